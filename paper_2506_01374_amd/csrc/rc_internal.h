// Internal declarations shared by the host-side translation units of librc.
#pragma once

#include <cstdint>
#include <string>
#include <vector>

#include "rc.h"

namespace rc {

struct KnobDef {
    const char *name;
    const char *xform;        // transformation class
    std::vector<int32_t> values;
    int32_t def;              // value in the untransformed program P0
};

// Knob table of an operator kind (empty for an unknown kind).
const std::vector<KnobDef> &knobs_for(int32_t kind);
// Index of a knob by name, -1 if absent.
int knob_index(int32_t kind, const char *name);

rc_status fail(rc_status s, const std::string &msg);
void clear_error();

bool desc_ok(const rc_op_desc *d);
// Knob value by name (asserts the name exists for the kind).
int32_t kv(const rc_op_desc *d, const rc_schedule *s, const char *name);

// Depth of the direct-to-LDS ring of bf16 GEMM stages 7.
int gemm_ring_stages(int tm, int tn, int tk, int nb, int waves, int occ);

// The same for the int8 product's ring (stages 2), the K of one of its splits,
// and the tiles that it runs at half height.
int gemm_i8_ring_stages(int tm, int tn, int tk, int waves, int occ);
int64_t gemm_i8_split_k(int64_t K, int tk, int splits);
int64_t gemm_i8_tail_tiles(int64_t tiles, int tm, int tn, int tk, int waves, int occ);

// Column split of a GEMM block over two launches (the "tail" knob).
bool gemm_tail_split(int tm, int tn, int tk, int nb, int waves, int occ, int st, int64_t M, int64_t N,
                     int64_t *main_cols, int64_t *tail_cols);

// Sizes of a kind of attention in serving (0 where it has none).
struct SeqDims {
    int64_t T, TK, B, H, Hkv, D, page, pages, width;
};
SeqDims seq_dims(const rc_op_desc *d);
int expected_dims(int32_t kind);
// Workgroups a CU for which keys are cut: `splits`, or twice that (outside the ring,
// where the pieces take more than a round).
int seqs_pieces(const rc_op_desc *d, const rc_schedule *s);
// Work items that an attention over sequences has at most, and blocks of rows
// that it cuts: of two pieces at least, which are fewer than two a workgroup that
// the keys are cut for (`splits`: seqs_pieces).
int64_t seqs_items(const rc_op_desc *d, int bm, int splits);
int64_t seqs_cut_blocks(const rc_op_desc *d, int bm, int splits);

// Legality with a reason; "" when legal.
std::string check_schedule(const rc_op_desc *d, const rc_schedule *s);

// Directory holding the kernel sources' embedded copy and the cache.
std::string cache_dir();

// rc_launch with the workspace given by the caller of this function (no
// allocation on any path that succeeds).
rc_status launch_plan(const rc_plan *p, const rc_args *a, void *workspace, size_t ws_bytes,
                      void *stream);

}  // namespace rc
