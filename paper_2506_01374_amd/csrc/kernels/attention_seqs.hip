// Attention over sequences of different lengths for gfx950: over a paged cache
// of keys and values (bf16, or int8 with an fp32 scale for each token and
// head), or over sequences packed behind each other; grouped heads, causal or
// not, any number of new rows a sequence.
//
// Compile-time schedule (generated prologue):
//   BM      rows of a work item (TileSize), see below
//   NW      waves of a workgroup (Parallel)
//   STAGES  keys and values go straight to registers, and 1: a tile is loaded,
//           then computed, 2: the next tile's loads are under way meanwhile; 3:
//           they go through a ring in shared memory (ComputeLocation)
//   OCC     waves per SIMD the register allocation must leave room for (with
//           the ring two)
//   SPLIT   1: the keys of a sequence are cut into pieces for several
//           workgroups, whose states rc_attention_seqs_join puts together
//   HD      head dimension: 64, 128 or 256
//   PAGED   1: K and V are [pages][HKV][page][HD], found through the table
//   I8      1: they hold int8 (PAGED)
//   LEAST   key tiles that a piece has at least (SPLIT)
//   SCALE_LOG2  log2(e) / sqrt(HD): scores are kept in log2 units
//
// The G query heads that share a K/V head are rows of one product: row r of
// sequence b and K/V head h is query head h G + r % G of the token r / G.  Row
// r sees the keys 0 .. vis, with vis the token's position (causal) or the last
// key's.  A row that sees none is 0.
//
// Scores, maxima and all sums are fp32.  Probabilities are rounded to bf16 for the
// second product, with int8 after V's scale is multiplied in: half a step, 2^-8, of
// each, which is what the output's own rounding may cost, where two terms of each
// would double the second product's matrix instructions.
//
// What is in the offsets, lengths and the table is on the device, and so is the
// division of work: every wave reads the lengths of all sequences and finds its
// workgroup's item (see find), so that a launch, a captured one too, serves
// whatever lengths it then meets.  Whatever they hold, no access leaves its
// buffer: offsets and lengths are clamped, and a page that is not in the cache
// is not seen.

typedef unsigned short bf16_t;
typedef unsigned int u32;
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef u32 u32x2 __attribute__((ext_vector_type(2)));
typedef u32 u32x4 __attribute__((ext_vector_type(4)));

#if STAGES == 3
#define QB (BM / 64)               // blocks of 16 rows of a wave
#define BN (HD == 256 ? 32 : 64)   // keys of a tile
#else
#define QB (BM / 16)
#define BN 32
#endif
#define NKS (HD / 32)              // MFMA steps of the score product
#define DE (HD / 16)               // elements of V that a lane takes of a key
#define ELT (I8 ? 1 : 2)           // bytes of an element of K and V
// The running maximum moves only when a score exceeds it by more than this
// (in log2 units): a stale one keeps every probability below 2^8
#define STALE 8.0f

struct SeqsArgs {
    const bf16_t *Q;               // [T][H][HD]
    const char *K, *V;
    const float *Ks, *Vs;          // [pages][HKV][page] (I8)
    const int *offsets;            // [B + 1]
    const int *lens;               // [B] (PAGED), or the offsets of K's rows [B + 1]
    const int *table;              // [B][width]
    bf16_t *O;
    float *P;                      // states of pieces (SPLIT)
    int T, TK, B, G, HKV, shift, pages, width, causal, slots;
    int by;                        // the join: see there
};

__device__ __forceinline__ int limit(int x, int lo, int hi) { return x < lo ? lo : x > hi ? hi : x; }
// byte e of w as a float
__device__ __forceinline__ float byte(u32 w, int e) { return (float)(signed char)(w >> (8 * e)); }
__device__ __forceinline__ float pow2(float x) { return __builtin_amdgcn_exp2f(x); }

// ---------------------------------------------------------------------------
// Division of work
// ---------------------------------------------------------------------------

struct Seq {
    int q0, n;          // rows q0 .. q0 + n - 1 of Q
    int k0;             // first row of K (packed)
    int len, keys;      // tokens; keys that there are (at most len)
    __device__ __forceinline__ int vis(int token, int causal) const {
        const int p = len - n + token;
        return causal && p < keys - 1 ? p : keys - 1;
    }
};

__device__ __forceinline__ Seq sequence(const SeqsArgs &a, int b) {
    Seq s;
    s.q0 = limit(a.offsets[b], 0, a.T);
    s.n = limit(a.offsets[b + 1], s.q0, a.T) - s.q0;
#if PAGED
    s.k0 = 0;
    s.len = limit(a.lens[b], 0, 1 << 30);
    s.keys = limit(s.len, 0, a.width << a.shift);
#else
    s.k0 = limit(a.lens[b], 0, a.TK);
    s.keys = s.len = limit(a.lens[b + 1], s.k0, a.TK) - s.k0;
#endif
    return s;
}

__device__ __forceinline__ int blocks_of(const SeqsArgs &a, const Seq &s) { return (int)(((long long)s.n * a.G + BM - 1) / BM); }
__device__ __forceinline__ int tiles_of(const Seq &s) { return (s.keys + BN - 1) / BN; }

struct Item {
    Seq s;
    int h, block, piece, pieces, slot;
};

// x + that of all lanes before, by moves between lanes without shared memory
__device__ __forceinline__ int scan(int x) {
#define FROM(how, rows) x += __builtin_amdgcn_update_dpp(0, x, how, rows, 0xF, false)
    FROM(0x111, 0xF);              // within rows of 16: 1, 2, 4, 8 lanes to the right
    FROM(0x112, 0xF);
    FROM(0x114, 0xF);
    FROM(0x118, 0xF);
    FROM(0x142, 0xA);              // the last lane of rows 0 and 2 to the next row
    FROM(0x143, 0xC);              // lane 31 to the two rows behind it
#undef FROM
    return x;
}
__device__ __forceinline__ int from_lane(int x, int lane) { return __builtin_amdgcn_readlane(x, lane); }

// A sequence's rows are cut into blocks of BM, and with SPLIT its keys into
// pieces of at most `most` tiles, the same number for each block.  `most` is
// the work of all sequences over the workgroups that it is cut for (a.slots), or
// half of that, so that pieces of blocks that are cut are at most 2 a.slots, or 4:
// each takes more than half of it.  The pieces' states are in this order too: sequence by sequence,
// its last block (the one that sees most keys) first, piece by piece, head by
// head.  Item `index` of that order (ITEMS), the first piece's of what row
// `index` of Q is in (ROWS), or of the `index`-th block that is cut (BLOCKS).
// Where there are more than SCANNED sequences, which are not cut then, they are not
// gone through: sequence b has the indexes of blocks from first_index(b) on, which
// are at least as many as its blocks, and is found by 64 of them at a time (8192
// sequences of 64 tokens, 8 heads: 802 us, 3860 where all lengths are read).
#define SCANNED 256
__device__ __forceinline__ int first_index(const SeqsArgs &a, int b) { return (int)((u32)limit(a.offsets[b], 0, a.T) * a.G / BM) + b; }
enum Find { ITEMS, ROWS, BLOCKS };
template <Find WHAT> __device__ __forceinline__ bool find(const SeqsArgs &a, int index, Item &item) {
    const int lane = threadIdx.x & 63;
    item.h = WHAT == ROWS ? 0 : index % a.HKV;
    int j = WHAT == ROWS ? index : index / a.HKV;
    int most = 1 << 30;
    Seq first = {};                // of the first 64 sequences
    if (lane < a.B) first = sequence(a, lane);
#if SPLIT
    unsigned long long work = 0;
    for (int c = 0; c < a.B; c += 64) {
        const Seq s = c == 0 || c + lane >= a.B ? first : sequence(a, c + lane);
        // (all of it is below 2^51, 24 bits at a time)
        const unsigned long long w = c + lane < a.B ? (unsigned long long)blocks_of(a, s) * tiles_of(s) : 0;
        work += (u32)from_lane(scan((int)(w & 0xFFFFFF)), 63) + ((unsigned long long)(u32)from_lane(scan((int)(w >> 24)), 63) << 24);
    }
    work = (work * a.HKV + a.slots - 1) / a.slots;
    most = work < LEAST ? LEAST : work > (1 << 30) ? 1 << 30 : (int)work;
    // A last piece more of many blocks can be a second round of workgroups: in the
    // ring, 25 blocks of 8 heads in 3 pieces for 2, with 15 single rows, 157 us for
    // 148.  There a piece counts as a workgroup, and a block that is not cut as the part
    // of one that its tiles are of `most`, with START tiles more for the start and the
    // end of each: with all blocks as workgroups, many short sequences leave a long one
    // whole (62 of 256 tokens and 5 rows, one of 32768: 268 us for 55; 32 of 300 to 8192
    // and 16 rows 74 for 65).  Cut blocks, each of more than `most` tiles, exceed what
    // their tiles take of a round by one piece each, so that the next `most` is at most
    // twice what all tiles and starts are over the workgroups.
    // (Outside the ring, where pieces are long, a second round comes in smaller ones:
    // 128 rows over int8 caches of 128 to 4096 tokens 92 us for 79, 64 over bf16 ones
    // of 64 to 8192 88 for 85; where all are as long and fit one round, 64 of 1600
    // int8 tokens, smaller ones take 56 for 47.  Of short pieces the count would take
    // what it gains, and over int8 caches of 64 to 8192 tokens 64 rows 58 for 56.)
    const int tries = STAGES == 3 ? 4 : most >= (I8 ? 64 : 32) ? 1 : 0;
    constexpr int PART = STAGES == 3 ? 32 : 1, START = 5;     // (a workgroup, in the units that are counted)
#pragma nounroll
    for (int t = 0; t < tries; ++t) {
        const float part = PART * __builtin_amdgcn_rcpf((float)(most + START));
        long long load = 0;
        bool cut = false;
        for (int c = 0; c < a.B; c += 64) {
            const Seq s = c == 0 || c + lane >= a.B ? first : sequence(a, c + lane);
            const int tiles = tiles_of(s), pieces = c + lane < a.B ? max(1, (tiles + most - 1) / most) : 1;
            const int each = STAGES != 3 || pieces > 1 ? PART * pieces : (int)((float)(tiles + START) * part);
            load += from_lane(scan(c + lane < a.B ? (int)min((long long)blocks_of(a, s) * each, 1ll << 24) : 0), 63);
            cut |= __builtin_amdgcn_ballot_w64(pieces > 1) != 0;
        }
        load *= a.HKV;
        if (!cut || load * 16 <= PART * a.slots * 17ll) break;
        most = STAGES == 3 ? (int)min((long long)(1 << 30), most * load / (PART * a.slots) + 1) : max(LEAST, (most + 1) / 2);
    }
#endif
    int slot = 0, c = 0, end = a.B;
#if !SPLIT
    if (a.B > SCANNED) {
        // only the last sequence whose first index is not past j
        for (int n = a.B, step; n > 1; n = end - c) {
            step = (n + 63) / 64;
            const unsigned long long before = __builtin_amdgcn_ballot_w64(lane * step < n && first_index(a, min(c + lane * step, a.B)) <= j);
            if (!before) return false;
            c += (63 - __builtin_clzll(before)) * step;
            end = min(end, c + step);
        }
        c = __builtin_amdgcn_readfirstlane(c);
        j = __builtin_amdgcn_readfirstlane(j - first_index(a, c));
    }
#endif
    for (; c < end; c += 64) {
        const Seq s = c == 0 || c + lane >= end ? first : sequence(a, c + lane);
        const int blocks = c + lane < end ? blocks_of(a, s) : 0, pieces = SPLIT ? max(1, (tiles_of(s) + most - 1) / most) : 1;
        const int cut = pieces > 1 ? blocks * pieces : 0;      // states that the sequence leaves
        const int items = WHAT == ITEMS ? blocks * pieces : pieces > 1 ? blocks : 0;
        const int sum = WHAT == ROWS ? 0 : scan(items), sums = SPLIT ? scan(cut) : 0;
        const unsigned long long past = __builtin_amdgcn_ballot_w64(WHAT == ROWS ? blocks > 0 && s.q0 <= j && j < s.q0 + s.n : sum > j);
        if (past) {
            const int at = __builtin_ctzll(past);
            item.s.q0 = from_lane(s.q0, at), item.s.n = from_lane(s.n, at), item.s.len = from_lane(s.len, at);
            item.s.keys = from_lane(s.keys, at);
            // (PAGED: which sequence, to find its row of the table)
            item.s.k0 = PAGED ? c + at : from_lane(s.k0, at);
            item.pieces = from_lane(pieces, at);
            slot += from_lane(sums - cut, at);
            if (WHAT == ROWS) {
                item.slot = slot;
                item.block = from_lane(blocks, at);            // how many there are
                return true;
            }
            const int i = j - from_lane(sum - items, at), order = WHAT == ITEMS ? i / item.pieces : i;
            item.block = from_lane(blocks, at) - 1 - order;
            item.piece = WHAT == ITEMS ? i % item.pieces : 0;
            item.slot = (slot + order * item.pieces + item.piece) * a.HKV + item.h;
            return true;
        }
        if (WHAT != ROWS) j -= from_lane(sum, 63);
        slot += from_lane(sums, 63);
    }
    return false;
}

// -inf (no key seen yet) as a finite number: what is -inf relative to it stays so
__device__ __forceinline__ float least_finite(float m) { return fmaxf(m, -0x1.fffffep127f); }

// State of a piece: m and l of its rows, then their sums of p V
#define STATE (BM * (HD + 2))

__device__ __forceinline__ u32 pack2(float a, float b) {
    return __builtin_bit_cast(u32, __builtin_convertvector((f32x2){a, b}, bf16x2));
}
// four outputs of a row, sums of p V over the sum of p: 0 where nothing was seen, or at
// -inf alone, whose values (0 times each) may be anything
__device__ __forceinline__ u32x2 outputs(const f32x4 &o, float sum) {
    const float inv = 1.f / sum;
    const u32x2 x = {pack2(o[0] * inv, o[1] * inv), pack2(o[2] * inv, o[3] * inv)};
    return sum == 0.f ? u32x2{} : x;
}
__device__ __forceinline__ f32x4 mfma(const bf16x8 &a, const bf16x8 &b, const f32x4 &c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
}

// ---------------------------------------------------------------------------
// Keys and values straight to registers
// ---------------------------------------------------------------------------
//
// A wave takes whole tiles of 32 keys, every NW-th of its workgroup's piece,
// and all BM rows.  S^T = K Q^T: a lane's part of K is what the matrix
// instruction takes from it, 16 consecutive bytes of key lane % 16, so that K
// needs no shared memory.  O^T = V^T P^T needs 8 keys of one channel from a
// lane: it loads the channels DE (lane % 16) .. + DE - 1 of 8 keys, pairs them
// up with a byte permute, and the e-th of DE instructions takes the channels
// DE i + e as its 16 rows.  The keys of a lane are those of its scores (4 (lane
// / 16) + r of each 16), so that P^T stays where it is.
//
// Bound by the cache's bytes where there are many, by the way to memory (lengths,
// table, tile) else: 64 rows over bf16 caches of 64 to 8192 tokens, 8 K/V heads of
// 128, 87 us (4.7 TB/s), over int8 ones 48 (4.4; a byte takes 1.5 vector
// instructions of a lane to widen); one row over 32768 tokens 25 (5.4).

// Values that are not finite, in a tile that some row does not see whole: 0 times
// one is a NaN.  O += V^T P^T takes them as 0, and +-1 in their place (a NaN both)
// times the keys that a row sees (1, or 0) says which of its sums are infinite.
__device__ __forceinline__ bool far(u32 half) { return (half & 0x7F80u) == 0x7F80u; }
__device__ __forceinline__ bf16x8 ones(const u32x4 &v, u32 but) {
    u32x4 f;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const u32 lo = v[j] & 0xFFFFu, hi = v[j] >> 16;
        f[j] = (far(lo) && lo != but ? 0x3F80u : 0u) | (far(hi) && hi != but ? 0x3F800000u : 0u);
    }
    return __builtin_bit_cast(bf16x8, f);
}
__device__ __forceinline__ bf16x8 seen(const f32x4 &s0, const f32x4 &s1) {
    const float none = -__builtin_inff();
    u32x4 f;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const f32x4 &s = j < 2 ? s0 : s1;
        f[j] = (s[2 * (j % 2)] == none ? 0u : 0x3F80u) | (s[2 * (j % 2) + 1] == none ? 0u : 0x3F800000u);
    }
    return __builtin_bit_cast(bf16x8, f);
}
__device__ __forceinline__ f32x4 add_far(const u32x4 &v, const bf16x8 &p, const bf16x8 &see, const f32x4 &o) {
    u32x4 f;
#pragma unroll
    for (int j = 0; j < 4; ++j) f[j] = v[j] & ~((far(v[j]) ? 0xFFFFu : 0u) | (far(v[j] >> 16) ? 0xFFFF0000u : 0u));
    f32x4 x = mfma(__builtin_bit_cast(bf16x8, f), p, o);
    const f32x4 up = mfma(ones(v, 0xFF80u), see, f32x4{}), down = mfma(ones(v, 0x7F80u), see, f32x4{});
#pragma unroll
    for (int r = 0; r < 4; ++r) x[r] += (up[r] > 0.f ? __builtin_inff() : 0.f) - (down[r] > 0.f ? __builtin_inff() : 0.f);
    return x;
}

#if STAGES < 3

struct Tile {
    u32x4 k[2][I8 ? NKS / 2 : NKS];
    u32 v[8][DE * ELT / 4];
#if I8
    f32x4 ks[2], vs[2];
#endif
    int held;          // of the two 16-key blocks
};

// (At most three waves a SIMD where there are two at least: with four, pieces that are
// cut for two crowd some of the CUs, 64 rows over int8 caches of 64 to 8192 tokens 58.6
// us for 56.0, 100 rows of D = 64 over bf16 ones 100.3 for 98.6.)
extern "C" __global__ __launch_bounds__(64 * NW) __attribute__((amdgpu_waves_per_eu(OCC, OCC == 2 ? 3 : 8))) void rc_attention_seqs(SeqsArgs a) {
    __shared__ __attribute__((aligned(16))) float osum[NW][BM][HD + 4];
    __shared__ float om[NW][BM], ol[NW][BM];
    const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int i = lane % 16, g = lane / 16;
    Item item;
    if (!find<ITEMS>(a, blockIdx.x, item)) return;
    const Seq s = item.s;
    const int rows = s.n * a.G, r0 = item.block * BM;

    // queries, and the last key that each sees (the first row the fewest)
    bf16x8 q[QB][NKS];
    int vis[QB];
    const int least = __builtin_amdgcn_readfirstlane(s.vis(r0 / a.G, a.causal));
#pragma unroll
    for (int b = 0; b < QB; ++b) {
        const int r = r0 + 16 * b + i, token = r / a.G;
        vis[b] = 1 << 30;          // (rows that there are not)
#pragma unroll
        for (int ks = 0; ks < NKS; ++ks) q[b][ks] = bf16x8{};
        if (r < rows) {
            vis[b] = s.vis(token, a.causal);
            const bf16_t *p = a.Q + ((size_t)(s.q0 + token) * a.HKV * a.G + item.h * a.G + r % a.G) * HD;
#pragma unroll
            for (int ks = 0; ks < NKS; ++ks)
                q[b][ks] = *(const bf16x8 *)(p + (I8 ? 64 * (ks / 2) + 16 * g + 8 * (ks % 2) : 32 * ks + 8 * g));
        }
    }

    // tiles of the block's last row, of the piece, of the wave
    const int last = s.vis((min(rows, r0 + BM) - 1) / a.G, a.causal);
    const int tiles = (max(last + 1, 0) + BN - 1) / BN, share = (tiles + item.pieces - 1) / item.pieces;
    const int t0 = item.piece * share + w, t1 = min(tiles, (item.piece + 1) * share);
    const int nt = __builtin_amdgcn_readfirstlane(t1 > t0 ? (t1 - t0 + NW - 1) / NW : 0);

    f32x4 o[QB][DE];
    float m[QB], l[QB];
#pragma unroll
    for (int b = 0; b < QB; ++b) {
        m[b] = -__builtin_inff();
        l[b] = 0.f;
#pragma unroll
        for (int e = 0; e < DE; ++e) o[b][e] = f32x4{0.f, 0.f, 0.f, 0.f};
    }

    int ids = 0;                           // pages of the 64 next blocks of 16 keys
#if PAGED
    constexpr u32 step = HD * ELT;
#else
    const u32 step = (u32)a.HKV * (HD * ELT);
#endif
    auto load = [&](int it, Tile &x) __attribute__((always_inline)) {
        x.held = 3;
#if PAGED
        if (it % 32 == 0) {
            const int key = (t0 + (it + lane / 2) * NW) * BN + 16 * (lane & 1);
            ids = it + lane / 2 < nt && key < s.keys ? a.table[(size_t)s.k0 * a.width + (key >> a.shift)] : -1;
        }
#endif
#pragma unroll
        for (int c = 0; c < 2; ++c) {
            const int key = (t0 + it * NW) * BN + 16 * c;
#if PAGED
            int id = __builtin_amdgcn_readlane(ids, (2 * it + c) % 64);
            if ((u32)id >= (u32)a.pages) id = 0, x.held &= ~(1 << c);
            const size_t row = (((size_t)id * a.HKV + item.h) << a.shift) + (key & ((1 << a.shift) - 1));
            constexpr int end = 15;
#else
            // rows past the sequence's last: that one, which is there
            const int from = min(key, s.keys - 1), end = s.keys - 1 - from;
            const size_t row = (size_t)(s.k0 + from) * a.HKV + item.h;
#endif
            const char *kp = a.K + row * (HD * ELT), *vp = a.V + row * (HD * ELT);
#pragma unroll
            for (int ks = 0; ks < (I8 ? NKS / 2 : NKS); ++ks)
                x.k[c][ks] = *(const u32x4 *)(kp + ((u32)min(i, end) * step + 16 * g) + 64 * ks);
#pragma unroll
            for (int j = 0; j < 4; ++j)
                __builtin_memcpy(x.v[4 * c + j], vp + ((u32)min(4 * g + j, end) * step + i * (DE * ELT)), DE * ELT);
#if I8
            x.ks[c] = *(const f32x4 *)((const char *)(a.Ks + row) + 16u * g);
            x.vs[c] = *(const f32x4 *)((const char *)(a.Vs + row) + 16u * g);
#endif
        }
        __builtin_amdgcn_sched_barrier(0);
    };

    // the largest over the lanes of a row
    auto over_lanes = [&](float v) {
        v = fmaxf(v, __shfl_xor(v, 16));
        return fmaxf(v, __shfl_xor(v, 32));
    };

    auto compute = [&](int it, Tile &x) __attribute__((always_inline)) {
        const int key0 = (t0 + it * NW) * BN;
        f32x4 sc[QB][2];
#pragma unroll
        for (int b = 0; b < QB; ++b)
#pragma unroll
            for (int c = 0; c < 2; ++c) sc[b][c] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int c = 0; c < 2; ++c)
#pragma unroll
            for (int ks = 0; ks < NKS; ++ks) {
#if I8
                u32x4 f;
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    const u32 t = x.k[c][ks / 2][2 * (ks % 2) + e];
                    f[2 * e] = pack2(byte(t, 0), byte(t, 1));
                    f[2 * e + 1] = pack2(byte(t, 2), byte(t, 3));
                }
                const bf16x8 k = __builtin_bit_cast(bf16x8, f);
#else
                const bf16x8 k = __builtin_bit_cast(bf16x8, x.k[c][ks]);
#endif
#pragma unroll
                for (int b = 0; b < QB; ++b) sc[b][c] = mfma(k, q[b][ks], sc[b][c]);
            }
        // a tile that some row does not see whole
        const bool masked = key0 + BN - 1 > least || x.held != 3;
        bool apart = false;                // values that are not finite, which some row does not see
#if I8
#pragma unroll
        for (int b = 0; b < QB; ++b)
#pragma unroll
            for (int c = 0; c < 2; ++c) sc[b][c] *= x.ks[c];
#endif
        if (masked) {
#pragma unroll
            for (int c = 0; c < 2; ++c)
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    const int key = key0 + 16 * c + 4 * g + r;
                    const bool there = x.held >> c & 1 && key < s.keys;
#pragma unroll
                    for (int b = 0; b < QB; ++b)
                        if (!there || key > vis[b]) sc[b][c][r] = -__builtin_inff();
                    // what is not a key of the sequence may hold anything
#if I8
                    if (!there) x.vs[c][r] = 0.f;
#else
                    bool some = false;
#pragma unroll
                    for (int e = 0; e < DE * ELT / 4; ++e) {
                        u32 &v = x.v[4 * c + r][e];
                        v = there ? v : 0;
                        some |= far(v) | far(v >> 16);
                    }
                    apart |= some;
#endif
                }
        }
        bf16x8 p[QB];
#pragma unroll
        for (int b = 0; b < QB; ++b) {
            float top = -__builtin_inff();
#pragma unroll
            for (int c = 0; c < 2; ++c)
#pragma unroll
                for (int r = 0; r < 4; ++r) top = fmaxf(top, sc[b][c][r]);
            if (__builtin_amdgcn_ballot_w64(top * SCALE_LOG2 > m[b] + STALE) != 0) {
                const float now = fmaxf(m[b], over_lanes(top) * SCALE_LOG2);
                // (all -inf so far: nothing to rescale)
                const float by = m[b] == now ? 1.f : pow2(m[b] - now);
                l[b] *= by;
#pragma unroll
                for (int e = 0; e < DE; ++e) o[b][e] *= by;
                m[b] = now;
            }
            const float minus = -least_finite(m[b]);
            float pr[2][4];
#pragma unroll
            for (int c = 0; c < 2; ++c)
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    pr[c][r] = pow2(__builtin_fmaf(sc[b][c][r], SCALE_LOG2, minus));
                    l[b] += pr[c][r];
#if I8
                    // V's scale goes into p; a key that the row does not see has none
                    pr[c][r] = masked && key0 + 16 * c + 4 * g + r > vis[b] ? 0.f : pr[c][r] * x.vs[c][r];
#endif
                }
            u32x4 f;
#pragma unroll
            for (int c = 0; c < 2; ++c) {
                f[2 * c] = pack2(pr[c][0], pr[c][1]);
                f[2 * c + 1] = pack2(pr[c][2], pr[c][3]);
            }
            p[b] = __builtin_bit_cast(bf16x8, f);
        }
        auto values = [&](int e) __attribute__((always_inline)) {
            u32x4 f;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
#if I8
                f[j] = pack2(byte(x.v[2 * j][e / 4], e % 4), byte(x.v[2 * j + 1][e / 4], e % 4));
#else
                f[j] = __builtin_amdgcn_perm(x.v[2 * j + 1][e / 2], x.v[2 * j][e / 2], e % 2 ? 0x07060302u : 0x05040100u);
#endif
            }
            return f;
        };
        if (!I8 && __builtin_amdgcn_ballot_w64(apart) != 0) {
#pragma unroll
            for (int e = 0; e < DE; ++e) {
                const u32x4 v = values(e);
#pragma unroll
                for (int b = 0; b < QB; ++b) o[b][e] = add_far(v, p[b], seen(sc[b][0], sc[b][1]), o[b][e]);
                __builtin_amdgcn_sched_barrier(0);
            }
            return;
        }
#pragma unroll
        for (int e = 0; e < DE; ++e) {
            const bf16x8 v = __builtin_bit_cast(bf16x8, values(e));
#pragma unroll
            for (int b = 0; b < QB; ++b) o[b][e] = mfma(v, p[b], o[b][e]);
        }
    };

#if STAGES == 1
#pragma nounroll
    for (int it = 0; it < nt; ++it) {
        Tile x;
        load(it, x);
        compute(it, x);
    }
#else
    // (the loads are issued without a branch: past the last tile, that one again)
    if (nt > 0) {
        Tile x, y;
        load(0, x);
        for (int it = 0; it < nt; it += 2) {
            load(min(it + 1, nt - 1), y);
            compute(it, x);
            if (it + 1 < nt) {
                load(min(it + 2, nt - 1), x);
                compute(it + 1, y);
            }
        }
    }
#endif

    // the waves' states, added with the weights of their maxima
#pragma unroll
    for (int b = 0; b < QB; ++b) {
        l[b] += __shfl_xor(l[b], 16);
        l[b] += __shfl_xor(l[b], 32);
        if (g == 0) om[w][16 * b + i] = m[b], ol[w][16 * b + i] = l[b];
#pragma unroll
        for (int r = 0; r < 4; ++r)
#pragma unroll
            for (int e = 0; e < DE; e += 4)
                *(f32x4 *)&osum[w][16 * b + i][DE * (4 * g + r) + e] = f32x4{o[b][e][r], o[b][e + 1][r], o[b][e + 2][r], o[b][e + 3][r]};
    }
    __syncthreads();
    float *state = a.P + (SPLIT ? (size_t)item.slot * STATE : 0);
    for (int c = threadIdx.x; c < BM * HD / 4; c += 64 * NW) {
        const int r = c / (HD / 4), d = c % (HD / 4) * 4;
        if (r0 + r >= rows) continue;
        float top = om[0][r];
#pragma unroll
        for (int v = 1; v < NW; ++v) top = fmaxf(top, om[v][r]);
        float sum = 0.f;
        f32x4 out = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int v = 0; v < NW; ++v) {
            const float by = om[v][r] == top ? 1.f : pow2(om[v][r] - top);
            sum += ol[v][r] * by;
            out += *(const f32x4 *)&osum[v][r][d] * by;
        }
        if (SPLIT && item.pieces > 1) {
            if (d == 0) state[r] = top, state[BM + r] = sum;
            *(f32x4 *)(state + 2 * BM + r * HD + d) = out;
        } else {
            const int row = r0 + r;
            bf16_t *p = a.O + ((size_t)(s.q0 + row / a.G) * a.HKV * a.G + item.h * a.G + row % a.G) * HD + d;
            *(u32x2 *)p = outputs(out, sum);
        }
    }
}

#endif

// ---------------------------------------------------------------------------
// Keys and values through shared memory, in turns (STAGES 3)
// ---------------------------------------------------------------------------
//
// Four waves of 16 QB rows each, or eight: four for the even key tiles of the
// piece, and four for the odd ones, with their own softmax states, put together
// at the end.  Waves w and w + 4 share a SIMD and take turns on its matrix cores:
// while one multiplies (O^T += V^T P^T of its tile, then S^T = K Q^T of its next),
// the other does its softmax (vector work); a barrier ends each turn.  Four waves
// alternate the same turns, two workgroups a CU, which fall out of step by
// themselves and fill each other's starts and ends, 17000 cycles a block (8
// prompts of 8192 tokens in all, 32 heads of 128: 148 us, with eight waves 180);
// eight are for few blocks, each of them done sooner (8 sequences of 64 new rows and
// 1000 tokens: blocks of 64 rows 19 us, with four 23).
// K and V go straight from memory to shared memory, into a ring of two tiles for
// each operand and half of the waves; the softmax turn issues the loads between its
// exponentials, K of the tile after the next and V of the next, into the places
// that the matrix turn before it has read, and waits for those of the softmax turn
// before.  16-byte chunks of a row are XOR-ed with the row's number (KSWZ, VSWZ),
// by the choice of what a lane fetches, so that fragment reads have no bank
// conflicts; V's are transposed by the reading instruction.
// An int8 tile goes through registers: a softmax turn widens what the one before
// has loaded to bf16 (exactly) and writes it, K of the next tile and V of this
// one, so that one place for each is enough.  K's scale is multiplied into the
// scores, V's into the probabilities.
//
// Bound by the issue of vector and matrix instructions together, at a clock that
// the power limits: a prompt of 16384 tokens, 32 heads of 128, 1.78 to 1.88 ms
// (1.23 to 1.17 PFLOP/s), matrix cores busy 62 % of the time at 1.9 GHz.  Over an
// int8 cache by vector instructions, more than a quarter of which widen (512 rows
// over 8192 tokens 110 us, over bf16 75 to 81).  Slower were: loads issued by the
// matrix turn (1972 -> 2147 us), V read by 16 bytes and paired by permutes (7 %
// more), the matrix turn without priority; no gain: none of the loads past a half's
// last tile, V and the second K tile loaded behind the first's wait, priority for a
// block's start and end, V's rows swizzled by their parity too.

#if STAGES == 3
#define ROWG 4                     // groups of rows
#define HALVES (NW / ROWG)         // 2: of the waves, 1: all of them take every tile
#define BNW (BN / ROWG)            // keys that a wave loads of a tile
#define KB (BN / 16)
#define DB (HD / 16)
#define CPR (HD / 8)               // 16-byte chunks of a row
#define RPL ((16 / CPR) > 0 ? (16 / CPR) : 1)
#define KSWZ(r) (((r) / RPL) % (CPR < 16 ? CPR : 16))
#define VSWZ(r) ((2 * (r)) & (CPR - 1))
#define TILE (BN * HD)
#define NPJ (BN / 32)              // MFMA steps of P V
#define NKF (KB * NKS)             // fragments of K and of V
#define NVF (NPJ * DB)
#define AHEAD 8                    // of them read ahead of their MFMAs
#define WL (TILE / 512 / ROWG)     // 1 KiB loads of a wave for a tile
#define RPI (512 / HD)             // rows of one
#define NL (TILE / 1024 / ROWG)    // 16-byte loads of a lane for a tile of int8

template <int V> struct IntC { static constexpr int value = V; };
// seq<A, B>(f): f(IntC<A>), ... f(IntC<B - 1>), every index a constant
template <class T, T... I> struct ISeq {};
template <int A, class F, int... I> __device__ __forceinline__ void seq_calls(F &f, ISeq<int, I...>) {
    (f(IntC<A + I>{}), ...);
}
template <int A, int B, class F> __device__ __forceinline__ void seq(F &&f) {
    if constexpr (B > A) seq_calls<A>(f, __make_integer_seq<ISeq, int, B - A>{});
}
// at most n loads of this wave are left in flight
#define WAIT_VM(n) __builtin_amdgcn_s_waitcnt(((n) & 15) | ((((n) >> 4) & 3) << 14) | (7 << 4) | (15 << 8))

// the lane's number, formed where it is used: held, it takes a register that the
// turns need
__device__ __forceinline__ int lane_here() {
    int x;
    asm volatile("v_mbcnt_lo_u32_b32 %0, -1, 0\n\tv_mbcnt_hi_u32_b32 %0, -1, %0" : "=v"(x));
    return x;
}

extern "C" __global__ __launch_bounds__(64 * NW) __attribute__((amdgpu_waves_per_eu(2, 2))) void rc_attention_seqs(SeqsArgs a) {
#if I8
    // K of each half's tile, then V; the last for the halves' states
    __shared__ __attribute__((aligned(16))) bf16_t ring[HALVES == 2 ? 5 : 2][TILE];
    __shared__ __attribute__((aligned(16))) float scales[HALVES][2][2][BN];   // of each half: two tiles' Ks (times SCALE_LOG2) and Vs
    __shared__ __attribute__((aligned(16))) float ones[BN];
    if (threadIdx.x < BN) ones[threadIdx.x] = 1.f;
#else
    __shared__ __attribute__((aligned(16))) bf16_t ring[4 * HALVES][TILE];    // K of each half's two tiles, then V
    __shared__ int again;
    if (threadIdx.x == 0) again = 0;
#endif
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int i = lane % 16, g = lane / 16, rg = wave % ROWG, sp = wave / ROWG;
    Item item;
    if (!find<ITEMS>(a, blockIdx.x, item)) return;
    const Seq s = item.s;
    const int rows = s.n * a.G, r0 = item.block * BM, r0w = r0 + 16 * QB * rg;

    // tiles of the block's last row, of the piece
    const int last_vis = s.vis((min(rows, r0 + BM) - 1) / a.G, a.causal);
    const int all = (max(last_vis + 1, 0) + BN - 1) / BN, share = (all + item.pieces - 1) / item.pieces;
    int kt0 = item.piece * share;
#if I8 && !SPLIT
    asm volatile("" : "+s"(kt0));          // (where it is known to be 0, more is held than there are registers for)
#endif
    const int n_kt = max(0, min(all, kt0 + share) - kt0);
    const int n_it = (n_kt + HALVES - 1) / HALVES, n_loc = (n_kt + HALVES - 1 - sp) / HALVES;        // turns; tiles of this half

    // loads: lane's byte offsets within the wave's rows of a tile
#if I8
    // (16 int8, two chunks in shared memory)
    const int row = lane / (HD / 16), chunk = lane % (HD / 16), rw = rg * BNW + row;
    // (elements of the first of them; 1024 / HD rows on the XOR-ed part changes
    // by a constant)
    const int k_to = sp * TILE + rw * HD + 8 * ((2 * chunk) ^ KSWZ(rw)), v_to = (HALVES + sp) * TILE + rw * HD + 8 * ((2 * chunk) ^ VSWZ(rw));
#else
#if PAGED
    constexpr u32 step = HD * 2;
#else
    const u32 step = (u32)a.HKV * (HD * 2);
#endif
    u32 k_src[WL], v_src[WL];
#pragma unroll
    for (int j = 0; j < WL; ++j) {
        const int r = j * RPI + lane / CPR, row = rg * BNW + r, c = lane % CPR;
        k_src[j] = r * step + 16 * (c ^ KSWZ(row));
        v_src[j] = r * step + 16 * (c ^ VSWZ(row));
    }
    typedef __attribute__((address_space(3))) bf16_t *lds_p;
    const u32 lds0 = (u32)(size_t)(lds_p)ring[0] + rg * (WL * 1024u);
    // K or V (v) of this half's slot b
    auto slot = [&](int v, int b) { return lds0 + (u32)(2 * HALVES * v + 2 * sp + b) * (TILE * 2u); };
    // (issued from inline assembly, which the compiler's own waits do not see:
    // it would drain them before every read of shared memory)
    auto dma = [&](const char *base, u32 off, u32 lds) {
        asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, %1" ::"v"(off), "s"(base), "s"(lds) : "memory", "m0");
    };
#endif
    // Where the wave's rows of the half's tile `it` start, and the last of them
    // that is a key (past the sequence's last key: that one, which is there).
    // Past the half's last tile: that one again, which nothing reads.
    struct From {
        size_t at;                         // bytes; of the scales elements
        int end;
    };
    const int last_key = s.keys - 1;
    int ids = 0;                           // pages of the wave's rows of 64 tiles
    auto first_key = [&](int it) { return min((kt0 + HALVES * it + sp) * BN + BNW * rg, last_key & ~(BNW - 1)); };
    auto rows_of = [&](int it) {
        it = min(it, max(n_loc - 1, 0));
        const int key = first_key(it);
        From f;
        f.end = last_key - key;
#if PAGED
        if (it % 64 == 0) {
            const int x = first_key(it + lane_here());
            ids = a.table[(size_t)s.k0 * a.width + (x >> a.shift)];
        }
        const int id = __builtin_amdgcn_readlane(ids, it % 64);
        f.at = (((size_t)((u32)id < (u32)a.pages ? id : 0) * a.HKV + item.h) << a.shift) + (key & ((1 << a.shift) - 1));
#else
        f.at = (size_t)(s.k0 + key) * a.HKV + item.h;
#endif
        if (!I8) f.at *= HD * 2;
        return f;
    };
#if I8
    // A tile on its way through registers: loaded in one softmax turn, widened
    // to bf16 and written to shared memory in the next
    u32x4 kx[NL], vx[NL];
    float sx = 0.f, sy = 0.f;
    auto fetch = [&](const char *src, const From &f, u32x4 (&x)[NL]) __attribute__((always_inline)) {
#pragma unroll
        for (int j = 0; j < NL; ++j) x[j] = *(const u32x4 *)(src + f.at * HD + (u32)(min(row + j * (1024 / HD), f.end) * HD + 16 * chunk));
    };
    auto fetch_scales = [&](const From &f) __attribute__((always_inline)) {
        const u32 at = 4 * min(lane % BNW, f.end);
        sx = *(const float *)((const char *)(a.Ks + f.at) + at);
        sy = *(const float *)((const char *)(a.Vs + f.at) + at);
    };
    auto widen = [&](const u32x4 (&x)[NL], int to, int swz) __attribute__((always_inline)) {
#pragma unroll
        for (int j = 0; j < NL; ++j)
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                u32x4 y;
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    const u32 t = x[j][2 * h + e];
                    y[2 * e] = pack2(byte(t, 0), byte(t, 1));
                    y[2 * e + 1] = pack2(byte(t, 2), byte(t, 3));
                }
                *(u32x4 *)(ring[0] + ((to + 1024 * j) ^ (8 * swz * j) ^ 8 * h)) = y;
                __builtin_amdgcn_sched_barrier(0);
            }
    };
    auto put_scales = [&](int b) __attribute__((always_inline)) {
        if (lane < 2 * BNW) scales[sp][b][lane / BNW][rg * BNW + lane % BNW] = lane < BNW ? sx * SCALE_LOG2 : sy;
    };
    From next = {0, BNW};
    if (n_kt > 0) {
        From f = rows_of(0);
        fetch(a.K, f, kx);
        fetch(a.V, f, vx);
        fetch_scales(f);
        next = rows_of(1);
        widen(kx, k_to, KSWZ(1024 / HD));
        put_scales(0);
        fetch(a.K, next, kx);
        fetch_scales(next);
    }
#else
    // loads j0 .. j1 - 1 of a tile; `edge`: rows past the last key fetch that one
    auto load = [&](const char *src, const u32 (&off)[WL], const From &f, u32 lds, int j0, int j1, auto edge) __attribute__((always_inline)) {
#pragma unroll
        for (int j = j0; j < j1; ++j) {
            u32 o = off[j];
            if constexpr (decltype(edge)::value) o -= (u32)max(j * RPI + lane / CPR - f.end, 0) * step;
            dma(src + f.at, o, lds + j * 1024u);
        }
    };
    auto load_whole = [&](const char *src, const u32 (&off)[WL], const From &f, u32 lds) __attribute__((always_inline)) {
        if (f.end < BNW - 1) load(src, off, f, lds, 0, WL, IntC<1>{});
        else load(src, off, f, lds, 0, WL, IntC<0>{});
    };

    // (nothing to see: the states below stay empty)
    From next = {0, BNW};
    if (n_kt > 0) {
        const From f = rows_of(0);
        next = rows_of(1);
        load_whole(a.K, k_src, f, slot(0, 0));
        load_whole(a.V, v_src, f, slot(1, 0));
        load_whole(a.K, k_src, next, slot(0, 1));
    }
#endif
    // is a page of the piece not held?
    bool gaps = false;
#if PAGED
    for (int p = (kt0 * BN >> a.shift) + lane; n_kt > 0 && p <= min(last_key, (kt0 + n_kt) * BN - 1) >> a.shift; p += 64)
        gaps |= (u32)a.table[(size_t)s.k0 * a.width + p] >= (u32)a.pages;
    gaps = __builtin_amdgcn_ballot_w64(gaps) != 0;
#endif
    auto held = [&](int key) {
        if (!PAGED || !gaps) return true;
        return (u32)a.table[(size_t)s.k0 * a.width + (min(key, last_key) >> a.shift)] < (u32)a.pages;
    };

    bf16x8 qf[QB][NKS];
    int vis[QB], least = 1 << 30, most = -1;           // (of the wave's first and last row)
    if (r0w < rows) {
        least = __builtin_amdgcn_readfirstlane(s.vis(r0w / a.G, a.causal));
        most = __builtin_amdgcn_readfirstlane(s.vis((min(rows, r0w + 16 * QB) - 1) / a.G, a.causal));
    }
#pragma unroll
    for (int b = 0; b < QB; ++b) {
        const int r = r0w + 16 * b + i, token = r / a.G;
        vis[b] = 1 << 30;          // (rows that there are not)
#pragma unroll
        for (int ks = 0; ks < NKS; ++ks) qf[b][ks] = bf16x8{};
        if (r < rows) {
            vis[b] = s.vis(token, a.causal);
            const bf16_t *p = a.Q + ((size_t)(s.q0 + token) * a.HKV * a.G + item.h * a.G + r % a.G) * HD;
#pragma unroll
            for (int ks = 0; ks < NKS; ++ks) qf[b][ks] = *(const bf16x8 *)(p + 32 * ks + 8 * g);
        }
    }
    // (their loads end before the loop, whose waits count the ring's alone)
#pragma unroll
    for (int b = 0; b < QB; ++b)
#pragma unroll
        for (int ks = 0; ks < NKS; ++ks) asm volatile("" ::"v"(qf[b][ks]));
    WAIT_VM(0);
    __syncthreads();

    f32x4 o[QB][DB];
    float m[QB];
#if I8
    float l[QB];                   // of a lane's own keys
#define SUM(b) l[b]
#else
    f32x4 l[QB];                   // of all keys, in each element
#define SUM(b) l[b][0]
#endif
    auto clear = [&] {
#pragma unroll
        for (int b = 0; b < QB; ++b) {
            m[b] = -__builtin_inff();
            l[b] = {};
#pragma unroll
            for (int d = 0; d < DB; ++d) o[b][d] = f32x4{0.f, 0.f, 0.f, 0.f};
        }
    };
    clear();

    typedef short v4i16 __attribute__((ext_vector_type(4)));
    typedef __attribute__((address_space(3))) v4i16 *lds_v4p;
    // Fragments, at an element of shared memory: of K at k0 + its tile's, with
    // the chunk 4 ks + g XOR-ed as above, which is an XOR of the whole index (a
    // tile starts at a multiple of HD); of V likewise
    constexpr int SLOTS = I8 ? 1 : 2;      // of a half's operand
    const int k0 = SLOTS * sp * TILE + i * HD + 8 * (g ^ KSWZ(i));
    const int vr = 4 * g + i / 4, v0 = SLOTS * (HALVES + sp) * TILE + vr * HD + 8 * ((lane & 3) / 2 ^ VSWZ(vr)) + (lane & 1) * 4;
    auto read_kf = [&](auto fc, int k) __attribute__((always_inline)) {
        constexpr int f = decltype(fc)::value;
        return *(const bf16x8 *)(ring[0] + (k ^ 32 * (f % NKS)) + (f / NKS) * 16 * HD);
    };
    auto read_v = [&](int v, int d, int j) __attribute__((always_inline)) {
        const bf16_t *const p = ring[0] + (v ^ 16 * d) + 32 * j * HD;
        const v4i16 x = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_v4p)(p));
        const v4i16 y = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_v4p)(p + 16 * HD));
        return __builtin_bit_cast(bf16x8, __builtin_shufflevector(x, y, 0, 1, 2, 3, 4, 5, 6, 7));
    };
    auto read_vf = [&](auto fc, int v) __attribute__((always_inline)) {
        constexpr int f = decltype(fc)::value;
        return read_v(v, f % DB, f / DB);
    };
    static_assert(NVF % AHEAD == 0 && NKF >= AHEAD, "fragment ring");
    f32x4 sc[QB][KB];
    // (P^T and the fragments under way are arguments: variables of the whole loop
    // would hold their registers through both turns)
    typedef bf16x8 Probs[NPJ][QB];
    typedef bf16x8 Frags[AHEAD];
    // S^T of a tile: its first AHEAD fragments are in fr
    auto qk = [&](int k, Frags &fr) __attribute__((always_inline)) {
        seq<0, NKF>([&](auto fc) __attribute__((always_inline)) {
            constexpr int f = decltype(fc)::value, kb = f / NKS, ks = f % NKS;
            const bf16x8 x = fr[f % AHEAD];
            if constexpr (f + AHEAD < NKF) fr[f % AHEAD] = read_kf(IntC<f + AHEAD>{}, k);
            seq<0, QB>([&](auto bc) __attribute__((always_inline)) {
                constexpr int b = decltype(bc)::value;
                sc[b][kb] = mfma(x, qf[b][ks], ks == 0 ? f32x4{} : sc[b][kb]);
            });
            if (!I8) __builtin_amdgcn_sched_barrier(0);        // (int8: the order pinned here would spill)
        });
    };
#if !I8
    const bf16x8 ones_row = __builtin_bit_cast(bf16x8, u32x4{0x3F803F80u, 0x3F803F80u, 0x3F803F80u, 0x3F803F80u});
#endif
    // O^T += V^T P^T of a tile, its first AHEAD fragments in fr, reading the
    // first fragments of the next K tile
    auto pv = [&](int v, int kn, const Probs &pf, Frags &fr) __attribute__((always_inline)) {
        seq<0, NVF>([&](auto fc) __attribute__((always_inline)) {
            constexpr int f = decltype(fc)::value, j = f / DB, d = f % DB;
            const bf16x8 x = fr[f % AHEAD];
            if constexpr (f + AHEAD < NVF) fr[f % AHEAD] = read_vf(IntC<f + AHEAD>{}, v);
            else fr[f % AHEAD] = read_kf(IntC<f + AHEAD - NVF>{}, kn);
            seq<0, QB>([&](auto bc) __attribute__((always_inline)) {
                constexpr int b = decltype(bc)::value;
                o[b][d] = mfma(x, pf[j][b], o[b][d]);
                // the sums of the rounded probabilities, a product with ones: two
                // instructions of the matrix cores for 16 additions
#if !I8
                if constexpr (d == 0) l[b] = mfma(ones_row, pf[j][b], l[b]);
#endif
            });
            if (!I8) __builtin_amdgcn_sched_barrier(0);        // (int8: the order pinned here would spill)
        });
    };
    auto key_of = [&](int it) { return (kt0 + HALVES * it + sp) * BN; };
    auto live = [&](int it) { return it < n_loc && key_of(it) <= most; };
    auto mask = [&](int it) __attribute__((always_inline)) {
#pragma unroll
        for (int kb = 0; kb < KB; ++kb) {
            const int key = key_of(it) + 16 * kb;
            const bool there = held(key);
#pragma unroll
            for (int b = 0; b < QB; ++b)
#pragma unroll
                for (int r = 0; r < 4; ++r)
                    if (!there || key + 4 * g + r > vis[b]) sc[b][kb][r] = -__builtin_inff();
        }
    };
    // Probabilities are relative to an offset m that is STALE above the largest
    // score of the tile that set it, so that they stay below 2 until a score is
    // past that by STALE + 1.  Whether one is, is seen in the probabilities
    // themselves (the top bit of the exponent, which a NaN has too): the maximum
    // of a tile's scores is needed only where the offset moves.
    auto move = [&](int b, const float *scale) __attribute__((always_inline)) {
        float top = -__builtin_inff();
#pragma unroll
        for (int kb = 0; kb < KB; ++kb)
#pragma unroll
            for (int r = 0; r < 4; ++r) top = fmaxf(top, sc[b][kb][r] * (I8 ? scale[16 * kb + r] : SCALE_LOG2));
        top = fmaxf(top, __shfl_xor(top, 16));
        top = fmaxf(top, __shfl_xor(top, 32));
        const float now = top > m[b] ? top + STALE : m[b];
        const float by = m[b] == now ? 1.f : pow2(m[b] - now);
        l[b] *= by;
#pragma unroll
        for (int d = 0; d < DB; ++d) o[b][d] *= by;
        m[b] = now;
    };
    auto masked = [&](int it) { return key_of(it) + BN - 1 > least || gaps; };
    // A tile that some row does not see whole is looked through for values that
    // are not finite: 0 times each of them.  Where there are any, the piece is
    // done again (see below): a second way through the turns would leave too few
    // registers for the first.
    bool far_seen = false;
    auto far_values = [&](int v) __attribute__((always_inline)) {
        f32x4 x = {0.f, 0.f, 0.f, 0.f};
        seq<0, NVF>([&](auto f) __attribute__((always_inline)) { x = mfma(read_vf(f, v), bf16x8{}, x); });
        const float y = (x[0] + x[1]) + (x[2] + x[3]);
        return __builtin_amdgcn_ballot_w64(y != y) != 0;
    };
#if I8
    // The softmax of tile `it`.  The values' scales are multiplied in; where some
    // row does not see a key, its scale may be anything.
    auto scaled = [&](int it, bool some, Probs &pf) __attribute__((always_inline)) {
        // (the scores of a tile that some row does not see whole have their
        // scales, and the mask, already)
        const float *const scale = (some ? ones : scales[sp][it & 1][0]) + 4 * g;
        u32 bits[QB] = {};
        float sum[QB] = {};
        auto all = [&](int first, int last) __attribute__((always_inline)) {
            seq<0, KB>([&](auto kc) __attribute__((always_inline)) {
                constexpr int kb = decltype(kc)::value;
                const f32x4 ks = *(const f32x4 *)(scale + 16 * kb), vs = *(const f32x4 *)&scales[sp][it & 1][1][16 * kb + 4 * g];
#pragma unroll
                for (int b = first; b < last; ++b) {
                    const float minus = -least_finite(m[b]);
                    float p[4];
#pragma unroll
                    for (int r = 0; r < 4; ++r) {
                        p[r] = pow2(__builtin_fmaf(sc[b][kb][r], ks[r], minus));
                        bits[b] |= __builtin_bit_cast(u32, p[r]);
                    }
                    sum[b] += (p[0] + p[1]) + (p[2] + p[3]);
#pragma unroll
                    for (int r = 0; r < 4; ++r) p[r] *= vs[r];
                    if (some) {
#pragma unroll
                        for (int r = 0; r < 4; ++r) p[r] = sc[b][kb][r] == -__builtin_inff() ? 0.f : p[r];
                    }
                    u32x4 w = __builtin_bit_cast(u32x4, pf[kb / 2][b]);
                    w[2 * (kb % 2)] = pack2(p[0], p[1]);
                    w[2 * (kb % 2) + 1] = pack2(p[2], p[3]);
                    pf[kb / 2][b] = __builtin_bit_cast(bf16x8, w);
                }
                __builtin_amdgcn_sched_barrier(0);
            });
        };
        all(0, QB);
        seq<0, QB>([&](auto bc) __attribute__((always_inline)) {
            constexpr int b = decltype(bc)::value;
            if (__builtin_amdgcn_ballot_w64(bits[b] >> 30 & 1) != 0) {
                move(b, scale);
                sum[b] = 0.f;
                all(b, b + 1);
            }
            l[b] += sum[b];
        });
    };
#else
    // probabilities of 16 keys; their bits
    auto probs = [&](int b, int kb, Probs &pf) __attribute__((always_inline)) {
        const float minus = -least_finite(m[b]);
        float p[4];
#pragma unroll
        for (int r = 0; r < 4; ++r) p[r] = pow2(__builtin_fmaf(sc[b][kb][r], SCALE_LOG2, minus));
        u32x4 w = __builtin_bit_cast(u32x4, pf[kb / 2][b]);
        const u32 x = pack2(p[0], p[1]), y = pack2(p[2], p[3]);
        w[2 * (kb % 2)] = x;
        w[2 * (kb % 2) + 1] = y;
        pf[kb / 2][b] = __builtin_bit_cast(bf16x8, w);
        return x | y;
    };
    // does one of two probabilities in `bits` have the exponent's top bit?
    auto past = [&](u32 bits) __attribute__((always_inline)) { return __builtin_amdgcn_ballot_w64((bits & 0x40004000u) != 0) != 0; };
    // The softmax turn of tile `it`, in KB x QB groups of exponentials with a share
    // of the loads in each; a turn that loads the sequence's last, partial tile
    // issues its loads first
    auto exps = [&](int it, auto act, Probs &pf) __attribute__((always_inline)) {
        u32 bits[QB] = {};
        const From kn = rows_of(it + 2), vn = next;
        next = kn;
        const u32 lk = slot(0, it & 1), lv = slot(1, (it + 1) & 1);
        auto groups = [&](auto loads) __attribute__((always_inline)) {
            seq<0, KB * QB>([&](auto gc) __attribute__((always_inline)) {
                constexpr int n = decltype(gc)::value, kb = n / QB, b = n % QB;
                constexpr int d0 = n * 2 * WL / (KB * QB), d1 = (n + 1) * 2 * WL / (KB * QB);
                if constexpr (decltype(loads)::value && d0 < WL && d1 > d0)
                    load(a.K, k_src, kn, lk, d0, d1 < WL ? d1 : WL, IntC<0>{});
                if constexpr (decltype(loads)::value && d1 > WL)
                    load(a.V, v_src, vn, lv, d0 > WL ? d0 - WL : 0, d1 - WL, IntC<0>{});
                if constexpr (decltype(act)::value) bits[b] |= probs(b, kb, pf);
                __builtin_amdgcn_sched_barrier(0);
            });
        };
        if (min(kn.end, vn.end) < BNW - 1) {
            load_whole(a.K, k_src, kn, lk);
            load_whole(a.V, v_src, vn, lv);
            groups(IntC<0>{});
        } else {
            groups(IntC<1>{});
        }
        if constexpr (decltype(act)::value) {
            seq<0, QB>([&](auto bc) __attribute__((always_inline)) {
                constexpr int b = decltype(bc)::value;
                if (past(bits[b])) {
                    move(b, nullptr);
#pragma unroll
                    for (int kb = 0; kb < KB; ++kb) probs(b, kb, pf);
                }
            });
        }
    };
#endif
    auto turn_end = [&] {
        __builtin_amdgcn_sched_barrier(0);
        __builtin_amdgcn_s_waitcnt(0xC07F);      // lgkmcnt(0): this wave's reads of shared memory are done
        asm volatile("s_barrier" ::: "memory");
    };
    if (sp == 1) turn_end();
    if (live(0)) {
        Frags fr;
        seq<0, AHEAD>([&](auto f) __attribute__((always_inline)) { fr[decltype(f)::value] = read_kf(f, k0); });
        qk(k0, fr);
    }
    turn_end();
#pragma nounroll
    for (int it = 0; it < n_it; ++it) {
        int v = v0 + (I8 ? 0 : (it & 1) * TILE), k = k0 + (I8 ? 0 : ((it + 1) & 1) * TILE);
#if I8
        // (what is formed from them is formed in each turn: held, it takes too
        // many registers)
        int kt = k_to, vt = v_to;
        asm volatile("" : "+v"(v), "+v"(k), "+v"(kt), "+v"(vt));
#endif
        Probs pf;
        const bool act = live(it), some = act && masked(it);
#if I8
        // K of the next tile and V of this one, which the matrix turn reads next,
        // and the scales that the next softmax turn reads
        widen(kx, kt, KSWZ(1024 / HD));
        widen(vx, vt, VSWZ(1024 / HD));
        put_scales((it + 1) & 1);
        __builtin_amdgcn_sched_barrier(0);
        const From kn = rows_of(it + 2);
        fetch(a.K, kn, kx);
        fetch(a.V, next, vx);
        fetch_scales(kn);
        next = kn;
        __builtin_amdgcn_sched_barrier(0);
        if (act) {
            if (some) {
#pragma unroll
                for (int kb = 0; kb < KB; ++kb) {
                    const f32x4 ks = *(const f32x4 *)&scales[sp][it & 1][0][16 * kb + 4 * g];
#pragma unroll
                    for (int b = 0; b < QB; ++b) sc[b][kb] *= ks;
                }
                mask(it);
            }
            scaled(it, some, pf);
        }
#else
        if (act) {
            if (some) mask(it);
            exps(it, IntC<1>{}, pf);
        } else {
            exps(it, IntC<0>{}, pf);
        }
        WAIT_VM(2 * WL);           // the loads of the softmax turn before this one have landed
#endif
        turn_end();
        // matrix turn: its waves go first at the issue port
        __builtin_amdgcn_s_setprio(2);
        if (act) {
            if (!I8 && some && !far_seen) far_seen = far_values(v);
            Frags fr;
            seq<0, AHEAD>([&](auto f) __attribute__((always_inline)) { fr[decltype(f)::value] = read_vf(f, v); });
            pv(v, k, pf, fr);
            if (live(it + 1)) qk(k, fr);
        }
        __builtin_amdgcn_s_setprio(0);
        turn_end();
    }
    WAIT_VM(0);
    if (HALVES == 2 && sp == 0) turn_end();
#if !I8
    if (far_seen) again = 1;
#endif
    __syncthreads();           // every wave is done with the ring (used again below)
#if !I8
    if (again) {
        // a tile after the other, with care for the values
        clear();
        for (int it = 0; it < n_it; ++it) {
            const From f = rows_of(it);
            load_whole(a.K, k_src, f, slot(0, 0));
            load_whole(a.V, v_src, f, slot(1, 0));
            WAIT_VM(0);
            __syncthreads();
            if (live(it)) {
                Frags fr;
                seq<0, AHEAD>([&](auto f) __attribute__((always_inline)) { fr[decltype(f)::value] = read_kf(f, k0); });
                qk(k0, fr);
                if (masked(it)) mask(it);
                Probs pf;
#pragma unroll
                for (int b = 0; b < QB; ++b) {
                    u32 bits = 0;
#pragma unroll
                    for (int kb = 0; kb < KB; ++kb) bits |= probs(b, kb, pf);
                    if (past(bits)) {
                        move(b, nullptr);
#pragma unroll
                        for (int kb = 0; kb < KB; ++kb) probs(b, kb, pf);
                    }
#pragma unroll
                    for (int j = 0; j < NPJ; ++j) {
                        const bf16x8 see = seen(sc[b][2 * j], sc[b][2 * j + 1]);
                        l[b] = mfma(ones_row, pf[j][b], l[b]);
#pragma unroll
                        for (int d = 0; d < DB; ++d) {
                            o[b][d] = add_far(__builtin_bit_cast(u32x4, read_v(v0, d, j)), pf[j][b], see, o[b][d]);
                            __builtin_amdgcn_sched_barrier(0);
                        }
                    }
                }
            }
            __syncthreads();
        }
    }
#endif

    // the two halves' states
#if I8
#pragma unroll
    for (int b = 0; b < QB; ++b) {
        l[b] += __shfl_xor(l[b], 16);
        l[b] += __shfl_xor(l[b], 32);
    }
#endif
#if HALVES == 2
    float *const other = (float *)ring[0] + rg * (QB * (32 + DB * 256));
    if (sp == 1) {
#pragma unroll
        for (int b = 0; b < QB; ++b) {
            if (g == 0) other[b * 32 + i] = m[b], other[b * 32 + 16 + i] = SUM(b);
#pragma unroll
            for (int d = 0; d < DB; ++d) *(f32x4 *)(other + QB * 32 + ((b * DB + d) * 64 + lane) * 4) = o[b][d];
        }
    }
    __syncthreads();
    if (sp == 1) return;
#endif
    float *state = a.P + (SPLIT ? (size_t)item.slot * STATE : 0);
    const int ie = lane_here() % 16, ge = lane_here() / 16;
#pragma unroll
    for (int b = 0; b < QB; ++b) {
#if HALVES == 2
        const float mo = other[b * 32 + ie], lo = other[b * 32 + 16 + ie], top = fmaxf(m[b], mo);
        const float by = m[b] == top ? 1.f : pow2(m[b] - top), byo = mo == top ? 1.f : pow2(mo - top);
        const float sum = SUM(b) * by + lo * byo;
#else
        const float top = m[b], sum = SUM(b);
#endif
        const int row = r0w + 16 * b + ie, r = row - r0;
        if (row >= rows) continue;
        if (SPLIT && item.pieces > 1 && ge == 0) state[r] = top, state[BM + r] = sum;
        bf16_t *p = a.O + ((size_t)(s.q0 + row / a.G) * a.HKV * a.G + item.h * a.G + row % a.G) * HD;
        auto sum_of = [&](int d) {
#if HALVES == 2
            return o[b][d] * by + *(const f32x4 *)(other + QB * 32 + ((b * DB + d) * 64 + 16 * ge + ie) * 4) * byo;
#else
            return o[b][d];
#endif
        };
        if (SPLIT && item.pieces > 1) {
#pragma unroll
            for (int d = 0; d < DB; ++d) *(f32x4 *)(state + 2 * BM + r * HD + 16 * d + 4 * ge) = sum_of(d);
            continue;
        }
        // two neighbouring sums of 16 channels: lanes 16 apart, of a row, trade
        // halves, so that each stores 16 bytes of one (64 prompts of 128 tokens 58.2 us
        // with 8 bytes, 52.6 with 16)
#pragma unroll
        for (int d = 0; d < DB; d += 2) {
            const u32x2 x = outputs(sum_of(d), sum), y = outputs(sum_of(d + 1), sum);
            const u32x2 lo = __builtin_bit_cast(u32x2, __builtin_amdgcn_permlane16_swap(x[0], y[0], false, false));
            const u32x2 hi = __builtin_bit_cast(u32x2, __builtin_amdgcn_permlane16_swap(x[1], y[1], false, false));
            *(u32x4 *)(p + 16 * (d + (ge & 1)) + 8 * (ge >> 1)) = u32x4{lo[0], hi[0], lo[1], hi[1]};
        }
    }
}
#endif

// ---------------------------------------------------------------------------
// The pieces of blocks that were cut
// ---------------------------------------------------------------------------
//
// A lane takes 4 channels.  By blocks (`by` 2): a workgroup takes the pieces of 2048
// / HD rows of a block, four or eight at once.  By rows, where there are few, which
// may have many pieces (`by` 1): a workgroup takes a row, a lane every 1024 / HD-th
// piece, eight at once.  The time is that of the way to memory and back, 6 us, and
// for large blocks of their states (26 MB of 200 blocks of 128 rows in two pieces,
// 10 us).
#if SPLIT
extern "C" __global__ __launch_bounds__(256) void rc_attention_seqs_join(SeqsArgs a) {
    __shared__ f32x4 po[4][HD / 4];
    __shared__ float pm[4], pl[4];
    const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), H = a.HKV * a.G;
    const size_t next = (size_t)a.HKV * STATE;          // of a block's next piece
    float m = -__builtin_inff(), l = 0.f;
    f32x4 o = {0.f, 0.f, 0.f, 0.f};
    auto add = [&](float mp, float lp, const f32x4 &op) {
        const float top = fmaxf(m, mp), x = m == top ? 1.f : pow2(m - top), y = mp == top ? 1.f : pow2(mp - top);
        l = l * x + lp * y;
        o = o * x + op * y;
        m = top;
    };
    constexpr int LANES = HD / 4, PAR = 64 / LANES;
    if (a.by == 2) {
        constexpr int ROWS_OF = 8 * PAR, SHARES = BM > ROWS_OF ? BM / ROWS_OF : 1;       // rows of a workgroup, workgroups of a block
        constexpr int ONCE = STAGES == 3 ? 4 : 8;
        Item item;
        if (!find<BLOCKS>(a, blockIdx.x / SHARES, item)) return;
        const int d = threadIdx.x % LANES * 4;
#pragma unroll
        for (int half = 0; half < 2; ++half) {
            const int r = blockIdx.x % SHARES * ROWS_OF + half * (ROWS_OF / 2) + threadIdx.x / LANES, row = item.block * BM + r;
            if (r >= BM || row >= item.s.n * a.G) continue;
            const float *state = a.P + (size_t)item.slot * STATE;
            m = -__builtin_inff(), l = 0.f;
            o = f32x4{0.f, 0.f, 0.f, 0.f};
            for (int p = 0; p < item.pieces; p += ONCE) {
                float mp[ONCE], lp[ONCE];
                f32x4 op[ONCE];
#pragma unroll
                for (int i = 0; i < ONCE; ++i) {
                    const float *x = state + (size_t)min(p + i, item.pieces - 1) * next;
                    mp[i] = x[r], lp[i] = x[BM + r];
                    op[i] = *(const f32x4 *)(x + 2 * BM + r * HD + d);
                }
#pragma unroll
                for (int i = 0; i < ONCE; ++i)
                    if (p + i < item.pieces) add(mp[i], lp[i], op[i]);
            }
            bf16_t *to = a.O + ((size_t)(item.s.q0 + row / a.G) * H + item.h * a.G + row % a.G) * HD + d;
            *(u32x2 *)to = outputs(o, l);
        }
        return;
    }
    const long long at = blockIdx.x;
    const int token = (int)(at / H), head = (int)(at % H);
    Item item;
    if (!find<ROWS>(a, token, item) || item.pieces == 1) return;
    const int row = (token - item.s.q0) * a.G + head % a.G, r = row % BM;
    const float *state = a.P + ((size_t)(item.slot + (item.block - 1 - row / BM) * item.pieces) * a.HKV + head / a.G) * STATE;
    const int part = lane / LANES, d = lane % LANES * 4;
    constexpr int step = 4 * PAR;
    for (int p0 = w * PAR + part; p0 - part < item.pieces; p0 += 8 * step) {
        float mp[8], lp[8];
        f32x4 op[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const float *x = state + (size_t)min(p0 + i * step, item.pieces - 1) * next;
            mp[i] = x[r], lp[i] = x[BM + r];
            op[i] = *(const f32x4 *)(x + 2 * BM + r * HD + d);
        }
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (p0 + i * step < item.pieces) add(mp[i], lp[i], op[i]);
    }
#pragma unroll
    for (int x = LANES; x < 64; x <<= 1) {
        const f32x4 other = {__shfl_xor(o[0], x), __shfl_xor(o[1], x), __shfl_xor(o[2], x), __shfl_xor(o[3], x)};
        add(__shfl_xor(m, x), __shfl_xor(l, x), other);
    }
    if (part == 0) po[w][d / 4] = o;
    if (lane == 0) pm[w] = m, pl[w] = l;
    __syncthreads();
    if (w) return;
#pragma unroll
    for (int x = 1; x < 4; ++x) add(pm[x], pl[x], po[x][d / 4]);
    if (part == 0) *(u32x2 *)(a.O + (size_t)at * HD + d) = outputs(o, l);
}
#endif
