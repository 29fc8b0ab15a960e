// Attention over sequences of different lengths for gfx950: over a paged cache
// of keys and values (bf16, or int8 with an fp32 scale for each token and
// head), or over sequences packed behind each other; grouped heads, causal or
// not, any number of new rows a sequence.
//
// Compile-time schedule (generated prologue):
//   BM      rows of a work item (TileSize), see below
//   NW      waves that share an item's keys (Parallel)
//   STAGES  1: a tile is loaded, then computed; 2: the next tile's loads are
//           under way meanwhile (ComputeLocation)
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

#define QB (BM / 16)               // blocks of 16 rows
#define BN 32                      // keys of a tile
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
};

__device__ __forceinline__ int limit(int x, int lo, int hi) { return x < lo ? lo : x > hi ? hi : x; }
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

// A sequence's rows are cut into blocks of BM, and with SPLIT its keys into
// pieces of at most `most` tiles, the same number for each block.  `most` is
// the work of all sequences over the workgroups that it is cut for (a.slots), so
// that pieces of blocks that are cut are at most 2 a.slots: each takes more than
// half of it.  Item j is piece by piece, the sequence's last block (the one that
// sees most keys) first, head by head; JOIN: block by block of what is cut.
template <bool JOIN> __device__ __forceinline__ bool find(const SeqsArgs &a, int index, Item &item) {
    const int lane = threadIdx.x & 63;
    item.h = index % a.HKV;
    int j = index / a.HKV;
    int most = 1 << 30;
#if SPLIT
    unsigned long long work = 0;
    for (int c = 0; c < a.B; c += 64) {
        unsigned long long w = 0;
        if (c + lane < a.B) {
            const Seq s = sequence(a, c + lane);
            w = (unsigned long long)blocks_of(a, s) * tiles_of(s);
        }
#pragma unroll
        for (int d = 1; d < 64; d <<= 1) w += __shfl_xor(w, d);
        work += w;
    }
    work = (work * a.HKV + a.slots - 1) / a.slots;
    most = work < LEAST ? LEAST : work > (1 << 30) ? 1 << 30 : (int)work;
#endif
    int slot = 0;
    for (int c = 0; c < a.B; c += 64) {
        Seq s = {};
        int blocks = 0, pieces = 1;
        if (c + lane < a.B) {
            s = sequence(a, c + lane);
            blocks = blocks_of(a, s);
            if (SPLIT) pieces = max(1, (tiles_of(s) + most - 1) / most);
        }
        const int cut = pieces > 1 ? blocks * pieces : 0;      // states that the sequence leaves
        const int items = JOIN ? (pieces > 1 ? blocks : 0) : blocks * pieces;
        int sum = items, sums = cut;
#pragma unroll
        for (int d = 1; d < 64; d <<= 1) {
            const int x = __shfl_up(sum, d), y = __shfl_up(sums, d);
            if (lane >= d) sum += x, sums += y;
        }
        const unsigned long long past = __builtin_amdgcn_ballot_w64(sum > j);
        if (past) {
            const int at = __builtin_ctzll(past);
            auto of = [&](int x) { return __builtin_amdgcn_readlane(x, at); };
            item.s.q0 = of(s.q0), item.s.n = of(s.n), item.s.k0 = of(s.k0), item.s.len = of(s.len), item.s.keys = of(s.keys);
            const int i = j - of(sum - items), k = of(blocks);
            item.pieces = of(pieces);
            const int order = JOIN ? i : i / item.pieces;
            item.block = k - 1 - order;
            item.piece = JOIN ? 0 : i % item.pieces;
            item.slot = ((slot + of(sums - cut)) + order * item.pieces + item.piece) * a.HKV + item.h;
            // (for readlane's sake: which sequence, to find its row of the table)
            item.s.k0 = PAGED ? c + at : item.s.k0;
            return true;
        }
        j -= __builtin_amdgcn_readlane(sum, 63);
        slot += __builtin_amdgcn_readlane(sums, 63);
    }
    return false;
}

// State of a piece: m and l of its rows, then their sums of p V
#define STATE (BM * (HD + 2))

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

__device__ __forceinline__ u32 pack2(float a, float b) {
    return __builtin_bit_cast(u32, __builtin_convertvector((f32x2){a, b}, bf16x2));
}
__device__ __forceinline__ f32x4 mfma(const bf16x8 &a, const bf16x8 &b, const f32x4 &c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
}
// byte e of w as a float
__device__ __forceinline__ float byte(u32 w, int e) { return (float)(signed char)(w >> (8 * e)); }

struct Tile {
    u32x4 k[2][I8 ? NKS / 2 : NKS];
    u32 v[8][DE * ELT / 4];
#if I8
    f32x4 ks[2], vs[2];
#endif
    int held;          // of the two 16-key blocks
};

extern "C" __global__ __launch_bounds__(64 * NW) void rc_attention_seqs(SeqsArgs a) {
    __shared__ __attribute__((aligned(16))) float osum[NW][BM][HD + 4];
    __shared__ float om[NW][BM], ol[NW][BM];
    const int lane = threadIdx.x & 63, w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int i = lane % 16, g = lane / 16;
    Item item;
    if (!find<false>(a, blockIdx.x, item)) return;
    const Seq s = item.s;
    const int rows = s.n * a.G, r0 = item.block * BM;

    // queries, and the last key that each sees
    bf16x8 q[QB][NKS];
    int vis[QB], least = 1 << 30;
#pragma unroll
    for (int b = 0; b < QB; ++b) {
        const int r = r0 + 16 * b + i, token = r / a.G;
        vis[b] = 1 << 30;          // (rows that there are not)
#pragma unroll
        for (int ks = 0; ks < NKS; ++ks) q[b][ks] = bf16x8{};
        if (r < rows) {
            vis[b] = s.vis(token, a.causal);
            least = min(least, vis[b]);
            const bf16_t *p = a.Q + ((size_t)(s.q0 + token) * a.HKV * a.G + item.h * a.G + r % a.G) * HD;
#pragma unroll
            for (int ks = 0; ks < NKS; ++ks)
                q[b][ks] = *(const bf16x8 *)(p + (I8 ? 64 * (ks / 2) + 16 * g + 8 * (ks % 2) : 32 * ks + 8 * g));
        }
    }
#pragma unroll
    for (int d = 1; d < 16; d <<= 1) least = min(least, __shfl_xor(least, d));
    least = __builtin_amdgcn_readfirstlane(least);

    // tiles of the block's last row, of the piece, of the wave
    const int last = s.vis((min(rows, r0 + BM) - 1) / a.G, a.causal);
    const int tiles = (max(last + 1, 0) + BN - 1) / BN, share = (tiles + item.pieces - 1) / item.pieces;
    const int t0 = item.piece * share + w, t1 = min(tiles, (item.piece + 1) * share);
    const int nt = __builtin_amdgcn_readfirstlane(t1 > t0 ? (t1 - t0 + NW - 1) / NW : 0);

    f32x4 o[QB][DE];
    float m[QB], minus[QB], l[QB];         // minus: -m, or 0 while no key was seen
#pragma unroll
    for (int b = 0; b < QB; ++b) {
        m[b] = -__builtin_inff();
        minus[b] = l[b] = 0.f;
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
                    u32 far = 0;
#pragma unroll
                    for (int e = 0; e < DE * ELT / 4; ++e) {
                        u32 &v = x.v[4 * c + r][e];
                        v = there ? v : 0;
                        far |= ((v & 0x7F80u) == 0x7F80u) | ((v & 0x7F800000u) == 0x7F800000u);
                    }
                    apart |= far != 0;
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
                minus[b] = now == -__builtin_inff() ? 0.f : -now;
            }
            float pr[2][4];
#pragma unroll
            for (int c = 0; c < 2; ++c)
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    pr[c][r] = pow2(__builtin_fmaf(sc[b][c][r], SCALE_LOG2, minus[b]));
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
            // Key by key, so that a row leaves out what it does not see (0 times
            // an infinity or a NaN is a NaN)
#pragma nounroll
            for (int k = 0; k < BN; ++k) {
                // (what is formed from V is formed anew: held, it takes as many registers again)
#pragma unroll
                for (int j = 0; j < 8; ++j)
#pragma unroll
                    for (int e = 0; e < DE * ELT / 4; ++e) asm volatile("" : "+v"(x.v[j][e]));
                const int at = k / 16 * 4 + k % 4;      // its place among the 8 of the lanes g = k % 16 / 4
                u32x4 only;
#pragma unroll
                for (int j = 0; j < 4; ++j) only[j] = g == k % 16 / 4 && at / 2 == j ? (at % 2 ? 0xFFFF0000u : 0xFFFFu) : 0u;
#pragma unroll
                for (int b = 0; b < QB; ++b)
#pragma unroll
                    for (int e = 0; e < DE; ++e) {
                        const f32x4 t = mfma(__builtin_bit_cast(bf16x8, values(e) & only),
                                             __builtin_bit_cast(bf16x8, __builtin_bit_cast(u32x4, p[b]) & only), f32x4{0.f, 0.f, 0.f, 0.f});
                        if (key0 + k <= vis[b]) o[b][e] += t;
                        __builtin_amdgcn_sched_barrier(0);
                    }
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
            const float inv = sum == 0.f ? 0.f : 1.f / sum;
            const int row = r0 + r;
            bf16_t *p = a.O + ((size_t)(s.q0 + row / a.G) * a.HKV * a.G + item.h * a.G + row % a.G) * HD + d;
            *(u32x2 *)p = u32x2{pack2(out[0] * inv, out[1] * inv), pack2(out[2] * inv, out[3] * inv)};
        }
    }
}

// ---------------------------------------------------------------------------
// Rows of sequences that were cut: a wave takes a row.
// ---------------------------------------------------------------------------
#if SPLIT
extern "C" __global__ __launch_bounds__(256) void rc_attention_seqs_join(SeqsArgs a) {
    const int lane = threadIdx.x & 63;
    const long long at = (long long)blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    Item item;
    if (!find<true>(a, (int)(at / BM), item)) return;
    const int r = (int)(at % BM), row = item.block * BM + r;
    if (row >= item.s.n * a.G) return;
    const float *state = a.P + (size_t)item.slot * STATE;
    const size_t next = (size_t)a.HKV * STATE;          // of the block's next piece
    float top = -__builtin_inff();
    for (int p = lane; p < item.pieces; p += 64) top = fmaxf(top, state[p * next + r]);
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) top = fmaxf(top, __shfl_xor(top, d));
    constexpr int PER = HD / 64;
    float sum = 0.f, out[PER] = {};
#pragma unroll 8
    for (int p = 0; p < item.pieces; ++p) {
        const float *x = state + p * next;
        const float by = x[r] == top ? 1.f : pow2(x[r] - top);
        sum += x[BM + r] * by;
#pragma unroll
        for (int e = 0; e < PER; ++e) out[e] += x[2 * BM + r * HD + lane * PER + e] * by;
    }
    const float inv = sum == 0.f ? 0.f : 1.f / sum;
    bf16_t *o = a.O + ((size_t)(item.s.q0 + row / a.G) * a.HKV * a.G + item.h * a.G + row % a.G) * HD + lane * PER;
#pragma unroll
    for (int e = 0; e < PER; ++e) o[e] = __builtin_bit_cast(bf16_t, (__bf16)(out[e] * inv));
}
#endif
