// int8 x int8 -> int32 MFMA matrix product for gfx950 with a fused epilogue:
//   acc[m][n] = sum_k A[m][k] B[n][k]              (int32, exact)
//   out[m][n] = acc * (sa[m] * sb[n]) (+ bias[n])  (fp32, rounded once)
// and the gated form, two products of one A:
//   out[m][n] = bf16(SiLU(g) * u).
// Both operands have K contiguous, the layout the matrix instructions take:
// 16 consecutive k are one register fragment of a lane.
//
// Compile-time schedule (generated prologue); the sizes are arguments:
//   TM TN TK     workgroup tile, TK in elements = bytes (TileSize); GATED: a
//                tile of TN weight rows is TN / 2 gate and TN / 2 up rows
//   WM WN WK     waves along M, N and K (Parallel); NT = 64 * WM * WN * WK
//   MF           MFMA shape: 16 -> v_mfma_i32_16x16x64_i8,
//                            32 -> v_mfma_i32_32x32x32_i8
//   STAGES       1: LDS double buffer with register prefetch of the next K
//                tile, any sizes (ComputeLocation); 2: a ring of NSTAGE LDS
//                buffers filled by direct-to-LDS buffer loads issued
//                NSTAGE - 1 tiles ahead (K a multiple of 16: a lane moves 16
//                aligned bytes); 3: streaming, for few rows of A - operands
//                go straight to registers in the MFMA's layout, the WK waves
//                of a tile take K in turns and add up through LDS
//   SPLITS       the K range cut over that many workgroups of a tile, whose
//                int32 sums rc_gemm_i8_join adds and finishes (Parallel)
//   ORDER        0: tile n fastest; 1: bands of 8 M tiles, m fastest within
//                a band, each XCD owning a contiguous range
//   TAIL         1 (ring): the last TAIL_TILES tiles, those of a partial round
//                of workgroups, run as twice as many of half the height
//   OCC          waves per SIMD the register allocation must leave room for
//   BIAS F32 GATED   operator flags: bias added, fp32 output, gated form
//
// Edges: rows past M or N read the last row and are not stored; a K tail
// reads zeros.

#define NT (64 * WM * WN * WK)
#define WTN (TN / WN)
#define FN (WTN / MF)
#define CPR (TK / 16)                                       // 16-byte chunks of a tile row
#define RPL ((16 / CPR) > 0 ? (16 / CPR) : 1)
#define TNO (GATED ? TN / 2 : TN)                           // output columns of a tile
#define WTO (GATED ? WTN / 2 : WTN)                         // of a wave

typedef unsigned short bf16_t;
typedef signed char i8;
typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef int i32x16 __attribute__((ext_vector_type(16)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef unsigned int u32x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));

#if MF == 16
typedef i32x4 accT;
#define ACCN 4
#define KSTEP 64
#else
typedef i32x16 accT;
#define ACCN 16
#define KSTEP 32
#endif

struct GemmI8Args {
    const i8 *A;                // [M][K]
    const i8 *B0, *B1;          // [N][K] (B1: the up weight of GATED)
    const float *sa;            // [M]
    const float *sb0, *sb1;     // [N]
    const float *bias;          // [N] (BIAS)
    void *C;                    // [M][N]
    int *P;                     // [SPLITS][M][GATED ? 2 : 1][N rounded up to 4] (SPLITS > 1)
    long long M;
    int N, K;
    int KP;                     // K of one split: a multiple of TK, or K
    int tail;                   // tiles that run in halves (TAIL)
};

template <int V> struct IntC { static constexpr int value = V; };
// seq<A, B>(f): f(IntC<A>), f(IntC<A + 1>), ... f(IntC<B - 1>), every index a
// constant
template <class T, T... I> struct ISeq {};
template <int A, class F, int... I> __device__ __forceinline__ void seq_calls(F &f, ISeq<int, I...>) {
    (f(IntC<A + I>{}), ...);
}
template <int A, int B, class F> __device__ __forceinline__ void seq(F &&f) {
    if constexpr (B > A) seq_calls<A>(f, __make_integer_seq<ISeq, int, B - A>{});
}

__device__ __forceinline__ accT mfma(const i32x4 &a, const i32x4 &b, const accT &c) {
#if MF == 16
    return __builtin_amdgcn_mfma_i32_16x16x64_i8(a, b, c, 0, 0, 0);
#else
    return __builtin_amdgcn_mfma_i32_32x32x32_i8(a, b, c, 0, 0, 0);
#endif
}

// XOR applied to a row's 16-byte chunk indices, so that the 16 lanes served
// together by a 128-bit LDS access (0-3, 12-15, 20-23 and 24-27, then 4-11,
// 16-19 and 28-31, and so on) hit distinct 16-byte columns of the 256 bytes
// that the banks span.
__device__ __forceinline__ int swz_x(int row) {
    if (CPR == 4) return (0x78 >> (row / 2 % 8 & 6)) & 3;   // 0, 2, 3, 1 by row / 4 % 4
    return (row / RPL) % CPR;
}
__device__ __forceinline__ int swz(int row, int chunk) { return row * TK + ((chunk ^ swz_x(row)) << 4); }

// 16 elements at p, of which `left` are in the row (the rest reads zero)
__device__ __forceinline__ i32x4 load16(const i8 *p, int left) {
    i32x4 v = {0, 0, 0, 0};
    if (left >= 16) {
        __builtin_memcpy(&v, p, 16);
    } else {
        unsigned w[4] = {0, 0, 0, 0};
#pragma unroll
        for (int j = 0; j < 16; ++j)
            if (j < left) w[j / 4] |= (unsigned)(unsigned char)p[j] << (8 * (j % 4));
        v = i32x4{(int)w[0], (int)w[1], (int)w[2], (int)w[3]};
    }
    return v;
}

__device__ __forceinline__ float silu(float x) {
    // x * sigmoid(x); exp(-x) as 2^(-x log2 e) on the hardware exp2 unit
    return x / (1.0f + __builtin_amdgcn_exp2f(-x * 1.4426950408889634f));
}

// Columns n .. n + 3 of row m from their sums (GATED: g, and u the second
// weight's); `whole`: all four exist and rows start on four columns.
__device__ __forceinline__ void finish(const GemmI8Args &a, long long m, int n, const int (&g)[4], const int (&u)[4], bool whole) {
    const float sa = a.sa[m];
    float v[4];
    auto one = [&](int r) {
        float y = (float)g[r] * (sa * a.sb0[n + r]);
#if GATED
        y = silu(y) * ((float)u[r] * (sa * a.sb1[n + r]));
#endif
#if BIAS
        y += a.bias[n + r];
#endif
        return y;
    };
    const size_t at = (size_t)m * a.N + n;
    if (whole) {
#pragma unroll
        for (int r = 0; r < 4; ++r) v[r] = one(r);
#if F32
        *(f32x4 *)((float *)a.C + at) = f32x4{v[0], v[1], v[2], v[3]};
#else
        u32x2 p;
        p[0] = __builtin_bit_cast(unsigned, __builtin_convertvector((f32x2){v[0], v[1]}, bf16x2));
        p[1] = __builtin_bit_cast(unsigned, __builtin_convertvector((f32x2){v[2], v[3]}, bf16x2));
        *(u32x2 *)((bf16_t *)a.C + at) = p;
#endif
        return;
    }
#pragma unroll
    for (int r = 0; r < 4; ++r) {
        if (n + r >= a.N) continue;
        const float y = one(r);
#if F32
        ((float *)a.C)[at + r] = y;
#else
        ((bf16_t *)a.C)[at + r] = __builtin_bit_cast(bf16_t, (__bf16)y);
#endif
    }
}

#if STAGES == 1
#define LDS_BYTES (2 * (TM + TN) * TK)
#elif STAGES == 2
#define LDS_BYTES (NSTAGE * (TM + TN) * TK)
#else
#define LDS_BYTES (WK * (TM / 16) * (TN / 16) * 1024)
#endif

// The tile of HM rows at row m0 and column tile nt, of K split kz.
template <int HM> __device__ __forceinline__ void product(const GemmI8Args &args, i8 *lds, long long m0, int nt, int kz) {
    constexpr int WTM = HM / WM, FM = WTM / MF;
    const int tid = threadIdx.x;
    const int lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);     // wave-uniform: scalar registers
    __builtin_assume(wave >= 0 && wave < WM * WN * WK);
    const int wm = wave / WN % WM, wn = wave % WN;
    const int ld = args.K, N = args.N;                             // rows of both operands are K long
    const int n0 = nt * TNO;                                       // first output column
    const int mrows = (int)min((long long)HM, args.M - m0);
    const int ncols = min(TNO, N - n0);
    // this split's K range: the operands start at its first k
    const int k_first = kz * args.KP;
    const int K = SPLITS > 1 ? min(args.KP, ld - k_first) : ld;
    const i8 *const Ab = args.A + (size_t)m0 * ld + k_first;
    const i8 *const B0 = args.B0 + (size_t)n0 * ld + k_first;
#if GATED
    const i8 *const B1 = args.B1 + (size_t)n0 * ld + k_first;
    // weight row b of the tile: of wave column b / WTN, its first WTO rows
    // gate and the others up, so that one lane ends up with both sums of an
    // output
#define SRC_ROW(b) ((b) / WTN * WTO + (b) % WTO)
#define SRC_UP(b) ((b) % WTN >= WTO)
#else
    const i8 *const B1 = B0;
#define SRC_ROW(b) (b)
#define SRC_UP(b) false
#endif

    accT acc[FM][FN];
#pragma unroll
    for (int i = 0; i < FM; ++i)
#pragma unroll
        for (int j = 0; j < FN; ++j)
#pragma unroll
            for (int r = 0; r < ACCN; ++r) acc[i][j][r] = 0;

    // byte offset of this lane's fragment of each k-step in a tile's rows
    constexpr int KS = TK / KSTEP;
    int foff[KS];
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) foff[ks] = swz(lane % MF, ks * (KSTEP / 16) + lane / MF);

#if STAGES == 1
    constexpr int BUF = (HM + TN) * TK;
    // chunk v of a tile: row v / CPR, chunk v % CPR of it
    constexpr int CH = ((HM + TN) * CPR + NT - 1) / NT;            // per thread
    const i8 *src[CH];
    int kc[CH], dst[CH];
#pragma unroll
    for (int i = 0; i < CH; ++i) {
        const int v = tid + i * NT;
        const int row = v / CPR, c = v % CPR;
        kc[i] = c * 16;
        if (row < HM) {
            dst[i] = swz(row, c);
            src[i] = Ab + (size_t)min(row, mrows - 1) * ld + kc[i];
        } else {
            const int b = row - HM;
            dst[i] = v < (HM + TN) * CPR ? HM * TK + swz(b, c) : -1;
            src[i] = (SRC_UP(b) ? B1 : B0) + (size_t)min(SRC_ROW(b), ncols - 1) * ld + kc[i];
        }
    }
    i32x4 reg[CH];
    auto fetch = [&](int k0) {
        if (k0 + TK <= K) {
#pragma unroll
            for (int i = 0; i < CH; ++i) __builtin_memcpy(&reg[i], src[i] + k0, 16);
        } else {
#pragma unroll
            for (int i = 0; i < CH; ++i) reg[i] = load16(src[i] + k0, K - k0 - kc[i]);
        }
    };
    auto put = [&](int b) {
#pragma unroll
        for (int i = 0; i < CH; ++i)
            if (dst[i] >= 0) *(i32x4 *)(lds + b * BUF + dst[i]) = reg[i];
    };
    const int tiles = (K + TK - 1) / TK;
    fetch(0);
    put(0);
    __syncthreads();
    for (int t = 0; t < tiles; ++t) {
        // buffer (t + 1) & 1 was last read in iteration t - 1, which ended
        // with a barrier
        if (t + 1 < tiles) fetch((t + 1) * TK);
        const i8 *la = lds + (t & 1) * BUF + wm * WTM * TK, *lb = lds + (t & 1) * BUF + (HM + wn * WTN) * TK;
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) {
            i32x4 fa[FM], fb[FN];
#pragma unroll
            for (int i = 0; i < FM; ++i) fa[i] = *(const i32x4 *)(la + i * MF * TK + foff[ks]);
#pragma unroll
            for (int j = 0; j < FN; ++j) fb[j] = *(const i32x4 *)(lb + j * MF * TK + foff[ks]);
#pragma unroll
            for (int i = 0; i < FM; ++i)
#pragma unroll
                for (int j = 0; j < FN; ++j) acc[i][j] = mfma(fb[j], fa[i], acc[i][j]);
        }
        if (t + 1 < tiles) put((t + 1) & 1);
        __syncthreads();
    }
#elif STAGES == 2
    // buffer_load_dwordx4 ... lds moves 64 lanes x 16 B into 1 KiB of LDS at
    // a wave-uniform base (M0); the swizzle is applied by choosing which
    // chunk a lane fetches.  Tile t goes to buffer t % NSTAGE; the fragments
    // of tile t + 1's first k-step are read during tile t's last one, so a
    // tile starts its MFMAs right after its one barrier, which also frees
    // the buffer of tile t - 1.  The loads are inline assembly, invisible to
    // the compiler's wait counts; the waits below order the ring (loads
    // complete in order).
    typedef __attribute__((address_space(3))) i8 *lds_p;
    constexpr int STAGE_BYTES = (HM + TN) * TK;
    constexpr int NWV = WM * WN;
    constexpr int A_WL = HM * TK / 1024 / NWV;          // wave-loads per wave, A tile
    constexpr int B_WL = TN * TK / 1024 / NWV;          // weight tile
    constexpr int LPT = A_WL + B_WL;
    constexpr int RPW = 1024 / TK;                      // rows of a wave-load
    constexpr unsigned OOB = 0x80000000u;               // past every tile's rows: loads zeros
    i8 *const ring = lds;
    // A resource covers the tile's rows from this split's first k on: rows
    // past M or N are out of its range and load zeros, and offsets stay in
    // 32 bits whatever the operands' sizes.
    auto rsrc = [](const void *base, int bytes) {
        const unsigned long long a = (unsigned long long)base;
        i32x4 r;
        r[0] = __builtin_amdgcn_readfirstlane((int)(unsigned)a);
        r[1] = __builtin_amdgcn_readfirstlane((int)((unsigned)(a >> 32) & 0xFFFFu));   // stride 0
        r[2] = __builtin_amdgcn_readfirstlane(bytes);
        r[3] = 0x00020000;                                                             // raw dword access
        return r;
    };
    const i32x4 rsA = rsrc(Ab, mrows * ld - k_first);
    const i32x4 rsB0 = rsrc(B0, ncols * ld - k_first);
#if GATED
    const i32x4 rsB1 = rsrc(B1, ncols * ld - k_first);
    // a wave-load's rows are all of one weight: 16 of them divide WTO
    i32x4 rsB[B_WL];
#pragma unroll
    for (int j = 0; j < B_WL; ++j) {
        const bool up = SRC_UP((wave * B_WL + j) * RPW);
#pragma unroll
        for (int q = 0; q < 4; ++q) rsB[j][q] = up ? rsB1[q] : rsB0[q];
    }
#endif
    unsigned a_off[A_WL], b_off[B_WL];                  // bytes, at k = 0
    auto chunk_k = [&](int row) { return (((lane % CPR) ^ swz_x(row)) << 4); };
    auto a_row = [&](int j) { return (wave * A_WL + j) * RPW + lane / CPR; };
    auto b_row = [&](int j) { return (wave * B_WL + j) * RPW + lane / CPR; };
#pragma unroll
    for (int j = 0; j < A_WL; ++j) a_off[j] = (unsigned)(a_row(j) * ld + chunk_k(a_row(j)));
#pragma unroll
    for (int j = 0; j < B_WL; ++j) b_off[j] = (unsigned)(SRC_ROW(b_row(j)) * ld + chunk_k(b_row(j)));
    // the last tile's chunks past K: zeros (called ahead of its loads)
    const int tiles = (K + TK - 1) / TK;
    auto mask_tail = [&]() {
        const int left = K - (tiles - 1) * TK;
#pragma unroll
        for (int j = 0; j < A_WL; ++j) a_off[j] = chunk_k(a_row(j)) < left ? a_off[j] : OOB;
#pragma unroll
        for (int j = 0; j < B_WL; ++j) b_off[j] = chunk_k(b_row(j)) < left ? b_off[j] : OOB;
    };
    auto dma = [&](unsigned off, const i32x4 &rs, int koff, unsigned to) __attribute__((always_inline)) {
        asm volatile("s_mov_b32 m0, %3\n\ts_nop 0\n\tbuffer_load_dwordx4 %0, %1, %2 offen lds"
                     :: "v"(off), "s"(rs), "s"(koff), "s"(to) : "memory", "m0");
    };
    const unsigned ring0 = (unsigned)(size_t)(lds_p)ring;
    // wave-load d of tile t into the buffer at LDS address sb
    auto issue_one = [&](auto dc, int t, unsigned sb) __attribute__((always_inline)) {
        constexpr int d = decltype(dc)::value;
        if constexpr (d < A_WL) {
            dma(a_off[d], rsA, t * TK, sb + (unsigned)((wave * A_WL + d) * 1024));
        } else {
            constexpr int j = d - A_WL;
#if GATED
            dma(b_off[j], rsB[j], t * TK, sb + (unsigned)(HM * TK + (wave * B_WL + j) * 1024));
#else
            dma(b_off[j], rsB0, t * TK, sb + (unsigned)(HM * TK + (wave * B_WL + j) * 1024));
#endif
        }
    };
    // s_waitcnt with only the vector-memory count constrained
#define WAIT_VM(n) __builtin_amdgcn_s_waitcnt(((n) & 15) | ((((n) >> 4) & 3) << 14) | (7 << 4) | (15 << 8))
    // Fragments: a row's A fragment is replaced by the next k-step's once its
    // MFMAs are issued; the weight's are used to the end of the k-step, and
    // have a second set.  (Two whole sets are 32 registers more in 256 x 256
    // tiles of 8 waves, which then spill.)
    i32x4 fa[FM], fb[2][FN];
    constexpr int NMF = FM * FN;
    // One k-step: its MFMAs, with the next k-step's fragment reads and this
    // k-step's share of a later tile's loads spread between them, in an order
    // the scheduler keeps: the matrix, LDS and memory pipes run side by side.
    constexpr auto b_before = [](int m) constexpr {                // weight reads before MFMA m
        const int r = (m * FN * 4 + 3 * NMF - 1) / (3 * NMF);
        return r < FN ? r : FN;
    };
    constexpr auto loads_before = [](int s) constexpr {
        const int d = NSTAGE > 3 || LPT > KS * NMF ? s * LPT / (KS * NMF) : s;
        return d < LPT ? d : LPT;
    };
    // `set`: the weight fragments to use; ln, ksn: LDS buffer and k-step of the next
    auto kstep = [&](auto set, unsigned ln, int ksn, auto ksc, auto loads, int t, unsigned sb) __attribute__((always_inline)) {
        constexpr int bs = decltype(set)::value;
        const i8 *la = ring + ln + wm * WTM * TK + foff[ksn];
        const i8 *lb = ring + ln + HM * TK + wn * WTN * TK + foff[ksn];
        seq<0, NMF>([&](auto mc) __attribute__((always_inline)) {
            constexpr int m = decltype(mc)::value, i = m / FN, j = m % FN;
            seq<b_before(m), b_before(m + 1)>([&](auto r) __attribute__((always_inline)) {
                fb[1 - bs][decltype(r)::value] = *(const i32x4 *)(lb + decltype(r)::value * MF * TK);
            });
            if constexpr (i > 0 && j == (FN > 1 ? 1 : 0)) fa[i - 1] = *(const i32x4 *)(la + (i - 1) * MF * TK);
            if constexpr (decltype(loads)::value) {
                constexpr int st = decltype(ksc)::value * NMF + m;
                seq<loads_before(st), loads_before(st + 1)>(
                    [&](auto d) __attribute__((always_inline)) { issue_one(d, t, sb); });
            }
            acc[i][j] = mfma(fb[bs][j], fa[i], acc[i][j]);
            __builtin_amdgcn_sched_barrier(0);
        });
        fa[FM - 1] = *(const i32x4 *)(la + (FM - 1) * MF * TK);
        __builtin_amdgcn_sched_barrier(0);
    };
    // buffers of tiles t, t + 1 and t - 1 (the one tile t + NSTAGE - 1 goes to)
    int cur = 0, nx = 1, fill = NSTAGE - 1;
    // tile t, its first k-step's weight fragments in set `par`
    auto tile = [&](int t, auto par, auto loads) __attribute__((always_inline)) {
        const unsigned sb = ring0 + (unsigned)(fill * STAGE_BYTES);
        seq<0, KS>([&](auto ksc) __attribute__((always_inline)) {
            constexpr int ks = decltype(ksc)::value, fs = (decltype(par)::value + ks) & 1;
            kstep(IntC<fs>{}, (unsigned)((ks + 1 < KS ? cur : nx) * STAGE_BYTES), ks + 1 < KS ? ks + 1 : 0, ksc, loads,
                  t + NSTAGE - 1, sb);
        });
        fill = cur;
        cur = nx;
        nx = nx + 1 == NSTAGE ? 0 : nx + 1;
    };
    // A barrier after which tile t + 1 is in LDS, `newer` later tiles' loads
    // being in flight, and no wave reads tile t - 1's buffer any more: its
    // last reads were consumed by MFMAs issued before the barrier.
#define RING_BARRIER(newer)                        \
    do {                                           \
        __builtin_amdgcn_sched_barrier(0);         \
        WAIT_VM((newer) * LPT);                    \
        asm volatile("s_barrier" ::: "memory");    \
        __builtin_amdgcn_sched_barrier(0);         \
    } while (0)
    seq<0, NSTAGE - 1>([&](auto u) __attribute__((always_inline)) {
        constexpr int t = decltype(u)::value;
        if (t < tiles) {
            if (t == tiles - 1) mask_tail();
            seq<0, LPT>([&](auto d) __attribute__((always_inline)) { issue_one(d, t, ring0 + (unsigned)(t * STAGE_BYTES)); });
        }
    });
    if (tiles >= NSTAGE - 1)
        RING_BARRIER(NSTAGE - 2);
    else
        RING_BARRIER(0);
#pragma unroll
    for (int i = 0; i < FM; ++i) fa[i] = *(const i32x4 *)(ring + (wm * WTM + i * MF) * TK + foff[0]);
#pragma unroll
    for (int j = 0; j < FN; ++j) fb[0][j] = *(const i32x4 *)(ring + HM * TK + (wn * WTN + j * MF) * TK + foff[0]);
    // Tiles with a later one to load, the last of them the one that loads the
    // last, perhaps partial tile.  An odd number of k-steps a tile swaps the
    // weight's sets: then two tiles an iteration, and what an odd tile left
    // over has read is moved to the first set.
    constexpr int SWAP = KS % 2;
    auto first_set = [&]() __attribute__((always_inline)) {
#pragma unroll
        for (int j = 0; j < FN; ++j) fb[0][j] = fb[1][j];
    };
    const int steady = tiles - (NSTAGE - 1);
    int t = 0;
#pragma nounroll
    for (; t + SWAP < steady; t += 1 + SWAP) {
        seq<0, 1 + SWAP>([&](auto p) __attribute__((always_inline)) {
            constexpr int u = decltype(p)::value;
            if (t + u == steady - 1) mask_tail();
            RING_BARRIER(NSTAGE - 3);
            tile(t + u, p, IntC<1>{});
        });
    }
    if (t < steady) {
        mask_tail();
        RING_BARRIER(NSTAGE - 3);
        tile(t, IntC<0>{}, IntC<1>{});
        if (SWAP) first_set();
        ++t;
    }
    // the last NSTAGE - 1 tiles, `left` after each: their waits are constants
    auto drain = [&](auto u, auto par) __attribute__((always_inline)) {
        constexpr int left = NSTAGE - 2 - decltype(u)::value;
        if constexpr (left > 0) RING_BARRIER(left - 1);
        tile(t, par, IntC<0>{});
        ++t;
    };
    seq<0, NSTAGE - 1>([&](auto u) __attribute__((always_inline)) {
        // (a swap needs at least NSTAGE - 1 tiles: every set is then known)
        if (SWAP || tiles > NSTAGE - 2 - decltype(u)::value) drain(u, IntC<SWAP ? decltype(u)::value & 1 : 0>{});
    });
#undef RING_BARRIER
#undef WAIT_VM
#elif STAGES == 3
    // Lane l holds 16 bytes of row l % 16 from k = 16 * (l / 16) of each
    // 64-deep MFMA step, so that a wave's load takes 64 bytes of 16 rows and
    // the TK / 64 loads of a batch take whole cache lines.  A batch is loaded
    // while the one before it is multiplied; enough waves on a CU keep the
    // memory busy.  Rows past M or N read the last row.
    static_assert(MF == 16 && WM == 1 && WN == 1, "one wave column");
    constexpr int NG = TK / 64;                         // MFMA steps of a batch
    unsigned ao[FM], bo[FN];
#pragma unroll
    for (int i = 0; i < FM; ++i) ao[i] = (unsigned)(min(i * 16 + lane % 16, mrows - 1) * ld + lane / 16 * 16);
#pragma unroll
    for (int j = 0; j < FN; ++j) bo[j] = (unsigned)(min(SRC_ROW(j * 16 + lane % 16), ncols - 1) * ld + lane / 16 * 16);
    struct Batch {
        i32x4 a[NG][FM], b[NG][FN];
    } f[2];
    auto fetch = [&](Batch &x, int k0) __attribute__((always_inline)) {
#pragma unroll
        for (int g = 0; g < NG; ++g) {
#pragma unroll
            for (int j = 0; j < FN; ++j) __builtin_memcpy(&x.b[g][j], (SRC_UP(j * 16) ? B1 : B0) + (k0 + g * 64) + bo[j], 16);
#pragma unroll
            for (int i = 0; i < FM; ++i) __builtin_memcpy(&x.a[g][i], Ab + (k0 + g * 64) + ao[i], 16);
        }
    };
    auto multiply = [&](const Batch &x) __attribute__((always_inline)) {
#pragma unroll
        for (int g = 0; g < NG; ++g)
#pragma unroll
            for (int i = 0; i < FM; ++i)
#pragma unroll
                for (int j = 0; j < FN; ++j) acc[i][j] = mfma(x.b[g][j], x.a[g][i], acc[i][j]);
    };
    const int whole = K / TK * TK;                      // whole batches
    int k0 = wave * TK;
    if (k0 < whole) fetch(f[0], k0);
    while (k0 < whole) {
        const int k1 = k0 + WK * TK, k2 = k1 + WK * TK;
        if (k1 < whole) fetch(f[1], k1);
        multiply(f[0]);
        if (k1 >= whole) break;
        if (k2 < whole) fetch(f[0], k2);
        multiply(f[1]);
        k0 = k2;
    }
    // what is left of K, a step a wave
    for (int k = whole + wave * 64; k < K; k += WK * 64) {
        const int left = K - k - lane / 16 * 16;
        i32x4 a[FM], b[FN];
#pragma unroll
        for (int i = 0; i < FM; ++i) a[i] = load16(Ab + k + ao[i], left);
#pragma unroll
        for (int j = 0; j < FN; ++j) b[j] = load16((SRC_UP(j * 16) ? B1 : B0) + k + bo[j], left);
#pragma unroll
        for (int i = 0; i < FM; ++i)
#pragma unroll
            for (int j = 0; j < FN; ++j) acc[i][j] = mfma(b[j], a[i], acc[i][j]);
    }
    // add the waves' sums: wave w finishes every WK-th of the output blocks
    i32x4(*const sums)[FM * FN][64] = (i32x4(*)[FM * FN][64])lds;
    if (WK > 1) {
#pragma unroll
        for (int i = 0; i < FM; ++i)
#pragma unroll
            for (int j = 0; j < FN; ++j) sums[wave][i * FN + j][lane] = acc[i][j];
        __syncthreads();
    }
    constexpr int FO = GATED ? FN / 2 : FN;
    for (int b = wave; b < FM * FO; b += WK) {
        const int i = b / FO, j = b % FO;
        i32x4 s = {0, 0, 0, 0}, u = {0, 0, 0, 0};
        if (WK > 1) {
#pragma unroll
            for (int w = 0; w < WK; ++w) {
                s += sums[w][i * FN + j][lane];
                if (GATED) u += sums[w][i * FN + FO + j][lane];
            }
        } else {
            // (one wave: its own sums, found without indexing registers)
#pragma unroll
            for (int x = 0; x < FM * FO; ++x)
                if (x == b) {
                    s = acc[x / FO][x % FO];
                    if (GATED) u = acc[x / FO][x % FO + FO % FN];
                }
        }
        const int ml = i * 16 + lane % 16, nl = j * 16 + 4 * (lane / 16);
        if (ml >= mrows || nl >= ncols) continue;
        const int sv[4] = {s[0], s[1], s[2], s[3]}, uv[4] = {u[0], u[1], u[2], u[3]};
        finish(args, m0 + ml, n0 + nl, sv, uv, (N & 3) == 0);
    }
    return;
#endif

    // ---- epilogue ---------------------------------------------------------
    // The weight fragment was the MFMA's first operand: a lane holds one
    // output row m and runs of 4 consecutive columns.
    const bool quads = (N & 3) == 0;
#if SPLITS > 1
    const int ldp = (N + 3) & ~3;                                  // of a partial row, per weight
#endif
#pragma unroll
    for (int i = 0; i < FM; ++i) {
        const int ml = wm * WTM + i * MF + lane % MF;
        if (ml >= mrows) continue;
#pragma unroll
        for (int j = 0; j < (GATED ? FN / 2 : FN); ++j) {
#pragma unroll
            for (int g = 0; g < ACCN / 4; ++g) {
                const int nl = wn * WTO + j * MF + g * 8 + 4 * (lane / MF);
                if (nl >= ncols) continue;
                int s[4], u[4];
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                    s[r] = acc[i][j][g * 4 + r];
                    u[r] = GATED ? acc[i][j + (GATED ? FN / 2 : 0)][g * 4 + r] : 0;
                }
#if SPLITS > 1
                // (columns past N up to the next four are stored too)
                int *p = args.P + (((size_t)kz * args.M + m0 + ml) * (GATED ? 2 : 1)) * ldp + n0 + nl;
                *(i32x4 *)p = i32x4{s[0], s[1], s[2], s[3]};
                if (GATED) *(i32x4 *)(p + ldp) = i32x4{u[0], u[1], u[2], u[3]};
#else
                finish(args, m0 + ml, n0 + nl, s, u, quads);
#endif
            }
        }
    }
}

extern "C" __global__ __launch_bounds__(NT) __attribute__((amdgpu_waves_per_eu(OCC, 8)))
void rc_gemm_i8(GemmI8Args args) {
    __shared__ __attribute__((aligned(1024))) i8 lds[LDS_BYTES];
    // ---- workgroup -> tile ----------------------------------------------
    const int ntn = (args.N + TNO - 1) / TNO;
    const int ntm = (int)((args.M + TM - 1) / TM);
    int bid = blockIdx.x;
    int blocks = (int)gridDim.x / SPLITS;                          // of one split
    const int kz = SPLITS > 1 ? bid / blocks : 0;
    bid -= kz * blocks;
#if TAIL
    // whole tiles first, then the halves of the others
    const int first = ntm * ntn - args.tail;
    const bool half = bid >= first;
    bid -= half ? first : 0;
    blocks = half ? 2 * args.tail : first;
#endif
#if ORDER == 1
    // Workgroups reach the 8 XCDs round-robin (workgroup b on XCD b % 8):
    // XCD x takes a contiguous range of the tiles, the first `rest` of them
    // one more.
    {
        const int per = blocks >> 3, rest = blocks & 7, x = bid & 7;
        bid = x * per + min(x, rest) + (bid >> 3);
    }
#endif
#if TAIL
    const int lower = half ? bid & 1 : 0;
    if (half) bid = first + (bid >> 1);
#endif
#if ORDER == 1
    // Within a band of 8 M tiles, m runs fastest: the 32 tiles an XCD's CUs
    // hold share 8 tiles of A and 4 of B.
    const int band = bid / (8 * ntn), rows = min(8, ntm - 8 * band), in = bid - band * 8 * ntn;
    const int mt = 8 * band + in % rows, nt = in / rows;
#else
    const int mt = bid / ntn, nt = bid % ntn;
#endif
    const long long m0 = (long long)mt * TM;
#if TAIL
    if (half) {
        if (m0 + lower * (TM / 2) < args.M) product<TM / 2>(args, lds, m0 + lower * (TM / 2), nt, kz);
        return;
    }
#endif
    product<TM>(args, lds, m0, nt, kz);
}

#if SPLITS > 1
// Adds the splits' int32 sums (exact in any order) and finishes the outputs,
// four columns a thread.
extern "C" __global__ __launch_bounds__(256) void rc_gemm_i8_join(GemmI8Args args) {
    const int N = args.N, quads = (N + 3) / 4, ldp = quads * 4;
    const size_t at = (size_t)blockIdx.x * 256 + threadIdx.x;
    if (at >= (size_t)args.M * quads) return;
    const long long m = (long long)(at / quads);
    const int n = (int)(at % quads) * 4;
    i32x4 s = {0, 0, 0, 0}, u = {0, 0, 0, 0};
#pragma unroll
    for (int z = 0; z < SPLITS; ++z) {
        const int *p = args.P + (((size_t)z * args.M + m) * (GATED ? 2 : 1)) * ldp + n;
        s += *(const i32x4 *)p;
        if (GATED) u += *(const i32x4 *)(p + ldp);
    }
    const int sv[4] = {s[0], s[1], s[2], s[3]}, uv[4] = {u[0], u[1], u[2], u[3]};
    finish(args, m, n, sv, uv, (N & 3) == 0);
}
#endif
