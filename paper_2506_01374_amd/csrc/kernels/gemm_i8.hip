// int8 x int8 -> int32 MFMA matrix product for gfx950 with a fused epilogue:
//   acc[m][n] = sum_k A[m][k] B[n][k]              (int32, exact)
//   out[m][n] = acc * sa[m] * sb[n] (+ bias[n])    (fp32, then the output's type)
// (the sum is converted, multiplied by sa and then by sb, each rounded in fp32:
// sa * sb first would leave fp32's range where the output does not)
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
//   STAGES       1: LDS double buffer with register prefetch of the next two
//                K tiles, any sizes (ComputeLocation); 2: a ring of NSTAGE LDS
//                buffers filled by direct-to-LDS buffer loads issued
//                NSTAGE - 1 tiles ahead (K a multiple of 16: a lane moves 16
//                aligned bytes; rows of another length are copied first, by
//                rc_pad_i8); 3: streaming, for few rows of A -
//                operands go straight to registers in the MFMA's layout, the
//                WK waves of a tile take K in turns and add up through LDS
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
//
// What bounds it, and what each stage measured (bf16 output):
//   few rows: the weight's way from memory.  Streaming 4096 x 14336 for one
//   row takes 10.1 us (5.8 TB/s; the ring 12.8, one wave a tile 27.8); the
//   ring 4096 x 4096 for 16 rows 5.5 us (streaming 6.4) and, gated, 14336 x
//   4096 26.5 us (4.4 TB/s).
//   many rows: the matrix cores, next to the tiles' way from L2 to LDS.  A CU
//   takes about 50 bytes a clock from L2, so that 64 of K of a 256 x 128 tile
//   (24 KB) need 490 clocks next to 512 of MFMAs, of a 256 x 256 tile 655 next
//   to 1024.  8192 x 8192 x 8192 in 256 x 256 tiles: 450 us, 2.44 POP/s; 2048 x
//   4096 x 14336 in 256 x 128 tiles, one round of workgroups: 124 us, 1.93.  A
//   256 x 256 tile costs some 10 us around its K loop: 3 to the first MFMA, 4
//   of stores, the rest between workgroups.
//   The double buffer is behind the ring (1024 x 4096 x 4096: 23.4 and 21.4
//   us); it is there for rows that are no whole 16-byte chunks.  With loads two
//   tiles ahead these take 31.5 us for K of 4099, with one 42.3, and 27.3 for K
//   of 4100, whose rows start on 4 bytes.
//   The 32 x 32 MFMA is about 5 % slower than the 16 x 16 one in the same tile.

#define NT (64 * WM * WN * WK)
#define WTN (TN / WN)
#define FN (WTN / MF)
#define CPR (TK / 16)                                       // 16-byte chunks of a tile row
#define RPL ((16 / CPR) > 0 ? (16 / CPR) : 1)
#define TNO (GATED ? TN / 2 : TN)                           // output columns of a tile
#define WTO (GATED ? WTN / 2 : WTN)                         // of a wave
// neighbouring output columns of a lane
#if STAGES != 3 && (TN / WN) / (GATED + 1) % 32 == 0
#define RUN 8
#else
#define RUN 4
#endif

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

// The row's last 16 elements v, moved down so that the last `left` of them
// (none to 16) are the first, with zeros behind them.
__device__ __forceinline__ void shift16(i32x4 &v, int left) {
    const unsigned by = (unsigned)(16 - min(max(left, 0), 16));
    i32x4 w = v;
    if (by & 8) w = i32x4{w[2], w[3], 0, 0};
    if (by & 4) w = i32x4{w[1], w[2], w[3], 0};
#pragma unroll
    for (int j = 0; j < 4; ++j)
        v[j] = by == 16 ? 0 : (int)__builtin_amdgcn_alignbyte(j < 3 ? (unsigned)w[j + 1] : 0u, (unsigned)w[j], by & 3);
}

// The first `left` elements at p, fewer than 16, and zeros.
__device__ __forceinline__ i32x4 bytes16(const i8 *p, int left) {
    unsigned long long w[2] = {0, 0};
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll 1
        for (int j = 0; j < 8 && 8 * h + j < left; ++j) w[h] |= (unsigned long long)(unsigned char)p[8 * h + j] << (8 * j);
    return i32x4{(int)w[0], (int)(w[0] >> 32), (int)w[1], (int)(w[1] >> 32)};
}

__device__ __forceinline__ float silu(float x) {
    // x * sigmoid(x); exp(-x) as 2^(-x log2 e) and the reciprocal on the
    // hardware's units, one step of fp32 off each, which a rounding to bf16
    // follows.  The reciprocal's results end at 2^-126: below x = -87.3, where
    // the value is under 10^-36, this is 0.
    return x * __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(-x * 1.4426950408889634f));
}

// R neighbouring columns' scales (and bias).
template <int R> struct Cols {
    float s[R];
#if GATED
    float u[R];
#endif
#if BIAS
    float b[R];
#endif
    // of column n on; `in`: all R exist (columns past the last repeat it)
    __device__ __forceinline__ void load(const GemmI8Args &a, int n, bool in) {
        if (in) {
            __builtin_memcpy(s, a.sb0 + n, sizeof s);
#if GATED
            __builtin_memcpy(u, a.sb1 + n, sizeof u);
#endif
#if BIAS
            __builtin_memcpy(b, a.bias + n, sizeof b);
#endif
        } else {
#pragma unroll
            for (int r = 0; r < R; ++r) {
                const int c = min(n + r, a.N - 1);
                s[r] = a.sb0[c];
#if GATED
                u[r] = a.sb1[c];
#endif
#if BIAS
                b[r] = a.bias[c];
#endif
            }
        }
    }
};

// Columns n .. n + R - 1 of row m from their sums (GATED: g, and u the second
// weight's).  Stores are of up to 16 bytes at any alignment.
template <int R>
__device__ __forceinline__ void finish(const GemmI8Args &a, long long m, int n, const int (&g)[R], const int (&u)[R], float sa,
                                       const Cols<R> &c, bool in) {
#if F32
    float v[R];
#else
    bf16_t v[R];
#endif
#pragma unroll
    for (int r = 0; r < R; ++r) {
        float y = (float)g[r] * sa * c.s[r];
#if GATED
        y = silu(y) * ((float)u[r] * sa * c.u[r]);
#endif
#if BIAS
        y += c.b[r];
#endif
#if F32
        v[r] = y;
#else
        v[r] = __builtin_bit_cast(bf16_t, (__bf16)y);
#endif
    }
#if F32
    float *out = (float *)a.C + (size_t)m * a.N + n;
#else
    bf16_t *out = (bf16_t *)a.C + (size_t)m * a.N + n;
#endif
    if (in) {
        __builtin_memcpy(out, v, sizeof v);
    } else {
#pragma unroll
        for (int r = 0; r < R; ++r)
            if (n + r < a.N) out[r] = v[r];
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
#define SRC_ROW(b) ((b) / WTN * WTO + SRC_IN((b) % WTO))
#define SRC_UP(b) ((b) % WTN >= WTO)
#else
    const i8 *const B1 = B0;
#define SRC_ROW(b) SRC_IN(b)
#define SRC_UP(b) false
#endif
    // Which output column a weight row of the tile is: a lane's sums of an
    // MFMA are runs of 4 columns; taking the rows in this order puts two such
    // runs side by side, so that a lane stores 16 bytes of bf16.
#if RUN == 8 && MF == 16
#define SRC_IN(b) ((b) / 32 * 32 + (b) / 4 % 4 * 8 + (b) / 16 % 2 * 4 + (b) % 4)
#elif RUN == 8
#define SRC_IN(b) ((b) / 16 * 16 + (b) / 4 % 2 * 8 + (b) / 8 % 2 * 4 + (b) % 4)
#else
#define SRC_IN(b) (b)
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
        // (threads past the tile's last chunk move it again)
        const int v = min(tid + i * NT, (HM + TN) * CPR - 1);
        const int row = v / CPR, c = v % CPR;
        kc[i] = c * 16;
        if (row < HM) {
            dst[i] = swz(row, c);
            src[i] = Ab + (size_t)min(row, mrows - 1) * ld;
        } else {
            const int b = row - HM;
            dst[i] = HM * TK + swz(b, c);
            src[i] = (SRC_UP(b) ? B1 : B0) + (size_t)min(SRC_ROW(b), ncols - 1) * ld;
        }
    }
    // Two tiles ahead of the one that is multiplied: of tile t + 1, whose
    // loads had an iteration's time, and of tile t + 2.
    i32x4 reg[2][CH];
    const int tiles = (K + TK - 1) / TK;
    auto plain = [&](i32x4 (&r)[CH], int t) __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < CH; ++i) __builtin_memcpy(&r[i], src[i] + (kc[i] + t * TK), 16);
    };
    // the last tile's too: the row's last 16 elements for a chunk that is not
    // whole or past the row (a branch around loads would make what follows wait
    // for all of them)
    auto fetch = [&](i32x4 (&r)[CH], int t) __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < CH; ++i) __builtin_memcpy(&r[i], src[i] + min(kc[i] + t * TK, K - 16), 16);
    };
    auto put = [&](const i32x4 (&r)[CH], int b) __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < CH; ++i) *(i32x4 *)(lds + b * BUF + dst[i]) = r[i];
    };
    auto multiply = [&](int b) __attribute__((always_inline)) {
        const i8 *la = lds + b * BUF + wm * WTM * TK, *lb = lds + b * BUF + (HM + wn * WTN) * TK;
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
    };
    auto ends = [&](i32x4 (&r)[CH], int t) __attribute__((always_inline)) {
        if (t * TK + TK > K)
#pragma unroll
            for (int i = 0; i < CH; ++i) shift16(r[i], K - t * TK - kc[i]);
    };
    if (ld < 16) {                                      // (rows shorter than a load: one tile)
#pragma unroll
        for (int i = 0; i < CH; ++i) reg[0][i] = bytes16(src[i] + kc[i], K - kc[i]);
    } else {
        fetch(reg[0], 0);
        if (tiles > 1) fetch(reg[1], 1);
        ends(reg[0], 0);
    }
    put(reg[0], 0);
    __syncthreads();
    // Tile t is in buffer 0 and t + 1 in reg[1].  Buffer (t + 1) & 1 was last
    // read in iteration t - 1, which ended with a barrier.
    int t = 0;
    for (; t + 3 < tiles; t += 2) {
        plain(reg[0], t + 2);
        multiply(0);
        put(reg[1], 1);
        __syncthreads();
        fetch(reg[1], t + 3);
        multiply(1);
        put(reg[0], 0);
        __syncthreads();
    }
    // one to three tiles are left
    if (t + 3 == tiles) {
        fetch(reg[0], t + 2);
        multiply(0);
        put(reg[1], 1);
        __syncthreads();
        multiply(1);
        ends(reg[0], t + 2);
        put(reg[0], 0);
        __syncthreads();
        multiply(0);
    } else {
        multiply(0);
        if (t + 2 == tiles) {
            ends(reg[1], t + 1);
            put(reg[1], 1);
            __syncthreads();
            multiply(1);
        }
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
    // the block of 16 x 16 outputs that this wave finishes first: its scales
    // are loaded ahead of K, not after it
    constexpr int FO = GATED ? FN / 2 : FN;
    int b_m, b_n;
    float b_sa = 0.f;
    Cols<4> b_cols = {};
    auto block = [&](int b) {
        b_m = b / FO * 16 + lane % 16;
        b_n = b % FO * 16 + 4 * (lane / 16);
        if (b_m < mrows && b_n < ncols) {
            b_sa = args.sa[m0 + b_m];
            b_cols.load(args, n0 + b_n, n0 + b_n + 4 <= N);
        }
    };
    if (wave < FM * FO) block(wave);
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
    // what is left of K, a step a wave: loads of the row's last 16 elements
    // where fewer are left, all under way before one is moved down
    for (int k = whole + wave * 64; k < K; k += WK * 64) {
        const int left = K - k - lane / 16 * 16, back = min(left - 16, 0);
        i32x4 a[FM], b[FN];
        if (ld >= 16) {
#pragma unroll
            for (int i = 0; i < FM; ++i) __builtin_memcpy(&a[i], Ab + (k + back) + (size_t)ao[i], 16);
#pragma unroll
            for (int j = 0; j < FN; ++j) __builtin_memcpy(&b[j], (SRC_UP(j * 16) ? B1 : B0) + (k + back) + (size_t)bo[j], 16);
#pragma unroll
            for (int i = 0; i < FM; ++i) shift16(a[i], left);
#pragma unroll
            for (int j = 0; j < FN; ++j) shift16(b[j], left);
        } else {
            // (a row shorter than a load)
#pragma unroll
            for (int i = 0; i < FM; ++i) a[i] = bytes16(Ab + k + ao[i], left);
#pragma unroll
            for (int j = 0; j < FN; ++j) b[j] = bytes16((SRC_UP(j * 16) ? B1 : B0) + k + bo[j], left);
        }
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
        if (b != wave) block(b);
        if (b_m >= mrows || b_n >= ncols) continue;
        const int sv[4] = {s[0], s[1], s[2], s[3]}, uv[4] = {u[0], u[1], u[2], u[3]};
        finish<4>(args, m0 + b_m, n0 + b_n, sv, uv, b_sa, b_cols, n0 + b_n + 4 <= N);
    }
    return;
#endif

    // ---- epilogue ---------------------------------------------------------
    // The weight fragment was the MFMA's first operand: a lane holds one
    // output row m and runs of RUN neighbouring columns, run q of a fragment
    // row at column run_at(q) of the tile.
    // (The lane is counted anew: kept from the start, it would hold a register
    // through the main loop, where 256 x 256 tiles of 8 waves have none left.)
    int el;
    asm volatile("v_mbcnt_lo_u32_b32 %0, -1, 0\n\tv_mbcnt_hi_u32_b32 %0, -1, %0" : "=v"(el));
    constexpr int RUNS = WTO / RUN / (64 / MF);
    auto run_at = [&](int q) { return wn * WTO + q * RUN * (64 / MF) + RUN * (el / MF); };
    auto sums_of = [&](auto ic, auto qc, int (&s)[RUN], int (&u)[RUN]) __attribute__((always_inline)) {
        constexpr int i = decltype(ic)::value, q = decltype(qc)::value, F = MF == 16 ? RUN / 4 : 1, G = MF == 16 ? 0 : q % 2;
        constexpr int j = MF == 16 ? q * F : q / 2;
#pragma unroll
        for (int r = 0; r < RUN; ++r) {
            s[r] = acc[i][j + (MF == 16 ? r / 4 : 0)][MF == 16 ? r % 4 : G * 8 + r];
            u[r] = GATED ? acc[i][j + (MF == 16 ? r / 4 : 0) + FN / 2][MF == 16 ? r % 4 : G * 8 + r] : 0;
        }
    };
#if SPLITS > 1
    const int ldp = (N + 3) & ~3;                                  // of a partial row, per weight
    // (one pointer, moved row by row: the scheduler would form all addresses
    // at once, next to all sums, and spill)
    int *row = args.P + (((size_t)kz * args.M + m0 + wm * WTM + el % MF) * (GATED ? 2 : 1)) * ldp + n0;
    seq<0, FM>([&](auto ic) __attribute__((always_inline)) {
        const int ml = wm * WTM + decltype(ic)::value * MF + el % MF;
        if constexpr (decltype(ic)::value > 0) row += (size_t)MF * (GATED ? 2 : 1) * ldp;
        asm volatile("" : "+v"(row));
        __builtin_amdgcn_sched_barrier(0);
        seq<0, RUNS>([&](auto qc) __attribute__((always_inline)) {
            int s[RUN], u[RUN];
            sums_of(ic, qc, s, u);
            const int nl = run_at(decltype(qc)::value);
#pragma unroll
            for (int r = 0; r < RUN; r += 4) {
                // (columns past N up to the next four are stored too)
                if (ml < mrows && nl + r < ncols) {
                    *(i32x4 *)(row + nl + r) = i32x4{s[r], s[r + 1], s[r + 2], s[r + 3]};
                    if (GATED) *(i32x4 *)(row + ldp + nl + r) = i32x4{u[r], u[r + 1], u[r + 2], u[r + 3]};
                }
            }
        });
    });
#else
    // All scales at once (a load behind every store's branch would cost its
    // whole latency each): columns of a whole tile without a test.
    auto store = [&](auto whole) __attribute__((always_inline)) {
        constexpr bool W = decltype(whole)::value;
        Cols<RUN> cols[RUNS];
        float sa[FM];
#pragma unroll
        for (int q = 0; q < RUNS; ++q) cols[q].load(args, n0 + run_at(q), W || n0 + run_at(q) + RUN <= N);
#pragma unroll
        for (int i = 0; i < FM; ++i) sa[i] = args.sa[m0 + min(wm * WTM + i * MF + el % MF, mrows - 1)];
        seq<0, FM>([&](auto ic) __attribute__((always_inline)) {
            constexpr int i = decltype(ic)::value;
            const int ml = wm * WTM + i * MF + el % MF;
            seq<0, RUNS>([&](auto qc) __attribute__((always_inline)) {
                constexpr int q = decltype(qc)::value;
                int s[RUN], u[RUN];
                sums_of(ic, qc, s, u);
                const int nl = run_at(q);
                if (ml < mrows && (W || nl < ncols))
                    finish<RUN>(args, m0 + ml, n0 + nl, s, u, sa[i], cols[q], W || n0 + nl + RUN <= N);
            });
        });
    };
    if (ncols == TNO)
        store(IntC<1>{});
    else
        store(IntC<0>{});
#endif
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
// four columns a thread.  Bound by memory: 67 MB of sums in and 17 MB out take
// 14.4 us, 5.8 TB/s.
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
    Cols<4> cols;
    cols.load(args, n, n + 4 <= N);
    finish<4>(args, m, n, sv, uv, args.sa[m], cols, n + 4 <= N);
}
#endif
