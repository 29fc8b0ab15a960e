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
//   WM WN        waves along M and N (Parallel); NT = 64 * WM * WN threads
//   MF           MFMA shape: 16 -> v_mfma_i32_16x16x64_i8,
//                            32 -> v_mfma_i32_32x32x32_i8
//   STAGES       1: LDS double buffer with register prefetch of the next K
//                tile, any sizes (ComputeLocation)
//   ORDER        0: tile n fastest; 1: bands of 8 M tiles, m fastest within
//                a band, each XCD owning a contiguous range
//   OCC          waves per SIMD the register allocation must leave room for
//   BIAS F32 GATED   operator flags: bias added, fp32 output, gated form
//
// Edges: rows past M or N read the last row and are not stored; a K tail
// reads zeros.

#define NT (64 * WM * WN)
#define WTM (TM / WM)
#define WTN (TN / WN)
#define FM (WTM / MF)
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
    long long M;
    int N, K;
};

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

extern "C" __global__ __launch_bounds__(NT) __attribute__((amdgpu_waves_per_eu(OCC, 8)))
void rc_gemm_i8(GemmI8Args args) {
    const int tid = threadIdx.x;
    const int lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);     // wave-uniform: scalar registers
    __builtin_assume(wave >= 0 && wave < WM * WN);
    const int wm = wave / WN, wn = wave % WN;
    const int K = args.K, N = args.N;

    // ---- workgroup -> tile ----------------------------------------------
    const int ntn = (N + TNO - 1) / TNO;
    const int ntm = (int)((args.M + TM - 1) / TM);
    int bid = blockIdx.x;
    int mt, nt;
#if ORDER == 1
    // Workgroups reach the 8 XCDs round-robin (workgroup b on XCD b % 8):
    // XCD x takes a contiguous range of the tiles, the first `rest` of them
    // one more.  Within a band of 8 M tiles, m runs fastest: the 32 tiles an
    // XCD's CUs hold share 8 tiles of A and 4 of B.
    {
        const int per = (int)gridDim.x >> 3, rest = (int)gridDim.x & 7, x = bid & 7;
        bid = x * per + min(x, rest) + (bid >> 3);
        const int band = bid / (8 * ntn), rows = min(8, ntm - 8 * band), in = bid - band * 8 * ntn;
        mt = 8 * band + in % rows;
        nt = in / rows;
    }
#else
    mt = bid / ntn;
    nt = bid % ntn;
#endif
    const long long m0 = (long long)mt * TM;
    const int n0 = nt * TNO;                                       // first output column
    const int mrows = (int)min((long long)TM, args.M - m0);
    const int ncols = min(TNO, N - n0);
    const i8 *const Ab = args.A + (size_t)m0 * K;
    const i8 *const B0 = args.B0 + (size_t)n0 * K;
#if GATED
    const i8 *const B1 = args.B1 + (size_t)n0 * K;
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
    __shared__ __attribute__((aligned(16))) i8 lds[2][(TM + TN) * TK];
    // chunk v of a tile: row v / CPR, chunk v % CPR of it
    constexpr int CH = ((TM + TN) * CPR + NT - 1) / NT;            // per thread
    const i8 *src[CH];
    int kc[CH], dst[CH];
#pragma unroll
    for (int i = 0; i < CH; ++i) {
        const int v = tid + i * NT;
        const int row = v / CPR, c = v % CPR;
        kc[i] = c * 16;
        if (row < TM) {
            dst[i] = swz(row, c);
            src[i] = Ab + (size_t)min(row, mrows - 1) * K + kc[i];
        } else {
            const int b = row - TM;
            dst[i] = v < (TM + TN) * CPR ? TM * TK + swz(b, c) : -1;
            src[i] = (SRC_UP(b) ? B1 : B0) + (size_t)min(SRC_ROW(b), ncols - 1) * K + kc[i];
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
            if (dst[i] >= 0) *(i32x4 *)(lds[b] + dst[i]) = reg[i];
    };
    const int tiles = (K + TK - 1) / TK;
    fetch(0);
    put(0);
    __syncthreads();
    for (int t = 0; t < tiles; ++t) {
        // buffer (t + 1) & 1 was last read in iteration t - 1, which ended
        // with a barrier
        if (t + 1 < tiles) fetch((t + 1) * TK);
        const i8 *la = lds[t & 1] + wm * WTM * TK, *lb = lds[t & 1] + (TM + wn * WTN) * TK;
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
#endif

    // ---- epilogue ---------------------------------------------------------
    // The weight fragment was the MFMA's first operand: a lane holds one
    // output row m and runs of 4 consecutive columns.
    const bool quads = (N & 3) == 0;
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
                finish(args, m0 + ml, n0 + nl, s, u, quads);
            }
        }
    }
}
