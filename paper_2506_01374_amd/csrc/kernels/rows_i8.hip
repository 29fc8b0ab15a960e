// Rows of bf16 to int8 with one fp32 scale a row, for gfx950: the plain
// quantisation, and the root-mean-square norm with the residual's addition
// in front of it.
//
// Compile-time schedule (generated prologue):
//   WAVES   waves that share a row (Parallel)
//   ROWS    rows of a workgroup (Parallel); 64 * WAVES * ROWS threads
//   VEC     elements of a global load, 1, 2, 4 or 8 (Vectorize).  A row need
//           not be whole vectors, nor start on a vector's alignment: the
//           last, partial vector is moved element by element
//   HELD    vectors a thread keeps in registers between the two passes over
//           its row (ComputeLocation), 64 * WAVES * VEC * HELD >= the row;
//           0: the second pass reads the row again
//   NORM    1: norm in front; RES  1: with the residual's addition
//
// With h the row (RES: h = bf16(x + r), which is stored), p = h w (NORM) or
// h, and a = max |p|:
//   NORM:  y = p / sqrt(mean h^2 + eps),   scale = max |y| / 127
//   else:  y = p,                          scale = a / 127
//   q = rint(y / scale) = rint(127 p / a), halves to the even integer.
// The norm's factor cancels from q, which so needs no sum: p is a product of
// two 8-bit significands, 127 p has at most 23 bits, and the remainder 127 p
// - q a of a trial q is exact in fp32, so q is the correctly rounded integer
// whatever the order in which the row was read (see quant).  The sum of
// squares and both statistics are fp32.
// A row of zeros has scale 0 and q 0.  A row that holds a NaN or an infinity,
// or (NORM) whose squares sum past fp32, has scale NaN and q 0: what is
// computed from it is NaN, not a silent zero.

typedef unsigned short bf16_t;
typedef unsigned int u32;

#define LANES (64 * WAVES)

struct RowsI8Args {
    const bf16_t *x;       // [rows][cols]
    const bf16_t *w;       // [cols] (NORM)
    const bf16_t *r;       // [rows][cols] (RES)
    signed char *q;        // [rows][cols]
    float *scale;          // [rows]
    bf16_t *h;             // [rows][cols] (RES); may be x or r
    long long rows;
    int cols;
    float eps;
};

__device__ __forceinline__ bf16_t f2bf(float x) { return __builtin_bit_cast(bf16_t, (__bf16)x); }
__device__ __forceinline__ float bf2f(u32 b) { return __builtin_bit_cast(float, b << 16); }

struct Vec {
    bf16_t e[VEC];
};

// Elements c .. c + VEC - 1 of a row of `cols`, zeros past its end.
__device__ __forceinline__ Vec load(const bf16_t *row, int c, int cols) {
    Vec v;
    if (c + VEC <= cols) {
        __builtin_memcpy(&v, row + c, sizeof v);
    } else {
#pragma unroll
        for (int j = 0; j < VEC; ++j) v.e[j] = c + j < cols ? row[c + j] : (bf16_t)0;
    }
    return v;
}

template <class T> __device__ __forceinline__ void store(T *row, const T (&v)[VEC], int c, int cols) {
    if (c + VEC <= cols) {
        __builtin_memcpy(row + c, v, sizeof v);
    } else {
#pragma unroll
        for (int j = 0; j < VEC; ++j)
            if (c + j < cols) row[c + j] = v[j];
    }
}

// rint(127 p / a) for |p| <= a, halves to even.  p and a are scaled by a
// power of two that brings a near 1, `inv` is near 1 / a.  The trial t is
// within one of the result, and 127 p - t a is exact: both terms are
// multiples of the smaller term's last bit, and their difference is below
// 2 a, so that it has no more bits than 127 p has (t = 0 leaves 127 p).
__device__ __forceinline__ int quant(float p, float a, float inv) {
    const float s = 127.f * p;
    const float t = __builtin_rintf(s * inv);
    const float rem = __builtin_fmaf(-t, a, s);
    const float twice = 2.f * __builtin_fabsf(rem);
    const int n = (int)t;
    // past half a step, or at the half and odd: the neighbour on that side
    const bool move = twice > a || (twice == a && (n & 1));
    return move ? n + (rem > 0.f ? 1 : -1) : n;
}

extern "C" __global__ __launch_bounds__(LANES * ROWS) void rc_rows_i8(RowsI8Args a) {
    const int tid = threadIdx.x;
    const int part = tid % LANES;                       // thread of its row
    const int slot = tid / LANES;                       // row of the workgroup
    const long long row_at = (long long)blockIdx.x * ROWS + slot;
    const bool live = row_at < a.rows;                  // (the last workgroup may have fewer rows)
    const long long base = (live ? row_at : 0) * a.cols;
    const int cols = live ? a.cols : 0;
    const bf16_t *x = a.x + base;
#if RES
    const bf16_t *r = a.r + base;
    bf16_t *ho = a.h + base;
#endif

    // one vector of the row: h in v (stored where RES), w in wv
    auto fetch = [&](int c, Vec &v, Vec &wv) {
        v = load(x, c, cols);
#if RES
        const Vec b = load(r, c, cols);
#pragma unroll
        for (int j = 0; j < VEC; ++j) v.e[j] = f2bf(bf2f(v.e[j]) + bf2f(b.e[j]));
        store(ho, v.e, c, cols);
#endif
#if NORM
        wv = load(a.w, c, cols);
#else
        (void)wv;
#endif
    };
    auto product = [&](const Vec &v, const Vec &wv, int j) {
#if NORM
        return bf2f(v.e[j]) * bf2f(wv.e[j]);
#else
        (void)wv;
        return bf2f(v.e[j]);
#endif
    };
    // |p| as bits: unsigned order is the order of the magnitudes, with NaN
    // above infinity, so the maximum keeps both
    u32 top = 0;
    float ss = 0.f;
    auto take = [&](const Vec &v, const Vec &wv) {
#pragma unroll
        for (int j = 0; j < VEC; ++j) {
            const u32 b = __builtin_bit_cast(u32, product(v, wv, j)) & 0x7FFFFFFFu;
            top = b > top ? b : top;
#if NORM
            const float h = bf2f(v.e[j]);
            ss = __builtin_fmaf(h, h, ss);
#endif
        }
    };

#if HELD
    Vec v[HELD], wv[HELD];
#pragma unroll
    for (int i = 0; i < HELD; ++i) fetch((i * LANES + part) * VEC, v[i], wv[i]);
#pragma unroll
    for (int i = 0; i < HELD; ++i) take(v[i], wv[i]);
#else
    for (int c = part * VEC; c < cols; c += LANES * VEC) {
        Vec v, wv;
        fetch(c, v, wv);
        take(v, wv);
    }
#endif

    // over the row's lanes and waves, in a fixed order
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
        const u32 o = (u32)__shfl_xor((int)top, d);
        top = o > top ? o : top;
#if NORM
        ss += __shfl_xor(ss, d);
#endif
    }
#if WAVES > 1
    __shared__ u32 tops[ROWS][WAVES];
    __shared__ float sums[ROWS][WAVES];
    if (part % 64 == 0) {
        tops[slot][part / 64] = top;
        sums[slot][part / 64] = ss;
    }
    __syncthreads();
    top = tops[slot][0];
    ss = sums[slot][0];
#pragma unroll
    for (int i = 1; i < WAVES; ++i) {
        const u32 o = tops[slot][i];
        top = o > top ? o : top;
        ss += sums[slot][i];
    }
#endif

    bool bad = top >= 0x7F800000u;
    float scale = __builtin_bit_cast(float, top);
#if NORM
    // (the host keeps eps at 2^-100 or more, next to which a square that
    // leaves fp32's normal range is nothing)
    bad |= !(ss < __builtin_inff());
    scale /= __builtin_sqrtf(ss / (float)a.cols + a.eps);
#endif
    scale /= 127.f;             // last, so that a small one is rounded once
    if (bad) scale = __builtin_nanf("");
    if (live && part == 0) a.scale[row_at] = scale;

    // a in [1, 2) times a power of two: p and a are brought there by its
    // inverse (exact), so that no product above leaves fp32's range
    const float am = __builtin_bit_cast(float, top);
    float up = 1.f;
    if (top < 0x20000000u) up = 18446744073709551616.f;             // a < 2^-63: 2^64
    if (top >= 0x5F800000u) up = 5.421010862427522e-20f;            // a >= 2^64: 2^-64
    const float as = am * up;
    const float inv = bad || top == 0u ? 0.f : __builtin_amdgcn_rcpf(as);
    auto emit = [&](const Vec &v, const Vec &wv, int c) {
        signed char o[VEC];
#pragma unroll
        for (int j = 0; j < VEC; ++j)
            o[j] = inv == 0.f ? (signed char)0 : (signed char)quant(product(v, wv, j) * up, as, inv);
        store(a.q + base, o, c, cols);
    };
#if HELD
#pragma unroll
    for (int i = 0; i < HELD; ++i) {
        const int c = (i * LANES + part) * VEC;
        if (c < cols) emit(v[i], wv[i], c);
    }
#else
    for (int c = part * VEC; c < cols; c += LANES * VEC) {
        Vec wv = {};
#if RES
        const Vec v = load(ho, c, cols);                 // its own store: x or r may be gone
#else
        const Vec v = load(x, c, cols);
#endif
#if NORM
        wv = load(a.w, c, cols);
#endif
        emit(v, wv, c);
    }
#endif
}
