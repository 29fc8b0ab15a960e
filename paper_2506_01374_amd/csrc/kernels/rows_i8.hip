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
// whatever the order in which the row was read (see nearest).  A product's
// exponent can leave fp32: a row whose a is not between 2^-63 and 2^64 takes
// its products, a and the remainders in 64 bits (see WIDE).  The sum of
// squares is fp32, of one vector's at a time, and where a thread has many
// vectors their sums carry what the additions drop: its error does not grow
// with the row.
// A row of zeros has scale 0 and q 0.  A row that holds a NaN or an infinity,
// or (NORM) whose squares sum or whose scale is past fp32, has scale NaN and q
// 0: what is computed from it is NaN, not a silent zero.
//
// Bound by memory with many rows: 2048 x 14336 plain, 88 MB, 16.7 us (5.3
// TB/s); the norm with the residual, 2048 x 4096, 59 MB, 12.6 us (4.7 TB/s),
// 8192 x 4096 43.4 us (5.4).  A row stays in registers between the passes:
// reading it again takes 18.8 us in the first of these.  Rows in 64 bits are
// read twice more: 2048 x 4096 of them, with the residual, take 21.3 us for 12.6.
// Bound by the way to memory and back with few rows: one row of 4096 takes 3.0
// us, of which an empty kernel takes 2.2, so that its waves are many and their
// loads all under way at once.

typedef unsigned short bf16_t;
typedef unsigned int u32;
typedef unsigned short u16x2 __attribute__((ext_vector_type(2)));

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

// VEC elements, two a word.
#define WORDS ((VEC + 1) / 2)
struct Vec {
    u32 w[WORDS];
    __device__ __forceinline__ float at(int j) const {
        return __builtin_bit_cast(float, j % 2 ? w[j / 2] & 0xFFFF0000u : w[j / 2] << 16);
    }
};

// Elements c .. c + VEC - 1 of a row of `cols`, zeros past its end.  In two
// steps, so that a thread's loads are all under way before it waits for one:
// `fetch` loads whole vectors without a branch (a lane whose vector is not
// whole loads the row's last one), `ends` puts right the lanes at the end.
__device__ __forceinline__ Vec fetch(const bf16_t *row, int c, int cols) {
    Vec v = {};
    if (cols >= VEC) __builtin_memcpy(&v, row + (c < cols - VEC ? c : cols - VEC), 2 * VEC);
    return v;
}

__device__ __forceinline__ void ends(Vec &v, const bf16_t *row, int c, int cols) {
    if (c + VEC <= cols) return;
#pragma unroll
    for (int i = 0; i < WORDS; ++i) v.w[i] = 0;
    if (c >= cols) return;
#pragma unroll
    for (int j = 0; j < VEC; ++j)
        if (c + j < cols) v.w[j / 2] |= (u32)row[c + j] << (16 * (j % 2));
}

// VEC elements of type T, packed in v, to a row of `cols` at c
template <class T, int W> __device__ __forceinline__ void store(T *row, const u32 (&v)[W], int c, int cols) {
    constexpr int PER = 4 / sizeof(T);                  // of a word
    if (c + VEC <= cols) {
        __builtin_memcpy(row + c, v, VEC * sizeof(T));
    } else {
#pragma unroll
        for (int j = 0; j < VEC; ++j)
            if (c + j < cols) row[c + j] = (T)(v[j / PER] >> (32 / PER * (j % PER)));
    }
}

// the low bytes of t, four a word
__device__ __forceinline__ void pack(u32 (&q)[(VEC + 3) / 4], const u32 (&t)[VEC]) {
#pragma unroll
    for (int i = 0; i < (VEC + 3) / 4; ++i) {
        const int j = 4 * i;
        q[i] = VEC > 1 ? __builtin_amdgcn_perm(t[j + (VEC > 1)], t[j], 0x0C0C0400u) : t[j];
        if (VEC > 3) q[i] = __builtin_amdgcn_perm(__builtin_amdgcn_perm(t[j + 3 * (VEC > 3)], t[j + 2 * (VEC > 3)], 0x0C0C0400u), q[i], 0x05040100u);
    }
}

// An integer t near s / a, |s| <= 127 a, as SHIFT + t: the last bit of a
// float there is 1, so that the addition rounds to an integer, which the low
// bits then are.
#define SHIFT 12582912.f        // 1.5 * 2^23
__device__ __forceinline__ float trial(float s, float inv) { return __builtin_fmaf(s, inv, SHIFT); }

// rint(s / a), halves to even, s = 127 p and |p| <= a.  The trial t is within
// one of the result, and s - t a is exact: both terms are multiples of the
// smaller term's last bit, and their difference is below 2 a, so that it has
// no more bits than s has (t = 0 leaves s).  Where it is below a / 2, or that
// with an even t, t is the result.
__device__ __forceinline__ int nearest(float s, float a, float inv) {
    const float t = trial(s, inv);
    const float rem = __builtin_fmaf(-(t - SHIFT), a, s);
    const float r = __builtin_fabsf(rem);
    const int n = __builtin_bit_cast(int, t);
    // past half a step, or at the half and odd: the neighbour on that side
    const bool move = r > 0.5f * a || (r == 0.5f * a && (n & 1));
    return move ? n + (rem > 0.f ? 1 : -1) : n;
}

extern "C" __global__ __launch_bounds__(LANES * ROWS) void rc_rows_i8(RowsI8Args a) {
    const int tid = threadIdx.x;
    const int part = tid % LANES;                       // thread of its row
    const int slot = ROWS > 1 ? __builtin_amdgcn_readfirstlane(tid / LANES) : 0;     // row of the workgroup
    const long long row_at = (long long)blockIdx.x * ROWS + slot;
    const bool live = row_at < a.rows;                  // (the last workgroup may have fewer rows)
    const long long base = (live ? row_at : 0) * a.cols;
    const int cols = live ? a.cols : 0;
    const bf16_t *x = a.x + base;
#if RES
    const bf16_t *r = a.r + base;
    bf16_t *ho = a.h + base;
#endif

    // a thread's vectors of the row: h in v (stored where RES), w in wv
    auto read = [&](int c, auto &v, auto &wv, int n) {
#pragma unroll
        for (int i = 0; i < n; ++i) v[i] = fetch(x, c + i * LANES * VEC, cols);
#if RES
        Vec b[HELD ? HELD : 1];
#pragma unroll
        for (int i = 0; i < n; ++i) b[i] = fetch(r, c + i * LANES * VEC, cols);
#endif
#if NORM
#pragma unroll
        for (int i = 0; i < n; ++i) wv[i] = fetch(a.w, c + i * LANES * VEC, cols);
#endif
#pragma unroll
        for (int i = 0; i < n; ++i) {
            const int ci = c + i * LANES * VEC;
            ends(v[i], x, ci, cols);
#if RES
            ends(b[i], r, ci, cols);
            Vec h = {};
#pragma unroll
            for (int j = 0; j < VEC; ++j) h.w[j / 2] |= (u32)f2bf(v[i].at(j) + b[i].at(j)) << (16 * (j % 2));
            store(ho, h.w, ci, cols);
            v[i] = h;
#endif
#if NORM
            ends(wv[i], a.w, ci, cols);
#endif
        }
    };
    auto product = [&](const Vec &v, const Vec &wv, int j) {
#if NORM
        return v.at(j) * wv.at(j);
#else
        (void)wv;
        return v.at(j);
#endif
    };
    // the maximum keeps a NaN: of magnitudes as bits, above all others (the
    // plain kind, two a word), or by the instruction
    float top = 0.f;
    u16x2 tops2 = {0, 0};
    float ss = 0.f;
#if NORM
    u32 bits = 0;               // of h whose squares did not reach fp32, without their signs
    auto gather = [&](const Vec &v) __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < WORDS; ++i)             // (in C it is formed ahead of the branch around it)
            asm("v_and_or_b32 %0, %1, %2, %0" : "+v"(bits) : "v"(v.w[i]), "s"(0x7FFF7FFFu));
    };
#if !HELD
    float lost = 0.f;           // what the additions to ss have dropped
#endif
#endif
    auto take = [&](const Vec &v, const Vec &wv) {
#if NORM
        float s = 0.f;
#pragma unroll
        for (int j = 0; j < VEC; ++j) {
            top = __builtin_elementwise_maximum(top, __builtin_fabsf(product(v, wv, j)));
            const float h = v.at(j);
            s = __builtin_fmaf(h, h, s);
        }
#if HELD
        if (s == 0.f) gather(v);
        ss += s;
#else
        // (a row of 2^24 equal values: 1e-3 off without, in one wave)
        s -= lost;
        const float sum = ss + s;
        lost = (sum - ss) - s;
        ss = sum;
#endif
#else
#pragma unroll
        for (int i = 0; i < WORDS; ++i)
            tops2 = __builtin_elementwise_max(tops2, __builtin_bit_cast(u16x2, v.w[i] & 0x7FFF7FFFu));
#endif
    };

#if HELD
    Vec v[HELD], wv[HELD];
    read(part * VEC, v, wv, HELD);
#pragma unroll
    for (int i = 0; i < HELD; ++i) take(v[i], wv[i]);
#else
    for (int c = part * VEC; c < cols; c += LANES * VEC) {
        Vec v[1], wv[1];
        read(c, v, wv, 1);
        take(v[0], wv[0]);
    }
#endif

    const auto put = [&](u32 (&q)[(VEC + 3) / 4], u32 keep, int c) __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < (VEC + 3) / 4; ++i) q[i] &= keep;
        store(a.q + base, q, c, cols);
    };
    // f(h, w, c) of each of the thread's vectors, read again
    const auto again = [&](auto &&f) __attribute__((always_inline)) {
        for (int c = part * VEC; c < cols; c += LANES * VEC) {
            // RES: its own store, as x or r may be gone
#if RES
            const bf16_t *src = ho;
#else
            const bf16_t *src = x;
#endif
            Vec h = fetch(src, c, cols), wv = {};
            ends(h, src, c, cols);
#if NORM
            wv = fetch(a.w, c, cols);
            ends(wv, a.w, c, cols);
#endif
            f(h, wv, c);
        }
    };

#if NORM
    // squares of which none reached fp32: its least value instead of 0 (next to
    // eps nothing), so that a row's 0 is the sum of zeros alone
#if !HELD
    if (ss == 0.f) again([&](const Vec &v, const Vec &, int) __attribute__((always_inline)) { gather(v); });
#endif
    if (ss == 0.f && bits) ss = 0x1p-149f;
#endif
#if !NORM
    top = __builtin_bit_cast(float, (u32)(tops2[0] > tops2[1] ? tops2[0] : tops2[1]) << 16);
#endif

    // over the row's lanes and waves, in a fixed order
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
        top = __builtin_elementwise_maximum(top, __shfl_xor(top, d));
#if NORM
        ss += __shfl_xor(ss, d);
#endif
    }
#if WAVES > 1
    __shared__ float tops[ROWS][WAVES], sums[ROWS][WAVES];
    if (part % 64 == 0) {
        tops[slot][part / 64] = top;
        sums[slot][part / 64] = ss;
    }
    __syncthreads();
    top = tops[slot][0];
    ss = sums[slot][0];
#pragma unroll
    for (int i = 1; i < WAVES; ++i) {
        top = __builtin_elementwise_maximum(top, tops[slot][i]);
        ss += sums[slot][i];
    }
#endif

#if NORM
    // The row in 64 bits, which hold every product of two bf16: where fp32 may
    // have lost the end of a product that counts (a below 2^-126 does), or
    // 1 / a and y could leave it; rows with a NaN or an infinity come here too.
    // Not rows of zeros, which padding makes many.
#define WIDE(top, ss) (!((top) >= 0x1p-63f && (top) < 0x1p64f) && !((top) == 0.f && (ss) == 0.f))
    const bool wide = live && WIDE(top, ss);
    bool any = wide;                                    // of the rows that share the barrier below
#if ROWS > 1 && WAVES > 1
    for (int s = 0; s < ROWS; ++s) {
        float t = tops[s][0], sum = sums[s][0];
        for (int i = 1; i < WAVES; ++i) {
            t = __builtin_elementwise_maximum(t, tops[s][i]);
            sum += sums[s][i];
        }
        any |= (long long)blockIdx.x * ROWS + s < a.rows && WIDE(t, sum);
    }
#endif
    if (any) {
        double most = 0;
        // (with held vectors instead of a second reading 8192 x 4096 would take
        // 73 registers, not 48, and leave room for fewer waves)
        again([&](const Vec &v, const Vec &wv, int) __attribute__((always_inline)) {
#pragma unroll
            for (int j = 0; j < VEC; ++j) {
                const double p = __builtin_fabs((double)v.at(j) * (double)wv.at(j));
                most = __builtin_fmax(most, p < __builtin_inf() ? p : __builtin_inf());
            }
        });
#pragma unroll
        for (int d = 1; d < 64; d <<= 1) most = __builtin_fmax(most, __shfl_xor(most, d));
#if WAVES > 1
        __shared__ double mosts[ROWS][WAVES];
        if (part % 64 == 0) mosts[slot][part / 64] = most;
        __syncthreads();
        for (int i = 0; i < WAVES; ++i) most = __builtin_fmax(most, mosts[slot][i]);
#endif
        if (wide) {
            float scale = (float)(most / __builtin_sqrt((double)(ss / (float)a.cols + a.eps)) / 127.);
            const bool bad = !(most < __builtin_inf()) || !(ss < __builtin_inff()) || !(scale < __builtin_inff());
            if (bad) scale = __builtin_nanf("");
            if (part == 0) a.scale[row_at] = scale;
            if (bad || most == 0) {
                u32 q[(VEC + 3) / 4] = {};
                for (int c = part * VEC; c < cols; c += LANES * VEC) put(q, 0u, c);
                return;
            }
            const double inv = 1 / most;
            again([&](const Vec &v, const Vec &wv, int c) __attribute__((always_inline)) {
                u32 o[VEC], q[(VEC + 3) / 4];
#pragma unroll
                for (int j = 0; j < VEC; ++j) {
                    // as in nearest; t is next to s / a by its last bits
                    const double s = (double)v.at(j) * (double)wv.at(j) * 127.;
                    const double t = __builtin_rint(s * inv), rem = __builtin_fma(-t, most, s), r = __builtin_fabs(rem);
                    const int n = (int)t;
                    const bool move = r > 0.5 * most || (r == 0.5 * most && (n & 1));
                    o[j] = (u32)(move ? n + (rem > 0 ? 1 : -1) : n);
                }
                pack(q, o);
                put(q, ~0u, c);
            });
            return;
        }
    }
    const bool bad = !(ss < __builtin_inff());
    float scale = top / __builtin_sqrtf(ss / (float)a.cols + a.eps);
    const float up = 1.f;
#else
    const bool bad = !(top < __builtin_inff());
    float scale = top;
    // a is brought near 1 by a power of two, and p with it (exact), so that no
    // product below leaves fp32's range
    float up = 1.f;
    if (top < 0x1p-63f) up = 0x1p64f;
    if (top >= 0x1p64f) up = 0x1p-64f;
#endif
    scale /= 127.f;             // last, so that a small one is rounded once
    if (bad) scale = __builtin_nanf("");
    if (live && part == 0) a.scale[row_at] = scale;

    const float as = bad || top == 0.f ? 1.f : top * up;
    // above 1 / a by its last bits: then the trial of p = a / 2, the one tie
    // that is met often, is 64, the even neighbour of 63.5
    const float inv = __builtin_amdgcn_rcpf(as) * 0x1.000004p0f;
    const u32 keep = bad ? 0u : ~0u;
    const auto emit = [&](const Vec &v, const Vec &wv, int c) __attribute__((always_inline)) {
        // trials of all elements, and again where one of them is not nearest
        u32 o[VEC], q[(VEC + 3) / 4];
        float far = 0.f;
#pragma unroll
        for (int j = 0; j < VEC; ++j) {
            const float s = product(v, wv, j) * (127.f * up);
            const float t = trial(s, inv);
            o[j] = __builtin_bit_cast(u32, t);
            float rem = __builtin_fmaf(-(t - SHIFT), as, s);
#if !NORM
            // Ties: an odd trial's last bit makes a remainder of a / 2 larger
            // (a and so a / 2 have 8 bits, their last one is 0), and no smaller
            // one as large.  (bf16 values of half the maximum are many; of a
            // norm's products few are, and every tie is done again.)
            rem = __builtin_bit_cast(float, __builtin_bit_cast(u32, rem) | (o[j] & 1));
#endif
            far = __builtin_fmaxf(far, __builtin_fabsf(rem));
        }
        pack(q, o);
        if (NORM ? far >= 0.5f * as : far > 0.5f * as) {
#pragma unroll
            for (int j = 0; j < VEC; ++j) o[j] = (u32)nearest(product(v, wv, j) * (127.f * up), as, inv);
            pack(q, o);
        }
        put(q, keep, c);
    };
#if HELD
#pragma unroll
    for (int i = 0; i < HELD; ++i) {
        const int c = (i * LANES + part) * VEC;
        if (c < cols) emit(v[i], wv[i], c);
    }
#else
    again(emit);
#endif
}
