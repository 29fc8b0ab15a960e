// New tokens' keys and values into a paged cache, and rows of a paged cache
// back into packed rows, for gfx950: bf16, or int8 with an fp32 scale for each
// token and head.
//
// Compile-time schedule (generated prologue):
//   WAVES   waves of a workgroup (Parallel); a wave moves a token
//   VEC     elements of a lane's load, 4 or 8 (Vectorize)
//   HD      head dimension: 64, 128 or 256
//   I8      1: the cache holds int8 and scales
//
// Sequence b has the packed rows offsets[b] .. offsets[b + 1] - 1, which are the
// newest of its lens[b] tokens; position p of it is slot p % page of page
// table[b][p / page], [pages][HKV][page][HD].  Whatever the offsets, lengths and
// the table hold, no access leaves its buffer: a row in no sequence is left
// out, and one whose page is not in the cache is not written, and read as 0.
//
// int8: scale = max |x| / 127 over a token's head, q = rint(127 x / max |x|),
// halves to the even integer, exactly rounded.  Zeros have scale 0 and q 0; a
// head that holds a NaN or an infinity has scale NaN and q 0.
//
// Bound by memory; for few tokens by the way through offsets, lengths and table,
// three loads one after the other, beside which the token's own are under way.
// 8000 rows of 8 heads of 128 written to an int8 cache take 13.5 us (3.7 TB/s), 16384
// read from one 22.4 (4.5); 64 rows written 6 and 777 of 4 heads of 64 read 5.6, of
// which the launch is the most.

typedef unsigned short bf16_t;
typedef unsigned int u32;

#define LANES (HD / VEC)           // lanes of a head
#define WORDS (VEC / 2)            // of a lane's bf16 elements

struct CacheArgs {
    bf16_t *k, *v;                 // [T][HKV][HD]
    char *K, *V;                   // [pages][HKV][page][HD]
    float *Ks, *Vs;                // [pages][HKV][page] (I8)
    const int *offsets, *lens, *table;
    int T, B, HKV, shift, pages, width;
};

typedef u32 Vec __attribute__((ext_vector_type(WORDS)));
#if VEC == 8
typedef u32 Bytes __attribute__((ext_vector_type(2)));
#define WORD(q, i) q[i]
#else
typedef u32 Bytes;
#define WORD(q, i) q
#endif

__device__ __forceinline__ float element(const Vec &x, int j) {
    return __builtin_bit_cast(float, j % 2 ? x[j / 2] & 0xFFFF0000u : x[j / 2] << 16);
}

// the larger of each half of two words
__device__ __forceinline__ u32 larger(u32 a, u32 b) {
    typedef unsigned short u16x2 __attribute__((ext_vector_type(2)));
    return __builtin_bit_cast(u32, __builtin_elementwise_max(__builtin_bit_cast(u16x2, a), __builtin_bit_cast(u16x2, b)));
}

// the same over the lanes of a head, in rows of 16 without shared memory: lanes 1
// and 2 away, then the mirror images in 8 and in 16 lanes, whose quads and halves
// are alike by then
__device__ __forceinline__ u32 over_head(u32 x) {
#define WITH(how) x = larger(x, (u32)__builtin_amdgcn_update_dpp(0, (int)x, how, 0xF, 0xF, true))
    WITH(0xB1);
    WITH(0x4E);
    WITH(0x141);
    if (LANES > 8) WITH(0x140);
#undef WITH
#pragma unroll
    for (int s = 16; s < LANES; s <<= 1) x = larger(x, (u32)__shfl_xor((int)x, s));
    return x;
}

// (row of the cache's slots, or -1 if the token has none; whether the row is a
// sequence's) of a packed row.  The wave narrows the sequences down 64-fold
// with each load, and finds the row's among the last 64 of them.
struct Place {
    long long slot;                // of head 0: (page HKV) page_size + slot
    bool row;
};
__device__ __forceinline__ Place place(const CacheArgs &a, int row) {
    const int lane = threadIdx.x & 63;
    Place p = {-1, false};
    int lo = 0, n = a.B;           // the row's sequence is among lo .. lo + n - 1
    while (n > 64) {
        const int step = (n + 63) / 64, at = lo + lane * step;
        // sequences that start at or before the row: the last of them holds it
        const unsigned long long before = __builtin_amdgcn_ballot_w64(at < lo + n && a.offsets[min(at, a.B)] <= row);
        if (!before) return p;
        const int last = 63 - __builtin_clzll(before);
        const int to = min(n, (last + 1) * step);
        lo += last * step;
        n = to - last * step;
    }
    const int b = min(lo + lane, a.B - 1);
    const int from = a.offsets[b], to = a.offsets[b + 1], len = a.lens[b];
    const unsigned long long in = __builtin_amdgcn_ballot_w64(lane < n && from <= row && row < to);
    if (!in) return p;
    const int at = __builtin_ctzll(in);
    p.row = true;
    const long long pos = (long long)__builtin_amdgcn_readlane(len, at) - __builtin_amdgcn_readlane(to, at) + row;
    if (pos < 0 || pos >> a.shift >= a.width) return p;
    const int id = __builtin_amdgcn_readfirstlane(a.table[(long long)(lo + at) * a.width + (pos >> a.shift)]);
    if ((u32)id >= (u32)a.pages) return p;
    p.slot = ((long long)id * a.HKV << a.shift) + (pos & ((1 << a.shift) - 1));
    return p;
}

// Integers near s / a, |s| <= 127 a, as SHIFT + t: the last bit of a float there
// is 1, so that the addition rounds to an integer, which the low bits then are.
#define SHIFT 12582912.f           // 1.5 * 2^23

// VEC of a head's elements x, the head's largest magnitude `as` after the factor
// `up`, as integers.  Trials of all, within one of the result, whose remainders s
// - t a are exact (127 x has 15 bits, a 8); again where one of them is not the
// nearest, or at a half and odd: an odd trial's last bit makes a remainder of a
// half larger (a / 2 has 8 bits, their last one is 0), and no smaller one as large.
__device__ __forceinline__ Bytes quantise(const Vec &x, float as, float up) {
    // above 1 / a by its last bits: the trial of a / 2, the one tie that is met
    // often, is 64 then, the even neighbour of 63.5
    const float inv = __builtin_amdgcn_rcpf(as) * 0x1.000004p0f;
    u32 t[VEC];
    float far = 0.f;
#pragma unroll
    for (int j = 0; j < VEC; ++j) {
        const float s = element(x, j) * (127.f * up), n = __builtin_fmaf(s, inv, SHIFT);
        t[j] = __builtin_bit_cast(u32, n);
        const float rem = __builtin_fmaf(-(n - SHIFT), as, s);
        far = fmaxf(far, __builtin_fabsf(__builtin_bit_cast(float, __builtin_bit_cast(u32, rem) | (t[j] & 1))));
    }
    if (far > 0.5f * as) {
#pragma unroll
        for (int j = 0; j < VEC; ++j) {
            const float s = element(x, j) * (127.f * up), n = __builtin_bit_cast(float, t[j]);
            const float rem = __builtin_fmaf(-(n - SHIFT), as, s), r = __builtin_fabsf(rem);
            if (r > 0.5f * as || (r == 0.5f * as && (t[j] & 1))) t[j] += rem > 0.f ? 1 : -1;
        }
    }
    Bytes q;
#pragma unroll
    for (int i = 0; i < VEC / 4; ++i) {
        const u32 lo = __builtin_amdgcn_perm(t[4 * i + 1], t[4 * i], 0x0C0C0400u);
        const u32 hi = __builtin_amdgcn_perm(t[4 * i + 3], t[4 * i + 2], 0x0C0C0400u);
        WORD(q, i) = __builtin_amdgcn_perm(hi, lo, 0x05040100u);
    }
    return q;
}

// K's chunks of VEC elements, then V's; four of a lane at once
#define AT_ONCE 4

extern "C" __global__ __launch_bounds__(64 * WAVES) void rc_kv_write(CacheArgs a) {
    const int lane = threadIdx.x & 63, row = blockIdx.x * WAVES + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    if (row >= a.T) return;
    const int chunks = a.HKV * LANES;
    const bf16_t *k = a.k + (size_t)row * a.HKV * HD, *v = a.v + (size_t)row * a.HKV * HD;
    Vec x[AT_ONCE];
    auto fetch = [&](int from) {
#pragma unroll
        for (int j = 0; j < AT_ONCE; ++j) {
            const int c = from + 64 * j;
            x[j] = Vec{};
            if (c < 2 * chunks) x[j] = *(const Vec *)((c >= chunks ? v - (size_t)chunks * VEC : k) + (size_t)c * VEC);
        }
    };
    fetch(lane);                                       // on their way while the place is found
    const Place p = place(a, row);
    if (p.slot < 0) return;
    for (int from = lane;;) {
#pragma unroll
        for (int j = 0; j < AT_ONCE; ++j) {
            const int c = from + 64 * j;
            const bool isv = c >= chunks, live = c < 2 * chunks;
            const int cc = isv ? c - chunks : c, h = cc / LANES, d = cc % LANES * VEC;
            const long long slot = p.slot + ((long long)h << a.shift);
#if I8
            // magnitudes as bits: above all others a NaN
            u32 most = 0;
#pragma unroll
            for (int e = 0; e < WORDS; ++e) most = larger(most, x[j][e] & 0x7FFF7FFFu);
            most = over_head(most);
            const float top = __builtin_bit_cast(float, max(most & 0xFFFF0000u, most << 16));
            const bool bad = !(top < __builtin_inff());
            // brought near 1 by a power of two, exactly, so that 127 x and its
            // remainders stay in fp32's range
            const float up = top < 0x1p-63f ? 0x1p64f : top >= 0x1p64f ? 0x1p-64f : 1.f;
            Bytes q = quantise(x[j], bad || top == 0.f ? 1.f : top * up, up);
            if (bad) q = Bytes{};
            if (live) {
                *(Bytes *)((isv ? a.V : a.K) + slot * HD + d) = q;
                if (d == 0) (isv ? a.Vs : a.Ks)[slot] = bad ? __builtin_nanf("") : top / 127.f;
            }
#else
            if (live) *(Vec *)((isv ? a.V : a.K) + (slot * HD + d) * 2) = x[j];
#endif
        }
        from += 64 * AT_ONCE;
        if (from - lane >= 2 * chunks) break;
        fetch(from);
    }
}

extern "C" __global__ __launch_bounds__(64 * WAVES) void rc_kv_read(CacheArgs a) {
    const int lane = threadIdx.x & 63, row = blockIdx.x * WAVES + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    if (row >= a.T) return;
    const int chunks = a.HKV * LANES;
    bf16_t *k = a.k + (size_t)row * a.HKV * HD, *v = a.v + (size_t)row * a.HKV * HD;
    const Place p = place(a, row);
    if (!p.row) return;
    const long long slot0 = p.slot < 0 ? 0 : p.slot;
    for (int from = lane; from - lane < 2 * chunks; from += 64 * AT_ONCE) {
        Vec x[AT_ONCE];
#if I8
        Bytes q[AT_ONCE];
        float s[AT_ONCE];
#endif
#pragma unroll
        for (int j = 0; j < AT_ONCE; ++j) {
            const int c = min(from + 64 * j, 2 * chunks - 1), isv = c >= chunks, cc = isv ? c - chunks : c;
            const long long slot = slot0 + ((long long)(cc / LANES) << a.shift);
            const long long at = slot * HD + cc % LANES * VEC;
#if I8
            q[j] = *(const Bytes *)((isv ? a.V : a.K) + at);
            s[j] = (isv ? a.Vs : a.Ks)[slot];
#else
            x[j] = *(const Vec *)((isv ? a.V : a.K) + 2 * at);
#endif
        }
#pragma unroll
        for (int j = 0; j < AT_ONCE; ++j) {
            const int c = from + 64 * j;
#if I8
#pragma unroll
            for (int e = 0; e < WORDS; ++e) {
                u32 y = 0;
#pragma unroll
                for (int b = 0; b < 2; ++b) {
                    const int n = 2 * e + b;
                    const float f = (float)(signed char)(WORD(q[j], n / 4) >> (8 * (n % 4))) * s[j];
                    y |= (u32)__builtin_bit_cast(bf16_t, (__bf16)f) << (16 * b);
                }
                x[j][e] = y;
            }
#endif
            if (p.slot < 0) x[j] = Vec{};
            if (c < 2 * chunks) *(Vec *)((c >= chunks ? v - (size_t)chunks * VEC : k) + (size_t)c * VEC) = x[j];
        }
    }
}
