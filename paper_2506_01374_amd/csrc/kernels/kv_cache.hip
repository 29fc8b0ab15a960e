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

struct Vec { u32 w[WORDS]; };
struct Bytes { u32 w[VEC / 4]; };

__device__ __forceinline__ float element(const Vec &x, int j) {
    return __builtin_bit_cast(float, j % 2 ? x.w[j / 2] & 0xFFFF0000u : x.w[j / 2] << 16);
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

extern "C" __global__ __launch_bounds__(64 * WAVES) void rc_kv_write(CacheArgs a) {
    const int lane = threadIdx.x & 63, row = blockIdx.x * WAVES + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    if (row >= a.T) return;
    const int chunks = a.HKV * LANES;                  // of K's row, then of V's
    const bf16_t *k = a.k + (size_t)row * a.HKV * HD, *v = a.v + (size_t)row * a.HKV * HD;
    auto fetch = [&](int c) {
        Vec x = {};
        const bool isv = c >= chunks;
        if (c < 2 * chunks) __builtin_memcpy(&x, (isv ? v : k) + (size_t)(isv ? c - chunks : c) * VEC, sizeof x);
        return x;
    };
    Vec x = fetch(lane);                               // on its way while the place is found
    const Place p = place(a, row);
    if (p.slot < 0) return;
    for (int c = lane; c - lane < 2 * chunks; c += 64) {
        const Vec next = fetch(c + 64);
        const bool isv = c >= chunks, live = c < 2 * chunks;
        const int cc = isv ? c - chunks : c, h = cc / LANES, d = cc % LANES * VEC;
        const long long slot = p.slot + ((long long)h << a.shift);
#if I8
        // magnitudes as bits: above all others a NaN
        u32 top = 0;
#pragma unroll
        for (int j = 0; j < VEC; ++j) top = max(top, __builtin_bit_cast(u32, element(x, j)) & 0x7FFFFFFFu);
#pragma unroll
        for (int s = 1; s < LANES; s <<= 1) top = max(top, (u32)__shfl_xor((int)top, s));
        const float most = __builtin_bit_cast(float, top);
        const bool bad = !(most < __builtin_inff());
        // near 1 by a power of two, exactly, so that 127 x and its remainders
        // stay in fp32's range
        const float up = most < 0x1p-63f ? 0x1p64f : most >= 0x1p64f ? 0x1p-64f : 1.f;
        const float as = bad || most == 0.f ? 1.f : most * up, inv = 1.f / as;
        Bytes q = {};
#pragma unroll
        for (int j = 0; j < VEC; ++j) {
            // s - t a is exact (127 x has 15 bits, a 8), and t within one of the result
            const float s = element(x, j) * (127.f * up);
            const float t = __builtin_rintf(s * inv), rem = __builtin_fmaf(-t, as, s), r = __builtin_fabsf(rem);
            const int n = (int)t;
            const bool move = r > 0.5f * as || (r == 0.5f * as && (n & 1));
            const int e = bad ? 0 : move ? n + (rem > 0.f ? 1 : -1) : n;
            q.w[j / 4] |= (u32)(e & 255) << (8 * (j % 4));
        }
        if (live) {
            __builtin_memcpy((isv ? a.V : a.K) + slot * HD + d, &q, sizeof q);
            if (d == 0) (isv ? a.Vs : a.Ks)[slot] = bad ? __builtin_nanf("") : most / 127.f;
        }
#else
        if (live) __builtin_memcpy((isv ? a.V : a.K) + (slot * HD + d) * 2, &x, sizeof x);
#endif
        x = next;
    }
}

extern "C" __global__ __launch_bounds__(64 * WAVES) void rc_kv_read(CacheArgs a) {
    const int lane = threadIdx.x & 63, row = blockIdx.x * WAVES + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    if (row >= a.T) return;
    const int chunks = a.HKV * LANES;
    bf16_t *k = a.k + (size_t)row * a.HKV * HD, *v = a.v + (size_t)row * a.HKV * HD;
    const Place p = place(a, row);
    if (!p.row) return;
    for (int c = lane; c < 2 * chunks; c += 64) {
        const bool isv = c >= chunks;
        const int cc = isv ? c - chunks : c, h = cc / LANES, d = cc % LANES * VEC;
        const long long slot = p.slot + ((long long)h << a.shift);
        Vec x = {};
        if (p.slot >= 0) {
#if I8
            Bytes q;
            __builtin_memcpy(&q, (isv ? a.V : a.K) + slot * HD + d, sizeof q);
            const float s = (isv ? a.Vs : a.Ks)[slot];
#pragma unroll
            for (int j = 0; j < VEC; ++j) {
                const __bf16 y = (__bf16)((float)(signed char)(q.w[j / 4] >> (8 * (j % 4))) * s);
                x.w[j / 2] |= (u32)__builtin_bit_cast(bf16_t, y) << (16 * (j % 2));
            }
#else
            __builtin_memcpy(&x, (isv ? a.V : a.K) + (slot * HD + d) * 2, sizeof x);
#endif
        }
        __builtin_memcpy((isv ? v : k) + (size_t)cc * VEC, &x, sizeof x);
    }
}
