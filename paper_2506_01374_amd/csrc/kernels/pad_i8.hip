// int8 rows of any length to rows of whole 16-byte chunks with zeros behind
// them, which add nothing to a product's sums: two or three matrices of rows
// of K, one after the other, a chunk a thread.
//
// Bound by memory: every row read and written once (2048 + 14336 rows of 4098,
// 134 MB: 26.8 us, 5.0 TB/s).  It pays where the product would otherwise read
// each row many times at addresses that start on no 16 bytes.
typedef signed char i8;
typedef int i32x4 __attribute__((ext_vector_type(4)));

struct PadI8Args {
    const i8 *A, *B0, *B1;      // [M][K], [N][K], and the rest [][K]
    i8 *out;                    // [rows][K rounded up to 16]
    long long rows, M;
    int N, K;
};

extern "C" __global__ __launch_bounds__(256) void rc_pad_i8(PadI8Args a) {
    const unsigned chunks = (a.K + 15) / 16;
    const unsigned at = blockIdx.x * 256u + threadIdx.x;      // the grid has less than 2^32 threads
    long long row = at / chunks;
    if (row >= a.rows) return;
    const int k = (int)(at % chunks) * 16;
    const i8 *src = a.A;
    if (row >= a.M) {
        row -= a.M;
        src = a.B0;
        if (row >= a.N) {
            row -= a.N;
            src = a.B1;
        }
    }
    src += (size_t)row * a.K + k;
    const int left = a.K - k;
    i32x4 v = {0, 0, 0, 0};
    if (left >= 16) {
        __builtin_memcpy(&v, src, 16);
    } else {
#pragma unroll
        for (int j = 0; j < 15; ++j)
            if (j < left) v[j / 4] |= (int)((unsigned)(unsigned char)src[j] << (8 * (j % 4)));
    }
    *(i32x4 *)(a.out + (size_t)at * 16) = v;
}
