// Dropout on rows whose mask is a function of a seed and is stored nowhere: the backward pass forms it anew.
//
//   t = round(65536 p);  value e of the rows (row-major) has a word w_e of 16 random bits;
//   out_e = w_e >= t ? x_e 65536 / (65536 - t) : 0,  + residual_e
//
// The words are those of Philox 4x32 in ten rounds (Salmon, Moraes, Dror and Shaw, "Parallel random numbers: as easy as 1, 2, 3",
// 2011): key = the seed's two halves, counter = (e / 8, offset), eight words of 16 bits each, the lower half of each result first.
// Neither the type nor the row count changes a value's word.
#include "scnn_dense.h"

namespace scnn {

// Eight words for block `i` of eight values: word k is bits 16 (k % 2) .. of c[k / 2].
__device__ __forceinline__ void philox(unsigned long long i, unsigned long long offset, unsigned long long seed, unsigned (&c)[4]) {
    c[0] = (unsigned)i;
    c[1] = (unsigned)(i >> 32);
    c[2] = (unsigned)offset;
    c[3] = (unsigned)(offset >> 32);
    unsigned k0 = (unsigned)seed, k1 = (unsigned)(seed >> 32);
#pragma unroll
    for (int r = 0; r < 10; ++r) {
        const unsigned long long p0 = (unsigned long long)0xD2511F53u * c[0], p1 = (unsigned long long)0xCD9E8D57u * c[2];
        c[0] = (unsigned)(p1 >> 32) ^ c[1] ^ k0;
        c[1] = (unsigned)p1;
        c[2] = (unsigned)(p0 >> 32) ^ c[3] ^ k1;
        c[3] = (unsigned)p0;
        k0 += 0x9E3779B9u;
        k1 += 0xBB67AE85u;
    }
}

struct DropoutArgs {
    const void *x, *residual;
    void* out;  // may be x or residual: a value is read by the thread that writes it, before it does
    long long rows, channels;
    const long long* rows_dev;
    unsigned long long seed, offset;
    const unsigned long long* rng;
    unsigned threshold;
    float scale;
};

// Eight values a thread and step, of one counter: ten rounds of two 32-bit products each are ten instructions a value, which memory hides.
// Under the profiler, on the same arrays again and again (the last-level cache holds them): 8192 x 4096 bf16 with a residual 30 us, 6.6 TB/s;
// 643072 x 35 fp16 16 us, 5.5 TB/s; 64 x 1024 fp32 2.6 us.  The first on arrays that change from call to call: 38.7 us, 5.2 TB/s.
template <typename T>
__global__ __launch_bounds__(256) void k_dropout(DropoutArgs p) {
    constexpr int V = kVec<T>, H = 8 / V;
    const long long n = rows_of(p.rows, p.rows_dev) * p.channels;
    const unsigned long long seed = p.rng ? p.rng[0] : p.seed, offset = p.rng ? p.rng[1] : p.offset;
    const T *x = (const T*)p.x, *residual = (const T*)p.residual;
    T* out = (T*)p.out;
    const long long step = (long long)gridDim.x * 256;
    for (long long i = (long long)blockIdx.x * 256 + threadIdx.x; i * 8 < n; i += step) {
        const long long at = i * 8;
        const int m = (int)(n - at < 8 ? n - at : 8);
        VecOf<T, V> a[H], b[H], y[H];
#pragma unroll
        for (int h = 0; h < H; ++h) {
            a[h] = load_raw<T>(x + at + h * V, m - h * V, false);
            b[h] = VecOf<T, V>{};
            if (residual) b[h] = load_raw<T>(residual + at + h * V, m - h * V, false);
        }
        unsigned c[4];
        philox((unsigned long long)i, offset, seed, c);
#pragma unroll
        for (int k = 0; k < 8; ++k) {
            const unsigned word = k & 1 ? c[k / 2] >> 16 : c[k / 2] & 0xffffu;
            float v = word >= p.threshold ? (float)a[k / V][k % V] * p.scale : 0.0f;
            if (residual) v += (float)b[k / V][k % V];
            y[k / V][k % V] = (T)v;
        }
#pragma unroll
        for (int h = 0; h < H; ++h) store_raw<T>(out + at + h * V, m - h * V, y[h]);
    }
}

hipError_t launch_dropout(int dtype, const void* x, const void* residual, void* out, long long rows, const long long* rows_dev,
                          long long channels, double p, unsigned long long seed, unsigned long long offset,
                          const unsigned long long* rng, hipStream_t s) {
    DropoutArgs a = {};
    a.x = x; a.residual = residual; a.out = out;
    a.rows = rows; a.channels = channels; a.rows_dev = rows_dev;
    a.seed = seed; a.offset = offset; a.rng = rng;
    a.threshold = (unsigned)__builtin_rint(p * 65536.0);
    a.scale = a.threshold < 65536 ? (float)(65536.0 / (65536.0 - (double)a.threshold)) : 0.0f;
    const long long blocks = (rows * channels + 2047) / 2048, most = 8LL * device_cu_count();
    const dim3 grid((unsigned)(blocks < most ? blocks : most));
    switch (dtype) {
        case SCNN_F32: hipLaunchKernelGGL((k_dropout<float>), grid, dim3(256), 0, s, a); break;
        case SCNN_BF16: hipLaunchKernelGGL((k_dropout<__bf16>), grid, dim3(256), 0, s, a); break;
        default: hipLaunchKernelGGL((k_dropout<_Float16>), grid, dim3(256), 0, s, a);
    }
    return hipGetLastError();
}

}  // namespace scnn
