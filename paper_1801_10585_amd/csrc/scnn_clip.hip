// Global norm of many gradient tensors and their scaling (clipping by the global norm).
//
//   norm = sqrt(sum over all entries of g^2),  scale = max_norm / (norm + 1e-6), at most 1,  out = g scale
//
// Bound by memory: every entry is read for the norm, then read again and written; nothing can be scaled before the last
// entry has been squared.  The tensors' addresses travel in the kernels' arguments (a table of up to 120 a launch),
// so that a call copies nothing to the device and can be captured in a graph.  A workgroup owns one chunk of one tensor.
// Squares are summed in fp64, which costs nothing beside the loads, so that no gradient of fp32 overflows its square and the
// order of addition does not show; the chunks' sums are stored and added in one fixed order by every workgroup of the second
// launch (some thousand numbers from the L2), which saves a launch between the two.  127 M bf16 entries in 60 tensors: 58 us for
// the squares (4.4 TB/s), 84 to scale them (6.0 TB/s, a part of the second read from the caches); 18 small tensors: 4 + 5 us.
#include "scnn_dense.h"

namespace scnn {

template <typename T>
__device__ __forceinline__ double sum_squares(const T* __restrict__ p, long long n) {
    constexpr int V = kVec<T>;
    double sum = 0.0;
    long long i = (long long)threadIdx.x * V;
    for (; i + 3 * 256 * V + V <= n; i += 4 * 256 * V) {  // four loads in flight
        float v[4][V];
#pragma unroll
        for (int k = 0; k < 4; ++k) load_elems<T>(p + i + k * 256 * V, V, true, v[k]);
#pragma unroll
        for (int k = 0; k < 4; ++k)
#pragma unroll
            for (int j = 0; j < V; ++j) sum += (double)v[k][j] * (double)v[k][j];
    }
    for (; i < n; i += 256 * V) {
        float v[V];
        load_elems<T>(p + i, (int)(n - i < V ? n - i : V), n >= V, v);
#pragma unroll
        for (int j = 0; j < V; ++j) sum += (double)v[j] * (double)v[j];
    }
    return sum;
}

// F: the product's type.
template <typename T, typename F>
__device__ __forceinline__ void scale_chunk(const T* p, T* q, long long n, F scale) {
    constexpr int V = kVec<T>;
    long long i = (long long)threadIdx.x * V;
    for (; i + 3 * 256 * V + V <= n; i += 4 * 256 * V) {
        float v[4][V];
#pragma unroll
        for (int k = 0; k < 4; ++k) load_elems<T>(p + i + k * 256 * V, V, true, v[k]);
#pragma unroll
        for (int k = 0; k < 4; ++k) {
#pragma unroll
            for (int j = 0; j < V; ++j) v[k][j] = (float)((F)v[k][j] * scale);
            store_elems<T>(q + i + k * 256 * V, V, v[k]);
        }
    }
    for (; i < n; i += 256 * V) {
        const int m = (int)(n - i < V ? n - i : V);
        float v[V];
        load_elems<T>(p + i, m, false, v);
#pragma unroll
        for (int j = 0; j < V; ++j) v[j] = (float)((F)v[j] * scale);
        store_elems<T>(q + i, m, v);
    }
}

// Sum over the workgroup's 256 threads, the same in each of them.
__device__ __forceinline__ double block_add(double v, double* s_part /*[4]*/) {
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) v += __shfl_xor(v, d, 64);
    if ((threadIdx.x & 63) == 0) s_part[threadIdx.x >> 6] = v;
    __syncthreads();
    return (s_part[0] + s_part[1]) + (s_part[2] + s_part[3]);
}

// The tensor that owns workgroup `block` of the launch: first[t] <= block < first[t + 1].
template <int N>
__device__ __forceinline__ int tensor_of(const ClipTable<N>& tab, unsigned block) {
    int lo = 0, hi = tab.n - 1;
    while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if (tab.t[mid].first <= block) lo = mid; else hi = mid - 1;
    }
    return lo;
}

template <int N>
__global__ __launch_bounds__(256) void k_grad_squares(ClipTable<N> tab, double* __restrict__ part) {
    __shared__ double s_part[4];
    const ClipTensor& t = tab.t[tensor_of(tab, blockIdx.x)];
    const long long at = (long long)(blockIdx.x - t.first) * tab.chunk;
    const long long n = t.count - at < tab.chunk ? t.count - at : tab.chunk;
    double sum;
    if (t.dtype == SCNN_F32) sum = sum_squares((const float*)t.src + at, n);
    else if (t.dtype == SCNN_BF16) sum = sum_squares((const __bf16*)t.src + at, n);
    else sum = sum_squares((const _Float16*)t.src + at, n);
    sum = block_add(sum, s_part);
    if (threadIdx.x == 0) part[tab.slot + blockIdx.x] = sum;
}

// result = {norm, scale}, by the launch with slot 0.  Without destinations (the norm alone) the grid is one workgroup.
template <int N>
__global__ __launch_bounds__(256) void k_grad_scale(ClipTable<N> tab, const double* __restrict__ part, int parts, double max_norm,
                                                    double* __restrict__ result) {
    __shared__ double s_part[4];
    double sum = 0.0;
    for (int i = threadIdx.x; i < parts; i += 256) sum += part[i];
    const double norm = sqrt(block_add(sum, s_part));
    double scale = max_norm / (norm + 1e-6);
    if (scale > 1.0) scale = 1.0;  // (NaN stays NaN)
    if (tab.slot == 0 && blockIdx.x == 0 && threadIdx.x == 0) {
        result[0] = norm;
        result[1] = scale;
    }
    if (tab.n == 0) return;
    // from the last chunk to the first: what the norm read last is what the caches still hold
    const unsigned block = gridDim.x - 1 - blockIdx.x;
    const ClipTensor& t = tab.t[tensor_of(tab, block)];
    if (scale == 1.0 && t.dst == t.src) return;  // in place and nothing to change
    const long long at = (long long)(block - t.first) * tab.chunk;
    const long long n = t.count - at < tab.chunk ? t.count - at : tab.chunk;
    auto all = [&](auto by) {
        if (t.dtype == SCNN_F32) scale_chunk((const float*)t.src + at, (float*)t.dst + at, n, by);
        else if (t.dtype == SCNN_BF16) scale_chunk((const __bf16*)t.src + at, (__bf16*)t.dst + at, n, by);
        else scale_chunk((const _Float16*)t.src + at, (_Float16*)t.dst + at, n, by);
    };
    // a scale that fp32 would hold in few bits or not at all multiplies in fp64: gradients of 10^38 have ordinary results
    if (scale < 0x1p-100) all(scale);
    else all((float)scale);
}

// Entries a workgroup takes: about 2048 workgroups of work where there is enough, never fewer than 4096 entries.
static long long chunk_of(long long total) {
    const long long per = round_up((total + 2047) / 2048, 2048);
    return per < 4096 ? 4096 : per;
}

long long grad_norm_parts(int n, const int64_t* counts) {
    long long total = 0, parts = 0;
    for (int i = 0; i < n; ++i) total += counts[i];
    const long long chunk = chunk_of(total);
    for (int i = 0; i < n; ++i) parts += (counts[i] + chunk - 1) / chunk;
    return parts;
}

template <int N>
static hipError_t grad_clip(int n, const void* const* src, void* const* dst, const int64_t* counts, const int* dtypes,
                            double max_norm, double* result, double* part, hipStream_t s) {
    long long total = 0;
    for (int i = 0; i < n; ++i) total += counts[i];
    const long long chunk = chunk_of(total);
    const int parts = (int)grad_norm_parts(n, counts);
    for (int pass = 0; pass < 2; ++pass) {
        ClipTable<N> tab;
        tab.chunk = chunk;
        long long slot = 0;
        int i = 0;
        do {
            tab.n = 0;
            tab.slot = (int)slot;
            unsigned blocks = 0;
            for (; i < n && tab.n < N; ++i) {
                if (counts[i] == 0) continue;
                ClipTensor& t = tab.t[tab.n++];
                t.src = src[i];
                t.dst = dst ? dst[i] : nullptr;
                t.count = counts[i];
                t.dtype = dtypes[i];
                t.first = blocks;
                blocks += (unsigned)((counts[i] + chunk - 1) / chunk);
            }
            if (pass == 0) {
                if (blocks) hipLaunchKernelGGL((k_grad_squares<N>), dim3(blocks), dim3(256), 0, s, tab, part);
            } else {
                if (!dst) {
                    tab.n = 0;
                    blocks = 1;
                }
                if (blocks || slot == 0)
                    hipLaunchKernelGGL((k_grad_scale<N>), dim3(blocks ? blocks : 1), dim3(256), 0, s, tab, part, parts, max_norm,
                                       result);
                if (!dst) break;
            }
            slot += blocks;
        } while (i < n);
    }
    return hipGetLastError();
}

hipError_t launch_grad_clip(int n, const void* const* src, void* const* dst, const int64_t* counts, const int* dtypes,
                            double max_norm, double* result, double* part, hipStream_t s) {
    return n <= 24 ? grad_clip<24>(n, src, dst, counts, dtypes, max_norm, result, part, s)
                   : grad_clip<120>(n, src, dst, counts, dtypes, max_norm, result, part, s);
}

}  // namespace scnn
