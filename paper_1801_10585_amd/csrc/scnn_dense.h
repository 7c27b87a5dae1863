// Shared by the layers on plain rows of values (linear layers, layer norm) and by gradient clipping: element types,
// vectors of them at any alignment, activations, sums across lanes.
#pragma once
#include <type_traits>

#include "scnn_internal.h"

namespace scnn {

template <int DTYPE> struct DenseType;
template <> struct DenseType<SCNN_F32> { using type = float; };
template <> struct DenseType<SCNN_BF16> { using type = __bf16; };
template <> struct DenseType<SCNN_F16> { using type = _Float16; };

// Elements of one 16-byte access.
template <typename T> constexpr int kVec = 16 / (int)sizeof(T);
template <typename T, int N> using VecOf = T __attribute__((ext_vector_type(N)));

template <typename T> using BitsAs = VecOf<T, kVec<T>>;

// Sixteen bytes from an address aligned to the element only (rows of odd widths start anywhere): the compiler makes one
// global access of 16 bytes of it, which the hardware takes at any address.  Of a vector that a row ends in, n < kVec elements
// are there, the others are 0: up to three fp32 one by one; up to seven of 16 bits as the row's last sixteen bytes, shifted,
// where the row is that long (`whole`), else in pieces of eight, four and two bytes.  (Without TAIL a row ends with a vector.)
template <typename T, bool TAIL = true>
__device__ __forceinline__ VecOf<T, kVec<T>> load_raw(const T* __restrict__ p, int n, bool whole) {
    VecOf<T, kVec<T>> r = {};
    if (n >= kVec<T>) {
        __builtin_memcpy(&r, p, 16);
    } else if constexpr (!TAIL) {
    } else if constexpr (sizeof(T) == 4) {
#pragma unroll
        for (int i = 0; i < 3; ++i)
            if (i < n) r[i] = p[i];
    } else if (n > 0) {
        typedef unsigned __int128 u128;
        u128 v = 0;
        if (whole) {
            __builtin_memcpy(&v, p + n - 8, 16);
            v >>= 16 * (8 - n);
        } else {
            int at = 0;
            if (n & 4) {
                unsigned long long q;
                __builtin_memcpy(&q, p, 8);
                v = q;
                at = 4;
            }
            if (n & 2) {
                unsigned q;
                __builtin_memcpy(&q, p + at, 4);
                v |= (u128)q << (16 * at);
                at += 2;
            }
            if (n & 1) {
                unsigned short q;
                __builtin_memcpy(&q, p + at, 2);
                v |= (u128)q << (16 * at);
            }
        }
        r = __builtin_bit_cast(BitsAs<T>, v);
    }
    return r;
}
template <typename T, bool TAIL = true>
__device__ __forceinline__ void load_elems(const T* __restrict__ p, int n, bool whole, float (&v)[kVec<T>]) {
    const VecOf<T, kVec<T>> r = load_raw<T, TAIL>(p, n, whole);
#pragma unroll
    for (int i = 0; i < kVec<T>; ++i) v[i] = (float)r[i];
}

// The first n elements of a vector; those of a row's last one in pieces of eight, four and two bytes.
template <typename T, bool TAIL = true>
__device__ __forceinline__ void store_raw(T* __restrict__ p, int n, VecOf<T, kVec<T>> r) {
    typedef unsigned __int128 u128;
    u128 v = __builtin_bit_cast(u128, r);
    if (n >= kVec<T>) {
        __builtin_memcpy(p, &v, 16);
        return;
    }
    if (!TAIL || n <= 0) return;
    if (sizeof(T) == 2 && (n & 4)) {
        __builtin_memcpy(p, &v, 8);
        v >>= 64;
        p += 4;
    }
    if (n & 2) {
        __builtin_memcpy(p, &v, 2 * sizeof(T));
        v >>= 16 * (int)sizeof(T);
        p += 2;
    }
    if (n & 1) __builtin_memcpy(p, &v, sizeof(T));
}
// Rounded once, to nearest even.
template <typename T, bool TAIL = true>
__device__ __forceinline__ void store_elems(T* __restrict__ p, int n, const float (&v)[kVec<T>]) {
    VecOf<T, kVec<T>> r;
#pragma unroll
    for (int i = 0; i < kVec<T>; ++i) r[i] = (T)v[i];
    store_raw<T, TAIL>(p, n, r);
}

// Rows of a call: the host's count, or the device's, held to the arrays' capacity.
__device__ __forceinline__ long long rows_of(long long rows, const long long* __restrict__ rows_dev) {
    if (!rows_dev) return rows;
    long long n = *rows_dev;
    // (the same in every lane, which the compiler does not know of a load: loops over rows stay scalar)
    n = (long long)((unsigned long long)(unsigned)__builtin_amdgcn_readfirstlane((int)((unsigned long long)n >> 32)) << 32 |
                    (unsigned)__builtin_amdgcn_readfirstlane((int)n));
    return n < 0 ? 0 : (n < rows ? n : rows);
}

// Grid of `blocks` workgroups of THREADS along one axis and `y` along another.  A launch holds fewer than 2^32 threads along an
// axis: what goes past 2^31 continues along z, and block_id is the number along both.  The last z may be part empty: kernels
// leave where block_id is past their work.
template <int THREADS> constexpr long long kBlocksX = (1LL << 31) / THREADS;
template <int THREADS> dim3 grid_of(long long blocks, unsigned y = 1) {
    if (blocks <= kBlocksX<THREADS>) return dim3((unsigned)blocks, y);
    return dim3((unsigned)kBlocksX<THREADS>, y, (unsigned)((blocks + kBlocksX<THREADS> - 1) / kBlocksX<THREADS>));
}
template <int THREADS> __device__ __forceinline__ long long block_id() { return blockIdx.z * kBlocksX<THREADS> + blockIdx.x; }

// Distribution function of the normal density, Phi(z) = erfc(-z / sqrt 2) / 2, and e = exp(-z^2 / 2) on the way.  With
// erfcx(x) = exp(x^2) erfc(x) as t P(t), t = 1 / (1 + 0.4 x), P of degree eight fitted for the least relative error over
// x >= 0 (1.3e-7), Phi of either side is a product, not a difference, at a fifth of the library function's instructions: behind a
// wide product, 33 M values of erfcf took 100 us, more than a third of the product.  Its error is 8 x 2^-24 of the value down
// to z = -2; below, the exponential's argument z^2 / 2 is rounded twice: 1.1 z^2 x 2^-24 of the value at most (2e-6 at -6, 7e-6 at
// -12).  (The argument in two parts keeps 8 x 2^-24 down to -13 and makes the layer of 8192 x 4096 -> 4096 bf16 5 per cent longer.)
__device__ __forceinline__ float normal_cdf(float z, float& e) {
    const float t = __builtin_amdgcn_rcpf(__builtin_fmaf(0.4f * 0.70710678f, __builtin_fabsf(z), 1.0f));
    e = __builtin_amdgcn_exp2f(z * z * -0.72134752f);
    float p = 0.05023009330f;
    p = __builtin_fmaf(p, t, -0.18275529146f);
    p = __builtin_fmaf(p, t, 0.16880626976f);
    p = __builtin_fmaf(p, t, -0.00531849405f);
    p = __builtin_fmaf(p, t, 0.14125579596f);
    p = __builtin_fmaf(p, t, 0.16860525310f);
    p = __builtin_fmaf(p, t, 0.20782974362f);
    p = __builtin_fmaf(p, t, 0.22567094862f);
    p = __builtin_fmaf(p, t, 0.22567580640f);
    const float tail = 0.5f * t * p * e;
    return z < 0.0f ? tail : 1.0f - tail;
}

// 1 / (1 + exp(-z)), below 0 good to (6 + 1.2 |z|) x 2^-24 of the value (the exponential's argument is rounded), 0 from -87.4 on.
__device__ __forceinline__ float logistic(float z) {
    return __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(z * -1.44269504f));
}

__device__ __forceinline__ float activate(float z, int act) {
    float e;
    switch (act) {
        case SCNN_ACT_RELU: return z < 0.0f ? 0.0f : z;  // (a NaN stays one)
        case SCNN_ACT_GELU: return z * normal_cdf(z, e);
        case SCNN_ACT_SILU: return z * logistic(z);
        default: return z;
    }
}

// g * d act(z) / dz
__device__ __forceinline__ float activate_back(float g, float z, int act) {
    switch (act) {
        case SCNN_ACT_RELU: return z <= 0.0f ? 0.0f : g;
        case SCNN_ACT_GELU: {
            float e;
            const float cdf = normal_cdf(z, e);
            return g * (cdf + z * e * 0.39894228f);
        }
        case SCNN_ACT_SILU: {
            const float s = logistic(z);
            return g * (s * (1.0f + z * (1.0f - s)));
        }
        default: return g;
    }
}

// Sum over groups of P lanes of a wave (P a power of two), the same bits in each of the group's lanes.
template <int P, typename F>
__device__ __forceinline__ F lanes_add(F v) {
#pragma unroll
    for (int d = 1; d < P; d <<= 1) {
        if constexpr (sizeof(F) == 8 && !std::is_same<F, double>::value) {  // (a pair of floats)
            F o;
            o.x = __shfl_xor(v.x, d, 64);
            o.y = __shfl_xor(v.y, d, 64);
            v += o;
        } else {
            v += __shfl_xor(v, d, 64);
        }
    }
    return v;
}

// out[c] = sum over p < parts of part[p * cols + c], in a fixed order, rounded once; columns [0, split) go to out0, the
// rest to out1 (either may be null).
hipError_t launch_column_sums(const float* part, int parts, long long cols, long long split, void* out0, void* out1,
                              int dtype, hipStream_t s);

// Tensors of a gradient list, as the kernels' argument: up to 120 of them fit the 4096 bytes that a launch may carry.  (A
// launch costs the host more the more it carries: lists of up to 24 take a table of that size.)
struct ClipTensor {
    const void* src;
    void* dst;
    long long count;
    unsigned first;  // first workgroup
    int dtype;
};
template <int N>
struct ClipTable {
    ClipTensor t[N];
    long long chunk;  // entries a workgroup
    int n;
    int slot;         // the launch's first partial sum
};
static_assert(sizeof(ClipTable<120>) + 64 <= 4096, "kernel arguments of one launch");

long long grad_norm_parts(int n, const int64_t* counts);  // partial sums (double) of a call
hipError_t launch_grad_clip(int n, const void* const* src, void* const* dst, const int64_t* counts, const int* dtypes,
                            double max_norm, double* result, double* part, hipStream_t s);

size_t norm_bwd_part_bytes(long long rows, int channels, int dtype);
hipError_t launch_norm_fwd(const void* x, long long rows, const long long* rows_dev, int channels, const void* gamma,
                           const void* beta, float eps, void* out, float* mean, float* rstd, int dtype, hipStream_t s);
hipError_t launch_norm_bwd(const void* x, const void* g, long long rows, const long long* rows_dev, int channels,
                           const void* gamma, const float* mean, const float* rstd, void* dx, void* dgamma, void* dbeta,
                           float* part, int dtype, hipStream_t s);

// A linear layer's call, forward (x, w, bias, residual, out, pre) or backward (x, w, pre, g, dx, dw, dbias).
struct LinearCall {
    const void *x, *w, *bias, *residual, *g;
    const void* pre_in;
    void *out, *pre, *dx, *dw, *dbias;
    long long rows, c_in, c_out;
    const long long* rows_dev;
    int act;
    void* workspace;
};
size_t linear_fwd_part_bytes(int dtype, long long rows, long long c_in, long long c_out);
size_t linear_bwd_bytes(int dtype, long long rows, long long c_in, long long c_out, int act);
hipError_t launch_linear_fwd(int dtype, const LinearCall& c, hipStream_t s);
hipError_t launch_linear_bwd(int dtype, const LinearCall& c, hipStream_t s);

}  // namespace scnn
