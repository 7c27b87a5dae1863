// Linear layers in 8-bit integers, for serving: out = act(z) + residual with z = (sum_k q[r, k] w[n, k]) x_scale[r] w_scale[n] + bias.
//
//   most = max(max_k |x[r, k]|, 2^-100),  x_scale[r] = most / 127,  q[r, k] = x[r, k] (127 / most) rounded to nearest even
// (fp32, both quotients rounded once), the same for the columns of a layer's weights, laid out as rows.  A row that holds a NaN
// or an infinity has scale NaN and q 0, so that its results are NaN.
//
// The sums are exact: 32-bit integers, |q w| <= 2^14 and fewer than 2^17 of them.  Rows of 8-bit values are filled up with zeros to
// a multiple of 64, so that every row begins on 64 bytes and k needs no ends.
#include "scnn_dense.h"

namespace scnn {

typedef int i4 __attribute__((ext_vector_type(4)));

constexpr float kLeast = 0x1p-100f;

// Bits of the largest magnitude, and of an infinity or NaN where there is one (the largest bits of all).
__device__ __forceinline__ unsigned magnitude(float v) { return __float_as_uint(v) & 0x7fffffffu; }
__device__ __forceinline__ unsigned wave_most(unsigned v) {
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
        const unsigned o = __shfl_xor(v, d, 64);
        v = o > v ? o : v;
    }
    return v;
}

struct Quantizer { float inverse, scale; };
__device__ __forceinline__ Quantizer quantizer(unsigned most) {
    Quantizer q;
    if (most >= 0x7f800000u) {
        q.inverse = 0.0f;
        q.scale = __uint_as_float(0x7fc00000u);
        return q;
    }
    const float m = fmaxf(__uint_as_float(most), kLeast);
    q.inverse = 127.0f / m;
    q.scale = m / 127.0f;
    return q;
}
// (an infinity or NaN times 0 would be NaN: such rows hold 0)
__device__ __forceinline__ int quantized(float v, const Quantizer& q) {
    return q.inverse == 0.0f ? 0 : (int)__builtin_rintf(v * q.inverse);
}

// A workgroup of P threads a row, H vectors of the row in a thread's registers; what a longer row has more is read again.
template <typename T, int P, int H>
__global__ __launch_bounds__(P) void k_quantize_rows(const T* __restrict__ x, long long rows_cap, const long long* __restrict__ rows_dev,
                                                     long long channels, long long width, signed char* __restrict__ out,
                                                     float* __restrict__ scale) {
    constexpr int V = kVec<T>;
    typedef signed char Q __attribute__((ext_vector_type(V)));
    __shared__ unsigned s_most[P / 64];
    const long long rows = rows_of(rows_cap, rows_dev), row = block_id<P>();
    if (row >= rows) return;
    const bool whole = channels >= V;
    const T* __restrict__ xr = x + row * channels;
    VecOf<T, V> held[H];
    unsigned most = 0;
    auto at = [&](long long j) { return (j * P + threadIdx.x) * V; };
    auto take = [&](long long c) {
        const long long n = channels - c;
        return load_raw<T>(xr + c, (int)(n < V ? (n > 0 ? n : 0) : V), whole);
    };
    auto look = [&](const VecOf<T, V>& v) {
#pragma unroll
        for (int i = 0; i < V; ++i) {
            const unsigned m = magnitude((float)v[i]);
            most = m > most ? m : most;
        }
    };
#pragma unroll
    for (int j = 0; j < H; ++j) held[j] = take(at(j));
#pragma unroll
    for (int j = 0; j < H; ++j) look(held[j]);
    for (long long j = H; at(j) < channels; ++j) look(take(at(j)));
    most = wave_most(most);
    if ((threadIdx.x & 63) == 0) s_most[threadIdx.x >> 6] = most;
    __syncthreads();
#pragma unroll
    for (int k = 0; k < P / 64; ++k) most = s_most[k] > most ? s_most[k] : most;
    const Quantizer q = quantizer(most);
    signed char* __restrict__ to = out + row * width;
    auto put = [&](long long c, const VecOf<T, V>& v) {
        Q r;
#pragma unroll
        for (int i = 0; i < V; ++i) r[i] = (signed char)quantized((float)v[i], q);
        if (c < width) __builtin_memcpy(to + c, &r, sizeof(r));
    };
#pragma unroll
    for (int j = 0; j < H; ++j) put(at(j), held[j]);
    for (long long j = H; at(j) < width; ++j) put(at(j), take(at(j)));
    if (threadIdx.x == 0) scale[row] = q.scale;
}

// 32 columns of w [c_in, c_out] a workgroup: their largest magnitudes, then their values as rows of q by way of LDS.
template <typename T>
__global__ __launch_bounds__(1024) void k_quantize_weight(const T* __restrict__ w, long long c_in, long long c_out, long long width,
                                                          signed char* __restrict__ out, float* __restrict__ scale) {
    __shared__ unsigned s_most[32][33];
    __shared__ signed char s_q[32][64 + 4];
    const int tc = threadIdx.x & 31, tr = threadIdx.x >> 5;
    const long long c0 = block_id<1024>() * 32, c = c0 + tc;
    if (c0 >= c_out) return;
    unsigned most = 0;
    if (c < c_out)
#pragma unroll 4
        for (long long k = tr; k < c_in; k += 32) {
            const unsigned m = magnitude((float)w[k * c_out + c]);
            most = m > most ? m : most;
        }
    s_most[tr][tc] = most;
    __syncthreads();
#pragma unroll
    for (int k = 0; k < 32; ++k) most = s_most[k][tc] > most ? s_most[k][tc] : most;
    const Quantizer q = quantizer(most);
    if (tr == 0 && c < c_out) scale[c] = q.scale;
    for (long long k0 = 0; k0 < width; k0 += 64) {
        __syncthreads();
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const long long k = k0 + h * 32 + tr;
            s_q[tc][h * 32 + tr] = (signed char)(k < c_in && c < c_out ? quantized((float)w[k * c_out + c], q) : 0);
        }
        __syncthreads();
        const int row = threadIdx.x >> 4, four = threadIdx.x & 15;
        if (row < 32 && c0 + row < c_out) *(int*)(out + (c0 + row) * width + k0 + four * 4) = *(const int*)&s_q[row][four * 4];
    }
}

struct Int8Args {
    const signed char *x, *w;
    const float *x_scale, *w_scale;
    const void *bias, *residual;
    void* out;
    long long m, n, width;
    const long long* rows_dev;
    int act;
};

// Epilogue of four neighbouring columns.
template <typename T>
__device__ __forceinline__ void finish4(const Int8Args& p, long long m, long long n, const i4& sum) {
    const float xs = p.x_scale[m];
    const int w = (int)(p.n - n < 4 ? p.n - n : 4);
#pragma unroll
    for (int j = 0; j < 4; ++j)
        if (j < w) {
            float z = (float)sum[j] * xs * p.w_scale[n + j];
            if (p.bias) z += (float)((const T*)p.bias)[n + j];
            z = activate(z, p.act);
            if (p.residual) z += (float)((const T*)p.residual)[m * p.n + n + j];
            ((T*)p.out)[m * p.n + n + j] = (T)z;
        }
}

// 64 x 64 outputs a workgroup of four waves, 64 k a step through registers into LDS.
template <typename T>
__global__ __launch_bounds__(256) void k_int8_tile(Int8Args p) {
    __shared__ i4 s_x[64][4], s_w[64][4];
    const long long m_end = rows_of(p.m, p.rows_dev);
    const unsigned tiles_n = (unsigned)((p.n + 63) / 64), block = (unsigned)block_id<256>();
    const long long m0 = (long long)(block / tiles_n) * 64, n0 = (long long)(block % tiles_n) * 64;
    if (m0 >= m_end) return;
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, i16 = lane & 15, q = lane >> 4;
    const int wm = (wave >> 1) * 32, wn = (wave & 1) * 32;
    const int r = tid >> 2, c = tid & 3;
    // (rows past the end are read from the last one, what they add up to is not stored)
    const signed char* __restrict__ xr = p.x + (m0 + r < m_end ? m0 + r : m_end - 1) * p.width + c * 16;
    const signed char* __restrict__ wr = p.w + (n0 + r < p.n ? n0 + r : p.n - 1) * p.width + c * 16;
    i4 acc[2][2] = {};
    i4 nx = *(const i4*)xr, nw = *(const i4*)wr;
    for (long long k = 0; k < p.width; k += 64) {
        __syncthreads();
        s_x[r][c ^ ((r >> 1) & 3)] = nx;
        s_w[r][c ^ ((r >> 1) & 3)] = nw;
        __syncthreads();
        if (k + 64 < p.width) {
            nx = *(const i4*)(xr + k + 64);
            nw = *(const i4*)(wr + k + 64);
        }
        i4 fx[2], fw[2];
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const int a = wm + i * 16 + i16, b = wn + i * 16 + i16;
            fx[i] = s_x[a][q ^ ((a >> 1) & 3)];
            fw[i] = s_w[b][q ^ ((b >> 1) & 3)];
        }
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
            for (int j = 0; j < 2; ++j) acc[i][j] = __builtin_amdgcn_mfma_i32_16x16x64_i8(fw[j], fx[i], acc[i][j], 0, 0, 0);
    }
    // lane: row m = lane % 16, columns n = 4 (lane / 16) .. + 3 of each block
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const long long m = m0 + wm + i * 16 + i16;
        if (m >= m_end) continue;
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            const long long n = n0 + wn + j * 16 + 4 * q;
            if (n < p.n) finish4<T>(p, m, n, acc[i][j]);
        }
    }
}

// ------------------------------------------------------------------ host side
template <typename T>
static hipError_t quantize(const void* x, long long rows, const long long* rows_dev, long long channels, signed char* q, float* scale,
                           hipStream_t s) {
    const long long width = int8_width(channels);
    hipLaunchKernelGGL((k_quantize_rows<T, 256, 4>), grid_of<256>(rows), dim3(256), 0, s, (const T*)x, rows, rows_dev, channels, width,
                       q, scale);
    return hipGetLastError();
}

hipError_t launch_quantize_rows(int dtype, const void* x, long long rows, const long long* rows_dev, long long channels,
                                signed char* q, float* scale, hipStream_t s) {
    switch (dtype) {
        case SCNN_F32: return quantize<float>(x, rows, rows_dev, channels, q, scale, s);
        case SCNN_BF16: return quantize<__bf16>(x, rows, rows_dev, channels, q, scale, s);
        default: return quantize<_Float16>(x, rows, rows_dev, channels, q, scale, s);
    }
}

template <typename T>
static hipError_t quantize_weight(const void* w, long long c_in, long long c_out, signed char* q, float* scale, hipStream_t s) {
    hipLaunchKernelGGL((k_quantize_weight<T>), grid_of<1024>((c_out + 31) / 32), dim3(1024), 0, s, (const T*)w, c_in, c_out,
                       int8_width(c_in), q, scale);
    return hipGetLastError();
}

hipError_t launch_quantize_weight(int dtype, const void* w, long long c_in, long long c_out, signed char* q, float* scale,
                                  hipStream_t s) {
    switch (dtype) {
        case SCNN_F32: return quantize_weight<float>(w, c_in, c_out, q, scale, s);
        case SCNN_BF16: return quantize_weight<__bf16>(w, c_in, c_out, q, scale, s);
        default: return quantize_weight<_Float16>(w, c_in, c_out, q, scale, s);
    }
}

struct Int8Space { size_t q, scale, total; };
static Int8Space int8_space(bool given, long long rows, long long c_in) {
    Int8Space a = {};
    if (given) return a;
    a.scale = (size_t)round_up(rows * int8_width(c_in), 256);
    a.total = a.scale + (size_t)round_up(rows * 4, 256);
    return a;
}
size_t linear_int8_bytes(int dtype, bool given, long long rows, long long c_in, long long c_out) {
    return int8_space(given, rows, c_in).total;
}

template <typename T>
static hipError_t linear_int8(int dtype, const Int8Call& c, hipStream_t s) {
    Int8Args p = {};
    const Int8Space at = int8_space(c.x_scale != nullptr, c.rows, c.c_in);
    p.x = (const signed char*)c.x;
    p.x_scale = c.x_scale;
    if (!c.x_scale) {
        signed char* const q = (signed char*)c.workspace + at.q;
        float* const scale = (float*)((char*)c.workspace + at.scale);
        const hipError_t e = quantize<T>(c.x, c.rows, c.rows_dev, c.c_in, q, scale, s);
        if (e != hipSuccess) return e;
        p.x = q;
        p.x_scale = scale;
    }
    p.w = c.w; p.w_scale = c.w_scale; p.bias = c.bias; p.residual = c.residual; p.out = c.out;
    p.m = c.rows; p.n = c.c_out; p.width = int8_width(c.c_in);
    p.rows_dev = c.rows_dev;
    p.act = c.act;
    const long long tiles = ((p.m + 63) / 64) * ((p.n + 63) / 64);
    hipLaunchKernelGGL((k_int8_tile<T>), grid_of<256>(tiles), dim3(256), 0, s, p);
    return hipGetLastError();
}

hipError_t launch_linear_int8(int dtype, const Int8Call& c, hipStream_t s) {
    switch (dtype) {
        case SCNN_F32: return linear_int8<float>(dtype, c, s);
        case SCNN_BF16: return linear_int8<__bf16>(dtype, c, s);
        default: return linear_int8<_Float16>(dtype, c, s);
    }
}

}  // namespace scnn
