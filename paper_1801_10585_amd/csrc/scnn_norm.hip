// Layer norm over the channels of rows [rows, C], forward and backward.
//
//   mean = sum_c x / C,  var = sum_c (x - mean)^2 / C,  rstd = 1 / sqrt(var + eps),  xh = (x - mean) rstd
//   out = xh gamma + beta
//   h = g gamma,  dx = rstd (h - sum_c(h) / C - xh sum_c(h xh) / C),  dgamma = sum_r g xh,  dbeta = sum_r g
//
// Both directions are bound by memory: a row is read once and kept in registers between its sums and its result (the
// deviations are summed around the mean that is already known, so nothing cancels).  The mean is summed and divided in fp64, and
// what its rounding to fp32 leaves is taken off every deviation too (64 channels around 10^4 with deviations of 1: 4e-7 off;
// 6e-4 without); a row of equal values, however large, has deviations of exactly 0.  The other sums are fp32.  The sums over rows
// behind dgamma and dbeta are formed a column a lane in registers while the rows go by, joined within the workgroup, and
// the workgroups' sums are added by a second launch in a fixed order: no atomics, the same bits every time.
// Forward: 643072 x 64 fp32 64 us (5.2 TB/s, as a large copy), 8192 x 4096 fp32 51 (5.2 TB/s).  Backward: 643072 x 64 fp32 104
// (4.8), 8192 x 4096 bf16 37 + 4 for the second launch (4.6), 209645 x 25 fp32 14.5 + 4 (3.5: vectors of rows of 100 bytes).
#include "scnn_dense.h"

namespace scnn {

// P threads hold a row (a group of lanes of a wave, or whole waves from 256 on), VPL 16-byte vectors each.
template <int P> constexpr int kNormBlock = P <= 64 ? 256 : P;
// The backward pass takes four rows of 256 threads at once: sixteen waves of loads in flight, and one set of sums.
template <int P> constexpr int kBackBlock = P <= 64 ? 256 : 1024;

// Sum over the P threads of a row.  Up to 64: lane exchanges.  Else s_part holds a value a wave of the workgroup, all of
// whose threads call it; two arrays in turn make one barrier a sum enough.
template <int P, typename F>
__device__ __forceinline__ F row_add(F v, F* s_part) {
    if constexpr (P <= 64) {
        return lanes_add<P>(v);
    } else {
        v = lanes_add<64>(v);
        if ((threadIdx.x & 63) == 0) s_part[threadIdx.x >> 6] = v;
        __syncthreads();
        F t = 0;
#pragma unroll
        for (int i = 0; i < P / 64; ++i) t += s_part[threadIdx.x / P * (P / 64) + i];
        return t;
    }
}

// Mean of a row from its sum: to nearest in fp64 (one step of Newton's after the product with 1 / C: exact where the quotient
// is a double, as in rows of equal values), as a float and what that leaves.
__device__ __forceinline__ float row_mean(double sum, double channels, double inv_c, float& rest) {
    double q = sum * inv_c;
    const double off = __builtin_fma(-q, channels, sum);
    if (off == off) q = __builtin_fma(off, inv_c, q);  // (an infinity stays one)
    const float mean = (float)q;
    rest = (float)(q - (double)mean);
    return mean;
}

template <typename T, int P, int VPL, bool TAIL>
__global__ __launch_bounds__(kNormBlock<P>) void k_norm_fwd(const T* __restrict__ x, long long rows_cap,
                                                            const long long* __restrict__ rows_dev, int channels,
                                                            const T* __restrict__ gamma, const T* __restrict__ beta,
                                                            float eps, T* __restrict__ out, float* __restrict__ mean_out,
                                                            float* __restrict__ rstd_out) {
    constexpr int V = kVec<T>, G = kNormBlock<P> / P;
    __shared__ float s_part[P <= 64 ? 1 : P / 64];
    __shared__ double s_mean[P <= 64 ? 1 : P / 64];
    const long long rows = rows_of(rows_cap, rows_dev);
    const bool whole = channels >= kVec<T>;
    const int t = threadIdx.x % P;
    const float inv_c = 1.0f / (float)channels;
    const double inv_c64 = 1.0 / (double)channels;
    for (long long row = (long long)blockIdx.x * G + threadIdx.x / P; row < rows; row += (long long)gridDim.x * G) {
        const T* __restrict__ xr = x + row * channels;
        float v[VPL][V];
        double sum = 0.0;
#pragma unroll
        for (int j = 0; j < VPL; ++j) {
            const int c = (j * P + t) * V;
            load_elems<T, TAIL>(xr + c, channels - c, whole, v[j]);
#pragma unroll
            for (int i = 0; i < V; ++i) sum += (double)v[j][i];
        }
        float rest;
        const float mean = row_mean(row_add<P>(sum, s_mean), (double)channels, inv_c64, rest);
        float sq = 0.0f;
#pragma unroll
        for (int j = 0; j < VPL; ++j) {
            const int c = (j * P + t) * V;
#pragma unroll
            for (int i = 0; i < V; ++i) {
                v[j][i] = c + i < channels ? (v[j][i] - mean) - rest : 0.0f;
                sq += v[j][i] * v[j][i];
            }
        }
        const float rstd = 1.0f / sqrtf(row_add<P>(sq, s_part) * inv_c + eps);
        T* __restrict__ yr = out + row * channels;
#pragma unroll
        for (int j = 0; j < VPL; ++j) {
            const int c = (j * P + t) * V;
            float ga[V], be[V];
            if (gamma) load_elems<T, TAIL>(gamma + c, channels - c, whole, ga);
            if (beta) load_elems<T, TAIL>(beta + c, channels - c, whole, be);
#pragma unroll
            for (int i = 0; i < V; ++i) {
                v[j][i] *= rstd;
                if (gamma) v[j][i] *= ga[i];
                if (beta) v[j][i] += be[i];
            }
            store_elems<T, TAIL>(yr + c, channels - c, v[j]);
        }
        if (t == 0) {
            if (mean_out) mean_out[row] = mean;
            if (rstd_out) rstd_out[row] = rstd;
        }
    }
}

// Rows too long for a workgroup's registers: read three times, the second and third time mostly from the L2.
template <typename T>
__global__ __launch_bounds__(1024) void k_norm_fwd_long(const T* __restrict__ x, long long rows_cap,
                                                        const long long* __restrict__ rows_dev, int channels,
                                                        const T* __restrict__ gamma, const T* __restrict__ beta, float eps,
                                                        T* __restrict__ out, float* __restrict__ mean_out,
                                                        float* __restrict__ rstd_out) {
    constexpr int V = kVec<T>, P = 1024;
    __shared__ float s_part[P / 64];
    __shared__ double s_mean[P / 64];
    const long long rows = rows_of(rows_cap, rows_dev);
    const bool whole = channels >= kVec<T>;
    const float inv_c = 1.0f / (float)channels;
    const double inv_c64 = 1.0 / (double)channels;
    for (long long row = blockIdx.x; row < rows; row += gridDim.x) {
        const T* __restrict__ xr = x + row * channels;
        T* __restrict__ yr = out + row * channels;
        double sum = 0.0;
        float sq = 0.0f;
        for (long long c = (long long)threadIdx.x * V; c < channels; c += P * V) {
            float v[V];
            load_elems<T>(xr + c, channels - (int)c, whole, v);
#pragma unroll
            for (int i = 0; i < V; ++i) sum += (double)v[i];
        }
        float rest;
        const float mean = row_mean(row_add<P>(sum, s_mean), (double)channels, inv_c64, rest);
        for (long long c = (long long)threadIdx.x * V; c < channels; c += P * V) {
            float v[V];
            load_elems<T>(xr + c, channels - (int)c, whole, v);
#pragma unroll
            for (int i = 0; i < V; ++i) {
                const float d = c + i < channels ? (v[i] - mean) - rest : 0.0f;
                sq += d * d;
            }
        }
        const float rstd = 1.0f / sqrtf(row_add<P>(sq, s_part) * inv_c + eps);
        for (long long c = (long long)threadIdx.x * V; c < channels; c += P * V) {
            const int n = channels - (int)c;
            float v[V], ga[V], be[V];
            load_elems<T>(xr + c, n, whole, v);
            if (gamma) load_elems<T>(gamma + c, n, whole, ga);
            if (beta) load_elems<T>(beta + c, n, whole, be);
#pragma unroll
            for (int i = 0; i < V; ++i) {
                v[i] = ((v[i] - mean) - rest) * rstd;
                if (gamma) v[i] *= ga[i];
                if (beta) v[i] += be[i];
            }
            store_elems<T>(yr + c, n, v);
        }
        if (threadIdx.x == 0) {
            if (mean_out) mean_out[row] = mean;
            if (rstd_out) rstd_out[row] = rstd;
        }
    }
}

// part [gridDim.x][2][channels]: this workgroup's sums of g xh and of g (not written where part is null).
template <typename T, int P, int VPL, bool TAIL>
__global__ __launch_bounds__(kBackBlock<P>) void k_norm_bwd(const T* __restrict__ x, const T* __restrict__ g,
                                                            long long rows_cap, const long long* __restrict__ rows_dev,
                                                            int channels, const T* __restrict__ gamma,
                                                            const float* __restrict__ mean_in,
                                                            const float* __restrict__ rstd_in, T* __restrict__ dx,
                                                            float* __restrict__ part) {
    constexpr int V = kVec<T>, B = kBackBlock<P>, G = B / P;
    typedef float f2 __attribute__((ext_vector_type(2)));
    __shared__ f2 s_part[2][P <= 64 ? 1 : B / 64];
    const long long rows = rows_of(rows_cap, rows_dev);
    const bool whole = channels >= kVec<T>;
    const int t = threadIdx.x % P, group = threadIdx.x / P;
    const float inv_c = 1.0f / (float)channels;
    float d_gamma[VPL][V], d_beta[VPL][V];
    VecOf<T, V> ga[VPL];
#pragma unroll
    for (int j = 0; j < VPL; ++j) {
        const int c = (j * P + t) * V;
        ga[j] = VecOf<T, V>{};
        if (gamma) ga[j] = load_raw<T, TAIL>(gamma + c, channels - c, whole);
#pragma unroll
        for (int i = 0; i < V; ++i) d_gamma[j][i] = d_beta[j][i] = 0.0f;
    }
    int turn = 0;
    // Rows as they lie in memory (half the registers with 16-bit types), the next one on its way while this one is summed
    // where the registers last.
    constexpr bool AHEAD = VPL == 1;
    VecOf<T, V> xr[VPL], gr[VPL], x_next[VPL], g_next[VPL];
    float mean_next = 0.0f, rstd_next = 0.0f;
    auto fetch = [&](long long row) {
        const bool live = row < rows;
        if (live) {
            mean_next = mean_in[row];
            rstd_next = rstd_in[row];
        }
#pragma unroll
        for (int j = 0; j < VPL; ++j) {
            const int c = (j * P + t) * V;
            x_next[j] = load_raw<T, TAIL>(x + row * channels + c, live ? channels - c : 0, whole);
            g_next[j] = load_raw<T, TAIL>(g + row * channels + c, live ? channels - c : 0, whole);
        }
    };
    if (AHEAD) fetch((long long)blockIdx.x * G + group);
    // (all groups of the workgroup go round together: row_add holds a barrier)
    for (long long row0 = (long long)blockIdx.x * G; row0 < rows; row0 += (long long)gridDim.x * G, turn ^= 1) {
        const long long row = row0 + group;
        const bool live = row < rows;
        if (!AHEAD) fetch(row);
        const float mean = mean_next, rstd = rstd_next;
        f2 sums = {0.0f, 0.0f};
#pragma unroll
        for (int j = 0; j < VPL; ++j) {
            xr[j] = x_next[j];
            gr[j] = g_next[j];
        }
        if (AHEAD) fetch(row + (long long)gridDim.x * G);
#pragma unroll
        for (int j = 0; j < VPL; ++j)
#pragma unroll
            for (int i = 0; i < V; ++i) {
                // (past the row's end g is 0, and so is everything below)
                const float xh = (j * P + t) * V + i < channels ? ((float)xr[j][i] - mean) * rstd : 0.0f;
                const float gi = (float)gr[j][i], h = gamma ? gi * (float)ga[j][i] : gi;
                d_gamma[j][i] += gi * xh;
                d_beta[j][i] += gi;
                sums.x += h;
                sums.y += h * xh;
            }
        if (!dx) continue;
        sums = row_add<P>(sums, s_part[turn]) * inv_c;
        if constexpr (sizeof(T) == 2) {
            // the compiler would keep the products of the first half in twice the registers: it may not know these values
            // any more
#pragma unroll
            for (int j = 0; j < VPL; ++j) asm volatile("" : "+v"(xr[j]), "+v"(gr[j]));
        }
        if (live)
#pragma unroll
            for (int j = 0; j < VPL; ++j) {
                const int c = (j * P + t) * V;
                float v[V];
#pragma unroll
                for (int i = 0; i < V; ++i) {
                    const float gi = (float)gr[j][i], h = gamma ? gi * (float)ga[j][i] : gi;
                    v[i] = rstd * (h - sums.x - ((float)xr[j][i] - mean) * rstd * sums.y);
                }
                store_elems<T, TAIL>(dx + row * channels + c, channels - c, v);
            }
    }
    if (!part) return;
    float* __restrict__ mine = part + (long long)blockIdx.x * 2 * channels;
    // the rows of a wave by lane exchanges, those of different waves in LDS
    constexpr int L = P <= 64 ? 4 : G;
    __shared__ float s_col[L][P * V];
    const int set = P <= 64 ? threadIdx.x >> 6 : group;
#pragma unroll
    for (int j = 0; j < VPL; ++j)
#pragma unroll
        for (int k = 0; k < 2; ++k) {
            __syncthreads();
#pragma unroll
            for (int i = 0; i < V; ++i) {
                float a = k ? d_beta[j][i] : d_gamma[j][i];
                if constexpr (P < 64)
#pragma unroll
                    for (int d = P; d < 64; d <<= 1) a += __shfl_xor(a, d, 64);
                if (P > 64 || (threadIdx.x & 63) < P) s_col[set][t * V + i] = a;
            }
            __syncthreads();
            for (int c = threadIdx.x; c < P * V; c += B) {
                const int cc = j * P * V + c;
                if (cc >= channels) break;
                float sum = s_col[0][c];
#pragma unroll
                for (int q = 1; q < L; ++q) sum += s_col[q][c];
                mine[(long long)k * channels + cc] = sum;
            }
        }
}

// dx of rows too long for a workgroup's registers; their dgamma and dbeta come from k_norm_cols_long.
template <typename T>
__global__ __launch_bounds__(1024) void k_norm_bwd_long(const T* __restrict__ x, const T* __restrict__ g,
                                                        long long rows_cap, const long long* __restrict__ rows_dev,
                                                        int channels, const T* __restrict__ gamma,
                                                        const float* __restrict__ mean_in,
                                                        const float* __restrict__ rstd_in, T* __restrict__ dx) {
    constexpr int V = kVec<T>, P = 1024;
    __shared__ float s_part[2][P / 64];
    const long long rows = rows_of(rows_cap, rows_dev);
    const bool whole = channels >= kVec<T>;
    const float inv_c = 1.0f / (float)channels;
    for (long long row = blockIdx.x; row < rows; row += gridDim.x) {
        const float mean = mean_in[row], rstd = rstd_in[row];
        const T* __restrict__ xr = x + row * channels;
        const T* __restrict__ gr = g + row * channels;
        float s_h = 0.0f, s_hx = 0.0f;
        for (int pass = 0; pass < 2; ++pass) {
            float m_h = 0.0f, m_hx = 0.0f;
            if (pass) {
                m_h = row_add<P>(s_h, s_part[0]) * inv_c;
                m_hx = row_add<P>(s_hx, s_part[1]) * inv_c;
            }
            for (long long c = (long long)threadIdx.x * V; c < channels; c += P * V) {
                const int n = channels - (int)c;
                float v[V], h[V], ga[V];
                load_elems<T>(xr + c, n, whole, v);
                load_elems<T>(gr + c, n, whole, h);
                if (gamma) load_elems<T>(gamma + c, n, whole, ga);
#pragma unroll
                for (int i = 0; i < V; ++i) {
                    v[i] = i < n ? (v[i] - mean) * rstd : 0.0f;
                    if (gamma) h[i] *= ga[i];
                    if (pass) {
                        h[i] = rstd * (h[i] - m_h - v[i] * m_hx);
                    } else {
                        s_h += h[i];
                        s_hx += h[i] * v[i];
                    }
                }
                if (pass) store_elems<T>(dx + row * channels + c, n, h);
            }
        }
    }
}

// part [gridDim.y][2][channels]: column sums of g xh and g over this workgroup's rows, a vector of columns a thread.
template <typename T>
__global__ __launch_bounds__(256) void k_norm_cols_long(const T* __restrict__ x, const T* __restrict__ g, long long rows_cap,
                                                        const long long* __restrict__ rows_dev, int channels,
                                                        const float* __restrict__ mean_in,
                                                        const float* __restrict__ rstd_in, float* __restrict__ part) {
    constexpr int V = kVec<T>;
    const long long rows = rows_of(rows_cap, rows_dev);
    const bool whole = channels >= kVec<T>;
    const long long c = ((long long)blockIdx.x * 256 + threadIdx.x) * V;
    if (c >= channels) return;
    const int n = channels - (int)c;
    float d_gamma[V], d_beta[V];
#pragma unroll
    for (int i = 0; i < V; ++i) d_gamma[i] = d_beta[i] = 0.0f;
    for (long long row = blockIdx.y; row < rows; row += gridDim.y) {
        const float mean = mean_in[row], rstd = rstd_in[row];
        float v[V], h[V];
        load_elems<T>(x + row * channels + c, n, whole, v);
        load_elems<T>(g + row * channels + c, n, whole, h);
#pragma unroll
        for (int i = 0; i < V; ++i) {
            d_gamma[i] += i < n ? h[i] * ((v[i] - mean) * rstd) : 0.0f;
            d_beta[i] += h[i];
        }
    }
    float* __restrict__ mine = part + (long long)blockIdx.y * 2 * channels;
#pragma unroll
    for (int i = 0; i < V; ++i)
        if (i < n) {
            mine[c + i] = d_gamma[i];
            mine[channels + c + i] = d_beta[i];
        }
}

// Sixteen columns a workgroup, 64 threads a column, each over every 64th part; their sums joined in order.  (The parts are
// some hundred to two thousand; with sixteen threads a column 820 parts took 13.7 us, a load behind the other.)
template <typename T>
__global__ __launch_bounds__(1024) void k_column_sums(const float* __restrict__ part, int parts, long long cols,
                                                      long long split, T* __restrict__ out0, T* __restrict__ out1) {
    __shared__ double s_sum[64][17];
    const int tc = threadIdx.x & 15, tp = threadIdx.x >> 4;
    const long long c = block_id<1024>() * 16 + tc;
    double sum = 0.0;
    if (c < cols)
#pragma unroll 8
        for (int p = tp; p < parts; p += 64) sum += (double)part[(long long)p * cols + c];
    s_sum[tp][tc] = sum;
    __syncthreads();
#pragma unroll
    for (int d = 32; d >= 4; d >>= 1) {
        if (tp < d) s_sum[tp][tc] += s_sum[tp + d][tc];
        __syncthreads();
    }
    if (tp != 0 || c >= cols) return;
    sum = (s_sum[0][tc] + s_sum[1][tc]) + (s_sum[2][tc] + s_sum[3][tc]);
    if (c < split) {
        if (out0) out0[c] = (T)(float)sum;
    } else if (out1) {
        out1[c - split] = (T)(float)sum;
    }
}

template <typename T>
static hipError_t column_sums(const float* part, int parts, long long cols, long long split, void* out0, void* out1,
                              hipStream_t s) {
    hipLaunchKernelGGL((k_column_sums<T>), grid_of<1024>((cols + 15) / 16), dim3(1024), 0, s, part, parts, cols, split,
                       (T*)out0, (T*)out1);
    return hipGetLastError();
}

hipError_t launch_column_sums(const float* part, int parts, long long cols, long long split, void* out0, void* out1,
                              int dtype, hipStream_t s) {
    if (cols < 1 || (!out0 && !out1)) return hipSuccess;
    switch (dtype) {
        case SCNN_F32: return column_sums<float>(part, parts, cols, split, out0, out1, s);
        case SCNN_BF16: return column_sums<__bf16>(part, parts, cols, split, out0, out1, s);
        default: return column_sums<_Float16>(part, parts, cols, split, out0, out1, s);
    }
}

static int dtype_vec(int dtype) { return dtype == SCNN_F32 ? 4 : 8; }

// Threads a row and vectors a thread: one vector a lane up to a wave; then, where rows are many, more vectors a lane before
// more waves a row, which meet at a barrier for every sum (forward, 8192 rows of 8192 bf16, 256 threads of four vectors
// against 1024 of one: 56 / 84 us); where they are few, and in the backward pass, whose sums of columns take the registers,
// more waves.  p = 0: longer rows than these hold.
struct NormShape { int p, vpl; };
static NormShape norm_shape(int channels, int dtype, long long rows, bool forward) {
    const int units = (int)(((long long)channels + dtype_vec(dtype) - 1) / dtype_vec(dtype));
    for (int p = 1; p <= 64; p <<= 1)
        if (units <= p) return {p, 1};
    if (units <= 128) return {64, 2};
    if (forward && rows >= 8LL * device_cu_count()) {
        if (units <= 256) return {64, 4};
        if (units <= 512) return {256, 2};
        if (units <= 1024) return {256, 4};
    }
    if (units <= 256) return {256, 1};
    if (units <= 512) return {512, 1};
    if (units <= 1024) return {1024, 1};
    if (units <= 2048) return {1024, 2};
    if (units <= 4096 && forward) return {1024, 4};
    return {0, 0};
}

// Workgroups of the backward pass.  Each leaves 2 * channels sums, written and read again in fp32: at most about a sixteenth
// of the bytes that the rows take in and out, but enough to fill the card with one workgroup a compute unit, and no more
// than four of four waves.
static int norm_parts(long long rows, int channels, int dtype) {
    const NormShape n = norm_shape(channels, dtype, rows, false);
    const long long cus = device_cu_count();
    if (n.p == 0) return (int)(rows < 1 ? 1 : (rows < cus ? rows : cus));
    const long long per = (n.p <= 64 ? 256 : 1024) / n.p;
    const long long e = dtype == SCNN_F32 ? 4 : 2;
    long long parts = rows * 3 * e / (16 * 16);
    if (parts > 4 * cus) parts = 4 * cus;
    if (n.p > 64) parts = cus;
    if (parts < cus) parts = cus;
    const long long need = (rows + per - 1) / per;
    if (parts > need) parts = need;
    return (int)(parts < 1 ? 1 : parts);
}

size_t norm_bwd_part_bytes(long long rows, int channels, int dtype) {
    return (size_t)norm_parts(rows, channels, dtype) * 2 * (size_t)channels * sizeof(float);
}

#define SCNN_NORM_SHAPES(F)                                                                                             \
    F(1, 1) F(2, 1) F(4, 1) F(8, 1) F(16, 1) F(32, 1) F(64, 1) F(64, 2) F(256, 1) F(512, 1) F(1024, 1) F(1024, 2)

template <typename T>
static hipError_t norm_fwd(const void* x, long long rows, const long long* rows_dev, int channels, const void* gamma,
                           const void* beta, float eps, void* out, float* mean, float* rstd, int dtype, hipStream_t s) {
    const NormShape n = norm_shape(channels, dtype, rows, true);
    const bool tail = channels % kVec<T> != 0;  // (code for a row's last elements costs registers)
    const long long per = n.p > 0 && n.p <= 64 ? 256 / n.p : 1;
    const int threads = n.p == 0 ? 1024 : (n.p <= 64 ? 256 : n.p);
    long long blocks = (rows + per - 1) / per;
    const long long most = (long long)device_cu_count() * (2048 / threads);
    if (blocks > most) blocks = most;
#define F(P, VPL)                                                                                                      \
    if (n.p == P && n.vpl == VPL)                                                                                      \
        hipLaunchKernelGGL((tail ? k_norm_fwd<T, P, VPL, true> : k_norm_fwd<T, P, VPL, false>), dim3((unsigned)blocks),   \
                           dim3(kNormBlock<P>), 0, s, (const T*)x, rows, rows_dev, channels, (const T*)gamma,            \
                           (const T*)beta, eps, (T*)out, mean, rstd);
    SCNN_NORM_SHAPES(F) F(64, 4) F(256, 2) F(256, 4) F(1024, 4)
#undef F
    if (n.p == 0)
        hipLaunchKernelGGL((k_norm_fwd_long<T>), dim3((unsigned)blocks), dim3(1024), 0, s, (const T*)x, rows, rows_dev,
                           channels, (const T*)gamma, (const T*)beta, eps, (T*)out, mean, rstd);
    return hipGetLastError();
}

hipError_t launch_norm_fwd(const void* x, long long rows, const long long* rows_dev, int channels, const void* gamma,
                           const void* beta, float eps, void* out, float* mean, float* rstd, int dtype, hipStream_t s) {
    if (rows < 1) return hipSuccess;
    switch (dtype) {
        case SCNN_F32: return norm_fwd<float>(x, rows, rows_dev, channels, gamma, beta, eps, out, mean, rstd, dtype, s);
        case SCNN_BF16: return norm_fwd<__bf16>(x, rows, rows_dev, channels, gamma, beta, eps, out, mean, rstd, dtype, s);
        default: return norm_fwd<_Float16>(x, rows, rows_dev, channels, gamma, beta, eps, out, mean, rstd, dtype, s);
    }
}

template <typename T>
static hipError_t norm_bwd(const void* x, const void* g, long long rows, const long long* rows_dev, int channels,
                           const void* gamma, const float* mean, const float* rstd, void* dx, void* dgamma, void* dbeta,
                           float* part, int dtype, hipStream_t s) {
    const NormShape n = norm_shape(channels, dtype, rows, false);
    const bool tail = channels % kVec<T> != 0;
    const int parts = norm_parts(rows, channels, dtype);
    float* const sums = dgamma || dbeta ? part : nullptr;
#define F(P, VPL)                                                                                                      \
    if (n.p == P && n.vpl == VPL)                                                                                      \
        hipLaunchKernelGGL((tail ? k_norm_bwd<T, P, VPL, true> : k_norm_bwd<T, P, VPL, false>), dim3((unsigned)parts),    \
                           dim3(kBackBlock<P>), 0, s, (const T*)x, (const T*)g, rows, rows_dev, channels,                \
                           (const T*)gamma, mean, rstd, (T*)dx, sums);
    SCNN_NORM_SHAPES(F)
#undef F
    if (n.p == 0) {
        if (dx) {
            const long long blocks = rows < 2 * device_cu_count() ? (rows < 1 ? 1 : rows) : 2 * device_cu_count();
            hipLaunchKernelGGL((k_norm_bwd_long<T>), dim3((unsigned)blocks), dim3(1024), 0, s, (const T*)x, (const T*)g,
                               rows, rows_dev, channels, (const T*)gamma, mean, rstd, (T*)dx);
        }
        if (sums) {
            const int wide = 256 * dtype_vec(dtype);
            hipLaunchKernelGGL((k_norm_cols_long<T>), dim3((unsigned)(((long long)channels + wide - 1) / wide), (unsigned)parts),
                               dim3(256), 0, s, (const T*)x, (const T*)g, rows, rows_dev, channels, mean, rstd, sums);
        }
    }
    hipError_t e = hipGetLastError();
    if (e != hipSuccess || !sums) return e;
    return launch_column_sums(sums, parts, 2LL * channels, channels, dgamma, dbeta, dtype, s);
}

hipError_t launch_norm_bwd(const void* x, const void* g, long long rows, const long long* rows_dev, int channels,
                           const void* gamma, const float* mean, const float* rstd, void* dx, void* dgamma, void* dbeta,
                           float* part, int dtype, hipStream_t s) {
    switch (dtype) {
        case SCNN_F32:
            return norm_bwd<float>(x, g, rows, rows_dev, channels, gamma, mean, rstd, dx, dgamma, dbeta, part, dtype, s);
        case SCNN_BF16:
            return norm_bwd<__bf16>(x, g, rows, rows_dev, channels, gamma, mean, rstd, dx, dgamma, dbeta, part, dtype, s);
        default:
            return norm_bwd<_Float16>(x, g, rows, rows_dev, channels, gamma, mean, rstd, dx, dgamma, dbeta, part, dtype, s);
    }
}

}  // namespace scnn
