// Linear layers in 8-bit integers, for serving: out = act(z) + residual with z = (sum_k q[r, k] w[n, k]) x_scale[r] w_scale[n] + bias.
//
//   most = max(max_k |x[r, k]|, 2^-100),  x_scale[r] = most / 127,  q[r, k] = x[r, k] (127 / most) rounded to nearest even
// (fp32, both quotients rounded once), the same for the columns of a layer's weights, laid out as rows.  A row that holds a NaN
// or an infinity has scale NaN and q 0, so that its results are NaN.
//
// The sums are exact: 32-bit integers, |q w| <= 2^14 and fewer than 2^17 of them.  Rows of 8-bit values are filled up with zeros to
// a multiple of 64, so that every row begins on 64 bytes and k needs no ends.
#include "scnn_tiles.h"

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

// P threads a row (a group of lanes of a wave, or a workgroup of whole waves), H vectors of the row in a thread's registers; what a
// longer row has more is read again.  Bound by memory, one reading of rows of up to 2 P vectors: 8192 x 4096 bf16 19 us (5.3 TB/s),
// 200000 x 64 bf16 8.4 us by 4 threads a row (16.4 by 16), 64 x 12288 fp16 4.2 us by 1024.
template <typename T, int P, int H>
__global__ __launch_bounds__(P < 256 ? 256 : P) void k_quantize_rows(const T* __restrict__ x, long long rows_cap,
                                                                     const long long* __restrict__ rows_dev, long long channels,
                                                                     long long width, signed char* __restrict__ out,
                                                                     float* __restrict__ scale) {
    constexpr int V = kVec<T>, B = P < 256 ? 256 : P, G = B / P;
    typedef signed char Q __attribute__((ext_vector_type(V)));
    __shared__ unsigned s_most[B / 64];
    const int t = threadIdx.x % P;
    const long long rows = rows_of(rows_cap, rows_dev), row = block_id<B>() * G + threadIdx.x / P;
    const bool live = row < rows, whole = channels >= V;
    const T* __restrict__ xr = x + row * channels;
    VecOf<T, V> held[H];
    unsigned most = 0;
    auto at = [&](long long j) { return (j * P + t) * V; };
    auto take = [&](long long c) {
        const long long n = live ? channels - c : 0;
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
#pragma unroll
    for (int d = 1; d < (P < 64 ? P : 64); d <<= 1) {
        const unsigned o = __shfl_xor(most, d, 64);
        most = o > most ? o : most;
    }
    if constexpr (P > 64) {
        if ((threadIdx.x & 63) == 0) s_most[threadIdx.x >> 6] = most;
        __syncthreads();
#pragma unroll
        for (int k = 0; k < P / 64; ++k) most = s_most[k] > most ? s_most[k] : most;
    }
    if (!live) return;
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
    if (t == 0) scale[row] = q.scale;
}

// Once for a layer.  32 columns of w [c_in, c_out] a workgroup, V of a row a thread: their largest magnitudes, then k_span rows of them as
// rows of q by way of LDS; workgroups along y each look at all of the columns, which the L2 has by then.  12288 x 1024 bf16 30 us (one
// workgroup a strip, value by value: 203).
template <typename T>
__global__ __launch_bounds__(1024) void k_quantize_weight(const T* __restrict__ w, long long c_in, long long c_out, long long width,
                                                          long long k_span, signed char* __restrict__ out, float* __restrict__ scale) {
    constexpr int V = kVec<T>, C = 32, TR = C / V, R = 1024 / TR, B = R / 32;  // R rows a step, B bytes of q a thread
    typedef signed char Q __attribute__((ext_vector_type(B)));
    __shared__ unsigned s_most[16][C];
    __shared__ float s_inverse[C];
    __shared__ __align__(16) signed char s_q[C][R + 16];
    const int tid = threadIdx.x, lane = tid & 63, tc = tid % TR * V, tr = tid / TR;
    const long long c0 = block_id<1024>() * C;
    if (c0 >= c_out) return;
    const int n = (int)(c_out - c0 - tc < V ? c_out - c0 - tc : V);  // (0 and less: no column of this thread's is there)
    const T* __restrict__ from = w + c0 + tc;
    auto take = [&](long long k) { return load_raw<T>(from + k * c_out, n, c_out >= V); };
    unsigned most[V] = {};
    for (long long k = tr; k < c_in; k += 4 * R) {
        VecOf<T, V> v[4];
#pragma unroll
        for (int u = 0; u < 4; ++u) v[u] = take(k + u * R < c_in ? k + u * R : k);
#pragma unroll
        for (int u = 0; u < 4; ++u)
#pragma unroll
            for (int i = 0; i < V; ++i) {
                const unsigned m = magnitude((float)v[u][i]);
                most[i] = m > most[i] ? m : most[i];
            }
    }
#pragma unroll
    for (int i = 0; i < V; ++i) {
#pragma unroll
        for (int d = TR; d < 64; d <<= 1) {
            const unsigned o = __shfl_xor(most[i], d, 64);
            most[i] = o > most[i] ? o : most[i];
        }
        if (lane < TR) s_most[tid >> 6][tc + i] = most[i];
    }
    __syncthreads();
    if (tid < C) {
        unsigned m = 0;
#pragma unroll
        for (int k = 0; k < 16; ++k) m = s_most[k][tid] > m ? s_most[k][tid] : m;
        const Quantizer q = quantizer(m);
        s_inverse[tid] = q.inverse;
        if (blockIdx.y == 0 && c0 + tid < c_out) scale[c0 + tid] = q.scale;
    }
    __syncthreads();
    Quantizer q[V];
#pragma unroll
    for (int i = 0; i < V; ++i) q[i].inverse = s_inverse[tc + i];
    const long long k_first = (long long)blockIdx.y * k_span, k_end = k_first + k_span < width ? k_first + k_span : width;
    VecOf<T, V> next = {};
    if (k_first + tr < c_in) next = take(k_first + tr);
    for (long long k0 = k_first; k0 < k_end; k0 += R) {
#pragma unroll
        for (int i = 0; i < V; ++i) s_q[tc + i][tr] = (signed char)quantized((float)next[i], q[i]);
        next = VecOf<T, V>{};
        if (k0 + R + tr < c_in) next = take(k0 + R + tr);
        __syncthreads();
        const int col = tid >> 5, at = (tid & 31) * B;
        if (c0 + col < c_out && k0 + at < k_end) *(Q*)(out + (c0 + col) * width + k0 + at) = *(const Q*)&s_q[col][at];
        __syncthreads();
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
    int* part;          // [splits][m][n], joined by k_int8_join; null: the tile ends the call itself
    long long k_split;  // bytes of a row that a workgroup sums, a multiple of 64
};

// Epilogue of C neighbouring columns of which w are there; everything is read before the first is written (out may be residual).
template <typename T, int C>
struct Beside { float scale[C]; VecOf<T, C> bias; };
template <typename T, int C>
__device__ __forceinline__ VecOf<T, C> some(const void* from, long long at, int w) {
    VecOf<T, C> v = {};
    if (!from) return v;
    const T* p = (const T*)from + at;
    if (w >= C) {
        __builtin_memcpy(&v, p, sizeof(v));
    } else {
#pragma unroll
        for (int j = 0; j < C; ++j)
            if (j < w) v[j] = p[j];
    }
    return v;
}
template <typename T, int C>
__device__ __forceinline__ Beside<T, C> beside(const Int8Args& p, long long n, int w) {
    Beside<T, C> b;
    if (w >= C) {
        __builtin_memcpy(b.scale, p.w_scale + n, sizeof(b.scale));
    } else {
#pragma unroll
        for (int j = 0; j < C; ++j) b.scale[j] = j < w ? p.w_scale[n + j] : 0.0f;
    }
    b.bias = some<T, C>(p.bias, n, w);
    return b;
}
template <typename T, int C>
__device__ __forceinline__ void finish(const Int8Args& p, long long m, long long n, int w, float xs, const int (&sum)[C],
                                       const Beside<T, C>& b, const VecOf<T, C>& residual) {
    VecOf<T, C> y;
    const long long at = m * p.n + n;
    float z[C];
    // (|sum| < 2^31: times a scale above 2^96 it may leave fp32 where z does not; by powers of two, so that every rounding is as before)
    const bool far = __builtin_fabsf(xs) > 0x1p96f;
    const float down = far ? xs * 0x1p-64f : xs, up = far ? 0x1p64f : 1.0f;
#pragma unroll
    for (int j = 0; j < C; ++j) {
        z[j] = (float)sum[j] * down * b.scale[j] * up;
        if (p.bias) z[j] += (float)b.bias[j];
    }
    activate_all<C>(z, p.act);
#pragma unroll
    for (int j = 0; j < C; ++j) {
        if (p.residual) z[j] += (float)residual[j];
        y[j] = (T)z[j];
    }
    if (w >= C) {
        // (tiles' results, where rows are whole vectors, leave the L2 to the operands: 8192 x 4096 x 4096 bf16 with silu and a residual
        // 150 us else, so 131; of 1303 columns it takes 2 per cent longer)
        if (C == 8 && (p.n & 7) == 0) __builtin_nontemporal_store(y, (VecOf<T, C> __attribute__((aligned(sizeof(T))))*)((T*)p.out + at));
        else __builtin_memcpy((T*)p.out + at, &y, sizeof(y));
    } else {
#pragma unroll
        for (int j = 0; j < C; ++j)
            if (j < w) ((T*)p.out)[at + j] = y[j];
    }
}
template <typename T, int C>
__device__ __forceinline__ void finish(const Int8Args& p, long long m, long long n, int w, float xs, const int (&sum)[C]) {
    finish<T, C>(p, m, n, w, xs, sum, beside<T, C>(p, n, w), some<T, C>(p.residual, m * p.n + n, w));
}

// BM x BN outputs a workgroup; a step is 128 bytes of every row, copied from memory to LDS without passing through registers, the
// next step's while this one's is multiplied.  (Steps of 64 bytes in three, four and five places: 3 to 12 per cent longer.)  Rows of a
// step are pieces of 16 bytes; piece c of row r lies at place c ^ spread(r), so that the lanes of a read meet different banks (the copy
// puts pieces down in the order of the lanes, whose addresses carry the permutation).  Rows past the arrays' ends are read from the last
// one, what they add up to is not stored; a row that ends in the middle of a step has its first half copied twice and multiplied once.
// The operands swap places at the instruction: its rows are the tile's columns n, in pairs of blocks (block b of a pair takes columns
// 8 (i / 4) + 4 b + i % 4, i < 16), so that a lane ends with eight neighbouring columns of one row.
// 8192 x 4096 x 4096 bf16 out, tiles of 256, in a graph: 123 us, with gelu and a residual 148, 2230 and 1860 TOP/s (the library's bare product
// 2030 to 2070); under the profiler the second 165, the least of 21 149.
// LDS has no conflict; one workgroup a unit, whose waves wait at a barrier a step, and an epilogue that nothing overlaps.  (Four waves
// of 128 x 128 one and a half times as long; without s_setprio 7 per cent longer; both halves' operands read ahead: no change.)
// 3001 x 1001 x 1303 fp32 out, tiles of 64: 13 us, four workgroups a unit, mostly their starts and ends.
template <bool PAIR>
__device__ __forceinline__ int spread(int r) { return PAIR ? (r & 3) | ((r >> 1) & 4) : r & 7; }  // (eight lanes read rows 0 to 7, PAIR: 0 to 3 and 8 to 11)

template <typename T, int BM, int BN, int WM, int WN>
__global__ __launch_bounds__(64 * WM * WN) void k_int8_ring(Int8Args p) {
    constexpr int P = 8, NT = 64 * WM * WN, A8 = BM * P, B8 = BN * P, AN = A8 / NT, BN8 = B8 / NT, SLOT = (A8 + B8) * 16;
    constexpr int TM = BM / WM / 16, TN = BN / WN / 16;
    static_assert(A8 % NT == 0 && B8 % NT == 0 && TN % 2 == 0, "whole pieces a thread, pairs of blocks");
    extern __shared__ __align__(1024) char s_ring[];
    const long long m_end = rows_of(p.m, p.rows_dev);
    unsigned tile_m, tile_n;
    const unsigned tiles_m = (unsigned)((p.m + BM - 1) / BM), tiles_n = (unsigned)((p.n + BN - 1) / BN), block = (unsigned)block_id<NT>();
    const bool any = block < tiles_m * tiles_n;
    tile_at(any ? block : 0, tiles_m, tiles_n, tile_m, tile_n);
    const long long m0 = any ? (long long)tile_m * BM : m_end, n0 = (long long)tile_n * BN;
    if (m0 >= m_end) return;
    const long long k_first = (long long)blockIdx.y * p.k_split;
    const int bytes = (int)(p.width - k_first < p.k_split ? p.width - k_first : p.k_split);  // (of every row: a multiple of 64)
    const int steps = (bytes + 127) / 128;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int wm = (wave / WN) * (TM * 16), wn = (wave % WN) * (TN * 16), q = lane >> 4, i16 = lane & 15;
    const unsigned ring = (unsigned)(size_t)(__attribute__((address_space(3))) char*)s_ring;

    // this thread's pieces: byte offsets from the tile's first value at the step's first k
    auto piece_a = [&](int e) { return (e % P) ^ spread<false>(e / P); };
    auto piece_b = [&](int e) { return (e % P) ^ spread<true>(e / P); };
    auto offset_of = [&](int r, int c, long long first, long long end) -> unsigned {
        const long long row = first + r < end ? r : end - 1 - first;
        return (unsigned)(row * p.width + c * 16);
    };
    unsigned at_a[AN], at_b[BN8];
#pragma unroll
    for (int i = 0; i < AN; ++i) at_a[i] = offset_of((i * NT + tid) / P, piece_a(i * NT + tid), m0, m_end);
#pragma unroll
    for (int i = 0; i < BN8; ++i) at_b[i] = offset_of((i * NT + tid) / P, piece_b(i * NT + tid), n0, p.n);
    const signed char *base_a = p.x + m0 * p.width + k_first, *base_b = p.w + n0 * p.width + k_first;
    // (half: pieces 4 to 7 of the last step, where the row has none: 64 bytes back)
    auto copy_step = [&](int slot, bool half) {
        const unsigned to = ring + slot * SLOT + wave * 1024;
#pragma unroll
        for (int i = 0; i < AN; ++i) copy_to_lds(base_a, at_a[i] - (half && piece_a(i * NT + tid) >= 4 ? 64u : 0u), to + i * NT * 16);
#pragma unroll
        for (int i = 0; i < BN8; ++i)
            copy_to_lds(base_b, at_b[i] - (half && piece_b(i * NT + tid) >= 4 ? 64u : 0u), to + A8 * 16 + i * NT * 16);
        base_a += 128;
        base_b += 128;
    };
    i4 acc[TM][TN];
#pragma unroll
    for (int i = 0; i < TM; ++i)
#pragma unroll
        for (int j = 0; j < TN; ++j) acc[i][j] = i4{0, 0, 0, 0};
    auto multiply = [&](const char* sa, const char* sb, int kk) {
        i4 fa[TM], fb[TN];
#pragma unroll
        for (int j = 0; j < TN; ++j) {
            const int r = wn + (j & ~1) * 16 + 8 * (i16 >> 2) + 4 * (j & 1) + (i16 & 3);
            fb[j] = *(const i4*)(sb + (r * P + ((kk * 4 + q) ^ spread<true>(r))) * 16);
        }
#pragma unroll
        for (int i = 0; i < TM; ++i) {
            const int r = wm + i * 16 + i16;
            fa[i] = *(const i4*)(sa + (r * P + ((kk * 4 + q) ^ spread<false>(r))) * 16);
        }
        __builtin_amdgcn_s_setprio(1);  // (a wave that multiplies goes before those that fetch)
#pragma unroll
        for (int i = 0; i < TM; ++i)
#pragma unroll
            for (int j = 0; j < TN; ++j) acc[i][j] = __builtin_amdgcn_mfma_i32_16x16x64_i8(fb[j], fa[i], acc[i][j], 0, 0, 0);
        __builtin_amdgcn_s_setprio(0);
    };
    const bool odd = (bytes & 127) != 0;
    copy_step(0, odd && steps == 1);
    for (int step = 0; step < steps; ++step) {
        // this step's copies have landed; its predecessor has been read by all waves, so that its place can be filled
        copies_and_barrier<0>();
        if (step + 1 < steps) copy_step((step + 1) & 1, odd && step + 2 == steps);
        const char* const s = s_ring + (step & 1) * SLOT;
        multiply(s, s + A8 * 16, 0);
        if (!odd || step + 1 < steps) multiply(s, s + A8 * 16, 1);
    }
    const long long m_lane = m0 + wm + i16;
    if (p.part) {
#pragma unroll
        for (int i = 0; i < TM; ++i)
#pragma unroll
            for (int j = 0; j < TN; j += 2) {
                const long long m = m_lane + i * 16, n = n0 + wn + j * 16 + 8 * q;
                if (m >= m_end || n >= p.n) continue;
                int* to = p.part + ((long long)blockIdx.y * p.m + m) * p.n + n;
                if (p.n - n >= 8) {
                    __builtin_memcpy(to, &acc[i][j], 16);
                    __builtin_memcpy(to + 4, &acc[i][j + 1], 16);
                } else {
#pragma unroll
                    for (int c = 0; c < 8; ++c)
                        if (c < p.n - n) to[c] = acc[i][j + c / 4][c % 4];
                }
            }
        return;
    }
    // what stands beside the sums is read for R rows at once
    constexpr int R = TM < 4 ? TM : 4;
    float xs[TM];
#pragma unroll
    for (int i = 0; i < TM; ++i) xs[i] = p.x_scale[m_lane + i * 16 < m_end ? m_lane + i * 16 : m_end - 1];
#pragma unroll
    for (int j = 0; j < TN; j += 2) {
        const long long n = n0 + wn + j * 16 + 8 * q;
        if (n >= p.n) continue;
        const int w = (int)(p.n - n < 8 ? p.n - n : 8);
        const Beside<T, 8> b = beside<T, 8>(p, n, w);
#pragma unroll
        for (int i0 = 0; i0 < TM; i0 += R) {
            VecOf<T, 8> residual[R];
#pragma unroll
            for (int r = 0; r < R; ++r) {
                const long long m = m_lane + (i0 + r) * 16;
                residual[r] = some<T, 8>(p.residual, (m < m_end ? m : m_end - 1) * p.n + n, w);
            }
#pragma unroll
            for (int r = 0; r < R; ++r) {
                const int i = i0 + r;
                const int sum[8] = {acc[i][j][0], acc[i][j][1], acc[i][j][2], acc[i][j][3],
                                    acc[i][j + 1][0], acc[i][j + 1][1], acc[i][j + 1][2], acc[i][j + 1][3]};
                if (m_lane + i * 16 < m_end) finish<T, 8>(p, m_lane + i * 16, n, w, xs[i], sum, b, residual[r]);
            }
        }
    }
}

// Up to 16 MB rows: bound by reading w once.  Eight waves share the k of 16 NB columns, operands straight from memory to the
// registers that the instruction wants, a lane 16 bytes of one row; their sums meet in LDS.  8 x 4096 -> 4096 in 8 bits: 6.4 us, 2.6 TB/s;
// 32 x 4096 -> 4096 8.9 (tiles of 64 longer than that up to 32 rows).
template <typename T, int MB, int NB>
__global__ __launch_bounds__(512) void k_int8_skinny(Int8Args p) {
    constexpr int W = 8, U = 4;
    __shared__ int s_sum[W][MB * NB][4][64];
    const long long m_end = rows_of(p.m, p.rows_dev);
    const long long n0 = block_id<512>() * (16 * NB);
    if (n0 >= p.n || m_end < 1) return;
    const long long k_first = (long long)blockIdx.y * p.k_split;
    const int bytes = (int)(p.width - k_first < p.k_split ? p.width - k_first : p.k_split);
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), q = lane >> 4, i16 = lane & 15;
    const signed char *x[MB], *w[NB];
#pragma unroll
    for (int i = 0; i < MB; ++i) x[i] = p.x + (16 * i + i16 < m_end ? 16 * i + i16 : m_end - 1) * p.width + k_first + q * 16;
#pragma unroll
    for (int j = 0; j < NB; ++j) w[j] = p.w + (n0 + 16 * j + i16 < p.n ? n0 + 16 * j + i16 : p.n - 1) * p.width + k_first + q * 16;
    i4 acc[MB][NB];
#pragma unroll
    for (int i = 0; i < MB; ++i)
#pragma unroll
        for (int j = 0; j < NB; ++j) acc[i][j] = i4{0, 0, 0, 0};
    // a wave's steps of 64 bytes lie next to each other
    const int steps = bytes / 64, each = (steps + W - 1) / W;
    const int from = wave * each, to = from + each < steps ? from + each : steps;
    for (int s = from; s < to; s += U) {
        i4 fx[U][MB], fw[U][NB];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const bool live = s + u < to;
            const long long at = (long long)(live ? s + u : s) * 64;
#pragma unroll
            for (int j = 0; j < NB; ++j) fw[u][j] = *(const i4*)(w[j] + at);
#pragma unroll
            for (int i = 0; i < MB; ++i) fx[u][i] = *(const i4*)(x[i] + at);
            if (!live)
#pragma unroll
                for (int j = 0; j < NB; ++j) fw[u][j] = i4{0, 0, 0, 0};
        }
#pragma unroll
        for (int u = 0; u < U; ++u)
#pragma unroll
            for (int i = 0; i < MB; ++i)
#pragma unroll
                for (int j = 0; j < NB; ++j) acc[i][j] = __builtin_amdgcn_mfma_i32_16x16x64_i8(fw[u][j], fx[u][i], acc[i][j], 0, 0, 0);
    }
#pragma unroll
    for (int i = 0; i < MB; ++i)
#pragma unroll
        for (int j = 0; j < NB; ++j)
#pragma unroll
            for (int c = 0; c < 4; ++c) s_sum[wave][i * NB + j][c][lane] = acc[i][j][c];
    __syncthreads();
    // four neighbouring columns a thread: lane (m, q) of block (i, j) as the instruction left them
    for (int e = threadIdx.x; e < MB * NB * 64; e += 512) {
        const int l = e & 63, b = e >> 6, i = b / NB, j = b % NB;
        const long long m = 16 * i + (l & 15), n = n0 + 16 * j + 4 * (l >> 4);
        if (m >= m_end || n >= p.n) continue;
        int sum[4] = {0, 0, 0, 0};
#pragma unroll
        for (int v = 0; v < W; ++v)
#pragma unroll
            for (int c = 0; c < 4; ++c) sum[c] += s_sum[v][b][c][l];
        const int width = (int)(p.n - n < 4 ? p.n - n : 4);
        if (p.part) {
            int* to4 = p.part + ((long long)blockIdx.y * p.m + m) * p.n + n;
#pragma unroll
            for (int c = 0; c < 4; ++c)
                if (c < width) to4[c] = sum[c];
        } else {
            finish<T, 4>(p, m, n, width, p.x_scale[m], sum);
        }
    }
}

// Joins the sums of a split k and ends the call: four neighbouring columns a thread.
template <typename T>
__global__ __launch_bounds__(256) void k_int8_join(Int8Args p, int splits) {
    const long long m_end = rows_of(p.m, p.rows_dev), quads = (p.n + 3) / 4;
    const long long id = block_id<256>() * 256 + threadIdx.x, m = id / quads, n = id % quads * 4;
    if (m >= m_end) return;
    const int w = (int)(p.n - n < 4 ? p.n - n : 4);
    const int* __restrict__ f = p.part + m * p.n + n;
    const long long step = p.m * p.n;
    int sum[4] = {0, 0, 0, 0};
#pragma unroll 8
    for (int s = 0; s < splits; ++s) {
        i4 v = {0, 0, 0, 0};
        if (w == 4) {
            __builtin_memcpy(&v, f + s * step, sizeof(v));
        } else {
#pragma unroll
            for (int c = 0; c < 4; ++c)
                if (c < w) v[c] = f[s * step + c];
        }
#pragma unroll
        for (int c = 0; c < 4; ++c) sum[c] += v[c];
    }
    finish<T, 4>(p, m, n, w, p.x_scale[m], sum);
}

// One row, brought to 8 bits by every workgroup for itself: bound by reading w once.  A wave takes R columns (rows of w), its first
// pieces of them on their way while the row is quantised; a lane multiplies 16 bytes at a time, four products an instruction.
// GIVEN: the row is there in 8 bits.  4096 -> 4096 bf16: 6.4 us, 2.6 TB/s of w, where the row's own reading, maximum and rounding come
// before the first product; one launch (as a quantisation and a product it took 26 us).
constexpr int kRowThreads = 256, kRowLds = 16384;  // bytes of the row in LDS at a time
template <typename T, int R, bool GIVEN>
__global__ __launch_bounds__(kRowThreads) void k_int8_row(Int8Args p, const T* __restrict__ x, int c_in) {
    constexpr int V = kVec<T>, P = kRowThreads, U = 4;
    __shared__ __align__(16) signed char s_x[kRowLds];
    __shared__ unsigned s_most[P / 64];
    if (rows_of(p.m, p.rows_dev) < 1) return;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const long long n0 = (block_id<P>() * (P / 64) + wave) * R;
    const int width = (int)p.width;
    const signed char* w[R];
#pragma unroll
    for (int r = 0; r < R; ++r) w[r] = p.w + (n0 + r < p.n ? n0 + r : p.n - 1) * p.width;
    i4 held[U][R];
    auto fetch = [&](int u, int k) {  // (past the row's end: its first bytes, times 0)
#pragma unroll
        for (int r = 0; r < R; ++r) held[u][r] = *(const i4*)(w[r] + (k < width ? k : 0));
    };
#pragma unroll
    for (int u = 0; u < U; ++u) fetch(u, (u * 64 + lane) * 16);
    Quantizer z = {0.0f, 0.0f};
    constexpr int H = 2;  // vectors of the row that a thread keeps between the two looks at them
    VecOf<T, V> mine[H];
    auto value = [&](int c) { return load_raw<T>(x + c, c < c_in ? c_in - c : 0, c_in >= V); };
    if constexpr (!GIVEN) {
        unsigned most = 0;
        auto look = [&](const VecOf<T, V>& v) {
#pragma unroll
            for (int i = 0; i < V; ++i) {
                const unsigned a = magnitude((float)v[i]);
                most = a > most ? a : most;
            }
        };
#pragma unroll
        for (int h = 0; h < H; ++h) mine[h] = value((h * P + threadIdx.x) * V);
#pragma unroll
        for (int h = 0; h < H; ++h) look(mine[h]);
        for (int c = (H * P + threadIdx.x) * V; c < c_in; c += P * V) look(value(c));
        most = wave_most(most);
        if (lane == 0) s_most[wave] = most;
        __syncthreads();
#pragma unroll
        for (int k = 0; k < P / 64; ++k) most = s_most[k] > most ? s_most[k] : most;
        z = quantizer(most);
    } else {
        z.scale = p.x_scale[0];
    }
    int acc[R];
#pragma unroll
    for (int r = 0; r < R; ++r) acc[r] = 0;
    for (int k0 = 0; k0 < width; k0 += kRowLds) {
        const int part = width - k0 < kRowLds ? width - k0 : kRowLds;
        __syncthreads();
        if constexpr (GIVEN) {
            for (int c = threadIdx.x * 16; c < part; c += P * 16) *(i4*)(s_x + c) = *(const i4*)(p.x + k0 + c);
        } else {
            typedef signed char Q __attribute__((ext_vector_type(V)));
            auto keep = [&](int c, const VecOf<T, V>& v) {
                Q b;
#pragma unroll
                for (int i = 0; i < V; ++i) b[i] = (signed char)quantized((float)v[i], z);
                *(Q*)(s_x + c) = b;
            };
            static_assert(H * P * V <= kRowLds, "the vectors that are kept are of the first part");
            if (k0 == 0)
#pragma unroll
                for (int h = 0; h < H; ++h)
                    if ((h * P + (int)threadIdx.x) * V < part) keep((h * P + threadIdx.x) * V, mine[h]);
            for (int c = (k0 == 0 ? H * P + threadIdx.x : threadIdx.x) * V; c < part; c += P * V) keep(c, value(k0 + c));
        }
        __syncthreads();
        for (int k = lane * 16; k < part; k += U * 1024) {
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const int at = k + u * 1024;
                const i4 v = at < part ? *(const i4*)(s_x + at) : i4{0, 0, 0, 0};
#pragma unroll
                for (int r = 0; r < R; ++r)
#pragma unroll
                    for (int c = 0; c < 4; ++c) acc[r] = __builtin_amdgcn_sdot4(v[c], held[u][r][c], acc[r], false);
                fetch(u, k0 + at + U * 1024);
            }
        }
    }
#pragma unroll
    for (int r = 0; r < R; ++r) {
        int sum[1] = {acc[r]};
#pragma unroll
        for (int d = 1; d < 64; d <<= 1) sum[0] += __shfl_xor(sum[0], d, 64);
        if (lane == r && n0 + r < p.n) finish<T, 1>(p, 0, n0 + r, 1, z.scale, sum);
    }
}

// ------------------------------------------------------------------ host side
template <typename T>
static hipError_t quantize(const void* x, long long rows, const long long* rows_dev, long long channels, signed char* q, float* scale,
                           hipStream_t s) {
    const long long width = int8_width(channels), units = width / kVec<T>;
#define F(P, H)                                                                                                           \
    hipLaunchKernelGGL((k_quantize_rows<T, P, H>), (grid_of<P < 256 ? 256 : P>((rows + (P < 256 ? 256 / P : 1) - 1) / (P < 256 ? 256 / P : 1))), \
                       dim3(P < 256 ? 256 : P), 0, s, (const T*)x, rows, rows_dev, channels, width, q, scale)
    if (units <= 8) F(4, 2);
    else if (units <= 32) F(16, 2);
    else if (units <= 128) F(64, 2);
    else if (units <= 512 || rows >= 4LL * device_cu_count()) F(256, 2);
    else F(1024, 2);
#undef F
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
    // as many workgroups as compute units, where the rows are enough for some steps each
    const long long width = int8_width(c_in), strips = (c_out + 31) / 32, least = 1024;
    long long splits = device_cu_count() / strips;
    if (splits > width / least) splits = width / least;
    if (splits < 1) splits = 1;
    const long long span = round_up((width + splits - 1) / splits, 256);
    hipLaunchKernelGGL((k_quantize_weight<T>), grid_of<1024>(strips, (unsigned)((width + span - 1) / span)), dim3(1024), 0, s, (const T*)w,
                       c_in, c_out, width, span, q, scale);
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

// Kernel of a product: one row, up to 32 rows straight from memory, or tiles of 256, 128 or 64 squared.  bf16 with silu and residual, rows
// given, us in a graph, of tiles of 256 / 128 / 64 (tiles of 64 x 128 lay between the last two, or above both):
//   8192 x 4096 x 4096 (m, k, n)  130 / 152 / 204        4096 x 4096 x 4096   66 / 74 / 104       16384 x 2048 x 1024  40 / 45 / 60
//   6000 x 4096 x 4096  117 / 111 / 155 (384 tiles of 256 on 256 units)     8192 x 1024 x 1024   25 / 17.0 / 19.9 (512 of 128)
//   5000 x 1000 x 1304   26 / 20.3 / 18.3 (440)          2048 x 2048 x 2048   35 / 18.7 / 17.4    3000 x 4096 x 1024   38 / 27.4 / 21.6
//   1000 x 12288 x 1000  38 / 31.4 / 31.5 (k split four ways, 64: twice)    1024 x 1024 x 1024   24 / 12.2 / 7.8
//   512 x 4096 x 4096    33 / 25.1 / 19.5                200000 x 64 x 64     51 / 26.4 / 15.8    300 x 300 x 3000   17.9 / 9.6 / 5.7
// The largest where their rounds over the units are 95 per cent full, 128 from two a unit on with k to hide their start and end, or where
// k is long.  k is split where workgroups are few, down to 1024 bytes of it: one a unit (tiles of 64: two).
enum class Int8Kind { kRow, kSkinny, kRing256, kRing128, kRing64 };
struct Int8Plan {
    Int8Kind kind;
    int bm, bn, splits;
    long long k_split;
};
static Int8Plan int8_plan(long long m, long long n, long long width) {
    Int8Plan t = {Int8Kind::kRow, 1, 1, 1, width};
    if (m <= 1) return t;
    const long long cus = device_cu_count();
    auto tiles = [&](long long bm, long long bn) { return ((m + bm - 1) / bm) * ((n + bn - 1) / bn); };
    long long want = cus;  // workgroups
    if (m <= 32) {
        t.kind = Int8Kind::kSkinny;
        t.bm = m <= 16 ? 16 : 32;
        t.bn = 16;
    } else {
        const long long largest = tiles(256, 256), rounds = (largest + cus - 1) / cus, large = tiles(128, 128);
        if (width >= 2048 && 20 * largest >= 19 * rounds * cus) t.kind = Int8Kind::kRing256, t.bm = t.bn = 256;
        else if ((width >= 1024 && large >= 2 * cus) || (width >= 8192 && 4 * large >= cus && m > 64)) t.kind = Int8Kind::kRing128, t.bm = t.bn = 128;
        else t.kind = Int8Kind::kRing64, t.bm = t.bn = 64, want = 2 * cus;
    }
    const long long all = tiles(t.bm, t.bn);
    if (all < want) {
        long long s = want / all, most = width / 1024;
        if (s > most) s = most;
        if (s > 1) t.k_split = round_up((width + s - 1) / s, t.kind == Int8Kind::kSkinny ? 512 : 128);
    }
    t.splits = (int)((width + t.k_split - 1) / t.k_split);
    return t;
}

struct Int8Space { size_t q, scale, part, total; };
static Int8Space int8_space(bool given, long long rows, long long c_in, long long c_out) {
    Int8Space a = {};
    const Int8Plan t = int8_plan(rows, c_out, int8_width(c_in));
    if (t.kind == Int8Kind::kRow) return a;
    if (!given) {
        a.scale = (size_t)round_up(rows * int8_width(c_in), 256);
        a.part = a.scale + (size_t)round_up(rows * 4, 256);
    }
    a.total = a.part + (t.splits > 1 ? (size_t)round_up(t.splits * rows * c_out * 4, 256) : 0);
    return a;
}
size_t linear_int8_bytes(int dtype, bool given, long long rows, long long c_in, long long c_out) {
    return int8_space(given, rows, c_in, c_out).total;
}

template <typename T, int BM, int BN, int WM, int WN>
static hipError_t ring(const Int8Args& p, long long tiles, int splits, hipStream_t s) {
    constexpr int lds = (BM + BN) * 256;
    auto kernel = k_int8_ring<T, BM, BN, WM, WN>;
    if (lds >= 65536) {
        const hipError_t e = hipFuncSetAttribute((const void*)kernel, hipFuncAttributeMaxDynamicSharedMemorySize, lds);
        if (e != hipSuccess) return e;
    }
    hipLaunchKernelGGL(kernel, grid_of<64 * WM * WN>(tiles, (unsigned)splits), dim3(64 * WM * WN), lds, s, p);
    return hipGetLastError();
}

template <typename T, bool GIVEN>
static void one_row(const Int8Args& p, const void* x, int c_in, hipStream_t s) {
    const long long cus = device_cu_count(), waves = kRowThreads / 64;
#define F(R) hipLaunchKernelGGL((k_int8_row<T, R, GIVEN>), grid_of<kRowThreads>((p.n + waves * R - 1) / (waves * R)), dim3(kRowThreads), 0, s, p, (const T*)x, c_in)
    if (p.n >= 4 * waves * cus) F(4);
    else if (p.n >= 2 * waves * cus) F(2);
    else F(1);
#undef F
}

template <typename T>
static hipError_t linear_int8(int dtype, const Int8Call& c, hipStream_t s) {
    Int8Args p = {};
    p.x = (const signed char*)c.x;
    p.x_scale = c.x_scale;
    p.w = c.w; p.w_scale = c.w_scale; p.bias = c.bias; p.residual = c.residual; p.out = c.out;
    p.m = c.rows; p.n = c.c_out; p.width = int8_width(c.c_in);
    p.rows_dev = c.rows_dev;
    p.act = c.act;
    const Int8Plan t = int8_plan(p.m, p.n, p.width);
    if (t.kind == Int8Kind::kRow) {
        if (c.x_scale) one_row<T, true>(p, c.x, (int)c.c_in, s);
        else one_row<T, false>(p, c.x, (int)c.c_in, s);
        return hipGetLastError();
    }
    const Int8Space at = int8_space(c.x_scale != nullptr, c.rows, c.c_in, c.c_out);
    if (!c.x_scale) {
        signed char* const q = (signed char*)c.workspace + at.q;
        float* const scale = (float*)((char*)c.workspace + at.scale);
        const hipError_t e = quantize<T>(c.x, c.rows, c.rows_dev, c.c_in, q, scale, s);
        if (e != hipSuccess) return e;
        p.x = q;
        p.x_scale = scale;
    }
    p.k_split = t.k_split;
    if (t.splits > 1) p.part = (int*)((char*)c.workspace + at.part);
    const long long tiles = ((p.m + t.bm - 1) / t.bm) * ((p.n + t.bn - 1) / t.bn);
    hipError_t e = hipSuccess;
    switch (t.kind) {
        case Int8Kind::kSkinny: {
            const dim3 grid = grid_of<512>(tiles, (unsigned)t.splits);
            if (t.bm == 16) hipLaunchKernelGGL((k_int8_skinny<T, 1, 1>), grid, dim3(512), 0, s, p);
            else hipLaunchKernelGGL((k_int8_skinny<T, 2, 1>), grid, dim3(512), 0, s, p);
            e = hipGetLastError();
            break;
        }
        case Int8Kind::kRing256: e = ring<T, 256, 256, 2, 4>(p, tiles, t.splits, s); break;
        case Int8Kind::kRing128: e = ring<T, 128, 128, 2, 2>(p, tiles, t.splits, s); break;
        default: e = ring<T, 64, 64, 2, 2>(p, tiles, t.splits, s);
    }
    if (e != hipSuccess || t.splits <= 1) return e;
    hipLaunchKernelGGL((k_int8_join<T>), grid_of<256>((p.m * ((p.n + 3) / 4) + 255) / 256), dim3(256), 0, s, p, t.splits);
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
