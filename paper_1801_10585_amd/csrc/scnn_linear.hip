// Linear layers on rows: out = act(x w + bias) + residual, and the gradients of x, w and bias.
//
//   forward   z [R, N] = x [R, K] w [K, N] + bias,  out = act(z) + residual
//   backward  dz = g act'(z),  dx [R, K] = dz w^T,  dw [K, N] = x^T dz,  dbias = sum_r dz
//
// All three products run through one tiled kernel (k_linear_tile): D [M, N] = sum_k A(m, k) B(k, n), where either operand
// lies in memory with k or with its other index contiguous.  A tile is staged in LDS the way it lies in memory; an operand
// whose k is contiguous is read from there in pieces of eight k a lane, the other by transposing LDS reads
// (ds_read_b64_tr_b16: sixteen lanes read four rows of sixteen values and each receives one column), so that no operand
// is laid out anew.  16-bit operands multiply as they are; fp32 operands are split into three bf16 numbers each while they
// are staged, and six of the nine products are multiplied (split8, split_products: as close to the exact sum as fp32
// products): 182 TFLOP/s on 4096 x 4096 x 4096 where the library's fp32 product reaches 147.  All sums are fp32.
#include "scnn_dense.h"

namespace scnn {

typedef float f4 __attribute__((ext_vector_type(4)));
typedef _Float16 h8 __attribute__((ext_vector_type(8)));
typedef short s4 __attribute__((ext_vector_type(4)));

// Byte offset of 16-byte piece c of row r of a staged tile.  K_CONTIG: rows of BK k (a row is one m or n); else rows of W
// values of one k.  Pieces are permuted within a row so that the lanes of a read hit different banks: by the row number
// for rows of k; in pairs (the 32 bytes that four lanes of a transposing read share) by the k for the others, of which one
// read takes the rows 8q .. 8q + 3, q < 4.
template <bool K_CONTIG, int W>
__device__ __forceinline__ int staged(int r, int c) {
    constexpr int CH = W / 8;
    if constexpr (K_CONTIG) {
        const int sw = CH >= 8 ? (r & 7) : ((r >> 1) & 3);
        return (r * CH + (c ^ sw)) * 16;
    } else {
        const int sw = ((r & 3) | ((r >> 1) & 4)) & (CH / 2 - 1);
        return (r * CH + (c ^ (sw << 1))) * 16;
    }
}

// Eight k (32 kk + 8 q .. + 7, q = lane / 16) of row or column `base` + lane % 16.
template <bool K_CONTIG, int W>
__device__ __forceinline__ u32x4 fragment(const char* tile, int base, int kk) {
    const int lane = threadIdx.x & 63, q = lane >> 4, i = lane & 15;
    if constexpr (K_CONTIG) {
        return *(const u32x4*)(tile + staged<true, W>(base + i, kk * 4 + q));
    } else {
        typedef __attribute__((address_space(3))) s4 lds_s4;
        const int k = kk * 32 + 8 * q + (i >> 2);
        const int c = (base >> 3) + ((i & 3) >> 1), in = (i & 1) * 8;
        union { s4 half[2]; u32x4 all; } r;
        r.half[0] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s4*)(tile + staged<false, W>(k, c) + in));
        r.half[1] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s4*)(tile + staged<false, W>(k + 4, c) + in));
        return r.all;
    }
}

// The same for columns in pairs of blocks: block b of the pair at `base` takes the columns base + 8 (i / 4) + 4 b + i % 4,
// i < 16, so that the two blocks' results of a lane are eight neighbouring columns (16 bytes of a 16-bit type; 64 bytes a row
// a store.  With 8 bytes a lane a wide layer's stores wrote 237 MB to memory for 134 MB of results.)
template <bool K_CONTIG, int W>
__device__ __forceinline__ int staged_pair(int r, int c) {  // rows of k: the rows of a read are 0-3, 8-11, 16-19, 24-27 (+ 4 b)
    if constexpr (K_CONTIG) return (r * (W / 8) + (c ^ (W >= 64 ? (r & 3) | ((r >> 1) & 4) : (r & 3)))) * 16;
    else return staged<false, W>(r, c);
}
template <bool K_CONTIG, int W>
__device__ __forceinline__ u32x4 fragment_pair(const char* tile, int base, int b, int kk) {
    const int lane = threadIdx.x & 63, q = lane >> 4, i = lane & 15;
    if constexpr (K_CONTIG) {
        return *(const u32x4*)(tile + staged_pair<true, W>(base + 8 * (i >> 2) + 4 * b + (i & 3), kk * 4 + q));
    } else {
        typedef __attribute__((address_space(3))) s4 lds_s4;
        const int k = kk * 32 + 8 * q + (i >> 2), c = (base >> 3) + (i & 3);
        union { s4 half[2]; u32x4 all; } r;
        r.half[0] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s4*)(tile + staged<false, W>(k, c) + 8 * b));
        r.half[1] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s4*)(tile + staged<false, W>(k + 4, c) + 8 * b));
        return r.all;
    }
}

// What a call multiplies.  `rows_k`: the device's row count bounds k (the filter's gradient), else m.
struct LinearArgs {
    const void* a;
    const void* b;
    long long m, n, k;
    const long long* rows_dev;
    const void* bias;
    const void* residual;
    void* out;
    void* pre;
    float* part;       // [splits][m][n], joined by k_linear_join; null: the tile ends the call itself
    long long k_split; // k a workgroup sums, a multiple of 64
    int act;
    int rows_k;
    const float* scale;  // fp16, nullable: what the sums are multiplied by (a power of two)
};

// Eight fp32 values as three bf16 numbers each, to nearest (split8), and what these leave of them, if anything: `lost`
// gathers the remainders' bits.  Nothing is left of 0 and of magnitudes from 2^-109 on, whose last bit is no smaller than
// bf16's smallest number; infinities and NaN leave NaN.
__device__ __forceinline__ void split8(const u32x4 (&x)[2], u32x4 (&part)[3], unsigned& lost) {
    typedef float f32x2 __attribute__((ext_vector_type(2)));
    typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        f32x2 v;
        v.x = __uint_as_float(x[i >> 1][(2 * i) & 3]);
        v.y = __uint_as_float(x[i >> 1][(2 * i + 1) & 3]);
#pragma unroll
        for (int k = 0; k < 3; ++k) {
            const unsigned p = __builtin_bit_cast(unsigned, __builtin_convertvector(v, bf16x2));
            part[k][i] = p;
            v.x -= __uint_as_float(p << 16);
            v.y -= __uint_as_float(p & 0xffff0000u);
        }
        lost |= __float_as_uint(v.x) | __float_as_uint(v.y);
    }
}

// Epilogue of four neighbouring columns: bias, activation, residual.
template <typename T>
__device__ __forceinline__ void finish4(const LinearArgs& p, long long m, long long n, float (&z)[4]) {
    const long long at = m * p.n + n;
    const int w = (int)(p.n - n < 4 ? p.n - n : 4);
    auto load4 = [&](const void* from, long long i, float (&v)[4]) {
        const T* f = (const T*)from + i;
        if (w == 4) {
            VecOf<T, 4> r;
            __builtin_memcpy(&r, f, sizeof(r));
#pragma unroll
            for (int j = 0; j < 4; ++j) v[j] = (float)r[j];
        } else {
#pragma unroll
            for (int j = 0; j < 4; ++j) v[j] = j < w ? (float)f[j] : 0.0f;
        }
    };
    auto store4 = [&](void* to, const float (&v)[4]) {
        T* f = (T*)to + at;
        if (w == 4) {
            VecOf<T, 4> r;
#pragma unroll
            for (int j = 0; j < 4; ++j) r[j] = (T)v[j];
            __builtin_memcpy(f, &r, sizeof(r));
        } else {
#pragma unroll
            for (int j = 0; j < 4; ++j)
                if (j < w) f[j] = (T)v[j];
        }
    };
    float t[4];
    if constexpr (std::is_same<T, _Float16>::value)
        if (p.scale) {
            const float by = *p.scale;
#pragma unroll
            for (int j = 0; j < 4; ++j) z[j] *= by;
        }
    if (p.bias) {
        load4(p.bias, n, t);
#pragma unroll
        for (int j = 0; j < 4; ++j) z[j] += t[j];
    }
    if (p.pre) store4(p.pre, z);
    if (p.act != SCNN_ACT_NONE)
#pragma unroll
        for (int j = 0; j < 4; ++j) z[j] = activate(z[j], p.act);
    if (p.residual) {
        load4(p.residual, at, t);
#pragma unroll
        for (int j = 0; j < 4; ++j) z[j] += t[j];
    }
    store4(p.out, z);
}

// The same for all of a wave's blocks, which lie inside the array: everything that is read is on its way before the first
// value is written.  (A load behind every store, which may be to the same place, was a fifth of a wide layer's time.)
// m: the lane's first row; n: its first column, of groups of C that lie GROUP apart (C = 8: pairs of blocks).
template <typename T, int TM, int TN, int C, int GROUP>
__device__ __forceinline__ void finish_tile(const LinearArgs& p, long long m, long long n, const f4 (&acc)[TM][TN]) {
    typedef VecOf<T, C> V;
    constexpr int J = TN * 4 / C;
    V bias[J], residual[TM][J];
    float by = 1.0f;
    if constexpr (std::is_same<T, _Float16>::value)
        if (p.scale) by = *p.scale;
#pragma unroll
    for (int j = 0; j < J; ++j) {
        bias[j] = V{};
        if (p.bias) __builtin_memcpy(&bias[j], (const T*)p.bias + n + j * GROUP, sizeof(V));
    }
    if (p.residual)
#pragma unroll
        for (int i = 0; i < TM; ++i)
#pragma unroll
            for (int j = 0; j < J; ++j)
                __builtin_memcpy(&residual[i][j], (const T*)p.residual + (m + i * 16) * p.n + n + j * GROUP, sizeof(V));
#pragma unroll
    for (int i = 0; i < TM; ++i)
#pragma unroll
        for (int j = 0; j < J; ++j) {
            const long long at = (m + i * 16) * p.n + n + j * GROUP;
            float z[C];
            V r;
#pragma unroll
            for (int c = 0; c < C; ++c) {
                z[c] = acc[i][j * (C / 4) + c / 4][c & 3];
                if constexpr (std::is_same<T, _Float16>::value) z[c] *= by;
                if (p.bias) z[c] += (float)bias[j][c];
                r[c] = (T)z[c];
            }
            if (p.pre) __builtin_memcpy((T*)p.pre + at, &r, sizeof(V));
            if (p.act != SCNN_ACT_NONE)
#pragma unroll
                for (int c = 0; c < C; ++c) z[c] = activate(z[c], p.act);
#pragma unroll
            for (int c = 0; c < C; ++c) {
                if (p.residual) z[c] += (float)residual[i][j][c];
                r[c] = (T)z[c];
            }
            __builtin_memcpy((T*)p.out + at, &r, sizeof(V));
        }
}

// Eight neighbouring values of a row of `cols`, 0 past its end and past the last row.
template <typename T>
__device__ __forceinline__ VecOf<T, 8> load8(const T* __restrict__ base, long long row, long long rows, long long col, long long cols) {
    constexpr int V = kVec<T>;
    VecOf<T, 8> v = {};
    if (row < rows && col < cols) {
        const T* __restrict__ p = base + row * cols + col;
        const int n = (int)(cols - col < 8 ? cols - col : 8);
        VecOf<T, V> half[8 / V];
#pragma unroll
        for (int i = 0; i < 8 / V; ++i) half[i] = load_raw<T>(p + i * V, n - i * V, cols >= V);
        __builtin_memcpy(&v, half, sizeof(v));
    }
    return v;
}

// BM x BN outputs a workgroup, BK values of k a step.  KG groups of WM x WN waves take the steps in turn, each with a staging
// area of its own, and join their sums at the end: waves enough to hide the latencies of short products without as many
// partial sums in memory.  The operands swap places at the instruction: its rows are the tile's columns n, so that a lane
// ends with four neighbouring n of one m (16 or 8 bytes a store).
template <typename T, bool AK, bool BK_, int BM, int BN, int BK, int WM, int WN, int KG>
__global__ __launch_bounds__(64 * WM * WN * KG) void k_linear_tile(LinearArgs p) {
    constexpr bool SPLIT = std::is_same<T, float>::value;
    constexpr int PARTS = SPLIT ? 3 : 1, NT = 64 * WM * WN;
    constexpr int AW = AK ? BK : BM, BW = BK_ ? BK : BN;          // values of a staged row
    constexpr int A8 = BM * BK / 8, B8 = BN * BK / 8;             // pieces of eight values
    constexpr int AN = (A8 + NT - 1) / NT, BN8 = (B8 + NT - 1) / NT, AREA = PARTS * (A8 + B8) * 16;
    constexpr int TM = BM / WM / 16, TN = BN / WN / 16;
    constexpr int JOIN = (KG - 1) * NT * TM * TN * 16;            // bytes in which the groups' sums meet
    __shared__ __align__(16) char s_stage[KG * AREA > JOIN ? KG * AREA : JOIN];
    const long long rows = rows_of(p.rows_k ? p.k : p.m, p.rows_dev);
    const long long m_end = p.rows_k ? p.m : rows, k_all = p.rows_k ? rows : p.k;
    const unsigned tiles_n = (unsigned)((p.n + BN - 1) / BN), block = (unsigned)block_id<NT * KG>();  // (tiles: up to 2^30)
    const long long m0 = (long long)(block / tiles_n) * BM, n0 = (long long)(block % tiles_n) * BN;
    if (m0 >= m_end) return;
    const long long k_first = (long long)blockIdx.y * p.k_split;
    const long long k_end = k_first + p.k_split < k_all ? k_first + p.k_split : k_all;
    const int group = KG == 1 ? 0 : __builtin_amdgcn_readfirstlane(threadIdx.x / NT);
    const int tid = threadIdx.x - group * NT, lane = tid & 63, wave = tid >> 6;
    const int wm = (wave / WN) * (TM * 16), wn = (wave % WN) * (TN * 16);
    char *const s_a = s_stage + group * AREA, *const s_b = s_a + PARTS * A8 * 16;

    f4 acc[TM][TN];
#pragma unroll
    for (int i = 0; i < TM; ++i)
#pragma unroll
        for (int j = 0; j < TN; ++j) acc[i][j] = f4{0.f, 0.f, 0.f, 0.f};

    // A tile that lies inside the arrays reads its pieces at 32-bit offsets from its first value, which moves on with k; the
    // others, and the last step of a k that ends inside it, ask for every piece where it lies.  (A multiplication of 64 bits
    // and four comparisons a piece cost as much as splitting its eight values.)
    VecOf<T, 8> ra[AN], rb[BN8];
    const long long wide_a = AK ? p.k : p.m, wide_b = BK_ ? p.k : p.n;
    const bool inside = m0 + BM <= m_end && n0 + BN <= p.n && A8 % NT == 0 && B8 % NT == 0 && wide_a < (1 << 22) && wide_b < (1 << 22);
    unsigned at_a[AN], at_b[BN8];
#pragma unroll
    for (int i = 0; i < AN; ++i) at_a[i] = (unsigned)((i * NT + tid) / (AW / 8)) * (unsigned)wide_a + (i * NT + tid) % (AW / 8) * 8;
#pragma unroll
    for (int i = 0; i < BN8; ++i) at_b[i] = (unsigned)((i * NT + tid) / (BW / 8)) * (unsigned)wide_b + (i * NT + tid) % (BW / 8) * 8;
    auto fetch = [&](long long k) {
        if (inside && k + BK <= k_end) {
            const T* __restrict__ pa = (const T*)p.a + (AK ? m0 * p.k + k : k * p.m + m0);
            const T* __restrict__ pb = (const T*)p.b + (BK_ ? n0 * p.k + k : k * p.n + n0);
#pragma unroll
            for (int i = 0; i < AN; ++i) __builtin_memcpy(&ra[i], pa + at_a[i], sizeof(ra[i]));
#pragma unroll
            for (int i = 0; i < BN8; ++i) __builtin_memcpy(&rb[i], pb + at_b[i], sizeof(rb[i]));
            return;
        }
        const bool any = k < k_end;  // (a group whose turn does not come stages zeros)
#pragma unroll
        for (int i = 0; i < AN; ++i) {
            const int e = i * NT + tid, r = e / (AW / 8), c = e % (AW / 8) * 8;
            if (A8 % NT == 0 || e < A8)
                ra[i] = AK ? load8<T>((const T*)p.a, m0 + r, any ? m_end : 0, k + c, p.k)
                           : load8<T>((const T*)p.a, k + r, k_end, m0 + c, p.m);
        }
#pragma unroll
        for (int i = 0; i < BN8; ++i) {
            const int e = i * NT + tid, r = e / (BW / 8), c = e % (BW / 8) * 8;
            if (B8 % NT == 0 || e < B8)
                rb[i] = BK_ ? load8<T>((const T*)p.b, n0 + r, any ? p.n : 0, k + c, p.k)
                            : load8<T>((const T*)p.b, k + r, k_end, n0 + c, p.n);
        }
    };
    unsigned lost = 0;  // bits of what the three parts of some value leave of it
    auto put = [&](char* tile, int pieces, int at, const VecOf<T, 8>& v) {
        if constexpr (SPLIT) {
            u32x4 x[2], part[3];
            __builtin_memcpy(x, &v, 32);
            split8(x, part, lost);
#pragma unroll
            for (int q = 0; q < 3; ++q) *(u32x4*)(tile + q * pieces * 16 + at) = part[q];
        } else {
            *(u32x4*)(tile + at) = __builtin_bit_cast(u32x4, v);
        }
    };
    fetch(k_first + group * BK);
    for (long long k0 = k_first; k0 < k_end; k0 += KG * BK) {
        __syncthreads();
#pragma unroll
        for (int i = 0; i < AN; ++i) {
            const int e = i * NT + tid;
            if (A8 % NT == 0 || e < A8) put(s_a, A8, staged<AK, AW>(e / (AW / 8), e % (AW / 8)), ra[i]);
        }
#pragma unroll
        for (int i = 0; i < BN8; ++i) {
            const int e = i * NT + tid;
            if (B8 % NT == 0 || e < B8) put(s_b, B8, staged<BK_, BW>(e / (BW / 8), e % (BW / 8)), rb[i]);
        }
        __syncthreads();
        if (k0 + KG * BK < k_end) fetch(k0 + (KG + group) * BK);
#pragma unroll
        for (int kk = 0; kk < BK / 32; ++kk) {
            u32x4 fa[TM][PARTS];
#pragma unroll
            for (int i = 0; i < TM; ++i)
#pragma unroll
                for (int q = 0; q < PARTS; ++q) fa[i][q] = fragment<AK, AW>(s_a + q * A8 * 16, wm + i * 16, kk);
#pragma unroll
            for (int j = 0; j < TN; ++j) {
                u32x4 fb[PARTS];
#pragma unroll
                for (int q = 0; q < PARTS; ++q) fb[q] = fragment<BK_, BW>(s_b + q * B8 * 16, wn + j * 16, kk);
#pragma unroll
                for (int i = 0; i < TM; ++i) {
                    if constexpr (SPLIT) {
                        f4 large, small;
                        split_products(fb, fa[i][0], fa[i][1], fa[i][2], large, small);
                        acc[i][j] += large + small;
                    } else if constexpr (std::is_same<T, __bf16>::value) {
                        acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, fb[0]),
                                                                            __builtin_bit_cast(bf16x8, fa[i][0]), acc[i][j], 0, 0, 0);
                    } else {
                        acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(h8, fb[0]),
                                                                           __builtin_bit_cast(h8, fa[i][0]), acc[i][j], 0, 0, 0);
                    }
                }
            }
        }
    }
    if constexpr (SPLIT) {
        // Values that the parts do not hold: too small ones leave something (lost), infinities and NaN, and magnitudes whose
        // products overflow though their sums might not, leave no finite sum.  A workgroup that met any sums its outputs
        // anew with fp32 products, the groups one k in KG of each four.
        bool odd = lost != 0;
#pragma unroll
        for (int i = 0; i < TM; ++i)
#pragma unroll
            for (int j = 0; j < TN; ++j)
#pragma unroll
                for (int c = 0; c < 4; ++c) odd |= (__float_as_uint(acc[i][j][c]) & 0x7f800000u) == 0x7f800000u;
        if (__syncthreads_or(odd)) {
            const int q = lane >> 4, i16 = lane & 15;
            auto at_a = [&](long long m, long long k) {
                return m < m_end && k < k_end ? (float)((const T*)p.a)[AK ? m * p.k + k : k * p.m + m] : 0.0f;
            };
            auto at_b = [&](long long n, long long k) {
                return n < p.n && k < k_end ? (float)((const T*)p.b)[BK_ ? n * p.k + k : k * p.n + n] : 0.0f;
            };
#pragma unroll
            for (int i = 0; i < TM; ++i)
#pragma unroll
                for (int j = 0; j < TN; ++j) acc[i][j] = f4{0.f, 0.f, 0.f, 0.f};
            for (long long k = k_first + 4 * group; k < k_end; k += 4 * KG)
#pragma unroll
                for (int i = 0; i < TM; ++i) {
                    const float va = at_a(m0 + wm + i * 16 + i16, k + q);
#pragma unroll
                    for (int j = 0; j < TN; ++j)
                        acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x4f32(at_b(n0 + wn + j * 16 + i16, k + q), va, acc[i][j], 0, 0, 0);
                }
        }
    }
    if constexpr (KG > 1) {
        __syncthreads();
        f4* const s_join = (f4*)s_stage;
        if (group > 0)
#pragma unroll
            for (int i = 0; i < TM; ++i)
#pragma unroll
                for (int j = 0; j < TN; ++j) s_join[(((group - 1) * TM + i) * TN + j) * NT + tid] = acc[i][j];
        __syncthreads();
        if (group > 0) return;
#pragma unroll
        for (int g = 0; g < KG - 1; ++g)
#pragma unroll
            for (int i = 0; i < TM; ++i)
#pragma unroll
                for (int j = 0; j < TN; ++j) acc[i][j] += s_join[((g * TM + i) * TN + j) * NT + tid];
    }
    // lane: row m = lane % 16, columns n = 4 (lane / 16) .. + 3 of each block
    if (!p.part && inside) {
        finish_tile<T, TM, TN, 4, 16>(p, m0 + wm + (lane & 15), n0 + wn + 4 * (lane >> 4), acc);
        return;
    }
#pragma unroll
    for (int i = 0; i < TM; ++i) {
        const long long m = m0 + wm + i * 16 + (lane & 15);
        if (m >= m_end) continue;
#pragma unroll
        for (int j = 0; j < TN; ++j) {
            const long long n = n0 + wn + j * 16 + 4 * (lane >> 4);
            if (n >= p.n) continue;
            float z[4] = {acc[i][j][0], acc[i][j][1], acc[i][j][2], acc[i][j][3]};
            if (p.part) {
                float* __restrict__ to = p.part + ((long long)blockIdx.y * p.m + m) * p.n + n;
#pragma unroll
                for (int c = 0; c < 4; ++c)
                    if (n + c < p.n) to[c] = z[c];
            } else {
                finish4<T>(p, m, n, z);
            }
        }
    }
}

// Tiles of a launch in the order of its workgroups.  Workgroup i runs on XCD i % 8: each XCD takes one run of neighbouring
// tiles, and within a run eight rows of tiles go side by side, so that the tiles that an L2 works on share their operands.
__device__ __forceinline__ void tile_at(unsigned block, unsigned tiles_m, unsigned tiles_n, unsigned& tm, unsigned& tn) {
    const unsigned all = tiles_m * tiles_n, each = all / kXcds, more = all % kXcds;
    const unsigned xcd = block % kXcds, i = block / kXcds;
    const unsigned at = xcd * each + (xcd < more ? xcd : more) + i;
    constexpr unsigned kSide = 8;
    const unsigned group = at / (kSide * tiles_n), in = at % (kSide * tiles_n);
    const unsigned side = tiles_m - group * kSide < kSide ? tiles_m - group * kSide : kSide;
    // (divisions leave the vector unit: the addresses that follow from these are to be scalar)
    tm = (unsigned)__builtin_amdgcn_readfirstlane((int)(group * kSide + in % side));
    tn = (unsigned)__builtin_amdgcn_readfirstlane((int)(in / side));
}

// Sixteen bytes a lane straight from memory to LDS: lane l's to lds + 16 l.
__device__ __forceinline__ void copy_to_lds(const void* base, unsigned offset, unsigned lds) {
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %1, %2" ::"s"(lds), "v"(offset), "s"(base) : "memory", "m0");
}
// Waits until at most N of this wave's copies are on their way and its LDS reads have arrived, then for the workgroup's
// other waves.
template <int N>
__device__ __forceinline__ void copies_and_barrier() {
    asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)\n\ts_barrier" ::"n"(N) : "memory");
}

// The same product for 16-bit operands whose rows begin on 16 bytes: tiles of BM x BN x BK go from memory to LDS without
// passing through registers, into a ring of STAGES, so that a step's copies have two steps of products to arrive.  The
// lanes' addresses carry the permutation of the pieces (staged), since the copy puts them down in the order of the lanes.
// Rows and columns past the arrays' ends are read from the last one inside; what they add up to is not stored.  k past a
// multiple of BK is staged through registers at the end, with zeros.  8192 x 4096 x 4096 bf16 (m, n, k): 226 us, 1219 TFLOP/s
// (the library's product 237), 253 with gelu, residual and pre, of whose time the matrix cores are busy 47 per cent (256 x 256
// tiles, one workgroup a unit: nothing multiplies while they end); 62 per cent in the products of 4096 x 4096 x 4096 (128 x 128
// tiles), LDS a third.
template <typename T, bool AK, bool BK_, int BM, int BN, int BK, int WM, int WN, int STAGES>
__global__ __launch_bounds__(64 * WM * WN) void k_linear_ring(LinearArgs p) {
    constexpr int NT = 64 * WM * WN, AW = AK ? BK : BM, BW = BK_ ? BK : BN;
    constexpr int A8 = BM * BK / 8, B8 = BN * BK / 8, AN = A8 / NT, BN8 = B8 / NT, SLOT = (A8 + B8) * 16;
    constexpr int TM = BM / WM / 16, TN = BN / WN / 16, COPIES = AN + BN8;
    constexpr bool PAIR = TN % 2 == 0;  // columns in pairs of blocks (fragment_pair)
    static_assert(A8 % NT == 0 && B8 % NT == 0, "whole pieces a thread");
    extern __shared__ __align__(1024) char s_ring[];
    const long long rows = rows_of(p.rows_k ? p.k : p.m, p.rows_dev);
    const long long m_end = p.rows_k ? p.m : rows, k_all = p.rows_k ? rows : p.k;
    unsigned tile_m, tile_n;
    const unsigned tiles_m = (unsigned)((p.m + BM - 1) / BM), tiles_n = (unsigned)((p.n + BN - 1) / BN), block = (unsigned)block_id<NT>();
    const bool any = block < tiles_m * tiles_n;
    tile_at(any ? block : 0, tiles_m, tiles_n, tile_m, tile_n);
    // (one way out: with two the compiler laid out the epilogue's branches so that a wide layer took 3 per cent longer)
    const long long m0 = any ? (long long)tile_m * BM : m_end, n0 = (long long)tile_n * BN;
    if (m0 >= m_end) return;
    const long long k_first = (long long)blockIdx.y * p.k_split;
    const long long k_end = k_first + p.k_split < k_all ? k_first + p.k_split : k_all;
    const int steps = k_end > k_first ? (int)((k_end - k_first) / BK) : 0;
    const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int wm = (wave / WN) * (TM * 16), wn = (wave % WN) * (TN * 16);
    const unsigned ring = (unsigned)(size_t)(__attribute__((address_space(3))) char*)s_ring;

    // This thread's pieces: byte offsets from the tile's first value at the step's first k.
    auto offset_of = [&](bool k_contig, bool pair, int w, int e, long long first, long long end, long long ld) -> unsigned {
        const int r = e / (w / 8);
        int c = e % (w / 8);
        if (k_contig) {
            c ^= pair ? (w >= 64 ? (r & 3) | ((r >> 1) & 4) : (r & 3)) : w / 8 >= 8 ? (r & 7) : ((r >> 1) & 3);
            const long long row = first + r < end ? r : end - 1 - first;
            return (unsigned)((row * ld + c * 8) * 2);
        }
        c ^= (((r & 3) | ((r >> 1) & 4)) & (w / 16 - 1)) << 1;
        const long long col = first + c * 8 < end ? c * 8 : end - 8 - first;  // (an array's width is a multiple of eight)
        return (unsigned)((r * ld + col) * 2);
    };
    unsigned at_a[AN], at_b[BN8];
#pragma unroll
    for (int i = 0; i < AN; ++i) at_a[i] = offset_of(AK, false, AW, i * NT + tid, m0, AK ? m_end : p.m, AK ? p.k : p.m);
#pragma unroll
    for (int i = 0; i < BN8; ++i) at_b[i] = offset_of(BK_, PAIR, BW, i * NT + tid, n0, p.n, BK_ ? p.k : p.n);
    const char* base_a = (const char*)p.a + (AK ? m0 * p.k + k_first : k_first * p.m + m0) * 2;
    const char* base_b = (const char*)p.b + (BK_ ? n0 * p.k + k_first : k_first * p.n + n0) * 2;
    const long long next_a = (AK ? (long long)BK : BK * p.m) * 2, next_b = (BK_ ? (long long)BK : BK * p.n) * 2;
    auto copy_step = [&](int slot) {
        const unsigned to = ring + slot * SLOT + wave * 1024;
#pragma unroll
        for (int i = 0; i < AN; ++i) copy_to_lds(base_a, at_a[i], to + i * NT * 16);
#pragma unroll
        for (int i = 0; i < BN8; ++i) copy_to_lds(base_b, at_b[i], to + A8 * 16 + i * NT * 16);
        base_a += next_a;
        base_b += next_b;
    };

    f4 acc[TM][TN];
#pragma unroll
    for (int i = 0; i < TM; ++i)
#pragma unroll
        for (int j = 0; j < TN; ++j) acc[i][j] = f4{0.f, 0.f, 0.f, 0.f};
    auto multiply = [&](const char* sa, const char* sb) {
#pragma unroll
        for (int kk = 0; kk < BK / 32; ++kk) {
            u32x4 fa[TM], fb[TN];
#pragma unroll
            for (int j = 0; j < TN; ++j)
                fb[j] = PAIR ? fragment_pair<BK_, BW>(sb, wn + (j & ~1) * 16, j & 1, kk) : fragment<BK_, BW>(sb, wn + j * 16, kk);
#pragma unroll
            for (int i = 0; i < TM; ++i) fa[i] = fragment<AK, AW>(sa, wm + i * 16, kk);
            // (a wave that multiplies goes before the other workgroup's waves, which then fetch: 1063 -> 1189 TFLOP/s on
            // 8192 x 4096 x 4096 with 128 x 128 tiles)
            __builtin_amdgcn_s_setprio(1);
#pragma unroll
            for (int i = 0; i < TM; ++i)
#pragma unroll
                for (int j = 0; j < TN; ++j) {
                    if constexpr (std::is_same<T, __bf16>::value)
                        acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, fb[j]),
                                                                            __builtin_bit_cast(bf16x8, fa[i]), acc[i][j], 0, 0, 0);
                    else
                        acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(h8, fb[j]),
                                                                           __builtin_bit_cast(h8, fa[i]), acc[i][j], 0, 0, 0);
                }
            __builtin_amdgcn_s_setprio(0);
        }
    };
    // STAGES - 1 steps are on their way before the first product.
#pragma unroll
    for (int i = 0; i < STAGES - 1; ++i)
        if (i < steps) copy_step(i);
    int slot = 0;
    for (int step = 0; step < steps; ++step) {
        // this step's copies have landed; its predecessor has been read by all waves, so that its slot can be filled
        if (step + STAGES - 1 <= steps) copies_and_barrier<(STAGES - 2) * COPIES>();
        else copies_and_barrier<0>();
        if (step + STAGES - 1 < steps) copy_step(slot == 0 ? STAGES - 1 : slot - 1);
        multiply(s_ring + slot * SLOT, s_ring + slot * SLOT + A8 * 16);
        slot = slot == STAGES - 1 ? 0 : slot + 1;
    }
    const long long k_tail = k_first + (long long)steps * BK;
    if (k_tail < k_end) {
        __syncthreads();
#pragma unroll
        for (int i = 0; i < AN; ++i) {
            const int e = i * NT + tid, r = e / (AW / 8), c = e % (AW / 8);
            const VecOf<T, 8> v = AK ? load8<T>((const T*)p.a, m0 + r, m_end, k_tail + c * 8, p.k)
                                     : load8<T>((const T*)p.a, k_tail + r, k_end, m0 + c * 8, p.m);
            *(u32x4*)(s_ring + staged<AK, AW>(r, c)) = __builtin_bit_cast(u32x4, v);
        }
#pragma unroll
        for (int i = 0; i < BN8; ++i) {
            const int e = i * NT + tid, r = e / (BW / 8), c = e % (BW / 8);
            const VecOf<T, 8> v = BK_ ? load8<T>((const T*)p.b, n0 + r, p.n, k_tail + c * 8, p.k)
                                      : load8<T>((const T*)p.b, k_tail + r, k_end, n0 + c * 8, p.n);
            *(u32x4*)(s_ring + A8 * 16 + (PAIR ? staged_pair<BK_, BW>(r, c) : staged<BK_, BW>(r, c))) = __builtin_bit_cast(u32x4, v);
        }
        __syncthreads();
        multiply(s_ring, s_ring + A8 * 16);
    }
    if (!p.part && m0 + BM <= m_end && n0 + BN <= p.n) {
        if constexpr (PAIR) finish_tile<T, TM, TN, 8, 32>(p, m0 + wm + (lane & 15), n0 + wn + 8 * (lane >> 4), acc);
        else finish_tile<T, TM, TN, 4, 16>(p, m0 + wm + (lane & 15), n0 + wn + 4 * (lane >> 4), acc);
        return;
    }
#pragma unroll
    for (int i = 0; i < TM; ++i) {
        const long long m = m0 + wm + i * 16 + (lane & 15);
        if (m >= m_end) continue;
#pragma unroll
        for (int j = 0; j < TN; ++j) {
            const long long n = n0 + wn + (PAIR ? (j & ~1) * 16 + 8 * (lane >> 4) + 4 * (j & 1) : j * 16 + 4 * (lane >> 4));
            if (n >= p.n) continue;
            float z[4] = {acc[i][j][0], acc[i][j][1], acc[i][j][2], acc[i][j][3]};
            if (p.part) __builtin_memcpy(p.part + ((long long)blockIdx.y * p.m + m) * p.n + n, z, 16);
            else finish4<T>(p, m, n, z);
        }
    }
}

// Joins the partial sums of a split k and ends the call: four neighbouring columns a thread, TS threads a quad, each over
// every TS-th split, their sums added in order.  (One thread a quad over 205 splits of a 35 x 19 filter: 92 us, each load
// behind the one before; sixteen: 5.)
template <typename T, int TS>
__global__ __launch_bounds__(256) void k_linear_join(LinearArgs p, int splits) {
    constexpr int Q = 256 / TS;
    __shared__ f4 s_sum[TS][Q];
    const long long m_end = p.rows_k ? p.m : rows_of(p.m, p.rows_dev);
    const long long quads = (p.n + 3) / 4;
    const int tq = threadIdx.x % Q, ts = threadIdx.x / Q;
    const long long id = block_id<256>() * Q + tq;
    const long long m = id / quads, n = id % quads * 4;
    f4 z = {0.f, 0.f, 0.f, 0.f};
    if (m < m_end) {
        const int w = (int)(p.n - n < 4 ? p.n - n : 4);
        const long long step = p.m * p.n;
        const float* __restrict__ f = p.part + m * p.n + n;
#pragma unroll 4
        for (int s = ts; s < splits; s += TS) {
            f4 v = {0.f, 0.f, 0.f, 0.f};
            if (w == 4) {
                __builtin_memcpy(&v, f + s * step, sizeof(v));
            } else {
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    if (j < w) v[j] = f[s * step + j];
            }
            z += v;
        }
    }
    s_sum[ts][tq] = z;
    __syncthreads();
    if (ts != 0 || m >= m_end) return;
#pragma unroll
    for (int i = 1; i < TS; ++i) z += s_sum[i][tq];
    float out[4] = {z[0], z[1], z[2], z[3]};
    finish4<T>(p, m, n, out);
}

// Largest finite magnitude of fp16 g [rows, cols] among this workgroup's values, as its bits: peak [gridDim.x].  A read of g, four
// loads a thread on their way: it makes a call of 4096 x 4096 -> 4096 longer by 7 us (290 / 284, 5 TB/s), small ones by 4.
constexpr int kPeaks = 256, kPeakThreads = 1024;
__global__ __launch_bounds__(kPeakThreads) void k_grad_peak(const _Float16* __restrict__ g, long long rows_cap,
                                                   const long long* __restrict__ rows_dev, long long cols,
                                                   unsigned* __restrict__ peak) {
    __shared__ unsigned s_max[kPeakThreads / 64];
    const long long n = rows_of(rows_cap, rows_dev) * cols, step = (long long)gridDim.x * kPeakThreads * 8;
    typedef VecOf<unsigned short, 8> Bits;
    Bits most = {};
    auto take = [&](VecOf<_Float16, 8> v) {
        const Bits bits = __builtin_bit_cast(Bits, v) & (unsigned short)0x7fff;
        const Bits fine = bits < (unsigned short)0x7c00 ? bits : Bits{};
        most = fine > most ? fine : most;
    };
    long long i = ((long long)blockIdx.x * kPeakThreads + threadIdx.x) * 8;
    for (; i + 3 * step + 8 <= n; i += 4 * step) {
        VecOf<_Float16, 8> v[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) v[k] = load_raw<_Float16>(g + i + k * step, 8, true);
#pragma unroll
        for (int k = 0; k < 4; ++k) take(v[k]);
    }
    for (; i < n; i += step) take(load_raw<_Float16>(g + i, (int)(n - i < 8 ? n - i : 8), n >= 8));
    unsigned top = 0;
#pragma unroll
    for (int j = 0; j < 8; ++j) top = most[j] > top ? most[j] : top;
    for (int d = 1; d < 64; d <<= 1) {
        const unsigned o = __shfl_xor(top, d, 64);
        top = o > top ? o : top;
    }
    if ((threadIdx.x & 63) == 0) s_max[threadIdx.x >> 6] = top;
    __syncthreads();
    if (threadIdx.x == 0) {
        for (int k = 1; k < kPeakThreads / 64; ++k) top = s_max[k] > top ? s_max[k] : top;
        peak[blockIdx.x] = top;
    }
}

// dz = g act'(pre) rounded to the operands' type (what the matrix instructions take), and this workgroup's column sums of
// the dz before that rounding: part [gridDim.y][cols].  A block is tn threads wide, each a 16-byte vector of columns.  Bound by
// memory: 4096 x 4096 bf16 gelu 21.5 us, 4.7 TB/s.
// fp16 with peaks: dz is held times the power of two that takes the largest finite |g| to 2^14 .. 2^15, so that none (slopes end
// at 1.13) passes fp16's end and only what is 2^-39 of that |g| and less is rounded to 0; unscale receives the inverse.
template <typename T>
__global__ __launch_bounds__(256) void k_act_back(const T* __restrict__ g, const T* __restrict__ pre, long long rows_cap,
                                                  const long long* __restrict__ rows_dev, long long cols, int act, int tn,
                                                  T* __restrict__ dz, float* __restrict__ part,
                                                  const unsigned* __restrict__ peak, int peaks, float* __restrict__ unscale) {
    constexpr int V = kVec<T>;
    __shared__ float s_sum[256][V];
    const long long rows = rows_of(rows_cap, rows_dev);
    float scale = 1.0f;
    if constexpr (std::is_same<T, _Float16>::value)
        if (peak) {
            __shared__ unsigned s_max[4];
            unsigned most = (int)threadIdx.x < peaks ? peak[threadIdx.x] : 0;
            for (int d = 1; d < 64; d <<= 1) {
                const unsigned o = __shfl_xor(most, d, 64);
                most = o > most ? o : most;
            }
            if ((threadIdx.x & 63) == 0) s_max[threadIdx.x >> 6] = most;
            __syncthreads();
            for (int i = 0; i < 4; ++i) most = s_max[i] > most ? s_max[i] : most;
            if (most > 0) {
                const float m = (float)__builtin_bit_cast(_Float16, (unsigned short)most);  // (normal in fp32: its exponent)
                const int up = 14 - ((int)(__float_as_uint(m) >> 23) - 127);
                scale = __uint_as_float((unsigned)(127 + up) << 23);
            }
            if (blockIdx.x == 0 && blockIdx.y == 0 && threadIdx.x == 0) *unscale = 1.0f / scale;
        }
    const int tc = threadIdx.x % tn, tr = threadIdx.x / tn, nr = 256 / tn;
    const long long c = ((long long)blockIdx.x * tn + tc) * V;
    const int n = (int)(cols - c < V ? cols - c : V);
    float sum[V];
#pragma unroll
    for (int i = 0; i < V; ++i) sum[i] = 0.0f;
    if (n > 0)
        for (long long row = (long long)blockIdx.y * nr + tr; row < rows; row += (long long)gridDim.y * nr) {
            float v[V], z[V];
            load_elems<T>(g + row * cols + c, n, cols >= V, v);
            if (act != SCNN_ACT_NONE) {
                load_elems<T>(pre + row * cols + c, n, cols >= V, z);
#pragma unroll
                for (int i = 0; i < V; ++i) v[i] = activate_back(v[i], z[i], act);
                if constexpr (std::is_same<T, _Float16>::value) {
                    float held[V];
#pragma unroll
                    for (int i = 0; i < V; ++i) held[i] = v[i] * scale;
                    store_elems<T>(dz + row * cols + c, n, held);
                } else {
                    store_elems<T>(dz + row * cols + c, n, v);
                }
            }
#pragma unroll
            for (int i = 0; i < V; ++i) sum[i] += v[i];
        }
    if (!part) return;
#pragma unroll
    for (int i = 0; i < V; ++i) s_sum[threadIdx.x][i] = sum[i];
    __syncthreads();
    for (int e = threadIdx.x; e < tn * V; e += 256) {
        const int col = e / V, i = e % V;
        const long long at = ((long long)blockIdx.x * tn + col) * V + i;
        if (at >= cols) continue;
        float t = 0.0f;
        for (int r = 0; r < nr; ++r) t += s_sum[r * tn + col][i];
        part[(long long)blockIdx.y * cols + at] = t;
    }
}

// Gradients of a narrow layer in one pass over its rows: bound by reading x, g and pre and writing dx once.  A workgroup
// keeps w in LDS and takes 64 rows at a time, the next ones on their way to registers meanwhile: dz = g act'(pre) is formed
// once, staged next to x, and read by both products, dx = dz w^T with its channels contiguous, dw += x^T dz by transposing
// reads; dw stays in the accumulators and the column sums of dz in registers until the workgroup's rows are done.  part
// [gridDim.x][c_in * c_out + c_out] then receives both, and one launch adds the workgroups' up.  P: widths up to P.
// 52417 rows of 35 -> 19 fp16, silu: 13.7 + 4 us, against 30 for the five launches of the general way; 643072 of 64 -> 64 with
// relu bf16 75 us, 4.4 TB/s, fp32 165 us, 4.0 TB/s.
template <int BYTES, int P> struct NarrowShape;  // threads; waves of dx (64 x P) and of dw (P x P), rows by columns
template <int BYTES> struct NarrowShape<BYTES, 32> { static constexpr int NT = 256, XM = 4, XN = 1, WM = 2, WN = 2; };
template <> struct NarrowShape<4, 64> { static constexpr int NT = 256, XM = 2, XN = 2, WM = 2, WN = 2; };
template <> struct NarrowShape<2, 64> { static constexpr int NT = 512, XM = 4, XN = 2, WM = 2, WN = 4; };

struct NarrowArgs {
    const void *x, *w, *pre, *g;
    void* dx;
    float* part;
    long long rows;
    const long long* rows_dev;
    int c_in, c_out, act;
};

// FINE: 16-bit types behind gelu or silu, whose dz has more bits than the type.  dz then enters both products as two bf16
// numbers (2^-17 of it are left out), bf16 operands as they are and fp16 ones as two bf16 numbers, which hold them exactly; of
// the products of parts all but low times low.  bf16 has fp32's range, so that no dz overflows or vanishes as it would in fp16.
// (Rounded to the type, dz cost dw of 52417 x 35 -> 19 fp16 half of its accuracy.  us a call in a graph, this against dz rounded:
// that layer 18.6 / 16.7; 643072 of 64 -> 64 gelu, bf16 97 / 88, fp16 105 / 89; 209645 of 24 -> 24 silu, bf16 23.0 / 21.5.  To look
// for infinities in the sums, not in what is staged, saved 2 to 20 us of these.)
template <typename T, int P, bool FINE>
__global__ __launch_bounds__((NarrowShape<sizeof(T), P>::NT)) void k_linear_bwd_narrow(NarrowArgs p) {
    constexpr bool SPLIT = std::is_same<T, float>::value, HALF = std::is_same<T, _Float16>::value;
    constexpr int ZP = SPLIT ? 3 : (FINE ? 2 : 1), XP = SPLIT ? 3 : (FINE && HALF ? 2 : 1);  // parts of dz; of x and w
    constexpr int ROWS = 64, CH = P / 8;
    typedef NarrowShape<sizeof(T), P> S;
    constexpr int NT = S::NT, PIECES = ROWS * CH, PN = PIECES / NT, WPIECES = P * CH, WPN = (WPIECES + NT - 1) / NT;
    constexpr int XM = ROWS / S::XM / 16, XN = P / S::XN / 16, WM = P / S::WM / 16, WN = P / S::WN / 16;
    __shared__ __align__(16) char s_w[XP * WPIECES * 16], s_z[(ZP + XP) * PIECES * 16];
    char* const s_x = s_z + ZP * PIECES * 16;
    const long long rows = rows_of(p.rows, p.rows_dev);
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
    const T *const x = (const T*)p.x, *const w = (const T*)p.w, *const pre = (const T*)p.pre, *const g = (const T*)p.g;
    const int c8 = tid % CH * 8;  // first column of this thread's pieces

    auto put_parts = [&](char* tile, int pieces, int at, const VecOf<float, 8>& v) {
        const bf16x8 high = __builtin_convertvector(v, bf16x8);
        const bf16x8 low = __builtin_convertvector(v - __builtin_convertvector(high, VecOf<float, 8>), bf16x8);
        *(u32x4*)(tile + at) = __builtin_bit_cast(u32x4, high);
        *(u32x4*)(tile + pieces * 16 + at) = __builtin_bit_cast(u32x4, low);
    };
    auto put = [&](char* tile, int pieces, int at, const VecOf<T, 8>& v, int& odd) {
        if constexpr (SPLIT) {
            u32x4 q[2], part[3];
            __builtin_memcpy(q, &v, 32);
#pragma unroll
            for (int i = 0; i < 8; ++i) odd |= split_exact(q[i >> 2][i & 3]) ? 0 : 1;
            scnn::split8(q, part);
#pragma unroll
            for (int k = 0; k < 3; ++k) *(u32x4*)(tile + k * pieces * 16 + at) = part[k];
        } else if constexpr (FINE && HALF) {
            put_parts(tile, pieces, at, __builtin_convertvector(v, VecOf<float, 8>));
        } else {
            *(u32x4*)(tile + at) = __builtin_bit_cast(u32x4, v);
        }
    };
    // w [c_in][c_out]: the contraction of dx runs along its rows
    int odd_w = 0;
#pragma unroll
    for (int i = 0; i < WPN; ++i) {
        const int e = i * NT + tid;
        if (WPIECES % NT == 0 || e < WPIECES)
            put(s_w, WPIECES, staged<true, P>(e / CH, e % CH), load8<T>(w, e / CH, p.dx ? p.c_in : 0, e % CH * 8, p.c_out), odd_w);
    }
    VecOf<T, 8> rx[PN], rg[PN], rp[PN];
    auto fetch = [&](long long first) {
#pragma unroll
        for (int i = 0; i < PN; ++i) {
            const long long row = first + (i * NT + tid) / CH;
            rg[i] = load8<T>(g, row, rows, c8, p.c_out);
            if (p.act != SCNN_ACT_NONE) rp[i] = load8<T>(pre, row, rows, c8, p.c_out);
            rx[i] = load8<T>(x, x ? row : rows, rows, c8, p.c_in);  // (null: dw is not asked for)
        }
    };
    f4 dw[WM][WN];
#pragma unroll
    for (int i = 0; i < WM; ++i)
#pragma unroll
        for (int j = 0; j < WN; ++j) dw[i][j] = f4{0.f, 0.f, 0.f, 0.f};
    float db[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) db[i] = 0.0f;
    auto multiply = [&](const auto& a, const auto& b, f4 acc) {  // (b's rows become the lanes' rows)
        constexpr int NA = sizeof(a) / 16, NB = sizeof(b) / 16;
        if constexpr (SPLIT) {
            f4 large, small;
            split_products(a, b[0], b[1], b[2], large, small);
            return acc + (large + small);
        } else if constexpr (FINE) {
#pragma unroll
            for (int i = NA - 1; i >= 0; --i)
#pragma unroll
                for (int j = NB - 1; j >= 0; --j)
                    if (i + j < 2)
                        acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a[i]), __builtin_bit_cast(bf16x8, b[j]), acc, 0, 0, 0);
            return acc;
        } else if constexpr (std::is_same<T, __bf16>::value) {
            return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a[0]), __builtin_bit_cast(bf16x8, b[0]), acc, 0, 0, 0);
        } else {
            return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(h8, a[0]), __builtin_bit_cast(h8, b[0]), acc, 0, 0, 0);
        }
    };
    const long long step = (long long)gridDim.x * ROWS;
    const int xm = wave / S::XN * XM * 16, xn = wave % S::XN * XN * 16, wm = wave / S::WN * WM * 16, wn = wave % S::WN * WN * 16;
    // The same with fp32 products, operands from memory, for values that the parts do not hold.
    const int q4 = lane >> 4, i16 = lane & 15;
    auto z_at = [&](long long row, int n) {
        if (row >= rows || n >= p.c_out) return 0.0f;
        const float v = (float)g[row * p.c_out + n];
        return p.act != SCNN_ACT_NONE ? activate_back(v, (float)pre[row * p.c_out + n], p.act) : v;
    };
    auto dx_fp32 = [&](long long at, f4 (&dx)[XM][XN]) {
        for (int k = 0; k < p.c_out; k += 4)
#pragma unroll
            for (int i = 0; i < XM; ++i) {
                const float vz = z_at(at + xm + i * 16 + i16, k + q4);
#pragma unroll
                for (int j = 0; j < XN; ++j) {
                    const int n = xn + j * 16 + i16;
                    const float vw = n < p.c_in && k + q4 < p.c_out ? (float)w[n * p.c_out + k + q4] : 0.0f;
                    dx[i][j] = __builtin_amdgcn_mfma_f32_16x16x4f32(vw, vz, dx[i][j], 0, 0, 0);
                }
            }
    };
    auto dw_fp32 = [&](long long at) {
        for (int k = 0; k < ROWS; k += 4)
#pragma unroll
            for (int i = 0; i < WM; ++i) {
                const int m = wm + i * 16 + i16;
                const float vx = at + k + q4 < rows && m < p.c_in ? (float)x[(at + k + q4) * p.c_in + m] : 0.0f;
#pragma unroll
                for (int j = 0; j < WN; ++j)
                    dw[i][j] = __builtin_amdgcn_mfma_f32_16x16x4f32(z_at(at + k + q4, wn + j * 16 + i16), vx, dw[i][j], 0, 0, 0);
            }
    };
    // FINE: low parts beside an infinity make a NaN of what should stay one; either shows in the sums, which the wave then forms
    // anew.
    auto odd_sums = [&](const auto& acc) {
        float none = 0.0f;
#pragma unroll
        for (int i = 0; i < (int)(sizeof(acc) / sizeof(acc[0])); ++i)
#pragma unroll
            for (int j = 0; j < (int)(sizeof(acc[0]) / 16); ++j)
#pragma unroll
                for (int c = 0; c < 4; ++c) none = __builtin_fmaf(acc[i][j][c], 0.0f, none);
        return __any(none != none) != 0;
    };
    long long first = (long long)blockIdx.x * ROWS;
    if (first < rows) fetch(first);
    for (; first < rows; first += step) {
        int odd = odd_w;
        if (first != (long long)blockIdx.x * ROWS) __syncthreads();  // (the tiles before these have been read)
#pragma unroll
        for (int i = 0; i < PN; ++i) {
            const int r = (i * NT + tid) / CH;
            VecOf<T, 8> z = rg[i];
            VecOf<float, 8> wide;
#pragma unroll
            for (int c = 0; c < 8; ++c) {
                float v = (float)rg[i][c];
                if (p.act != SCNN_ACT_NONE) {
                    v = first + r < rows && c8 + c < p.c_out ? activate_back(v, (float)rp[i][c], p.act) : 0.0f;
                    z[c] = (T)v;  // (fp32; relu's dz is g or 0)
                }
                wide[c] = v;
                db[c] += v;
            }
            if constexpr (FINE) put_parts(s_z, PIECES, staged<false, P>(r, tid % CH), wide);
            else put(s_z, PIECES, staged<false, P>(r, tid % CH), z, odd);
            if (x) put(s_x, PIECES, staged<false, P>(r, tid % CH), rx[i], odd);
        }
        bool exact = true;
        if constexpr (SPLIT) exact = !__syncthreads_or(odd);
        else __syncthreads();
        if (first + step < rows) fetch(first + step);
        // dz [64][c_out], rows of dz one way and columns the other
        auto rows_of_z = [&](int base, int kk, u32x4 (&f)[ZP]) {
            const int r = base + (lane & 15);
#pragma unroll
            for (int q = 0; q < ZP; ++q) f[q] = *(const u32x4*)(s_z + q * PIECES * 16 + staged<false, P>(r, kk * 4 + (lane >> 4)));
        };
        f4 dx[XM][XN];
#pragma unroll
        for (int i = 0; i < XM; ++i)
#pragma unroll
            for (int j = 0; j < XN; ++j) dx[i][j] = f4{0.f, 0.f, 0.f, 0.f};
        if (exact) {
            if (p.dx)
#pragma unroll
                for (int kk = 0; kk < P / 32; ++kk) {
                    if (kk * 32 >= p.c_out) break;
                    u32x4 fz[XM][ZP];
#pragma unroll
                    for (int i = 0; i < XM; ++i) rows_of_z(xm + i * 16, kk, fz[i]);
#pragma unroll
                    for (int j = 0; j < XN; ++j) {
                        if (xn + j * 16 >= p.c_in) break;
                        u32x4 fw[XP];
#pragma unroll
                        for (int q = 0; q < XP; ++q) fw[q] = fragment<true, P>(s_w + q * WPIECES * 16, xn + j * 16, kk);
#pragma unroll
                        for (int i = 0; i < XM; ++i) dx[i][j] = multiply(fw, fz[i], dx[i][j]);
                    }
                }
            if (x)
#pragma unroll
                for (int kk = 0; kk < ROWS / 32; ++kk) {
                    if (wm >= p.c_in) break;
                    u32x4 fx[WM][XP];
#pragma unroll
                    for (int i = 0; i < WM; ++i)
#pragma unroll
                        for (int q = 0; q < XP; ++q) fx[i][q] = fragment<false, P>(s_x + q * PIECES * 16, wm + i * 16, kk);
#pragma unroll
                    for (int j = 0; j < WN; ++j) {
                        if (wn + j * 16 >= p.c_out) break;
                        u32x4 fz[ZP];
#pragma unroll
                        for (int q = 0; q < ZP; ++q) fz[q] = fragment<false, P>(s_z + q * PIECES * 16, wn + j * 16, kk);
#pragma unroll
                        for (int i = 0; i < WM; ++i) dw[i][j] = multiply(fz, fx[i], dw[i][j]);
                    }
                }
        } else if constexpr (SPLIT) {
            // a value among these rows or in w that the three parts do not hold
            if (p.dx) dx_fp32(first, dx);
            if (x) dw_fp32(first);
        }
        if constexpr (FINE)
            if (p.dx && odd_sums(dx)) {
#pragma unroll
                for (int i = 0; i < XM; ++i)
#pragma unroll
                    for (int j = 0; j < XN; ++j) dx[i][j] = f4{0.f, 0.f, 0.f, 0.f};
                dx_fp32(first, dx);
            }
        if (p.dx)
#pragma unroll
            for (int i = 0; i < XM; ++i) {
                const long long row = first + xm + i * 16 + (lane & 15);
                if (row >= rows) continue;
#pragma unroll
                for (int j = 0; j < XN; ++j) {
                    const int n = xn + j * 16 + 4 * (lane >> 4);
                    T* __restrict__ to = (T*)p.dx + row * p.c_in + n;
                    if (n + 4 <= p.c_in) {
                        VecOf<T, 4> v;
#pragma unroll
                        for (int c = 0; c < 4; ++c) v[c] = (T)dx[i][j][c];
                        __builtin_memcpy(to, &v, sizeof(v));
                    } else {
#pragma unroll
                        for (int c = 0; c < 4; ++c)
                            if (n + c < p.c_in) to[c] = (T)dx[i][j][c];
                    }
                }
            }
    }
    if (!p.part) return;
    if constexpr (FINE)
        if (x && odd_sums(dw)) {
#pragma unroll
            for (int i = 0; i < WM; ++i)
#pragma unroll
                for (int j = 0; j < WN; ++j) dw[i][j] = f4{0.f, 0.f, 0.f, 0.f};
            for (long long at = (long long)blockIdx.x * ROWS; at < rows; at += step) dw_fp32(at);
        }
    float* __restrict__ mine = p.part + (long long)blockIdx.x * ((long long)p.c_in * p.c_out + p.c_out);
#pragma unroll
    for (int i = 0; i < WM; ++i) {
        const int m = wm + i * 16 + (lane & 15);
        if (m >= p.c_in) continue;
#pragma unroll
        for (int j = 0; j < WN; ++j) {
            const int n = wn + j * 16 + 4 * (lane >> 4);
#pragma unroll
            for (int c = 0; c < 4; ++c)
                if (n + c < p.c_out) mine[m * p.c_out + n + c] = dw[i][j][c];
        }
    }
    // column sums: threads with the same columns lie CH apart
    __syncthreads();
    float(*s_db)[P] = (float(*)[P])s_z;
    static_assert(NT / CH * P * 4 <= (ZP + XP) * PIECES * 16, "room for the column sums");
#pragma unroll
    for (int c = 0; c < 8; ++c) s_db[tid / CH][c8 + c] = db[c];
    __syncthreads();
    if (tid < p.c_out) {
        float sum = 0.0f;
        for (int r = 0; r < NT / CH; ++r) sum += s_db[r][tid];
        mine[p.c_in * p.c_out + tid] = sum;
    }
}

// A narrow layer forward: bound by reading x and writing out.  w stays in registers, as the operand of every product of its
// wave; a wave takes 16 rows at a time, each lane eight neighbouring channels of a row straight from memory, which is how
// the instruction wants them, the next rows on their way meanwhile.  No LDS, no barrier.  Widths up to P.
// us, this against tiles of 64 x 64: 209645 rows of 24 -> 24 fp32 15.7 / 26.0, bf16 11.7 / 21.8; 100000 of 8 -> 16 fp32 8.8 /
// 12.9.  With 64 channels its registers cost the occupancy that streaming needs: 643072 of 64 -> 64 bf16 59.6 / 52.3.
struct NarrowFwdArgs {
    const void *x, *w, *bias, *residual;
    void *out, *pre;
    long long rows;
    const long long* rows_dev;
    int c_in, c_out, act;
};

template <typename T, int P>
__global__ __launch_bounds__(256) void k_linear_fwd_narrow(NarrowFwdArgs p) {
    constexpr bool SPLIT = std::is_same<T, float>::value;
    constexpr int PARTS = SPLIT ? 3 : 1, KB = P / 32, NB = P / 16;
    typedef VecOf<T, 4> V4;
    const long long rows = rows_of(p.rows, p.rows_dev);
    const int lane = threadIdx.x & 63, i16 = lane & 15, q = lane >> 4;
    const T *const x = (const T*)p.x, *const w = (const T*)p.w;
    int odd_w = 0;
    // lane: column n = 16 j + lane % 16 of w, k = 32 kk + 8 (lane / 16) .. + 7
    u32x4 fw[KB][NB][PARTS];
#pragma unroll
    for (int kk = 0; kk < KB; ++kk)
#pragma unroll
        for (int j = 0; j < NB; ++j) {
            VecOf<T, 8> v = {};
            const int n = j * 16 + i16;
#pragma unroll
            for (int c = 0; c < 8; ++c) {
                const int k = kk * 32 + q * 8 + c;
                if (k < p.c_in && n < p.c_out) v[c] = w[k * p.c_out + n];
            }
            if constexpr (SPLIT) {
                u32x4 two[2];
                __builtin_memcpy(two, &v, 32);
#pragma unroll
                for (int c = 0; c < 8; ++c) odd_w |= split_exact(two[c >> 2][c & 3]) ? 0 : 1;
                scnn::split8(two, fw[kk][j]);
            } else {
                fw[kk][j][0] = __builtin_bit_cast(u32x4, v);
            }
        }
    // (a value of w that the parts do not hold makes every row of the call multiply in fp32)
    odd_w = __any(odd_w);
    V4 bias[NB];
#pragma unroll
    for (int j = 0; j < NB; ++j) {
        bias[j] = V4{};
        if (p.bias)
#pragma unroll
            for (int c = 0; c < 4; ++c)
                if (j * 16 + 4 * q + c < p.c_out) bias[j][c] = ((const T*)p.bias)[j * 16 + 4 * q + c];
    }
    VecOf<T, 8> next[KB];
    auto fetch = [&](long long first) {
#pragma unroll
        for (int kk = 0; kk < KB; ++kk) next[kk] = load8<T>(x, first + i16, rows, kk * 32 + q * 8, p.c_in);
    };
    const long long step = (long long)gridDim.x * 64;
    long long first = (long long)blockIdx.x * 64 + (threadIdx.x >> 6) * 16;
    if (first < rows) fetch(first);
    const bool aligned4 = p.c_out % 4 == 0;
    for (; first < rows; first += step) {
        VecOf<T, 8> now[KB];
#pragma unroll
        for (int kk = 0; kk < KB; ++kk) now[kk] = next[kk];
        const long long row = first + i16;
        V4 residual[NB];
        if (p.residual)
#pragma unroll
            for (int j = 0; j < NB; ++j) {
                const int n = j * 16 + 4 * q;
                residual[j] = V4{};
                if (row < rows && n < p.c_out) {
                    const T* __restrict__ from = (const T*)p.residual + row * p.c_out + n;
                    if (aligned4 || n + 4 <= p.c_out) {
                        __builtin_memcpy(&residual[j], from, sizeof(V4));
                    } else {
#pragma unroll
                        for (int c = 0; c < 4; ++c)
                            if (n + c < p.c_out) residual[j][c] = from[c];
                    }
                }
            }
        if (first + step < rows) fetch(first + step);
        f4 acc[NB];
#pragma unroll
        for (int j = 0; j < NB; ++j) acc[j] = f4{0.f, 0.f, 0.f, 0.f};
        int odd = odd_w;
#pragma unroll
        for (int kk = 0; kk < KB; ++kk) {
            if (kk * 32 >= p.c_in) break;
            u32x4 fx[PARTS];
            if constexpr (SPLIT) {
                u32x4 two[2];
                __builtin_memcpy(two, &now[kk], 32);
#pragma unroll
                for (int c = 0; c < 8; ++c) odd |= split_exact(two[c >> 2][c & 3]) ? 0 : 1;
                scnn::split8(two, fx);
            } else {
                fx[0] = __builtin_bit_cast(u32x4, now[kk]);
            }
#pragma unroll
            for (int j = 0; j < NB; ++j) {
                if (j * 16 >= p.c_out) break;
                if constexpr (SPLIT) {
                    f4 large, small;
                    split_products(fw[kk][j], fx[0], fx[1], fx[2], large, small);
                    acc[j] += large + small;
                } else if constexpr (std::is_same<T, __bf16>::value) {
                    acc[j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, fw[kk][j][0]),
                                                                     __builtin_bit_cast(bf16x8, fx[0]), acc[j], 0, 0, 0);
                } else {
                    acc[j] = __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(h8, fw[kk][j][0]),
                                                                    __builtin_bit_cast(h8, fx[0]), acc[j], 0, 0, 0);
                }
            }
        }
        if constexpr (SPLIT)
            if (__any(odd)) {
                // fp32 products, operands from memory
#pragma unroll
                for (int j = 0; j < NB; ++j) acc[j] = f4{0.f, 0.f, 0.f, 0.f};
                for (int k = 0; k < p.c_in; k += 4) {
                    const float vx = row < rows && k + q < p.c_in ? (float)x[row * p.c_in + k + q] : 0.0f;
#pragma unroll
                    for (int j = 0; j < NB; ++j) {
                        const int n = j * 16 + i16;
                        const float vw = n < p.c_out && k + q < p.c_in ? (float)w[(k + q) * p.c_out + n] : 0.0f;
                        acc[j] = __builtin_amdgcn_mfma_f32_16x16x4f32(vw, vx, acc[j], 0, 0, 0);
                    }
                }
            }
        if (row >= rows) continue;
#pragma unroll
        for (int j = 0; j < NB; ++j) {
            const int n = j * 16 + 4 * q;
            if (n >= p.c_out) break;
            const long long at = row * p.c_out + n;
            auto put = [&](void* to, const V4& v) {
                T* __restrict__ f = (T*)to + at;
                if (aligned4 || n + 4 <= p.c_out) {
                    __builtin_memcpy(f, &v, sizeof(V4));
                } else {
#pragma unroll
                    for (int c = 0; c < 4; ++c)
                        if (n + c < p.c_out) f[c] = v[c];
                }
            };
            f4 z = acc[j];
            V4 v;
#pragma unroll
            for (int c = 0; c < 4; ++c) {
                if (p.bias) z[c] += (float)bias[j][c];
                v[c] = (T)z[c];
            }
            if (p.pre) put(p.pre, v);
            if (p.act != SCNN_ACT_NONE)
#pragma unroll
                for (int c = 0; c < 4; ++c) z[c] = activate(z[c], p.act);
#pragma unroll
            for (int c = 0; c < 4; ++c) {
                if (p.residual) z[c] += (float)residual[j][c];
                v[c] = (T)z[c];
            }
            put(p.out, v);
        }
    }
}

// One to four rows: bound by reading w once.  `lanes` threads (a power of two up to 64) hold 16 bytes each of a row of w,
// every group of them four neighbouring k at a time, against x of the workgroup's k in LDS; fp32 products and sums.  The
// groups' sums meet by lane exchanges and in LDS, those of a split k in k_linear_join.  (Threads that walked down w in strips
// of 64 bytes, a load of x beside each of w, took 86 us for 8 x 4096 by 4096 x 4096 bf16, 216 for 8 x 12288 by 12288 x 1024.)
// (256 threads: 21 us against 11 for 2 x 999 by 999 x 4001 fp32.)
constexpr int kFewK = 1024;  // the most k of a workgroup
template <typename T, int R>
__global__ __launch_bounds__(1024) void k_linear_few(LinearArgs p, int lanes) {
    constexpr int V = kVec<T>;
    __shared__ __align__(16) float s_x[R][kFewK];
    __shared__ float s_sum[16][64 * V];
    const long long m_end = rows_of(p.m, p.rows_dev);
    const long long k_first = (long long)blockIdx.y * p.k_split;
    const int k_count = (int)(p.k - k_first < p.k_split ? p.k - k_first : p.k_split);
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, tc = tid & (lanes - 1), group = tid / lanes, groups = 1024 / lanes;
    const long long n_first = block_id<1024>() * lanes * V, n = n_first + tc * V;
    const int w = (int)(p.n - n < V ? p.n - n : V);
    const T *const x = (const T*)p.a, *const wt = (const T*)p.b + k_first * p.n + n;
#pragma unroll
    for (int r = 0; r < R; ++r)
        for (int k = tid; k < kFewK; k += 1024)
            s_x[r][k] = r < m_end && k < k_count ? (float)x[r * p.k + k_first + k] : 0.0f;
    __syncthreads();
    float acc[R][V];
#pragma unroll
    for (int r = 0; r < R; ++r)
#pragma unroll
        for (int i = 0; i < V; ++i) acc[r][i] = 0.0f;
#pragma unroll 2
    for (int k = group * 4; k < k_count; k += groups * 4) {
        VecOf<T, V> wv[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) wv[j] = load_raw<T>(wt + (long long)(k + j) * p.n, k + j < k_count ? w : 0, p.n >= V);
#pragma unroll
        for (int r = 0; r < R; ++r) {
            const f4 xv = *(const f4*)&s_x[r][k];
#pragma unroll
            for (int j = 0; j < 4; ++j)
#pragma unroll
                for (int i = 0; i < V; ++i) acc[r][i] += xv[j] * (float)wv[j][i];
        }
    }
    for (int d = lanes; d < 64; d <<= 1)  // (all sums a step at a time: an exchange takes a hundred clocks to come back)
#pragma unroll
        for (int r = 0; r < R; ++r)
#pragma unroll
            for (int i = 0; i < V; ++i) acc[r][i] += __shfl_xor(acc[r][i], d, 64);
#pragma unroll
    for (int r = 0; r < R; ++r) {
        if (r >= m_end) break;  // (the same for all threads)
        if (r > 0) __syncthreads();
        if (lane < lanes)
#pragma unroll
            for (int i = 0; i < V; ++i) s_sum[wave][tc * V + i] = acc[r][i];
        __syncthreads();
        const int c = tid * 4;
        const long long col = n_first + c;
        if (c < lanes * V && col < p.n) {
            float z[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int q = 0; q < 16; ++q)
#pragma unroll
                for (int j = 0; j < 4; ++j) z[j] += s_sum[q][c + j];
            if (p.part) {
                float* __restrict__ to = p.part + ((long long)blockIdx.y * p.m + r) * p.n + col;
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    if (col + j < p.n) to[j] = z[j];
            } else {
                finish4<T>(p, r, col, z);
            }
        }
    }
}

// ------------------------------------------------------------------ host side
// Kernel of a product: few rows, tiles staged through registers (any type, width and alignment), or tiles copied to LDS
// (16-bit types, rows that begin on 16 bytes).
enum class TileKind { kFew, kStaged, kStagedGroups, kStaged128, kRing256, kRing128, kRing64x128, kRing64, kRing32 };
struct TilePlan {
    TileKind kind;
    int bm, bn;
    int splits;
    long long k_split;
    int lanes;  // k_linear_few's
};

// The most k that one chain of 16-bit matrix instructions sums: the instruction cuts its sum off downwards at every step
// of 32 k, half a last bit on average, so that 65536 k may leave 2^10 last bits of 2^-24, an eighth of fp16's rounding.
constexpr long long kChain = 65536;

// bf16, best of several launches, us, of 128 x 128 / 64 x 128 / 64 x 64 / 32 x 64 tiles:
//   8192 x 4096 x 4096 (m, n, k)   231 / - / - / -          2048 x 2048 x 2048   29 / 24 / 29 / 37
//   2048 x 2048 x 512             12.3 / 10.7 / 10.9 / 14   1024 x 1024 x 1024   18 / 12.6 / 8.0 / 7.6
//   64 x 1024 x 12288             14.1 / 13.1 / 12.5 / 11.4   16 x 4096 x 4096   12.2 / 10.5 / 12.9 / 9.6
//   3000 x 2000 x 2000              39 / 49 / 60 / 84       5000 x 1304 x 1000   23.8 / 30.8 / 33.7 / 44.7
//   200000 x 64 x 32                31 / 34 / 16 / 23       100000 x 128 x 128   18.4 / 19.4 / 16.1 / 22
// 256 x 256 tiles run one a unit, 128 x 128 two; where the last round of the larger ones is part empty they lose more than they
// save.  us of 256 x 256 / 128 x 128, bf16, 4096 columns, k 4096, by rows (rounds of 256 x 256 tiles on 256 units), without and
// with gelu, residual and pre:
//   7936 (1.94)  224 / 231  272 / 270      8192 (2)     232 / 238  274 / 282      8448 (2.06)  299 / 253  345 / 287
//   10240 (2.5)  314 / 284  377 / 331      11264 (2.75) 329 / 319  386 / 366      11776 (2.88) 334 / 340  393 / 388
//   12288 (3)    342 / 352  405 / 406      14336 (3.5)  441 / 407  510 / 475      16384 (4)    463 / 468  509 / 614
// They are taken from two rounds on, at least 95 per cent full.
// Large tiles read their operands least and pay from five on four compute units (one of 64 x 128 a unit) on, with k to hide
// their start and end, where both sides fill them; short tiles for few rows; else 64 x 64.  k is split where that leaves
// compute units without a tile: one workgroup a unit was the fastest of 1, 2, 4 and 8 at 12 of 16 shapes, within 15 per cent
// of it at the others.
static TilePlan tile_plan(int dtype, long long m, long long n, long long k, bool forward, bool ring) {
    TilePlan t = {TileKind::kStaged, 64, 64, 1, round_up(k < 1 ? 1 : k, 64), 0};
    if (m < 1) return t;
    // us, few rows against tiles, 4096 x 4096: fp32 1 row 17.8, 4 rows 21.4, 8 rows 32.4 / 30; bf16 10.8, 17.2, 25.9 / 10.8
    if (forward && m <= (ring ? 1 : 4) && k <= (1 << 24)) {  // (2^14 workgroups along a split k)
        // Up to kFewK k one launch does, with few lanes a row of w so that there are more workgroups; a longer k is split for
        // two workgroups a compute unit, 64 lanes a row.
        t.kind = TileKind::kFew;
        const int v = dtype == SCNN_F32 ? 4 : 8, most = k > kFewK ? 64 : (n * k <= (1 << 20) ? 4 : 16);
        for (t.lanes = 1; t.lanes < most && (long long)t.lanes * v < n; t.lanes <<= 1) {}
        const long long strips = (n + (long long)t.lanes * v - 1) / ((long long)t.lanes * v), least = 4 * 1024 / t.lanes;
        if (k <= kFewK) {
            t.k_split = kFewK;
        } else {
            t.k_split = round_up(k * strips / (2LL * device_cu_count()) + 1, least);
            if (t.k_split > kFewK) t.k_split = kFewK;
        }
        t.splits = (int)((k + t.k_split - 1) / t.k_split);
        return t;
    }
    const long long cus = device_cu_count();
    auto tiles = [&](long long bm, long long bn) { return ((m + bm - 1) / bm) * ((n + bn - 1) / bn); };
    if (ring) {
        const long long largest = tiles(256, 256), rounds = (largest + cus - 1) / cus;
        if (k >= 512 && m > 128 && n > 128 && rounds >= 2 && 20 * largest >= 19 * rounds * cus) t.kind = TileKind::kRing256, t.bm = t.bn = 256;
        else if (k >= 512 && m > 64 && n > 64 && 4 * tiles(128, 128) >= 5 * cus) t.kind = TileKind::kRing128, t.bm = t.bn = 128;
        else if (k >= 512 && m > 32 && n > 64 && tiles(64, 128) >= cus) t.kind = TileKind::kRing64x128, t.bn = 128;
        else if (m <= 32) t.kind = TileKind::kRing32, t.bm = 32;
        else t.kind = TileKind::kRing64;
    }
    // fp32, us, of 128 x 128 / 64 x 64 / 64 x 64 by four groups of waves, the last with a workgroup a compute unit:
    //   4096 x 4096 x 4096   756 / 928 / 1080 (the library's product 960)   100000 x 128 x 128   39 / 35 / 79
    //   2560 x 2560 x 1024   101 / 111 / 138 (400 tiles of 128 x 128)       3000 x 2000 x 2000   236 / 222 / 249 (384)
    //   1024 x 1024 x 1024    36 / 31 / 22.5    64 x 1024 x 12288    36 / 26 / 24.3    32 x 64 x 200000 (x^T dz)   69 / 32 / 28
    if (!ring) {
        if (k >= 512 && m > 64 && n > 64 && 2 * tiles(128, 128) > 3 * cus) t.kind = TileKind::kStaged128, t.bm = t.bn = 128;
        else if (k >= 256 && tiles(64, 64) < 2 * cus) t.kind = TileKind::kStagedGroups;
    }
    const long long all = tiles(t.bm, t.bn), want = cus;
    if (all < want) {
        long long s = want / all, most = (k + 255) / 256;
        if (s > most) s = most;
        if (s > 1) t.k_split = round_up((k + s - 1) / s, 64);
    }
    if (t.k_split > kChain) t.k_split = kChain;
    t.splits = (int)((k + t.k_split - 1) / t.k_split);
    if (t.splits < 1) t.splits = 1;
    return t;
}

// Workspace of a product's partial sums: it must do for either way of staging, which the arrays' addresses decide.
static size_t part_bytes(int dtype, long long m, long long n, long long k, bool forward) {
    size_t most = 0;
    for (int ring = 0; ring <= (dtype == SCNN_F32 ? 0 : 1); ++ring) {
        const TilePlan t = tile_plan(dtype, m, n, k, forward, ring != 0);
        const size_t b = t.splits > 1 ? (size_t)round_up((long long)t.splits * m * n * 4, 256) : 0;
        if (b > most) most = b;
    }
    return most;
}

template <typename T, bool AK, bool BK_, int BM, int BN, int WM, int WN, int STAGES>
static hipError_t ring(const LinearArgs& p, long long tiles, int splits, hipStream_t s) {
    constexpr int BK = 64, lds = (BM + BN) * BK * 2 * STAGES;
    const dim3 grid = grid_of<64 * WM * WN>(tiles, (unsigned)splits);
    auto kernel = k_linear_ring<T, AK, BK_, BM, BN, BK, WM, WN, STAGES>;
    if (lds >= 65536) {
        const hipError_t e = hipFuncSetAttribute((const void*)kernel, hipFuncAttributeMaxDynamicSharedMemorySize, lds);
        if (e != hipSuccess) return e;
    }
    hipLaunchKernelGGL(kernel, grid, dim3(64 * WM * WN), lds, s, p);
    return hipGetLastError();
}

template <typename T>
static hipError_t join(const LinearArgs& p, int splits, hipStream_t s) {
    const long long quads = p.m * ((p.n + 3) / 4);
    if (splits >= 8)
        hipLaunchKernelGGL((k_linear_join<T, 16>), grid_of<256>((quads + 15) / 16), dim3(256), 0, s, p, splits);
    else
        hipLaunchKernelGGL((k_linear_join<T, 4>), grid_of<256>((quads + 63) / 64), dim3(256), 0, s, p, splits);
    return hipGetLastError();
}

template <typename T>
static hipError_t few_rows(const LinearArgs& p, const TilePlan& t, hipStream_t s) {
    const long long wide = (long long)t.lanes * kVec<T>;
    const dim3 grid = grid_of<1024>((p.n + wide - 1) / wide, (unsigned)t.splits);
    if (p.m == 1) hipLaunchKernelGGL((k_linear_few<T, 1>), grid, dim3(1024), 0, s, p, t.lanes);
    else hipLaunchKernelGGL((k_linear_few<T, 4>), grid, dim3(1024), 0, s, p, t.lanes);
    return hipGetLastError();
}

template <typename T, bool AK, bool BK_>
static hipError_t product(int dtype, LinearArgs p, bool forward, hipStream_t s) {
    bool copies = false;
    if constexpr (sizeof(T) == 2) {
        // rows of both operands begin on 16 bytes, and a tile's rows lie within 32-bit offsets
        const long long wa = AK ? p.k : p.m, wb = BK_ ? p.k : p.n;
        copies = wa % 8 == 0 && wb % 8 == 0 && wa < (1 << 22) && wb < (1 << 22) && ((uintptr_t)p.a & 15) == 0 &&
                 ((uintptr_t)p.b & 15) == 0 && p.n % 8 == 0;
    }
    const TilePlan t = tile_plan(dtype, p.m, p.n, p.k, forward, copies);
    p.k_split = t.k_split;
    if (t.splits <= 1) p.part = nullptr;
    hipError_t e = hipSuccess;
    constexpr int BK = std::is_same<T, float>::value ? 32 : 64;
    const long long tiles = ((p.n + t.bn - 1) / t.bn) * ((p.m + t.bm - 1) / t.bm);
    const dim3 by256 = grid_of<256>(tiles, (unsigned)t.splits), by1024 = grid_of<1024>(tiles, (unsigned)t.splits);
    if (t.kind == TileKind::kFew) {
        e = few_rows<T>(p, t, s);  // (only the forward product is planned so)
    } else if (t.kind == TileKind::kStaged) {
        hipLaunchKernelGGL((k_linear_tile<T, AK, BK_, 64, 64, BK, 2, 2, 1>), by256, dim3(256), 0, s, p);
        e = hipGetLastError();
    } else if (t.kind == TileKind::kStagedGroups) {
        hipLaunchKernelGGL((k_linear_tile<T, AK, BK_, 64, 64, BK, 2, 2, 4>), by1024, dim3(1024), 0, s, p);
        e = hipGetLastError();
    } else if (t.kind == TileKind::kStaged128) {
        hipLaunchKernelGGL((k_linear_tile<T, AK, BK_, 128, 128, BK, 2, 2, 1>), by256, dim3(256), 0, s, p);
        e = hipGetLastError();
    } else if constexpr (sizeof(T) == 2) {
        if (t.kind == TileKind::kRing256) e = ring<T, AK, BK_, 256, 256, 2, 4, 2>(p, tiles, t.splits, s);
        else if (t.kind == TileKind::kRing128) e = ring<T, AK, BK_, 128, 128, 2, 2, 2>(p, tiles, t.splits, s);
        else if (t.kind == TileKind::kRing64x128) e = ring<T, AK, BK_, 64, 128, 2, 2, 3>(p, tiles, t.splits, s);
        else if (t.kind == TileKind::kRing64) e = ring<T, AK, BK_, 64, 64, 2, 2, 2>(p, tiles, t.splits, s);
        else e = ring<T, AK, BK_, 32, 64, 1, 4, 4>(p, tiles, t.splits, s);
    }
    if (e != hipSuccess || t.splits <= 1) return e;
    return join<T>(p, t.splits, s);
}

// Widths that k_linear_fwd_narrow takes (w in registers).
static bool narrow_forward(long long c_in, long long c_out) { return c_in <= 32 && c_out <= 32; }

// Widths that k_linear_bwd_narrow takes (w and 64 rows of x and dz in LDS): its P, 0 for wider layers.
static int narrow_width(long long c_in, long long c_out) {
    const long long c = c_in > c_out ? c_in : c_out;
    if (c <= 32) return 32;
    return c <= 64 ? 64 : 0;  // (128, 16-bit types: 69 us against 57 for its three products apart on 100000 rows of 128 -> 128)
}

template <typename T>
static hipError_t narrow_fwd(const LinearCall& c, hipStream_t s) {
    NarrowFwdArgs p = {};
    p.x = c.x; p.w = c.w; p.bias = c.bias; p.residual = c.residual; p.out = c.out; p.pre = c.pre;
    p.rows = c.rows;
    p.rows_dev = c.rows_dev;
    p.c_in = (int)c.c_in; p.c_out = (int)c.c_out; p.act = c.act;
    long long blocks = (c.rows + 63) / 64;
    const long long most = 4LL * device_cu_count();
    if (blocks > most) blocks = most;
    hipLaunchKernelGGL((k_linear_fwd_narrow<T, 32>), dim3((unsigned)blocks), dim3(256), 0, s, p);
    return hipGetLastError();
}

size_t linear_fwd_part_bytes(int dtype, long long rows, long long c_in, long long c_out) {
    if (rows > 4 && narrow_forward(c_in, c_out)) return 0;
    return part_bytes(dtype, rows, c_out, c_in, true);
}

hipError_t launch_linear_fwd(int dtype, const LinearCall& c, hipStream_t s) {
    if (c.rows < 1) return hipSuccess;
    LinearArgs p = {};
    p.a = c.x; p.b = c.w;
    p.m = c.rows; p.n = c.c_out; p.k = c.c_in;
    p.rows_dev = c.rows_dev;
    p.bias = c.bias; p.residual = c.residual; p.out = c.out; p.pre = c.pre;
    p.part = (float*)c.workspace;
    p.act = c.act;
    if (p.m > 4 && narrow_forward(c.c_in, c.c_out)) {
        switch (dtype) {
            case SCNN_F32: return narrow_fwd<float>(c, s);
            case SCNN_BF16: return narrow_fwd<__bf16>(c, s);
            default: return narrow_fwd<_Float16>(c, s);
        }
    }
    switch (dtype) {
        case SCNN_F32: return product<float, true, false>(dtype, p, true, s);
        case SCNN_BF16: return product<__bf16, true, false>(dtype, p, true, s);
        default: return product<_Float16, true, false>(dtype, p, true, s);
    }
}

// Row slices of k_act_back and its block's width in threads.
struct BackPlan { int tn, parts; };
static BackPlan back_plan(long long rows, long long cols, int dtype) {
    const int v = dtype == SCNN_F32 ? 4 : 8;
    BackPlan b = {1, 1};
    while (b.tn < 64 && (long long)b.tn * v < cols) b.tn <<= 1;
    const long long strips = (cols + (long long)b.tn * v - 1) / ((long long)b.tn * v), nr = 256 / b.tn;
    long long parts = 4LL * device_cu_count() / strips;
    const long long need = (rows + nr - 1) / nr;
    if (parts > need) parts = need;
    b.parts = (int)(parts < 1 ? 1 : parts);
    return b;
}

// Two workgroups a compute unit, but at least two tiles of 64 rows each, and no longer chains than kChain rows.
static int narrow_groups(long long rows) {
    long long n = (rows + 127) / 128, most = 2LL * device_cu_count();
    if (most < (rows + kChain - 1) / kChain) most = (rows + kChain - 1) / kChain;
    if (n > most) n = most;
    return (int)(n < 1 ? 1 : n);
}

template <typename T>
static hipError_t narrow_bwd(int dtype, const LinearCall& c, int width, hipStream_t s) {
    NarrowArgs p = {};
    p.x = c.dw ? c.x : nullptr; p.w = c.w; p.pre = c.pre_in; p.g = c.g; p.dx = c.rows > 0 ? c.dx : nullptr;
    p.part = c.dw || c.dbias ? (float*)c.workspace : nullptr;
    p.rows = c.rows;
    p.rows_dev = c.rows_dev;
    p.c_in = (int)c.c_in; p.c_out = (int)c.c_out; p.act = c.act;
    if (!p.part && !p.dx) return hipSuccess;
    const int groups = narrow_groups(c.rows);
    constexpr bool PARTS = sizeof(T) == 2;
    const bool fine = PARTS && (c.act == SCNN_ACT_GELU || c.act == SCNN_ACT_SILU);
    auto kernel = width == 32 ? (fine ? k_linear_bwd_narrow<T, 32, PARTS> : k_linear_bwd_narrow<T, 32, false>)
                              : (fine ? k_linear_bwd_narrow<T, 64, PARTS> : k_linear_bwd_narrow<T, 64, false>);
    const int threads = width == 32 ? NarrowShape<sizeof(T), 32>::NT : NarrowShape<sizeof(T), 64>::NT;
    hipLaunchKernelGGL(kernel, dim3(groups), dim3(threads), 0, s, p);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess || !p.part) return e;
    const long long filter = c.c_in * c.c_out;
    return launch_column_sums(p.part, groups, filter + c.c_out, filter, c.dw, c.dbias, dtype, s);
}

// fp16 gradients of gelu and silu hold a scaled dz.
static bool scaled_dz(int dtype, int act) { return dtype == SCNN_F16 && (act == SCNN_ACT_GELU || act == SCNN_ACT_SILU); }

struct BackSpace { size_t dz, peak, sums, dx, dw, total; };
static BackSpace back_space(int dtype, long long rows, long long c_in, long long c_out, int act) {
    BackSpace b = {};
    const size_t e = dtype == SCNN_F32 ? 4 : 2;
    size_t at = 0;
    b.dz = at;
    if (act != SCNN_ACT_NONE) at += (size_t)round_up(rows * c_out * (long long)e, 256);
    b.peak = at;  // (behind the peaks: the inverse of the scale)
    if (scaled_dz(dtype, act)) at += round_up((kPeaks + 1) * 4, 256);
    b.sums = at;
    at += (size_t)round_up((long long)back_plan(rows, c_out, dtype).parts * c_out * 4, 256);
    b.dx = b.dw = at;  // (the two products run one after the other and share their partial sums' place)
    const size_t dx = part_bytes(dtype, rows, c_in, c_out, false), dw = part_bytes(dtype, c_in, c_out, rows, false);
    b.total = at + (dx > dw ? dx : dw);
    return b;
}

size_t linear_bwd_bytes(int dtype, long long rows, long long c_in, long long c_out, int act) {
    if (narrow_width(c_in, c_out) != 0)
        return (size_t)round_up((long long)narrow_groups(rows) * (c_in * c_out + c_out) * 4, 256);
    return back_space(dtype, rows, c_in, c_out, act).total;
}

template <typename T>
static hipError_t linear_bwd_typed(int dtype, const LinearCall& c, hipStream_t s) {
    if (const int width = narrow_width(c.c_in, c.c_out)) return narrow_bwd<T>(dtype, c, width, s);
    const BackSpace at = back_space(dtype, c.rows, c.c_in, c.c_out, c.act);
    char* const ws = (char*)c.workspace;
    const void* dz = c.g;
    if (c.act != SCNN_ACT_NONE) dz = ws + at.dz;
    const bool products = c.dx || c.dw;
    LinearArgs p = {};
    unsigned* peak = nullptr;
    int peaks = 0;
    if constexpr (std::is_same<T, _Float16>::value)
        if (products && scaled_dz(dtype, c.act)) {
            peak = (unsigned*)(ws + at.peak);
            p.scale = (const float*)(peak + kPeaks);
            const long long need = (c.rows * c.c_out + kPeakThreads * 8 - 1) / (kPeakThreads * 8);
            peaks = (int)(need < 1 ? 1 : (need < kPeaks ? need : kPeaks));
            hipLaunchKernelGGL(k_grad_peak, dim3((unsigned)peaks), dim3(kPeakThreads), 0, s, (const _Float16*)c.g, c.rows, c.rows_dev,
                               c.c_out, peak);
        }
    if (c.dbias || (products && c.act != SCNN_ACT_NONE)) {
        const BackPlan b = back_plan(c.rows, c.c_out, dtype);
        const long long wide = (long long)b.tn * kVec<T>;
        float* const sums = c.dbias ? (float*)(ws + at.sums) : nullptr;
        hipLaunchKernelGGL((k_act_back<T>), dim3((unsigned)((c.c_out + wide - 1) / wide), (unsigned)b.parts), dim3(256), 0, s,
                           (const T*)c.g, (const T*)c.pre_in, c.rows, c.rows_dev, c.c_out, c.act, b.tn, (T*)(ws + at.dz), sums,
                           peak, peaks, (float*)p.scale);
        if (c.dbias) {
            const hipError_t e = launch_column_sums(sums, b.parts, c.c_out, c.c_out, c.dbias, nullptr, dtype, s);
            if (e != hipSuccess) return e;
        }
    }
    p.rows_dev = c.rows_dev;
    p.act = SCNN_ACT_NONE;
    if (c.dx && c.rows > 0) {
        p.a = dz; p.b = c.w; p.out = c.dx;
        p.m = c.rows; p.n = c.c_in; p.k = c.c_out;
        p.part = (float*)(ws + at.dx);
        const hipError_t e = product<T, true, true>(dtype, p, false, s);
        if (e != hipSuccess) return e;
    }
    if (c.dw) {
        p.a = c.x; p.b = dz; p.out = c.dw;
        p.m = c.c_in; p.n = c.c_out; p.k = c.rows;
        p.rows_k = 1;
        p.part = (float*)(ws + at.dw);
        return product<T, false, false>(dtype, p, false, s);
    }
    return hipGetLastError();
}

hipError_t launch_linear_bwd(int dtype, const LinearCall& c, hipStream_t s) {
    switch (dtype) {
        case SCNN_F32: return linear_bwd_typed<float>(dtype, c, s);
        case SCNN_BF16: return linear_bwd_typed<__bf16>(dtype, c, s);
        default: return linear_bwd_typed<_Float16>(dtype, c, s);
    }
}

}  // namespace scnn
