// Group norm with an activation over the samples of rows [rows, C], forward and backward, and where the samples begin.
//
// Sample b has the rows offsets[b] .. offsets[b + 1] - 1, group j the columns j C/G .. (j + 1) C/G - 1, n = rows of b times C/G.
//   mean = sum x / n,  var = sum (x - mean)^2 / n,  rstd = 1 / sqrt(var + eps),  xh = (x - mean) rstd,  z = xh gamma + beta
//   out = act(z)
//   dz = g act'(z),  h = dz gamma,  dx = rstd (h - sum(h) / n - xh sum(h xh) / n)   (sums over the sample's group),
//   dgamma = sum_r dz xh,  dbeta = sum_r dz
//
// Bound by memory.  A sample is as long as it likes and its group's sums have to be known before its first result: the rows are
// read twice, in three launches: sums over blocks of rows (k_group_sums, k_group_back_sums), the blocks' sums joined for each
// sample and group (k_group_join, k_group_back_join), results (k_group_apply, k_group_back).  Short calls do all of it in one
// workgroup a sample (k_group_one, k_group_back_one), which finds its rows in the L2 the second time.
//
// Blocks of rows are cut without regard to the samples, whose sizes only the device knows: block i keeps one set of sums for
// every sample that it meets, in place i + b (along the rows either i or b grows by one, so that no place is taken twice), and
// sets what no pair (i, b) takes to 0.  Sums are added in a fixed order: the same bits every time.
// The forward sums are those of x - s and its square, s the first value of the sample's group, in fp64: what cancels in
// var = (sum d^2 - (sum d)^2 / n) / n is then bits that fp64 has to spare (a spread of 1e-5 of the distance between s and the
// mean leaves 2^-53 x 1e10 of it), and a group of equal values has exactly none.
#include "scnn_dense.h"

namespace scnn {

constexpr int kGroupThreads = 512;
constexpr int kOneThreads = 256;  // of a workgroup that does a sample by itself

// How threads lie over columns.  A workgroup takes `wide` columns from c0 on: tv threads a row, a vector each, `reps` rows at
// a time.  Rows of all C columns that are no whole number of vectors run on without a gap (flat): `active` vectors are `reps`
// whole rows, so that a thread meets the same columns at every step.  Either way value (thread, i) is number thread V + i of a
// step, and row k's column c number k pitch + c.
struct GroupLayout {
    int tv, reps, active, pitch, flat;
    int wide, slabs, pieces;  // a slab is whole groups (pieces 1), or one of `pieces` pieces of a group
};

struct GroupArgs {
    const void *x, *g, *gamma, *beta;
    void* out;             // forward: out, backward: dx
    float *mean, *rstd;    // [batch][groups]: written forward, read backward
    const long long* offsets;
    long long each;        // rows of a sample where offsets is null
    long long rows, chunk; // of a block
    long long batch, blocks, places;
    int channels, groups, per, act;
    float eps;
    void* part;            // places x: forward double [groups * pieces][2], backward float [2][channels]
    void* stat;            // [batch][groups]: forward {mean, rest, rstd, -}, backward {sum h / n, sum h xh / n}
    int parts_wanted;      // backward: dgamma or dbeta are
    GroupLayout l;
};

__device__ __forceinline__ long long first_row(const GroupArgs& p, long long b) {
    if (!p.offsets) return b * p.each;
    const long long r = p.offsets[b];
    return r < 0 ? 0 : (r < p.rows ? r : p.rows);
}
__device__ __forceinline__ long long end_row(const GroupArgs& p, long long b, long long first) {
    const long long r = first_row(p, b + 1);
    return r < first ? first : r;
}

// Number of the ascending keys key(0 .. n - 1) that are below or at `limit`, by a wave: 64 of them are asked at once.
template <typename F>
__device__ __forceinline__ long long count_up_to(long long n, long long limit, F key) {
    const int lane = threadIdx.x & 63;
    long long lo = 0, hi = n;
    while (hi - lo > 64) {
        const long long step = (hi - lo + 63) / 64, at = lo + (lane + 1) * step - 1;
        const int c = __popcll(__ballot(at < hi && key(at) <= limit));
        lo += c * step;
        if (lo > hi) lo = hi;
        if (lo + step - 1 < hi) hi = lo + step - 1;
    }
    return lo + __popcll(__ballot(lo + lane < hi && key(lo + lane) <= limit));
}

// The sample that row `r` lies in or, between samples, the next one; at most the last.
__device__ __forceinline__ long long sample_at(const GroupArgs& p, long long r) {
    long long b;
    if (!p.offsets) b = p.each > 0 ? r / p.each : 0;
    else b = count_up_to(p.batch, r, [&](long long k) { return first_row(p, k + 1); });
    return b < p.batch ? b : p.batch - 1;
}

// A thread's vectors among the rows lo .. hi - 1: `full` whole ones, then `part` of n values.
struct Walk {
    long long at, step;
    int full, part, n;
};
template <int V>
__device__ __forceinline__ Walk walk_of(const GroupArgs& p, int c0, int c1, long long lo, long long hi) {
    const int t = threadIdx.x;
    Walk w = {0, 0, 0, 0, 0};
    if (t >= p.l.active || hi <= lo) return w;
    if (p.l.flat) {
        const long long all = (hi - lo) * p.channels, mine = all - (long long)t * V;
        w.at = lo * p.channels + (long long)t * V;
        w.step = (long long)p.l.active * V;
        if (mine <= 0) return w;
        w.full = (int)(mine >= V ? (mine - V) / w.step + 1 : 0);
        const long long left = mine - w.full * w.step;
        if (left > 0) w.part = 1, w.n = (int)left;
    } else {
        const int k = t / p.l.tv, c = c0 + (t - k * p.l.tv) * V, n = c1 - c;
        w.at = (lo + k) * p.channels + c;
        w.step = (long long)p.l.reps * p.channels;
        const long long rows = hi - lo - k;
        if (n <= 0 || rows <= 0) return w;
        const int count = (int)((rows - 1) / p.l.reps + 1);
        if (n >= V) w.full = count;
        else w.part = count, w.n = n;
    }
    return w;
}

// Calls body(position, number of values) for a thread's vectors, U at a time: take() loads, then use().
template <int U, typename Take, typename Use, typename Part>
__device__ __forceinline__ void walk(const Walk& w, Take take, Use use, Part part) {
    long long at = w.at;
    int k = 0;
    for (; k + U <= w.full; k += U, at += U * w.step) {
#pragma unroll
        for (int u = 0; u < U; ++u) take(u, at + u * w.step);
#pragma unroll
        for (int u = 0; u < U; ++u) use(u, at + u * w.step);
    }
    for (; k < w.full; ++k, at += w.step) {
        take(0, at);
        use(0, at);
    }
    for (k = 0; k < w.part; ++k, at += w.step)
        for (int i = 0; i < w.n; ++i) part(i, at + i);
}

// Columns of this workgroup's slab, its first group and the number of its groups.
struct Slab { int c0, c1, j0, ng; };
__device__ __forceinline__ Slab slab_of(const GroupArgs& p) {
    const int s = blockIdx.y;
    Slab a;
    if (p.l.pieces > 1) {
        a.j0 = s / p.l.pieces;
        a.ng = 1;
        a.c0 = a.j0 * p.per + (s - a.j0 * p.l.pieces) * p.l.wide;
        a.c1 = a.c0 + p.l.wide < (a.j0 + 1) * p.per ? a.c0 + p.l.wide : (a.j0 + 1) * p.per;
    } else {
        a.c0 = s * p.l.wide;
        a.c1 = a.c0 + p.l.wide < p.channels ? a.c0 + p.l.wide : p.channels;
        a.j0 = a.c0 / p.per;
        a.ng = (a.c1 - a.c0) / p.per;
    }
    return a;
}

// Group of value i of this thread.  (Values past the slab's end take its last one.)
__device__ __forceinline__ int group_of(const GroupArgs& p, const Slab& a, int t, int i, int v) {
    int c;
    if (p.l.flat) c = (t * v + i) % p.channels;
    else c = a.c0 + t % p.l.tv * v + i;
    if (c >= a.c1) c = a.c1 - 1;
    return p.l.pieces > 1 ? a.j0 : c / p.per;
}
__device__ __forceinline__ int column_of(const GroupArgs& p, const Slab& a, int t, int i, int v) {
    const int c = p.l.flat ? (t * v + i) % p.channels : a.c0 + t % p.l.tv * v + i;
    return c < a.c1 ? c : a.c1 - 1;
}

__device__ __forceinline__ float finite_or_zero(float v) { return __builtin_fabsf(v) < __builtin_huge_valf() ? v : 0.0f; }

// Power of two of lanes that add n values: at most a wave.
__device__ __forceinline__ int lanes_for(int n) {
    int q = 1;
    while (q < n && q < 64) q <<= 1;
    return q;
}

// Sums over the slab's groups of per-value numbers: value (thread, i) of all threads in s_all, then done(group, sum) by one lane a
// group.  All threads of the workgroup call it.
template <int V, typename F>
__device__ __forceinline__ void add_groups(const GroupArgs& p, const Slab& a, const double (&v)[V], double* s_all, F done) {
    __syncthreads();
    if ((int)threadIdx.x < p.l.active)
#pragma unroll
        for (int i = 0; i < V; ++i) s_all[threadIdx.x * V + i] = v[i];
    __syncthreads();
    const int w = p.l.pieces > 1 ? a.c1 - a.c0 : p.per, n = w * p.l.reps, q = lanes_for(n);
    const int set = threadIdx.x / q, sets = blockDim.x / q, in = threadIdx.x & (q - 1);
    for (int j0 = 0; j0 < a.ng; j0 += sets) {
        const int j = j0 + set;
        double sum = 0.0;
        if (j < a.ng)
            for (int e = in; e < n; e += q) {
                const int k = e / w;
                sum += s_all[k * p.l.pitch + j * w + (e - k * w)];
            }
        for (int d = 1; d < q; d <<= 1) sum += __shfl_xor(sum, d, 64);
        if (in == 0 && j < a.ng) done(j, sum);
    }
}

// Sums of d = x - s and of d^2 over the rows lo .. hi - 1, s the first value of each group in row `origin`.
template <typename T>
__device__ __forceinline__ void forward_sums(const GroupArgs& p, const Slab& a, long long origin, long long lo, long long hi,
                                             double (&s1)[kVec<T>], double (&s2)[kVec<T>]) {
    constexpr int V = kVec<T>, U = 4;
    const T* __restrict__ x = (const T*)p.x;
    double s[V];
#pragma unroll
    for (int i = 0; i < V; ++i) {
        s1[i] = s2[i] = 0.0;
        s[i] = (double)finite_or_zero((float)x[origin * p.channels + (long long)group_of(p, a, threadIdx.x, i, V) * p.per]);
    }
    VecOf<T, V> r[U];
    walk<U>(walk_of<V>(p, a.c0, a.c1, lo, hi), [&](int u, long long at) { __builtin_memcpy(&r[u], x + at, 16); },
            [&](int u, long long) {
#pragma unroll
                for (int i = 0; i < V; ++i) {
                    const double d = (double)(float)r[u][i] - s[i];
                    s1[i] += d;
                    s2[i] = __builtin_fma(d, d, s2[i]);
                }
            },
            [&](int i, long long at) {
                const double v = (double)(float)x[at];
#pragma unroll
                for (int c = 0; c < V; ++c)
                    if (c == i) {
                        const double d = v - s[c];
                        s1[c] += d;
                        s2[c] = __builtin_fma(d, d, s2[c]);
                    }
            });
}

struct GroupStat { float mean, rest, rstd, none; };
// Statistics of n values from their sums about s.
__device__ __forceinline__ GroupStat stat_of(double s, double s1, double s2, double n, float eps) {
    const double off = s1 / n, mean = s + off;
    double var = (s2 - s1 * off) / n;
    if (var < 0.0) var = 0.0;  // (a NaN stays one)
    GroupStat r;
    r.mean = (float)mean;
    r.rest = (float)(mean - (double)r.mean);
    r.rstd = (float)(1.0 / sqrt(var + (double)eps));
    r.none = 0.0f;
    return r;
}

// Results of the rows lo .. hi - 1 of a sample whose statistics are stat[group - first].
template <typename T>
__device__ __forceinline__ void forward_rows(const GroupArgs& p, const Slab& a, const GroupStat* stat, int first, long long lo,
                                             long long hi) {
    constexpr int V = kVec<T>, U = 4;
    const T* __restrict__ x = (const T*)p.x;
    T* __restrict__ out = (T*)p.out;
    float mean[V], rest[V], scale[V], beta[V];
#pragma unroll
    for (int i = 0; i < V; ++i) {
        const GroupStat s = stat[group_of(p, a, threadIdx.x, i, V) - first];
        const int c = column_of(p, a, threadIdx.x, i, V);
        mean[i] = s.mean;
        rest[i] = s.rest;
        scale[i] = p.gamma ? s.rstd * (float)((const T*)p.gamma)[c] : s.rstd;
        beta[i] = p.beta ? (float)((const T*)p.beta)[c] : 0.0f;
    }
    VecOf<T, V> r[U];
    walk<U>(walk_of<V>(p, a.c0, a.c1, lo, hi), [&](int u, long long at) { __builtin_memcpy(&r[u], x + at, 16); },
            [&](int u, long long at) {
                VecOf<T, V> y;
#pragma unroll
                for (int i = 0; i < V; ++i)
                    y[i] = (T)activate(__builtin_fmaf(((float)r[u][i] - mean[i]) - rest[i], scale[i], beta[i]), p.act);
                __builtin_memcpy(out + at, &y, 16);
            },
            [&](int i, long long at) {
                const float v = (float)x[at];
#pragma unroll
                for (int c = 0; c < V; ++c)
                    if (c == i) out[at] = (T)activate(__builtin_fmaf((v - mean[c]) - rest[c], scale[c], beta[c]), p.act);
            });
}

// Rows of block i, and the samples whose sums it keeps.
struct Block { long long r0, r1, b0, b1; };
__device__ __forceinline__ Block block_of(const GroupArgs& p, long long i) {
    Block k;
    k.r0 = i * p.chunk;
    k.r1 = k.r0 + p.chunk < p.rows ? k.r0 + p.chunk : p.rows;
    k.b0 = i == 0 ? 0 : sample_at(p, k.r0);
    k.b1 = i + 1 == p.blocks ? p.batch - 1 : sample_at(p, k.r1);
    return k;
}

template <typename T>
__global__ __launch_bounds__(kGroupThreads) void k_group_sums(GroupArgs p) {
    constexpr int V = kVec<T>;
    __shared__ double s_all[kGroupThreads * V];
    const long long i = block_id<kGroupThreads>();
    if (i >= p.blocks) return;
    const Slab a = slab_of(p);
    const Block k = block_of(p, i);
    const int to = p.l.pieces > 1 ? (int)blockIdx.y : a.j0;
    for (long long b = k.b0; b <= k.b1; ++b) {
        const long long first = first_row(p, b), end = end_row(p, b, first);
        const long long lo = first > k.r0 ? first : k.r0, hi = end < k.r1 ? end : k.r1;
        double* const part = (double*)p.part + ((i + b) * p.groups * p.l.pieces + to) * 2;
        if (hi <= lo) {
            for (int j = threadIdx.x; j < 2 * a.ng; j += blockDim.x) part[j] = 0.0;
            continue;
        }
        double s1[V], s2[V];
        forward_sums<T>(p, a, first, lo, hi, s1, s2);
        add_groups<V>(p, a, s1, s_all, [&](int j, double sum) { part[2 * j] = sum; });
        add_groups<V>(p, a, s2, s_all, [&](int j, double sum) { part[2 * j + 1] = sum; });
    }
}

// Sum over the Q threads (a power of two up to 256) of each of a workgroup's sets; all 256 threads call it.
__device__ __forceinline__ double set_add(double v, int q, double* s_wave) {
    for (int d = 1; d < q && d < 64; d <<= 1) v += __shfl_xor(v, d, 64);
    if (q <= 64) return v;
    __syncthreads();
    if ((threadIdx.x & 63) == 0) s_wave[threadIdx.x >> 6] = v;
    __syncthreads();
    const int w = threadIdx.x / q * (q / 64);
    v = 0.0;
    for (int k = 0; k < q / 64; ++k) v += s_wave[w + k];
    return v;
}

// Q threads for each sample and group.
template <typename T>
__global__ __launch_bounds__(256) void k_group_join(GroupArgs p, int q) {
    __shared__ double s_wave[4];
    const long long id = block_id<256>() * (256 / q) + threadIdx.x / q;
    const int in = threadIdx.x & (q - 1);
    const bool live = id < p.batch * p.groups;
    const long long b = live ? id / p.groups : 0;
    const int j = (int)(live ? id % p.groups : 0);
    const long long first = first_row(p, b), end = end_row(p, b, first);
    double s1 = 0.0, s2 = 0.0;
    if (live && end > first) {
        const long long n = ((end - 1) / p.chunk - first / p.chunk + 1) * p.l.pieces;
        const double* __restrict__ part = (const double*)p.part;
        const long long from = (first / p.chunk + b) * p.l.pieces * p.groups + (long long)j * p.l.pieces;
#pragma unroll 4
        for (long long e = in; e < n; e += q) {
            const long long i = p.l.pieces > 1 ? e / p.l.pieces : e;
            const double* at = part + (from + i * p.l.pieces * p.groups + (e - i * p.l.pieces)) * 2;
            s1 += at[0];
            s2 += at[1];
        }
    }
    s1 = set_add(s1, q, s_wave);
    s2 = set_add(s2, q, s_wave);
    if (!live || in != 0) return;
    GroupStat r = {0.0f, 0.0f, 0.0f, 0.0f};
    if (end > first) {
        const float s = finite_or_zero((float)((const T*)p.x)[first * p.channels + (long long)j * p.per]);
        r = stat_of((double)s, s1, s2, (double)(end - first) * p.per, p.eps);
    }
    ((GroupStat*)p.stat)[id] = r;
    if (p.mean) p.mean[id] = r.mean;
    if (p.rstd) p.rstd[id] = r.rstd;
}

template <typename T>
__global__ __launch_bounds__(kGroupThreads) void k_group_apply(GroupArgs p) {
    const long long i = block_id<kGroupThreads>();
    if (i >= p.blocks) return;
    const Slab a = slab_of(p);
    const Block k = block_of(p, i);
    for (long long b = k.b0; b <= k.b1; ++b) {
        const long long first = first_row(p, b), end = end_row(p, b, first);
        const long long lo = first > k.r0 ? first : k.r0, hi = end < k.r1 ? end : k.r1;
        if (hi > lo) forward_rows<T>(p, a, (const GroupStat*)p.stat + b * p.groups, 0, lo, hi);
    }
}

// A sample's slab of whole groups by one workgroup.
template <typename T>
__global__ __launch_bounds__(kOneThreads) void k_group_one(GroupArgs p) {
    constexpr int V = kVec<T>;
    __shared__ double s_all[kOneThreads * V];
    __shared__ union { double sum; GroupStat stat; } s_group[kOneThreads * V];
    const long long b = block_id<kOneThreads>();
    if (b >= p.batch) return;
    const Slab a = slab_of(p);
    const long long first = first_row(p, b), end = end_row(p, b, first), id = b * p.groups + a.j0;
    const T* __restrict__ x = (const T*)p.x;
    if (end > first) {
        double s1[V], s2[V];
        forward_sums<T>(p, a, first, first, end, s1, s2);
        add_groups<V>(p, a, s1, s_all, [&](int j, double sum) { s_group[j].sum = sum; });
        add_groups<V>(p, a, s2, s_all, [&](int j, double sum) {
            const float s = finite_or_zero((float)x[first * p.channels + (long long)(a.j0 + j) * p.per]);
            s_group[j].stat = stat_of((double)s, s_group[j].sum, sum, (double)(end - first) * p.per, p.eps);
        });
        __syncthreads();
        forward_rows<T>(p, a, &s_group[0].stat, a.j0, first, end);
    }
    for (int j = threadIdx.x; j < a.ng; j += blockDim.x) {
        if (p.mean) p.mean[id + j] = end > first ? s_group[j].stat.mean : 0.0f;
        if (p.rstd) p.rstd[id + j] = end > first ? s_group[j].stat.rstd : 0.0f;
    }
}

// What the backward pass knows of a thread's columns.
template <int V>
struct BackColumns { float mean[V], rstd[V], gamma[V], beta[V]; };
template <typename T>
__device__ __forceinline__ BackColumns<kVec<T>> back_columns(const GroupArgs& p, const Slab& a, long long b) {
    constexpr int V = kVec<T>;
    BackColumns<V> k;
#pragma unroll
    for (int i = 0; i < V; ++i) {
        const long long s = b * p.groups + group_of(p, a, threadIdx.x, i, V);
        const int c = column_of(p, a, threadIdx.x, i, V);
        k.mean[i] = p.mean[s];
        k.rstd[i] = p.rstd[s];
        k.gamma[i] = p.gamma ? (float)((const T*)p.gamma)[c] : 1.0f;
        k.beta[i] = p.beta ? (float)((const T*)p.beta)[c] : 0.0f;
    }
    return k;
}
// xh and dz of a value.  relu's slope hangs on the sign of z alone, which is found in fp64: in fp32 one value in some ten
// million lies on the wrong side and takes a whole gradient with it.
template <int V>
__device__ __forceinline__ void back_value(const BackColumns<V>& k, int i, float x, float g, int act, float& xh, float& dz) {
    const float d = x - k.mean[i];
    xh = d * k.rstd[i];
    if (act == SCNN_ACT_RELU) {
        const double z = __builtin_fma(((double)x - (double)k.mean[i]) * (double)k.rstd[i], (double)k.gamma[i], (double)k.beta[i]);
        dz = z <= 0.0 ? 0.0f : g;
    } else {
        dz = activate_back(g, __builtin_fmaf(xh, k.gamma[i], k.beta[i]), act);
    }
}

template <typename T>
__device__ __forceinline__ void backward_sums(const GroupArgs& p, const Slab& a, const BackColumns<kVec<T>>& k, long long lo,
                                              long long hi, float (&da)[kVec<T>], float (&db)[kVec<T>]) {
    constexpr int V = kVec<T>, U = 2;
    const T *__restrict__ x = (const T*)p.x, *__restrict__ g = (const T*)p.g;
#pragma unroll
    for (int i = 0; i < V; ++i) da[i] = db[i] = 0.0f;
    VecOf<T, V> r[U], q[U];
    walk<U>(walk_of<V>(p, a.c0, a.c1, lo, hi),
            [&](int u, long long at) {
                __builtin_memcpy(&r[u], x + at, 16);
                __builtin_memcpy(&q[u], g + at, 16);
            },
            [&](int u, long long) {
#pragma unroll
                for (int i = 0; i < V; ++i) {
                    float xh, dz;
                    back_value<V>(k, i, (float)r[u][i], (float)q[u][i], p.act, xh, dz);
                    da[i] = __builtin_fmaf(dz, xh, da[i]);
                    db[i] += dz;
                }
            },
            [&](int i, long long at) {
                const float v = (float)x[at], w = (float)g[at];
#pragma unroll
                for (int c = 0; c < V; ++c)
                    if (c == i) {
                        float xh, dz;
                        back_value<V>(k, c, v, w, p.act, xh, dz);
                        da[c] = __builtin_fmaf(dz, xh, da[c]);
                        db[c] += dz;
                    }
            });
}

// Sums over a step's rows: done(column of the slab, sum).
template <int V, typename F>
__device__ __forceinline__ void add_columns(const GroupArgs& p, const Slab& a, const float (&v)[V], float* s_all, F done) {
    __syncthreads();
    if ((int)threadIdx.x < p.l.active)
#pragma unroll
        for (int i = 0; i < V; ++i) s_all[threadIdx.x * V + i] = v[i];
    __syncthreads();
    for (int c = threadIdx.x; c < a.c1 - a.c0; c += blockDim.x) {
        float sum = s_all[c];
        for (int k = 1; k < p.l.reps; ++k) sum += s_all[k * p.l.pitch + c];
        done(c, sum);
    }
}

// stat: {sum h / n, sum h xh / n} of group - first.
template <typename T>
__device__ __forceinline__ void backward_rows(const GroupArgs& p, const Slab& a, const BackColumns<kVec<T>>& k, const float2* stat,
                                              int first, long long lo, long long hi) {
    constexpr int V = kVec<T>, U = 2;
    const T *__restrict__ x = (const T*)p.x, *__restrict__ g = (const T*)p.g;
    T* __restrict__ dx = (T*)p.out;
    float m_h[V], m_hx[V];
#pragma unroll
    for (int i = 0; i < V; ++i) {
        const float2 s = stat[group_of(p, a, threadIdx.x, i, V) - first];
        m_h[i] = s.x;
        m_hx[i] = s.y;
    }
    auto value = [&](int i, float v, float w) {
        float xh, dz;
        back_value<V>(k, i, v, w, p.act, xh, dz);
        return k.rstd[i] * (dz * k.gamma[i] - m_h[i] - xh * m_hx[i]);
    };
    VecOf<T, V> r[U], q[U];
    walk<U>(walk_of<V>(p, a.c0, a.c1, lo, hi),
            [&](int u, long long at) {
                __builtin_memcpy(&r[u], x + at, 16);
                __builtin_memcpy(&q[u], g + at, 16);
            },
            [&](int u, long long at) {
                VecOf<T, V> y;
#pragma unroll
                for (int i = 0; i < V; ++i) y[i] = (T)value(i, (float)r[u][i], (float)q[u][i]);
                __builtin_memcpy(dx + at, &y, 16);
            },
            [&](int i, long long at) {
                const float v = (float)x[at], w = (float)g[at];
#pragma unroll
                for (int c = 0; c < V; ++c)
                    if (c == i) dx[at] = (T)value(c, v, w);
            });
}

template <typename T>
__global__ __launch_bounds__(kGroupThreads) void k_group_back_sums(GroupArgs p) {
    constexpr int V = kVec<T>;
    __shared__ float s_all[kGroupThreads * V];
    const long long i = block_id<kGroupThreads>();
    if (i >= p.blocks) return;
    const Slab a = slab_of(p);
    const Block k = block_of(p, i);
    for (long long b = k.b0; b <= k.b1; ++b) {
        const long long first = first_row(p, b), end = end_row(p, b, first);
        const long long lo = first > k.r0 ? first : k.r0, hi = end < k.r1 ? end : k.r1;
        float* const part = (float*)p.part + (i + b) * 2 * p.channels + a.c0;
        if (hi <= lo) {
            for (int c = threadIdx.x; c < a.c1 - a.c0; c += blockDim.x) part[c] = part[p.channels + c] = 0.0f;
            continue;
        }
        float da[V], db[V];
        backward_sums<T>(p, a, back_columns<T>(p, a, b), lo, hi, da, db);
        add_columns<V>(p, a, da, s_all, [&](int c, float sum) { part[c] = sum; });
        add_columns<V>(p, a, db, s_all, [&](int c, float sum) { part[p.channels + c] = sum; });
    }
}

template <typename T>
__global__ __launch_bounds__(256) void k_group_back_join(GroupArgs p, int q) {
    __shared__ double s_wave[4];
    const long long id = block_id<256>() * (256 / q) + threadIdx.x / q;
    const int in = threadIdx.x & (q - 1);
    const bool live = id < p.batch * p.groups;
    const long long b = live ? id / p.groups : 0;
    const int j = (int)(live ? id % p.groups : 0);
    const long long first = first_row(p, b), end = end_row(p, b, first);
    double m_h = 0.0, m_hx = 0.0;
    if (live && end > first) {
        const long long n = ((end - 1) / p.chunk - first / p.chunk + 1) * p.per;
        const float* __restrict__ part = (const float*)p.part + (first / p.chunk + b) * 2 * p.channels + (long long)j * p.per;
        const T* __restrict__ gamma = (const T*)p.gamma;
#pragma unroll 4
        for (long long e = in; e < n; e += q) {
            const long long i = e / p.per;
            const int c = (int)(e - i * p.per);
            const float* at = part + i * 2 * p.channels + c;
            const double by = gamma ? (double)(float)gamma[(long long)j * p.per + c] : 1.0;
            m_hx += by * (double)at[0];
            m_h += by * (double)at[p.channels];
        }
    }
    m_h = set_add(m_h, q, s_wave);
    m_hx = set_add(m_hx, q, s_wave);
    if (!live || in != 0) return;
    const double n = end > first ? (double)(end - first) * p.per : 1.0;
    ((float2*)p.stat)[id] = make_float2((float)(m_h / n), (float)(m_hx / n));
}

template <typename T>
__global__ __launch_bounds__(kGroupThreads) void k_group_back(GroupArgs p) {
    const long long i = block_id<kGroupThreads>();
    if (i >= p.blocks) return;
    const Slab a = slab_of(p);
    const Block k = block_of(p, i);
    for (long long b = k.b0; b <= k.b1; ++b) {
        const long long first = first_row(p, b), end = end_row(p, b, first);
        const long long lo = first > k.r0 ? first : k.r0, hi = end < k.r1 ? end : k.r1;
        if (hi > lo) backward_rows<T>(p, a, back_columns<T>(p, a, b), (const float2*)p.stat + b * p.groups, 0, lo, hi);
    }
}

// part [batch][2][channels]
template <typename T>
__global__ __launch_bounds__(kOneThreads) void k_group_back_one(GroupArgs p) {
    constexpr int V = kVec<T>;
    __shared__ float s_all[kOneThreads * V];
    __shared__ float s_col[2][kOneThreads * V];
    __shared__ float2 s_stat[kOneThreads * V];
    const long long b = block_id<kOneThreads>();
    if (b >= p.batch) return;
    const Slab a = slab_of(p);
    const long long first = first_row(p, b), end = end_row(p, b, first);
    float* const part = (float*)p.part + b * 2 * p.channels + a.c0;
    const int wide = a.c1 - a.c0;
    if (end <= first) {
        if (p.parts_wanted)
            for (int c = threadIdx.x; c < wide; c += blockDim.x) part[c] = part[p.channels + c] = 0.0f;
        return;
    }
    const BackColumns<V> k = back_columns<T>(p, a, b);
    float da[V], db[V];
    backward_sums<T>(p, a, k, first, end, da, db);
    add_columns<V>(p, a, da, s_all, [&](int c, float sum) { s_col[0][c] = sum; });
    add_columns<V>(p, a, db, s_all, [&](int c, float sum) { s_col[1][c] = sum; });
    __syncthreads();
    if (p.parts_wanted)
        for (int c = threadIdx.x; c < wide; c += blockDim.x) {
            part[c] = s_col[0][c];
            part[p.channels + c] = s_col[1][c];
        }
    if (!p.out) return;
    const int q = lanes_for(p.per), set = threadIdx.x / q, sets = blockDim.x / q, in = threadIdx.x & (q - 1);
    const double n = (double)(end - first) * p.per;
    for (int j0 = 0; j0 < a.ng; j0 += sets) {
        const int j = j0 + set;
        double m_h = 0.0, m_hx = 0.0;
        if (j < a.ng)
            for (int e = in; e < p.per; e += q) {
                const int c = j * p.per + e;
                const double by = p.gamma ? (double)(float)((const T*)p.gamma)[a.c0 + c] : 1.0;
                m_hx += by * (double)s_col[0][c];
                m_h += by * (double)s_col[1][c];
            }
        for (int d = 1; d < q; d <<= 1) {
            m_h += __shfl_xor(m_h, d, 64);
            m_hx += __shfl_xor(m_hx, d, 64);
        }
        if (in == 0 && j < a.ng) s_stat[j] = make_float2((float)(m_h / n), (float)(m_hx / n));
    }
    __syncthreads();
    backward_rows<T>(p, a, k, s_stat, a.j0, first, end);
}

// offsets[b]: the rows whose sample index is below b, a wave a sample.
__global__ __launch_bounds__(256) void k_sample_offsets(const int* __restrict__ coords, int stride, long long rows_cap,
                                                        const long long* __restrict__ rows_dev, long long batch,
                                                        long long* __restrict__ offsets) {
    const long long b = block_id<256>() * 4 + (threadIdx.x >> 6);
    if (b > batch) return;
    const long long rows = rows_of(rows_cap, rows_dev);
    const long long n = count_up_to(rows, b - 1, [&](long long r) { return (long long)coords[r * stride]; });
    if ((threadIdx.x & 63) == 0) offsets[b] = n;
}

// ------------------------------------------------------------------ host side
static int group_vec(int dtype) { return dtype == SCNN_F32 ? 4 : 8; }

// Slabs of no more columns than `threads` vectors.
static GroupLayout group_layout(int channels, int per, int dtype, int threads) {
    const int v = group_vec(dtype);
    GroupLayout l = {};
    l.slabs = l.pieces = 1;
    l.wide = channels;
    int even = 1;  // the largest power of two that both the vector and a row are a multiple of
    while (even < v && channels % (2 * even) == 0) even *= 2;
    const long long period = channels / even;  // vectors after which a run of rows meets the same columns
    if (even < v && period <= 256) {
        l.flat = 1;
        l.active = (int)(256 / period * period);
        l.reps = (int)((long long)l.active * v / channels);
        l.tv = l.active;
        l.pitch = channels;
        return l;
    }
    l.tv = (int)(((long long)channels + v - 1) / v);
    if (l.tv > threads) {
        const long long most = (long long)threads * v;
        if (per <= most) {
            l.wide = (int)(most / per * per);
            l.slabs = (int)(((long long)channels + l.wide - 1) / l.wide);
        } else {
            l.pieces = (int)((per + most - 1) / most);
            l.wide = (int)round_up((per + l.pieces - 1) / l.pieces, v);
            l.slabs = channels / per * l.pieces;
        }
        l.tv = (l.wide + v - 1) / v;
    }
    l.reps = l.tv >= 256 ? 1 : 256 / l.tv;
    l.active = l.tv * l.reps;
    l.pitch = l.tv * v;
    return l;
}

// Rows of a block: four workgroups of 256 threads a compute unit, but no fewer than four vectors a thread.
static long long group_chunk(const GroupLayout& l, long long rows) {
    const long long want = 4LL * 256 * device_cu_count() / ((l.active + 63) / 64 * 64) / l.slabs;
    long long chunk = (rows + (want < 1 ? 1 : want) - 1) / (want < 1 ? 1 : want);
    if (chunk < 4LL * l.reps) chunk = 4LL * l.reps;
    return round_up(chunk, l.reps);
}

// Calls that one workgroup a sample does best.
static bool group_short(long long rows, long long batch, int channels, int dtype) {
    const long long bytes = rows * channels * (dtype == SCNN_F32 ? 4 : 2);
    return bytes <= (64 << 10) || bytes / batch <= (32 << 10);
}

struct GroupSpace { GroupLayout l; long long blocks, chunk, places; size_t part, stat, total; bool one; };
static GroupSpace group_space(long long rows, long long batch, int channels, int groups, int dtype, bool back) {
    GroupSpace s = {};
    s.l = group_layout(channels, channels / groups, dtype, kOneThreads);
    s.one = s.l.pieces == 1 && group_short(rows, batch, channels, dtype);
    if (!s.one) s.l = group_layout(channels, channels / groups, dtype, kGroupThreads);
    s.chunk = group_chunk(s.l, rows);
    s.blocks = rows < 1 ? 1 : (rows + s.chunk - 1) / s.chunk;
    s.places = s.one ? batch : s.blocks + batch - 1;
    if (s.one && !back) return s;
    const size_t place = back ? (size_t)channels * 8 : (size_t)groups * s.l.pieces * 16;
    s.stat = (size_t)round_up((long long)(s.places * place), 256);
    s.total = s.stat;
    if (!s.one) s.total += (size_t)round_up(batch * groups * (back ? 8LL : 16LL), 256);
    return s;
}

size_t group_norm_bytes(int dtype, long long rows, long long batch, int channels, int groups, bool back) {
    return group_space(rows, batch, channels, groups, dtype, back).total;
}

static GroupArgs group_args(int dtype, const GroupCall& c, bool back, GroupSpace& s) {
    GroupArgs p = {};
    p.x = c.x; p.g = c.g; p.gamma = c.gamma; p.beta = c.beta;
    p.out = back ? c.dx : c.out;
    p.mean = c.mean; p.rstd = c.rstd;
    p.offsets = c.offsets;
    p.rows = c.rows; p.batch = c.batch;
    p.each = c.rows / c.batch;
    p.channels = c.channels; p.groups = c.groups; p.per = c.channels / c.groups; p.act = c.act;
    p.eps = c.eps;
    s = group_space(c.rows, c.batch, c.channels, c.groups, dtype, back);
    p.l = s.l;
    p.chunk = s.chunk; p.blocks = s.blocks; p.places = s.places;
    p.part = (char*)c.workspace + s.part;
    p.stat = (char*)c.workspace + s.stat;
    p.parts_wanted = c.dgamma || c.dbeta;
    return p;
}

// Threads that join the sums of a sample's group, about n of them.
static int join_threads(long long n) {
    int q = 1;
    while (q < 256 && q < n) q <<= 1;
    return q;
}

template <typename T>
static hipError_t group_fwd(int dtype, const GroupCall& c, hipStream_t s) {
    GroupSpace at;
    const GroupArgs p = group_args(dtype, c, false, at);
    const unsigned threads = (unsigned)((p.l.active + 63) / 64 * 64);
    if (at.one) {
        hipLaunchKernelGGL((k_group_one<T>), grid_of<kOneThreads>(c.batch, p.l.slabs), dim3(threads), 0, s, p);
        return hipGetLastError();
    }
    const dim3 grid = grid_of<kGroupThreads>(p.blocks, p.l.slabs);
    hipLaunchKernelGGL((k_group_sums<T>), grid, dim3(threads), 0, s, p);
    const int q = join_threads((p.blocks / p.batch + 1) * p.l.pieces);
    hipLaunchKernelGGL((k_group_join<T>), grid_of<256>((p.batch * p.groups + 256 / q - 1) / (256 / q)), dim3(256), 0, s, p, q);
    hipLaunchKernelGGL((k_group_apply<T>), grid, dim3(threads), 0, s, p);
    return hipGetLastError();
}

template <typename T>
static hipError_t group_bwd(int dtype, const GroupCall& c, hipStream_t s) {
    GroupSpace at;
    const GroupArgs p = group_args(dtype, c, true, at);
    const unsigned threads = (unsigned)((p.l.active + 63) / 64 * 64);
    if (at.one) {
        hipLaunchKernelGGL((k_group_back_one<T>), grid_of<kOneThreads>(c.batch, p.l.slabs), dim3(threads), 0, s, p);
    } else {
        const dim3 grid = grid_of<kGroupThreads>(p.blocks, p.l.slabs);
        hipLaunchKernelGGL((k_group_back_sums<T>), grid, dim3(threads), 0, s, p);
        if (p.out) {
            const int q = join_threads((p.blocks / p.batch + 1) * p.per);
            hipLaunchKernelGGL((k_group_back_join<T>), grid_of<256>((p.batch * p.groups + 256 / q - 1) / (256 / q)), dim3(256), 0,
                               s, p, q);
            hipLaunchKernelGGL((k_group_back<T>), grid, dim3(threads), 0, s, p);
        }
    }
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess || !p.parts_wanted) return e;
    return launch_column_sums((const float*)p.part, (int)p.places, 2LL * p.channels, p.channels, c.dgamma, c.dbeta, dtype, s);
}

hipError_t launch_group_fwd(int dtype, const GroupCall& c, hipStream_t s) {
    switch (dtype) {
        case SCNN_F32: return group_fwd<float>(dtype, c, s);
        case SCNN_BF16: return group_fwd<__bf16>(dtype, c, s);
        default: return group_fwd<_Float16>(dtype, c, s);
    }
}

hipError_t launch_group_bwd(int dtype, const GroupCall& c, hipStream_t s) {
    switch (dtype) {
        case SCNN_F32: return group_bwd<float>(dtype, c, s);
        case SCNN_BF16: return group_bwd<__bf16>(dtype, c, s);
        default: return group_bwd<_Float16>(dtype, c, s);
    }
}

hipError_t launch_sample_offsets(const int* coords, int stride, long long rows, const long long* rows_dev, long long batch,
                                 long long* offsets, hipStream_t s) {
    hipLaunchKernelGGL(k_sample_offsets, grid_of<256>((batch + 4) / 4), dim3(256), 0, s, coords, stride, rows, rows_dev, batch, offsets);
    return hipGetLastError();
}

}  // namespace scnn
