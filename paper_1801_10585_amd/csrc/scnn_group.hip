// Group norm with an activation over the samples of rows [rows, C], forward and backward, and where the samples begin.
//
// Sample b has the rows offsets[b] .. offsets[b + 1] - 1, group j the columns j C/G .. (j + 1) C/G - 1, n = rows of b times C/G.
//   mean = sum x / n,  var = sum (x - mean)^2 / n,  rstd = 1 / sqrt(var + eps),  xh = (x - mean) rstd,  z = xh gamma + beta
//   out = act(z)
//   dz = g act'(z),  h = dz gamma,  dx = rstd (h - sum(h) / n - xh sum(h xh) / n)   (sums over the sample's group),
//   dgamma = sum_r dz xh,  dbeta = sum_r dz
//
// Bound by memory.  A sample is as long as it likes and its group's sums have to be known before its first result: the rows are
// read twice, in two launches: sums over blocks of rows (k_group_sums, k_group_back_sums), then results (k_group_apply,
// k_group_back), every workgroup joining the sums of the samples that it meets; where these are many a launch between
// joins them (k_group_join).  Samples of few values are done by a workgroup each, which keeps its rows in registers
// (k_group_one, k_group_back_one).
//
// Blocks of rows are cut without regard to the samples, whose sizes only the device knows: block i keeps one set of sums for
// every sample that it meets, in place i + b (along the rows either i or b grows by one, so that no place is taken twice), and
// sets what no pair (i, b) takes to 0.  Sums are added in a fixed order: the same bits every time.
// The forward sums are those of x - s and its square, s the first value of the sample's group, in fp64: what cancels in
// var = (sum d^2 - (sum d)^2 / n) / n is then bits that fp64 has to spare (a spread of 1e-5 of the distance between s and the
// mean leaves 2^-53 x 1e10 of it), and a group of equal values has exactly none.
#include "scnn_dense.h"

namespace scnn {

constexpr int kGroupThreads = 512;  // most threads of a workgroup that takes a block of rows
constexpr int kHereGroups = 64;     // most groups of a slab whose sums a workgroup joins by itself

// How threads lie over columns.  A workgroup takes `wide` columns from c0 on: tv threads a row, a vector each, `reps` rows at
// a time.  Rows of all C columns that are no whole number of vectors run on without a gap (flat): `active` vectors are `reps`
// whole rows, so that a thread meets the same columns at every step.  Either way value (thread, i) is number thread V + i of a
// step, and row k's column c number k pitch + c.
struct GroupLayout {
    int tv, reps, active, pitch, flat;
    int wide, slabs, pieces;  // a slab is whole groups (pieces 1), or one of `pieces` pieces of a group
    int merged;               // a vector's columns are of one group
    float inv_tv, inv_per, inv_c;
};

struct GroupArgs {
    const void *x, *g, *gamma, *beta;
    void *out, *dgamma, *dbeta;  // out: forward out, backward dx
    float *mean, *rstd;          // [batch][groups]: written forward, read backward
    const long long* offsets;
    long long each;              // rows of a sample where offsets is null
    long long rows, chunk;       // chunk: rows of a block
    long long batch, blocks, places;
    int channels, groups, per, act;
    float eps;
    float* cols;                 // backward: [places][2][channels], sums of dz xh and dz over a place's rows; null: not wanted
    void* part;                  // [places][groups * pieces]: forward {sum d, sum d^2} in fp64, backward {sum h, sum h xh} in fp32
    void* stat;                  // [batch][groups] of k_group_join; null: joined where they are used
    GroupLayout l;
};

// a / d for whole numbers a < 2^21 by way of 1 / d in fp32: (a + 1/2) / d is no nearer to a whole number than 1 / (2 d).
__device__ __forceinline__ int quotient(int a, float inverse) { return (int)(((float)a + 0.5f) * inverse); }

// The samples' bounds.  Up to 63 samples a wave holds them all, a lane each.
struct Bounds {
    const long long* offsets;
    long long each, rows, batch, lane_row;
    bool here;
};
__device__ __forceinline__ Bounds bounds_of(const GroupArgs& p) {
    Bounds s = {p.offsets, p.each, p.rows, p.batch, 0, p.offsets != nullptr && p.batch < 64};
    const int lane = threadIdx.x & 63;
    if (s.here) {
        const long long r = p.offsets[lane <= p.batch ? lane : p.batch];
        s.lane_row = r < 0 ? 0 : (r < p.rows ? r : p.rows);
    }
    return s;
}
__device__ __forceinline__ long long uniform(long long v) {
    return (long long)((unsigned long long)(unsigned)__builtin_amdgcn_readfirstlane((int)((unsigned long long)v >> 32)) << 32 |
                       (unsigned)__builtin_amdgcn_readfirstlane((int)v));
}
__device__ __forceinline__ long long first_row(const Bounds& s, long long b) {
    if (!s.offsets) return b * s.each;
    if (s.here) {
        const int lane = __builtin_amdgcn_readfirstlane((int)b);
        return (long long)((unsigned long long)(unsigned)__builtin_amdgcn_readlane((int)((unsigned long long)s.lane_row >> 32), lane) << 32 |
                           (unsigned)__builtin_amdgcn_readlane((int)s.lane_row, lane));
    }
    const long long r = s.offsets[b];
    return r < 0 ? 0 : (r < s.rows ? r : s.rows);
}
struct Rows { long long first, end; };
// (the same in every lane of a workgroup, where b is)
__device__ __forceinline__ Rows rows_of_sample(const Bounds& s, long long b) {
    Rows r;
    r.first = uniform(first_row(s, b));
    r.end = uniform(first_row(s, b + 1));
    if (r.end < r.first) r.end = r.first;
    return r;
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
__device__ __forceinline__ long long sample_at(const Bounds& s, long long r) {
    long long b;
    if (!s.offsets) {
        b = s.each > 0 ? r / s.each : 0;
    } else if (s.here) {
        const int lane = threadIdx.x & 63;
        b = __popcll(__ballot(lane > 0 && lane <= s.batch && s.lane_row <= r));
    } else {
        b = count_up_to(s.batch, r, [&](long long k) { return first_row(s, k + 1); });
    }
    return uniform(b < s.batch ? b : s.batch - 1);
}

// Rows of block i, and the samples whose sums it keeps.
struct Block { long long r0, r1, b0, b1; };
__device__ __forceinline__ Block block_of(const GroupArgs& p, const Bounds& s, long long i) {
    Block k;
    k.r0 = i * p.chunk;
    k.r1 = k.r0 + p.chunk < p.rows ? k.r0 + p.chunk : p.rows;
    k.b0 = i == 0 ? 0 : sample_at(s, k.r0);
    k.b1 = i + 1 == p.blocks ? p.batch - 1 : sample_at(s, k.r1);
    return k;
}

// Columns of this workgroup's slab, its first group, the number of its groups and their width in it.
struct Slab { int c0, c1, j0, ng, w; };
__device__ __forceinline__ Slab slab_of(const GroupArgs& p) {
    const int s = blockIdx.y;
    Slab a;
    if (p.l.pieces > 1) {
        a.j0 = s / p.l.pieces;
        a.ng = 1;
        a.c0 = a.j0 * p.per + (s - a.j0 * p.l.pieces) * p.l.wide;
        a.c1 = a.c0 + p.l.wide < (a.j0 + 1) * p.per ? a.c0 + p.l.wide : (a.j0 + 1) * p.per;
        a.w = a.c1 - a.c0;
    } else {
        a.c0 = s * p.l.wide;
        a.c1 = a.c0 + p.l.wide < p.channels ? a.c0 + p.l.wide : p.channels;
        a.j0 = p.l.slabs > 1 ? a.c0 / p.per : 0;
        a.ng = p.l.slabs > 1 ? (a.c1 - a.c0) / p.per : p.groups;
        a.w = p.per;
    }
    return a;
}

// This thread's place: its row among a step's, its first column in the slab.
struct Place { int row, col; };
template <int V>
__device__ __forceinline__ Place place_of(const GroupArgs& p) {
    const int t = threadIdx.x;
    if (p.l.flat) return {0, t * V};
    const int k = quotient(t, p.l.inv_tv);
    return {k, (t - k * p.l.tv) * V};
}
// Column in the slab of value i of this thread.  (Values past the slab's end take its last column.)
__device__ __forceinline__ int column_of(const GroupArgs& p, const Slab& a, const Place& t, int i) {
    int c = t.col + i;
    if (p.l.flat) c -= quotient(c, p.l.inv_c) * p.channels;
    return c < a.c1 - a.c0 ? c : a.c1 - a.c0 - 1;
}
// Group in the slab of a column of it.
__device__ __forceinline__ int group_of(const GroupArgs& p, int column) { return p.l.pieces > 1 ? 0 : quotient(column, p.l.inv_per); }

// A thread's vectors among the rows lo .. hi - 1: `full` whole ones, then `part` of n values.
struct Walk {
    long long at, step;
    int full, part, n;
};
template <int V>
__device__ __forceinline__ Walk walk_of(const GroupArgs& p, const Slab& a, const Place& t, long long lo, long long hi) {
    Walk w = {0, 0, 0, 0, 0};
    if ((int)threadIdx.x >= p.l.active || hi <= lo) return w;
    const unsigned rows = (unsigned)(hi - lo), steps = rows / (unsigned)p.l.reps;  // (rows: fewer than 2^31)
    const int left = (int)(rows - steps * (unsigned)p.l.reps);
    w.step = (long long)p.l.reps * p.channels;
    w.full = (int)steps;
    if (p.l.flat) {
        w.at = lo * p.channels + t.col;
        const int n = left * p.channels - t.col;  // (fewer than a step's values)
        if (n >= V) ++w.full;
        else if (n > 0) w.part = 1, w.n = n;
    } else {
        w.at = (lo + t.row) * p.channels + a.c0 + t.col;
        if (t.row < left) ++w.full;
        const int n = a.c1 - a.c0 - t.col;
        if (n < V) {
            w.part = n > 0 ? w.full : 0;
            w.n = n;
            w.full = 0;
        }
    }
    return w;
}

template <typename T> using Loose = VecOf<T, kVec<T>> __attribute__((aligned(sizeof(T))));  // (at any element's address)
template <typename T> __device__ __forceinline__ VecOf<T, kVec<T>> take(const T* p) { return *(const Loose<T>*)p; }
// Results are not read again soon: they leave the L2 to the rows.
template <typename T> __device__ __forceinline__ void put(T* p, VecOf<T, kVec<T>> v) { __builtin_nontemporal_store(v, (Loose<T>*)p); }

__device__ __forceinline__ float finite_or_zero(float v) { return __builtin_fabsf(v) < __builtin_huge_valf() ? v : 0.0f; }

// Power of two of lanes that add n values: at most a wave.
__device__ __forceinline__ int lanes_for(int n) {
    int q = 1;
    while (q < n && q < 64) q <<= 1;
    return q;
}

// Accumulators of a thread: one a column, or two for all of a vector's columns where these are of one group.
template <typename T, bool M> constexpr int kSums = M ? 2 : kVec<T>;

// Sums over the slab's groups of the threads' numbers, then done(group, sum) by one lane a group.  All threads of the workgroup call it.
// s_all: a number a thread (merged), or a vector of them.
template <typename T, bool M, typename F>
__device__ __forceinline__ void add_groups(const GroupArgs& p, const Slab& a, const double (&v)[kSums<T, M>], double* s_all, F done) {
    constexpr int V = kVec<T>;
    __syncthreads();
    if ((int)threadIdx.x < p.l.active) {
        if constexpr (M) {
            s_all[threadIdx.x] = v[0] + v[1];
        } else {
#pragma unroll
            for (int i = 0; i < V; ++i) s_all[threadIdx.x * V + i] = v[i];
        }
    }
    __syncthreads();
    const int w = M ? (a.w + V - 1) / V : a.w, pitch = M ? p.l.tv : p.l.pitch, n = w * p.l.reps, q = lanes_for(n);
    const float inv = 1.0f / (float)w;
    const int set = threadIdx.x / q, sets = blockDim.x / q, in = threadIdx.x & (q - 1);
    for (int j0 = 0; j0 < a.ng; j0 += sets) {
        const int j = j0 + set;
        double sum = 0.0;
        if (j < a.ng)
            for (int e = in; e < n; e += q) {
                const int k = quotient(e, inv);
                sum += s_all[k * pitch + j * w + (e - k * w)];
            }
        for (int d = 1; d < q; d <<= 1) sum += __shfl_xor(sum, d, 64);
        if (in == 0 && j < a.ng) done(j, sum);
    }
}

// The first value of each accumulator's group in row `origin`.
template <typename T, bool M>
__device__ __forceinline__ void first_values(const GroupArgs& p, const Slab& a, const Place& t, long long origin, float (&s)[kSums<T, M>]) {
    const T* __restrict__ x = (const T*)p.x + origin * p.channels + (long long)a.j0 * p.per;
#pragma unroll
    for (int i = 0; i < kSums<T, M>; ++i)
        s[i] = M && i ? s[0] : (float)x[(long long)group_of(p, column_of(p, a, t, i)) * p.per];
#pragma unroll
    for (int i = 0; i < kSums<T, M>; ++i) s[i] = finite_or_zero(s[i]);
}
template <typename T, bool M>
__device__ __forceinline__ void add_value(float x, int i, const double (&s)[kSums<T, M>], double (&s1)[kSums<T, M>], double (&s2)[kSums<T, M>]) {
    const int k = M ? i & 1 : i;
    const double d = (double)x - s[k];
    s1[k] += d;
    s2[k] = __builtin_fma(d, d, s2[k]);
}

// U vectors of a thread on their way: number k, k + 1, ... upwards, or k - 1, k - 2, ... downwards (the last ones of a block are
// what the L2 still has when its rows are read again).
template <typename T, int U, bool DOWN>
__device__ __forceinline__ void fetch(const T* __restrict__ x, const Walk& w, int k, VecOf<T, kVec<T>> (&r)[U]) {
    const T* at = x + w.at + (long long)(DOWN ? k - 1 : k) * w.step;
    const int n = DOWN ? k : w.full - k;
#pragma unroll
    for (int u = 0; u < U; ++u)
        if (u < n) r[u] = take(at + (DOWN ? -u : u) * w.step);
}
// Sums over a thread's vectors from number k on, of which the first U are there, and over its odd values.
template <typename T, bool M, int U>
__device__ __forceinline__ void sum_from(const T* __restrict__ x, const Walk& w, int k, VecOf<T, kVec<T>> (&r)[U], const double (&s)[kSums<T, M>],
                                         double (&s1)[kSums<T, M>], double (&s2)[kSums<T, M>]) {
    constexpr int V = kVec<T>;
    while (k < w.full) {
#pragma unroll
        for (int u = 0; u < U; ++u)
            if (u < w.full - k) {
#pragma unroll
                for (int i = 0; i < V; ++i) {
                    add_value<T, M>((float)r[u][i], i, s, s1, s2);
                    if (i % 4 == 3) __builtin_amdgcn_sched_barrier(0);  // (the compiler would take all of them apart at once, in twice the registers)
                }
            }
        k += U;
        fetch<T, U, false>(x, w, k, r);
    }
    long long at = w.at + (long long)w.full * w.step;
    for (k = 0; k < w.part; ++k, at += w.step)
#pragma unroll
        for (int i = 0; i < V - 1; ++i)
            if (i < w.n) add_value<T, M>((float)x[at + i], i, s, s1, s2);
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

// What the forward pass knows of a thread's columns.
template <int V>
struct Columns { float mean[V], rest[V], scale[V], beta[V]; };
template <typename T>
__device__ __forceinline__ Columns<kVec<T>> columns_of(const GroupArgs& p, const Slab& a, const Place& t, const GroupStat* stat) {
    constexpr int V = kVec<T>;
    Columns<V> k;
#pragma unroll
    for (int i = 0; i < V; ++i) {
        const int c = column_of(p, a, t, i);
        const GroupStat s = stat[group_of(p, c)];
        k.mean[i] = s.mean;
        k.rest[i] = s.rest;
        k.scale[i] = p.gamma ? s.rstd * (float)((const T*)p.gamma)[a.c0 + c] : s.rstd;
        k.beta[i] = p.beta ? (float)((const T*)p.beta)[a.c0 + c] : 0.0f;
    }
    return k;
}
template <int V>
__device__ __forceinline__ float forward_value(const Columns<V>& k, int i, float x, int act) {
    return activate(__builtin_fmaf((x - k.mean[i]) - k.rest[i], k.scale[i], k.beta[i]), act);
}
template <typename T>
__device__ __forceinline__ void forward_vector(const GroupArgs& p, const Columns<kVec<T>>& k, long long at, VecOf<T, kVec<T>> r) {
    VecOf<T, kVec<T>> y;
#pragma unroll
    for (int i = 0; i < kVec<T>; ++i) {
        y[i] = (T)forward_value<kVec<T>>(k, i, (float)r[i], p.act);
        if (i % 4 == 3) __builtin_amdgcn_sched_barrier(0);
    }
    put((T*)p.out + at, y);
}
// A thread's vectors from number k - 1 down to `from`, of which the first U are there.
template <typename T, int U>
__device__ __forceinline__ void forward_down(const GroupArgs& p, const Columns<kVec<T>>& c, const Walk& w, int from, int k,
                                             VecOf<T, kVec<T>> (&r)[U]) {
    while (k > from) {
        const long long at = w.at + (long long)(k - 1) * w.step;
#pragma unroll
        for (int u = 0; u < U; ++u)
            if (u < k - from) {
                forward_vector<T>(p, c, at - u * w.step, r[u]);
                __builtin_amdgcn_sched_barrier(0);
            }
        k -= U;
        fetch<T, U, true>((const T*)p.x, w, k, r);
    }
}
template <typename T>
__device__ __forceinline__ void forward_part(const GroupArgs& p, const Columns<kVec<T>>& c, const Walk& w) {
    long long at = w.at + (long long)w.full * w.step;
    for (int k = 0; k < w.part; ++k, at += w.step)
#pragma unroll
        for (int i = 0; i < kVec<T> - 1; ++i)
            if (i < w.n) ((T*)p.out)[at + i] = (T)forward_value<kVec<T>>(c, i, (float)((const T*)p.x)[at + i], p.act);
}

template <typename T, bool M>
__global__ __launch_bounds__(kGroupThreads, 4) void k_group_sums(GroupArgs p) {
    constexpr int V = kVec<T>, A = kSums<T, M>;
    __shared__ double s_all[kGroupThreads * (M ? 1 : V)];
    const long long i = block_id<kGroupThreads>();
    if (i >= p.blocks) return;
    const Bounds s = bounds_of(p);
    const Slab a = slab_of(p);
    const Place t = place_of<V>(p);
    const Block k = block_of(p, s, i);
    const int to = p.l.pieces > 1 ? (int)blockIdx.y : a.j0;
    for (long long b = k.b0; b <= k.b1; ++b) {
        const Rows r = rows_of_sample(s, b);
        const long long lo = r.first > k.r0 ? r.first : k.r0, hi = r.end < k.r1 ? r.end : k.r1;
        double* const part = (double*)p.part + ((i + b) * p.groups * p.l.pieces + to) * 2;
        if (hi <= lo) {
            for (int j = threadIdx.x; j < 2 * a.ng; j += blockDim.x) part[j] = 0.0;
            continue;
        }
        float near[A];
        double from[A], s1[A], s2[A];
        first_values<T, M>(p, a, t, r.first, near);
        const Walk w = walk_of<V>(p, a, t, lo, hi);
        // (the first vectors are on their way with the values that they are taken about)
        VecOf<T, V> x[4];
        fetch<T, 4, false>((const T*)p.x, w, 0, x);
#pragma unroll
        for (int c = 0; c < A; ++c) {
            from[c] = (double)near[c];
            s1[c] = s2[c] = 0.0;
        }
        sum_from<T, M, 4>((const T*)p.x, w, 0, x, from, s1, s2);
        add_groups<T, M>(p, a, s1, s_all, [&](int j, double sum) { part[2 * j] = sum; });
        add_groups<T, M>(p, a, s2, s_all, [&](int j, double sum) { part[2 * j + 1] = sum; });
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

template <typename T>
__device__ __forceinline__ GroupStat joined_stat(const GroupArgs& p, const Rows& r, int j, double s1, double s2) {
    const float s = finite_or_zero((float)((const T*)p.x)[r.first * p.channels + (long long)j * p.per]);
    return stat_of((double)s, s1, s2, (double)(r.end - r.first) * p.per, p.eps);
}

// The places that hold the sums of a sample: from, and how many.
__device__ __forceinline__ long long places_of(const GroupArgs& p, long long b, const Rows& r, long long& count) {
    const long long i0 = (long long)((unsigned)r.first / (unsigned)p.chunk), i1 = (long long)((unsigned)(r.end - 1) / (unsigned)p.chunk);
    count = i1 - i0 + 1;
    return i0 + b;
}

// Q threads for each sample and group.  BACK: means of h and h xh, else the statistics.
template <typename T, bool BACK>
__global__ __launch_bounds__(256) void k_group_join(GroupArgs p, int q) {
    typedef typename std::conditional<BACK, float, double>::type F;
    __shared__ double s_wave[4];
    const long long id = block_id<256>() * (256 / q) + threadIdx.x / q;
    const int in = threadIdx.x & (q - 1);
    const bool live = id < p.batch * p.groups;
    const long long b = live ? id / p.groups : 0;
    const int j = (int)(live ? id - b * p.groups : 0);
    Bounds s = {p.offsets, p.each, p.rows, p.batch, 0, false};  // (b differs from lane to lane)
    Rows r = {first_row(s, b), first_row(s, b + 1)};
    if (r.end < r.first) r.end = r.first;
    double s1 = 0.0, s2 = 0.0;
    if (live && r.end > r.first) {
        long long count;
        const long long from = places_of(p, b, r, count);
        const F* __restrict__ part = (const F*)p.part;
        const unsigned pieces = (unsigned)p.l.pieces;
        const long long n = count * pieces;
#pragma unroll 4
        for (long long e = in; e < n; e += q) {
            const long long i = pieces > 1 ? e / pieces : e;
            const F* at = part + (((from + i) * p.groups + j) * pieces + (e - i * pieces)) * 2;
            s1 += (double)at[0];
            s2 += (double)at[1];
        }
    }
    s1 = set_add(s1, q, s_wave);
    s2 = set_add(s2, q, s_wave);
    if (!live || in != 0) return;
    if constexpr (BACK) {
        const double n = r.end > r.first ? (double)(r.end - r.first) * p.per : 1.0;
        ((float2*)p.stat)[id] = make_float2((float)(s1 / n), (float)(s2 / n));
    } else {
        GroupStat v = {0.0f, 0.0f, 0.0f, 0.0f};
        if (r.end > r.first) v = joined_stat<T>(p, r, j, s1, s2);
        ((GroupStat*)p.stat)[id] = v;
        if (p.mean) p.mean[id] = v.mean;
        if (p.rstd) p.rstd[id] = v.rstd;
    }
}

// The sums of a sample's groups by one workgroup: threads side by side take neighbouring groups of a place, their sums meet in
// s_two, then done(group of the slab, sums) by one lane a group.  (Reads the places' lines whole: a lane a place took four times as
// long.)  All threads call it; up to kHereGroups groups.
template <typename F, typename D>
__device__ __forceinline__ void join_here(const GroupArgs& p, const Slab& a, long long b, const Rows& r, double2* s_two, D done) {
    const int ng = a.ng, sets = (int)blockDim.x / ng, set = threadIdx.x / ng, j = threadIdx.x - set * ng;
    long long count;
    const long long from = places_of(p, b, r, count);
    double2 sum = make_double2(0.0, 0.0);
    if (set < sets) {
        const F* __restrict__ part = (const F*)p.part + ((from + set) * p.groups + a.j0 + j) * 2;
        const long long step = (long long)sets * p.groups * 2;
#pragma unroll 8
        for (long long i = set; i < count; i += sets, part += step) {
            sum.x += (double)part[0];
            sum.y += (double)part[1];
        }
    }
    __syncthreads();
    s_two[threadIdx.x] = sum;
    __syncthreads();
    int q = 1;
    while (2 * q * ng <= (int)blockDim.x && q < 64 && q < sets) q <<= 1;
    const int k = threadIdx.x / q, in = threadIdx.x & (q - 1);
    sum = make_double2(0.0, 0.0);
    if (k < ng)
        for (int e = in; e < sets; e += q) {
            sum.x += s_two[e * ng + k].x;
            sum.y += s_two[e * ng + k].y;
        }
    for (int d = 1; d < q; d <<= 1) {
        sum.x += __shfl_xor(sum.x, d, 64);
        sum.y += __shfl_xor(sum.y, d, 64);
    }
    if (k < ng && in == 0) done(k, sum);
}

template <typename T>
__global__ __launch_bounds__(kGroupThreads, 4) void k_group_apply(GroupArgs p) {
    constexpr int V = kVec<T>, U = 16 / V;
    __shared__ double2 s_two[kGroupThreads];
    __shared__ GroupStat s_stat[kHereGroups];
    const long long i = block_id<kGroupThreads>();
    if (i >= p.blocks) return;
    const Bounds s = bounds_of(p);
    const Slab a = slab_of(p);
    const Place t = place_of<V>(p);
    const Block k = block_of(p, s, i);
    for (long long b = k.b0; b <= k.b1; ++b) {
        const Rows r = rows_of_sample(s, b);
        const long long lo = r.first > k.r0 ? r.first : k.r0, hi = r.end < k.r1 ? r.end : k.r1, id = b * p.groups + a.j0;
        if (!p.stat && r.end == r.first)  // (by every workgroup that passes the empty sample)
            for (int j = threadIdx.x; j < a.ng; j += blockDim.x) {
                if (p.mean) p.mean[id + j] = 0.0f;
                if (p.rstd) p.rstd[id + j] = 0.0f;
            }
        if (hi <= lo) continue;
        const Walk w = walk_of<V>(p, a, t, lo, hi);
        // (the last vectors are on their way while the sums are joined)
        VecOf<T, V> x[U];
        fetch<T, U, true>((const T*)p.x, w, w.full, x);
        const GroupStat* stat = (const GroupStat*)p.stat + id;
        if (!p.stat) {
            join_here<double>(p, a, b, r, s_two, [&](int j, double2 sum) {
                const GroupStat v = joined_stat<T>(p, r, a.j0 + j, sum.x, sum.y);
                s_stat[j] = v;
                if (r.first >= k.r0) {
                    if (p.mean) p.mean[id + j] = v.mean;
                    if (p.rstd) p.rstd[id + j] = v.rstd;
                }
            });
            __syncthreads();
            stat = s_stat;
        }
        const Columns<V> c = columns_of<T>(p, a, t, stat);
        forward_down<T, U>(p, c, w, 0, w.full, x);
        forward_part<T>(p, c, w);
    }
}

// A sample's slab of whole groups by one workgroup of up to B threads, H vectors a thread in registers; what a larger sample has
// more is read again.
template <typename T, bool M, int B, int H>
__global__ __launch_bounds__(B) void k_group_one(GroupArgs p) {
    constexpr int V = kVec<T>, A = kSums<T, M>;
    __shared__ double s_all[B * (M ? 1 : V)];
    __shared__ union { double sum; GroupStat stat; } s_group[M ? B : B * V / 4];
    const long long b = block_id<B>();
    if (b >= p.batch) return;
    const Bounds s = {p.offsets, p.each, p.rows, p.batch, 0, false};
    const Slab a = slab_of(p);
    const Place t = place_of<V>(p);
    const Rows r = rows_of_sample(s, b);
    const long long id = b * p.groups + a.j0;
    if (r.end > r.first) {
        const T* __restrict__ x = (const T*)p.x;
        const Walk w = walk_of<V>(p, a, t, r.first, r.end);
        float near[A];
        double from[A], s1[A], s2[A];
        first_values<T, M>(p, a, t, r.first, near);
        VecOf<T, V> held[H];
#pragma unroll
        for (int h = 0; h < H; ++h)
            if (h < w.full) held[h] = take(x + w.at + h * w.step);
#pragma unroll
        for (int c = 0; c < A; ++c) {
            from[c] = (double)near[c];
            s1[c] = s2[c] = 0.0;
        }
#pragma unroll
        for (int h = 0; h < H; ++h)
            if (h < w.full) {
#pragma unroll
                for (int i = 0; i < V; ++i) add_value<T, M>((float)held[h][i], i, from, s1, s2);
                __builtin_amdgcn_sched_barrier(0);
            }
        VecOf<T, V> more[4];
        fetch<T, 4, false>(x, w, H, more);
        sum_from<T, M, 4>(x, w, H, more, from, s1, s2);
        add_groups<T, M>(p, a, s1, s_all, [&](int j, double sum) { s_group[j].sum = sum; });
        add_groups<T, M>(p, a, s2, s_all, [&](int j, double sum) {
            const GroupStat v = joined_stat<T>(p, r, a.j0 + j, s_group[j].sum, sum);
            s_group[j].stat = v;
            if (p.mean) p.mean[id + j] = v.mean;
            if (p.rstd) p.rstd[id + j] = v.rstd;
        });
        __syncthreads();
        const Columns<V> c = columns_of<T>(p, a, t, &s_group[0].stat);
#pragma unroll
        for (int h = 0; h < H; ++h)
            if (h < w.full) {
                forward_vector<T>(p, c, w.at + h * w.step, held[h]);
                __builtin_amdgcn_sched_barrier(0);
            }
        if (w.full > H) {
            fetch<T, 4, true>(x, w, w.full, more);
            forward_down<T, 4>(p, c, w, H, w.full, more);
        }
        forward_part<T>(p, c, w);
    } else {
        for (int j = threadIdx.x; j < a.ng; j += blockDim.x) {
            if (p.mean) p.mean[id + j] = 0.0f;
            if (p.rstd) p.rstd[id + j] = 0.0f;
        }
    }
}

// What the backward pass knows of a thread's columns (mean and rstd once where they are of one group).
template <int V, int A>
struct BackColumns { float mean[A], rstd[A], gamma[V], beta[V]; };
template <typename T, bool M>
__device__ __forceinline__ BackColumns<kVec<T>, M ? 1 : kVec<T>> back_columns(const GroupArgs& p, const Slab& a, const Place& t, long long b) {
    constexpr int V = kVec<T>;
    BackColumns<V, M ? 1 : V> k;
#pragma unroll
    for (int i = 0; i < V; ++i) {
        const int c = column_of(p, a, t, i);
        if (!M || i == 0) {
            const long long s = b * p.groups + a.j0 + group_of(p, c);
            k.mean[i] = p.mean[s];
            k.rstd[i] = p.rstd[s];
        }
        k.gamma[i] = p.gamma ? (float)((const T*)p.gamma)[a.c0 + c] : 1.0f;
        k.beta[i] = p.beta ? (float)((const T*)p.beta)[a.c0 + c] : 0.0f;
    }
    return k;
}
// xh and dz of a value.  relu's slope hangs on the sign of z alone, and in fp32 one z in some ten million lies on the wrong side of
// 0 and takes a whole gradient with it: what is nearer to 0 than 8 roundings of its parts (three are made) is formed anew in fp64.
template <int V, int A>
__device__ __forceinline__ void back_value(const BackColumns<V, A>& k, int i, float x, float g, int act, float& xh, float& dz) {
    const float mean = k.mean[A == 1 ? 0 : i], rstd = k.rstd[A == 1 ? 0 : i];
    xh = (x - mean) * rstd;
    float z = __builtin_fmaf(xh, k.gamma[i], k.beta[i]);
    if (act == SCNN_ACT_RELU) {
        if (__builtin_fabsf(z) <= 0x1p-21f * (__builtin_fabsf(xh * k.gamma[i]) + __builtin_fabsf(k.beta[i]))) {
            float m = mean, r = rstd, c = k.gamma[i], o = k.beta[i];
            asm volatile("" : "+v"(m), "+v"(r), "+v"(c), "+v"(o));  // (else all columns' values are held in fp64 besides)
            const double far = __builtin_fma(((double)x - (double)m) * (double)r, (double)c, (double)o);
            z = far <= 0.0 ? 0.0f : 1.0f;
        }
    }
    dz = activate_back(g, z, act);
}
template <int V, int A>
__device__ __forceinline__ void back_add(const BackColumns<V, A>& k, int i, float x, float g, int act, float (&da)[V], float (&db)[V], float& dz) {
    float xh;
    back_value<V, A>(k, i, x, g, act, xh, dz);
    da[i] = __builtin_fmaf(dz, xh, da[i]);
    db[i] += dz;
}

template <typename T, bool M, int U>
__device__ __forceinline__ void back_sum_from(const GroupArgs& p, const BackColumns<kVec<T>, M ? 1 : kVec<T>>& c, const Walk& w, int k,
                                              VecOf<T, kVec<T>> (&r)[U], VecOf<T, kVec<T>> (&q)[U], float (&da)[kVec<T>], float (&db)[kVec<T>]) {
    constexpr int V = kVec<T>, A = M ? 1 : V;
    const T *__restrict__ x = (const T*)p.x, *__restrict__ g = (const T*)p.g;
    float dz;
    while (k < w.full) {
#pragma unroll
        for (int u = 0; u < U; ++u)
            if (u < w.full - k) {
#pragma unroll
                for (int i = 0; i < V; ++i) {
                    back_add<V, A>(c, i, (float)r[u][i], (float)q[u][i], p.act, da, db, dz);
                    if (i % 4 == 3) __builtin_amdgcn_sched_barrier(0);
                }
            }
        k += U;
        fetch<T, U, false>(x, w, k, r);
        fetch<T, U, false>(g, w, k, q);
    }
    long long at = w.at + (long long)w.full * w.step;
    for (k = 0; k < w.part; ++k, at += w.step)
#pragma unroll
        for (int i = 0; i < V - 1; ++i)
            if (i < w.n) back_add<V, A>(c, i, (float)x[at + i], (float)g[at + i], p.act, da, db, dz);
}

// Sums over a step's rows: done(column of the slab, sum) by one lane a column.  All threads call it; s_all: a vector a thread.
template <int V, typename F>
__device__ __forceinline__ void add_columns(const GroupArgs& p, const Slab& a, const float (&v)[V], float* s_all, F done) {
    __syncthreads();
    if ((int)threadIdx.x < p.l.active)
#pragma unroll
        for (int i = 0; i < V; ++i) s_all[threadIdx.x * V + i] = v[i];
    __syncthreads();
    const int wide = a.c1 - a.c0;
    int q = 1;
    while (2 * q * wide <= (int)blockDim.x && q < p.l.reps && q < 64) q <<= 1;
    const int sets = blockDim.x / q, in = threadIdx.x & (q - 1);
    for (int c0 = 0; c0 < wide; c0 += sets) {
        const int c = c0 + threadIdx.x / q;
        float sum = 0.0f;
        if (c < wide)
            for (int k = in; k < p.l.reps; k += q) sum += s_all[k * p.l.pitch + c];
        for (int d = 1; d < q; d <<= 1) sum += __shfl_xor(sum, d, 64);
        if (c < wide && in == 0) done(c, sum);
    }
}

// Sums of h and h xh over the slab's groups from the columns' sums of dz xh and dz: done(group, sum h, sum h xh).
template <typename T, typename F>
__device__ __forceinline__ void back_groups(const GroupArgs& p, const Slab& a, const float* s_a, const float* s_b, F done) {
    const T* __restrict__ gamma = p.gamma ? (const T*)p.gamma + a.c0 : nullptr;
    const int q = lanes_for(a.w), set = threadIdx.x / q, sets = blockDim.x / q, in = threadIdx.x & (q - 1);
    for (int j0 = 0; j0 < a.ng; j0 += sets) {
        const int j = j0 + set;
        double h = 0.0, hx = 0.0;
        if (j < a.ng)
            for (int e = in; e < a.w; e += q) {
                const int c = j * a.w + e;
                const double by = gamma ? (double)(float)gamma[c] : 1.0;
                hx += by * (double)s_a[c];
                h += by * (double)s_b[c];
            }
        for (int d = 1; d < q; d <<= 1) {
            h += __shfl_xor(h, d, 64);
            hx += __shfl_xor(hx, d, 64);
        }
        if (in == 0 && j < a.ng) done(j, h, hx);
    }
}

template <int V, int A>
struct Means { float h[A], hx[A]; };
template <typename T, bool M>
__device__ __forceinline__ Means<kVec<T>, M ? 1 : kVec<T>> means_of(const GroupArgs& p, const Slab& a, const Place& t, const float2* stat) {
    constexpr int V = kVec<T>, A = M ? 1 : V;
    Means<V, A> m;
#pragma unroll
    for (int i = 0; i < A; ++i) {
        const float2 s = stat[group_of(p, column_of(p, a, t, i))];
        m.h[i] = s.x;
        m.hx[i] = s.y;
    }
    return m;
}
template <int V, int A>
__device__ __forceinline__ float back_result(const BackColumns<V, A>& k, const Means<V, A>& m, int i, float xh, float dz) {
    const int j = A == 1 ? 0 : i;
    return k.rstd[j] * (dz * k.gamma[i] - m.h[j] - xh * m.hx[j]);
}
template <typename T, bool M>
__device__ __forceinline__ void back_vector(const GroupArgs& p, const BackColumns<kVec<T>, M ? 1 : kVec<T>>& k,
                                            const Means<kVec<T>, M ? 1 : kVec<T>>& m, long long at, VecOf<T, kVec<T>> r, VecOf<T, kVec<T>> q) {
    constexpr int V = kVec<T>, A = M ? 1 : V;
    VecOf<T, V> y;
#pragma unroll
    for (int i = 0; i < V; ++i) {
        float xh, dz;
        back_value<V, A>(k, i, (float)r[i], (float)q[i], p.act, xh, dz);
        y[i] = (T)back_result<V, A>(k, m, i, xh, dz);
        if (i % 4 == 3) __builtin_amdgcn_sched_barrier(0);
    }
    put((T*)p.out + at, y);
}
// A thread's vectors from number k - 1 down to `from`, of which the first U are there, and its odd values.
template <typename T, bool M, int U>
__device__ __forceinline__ void back_down(const GroupArgs& p, const BackColumns<kVec<T>, M ? 1 : kVec<T>>& c,
                                          const Means<kVec<T>, M ? 1 : kVec<T>>& m, const Walk& w, int from, int k,
                                          VecOf<T, kVec<T>> (&r)[U], VecOf<T, kVec<T>> (&q)[U]) {
    constexpr int V = kVec<T>, A = M ? 1 : V;
    const T *__restrict__ x = (const T*)p.x, *__restrict__ g = (const T*)p.g;
    while (k > from) {
        const long long at = w.at + (long long)(k - 1) * w.step;
#pragma unroll
        for (int u = 0; u < U; ++u)
            if (u < k - from) {
                back_vector<T, M>(p, c, m, at - u * w.step, r[u], q[u]);
                __builtin_amdgcn_sched_barrier(0);
            }
        k -= U;
        fetch<T, U, true>(x, w, k, r);
        fetch<T, U, true>(g, w, k, q);
    }
    long long at = w.at + (long long)w.full * w.step;
    for (int n = 0; n < w.part; ++n, at += w.step)
#pragma unroll
        for (int i = 0; i < V - 1; ++i)
            if (i < w.n) {
                float xh, dz;
                back_value<V, A>(c, i, (float)x[at + i], (float)g[at + i], p.act, xh, dz);
                ((T*)p.out)[at + i] = (T)back_result<V, A>(c, m, i, xh, dz);
            }
}

template <typename T, bool M>
__global__ __launch_bounds__(kGroupThreads, 4) void k_group_back_sums(GroupArgs p) {
    constexpr int V = kVec<T>, U = 8 / V;
    __shared__ float s_all[kGroupThreads * V];
    __shared__ float s_col[2][kGroupThreads * V];
    const long long i = block_id<kGroupThreads>();
    if (i >= p.blocks) return;
    const Bounds s = bounds_of(p);
    const Slab a = slab_of(p);
    const Place t = place_of<V>(p);
    const Block k = block_of(p, s, i);
    const int wide = a.c1 - a.c0, to = p.l.pieces > 1 ? (int)blockIdx.y : a.j0;
    for (long long b = k.b0; b <= k.b1; ++b) {
        const Rows r = rows_of_sample(s, b);
        const long long lo = r.first > k.r0 ? r.first : k.r0, hi = r.end < k.r1 ? r.end : k.r1;
        float* const cols = p.cols + (i + b) * 2 * p.channels + a.c0;
        float* const part = (float*)p.part + ((i + b) * p.groups * p.l.pieces + to) * 2;
        if (hi <= lo) {
            if (p.cols)
                for (int c = threadIdx.x; c < wide; c += blockDim.x) cols[c] = cols[p.channels + c] = 0.0f;
            for (int j = threadIdx.x; j < 2 * a.ng; j += blockDim.x) part[j] = 0.0f;
            continue;
        }
        float da[V], db[V];
#pragma unroll
        for (int c = 0; c < V; ++c) da[c] = db[c] = 0.0f;
        const Walk w = walk_of<V>(p, a, t, lo, hi);
        VecOf<T, V> x[U], g[U];
        fetch<T, U, false>((const T*)p.x, w, 0, x);
        fetch<T, U, false>((const T*)p.g, w, 0, g);
        back_sum_from<T, M, U>(p, back_columns<T, M>(p, a, t, b), w, 0, x, g, da, db);
        add_columns<V>(p, a, da, s_all, [&](int c, float sum) {
            s_col[0][c] = sum;
            if (p.cols) cols[c] = sum;
        });
        add_columns<V>(p, a, db, s_all, [&](int c, float sum) {
            s_col[1][c] = sum;
            if (p.cols) cols[p.channels + c] = sum;
        });
        if (!p.out) continue;
        __syncthreads();
        back_groups<T>(p, a, s_col[0], s_col[1], [&](int j, double h, double hx) {
            part[2 * j] = (float)h;
            part[2 * j + 1] = (float)hx;
        });
        __syncthreads();
    }
}

// Four columns of the places' sums of dz xh and dz by one workgroup.
template <typename T>
__device__ __forceinline__ void back_columns_sum(const GroupArgs& p, long long at, double2* s_two) {
    double* const s_sum = (double*)s_two;
    const int c4 = threadIdx.x & 3, threads = blockDim.x / 4;
    const long long cols = 2LL * p.channels, c = at * 4 + c4;
    double sum = 0.0;
    if (c < cols)
#pragma unroll 8
        for (long long i = threadIdx.x >> 2; i < p.places; i += threads) sum += (double)p.cols[i * cols + c];
#pragma unroll
    for (int d = 4; d < 64; d <<= 1) sum += __shfl_xor(sum, d, 64);
    if ((threadIdx.x & 63) < 4) s_sum[threadIdx.x >> 6 << 2 | c4] = sum;
    __syncthreads();
    if (threadIdx.x >= 4 || c >= cols) return;
    sum = 0.0;
    for (int w = 0; w < (int)blockDim.x / 64; ++w) sum += s_sum[w << 2 | c4];
    T* const to = (T*)(c < p.channels ? p.dgamma : p.dbeta);
    if (to) to[c < p.channels ? c : c - p.channels] = (T)(float)sum;
}

// Workgroups past the blocks add the columns' sums.
template <typename T, bool M>
__global__ __launch_bounds__(kGroupThreads, 4) void k_group_back(GroupArgs p) {
    constexpr int V = kVec<T>, U = 8 / V;
    __shared__ double2 s_two[kGroupThreads];
    __shared__ float2 s_stat[kHereGroups];
    const long long i = block_id<kGroupThreads>();
    if (i >= p.blocks) {
        if (blockIdx.y == 0 && p.cols && (i - p.blocks) * 4 < 2LL * p.channels) back_columns_sum<T>(p, i - p.blocks, s_two);
        return;
    }
    const Bounds s = bounds_of(p);
    const Slab a = slab_of(p);
    const Place t = place_of<V>(p);
    const Block k = block_of(p, s, i);
    for (long long b = k.b0; b <= k.b1; ++b) {
        const Rows r = rows_of_sample(s, b);
        const long long lo = r.first > k.r0 ? r.first : k.r0, hi = r.end < k.r1 ? r.end : k.r1;
        if (hi <= lo) continue;
        const Walk w = walk_of<V>(p, a, t, lo, hi);
        VecOf<T, V> x[U], g[U];
        fetch<T, U, true>((const T*)p.x, w, w.full, x);
        fetch<T, U, true>((const T*)p.g, w, w.full, g);
        const float2* stat = (const float2*)p.stat + b * p.groups + a.j0;
        if (!p.stat) {
            const double n = (double)(r.end - r.first) * p.per;
            join_here<float>(p, a, b, r, s_two, [&](int j, double2 sum) { s_stat[j] = make_float2((float)(sum.x / n), (float)(sum.y / n)); });
            __syncthreads();
            stat = s_stat;
        }
        const auto c = back_columns<T, M>(p, a, t, b);
        const auto m = means_of<T, M>(p, a, t, stat);
        back_down<T, M, U>(p, c, m, w, 0, w.full, x, g);
    }
}

// cols [batch][2][channels]; with one sample dgamma and dbeta themselves.
template <typename T, bool M, int B, int H>
__global__ __launch_bounds__(B) void k_group_back_one(GroupArgs p) {
    constexpr int V = kVec<T>, A = M ? 1 : V;
    __shared__ float s_all[B * V];
    __shared__ float s_col[2][B * V / 4];
    __shared__ float2 s_stat[M ? B : B * V / 4];
    const long long b = block_id<B>();
    if (b >= p.batch) return;
    const Bounds s = {p.offsets, p.each, p.rows, p.batch, 0, false};
    const Slab a = slab_of(p);
    const Place t = place_of<V>(p);
    const Rows r = rows_of_sample(s, b);
    const int wide = a.c1 - a.c0;
    auto give = [&](int c, float da, float db) {
        if (p.batch == 1) {
            if (p.dgamma) ((T*)p.dgamma)[a.c0 + c] = (T)da;
            if (p.dbeta) ((T*)p.dbeta)[a.c0 + c] = (T)db;
        } else if (p.cols) {
            p.cols[b * 2 * p.channels + a.c0 + c] = da;
            p.cols[(b * 2 + 1) * p.channels + a.c0 + c] = db;
        }
    };
    if (r.end == r.first) {
        for (int c = threadIdx.x; c < wide; c += blockDim.x) give(c, 0.0f, 0.0f);
        return;
    }
    const T *__restrict__ x = (const T*)p.x, *__restrict__ g = (const T*)p.g;
    const Walk w = walk_of<V>(p, a, t, r.first, r.end);
    VecOf<T, V> held[H], grad[H];
#pragma unroll
    for (int h = 0; h < H; ++h)
        if (h < w.full) {
            held[h] = take(x + w.at + h * w.step);
            grad[h] = take(g + w.at + h * w.step);
        }
    const BackColumns<V, A> k = back_columns<T, M>(p, a, t, b);
    float da[V], db[V], dz[H][V];
#pragma unroll
    for (int c = 0; c < V; ++c) da[c] = db[c] = 0.0f;
#pragma unroll
    for (int h = 0; h < H; ++h)
        if (h < w.full)
        {
#pragma unroll
            for (int i = 0; i < V; ++i) back_add<V, A>(k, i, (float)held[h][i], (float)grad[h][i], p.act, da, db, dz[h][i]);
            __builtin_amdgcn_sched_barrier(0);
        }
    VecOf<T, V> more[2], more_g[2];
    fetch<T, 2, false>(x, w, H, more);
    fetch<T, 2, false>(g, w, H, more_g);
    back_sum_from<T, M, 2>(p, k, w, H, more, more_g, da, db);
    add_columns<V>(p, a, da, s_all, [&](int c, float sum) { s_col[0][c] = sum; });
    add_columns<V>(p, a, db, s_all, [&](int c, float sum) { s_col[1][c] = sum; });
    __syncthreads();
    for (int c = threadIdx.x; c < wide; c += blockDim.x) give(c, s_col[0][c], s_col[1][c]);
    if (!p.out) return;
    const double n = (double)(r.end - r.first) * p.per;
    back_groups<T>(p, a, s_col[0], s_col[1], [&](int j, double h, double hx) { s_stat[j] = make_float2((float)(h / n), (float)(hx / n)); });
    __syncthreads();
    const Means<V, A> m = means_of<T, M>(p, a, t, s_stat);
#pragma unroll
    for (int h = 0; h < H; ++h)
        if (h < w.full) {
            VecOf<T, V> y;
#pragma unroll
            for (int i = 0; i < V; ++i) {
                const int j = A == 1 ? 0 : i;
                y[i] = (T)back_result<V, A>(k, m, i, ((float)held[h][i] - k.mean[j]) * k.rstd[j], dz[h][i]);
            }
            put((T*)p.out + w.at + h * w.step, y);
            __builtin_amdgcn_sched_barrier(0);
        }
    if (w.full > H) {
        fetch<T, 2, true>(x, w, w.full, more);
        fetch<T, 2, true>(g, w, w.full, more_g);
    }
    back_down<T, M, 2>(p, k, m, w, H, w.full, more, more_g);
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

// Slabs of up to `most` columns for workgroups of up to `threads` threads.
static GroupLayout group_layout(int channels, int per, int dtype, int threads, int most) {
    const int v = group_vec(dtype);
    GroupLayout l = {};
    l.slabs = l.pieces = 1;
    l.wide = channels;
    int even = 1;  // the largest power of two that both the vector and a row are a multiple of
    while (even < v && channels % (2 * even) == 0) even *= 2;
    const long long period = channels / even;  // vectors after which a run of rows meets the same columns
    if (even < v && period <= threads && (long long)channels <= most) {
        l.flat = 1;
        l.active = (int)(threads / period * period);
        l.reps = (int)((long long)l.active * v / channels);
        l.tv = l.active;
        l.pitch = channels;
    } else {
        if (channels > most) {
            if (per <= most) {
                l.wide = most / per * per;
                l.slabs = (channels + l.wide - 1) / l.wide;
            } else {
                l.pieces = (per + most - 1) / most;
                l.wide = (int)round_up((per + l.pieces - 1) / l.pieces, v);
                l.pieces = (per + l.wide - 1) / l.wide;
                l.slabs = channels / per * l.pieces;
            }
        }
        l.tv = (l.wide + v - 1) / v;
        l.reps = l.tv >= threads ? 1 : threads / l.tv;
        l.active = l.tv * l.reps;
        l.pitch = l.tv * v;
        l.merged = l.pieces > 1 || per % v == 0;
    }
    l.inv_tv = 1.0f / (float)l.tv;
    l.inv_per = 1.0f / (float)per;
    l.inv_c = 1.0f / (float)channels;
    return l;
}
static unsigned group_threads(const GroupLayout& l) { return (unsigned)((l.active + 63) / 64 * 64); }

// Rows of a block: four workgroups of 256 threads a compute unit, but no fewer than two vectors a thread.
static long long group_chunk(const GroupLayout& l, long long rows) {
    long long want = 4LL * 256 * device_cu_count() / group_threads(l) / l.slabs;
    if (want < 1) want = 1;
    long long chunk = (rows + want - 1) / want;
    if (chunk < 2LL * l.reps) chunk = 2LL * l.reps;
    return round_up(chunk, l.reps);
}

// A workgroup a sample and slab, its values in registers: up to kOneHeld (backward half as many) on the average.
constexpr long long kOneHeld = 32768;
constexpr int kOneThreads = 1024, kOneOdd = 512;  // threads where vectors are of one group, and where they are not
static bool group_one(long long rows, long long batch, int channels, int per, int dtype, bool back, GroupLayout& l) {
    const int v = group_vec(dtype), least = 64 / (16 / v);  // (64 bytes of a row)
    const long long held = back ? kOneHeld / 2 : kOneHeld, values = rows * channels / batch;
    const bool merged = per % v == 0;
    const int threads = merged ? kOneThreads : kOneOdd;
    int most = threads * v / 4;
    if (per > most) return false;
    if (merged) {
        // narrower slabs where a sample has more values than that, or compute units would idle
        long long want = (values + held - 1) / held;
        if (want * batch < device_cu_count() && values > 4096) want = device_cu_count() / batch;
        if (want > 1) {
            long long wide = (channels + want - 1) / want;
            if (wide < least) wide = least;
            wide = (wide + per - 1) / per * per;
            if (wide < most) most = (int)wide;
        }
    }
    if (rows * (channels < most ? channels : most) > held * batch) return false;
    l = group_layout(channels, per, dtype, threads, most);
    return l.pieces == 1;
}

struct GroupSpace { GroupLayout l; long long blocks, chunk, places; size_t part, cols, stat, total; bool one, joined; };
static GroupSpace group_space(long long rows, long long batch, int channels, int groups, int dtype, bool back) {
    GroupSpace s = {};
    const int per = channels / groups;
    s.one = group_one(rows, batch, channels, per, dtype, back, s.l);
    if (s.one) {
        s.places = batch;
        if (back && batch > 1) s.total = (size_t)round_up(batch * channels * 8, 256);
        return s;
    }
    s.l = group_layout(channels, per, dtype, 256, kGroupThreads * group_vec(dtype));
    s.chunk = group_chunk(s.l, rows);
    s.blocks = rows < 1 ? 1 : (rows + s.chunk - 1) / s.chunk;
    s.places = s.blocks + batch - 1;
    const int ng = s.l.wide / per;  // (of a slab)
    s.joined = s.l.pieces > 1 || ng > kHereGroups || (s.blocks / batch + 1) * ng > 2048;
    s.cols = (size_t)round_up(s.places * groups * s.l.pieces * (back ? 8LL : 16LL), 256);
    s.stat = s.cols + (back ? (size_t)round_up(s.places * channels * 8LL, 256) : 0);
    s.total = s.stat + (s.joined ? (size_t)round_up(batch * groups * (back ? 8LL : 16LL), 256) : 0);
    return s;
}

size_t group_norm_bytes(int dtype, long long rows, long long batch, int channels, int groups, bool back) {
    return group_space(rows, batch, channels, groups, dtype, back).total;
}

static GroupArgs group_args(int dtype, const GroupCall& c, bool back, GroupSpace& s) {
    GroupArgs p = {};
    p.x = c.x; p.g = c.g; p.gamma = c.gamma; p.beta = c.beta;
    p.out = back ? c.dx : c.out;
    p.dgamma = c.dgamma; p.dbeta = c.dbeta;
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
    if (c.dgamma || c.dbeta) p.cols = (float*)((char*)c.workspace + s.cols);
    if (s.joined) p.stat = (char*)c.workspace + s.stat;
    return p;
}

// A launch that joins the places' sums, about as many threads for a sample's group as it has places.
template <typename T, bool BACK>
static void group_join(const GroupArgs& p, hipStream_t s) {
    const long long n = (p.blocks / p.batch + 1) * p.l.pieces;
    int q = 1;
    while (q < 256 && q < n) q <<= 1;
    hipLaunchKernelGGL((k_group_join<T, BACK>), grid_of<256>((p.batch * p.groups + 256 / q - 1) / (256 / q)), dim3(256), 0, s, p, q);
}

template <typename T>
static hipError_t group_fwd(int dtype, const GroupCall& c, hipStream_t s) {
    GroupSpace at;
    const GroupArgs p = group_args(dtype, c, false, at);
    const dim3 threads(group_threads(p.l));
    if (at.one) {
        if (p.l.merged) hipLaunchKernelGGL((k_group_one<T, true, kOneThreads, 32 / kVec<T>>), grid_of<kOneThreads>(c.batch, p.l.slabs), threads, 0, s, p);
        else hipLaunchKernelGGL((k_group_one<T, false, kOneOdd, 8>), grid_of<kOneOdd>(c.batch, p.l.slabs), threads, 0, s, p);
        return hipGetLastError();
    }
    const dim3 grid = grid_of<kGroupThreads>(p.blocks, p.l.slabs);
    hipLaunchKernelGGL((p.l.merged ? k_group_sums<T, true> : k_group_sums<T, false>), grid, threads, 0, s, p);
    if (p.stat) group_join<T, false>(p, s);
    hipLaunchKernelGGL((k_group_apply<T>), grid, threads, 0, s, p);
    return hipGetLastError();
}

template <typename T>
static hipError_t group_bwd(int dtype, const GroupCall& c, hipStream_t s) {
    GroupSpace at;
    const GroupArgs p = group_args(dtype, c, true, at);
    const dim3 threads(group_threads(p.l));
    hipError_t e;
    if (at.one) {
        if (p.l.merged) hipLaunchKernelGGL((k_group_back_one<T, true, kOneThreads, 16 / kVec<T>>), grid_of<kOneThreads>(c.batch, p.l.slabs), threads, 0, s, p);
        else hipLaunchKernelGGL((k_group_back_one<T, false, kOneOdd, 4>), grid_of<kOneOdd>(c.batch, p.l.slabs), threads, 0, s, p);
        e = hipGetLastError();
        if (c.batch == 1) return e;
    } else {
        hipLaunchKernelGGL((p.l.merged ? k_group_back_sums<T, true> : k_group_back_sums<T, false>),
                           grid_of<kGroupThreads>(p.blocks, p.l.slabs), threads, 0, s, p);
        if (p.out) {
            if (p.stat) group_join<T, true>(p, s);
            const long long more = p.cols ? (2LL * p.channels + 3) / 4 : 0;
            hipLaunchKernelGGL((p.l.merged ? k_group_back<T, true> : k_group_back<T, false>),
                               grid_of<kGroupThreads>(p.blocks + more, p.l.slabs), threads, 0, s, p);
            return hipGetLastError();
        }
        e = hipGetLastError();
    }
    if (e != hipSuccess || !p.cols) return e;
    return launch_column_sums(p.cols, (int)p.places, 2LL * p.channels, p.channels, c.dgamma, c.dbeta, dtype, s);
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
