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
// (k_group_one, k_group_back_one).  Only the device knows the sizes of samples that offsets name: where one of them could hold a workgroup
// up, it leaves those above `over` rows to the blocks of rows, which then take no others.
//
// Blocks of rows are cut without regard to the samples, whose sizes only the device knows: block i keeps one set of sums for
// every sample that it meets, in place i + b (along the rows either i or b grows by one, so that no place is taken twice), and
// sets what no pair (i, b) takes to 0.  Sums are added in a fixed order: the same bits every time.
// The forward sums are those of x - s and its square, s the first value of the sample's group, in fp64: what cancels in
// var = (sum d^2 - (sum d)^2 / n) / n is then bits that fp64 has to spare (a spread of 1e-5 of the distance between s and the
// mean leaves 2^-53 x 1e10 of it), and a group of equal values has exactly none.
#include "scnn_dense.h"

namespace scnn {

constexpr int kGroupThreads = 256;  // most threads of a workgroup that takes a block of rows
constexpr int kHereGroups = 64;     // most groups of a slab whose sums a workgroup joins by itself

// How threads lie over columns.  A workgroup takes `wide` columns from c0 on: tv threads a row, a vector each, `reps` rows at
// a time.  Rows of all C columns that are no whole number of vectors run on without a gap (flat): `active` vectors are `reps`
// whole rows, so that a thread meets the same columns at every step; value i of thread t is then number t V + i of a step, and row k's
// column c number k C + c.
struct GroupLayout {
    int tv, reps, active, flat;
    int wide, slabs, pieces;  // a slab is whole groups (pieces 1), or one of `pieces` pieces of a group
    int merged;               // a vector's columns are of one group, and none is cut
    int sub;                  // 2^sub neighbouring values of a vector are of one group, whatever the vector
    float inv_tv, inv_per, inv_c;
    double inv_reps;
};

struct GroupArgs {
    const void *x, *g, *gamma, *beta;
    void *out, *dgamma, *dbeta;  // out: forward out, backward dx
    float *mean, *rstd;          // [batch][groups]: written forward, read backward
    const long long* offsets;
    long long each;              // rows of a sample where offsets is null
    long long rows, chunk;       // chunk: rows of a block
    long long over;              // samples of more rows are the blocks', the others a workgroup's each; 0: no such division
    long long batch, blocks, places, sum_blocks;
    double inv_each, inv_chunk;
    int channels, groups, per, act;
    float eps;
    float* cols;                 // backward: [places][2][channels], sums of dz xh and dz over a place's rows ([blocks] with `over`); null: not wanted
    void* part;                  // [places][groups * pieces]: forward {sum d, sum d^2} in fp64, backward {sum h, sum h xh} in fp32
    void* stat;                  // [batch][groups] of k_group_join; null: joined where they are used
    GroupLayout l;
};

// a / d for whole numbers a < 2^21 by way of 1 / d in fp32: (a + 1/2) / d is no nearer to a whole number than 1 / (2 d).
__device__ __forceinline__ int quotient(int a, float inverse) { return (int)(((float)a + 0.5f) * inverse); }
// The same for a < 2^31.  (A division of 64 bits is a hundred instructions.)
__device__ __forceinline__ long long quotient(long long a, double inverse) { return (long long)(unsigned)(((double)(unsigned)a + 0.5) * inverse); }

// The samples' bounds.  Up to 63 samples a wave holds them all, a lane each.
struct Bounds {
    const long long* offsets;
    long long each, rows, batch, lane_row;
    double inv_each;
    bool here;
};
__device__ __forceinline__ Bounds bounds_of(const GroupArgs& p) {
    Bounds s = {p.offsets, p.each, p.rows, p.batch, 0, p.inv_each, p.offsets != nullptr && p.batch < 64};
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
    if (s.here)  // (rows: fewer than 2^31)
        return (unsigned)__builtin_amdgcn_readlane((int)s.lane_row, __builtin_amdgcn_readfirstlane((int)b));
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
        b = s.each > 0 ? quotient(r, s.inv_each) : 0;
    } else if (s.here) {
        const int lane = threadIdx.x & 63;
        b = __popcll(__ballot(lane > 0 && lane <= s.batch && s.lane_row <= r));
    } else {
        b = count_up_to(s.batch, r, [&](long long k) { return first_row(s, k + 1); });
    }
    return uniform(b < s.batch ? b : s.batch - 1);
}

// Rows of block i, and the samples whose sums it keeps.  (Of those above `over` rows, which is no less than a block's, a block holds an end
// at least: only the samples of its first and its last row are looked at.)
struct Block { long long r0, r1, b0, b1; };
template <bool OVER>
__device__ __forceinline__ Block block_of(const GroupArgs& p, const Bounds& s, long long i) {
    Block k;
    k.r0 = i * p.chunk;
    k.r1 = k.r0 + p.chunk < p.rows ? k.r0 + p.chunk : p.rows;
    k.b0 = i == 0 && !OVER ? 0 : sample_at(s, k.r0);
    k.b1 = OVER ? sample_at(s, k.r1 - 1) : (i + 1 == p.blocks ? p.batch - 1 : sample_at(s, k.r1));
    return k;
}
__device__ __forceinline__ bool any_over(const GroupArgs& p, const Bounds& s, const Block& k) {
    const Rows a = rows_of_sample(s, k.b0), b = rows_of_sample(s, k.b1);
    return a.end - a.first > p.over || b.end - b.first > p.over;
}
template <bool OVER>
__device__ __forceinline__ long long next_sample(const Block& k, long long b) { return OVER && b < k.b1 ? k.b1 : b + 1; }

// Columns of slab s, its first group, the number of its groups and their width in it.
struct Slab { int c0, c1, j0, ng, w; };
__device__ __forceinline__ Slab slab_of(const GroupArgs& p, int s) {
    if (p.l.slabs == 1) return {0, p.channels, 0, p.groups, p.per};
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
        a.j0 = a.c0 / p.per;
        a.ng = (a.c1 - a.c0) / p.per;
        a.w = p.per;
    }
    return a;
}

// This thread's place: its row among a step's, its first column in the slab.  A vector that the slab's end cuts is the slab's last whole
// one instead (it may begin before the slab), of which the first `other` values are another thread's: read, but neither
// added nor written.  (Cut vectors taken value by value behind the others: forward 60000 x 517 bf16 in 11 groups 122 us, so 59 at the time.)
struct Place { int row, col, other; };
template <int V>
__device__ __forceinline__ Place place_of(const GroupArgs& p, const Slab& a) {
    const int t = threadIdx.x;
    if (p.l.flat) return {0, t * V, 0};
    const int k = quotient(t, p.l.inv_tv), c = (t - k * p.l.tv) * V, over = c + V - (a.c1 - a.c0);
    return over <= 0 ? Place{k, c, 0} : Place{k, c - over, over < V ? over : V};
}
// Column in the slab of value i of this thread, or one of the slab's where it has none.
__device__ __forceinline__ int column_of(const GroupArgs& p, const Slab& a, const Place& t, int i) {
    int c = t.col + i;
    c -= quotient(c, p.l.inv_c) * p.channels;  // (inv_c is 0 where rows do not run on)
    return c < 0 ? 0 : (c < a.c1 - a.c0 ? c : a.c1 - a.c0 - 1);
}
// Group in the slab of a column of it.
__device__ __forceinline__ int group_of(const GroupArgs& p, int column) { return quotient(column, p.l.inv_per); }  // (inv_per is 0 in pieces)

// A thread's vectors among the rows lo .. hi - 1: `full` whole ones, of which all threads that have any have `common` (the same in every
// lane); behind those of rows that run on, n values.
struct Walk {
    long long at, step;
    int full, n, common, other;
};
template <int V>
__device__ __forceinline__ Walk walk_of(const GroupArgs& p, const Slab& a, const Place& t, long long lo, long long hi) {
    Walk w = {0, 0, 0, 0, 0, t.other};
    if (hi <= lo) return w;
    const int steps = __builtin_amdgcn_readfirstlane((int)quotient(hi - lo, p.l.inv_reps));
    w.common = steps;
    if ((int)threadIdx.x >= p.l.active || t.other >= V) return w;
    const int left = (int)(hi - lo - (long long)steps * p.l.reps);
    w.step = (long long)p.l.reps * p.channels;
    w.full = steps;
    if (p.l.flat) {
        w.at = lo * p.channels + t.col;
        const int n = left * p.channels - t.col;  // (fewer than a step's values)
        if (n >= V) ++w.full;
        else if (n > 0) w.n = n;
    } else {
        w.at = (lo + t.row) * p.channels + a.c0 + t.col;
        if (t.row < left) ++w.full;
    }
    return w;
}

template <typename T> using Loose = VecOf<T, kVec<T>> __attribute__((aligned(sizeof(T))));  // (at any element's address)
template <typename T> __device__ __forceinline__ VecOf<T, kVec<T>> take(const T* p) { return *(const Loose<T>*)p; }
// Results are not read again soon: they leave the L2 to the rows.
template <typename T> __device__ __forceinline__ void put(T* p, VecOf<T, kVec<T>> v, int other) {
    typedef unsigned __int128 u128;
    if (other == 0) __builtin_nontemporal_store(v, (Loose<T>*)p);
    else store_raw<T>(p + other, kVec<T> - other, __builtin_bit_cast(VecOf<T, kVec<T>>, __builtin_bit_cast(u128, v) >> (other * 8 * (int)sizeof(T))));
}

// Vector number k of a thread, counted from its first one or, DOWN, from its last one (the last ones of a block are what the L2 still
// has when its rows are read again).
template <bool DOWN> __device__ __forceinline__ long long position(const Walk& w, int k) { return w.at + (long long)(DOWN ? w.full - 1 - k : k) * w.step; }
// U vectors of a thread on their way, from number k on.
template <typename T, int U, bool DOWN>
__device__ __forceinline__ void fetch(const T* __restrict__ x, const Walk& w, int k, VecOf<T, kVec<T>> (&r)[U]) {
#pragma unroll
    for (int u = 0; u < U; ++u)
        if (k + u < w.full) r[u] = take(x + position<DOWN>(w, k + u));
}
// Calls use(slot, k) for a thread's vectors from number k up to `end`; the first U are there, and each slot is loaded again as soon as it
// was used: load(slot, k).  Steps that all threads have run without a condition, so that a wait counts the loads behind it.  (Loaded all at
// once behind the last use: forward 643072 x 64 fp32 82.6 us, so 78.5; backward 209645 x 25 fp32 37, so 33.)
template <int U, typename Use, typename Load>
__device__ __forceinline__ void walk(const Walk& w, int k, int end, Use use, Load load) {
    if (k >= end) return;
    for (const int common = w.common - (w.full - end); k + 2 * U <= common; k += U)
#pragma unroll
        for (int u = 0; u < U; ++u) {
            use(u, k + u);
            load(u, k + U + u);
            __builtin_amdgcn_sched_barrier(0);
        }
    for (; k < end; k += U)
#pragma unroll
        for (int u = 0; u < U; ++u)
            if (k + u < end) {
                use(u, k + u);
                if (k + U + u < end) load(u, k + U + u);
                __builtin_amdgcn_sched_barrier(0);
            }
}

__device__ __forceinline__ float finite_or_zero(float v) { return __builtin_fabsf(v) < __builtin_huge_valf() ? v : 0.0f; }

struct Two { double a, b; };
__device__ __forceinline__ Two lanes_two(Two v, int q) {
    for (int d = 1; d < q; d <<= 1) {
        v.a += __shfl_xor(v.a, d, 64);
        v.b += __shfl_xor(v.b, d, 64);
    }
    return v;
}

// ------------------------------------------------------------------ forward
// Accumulators of a thread: one a column, or two for all of a vector's columns where these are of one group.
template <typename T, bool M> constexpr int kSums = M ? 2 : kVec<T>;
template <typename T, bool M>
struct Sums { double s[kSums<T, M>], one[kSums<T, M>], two[kSums<T, M>]; };

// The first value of each accumulator's group in row `origin`.
template <typename T, bool M>
__device__ __forceinline__ void first_values(const GroupArgs& p, const Slab& a, const Place& t, long long origin, float (&s)[kSums<T, M>]) {
    const T* __restrict__ x = (const T*)p.x + origin * p.channels + (long long)a.j0 * p.per;
#pragma unroll
    for (int i = 0; i < kSums<T, M>; ++i)
        s[i] = M && i ? s[0] : (float)x[(long long)group_of(p, column_of(p, a, t, i)) * p.per];
}
template <typename T, bool M>
__device__ __forceinline__ void begin_sums(const float (&near)[kSums<T, M>], Sums<T, M>& v) {
#pragma unroll
    for (int i = 0; i < kSums<T, M>; ++i) {
        v.s[i] = (double)finite_or_zero(near[i]);
        v.one[i] = v.two[i] = 0.0;
    }
}
template <typename T, bool M>
__device__ __forceinline__ void add_value(float x, int i, Sums<T, M>& v) {
    const int k = M ? i & 1 : i;
    const double d = (double)x - v.s[k];
    v.one[k] += d;
    v.two[k] = __builtin_fma(d, d, v.two[k]);
}
// Sums over a thread's vectors from number k on, of which the first U are there, and over its odd values.
template <typename T, bool M, int U>
__device__ __forceinline__ void sum_from(const T* __restrict__ x, const Walk& w, int k, VecOf<T, kVec<T>> (&r)[U], Sums<T, M>& v) {
    constexpr int V = kVec<T>;
    walk<U>(w, k, w.full,
            [&](int u, int) {
#pragma unroll
                for (int i = 0; i < V; ++i) add_value<T, M>((float)r[u][i], i, v);
            },
            [&](int u, int n) { r[u] = take(x + position<false>(w, n)); });
    if (w.n) {
        const long long at = w.at + (long long)w.full * w.step;
#pragma unroll
        for (int i = 0; i < V - 1; ++i)
            if (i < w.n) add_value<T, M>((float)x[at + i], i, v);
    }
}

// Lanes that add the n values of each of `groups` sums, as a power of two: no more than there are values, threads for them all, or lanes
// of a wave.
__device__ __forceinline__ int lane_bits(int n, int groups) {
    int q = 0;
    while (1 << q < n && q < 6 && 2 * groups << q <= (int)blockDim.x) ++q;
    return q;
}
// Where the numbers of a step lie in LDS: number i of each thread beside that of the others (lanes that write meet different banks), the
// arrays of two i one number apart from being so many banks apart.  2^sub neighbouring values are one number, 2^v a vector.
__device__ __forceinline__ int step_at(const GroupArgs& p, int v, int sub, int row, int column) {
    const int e = p.l.flat ? row * p.channels + column : column >> sub, each = v - sub;
    return (e & ((1 << each) - 1)) * (p.l.active + 1) + (p.l.flat ? e >> each : row * p.l.tv + (e >> each));
}

// Sums over the slab's groups of the threads' pairs, then done(group, sums) by one lane a group.  All threads of the workgroup call it.
template <typename T, bool M, typename F>
__device__ __forceinline__ void add_groups(const GroupArgs& p, const Slab& a, const Place& t, const Sums<T, M>& v, Two* s_all, F done) {
    constexpr int V = kVec<T>;
    constexpr int VB = V == 8 ? 3 : 2;
    const int sub = M ? VB : p.l.sub, w = (a.w + (1 << sub) - 1) >> sub, next = p.l.active + 1;
    Two* const mine = s_all + threadIdx.x - (t.other >> sub) * next;
    if ((int)threadIdx.x < p.l.active) {
        if constexpr (M) {
            s_all[threadIdx.x] = {v.one[0] + v.one[1], v.two[0] + v.two[1]};
        } else if (sub == 0) {
#pragma unroll
            for (int i = 0; i < V; ++i)
                if (i >= t.other) mine[i * next] = {v.one[i], v.two[i]};
        } else if (sub == 1) {
#pragma unroll
            for (int i = 0; i < V; i += 2)
                if (i >= t.other) mine[i / 2 * next] = {v.one[i] + v.one[i + 1], v.two[i] + v.two[i + 1]};
        } else if constexpr (V == 8) {
#pragma unroll
            for (int i = 0; i < V; i += 4)
                if (i >= t.other)
                    mine[i / 4 * next] = {(v.one[i] + v.one[i + 1]) + (v.one[i + 2] + v.one[i + 3]), (v.two[i] + v.two[i + 1]) + (v.two[i + 2] + v.two[i + 3])};
        }
    }
    __syncthreads();
    const int n = w * p.l.reps, bits = lane_bits(n, a.ng), q = 1 << bits;
    const float inv = 1.0f / (float)w;
    const int set = threadIdx.x >> bits, sets = blockDim.x >> bits, in = threadIdx.x & (q - 1);
    for (int j0 = 0; j0 < a.ng; j0 += sets) {
        const int j = j0 + set;
        Two sum = {0.0, 0.0};
        if (j < a.ng)
            for (int e = in; e < n; e += q) {
                const int k = quotient(e, inv);
                const Two o = s_all[step_at(p, VB, sub, k, (j * w + (e - k * w)) << sub)];
                sum.a += o.a;
                sum.b += o.b;
            }
        sum = lanes_two(sum, q);
        if (in == 0 && j < a.ng) done(j, sum);
    }
}

struct GroupStat { float mean, rest, rstd, none; };
// Statistics of n values from their sums about s.
__device__ __forceinline__ GroupStat stat_of(float near, Two sum, double n, float eps) {
    const double s = (double)finite_or_zero(near), inv = 1.0 / n, off = sum.a * inv, mean = s + off;
    double var = (sum.b - sum.a * off) * inv;
    if (var < 0.0) var = 0.0;  // (a NaN stays one)
    // 1 / sqrt by one step of Newton's from the instruction's estimate (2^-23 or better): far past fp32's rounding
    const double v = var + (double)eps, y = __builtin_amdgcn_rsq(v), half = __builtin_fma(-0.5 * v * y, y, 0.5);
    GroupStat r;
    r.mean = (float)mean;
    r.rest = (float)(mean - (double)r.mean);
    r.rstd = half == half ? (float)__builtin_fma(y, half, y) : (float)y;  // (no step from 0, infinity and NaN)
    r.none = 0.0f;
    return r;
}

// gamma and beta of a thread's columns, 1 and 0 where there are none.
template <typename T>
struct Affine { VecOf<T, kVec<T>> gamma, beta; };
template <typename T>
__device__ __forceinline__ VecOf<T, kVec<T>> column_values(const GroupArgs& p, const Slab& a, const Place& t, const void* from, float none) {
    constexpr int V = kVec<T>;
    VecOf<T, V> v;
    if (!from) {
#pragma unroll
        for (int i = 0; i < V; ++i) v[i] = (T)none;
    } else if (!p.l.flat) {
        v = take((const T*)from + a.c0 + t.col);
    } else {
#pragma unroll
        for (int i = 0; i < V; ++i) v[i] = ((const T*)from)[a.c0 + column_of(p, a, t, i)];
    }
    return v;
}
template <typename T>
__device__ __forceinline__ Affine<T> affine_of(const GroupArgs& p, const Slab& a, const Place& t) {
    return {column_values<T>(p, a, t, p.gamma, 1.0f), column_values<T>(p, a, t, p.beta, 0.0f)};
}

// What the forward pass knows of a thread's columns (mean and what its rounding leaves once, where they are of one group).
template <int V, int A>
struct Columns { float mean[A], rest[A], scale[V], beta[V]; };
template <typename T, bool M>
__device__ __forceinline__ Columns<kVec<T>, M ? 1 : kVec<T>> columns_of(const GroupArgs& p, const Slab& a, const Place& t, const Affine<T>& f,
                                                                       const GroupStat* stat) {
    constexpr int V = kVec<T>, A = M ? 1 : V;
    Columns<V, A> k;
    GroupStat s = {};
#pragma unroll
    for (int i = 0; i < V; ++i) {
        if (i < A) {
            s = stat[group_of(p, column_of(p, a, t, i))];
            k.mean[i] = s.mean;
            k.rest[i] = s.rest;
        }
        k.scale[i] = s.rstd * (float)f.gamma[i];
        k.beta[i] = (float)f.beta[i];
    }
    return k;
}
template <int V, int A>
__device__ __forceinline__ float forward_value(const Columns<V, A>& k, int i, float x) {  // z
    const int j = A == 1 ? 0 : i;
    return __builtin_fmaf((x - k.mean[j]) - k.rest[j], k.scale[i], k.beta[i]);
}
template <typename T, int A>
__device__ __forceinline__ void forward_vector(const GroupArgs& p, const Columns<kVec<T>, A>& k, const Walk& w, long long at, VecOf<T, kVec<T>> r) {
    constexpr int V = kVec<T>;
    VecOf<T, V> y;
    float z[V];
#pragma unroll
    for (int i = 0; i < V; ++i) z[i] = forward_value<V, A>(k, i, (float)r[i]);
    activate_all<V>(z, p.act);
#pragma unroll
    for (int i = 0; i < V; ++i) y[i] = (T)z[i];
    put((T*)p.out + at, y, A == 1 ? 0 : w.other);
}
// A thread's vectors from its last down to number `from`, of which the first U are there, and its odd values.
template <typename T, int A, int U>
__device__ __forceinline__ void forward_down(const GroupArgs& p, const Columns<kVec<T>, A>& c, const Walk& w, int from,
                                             VecOf<T, kVec<T>> (&r)[U]) {
    walk<U>(w, 0, w.full - from, [&](int u, int n) { forward_vector<T, A>(p, c, w, position<true>(w, n), r[u]); },
            [&](int u, int n) { r[u] = take((const T*)p.x + position<true>(w, n)); });
    if (w.n) {
        const long long at = w.at + (long long)w.full * w.step;
#pragma unroll
        for (int i = 0; i < kVec<T> - 1; ++i)
            if (i < w.n) ((T*)p.out)[at + i] = (T)activate(forward_value<kVec<T>, A>(c, i, (float)((const T*)p.x)[at + i]), p.act);
    }
}

constexpr int kAhead = 4;  // vectors of x that a thread of the blocks' kernels has on their way

// Sums of a block's rows.  643072 x 64 fp32 in 8 groups: 26 us, 6.4 TB/s of x (caches hold some of it), bound by memory; the fp64 sums of
// 23651 x 16 bf16 take 9 us, where a workgroup has one step: its start, two loads behind one another, LDS.
template <typename T, bool M, bool OVER>
__device__ __forceinline__ void block_sums(const GroupArgs& p, long long i, int slab, char* s_step) {
    constexpr int V = kVec<T>;
    if (i >= p.blocks) return;
    const Bounds s = bounds_of(p);
    const Block k = block_of<OVER>(p, s, i);
    if (OVER && !any_over(p, s, k)) return;
    const Slab a = slab_of(p, slab);
    const Place t = place_of<V>(p, a);
    const int to = p.l.pieces > 1 ? slab : a.j0;
    for (long long b = k.b0; b <= k.b1; b = next_sample<OVER>(k, b)) {
        const Rows r = rows_of_sample(s, b);
        if (OVER && r.end - r.first <= p.over) continue;
        const long long lo = r.first > k.r0 ? r.first : k.r0, hi = r.end < k.r1 ? r.end : k.r1;
        Two* const part = (Two*)p.part + (i + b) * p.groups * p.l.pieces + to;
        if (hi <= lo) {
            for (int j = threadIdx.x; j < a.ng; j += blockDim.x) part[j] = {0.0, 0.0};
            continue;
        }
        // (the first vectors are on their way with the values that they are taken about)
        float near[kSums<T, M>];
        const Walk w = walk_of<V>(p, a, t, lo, hi);
        VecOf<T, V> x[kAhead];
        first_values<T, M>(p, a, t, r.first, near);
        fetch<T, kAhead, false>((const T*)p.x, w, 0, x);
        Sums<T, M> v;
        begin_sums<T, M>(near, v);
        sum_from<T, M, kAhead>((const T*)p.x, w, 0, x, v);
        add_groups<T, M>(p, a, t, v, (Two*)s_step, [&](int j, Two sum) { part[j] = sum; });
        if (b < k.b1) __syncthreads();
    }
}
template <typename T, bool M>
__global__ __launch_bounds__(kGroupThreads, 2) void k_group_sums(GroupArgs p) {
    extern __shared__ __align__(16) char s_step[];
    block_sums<T, M, false>(p, block_id<kGroupThreads>(), blockIdx.y, s_step);
}

// Sum over the Q threads (a power of two up to 256) of each of a workgroup's sets; all 256 threads call it.
__device__ __forceinline__ Two set_add(Two v, int q, Two* s_wave) {
    v = lanes_two(v, q < 64 ? q : 64);
    if (q <= 64) return v;
    if ((threadIdx.x & 63) == 0) s_wave[threadIdx.x >> 6] = v;
    __syncthreads();
    const int w = threadIdx.x / q * (q / 64);
    v = {0.0, 0.0};
    for (int k = 0; k < q / 64; ++k) {
        v.a += s_wave[w + k].a;
        v.b += s_wave[w + k].b;
    }
    return v;
}

// The places that hold the sums of a sample: from, and how many.
__device__ __forceinline__ long long places_of(const GroupArgs& p, long long b, const Rows& r, int& count) {
    const long long i0 = quotient(r.first, p.inv_chunk), i1 = quotient(r.end - 1, p.inv_chunk);
    count = (int)(i1 - i0) + 1;
    return i0 + b;
}
template <typename T>
__device__ __forceinline__ float near_value(const GroupArgs& p, const Rows& r, int j) {
    return (float)((const T*)p.x)[r.first * p.channels + (long long)j * p.per];
}

// Q threads for each sample and group.  BACK: means of h and h xh, else the statistics.
template <typename T, bool BACK>
__global__ __launch_bounds__(256) void k_group_join(GroupArgs p, int q) {
    typedef typename std::conditional<BACK, float, double>::type F;
    __shared__ Two s_wave[4];
    const long long id = block_id<256>() * (256 / q) + threadIdx.x / q;
    const int in = threadIdx.x & (q - 1);
    bool live = id < p.batch * p.groups;
    const long long b = live ? id / p.groups : 0;
    const int j = (int)(live ? id - b * p.groups : 0);
    const Bounds s = {p.offsets, p.each, p.rows, p.batch, 0, p.inv_each, false};  // (b differs from lane to lane)
    Rows r = {first_row(s, b), first_row(s, b + 1)};
    if (r.end < r.first) r.end = r.first;
    live = live && (p.over == 0 || r.end - r.first > p.over);
    Two sum = {0.0, 0.0};
    if (live && r.end > r.first) {
        int count;
        const long long from = places_of(p, b, r, count);
        const F* __restrict__ part = (const F*)p.part;
        const int pieces = p.l.pieces;
        const long long n = (long long)count * pieces;
        // (four at a time: a load behind the other takes a microsecond each)
        for (long long e0 = in; e0 < n; e0 += 4LL * q) {
            F two[4][2];
#pragma unroll
            for (int u = 0; u < 4; ++u) {
                const long long e = e0 + u * q < n ? e0 + u * q : n - 1, i = pieces > 1 ? e / pieces : e;
                __builtin_memcpy(two[u], part + (((from + i) * p.groups + j) * pieces + (e - i * pieces)) * 2, sizeof(two[u]));
            }
#pragma unroll
            for (int u = 0; u < 4; ++u)
                if (e0 + u * q < n) {
                    sum.a += (double)two[u][0];
                    sum.b += (double)two[u][1];
                }
        }
    }
    sum = set_add(sum, q, s_wave);
    if (!live || in != 0) return;
    if constexpr (BACK) {
        const double n = r.end > r.first ? (double)(r.end - r.first) * p.per : 1.0;
        ((float2*)p.stat)[id] = make_float2((float)(sum.a / n), (float)(sum.b / n));
    } else {
        GroupStat v = {0.0f, 0.0f, 0.0f, 0.0f};
        if (r.end > r.first) v = stat_of(near_value<T>(p, r, j), sum, (double)(r.end - r.first) * p.per, p.eps);
        ((GroupStat*)p.stat)[id] = v;
        if (p.mean) p.mean[id] = v.mean;
        if (p.rstd) p.rstd[id] = v.rstd;
    }
}

// The sums of a sample's groups by one workgroup: threads side by side take neighbouring groups of a place, their sums meet in
// s_two, then one lane a group ends with them (group k < ng, lane 0 of its q).  All threads call it; up to kHereGroups groups.
struct Joiner { int sets, set, j, q, k, in; };
__device__ __forceinline__ Joiner joiner_of(const Slab& a) {
    Joiner o;
    const float inv = 1.0f / (float)a.ng;
    o.sets = quotient((int)blockDim.x, inv);
    o.set = quotient((int)threadIdx.x, inv);
    o.j = threadIdx.x - o.set * a.ng;
    const int bits = lane_bits(o.sets, a.ng);
    o.q = 1 << bits;
    o.k = threadIdx.x >> bits;
    o.in = threadIdx.x & (o.q - 1);
    return o;
}
template <typename F>
__device__ __forceinline__ Two join_here(const GroupArgs& p, const Slab& a, const Joiner& o, long long b, const Rows& r, Two* s_two) {
    int count;
    const long long from = places_of(p, b, r, count);
    Two sum = {0.0, 0.0};
    if (o.set < o.sets) {
        const F* __restrict__ part = (const F*)p.part + (from * p.groups + a.j0 + o.j) * 2;
        for (int i = o.set; i < count; i += 4 * o.sets) {  // (four at a time, as in k_group_join)
            F two[4][2];
#pragma unroll
            for (int u = 0; u < 4; ++u)
                __builtin_memcpy(two[u], part + (long long)(i + u * o.sets < count ? i + u * o.sets : count - 1) * p.groups * 2, sizeof(two[u]));
#pragma unroll
            for (int u = 0; u < 4; ++u)
                if (i + u * o.sets < count) {
                    sum.a += (double)two[u][0];
                    sum.b += (double)two[u][1];
                }
        }
    }
    __syncthreads();
    s_two[threadIdx.x] = sum;
    __syncthreads();
    sum = {0.0, 0.0};
    if (o.k < a.ng)
        for (int e = o.in; e < o.sets; e += o.q) {
            sum.a += s_two[e * a.ng + o.k].a;
            sum.b += s_two[e * a.ng + o.k].b;
        }
    return lanes_two(sum, o.q);
}

// Results of a block's rows, its last ones first.  643072 x 64 fp32: 50 us, 6.5 TB/s read and written, bound by memory.
template <typename T, bool M, bool OVER>
__global__ __launch_bounds__(kGroupThreads, 2) void k_group_apply(GroupArgs p) {
    constexpr int V = kVec<T>, A = M ? 1 : V;
    __shared__ Two s_two[kGroupThreads];
    __shared__ GroupStat s_stat[kHereGroups];
    const long long i = block_id<kGroupThreads>();
    if (i >= p.blocks) return;
    const Bounds s = bounds_of(p);
    const Block k = block_of<OVER>(p, s, i);
    if (OVER && !any_over(p, s, k)) return;
    const Slab a = slab_of(p, blockIdx.y);
    const Place t = place_of<V>(p, a);
    const Affine<T> f = affine_of<T>(p, a, t);
    const Joiner o = joiner_of(a);
    for (long long b = k.b0; b <= k.b1; b = next_sample<OVER>(k, b)) {
        const Rows r = rows_of_sample(s, b);
        if (OVER && r.end - r.first <= p.over) continue;
        const long long lo = r.first > k.r0 ? r.first : k.r0, hi = r.end < k.r1 ? r.end : k.r1, id = b * p.groups + a.j0;
        if (!p.stat && r.end == r.first)  // (by every workgroup that passes the empty sample)
            for (int j = threadIdx.x; j < a.ng; j += blockDim.x) {
                if (p.mean) p.mean[id + j] = 0.0f;
                if (p.rstd) p.rstd[id + j] = 0.0f;
            }
        if (hi <= lo) continue;
        const Walk w = walk_of<V>(p, a, t, lo, hi);
        // (the last vectors are on their way while the sums are joined)
        VecOf<T, V> x[kAhead];
        fetch<T, kAhead, true>((const T*)p.x, w, 0, x);
        const GroupStat* stat = (const GroupStat*)p.stat + id;
        if (!p.stat) {
            const bool ends = o.k < a.ng && o.in == 0;
            const float near = ends ? near_value<T>(p, r, a.j0 + o.k) : 0.0f;
            const Two sum = join_here<double>(p, a, o, b, r, s_two);
            if (ends) {
                const GroupStat v = stat_of(near, sum, (double)(r.end - r.first) * p.per, p.eps);
                s_stat[o.k] = v;
                if (r.first >= k.r0) {
                    if (p.mean) p.mean[id + o.k] = v.mean;
                    if (p.rstd) p.rstd[id + o.k] = v.rstd;
                }
            }
            __syncthreads();
            stat = s_stat;
        }
        const Columns<V, A> c = columns_of<T, M>(p, a, t, f, stat);
        forward_down<T, A, kAhead>(p, c, w, 0, x);
    }
}

// A sample's slab of whole groups by one workgroup of up to B threads, H vectors a thread in registers; what a larger sample has
// more is read again.  One launch and one reading: 512 x 24 fp32 in 8 groups 7 us, bound by latency (a load, LDS, a store).
template <typename T, bool M, int H, bool OVER>
__device__ __forceinline__ void one_forward(const GroupArgs& p, long long b, char* s_step) {
    constexpr int V = kVec<T>, A = M ? 1 : V;
    GroupStat* const s_stat = (GroupStat*)s_step;
    Two* const s_all = (Two*)(s_stat + p.l.wide / p.per);
    if (b >= p.batch) return;
    const Bounds s = {p.offsets, p.each, p.rows, p.batch, 0, p.inv_each, false};
    const Slab a = slab_of(p, blockIdx.y);
    const Place t = place_of<V>(p, a);
    const Rows r = rows_of_sample(s, b);
    const long long id = b * p.groups + a.j0;
    if (r.end == r.first) {
        for (int j = threadIdx.x; j < a.ng; j += blockDim.x) {
            if (p.mean) p.mean[id + j] = 0.0f;
            if (p.rstd) p.rstd[id + j] = 0.0f;
        }
        return;
    }
    if (OVER && r.end - r.first > p.over) return;
    const T* __restrict__ x = (const T*)p.x;
    const Walk w = walk_of<V>(p, a, t, r.first, r.end);
    float near[kSums<T, M>];
    first_values<T, M>(p, a, t, r.first, near);
    VecOf<T, V> held[H];
    fetch<T, H, false>(x, w, 0, held);
    const Affine<T> f = affine_of<T>(p, a, t);
    Sums<T, M> v;
    begin_sums<T, M>(near, v);
#pragma unroll
    for (int h = 0; h < H; ++h)
        if (h < w.full) {
#pragma unroll
            for (int i = 0; i < V; ++i) add_value<T, M>((float)held[h][i], i, v);
            __builtin_amdgcn_sched_barrier(0);
        }
    VecOf<T, V> more[2];
    fetch<T, 2, false>(x, w, H, more);
    sum_from<T, M, 2>(x, w, H, more, v);
    add_groups<T, M>(p, a, t, v, s_all, [&](int j, Two sum) {
        const GroupStat g = stat_of(near_value<T>(p, r, a.j0 + j), sum, (double)(r.end - r.first) * p.per, p.eps);
        s_stat[j] = g;
        if (p.mean) p.mean[id + j] = g.mean;
        if (p.rstd) p.rstd[id + j] = g.rstd;
    });
    __syncthreads();
    const Columns<V, A> c = columns_of<T, M>(p, a, t, f, s_stat);
#pragma unroll
    for (int h = 0; h < H; ++h)
        if (h < w.full) {
            forward_vector<T, A>(p, c, w, position<false>(w, h), held[h]);
            __builtin_amdgcn_sched_barrier(0);
        }
    if (w.full > H) fetch<T, 2, true>(x, w, 0, more);
    forward_down<T, A, 2>(p, c, w, H, more);
}
template <typename T, bool M, int B, int H>
__global__ __launch_bounds__(B, 2) void k_group_one(GroupArgs p) {
    extern __shared__ __align__(16) char s_step[];
    one_forward<T, M, H, false>(p, block_id<B>(), s_step);
}
// Number of a workgroup among those behind the ones that take a sample and slab each, which lie along the grid's x and y: in further columns
// of the grid or in further rows; below 0: it is one of these.
__device__ __forceinline__ long long number_behind(const GroupArgs& p, long long id) {
    const int y = blockIdx.y;
    if (y >= p.l.slabs) return (y - p.l.slabs) * p.batch + id;
    return id < p.batch ? -1 : (id - p.batch) * p.l.slabs + y;
}
// Samples of up to `over` rows; workgroups behind theirs add the blocks' sums of the others.
template <typename T, bool M, int B, int H>
__global__ __launch_bounds__(B, 2) void k_group_one_sums(GroupArgs p, GroupArgs blocks) {
    extern __shared__ __align__(16) char s_step[];
    const long long id = block_id<B>(), at = number_behind(p, id);
    if (at < 0) one_forward<T, M, H, true>(p, id, s_step);
    else if (at < blocks.blocks * blocks.l.slabs) block_sums<T, M, true>(blocks, (unsigned)at / blocks.l.slabs, (unsigned)at % blocks.l.slabs, s_step);
}

// ------------------------------------------------------------------ backward
// What the backward pass knows of a thread's columns (mean and rstd once where they are of one group).
template <int V, int A>
struct BackColumns { float mean[A], rstd[A], gamma[V], beta[V]; };
template <typename T, bool M>
__device__ __forceinline__ BackColumns<kVec<T>, M ? 1 : kVec<T>> back_columns(const GroupArgs& p, const Slab& a, const Place& t, const Affine<T>& f,
                                                                             long long b) {
    constexpr int V = kVec<T>, A = M ? 1 : V;
    BackColumns<V, A> k;
#pragma unroll
    for (int i = 0; i < A; ++i) {
        const long long s = b * p.groups + a.j0 + group_of(p, column_of(p, a, t, i));
        k.mean[i] = p.mean[s];
        k.rstd[i] = p.rstd[s];
    }
#pragma unroll
    for (int i = 0; i < V; ++i) {
        k.gamma[i] = (float)f.gamma[i];
        k.beta[i] = (float)f.beta[i];
    }
    return k;
}
// xh and dz of N values of a thread, whose columns are those from i0 on.  relu's slope hangs on the sign of z alone, and in fp32 one z
// in some ten million lies on the wrong side of 0 and takes a whole gradient with it: what is nearer to 0 than 8 roundings of its
// parts (three are made) is formed anew in fp64.
template <int V, int A, int N>
__device__ __forceinline__ void back_values(const BackColumns<V, A>& k, int i0, const float (&x)[N], const float (&g)[N], int act, float (&xh)[N],
                                            float (&dz)[N]) {
    float z[N];
#pragma unroll
    for (int i = 0; i < N; ++i) {
        const int j = A == 1 ? 0 : i0 + i;
        xh[i] = (x[i] - k.mean[j]) * k.rstd[j];
        z[i] = __builtin_fmaf(xh[i], k.gamma[i0 + i], k.beta[i0 + i]);
    }
    if (act == SCNN_ACT_RELU) {
        bool near = false;
#pragma unroll
        for (int i = 0; i < N; ++i)
            near |= __builtin_fabsf(z[i]) <= 0x1p-21f * (__builtin_fabsf(xh[i] * k.gamma[i0 + i]) + __builtin_fabsf(k.beta[i0 + i]));
        if (near)
#pragma unroll
            for (int i = 0; i < N; ++i) {
                float m = k.mean[A == 1 ? 0 : i0 + i], r = k.rstd[A == 1 ? 0 : i0 + i], c = k.gamma[i0 + i], o = k.beta[i0 + i];
                asm volatile("" : "+v"(m), "+v"(r), "+v"(c), "+v"(o));  // (else all columns' values are held in fp64 besides)
                const double far = __builtin_fma(((double)x[i] - (double)m) * (double)r, (double)c, (double)o);
                z[i] = far <= 0.0 ? 0.0f : 1.0f;  // (a NaN's slope is 1, as with activate_back)
            }
    }
    activate_back_all<N>(g, z, act, dz);
}
template <int V>
struct BackSums { float a[V], b[V]; };  // of dz xh and dz
template <int V, int A, int N>
__device__ __forceinline__ void back_add(const BackColumns<V, A>& k, int i0, const float (&x)[N], const float (&g)[N], int act, BackSums<V>& v,
                                         float (&dz)[N]) {
    float xh[N];
    back_values<V, A, N>(k, i0, x, g, act, xh, dz);
#pragma unroll
    for (int i = 0; i < N; ++i) {
        v.a[i0 + i] = __builtin_fmaf(dz[i], xh[i], v.a[i0 + i]);
        v.b[i0 + i] += dz[i];
    }
}
template <typename T>
__device__ __forceinline__ void apart(VecOf<T, kVec<T>> r, float (&v)[kVec<T>]) {
#pragma unroll
    for (int i = 0; i < kVec<T>; ++i) v[i] = (float)r[i];
}

// A thread's sums are fp32 over runs of kRun of its vectors and fp64 over the runs: what a sum is off by does not grow with the rows.
// (16384 additions of 0.1 behind each other in fp32 are off by 1.5e-4 of their sum, and a gradient of equal values, whose dx is 0, has as
// much in every dx.)
constexpr int kRun = 32;

// Sums over a thread's vectors from number k on, of which the first U are there; U divides k and kRun.
template <typename T, int A, int U>
__device__ __forceinline__ void back_sum_from(const GroupArgs& p, const BackColumns<kVec<T>, A>& c, const Walk& w, int k,
                                              VecOf<T, kVec<T>> (&r)[U], VecOf<T, kVec<T>> (&q)[U], BackSums<kVec<T>>& v) {
    constexpr int V = kVec<T>;
    const T *__restrict__ x = (const T*)p.x, *__restrict__ g = (const T*)p.g;
    double a[V] = {}, b[V] = {};
    walk<U>(w, k, w.full,
            [&](int u, int n) {
                float xs[V], gs[V], dz[V];
                apart<T>(r[u], xs);
                apart<T>(q[u], gs);
                back_add<V, A, V>(c, 0, xs, gs, p.act, v, dz);
                if (u == U - 1 && (n & (kRun - 1)) == kRun - 1)
#pragma unroll
                    for (int i = 0; i < V; ++i) {
                        a[i] += (double)v.a[i];
                        b[i] += (double)v.b[i];
                        v.a[i] = v.b[i] = 0.0f;
                    }
            },
            [&](int u, int n) {
                r[u] = take(x + position<false>(w, n));
                q[u] = take(g + position<false>(w, n));
            });
    if (w.full >= kRun)
#pragma unroll
        for (int i = 0; i < V; ++i) {
            v.a[i] = (float)(a[i] + (double)v.a[i]);
            v.b[i] = (float)(b[i] + (double)v.b[i]);
        }
}
// And over its odd values.
template <typename T, int A>
__device__ __forceinline__ void back_sum_odd(const GroupArgs& p, const BackColumns<kVec<T>, A>& c, const Walk& w, BackSums<kVec<T>>& v) {
    constexpr int V = kVec<T>;
    if (w.n) {
        const long long at = w.at + (long long)w.full * w.step;
#pragma unroll
        for (int i = 0; i < V - 1; ++i)
            if (i < w.n) {
                const float xs[1] = {(float)((const T*)p.x)[at + i]}, gs[1] = {(float)((const T*)p.g)[at + i]};
                float dz[1];
                back_add<V, A, 1>(c, i, xs, gs, p.act, v, dz);
            }
    }
}

// Sums over a step's rows, given to s_col [2][wide].  All threads call it and meet at its end; s_all: a step's numbers, as in add_groups.
// (Rows one behind the other put all lanes of a sum in one bank: 64 samples of 512 x 256 bf16 took 36.9 us, so 26.6 at the time.)
template <int V>
__device__ __forceinline__ void add_columns(const GroupArgs& p, const Slab& a, const Place& t, const BackSums<V>& v, float2* s_all, float* s_col) {
    const int wide = a.c1 - a.c0;
    if ((int)threadIdx.x < p.l.active)
#pragma unroll
        for (int i = 0; i < V; ++i)
            if (i >= t.other) s_all[(i - t.other) * (p.l.active + 1) + threadIdx.x] = make_float2(v.a[i], v.b[i]);
    __syncthreads();
    const int bits = lane_bits(p.l.reps, wide), q = 1 << bits, sets = blockDim.x >> bits, in = threadIdx.x & (q - 1);
    for (int c0 = 0; c0 < wide; c0 += sets) {
        const int c = c0 + (threadIdx.x >> bits);
        float2 sum = make_float2(0.0f, 0.0f);
        if (c < wide)
            for (int k = in; k < p.l.reps; k += q) {
                const float2 o = s_all[step_at(p, V == 8 ? 3 : 2, 0, k, c)];
                sum.x += o.x;
                sum.y += o.y;
            }
        for (int d = 1; d < q; d <<= 1) {
            sum.x += __shfl_xor(sum.x, d, 64);
            sum.y += __shfl_xor(sum.y, d, 64);
        }
        if (c < wide && in == 0) {
            s_col[c] = sum.x;
            s_col[wide + c] = sum.y;
        }
    }
    __syncthreads();
}

// Sums of h and h xh over the slab's groups from the columns' sums of dz xh and dz: done(group, {sum h, sum h xh}) by one lane a group.
template <typename T, typename F>
__device__ __forceinline__ void back_groups(const GroupArgs& p, const Slab& a, const float* s_col, F done) {
    const T* __restrict__ gamma = p.gamma ? (const T*)p.gamma + a.c0 : nullptr;
    const int wide = a.c1 - a.c0, bits = lane_bits(a.w, a.ng), q = 1 << bits, set = threadIdx.x >> bits, sets = blockDim.x >> bits,
              in = threadIdx.x & (q - 1);
    for (int j0 = 0; j0 < a.ng; j0 += sets) {
        const int j = j0 + set;
        Two sum = {0.0, 0.0};
        if (j < a.ng)
            for (int e = in; e < a.w; e += q) {
                const int c = j * a.w + e;
                const double by = gamma ? (double)(float)gamma[c] : 1.0;
                sum.a += by * (double)s_col[wide + c];
                sum.b += by * (double)s_col[c];
            }
        sum = lanes_two(sum, q);
        if (in == 0 && j < a.ng) done(j, sum);
    }
}

template <int A>
struct Means { float h[A], hx[A]; };
template <typename T, bool M>
__device__ __forceinline__ Means<M ? 1 : kVec<T>> means_of(const GroupArgs& p, const Slab& a, const Place& t, const float2* stat) {
    constexpr int A = M ? 1 : kVec<T>;
    Means<A> m;
#pragma unroll
    for (int i = 0; i < A; ++i) {
        const float2 s = stat[group_of(p, column_of(p, a, t, i))];
        m.h[i] = s.x;
        m.hx[i] = s.y;
    }
    return m;
}
template <int V, int A>
__device__ __forceinline__ float back_result(const BackColumns<V, A>& k, const Means<A>& m, int i, float xh, float dz) {
    const int j = A == 1 ? 0 : i;
    return k.rstd[j] * (dz * k.gamma[i] - m.h[j] - xh * m.hx[j]);
}
// A thread's vectors from its last down to number `from`, of which the first U are there, and its odd values.
template <typename T, int A, int U>
__device__ __forceinline__ void back_down(const GroupArgs& p, const BackColumns<kVec<T>, A>& c, const Means<A>& m, const Walk& w, int from,
                                          VecOf<T, kVec<T>> (&r)[U], VecOf<T, kVec<T>> (&q)[U]) {
    constexpr int V = kVec<T>;
    const T *__restrict__ x = (const T*)p.x, *__restrict__ g = (const T*)p.g;
    walk<U>(w, 0, w.full - from,
            [&](int u, int n) {
                VecOf<T, V> y;
                float xs[V], gs[V], xh[V], dz[V];
                apart<T>(r[u], xs);
                apart<T>(q[u], gs);
                back_values<V, A, V>(c, 0, xs, gs, p.act, xh, dz);
#pragma unroll
                for (int i = 0; i < V; ++i) y[i] = (T)back_result<V, A>(c, m, i, xh[i], dz[i]);
                put((T*)p.out + position<true>(w, n), y, A == 1 ? 0 : w.other);
            },
            [&](int u, int n) {
                r[u] = take(x + position<true>(w, n));
                q[u] = take(g + position<true>(w, n));
            });
    if (w.n) {
        const long long at = w.at + (long long)w.full * w.step;
#pragma unroll
        for (int i = 0; i < V - 1; ++i)
            if (i < w.n) {
                const float xs[1] = {(float)x[at + i]}, gs[1] = {(float)g[at + i]};
                float xh[1], dz[1];
                back_values<V, A, 1>(c, i, xs, gs, p.act, xh, dz);
                ((T*)p.out)[at + i] = (T)back_result<V, A>(c, m, i, xh[0], dz[0]);
            }
    }
}

constexpr int kBackAhead = 2;  // vectors of x and of g

// LDS: a step's numbers, then the columns' sums.
__host__ __device__ __forceinline__ int step_values(const GroupLayout& l, int v) { return v * (l.active + 1); }

// Sums of a block's rows, of columns first: dgamma and dbeta want these, and those of a group's h and h xh follow from them by gamma.
// 209645 x 25 fp32 in 5 groups, relu: 15 us, 2.9 TB/s of x and g: eleven steps a workgroup with a start and an end around them.
template <typename T, bool M, bool OVER>
__device__ __forceinline__ void block_back_sums(const GroupArgs& p, long long i, int slab, char* s_step) {
    constexpr int V = kVec<T>, A = M ? 1 : V, U = kBackAhead;
    float2* const s_all = (float2*)s_step;
    float* const s_col = (float*)(s_all + step_values(p.l, V));
    if (i >= p.blocks) return;
    const Bounds s = bounds_of(p);
    const Slab a = slab_of(p, slab);
    const Place t = place_of<V>(p, a);
    const Affine<T> f = affine_of<T>(p, a, t);
    const Block k = block_of<OVER>(p, s, i);
    const int wide = a.c1 - a.c0, to = p.l.pieces > 1 ? slab : a.j0;
    bool first = true;
    for (long long b = k.b0; b <= k.b1; b = next_sample<OVER>(k, b)) {
        const Rows r = rows_of_sample(s, b);
        if (OVER && r.end - r.first <= p.over) continue;
        const long long lo = r.first > k.r0 ? r.first : k.r0, hi = r.end < k.r1 ? r.end : k.r1;
        float* const cols = p.cols + (OVER ? i : i + b) * 2 * p.channels + a.c0;
        float2* const part = (float2*)p.part + (i + b) * p.groups * p.l.pieces + to;
        if (hi <= lo) {
            if (OVER) continue;
            if (p.cols)
                for (int c = threadIdx.x; c < wide; c += blockDim.x) cols[c] = cols[p.channels + c] = 0.0f;
            for (int j = threadIdx.x; j < a.ng; j += blockDim.x) part[j] = make_float2(0.0f, 0.0f);
            continue;
        }
        const Walk w = walk_of<V>(p, a, t, lo, hi);
        VecOf<T, V> x[U], g[U];
        fetch<T, U, false>((const T*)p.x, w, 0, x);
        fetch<T, U, false>((const T*)p.g, w, 0, g);
        BackSums<V> v = {};
        const BackColumns<V, A> c = back_columns<T, M>(p, a, t, f, b);
        back_sum_from<T, A, U>(p, c, w, 0, x, g, v);
        back_sum_odd<T, A>(p, c, w, v);
        add_columns<V>(p, a, t, v, s_all, s_col);
        if (p.cols)
            for (int c = threadIdx.x; c < wide; c += blockDim.x) {
                cols[c] = OVER && !first ? cols[c] + s_col[c] : s_col[c];
                cols[p.channels + c] = OVER && !first ? cols[p.channels + c] + s_col[wide + c] : s_col[wide + c];
            }
        first = false;
        if (p.out) back_groups<T>(p, a, s_col, [&](int j, Two sum) { part[j] = make_float2((float)sum.a, (float)sum.b); });
        if (b < k.b1) __syncthreads();
    }
    if (OVER && p.cols && first)
        for (int c = threadIdx.x; c < wide; c += blockDim.x) p.cols[i * 2 * p.channels + a.c0 + c] = p.cols[(i * 2 + 1) * p.channels + a.c0 + c] = 0.0f;
}
template <typename T, bool M>
__global__ __launch_bounds__(kGroupThreads, 2) void k_group_back_sums(GroupArgs p) {
    extern __shared__ __align__(16) char s_step[];
    block_back_sums<T, M, false>(p, block_id<kGroupThreads>(), blockIdx.y, s_step);
}

// 4 N columns of the places' sums of dz xh and dz by one workgroup, four neighbours a thread.
template <typename T, int N>
__device__ __forceinline__ void back_columns_sum(const GroupArgs& p, long long at, double* s_sum) {
    constexpr int U = 4;
    const int cn = threadIdx.x & (N - 1), threads = blockDim.x / N;
    const long long cols = 2LL * p.channels, c = (at * N + cn) * 4;
    const int n = (int)(cols - c < 4 ? cols - c : 4);
    double sum[4] = {0.0, 0.0, 0.0, 0.0};
    if (n > 0)
        for (long long i = threadIdx.x / N; i < p.places; i += U * threads) {
            float v[U][4];
#pragma unroll
            for (int u = 0; u < U; ++u) {
                const float* from = p.cols + (i + u * threads < p.places ? i + u * threads : p.places - 1) * cols + c;
#pragma unroll
                for (int k = 0; k < 4; ++k) v[u][k] = from[k < n ? k : 0];
            }
#pragma unroll
            for (int u = 0; u < U; ++u)
                if (i + u * threads < p.places)
#pragma unroll
                    for (int k = 0; k < 4; ++k) sum[k] += (double)v[u][k];
        }
#pragma unroll
    for (int k = 0; k < 4; ++k) {
#pragma unroll
        for (int d = N; d < 64; d <<= 1) sum[k] += __shfl_xor(sum[k], d, 64);
        if ((threadIdx.x & 63) < N) s_sum[((threadIdx.x >> 6) * N + cn) * 4 + k] = sum[k];
    }
    __syncthreads();
    if (threadIdx.x >= N * 4) return;
    const long long out = at * N * 4 + threadIdx.x;
    if (out >= cols) return;
    double all = 0.0;
    for (int w = 0; w < (int)blockDim.x / 64; ++w) all += s_sum[w * N * 4 + threadIdx.x];
    T* const to = (T*)(out < p.channels ? p.dgamma : p.dbeta);
    if (to) to[out < p.channels ? out : out - p.channels] = (T)(float)all;
}

// Columns of a workgroup that adds them: 64 bytes of a place, or 16 where these are many.
template <bool OVER> constexpr int kSumColumns = OVER ? 4 : 16;

// Gradients of a block's rows; workgroups past the blocks add the columns' sums.  209645 x 25 fp32 in 5 groups, relu: 15 us, 4.3 TB/s.
template <typename T, bool M, bool OVER>
__global__ __launch_bounds__(kGroupThreads, 2) void k_group_back(GroupArgs p) {
    constexpr int V = kVec<T>, A = M ? 1 : V, U = kBackAhead;
    __shared__ Two s_two[kGroupThreads];
    __shared__ float2 s_stat[kHereGroups];
    const long long i = block_id<kGroupThreads>();
    if (i >= p.blocks) {
        if (blockIdx.y == 0 && i - p.blocks < p.sum_blocks) back_columns_sum<T, kSumColumns<OVER> / 4>(p, i - p.blocks, (double*)s_two);
        return;
    }
    const Bounds s = bounds_of(p);
    const Block k = block_of<OVER>(p, s, i);
    if (OVER && !any_over(p, s, k)) return;
    const Slab a = slab_of(p, blockIdx.y);
    const Place t = place_of<V>(p, a);
    const Affine<T> f = affine_of<T>(p, a, t);
    const Joiner o = joiner_of(a);
    for (long long b = k.b0; b <= k.b1; b = next_sample<OVER>(k, b)) {
        const Rows r = rows_of_sample(s, b);
        if (OVER && r.end - r.first <= p.over) continue;
        const long long lo = r.first > k.r0 ? r.first : k.r0, hi = r.end < k.r1 ? r.end : k.r1;
        if (hi <= lo) continue;
        const Walk w = walk_of<V>(p, a, t, lo, hi);
        VecOf<T, V> x[U], g[U];
        fetch<T, U, true>((const T*)p.x, w, 0, x);
        fetch<T, U, true>((const T*)p.g, w, 0, g);
        const BackColumns<V, A> c = back_columns<T, M>(p, a, t, f, b);
        const float2* stat = (const float2*)p.stat + b * p.groups + a.j0;
        if (!p.stat) {
            const Two sum = join_here<float>(p, a, o, b, r, s_two);
            if (o.k < a.ng && o.in == 0) {
                const double inv = 1.0 / ((double)(r.end - r.first) * p.per);
                s_stat[o.k] = make_float2((float)(sum.a * inv), (float)(sum.b * inv));
            }
            __syncthreads();
            stat = s_stat;
        }
        back_down<T, A, U>(p, c, means_of<T, M>(p, a, t, stat), w, 0, x, g);
    }
}

// Backward by a workgroup a sample and slab, x, g and dz in registers.  cols [batch][2][channels]; with one sample dgamma and dbeta
// themselves.  64 samples of 512 x 256 bf16 in 32 groups, silu: 15 us, 3.4 TB/s, bound by the instructions of silu and its slope and by
// what a workgroup does between its loads and its stores; k_column_sums behind it 4 us.
template <typename T, bool M, int H, bool OVER>
__device__ __forceinline__ void one_back(const GroupArgs& p, long long b, char* s_step) {
    constexpr int V = kVec<T>, A = M ? 1 : V;
    float2* const s_all = (float2*)s_step;
    float* const s_col = (float*)(s_all + step_values(p.l, V));
    float2* const s_stat = s_all;  // (when the columns' sums are done)
    if (b >= p.batch) return;
    const Bounds s = {p.offsets, p.each, p.rows, p.batch, 0, p.inv_each, false};
    const Slab a = slab_of(p, blockIdx.y);
    const Place t = place_of<V>(p, a);
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
    if (r.end == r.first || (OVER && r.end - r.first > p.over)) {
        for (int c = threadIdx.x; c < wide; c += blockDim.x) give(c, 0.0f, 0.0f);
        return;
    }
    const T *__restrict__ x = (const T*)p.x, *__restrict__ g = (const T*)p.g;
    const Walk w = walk_of<V>(p, a, t, r.first, r.end);
    VecOf<T, V> held[H], grad[H];
    const Affine<T> f = affine_of<T>(p, a, t);
    const BackColumns<V, A> k = back_columns<T, M>(p, a, t, f, b);
    BackSums<V> v = {};
    VecOf<T, V> more[2], more_g[2];
    if (w.full > H) {  // (what is read again comes first: its sums in fp64 and the held values would not both fit the registers)
        fetch<T, 2, false>(x, w, H, more);
        fetch<T, 2, false>(g, w, H, more_g);
        back_sum_from<T, A, 2>(p, k, w, H, more, more_g, v);
    }
    fetch<T, H, false>(x, w, 0, held);
    fetch<T, H, false>(g, w, 0, grad);
    float dz[H][V];
#pragma unroll
    for (int h = 0; h < H; ++h)
        if (h < w.full) {
            float xs[V], gs[V];
            apart<T>(held[h], xs);
            apart<T>(grad[h], gs);
            back_add<V, A, V>(k, 0, xs, gs, p.act, v, dz[h]);
            __builtin_amdgcn_sched_barrier(0);
        }
    back_sum_odd<T, A>(p, k, w, v);
    add_columns<V>(p, a, t, v, s_all, s_col);
    for (int c = threadIdx.x; c < wide; c += blockDim.x) give(c, s_col[c], s_col[wide + c]);
    if (!p.out) return;
    const double inv = 1.0 / ((double)(r.end - r.first) * p.per);
    back_groups<T>(p, a, s_col, [&](int j, Two sum) { s_stat[j] = make_float2((float)(sum.a * inv), (float)(sum.b * inv)); });
    __syncthreads();
    const Means<A> m = means_of<T, M>(p, a, t, s_stat);
#pragma unroll
    for (int h = 0; h < H; ++h)
        if (h < w.full) {
            VecOf<T, V> y;
#pragma unroll
            for (int i = 0; i < V; ++i) {
                const int j = A == 1 ? 0 : i;
                y[i] = (T)back_result<V, A>(k, m, i, ((float)held[h][i] - k.mean[j]) * k.rstd[j], dz[h][i]);
            }
            put((T*)p.out + w.at + h * w.step, y, A == 1 ? 0 : w.other);
            __builtin_amdgcn_sched_barrier(0);
        }
    if (w.full > H) {
        fetch<T, 2, true>(x, w, 0, more);
        fetch<T, 2, true>(g, w, 0, more_g);
    }
    back_down<T, A, 2>(p, k, m, w, H, more, more_g);
}
template <typename T, bool M, int B, int H>
__global__ __launch_bounds__(B, 2) void k_group_back_one(GroupArgs p) {
    extern __shared__ __align__(16) char s_step[];
    one_back<T, M, H, false>(p, block_id<B>(), s_step);
}
// As k_group_one_sums.
template <typename T, bool M, int B, int H>
__global__ __launch_bounds__(B, 2) void k_group_back_one_sums(GroupArgs p, GroupArgs blocks) {
    extern __shared__ __align__(16) char s_step[];
    const long long id = block_id<B>(), at = number_behind(p, id);
    if (at < 0) one_back<T, M, H, true>(p, id, s_step);
    else if (at < blocks.blocks * blocks.l.slabs) block_back_sums<T, M, true>(blocks, (unsigned)at / blocks.l.slabs, (unsigned)at % blocks.l.slabs, s_step);
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
    const int period = channels / even;  // vectors after which a run of rows meets the same columns
    // Values of a step: of rows that run on, and of rows that each begin with a vector (loads at any address, a cut vector a row).  The
    // first where they are as many, or nearly.  us of the first / second, bf16, relu: backward 60000 x 516 112 / 88, 100000 x 260
    // 78 / 70, 100000 x 165 66 / 55; fp32: 100000 x 258 116 / 96 (all some 10 per cent shorter since).
    const int row = (channels + v - 1) / v, runs = threads / period * period * v, rows = (row >= threads ? 1 : threads / row) * channels;
    if (even < v && period <= threads && channels <= most && 8LL * runs >= 7LL * rows) {
        l.flat = 1;
        l.active = threads / period * period;
        l.reps = (int)((long long)l.active * v / channels);
        l.tv = l.active;
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
        l.merged = per % v == 0;
        while (1 << l.sub < v && per % (2 << l.sub) == 0) ++l.sub;
    }
    l.inv_tv = 1.0f / (float)l.tv;
    l.inv_per = l.pieces > 1 ? 0.0f : 1.0f / (float)per;
    l.inv_c = l.flat ? 1.0f / (float)channels : 0.0f;
    l.inv_reps = 1.0 / (double)l.reps;
    return l;
}
static unsigned group_threads(const GroupLayout& l) { return (unsigned)((l.active + 63) / 64 * 64); }
// Bytes of LDS: pairs in fp64 for `sub` neighbours (and a group's statistics), pairs in fp32 and the columns' sums.
static unsigned sums_lds(const GroupLayout& l, int v) { return (unsigned)((l.merged ? 1 : v >> l.sub) * (l.active + 1) * 16); }
static unsigned one_lds(const GroupLayout& l, int v, int per) { return sums_lds(l, v) + (unsigned)(l.wide / per) * 16; }
static unsigned back_lds(const GroupLayout& l, int v) { return (unsigned)(step_values(l, v) + l.wide) * 8; }

// Rows of a block: two workgroups of 256 threads a compute unit (what a workgroup does before and after its rows costs all its waves
// as much as some vectors each), but no fewer than two vectors a thread; one where that makes no more than a workgroup a unit.
static long long group_chunk(const GroupLayout& l, long long rows) {
    if ((rows + l.reps - 1) / l.reps * l.slabs <= device_cu_count()) return l.reps;
    long long want = 2LL * device_cu_count() / l.slabs;
    if (want < 1) want = 1;
    long long chunk = (rows + want - 1) / want;
    if (chunk < 2LL * l.reps) chunk = 2LL * l.reps;
    return round_up(chunk, l.reps);
}

// A workgroup a sample and slab, its values in registers: 16384 of them, in 256 threads, or in 512 where workgroups are few; samples of
// up to twice that on the average.  Only the device knows how unequal samples are that offsets name, and a workgroup takes 0.3 us a
// thousand values: they are up to half of it in calls of more than 2^24 values, and these up to 2^28 (and see kOneMost).
// us of this / of blocks of rows, in a graph, at the time: backward 64 samples of 512 x 256 bf16 20 / 39, forward 512 x 24 fp32 7.5 / 14;
// forward and backward 4096 samples of about 128 x 64 bf16 39 / 105 and 87 / 141, of 16 x 512 fp32 49 / 107 and 105 / 187; 1024 equal
// ones of 512 x 64 fp32 52 / 80 and 88 / 124.
constexpr int kOneFew = 512, kOneMany = 256;
constexpr long long kOneHeld = 16384, kOneAny = 1LL << 24, kOneAll = 1LL << 28;
static bool group_one(long long rows, long long batch, int channels, int per, int dtype, bool equal, GroupLayout& l, int& threads) {
    const int v = group_vec(dtype), least = 64 / (16 / v);  // (64 bytes of a row)
    const long long values = rows * channels / batch, cus = device_cu_count();
    int most = kOneMany * v / 2;
    if (per > most) return false;
    if (per % v == 0) {
        // narrower slabs where a sample has more values than that, or compute units would idle
        long long want = (values + kOneHeld - 1) / kOneHeld;
        if (want * batch < cus && values > 4096) want = cus / batch;
        if (want > 1) {
            long long wide = (channels + want - 1) / want;
            if (wide < least) wide = least;
            wide = (wide + per - 1) / per * per;
            if (wide < most) most = (int)wide;
        }
    }
    const long long held = rows * (channels < most ? channels : most);
    if (held > 2 * kOneHeld * batch) return false;
    if (!equal && rows * channels > kOneAny && (rows * channels > kOneAll || 2 * held > kOneHeld * batch)) return false;
    threads = kOneFew;
    l = group_layout(channels, per, dtype, threads, most);
    if (batch * l.slabs >= cus || one_lds(l, v, per) > 60000) {
        threads = kOneMany;
        l = group_layout(channels, per, dtype, threads, most);
    }
    return l.pieces == 1 && l.slabs <= 65535;  // (a launch's second axis)
}

// With offsets, samples above `over` rows are left to the blocks: their sums are added beside the others' work, and one more launch ends at
// once where there are none.  A workgroup keeps up to kOneMost values, 20 us of it, or as many as a block's rows; calls of up to twice as many
// are not divided.  us in a graph of one sample with all rows (a workgroup for it) / of equal ones (undivided): 64 samples in 131072 x 16
// fp32 forward 16 (442) / 15 (12.7), backward 22 (679) / 23 (19.9); 512 in 262144 x 64 bf16 29 (2770) / 23 (19.7) and 42 (3630) / 44 (39.6);
// 32768 in 4194304 x 64 bf16 348 (85700) / 263 (230) and 652 (136600) / 615 (584).
constexpr long long kOneMost = 65536;

struct GroupSpace {
    GroupLayout one_l, l;  // of a workgroup a sample, of blocks
    long long blocks, chunk, places, over;
    size_t part, stat, total;  // (the columns' sums, where there are some, come first)
    bool one, joined;
    int threads;
    bool any_blocks() const { return !one || over; }
};
static GroupSpace group_space(long long rows, long long batch, int channels, int groups, int dtype, bool equal, bool back) {
    GroupSpace s = {};
    const int per = channels / groups;
    s.one = group_one(rows, batch, channels, per, dtype, equal, s.one_l, s.threads);
    const bool divided = s.one && !equal && rows * s.one_l.wide > 2 * kOneMost;
    if (s.one && !divided) {
        if (back && batch > 1) s.total = (size_t)round_up(batch * channels * 8, 256);
        return s;
    }
    s.l = group_layout(channels, per, dtype, kGroupThreads, kGroupThreads * group_vec(dtype));
    s.chunk = group_chunk(s.l, rows);
    s.blocks = rows < 1 ? 1 : (rows + s.chunk - 1) / s.chunk;
    s.places = s.blocks + batch - 1;
    if (divided) s.over = s.chunk > kOneMost / s.one_l.wide ? s.chunk : kOneMost / s.one_l.wide;
    const int ng = s.l.wide / per;  // (of a slab)
    s.joined = s.l.pieces > 1 || ng > kHereGroups || (!divided && (s.blocks / batch + 1) * ng > 2048);
    // (divided, the columns' sums of samples and of blocks lie behind each other)
    if (back) s.part = (size_t)round_up((divided ? batch + s.blocks : s.places) * channels * 8LL, 256);
    s.stat = s.part + (size_t)round_up(s.places * groups * s.l.pieces * (back ? 8LL : 16LL), 256);
    s.total = s.stat + (s.joined ? (size_t)round_up(batch * groups * (back ? 8LL : 16LL), 256) : 0);
    return s;
}

size_t group_norm_bytes(int dtype, long long rows, long long batch, int channels, int groups, bool back) {
    const size_t equal = group_space(rows, batch, channels, groups, dtype, true, back).total;
    const size_t any = group_space(rows, batch, channels, groups, dtype, false, back).total;
    return equal > any ? equal : any;
}

// Arguments of the workgroups that take a sample each, and of the blocks'.
struct GroupBoth { GroupArgs one, blocks; };
static GroupBoth group_args(const GroupCall& c, bool back, const GroupSpace& s) {
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
    p.over = s.over;
    p.inv_each = p.each > 0 ? 1.0 / (double)p.each : 0.0;
    if (c.dgamma || c.dbeta) p.cols = (float*)c.workspace;
    GroupBoth a = {p, p};
    a.one.l = s.one_l;
    if (!s.any_blocks()) return a;
    a.blocks.l = s.l;
    a.blocks.chunk = s.chunk; a.blocks.blocks = s.blocks; a.blocks.places = s.places;
    a.blocks.inv_chunk = 1.0 / (double)s.chunk;
    a.blocks.part = (char*)c.workspace + s.part;
    if (p.cols && s.over) a.blocks.cols = p.cols + c.batch * 2 * c.channels;
    if (s.joined) a.blocks.stat = (char*)c.workspace + s.stat;
    return a;
}

// A launch that joins the places' sums, about as many threads for a sample's group as it has places.
template <typename T, bool BACK>
static void group_join(const GroupArgs& p, hipStream_t s) {
    const long long n = (p.blocks / p.batch + 1) * p.l.pieces;
    int q = 1;
    while (q < 256 && q < n) q <<= 1;
    hipLaunchKernelGGL((k_group_join<T, BACK>), grid_of<256>((p.batch * p.groups + 256 / q - 1) / (256 / q)), dim3(256), 0, s, p, q);
}

// The first launch where a workgroup takes a sample: alone, or with the blocks' sums of longer ones behind it (in rows of the grid, which are
// started last, where there are several already: 64 samples in 19200 x 64 fp32 backward 13.3 us, in columns 15.2).
template <typename F>
static void one_launch(const GroupBoth& p, const GroupSpace& at, unsigned one, unsigned sums, F launch) {
    const unsigned t1 = group_threads(p.one.l);
    const long long batch = p.one.batch;
    const int y = p.one.l.slabs;
    if (!at.over) return launch(batch, y, dim3(t1), one);
    const unsigned t2 = group_threads(p.blocks.l);
    const long long more = at.blocks * p.blocks.l.slabs, rows = (more + batch - 1) / batch;
    const bool below = y > 1 && y + rows <= 65535 && batch <= 1 << 20;
    launch(batch + (below ? 0 : (more + y - 1) / y), below ? y + (int)rows : y, dim3(t1 > t2 ? t1 : t2), sums > one ? sums : one);
}
template <typename T, bool M, int B, int H>
static void one_fwd(const GroupBoth& p, const GroupSpace& at, hipStream_t s) {
    constexpr int V = kVec<T>;
    one_launch(p, at, one_lds(p.one.l, V, p.one.per), at.over ? sums_lds(p.blocks.l, V) : 0, [&](long long n, int y, dim3 threads, unsigned lds) {
        if (at.over) hipLaunchKernelGGL((k_group_one_sums<T, M, B, H>), grid_of<B>(n, y), threads, lds, s, p.one, p.blocks);
        else hipLaunchKernelGGL((k_group_one<T, M, B, H>), grid_of<B>(n, y), threads, lds, s, p.one);
    });
}
template <typename T, bool M, int B, int H>
static void one_bwd(const GroupBoth& p, const GroupSpace& at, hipStream_t s) {
    constexpr int V = kVec<T>;
    one_launch(p, at, back_lds(p.one.l, V), at.over ? back_lds(p.blocks.l, V) : 0, [&](long long n, int y, dim3 threads, unsigned lds) {
        if (at.over) hipLaunchKernelGGL((k_group_back_one_sums<T, M, B, H>), grid_of<B>(n, y), threads, lds, s, p.one, p.blocks);
        else hipLaunchKernelGGL((k_group_back_one<T, M, B, H>), grid_of<B>(n, y), threads, lds, s, p.one);
    });
}

template <typename T, bool M>
static hipError_t group_fwd(const GroupBoth& p, const GroupSpace& at, hipStream_t s) {
    constexpr int V = kVec<T>;
    if (at.one) {
        if (at.threads == kOneFew) one_fwd<T, M, kOneFew, 32 / V>(p, at, s);
        else one_fwd<T, M, kOneMany, 64 / V>(p, at, s);
        if (!at.over) return hipGetLastError();
    }
    const GroupArgs& b = p.blocks;
    const dim3 threads(group_threads(b.l)), grid = grid_of<kGroupThreads>(b.blocks, b.l.slabs);
    if (!at.one) hipLaunchKernelGGL((k_group_sums<T, M>), grid, threads, sums_lds(b.l, V), s, b);
    if (b.stat) group_join<T, false>(b, s);
    if (at.over) hipLaunchKernelGGL((k_group_apply<T, M, true>), grid, threads, 0, s, b);
    else hipLaunchKernelGGL((k_group_apply<T, M, false>), grid, threads, 0, s, b);
    return hipGetLastError();
}

template <typename T, bool M>
static hipError_t group_bwd(int dtype, const GroupBoth& p, const GroupSpace& at, hipStream_t s) {
    constexpr int V = kVec<T>;
    GroupArgs b = p.blocks;
    if (at.one) {
        if (at.threads == kOneFew) one_bwd<T, M, kOneFew, 32 / V>(p, at, s);
        else one_bwd<T, M, kOneMany, 64 / V>(p, at, s);
    } else {
        hipLaunchKernelGGL((k_group_back_sums<T, M>), grid_of<kGroupThreads>(b.blocks, b.l.slabs), dim3(group_threads(b.l)), back_lds(b.l, V), s, b);
    }
    // the columns' sums, of samples and blocks behind each other where both took some
    const long long parts = at.one ? b.batch + (at.over ? b.blocks : 0) : b.places;
    b.cols = p.one.cols;
    if (b.out && (!at.one || at.over)) {
        if (b.stat) group_join<T, true>(b, s);
        b.places = parts;
        const int wide = at.over ? kSumColumns<true> : kSumColumns<false>;
        const bool here = b.cols && (!at.over || parts <= 1024);  // (4608 places of 128: 17 us here, so 8 in a launch of their own)
        b.sum_blocks = here ? (2LL * b.channels + wide - 1) / wide : 0;
        const dim3 grid = grid_of<kGroupThreads>(b.blocks + b.sum_blocks, b.l.slabs), threads(group_threads(b.l));
        if (at.over) hipLaunchKernelGGL((k_group_back<T, M, true>), grid, threads, 0, s, b);
        else hipLaunchKernelGGL((k_group_back<T, M, false>), grid, threads, 0, s, b);
        if (here || !b.cols) return hipGetLastError();
    }
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess || !b.cols || (at.one && b.batch == 1)) return e;
    return launch_column_sums(b.cols, (int)parts, 2LL * b.channels, b.channels, b.dgamma, b.dbeta, dtype, s);
}

template <typename T>
static hipError_t group_norm(int dtype, const GroupCall& c, bool back, hipStream_t s) {
    const GroupSpace at = group_space(c.rows, c.batch, c.channels, c.groups, dtype, c.offsets == nullptr, back);
    const GroupBoth p = group_args(c, back, at);
    const bool merged = at.one ? p.one.l.merged : p.blocks.l.merged;  // (of both the same: whether a group is whole vectors)
    if (back) return merged ? group_bwd<T, true>(dtype, p, at, s) : group_bwd<T, false>(dtype, p, at, s);
    return merged ? group_fwd<T, true>(p, at, s) : group_fwd<T, false>(p, at, s);
}
static hipError_t group_norm(int dtype, const GroupCall& c, bool back, hipStream_t s) {
    switch (dtype) {
        case SCNN_F32: return group_norm<float>(dtype, c, back, s);
        case SCNN_BF16: return group_norm<__bf16>(dtype, c, back, s);
        default: return group_norm<_Float16>(dtype, c, back, s);
    }
}
hipError_t launch_group_fwd(int dtype, const GroupCall& c, hipStream_t s) { return group_norm(dtype, c, false, s); }
hipError_t launch_group_bwd(int dtype, const GroupCall& c, hipStream_t s) { return group_norm(dtype, c, true, s); }

hipError_t launch_sample_offsets(const int* coords, int stride, long long rows, const long long* rows_dev, long long batch,
                                 long long* offsets, hipStream_t s) {
    hipLaunchKernelGGL(k_sample_offsets, grid_of<256>((batch + 4) / 4), dim3(256), 0, s, coords, stride, rows, rows_dev, batch, offsets);
    return hipGetLastError();
}

}  // namespace scnn
