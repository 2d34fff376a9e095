// Log probabilities of class labels, their entropy and best classes, the gradient, and the loss made of them (ftp_logprob,
// ftp_logprob_backward, ftp_loss_logprob).
//
// Logits are read once: a row stays in the registers of a warp (short rows), of a block, or of a cluster of up to 16 blocks that
// exchange their parts through distributed shared memory.  With the row's maximum m the sums are s = sum 2^a and t = sum a 2^a,
// a = (z - m) log2 e, and lse = m + log s, entropy = log s - (t / s) log 2.
//
// The best classes come without sorting: a row is cut into 32 parts, and the top-th largest of the parts' maxima is a
// bound that at least `top` values reach and few more do (for 8 of 32 parts about 9).  Those are collected in shared memory and
// each finds its own place by counting the better ones.  Where equal values overflow the list, the places are found one by one, each in a
// reading of the whole row: right, but slow (8 best of 4096 x 32000 bf16: 68 us of normal values, 1390 of equal ones).
// A value and its class make one 64-bit key whose order is descending value, then ascending class.
#include <cooperative_groups.h>

#include <atomic>

#include "arrays.cuh"
#include "row_ring.hpp"

using namespace ftp;
using namespace ftp::arr;
namespace cg = cooperative_groups;

namespace {

constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;
constexpr float kLeast = -160.f;                       // 2^-160 is 0 in fp32: where a = -inf would make 0 * inf
constexpr int kTop = FTP_TOP_MAX;
constexpr int kParts = 32;                             // parts of a row, whose maxima bound its best values
constexpr int kListBlock = 512, kListWarp = 64;        // candidates
constexpr int kCountHere = 4096;                       // rows whose labels every block counts by itself

struct LpArgs {
    const void* z;
    void* dz;
    long long z_stride, dz_stride;
    const long long* labels;
    float *logp, *lse, *entropy, *top_logp;
    long long* top_index;
    int top;
    // gradient
    const float *lse_in, *entropy_in, *dlogp, *dentropy;
    // loss
    float scale;
    const int* counts;           // labelled rows counted by block, null: count the labels
    int n_counts;
    float* sums;                 // a sum of log probabilities for each block; null: no loss
    long long n, rows;
    int c, p;
};

enum { kStats = 0, kLoss = 1 };

__device__ __forceinline__ float ex2(float v) { float r; asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(v)); return r; }
__device__ __forceinline__ float minus_inf() { return __uint_as_float(0xff800000u); }

// Key of a value and its class; a NaN ranks as -infinity, -0 as 0.  Every key of a class is above 0.
__device__ __forceinline__ unsigned long long key_of(float v, int cls)
{
    const unsigned b = __float_as_uint(fmaxf(v, minus_inf()) + 0.f);
    const unsigned up = b & 0x80000000u ? ~b : b | 0x80000000u;
    return ((unsigned long long)up << 32) | (0xffffffffu - (unsigned)cls);
}
__device__ __forceinline__ int class_of(unsigned long long key) { return (int)(0xffffffffu - (unsigned)key); }
__device__ __forceinline__ float value_of(unsigned long long key)
{
    const unsigned up = (unsigned)(key >> 32);
    return __uint_as_float(up & 0x80000000u ? up & 0x7fffffffu : ~up);
}
__device__ __forceinline__ unsigned long long lanes_best(unsigned long long v, int width)
{
    for (int d = width >> 1; d >= 1; d >>= 1) {
        const unsigned long long u = __shfl_xor_sync(0xffffffffu, v, d);
        if (u > v) v = u;
    }
    return v;
}

// What a row (or a part of it) comes to: maximum, sum of 2^a and of a 2^a.
struct Sums { float m, s, t; };
__device__ __forceinline__ Sums join(const Sums& a, const Sums& b)
{
    if (b.s == 0.f) return a;
    if (a.s == 0.f) return b;
    const float m = fmaxf(a.m, b.m);
    const float da = (a.m - m) * kLog2e, db = (b.m - m) * kLog2e, fa = ex2(da), fb = ex2(db);
    return {m, a.s * fa + b.s * fb, (a.t + a.s * fmaxf(da, kLeast)) * fa + (b.t + b.s * fmaxf(db, kLeast)) * fb};
}

struct RowResult { float m, log_s, lse, entropy; bool empty; };
__device__ __forceinline__ RowResult result_of(const Sums& r)
{
    RowResult o;
    o.empty = r.s == 0.f;                          // every class ruled out
    o.m = r.m;
    o.log_s = logf(r.s);
    o.lse = r.m + o.log_s;
    o.entropy = o.empty ? 0.f : o.log_s - r.t / r.s * kLn2;
    return o;
}
// Log probability of a class of logit z.
__device__ __forceinline__ float logp_of(const RowResult& r, float z) { return r.empty ? minus_inf() : (z - r.m) - r.log_s; }

// The logit of a row's label, and what stands in its place (has: 1 yes, 0 no label, -1 out of range).
struct Label { long long cls; float z; int has; };
template <class T> __device__ __forceinline__ Label read_label(const LpArgs& a, long long row, const T* z, long long class_stride)
{
    Label l{a.labels ? a.labels[row] : -1, 0.f, 0};
    if (l.cls >= a.c) { l.has = -1; l.cls = -1; }
    else if (l.cls >= 0) { l.has = 1; l.z = to_f(z[l.cls * class_stride]); }
    else l.cls = -1;
    return l;
}
__device__ __forceinline__ float logp_of_label(const RowResult& r, const Label& l)
{
    return l.has > 0 ? logp_of(r, l.z) : l.has == 0 ? 0.f : nan_f();
}
__device__ __forceinline__ void write_stats(const LpArgs& a, long long row, const RowResult& r, const Label& l)
{
    if (a.logp) a.logp[row] = logp_of_label(r, l);
    if (a.lse) a.lse[row] = r.lse;
    if (a.entropy) a.entropy[row] = r.entropy;
}

// (z - m) log2 e.  The difference comes first: logits of the type's lowest value, which masks use, would overflow otherwise.
__device__ __forceinline__ float exponent_of(float z, float m) { return (z - m) * kLog2e; }

// Labelled rows of the whole call, counted by all threads of a block.
__device__ __forceinline__ float labelled_rows(const LpArgs& a)
{
    __shared__ int red[32];
    int k = 0;
    if (a.counts) for (int i = threadIdx.x; i < a.n_counts; i += blockDim.x) k += a.counts[i];
    else for (long long i = threadIdx.x; i < a.rows; i += blockDim.x) k += a.labels[i] >= 0;
    k = __reduce_add_sync(0xffffffffu, k);
    if ((threadIdx.x & 31) == 0) red[threadIdx.x >> 5] = k;
    __syncthreads();
    k = 0;
    for (int i = 0; i < (int)(blockDim.x >> 5); ++i) k += red[i];
    return (float)k;
}

// ---- matrices ---------------------------------------------------------------------------------------------------
// Largest value of packs, two 16-bit values to an instruction; NaNs are passed over.
template <class T, int V> struct Largest {
    float v = minus_inf();
    __device__ __forceinline__ void take(const Pack<T, V>& p)
    {
#pragma unroll
        for (int j = 0; j < V; ++j) v = fmaxf(v, to_f(p.get(j)));
    }
    __device__ __forceinline__ float value() const { return v; }
};
__device__ __forceinline__ __nv_bfloat162 max_two(__nv_bfloat162 a, __nv_bfloat162 b) { return __hmax2(a, b); }
__device__ __forceinline__ __half2 max_two(__half2 a, __half2 b) { return __hmax2(a, b); }
template <class T, class T2> struct LargestPairs {
    T2 v;
    __device__ __forceinline__ LargestPairs() { v.x = v.y = from_f<T>(minus_inf()); }
    __device__ __forceinline__ void take(const Pack<T, 8>& p)
    {
        const T2* w = reinterpret_cast<const T2*>(p.w);
        v = max_two(v, max_two(max_two(w[0], w[1]), max_two(w[2], w[3])));
    }
    __device__ __forceinline__ float value() const { return fmaxf(to_f(v.x), to_f(v.y)); }
};
template <> struct Largest<__nv_bfloat16, 8> : LargestPairs<__nv_bfloat16, __nv_bfloat162> {};
template <> struct Largest<__half, 8> : LargestPairs<__half, __half2> {};

// Order of fp32 values as unsigned numbers (no NaNs).
__device__ __forceinline__ unsigned order_of(float v)
{
    const unsigned b = __float_as_uint(v + 0.f);
    return b & 0x80000000u ? ~b : b | 0x80000000u;
}
// A bound that `top` of the 32 lanes' values reach at least: the maximum, taken away `top` - 1 times with all that are equal to it.  (Equal
// ones count as one, so that the bound is lower than it need be where maxima tie, as those of 16 bits often do.)
__device__ __forceinline__ float bound_of(float v, int top)
{
    unsigned mine = order_of(v), best = 0;
    for (int k = 0; k < top; ++k) {
        best = __reduce_max_sync(0xffffffffu, mine);
        if (best == order_of(minus_inf())) break;
        if (mine == best) mine = order_of(minus_inf());
    }
    return __uint_as_float(best & 0x80000000u ? best & 0x7fffffffu : ~best);
}

// The `top` best of `m` keys in `list`, found by `threads` threads by counting; write(place, key) for each.
template <class F> __device__ __forceinline__ void place(const unsigned long long* list, int m, int top, int t, int threads, F write)
{
    for (int i = t; i < m; i += threads) {
        const unsigned long long k = list[i];
        int better = 0;
        for (int j = 0; j < m; ++j) better += list[j] > k;
        if (better < top) write(better, k);
    }
}

// Sums of `n` lanes, a power of two up to 32, of which lane i has those numbered i modulo n; every lane has the result.
__device__ __forceinline__ Sums join_lanes(Sums s, int n)
{
    const int lane = threadIdx.x & 31;
#pragma unroll
    for (int d = 16; d >= 1; d >>= 1)
        if (d < n) {
            const Sums o{__shfl_xor_sync(0xffffffffu, s.m, d), __shfl_xor_sync(0xffffffffu, s.s, d), __shfl_xor_sync(0xffffffffu, s.t, d)};
            s = lane & d ? join(o, s) : join(s, o);            // (the same bits in all lanes)
        }
    return s;
}

__device__ __forceinline__ Sums join_lanes(const Sums* of, int n) { return join_lanes(of[threadIdx.x & (n - 1)], n); }

// Adds a vector's exponents to the sums of a thread, which are A side by side.
template <int MODE, int V, int A> __device__ __forceinline__ void take_sums(const Vals<V>& z, float shift, Vals<A>& s, Vals<A>& t)
{
#pragma unroll
    for (int i = 0; i < V; i += A) {
        Vals<A> x, e;
#pragma unroll
        for (int j = 0; j < A; ++j) x.v[j] = z.v[i + j];
        x = mul(add(x, all<A>(-shift)), all<A>(kLog2e));
#pragma unroll
        for (int j = 0; j < A; ++j) {
            if (MODE == kStats) x.v[j] = max_nan(x.v[j], kLeast);
            e.v[j] = ex2(x.v[j]);
        }
        s = add(s, e);
        if (MODE == kStats) t = fma(e, x, t);
    }
}

// dlogits of a vector of places e ..: g 2^((z - m) log2 e), less f at the label's place `at`; 0 if f is.
template <int V> __device__ __forceinline__ Vals<V> loss_grads(const Vals<V>& z, float m, float g, float f, int e, int at)
{
    Vals<V> x = mul(add(z, all<V>(-m)), all<V>(kLog2e));
#pragma unroll
    for (int j = 0; j < V; ++j) x.v[j] = ex2(x.v[j]);
    x = mul(x, all<V>(g));
    if (f == 0.f) x = all<V>(0.f);                              // (whatever the logits are)
    if ((unsigned)(at - e) < (unsigned)V && at >= 0) {
#pragma unroll
        for (int j = 0; j < V; ++j)
            if (e + j == at) x.v[j] -= f;
    }
    return x;
}

// How many keys a warp's list holds.  Where equal values overflowed it, the best classes take their places one after the other.
template <class T> __device__ __forceinline__ int best_of_list(const LpArgs& a, const T* zr, int found, unsigned long long* list, int lane)
{
    if (found <= kListWarp) return found;
    unsigned long long before = ~0ull;
    __syncwarp();
    for (int k = 0; k < a.top; ++k) {
        unsigned long long best = 0;
        for (int e = lane; e < a.c; e += 32) {
            const unsigned long long key = key_of(to_f(zr[e]), e);
            if (key < before && key > best) best = key;
        }
        before = lanes_best(best, 32);
        if (lane == 0) list[k] = before;
    }
    __syncwarp();
    return a.top;
}

// Rows that a warp holds in its registers, as NV vectors of V logits a lane.  SHIFT as in norm.cu: vectors lie on the 16-byte grid below
// the row's start.
constexpr int kRowWarps = 8;

template <class T, int V, int NV, bool SHIFT, int MODE>
__global__ void __launch_bounds__(kRowWarps * 32, 2) logprob_warp_rows_kernel(LpArgs a)
{
    __shared__ unsigned long long lists[kRowWarps][kListWarp];
    __shared__ int counts[kRowWarps];
    __shared__ float totals[kRowWarps];
    previous_launches();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    unsigned long long* list = lists[warp];
    int* count = counts + warp;
    const bool want_top = MODE == kStats && a.top > 0;
    float over = 0.f, total = 0.f;
    if (MODE == kLoss) {
        const float k = labelled_rows(a);
        over = k > 0.f ? a.scale / k : 0.f;
    }
    for (long long row = (long long)blockIdx.x * kRowWarps + warp; row < a.rows; row += (long long)gridDim.x * kRowWarps) {
        const T* zr = static_cast<const T*>(a.z) + row * a.z_stride;
        const int o = SHIFT ? (int)((reinterpret_cast<uintptr_t>(zr) / sizeof(T)) & (V - 1)) : 0, last = o + a.c;
        Pack<T, V> raw[NV];
        const Reach<T, V> in = reach<T, V>(zr, o, last, static_cast<const T*>(a.z), static_cast<const T*>(a.z) + (a.rows - 1) * a.z_stride + a.c);
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            raw[i] = filled<T, V>(from_f<T>(minus_inf()));
            load_whole<T, V>(raw[i], zr - o, (i * 32 + lane) * V, in.lo, in.hi);
        }
        Label label{-1, 0.f, 0};
        if (MODE == kLoss || lane == 0) label = read_label<T>(a, row, zr, 1);
        if (SHIFT || a.c % V) {
            if (!in.all) {
#pragma unroll
                for (int i = 0; i < NV; ++i) load_rest<T, V>(raw[i], zr - o, (i * 32 + lane) * V, o, last);
            }
#pragma unroll
            for (int i = 0; i < NV; ++i) keep_part<T, V>(raw[i], (i * 32 + lane) * V, o, last, from_f<T>(minus_inf()));
        }
        Largest<T, V> most;
#pragma unroll
        for (int i = 0; i < NV; ++i) most.take(raw[i]);
        const float mine = most.value(), m = lanes_max(mine), shift = m == minus_inf() ? 0.f : m;
        Vals<V> s = all<V>(0.f), x2 = all<V>(0.f);
#pragma unroll
        for (int i = 0; i < NV; ++i) take_sums<MODE>(values(raw[i]), shift, s, x2);
        Sums sums{shift, lanes_sum(sum_of(s)), 0.f};
        if (MODE == kStats) sums.t = lanes_sum(sum_of(x2));
        const RowResult r = result_of(sums);
        if (MODE == kStats && lane == 0) write_stats(a, row, r, label);
        if (want_top) {
            if (lane == 0) *count = 0;
            __syncwarp();
            const float bound = bound_of(mine, a.top);
            if (mine >= bound) {
#pragma unroll
                for (int i = 0; i < NV; ++i) {
                    const int e = (i * 32 + lane) * V;
#pragma unroll
                    for (int j = 0; j < V; ++j) {
                        const float v = fmaxf(to_f(raw[i].get(j)), minus_inf());
                        if (v >= bound && e + j >= o && e + j < last) {
                            const int at = atomicAdd(count, 1);
                            if (at < kListWarp) list[at] = key_of(v, e + j - o);
                        }
                    }
                }
            }
            __syncwarp();
            const int found = best_of_list<T>(a, zr, *count, list, lane);
            place(list, found, a.top, lane, 32, [&](int at, unsigned long long k) {
                if (a.top_logp) a.top_logp[row * a.top + at] = logp_of(r, value_of(k));
                if (a.top_index) a.top_index[row * a.top + at] = class_of(k);
            });
            __syncwarp();
        }
        if (MODE == kLoss) {
            if (lane == 0 && label.has) total += logp_of_label(r, label);
            __syncwarp();                        // lane 0 has the label's logit, which another lane may write over (dlogits in its place)
            if (a.dz) {
                T* dr = static_cast<T*>(a.dz) + row * a.dz_stride - o;
                const float f = label.has > 0 ? (r.empty ? 0.f : over) : label.has == 0 ? 0.f : nan_f(), g = f == 0.f ? 0.f : f / sums.s;
                const int at = label.has > 0 ? (int)label.cls + o : -1;
#pragma unroll
                for (int i = 0; i < NV; ++i) {
                    const int e = (i * 32 + lane) * V;
                    if (e < last) store_part<T, V>(dr, e, o, last, rounded<T, V>(loss_grads(values(raw[i]), sums.m, g, f, e, at)));
                }
            }
        }
    }
    if (MODE == kLoss && a.sums) {
        if (lane == 0) totals[warp] = total;
        __syncthreads();
        if (threadIdx.x == 0) {
            float s = 0.f;
            for (int i = 0; i < kRowWarps; ++i) s += totals[i];
            a.sums[blockIdx.x] = s;
        }
    }
}

// Many long rows: a warp streams a row, four vectors a lane at a time with the next four on their way, and keeps a running maximum that
// the sums are brought to when it grows.  Without barriers, and with what a row costs once (400 instructions) spread over all of its values
// in a lane: 4096 x 32000 bf16 with the eight best take 122 us with a block a row.  The row is cut into up to 32 units of batches, and the
// largest value of each lane in each unit stays in shared memory: where one reaches the bound, the whole warp looks the lane's values over.
constexpr int kStreamWarps = 4, kBatch = 4, kUnits = 32;

template <class T, bool SHIFT> __global__ void __launch_bounds__(kStreamWarps * 32, 7) logprob_stream_rows_kernel(LpArgs a)
{
    constexpr int V = 16 / sizeof(T), kWide = 32 * V * kBatch;              // places of a batch
    __shared__ unsigned long long lists[kStreamWarps][kListWarp];
    __shared__ int counts[kStreamWarps];
    __shared__ float largest_of[kStreamWarps][kUnits][32];
    previous_launches();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    unsigned long long* list = lists[warp];
    int* count = counts + warp;
    for (long long row = (long long)blockIdx.x * kStreamWarps + warp; row < a.rows; row += (long long)gridDim.x * kStreamWarps) {
        const T* zr = static_cast<const T*>(a.z) + row * a.z_stride;
        const int o = SHIFT ? (int)((reinterpret_cast<uintptr_t>(zr) / sizeof(T)) & (V - 1)) : 0, last = o + a.c;
        const int batches = (last + kWide - 1) / kWide, unit = (batches + kUnits - 1) / kUnits, units = (batches + unit - 1) / unit;
        const T* grid = zr - o;
        Label label{-1, 0.f, 0};
        if (lane == 0) label = read_label<T>(a, row, zr, 1);
        Pack<T, V> next[kBatch];
        auto fetch = [&](int b) {
            const int e = b * kWide + lane * V;
            if ((!SHIFT || b > 0) && (b + 1) * kWide <= last) {
#pragma unroll
                for (int i = 0; i < kBatch; ++i) next[i] = load_pack<T, V>(grid + e + i * 32 * V);
            } else {
#pragma unroll
                for (int i = 0; i < kBatch; ++i) {
                    next[i] = filled<T, V>(from_f<T>(minus_inf()));
                    load_whole<T, V>(next[i], grid, e + i * 32 * V, o, last);
                }
#pragma unroll
                for (int i = 0; i < kBatch; ++i) load_rest<T, V>(next[i], grid, e + i * 32 * V, o, last);
            }
        };
        fetch(0);
        float most = minus_inf(), shift = 0.f;
        Vals<4> s = all<4>(0.f), x2 = all<4>(0.f);
        int b = 0;
        for (int u = 0; u < units; ++u) {
            float here_most = minus_inf();
            for (const int end = min(batches, (u + 1) * unit); b < end;) {
                Pack<T, V> raw[kBatch];
                Largest<T, V> here;
#pragma unroll
                for (int i = 0; i < kBatch; ++i) { raw[i] = next[i]; here.take(raw[i]); }
                if (++b < batches) fetch(b);
                const float big = here.value();
                here_most = fmaxf(here_most, big);
                if (__any_sync(0xffffffffu, big > most)) {
                    most = fmaxf(most, big);
                    const float to = most == minus_inf() ? 0.f : most;
                    // (a sum of 0 has no maximum yet, and one far below the new maximum counts for nothing: neither must make 0 * inf)
                    const float d = sum_of(s) == 0.f ? 0.f : fmaxf((shift - to) * kLog2e, kLeast), f = ex2(d);
                    x2 = mul(fma(s, all<4>(d), x2), all<4>(f));
                    s = mul(s, all<4>(f));
                    shift = to;
                }
#pragma unroll
                for (int i = 0; i < kBatch; ++i) {
                    keep_packed(raw[i]);
                    take_sums<kStats>(values(raw[i]), shift, s, x2);
                }
            }
            if (a.top > 0) largest_of[warp][u][lane] = here_most;
        }
        const float m = lanes_max(most), to = m == minus_inf() ? 0.f : m;
        Sums sums{to, sum_of(s), sum_of(x2)};
        {
            const float d = sums.s == 0.f ? 0.f : fmaxf((shift - to) * kLog2e, kLeast), f = ex2(d);
            sums.t = lanes_sum(fmaf(sums.s, d, sums.t) * f);
            sums.s = lanes_sum(sums.s * f);
        }
        const RowResult r = result_of(sums);
        if (lane == 0) write_stats(a, row, r, label);
        if (a.top == 0) continue;
        if (lane == 0) *count = 0;
        __syncwarp();
        const float bound = bound_of(most, a.top);
        for (int u = 0; u < units; ++u) {
            for (unsigned who = __ballot_sync(0xffffffffu, largest_of[warp][u][lane] >= bound); who; who &= who - 1) {
                const int first = (__ffs(who) - 1) * V, end = min(batches, (u + 1) * unit);
                // a batch has 32 values of each lane (16 in fp32): one for each lane to look at
                for (int at = u * unit; at < end; ++at) {
                    const int e = at * kWide + (lane / V % kBatch) * 32 * V + first + lane % V;
                    if (lane >= V * kBatch || e < o || e >= last) continue;
                    const float v = fmaxf(to_f(grid[e]), minus_inf());
                    if (v >= bound) {
                        const int place = atomicAdd(count, 1);
                        if (place < kListWarp) list[place] = key_of(v, e - o);
                    }
                }
                __syncwarp();
            }
        }
        __syncwarp();
        const int found = best_of_list<T>(a, zr, *count, list, lane);
        place(list, found, a.top, lane, 32, [&](int at, unsigned long long k) {
            if (a.top_logp) a.top_logp[row * a.top + at] = logp_of(r, value_of(k));
            if (a.top_index) a.top_index[row * a.top + at] = class_of(k);
        });
        __syncwarp();
    }
}

// Longer rows: TH threads of a block have a row, or with a cluster its part of one, in shared memory, and the next ones are on their
// way into the other stages.  A thread copies (cp.async, 16 bytes each) what it will read itself, every TH-th vector, so that no barrier
// stands between copy and use, and the passes over the row are short loops: with the row in registers instead they had to be
// unrolled in full and waited for instructions more than for anything else (4096 x 32000 bf16 with the eight best: 159 us).
// What is left to do for a row once its sums and its list of candidates are there, a thousand cycles of one warp, is one more warp's
// (FIN), while the others are at the next row.  Blocks of a cluster, and the loss, whose delta needs the sums at once, do without.
constexpr int kStageMost = 64 * 1024;            // bytes of a part: 32768 classes of 16 bits, 16384 of 32

struct BlockShared {
    unsigned long long list[kListBlock];
    unsigned long long best[2][kTop];            // a block's own best, for the cluster; of this row and the one before
    unsigned long long round[32];
    float parts[kParts];
    Sums sums[2][32];                            // of the warps; of this row and the one before
    int count[2];
    Sums whole[2];
};

__device__ __forceinline__ void copy_16(void* to, const void* from)
{
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"((unsigned)__cvta_generic_to_shared(to)), "l"(from) : "memory");
}
__device__ __forceinline__ void copies_of_row_end() { asm volatile("cp.async.commit_group;" ::: "memory"); }
// Waits until all but the last `left` rows' copies of this thread have arrived.
__device__ __forceinline__ void wait_rows(int left)
{
    if (left <= 0) asm volatile("cp.async.wait_group 0;" ::: "memory");
    else if (left == 1) asm volatile("cp.async.wait_group 1;" ::: "memory");
    else if (left == 2) asm volatile("cp.async.wait_group 2;" ::: "memory");
    else asm volatile("cp.async.wait_group 3;" ::: "memory");
}

template <class T, bool SHIFT, int MODE, int TH, bool FIN>
__global__ void __launch_bounds__(TH + (FIN ? 32 : 0), TH == 128 ? 3 : 1)
logprob_block_rows_kernel(LpArgs a, int cluster, int part, int stages, bool dz_vec)
{
    constexpr int V = 16 / sizeof(T), kWarps = TH / 32, kLanes = TH / kParts, kStep = TH * V, kAll = TH + (FIN ? 32 : 0);
    extern __shared__ __align__(16) unsigned char ring[];
    __shared__ BlockShared sh;
    previous_launches();
    const int t = threadIdx.x, lane = t & 31;
    const int rank = FIN ? 0 : (int)(blockIdx.x % cluster);
    const long long step = FIN ? gridDim.x : gridDim.x / cluster;
    const bool want_top = MODE == kStats && a.top > 0;
    float over = 0.f, total = 0.f;
    if (MODE == kLoss) {
        const float k = labelled_rows(a);
        over = k > 0.f ? a.scale / k : 0.f;
    }
    if (t < 2) sh.count[t] = 0;
    __syncthreads();
    long long row = FIN ? blockIdx.x : blockIdx.x / cluster;
    int turn = 0;
    auto sync_rows = [&] { if constexpr (FIN) group_barrier(1, kAll); else __syncthreads(); };
    auto sync_list = [&] { if constexpr (FIN) group_barrier(2, kAll); else __syncthreads(); };
    if (FIN && t >= TH) {
        for (; row < a.rows; row += step, turn ^= 1) {
            Label label{-1, 0.f, 0};
            if (lane == 0) label = read_label<T>(a, row, static_cast<const T*>(a.z) + row * a.z_stride, 1);
            sync_rows();                         // (this also says that the list of the row before has been read)
            const RowResult r = result_of(join_lanes(sh.sums[turn], kWarps));
            if (lane == 0) write_stats(a, row, r, label);
            if (!want_top) continue;
            sync_list();
            int found = sh.count[turn];
            if (found > kListBlock) { sync_list(); found = a.top; }
            place(sh.list, found, a.top, lane, 32, [&](int at, unsigned long long k) {
                if (a.top_logp) a.top_logp[row * a.top + at] = logp_of(r, value_of(k));
                if (a.top_index) a.top_index[row * a.top + at] = class_of(k);
            });
        }
        return;
    }
    auto shift_of = [&](const T* zr) { return SHIFT ? (int)((reinterpret_cast<uintptr_t>(zr) / sizeof(T)) & (V - 1)) : 0; };
    // places [first, last) of the row, on the grid that starts o below it, are this block's; a thread's vectors start at first + t V + k kStep
    auto fetch = [&](long long row, int stage) {
        if (row < a.rows) {
            const T* zr = static_cast<const T*>(a.z) + row * a.z_stride;
            const int o = shift_of(zr), first = rank * part, last = min(o + a.c, first + part), mine = last - first - t * V;
            T* to = reinterpret_cast<T*>(ring + (size_t)stage * part * sizeof(T)) + t * V;
            zr -= o;
            const T* from = zr + first + t * V;
            const int whole = mine < V ? 0 : (mine - V) / kStep + 1;                    // vectors that end before `last`
            const bool head = SHIFT && o > 0 && rank == 0 && t == 0;                    // the first one starts before the row
#pragma unroll 4
            for (int k = head ? 1 : 0; k < whole; ++k) copy_16(to + k * kStep, from + k * kStep);
            auto across = [&](int k) {
                Pack<T, V> p = filled<T, V>(from_f<T>(minus_inf()));
                load_rest<T, V>(p, zr, first + t * V + k * kStep, o, last);
                store_pack<T, V>(to + k * kStep, p);
            };
            if (head) across(0);
            if (whole * kStep < mine && !(head && whole == 0)) across(whole);
        }
        copies_of_row_end();
    };
    for (int i = 0; i + 1 < stages; ++i) fetch(row + i * step, i);
    int stage = 0;
    for (; row < a.rows; row += step, turn ^= 1) {
        const T* zr = static_cast<const T*>(a.z) + row * a.z_stride;
        const int o = shift_of(zr), first = rank * part, last = min(o + a.c, first + part);
        const T* mine_at = reinterpret_cast<const T*>(ring + (size_t)stage * part * sizeof(T)) + t * V;
        const int vectors = max(0, (last - first - t * V + kStep - 1) / kStep);
        Label label{-1, 0.f, 0};
        if (!FIN && (MODE == kLoss || t == 0)) label = read_label<T>(a, row, zr, 1);
        fetch(row + (stages - 1) * step, stage == 0 ? stages - 1 : stage - 1);
        wait_rows(stages - 1);
        stage = stage + 1 == stages ? 0 : stage + 1;
        Largest<T, V> most;
#pragma unroll 4
        for (int k = 0; k < vectors; ++k) most.take(load_pack<T, V>(mine_at + k * kStep));
        const float mine = most.value();
        // largest of a part of the row, and of the warp, which the exponents are taken from
        const float part_max = lanes_max(mine, kLanes);
        if (want_top && lane % kLanes == 0) sh.parts[t / kLanes] = part_max;
        const float m = lanes_max(part_max), shift = m == minus_inf() ? 0.f : m;
        Vals<V> s = all<V>(0.f), x2 = all<V>(0.f);
#pragma unroll 4
        for (int k = 0; k < vectors; ++k) take_sums<MODE>(values(load_pack<T, V>(mine_at + k * kStep)), shift, s, x2);
        Sums sums{shift, lanes_sum(sum_of(s)), 0.f};
        if (MODE == kStats) sums.t = lanes_sum(sum_of(x2));
        if (lane == 0) sh.sums[turn][t >> 5] = sums;
        sync_rows();
        if (!FIN && (t < 32 || MODE == kLoss || cluster > 1)) sums = join_lanes(sh.sums[turn], kWarps);
        if (t == 0) sh.count[turn ^ 1] = 0;
        // the best classes of this part
        int found = 0;
        if (want_top) {
            const float bound = bound_of(sh.parts[lane], a.top);
            if (mine >= bound) {
                for (int k = 0; k < vectors; ++k) {
                    const Pack<T, V> p = load_pack<T, V>(mine_at + k * kStep);
                    Largest<T, V> here;
                    here.take(p);
                    if (here.value() < bound) continue;
                    const int e = first + t * V + k * kStep;
#pragma unroll
                    for (int j = 0; j < V; ++j) {
                        const float v = fmaxf(to_f(p.get(j)), minus_inf());
                        if (v >= bound && e + j >= o && e + j < last) {
                            const int at = atomicAdd(&sh.count[turn], 1);
                            if (at < kListBlock) sh.list[at] = key_of(v, e + j - o);
                        }
                    }
                }
            }
            sync_list();
            found = sh.count[turn];
            if (found > kListBlock) {                             // too many equal ones: one place after the other
                unsigned long long before = ~0ull;
                const int places = min(a.top, found);
                for (int k = 0; k < places; ++k) {
                    unsigned long long best = 0;
                    for (int e = max(first, o) + t; e < last; e += TH) {
                        const unsigned long long key = key_of(to_f(zr[e - o]), e - o);
                        if (key < before && key > best) best = key;
                    }
                    best = lanes_best(best, 32);
                    group_barrier(3, TH);
                    if (lane == 0) sh.round[t >> 5] = best;
                    group_barrier(3, TH);
                    before = lanes_best(sh.round[lane & (kWarps - 1)], 32);
                    if (t == 0) sh.list[k] = before;
                }
                found = places;
                sync_list();
            }
        }
        if (!FIN && cluster > 1) {
            cg::cluster_group cl = cg::this_cluster();
            if (want_top) {
                if (t < kTop) sh.best[turn][t] = 0;
                __syncthreads();
                place(sh.list, found, a.top, t, TH, [&](int at, unsigned long long k) { sh.best[turn][at] = k; });
            }
            if (t == 0) sh.whole[turn] = sums;
            // one barrier a row: what is read here is written again for the row after the next, behind the next row's barrier (300 bf16
            // rows of 250000 classes without best ones: 102 us; with a second barrier and each thread joining all blocks' sums one after the other
            // 140)
            cl.sync();
            if (MODE == kLoss || rank == 0) sums = join_lanes(*cl.map_shared_rank(&sh.whole[turn], lane & (cluster - 1)), cluster);
            if (want_top && rank == 0) {
                found = cluster * a.top;
                for (int i = t; i < found; i += TH) sh.list[i] = cl.map_shared_rank(sh.best[turn], i / a.top)[i % a.top];
                __syncthreads();
            }
        }
        if (!FIN && MODE == kStats && rank == 0) {                // (cluster > 1: a row alone has the warp above)
            const RowResult r = result_of(sums);
            if (t == 0) write_stats(a, row, r, label);
            if (want_top)
                place(sh.list, found, a.top, t, TH, [&](int at, unsigned long long k) {
                    if (a.top_logp) a.top_logp[row * a.top + at] = logp_of(r, value_of(k));
                    if (a.top_index) a.top_index[row * a.top + at] = class_of(k);
                });
        }
        if (MODE == kLoss) {
            const RowResult r = result_of(sums);
            if (t == 0 && rank == 0 && label.has) total += logp_of_label(r, label);
            if (a.dz) {
                T* dr = static_cast<T*>(a.dz) + row * a.dz_stride - o;
                const float f = label.has > 0 ? (r.empty ? 0.f : over) : label.has == 0 ? 0.f : nan_f(), g = f == 0.f ? 0.f : f / sums.s;
                const int at = label.has > 0 ? (int)label.cls + o : -1;
#pragma unroll 2
                for (int k = 0; k < vectors; ++k) {
                    const int e = first + t * V + k * kStep;
                    const Pack<T, V> d = rounded<T, V>(loss_grads(values(load_pack<T, V>(mine_at + k * kStep)), sums.m, g, f, e, at));
                    if (dz_vec) store_part<T, V>(dr, e, o, last, d);
                    else {
#pragma unroll
                        for (int j = 0; j < V; ++j)
                            if (e + j >= o && e + j < last) dr[e + j] = d.get(j);
                    }
                }
            }
        }
    }
    if (!FIN && cluster > 1) cg::this_cluster().sync();           // the others read this block's part
    wait_rows(0);
    if (MODE == kLoss && a.sums && t == 0) a.sums[blockIdx.x] = total;
}

// ---- maps -------------------------------------------------------------------------------------------------------
// As in norm.cu: a lane has V pixels (4 bytes of them, or one value), `share` warps split the classes, up to CPT of them to a warp, in
// registers.  CPT = 0: any number, read again for every pass.  If share is 1 the warps of a block take a tile each and need no barrier.
constexpr int kMapWarps = 16;

// Best of each pixel over the warps of the block; `red`: a value a thread, not read or written by others until the next barrier.
template <class V, class F> __device__ __forceinline__ V across_warps(V v, int share, V* red, F better)
{
    if (share == 1) return v;
    const int lane = threadIdx.x & 31;
    red[threadIdx.x] = v;
    __syncthreads();
    v = red[lane];
    for (int w = 1; w < share; ++w) v = better(v, red[w * 32 + lane]);
    return v;
}

template <class T, int V, int CPT, int MODE, bool TOP>
__device__ __forceinline__ void logprob_tile(const LpArgs& a, long long n, int px, int first, int per, int share, float over, float& total,
                                             float (*red)[32 * kMapWarps * V], unsigned long long (*keys)[TOP ? 32 * kMapWarps : 1])
{
    const int count = min(per, a.c - first);
    const bool live = px < a.p;
    const long long row = n * a.p + px;
    const T* zt = static_cast<const T*>(a.z) + n * a.z_stride + px;
    const unsigned bytes = (unsigned)a.p * sizeof(T);
    const char* base = reinterpret_cast<const char*>(zt + (long long)first * a.p);
    auto load = [&](int i) {
        Pack<T, V> r = filled<T, V>(from_f<T>(minus_inf()));
        if (live && i < count) r = load_pack<T, V>(reinterpret_cast<const T*>(base + (unsigned long long)bytes * (unsigned)i));
        return r;
    };
    Pack<T, V> raw[CPT ? CPT : 1];
    if constexpr (CPT > 0) {
#pragma unroll
        for (int i = 0; i < CPT; ++i) raw[i] = filled<T, V>(from_f<T>(minus_inf()));
        if (live) {
#pragma unroll
            for (int i0 = 0; i0 < CPT; i0 += 8) {
                if (i0 + 8 <= count) {
#pragma unroll
                    for (int i = i0; i < i0 + 8; ++i) raw[i] = load_pack<T, V>(reinterpret_cast<const T*>(base + (unsigned long long)bytes * (unsigned)i));
                } else {
#pragma unroll
                    for (int i = i0; i < i0 + 8; ++i)
                        if (i < count) raw[i] = load_pack<T, V>(reinterpret_cast<const T*>(base + (unsigned long long)bytes * (unsigned)i));
                }
            }
        }
    }
    Label label[V];
    if (live && (MODE == kLoss || first == 0)) {
#pragma unroll
        for (int j = 0; j < V; ++j) label[j] = read_label<T>(a, row + j, zt + j, a.p);
    }
    auto each = [&](auto f) {
        if constexpr (CPT > 0) {
#pragma unroll
            for (int i0 = 0; i0 < CPT; i0 += 8) {               // eight without a test, where there are as many
                if (i0 + 8 <= count) {
#pragma unroll
                    for (int i = i0; i < i0 + 8; ++i) f(raw[i], i);
                } else {
#pragma unroll
                    for (int i = i0; i < i0 + 8; ++i)
                        if (i < count) f(raw[i], i);
                }
            }
        } else {
            for (int i = 0; i < count; ++i) {
                Pack<T, V> r = load(i);
                f(r, i);
            }
        }
    };
    Vals<V> m = all<V>(minus_inf()), s = all<V>(0.f), t = all<V>(0.f);
    each([&](const Pack<T, V>& r, int) {
        const Vals<V> z = values(r);
#pragma unroll
        for (int j = 0; j < V; ++j) m.v[j] = fmaxf(m.v[j], z.v[j]);
    });
#pragma unroll
    for (int j = 0; j < V; ++j) {
        m.v[j] = across_warps(m.v[j], share, red[0] + j * 32 * kMapWarps, [](float x, float y) { return fmaxf(x, y); });
        if (m.v[j] == minus_inf()) m.v[j] = 0.f;
    }
    const Vals<V> minus_m = mul(m, all<V>(-1.f));
    constexpr bool kKeep = MODE == kLoss && CPT > 0 && sizeof(T) == 4;         // the exponentials take the logits' registers
    each([&](Pack<T, V>& r, int) {
        Vals<V> x = mul(add(values(r), minus_m), all<V>(kLog2e)), e;
#pragma unroll
        for (int j = 0; j < V; ++j) {
            if (MODE == kStats) x.v[j] = max_nan(x.v[j], kLeast);
            e.v[j] = ex2(x.v[j]);
        }
        s = add(s, e);
        if (MODE == kStats) t = fma(e, x, t);
        if (kKeep) r = rounded<T, V>(e);
    });
    // (three buffers in turn: each is written again only after a barrier that follows its last reading)
#pragma unroll
    for (int j = 0; j < V; ++j) {
        s.v[j] = across_warps(s.v[j], share, red[1] + j * 32 * kMapWarps, [](float x, float y) { return x + y; });
        if (MODE == kStats) t.v[j] = across_warps(t.v[j], share, red[2] + j * 32 * kMapWarps, [](float x, float y) { return x + y; });
    }
    RowResult r[V];
#pragma unroll
    for (int j = 0; j < V; ++j) r[j] = result_of(Sums{m.v[j], s.v[j], t.v[j]});
    if (MODE == kStats && live && first == 0) {
#pragma unroll
        for (int j = 0; j < V; ++j) write_stats(a, row + j, r[j], label[j]);
    }
    if constexpr (TOP) {
        // Every place looks at every class (8 x 21 x 416 x 416: 34 us without best classes, 57 with one, 120 with 5, 359 with 20).
        unsigned long long before = ~0ull;
        for (int k = 0; k < a.top; ++k) {
            unsigned long long best = 0;
            each([&](const Pack<T, V>& q, int i) {
                const unsigned long long key = key_of(to_f(q.get(0)), first + i);
                if (key < before && key > best) best = key;
            });
            before = across_warps(best, share, keys[k & 1], [](unsigned long long x, unsigned long long y) { return x > y ? x : y; });
            if (live && first == 0) {
                const long long at = (n * a.top + k) * a.p + px;
                if (a.top_logp) a.top_logp[at] = logp_of(r[0], value_of(before));
                if (a.top_index) a.top_index[at] = class_of(before);
            }
        }
    }
    if (MODE == kLoss) {
        Vals<V> g, f;
#pragma unroll
        for (int j = 0; j < V; ++j) {
            if (!live) { f.v[j] = g.v[j] = 0.f; continue; }
            f.v[j] = label[j].has > 0 ? (r[j].empty ? 0.f : over) : label[j].has == 0 ? 0.f : nan_f();
            g.v[j] = f.v[j] == 0.f ? 0.f : f.v[j] / s.v[j];
            if (first == 0 && label[j].has) total += logp_of_label(r[j], label[j]);
        }
        if (a.dz && live) {
            char* out = reinterpret_cast<char*>(static_cast<T*>(a.dz) + n * a.dz_stride + (long long)first * a.p + px);
            each([&](const Pack<T, V>& q, int i) {
                Vals<V> x = values(q);
                if (!kKeep) {
                    x = mul(add(x, minus_m), all<V>(kLog2e));
#pragma unroll
                    for (int j = 0; j < V; ++j) x.v[j] = ex2(x.v[j]);
                }
                x = mul(x, g);
#pragma unroll
                for (int j = 0; j < V; ++j) {
                    if (f.v[j] == 0.f) x.v[j] = 0.f;            // (whatever the logits are)
                    if (first + i == (int)label[j].cls) x.v[j] -= f.v[j];
                }
                store_pack<T, V>(reinterpret_cast<T*>(out + (unsigned long long)bytes * (unsigned)i), rounded<T, V>(x));
            });
        }
    }
}

// MOST: warps of a block at most.  Blocks of four are held to 64 registers in the loss, for 32 warps an SM (90 registers and 20 warps: a map of
// 21 classes and 416 x 416 pixels takes 59 us instead of 55).
template <class T, int V, int CPT, int MODE, bool TOP, int MOST>
__global__ void __launch_bounds__(32 * MOST, MOST == 4 && MODE == kLoss ? 8 : 1) logprob_map_kernel(LpArgs a, int share, int per, int tiles)
{
    __shared__ float red[3][32 * kMapWarps * V];
    __shared__ unsigned long long keys[2][TOP ? 32 * kMapWarps : 1];
    previous_launches();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, warps = blockDim.x >> 5, groups = warps / share;
    const int first = (warp & (share - 1)) * per;
    float over = 0.f, total = 0.f;
    if (MODE == kLoss) {
        const float k = labelled_rows(a);
        over = k > 0.f ? a.scale / k : 0.f;
    }
    for (Walk w(blockIdx.x * groups + warp / share, gridDim.x * groups, tiles); w.hi < a.n; w.advance()) {
        logprob_tile<T, V, CPT, MODE, TOP>(a, w.hi, w.lo * 32 * V + lane * V, first, per, share, over, total, red, keys);
        if (TOP && share > 1) __syncthreads();                  // (the keys' two buffers start over)
    }
    if (MODE == kLoss && a.sums) {
        total = lanes_sum(total);
        __syncthreads();
        if (lane == 0) red[0][warp] = total;
        __syncthreads();
        if (threadIdx.x == 0) {
            float sum = 0.f;
            for (int w = 0; w < warps; ++w) sum += red[0][w];
            a.sums[blockIdx.x] = sum;
        }
    }
}

// ---- the loss around them ---------------------------------------------------------------------------------------
__global__ void __launch_bounds__(256) count_labels_kernel(const long long* labels, long long rows, int* counts)
{
    __shared__ int red[8];
    previous_launches();
    next_launch();
    int k = 0;
    for (long long i = (long long)blockIdx.x * 256 + threadIdx.x; i < rows; i += (long long)gridDim.x * 256) k += labels[i] >= 0;
    k = __reduce_add_sync(0xffffffffu, k);
    if ((threadIdx.x & 31) == 0) red[threadIdx.x >> 5] = k;
    __syncthreads();
    if (threadIdx.x == 0) {
        k = 0;
        for (int i = 0; i < 8; ++i) k += red[i];
        counts[blockIdx.x] = k;
    }
}

__global__ void __launch_bounds__(512) loss_finish_kernel(LpArgs a, int sums, float* loss)
{
    __shared__ float red[16];
    previous_launches();
    const float k = labelled_rows(a);
    float s = 0.f;
    for (int i = threadIdx.x; i < sums; i += 512) s += a.sums[i];
    s = lanes_sum(s, 32);
    if ((threadIdx.x & 31) == 0) red[threadIdx.x >> 5] = s;
    __syncthreads();
    if (threadIdx.x == 0) {
        s = 0.f;
        for (int i = 0; i < 16; ++i) s += red[i];
        *loss = k > 0.f ? -s / k : 0.f;
    }
}

// ---- gradient ---------------------------------------------------------------------------------------------------
// What a row's classes share: dlogits = w_l (class = label) - p (w_l + w_h (log p + entropy)) = w_l (class = label) - p (base + slope x)
// with x = log2 p.
struct RowGrad { float lse, wl, base, slope; int cls; };
__device__ __forceinline__ RowGrad row_grad(const LpArgs& a, long long row)
{
    RowGrad r;
    r.lse = a.lse_in[row];
    const long long cls = a.labels ? a.labels[row] : -1;
    r.cls = cls >= 0 && cls < a.c ? (int)cls : -1;
    r.wl = a.dlogp && r.cls >= 0 ? a.dlogp[row] : 0.f;
    if (cls >= a.c) r.wl = nan_f();
    const float wh = a.dentropy ? a.dentropy[row] : 0.f;
    r.base = a.dentropy ? fmaf(wh, a.entropy_in[row], r.wl) : r.wl;
    r.slope = wh * kLn2;
    if (r.lse == minus_inf()) { r.lse = INFINITY; r.wl = r.base = r.slope = 0.f; }         // nothing left: all p are 0
    return r;
}
template <int V> __device__ __forceinline__ Vals<V> class_grads(const Vals<V>& z, const Vals<V>& minus_lse, const Vals<V>& slope, const Vals<V>& base)
{
    Vals<V> x = mul(add(z, minus_lse), all<V>(kLog2e)), p;
#pragma unroll
    for (int j = 0; j < V; ++j) { x.v[j] = max_nan(x.v[j], kLeast); p.v[j] = ex2(x.v[j]); }
    return mul(mul(p, all<V>(-1.f)), fma(slope, x, base));
}

template <class T, int V, bool SHIFT> __global__ void __launch_bounds__(256) logprob_bwd_rows_kernel(LpArgs a, int segments)
{
    previous_launches();
    constexpr int kPer = 4, kSegment = 32 * V * kPer;
    const int lane = threadIdx.x & 31;
    for (Walk w(blockIdx.x * 8 + (threadIdx.x >> 5), gridDim.x * 8, segments); w.hi < a.rows; w.advance()) {
        const long long row = w.hi;
        const int first = w.lo * kSegment + lane * V;
        const T* zr = static_cast<const T*>(a.z) + row * a.z_stride;
        const int o = SHIFT ? (int)((reinterpret_cast<uintptr_t>(zr) / sizeof(T)) & (V - 1)) : 0;
        const int hi = o + a.c;
        const Reach<T, V> in = reach<T, V>(zr, o, hi, static_cast<const T*>(a.z), static_cast<const T*>(a.z) + (a.rows - 1) * a.z_stride + a.c);
        zr -= o;
        T* dr = static_cast<T*>(a.dz) + row * a.dz_stride - o;
        Pack<T, V> raw[kPer];
#pragma unroll
        for (int i = 0; i < kPer; ++i) {
            raw[i] = zero_pack<T, V>();
            load_whole<T, V>(raw[i], zr, first + i * 32 * V, in.lo, in.hi);          // (places outside the row are not stored: they may hold anything)
        }
        const RowGrad r = row_grad(a, row);
        if ((SHIFT || a.c % V) && !in.all) {
#pragma unroll
            for (int i = 0; i < kPer; ++i) load_rest<T, V>(raw[i], zr, first + i * 32 * V, o, hi);
        }
        const int at = r.cls >= 0 ? r.cls + o : -1;
#pragma unroll
        for (int i = 0; i < kPer; ++i) {
            const int e = first + i * 32 * V;
            if (e >= hi) continue;
            Vals<V> d = class_grads(values(raw[i]), all<V>(-r.lse), all<V>(r.slope), all<V>(r.base));
            if ((unsigned)(at - e) < (unsigned)V && at >= 0) {
#pragma unroll
                for (int j = 0; j < V; ++j)
                    if (e + j == at) d.v[j] += r.wl;
            }
            store_part<T, V>(dr, e, o, hi, rounded<T, V>(d));
        }
    }
}

template <class T, int V> __global__ void __launch_bounds__(256) logprob_bwd_map_kernel(LpArgs a, int tiles)
{
    previous_launches();
    constexpr int kSlab = 16, kAhead = 8;
    const int lane = threadIdx.x & 31;
    const int c0 = blockIdx.y * kSlab, c1 = min(a.c, c0 + kSlab);
    for (Walk w(blockIdx.x * 8 + (threadIdx.x >> 5), gridDim.x * 8, tiles); w.hi < a.n; w.advance()) {
        const long long n = w.hi;
        const int px = w.lo * 32 * V + lane * V;
        if (px >= a.p) continue;
        const T* zt = static_cast<const T*>(a.z) + n * a.z_stride + px;
        T* dt = static_cast<T*>(a.dz) + n * a.dz_stride + px;
        Vals<V> minus_lse, slope, base, wl;
        int cls[V];
#pragma unroll
        for (int j = 0; j < V; ++j) {
            const RowGrad r = row_grad(a, n * a.p + px + j);
            minus_lse.v[j] = -r.lse; slope.v[j] = r.slope; base.v[j] = r.base; wl.v[j] = r.wl; cls[j] = r.cls;
        }
        for (int ch = c0; ch < c1; ch += kAhead) {
            Pack<T, V> raw[kAhead];
#pragma unroll
            for (int i = 0; i < kAhead; ++i)
                if (ch + i < c1) raw[i] = load_pack<T, V>(zt + (long long)(ch + i) * a.p);
#pragma unroll
            for (int i = 0; i < kAhead; ++i) {
                if (ch + i >= c1) continue;
                Vals<V> d = class_grads(values(raw[i]), minus_lse, slope, base);
#pragma unroll
                for (int j = 0; j < V; ++j)
                    if (ch + i == cls[j]) d.v[j] += wl.v[j];
                store_pack<T, V>(dt + (long long)(ch + i) * a.p, rounded<T, V>(d));
            }
        }
    }
}

// ---- host -------------------------------------------------------------------------------------------------------
constexpr int kMostBlocks = kLossBlocksPerSm * kSms;         // blocks of a loss, each with a sum
constexpr int kMostCounts = 1024;

template <class T, int V, int NV, bool SHIFT, int MODE> int run_warp_rows(const LpArgs& a, int* blocks, cudaStream_t st)
{
    const int fit = resident<logprob_warp_rows_kernel<T, V, NV, SHIFT, MODE>>(kRowWarps * 32, 0);
    const long long want = (a.rows + kRowWarps - 1) / kRowWarps, most = (long long)kSms * (fit < kLossBlocksPerSm ? fit : kLossBlocksPerSm);
    *blocks = (int)(want < most ? want : most);
    launch(logprob_warp_rows_kernel<T, V, NV, SHIFT, MODE>, dim3(*blocks), dim3(kRowWarps * 32), 0, LaunchStream{st, true}, a);
    return launched();
}
template <class T, bool SHIFT, int MODE, int TH, bool FIN> int run_block_rows(const LpArgs& a, int cluster, int share, bool dz_vec, int* blocks, cudaStream_t st)
{
    auto kernel = logprob_block_rows_kernel<T, SHIFT, MODE, TH, FIN>;
    const int threads = TH + (FIN ? 32 : 0), stage = share * 16;
    const RowRing shape = row_ring(resident<logprob_block_rows_kernel<T, SHIFT, MODE, TH, FIN>>(threads, 0), stage, MODE == kLoss);
    const int fit = shape.blocks;
    int stages = shape.stages;
    const size_t ring = (size_t)stages * stage;
    long long slots = (long long)kSms * fit;
    if (cluster > 1) {
        // a cluster stays within a GPC, whose SMs it need not divide: clusters that are not held at once would run after the others, each
        // with as many rows (399 bf16 rows of 84120 classes and their gradient: 146 us with 148 / 4 clusters, 99 with those that fit, both with two
        // barriers a row; 85 now)
        static std::atomic<int> held[5][33];
        std::atomic<int>& at = held[31 - __builtin_clz(cluster)][fit];
        if (at.load(std::memory_order_relaxed) == 0) {
            cudaLaunchAttribute dim{};
            dim.id = cudaLaunchAttributeClusterDimension;
            dim.val.clusterDim.x = cluster; dim.val.clusterDim.y = dim.val.clusterDim.z = 1;
            cudaLaunchConfig_t ask{};
            ask.gridDim = dim3(cluster); ask.blockDim = dim3(threads); ask.dynamicSmemBytes = ring; ask.attrs = &dim; ask.numAttrs = 1;
            int n = 0;
            if (!allow_smem(kernel, ring, kRingBytes) ||
                (cluster > 8 && cudaFuncSetAttribute(kernel, cudaFuncAttributeNonPortableClusterSizeAllowed, 1) != cudaSuccess) ||
                cudaOccupancyMaxActiveClusters(&n, kernel, &ask) != cudaSuccess || n < 1) return refused();
            at.store(n, std::memory_order_relaxed);
        }
        slots = at.load(std::memory_order_relaxed);
    }
    const long long each = (a.rows + slots - 1) / slots;      // rows of a block: no more stages than that
    if (stages > each) stages = (int)each;
    const size_t smem = (size_t)stages * stage;
    *blocks = (int)(a.rows < slots ? a.rows : slots) * cluster;
    cudaLaunchAttribute at[2] = {};
    at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at[0].val.programmaticStreamSerializationAllowed = 1;
    at[1].id = cudaLaunchAttributeClusterDimension;
    at[1].val.clusterDim.x = cluster; at[1].val.clusterDim.y = at[1].val.clusterDim.z = 1;
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = dim3(*blocks); cfg.blockDim = dim3(threads); cfg.dynamicSmemBytes = smem; cfg.stream = st;
    cfg.attrs = at; cfg.numAttrs = cluster > 1 ? 2 : 1;
    if (!allow_smem(kernel, smem, kRingBytes) ||
        (cluster > 8 && cudaFuncSetAttribute(kernel, cudaFuncAttributeNonPortableClusterSizeAllowed, 1) != cudaSuccess)) return refused();
    if (cudaLaunchKernelEx(&cfg, kernel, a, cluster, share * (int)(16 / sizeof(T)), stages, dz_vec) != cudaSuccess) return refused();
    return launched();
}
// A cluster shares a row that is longer than a stage, or that few rows leave to few blocks; rows of up to 16 KB take 128 threads.
template <class T, bool SHIFT, int MODE> int pick_block_rows(const LpArgs& a, bool dz_vec, int* blocks, cudaStream_t st)
{
    constexpr int V = 16 / sizeof(T);
    const int vecs = (a.c + (SHIFT ? V - 1 : 0) + V - 1) / V;
    int cluster = 1;
    auto share = [&] { return (vecs + cluster - 1) / cluster; };
    while (share() * 16 > kStageMost) cluster *= 2;
    while (cluster < 16 && a.rows * cluster * 2 <= kSms && share() > 512) cluster *= 2;
    constexpr bool kFin = MODE == kStats;
    if constexpr (MODE == kStats) {
        // a warp a row from 8 rows an SM on, and from 3 on where a row would take a cluster (us with 8 best classes, warps against
        // blocks: bf16 1200 rows of 16000 21 against 30, f32 1200 of 5000 13 against 20, f16 1200 of 32000 42 against 40, bf16 1000 of
        // 32000 37 against 33; against clusters: 900 of 50000 54 against 89, f32 600 of 120000 208 against 266, 300 of them 200 against 136).
        // (Near 8 rows an SM the rule is up to 5 % on the slower side, as for the f16 rows above.)
        if (a.rows >= (cluster > 1 ? 3 : 8) * kSms) {
            const int fit = resident<logprob_stream_rows_kernel<T, SHIFT>>(kStreamWarps * 32, 0);
            const long long want = (a.rows + kStreamWarps - 1) / kStreamWarps, most = (long long)kSms * fit;
            *blocks = (int)(want < most ? want : most);
            launch(logprob_stream_rows_kernel<T, SHIFT>, dim3(*blocks), dim3(kStreamWarps * 32), 0, LaunchStream{st, true}, a);
            return launched();
        }
    }
    if (cluster > 1) return run_block_rows<T, SHIFT, MODE, 512, false>(a, cluster, share(), dz_vec, blocks, st);
    if (share() <= 1024) return run_block_rows<T, SHIFT, MODE, 128, kFin>(a, 1, share(), dz_vec, blocks, st);
    return run_block_rows<T, SHIFT, MODE, 512, kFin>(a, 1, share(), dz_vec, blocks, st);
}

// Warps hold rows of up to 1024 classes (2048 of 16 bits), blocks longer ones.  A thread has 1, 2, 4 or 8 vectors: with 1 and 8 alone
// 16037 bf16 rows of 479 classes and their 5 best took 41 us, with 2 vectors they take 21.
template <class T, int MODE> int rows(const LpArgs& a, int* blocks, cudaStream_t st)
{
    constexpr int V = 16 / sizeof(T);
    const bool one = a.rows == 1;
    const bool grid = aligned(a.z, 16) && (one || a.z_stride % V == 0);
    const bool same = !a.dz || (((reinterpret_cast<uintptr_t>(a.z) ^ reinterpret_cast<uintptr_t>(a.dz)) & 15) == 0 &&
                                (one || (a.z_stride - a.dz_stride) % V == 0));
    const int vecs = (a.c + (grid ? 0 : V - 1) + V - 1) / V;
    if (vecs > 32 * 8) return grid ? pick_block_rows<T, false, MODE>(a, same, blocks, st) : pick_block_rows<T, true, MODE>(a, same, blocks, st);
    if (!same) return a.c <= 32 * 8 ? run_warp_rows<T, 1, 8, false, MODE>(a, blocks, st) : a.c <= 32 * 32 ? run_warp_rows<T, 1, 32, false, MODE>(a, blocks, st)
                                                                                         : run_warp_rows<T, 1, 64, false, MODE>(a, blocks, st);
#define GO(SHIFT)                                                                              \
    do {                                                                                       \
        if (V == 8 && vecs <= 32) return run_warp_rows<T, V, 1, SHIFT, MODE>(a, blocks, st);   \
        if (vecs <= 32 * 2) return run_warp_rows<T, V, 2, SHIFT, MODE>(a, blocks, st);         \
        if (vecs <= 32 * 4) return run_warp_rows<T, V, 4, SHIFT, MODE>(a, blocks, st);         \
        return run_warp_rows<T, V, 8, SHIFT, MODE>(a, blocks, st);                             \
    } while (0)
    if (grid) GO(false);
    GO(true);
#undef GO
}

// Warps that share a tile's classes, and classes of each: the fewest warps of up to 32 classes; 16 warps and any number of classes beyond.
template <class T, int V, int MODE, bool TOP> int run_map(const LpArgs& a, int* blocks, cudaStream_t st)
{
    const long long tiles = (a.p + 32 * V - 1) / (32 * V), all = a.n * tiles;
    int share = 1;
    while (share < kMapWarps && (a.c + share - 1) / share > 32) share *= 2;
    const int per = (a.c + share - 1) / share, warps = share > 1 ? share : 4, groups = warps / share;
    const LaunchStream ls{st, true};
#define GO(...)                                                                                                                              \
    do {                                                                                                                                     \
        const int fit = resident<__VA_ARGS__>(warps * 32, 0);                                                                                \
        const long long want = (all + groups - 1) / groups, most = (long long)kSms * (fit < kLossBlocksPerSm ? fit : kLossBlocksPerSm);                                    \
        *blocks = (int)(want < most ? want : most);                                                                                          \
        launch(__VA_ARGS__, dim3(*blocks), dim3(warps * 32), 0, ls, a, share, per, (int)tiles);                                              \
        return launched();                                                                                                                   \
    } while (0)
    if (warps <= 4) {
        if (per <= 8) GO(logprob_map_kernel<T, V, 8, MODE, TOP, 4>);
        if (per <= 24) GO(logprob_map_kernel<T, V, 24, MODE, TOP, 4>);
        GO(logprob_map_kernel<T, V, 32, MODE, TOP, 4>);
    }
    if (per <= 32) GO(logprob_map_kernel<T, V, 32, MODE, TOP, kMapWarps>);
    GO(logprob_map_kernel<T, V, 0, MODE, TOP, kMapWarps>);
#undef GO
}

template <class T> bool map_vector(const LpArgs& a, int v)
{
    if (v == 1) return true;
    auto fits = [&](const void* p, long long stride) { return !p || (aligned(p, v * sizeof(T)) && (a.n == 1 || stride % v == 0)); };
    return a.p % v == 0 && fits(a.z, a.z_stride) && fits(a.dz, a.dz_stride);
}

template <class T, int MODE> int forward(const LpArgs& a, int* blocks, cudaStream_t st)
{
    if (a.p == 1) return rows<T, MODE>(a, blocks, st);
    if constexpr (MODE == kStats)
        if (a.top > 0) return run_map<T, 1, MODE, true>(a, blocks, st);
    constexpr int V = 4 / sizeof(T);
    if (map_vector<T>(a, V)) return run_map<T, V, MODE, false>(a, blocks, st);
    return run_map<T, 1, MODE, false>(a, blocks, st);
}
template <int MODE> int forward(int type, const LpArgs& a, int* blocks, cudaStream_t st)
{
    if (type == FTP_TYPE_F32) return forward<float, MODE>(a, blocks, st);
    if (type == FTP_TYPE_BF16) return forward<__nv_bfloat16, MODE>(a, blocks, st);
    return forward<__half, MODE>(a, blocks, st);
}

template <class T, int V, bool SHIFT> int bwd_rows(const LpArgs& a, LaunchStream ls)
{
    const long long width = a.c + (SHIFT ? V - 1 : 0), segments = (width + 128 * V - 1) / (128 * V);
    const long long want = (a.rows * segments + 7) / 8, most = 8LL * kSms;
    launch(logprob_bwd_rows_kernel<T, V, SHIFT>, dim3((unsigned)(want < most ? want : most)), dim3(256), 0, ls, a, (int)segments);
    return launched();
}
template <class T, int V> int bwd_map(const LpArgs& a, LaunchStream ls)
{
    const long long tiles = (a.p + 32 * V - 1) / (32 * V), slabs = (a.c + 15) / 16;
    const long long want = (a.n * tiles + 7) / 8, most = (8LL * kSms + slabs - 1) / slabs;
    launch(logprob_bwd_map_kernel<T, V>, dim3((unsigned)(want < most ? want : most), (unsigned)slabs), dim3(256), 0, ls, a, (int)tiles);
    return launched();
}
template <class T> int backward(const LpArgs& a, LaunchStream ls)
{
    constexpr int V = 16 / sizeof(T);
    if (a.p > 1) return map_vector<T>(a, V) ? bwd_map<T, V>(a, ls) : bwd_map<T, 1>(a, ls);
    const bool one = a.rows == 1;
    const bool same = ((reinterpret_cast<uintptr_t>(a.z) ^ reinterpret_cast<uintptr_t>(a.dz)) & 15) == 0 &&
                      (one || (a.z_stride - a.dz_stride) % V == 0);
    if (!same) return bwd_rows<T, 1, false>(a, ls);
    if (aligned(a.z, 16) && (one || a.z_stride % V == 0)) return bwd_rows<T, V, false>(a, ls);
    return bwd_rows<T, V, true>(a, ls);
}

int check_classes(const ftp_dims* d, long long* rows)
{
    const int rc = check_dims(d, rows);
    return rc != FTP_OK ? rc : d->c > FTP_CLASSES_MAX ? FTP_ERR_TOO_LARGE : FTP_OK;
}

constexpr size_t kLossWorkspace = (size_t)kMostBlocks * 4 + (size_t)kMostCounts * 4;

}  // namespace

extern "C" {

int ftp_logprob(const ftp_dims* d, const void* logits, long long logits_stride, const long long* labels,
                float* logp, float* lse, float* entropy, int top, float* top_logp, long long* top_index, void* stream)
{
    long long rows = 0;
    const int rc = check_classes(d, &rows);
    if (rc != FTP_OK) return rc;
    if (top < 0 || top > FTP_TOP_MAX || top > d->c) return FTP_ERR_ARG;
    if (rows == 0) return FTP_OK;
    if ((top > 0) != (top_logp || top_index) || (!logp && !lse && !entropy && !top)) return FTP_ERR_ARG;
    if (!logits || !aligned(logits, type_size(d->type)) || !fix_stride(d, &logits_stride) || (logp && !labels)) return FTP_ERR_ARG;
    if (!aligned(labels, 8) || !aligned(logp, 4) || !aligned(lse, 4) || !aligned(entropy, 4) || !aligned(top_logp, 4) || !aligned(top_index, 8))
        return FTP_ERR_ARG;
    LpArgs a{};
    a.z = logits; a.z_stride = logits_stride; a.labels = logp ? labels : nullptr;
    a.logp = logp; a.lse = lse; a.entropy = entropy; a.top = top; a.top_logp = top_logp; a.top_index = top_index;
    a.n = d->n; a.rows = rows; a.c = (int)d->c; a.p = (int)d->p;
    int blocks = 0;
    return forward<kStats>(d->type, a, &blocks, static_cast<cudaStream_t>(stream));
}

int ftp_logprob_backward(const ftp_dims* d, const void* logits, long long logits_stride, const long long* labels,
                         const float* lse, const float* entropy, const float* dlogp, const float* dentropy,
                         void* dlogits, long long dlogits_stride, void* stream)
{
    long long rows = 0;
    const int rc = check_classes(d, &rows);
    if (rc != FTP_OK) return rc;
    if (rows == 0) return FTP_OK;
    if (!logits || !dlogits || !lse || (dlogp && !labels) || (dentropy && !entropy)) return FTP_ERR_ARG;
    const size_t size = type_size(d->type);
    if (!aligned(logits, size) || !aligned(dlogits, size) || !fix_stride(d, &logits_stride) || !fix_stride(d, &dlogits_stride)) return FTP_ERR_ARG;
    if (!aligned(labels, 8) || !aligned(lse, 4) || !aligned(entropy, 4) || !aligned(dlogp, 4) || !aligned(dentropy, 4)) return FTP_ERR_ARG;
    LpArgs a{};
    a.z = logits; a.z_stride = logits_stride; a.dz = dlogits; a.dz_stride = dlogits_stride; a.labels = dlogp ? labels : nullptr;
    a.lse_in = lse; a.entropy_in = entropy; a.dlogp = dlogp; a.dentropy = dentropy;
    a.n = d->n; a.rows = rows; a.c = (int)d->c; a.p = (int)d->p;
    const LaunchStream ls{static_cast<cudaStream_t>(stream), true};
    if (d->type == FTP_TYPE_F32) return backward<float>(a, ls);
    if (d->type == FTP_TYPE_BF16) return backward<__nv_bfloat16>(a, ls);
    return backward<__half>(a, ls);
}

int ftp_loss_logprob_workspace(const ftp_dims* d, size_t* bytes)
{
    long long rows = 0;
    const int rc = check_classes(d, &rows);
    if (rc != FTP_OK) return rc;
    if (!bytes) return FTP_ERR_ARG;
    *bytes = kLossWorkspace;
    return FTP_OK;
}

int ftp_loss_logprob(const ftp_dims* d, const void* logits, long long logits_stride, const long long* labels, float scale,
                     void* dlogits, long long dlogits_stride, float* loss_out, void* workspace, size_t workspace_bytes,
                     void* stream)
{
    long long rows = 0;
    const int rc = check_classes(d, &rows);
    if (rc != FTP_OK) return rc;
    if (rows >= (1LL << 31)) return FTP_ERR_TOO_LARGE;
    if ((rows > 0 && !dlogits && !loss_out) || !(scale >= -3.0e38f && scale <= 3.0e38f) || !aligned(loss_out, 4)) return FTP_ERR_ARG;
    if (!workspace || !aligned(workspace, 16) || workspace_bytes < kLossWorkspace) return FTP_ERR_ARG;
    const cudaStream_t st = static_cast<cudaStream_t>(stream);
    if (rows == 0) return !loss_out || cudaMemsetAsync(loss_out, 0, 4, st) == cudaSuccess ? FTP_OK : refused();
    const size_t size = type_size(d->type);
    if (!logits || !labels || !aligned(logits, size) || !aligned(dlogits, size) || !aligned(labels, 8)) return FTP_ERR_ARG;
    if (!fix_stride(d, &logits_stride) || (dlogits && !fix_stride(d, &dlogits_stride))) return FTP_ERR_ARG;
    LpArgs a{};
    a.z = logits; a.z_stride = logits_stride; a.dz = dlogits; a.dz_stride = dlogits ? dlogits_stride : 0; a.labels = labels;
    a.scale = scale; a.n = d->n; a.rows = rows; a.c = (int)d->c; a.p = (int)d->p;
    a.sums = loss_out ? static_cast<float*>(workspace) : nullptr;
    const LaunchStream ls{st, true};
    if (rows > kCountHere) {
        int* counts = reinterpret_cast<int*>(static_cast<float*>(workspace) + kMostBlocks);
        const long long want = (rows + 2047) / 2048;
        a.n_counts = (int)(want < kMostCounts ? want : kMostCounts);
        launch(count_labels_kernel, dim3(a.n_counts), dim3(256), 0, ls, labels, rows, counts);
        a.counts = counts;
    }
    int blocks = 0;
    const int rf = forward<kLoss>(d->type, a, &blocks, st);
    if (rf != FTP_OK || !loss_out) return rf;
    launch(loss_finish_kernel, dim3(1), dim3(512), 0, ls, a, blocks, loss_out);
    return launched();
}

}  // extern "C"
