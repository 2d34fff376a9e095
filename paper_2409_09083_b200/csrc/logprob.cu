// Log probabilities of class labels, their entropy and best classes, the gradient, and the loss made of them (ftp_logprob,
// ftp_logprob_backward, ftp_loss_logprob).
//
// Logits are read once: a row stays in the registers of a warp (short rows), of a block, or of a cluster of up to 16 blocks that
// exchange their parts through distributed shared memory.  With the row's maximum m the sums are s = sum 2^a and t = sum a 2^a,
// a = (z - m) log2 e, and lse = m + log s, entropy = log s - (t / s) log 2.
//
// The best classes come without sorting: a row is cut into 32 parts, and the top-th largest of the parts' maxima is a
// bound that at least `top` values reach and few more do (for 8 of 32 parts about 9).  Those are collected in shared memory and
// each finds its own place by counting the better ones.  Where equal values overflow the list, the places are found one by one.
// A value and its class make one 64-bit key whose order is descending value, then ascending class.
#include <cooperative_groups.h>

#include "arrays.cuh"

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

template <class T, int V> __device__ __forceinline__ Pack<T, V> load_logits(const T* base, int e, int lo, int hi)
{
    if (e >= lo && e + V <= hi) return load_pack<T, V>(base + e);
    Pack<T, V> r;
#pragma unroll
    for (int j = 0; j < V; ++j) r.v[j] = e + j >= lo && e + j < hi ? base[e + j] : from_f<T>(minus_inf());
    return r;
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
// A group of TPR threads (a warp, or the block) holds a row, or with a cluster its part of one, as NV vectors of V logits a
// thread.  SHIFT as in norm.cu: vectors lie on the 16-byte grid below the row's start.
template <int TPR> struct RowShared {
    static constexpr int kGroups = TPR == 32 ? 8 : 1;
    static constexpr int kList = TPR == 32 ? kListWarp : kListBlock;
    unsigned long long list[kGroups][kList];
    unsigned long long best[kTop];           // a block's own best, for the cluster
    float parts[kParts];
    float bound;
    float red[2][32];
    int count[kGroups];
    unsigned long long round[32];
    Sums sums;
};

// The `top` best of `m` keys in `list`, by counting; write(place, key) for each.
template <int TPR, class F> __device__ __forceinline__ void place(const unsigned long long* list, int m, int top, int t, F write)
{
    for (int i = t; i < m; i += TPR) {
        const unsigned long long k = list[i];
        int better = 0;
        for (int j = 0; j < m; ++j) better += list[j] > k;
        if (better < top) write(better, k);
    }
}

template <class T, int V, int NV, int TPR, bool SHIFT, int MODE>
__global__ void __launch_bounds__(TPR == 32 ? 256 : 512) logprob_rows_kernel(LpArgs a, int cluster, int part)
{
    __shared__ RowShared<TPR> sh;
    previous_launches();
    constexpr int kGroups = RowShared<TPR>::kGroups;
    const int t = threadIdx.x & (TPR - 1), group = threadIdx.x / TPR, lane = threadIdx.x & 31;
    const int rank = TPR == 32 ? 0 : (int)(blockIdx.x % cluster);
    const long long step = (long long)(gridDim.x / cluster) * kGroups;
    float over = 0.f, total = 0.f;
    if (MODE == kLoss) {
        const float k = labelled_rows(a);
        over = k > 0.f ? a.scale / k : 0.f;
    }
    for (long long row0 = (long long)(blockIdx.x / cluster) * kGroups; row0 < a.rows; row0 += step) {
        const long long row = row0 + group;
        if (TPR == 32 && row >= a.rows) break;                   // (a warp of its own: nobody waits for it)
        const T* zr = static_cast<const T*>(a.z) + row * a.z_stride;
        const int o = SHIFT ? (int)((reinterpret_cast<uintptr_t>(zr) / sizeof(T)) & (V - 1)) : 0;
        const int hi = o + a.c, first = rank * part, last = min(hi, first + part);
        Label label{-1, 0.f, 0};
        label = read_label<T>(a, row, zr, 1);
        zr -= o;
        Pack<T, V> raw[NV];
        float big = minus_inf();
#pragma unroll
        for (int i = 0; i < NV; ++i) raw[i] = load_logits<T, V>(zr, first + (i * TPR + t) * V, o, last);
#pragma unroll
        for (int i = 0; i < NV; ++i)
#pragma unroll
            for (int j = 0; j < V; ++j) big = fmaxf(big, to_f(raw[i].v[j]));
        // the row's maximum, and the parts' ones
        float part_max = big, m;
        if (TPR == 32) m = lanes_max(big, 32);
        else {
            part_max = lanes_max(big, TPR / kParts);
            if (t % (TPR / kParts) == 0) sh.parts[t / (TPR / kParts)] = part_max;
            if (t == 0) sh.count[0] = 0;
            __syncthreads();
            part_max = sh.parts[lane];
            m = lanes_max(part_max, 32);
        }
        if (TPR == 32) {
            if (lane == 0) sh.count[group] = 0;
            __syncwarp();
        }
        float bound = minus_inf();
        const bool want_top = MODE == kStats && a.top > 0;
        if (want_top && (TPR == 32 || t < 32)) {
            int better = 0;
#pragma unroll
            for (int i = 0; i < 32; ++i) {
                const float v = __shfl_sync(0xffffffffu, part_max, i);
                better += v > part_max || (v == part_max && i < lane);
            }
            const unsigned who = __ballot_sync(0xffffffffu, better == a.top - 1);
            bound = __shfl_sync(0xffffffffu, part_max, __ffs(who) - 1);
            if (TPR != 32 && t == 0) sh.bound = bound;
        }
        const float shift = m == minus_inf() ? 0.f : m;
        float s = 0.f, tt = 0.f;
#pragma unroll
        for (int i = 0; i < NV; ++i)
#pragma unroll
            for (int j = 0; j < V; ++j) {
                const float x = max_nan(exponent_of(to_f(raw[i].v[j]), shift), kLeast), e = ex2(x);
                s += e;
                if (MODE == kStats) tt = fmaf(e, x, tt);
            }
        s = lanes_sum(s, 32);
        if (MODE == kStats) tt = lanes_sum(tt, 32);
        if (TPR != 32) {
            if (lane == 0) { sh.red[0][t >> 5] = s; sh.red[1][t >> 5] = tt; }
            __syncthreads();
            s = lanes_sum(lane < TPR / 32 ? sh.red[0][lane] : 0.f, 32);
            if (MODE == kStats) tt = lanes_sum(lane < TPR / 32 ? sh.red[1][lane] : 0.f, 32);
            bound = sh.bound;
        }
        Sums sums{shift, s, tt};
        // the best classes of this part
        int found = 0;
        if (want_top) {
            if (big >= bound) {
#pragma unroll
                for (int i = 0; i < NV; ++i) {
                    const int e = first + (i * TPR + t) * V;
#pragma unroll
                    for (int j = 0; j < V; ++j) {
                        const float v = fmaxf(to_f(raw[i].v[j]), minus_inf());
                        if (v >= bound && e + j >= o && e + j < last) {
                            const int at = atomicAdd(&sh.count[group], 1);
                            if (at < RowShared<TPR>::kList) sh.list[group][at] = key_of(v, e + j - o);
                        }
                    }
                }
            }
            if (TPR == 32) __syncwarp(); else __syncthreads();
            found = sh.count[group];
            if (found > RowShared<TPR>::kList) {                  // too many equal ones: one place after the other
                unsigned long long before = ~0ull;
                const int places = min(a.top, found);
                for (int k = 0; k < places; ++k) {
                    unsigned long long mine = 0;
#pragma unroll
                    for (int i = 0; i < NV; ++i) {
                        const int e = first + (i * TPR + t) * V;
#pragma unroll
                        for (int j = 0; j < V; ++j) {
                            const unsigned long long key = e + j >= o && e + j < last ? key_of(to_f(raw[i].v[j]), e + j - o) : 0ull;
                            if (key < before && key > mine) mine = key;
                        }
                    }
                    mine = lanes_best(mine, 32);
                    if (TPR != 32) {
                        __syncthreads();
                        if (lane == 0) sh.round[t >> 5] = mine;
                        __syncthreads();
                        mine = lanes_best(lane < TPR / 32 ? sh.round[lane] : 0ull, 32);
                    }
                    before = mine;
                    if (t == 0) sh.list[group][k] = mine;
                }
                found = places;
                if (TPR == 32) __syncwarp(); else __syncthreads();
            }
        }
        if (TPR != 32 && cluster > 1) {
            cg::cluster_group cl = cg::this_cluster();
            if (want_top) {
                if (t < kTop) sh.best[t] = 0;
                __syncthreads();
                place<TPR>(sh.list[0], found, a.top, t, [&](int at, unsigned long long k) { sh.best[at] = k; });
            }
            if (t == 0) sh.sums = sums;
            cl.sync();
            sums = *cl.map_shared_rank(&sh.sums, 0);
            for (int r = 1; r < cluster; ++r) sums = join(sums, *cl.map_shared_rank(&sh.sums, r));
            if (want_top && rank == 0) {
                found = cluster * a.top;
                for (int i = t; i < found; i += TPR) sh.list[0][i] = cl.map_shared_rank(sh.best, i / a.top)[i % a.top];
                __syncthreads();
            }
        }
        const RowResult r = result_of(sums);
        if (MODE == kStats && rank == 0) {
            if (t == 0) write_stats(a, row, r, label);
            if (want_top)
                place<TPR>(sh.list[group], found, a.top, t, [&](int at, unsigned long long k) {
                    if (a.top_logp) a.top_logp[row * a.top + at] = logp_of(r, value_of(k));
                    if (a.top_index) a.top_index[row * a.top + at] = class_of(k);
                });
        }
        if (MODE == kLoss) {
            if (t == 0 && rank == 0 && label.has) total += logp_of_label(r, label);
            if (a.dz) {
                T* dr = static_cast<T*>(a.dz) + row * a.dz_stride - o;
                const float f = label.has > 0 ? (r.empty ? 0.f : over) : label.has == 0 ? 0.f : nan_f();
                const float g = f / sums.s;
                const bool nothing = f == 0.f;
                const int at = label.has > 0 ? (int)label.cls + o : -1;
#pragma unroll
                for (int i = 0; i < NV; ++i) {
                    const int e = first + (i * TPR + t) * V;
                    if (e >= last) continue;
                    Pack<T, V> d;
#pragma unroll
                    for (int j = 0; j < V; ++j) {
                        const float x = ex2(exponent_of(to_f(raw[i].v[j]), sums.m)) * g;
                        d.v[j] = from_f<T>(nothing ? 0.f : e + j == at ? x - f : x);
                    }
                    store_part<T, V>(dr, e, o, last, d);
                }
            }
        }
        if (TPR != 32) {                                  // before the next row's values take the places of these
            if (cluster > 1) cg::this_cluster().sync();
            else __syncthreads();
        } else __syncwarp();
    }
    if (MODE == kLoss && a.sums) {
        __shared__ float red[8];
        if (TPR == 32) {
            if (lane == 0) red[group] = total;
            __syncthreads();
            if (threadIdx.x == 0) {
                float s = 0.f;
                for (int i = 0; i < kGroups; ++i) s += red[i];
                a.sums[blockIdx.x] = s;
            }
        } else if (t == 0) a.sums[blockIdx.x] = total;
    }
}

// ---- maps -------------------------------------------------------------------------------------------------------
// Tiles as in norm.cu: lp lanes of V pixels each, channels shared out to groups, CPT of them in a thread's registers (0: any number,
// read again for each pass).  TOP: the best classes, found one after the other.
template <class T, int V, int CPT, int MODE, bool TOP>
__global__ void __launch_bounds__(256) logprob_map_kernel(LpArgs a, int lp, int tiles)
{
    constexpr int kWarps = 8;
    __shared__ float red[2][kWarps * 32 * V];
    __shared__ unsigned long long round[2][TOP ? kWarps * 32 : 1];
    previous_launches();
    const int l = threadIdx.x & (lp - 1), g = threadIdx.x / lp, groups = blockDim.x / lp, lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int slots = CPT ? CPT : (a.c + groups - 1) / groups;
    float over = 0.f, total = 0.f;
    if (MODE == kLoss) {
        const float k = labelled_rows(a);
        over = k > 0.f ? a.scale / k : 0.f;
    }
    for (long long tile = blockIdx.x; tile < a.n * tiles; tile += gridDim.x) {
        const long long n = tile / tiles;
        const int px = (int)(tile - n * tiles) * lp * V + l * V;
        const bool live = px < a.p;
        const long long row = n * a.p + px;
        const T* zt = static_cast<const T*>(a.z) + n * a.z_stride + px;
        auto load = [&](int i) {
            const int ch = g + i * groups;
            if (live && ch < a.c) return load_pack<T, V>(zt + (long long)ch * a.p);
            Pack<T, V> r;
#pragma unroll
            for (int j = 0; j < V; ++j) r.v[j] = from_f<T>(minus_inf());
            return r;
        };
        Pack<T, V> raw[CPT ? CPT : 1];
        if constexpr (CPT > 0) {
#pragma unroll
            for (int i = 0; i < CPT; ++i) raw[i] = load(i);
        }
        Label label[V];
        if (live && (MODE == kLoss || g == 0)) {
#pragma unroll
            for (int j = 0; j < V; ++j) label[j] = read_label<T>(a, row + j, zt + j, a.p);
        }
        auto each = [&](auto f) {
            if constexpr (CPT > 0) {
#pragma unroll
                for (int i = 0; i < CPT; ++i) f(raw[i], i);
            } else
                for (int i = 0; i < slots; ++i) f(load(i), i);
        };
        float m[V], s[V], t[V];
#pragma unroll
        for (int j = 0; j < V; ++j) { m[j] = minus_inf(); s[j] = t[j] = 0.f; }
        each([&](const Pack<T, V>& r, int) {
#pragma unroll
            for (int j = 0; j < V; ++j) m[j] = fmaxf(m[j], to_f(r.v[j]));
        });
#pragma unroll
        for (int j = 0; j < V; ++j)
            for (int d = 16; d >= lp; d >>= 1) m[j] = fmaxf(m[j], __shfl_xor_sync(0xffffffffu, m[j], d));
        if (lane < lp) {
#pragma unroll
            for (int j = 0; j < V; ++j) red[0][(warp * V + j) * lp + lane] = m[j];
        }
        __syncthreads();
#pragma unroll
        for (int j = 0; j < V; ++j) {
            m[j] = minus_inf();
#pragma unroll
            for (int w = 0; w < kWarps; ++w) m[j] = fmaxf(m[j], red[0][(w * V + j) * lp + (lane & (lp - 1))]);
            if (m[j] == minus_inf()) m[j] = 0.f;
        }
        each([&](const Pack<T, V>& r, int) {
#pragma unroll
            for (int j = 0; j < V; ++j) {
                const float x = max_nan(exponent_of(to_f(r.v[j]), m[j]), kLeast), e = ex2(x);
                s[j] += e;
                if (MODE == kStats) t[j] = fmaf(e, x, t[j]);
            }
        });
        // sums over the channels; the second buffer, then the first again, which all threads have read by the barrier in between
        auto sum_up = [&](float (&v)[V], float* buffer) {
#pragma unroll
            for (int j = 0; j < V; ++j)
                for (int d = 16; d >= lp; d >>= 1) v[j] += __shfl_xor_sync(0xffffffffu, v[j], d);
            if (lane < lp) {
#pragma unroll
                for (int j = 0; j < V; ++j) buffer[(warp * V + j) * lp + lane] = v[j];
            }
            __syncthreads();
#pragma unroll
            for (int j = 0; j < V; ++j) {
                v[j] = 0.f;
#pragma unroll
                for (int w = 0; w < kWarps; ++w) v[j] += buffer[(w * V + j) * lp + (lane & (lp - 1))];
            }
        };
        sum_up(s, red[1]);
        if (MODE == kStats) sum_up(t, red[0]);
        RowResult r[V];
#pragma unroll
        for (int j = 0; j < V; ++j) r[j] = result_of(Sums{m[j], s[j], t[j]});
        if (MODE == kStats && live && g == 0) {
#pragma unroll
            for (int j = 0; j < V; ++j) write_stats(a, row + j, r[j], label[j]);
        }
        if constexpr (TOP) {
            unsigned long long before = ~0ull;
            for (int k = 0; k < a.top; ++k) {
                unsigned long long mine = 0;
                each([&](const Pack<T, V>& q, int i) {
                    const int ch = g + i * groups;
                    const unsigned long long key = ch < a.c ? key_of(to_f(q.v[0]), ch) : 0ull;
                    if (key < before && key > mine) mine = key;
                });
                for (int d = 16; d >= lp; d >>= 1) {
                    const unsigned long long u = __shfl_xor_sync(0xffffffffu, mine, d);
                    if (u > mine) mine = u;
                }
                if (lane < lp) round[k & 1][warp * lp + lane] = mine;
                __syncthreads();
                mine = 0;
#pragma unroll
                for (int w = 0; w < kWarps; ++w) {
                    const unsigned long long u = round[k & 1][w * lp + (lane & (lp - 1))];
                    if (u > mine) mine = u;
                }
                before = mine;
                if (live && g == 0) {
                    const long long at = (n * a.top + k) * a.p + px;
                    if (a.top_logp) a.top_logp[at] = logp_of(r[0], value_of(mine));
                    if (a.top_index) a.top_index[at] = class_of(mine);
                }
            }
        }
        if (MODE == kLoss) {
            float f[V], gr[V];
            if (live) {
#pragma unroll
                for (int j = 0; j < V; ++j) {
                    f[j] = label[j].has > 0 ? (r[j].empty ? 0.f : over) : label[j].has == 0 ? 0.f : nan_f();
                    gr[j] = f[j] / s[j];
                    if (g == 0 && label[j].has) total += logp_of_label(r[j], label[j]);
                }
                if (a.dz) {
                    T* dt = static_cast<T*>(a.dz) + n * a.dz_stride + px;
                    each([&](const Pack<T, V>& q, int i) {
                        const int ch = g + i * groups;
                        if (ch >= a.c) return;
                        Pack<T, V> d;
#pragma unroll
                        for (int j = 0; j < V; ++j) {
                            const float x = ex2(exponent_of(to_f(q.v[j]), m[j])) * gr[j];
                            d.v[j] = from_f<T>(f[j] == 0.f ? 0.f : ch == label[j].cls ? x - f[j] : x);
                        }
                        store_pack<T, V>(dt + (long long)ch * a.p, d);
                    });
                }
            }
        }
        __syncthreads();
    }
    if (MODE == kLoss && a.sums) {
        total = lanes_sum(total, 32);
        __syncthreads();
        if (lane == 0) red[0][warp] = total;
        __syncthreads();
        if (threadIdx.x == 0) {
            float sum = 0.f;
            for (int w = 0; w < kWarps; ++w) sum += red[0][w];
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
// What a row's classes share: dlogits = w_l (class = label) - p (w_l + w_h (log p + entropy)).
struct RowGrad { float lse, wl, wh, h; long long cls; bool empty; };
__device__ __forceinline__ RowGrad row_grad(const LpArgs& a, long long row)
{
    RowGrad r;
    r.lse = a.lse_in[row];
    r.cls = a.labels ? a.labels[row] : -1;
    r.wl = a.dlogp && r.cls >= 0 ? a.dlogp[row] : 0.f;
    if (r.cls >= a.c) r.wl = nan_f();
    r.wh = a.dentropy ? a.dentropy[row] : 0.f;
    r.h = a.dentropy ? a.entropy_in[row] : 0.f;
    r.empty = r.lse == minus_inf();
    return r;
}
__device__ __forceinline__ float class_grad(const RowGrad& r, float z, bool hit)
{
    const float lp = max_nan(z - r.lse, -110.f), p = ex2(lp * kLog2e);       // e^-110 is 0 in fp32
    const float d = (hit ? r.wl : 0.f) - p * fmaf(r.wh, lp + r.h, r.wl);
    return r.empty ? 0.f : d;
}

template <class T, int V, bool SHIFT> __global__ void __launch_bounds__(256) logprob_bwd_rows_kernel(LpArgs a, int segments)
{
    previous_launches();
    constexpr int kPer = 4, kSegment = 32 * V * kPer;
    const int lane = threadIdx.x & 31;
    for (long long task = (long long)blockIdx.x * 8 + (threadIdx.x >> 5); task < a.rows * segments; task += (long long)gridDim.x * 8) {
        const long long row = segments == 1 ? task : task / segments;
        const int first = (int)(task - row * segments) * kSegment + lane * V;
        const T* zr = static_cast<const T*>(a.z) + row * a.z_stride;
        const int o = SHIFT ? (int)((reinterpret_cast<uintptr_t>(zr) / sizeof(T)) & (V - 1)) : 0;
        const int hi = o + a.c;
        zr -= o;
        T* dr = static_cast<T*>(a.dz) + row * a.dz_stride - o;
        Pack<T, V> raw[kPer];
#pragma unroll
        for (int i = 0; i < kPer; ++i) raw[i] = load_logits<T, V>(zr, first + i * 32 * V, o, hi);
        const RowGrad r = row_grad(a, row);
        const long long at = r.cls + o;
#pragma unroll
        for (int i = 0; i < kPer; ++i) {
            const int e = first + i * 32 * V;
            if (e >= hi) continue;
            Pack<T, V> d;
#pragma unroll
            for (int j = 0; j < V; ++j) d.v[j] = from_f<T>(class_grad(r, to_f(raw[i].v[j]), r.cls >= 0 && e + j == at));
            store_part<T, V>(dr, e, o, hi, d);
        }
    }
}

template <class T, int V> __global__ void __launch_bounds__(256) logprob_bwd_map_kernel(LpArgs a, int tiles, int slabs)
{
    previous_launches();
    constexpr int kSlab = 16, kAhead = 4;
    const int lane = threadIdx.x & 31;
    for (long long task = (long long)blockIdx.x * 8 + (threadIdx.x >> 5); task < a.n * tiles * slabs; task += (long long)gridDim.x * 8) {
        const long long at = task / slabs, n = at / tiles;
        const int c0 = (int)(task - at * slabs) * kSlab, c1 = min(a.c, c0 + kSlab);
        const int px = (int)(at - n * tiles) * 32 * V + lane * V;
        if (px >= a.p) continue;
        const T* zt = static_cast<const T*>(a.z) + n * a.z_stride + px;
        T* dt = static_cast<T*>(a.dz) + n * a.dz_stride + px;
        RowGrad r[V];
#pragma unroll
        for (int j = 0; j < V; ++j) r[j] = row_grad(a, n * a.p + px + j);
        for (int ch = c0; ch < c1; ch += kAhead) {
            Pack<T, V> raw[kAhead];
#pragma unroll
            for (int i = 0; i < kAhead; ++i)
                if (ch + i < c1) raw[i] = load_pack<T, V>(zt + (long long)(ch + i) * a.p);
#pragma unroll
            for (int i = 0; i < kAhead; ++i) {
                if (ch + i >= c1) continue;
                Pack<T, V> d;
#pragma unroll
                for (int j = 0; j < V; ++j) d.v[j] = from_f<T>(class_grad(r[j], to_f(raw[i].v[j]), ch + i == r[j].cls));
                store_pack<T, V>(dt + (long long)(ch + i) * a.p, d);
            }
        }
    }
}

// ---- host -------------------------------------------------------------------------------------------------------
constexpr int kMostBlocks = 8 * kSms;         // blocks of a loss, each with a sum
constexpr int kMostCounts = 1024;

template <class T, int V, int NV, int TPR, bool SHIFT, int MODE> int run_rows(const LpArgs& a, int cluster, int part, int* blocks, cudaStream_t st)
{
    auto kernel = logprob_rows_kernel<T, V, NV, TPR, SHIFT, MODE>;
    const int threads = TPR == 32 ? 256 : 512, per = TPR == 32 ? 8 : 1;
    const long long want = (a.rows + per - 1) / per, most = (TPR == 32 ? kMostBlocks : 4 * kSms) / cluster;
    *blocks = (int)(want < most ? want : most) * cluster;
    cudaLaunchAttribute at[2] = {};
    at[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at[0].val.programmaticStreamSerializationAllowed = 1;
    at[1].id = cudaLaunchAttributeClusterDimension;
    at[1].val.clusterDim.x = cluster; at[1].val.clusterDim.y = at[1].val.clusterDim.z = 1;
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = dim3(*blocks); cfg.blockDim = dim3(threads); cfg.stream = st;
    cfg.attrs = at; cfg.numAttrs = cluster > 1 ? 2 : 1;
    if (cluster > 8 && cudaFuncSetAttribute(kernel, cudaFuncAttributeNonPortableClusterSizeAllowed, 1) != cudaSuccess) return FTP_ERR_CUDA;
    if (cudaLaunchKernelEx(&cfg, kernel, a, cluster, part) != cudaSuccess) return FTP_ERR_CUDA;
    return launched();
}

// Warps hold rows of up to 1024 classes (2048 of 16 bits); blocks hold parts of up to 16384 classes (32768 of 16 bits), and a cluster shares a
// row that is longer, or that few rows leave to few blocks.
template <class T, int V, bool SHIFT, int MODE> int pick_rows(const LpArgs& a, int* blocks, cudaStream_t st)
{
    const int vecs = (a.c + (SHIFT ? V - 1 : 0) + V - 1) / V;
    constexpr int kSmall = 8 / V ? 8 / V : 1, kMid = V == 8 ? 4 : 32 / V, kWide = V == 8 ? 8 : 32 / V;
    if (vecs <= 32 * kSmall) return run_rows<T, V, kSmall, 32, SHIFT, MODE>(a, 1, vecs * V, blocks, st);
    if (vecs <= 32 * kMid) return run_rows<T, V, kMid, 32, SHIFT, MODE>(a, 1, vecs * V, blocks, st);
    int cluster = 1;
    auto share = [&] { return (vecs + cluster - 1) / cluster; };
    while (share() > 512 * kWide) cluster *= 2;
    while (cluster < 16 && a.rows * cluster * 2 <= 2 * kSms && share() > 512 * kSmall) cluster *= 2;
    if (share() <= 512 * kSmall) return run_rows<T, V, kSmall, 512, SHIFT, MODE>(a, cluster, share() * V, blocks, st);
    if (share() <= 512 * kMid) return run_rows<T, V, kMid, 512, SHIFT, MODE>(a, cluster, share() * V, blocks, st);
    return run_rows<T, V, kWide, 512, SHIFT, MODE>(a, cluster, share() * V, blocks, st);
}

template <class T, int MODE> int rows(const LpArgs& a, int* blocks, cudaStream_t st)
{
    constexpr int V = 16 / sizeof(T);
    const bool one = a.rows == 1;
    const bool grid = aligned(a.z, 16) && (one || a.z_stride % V == 0);
    const bool same = !a.dz || (((reinterpret_cast<uintptr_t>(a.z) ^ reinterpret_cast<uintptr_t>(a.dz)) & 15) == 0 &&
                                (one || (a.z_stride - a.dz_stride) % V == 0));
    if (same) return grid ? pick_rows<T, V, false, MODE>(a, blocks, st) : pick_rows<T, V, true, MODE>(a, blocks, st);
    return pick_rows<T, 1, false, MODE>(a, blocks, st);
}

template <class T, int V, int MODE, bool TOP> int run_map(const LpArgs& a, int* blocks, cudaStream_t st)
{
    int lp = 32;
    auto per = [&] { return (a.c + 256 / lp - 1) / (256 / lp); };
    while (per() > 4 && lp * V > 32) lp >>= 1;
    const long long tiles = (a.p + lp * V - 1) / (lp * V), all = a.n * tiles;
    const LaunchStream ls{st, true};
    auto go = [&](auto kernel, int per_sm) {
        const long long most = (long long)kSms * per_sm;
        *blocks = (int)(all < most ? all : most);
        launch(kernel, dim3(*blocks), dim3(256), 0, ls, a, lp, (int)tiles);
        return launched();
    };
    if (per() <= 1) return go(logprob_map_kernel<T, V, 1, MODE, TOP>, 8);
    if (per() <= 4) return go(logprob_map_kernel<T, V, 4, MODE, TOP>, 4);
    if (per() <= 16) return go(logprob_map_kernel<T, V, 16, MODE, TOP>, 2);
    return go(logprob_map_kernel<T, V, 0, MODE, TOP>, 4);
}

template <class T> bool map_vector(const LpArgs& a, int v)
{
    auto fits = [&](const void* p, long long stride) { return !p || (aligned(p, v * sizeof(T)) && (a.n == 1 || stride % v == 0)); };
    return a.p % v == 0 && fits(a.z, a.z_stride) && fits(a.dz, a.dz_stride);
}

template <class T, int MODE> int forward(const LpArgs& a, int* blocks, cudaStream_t st)
{
    if (a.p == 1) return rows<T, MODE>(a, blocks, st);
    if constexpr (MODE == kStats)
        if (a.top > 0) return run_map<T, 1, MODE, true>(a, blocks, st);
    constexpr int V = 16 / sizeof(T);
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
    const long long want = (a.n * tiles * slabs + 7) / 8, most = 8LL * kSms;
    launch(logprob_bwd_map_kernel<T, V>, dim3((unsigned)(want < most ? want : most)), dim3(256), 0, ls, a, (int)tiles, (int)slabs);
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
    if (rows == 0) return !loss_out || cudaMemsetAsync(loss_out, 0, 4, st) == cudaSuccess ? FTP_OK : FTP_ERR_CUDA;
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
