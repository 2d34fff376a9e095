// Channel norm, forward and backward (ftp_norm_forward, ftp_norm_backward).
//
// Both directions are bound by memory: forward reads x and writes y, backward reads x (or its checkpoint) and dy and writes dx.
// So a row of values is read once and stays in registers between its statistics and its result.  Two layouts: matrices (p = 1), where
// the threads of a group lie along the row, and maps (p > 1), where the lanes of a warp lie along the pixels of a plane and a thread holds
// up to 32 channels of its pixels.
//
// The variance is the mean of (x - mean)^2 over values in registers, not E x^2 - mean^2.  dweight and dbias: a thread (in maps: a lane)
// keeps the same columns for all its rows and sums them in registers; each block writes one partial set and a second launch adds the
// sets in a fixed order.
#include <algorithm>
#include "arrays.cuh"

using namespace ftp;
using namespace ftp::arr;

namespace {

struct NormArgs {
    const void* x;               // backward: null if the values come from the checkpoint
    const void* dy;
    void* out;                   // y or dx
    long long x_stride, dy_stride, out_stride;
    const float* weight;         // null: 1
    const float* bias;           // null: 0
    float* mean;                 // forward: may be null
    float* rstd;
    CkptView ck;
    float* partials;             // backward: [blocks][2][c], null: not wanted
    long long n, rows;           // samples; n * p
    int c, p;
    float eps;
    int w_vec;                   // weight and bias are 16-byte aligned
};

// Adds over the `tpr` threads of a group: a power of two of lanes, or whole warps -- the block, or with a barrier `number` of their own (an SM
// has 64 barriers and a kernel that names them at run time takes 16 a block: for kernels of one
// block an SM).  `red`: K floats a warp, not read or written by anyone else until the group has passed another barrier.
template <int K, bool NAMED = false> __device__ __forceinline__ void group_sum(float (&v)[K], int tpr, int number, float* red)
{
#pragma unroll
    for (int k = 0; k < K; ++k) v[k] = lanes_sum(v[k], tpr);
    if (tpr <= 32) return;
    const int warp = threadIdx.x >> 5, per = tpr >> 5, first = NAMED ? (number - 1) * per : 0;
    if ((threadIdx.x & 31) == 0) {
#pragma unroll
        for (int k = 0; k < K; ++k) red[warp * K + k] = v[k];
    }
    if constexpr (NAMED) group_barrier(number, tpr);
    else __syncthreads();
#pragma unroll
    for (int k = 0; k < K; ++k) v[k] = 0.f;
#pragma unroll 4
    for (int i = 0; i < per; ++i)
#pragma unroll
        for (int k = 0; k < K; ++k) v[k] += red[(first + i) * K + k];
}

// weight or bias of columns [col, col + V) (null: `none`); columns outside [0, c) read as `none`.  FAST: there, whole and aligned.
template <bool FAST, int V> __device__ __forceinline__ void load_cols(const float* w, int col, int c, float none, float* out)
{
    if constexpr (FAST) {
#pragma unroll
        for (int j = 0; j < V; j += 4) {
            const float4 q = __ldg(reinterpret_cast<const float4*>(w + col + j));
            out[j] = q.x; out[j + 1] = q.y; out[j + 2] = q.z; out[j + 3] = q.w;
        }
    } else {
#pragma unroll
        for (int j = 0; j < V; ++j) out[j] = w && (unsigned)(col + j) < (unsigned)c ? __ldg(w + col + j) : none;
    }
}

// x of a row as it is read: packs of the array, or steps of the checkpoint.  hats() gives (x - mean) rstd from rstd and -mean rstd:
// one multiply-add, off by no more than the rounding of mean itself; q (step rstd) is as exact, the step being a power of two.
template <class T, int V, bool CK> struct Raw;
template <class T, int V> struct Raw<T, V, false> {
    Pack<T, V> a;
    __device__ __forceinline__ void clear() { a = zero_pack<T, V>(); }
    __device__ __forceinline__ Vals<V> hats(float rstd, float shift) const { return fma(values(a), all<V>(rstd), all<V>(shift)); }
    __device__ __forceinline__ Vals<V> hats(const Vals<V>& rstd, const Vals<V>& shift) const { return fma(values(a), rstd, shift); }
};
template <class T, int V> struct Raw<T, V, true> {
    Pack<unsigned char, V> q;
    unsigned e;
    __device__ __forceinline__ void clear()
    {
        e = 1;
        q = zero_pack<unsigned char, V>();
    }
    __device__ __forceinline__ Vals<V> hats(float rstd, float shift) const { return fma(steps_of(q), all<V>(rstd * step_of(e)), all<V>(shift)); }
    __device__ __forceinline__ Vals<V> hats(const Vals<V>& rstd, const Vals<V>& shift) const { return fma(steps_of(q), mul(rstd, all<V>(step_of(e))), shift); }
};

// ---- matrices ---------------------------------------------------------------------------------------------------
// A group of `tpr` threads holds a row as VPT vectors of V values a thread: vector i * tpr + t.  FAST: every vector lies in the row as a
// whole, and weight and bias are there and aligned.  SHIFT: rows start at any multiple of the value's size, and the vectors lie on
// the 16-byte grid below the row's start (x and y the same distance above it); then column = place - o.  With V = 1 any alignment goes.
enum { kFast, kEdge, kShift };

// Values wait in registers as they were read and are widened again in each of the three passes: with 8 vectors a thread a warp holds
// 2048 values of 16 bits, and exchanges, barriers and addresses are shared by 64 values of each lane.
template <class T, int V, int VPT, int FORM, bool CK, int MOST>
__global__ void __launch_bounds__(MOST, MOST > 128 ? 1 : 6) norm_fwd_rows_kernel(NormArgs a, int tpr)
{
    constexpr bool kWhole = FORM == kFast || V == 1;
    __shared__ float red[2][16];
    constexpr bool kEdges = CK && FORM == kShift;
    __shared__ __align__(16) Pack<T, V> edge[kEdges ? 2 : 1][kEdges ? 16 : 1][kEdges ? VPT : 1];       // first vectors of the warps, of this row and the one before
    int turn = 0;
    previous_launches();
    const int per = tpr > 32 ? 1 : blockDim.x / tpr, t = threadIdx.x & (tpr - 1), group = tpr > 32 ? 0 : threadIdx.x / tpr;
    const float inv_c = 1.f / (float)a.c;
    const long long step = (long long)gridDim.x * per;
    for (long long row0 = (long long)blockIdx.x * per; row0 < a.rows; row0 += step, turn ^= 1) {
        const long long row = row0 + group;
        const bool live = row < a.rows;
        const T* xr = static_cast<const T*>(a.x) + row * a.x_stride;
        const int o = FORM == kShift ? (int)((reinterpret_cast<uintptr_t>(xr) / sizeof(T)) & (V - 1)) : 0;
        const int hi = live ? o + a.c : 0;
        const Reach<T, V> in = reach<T, V>(xr, o, o + a.c, static_cast<const T*>(a.x), static_cast<const T*>(a.x) + (a.rows - 1) * a.x_stride + a.c);
        xr += t * V - o;
        Pack<T, V> raw[VPT];
#pragma unroll
        for (int i = 0; i < VPT; ++i) {
            const int e = (i * tpr + t) * V;
            raw[i] = zero_pack<T, V>();
            if (kWhole) { if (e < hi) raw[i] = load_pack<T, V>(xr + i * tpr * V); }
            else if (live) load_whole<T, V>(raw[i], xr - t * V, e, in.lo, in.hi);
        }
        if (!kWhole && live) {
            if (!in.all) {
#pragma unroll
                for (int i = 0; i < VPT; ++i) load_rest<T, V>(raw[i], xr - t * V, (i * tpr + t) * V, o, hi);
            }
#pragma unroll
            for (int i = 0; i < VPT; ++i) keep_part<T, V>(raw[i], (i * tpr + t) * V, o, hi, from_f<T>(0.f));
        }
        if constexpr (kEdges) {                                 // (read behind the barriers, or the warp's exchanges, of the sums)
            if ((threadIdx.x & 31) == 0) {
#pragma unroll
                for (int i = 0; i < VPT; ++i) edge[turn][threadIdx.x >> 5][i] = raw[i];
            }
            __syncwarp();
        }
        Vals<V> acc = values(raw[0]);
#pragma unroll
        for (int i = 1; i < VPT; ++i) acc = add(acc, values(raw[i]));
        float s[1] = {sum_of(acc)};
        group_sum<1>(s, tpr, 0, red[0]);
        const float mean = a.c == 1 ? s[0] : s[0] * inv_c;
        acc = all<V>(0.f);
#pragma unroll
        for (int i = 0; i < VPT; ++i) keep_packed(raw[i]);
#pragma unroll
        for (int i = 0; i < VPT; ++i) {
            const int e = (i * tpr + t) * V;
            Vals<V> d = add(values(raw[i]), all<V>(e < hi ? -mean : 0.f));       // (a vector that is not there stays 0)
            if (!kWhole && (e < o || e + V > hi)) {                               // nor places before or behind the row
#pragma unroll
                for (int j = 0; j < V; ++j)
                    if (e + j < o || e + j >= hi) d.v[j] = 0.f;
            }
            acc = fma(d, d, acc);
        }
        s[0] = sum_of(acc);
        group_sum<1>(s, tpr, 0, red[1]);
#pragma unroll
        for (int i = 0; i < VPT; ++i) keep_packed(raw[i]);
        const float rstd = 1.f / sqrtf(s[0] * inv_c + a.eps);
        if (live && t == 0) {
            if (a.mean) a.mean[row] = mean;
            if (a.rstd) a.rstd[row] = rstd;
        }
        T* yr = static_cast<T*>(a.out) + row * a.out_stride + t * V - o;
        unsigned char* qr = a.ck.q + row * a.ck.pitch + t * V;
        unsigned char* er = a.ck.steps + row * a.ck.blocks + t * V / kBlock;
        // The checkpoint first, before y may have been written over x: columns [e, e + V) of the row are places o further on, across a vector
        // of this lane and of the next one, which for the last lane of a warp lies in shared memory.
        if constexpr (CK) {
            auto columns = [&](const Pack<T, V>& mine, int i) {
                if constexpr (FORM == kShift) {
                    Pack<T, V> next = from_next_lane(mine);
                    if ((t & 31) == 31 || t == tpr - 1) {
                        const int w = (t >> 5) + 1, warps = tpr >> 5;          // (the last warp goes on with the first one's next vector)
                        next = zero_pack<T, V>();
                        if (w < warps) next = edge[turn][w][i];
                        else if (i + 1 < VPT && warps > 0) next = edge[turn][tpr > 32 ? 0 : threadIdx.x >> 5][(i + 1) % VPT];
                    }
                    return values(window<T, V>(mine, next, o));
                } else return values(mine);
            };
            bool any = false;
#pragma unroll
            for (int i = 0; i < VPT; ++i) {                         // as if all values were finite
                const int skip = i * tpr * V;
                const Vals<V> k = columns(raw[i], i);
                const float big = largest(k);
                any |= special<T>(big);
                const unsigned ex = step_exponent(big);
                if (live && skip + t * V < a.ck.pitch) {
                    store_pack<unsigned char, V>(qr + skip, to_steps(k, ex));
                    if (t % (kBlock / V) == 0) er[(unsigned)skip / kBlock] = (unsigned char)ex;
                }
            }
            if (__any_sync(0xffffffffu, any)) {                     // the blocks with others once more
#pragma unroll 1
                for (int i = 0; i < VPT; ++i) {
                    const int skip = i * tpr * V, e = skip + t * V;
                    Pack<T, V> again = zero_pack<T, V>();
                    load_whole<T, V>(again, xr - t * V, e, o, hi);
                    load_rest<T, V>(again, xr - t * V, e, o, hi);
                    const Vals<V> k = columns(again, i);
                    if (special<T>(largest(k))) {
                        unsigned ex;
                        const Pack<unsigned char, V> st = to_steps_special<T, V>(k, ex);
                        if (live && e < a.ck.pitch) {
                            store_pack<unsigned char, V>(qr + skip, st);
                            if (t % (kBlock / V) == 0) er[(unsigned)skip / kBlock] = (unsigned char)ex;
                        }
                    }
                    __syncwarp();
                }
            }
        }
#pragma unroll
        for (int i = 0; i < VPT; ++i) keep_packed(raw[i]);
#pragma unroll
        for (int i = 0; i < VPT; ++i) {
            const int skip = i * tpr * V, e = skip + t * V;
            if (e >= hi) continue;
            Vals<V> w, b;
            load_cols<FORM == kFast, V>(a.weight, e - o, a.c, 1.f, w.v);
            load_cols<FORM == kFast, V>(a.bias, e - o, a.c, 0.f, b.v);
            const Pack<T, V> y = rounded<T, V>(fma(mul(add(values(raw[i]), all<V>(-mean)), all<V>(rstd)), w, b));
            if (kWhole) store_pack<T, V>(yr + skip, y);
            else store_part<T, V>(yr - t * V, e, o, hi, y);
        }
    }
}

// Rows longer than a block's registers: three passes over the row, the second and third from L2.
template <class T, bool CK> __global__ void __launch_bounds__(1024) norm_fwd_long_rows_kernel(NormArgs a)
{
    __shared__ float red[2][32];
    previous_launches();
    for (long long row = blockIdx.x; row < a.rows; row += gridDim.x) {
        const T* xr = static_cast<const T*>(a.x) + row * a.x_stride;
        T* yr = static_cast<T*>(a.out) + row * a.out_stride;
        float s[1] = {0.f}, q[1] = {0.f};
        for (int e = threadIdx.x; e < a.c; e += 1024) s[0] += to_f(xr[e]);
        group_sum<1>(s, 1024, 0, red[0]);
        const float mean = s[0] / (float)a.c;
        for (int e = threadIdx.x; e < a.c; e += 1024) { const float d = to_f(xr[e]) - mean; q[0] = fmaf(d, d, q[0]); }
        group_sum<1>(q, 1024, 0, red[1]);
        const float rstd = 1.f / sqrtf(q[0] / (float)a.c + a.eps);
        if (threadIdx.x == 0) {
            if (a.mean) a.mean[row] = mean;
            if (a.rstd) a.rstd[row] = rstd;
        }
        const int end = (a.c + kBlock - 1) / kBlock * kBlock;         // whole warps, for the blocks of a checkpoint
        for (int e = threadIdx.x; e < end; e += 1024) {
            Pack<T, 1> v = zero_pack<T, 1>();
            if (e < a.c) v.set(0, xr[e]);
            if (CK) {
                const float big = largest(values(v));
                unsigned ex = step_exponent(big);
                const Pack<unsigned char, 1> st = special<T>(big) ? to_steps_special<T, 1>(values(v), ex) : to_steps(values(v), ex);
                a.ck.q[row * a.ck.pitch + e] = st.get(0);
                if (e % kBlock == 0) a.ck.steps[row * a.ck.blocks + e / kBlock] = (unsigned char)ex;
            }
            if (e < a.c)
                yr[e] = from_f<T>(fmaf((to_f(v.get(0)) - mean) * rstd, a.weight ? a.weight[e] : 1.f, a.bias ? a.bias[e] : 0.f));
        }
    }
}

// Backward pass of matrices; the same spread of a row over a group, a block's groups (each with a barrier of its own) taking rows in
// turn.  A thread's columns are the same in every row, so dweight and dbias of its columns add up in registers over all rows of the block.
// SHIFT keeps that true for rows off the 16-byte grid: a group's rows are a multiple of V rows apart, so that all of them start the
// same distance o behind the grid, and place e is column e - o in each.
// The next row's values are on their way while a row is summed: with one block of 512 threads an SM, whose 128 registers a thread hold the
// sums, 32 KB are always in flight.
template <class T, int V, bool SHIFT, bool CK> struct RowX {
    Raw<T, V, CK> raw;
    __device__ __forceinline__ Vals<V> hats(float rstd, float shift, int, int) const { return raw.hats(rstd, shift); }
};
template <class T, int V> struct RowX<T, V, true, true> {
    ShiftedSteps<V> steps;
    Raw<T, V, true> raw;                                 // where o = 0
    __device__ __forceinline__ Vals<V> hats(float rstd, float shift, int e, int o) const
    {
        return o == 0 ? raw.hats(rstd, shift) : fma(steps.numbers(o), steps.scales(e - o, rstd), all<V>(shift));
    }
};
template <class T, int V, int VPT, bool SHIFT, bool CK> struct RowIn {
    RowX<T, V, SHIFT, CK> x[VPT];
    Pack<T, V> dy[VPT];
    float mean, rstd;
};
// Where a thread's first vector of a row lies; the others follow at multiples of tpr vectors.  (The checkpoint's: of the row itself.)
template <class T> struct RowAt {
    const T *x, *dy;
    T* out;
    const unsigned char *q, *e;
    const float *mean, *rstd;
};
template <class T, int V, int VPT, int FORM, bool CK>
__device__ __forceinline__ void load_row(const NormArgs& a, const RowAt<T>& at, bool live, int o, int tpr, int t, RowIn<T, V, VPT, FORM == kShift, CK>& in)
{
    constexpr bool kWhole = FORM == kFast || V == 1;
    const int hi = o + a.c;
    Reach<T, V> rd{o, hi, true}, rx{o, hi, true};
    if (!kWhole && live) {
        rd = reach<T, V>(at.dy - t * V + o, o, hi, static_cast<const T*>(a.dy), static_cast<const T*>(a.dy) + (a.rows - 1) * a.dy_stride + a.c);
        if constexpr (!CK) rx = reach<T, V>(at.x - t * V + o, o, hi, static_cast<const T*>(a.x), static_cast<const T*>(a.x) + (a.rows - 1) * a.x_stride + a.c);
    }
    in.mean = in.rstd = 0.f;
    if (live) { in.mean = *at.mean; in.rstd = *at.rstd; }
#pragma unroll
    for (int i = 0; i < VPT; ++i) {
        const int skip = i * tpr * V, e = skip + t * V;
        in.dy[i] = zero_pack<T, V>();
        in.x[i].raw.clear();
        if (live && e < hi) {
            if (kWhole) in.dy[i] = load_pack<T, V>(at.dy + skip);
            else load_whole<T, V>(in.dy[i], at.dy - t * V, e, rd.lo, rd.hi);
            if constexpr (CK) {
                if constexpr (FORM == kShift) {
                    if (o > 0) { in.x[i].steps.load(at.q, at.e, e - o, o, (int)a.ck.pitch); continue; }
                }
                in.x[i].raw.q = load_pack<unsigned char, V>(at.q + e);
                in.x[i].raw.e = at.e[(unsigned)e / kBlock];
            } else {
                if (kWhole) in.x[i].raw.a = load_pack<T, V>(at.x + skip);
                else load_whole<T, V>(in.x[i].raw.a, at.x - t * V, e, rx.lo, rx.hi);
            }
        } else if constexpr (CK && FORM == kShift) {
            in.x[i].steps.lo = in.x[i].steps.hi = zero_pack<unsigned char, V>();
            in.x[i].steps.e0 = in.x[i].steps.e1 = 1;
        }
    }
    if (!kWhole && live && !(rd.all && rx.all)) {
#pragma unroll
        for (int i = 0; i < VPT; ++i) {
            const int e = (i * tpr + t) * V;
            load_rest<T, V>(in.dy[i], at.dy - t * V, e, o, hi);
            if constexpr (!CK) load_rest<T, V>(in.x[i].raw.a, at.x - t * V, e, o, hi);
        }
    }
}

template <class T, int V, int VPT, int FORM, bool CK>
__global__ void __launch_bounds__(512, 1) norm_bwd_rows_kernel(NormArgs a, int tpr)
{
    constexpr bool kWhole = FORM == kFast || V == 1;
    constexpr int E = V * VPT;
    extern __shared__ __align__(16) float smem[];      // the weights of each thread's columns; at the end a set of columns per group, to be added
    __shared__ float red[2][32];
    __shared__ int shifts[64];
    previous_launches();
    next_launch();
    const int per = blockDim.x / tpr, group = threadIdx.x / tpr, t = threadIdx.x - group * tpr;
    const float inv_c = 1.f / (float)a.c;
    Vals<E> dw = all<E>(0.f), db = all<E>(0.f);
    const long long step = (long long)gridDim.x * per;
    long long row = (long long)blockIdx.x * per + group;
    RowAt<T> at;
    at.dy = static_cast<const T*>(a.dy) + row * a.dy_stride;
    const int o = FORM == kShift ? (int)((reinterpret_cast<uintptr_t>(at.dy) / sizeof(T)) & (V - 1)) : 0;
    const int hi = o + a.c;
    at.dy += t * V - o;
    at.x = static_cast<const T*>(a.x) + row * a.x_stride + t * V - o;
    at.out = static_cast<T*>(a.out) + row * a.out_stride + t * V - o;
    at.q = a.ck.q + row * a.ck.pitch;
    at.e = a.ck.steps + row * a.ck.blocks;
    at.mean = a.mean + row;
    at.rstd = a.rstd + row;
    RowIn<T, V, VPT, FORM == kShift, CK> next;
    load_row<T, V, VPT, FORM, CK>(a, at, row < a.rows, o, tpr, t, next);
    float4* weights = reinterpret_cast<float4*>(smem) + threadIdx.x;
    {
        Vals<E> w = all<E>(0.f);
#pragma unroll
        for (int i = 0; i < VPT; ++i) {
            const int e = (i * tpr + t) * V;
            if (e < hi) load_cols<FORM == kFast, V>(a.weight, e - o, a.c, 1.f, w.v + i * V);
        }
        if constexpr (E % 4 == 0) {
#pragma unroll
            for (int j = 0; j < E; j += 4) weights[j / 4 * blockDim.x] = make_float4(w.v[j], w.v[j + 1], w.v[j + 2], w.v[j + 3]);
        } else smem[threadIdx.x] = w.v[0];
    }
    int turn = 0;
    // (groups narrower than a warp stay together: a warp goes on until none of its rows is left)
    for (long long first = (long long)blockIdx.x * per + (tpr < 32 ? (threadIdx.x & ~31) / tpr : group); first < a.rows; first += step, turn ^= 1) {
        const float rstd = next.rstd, shift = -next.mean * next.rstd;
        if (!kWhole) {
#pragma unroll
            for (int i = 0; i < VPT; ++i) {
                keep_part<T, V>(next.dy[i], (i * tpr + t) * V, o, hi, from_f<T>(0.f));
                if constexpr (!CK) keep_part<T, V>(next.x[i].raw.a, (i * tpr + t) * V, o, hi, from_f<T>(0.f));
            }
        }
        Vals<E> d, hat;
#pragma unroll
        for (int i = 0; i < VPT; ++i) {
            const Vals<V> di = values(next.dy[i]), hi = next.x[i].hats(rstd, shift, (i * tpr + t) * V, o);
#pragma unroll
            for (int j = 0; j < V; ++j) { d.v[i * V + j] = di.v[j]; hat.v[i * V + j] = hi.v[j]; }
        }
        const bool live = row < a.rows;
        row += step;
        at.x += step * a.x_stride; at.dy += step * a.dy_stride;
        at.q += step * a.ck.pitch; at.e += step * a.ck.blocks;
        at.mean += step; at.rstd += step;
        load_row<T, V, VPT, FORM, CK>(a, at, row < a.rows, o, tpr, t, next);
        dw = fma(d, hat, dw);
        db = add(db, d);
        Vals<E> w;                                     // (16 registers more would spill)
        if constexpr (E % 4 == 0) {
#pragma unroll
            for (int j = 0; j < E; j += 4) {
                const float4 q = weights[j / 4 * blockDim.x];
                w.v[j] = q.x; w.v[j + 1] = q.y; w.v[j + 2] = q.z; w.v[j + 3] = q.w;
            }
        } else w.v[0] = smem[threadIdx.x];
        const Vals<E> g = mul(d, w);
        float s[2] = {sum_of(g), sum_of(mul(g, hat))};
        group_sum<2, true>(s, tpr, group + 1, red[turn]);
        if (a.out && live) {
            const Vals<E> dx = fma(hat, all<E>(-s[1] * inv_c * rstd), fma(g, all<E>(rstd), all<E>(-s[0] * inv_c * rstd)));
#pragma unroll
            for (int i = 0; i < VPT; ++i) {
                const int skip = i * tpr * V, e = skip + t * V;
                Vals<V> v;
#pragma unroll
                for (int j = 0; j < V; ++j) v.v[j] = dx.v[i * V + j];
                if (e < hi) {
                    if (kWhole) store_pack<T, V>(at.out + skip, rounded<T, V>(v));
                    else store_part<T, V>(at.out - t * V, e, o, hi, rounded<T, V>(v));
                }
            }
        }
        at.out += step * a.out_stride;
    }
    if (!a.partials) return;
    const int width = tpr * E;
    float* set = a.partials + (long long)blockIdx.x * 2 * a.c;
    if (t == 0) shifts[group] = o;
    for (int k = 0; k < 2; ++k) {
        __syncthreads();
#pragma unroll
        for (int i = 0; i < VPT; ++i)
#pragma unroll
            for (int j = 0; j < V; ++j) smem[group * width + (i * tpr + t) * V + j] = k ? db.v[i * V + j] : dw.v[i * V + j];
        __syncthreads();
        for (int col = threadIdx.x; col < a.c; col += blockDim.x) {
            float s = 0.f;
            for (int g = 0; g < per; ++g) s += smem[g * width + col + shifts[g]];
            set[(long long)k * a.c + col] = s;
        }
    }
}

// Rows longer than that: two passes, the column sums of the block in its partial set itself (a thread's own columns), read and written for every
// row: 1000 x 12000 fp32 takes 82 us, 22 of which are its bytes once.
template <class T, bool CK> __global__ void __launch_bounds__(1024) norm_bwd_long_rows_kernel(NormArgs a)
{
    __shared__ float red[2][64];
    previous_launches();
    const float inv_c = 1.f / (float)a.c;
    float* set = a.partials ? a.partials + (long long)blockIdx.x * 2 * a.c : nullptr;
    int turn = 0;
    for (long long row = blockIdx.x; row < a.rows; row += gridDim.x, turn ^= 1) {
        const T* xr = static_cast<const T*>(a.x) + row * a.x_stride;
        const T* dyr = static_cast<const T*>(a.dy) + row * a.dy_stride;
        const unsigned char* qr = a.ck.q + row * a.ck.pitch;
        const unsigned char* er = a.ck.steps + row * a.ck.blocks;
        const float mean = a.mean[row], rstd = a.rstd[row];
        const float shift = -mean * rstd;
        auto hat_of = [&](int e) {
            Raw<T, 1, CK> r;
            if constexpr (CK) { r.q.w[0] = qr[e]; r.e = er[e / kBlock]; }
            else r.a.w[0] = bits_of(xr[e]);
            return r.hats(rstd, shift).v[0];
        };
        float s[2] = {0.f, 0.f};
        for (int e = threadIdx.x; e < a.c; e += 1024) {
            const float g = to_f(dyr[e]) * (a.weight ? a.weight[e] : 1.f);
            s[0] += g;
            s[1] = fmaf(g, hat_of(e), s[1]);
        }
        group_sum<2>(s, 1024, 0, red[turn]);
        const float m0 = s[0] * inv_c, m1 = s[1] * inv_c;
        const bool first = row == blockIdx.x;
        for (int e = threadIdx.x; e < a.c; e += 1024) {
            const float d = to_f(dyr[e]), hat = hat_of(e);
            if (set) {
                set[e] = fmaf(d, hat, first ? 0.f : set[e]);
                set[a.c + e] = d + (first ? 0.f : set[a.c + e]);
            }
            if (a.out)
                static_cast<T*>(a.out)[row * a.out_stride + e] =
                    from_f<T>((fmaf(d, a.weight ? a.weight[e] : 1.f, -m0) - hat * m1) * rstd);
        }
    }
}

// ---- maps -------------------------------------------------------------------------------------------------------
// A tile is 32 V pixels of one sample with all channels: a lane has V pixels (4 bytes of them, or one value), and `share` warps split
// the channels, `per` <= CPT to a warp, which stay in registers.  If share > 1 these are the block; if one warp holds all channels, the
// warps of a block take a tile each and need no barrier.
struct Tile { long long n, row; int px, first, count; bool live; };

__device__ __forceinline__ Tile tile_of(const NormArgs& a, const Walk& w, int pixels, int at, int first, int per)
{
    Tile t;
    t.n = w.hi;
    t.px = w.lo * pixels + at;
    t.live = t.px < a.p;
    t.row = t.n * a.p + t.px;
    t.first = first;
    t.count = min(per, a.c - first);
    return t;
}

// Adds K values of each pixel over the `share` warps of the block, in their order (1: the warp's own).  A block's last warp may have fewer
// channels and come here by another branch than the others, where __syncthreads() would have to be one place of the program for all.
template <int K, int V> __device__ __forceinline__ void pixel_sum(Vals<V> (&v)[K], int share, float* red)
{
    if (share == 1) return;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
#pragma unroll
    for (int k = 0; k < K; ++k)
#pragma unroll
        for (int j = 0; j < V; ++j) red[((warp * K + k) * V + j) * 32 + lane] = v[k].v[j];
    block_barrier();
#pragma unroll
    for (int k = 0; k < K; ++k) v[k] = all<V>(0.f);
#pragma unroll 4
    for (int w = 0; w < share; ++w)
#pragma unroll
        for (int k = 0; k < K; ++k)
#pragma unroll
            for (int j = 0; j < V; ++j) v[k].v[j] += red[((w * K + k) * V + j) * 32 + lane];
}

// Bytes from a place of channel 0 to the same place of channel i: one wide multiply-add.
__device__ __forceinline__ const char* plane(const char* base, unsigned bytes, int i) { return base + (unsigned long long)bytes * (unsigned)i; }
__device__ __forceinline__ char* plane(char* base, unsigned bytes, int i) { return base + (unsigned long long)bytes * (unsigned)i; }

// Weight and bias of all channels, in shared memory.
__device__ __forceinline__ void stage_cols(const NormArgs& a, float2* wb)
{
    for (int i = threadIdx.x; i < a.c; i += blockDim.x) wb[i] = make_float2(a.weight ? a.weight[i] : 1.f, a.bias ? a.bias[i] : 0.f);
    __syncthreads();
}

// FULL: all CPT channels and all pixels of the tile are there, which spares four tests for every value.
template <class T, int V, int CPT, bool CK, bool FULL>
__device__ __forceinline__ void norm_fwd_tile(const NormArgs& a, const Tile& t, int share, float* red, int half, const float2* wb)
{
    const int count = FULL ? CPT : t.count;
    const bool live = FULL || t.live;
    const unsigned bytes = (unsigned)a.p * sizeof(T);
    const float inv_c = 1.f / (float)a.c;
    const char* xt = reinterpret_cast<const char*>(static_cast<const T*>(a.x) + t.n * a.x_stride + (long long)t.first * a.p + t.px);
    char* yt = reinterpret_cast<char*>(static_cast<T*>(a.out) + t.n * a.out_stride + (long long)t.first * a.p + t.px);
    Pack<T, V> raw[CPT];
#pragma unroll
    for (int i = 0; i < CPT; ++i) {
        if (!FULL) raw[i] = zero_pack<T, V>();
        if (i < count && live) raw[i] = load_pack<T, V>(reinterpret_cast<const T*>(plane(xt, bytes, i)));
    }
    Vals<V> s[1] = {all<V>(0.f)};
#pragma unroll
    for (int i = 0; i < CPT; ++i) s[0] = add(s[0], values(raw[i]));
    pixel_sum<1, V>(s, share, red);
    const Vals<V> mean = a.c == 1 ? s[0] : mul(s[0], all<V>(inv_c)), minus = mul(mean, all<V>(-1.f));
    s[0] = all<V>(0.f);
#pragma unroll
    for (int i = 0; i < CPT; ++i) keep_packed(raw[i]);
#pragma unroll
    for (int i = 0; i < CPT; ++i)
        if (i < count) { const Vals<V> d = add(values(raw[i]), minus); s[0] = fma(d, d, s[0]); }
    pixel_sum<1, V>(s, share, red + half);
#pragma unroll
    for (int i = 0; i < CPT; ++i) keep_packed(raw[i]);
    Vals<V> rstd;
#pragma unroll
    for (int j = 0; j < V; ++j) rstd.v[j] = 1.f / sqrtf(s[0].v[j] * inv_c + a.eps);
    if (live && t.first == 0) {
#pragma unroll
        for (int j = 0; j < V; ++j) {
            if (a.mean) a.mean[t.row + j] = mean.v[j];
            if (a.rstd) a.rstd[t.row + j] = rstd.v[j];
        }
    }
    const long long run = t.n * a.c + t.first;
    char* qt = reinterpret_cast<char*>(a.ck.q + run * a.ck.pitch + t.px);
    unsigned char* et = a.ck.steps + run * a.ck.blocks + t.px / kBlock;
    if constexpr (CK) {                                         // the checkpoint first, before y may have been written over x
        bool any = false;
#pragma unroll
        for (int i = 0; i < CPT; ++i) {                         // as if all values were finite
            if (i >= count) continue;
            const Vals<V> v = values(raw[i]);
            const float big = largest(v);
            any |= special<T>(big);
            const unsigned ex = step_exponent(big);
            if (FULL || t.px < a.ck.pitch) {
                store_pack<unsigned char, V>(reinterpret_cast<unsigned char*>(plane(qt, (unsigned)a.ck.pitch, i)), to_steps(v, ex));
                if (t.px % kBlock == 0) et[(unsigned long long)(unsigned)a.ck.blocks * i] = (unsigned char)ex;
            }
        }
        if (__any_sync(0xffffffffu, any)) {                     // the blocks with others once more
#pragma unroll 1
            for (int i = 0; i < count; ++i) {
                Pack<T, V> again = zero_pack<T, V>();
                if (live) again = load_pack<T, V>(reinterpret_cast<const T*>(plane(xt, bytes, i)));
                const Vals<V> v = values(again);
                if (special<T>(largest(v))) {
                    unsigned ex;
                    const Pack<unsigned char, V> st = to_steps_special<T, V>(v, ex);
                    if (FULL || t.px < a.ck.pitch) {
                        store_pack<unsigned char, V>(reinterpret_cast<unsigned char*>(plane(qt, (unsigned)a.ck.pitch, i)), st);
                        if (t.px % kBlock == 0) et[(unsigned long long)(unsigned)a.ck.blocks * i] = (unsigned char)ex;
                    }
                }
                __syncwarp();
            }
        }
    }
#pragma unroll
    for (int i = 0; i < CPT; ++i) {
        if (i >= count || !live) continue;
        const float2 c = wb[t.first + i];
        store_pack<T, V>(reinterpret_cast<T*>(plane(yt, bytes, i)),
                         rounded<T, V>(fma(add(values(raw[i]), minus), mul(rstd, all<V>(c.x)), all<V>(c.y))));
    }
}

template <class T, int V, int CPT, bool CK, int MOST>
__global__ void __launch_bounds__(MOST, MOST == 256 ? 3 : 1) norm_fwd_map_kernel(NormArgs a, int share, int per, int tiles)
{
    extern __shared__ float smem[];                      // weight and bias, then [2][warps][V * 32]
    previous_launches();
    float2* wb = reinterpret_cast<float2*>(smem);
    float* red = smem + 2 * a.c;
    stage_cols(a, wb);
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, group = warp / share, groups = (blockDim.x >> 5) / share;
    for (Walk w(blockIdx.x * groups + group, gridDim.x * groups, tiles); w.hi < a.n; w.advance()) {
        const Tile t = tile_of(a, w, 32 * V, lane * V, (warp & (share - 1)) * per, per);
        if (t.count == CPT && t.px - lane * V + 32 * V <= a.p) norm_fwd_tile<T, V, CPT, CK, true>(a, t, share, red, blockDim.x * V, wb);
        else norm_fwd_tile<T, V, CPT, CK, false>(a, t, share, red, blockDim.x * V, wb);
    }
}

// More channels than registers hold: three passes over the tile, the second and third from L2.
template <class T, int V, bool CK> __global__ void __launch_bounds__(512) norm_fwd_long_map_kernel(NormArgs a, int tiles)
{
    __shared__ float red[2][512 * V];
    previous_launches();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, warps = blockDim.x >> 5;
    for (Walk w(blockIdx.x, gridDim.x, tiles); w.hi < a.n; w.advance()) {
        const Tile t = tile_of(a, w, 32 * V, lane * V, 0, a.c);
        const T* xt = static_cast<const T*>(a.x) + t.n * a.x_stride + t.px;
        T* yt = static_cast<T*>(a.out) + t.n * a.out_stride + t.px;
        auto load = [&](int ch) { return t.live ? values(load_pack<T, V>(xt + (long long)ch * a.p)) : all<V>(0.f); };
        Vals<V> s[1] = {all<V>(0.f)};
        for (int ch = warp; ch < a.c; ch += warps) s[0] = add(s[0], load(ch));
        pixel_sum<1, V>(s, warps, red[0]);
        Vals<V> mean, rstd;
#pragma unroll
        for (int j = 0; j < V; ++j) mean.v[j] = s[0].v[j] / (float)a.c;
        const Vals<V> minus = mul(mean, all<V>(-1.f));
        s[0] = all<V>(0.f);
        for (int ch = warp; ch < a.c; ch += warps) { const Vals<V> d = add(load(ch), minus); s[0] = fma(d, d, s[0]); }
        pixel_sum<1, V>(s, warps, red[1]);
#pragma unroll
        for (int j = 0; j < V; ++j) rstd.v[j] = 1.f / sqrtf(s[0].v[j] / (float)a.c + a.eps);
        if (t.live && warp == 0) {
#pragma unroll
            for (int j = 0; j < V; ++j) {
                if (a.mean) a.mean[t.row + j] = mean.v[j];
                if (a.rstd) a.rstd[t.row + j] = rstd.v[j];
            }
        }
        for (int ch = warp; ch < a.c; ch += warps) {
            const Vals<V> x = load(ch);
            if (CK) {
                const float big = largest(x);
                unsigned ex = step_exponent(big);
                const Pack<unsigned char, V> st = special<T>(big) ? to_steps_special<T, V>(x, ex) : to_steps(x, ex);
                if (t.px < a.ck.pitch) {
                    const long long run = t.n * a.c + ch;
                    store_pack<unsigned char, V>(a.ck.q + run * a.ck.pitch + t.px, st);
                    if (t.px % kBlock == 0) a.ck.steps[run * a.ck.blocks + t.px / kBlock] = (unsigned char)ex;
                }
            }
            if (t.live) {
                const float w = a.weight ? __ldg(a.weight + ch) : 1.f, b = a.bias ? __ldg(a.bias + ch) : 0.f;
                store_pack<T, V>(yt + (long long)ch * a.p, rounded<T, V>(fma(mul(add(x, minus), rstd), all<V>(w), all<V>(b))));
            }
        }
    }
}

// Sums over the 32 lanes of N values a lane: lane l < N ends with the sum of value l.  Halving: at each step a lane gives half of its
// values to the lane across and keeps the other half, N - 1 exchanges in all instead of 5 N.
template <int N> __device__ __forceinline__ float across_lanes(float (&v)[N], int lane)
{
#pragma unroll
    for (int h = N / 2; h >= 1; h >>= 1) {
        const bool up = lane & h;
#pragma unroll
        for (int i = 0; i < h; ++i) {
            const float give = up ? v[i] : v[i + h], keep = up ? v[i + h] : v[i];
            v[i] = keep + __shfl_xor_sync(0xffffffffu, give, h);
        }
    }
    float s = v[0];
#pragma unroll
    for (int d = 16; d >= N; d >>= 1) s += __shfl_xor_sync(0xffffffffu, s, d);
    return s;
}

template <class T, int V, bool CK>
__device__ __forceinline__ void load_map(const NormArgs& a, const Tile& t, int ch, Raw<T, V, CK>& x, Pack<T, V>& dy)
{
    const long long at = (long long)ch * a.p + t.px;
    dy = zero_pack<T, V>();
    if constexpr (CK) {
        x.e = 1;
        x.q = zero_pack<unsigned char, V>();
    } else x.a = zero_pack<T, V>();
    if (!t.live) return;
    dy = load_pack<T, V>(static_cast<const T*>(a.dy) + t.n * a.dy_stride + at);
    if constexpr (CK) {
        const long long run = t.n * a.c + ch;
        x.q = load_pack<unsigned char, V>(a.ck.q + run * a.ck.pitch + t.px);
        x.e = a.ck.steps[run * a.ck.blocks + t.px / kBlock];
    } else x.a = load_pack<T, V>(static_cast<const T*>(a.x) + t.n * a.x_stride + at);
}

// FULL as above.  Adds this tile's part of the warp's channel sums to dw and db: with up to 16 channels each lane sums its pixels in
// registers; with more, lane l gets the sums of channel l, which takes two exchanges for each value.
template <int CPT> struct ChannelSums {
    static constexpr bool kOwn = CPT <= 16;
    static constexpr int kRegs = kOwn ? CPT : 1;
    float dw[kRegs], db[kRegs];
};
template <class T, int V, int CPT, bool CK, bool FULL>
__device__ __forceinline__ void norm_bwd_tile(const NormArgs& a, const Tile& t, int share, float* red, const float2* wb, ChannelSums<CPT>& cs)
{
    constexpr bool kOwn = ChannelSums<CPT>::kOwn;
    const int lane = threadIdx.x & 31, count = FULL ? CPT : t.count;
    const bool live = FULL || t.live;
    const unsigned bytes = (unsigned)a.p * sizeof(T);
    const float inv_c = 1.f / (float)a.c;
    const long long at = (long long)t.first * a.p + t.px, run = t.n * a.c + t.first;
    const char* xt = reinterpret_cast<const char*>(static_cast<const T*>(a.x) + t.n * a.x_stride + at);
    const char* dt = reinterpret_cast<const char*>(static_cast<const T*>(a.dy) + t.n * a.dy_stride + at);
    const char* qt = reinterpret_cast<const char*>(a.ck.q + run * a.ck.pitch + t.px);
    const unsigned char* et = a.ck.steps + run * a.ck.blocks + t.px / kBlock;
    Raw<T, V, CK> x[CPT];
    Pack<T, V> dy[CPT];
#pragma unroll
    for (int i = 0; i < CPT; ++i) {
        if (!FULL) { dy[i] = zero_pack<T, V>(); x[i].clear(); }
        if (i < count && live) {
            dy[i] = load_pack<T, V>(reinterpret_cast<const T*>(plane(dt, bytes, i)));
            if constexpr (CK) {
                x[i].q = load_pack<unsigned char, V>(reinterpret_cast<const unsigned char*>(plane(qt, (unsigned)a.ck.pitch, i)));
                x[i].e = et[(unsigned long long)(unsigned)a.ck.blocks * i];
            } else x[i].a = load_pack<T, V>(reinterpret_cast<const T*>(plane(xt, bytes, i)));
        }
    }
    Vals<V> rstd, shift, s[2] = {all<V>(0.f), all<V>(0.f)};
#pragma unroll
    for (int j = 0; j < V; ++j) {
        rstd.v[j] = live ? a.rstd[t.row + j] : 0.f;
        shift.v[j] = live ? -a.mean[t.row + j] * rstd.v[j] : 0.f;
    }
    float sums[kOwn ? 1 : CPT];
    constexpr bool kAgain = CK && V == 4;                       // steps are decoded twice: 32 registers of hats less
    Vals<V> hat[kAgain ? 1 : CPT];
#pragma unroll
    for (int i = 0; i < CPT; ++i) {
        if (!kOwn) sums[i] = 0.f;
        if (i >= count) continue;
        const float w = wb[t.first + i].x;
        hat[kAgain ? 0 : i] = x[i].hats(rstd, shift);
        const Vals<V> d = values(dy[i]), dh = mul(d, hat[kAgain ? 0 : i]);
        s[0] = fma(d, all<V>(w), s[0]);
        s[1] = fma(dh, all<V>(w), s[1]);
        if constexpr (kOwn) { cs.dw[i] += sum_of(dh); cs.db[i] += sum_of(d); }
        else sums[i] = sum_of(dh);
    }
    if constexpr (!kOwn)
        if (a.partials) {
            cs.dw[0] += across_lanes<CPT>(sums, lane);
#pragma unroll
            for (int i = 0; i < CPT; ++i) sums[i] = i < count ? sum_of(values(dy[i])) : 0.f;
            cs.db[0] += across_lanes<CPT>(sums, lane);
        }
    pixel_sum<2, V>(s, share, red);
    if (!a.out) return;
    const Vals<V> m0 = mul(mul(s[0], all<V>(-inv_c)), rstd), m1 = mul(mul(s[1], all<V>(-inv_c)), rstd);
    char* out = reinterpret_cast<char*>(static_cast<T*>(a.out) + t.n * a.out_stride + at);
    if constexpr (kAgain) {
#pragma unroll
        for (int i = 0; i < CPT; ++i) asm volatile("" : "+r"(x[i].q.w[0]));       // (or the compiler keeps them after all)
    }
#pragma unroll
    for (int i = 0; i < CPT; ++i)
        if (i < count && live)
            store_pack<T, V>(reinterpret_cast<T*>(plane(out, bytes, i)),
                             rounded<T, V>(fma(kAgain ? x[i].hats(rstd, shift) : hat[kAgain ? 0 : i], m1, fma(values(dy[i]), mul(rstd, all<V>(wb[t.first + i].x)), m0))));
}

template <class T, int V, int CPT, bool CK>
__global__ void __launch_bounds__(512) norm_bwd_map_kernel(NormArgs a, int share, int per, int tiles)
{
    extern __shared__ float smem[];                      // weight and bias, then [2][warps][2][V * 32]
    previous_launches();
    next_launch();
    float2* wb = reinterpret_cast<float2*>(smem);
    float* red = smem + 2 * a.c;
    stage_cols(a, wb);
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, group = warp / share, groups = (blockDim.x >> 5) / share;
    const int half = blockDim.x * V * 2;
    ChannelSums<CPT> cs;
#pragma unroll
    for (int i = 0; i < ChannelSums<CPT>::kRegs; ++i) cs.dw[i] = cs.db[i] = 0.f;
    int turn = 0;
    for (Walk w(blockIdx.x * groups + group, gridDim.x * groups, tiles); w.hi < a.n; w.advance(), turn ^= 1) {
        const Tile t = tile_of(a, w, 32 * V, lane * V, (warp & (share - 1)) * per, per);
        if (t.count == CPT && t.px - lane * V + 32 * V <= a.p)
            norm_bwd_tile<T, V, CPT, CK, true>(a, t, share, red + turn * half, wb, cs);
        else
            norm_bwd_tile<T, V, CPT, CK, false>(a, t, share, red + turn * half, wb, cs);
    }
    if (!a.partials) return;
    float dw = cs.dw[0], db = cs.db[0];
    if constexpr (ChannelSums<CPT>::kOwn) { dw = across_lanes<CPT>(cs.dw, lane); db = across_lanes<CPT>(cs.db, lane); }
    __syncthreads();
    red[threadIdx.x] = dw;
    red[blockDim.x + threadIdx.x] = db;
    __syncthreads();
    const int ch = (warp & (share - 1)) * per + lane;
    if (group == 0 && lane < per && ch < a.c) {
        float* set = a.partials + (long long)blockIdx.x * 2 * a.c;
        for (int k = 0; k < 2; ++k) {
            float s = 0.f;
            for (int g = 0; g < groups; ++g) s += red[k * blockDim.x + g * share * 32 + threadIdx.x];
            set[(long long)k * a.c + ch] = s;
        }
    }
}

// More channels than that: two passes, the sums of a channel grow in the block's own set.
template <class T, int V, bool CK> __global__ void __launch_bounds__(512) norm_bwd_long_map_kernel(NormArgs a, int tiles)
{
    __shared__ float red[2][512 * V * 2 <= 2048 ? 512 * V * 2 : 2048];
    previous_launches();
    next_launch();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, warps = blockDim.x >> 5;
    const float inv_c = 1.f / (float)a.c;
    float* set = a.partials ? a.partials + (long long)blockIdx.x * 2 * a.c : nullptr;
    int turn = 0;
    bool first = true;
    for (Walk w(blockIdx.x, gridDim.x, tiles); w.hi < a.n; w.advance(), turn ^= 1, first = false) {
        const Tile t = tile_of(a, w, 32 * V, lane * V, 0, a.c);
        Vals<V> rstd, shift, s[2] = {all<V>(0.f), all<V>(0.f)};
#pragma unroll
        for (int j = 0; j < V; ++j) {
            rstd.v[j] = t.live ? a.rstd[t.row + j] : 0.f;
            shift.v[j] = t.live ? -a.mean[t.row + j] * rstd.v[j] : 0.f;
        }
        Raw<T, V, CK> x;
        Pack<T, V> dy;
        for (int ch = warp; ch < a.c; ch += warps) {
            load_map<T, V, CK>(a, t, ch, x, dy);
            const float w = a.weight ? __ldg(a.weight + ch) : 1.f;
            const Vals<V> d = values(dy), dh = mul(d, x.hats(rstd, shift));
            s[0] = fma(d, all<V>(w), s[0]);
            s[1] = fma(dh, all<V>(w), s[1]);
            if (set) {
                const float w1 = lanes_sum(sum_of(dh)), b1 = lanes_sum(sum_of(d));
                if (lane == 0) {
                    set[ch] = w1 + (first ? 0.f : set[ch]);
                    set[a.c + ch] = b1 + (first ? 0.f : set[a.c + ch]);
                }
            }
        }
        pixel_sum<2, V>(s, warps, red[turn]);
        if (!a.out) continue;
        const Vals<V> m0 = mul(mul(s[0], all<V>(-inv_c)), rstd), m1 = mul(mul(s[1], all<V>(-inv_c)), rstd);
        for (int ch = warp; ch < a.c; ch += warps) {
            load_map<T, V, CK>(a, t, ch, x, dy);
            const float w = a.weight ? __ldg(a.weight + ch) : 1.f;
            if (t.live)
                store_pack<T, V>(static_cast<T*>(a.out) + t.n * a.out_stride + (long long)ch * a.p + t.px,
                                 rounded<T, V>(fma(x.hats(rstd, shift), m1, fma(mul(values(dy), all<V>(w)), rstd, m0))));
        }
    }
}

// ---- sum of the partial sets ------------------------------------------------------------------------------------
// Columns 0 .. 2 c - 1 of `sets` sets: 32 columns a block, its 32 warps take every 32nd set, then one adds the 32 sums.
__global__ void __launch_bounds__(1024) norm_reduce_kernel(const float* partials, int sets, int c, float* dweight, float* dbias)
{
    __shared__ float part[32][33];
    previous_launches();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const long long width = 2LL * c, col = (long long)blockIdx.x * 32 + lane;
    float s = 0.f;
    if (col < width)
#pragma unroll 8
        for (int i = warp; i < sets; i += 32) s += partials[i * width + col];
    part[warp][lane] = s;
    __syncthreads();
    s = lanes_sum(part[lane][warp]);
    const long long own = (long long)blockIdx.x * 32 + warp;
    if (lane == 0 && own < width) {
        if (own < c) dweight[own] = s; else dbias[own - c] = s;
    }
}

// ---- host -------------------------------------------------------------------------------------------------------
int pow2_at_least(long long v) { int r = 1; while (r < v) r <<= 1; return r; }

// Blocks an SM of a backward pass, each with a partial set.
constexpr int kRowSets = 2, kMapSets = 6;
unsigned fewer(long long a, long long b) { return (unsigned)(a < b ? a : b); }

template <class T, int V, int VPT, int FORM, bool CK, int MOST = 128> int run_fwd_rows(const NormArgs& a, int tpr, LaunchStream ls)
{
    const int threads = tpr > 32 ? tpr : 128, per = tpr > 32 ? 1 : threads / tpr;
    const long long fit = (long long)kSms * resident<norm_fwd_rows_kernel<T, V, VPT, FORM, CK, MOST>>(threads, 0);
    launch(norm_fwd_rows_kernel<T, V, VPT, FORM, CK, MOST>, dim3(fewer((a.rows + per - 1) / per, fit)), dim3(threads), 0, ls, a, tpr);
    return launched();
}
// As many vectors to a thread as let a warp hold the row, up to 8 (128 bytes a thread as read); then more warps.
template <class T, int V, int FORM, bool CK> int pick_fwd_rows(const NormArgs& a, LaunchStream ls)
{
    const long long vecs = (a.c + (FORM == kShift ? V - 1 : 0) + V - 1) / V;
    const int least = kBlock / V < 8 ? 8 : kBlock / V;
    auto group = [&](int vpt) { const int t = pow2_at_least((vecs + vpt - 1) / vpt); return t < least ? least : t; };
    constexpr int kWide = V == 1 ? 32 : 8;
    if (vecs <= 32) return run_fwd_rows<T, V, 1, FORM, CK>(a, group(1), ls);
    if (vecs <= 4 * 32) return run_fwd_rows<T, V, 4, FORM, CK>(a, 32, ls);
    if (vecs <= kWide * 128) return run_fwd_rows<T, V, kWide, FORM, CK>(a, group(kWide) < 32 ? 32 : group(kWide), ls);
    if (vecs <= kWide * 512) return run_fwd_rows<T, V, kWide, FORM, CK, 512>(a, group(kWide), ls);
    launch(norm_fwd_long_rows_kernel<T, CK>, dim3(fewer(a.rows, 2 * kSms)), dim3(1024), 0, ls, a);
    return launched();
}
template <class T, bool CK> int fwd_rows(const NormArgs& a, LaunchStream ls)
{
    constexpr int V = 16 / sizeof(T);
    const bool one = a.rows == 1;
    const bool on_grid = aligned(a.x, 16) && aligned(a.out, 16) && (one || (a.x_stride % V == 0 && a.out_stride % V == 0));
    const bool same = ((reinterpret_cast<uintptr_t>(a.x) ^ reinterpret_cast<uintptr_t>(a.out)) & 15) == 0 &&
                      (one || (a.x_stride - a.out_stride) % V == 0);
    if (on_grid) return a.c % V == 0 && a.weight && a.bias && a.w_vec ? pick_fwd_rows<T, V, kFast, CK>(a, ls) : pick_fwd_rows<T, V, kEdge, CK>(a, ls);
    if (same) return pick_fwd_rows<T, V, kShift, CK>(a, ls);
    return pick_fwd_rows<T, 1, kEdge, CK>(a, ls);
}

int sum_sets(const NormArgs& a, int sets, float* dweight, float* dbias, LaunchStream ls)
{
    if (!a.partials) return launched();
    launch(norm_reduce_kernel, dim3((unsigned)((2LL * a.c + 31) / 32)), dim3(1024), 0, ls, (const float*)a.partials, sets, a.c, dweight, dbias);
    return launched();
}

template <class T, int V, int VPT, int FORM, bool CK> int run_bwd_rows(const NormArgs& a, int tpr, float* dweight, float* dbias, LaunchStream ls)
{
    const int per = 512 / tpr, threads = per * tpr;
    const size_t smem = (size_t)threads * VPT * V * 4;
    int blocks = fewer((a.rows + per - 1) / per, kSms);
    // rows of a group a multiple of V rows apart (unless each has one row only)
    if (FORM == kShift && (long long)blocks * per < a.rows)
        while ((blocks * per) % V) --blocks;
    if (!allow_smem(norm_bwd_rows_kernel<T, V, VPT, FORM, CK>, smem, (size_t)512 * VPT * V * 4)) return refused();
    launch(norm_bwd_rows_kernel<T, V, VPT, FORM, CK>, dim3(blocks), dim3(threads), smem, ls, a, tpr);
    return sum_sets(a, blocks, dweight, dbias, ls);
}
// 16 values to a thread (8 in fp32, whose values as read take the registers of two); rows of up to 8192 columns.  32 values of 16 bits
// up to 16384, though they spill 736 to 1328 bytes a thread: 2020 fp16 rows of 15353, forward and backward with a checkpoint, take 312 us, and 356
// with rows read twice.
template <class T, int V, int FORM, bool CK> int pick_bwd_rows(const NormArgs& a, float* dweight, float* dbias, LaunchStream ls)
{
    const long long vecs = (a.c + (FORM == kShift ? V - 1 : 0) + V - 1) / V;
    const int least = kBlock / V < 8 ? 8 : kBlock / V;
    auto group = [&](int vpt) {                            // lanes of a warp by powers of two, then whole warps
        const long long t = (vecs + vpt - 1) / vpt;
        return t > 32 ? (int)(t + 31) / 32 * 32 : pow2_at_least(t) < least ? least : pow2_at_least(t);
    };
    constexpr int kWide = 16 / V;
    if (vecs <= 32) return run_bwd_rows<T, V, 1, FORM, CK>(a, group(1), dweight, dbias, ls);
    if constexpr (sizeof(T) == 4)
        if (vecs <= kWide / 2 * 512) return run_bwd_rows<T, V, kWide / 2, FORM, CK>(a, group(kWide / 2), dweight, dbias, ls);
    if (vecs <= kWide * 512) return run_bwd_rows<T, V, kWide, FORM, CK>(a, group(kWide), dweight, dbias, ls);
    if constexpr (V == 8)
        if (vecs <= 2 * kWide * 512) return run_bwd_rows<T, V, 2 * kWide, FORM, CK>(a, group(2 * kWide), dweight, dbias, ls);
    const int blocks = fewer(a.rows, 2 * kSms);
    launch(norm_bwd_long_rows_kernel<T, CK>, dim3(blocks), dim3(1024), 0, ls, a);
    return sum_sets(a, blocks, dweight, dbias, ls);
}
template <class T, bool CK> int bwd_rows(const NormArgs& a, float* dweight, float* dbias, LaunchStream ls)
{
    constexpr int V = 16 / sizeof(T);
    const bool one = a.rows == 1;
    auto on_grid = [&](const void* p, long long stride) { return !p || (aligned(p, 16) && (one || stride % V == 0)); };
    // the same distance above the grid as dy, in every row
    auto like_dy = [&](const void* p, long long stride) {
        return !p || (((reinterpret_cast<uintptr_t>(p) ^ reinterpret_cast<uintptr_t>(a.dy)) & 15) == 0 && (one || (stride - a.dy_stride) % V == 0));
    };
    if (on_grid(a.x, a.x_stride) && on_grid(a.dy, a.dy_stride) && on_grid(a.out, a.out_stride))
        return a.c % V == 0 && a.weight && a.w_vec ? pick_bwd_rows<T, V, kFast, CK>(a, dweight, dbias, ls) : pick_bwd_rows<T, V, kEdge, CK>(a, dweight, dbias, ls);
    if (like_dy(a.x, a.x_stride) && like_dy(a.out, a.out_stride)) return pick_bwd_rows<T, V, kShift, CK>(a, dweight, dbias, ls);
    return pick_bwd_rows<T, 1, kEdge, CK>(a, dweight, dbias, ls);
}

// Shape of a launch over maps: warps that share a tile's channels, channels of each, warps of a block.
struct MapShapeOf { int share, per, warps; };
MapShapeOf map_shape(int c, int most)
{
    MapShapeOf m{};
    m.share = pow2_at_least((c + most - 1) / most);
    m.per = (c + m.share - 1) / m.share;
    m.warps = m.share > 1 ? m.share : 4;
    return m;
}

template <class T, int V, bool CK> int fwd_map(const NormArgs& a, LaunchStream ls)
{
    const long long tiles = (a.p + 32 * V - 1) / (32 * V), all = a.n * tiles;
    if constexpr (V < 4)
        if (a.c > 1024) {
            launch(norm_fwd_long_map_kernel<T, V, CK>, dim3(fewer(all, 4 * kSms)), dim3(512), 0, ls, a, (int)tiles);
            return launched();
        }
    const MapShapeOf m = map_shape(a.c, V == 4 ? 8 : a.c <= 128 && (CK || V == 2) ? 16 : 32);
    const size_t smem = (size_t)a.c * 8 + 2 * (size_t)m.warps * 32 * V * 4;
    const long long blocks = (all + m.warps / m.share - 1) / (m.warps / m.share);
#define GO(...)                                                                                                                             \
    do {                                                                                                                                    \
        launch(__VA_ARGS__, dim3(fewer(blocks, (long long)kSms * std::min(cap, resident<__VA_ARGS__>(m.warps * 32, smem)))), dim3(m.warps * 32), smem, ls, \
               a, m.share, m.per, (int)tiles);                                                                                              \
        return launched();                                                                                                                  \
    } while (0)
    // 16 warps an SM with 32 loads each on their way: with 20 and 24 the map of 16 x 32 x 304 x 304 takes 72 and 74 us instead of 64.  With
    // a checkpoint to write the kernel is closer to the issue rate and takes all it can get (123 us with 16 warps, 111 with 24).  (Both measured on
    // fp32 maps.)  More than 512 channels take blocks of 1024 threads, whose 64 registers spill with 32 channels a thread and a checkpoint (180
    // bytes; 460 with two 16-bit pixels: 8 x 700 x 52 x 52 bf16 27 us, 45 with a checkpoint).
    const int cap = CK ? 32 : 16 / m.warps > 0 ? 16 / m.warps : 1;
    if (m.per <= 8 && m.warps <= 8) GO(norm_fwd_map_kernel<T, V, 8, CK, 256>);
    if constexpr (V == 4) GO(norm_fwd_map_kernel<T, V, 8, CK, 512>);
    else {
        if constexpr (CK || V == 2)
            if (m.per <= 16 && m.warps <= 8) GO(norm_fwd_map_kernel<T, V, 16, CK, 256>);
        if (m.warps <= 8) GO(norm_fwd_map_kernel<T, V, 32, CK, 256>);
        GO(norm_fwd_map_kernel<T, V, 32, CK, 1024>);
    }
#undef GO
}
template <class T, int V, bool CK> int bwd_map(const NormArgs& a, float* dweight, float* dbias, LaunchStream ls)
{
    const long long tiles = (a.p + 32 * V - 1) / (32 * V), all = a.n * tiles;
    if constexpr (V < 4)
        if (a.c > 512) {
            const int blocks = fewer(all, 2 * kSms);
            launch(norm_bwd_long_map_kernel<T, V, CK>, dim3(blocks), dim3(512 / V), 0, ls, a, (int)tiles);
            return sum_sets(a, blocks, dweight, dbias, ls);
        }
    // (Two 16-bit pixels with 16 and 32 channels a thread spill 390 to 740 bytes: 8 x 64 x 208 x 208 bf16 48 us, f32 50; 8 x 512 x 104 x 104 bf16
    // 98 us, f32 129, with twice the bytes to move.)
    const MapShapeOf m = map_shape(a.c, V == 4 ? 8 : CK && V == 2 && a.c <= 128 ? 8 : a.c <= 256 ? 16 : 32);
    const size_t smem = (size_t)a.c * 8 + 4 * (size_t)m.warps * 32 * V * 4;
    const long long want = (all + m.warps / m.share - 1) / (m.warps / m.share);
#define GO(...)                                                                                                    \
    do {                                                                                                           \
        const int fit = resident<__VA_ARGS__>(m.warps * 32, smem), blocks = fewer(want, (long long)kSms * (fit < kMapSets ? fit : kMapSets)); \
        launch(__VA_ARGS__, dim3(blocks), dim3(m.warps * 32), smem, ls, a, m.share, m.per, (int)tiles);            \
        return sum_sets(a, blocks, dweight, dbias, ls);                                                            \
    } while (0)
    if (m.per <= 8) GO(norm_bwd_map_kernel<T, V, 8, CK>);
    if constexpr (V < 4) {
        if (m.per <= 16) GO(norm_bwd_map_kernel<T, V, 16, CK>);
        GO(norm_bwd_map_kernel<T, V, 32, CK>);
    } else return FTP_ERR_ARG;                            // (per is at most 8)
#undef GO
}

// Whether arrays can be read v pixels at a time.
template <class T> bool map_words(const NormArgs& a, int v)
{
    auto fits = [&](const void* p, long long stride) { return !p || (aligned(p, v * sizeof(T)) && (a.n == 1 || stride % v == 0)); };
    return a.p % v == 0 && fits(a.x, a.x_stride) && fits(a.dy, a.dy_stride) && fits(a.out, a.out_stride);
}
// With a checkpoint, four pixels a lane and 8 channels a thread where 16 warps hold the channels that way: its addresses, exponents and bytes
// cost more than the arithmetic and are shared by four values then (8 x 64 x 208 x 208: one pixel and 16 channels 50 us forward, 54 us
// backward).  Without one, more channels a thread and fewer barriers are worth more.
template <class T, bool CK> bool map_quads(const NormArgs& a) { return CK && a.c <= 128 && map_words<T>(a, 4); }

template <class T, bool CK> int forward(const NormArgs& a, LaunchStream ls)
{
    if (a.p == 1) return fwd_rows<T, CK>(a, ls);
    if constexpr (CK)
        if (map_quads<T, CK>(a)) return fwd_map<T, 4, CK>(a, ls);
    if constexpr (sizeof(T) == 2)
        if (map_words<T>(a, 2)) return fwd_map<T, 2, CK>(a, ls);
    return fwd_map<T, 1, CK>(a, ls);
}
template <class T, bool CK> int backward(const NormArgs& a, float* dweight, float* dbias, LaunchStream ls)
{
    if (a.p == 1) return bwd_rows<T, CK>(a, dweight, dbias, ls);
    if constexpr (CK)
        if (map_quads<T, CK>(a)) return bwd_map<T, 4, CK>(a, dweight, dbias, ls);
    if constexpr (sizeof(T) == 2)
        if (map_words<T>(a, 2)) return bwd_map<T, 2, CK>(a, dweight, dbias, ls);
    return bwd_map<T, 1, CK>(a, dweight, dbias, ls);
}
template <class T> int forward(const NormArgs& a, bool ck, LaunchStream ls) { return ck ? forward<T, true>(a, ls) : forward<T, false>(a, ls); }
template <class T> int backward(const NormArgs& a, bool ck, float* dw, float* db, LaunchStream ls)
{
    return ck ? backward<T, true>(a, dw, db, ls) : backward<T, false>(a, dw, db, ls);
}

size_t workspace_bytes(const ftp_dims* d) { return (size_t)kSms * (d->p == 1 ? kRowSets : kMapSets) * 2 * (size_t)d->c * 4; }

}  // namespace

extern "C" {

int ftp_norm_forward(const ftp_dims* d, const void* x, long long x_stride, const float* weight, const float* bias, float eps,
                     void* y, long long y_stride, float* mean, float* rstd, void* ckpt, void* stream)
{
    long long rows = 0;
    const int rc = check_dims(d, &rows);
    if (rc != FTP_OK) return rc;
    if (!(eps >= 0.f && eps <= 3.0e38f)) return FTP_ERR_ARG;
    if (rows == 0) return FTP_OK;
    const size_t size = type_size(d->type);
    if (!x || !y || !aligned(x, size) || !aligned(y, size) || !fix_stride(d, &x_stride) || !fix_stride(d, &y_stride)) return FTP_ERR_ARG;
    if (!aligned(weight, 4) || !aligned(bias, 4) || !aligned(mean, 4) || !aligned(rstd, 4) || !aligned(ckpt, 16)) return FTP_ERR_ARG;
    NormArgs a{};
    a.x = x; a.out = y; a.x_stride = x_stride; a.out_stride = y_stride;
    a.weight = weight; a.bias = bias; a.mean = mean; a.rstd = rstd; a.ck = ckpt_view(d, ckpt);
    a.n = d->n; a.rows = rows; a.c = (int)d->c; a.p = (int)d->p; a.eps = eps;
    a.w_vec = aligned(weight, 16) && aligned(bias, 16);
    const LaunchStream ls{static_cast<cudaStream_t>(stream), true};
    if (d->type == FTP_TYPE_F32) return forward<float>(a, ckpt != nullptr, ls);
    if (d->type == FTP_TYPE_BF16) return forward<__nv_bfloat16>(a, ckpt != nullptr, ls);
    return forward<__half>(a, ckpt != nullptr, ls);
}

int ftp_norm_workspace(const ftp_dims* d, size_t* bytes)
{
    long long rows = 0;
    const int rc = check_dims(d, &rows);
    if (rc != FTP_OK) return rc;
    if (!bytes) return FTP_ERR_ARG;
    *bytes = workspace_bytes(d);
    return FTP_OK;
}

int ftp_norm_backward(const ftp_dims* d, const void* x, long long x_stride, const void* ckpt, const void* dy, long long dy_stride,
                      const float* weight, const float* mean, const float* rstd, void* dx, long long dx_stride,
                      float* dweight, float* dbias, void* workspace, size_t workspace_size, void* stream)
{
    long long rows = 0;
    const int rc = check_dims(d, &rows);
    if (rc != FTP_OK) return rc;
    if ((dweight == nullptr) != (dbias == nullptr) || (rows > 0 && !dx && !dweight)) return FTP_ERR_ARG;
    if (!aligned(dweight, 4) || !aligned(dbias, 4)) return FTP_ERR_ARG;
    if (dweight && (!workspace || !aligned(workspace, 16) || workspace_size < workspace_bytes(d))) return FTP_ERR_ARG;
    const cudaStream_t st = static_cast<cudaStream_t>(stream);
    if (rows == 0) {                                     // sums over nothing
        if (dweight && (cudaMemsetAsync(dweight, 0, (size_t)d->c * 4, st) != cudaSuccess ||
                        cudaMemsetAsync(dbias, 0, (size_t)d->c * 4, st) != cudaSuccess)) return refused();
        return FTP_OK;
    }
    if ((x == nullptr) == (ckpt == nullptr) || !dy || !mean || !rstd) return FTP_ERR_ARG;
    const size_t size = type_size(d->type);
    if (!aligned(x, size) || !aligned(dy, size) || !aligned(dx, size) || !aligned(ckpt, 16)) return FTP_ERR_ARG;
    if (!aligned(weight, 4) || !aligned(mean, 4) || !aligned(rstd, 4)) return FTP_ERR_ARG;
    if ((x && !fix_stride(d, &x_stride)) || !fix_stride(d, &dy_stride) || (dx && !fix_stride(d, &dx_stride))) return FTP_ERR_ARG;
    NormArgs a{};
    a.x = x; a.dy = dy; a.out = dx; a.x_stride = x ? x_stride : 0; a.dy_stride = dy_stride; a.out_stride = dx ? dx_stride : 0;
    a.weight = weight; a.mean = const_cast<float*>(mean); a.rstd = const_cast<float*>(rstd); a.ck = ckpt_view(d, ckpt);
    a.partials = dweight ? static_cast<float*>(workspace) : nullptr;
    a.n = d->n; a.rows = rows; a.c = (int)d->c; a.p = (int)d->p;
    a.w_vec = aligned(weight, 16);
    const LaunchStream ls{st, true};
    if (d->type == FTP_TYPE_F32) return backward<float>(a, ckpt != nullptr, dweight, dbias, ls);
    if (d->type == FTP_TYPE_BF16) return backward<__nv_bfloat16>(a, ckpt != nullptr, dweight, dbias, ls);
    return backward<__half>(a, ckpt != nullptr, dweight, dbias, ls);
}

}  // extern "C"
