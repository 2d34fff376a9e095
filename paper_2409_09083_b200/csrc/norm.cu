// Channel norm, forward and backward (ftp_norm_forward, ftp_norm_backward).
//
// Both directions are bound by memory: forward reads x and writes y, backward reads x (or its checkpoint) and dy and writes dx.
// So a row of values is read once and stays in registers between its statistics and its result, and a block takes rows until
// none are left.  Two layouts: matrices (p = 1), where the threads of a group lie along the row, and maps (p > 1), where the
// lanes of a warp lie along the pixels of a plane and groups of threads share out the channels.
//
// The variance is the mean of (x - mean)^2 over values in registers, not E x^2 - mean^2.  dweight and dbias: a thread keeps the
// same columns (channels) for all its rows and sums them in registers; each block writes one partial set and a second launch adds
// the sets in a fixed order.
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

constexpr int kRowThreads = 256;       // matrices: threads of a block whose rows are shorter than that many vectors
constexpr int kMapThreads = 256;

// Adds over the `tpr` threads of a group; tpr a power of two, groups within a warp or a whole number of warps.  `red`: a float a warp,
// not read or written by anyone else until another barrier has passed.
template <int K> __device__ __forceinline__ void group_sum(float (&v)[K], int tpr, float* red)
{
#pragma unroll
    for (int k = 0; k < K; ++k) v[k] = lanes_sum(v[k], tpr < 32 ? tpr : 32);
    if (tpr <= 32) return;
    const int warp = threadIdx.x >> 5, per = tpr >> 5, first = warp & ~(per - 1);
    if ((threadIdx.x & 31) == 0) {
#pragma unroll
        for (int k = 0; k < K; ++k) red[warp * K + k] = v[k];
    }
    __syncthreads();
#pragma unroll
    for (int k = 0; k < K; ++k) {
        float s = 0.f;
        for (int i = 0; i < per; ++i) s += red[(first + i) * K + k];
        v[k] = s;
    }
}

// weight or bias of columns [col, col + V) (null: `none`); columns outside [0, c) read as `none`.
template <int V> __device__ __forceinline__ void load_cols(const float* w, int col, int c, bool vec, float none, float (&out)[V])
{
    if (w && vec && V % 4 == 0 && col >= 0 && (col & 3) == 0 && col + V <= c) {
#pragma unroll
        for (int j = 0; j < V; j += 4) {
            const float4 q = __ldg(reinterpret_cast<const float4*>(w + col + j));
            out[j] = q.x; out[(j + 1) % V] = q.y; out[(j + 2) % V] = q.z; out[(j + 3) % V] = q.w;
        }
        return;
    }
#pragma unroll
    for (int j = 0; j < V; ++j) out[j] = w && col + j >= 0 && col + j < c ? __ldg(w + col + j) : none;
}

// The checkpoint's bytes of V values whose block is spread over 32 / V neighbouring lanes (all lanes take part).
template <class T, int V> __device__ __forceinline__ Pack<unsigned char, V> make_steps(const Pack<T, V>& a, unsigned& e)
{
    unsigned big = 0;
#pragma unroll
    for (int j = 0; j < V; ++j) big = max(big, magnitude_bits(to_f(a.v[j])));
#pragma unroll
    for (int d = kBlock / V / 2; d >= 1; d >>= 1) big = max(big, __shfl_xor_sync(0xffffffffu, big, d));
    e = step_exponent(big);
    const float inverse = inverse_step(e), most = most_steps<T>(e);
    Pack<unsigned char, V> q;
#pragma unroll
    for (int j = 0; j < V; ++j) q.v[j] = (unsigned char)to_steps(to_f(a.v[j]), inverse, most);
    return q;
}

template <int V> __device__ __forceinline__ void read_steps(const Pack<unsigned char, V>& q, float step, float (&out)[V])
{
    if constexpr (V % 4 == 0) {
#pragma unroll
        for (int j = 0; j < V; j += 4) {
            unsigned w;
            __builtin_memcpy(&w, &q.v[j], 4);
            float f[4];
            from_steps(w, step, f);
#pragma unroll
            for (int k = 0; k < 4; ++k) out[j + k] = f[k];
        }
    } else {
#pragma unroll
        for (int j = 0; j < V; ++j) out[j] = from_step(q.v[j], step);
    }
}

// What a row's x is read as: packs of the array, or steps of the checkpoint.
template <class T, int V, bool CK> struct Raw;
template <class T, int V> struct Raw<T, V, false> {
    Pack<T, V> a;
    __device__ __forceinline__ void values(float (&out)[V]) const
    {
#pragma unroll
        for (int j = 0; j < V; ++j) out[j] = to_f(a.v[j]);
    }
};
template <class T, int V> struct Raw<T, V, true> {
    Pack<unsigned char, V> q;
    unsigned char e;
    __device__ __forceinline__ void values(float (&out)[V]) const { read_steps<V>(q, step_of(e), out); }
};

// ---- matrices ---------------------------------------------------------------------------------------------------
// A group of `tpr` threads holds a row as VPT vectors of V values a thread: vector i * tpr + t.  SHIFT: rows start at any
// multiple of the value's size, and the vectors lie on the 16-byte grid below the row's start (x and y the same distance above
// it); then column = place - o.  With V = 1 any alignment goes.
template <class T, int V, int VPT, bool SHIFT, bool CK>
__global__ void __launch_bounds__(1024) norm_fwd_rows_kernel(NormArgs a, int tpr)
{
    __shared__ float red[2][32];
    previous_launches();
    const int per = blockDim.x / tpr, t = threadIdx.x & (tpr - 1);
    for (long long row0 = (long long)blockIdx.x * per; row0 < a.rows; row0 += (long long)gridDim.x * per) {
        const long long row = row0 + threadIdx.x / tpr;
        const bool live = row < a.rows;
        const T* xr = static_cast<const T*>(a.x) + row * a.x_stride;
        T* yr = static_cast<T*>(a.out) + row * a.out_stride;
        const int o = SHIFT ? (int)((reinterpret_cast<uintptr_t>(xr) / sizeof(T)) & (V - 1)) : 0;
        const int hi = live ? o + a.c : 0;
        xr -= o; yr -= o;
        Pack<T, V> raw[VPT];
        float s[1] = {0.f};
#pragma unroll
        for (int i = 0; i < VPT; ++i) {
            const int e = (i * tpr + t) * V;
            raw[i] = e < hi ? load_part<T, V>(xr, e, o, hi) : zero_pack<T, V>();
        }
#pragma unroll
        for (int i = 0; i < VPT; ++i)
#pragma unroll
            for (int j = 0; j < V; ++j) s[0] += to_f(raw[i].v[j]);
        group_sum<1>(s, tpr, red[0]);
        const float mean = s[0] / (float)a.c;
        float q[1] = {0.f};
#pragma unroll
        for (int i = 0; i < VPT; ++i) {
            const int e = (i * tpr + t) * V;
#pragma unroll
            for (int j = 0; j < V; ++j) {
                const float d = to_f(raw[i].v[j]) - mean;
                if (e + j >= o && e + j < hi) q[0] = fmaf(d, d, q[0]);
            }
        }
        group_sum<1>(q, tpr, red[1]);
        const float rstd = 1.f / sqrtf(q[0] / (float)a.c + a.eps);
        if (live && t == 0) {
            if (a.mean) a.mean[row] = mean;
            if (a.rstd) a.rstd[row] = rstd;
        }
#pragma unroll
        for (int i = 0; i < VPT; ++i) {
            const int e = (i * tpr + t) * V;
            if (CK) {
                unsigned ex;
                const Pack<unsigned char, V> st = make_steps<T, V>(raw[i], ex);
                if (live && e < a.ck.pitch) {
                    store_pack<unsigned char, V>(a.ck.q + row * a.ck.pitch + e, st);
                    if (e % kBlock == 0) a.ck.steps[row * a.ck.blocks + e / kBlock] = (unsigned char)ex;
                }
            }
            if (e < hi) {
                float w[V], b[V];
                load_cols<V>(a.weight, e - o, a.c, a.w_vec, 1.f, w);
                load_cols<V>(a.bias, e - o, a.c, a.w_vec, 0.f, b);
                Pack<T, V> y;
#pragma unroll
                for (int j = 0; j < V; ++j) y.v[j] = from_f<T>(fmaf((to_f(raw[i].v[j]) - mean) * rstd, w[j], b[j]));
                store_part<T, V>(yr, e, o, hi, y);
            }
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
        group_sum<1>(s, 1024, red[0]);
        const float mean = s[0] / (float)a.c;
        for (int e = threadIdx.x; e < a.c; e += 1024) { const float d = to_f(xr[e]) - mean; q[0] = fmaf(d, d, q[0]); }
        group_sum<1>(q, 1024, red[1]);
        const float rstd = 1.f / sqrtf(q[0] / (float)a.c + a.eps);
        if (threadIdx.x == 0) {
            if (a.mean) a.mean[row] = mean;
            if (a.rstd) a.rstd[row] = rstd;
        }
        const int end = (a.c + kBlock - 1) / kBlock * kBlock;         // whole warps, for the blocks of a checkpoint
        for (int e = threadIdx.x; e < end; e += 1024) {
            Pack<T, 1> v = zero_pack<T, 1>();
            if (e < a.c) v.v[0] = xr[e];
            if (CK) {
                unsigned ex;
                const Pack<unsigned char, 1> st = make_steps<T, 1>(v, ex);
                a.ck.q[row * a.ck.pitch + e] = st.v[0];
                if (e % kBlock == 0) a.ck.steps[row * a.ck.blocks + e / kBlock] = (unsigned char)ex;
            }
            if (e < a.c)
                yr[e] = from_f<T>(fmaf((to_f(v.v[0]) - mean) * rstd, a.weight ? a.weight[e] : 1.f, a.bias ? a.bias[e] : 0.f));
        }
    }
}

// Backward pass of matrices; the same spread of a row over a group.  A thread's columns are the same in every row, so dweight and
// dbias of its columns add up in registers over all rows of the block.
template <class T, int V, int VPT, bool CK>
__global__ void __launch_bounds__(V* VPT >= 16 ? 512 : 1024) norm_bwd_rows_kernel(NormArgs a, int tpr)
{
    extern __shared__ float smem[];                    // a set of columns per group, to add the groups of the block
    __shared__ float red[2][64];
    previous_launches();
    const int per = blockDim.x / tpr, t = threadIdx.x & (tpr - 1);
    const float inv_c = 1.f / (float)a.c;
    float dw[VPT][V], db[VPT][V];
#pragma unroll
    for (int i = 0; i < VPT; ++i)
#pragma unroll
        for (int j = 0; j < V; ++j) dw[i][j] = db[i][j] = 0.f;
    int turn = 0;
    for (long long row0 = (long long)blockIdx.x * per; row0 < a.rows; row0 += (long long)gridDim.x * per, turn ^= 1) {
        const long long row = row0 + threadIdx.x / tpr;
        const bool live = row < a.rows;
        const int c = live ? a.c : 0;
        Raw<T, V, CK> x[VPT];
        Pack<T, V> dy[VPT];
#pragma unroll
        for (int i = 0; i < VPT; ++i) {
            const int e = (i * tpr + t) * V;
            if (e < c) {
                dy[i] = load_part<T, V>(static_cast<const T*>(a.dy) + row * a.dy_stride, e, 0, c);
                if constexpr (CK) {
                    x[i].q = load_pack<unsigned char, V>(a.ck.q + row * a.ck.pitch + e);
                    x[i].e = a.ck.steps[row * a.ck.blocks + e / kBlock];
                } else x[i].a = load_part<T, V>(static_cast<const T*>(a.x) + row * a.x_stride, e, 0, c);
            }
        }
        const float mean = live ? a.mean[row] : 0.f, rstd = live ? a.rstd[row] : 0.f;
        float s[2] = {0.f, 0.f};
#pragma unroll
        for (int i = 0; i < VPT; ++i) {
            const int e = (i * tpr + t) * V;
            if (e >= c) continue;
            float xv[V], w[V];
            x[i].values(xv);
            load_cols<V>(a.weight, e, a.c, a.w_vec, 1.f, w);
#pragma unroll
            for (int j = 0; j < V; ++j) {
                const float d = to_f(dy[i].v[j]), hat = (xv[j] - mean) * rstd, g = d * w[j];
                if (e + j < c) { s[0] += g; s[1] = fmaf(g, hat, s[1]); }
                dw[i][j] = fmaf(d, hat, dw[i][j]);
                db[i][j] += d;
            }
        }
        group_sum<2>(s, tpr, red[turn]);
        if (!a.out) continue;
        const float m0 = s[0] * inv_c, m1 = s[1] * inv_c;
#pragma unroll
        for (int i = 0; i < VPT; ++i) {
            const int e = (i * tpr + t) * V;
            if (e >= c) continue;
            float xv[V], w[V];
            x[i].values(xv);
            load_cols<V>(a.weight, e, a.c, a.w_vec, 1.f, w);
            Pack<T, V> dx;
#pragma unroll
            for (int j = 0; j < V; ++j) {
                const float hat = (xv[j] - mean) * rstd;
                dx.v[j] = from_f<T>((fmaf(to_f(dy[i].v[j]), w[j], -m0) - hat * m1) * rstd);
            }
            store_part<T, V>(static_cast<T*>(a.out) + row * a.out_stride, e, 0, c, dx);
        }
    }
    if (!a.partials) return;
    next_launch();
    const int width = tpr * VPT * V;
    float* set = a.partials + (long long)blockIdx.x * 2 * a.c;
    for (int k = 0; k < 2; ++k) {
        __syncthreads();
#pragma unroll
        for (int i = 0; i < VPT; ++i)
#pragma unroll
            for (int j = 0; j < V; ++j) smem[(threadIdx.x / tpr) * width + (i * tpr + t) * V + j] = k ? db[i][j] : dw[i][j];
        __syncthreads();
        for (int e = threadIdx.x; e < a.c; e += blockDim.x) {
            float s = 0.f;
            for (int g = 0; g < per; ++g) s += smem[g * width + e];
            set[(long long)k * a.c + e] = s;
        }
    }
}

// Rows longer than that: two passes, the column sums of the block in its partial set itself (a thread's own columns).
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
        auto hat_of = [&](int e) { return ((CK ? from_step(qr[e], step_of(er[e / kBlock])) : to_f(xr[e])) - mean) * rstd; };
        float s[2] = {0.f, 0.f};
        for (int e = threadIdx.x; e < a.c; e += 1024) {
            const float g = to_f(dyr[e]) * (a.weight ? a.weight[e] : 1.f);
            s[0] += g;
            s[1] = fmaf(g, hat_of(e), s[1]);
        }
        group_sum<2>(s, 1024, red[turn]);
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
// A tile is lp * V pixels of one sample with all channels: lane l < lp of a group of lp threads has pixels l * V .. of
// channels g, g + groups, ...  (CPT of them in registers, or any number if CPT is 0, then read again for every pass).
struct Tile { long long n; int px; bool live; long long row; };

__device__ __forceinline__ Tile tile_of(const NormArgs& a, long long tile, int tiles, int pixels, int at)
{
    Tile t;
    t.n = tile / tiles;
    t.px = (int)(tile - t.n * tiles) * pixels + at;
    t.live = t.px < a.p;
    t.row = t.n * a.p + t.px;
    return t;
}

// Sums over the channels of each pixel: over the lanes of a warp that share pixels, then over the warps.  `red`: [warps][pixels * K].
template <int K, int V> __device__ __forceinline__ void pixel_sum(float (&v)[K][V], int lp, float* red)
{
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, warps = blockDim.x >> 5;
#pragma unroll
    for (int k = 0; k < K; ++k)
#pragma unroll
        for (int j = 0; j < V; ++j)
            for (int d = 16; d >= lp; d >>= 1) v[k][j] += __shfl_xor_sync(0xffffffffu, v[k][j], d);
    if (lane < lp) {
#pragma unroll
        for (int k = 0; k < K; ++k)
#pragma unroll
            for (int j = 0; j < V; ++j) red[((warp * K + k) * V + j) * lp + lane] = v[k][j];
    }
    __syncthreads();
#pragma unroll
    for (int k = 0; k < K; ++k)
#pragma unroll
        for (int j = 0; j < V; ++j) {
            float s = 0.f;
            for (int w = 0; w < warps; ++w) s += red[((w * K + k) * V + j) * lp + (lane & (lp - 1))];
            v[k][j] = s;
        }
}

template <class T, int V, int CPT, bool CK>
__global__ void __launch_bounds__(512) norm_fwd_map_kernel(NormArgs a, int lp, int tiles)
{
    extern __shared__ float smem[];
    previous_launches();
    const int l = threadIdx.x & (lp - 1), g = threadIdx.x / lp, groups = blockDim.x / lp;
    const int red = (blockDim.x >> 5) * lp * V;
    const int slots = CPT ? CPT : (a.c + groups - 1) / groups;
    for (long long tile = blockIdx.x; tile < a.n * tiles; tile += gridDim.x) {
        const Tile t = tile_of(a, tile, tiles, lp * V, l * V);
        const T* xt = static_cast<const T*>(a.x) + t.n * a.x_stride + t.px;
        T* yt = static_cast<T*>(a.out) + t.n * a.out_stride + t.px;
        auto load = [&](int i) {
            const int ch = g + i * groups;
            return t.live && ch < a.c ? load_pack<T, V>(xt + (long long)ch * a.p) : zero_pack<T, V>();
        };
        Pack<T, V> raw[CPT ? CPT : 1];
        float s[1][V], q[1][V];
#pragma unroll
        for (int j = 0; j < V; ++j) s[0][j] = q[0][j] = 0.f;
        if constexpr (CPT > 0) {
#pragma unroll
            for (int i = 0; i < CPT; ++i) raw[i] = load(i);
        }
        auto sum = [&](const Pack<T, V>& r) {
#pragma unroll
            for (int j = 0; j < V; ++j) s[0][j] += to_f(r.v[j]);
        };
        if constexpr (CPT > 0) {
#pragma unroll
            for (int i = 0; i < CPT; ++i) sum(raw[i]);
        } else
            for (int i = 0; i < slots; ++i) sum(load(i));
        pixel_sum<1, V>(s, lp, smem);
        float mean[V], rstd[V];
#pragma unroll
        for (int j = 0; j < V; ++j) mean[j] = s[0][j] / (float)a.c;
        auto square = [&](const Pack<T, V>& r, int i) {
            if (g + i * groups >= a.c) return;
#pragma unroll
            for (int j = 0; j < V; ++j) { const float d = to_f(r.v[j]) - mean[j]; q[0][j] = fmaf(d, d, q[0][j]); }
        };
        if constexpr (CPT > 0) {
#pragma unroll
            for (int i = 0; i < CPT; ++i) square(raw[i], i);
        } else
            for (int i = 0; i < slots; ++i) square(load(i), i);
        pixel_sum<1, V>(q, lp, smem + red);
#pragma unroll
        for (int j = 0; j < V; ++j) rstd[j] = 1.f / sqrtf(q[0][j] / (float)a.c + a.eps);
        if (t.live && g == 0) {
#pragma unroll
            for (int j = 0; j < V; ++j) {
                if (a.mean) a.mean[t.row + j] = mean[j];
                if (a.rstd) a.rstd[t.row + j] = rstd[j];
            }
        }
        auto finish = [&](const Pack<T, V>& r, int i) {
            const int ch = g + i * groups;
            if (CK) {
                unsigned ex;
                const Pack<unsigned char, V> st = make_steps<T, V>(r, ex);
                if (ch < a.c && t.px < a.ck.pitch) {
                    const long long run = t.n * a.c + ch;
                    store_pack<unsigned char, V>(a.ck.q + run * a.ck.pitch + t.px, st);
                    if (t.px % kBlock == 0) a.ck.steps[run * a.ck.blocks + t.px / kBlock] = (unsigned char)ex;
                }
            }
            if (t.live && ch < a.c) {
                const float w = a.weight ? __ldg(a.weight + ch) : 1.f, b = a.bias ? __ldg(a.bias + ch) : 0.f;
                Pack<T, V> y;
#pragma unroll
                for (int j = 0; j < V; ++j) y.v[j] = from_f<T>(fmaf((to_f(r.v[j]) - mean[j]) * rstd[j], w, b));
                store_pack<T, V>(yt + (long long)ch * a.p, y);
            }
        };
        if constexpr (CPT > 0) {
#pragma unroll
            for (int i = 0; i < CPT; ++i) finish(raw[i], i);
        } else
            for (int i = 0; i < slots; ++i) finish(load(i), i);
    }
}

template <class T, int V, int CPT, bool CK>
__global__ void __launch_bounds__(512) norm_bwd_map_kernel(NormArgs a, int lp, int tiles)
{
    extern __shared__ float smem[];
    previous_launches();
    const int l = threadIdx.x & (lp - 1), g = threadIdx.x / lp, groups = blockDim.x / lp;
    const int red = (blockDim.x >> 5) * lp * V * 2;
    const int slots = CPT ? CPT : (a.c + groups - 1) / groups;
    const float inv_c = 1.f / (float)a.c;
    constexpr int R = CPT ? CPT : 1;
    float dw[R], db[R];
#pragma unroll
    for (int i = 0; i < R; ++i) dw[i] = db[i] = 0.f;
    float* set = a.partials ? a.partials + (long long)blockIdx.x * 2 * a.c : nullptr;
    int turn = 0;
    for (long long tile = blockIdx.x; tile < a.n * tiles; tile += gridDim.x, turn ^= 1) {
        const Tile t = tile_of(a, tile, tiles, lp * V, l * V);
        const T* xt = static_cast<const T*>(a.x) + t.n * a.x_stride + t.px;
        const T* dyt = static_cast<const T*>(a.dy) + t.n * a.dy_stride + t.px;
        auto load = [&](int i, Raw<T, V, CK>& x, Pack<T, V>& dy) {
            const int ch = g + i * groups;
            const bool there = t.live && ch < a.c;
            dy = there ? load_pack<T, V>(dyt + (long long)ch * a.p) : zero_pack<T, V>();
            if constexpr (CK) {
                const long long run = t.n * a.c + ch;
                x.e = 0;
                if (there) {
                    x.q = load_pack<unsigned char, V>(a.ck.q + run * a.ck.pitch + t.px);
                    x.e = a.ck.steps[run * a.ck.blocks + t.px / kBlock];
                } else
                    for (int j = 0; j < V; ++j) x.q.v[j] = 0;
            } else x.a = there ? load_pack<T, V>(xt + (long long)ch * a.p) : zero_pack<T, V>();
        };
        Raw<T, V, CK> x[R];
        Pack<T, V> dy[R];
        if constexpr (CPT > 0) {
#pragma unroll
            for (int i = 0; i < CPT; ++i) load(i, x[i], dy[i]);
        }
        float mean[V], rstd[V], s[2][V];
#pragma unroll
        for (int j = 0; j < V; ++j) {
            mean[j] = t.live ? a.mean[t.row + j] : 0.f;
            rstd[j] = t.live ? a.rstd[t.row + j] : 0.f;
            s[0][j] = s[1][j] = 0.f;
        }
        auto sum = [&](const Raw<T, V, CK>& xr, const Pack<T, V>& dr, int i, float& dw_i, float& db_i) {
            const int ch = g + i * groups;
            if (ch >= a.c) return;
            const float w = a.weight ? __ldg(a.weight + ch) : 1.f;
            float xv[V];
            xr.values(xv);
#pragma unroll
            for (int j = 0; j < V; ++j) {
                const float d = to_f(dr.v[j]), hat = (xv[j] - mean[j]) * rstd[j], gr = d * w;
                s[0][j] += gr;
                s[1][j] = fmaf(gr, hat, s[1][j]);
                dw_i = fmaf(d, hat, dw_i);
                db_i += d;
            }
        };
        if constexpr (CPT > 0) {
#pragma unroll
            for (int i = 0; i < CPT; ++i) sum(x[i], dy[i], i, dw[i], db[i]);
        } else {
            for (int i = 0; i < slots; ++i) {
                float w1 = 0.f, b1 = 0.f;
                load(i, x[0], dy[0]);
                sum(x[0], dy[0], i, w1, b1);
                if (set) {                                   // the channel's sums grow in the block's own set
                    w1 = lanes_sum(w1, lp); b1 = lanes_sum(b1, lp);
                    const int ch = g + i * groups;
                    if (l == 0 && ch < a.c) {
                        const bool first = tile == blockIdx.x;
                        set[ch] = w1 + (first ? 0.f : set[ch]);
                        set[a.c + ch] = b1 + (first ? 0.f : set[a.c + ch]);
                    }
                }
            }
        }
        pixel_sum<2, V>(s, lp, smem + turn * red);
        auto finish = [&](const Raw<T, V, CK>& xr, const Pack<T, V>& dr, int i) {
            const int ch = g + i * groups;
            if (!t.live || ch >= a.c) return;
            const float w = a.weight ? __ldg(a.weight + ch) : 1.f;
            float xv[V];
            xr.values(xv);
            Pack<T, V> dx;
#pragma unroll
            for (int j = 0; j < V; ++j) {
                const float hat = (xv[j] - mean[j]) * rstd[j];
                dx.v[j] = from_f<T>((fmaf(to_f(dr.v[j]), w, -s[0][j] * inv_c) - hat * (s[1][j] * inv_c)) * rstd[j]);
            }
            store_pack<T, V>(static_cast<T*>(a.out) + t.n * a.out_stride + t.px + (long long)ch * a.p, dx);
        };
        if (!a.out) continue;
        if constexpr (CPT > 0) {
#pragma unroll
            for (int i = 0; i < CPT; ++i) finish(x[i], dy[i], i);
        } else
            for (int i = 0; i < slots; ++i) { load(i, x[0], dy[0]); finish(x[0], dy[0], i); }
    }
    if (CPT == 0 || !set) return;
    next_launch();
#pragma unroll
    for (int i = 0; i < R; ++i) {
        const float w1 = lanes_sum(dw[i], lp), b1 = lanes_sum(db[i], lp);
        const int ch = g + i * groups;
        if (l == 0 && ch < a.c) { set[ch] = w1; set[a.c + ch] = b1; }
    }
}

// ---- sum of the partial sets ------------------------------------------------------------------------------------
// Columns 0 .. 2 c - 1 of `sets` sets: 32 columns a block, its 8 warps take every eighth set, then one adds the eight sums.
__global__ void __launch_bounds__(256) norm_reduce_kernel(const float* partials, int sets, int c, float* dweight, float* dbias)
{
    __shared__ float part[8][33];
    previous_launches();
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const long long col = (long long)blockIdx.x * 32 + lane, width = 2LL * c;
    float s = 0.f;
    if (col < width)
        for (int i = warp; i < sets; i += 8) s += partials[i * width + col];
    part[warp][lane] = s;
    __syncthreads();
    if (warp == 0 && col < width) {
        s = 0.f;
#pragma unroll
        for (int i = 0; i < 8; ++i) s += part[i][lane];
        if (col < c) dweight[col] = s; else dbias[col - c] = s;
    }
}

// ---- host -------------------------------------------------------------------------------------------------------
int pow2_at_least(long long v) { int r = 1; while (r < v) r <<= 1; return r; }

constexpr int kMostSets = 4 * kSms;           // blocks of a backward pass, each with a partial set

template <class T, int V, int VPT, bool SHIFT, bool CK> int run_fwd_rows(const NormArgs& a, int tpr, LaunchStream ls)
{
    const int threads = tpr > kRowThreads ? tpr : kRowThreads, per = threads / tpr;
    const long long want = (a.rows + per - 1) / per, most = (long long)kSms * (2048 / threads);
    launch(norm_fwd_rows_kernel<T, V, VPT, SHIFT, CK>, dim3((unsigned)(want < most ? want : most)), dim3(threads), 0, ls, a, tpr);
    return launched();
}
template <class T, int V, bool SHIFT, bool CK> int pick_fwd_rows(const NormArgs& a, LaunchStream ls)
{
    const long long vecs = (a.c + (SHIFT ? V - 1 : 0) + V - 1) / V;
    const int least = V == 1 ? 32 : 8;
    auto group = [&](int vpt) { const int t = pow2_at_least((vecs + vpt - 1) / vpt); return t < least ? least : t; };
    if constexpr (V == 1) {
        if (vecs <= 4 * 1024) return run_fwd_rows<T, V, 4, SHIFT, CK>(a, group(4), ls);
        if (vecs <= 16 * 1024) return run_fwd_rows<T, V, 16, SHIFT, CK>(a, group(16), ls);
    } else {
        if (vecs <= 512) return run_fwd_rows<T, V, 1, SHIFT, CK>(a, group(1), ls);
        if (vecs <= 2 * 1024) return run_fwd_rows<T, V, 2, SHIFT, CK>(a, group(2), ls);
        if (vecs <= 8 * 1024) return run_fwd_rows<T, V, 8, SHIFT, CK>(a, group(8), ls);
    }
    launch(norm_fwd_long_rows_kernel<T, CK>, dim3((unsigned)(a.rows < 2 * kSms ? a.rows : 2 * kSms)), dim3(1024), 0, ls, a);
    return launched();
}
template <class T, bool CK> int fwd_rows(const NormArgs& a, LaunchStream ls)
{
    constexpr int V = 16 / sizeof(T);
    const bool one = a.rows == 1;
    const bool on_grid = aligned(a.x, 16) && aligned(a.out, 16) && (one || (a.x_stride % V == 0 && a.out_stride % V == 0));
    const bool same = ((reinterpret_cast<uintptr_t>(a.x) ^ reinterpret_cast<uintptr_t>(a.out)) & 15) == 0 &&
                      (one || (a.x_stride - a.out_stride) % V == 0);
    if (on_grid) return pick_fwd_rows<T, V, false, CK>(a, ls);
    if constexpr (!CK)
        if (same) return pick_fwd_rows<T, V, true, false>(a, ls);
    return pick_fwd_rows<T, 1, false, CK>(a, ls);
}

int sum_sets(const NormArgs& a, int sets, float* dweight, float* dbias, LaunchStream ls)
{
    if (!a.partials) return launched();
    launch(norm_reduce_kernel, dim3((unsigned)((2LL * a.c + 31) / 32)), dim3(256), 0, ls, (const float*)a.partials, sets, a.c, dweight, dbias);
    return launched();
}

template <class T, int V, int VPT, bool CK> int run_bwd_rows(const NormArgs& a, int tpr, float* dweight, float* dbias, LaunchStream ls)
{
    const int threads = tpr > kRowThreads ? tpr : kRowThreads, per = threads / tpr;
    const size_t smem = a.partials ? (size_t)threads * VPT * V * 4 : 0;
    const long long want = (a.rows + per - 1) / per;
    const long long most = threads <= 256 ? 4 * kSms : threads <= 512 ? 2 * kSms : kSms;
    const int blocks = (int)(want < most ? want : most);
    if (!allow_smem(norm_bwd_rows_kernel<T, V, VPT, CK>, smem)) return FTP_ERR_CUDA;
    launch(norm_bwd_rows_kernel<T, V, VPT, CK>, dim3(blocks), dim3(threads), smem, ls, a, tpr);
    return sum_sets(a, blocks, dweight, dbias, ls);
}
template <class T, int V, bool CK> int pick_bwd_rows(const NormArgs& a, float* dweight, float* dbias, LaunchStream ls)
{
    const long long vecs = (a.c + V - 1) / V;
    const int least = V == 1 ? 32 : 8;
    auto group = [&](int vpt) { const int t = pow2_at_least((vecs + vpt - 1) / vpt); return t < least ? least : t; };
    if constexpr (V == 1) {
        if (vecs <= 4 * 1024) return run_bwd_rows<T, V, 4, CK>(a, group(4), dweight, dbias, ls);
        if (vecs <= 16 * 512) return run_bwd_rows<T, V, 16, CK>(a, group(16), dweight, dbias, ls);
    } else {
        if (vecs <= 1024) return run_bwd_rows<T, V, 1, CK>(a, group(1), dweight, dbias, ls);
        if (vecs <= 4 * 512) return run_bwd_rows<T, V, 4, CK>(a, group(4), dweight, dbias, ls);
    }
    const int blocks = (int)(a.rows < 2 * kSms ? a.rows : 2 * kSms);
    launch(norm_bwd_long_rows_kernel<T, CK>, dim3(blocks), dim3(1024), 0, ls, a);
    return sum_sets(a, blocks, dweight, dbias, ls);
}
template <class T, bool CK> int bwd_rows(const NormArgs& a, float* dweight, float* dbias, LaunchStream ls)
{
    constexpr int V = 16 / sizeof(T);
    auto on_grid = [&](const void* p, long long stride) { return !p || (aligned(p, 16) && (a.rows == 1 || stride % V == 0)); };
    if (on_grid(a.x, a.x_stride) && on_grid(a.dy, a.dy_stride) && on_grid(a.out, a.out_stride))
        return pick_bwd_rows<T, V, CK>(a, dweight, dbias, ls);
    return pick_bwd_rows<T, 1, CK>(a, dweight, dbias, ls);
}

// Tile shape of maps: as many lanes along the pixels as leave a thread at most `most` channels, but tiles of 32 pixels at least.
struct MapShapeOf { int lp, threads, cpt; };
MapShapeOf map_shape(int c, int V, int most)
{
    MapShapeOf m{32, kMapThreads, 0};
    auto per = [&] { return (c + m.threads / m.lp - 1) / (m.threads / m.lp); };
    while (per() > 4 && m.lp * V > 32) m.lp >>= 1;
    if (per() > most) m.threads = 512;
    m.cpt = per();
    return m;
}

template <class T, int V, bool CK> int fwd_map(const NormArgs& a, LaunchStream ls)
{
    const MapShapeOf m = map_shape(a.c, V, 16);
    const long long tiles = (a.p + m.lp * V - 1) / (m.lp * V), all = a.n * tiles;
    const size_t smem = 2 * (size_t)(m.threads / 32) * m.lp * V * 4;
    auto go = [&](auto kernel, int per_sm) {
        const long long most = (long long)kSms * per_sm;
        if (!allow_smem(kernel, smem)) return (int)FTP_ERR_CUDA;
        launch(kernel, dim3((unsigned)(all < most ? all : most)), dim3(m.threads), smem, ls, a, m.lp, (int)tiles);
        return launched();
    };
    if (m.cpt <= 1) return go(norm_fwd_map_kernel<T, V, 1, CK>, 8);
    if (m.cpt <= 4) return go(norm_fwd_map_kernel<T, V, 4, CK>, 6);
    if (m.cpt <= 16) return go(norm_fwd_map_kernel<T, V, 16, CK>, 2);
    return go(norm_fwd_map_kernel<T, V, 0, CK>, 4);
}
template <class T, int V, bool CK> int bwd_map(const NormArgs& a, float* dweight, float* dbias, LaunchStream ls)
{
    const MapShapeOf m = map_shape(a.c, V, 8);
    const long long tiles = (a.p + m.lp * V - 1) / (m.lp * V), all = a.n * tiles;
    const size_t smem = 4 * (size_t)(m.threads / 32) * m.lp * V * 4;
    auto go = [&](auto kernel, int per_sm) {
        const long long most = (long long)kSms * per_sm;
        const int blocks = (int)(all < most ? all : most);
        if (!allow_smem(kernel, smem)) return (int)FTP_ERR_CUDA;
        launch(kernel, dim3(blocks), dim3(m.threads), smem, ls, a, m.lp, (int)tiles);
        return sum_sets(a, blocks, dweight, dbias, ls);
    };
    if (m.cpt <= 1) return go(norm_bwd_map_kernel<T, V, 1, CK>, 4);
    if (m.cpt <= 4) return go(norm_bwd_map_kernel<T, V, 4, CK>, 4);
    if (m.cpt <= 8) return go(norm_bwd_map_kernel<T, V, 8, CK>, 2);
    return go(norm_bwd_map_kernel<T, V, 0, CK>, 3);
}

// The widest vector of pixels that divides a plane and lies on its own grid in every array.
template <class T> int map_vector(const NormArgs& a, int most)
{
    auto fits = [&](const void* p, long long stride, int v) { return !p || (aligned(p, v * sizeof(T)) && (a.n == 1 || stride % v == 0)); };
    for (int v = most; v > 1; v = v == 8 ? 2 : 1)
        if (a.p % v == 0 && fits(a.x, a.x_stride, v) && fits(a.dy, a.dy_stride, v) && fits(a.out, a.out_stride, v)) return v;
    return 1;
}

template <class T, bool CK> int forward(const NormArgs& a, LaunchStream ls)
{
    if (a.p == 1) return fwd_rows<T, CK>(a, ls);
    if constexpr (sizeof(T) == 4)
        return map_vector<T>(a, 4) == 4 ? fwd_map<T, 4, CK>(a, ls) : fwd_map<T, 1, CK>(a, ls);
    else {
        const int v = map_vector<T>(a, 8);
        return v == 8 ? fwd_map<T, 8, CK>(a, ls) : v == 2 ? fwd_map<T, 2, CK>(a, ls) : fwd_map<T, 1, CK>(a, ls);
    }
}
template <class T, bool CK> int backward(const NormArgs& a, float* dweight, float* dbias, LaunchStream ls)
{
    if (a.p == 1) return bwd_rows<T, CK>(a, dweight, dbias, ls);
    if constexpr (sizeof(T) == 4)
        return map_vector<T>(a, 4) == 4 ? bwd_map<T, 4, CK>(a, dweight, dbias, ls) : bwd_map<T, 1, CK>(a, dweight, dbias, ls);
    else {
        const int v = map_vector<T>(a, 8);
        return v == 8 ? bwd_map<T, 8, CK>(a, dweight, dbias, ls)
             : v == 2 ? bwd_map<T, 2, CK>(a, dweight, dbias, ls) : bwd_map<T, 1, CK>(a, dweight, dbias, ls);
    }
}
template <class T> int forward(const NormArgs& a, bool ck, LaunchStream ls) { return ck ? forward<T, true>(a, ls) : forward<T, false>(a, ls); }
template <class T> int backward(const NormArgs& a, bool ck, float* dw, float* db, LaunchStream ls)
{
    return ck ? backward<T, true>(a, dw, db, ls) : backward<T, false>(a, dw, db, ls);
}

size_t workspace_bytes(const ftp_dims* d) { return (size_t)kMostSets * 2 * (size_t)d->c * 4; }

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
                        cudaMemsetAsync(dbias, 0, (size_t)d->c * 4, st) != cudaSuccess)) return FTP_ERR_CUDA;
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
