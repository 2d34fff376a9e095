// What the operators on arrays [n, c, p] share (norm.cu, ckpt.cu, logprob.cu): types, vectors of 16 bytes, sums over a group of
// threads, the 8-bit checkpoint's arithmetic, host checks.
//
// An array is n samples of c channels of p pixels, each sample dense, `stride` elements from one sample to the next; p = 1 is
// a matrix of n rows.  Values are fp32, bf16 or fp16; every sum and statistic is held in fp32.
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>

#include <cstdint>

#include "ftp.h"
#include "launch.cuh"

namespace ftp {
namespace arr {

constexpr int kSms = 148;                     // multiprocessors of a B200: the unit of the persistent grids

// ---- values -----------------------------------------------------------------------------------------------------
__device__ __forceinline__ float to_f(float v) { return v; }
__device__ __forceinline__ float to_f(__nv_bfloat16 v) { return __bfloat162float(v); }
__device__ __forceinline__ float to_f(__half v) { return __half2float(v); }
template <class T> __device__ __forceinline__ T from_f(float v);
template <> __device__ __forceinline__ float from_f<float>(float v) { return v; }
template <> __device__ __forceinline__ __nv_bfloat16 from_f<__nv_bfloat16>(float v) { return __float2bfloat16_rn(v); }
template <> __device__ __forceinline__ __half from_f<__half>(float v) { return __float2half_rn(v); }

__device__ __forceinline__ unsigned bits_of(float v) { return __float_as_uint(v); }
__device__ __forceinline__ unsigned bits_of(__nv_bfloat16 v) { return __bfloat16_as_ushort(v); }
__device__ __forceinline__ unsigned bits_of(__half v) { return __half_as_ushort(v); }
__device__ __forceinline__ unsigned bits_of(unsigned char v) { return v; }
template <class T> __device__ __forceinline__ T of_bits(unsigned b);
template <> __device__ __forceinline__ float of_bits<float>(unsigned b) { return __uint_as_float(b); }
template <> __device__ __forceinline__ __nv_bfloat16 of_bits<__nv_bfloat16>(unsigned b) { return __ushort_as_bfloat16((unsigned short)b); }
template <> __device__ __forceinline__ __half of_bits<__half>(unsigned b) { return __ushort_as_half((unsigned short)b); }
template <> __device__ __forceinline__ unsigned char of_bits<unsigned char>(unsigned b) { return (unsigned char)b; }

// V values side by side, moved as one word of up to 16 bytes.  They are kept as the 32-bit registers that they come in: an array of 16-bit
// values the compiler takes apart and puts together again wherever paths meet (log probabilities of 4096 x 32000 bf16, a warp a row: 65 M
// instructions and 652 bytes of spills that way, 55 M and 76 this way; 144 and 120 us).
template <class T, int V> struct Pack {
    static constexpr int kBits = 8 * sizeof(T), kPer = 32 / kBits, kWords = (V + kPer - 1) / kPer;
    unsigned w[kWords];
    __device__ __forceinline__ T get(int j) const { return of_bits<T>(kBits == 32 ? w[j] : w[j / kPer] >> (kBits * (j % kPer))); }
    __device__ __forceinline__ void set(int j, T v)
    {
        if constexpr (kBits == 32) w[j] = bits_of(v);
        else {
            const unsigned at = kBits * (j % kPer), mask = ((1u << (kBits % 32)) - 1u) << at;
            w[j / kPer] = (w[j / kPer] & ~mask) | (bits_of(v) << at);
        }
    }
};

template <class T, int V> __device__ __forceinline__ Pack<T, V> load_pack(const T* p)
{
    constexpr int kBytes = sizeof(T) * V;
    Pack<T, V> r;
    if constexpr (kBytes == 16) { const uint4 q = *reinterpret_cast<const uint4*>(p); r.w[0] = q.x; r.w[1] = q.y; r.w[2] = q.z; r.w[3] = q.w; }
    else if constexpr (kBytes == 8) { const uint2 q = *reinterpret_cast<const uint2*>(p); r.w[0] = q.x; r.w[1] = q.y; }
    else if constexpr (kBytes == 4) r.w[0] = *reinterpret_cast<const unsigned*>(p);
    else if constexpr (kBytes == 2) r.w[0] = *reinterpret_cast<const unsigned short*>(p);
    else r.w[0] = *reinterpret_cast<const unsigned char*>(p);
    return r;
}
template <class T, int V> __device__ __forceinline__ void store_pack(T* p, const Pack<T, V>& a)
{
    constexpr int kBytes = sizeof(T) * V;
    if constexpr (kBytes == 16) *reinterpret_cast<uint4*>(p) = make_uint4(a.w[0], a.w[1], a.w[2], a.w[3]);
    else if constexpr (kBytes == 8) *reinterpret_cast<uint2*>(p) = make_uint2(a.w[0], a.w[1]);
    else if constexpr (kBytes == 4) *reinterpret_cast<unsigned*>(p) = a.w[0];
    else if constexpr (kBytes == 2) *reinterpret_cast<unsigned short*>(p) = (unsigned short)a.w[0];
    else *reinterpret_cast<unsigned char*>(p) = (unsigned char)a.w[0];
}
template <class T, int V> __device__ __forceinline__ Pack<T, V> zero_pack()
{
    Pack<T, V> r;
#pragma unroll
    for (int j = 0; j < Pack<T, V>::kWords; ++j) r.w[j] = 0u;
    return r;
}

// Keeps 16-bit values packed: without it the compiler holds on to their fp32 forms between two passes, in twice the registers.
template <class T, int V> __device__ __forceinline__ void keep_packed(Pack<T, V>& a)
{
    if constexpr (sizeof(T) == 2 && V % 2 == 0) {
#pragma unroll
        for (int j = 0; j < Pack<T, V>::kWords; ++j) asm volatile("" : "+r"(a.w[j]));
    }
}

// Values [e, e + V) of a row of which only [lo, hi) exist, `base` aligned for whole words; what does not exist reads as `fill` and is
// not written.  Words that lie across an end of the row come in three steps, so that no branch stands between any two loads and none is
// waited for before it is used: load_whole of all a thread's words, each one predicated instruction, with the bounds that reach()
// widens where the neighbouring memory is the array's too; load_rest, value by value, for the first and last rows, where it is not;
// and keep_part, where the values are used, which puts `fill` in the places that are not the row's.  Places are ints, relative to the
// row or segment: wide ones cost more than the arithmetic.
template <class T, int V> struct Reach {
    int lo, hi;          // of load_whole
    bool all;            // nothing is left to load_rest
};
// `row`: first value of the row, `count` values; [begin, end) the array, from its first value to its last.
template <class T, int V> __device__ __forceinline__ Reach<T, V> reach(const T* row, int lo, int hi, const T* begin, const T* end)
{
    const bool before = row - begin >= V, behind = end - (row + (hi - lo)) >= V;
    return {before ? lo - (V - 1) : lo, behind ? hi + V - 1 : hi, before && behind};
}
template <class T, int V> __device__ __forceinline__ void keep_part(Pack<T, V>& r, int e, int lo, int hi, T fill)
{
    if (V > 1 && (e < lo || e + V > hi)) {
#pragma unroll
        for (int j = 0; j < V; ++j)
            if (e + j < lo || e + j >= hi) r.set(j, fill);
    }
}
template <class T, int V> __device__ __forceinline__ Pack<T, V> filled(T fill)
{
    Pack<T, V> r;
    const unsigned b = sizeof(T) == 2 ? bits_of(fill) * 0x10001u : bits_of(fill);
#pragma unroll
    for (int j = 0; j < Pack<T, V>::kWords; ++j) r.w[j] = b;
    return r;
}
template <class T, int V> __device__ __forceinline__ void load_whole(Pack<T, V>& r, const T* base, int e, int lo, int hi)
{
    if (e >= lo && e + V <= hi) r = load_pack<T, V>(base + e);
}
template <class T, int V> __device__ __forceinline__ void load_rest(Pack<T, V>& r, const T* base, int e, int lo, int hi)
{
    if (V > 1 && e < hi && e + V > lo && (e < lo || e + V > hi)) {
#pragma unroll
        for (int j = 0; j < V; ++j)
            if (e + j >= lo && e + j < hi) r.set(j, base[e + j]);
    }
}
template <class T, int V> __device__ __forceinline__ void store_part(T* base, int e, int lo, int hi, const Pack<T, V>& a)
{
    if (e >= lo && e + V <= hi) { store_pack<T, V>(base + e, a); return; }
#pragma unroll
    for (int j = 0; j < V; ++j)
        if (e + j >= lo && e + j < hi) base[e + j] = a.get(j);
}

// Values [o, o + V) of the 2 V in `lo` and `hi`, 0 <= o < V: a vector that lies across two words of the grid.
template <class T, int V> __device__ __forceinline__ Pack<T, V> window(const Pack<T, V>& lo, const Pack<T, V>& hi, int o)
{
    constexpr int N = Pack<T, V>::kWords;
    static_assert(sizeof(T) * V >= 4, "whole words");
    const unsigned bytes = (unsigned)o * sizeof(T), bits = (bytes & 3u) * 8u;
    unsigned w[2 * N + 1];
#pragma unroll
    for (int j = 0; j < N; ++j) { w[j] = lo.w[j]; w[N + j] = hi.w[j]; }
    w[2 * N] = 0u;
#pragma unroll
    for (int d = 1; d < N; d <<= 1) {
        const bool move = (bytes >> 2) & d;
#pragma unroll
        for (int j = 0; j + d <= 2 * N; ++j) w[j] = move ? w[j + d] : w[j];
    }
    Pack<T, V> r;
#pragma unroll
    for (int j = 0; j < N; ++j) r.w[j] = __funnelshift_r(w[j], w[j + 1], bits);
    return r;
}
// The pack of the next lane.
template <class T, int V> __device__ __forceinline__ Pack<T, V> from_next_lane(const Pack<T, V>& a)
{
    Pack<T, V> r;
#pragma unroll
    for (int j = 0; j < Pack<T, V>::kWords; ++j) r.w[j] = __shfl_down_sync(0xffffffffu, a.w[j], 1);
    return r;
}

// V values as fp32, in pairs where V is even: the packed fp32 instructions of sm_100 do two values in one issue slot, and all of
// the kernels here are closer to the issue rate than to anything else but memory.
template <int V> struct Vals { float v[V]; };

template <int V> __device__ __forceinline__ Vals<V> all(float s)
{
    Vals<V> r;
#pragma unroll
    for (int j = 0; j < V; ++j) r.v[j] = s;
    return r;
}
template <int V> __device__ __forceinline__ Vals<V> fma(const Vals<V>& a, const Vals<V>& b, const Vals<V>& c)
{
    Vals<V> r;
    if constexpr (V % 2 == 0) {
#pragma unroll
        for (int j = 0; j < V; j += 2) {
            const float2 d = __ffma2_rn(make_float2(a.v[j], a.v[j + 1]), make_float2(b.v[j], b.v[j + 1]), make_float2(c.v[j], c.v[j + 1]));
            r.v[j] = d.x; r.v[j + 1] = d.y;
        }
    } else {
#pragma unroll
        for (int j = 0; j < V; ++j) r.v[j] = fmaf(a.v[j], b.v[j], c.v[j]);
    }
    return r;
}
template <int V> __device__ __forceinline__ Vals<V> add(const Vals<V>& a, const Vals<V>& b)
{
    Vals<V> r;
    if constexpr (V % 2 == 0) {
#pragma unroll
        for (int j = 0; j < V; j += 2) {
            const float2 d = __fadd2_rn(make_float2(a.v[j], a.v[j + 1]), make_float2(b.v[j], b.v[j + 1]));
            r.v[j] = d.x; r.v[j + 1] = d.y;
        }
    } else {
#pragma unroll
        for (int j = 0; j < V; ++j) r.v[j] = a.v[j] + b.v[j];
    }
    return r;
}
template <int V> __device__ __forceinline__ Vals<V> mul(const Vals<V>& a, const Vals<V>& b)
{
    Vals<V> r;
    if constexpr (V % 2 == 0) {
#pragma unroll
        for (int j = 0; j < V; j += 2) {
            const float2 d = __fmul2_rn(make_float2(a.v[j], a.v[j + 1]), make_float2(b.v[j], b.v[j + 1]));
            r.v[j] = d.x; r.v[j + 1] = d.y;
        }
    } else {
#pragma unroll
        for (int j = 0; j < V; ++j) r.v[j] = a.v[j] * b.v[j];
    }
    return r;
}
template <int V> __device__ __forceinline__ float sum_of(const Vals<V>& a)
{
    if constexpr (V >= 4) {
        Vals<V / 2> lo, hi;
#pragma unroll
        for (int j = 0; j < V / 2; ++j) { lo.v[j] = a.v[j]; hi.v[j] = a.v[j + V / 2]; }
        return sum_of(add(lo, hi));
    } else if constexpr (V == 2) return a.v[0] + a.v[1];
    else return a.v[0];
}

template <int V> __device__ __forceinline__ Vals<V> values(const Pack<float, V>& p)
{
    Vals<V> r;
#pragma unroll
    for (int j = 0; j < V; ++j) r.v[j] = __uint_as_float(p.w[j]);
    return r;
}
template <int V> __device__ __forceinline__ Vals<V> values(const Pack<__nv_bfloat16, V>& p)
{
    Vals<V> r;
#pragma unroll
    for (int j = 0; j < V; ++j) r.v[j] = __uint_as_float(j % 2 ? p.w[j / 2] & 0xffff0000u : p.w[j / 2] << 16);
    return r;
}
template <int V> __device__ __forceinline__ Vals<V> values(const Pack<__half, V>& p)
{
    Vals<V> r;
    if constexpr (V == 1) r.v[0] = to_f(p.get(0));
    else {
#pragma unroll
        for (int j = 0; j < V; j += 2) {
            const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&p.w[j / 2]));
            r.v[j] = f.x; r.v[j + 1] = f.y;
        }
    }
    return r;
}
// Rounds V values to the array's type, two to an instruction where it has one.
template <class T, int V> __device__ __forceinline__ Pack<T, V> rounded(const Vals<V>& a)
{
    Pack<T, V> r;
    if constexpr (sizeof(T) == 2 && V % 2 == 0) {
#pragma unroll
        for (int j = 0; j < V; j += 2) {
            if constexpr (__is_same(T, __nv_bfloat16)) {
                const __nv_bfloat162 w = __floats2bfloat162_rn(a.v[j], a.v[j + 1]);
                r.w[j / 2] = *reinterpret_cast<const unsigned*>(&w);
            } else {
                const __half2 w = __floats2half2_rn(a.v[j], a.v[j + 1]);
                r.w[j / 2] = *reinterpret_cast<const unsigned*>(&w);
            }
        }
    } else {
#pragma unroll
        for (int j = 0; j < V; ++j) r.w[j] = bits_of(from_f<T>(a.v[j]));
    }
    return r;
}

// Index hi * n + lo, walked in equal steps without a division for each (64 bits of one are a hundred instructions).
struct Walk {
    long long hi;
    int lo, n, step_hi, step_lo;
    __device__ __forceinline__ Walk(unsigned start, unsigned step, int n_) : n(n_)
    {
        hi = start / (unsigned)n; lo = (int)(start % (unsigned)n);
        step_hi = (int)(step / (unsigned)n); step_lo = (int)(step % (unsigned)n);
    }
    __device__ __forceinline__ void advance()
    {
        hi += step_hi; lo += step_lo;
        if (lo >= n) { lo -= n; ++hi; }
    }
};

// ---- sums -------------------------------------------------------------------------------------------------------
// Sum over `width` neighbouring lanes (a power of two); every lane has it.
__device__ __forceinline__ float lanes_sum(float v, int width = 32)
{
#pragma unroll
    for (int d = 16; d >= 1; d >>= 1)
        if (d < width) v += __shfl_xor_sync(0xffffffffu, v, d);
    return v;
}
__device__ __forceinline__ float lanes_max(float v, int width = 32)
{
#pragma unroll
    for (int d = 16; d >= 1; d >>= 1)
        if (d < width) v = fmaxf(v, __shfl_xor_sync(0xffffffffu, v, d));
    return v;
}
// Barrier of `threads` threads (whole warps) of the block; groups of one block use numbers of their own, 1 to 15.
__device__ __forceinline__ void group_barrier(int number, int threads)
{
    asm volatile("bar.sync %0, %1;" ::"r"(number), "r"(threads) : "memory");
}
// Barrier of all warps of the block, from whichever place of the program each comes to it.
__device__ __forceinline__ void block_barrier() { asm volatile("bar.sync 0;" ::: "memory"); }

__device__ __forceinline__ float max_nan(float a, float b) { float r; asm("max.NaN.f32 %0, %1, %2;" : "=f"(r) : "f"(a), "f"(b)); return r; }
__device__ __forceinline__ float nan_f() { return __uint_as_float(0x7fffffffu); }

// ---- the 8-bit checkpoint ---------------------------------------------------------------------------------------
// Blocks of 32 consecutive values of a row or plane: one byte e stands for the step 2^(e - 127), a signed byte q for the value
// q * step.  e is the least in [1, 249] with 127 * step >= the largest finite magnitude of the block, so q = round(x / step)
// is at most 127, both x / step and q * step are exact in fp32, and the value kept is the same bits in every implementation.
// q = -128 marks an infinity or NaN and reads as NaN.  64 * 2^122 and (fp16) 64 * 2^10 would be infinite: the largest finite
// values of a type are held to 63 steps.
constexpr int kBlock = 32;

// 127 * 2^k = 1.984375 * 2^(k + 6): the exponent field of the magnitude minus 6, one more if its fraction is above 0x7e0000.
__device__ __forceinline__ unsigned step_exponent(float largest)
{
    const int e = (int)((__float_as_uint(largest) + 0x1ffffu) >> 23) - 6;
    return e < 1 ? 1u : (unsigned)e;
}
__device__ __forceinline__ float step_of(unsigned e) { return __uint_as_float(e << 23); }
__device__ __forceinline__ float inverse_step(unsigned e) { return __uint_as_float((254u - e) << 23); }
// Blocks for which rounding alone is not all: an infinity or NaN in them, or a largest value that rounds to 64 steps of a step too large.
template <class T> __device__ __forceinline__ bool special(float largest)
{
    constexpr float last = sizeof(T) == 2 && !__is_same(T, __nv_bfloat16) ? 65024.f : 1.984375f * 0x1p127f;   // 127 of the last step that is not
    return !(largest <= last);
}

// Largest magnitude of a block that is spread, V values each, over 32 / V neighbouring lanes (all lanes of the warp take part); NaN if
// there is one among them.
template <int V> __device__ __forceinline__ float largest(const Vals<V>& x, unsigned lanes = 0xffffffffu)
{
    float big = fabsf(x.v[0]);
#pragma unroll
    for (int j = 1; j < V; ++j) big = max_nan(big, fabsf(x.v[j]));
    if constexpr (V == 1) return __uint_as_float(__reduce_max_sync(lanes, __float_as_uint(big)));     // (a NaN's bits are above all)
#pragma unroll
    for (int d = kBlock / V / 2; d >= 1; d >>= 1) big = max_nan(big, __shfl_xor_sync(lanes, big, d));
    return big;
}

// The steps of V values of a block that is not special().  Adding 1.5 * 2^23 rounds to the nearest integer, ties to even, and leaves it
// in the low byte.
template <int V> __device__ __forceinline__ Pack<unsigned char, V> to_steps(const Vals<V>& x, unsigned e)
{
    Pack<unsigned char, V> q;
    const Vals<V> s = fma(x, all<V>(inverse_step(e)), all<V>(12582912.f));
    if constexpr (V % 4 == 0) {
#pragma unroll
        for (int j = 0; j < V; j += 4) {
            const unsigned lo = __byte_perm(__float_as_uint(s.v[j]), __float_as_uint(s.v[j + 1]), 0x0040);
            const unsigned hi = __byte_perm(__float_as_uint(s.v[j + 2]), __float_as_uint(s.v[j + 3]), 0x0040);
            q.w[j / 4] = __byte_perm(lo, hi, 0x5410);
        }
    } else if constexpr (V == 2) q.w[0] = __byte_perm(__float_as_uint(s.v[0]), __float_as_uint(s.v[1]), 0x0040) & 0xffffu;
    else q.w[0] = __float_as_uint(s.v[0]) & 0xffu;
    return q;
}

// The same for a special block, by the lanes that hold it: largest finite magnitude, then each value by itself.
template <class T, int V> __device__ __noinline__ Pack<unsigned char, V> to_steps_special(const Vals<V> x, unsigned& e)
{
    constexpr int kLanes = kBlock / V;
    const unsigned lanes = kLanes == 32 ? 0xffffffffu : ((1u << (kLanes % 32)) - 1u) << (threadIdx.x & 31 & ~(kLanes - 1));
    Vals<V> finite;
#pragma unroll
    for (int j = 0; j < V; ++j) finite.v[j] = fabsf(x.v[j]) < INFINITY ? x.v[j] : 0.f;
    const float big = largest(finite, lanes);
    e = step_exponent(big);
    const float inverse = inverse_step(e), most = special<T>(big) ? 63.f : 127.f;
    Pack<unsigned char, V> q = zero_pack<unsigned char, V>();
#pragma unroll
    for (int j = 0; j < V; ++j) {
        const float s = fminf(fmaxf(finite.v[j] * inverse, -most), most) + 12582912.f;
        q.set(j, fabsf(x.v[j]) < INFINITY ? (unsigned char)__float_as_uint(s) : (unsigned char)0x80u);
    }
    return q;
}

// The steps as numbers: a byte plus 128 in the low bits of 2^23 is the float 2^23 + q + 128.  -128 becomes NaN.
template <int V> __device__ __forceinline__ Vals<V> steps_of(const Pack<unsigned char, V>& q)
{
    Vals<V> r;
    bool marked = false;
#pragma unroll
    for (int i = 0; i < Pack<unsigned char, V>::kWords; ++i) {
        const unsigned u = q.w[i] ^ 0x80808080u;
        constexpr int kHere = V < 4 ? V : 4;
        constexpr unsigned kTops = V >= 4 ? 0x80808080u : V == 2 ? 0x8080u : 0x80u;
#pragma unroll
        for (int k = 0; k < kHere; ++k) r.v[4 * i + k] = __uint_as_float(__byte_perm(u, 0x4b000000u, 0x7540 + k));
        marked |= ((u - 0x01010101u) & ~u & kTops) != 0u;      // a byte of u is 0
    }
    r = add(r, all<V>(-8388736.f));
    if (marked) {
#pragma unroll
        for (int j = 0; j < V; ++j)
            if (r.v[j] == -128.f) r.v[j] = nan_f();
    }
    return r;
}

// Steps of columns [col, col + V) of a run, col a multiple of V less o (0 < o < V): they lie across two words of the run and, it may be,
// across two blocks.  Columns before the run or behind its padding are 0.
template <int V> struct ShiftedSteps {
    Pack<unsigned char, V> lo, hi;
    unsigned e0, e1;
    __device__ __forceinline__ void load(const unsigned char* q, const unsigned char* steps, int col, int o, int padded)
    {
        const int at = col + o;
        lo = hi = zero_pack<unsigned char, V>();
        if (at >= V && at - V < padded) lo = load_pack<unsigned char, V>(q + at - V);
        if (at < padded) hi = load_pack<unsigned char, V>(q + at);
        e0 = steps[max(0, min(col, padded - 1)) / kBlock];
        e1 = steps[min(max(0, col + V - 1), padded - 1) / kBlock];
    }
    // the numbers of steps, and each one's step times `by`
    __device__ __forceinline__ Vals<V> numbers(int o) const { return steps_of(window<unsigned char, V>(lo, hi, V - o)); }
    __device__ __forceinline__ Vals<V> scales(int col, float by) const
    {
        const float s0 = step_of(e0) * by, s1 = step_of(e1) * by;
        const int second = (col + V - 1) & ~(kBlock - 1);            // first column of the block that the last one is in
        Vals<V> r;
#pragma unroll
        for (int j = 0; j < V; ++j) r.v[j] = col + j >= second ? s1 : s0;
        return r;
    }
};

// Where a checkpoint lies: q bytes of run r (a row or plane of `len` values) at r * pitch, its step bytes at steps + r * blocks.
struct CkptView {
    unsigned char* q;
    unsigned char* steps;
    long long pitch;
    int blocks;
};

// ---- host -------------------------------------------------------------------------------------------------------
inline int type_size(int type) { return type == FTP_TYPE_F32 ? 4 : 2; }

// FTP_OK with *rows = n * p (0: nothing to do), or an error.  Any count fits 62 bits after this.
inline int check_dims(const ftp_dims* d, long long* rows)
{
    if (!d || d->struct_size != (int)sizeof(ftp_dims)) return FTP_ERR_ARG;
    if (d->type != FTP_TYPE_F32 && d->type != FTP_TYPE_BF16 && d->type != FTP_TYPE_F16) return FTP_ERR_ARG;
    if (d->n < 0 || d->c < 1 || d->p < 0) return FTP_ERR_ARG;
    constexpr long long kMost = 1LL << 30;
    if (d->n >= kMost || d->c >= kMost || d->p >= kMost) return FTP_ERR_TOO_LARGE;
    if (d->n > 0 && d->p > 0) {
        const long long rows_ = d->n * d->p;
        if (rows_ >= (1LL << 40) || d->c > ((1LL << 46) / rows_)) return FTP_ERR_TOO_LARGE;
    }
    *rows = d->n * d->p;
    return FTP_OK;
}
// A sample stride of 0 stands for a dense array; any other must hold a sample.
inline bool fix_stride(const ftp_dims* d, long long* stride)
{
    const long long dense = d->c * d->p;
    if (*stride == 0) *stride = dense;
    return *stride >= dense && *stride < (1LL << 46) / (d->n > 0 ? d->n : 1);
}
inline bool aligned(const void* p, size_t to) { return (reinterpret_cast<uintptr_t>(p) & (to - 1)) == 0; }

// Runs that a checkpoint cuts into blocks: the rows of a matrix, or the planes of maps.
inline long long run_length(const ftp_dims* d) { return d->p == 1 ? d->c : d->p; }
inline long long run_count(const ftp_dims* d) { return d->p == 1 ? d->n : d->n * d->c; }
inline CkptView ckpt_view(const ftp_dims* d, const void* ckpt)
{
    CkptView v{};
    v.blocks = (int)((run_length(d) + kBlock - 1) / kBlock);
    v.pitch = (long long)v.blocks * kBlock;
    v.q = static_cast<unsigned char*>(const_cast<void*>(ckpt));
    v.steps = v.q ? v.q + run_count(d) * v.pitch : nullptr;
    return v;
}

// Dynamic shared memory of a launch; 48 KB together with the kernel's own (16 KB at most here) need no leave.  The leave is the process's, not
// the launch's: `most`, what any launch of this kernel takes, is the only value that it is ever given, so that no thread lowers it between another
// one's asking and its launch.
template <class K> inline bool allow_smem(K kernel, size_t bytes, size_t most)
{
    return bytes <= 32 * 1024 || (bytes <= most && cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)most) == cudaSuccess);
}
// Blocks of a kernel that an SM holds at once, from its registers (asked for once) and the launch's shared memory: persistent grids are
// that many an SM, or their last blocks would wait for the first to end.
template <auto K> inline int resident(int threads, size_t smem)
{
    static const cudaFuncAttributes at = [] { cudaFuncAttributes a{}; if (cudaFuncGetAttributes(&a, K) != cudaSuccess) a.numRegs = 255; return a; }();
    const int regs = (at.numRegs + 7) / 8 * 8;
    const size_t shared = smem + at.sharedSizeBytes + 1024;
    const int by_regs = 65536 / (regs * threads), by_smem = (int)(233472 / shared), by_threads = 2048 / threads;
    int n = by_regs < by_smem ? by_regs : by_smem;
    n = n < by_threads ? n : by_threads;
    return n < 1 ? 1 : n > 32 ? 32 : n;
}
inline int launched() { return cudaGetLastError() == cudaSuccess ? FTP_OK : FTP_ERR_CUDA; }
// A runtime call was refused: the error that it left with the thread is this call's, not the next one's.
inline int refused()
{
    cudaGetLastError();
    return FTP_ERR_CUDA;
}

}  // namespace arr
}  // namespace ftp
