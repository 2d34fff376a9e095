// 8-bit checkpoints on their own (ftp_ckpt_bytes, ftp_ckpt_save, ftp_ckpt_load); format and arithmetic in arrays.cuh.
//
// Both are bound by memory.  A warp takes segments of a run, all values of a segment in registers; the 32 values of a block lie in
// 32 / V neighbouring lanes, whose largest magnitude takes log2(32 / V) exchanges.  Where runs are whole blocks and the array is
// dense, the array is one run: the blocks are the same.
#include "arrays.cuh"

using namespace ftp;
using namespace ftp::arr;

namespace {

struct CkptArgs {
    void* x;
    const void* end;                // behind the array's last value
    CkptView ck;
    long long runs, len;            // runs of `len` values
    long long run_stride;           // between runs of a sample
    long long sample_stride;        // between samples
    long long per_sample;           // runs of a sample
};

constexpr int kThreads = 256;
constexpr int kPer = 4;             // vectors of a lane in a segment

// SHIFT: runs start at any multiple of the value's size, o values behind the 16-byte grid.  What is saved is read on the grid and moved
// to the run's own columns, with the next lane's word; what is loaded lies on the grid and takes its steps from two words of the run.
template <class T, int V, bool SAVE, bool SHIFT> __global__ void __launch_bounds__(kThreads) ckpt_kernel(CkptArgs a, int segments)
{
    previous_launches();
    constexpr int kSegment = 32 * V * kPer;
    const int lane = threadIdx.x & 31;
    for (Walk w(blockIdx.x * (kThreads / 32) + (threadIdx.x >> 5), gridDim.x * (kThreads / 32), segments); w.hi < a.runs; w.advance()) {
        const long long run = w.hi, start = (long long)w.lo * kSegment;
        const long long n = a.per_sample == 1 ? run : run / a.per_sample;
        // from here on places are relative to the segment
        T* x = static_cast<T*>(a.x) + n * a.sample_stride + (run - n * a.per_sample) * a.run_stride + start;
        const int o = SHIFT ? (int)((reinterpret_cast<uintptr_t>(x) / sizeof(T)) & (V - 1)) : 0;
        unsigned char* q = a.ck.q + run * a.ck.pitch + start;
        unsigned char* steps = a.ck.steps + run * a.ck.blocks + (start >> 5);
        const long long left = a.len - start, room = a.ck.pitch - start;
        const int len = (int)(left < kSegment + V ? left : kSegment + V), padded = (int)(room < kSegment ? room : kSegment);
        if constexpr (SAVE) {
            Pack<T, V> raw[kPer];
            const Reach<T, V> in = reach<T, V>(x, o, o + len, static_cast<const T*>(a.x), static_cast<const T*>(a.end));
#pragma unroll
            for (int i = 0; i < kPer; ++i) {
                raw[i] = zero_pack<T, V>();
                load_whole<T, V>(raw[i], x - o, (i * 32 + lane) * V, in.lo, in.hi);
            }
            if (SHIFT || len % V) {
                if (!in.all) {
#pragma unroll
                    for (int i = 0; i < kPer; ++i) load_rest<T, V>(raw[i], x - o, (i * 32 + lane) * V, o, o + len);
                }
#pragma unroll
                for (int i = 0; i < kPer; ++i) keep_part<T, V>(raw[i], (i * 32 + lane) * V, o, o + len, from_f<T>(0.f));
            }
            if constexpr (SHIFT) {
                Pack<T, V> after[kPer];
#pragma unroll
                for (int i = 0; i < kPer; ++i) {
                    const Pack<T, V> next = from_next_lane(raw[i]);
                    after[i] = zero_pack<T, V>();
                    if (lane == 31) load_whole<T, V>(after[i], x - o, (i * 32 + 32) * V, in.lo, in.hi);
                    else after[i] = next;
                }
#pragma unroll
                for (int i = 0; i < kPer; ++i)
                    if (lane == 31) {
                        if (!in.all) load_rest<T, V>(after[i], x - o, (i * 32 + 32) * V, o, o + len);
                        keep_part<T, V>(after[i], (i * 32 + 32) * V, o, o + len, from_f<T>(0.f));
                    }
#pragma unroll
                for (int i = 0; i < kPer; ++i) raw[i] = window<T, V>(raw[i], after[i], o);
            }
            // every block as if it held finite values only, then the others again
            float big[kPer];
            bool any = false;
#pragma unroll
            for (int i = 0; i < kPer; ++i) {
                big[i] = largest(values(raw[i]));
                any |= special<T>(big[i]);
            }
#pragma unroll
            for (int i = 0; i < kPer; ++i) {
                const int e = (i * 32 + lane) * V;
                const unsigned ex = step_exponent(big[i]);
                if (e < padded) {
                    store_pack<unsigned char, V>(q + e, to_steps(values(raw[i]), ex));
                    if (lane % (kBlock / V) == 0) steps[(unsigned)e >> 5] = (unsigned char)ex;
                }
            }
            if (!__any_sync(0xffffffffu, any)) continue;
#pragma unroll
            for (int i = 0; i < kPer; ++i) {
                const int e = (i * 32 + lane) * V;
                if (!special<T>(big[i])) continue;
                unsigned ex;
                const Pack<unsigned char, V> b = to_steps_special<T, V>(values(raw[i]), ex);
                if (e < padded) {
                    store_pack<unsigned char, V>(q + e, b);
                    if (lane % (kBlock / V) == 0) steps[(unsigned)e >> 5] = (unsigned char)ex;
                }
            }
        } else if constexpr (SHIFT) {
            // places of the run's grid, o of which lie before it; columns of the whole run, of which this is the part from `start` on
            const unsigned char *q0 = q - start, *steps0 = steps - (start >> 5);
            const long long all_places = a.len + o - start;
            const int hi = (int)(all_places < kSegment ? all_places : kSegment), lo = start == 0 ? o : 0;
            ShiftedSteps<V> in[kPer];
#pragma unroll
            for (int i = 0; i < kPer; ++i) {
                const int e = (i * 32 + lane) * V;
                if (e >= hi) continue;
                if (o == 0) { in[i].hi = load_pack<unsigned char, V>(q + e); in[i].e0 = in[i].e1 = steps[(unsigned)e >> 5]; }
                else in[i].load(q0, steps0, (int)start + e - o, o, (int)a.ck.pitch);
            }
#pragma unroll
            for (int i = 0; i < kPer; ++i) {
                const int e = (i * 32 + lane) * V;
                if (e >= hi) continue;
                const Vals<V> v = o == 0 ? mul(steps_of(in[i].hi), all<V>(step_of(in[i].e0))) : mul(in[i].numbers(o), in[i].scales((int)start + e - o, 1.f));
                store_part<T, V>(x - o, e, lo, hi, rounded<T, V>(v));
            }
        } else {
            Pack<unsigned char, V> b[kPer];
            unsigned ex[kPer];
            const int hi = len < kSegment ? len : kSegment;
#pragma unroll
            for (int i = 0; i < kPer; ++i) {
                const int e = (i * 32 + lane) * V;
                ex[i] = 1;
                if (e < hi) { b[i] = load_pack<unsigned char, V>(q + e); ex[i] = steps[(unsigned)e >> 5]; }
            }
#pragma unroll
            for (int i = 0; i < kPer; ++i) {
                const int e = (i * 32 + lane) * V;
                if (e < hi) store_part<T, V>(x, e, 0, hi, rounded<T, V>(mul(steps_of(b[i]), all<V>(step_of(ex[i])))));
            }
        }
    }
}

template <class T, bool SAVE, bool SHIFT> int run(const CkptArgs& a, LaunchStream ls)
{
    constexpr int V = 16 / sizeof(T);
    const long long segment = 32 * V * kPer, places = SAVE ? a.ck.pitch : a.len + (SHIFT ? V - 1 : 0);
    const long long segments = (places + segment - 1) / segment, tasks = a.runs * segments;
    const long long want = (tasks + kThreads / 32 - 1) / (kThreads / 32), most = 8LL * kSms;
    launch(ckpt_kernel<T, V, SAVE, SHIFT>, dim3((unsigned)(want < most ? want : most)), dim3(kThreads), 0, ls, a, (int)segments);
    return launched();
}
template <class T, bool SAVE> int pick(const CkptArgs& a, LaunchStream ls)
{
    constexpr int V = 16 / sizeof(T);
    const bool grid = aligned(a.x, 16) && (a.runs == 1 || (a.run_stride % V == 0 && a.sample_stride % V == 0));
    return grid ? run<T, SAVE, false>(a, ls) : run<T, SAVE, true>(a, ls);
}

template <bool SAVE> int ckpt(const ftp_dims* d, const void* x, long long x_stride, const void* ck, void* stream)
{
    long long rows = 0;
    const int rc = check_dims(d, &rows);
    if (rc != FTP_OK) return rc;
    if (rows == 0) return FTP_OK;
    if (!x || !ck || !aligned(x, type_size(d->type)) || !aligned(ck, 16) || !fix_stride(d, &x_stride)) return FTP_ERR_ARG;
    CkptArgs a{};
    a.end = static_cast<const char*>(x) + ((d->n - 1) * x_stride + d->c * d->p) * type_size(d->type);
    a.x = const_cast<void*>(x); a.ck = ckpt_view(d, ck);
    a.len = run_length(d); a.runs = run_count(d); a.run_stride = a.len; a.sample_stride = x_stride; a.per_sample = d->p == 1 ? 1 : d->c;
    if (x_stride == d->c * d->p || d->n == 1) {
        a.per_sample = 1; a.sample_stride = a.len;            // runs lie one behind the other
        // (a run off the grid is walked with 32-bit columns)
        if (a.len % kBlock == 0 && a.runs * a.ck.blocks < (aligned(x, 16) ? 1LL << 31 : 1LL << 25)) {
            a.len *= a.runs; a.ck.pitch *= a.runs; a.ck.blocks *= (int)a.runs;
            a.runs = 1;
        }
    }
    const LaunchStream ls{static_cast<cudaStream_t>(stream), true};
    if (d->type == FTP_TYPE_F32) return pick<float, SAVE>(a, ls);
    if (d->type == FTP_TYPE_BF16) return pick<__nv_bfloat16, SAVE>(a, ls);
    return pick<__half, SAVE>(a, ls);
}

}  // namespace

extern "C" {

int ftp_ckpt_bytes(const ftp_dims* d, size_t* bytes)
{
    long long rows = 0;
    const int rc = check_dims(d, &rows);
    if (rc != FTP_OK) return rc;
    if (!bytes) return FTP_ERR_ARG;
    *bytes = rows ? (size_t)run_count(d) * (size_t)((run_length(d) + kBlock - 1) / kBlock) * (kBlock + 1) : 0;
    return FTP_OK;
}

int ftp_ckpt_save(const ftp_dims* d, const void* x, long long x_stride, void* ck, void* stream)
{
    return ckpt<true>(d, x, x_stride, ck, stream);
}

int ftp_ckpt_load(const ftp_dims* d, const void* ck, void* x, long long x_stride, void* stream)
{
    return ckpt<false>(d, x, x_stride, ck, stream);
}

}  // extern "C"
