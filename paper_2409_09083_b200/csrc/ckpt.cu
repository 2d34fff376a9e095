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
    CkptView ck;
    long long runs, len;            // runs of `len` values
    long long run_stride;           // between runs of a sample
    long long sample_stride;        // between samples
    long long per_sample;           // runs of a sample
};

constexpr int kThreads = 256;
constexpr int kPer = 4;             // vectors of a lane in a segment

template <class T, int V, bool SAVE> __global__ void __launch_bounds__(kThreads) ckpt_kernel(CkptArgs a, int segments)
{
    previous_launches();
    constexpr int kSegment = 32 * V * kPer;
    const int lane = threadIdx.x & 31;
    for (Walk w(blockIdx.x * (kThreads / 32) + (threadIdx.x >> 5), gridDim.x * (kThreads / 32), segments); w.hi < a.runs; w.advance()) {
        const long long run = w.hi, start = (long long)w.lo * kSegment;
        const long long n = a.per_sample == 1 ? run : run / a.per_sample;
        // from here on places are relative to the segment
        T* x = static_cast<T*>(a.x) + n * a.sample_stride + (run - n * a.per_sample) * a.run_stride + start;
        unsigned char* q = a.ck.q + run * a.ck.pitch + start;
        unsigned char* steps = a.ck.steps + run * a.ck.blocks + (start >> 5);
        const int len = (int)(a.len - start < kSegment ? a.len - start : kSegment), padded = (int)(a.ck.pitch - start < kSegment ? a.ck.pitch - start : kSegment);
        if constexpr (SAVE) {
            Pack<T, V> raw[kPer];
#pragma unroll
            for (int i = 0; i < kPer; ++i) {
                raw[i] = zero_pack<T, V>();
                load_whole<T, V>(raw[i], x, (i * 32 + lane) * V, 0, len);
            }
            if (V > 1 && len % V) {
#pragma unroll
                for (int i = 0; i < kPer; ++i) load_rest<T, V>(raw[i], x, (i * 32 + lane) * V, 0, len);
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
        } else {
            Pack<unsigned char, V> b[kPer];
            unsigned ex[kPer];
#pragma unroll
            for (int i = 0; i < kPer; ++i) {
                const int e = (i * 32 + lane) * V;
                ex[i] = 1;
                if (e < len) { b[i] = load_pack<unsigned char, V>(q + e); ex[i] = steps[(unsigned)e >> 5]; }
            }
#pragma unroll
            for (int i = 0; i < kPer; ++i) {
                const int e = (i * 32 + lane) * V;
                if (e < len) store_part<T, V>(x, e, 0, len, rounded<T, V>(mul(steps_of(b[i]), all<V>(step_of(ex[i])))));
            }
        }
    }
}

template <class T, int V, bool SAVE> int run(const CkptArgs& a, LaunchStream ls)
{
    const long long segment = 32 * V * kPer, segments = (a.ck.pitch + segment - 1) / segment, tasks = a.runs * segments;
    const long long want = (tasks + kThreads / 32 - 1) / (kThreads / 32), most = 8LL * kSms;
    launch(ckpt_kernel<T, V, SAVE>, dim3((unsigned)(want < most ? want : most)), dim3(kThreads), 0, ls, a, (int)segments);
    return launched();
}
template <class T, bool SAVE> int pick(const CkptArgs& a, LaunchStream ls)
{
    constexpr int V = 16 / sizeof(T);
    const bool grid = aligned(a.x, 16) && (a.runs == 1 || (a.run_stride % V == 0 && a.sample_stride % V == 0));
    return grid ? run<T, V, SAVE>(a, ls) : run<T, 1, SAVE>(a, ls);
}

template <bool SAVE> int ckpt(const ftp_dims* d, const void* x, long long x_stride, const void* ck, void* stream)
{
    long long rows = 0;
    const int rc = check_dims(d, &rows);
    if (rc != FTP_OK) return rc;
    if (rows == 0) return FTP_OK;
    if (!x || !ck || !aligned(x, type_size(d->type)) || !aligned(ck, 16) || !fix_stride(d, &x_stride)) return FTP_ERR_ARG;
    CkptArgs a{};
    a.x = const_cast<void*>(x); a.ck = ckpt_view(d, ck);
    a.len = run_length(d); a.runs = run_count(d); a.run_stride = a.len; a.sample_stride = x_stride; a.per_sample = d->p == 1 ? 1 : d->c;
    if (x_stride == d->c * d->p || d->n == 1) {
        a.per_sample = 1; a.sample_stride = a.len;            // runs lie one behind the other
        if (a.len % kBlock == 0 && a.runs * a.ck.blocks < (1LL << 31)) {
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
