// top_logits.cu -- the K largest logits of each row (sats_top_logits).
#include "internal.h"
#include "rows.cuh"

namespace sats {
namespace {
constexpr int kSelThreads = 512, kSelPerSm = 2;
}
}  // namespace sats
#include "logits.cuh"

namespace sats {
namespace {

struct TopParams {
    const void *z;
    int64_t ld;
    int T, V, K;
    float *values;
    int32_t *idx;
    int cluster, cached;
};

template <bool F32>
__global__ void __launch_bounds__(kSelThreads, kSelPerSm) top_kernel(const TopParams p)
{
    extern __shared__ __align__(16) uint4 smem[];
    __shared__ Shared sh;
    const int row = blockIdx.x / p.cluster;
    unsigned long long *list = reinterpret_cast<unsigned long long *>(smem + p.cached);
    Ctx<F32> c{Row<F32>(p.z, row, p.ld, p.V)};
    set_ctx(c, smem, p.cached, p.cluster, &sh);
    start_row(c, smem);
    uint32_t kmax, bound;
    load_row(c, smem, p.K, reinterpret_cast<uint32_t *>(list), &kmax, &bound);
    bool ok;
    int n = gather_list(c, list, bound, Cut{kKeyNone, INT_MIN}, &ok);
    if (!ok) {   // (the same in every CTA of the row)
        const Cut cut = cut_count(c, kmax, p.K);
        n = gather_list(c, list, max(cut.key, kKeyNone + 1), cut, &ok);   // at most K
    }
    if (c.rank != 0) return;   // (nobody reads this CTA's memory any more)
    if (n <= kSmall) {
        const Small e(list, n);
        const int at = e.larger(list, n);
        if (e.on && e.part == 0 && at < p.K) {
            p.values[(size_t)row * p.K + at] = key_float(e.key());
            p.idx[(size_t)row * p.K + at] = e.idx();
        }
        for (int i = n + threadIdx.x; i < p.K; i += kSelThreads) {
            p.values[(size_t)row * p.K + i] = -INFINITY;
            p.idx[(size_t)row * p.K + i] = -1;
        }
        return;
    }
    sort_list(list, n);
    for (int i = threadIdx.x; i < p.K; i += kSelThreads) {
        const unsigned long long e = i < n ? list[i] : 0ull;
        p.values[(size_t)row * p.K + i] = i < n ? key_float((uint32_t)(e >> 32)) : -INFINITY;
        p.idx[(size_t)row * p.K + i] = i < n ? (int32_t)~(uint32_t)e : -1;
    }
}

template <bool F32>
sats_status top_logits(const void *logits, int64_t ld, int T, int V, int K, float *values, int32_t *idx, void *stream)
{
    const sats_status s = check_rows(logits, ld, T, V, RowElem<F32>::kBytes);
    if (s != SATS_OK) return s;
    if (K < 1 || K > V) return SATS_EINVAL;
    if (K > kMaxTop) return SATS_ESHAPE;
    if (T == 0) return SATS_OK;
    if (!values || !idx) return SATS_EINVAL;
    TopParams p{};
    p.z = logits; p.ld = ld; p.T = T; p.V = V; p.K = K; p.values = values; p.idx = idx;
    const cudaError_t e = launch_rows<F32, top_kernel<F32>>(p, T, static_cast<cudaStream_t>(stream));
    return e == cudaSuccess ? SATS_OK : cuda_fail(e, "top-logits kernel launch");
}

}  // namespace
}  // namespace sats

extern "C" {

sats_status sats_top_logits(const void *logits, int64_t ld, int T, int V, int K, float *values, int32_t *idx,
                            void *stream)
{
    return sats::top_logits<false>(logits, ld, T, V, K, values, idx, stream);
}

sats_status sats_top_logits_f32(const float *logits, int64_t ld, int T, int V, int K, float *values, int32_t *idx,
                                void *stream)
{
    return sats::top_logits<true>(logits, ld, T, V, K, values, idx, stream);
}

}  // extern "C"
