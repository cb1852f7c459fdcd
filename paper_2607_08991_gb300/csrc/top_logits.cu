// top_logits.cu -- the K largest logits of each row (sats_top_logits).
#include "internal.h"
#include "rows.cuh"

namespace sats {
namespace {
constexpr int kSelThreads = 256, kSelPerSm = 3;
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
    int cap;   // entries of the list
};

template <bool F32>
__global__ void __launch_bounds__(kSelThreads, kSelPerSm) top_kernel(const TopParams p)
{
    extern __shared__ __align__(16) uint4 smem[];
    __shared__ Shared sh;
    const int row = (int)(blockIdx.x >> (31 - __clz(p.cluster)));
    unsigned long long *list = reinterpret_cast<unsigned long long *>(smem + p.cached);
    Ctx<F32> c{Row<F32>(p.z, row, p.ld, p.V)};
    set_ctx(c, smem, p.cached, p.cluster, &sh, p.cap);
    start_row(c, smem);
    uint32_t kmax, bound;
    load_row(c, smem, p.K, reinterpret_cast<uint32_t *>(list), &kmax, &bound);
    float *values = p.values + (size_t)row * p.K;
    int32_t *idx = p.idx + (size_t)row * p.K;
    {
        // each CTA orders its own candidates and hands them to all others; a candidate's place in the row is its place
        // in its CTA's list and, found by halving, in every other one
        const int C = c.C, seg = c.cap / C, tid = threadIdx.x;
        unsigned long long *own = list + c.rank * seg;
        const int here = collect(c, own, seg, bound, Cut{kKeyNone, INT_MIN});
        const bool fits = here <= min(seg, kSmall);
        if (fits) {
            const Small e(own, here);
            const int at = e.larger(own, here);
            __syncthreads();
            if (e.on && e.part == 0) {
                own[at] = e.e;
                for (int q = 1; q < C; ++q) st_peer_u64(peer_addr(own + at, (c.rank + q) & (C - 1)), e.e);
            }
        }
        if (tid < C) st_peer_u32(peer_addr(&sh.cnt[c.rank], tid), fits ? (uint32_t)here : 0xffffffffu);
        if (C > 1) cluster_sync_all();
        else __syncthreads();
        bool all = true;
        int n = 0;
        for (int k = 0; k < C; ++k) {
            all = all && sh.cnt[k] != 0xffffffffu;
            n += (int)sh.cnt[k];
        }
        if (all) {   // (the same in every CTA of the row)
            if (tid < here) {
                const unsigned long long e = own[tid];
                int at = tid;
                for (int q = 1; q < C; ++q) {
                    const unsigned k = (c.rank + q) & (C - 1);
                    const unsigned long long *other = list + k * seg;
                    int lo = 0, hi = (int)sh.cnt[k];
                    while (lo < hi) {
                        const int mid = (lo + hi) / 2;
                        if (other[mid] > e) lo = mid + 1;
                        else hi = mid;
                    }
                    at += lo;
                }
                if (at < p.K) {
                    values[at] = key_float((uint32_t)(e >> 32));
                    idx[at] = (int32_t)~(uint32_t)e;
                }
            }
            if (c.rank == 0)
                for (int i = n + tid; i < p.K; i += kSelThreads) {
                    values[i] = -INFINITY;
                    idx[i] = -1;
                }
            return;
        }
    }
    // more candidates than that: one list of all of them, or of exactly the K largest
    bool ok;
    int n = gather_list(c, list, bound, Cut{kKeyNone, INT_MIN}, &ok);
    if (!ok) {   // (the same in every CTA of the row)
        const Cut cut = cut_count(c, kmax, p.K);
        n = gather_list(c, list, max(cut.key, kKeyNone + 1), cut, &ok);   // at most K
    }
    if (c.rank != 0) return;   // (nobody reads this CTA's memory any more)
    sort_list(list, n);
    for (int i = threadIdx.x; i < p.K; i += kSelThreads) {
        const unsigned long long e = i < n ? list[i] : 0ull;
        values[i] = i < n ? key_float((uint32_t)(e >> 32)) : -INFINITY;
        idx[i] = i < n ? (int32_t)~(uint32_t)e : -1;
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
    p.cap = K <= kListCap / 16 ? kListCap / 4 : kListCap;   // (a small one leaves room for another CTA)
    const cudaError_t e = launch_rows<F32, top_kernel<F32>>(p, T, p.cap, K, static_cast<cudaStream_t>(stream));
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
