// top_logits.cu -- the K largest logits of each row (sats_top_logits).
#include "internal.h"
#include "rows.cuh"

namespace sats {
namespace {
constexpr int kSelThreads = 256, kSelPerSm = 4;
}
}  // namespace sats
#include "logits.cuh"

namespace sats {
namespace {

constexpr size_t kMaxSmem = (size_t)kListCap * 12 + (size_t)kMaxGroups * kSelThreads * 4;

struct TopParams {
    const void *z;
    int64_t ld;
    int T, V, K;
    float *values;
    int32_t *idx;
    int cluster;
    int cap;          // entries of the list
    Groups groups;
};

// The row streams through registers once; only the groups whose maximum reaches the bound are read again, from the L2.
template <bool F32>
__global__ void __launch_bounds__(kSelThreads, kSelPerSm) top_kernel(const TopParams p)
{
    extern __shared__ __align__(16) uint4 smem[];
    __shared__ Shared sh;
    const int row = (int)(blockIdx.x >> (31 - __clz(p.cluster))), tid = threadIdx.x;
    unsigned long long *list = reinterpret_cast<unsigned long long *>(smem);
    float *gm = reinterpret_cast<float *>(list + p.cap);
    int *hits = reinterpret_cast<int *>(gm + kMaxGroups * kSelThreads);   // p.cap groups to read again
    Ctx<F32> c{Row<F32>(p.z, row, p.ld, p.V)};
    set_ctx<F32>(c, nullptr, 0, p.cluster, &sh, p.cap);
    if (c.C > 1) cluster_arrive();
    uint32_t *scratch = reinterpret_cast<uint32_t *>(list);
    for (int i = tid; i < kBoundBins; i += kSelThreads) scratch[i] = 0u;
    float hi = -INFINITY, lo = INFINITY;
    const int mine = group_maxima(c, p.groups, gm, &hi, &lo);
    uint32_t top;
    uint32_t bound = group_bound(&sh, scratch, (p.K + c.C - 1) >> (31 - __clz(c.C)), hi, lo, &top, [&](auto f) {
        for (int g = 0; g < mine; ++g) f(gm[g * kSelThreads + tid]);
    });
    if (c.C > 1) {
        cluster_wait();
        if (tid < c.C) {
            st_peer_u32(peer_addr(&sh.kmax[c.rank], tid), top);
            st_peer_u32(peer_addr(&sh.bound[c.rank], tid), bound);
        }
        cluster_sync_all();
        for (int k = 0; k < c.C; ++k) {
            top = max(top, sh.kmax[k]);
            bound = min(bound, sh.bound[k]);
        }
    }
    float *values = p.values + (size_t)row * p.K;
    int32_t *idx = p.idx + (size_t)row * p.K;
    {
        // each CTA orders its own candidates and hands them to all others; a candidate's place in the row is its place
        // in its CTA's list and, found by halving, in every other one
        const int C = c.C, seg = c.cap / C;
        unsigned long long *own = list + c.rank * seg;
        collect_groups(c, p.groups, gm, mine, hits, key_float(bound), own, seg);
        const int here = (int)sh.nlist;
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
        const Cut cut = cut_count(c, top, p.K);
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
    const int64_t bytes = (int64_t)V * RowElem<F32>::kBytes;
    p.cluster = logits_cluster(T, bytes, K, 0);
    p.cap = K <= kListCap / 16 ? kListCap / 4 : kListCap;
    // enough groups for a close bound, 64 times as many as it has to be reached by: 4 to kMaxGroups a thread
    int groups = 4;
    while (groups < kMaxGroups && (int64_t)groups * kSelThreads * p.cluster < 64 * (int64_t)K) groups *= 2;
    p.groups = plan_groups(bytes, p.cluster, groups);
    const size_t smem = (size_t)p.cap * 12 + (size_t)kMaxGroups * kSelThreads * 4;
    const cudaError_t e = launch_clusters<top_kernel<F32>>((int64_t)T * p.cluster, kSelThreads, smem, kMaxSmem, p.cluster,
                                                           static_cast<cudaStream_t>(stream), p);
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
