// top_logits.cu -- the K largest logits of each row (sats_top_logits).
#include <algorithm>

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
static_assert(kListCap * 8 <= kMaxGroups * kSelThreads * 4 && kListCap >= 2 * 512, "where the list's entries are placed");

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

// Puts the n entries of the list (the largest is `top`) where they belong in descending order, without sorting:
// equal steps of the logit give each entry a run of places, the entries of its step (a few, as a rule) its place there.
// (1216 rows at K 1000: 127 us, with a bitonic sort of the list 202.)
// False where a step has too many.  other: room for the list; count: 2 kPlaceSteps words behind it.
constexpr int kPlaceSteps = 512, kPlaceMost = 128;
__device__ __forceinline__ bool put_by_steps(const unsigned long long *list, int n, uint32_t top,
                                             unsigned long long *other, uint32_t *count, Shared *sh, float *values,
                                             int32_t *idx, int K)
{
    constexpr int kPer = kListCap / kSelThreads, kRun = kPlaceSteps / kSelThreads;
    const int tid = threadIdx.x;
    __syncthreads();
    uint32_t low = 0xffffffffu;
    for (int i = tid; i < n; i += kSelThreads) low = min(low, (uint32_t)(list[i] >> 32));
    low = __reduce_min_sync(0xffffffffu, low);
    if ((tid & 31) == 0) sh->klow[tid >> 5] = low;
    for (int i = tid; i < kPlaceSteps; i += kSelThreads) count[i] = 0u;
    __syncthreads();
    low = __reduce_min_sync(0xffffffffu, sh->klow[tid & (kSelWarps - 1)]);
    const float ft = key_float(top), range = ft - key_float(low);
    if (!(range > 0.f && range < INFINITY)) return false;
    const float scale = (float)kPlaceSteps / range;
    if (scale == INFINITY) return false;
    uint32_t *first = count + kPlaceSteps;
    const auto step_of = [&](unsigned long long e) {
        return (int)fminf((ft - key_float((uint32_t)(e >> 32))) * scale, (float)(kPlaceSteps - 1));
    };
    uint32_t at[kPer];
#pragma unroll
    for (int k = 0; k < kPer; ++k)
        if (tid + k * kSelThreads < n) at[k] = atomicAdd(count + step_of(list[tid + k * kSelThreads]), 1u);
    __syncthreads();
    uint32_t run[kRun], sum = 0, most = 0;
#pragma unroll
    for (int k = 0; k < kRun; ++k) {
        run[k] = count[tid * kRun + k];
        most = max(most, run[k]);
        sum += run[k];
    }
    if (__syncthreads_or(most > (uint32_t)kPlaceMost)) return false;
    unsigned long long total;
    uint32_t from = (uint32_t)block_scan_u64(sum, sh, &total);
#pragma unroll
    for (int k = 0; k < kRun; ++k) {
        first[tid * kRun + k] = from;
        from += run[k];
    }
    __syncthreads();
#pragma unroll
    for (int k = 0; k < kPer; ++k)
        if (tid + k * kSelThreads < n) {
            const unsigned long long e = list[tid + k * kSelThreads];
            other[first[step_of(e)] + at[k]] = e;
        }
    __syncthreads();
    for (int i = tid; i < n; i += kSelThreads) {   // (neighbours have the same step, or nearly)
        const unsigned long long e = other[i];
        const int s = step_of(e), f = (int)first[s], m = (int)count[s];
        int place = f;
        for (int j = f; j < f + m; ++j) place += other[j] > e;
        if (place < K) {
            values[place] = key_float((uint32_t)(e >> 32));
            idx[place] = (int32_t)~(uint32_t)e;
        }
    }
    for (int i = n + tid; i < K; i += kSelThreads) {
        values[i] = -INFINITY;
        idx[i] = -1;
    }
    return true;
}

// The row streams through registers once; only the groups whose maximum reaches the bound are read again, from the L2.
// 2048 rows of 128256 bf16 logits at K 64 take 106 us, 4.95 TB/s, where 78 us is the stream: the rest is the chain after
// it (histogram, one or two exchanges, the candidates), 6 to 8 us that the three other CTAs on the SM cover in part; one
// row of 151936 takes 10.8 us.  With the rows kept in shared memory (2 CTAs to an SM) it was 210, with clusters that stay
// for many rows and fetch ahead 329.  At K 400 and 1000 1216 rows take 90 and 126 us, at K 64 63.
// FEW: few_groups.
template <bool F32, bool FEW>
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
    const int R = (p.K + c.C - 1) >> (31 - __clz(c.C));
    uint32_t bound;
    if constexpr (FEW)
        bound = element_bound(c, scratch, R, &top);
    else
        bound = group_bound(&sh, scratch, R, hi, lo, &top, [&](auto f) {
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
        if (tid < C) {
            st_peer_u32(peer_addr(&sh.cnt[c.rank], tid), fits ? (uint32_t)here : 0xffffffffu);
            st_peer_u32(peer_addr(&sh.above[c.rank], tid), (uint32_t)here);
        }
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
    bool there = true;
    int n = 0, before = 0;
    for (int k = 0; k < c.C; ++k) {
        if (k == (int)c.rank) before = n;
        there = there && sh.above[k] <= (uint32_t)(c.cap / c.C);
        n += (int)sh.above[k];
    }
    if (there) {   // (the same in every CTA of the row)
        unsigned long long *own = list + c.rank * (c.cap / c.C);
        if (c.C > 1) {
            // the first CTA's list behind its own entries: the others' places there are free
            const int mine = (int)sh.nlist;
            if (c.rank != 0)
                for (int i = tid; i < mine; i += kSelThreads) st_peer_u64(peer_addr(list + before + i, 0), own[i]);
            cluster_sync_all();
        }
    } else {
        bool ok;
        n = gather_list(c, list, bound, Cut{kKeyNone, INT_MIN}, &ok);
        if (!ok) {   // (the same in every CTA of the row)
            const Cut cut = cut_count(c, top, p.K);
            n = gather_list(c, list, max(cut.key, kKeyNone + 1), cut, &ok);   // at most K
        }
    }
    if (c.rank != 0) return;   // (nobody reads this CTA's memory any more)
    unsigned long long *other = reinterpret_cast<unsigned long long *>(gm);
    if (put_by_steps(list, n, top, other, reinterpret_cast<uint32_t *>(other + p.cap), &sh, values, idx, p.K)) return;
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
    const int64_t ctas = (int64_t)T * p.cluster;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    const int granules = (int)std::min<int64_t>((bytes + 15) / 16 / p.cluster, 1 << 20);   // (a group has one at least)
    const cudaError_t e =
        few_groups(granules, granules * RowElem<F32>::kPer, (K + p.cluster - 1) / p.cluster)
            ? launch_clusters<top_kernel<F32, true>>(ctas, kSelThreads, smem, kMaxSmem, p.cluster, st, p)
            : launch_clusters<top_kernel<F32, false>>(ctas, kSelThreads, smem, kMaxSmem, p.cluster, st, p);
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
