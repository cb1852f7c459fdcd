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

constexpr int kTurn = 8;               // granules in flight per thread
constexpr int kMaxGroups = 16;         // groups of a thread, at most
constexpr size_t kMaxSmem = (size_t)kListCap * 12 + (size_t)kMaxGroups * kSelThreads * 4;

struct TopParams {
    const void *z;
    int64_t ld;
    int T, V, K;
    float *values;
    int32_t *idx;
    int cluster;
    int cap;          // entries of the list
    int size, turns;  // granules of a group: `size` (1, 2, 4 or 8) in each of `turns` (1 unless size is 8) turns
};

// The maxima of a thread's groups of U granules in each of `turns` turns, to gm[group][thread]; the largest and the
// least above -inf.  Granules go to the threads in turn.
template <bool F32, int U>
__device__ __forceinline__ void group_maxima(const Ctx<F32> &c, int turns, float *gm, float *hi, float *lo)
{
    constexpr int kPer = kTurn / U;
    const int tid = threadIdx.x;
    float most = -INFINITY;   // (of a group that goes on)
    int left = turns;
    for (int v0 = tid; v0 < c.n; v0 += kTurn * kSelThreads) {
        uint4 x[kTurn];
#pragma unroll
        for (int k = 0; k < kTurn; ++k) {
            const uint32_t none = F32 ? 0xff800000u : 0xff80ff80u;
            x[k] = v0 + k * kSelThreads < c.n ? load_granule<F32>(c.r, c.gb + v0 + k * kSelThreads)
                                              : make_uint4(none, none, none, none);
        }
#pragma unroll
        for (int g = 0; g < kPer; ++g) {
            float m = granule_max<F32>(x[g * U]);
#pragma unroll
            for (int k = 1; k < U; ++k) m = fmaxf(m, granule_max<F32>(x[g * U + k]));
            most = fmaxf(most, m);
            if (U == kTurn && --left > 0 && v0 + kTurn * kSelThreads < c.n) continue;
            *gm = most;
            gm += kSelThreads;
            *hi = fmaxf(*hi, most);
            if (most > -INFINITY) *lo = fminf(*lo, most);
            most = -INFINITY;
            left = turns;
        }
    }
}

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
    switch (p.size) {
    case 1: group_maxima<F32, 1>(c, 1, gm + tid, &hi, &lo); break;
    case 2: group_maxima<F32, 2>(c, 1, gm + tid, &hi, &lo); break;
    case 4: group_maxima<F32, 4>(c, 1, gm + tid, &hi, &lo); break;
    default: group_maxima<F32, 8>(c, p.turns, gm + tid, &hi, &lo); break;
    }
    // granule j of group g of thread t is number (g S + j) kSelThreads + t of the CTA's
    const int S = p.size * p.turns, turns = tid < c.n ? (c.n - tid + kTurn * kSelThreads - 1) / (kTurn * kSelThreads) : 0;
    const int mine = (turns * kTurn + S - 1) / S;   // kMaxGroups at most
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
        constexpr int E = RowElem<F32>::kPer;
        const int C = c.C, seg = c.cap / C;
        unsigned long long *own = list + c.rank * seg;
        const float fb = key_float(bound);
        if (tid == 0) sh.nlist = sh.nhits = 0;
        __syncthreads();
        for (int g = 0; g < mine; ++g)
            if (gm[g * kSelThreads + tid] >= fb) {
                const uint32_t at = atomicAdd(&sh.nhits, 1u);
                if (at < (uint32_t)seg) hits[at] = g * kSelThreads + tid;
            }
        __syncthreads();
        const int nhits = min((int)sh.nhits, seg);   // (a group has a candidate: with more groups there are too many of them)
        for (int w = tid; w < nhits * S; w += kSelThreads) {
            const int h = hits[w / S], v = (h / kSelThreads * S + w % S) * kSelThreads + h % kSelThreads;
            if (v >= c.n) continue;
            const uint4 x = load_granule<F32>(c.r, c.gb + v);
            if (!(granule_max<F32>(x) >= fb)) continue;
            float f[E];
            granule_floats<F32>(c.clean(x), f);
            const int i0 = c.r.first(c.gb + v);
#pragma unroll
            for (int j = 0; j < E; ++j)
                if (f[j] >= fb && f[j] > -INFINITY) {
                    const uint32_t at = atomicAdd(&sh.nlist, 1u);
                    if (at < (uint32_t)seg) own[at] = ((unsigned long long)key_of(f[j]) << 32) | (uint32_t)~(uint32_t)(i0 + j);
                }
        }
        __syncthreads();
        const int here = (int)sh.nlist;
        const bool fits = (int)sh.nhits <= seg && here <= min(seg, kSmall);
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
    int64_t groups = 4;
    while (groups < kMaxGroups && groups * kSelThreads * p.cluster < 64 * (int64_t)K) groups *= 2;
    const int64_t each = (bytes / 16 / p.cluster + 4 + kSelThreads - 1) / kSelThreads;   // granules of a thread, at most
    const int64_t rounded = (each + kTurn - 1) / kTurn * kTurn;
    p.size = p.turns = 1;
    while (p.size < kTurn && p.size * groups < rounded) p.size *= 2;
    while ((int64_t)p.size * p.turns * groups < rounded) p.turns *= 2;
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
