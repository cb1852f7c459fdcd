// logits.cuh -- the top logits of a row and the drawing of a token from it: what top_logits.cu and sample.cu share.
//
// One row per thread-block cluster.  Where few of the row's largest logits are asked for, both calls start alike:
//   - while the row arrives, each thread keeps the maxima of a few groups of its elements.  At least R groups have
//     their maximum at or above the R-th largest of these maxima, so that at least R elements do: with
//     R = ceil(K / C) in each of C CTAs, the least of their bounds has K elements of the row at or above it;
//   - the elements at or above the bound (about K of them in a row of no particular order) go to a list, which is put in
//     order: descending logits, ties by the lower index.
// A row whose list would not fit (many equal logits, or large ones that share few groups) takes the general way: the
// exact K-th largest key by bisection over the keys, counting in every step (2048 rows of 5000 logits at K 1000, when
// all of them took it: 351 us, against 75 with a bound).
#pragma once

#include <climits>
#include <cmath>

#include "internal.h"
#include "rows.cuh"

namespace sats {
namespace {

constexpr int kSelWarps = kSelThreads / 32;   // (kSelThreads: the including file's choice)
constexpr int kMaxTop = 1024;          // largest K of the list's way
constexpr int kListCap = 2048;         // entries of the list
constexpr uint32_t kKeyNone = 0x007fffffu;   // key of -inf: never selected
constexpr int kFew = 8;                // elements per thread at the end of a search

// Keys order as the floats do; both zeros have one key.  NaN has none (cleaned to -inf before).
__device__ __forceinline__ uint32_t key_of(float x)
{
    const uint32_t b = __float_as_uint(x + 0.f);
    return b ^ ((uint32_t)((int32_t)b >> 31) | 0x80000000u);
}
__device__ __forceinline__ float key_float(uint32_t k)
{
    return __uint_as_float((k & 0x80000000u) ? k ^ 0x80000000u : ~k);
}

// ------------------------------------------------------------------ the row in a cluster
struct Shared {
    unsigned long long wsum[kSelWarps];
    unsigned long long scan[kSelWarps];
    unsigned long long slot[2][2][kRowMaxCluster];   // the CTAs' values, one or two of each; two buffers in turn
    uint32_t kmax[kRowMaxCluster], bound[kRowMaxCluster];
    int part[kSelWarps];
    uint32_t ktop[kSelWarps], klow[kSelWarps];
    int border;
    uint32_t nlist, nhits;
    int found_idx;
    uint32_t found_key;
    uint32_t kminp;
    // the nucleus: steps of the border, and of each CTA the entries, the tokens kept and their mass
    uint32_t bin0, bin1, cnt[kRowMaxCluster], above[kRowMaxCluster];
    unsigned long long mass[kRowMaxCluster];
};

template <bool F32>
struct Ctx {
    Row<F32> r;
    int gb, n;            // this CTA's granules: gb .. gb + n
    int wb, we;           // this warp's, within them
    int cached;           // of them in shared memory
    const uint4 *cache;
    Shared *sh;
    int C;
    unsigned rank;
    int turn;             // of the all-reduce buffers
    int cap;              // entries of the list, kListCap at most

    // Granule v of this CTA's; get: with NaN replaced by -inf.
    __device__ __forceinline__ uint4 raw(int v) const { return v < cached ? cache[v] : load_granule<F32>(r, gb + v); }
    __device__ __forceinline__ uint4 get(int v) const { return clean(raw(v)); }
    static __device__ __forceinline__ uint4 clean(uint4 x)
    {
        if constexpr (F32) {
            x.x = __float_as_uint(fmaxf(__uint_as_float(x.x), -INFINITY));
            x.y = __float_as_uint(fmaxf(__uint_as_float(x.y), -INFINITY));
            x.z = __float_as_uint(fmaxf(__uint_as_float(x.z), -INFINITY));
            x.w = __float_as_uint(fmaxf(__uint_as_float(x.w), -INFINITY));
        } else {
            x.x = bf16x2_max(x.x, 0xff80ff80u);
            x.y = bf16x2_max(x.y, 0xff80ff80u);
            x.z = bf16x2_max(x.z, 0xff80ff80u);
            x.w = bf16x2_max(x.w, 0xff80ff80u);
        }
        return x;
    }
    // One element of granule v.
    __device__ __forceinline__ float get(int v, int j) const
    {
        float x;
        if constexpr (F32) {
            x = v < cached ? reinterpret_cast<const float *>(cache + v)[j] : __uint_as_float(pick(load_granule<F32>(r, gb + v), j));
        } else {
            x = v < cached ? __uint_as_float((uint32_t)reinterpret_cast<const uint16_t *>(cache + v)[j] << 16)
                           : __uint_as_float(pick(load_granule<F32>(r, gb + v), j >> 1) << ((j & 1) ? 0 : 16) & 0xffff0000u);
        }
        return x == x ? x : -INFINITY;
    }
    static __device__ __forceinline__ uint32_t pick(const uint4 &x, int w)
    {
        return w == 0 ? x.x : w == 1 ? x.y : w == 2 ? x.z : x.w;
    }
};

__device__ __forceinline__ unsigned long long warp_sum_u64(unsigned long long v)
{
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    return v;
}

// Sum over the CTA; the warps' parts stay in sh->wsum until the next call.  Every thread gets the total.
__device__ __forceinline__ unsigned long long block_sum_u64(unsigned long long v, Shared *sh)
{
    v = warp_sum_u64(v);
    __syncthreads();   // (whoever still reads the parts of the last call)
    if ((threadIdx.x & 31) == 0) sh->wsum[threadIdx.x >> 5] = v;
    __syncthreads();
    unsigned long long t = 0;
#pragma unroll
    for (int w = 0; w < kSelWarps; ++w) t += sh->wsum[w];
    return t;
}

// Exclusive sums of the threads' values over the CTA, the total in *total.
__device__ __forceinline__ unsigned long long block_scan_u64(unsigned long long v, Shared *sh, unsigned long long *total)
{
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    unsigned long long incl = v;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const unsigned long long u = __shfl_up_sync(0xffffffffu, incl, o);
        if (lane >= o) incl += u;
    }
    __syncthreads();
    if (lane == 31) sh->scan[warp] = incl;
    __syncthreads();
    unsigned long long before = 0, t = 0;
#pragma unroll
    for (int w = 0; w < kSelWarps; ++w) {
        if (w < warp) before += sh->scan[w];
        t += sh->scan[w];
    }
    *total = t;
    return before + incl - v;
}

// The CTAs' values, in every CTA's slots; returns their buffer (of second values: behind the first ones).
template <bool F32>
__device__ __forceinline__ const unsigned long long *cluster_gather(Ctx<F32> &c, unsigned long long v,
                                                                    unsigned long long second = 0)
{
    unsigned long long (*slot)[kRowMaxCluster] = c.sh->slot[c.turn];
    c.turn ^= 1;
    if (c.C == 1) {
        if (threadIdx.x == 0) {
            slot[0][0] = v;
            slot[1][0] = second;
        }
        __syncthreads();
        return slot[0];
    }
    if (threadIdx.x < (unsigned)c.C) {
        st_peer_u64(peer_addr(&slot[0][c.rank], threadIdx.x), v);
        st_peer_u64(peer_addr(&slot[1][c.rank], threadIdx.x), second);
    }
    cluster_sync_all();
    return slot[0];
}

__device__ __forceinline__ unsigned long long slot_sum(const unsigned long long *slot, int C)
{
    unsigned long long t = 0;
    for (int k = 0; k < C; ++k) t += slot[k];
    return t;
}

template <bool F32>
__device__ __forceinline__ unsigned long long cluster_sum(Ctx<F32> &c, unsigned long long v)
{
    return slot_sum(cluster_gather(c, block_sum_u64(v, c.sh)), c.C);
}

// What is kept: keys above `key`, and of those equal to it the ones up to index `idx` (INT_MIN: none; the places of a
// granule before the row have indices below 0).
struct Cut {
    uint32_t key;
    int idx;
    __device__ __forceinline__ bool keeps(uint32_t k, int i) const { return k > key || (k == key && i <= idx); }
};

// A sum over the row's tokens is given by a functor: elem(logit, key, index) for one of them, granule(c, v) for the
// ones of granule v.  ByElem makes one of a function of an element.
template <typename F>
struct ByElem {
    F f;
    __device__ __forceinline__ unsigned long long elem(float x, uint32_t k, int i) const { return f(x, k, i); }
    template <bool F32>
    __device__ __forceinline__ unsigned long long granule(const Ctx<F32> &c, int v) const
    {
        constexpr int E = RowElem<F32>::kPer;
        float x[E];
        granule_floats<F32>(c.get(v), x);
        const int i0 = c.r.first(c.gb + v);
        unsigned long long s = 0;
#pragma unroll
        for (int j = 0; j < E; ++j) {
            const uint32_t k = key_of(x[j]);
            if (k > kKeyNone) s += f(x[j], k, i0 + j);   // (places outside the row are -inf)
        }
        return s;
    }
};
template <typename F>
__device__ __forceinline__ ByElem<F> by_elem(F f) { return ByElem<F>{f}; }

// Sum over this thread's granules, lanes in turn over the warp's run of them.
template <bool F32, typename S>
__device__ __forceinline__ unsigned long long thread_sum(const Ctx<F32> &c, const S &f)
{
    unsigned long long s = 0;
    for (int v = c.wb + (int)(threadIdx.x & 31); v < c.we; v += 32) s += f.granule(c, v);
    return s;
}

// The first token in the vocabulary's order at which the running sum of f passes `target` (which is below the sum
// over the row): found(idx, key) by one thread.  The warps' sums are in sh->wsum (block_sum_u64 of thread_sum), the
// CTAs' are in `slot`.  The CTA that holds the token narrows a run of granules down
// sixteenfold a step until its threads have a few elements each.
template <bool F32, typename S, typename Found>
__device__ __forceinline__ void locate(Ctx<F32> &c, unsigned long long target, const S &f,
                                       const unsigned long long *slot, Found found)
{
    Shared *sh = c.sh;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    unsigned long long before = 0;
    for (unsigned k = 0; k < c.rank; ++k) before += slot[k];
    if (target >= before && target - before < slot[c.rank]) {   // (one CTA)
        unsigned long long t = target - before;
        int a = 0, b = c.n, per = (c.n + kSelWarps - 1) / kSelWarps;
        for (;;) {
            int w = 0;
            while (w < kSelWarps - 1 && t >= sh->wsum[w]) t -= sh->wsum[w++];
            a = a + w * per;
            b = min(b, a + per);
            if (b - a <= kSelThreads * kFew / RowElem<F32>::kPer) break;
            per = (b - a + kSelWarps - 1) / kSelWarps;
            unsigned long long s = 0;
            const int wb = min(b, a + warp * per), we = min(b, wb + per);
            for (int v = wb + lane; v < we; v += 32) s += f.granule(c, v);
            block_sum_u64(s, sh);
        }
        // a few elements per thread, in order
        constexpr int E = RowElem<F32>::kPer;
        const int n = (b - a) * E, each = (n + kSelThreads - 1) / kSelThreads, first = tid * each;
        const int i0 = c.r.first(c.gb + a);
        const auto at = [&](int e, uint32_t *k) {
            const float x = c.get(a + e / E, e % E);
            *k = key_of(x);
            return *k > kKeyNone ? f.elem(x, *k, i0 + e) : 0ull;
        };
        uint32_t k;
        unsigned long long s = 0, total;
        for (int e = first; e < min(n, first + each); ++e) s += at(e, &k);
        unsigned long long run = block_scan_u64(s, sh, &total);
        if (t >= run && t - run < s) {   // (one thread)
            int e = first;
            for (const int last = min(n, first + each) - 1;; ++e) {
                run += at(e, &k);
                if (run > t || e == last) break;   // (t is below the sum of the thread's elements)
            }
            found(i0 + e, k);
        }
    }
}

// The same, with the sums to be taken first; *idx, *key in every CTA.
template <bool F32, typename S>
__device__ void sum_and_locate(Ctx<F32> &c, unsigned long long target, const S &f, int *idx, uint32_t *key)
{
    const unsigned long long mine = block_sum_u64(thread_sum(c, f), c.sh);
    const unsigned long long *slot = cluster_gather(c, mine);
    Shared *sh = c.sh;
    locate(c, target, f, slot, [&](int i, uint32_t k) {
        for (int q = 0; q < c.C; ++q) {
            st_peer_u32(peer_addr(&sh->found_idx, q), (uint32_t)i);
            st_peer_u32(peer_addr(&sh->found_key, q), k);
        }
    });
    if (c.C > 1) cluster_sync_all();
    else __syncthreads();
    *idx = sh->found_idx;
    *key = sh->found_key;
}

// The largest key at which sum(f over keys >= it) is at least `want` (1 <= want <= the sum over all): between kmin and
// kmax, the least and the largest key that f counts.  The sum over the keys above it in *above.
template <bool F32, typename F>
__device__ uint32_t bisect_key(Ctx<F32> &c, uint32_t kmin, uint32_t kmax, unsigned long long want, F f,
                               unsigned long long *above)
{
    uint32_t lo = kmin, hi = kmax + 1;   // sum(lo) >= want > sum(hi)
    unsigned long long s_hi = 0;
    while (hi - lo > 1) {
        const uint32_t mid = lo + (hi - lo) / 2;
        const auto from_mid = by_elem([&](float x, uint32_t k, int i) { return k >= mid ? f(x, k, i) : 0ull; });
        const unsigned long long s = cluster_sum(c, thread_sum(c, from_mid));
        if (s >= want) lo = mid;
        else { hi = mid; s_hi = s; }
    }
    *above = s_hi;
    return lo;
}

// The cut that keeps the k largest (ties by the lower index); no cut where the row has no more than k.
template <bool F32>
__device__ Cut cut_count(Ctx<F32> &c, uint32_t kmax, int k)
{
    const auto one = [](float, uint32_t, int) { return 1ull; };
    if (cluster_sum(c, thread_sum(c, by_elem(one))) <= (unsigned long long)k) return Cut{kKeyNone, INT_MIN};
    unsigned long long above;
    Cut cut;
    cut.key = bisect_key(c, kKeyNone + 1, kmax, (unsigned long long)k, one, &above);
    const uint32_t at = cut.key;
    uint32_t key;
    sum_and_locate(c, (unsigned long long)k - above - 1ull,
                   by_elem([at](float, uint32_t q, int) { return q == at ? 1ull : 0ull; }), &cut.idx, &key);
    return cut;
}

// ------------------------------------------------------------------ the list
constexpr int kListPer = kListCap / kSelThreads;   // list entries of a thread, in a row

// Sorts n2 (a power of two) words descending; all threads of the CTA.
__device__ void sort_desc(unsigned long long *a, int n2)
{
    __syncthreads();
    for (int k = 2; k <= n2; k <<= 1) {
        for (int j = k >> 1; j > 0; j >>= 1) {
            for (int t = threadIdx.x; t < n2 / 2; t += kSelThreads) {
                const int i = 2 * t - (t & (j - 1));
                const unsigned long long x = a[i], y = a[i + j];
                if ((x < y) == ((i & k) == 0)) {
                    a[i] = y;
                    a[i + j] = x;
                }
            }
            // pairs at a distance of at most 32 stay within the 64 words of one warp's pairs
            if (j > 32 || (j == 1 && k >= 64)) __syncthreads();
            else __syncwarp();
        }
    }
    __syncthreads();
}

__device__ __forceinline__ int pow2_at_least(int n) { return n <= 1 ? 1 : 1 << (32 - __clz(n - 1)); }

// Brings the CTAs' parts of the list (sh->nlist entries each, of which up to c.cap are there) together in the
// cluster's first CTA.  Returns how many there are (in every CTA); *ok: they fit and are there.
template <bool F32>
__device__ int push_list(Ctx<F32> &c, unsigned long long *list, bool *ok)
{
    const uint32_t mine = c.sh->nlist;
    const unsigned long long *slot = cluster_gather(c, (unsigned long long)mine);
    unsigned long long total = 0, before = 0;
    for (int k = 0; k < c.C; ++k) {
        if (k < (int)c.rank) before += slot[k];
        total += slot[k];
    }
    *ok = total <= (unsigned long long)c.cap;
    if (*ok && c.C > 1) {
        if (c.rank != 0)
            for (uint32_t i = threadIdx.x; i < mine; i += kSelThreads)
                st_peer_u64(peer_addr(list + before + i, 0), list[i]);
        cluster_sync_all();
    }
    return (int)(total < (unsigned long long)INT_MAX ? total : INT_MAX);
}

// This CTA's elements with keys from `bound` on that `cut` keeps, to `list`, in no order; returns how many there are (of
// which `cap` at most are in the list).
template <bool F32>
__device__ int collect(Ctx<F32> &c, unsigned long long *list, int cap, uint32_t bound, Cut cut)
{
    constexpr int E = RowElem<F32>::kPer;
    Shared *sh = c.sh;
    const float fb = key_float(bound);
    if (threadIdx.x == 0) sh->nlist = 0;
    __syncthreads();
    for (int v = c.wb + (int)(threadIdx.x & 31); v < c.we; v += 32) {
        const uint4 x = c.raw(v);
        if (!(granule_max<F32>(x) >= fb)) continue;
        float f[E];
        granule_floats<F32>(c.clean(x), f);
        const int i0 = c.r.first(c.gb + v);
#pragma unroll
        for (int j = 0; j < E; ++j) {
            if (!(f[j] >= fb)) continue;
            const uint32_t k = key_of(f[j]);
            if (k >= bound && k > kKeyNone && cut.keeps(k, i0 + j)) {
                const uint32_t at = atomicAdd(&sh->nlist, 1u);
                if (at < (uint32_t)cap) list[at] = ((unsigned long long)k << 32) | (uint32_t)~(uint32_t)(i0 + j);
            }
        }
    }
    __syncthreads();
    return (int)sh->nlist;
}

// The same of the whole row, to the list of the cluster's first CTA (push_list).
template <bool F32>
__device__ int gather_list(Ctx<F32> &c, unsigned long long *list, uint32_t bound, Cut cut, bool *ok)
{
    collect(c, list, c.cap, bound, cut);
    return push_list(c, list, ok);
}

// Pads the list with zeros and sorts it; n <= kListCap.  (First CTA.)
__device__ void sort_list(unsigned long long *list, int n)
{
    const int n2 = pow2_at_least(n);
    for (int i = n + threadIdx.x; i < n2; i += kSelThreads) list[i] = 0ull;
    sort_desc(list, n2);
}

// A list of at most kSmall entries needs no sorting: each is compared with all others, by kSelThreads / (the entries'
// number, rounded up to a power of two) threads each.  (128 entries: sorting took 3 us, this a fifth of it.)
constexpr int kSmall = 256;   // (at most kSelThreads)
static_assert(kSmall <= kSelThreads, "a thread per entry");
struct Small {
    unsigned long long e;   // (key << 32) | ~index
    int i, part, per;       // the entry, the thread's part of the comparisons, threads per entry (a power of two <= 16)
    bool on;

    __device__ __forceinline__ Small(const unsigned long long *list, int n)
    {
        const int n2 = max(32, pow2_at_least(n));
        per = kSelThreads / n2;
        i = (int)threadIdx.x / per;
        part = (int)threadIdx.x & (per - 1);
        on = i < n;
        e = on ? list[i] : 0ull;
    }
    __device__ __forceinline__ uint32_t key() const { return (uint32_t)(e >> 32); }
    __device__ __forceinline__ int idx() const { return (int)~(uint32_t)e; }
    // Weights lie behind the entries.
    __device__ __forceinline__ void put_weight(unsigned long long *list, unsigned long long w) const
    {
        if (part == 0 && on) list[kSmall + i] = w;
    }
    // Number of the entries before this one in descending order, and (weights given) their sum.
    __device__ __forceinline__ int larger(const unsigned long long *list, int n) const
    {
        int rank = 0;
        for (int j = part; j < n; j += per) rank += list[j] > e;
        for (int o = per / 2; o > 0; o >>= 1) rank += __shfl_xor_sync(0xffffffffu, rank, o);
        return rank;
    }
    __device__ __forceinline__ void larger(const unsigned long long *list, int n, int *rank, unsigned long long *sum) const
    {
        int r = 0;
        unsigned long long s = 0;
        for (int j = part; j < n; j += per)
            if (list[j] > e) {
                ++r;
                s += list[kSmall + j];
            }
        for (int o = per / 2; o > 0; o >>= 1) {
            r += __shfl_xor_sync(0xffffffffu, r, o);
            s += __shfl_xor_sync(0xffffffffu, s, o);
        }
        *rank = r;
        *sum = s;
    }
    // Sum of the weights of the entries with lower indices.
    __device__ __forceinline__ unsigned long long earlier(const unsigned long long *list, int n) const
    {
        unsigned long long s = 0;
        for (int j = part; j < n; j += per)
            if ((uint32_t)list[j] > (uint32_t)e) s += list[kSmall + j];
        for (int o = per / 2; o > 0; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
        return s;
    }
};

// ------------------------------------------------------------------ the bound
// A key that the maxima of at least R of the CTA's groups reach (kKeyNone + 1 if there are not so many, or R is 0), and
// the largest key in *top.  hi, lo: the largest of the thread's maxima and the least above -inf; each(f): f(maximum) for
// all of them.  A histogram of the maxima from the largest down, in equal steps; scratch: its kBoundBins words, zero, a
// barrier ahead.
constexpr int kBoundBins = 512;
template <typename Each>
__device__ __forceinline__ uint32_t group_bound(Shared *sh, uint32_t *scratch, int R, float hi, float lo, uint32_t *top,
                                                Each each)
{
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const uint32_t khi = __reduce_max_sync(0xffffffffu, key_of(hi));
    uint32_t klo = __reduce_min_sync(0xffffffffu, key_of(lo));
    if (lane == 0) {
        sh->ktop[warp] = khi;
        sh->klow[warp] = klo;
    }
    if (threadIdx.x == 0) sh->border = kBoundBins;
    __syncthreads();
    *top = __reduce_max_sync(0xffffffffu, sh->ktop[lane & (kSelWarps - 1)]);
    if (R <= 0) return kKeyNone + 1;
    klo = __reduce_min_sync(0xffffffffu, sh->klow[lane & (kSelWarps - 1)]);
    const float ft = key_float(*top), range = ft - key_float(klo);
    const float scale = range > 0.f && range < INFINITY ? (float)kBoundBins / range : 0.f;   // (0: one step)
    const auto bin = [&](float g) { return scale > 0.f ? (int)fminf((ft - g) * scale, (float)(kBoundBins - 1)) : 0; };
    each([&](float g) {
        if (g > -INFINITY) atomicAdd(scratch + bin(g), 1u);
    });
    __syncthreads();
    if (warp == 0) {
        constexpr int kPer = kBoundBins / 32;
        uint32_t n[kPer], sum = 0;
#pragma unroll
        for (int k = 0; k < kPer; ++k) {
            n[k] = scratch[lane * kPer + k];
            sum += n[k];
        }
        uint32_t incl = sum;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const uint32_t u = __shfl_up_sync(0xffffffffu, incl, o);
            if (lane >= o) incl += u;
        }
        uint32_t run = incl - sum;
        if (run < (uint32_t)R && incl >= (uint32_t)R) {   // (at most one lane)
            int b = lane * kPer;
#pragma unroll
            for (int k = 0; k < kPer; ++k) {
                run += n[k];
                b += run < (uint32_t)R;
            }
            sh->border = b;
        }
    }
    __syncthreads();
    // the least maximum down to that step; everything, where there are fewer than R
    const int border = sh->border;
    float at = INFINITY;
    each([&](float g) {
        if (g > -INFINITY && bin(g) <= border) at = fminf(at, g);
    });
    klo = __reduce_min_sync(0xffffffffu, key_of(at));
    if (lane == 0) sh->klow[warp] = klo;
    __syncthreads();
    klo = __reduce_min_sync(0xffffffffu, sh->klow[lane & (kSelWarps - 1)]);
    return border < kBoundBins ? klo : kKeyNone + 1;
}

// The same with every element a group: where the granules are too few for groups of them to give a close bound.
template <bool F32>
__device__ __noinline__ uint32_t element_bound(const Ctx<F32> &c, uint32_t *scratch, int R, uint32_t *top)
{
    constexpr int E = RowElem<F32>::kPer;
    const auto each = [&](auto f) {
        for (int v = threadIdx.x; v < c.n; v += kSelThreads) {
            float x[E];
            granule_floats<F32>(c.get(v), x);
#pragma unroll
            for (int j = 0; j < E; ++j) f(x[j]);
        }
    };
    float hi = -INFINITY, lo = INFINITY;
    each([&](float x) {
        hi = fmaxf(hi, x);
        if (x > -INFINITY) lo = fminf(lo, x);
    });
    return group_bound(c.sh, scratch, R, hi, lo, top, each);
}
// (With fewer groups than R there is no bound at all, with not many more a loose one; a short row the list takes whole.)
__host__ __device__ inline bool few_groups(int groups, int elements, int R) { return groups < 2 * R && elements > 512; }

// ------------------------------------------------------------------ groups of a row that streams through registers
constexpr int kTurn = 8;               // granules in flight per thread
constexpr int kMaxGroups = 16;         // groups of a thread, at most

// Granules of a group: `size` (1, 2, 4 or 8) in each of `turns` (1 unless size is 8) turns.
struct Groups {
    int size, turns;
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

// Their maxima to gm[group][thread], kMaxGroups at most; returns how many groups the thread has.
template <bool F32>
__device__ __forceinline__ int group_maxima(const Ctx<F32> &c, Groups q, float *gm, float *hi, float *lo)
{
    const int tid = threadIdx.x;
    switch (q.size) {
    case 1: group_maxima<F32, 1>(c, 1, gm + tid, hi, lo); break;
    case 2: group_maxima<F32, 2>(c, 1, gm + tid, hi, lo); break;
    case 4: group_maxima<F32, 4>(c, 1, gm + tid, hi, lo); break;
    default: group_maxima<F32, 8>(c, q.turns, gm + tid, hi, lo); break;
    }
    const int S = q.size * q.turns, turns = tid < c.n ? (c.n - tid + kTurn * kSelThreads - 1) / (kTurn * kSelThreads) : 0;
    return (turns * kTurn + S - 1) / S;
}

// The CTA's elements from fb on, read again in the groups whose maximum is: to `own`, in no order; sh->nlist says how many
// there are (or more than cap), of which the first cap are there.  hits: cap words.
template <bool F32>
__device__ __forceinline__ void collect_groups(const Ctx<F32> &c, Groups q, const float *gm, int mine, int *hits, float fb,
                                               unsigned long long *own, int cap)
{
    constexpr int E = RowElem<F32>::kPer;
    Shared *sh = c.sh;
    const int tid = threadIdx.x, S = q.size * q.turns;
    if (tid == 0) sh->nlist = sh->nhits = 0;
    __syncthreads();
    for (int g = 0; g < mine; ++g)
        if (gm[g * kSelThreads + tid] >= fb) {
            const uint32_t at = atomicAdd(&sh->nhits, 1u);
            if (at < (uint32_t)cap) hits[at] = g * kSelThreads + tid;
        }
    __syncthreads();
    const int nhits = min((int)sh->nhits, cap);
    // granule j of group g of thread t is number (g S + j) kSelThreads + t of the CTA's
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
                const uint32_t at = atomicAdd(&sh->nlist, 1u);
                if (at < (uint32_t)cap) own[at] = ((unsigned long long)key_of(f[j]) << 32) | (uint32_t)~(uint32_t)(i0 + j);
            }
    }
    __syncthreads();
    // (a group has a candidate: with more groups than that there are too many of them)
    if (tid == 0 && sh->nhits > (uint32_t)cap) sh->nlist = sh->nhits;
    __syncthreads();
}

template <bool F32>
__device__ __forceinline__ void set_ctx(Ctx<F32> &c, const uint4 *cache, int cached, int C, Shared *sh,
                                        int cap = kListCap)
{
    c.C = C;
    c.cap = cap;
    c.rank = blockIdx.x & (C - 1);
    const int per = (c.r.G + C - 1) >> (31 - __clz(C));   // (C is a power of two)
    c.gb = min(c.r.G, (int)c.rank * per);
    c.n = min(c.r.G - c.gb, per);
    const int wper = (c.n + kSelWarps - 1) / kSelWarps, warp = threadIdx.x >> 5;
    c.wb = min(c.n, warp * wper);
    c.we = min(c.n, c.wb + wper);
    c.cached = cached;
    c.cache = cache;
    c.sh = sh;
    c.turn = 0;
}

// ------------------------------------------------------------------ launches (host)
constexpr int kSms = 152;

// CTAs of a row: one where the rows alone fill the GPU, more where they do not, as long as each has a few granules per
// thread; with few rows so many that a row's list of `want` entries falls to them in parts of at most kSmall; and so many
// that a share of at most `share` bytes (0: any) is left to each.  Top logits of 128256 bf16 ones with 1 / 2 / 4 / 8 CTAs
// (us): 38 rows, K 64 15.4 / 13.0 / 11.6 / 12.1; 76 rows 18.3 / 14.6 / 13.2 / 21.3; 304 rows 23.2 / 22.4 / 34.6 / 51.2;
// 1216 rows 63 / 75 / 102 / 170.  At K 1000: 38 rows 33.8 / 23.3 / 20.0 / 19.4, 76 rows 40 / 25.5 / 22.5 / 32.5 (here the
// rule's 8 are not the best: clusters of eight begin a second wave), 152 rows 45 / 29 / 36 / 51, 304 rows 49 / 39 / 53 / 88.
int logits_cluster(int rows, int64_t row_bytes, int want, size_t share)
{
    int C = 1;
    while (C < kRowMaxCluster && ((share && row_bytes > (int64_t)C * (int64_t)share) ||
                                  (((int64_t)rows * C < 2 * kSms || (want > C * (kSmall * 3 / 4) && rows < kSms)) &&
                                   row_bytes >= 2 * (int64_t)C * kSelThreads * 16)))
        C *= 2;
    return C;
}

// Groups of a row's granules for `groups` (4 to kMaxGroups) of each thread.
Groups plan_groups(int64_t row_bytes, int cluster, int groups)
{
    const int64_t each = (row_bytes / 16 / cluster + 4 + kSelThreads - 1) / kSelThreads;   // granules of a thread, at most
    const int64_t rounded = (each + kTurn - 1) / kTurn * kTurn;
    Groups q{1, 1};
    while (q.size < kTurn && q.size * groups < rounded) q.size *= 2;
    while ((int64_t)q.size * q.turns * groups < rounded) q.turns *= 2;
    return q;
}

sats_status check_rows(const void *logits, int64_t ld, int rows, int V, int bytes)
{
    if (rows < 0 || V < 1 || ld < V) return SATS_EINVAL;
    if (V > INT_MAX - 64 || rows > INT_MAX / kRowMaxCluster || ld > (int64_t)1 << 40) return SATS_ESHAPE;
    if (rows > 0 && (!logits || reinterpret_cast<uintptr_t>(logits) % bytes)) return SATS_EINVAL;
    return SATS_OK;
}

}  // namespace
}  // namespace sats
