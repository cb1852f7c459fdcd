// logits.cu -- the top logits of a row and the drawing of a token from it (sats_top_logits, sats_sample).
//
// One row per thread-block cluster.  The row's share of a CTA is brought to shared memory once; all passes after
// that run there.  Both calls start from the row's largest logits:
//   - while the row arrives, each thread keeps the maxima of a few groups of its elements.  At least R groups have
//     their maximum at or above the R-th largest of these maxima, so that at least R elements do: with
//     R = ceil(K / C) in each of C CTAs, the least of their bounds has K elements of the row at or above it;
//   - the elements at or above the bound (about K of them in a row of no particular order) go to a list in the first
//     CTA, which sorts it: descending logits, ties by the lower index.
// A row whose list would not fit (many equal logits, or large ones that share few groups) takes the general way: the
// exact K-th largest key by bisection over the keys, counting in every step.
//
// Drawing needs sums over up to V tokens that decide next to borders as close as the smallest token's probability.
// A token's weight is therefore a whole number, w = 2^F exp((z - max) / T) to about 35 bits relative (never less
// than 2^-F absolute), computed in pairs of floats; sums of whole numbers do not depend on their order, and every
// decision (the nucleus, the drawn token) is the same in whichever grouping it is found.
#include <climits>
#include <cmath>

#include "internal.h"
#include "rows.cuh"

namespace sats {
namespace {

constexpr int kMaxTop = 1024;          // largest K of the list's way
constexpr int kListCap = 2048;         // entries of the list
constexpr uint32_t kKeyNone = 0x007fffffu;   // key of -inf: never selected
constexpr int kAhead = 8;              // granules in flight per thread while the row arrives
constexpr size_t kShare = 64 * 1024;   // of a row's bytes per CTA, where the cluster allows
constexpr size_t kMaxCache = 184 * 1024;

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

// ------------------------------------------------------------------ weights
// 2^(j / 1024) in two floats: the leading 24 bits, and the rest times 2^41.
struct Exp2Table {
    float v[1024][2];
};
constexpr Exp2Table make_exp2_table()
{
    Exp2Table t{};
    for (int j = 0; j < 1024; ++j) {
        const double x = j * (0.69314718055994530942 / 1024.0);
        double term = 1.0, sum = 0.0;
        for (int k = 24; k > 0; --k) sum = (1.0 + sum) * (x / k);   // exp(x) - 1
        term += sum;
        const float hi = (float)term;
        t.v[j][0] = hi;
        t.v[j][1] = (float)((term - (double)hi) * 2199023255552.0);
    }
    return t;
}
__device__ const Exp2Table kExp2 = make_exp2_table();

// How a row's weights are scaled.
struct Scale {
    float top;        // the row's largest logit
    float chi, clo;   // log2(e) / T in two floats
    int F;            // fraction bits of a weight
    bool hard;        // only the largest logits weigh anything (they are +inf, or T next to nothing)
};

// chi + clo = log2(e) / T to twice the precision.
__device__ __forceinline__ void set_scale(Scale &s, float top, float T, int V)
{
    constexpr float Lh = 1.44269504f, Ll = 1.92596299e-8f;   // log2(e) in two floats
    s.top = top;
    s.hard = top == INFINITY || T < 1e-30f;
    s.chi = __fdiv_rn(Lh, T);
    s.clo = __fdiv_rn(__fadd_rn(fmaf(-s.chi, T, Lh), Ll), T);
    const int bits = 32 - __clz(V - 1);       // V - 1 < 2^bits
    s.F = min(50, 62 - (V > 1 ? bits : 0));   // V weights of at most 2^F + 1 stay below 2^63
}

// round-to-odd keeps the sums unbiased: what the shift drops counts as one half of the last place kept.
__device__ __forceinline__ unsigned long long weight(float z, const Scale &s, const float2 *tab)
{
    if (s.hard) return z == s.top ? (1ull << s.F) | 1ull : 0ull;
    // x = z - top exactly, in two floats
    const float xh = __fsub_rn(z, s.top);
    const float bv = __fsub_rn(z, xh), av = __fadd_rn(xh, bv);
    const float xl = __fadd_rn(__fsub_rn(z, av), __fsub_rn(bv, s.top));
    const float p = __fmul_rn(xh, s.chi);
    if (!(p > -(float)(s.F - 1))) return 0ull;   // (-inf among them)
    const float e = fmaf(xl, s.chi, fmaf(xh, s.clo, fmaf(xh, s.chi, -p)));
    // p = g / 1024 + rest, exactly
    constexpr float kMagic = 12288.f;            // 1.5 * 2^13: one unit in the last place is 2^-10
    const float m = __fadd_rn(p, kMagic);
    const int g = __float_as_int(m) - __float_as_int(kMagic);
    const float r = __fadd_rn(__fsub_rn(p, __fsub_rn(m, kMagic)), e);   // |r| <= 2^-11, and a little
    // 2^r - 1, times 2^41
    constexpr float L = 0.69314718055994530942f, S41 = 2199023255552.f;
    const float q = r * fmaf(r, fmaf(r, S41 * (L * L * L / 6.f), S41 * (L * L / 2.f)), S41 * L);
    const float2 t = tab[g & 1023];
    const int lo = __float2int_rn(fmaf(t.x, q, t.y));
    const uint32_t hi24 = __float_as_uint(t.x) - 0x3f000000u;   // t.x = hi24 / 2^23
    const unsigned long long w = ((unsigned long long)hi24 << 18) + (long long)lo;   // 41 fraction bits
    const int down = 61 - s.F - (g >> 10);       // in 0..61 (p > 1 - F)
    return ((w << 20) >> down) | 1ull;
}

// f * total for 0 <= f < 1, exactly and rounded down (and up): shares of a mass at a border are not to depend on a
// rounded product.
__device__ __forceinline__ unsigned long long share_floor(float f, unsigned long long total, bool *exact)
{
    const uint32_t b = __float_as_uint(f), ex = b >> 23;
    const uint32_t m = ex ? (b & 0x7fffffu) | 0x800000u : b;   // f = m 2^-down
    const int down = ex ? 150 - (int)ex : 149;                 // 24 or more
    const unsigned long long lo = total * m, hi = __umul64hi(total, (unsigned long long)m);
    unsigned long long r, rest;
    if (down < 64) {
        r = (hi << (64 - down)) | (lo >> down);                // (below 2^63: f < 1)
        rest = lo << (64 - down);
    } else if (down < 128) {
        r = down == 64 ? hi : hi >> (down - 64);
        rest = lo | (down == 64 ? 0ull : hi << (128 - down));
    } else {
        r = 0;
        rest = lo | hi;
    }
    *exact = rest == 0;
    return r;
}
__device__ __forceinline__ unsigned long long share_floor(float f, unsigned long long total)
{
    bool exact;
    return share_floor(f, total, &exact);
}
__device__ __forceinline__ unsigned long long share_ceil(float f, unsigned long long total)
{
    bool exact;
    const unsigned long long r = share_floor(f, total, &exact);
    return exact ? r : r + 1ull;
}

// ------------------------------------------------------------------ the row in a cluster
struct Shared {
    unsigned long long wsum[kRowWarps];
    unsigned long long scan[kRowWarps];
    unsigned long long slot[2][kRowMaxCluster];      // all-reduce, two buffers in turn
    uint32_t kmax[kRowMaxCluster], bound[kRowMaxCluster], cnt[kRowMaxCluster];
    int part[2][kRowWarps];
    uint32_t ktop[kRowWarps];
    uint32_t nlist;
    int found_idx;
    uint32_t found_key;
    uint32_t kminp;
    int flag;
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

    // Granule v of this CTA's, NaN replaced by -inf.
    __device__ __forceinline__ uint4 get(int v) const
    {
        uint4 x = v < cached ? cache[v] : load_granule<F32>(r, gb + v);
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
    for (int w = 0; w < kRowWarps; ++w) t += sh->wsum[w];
    return t;
}

// The CTAs' values, in every CTA's slots; returns their buffer.
template <bool F32>
__device__ __forceinline__ const unsigned long long *cluster_gather(Ctx<F32> &c, unsigned long long v)
{
    unsigned long long *slot = c.sh->slot[c.turn];
    c.turn ^= 1;
    if (c.C == 1) {
        if (threadIdx.x == 0) slot[0] = v;
        __syncthreads();
        return slot;
    }
    if (threadIdx.x < (unsigned)c.C) st_peer_u64(peer_addr(slot + c.rank, threadIdx.x), v);
    cluster_sync_all();
    return slot;
}

template <bool F32>
__device__ __forceinline__ unsigned long long cluster_sum(Ctx<F32> &c, unsigned long long v)
{
    const unsigned long long *slot = cluster_gather(c, block_sum_u64(v, c.sh));
    unsigned long long t = 0;
    for (int k = 0; k < c.C; ++k) t += slot[k];
    return t;
}

// What is kept: keys above `key`, and of those equal to it the ones up to index `idx`.
struct Cut {
    uint32_t key;
    int idx;
    __device__ __forceinline__ bool keeps(uint32_t k, int i) const { return k > key || (k == key && i <= idx); }
};

// Sum of f(logit, key, index) over granule v.
template <bool F32, typename F>
__device__ __forceinline__ unsigned long long granule_sum(const Ctx<F32> &c, int v, F f)
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

// Sum over this thread's granules, lanes in turn over the warp's run of them.
template <bool F32, typename F>
__device__ __forceinline__ unsigned long long thread_sum(const Ctx<F32> &c, F f)
{
    unsigned long long s = 0;
    for (int v = c.wb + (int)(threadIdx.x & 31); v < c.we; v += 32) s += granule_sum(c, v, f);
    return s;
}

// The first token in the vocabulary's order at which the running sum of f passes `target` (which is below the sum
// over the row): *idx, *key in every CTA.  The CTA that holds it narrows a run of granules down sixteenfold a step.
template <bool F32, typename F>
__device__ void locate(Ctx<F32> &c, unsigned long long target, F f, int *idx, uint32_t *key)
{
    Shared *sh = c.sh;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const unsigned long long mine = block_sum_u64(thread_sum(c, f), sh);
    const unsigned long long *slot = cluster_gather(c, mine);
    unsigned long long before = 0;
    for (unsigned k = 0; k < c.rank; ++k) before += slot[k];
    if (target >= before && target - before < mine) {   // (one CTA)
        unsigned long long t = target - before;
        int a = 0, b = c.n, per = (c.n + kRowWarps - 1) / kRowWarps;
        for (;;) {
            int w = 0;
            while (w < kRowWarps - 1 && t >= sh->wsum[w]) t -= sh->wsum[w++];
            a = a + w * per;
            b = min(b, a + per);
            if (b - a <= 32) break;
            per = (b - a + kRowWarps - 1) / kRowWarps;
            unsigned long long s = 0;
            const int wb = min(b, a + warp * per), we = min(b, wb + per);
            for (int v = wb + lane; v < we; v += 32) s += granule_sum(c, v, f);
            block_sum_u64(s, sh);
        }
        if (warp == 0) {
            const int v = a + lane;
            const unsigned long long s = v < b ? granule_sum(c, v, f) : 0ull;
            unsigned long long incl = s;
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) {
                const unsigned long long u = __shfl_up_sync(0xffffffffu, incl, o);
                if (lane >= o) incl += u;
            }
            const unsigned long long excl = incl - s;
            if (t >= excl && t < incl) {
                constexpr int E = RowElem<F32>::kPer;
                float x[E];
                granule_floats<F32>(c.get(v), x);
                const int i0 = c.r.first(c.gb + v);
                unsigned long long run = excl;
                bool hit = false;
#pragma unroll
                for (int j = 0; j < E; ++j) {
                    const uint32_t k = key_of(x[j]);
                    if (k > kKeyNone) run += f(x[j], k, i0 + j);
                    if (!hit && run > t) {
                        hit = true;
                        for (int q = 0; q < c.C; ++q) {
                            st_peer_u32(peer_addr(&sh->found_idx, q), (uint32_t)(i0 + j));
                            st_peer_u32(peer_addr(&sh->found_key, q), k);
                        }
                    }
                }
            }
        }
    }
    if (c.C > 1) cluster_sync_all();
    else __syncthreads();
    *idx = sh->found_idx;
    *key = sh->found_key;
}

// The largest key at which sum(f over keys >= it) is at least `want` (1 <= want <= the sum over all), the sum over
// the keys above it in *above.
template <bool F32, typename F>
__device__ uint32_t bisect_key(Ctx<F32> &c, uint32_t kmax, unsigned long long want, F f, unsigned long long *above)
{
    uint32_t lo = kKeyNone + 1, hi = kmax + 1;   // sum(lo) >= want > sum(hi)
    unsigned long long s_hi = 0;
    while (hi - lo > 1) {
        const uint32_t mid = lo + (hi - lo) / 2;
        const unsigned long long s =
            cluster_sum(c, thread_sum(c, [&](float x, uint32_t k, int i) { return k >= mid ? f(x, k, i) : 0ull; }));
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
    if (cluster_sum(c, thread_sum(c, one)) <= (unsigned long long)k) return Cut{kKeyNone, -1};
    unsigned long long above;
    Cut cut;
    cut.key = bisect_key(c, kmax, (unsigned long long)k, one, &above);
    const uint32_t at = cut.key;
    uint32_t key;
    locate(c, (unsigned long long)k - above - 1ull, [at](float, uint32_t q, int) { return q == at ? 1ull : 0ull; },
           &cut.idx, &key);
    return cut;
}

// ------------------------------------------------------------------ the list
// Sorts n2 (a power of two) words descending; all threads of the CTA.
__device__ void sort_desc(unsigned long long *a, int n2)
{
    __syncthreads();
    for (int k = 2; k <= n2; k <<= 1) {
        for (int j = k >> 1; j > 0; j >>= 1) {
            for (int t = threadIdx.x; t < n2 / 2; t += kRowThreads) {
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

// Elements with keys from `bound` on that `cut` keeps, to the list of the cluster's first CTA, in no order.  Returns
// how many there are (in every CTA; the list is complete only if they fit, and `ok` says so).
template <bool F32>
__device__ int gather_list(Ctx<F32> &c, unsigned long long *list, uint32_t bound, Cut cut, bool *ok)
{
    constexpr int E = RowElem<F32>::kPer;
    Shared *sh = c.sh;
    const float fb = key_float(bound);
    if (threadIdx.x == 0) sh->nlist = 0;
    __syncthreads();
    for (int v = c.wb + (int)(threadIdx.x & 31); v < c.we; v += 32) {
        const uint4 x = c.get(v);
        if (!(granule_max<F32>(x) >= fb)) continue;
        float f[E];
        granule_floats<F32>(x, f);
        const int i0 = c.r.first(c.gb + v);
#pragma unroll
        for (int j = 0; j < E; ++j) {
            const uint32_t k = key_of(f[j]);
            if (k >= bound && k > kKeyNone && cut.keeps(k, i0 + j)) {
                const uint32_t at = atomicAdd(&sh->nlist, 1u);
                if (at < kListCap) list[at] = ((unsigned long long)k << 32) | (uint32_t)~(uint32_t)(i0 + j);
            }
        }
    }
    __syncthreads();
    const uint32_t mine = sh->nlist;
    const unsigned long long *slot = cluster_gather(c, (unsigned long long)mine);
    unsigned long long total = 0, before = 0;
    for (int k = 0; k < c.C; ++k) {
        if (k < (int)c.rank) before += slot[k];
        total += slot[k];
    }
    *ok = total <= kListCap;
    if (*ok && c.C > 1) {
        if (c.rank != 0)
            for (uint32_t i = threadIdx.x; i < mine; i += kRowThreads)
                st_peer_u64(peer_addr(list + before + i, 0), list[i]);
        cluster_sync_all();
    }
    return (int)(total < (unsigned long long)INT_MAX ? total : INT_MAX);
}

// Pads the list with zeros and sorts it; n <= kListCap.  (First CTA.)
__device__ void sort_list(unsigned long long *list, int n)
{
    const int n2 = pow2_at_least(n);
    for (int i = n + threadIdx.x; i < n2; i += kRowThreads) list[i] = 0ull;
    sort_desc(list, n2);
}

// Brings the row in and finds its largest key and, for want > 0, a bound with at least `want` elements at or above
// it (or below every element, if there are not so many).
template <bool F32>
__device__ void load_row(Ctx<F32> &c, uint4 *cache, int want, uint32_t *kmax, uint32_t *bound)
{
    constexpr int NG = F32 ? 4 : 8;   // groups of a thread
    Shared *sh = c.sh;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    uint32_t gm[4] = {0xff800000u, 0xff800000u, 0xff800000u, 0xff800000u};
    if constexpr (!F32)
        for (int k = 0; k < 4; ++k) gm[k] = 0xff80ff80u;
    const auto join = [&](const uint4 &x) {
        if constexpr (F32) {
            gm[0] = __float_as_uint(fmaxf(__uint_as_float(gm[0]), __uint_as_float(x.x)));
            gm[1] = __float_as_uint(fmaxf(__uint_as_float(gm[1]), __uint_as_float(x.y)));
            gm[2] = __float_as_uint(fmaxf(__uint_as_float(gm[2]), __uint_as_float(x.z)));
            gm[3] = __float_as_uint(fmaxf(__uint_as_float(gm[3]), __uint_as_float(x.w)));
        } else {
            gm[0] = bf16x2_max(gm[0], x.x);
            gm[1] = bf16x2_max(gm[1], x.y);
            gm[2] = bf16x2_max(gm[2], x.z);
            gm[3] = bf16x2_max(gm[3], x.w);
        }
    };
    if (c.C > 1) cluster_arrive();
    const int end = min(c.we, c.cached);
    for (int i = 0; i < kAhead; ++i) {
        const int v = c.wb + lane + 32 * i;
        if (v < end) fetch_granule<F32>(c.r, c.gb + v, cache + v);
        cp_async_commit();
    }
    for (int v = c.wb + lane; v < end; v += 32) {
        cp_async_wait<kAhead - 1>();
        join(cache[v]);
        const int next = v + 32 * kAhead;
        if (next < end) fetch_granule<F32>(c.r, c.gb + next, cache + next);
        cp_async_commit();
    }
    for (int v = max(c.wb, c.cached) + lane; v < c.we; v += 32) join(load_granule<F32>(c.r, c.gb + v));

    uint32_t key[NG], top = 0;
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        if constexpr (F32) {
            key[k] = key_of(__uint_as_float(gm[k]));
        } else {
            key[2 * k] = key_of(bf16_lo(gm[k]));
            key[2 * k + 1] = key_of(bf16_hi(gm[k]));
        }
    }
#pragma unroll
    for (int k = 0; k < NG; ++k) top = max(top, key[k]);
    top = __reduce_max_sync(0xffffffffu, top);
    if (lane == 0) sh->ktop[warp] = top;
    __syncthreads();
    top = sh->ktop[lane & (kRowWarps - 1)];
    top = __reduce_max_sync(0xffffffffu, top);

    uint32_t low = kKeyNone + 1;
    if (want > 0) {
        // the want-th largest of this CTA's group maxima, or a little below it
        const int R = (want + c.C - 1) / c.C;
        constexpr int kShift = F32 ? 0 : 16;         // bf16 keys differ in their upper halves alone
        uint32_t lo = (kKeyNone >> kShift) + (F32 ? 1 : 0), hi = (top >> kShift) + 1;   // count(lo) >= R is assumed: see below
        int turn = 0;
        while (hi - lo > 1) {
            const uint32_t mid = lo + (hi - lo) / 2;
            int n = 0;
#pragma unroll
            for (int k = 0; k < NG; ++k) n += (key[k] >> kShift) >= mid;
            n = __reduce_add_sync(0xffffffffu, n);
            if (lane == 0) sh->part[turn][warp] = n;
            __syncthreads();
            n = __reduce_add_sync(0xffffffffu, lane < kRowWarps ? sh->part[turn][lane] : 0);
            turn ^= 1;
            if (n >= R) {
                lo = mid;
                if (n <= R + (R >> 3)) break;
            } else {
                hi = mid;
            }
        }
        low = max(lo << kShift, kKeyNone + 1);   // the search ends at its lower end if there are fewer than R
    }
    if (c.C > 1) {
        cluster_wait();
        if (tid < c.C) {
            st_peer_u32(peer_addr(&sh->kmax[c.rank], tid), top);
            st_peer_u32(peer_addr(&sh->bound[c.rank], tid), low);
        }
        cluster_sync_all();
        for (int k = 0; k < c.C; ++k) {
            top = max(top, sh->kmax[k]);
            low = min(low, sh->bound[k]);
        }
    } else {
        __syncthreads();
    }
    *kmax = top;
    *bound = low;
}

template <bool F32>
__device__ __forceinline__ void set_ctx(Ctx<F32> &c, const uint4 *cache, int cached, int C, Shared *sh)
{
    c.C = C;
    c.rank = blockIdx.x % C;
    const int per = (c.r.G + C - 1) / C;
    c.gb = min(c.r.G, (int)c.rank * per);
    c.n = min(c.r.G - c.gb, per);
    const int wper = (c.n + kRowWarps - 1) / kRowWarps, warp = threadIdx.x >> 5;
    c.wb = min(c.n, warp * wper);
    c.we = min(c.n, c.wb + wper);
    c.cached = cached;
    c.cache = cache;
    c.sh = sh;
    c.turn = 0;
}

// The lowest index that has the largest key.
template <bool F32>
__device__ int lowest_at(Ctx<F32> &c, uint32_t kmax)
{
    constexpr int E = RowElem<F32>::kPer;
    const float fm = key_float(kmax);
    int best = INT_MAX;
    for (int v = c.wb + (int)(threadIdx.x & 31); v < c.we && best == INT_MAX; v += 32) {
        const uint4 x = c.get(v);
        if (!(granule_max<F32>(x) >= fm)) continue;
        float f[E];
        granule_floats<F32>(x, f);
        const int i0 = c.r.first(c.gb + v);
#pragma unroll
        for (int j = E - 1; j >= 0; --j)
            if (f[j] >= fm) best = i0 + j;
    }
    best = __reduce_min_sync(0xffffffffu, best);
    __syncthreads();
    if ((threadIdx.x & 31) == 0) c.sh->part[0][threadIdx.x >> 5] = best;
    __syncthreads();
    best = __reduce_min_sync(0xffffffffu, c.sh->part[0][threadIdx.x & (kRowWarps - 1)]);
    const unsigned long long *slot = cluster_gather(c, (unsigned long long)(unsigned)best);
    for (int k = 0; k < c.C; ++k) best = min(best, (int)(unsigned)slot[k]);
    return best;
}

struct TopParams {
    const void *z;
    int64_t ld;
    int T, V, K;
    float *values;
    int32_t *idx;
    int cluster, cached;
};

template <bool F32>
__global__ void __launch_bounds__(kRowThreads, 2) top_kernel(const TopParams p)
{
    extern __shared__ __align__(16) uint4 smem[];
    __shared__ Shared sh;
    const int row = blockIdx.x / p.cluster;
    unsigned long long *list = reinterpret_cast<unsigned long long *>(smem + p.cached);
    Ctx<F32> c{Row<F32>(p.z, row, p.ld, p.V)};
    set_ctx(c, smem, p.cached, p.cluster, &sh);
    uint32_t kmax, bound;
    load_row(c, smem, p.K, &kmax, &bound);
    bool ok;
    int n = gather_list(c, list, bound, Cut{kKeyNone, -1}, &ok);
    if (!ok) {   // (the same in every CTA of the row)
        const Cut cut = cut_count(c, kmax, p.K);
        n = gather_list(c, list, max(cut.key, kKeyNone + 1), cut, &ok);   // at most K
    }
    if (c.rank != 0) return;   // (nobody reads this CTA's memory any more)
    sort_list(list, n);
    for (int i = threadIdx.x; i < p.K; i += kRowThreads) {
        const unsigned long long e = i < n ? list[i] : 0ull;
        p.values[(size_t)row * p.K + i] = i < n ? key_float((uint32_t)(e >> 32)) : -INFINITY;
        p.idx[(size_t)row * p.K + i] = i < n ? (int32_t)~(uint32_t)e : -1;
    }
}

struct SampleParams {
    const void *z;
    int64_t ld;
    int B, V;
    const float *temperature;
    const int32_t *top_k;
    const float *top_p, *min_p, *u;
    int32_t *ids;
    float *logprob;
    int32_t *n_kept;
    int32_t *status;
    int cluster, cached;
};

__device__ __forceinline__ void put_sample(const SampleParams &p, int row, int id, float logprob, long long n)
{
    p.ids[row] = id;
    if (p.logprob) p.logprob[row] = logprob;
    if (p.n_kept) p.n_kept[row] = (int32_t)n;
}

// log(weight of z / total): the top logit is always kept, the total is 2^F or more.
__device__ __forceinline__ float log_share(float z, float T, const Scale &s, unsigned long long total)
{
    const float rest = (float)(long long)(total - (1ull << s.F)) * exp2f(-(float)s.F);
    return (z == s.top ? 0.f : (z - s.top) / T) - log1pf(rest);
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
    for (int w = 0; w < kRowWarps; ++w) {
        if (w < warp) before += sh->scan[w];
        t += sh->scan[w];
    }
    *total = t;
    return before + incl - v;
}

constexpr int kListPer = kListCap / kRowThreads;   // list entries of a thread, in a row

template <bool F32>
__global__ void __launch_bounds__(kRowThreads, 2) sample_kernel(const SampleParams p)
{
    extern __shared__ __align__(16) uint4 smem[];
    __shared__ Shared sh;
    __shared__ float2 tab[1024];
    const int row = blockIdx.x / p.cluster, tid = threadIdx.x;
    unsigned long long *list = reinterpret_cast<unsigned long long *>(smem + p.cached);
    const float T = p.temperature ? p.temperature[row] : 1.f;
    const float top_p = p.top_p ? p.top_p[row] : 1.f, min_p = p.min_p ? p.min_p[row] : 0.f;
    const float u = p.u[row];
    int k = p.top_k ? p.top_k[row] : 0;
    if (!(T >= 0.f) || T == INFINITY || top_p != top_p || !(min_p <= 1.f) || !(u >= 0.f && u < 1.f)) {
        if (blockIdx.x % p.cluster == 0 && tid == 0) {
            put_sample(p, row, -1, __int_as_float(0x7fffffff), 0);
            if (p.status) atomicOr(p.status, kStatusBadToken);
        }
        return;   // (every CTA of the row)
    }
    if (k < 0 || k >= p.V) k = 0;
    const bool greedy = T == 0.f || k == 1 || top_p <= 0.f;
    const bool nucleus = top_p < 1.f;
    // the list serves a top-k that fits it, and without one the nucleus if it lies within the largest logits
    const int want = greedy ? 0 : (k > 0 && k <= kMaxTop ? k : (k == 0 && nucleus ? kMaxTop : 0));
    for (int i = tid; i < 1024; i += kRowThreads) tab[i] = make_float2(kExp2.v[i][0], kExp2.v[i][1]);
    Ctx<F32> c{Row<F32>(p.z, row, p.ld, p.V)};
    set_ctx(c, smem, p.cached, p.cluster, &sh);
    uint32_t kmax, bound;
    load_row(c, smem, want, &kmax, &bound);
    if (kmax <= kKeyNone) {   // nothing can be drawn
        if (c.rank == 0 && tid == 0) put_sample(p, row, -1, -INFINITY, 0);
        return;
    }
    if (greedy) {
        const int id = lowest_at(c, kmax);
        if (c.rank == 0 && tid == 0) put_sample(p, row, id, 0.f, 1);
        return;
    }
    Scale s;
    set_scale(s, key_float(kmax), T, p.V);
    // min-p as the least key that is kept: exp((z - top) / T) >= min_p where z >= top + T log(min_p)
    uint32_t kminp = 0;
    if (min_p > 0.f) {
        if (tid == 0) {
            const double v = s.hard ? (double)s.top : (double)s.top + (double)T * log((double)min_p);
            float f = (float)v;
            if ((double)f < v) f = nextafterf(f, INFINITY);
            sh.kminp = key_of(f);
        }
        __syncthreads();
        kminp = sh.kminp;
    }
    const auto mass = [&](float x, uint32_t, int) { return weight(x, s, tab); };

    const bool only_minp = k == 0 && !nucleus && kminp > kKeyNone;
    if (want > 0 || only_minp) {
        unsigned long long Z = 0;
        if (k == 0 && nucleus) Z = cluster_sum(c, thread_sum(c, mass));
        // with a top-k the list must hold all of it: its mass is what top-p refers to
        const uint32_t from = k > 0 ? bound : max(want > 0 ? bound : kKeyNone + 1, kminp);
        bool ok;
        const int n = gather_list(c, list, from, Cut{kKeyNone, -1}, &ok);
        if (ok) {
            if (c.rank == 0) {
                sort_list(list, n);
                int m = k > 0 ? min(n, k) : n;
                unsigned long long w[kListPer], sum = 0, total;
                if (nucleus || k > 0) {
                    int in_minp = 0;
#pragma unroll
                    for (int j = 0; j < kListPer; ++j) {
                        const int i = tid * kListPer + j;
                        const uint32_t key = i < m ? (uint32_t)(list[i] >> 32) : 0u;
                        w[j] = i < m ? weight(key_float(key), s, tab) : 0ull;
                        sum += w[j];
                        in_minp += i < m && key >= kminp;
                    }
                    unsigned long long run = block_scan_u64(sum, &sh, &total);
                    if (k > 0) Z = total;
                    const unsigned long long target = nucleus ? share_ceil(top_p, Z) : ~0ull;
                    int in_p = 0;
#pragma unroll
                    for (int j = 0; j < kListPer; ++j) {
                        in_p += tid * kListPer + j < m && run < target;
                        run += w[j];
                    }
                    const unsigned long long both =
                        block_sum_u64(((unsigned long long)(unsigned)in_p << 32) | (unsigned)in_minp, &sh);
                    // the nucleus may reach beyond the list
                    if (k == 0 && total < target && from > kminp && from > kKeyNone + 1) m = -1;
                    else m = min((int)(both >> 32), (int)(uint32_t)both);
                }
                if (m > 0) {
                    // the kept ones in the vocabulary's order
                    const int m2 = pow2_at_least(m);
                    __syncthreads();
                    for (int i = tid; i < m2; i += kRowThreads) {
                        const unsigned long long e = list[i];
                        list[i] = i < m ? (e << 32) | (e >> 32) : 0ull;
                    }
                    sort_desc(list, m2);
                    sum = 0;
#pragma unroll
                    for (int j = 0; j < kListPer; ++j) {
                        const int i = tid * kListPer + j;
                        w[j] = i < m ? weight(key_float((uint32_t)list[i]), s, tab) : 0ull;
                        sum += w[j];
                    }
                    unsigned long long run = block_scan_u64(sum, &sh, &total);
                    const unsigned long long target = share_floor(u, total);
#pragma unroll
                    for (int j = 0; j < kListPer; ++j) {
                        const unsigned long long next = run + w[j];
                        if (target >= run && target < next) {   // one entry
                            const unsigned long long e = list[tid * kListPer + j];
                            put_sample(p, row, (int)~(uint32_t)(e >> 32),
                                       log_share(key_float((uint32_t)e), T, s, total), m);
                        }
                        run = next;
                    }
                }
                if (k == 0) {   // the others wait to hear whether that was all
                    __syncthreads();
                    if (tid < c.C) st_peer_u32(peer_addr(&sh.flag, tid), m > 0);
                }
            }
            if (k > 0) return;
            if (c.C > 1) cluster_sync_all();
            else __syncthreads();
            if (sh.flag) return;
        }
    }

    // the general way: the cuts one after the other, over the whole row
    Cut cut{kKeyNone, -1};
    if (k > 0) cut = cut_count(c, kmax, k);
    if (nucleus) {
        const Cut by_k = cut;
        const auto kept = [&](float x, uint32_t q, int i) { return by_k.keeps(q, i) ? weight(x, s, tab) : 0ull; };
        const unsigned long long Z = cluster_sum(c, thread_sum(c, kept));
        const unsigned long long want_mass = max(share_ceil(top_p, Z), 1ull);
        unsigned long long above;
        const uint32_t key = bisect_key(c, kmax, want_mass, kept, &above);
        // ties at the border: the first of them that reach the mass
        const unsigned long long w = weight(key_float(key), s, tab);
        const unsigned long long ties = (want_mass - above + w - 1ull) / w;
        uint32_t at;
        locate(c, ties - 1ull, [=](float, uint32_t q, int i) { return q == key && by_k.keeps(q, i) ? 1ull : 0ull; },
               &cut.idx, &at);
        cut.key = key;
    }
    if (kminp > cut.key) cut = Cut{kminp - 1u, -1};
    const Cut last = cut;
    const unsigned long long count =
        cluster_sum(c, thread_sum(c, [&](float, uint32_t q, int i) { return last.keeps(q, i) ? 1ull : 0ull; }));
    const auto kept = [&](float x, uint32_t q, int i) { return last.keeps(q, i) ? weight(x, s, tab) : 0ull; };
    const unsigned long long total = cluster_sum(c, thread_sum(c, kept));
    int id;
    uint32_t key;
    locate(c, share_floor(u, total), kept, &id, &key);
    if (c.rank == 0 && tid == 0) put_sample(p, row, id, log_share(key_float(key), T, s, total), (long long)count);
}

int logits_cluster(int rows, int64_t row_bytes)
{
    int C = 1;
    while (C < kRowMaxCluster && (row_bytes > (int64_t)C * (int64_t)kShare ||
                                  ((int64_t)rows * C < 2 * 152 && row_bytes >= 2 * (int64_t)C * kRowThreads * 16)))
        C *= 2;
    return C;
}

// Cluster and shared memory of a launch over `rows` rows.
template <bool F32, typename P>
cudaError_t launch_rows(void (*kern)(const P), P p, int rows, cudaStream_t st)
{
    const int64_t bytes = (int64_t)p.V * RowElem<F32>::kBytes;
    p.cluster = logits_cluster(rows, bytes);
    const size_t share = (size_t)((bytes + 32 + p.cluster - 1) / p.cluster) + 32;
    p.cached = (int)((share < kMaxCache ? share : kMaxCache) / 16);
    const size_t smem = (size_t)p.cached * 16 + kListCap * 8;
    if (smem > 32 * 1024) {
        const cudaError_t e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                                   (int)(kMaxCache + kListCap * 8));
        if (e != cudaSuccess) return e;
    }
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)rows * (unsigned)p.cluster);
    cfg.blockDim = dim3(kRowThreads);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = st;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = (unsigned)p.cluster;
    attr[0].val.clusterDim.y = 1;
    attr[0].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, kern, p);
}

sats_status check_rows(const void *logits, int64_t ld, int rows, int V, int bytes)
{
    if (rows < 0 || V < 1 || ld < V) return SATS_EINVAL;
    if (V > INT_MAX - 64 || rows > INT_MAX / kRowMaxCluster || ld > (int64_t)1 << 40) return SATS_ESHAPE;
    if (rows > 0 && (!logits || reinterpret_cast<uintptr_t>(logits) % bytes)) return SATS_EINVAL;
    return SATS_OK;
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
    const cudaError_t e = launch_rows<F32, TopParams>(top_kernel<F32>, p, T, static_cast<cudaStream_t>(stream));
    return e == cudaSuccess ? SATS_OK : cuda_fail(e, "top-logits kernel launch");
}

template <bool F32>
sats_status sample(const void *logits, int64_t ld, int B, int V, const float *temperature, const int32_t *top_k,
                   const float *top_p, const float *min_p, const float *u, int32_t *ids, float *logprob,
                   int32_t *n_kept, int32_t *dev_status, void *stream)
{
    const sats_status s = check_rows(logits, ld, B, V, RowElem<F32>::kBytes);
    if (s != SATS_OK || B == 0) return s;
    if (!u || !ids) return SATS_EINVAL;
    SampleParams p{};
    p.z = logits; p.ld = ld; p.B = B; p.V = V; p.temperature = temperature; p.top_k = top_k; p.top_p = top_p;
    p.min_p = min_p; p.u = u; p.ids = ids; p.logprob = logprob; p.n_kept = n_kept; p.status = dev_status;
    const cudaError_t e = launch_rows<F32, SampleParams>(sample_kernel<F32>, p, B, static_cast<cudaStream_t>(stream));
    return e == cudaSuccess ? SATS_OK : cuda_fail(e, "sampling kernel launch");
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

sats_status sats_sample(const void *logits, int64_t ld, int B, int V, const float *temperature, const int32_t *top_k,
                        const float *top_p, const float *min_p, const float *u, int32_t *ids, float *logprob,
                        int32_t *n_kept, int32_t *dev_status, void *stream)
{
    return sats::sample<false>(logits, ld, B, V, temperature, top_k, top_p, min_p, u, ids, logprob, n_kept, dev_status,
                               stream);
}

sats_status sats_sample_f32(const float *logits, int64_t ld, int B, int V, const float *temperature,
                            const int32_t *top_k, const float *top_p, const float *min_p, const float *u, int32_t *ids,
                            float *logprob, int32_t *n_kept, int32_t *dev_status, void *stream)
{
    return sats::sample<true>(logits, ld, B, V, temperature, top_k, top_p, min_p, u, ids, logprob, n_kept, dev_status,
                              stream);
}

}  // extern "C"
