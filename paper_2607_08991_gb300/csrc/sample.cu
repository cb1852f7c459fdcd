// sample.cu -- drawing a token from each row of logits (sats_sample).
//
// Rows of bf16 logits are drawn by sample_values_kernel, which counts their values; fp32 rows, short ones and very long
// ones by sample_kernel, which brings the row's share of a CTA to shared memory once and makes all its passes there.
//
// Drawing needs sums over up to V tokens that decide next to borders as close as the smallest token's probability.
// A token's weight is therefore a whole number, w = 2^F exp((z - max) / T) to about 35 bits relative (never less
// than 2^-F absolute), computed in pairs of floats; sums of whole numbers do not depend on their order, and every
// decision (the nucleus, the drawn token) is the same in whichever grouping it is found.
#include <algorithm>

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

constexpr int kAhead = 8;              // granules in flight per thread while the row arrives
// Of a row's bytes per CTA, where the cluster allows (300 fp32 top-p rows with 128 KB 307 us, with 64 KB 233).
constexpr size_t kShare = 64 * 1024;
constexpr size_t kMaxCache = 182 * 1024;
constexpr size_t kMaxSmem = kMaxCache + (size_t)kListCap * 8;
static_assert(kMaxSmem + 13 * 1024 <= kSmemPerCta, "with the kernel's static part");

// ------------------------------------------------------------------ weights
// 2^(-j / 1024) in two floats.
struct Exp2Table {
    float2 v[1024];
};
constexpr Exp2Table make_exp2_table()
{
    Exp2Table t{};
    for (int j = 0; j < 1024; ++j) {
        const double x = -j * (0.69314718055994530942 / 1024.0);
        double rest = 0.0;
        for (int k = 24; k > 0; --k) rest = (1.0 + rest) * (x / k);   // exp(x) - 1
        const double v = 1.0 + rest;
        t.v[j].x = (float)v;
        t.v[j].y = (float)(v - (double)t.v[j].x);
    }
    return t;
}
__device__ const Exp2Table kExp2 = make_exp2_table();

// How a row's weights are scaled.
struct Scale {
    float top;        // the row's largest logit
    float chi, clo;   // log2(e) / T in two floats
    float magic;      // 1.5 * 2^(23 - F): one unit in the last place is 2^-F
    int F;            // fraction bits of a weight, 43 at most
    bool hard;        // only the largest logits weigh anything (they are +inf, or T is next to nothing)
};

// chi + clo = log2(e) / T to twice the precision.
__device__ __forceinline__ void set_scale(Scale &s, float top, float T, int V)
{
    constexpr float Lh = 1.44269504f, Ll = 1.92596299e-8f;   // log2(e) in two floats
    s.top = top;
    s.hard = top == INFINITY || T < 1e-30f;
    s.chi = __fdiv_rn(Lh, T);
    s.clo = __fdiv_rn(__fadd_rn(fmaf(-s.chi, T, Lh), Ll), T);
    s.F = min(43, 62 - (32 - __clz(V)));      // V weights of 2^F stay below 2^62
    s.magic = __int_as_float(((127 + 23 - s.F) << 23) | 0x400000);
}

constexpr float kMagicG = 12288.f;   // 1.5 * 2^13: one unit in the last place is 2^-10
constexpr float kMagicW = 6.f;       // 1.5 * 2^2: 2^-21

// Two weights 2^F exp((z - top) / T) as whole numbers (i1 << (F - 21)) + i2, where z <= top; `in` says whether they
// can be other than 0 (false for NaN and -inf, whose numbers mean nothing).  g: g / 1024 octaves below the top.
// Sums of floats in pairs throughout; relative error about 2^-35, from the rounding of r L and T.x q to 24 bits.
struct Weights2 {
    int i1[2], i2[2], g[2];
    bool in[2];
};
__device__ __forceinline__ Weights2 weights2(f32x2 z, const Scale &s, const float2 *tab)
{
    const auto both = [](float v) { return pack2(v, v); };
    constexpr float L = 0.69314718055994530942f;
    const f32x2 minus1 = both(-1.f), nt = both(-s.top), chi = both(s.chi);
    const f32x2 xh = fadd2(z, nt);
    const f32x2 bv = ffma2(xh, minus1, z);
    const f32x2 xl = fadd2(ffma2(fadd2(xh, bv), minus1, z), fadd2(bv, nt));   // xh + xl = z - top, exactly
    // y - e = (top - z) log2(e) / T
    const f32x2 y = fmul2(xh, both(-s.chi));
    const f32x2 e = ffma2(xl, chi, ffma2(xh, both(s.clo), ffma2(xh, chi, y)));
    // y = g / 1024 - what r starts from, exactly
    const f32x2 m = fadd2(y, both(kMagicG));
    const f32x2 r = fadd2(ffma2(y, minus1, fadd2(m, both(-kMagicG))), e);   // |r| <= 2^-11, and a little
    // q = 2^r - 1 (the next term is below 2^-37)
    const f32x2 q = fmul2(r, ffma2(r, both(L * L / 2.f), both(L)));
    const float2 mm = unpack2(m), yy = unpack2(y);
    Weights2 w;
    w.g[0] = __float_as_int(mm.x) - __float_as_int(kMagicG);
    w.g[1] = __float_as_int(mm.y) - __float_as_int(kMagicG);
    w.in[0] = yy.x < 60.f;
    w.in[1] = yy.y < 60.f;
    const float2 t0 = tab[w.g[0] & 1023], t1 = tab[w.g[1] & 1023];
    const f32x2 tx = pack2(t0.x, t1.x);
    const f32x2 lo = ffma2(tx, q, pack2(t0.y, t1.y));
    // h + l = 2^(-(g mod 1024) / 1024 + r), scaled by 2^(-(g div 1024))
    const f32x2 h = fadd2(tx, lo);
    const f32x2 l = ffma2(ffma2(tx, minus1, h), minus1, lo);
    const f32x2 sc = pack2(__int_as_float(0x3f800000 - ((w.g[0] << 13) & 0xff800000)),
                           __int_as_float(0x3f800000 - ((w.g[1] << 13) & 0xff800000)));
    const f32x2 hs = fmul2(h, sc);
    const f32x2 m1 = fadd2(hs, both(kMagicW));
    const f32x2 d = ffma2(l, sc, ffma2(fadd2(m1, both(-kMagicW)), minus1, hs));
    const float2 a = unpack2(m1), b = unpack2(fadd2(d, both(s.magic)));
    w.i1[0] = __float_as_int(a.x) - __float_as_int(kMagicW);
    w.i1[1] = __float_as_int(a.y) - __float_as_int(kMagicW);
    w.i2[0] = __float_as_int(b.x) - __float_as_int(s.magic);
    w.i2[1] = __float_as_int(b.y) - __float_as_int(s.magic);
    return w;
}

__device__ __forceinline__ unsigned long long whole_weight(int i1, int i2, const Scale &s)
{
    return ((unsigned long long)(unsigned)i1 << (s.F - 21)) + (long long)i2;
}

// One weight.
__device__ __forceinline__ unsigned long long weight(float z, const Scale &s, const float2 *tab)
{
    if (s.hard) return z == s.top ? 1ull << s.F : 0ull;
    const Weights2 w = weights2(pack2(z, z), s, tab);
    return w.in[0] ? whole_weight(w.i1[0], w.i2[0], s) : 0ull;
}

// f * total for 0 <= f < 1 (not -0), exactly and rounded down (and up): shares of a mass at a border are not to depend on a
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

// Granules whose weights' parts add up in 32 bits (256 weights of at most 2^21 and less).
constexpr int kFlush = 32;

// The kept tokens' weights.
struct KeptMass {
    const Scale &s;
    const float2 *tab;
    Cut cut;
    float at;   // the cut's key as a logit
    __device__ __forceinline__ KeptMass(const Scale &s_, const float2 *t_, Cut c_)
        : s(s_), tab(t_), cut(c_), at(key_float(c_.key)) {}
    __device__ __forceinline__ unsigned long long elem(float x, uint32_t k, int i) const
    {
        return cut.keeps(k, i) ? weight(x, s, tab) : 0ull;
    }
    __device__ __forceinline__ bool keeps(float x, int i) const { return x > at || (x == at && i <= cut.idx); }
    template <bool F32>
    __device__ __forceinline__ unsigned long long granule(const Ctx<F32> &c, int v) const
    {
        int n = 0;
        return granule(c, v, n);
    }
    // ... and their number, added to n
    template <bool F32>
    __device__ __forceinline__ unsigned long long granule(const Ctx<F32> &c, int v, int &n) const
    {
        int a1 = 0, a2 = 0;
        add(c, v, a1, a2, n);
        return whole_weight(a1, a2, s);   // (eight weights at most)
    }
    // (CUT: something is cut; without, every token above -inf is kept)
    template <bool CUT = true, bool F32>
    __device__ __forceinline__ void add(const Ctx<F32> &c, int v, int &a1, int &a2, int &n) const
    {
        constexpr int P = RowElem<F32>::kPer / 2;
        const uint4 x = c.raw(v);
        if (CUT && !(granule_max<F32>(x) >= at)) return;
        f32x2 z[P];
        granule_pairs<F32>(c.clean(x), z);
        const int i0 = c.r.first(c.gb + v);
        const auto kept = [&](float f, int i) { return CUT ? keeps(f, i) : f > -INFINITY; };
        if (s.hard) {
#pragma unroll
            for (int j = 0; j < P; ++j) {
                const float2 y = unpack2(z[j]);
                const bool k0 = kept(y.x, i0 + 2 * j), k1 = kept(y.y, i0 + 2 * j + 1);
                n += k0 + k1;
                a1 += ((k0 && y.x == s.top) + (k1 && y.y == s.top)) << 21;
            }
        } else {
#pragma unroll
            for (int j = 0; j < P; ++j) {
                const float2 y = unpack2(z[j]);
                const Weights2 w = weights2(z[j], s, tab);
                const bool k0 = kept(y.x, i0 + 2 * j), k1 = kept(y.y, i0 + 2 * j + 1);
                n += k0 + k1;
                if (k0 && w.in[0]) { a1 += w.i1[0]; a2 += w.i2[0]; }
                if (k1 && w.in[1]) { a1 += w.i1[1]; a2 += w.i2[1]; }
            }
        }
    }
    // Sum over this thread's granules.
    template <bool CUT, bool F32>
    __device__ __forceinline__ unsigned long long over_row(const Ctx<F32> &c, int &n) const
    {
        unsigned long long sum = 0;
        for (int v0 = c.wb + (int)(threadIdx.x & 31); v0 < c.we; v0 += 32 * kFlush) {
            int a1 = 0, a2 = 0;
            for (int v = v0; v < min(c.we, v0 + 32 * kFlush); v += 32) add<CUT>(c, v, a1, a2, n);
            sum += whole_weight(a1, a2, s);
        }
        return sum;
    }
};

// ------------------------------------------------------------------ the row
// Sends for a thread's first granules.
template <bool F32>
__device__ __forceinline__ void start_row(const Ctx<F32> &c, uint4 *cache)
{
    if (c.C > 1) cluster_arrive();   // (load_row waits)
    const int end = min(c.we, c.cached);
    for (int i = 0; i < kAhead; ++i) {
        const int v = c.wb + (int)(threadIdx.x & 31) + 32 * i;
        if (v < end) fetch_granule<F32>(c.r, c.gb + v, cache + v);
        cp_async_commit();
    }
}

// Brings the row in and finds its largest key and, for want > 0, a bound with at least `want` elements at or above
// it (or below every element, if there are not so many).  scratch: kBoundBins words.
__host__ __device__ constexpr int groups_of(bool f32) { return f32 ? 4 : 8; }   // of a thread
template <bool FEW, bool F32>
__device__ void load_row(Ctx<F32> &c, uint4 *cache, int want, uint32_t *scratch, uint32_t *kmax, uint32_t *bound)
{
    constexpr int NG = groups_of(F32);
    Shared *sh = c.sh;
    const int tid = threadIdx.x, lane = tid & 31;
    if (want > 0)
        for (int i = tid; i < kBoundBins; i += kSelThreads) scratch[i] = 0u;
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
    const int end = min(c.we, c.cached);
    for (int v = c.wb + lane; v < end; v += 32) {
        cp_async_wait<kAhead - 1>();
        join(cache[v]);
        const int next = v + 32 * kAhead;
        if (next < end) fetch_granule<F32>(c.r, c.gb + next, cache + next);
        cp_async_commit();
    }
    for (int v = max(c.wb, c.cached) + lane; v < c.we; v += 32) join(load_granule<F32>(c.r, c.gb + v));

    // the groups' maxima
    float g[NG], hi = -INFINITY, lo = INFINITY;
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        if constexpr (F32) {
            g[k] = fmaxf(__uint_as_float(gm[k]), -INFINITY);
        } else {
            g[2 * k] = fmaxf(bf16_lo(gm[k]), -INFINITY);
            g[2 * k + 1] = fmaxf(bf16_hi(gm[k]), -INFINITY);
        }
    }
#pragma unroll
    for (int k = 0; k < NG; ++k) {
        hi = fmaxf(hi, g[k]);
        if (want > 0 && g[k] > -INFINITY) lo = fminf(lo, g[k]);
    }
    uint32_t top, low;
    const int R = (want + c.C - 1) >> (31 - __clz(c.C));
    bool few = false;
    if constexpr (FEW) {
        few = few_groups(min(c.n, kSelThreads) * NG, min(c.n, 1 << 20) * RowElem<F32>::kPer, R);
        if (few) {
            __syncthreads();   // (others' granules)
            low = element_bound(c, scratch, R, &top);
        }
    }
    if (!few) {
        low = group_bound(sh, scratch, R, hi, lo, &top, [&](auto f) {
#pragma unroll
            for (int k = 0; k < NG; ++k) f(g[k]);
        });
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

// ------------------------------------------------------------------ the nucleus
// Where the mass from the top reaches a share of the whole, in two passes over the row.  The first counts the tokens in
// 2048 equal steps of the weight's logarithm, each as 4096 times its weight relative to the middle of its step (right
// to kOff): no exponential, one addition in shared memory a token.  From all CTAs' counts follow the steps in which the
// border can lie, as a rule one or two.  The second pass takes the exact weights: of all tokens, of the ones above these
// steps, and a list of the ones within, which settles the border; that it lies there at all is checked.  (A step's 32 bits
// hold 2^20 tokens of a CTA, less a few: rows of over 8 million logits can run them over, to any number.  A border that
// they then put in a wrong place fails that check; counts of 0 in all, as 2^20 alike in each CTA leave, put it nowhere.)
constexpr int kBins = 2048;
static_assert(2 * kBins * 4 <= kListCap * 8, "the counts, and their exchange, lie where the list does");
// Half a 1 / 1024 octave, the straight line instead of the power within a step, the rounding to 1 / 4096.
constexpr float kOff = 7e-4f;

struct Nucleus {
    Cut cut;
    bool sums;   // sh->wsum has the warps' kept mass, sh->mass and sh->above the CTAs' and their numbers of kept tokens
};

// Ties at one key, `above` the mass before them: the cut at the first of them with which the mass reaches `want`.
template <bool F32>
__device__ Cut cut_ties(Ctx<F32> &c, uint32_t key, unsigned long long w, unsigned long long above,
                        unsigned long long want, Cut by_k)
{
    const unsigned long long ties = (want - above + w - 1ull) / w;
    Cut cut;
    uint32_t at;
    sum_and_locate(c, ties - 1ull,
                   by_elem([=](float, uint32_t q, int i) { return q == key && by_k.keeps(q, i) ? 1ull : 0ull; }),
                   &cut.idx, &at);
    cut.key = key;
    return cut;
}

// The parts of a list that lie `seg` entries apart (sh->cnt of each), one behind another.
__device__ __noinline__ void one_behind_another(unsigned long long *list, int seg, int n, int C, Shared *sh)
{
    for (int i0 = 0; i0 < n; i0 += kSelThreads) {   // (from the first on: nothing is overwritten before it is read)
        const int i = i0 + (int)threadIdx.x;
        unsigned long long e = 0;
        if (i < n) {
            int k = 0, from = 0;
            while (i - from >= (int)sh->cnt[k]) from += (int)sh->cnt[k++];
            e = list[k * seg + i - from];
        }
        __syncthreads();
        if (i < n) list[i] = e;
        __syncthreads();
    }
}

// The last entry, from the largest down, that the mass `want` still reaches: to sh->found_key and found_idx.  For lists
// that are sorted for it.
__device__ __noinline__ void cut_in_list(unsigned long long *list, int n, unsigned long long want, Scale s,
                                         const float2 *tab, Shared *sh)
{
    sort_list(list, n);
    const int first = (int)threadIdx.x * kListPer;
    unsigned long long sum = 0, rest;
    for (int i = first; i < min(n, first + kListPer); ++i) sum += weight(key_float((uint32_t)(list[i] >> 32)), s, tab);
    unsigned long long before = block_scan_u64(sum, sh, &rest);
    for (int i = first; i < min(n, first + kListPer); ++i) {
        const unsigned long long x = list[i], w = weight(key_float((uint32_t)(x >> 32)), s, tab);
        if (before < want && want - before <= w) {   // (one thread)
            sh->found_key = (uint32_t)(x >> 32);
            sh->found_idx = (int)~(uint32_t)x;
        }
        before += w;
    }
}

// Gives each CTA its run of the kBins words `count` of all CTAs, one CTA's behind another's: to `got`, or in place where
// there is one CTA.  A barrier ahead.
template <bool F32>
__device__ __forceinline__ uint32_t *exchange_counts(Ctx<F32> &c, uint32_t *count, uint32_t *got)
{
    if (c.C == 1) return count;
    const int nb = kBins / c.C;
    for (int i = threadIdx.x; i < kBins / 4; i += kSelThreads) {
        const uint4 q = reinterpret_cast<const uint4 *>(count)[i];
        const int b = 4 * i;
        st_peer_v4(peer_addr(got + c.rank * nb + b % nb, b / nb), __uint_as_float(q.x), __uint_as_float(q.y),
                   __uint_as_float(q.z), __uint_as_float(q.w));
    }
    cluster_sync_all();
    return got;
}

// Where more tokens than the list holds lie in the steps [d0, d1) of 1 / 1024 octave that have the border, with `want` of
// mass to be reached there: their exact masses step by step, and the list of the one step that has it, as cut_by_counts
// leaves it (the CTAs' parts in every CTA, sh->cnt).  Returns what of the mass is to be reached in the list; 0 where that
// does not do.  (300 fp32 rows of 100003 with a temperature of 20 and top-p 0.5: 490 us, by bisection 2760.)
template <bool FILTERED, bool F32>
__device__ __noinline__ unsigned long long list_of_one_step(Ctx<F32> c, Scale s, const float2 *tab, Cut by_k,
                                                            unsigned long long *list, int d0, int d1, unsigned long long want)
{
    constexpr int E = RowElem<F32>::kPer, P = E / 2, kFine = 128;
    static_assert((kRowMaxCluster + 1) * kFine + 1 <= kListCap && kFine <= kSelThreads, "the masses lie where the list does");
    Shared *sh = c.sh;
    const KeptMass all(s, tab, by_k);
    const int tid = threadIdx.x, lane = tid & 31, C = c.C;
    if ((unsigned)(d1 - d0) > (unsigned)kFine) return 0;
    unsigned long long *fine = list + kRowMaxCluster * kFine, *before = fine + kFine;
    // f(logit, index, step) for the tokens of a run of steps
    const auto over = [&](int from, int n, auto f) {
        const f32x2 nt = pack2(-s.top, -s.top), chi = pack2(-s.chi, -s.chi), magic = pack2(kMagicG, kMagicG);
        for (int v = c.wb + lane; v < c.we; v += 32) {
            f32x2 z[P];
            granule_pairs<F32>(c.get(v), z);
            const int i0 = c.r.first(c.gb + v);
#pragma unroll
            for (int j = 0; j < P; ++j) {
                const f32x2 y2 = fmul2(fadd2(z[j], nt), chi);   // (as weights2 does)
                const float2 x = unpack2(z[j]), y = unpack2(y2), m = unpack2(fadd2(y2, magic));
                const int base = __float_as_int(kMagicG) + from, i = i0 + 2 * j;
                const int a = __float_as_int(m.x) - base, b = __float_as_int(m.y) - base;
                if (y.x < 60.f && (unsigned)a < (unsigned)n && (!FILTERED || all.keeps(x.x, i))) f(x.x, i, a);
                if (y.y < 60.f && (unsigned)b < (unsigned)n && (!FILTERED || all.keeps(x.y, i + 1))) f(x.y, i + 1, b);
            }
        }
    };
    __syncthreads();
    if (tid < kFine) fine[tid] = 0;
    __syncthreads();
    over(d0, d1 - d0, [&](float x, int, int d) { atomicAdd(fine + d, weight(x, s, tab)); });
    __syncthreads();
    if (tid < kFine)
        for (int q = 0; q < C; ++q) st_peer_u64(peer_addr(list + c.rank * kFine + tid, q), fine[tid]);
    if (tid == 0) {
        sh->nlist = 0;
        sh->border = -1;
    }
    if (C > 1) cluster_sync_all();
    else __syncthreads();
    unsigned long long m = 0, total;
    if (tid < kFine)
        for (int k = 0; k < C; ++k) m += list[k * kFine + tid];
    const unsigned long long run = block_scan_u64(m, sh, &total);
    if (run < want && want - run <= m) {   // (one thread)
        sh->border = tid;
        *before = run;
    }
    __syncthreads();
    const int border = sh->border;
    if (border < 0) return 0;   // (the same in every CTA of the row)
    want -= *before;
    if (C > 1) cluster_sync_all();   // (all have read the masses)
    else __syncthreads();
    const int seg = kListCap / C;
    unsigned long long *own = list + c.rank * seg;
    over(d0 + border, 1, [&](float x, int i, int) {
        const uint32_t at = atomicAdd(&sh->nlist, 1u);
        if (at < (uint32_t)seg) own[at] = ((unsigned long long)key_of(x) << 32) | (uint32_t)~(uint32_t)i;
    });
    __syncthreads();
    const int here = (int)sh->nlist;
    if (here <= seg)
        for (int q = 1; q < C; ++q) {
            const unsigned to = (c.rank + q) % C;
            for (int i = tid; i < here; i += kSelThreads) st_peer_u64(peer_addr(own + i, to), own[i]);
        }
    if (tid < C) st_peer_u32(peer_addr(&sh->cnt[c.rank], tid), (uint32_t)here);
    if (C > 1) cluster_sync_all();
    else __syncthreads();
    for (int k = 0; k < C; ++k)
        if (sh->cnt[k] > (uint32_t)seg) return 0;
    return want;
}

// The cut that keeps, of what by_k keeps, the largest up to a share top_p < 1 of the mass, by counts and exact weights;
// false (the same in every CTA of the row) where the border does not lie where the counts have it, or among more
// tokens than the list holds.
template <bool FILTERED, bool F32>
__device__ bool cut_by_counts(Ctx<F32> &c, const Scale &s, const float2 *tab, unsigned long long *list, Cut by_k,
                              float top_p, Nucleus *res)
{
    constexpr int E = RowElem<F32>::kPer, P = E / 2;
    Shared *sh = c.sh;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, C = c.C;
    const KeptMass all(s, tab, by_k);
    // steps as fine as 128 logits, or what weighs more than 2^-64, allow
    int shift = 0;
    while (shift < 5 && (float)(2 << shift) < 128.f * s.chi) ++shift;
    uint32_t *count = reinterpret_cast<uint32_t *>(list), *got = count + kBins;
    for (int i = tid; i < kBins / 4; i += kSelThreads) reinterpret_cast<uint4 *>(count)[i] = make_uint4(0, 0, 0, 0);
    __syncthreads();
    {
        const f32x2 nt = pack2(-s.top, -s.top), chi = pack2(-s.chi, -s.chi), magic = pack2(kMagicG, kMagicG);
        const uint32_t mask = (1u << shift) - 1u;
        const auto add = [&](float y, float m) {
            if (!(y < 60.f)) return;
            const uint32_t d = (uint32_t)(__float_as_int(m) - __float_as_int(kMagicG));   // 1 / 1024 octaves below the top
            const int v = 4096 + (((int)mask - 2 * (int)(d & mask)) * 2839 >> 11);         // ln 2 * 2 = 2839 / 2048
            atomicAdd(count + min(d >> shift, (uint32_t)kBins - 1u), (uint32_t)v);
        };
        for (int v = c.wb + lane; v < c.we; v += 32) {
            f32x2 z[P];
            granule_pairs<F32>(c.get(v), z);
            const int i0 = c.r.first(c.gb + v);
#pragma unroll
            for (int j = 0; j < P; ++j) {
                const f32x2 y2 = fmul2(fadd2(z[j], nt), chi);   // (as weights2 does)
                const float2 f = unpack2(z[j]), y = unpack2(y2), m = unpack2(fadd2(y2, magic));
                if (!FILTERED || all.keeps(f.x, i0 + 2 * j)) add(y.x, m.x);
                if (!FILTERED || all.keeps(f.y, i0 + 2 * j + 1)) add(y.y, m.y);
            }
        }
    }
    __syncthreads();
    const int nb = kBins / C;
    got = exchange_counts(c, count, got);
    constexpr int kMost = kBins / kSelThreads;
    const int per = (nb + kSelThreads - 1) / kSelThreads;
    unsigned long long m[kMost], mine = 0;   // masses in whole numbers: their sums are the same in every CTA
#pragma unroll
    for (int j = 0; j < kMost; ++j) {
        const int b = tid * per + j;
        m[j] = 0;
        if (j < per && b < nb) {
            unsigned long long n = 0;
            for (int k = 0; k < C; ++k) n += got[k * nb + b];
            const float mid = ((float)((c.rank * nb + b) << shift) + 0.5f * (float)(1 << shift)) * (1.f / 1024.f);
            m[j] = (unsigned long long)__float2ll_rn((float)n * exp2f(20.f - mid));
        }
        mine += m[j];
    }
    unsigned long long total;
    unsigned long long run = block_scan_u64(mine, sh, &total);
    const unsigned long long *slot = cluster_gather(c, total);
    const unsigned long long Zs = slot_sum(slot, C);
    if (Zs == 0) return false;   // (the same in every CTA of the row; from here on one step is the border's, each way)
    for (unsigned k = 0; k < c.rank; ++k) run += slot[k];
    {
        const float rest = 1.f - top_p;
        const auto reached = [&](unsigned long long cum, float off) {   // cum / Z >= top_p, both sides off by a factor
            return (float)cum * (rest * (1.f + off)) >= (float)(Zs - cum) * (top_p * (1.f - off));
        };
#pragma unroll
        for (int j = 0; j < kMost; ++j) {
            if (m[j] != 0) {
                const uint32_t b = c.rank * nb + tid * per + j;
                if (!reached(run, kOff) && reached(run + m[j], kOff))   // (one thread)
                    for (int k = 0; k < C; ++k) st_peer_u32(peer_addr(&sh->bin0, k), b);
                if (!reached(run, -kOff) && reached(run + m[j], -kOff))   // (one thread)
                    for (int k = 0; k < C; ++k) st_peer_u32(peer_addr(&sh->bin1, k), b);
            }
            run += m[j];
        }
    }
    if (tid == 0) sh->nlist = 0;
    if (C > 1) cluster_sync_all();
    else __syncthreads();

    // exact weights; each CTA's entries have a part of the list of their own, in every CTA
    const int seg = kListCap / C;
    unsigned long long *own = list + c.rank * seg;
    const int d0 = (int)sh->bin0 << shift, d1 = sh->bin1 >= kBins - 1u ? INT_MAX : (int)(sh->bin1 + 1u) << shift;
    unsigned long long w_all = 0, w_above = 0;
    int n_above = 0;
    for (int v0 = c.wb + lane; v0 < c.we; v0 += 32 * kFlush) {
        int a1 = 0, a2 = 0, t1 = 0, t2 = 0;
        for (int v = v0; v < min(c.we, v0 + 32 * kFlush); v += 32) {
            f32x2 z[P];
            granule_pairs<F32>(c.get(v), z);
            const int i0 = c.r.first(c.gb + v);
#pragma unroll
            for (int j = 0; j < P; ++j) {
                const Weights2 w = weights2(z[j], s, tab);
                const float2 y = unpack2(z[j]);
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const float f = h ? y.y : y.x;
                    const int i = i0 + 2 * j + h, d = w.g[h];
                    const bool in = w.in[h] && (!FILTERED || all.keeps(f, i));
                    if (in) { t1 += w.i1[h]; t2 += w.i2[h]; }
                    if (in && d < d0) { a1 += w.i1[h]; a2 += w.i2[h]; ++n_above; }
                    if (in && (unsigned)(d - d0) < (unsigned)(d1 - d0)) {
                        const uint32_t at = atomicAdd(&sh->nlist, 1u);
                        if (at < (uint32_t)seg) own[at] = ((unsigned long long)key_of(f) << 32) | (uint32_t)~(uint32_t)i;
                    }
                }
            }
        }
        w_all += whole_weight(t1, t2, s);
        w_above += whole_weight(a1, a2, s);
    }
    w_all = warp_sum_u64(w_all);
    w_above = warp_sum_u64(w_above);
    n_above = (int)__reduce_add_sync(0xffffffffu, n_above);
    if (lane == 0) {
        sh->scan[warp] = w_all;
        sh->wsum[warp] = w_above;
        sh->part[warp] = n_above;
    }
    __syncthreads();
    w_all = w_above = 0;
    for (int w = 0; w < kSelWarps; ++w) {
        w_all += sh->scan[w];
        w_above += sh->wsum[w];
    }
    n_above = (int)__reduce_add_sync(0xffffffffu, lane < kSelWarps ? sh->part[lane] : 0);
    const int here = (int)sh->nlist;
    if (here <= seg)
        for (int q = 1; q < C; ++q) {   // (each CTA begins with its neighbour)
            const unsigned to = (c.rank + q) % C;
            for (int i = tid; i < here; i += kSelThreads) st_peer_u64(peer_addr(own + i, to), own[i]);
        }
    if (tid < C) {
        st_peer_u32(peer_addr(&sh->cnt[c.rank], tid), (uint32_t)here);
        st_peer_u32(peer_addr(&sh->above[c.rank], tid), (uint32_t)n_above);
    }
    slot = cluster_gather(c, w_all, w_above);
    const unsigned long long Z = slot_sum(slot, C), A = slot_sum(slot + kRowMaxCluster, C), target = share_ceil(top_p, Z);
    if (A >= target) return false;
    unsigned long long want = target - A;
    bool fits = true;
    for (int k = 0; k < C; ++k) fits = fits && sh->cnt[k] <= (uint32_t)seg;
    if (!fits) {
        want = list_of_one_step<FILTERED>(c, s, tab, by_k, list, d0, d1, want);
        if (want == 0) return false;   // (the same in every CTA of the row)
    }
    int n = 0, off = 0;   // entries; of the CTAs before this one
    for (int k = 0; k < C; ++k) {
        if (k < (int)c.rank) off += (int)sh->cnt[k];
        n += (int)sh->cnt[k];
    }
    if (n == 0) return false;
    // every CTA does what follows: the entries one behind another, and the last one that is kept
    if (tid == 0) sh->found_idx = -1;
    if (C > 1) one_behind_another(list, seg, n, C, sh);
    else __syncthreads();
    if (n <= kSmall) {
        const Small m(list, n);
        const unsigned long long w = m.on ? weight(key_float(m.key()), s, tab) : 0ull;
        m.put_weight(list, w);
        __syncthreads();
        int rank;
        unsigned long long before;
        m.larger(list, n, &rank, &before);
        if (m.on && m.part == 0 && before < want && want - before <= w) {   // (one thread)
            sh->found_key = m.key();
            sh->found_idx = m.idx();
        }
    } else {
        cut_in_list(list, n, want, s, tab, sh);
    }
    __syncthreads();
    const Cut cut{sh->found_key, sh->found_idx};
    *res = Nucleus{cut, false};
    if (cut.idx < 0 || n > kSmall || !fits) return cut.idx >= 0;
    // what is kept of the CTAs, a warp each; then of this CTA's warps
    if (warp < C) {
        int from = 0;
        for (int k = 0; k < warp; ++k) from += (int)sh->cnt[k];
        unsigned long long w = 0;
        int kept = 0;
        for (int i = from + lane; i < from + (int)sh->cnt[warp]; i += 32)
            if (cut.keeps((uint32_t)(list[i] >> 32), (int)~(uint32_t)list[i])) {
                w += list[kSmall + i];
                ++kept;
            }
        w = warp_sum_u64(w);
        kept = (int)__reduce_add_sync(0xffffffffu, kept);
        if (lane == 0) {
            sh->mass[warp] = slot[kRowMaxCluster + warp] + w;
            sh->above[warp] += (uint32_t)kept;
        }
    }
    const int wper = (c.n + kSelWarps - 1) / kSelWarps;
    unsigned long long w = 0;
    for (int i = off + lane; i < off + here; i += 32) {
        const unsigned long long e = list[i];
        const int idx = (int)~(uint32_t)e, v = (int)(((unsigned)idx + (unsigned)c.r.head) / E) - c.gb;
        if (v >= warp * wper && v < (warp + 1) * wper && cut.keeps((uint32_t)(e >> 32), idx)) w += list[kSmall + i];
    }
    w = warp_sum_u64(w);
    if (lane == 0) sh->wsum[warp] += w;
    __syncthreads();
    res->sums = true;
    return true;
}

// The same in any case: where the counts do not do, the key by bisection and its ties by their order.
template <bool F32>
__device__ Nucleus cut_mass(Ctx<F32> &c, const Scale &s, const float2 *tab, unsigned long long *list, uint32_t kmax,
                            Cut by_k, float top_p)
{
    Nucleus res;
    if (!s.hard && (by_k.key > kKeyNone ? cut_by_counts<true>(c, s, tab, list, by_k, top_p, &res)
                                        : cut_by_counts<false>(c, s, tab, list, by_k, top_p, &res)))
        return res;
    const KeptMass all(s, tab, by_k);
    const auto f = [&](float x, uint32_t q, int i) { return by_k.keeps(q, i) ? weight(x, s, tab) : 0ull; };
    const unsigned long long Z = cluster_sum(c, thread_sum(c, all)), want = share_ceil(top_p, Z);
    unsigned long long above = 0;
    const uint32_t key = s.hard ? kmax : bisect_key(c, kKeyNone + 1, kmax, want, f, &above);
    return Nucleus{cut_ties(c, key, weight(key_float(key), s, tab), above, want, by_k), false};
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
    if ((threadIdx.x & 31) == 0) c.sh->part[threadIdx.x >> 5] = best;
    __syncthreads();
    best = __reduce_min_sync(0xffffffffu, c.sh->part[threadIdx.x & (kSelWarps - 1)]);
    const unsigned long long *slot = cluster_gather(c, (unsigned long long)(unsigned)best);
    for (int k = 0; k < c.C; ++k) best = min(best, (int)(unsigned)slot[k]);
    return best;
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
    Groups groups;
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

// The draw from a list of the row's largest n >= k entries that is sorted for it.
__device__ __noinline__ void draw_from_list(const SampleParams &p, int row, unsigned long long *list, int n, int k,
                                            float top_p, uint32_t kminp, float u, float T, Scale s, const float2 *tab,
                                            Shared *sh)
{
    sort_list(list, n);
    const int first = (int)threadIdx.x * kListPer;
    const auto weight_at = [&](int i, int shift) { return weight(key_float((uint32_t)(list[i] >> shift)), s, tab); };
    int m = min(n, k);
    unsigned long long sum = 0, total;
    if (top_p < 1.f || kminp > 0) {
        int in_p = 0, in_minp = 0;
        for (int i = first; i < min(m, first + kListPer); ++i) {
            sum += weight_at(i, 32);
            in_minp += (uint32_t)(list[i] >> 32) >= kminp;
        }
        unsigned long long run = block_scan_u64(sum, sh, &total);
        const unsigned long long target = top_p < 1.f ? share_ceil(top_p, total) : ~0ull;
        for (int i = first; i < min(m, first + kListPer); ++i) {
            in_p += run < target;
            run += weight_at(i, 32);
        }
        const unsigned long long both = block_sum_u64(((unsigned long long)(unsigned)in_p << 32) | (unsigned)in_minp, sh);
        m = min((int)(both >> 32), (int)(uint32_t)both);
    }
    // the kept ones in the vocabulary's order
    const int m2 = pow2_at_least(m);
    __syncthreads();
    for (int i = threadIdx.x; i < m2; i += kSelThreads) {
        const unsigned long long e = list[i];
        list[i] = i < m ? (e << 32) | (e >> 32) : 0ull;
    }
    sort_desc(list, m2);
    sum = 0;
    for (int i = first; i < min(m, first + kListPer); ++i) sum += weight_at(i, 0);
    unsigned long long run = block_scan_u64(sum, sh, &total);
    const unsigned long long target = share_floor(u, total);
    for (int i = first; i < min(m, first + kListPer); ++i) {
        const unsigned long long next = run + weight_at(i, 0);
        if (target >= run && target < next) {   // one entry
            const unsigned long long e = list[i];
            put_sample(p, row, (int)~(uint32_t)(e >> 32), log_share(key_float((uint32_t)e), T, s, total), m);
        }
        run = next;
    }
}

// What a row asks for.
struct Settings {
    float T, top_p, min_p, u;
    int k;                  // 0: off
    bool bad, greedy, nucleus;

    __device__ __forceinline__ Settings(const SampleParams &p, int row)
    {
        T = p.temperature ? p.temperature[row] : 1.f;
        top_p = p.top_p ? p.top_p[row] : 1.f;
        min_p = p.min_p ? p.min_p[row] : 0.f;
        u = p.u[row] + 0.f;   // (-0 is 0)
        k = p.top_k ? p.top_k[row] : 0;
        bad = !(T >= 0.f) || T == INFINITY || top_p != top_p || !(min_p <= 1.f) || !(u >= 0.f && u < 1.f);
        if (k < 0 || k >= p.V) k = 0;
        greedy = T == 0.f || k == 1 || top_p <= 0.f;
        nucleus = top_p < 1.f;
    }
};

__device__ __forceinline__ void put_bad(const SampleParams &p, int row)
{
    put_sample(p, row, -1, __int_as_float(0x7fffffff), 0);
    if (p.status) atomicOr(p.status, kStatusBadToken);
}

// min-p as the least key that is kept: exp((z - top) / T) >= min_p where z >= top + T log(min_p).  All threads.
__device__ __forceinline__ uint32_t least_key(const Settings &set, const Scale &s, Shared *sh)
{
    if (!(set.min_p > 0.f)) return 0;
    if (threadIdx.x == 0) {
        const double v = s.hard ? (double)s.top : (double)s.top + (double)set.T * log((double)set.min_p);
        float f = (float)v;
        if ((double)f < v) f = nextafterf(f, INFINITY);
        sh->kminp = key_of(f);
    }
    __syncthreads();
    return sh->kminp;
}

// The draw from the n largest entries of a row, the k largest among them (k 0: all that is kept is).
__device__ __forceinline__ void draw_list(const SampleParams &p, int row, const Settings &set, const Scale &s,
                                          unsigned long long *list, int n, uint32_t kminp, const float2 *tab, Shared *sh)
{
    const int k = set.k > 0 ? set.k : INT_MAX;
    const float T = set.T, u = set.u, top_p = set.top_p;
    if (n <= kSmall) {
        const Small e(list, n);
        const unsigned long long w = e.on ? weight(key_float(e.key()), s, tab) : 0ull;
        e.put_weight(list, w);
        __syncthreads();
        int at;
        unsigned long long above;
        e.larger(list, n, &at, &above);
        bool kept = e.on && at < k && e.key() >= kminp;
        if (set.nucleus) {
            const unsigned long long Z = block_sum_u64(e.on && e.part == 0 && at < k ? w : 0ull, sh);
            kept = kept && above < share_ceil(top_p, Z);
        }
        const int m = __syncthreads_count(kept && e.part == 0);
        e.put_weight(list, kept ? w : 0ull);
        const unsigned long long total = block_sum_u64(kept && e.part == 0 ? w : 0ull, sh);
        const unsigned long long before = e.earlier(list, n), target = share_floor(u, total);
        if (kept && e.part == 0 && target >= before && target - before < w)   // one entry
            put_sample(p, row, e.idx(), log_share(key_float(e.key()), T, s, total), m);
        return;
    }
    draw_from_list(p, row, list, n, k, set.nucleus ? top_p : 1.f, kminp, u, T, s, tab, sh);
}

// The draw in any case, after start_row.
template <bool FEW, bool F32>
__device__ __forceinline__ void sample_row(Ctx<F32> &c, const SampleParams &p, int row, const Settings &set, uint4 *cache,
                                           unsigned long long *list, const float2 *tab)
{
    Shared &sh = *c.sh;
    const int tid = threadIdx.x, k = set.k;
    const float T = set.T, u = set.u, top_p = set.top_p;
    const int want = !set.greedy && k > 0 && k <= kMaxTop ? k : 0;   // what the list serves
    uint32_t kmax, bound;
    load_row<FEW>(c, cache, want, reinterpret_cast<uint32_t *>(list), &kmax, &bound);
    if (kmax <= kKeyNone) {   // nothing can be drawn
        if (c.rank == 0 && tid == 0) put_sample(p, row, -1, -INFINITY, 0);
        return;
    }
    if (set.greedy) {
        const int id = lowest_at(c, kmax);
        if (c.rank == 0 && tid == 0) put_sample(p, row, id, 0.f, 1);
        return;
    }
    Scale s;
    set_scale(s, key_float(kmax), T, p.V);
    const uint32_t kminp = least_key(set, s, &sh);

    if (want > 0) {
        bool ok;
        const int n = gather_list(c, list, bound, Cut{kKeyNone, INT_MIN}, &ok);
        if (ok) {   // (the same in every CTA of the row)
            if (c.rank != 0) return;   // (nobody reads this CTA's memory any more)
            draw_list(p, row, set, s, list, n, kminp, tab, &sh);
            return;
        }
    }

    // over the whole row: the cuts one after the other, then the kept mass and the token in it
    Cut cut{kKeyNone, INT_MIN};
    if (k > 0) cut = cut_count(c, kmax, k);
    bool sums = false;
    if (set.nucleus) {
        const Nucleus q = cut_mass(c, s, tab, list, kmax, cut, top_p);
        cut = q.cut;
        sums = q.sums;
    }
    if (kminp > cut.key) {
        cut = Cut{kminp, INT_MAX};
        sums = false;
    }
    const KeptMass kept(s, tab, cut);
    const unsigned long long *mass = sh.mass;
    unsigned long long count = 0;
    if (sums) {
        for (int q = 0; q < c.C; ++q) count += sh.above[q];
    } else {
        int n = 0;
        unsigned long long mine = cut.key > kKeyNone ? kept.template over_row<true>(c, n) : kept.template over_row<false>(c, n);
        n = (int)__reduce_add_sync(0xffffffffu, n);
        __syncthreads();
        if ((tid & 31) == 0) sh.part[tid >> 5] = n;
        mine = block_sum_u64(mine, &sh);
        n = __reduce_add_sync(0xffffffffu, (tid & 31) < kSelWarps ? sh.part[tid & 31] : 0);
        mass = cluster_gather(c, mine, (unsigned long long)(unsigned)n);
        count = slot_sum(mass + kRowMaxCluster, c.C);
    }
    const unsigned long long total = slot_sum(mass, c.C);
    locate(c, share_floor(u, total), kept, mass, [&](int id, uint32_t key) {
        put_sample(p, row, id, log_share(key_float(key), T, s, total), (long long)count);
    });
}

// The row in shared memory, three CTAs of 256 threads to an SM (1024 x 1, 512 x 2, 256 x 4 and 128 x 6 were slower).  300 rows
// of 100003 fp32 logits with top-p take 233 us, where reading them takes 18: the counting pass issues about 25 and the
// exact pass about 60 instructions an element (a weight of 35 bits is some 20 operations on pairs of floats), over half of
// the issue slots that there are, and five barriers of the cluster stand between the passes.  Four rows of 1000: 10.8 us.
//
// FEW: there may be few_groups (the calls to see to it cost 4 to 8 % of the other draws).
template <bool F32, bool FEW>
__global__ void __launch_bounds__(kSelThreads, kSelPerSm) sample_kernel(const SampleParams p)
{
    extern __shared__ __align__(16) uint4 smem[];
    __shared__ Shared sh;
    __shared__ float2 tab[1024];
    const int row = (int)(blockIdx.x >> (31 - __clz(p.cluster))), tid = threadIdx.x;
    unsigned long long *list = reinterpret_cast<unsigned long long *>(smem + p.cached);
    Ctx<F32> c{Row<F32>(p.z, row, p.ld, p.V)};
    set_ctx(c, smem, p.cached, p.cluster, &sh);
    start_row(c, smem);
    const Settings set(p, row);
    if (set.bad) {
        if (c.rank == 0 && tid == 0) put_bad(p, row);
        cp_async_wait<0>();
        if (c.C > 1) cluster_wait();
        return;   // (every CTA of the row)
    }
    if (!set.greedy)
        for (int i = tid; i < 1024; i += kSelThreads) tab[i] = kExp2.v[i];
    sample_row<FEW>(c, p, row, set, smem, list, tab);
}

// ------------------------------------------------------------------ bf16 rows by their values
// A bf16 row has few different values that weigh anything: the tokens of each are counted while the row streams through
// registers, and all that is asked for (the k-th largest, the mass, the nucleus' border, the kept mass of every CTA)
// follows exactly from the counts and one weight per value.  Only the CTA in which the token lies reads its tokens again
// (from the L2) and adds their weights from a table of the values.
//
// 512 rows of 128256 bf16 logits (19 us of reading) take 135 us free, 165 with top-p, 155 with a top-k of up to 1000, 90
// with min-p, 74 with a top-k of 50, 53 greedy; with the row in shared memory (sample_kernel) they take 159, 373, 198, 115,
// 101 and 59.  A count is about ten instructions a token, an addition in shared memory among them: 57 us until
// the row is counted, 36 if it were only read.  Then 25 to 50 us go into the weights of 4096 values, the border and two
// exchanges, and 35 to 45 into the one CTA of a row that adds its tokens' weights (two lookups of 8 bytes in the table
// cost a conflict of banks each): chains of latency, covered by three other CTAs on the SM.
//
// The values of magnitudes from 2^-10 to below 2^6 have a step each, in descending order.  Smaller ones are listed one by
// one; of those from -2^6 down, which have no weight, the number is known.  What does not fit this (larger logits, many tiny
// ones, a border among the listed ones) is drawn the general way.
constexpr int kSteps = 2 * kBins;   // two counts of 16 bits in a word
constexpr int kFewMax = kSelThreads;
constexpr int kLeastMag = 117 << 7, kFarMag = 133 << 7;   // magnitudes as bits
static_assert(kFarMag - kLeastMag == kSteps / 2, "a step for each value");
constexpr int kValuesPerSm = 4;   // (3, with more registers: 256 mixed rows 83 us, 512 free ones 140; with 4 81 and 135)
// Tokens of a row: with 4096 steps a row, short rows of a free draw are slower this way (512 rows of 8000: 31 us against
// 22; of 32000: 52 against 49), all others faster (of 8000 with top-p 42 against 49, top-k 43 against 70; of 2000 with top-p
// 34 against 40, free 26 against 15).  One rule whatever the settings: which of them a row uses the host does not know.
constexpr int kValuesFrom = 4096;
constexpr int kValuesTo = 65536 - 128;     // of a CTA: counts of 16 bits
// Of a row's bytes per CTA, where the cluster allows: 256 mixed rows of 151936 take 81 us with 4 CTAs and 98 with 8, 512
// top-p rows of 128256 165 with 4 CTAs, 177 with 2 and 209 with 8.
constexpr size_t kValuesShare = 96 * 1024;
constexpr int kValuesTop = 192;            // the largest top-k that goes by a list (of which kSmall need no sorting)
constexpr uint32_t kNoWay = 0xffffffffu;

__device__ __forceinline__ uint32_t max_u16x2(uint32_t a, uint32_t b)
{
    uint32_t d;
    asm("max.u16x2 %0, %1, %2;" : "=r"(d) : "r"(a), "r"(b));
    return d;
}
__device__ __forceinline__ uint32_t min_u16x2(uint32_t a, uint32_t b)
{
    uint32_t d;
    asm("min.u16x2 %0, %1, %2;" : "=r"(d) : "r"(a), "r"(b));
    return d;
}

__device__ __forceinline__ float step_value(int step)
{
    const uint32_t m = step < kSteps / 2 ? (uint32_t)(kFarMag - 1 - step) : (uint32_t)(kLeastMag + step - kSteps / 2) | 0x8000u;
    return __uint_as_float(m << 16);
}
__device__ __forceinline__ int step_of(uint32_t bits)   // (of a value that has one)
{
    const int m = (int)(bits & 0x7fffu) - kLeastMag;
    return bits & 0x8000u ? kSteps / 2 + m : kSteps / 2 - 1 - m;
}

// The steps of a granule's eight values, in pairs; false: not all of them have one.
__device__ __forceinline__ bool granule_steps(const uint4 &q, uint32_t (&step)[4])
{
    const uint32_t w[4] = {q.x, q.y, q.z, q.w};
    uint32_t big = 0, least = 0xffffffffu;
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        const uint32_t mag = w[k] & 0x7fff7fffu;
        big = max_u16x2(big, mag);
        least = min_u16x2(least, mag);
        uint32_t neg;   // all ones in the halves of negative values
        asm("prmt.b32 %0, %1, 0, 0xbb99;" : "=r"(neg) : "r"(w[k]));
        // with m = mag - kLeastMag (below 2048): 2047 - m, or 2048 + m of a negative value
        step[k] = ((mag + 0x10001u * (0x8000u - kLeastMag)) ^ neg ^ 0x07ff07ffu) & 0x0fff0fffu;
    }
    return (((least + 0x10001u * (0x8000u - kLeastMag)) & ~(big + 0x10001u * (0x8000u - kFarMag))) & 0x80008000u) == 0x80008000u;
}

__device__ __forceinline__ uint32_t granule_elem16(const uint4 &q, int j)
{
    const uint32_t w = j < 4 ? (j < 2 ? q.x : q.y) : (j < 6 ? q.z : q.w);
    return (w >> ((j & 1) * 16)) & 0xffffu;
}
// Which of the eight have no step, as bits.
__device__ __forceinline__ uint32_t odd_ones(const uint4 &q)
{
    const uint32_t w[4] = {q.x, q.y, q.z, q.w};
    uint32_t odd = 0;
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        const uint32_t lo = w[k] & 0x7fffu, hi = (w[k] >> 16) & 0x7fffu;
        odd |= lo - kLeastMag >= kFarMag - kLeastMag ? 1u << (2 * k) : 0u;
        odd |= hi - kLeastMag >= kFarMag - kLeastMag ? 2u << (2 * k) : 0u;
    }
    return odd;
}

struct ValueShared {
    float few[kFewMax];
    unsigned long long part[kSelWarps][kRowMaxCluster], few_mass[kSelWarps], few_kept[kSelWarps];
    uint32_t part_n[kSelWarps], few_n[kSelWarps];
    // written by the CTAs of the row
    unsigned long long mass[kRowMaxCluster][kRowMaxCluster];   // [of the sender's steps][of the CTA]
    unsigned long long listed[kRowMaxCluster];                 // kept ones among the listed
    uint32_t n[kRowMaxCluster], listed_n[kRowMaxCluster], there[kRowMaxCluster], below[kRowMaxCluster],
        counted[kRowMaxCluster];
    uint32_t border, ties, ties_kept;   // the last kept step; its tokens in this CTA, and the kept ones among them
    unsigned long long of_k;            // mass of the k largest
};

// A token's weight from the table (0 where it is cut), for `locate`.
struct TableMass {
    const unsigned long long *table;
    const Scale &s;
    const float2 *tab;
    uint32_t kminp;
    bool listed;             // the ones without a step are kept, from kminp on
    int tie, idx;            // a step of which only the tokens up to an index are kept (-1: none), its weight 0 in the table
    unsigned long long tie_w;

    __device__ __forceinline__ unsigned long long elem(float x, uint32_t k, int i) const
    {
        const uint32_t bits = __float_as_uint(x) >> 16;
        const int mag = (int)(bits & 0x7fffu);
        if (mag >= kFarMag) return 0ull;
        if (mag < kLeastMag) return listed && k >= kminp ? weight(x, s, tab) : 0ull;
        const int step = step_of(bits);
        return step == tie ? (i <= idx ? tie_w : 0ull) : table[step];
    }
    // i0: the index of the first of them
    __device__ __forceinline__ unsigned long long granule(const uint4 &q, int i0) const
    {
        uint32_t step[4], odd = granule_steps(q, step) ? 0u : odd_ones(q);
        unsigned long long a = 0, b = 0;
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            a += table[step[k] & 0xffffu];
            b += table[step[k] >> 16];
        }
        if (tie >= 0) {
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                if ((int)(step[k] & 0xffffu) == tie && !(odd & (1u << (2 * k))) && i0 + 2 * k <= idx) a += tie_w;
                if ((int)(step[k] >> 16) == tie && !(odd & (2u << (2 * k))) && i0 + 2 * k + 1 <= idx) b += tie_w;
            }
        }
        for (; odd != 0; odd &= odd - 1u) {
            const int j = __ffs(odd) - 1;
            const uint32_t w = step[j >> 1], x = granule_elem16(q, j) << 16;
            a -= table[j & 1 ? w >> 16 : w & 0xffffu];
            a += elem(__uint_as_float(x), key_of(__uint_as_float(x)), i0 + j);   // (-inf and NaN weigh nothing)
        }
        return a + b;
    }
};

// The tokens of one value.
struct TieCount {
    uint32_t bits;   // of it
    __device__ __forceinline__ unsigned long long elem(float x, uint32_t, int) const
    {
        return __float_as_uint(x) >> 16 == bits;
    }
    __device__ __forceinline__ unsigned long long granule(const uint4 &q, int) const
    {
        const uint32_t w[4] = {q.x, q.y, q.z, q.w};
        uint32_t n = 0;
#pragma unroll
        for (int k = 0; k < 4; ++k) n += ((w[k] & 0xffffu) == bits) + (w[k] >> 16 == bits);
        return n;
    }
};

// The first token of this CTA's, in order, at which the running sum of f passes `target` (below their sum): found(idx,
// key) by one thread.  Sums of kSegGranules granules each, then the elements of the ones that hold it.  seg: kSegs words.
constexpr int kSegGranules = 128, kSegs = 64;
static_assert(kSegs % kSelWarps == 0 && kValuesTo / 8 + kSelWarps <= kSegs * kSegGranules && kSegs <= kSelThreads,
              "a thread per sum");
static_assert(kSegGranules * 8 == kSelThreads * 4, "four elements of them per thread");
template <typename S, typename Found>
__device__ __forceinline__ void find_in_share(const Ctx<false> &c, unsigned long long target, const S &f,
                                              unsigned long long *seg, Found found)
{
    constexpr int U = kSegGranules / 32;
    Shared *sh = c.sh;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int wper = (c.n + kSelWarps - 1) / kSelWarps, each = (wper + kSegGranules - 1) / kSegGranules;   // sums of a warp
    for (int i = 0; i < each; ++i) {
        uint4 x[U];
#pragma unroll
        for (int k = 0; k < U; ++k) {
            const int v = c.wb + kSegGranules * i + 32 * k + lane;
            if (v < c.we) x[k] = load_granule<false>(c.r, c.gb + v);
        }
        unsigned long long a = 0;
#pragma unroll
        for (int k = 0; k < U; ++k) {
            const int v = c.wb + kSegGranules * i + 32 * k + lane;
            if (v < c.we) a += f.granule(x[k], c.r.first(c.gb + v));
        }
        a = warp_sum_u64(a);
        if (lane == 0) seg[warp * each + i] = a;
    }
    __syncthreads();
    unsigned long long mine = tid < kSelWarps * each ? seg[tid] : 0ull, total;
    unsigned long long run = block_scan_u64(mine, sh, &total);
    if (target >= run && target - run < mine) {   // (one thread)
        sh->border = tid;
        sh->mass[0] = run;
    }
    __syncthreads();
    const int at = sh->border, w = at / each, v = w * wper + kSegGranules * (at - w * each) + (tid >> 1);
    target -= sh->mass[0];
    const int j0 = (tid & 1) * 4, i0 = c.r.first(c.gb + v) + j0;
    const bool on = v < min(c.n, (w + 1) * wper);
    const uint4 q = on ? load_granule<false>(c.r, c.gb + v) : make_uint4(0xff80ff80u, 0xff80ff80u, 0xff80ff80u, 0xff80ff80u);
    unsigned long long m[4];
    mine = 0;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const float x = __uint_as_float(granule_elem16(q, j0 + j) << 16);
        m[j] = x > -INFINITY ? f.elem(x, key_of(x), i0 + j) : 0ull;   // (a NaN is not above it)
        mine += m[j];
    }
    run = block_scan_u64(mine, sh, &total);
    if (target >= run && target - run < mine) {   // (one thread)
        int j = 0;
        while (j < 3 && target - run >= m[j]) run += m[j++];
        found(i0 + j, key_of(__uint_as_float(granule_elem16(q, j0 + j) << 16)));
    }
}

__device__ __noinline__ void sample_row_again(Ctx<false> c, const SampleParams &p, int row, const Settings &set,
                                              unsigned long long *list, const float2 *tab)
{
    start_row(c, nullptr);
    sample_row<false>(c, p, row, set, static_cast<uint4 *>(nullptr), list, tab);
}

__global__ void __launch_bounds__(kSelThreads, kValuesPerSm) sample_values_kernel(const SampleParams p)
{
    extern __shared__ __align__(16) uint4 smem[];
    __shared__ Shared sh;
    __shared__ ValueShared sv;
    __shared__ float2 tab[1024];
    const int row = (int)(blockIdx.x >> (31 - __clz(p.cluster))), tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    Ctx<false> c{Row<false>(p.z, row, p.ld, p.V)};
    set_ctx(c, nullptr, 0, p.cluster, &sh);
    const int C = c.C;
    if (C > 1) cluster_arrive();
    const Settings set(p, row);
    if (set.bad) {
        if (c.rank == 0 && tid == 0) put_bad(p, row);
        if (C > 1) cluster_wait();
        return;   // (every CTA of the row)
    }
    unsigned long long *list = reinterpret_cast<unsigned long long *>(smem);
    if (!set.greedy)
        for (int i = tid; i < 1024; i += kSelThreads) tab[i] = kExp2.v[i];
    bool met = C == 1;   // every CTA of the row runs
    if (!set.greedy && (set.k > 0 ? set.k <= kValuesTop : set.min_p > 0.f && !set.nucleus)) {
        // few tokens are kept, as a rule: a list of the k largest, or of the ones that min-p keeps
        uint32_t *scratch = reinterpret_cast<uint32_t *>(list);
        float *gm = reinterpret_cast<float *>(list + kListCap);
        int *hits = reinterpret_cast<int *>(gm + kMaxGroups * kSelThreads);
        for (int i = tid; i < kBoundBins; i += kSelThreads) scratch[i] = 0u;
        float hi = -INFINITY, lo = INFINITY;
        const int mine = group_maxima(c, p.groups, gm, &hi, &lo);
        uint32_t top;
        uint32_t bound = group_bound(&sh, scratch, (set.k + C - 1) >> (31 - __clz(C)), hi, lo, &top, [&](auto f) {
            for (int g = 0; g < mine; ++g) f(gm[g * kSelThreads + tid]);
        });
        if (C > 1) {
            cluster_wait();
            met = true;
            if (tid < C) {
                st_peer_u32(peer_addr(&sh.kmax[c.rank], tid), top);
                st_peer_u32(peer_addr(&sh.bound[c.rank], tid), bound);
            }
            cluster_sync_all();
            for (int k = 0; k < C; ++k) {
                top = max(top, sh.kmax[k]);
                bound = min(bound, sh.bound[k]);
            }
        }
        if (top <= kKeyNone) {   // nothing can be drawn
            if (c.rank == 0 && tid == 0) put_sample(p, row, -1, -INFINITY, 0);
            return;
        }
        Scale s;
        set_scale(s, key_float(top), set.T, p.V);
        const uint32_t kminp = least_key(set, s, &sh);
        if (set.k == 0) bound = max(kminp, kKeyNone + 1);
        collect_groups(c, p.groups, gm, mine, hits, key_float(bound), list, kListCap);
        bool ok;
        const int n = push_list(c, list, &ok);
        if (ok && (set.k > 0 || n <= kSmall)) {   // (the same in every CTA of the row)
            if (c.rank != 0) return;   // (nobody reads this CTA's memory any more)
            draw_list(p, row, set, s, list, n, kminp, tab, &sh);
            return;
        }
        __syncthreads();
    }
    uint32_t *count = reinterpret_cast<uint32_t *>(smem), *got = count + kBins;
    unsigned long long *table = list, *seg = table + kSteps;   // (after the counts)
    if (!set.greedy)
        for (int i = tid; i < kBins / 4; i += kSelThreads) smem[i] = make_uint4(0, 0, 0, 0);
    if (tid == 0) {
        sh.nlist = 0;
        sv.border = kNoWay;
        sv.of_k = 0;
    }
    __syncthreads();

    // the row
    uint32_t most = 0xff80ff80u, below = 0;
    bool far = false;
    {
        constexpr int U = 4;
        const auto add = [&](uint32_t step) { atomicAdd(count + (step >> 1), 1u << ((step & 1u) << 4)); };
        for (int v0 = tid; v0 < c.n; v0 += U * kSelThreads) {
            uint4 x[U];
#pragma unroll
            for (int k = 0; k < U; ++k)
                x[k] = v0 + k * kSelThreads < c.n ? load_granule<false>(c.r, c.gb + v0 + k * kSelThreads)
                                                  : make_uint4(0xff80ff80u, 0xff80ff80u, 0xff80ff80u, 0xff80ff80u);
#pragma unroll
            for (int k = 0; k < U; ++k) {
                const uint4 q = x[k];
                most = bf16x2_max(most, bf16x2_max(bf16x2_max(q.x, q.y), bf16x2_max(q.z, q.w)));
                if (set.greedy || v0 + k * kSelThreads >= c.n) continue;
                uint32_t step[4];
                if (granule_steps(q, step)) {
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        add(step[j] & 0xffffu);
                        add(step[j] >> 16);
                    }
                } else {
                    uint32_t odd = odd_ones(q);
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        if (!(odd & (1u << (2 * j)))) add(step[j] & 0xffffu);
                        if (!(odd & (2u << (2 * j)))) add(step[j] >> 16);
                    }
                    for (; odd != 0; odd &= odd - 1u) {
                        const uint32_t b = granule_elem16(q, __ffs(odd) - 1), mag = b & 0x7fffu;
                        if (mag > 0x7f80u || b == 0xff80u) continue;   // NaN, -inf
                        if (mag >= kFarMag) {
                            if (b & 0x8000u) ++below;
                            else far = true;
                        } else {
                            const uint32_t at = atomicAdd(&sh.nlist, 1u);
                            if (at < kFewMax) sv.few[at] = __uint_as_float(b << 16);
                        }
                    }
                }
            }
        }
    }
    {
        const float m = fmaxf(fmaxf(bf16_lo(most), bf16_hi(most)), -INFINITY);
        const uint32_t key = __reduce_max_sync(0xffffffffu, key_of(m));
        below = __reduce_add_sync(0xffffffffu, below);
        if (lane == 0) {
            sh.ktop[warp] = key;
            sh.part[warp] = (int)below;
        }
    }
    far = __syncthreads_or(far);
    const int nfew = (int)sh.nlist;
    uint32_t kmax = __reduce_max_sync(0xffffffffu, sh.ktop[lane & (kSelWarps - 1)]);
    if (!met) cluster_wait();
    if (tid < C) {
        st_peer_u32(peer_addr(&sh.kmax[c.rank], tid), kmax);
        st_peer_u32(peer_addr(&sv.there[c.rank], tid), far ? kNoWay : (uint32_t)nfew);
        uint32_t n = 0;
        for (int w = 0; w < kSelWarps; ++w) n += (uint32_t)sh.part[w];
        st_peer_u32(peer_addr(&sv.below[c.rank], tid), n);
    }
    if (!set.greedy) {
        got = exchange_counts(c, count, got);
        if (C == 1) __syncthreads();
    } else if (C > 1) {
        cluster_sync_all();
    } else {
        __syncthreads();
    }
    unsigned first = 0;   // the first CTA that has the largest logit
    kmax = sh.kmax[0];
    for (int k = 1; k < C; ++k)
        if (sh.kmax[k] > kmax) {
            kmax = sh.kmax[k];
            first = k;
        }
    if (kmax <= kKeyNone) {   // nothing can be drawn
        if (c.rank == 0 && tid == 0) put_sample(p, row, -1, -INFINITY, 0);
        return;
    }
    if (set.greedy) {
        if (c.rank != first) return;
        Ctx<false> one = c;
        one.C = 1;
        one.rank = 0;
        const int id = lowest_at(one, kmax);
        if (tid == 0) put_sample(p, row, id, 0.f, 1);
        return;
    }
    Scale s;
    set_scale(s, key_float(kmax), set.T, p.V);
    uint32_t all_below = 0, all_few = 0;
    bool way = !s.hard;
    for (int k = 0; k < C; ++k) {
        way = way && sv.there[k] <= (uint32_t)kFewMax;
        all_few += sv.there[k];
        all_below += sv.below[k];
    }
    // (what lies below the steps has no weight: 45 octaves below the top and more)
    way = way && (all_below == 0 || s.top + 64.f >= 31.4f * set.T);
    const uint32_t kminp = least_key(set, s, &sh);
    int last = kSteps - 1;   // min-p: the last step that is kept
    if (kminp > 0) {
        const uint32_t b = __float_as_uint(key_float(kminp)), up = b & 0x80000000u ? b >> 16 : (b + 0xffffu) >> 16;
        const int mag = (int)(up & 0x7fffu);   // (up: the least bf16 value from there on)
        if (mag < kLeastMag) last = kSteps / 2 - 1;
        else if (mag < kFarMag) last = step_of(up);
        else way = way && all_below == 0;   // (it is -2^6 or below: larger than the top it cannot be)
    }
    if (!way) {   // (the same in every CTA of the row)
        __syncthreads();
        sample_row_again(c, p, row, set, reinterpret_cast<unsigned long long *>(smem), tab);
        return;
    }

    // the listed ones' masses: of all, and of what min-p keeps
    if (32 * warp < nfew) {
        const bool on = tid < nfew;
        const float x = on ? sv.few[tid] : 0.f;
        const unsigned long long w = on ? weight(x, s, tab) : 0ull;
        const bool in = on && key_of(x) >= kminp;
        const unsigned long long a = warp_sum_u64(w), b = warp_sum_u64(in ? w : 0ull);
        const uint32_t n = (uint32_t)__popc(__ballot_sync(0xffffffffu, in));
        if (lane == 0) {
            sv.few_mass[warp] = a;
            sv.few_kept[warp] = b;
            sv.few_n[warp] = n;
        }
    }
    // a run of steps per CTA, of it a run per thread: the masses of the CTAs' tokens there (up to `last`, the rest apart)
    const int nw = kBins / C, per = (nw + kSelThreads - 1) / kSelThreads;   // words
    const int w0 = min(nw, tid * per), w1 = min(nw, w0 + per);
    const int base = (int)c.rank * nw, b0 = 2 * (base + w0), b1 = 2 * (base + w1);
    const auto counted = [&](int k, int b) { return (got[k * nw + (b >> 1) - base] >> ((b & 1) << 4)) & 0xffffu; };
    const auto in_step = [&](int b) {
        uint32_t t = 0;
        for (int k = 0; k < C; ++k) t += counted(k, b);
        return t;
    };
    unsigned long long acc[kRowMaxCluster], mine = 0;
    uint32_t n = 0, tokens = 0;
#pragma unroll
    for (int k = 0; k < kRowMaxCluster; ++k) acc[k] = 0;
    for (int w = w0; w < w1; ++w) {
        const int b = 2 * (base + w);
        uint32_t any = 0;
        for (int k = 0; k < C; ++k) any |= got[k * nw + w];
        if (any == 0) continue;
        const Weights2 q = weights2(pack2(step_value(b), step_value(b + 1)), s, tab);
        // (steps above the top are empty)
        const unsigned long long wa = q.in[0] ? whole_weight(q.i1[0], q.i2[0], s) : 0ull;
        const unsigned long long wb = q.in[1] ? whole_weight(q.i1[1], q.i2[1], s) : 0ull;
        const bool ina = b <= last, inb = b + 1 <= last;
#pragma unroll
        for (int k = 0; k < kRowMaxCluster; ++k) {
            if (k >= C) break;
            const uint32_t x = got[k * nw + w], na = x & 0xffffu, nb = x >> 16;
            const unsigned long long ma = na * wa, mb = nb * wb;
            tokens += na + nb;
            n += (ina ? na : 0u) + (inb ? nb : 0u);
            acc[k] += (ina ? ma : 0ull) + (inb ? mb : 0ull);
            mine += ma + mb;
        }
    }
    const auto drop = [&]() {
        n = 0;
#pragma unroll
        for (int k = 0; k < kRowMaxCluster; ++k) acc[k] = 0;
    };
    bool cut = set.nucleus;
    uint32_t all_tokens = 0;
    if (set.nucleus || set.k > 0) {
        unsigned long long total, total_n = 0;
        unsigned long long run = block_scan_u64(mine, &sh, &total);
        uint32_t run_n = 0;
        if (set.k > 0) run_n = (uint32_t)block_scan_u64(tokens, &sh, &total_n);
        unsigned long long few = 0;
        for (int w = 0; 32 * w < nfew; ++w) few += sv.few_mass[w];
        if (tid < C) st_peer_u32(peer_addr(&sv.counted[c.rank], tid), (uint32_t)total_n);
        const unsigned long long *slot = cluster_gather(c, total, few);
        few = slot_sum(slot + kRowMaxCluster, C);
        unsigned long long Z = slot_sum(slot, C) + few;
        for (unsigned k = 0; k < c.rank; ++k) {
            run += slot[k];
            run_n += sv.counted[k];
        }
        if (b0 >= kSteps / 2) {   // (the listed ones are between the positive and the negative steps)
            run += few;
            run_n += all_few;
        }
        uint32_t most_n = 0xffffffffu;
        if (set.k > 0) {
            all_tokens = all_few;
            for (int k = 0; k < C; ++k) all_tokens += sv.counted[k];
            if ((uint32_t)set.k < all_tokens) {
                most_n = (uint32_t)set.k;
                cut = true;
            }
        }
        // the thread's steps in order, while `more` says so: more(step, tokens before, mass before, tokens, weight)
        const auto walk = [&](auto more) {
            unsigned long long m = run;
            uint32_t before = run_n;
            for (int b = b0; b < b1; ++b) {
                const uint32_t t = in_step(b);
                if (t == 0) continue;
                const unsigned long long w = weight(step_value(b), s, tab);
                if (!more(b, before, m, t, w)) return;
                m += t * w;
                before += t;
            }
        };
        unsigned long long target = ~0ull;
        if (set.nucleus) {
            if (most_n != 0xffffffffu) {
                if (run_n < most_n && run_n + tokens >= most_n)   // (one thread)
                    walk([&](int, uint32_t before, unsigned long long m, uint32_t t, unsigned long long w) {
                        if (before + t < most_n) return true;
                        m += (most_n - before) * w;
                        for (int k = 0; k < C; ++k) st_peer_u64(peer_addr(&sv.of_k, k), m);
                        return false;
                    });
                if (C > 1) cluster_sync_all();
                else __syncthreads();
                Z = sv.of_k;   // (0: the k-th largest is a listed one)
            }
            target = share_ceil(set.top_p, Z);
        }
        if (run >= target || run_n >= most_n) {
            drop();
        } else if (cut && (run + mine >= target || (most_n != 0xffffffffu && run_n + tokens >= most_n))) {   // (one thread)
            drop();
            walk([&](int b, uint32_t before, unsigned long long m, uint32_t t, unsigned long long w) {
                uint32_t left = min(t, most_n - before);
                bool border = most_n != 0xffffffffu && before + t >= most_n;
                if (target - m <= left * w) {
                    border = true;
                    left = (uint32_t)((target - m + w - 1ull) / w);
                }
                if (b <= last) n += left;
                for (int k = 0; k < C; ++k) {
                    const uint32_t there = counted(k, b), kept = min(there, left);
                    left -= kept;
#pragma unroll
                    for (int q = 0; q < kRowMaxCluster; ++q)
                        if (q == k && b <= last) acc[q] += kept * w;
                    if (border) {
                        st_peer_u32(peer_addr(&sv.border, k), (uint32_t)b);
                        st_peer_u32(peer_addr(&sv.ties, k), there);
                        st_peer_u32(peer_addr(&sv.ties_kept, k), kept);
                    }
                }
                return !border;
            });
        }
    }
#pragma unroll
    for (int k = 0; k < kRowMaxCluster; ++k) {
        if (k >= C) break;
        const unsigned long long a = warp_sum_u64(acc[k]);
        if (lane == 0) sv.part[warp][k] = a;
    }
    n = __reduce_add_sync(0xffffffffu, n);
    if (lane == 0) sv.part_n[warp] = n;
    __syncthreads();
    if (tid < C * C) {
        const int k = tid & (C - 1), to = tid >> (31 - __clz(C));
        unsigned long long a = 0;
        for (int w = 0; w < kSelWarps; ++w) a += sv.part[w][k];
        st_peer_u64(peer_addr(&sv.mass[c.rank][k], to), a);
    }
    if (tid < C) {
        unsigned long long kept = 0;
        uint32_t kept_n = 0;
        n = 0;
        for (int w = 0; w < kSelWarps; ++w) n += sv.part_n[w];
        for (int w = 0; 32 * w < nfew; ++w) {
            kept += sv.few_kept[w];
            kept_n += sv.few_n[w];
        }
        st_peer_u32(peer_addr(&sv.n[c.rank], tid), n);
        st_peer_u32(peer_addr(&sv.listed_n[c.rank], tid), kept_n);
        st_peer_u64(peer_addr(&sv.listed[c.rank], tid), kept);
    }
    if (C > 1) cluster_sync_all();
    else __syncthreads();
    const int border = (int)sv.border;
    if (cut && border < 0) {   // (the same in every CTA of the row)
        sample_row_again(c, p, row, set, reinterpret_cast<unsigned long long *>(smem), tab);
        return;
    }
    const bool listed = !cut || border >= kSteps / 2;
    unsigned long long total = 0, before = 0, here = 0;
    uint32_t kept_n = cut || kminp > 0 ? 0u : all_below;
    for (int k = 0; k < C; ++k) {
        unsigned long long a = listed ? sv.listed[k] : 0ull;
        for (int q = 0; q < C; ++q) a += sv.mass[q][k];
        if (k < (int)c.rank) before += a;
        if (k == (int)c.rank) here = a;
        total += a;
        kept_n += sv.n[k] + (listed ? sv.listed_n[k] : 0u);
    }
    if (set.k > 0) kept_n = min(kept_n, (uint32_t)set.k);
    const unsigned long long target = share_floor(set.u, total);
    if (target < before || target - before >= here) return;   // another CTA has it

    // this CTA alone from here on
    Ctx<false> one = c;
    one.C = 1;
    one.rank = 0;
    TableMass mass{table, s, tab, kminp, listed, -1, INT_MIN, 0ull};
    if (cut && border <= last && sv.ties_kept < sv.ties) {
        mass.tie = border;
        mass.tie_w = weight(step_value(border), s, tab);
        if (sv.ties_kept > 0) {
            find_in_share(one, (unsigned long long)sv.ties_kept - 1ull, TieCount{__float_as_uint(step_value(border)) >> 16},
                          seg, [&](int i, uint32_t) { sh.found_idx = i; });
            __syncthreads();
            mass.idx = sh.found_idx;
        }
    }
    const int end = min(last, cut ? border : kSteps - 1);
    const int begin = fabsf(s.top) >= step_value(kSteps / 2 - 1) ? step_of(__float_as_uint(s.top) >> 16) : kSteps / 2 - 1;
    for (int b = 2 * tid; b < kSteps; b += 2 * kSelThreads) {
        ulonglong2 w = make_ulonglong2(0ull, 0ull);
        if (b <= end && b + 1 >= begin) {
            const Weights2 q = weights2(pack2(step_value(b), step_value(b + 1)), s, tab);
            if (q.in[0] && b != mass.tie) w.x = whole_weight(q.i1[0], q.i2[0], s);
            if (q.in[1] && b + 1 <= end && b + 1 != mass.tie) w.y = whole_weight(q.i1[1], q.i2[1], s);
        }
        *reinterpret_cast<ulonglong2 *>(table + b) = w;
    }
    __syncthreads();
    find_in_share(one, target - before, mass, seg, [&](int id, uint32_t key) {
        put_sample(p, row, id, log_share(key_float(key), set.T, s, total), (long long)kept_n);
    });
}

constexpr size_t kValuesSmem = std::max<size_t>((kSteps + kSegs) * 8, kListCap * 12 + kMaxGroups * kSelThreads * 4);

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
    const int64_t bytes = (int64_t)V * RowElem<F32>::kBytes;
    p.cluster = logits_cluster(B, bytes, 0, kValuesShare);
    if (!F32 && V >= kValuesFrom && V / p.cluster < kValuesTo) {
        p.groups = plan_groups(bytes, p.cluster, kMaxGroups);
        const cudaError_t e = launch_clusters<sample_values_kernel>((int64_t)B * p.cluster, kSelThreads, kValuesSmem, kValuesSmem,
                                                                    p.cluster, static_cast<cudaStream_t>(stream), p);
        return e == cudaSuccess ? SATS_OK : cuda_fail(e, "sampling kernel launch");
    }
    p.cluster = logits_cluster(B, bytes, 0, kShare);
    const size_t share = (size_t)((bytes + 32 + p.cluster - 1) / p.cluster) + 32;
    p.cached = (int)((share < kMaxCache ? share : kMaxCache) / 16);
    const int granules = (int)std::min<int64_t>((bytes + 15) / 16 / p.cluster, 1 << 20);
    const bool few = top_k && few_groups(std::min(granules, kSelThreads) * groups_of(F32), granules * RowElem<F32>::kPer,
                                         std::min(V, kMaxTop) / p.cluster);
    const int64_t ctas = (int64_t)B * p.cluster;
    const size_t smem = (size_t)p.cached * 16 + kListCap * 8;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    const cudaError_t e = few ? launch_clusters<sample_kernel<F32, true>>(ctas, kSelThreads, smem, kMaxSmem, p.cluster, st, p)
                              : launch_clusters<sample_kernel<F32, false>>(ctas, kSelThreads, smem, kMaxSmem, p.cluster, st, p);
    return e == cudaSuccess ? SATS_OK : cuda_fail(e, "sampling kernel launch");
}

}  // namespace
}  // namespace sats

extern "C" {

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
