// sample.cu -- drawing a token from each row of logits (sats_sample).
//
// The row's share of a CTA is brought to shared memory once; all passes after that run there.
//
// Drawing needs sums over up to V tokens that decide next to borders as close as the smallest token's probability.
// A token's weight is therefore a whole number, w = 2^F exp((z - max) / T) to about 35 bits relative (never less
// than 2^-F absolute), computed in pairs of floats; sums of whole numbers do not depend on their order, and every
// decision (the nucleus, the drawn token) is the same in whichever grouping it is found.
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
constexpr size_t kShare = 64 * 1024;   // of a row's bytes per CTA, where the cluster allows
constexpr size_t kMaxCache = 184 * 1024;
constexpr size_t kMaxSmem = kMaxCache + (size_t)kListCap * 8;
static_assert(kMaxSmem + 11 * 1024 <= kSmemPerCta, "with the kernel's static part");

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
template <bool F32>
__device__ void load_row(Ctx<F32> &c, uint4 *cache, int want, uint32_t *scratch, uint32_t *kmax, uint32_t *bound)
{
    constexpr int NG = F32 ? 4 : 8;   // groups of a thread
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
    uint32_t top;
    uint32_t low = group_bound(sh, scratch, (want + c.C - 1) >> (31 - __clz(c.C)), hi, lo, &top, [&](auto f) {
#pragma unroll
        for (int k = 0; k < NG; ++k) f(g[k]);
    });
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
// steps, and a list of the ones within, which settles the border; that it lies there at all is checked.
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
    // a run of steps per CTA: its counts in all CTAs
    const int nb = kBins / C;
    if (C > 1) {
        for (int i = tid; i < kBins / 4; i += kSelThreads) {
            const uint4 q = reinterpret_cast<const uint4 *>(count)[i];
            const int b = 4 * i;
            st_peer_v4(peer_addr(got + c.rank * nb + b % nb, b / nb), __uint_as_float(q.x), __uint_as_float(q.y),
                       __uint_as_float(q.z), __uint_as_float(q.w));
        }
        cluster_sync_all();
    } else {
        got = count;
    }
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
    unsigned long long Zs = slot_sum(slot, C);
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
    int n = 0, off = 0;   // entries; of the CTAs before this one
    bool fits = A < target;
    for (int k = 0; k < C; ++k) {
        fits = fits && sh->cnt[k] <= (uint32_t)seg;
        if (k < (int)c.rank) off += (int)sh->cnt[k];
        n += (int)sh->cnt[k];
    }
    if (!fits || n == 0) return false;
    const unsigned long long want = target - A;
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
    if (cut.idx < 0 || n > kSmall) return cut.idx >= 0;
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

template <bool F32>
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
    const float T = p.temperature ? p.temperature[row] : 1.f;
    const float top_p = p.top_p ? p.top_p[row] : 1.f, min_p = p.min_p ? p.min_p[row] : 0.f;
    const float u = p.u[row];
    int k = p.top_k ? p.top_k[row] : 0;
    if (!(T >= 0.f) || T == INFINITY || top_p != top_p || !(min_p <= 1.f) || !(u >= 0.f && u < 1.f)) {
        if (c.rank == 0 && tid == 0) {
            put_sample(p, row, -1, __int_as_float(0x7fffffff), 0);
            if (p.status) atomicOr(p.status, kStatusBadToken);
        }
        cp_async_wait<0>();
        if (c.C > 1) cluster_wait();
        return;   // (every CTA of the row)
    }
    if (k < 0 || k >= p.V) k = 0;
    const bool greedy = T == 0.f || k == 1 || top_p <= 0.f;
    const bool nucleus = top_p < 1.f;
    const int want = !greedy && k > 0 && k <= kMaxTop ? k : 0;   // what the list serves
    if (!greedy)
        for (int i = tid; i < 1024; i += kSelThreads) tab[i] = kExp2.v[i];
    uint32_t kmax, bound;
    load_row(c, smem, want, reinterpret_cast<uint32_t *>(list), &kmax, &bound);
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

    if (want > 0) {
        bool ok;
        const int n = gather_list(c, list, bound, Cut{kKeyNone, INT_MIN}, &ok);
        if (ok) {   // (the same in every CTA of the row)
            if (c.rank != 0) return;   // (nobody reads this CTA's memory any more)
            if (n <= kSmall) {
                const Small e(list, n);
                const unsigned long long w = e.on ? weight(key_float(e.key()), s, tab) : 0ull;
                e.put_weight(list, w);
                __syncthreads();
                int at;
                unsigned long long above;
                e.larger(list, n, &at, &above);
                bool kept = e.on && at < k && e.key() >= kminp;
                if (nucleus) {
                    const unsigned long long Z = block_sum_u64(e.on && e.part == 0 && at < k ? w : 0ull, &sh);
                    kept = kept && above < share_ceil(top_p, Z);
                }
                const int m = __syncthreads_count(kept && e.part == 0);
                e.put_weight(list, kept ? w : 0ull);
                const unsigned long long total = block_sum_u64(kept && e.part == 0 ? w : 0ull, &sh);
                const unsigned long long before = e.earlier(list, n), target = share_floor(u, total);
                if (kept && e.part == 0 && target >= before && target - before < w)   // one entry
                    put_sample(p, row, e.idx(), log_share(key_float(e.key()), T, s, total), m);
                return;
            }
            draw_from_list(p, row, list, n, k, nucleus ? top_p : 1.f, kminp, u, T, s, tab, &sh);
            return;
        }
    }

    // over the whole row: the cuts one after the other, then the kept mass and the token in it
    Cut cut{kKeyNone, INT_MIN};
    if (k > 0) cut = cut_count(c, kmax, k);
    bool sums = false;
    if (nucleus) {
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
        unsigned long long mine = cut.key > kKeyNone ? kept.over_row<true>(c, n) : kept.over_row<false>(c, n);
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
    p.cluster = logits_cluster(B, bytes, 0, kShare);
    const size_t share = (size_t)((bytes + 32 + p.cluster - 1) / p.cluster) + 32;
    p.cached = (int)((share < kMaxCache ? share : kMaxCache) / 16);
    const cudaError_t e = launch_clusters<sample_kernel<F32>>((int64_t)B * p.cluster, kSelThreads,
                                                              (size_t)p.cached * 16 + kListCap * 8, kMaxSmem, p.cluster,
                                                              static_cast<cudaStream_t>(stream), p);
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
