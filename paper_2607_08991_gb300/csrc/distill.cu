// distill.cu -- distillation of a row of logits from a teacher's top logits, mixed with the next-token cross
// entropy, forward and backward (sats_distill_loss, sats_distill_grad, sats_distill_loss_grad).
//
// For a row z of V logits, teacher entries (i_k, g_k), a label y, a temperature tau and a share alpha:
//     q   = softmax over the entries of g / tau,   p^tau = softmax(z / tau),   p = softmax(z)
//     KD  = tau^2 sum_k q_k (log q_k - log p^tau_{i_k}),     CE = log sum_j exp z_j - z_y
//     loss = alpha KD + (1 - alpha) CE
//     d loss / d z_j = alpha tau (p^tau_j - sum_{k: i_k = j} q_k) + (1 - alpha) (p_j - [j = y])
// Everything is kept in base 2: with c = log2(e) / tau and m the row's maximum, w_j = 2^((z_j - m) c) and S = sum w_j
// give p^tau_j = w_j / S and log2 p^tau_j = (z_j - m) c - log2 S.  The difference comes first: it is exact where w_j
// is large, and a row of the type's lowest values overflows nowhere.  While a thread reads, m is its own running
// maximum (one pass); the threads' sums are joined over the row's CTAs at the end.
#include <climits>
#include <cmath>

#include "internal.h"
#include "rows.cuh"

namespace sats {
namespace {

constexpr float kLog2e = 1.44269504088896340736f, kLn2 = 0.69314718055994530942f;
constexpr int kMaxEntries = 1024;             // teacher entries of a row
constexpr float kMinTau = 0x1p-10f;           // to its inverse: a log-sum-exp at tau keeps some of its bits
constexpr size_t kMaxCache = 180 * 1024;      // of a row's share in shared memory
constexpr size_t kMaxSmem = kSmemPerCta - 2 * 1024;   // dynamic: a row's share, two tables of entries
// Threads, CTAs to an SM and the share of a row that a CTA of the one-pass kernel has on chip (where the cluster allows),
// 4096 rows of 128256 bf16 logits before its clusters stayed for many rows (us): 256 x 3, 72 KB 450; 256 x 4, 72 KB 455;
// 256 x 4, 40 KB 563; 512 x 2, 72 KB 581; 128 x 8, 40 KB 460.  The backward pass with 256 x 4 takes 197 us where 512 x 2
// took 273 (1000 rows of 151936 fp32 logits), the loss 352 where it took 371 (8192 rows of 151936 bf16 ones).  Powers of
// two: sums over warps halve their number.
constexpr size_t kStepShare = 72 * 1024;
constexpr int kLossThreads = 256, kGradThreads = 256, kStepThreads = 256, kStepPerSm = 3;

struct DistillParams {
    const void *z;
    int64_t ldz;
    int T, V;
    const int32_t *idx;
    const float *val;
    int K;
    const int32_t *labels;
    float tau, alpha;
    float *loss, *lse;        // lse: [T][2], of z / tau and of z
    const float *lse_in;
    const float *g;
    void *d;
    int64_t ldd;
    int32_t *status;
    int cluster;              // CTAs of a row
    int cached;               // granules of a CTA's share that stay in shared memory
    int slots;                // of the table of entries' indices (a power of two)
    int withheld;             // a row whose sums the second CTA does not send to the first (the self-test's; -1)
};

// Sums of 2^((z - m) c) for one or two c, m the largest z so far.
template <int NT>
struct RunSum {
    float m;
    float s[NT];
};

// What is subtracted from logits whose maximum is m (-inf - (-inf) would be NaN).
__device__ __forceinline__ float offset_of(float m) { return m == -INFINITY ? 0.f : m; }

// Adds N granules' elements.
template <bool F32, int NT, int N>
__device__ __forceinline__ void run_add(RunSum<NT> &r, const uint4 (&v)[N], const float (&c)[NT])
{
    constexpr int P = RowElem<F32>::kPer / 2;
    float gm = granule_max<F32>(v[0]);
#pragma unroll
    for (int k = 1; k < N; ++k) gm = fmaxf(gm, granule_max<F32>(v[k]));
    if (gm > r.m) {
#pragma unroll
        for (int t = 0; t < NT; ++t) r.s[t] *= ex2_approx((r.m - gm) * c[t]);   // (from -inf: a factor of 0)
        r.m = gm;
    }
    const float off = -offset_of(r.m);
    const f32x2 off2 = pack2(off, off);
#pragma unroll
    for (int k = 0; k < N; ++k) {
        f32x2 x[P];
        granule_pairs<F32>(v[k], x);
#pragma unroll
        for (int j = 0; j < P; ++j) x[j] = fadd2(x[j], off2);
#pragma unroll
        for (int t = 0; t < NT; ++t) {
            const f32x2 c2 = pack2(c[t], c[t]);
            f32x2 e[P];
#pragma unroll
            for (int j = 0; j < P; ++j) {
                const float2 y = unpack2(fmul2(x[j], c2));
                e[j] = pack2(ex2_approx(y.x), ex2_approx(y.y));
            }
#pragma unroll
            for (int w = P / 2; w > 0; w >>= 1)
#pragma unroll
                for (int j = 0; j < w; ++j) e[j] = fadd2(e[j], e[j + w]);
            r.s[t] += hsum2(e[0]);
        }
    }
}

// The largest of the warp's values (no NaN among them): as whole numbers that order like them.
__device__ __forceinline__ float warp_max(float v)
{
    const int b = __float_as_int(v);
    const int m = __reduce_max_sync(0xffffffffu, b ^ ((b >> 31) & 0x7fffffff));
    return __int_as_float(m ^ ((m >> 31) & 0x7fffffff));
}

// Joins the sums of N lanes (a power of two), each lane's own in a warp's first N lanes or repeated every N lanes:
// brings them to the largest maximum, then adds.
template <int NT>
__device__ __forceinline__ void warp_join(RunSum<NT> &sum, const float (&c)[NT], int N)
{
    const float m = warp_max(sum.m);
#pragma unroll
    for (int t = 0; t < NT; ++t) {
        // (a lane that has seen nothing above -inf has the sum 0, or NaN if it has seen one)
        float v = sum.s[t] * (sum.m == m ? 1.f : ex2_approx((sum.m - m) * c[t]));
        for (int o = N / 2; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
        sum.s[t] = v;
    }
    sum.m = m;
}
__device__ __forceinline__ float load_logit(const void *z, int64_t at, bool f32)
{
    if (f32) return reinterpret_cast<const volatile float *>(z)[at];
    return __uint_as_float((uint32_t)reinterpret_cast<const volatile uint16_t *>(z)[at] << 16);
}

// Round to nearest, ties to even; a NaN stays one.
__device__ __forceinline__ uint32_t bf16_bits(float lo, float hi)
{
    uint32_t r;
    asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
    return r;
}

template <bool F32>
__device__ __forceinline__ uint4 pack_granule(const float2 (&f)[RowElem<F32>::kPer / 2])
{
    if constexpr (F32)
        return make_uint4(__float_as_uint(f[0].x), __float_as_uint(f[0].y), __float_as_uint(f[1].x), __float_as_uint(f[1].y));
    else
        return make_uint4(bf16_bits(f[0].x, f[0].y), bf16_bits(f[1].x, f[1].y), bf16_bits(f[2].x, f[2].y),
                          bf16_bits(f[3].x, f[3].y));
}

template <bool F32>
__device__ __forceinline__ void store_elem(void *d, int64_t at, uint32_t bits)
{
    if constexpr (F32) reinterpret_cast<uint32_t *>(d)[at] = bits;
    else reinterpret_cast<uint16_t *>(d)[at] = (uint16_t)bits;
}

template <bool F32>
__device__ __forceinline__ uint32_t granule_elem(const uint4 &v, int j)
{
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
    if constexpr (F32) return w[j];
    else return (w[j >> 1] >> ((j & 1) * 16)) & 0xffffu;
}

__device__ __forceinline__ void st_row_v4(void *p, const uint4 &v)
{
    asm volatile("st.global.cs.v4.u32 [%0], {%1, %2, %3, %4};" ::"l"(p), "r"(v.x), "r"(v.y), "r"(v.z), "r"(v.w)
                 : "memory");
}

// Elements [from, to) of a granule whose first element is number `first` of a row, one by one.
template <bool F32>
__device__ __noinline__ void put_elements(char *out, int first, int V, uint4 o, int from, int to)
{
    constexpr int E = RowElem<F32>::kPer;
#pragma unroll
    for (int j = 0; j < E; ++j)
        if (j >= from && j < to && (unsigned)(first + j) < (unsigned)V) store_elem<F32>(out, first + j, granule_elem<F32>(o, j));
}

// Stores a warp's run of consecutive granules, 32 in each turn, to a row of the output that does not lie on their
// 16-byte boundaries.  A vector of the output is the end of one granule and the beginning of the next: a lane takes the
// one before its own from the lane before it, the first lane from the last one's of the turn before.  What has no whole
// neighbour goes element by element: the ends of the run.
template <bool F32>
struct Shifted {
    char *out;
    int V, cut;            // elements of a granule that complete the vector begun by the one before it
    uint32_t last[4];      // the lane's granule of the turn before
    int was;               // 1: there was one, 2: and it was all row

    __device__ __forceinline__ Shifted(char *o, const Row<F32> &r, int v) : out(o), V(v), last{0, 0, 0, 0}, was(0)
    {
        constexpr int E = RowElem<F32>::kPer, B = RowElem<F32>::kBytes;
        const int at = (int)((reinterpret_cast<uintptr_t>(o) / B - (uintptr_t)r.head) & (E - 1));   // of a granule in its vector
        cut = E - at;      // (at is not 0: the boundaries differ)
    }
    // All lanes; first: the granule's first element; state: 0 where there is none, else as `was`.  After the last turn
    // once more with nothing.
    __device__ __forceinline__ void put(int first, int state, const uint4 &o)
    {
        constexpr int E = RowElem<F32>::kPer, B = RowElem<F32>::kBytes;
        const int lane = threadIdx.x & 31, from = (lane + 31) & 31;
        const bool end = lane == 31;
        uint32_t w[8] = {0, 0, 0, 0, o.x, o.y, o.z, o.w};
#pragma unroll
        for (int k = 0; k < 4; ++k) w[k] = __shfl_sync(0xffffffffu, end ? last[k] : w[4 + k], from);
        const int left = __shfl_sync(0xffffffffu, end ? was : state, from);
        const int skip = cut * B;
        if ((state & 2) && (left & 2)) {
            uint4 v = make_uint4(0, 0, 0, 0);
            const int bits = (skip & 3) * 8;
            switch (skip >> 2) {   // (the same in every lane)
            case 0: v = make_uint4(__funnelshift_r(w[0], w[1], bits), __funnelshift_r(w[1], w[2], bits),
                                   __funnelshift_r(w[2], w[3], bits), __funnelshift_r(w[3], w[4], bits)); break;
            case 1: v = make_uint4(__funnelshift_r(w[1], w[2], bits), __funnelshift_r(w[2], w[3], bits),
                                   __funnelshift_r(w[3], w[4], bits), __funnelshift_r(w[4], w[5], bits)); break;
            case 2: v = make_uint4(__funnelshift_r(w[2], w[3], bits), __funnelshift_r(w[3], w[4], bits),
                                   __funnelshift_r(w[4], w[5], bits), __funnelshift_r(w[5], w[6], bits)); break;
            default: v = make_uint4(__funnelshift_r(w[3], w[4], bits), __funnelshift_r(w[4], w[5], bits),
                                    __funnelshift_r(w[5], w[6], bits), __funnelshift_r(w[6], w[7], bits)); break;
            }
            st_row_v4(out + ((int64_t)(first - E) * B + skip), v);
        } else {
            if (left) put_elements<F32>(out, first - E, V, make_uint4(w[0], w[1], w[2], w[3]), cut, E);
            if (state) put_elements<F32>(out, first, V, o, 0, cut);
        }
        last[0] = o.x;
        last[1] = o.y;
        last[2] = o.z;
        last[3] = o.w;
        was = state;
    }
};

// A row's entries in shared memory (of K each).
struct Entries {
    int *i;       // -1: absent
    float *g;     // the teacher's value, -inf where absent
    float *z;     // the row's logit there

    __device__ __forceinline__ Entries(void *at, int K)
        : i(reinterpret_cast<int *>(at)), g(reinterpret_cast<float *>(i + K)), z(g + K)
    {
    }
};

// What makes shares of the values: log2 q = (g - m) c - l2, m their maximum, l2 = log2 sum 2^((g - m) c).
struct Shares {
    float m, c, l2;
    __device__ __forceinline__ float log2_of(float g) const { return fmaf(g - m, c, -l2); }
};

// Indices seen, to tell whether one occurs twice: open addressing, at least twice as many slots as entries.
struct Seen {
    int *slot;
    unsigned mask;
    __device__ __forceinline__ bool before(int i) const
    {
        unsigned at = ((unsigned)i * 2654435761u >> 16) & mask;
        for (;;) {
            const int was = atomicCAS(slot + at, -1, i);
            if (was == -1) return false;
            if (was == i) return true;
            at = (at + 1) & mask;
        }
    }
};

// Facts about a row's entries that its threads join.
enum { kEntryTwice = 1, kEntryNan = 2, kEntryLabel = 4 };

// One entry of a row: its index, its value and its logit to shared memory.  *gm: the largest value of the thread's.
__device__ __forceinline__ void put_entry(const Entries &e, const DistillParams &p, int k, int i, float g, float z,
                                          int label, bool report, float *gm, int *facts)
{
    const bool there = i >= 0 && i < p.V;
    e.i[k] = there ? i : -1;
    e.g[k] = there ? g : -INFINITY;
    e.z[k] = z;
    if (there) {
        *gm = fmaxf(*gm, g);
        *facts |= (g != g ? kEntryNan : 0) | (i == label ? kEntryLabel : 0);
    }
    if (i >= p.V && report && p.status) atomicOr(p.status, kStatusBadToken);
}

// A warp's part of the row's shares, from its threads' own entries and their largest value: {maximum, sum, facts}.
template <int TH>
__device__ __forceinline__ float4 warp_shares(const Entries &e, int K, float c, float gm, int facts)
{
    gm = warp_max(gm);
    const float off = offset_of(gm);
    float sum = 0.f;
    for (int k = threadIdx.x; k < K; k += TH) sum += exp2f((e.g[k] - off) * c);
    return make_float4(gm, warp_sum(sum), __int_as_float((int)__reduce_or_sync(0xffffffffu, facts)), 0.f);
}

// The CTA's, from all warps' parts (in shared memory; a barrier before).  Returns whether any entry has a share
// (entries of no weight at all are absent ones).
template <int WARPS>
__device__ __forceinline__ bool join_shares(const float4 *part, float c, Shares *s, int *facts)
{
    const float4 v = part[threadIdx.x & (WARPS - 1)];
    s->m = warp_max(v.x);
    s->c = c;
    float sum = v.y * (v.x == s->m ? 1.f : exp2f((v.x - s->m) * c));
#pragma unroll
    for (int o = WARPS / 2; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
    s->l2 = log2f(sum);
    *facts = (int)__reduce_or_sync(0xffffffffu, __float_as_int(v.z));
    return s->m > -INFINITY || (*facts & kEntryNan);
}

// All of it at once, with one barrier.
template <bool F32, int TH>
__device__ __forceinline__ bool load_entries(const Entries &e, const DistillParams &p, int row, int label, int lo,
                                             int hi, float c, float4 *part, bool report, Shares *s, int *facts)
{
    float gm = -INFINITY;
    int mine = 0;
    for (int k = threadIdx.x; k < p.K; k += TH) {
        const int i = p.idx[(size_t)row * p.K + k];
        const float z = i >= lo && i < hi ? load_logit(p.z, (int64_t)row * p.ldz + i, F32) : 0.f;
        put_entry(e, p, k, i, p.val[(size_t)row * p.K + k], z, label, report, &gm, &mine);
    }
    const float4 w = warp_shares<TH>(e, p.K, c, gm, mine);
    if ((threadIdx.x & 31) == 0) part[threadIdx.x >> 5] = w;
    __syncthreads();
    return join_shares<TH / 32>(part, c, s, facts);
}

// A thread's part of KD / (tau^2 ln 2), l2 = log2 of the row's sum at tau.
template <int TH>
__device__ __forceinline__ float kd_part(const Entries &e, int K, const Shares &s, float off, float l2)
{
    float kd = 0.f;
    for (int o = threadIdx.x; o < K; o += TH) {
        const float lq = s.log2_of(e.g[o]), q = exp2f(lq);
        if (!(q == 0.f)) kd += q * (lq - fmaf(e.z[o] - off, s.c, -l2));   // (0 log 0 = 0)
    }
    return kd;
}

// d_j = A 2^(x_0) + B 2^(x_1), less the targets; with one exponential (NT 1) it is one of the two, or both at tau = 1
// in A.  From sums, x = (z - off) c; from log-sum-exps, x = (z / tau - lse) log2 e: the difference comes first, it is
// exact where the probability is large.  A coefficient of 0 is exactly 0, also for a row that has no sum (but at its NaN and
// +inf logits).
template <int NT, bool LSE>
struct GradFn {
    float A, B, s0, a0, m0, a1;
    __device__ __forceinline__ float2 operator()(f32x2 x) const
    {
        const f32x2 x0 = LSE ? ffma2(x, pack2(s0, s0), pack2(a0, a0)) : fadd2(x, pack2(a0, a0));
        const float2 e0 = unpack2(fmul2(x0, pack2(m0, m0)));
        f32x2 d = fmul2(pack2(A, A), pack2(ex2_approx(e0.x), ex2_approx(e0.y)));
        if constexpr (NT == 2) {
            const f32x2 x1 = LSE ? fadd2(x, pack2(a1, a1)) : x0;
            const float2 e1 = unpack2(fmul2(x1, pack2(kLog2e, kLog2e)));
            d = ffma2(pack2(B, B), pack2(ex2_approx(e1.x), ex2_approx(e1.y)), d);
        }
        return unpack2(d);
    }
    __device__ __forceinline__ float operator()(float x) const { return (*this)(pack2(x, x)).x; }
    template <bool F32>
    __device__ __forceinline__ uint4 granule(const uint4 &x) const
    {
        constexpr int P = RowElem<F32>::kPer / 2;
        f32x2 f[P];
        float2 d[P];
        granule_pairs<F32>(x, f);
#pragma unroll
        for (int j = 0; j < P; ++j) d[j] = (*this)(f[j]);
        return pack_granule<F32>(d);
    }
};

// Stores granule g of the gradient's row `out`, which lies on the same 16-byte boundaries as the logits' row.
// (The ends of a row out of line: their stores would be executed without effect for every granule otherwise.)
template <bool F32>
__device__ __noinline__ void put_edge_granule(char *out, int first, int V, uint4 o)
{
    constexpr int E = RowElem<F32>::kPer;
#pragma unroll
    for (int j = 0; j < E; ++j)
        if ((unsigned)(first + j) < (unsigned)V) store_elem<F32>(out, first + j, granule_elem<F32>(o, j));
}
template <bool F32>
__device__ __forceinline__ void put_granule(char *out, const Row<F32> &r, int g, const uint4 &o)
{
    if (r.whole(g)) st_row_v4(out + (int64_t)r.first(g) * RowElem<F32>::kBytes, o);
    else put_edge_granule<F32>(out, r.first(g), r.V, o);
}

// The places of the entries and the label within [lo, hi), each computed as a whole and rounded once; after everybody's
// stores and a barrier.  up: the row's upstream gradient, wt, wh: the terms' shares (wt 0: no entries).
template <bool F32, int TH, typename G>
__device__ __forceinline__ void put_targets(char *out, const DistillParams &p, const Entries &e, const Shares &s,
                                            int facts, int lo, int hi, float up, float wt, float wh, int label,
                                            float zy, const G &grad)
{
    if (wt > 0.f)
        for (int o = threadIdx.x; o < p.K; o += TH) {
            const int i = e.i[o];
            if (i < lo || i >= hi) continue;
            float q = exp2f(s.log2_of(e.g[o]));
            if (facts & kEntryTwice) {   // an index's first entry adds them all, in their order
                q = 0.f;
                bool first = true;
                for (int k = 0; k < p.K; ++k)
                    if (e.i[k] == i) {
                        first &= k >= o;
                        q += exp2f(s.log2_of(e.g[k]));
                    }
                if (!first) continue;
            }
            float d = fmaf(-up * wt * p.tau, q, grad(e.z[o]));
            if (i == label) d -= up * wh;
            store_elem<F32>(out, i, F32 ? __float_as_uint(d) : bf16_bits(d, 0.f) & 0xffffu);
        }
    // the label, where it is not one of the entries
    if (threadIdx.x == 0 && wh > 0.f && label >= lo && label < hi && !(wt > 0.f && (facts & kEntryLabel))) {
        const float d = grad(zy) - up * wh;
        store_elem<F32>(out, label, F32 ? __float_as_uint(d) : bf16_bits(d, 0.f) & 0xffffu);
    }
}

template <int NT>
__device__ __forceinline__ void put_sum(float (&at)[4], const RunSum<NT> &sum)
{
    at[0] = sum.m;
#pragma unroll
    for (int t = 0; t < NT; ++t) at[1 + t] = sum.s[t];
}
template <int NT>
__device__ __forceinline__ RunSum<NT> get_sum(const float (&at)[4])
{
    RunSum<NT> sum;
    sum.m = at[0];
#pragma unroll
    for (int t = 0; t < NT; ++t) sum.s[t] = at[1 + t];
    return sum;
}
template <int NT>
__device__ __forceinline__ RunSum<NT> empty_sum()
{
    RunSum<NT> sum;
    sum.m = -INFINITY;
#pragma unroll
    for (int t = 0; t < NT; ++t) sum.s[t] = 0.f;
    return sum;
}

// Adds the granules from v0 on of a CTA's n, from memory, to a thread's sum.
template <bool F32, int NT, int TH>
__device__ __forceinline__ void stream_sum(RunSum<NT> &sum, const Row<F32> &r, int gb, int v0, int n, const float (&c)[NT])
{
    int v = v0 + threadIdx.x;
    for (; v + 3 * TH < n; v += 4 * TH) {
        uint4 x[4];
#pragma unroll
        for (int k = 0; k < 4; ++k) x[k] = load_granule<F32>(r, gb + v + k * TH);
        run_add<F32, NT, 4>(sum, x, c);
    }
    if (v < n) {   // (the last up to three, in flight together as well)
        uint4 x[3];
#pragma unroll
        for (int k = 0; k < 3; ++k) {
            const uint32_t none = F32 ? 0xff800000u : 0xff80ff80u;
            x[k] = v + k * TH < n ? load_granule<F32>(r, gb + v + k * TH) : make_uint4(none, none, none, none);
        }
        run_add<F32, NT, 3>(sum, x, c);
    }
}

// The exponents' factors: c[0] is tau's, c[1] (NT 2) that of temperature 1.
template <int NT>
__device__ __forceinline__ void set_factors(float (&c)[NT], const DistillParams &p, float ctau)
{
    c[0] = NT == 2 || p.alpha > 0.f ? ctau : kLog2e;
    if constexpr (NT == 2) c[1] = kLog2e;
}

// The loss of a row from its sum, by one thread; kd: KD / (tau^2 ln 2).
template <int NT>
__device__ __forceinline__ void put_loss(const DistillParams &p, int row, const float (&l2)[NT], float off, float kd,
                                         float wt, float wh, float zy)
{
    constexpr int H = NT - 1;   // the sums at temperature 1
    float loss = 0.f;
    if (wt > 0.f) loss += wt * p.tau * p.tau * kLn2 * kd;
    if (wh > 0.f) loss += wh * fmaf(kLn2, l2[H], off - zy);
    p.loss[row] = loss;
    if (p.lse) {
        p.lse[2 * (size_t)row] = fmaf(kLn2, l2[0], off / p.tau);   // (NT 1 is tau = 1 here)
        p.lse[2 * (size_t)row + 1] = fmaf(kLn2, l2[H], off);
    }
}

// A CTA's run of a row's granules: first, number.
template <bool F32>
__device__ __forceinline__ int2 run_of(const Row<F32> &r, int C, int rank)
{
    const int per = (r.G + C - 1) >> (31 - __clz(C)), gb = min(r.G, rank * per);   // (C is a power of two)
    return make_int2(gb, min(r.G - gb, per));
}

// The granules [x, y) of a run that are all row (the row's first and last may not be).
template <bool F32>
__device__ __forceinline__ int2 whole_of(const Row<F32> &r, int2 run)
{
    const int x = run.x == 0 && run.y > 0 && !r.whole(0) ? 1 : 0;
    const int y = run.x + run.y == r.G && run.y > 0 && !r.whole(r.G - 1) ? run.y - 1 : run.y;
    return make_int2(x, y);
}

// ------------------------------------------------------------------ the loss
// One row per cluster, read once: bounded by HBM.  8192 rows of 151936 bf16 logits (one in twenty ignored) take 352 us,
// 6.71 TB/s of what is read (a copy reaches 6.78); 37 rows of 128256 fp32 ones with two temperatures 11 us, most of it a
// launch and two barriers of the cluster.  With 50 entries at tau 2 (two exponentials an element) the 8192 rows take 401.
template <bool F32, int NT, int TH>
__global__ void __launch_bounds__(TH, 1024 / TH) distill_loss_kernel(const DistillParams p)
{
    constexpr int WARPS = TH / 32;
    extern __shared__ __align__(16) uint4 smem[];
    __shared__ float4 part[WARPS];
    __shared__ float wsum[WARPS][4], wkd[WARPS];
    __shared__ __align__(16) float csum[kRowMaxCluster][4];
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int C = p.cluster, row = blockIdx.x / C, rank = blockIdx.x % C;
    const int label = p.labels ? p.labels[row] : 0;
    const bool bad = p.labels && label >= p.V;
    if (label < 0 || bad) {   // an ignored row: nothing of it is read, all its CTAs leave here
        if (rank == 0 && tid == 0) {
            if (bad && p.status) atomicOr(p.status, kStatusBadToken);
            p.loss[row] = 0.f;
            if (p.lse) p.lse[2 * (size_t)row] = p.lse[2 * (size_t)row + 1] = 0.f;
        }
        return;
    }
    if (C > 1) cluster_arrive();
    const Row<F32> r(p.z, row, p.ldz, p.V);
    const int2 run = run_of(r, C, rank);
    const float ctau = kLog2e / p.tau;
    float c[NT];
    set_factors(c, p, ctau);
    const Entries ent(smem, p.K);
    Shares shares;
    int facts;
    const bool any = p.alpha > 0.f && p.K > 0 && rank == 0 &&
                     load_entries<F32, TH>(ent, p, row, label, 0, p.V, ctau, part, true, &shares, &facts);
    const bool hard = p.alpha < 1.f && p.labels;
    const float zy = hard ? load_logit(p.z, (int64_t)row * p.ldz + label, F32) : 0.f;

    RunSum<NT> sum = empty_sum<NT>();
    stream_sum<F32, NT, TH>(sum, r, run.x, 0, run.y, c);
    warp_join(sum, c, 32);
    if (lane == 0) put_sum(wsum[warp], sum);
    __syncthreads();
    sum = get_sum<NT>(wsum[lane & (WARPS - 1)]);
    warp_join(sum, c, WARPS);
    if (C > 1) {
        cluster_wait();
        if (tid < C) st_peer_v4(peer_addr(csum[rank], tid), sum.m, sum.s[0], sum.s[NT - 1], 0.f);
        cluster_sync_all();
        if (rank != 0) return;
        sum = get_sum<NT>(csum[lane & (C - 1)]);
        warp_join(sum, c, C);
    }
    const float off = offset_of(sum.m);
    float l2[NT];
#pragma unroll
    for (int t = 0; t < NT; ++t) l2[t] = log2f(sum.s[t]);
    float kd = 0.f;
    if (any) {
        kd = warp_sum(kd_part<TH>(ent, p.K, shares, off, l2[0]));
        if (lane == 0) wkd[warp] = kd;
        __syncthreads();
        kd = 0.f;
        for (int w = 0; w < WARPS; ++w) kd += wkd[w];
    }
    if (tid == 0) put_loss(p, row, l2, off, kd, any ? p.alpha : 0.f, hard ? 1.f - p.alpha : 0.f, zy);
}

// ------------------------------------------------------------------ the gradient from the log-sum-exps
// p.cluster CTAs per row that need nothing of one another; the row streams through registers, four granules in
// flight per thread.  Bounded by HBM: 1000 rows of 151936 fp32 logits, read and written, 195 us or 6.1 TB/s of the rows
// that count (one granule in flight: 273 us); 221 us where the gradient's rows lie on other 16-byte boundaries (element by
// element 367).
template <bool F32, int NT, int TH>
__global__ void __launch_bounds__(TH, 1024 / TH) distill_grad_kernel(const DistillParams p)
{
    constexpr int WARPS = TH / 32, E = RowElem<F32>::kPer, B = RowElem<F32>::kBytes;
    extern __shared__ __align__(16) uint4 smem[];
    __shared__ float4 part[WARPS];
    const int tid = threadIdx.x;
    const int C = p.cluster, row = blockIdx.x / C, rank = blockIdx.x % C;
    const Row<F32> r(p.z, row, p.ldz, p.V);
    const int2 run = run_of(r, C, rank);
    const int lo = max(0, r.first(run.x)), hi = (int)min((int64_t)p.V, (int64_t)r.first(run.x) + (int64_t)run.y * E);
    char *out = reinterpret_cast<char *>(p.d) + (size_t)((int64_t)row * p.ldd) * B;
    // whether the output's vectors lie on the same boundaries as the input's
    const bool same = ((reinterpret_cast<uintptr_t>(out) - (uintptr_t)r.head * B) & 15u) == 0;
    const Entries ent(smem, p.K);
    const Seen seen{reinterpret_cast<int *>(ent.z + p.K), (unsigned)p.slots - 1u};
    const int label = p.labels ? p.labels[row] : 0;
    const bool bad = p.labels && label >= p.V, ignored = label < 0 || bad;
    if (bad && rank == 0 && tid == 0 && p.status) atomicOr(p.status, kStatusBadToken);

    bool any = false;
    Shares shares;
    int facts = 0;
    const bool hard = !ignored && p.alpha < 1.f && p.labels;
    float zy = 0.f;
    if (!ignored) {
        const float ctau = kLog2e / p.tau;
        if (p.alpha > 0.f && p.K > 0)
            any = load_entries<F32, TH>(ent, p, row, label, lo, hi, ctau, part, rank == 0, &shares, &facts);
        if (hard && label >= lo && label < hi) zy = load_logit(p.z, (int64_t)row * p.ldz + label, F32);
        __syncthreads();   // in place: the targets' logits are read before anybody stores
    }
    const float wt = any ? p.alpha : 0.f, wh = hard ? 1.f - p.alpha : 0.f;
    const float up = ignored ? 0.f : p.g ? p.g[row] : 1.f;
    GradFn<NT, true> grad;
    const bool tau_first = NT == 2 || p.alpha > 0.f;   // what the first exponential is of
    grad.A = NT == 2 ? up * wt * p.tau : up * (wt * p.tau + wh);
    grad.B = NT == 2 ? up * wh : 0.f;
    grad.s0 = tau_first ? 1.f / p.tau : 1.f;
    grad.m0 = kLog2e;
    grad.a0 = grad.A == 0.f ? -INFINITY : -p.lse_in[2 * (size_t)row + (tau_first ? 0 : 1)];
    grad.a1 = grad.B == 0.f ? -INFINITY : -p.lse_in[2 * (size_t)row + 1];

    if (same) {
        constexpr int U = 4;
        int v = tid;
        if (!ignored)
            for (; v + (U - 1) * TH < run.y; v += U * TH) {
                uint4 x[U];
#pragma unroll
                for (int k = 0; k < U; ++k) x[k] = load_granule<F32>(r, run.x + v + k * TH);
#pragma unroll
                for (int k = 0; k < U; ++k) put_granule<F32>(out, r, run.x + v + k * TH, grad.template granule<F32>(x[k]));
            }
        if (!ignored) {   // (the last up to three, in flight together as well)
            uint4 x[U - 1];
#pragma unroll
            for (int k = 0; k < U - 1; ++k)
                if (v + k * TH < run.y) x[k] = load_granule<F32>(r, run.x + v + k * TH);
#pragma unroll
            for (int k = 0; k < U - 1; ++k)
                if (v + k * TH < run.y) put_granule<F32>(out, r, run.x + v + k * TH, grad.template granule<F32>(x[k]));
        } else {
            for (; v < run.y; v += TH) put_granule<F32>(out, r, run.x + v, make_uint4(0, 0, 0, 0));
        }
    } else {
        constexpr int U = 4;
        const int wper = (run.y + WARPS - 1) / WARPS, w0 = min(run.y, (tid >> 5) * wper), w1 = min(run.y, w0 + wper);
        Shifted<F32> to(out, r, p.V);
        for (int v0 = w0; v0 < w1; v0 += 32 * U) {
            uint4 x[U];
#pragma unroll
            for (int k = 0; k < U; ++k) {
                const int v = v0 + 32 * k + (tid & 31);
                x[k] = v < w1 && !ignored ? load_granule<F32>(r, run.x + v) : make_uint4(0, 0, 0, 0);
            }
#pragma unroll
            for (int k = 0; k < U; ++k) {
                const int v = v0 + 32 * k + (tid & 31);
                const uint4 o = ignored ? make_uint4(0, 0, 0, 0) : grad.template granule<F32>(x[k]);
                to.put(r.first(run.x + v), v < w1 ? 1 + 2 * r.whole(run.x + v) : 0, o);
            }
        }
        to.put(r.first(run.x + w0 + ((w1 - w0 + 32 * U - 1) / (32 * U)) * 32 * U + (tid & 31)), 0, make_uint4(0, 0, 0, 0));
    }
    if (ignored) return;
    bool twice = false;
    if (any) {
        for (int i = tid; i < p.slots; i += TH) seen.slot[i] = -1;
        __syncthreads();
        for (int o = tid; o < p.K; o += TH)
            if (ent.i[o] >= lo && ent.i[o] < hi) twice |= seen.before(ent.i[o]);
    }
    if (__syncthreads_or(twice)) facts |= kEntryTwice;
    put_targets<F32, TH>(out, p, ent, shares, facts, lo, hi, up, wt, wh, label, zy, grad);
}

// ------------------------------------------------------------------ both in one pass
// Clusters that stay for many rows.  A row's share of a CTA is in shared memory from the sums to the gradient; as soon
// as a thread has a granule's gradient it sends for the same granule of the cluster's next row, into the same place:
// nobody else touches it, so the next row arrives while this one is stored, without a barrier.  The CTAs of a row
// exchange their sums by stores that count on an mbarrier of the receiver (a cluster barrier would wait for the
// gradient's stores as well).  A CTA whose wait gives up says so in the status word; its mbarriers' phases are out of step
// from then on, so that it neither arms nor waits nor sends any more and leaves NaN in its part of all rows to come.  The
// others miss its sums in the next row, and do the same after one more limit at most.
// 4096 rows of 128256 bf16 logits with 64 entries, read once and written once, take 377 us, 5.4 TB/s; one row per cluster
// and launch took 450.  Without entries it is 333 us, with 1000 of them 544, at tau 2 (two exponentials) 466: what bounds
// it is the issue of instructions (an exponential an element in the sums and another in the gradient, 24 warps to an SM)
// and the latency of the chain sums - exchange - gradient in each row, which two other CTAs on the SM cover in part.
// SHIFT: some rows of the gradient lie on other 16-byte boundaries than the logits' rows; a warp then has a run of
// consecutive granules (as Shifted wants them) and not every eighth run of 32, which is 6 % faster.
template <bool F32, int NT, bool SHIFT, int TH>
__global__ void __launch_bounds__(TH, kStepPerSm * kStepThreads / TH) distill_step_kernel(const DistillParams p)
{
    constexpr int WARPS = TH / 32, E = RowElem<F32>::kPer, B = RowElem<F32>::kBytes;
    constexpr int kLate = 4;                 // of a thread's granules that may still be on their way when a row begins
    constexpr int kBatch = F32 ? 4 : 2;      // granules summed together
    extern __shared__ __align__(16) uint4 row_smem[];
    __shared__ float4 part[WARPS];
    __shared__ float wsum[WARPS][4], wkd[WARPS];
    __shared__ __align__(16) float csum[2][kRowMaxCluster][4];
    __shared__ uint64_t arrived[2];
    __shared__ int gave_up;                  // set between a row's first barrier and its last one, read before the first
    __shared__ float label_logit;            // the first thread's: in place, it is read before the row's sums go out
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int C = p.cluster, rank = blockIdx.x % C, stride = gridDim.x / C;
    char *tables = reinterpret_cast<char *>(row_smem + p.cached);   // entries, two of them in turn, and their indices' table
    const size_t table_bytes = (size_t)p.K * 12;
    const Seen seen{reinterpret_cast<int *>(tables + 2 * table_bytes), (unsigned)p.slots - 1u};
    const float ctau = kLog2e / p.tau;
    float c[NT];
    set_factors(c, p, ctau);
    const bool soft = p.alpha > 0.f && p.K > 0, hard = p.alpha < 1.f && p.labels;
    const float wh = hard ? 1.f - p.alpha : 0.f;
    // a thread's places in shared memory, the same for every row: at0 and every kHop-th after it, before `end`
    constexpr int kHop = SHIFT ? 32 : TH;
    const int wper = (p.cached + WARPS - 1) / WARPS;
    const int at0 = SHIFT ? warp * wper + lane : tid, end = SHIFT ? min(p.cached, (warp + 1) * wper) : p.cached;
    const int turns = SHIFT ? (wper + 31) / 32 : (p.cached + TH - 1) / TH;
    const auto place = [&](int i) { return SHIFT && at0 + kHop * i >= end ? INT_MAX : at0 + kHop * i; };

    const auto label_of = [&](int row) { return p.labels && row < p.T ? p.labels[row] : 0; };
    const auto alive = [&](int row, int label) { return row < p.T && label >= 0 && label < p.V; };

    if (tid == 0) {
        mbar_init(&arrived[0], 1);
        mbar_init(&arrived[1], 1);
        mbar_init_fence();
        gave_up = 0;
    }
    if (soft)
        for (int i = tid; i < p.slots; i += TH) seen.slot[i] = -1;
    int row = blockIdx.x / C, label = label_of(row), uses = 0;
    {
        const Row<F32> r(p.z, row, p.ldz, p.V);
        const int2 run = run_of(r, C, rank);
        const int n = alive(row, label) ? min(run.y, p.cached) : 0;
        for (int i = 0; i < turns; ++i) {
            const int v = place(i);
            if (v < n) fetch_granule<F32>(r, run.x + v, row_smem + v);
            cp_async_commit();
        }
    }
    if (C > 1) cluster_sync_all();   // every CTA runs, and its mbarriers are there
    else __syncthreads();

    for (; row < p.T; row += stride) {
        const Row<F32> r(p.z, row, p.ldz, p.V);
        const int2 run = run_of(r, C, rank);
        const int n = run.y, nc = min(n, p.cached);
        const int lo = max(0, r.first(run.x)), hi = (int)min((int64_t)p.V, (int64_t)r.first(run.x) + (int64_t)n * E);
        char *out = reinterpret_cast<char *>(p.d) + (size_t)((int64_t)row * p.ldd) * B;
        // whether the output's vectors lie on the same boundaries as the input's
        const bool same = ((reinterpret_cast<uintptr_t>(out) - (uintptr_t)r.head * B) & 15u) == 0;
        const bool live = alive(row, label);
        const int nlabel = label_of(row + stride);
        const bool next = alive(row + stride, nlabel);
        const Row<F32> nr(p.z, next ? row + stride : row, p.ldz, p.V);
        const int2 nrun = run_of(nr, C, rank);
        const int nn = next ? min(nrun.y, p.cached) : 0;

        const int turn = uses & 1;
        const Entries ent(tables + turn * table_bytes, p.K);
        GradFn<NT, false> grad;
        Shares shares;
        float up = 0.f, wt = 0.f, off = 0.f, l2[NT];
        int facts = 0;
        bool any = false;
        if (live) {
            const bool alone = *(volatile int *)&gave_up != 0;   // (the same in all threads)
            // the entries and the label's logit are on their way while the row is summed
            if (soft)
                for (int k = tid; k < p.K; k += TH) {
                    cp_async4(ent.i + k, p.idx + (size_t)row * p.K + k);
                    cp_async4(ent.g + k, p.val + (size_t)row * p.K + k);
                }
            cp_async_commit();
            const float zy = hard && tid == 0 ? load_logit(p.z, (int64_t)row * p.ldz + label, F32) : 0.f;
            up = p.g ? p.g[row] : 1.f;

            RunSum<NT> sum = empty_sum<NT>();
            int v = at0;
            const int stop = min(nc, end);
            const auto batches = [&](int until) {
                for (; v + (kBatch - 1) * kHop < until; v += kBatch * kHop) {
                    uint4 x[kBatch];
#pragma unroll
                    for (int k = 0; k < kBatch; ++k) x[k] = row_smem[v + k * kHop];
                    run_add<F32, NT, kBatch>(sum, x, c);
                }
            };
            cp_async_wait<kLate + 1>();   // (the last group is the entries')
            batches(min(stop, (SHIFT ? warp * wper : 0) + (turns - kLate) * kHop));
            cp_async_wait<0>();
            batches(stop);
            for (; v < stop; v += kHop) {
                const uint4 one[1] = {row_smem[v]};
                run_add<F32, NT, 1>(sum, one, c);
            }
            stream_sum<F32, NT, TH>(sum, r, run.x, nc, n, c);
            if (soft) {
                float gm = -INFINITY;
                int mine = 0;
                const int from = rank ? lo : 0, to = rank ? hi : p.V;
                constexpr int U = 4;   // entries of a thread whose logits are on their way together
                for (int k0 = tid; k0 < p.K; k0 += U * TH) {
                    int i[U];
                    float z[U];
#pragma unroll
                    for (int u = 0; u < U; ++u) {
                        i[u] = k0 + u * TH < p.K ? ent.i[k0 + u * TH] : -1;
                        z[u] = i[u] >= from && i[u] < to ? load_logit(p.z, (int64_t)row * p.ldz + i[u], F32) : 0.f;
                    }
#pragma unroll
                    for (int u = 0; u < U; ++u) {
                        const int k = k0 + u * TH;
                        if (k >= p.K) break;
                        put_entry(ent, p, k, i[u], ent.g[k], z[u], label, rank == 0, &gm, &mine);
                        if (i[u] >= lo && i[u] < hi && seen.before(i[u])) mine |= kEntryTwice;
                    }
                }
                const float4 w = warp_shares<TH>(ent, p.K, ctau, gm, mine);
                if (lane == 0) part[warp] = w;
            }
            warp_join(sum, c, 32);
            if (lane == 0) put_sum(wsum[warp], sum);
            if (tid == 0) label_logit = zy;
            __syncthreads();
            sum = get_sum<NT>(wsum[lane & (WARPS - 1)]);
            warp_join(sum, c, WARPS);
            bool met = true;
            if (C > 1) {
                if (tid == 0 && !alone) mbar_arrive_expect_tx(&arrived[turn], 16u * C);
                if (tid < C && !alone && !(row == p.withheld && rank == 1 && tid == 0))
                    st_async_v4(peer_addr(csum[turn][rank], tid), sum.m, sum.s[0], sum.s[NT - 1], 0.f,
                                peer_addr(&arrived[turn], tid));
            }
            if (soft) {
                any = join_shares<WARPS>(part, ctau, &shares, &facts);
                for (int i = tid; i < p.slots; i += TH) seen.slot[i] = -1;   // (all have looked; a barrier ahead of the next row)
            }
            if (C > 1) {
                met = !alone && mbar_wait<false, true>(&arrived[turn], (uses >> 1) & 1, &gave_up);
                sum = get_sum<NT>(csum[turn][lane & (C - 1)]);
                warp_join(sum, c, C);
                if (!met) {
                    sum.s[0] = sum.s[NT - 1] = __int_as_float(0x7fffffff);
                    if (!alone) {
                        *(volatile int *)&gave_up = 1;   // (who still waits gives up with it)
                        if (p.status) atomicOr(p.status, kStatusTimeout);
                    }
                }
            }
            ++uses;
            wt = any ? p.alpha : 0.f;
            off = offset_of(sum.m);
#pragma unroll
            for (int t = 0; t < NT; ++t) l2[t] = log2f(sum.s[t]);
            grad.A = NT == 2 ? up * wt * p.tau : up * (wt * p.tau + wh);
            grad.B = NT == 2 ? up * wh : 0.f;
            if (grad.A != 0.f) grad.A /= sum.s[0];
            if (grad.B != 0.f) grad.B /= sum.s[NT - 1];
            grad.s0 = 1.f;
            grad.a0 = grad.a1 = -off;
            grad.m0 = c[0];
        }
        // the gradient, and the next row's granules into the places that become free
        const auto value = [&](int v) {
            if (!live) return make_uint4(0, 0, 0, 0);   // an ignored row: nothing of it is read
            return grad.template granule<F32>(v < nc ? row_smem[v] : load_granule<F32>(r, run.x + v));
        };
        const auto send = [&](int i) {
            const int v = place(i);
            if (v < nn) fetch_granule<F32>(nr, nrun.x + v, row_smem + v);
            cp_async_commit();
        };
        if (!SHIFT || same) {
            const int2 whole = whole_of(r, run), nwhole = whole_of(nr, nrun);
            // turns in which the whole warp (all threads) has whole granules to store and to send for
            const int first = SHIFT ? warp * wper : 0, last = min(min(min(whole.y, nc), min(nwhole.y, nn)), end);
            const int plain1 = live && next && last > first ? (last - first) / kHop : 0;
            const auto turn_of = [&](int i) {
                const int v = place(i);
                if (v < nc) put_granule<F32>(out, r, run.x + v, value(v));
                send(i);
            };
            int i = 0;
            if (first < max(whole.x, nwhole.x)) turn_of(i++);
            char *dst = out + ((int64_t)r.first(run.x) * B + (int64_t)at0 * 16);   // (aligned)
            const char *src = nr.base + ((size_t)nrun.x + at0) * 16;
            uint4 *at = row_smem + at0;
            for (; i + kBatch <= plain1; i += kBatch) {
                uint4 x[kBatch];
#pragma unroll
                for (int k = 0; k < kBatch; ++k) x[k] = at[(i + k) * kHop];
#pragma unroll
                for (int k = 0; k < kBatch; ++k) {
                    const size_t o = (size_t)(i + k) * (kHop * 16);
                    st_row_v4(dst + o, grad.template granule<F32>(x[k]));
                    cp_async16(at + (i + k) * kHop, src + o);
                    cp_async_commit();
                }
            }
            for (; i < turns; ++i) turn_of(i);
            for (int v = nc + tid; v < n; v += TH) put_granule<F32>(out, r, run.x + v, value(v));
        } else {
            Shifted<F32> to(out, r, p.V);
            for (int i = 0; i < turns; ++i) {
                const int v = place(i);
                const bool on = v < nc;
                const uint4 o = on ? value(v) : make_uint4(0, 0, 0, 0);
                send(i);
                to.put(r.first(run.x + at0 + 32 * i), on ? 1 + 2 * r.whole(run.x + v) : 0, o);
            }
            to.put(r.first(run.x + at0 + 32 * turns), 0, make_uint4(0, 0, 0, 0));
            for (int v0 = nc + 32 * warp; v0 < n; v0 += TH) {   // (what did not fit: each turn a run of its own)
                const int v = v0 + lane;
                to.put(r.first(run.x + v), v < n ? 1 + 2 * r.whole(run.x + v) : 0,
                       v < n ? value(v) : make_uint4(0, 0, 0, 0));
                to.put(r.first(run.x + v + 32), 0, make_uint4(0, 0, 0, 0));
            }
        }
        if (live) {
            const float zy = tid == 0 ? label_logit : 0.f;
            if (rank == 0 && any) {
                const float kd = warp_sum(kd_part<TH>(ent, p.K, shares, off, l2[0]));
                if (lane == 0) wkd[warp] = kd;
            }
            __syncthreads();
            if (rank == 0 && tid == 0) {
                float kd = 0.f;
                for (int w = 0; any && w < WARPS; ++w) kd += wkd[w];
                put_loss(p, row, l2, off, kd, wt, wh, zy);
            }
            put_targets<F32, TH>(out, p, ent, shares, facts, lo, hi, up, wt, wh, label, zy, grad);
        } else if (rank == 0 && tid == 0) {
            p.loss[row] = 0.f;
            if (label >= p.V && p.status) atomicOr(p.status, kStatusBadToken);
        }
        label = nlabel;
    }
    if (C > 1) {
        cluster_sync_all();   // nobody leaves while another may still write to its memory
        if (gave_up) {        // what it has not waited for has a millisecond to arrive
            const unsigned long long t0 = global_ns();
            while (global_ns() - t0 < 1000000ull) __nanosleep(1000);
        }
    }
}

size_t al16(size_t v) { return (v + 15) & ~(size_t)15; }

// CTAs of a row: one where the rows alone fill the GPU with `fill` CTAs to an SM, more where they do not, as long as each
// still has a granule for each of `threads`; and as many as it takes for the share that stays on chip to leave room for
// other CTAs on the SM.  Measured with 1 / 2 / 4 / 8 CTAs a row (us; 151936 bf16 or fp32 logits): loss of 76
// rows 20.0 / 14.1 / 11.4 / 10.8, of 304 rows 25.6 / 22.1 / 23.6 / 31.7 (the rule's 1 is not the best there), of 1216 rows
// 61 / 69 / 77 / 103 (a cluster costs about a microsecond of every wave); gradient of 76 rows 46 / 30 / 26 / 22, of 304 rows
// 73 / 66 / 67 / 67, of 1216 rows 236 / 234 / 239 / 241.
int row_cluster(int T, int64_t row_bytes, size_t share, int fill, int threads)
{
    int C = 1;
    while (C < kRowMaxCluster && ((share && row_bytes > (int64_t)C * (int64_t)share) ||
                                  ((int64_t)T * C < fill * 152 && row_bytes >= 2 * (int64_t)C * threads * 16)))
        C *= 2;
    return C;
}

static_assert((kLossThreads & (kLossThreads - 1)) == 0 && (kGradThreads & (kGradThreads - 1)) == 0 &&
                  (kStepThreads & (kStepThreads - 1)) == 0 && kLossThreads <= 1024 && kGradThreads >= 64 &&
                  kStepThreads >= 64,
              "the sums over warps halve their number");

// Rows that are short go to smaller CTAs, more of them to an SM: what a row costs apart from its elements (the sums over
// warps, the exchange, the entries) is latency.  8192 rows of bf16 logits with 128 / 256 threads (us): loss of 1000 logits
// 19 / 28, gradient 34 / 59, both in one pass 52 / 86; 4000 rows of 16000 30 / 36, 57 / 65 and 64 / 76, of 32000 46 / 49,
// 98 / 102 and 127 / 108, of 128256 159 / 156 and 345 / 333 (loss and gradient).  With 1000 entries the one-pass kernel is
// slower with fewer threads (8000 logits: 283 / 237), with 200 not (93 / 119).
constexpr int kShortThreads = 128;
constexpr int64_t kShortBytes = 32 * 1024;
bool short_rows(const DistillParams &p, int64_t bytes) { return p.cluster == 1 && bytes <= kShortBytes; }

// Two exponentials per element only where both temperatures count and differ.
bool two_sums(const DistillParams &p) { return p.tau != 1.f && p.alpha > 0.f && p.alpha < 1.f; }

template <bool F32, int TH>
cudaError_t launch_loss(const DistillParams &p, cudaStream_t st)
{
    const size_t smem = (size_t)p.K * 12;
    const bool two = two_sums(p) || (p.lse && p.tau != 1.f);   // both log-sum-exps are asked for
    const int64_t ctas = (int64_t)p.T * p.cluster;
    return two ? launch_clusters<distill_loss_kernel<F32, 2, TH>>(ctas, TH, smem, kMaxSmem, p.cluster, st, p)
               : launch_clusters<distill_loss_kernel<F32, 1, TH>>(ctas, TH, smem, kMaxSmem, p.cluster, st, p);
}

template <bool F32>
cudaError_t launch_loss(DistillParams p, cudaStream_t st)
{
    const int64_t bytes = (int64_t)p.V * RowElem<F32>::kBytes;
    p.cluster = row_cluster(p.T, bytes, 0, 2, kLossThreads);
    return short_rows(p, bytes) ? launch_loss<F32, kShortThreads>(p, st) : launch_loss<F32, kLossThreads>(p, st);
}

// Shared memory for a row's entries, `copies` of them, and the table of their indices.
size_t plan_entries(DistillParams &p, int copies)
{
    p.slots = 32;
    while (p.slots < 2 * p.K) p.slots *= 2;
    return copies * ((size_t)p.K * 12) + (size_t)p.slots * 4;
}

template <bool F32, int TH>
cudaError_t launch_grad(const DistillParams &p, size_t smem, cudaStream_t st)
{
    // (the CTAs of a row need no cluster)
    const int64_t ctas = (int64_t)p.T * p.cluster;
    return two_sums(p) ? launch_clusters<distill_grad_kernel<F32, 2, TH>>(ctas, TH, smem, kMaxSmem, 1, st, p)
                       : launch_clusters<distill_grad_kernel<F32, 1, TH>>(ctas, TH, smem, kMaxSmem, 1, st, p);
}

template <bool F32>
cudaError_t launch_grad(DistillParams p, cudaStream_t st)
{
    const int64_t bytes = (int64_t)p.V * RowElem<F32>::kBytes;
    p.cluster = row_cluster(p.T, bytes, 0, 4, kGradThreads);
    const size_t smem = plan_entries(p, 1);
    return short_rows(p, bytes) ? launch_grad<F32, kShortThreads>(p, smem, st) : launch_grad<F32, kGradThreads>(p, smem, st);
}

template <bool F32, int NT, bool SHIFT, int TH>
cudaError_t launch_step(const DistillParams &p, size_t smem, cudaStream_t st)
{
    // as many clusters as the GPU holds at a time, each for every so many rows
    int fit = 0;
    const cudaError_t e = resident_clusters<distill_step_kernel<F32, NT, SHIFT, TH>>(TH, smem, kMaxSmem, p.cluster, &fit);
    if (e != cudaSuccess) return e;
    const int64_t clusters = p.T < fit ? p.T : fit < 1 ? 1 : fit;
    return launch_clusters<distill_step_kernel<F32, NT, SHIFT, TH>>(clusters * p.cluster, TH, smem, kMaxSmem, p.cluster, st, p);
}

template <bool F32, int NT, bool SHIFT>
cudaError_t launch_step(DistillParams p, cudaStream_t st)
{
    const int64_t bytes = (int64_t)p.V * RowElem<F32>::kBytes;
    const size_t entries = plan_entries(p, 2);
    p.cluster = row_cluster(p.T, bytes, kStepShare, 2, 2 * kStepThreads);
    const size_t share = al16((size_t)((bytes + 32 + p.cluster - 1) / p.cluster) + 32);
    p.cached = (int)((share < kMaxCache ? share : kMaxCache) / 16);
    const size_t smem = (size_t)p.cached * 16 + entries;
    return short_rows(p, bytes) && p.K <= 2 * kShortThreads ? launch_step<F32, NT, SHIFT, kShortThreads>(p, smem, st)
                                : launch_step<F32, NT, SHIFT, kStepThreads>(p, smem, st);
}

template <bool F32>
cudaError_t launch_step(const DistillParams &p, cudaStream_t st)
{
    constexpr int B = RowElem<F32>::kBytes;
    const bool same = (reinterpret_cast<uintptr_t>(p.z) - reinterpret_cast<uintptr_t>(p.d)) % 16 == 0 &&
                      (p.T == 1 || (p.ldz - p.ldd) * B % 16 == 0);
    if (two_sums(p)) return same ? launch_step<F32, 2, false>(p, st) : launch_step<F32, 2, true>(p, st);
    return same ? launch_step<F32, 1, false>(p, st) : launch_step<F32, 1, true>(p, st);
}

// What the three calls have in common; their own outputs are checked by each.
template <bool F32>
sats_status check_distill(const DistillParams &p)
{
    constexpr int B = RowElem<F32>::kBytes;
    if (p.T < 0 || p.V < 1 || p.ldz < p.V || p.K < 0) return SATS_EINVAL;
    if (!(p.tau >= kMinTau && p.tau <= 1.f / kMinTau) || !(p.alpha >= 0.f && p.alpha <= 1.f)) return SATS_EINVAL;
    if (p.K > kMaxEntries || p.V > INT_MAX - 64 || p.T > INT_MAX / kRowMaxCluster) return SATS_ESHAPE;
    if (p.ldz > (int64_t)1 << 40 || p.ldd > (int64_t)1 << 40) return SATS_ESHAPE;
    if (p.T == 0) return SATS_OK;
    if (!p.z || reinterpret_cast<uintptr_t>(p.z) % B) return SATS_EINVAL;
    if (p.K > 0 && (!p.idx || !p.val)) return SATS_EINVAL;
    if (!(p.alpha > 0.f && p.K > 0) && !(p.alpha < 1.f && p.labels)) return SATS_EINVAL;   // neither term
    return SATS_OK;
}

// The gradient may overwrite the logits (the same rows at the same places) or lie between their rows, equally far apart;
// any other overlap of the two areas is refused.
template <bool F32>
bool bad_overlap(const DistillParams &p)
{
    constexpr int B = RowElem<F32>::kBytes;
    const uintptr_t z0 = reinterpret_cast<uintptr_t>(p.z), d0 = reinterpret_cast<uintptr_t>(p.d);
    const uintptr_t z1 = z0 + (uintptr_t)((p.T - 1) * p.ldz + p.V) * B, d1 = d0 + (uintptr_t)((p.T - 1) * p.ldd + p.V) * B;
    if (z0 == d0 && (p.T == 1 || p.ldz == p.ldd)) return false;
    if (!(z0 < d1 && d0 < z1)) return false;
    if (p.T == 1 || p.ldz != p.ldd) return true;
    // how far behind the beginning of a row of the logits one of the gradient begins
    const uintptr_t step = (uintptr_t)p.ldz * B, row = (uintptr_t)p.V * B;
    const uintptr_t behind = d0 >= z0 ? (d0 - z0) % step : (step - (z0 - d0) % step) % step;
    return behind < row || behind > step - row;
}

sats_status launched(cudaError_t e) { return e == cudaSuccess ? SATS_OK : cuda_fail(e, "distillation kernel launch"); }

template <bool F32>
sats_status distill_loss(const void *logits, int64_t ld, int T, int V, const int32_t *idx, const float *val, int K,
                         const int32_t *labels, float tau, float alpha, float *loss, float *lse, int32_t *dev_status,
                         void *stream)
{
    DistillParams p{};
    p.z = logits; p.ldz = ld; p.T = T; p.V = V; p.idx = idx; p.val = val; p.K = K; p.labels = labels;
    p.tau = tau; p.alpha = alpha; p.loss = loss; p.lse = lse; p.status = dev_status;
    const sats_status s = check_distill<F32>(p);
    if (s != SATS_OK || T == 0) return s;
    if (!loss) return SATS_EINVAL;
    return launched(launch_loss<F32>(p, static_cast<cudaStream_t>(stream)));
}

template <bool F32>
sats_status distill_grad(const void *logits, int64_t ld, int T, int V, const int32_t *idx, const float *val, int K,
                         const int32_t *labels, float tau, float alpha, const float *lse, const float *g,
                         void *dlogits, int64_t ld_d, int32_t *dev_status, void *stream)
{
    DistillParams p{};
    p.z = logits; p.ldz = ld; p.T = T; p.V = V; p.idx = idx; p.val = val; p.K = K; p.labels = labels;
    p.tau = tau; p.alpha = alpha; p.lse_in = lse; p.g = g; p.d = dlogits; p.ldd = ld_d; p.status = dev_status;
    const sats_status s = check_distill<F32>(p);
    if (s != SATS_OK) return s;
    if (ld_d < V) return SATS_EINVAL;
    if (T == 0) return SATS_OK;
    if (!lse || !dlogits || reinterpret_cast<uintptr_t>(dlogits) % RowElem<F32>::kBytes || bad_overlap<F32>(p))
        return SATS_EINVAL;
    return launched(launch_grad<F32>(p, static_cast<cudaStream_t>(stream)));
}

template <bool F32>
sats_status distill_loss_grad(const void *logits, int64_t ld, int T, int V, const int32_t *idx, const float *val,
                              int K, const int32_t *labels, float tau, float alpha, const float *g, float *loss,
                              void *dlogits, int64_t ld_d, int32_t *dev_status, void *stream, int withheld = -1)
{
    DistillParams p{};
    p.z = logits; p.ldz = ld; p.T = T; p.V = V; p.idx = idx; p.val = val; p.K = K; p.labels = labels;
    p.tau = tau; p.alpha = alpha; p.loss = loss; p.g = g; p.d = dlogits; p.ldd = ld_d; p.status = dev_status;
    p.withheld = withheld;
    const sats_status s = check_distill<F32>(p);
    if (s != SATS_OK) return s;
    if (ld_d < V) return SATS_EINVAL;
    if (T == 0) return SATS_OK;
    if (!loss || !dlogits || reinterpret_cast<uintptr_t>(dlogits) % RowElem<F32>::kBytes || bad_overlap<F32>(p))
        return SATS_EINVAL;
    return launched(launch_step<F32>(p, static_cast<cudaStream_t>(stream)));
}

}  // namespace
}  // namespace sats

extern "C" {

sats_status sats_distill_loss(const void *logits, int64_t ld, int T, int V, const int32_t *top_idx,
                              const float *top_val, int K, const int32_t *labels, float tau, float alpha, float *loss,
                              float *lse, int32_t *dev_status, void *stream)
{
    return sats::distill_loss<false>(logits, ld, T, V, top_idx, top_val, K, labels, tau, alpha, loss, lse, dev_status,
                                     stream);
}

sats_status sats_distill_loss_f32(const float *logits, int64_t ld, int T, int V, const int32_t *top_idx,
                                  const float *top_val, int K, const int32_t *labels, float tau, float alpha,
                                  float *loss, float *lse, int32_t *dev_status, void *stream)
{
    return sats::distill_loss<true>(logits, ld, T, V, top_idx, top_val, K, labels, tau, alpha, loss, lse, dev_status,
                                    stream);
}

sats_status sats_distill_grad(const void *logits, int64_t ld, int T, int V, const int32_t *top_idx,
                              const float *top_val, int K, const int32_t *labels, float tau, float alpha,
                              const float *lse, const float *g, void *dlogits, int64_t ld_d, int32_t *dev_status,
                              void *stream)
{
    return sats::distill_grad<false>(logits, ld, T, V, top_idx, top_val, K, labels, tau, alpha, lse, g, dlogits, ld_d,
                                     dev_status, stream);
}

sats_status sats_distill_grad_f32(const float *logits, int64_t ld, int T, int V, const int32_t *top_idx,
                                  const float *top_val, int K, const int32_t *labels, float tau, float alpha,
                                  const float *lse, const float *g, float *dlogits, int64_t ld_d,
                                  int32_t *dev_status, void *stream)
{
    return sats::distill_grad<true>(logits, ld, T, V, top_idx, top_val, K, labels, tau, alpha, lse, g, dlogits, ld_d,
                                    dev_status, stream);
}

sats_status sats_distill_loss_grad(const void *logits, int64_t ld, int T, int V, const int32_t *top_idx,
                                   const float *top_val, int K, const int32_t *labels, float tau, float alpha,
                                   const float *g, float *loss, void *dlogits, int64_t ld_d, int32_t *dev_status,
                                   void *stream)
{
    return sats::distill_loss_grad<false>(logits, ld, T, V, top_idx, top_val, K, labels, tau, alpha, g, loss, dlogits,
                                          ld_d, dev_status, stream);
}

sats_status sats_distill_loss_grad_f32(const float *logits, int64_t ld, int T, int V, const int32_t *top_idx,
                                       const float *top_val, int K, const int32_t *labels, float tau, float alpha,
                                       const float *g, float *loss, float *dlogits, int64_t ld_d,
                                       int32_t *dev_status, void *stream)
{
    return sats::distill_loss_grad<true>(logits, ld, T, V, top_idx, top_val, K, labels, tau, alpha, g, loss, dlogits,
                                         ld_d, dev_status, stream);
}

sats_status sats_selftest_distill_timeout(const void *logits, int64_t ld, int T, int V, const int32_t *labels,
                                          float *loss, void *dlogits, int64_t ld_d, int row, int32_t *dev_status,
                                          void *stream)
{
    if (row < 0 || row >= T) return SATS_EINVAL;
    return sats::distill_loss_grad<false>(logits, ld, T, V, nullptr, nullptr, 0, labels, 1.f, 0.f, nullptr, loss, dlogits,
                                          ld_d, dev_status, stream, row);
}

}  // extern "C"
