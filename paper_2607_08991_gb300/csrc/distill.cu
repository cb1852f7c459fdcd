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
constexpr int kAhead = 8;                     // granules in flight per thread on the way to shared memory
constexpr int kHashSlots = 2 * kMaxEntries;
constexpr size_t kMaxCache = 192 * 1024;      // of a row's share in shared memory

constexpr size_t kGradShare = 72 * 1024;      // of a row per CTA, where the cluster allows: several CTAs to an SM
constexpr size_t kMaxSmem = kMaxCache + (size_t)kRowThreads * 16 + (size_t)kMaxEntries * 12;

enum { kLoss = 0, kLossGrad = 1, kGrad = 2 };

// Threads of a CTA, and CTAs that an SM is to hold.
template <int MODE>
struct Shape {
    static constexpr int kThreads = MODE == kLoss ? 512 : 256;
    static constexpr int kWarps = kThreads / 32;
    static constexpr int kPerSm = MODE == kGrad ? 4 : MODE == kLossGrad ? 3 : 2;
};

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
    int work;                 // granules of shared memory behind them: the stage, and before that the hash table
};

// Sums of 2^((z - m) c) for one or two c, m the largest z so far.
template <int NT>
struct RunSum {
    float m;
    float s[NT];
};

template <int NT>
__device__ __forceinline__ void run_join(RunSum<NT> &a, const RunSum<NT> &b, const float (&c)[NT])
{
    const float m = fmaxf(a.m, b.m);
#pragma unroll
    for (int t = 0; t < NT; ++t) {
        // (a side that has seen nothing above -inf has the sum 0, or NaN if it has seen one)
        const float fa = a.m == m ? 1.f : ex2_approx((a.m - m) * c[t]);
        const float fb = b.m == m ? 1.f : ex2_approx((b.m - m) * c[t]);
        a.s[t] = a.s[t] * fa + b.s[t] * fb;
    }
    a.m = m;
}

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

template <int WARPS>
__device__ __forceinline__ float block_max(float v, float *part)
{
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) v = fmaxf(v, __shfl_xor_sync(0xffffffffu, v, o));
    if ((threadIdx.x & 31) == 0) part[threadIdx.x >> 5] = v;
    __syncthreads();
    v = part[threadIdx.x & (WARPS - 1)];
#pragma unroll
    for (int o = WARPS / 2; o > 0; o >>= 1) v = fmaxf(v, __shfl_xor_sync(0xffffffffu, v, o));
    return v;
}

template <int WARPS>
__device__ __forceinline__ float block_sum(float v, float *part)
{
    v = warp_sum(v);
    if ((threadIdx.x & 31) == 0) part[threadIdx.x >> 5] = v;
    __syncthreads();
    v = part[threadIdx.x & (WARPS - 1)];
#pragma unroll
    for (int o = WARPS / 2; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    return v;
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

// Stores the elements of the n granules from g0 on (their values in `stage`) to a row of the output that does not
// lie on the granules' boundaries: whole 16-byte vectors of the output where these granules cover them, single
// elements at both ends.  All threads of the CTA; `stage` complete before, free again after the call's end and a sync.
template <bool F32, int TH>
__device__ __forceinline__ void store_shifted(char *out, const Row<F32> &r, int g0, int n, const uint4 *stage)
{
    constexpr int E = RowElem<F32>::kPer, B = RowElem<F32>::kBytes;
    const int f0 = r.first(g0);
    const int64_t lo = f0 > 0 ? f0 : 0;
    const int64_t end = (int64_t)f0 + (int64_t)n * E, hi = end < r.V ? end : r.V;
    const int oh = (int)(reinterpret_cast<uintptr_t>(out) & 15u) / B;
    const int64_t o0 = (lo + oh) / E, o1 = (hi + oh + E - 1) / E;
    for (int64_t o = o0 + threadIdx.x; o < o1; o += TH) {
        const int64_t e0 = o * E - oh;
        uint32_t w[4];
        const bool full = e0 >= lo && e0 + E <= hi;
        if constexpr (F32) {
            const uint32_t *s = reinterpret_cast<const uint32_t *>(stage);
#pragma unroll
            for (int j = 0; j < E; ++j) {
                const int64_t e = e0 + j;
                w[j] = e >= lo && e < hi ? s[e - f0] : 0u;
                if (!full && e >= lo && e < hi) store_elem<F32>(out, e, w[j]);
            }
        } else {
            const uint16_t *s = reinterpret_cast<const uint16_t *>(stage);
#pragma unroll
            for (int j = 0; j < E / 2; ++j) {
                const int64_t e = e0 + 2 * j;
                const uint32_t a = e >= lo && e < hi ? s[e - f0] : 0u;
                const uint32_t b = e + 1 >= lo && e + 1 < hi ? s[e + 1 - f0] : 0u;
                w[j] = a | (b << 16);
                if (!full) {
                    if (e >= lo && e < hi) store_elem<F32>(out, e, a);
                    if (e + 1 >= lo && e + 1 < hi) store_elem<F32>(out, e + 1, b);
                }
            }
        }
        if (full) st_row_v4(out + e0 * B, make_uint4(w[0], w[1], w[2], w[3]));
    }
}

// A row's entries in shared memory (of K each).
struct Entries {
    int *i;       // -1: absent
    float *lq;    // log2 q
    float *z;     // the row's logit there
};

// Fills them in; whether any entry has a share.  All threads; part: 2 WARPS floats.
template <bool F32, int TH>
__device__ __forceinline__ bool load_entries(const Entries &e, const DistillParams &p, int row, float c, float *part,
                                             bool report)
{
    float gm = -INFINITY;
    bool nan = false;
    for (int k = threadIdx.x; k < p.K; k += TH) {
        const int i = p.idx[(size_t)row * p.K + k];
        const bool there = i >= 0 && i < p.V;
        const float g = there ? p.val[(size_t)row * p.K + k] : -INFINITY;
        e.i[k] = there ? i : -1;
        e.lq[k] = g;
        e.z[k] = there ? load_logit(p.z, (int64_t)row * p.ldz + i, F32) : 0.f;
        gm = fmaxf(gm, g);
        nan |= g != g;
        if (i >= p.V && report && p.status) atomicOr(p.status, kStatusBadToken);
    }
    gm = block_max<TH / 32>(gm, part);
    if (!__syncthreads_or(gm > -INFINITY || nan)) return false;   // (entries of no weight at all are absent ones)
    float sum = 0.f;
    for (int k = threadIdx.x; k < p.K; k += TH) {
        const float l = (e.lq[k] - gm) * c;
        e.lq[k] = l;
        sum += exp2f(l);
    }
    const float l2 = log2f(block_sum<TH / 32>(sum, part + TH / 32));
    for (int k = threadIdx.x; k < p.K; k += TH) e.lq[k] -= l2;
    return true;
}

// One row per cluster of p.cluster CTAs.
// MODE kLoss reads the row once; kLossGrad keeps it in shared memory between the sums and the gradient (what does
// not fit is read again); kGrad needs no sums, they come in lse_in.
// NT: 2 where sums at tau and at 1 are both needed and differ, c[0] being tau's.
template <bool F32, int MODE, int NT>
__global__ void __launch_bounds__(Shape<MODE>::kThreads, Shape<MODE>::kPerSm) distill_kernel(const DistillParams p)
{
    extern __shared__ __align__(16) uint4 row_smem[];
    constexpr int TH = Shape<MODE>::kThreads, WARPS = Shape<MODE>::kWarps;
    __shared__ float part[3 * WARPS];
    __shared__ float wsum[WARPS][4];
    __shared__ __align__(16) float csum[kRowMaxCluster][4];
    constexpr int E = RowElem<F32>::kPer, B = RowElem<F32>::kBytes;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int C = p.cluster, row = blockIdx.x / C;
    const unsigned rank = blockIdx.x % C;
    const Row<F32> r(p.z, row, p.ldz, p.V);
    const int per = (r.G + C - 1) / C, gb = min(r.G, (int)rank * per), n = min(r.G - gb, per);
    const float ctau = kLog2e / p.tau;
    float c[NT];
    c[0] = NT == 2 || p.alpha > 0.f ? ctau : kLog2e;
    if constexpr (NT == 2) c[1] = kLog2e;

    // an ignored row: nothing of it is read
    const int label = p.labels ? p.labels[row] : 0;
    const bool bad = p.labels && label >= p.V;
    if (bad && rank == 0 && tid == 0 && p.status) atomicOr(p.status, kStatusBadToken);
    char *out = MODE == kLoss ? nullptr : reinterpret_cast<char *>(p.d) + (size_t)((int64_t)row * p.ldd) * B;
    // whether output vectors lie on the same boundaries as the input's
    const bool same = MODE == kLoss || ((reinterpret_cast<uintptr_t>(out) - (uintptr_t)r.head * B) & 15u) == 0;
    uint4 *stage = row_smem + p.cached;
    Entries ent;
    ent.i = reinterpret_cast<int *>(stage + p.work);
    ent.lq = reinterpret_cast<float *>(ent.i + p.K);
    ent.z = ent.lq + p.K;
    if (label < 0 || bad) {
        if (rank == 0 && tid == 0) {
            if (MODE != kGrad && p.loss) p.loss[row] = 0.f;
            if (MODE != kGrad && p.lse) p.lse[2 * (size_t)row] = p.lse[2 * (size_t)row + 1] = 0.f;
        }
        if constexpr (MODE != kLoss) {
            const uint4 zero = make_uint4(0, 0, 0, 0);
            if (!same) stage[tid] = zero;
            __syncthreads();
            for (int v0 = 0; v0 < n; v0 += TH) {
                const int g = gb + v0 + tid;
                if (!same) {
                    store_shifted<F32, TH>(out, r, gb + v0, min(TH, n - v0), stage);
                } else if (v0 + tid < n) {
                    if (r.whole(g)) st_row_v4(out + (int64_t)r.first(g) * B, zero);
                    else
                        for (int j = 0; j < E; ++j)
                            if (r.inside(r.first(g) + j)) store_elem<F32>(out, r.first(g) + j, 0u);
                }
            }
        }
        return;   // (all CTAs of the row leave here: none of them waits)
    }

    if (MODE != kGrad && C > 1) cluster_arrive();
    // start the row on its way first: the entries are small
    if constexpr (MODE == kLossGrad) {
        for (int i = 0; i < kAhead; ++i) {
            const int v = tid + i * TH;
            if (v < min(n, p.cached)) fetch_granule<F32>(r, gb + v, row_smem + v);
            cp_async_commit();
        }
    }
    bool any = false;   // the row has an entry with a share
    if (p.alpha > 0.f && p.K > 0 && (MODE != kLoss || rank == 0))
        any = load_entries<F32, TH>(ent, p, row, ctau, part, rank == 0);
    const bool hard = p.alpha < 1.f && p.labels;
    const float zy = hard ? load_logit(p.z, (int64_t)row * p.ldz + label, F32) : 0.f;
    const float wt = any ? p.alpha : 0.f, wh = hard ? 1.f - p.alpha : 0.f;

    float off = 0.f, inv[NT];   // 2^((z - off) c) * inv = probability; MODE kGrad: see there
    if constexpr (MODE != kGrad) {
        RunSum<NT> sum;
        sum.m = -INFINITY;
#pragma unroll
        for (int t = 0; t < NT; ++t) sum.s[t] = 0.f;
        int done = 0;
        if constexpr (MODE == kLossGrad) {
            const int nc = min(n, p.cached);
            for (int i = 0; tid + i * TH < nc; ++i) {
                cp_async_wait<kAhead - 1>();
                const int v = tid + i * TH, next = v + kAhead * TH;
                const uint4 one[1] = {row_smem[v]};
                if (next < nc) fetch_granule<F32>(r, gb + next, row_smem + next);
                cp_async_commit();
                run_add<F32, NT, 1>(sum, one, c);
            }
            done = nc;
        }
        int v = done + tid;
        for (; v + 3 * TH < n; v += 4 * TH) {
            uint4 x[4];
#pragma unroll
            for (int k = 0; k < 4; ++k) x[k] = load_granule<F32>(r, gb + v + k * TH);
            run_add<F32, NT, 4>(sum, x, c);
        }
        for (; v < n; v += TH) {
            const uint4 one[1] = {load_granule<F32>(r, gb + v)};
            run_add<F32, NT, 1>(sum, one, c);
        }
        // the warp, the CTA, the cluster
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) {
            RunSum<NT> other;
            other.m = __shfl_xor_sync(0xffffffffu, sum.m, o);
#pragma unroll
            for (int t = 0; t < NT; ++t) other.s[t] = __shfl_xor_sync(0xffffffffu, sum.s[t], o);
            run_join(sum, other, c);
        }
        if (lane == 0) {
            wsum[warp][0] = sum.m;
#pragma unroll
            for (int t = 0; t < NT; ++t) wsum[warp][1 + t] = sum.s[t];
        }
        __syncthreads();
        sum.m = wsum[lane & (WARPS - 1)][0];
#pragma unroll
        for (int t = 0; t < NT; ++t) sum.s[t] = wsum[lane & (WARPS - 1)][1 + t];
#pragma unroll
        for (int o = WARPS / 2; o > 0; o >>= 1) {
            RunSum<NT> other;
            other.m = __shfl_xor_sync(0xffffffffu, sum.m, o);
#pragma unroll
            for (int t = 0; t < NT; ++t) other.s[t] = __shfl_xor_sync(0xffffffffu, sum.s[t], o);
            run_join(sum, other, c);
        }
        if (C > 1) {
            cluster_wait();
            if (tid < C) st_peer_v4(peer_addr(csum[rank], tid), sum.m, sum.s[0], sum.s[NT - 1], 0.f);
            cluster_sync_all();
            sum.m = -INFINITY;
#pragma unroll
            for (int t = 0; t < NT; ++t) sum.s[t] = 0.f;
            for (int k = 0; k < C; ++k) {
                RunSum<NT> other;
                other.m = csum[k][0];
#pragma unroll
                for (int t = 0; t < NT; ++t) other.s[t] = csum[k][1 + t];
                run_join(sum, other, c);
            }
        }
        float l2[NT];
        off = offset_of(sum.m);
#pragma unroll
        for (int t = 0; t < NT; ++t) {
            l2[t] = log2f(sum.s[t]);
            inv[t] = 1.f / sum.s[t];
        }
        if (rank == 0) {
            float kd = 0.f;
            if (any) {
                for (int o = tid; o < p.K; o += TH) {
                    const float q = exp2f(ent.lq[o]);
                    if (!(q == 0.f)) kd += q * (ent.lq[o] - fmaf(ent.z[o] - off, ctau, -l2[0]));   // (0 log 0 = 0)
                }
                kd = block_sum<WARPS>(kd, part + 2 * WARPS);
            }
            if (tid == 0) {
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
        }
    }

    if constexpr (MODE != kLoss) {
        const float up = p.g ? p.g[row] : 1.f;
        // d_j = A 2^(x_0) + B 2^(x_1) less the targets; NT 1: one of the two, or both at tau = 1 in A
        float A, Bq = 0.f;
        float itau = 1.f, l0 = 0.f, l1 = 0.f;
        if constexpr (NT == 2) {
            A = up * wt * p.tau;
            Bq = up * wh;
        } else {
            A = up * (wt * p.tau + wh);
        }
        if constexpr (MODE == kLossGrad) {
            // (a row of no weight has the gradient 0, also where it has no sum)
            if (A != 0.f) A *= inv[0];
            if constexpr (NT == 2)
                if (Bq != 0.f) Bq *= inv[1];
        } else {
            // p = 2^((z / tau - lse) log2 e): the difference first, it is exact where p is large
            itau = NT == 2 || p.alpha > 0.f ? 1.f / p.tau : 1.f;
            l0 = p.lse_in[2 * (size_t)row + (NT == 2 || p.alpha > 0.f ? 0 : 1)];
            if constexpr (NT == 2) l1 = p.lse_in[2 * (size_t)row + 1];
            if (A == 0.f) l0 = INFINITY;
            if (Bq == 0.f) l1 = INFINITY;
            __syncthreads();   // in place: the targets' logits are read before anybody stores
        }
        // the two steps of an exponent: to pairs, and to single values the same way
        const float s0 = MODE == kLossGrad ? 1.f : itau, a0 = MODE == kLossGrad ? -off : -l0;
        const float a1 = MODE == kLossGrad ? -off : -l1;
        const float m0 = MODE == kLossGrad ? c[0] : kLog2e, m1 = kLog2e;
        const auto grad2 = [&](f32x2 x) {
            const f32x2 x0 = MODE == kLossGrad ? fadd2(x, pack2(a0, a0)) : ffma2(x, pack2(s0, s0), pack2(a0, a0));
            const float2 e0 = unpack2(fmul2(x0, pack2(m0, m0)));
            f32x2 d = fmul2(pack2(A, A), pack2(ex2_approx(e0.x), ex2_approx(e0.y)));
            if constexpr (NT == 2) {
                const f32x2 x1 = MODE == kLossGrad ? x0 : fadd2(x, pack2(a1, a1));
                const float2 e1 = unpack2(fmul2(x1, pack2(m1, m1)));
                d = ffma2(pack2(Bq, Bq), pack2(ex2_approx(e1.x), ex2_approx(e1.y)), d);
            }
            return unpack2(d);
        };
        const auto grad = [&](float x) { return grad2(pack2(x, x)).x; };
        const auto one = [&](const uint4 &x) {
            f32x2 f[E / 2];
            float2 d[E / 2];
            granule_pairs<F32>(x, f);
#pragma unroll
            for (int j = 0; j < E / 2; ++j) d[j] = grad2(f[j]);
            return pack_granule<F32>(d);
        };
        const auto put = [&](int g, const uint4 &o) {
            if (r.whole(g)) st_row_v4(out + (int64_t)r.first(g) * B, o);
            else
#pragma unroll
                for (int j = 0; j < E; ++j)
                    if (r.inside(r.first(g) + j)) store_elem<F32>(out, r.first(g) + j, granule_elem<F32>(o, j));
        };
        const auto fetched = [&](int v) {
            return MODE == kLossGrad && v < p.cached ? row_smem[v] : load_granule<F32>(r, gb + v);
        };
        if (same) {
            constexpr int U = MODE == kGrad ? 4 : 1;   // loads in flight per thread
            int v = tid;
            for (; v + (U - 1) * TH < n; v += U * TH) {
                uint4 x[U];
#pragma unroll
                for (int k = 0; k < U; ++k) x[k] = fetched(v + k * TH);
#pragma unroll
                for (int k = 0; k < U; ++k) put(gb + v + k * TH, one(x[k]));
            }
            for (; v < n; v += TH) put(gb + v, one(fetched(v)));
        } else {
            for (int v0 = 0; v0 < n; v0 += TH) {
                if (v0 + tid < n) stage[tid] = one(fetched(v0 + tid));
                __syncthreads();
                store_shifted<F32, TH>(out, r, gb + v0, min(TH, n - v0), stage);
                __syncthreads();
            }
        }
        // the targets' places, each computed as a whole and rounded once, after everybody's stores
        const int lo = max(0, r.first(gb)), hi = (int)min((int64_t)p.V, (int64_t)r.first(gb) + (int64_t)n * E);
        bool twice = false;
        int *hash = reinterpret_cast<int *>(row_smem);   // (over the cached row, which nobody needs any more)
        if (any) {
            // does an index occur twice?  (open addressing; as many slots as twice the entries)
            __syncthreads();
            for (int i = tid; i < kHashSlots; i += TH) hash[i] = -1;
            __syncthreads();
            for (int o = tid; o < p.K; o += TH) {
                const int i = ent.i[o];
                if (i < lo || i >= hi) continue;
                unsigned slot = ((unsigned)i * 2654435761u) >> 21;
                static_assert(kHashSlots == 2048, "the shift above");
                for (;;) {
                    const int was = atomicCAS(&hash[slot], -1, i);
                    if (was == -1) break;
                    if (was == i) { twice = true; break; }
                    slot = (slot + 1) & (kHashSlots - 1);
                }
            }
        }
        twice = __syncthreads_or(twice);
        bool labelled = false;
        if (any)
            for (int o = tid; o < p.K; o += TH) {
                const int i = ent.i[o];
                if (i < lo || i >= hi) continue;
                float q = exp2f(ent.lq[o]);
                if (twice) {   // an index's first entry adds them all, in their order
                    q = 0.f;
                    bool first = true;
                    for (int k = 0; k < p.K; ++k)
                        if (ent.i[k] == i) {
                            first &= k >= o;
                            q += exp2f(ent.lq[k]);
                        }
                    if (!first) continue;
                }
                float d = fmaf(-up * wt * p.tau, q, grad(ent.z[o]));
                if (hard && i == label) {
                    d -= up * wh;
                    labelled = true;
                }
                store_elem<F32>(out, i, F32 ? __float_as_uint(d) : bf16_bits(d, 0.f) & 0xffffu);
            }
        // the label, where it is not one of the entries
        if (hard && label >= lo && label < hi && !__syncthreads_or(labelled) && tid == 0) {
            const float d = grad(zy) - up * wh;
            store_elem<F32>(out, label, F32 ? __float_as_uint(d) : bf16_bits(d, 0.f) & 0xffffu);
        }
    }
}

size_t al16(size_t v) { return (v + 15) & ~(size_t)15; }

// CTAs of a row: one where the rows alone fill the GPU, more where they do not, as long as each still has a granule
// per thread; and as many as it takes for the share that stays on chip to leave room for other CTAs on the SM.
int row_cluster(int T, int64_t row_bytes, size_t share)
{
    int C = 1;
    while (C < kRowMaxCluster && ((share && row_bytes > (int64_t)C * (int64_t)share) ||
                                  ((int64_t)T * C < 2 * 152 && row_bytes >= 2 * (int64_t)C * kRowThreads * 16)))
        C *= 2;
    return C;
}

template <bool F32, int MODE, int NT>
cudaError_t launch_distill(DistillParams p, cudaStream_t st)
{
    const int64_t bytes = (int64_t)p.V * RowElem<F32>::kBytes;
    p.cluster = row_cluster(p.T, bytes, MODE == kLossGrad ? kGradShare : 0);
    p.cached = p.work = 0;
    if (MODE == kLossGrad) {
        const size_t share = al16((size_t)((bytes + 32 + p.cluster - 1) / p.cluster) + 32);
        p.cached = (int)((share < kMaxCache ? share : kMaxCache) / 16);
    }
    if (MODE != kLoss) {
        // a stage where the gradient's rows do not lie on the logits' 16-byte boundaries; room for the hash table
        constexpr int B = RowElem<F32>::kBytes;
        const bool same = (reinterpret_cast<uintptr_t>(p.z) - reinterpret_cast<uintptr_t>(p.d)) % 16 == 0 &&
                          (p.T == 1 || (p.ldz - p.ldd) * B % 16 == 0);
        p.work = same ? 0 : Shape<MODE>::kThreads;
        const int least = p.K > 0 ? kHashSlots * 4 / 16 : 0;
        if (p.cached + p.work < least) p.work = least - p.cached;
    }
    const size_t smem = ((size_t)p.cached + p.work) * 16 + (size_t)p.K * 12;
    auto kern = distill_kernel<F32, MODE, NT>;
    if (smem > 40 * 1024) {
        const cudaError_t e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)kMaxSmem);
        if (e != cudaSuccess) return e;
    }
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)p.T * (unsigned)p.cluster);
    cfg.blockDim = dim3(Shape<MODE>::kThreads);
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

template <bool F32, int MODE>
cudaError_t launch_distill_nt(const DistillParams &p, cudaStream_t st)
{
    const bool both = MODE == kLoss ? p.lse != nullptr || (p.alpha > 0.f && p.alpha < 1.f)
                                    : p.alpha > 0.f && p.alpha < 1.f;
    return p.tau != 1.f && both ? launch_distill<F32, MODE, 2>(p, st) : launch_distill<F32, MODE, 1>(p, st);
}

// What the three calls have in common; MODE's own outputs are checked by the entries.
template <bool F32>
sats_status check_distill(const DistillParams &p)
{
    constexpr int B = RowElem<F32>::kBytes;
    if (p.T < 0 || p.V < 1 || p.ldz < p.V || p.K < 0) return SATS_EINVAL;
    if (!(p.tau > 0.f) || std::isinf(p.tau) || !(p.alpha >= 0.f && p.alpha <= 1.f)) return SATS_EINVAL;
    if (p.K > kMaxEntries || p.V > INT_MAX - 64 || p.T > INT_MAX / kRowMaxCluster) return SATS_ESHAPE;
    if (p.ldz > (int64_t)1 << 40 || p.ldd > (int64_t)1 << 40) return SATS_ESHAPE;
    if (p.T == 0) return SATS_OK;
    if (!p.z || reinterpret_cast<uintptr_t>(p.z) % B) return SATS_EINVAL;
    if (p.K > 0 && (!p.idx || !p.val)) return SATS_EINVAL;
    if (!(p.alpha > 0.f && p.K > 0) && !(p.alpha < 1.f && p.labels)) return SATS_EINVAL;   // neither term
    return SATS_OK;
}

// The gradient may overwrite the logits (the same rows at the same places); any other overlap is refused.
template <bool F32>
bool bad_overlap(const DistillParams &p)
{
    constexpr int B = RowElem<F32>::kBytes;
    const uintptr_t z0 = reinterpret_cast<uintptr_t>(p.z), d0 = reinterpret_cast<uintptr_t>(p.d);
    const uintptr_t z1 = z0 + (uintptr_t)((p.T - 1) * p.ldz + p.V) * B, d1 = d0 + (uintptr_t)((p.T - 1) * p.ldd + p.V) * B;
    if (z0 == d0 && (p.T == 1 || p.ldz == p.ldd)) return false;
    return z0 < d1 && d0 < z1;
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
    return launched(launch_distill_nt<F32, kLoss>(p, static_cast<cudaStream_t>(stream)));
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
    return launched(launch_distill_nt<F32, kGrad>(p, static_cast<cudaStream_t>(stream)));
}

template <bool F32>
sats_status distill_loss_grad(const void *logits, int64_t ld, int T, int V, const int32_t *idx, const float *val,
                              int K, const int32_t *labels, float tau, float alpha, const float *g, float *loss,
                              void *dlogits, int64_t ld_d, int32_t *dev_status, void *stream)
{
    DistillParams p{};
    p.z = logits; p.ldz = ld; p.T = T; p.V = V; p.idx = idx; p.val = val; p.K = K; p.labels = labels;
    p.tau = tau; p.alpha = alpha; p.loss = loss; p.g = g; p.d = dlogits; p.ldd = ld_d; p.status = dev_status;
    const sats_status s = check_distill<F32>(p);
    if (s != SATS_OK) return s;
    if (ld_d < V) return SATS_EINVAL;
    if (T == 0) return SATS_OK;
    if (!loss || !dlogits || reinterpret_cast<uintptr_t>(dlogits) % RowElem<F32>::kBytes || bad_overlap<F32>(p))
        return SATS_EINVAL;
    return launched(launch_distill_nt<F32, kLossGrad>(p, static_cast<cudaStream_t>(stream)));
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

}  // extern "C"
