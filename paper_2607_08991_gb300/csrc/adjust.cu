// adjust.cu -- penalties for repeated tokens, biases and masks on rows of logits (sats_adjust_logits), and the gradient
// of that (sats_adjust_logits_grad).
//
// A row is cut into slices of the vocabulary, a CTA each.  The CTA reads the row's whole history and counts, in shared
// memory, the ids that fall into its slice (whole numbers: the counts do not depend on an order); meanwhile the slice's
// logits arrive in shared memory.  The few logits whose token was counted or has a bias are changed there, each by
// one thread that claims its count, from the logit as it came and in fp32, rounded once.  Then the slice goes out in
// 16-byte vectors with the mask's bits applied on the way.  So the row is read and written once whatever it holds, and
// in place only what changes is touched.
#include <algorithm>
#include <climits>
#include <cuda_bf16.h>

#include "internal.h"
#include "rows.cuh"

namespace sats {
namespace {

constexpr int kAdjThreads = 512;
constexpr int kMaxBiases = 1024;
constexpr int kNarrowHist = 1 << 15;   // histories shorter than this fit 16-bit counts
constexpr size_t kMaxAdjSmem = 200 * 1024;

struct AdjustParams {
    const void *src;         // the logits, or the gradient that comes in
    const void *z;           // the logits
    void *out;
    int64_t ld_src, ld_z, ld_out;
    int B, V, L;
    const int32_t *hist;
    int64_t ld_hist;
    const int32_t *hist_len, *n_prompt;
    const float *rep, *pres, *freq;
    const int32_t *bias_idx;
    const float *bias_val;
    int M;
    const uint32_t *mask;
    int64_t ld_mask;
    int n_masks;
    const int32_t *mask_row;
    int32_t *status;
    int S, slices;           // elements of a slice (a multiple of 32), slices of a row
    bool wide;               // 32-bit counts
};

// Calls f(id, position) for the ids at positions [0, n), spread over the CTA; whole 16-byte vectors where they lie inside,
// four of a thread in flight.
template <typename F>
__device__ __forceinline__ void for_each_id(const int32_t *p, int n, F f)
{
    constexpr int kFlight = 4;
    const int lead = (int)((reinterpret_cast<uintptr_t>(p) >> 2) & 3);   // ids between the vector boundary and the first
    const int vectors = (int)(((int64_t)n + lead + 3) >> 2);
    const int4 *base = reinterpret_cast<const int4 *>(p - lead);
    for (int v0 = threadIdx.x; v0 < vectors; v0 += kAdjThreads * kFlight) {
        int4 q[kFlight];
#pragma unroll
        for (int i = 0; i < kFlight; ++i) {
            const int v = v0 + i * kAdjThreads, at = 4 * v - lead;
            q[i] = make_int4(-1, -1, -1, -1);
            if (v >= vectors) continue;
            if (at >= 0 && at <= n - 4) q[i] = __ldg(base + v);
            else {
                if (at >= 0) q[i].x = __ldg(p + at);
                if (at + 1 >= 0 && at + 1 < n) q[i].y = __ldg(p + at + 1);
                if (at + 2 >= 0 && at + 2 < n) q[i].z = __ldg(p + at + 2);
                if (at + 3 < n) q[i].w = __ldg(p + at + 3);
            }
        }
#pragma unroll
        for (int i = 0; i < kFlight; ++i) {
            const int at = 4 * (v0 + i * kAdjThreads) - lead;
            f(q[i].x, at);
            f(q[i].y, at + 1);
            f(q[i].z, at + 2);
            f(q[i].w, at + 3);
        }
    }
}

template <bool F32>
__device__ __forceinline__ float load_elem(const void *p, int64_t i)
{
    if constexpr (F32) return *(static_cast<const volatile float *>(p) + i);
    else return __uint_as_float((uint32_t) * (static_cast<const volatile uint16_t *>(p) + i) << 16);
}

template <bool F32>
__device__ __forceinline__ void store_elem(void *p, int64_t i, float v)
{
    if constexpr (F32) static_cast<float *>(p)[i] = v;
    else static_cast<__nv_bfloat16 *>(p)[i] = __float2bfloat16_rn(v);
}

// The counts of a slice's tokens.  Forward: a field of 16 (or 32) bits each, the top bit for "in the prompt", the others the
// number of generated ones.  Gradient: a bit each.
template <bool GRAD>
struct Counts {
    uint32_t *w;
    bool wide;

    __device__ __forceinline__ void mark(int i, bool generated)
    {
        if constexpr (GRAD) {
            const uint32_t bit = 1u << (i & 31);
            if (!(*static_cast<volatile uint32_t *>(w + (i >> 5)) & bit)) atomicOr(w + (i >> 5), bit);
        } else if (wide) {
            if (generated) atomicAdd(w + i, 1u);
            else if (!(*static_cast<volatile uint32_t *>(w + i) >> 31)) atomicOr(w + i, 0x80000000u);
        } else {
            const int sh = 16 * (i & 1);
            uint32_t *p = w + (i >> 1);
            if (generated) atomicAdd(p, 1u << sh);
            else if (!(*static_cast<volatile uint32_t *>(p) & (0x8000u << sh))) atomicOr(p, 0x8000u << sh);
        }
    }
    // The token's field, which is 0 from then on: one thread gets it.  Bit 31: seen; below: how often generated.
    __device__ __forceinline__ uint32_t claim(int i)
    {
        if constexpr (GRAD) {
            const uint32_t bit = 1u << (i & 31);
            if (!(*static_cast<volatile uint32_t *>(w + (i >> 5)) & bit)) return 0u;
            return atomicAnd(w + (i >> 5), ~bit) & bit ? 0x80000000u : 0u;
        } else if (wide) {
            if (!*static_cast<volatile uint32_t *>(w + i)) return 0u;
            const uint32_t f = atomicExch(w + i, 0u);
            return f ? f | 0x80000000u : 0u;
        } else {
            const int sh = 16 * (i & 1);
            uint32_t *p = w + (i >> 1);
            if (!(*static_cast<volatile uint32_t *>(p) >> sh & 0xffffu)) return 0u;
            const uint32_t f = atomicAnd(p, ~(0xffffu << sh)) >> sh & 0xffffu;
            return f ? (f & 0x7fffu) | 0x80000000u : 0u;
        }
    }
};

// A setting of the row; outside its range it is off and noted.
__device__ __forceinline__ float setting(const float *p, int row, float off, bool positive, bool *bad)
{
    if (!p) return off;
    const float v = p[row];
    if (isfinite(v) && (!positive || v > 0.f)) return v;
    *bad = true;
    return off;
}

// 4 (fp32) or 8 (bf16) elements at byte `off` of shared memory, wherever that is.
template <bool F32>
__device__ __forceinline__ uint4 load_anywhere(const char *stage, int off, bool aligned)
{
    if (aligned) return *reinterpret_cast<const uint4 *>(stage + off);
    const uint32_t *p = reinterpret_cast<const uint32_t *>(stage + (off & ~3));
    const uint32_t a = p[0], b = p[1], c = p[2], d = p[3];
    if (F32 || (off & 2) == 0) return make_uint4(a, b, c, d);
    const uint32_t e = p[4];
    return make_uint4(__funnelshift_r(a, b, 16), __funnelshift_r(b, c, 16), __funnelshift_r(c, d, 16),
                      __funnelshift_r(d, e, 16));
}

template <bool F32, bool GRAD, bool INPLACE>
__global__ void __launch_bounds__(kAdjThreads) adjust_kernel(const AdjustParams p)
{
    constexpr int ES = RowElem<F32>::kBytes, E = RowElem<F32>::kPer;
    constexpr uint32_t kBanned = GRAD ? 0u : (F32 ? 0xff800000u : 0xff80u);
    extern __shared__ __align__(16) char smem[];
    __shared__ int n_bias;
    const int tid = threadIdx.x;
    char *stage = smem;
    const size_t stage_bytes = INPLACE ? 0 : (size_t)p.S * ES + 32;
    uint32_t *table = reinterpret_cast<uint32_t *>(smem + stage_bytes);
    const int table_words = p.hist ? (GRAD ? p.S / 32 : (p.wide ? p.S : p.S / 2)) : 0;
    uint32_t *mask_words = table + table_words;   // S / 32 + 1
    int2 *biases = reinterpret_cast<int2 *>(mask_words + (p.mask ? p.S / 32 + 2 : 0));
    bool bad = false;

    const int64_t units = (int64_t)p.B * p.slices;
    for (int64_t u = blockIdx.x; u < units; u += gridDim.x) {
        const int row = (int)(u / p.slices);
        const int e0 = (int)(u - (int64_t)row * p.slices) * p.S;
        const int n = min(p.S, p.V - e0);
        const Row<F32> in(p.src, row, p.ld_src, p.V), to(p.out, row, p.ld_out, p.V);
        char *const out = static_cast<char *>(p.out) + (row * p.ld_out + e0) * ES;

        // the slice's logits on their way to shared memory: its granules, from byte 0 on
        const int ga = (in.head + e0) / E;
        if constexpr (!INPLACE) {
            const int gb = (int)(((int64_t)in.head + e0 + n + E - 1) / E);
            for (int g = ga + tid; g < gb; g += kAdjThreads) {
                char *const at = stage + (size_t)(g - ga) * 16;
                if (in.whole(g)) cp_async16(at, in.base + (size_t)g * 16);
                else {
#pragma unroll
                    for (int j = 0; j < E; ++j)
                        if (in.inside(in.first(g) + j)) {
                            if constexpr (F32)
                                reinterpret_cast<float *>(at)[j] = reinterpret_cast<const float *>(in.base)[(size_t)g * E + j];
                            else
                                reinterpret_cast<uint16_t *>(at)[j] =
                                    reinterpret_cast<const uint16_t *>(in.base)[(size_t)g * E + j];
                        }
                }
            }
            cp_async_commit();
        }

        // the row's settings
        int len = 0, prompt = 0;
        const float rep = setting(p.rep, row, 1.f, true, &bad);
        const float pres = GRAD ? 0.f : setting(p.pres, row, 0.f, false, &bad);
        const float freq = GRAD ? 0.f : setting(p.freq, row, 0.f, false, &bad);
        const int32_t *hist = nullptr;
        if (p.hist) {
            hist = p.hist + row * p.ld_hist;
            len = p.hist_len ? p.hist_len[row] : p.L;
            if (len < 0 || len > p.L) {
                bad = true;
                len = len < 0 ? 0 : p.L;
            }
            if (p.n_prompt) prompt = p.n_prompt[row];
            if (rep == 1.f && pres == 0.f && freq == 0.f) len = 0;   // nothing would change
        }
        const uint32_t *mask = nullptr;
        if (p.mask) {
            int m = p.mask_row ? p.mask_row[row] : row;
            if (m >= p.n_masks) {
                bad = true;
                m = -1;
            }
            if (m >= 0) mask = p.mask + m * p.ld_mask;
        }

        Counts<GRAD> counts{table, p.wide};
        if (len > 0) {
            const int words = GRAD ? (n + 31) / 32 : (p.wide ? n : (n + 1) / 2);
            for (int i = tid; i < words; i += kAdjThreads) table[i] = 0u;
        }
        if (mask) {
            const int words = (n + 31) / 32;
            for (int i = tid; i < words + 1; i += kAdjThreads) mask_words[i] = i < words ? __ldg(mask + e0 / 32 + i) : 0u;
        }
        if (tid == 0) n_bias = 0;
        __syncthreads();

        for_each_id(hist, len, [&](int id, int at) {
            const int i = (int)((unsigned)id - (unsigned)e0);
            if ((unsigned)i < (unsigned)n && id >= 0) counts.mark(i, at >= prompt);
            else if (id >= p.V) bad = true;
        });
        if constexpr (!GRAD) {
            for (int j = tid; j < p.M; j += kAdjThreads) {
                const int id = p.bias_idx[(int64_t)row * p.M + j];
                const int i = (int)((unsigned)id - (unsigned)e0);
                if (id >= p.V) bad = true;
                else if (id >= 0 && (unsigned)i < (unsigned)n) {
                    const float b = p.bias_val[(int64_t)row * p.M + j];
                    if (b < INFINITY) biases[atomicAdd(&n_bias, 1)] = make_int2(i, j);
                    else bad = true;   // NaN or +inf
                }
            }
        }
        if constexpr (!INPLACE) cp_async_wait<0>();
        __syncthreads();

        // one logit, from what it was; count: a field of claim()
        char *const held = INPLACE ? out : stage + ((size_t)(in.head + e0) - (size_t)ga * E) * ES;   // element 0 of the slice
        auto change = [&](int i, uint32_t count, float bias) {
            float v = load_elem<F32>(held, i);
            if constexpr (GRAD) {
                const float z = load_elem<F32>(p.z, row * p.ld_z + e0 + i);
                v = z > 0.f ? __fdiv_rn(v, rep) : __fmul_rn(v, rep);
            } else {
                if (count) v = v > 0.f ? __fdiv_rn(v, rep) : __fmul_rn(v, rep);
                const uint32_t c = count & 0x7fffffffu;
                if (c) v = __fsub_rn(__fsub_rn(v, __fmul_rn(freq, __uint2float_rn(c))), pres);
                v = bias > -INFINITY ? __fadd_rn(v, bias) : -INFINITY;
            }
            store_elem<F32>(held, i, v);
        };
        if constexpr (!GRAD) {
            // of equal tokens' biases the last one counts; its thread changes the logit as a whole
            for (int a = tid; a < n_bias; a += kAdjThreads) {
                const int2 mine = biases[a];
                bool last = true;
                for (int b = 0; b < n_bias; ++b) last = last && !(biases[b].x == mine.x && biases[b].y > mine.y);
                if (last) change(mine.x, len > 0 ? counts.claim(mine.x) : 0u, p.bias_val[(int64_t)row * p.M + mine.y]);
            }
            if (p.M > 0) __syncthreads();
        }
        for_each_id(hist, len, [&](int id, int) {
            const int i = (int)((unsigned)id - (unsigned)e0);
            if ((unsigned)i < (unsigned)n && id >= 0) {
                const uint32_t c = counts.claim(i);
                if (c) change(i, c, 0.f);
            }
        });
        __syncthreads();

        // out with it (in place: with what the mask bans)
        if (!INPLACE || mask) {
            const int g0 = (to.head + e0) / E, g1 = (int)(((int64_t)to.head + e0 + n + E - 1) / E);
            const int shift = INPLACE ? 0 : (int)((held - stage) + ((int64_t)g0 * E - to.head - e0) * ES);   // stage byte of g0
            const bool aligned = (shift & 15) == 0;
            for (int g = g0 + tid; g < g1; g += kAdjThreads) {
                const int i0 = to.first(g) - e0;                     // of the slice
                const bool whole = i0 >= 0 && i0 <= n - E;
                uint32_t allow = 0xffffffffu;
                if (mask) {
                    const int at = max(i0, 0);
                    allow = __funnelshift_r(mask_words[at >> 5], mask_words[(at >> 5) + 1], at & 31);
                    if (i0 < 0) allow <<= -i0;
                }
                if (INPLACE && (allow & ((1u << E) - 1u)) == (1u << E) - 1u) continue;
                uint4 *const dst = reinterpret_cast<uint4 *>(const_cast<char *>(to.base) + (size_t)g * 16);
                if (whole && (!INPLACE || (allow & ((1u << E) - 1u)) == 0u)) {
                    uint4 v = make_uint4(0u, 0u, 0u, 0u);
                    if constexpr (!INPLACE) v = load_anywhere<F32>(stage, shift + (g - g0) * 16, aligned);
                    if (mask) {
                        uint32_t *w = reinterpret_cast<uint32_t *>(&v);
#pragma unroll
                        for (int k = 0; k < 4; ++k) {
                            if constexpr (F32) {
                                if (!(allow >> k & 1u)) w[k] = kBanned;
                            } else {
                                if (!(allow >> (2 * k) & 1u)) w[k] = (w[k] & 0xffff0000u) | kBanned;
                                if (!(allow >> (2 * k + 1) & 1u)) w[k] = (w[k] & 0xffffu) | kBanned << 16;
                            }
                        }
                    }
                    *dst = v;
                } else {
#pragma unroll
                    for (int j = 0; j < E; ++j) {
                        const int i = i0 + j;
                        if ((unsigned)i >= (unsigned)n) continue;
                        const bool ok = allow >> j & 1u;
                        if (INPLACE && ok) continue;
                        if constexpr (F32) reinterpret_cast<uint32_t *>(dst)[j] = ok ? reinterpret_cast<const uint32_t *>(held)[i] : kBanned;
                        else reinterpret_cast<uint16_t *>(dst)[j] = ok ? reinterpret_cast<const uint16_t *>(held)[i] : (uint16_t)kBanned;
                    }
                }
            }
        }
        __syncthreads();
    }
    if (bad && p.status) atomicOr(p.status, kStatusBadToken);
}

// ------------------------------------------------------------------ host
// Two areas of rows that are the same, lie beside one another, or (equally far apart) between one another's rows.
bool bad_overlap(const void *a, int64_t lda, const void *b, int64_t ldb, int rows, int V, int bytes)
{
    const uintptr_t a0 = reinterpret_cast<uintptr_t>(a), b0 = reinterpret_cast<uintptr_t>(b);
    const uintptr_t a1 = a0 + (uintptr_t)((rows - 1) * lda + V) * bytes, b1 = b0 + (uintptr_t)((rows - 1) * ldb + V) * bytes;
    if (a0 == b0 && (rows == 1 || lda == ldb)) return false;
    if (!(a0 < b1 && b0 < a1)) return false;
    if (rows == 1 || lda != ldb) return true;
    const uintptr_t step = (uintptr_t)lda * bytes, row = (uintptr_t)V * bytes;
    const uintptr_t behind = b0 >= a0 ? (b0 - a0) % step : (step - (a0 - b0) % step) % step;
    return behind < row || behind > step - row;
}

bool bad_rows(const void *p, int64_t ld, int V, int bytes)
{
    return !p || reinterpret_cast<uintptr_t>(p) % bytes || ld < V;
}

size_t adjust_smem(const AdjustParams &p, bool grad, bool in_place, int es)
{
    const size_t S = (size_t)p.S;
    size_t n = in_place ? 0 : S * es + 32;
    if (p.hist) n += grad ? S / 8 : S * (p.wide ? 4 : 2);
    if (p.mask) n += S / 8 + 8;
    return n + (size_t)p.M * 8;
}

template <bool F32, bool GRAD, bool INPLACE>
cudaError_t launch_adjust(AdjustParams p, cudaStream_t st)
{
    p.wide = p.L >= kNarrowHist;
    // Slices as large as 16384 tokens where the rows fill the GPU twice over, so that few CTAs read a row's history.
    int sms = 0, dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e == cudaSuccess) e = cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev);
    if (e != cudaSuccess) return e;
    p.S = 16384;
    while (p.S > 2048 && (int64_t)p.B * (((int64_t)p.V + p.S - 1) / p.S) < 2 * sms) p.S /= 2;
    p.slices = (int)(((int64_t)p.V + p.S - 1) / p.S);
    const size_t smem = adjust_smem(p, GRAD, INPLACE, RowElem<F32>::kBytes);
    e = allow_smem<adjust_kernel<F32, GRAD, INPLACE>>(kMaxAdjSmem);
    if (e != cudaSuccess) return e;
    const int64_t units = (int64_t)p.B * p.slices;
    adjust_kernel<F32, GRAD, INPLACE><<<(unsigned)std::min<int64_t>(units, INT_MAX), kAdjThreads, smem, st>>>(p);
    return cudaGetLastError();
}

// What both calls have in common.
sats_status check_adjust(const AdjustParams &p, int n_masks, int bytes)
{
    if (p.B < 0 || p.V < 1 || p.L < 0 || p.M < 0 || n_masks < 0 || p.ld_z < p.V || p.ld_hist < 0) return SATS_EINVAL;
    if (p.V > INT_MAX - 64 || p.B > INT_MAX / kRowMaxCluster || p.L > 1 << 30 || p.M > kMaxBiases) return SATS_ESHAPE;
    if (std::max({p.ld_z, p.ld_src, p.ld_out, p.ld_hist, p.ld_mask}) > (int64_t)1 << 40) return SATS_ESHAPE;
    if (p.B == 0) return SATS_OK;
    if (bad_rows(p.z, p.ld_z, p.V, bytes) || bad_rows(p.src, p.ld_src, p.V, bytes) || bad_rows(p.out, p.ld_out, p.V, bytes))
        return SATS_EINVAL;
    if (p.mask && (p.ld_mask < (p.V + 31) / 32 || (!p.mask_row && n_masks < p.B))) return SATS_EINVAL;
    if ((p.mask_row && !p.mask) || (p.M > 0 && (!p.bias_idx || !p.bias_val))) return SATS_EINVAL;
    if (!p.hist && p.L > 0) return SATS_EINVAL;
    if (bad_overlap(p.src, p.ld_src, p.out, p.ld_out, p.B, p.V, bytes)) return SATS_EINVAL;
    if (p.z != p.src && bad_overlap(p.z, p.ld_z, p.out, p.ld_out, p.B, p.V, bytes)) return SATS_EINVAL;
    return SATS_OK;
}

template <bool F32>
sats_status adjust(const void *logits, int64_t ld, int B, int V, const int32_t *hist, int64_t ld_hist, int L,
                   const int32_t *hist_len, const int32_t *n_prompt, const float *rep, const float *pres,
                   const float *freq, const int32_t *bias_idx, const float *bias_val, int M, const void *mask,
                   int64_t ld_mask, int n_masks, const int32_t *mask_row, void *out, int64_t ld_out,
                   int32_t *dev_status, void *stream)
{
    AdjustParams p{};
    p.src = p.z = logits; p.ld_src = p.ld_z = ld; p.out = out; p.ld_out = ld_out; p.B = B; p.V = V;
    p.hist = hist; p.ld_hist = ld_hist; p.L = L; p.hist_len = hist_len; p.n_prompt = n_prompt;
    p.rep = rep; p.pres = pres; p.freq = freq; p.bias_idx = bias_idx; p.bias_val = bias_val; p.M = M;
    p.mask = static_cast<const uint32_t *>(mask); p.ld_mask = ld_mask; p.n_masks = n_masks; p.mask_row = mask_row;
    p.status = dev_status;
    const sats_status s = check_adjust(p, n_masks, RowElem<F32>::kBytes);
    if (s != SATS_OK || B == 0) return s;
    if (L == 0) p.hist = nullptr;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    const cudaError_t e = out == logits ? launch_adjust<F32, false, true>(p, st) : launch_adjust<F32, false, false>(p, st);
    return e == cudaSuccess ? SATS_OK : cuda_fail(e, "adjusted logits kernel launch");
}

template <bool F32>
sats_status adjust_grad(const void *logits, int64_t ld, int B, int V, const int32_t *hist, int64_t ld_hist, int L,
                        const int32_t *hist_len, const float *rep, const void *mask, int64_t ld_mask, int n_masks,
                        const int32_t *mask_row, const void *dout, int64_t ld_dout, void *dlogits, int64_t ld_d,
                        int32_t *dev_status, void *stream)
{
    AdjustParams p{};
    p.z = logits; p.ld_z = ld; p.src = dout; p.ld_src = ld_dout; p.out = dlogits; p.ld_out = ld_d; p.B = B; p.V = V;
    p.hist = hist; p.ld_hist = ld_hist; p.L = L; p.hist_len = hist_len; p.rep = rep;
    p.mask = static_cast<const uint32_t *>(mask); p.ld_mask = ld_mask; p.n_masks = n_masks; p.mask_row = mask_row;
    p.status = dev_status;
    const sats_status s = check_adjust(p, n_masks, RowElem<F32>::kBytes);
    if (s != SATS_OK || B == 0) return s;
    if (L == 0 || !rep) p.hist = nullptr;
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    const cudaError_t e = dlogits == dout ? launch_adjust<F32, true, true>(p, st) : launch_adjust<F32, true, false>(p, st);
    return e == cudaSuccess ? SATS_OK : cuda_fail(e, "adjusted logits gradient kernel launch");
}

}  // namespace
}  // namespace sats

extern "C" {

sats_status sats_adjust_logits(const void *logits, int64_t ld, int B, int V, const int32_t *hist, int64_t ld_hist, int L,
                               const int32_t *hist_len, const int32_t *n_prompt, const float *repetition,
                               const float *presence, const float *frequency, const int32_t *bias_idx,
                               const float *bias_val, int M, const void *mask, int64_t ld_mask, int n_masks,
                               const int32_t *mask_row, void *out, int64_t ld_out, int32_t *dev_status, void *stream)
{
    return sats::adjust<false>(logits, ld, B, V, hist, ld_hist, L, hist_len, n_prompt, repetition, presence, frequency,
                               bias_idx, bias_val, M, mask, ld_mask, n_masks, mask_row, out, ld_out, dev_status, stream);
}

sats_status sats_adjust_logits_f32(const float *logits, int64_t ld, int B, int V, const int32_t *hist, int64_t ld_hist,
                                   int L, const int32_t *hist_len, const int32_t *n_prompt, const float *repetition,
                                   const float *presence, const float *frequency, const int32_t *bias_idx,
                                   const float *bias_val, int M, const void *mask, int64_t ld_mask, int n_masks,
                                   const int32_t *mask_row, float *out, int64_t ld_out, int32_t *dev_status,
                                   void *stream)
{
    return sats::adjust<true>(logits, ld, B, V, hist, ld_hist, L, hist_len, n_prompt, repetition, presence, frequency,
                              bias_idx, bias_val, M, mask, ld_mask, n_masks, mask_row, out, ld_out, dev_status, stream);
}

sats_status sats_adjust_logits_grad(const void *logits, int64_t ld, int B, int V, const int32_t *hist, int64_t ld_hist,
                                    int L, const int32_t *hist_len, const float *repetition, const void *mask,
                                    int64_t ld_mask, int n_masks, const int32_t *mask_row, const void *dout,
                                    int64_t ld_dout, void *dlogits, int64_t ld_d, int32_t *dev_status, void *stream)
{
    return sats::adjust_grad<false>(logits, ld, B, V, hist, ld_hist, L, hist_len, repetition, mask, ld_mask, n_masks,
                                    mask_row, dout, ld_dout, dlogits, ld_d, dev_status, stream);
}

sats_status sats_adjust_logits_grad_f32(const float *logits, int64_t ld, int B, int V, const int32_t *hist,
                                        int64_t ld_hist, int L, const int32_t *hist_len, const float *repetition,
                                        const void *mask, int64_t ld_mask, int n_masks, const int32_t *mask_row,
                                        const float *dout, int64_t ld_dout, float *dlogits, int64_t ld_d,
                                        int32_t *dev_status, void *stream)
{
    return sats::adjust_grad<true>(logits, ld, B, V, hist, ld_hist, L, hist_len, repetition, mask, ld_mask, n_masks,
                                   mask_row, dout, ld_dout, dlogits, ld_d, dev_status, stream);
}

}  // extern "C"
