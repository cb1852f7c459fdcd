// adjust.cu -- penalties for repeated tokens, biases and masks on rows of logits (sats_adjust_logits), and the gradient
// of that (sats_adjust_logits_grad).
//
// A CTA has a slice of a row, up to 2048 of the output's 16-byte vectors.  While its logits arrive in shared memory, it
// reads the row's history and counts, in a table in shared memory, the ids that fall into the slice (whole numbers: they
// do not depend on an order); whoever counts a token first puts it on a list.  The listed logits are changed in shared
// memory, each by one thread, from the logit as it came and in fp32, rounded once; then the slice goes out with the
// mask's bits applied on the way.  So a row is read and written once, in whole vectors, whatever is changed in it; in
// place only what changes is touched.  What is read is asked for at the start, the ids as soon as the row's settings and
// length say which: a CTA's life is one wait for the row's vectors and three barriers, and three CTAs to an SM keep the
// memory busy.  (Ids asked for before the settings are there, up to the histories' capacity: 256 rows 1 us less, a gradient of
// 1024 rows as well; but then histories that do not count are read.)
//
// Bound by HBM for the gradient of many rows (1024 rows of 128256 bf16 logits 89.5 us, 5.9 TB/s); by the instructions and waits
// of a slice where every slice has thousands of ids to look at (256 rows of 151936 bf16 logits with 4096 ids 50 us, 3.1
// TB/s; 77 rows of 50001 fp32 logits with 30000 ids 43 us); by the chain settings and ids - table - logits for few rows (one
// row with 2000 ids 3.2 us).  Times of the GPU alone, from graphs.  256 threads to a CTA: 512, with slices of 2 to 4 vectors a
// thread, took 57 to 70 us for the 256 rows and 105 to 132 for the gradient.
// Other ways, measured on 256 rows / on the gradient of 1024 (us): every slice reads what it needs when it needs it, and
// the ids twice 69 / 183; one kernel that moves the rows and one of a CTA a row that changes single logits behind it, ids in a
// hash table 54 / 107, by bits and their running counts 47 / 115 (each read and written in a sector of 32 bytes); a cluster a
// row, one CTA of which counts 105 / 131; a cluster whose CTAs count the ids once, through distributed shared memory 99 /
// 172; slices that go over their tables in place of lists 63 / 105; CTAs that stay, the next slice arriving meanwhile 65 / 125.
#include <algorithm>
#include <climits>
#include <cuda_bf16.h>

#include "internal.h"
#include "rows.cuh"

namespace sats {
namespace {

constexpr int kAdjThreads = 256;
constexpr int kMostEach = 8;           // vectors of a slice per thread
constexpr int kKeep = 2;               // vectors of ids of a thread that are asked for at the start
constexpr int kMaxBiases = 1024, kBiasEach = kMaxBiases / kAdjThreads;
constexpr int kNarrowHist = 1 << 14;   // histories shorter than this fit 16-bit fields
constexpr size_t kMaxAdjSmem = 68 * 1024;   // three CTAs to an SM, with the kernel's static part

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
    int each, slices;        // vectors of a slice per thread; slices of a row
    int listed;              // places of the list
    bool wide;               // 32-bit fields
};

__device__ __forceinline__ const uint32_t *row_mask(const AdjustParams &p, int row, bool *bad)
{
    if (!p.mask) return nullptr;
    const int m = p.mask_row ? p.mask_row[row] : row;
    if (m >= p.n_masks) *bad = true;
    return m >= 0 && m < p.n_masks ? p.mask + m * p.ld_mask : nullptr;
}

// Bits of 8 tokens from f on, from mask words of which the first is word w0; f may lie before 0.
__device__ __forceinline__ uint32_t staged_bits(const uint32_t *words, int w0, int f)
{
    const int at = max(f, 0);
    const uint32_t *const w = words + ((at >> 5) - w0);
    return __funnelshift_r(w[0], w[1], at & 31) << (at - f);
}

// The vector of ids at place v of a history: its positions 4 v - lead.. where they are below n (others: -1).
__device__ __forceinline__ int4 load_ids(const int32_t *p, int lead, int v, int n)
{
    const int at = 4 * v - lead;
    if (at >= 0 && at <= n - 4) return __ldg(reinterpret_cast<const int4 *>(p - lead) + v);
    int4 q = make_int4(-1, -1, -1, -1);
    if (at >= 0 && at < n) q.x = __ldg(p + at);
    if (at + 1 >= 0 && at + 1 < n) q.y = __ldg(p + at + 1);
    if (at + 2 >= 0 && at + 2 < n) q.z = __ldg(p + at + 2);
    if (at + 3 >= 0 && at + 3 < n) q.w = __ldg(p + at + 3);
    return q;
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

// A setting of the row; outside its range it is off and noted.
__device__ __forceinline__ float checked(float v, float off, bool positive, bool *bad)
{
    if (isfinite(v) && (!positive || v > 0.f)) return v;
    *bad = true;
    return off;
}

// 4 (fp32) or 8 (bf16) elements at byte `off` of shared memory, wherever that is.
template <bool F32>
__device__ __forceinline__ uint4 load_anywhere(const char *stage, int off)
{
    if ((off & 15) == 0) return *reinterpret_cast<const uint4 *>(stage + off);
    const uint32_t *p = reinterpret_cast<const uint32_t *>(stage + (off & ~3));
    const uint32_t a = p[0], b = p[1], c = p[2], d = p[3];
    if (F32 || (off & 2) == 0) return make_uint4(a, b, c, d);
    const uint32_t e = p[4];
    return make_uint4(__funnelshift_r(a, b, 16), __funnelshift_r(b, c, 16), __funnelshift_r(c, d, 16),
                      __funnelshift_r(d, e, 16));
}

// A logit or gradient that one's token scales.
__device__ __forceinline__ float scaled(float v, float z, float rep) { return z > 0.f ? __fdiv_rn(v, rep) : __fmul_rn(v, rep); }

// A logit with its token's field (bit 31: in the prompt, bit 30: has a bias, below: times generated), then its bias.
__device__ __forceinline__ float penalised(float v, uint32_t f, float rep, float freq, float pres)
{
    const uint32_t made = f & 0x3fffffffu;
    if (f & ~0x40000000u) v = scaled(v, v, rep);
    if (made) v = __fsub_rn(__fsub_rn(v, __fmul_rn(freq, __uint2float_rn(made))), pres);
    return v;
}
__device__ __forceinline__ float biased(float v, float add) { return add > -INFINITY ? __fadd_rn(v, add) : -INFINITY; }

// A vector with what its bits do not allow banned.
template <bool F32, bool GRAD>
__device__ __forceinline__ uint4 ban(const uint4 &v, uint32_t allow)
{
    constexpr uint32_t kBanned = GRAD ? 0u : (F32 ? 0xff800000u : 0xff80u);
    uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        if constexpr (F32) {
            if (!(allow >> i & 1u)) w[i] = kBanned;
        } else {
            if (!(allow >> (2 * i) & 1u)) w[i] = (w[i] & 0xffff0000u) | kBanned;
            if (!(allow >> (2 * i + 1) & 1u)) w[i] = (w[i] & 0xffffu) | kBanned << 16;
        }
    }
    return make_uint4(w[0], w[1], w[2], w[3]);
}

// Vector g of a row element by element (src: its first one's value); in place only what is banned.
template <bool F32, bool GRAD, bool INPLACE>
__device__ __forceinline__ void store_edge(const Row<F32> &to, int g, const char *src, uint32_t allow)
{
    constexpr int E = RowElem<F32>::kPer;
    constexpr uint32_t kBanned = GRAD ? 0u : (F32 ? 0xff800000u : 0xff80u);
    char *const dst = const_cast<char *>(to.base) + (size_t)g * 16;
#pragma unroll
    for (int j = 0; j < E; ++j) {
        const bool ok = allow >> j & 1u;
        if (!to.inside(to.first(g) + j) || (INPLACE && ok)) continue;
        if constexpr (F32) reinterpret_cast<uint32_t *>(dst)[j] = ok ? reinterpret_cast<const uint32_t *>(src)[j] : kBanned;
        else reinterpret_cast<uint16_t *>(dst)[j] = ok ? reinterpret_cast<const uint16_t *>(src)[j] : (uint16_t)kBanned;
    }
}

// The slice's table.  Forward: a field for each token, of 16 or (wide) 32 bits: the top bit for "in the prompt", the next for
// "has a bias", the others the number of times it was generated.  Gradient: a bit for each token.
template <bool GRAD>
struct Table {
    uint32_t *w;
    bool wide;

    __device__ __forceinline__ int words(int n) const { return GRAD ? (n + 31) / 32 : (wide ? n : (n + 1) / 2); }
    // Adds or (bit) sets; whether the token was not in the table yet.
    __device__ __forceinline__ bool generated(int i)
    {
        if (wide) return atomicAdd(w + i, 1u) == 0u;
        const int sh = 16 * (i & 1);
        return (atomicAdd(w + (i >> 1), 1u << sh) >> sh & 0xffffu) == 0u;
    }
    __device__ __forceinline__ bool set(int i, uint32_t bit)   // bit: 2 the prompt's, 1 the bias'
    {
        if constexpr (GRAD) return !(atomicOr(w + (i >> 5), 1u << (i & 31)) >> (i & 31) & 1u);
        if (wide) return atomicOr(w + i, bit << 30) == 0u;
        const int sh = 16 * (i & 1);
        return (atomicOr(w + (i >> 1), bit << (14 + sh)) >> sh & 0xffffu) == 0u;
    }
    // Bit 31: the prompt's, bit 30: the bias', below: the count.
    __device__ __forceinline__ uint32_t field(int i) const
    {
        if (wide) return w[i];
        const uint32_t f = w[i >> 1] >> 16 * (i & 1) & 0xffffu;
        return f >> 14 << 30 | (f & 0x3fffu);
    }
};

template <bool F32, bool GRAD, bool INPLACE>
__global__ void __launch_bounds__(kAdjThreads, GRAD ? 6 : 4) adjust_kernel(const __grid_constant__ AdjustParams p)
{
    constexpr int ES = RowElem<F32>::kBytes, E = RowElem<F32>::kPer;
    constexpr uint32_t kAll = (1u << E) - 1u;
    extern __shared__ __align__(16) char smem[];
    __shared__ uint32_t mask_words[kAdjThreads * kMostEach * E / 32 + 2];
    __shared__ uint16_t aside[kAdjThreads * 4 * kKeep];   // token of the slice, bit 15: of the prompt
    __shared__ int n_listed, n_bias;
    const int tid = threadIdx.x;
    const int vectors = kAdjThreads * p.each, S = vectors * E;   // of a slice
    char *const stage = smem;
    Table<GRAD> table{reinterpret_cast<uint32_t *>(smem + (INPLACE ? 0 : vectors * 16 + 32)), p.wide};
    const int table_words = p.hist || p.M > 0 ? table.words(S) : 0;
    uint16_t *const list = reinterpret_cast<uint16_t *>(table.w + table_words);
    uint32_t *const biases = reinterpret_cast<uint32_t *>(list + p.listed);   // token << 16 | place in the row's list
    bool bad = false;

    const int64_t units = (int64_t)p.B * p.slices;
    for (int64_t u = blockIdx.x; u < units; u += gridDim.x) {
        const int row = (int)(u / p.slices);
        const int gs = (int)(u - (int64_t)row * p.slices) * vectors;   // the slice's first vector
        const Row<F32> in(p.src, row, p.ld_src, p.V), to(p.out, row, p.ld_out, p.V);
        const int ge = min(to.G, gs + vectors);
        const int base = to.first(gs);                                  // token i of the slice is base + i of the row
        const int e0 = max(base, 0), e1 = (int)min((int64_t)p.V, (int64_t)base + S);
        if (gs >= ge) continue;

        // ---- what is read, all of it but the ids asked for before anything is looked at
        const int ga = (in.head + e0) / E;                              // byte 0 of the stage
        if constexpr (!INPLACE) {
            const int gb = (int)(((int64_t)in.head + e1 + E - 1) / E);
            const int g0 = in.whole(ga) ? ga : ga + 1, g1 = in.whole(gb - 1) ? gb : gb - 1;   // a row's ends may be parts of vectors
            const char *from = in.base + (size_t)(g0 + tid) * 16;
            char *at = stage + (g0 - ga + tid) * 16;
            for (int g = g0 + tid; g < g1; g += kAdjThreads, from += kAdjThreads * 16, at += kAdjThreads * 16) cp_async16(at, from);
            if (tid == 0 && g0 > ga) *reinterpret_cast<uint4 *>(stage) = load_edge_granule<F32>(in.base, in.first(ga), in.V, ga);
            if (tid == 32 && g1 < gb && gb - 1 >= g0)
                *reinterpret_cast<uint4 *>(stage + (gb - 1 - ga) * 16) = load_edge_granule<F32>(in.base, in.first(gb - 1), in.V, gb - 1);
            cp_async_commit();
        }
        float rep = p.rep ? p.rep[row] : 1.f;
        float pres = !GRAD && p.pres ? p.pres[row] : 0.f;
        float freq = !GRAD && p.freq ? p.freq[row] : 0.f;
        int len = p.hist ? (p.hist_len ? p.hist_len[row] : p.L) : 0;
        const int prompt = !GRAD && p.n_prompt ? p.n_prompt[row] : 0;
        int bias_id[kBiasEach];
        float bias_add[kBiasEach];
        if constexpr (!GRAD) {
#pragma unroll
            for (int k = 0; k < kBiasEach; ++k) {
                bias_id[k] = -1;
                if (tid + k * kAdjThreads < p.M) {
                    bias_id[k] = p.bias_idx[(int64_t)row * p.M + tid + k * kAdjThreads];
                    bias_add[k] = p.bias_val[(int64_t)row * p.M + tid + k * kAdjThreads];
                }
            }
        }
        const uint32_t *const mask = row_mask(p, row, &bad);

        for (int i = tid; i < table_words / 4; i += kAdjThreads) reinterpret_cast<uint4 *>(table.w)[i] = make_uint4(0u, 0u, 0u, 0u);
        if (tid == 0) n_listed = n_bias = 0;
        rep = checked(rep, 1.f, true, &bad);
        pres = checked(pres, 0.f, false, &bad);
        freq = checked(freq, 0.f, false, &bad);
        if (len < 0 || len > p.L) {
            bad = true;
            len = len < 0 ? 0 : p.L;
        }
        if (rep == 1.f && pres == 0.f && freq == 0.f) len = 0;   // nothing would change
        // ids: of a row that has settings, as many as count, and nothing else of the history
        const int32_t *const hist = p.hist ? p.hist + row * p.ld_hist : nullptr;
        const int lead = (int)((reinterpret_cast<uintptr_t>(hist) >> 2) & 3);   // ids between the vector boundary and the first
        int4 ids[kKeep];
#pragma unroll
        for (int k = 0; k < kKeep; ++k) ids[k] = load_ids(hist, lead, tid + k * kAdjThreads, len);
        const int w0 = e0 >> 5;
        if (mask) {
            const int n = ((e1 - 1) >> 5) - w0 + 1;
            for (int i = tid; i < n; i += kAdjThreads) cp_async4(mask_words + i, mask + w0 + i);
            cp_async_commit();
        }
        __syncthreads();

        // ---- which tokens, how often
        // A thread puts the few of its ids that fall into the slice aside; a warp then enters as many at a time as its lanes
        // have, instead of at every id the one lane in ten that has one.
        const uint32_t here = (uint32_t)(e1 - e0), low = (uint32_t)e0;
        const int skew = e0 - base;
        uint16_t *const mine = aside + tid;
        int n_aside = 0;
        const auto look = [&](int id, bool early) {   // (an absent id is below 0)
            const uint32_t i = (uint32_t)id - low;
            if (i < here) {
                mine[n_aside * kAdjThreads] = (uint16_t)((i + skew) | (early ? 0x8000u : 0u));
                ++n_aside;
            }
        };
        const auto enter = [&] {
            for (int k = 0; __any_sync(0xffffffffu, k < n_aside); ++k) {
                if (k >= n_aside) continue;
                const uint32_t x = mine[k * kAdjThreads];
                const int i = (int)(x & 0x7fffu);
                if (GRAD || (x & 0x8000u) ? table.set(i, 2u) : table.generated(i)) list[atomicAdd(&n_listed, 1)] = (uint16_t)i;
            }
            n_aside = 0;
        };
        const bool last_slice = e1 == p.V;   // looks for ids that are no tokens
        const auto look4 = [&](const int4 &q, int at) {
            look(q.x, at < prompt);
            look(q.y, at + 1 < prompt);
            look(q.z, at + 2 < prompt);
            look(q.w, at + 3 < prompt);
            if (last_slice) bad = bad || max(max(q.x, q.y), max(q.z, q.w)) >= p.V;
        };
        const int id_vectors = len > 0 ? (int)(((int64_t)len + lead + 3) >> 2) : 0;
        // the vectors that lie wholly in the history, then (one thread each) what is before and behind them
        const int whole0 = lead > 0 ? 1 : 0, whole1 = (int)(((int64_t)len + lead) >> 2);
        const int4 *const vectors4 = reinterpret_cast<const int4 *>(hist - lead);
        for (int v0 = tid & ~31; v0 < id_vectors; v0 += kKeep * kAdjThreads) {   // (the same turns for a whole warp)
            const int v1 = v0 + (tid & 31);
            if (v0 > 0 && v0 >= kKeep * kAdjThreads) {
#pragma unroll
                for (int k = 0; k < kKeep; ++k) {
                    const int v = v1 + k * kAdjThreads;
                    ids[k] = v >= whole0 && v < whole1 ? __ldg(vectors4 + v) : make_int4(-1, -1, -1, -1);
                }
            }
#pragma unroll
            for (int k = 0; k < kKeep; ++k) {
                const int v = v1 + k * kAdjThreads;
                if (v >= whole0 && v < whole1) look4(ids[k], 4 * v - lead);
                else if (v < id_vectors) look4(load_ids(hist, lead, v, len), 4 * v - lead);
            }
            enter();
        }
        if constexpr (!GRAD) {
#pragma unroll
            for (int k = 0; k < kBiasEach; ++k) {
                const int id = bias_id[k];
                if (id < 0) continue;
                if (id >= p.V || !(bias_add[k] < INFINITY)) bad = true;   // no token, NaN or +inf
                else if (id >= e0 && id < e1) {
                    if (table.set(id - base, 1u)) list[atomicAdd(&n_listed, 1)] = (uint16_t)(id - base);
                    biases[atomicAdd(&n_bias, 1)] = (uint32_t)(id - base) << 16 | (uint32_t)(tid + k * kAdjThreads);
                }
            }
        }
        cp_async_wait<0>();
        __syncthreads();

        // ---- the listed logits; element 0 of the slice lies at byte `first` of the stage (in place: of the row)
        const int64_t out = row * p.ld_out + base;
        const int first = (in.head + base - ga * E) * ES;   // (may lie before it, if the slice begins before the row)
        if (n_listed > 0) {
            const auto change = [&](int i, bool has_bias, float add) {
                char *const at = INPLACE ? static_cast<char *>(p.out) + (out + i) * ES : stage + first + i * ES;
                float v = load_elem<F32>(at, 0);
                if constexpr (GRAD) v = scaled(v, load_elem<F32>(p.z, row * p.ld_z + base + i), rep);
                else v = penalised(v, table.field(i), rep, freq, pres);
                store_elem<F32>(at, 0, has_bias ? biased(v, add) : v);
            };
            for (int k = tid; k < n_listed; k += kAdjThreads) {
                const int i = list[k];
                if (GRAD || !(table.field(i) & 0x40000000u)) change(i, false, 0.f);
            }
            if constexpr (!GRAD) {
                // of equal tokens' biases the last one counts; its thread changes the logit as a whole
                for (int a = tid; a < n_bias; a += kAdjThreads) {
                    const uint32_t mine = biases[a];
                    bool last = true;
                    for (int b = 0; b < n_bias; ++b) last = last && !(biases[b] > mine && (biases[b] ^ mine) < 65536u);
                    if (last) change((int)(mine >> 16), true, p.bias_val[(int64_t)row * p.M + (mine & 0xffffu)]);
                }
            }
            __syncthreads();
        }

        // ---- out with it (in place: with what the mask bans)
        if (!INPLACE || mask) {
            const int g0 = to.whole(gs) ? gs : gs + 1, g1 = to.whole(ge - 1) ? ge : ge - 1;
            const int shift = first + (to.first(gs) - base) * ES;   // stage byte of vector gs
            uint4 *dst = reinterpret_cast<uint4 *>(const_cast<char *>(to.base) + (size_t)(g0 + tid) * 16);
            int held = shift + (g0 - gs + tid) * 16, f = to.first(g0 + tid);
            for (int g = g0 + tid; g < g1; g += kAdjThreads, dst += kAdjThreads, held += kAdjThreads * 16, f += kAdjThreads * E) {
                uint4 v = make_uint4(0u, 0u, 0u, 0u);
                if constexpr (!INPLACE) v = load_anywhere<F32>(stage, held);
                if (mask) {
                    const uint32_t allow = staged_bits(mask_words, w0, f);
                    if (INPLACE && (allow & kAll) != 0u) {
                        if ((allow & kAll) != kAll) store_edge<F32, GRAD, true>(to, g, nullptr, allow);
                        continue;
                    }
                    v = ban<F32, GRAD>(v, allow);
                }
                *dst = v;
            }
            if (tid == 0 && g0 > gs)
                store_edge<F32, GRAD, INPLACE>(to, gs, stage + shift, mask ? staged_bits(mask_words, w0, to.first(gs)) : kAll);
            if (tid == 32 && g1 < ge && ge - 1 >= g0)
                store_edge<F32, GRAD, INPLACE>(to, ge - 1, stage + shift + (ge - 1 - gs) * 16,
                                               mask ? staged_bits(mask_words, w0, to.first(ge - 1)) : kAll);
        }
        if (gridDim.x < units) __syncthreads();
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

template <bool F32, bool GRAD, bool INPLACE>
cudaError_t launch_adjust(AdjustParams p, cudaStream_t st)
{
    int sms = 0, dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e == cudaSuccess) e = cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev);
    if (e != cudaSuccess) return e;
    p.wide = p.L >= kNarrowHist;
    const int64_t ids = (int64_t)(p.hist ? p.L : 0) + p.M;
    constexpr int E = RowElem<F32>::kPer;
    const int64_t granules = ((int64_t)p.V + E - 1) / E + 1;   // (a row may begin inside one)
    p.each = kMostEach;
    while (p.each > 1 && (int64_t)p.B * ((granules + kAdjThreads * p.each - 1) / (kAdjThreads * p.each)) < 2 * sms) p.each /= 2;
    size_t smem = 0;
    for (;; --p.each) {
        const size_t S = (size_t)kAdjThreads * p.each * E;
        p.listed = (int)((std::min<int64_t>(ids, S) + 3) / 4 * 4);
        smem = INPLACE ? 0 : S * (16 / E) + 32;
        if (ids > 0) smem += (GRAD ? S / 8 : S * (p.wide ? 4 : 2)) + (size_t)p.listed * 2 + (size_t)p.M * 4;
        if (smem <= kMaxAdjSmem || p.each == 1) break;
    }
    p.slices = (int)((granules + kAdjThreads * p.each - 1) / (kAdjThreads * p.each));
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
    if (p.V > INT_MAX - 64 || p.B > INT_MAX / kRowMaxCluster || p.L >= 1 << 30 || p.M > kMaxBiases) return SATS_ESHAPE;
    if (std::max({p.ld_z, p.ld_src, p.ld_out, p.ld_hist, p.ld_mask}) > (int64_t)1 << 40) return SATS_ESHAPE;
    if (p.B == 0) return SATS_OK;
    if (bad_rows(p.z, p.ld_z, p.V, bytes) || bad_rows(p.src, p.ld_src, p.V, bytes) || bad_rows(p.out, p.ld_out, p.V, bytes))
        return SATS_EINVAL;
    if (p.mask && (p.ld_mask < (p.V + 31) / 32 || (!p.mask_row && n_masks < p.B))) return SATS_EINVAL;
    if ((p.mask_row && !p.mask) || (p.M > 0 && (!p.bias_idx || !p.bias_val))) return SATS_EINVAL;
    if (!p.hist && p.L > 0) return SATS_EINVAL;
    const void *const words[] = {p.hist, p.hist_len, p.n_prompt, p.rep, p.pres, p.freq, p.bias_idx, p.bias_val, p.mask, p.mask_row,
                                 p.status};
    for (const void *w : words)
        if (reinterpret_cast<uintptr_t>(w) % 4) return SATS_EINVAL;
    if (bad_overlap(p.src, p.ld_src, p.out, p.ld_out, p.B, p.V, bytes)) return SATS_EINVAL;
    // (a thread reads its logit and then writes its gradient, others theirs meanwhile: over the logits only if they are
    // what comes in, row for row)
    const bool alike = p.z == p.src && (p.B == 1 || p.ld_z == p.ld_src);
    if (!alike && (p.z == p.out || bad_overlap(p.z, p.ld_z, p.out, p.ld_out, p.B, p.V, bytes))) return SATS_EINVAL;
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
