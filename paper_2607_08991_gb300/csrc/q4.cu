// q4.cu -- 4-bit weights with group scales: the product of rows of activations with them on the tensor cores
// (sats_q4_matmul), their making from bf16 weights and reading back (sats_q4_quantize, sats_q4_dequantize), and the
// handle that keeps them packed (sats_q4_create).
//
// A weight is s q, q a whole number from -8 to 7 and s the bf16 scale of its group of G (32, 64, 128) consecutive k: 11
// significant bits at most, which is what fp16 has.  So the product runs in fp16 MMAs without rounding a weight: every
// column's scales are divided by a power of two (kept beside them) that puts the largest at 2^10..2^11, and every
// token's activations by one that puts the largest at 2^14..2^15; fp32 activations go as two fp16 parts.
//
// The weights are the A operand (128 of them a tile, M) and stay 4 bits wide until they are in registers: warpgroups (two,
// four in the kernel for many tokens) turn a stage of 128 k into fp16 pairs and store them to TMEM, where the MMA reads its
// A operand from; only the activations (N, the tokens) lie in shared memory as the MMA wants them.  Through shared memory
// the fp16 weights would cost four times the bytes that arrive from HBM, written once and read once.
#include <algorithm>
#include <climits>
#include <cuda_fp16.h>
#include <new>

#include "rows.cuh"
#include "tc_common.cuh"

struct sats_q4 {
    int K = 0, N = 0, G = 0, device = 0;
    uint8_t *blk = nullptr;   // [row tiles][stages]: blocks as described at kCodeBytes
    int *col_exp = nullptr;   // [N rounded up to 128]: the power of two that a column's scales were divided by
};

namespace sats {
namespace {
using namespace tc;

constexpr int kRows = 128;                    // columns of the weight matrix in a tile (MMA M)
constexpr int kStageK = 128;                  // k of a stage
constexpr int kCodeBytes = kRows * kStageK / 2;
// A block: for each half of 64 k and each piece of 32 k the 16 bytes of every row (row after row), then the fp16 scales,
// group after group, 128 rows each.
// A word holds 8 codes u = q + 8, those of k = 2p in its low and 2p + 1 in its high half, p = 0..3: bits 6..9, 10..13,
// 2..5 of the half, and for p = 3 bits 14..17 of the word (even) and 30, 31, 0, 1 (odd): as it is and rotated by 8 bits the
// word has every pair at bits 6..9 or 2..5 of its halves, where with the exponent of 1024 they read as fp16 numbers.
constexpr int kMaxK = 65536;
constexpr int64_t kMaxQ4N = (int64_t)1 << 24;
constexpr int kMaxCtas = 320;                 // of the product's kernel
constexpr int kLoShift = 11;                  // the second part of an fp32 activation is kept 2^11 times larger
constexpr int kMaxSplitWaves = 16;            // tiles of more waves are not split: the last, uneven one is 1 of 17 (plan_q4)
constexpr int kMaxSplitTiles = kMaxSplitWaves * kMaxCtas;
constexpr int kDirectTokens = 16;             // columns (fp32 activations: two a token) that a CTA may stage itself
constexpr int kCtlBytes = 256;

__host__ __device__ constexpr int block_bytes(int G) { return kCodeBytes + kStageK / G * kRows * 2; }
__host__ __device__ constexpr int div_up(int a, int b) { return (a + b - 1) / b; }

// ------------------------------------------------------------------ quantising
// amax over the group, s = bf16(amax / 7), q = w / s rounded half to even.  amax / 7 is further than 2^-12 (relative) from
// the middle of two bf16 numbers, so a product with 1 / 7 decides as the division does; w / s is either a tie or further
// than 2^-10 from one (a ratio of two numbers of 8 bits), so a product with 1 / s, off by 2^-20 at most, that is first
// rounded to a multiple of 2^-11 does.  A group with an infinity or a NaN gets the scale NaN and codes 0.
//
// A warp has 128 columns and 16 rows: a thread's 16 x 4 values stay in registers between amax and codes, so W is read
// once; the warps of a group meet in shared memory for its amax.  The codes of two rows are one multiply-add of the whole
// numbers' floating-point bits.  (A 4096 x 14336 layer 29 us, 5.2 TB/s, half of the issue slots taken.)
constexpr int kQuantWarps = 8, kQuantRows = 16, kQuantCols = 128;

// Whether rows of `elems` elements from p on can be read or written in vectors of four elements.
bool in_fours(const void *p, int64_t elems, int elem_bytes)
{
    return reinterpret_cast<uintptr_t>(p) % (4 * elem_bytes) == 0 && elems % 4 == 0;
}

// Four bytes of each lane, for columns n..n + 3 of a row of bytes that starts anywhere; inside: all lanes' columns are there.
__device__ __forceinline__ void store_row_bytes(uint8_t *row, int n, int N, uint32_t v, int lane, bool inside)
{
    // The aligned word that begins `lead` bytes before n: the last bytes of the lane before and the first of this one.
    // What is left at the warp's ends goes out byte by byte.
    const int lead = (int)(reinterpret_cast<uintptr_t>(row + n) & 3u);   // the same in all lanes
    const uint32_t w = __funnelshift_l(__shfl_up_sync(0xffffffffu, v, 1), v, 8 * lead);
    uint8_t *const at = row + (n - lead);
    if ((lane > 0 || lead == 0) && (inside || n - lead + 4 <= N)) *reinterpret_cast<uint32_t *>(at) = w;
    else {
#pragma unroll
        for (int j = 0; j < 4; ++j)
            if ((lane > 0 || j >= lead) && n - lead + j < N) at[j] = (uint8_t)(w >> 8 * j);
    }
    if (lane == 31 && lead > 0) {
#pragma unroll
        for (int j = 1; j < 4; ++j)
            if (j >= 4 - lead && n + j < N) row[n + j] = (uint8_t)(v >> 8 * j);
    }
}

__device__ __forceinline__ float rcp_approx(float x)   // 1 / x to 1 ulp
{
    float y;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

template <bool FOURS, bool OUT4>
__global__ void __launch_bounds__(32 * kQuantWarps, 3) q4_quantize_kernel(const uint16_t *W, int64_t ld, int K, int N, int G,
                                                                       uint8_t *codes, uint16_t *scales)
{
    __shared__ uint32_t tops[kQuantWarps][32][4];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int n = blockIdx.x * kQuantCols + 4 * lane;
    const int per = G / kQuantRows;   // warps of a group
    for (int k0 = (blockIdx.y * kQuantWarps + warp) * kQuantRows; k0 - warp * kQuantRows < K;
         k0 += gridDim.y * kQuantWarps * kQuantRows) {
        uint32_t w[kQuantRows][2];   // columns n, n + 1 and n + 2, n + 3
        const uint16_t *from = W + (int64_t)k0 * ld + n;
        const int rows = K - k0;
        const bool inside = rows >= kQuantRows && (blockIdx.x + 1) * kQuantCols <= N;   // the warp's whole tile
        if (FOURS && inside) {
#pragma unroll
            for (int i = 0; i < kQuantRows; ++i, from += ld) {
                const uint2 q = __ldcs(reinterpret_cast<const uint2 *>(from));
                w[i][0] = q.x;
                w[i][1] = q.y;
            }
        } else {
#pragma unroll
            for (int i = 0; i < kQuantRows; ++i, from += ld) {
                w[i][0] = w[i][1] = 0u;
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    if (i < rows && n + j < N) w[i][j >> 1] |= (uint32_t)from[j] << 16 * (j & 1);
            }
        }
        // magnitudes as whole numbers: they order as the values do, infinities and NaN above
        uint32_t m[2] = {0u, 0u};
#pragma unroll
        for (int i = 0; i < kQuantRows; ++i)
#pragma unroll
            for (int j = 0; j < 2; ++j) m[j] = __vmaxu2(m[j], w[i][j] & 0x7fff7fffu);
        uint32_t top[4] = {m[0] & 0xffffu, m[0] >> 16, m[1] & 0xffffu, m[1] >> 16};
        *reinterpret_cast<uint4 *>(tops[warp][lane]) = make_uint4(top[0], top[1], top[2], top[3]);
        __syncthreads();
        for (int o = warp / per * per; o < (warp / per + 1) * per; ++o) {
            const uint4 t = *reinterpret_cast<const uint4 *>(tops[o][lane]);
            top[0] = max(top[0], t.x);
            top[1] = max(top[1], t.y);
            top[2] = max(top[2], t.z);
            top[3] = max(top[3], t.w);
        }
        __syncthreads();
        if (k0 >= K) continue;
        float s[4], r[4];
        uint16_t sb[4];
        bool slow = false;   // subnormal scales and groups that are not finite
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            sb[j] = top[j] >= 0x7f80u ? 0x7fc0u : bf16_bits(__fmul_rn(__uint_as_float(top[j] << 16), 1.f / 7.f));
            s[j] = __uint_as_float((uint32_t)sb[j] << 16);
            const bool fine = s[j] >= 1.17549435e-38f;
            slow = slow || (!fine && top[j] != 0u);
            r[j] = fine ? rcp_approx(s[j]) : 0.f;
        }
        if (k0 % G == 0) {
            uint16_t *const p = scales + (int64_t)(k0 / G) * N + n;
#pragma unroll
            for (int j = 0; j < 4; ++j)
                if (n + j < N) p[j] = sb[j];
        }
        const f32x2 r01 = pack2(r[0], r[1]), r23 = pack2(r[2], r[3]);
        const f32x2 grid = pack2(6144.f, 6144.f), no_grid = pack2(-6144.f, -6144.f);   // 1.5 x 2^12: multiples of 2^-11
        const f32x2 whole = pack2(12582920.f, 12582920.f);                             // 1.5 x 2^23 + 8: of 1; bits: q + 8
        uint8_t *to = codes + (int64_t)(k0 / 2) * N;
        auto rounded = [&](uint32_t v, f32x2 rr) {
            return fadd2(fadd2(ffma2(bf16x2_to_f32x2(v), rr, grid), no_grid), whole);
        };
        const auto code4 = [&](int i) {   // of rows i and i + 1
            uint32_t b[4];
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                const float2 even = unpack2(rounded(w[i][j], j ? r23 : r01)), odd = unpack2(rounded(w[i + 1][j], j ? r23 : r01));
                b[2 * j] = __float_as_uint(odd.x) * 16u + __float_as_uint(even.x);
                b[2 * j + 1] = __float_as_uint(odd.y) * 16u + __float_as_uint(even.y);
            }
            return __byte_perm(__byte_perm(b[0], b[1], 0x0040), __byte_perm(b[2], b[3], 0x0040), 0x5410) ^ 0x88888888u;
        };
        if (OUT4 && inside && !__any_sync(0xffffffffu, slow)) {
#pragma unroll
            for (int i = 0; i < kQuantRows; i += 2, to += N) __stcs(reinterpret_cast<uint32_t *>(to + n), code4(i));
            continue;
        }
#pragma unroll
        for (int i = 0; i < kQuantRows; i += 2, to += N) {
            if (i >= rows) break;
            uint32_t v = code4(i);
            if (slow) {
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const float sj = s[j];
                    if (sj >= 1.17549435e-38f) continue;
                    uint32_t c = 0;
#pragma unroll
                    for (int o = 0; o < 2; ++o) {
                        const float x = __uint_as_float(w[i + o][j >> 1] >> 16 * (j & 1) << 16);
                        const float q = sj > 0.f ? fminf(fmaxf(rintf(__fdiv_rn(x, sj)), -7.f), 7.f) : 0.f;
                        c |= ((uint32_t)(int)q & 15u) << 4 * o;
                    }
                    v = (v & ~(0xffu << 8 * j)) | c << 8 * j;
                }
            }
            store_row_bytes(to, n, N, v, lane, inside);
        }
    }
}

// Eight bytes of codes of a thread at a time; a nibble's value from the bits of a float.
constexpr int kReadRows = 16;   // of codes, 32 of values: within a group

__device__ __forceinline__ float code_value(uint32_t nibble)   // (what lies above the nibble does not matter)
{
    return __uint_as_float(((nibble & 15u) ^ 8u) | 0x4b000000u) - 8388616.f;
}

template <bool FOURS>
__global__ void __launch_bounds__(256) q4_dequantize_kernel(const uint8_t *codes, const uint16_t *scales, int K, int N, int G,
                                                            float *values)
{
    constexpr int C = FOURS ? 4 : 1;
    const int64_t n = ((int64_t)blockIdx.x * 256 + threadIdx.x) * C;
    if (n >= N) return;
    const int rows = K / 2;
    for (int i0 = blockIdx.y * kReadRows; i0 < rows; i0 += gridDim.y * kReadRows) {
        float s[C];
#pragma unroll
        for (int j = 0; j < C; ++j) s[j] = __uint_as_float((uint32_t)scales[(int64_t)(2 * i0 / G) * N + n + j] << 16);
        const uint8_t *from = codes + (int64_t)i0 * N + n;
        float *to = values + (int64_t)i0 * 2 * N + n;
        const auto code = [&] {
            if constexpr (FOURS) return __ldcs(reinterpret_cast<const uint32_t *>(from));
            else return (uint32_t)__ldcs(from);
        };
        const auto put = [&](uint32_t c) {
#pragma unroll
            for (int o = 0; o < 2; ++o, to += N) {
                float v[C];
#pragma unroll
                for (int j = 0; j < C; ++j) v[j] = code_value(c >> (8 * j + 4 * o)) * s[j];
                if constexpr (FOURS) __stcs(reinterpret_cast<float4 *>(to), make_float4(v[0], v[1], v[2], v[3]));
                else __stcs(to, v[0]);
            }
        };
        if (i0 + kReadRows <= rows) {
            uint32_t c[kReadRows];
#pragma unroll
            for (int i = 0; i < kReadRows; ++i, from += N) c[i] = code();
#pragma unroll
            for (int i = 0; i < kReadRows; ++i) put(c[i]);
        } else
            for (int i = i0; i < rows; ++i, from += N) put(code());
    }
}

// ------------------------------------------------------------------ packing
// The power of two of each column: its largest finite scale becomes 2^10..2^11 (64 times what the block holds).
__global__ void __launch_bounds__(128) q4_columns_kernel(const uint16_t *scales, int groups, int N, int *col_exp)
{
    const int64_t n = (int64_t)blockIdx.x * 128 + threadIdx.x;
    uint32_t top = 0;
    if (n < N)
        for (int g = 0; g < groups; ++g) {
            const uint32_t s = scales[(int64_t)g * N + n] & 0x7fffu;
            if (s < 0x7f80u) top = max(top, s);
        }
    col_exp[n] = top ? ilogbf(__uint_as_float(top << 16)) - 10 : 0;
}

__global__ void __launch_bounds__(128) q4_pack_kernel(const uint8_t *codes, const uint16_t *scales, int K, int N, int G,
                                                      const int *col_exp, uint8_t *blk)
{
    const int r = threadIdx.x, ks = blockIdx.x;
    const int64_t rt = (int64_t)blockIdx.z * 65535 + blockIdx.y, n = rt * kRows + r;
    if (rt * kRows >= N) return;
    uint8_t *const b = blk + (rt * gridDim.x + ks) * block_bytes(G);
    for (int piece = 0; piece < 4; ++piece) {
        uint32_t w[4];
        for (int i = 0; i < 4; ++i) {
            uint32_t v = 0;
            for (int p = 0; p < 4; ++p) {
                const int k = ks * kStageK + piece * 32 + i * 8 + 2 * p;
                const uint32_t c = (n < N && k < K) ? codes[(int64_t)(k / 2) * N + n] : 0u;
                const uint32_t even = (c & 15u) ^ 8u, odd = (c >> 4) ^ 8u;   // q + 8
                if (p < 3) {
                    const int at = p == 0 ? 6 : p == 1 ? 10 : 2;
                    v |= even << at | odd << (at + 16);
                } else v |= even << 14 | odd << 30 | odd >> 2;
            }
            w[i] = v;
        }
        reinterpret_cast<uint4 *>(b)[piece * kRows + r] = make_uint4(w[0], w[1], w[2], w[3]);
    }
    __half *const sc = reinterpret_cast<__half *>(b + kCodeBytes);
    for (int j = 0; j < kStageK / G; ++j) {
        const int g = (ks * kStageK) / G + j;
        float s = 0.f;
        if (n < N && g * G < K) s = __uint_as_float((uint32_t)scales[(int64_t)g * N + n] << 16);
        sc[j * kRows + r] = __float2half_rn(scalbnf(s, -col_exp[n] - 6));
    }
}

// ------------------------------------------------------------------ activations
// 8 values times f1 f2 as fp16 pairs, first and (fp32) second parts.
template <bool F32>
__device__ __forceinline__ void split8(const float (&x)[8], float f1, float f2, uint32_t (&hi)[4], uint32_t (&lo)[4])
{
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        __half h[2], l[2];
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            const float v = x[2 * i + j] * f1 * f2;
            h[j] = __float2half_rn(v);
            const float rest = (v - __half2float(h[j])) * (float)(1 << kLoShift);
            l[j] = __float2half_rn(isfinite(rest) ? rest : 0.f);
        }
        hi[i] = (uint32_t)__half_as_ushort(h[0]) | (uint32_t)__half_as_ushort(h[1]) << 16;
        lo[i] = F32 ? (uint32_t)__half_as_ushort(l[0]) | (uint32_t)__half_as_ushort(l[1]) << 16 : 0u;
    }
}

// Tokens in tiles; for a tile and a stage of 128 k two halves of 64 k, each TN rows of 128 bytes in the order that the
// 128-byte swizzle of the MMA's operand has.  With fp32 activations the first TN / 2 rows are the tokens' first parts,
// the others their second ones.
constexpr int kStageThreads = 256;

struct StageParams {
    const void *x;
    char *xs;
    int *tok_exp;
    int B, K, KS, TN, per_tile;   // per_tile: tokens of a tile
};

// 8 consecutive activations from k on, 0 from K on; fours: x begins on a 16-byte boundary (K is a multiple of 8).
template <bool F32>
__device__ __forceinline__ void load8(const void *x, int64_t token, int k, int K, bool fours, float (&v)[8])
{
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = 0.f;
    if (k >= K) return;
    if constexpr (F32) {
        const float *const at = static_cast<const float *>(x) + token * K + k;
        if (fours) {
            const float4 q = *reinterpret_cast<const float4 *>(at), r = *reinterpret_cast<const float4 *>(at + 4);
            v[0] = q.x; v[1] = q.y; v[2] = q.z; v[3] = q.w; v[4] = r.x; v[5] = r.y; v[6] = r.z; v[7] = r.w;
        } else {
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = at[i];
        }
    } else {
        const uint16_t *const at = static_cast<const uint16_t *>(x) + token * K + k;
        if (fours) unpack8(*reinterpret_cast<const uint4 *>(at), v);
        else {
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = __uint_as_float((uint32_t)at[i] << 16);
        }
    }
}

// Largest finite magnitude, as its bits.
__device__ __forceinline__ uint32_t largest8(const float (&v)[8])
{
    uint32_t top = 0;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        const uint32_t m = __float_as_uint(v[j]) & 0x7fffffffu;
        if (m < 0x7f800000u) top = max(top, m);
    }
    return top;
}

// The power of two that puts a token's largest magnitude (its bits) at 2^14..2^15, and factors whose product divides by it
// (2^-e alone can be out of range).
__device__ __forceinline__ int token_power(uint32_t top) { return top ? ilogbf(__uint_as_float(top)) - 14 : 0; }
__device__ __forceinline__ float2 power_factors(int e) { return make_float2(scalbnf(1.f, -e / 2), scalbnf(1.f, -e - -e / 2)); }

// One CTA to a token: all of it in registers up to K = 8192, so that it is read once.
template <bool F32>
__global__ void __launch_bounds__(kStageThreads) q4_stage_kernel(const StageParams p)
{
    constexpr int kHeld = 4;
    grid_launch_dependents();
    __shared__ uint32_t top_s[kStageThreads / 32];
    const int tid = threadIdx.x, pieces = p.KS * 16;
    const int64_t b = blockIdx.x;
    const bool fours = (reinterpret_cast<uintptr_t>(p.x) & 15u) == 0;
    grid_dependency_wait();
    float v[kHeld][8];
#pragma unroll
    for (int k = 0; k < kHeld; ++k) load8<F32>(p.x, b, (tid + k * kStageThreads) * 8, p.K, fours, v[k]);
    uint32_t top = 0;
#pragma unroll
    for (int k = 0; k < kHeld; ++k) top = max(top, largest8(v[k]));
    for (int c = tid + kHeld * kStageThreads; c < pieces; c += kStageThreads) {
        float w[8];
        load8<F32>(p.x, b, c * 8, p.K, fours, w);
        top = max(top, largest8(w));
    }
    top = __reduce_max_sync(0xffffffffu, top);
    if ((tid & 31) == 0) top_s[tid >> 5] = top;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < kStageThreads / 32; ++i) top = max(top, top_s[i]);
    const int e = token_power(top);
    if (tid == 0) p.tok_exp[b] = e;
    const float2 f = power_factors(e);

    const int tile = (int)(b / p.per_tile), row = (int)(b % p.per_tile);
    char *const base = p.xs + (int64_t)tile * p.KS * p.TN * 256;
    const auto put = [&](int c, const float (&w)[8]) {   // 8 consecutive k are 16 bytes of a row
        uint32_t hi[4], lo[4];
        split8<F32>(w, f.x, f.y, hi, lo);
        char *const half = base + (int64_t)(c >> 3) * p.TN * 128;
        const int piece = c & 7;
        *reinterpret_cast<uint4 *>(half + row * 128 + ((piece ^ (row & 7)) << 4)) = make_uint4(hi[0], hi[1], hi[2], hi[3]);
        if constexpr (F32) {
            const int r = p.TN / 2 + row;
            *reinterpret_cast<uint4 *>(half + r * 128 + ((piece ^ (r & 7)) << 4)) = make_uint4(lo[0], lo[1], lo[2], lo[3]);
        }
    };
#pragma unroll
    for (int k = 0; k < kHeld; ++k)
        if (tid + k * kStageThreads < pieces) put(tid + k * kStageThreads, v[k]);
    for (int c = tid + kHeld * kStageThreads; c < pieces; c += kStageThreads) {
        float w[8];
        load8<F32>(p.x, b, c * 8, p.K, fours, w);
        put(c, w);
    }
}

// ------------------------------------------------------------------ the product
struct Q4Params {
    const uint8_t *blk;
    const int *col_exp;
    const char *xs;
    const int *tok_exp;
    void *y;
    int64_t ld_y;
    int B, N, KS, TT, per_tile;   // TT: token tiles
    int G;
    int per, rem;                 // units of a CTA: per, one more for the first rem
    bool whole;                   // a unit is a tile, else a stage of 128 k
    bool y_f32;
    int stages;                   // of the shared-memory ring
    const void *x;                // the kernels that stage it themselves
    int K;
    int slots;                    // .. stages of x that a CTA has, at most
    float *partial;               // [2 kMaxCtas][R][128]
    int *counters;                // [tiles], 0 between calls
    int *ctl;
};

constexpr int kQ4MaxStages = 8;

// The first unit of CTA c.
__device__ __forceinline__ int first_unit(const Q4Params &p, int c) { return c * p.per + min(c, p.rem); }
// The CTA of a unit.
__device__ __forceinline__ int unit_cta(const Q4Params &p, int u)
{
    const int longer = p.rem * (p.per + 1);
    return u < longer ? u / (p.per + 1) : p.rem + (u - longer) / p.per;
}

// A place in the ring of `n` slots and the parity of its use.
struct Slot {
    int i = 0;
    uint32_t parity = 0;
    __device__ __forceinline__ void next(int n)
    {
        if (++i == n) {
            i = 0;
            parity ^= 1u;
        }
    }
};

// D += A B with A (fp16) in TMEM.
__device__ __forceinline__ void mma_f16_tmem_if(uint32_t lead, uint32_t d_tmem, uint32_t a_tmem, uint64_t b,
                                                uint32_t idesc, uint32_t acc)
{
    asm volatile(
        "{\n\t.reg .pred p, q;\n\tsetp.ne.b32 p, %4, 0;\n\tsetp.ne.b32 q, %5, 0;\n\t"
        "@q tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}"
        ::"r"(d_tmem), "r"(a_tmem), "l"(b), "r"(idesc), "r"(acc), "r"(lead)
        : "memory");
}

__device__ __forceinline__ void tmem_st32(uint32_t taddr, const uint32_t (&r)[32])
{
    __syncwarp();   // (as tmem_ld16)
    asm volatile(
        "tcgen05.st.sync.aligned.32x32b.x32.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, "
        "%16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31, %32};"
        ::"r"(taddr), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]),
        "r"(r[9]), "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15]), "r"(r[16]), "r"(r[17]),
        "r"(r[18]), "r"(r[19]), "r"(r[20]), "r"(r[21]), "r"(r[22]), "r"(r[23]), "r"(r[24]), "r"(r[25]), "r"(r[26]),
        "r"(r[27]), "r"(r[28]), "r"(r[29]), "r"(r[30]), "r"(r[31])
        : "memory");
}

__device__ __forceinline__ void tmem_st16(uint32_t taddr, const uint32_t (&r)[16])
{
    __syncwarp();
    asm volatile(
        "tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16};"
        ::"r"(taddr), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]),
        "r"(r[9]), "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15])
        : "memory");
}

__device__ __forceinline__ void tmem_st_wait() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }

// (Whole numbers read as the low bits of a float of known exponent: a published technique, for fp16 weights in Kim et al.,
// "Who Says Elephants Can't Run", 2022.)
// The 8 codes of a word times the group's scale (t: a 64th of it), as fp16 pairs in the order of k.  At bits 6..9 a field
// reads as 64 (16 + u): 64 (16 + u) t - 1536 t = (u - 8) 64 t in one multiply-add, exact in its product, in 1536 t (10 bits)
// and in the result (11 bits).  At bits 2..5 it reads as 1024 + 4 u, from which 1056 leaves 4 (u - 8): a subtraction and a
// product, which the multiply-add pipe has time for, where a shift to bits 6..9 would go to the logic pipe like the masks.
struct Scale {
    __half2 t, c, t16;
    __device__ __forceinline__ explicit Scale(__half s)
    {
        t = __half2half2(s);
        c = __hmul2(t, __float2half2_rn(-1536.f));
        t16 = __hmul2(t, __float2half2_rn(16.f));
    }
};

__device__ __forceinline__ void dequant8(uint32_t w, const Scale &s, uint32_t *out)
{
    const uint32_t rot = __byte_perm(w, w, 0x0321);
    // (v & mask) | the exponents of 1024, said as one operation of three operands
    const auto field = [](uint32_t v, uint32_t mask) {
        uint32_t d;
        asm("lop3.b32 %0, %1, %2, %3, 0xea;" : "=r"(d) : "r"(v), "r"(mask), "r"(0x64006400u));
        return d;
    };
    const auto half = [](uint32_t v) { return *reinterpret_cast<const __half2 *>(&v); };
    const auto word = [](__half2 h) { return *reinterpret_cast<const uint32_t *>(&h); };
    const __half2 k1056 = __float2half2_rn(1056.f);
    out[0] = word(__hfma2(half(field(w, 0x03c003c0u)), s.t, s.c));
    out[1] = word(__hmul2(__hsub2(half(field(rot, 0x003c003cu)), k1056), s.t16));
    out[2] = word(__hmul2(__hsub2(half(field(w, 0x003c003cu)), k1056), s.t16));
    out[3] = word(__hfma2(half(field(rot, 0x03c003c0u)), s.t, s.c));
}

// warp_wait (tc_common.cuh) with fewer instructions while it waits: the limit and the abort flag are looked at after every
// 16 tries, each of which the hardware suspends for a while.
__device__ __forceinline__ bool role_wait(uint64_t *bar, uint32_t parity, volatile int *abort)
{
    bool ok = mbar_try_wait(bar, parity);
    if (!__all_sync(0xffffffffu, ok)) {
        const unsigned long long t0 = global_ns();
        for (;;) {
#pragma unroll 1
            for (int i = 0; i < 16 && !ok; ++i) ok = mbar_try_wait(bar, parity);
            if (__all_sync(0xffffffffu, ok)) break;
            if (__any_sync(0xffffffffu, *abort != 0 || global_ns() - t0 > kWaitLimitNs)) return false;
        }
    }
    __syncwarp();
    return true;
}

// A row's 128 codes of a block with their scales, and their way to TMEM.
struct Codes {
    uint4 q[4];
    __half sc[4];

    __device__ __forceinline__ void load(const char *block, int per, int r)   // per: groups of a block
    {
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            q[j] = reinterpret_cast<const uint4 *>(block)[j * kRows + r];
            sc[j] = reinterpret_cast<const __half *>(block + kCodeBytes)[((j * per) >> 2) * kRows + r];
        }
    }
    __device__ __forceinline__ void store(uint32_t taddr) const
    {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            uint32_t v[32];
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                const Scale t(sc[2 * h + j]);
                const uint4 c = q[2 * h + j];
                dequant8(c.x, t, v + 16 * j);
                dequant8(c.y, t, v + 16 * j + 4);
                dequant8(c.z, t, v + 16 * j + 8);
                dequant8(c.w, t, v + 16 * j + 12);
            }
            tmem_st32(taddr + h * 32, v);
        }
    }
};

struct Q4Bars {
    uint64_t full[kQ4MaxStages], empty[kQ4MaxStages];
    uint64_t a_full[4], a_empty[4];
    uint64_t d_full[4], d_empty[4];   // (with as many accumulators as stages of weights, d_full says that these are free, too)
    uint64_t group[2];
    uint64_t x_full;
    uint64_t drain;
};

constexpr int kDeqGroups = 2;   // warpgroups that turn weights to fp16

template <int EG>
constexpr int q4_threads() { return 32 * (2 + 4 * kDeqGroups + 4 * EG); }

// Columns [c, c + n) of this warp's lanes added to acc; n 8, 16 or a multiple of 16.
template <int n>
__device__ __forceinline__ void add_columns(uint32_t taddr, float (&acc)[n])
{
    if constexpr (n == 8) {
        float v[8];
        tmem_ld8(taddr, v);
        tmem_ld_wait();
#pragma unroll
        for (int i = 0; i < 8; ++i) acc[i] += v[i];
    } else {
#pragma unroll
        for (int c = 0; c < n; c += 16) {
            float v[16];
            tmem_ld16(taddr + c, v);
            tmem_ld_wait();
#pragma unroll
            for (int i = 0; i < 16; ++i) acc[c + i] += v[i];
        }
    }
}

// v 2^e for a sum v of scaled products (1e-30 < |v| < 1e30, or 0) and any e that two scales' exponents add up to: rounded once
// where the result is subnormal (below e = -252 it is 0).
__device__ __forceinline__ float times_pow2(float v, int e)
{
    e = max(e, -252);
    const int half = e >> 1;
    return v * __int_as_float((half + 127) << 23) * __int_as_float((e - half + 127) << 23);
}

// R: tokens of a tile that are there (columns of the accumulator that are used); TN >= 16: the MMA's N, whose rows past
// R read whatever lies behind them in shared memory and land in columns that nobody reads.  NA, ND: stages of fp16 weights
// and accumulators in TMEM; EG: warpgroups that add the sums up; PER_SM: resident CTAs.
// DIRECT (a few tokens): the CTA brings the activations of its stages to shared memory itself, at its start, with a power of
// two of its own for each token; no second kernel, and the ring holds weights alone.
template <int R, int NA, int ND, int EG, int PER_SM, bool F32, bool DIRECT>
__global__ void __launch_bounds__(q4_threads<EG>(), PER_SM) q4_matmul_kernel(const __grid_constant__ Q4Params p)
{
    constexpr int TN = R < 16 ? 16 : R;
    constexpr int kCols = (ND * TN + NA * 64) <= 256 ? 256 : 512;   // TMEM: accumulators, then the weights
    constexpr int kX = R * 256;                                    // bytes of the activations of a stage
    constexpr uint32_t kIdesc = (1u << 4) | ((uint32_t)(TN >> 3) << 17) | ((uint32_t)(kRows >> 4) << 24);
    constexpr int kGroups = kDeqGroups;
    constexpr int kDeq = 4 * EG, kLoad = kDeq + 4 * kGroups, kMma = kLoad + 1;   // first warps of the roles
    static_assert(ND * TN + NA * 64 <= kCols && kCols * PER_SM <= 512 && NA <= 4 && ND <= 4, "TMEM");
    extern __shared__ char smem_raw[];
    __shared__ Q4Bars bars;
    __shared__ uint32_t tmem_slot;
    __shared__ volatile int abort_flag;
    __shared__ int last_flag[EG];
    __shared__ uint32_t tops[DIRECT ? R : 1];

    const int warp = uniform_warp(), lane = threadIdx.x & 31;
    char *const ring = smem_raw + (-smem_addr(smem_raw) & 1023u);   // (not through an integer: loads stay shared-memory loads)
    const int blk = block_bytes(p.G);
    char *const wring = ring + (size_t)(DIRECT ? p.slots : p.stages) * kX;
    constexpr int kLoaded = DIRECT ? 0 : kX;   // of x, with each stage of the ring
    const int u0 = first_unit(p, blockIdx.x), u1 = first_unit(p, blockIdx.x + 1);
    const int n_it = p.whole ? (u1 - u0) * p.KS : u1 - u0;
    const int tile0 = p.whole ? u0 : u0 / p.KS, ks0 = p.whole ? 0 : u0 - tile0 * p.KS;

    if (threadIdx.x == 0) {
        for (int i = 0; i < kQ4MaxStages; ++i) {
            mbar_init(&bars.full[i], 1);
            mbar_init(&bars.empty[i], DIRECT ? 4 : 5);   // four warps that have read the codes, the MMAs that have read the activations
        }
        for (int i = 0; i < 4; ++i) {
            mbar_init(&bars.a_full[i], 4);
            mbar_init(&bars.a_empty[i], 1);
        }
        for (int i = 0; i < 4; ++i) {
            mbar_init(&bars.d_full[i], 1);
            mbar_init(&bars.d_empty[i], 4 * EG);
        }
        mbar_init(&bars.group[0], 4);
        mbar_init(&bars.group[1], 4);
        mbar_init(&bars.x_full, kLoad);
        mbar_init(&bars.drain, 1);
        abort_flag = 0;
        mbar_init_fence();
    }
    if (DIRECT && threadIdx.x < R) tops[threadIdx.x] = 0u;
    if (warp == kMma) tmem_alloc(&tmem_slot, kCols);
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = tmem_slot;
    // the next kernel, if it asks to, may come to the SMs that this one leaves free
    if constexpr (DIRECT) grid_launch_dependents();

    if (DIRECT && warp < kLoad) {
        // ---- the activations: 8 consecutive k of a token are 16 bytes of a row
        constexpr int kThreads = 32 * kLoad;
        grid_dependency_wait();
        const int n_slots = min(n_it, p.KS), groups = n_slots * 16, first = n_it < p.KS ? ks0 : 0;
        const bool fours = (reinterpret_cast<uintptr_t>(p.x) & 15u) == 0;
        const auto values = [&](int piece, bool there, float (&v)[8]) {
            const int b = piece / groups, g = piece - b * groups;
            int ks = first + (g >> 4);
            if (ks >= p.KS) ks -= p.KS;
            load8<F32>(p.x, b, there ? ks * kStageK + (g & 15) * 8 : p.K, p.K, fours, v);
        };
        // all tokens' pieces at once; the first kHeld of a thread stay in registers between the two steps
        constexpr int kHeld = 2;
        float kept[kHeld][8];
        const int total = p.B * groups;
        const auto largest = [&](int i, const float (&v)[8]) {   // (a multiple of 16 pieces to a token: half a warp has one token)
            uint32_t top = largest8(v);
#pragma unroll
            for (int o = 8; o > 0; o >>= 1) top = max(top, __shfl_xor_sync(0xffffffffu, top, o));
            if ((lane & 15) == 0 && i < total) atomicMax(&tops[i / groups], top);
        };
        const auto put = [&](int i, const float (&v)[8]) {
            const int b = i / groups, g = i - b * groups;
            const float2 f = power_factors(token_power(tops[b]));
            uint32_t hi[4], lo[4];
            split8<F32>(v, f.x, f.y, hi, lo);
            char *const half = ring + (size_t)(g >> 3) * (R * 128);
            const int piece = g & 7;
            *reinterpret_cast<uint4 *>(half + b * 128 + ((piece ^ (b & 7)) << 4)) = make_uint4(hi[0], hi[1], hi[2], hi[3]);
            if constexpr (F32) {
                const int r = R / 2 + b;
                *reinterpret_cast<uint4 *>(half + r * 128 + ((piece ^ (r & 7)) << 4)) = make_uint4(lo[0], lo[1], lo[2], lo[3]);
            }
        };
#pragma unroll
        for (int k = 0; k < kHeld; ++k) {
            const int i = threadIdx.x + k * kThreads;
            values(i, i < total, kept[k]);
        }
#pragma unroll
        for (int k = 0; k < kHeld; ++k) largest(threadIdx.x + k * kThreads, kept[k]);
        for (int i0 = kHeld * kThreads; i0 < total; i0 += kThreads) {
            const int i = i0 + threadIdx.x;
            float v[8];
            values(i, i < total, v);
            largest(i, v);
        }
        named_barrier(3, kThreads);
#pragma unroll
        for (int k = 0; k < kHeld; ++k)
            if (threadIdx.x + k * kThreads < total) put(threadIdx.x + k * kThreads, kept[k]);
        for (int i = threadIdx.x + kHeld * kThreads; i < total; i += kThreads) {
            float v[8];
            values(i, true, v);
            put(i, v);
        }
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");   // the MMAs read what has been written here
        __syncwarp();
        if (lane == 0) mbar_arrive(&bars.x_full);
    }
    if (warp == kLoad) {
        // ---- loads
        const uint32_t lead = elect_one();
        const int ahead = min(n_it, p.stages);
        // the weights do not depend on the kernel that stages the activations
        int ks = ks0, tt = tile0 % p.TT;
        const uint8_t *w = p.blk + ((int64_t)(tile0 / p.TT) * p.KS + ks) * blk;
        auto step_w = [&](int &ks_, int &tt_) {   // (the same row tile again for the next token tile)
            w += blk;
            if (++ks_ == p.KS) {
                ks_ = 0;
                if (++tt_ == p.TT) tt_ = 0;
                else w -= (int64_t)p.KS * blk;
            }
        };
        for (int it = 0; it < ahead; ++it) {
            mbar_expect_if(lead, &bars.full[it], (uint32_t)(blk + kLoaded));
            bulk_load_shared_if(lead, wring + (size_t)it * blk, w, (uint32_t)blk, &bars.full[it]);
            step_w(ks, tt);
        }
        if constexpr (!DIRECT) grid_dependency_wait();
        int xks = ks0, xtt = tile0 % p.TT;
        const char *x = p.xs + ((int64_t)xtt * p.KS + xks) * kX;
        auto step_x = [&] {
            x += kX;
            if (++xks == p.KS) {
                xks = 0;
                if (++xtt == p.TT) {
                    xtt = 0;
                    x = p.xs;
                }
            }
        };
        if constexpr (!DIRECT)
            for (int it = 0; it < ahead; ++it) {
                bulk_load_shared_if(lead, ring + (size_t)it * kX, x, (uint32_t)kX, &bars.full[it]);
                step_x();
            }
        Slot s;   // parity: of the use before
        s.i = ahead == p.stages ? 0 : ahead;
        int issued = ahead;
        for (int it = ahead; it < n_it; ++it) {
            if (!role_wait(&bars.empty[s.i], s.parity, &abort_flag)) {
                if (lane == 0) set_timeout(p.ctl, &abort_flag);
                break;
            }
            mbar_expect_if(lead, &bars.full[s.i], (uint32_t)(blk + kLoaded));
            bulk_load_shared_if(lead, wring + (size_t)s.i * blk, w, (uint32_t)blk, &bars.full[s.i]);
            if constexpr (!DIRECT) {
                bulk_load_shared_if(lead, ring + (size_t)s.i * kX, x, (uint32_t)kX, &bars.full[s.i]);
                step_x();
            }
            step_w(ks, tt);
            s.next(p.stages);
            issued = it + 1;
        }
        // nothing may arrive after the CTA's end
        int never = 0;
        for (int it = max(0, issued - p.stages); it < issued; ++it)
            role_wait(&bars.full[it % p.stages], (uint32_t)((it / p.stages) & 1), &never);
    } else if (warp == kMma) {
        // ---- MMAs
        const uint32_t lead = elect_one();
        // This warp's instructions are one chain, the longest of a small tile's stage, so its places in the rings are
        // literals and cost no arithmetic between the MMAs: it takes U stages a turn (one token through a 4096 x 128256
        // head 61 -> 56 us).
        constexpr int U = NA == ND ? NA : NA * ND / (NA % 2 == 0 && ND % 2 == 0 ? 2 : 1);
        bool ok = true;
        Slot s;
        const uint64_t desc0 = smem_desc(smem_addr(ring));
        int slot = n_it < p.KS ? 0 : ks0;   // (DIRECT) of x
        if constexpr (DIRECT) ok = role_wait(&bars.x_full, 0u, &abort_flag);
        uint32_t odd = 0;
        for (int it0 = 0; it0 < n_it && ok; it0 += U, odd ^= 1u) {
#pragma unroll
            for (int j = 0; j < U; ++j) {
                if (it0 + j >= n_it) break;
                const int a = j % NA, d = j % ND;
                const uint32_t a_parity = (U / NA * odd + j / NA) & 1u, d_parity = (U / ND * odd + j / ND) & 1u;
                if constexpr (!DIRECT) ok = role_wait(&bars.full[s.i], s.parity, &abort_flag);
                if (ok && (it0 > 0 || j >= ND)) ok = role_wait(&bars.d_empty[d], d_parity ^ 1u, &abort_flag);
                if (ok) ok = role_wait(&bars.a_full[a], a_parity, &abort_flag);
                if (!ok) break;
                tc_fence_after();
                const uint64_t desc = desc0 + (uint64_t)((DIRECT ? slot : s.i) * (kX >> 4));
#pragma unroll
                for (int k = 0; k < 8; ++k)   // 16 k: 8 columns of TMEM, 32 bytes of the swizzled rows
                    mma_f16_tmem_if(lead, tmem + d * TN, tmem + ND * TN + a * 64 + k * 8,
                                    desc + (k >> 2) * (R * 128 >> 4) + 2 * (k & 3), kIdesc, (uint32_t)(k > 0));
                if constexpr (!DIRECT) mma_commit_if(lead, &bars.empty[s.i]);
                if constexpr (NA != ND) mma_commit_if(lead, &bars.a_empty[a]);
                mma_commit_if(lead, &bars.d_full[d]);
                if constexpr (DIRECT) slot = slot + 1 == p.KS ? 0 : slot + 1;
                else s.next(p.stages);
            }
        }
        if (!ok && lane == 0) set_timeout(p.ctl, &abort_flag);
        mma_commit_if(lead, &bars.drain);
        int never = 0;
        role_wait(&bars.drain, 0u, &never);
    } else if (warp >= kDeq) {
        // ---- weights to fp16: the warpgroups take turns at the stages
        const int group = (warp - kDeq) >> 2, quad = warp & 3, r = quad * 32 + lane;
        const int per = kStageK / p.G;
        const uint32_t dst = tmem + ((uint32_t)(quad * 32) << 16) + ND * TN;
        bool ok = true;
        Slot s, a;
        for (int i = 0; i < group; ++i) {
            s.next(p.stages);
            a.next(NA);
        }
        for (int it = group; it < n_it; it += kGroups) {
            ok = role_wait(&bars.full[s.i], s.parity, &abort_flag);
            if (!ok) break;
            const char *const w = wring + (size_t)s.i * blk;
            Codes q;
            q.load(w, per, r);
            __syncwarp();
            if (lane == 0) mbar_arrive(&bars.empty[s.i]);
            if (it >= NA) ok = role_wait(NA == ND ? &bars.d_full[a.i] : &bars.a_empty[a.i], a.parity ^ 1u, &abort_flag);
            if (!ok) break;
            tc_fence_after();
            q.store(dst + a.i * 64);
            tmem_st_wait();
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(&bars.a_full[a.i]);
#pragma unroll
            for (int i = 0; i < kGroups; ++i) {
                s.next(p.stages);
                a.next(NA);
            }
        }
        if (!ok && lane == 0) set_timeout(p.ctl, &abort_flag);
    } else {
        // ---- sums: each stage's 128 products are added up by the MMAs, the stages here in fp32 (the accumulator truncates).
        // Warpgroup e has columns [e C, (e + 1) C); with fp32 activations R / 2 second parts follow R / 2 first ones, so
        // each warpgroup takes half of both.
        constexpr int C = R / EG, kOut = F32 ? C / 2 : C;
        constexpr int kPieces = F32 && EG > 1 ? 2 : 1, P = C / kPieces;
        const int e = warp >> 2, quad = warp & 3, r = quad * 32 + lane;
        const uint32_t src = tmem + ((uint32_t)(quad * 32) << 16) + e * P;
        // (the tokens' powers of two come from the preceding kernel: for what is read with plain loads a role waits itself)
        if constexpr (!DIRECT) grid_dependency_wait();
        // The power of two that token i's activations were divided by (in this CTA).
        const auto token_exp = [&](int token0, int i) {
            if constexpr (!DIRECT) return p.tok_exp[token0 + i];
            else return token_power(tops[i]);
        };
        // A barrier of the warpgroup whose wait is bounded like the others (a warp that has given up is not coming).
        uint32_t group_parity = 0;
        const auto group_sync = [&] {
            __syncwarp();
            if (lane == 0) mbar_arrive(&bars.group[e]);
            const bool all = role_wait(&bars.group[e], group_parity, &abort_flag);
            group_parity ^= 1u;
            return all;
        };
        float acc[kPieces][P];
#pragma unroll
        for (int j = 0; j < kPieces; ++j)
#pragma unroll
            for (int i = 0; i < P; ++i) acc[j][i] = 0.f;
        bool ok = true;
        Slot d;
        int ks = ks0, tile = tile0;
        for (int it = 0; it < n_it; ++it) {
            ok = role_wait(&bars.d_full[d.i], d.parity, &abort_flag);
            if (!ok) break;
            tc_fence_after();
#pragma unroll
            for (int j = 0; j < kPieces; ++j) add_columns<P>(src + d.i * TN + j * (R / 2), acc[j]);
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(&bars.d_empty[d.i]);
            d.next(ND);
            const bool tile_end = ++ks == p.KS;
            if (!tile_end && it != n_it - 1) continue;

            // the end of a tile or of this CTA's share of one
            float sum[kOut];
#pragma unroll
            for (int i = 0; i < kOut; ++i) {
                if constexpr (!F32) sum[i] = acc[0][i];
                else if constexpr (kPieces == 2) sum[i] = acc[0][i] + acc[1][i] * (1.f / (1 << kLoShift));
                else sum[i] = acc[0][i] + acc[0][i + kOut] * (1.f / (1 << kLoShift));
            }
            const int tt = tile % p.TT, token0 = tt * p.per_tile + e * kOut;
            const int n = (tile / p.TT) * kRows + r;
            const int tokens = min(p.per_tile - e * kOut, p.B - token0);   // (of the next ones, if more than kOut)
            {
                const int ce = n < p.N ? p.col_exp[n] : 0;
#pragma unroll
                for (int i = 0; i < kOut; ++i)
                    if (i < tokens) sum[i] = times_pow2(sum[i], ce + token_exp(token0, i));
            }
            bool write = true;
            if (!p.whole && (u0 > tile * p.KS || !tile_end)) {
                // the CTAs of the tile leave their sums in the workspace; the last one to come adds them in order
                const int t0 = tile * p.KS, c0 = unit_cta(p, t0), c1 = unit_cta(p, t0 + p.KS - 1);
                auto slot = [&](int c) {   // a CTA's second slot is for the tile that it begins
                    return p.partial + ((size_t)(2 * c + (first_unit(p, c) < t0 ? 1 : 0)) * R + e * kOut) * kRows + r;
                };
                float *const mine = slot(blockIdx.x);
#pragma unroll
                for (int i = 0; i < kOut; ++i)
                    if (i < tokens) __stcg(mine + i * kRows, sum[i]);
                __threadfence();
                if (!(ok = group_sync())) break;
                if (r == 0) {
                    const int old = atom_add_acq_rel_gpu(p.counters + EG * tile + e, 1);
                    last_flag[e] = old == c1 - c0;
                    if (old == c1 - c0) p.counters[EG * tile + e] = 0;
                }
                if (!(ok = group_sync())) break;
                write = last_flag[e] != 0;
                if (write) {
                    __threadfence();
                    // a few tokens at a time, of which a few CTAs' sums are on their way
                    constexpr int kTok = kOut < 8 ? kOut : 8, kAtOnce = 4;
#pragma unroll
                    for (int i0 = 0; i0 < kOut; i0 += kTok) {
                        if (i0 >= tokens) break;
#pragma unroll
                        for (int i = 0; i < kTok; ++i) sum[i0 + i] = 0.f;
                        for (int c = c0; c <= c1; c += kAtOnce) {
                            float part[kAtOnce][kTok];
#pragma unroll
                            for (int j = 0; j < kAtOnce; ++j) {
                                const float *const from = slot(min(c + j, c1));
#pragma unroll
                                for (int i = 0; i < kTok; ++i)
                                    part[j][i] = i0 + i < tokens && c + j <= c1 ? __ldcg(from + (i0 + i) * kRows) : 0.f;
                            }
#pragma unroll
                            for (int j = 0; j < kAtOnce; ++j)
#pragma unroll
                                for (int i = 0; i < kTok; ++i) sum[i0 + i] += part[j][i];
                        }
                    }
                }
            }
            if (write && n < p.N) {
#pragma unroll
                for (int i = 0; i < kOut; ++i) {
                    if (i < tokens) {
                        const int64_t at = (int64_t)(token0 + i) * p.ld_y + n;
                        if (p.y_f32) static_cast<float *>(p.y)[at] = sum[i];
                        else static_cast<__nv_bfloat16 *>(p.y)[at] = __float2bfloat16_rn(sum[i]);
                    }
                }
            }
#pragma unroll
            for (int j = 0; j < kPieces; ++j)
#pragma unroll
                for (int i = 0; i < P; ++i) acc[j][i] = 0.f;
            if (tile_end) {
                ks = 0;
                ++tile;
            }
        }
        if (!ok && lane == 0) set_timeout(p.ctl, &abort_flag);
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    if (warp == kMma) tmem_dealloc(tmem, kCols);
}

// ------------------------------------------------------------------ the product for many tokens
// Two row tiles (256 columns of the weights) to a tile of 128 columns of activations, so that these come through the L2
// half as often: at 128 x 128 they are 41 KB a stage of 512 cycles of MMAs, more than the L2 gives every SM (2048
// tokens through 4096 x 14336 took 279 us, 179 of them without dequantising, MMAs or sums).  Each row tile has an
// accumulator; while the MMAs of a stage fill one, two warpgroups add the other's 128 products up, in registers like the
// kernel above: 128 sums a thread, for which they take registers from the other warps.  2048 tokens 197 us, of which
// writing the results 30 (the sums are not read meanwhile); with sums that stay in the accumulators for all of K 187, but
// those are cut off K / 16 times.
constexpr int kWideR = 128, kWideGroups = 4, kWideEpi = 8;
constexpr int kWideThreads = 32 * (kWideEpi + 4 * kWideGroups + 4);   // (two warps of the last four: loads, MMAs)
constexpr int kWideNA = 4;
constexpr int kWideStages = 4;
// Registers a thread at the launch, and of the three kinds of warpgroups from then on: what is given up has to cover
// what is taken, or the taking waits for ever.
constexpr int kWideRegs = 72, kWideEpiRegs = 152, kWideDeqRegs = 40, kWideRestRegs = 32;
static_assert(kWideEpiRegs * 32 * kWideEpi + kWideDeqRegs * 128 * kWideGroups + kWideRestRegs * 128 <= kWideRegs * kWideThreads,
              "registers that there are");

template <int n>
__device__ __forceinline__ void more_registers()
{
    __syncwarp();
    asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(n));
}
template <int n>
__device__ __forceinline__ void fewer_registers()
{
    __syncwarp();
    asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(n));
}

struct WideBars {
    uint64_t full[kWideStages], empty[kWideStages];
    uint64_t a_full[kWideNA], a_empty[kWideNA];
    uint64_t d_full[2], d_empty[2];
    uint64_t drain;
};

template <bool F32>
__global__ void __launch_bounds__(kWideThreads, 1) q4_wide_kernel(const __grid_constant__ Q4Params p)
{
    constexpr int R = kWideR, kX = R * 256, kCols = 512;
    constexpr uint32_t kIdesc = (1u << 4) | ((uint32_t)(R >> 3) << 17) | ((uint32_t)(kRows >> 4) << 24);
    constexpr int kLoad = kWideEpi + 4 * kWideGroups, kMma = kLoad + 1;
    extern __shared__ char smem_raw[];
    __shared__ WideBars bars;
    __shared__ uint32_t tmem_slot;
    __shared__ volatile int abort_flag;

    const int warp = uniform_warp(), lane = threadIdx.x & 31;
    char *const ring = smem_raw + (-smem_addr(smem_raw) & 1023u);
    const int blk = block_bytes(p.G);
    char *const wring = ring + (size_t)p.stages * kX;
    const int tile0 = first_unit(p, blockIdx.x), n_tiles = first_unit(p, blockIdx.x + 1) - tile0;   // pairs of row tiles
    const int n_it = n_tiles * p.KS, last_rt = (p.N - 1) / kRows;

    if (threadIdx.x == 0) {
        for (int i = 0; i < kWideStages; ++i) {
            mbar_init(&bars.full[i], 1);
            mbar_init(&bars.empty[i], 9);   // four warps to each of the two blocks of codes, the MMAs
        }
        for (int i = 0; i < kWideNA; ++i) {
            mbar_init(&bars.a_full[i], 4);
            mbar_init(&bars.a_empty[i], 1);
        }
        for (int i = 0; i < 2; ++i) {
            mbar_init(&bars.d_full[i], 1);
            mbar_init(&bars.d_empty[i], kWideEpi);
        }
        mbar_init(&bars.drain, 1);
        abort_flag = 0;
        mbar_init_fence();
    }
    if (warp == kMma) tmem_alloc(&tmem_slot, kCols);
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = tmem_slot;

    if (warp >= kLoad) {
        fewer_registers<kWideRestRegs>();
        if (warp == kLoad) {
            // ---- loads
            const uint32_t lead = elect_one();
            grid_dependency_wait();
            int tile = tile0, ks = 0, issued = 0;
            const uint8_t *w = nullptr;
            const char *x = nullptr;
            int64_t second = 0;   // how far the second row tile's blocks lie behind the first's (0: there is none)
            Slot s;
            for (int it = 0; it < n_it; ++it) {
                if (ks == 0) {
                    const int rt = tile / p.TT * 2;
                    w = p.blk + (int64_t)rt * p.KS * blk;
                    x = p.xs + (int64_t)(tile % p.TT) * p.KS * kX;
                    second = rt < last_rt ? (int64_t)p.KS * blk : 0;
                }
                if (it >= p.stages && !role_wait(&bars.empty[s.i], s.parity ^ 1u, &abort_flag)) {
                    if (lane == 0) set_timeout(p.ctl, &abort_flag);
                    break;
                }
                mbar_expect_if(lead, &bars.full[s.i], (uint32_t)(2 * blk + kX));
                bulk_load_shared_if(lead, wring + (size_t)s.i * 2 * blk, w, (uint32_t)blk, &bars.full[s.i]);
                bulk_load_shared_if(lead, wring + (size_t)(s.i * 2 + 1) * blk, w + second, (uint32_t)blk, &bars.full[s.i]);
                bulk_load_shared_if(lead, ring + (size_t)s.i * kX, x, (uint32_t)kX, &bars.full[s.i]);
                w += blk;
                x += kX;
                issued = it + 1;
                s.next(p.stages);
                if (++ks == p.KS) {
                    ks = 0;
                    ++tile;
                }
            }
            // nothing may arrive after the CTA's end
            int never = 0;
            for (int it = max(0, issued - p.stages); it < issued; ++it)
                role_wait(&bars.full[it % p.stages], (uint32_t)((it / p.stages) & 1), &never);
        } else if (warp == kMma) {
            // ---- MMAs: of a stage the first row tile's, then the second's
            const uint32_t lead = elect_one();
            bool ok = true;
            Slot s;
            const uint64_t desc0 = smem_desc(smem_addr(ring));
            uint32_t odd = 0;        // of the turn through the four places for weights
            for (int it0 = 0; it0 < n_it && ok; it0 += 2, odd ^= 1u) {
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const int d = j & 1;
                    const uint32_t before = (uint32_t)(j >> 1) ^ 1u;   // parity of the accumulator's use before
                    if (it0 + (j >> 1) >= n_it) break;
                    if (d == 0) ok = role_wait(&bars.full[s.i], s.parity, &abort_flag);
                    if (ok && it0 + (j >> 1) > 0) ok = role_wait(&bars.d_empty[d], before, &abort_flag);
                    if (ok) ok = role_wait(&bars.a_full[j], odd, &abort_flag);
                    if (!ok) break;
                    tc_fence_after();
                    const uint64_t desc = desc0 + (uint64_t)(s.i * (kX >> 4));
#pragma unroll
                    for (int k = 0; k < 8; ++k)
                        mma_f16_tmem_if(lead, tmem + d * R, tmem + 2 * R + j * 64 + k * 8,
                                        desc + (k >> 2) * (R * 128 >> 4) + 2 * (k & 3), kIdesc, (uint32_t)(k > 0));
                    mma_commit_if(lead, &bars.a_empty[j]);
                    mma_commit_if(lead, &bars.d_full[d]);
                    if (d == 1) {
                        mma_commit_if(lead, &bars.empty[s.i]);
                        s.next(p.stages);
                    }
                }
            }
            if (!ok && lane == 0) set_timeout(p.ctl, &abort_flag);
            mma_commit_if(lead, &bars.drain);
            int never = 0;
            role_wait(&bars.drain, 0u, &never);
        }
    } else if (warp >= kWideEpi) {
        // ---- weights to fp16: the warpgroups take turns at the blocks, two to a stage
        fewer_registers<kWideDeqRegs>();
        static_assert(kWideGroups == kWideNA, "a warpgroup has one place in TMEM");
        const int group = (warp - kWideEpi) >> 2, quad = warp & 3, r = quad * 32 + lane;
        const int per = kStageK / p.G;
        const uint32_t dst = tmem + ((uint32_t)(quad * 32) << 16) + 2 * R + group * 64;
        bool ok = true;
        Slot s;
        uint32_t used = 0;   // times this place has been
        if (group >= 2) s.next(p.stages);
        for (int it = group >> 1; it < n_it; it += 2, ++used) {
            ok = role_wait(&bars.full[s.i], s.parity, &abort_flag);
            if (!ok) break;
            if (used > 0) ok = role_wait(&bars.a_empty[group], (used - 1) & 1u, &abort_flag);
            if (!ok) break;
            tc_fence_after();
            const char *const block = wring + (size_t)(s.i * 2 + (group & 1)) * blk;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const uint4 q = reinterpret_cast<const uint4 *>(block)[j * kRows + r];
                const Scale t(reinterpret_cast<const __half *>(block + kCodeBytes)[((j * per) >> 2) * kRows + r]);
                uint32_t v[16];
                dequant8(q.x, t, v);
                dequant8(q.y, t, v + 4);
                dequant8(q.z, t, v + 8);
                dequant8(q.w, t, v + 12);
                tmem_st16(dst + j * 16, v);
            }
            __syncwarp();
            if (lane == 0) mbar_arrive(&bars.empty[s.i]);
            tmem_st_wait();
            tc_fence_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(&bars.a_full[group]);
            s.next(p.stages);
            s.next(p.stages);
        }
        if (!ok && lane == 0) set_timeout(p.ctl, &abort_flag);
    } else {
        // ---- sums and results: warpgroup e has the columns [64 e, 64 e + 64) of both row tiles (fp32 activations: half
        // of the first and of the second parts)
        more_registers<kWideEpiRegs>();
        constexpr int kOut = F32 ? 32 : 64;
        const int e = warp >> 2, quad = warp & 3, r = quad * 32 + lane;
        const uint32_t src = tmem + ((uint32_t)(quad * 32) << 16) + e * kOut;
        grid_dependency_wait();   // (the tokens' powers of two)
        const bool twos = (reinterpret_cast<uintptr_t>(p.y) & 3u) == 0 && p.ld_y % 2 == 0;
        f32x2 acc[2][32];         // columns src + 0.. and (fp32 activations, from the 16th pair on) src + R / 2 + 0..
#pragma unroll
        for (int i = 0; i < 32; ++i) acc[0][i] = acc[1][i] = pack2(0.f, 0.f);
        bool ok = true;
        int ks = 0, tile = tile0;
        for (int it = 0; it < n_it && ok; ++it) {
            const bool tile_end = ks + 1 == p.KS;
#pragma unroll
            for (int d = 0; d < 2; ++d) {
                if (ok) ok = role_wait(&bars.d_full[d], (uint32_t)(it & 1), &abort_flag);
                if (!ok) break;
                tc_fence_after();
#pragma unroll
                for (int c = 0; c < 64; c += 16) {
                    float v[16];
                    tmem_ld16(src + d * R + (F32 && c >= 32 ? R / 2 - 32 : 0) + c, v);
                    tmem_ld_wait();
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        f32x2 &a = acc[d][c / 2 + i];
                        const f32x2 b = pack2(v[2 * i], v[2 * i + 1]);
                        a = fadd2(a, b);
                    }
                }
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(&bars.d_empty[d]);
            }
            if (!ok) break;
            if (tile_end) {
                const int token0 = tile % p.TT * p.per_tile + e * kOut, tokens = min(kOut, p.B - token0);
                // a lane has two tokens' powers of two: loads between the stores would each wait for the L2
                int te[2];
#pragma unroll
                for (int i = 0; i < 2; ++i)
                    te[i] = i * 32 + lane < tokens ? p.tok_exp[token0 + i * 32 + lane] : 0;
                const bool near_tokens = __all_sync(0xffffffffu, abs(te[0]) <= 40 && abs(te[1]) <= 40);
#pragma unroll
                for (int d = 0; d < 2; ++d) {
                    const int n = (tile / p.TT * 2 + d) * kRows + r, n0 = n & ~1;
                    const int ce = n < p.N ? p.col_exp[n] : 0;
                    // powers of two that are far from fp32's ends in every lane: one factor (the sums are 0 or 2^-60 to 2^60)
                    const bool near = near_tokens && __all_sync(0xffffffffu, abs(ce) <= 40);
                    const auto times = [&](float v, int i) {
                        const int t = __shfl_sync(0xffffffffu, te[i / 32], i % 32);
                        return near ? v * __int_as_float((ce + 127 + t) << 23) : times_pow2(v, ce + t);
                    };
                    uint16_t *at = static_cast<uint16_t *>(p.y) + (int64_t)(token0 + (lane & 1)) * p.ld_y + n0;
                    const uint32_t pick = lane & 1 ? 0x3276u : 0x5410u;
                    int left = tokens - (lane & 1);
#pragma unroll
                    for (int i = 0; i < kOut; i += 2, at += 2 * p.ld_y, left -= 2) {
                        float2 v = unpack2(acc[d][i / 2]);
                        if constexpr (F32) {
                            const float2 lo = unpack2(acc[d][16 + i / 2]);
                            v.x += lo.x * (1.f / (1 << kLoShift));
                            v.y += lo.y * (1.f / (1 << kLoShift));
                        }
                        const float v0 = times(v.x, i), v1 = times(v.y, i + 1);
                        // two lanes' columns of a token in one store: the even lane writes the first token's, the odd one the second's
                        const __nv_bfloat162 h = __floats2bfloat162_rn(v0, v1);
                        const uint32_t mine = *reinterpret_cast<const uint32_t *>(&h);
                        const uint32_t both = __byte_perm(mine, __shfl_xor_sync(0xffffffffu, mine, 1), pick);
                        if (left <= 0) continue;
                        if (twos && n0 + 1 < p.N) *reinterpret_cast<uint32_t *>(at) = both;
                        else {
                            if (n0 < p.N) at[0] = (uint16_t)both;
                            if (n0 + 1 < p.N) at[1] = (uint16_t)(both >> 16);
                        }
                    }
#pragma unroll
                    for (int i = 0; i < 32; ++i) acc[d][i] = pack2(0.f, 0.f);
                }
                ++tile;
            }
            ks = tile_end ? 0 : ks + 1;
        }
        if (!ok && lane == 0) set_timeout(p.ctl, &abort_flag);
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    if (warp == kMma) tmem_dealloc(tmem, kCols);
}

// ------------------------------------------------------------------ host
// Tokens of a tile: fp32 activations take two columns each.
int tile_tokens(int B, bool f32)
{
    const int64_t cols = (int64_t)B * (f32 ? 2 : 1);
    return cols <= 8 ? 8 : cols <= 16 ? 16 : cols <= 32 ? 32 : cols <= 64 ? 64 : 128;
}

struct Q4Layout {
    size_t counters, tok_exp, partial, xs, total;
};

size_t up256(size_t v) { return (v + 255) & ~(size_t)255; }

// The counters, which are 0 between calls, have the same place in every call's layout: a workspace serves smaller batches
// and other weights, too.  Room for either type of activations.
Q4Layout q4_layout(int K, int N, int B)
{
    Q4Layout L{};
    const int b = std::max(B, 1);
    size_t xs = 0, partial = 0;
    for (int f = 0; f < 2; ++f) {
        const int TN = tile_tokens(b, f != 0);
        const size_t tt = (size_t)div_up(b, f ? TN / 2 : TN);
        xs = std::max(xs, tt * div_up(K, kStageK) * TN * 256);
        partial = std::max(partial, (size_t)2 * kMaxCtas * TN * kRows * 4);
    }
    L.counters = kCtlBytes;
    L.tok_exp = L.counters + up256((size_t)kMaxSplitTiles * 2 * 4);
    L.partial = L.tok_exp + up256((size_t)b * 4);
    L.xs = L.partial + up256(partial);
    L.total = L.xs + xs;
    return L;
}

bool q4_shape_ok(int64_t K, int64_t N, int G)
{
    return K >= 8 && K <= kMaxK && K % 8 == 0 && N >= 1 && N <= kMaxQ4N && (G == 32 || G == 64 || G == 128);
}

constexpr int kSmemPair = 110 * 1024, kSmemOne = 222 * 1024;   // of a CTA, two or one to an SM
constexpr int kDirectRing = 4;   // stages of weights that have to fit beside the activations

// How the stages go to the CTAs.
void plan_q4(Q4Params &p, int R, int per_sm, int *grid)
{
    const int tiles = div_up(p.N, kRows) * p.TT;
    const int most = std::min(kMaxCtas, per_sm * sm_count());
    // Whole tiles where that is at most so many stages more for the busiest CTA, else any number of stages each, and an
    // exchange of sums.  Whole / divided (us, bf16 activations, fp32 results): one token, K 4096, 1003 tiles (23 stages more)
    // 55.6 / 59.1, 152 tiles (16) 13.3 / 13.7, 456 tiles (16) 34.7 / 30.2; K 8192, 152 tiles (32) 33.6 / 22.0; 24 tokens, K 4096,
    // 699 tiles (23) 51.1 / 55.7, 152 tiles (16) 21.7 / 18.2; K 8192, 456 tiles (32) 73.3 / 62.4.  Wide tiles, 128 tokens: K 4096, 350
    // tiles (23) 69.7 / 70.6, 76 tiles (16) 25.5 / 24.2; K 8192, 76 tiles (32) 42.4 / 34.2, 175 tiles (55) 77.5 / 63.8.  Below
    // 8 stages whole tiles win everywhere, by 5 to 40 %.
    const int loss = R >= 64 ? 32 : 16;
    const int64_t waves = (tiles + most - 1) / most;
    p.whole = waves > kMaxSplitWaves || waves * p.KS - (int64_t)tiles * p.KS / most <= loss;
    const int units = p.whole ? tiles : tiles * p.KS;
    *grid = std::min(most, units);
    p.per = units / *grid;
    p.rem = units % *grid;
    p.slots = std::min<int64_t>(p.KS, (int64_t)(p.per + (p.rem > 0 ? 1 : 0)) * (p.whole ? p.KS : 1));
}

// Places of a ring, at most n, of which kDeqGroups warpgroups take the stages in turns.  With an odd number of places a warpgroup sees
// every second use of one, and by the parity it waits for, the use before last passes for its own while the other
// warpgroup's between is still arriving.  That one has arrived once the MMAs of the stage n before are done; a warpgroup that
// has finished its own stage before knows this of the stage NA + kDeqGroups before.  (128 columns had 5 places and 4 of
// weights: a result of 256 tokens in 250 had a tile with wrong stages.)
int ring_stages(int n, int NA) { return n % kDeqGroups != 0 && n < NA + kDeqGroups ? n / kDeqGroups * kDeqGroups : n; }

template <int R, int NA, int ND, int EG, int PER_SM, bool F32, bool DIRECT>
cudaError_t launch_q4(const Q4Params &planned, int grid, cudaStream_t st)
{
    static std::atomic<int> configured[64];
    Q4Params p = planned;
    const int stage = block_bytes(p.G) + (DIRECT ? 0 : R * 256);
    const int kept = 1024 + (DIRECT ? p.slots * R * 256 : 0);
    p.stages = std::min(kQ4MaxStages, ((PER_SM == 2 ? kSmemPair : kSmemOne) - kept) / stage);
    p.stages = ring_stages(p.stages, NA);
    const size_t smem = (size_t)p.stages * stage + kept;
    const cudaError_t e = set_smem(q4_matmul_kernel<R, NA, ND, EG, PER_SM, F32, DIRECT>, smem, configured);
    if (e != cudaSuccess) return e;
    return launch_pdl_cfg(q4_matmul_kernel<R, NA, ND, EG, PER_SM, F32, DIRECT>, dim3(grid), q4_threads<EG>(), smem, st, p);
}

// Whether the kernel for many tokens takes a call: pairs of row tiles that fill the SMs evenly enough.  With it / without
// (us, 128 to 2048 tokens): three quarters of a wave, K 4096 35.0 / 46.6, K 1024 16.7 / 22.0; 0.45 of one 33.7 / 27.2 and 16.3 / 13.3;
// one and a half waves 66.3 / 72.8; 1.1 waves (0.55 of two) 65.1 / 66.5.  (From half of a wave on it would win, too: 34.2 / 43.8.)
bool plan_wide(Q4Params &p, int R, int *grid)
{
    const int sms = std::min(kMaxCtas, sm_count());
    const int64_t pairs = (int64_t)div_up(div_up(p.N, kRows), 2) * p.TT, waves = (pairs + sms - 1) / sms;
    if (p.y_f32 || R != kWideR || pairs * 4 < waves * sms * 3) return false;
    *grid = sms;
    p.per = (int)(pairs / sms);
    p.rem = (int)(pairs % sms);
    return true;
}

template <bool F32>
cudaError_t launch_wide(const Q4Params &planned, int grid, cudaStream_t st)
{
    static std::atomic<int> configured[64];
    // (asked once: a build that gives the threads fewer registers must not begin to exchange them)
    static std::atomic<int> registers{0};
    if (registers.load() == 0) {
        cudaFuncAttributes attr{};
        const cudaError_t e = cudaFuncGetAttributes(&attr, q4_wide_kernel<F32>);
        if (e != cudaSuccess) return e;
        registers.store(attr.numRegs);
    }
    if (registers.load() < kWideRegs) return cudaErrorInvalidDeviceFunction;
    Q4Params p = planned;
    const int stage = 2 * block_bytes(p.G) + kWideR * 256;
    p.stages = std::min(kWideStages, (kSmemOne - 1024) / stage);
    const size_t smem = (size_t)p.stages * stage + 1024;
    const cudaError_t e = set_smem(q4_wide_kernel<F32>, smem, configured);
    if (e != cudaSuccess) return e;
    return launch_pdl_cfg(q4_wide_kernel<F32>, dim3(grid), kWideThreads, smem, st, p);
}

template <bool F32>
cudaError_t run_q4(const sats_q4 *w, const void *x, int B, void *y, int64_t ld_y, bool y_f32, char *ws, cudaStream_t st)
{
    const Q4Layout L = q4_layout(w->K, w->N, B);
    const int TN = tile_tokens(B, F32);
    Q4Params p{};
    p.blk = w->blk; p.col_exp = w->col_exp; p.xs = ws + L.xs;
    p.tok_exp = reinterpret_cast<int *>(ws + L.tok_exp);
    p.y = y; p.ld_y = ld_y; p.B = B; p.N = w->N; p.G = w->G; p.y_f32 = y_f32;
    p.KS = div_up(w->K, kStageK);
    p.per_tile = F32 ? TN / 2 : TN;
    p.TT = div_up(B, p.per_tile);
    p.partial = reinterpret_cast<float *>(ws + L.partial);
    p.counters = reinterpret_cast<int *>(ws + L.counters);
    p.ctl = reinterpret_cast<int *>(ws);

    p.x = x;
    p.K = w->K;
    int grid = 0;
    plan_q4(p, TN, TN <= 32 ? 2 : 1, &grid);
    if (TN <= kDirectTokens && 1024 + p.slots * TN * 256 + kDirectRing * block_bytes(p.G) <= kSmemPair)
        return TN == 8 ? launch_q4<8, 3, 3, 1, 2, F32, true>(p, grid, st) : launch_q4<16, 3, 3, 1, 2, F32, true>(p, grid, st);

    StageParams sp{x, ws + L.xs, reinterpret_cast<int *>(ws + L.tok_exp), B, w->K, p.KS, TN, p.per_tile};
    const cudaError_t e = launch_pdl_threads(q4_stage_kernel<F32>, dim3(B), kStageThreads, st, sp);
    if (e != cudaSuccess) return e;
    int wide = 0;
    if (plan_wide(p, TN, &wide)) return launch_wide<F32>(p, wide, st);
    switch (TN) {
    case 8: return launch_q4<8, 3, 3, 1, 2, F32, false>(p, grid, st);
    case 16: return launch_q4<16, 3, 3, 1, 2, F32, false>(p, grid, st);
    case 32: return launch_q4<32, 2, 2, 1, 2, F32, false>(p, grid, st);
    case 64: return launch_q4<64, 4, 2, 1, 1, F32, false>(p, grid, st);
    default: return launch_q4<128, 4, 2, 2, 1, F32, false>(p, grid, st);
    }
}

// Whether `n` bytes from a on and `rows` rows of `row` bytes, `step` apart, from b on have a byte in common.
bool overlap(const void *a, size_t n, const void *b, size_t rows, size_t row, size_t step)
{
    const uintptr_t a0 = reinterpret_cast<uintptr_t>(a), b0 = reinterpret_cast<uintptr_t>(b);
    if (a0 + n <= b0 || b0 + (rows - 1) * step + row <= a0) return false;
    if (a0 <= b0) return true;
    const size_t in = (a0 - b0) % step;   // a begins in, or behind, a row that is there
    return in < row || ((a0 - b0) / step + 1 < rows && in + n > step);
}

template <bool F32>
sats_status q4_matmul(const sats_q4 *w, const void *x, int B, void *y, int64_t ld_y, int y_f32, void *ws, size_t ws_bytes,
                      void *stream)
{
    if (!w || !ws || B < 0) return SATS_EINVAL;
    if (reinterpret_cast<uintptr_t>(ws) % 256) return SATS_EINVAL;
    if (ld_y < w->N) return SATS_EINVAL;
    if (B > 1 << 20 || ld_y > (int64_t)1 << 40) return SATS_ESHAPE;
    const size_t need = q4_layout(w->K, w->N, B).total;
    if (ws_bytes < need) return SATS_ENOSPACE;
    if (B == 0) return SATS_OK;
    if (!x || !y || reinterpret_cast<uintptr_t>(x) % (F32 ? 4 : 2) || reinterpret_cast<uintptr_t>(y) % (y_f32 ? 4 : 2))
        return SATS_EINVAL;
    // (CTAs write results while others still read activations)
    const size_t x_bytes = (size_t)B * w->K * (F32 ? 4 : 2), y_es = y_f32 ? 4 : 2, row = w->N * y_es, step = ld_y * y_es;
    if (overlap(x, x_bytes, y, B, row, step) || overlap(ws, need, x, 1, x_bytes, x_bytes) || overlap(ws, need, y, B, row, step))
        return SATS_EINVAL;
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return cuda_fail(e, "cudaGetDevice");
    if (dev != w->device) return SATS_EINVAL;
    e = run_q4<F32>(w, x, B, y, ld_y, y_f32 != 0, static_cast<char *>(ws), static_cast<cudaStream_t>(stream));
    return e == cudaSuccess ? SATS_OK : cuda_fail(e, "4-bit product kernel launch");
}

}  // namespace
}  // namespace sats

using namespace sats;

extern "C" {

sats_status sats_q4_quantize(const void *W, int64_t ld, int K, int N, int G, uint8_t *codes, void *scales, void *stream)
{
    if (ld < N) return SATS_EINVAL;
    if (!q4_shape_ok(K, N, G) || ld > (int64_t)1 << 40) return SATS_ESHAPE;
    if (!W || !codes || !scales || reinterpret_cast<uintptr_t>(W) % 2 || reinterpret_cast<uintptr_t>(scales) % 2)
        return SATS_EINVAL;
    const dim3 grid(div_up(N, kQuantCols), div_up(K, kQuantWarps * kQuantRows));
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    const uint16_t *const w = static_cast<const uint16_t *>(W);
    uint16_t *const sc = static_cast<uint16_t *>(scales);
    const bool in4 = in_fours(W, ld, 2), out4 = in_fours(codes, N, 1);
    const auto kernel = in4 ? (out4 ? q4_quantize_kernel<true, true> : q4_quantize_kernel<true, false>)
                            : (out4 ? q4_quantize_kernel<false, true> : q4_quantize_kernel<false, false>);
    kernel<<<grid, 32 * kQuantWarps, 0, st>>>(w, ld, K, N, G, codes, sc);
    const cudaError_t e = cudaGetLastError();
    return e == cudaSuccess ? SATS_OK : cuda_fail(e, "quantising kernel launch");
}

sats_status sats_q4_dequantize(const uint8_t *codes, const void *scales, int K, int N, int G, float *values, void *stream)
{
    if (!q4_shape_ok(K, N, G)) return SATS_ESHAPE;
    if (!codes || !scales || !values || reinterpret_cast<uintptr_t>(scales) % 2 || reinterpret_cast<uintptr_t>(values) % 4)
        return SATS_EINVAL;
    const bool fours = in_fours(codes, N, 1) && in_fours(values, N, 4);
    const dim3 grid(div_up(N, fours ? 1024 : 256), div_up(K / 2, kReadRows));
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    const uint16_t *const sc = static_cast<const uint16_t *>(scales);
    if (fours) q4_dequantize_kernel<true><<<grid, 256, 0, st>>>(codes, sc, K, N, G, values);
    else q4_dequantize_kernel<false><<<grid, 256, 0, st>>>(codes, sc, K, N, G, values);
    const cudaError_t e = cudaGetLastError();
    return e == cudaSuccess ? SATS_OK : cuda_fail(e, "reading back kernel launch");
}

sats_status sats_q4_create(const uint8_t *codes, const void *scales, int K, int N, int G, void *stream, sats_q4 **out)
{
    if (!out) return SATS_EINVAL;
    *out = nullptr;
    if (!codes || !scales || reinterpret_cast<uintptr_t>(scales) % 2) return SATS_EINVAL;
    if (!q4_shape_ok(K, N, G)) return SATS_ESHAPE;
    sats_q4 *w = new (std::nothrow) sats_q4();
    if (!w) return cuda_fail(cudaErrorMemoryAllocation, "host allocation");
    w->K = K;
    w->N = N;
    w->G = G;
    cudaGetDevice(&w->device);
    const int rt = div_up(N, kRows), ks = div_up(K, kStageK);
    cudaStream_t st = static_cast<cudaStream_t>(stream);
    const uint16_t *sc = static_cast<const uint16_t *>(scales);
    cudaError_t e = cudaMalloc(&w->blk, (size_t)rt * ks * block_bytes(G));
    if (e == cudaSuccess) e = cudaMalloc(&w->col_exp, (size_t)rt * kRows * sizeof(int));
    if (e == cudaSuccess) {
        q4_columns_kernel<<<rt, 128, 0, st>>>(sc, div_up(K, G), N, w->col_exp);
        q4_pack_kernel<<<dim3(ks, std::min(rt, 65535), div_up(rt, 65535)), 128, 0, st>>>(codes, sc, K, N, G, w->col_exp, w->blk);
        e = cudaGetLastError();
    }
    if (e == cudaSuccess) e = cudaStreamSynchronize(st);
    if (e != cudaSuccess) {
        cudaFree(w->blk);
        cudaFree(w->col_exp);
        delete w;
        return cuda_fail(e, "4-bit weights: allocation or packing");
    }
    *out = w;
    return SATS_OK;
}

sats_status sats_q4_destroy(sats_q4 *w)
{
    if (!w) return SATS_EINVAL;
    // (the device that may still be at work with it, whichever is the current one)
    int dev = w->device;
    cudaGetDevice(&dev);
    if (dev != w->device) cudaSetDevice(w->device);
    cudaDeviceSynchronize();
    const cudaError_t e1 = cudaFree(w->blk), e2 = cudaFree(w->col_exp);
    if (dev != w->device) cudaSetDevice(dev);
    delete w;
    if (e1 != cudaSuccess) return cuda_fail(e1, "cudaFree");
    return e2 == cudaSuccess ? SATS_OK : cuda_fail(e2, "cudaFree");
}

sats_status sats_q4_shape(const sats_q4 *w, int *K, int *N, int *G)
{
    if (!w) return SATS_EINVAL;
    if (K) *K = w->K;
    if (N) *N = w->N;
    if (G) *G = w->G;
    return SATS_OK;
}

size_t sats_q4_workspace_bytes(int K, int N, int B)
{
    if (!q4_shape_ok(K, N, 32) || B < 0 || B > 1 << 20) return 0;
    return q4_layout(K, N, B).total;
}

sats_status sats_q4_matmul(const sats_q4 *w, const void *x, int B, void *y, int64_t ld_y, int y_f32, void *ws,
                           size_t ws_bytes, void *stream)
{
    return q4_matmul<false>(w, x, B, y, ld_y, y_f32, ws, ws_bytes, stream);
}

sats_status sats_q4_matmul_f32(const sats_q4 *w, const float *x, int B, void *y, int64_t ld_y, int y_f32, void *ws,
                               size_t ws_bytes, void *stream)
{
    return q4_matmul<true>(w, x, B, y, ld_y, y_f32, ws, ws_bytes, stream);
}

}  // extern "C"
