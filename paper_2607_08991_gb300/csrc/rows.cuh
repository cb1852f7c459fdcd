// rows.cuh -- rows of vocabulary logits on a thread-block cluster (sm_103a): what the kernels of distill.cu and
// logits.cuh share.
//
// A row of V logits (bf16 or fp32) is cut into granules of 16 bytes on the row's own 16-byte boundaries, so that a
// row that starts anywhere still moves in whole vectors; the places of the first and last granule that lie outside
// the row read as -inf.  The C CTAs of a cluster take consecutive runs of granules.
#pragma once

#include <atomic>
#include <cstdint>
#include <cuda_runtime.h>

#include "common.cuh"

namespace sats {

constexpr int kRowMaxCluster = 8;   // the portable limit

template <bool F32>
struct RowElem {
    static constexpr int kBytes = F32 ? 4 : 2;
    static constexpr int kPer = 16 / kBytes;   // elements of a granule
};

template <bool F32>
struct Row {
    const char *base;   // the first granule (16-byte aligned)
    int head;           // elements of it that lie before the row
    int V;
    int G;              // granules

    __device__ __forceinline__ Row(const void *logits, int64_t row, int64_t ld, int v)
    {
        constexpr int B = RowElem<F32>::kBytes, E = RowElem<F32>::kPer;
        const uintptr_t a = reinterpret_cast<uintptr_t>(logits) + (uintptr_t)(row * ld) * B;
        head = (int)(a & 15u) / B;
        base = reinterpret_cast<const char *>(a & ~(uintptr_t)15);
        V = v;
        G = (int)(((int64_t)head + v + E - 1) / E);
    }
    // Vocabulary index of a granule's first element (below 0 in the first granule of a row that starts inside it).
    __device__ __forceinline__ int first(int g) const { return (int)((unsigned)g * RowElem<F32>::kPer - (unsigned)head); }
    __device__ __forceinline__ bool inside(int idx) const { return (unsigned)idx < (unsigned)V; }
    // Whether the granule is all row.
    __device__ __forceinline__ bool whole(int g) const
    {
        const int f = first(g);
        return f >= 0 && f <= V - RowElem<F32>::kPer;
    }
};

// Streaming loads: a row is read once (and, by the calls that may work in place, written afterwards: not the
// read-only path).
__device__ __forceinline__ uint4 ld_row_v4(const void *p)
{
    uint4 v;
    asm volatile("ld.global.L1::no_allocate.v4.u32 {%0, %1, %2, %3}, [%4];"
                 : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w)
                 : "l"(p)
                 : "memory");
    return v;
}

template <bool F32>
__device__ __noinline__ uint4 load_edge_granule(const char *base, int first, int V, int g)
{
    constexpr int E = RowElem<F32>::kPer;
    uint32_t w[4];
    if constexpr (F32) {
        const volatile uint32_t *p = reinterpret_cast<const volatile uint32_t *>(base) + (size_t)g * E;
#pragma unroll
        for (int j = 0; j < 4; ++j) w[j] = (unsigned)(first + j) < (unsigned)V ? p[j] : 0xff800000u;
    } else {
        const volatile uint16_t *p = reinterpret_cast<const volatile uint16_t *>(base) + (size_t)g * E;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const uint32_t lo = (unsigned)(first + 2 * j) < (unsigned)V ? p[2 * j] : 0xff80u;
            const uint32_t hi = (unsigned)(first + 2 * j + 1) < (unsigned)V ? p[2 * j + 1] : 0xff80u;
            w[j] = lo | (hi << 16);
        }
    }
    return make_uint4(w[0], w[1], w[2], w[3]);
}

template <bool F32>
__device__ __forceinline__ uint4 load_granule(const Row<F32> &r, int g)
{
    if (r.whole(g)) return ld_row_v4(r.base + (size_t)g * 16);
    return load_edge_granule<F32>(r.base, r.first(g), r.V, g);
}

// 16 bytes global -> shared without a register in between; both 16-byte aligned.
__device__ __forceinline__ void cp_async16(void *dst, const void *src)
{
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(smem_addr(dst)), "l"(src) : "memory");
}
__device__ __forceinline__ void cp_async4(void *dst, const void *src)   // (4 bytes)
{
    asm volatile("cp.async.ca.shared.global [%0], [%1], 4;" ::"r"(smem_addr(dst)), "l"(src) : "memory");
}
__device__ __forceinline__ void cp_async_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void cp_async_wait()
{
    asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory");
}

// Brings granule g of the row to dst; complete after a cp_async_wait of this thread.
template <bool F32>
__device__ __forceinline__ void fetch_granule(const Row<F32> &r, int g, uint4 *dst)
{
    if (r.whole(g)) cp_async16(dst, r.base + (size_t)g * 16);
    else *dst = load_edge_granule<F32>(r.base, r.first(g), r.V, g);
}

// Both halves at once, each rounded once.
__device__ __forceinline__ f32x2 fadd2(f32x2 a, f32x2 b)
{
    f32x2 d;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(a), "l"(b));
    return d;
}
__device__ __forceinline__ f32x2 fmul2(f32x2 a, f32x2 b)
{
    f32x2 d;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(a), "l"(b));
    return d;
}

// A granule's elements as pairs of floats.
template <bool F32>
__device__ __forceinline__ void granule_pairs(const uint4 &v, f32x2 (&f)[RowElem<F32>::kPer / 2])
{
    if constexpr (F32) {
        f[0] = pack2(__uint_as_float(v.x), __uint_as_float(v.y));
        f[1] = pack2(__uint_as_float(v.z), __uint_as_float(v.w));
    } else {
        f[0] = bf16x2_to_f32x2(v.x);
        f[1] = bf16x2_to_f32x2(v.y);
        f[2] = bf16x2_to_f32x2(v.z);
        f[3] = bf16x2_to_f32x2(v.w);
    }
}

template <bool F32>
__device__ __forceinline__ void granule_floats(const uint4 &v, float (&f)[RowElem<F32>::kPer])
{
    if constexpr (F32) {
        f[0] = __uint_as_float(v.x);
        f[1] = __uint_as_float(v.y);
        f[2] = __uint_as_float(v.z);
        f[3] = __uint_as_float(v.w);
    } else {
        unpack8(v, f);
    }
}

// Larger of two bf16 pairs; a NaN gives way to a number.
__device__ __forceinline__ uint32_t bf16x2_max(uint32_t a, uint32_t b)
{
    uint32_t d;
    asm("max.bf16x2 %0, %1, %2;" : "=r"(d) : "r"(a), "r"(b));
    return d;
}

// The granule's largest element (a NaN gives way to a number; -inf if nothing is larger).
template <bool F32>
__device__ __forceinline__ float granule_max(const uint4 &v)
{
    if constexpr (F32) {
        return fmaxf(fmaxf(__uint_as_float(v.x), __uint_as_float(v.y)), fmaxf(__uint_as_float(v.z), __uint_as_float(v.w)));
    } else {
        const uint32_t m = bf16x2_max(bf16x2_max(v.x, v.y), bf16x2_max(v.z, v.w));
        return fmaxf(bf16_lo(m), bf16_hi(m));
    }
}

// ------------------------------------------------------------------ clusters
// A barrier of all threads of all CTAs of the cluster, in two halves.  A kernel arrives at its start and waits before
// it first reaches another CTA's memory: that CTA has to run by then.
__device__ __forceinline__ void cluster_arrive() { asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory"); }
__device__ __forceinline__ void cluster_wait() { asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory"); }

// Both together; orders shared-memory accesses across the cluster.
__device__ __forceinline__ void cluster_sync_all()
{
    cluster_arrive();
    cluster_wait();
}

// The address, in CTA `rank` of the cluster, of what `p` is in this CTA.
__device__ __forceinline__ uint32_t peer_addr(const void *p, unsigned rank)
{
    uint32_t r;
    asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(r) : "r"(smem_addr(p)), "r"(rank));
    return r;
}
__device__ __forceinline__ void st_peer_u32(uint32_t addr, uint32_t v)
{
    asm volatile("st.shared::cluster.u32 [%0], %1;" ::"r"(addr), "r"(v) : "memory");
}
__device__ __forceinline__ void st_peer_u64(uint32_t addr, uint64_t v)
{
    asm volatile("st.shared::cluster.u64 [%0], %1;" ::"r"(addr), "l"(v) : "memory");
}
__device__ __forceinline__ void st_peer_v4(uint32_t addr, float a, float b, float c, float d)
{
    asm volatile("st.shared::cluster.v4.f32 [%0], {%1, %2, %3, %4};" ::"r"(addr), "f"(a), "f"(b), "f"(c), "f"(d)
                 : "memory");
}

// The same without a barrier: counts 16 bytes on the mbarrier `bar` of the CTA written to (both addresses its).
__device__ __forceinline__ void st_async_v4(uint32_t addr, float a, float b, float c, float d, uint32_t bar)
{
    asm volatile("st.async.shared::cluster.mbarrier::complete_tx::bytes.v4.f32 [%0], {%1, %2, %3, %4}, [%5];"
                 ::"r"(addr), "f"(a), "f"(b), "f"(c), "f"(d), "r"(bar)
                 : "memory");
}

// 2^x (2 ulp; results below the normal range are 0).
__device__ __forceinline__ float ex2_approx(float x)
{
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

// ------------------------------------------------------------------ launches (host)
// Shared memory that a CTA may have, less what the system takes.
constexpr size_t kSmemPerCta = 227 * 1024;

// Lets Kern have up to max_smem bytes of dynamic shared memory on the current device; asked once per device.
template <auto Kern>
cudaError_t allow_smem(size_t max_smem)
{
    static std::atomic<uint64_t> done{0};
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return e;
    const uint64_t bit = 1ull << (dev & 63);
    if (dev < 64 && (done.load(std::memory_order_relaxed) & bit)) return cudaSuccess;
    e = cudaFuncSetAttribute(Kern, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)max_smem);
    if (e == cudaSuccess && dev < 64) done.fetch_or(bit, std::memory_order_relaxed);
    return e;
}

struct ClusterConfig {
    cudaLaunchConfig_t cfg = {};
    cudaLaunchAttribute attr[1];

    ClusterConfig(int64_t ctas, int threads, size_t smem, int cluster, cudaStream_t st)
    {
        cfg.gridDim = dim3((unsigned)ctas);
        cfg.blockDim = dim3(threads);
        cfg.dynamicSmemBytes = smem;
        cfg.stream = st;
        attr[0].id = cudaLaunchAttributeClusterDimension;
        attr[0].val.clusterDim.x = (unsigned)cluster;
        attr[0].val.clusterDim.y = 1;
        attr[0].val.clusterDim.z = 1;
        cfg.attrs = attr;
        cfg.numAttrs = 1;
    }
};

// Launches Kern with `ctas` CTAs in clusters of `cluster`; max_smem: the most dynamic shared memory it is ever given.
template <auto Kern, typename P>
cudaError_t launch_clusters(int64_t ctas, int threads, size_t smem, size_t max_smem, int cluster, cudaStream_t st,
                            const P &p)
{
    const cudaError_t e = allow_smem<Kern>(max_smem);
    if (e != cudaSuccess) return e;
    ClusterConfig c(ctas, threads, smem, cluster, st);
    return cudaLaunchKernelEx(&c.cfg, Kern, p);
}

// Clusters of this shape that the current device holds at a time (the last answer is kept per host thread).
template <auto Kern>
cudaError_t resident_clusters(int threads, size_t smem, size_t max_smem, int cluster, int *n)
{
    struct Last {
        int dev = -1, cluster = 0, n = 0;
        size_t smem = 0;
    };
    static thread_local Last last;
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return e;
    if (last.dev != dev || last.cluster != cluster || last.smem != smem) {
        e = allow_smem<Kern>(max_smem);
        if (e != cudaSuccess) return e;
        ClusterConfig c((int64_t)cluster, threads, smem, cluster, nullptr);
        int got = 0;
        e = cudaOccupancyMaxActiveClusters(&got, Kern, &c.cfg);
        if (e != cudaSuccess) return e;
        last.dev = dev;
        last.cluster = cluster;
        last.smem = smem;
        last.n = got;
    }
    *n = last.n;
    return cudaSuccess;
}

}  // namespace sats
