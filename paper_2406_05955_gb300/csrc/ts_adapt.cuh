// ts_adapt.cuh -- helpers of the low-rank adapters' kernels (ts_adapt.cu, ts_adapt_wide.cu, ts_adapt_grads.cu).
#pragma once

#include <atomic>

#include "ts_adapt.h"
#include "ts_grouped.h"
#include "ts_kernels.cuh"

namespace tsffn {
namespace {

constexpr int kThreads = 256;
constexpr int kWarps = kThreads / kWarp;
constexpr int kChunk = 256;  // bytes of a row of x, A, y or out in a chunk
constexpr int kMaxCluster = 8;
constexpr int kSms = 152;

// ---- matrix instructions, asynchronous copies, clusters ---------------------------------------
__device__ __forceinline__ void mma(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
    asm volatile("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
                 : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
                 : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ void ldmatrix4(uint32_t (&v)[4], uint32_t at) {
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0,%1,%2,%3}, [%4];"
                 : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3]) : "r"(at) : "memory");
}
__device__ __forceinline__ void ldmatrix4_t(uint32_t (&v)[4], uint32_t at) {
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0,%1,%2,%3}, [%4];"
                 : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3]) : "r"(at) : "memory");
}
// 16 bytes, or zeros.
__device__ __forceinline__ void copy16(uint32_t to, const void* from, bool in) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(to), "l"(from), "r"(in ? 16 : 0) : "memory");
}
__device__ __forceinline__ void copy4(uint32_t to, const void* from, bool in) {
    asm volatile("cp.async.ca.shared.global [%0], [%1], 4, %2;" ::"r"(to), "l"(from), "r"(in ? 4 : 0) : "memory");
}
__device__ __forceinline__ void copies_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void copies_wait() {
    asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory");
}
__device__ __forceinline__ void copies_wait_all() { asm volatile("cp.async.wait_all;" ::: "memory"); }
// An arrival (one of those that `bar` counts) when the copies that this thread has issued are there.
__device__ __forceinline__ void copies_arrive(uint64_t* bar) {
    asm volatile("cp.async.mbarrier.arrive.noinc.shared::cta.b64 [%0];" ::"r"(smem_u32(bar)) : "memory");
}
__device__ __forceinline__ void cluster_arrive() { asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory"); }
__device__ __forceinline__ void cluster_wait() { asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory"); }
__device__ __forceinline__ uint32_t cluster_rank() {
    uint32_t r;
    asm volatile("mov.u32 %0, %cluster_ctarank;" : "=r"(r));
    return r;
}
__device__ __forceinline__ float4 cluster_ld4(uint32_t at, uint32_t rank) {
    uint32_t a;
    float4 v;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(a) : "r"(at), "r"(rank));
    asm volatile("ld.shared::cluster.v4.f32 {%0,%1,%2,%3}, [%4];" : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w) : "r"(a) : "memory");
    return v;
}

// Byte of 16-byte piece `c` of row `row` in rows of PITCH bytes, pieces permuted so that 8 rows' same piece lie in 8 banks.
template <int PITCH>
__device__ __forceinline__ int place(int row, int c) {
    static_assert(PITCH >= 128, "");
    return row * PITCH + ((c ^ (row & 7)) << 4);
}

// fp32 as a sum of P bf16 numbers, 8 significant bits each; an infinity or NaN is the first alone.
template <int P>
__device__ __forceinline__ void split(float v, __nv_bfloat16 (&p)[P]) {
    p[0] = __float2bfloat16_rn(v);
    const bool finite = fabsf(__bfloat162float(p[0])) < INFINITY;
#pragma unroll
    for (int i = 1; i < P; ++i) {
        v -= __bfloat162float(p[i - 1]);
        p[i] = __float2bfloat16_rn(finite ? v : 0.0f);
    }
}

// ---- the 5th-generation tensor cores (one CTA) ------------------------------------------------
__device__ __forceinline__ bool elect_one() {
    uint32_t p;
    asm volatile("{\n\t.reg .pred p;\n\telect.sync _|p, 0xffffffff;\n\tselp.u32 %0, 1, 0, p;\n\t}" : "=r"(p));
    return p != 0;
}
__device__ __forceinline__ void tc_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tc_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tc_mma(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t accumulate) {
    asm volatile(
        "{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n\t}" ::"r"(d),
        "l"(a), "l"(b), "r"(idesc), "r"(accumulate)
        : "memory");
}
__device__ __forceinline__ void tc_commit(uint64_t* bar) {
    asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(smem_u32(bar)) : "memory");
}
// 32 lanes x 4 or 8 columns, a lane a thread
__device__ __forceinline__ void tc_ld4(uint32_t at, float* v) {
    uint32_t r[4];
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x4.b32 {%0,%1,%2,%3}, [%4];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(at) : "memory");
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = __uint_as_float(r[i]);
}
__device__ __forceinline__ void tc_ld8(uint32_t at, float* v) {
    uint32_t r[8];
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x8.b32 {%0,%1,%2,%3,%4,%5,%6,%7}, [%8];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7])
                 : "r"(at)
                 : "memory");
#pragma unroll
    for (int i = 0; i < 8; ++i) v[i] = __uint_as_float(r[i]);
}
// the values of the loads before: not to be used earlier
template <int N>
__device__ __forceinline__ void tc_ld_wait(float (&v)[N]) {
    asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory");
#pragma unroll
    for (int i = 0; i < N; ++i) asm volatile("" : "+f"(v[i]));
}
// shared-memory descriptors with the 128-byte swizzle: k along the 128-byte rows (atoms of 8 rows, 1024 bytes apart), or 64
// columns along them (8 of k an atom, `block` bytes between blocks of 64 columns)
__device__ __forceinline__ uint64_t desc_k(uint32_t at) {
    return (uint64_t)((at & 0x3FFFFu) >> 4) | (uint64_t)1 << 16 | (uint64_t)(1024 >> 4) << 32 | (uint64_t)1 << 46 | (uint64_t)2 << 61;
}
__device__ __forceinline__ uint64_t desc_n(uint32_t at, uint32_t block) {
    return (uint64_t)((at & 0x3FFFFu) >> 4) | (uint64_t)(block >> 4) << 16 | (uint64_t)(1024 >> 4) << 32 | (uint64_t)1 << 46 |
           (uint64_t)2 << 61;
}
// D fp32, A and B bf16, 128 rows, n columns; whether A's rows and B's columns lie along the 128 bytes (and not k)
constexpr uint32_t idesc(int n, bool a_rows, bool b_columns) {
    return (1u << 4) | (1u << 7) | (1u << 10) | (a_rows ? 1u << 15 : 0u) | (b_columns ? 1u << 16 : 0u) | (uint32_t)(n >> 3) << 17 | (8u << 24);
}

template <int COLUMNS>
__device__ __forceinline__ void tc_alloc(uint32_t* to) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(to)), "r"(COLUMNS) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
}
template <int COLUMNS>
__device__ __forceinline__ void tc_free(uint32_t at) {
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(at), "r"(COLUMNS) : "memory");
}

// The tile of a cluster: up to MT rows of one adapter.
struct TileRows {
    int id, first, count;
};

// By the list: tile number `tile` of all groups' in a row, the rows without an adapter last.
template <int MT>
__device__ __forceinline__ void find_listed(const AdaptLaunch& L, int tile, TileRows* found, int* rows) {
    __shared__ int sums[kWarp];
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    int begin = 0, end = 0;
    if (tid <= L.n_adapters) {
        begin = min(max(L.offsets[tid], 0), L.rows);
        end = min(max(L.offsets[tid + 1], begin), L.rows);
    }
    const int tiles = (end - begin + MT - 1) / MT;
    int upto = tiles;
#pragma unroll
    for (int o = 1; o < kWarp; o <<= 1) {
        const int v = __shfl_up_sync(0xffffffffu, upto, o);
        if (lane >= o) upto += v;
    }
    if (lane == kWarp - 1) sums[warp] = upto;
    if (tid == 0) *found = {-1, 0, 0};
    __syncthreads();
    for (int w = 0; w < warp; ++w) upto += sums[w];
    if (tile < upto && tile >= upto - tiles) {
        const int first = begin + (tile - (upto - tiles)) * MT;
        *found = {tid, first, min(MT, end - first)};
    }
    __syncthreads();
    if (tid < MT) {
        const int row = tid < found->count ? L.list[found->first + tid] : -1;
        rows[tid] = (unsigned)row < (unsigned)L.rows ? row : -1;
    }
}

// Clusters of `ctas` CTAs of a kernel that can be on the device at once: a cluster has to fit into a part of it, so of the
// larger ones there are fewer than the SMs divided by their size (of 8 CTAs, one on an SM: 15 on 152 SMs). Asked for once.
template <typename K>
int resident_clusters(K kernel, int ctas, int threads, int smem, std::atomic<int> (&known)[kMaxCluster + 1]) {
    int n = known[ctas].load(std::memory_order_relaxed);
    if (n == 0) {
        cudaLaunchConfig_t cfg = launch_shape(dim3((unsigned)ctas), threads, nullptr);
        cfg.dynamicSmemBytes = smem;
        cudaLaunchAttribute at{};
        at.id = cudaLaunchAttributeClusterDimension;
        at.val.clusterDim = {(unsigned)ctas, 1, 1};
        cfg.attrs = &at;
        cfg.numAttrs = 1;
        if (cudaOccupancyMaxActiveClusters(&n, kernel, &cfg) != cudaSuccess || n < 1) n = kSms / ctas;
        known[ctas].store(n, std::memory_order_relaxed);
    }
    return n;
}

}  // namespace
}  // namespace tsffn
