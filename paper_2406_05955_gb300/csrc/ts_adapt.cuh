// ts_adapt.cuh -- device helpers of the low-rank adapters' kernels (ts_adapt.cu, ts_adapt_wide.cu).
#pragma once

#include "ts_adapt.h"
#include "ts_kernels.cuh"

namespace tsffn {
namespace {

constexpr int kThreads = 256;
constexpr int kWarps = kThreads / kWarp;
constexpr int kChunk = 256;  // bytes of a row of x, A, y or out in a chunk
constexpr int kMaxCluster = 8;
constexpr int kSms = 152;
constexpr int kResidentCtas = 2 * kSms;

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
__device__ __forceinline__ void ldmatrix2_t(uint32_t (&v)[2], uint32_t at) {
    asm volatile("ldmatrix.sync.aligned.m8n8.x2.trans.shared.b16 {%0,%1}, [%2];" : "=r"(v[0]), "=r"(v[1]) : "r"(at) : "memory");
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

// The tile of a cluster: up to MT rows of one adapter.
struct TileRows {
    int id, rank, first, count;
};

// By the list: tile number `tile` of all groups' in a row, the rows without an adapter last.
template <int MT>
__device__ __forceinline__ void find_listed(const AdaptLaunch& L, int tile, TileRows* found, int* rows) {
    __shared__ int sums[kWarps];
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
    if (tid == 0) *found = {-1, 0, 0, 0};
    __syncthreads();
    for (int w = 0; w < warp; ++w) upto += sums[w];
    if (tile < upto && tile >= upto - tiles) {
        const int first = begin + (tile - (upto - tiles)) * MT;
        *found = {tid, 0, first, min(MT, end - first)};
    }
    __syncthreads();
    if (tid < MT) {
        const int row = tid < found->count ? L.list[found->first + tid] : -1;
        rows[tid] = (unsigned)row < (unsigned)L.rows ? row : -1;
    }
}

}  // namespace
}  // namespace tsffn
