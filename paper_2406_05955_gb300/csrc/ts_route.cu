// ts_route.cu -- routing of many tokens (Sec. 4: top_k of the experts by router logit, softmax over the picked ones).
//
// Picking: as many lanes of a token as give each at most 8 experts hold its logits in registers; top_k rounds of a
// maximum over them (a lower expert wins a tie). Placing: the picks are sorted by expert, in token order, by a counting
// sort of one cluster of CTAs: every warp counts the picks of its own contiguous part, the counts are summed over the
// warps and, through distributed shared memory, over the CTAs, and a pick's row is its expert's first row plus the
// picks of that expert before it. Nothing is atomic, so rows do not depend on timing, and no scratch is needed.
// Few tokens are picked by the CTA that places them: one launch instead of two.
//
// Latency bounds it: logits and lists are 2.9 MB for 8192 tokens of 64 experts, 0.4 us of memory time; picking and the
// placing's chain of counts, cluster barrier and scan take 10.1 us (4 tokens of 8 experts: 3.7).
#include "ts_grouped.h"
#include "ts_kernels.cuh"

namespace tsffn {
namespace {

constexpr int kPer = 8;  // experts of a lane
constexpr int kPickThreads = 128;
constexpr int kPlaceThreads = 1024;
constexpr int kPlaceWarps = kPlaceThreads / kWarp;
constexpr int kPlaceCtas = 8, kPlaceMost = 16;  // CTAs of the cluster

// The picks of token t by G lanes of a warp, of which this is lane `sub`; all lanes of the warp take part (t may be
// behind the last token).
template <int G>
__device__ __forceinline__ void pick(const RouteLaunch& L, int t, int sub) {
    const bool in = t < L.tokens;
    float v[kPer];
    const float* x = L.logits + (size_t)(in ? t : 0) * L.n_experts + sub * kPer;
    const int n = in ? L.n_experts - sub * kPer : 0;  // experts from this lane's on
    if ((L.n_experts & 3) == 0 && (reinterpret_cast<uintptr_t>(L.logits) & 15u) == 0) {
#pragma unroll
        for (int i = 0; i < kPer; i += 4) {
            const float4 f = i < n ? *reinterpret_cast<const float4*>(x + i) : make_float4(-INFINITY, -INFINITY, -INFINITY, -INFINITY);
            v[i] = f.x, v[i + 1] = f.y, v[i + 2] = f.z, v[i + 3] = f.w;
        }
    } else {
#pragma unroll
        for (int i = 0; i < kPer; ++i) v[i] = i < n ? x[i] : -INFINITY;
    }
    // keys that order as the numbers do; 0 for what is never picked (-infinity, NaN)
    unsigned key[kPer];
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
        const unsigned u = __float_as_uint(v[i] + 0.0f);  // (-0 is 0)
        key[i] = v[i] > -INFINITY ? ((u >> 31) ? ~u : u | 0x80000000u) : 0u;
    }
    // A round: the lanes' largest keys, the largest of the token's, and the first lane that has it, whose first expert with
    // it is picked. That lane stores it; all know the number.
    const unsigned group = (G == 32 ? 0xffffffffu : (1u << (G & 31)) - 1u) << ((threadIdx.x & 31) / G * G);
    float val[kMaxRouteK], top = 0.0f, sum = 0.0f;
#pragma unroll
    for (int j = 0; j < kMaxRouteK; ++j) {
        val[j] = 0.0f;
        if (j >= L.top_k) break;
        unsigned mine = key[0];
        int at = 0;
#pragma unroll
        for (int i = 1; i < kPer; ++i)
            if (key[i] > mine) {
                mine = key[i];
                at = i;
            }
        unsigned best = mine;
        if constexpr (G == 32) {
            best = __reduce_max_sync(0xffffffffu, mine);
        } else {
#pragma unroll
            for (int o = G / 2; o > 0; o >>= 1) best = max(best, __shfl_xor_sync(0xffffffffu, best, o));
        }
        bool winner = true;
        if constexpr (G > 1)
            winner = (threadIdx.x & 31) == (unsigned)__ffs(__ballot_sync(0xffffffffu, mine == best) & group) - 1u;
        if (winner && in) L.sel[(size_t)t * L.top_k + j] = best ? sub * kPer + at : -1;
        if (best) {
            const float b = __uint_as_float((best >> 31) ? best & 0x7fffffffu : ~best);
            if (j == 0) top = b;
            val[j] = b == top ? 1.0f : expf(b - top);  // (infinity - infinity among the first)
            sum += val[j];
        }
#pragma unroll
        for (int i = 0; i < kPer; ++i)
            if (winner && i == at) key[i] = 0u;
    }
    if (in && sub == 0)
#pragma unroll
        for (int j = 0; j < kMaxRouteK; ++j)
            if (j < L.top_k) L.w[(size_t)t * L.top_k + j] = val[j] > 0.0f ? __fdiv_rn(val[j], sum) : 0.0f;
}

template <int G>
__global__ void __launch_bounds__(kPickThreads) k_route_pick(const RouteLaunch L) {
    pdl_launch_dependents();  // the placing CTAs set up meanwhile
    pdl_wait();
    const long long i = (long long)blockIdx.x * kPickThreads + threadIdx.x;
    pick<G>(L, (int)(i / G), (int)(i % G));
}

__device__ __forceinline__ uint32_t cluster_rank() {
    uint32_t r;
    asm volatile("mov.u32 %0, %cluster_ctarank;" : "=r"(r));
    return r;
}
__device__ __forceinline__ uint32_t cluster_size() {
    uint32_t r;
    asm volatile("mov.u32 %0, %cluster_nctarank;" : "=r"(r));
    return r;
}
__device__ __forceinline__ void cluster_sync() {
    asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}
__device__ __forceinline__ int cluster_ld(const int* p, uint32_t rank) {
    uint32_t a;
    int v;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(a) : "r"(smem_u32(p)), "r"(rank));
    asm volatile("ld.shared::cluster.s32 %0, [%1];" : "=r"(v) : "r"(a) : "memory");
    return v;
}

// The lanes of the warp with the same expert as this one (e < 2^bits; -1: no pick, whose mask is not used), by a ballot a
// bit (8192 tokens, 6 of 64 experts: 17.6 us, 19.3 with __match_any_sync).
__device__ __forceinline__ unsigned same_expert(int e, int bits) {
    unsigned same = __ballot_sync(0xffffffffu, e >= 0);
    for (int b = 0; b < bits; ++b) {
        const bool set = (e >> b) & 1;
        const unsigned votes = __ballot_sync(0xffffffffu, set);
        same &= set ? votes : ~votes;
    }
    return same;
}

// The picks i, i + 32, ... of a lane, all on their way at once; -1 behind the last one.
constexpr int kAhead = 8;
__device__ __forceinline__ void load_picks(const RouteLaunch& L, int i, int end, int (&e)[kAhead]) {
#pragma unroll
    for (int u = 0; u < kAhead; ++u) e[u] = i + u * kWarp < end ? L.sel[i + u * kWarp] : -1;
}

// G > 0: picks first (one CTA).
template <int G>
__global__ void __launch_bounds__(kPlaceThreads) k_route_place(const RouteLaunch L) {
    __shared__ int count[kPlaceWarps][kMaxRouteExperts];
    __shared__ int total_here[kMaxRouteExperts], first[kMaxRouteExperts], sums[kMaxRouteExperts / kWarp];
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, E = L.n_experts;
    if constexpr (G > 0) {
        pdl_wait();
        for (int i = tid; i - tid < L.tokens * G; i += kPlaceThreads) pick<G>(L, i / G, i % G);
        __syncthreads();  // (orders the picks' stores before the loads below)
    }
    const uint32_t rank = cluster_rank(), ctas = cluster_size();
    const int bits = 32 - __clz(E - 1);
    const int total = L.tokens * L.top_k;
    const int part = (int)(((long long)total + ctas * kPlaceThreads - 1) / (ctas * kPlaceThreads)) * kWarp;  // of a warp
    const int begin = (int)min((long long)total, (long long)(rank * kPlaceWarps + warp) * part);
    const int end = min(total, begin + part);
    for (int e = lane; e < E; e += kWarp) count[warp][e] = 0;
    __syncwarp();
    if constexpr (G == 0) pdl_wait();  // for the picks
    for (int i0 = begin; i0 < end; i0 += kAhead * kWarp) {
        int es[kAhead];
        load_picks(L, i0 + lane, end, es);
#pragma unroll
        for (int u = 0; u < kAhead; ++u) {
            if (i0 + u * kWarp >= end) break;
            const unsigned same = same_expert(es[u], bits);
            if (es[u] >= 0 && (same & ((1u << lane) - 1u)) == 0u) count[warp][es[u]] += __popc(same);
            __syncwarp();
        }
    }
    __syncthreads();
    if (tid < E) {  // the counts of the warps before, and the CTA's
        int sum = 0;
#pragma unroll 8
        for (int w = 0; w < kPlaceWarps; ++w) {
            const int c = count[w][tid];
            count[w][tid] = sum;
            sum += c;
        }
        total_here[tid] = sum;
    }
    int before = 0, all = 0;  // of expert tid: in the CTAs before, and in all
    if (ctas > 1) {
        cluster_sync();
        if (tid < E)
            for (uint32_t c = 0; c < ctas; ++c) {
                const int v = cluster_ld(&total_here[tid], c);
                before += c < rank ? v : 0;
                all += v;
            }
        cluster_sync();  // no CTA leaves while another reads its counts
    } else if (tid < E) {
        all = total_here[tid];
    }
    // first rows: an exclusive scan over the experts, by the first 8 warps
    int scan = all;
    if (tid < kMaxRouteExperts) {
#pragma unroll
        for (int o = 1; o < kWarp; o <<= 1) {
            const int v = __shfl_up_sync(0xffffffffu, scan, o);
            if (lane >= o) scan += v;
        }
        if (lane == kWarp - 1) sums[warp] = scan;
    }
    __syncthreads();
    if (tid < kMaxRouteExperts) {
        for (int w = 0; w < warp; ++w) scan += sums[w];
        if (tid < E) {
            first[tid] = scan - all + before;
            if (rank == 0) L.offsets[tid + 1] = scan;
        }
        if (tid == 0 && rank == 0) {
            L.offsets[0] = 0;
            if (L.shape != nullptr) L.shape[0] = L.tokens, L.shape[1] = L.top_k;
        }
    }
    __syncthreads();
    for (int i0 = begin; i0 < end; i0 += kAhead * kWarp) {
        int es[kAhead];
        load_picks(L, i0 + lane, end, es);
#pragma unroll
        for (int u = 0; u < kAhead; ++u) {
            const int i = i0 + u * kWarp + lane, e = es[u];
            if (i0 + u * kWarp >= end) break;
            const unsigned same = same_expert(e, bits);
            const unsigned ahead = same & ((1u << lane) - 1u);
            const int at = e >= 0 ? first[e] + count[warp][e] + __popc(ahead) : -1;
            __syncwarp();
            if (e >= 0) {
                if (ahead == 0u) count[warp][e] += __popc(same);
                L.rows[at] = (int32_t)((unsigned)i / (unsigned)L.top_k);
            }
            if (i < end) L.slots[i] = at;
            __syncwarp();
        }
    }
}

template <int G>
cudaError_t launch(const RouteLaunch& a, cudaStream_t stream) {
    // One launch as long as the one CTA picks in one round. Calls among others on a stream, which the caller bounds: 4 and 1024
    // tokens of 8 experts and 128 of 64 take 6.8 us so and 8.8 in two launches. In a graph: 3.7 us (in two launches 3.9), 5.5 (5.0)
    // and 6.8 (5.6); beyond one round the CTA falls behind: 2048 tokens of 8 experts 8.5 (5.2), 512 of 64 20.0 (6.5).
    const bool fused = (long long)a.tokens * G <= kPlaceThreads;
    if (fused) return launch_after(k_route_place<G>, launch_shape(dim3(1), kPlaceThreads, stream), a);
    const long long lanes = (long long)a.tokens * G;
    const cudaError_t picked = launch_after(
        k_route_pick<G>, launch_shape(dim3((unsigned)((lanes + kPickThreads - 1) / kPickThreads)), kPickThreads, stream), a);
    if (picked != cudaSuccess) return picked;
    // 16 CTAs from 16384 picks on: 8192 tokens, 6 of 64 experts, 14.5 -> 11.9 us; 4096 tokens, 2 of 8, 6.8 -> 7.1.
    const unsigned ctas = (long long)a.tokens * a.top_k >= 16384 ? kPlaceMost : kPlaceCtas;
    if (ctas > kPlaceCtas) {
        const cudaError_t e = cudaFuncSetAttribute(k_route_place<0>, cudaFuncAttributeNonPortableClusterSizeAllowed, 1);
        if (e != cudaSuccess) return e;
    }
    cudaLaunchConfig_t cfg = launch_shape(dim3(ctas), kPlaceThreads, stream);
    cudaLaunchAttribute at[2]{};
    at[0].id = cudaLaunchAttributeClusterDimension;
    at[0].val.clusterDim = {ctas, 1, 1};
    at[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at[1].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = at;
    cfg.numAttrs = 2;
    return cudaLaunchKernelEx(&cfg, k_route_place<0>, a);
}

}  // namespace

cudaError_t launch_route(const RouteLaunch& a, cudaStream_t stream) {
    const int lanes = (a.n_experts + kPer - 1) / kPer;
    if (lanes <= 1) return launch<1>(a, stream);
    if (lanes <= 2) return launch<2>(a, stream);
    if (lanes <= 4) return launch<4>(a, stream);
    if (lanes <= 8) return launch<8>(a, stream);
    if (lanes <= 16) return launch<16>(a, stream);
    return launch<32>(a, stream);
}

}  // namespace tsffn
