// ts_balance.cu -- how evenly tokens are routed (ts_balance), and the gradient of the router's logits from that and from
// the routing weights (ts_route_backward).
//
//     p[t] = softmax of token t's logits, P_e = mean of p[t][e] over the live tokens, f_e = picks of expert e / all picks
//     loss = E sum_e f_e P_e                       (1 where both are even; picks have no gradient)
//     dlogits[t][e] = dloss E / (picks tokens) p_e (counts_e - sum_j counts_j p_j)
//                     + sum over the picks i of e: w_i (dw_i - sum_j w_j dw_j)
// As many lanes of a token as give each at most 8 experts hold its logits in registers. Sums over tokens are taken in an
// order that depends on the sizes alone, by thread, CTA and over the CTAs, through distributed shared memory where one cluster
// has the tokens and in a second launch otherwise; counts are whole numbers, whose atomics in shared memory give the same
// sums in any order.
//
// Latency bounds both: 8192 tokens of 64 experts are 2 MB. Both of them in a row: 512 tokens, 2 of 8 experts, 9.0 us; 8192, 6
// of 64, 10.9 (three launches).
#include "ts_adapt.h"
#include "ts_grouped.h"
#include "ts_kernels.cuh"

namespace tsffn {
namespace {

constexpr int kPer = 8;  // experts of a lane
constexpr int kThreads = 512;
constexpr int kWarps = kThreads / kWarp;
constexpr int kCluster = 8;
constexpr int kMostCtas = 152;
constexpr int kJoinThreads = 1024;
constexpr int kBackThreads = 128;

__device__ __forceinline__ float max_over(float v, int lanes) {
    for (int o = lanes / 2; o > 0; o >>= 1) v = fmaxf(v, __shfl_xor_sync(0xffffffffu, v, o));
    return v;
}
__device__ __forceinline__ float sum_over(float v, int lanes) {
    for (int o = lanes / 2; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
    return v;
}

// This lane's probabilities of token t (of G lanes, this being number `sub`); whether the token is live: it has a logit that
// is neither -infinity nor NaN, which count for nothing. Infinities share the weight. All lanes of the warp take part.
template <int G>
__device__ __forceinline__ bool probabilities(const float* logits, int n_experts, int t, bool in, int sub, float (&p)[kPer]) {
    const float* x = logits + (size_t)(in ? t : 0) * n_experts + sub * kPer;
    const int n = in ? n_experts - sub * kPer : 0;
    if ((n_experts & 3) == 0 && (reinterpret_cast<uintptr_t>(logits) & 15u) == 0) {
#pragma unroll
        for (int i = 0; i < kPer; i += 4) {
            const float4 f = i < n ? *reinterpret_cast<const float4*>(x + i) : make_float4(-INFINITY, -INFINITY, -INFINITY, -INFINITY);
            p[i] = f.x, p[i + 1] = f.y, p[i + 2] = f.z, p[i + 3] = f.w;
        }
    } else {
#pragma unroll
        for (int i = 0; i < kPer; ++i) p[i] = i < n ? x[i] : -INFINITY;
    }
    float top = -INFINITY;
#pragma unroll
    for (int i = 0; i < kPer; ++i) top = fmaxf(top, p[i]);  // (of a number and NaN, the number)
    top = max_over(top, G);
    float sum = 0.0f;
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
        p[i] = !(p[i] > -INFINITY) ? 0.0f : p[i] == top ? 1.0f : expf(p[i] - top);
        sum += p[i];
    }
    sum = sum_over(sum, G);
    const bool live = top > -INFINITY;
#pragma unroll
    for (int i = 0; i < kPer; ++i) p[i] = live ? __fdiv_rn(p[i], sum) : 0.0f;
    return live;
}

// What a CTA has of its tokens, in shared memory: sums of p, counts, live tokens.
struct Sums {
    float share[kMaxRouteExperts];
    int counts[kMaxRouteExperts];
    int live;
};
// The same as a record of `work`.
__host__ __device__ constexpr int record(int n_experts) { return 2 * n_experts + 1; }

// The outputs, given expert threadIdx.x's sum and count; by the whole CTA, of which the first 256 threads have experts.
__device__ __forceinline__ void finish(const BalanceLaunch& L, float sum, int count, int tokens) {
    constexpr int kW = kMaxRouteExperts / kWarp;
    __shared__ double terms[kW];
    __shared__ int picks[kW];
    const int e = threadIdx.x, lane = e & 31, warp = e >> 5;
    if (warp < kW) {
        const double mean = e < L.n_experts && tokens > 0 ? (double)sum / tokens : 0.0;
        double term = 0.0;
        int n = 0;
        if (e < L.n_experts) {
            L.share[e] = (float)mean;
            L.counts[e] = n = count;
            term = mean * count;
        }
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) term += __shfl_xor_sync(0xffffffffu, term, o);
        n = __reduce_add_sync(0xffffffffu, n);
        if (lane == 0) {
            terms[warp] = term;
            picks[warp] = n;
        }
    }
    __syncthreads();
    if (e == 0) {
        double term = 0.0;
        int n = 0;
#pragma unroll
        for (int w = 0; w < kW; ++w) {
            term += terms[w];
            n += picks[w];
        }
        *L.loss = n > 0 ? (float)(L.n_experts * term / (double)n) : 0.0f;
        L.totals[0] = tokens;
        L.totals[1] = n;
    }
}

__device__ __forceinline__ uint32_t cluster_rank() {
    uint32_t r;
    asm volatile("mov.u32 %0, %cluster_ctarank;" : "=r"(r));
    return r;
}
__device__ __forceinline__ void cluster_sync() {
    asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}
__device__ __forceinline__ uint32_t cluster_ld(const void* p, uint32_t rank) {
    uint32_t a, v;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(a) : "r"(smem_u32(p)), "r"(rank));
    asm volatile("ld.shared::cluster.u32 %0, [%1];" : "=r"(v) : "r"(a) : "memory");
    return v;
}

// JOIN: the grid is one cluster, whose first CTA sums up and finishes; else the sums go to `work`.
template <int G, bool JOIN>
__global__ void __launch_bounds__(kThreads) k_balance(const BalanceLaunch L) {
    __shared__ float sums[kWarps][G * kPer];
    __shared__ Sums all;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, sub = lane % G;
    for (int e = tid; e < kMaxRouteExperts; e += kThreads) all.counts[e] = 0;
    if (tid == 0) all.live = 0;
    __syncthreads();
    pdl_wait();
    pdl_launch_dependents();
    constexpr int kTokens = kThreads / G;  // of a CTA at once
    float sum[kPer] = {};
    int live = 0;
    for (long long t0 = (long long)blockIdx.x * kTokens; t0 < L.tokens; t0 += (long long)gridDim.x * kTokens) {
        const long long t = t0 + tid / G;
        float p[kPer];
        live += probabilities<G>(L.logits, L.n_experts, (int)t, t < L.tokens, sub, p);
#pragma unroll
        for (int i = 0; i < kPer; ++i) sum[i] += p[i];
    }
    const int picks = L.tokens * L.top_k;
#pragma unroll 4
    for (int i = blockIdx.x * kThreads + tid; i < picks; i += gridDim.x * kThreads) {
        const int e = L.sel[i];
        if ((unsigned)e < (unsigned)L.n_experts) atomicAdd(&all.counts[e], 1);
    }
    live = __reduce_add_sync(0xffffffffu, sub == 0 ? live : 0);
    if (lane == 0 && live > 0) atomicAdd(&all.live, live);
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
#pragma unroll
        for (int o = G; o < kWarp; o <<= 1) sum[i] += __shfl_xor_sync(0xffffffffu, sum[i], o);
        if (lane < G) sums[warp][sub * kPer + i] = sum[i];
    }
    __syncthreads();
    if (tid < L.n_experts) {
        float s = 0.0f;
#pragma unroll
        for (int w = 0; w < kWarps; ++w) s += sums[w][tid];
        all.share[tid] = s;
    }
    if constexpr (JOIN) {
        if (gridDim.x > 1) cluster_sync();
        else __syncthreads();
        if (cluster_rank() == 0) {
            float s = 0.0f;
            int n = 0, tokens = 0;
            uint32_t part[kCluster][3];
#pragma unroll
            for (int c = 0; c < kCluster; ++c)
                if (c < (int)gridDim.x && tid < kMaxRouteExperts) {
                    const int e = min(tid, L.n_experts - 1);
                    part[c][0] = cluster_ld(&all.share[e], (uint32_t)c);
                    part[c][1] = cluster_ld(&all.counts[e], (uint32_t)c);
                    part[c][2] = cluster_ld(&all.live, (uint32_t)c);
                }
#pragma unroll
            for (int c = 0; c < kCluster; ++c)
                if (c < (int)gridDim.x && tid < kMaxRouteExperts) {
                    s += __uint_as_float(part[c][0]);
                    n += (int)part[c][1];
                    tokens += (int)part[c][2];
                }
            finish(L, s, n, tokens);
        }
        __syncwarp();
        if (gridDim.x > 1) cluster_sync();  // no CTA leaves while another reads its sums
    } else {
        float* const to = L.work + (size_t)blockIdx.x * record(L.n_experts);
        if (tid < L.n_experts) {
            to[tid] = all.share[tid];
            to[L.n_experts + tid] = __int_as_float(all.counts[tid]);
        }
        if (tid == 0) to[2 * L.n_experts] = __int_as_float(all.live);
    }
}

// E2: experts, rounded up to a power of two; as many threads as there are of those share an expert's records.
template <int E2>
__global__ void __launch_bounds__(kJoinThreads) k_balance_join(const BalanceLaunch L, int ctas) {
    constexpr int kParts = kJoinThreads / E2;
    __shared__ float share[kParts][E2];
    __shared__ int counts[kParts][E2], live[kWarp];
    const int tid = threadIdx.x, e = tid % E2, part = tid / E2, E = L.n_experts;
    pdl_wait();
    pdl_launch_dependents();
    float sum = 0.0f;
    int count = 0, tokens = 0;
    if (e < E) {
#pragma unroll 8
        for (int c = part; c < ctas; c += kParts) {
            const float* from = L.work + (size_t)c * record(E);
            sum += from[e];
            count += __float_as_int(from[E + e]);
        }
    }
    share[part][e] = sum;
    counts[part][e] = count;
    for (int c = tid; c < ctas; c += kJoinThreads) tokens += __float_as_int(L.work[(size_t)c * record(E) + 2 * E]);
    tokens = __reduce_add_sync(0xffffffffu, tokens);
    if ((tid & 31) == 0) live[tid >> 5] = tokens;
    __syncthreads();
    tokens = 0;
#pragma unroll
    for (int w = 0; w < kWarp; ++w) tokens += live[w];
    sum = 0.0f;
    count = 0;
    if (tid < E) {
#pragma unroll 8
        for (int i = 0; i < kParts; ++i) {
            sum += share[i][tid];
            count += counts[i][tid];
        }
    }
    finish(L, sum, count, tokens);
}

template <int G>
__global__ void __launch_bounds__(kBackThreads) k_route_backward(const RouteBackwardLaunch L) {
    const int sub = threadIdx.x % G;
    pdl_wait();
    pdl_launch_dependents();
    const long long i = (long long)blockIdx.x * kBackThreads + threadIdx.x;
    const bool in = i / G < L.tokens;
    const int t = in ? (int)(i / G) : 0, first = sub * kPer;
    // everything that is read, at once
    float w[kMaxRouteK], dw[kMaxRouteK], count[kPer], dloss = 0.0f, tokens = 0.0f, picks = 0.0f;
    int sel[kMaxRouteK];
    const bool balance = L.counts != nullptr, weights = L.dw != nullptr && in;
    const size_t at = (size_t)t * L.top_k;
#pragma unroll
    for (int j = 0; j < kMaxRouteK; ++j) {
        const bool there = weights && j < L.top_k;
        sel[j] = there ? L.sel[at + j] : -1;
        w[j] = there ? L.w[at + j] : 0.0f;
        dw[j] = there ? L.dw[at + j] : 0.0f;
    }
#pragma unroll
    for (int j = 0; j < kPer; ++j) count[j] = balance && first + j < L.n_experts ? (float)L.counts[first + j] : 0.0f;
    if (balance) {
        dloss = *L.dloss;
        tokens = (float)L.totals[0];
        picks = (float)L.totals[1];
    }
    float d[kPer] = {};
    if (balance) {
        float p[kPer], dot = 0.0f;
        probabilities<G>(L.logits, L.n_experts, t, in, sub, p);
        const float f = picks > 0.0f && tokens > 0.0f ? dloss * ((float)L.n_experts / picks / tokens) : 0.0f;
#pragma unroll
        for (int j = 0; j < kPer; ++j) dot = fmaf(count[j], p[j], dot);
        dot = sum_over(dot, G);
#pragma unroll
        for (int j = 0; j < kPer; ++j) d[j] = p[j] > 0.0f ? f * p[j] * (count[j] - dot) : 0.0f;  // (f may be infinite)
    }
    float mean = 0.0f;
#pragma unroll
    for (int j = 0; j < kMaxRouteK; ++j)
        if ((unsigned)sel[j] < (unsigned)L.n_experts) mean = fmaf(w[j], dw[j], mean);
#pragma unroll
    for (int j = 0; j < kMaxRouteK; ++j) {
        const float g = w[j] * (dw[j] - mean);
#pragma unroll
        for (int e = 0; e < kPer; ++e)
            if (sel[j] == first + e && sel[j] < L.n_experts) d[e] += g;
    }
    if (!in) return;
    float* to = L.dlogits + (size_t)t * L.n_experts + first;
    const int n = L.n_experts - first;
    if ((L.n_experts & 3) == 0 && (reinterpret_cast<uintptr_t>(L.dlogits) & 15u) == 0) {
#pragma unroll
        for (int e = 0; e < kPer; e += 4)
            if (e < n) *reinterpret_cast<float4*>(to + e) = make_float4(d[e], d[e + 1], d[e + 2], d[e + 3]);
    } else {
#pragma unroll
        for (int e = 0; e < kPer; ++e)
            if (e < n) to[e] = d[e];
    }
}

int lanes_of(int n_experts) {
    int g = 1;
    while (g * kPer < n_experts) g *= 2;
    return g;
}
// One cluster as long as its threads have one token each in turn, or two: a turn takes 1.5 us, the second launch 4.
bool one_cluster(int tokens, int n_experts) { return (long long)tokens * lanes_of(n_experts) <= 2ll * kCluster * kThreads; }
unsigned balance_ctas(int tokens, int n_experts) {
    const long long ctas = ((long long)tokens * lanes_of(n_experts) + kThreads - 1) / kThreads;
    const long long most = one_cluster(tokens, n_experts) ? kCluster : kMostCtas;
    return (unsigned)(ctas < 1 ? 1 : ctas < most ? ctas : most);
}

template <typename A>
void (*pick(int lanes, void (*const (&k)[6])(A)))(A) {
    int i = 0;
    while (lanes > 1) lanes /= 2, ++i;
    return k[i];
}

}  // namespace

size_t balance_work(int tokens, int n_experts) {
    return one_cluster(tokens, n_experts) ? 0 : (size_t)balance_ctas(tokens, n_experts) * record(n_experts);
}

cudaError_t launch_balance(const BalanceLaunch& a, cudaStream_t stream) {
    static constexpr void (*kJoined[])(BalanceLaunch) = {k_balance<1, true>, k_balance<2, true>, k_balance<4, true>,
                                                         k_balance<8, true>, k_balance<16, true>, k_balance<32, true>};
    static constexpr void (*kApart[])(BalanceLaunch) = {k_balance<1, false>, k_balance<2, false>, k_balance<4, false>,
                                                        k_balance<8, false>, k_balance<16, false>, k_balance<32, false>};
    const unsigned ctas = balance_ctas(a.tokens, a.n_experts);
    const int lanes = lanes_of(a.n_experts);
    if (one_cluster(a.tokens, a.n_experts)) {
        cudaLaunchConfig_t cfg = launch_shape(dim3(ctas), kThreads, stream);
        cudaLaunchAttribute at[2]{};
        at[0].id = cudaLaunchAttributeClusterDimension;
        at[0].val.clusterDim = {ctas, 1, 1};
        at[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
        at[1].val.programmaticStreamSerializationAllowed = 1;
        cfg.attrs = at;
        cfg.numAttrs = 2;
        return cudaLaunchKernelEx(&cfg, pick(lanes, kJoined), a);
    }
    const cudaError_t e = launch_after(pick(lanes, kApart), launch_shape(dim3(ctas), kThreads, stream), a);
    if (e != cudaSuccess) return e;
    const auto join = a.n_experts <= 32 ? k_balance_join<32> : a.n_experts <= 64 ? k_balance_join<64>
                                      : a.n_experts <= 128 ? k_balance_join<128> : k_balance_join<256>;
    return launch_after(join, launch_shape(dim3(1), kJoinThreads, stream), a, (int)ctas);
}

cudaError_t launch_route_backward(const RouteBackwardLaunch& a, cudaStream_t stream) {
    static constexpr void (*kKernels[])(RouteBackwardLaunch) = {k_route_backward<1>, k_route_backward<2>, k_route_backward<4>,
                                                                k_route_backward<8>, k_route_backward<16>, k_route_backward<32>};
    const int g = lanes_of(a.n_experts);
    const long long lanes = (long long)a.tokens * g;
    return launch_after(pick(g, kKernels), launch_shape(dim3((unsigned)((lanes + kBackThreads - 1) / kBackThreads)), kBackThreads, stream), a);
}

}  // namespace tsffn
