// ts_balance.cu -- how evenly tokens are routed (ts_balance), and the gradient of the router's logits from that and from
// the routing weights (ts_route_backward).
//
//     p[t] = softmax of token t's logits, P_e = mean of p[t][e] over the live tokens, f_e = picks of expert e / all picks
//     loss = E sum_e f_e P_e                       (1 where both are even; picks have no gradient)
//     dlogits[t][e] = dloss E / (picks tokens) p_e (counts_e - sum_j counts_j p_j)
//                     + sum over the picks i of e: w_i (dw_i - sum_j w_j dw_j)
// As many lanes of a token as give each at most 8 experts hold its logits in registers. Sums over tokens are taken in an
// order that depends on the sizes alone, by thread, CTA and, in a second launch, over the CTAs; counts are whole numbers,
// whose atomics in shared memory give the same sums in any order.
#include "ts_adapt.h"
#include "ts_grouped.h"
#include "ts_kernels.cuh"

namespace tsffn {
namespace {

constexpr int kPer = 8;  // experts of a lane
constexpr int kThreads = 256;
constexpr int kWarps = kThreads / kWarp;
constexpr int kMostCtas = 152;
constexpr int kJoinThreads = 1024;

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

// Sums of p over a CTA's tokens [n_experts], then its counts and its live tokens, as one record of `work`.
__host__ __device__ constexpr int record(int n_experts) { return 2 * n_experts + 1; }

template <int G>
__global__ void __launch_bounds__(kThreads) k_balance(const BalanceLaunch L) {
    __shared__ float sums[kWarps][kMaxRouteExperts];
    __shared__ int counts[kMaxRouteExperts], live_tokens;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, sub = lane % G;
    for (int e = tid; e < kMaxRouteExperts; e += kThreads) counts[e] = 0;
    if (tid == 0) live_tokens = 0;
    __syncthreads();
    pdl_wait();
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
    const long long picks = (long long)L.tokens * L.top_k;
    for (long long i = (long long)blockIdx.x * kThreads + tid; i < picks; i += (long long)gridDim.x * kThreads) {
        const int e = L.sel[i];
        if ((unsigned)e < (unsigned)L.n_experts) atomicAdd(&counts[e], 1);
    }
    if (sub == 0 && live > 0) atomicAdd(&live_tokens, live);
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
#pragma unroll
        for (int o = G; o < kWarp; o <<= 1) sum[i] += __shfl_xor_sync(0xffffffffu, sum[i], o);
        if (lane < G) sums[warp][sub * kPer + i] = sum[i];
    }
    __syncthreads();
    float* to = L.work + (size_t)blockIdx.x * record(L.n_experts);
    for (int e = tid; e < L.n_experts; e += kThreads) {
        float s = 0.0f;
#pragma unroll
        for (int w = 0; w < kWarps; ++w) s += sums[w][e];
        to[e] = s;
        to[L.n_experts + e] = __int_as_float(counts[e]);
    }
    if (tid == 0) to[2 * L.n_experts] = __int_as_float(live_tokens);
}

__global__ void __launch_bounds__(kJoinThreads) k_balance_join(const BalanceLaunch L, int ctas) {
    constexpr int kParts = kJoinThreads / kMaxRouteExperts;
    __shared__ float share[kParts][kMaxRouteExperts];
    __shared__ int counts[kParts][kMaxRouteExperts], live[kWarp];
    __shared__ double terms[kMaxRouteExperts];
    __shared__ long long picks_of[kMaxRouteExperts];
    const int tid = threadIdx.x, e = tid % kMaxRouteExperts, part = tid / kMaxRouteExperts, E = L.n_experts;
    pdl_wait();
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
    if (part == 0) {
#pragma unroll
        for (int i = 1; i < kParts; ++i) {
            sum += share[i][e];
            count += counts[i][e];
        }
        const double mean = tokens > 0 ? (double)sum / tokens : 0.0;
        if (e < E) {
            L.share[e] = (float)mean;
            L.counts[e] = count;
        }
        terms[e] = e < E ? mean * count : 0.0;
        picks_of[e] = e < E ? count : 0;
    }
    __syncthreads();
    for (int half = kMaxRouteExperts / 2; half > 0; half /= 2) {
        if (tid < half) {
            terms[tid] += terms[tid + half];
            picks_of[tid] += picks_of[tid + half];
        }
        __syncthreads();
    }
    if (tid == 0) {
        *L.loss = picks_of[0] > 0 ? (float)(E * terms[0] / (double)picks_of[0]) : 0.0f;
        L.totals[0] = tokens;
        L.totals[1] = (int)picks_of[0];
    }
}

template <int G>
__global__ void __launch_bounds__(kThreads) k_route_backward(const RouteBackwardLaunch L) {
    const int sub = threadIdx.x % G;
    pdl_wait();
    const long long i = (long long)blockIdx.x * kThreads + threadIdx.x;
    const bool in = i / G < L.tokens;
    const int t = in ? (int)(i / G) : 0, first = sub * kPer;
    float d[kPer] = {};
    if (L.counts != nullptr) {
        float p[kPer], count[kPer], dot = 0.0f;
        probabilities<G>(L.logits, L.n_experts, t, in, sub, p);
        const float tokens = (float)L.totals[0], picks = (float)L.totals[1];
        const float f = picks > 0.0f && tokens > 0.0f ? *L.dloss * ((float)L.n_experts / picks / tokens) : 0.0f;
#pragma unroll
        for (int j = 0; j < kPer; ++j) {
            count[j] = first + j < L.n_experts ? (float)L.counts[first + j] : 0.0f;
            dot = fmaf(count[j], p[j], dot);
        }
        dot = sum_over(dot, G);
#pragma unroll
        for (int j = 0; j < kPer; ++j) d[j] = f * p[j] * (count[j] - dot);
    }
    if (L.dw != nullptr && in) {
        const size_t at = (size_t)t * L.top_k;
        float mean = 0.0f, w[kMaxRouteK], dw[kMaxRouteK];
        int sel[kMaxRouteK];
#pragma unroll
        for (int j = 0; j < kMaxRouteK; ++j) {
            sel[j] = j < L.top_k ? L.sel[at + j] : -1;
            const bool some = (unsigned)sel[j] < (unsigned)L.n_experts;
            w[j] = some ? L.w[at + j] : 0.0f;
            dw[j] = some ? L.dw[at + j] : 0.0f;
            mean = fmaf(w[j], dw[j], mean);
        }
#pragma unroll
        for (int j = 0; j < kMaxRouteK; ++j)
#pragma unroll
            for (int e = 0; e < kPer; ++e)
                if (sel[j] == first + e && sel[j] < L.n_experts) d[e] = fmaf(w[j], dw[j] - mean, d[e]);
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
unsigned balance_ctas(int tokens, int n_experts) {
    const long long ctas = ((long long)tokens * lanes_of(n_experts) + kThreads - 1) / kThreads;
    return (unsigned)(ctas < 1 ? 1 : ctas < kMostCtas ? ctas : kMostCtas);
}

template <typename A>
void (*pick(int lanes, void (*const (&k)[6])(A)))(A) {
    int i = 0;
    while (lanes > 1) lanes /= 2, ++i;
    return k[i];
}

}  // namespace

size_t balance_work(int tokens, int n_experts) { return (size_t)balance_ctas(tokens, n_experts) * record(n_experts); }

cudaError_t launch_balance(const BalanceLaunch& a, cudaStream_t stream) {
    static constexpr void (*kKernels[])(BalanceLaunch) = {k_balance<1>, k_balance<2>, k_balance<4>,
                                                          k_balance<8>, k_balance<16>, k_balance<32>};
    const unsigned ctas = balance_ctas(a.tokens, a.n_experts);
    const cudaError_t e = launch_after(pick(lanes_of(a.n_experts), kKernels), launch_shape(dim3(ctas), kThreads, stream), a);
    if (e != cudaSuccess) return e;
    return launch_after(k_balance_join, launch_shape(dim3(1), kJoinThreads, stream), a, (int)ctas);
}

cudaError_t launch_route_backward(const RouteBackwardLaunch& a, cudaStream_t stream) {
    static constexpr void (*kKernels[])(RouteBackwardLaunch) = {k_route_backward<1>, k_route_backward<2>, k_route_backward<4>,
                                                                k_route_backward<8>, k_route_backward<16>, k_route_backward<32>};
    const int g = lanes_of(a.n_experts);
    const long long lanes = (long long)a.tokens * g;
    return launch_after(pick(g, kKernels), launch_shape(dim3((unsigned)((lanes + kThreads - 1) / kThreads)), kThreads, stream), a);
}

}  // namespace tsffn
