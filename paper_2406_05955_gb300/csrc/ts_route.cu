// ts_route.cu -- routing of many tokens (Sec. 4: top_k of the experts by router logit, softmax over the picked ones):
// k_route_pick chooses each token's experts, k_route_place sorts the picks by expert, in token order. The sort is a
// counting sort: every warp counts the picks of its own contiguous part, the counts are summed in order, and a pick's
// row is its expert's first row plus the picks of that expert before it. Nothing is atomic, so rows do not depend on
// timing.
#include "ts_grouped.h"
#include "ts_kernels.cuh"

namespace tsffn {
namespace {

constexpr int kPlaceThreads = 1024;
constexpr int kPlaceWarps = kPlaceThreads / kWarp;

// One token a thread: top_k rounds of the largest logit left.
__global__ void __launch_bounds__(128) k_route_pick(const RouteLaunch L) {
    const int t = blockIdx.x * 128 + threadIdx.x;
    if (t >= L.tokens) return;
    const float* x = L.logits + (size_t)t * L.n_experts;
    int sel[kMaxRouteK];
    float v[kMaxRouteK];
    int n = 0;
    for (; n < L.top_k; ++n) {
        float best = -INFINITY;
        int at = -1;
        for (int e = 0; e < L.n_experts; ++e) {
            bool taken = false;
            for (int j = 0; j < n; ++j) taken |= sel[j] == e;
            if (!taken && x[e] > best) {
                best = x[e];
                at = e;
            }
        }
        if (at < 0) break;
        sel[n] = at;
        v[n] = best;
    }
    const float top = v[0];
    float sum = 0.0f;
    for (int j = 0; j < n; ++j) {
        v[j] = v[j] == top ? 1.0f : expf(v[j] - top);  // infinity - infinity among them
        sum += v[j];
    }
    for (int j = 0; j < L.top_k; ++j) {
        L.sel[(size_t)t * L.top_k + j] = j < n ? sel[j] : -1;
        L.w[(size_t)t * L.top_k + j] = j < n ? __fdiv_rn(v[j], sum) : 0.0f;
    }
}

// One block: 32 warps, each with a contiguous part of the picks.
__global__ void __launch_bounds__(kPlaceThreads) k_route_place(const RouteLaunch L) {
    __shared__ int count[kPlaceWarps][kMaxRouteExperts];
    __shared__ int first[kMaxRouteExperts + 1];
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, E = L.n_experts;
    const long long total = (long long)L.tokens * L.top_k;
    const long long part = (total + kPlaceThreads - 1) / kPlaceThreads * kWarp;  // per warp, whole warps of picks
    const long long begin = warp * part, end = min(total, begin + part);
    for (int i = lane; i < E; i += kWarp) count[warp][i] = 0;
    __syncwarp();
    for (long long i = begin + lane; i - lane < end; i += kWarp) {
        const int e = i < end ? L.sel[i] : -1;
        const unsigned same = __match_any_sync(0xffffffffu, e);
        if (e >= 0 && (same & ((1u << lane) - 1u)) == 0u) count[warp][e] += __popc(same);
        __syncwarp();
    }
    __syncthreads();
    if (tid < E) {  // the counts of the warps before, and the expert's total
        int sum = 0;
        for (int w = 0; w < kPlaceWarps; ++w) {
            const int c = count[w][tid];
            count[w][tid] = sum;
            sum += c;
        }
        first[tid + 1] = sum;
    }
    __syncthreads();
    if (tid == 0) {
        first[0] = 0;
        for (int e = 0; e < E; ++e) first[e + 1] += first[e];
    }
    __syncthreads();
    if (tid <= E) L.offsets[tid] = first[tid];
    for (long long i = begin + lane; i - lane < end; i += kWarp) {
        const int e = i < end ? L.sel[i] : -1;
        const unsigned same = __match_any_sync(0xffffffffu, e);
        const unsigned before = same & ((1u << lane) - 1u);
        const int at = e >= 0 ? first[e] + count[warp][e] + __popc(before) : -1;
        __syncwarp();
        if (e >= 0) {
            if (before == 0u) count[warp][e] += __popc(same);
            L.rows[at] = (int32_t)(i / L.top_k);
        }
        if (i < end) L.slots[i] = at;
        __syncwarp();
    }
}

}  // namespace

cudaError_t launch_route(const RouteLaunch& a, cudaStream_t stream) {
    if (a.tokens > 0) k_route_pick<<<(a.tokens + 127) / 128, 128, 0, stream>>>(a);
    k_route_place<<<1, kPlaceThreads, 0, stream>>>(a);
    return cudaGetLastError();
}

}  // namespace tsffn
