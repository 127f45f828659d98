// ts_combine_bwd.cu -- the backward pass of ts_combine_rows: y[t] = sum_j w[t][j] src[slots[t][j]] gives
//     dsrc[r] = (sum over the j with slots[t][j] = r of w[t][j]) dy[t]  for the token t = rows[r],
//     dw[t][j] = <dy[t], src[slots[t][j]]>.
// A CTA has a token: dy[t] is read once for all of its rows. A row is written by the token that `rows` names, so one that
// slots names twice is still written once, and the same bits come out each time.
//
// Memory bounds it: dy and the rows read, the rows written. 4096 tokens of 2 rows of 4096, dy fp32, rows bf16, one in 20 without
// a row: 29.3 us (6.5 TB/s); 32 tokens 3.0.
#include "ts_adapt.h"
#include "ts_grouped.h"
#include "ts_kernels.cuh"

namespace tsffn {
namespace {

constexpr int kThreads = 256;
constexpr int kWarps = kThreads / kWarp;
constexpr int kVec = 8;  // elements of a thread's step

// `V` elements at p in fp32: 16-byte loads where V is 8.
template <typename T, int V>
__device__ __forceinline__ void load(const T* p, float (&v)[V]) {
    if constexpr (V == 1) {
        v[0] = Vec<T>::load1(p, 0);
    } else {
#pragma unroll
        for (int i = 0; i < V; i += Vec<T>::N) Vec<T>::unpack(ld_stream(p + i), v + i);
    }
}
template <typename T, int V>
__device__ __forceinline__ void store(T* p, const float (&v)[V]) {
    if constexpr (V == 1) {
        Vec<T>::store1(p, 0, v[0]);
    } else if constexpr (sizeof(T) == 4) {
#pragma unroll
        for (int i = 0; i < V; i += 4) __stcs(reinterpret_cast<float4*>(p + i), make_float4(v[i], v[i + 1], v[i + 2], v[i + 3]));
    } else {
        uint32_t w[V / 2];
#pragma unroll
        for (int i = 0; i < V; i += 2) {
            const __nv_bfloat162 b = __floats2bfloat162_rn(v[i], v[i + 1]);
            w[i / 2] = *reinterpret_cast<const uint32_t*>(&b);
        }
        __stcs(reinterpret_cast<uint4*>(p), make_uint4(w[0], w[1], w[2], w[3]));
    }
}

template <typename TD, typename TS, int V, int K>  // K: top_k rounded up to 2, 4 or 8
__global__ void __launch_bounds__(kThreads) k_combine_backward(const CombineBackwardLaunch L) {
    __shared__ float part[kWarps][K];
    const int t = blockIdx.x, lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    pdl_wait();
    pdl_launch_dependents();
    int slot[K];
    float w[K], dot[K] = {};
    bool mine[K];  // this token writes the row here
#pragma unroll
    for (int j = 0; j < K; ++j) {
        slot[j] = j < L.top_k ? L.slots[(size_t)t * L.top_k + j] : -1;
        if ((unsigned)slot[j] >= (unsigned)L.n_rows) slot[j] = -1;
        w[j] = j < L.top_k ? L.w[(size_t)t * L.top_k + j] : 0.0f;
        mine[j] = slot[j] >= 0 && L.rows[slot[j]] == t;
    }
#pragma unroll
    for (int j = 1; j < K; ++j)  // a row that the token has twice: at its first place, with both weights
#pragma unroll
        for (int i = 0; i < j; ++i)
            if (mine[j] && mine[i] && slot[i] == slot[j]) {
                w[i] += w[j];
                mine[j] = false;
            }
    for (int64_t i = (int64_t)threadIdx.x * V; i < L.n; i += kThreads * V) {
        float dy[V], v[V];
        load<TD, V>(static_cast<const TD*>(L.dy) + (size_t)t * L.n + i, dy);
#pragma unroll
        for (int j = 0; j < K; ++j) {
            if (slot[j] < 0) continue;
            const size_t at = (size_t)slot[j] * L.n + i;
            load<TS, V>(static_cast<const TS*>(L.src) + at, v);
#pragma unroll
            for (int e = 0; e < V; ++e) {
                dot[j] = fmaf(dy[e], v[e], dot[j]);
                v[e] = w[j] * dy[e];
            }
            if (mine[j]) store<TS, V>(static_cast<TS*>(L.dsrc) + at, v);
        }
    }
#pragma unroll
    for (int j = 0; j < K; ++j) {
        const float s = warp_sum(dot[j]);
        if (lane == 0) part[warp][j] = s;
    }
    __syncthreads();
    if (threadIdx.x < L.top_k) {
        float s = 0.0f;
#pragma unroll
        for (int i = 0; i < kWarps; ++i) s += part[i][threadIdx.x];
        L.dw[(size_t)t * L.top_k + threadIdx.x] = s;
    }
}

template <typename TD, typename TS, int V>
auto by_top_k(int top_k) {
    return top_k <= 2 ? k_combine_backward<TD, TS, V, 2> : top_k <= 4 ? k_combine_backward<TD, TS, V, 4>
                                                                      : k_combine_backward<TD, TS, V, kMaxRouteK>;
}
template <typename TD, typename TS>
auto by_step(bool vec, int top_k) {
    return vec ? by_top_k<TD, TS, kVec>(top_k) : by_top_k<TD, TS, 1>(top_k);
}

}  // namespace

cudaError_t launch_combine_backward(const CombineBackwardLaunch& a, bool dy_f32, bool src_f32, cudaStream_t stream) {
    const bool vec = a.n % kVec == 0 && (((uintptr_t)a.dy | (uintptr_t)a.src | (uintptr_t)a.dsrc) & 15u) == 0;
    const auto kernel = dy_f32 ? (src_f32 ? by_step<float, float>(vec, a.top_k) : by_step<float, __nv_bfloat16>(vec, a.top_k))
                               : (src_f32 ? by_step<__nv_bfloat16, float>(vec, a.top_k)
                                          : by_step<__nv_bfloat16, __nv_bfloat16>(vec, a.top_k));
    return launch_after(kernel, launch_shape(dim3((unsigned)a.tokens), kThreads, stream), a);
}

}  // namespace tsffn
