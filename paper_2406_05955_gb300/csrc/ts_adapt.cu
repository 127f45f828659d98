// ts_adapt.cu -- low-rank adapters of many requests beside a shared projection: h[t] = s_i x[t] A_i^T and
// out[t] = y[t] + h[t] B_i for the adapter i of row t (ts_adapt_rows), and the sums over rows of h^T x that are the
// gradients of A and B (ts_adapter_grads). With A and B exchanged the first is also the backward pass by rows.
#include <cuda_fp8.h>

#include "ts_adapt.h"
#include "ts_grouped.h"
#include "ts_kernels.cuh"

namespace tsffn {
namespace {

constexpr int kThreads = 256;

template <typename TY>
__global__ void __launch_bounds__(kThreads) k_adapt(const AdaptLaunch L) {
    __shared__ float h[kMaxRank];
    pdl_wait();
    const int at = blockIdx.x, warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    int row = at, id;
    if (L.list != nullptr) {
        row = L.list[at];
        for (id = 0; id < L.n_adapters && L.offsets[id + 1] <= at;) ++id;
    } else {
        id = L.ids[row];
    }
    if ((unsigned)row >= (unsigned)L.rows) return;
    const bool some = (unsigned)id < (unsigned)L.n_adapters;
    const int rank = !some ? 0 : L.ranks != nullptr ? min(max(L.ranks[id], 0), L.r) : L.r;
    const __nv_bfloat16* x = static_cast<const __nv_bfloat16*>(L.x) + row * L.ldx;
    for (int j = warp; j < L.r; j += kThreads / kWarp) {
        float sum = 0.0f;
        if (j < rank) {
            const __nv_bfloat16* a = static_cast<const __nv_bfloat16*>(L.a) + ((size_t)id * L.r + j) * L.k;
            for (int i = lane; i < L.k; i += kWarp) sum = fmaf(__bfloat162float(x[i]), __bfloat162float(a[i]), sum);
            sum = warp_sum(sum) * (L.scale != nullptr ? L.scale[id] : 1.0f);
        }
        if (lane == 0) {
            h[j] = sum;
            if (L.h != nullptr) L.h[(size_t)row * L.r + j] = sum;
        }
    }
    __syncthreads();
    if (L.out == nullptr || (rank == 0 && L.out == L.y)) return;
    const TY* y = static_cast<const TY*>(L.y) + row * L.ldy;
    TY* out = static_cast<TY*>(L.out) + row * L.ldo;
    const __nv_bfloat16* b = static_cast<const __nv_bfloat16*>(L.b) + (size_t)(some ? id : 0) * L.r * L.n;
    for (int i = threadIdx.x; i < L.n; i += kThreads) {
        float sum = 0.0f;
        for (int j = 0; j < rank; ++j) sum = fmaf(h[j], __bfloat162float(b[(size_t)j * L.n + i]), sum);
        Vec<TY>::store1(out, i, Vec<TY>::load1(y, i) + sum);
    }
}

template <bool E8>
__global__ void __launch_bounds__(kThreads) k_adapter_grads(const AdapterGradsLaunch L) {
    constexpr int kAtOnce = 16;
    pdl_wait();
    const int id = blockIdx.y, i = blockIdx.x * kThreads + threadIdx.x;
    if (i >= L.k) return;
    const int begin = L.offsets[id], end = min(L.offsets[id + 1], L.rows);
    for (int j0 = 0; j0 < L.r; j0 += kAtOnce) {
        float sum[kAtOnce] = {};
        for (int at = begin; at < end; ++at) {
            const int row = L.list[at];
            if ((unsigned)row >= (unsigned)L.rows) continue;
            float v;
            if constexpr (E8) {
                const __nv_fp8_e4m3 q = static_cast<const __nv_fp8_e4m3*>(L.x)[row * L.ldx + i];
                v = (float)q * L.x_scale[(int64_t)(i / kScaleBlock) * L.ld_scale + row];
            } else {
                v = __bfloat162float(static_cast<const __nv_bfloat16*>(L.x)[row * L.ldx + i]);
            }
#pragma unroll
            for (int j = 0; j < kAtOnce; ++j)
                if (j0 + j < L.r) sum[j] = fmaf(L.h[(size_t)row * L.r + j0 + j], v, sum[j]);
        }
#pragma unroll
        for (int j = 0; j < kAtOnce; ++j)
            if (j0 + j < L.r) {
                float* g = L.grad + ((size_t)id * L.r + j0 + j) * L.k + i;
                *g = L.accumulate ? *g + sum[j] : sum[j];
            }
    }
}

}  // namespace

cudaError_t prepare_adapt() { return cudaSuccess; }

cudaError_t launch_adapt(const AdaptLaunch& a, bool y_f32, cudaStream_t stream) {
    return launch_after(y_f32 ? k_adapt<float> : k_adapt<__nv_bfloat16>, launch_shape(dim3((unsigned)a.rows), kThreads, stream), a);
}

cudaError_t launch_adapter_grads(const AdapterGradsLaunch& a, bool e4m3, cudaStream_t stream) {
    return launch_after(e4m3 ? k_adapter_grads<true> : k_adapter_grads<false>,
                        launch_shape(dim3((unsigned)((a.k + kThreads - 1) / kThreads), (unsigned)a.n_adapters), kThreads, stream), a);
}

}  // namespace tsffn
