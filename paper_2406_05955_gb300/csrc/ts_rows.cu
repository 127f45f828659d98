// ts_rows.cu -- rows in the experts' order: copied (ts_gather_rows), rounded to e4m3 with a scale for each 128
// elements (ts_quant_rows), and summed back by token (ts_combine_rows). All are one pass over the data.
#include <cuda_fp8.h>

#include "ts_grouped.h"
#include "ts_kernels.cuh"

namespace tsffn {
namespace {

constexpr int kRowThreads = 256;
constexpr float kE4m3Max = 448.0f;
constexpr float kMinScale = 7.8886090522101181e-31f;  // 2^-100

// Source row of output row r; -1: none (behind the count, or a list entry out of range).
__device__ __forceinline__ int source_row(const RowsLaunch& L, int r) {
    if (r >= L.max_rows || (L.n != nullptr && r >= *L.n)) return -1;
    const int s = L.rows != nullptr ? L.rows[r] : r;
    return (unsigned)s < (unsigned)L.n_src ? s : -1;
}

__global__ void __launch_bounds__(kRowThreads) k_gather_rows(const RowsLaunch L, int64_t src_bytes, int row_bytes) {
    const int r = blockIdx.x, s = source_row(L, r);
    if (s < 0) return;
    const uint4* from = reinterpret_cast<const uint4*>(static_cast<const char*>(L.x) + s * src_bytes);
    uint4* to = reinterpret_cast<uint4*>(static_cast<char*>(L.out) + (int64_t)r * row_bytes);
    for (int i = threadIdx.x; i < row_bytes / 16; i += kRowThreads) to[i] = from[i];
}

// A block of 128 elements per warp, 4 a lane.
template <typename T>
__global__ void __launch_bounds__(kRowThreads) k_quant_rows(const RowsLaunch L) {
    const int r = blockIdx.x, s = source_row(L, r), lane = threadIdx.x & 31;
    if (s < 0) return;
    const T* from = static_cast<const T*>(L.x) + s * L.ldx;
    uint32_t* to = reinterpret_cast<uint32_t*>(static_cast<char*>(L.out) + (int64_t)r * L.k);
    for (int b = threadIdx.x >> 5; b * kScaleBlock < L.k; b += kRowThreads / kWarp) {
        const int i = b * kScaleBlock + 4 * lane;  // k is a multiple of 4
        float v[4], top = 0.0f;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            v[j] = i < L.k ? Vec<T>::load1(from, i + j) : 0.0f;
            top = fmaxf(top, fabsf(v[j]));
        }
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
        const float scale = top > 0.0f ? fmaxf(__fdiv_rn(top, kE4m3Max), kMinScale) : 1.0f;
        if (lane == 0) L.scale[(size_t)b * L.max_rows + r] = scale;
        uint32_t q = 0u;
#pragma unroll
        for (int j = 0; j < 4; ++j)
            q |= (uint32_t)__nv_cvt_float_to_fp8(__fdiv_rn(v[j], scale), __NV_SATFINITE, __NV_E4M3) << (8 * j);
        if (i < L.k) to[i / 4] = q;
    }
}

template <typename T>
__global__ void __launch_bounds__(kRowThreads) k_combine(const CombineLaunch L) {
    const int t = blockIdx.x;
    for (int i = threadIdx.x; i < L.n; i += kRowThreads) {
        float sum = 0.0f;
        for (int j = 0; j < L.top_k; ++j) {
            const int s = L.slots[(size_t)t * L.top_k + j];
            if ((unsigned)s < (unsigned)L.n_rows)
                sum = fmaf(L.w[(size_t)t * L.top_k + j], Vec<T>::load1(L.src, (size_t)s * L.n + i), sum);
        }
        L.y[(size_t)t * L.n + i] = sum;
    }
}

}  // namespace

cudaError_t launch_gather_rows(const RowsLaunch& a, int elem_bytes, cudaStream_t stream) {
    k_gather_rows<<<a.max_rows, kRowThreads, 0, stream>>>(a, a.ldx * elem_bytes, a.k * elem_bytes);
    return cudaGetLastError();
}

cudaError_t launch_quant_rows(const RowsLaunch& a, bool f32, cudaStream_t stream) {
    if (f32) k_quant_rows<float><<<a.max_rows, kRowThreads, 0, stream>>>(a);
    else k_quant_rows<__nv_bfloat16><<<a.max_rows, kRowThreads, 0, stream>>>(a);
    return cudaGetLastError();
}

cudaError_t launch_combine(const CombineLaunch& a, bool f32, cudaStream_t stream) {
    if (f32) k_combine<float><<<a.tokens, kRowThreads, 0, stream>>>(a);
    else k_combine<__nv_bfloat16><<<a.tokens, kRowThreads, 0, stream>>>(a);
    return cudaGetLastError();
}

}  // namespace tsffn
