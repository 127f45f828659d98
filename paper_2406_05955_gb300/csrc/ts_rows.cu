// ts_rows.cu -- rows in the experts' order: copied (ts_gather_rows), rounded to e4m3 with a scale for each 128
// elements (ts_quant_rows), and summed back by token (ts_combine_rows). All are one pass over the data and bound by
// memory; what matters is that each thread has several 16-byte loads on their way and that whole sectors are written.
// 8192 rows of 4096 bf16: copied in 21.8 us (6.2 TB/s), rounded in 18.6 (5.4); of 14336: 72.7 (6.5) and 57.8 (6.1).
#include <cuda_fp8.h>

#include "ts_grouped.h"
#include "ts_kernels.cuh"

namespace tsffn {
namespace {

constexpr int kRowThreads = 256;
constexpr int kRowsPerCta = kRowThreads / kWarp;  // a warp per row
constexpr int kLoads = 4;                         // 16-byte loads of a lane
constexpr float kE4m3Max = 448.0f;
constexpr float kMinScale = 7.8886090522101181e-31f;  // 2^-100

// Source row of output row r; -1: none (behind the count, or a list entry out of range).
__device__ __forceinline__ int source_row(const RowsLaunch& L, int r) {
    if (r >= L.max_rows || (L.n != nullptr && r >= *L.n)) return -1;
    const int s = L.rows != nullptr ? L.rows[r] : r;
    return (unsigned)s < (unsigned)L.n_src ? s : -1;
}

// A warp copies 2 KB of a row.
__global__ void __launch_bounds__(kRowThreads) k_gather_rows(const RowsLaunch L, int64_t src_bytes, int row_bytes) {
    pdl_wait();
    const int r = blockIdx.x * kRowsPerCta + (threadIdx.x >> 5), lane = threadIdx.x & 31, s = source_row(L, r);
    if (s < 0) return;
    const int at = blockIdx.y * (16 * kLoads * kWarp) + 16 * lane;
    const char* from = static_cast<const char*>(L.x) + s * src_bytes + at;
    char* to = static_cast<char*>(L.out) + (int64_t)r * row_bytes + at;
    uint4 v[kLoads];
#pragma unroll
    for (int i = 0; i < kLoads; ++i)
        if (at + 16 * kWarp * i < row_bytes) v[i] = ld_stream(from + 16 * kWarp * i);
#pragma unroll
    for (int i = 0; i < kLoads; ++i)
        if (at + 16 * kWarp * i < row_bytes) *reinterpret_cast<uint4*>(to + 16 * kWarp * i) = v[i];
}

// Two quotients x / scale, for inv = 1 / scale: the products with inv, corrected once by their remainders (Markstein's
// division, correctly rounded but for rare last bits: none of 2 10^7 pairs), 3 instructions for both where a division takes
// about 10. The rounding to e4m3 that follows is of this fp32 quotient.
__device__ __forceinline__ float2 quotients(float a, float b, float scale, float inv) {
    const float2 x = make_float2(a, b), i = make_float2(inv, inv), q = __fmul2_rn(x, i);
    return __ffma2_rn(__ffma2_rn(q, make_float2(-scale, -scale), x), i, q);
}

// Largest magnitude of a 16-byte load's elements (NaN left out; a maximum in bf16 is exact).
template <typename T>
__device__ __forceinline__ float largest(const uint4& v) {
    if constexpr (sizeof(T) == 2) {
        const __nv_bfloat162* h = reinterpret_cast<const __nv_bfloat162*>(&v);
        const __nv_bfloat162 m = __hmax2(__hmax2(__habs2(h[0]), __habs2(h[1])), __hmax2(__habs2(h[2]), __habs2(h[3])));
        return fmaxf(__low2float(m), __high2float(m));
    } else {
        float f[4];
        Vec<T>::unpack(v, f);
        return fmaxf(fmaxf(fabsf(f[0]), fabsf(f[1])), fmaxf(fabsf(f[2]), fabsf(f[3])));
    }
}

// A warp takes 8 (bf16) or 4 (fp32) blocks of 128 elements of a row, 16 or 32 lanes a block; a CTA the same blocks of 8
// rows, so that their scales, which lie together by block, are written 32 bytes at a time.
template <typename T>
__global__ void __launch_bounds__(kRowThreads) k_quant_rows(const RowsLaunch L) {
    constexpr int N = Vec<T>::N, kLanes = kScaleBlock / N;       // elements of a load, lanes of a block
    constexpr int kPer = kWarp / kLanes, kBlocks = kLoads * kPer;  // blocks of a load, of a warp
    __shared__ float scales[kBlocks][kRowsPerCta];
    __shared__ bool live[kRowsPerCta];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    pdl_wait();
    const int r = blockIdx.x * kRowsPerCta + warp, s = source_row(L, r);
    if (lane == 0) live[warp] = s >= 0;
    if (s >= 0) {
        const int at = blockIdx.y * (kBlocks * kScaleBlock) + N * lane;
        const T* from = static_cast<const T*>(L.x) + s * L.ldx + at;
        char* to = static_cast<char*>(L.out) + (int64_t)r * L.k + at;
        uint4 raw[kLoads];
#pragma unroll
        for (int i = 0; i < kLoads; ++i)
            raw[i] = at + N * kWarp * i < L.k ? ld_stream(from + N * kWarp * i) : make_uint4(0u, 0u, 0u, 0u);
#pragma unroll
        for (int i = 0; i < kLoads; ++i) {
            float v[N], top = largest<T>(raw[i]);
            Vec<T>::unpack(raw[i], v);
#pragma unroll
            for (int o = kLanes / 2; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
            const float scale = top > 0.0f ? fmaxf(__fdiv_rn(top, kE4m3Max), kMinScale) : 1.0f, inv = __frcp_rn(scale);
            if (lane % kLanes == 0) scales[i * kPer + lane / kLanes][warp] = scale;
            uint32_t q[N / 4];
#pragma unroll
            for (int j = 0; j < N; j += 4) {
                const float2 a = quotients(v[j], v[j + 1], scale, inv);
                const float2 b = quotients(v[j + 2], v[j + 3], scale, inv);
                q[j / 4] = (uint32_t)__nv_cvt_float2_to_fp8x2(a, __NV_SATFINITE, __NV_E4M3) |
                           (uint32_t)__nv_cvt_float2_to_fp8x2(b, __NV_SATFINITE, __NV_E4M3) << 16;
            }
            if (at + N * kWarp * i < L.k) {
                if constexpr (N == 8) *reinterpret_cast<uint2*>(to + N * kWarp * i) = make_uint2(q[0], q[1]);
                else *reinterpret_cast<uint32_t*>(to + N * kWarp * i) = q[0];
            }
        }
    }
    __syncthreads();
    const int b = threadIdx.x / kRowsPerCta, row = threadIdx.x % kRowsPerCta;
    const int block = blockIdx.y * kBlocks + b;
    if (b < kBlocks && block * kScaleBlock < L.k && live[row])
        L.scale[(size_t)block * L.max_rows + blockIdx.x * kRowsPerCta + row] = scales[b][row];
}

// A thread sums 16 bytes' elements of a token (VEC), its rows' loads on their way together, or one element. 4096 tokens
// of 2 rows, n = 4096, fp32: 30.5 us (6.6 TB/s), bf16 21.1. Measured at 36 us before it waited for less: without the
// streaming loads and stores 48, with registers for 8 rows (fewer threads on an SM) 41, with two or four times 16 bytes a
// thread 41 and 46.
template <typename T, bool VEC, int K>  // K: top_k rounded up to 2, 4 or 8
__global__ void __launch_bounds__(kRowThreads) k_combine(const CombineLaunch L) {
    constexpr int N = VEC ? Vec<T>::N : 1;
    const int t = blockIdx.y, i = (blockIdx.x * kRowThreads + threadIdx.x) * N;
    pdl_wait();
    if (i >= L.n) return;
    int s[K];
    float w[K], sum[N] = {};
#pragma unroll
    for (int j = 0; j < K; ++j) {
        s[j] = j < L.top_k ? L.slots[(size_t)t * L.top_k + j] : -1;
        w[j] = j < L.top_k ? L.w[(size_t)t * L.top_k + j] : 0.0f;
    }
    uint4 raw[K];
#pragma unroll
    for (int j = 0; j < K; ++j) {
        if ((unsigned)s[j] >= (unsigned)L.n_rows) continue;
        const T* from = static_cast<const T*>(L.src) + (size_t)s[j] * L.n + i;
        if constexpr (VEC) raw[j] = ld_stream(from);
        else raw[j].x = __float_as_uint(Vec<T>::load1(from, 0));
    }
#pragma unroll
    for (int j = 0; j < K; ++j) {
        if ((unsigned)s[j] >= (unsigned)L.n_rows) continue;
        float v[N];
        if constexpr (VEC) Vec<T>::unpack(raw[j], v);
        else v[0] = __uint_as_float(raw[j].x);
#pragma unroll
        for (int e = 0; e < N; ++e) sum[e] = fmaf(w[j], v[e], sum[e]);
    }
    float* y = L.y + (size_t)t * L.n + i;
    if constexpr (VEC) {
#pragma unroll
        for (int e = 0; e < N; e += 4)
            __stcs(reinterpret_cast<float4*>(y + e), make_float4(sum[e], sum[e + 1], sum[e + 2], sum[e + 3]));
    } else {
        y[0] = sum[0];
    }
}

template <typename T, bool VEC>
auto pick_combine(int top_k) {
    return top_k <= 2 ? k_combine<T, VEC, 2> : top_k <= 4 ? k_combine<T, VEC, 4> : k_combine<T, VEC, kMaxRouteK>;
}

dim3 row_grid(const RowsLaunch& a, int row, int per_cta) {
    return dim3((unsigned)((a.max_rows + kRowsPerCta - 1) / kRowsPerCta), (unsigned)((row + per_cta - 1) / per_cta));
}

}  // namespace

cudaError_t launch_gather_rows(const RowsLaunch& a, int elem_bytes, cudaStream_t stream) {
    const int bytes = a.k * elem_bytes;
    return launch_after(k_gather_rows, launch_shape(row_grid(a, bytes, 16 * kLoads * kWarp), kRowThreads, stream), a,
                        a.ldx * elem_bytes, bytes);
}

cudaError_t launch_quant_rows(const RowsLaunch& a, bool f32, cudaStream_t stream) {
    return launch_after(f32 ? k_quant_rows<float> : k_quant_rows<__nv_bfloat16>,
                        launch_shape(row_grid(a, a.k, (f32 ? 4 : 8) * kLoads * kWarp), kRowThreads, stream), a);
}

cudaError_t launch_combine(const CombineLaunch& a, bool f32, cudaStream_t stream) {
    const int size = f32 ? 4 : 8;  // elements of 16 bytes
    const bool vec = a.n % size == 0 && (((uintptr_t)a.src | (uintptr_t)a.y) & 15u) == 0;
    const int per = kRowThreads * (vec ? size : 1);
    const unsigned gx = (unsigned)((a.n + per - 1) / per);
    const auto kernel = f32 ? (vec ? pick_combine<float, true>(a.top_k) : pick_combine<float, false>(a.top_k))
                            : (vec ? pick_combine<__nv_bfloat16, true>(a.top_k) : pick_combine<__nv_bfloat16, false>(a.top_k));
    for (int t = 0; t < a.tokens; t += 65535) {  // the grid's second dimension ends there
        CombineLaunch b = a;
        b.slots += (size_t)t * a.top_k;
        b.w += (size_t)t * a.top_k;
        b.y += (size_t)t * a.n;
        const dim3 grid(gx, (unsigned)(a.tokens - t < 65535 ? a.tokens - t : 65535));
        const cudaError_t e = launch_after(kernel, launch_shape(grid, kRowThreads, stream), b);
        if (e != cudaSuccess) return e;
    }
    return cudaSuccess;
}

}  // namespace tsffn
