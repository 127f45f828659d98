// ts_drelu.cu -- the gated activation c = max(0, g) max(0, u) of products that were computed apart (ts_drelu_rows), what
// its backward pass needs kept in 8 bits, and that pass (ts_drelu_rows_backward).
//
// Only neurons of which both factors are positive have a gradient: dg = dc u, du = dc g there, 0 elsewhere. So the factors
// are kept as zero wherever the other one is not positive, and one e4m3 number says both the value and the mask: a
// positive factor is never rounded to zero. The scale of 128 elements is a power of two: values lose nothing but their
// last bits (2^-4 relative), c = g u of kept factors (4 and 4 significant bits) is exact in bf16, and nothing depends on
// how a quotient is rounded.
//
// One pass over memory bounds both: 8 and 10 bytes an element of bf16. 8092 rows of 14336, bf16: 145 us and 171 (6.4 and 6.8
// TB/s of those bytes, in a launch each; calls in a row 318 together).
#include <cuda_fp8.h>

#include "ts_adapt.h"
#include "ts_grouped.h"
#include "ts_kernels.cuh"

namespace tsffn {
namespace {

constexpr int kThreads = 256;
constexpr int kRows = kThreads / kWarp;  // a warp per row
constexpr int kLoads = 4;                // 16-byte loads of a lane from each input

// 2^e of the smallest power of two with top / 2^e <= 448 = 1.75 2^8, at least 2^-100 (top is positive and finite).
__device__ __forceinline__ int scale_exponent(float top) {
    const unsigned u = __float_as_uint(top);
    return max((int)(u >> 23) - 127 - 8 + ((u & 0x7fffffu) > 0x600000u), -100);
}
__device__ __forceinline__ float power_of_two(int e) { return __uint_as_float((unsigned)(e + 127) << 23); }

// N elements rounded to bf16, stored together.
template <int N>
__device__ __forceinline__ void store_bf16(void* to, const float (&v)[N]) {
    uint32_t w[N / 2];
#pragma unroll
    for (int i = 0; i < N; i += 2) {
        const __nv_bfloat162 p = __floats2bfloat162_rn(v[i], v[i + 1]);
        w[i / 2] = *reinterpret_cast<const uint32_t*>(&p);
    }
    if constexpr (N == 8) __stcs(static_cast<uint4*>(to), make_uint4(w[0], w[1], w[2], w[3]));
    else __stcs(static_cast<uint2*>(to), make_uint2(w[0], w[1]));
}

// N factors of one lane (of the LANES lanes that have a block) in e4m3 of a common scale, which is returned.
template <int N, int LANES>
__device__ __forceinline__ float keep(const float (&p)[N], uint32_t (&q)[N / 4]) {
    constexpr float kLargest = 3.19014718988379809e38f;  // 1.875 2^127: what is beyond (infinity) is kept as this
    float top = 0.0f;
#pragma unroll
    for (int i = 0; i < N; ++i) top = fmaxf(top, p[i]);
#pragma unroll
    for (int o = LANES / 2; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
    const int e = top > 0.0f ? scale_exponent(fminf(top, kLargest)) : 0;
    const float inverse = power_of_two(-e);
#pragma unroll
    for (int i = 0; i < N; i += 4) {
        float v[4];
#pragma unroll
        for (int j = 0; j < 4; ++j)  // what is below the smallest e4m3 number, 2^-9, becomes that
            v[j] = p[i + j] > 0.0f ? fmaxf(fminf(p[i + j], kLargest) * inverse, 0.001953125f) : 0.0f;
        q[i / 4] = (uint32_t)__nv_cvt_float2_to_fp8x2(make_float2(v[0], v[1]), __NV_SATFINITE, __NV_E4M3) |
                   (uint32_t)__nv_cvt_float2_to_fp8x2(make_float2(v[2], v[3]), __NV_SATFINITE, __NV_E4M3) << 16;
    }
    return power_of_two(e);
}

template <int N>
__device__ __forceinline__ void store_e4m3(uint8_t* to, const uint32_t (&q)[N / 4]) {
    if constexpr (N == 8) __stcs(reinterpret_cast<uint2*>(to), make_uint2(q[0], q[1]));
    else __stcs(reinterpret_cast<uint32_t*>(to), q[0]);
}

// The rows that a call is about: none where the device's count is negative.
__device__ __forceinline__ int live_rows(const int32_t* n, int rows) { return n != nullptr ? max(0, min(rows, *n)) : rows; }

// A warp takes 8 (bf16) or 4 (fp32) blocks of 128 elements of a row, a CTA the same blocks of 8 rows, so that their scales,
// which lie together by block, are written 32 bytes at a time.
template <typename T, bool KEEP>
__global__ void __launch_bounds__(kThreads) k_drelu(const DreluLaunch L) {
    constexpr int N = Vec<T>::N, kLanes = kScaleBlock / N, kPer = kWarp / kLanes, kBlocks = kLoads * kPer;
    __shared__ float scales[2][kBlocks][kRows];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    pdl_wait();
    pdl_launch_dependents();
    const int rows = live_rows(L.n, L.rows), r = blockIdx.x * kRows + warp;
    if (r < rows) {
        const int at = blockIdx.y * (kBlocks * kScaleBlock) + N * lane;
        const T* g = static_cast<const T*>(L.g) + r * L.ldg + at;
        const T* u = static_cast<const T*>(L.u) + r * L.ldu + at;
        uint4 rg[kLoads], ru[kLoads];
#pragma unroll
        for (int i = 0; i < kLoads; ++i) {
            const bool in = at + N * kWarp * i < L.m;
            rg[i] = in ? ld_stream(g + N * kWarp * i) : make_uint4(0u, 0u, 0u, 0u);
            ru[i] = in ? ld_stream(u + N * kWarp * i) : make_uint4(0u, 0u, 0u, 0u);
        }
#pragma unroll
        for (int i = 0; i < kLoads; ++i) {
            float pg[N], pu[N], c[N];
            Vec<T>::unpack(rg[i], pg);
            Vec<T>::unpack(ru[i], pu);
#pragma unroll
            for (int j = 0; j < N; ++j) {
                const bool both = pg[j] > 0.0f && pu[j] > 0.0f;
                pg[j] = both ? pg[j] : 0.0f;
                pu[j] = both ? pu[j] : 0.0f;
                c[j] = both ? pg[j] * pu[j] : 0.0f;
            }
            const int step = N * kWarp * i;
            const bool in = at + step < L.m;
            if (in) store_bf16<N>(static_cast<__nv_bfloat16*>(L.c) + r * L.ldc + at + step, c);
            if constexpr (KEEP) {
                uint32_t qg[N / 4], qu[N / 4];
                const float sg = keep<N, kLanes>(pg, qg), su = keep<N, kLanes>(pu, qu);
                if (lane % kLanes == 0) {
                    scales[0][i * kPer + lane / kLanes][warp] = sg;
                    scales[1][i * kPer + lane / kLanes][warp] = su;
                }
                if (in) {
                    const size_t to = (size_t)r * L.m + at + step;
                    store_e4m3<N>(L.q_gate + to, qg);
                    store_e4m3<N>(L.q_up + to, qu);
                }
            }
        }
    }
    if constexpr (KEEP) {
        __syncthreads();
        for (int i = threadIdx.x; i < 2 * kBlocks * kRows; i += kThreads) {
            const int which = i / (kBlocks * kRows), b = i / kRows % kBlocks, row = i % kRows;
            const int block = blockIdx.y * kBlocks + b, to = blockIdx.x * kRows + row;
            if (block * kScaleBlock < L.m && to < rows)
                (which ? L.s_up : L.s_gate)[(size_t)block * L.rows + to] = scales[which][b][row];
        }
    }
}

// Four e4m3 numbers times `scale`.
__device__ __forceinline__ void wide(uint32_t q, float scale, float* v) {
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const __half2_raw h = __nv_cvt_fp8x2_to_halfraw2((__nv_fp8x2_storage_t)(q >> 16 * i), __NV_E4M3);
        const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&h));
        v[2 * i] = f.x * scale;
        v[2 * i + 1] = f.y * scale;
    }
}

template <typename T>
__global__ void __launch_bounds__(kThreads) k_drelu_backward(const DreluBackwardLaunch L) {
    constexpr int N = Vec<T>::N;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    pdl_wait();
    pdl_launch_dependents();
    const int rows = live_rows(L.n, L.rows), r = blockIdx.x * kRows + warp;
    if (r >= rows) return;
    const int at = blockIdx.y * (N * kWarp * kLoads) + N * lane;
    uint4 rd[kLoads];
    uint2 rg[kLoads], ru[kLoads];
    float sg[kLoads], su[kLoads];
#pragma unroll
    for (int i = 0; i < kLoads; ++i) {
        const int col = at + N * kWarp * i;
        if (col >= L.m) break;
        const size_t q = (size_t)r * L.m + col, s = (size_t)(col / kScaleBlock) * L.rows + r;
        rd[i] = ld_stream(static_cast<const T*>(L.dc) + r * L.ldd + col);
        if constexpr (N == 8) {
            rg[i] = __ldcs(reinterpret_cast<const uint2*>(L.q_gate + q));
            ru[i] = __ldcs(reinterpret_cast<const uint2*>(L.q_up + q));
        } else {
            rg[i].x = __ldcs(reinterpret_cast<const unsigned*>(L.q_gate + q));
            ru[i].x = __ldcs(reinterpret_cast<const unsigned*>(L.q_up + q));
        }
        sg[i] = L.s_gate[s];
        su[i] = L.s_up[s];
    }
#pragma unroll
    for (int i = 0; i < kLoads; ++i) {
        const int col = at + N * kWarp * i;
        if (col >= L.m) break;
        float dc[N], pg[N], pu[N], dg[N], du[N], c[N];
        Vec<T>::unpack(rd[i], dc);
        wide(rg[i].x, sg[i], pg);
        wide(ru[i].x, su[i], pu);
        if constexpr (N == 8) {
            wide(rg[i].y, sg[i], pg + 4);
            wide(ru[i].y, su[i], pu + 4);
        }
#pragma unroll
        for (int j = 0; j < N; ++j) {
            const bool both = pg[j] > 0.0f && pu[j] > 0.0f;
            dg[j] = both ? dc[j] * pu[j] : 0.0f;
            du[j] = both ? dc[j] * pg[j] : 0.0f;
            c[j] = both ? pg[j] * pu[j] : 0.0f;
        }
        store_bf16<N>(static_cast<__nv_bfloat16*>(L.dg) + r * L.ldg + col, dg);
        store_bf16<N>(static_cast<__nv_bfloat16*>(L.du) + r * L.ldu + col, du);
        if (L.c != nullptr) store_bf16<N>(static_cast<__nv_bfloat16*>(L.c) + r * L.ldc + col, c);
    }
}

cudaLaunchConfig_t shape(int rows, int m, bool f32, cudaStream_t stream) {
    const int per = (f32 ? 4 : 8) * kWarp * kLoads;
    return launch_shape(dim3((unsigned)((rows + kRows - 1) / kRows), (unsigned)((m + per - 1) / per)), kThreads, stream);
}

}  // namespace

cudaError_t launch_drelu(const DreluLaunch& a, bool f32, cudaStream_t stream) {
    const bool kept = a.q_gate != nullptr;
    const auto kernel = f32 ? (kept ? k_drelu<float, true> : k_drelu<float, false>)
                            : (kept ? k_drelu<__nv_bfloat16, true> : k_drelu<__nv_bfloat16, false>);
    return launch_after(kernel, shape(a.rows, a.m, f32, stream), a);
}

cudaError_t launch_drelu_backward(const DreluBackwardLaunch& a, bool f32, cudaStream_t stream) {
    return launch_after(f32 ? k_drelu_backward<float> : k_drelu_backward<__nv_bfloat16>, shape(a.rows, a.m, f32, stream), a);
}

}  // namespace tsffn
