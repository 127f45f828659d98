// ts_grouped.cu -- products of ragged groups of rows with each group's own weights: y = x W_e, or
// max(0, x W_e) max(0, x U_e) (Eq. 1 with the dReLU of Eq. 2), over bf16 weights or e4m3 ones with a scale for
// each 128 x 128 block (and one for each 128 elements of a row of x).
#include <cuda_fp8.h>

#include "ts_grouped.h"
#include "ts_kernels.cuh"

namespace tsffn {
namespace {

constexpr int kT = 64;   // rows and columns of a block's tile
constexpr int kKT = 16;  // of k per step

__device__ __forceinline__ float elem(const void* p, size_t i, bool e4m3) {
    if (e4m3) return float(static_cast<const __nv_fp8_e4m3*>(p)[i]);
    return __bfloat162float(static_cast<const __nv_bfloat16*>(p)[i]);
}

// One 64 x 64 tile of y per block, 4 x 4 outputs a thread; tiles of rows are numbered group by group.
template <bool E4M3, bool GATED, bool KN>
__global__ void __launch_bounds__(256) k_grouped(const GroupedLaunch L) {
    __shared__ float xs[kKT][kT + 4], wt[GATED ? 2 : 1][kKT][kT + 4];
    int tile = blockIdx.y, g = -1, r0 = 0, r1 = 0;
    for (int e = 0; e < L.n_groups; ++e) {
        const int a = L.offsets ? L.offsets[e] : 0, b = L.offsets ? L.offsets[e + 1] : L.rows;
        if (a < 0 || b < a || b > L.rows) {
            if (threadIdx.x == 0) atomicOr(L.status, kStatusBadIndex);
            continue;
        }
        const int t = (b - a + kT - 1) / kT;
        if (tile < t) {
            g = e;
            r0 = a + tile * kT;
            r1 = min(b, r0 + kT);
            break;
        }
        tile -= t;
    }
    if (g < 0) return;
    const GroupWeights gw = L.weights[g];
    const int c0 = blockIdx.x * kT, tid = threadIdx.x, tx = tid & 15, ty = tid >> 4;
    const int kb_n = (L.k + kScaleBlock - 1) / kScaleBlock;
    float acc[GATED ? 2 : 1][4][4] = {};
    for (int k0 = 0; k0 < L.k; k0 += kKT) {
        for (int i = tid; i < kT * kKT; i += 256) {
            const int r = i / kKT, kk = k0 + i % kKT;
            float v = 0.0f;
            if (r0 + r < r1 && kk < L.k) {
                v = elem(L.x, (size_t)(r0 + r) * L.ldx + kk, E4M3);
                if (E4M3) v *= L.x_scale[(size_t)(kk / kScaleBlock) * L.ld_scale + r0 + r];
            }
            xs[i % kKT][r] = v;
            const int c = KN ? i % kT : i / kKT, kw = KN ? i / kT : i % kKT;
#pragma unroll
            for (int p = 0; p < (GATED ? 2 : 1); ++p) {
                float u = 0.0f;
                if (c0 + c < L.n && k0 + kw < L.k) {
                    const size_t at = KN ? (size_t)(k0 + kw) * L.n + c0 + c : (size_t)(c0 + c) * L.k + k0 + kw;
                    u = elem(p ? gw.u : gw.w, at, E4M3);
                    if (E4M3) u *= (p ? gw.us : gw.ws)[(size_t)((c0 + c) / kScaleBlock) * kb_n + (k0 + kw) / kScaleBlock];
                }
                wt[p][kw][c] = u;
            }
        }
        __syncthreads();
#pragma unroll
        for (int kk = 0; kk < kKT; ++kk)
#pragma unroll
            for (int p = 0; p < (GATED ? 2 : 1); ++p)
#pragma unroll
                for (int i = 0; i < 4; ++i)
#pragma unroll
                    for (int j = 0; j < 4; ++j)
                        acc[p][i][j] = fmaf(xs[kk][ty * 4 + i], wt[p][kk][tx + 16 * j], acc[p][i][j]);
        __syncthreads();
    }
    for (int i = 0; i < 4; ++i)
        for (int j = 0; j < 4; ++j) {
            const int r = r0 + ty * 4 + i, c = c0 + tx + 16 * j;
            if (r >= r1 || c >= L.n) continue;
            float v = acc[0][i][j];
            if (GATED) v = v > 0.0f && acc[GATED ? 1 : 0][i][j] > 0.0f ? v * acc[GATED ? 1 : 0][i][j] : 0.0f;
            const size_t at = (size_t)r * L.ldy + c;
            if (L.y_f32) static_cast<float*>(L.y)[at] = v;
            else static_cast<__nv_bfloat16*>(L.y)[at] = __float2bfloat16_rn(v);
        }
}

}  // namespace

cudaError_t launch_grouped(const GroupedLaunch& a, bool e4m3, bool gated, bool kn, cudaStream_t stream) {
    const int groups = a.offsets ? a.n_groups : 1;
    const dim3 grid((unsigned)((a.n + kT - 1) / kT), (unsigned)((a.rows + kT - 1) / kT + groups));
    if (e4m3)
        gated ? k_grouped<true, true, false><<<grid, 256, 0, stream>>>(a)
              : k_grouped<true, false, false><<<grid, 256, 0, stream>>>(a);
    else if (gated)
        k_grouped<false, true, false><<<grid, 256, 0, stream>>>(a);
    else
        kn ? k_grouped<false, false, true><<<grid, 256, 0, stream>>>(a)
           : k_grouped<false, false, false><<<grid, 256, 0, stream>>>(a);
    return cudaGetLastError();
}

}  // namespace tsffn
