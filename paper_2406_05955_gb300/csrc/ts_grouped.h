// ts_grouped.h -- launch parameters and launchers of the operators over many tokens (ts_route.cu, ts_rows.cu, ts_grouped.cu).
#pragma once

#include <cuda_runtime.h>
#include <stdint.h>

namespace tsffn {

constexpr int kMaxRouteExperts = 256;
constexpr int kMaxRouteK = 8;
constexpr int kMaxGroups = 256;
constexpr int kScaleBlock = 128;  // elements of one scale, along k and along n

struct RouteLaunch {
    const float* logits;  // [tokens][n_experts]
    int tokens, n_experts, top_k;
    int32_t* sel;         // [tokens][top_k]
    float* w;             // [tokens][top_k]
    int32_t* offsets;     // [n_experts + 1]
    int32_t* rows;        // [tokens * top_k]
    int32_t* slots;       // [tokens][top_k]
};

struct RowsLaunch {
    const void* x;        // [n_src] rows of k elements, ldx elements apart
    int64_t ldx;
    int n_src, k;
    const int32_t* rows;  // [max_rows] or nullptr
    const int32_t* n;     // device count or nullptr
    int max_rows;
    void* out;            // [max_rows][k]: copied, or e4m3
    float* scale;         // [k / 128][max_rows] (quantised rows)
};

struct CombineLaunch {
    const void* src;      // [n_rows][n]
    int n_rows, n;
    const int32_t* slots;
    const float* w;
    int tokens, top_k;
    float* y;
};

// Weights of one group.
struct GroupWeights {
    const void* w;
    const void* u;   // gated
    const float* ws; // TS_E4M3 scales
    const float* us;
};

struct GroupedLaunch {
    int n_groups, n, k;
    const GroupWeights* weights;  // device [n_groups]
    const void* x;
    int64_t ldx;
    const float* x_scale;         // [k / 128][ld_scale]
    int64_t ld_scale;
    const int32_t* offsets;       // [n_groups + 1] or nullptr (one group)
    int rows;
    void* y;
    int64_t ldy;
    int y_f32;
    unsigned* status;
};

cudaError_t launch_route(const RouteLaunch& a, cudaStream_t stream);
cudaError_t launch_gather_rows(const RowsLaunch& a, int elem_bytes, cudaStream_t stream);
cudaError_t launch_quant_rows(const RowsLaunch& a, bool f32, cudaStream_t stream);
cudaError_t launch_combine(const CombineLaunch& a, bool f32, cudaStream_t stream);
cudaError_t launch_grouped(const GroupedLaunch& a, bool e4m3, bool gated, bool kn, cudaStream_t stream);

}  // namespace tsffn
