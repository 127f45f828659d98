// ts_adapt.h -- launch parameters and launchers of what an adapted layer needs beside its frozen weights: low-rank adapters
// and their gradients (ts_adapt.cu), the gated activation kept in 8 bits (ts_drelu.cu), the balance loss and the gradient
// of routing (ts_balance.cu), the backward pass of combined rows (ts_combine_bwd.cu).
#pragma once

#include <cuda_runtime.h>
#include <stdint.h>

namespace tsffn {

constexpr int kMaxAdapters = 255;  // and one group of rows that have none: kMaxRouteExperts
constexpr int kMaxRank = 128;
constexpr int kFewRows = 512;      // of a call without a list
constexpr int kWideRank = 64;      // of the kernel of ts_adapt_wide.cu

struct AdaptLaunch {
    const void* x;           // [rows] rows of k bf16, ldx apart
    int64_t ldx;
    int rows, k;
    const void* a;           // [n_adapters][r][k] bf16
    const void* b;           // [n_adapters][r][n] bf16
    const float* scale;      // [n_adapters] or nullptr
    const int32_t* ranks;    // [n_adapters] or nullptr
    int n_adapters, r, n;
    const int32_t* ids;      // [rows] (calls without a list)
    const int32_t* list;     // [rows], by adapter, or nullptr
    const int32_t* offsets;  // [n_adapters + 2]
    const void* y;           // [rows] rows of n, ldy apart, or nullptr
    int64_t ldy;
    void* out;               // the same, ldo apart (nullptr: h alone)
    int64_t ldo;
    float* h;                // [rows][r] or nullptr
    int test_stall;          // ts_adapt_set_test_stall
};

// The most tiles of up to mt rows that a list of so many rows, and those of no adapter, can have.
inline long long most_tiles(int rows, int n_adapters, int mt) {
    return (long long)rows / mt + (rows < n_adapters + 1 ? rows : n_adapters + 1);
}

struct AdapterGradsLaunch {
    const float* h;          // [rows][r]
    int r;
    const void* x;           // [rows] rows of k, ldx apart, bf16 or e4m3
    int64_t ldx;
    const float* x_scale;    // [k / 128][ld_scale] (e4m3)
    int64_t ld_scale;
    int rows, k, n_adapters;
    const int32_t* list;
    const int32_t* offsets;
    float* grad;             // [n_adapters][r][k]
    int accumulate;
    int follows;             // what it reads was there before the kernel before it, which is one of these too, began
    int test_stall;          // ts_adapt_set_test_stall
};

struct DreluLaunch {
    const void* g;           // [rows] rows of m, ldg apart
    const void* u;
    int64_t ldg, ldu;
    const int32_t* n;        // device count or nullptr
    int rows, m;
    void* c;                 // bf16, ldc apart
    int64_t ldc;
    uint8_t* q_gate;         // [rows][m] e4m3, or all four nullptr
    uint8_t* q_up;
    float* s_gate;           // [m / 128][rows]
    float* s_up;
};

struct DreluBackwardLaunch {
    const void* dc;          // [rows] rows of m, ldd apart
    int64_t ldd;
    const uint8_t* q_gate;
    const uint8_t* q_up;
    const float* s_gate;
    const float* s_up;
    const int32_t* n;
    int rows, m;
    void* dg;                // bf16
    void* du;
    void* c;                 // or nullptr
    int64_t ldg, ldu, ldc;
};

struct BalanceLaunch {
    const float* logits;     // [tokens][n_experts]
    int tokens, n_experts, top_k;
    const int32_t* sel;      // [tokens][top_k]
    float* loss;             // [1]
    int32_t* counts;         // [n_experts]
    float* share;            // [n_experts]
    int32_t* totals;         // {live tokens, picks}
    float* work;             // balance_work floats
};

struct RouteBackwardLaunch {
    const float* logits;     // [tokens][n_experts]
    int tokens, n_experts, top_k;
    const int32_t* sel;      // [tokens][top_k]
    const float* w;
    const float* dw;         // or nullptr
    const int32_t* counts;   // and totals, dloss; or all nullptr
    const int32_t* totals;
    const float* dloss;
    float* dlogits;
};

struct CombineBackwardLaunch {
    const void* dy;          // [tokens][n]
    const void* src;         // [n_rows][n]
    int n_rows, n;
    const int32_t* slots;    // [tokens][top_k]
    const float* w;
    const int32_t* rows;     // [n_rows]
    int tokens, top_k;
    void* dsrc;              // [n_rows][n]
    float* dw;               // [tokens][top_k]
};

size_t balance_work(int tokens, int n_experts);  // floats

cudaError_t launch_list_rows(const int32_t* ids, int n_rows, int n_groups, int32_t* rows, int32_t* offsets,
                             cudaStream_t stream);
cudaError_t launch_adapt(const AdaptLaunch& a, bool y_f32, cudaStream_t stream);
cudaError_t launch_adapt_wide(const AdaptLaunch& a, bool y_f32, cudaStream_t stream);
// How many waits of the kernels on the current device have given up so far: copied on `stream`.
cudaError_t adapt_wide_timeouts(unsigned* n, cudaStream_t stream);
cudaError_t adapter_grads_timeouts(unsigned* n, cudaStream_t stream);
cudaError_t launch_adapter_grads(const AdapterGradsLaunch& a, bool e4m3, cudaStream_t stream);
cudaError_t launch_drelu(const DreluLaunch& a, bool f32, cudaStream_t stream);
cudaError_t launch_drelu_backward(const DreluBackwardLaunch& a, bool f32, cudaStream_t stream);
cudaError_t launch_balance(const BalanceLaunch& a, cudaStream_t stream);
cudaError_t launch_route_backward(const RouteBackwardLaunch& a, cudaStream_t stream);
cudaError_t launch_combine_backward(const CombineBackwardLaunch& a, bool dy_f32, bool src_f32, cudaStream_t stream);

}  // namespace tsffn
