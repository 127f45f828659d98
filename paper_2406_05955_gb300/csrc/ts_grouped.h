// ts_grouped.h -- launch parameters and launchers of the operators over many tokens (ts_route.cu, ts_rows.cu, ts_grouped.cu).
#pragma once

#include <cuda.h>
#include <cuda_runtime.h>
#include <stdint.h>

namespace tsffn {

constexpr int kMaxRouteExperts = 256;
constexpr int kMaxRouteK = 8;
constexpr int kMaxGroups = 256;
// Up to these sizes the kernels' 32-bit counts and the grids' second dimension hold.
constexpr int kMaxGroupedK = 1 << 28;
constexpr int kMaxRowElems = 1 << 24;  // of a row that is copied or rounded
constexpr int kMaxRows = 1 << 30;      // rows, and outputs of a product
constexpr int kScaleBlock = 128;  // elements of one scale, along k and along n

struct RouteLaunch {
    const float* logits;  // [tokens][n_experts]
    int tokens, n_experts, top_k;
    int32_t* sel;         // [tokens][top_k]
    float* w;             // [tokens][top_k]
    int32_t* offsets;     // [n_experts + 1]
    int32_t* rows;        // [tokens * top_k]
    int32_t* slots;       // [tokens][top_k]
    int32_t* shape;       // nullptr, or {tokens, top_k} of what sel and w hold
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

// Weights of one group: where TMA finds them, and TS_E4M3 scales. Device memory.
struct GroupWeights {
    CUtensorMap w;
    CUtensorMap u;   // gated
    const float* ws;
    const float* us;
};

constexpr int kXMaps = 5;         // maps of x: boxes of 8, 16, 32, 64 and 128 rows
constexpr int kMaxTileRows = 256; // rows of x of a tile
constexpr int kEpiWarps = 8;

// A CTA pair's tiles of the products, and the parts of tiles that several pairs share.
struct GroupedLaunch {
    CUtensorMap x[kXMaps];
    int n_groups, n, k;
    const GroupWeights* weights;  // device [n_groups]
    const float* x_scale;         // [k / 128][ld_scale]
    int64_t ld_scale;
    const int32_t* offsets;       // [n_groups + 1] or nullptr (one group)
    int rows;
    void* y;
    int64_t ldy;
    int y_f32;
    int y_vec;                    // bf16 rows of y start on 16-byte boundaries
    int pairs;                    // CTA pairs of the grid
    int part_chunks;              // 64-column chunks of a warp's part in `partial`: 1 or 2
    float* partial;               // [pairs][2][2 CTAs][kEpiWarps][part_chunks * 2048]
    unsigned* arrived;            // [2 * pairs][2 CTAs][kEpiWarps], zero between calls
    unsigned* status;
    int test_stall;               // ts_grouped_set_test_stall
};

// Whether an e4m3 product takes the rows of x as the MMA's M (see Kind in ts_grouped.cu): where the groups have enough of
// them on average to fill a tile of 256 reasonably. Over 8 groups of 65 rows (d = 4096, m = 14336) gated products take 202
// us so and 207 otherwise, of 49 201 and 195; down products of 128 rows 110 and 101. All of that is over equal groups: the
// host knows the buffer's rows and the number of groups, not which groups have rows, nor how many rows lie behind the last one.
inline bool grouped_x_is_m(bool e4m3, bool gated, long long rows, int groups) {
    return e4m3 && rows > (gated ? 64ll : 128ll) * groups;
}

// Bytes of GroupedLaunch::partial for tiles of up to `rows` rows, and entries of `arrived`.
inline int grouped_part_chunks(int rows) { return rows > 64 ? 2 : 1; }  // (rows as M have two from 65 rows on)
inline size_t grouped_partial_bytes(int pairs, int chunks) { return (size_t)pairs * 2 * 2 * kEpiWarps * chunks * 2048 * 4; }
inline size_t grouped_arrived(int pairs) { return (size_t)pairs * 2 * 2 * kEpiWarps; }

// Tensor map of a [rows][cols] matrix (ld elements apart) whose boxes are 128 bytes wide and box_rows high, with the
// 128-byte swizzle; false where it cannot be made.
bool grouped_map(CUtensorMap* m, const void* p, bool e4m3, int64_t cols, int64_t rows, int64_t ld, int box_rows);
constexpr int grouped_w_box(bool gated, bool kn) { return gated || kn ? 64 : 128; }
cudaError_t prepare_grouped();
// CTA pairs that can be resident at once (the kernels take the same shared memory and threads).
int grouped_pairs();

// Launches a kernel whose threads wait (pdl_wait) for what is before it on the stream before they read or write anything in
// memory: its CTAs are then brought up while that ends, and calls in a row take 1 to 3 us less each (one row,
// 4096 x 14336 e4m3: 25.3 -> 23.1 us; 16 rows, 4096 x 4096 bf16: 18.5 -> 15.7).
template <typename... Args>
cudaError_t launch_after(void (*kernel)(Args...), cudaLaunchConfig_t cfg, const Args&... args) {
    cudaLaunchAttribute at{};
    at.id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at.val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = &at;
    cfg.numAttrs = 1;
    return cudaLaunchKernelEx(&cfg, kernel, args...);
}
inline cudaLaunchConfig_t launch_shape(dim3 grid, int threads, cudaStream_t stream) {
    cudaLaunchConfig_t cfg{};
    cfg.gridDim = grid;
    cfg.blockDim = dim3((unsigned)threads);
    cfg.stream = stream;
    return cfg;
}

cudaError_t launch_route(const RouteLaunch& a, cudaStream_t stream);
cudaError_t launch_gather_rows(const RowsLaunch& a, int elem_bytes, cudaStream_t stream);
cudaError_t launch_quant_rows(const RowsLaunch& a, bool f32, cudaStream_t stream);
cudaError_t launch_combine(const CombineLaunch& a, bool f32, cudaStream_t stream);
cudaError_t launch_grouped(const GroupedLaunch& a, bool e4m3, bool gated, bool kn, cudaStream_t stream);

}  // namespace tsffn
