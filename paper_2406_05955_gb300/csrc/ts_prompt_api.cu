// ts_prompt_api.cu -- the C ABI of the operators over many tokens (include/ts_ffn.h): argument checks, handles, launches.
#include <stdint.h>

#include <algorithm>
#include <new>
#include <vector>

#include "ts_arena.h"
#include "ts_ffn.h"
#include "ts_grouped.h"
#include "ts_kernels.cuh"

using namespace tsffn;

namespace {

bool aligned16(const void* p) { return ((uintptr_t)p & 15u) == 0; }
ts_status launched(cudaError_t e) { return e == cudaSuccess ? TS_OK : TS_ERR_CUDA; }
int elem_size(ts_dtype dt) { return dt == TS_F32 ? 4 : dt == TS_BF16 ? 2 : 1; }

// Arguments that ts_gather_rows and ts_quant_rows share.
ts_status check_rows(const void* x, int64_t ldx, ts_dtype dtype, int n_src, int k, int max_rows, const void* out) {
    if (dtype != TS_F32 && dtype != TS_BF16) return TS_ERR_INVALID_ARG;
    if (n_src < 0 || k < 1 || max_rows < 0 || ldx < k) return TS_ERR_INVALID_ARG;
    if (max_rows == 0) return TS_OK;
    if (!out || (!x && n_src > 0)) return TS_ERR_INVALID_ARG;
    const int64_t size = elem_size(dtype);
    if (!aligned16(x) || !aligned16(out) || ldx * size % 16 != 0 || k * size % 16 != 0) return TS_ERR_INVALID_ARG;
    return TS_OK;
}

}  // namespace

struct ts_grouped {
    int n_groups = 0, n = 0, k = 0, max_rows = 0;
    ts_dtype dt = TS_BF16;
    ts_layout layout = TS_NK;
    bool gated = false;
    Arena arena;
    GroupWeights* weights = nullptr;  // device [n_groups]
    unsigned* status = nullptr;
    int pairs = 0, part_chunks = 1;
    float* partial = nullptr;
    unsigned* arrived = nullptr;
};

namespace {

// Tensor maps of the weights, scratch and its contents.
ts_status grouped_init(ts_grouped* h, std::vector<GroupWeights>& table, int n_groups, int n, int k, ts_dtype wdtype,
                       ts_layout layout, const void* const* w, const void* const* w_up, const float* const* scale,
                       const float* const* scale_up, int max_rows) {
    const bool e8 = wdtype == TS_E4M3, gated = w_up != nullptr, kn = layout == TS_KN;
    h->n_groups = n_groups;
    h->n = n;
    h->k = k;
    h->max_rows = max_rows;
    h->dt = wdtype;
    h->layout = layout;
    h->gated = gated;
    if (prepare_grouped() != cudaSuccess) return TS_ERR_CUDA;
    h->pairs = grouped_pairs(e8, gated, kn);
    if (h->pairs < 1) return TS_ERR_CUDA;
    h->part_chunks = grouped_part_chunks(max_rows);
    const int box = grouped_w_box(gated, kn);
    const int64_t cols = kn ? n : k, rows = kn ? k : n;
    for (int e = 0; e < n_groups; ++e) {
        GroupWeights& g = table[(size_t)e];
        g.ws = e8 ? scale[e] : nullptr;
        g.us = e8 && gated ? scale_up[e] : nullptr;
        if (!grouped_map(&g.w, w[e], e8, cols, rows, cols, box)) return TS_ERR_CUDA;
        if (gated && !grouped_map(&g.u, w_up[e], e8, cols, rows, cols, box)) return TS_ERR_CUDA;
    }
    const size_t bytes = sizeof(GroupWeights) * (size_t)n_groups;
    const size_t o_w = h->arena.take(bytes), o_status = h->arena.take(sizeof(unsigned));
    const size_t o_arrived = h->arena.take(grouped_arrived(h->pairs) * sizeof(unsigned));
    const size_t o_partial = h->arena.take(grouped_partial_bytes(h->pairs, h->part_chunks));
    const ts_status s = alloc_arena(&h->arena);
    if (s != TS_OK) return s;
    h->weights = h->arena.at<GroupWeights>(o_w);
    h->status = h->arena.at<unsigned>(o_status);
    h->arrived = h->arena.at<unsigned>(o_arrived);
    h->partial = h->arena.at<float>(o_partial);
    if (cudaMemcpy(h->weights, table.data(), bytes, cudaMemcpyHostToDevice) != cudaSuccess ||
        cudaStreamSynchronize(cudaStreamLegacy) != cudaSuccess)
        return TS_ERR_CUDA;
    return TS_OK;
}

}  // namespace

extern "C" {

ts_status ts_route(const float* logits, int tokens, int n_experts, int top_k, int32_t* sel, float* w,
                   int32_t* offsets, int32_t* rows, int32_t* slots, cudaStream_t stream) {
    if (tokens < 0 || n_experts < 1 || n_experts > kMaxRouteExperts || top_k < 1 || top_k > kMaxRouteK ||
        top_k > n_experts || !offsets || (long long)tokens * top_k > INT32_MAX)
        return TS_ERR_INVALID_ARG;
    if (tokens > 0 && (!logits || !sel || !w || !rows || !slots)) return TS_ERR_INVALID_ARG;
    return launched(launch_route({logits, tokens, n_experts, top_k, sel, w, offsets, rows, slots}, stream));
}

ts_status ts_gather_rows(const void* x, int64_t ldx, ts_dtype dtype, int n_src, int k, const int32_t* rows,
                         const int32_t* n, int max_rows, void* out, cudaStream_t stream) {
    const ts_status s = check_rows(x, ldx, dtype, n_src, k, max_rows, out);
    if (s != TS_OK || max_rows == 0) return s;
    return launched(launch_gather_rows({x, ldx, n_src, k, rows, n, max_rows, out, nullptr}, elem_size(dtype), stream));
}

ts_status ts_quant_rows(const void* x, int64_t ldx, ts_dtype dtype, int n_src, int k, const int32_t* rows,
                        const int32_t* n, int max_rows, void* q, float* scale, cudaStream_t stream) {
    const ts_status s = check_rows(x, ldx, dtype, n_src, k, max_rows, q);
    if (s != TS_OK) return s;
    if (k % 16 != 0) return TS_ERR_INVALID_ARG;
    if (max_rows == 0) return TS_OK;
    if (!scale) return TS_ERR_INVALID_ARG;
    return launched(launch_quant_rows({x, ldx, n_src, k, rows, n, max_rows, q, scale}, dtype == TS_F32, stream));
}

ts_status ts_combine_rows(const void* src, ts_dtype dtype, int n_rows, int n, const int32_t* slots, const float* w,
                          int tokens, int top_k, float* y, cudaStream_t stream) {
    if ((dtype != TS_F32 && dtype != TS_BF16) || n_rows < 0 || n < 1 || tokens < 0 || top_k < 1 || top_k > kMaxRouteK)
        return TS_ERR_INVALID_ARG;
    if (tokens == 0) return TS_OK;
    if ((!src && n_rows > 0) || !slots || !w || !y) return TS_ERR_INVALID_ARG;
    return launched(launch_combine({src, n_rows, n, slots, w, tokens, top_k, y}, dtype == TS_F32, stream));
}

ts_status ts_grouped_create(ts_grouped** out, int n_groups, int n, int k, ts_dtype wdtype, ts_layout layout,
                            const void* const* w, const void* const* w_up, const float* const* scale,
                            const float* const* scale_up, int max_rows) {
    if (!out || n_groups < 1 || n_groups > kMaxGroups || n < 1 || k < 1 || max_rows < 1 || !w) return TS_ERR_INVALID_ARG;
    if (layout != TS_NK && layout != TS_KN) return TS_ERR_INVALID_ARG;
    if (wdtype == TS_F32 || wdtype == TS_INT4) return TS_ERR_UNSUPPORTED;
    if (wdtype != TS_BF16 && wdtype != TS_E4M3) return TS_ERR_INVALID_ARG;
    const bool e8 = wdtype == TS_E4M3, gated = w_up != nullptr;
    if (k % (e8 ? 16 : 8) != 0 || (layout == TS_KN && n % 8 != 0)) return TS_ERR_INVALID_ARG;
    if (layout == TS_KN && (e8 || gated)) return TS_ERR_UNSUPPORTED;
    if (e8 != (scale != nullptr) || (e8 && gated) != (scale_up != nullptr)) return TS_ERR_INVALID_ARG;
    for (int e = 0; e < n_groups; ++e)
        if (!w[e] || !aligned16(w[e]) || (gated && (!w_up[e] || !aligned16(w_up[e]))) || (e8 && !scale[e]) ||
            (e8 && gated && !scale_up[e]))
            return TS_ERR_INVALID_ARG;
    std::vector<GroupWeights> table;
    ts_grouped* h = nullptr;
    try {
        table.resize((size_t)n_groups);
        h = new ts_grouped;
        h->arena.guards.reserve(8);
    } catch (const std::bad_alloc&) {
        delete h;
        return TS_ERR_OOM;
    }
    const ts_status s = grouped_init(h, table, n_groups, n, k, wdtype, layout, w, w_up, scale, scale_up, max_rows);
    if (s != TS_OK) {
        ts_grouped_destroy(h);
        return s;
    }
    *out = h;
    return TS_OK;
}

void ts_grouped_destroy(ts_grouped* h) {
    if (!h) return;
    if (h->arena.base) cudaFree(h->arena.base);
    delete h;
}

ts_status ts_grouped_forward(ts_grouped* h, const void* x, int64_t ldx, const float* x_scale, int64_t ld_scale,
                             const int32_t* offsets, int rows, void* y, int64_t ldy, ts_dtype ydtype,
                             cudaStream_t stream) {
    if (!h || rows < 0 || rows > h->max_rows || (ydtype != TS_F32 && ydtype != TS_BF16)) return TS_ERR_INVALID_ARG;
    if (!offsets && h->n_groups != 1) return TS_ERR_INVALID_ARG;
    if (rows == 0) return TS_OK;
    const bool e8 = h->dt == TS_E4M3;
    if (!x || !y || !aligned16(x) || ldx < h->k || ldx * elem_size(h->dt) % 16 != 0 || ldy < h->n)
        return TS_ERR_INVALID_ARG;
    if (e8 ? (!x_scale || ld_scale < rows) : x_scale != nullptr) return TS_ERR_INVALID_ARG;
    GroupedLaunch a;
    // boxes of up to half of the widest tile that so many rows can give
    const int widest = std::min(kMaxTileRows, (rows + 15) / 16 * 16);
    for (int i = 0; i < kXMaps; ++i) {
        if (!grouped_map(&a.x[i], x, e8, h->k, rows, ldx, 8 << i)) return TS_ERR_CUDA;
        if ((8 << i) >= widest / 2) break;
    }
    a.n_groups = h->n_groups;
    a.n = h->n;
    a.k = h->k;
    a.weights = h->weights;
    a.x_scale = x_scale;
    a.ld_scale = ld_scale;
    a.offsets = offsets;
    a.rows = rows;
    a.y = y;
    a.ldy = ldy;
    a.y_f32 = ydtype == TS_F32;
    a.y_vec = ldy % 8 == 0 && aligned16(y);
    a.pairs = h->pairs;
    a.part_chunks = h->part_chunks;
    a.partial = h->partial;
    a.arrived = h->arrived;
    a.status = h->status;
    return launched(launch_grouped(a, e8, h->gated, h->layout == TS_KN, stream));
}

ts_status ts_grouped_get_error(ts_grouped* h, cudaStream_t stream) {
    if (!h) return TS_ERR_INVALID_ARG;
    unsigned bits = 0;
    if (cudaMemcpyAsync(&bits, h->status, sizeof bits, cudaMemcpyDeviceToHost, stream) != cudaSuccess ||
        cudaMemsetAsync(h->status, 0, sizeof bits, stream) != cudaSuccess || cudaStreamSynchronize(stream) != cudaSuccess)
        return TS_ERR_CUDA;
    return bits & kStatusTimeout ? TS_ERR_TIMEOUT : bits & kStatusBadIndex ? TS_ERR_BAD_INDEX : TS_OK;
}

ts_status ts_grouped_check_scratch(ts_grouped* h, cudaStream_t stream) {
    return h ? check_arena(h->arena, stream) : TS_ERR_INVALID_ARG;
}

}  // extern "C"
