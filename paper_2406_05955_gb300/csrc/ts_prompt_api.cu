// ts_prompt_api.cu -- the C ABI of the operators over many tokens (include/ts_ffn.h): argument checks, handles, scratch,
// launches, and the forward of a whole layer of experts, which is those operators in a row.
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
bool aligned_for(const void* p, ts_dtype dt) { return (uintptr_t)p % (unsigned)elem_size(dt) == 0; }

// Arguments that ts_gather_rows and ts_quant_rows share.
ts_status check_rows(const void* x, int64_t ldx, ts_dtype dtype, int n_src, int k, int max_rows, const void* out) {
    if (dtype != TS_F32 && dtype != TS_BF16) return TS_ERR_INVALID_ARG;
    if (n_src < 0 || k < 1 || max_rows < 0 || ldx < k) return TS_ERR_INVALID_ARG;
    if (k > kMaxRowElems || max_rows > kMaxRows) return TS_ERR_UNSUPPORTED;
    if (max_rows == 0) return TS_OK;
    if (!out || (!x && n_src > 0)) return TS_ERR_INVALID_ARG;
    const int64_t size = elem_size(dtype);
    if (!aligned16(x) || !aligned16(out) || ldx * size % 16 != 0 || k * size % 16 != 0) return TS_ERR_INVALID_ARG;
    return TS_OK;
}

// Products of one kind and size, without scratch.
struct Products {
    int n_groups = 0, n = 0, k = 0;
    ts_dtype dt = TS_BF16;
    bool gated = false, kn = false;
    GroupWeights* weights = nullptr;  // device [n_groups]
};

// Scratch that products of up to max_rows rows can share, one launch at a time.
struct ProductScratch {
    int pairs = 0, part_chunks = 1;
    size_t o_partial = 0, o_arrived = 0, o_status = 0;
    float* partial = nullptr;
    unsigned* arrived = nullptr;
    unsigned* status = nullptr;
    int device = -1;

    // False where the kernels cannot be resident.
    bool plan(Arena* ar, int max_rows) {
        if (cudaGetDevice(&device) != cudaSuccess) return false;
        pairs = grouped_pairs();
        part_chunks = grouped_part_chunks(max_rows);
        if (pairs < 1) return false;
        o_status = ar->take(sizeof(unsigned));
        o_arrived = ar->take(grouped_arrived(pairs) * sizeof(unsigned));
        o_partial = ar->take(grouped_partial_bytes(pairs, part_chunks));
        return true;
    }
    void place(const Arena& ar) {
        status = ar.at<unsigned>(o_status);
        arrived = ar.at<unsigned>(o_arrived);
        partial = ar.at<float>(o_partial);
    }
};

// Whether a handle's device is the current one.
bool here(int device) {
    int now = -1;
    return cudaGetDevice(&now) == cudaSuccess && now == device;
}

// Whether the weights and scales that a product of n_groups groups needs are there, aligned.
bool weights_ok(int n_groups, bool e8, const void* const* w, const float* const* scale) {
    if (!w || e8 != (scale != nullptr)) return false;
    for (int i = 0; i < n_groups; ++i)
        if (!w[i] || !aligned16(w[i]) || (e8 && !scale[i])) return false;
    return true;
}

// Maps of a product's weights in `table`, the host copy of P.weights.
bool map_weights(const Products& P, GroupWeights* table, const void* const* w, const void* const* w_up,
                 const float* const* scale, const float* const* scale_up) {
    const bool e8 = P.dt == TS_E4M3;
    const int box = grouped_w_box(P.gated, P.kn);
    const int64_t cols = P.kn ? P.n : P.k, rows = P.kn ? P.k : P.n;
    for (int i = 0; i < P.n_groups; ++i) {
        GroupWeights& g = table[i];
        g.ws = e8 ? scale[i] : nullptr;
        g.us = e8 && P.gated ? scale_up[i] : nullptr;
        if (!grouped_map(&g.w, w[i], e8, cols, rows, cols, box)) return false;
        if (P.gated && !grouped_map(&g.u, w_up[i], e8, cols, rows, cols, box)) return false;
    }
    return true;
}

// Copies to device memory and waits for the default stream: what alloc_arena and this have written there is in place
// before a kernel of any stream can read it.
ts_status copy_in(void* to, const void* from, size_t bytes) {
    return cudaMemcpy(to, from, bytes, cudaMemcpyHostToDevice) == cudaSuccess &&
                   cudaStreamSynchronize(cudaStreamLegacy) == cudaSuccess
               ? TS_OK
               : TS_ERR_CUDA;
}

ts_status run_products(const Products& P, const ProductScratch& S, const void* x, int64_t ldx, const float* x_scale,
                       int64_t ld_scale, const int32_t* offsets, int rows, void* y, int64_t ldy, bool y_f32,
                       cudaStream_t stream, bool test_stall = false) {
    const bool e8 = P.dt == TS_E4M3;
    GroupedLaunch a;
    // boxes of up to half of the widest tile that so many rows can give
    const int widest = grouped_x_is_m(e8, P.gated, rows, P.n_groups) ? kMaxTileRows
                                                                     : std::min(kMaxTileRows, (rows + 15) / 16 * 16);
    for (int i = 0; i < kXMaps; ++i) {
        if (!grouped_map(&a.x[i], x, e8, P.k, rows, ldx, 8 << i)) return TS_ERR_CUDA;
        if ((8 << i) >= widest / 2) break;
    }
    a.n_groups = P.n_groups;
    a.n = P.n;
    a.k = P.k;
    a.weights = P.weights;
    a.x_scale = x_scale;
    a.ld_scale = ld_scale;
    a.offsets = offsets;
    a.rows = rows;
    a.y = y;
    a.ldy = ldy;
    a.y_f32 = y_f32;
    a.y_vec = ldy % 8 == 0 && aligned16(y);
    a.pairs = S.pairs;
    a.part_chunks = S.part_chunks;
    a.partial = S.partial;
    a.arrived = S.arrived;
    a.status = S.status;
    a.test_stall = test_stall;
    return launched(launch_grouped(a, e8, P.gated, P.kn, stream));
}

ts_status read_status(const ProductScratch& S, cudaStream_t stream) {
    unsigned bits = 0;
    if (cudaMemcpyAsync(&bits, S.status, sizeof bits, cudaMemcpyDeviceToHost, stream) != cudaSuccess ||
        cudaMemsetAsync(S.status, 0, sizeof bits, stream) != cudaSuccess || cudaStreamSynchronize(stream) != cudaSuccess)
        return TS_ERR_CUDA;
    // a launch that gave up may have left tiles half counted (and the next one may be on another stream)
    if ((bits & kStatusTimeout) &&
        (cudaMemsetAsync(S.arrived, 0, grouped_arrived(S.pairs) * sizeof(unsigned), stream) != cudaSuccess ||
         cudaStreamSynchronize(stream) != cudaSuccess))
        return TS_ERR_CUDA;
    return bits & kStatusTimeout ? TS_ERR_TIMEOUT : bits & kStatusBadIndex ? TS_ERR_BAD_INDEX : TS_OK;
}

// Sizes that ts_experts_create and ts_prompt_create take alike.
ts_status check_experts(int d, int m, int n_experts, int top_k, ts_dtype wdtype) {
    if (d < 1 || m < 1 || n_experts < 1 || n_experts > kMaxRouteExperts || top_k < 1 || top_k > kMaxRouteK ||
        top_k > n_experts)
        return TS_ERR_INVALID_ARG;
    if (wdtype == TS_F32 || wdtype == TS_INT4) return TS_ERR_UNSUPPORTED;
    if (wdtype != TS_BF16 && wdtype != TS_E4M3) return TS_ERR_INVALID_ARG;
    if (d > kMaxRowElems || m > kMaxRowElems) return TS_ERR_UNSUPPORTED;
    const int step = wdtype == TS_E4M3 ? 16 : 8;
    return d % step == 0 && m % step == 0 ? TS_OK : TS_ERR_INVALID_ARG;
}

}  // namespace

struct ts_grouped {
    Products p;
    ProductScratch s;
    Arena arena;
    int max_rows = 0;
    bool test_stall = false;  // ts_grouped_set_test_stall
};

struct ts_experts {
    int d = 0, m = 0, n_experts = 0, top_k = 0;
    ts_dtype dt = TS_BF16;
    bool routed = false;
    int device = -1;
    Products router, gate_up, down;
    Arena arena;
};

struct ts_prompt {
    int d = 0, m = 0, n_experts = 0, top_k = 0, max_tokens = 0;
    ts_dtype dt = TS_BF16;
    Arena arena;
    ProductScratch s;
    float* logits = nullptr;          // [max_tokens][n_experts]
    int32_t* sel = nullptr;           // [max_tokens][top_k]
    float* w = nullptr;
    int32_t* slots = nullptr;
    int32_t* rows = nullptr;          // [max_tokens * top_k]
    int32_t* offsets = nullptr;       // [n_experts + 1]
    int32_t* shape = nullptr;         // {tokens, top_k} of sel and w, by the forward that ran last (of a call or a replay)
    void* x = nullptr;                // [rows][d] in the experts' order, bf16 or e4m3
    float* x_scale = nullptr;         // [d / 128][rows]
    __nv_bfloat16* c = nullptr;       // [rows][m]
    void* cq = nullptr;               // [rows][m] e4m3
    float* c_scale = nullptr;         // [m / 128][rows]
    float* y = nullptr;               // [rows][d]
    int last_tokens = 0, last_k = 0;  // of the last call; last_k 0: none, without a router, or failed
};

extern "C" {

ts_status ts_route(const float* logits, int tokens, int n_experts, int top_k, int32_t* sel, float* w,
                   int32_t* offsets, int32_t* rows, int32_t* slots, cudaStream_t stream) {
    if (tokens < 0 || n_experts < 1 || n_experts > kMaxRouteExperts || top_k < 1 || top_k > kMaxRouteK ||
        top_k > n_experts || !offsets || (long long)tokens * top_k >= 1ll << 30)
        return TS_ERR_INVALID_ARG;
    if (tokens > 0 && (!logits || !sel || !w || !rows || !slots)) return TS_ERR_INVALID_ARG;
    return launched(launch_route({logits, tokens, n_experts, top_k, sel, w, offsets, rows, slots, nullptr}, stream));
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
    if (n > kMaxRows || tokens > kMaxRows) return TS_ERR_UNSUPPORTED;
    if (tokens == 0) return TS_OK;
    if ((!src && n_rows > 0) || !aligned_for(src, dtype) || !slots || !w || !y) return TS_ERR_INVALID_ARG;
    return launched(launch_combine({src, n_rows, n, slots, w, tokens, top_k, y}, dtype == TS_F32, stream));
}

// ---------------------------------------------------------------------------
// grouped products
// ---------------------------------------------------------------------------
ts_status ts_grouped_create(ts_grouped** out, int n_groups, int n, int k, ts_dtype wdtype, ts_layout layout,
                            const void* const* w, const void* const* w_up, const float* const* scale,
                            const float* const* scale_up, int max_rows) {
    if (!out || n_groups < 1 || n_groups > kMaxGroups || n < 1 || k < 1 || max_rows < 1 || !w) return TS_ERR_INVALID_ARG;
    if (layout != TS_NK && layout != TS_KN) return TS_ERR_INVALID_ARG;
    if (wdtype == TS_F32 || wdtype == TS_INT4) return TS_ERR_UNSUPPORTED;
    if (wdtype != TS_BF16 && wdtype != TS_E4M3) return TS_ERR_INVALID_ARG;
    const bool e8 = wdtype == TS_E4M3, gated = w_up != nullptr;
    if (k > kMaxGroupedK || n > kMaxRows || max_rows > kMaxRows) return TS_ERR_UNSUPPORTED;
    if (k % (e8 ? 16 : 8) != 0 || (layout == TS_KN && n % 8 != 0)) return TS_ERR_INVALID_ARG;
    if (layout == TS_KN && (e8 || gated)) return TS_ERR_UNSUPPORTED;
    if (!weights_ok(n_groups, e8, w, scale) || (gated && !weights_ok(n_groups, e8, w_up, scale_up)) || (!gated && scale_up))
        return TS_ERR_INVALID_ARG;
    if (prepare_grouped() != cudaSuccess) return TS_ERR_CUDA;
    ts_grouped* h = nullptr;
    ts_status s = TS_ERR_OOM;
    try {
        h = new ts_grouped;
        std::vector<GroupWeights> table((size_t)n_groups);
        const size_t bytes = sizeof(GroupWeights) * table.size();
        h->p.n_groups = n_groups;
        h->p.n = n;
        h->p.k = k;
        h->p.dt = wdtype;
        h->p.gated = gated;
        h->p.kn = layout == TS_KN;
        h->max_rows = max_rows;
        const size_t o_w = h->arena.take(bytes);
        if (!map_weights(h->p, table.data(), w, w_up, scale, scale_up) || !h->s.plan(&h->arena, max_rows)) s = TS_ERR_CUDA;
        else s = alloc_arena(&h->arena);
        if (s == TS_OK) {
            h->s.place(h->arena);
            h->p.weights = h->arena.at<GroupWeights>(o_w);
            s = copy_in(h->p.weights, table.data(), bytes);
        }
    } catch (const std::bad_alloc&) {
        s = TS_ERR_OOM;
    }
    if (s != TS_OK) {
        ts_grouped_destroy(h);
        return s;
    }
    *out = h;
    return TS_OK;
}

void ts_grouped_destroy(ts_grouped* h) {
    if (!h) return;
    free_arena(&h->arena);
    delete h;
}

ts_status ts_grouped_forward(ts_grouped* h, const void* x, int64_t ldx, const float* x_scale, int64_t ld_scale,
                             const int32_t* offsets, int rows, void* y, int64_t ldy, ts_dtype ydtype,
                             cudaStream_t stream) {
    if (!h || rows < 0 || rows > h->max_rows || (ydtype != TS_F32 && ydtype != TS_BF16)) return TS_ERR_INVALID_ARG;
    if (!offsets && h->p.n_groups != 1) return TS_ERR_INVALID_ARG;
    if (rows == 0) return TS_OK;
    if (!here(h->s.device) || !x || !y || !aligned16(x) || ldx < h->p.k || ldx * elem_size(h->p.dt) % 16 != 0 ||
        ldy < h->p.n || !aligned_for(y, ydtype))
        return TS_ERR_INVALID_ARG;
    if (h->p.dt == TS_E4M3 ? (!x_scale || ld_scale < rows) : x_scale != nullptr) return TS_ERR_INVALID_ARG;
    return run_products(h->p, h->s, x, ldx, x_scale, ld_scale, offsets, rows, y, ldy, ydtype == TS_F32, stream, h->test_stall);
}

ts_status ts_grouped_get_error(ts_grouped* h, cudaStream_t stream) {
    return h ? read_status(h->s, stream) : TS_ERR_INVALID_ARG;
}

ts_status ts_grouped_set_test_stall(ts_grouped* h, int on) {
    if (!h) return TS_ERR_INVALID_ARG;
    h->test_stall = on != 0;
    return TS_OK;
}

ts_status ts_grouped_check_scratch(ts_grouped* h, cudaStream_t stream) {
    return h ? check_arena(h->arena, stream) : TS_ERR_INVALID_ARG;
}

// ---------------------------------------------------------------------------
// layers of experts over many tokens
// ---------------------------------------------------------------------------
ts_status ts_experts_create(ts_experts** out, int d, int m, int n_experts, int top_k, ts_dtype wdtype,
                            const void* w_router, const void* const* w_gate, const void* const* w_up,
                            const void* const* w_down, const float* const* s_gate, const float* const* s_up,
                            const float* const* s_down) {
    if (!out) return TS_ERR_INVALID_ARG;
    const ts_status sizes = check_experts(d, m, n_experts, top_k, wdtype);
    if (sizes != TS_OK) return sizes;
    const bool e8 = wdtype == TS_E4M3;
    if ((!w_router && n_experts > 1) || (w_router && !aligned16(w_router)) || !weights_ok(n_experts, e8, w_gate, s_gate) ||
        !weights_ok(n_experts, e8, w_up, s_up) || !weights_ok(n_experts, e8, w_down, s_down))
        return TS_ERR_INVALID_ARG;
    if (prepare_grouped() != cudaSuccess) return TS_ERR_CUDA;
    ts_experts* h = nullptr;
    ts_status s = TS_ERR_OOM;
    try {
        h = new ts_experts;
        h->d = d;
        h->m = m;
        h->n_experts = n_experts;
        h->top_k = top_k;
        h->dt = wdtype;
        h->routed = w_router != nullptr;
        cudaGetDevice(&h->device);
        auto set = [](Products& p, int groups, int n, int k, ts_dtype dt, bool gated, bool kn) {
            p.n_groups = groups;
            p.n = n;
            p.k = k;
            p.dt = dt;
            p.gated = gated;
            p.kn = kn;
        };
        set(h->gate_up, n_experts, m, d, wdtype, true, false);
        set(h->down, n_experts, d, m, wdtype, false, !e8);
        set(h->router, 1, n_experts, d, TS_BF16, false, false);
        std::vector<GroupWeights> table(2 * (size_t)n_experts + 1);
        GroupWeights *gu = table.data(), *dn = gu + n_experts, *rt = dn + n_experts;
        const size_t bytes = sizeof(GroupWeights) * table.size(), o_w = h->arena.take(bytes);
        if (!map_weights(h->gate_up, gu, w_gate, w_up, s_gate, s_up) ||
            !map_weights(h->down, dn, w_down, nullptr, s_down, nullptr) ||
            (w_router && !map_weights(h->router, rt, &w_router, nullptr, nullptr, nullptr)))
            s = TS_ERR_CUDA;
        else
            s = alloc_arena(&h->arena);
        if (s == TS_OK) {
            h->gate_up.weights = h->arena.at<GroupWeights>(o_w);
            h->down.weights = h->gate_up.weights + n_experts;
            h->router.weights = h->down.weights + n_experts;
            s = copy_in(h->gate_up.weights, table.data(), bytes);
        }
    } catch (const std::bad_alloc&) {
        s = TS_ERR_OOM;
    }
    if (s != TS_OK) {
        ts_experts_destroy(h);
        return s;
    }
    *out = h;
    return TS_OK;
}

void ts_experts_destroy(ts_experts* h) {
    if (!h) return;
    free_arena(&h->arena);
    delete h;
}

ts_status ts_prompt_create(ts_prompt** out, int d, int m, int n_experts, int top_k, ts_dtype wdtype, int max_tokens) {
    if (!out || max_tokens < 1) return TS_ERR_INVALID_ARG;
    const ts_status sizes = check_experts(d, m, n_experts, top_k, wdtype);
    if (sizes != TS_OK) return sizes;
    if ((long long)max_tokens * top_k >= 1ll << 30) return TS_ERR_INVALID_ARG;
    if (prepare_grouped() != cudaSuccess) return TS_ERR_CUDA;
    const bool e8 = wdtype == TS_E4M3;
    ts_prompt* p = nullptr;
    ts_status s = TS_ERR_OOM;
    try {
        p = new ts_prompt;
        p->d = d;
        p->m = m;
        p->n_experts = n_experts;
        p->top_k = top_k;
        p->dt = wdtype;
        p->max_tokens = max_tokens;
        Arena& ar = p->arena;
        const size_t tokens = (size_t)max_tokens, rows = tokens * (size_t)top_k, db = ((size_t)d + 127) / 128,
                     mb = ((size_t)m + 127) / 128;
        const size_t o_logits = ar.take(tokens * (size_t)n_experts * 4), o_sel = ar.take(rows * 4), o_w = ar.take(rows * 4),
                     o_slots = ar.take(rows * 4), o_rows = ar.take(rows * 4), o_off = ar.take(((size_t)n_experts + 1) * 4), o_shape = ar.take(8),
                     o_x = ar.take(rows * (size_t)d * (e8 ? 1 : 2)), o_c = ar.take(rows * (size_t)m * 2),
                     o_y = ar.take(rows * (size_t)d * 4), o_xs = ar.take(e8 ? db * rows * 4 : 0),
                     o_cq = ar.take(e8 ? rows * (size_t)m : 0), o_cs = ar.take(e8 ? mb * rows * 4 : 0);
        s = p->s.plan(&ar, (int)rows) ? alloc_arena(&ar) : TS_ERR_CUDA;
        if (s == TS_OK && cudaStreamSynchronize(cudaStreamLegacy) != cudaSuccess) s = TS_ERR_CUDA;
        if (s == TS_OK) {
            p->s.place(ar);
            p->logits = ar.at<float>(o_logits);
            p->sel = ar.at<int32_t>(o_sel);
            p->w = ar.at<float>(o_w);
            p->slots = ar.at<int32_t>(o_slots);
            p->rows = ar.at<int32_t>(o_rows);
            p->offsets = ar.at<int32_t>(o_off);
            p->shape = ar.at<int32_t>(o_shape);
            p->x = ar.at<char>(o_x);
            p->c = ar.at<__nv_bfloat16>(o_c);
            p->y = ar.at<float>(o_y);
            p->x_scale = ar.at<float>(o_xs);
            p->cq = ar.at<char>(o_cq);
            p->c_scale = ar.at<float>(o_cs);
        }
    } catch (const std::bad_alloc&) {
        s = TS_ERR_OOM;
    }
    if (s != TS_OK) {
        ts_prompt_destroy(p);
        return s;
    }
    *out = p;
    return TS_OK;
}

void ts_prompt_destroy(ts_prompt* p) {
    if (!p) return;
    free_arena(&p->arena);
    delete p;
}

ts_status ts_prompt_forward(ts_prompt* p, ts_experts* e, const void* x, int tokens, float* y, cudaStream_t stream) {
    if (!p || !e || e->d != p->d || e->m != p->m || e->dt != p->dt || e->n_experts > p->n_experts || e->top_k > p->top_k ||
        tokens < 0 || tokens > p->max_tokens)
        return TS_ERR_INVALID_ARG;
    if (tokens == 0) {
        p->last_tokens = 0;
        p->last_k = e->routed ? e->top_k : 0;
        return TS_OK;
    }
    if (!here(p->s.device) || e->device != p->s.device || !x || !y || !aligned16(x)) return TS_ERR_INVALID_ARG;
    const int d = p->d, m = p->m, rows = e->routed ? tokens * e->top_k : tokens;
    const bool e8 = p->dt == TS_E4M3;
    const int32_t *offsets = nullptr, *count = nullptr, *list = nullptr;
    ts_status s = TS_OK;
    p->last_k = 0;
    if (e->routed) {
        s = run_products(e->router, p->s, x, d, nullptr, 0, nullptr, tokens, p->logits, e->n_experts, true, stream);
        if (s == TS_OK)
            s = launched(launch_route(
                {p->logits, tokens, e->n_experts, e->top_k, p->sel, p->w, p->offsets, p->rows, p->slots, p->shape}, stream));
        if (s != TS_OK) return s;
        offsets = p->offsets;
        count = p->offsets + e->n_experts;
        list = p->rows;
    }
    // the rows in the experts' order (a single expert takes bf16 rows as they are)
    const void* xr = x;
    if (e8) {
        s = launched(launch_quant_rows({x, d, tokens, d, list, count, rows, p->x, p->x_scale}, false, stream));
        xr = p->x;
    } else if (e->routed) {
        s = launched(launch_gather_rows({x, d, tokens, d, list, count, rows, p->x, nullptr}, 2, stream));
        xr = p->x;
    }
    if (s == TS_OK)
        s = run_products(e->gate_up, p->s, xr, d, e8 ? p->x_scale : nullptr, rows, offsets, rows, p->c, m, false, stream);
    const void* c = p->c;
    if (s == TS_OK && e8) {
        s = launched(launch_quant_rows({p->c, m, rows, m, nullptr, count, rows, p->cq, p->c_scale}, false, stream));
        c = p->cq;
    }
    if (s == TS_OK)
        s = run_products(e->down, p->s, c, m, e8 ? p->c_scale : nullptr, rows, offsets, rows, e->routed ? p->y : y, d, true,
                         stream);
    if (s == TS_OK && e->routed) {
        s = launched(launch_combine({p->y, rows, d, p->slots, p->w, tokens, e->top_k, y}, true, stream));
        if (s == TS_OK) {
            p->last_tokens = tokens;
            p->last_k = e->top_k;
        }
    }
    return s;
}

ts_status ts_prompt_get_routing(ts_prompt* p, cudaStream_t stream, int32_t* sel, float* w) {
    if (!p || p->last_k == 0 || !sel || !w) return TS_ERR_INVALID_ARG;
    const size_t bytes = (size_t)p->last_tokens * (size_t)p->last_k * 4;
    if (bytes == 0) return cudaStreamSynchronize(stream) == cudaSuccess ? TS_OK : TS_ERR_CUDA;
    int32_t shape[2] = {0, 0};
    if (cudaMemcpyAsync(shape, p->shape, sizeof shape, cudaMemcpyDeviceToHost, stream) != cudaSuccess ||
        cudaStreamSynchronize(stream) != cudaSuccess)
        return TS_ERR_CUDA;
    if (shape[0] != p->last_tokens || shape[1] != p->last_k) return TS_ERR_INVALID_ARG;
    if (cudaMemcpyAsync(sel, p->sel, bytes, cudaMemcpyDeviceToHost, stream) != cudaSuccess ||
        cudaMemcpyAsync(w, p->w, bytes, cudaMemcpyDeviceToHost, stream) != cudaSuccess ||
        cudaStreamSynchronize(stream) != cudaSuccess)
        return TS_ERR_CUDA;
    return TS_OK;
}

ts_status ts_prompt_get_error(ts_prompt* p, cudaStream_t stream) {
    return p ? read_status(p->s, stream) : TS_ERR_INVALID_ARG;
}

ts_status ts_prompt_check_scratch(ts_prompt* p, cudaStream_t stream) {
    return p ? check_arena(p->arena, stream) : TS_ERR_INVALID_ARG;
}

}  // extern "C"
