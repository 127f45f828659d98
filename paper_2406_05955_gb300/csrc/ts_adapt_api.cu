// ts_adapt_api.cu -- the C ABI of what an adapted layer needs beside its frozen weights (include/ts_ffn.h): argument checks
// and launches. None of these operators keeps anything between calls.
#include <stdint.h>

#include <atomic>

#include "ts_adapt.h"
#include "ts_ffn.h"
#include "ts_grouped.h"
#include "ts_kernels.cuh"

using namespace tsffn;

namespace {

bool aligned16(const void* p) { return ((uintptr_t)p & 15u) == 0; }
bool aligned4(const void* p) { return ((uintptr_t)p & 3u) == 0; }
std::atomic<int> test_stall{0};  // ts_adapt_set_test_stall

// The device's counts of waits that gave up only grow, and what callers have been told of them is kept here: nothing that one
// stream's kernel counts while another stream asks can be erased.
constexpr int kDevices = 64;
std::atomic<unsigned> told[kDevices][2];
bool moved_on(std::atomic<unsigned>& to, unsigned now) {
    unsigned had = to.load();
    while ((int)(now - had) > 0)  // (another caller may have been told of later ones)
        if (to.compare_exchange_weak(had, now)) return true;
    return false;
}
ts_status launched(cudaError_t e) { return e == cudaSuccess ? TS_OK : TS_ERR_CUDA; }
int elem_size(ts_dtype dt) { return dt == TS_F32 ? 4 : dt == TS_BF16 ? 2 : 1; }

// Rows of `cols` elements, `ld` apart, each on a 16-byte boundary.
bool rows_ok(const void* p, int64_t ld, int cols, ts_dtype dt) {
    return p != nullptr && aligned16(p) && ld >= cols && ld * elem_size(dt) % 16 == 0;
}

// Memory that a call reads or writes: rows of `bytes` bytes, `pitch` apart.
struct Region {
    const void* p;
    int64_t pitch;
    int rows;
    int64_t bytes;
};
Region rows_of(const void* p, int64_t ld, int rows, int cols, ts_dtype dt) {
    return {p, ld * elem_size(dt), rows, (int64_t)cols * elem_size(dt)};
}
Region whole(const void* p, int64_t bytes) { return {p, bytes, 1, bytes}; }

// Whether they share a byte. Rows that lie between those of the other, as columns of one buffer do, share none; that is looked
// for where the pitch is the same.
bool overlap(const Region& a, const Region& b) {
    if (a.p == nullptr || b.p == nullptr || a.rows <= 0 || b.rows <= 0 || a.bytes <= 0 || b.bytes <= 0) return false;
    const int64_t d = (int64_t)((uintptr_t)b.p - (uintptr_t)a.p);
    if (d >= (a.rows - 1) * a.pitch + a.bytes || -d >= (b.rows - 1) * b.pitch + b.bytes) return false;
    if (a.pitch != b.pitch || (a.rows == 1 && b.rows == 1)) return true;
    // row i + q of b begins d + q pitch behind row i of a: the two q that bring it nearest, from above and from below
    const int64_t rest = (d % a.pitch + a.pitch) % a.pitch, q = (rest - d) / a.pitch;
    const auto there = [&](int64_t i) { return i > -a.rows && i < b.rows; };
    return (rest < a.bytes && there(q)) || (a.pitch - rest < b.bytes && there(q - 1));
}

bool same_rows(const Region& a, const Region& b) { return a.p == b.p && (a.pitch == b.pitch || a.rows == 1) && a.bytes == b.bytes; }

// Whether any of `outs` shares memory with another of them or with any of `ins`.
template <size_t N, size_t M>
bool overlap(const Region (&outs)[N], const Region (&ins)[M]) {
    for (size_t i = 0; i < N; ++i) {
        for (const Region& in : ins)
            if (overlap(outs[i], in)) return true;
        for (size_t j = 0; j < i; ++j)
            if (overlap(outs[i], outs[j])) return true;
    }
    return false;
}

// The counts that ts_adapt_rows and ts_adapter_grads share.
ts_status check_adapters(int rows, int k, int n_adapters, int r) {
    if (rows < 0 || k < 1 || n_adapters < 1 || n_adapters > kMaxAdapters || r < 1 || r > kMaxRank) return TS_ERR_INVALID_ARG;
    return rows > kMaxRows || k > kMaxRowElems ? TS_ERR_UNSUPPORTED : TS_OK;
}

ts_status check_routing(int tokens, int n_experts, int top_k) {
    return tokens < 0 || n_experts < 1 || n_experts > kMaxRouteExperts || top_k < 1 || top_k > kMaxRouteK ||
                   top_k > n_experts || (long long)tokens * top_k >= 1ll << 30
               ? TS_ERR_INVALID_ARG
               : TS_OK;
}

// Sizes of the gated activation: rows of e4m3 numbers start on 16-byte boundaries.
ts_status check_drelu(ts_dtype dtype, int rows, int m) {
    if ((dtype != TS_F32 && dtype != TS_BF16) || rows < 0 || m < 1 || m % 16 != 0) return TS_ERR_INVALID_ARG;
    return rows > kMaxRows || m > kMaxRowElems ? TS_ERR_UNSUPPORTED : TS_OK;
}

}  // namespace

extern "C" {

ts_status ts_list_rows(const int32_t* ids, int n_rows, int n_groups, int32_t* rows, int32_t* offsets, cudaStream_t stream) {
    if (n_rows < 0 || n_rows >= 1 << 30 || n_groups < 1 || n_groups > kMaxAdapters || !aligned4(ids) || !aligned4(rows) ||
        !offsets || !aligned4(offsets) || (n_rows > 0 && (!ids || !rows)))
        return TS_ERR_INVALID_ARG;
    // ids are read again while rows and offsets are written
    const Region rid = whole(ids, 4ll * n_rows), rr = whole(rows, 4ll * n_rows), ro = whole(offsets, 4ll * (n_groups + 2));
    if (overlap(rr, rid) || overlap(ro, rid) || overlap(rr, ro)) return TS_ERR_INVALID_ARG;
    return launched(launch_list_rows(ids, n_rows, n_groups, rows, offsets, stream));
}

ts_status ts_adapt_rows(const void* x, int64_t ldx, int rows, int k, const void* a, const void* b, const float* scale,
                        const int32_t* ranks, int n_adapters, int r, int n, const int32_t* ids, const int32_t* list,
                        const int32_t* offsets, const void* y, int64_t ldy, ts_dtype ydtype, void* out, int64_t ldo, float* h,
                        cudaStream_t stream) {
    ts_status s = check_adapters(rows, k, n_adapters, r);
    if (s == TS_OK) s = check_adapters(rows, n, n_adapters, r);
    if (s != TS_OK) return s;
    if ((ydtype != TS_F32 && ydtype != TS_BF16) || k % 8 != 0 || n % 8 != 0) return TS_ERR_INVALID_ARG;
    if (rows == 0) return TS_OK;
    if (!rows_ok(x, ldx, k, TS_BF16) || !a || !aligned16(a) || !b || !aligned16(b) || !aligned4(scale) || !aligned4(ranks) ||
        !aligned4(h))
        return TS_ERR_INVALID_ARG;
    if (list ? !offsets || !aligned4(list) || !aligned4(offsets) : !ids || !aligned4(ids) || rows > kFewRows)
        return TS_ERR_INVALID_ARG;
    if (!out ? y != nullptr || !h : !rows_ok(y, ldy, n, ydtype) || !rows_ok(out, ldo, n, ydtype) || (out == y && ldo != ldy))
        return TS_ERR_INVALID_ARG;
    // Other CTAs read x while one writes out, and y in other places than it writes: out is y itself, or apart from both.
    const Region rx = rows_of(x, ldx, rows, k, TS_BF16), ry = rows_of(y, ldy, rows, n, ydtype), ro = rows_of(out, ldo, rows, n, ydtype),
                 rh = rows_of(h, r, rows, r, TS_F32);
    if (overlap(ro, rx) || (out != y && overlap(ro, ry)) || overlap(rh, rx) || overlap(rh, ry) || overlap(rh, ro))
        return TS_ERR_INVALID_ARG;
    return launched(launch_adapt({x, ldx, rows, k, a, b, scale, ranks, n_adapters, r, n, list ? nullptr : ids, list,
                                  list ? offsets : nullptr, y, ldy, out, ldo, h, test_stall.load()},
                                 ydtype == TS_F32, stream));
}

ts_status ts_adapt_get_error(cudaStream_t stream) {
    int dev = 0;
    unsigned n[2] = {0, 0};
    if (cudaGetDevice(&dev) != cudaSuccess || dev < 0 || dev >= kDevices || adapt_wide_timeouts(&n[0], stream) != cudaSuccess ||
        adapter_grads_timeouts(&n[1], stream) != cudaSuccess || cudaStreamSynchronize(stream) != cudaSuccess)
        return TS_ERR_CUDA;
    const bool rows = moved_on(told[dev][0], n[0]), grads = moved_on(told[dev][1], n[1]);
    return rows || grads ? TS_ERR_TIMEOUT : TS_OK;
}

void ts_adapt_set_test_stall(int on) { test_stall = on != 0; }

ts_status ts_adapter_grads(const float* h, int r, const void* x, int64_t ldx, ts_dtype xdtype, const float* x_scale,
                           int64_t ld_scale, int rows, int k, int n_adapters, const int32_t* list, const int32_t* offsets,
                           float* grad, int accumulate, cudaStream_t stream) {
    const ts_status s = check_adapters(rows, k, n_adapters, r);
    if (s != TS_OK) return s;
    const bool e8 = xdtype == TS_E4M3;
    if ((!e8 && xdtype != TS_BF16) || k % (e8 ? 16 : 8) != 0 || !grad || !aligned16(grad) || !offsets || !aligned4(offsets))
        return TS_ERR_INVALID_ARG;
    if (rows > 0 && (!h || !aligned4(h) || !rows_ok(x, ldx, k, xdtype) || !list || !aligned4(list) ||
                     (e8 ? !x_scale || !aligned4(x_scale) || ld_scale < rows : x_scale != nullptr)))
        return TS_ERR_INVALID_ARG;
    const Region to = whole(grad, 4ll * n_adapters * r * k);
    if (overlap(to, rows_of(h, r, rows, r, TS_F32)) || overlap(to, rows_of(x, ldx, rows, k, xdtype)) ||
        overlap(to, rows_of(x_scale, ld_scale, (k + kScaleBlock - 1) / kScaleBlock, rows, TS_F32)))
        return TS_ERR_INVALID_ARG;
    return launched(launch_adapter_grads(
        {h, r, x, ldx, x_scale, ld_scale, rows, k, n_adapters, list, offsets, grad, accumulate != 0, 0, test_stall.load()}, e8,
        stream));
}

ts_status ts_adapters_backward(const void* dy, int64_t ldy, int rows, int n, const void* a, const void* b, const float* scale,
                               const int32_t* ranks, int n_adapters, int r, int k, const int32_t* list, const int32_t* offsets,
                               const float* h, const void* x, int64_t ldx, ts_dtype xdtype, const float* x_scale,
                               int64_t ld_scale, const void* dx, int64_t lddx, ts_dtype dxdtype, void* out, int64_t ldo, float* dh,
                               float* da, float* db, int accumulate, cudaStream_t stream) {
    if (!offsets || !aligned4(offsets) || (rows > 0 && (!list || !dh))) return TS_ERR_INVALID_ARG;
    // all of it is checked before any of it is launched
    const bool e8 = xdtype == TS_E4M3;
    ts_status s = check_adapters(rows, k, n_adapters, r);
    if (s == TS_OK) s = check_adapters(rows, n, n_adapters, r);
    if (s != TS_OK) return s;
    if ((!e8 && xdtype != TS_BF16) || k % (e8 ? 16 : 8) != 0 || n % 8 != 0 || !da || !aligned16(da) || !db || !aligned16(db))
        return TS_ERR_INVALID_ARG;
    if (rows > 0 && (!h || !aligned4(h) || !rows_ok(x, ldx, k, xdtype) ||
                     (e8 ? !x_scale || !aligned4(x_scale) || ld_scale < rows : x_scale != nullptr)))
        return TS_ERR_INVALID_ARG;
    // dy, x and h are read after out and dh were written, and beside da and db (dx before these)
    if (rows > 0) {
        const Region outs[4] = {rows_of(out, ldo, rows, k, dxdtype), rows_of(dh, r, rows, r, TS_F32),
                                whole(da, 4ll * n_adapters * r * k), whole(db, 4ll * n_adapters * r * n)};
        const Region ins[4] = {rows_of(dy, ldy, rows, n, TS_BF16), rows_of(h, r, rows, r, TS_F32), rows_of(x, ldx, rows, k, xdtype),
                               rows_of(x_scale, ld_scale, (k + kScaleBlock - 1) / kScaleBlock, rows, TS_F32)};
        if (overlap(outs, ins)) return TS_ERR_INVALID_ARG;
    }
    s = ts_adapt_rows(dy, ldy, rows, n, b, a, scale, ranks, n_adapters, r, k, nullptr, list, offsets, dx, lddx, dxdtype, out, ldo,
                      dh, stream);
    if (s != TS_OK) return s;
    const int add = accumulate != 0, stall = test_stall.load();
    const cudaError_t e = launch_adapter_grads(
        {dh, r, x, ldx, x_scale, ld_scale, rows, k, n_adapters, list, offsets, da, add, 0, stall}, e8, stream);
    if (e != cudaSuccess) return TS_ERR_CUDA;
    return launched(launch_adapter_grads(
        {h, r, dy, ldy, nullptr, 0, rows, n, n_adapters, list, offsets, db, add, 1, stall}, false, stream));
}

ts_status ts_drelu_rows(const void* g, int64_t ldg, const void* u, int64_t ldu, ts_dtype dtype, const int32_t* n, int rows,
                        int m, void* c, int64_t ldc, void* q_gate, void* q_up, float* s_gate, float* s_up,
                        cudaStream_t stream) {
    const ts_status s = check_drelu(dtype, rows, m);
    if (s != TS_OK || rows == 0) return s;
    if (!rows_ok(g, ldg, m, dtype) || !rows_ok(u, ldu, m, dtype) || !rows_ok(c, ldc, m, TS_BF16) || !aligned4(n))
        return TS_ERR_INVALID_ARG;
    const bool kept = q_gate != nullptr;
    if (kept != (q_up != nullptr) || kept != (s_gate != nullptr) || kept != (s_up != nullptr) || !aligned16(q_gate) ||
        !aligned16(q_up) || !aligned4(s_gate) || !aligned4(s_up))
        return TS_ERR_INVALID_ARG;
    // c may lie over a bf16 g or u, element for element: a thread reads what it then writes
    const Region rg = rows_of(g, ldg, rows, m, dtype), ru = rows_of(u, ldu, rows, m, dtype), rc = rows_of(c, ldc, rows, m, TS_BF16);
    const int blocks = (m + kScaleBlock - 1) / kScaleBlock;
    const Region kept_to[4] = {whole(q_gate, (int64_t)rows * m), whole(q_up, (int64_t)rows * m), whole(s_gate, 4ll * rows * blocks),
                               whole(s_up, 4ll * rows * blocks)},
                 others[3] = {rg, ru, rc};
    if ((!same_rows(rc, rg) && overlap(rc, rg)) || (!same_rows(rc, ru) && overlap(rc, ru)) || overlap(kept_to, others))
        return TS_ERR_INVALID_ARG;
    return launched(launch_drelu({g, u, ldg, ldu, n, rows, m, c, ldc, static_cast<uint8_t*>(q_gate),
                                  static_cast<uint8_t*>(q_up), s_gate, s_up},
                                 dtype == TS_F32, stream));
}

ts_status ts_drelu_rows_backward(const void* dc, int64_t ldd, ts_dtype dtype, const void* q_gate, const void* q_up,
                                 const float* s_gate, const float* s_up, const int32_t* n, int rows, int m, void* dg,
                                 int64_t ldg, void* du, int64_t ldu, void* c, int64_t ldc, cudaStream_t stream) {
    const ts_status s = check_drelu(dtype, rows, m);
    if (s != TS_OK || rows == 0) return s;
    if (!rows_ok(dc, ldd, m, dtype) || !rows_ok(dg, ldg, m, TS_BF16) || !rows_ok(du, ldu, m, TS_BF16) || !aligned4(n) ||
        (c && !rows_ok(c, ldc, m, TS_BF16)) || !q_gate || !aligned16(q_gate) || !q_up || !aligned16(q_up) || !s_gate ||
        !aligned4(s_gate) || !s_up || !aligned4(s_up))
        return TS_ERR_INVALID_ARG;
    // dg, du or c may lie over a bf16 dc, element for element
    const int blocks = (m + kScaleBlock - 1) / kScaleBlock;
    const Region rd = rows_of(dc, ldd, rows, m, dtype);
    const Region outs[3] = {rows_of(dg, ldg, rows, m, TS_BF16), rows_of(du, ldu, rows, m, TS_BF16), rows_of(c, ldc, rows, m, TS_BF16)},
                 ins[4] = {whole(q_gate, (int64_t)rows * m), whole(q_up, (int64_t)rows * m), whole(s_gate, 4ll * rows * blocks),
                           whole(s_up, 4ll * rows * blocks)};
    if (overlap(outs, ins)) return TS_ERR_INVALID_ARG;
    for (const Region& out : outs)
        if (!same_rows(out, rd) && overlap(out, rd)) return TS_ERR_INVALID_ARG;
    return launched(launch_drelu_backward({dc, ldd, static_cast<const uint8_t*>(q_gate), static_cast<const uint8_t*>(q_up),
                                           s_gate, s_up, n, rows, m, dg, du, c, ldg, ldu, ldc},
                                          dtype == TS_F32, stream));
}

long long ts_balance_work(int tokens, int n_experts) {
    return check_routing(tokens, n_experts, 1) == TS_OK ? (long long)balance_work(tokens, n_experts) : -1;
}

ts_status ts_balance(const float* logits, int tokens, int n_experts, const int32_t* sel, int top_k, float* loss,
                     int32_t* counts, float* share, int32_t* totals, float* work, cudaStream_t stream) {
    const ts_status s = check_routing(tokens, n_experts, top_k);
    if (s != TS_OK) return s;
    if (!loss || !aligned4(loss) || !counts || !aligned4(counts) || !share || !aligned4(share) || !totals ||
        !aligned4(totals) || (!work && balance_work(tokens, n_experts) > 0) || !aligned4(work) || !aligned4(logits) ||
        !aligned4(sel) || (tokens > 0 && (!logits || !sel)))
        return TS_ERR_INVALID_ARG;
    const Region outs[5] = {whole(loss, 4), whole(counts, 4ll * n_experts), whole(share, 4ll * n_experts), whole(totals, 8),
                            whole(work, 4ll * (int64_t)balance_work(tokens, n_experts))},
                 ins[2] = {whole(logits, 4ll * tokens * n_experts), whole(sel, 4ll * tokens * top_k)};
    if (overlap(outs, ins)) return TS_ERR_INVALID_ARG;
    return launched(launch_balance({logits, tokens, n_experts, top_k, sel, loss, counts, share, totals, work}, stream));
}

ts_status ts_route_backward(const float* logits, int tokens, int n_experts, const int32_t* sel, const float* w, int top_k,
                            const float* dw, const int32_t* counts, const int32_t* totals, const float* dloss, float* dlogits,
                            cudaStream_t stream) {
    const ts_status s = check_routing(tokens, n_experts, top_k);
    if (s != TS_OK) return s;
    const bool balance = counts != nullptr;
    if (balance != (totals != nullptr) || balance != (dloss != nullptr) || !aligned4(counts) || !aligned4(totals) ||
        !aligned4(dloss))
        return TS_ERR_INVALID_ARG;
    if (tokens == 0) return TS_OK;
    if ((!balance && !dw) || (balance && !logits) || !aligned4(logits) || !dlogits || !aligned4(dlogits) || !aligned4(dw) ||
        !aligned4(sel) || !aligned4(w) || (dw && (!sel || !w)))
        return TS_ERR_INVALID_ARG;
    // dlogits may be logits: a token's lanes read theirs before they write
    const int64_t all = 4ll * tokens * n_experts, picks = 4ll * tokens * top_k;
    const Region outs[1] = {whole(dlogits, all)};
    const Region ins[7] = {whole(dlogits != logits ? logits : nullptr, all), whole(dw ? sel : nullptr, picks), whole(dw ? w : nullptr, picks),
                           whole(dw, picks), whole(counts, 4ll * n_experts), whole(totals, 8), whole(dloss, 4)};
    if (overlap(outs, ins)) return TS_ERR_INVALID_ARG;
    return launched(launch_route_backward({logits, tokens, n_experts, top_k, sel, w, dw, counts, totals, dloss, dlogits}, stream));
}

ts_status ts_combine_rows_backward(const void* dy, ts_dtype dydtype, const void* src, ts_dtype dtype, int n_rows, int n,
                                   const int32_t* slots, const float* w, const int32_t* rows, int tokens, int top_k,
                                   void* dsrc, float* dw, cudaStream_t stream) {
    if ((dtype != TS_F32 && dtype != TS_BF16) || (dydtype != TS_F32 && dydtype != TS_BF16) || n_rows < 0 || n < 1 ||
        tokens < 0 || top_k < 1 || top_k > kMaxRouteK)
        return TS_ERR_INVALID_ARG;
    if (n > kMaxRows || tokens > kMaxRows) return TS_ERR_UNSUPPORTED;
    if (tokens == 0) return TS_OK;
    const unsigned size = (unsigned)elem_size(dtype);
    if (!dy || (uintptr_t)dy % (unsigned)elem_size(dydtype) != 0 || (uintptr_t)src % size != 0 || (uintptr_t)dsrc % size != 0 ||
        (n_rows > 0 && (!src || !rows || !dsrc)) || !aligned4(rows) || !slots || !aligned4(slots) || !w ||
        !aligned4(w) || !dw || !aligned4(dw))
        return TS_ERR_INVALID_ARG;
    // a token's CTA writes rows of dsrc while others read dy and rows of src
    const Region to = rows_of(dsrc, n, n_rows, n, dtype);
    if (overlap(to, rows_of(src, n, n_rows, n, dtype)) || overlap(to, rows_of(dy, n, tokens, n, dydtype))) return TS_ERR_INVALID_ARG;
    return launched(launch_combine_backward({dy, src, n_rows, n, slots, w, rows, tokens, top_k, dsrc, dw}, dydtype == TS_F32,
                                            dtype == TS_F32, stream));
}

}  // extern "C"
