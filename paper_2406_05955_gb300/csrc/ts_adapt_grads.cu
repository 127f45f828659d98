// ts_adapt_grads.cu -- gradients of low-rank adapters: grad[i] = sum over the rows t of adapter i of h[t]^T x[t]
// (ts_adapter_grads).
//
// A cluster of CTAs has 128 columns of x. The rows are taken in chunks of up to 64 of one adapter, and its CTAs divide the
// chunks evenly, whichever adapters' they are: each stores the sums of adapters that lie in its part; those that reach into
// other parts are summed over distributed shared memory at the end, in the order of the CTAs. Adapters of up to 8 rows are
// no chunk's: warps sum them as they are.
//
// The rows are the products' k, gathered by the list. x is exact in bf16 (e4m3 rows too: the scale that 128 of their columns share
// is multiplied into h), h is split into three bf16 numbers of 8 bits each, so products and sums are as in fp32. The columns of
// x are the M of the tensor cores and the three parts of h, side by side, their N: one instruction for 16 rows (r up to
// 64), sums in tensor memory.
//
// Memory bounds it in principle: x once, h once for each 128 columns from L2. What it spends is latency: chunks in a row,
// each split, widened (e4m3) and multiplied between barriers by the 16 warps that an SM has room for; an SM issues 1.5
// instructions a cycle. 8192 rows, k = 4096, r = 32: 34 us from e4m3 rows (35 MB), 30 from bf16 ones (68 MB; r = 64 45, r = 128 71); 64 rows of one
// adapter, k = 512, r = 12: 4. Measured on the way: products by the warps' matrix instructions 98 and 40; rows divided
// instead of chunks, so that every CTA joins, 34 and 31 (64 rows of 8 adapters, k = 512, 10 us, now 5.7); two sets of parts,
// so that one is split while the other is multiplied by a warp of its own, no faster; 512 threads where two CTAs share an SM
// 10% slower (64 registers each), where one has it (r above 32) 10% faster; each of the later parts' sums tested for infinities, and not
// only the third's once a warp, 3% slower at r = 64 and 7 at 128. Adapters of up to 8 rows as chunks: a pass over 4
// rows of 28 adapters, k = 1520, n = 3504, r = 29, 43 us, now 25; 84 rows of 40, k = 13920, n = 2064, r = 4, 68 and 42 (48 if
// warps take up to 4 rows only).
#include <cuda_fp8.h>

#include <atomic>

#include "ts_adapt.cuh"
#include "ts_grouped.h"

namespace tsffn {
namespace {

__device__ unsigned grads_timeouts;  // waits that gave up, ever

constexpr int kGradCols = 128, kGradRows = 64;
constexpr int kFewest = 8, kShare = 8;  // rows of an adapter that warps sum by themselves, and components of a warp

// Four numbers as three bf16 numbers each, cut off (8, 8 and the last 8 bits: nothing is lost). An infinity or NaN is the
// first alone.
__device__ __forceinline__ void cut(const float4& v, uint2 (&p)[3]) {
    float f[4] = {v.x, v.y, v.z, v.w}, rest[4];
    uint32_t w[3][4];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        w[0][e] = __float_as_uint(f[e]);
        rest[e] = f[e] - __uint_as_float(w[0][e] & 0xffff0000u);
        w[1][e] = __float_as_uint(rest[e]);
        w[2][e] = __float_as_uint(rest[e] - __uint_as_float(w[1][e] & 0xffff0000u));
    }
    // (a remainder is NaN where the number is not finite, and else it is finite)
    if (const float odd = (rest[0] + rest[1]) + (rest[2] + rest[3]); odd != odd) {
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (!(fabsf(f[e]) < INFINITY)) {
                w[0][e] = f[e] != f[e] ? 0x7fff0000u : w[0][e];
                w[1][e] = w[2][e] = 0u;
            }
    }
#pragma unroll
    for (int q = 0; q < 3; ++q) p[q] = make_uint2(__byte_perm(w[q][0], w[q][1], 0x7632), __byte_perm(w[q][2], w[q][3], 0x7632));
}

// 16 e4m3 numbers in bf16 (exact).
__device__ __forceinline__ void widen(const uint4& v, uint4 (&to)[2]) {
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
    uint32_t b[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        const __half2_raw f = __nv_cvt_fp8x2_to_halfraw2((__nv_fp8x2_storage_t)(w[e / 2] >> 16 * (e & 1)), __NV_E4M3);
        const __nv_bfloat162 t = __float22bfloat162_rn(__half22float2(*reinterpret_cast<const __half2*>(&f)));
        b[e] = *reinterpret_cast<const uint32_t*>(&t);
    }
    to[0] = make_uint4(b[0], b[1], b[2], b[3]);
    to[1] = make_uint4(b[4], b[5], b[6], b[7]);
}

template <int RP, bool E8>
struct Grads {
    static constexpr int kXBytes = kGradRows * kGradCols * (E8 ? 1 : 2), kHBytes = kGradRows * RP * 4;
    static constexpr int kCtas = RP <= 32 ? 2 : 1;    // on an SM
    static constexpr int kThreads = 512 / kCtas;
    static constexpr int kSides = kThreads / kGradCols;  // threads that share a column's components
    static constexpr int kStages = RP <= 64 ? 3 : 2;
    static constexpr int kRing = kStages + 2;         // chunks whose rows are known
    // x starts on 1024 bytes in a stage; h, and for e4m3 rows their scales, lie in rings of their own
    static constexpr int kWideBytes = E8 ? kGradRows * kGradCols * 2 : 0;  // a chunk of x in bf16
    static constexpr int kBlock = kGradRows * 128;                         // 64 columns of a chunk
    static constexpr int kPart = (3 * RP + 63) / 64 * kBlock;              // h of a chunk, its parts side by side
    static constexpr int kScaleBytes = E8 ? kGradRows * 4 : 0;
    static constexpr int kSums = RP * kGradCols * 4;                       // of an adapter that began in another part
    static constexpr int kRows = kStages * kXBytes + kWideBytes + kPart + kStages * (kHBytes + kScaleBytes);
    static constexpr int kSmem = 1024 + kRows + kSums;
    static constexpr int kColumns = RP == 16 ? 64 : RP == 32 ? 128 : RP == 64 ? 256 : 512;  // of tensor memory
    static constexpr int kN = RP <= 64 ? 3 * RP : 3 * RP / 2;              // of an instruction
    static constexpr int kMine = RP / kSides;                              // components of a thread's column
    static_assert(kMine * kSides == RP && kMine % 8 == 0 && kThreads > kMaxAdapters, "");
    static_assert(kRows >= kSums && 3 * RP <= kColumns, "those of one that goes on in another part lie where rows were");
};

// Where chunks of up to 64 entries, each of one adapter of more than kFewest, lie in entries `at` .. end - 1 of the list, `id`
// being the adapter of `at`; `first` adapter's entries begin at offs[id].
struct Chunks {
    int id, at, end, n_adapters;
    // The next chunk's entries; none: 0.
    __device__ __forceinline__ int next(const int* offs, int& first, int& of) {
        if (at >= end) return 0;
        if (id + 1 < n_adapters && offs[id + 1] <= at) {
            do ++id;
            while (id + 1 < n_adapters && offs[id + 1] - offs[id] <= kFewest);
            at = max(at, offs[id]);
            if (at >= end) return 0;
        }
        first = at;
        of = id;
        const int n = min(min(kGradRows, offs[id + 1] - at), end - at);
        at += n;
        return n;
    }
};

template <int RP, bool E8>
__global__ void __launch_bounds__(Grads<RP, E8>::kThreads, Grads<RP, E8>::kCtas) k_adapter_grads(const __grid_constant__ AdapterGradsLaunch L, int ctas) {
    using G = Grads<RP, E8>;
    constexpr int kThreads = G::kThreads, kWarps = kThreads / kWarp;
    extern __shared__ unsigned char raw[];
    __shared__ int offs[kMaxAdapters + 1];
    __shared__ uint2 x_at[G::kRing][kGradRows], h_at[G::kRing][kGradRows];  // first byte of a chunk's rows (none: the highest bit)
    __shared__ int rows[E8 ? G::kRing : 1][kGradRows];
    __shared__ int ids[G::kRing];  // a chunk's adapter
    __shared__ int part_at[kMaxCluster + 1], part_id[kMaxCluster + 1];  // a CTA's first entry and its adapter
    __shared__ int sums[kWarps], split, few;  // an adapter is in several parts; there are adapters of few rows, or none
    __shared__ uint64_t done;
    __shared__ uint32_t tmem;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const uint32_t cta = cluster_rank();
    unsigned char* const smem = raw + (-smem_u32(raw) & 1023u);
    unsigned char* const wide = smem + G::kStages * G::kXBytes;
    unsigned char* const parts = wide + G::kWideBytes;
    unsigned char* const hs = parts + G::kPart;
    unsigned char* const scales = hs + G::kStages * G::kHBytes;
    float* const begun = reinterpret_cast<float*>(smem + G::kRows);  // sums [RP][128] of the adapter that began in another part
    float* const goes_on = reinterpret_cast<float*>(smem);           // and of the one that goes on in another
    const uint32_t smem0 = smem_u32(smem), hs0 = smem_u32(hs), scales0 = smem_u32(scales);
    const int col0 = (int)(blockIdx.x / ctas) * kGradCols;
    const bool h_vec = L.r % 4 == 0 && (reinterpret_cast<uintptr_t>(L.h) & 15u) == 0;
    const int quarter = (warp & 3) * 32, side = warp >> 2;
    if (tid == 0) {
        mbar_init(&done, 1);
        mbar_fence_init();
        split = few = 0;
    }
    if (!L.follows) pdl_wait();
    pdl_launch_dependents();  // one that follows fills the SMs that this one leaves
    if (warp == 0) tc_alloc<G::kColumns>(&tmem);
    if (tid <= L.n_adapters) offs[tid] = min(max(L.offsets[tid], 0), L.rows);
    tc_before();
    __syncthreads();
    tc_after();
    const uint32_t d = tmem;
    int nc = 0;
    {
        const int count = tid < L.n_adapters ? offs[tid + 1] - offs[tid] : 0, n = count > kFewest ? (count + kGradRows - 1) / kGradRows : 0;
        if (tid < L.n_adapters && count <= kFewest && (count > 0 || !L.accumulate)) few = 1;
        int upto = n, total = 0;
#pragma unroll
        for (int o = 1; o < kWarp; o <<= 1) {
            const int v = __shfl_up_sync(0xffffffffu, upto, o);
            if (lane >= o) upto += v;
        }
        if (lane == kWarp - 1) sums[warp] = upto;
        __syncthreads();
#pragma unroll
        for (int w = 0; w < kWarps; ++w) {
            upto += w < warp ? sums[w] : 0;
            total += sums[w];
        }
        for (int c = 0; c <= ctas; ++c) {
            const int at = (int)((long long)total * c / ctas), nth = at - (upto - n);
            if (nth >= 0 && nth < n) {
                part_at[c] = offs[tid] + nth * kGradRows;
                part_id[c] = tid;
                if (nth > 0) split = 1;
            }
            if (at == total && tid == 0) {
                part_at[c] = offs[L.n_adapters];
                part_id[c] = L.n_adapters - 1;
            }
            nc = c == (int)cta ? -at : c == (int)cta + 1 ? nc + at : nc;
        }
    }
    __syncthreads();
    const int begin = part_at[cta], end = part_at[cta + 1], first_id = part_id[cta];
    bool failed = false;

    // The 16-byte pieces that a thread copies: the same one of every few rows of x, and of h those that it then splits.
    constexpr int kPieces = kGradCols * (E8 ? 1 : 2) / 16, kXStep = kThreads / kPieces, kQuads = RP / 4, kHStep = kThreads / kQuads;
    // Which rows a warp has is so that what 8 lanes (16 bytes of x in bf16) or 16 (8 bytes of h's parts) write is in all banks.
    const int x_row = E8 ? tid >> 4 << 1 | (tid >> 2 & 1) : tid / kPieces;
    const int x_piece = E8 ? (tid >> 3 & 1) << 2 | (tid & 3) : tid % kPieces;
    constexpr int kTurn = RP == 16 ? 1 : RP == 32 ? 2 : 0;  // the three lowest bits of a row, turned to the left
    const int h_nth = tid / kQuads, h_row = (h_nth & ~7) | (h_nth << kTurn & 7) | (h_nth & 7) >> (3 - kTurn), h_quad = tid % kQuads;
    const bool x_in = col0 + x_piece * (E8 ? 16 : 8) < L.k, h_in = h_quad * 4 < L.r;
    const uint32_t x_to = E8 ? tid * 16 : (x_piece >> 3) * G::kBlock + place<128>(x_row, x_piece & 7);
    const char* const x_from = static_cast<const char*>(L.x) + (x_in ? (int64_t)col0 * (E8 ? 1 : 2) + x_piece * 16 : 0);
    const char* const h_from = reinterpret_cast<const char*>(L.h) + (h_in ? h_quad * 16 : 0);
    const float* const scale_from = E8 ? L.x_scale + (int64_t)(col0 / kScaleBlock) * L.ld_scale : nullptr;
    uint32_t part_to[3];
#pragma unroll
    for (int t = 0; t < 3; ++t) {
        const int c = t * RP + h_quad * 4;
        part_to[t] = (c >> 6) * G::kBlock + place<128>(h_row, (c & 63) >> 3) + (c & 7) * 2;
    }
    static_assert(kXStep % 8 == 0 && kHStep % 8 == 0, "a thread's rows are permuted alike");

    // Copies 16 bytes (or N) of the row at `at`, zeros where there is none.
    const auto from = [](const char* base, const uint2& at) { return base + ((uint64_t)(at.y & 0x7fffffffu) << 32 | at.x); };
    const auto issue = [&](int i, int stage, int ring) {  // chunk i, its places in the rings of rows and of what is known of them
        if (i < nc) {
            const uint32_t to = smem0 + stage * G::kXBytes + x_to;
#pragma unroll
            for (int p = 0; p < kGradRows / kXStep; ++p) {
                const uint2 at = x_at[ring][x_row + p * kXStep];
                copy16(to + p * (E8 ? kThreads * 16 : kXStep * 128), from(x_from, at), x_in && (int)at.y >= 0);
            }
            const uint32_t h = hs0 + stage * G::kHBytes + tid * 16;
            if (h_vec) {
#pragma unroll
                for (int p = 0; p < kGradRows / kHStep; ++p) {
                    const uint2 at = h_at[ring][h_row + p * kHStep];
                    copy16(h + p * kThreads * 16, from(h_from, at), h_in && (int)at.y >= 0);
                }
            } else {
#pragma unroll 1
                for (int p = 0; p < kGradRows / kHStep; ++p)
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const uint2 at = h_at[ring][h_row + p * kHStep];
                        const bool in = (int)at.y >= 0 && h_quad * 4 + e < L.r;
                        copy4(h + p * kThreads * 16 + e * 4, in ? from(h_from, at) + e * 4 : reinterpret_cast<const char*>(L.h), in);
                    }
            }
            if (E8 && tid < kGradRows) {
                const int row = rows[ring][tid];
                copy4(scales0 + stage * G::kScaleBytes + tid * 4, scale_from + max(row, 0), row >= 0);
            }
        }
        copies_commit();
    };
    // The first two warps look up the rows of chunks, two turns before their copies are issued.
    const bool looks = tid < kGradRows;
    Chunks ahead{first_id, begin, end, L.n_adapters};
    const auto look_up = [&](int& of) {
        if (!looks) return -1;
        int first = 0;
        const int n = ahead.next(offs, first, of);
        return tid < n ? L.list[first + tid] : -1;  // (what a turn loads the next one looks at)
    };
    const auto know = [&](int ring, int row, int of) {
        if (!looks) return;
        if ((unsigned)row >= (unsigned)L.rows) row = -1;
        const uint64_t x = row < 0 ? 1ull << 63 : (uint64_t)(row * L.ldx * (E8 ? 1 : 2)), h = row < 0 ? 1ull << 63 : (uint64_t)row * L.r * 4;
        x_at[ring][tid] = make_uint2((uint32_t)x, (uint32_t)(x >> 32));
        h_at[ring][tid] = make_uint2((uint32_t)h, (uint32_t)(h >> 32));
        if (E8) rows[ring][tid] = row;
        if (tid == 0) ids[ring] = of;
    };
    const auto after = [](int at, int n) { return at + 1 == n ? 0 : at + 1; };
    float sum[G::kMine] = {};
    // What the tensor cores have added up. An infinity in x makes NaN of a second or third part of h that is 0, where h is not: where
    // x is not finite (and so the third parts' sum), the first parts' sum counts alone, whose infinities and NaN are the product's.
    const auto take_over = [&] {
        float v[G::kMine];
        bool odd = false;
#pragma unroll
        for (int q = 2; q >= 0; --q) {
#pragma unroll
            for (int j = 0; j < G::kMine; j += 8) tc_ld8(d + ((uint32_t)quarter << 16) + q * RP + side * G::kMine + j, v + j);
            tc_ld_wait(v);
            if (q == 2) {
                float any[4] = {v[0], v[1], v[2], v[3]};
#pragma unroll
                for (int j = 4; j < G::kMine; ++j) any[j & 3] += v[j];
                odd = __any_sync(0xffffffffu, !(fabsf((any[0] + any[1]) + (any[2] + any[3])) < INFINITY));
            }
            if (q > 0 && odd)
#pragma unroll
                for (int j = 0; j < G::kMine; ++j) v[j] = fabsf(v[j]) < INFINITY ? v[j] : 0.0f;
#pragma unroll
            for (int j = 0; j < G::kMine; ++j) sum[j] += v[j];
        }
    };
    const int col = quarter + lane;
    const auto keep = [&](float* to) {
#pragma unroll
        for (int j = 0; j < G::kMine; ++j) to[(side * G::kMine + j) * kGradCols + col] = sum[j];
    };
    const auto finish = [&](int id) {
        if (offs[id] >= begin && offs[id + 1] <= end) {
            if (col0 + col < L.k) {
                float* const to = L.grad + ((size_t)id * L.r + side * G::kMine) * L.k + col0 + col;
#pragma unroll
                for (int j = 0; j < G::kMine; ++j)
                    if (side * G::kMine + j < L.r) to[(size_t)j * L.k] = L.accumulate ? to[(size_t)j * L.k] + sum[j] : sum[j];
            }
        } else {
            keep(offs[id] <= begin ? begun : goes_on);  // (the last one goes on: no rows come any more)
        }
#pragma unroll
        for (int j = 0; j < G::kMine; ++j) sum[j] = 0.0f;
    };

    if (nc > 0) {
        int ring[G::kStages], of[G::kStages], next_of = 0;
#pragma unroll
        for (int i = 0; i < G::kStages; ++i) ring[i] = look_up(of[i] = 0);
        int next = look_up(next_of);
#pragma unroll
        for (int i = 0; i < G::kStages; ++i) know(i, ring[i], of[i]);
        __syncthreads();
#pragma unroll
        for (int i = 0; i < G::kStages; ++i) issue(i, i, i);
        int stage = G::kStages - 1, last = 0, known = G::kStages, coming = G::kStages - 1, here = G::kRing - 1;
        int id = -1, nth = 0;  // the adapter of the last chunk, and how many of its chunks there were
        for (int i = 0; i < nc; ++i) {
            last = stage;
            stage = after(stage, G::kStages);
            here = after(here, G::kRing);
            const int now = ids[here];
            if (i == 0) copies_wait<G::kStages - 1>();
            else copies_wait<G::kStages - 2>();
            if (E8) __syncthreads();  // (the scales)
            know(known, next, next_of);
            known = after(known, G::kRing);
            next = look_up(next_of);
            if (i > 0) {  // the last chunk's products are done: what they read may be overwritten
                if (!failed) failed = !mbar_wait(&done, (i - 1) & 1);
                coming = after(coming, G::kRing);
                issue(i - 1 + G::kStages, last, coming);
                if (now != id || (nth & 3) == 0) {  // (every 256 rows too: the tensor cores cut bits off a long sum)
                    tc_after();
                    take_over();
                    if (now != id) finish(id);
                }
            }
            if (now != id) nth = 0;
            id = now;
#pragma unroll
            for (int p = 0; p < kGradRows / kHStep; ++p) {
                float4 v = reinterpret_cast<const float4*>(hs + stage * G::kHBytes)[p * kThreads + tid];
                if constexpr (E8) {
                    const float s = reinterpret_cast<const float*>(scales + stage * G::kScaleBytes)[h_row + p * kHStep];
                    v.x *= s, v.y *= s, v.z *= s, v.w *= s;
                }
                uint2 q[3];
                cut(v, q);
#pragma unroll
                for (int t = 0; t < 3; ++t) *reinterpret_cast<uint2*>(parts + part_to[t] + p * kHStep * 128) = q[t];
            }
            if constexpr (E8) {
#pragma unroll
                for (int p = 0; p < kGradRows / kXStep; ++p) {
                    uint4 b[2];
                    widen(*reinterpret_cast<const uint4*>(smem + stage * G::kXBytes + x_to + p * kThreads * 16), b);
                    unsigned char* const to = wide + (x_piece >> 2) * G::kBlock + p * kXStep * 128;
                    *reinterpret_cast<uint4*>(to + place<128>(x_row, x_piece * 2 & 7)) = b[0];
                    *reinterpret_cast<uint4*>(to + place<128>(x_row, (x_piece * 2 + 1) & 7)) = b[1];
                }
            }
            fence_proxy_async_smem();
            tc_before();
            __syncthreads();
            if (warp == 0 && elect_one()) {
                tc_after();
                const uint32_t x = E8 ? smem_u32(wide) : smem0 + (uint32_t)stage * G::kXBytes;
#pragma unroll
                for (int ks = 0; ks < kGradRows / 16; ++ks)
#pragma unroll
                    for (int n = 0; n < 3 * RP; n += G::kN)
                        tc_mma(d + n, desc_n(x, G::kBlock) + 128 * ks, desc_n(smem_u32(parts) + n / 64 * G::kBlock, G::kBlock) + 128 * ks,
                               idesc(G::kN, true, true), (nth & 3) != 0 || ks > 0);
                if (!(L.test_stall && i == nc - 1)) tc_commit(&done);
            }
            ++nth;
        }
        copies_wait<0>();
        if (!failed) failed = !mbar_wait(&done, (nc - 1) & 1);
        tc_after();
        take_over();
        __syncthreads();
        finish(id);
        tc_before();
    }
    if (failed) atomicAdd(&grads_timeouts, 1u);
    __syncthreads();
    if (warp == 0) {
        tc_after();
        tc_free<G::kColumns>(d);
    }

    // adapters of few rows, or none: a warp takes some components of one
    const int shares = (L.r + kShare - 1) / kShare;
    for (int u = few ? (int)cta * kWarps + warp : L.n_adapters * shares; u < L.n_adapters * shares; u += ctas * kWarps) {
        const int id = u / shares, j0 = (u - id * shares) * kShare, n = offs[id + 1] - offs[id], at = col0 + lane * 4;
        if (n > kFewest || (n <= 0 && L.accumulate)) continue;
        const bool in = at < L.k;
        int row = lane < n ? L.list[offs[id] + lane] : -1;
        if ((unsigned)row >= (unsigned)L.rows) row = -1;
        int of[kFewest];
        float v[kFewest][4];
#pragma unroll
        for (int t = 0; t < kFewest; ++t) {
            of[t] = __shfl_sync(0xffffffffu, row, t);
            uint2 w = make_uint2(0u, 0u);
            float scale = 1.0f;
            if (in && of[t] >= 0) {
                const char* const from = static_cast<const char*>(L.x) + (of[t] * L.ldx + at) * (E8 ? 1 : 2);
                if constexpr (E8) {
                    w.x = *reinterpret_cast<const uint32_t*>(from);
                    scale = scale_from[of[t]];
                } else {
                    w = *reinterpret_cast<const uint2*>(from);
                }
            }
            if constexpr (E8) {
#pragma unroll
                for (int e = 0; e < 4; e += 2) {
                    const __half2_raw f = __nv_cvt_fp8x2_to_halfraw2((__nv_fp8x2_storage_t)(w.x >> 8 * e), __NV_E4M3);
                    const float2 two = __half22float2(*reinterpret_cast<const __half2*>(&f));
                    v[t][e] = two.x * scale;
                    v[t][e + 1] = two.y * scale;
                }
            } else {
                v[t][0] = bf16lo(w.x), v[t][1] = bf16hi(w.x), v[t][2] = bf16lo(w.y), v[t][3] = bf16hi(w.y);
            }
        }
        float h[kFewest];
#pragma unroll
        for (int t = 0; t < kFewest; ++t) h[t] = of[t] >= 0 && lane < kShare && j0 + lane < L.r ? L.h[(size_t)of[t] * L.r + j0 + lane] : 0.0f;
        float* to = L.grad + ((size_t)id * L.r + j0) * L.k + at;
#pragma unroll 4
        for (int j = 0; j < min(kShare, L.r - j0); ++j, to += L.k) {
            float4 s = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
#pragma unroll
            for (int t = 0; t < kFewest; ++t) {
                if (t >= n) break;
                const float a = __shfl_sync(0xffffffffu, h[t], j);
                s.x = fmaf(a, v[t][0], s.x), s.y = fmaf(a, v[t][1], s.y), s.z = fmaf(a, v[t][2], s.z), s.w = fmaf(a, v[t][3], s.w);
            }
            if (!in) continue;
            if (L.accumulate) {
                const float4 had = *reinterpret_cast<const float4*>(to);
                s.x += had.x, s.y += had.y, s.z += had.z, s.w += had.w;
            }
            *reinterpret_cast<float4*>(to) = s;
        }
    }

    if (L.follows) pdl_wait();  // (what comes after this kernel comes after the one before it too)
    // Adapters of several parts: each of their CTAs sums some of the elements. A CTA can have two such adapters.
    if (ctas == 1 || !split) return;
    __syncthreads();
    cluster_arrive();
    cluster_wait();
    int did = -1;
    for (int side = 0; side < 2 && begin < end; ++side) {
        const int at = side == 0 ? begin : end - 1;  // an entry of the adapter
        int id = first_id;
        while (id + 1 < L.n_adapters && offs[id + 1] <= at) ++id;
        const int from = offs[id], to = offs[id + 1];
        if (id == did || (from >= begin && to <= end)) continue;
        did = id;
        int parties = 0, nth = 0;
        unsigned in = 0;
        for (int c = 0; c < ctas; ++c)
            if (part_at[c] < part_at[c + 1] && part_at[c] < to && part_at[c + 1] > from) {
                nth = c == (int)cta ? parties : nth;
                ++parties;
                in |= 1u << c;
            }
        float* const grad = L.grad + (size_t)id * L.r * L.k;
        for (int p = nth * kThreads + tid; p < RP * kGradCols / 4; p += kThreads * parties) {
            const int j = p / (kGradCols / 4), c4 = col0 + p % (kGradCols / 4) * 4;
            if (j >= L.r || c4 >= L.k) continue;
            float4 v[kMaxCluster];
#pragma unroll
            for (int c = 0; c < kMaxCluster; ++c)
                v[c] = (in >> c & 1) ? cluster_ld4(smem_u32(from <= part_at[c] ? begun : goes_on) + 16 * p, (uint32_t)c)
                                     : make_float4(0.0f, 0.0f, 0.0f, 0.0f);
            float4 s = v[0];
#pragma unroll
            for (int c = 1; c < kMaxCluster; ++c) s.x += v[c].x, s.y += v[c].y, s.z += v[c].z, s.w += v[c].w;
            float4* const out = reinterpret_cast<float4*>(grad + (size_t)j * L.k + c4);
            if (L.accumulate) {
                const float4 had = *out;
                s.x += had.x, s.y += had.y, s.z += had.z, s.w += had.w;
            }
            *out = s;
        }
    }
    __syncthreads();
    cluster_arrive();
    cluster_wait();
}

template <int RP, bool E8>
cudaError_t launch(const AdapterGradsLaunch& a, cudaStream_t stream) {
    using G = Grads<RP, E8>;
    const auto kernel = k_adapter_grads<RP, E8>;
    static std::atomic<int> known[kMaxCluster + 1];
    const cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, G::kSmem);
    if (e != cudaSuccess) return e;
    // The cluster whose rounds take the least time: measured, in 0.1 us, 8 a chunk (10 beside another CTA on the SM), 28 to begin
    // and 17 + 3 c to join. Where two have an SM, seven eighths of the places are counted on.
    const int some = a.rows / (kFewest + 1);  // adapters that may have chunks
    const long long blocks = (a.k + kGradCols - 1) / kGradCols, chunks = a.rows / kGradRows + (some < a.n_adapters ? some : a.n_adapters);
    const int warps = G::kThreads / kWarp, shares = (a.r + kShare - 1) / kShare;
    int ctas = 1;
    long long best = INT64_MAX;
    for (int c = 1; c <= kMaxCluster; ++c) {
        const int fit = G::kCtas == 1 ? resident_clusters(kernel, c, G::kThreads, G::kSmem, known) : G::kCtas * kSms * 7 / 8 / c;
        const long long rounds = (blocks + fit - 1) / fit, chunk = blocks * c > kSms && G::kCtas > 1 ? 10 : 8;
        const long long time = rounds * ((chunks + c - 1) / c * chunk + 28 + (c > 1 ? 17 + 3 * c : 0) + (a.n_adapters * shares + warps * c - 1) / (warps * c) * 5);
        if (time < best) best = time, ctas = c;
    }
    cudaLaunchConfig_t cfg = launch_shape(dim3((unsigned)(blocks * ctas)), G::kThreads, stream);
    cfg.dynamicSmemBytes = G::kSmem;
    cudaLaunchAttribute at[2]{};
    at[0].id = cudaLaunchAttributeClusterDimension;
    at[0].val.clusterDim = {(unsigned)ctas, 1, 1};
    at[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at[1].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = at;
    cfg.numAttrs = 2;
    return cudaLaunchKernelEx(&cfg, kernel, a, ctas);
}

template <bool E8>
cudaError_t launch_rank(const AdapterGradsLaunch& a, cudaStream_t stream) {
    if (a.r <= 16) return launch<16, E8>(a, stream);
    if (a.r <= 32) return launch<32, E8>(a, stream);
    return a.r <= 64 ? launch<64, E8>(a, stream) : launch<128, E8>(a, stream);
}

}  // namespace

cudaError_t launch_adapter_grads(const AdapterGradsLaunch& a, bool e4m3, cudaStream_t stream) {
    return e4m3 ? launch_rank<true>(a, stream) : launch_rank<false>(a, stream);
}

cudaError_t adapter_grads_timeouts(unsigned* n, cudaStream_t stream) {
    return cudaMemcpyFromSymbolAsync(n, grads_timeouts, sizeof *n, 0, cudaMemcpyDeviceToHost, stream);
}

}  // namespace tsffn
