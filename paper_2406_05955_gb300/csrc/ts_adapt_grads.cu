// ts_adapt_grads.cu -- gradients of low-rank adapters: grad[i] = sum over the rows t of adapter i of h[t]^T x[t]
// (ts_adapter_grads).
//
// A CTA has 128 columns of x; the rows of an adapter come in chunks of 64, gathered by the list, and are the products' k.
// x is exact in bf16 (e4m3 rows too: the scale that 128 of their columns share is multiplied into h), h is split into three bf16
// numbers of 8 bits each. An adapter of many rows is shared by the CTAs of a cluster, whose sums meet through distributed
// shared memory in the order of the CTAs; the others go to one CTA each. Which are which follows from the numbers of rows in
// the list, so one with nearly all rows does not wait for one CTA.
//
// Ranks up to 64: the columns of x are the M of the tensor cores and the three parts of h, side by side, their N: one
// instruction for 16 rows, sums in tensor memory. Above: the warps' matrix instructions, a part at a time.
//
// Memory bounds it: x once, h once for each 128 columns from L2.
#include <cuda_fp8.h>

#include "ts_adapt.cuh"
#include "ts_grouped.h"

namespace tsffn {
namespace {

__device__ unsigned grads_status;

constexpr int kGradCols = 128, kGradRows = 64;
constexpr int kIdRing = 8;

// Whether an adapter's rows are shared by the CTAs of a cluster: where one CTA would have more than twice the even share.
__device__ __forceinline__ bool shared_rows(int count, int even) { return count > max(2 * even, kGradRows); }

// First entry of adapter `id` in the list, and their number.
__device__ __forceinline__ int2 entries(const AdapterGradsLaunch& L, int id) {
    const int begin = min(max(L.offsets[id], 0), L.rows);
    return make_int2(begin, min(max(L.offsets[id + 1], begin), L.rows) - begin);
}

// The adapters of a CTA: `sums(id, first entry, entries, whether the cluster shares them)` for each. Those that are shared go
// round by cluster, the others by CTA.
template <typename F>
__device__ __forceinline__ void each_adapter(const AdapterGradsLaunch& L, int ctas, uint32_t cta, int even, const F& sums) {
    // thread t looks at adapter t, and the masks say which ones are this CTA's
    __shared__ unsigned bigs[kWarps], smalls[kWarps];
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int count = tid < L.n_adapters ? entries(L, tid).y : 0;
    const bool big = ctas > 1 && shared_rows(count, even);
    const bool small = tid < L.n_adapters && !big && !(count == 0 && L.accumulate);
    const unsigned big_here = __ballot_sync(0xffffffffu, big), small_here = __ballot_sync(0xffffffffu, small);
    if (lane == 0) {
        bigs[warp] = big_here;
        smalls[warp] = small_here;
    }
    __syncthreads();
    unsigned nth_big = __popc(big_here & ((1u << lane) - 1u)), nth_small = __popc(small_here & ((1u << lane) - 1u));
    for (int w = 0; w < warp; ++w) {
        nth_big += __popc(bigs[w]);
        nth_small += __popc(smalls[w]);
    }
    __syncthreads();
    const unsigned my_big = __ballot_sync(0xffffffffu, big && nth_big % gridDim.y == blockIdx.y);
    const unsigned my_small = __ballot_sync(0xffffffffu, small && nth_small % (gridDim.y * ctas) == blockIdx.y * ctas + cta);
    if (lane == 0) {
        bigs[warp] = my_big;
        smalls[warp] = my_small;
    }
    __syncthreads();
    for (int shared = 1; shared >= 0; --shared)
        for (int w = 0; w < kWarps; ++w)
            for (unsigned m = shared ? bigs[w] : smalls[w]; m != 0u; m &= m - 1u) {
                const int id = w * kWarp + __ffs(m) - 1;
                const int2 of = entries(L, id);
                sums(id, of.x, of.y, shared != 0);
            }
}

// The part of the list that a CTA has of an adapter's entries: chunks c0 .. c0 + nc - 1 of those from `begin` on.
struct Share {
    int first, end, nc;
    __device__ Share(int begin, int count, int parties, int me) {
        const int chunks = (count + kGradRows - 1) / kGradRows;
        const int c0 = (int)((long long)chunks * me / parties);
        nc = (int)((long long)chunks * (me + 1) / parties) - c0;
        first = begin + c0 * kGradRows;
        end = begin + count;
    }
    // thread's row of chunk i
    __device__ int row(const AdapterGradsLaunch& L, int i) const {
        const int at = first + i * kGradRows + (int)threadIdx.x;
        const int r = threadIdx.x < kGradRows && i < nc && at < end ? L.list[at] : -1;
        return (unsigned)r < (unsigned)L.rows ? r : -1;
    }
};

// The cluster's sums [RP][128 columns] of shared memory at `at`, summed and stored. Ends with a cluster barrier: what is there
// may then be overwritten.
template <int RP>
__device__ __forceinline__ void join_sums(const AdapterGradsLaunch& L, float* grad, uint32_t at, int col0, int ctas, uint32_t cta) {
    __syncthreads();
    cluster_arrive();
    cluster_wait();
    constexpr int kQuads = RP * kGradCols / 4;
    for (int p = (int)cta * kThreads + threadIdx.x; p < kQuads; p += kThreads * ctas) {
        const int j = p / (kGradCols / 4), col = col0 + p % (kGradCols / 4) * 4;
        if (j >= L.r || col >= L.k) continue;
        float4 v[kMaxCluster];
#pragma unroll
        for (int c = 0; c < kMaxCluster; ++c)
            if (c < ctas) v[c] = cluster_ld4(at + 16 * p, (uint32_t)c);
        float4* const to = reinterpret_cast<float4*>(grad + (size_t)j * L.k + col);
        float4 s = v[0];
#pragma unroll
        for (int c = 1; c < kMaxCluster; ++c)
            if (c < ctas) s.x += v[c].x, s.y += v[c].y, s.z += v[c].z, s.w += v[c].w;
        if (L.accumulate) {
            const float4 had = *to;
            s.x += had.x, s.y += had.y, s.z += had.z, s.w += had.w;
        }
        *to = s;
    }
    __syncthreads();
    cluster_arrive();
    cluster_wait();
}

// Four numbers as three bf16 numbers each, cut off (8, 8 and the last 8 bits: nothing is lost). An infinity or NaN is the
// first alone.
__device__ __forceinline__ void cut(const float4& v, uint2 (&p)[3]) {
    float f[4] = {v.x, v.y, v.z, v.w}, hi[4];
    uint32_t w[3][4];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        w[0][e] = __float_as_uint(f[e]);
        hi[e] = __uint_as_float(w[0][e] & 0xffff0000u);
        const float rest = f[e] - hi[e];
        w[1][e] = __float_as_uint(rest);
        w[2][e] = __float_as_uint(rest - __uint_as_float(w[1][e] & 0xffff0000u));
    }
    if (!(fabsf(f[0]) < INFINITY) || !(fabsf(f[1]) < INFINITY) || !(fabsf(f[2]) < INFINITY) || !(fabsf(f[3]) < INFINITY)) {
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

// ---------------------------------------------------------------------------
// r up to 64
// ---------------------------------------------------------------------------
template <int RP, bool E8>
struct Wide {
    static constexpr int kXBytes = kGradRows * kGradCols * (E8 ? 1 : 2), kHBytes = kGradRows * RP * 4;
    static constexpr int kStages = 3;
    // x starts on 1024 bytes in a stage; h, and for e4m3 rows their scales, lie in rings of their own
    static constexpr int kWideBytes = E8 ? 2 * kGradRows * kGradCols * 2 : 0;  // two chunks of x in bf16
    static constexpr int kBlock = kGradRows * 128;                             // 64 columns of a chunk
    static constexpr int kPart = (3 * RP + 63) / 64 * kBlock;                  // h of a chunk, its parts side by side
    static constexpr int kScaleBytes = E8 ? kGradRows * 4 : 0;
    static constexpr int kSmem = 1024 + kStages * (kXBytes + kHBytes + kScaleBytes) + kWideBytes + 2 * kPart;
    static constexpr int kColumns = RP == 16 ? 64 : RP == 32 ? 128 : 256;      // of tensor memory
    static constexpr int kMine = RP / 2;                                       // components of a thread's column
    static_assert(kStages * kXBytes + kWideBytes >= RP * kGradCols * 4 && kStages + 2 <= kIdRing && 3 * RP <= kColumns, "");
};

template <int RP, bool E8>
__global__ void __launch_bounds__(kThreads, RP <= 32 ? 2 : 1) k_adapter_grads_wide(const __grid_constant__ AdapterGradsLaunch L, int ctas, int even) {
    using G = Wide<RP, E8>;
    extern __shared__ unsigned char raw[];
    __shared__ int ids[kIdRing][kGradRows];
    __shared__ uint64_t done[2];
    __shared__ uint32_t tmem;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const uint32_t cta = cluster_rank();
    unsigned char* const smem = reinterpret_cast<unsigned char*>((reinterpret_cast<uintptr_t>(raw) + 1023) & ~(uintptr_t)1023);
    unsigned char* const wide = smem + G::kStages * G::kXBytes;
    unsigned char* const parts = wide + G::kWideBytes;
    unsigned char* const hs = parts + 2 * G::kPart;
    unsigned char* const scales = hs + G::kStages * G::kHBytes;
    const uint32_t smem0 = smem_u32(smem), hs0 = smem_u32(hs), scales0 = smem_u32(scales);
    const int col0 = (int)(blockIdx.x / ctas) * kGradCols;
    const bool h_vec = L.r % 4 == 0 && (reinterpret_cast<uintptr_t>(L.h) & 15u) == 0;
    const int quarter = (warp & 3) * 32, half = warp >> 2;
    if (tid == 0) {
        mbar_init(&done[0], 1);
        mbar_init(&done[1], 1);
        mbar_fence_init();
    }
    pdl_wait();
    if (warp == 0) tc_alloc<G::kColumns>(&tmem);
    tc_before();
    __syncthreads();
    tc_after();
    const uint32_t d = tmem;
    bool failed = false;
    unsigned uses = 0;  // chunks multiplied so far

    const auto sums = [&](int id, int begin, int count, bool join) {
        const Share S(begin, count, join ? ctas : 1, join ? (int)cta : 0);
        const auto issue = [&](int i) {
            if (i < S.nc) {
                const uint32_t to = smem0 + (uint32_t)(i % G::kStages) * G::kXBytes;
                const int* const rows = ids[i % kIdRing];
                constexpr int kPieces = kGradCols * (E8 ? 1 : 2) / 16;
                const int c = tid % kPieces, col = col0 + c * (E8 ? 16 : 8);
#pragma unroll
                for (int p = 0; p < kGradRows * kPieces / kThreads; ++p) {
                    const int row = tid / kPieces + p * (kThreads / kPieces), at = rows[row];
                    const bool in = at >= 0 && col < L.k;
                    const char* const from = static_cast<const char*>(L.x) + (in ? (at * L.ldx + col) * (E8 ? 1 : 2) : 0);
                    copy16(E8 ? to + (tid + p * kThreads) * 16 : to + (c >> 3) * G::kBlock + place<128>(row, c & 7), from, in);
                }
                const uint32_t h = hs0 + (uint32_t)(i % G::kStages) * G::kHBytes;
                if (h_vec) {
#pragma unroll
                    for (int p = 0; p < kGradRows * (RP / 4) / kThreads; ++p) {
                        const int at = tid + p * kThreads, row = rows[at / (RP / 4)], j = at % (RP / 4) * 4;
                        const bool in = row >= 0 && j < L.r;
                        copy16(h + at * 16, in ? L.h + (size_t)row * L.r + j : L.h, in);
                    }
                } else {  // (a thread copies what it reads)
#pragma unroll
                    for (int p = 0; p < kGradRows * (RP / 4) / kThreads; ++p)
#pragma unroll
                        for (int e = 0; e < 4; ++e) {
                            const int at = tid + p * kThreads, row = rows[at / (RP / 4)], j = at % (RP / 4) * 4 + e;
                            const bool in = row >= 0 && j < L.r;
                            copy4(h + at * 16 + e * 4, in ? L.h + (size_t)row * L.r + j : L.h, in);
                        }
                }
                if (E8 && tid < kGradRows) {
                    const bool in = rows[tid] >= 0;
                    copy4(scales0 + (uint32_t)(i % G::kStages) * G::kScaleBytes + tid * 4,
                          in ? L.x_scale + (int64_t)(col0 / kScaleBlock) * L.ld_scale + rows[tid] : L.x_scale, in);
                }
            }
            copies_commit();
        };
        float sum[G::kMine] = {};
        __syncthreads();  // (of what the last adapter has in shared memory)
        int next = -1;
        for (int i = 0; i < G::kStages; ++i) {
            next = S.row(L, i);
            if (tid < kGradRows) ids[i][tid] = next;
        }
        next = S.row(L, G::kStages);
        __syncthreads();
#pragma unroll
        for (int i = 0; i < G::kStages; ++i) issue(i);
        for (int i = 0; i < S.nc; ++i) {
            if (i == 0) copies_wait<G::kStages - 1>();
            else copies_wait<G::kStages - 2>();
            if (E8) __syncthreads();  // (the scales)
            if (tid < kGradRows) ids[(i + G::kStages) % kIdRing][tid] = next;
            next = S.row(L, i + G::kStages + 1);
            unsigned char* const part = parts + (i & 1) * G::kPart;
            const float4* const h = reinterpret_cast<const float4*>(hs + (i % G::kStages) * G::kHBytes);
#pragma unroll
            for (int p = 0; p < kGradRows * (RP / 4) / kThreads; ++p) {
                const int at = tid + p * kThreads, row = at / (RP / 4), j = at % (RP / 4) * 4;
                float4 v = h[at];
                if constexpr (E8) {
                    const float s = reinterpret_cast<const float*>(scales + (i % G::kStages) * G::kScaleBytes)[row];
                    v.x *= s, v.y *= s, v.z *= s, v.w *= s;
                }
                uint2 q[3];
                cut(v, q);
#pragma unroll
                for (int t = 0; t < 3; ++t) {
                    const int c = t * RP + j;
                    *reinterpret_cast<uint2*>(part + (c >> 6) * G::kBlock + place<128>(row, (c & 63) >> 3) + (c & 7) * 2) = q[t];
                }
            }
            if constexpr (E8) {
                unsigned char* const to = wide + (i & 1) * (kGradRows * kGradCols * 2);
#pragma unroll
                for (int p = 0; p < kGradRows * kGradCols / 16 / kThreads; ++p) {
                    const int at = tid + p * kThreads, row = at / (kGradCols / 16), c = at % (kGradCols / 16) * 2;
                    uint4 b[2];
                    widen(reinterpret_cast<const uint4*>(smem + (i % G::kStages) * G::kXBytes)[at], b);
                    *reinterpret_cast<uint4*>(to + (c >> 3) * G::kBlock + place<128>(row, c & 7)) = b[0];
                    *reinterpret_cast<uint4*>(to + (c >> 3) * G::kBlock + place<128>(row, (c + 1) & 7)) = b[1];
                }
            }
            fence_proxy_async_smem();
            tc_before();
            __syncthreads();
            if (warp == 0 && elect_one()) {
                tc_after();
                const uint32_t x = E8 ? smem_u32(wide) + (i & 1) * (kGradRows * kGradCols * 2) : smem0 + (uint32_t)(i % G::kStages) * G::kXBytes;
#pragma unroll
                for (int ks = 0; ks < kGradRows / 16; ++ks)
                    tc_mma(d, desc_n(x, G::kBlock) + 128 * ks, desc_n(smem_u32(part), G::kBlock) + 128 * ks, idesc(3 * RP, true, true),
                           (i & 3) != 0 || ks > 0);
                if (!(L.test_stall && i == S.nc - 1)) tc_commit(&done[uses & 1]);
            }
            ++uses;
            // Every 256 rows the sums leave the tensor cores, which cut bits off a long one; what is read then is complete.
            const bool take = (i & 3) == 3 || i == S.nc - 1;
            if (i > 0 && !failed) failed = !mbar_wait(&done[(uses - 2) & 1], (uses - 2) >> 1 & 1);
            if (take) {
                if (!failed) failed = !mbar_wait(&done[(uses - 1) & 1], (uses - 1) >> 1 & 1);
                tc_after();
                float v[G::kMine];
#pragma unroll
                for (int q = 2; q >= 0; --q) {
#pragma unroll
                    for (int j = 0; j < G::kMine; j += 8) tc_ld8(d + ((uint32_t)quarter << 16) + q * RP + half * G::kMine + j, v + j);
                    tc_ld_wait(v);
#pragma unroll
                    for (int j = 0; j < G::kMine; ++j) sum[j] += v[j];
                }
                tc_before();
            }
            if (i > 0) issue(i - 1 + G::kStages);
        }
        copies_wait<0>();
        float* const grad = L.grad + (size_t)id * L.r * L.k;
        const int col = quarter + lane;
        if (join) {
            __syncthreads();  // the stages hold the sums now
#pragma unroll
            for (int j = 0; j < G::kMine; ++j) reinterpret_cast<float*>(smem)[(half * G::kMine + j) * kGradCols + col] = sum[j];
            join_sums<RP>(L, grad, smem0, col0, ctas, cta);
            return;
        }
        if (col0 + col < L.k)
#pragma unroll
            for (int j = 0; j < G::kMine; ++j)
                if (half * G::kMine + j < L.r) {
                    float* const to = grad + (size_t)(half * G::kMine + j) * L.k + col0 + col;
                    *to = L.accumulate ? *to + sum[j] : sum[j];
                }
    };
    each_adapter(L, ctas, cta, even, sums);
    if (failed) atomicOr(&grads_status, kStatusTimeout);
    tc_before();
    __syncthreads();
    if (warp == 0) {
        tc_after();
        tc_free<G::kColumns>(d);
    }
}

// ---------------------------------------------------------------------------
// r above 64
// ---------------------------------------------------------------------------
template <int RP, bool E8>
struct Grads {
    static constexpr int kXPitch = kGradCols * (E8 ? 1 : 2);
    static constexpr int kXBytes = kGradRows * kXPitch, kHBytes = kGradRows * RP * 4, kScaleBytes = E8 ? kGradRows * 4 : 0;
    static constexpr int kStage = kXBytes + kHBytes + kScaleBytes;
    static constexpr int kStages = 3;
    static constexpr int kHPitch = RP * 2 + 16;
    static constexpr int kPartBytes = kGradRows * kHPitch;
    static constexpr int kWide = E8 ? kGradRows * kChunk : 0;  // x in bf16
    static constexpr int kSmem = kStages * kStage + 3 * kPartBytes + kWide;
    static constexpr int kMGroups = RP == 16 ? 1 : 2;          // ways that the warps share the components
    static constexpr int kMT = RP / 16 / kMGroups;             // 16-component tiles of a warp
    static constexpr int kNT = kGradCols / 8 / (kWarps / kMGroups);
    static_assert(kStages * kStage >= RP * kGradCols * 4 && kStages + 2 <= kIdRing, "");
};

template <int RP, bool E8>
__global__ void __launch_bounds__(kThreads) k_adapter_grads(const __grid_constant__ AdapterGradsLaunch L, int ctas, int even) {
    using G = Grads<RP, E8>;
    extern __shared__ __align__(128) unsigned char smem[];
    __shared__ int ids[kIdRing][kGradRows];
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const uint32_t cta = cluster_rank();
    unsigned char* const parts = smem + G::kStages * G::kStage;
    unsigned char* const wide = parts + 3 * G::kPartBytes;
    const uint32_t smem0 = smem_u32(smem), parts0 = smem_u32(parts), wide0 = smem_u32(wide);
    const int col0 = (int)(blockIdx.x / ctas) * kGradCols;
    const bool h_vec = L.r % 4 == 0 && (reinterpret_cast<uintptr_t>(L.h) & 15u) == 0;
    pdl_wait();

    const auto sums = [&](int id, int begin, int count, bool join) {
        const Share S(begin, count, join ? ctas : 1, join ? (int)cta : 0);
        const int nc = S.nc;
        const auto issue = [&](int i) {
            if (i < nc) {
                const uint32_t to = smem0 + (uint32_t)(i % G::kStages) * G::kStage;
                const int* const rows = ids[i % kIdRing];
                constexpr int kPieces = G::kXPitch / 16;
#pragma unroll
                for (int p = tid; p < kGradRows * kPieces; p += kThreads) {
                    const int row = p / kPieces, c = p % kPieces, col = col0 + c * (E8 ? 16 : 8);
                    const bool in = rows[row] >= 0 && col < L.k;
                    const char* const from = static_cast<const char*>(L.x) + (in ? (rows[row] * L.ldx + col) * (E8 ? 1 : 2) : 0);
                    copy16(to + (E8 ? p * 16 : place<kChunk>(row, c)), from, in);
                }
                const uint32_t h = to + G::kXBytes;
                if (h_vec) {
                    for (int p = tid; p < kGradRows * (RP / 4); p += kThreads) {
                        const int row = p / (RP / 4), j = p % (RP / 4) * 4;
                        const bool in = rows[row] >= 0 && j < L.r;
                        copy16(h + p * 16, in ? L.h + (size_t)rows[row] * L.r + j : L.h, in);
                    }
                } else {
                    for (int p = tid; p < kGradRows * RP; p += kThreads) {
                        const int row = p / RP, j = p % RP;
                        const bool in = rows[row] >= 0 && j < L.r;
                        copy4(h + p * 4, in ? L.h + (size_t)rows[row] * L.r + j : L.h, in);
                    }
                }
                if (E8 && tid < kGradRows) {
                    const bool in = rows[tid] >= 0;
                    copy4(h + G::kHBytes + tid * 4,
                          in ? L.x_scale + (int64_t)(col0 / kScaleBlock) * L.ld_scale + rows[tid] : L.x_scale, in);
                }
            }
            copies_commit();
        };
        float acc[G::kMT][G::kNT][4] = {}, sum[G::kMT][G::kNT][4] = {};
        int next = -1;
        __syncthreads();  // (of what the last sums have in shared memory)
        for (int i = 0; i < G::kStages; ++i) {
            next = S.row(L, i);
            if (tid < kGradRows) ids[i][tid] = next;
        }
        next = S.row(L, G::kStages);
        __syncthreads();
#pragma unroll
        for (int i = 0; i < G::kStages - 1; ++i) issue(i);
        const int mg = warp % G::kMGroups, n0 = warp / G::kMGroups * G::kNT * 8;
        for (int i = 0; i < nc; ++i) {
            copies_wait<G::kStages - 2>();
            __syncthreads();
            if (tid < kGradRows) ids[(i + G::kStages) % kIdRing][tid] = next;
            next = S.row(L, i + G::kStages + 1);
            issue(i + G::kStages - 1);
            const unsigned char* const stage = smem + (i % G::kStages) * G::kStage;
            const float* const h = reinterpret_cast<const float*>(stage + G::kXBytes);
#pragma unroll 4
            for (int p = tid; p < kGradRows * (RP / 4); p += kThreads) {
                const int row = p / (RP / 4), j = p % (RP / 4) * 4;
                float4 v = reinterpret_cast<const float4*>(h)[p];
                if constexpr (E8) {
                    const float s = reinterpret_cast<const float*>(stage + G::kXBytes + G::kHBytes)[row];
                    v.x *= s, v.y *= s, v.z *= s, v.w *= s;
                }
                uint2 q[3];
                cut(v, q);
#pragma unroll
                for (int t = 0; t < 3; ++t) *reinterpret_cast<uint2*>(parts + t * G::kPartBytes + row * G::kHPitch + j * 2) = q[t];
            }
            if constexpr (E8) {
#pragma unroll
                for (int p = tid; p < kGradRows * kGradCols / 16; p += kThreads) {
                    const int row = p / (kGradCols / 16), c = p % (kGradCols / 16) * 2;
                    uint4 b[2];
                    widen(reinterpret_cast<const uint4*>(stage)[p], b);
                    *reinterpret_cast<uint4*>(wide + place<kChunk>(row, c)) = b[0];
                    *reinterpret_cast<uint4*>(wide + place<kChunk>(row, c + 1)) = b[1];
                }
            }
            __syncthreads();
            const uint32_t x0 = E8 ? wide0 : smem0 + (uint32_t)(i % G::kStages) * G::kStage;
#pragma unroll
            for (int ks = 0; ks < kGradRows / 16; ++ks) {
                uint32_t w[G::kNT / 2][4];
#pragma unroll
                for (int t = 0; t < G::kNT; t += 2)
                    ldmatrix4_t(w[t / 2], x0 + place<kChunk>(ks * 16 + (lane & 15), n0 / 8 + t + (lane >> 4)));
#pragma unroll
                for (int m = 0; m < G::kMT; ++m)
#pragma unroll
                    for (int q = 2; q >= 0; --q) {
                        uint32_t a[4];
                        ldmatrix4_t(a, parts0 + q * G::kPartBytes + (ks * 16 + (lane & 7) + (lane >> 4) * 8) * G::kHPitch +
                                           ((mg * G::kMT + m) * 16 + ((lane >> 3) & 1) * 8) * 2);
#pragma unroll
                        for (int t = 0; t < G::kNT; t += 2) {
                            mma(acc[m][t], a, w[t / 2][0], w[t / 2][1]);
                            mma(acc[m][t + 1], a, w[t / 2][2], w[t / 2][3]);
                        }
                    }
            }
#pragma unroll
            for (int m = 0; m < G::kMT; ++m)
#pragma unroll
                for (int t = 0; t < G::kNT; ++t)
#pragma unroll
                    for (int e = 0; e < 4; ++e) {  // (the tensor cores cut bits off a long sum)
                        sum[m][t][e] += acc[m][t][e];
                        acc[m][t][e] = 0.0f;
                    }
        }
        float* const grad = L.grad + (size_t)id * L.r * L.k;
        if (!join) {
#pragma unroll
            for (int m = 0; m < G::kMT; ++m)
#pragma unroll
                for (int t = 0; t < G::kNT; ++t)
#pragma unroll
                    for (int e = 0; e < 4; e += 2) {
                        const int j = (mg * G::kMT + m) * 16 + lane / 4 + e * 4, col = col0 + n0 + t * 8 + (lane & 3) * 2;
                        if (j >= L.r || col >= L.k) continue;
                        float2* const to = reinterpret_cast<float2*>(grad + (size_t)j * L.k + col);
                        float2 v = make_float2(sum[m][t][e], sum[m][t][e + 1]);
                        if (L.accumulate) {
                            const float2 had = *to;
                            v.x += had.x, v.y += had.y;
                        }
                        *to = v;
                    }
            return;
        }
        copies_wait<0>();
        __syncthreads();  // the stages hold the sums now
        float* const mine = reinterpret_cast<float*>(smem);
#pragma unroll
        for (int m = 0; m < G::kMT; ++m)
#pragma unroll
            for (int t = 0; t < G::kNT; ++t)
#pragma unroll
                for (int e = 0; e < 4; e += 2)
                    *reinterpret_cast<float2*>(mine + ((mg * G::kMT + m) * 16 + lane / 4 + e * 4) * kGradCols + n0 + t * 8 + (lane & 3) * 2) =
                        make_float2(sum[m][t][e], sum[m][t][e + 1]);
        join_sums<RP>(L, grad, smem0, col0, ctas, cta);
    };

    each_adapter(L, ctas, cta, even, sums);
}

template <typename Kernel>
cudaError_t launch(Kernel kernel, int smem, const AdapterGradsLaunch& a, cudaStream_t stream) {
    const cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, smem);
    if (e != cudaSuccess) return e;
    // about two rounds of CTAs, in clusters of 8: fewer where there are no more adapters or chunks than that
    const int blocks = (a.k + kGradCols - 1) / kGradCols;
    int ctas = kMaxCluster;
    while (ctas > 1 && (long long)ctas * kGradRows / 2 >= a.rows) ctas /= 2;
    const int wish = (kResidentCtas * 2 + blocks * ctas - 1) / (blocks * ctas);
    const int ys = wish < a.n_adapters ? wish : a.n_adapters;
    const int even = (int)((long long)a.rows * blocks / kResidentCtas);
    cudaLaunchConfig_t cfg = launch_shape(dim3((unsigned)(blocks * ctas), (unsigned)ys), kThreads, stream);
    cfg.dynamicSmemBytes = smem;
    cudaLaunchAttribute at[2]{};
    at[0].id = cudaLaunchAttributeClusterDimension;
    at[0].val.clusterDim = {(unsigned)ctas, 1, 1};
    at[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at[1].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = at;
    cfg.numAttrs = 2;
    return cudaLaunchKernelEx(&cfg, kernel, a, ctas, even);
}

template <bool E8>
cudaError_t launch_rank(const AdapterGradsLaunch& a, cudaStream_t stream) {
    if (a.r <= 16) return launch(k_adapter_grads_wide<16, E8>, Wide<16, E8>::kSmem, a, stream);
    if (a.r <= 32) return launch(k_adapter_grads_wide<32, E8>, Wide<32, E8>::kSmem, a, stream);
    if (a.r <= 64) return launch(k_adapter_grads_wide<64, E8>, Wide<64, E8>::kSmem, a, stream);
    return launch(k_adapter_grads<128, E8>, Grads<128, E8>::kSmem, a, stream);
}

}  // namespace

cudaError_t launch_adapter_grads(const AdapterGradsLaunch& a, bool e4m3, cudaStream_t stream) {
    return e4m3 ? launch_rank<true>(a, stream) : launch_rank<false>(a, stream);
}

cudaError_t adapter_grads_status(unsigned* bits, cudaStream_t stream) {
    static const unsigned zero = 0;
    cudaError_t e = cudaMemcpyFromSymbolAsync(bits, grads_status, sizeof *bits, 0, cudaMemcpyDeviceToHost, stream);
    if (e == cudaSuccess) e = cudaMemcpyToSymbolAsync(grads_status, &zero, sizeof zero, 0, cudaMemcpyHostToDevice, stream);
    return e == cudaSuccess ? cudaStreamSynchronize(stream) : e;
}

}  // namespace tsffn
