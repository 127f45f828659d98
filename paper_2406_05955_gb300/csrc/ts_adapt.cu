// ts_adapt.cu -- low-rank adapters of many requests beside a shared projection: h[t] = s_i x[t] A_i^T and
// out[t] = y[t] + h[t] B_i for the adapter i of row t (ts_adapt_rows), and the sums over rows of h^T x that are the
// gradients of A and B (ts_adapter_grads). With A and B exchanged the first is also the backward pass by rows.
//
// Both products in one launch. A cluster of CTAs has a tile of up to 16 or 64 rows of one adapter: each CTA sums its part
// of k for the whole tile, the parts of h meet through distributed shared memory, summed in the same order by all, and each
// CTA adds h B_i to its part of the columns. One ring of chunks, 256 bytes of each row wide, carries x and A_i and then y and B_i: while h is
// being joined the first chunks of y are already on their way. Rows of a tile are gathered (a list by adapter), so they
// come by 16-byte asynchronous copies.
//
// Memory bounds it: x, y and out are 2 k + 2 n elements a row, the products 2 r flops for each of them.
#include <cuda_fp8.h>

#include "ts_adapt.cuh"
#include "ts_grouped.h"

namespace tsffn {
namespace {

// ---------------------------------------------------------------------------
// h and out
// ---------------------------------------------------------------------------
// MT: rows of a tile. RP: r rounded up to 16, 32, 64 or 128.
template <int MT, int RP, typename TY>
struct Tile {
    static constexpr int kCols = kChunk / 2;                          // of x and A in a chunk
    static constexpr int kOutCols = kChunk / (int)sizeof(TY);         // of y and out
    static constexpr int kBPitch = kOutCols * 2;                      // bytes of a row of B
    static constexpr int kParts = sizeof(TY) == 2 ? 2 : 3;            // bf16 numbers that h enters the second product as
    static constexpr int kStage = (MT + RP) * kChunk;
    static constexpr int kMTiles = MT / 16;
    static constexpr int kSides = kWarps / kMTiles;                   // warps that share 16 rows
    static constexpr int kNSplit = MT == 64 && RP == 128 ? 2 : 1;     // ways that those share r in the first product
    static constexpr int kSlabs = kSides / kNSplit;                   // and k
    static constexpr int kNT = RP / 8 / kNSplit;                      // 8-column tiles of a warp in the first product
    static constexpr int kOT = kOutCols / 8 / kSides;                 // and in the second
    static constexpr int kHPitch = RP * 2 + 16;
    static constexpr int kSlabBytes = MT * RP * 4;
    static constexpr int kPartBytes = MT * kHPitch;
    // the sums of h of this CTA (a slab for each warp of 16 rows; 64 rows' two warps add to one), and h as bf16 numbers
    static constexpr int kFixed = (MT == 16 ? kSlabs : 1) * kSlabBytes + kParts * kPartBytes;
    // two CTAs on an SM where two stages fit (the loads in flight of two cover the latency, and one works while the other joins)
    static constexpr int kHalf = 113 * 1024 - kFixed, kWhole = 226 * 1024 - kFixed;
    static constexpr int kWish = MT == 16 ? 8 : 4;
    static constexpr int kFit = kHalf >= 2 * kStage ? kHalf / kStage : kWhole / kStage;
    static constexpr int kStages = kFit < kWish ? kFit : kWish;
    static constexpr int kSmem = kStages * kStage + kFixed;
    static constexpr int kCtas = kSmem <= 113 * 1024 && RP <= 64 ? 2 : 1;  // on an SM
    static_assert(kStages >= 2, "");
};

// Without a list, of up to 64 rows: tile number t is there if row t is the first, 17th, 33rd or 49th of its adapter.
template <int MT>
__device__ __forceinline__ void find_few(const AdaptLaunch& L, int t, TileRows* found, int* rows) {
    static_assert(kFewRows == 64, "");
    if (threadIdx.x >= kWarp) return;
    const int lane = threadIdx.x;
    int id[2];
    unsigned same[2];
    const int mine = min((unsigned)L.ids[t], (unsigned)L.n_adapters);
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const int row = lane + i * kWarp;
        id[i] = row < L.rows ? (int)min((unsigned)L.ids[row], (unsigned)L.n_adapters) : -1;
        same[i] = __ballot_sync(0xffffffffu, id[i] == mine);
    }
    const unsigned long long all = (unsigned long long)same[1] << 32 | same[0];
    const int before = __popcll(all & ((1ull << t) - 1ull));
    const bool leads = before % MT == 0;
    if (lane == 0) *found = {leads ? mine : -1, 0, 0, leads ? min(MT, __popcll(all) - before) : 0};
    for (int i = lane; i < MT; i += kWarp) rows[i] = -1;
    __syncwarp();
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const int row = lane + i * kWarp, at = __popcll(all & ((1ull << row) - 1ull)) - before;
        if (id[i] == mine && at >= 0 && at < MT) rows[at] = row;
    }
}

template <int MT, int RP, typename TY>
__global__ void __launch_bounds__(kThreads, Tile<MT, RP, TY>::kCtas) k_adapt(const __grid_constant__ AdaptLaunch L, int ctas) {
    using T = Tile<MT, RP, TY>;
    extern __shared__ __align__(128) unsigned char smem[];
    __shared__ TileRows found;
    __shared__ int rows[MT];
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const uint32_t cta = cluster_rank();
    unsigned char* const parts = smem + T::kStages * T::kStage;
    unsigned char* const slabs = parts + T::kParts * T::kPartBytes;
    const uint32_t smem0 = smem_u32(smem), parts0 = smem_u32(parts);
    pdl_wait();
    if (L.list != nullptr) find_listed<MT>(L, (int)(blockIdx.x / ctas), &found, rows);
    else find_few<MT>(L, (int)(blockIdx.x / ctas), &found, rows);
    __syncthreads();
    const int id = found.id, count = found.count;
    if (id < 0) return;
    const bool some = id < L.n_adapters;
    const int rank = !some ? 0 : L.ranks != nullptr ? min(max(L.ranks[id], 0), L.r) : L.r;
    const __nv_bfloat16* const x = static_cast<const __nv_bfloat16*>(L.x);
    const __nv_bfloat16* const a = static_cast<const __nv_bfloat16*>(L.a) + (size_t)(some ? id : 0) * L.r * L.k;
    const __nv_bfloat16* const b = static_cast<const __nv_bfloat16*>(L.b) + (size_t)(some ? id : 0) * L.r * L.n;
    const TY* const y = static_cast<const TY*>(L.y);
    TY* const out = static_cast<TY*>(L.out);
    const float scale = some && L.scale != nullptr ? L.scale[id] : 1.0f;
    if (rank == 0) {
        if (L.h != nullptr && cta == 0 && blockIdx.y == 0)
            for (int i = tid; i < count * L.r; i += kThreads)
                if (rows[i / L.r] >= 0) L.h[(size_t)rows[i / L.r] * L.r + i % L.r] = 0.0f;
        if (out == y) return;  // (of both nullptr too)
    }

    // this CTA's chunks: of k, and then of n, which the clusters of a tile share as well
    const int k_chunks = rank > 0 ? (L.k + T::kCols - 1) / T::kCols : 0;
    const int n_chunks = out != nullptr ? (L.n + T::kOutCols - 1) / T::kOutCols : 0;
    const int k0 = (int)((long long)k_chunks * cta / ctas), nk = (int)((long long)k_chunks * (cta + 1) / ctas) - k0;
    const int all = ctas * (int)gridDim.y, me = (int)(blockIdx.y * ctas + cta);
    const int n0 = (int)((long long)n_chunks * me / all), nn = (int)((long long)n_chunks * (me + 1) / all) - n0;

    // A thread copies the same 16-byte piece of every 16th row of a chunk of x or y, and of the rows of A or B: where it
    // reads moves on by a chunk from one call to the next.
    constexpr int kPieces = kChunk / 16, kRowStep = kThreads / kPieces, kMine = MT / kRowStep;
    const int piece = tid % kPieces, row0 = tid / kPieces;
    const uint32_t to0 = smem0 + place<kChunk>(row0, piece);
    const char* src[kMine];
    bool there[kMine];
#pragma unroll
    for (int p = 0; p < kMine; ++p) {
        const int row = rows[row0 + p * kRowStep];
        there[p] = row >= 0;
        src[p] = reinterpret_cast<const char*>(x + (there[p] ? row * L.ldx : 0) + k0 * T::kCols + piece * 8);
    }
    const char* mat = reinterpret_cast<const char*>(a + (size_t)row0 * L.k + k0 * T::kCols + piece * 8);
    int col = k0 * T::kCols + piece * 8;
    const auto issue = [&](int i) {
        if (i < nk + nn) {
            const uint32_t to = to0 + (uint32_t)(i % T::kStages) * T::kStage;
            if (i == nk) {
                col = n0 * T::kOutCols + piece * (16 / (int)sizeof(TY));
#pragma unroll
                for (int p = 0; p < kMine; ++p)
                    src[p] = reinterpret_cast<const char*>(y + (there[p] ? rows[row0 + p * kRowStep] * L.ldy : 0) + col);
                constexpr int kBPieces = T::kBPitch / 16;
                mat = reinterpret_cast<const char*>(b + (size_t)(tid / kBPieces) * L.n + n0 * T::kOutCols + tid % kBPieces * 8);
            }
            const bool in = col < (i < nk ? L.k : L.n);
#pragma unroll
            for (int p = 0; p < kMine; ++p) {
                const bool take = in && there[p];
                copy16(to + p * kRowStep * kChunk, take ? src[p] : reinterpret_cast<const char*>(x), take);
                src[p] += kChunk;
            }
            if (i < nk) {
                const int64_t step = (int64_t)kRowStep * L.k * 2;
                const char* from = mat;
#pragma unroll
                for (int p = 0; p < RP / kRowStep; ++p) {
                    const bool take = in && row0 + p * kRowStep < rank;
                    copy16(to + MT * kChunk + p * kRowStep * kChunk, take ? from : reinterpret_cast<const char*>(x), take);
                    from += step;
                }
                mat += kChunk;
                col += T::kCols;
            } else {
                constexpr int kBPieces = T::kBPitch / 16, kBStep = kThreads / kBPieces;
                const int b_row = tid / kBPieces, b_col = col - piece * (16 / (int)sizeof(TY)) + tid % kBPieces * 8;
                const uint32_t b_to = smem0 + (uint32_t)(i % T::kStages) * T::kStage + MT * kChunk + place<T::kBPitch>(b_row, tid % kBPieces);
                const int64_t step = (int64_t)kBStep * L.n * 2;
                const char* from = mat;
                if (rank > 0) {
#pragma unroll
                    for (int p = 0; p < (RP + kBStep - 1) / kBStep; ++p) {
                        const bool take = b_col < L.n && b_row + p * kBStep < rank;
                        if (RP >= kBStep || b_row < RP)
                            copy16(b_to + p * kBStep * T::kBPitch, take ? from : reinterpret_cast<const char*>(x), take);
                        from += step;
                    }
                }
                mat += T::kBPitch;
                col += T::kOutCols;
            }
        }
        copies_commit();
    };

    const int m0 = (warp % T::kMTiles) * 16, side = warp / T::kMTiles;
    const bool live = m0 < count;
    // The tensor cores cut bits off a long sum: `sum` takes over what 8 steps of 16 have added.
    float acc[T::kNT][4] = {}, sum[T::kNT][4] = {};
    const auto take_over = [&] {
#pragma unroll
        for (int t = 0; t < T::kNT; ++t)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                sum[t][e] += acc[t][e];
                acc[t][e] = 0.0f;
            }
    };

    // h of the whole tile: this CTA's sums over its warps, all CTAs' over the cluster.
    const auto join = [&] {
        take_over();
        const int j0 = T::kNSplit == 2 ? side * T::kNT * 8 : 0;
        float4* const mine = reinterpret_cast<float4*>(slabs);
        const auto store = [&](float* to, bool add) {
#pragma unroll
            for (int t = 0; t < T::kNT; ++t)
#pragma unroll
                for (int e = 0; e < 4; e += 2) {
                    float2* const p = reinterpret_cast<float2*>(to + (m0 + lane / 4 + e * 4) * RP + j0 + t * 8 + (lane & 3) * 2);
                    const float2 had = add ? *p : make_float2(0.0f, 0.0f);
                    *p = make_float2(had.x + sum[t][e], had.y + sum[t][e + 1]);
                }
        };
        if constexpr (MT == 16) {
            store(reinterpret_cast<float*>(slabs + side * T::kSlabBytes), false);
            __syncthreads();
            for (int i = tid; i < MT * RP / 4; i += kThreads) {
                float4 s = mine[i];
#pragma unroll
                for (int w = 1; w < T::kSlabs; ++w) {
                    const float4 v = mine[w * (MT * RP / 4) + i];
                    s.x += v.x, s.y += v.y, s.z += v.z, s.w += v.w;
                }
                mine[i] = s;
            }
        } else {
            float* const to = reinterpret_cast<float*>(slabs);
            if (T::kSlabs == 1 || side == 0) store(to, false);
            __syncthreads();
            if (T::kSlabs == 2 && side == 1) store(to, true);
        }
        __syncthreads();
        if (ctas > 1) {
            cluster_arrive();
            cluster_wait();
        }
        const uint32_t at = smem_u32(slabs);
        for (int i = tid; i < MT * RP / 4; i += kThreads) {
            float4 s = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
            if (ctas > 1) {
                float4 v[kMaxCluster];
#pragma unroll
                for (int c = 0; c < kMaxCluster; ++c)
                    if (c < ctas) v[c] = cluster_ld4(at + 16 * i, (uint32_t)c);
#pragma unroll
                for (int c = 0; c < kMaxCluster; ++c)
                    if (c < ctas) s.x += v[c].x, s.y += v[c].y, s.z += v[c].z, s.w += v[c].w;
            } else {
                s = mine[i];
            }
            const int row = i / (RP / 4), j = i % (RP / 4) * 4;
            const float h[4] = {j < rank ? s.x * scale : 0.0f, j + 1 < rank ? s.y * scale : 0.0f,  // (x may hold NaN)
                                j + 2 < rank ? s.z * scale : 0.0f, j + 3 < rank ? s.w * scale : 0.0f};
            __nv_bfloat16 p[4][T::kParts];
#pragma unroll
            for (int e = 0; e < 4; ++e) split<T::kParts>(h[e], p[e]);
#pragma unroll
            for (int q = 0; q < T::kParts; ++q) {
                __nv_bfloat162 two[2] = {__halves2bfloat162(p[0][q], p[1][q]), __halves2bfloat162(p[2][q], p[3][q])};
                *reinterpret_cast<uint2*>(parts + q * T::kPartBytes + row * T::kHPitch + j * 2) = *reinterpret_cast<const uint2*>(two);
            }
            if (L.h != nullptr && blockIdx.y == 0 && row % ctas == (int)cta && rows[row] >= 0)
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    if (j + e < L.r) L.h[(size_t)rows[row] * L.r + j + e] = h[e];
        }
        __syncthreads();
        if (ctas > 1) cluster_arrive();  // (waited for at the end: no CTA leaves while another reads its sums)
    };

#pragma unroll
    for (int i = 0; i < T::kStages - 1; ++i) issue(i);
    for (int i = 0; i < nk + nn; ++i) {
        copies_wait<T::kStages - 2>();
        __syncthreads();
        issue(i + T::kStages - 1);
        const int stage = (i % T::kStages) * T::kStage;
        const uint32_t first = smem0 + stage, second = first + MT * kChunk;
        if (i < nk) {
            if (live) {
                constexpr int kSteps = T::kCols / 16, kMySteps = kSteps / T::kSlabs;
#pragma unroll
                for (int u = 0; u < kMySteps; ++u) {
                    const int ks = T::kSlabs > 1 ? side * kMySteps + u : u;
                    uint32_t xa[4];
                    ldmatrix4(xa, first + place<kChunk>(m0 + (lane & 15), ks * 2 + (lane >> 4)));
#pragma unroll
                    for (int t = 0; t < T::kNT; t += 2) {
                        uint32_t w[4];
                        const int j0 = (T::kNSplit == 2 ? side * T::kNT : 0) * 8 + t * 8;
                        ldmatrix4(w, second + place<kChunk>(j0 + (lane & 7) + ((lane >> 4) << 3), ks * 2 + ((lane >> 3) & 1)));
                        mma(acc[t], xa, w[0], w[1]);
                        mma(acc[t + 1], xa, w[2], w[3]);
                    }
                }
                if (MT > 16 || (i & 7) == 7) take_over();
            }
            continue;
        }
        if (i == nk && rank > 0) join();
        if (live) {
            float o[T::kOT][4];
            const int c0 = side * T::kOT * 8;  // this warp's first column in the chunk
            unsigned char* const tile = smem + stage;
            constexpr int kPer = 16 / (int)sizeof(TY);
            const auto at = [&](int t, int e) -> unsigned char* {  // of o[t][e] and the next one
                const int row = m0 + lane / 4 + e * 4, c = c0 + t * 8 + (lane & 3) * 2;
                return tile + place<kChunk>(row, c / kPer) + c % kPer * (int)sizeof(TY);
            };
            // sums for bf16 begin with y; fp32 ones add it last, as the tensor cores cut bits off a long sum
#pragma unroll
            for (int t = 0; t < T::kOT; ++t)
#pragma unroll
                for (int e = 0; e < 4; e += 2) {
                    const uint32_t v = sizeof(TY) == 2 ? *reinterpret_cast<const uint32_t*>(at(t, e)) : 0u;
                    o[t][e] = bf16lo(v);
                    o[t][e + 1] = bf16hi(v);
                }
            if (rank > 0) {
#pragma unroll
                for (int ks = 0; ks < RP / 16; ++ks) {
                    uint32_t h[T::kParts][4];
#pragma unroll
                    for (int q = 0; q < T::kParts; ++q)
                        ldmatrix4(h[q], parts0 + q * T::kPartBytes + (m0 + (lane & 15)) * T::kHPitch + ks * 32 + (lane >> 4) * 16);
                    const int j = ks * 16 + (lane & 15);
                    if constexpr (T::kOT == 1) {
                        uint32_t w[2];
                        ldmatrix2_t(w, second + place<T::kBPitch>(j, c0 / 8));
#pragma unroll
                        for (int q = T::kParts - 1; q >= 0; --q) mma(o[0], h[q], w[0], w[1]);
                    } else {
#pragma unroll
                        for (int t = 0; t < T::kOT; t += 2) {
                            uint32_t w[4];
                            ldmatrix4_t(w, second + place<T::kBPitch>(j, c0 / 8 + t + (lane >> 4)));
#pragma unroll
                            for (int q = T::kParts - 1; q >= 0; --q) {
                                mma(o[t], h[q], w[0], w[1]);
                                mma(o[t + 1], h[q], w[2], w[3]);
                            }
                        }
                    }
                }
            }
#pragma unroll
            for (int t = 0; t < T::kOT; ++t)
#pragma unroll
                for (int e = 0; e < 4; e += 2) {
                    if constexpr (sizeof(TY) == 2) {
                        *reinterpret_cast<__nv_bfloat162*>(at(t, e)) = __floats2bfloat162_rn(o[t][e], o[t][e + 1]);
                    } else {
                        float2* const p = reinterpret_cast<float2*>(at(t, e));
                        *p = make_float2(p->x + o[t][e], p->y + o[t][e + 1]);
                    }
                }
            __syncwarp();
            constexpr int kSeg = T::kOT * 8 / kPer;  // 16-byte pieces of a row of this warp
            const int col0 = (n0 + i - nk) * T::kOutCols;
#pragma unroll
            for (int p = lane; p < 16 * kSeg; p += kWarp) {
                const int row = m0 + p / kSeg, c = c0 / kPer + p % kSeg, to = col0 + c * kPer;
                if (rows[row] >= 0 && to < L.n)
                    *reinterpret_cast<uint4*>(out + rows[row] * L.ldo + to) = *reinterpret_cast<const uint4*>(tile + place<kChunk>(row, c));
            }
        }
    }
    if (rank > 0) {
        if (nn == 0) join();
        if (ctas > 1) cluster_wait();
    }
}

// ---------------------------------------------------------------------------
// gradients
// ---------------------------------------------------------------------------
// A CTA has 128 columns of x; the rows of an adapter come in chunks of 64. h is the transposed operand and is split into
// three bf16 numbers, x is exact in bf16 (e4m3 rows too: the scale that 128 of their columns share is multiplied into h).
constexpr int kGradCols = 128, kGradRows = 64;
constexpr int kIdRing = 8;

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

// Whether an adapter's rows are shared by the CTAs of a cluster: where one CTA would have more than twice the even share.
__device__ __forceinline__ bool shared_rows(int count, int even) { return count > max(2 * even, kGradRows); }

// First entry of adapter `id` in the list, and their number.
__device__ __forceinline__ int2 entries(const AdapterGradsLaunch& L, int id) {
    const int begin = min(max(L.offsets[id], 0), L.rows);
    return make_int2(begin, min(max(L.offsets[id + 1], begin), L.rows) - begin);
}

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

    // The sums over entries begin .. begin + count - 1 of the list, of which `mine` are this CTA's; shared: the cluster's CTAs
    // join theirs.
    const auto sums = [&](int id, int begin, int count, bool join) {
        const int chunks = (count + kGradRows - 1) / kGradRows, parties = join ? ctas : 1, me = join ? (int)cta : 0;
        const int c0 = (int)((long long)chunks * me / parties), nc = (int)((long long)chunks * (me + 1) / parties) - c0;
        const int first = begin + c0 * kGradRows, end = begin + count;
        const auto listed = [&](int i) {
            const int at = first + i * kGradRows + tid;
            const int row = tid < kGradRows && i < nc && at < end ? L.list[at] : -1;
            return (unsigned)row < (unsigned)L.rows ? row : -1;
        };
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
            next = listed(i);
            if (tid < kGradRows) ids[i][tid] = next;
        }
        next = listed(G::kStages);
        __syncthreads();
#pragma unroll
        for (int i = 0; i < G::kStages - 1; ++i) issue(i);
        const int mg = warp % G::kMGroups, n0 = warp / G::kMGroups * G::kNT * 8;
        for (int i = 0; i < nc; ++i) {
            copies_wait<G::kStages - 2>();
            __syncthreads();
            if (tid < kGradRows) ids[(i + G::kStages) % kIdRing][tid] = next;
            next = listed(i + G::kStages + 1);
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
                __nv_bfloat16 q[4][3];
                split<3>(v.x, q[0]);
                split<3>(v.y, q[1]);
                split<3>(v.z, q[2]);
                split<3>(v.w, q[3]);
#pragma unroll
                for (int t = 0; t < 3; ++t) {
                    __nv_bfloat162 two[2] = {__halves2bfloat162(q[0][t], q[1][t]), __halves2bfloat162(q[2][t], q[3][t])};
                    *reinterpret_cast<uint2*>(parts + t * G::kPartBytes + row * G::kHPitch + j * 2) = *reinterpret_cast<const uint2*>(two);
                }
            }
            if constexpr (E8) {
#pragma unroll
                for (int p = tid; p < kGradRows * kGradCols / 16; p += kThreads) {
                    const int row = p / (kGradCols / 16), c = p % (kGradCols / 16) * 2;
                    const uint4 v = reinterpret_cast<const uint4*>(stage)[p];
                    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
                    uint32_t b[8];
#pragma unroll
                    for (int e = 0; e < 8; ++e) {
                        const __half2_raw f = __nv_cvt_fp8x2_to_halfraw2((__nv_fp8x2_storage_t)(w[e / 2] >> 16 * (e & 1)), __NV_E4M3);
                        const __nv_bfloat162 t = __float22bfloat162_rn(__half22float2(*reinterpret_cast<const __half2*>(&f)));
                        b[e] = *reinterpret_cast<const uint32_t*>(&t);
                    }
                    *reinterpret_cast<uint4*>(wide + place<kChunk>(row, c)) = make_uint4(b[0], b[1], b[2], b[3]);
                    *reinterpret_cast<uint4*>(wide + place<kChunk>(row, c + 1)) = make_uint4(b[4], b[5], b[6], b[7]);
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
        __syncthreads();
        cluster_arrive();
        cluster_wait();
        constexpr int kQuads = RP * kGradCols / 4;
        for (int p = (int)cta * kThreads + tid; p < kQuads; p += kThreads * ctas) {
            const int j = p / (kGradCols / 4), col = col0 + p % (kGradCols / 4) * 4;
            if (j >= L.r || col >= L.k) continue;
            float4 v[kMaxCluster];
#pragma unroll
            for (int c = 0; c < kMaxCluster; ++c)
                if (c < ctas) v[c] = cluster_ld4(smem0 + 16 * p, (uint32_t)c);
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
    };

    // Adapters whose rows are shared go round by cluster, the others by CTA: thread t looks at adapter t, and the masks say
    // which ones are this CTA's.
    __shared__ unsigned bigs[kWarps], smalls[kWarps];
    const int count_of_mine = tid < L.n_adapters ? entries(L, tid).y : 0;
    const bool big = ctas > 1 && shared_rows(count_of_mine, even);
    const bool small = tid < L.n_adapters && !big && !(count_of_mine == 0 && L.accumulate);
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
    for (int w = 0; w < kWarps; ++w)
        for (unsigned m = bigs[w]; m != 0u; m &= m - 1u) {
            const int id = w * kWarp + __ffs(m) - 1;
            const int2 of = entries(L, id);
            sums(id, of.x, of.y, true);
        }
    for (int w = 0; w < kWarps; ++w)
        for (unsigned m = smalls[w]; m != 0u; m &= m - 1u) {
            const int id = w * kWarp + __ffs(m) - 1;
            const int2 of = entries(L, id);
            sums(id, of.x, of.y, false);
        }
}

template <int MT, int RP, typename TY>
cudaError_t launch_tiles(const AdaptLaunch& a, long long tiles, int ctas, cudaStream_t stream) {
    // Few tiles: several clusters have one, each with its own h and a part of the columns, of 2 chunks a CTA at least.
    const long long chunks = (a.n + Tile<MT, RP, TY>::kOutCols - 1) / Tile<MT, RP, TY>::kOutCols;
    long long sharing = a.out != nullptr ? kResidentCtas / (tiles * ctas) : 1;
    if (sharing > chunks / (2 * ctas)) sharing = chunks / (2 * ctas);
    if (sharing < 1) sharing = 1;
    const auto kernel = k_adapt<MT, RP, TY>;
    constexpr int kSmem = Tile<MT, RP, TY>::kSmem;
    const cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kSmem);
    if (e != cudaSuccess) return e;
    cudaLaunchConfig_t cfg = launch_shape(dim3((unsigned)(tiles * ctas), (unsigned)sharing), kThreads, stream);
    cfg.dynamicSmemBytes = kSmem;
    cudaLaunchAttribute at[2]{};
    at[0].id = cudaLaunchAttributeClusterDimension;
    at[0].val.clusterDim = {(unsigned)ctas, 1, 1};
    at[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at[1].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = at;
    cfg.numAttrs = 2;
    return cudaLaunchKernelEx(&cfg, kernel, a, ctas);
}

template <int MT, typename TY>
cudaError_t launch_rank(const AdaptLaunch& a, long long tiles, int ctas, cudaStream_t stream) {
    if (a.r <= 16) return launch_tiles<MT, 16, TY>(a, tiles, ctas, stream);
    if (a.r <= 32) return launch_tiles<MT, 32, TY>(a, tiles, ctas, stream);
    if (a.r <= 64) return launch_tiles<MT, 64, TY>(a, tiles, ctas, stream);
    return launch_tiles<MT, 128, TY>(a, tiles, ctas, stream);
}

template <typename TY>
cudaError_t launch_type(const AdaptLaunch& a, cudaStream_t stream) {
    if (a.list == nullptr) return launch_rank<16, TY>(a, a.rows, kMaxCluster, stream);
    const bool small = a.rows < 512 || a.rows / a.n_adapters <= 24;
    if (!small && a.r <= kWideRank) return launch_adapt_wide(a, sizeof(TY) == 4, stream);
    const int mt = small ? 16 : 64;
    int ctas = kMaxCluster;
    while (ctas > 1 && a.rows / mt * ctas > 2 * kResidentCtas) ctas /= 2;
    const long long tiles = most_tiles(a.rows, a.n_adapters, mt);
    return small ? launch_rank<16, TY>(a, tiles, ctas, stream) : launch_tiles<64, 128, TY>(a, tiles, ctas, stream);
}

template <int RP, bool E8>
cudaError_t launch_grads(const AdapterGradsLaunch& a, cudaStream_t stream) {
    const auto kernel = k_adapter_grads<RP, E8>;
    constexpr int kSmem = Grads<RP, E8>::kSmem;
    const cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kSmem);
    if (e != cudaSuccess) return e;
    // about two rounds of CTAs, in clusters of 8: fewer where there are no more adapters or chunks than that
    const int blocks = (a.k + kGradCols - 1) / kGradCols;
    int ctas = kMaxCluster;
    while (ctas > 1 && (long long)ctas * kGradRows / 2 >= a.rows) ctas /= 2;
    const int wish = (kResidentCtas * 2 + blocks * ctas - 1) / (blocks * ctas);
    const int ys = wish < a.n_adapters ? wish : a.n_adapters;
    const int even = (int)((long long)a.rows * blocks / kResidentCtas);
    cudaLaunchConfig_t cfg = launch_shape(dim3((unsigned)(blocks * ctas), (unsigned)ys), kThreads, stream);
    cfg.dynamicSmemBytes = kSmem;
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
cudaError_t launch_grads_rank(const AdapterGradsLaunch& a, cudaStream_t stream) {
    if (a.r <= 16) return launch_grads<16, E8>(a, stream);
    if (a.r <= 32) return launch_grads<32, E8>(a, stream);
    if (a.r <= 64) return launch_grads<64, E8>(a, stream);
    return launch_grads<128, E8>(a, stream);
}

}  // namespace

cudaError_t launch_adapt(const AdaptLaunch& a, bool y_f32, cudaStream_t stream) {
    return y_f32 ? launch_type<float>(a, stream) : launch_type<__nv_bfloat16>(a, stream);
}

cudaError_t launch_adapter_grads(const AdapterGradsLaunch& a, bool e4m3, cudaStream_t stream) {
    return e4m3 ? launch_grads_rank<true>(a, stream) : launch_grads_rank<false>(a, stream);
}

}  // namespace tsffn
