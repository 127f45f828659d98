// ts_adapt.cu -- low-rank adapters of many requests beside a shared projection: h[t] = s_i x[t] A_i^T and
// out[t] = y[t] + h[t] B_i for the adapter i of row t (ts_adapt_rows), of few rows or ranks above 64; ts_adapt_wide.cu has
// the others. With A and B exchanged it is also the backward pass by rows.
//
// Both products in one launch. A cluster of CTAs has a tile of up to 16 or 64 rows of one adapter: each CTA sums its part
// of k for the whole tile, the parts of h meet through distributed shared memory, summed in the same order by all, and each
// CTA adds h B_i to its part of the columns. One ring of chunks, 256 to 1024 bytes of each row wide, carries x and A_i and
// then y and B_i: while h is being joined the first chunks of y are already on their way. Rows of a tile are gathered (by
// a list, or by the rows' ids here), so they come by 16-byte asynchronous copies.
//
// Few rows are bound by the chain launch / ids / first chunk / sums of h / join / last chunk, not by bytes. Calls in a row,
// bf16 unless stated: 1 row, k = 4096, n = 14336, r = 16: 5.4 us; 64 rows of 64 adapters, k = n = 4096, r = 16, fp32: 9.5
// (12.5 MB, 1.3 TB/s; in chunks of 256 bytes 14.0); 300 rows of 20, k = 1408, n = 512, r = 40, fp32: 7.4. The matrix
// instructions of a warp do for it: they take 3% of the time.
#include "ts_adapt.cuh"
#include "ts_grouped.h"

namespace tsffn {
namespace {

// ---------------------------------------------------------------------------
// h and out
// ---------------------------------------------------------------------------
// MT: rows of a tile. RP: r rounded up to 16, 32, 64 or 128. CHUNK: bytes of a row in a chunk.
template <int MT, int RP, int CHUNK, typename TY>
struct Tile {
    static constexpr int kChunk = CHUNK;
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
    // the sums of h of this CTA (a slab for each warp that has a part of k), and h as bf16 numbers
    static constexpr int kFixed = kSlabs * kSlabBytes + kParts * kPartBytes;
    // two CTAs on an SM where two stages fit (the loads in flight of two cover the latency, and one works while the other joins)
    static constexpr int kHalf = 113 * 1024 - kFixed, kWhole = 226 * 1024 - kFixed;
    static constexpr int kWish = MT == 16 ? 6 : 4;
    static constexpr int kFit = kHalf >= 2 * kStage ? kHalf / kStage : kWhole / kStage;
    static constexpr int kStages = kFit < kWish ? kFit : kWish;
    static constexpr int kSmem = kStages * kStage + kFixed;
    static constexpr int kCtas = kSmem <= 113 * 1024 && RP <= 64 ? 2 : 1;  // on an SM
    static_assert(kStages >= 2 && kOT % 2 == 0 && (MT == 16 || kSlabs == 1), "");
};

// Without a list, of up to 512 rows: the same tiles, from the rows' ids. Thread t looks at rows 2 t and 2 t + 1.
template <int MT>
__device__ __forceinline__ void find_few(const AdaptLaunch& L, int tile, TileRows* found, int* rows) {
    static_assert(kFewRows == 2 * kThreads, "");
    __shared__ int counts[kMaxAdapters + 1], sums[kWarps];
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    int id[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const int row = 2 * tid + i;
        id[i] = row < L.rows ? (int)min((unsigned)L.ids[row], (unsigned)L.n_adapters) : -1;
    }
    counts[tid] = 0;
    if (tid == 0) *found = {-1, 0, 0};
    if (tid < MT) rows[tid] = -1;
    __syncthreads();
#pragma unroll
    for (int i = 0; i < 2; ++i)
        if (id[i] >= 0) atomicAdd(&counts[id[i]], 1);
    __syncthreads();
    const int tiles = (counts[tid] + MT - 1) / MT;
    int upto = tiles;
#pragma unroll
    for (int o = 1; o < kWarp; o <<= 1) {
        const int v = __shfl_up_sync(0xffffffffu, upto, o);
        if (lane >= o) upto += v;
    }
    if (lane == kWarp - 1) sums[warp] = upto;
    __syncthreads();
    for (int w = 0; w < warp; ++w) upto += sums[w];
    if (tile < upto && tile >= upto - tiles) {
        const int first = (tile - (upto - tiles)) * MT;
        *found = {tid, first, min(MT, counts[tid] - first)};
    }
    __syncthreads();
    // its rows, ascending: those of the warps before, of the lanes before, the thread's own
    const int mine = found->id, n = (id[0] == mine) + (id[1] == mine);
    const unsigned one = __ballot_sync(0xffffffffu, n >= 1), two = __ballot_sync(0xffffffffu, n == 2);
    const unsigned before = (1u << lane) - 1u;
    int at = __popc(one & before) + __popc(two & before);
    if (lane == 0) sums[warp] = __popc(one) + __popc(two);
    __syncthreads();
    for (int w = 0; w < warp; ++w) at += sums[w];
    at -= found->first;
#pragma unroll
    for (int i = 0; i < 2; ++i)
        if (id[i] == mine && mine >= 0) {
            if (at >= 0 && at < MT) rows[at] = 2 * tid + i;
            ++at;
        }
}

template <int MT, int RP, int CHUNK, typename TY>
__global__ void __launch_bounds__(kThreads, Tile<MT, RP, CHUNK, TY>::kCtas) k_adapt(const __grid_constant__ AdaptLaunch L, int ctas) {
    using T = Tile<MT, RP, CHUNK, TY>;
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
    constexpr int kPieces = T::kChunk / 16, kRowStep = kThreads / kPieces, kMine = MT / kRowStep;
    const int piece = tid % kPieces, row0 = tid / kPieces;
    const uint32_t to0 = smem0 + place<T::kChunk>(row0, piece);
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
    const auto flip = [](int step) { return (uint32_t)(step & 4) << 4; };  // (a row 4 further on has its pieces permuted another way)
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
                if (there[p]) copy16((to ^ flip(p * kRowStep)) + p * kRowStep * T::kChunk, in ? src[p] : reinterpret_cast<const char*>(x), in);
                src[p] += T::kChunk;
            }
            if (i < nk) {
                const int64_t step = (int64_t)kRowStep * L.k * 2;
                const char* from = mat;
#pragma unroll
                for (int p = 0; p < RP / kRowStep; ++p) {
                    const bool take = in && row0 + p * kRowStep < rank;
                    copy16((to ^ flip(p * kRowStep)) + (MT + p * kRowStep) * T::kChunk, take ? from : reinterpret_cast<const char*>(x), take);
                    from += step;
                }
                mat += T::kChunk;
                col += T::kCols;
            } else {
                constexpr int kBPieces = T::kBPitch / 16, kBStep = kThreads / kBPieces;
                const int b_row = tid / kBPieces, b_col = col - piece * (16 / (int)sizeof(TY)) + tid % kBPieces * 8;
                const uint32_t b_to = smem0 + (uint32_t)(i % T::kStages) * T::kStage + MT * T::kChunk + place<T::kBPitch>(b_row, tid % kBPieces);
                const int64_t step = (int64_t)kBStep * L.n * 2;
                const char* from = mat;
                if (rank > 0) {
#pragma unroll
                    for (int p = 0; p < (RP + kBStep - 1) / kBStep; ++p) {
                        const bool take = b_col < L.n && b_row + p * kBStep < rank;
                        if (RP >= kBStep || b_row < RP)
                            copy16((b_to ^ flip(p * kBStep)) + p * kBStep * T::kBPitch, take ? from : reinterpret_cast<const char*>(x), take);
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
        float* const to = reinterpret_cast<float*>(slabs + (MT == 16 ? side * T::kSlabBytes : 0));
#pragma unroll
        for (int t = 0; t < T::kNT; ++t)
#pragma unroll
            for (int e = 0; e < 4; e += 2)
                *reinterpret_cast<float2*>(to + (m0 + lane / 4 + e * 4) * RP + j0 + t * 8 + (lane & 3) * 2) = make_float2(sum[t][e], sum[t][e + 1]);
        __syncthreads();
        if constexpr (MT == 16) {
            for (int i = tid; i < MT * RP / 4; i += kThreads) {
                float4 s = mine[i];
#pragma unroll
                for (int w = 1; w < T::kSlabs; ++w) {
                    const float4 v = mine[w * (MT * RP / 4) + i];
                    s.x += v.x, s.y += v.y, s.z += v.z, s.w += v.w;
                }
                mine[i] = s;
            }
            __syncthreads();
        }
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
        const uint32_t first = smem0 + stage, second = first + MT * T::kChunk;
        if (i < nk) {
            if (live) {
                constexpr int kSteps = T::kCols / 16, kMySteps = kSteps / T::kSlabs;
#pragma unroll
                for (int u = 0; u < kMySteps; ++u) {
                    const int ks = T::kSlabs > 1 ? side * kMySteps + u : u;
                    uint32_t xa[4];
                    ldmatrix4(xa, first + place<T::kChunk>(m0 + (lane & 15), ks * 2 + (lane >> 4)));
#pragma unroll
                    for (int t = 0; t < T::kNT; t += 2) {
                        uint32_t w[4];
                        const int j0 = (T::kNSplit == 2 ? side * T::kNT : 0) * 8 + t * 8;
                        ldmatrix4(w, second + place<T::kChunk>(j0 + (lane & 7) + ((lane >> 4) << 3), ks * 2 + ((lane >> 3) & 1)));
                        mma(acc[t], xa, w[0], w[1]);
                        mma(acc[t + 1], xa, w[2], w[3]);
                    }
                }
                if (MT > 16 || (i + 1) % (8 / kMySteps) == 0) take_over();
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
                return tile + place<T::kChunk>(row, c / kPer) + c % kPer * (int)sizeof(TY);
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
            if (rank > 0) {  // (without an adapter y goes out as it came)
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
            }
            __syncwarp();
            constexpr int kSeg = T::kOT * 8 / kPer;  // 16-byte pieces of a row of this warp
            const int col0 = (n0 + i - nk) * T::kOutCols;
#pragma unroll
            for (int p = lane; p < 16 * kSeg; p += kWarp) {
                const int row = m0 + p / kSeg, c = c0 / kPer + p % kSeg, to = col0 + c * kPer;
                if (rows[row] >= 0 && to < L.n)
                    *reinterpret_cast<uint4*>(out + rows[row] * L.ldo + to) = *reinterpret_cast<const uint4*>(tile + place<T::kChunk>(row, c));
            }
        }
    }
    if (rank > 0) {
        if (nn == 0) join();
        if (ctas > 1) cluster_wait();
    }
}

template <int MT, int RP, int CHUNK, typename TY>
cudaError_t launch_tiles(const AdaptLaunch& a, long long tiles, cudaStream_t stream) {
    using T = Tile<MT, RP, CHUNK, TY>;
    // A large cluster has less of a row's bytes in each CTA, but takes longer to find its place beside others. 300 rows of 20
    // adapters, k = 1408, n = 512, clusters of 8 and of 4: r = 64, fp32 9.7 and 8.1 us, r = 16, bf16 6.3 and 5.9; k = n = 4096, 32 rows
    // of 32, r = 16, bf16 5.8 and 7.1; and alone on their SMs, 100 rows of 10, k = 2048, n = 1408, r = 32, bf16 6.2 and 6.8.
    constexpr int kResident = kSms * T::kCtas;
    const long long row_bytes = 2ll * a.k + (a.out != nullptr ? (long long)a.n * (int)sizeof(TY) : 0);
    int ctas = kMaxCluster;
    while (ctas > 1 && (tiles * ctas > kResident + kResident / 8 || (tiles * ctas > kSms && row_bytes < 900 * ctas))) ctas /= 2;
    // Few tiles: several clusters have one, each with its own h and a part of the columns, of a chunk a CTA at least.
    const long long n_chunks = a.out != nullptr ? (a.n + T::kOutCols - 1) / T::kOutCols : 0;
    long long sharing = kResident / (tiles * ctas);
    if (sharing > n_chunks / ctas) sharing = n_chunks / ctas;
    if (sharing < 1) sharing = 1;
    const auto kernel = k_adapt<MT, RP, CHUNK, TY>;
    const cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, T::kSmem);
    if (e != cudaSuccess) return e;
    cudaLaunchConfig_t cfg = launch_shape(dim3((unsigned)(tiles * ctas), (unsigned)sharing), kThreads, stream);
    cfg.dynamicSmemBytes = T::kSmem;
    cudaLaunchAttribute at[2]{};
    at[0].id = cudaLaunchAttributeClusterDimension;
    at[0].val.clusterDim = {(unsigned)ctas, 1, 1};
    at[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at[1].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = at;
    cfg.numAttrs = 2;
    return cudaLaunchKernelEx(&cfg, kernel, a, ctas);
}

template <typename TY>
cudaError_t launch_few(const AdaptLaunch& a, cudaStream_t stream) {
    // The wider chunks the better, as each costs the warps a round of latencies, down to two stages of them and up to what leaves
    // each CTA one at least. Microseconds, k = n = 4096: r = 16, chunks of 512 bytes and of 1024, 64 rows of 64 adapters, fp32, 11.0
    // and 9.6, 4 of 4, bf16 5.6 and 5.8 (1 row, n = 14336, 5.6 and 6.4); r = 64, of 256 (two CTAs on an SM), 512 (one) and 1024,
    // 32 of 32, bf16 14.5, 10.7 and 9.9, 1 row 8.7, 7.7 and 8.1; r = 128, of 256 and 512, 256 rows of 8, fp32 24.6 and 18.5. r = 32 has
    // its best with two CTAs: 8 of 8, bf16 6.4, and 6.6 with one and chunks of 1024.
    const long long tiles = most_tiles(a.rows, a.n_adapters, 16);
    const bool wide = tiles >= 8 && 2ll * a.k + (long long)a.n * (int)sizeof(TY) >= 8192;
    if (a.r <= 16) return wide ? launch_tiles<16, 16, 1024, TY>(a, tiles, stream) : launch_tiles<16, 16, 512, TY>(a, tiles, stream);
    if (a.r <= 32) return launch_tiles<16, 32, 512, TY>(a, tiles, stream);
    if (a.r <= 64) return wide ? launch_tiles<16, 64, 1024, TY>(a, tiles, stream) : launch_tiles<16, 64, 512, TY>(a, tiles, stream);
    return launch_tiles<16, 128, 512, TY>(a, tiles, stream);
}

template <typename TY>
cudaError_t launch_type(const AdaptLaunch& a, cudaStream_t stream) {
    // Tiles of 16 rows begin sooner, and read A and B 8 times as often. By the time of a tile, in 2 ns: 30 + r of 16 rows, 210 of 128 after
    // 6000 (r above 64: 340 of 64 after 4000). n = k = 4096, bf16, microseconds with the list's 6, 16 rows and 128, of 4, 30 and 100
    // adapters: r = 8, 4096 rows 27, 28, 30 and 32, 39, 63; 8192 50, 51, 52 and 47, 65, 74. r = 32, 2048 rows 23, 23, 37 and
    // 24, 31, 62; 4096 36, 37, 41 and 33, 41, 65; 8192 65, 66, 70 and 48, 67, 76. r = 64, 1024 rows 18, 26, 36 and 26, 33, 63;
    // 4096 53, 57, 61 and 37, 46, 71; 8192 102, 103, 106 and 52, 73, 85. r = 128 (and 64 rows), 1024 rows 26, 45, 55 and 50, 57, 101;
    // 4096 84, 88, 96 and 59, 102, 104; 8192 160, 165, 170 and 103, 103, 190. n = 2048, k = 1408, fp32 has the same order. The host
    // knows how many adapters there are, not how many have rows: of large pools of which few are hit it takes 16 rows too long (8192
    // rows of one adapter of 255, r = 64, about twice the time), and of r = 128 it takes 64 rows at 4096 of 30 and 8192 of 100, for 16% and 12%.
    const long long few = most_tiles(a.rows, a.n_adapters, 16) * (30 + a.r);
    const bool wide = a.r <= kWideRank;
    const long long many = wide ? 6000 + 210 * most_tiles(a.rows, a.n_adapters, 128) : 4000 + 340 * most_tiles(a.rows, a.n_adapters, 64);
    if (a.list == nullptr || few <= many) return launch_few<TY>(a, stream);
    if (wide) return launch_adapt_wide(a, sizeof(TY) == 4, stream);
    return launch_tiles<64, 128, 256, TY>(a, most_tiles(a.rows, a.n_adapters, 64), stream);
}

}  // namespace

cudaError_t launch_adapt(const AdaptLaunch& a, bool y_f32, cudaStream_t stream) {
    return y_f32 ? launch_type<float>(a, stream) : launch_type<__nv_bfloat16>(a, stream);
}

}  // namespace tsffn
