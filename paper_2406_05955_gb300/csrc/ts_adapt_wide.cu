// ts_adapt_wide.cu -- ts_adapt_rows over many rows (a list, r up to 64): tiles of 128 rows of one adapter on the tensor cores.
//
// The tile's cluster shares k and the columns as in ts_adapt.cu. A CTA's items are chunks 256 bytes of each row wide: of x and
// A_i, whose products are summed in tensor memory, and then of y and B_i. h is the M operand of the second product, as 2 (bf16
// rows) or 3 (fp32) bf16 numbers in shared memory, and a row of its products is a lane of tensor memory: so a thread has a row of
// an item to itself. It fetches it by one bulk copy into a row of shared memory and adds to it in place; its warp writes the
// 32 rows, two at a time.
//
// Sixteen warps, four an item, take items of y in turn (and copy x, 16 bytes at a time, in the order the tensor cores want), four
// copy A and B, one issues the products. They wait for one another by barriers in shared memory only.
//
// Memory bounds it where the tiles fill the device, latencies otherwise: a row of an item is fetched, added to and written
// in a chain that takes a warp 4700 cycles for 8 KB, so that many warps have to be at it. Measured on the way, 8192 rows,
// k = 4096, n = 14336, r = 64, bf16: eight warps that do everything, a CTA barrier an item, 130 us; sixteen so, or two CTAs
// of half the item, 130-140; a warp of its own for the products 122; a row a thread, bulk copies of 256 bytes both ways, two
// groups of warps with two items each 112 (a warp's 32 copies take 2000-2600 cycles to issue); of 512 bytes and one item 117;
// written by 16-byte stores 110; four groups with an item each 96 (4.9 TB/s; 5.6 while y is added to).
#include "ts_adapt.cuh"
#include "ts_grouped.h"

namespace tsffn {
namespace {

__device__ unsigned wide_timeouts;  // waits that gave up, ever

constexpr int kTileRows = 128;
constexpr int kGroup = kTileRows, kGroups = 4, kWorkers = kGroups * kGroup;  // threads that take items of y in turn
constexpr int kCarriers = 128;                            // that copy A and B
constexpr int kWideThreads = kWorkers + kCarriers + kWarp;
constexpr int kSlots = 4;                                 // items of rows: one of each group
constexpr int kPitch = kChunk + 16;                       // bytes from a row of y to the next: 8 rows' same piece lie in 8 banks
constexpr int kSlotBytes = kTileRows * kPitch;
static_assert(kSlots == kGroups && kSlotBytes % 1024 == 0 && kSlotBytes >= kTileRows * kChunk, "x starts on 1024 bytes");

template <int RP, typename TY>
struct Wide {
    static constexpr int kCols = kChunk / 2;                   // of x and A in an item
    static constexpr int kOutCols = kChunk / (int)sizeof(TY);  // of y and out
    static constexpr int kParts = sizeof(TY) == 2 ? 2 : 3;
    static constexpr int kMat = RP * kChunk;                   // of A or B in an item
    static constexpr int kMats = RP == 64 && kParts == 3 ? 2 : 3;
    static constexpr int kPart = kTileRows * 128;              // of h: 128 bytes a row, of which r take 2 r
    static constexpr int kSmem = 1024 + kSlots * kSlotBytes + kMats * kMat + kParts * kPart;
    static constexpr int kMine = RP / kGroups;                 // components of a thread's row
    static_assert(kTileRows * RP * 4 <= kParts * kPart, "the sums lie where h will");
};

template <int RP, typename TY>
__global__ void __launch_bounds__(kWideThreads, 1) k_adapt_wide(const __grid_constant__ AdaptLaunch L, int ctas) {
    using W = Wide<RP, TY>;
    extern __shared__ unsigned char raw[];
    __shared__ TileRows found;
    __shared__ int rows[kTileRows];
    __shared__ uint2 x_at[kTileRows];     // first byte of each row of x (none: the highest bit)
    __shared__ char* out_at[kTileRows];   // and of out (nullptr)
    __shared__ uint64_t come_x[kSlots], come_y[kSlots][kGroup / kWarp], come_mat[W::kMats];  // an item's copies
    __shared__ uint64_t done[kSlots];           // its products
    __shared__ uint64_t have_h, have_read[2];   // h as bf16 numbers; an item's products are in registers (two take turns)
    __shared__ uint32_t tmem;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const uint32_t cta = cluster_rank();
    unsigned char* const smem = raw + (-smem_u32(raw) & 1023u);
    unsigned char* const mats = smem + kSlots * kSlotBytes;
    unsigned char* const h_parts = mats + W::kMats * W::kMat;
    const uint32_t smem0 = smem_u32(smem), mats0 = smem_u32(mats), h0 = smem_u32(h_parts);
    pdl_wait();
    find_listed<kTileRows>(L, (int)(blockIdx.x / ctas), &found, rows);
    __syncthreads();
    const int id = found.id, count = found.count;
    if (id < 0) return;
    const bool some = id < L.n_adapters;
    const int rank = !some ? 0 : L.ranks != nullptr ? min(max(L.ranks[id], 0), L.r) : L.r;
    const float scale = some && L.scale != nullptr ? L.scale[id] : 1.0f;
    const __nv_bfloat16* const x = static_cast<const __nv_bfloat16*>(L.x);
    const __nv_bfloat16* const a = static_cast<const __nv_bfloat16*>(L.a) + (size_t)(some ? id : 0) * L.r * L.k;
    const __nv_bfloat16* const b = static_cast<const __nv_bfloat16*>(L.b) + (size_t)(some ? id : 0) * L.r * L.n;
    const TY* const y = static_cast<const TY*>(L.y);
    TY* const out = static_cast<TY*>(L.out);
    if (rank == 0) {
        if (L.h != nullptr && cta == 0 && blockIdx.y == 0)
            for (int i = tid; i < count * L.r; i += kWideThreads)
                if (rows[i / L.r] >= 0) L.h[(size_t)rows[i / L.r] * L.r + i % L.r] = 0.0f;
        if (out == y) return;  // (of both nullptr too)
    }
    if (tid < kTileRows) {
        const int row = rows[tid];
        const uint64_t at = row < 0 ? 1ull << 63 : (uint64_t)(row * L.ldx * 2);
        x_at[tid] = make_uint2((uint32_t)at, (uint32_t)(at >> 32));
        out_at[tid] = row < 0 ? nullptr : reinterpret_cast<char*>(out + row * L.ldo);
    }
    if (tid == 0) {
        for (int i = 0; i < kSlots; ++i) {
            mbar_init(&come_x[i], kWorkers);
            for (int q = 0; q < kGroup / kWarp; ++q) mbar_init(&come_y[i][q], 1);
            mbar_init(&done[i], 1);
        }
        for (int i = 0; i < W::kMats; ++i) mbar_init(&come_mat[i], kCarriers);
        mbar_init(&have_h, kWorkers);
        for (int i = 0; i < 2; ++i) mbar_init(&have_read[i], kGroup / kWarp);
        mbar_fence_init();
    }
    if (warp == 0 && rank > 0) tc_alloc<512>(&tmem);
    tc_before();
    __syncthreads();
    tc_after();
    // Tensor memory: sums of h over 256 of k, four in turn, and the two groups' products. What a sum was in is used again 8 items
    // later, which the rows' warps fetch after they have read it.
    const uint32_t t_h = rank > 0 ? tmem : 0, t_out = t_h + 256;

    const int k_chunks = rank > 0 ? (L.k + W::kCols - 1) / W::kCols : 0;
    const int n_chunks = out != nullptr ? (L.n + W::kOutCols - 1) / W::kOutCols : 0;
    const int k0 = (int)((long long)k_chunks * cta / ctas), nk = (int)((long long)k_chunks * (cta + 1) / ctas) - k0;
    const int all = ctas * (int)gridDim.y, me = (int)(blockIdx.y * ctas + cta);
    const int n0 = (int)((long long)n_chunks * me / all), nn = (int)((long long)n_chunks * (me + 1) / all) - n0;
    const int total = nk + nn;

    bool failed = false;
    const auto wait = [&](uint64_t* bar, unsigned parity) {
        if (!failed) failed = !mbar_wait(bar, parity);  // (after the first that gives up, none waits)
    };
    const auto products = [&](int i) { wait(&done[i & 3], i >> 2 & 1); };  // of item i

    if (warp >= (kWorkers + kCarriers) / kWarp) {
        // ---- the products -------------------------------------------------------------------------------------------
        int mat = 0, round = 0;
        for (int i = 0; i <= total && rank > 0; ++i) {
            if (i == nk) {
                if (ctas > 1) {  // the join's barriers are all threads'
                    for (int j = 0; j < 2; ++j) {
                        cluster_arrive();
                        cluster_wait();
                    }
                }
                wait(&have_h, 0);
            }
            if (i == total) break;
            if (i < nk) wait(&come_x[i & 3], i >> 2 & 1);
            else if (i >= nk + 2) wait(&have_read[i & 1], ((i - nk) / 2 - 1) & 1);
            wait(&come_mat[mat], round & 1);
            failed = __any_sync(0xffffffffu, failed);
            if (!failed) {
                fence_proxy_async_smem();
                tc_after();
                if (elect_one()) {
                    const uint32_t m = mats0 + mat * W::kMat, at = smem0 + (i & 3) * kSlotBytes;
                    if (i < nk) {
                        const uint32_t d = t_h + (i >> 1 & 3) * 64;
#pragma unroll
                        for (int ks = 0; ks < W::kCols / 16; ++ks)
                            tc_mma(d, desc_k(at + (ks >> 2) * (kTileRows * 128)) + 2 * (ks & 3), desc_k(m + (ks >> 2) * (RP * 128)) + 2 * (ks & 3),
                                   idesc(RP, false, false), (i & 1) != 0 || ks > 0);
                    } else {
#pragma unroll
                        for (int q = W::kParts - 1; q >= 0; --q)
#pragma unroll
                            for (int ks = 0; ks < RP / 16; ++ks)
                                tc_mma(t_out + (i & 1) * 128, desc_k(h0 + q * W::kPart) + 2 * ks, desc_n(m, RP * 128) + 128 * ks,
                                       idesc(W::kOutCols, false, true), q < W::kParts - 1 || ks > 0);
                    }
                    if (!(L.test_stall && i == total - 1)) tc_commit(&done[i & 3]);
                }
                __syncwarp();
            }
            if (++mat == W::kMats) mat = 0, ++round;
        }
    } else if (warp >= kWorkers / kWarp) {
        // ---- A and B ------------------------------------------------------------------------------------------------
        const int t = tid - kWorkers;
        constexpr int kAStep = kCarriers / 16, kBPieces = W::kOutCols / 8, kBStep = kCarriers / kBPieces;
        const int a_row = t / 16, a_piece = t % 16, b_row = t / kBPieces, b_piece = t % kBPieces;
        const uint32_t a_to = (a_piece >> 3) * (RP * 128), b_to = (b_piece >> 3) * (RP * 128);
        const int64_t a_step = (int64_t)kAStep * L.k * 2, b_step = (int64_t)kBStep * L.n * 2;
        // The join's barriers are all threads': the first is arrived at before the first part of B is copied, and waited for
        // before the first that comes after products of h.
        bool met = rank == 0 || ctas == 1;
        const auto meet = [&] {
            if (met) return;
            cluster_wait();
            cluster_arrive();
            cluster_wait();
            met = true;
        };
        int mat = 0;
        for (int i = 0; i < total && rank > 0; ++i) {
            if (i == nk && !met) cluster_arrive();
            if (i == nk + W::kMats) meet();
            if (i >= W::kMats) products(i - W::kMats);
            const uint32_t to = mats0 + mat * W::kMat;
            if (i < nk) {
                const int col = (k0 + i) * W::kCols + a_piece * 8;
                const bool in = col < L.k;
                const char* from = reinterpret_cast<const char*>(a + (size_t)a_row * L.k + (in ? col : 0));
#pragma unroll
                for (int j = 0; j < RP / kAStep; ++j) {
                    const int row = a_row + j * kAStep;
                    const bool take = in && row < rank;
                    copy16(to + a_to + place<128>(row, a_piece & 7), take ? from : reinterpret_cast<const char*>(a), take);
                    from += a_step;
                }
            } else {
                const int col = (n0 + i - nk) * W::kOutCols + b_piece * 8;
                const bool in = col < L.n;
                const char* from = reinterpret_cast<const char*>(b + (size_t)b_row * L.n + (in ? col : 0));
#pragma unroll
                for (int j = 0; j < RP / kBStep; ++j) {
                    const int row = b_row + j * kBStep;
                    const bool take = in && row < rank;
                    copy16(to + b_to + place<128>(row, b_piece & 7), take ? from : reinterpret_cast<const char*>(b), take);
                    from += b_step;
                }
            }
            copies_arrive(&come_mat[mat]);
            if (++mat == W::kMats) mat = 0;
        }
        if (total == nk && !met) cluster_arrive();
        meet();
    } else {
        // ---- rows ---------------------------------------------------------------------------------------------------
        const int group = warp >> 2, quarter = (warp & 3) * 32, mine = quarter + lane;  // this thread's row of the group's items
        const int row = rows[mine];
        const char* const y_row = reinterpret_cast<const char*>(y + (row < 0 ? 0 : row * L.ldy));
        const int there = __popc(__ballot_sync(0xffffffffu, row >= 0));
        const auto bytes = [&](int i) { return min(kChunk, (L.n - (n0 + i - nk) * W::kOutCols) * (int)sizeof(TY)); };  // of a row
        const auto at_col = [&](int i) { return (int64_t)(n0 + i - nk) * kChunk; };
        // x: a warp copies a fourth of 32 rows, 4 lanes a row
        const int piece = group * 4 + (lane & 3), x_row = quarter + (lane >> 2);
        const uint32_t x_to = (piece >> 3) * (kTileRows * 128) + place<128>(x_row, piece & 7);
        const auto fetch = [&](int i) {  // item i
            if (i >= total) return;
            if (i < nk) {
                const int col = (k0 + i) * W::kCols + piece * 8;
                const bool in = col < L.k;
                const char* const base = reinterpret_cast<const char*>(x + (in ? col : 0));
                const uint32_t to = smem0 + (i & 3) * kSlotBytes;
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const uint2 at = x_at[x_row + j * 8];
                    copy16(to + x_to + j * 8 * 128, base + ((uint64_t)(at.y & 0x7fffffffu) << 32 | at.x), in && (int)at.y >= 0);
                }
                copies_arrive(&come_x[i & 3]);
            } else if ((i & 3) == group) {
                uint64_t* const bar = &come_y[i & 3][warp & 3];
                const int n = bytes(i);
                if (i < nk + kSlots) fence_proxy_async_smem();  // (x was there)
                if (lane == 0) mbar_arrive_expect_tx(bar, (unsigned)(there * n));
                __syncwarp();
                if (row >= 0) tma_load_1d(smem + (i & 3) * kSlotBytes + mine * kPitch, y_row + at_col(i), (unsigned)n, bar);
            }
        };
#pragma unroll 1
        for (int i = 0; i < kSlots; ++i) fetch(i);
        if (rank > 0) {
            float sum[W::kMine] = {};
            for (int i = 1; i <= nk; ++i) {
                products(i - 1);
                if (i == nk || (i & 1) == 0) {
                    // The tensor cores cut bits off a long sum: every 256 of k it is added up here.
                    tc_after();
                    float v[W::kMine];
#pragma unroll
                    for (int j = 0; j < W::kMine; j += W::kMine < 8 ? 4 : 8) {
                        const uint32_t at = t_h + ((i - 1) >> 1 & 3) * 64 + ((uint32_t)quarter << 16) + group * W::kMine + j;
                        if constexpr (W::kMine < 8) tc_ld4(at, v + j);
                        else tc_ld8(at, v + j);
                    }
                    tc_ld_wait(v);
#pragma unroll
                    for (int j = 0; j < W::kMine; ++j) sum[j] += v[j];
                    tc_before();
                }
                fetch(i - 1 + kSlots);
            }
            // h of the whole tile, summed over the cluster, as bf16 numbers. The sums lie where those will.
            constexpr int kQuads = RP / 4, kAll = kTileRows * kQuads / kWorkers;
            float4* const sums = reinterpret_cast<float4*>(h_parts);
#pragma unroll
            for (int j = 0; j < W::kMine; j += 4)  // (a row's quads are permuted: whole rows would lie in the same banks)
                sums[mine * kQuads + (((group * W::kMine + j) / 4) ^ (mine & (kQuads - 1)))] = make_float4(sum[j], sum[j + 1], sum[j + 2], sum[j + 3]);
            named_bar_sync(1, kWorkers);
            if (ctas > 1) {
                cluster_arrive();
                cluster_wait();
            }
            float4 h[kAll];
#pragma unroll
            for (int i = 0; i < kAll; ++i) {
                const int at = tid + i * kWorkers;
                if (ctas > 1) {
                    float4 v[kMaxCluster];
#pragma unroll
                    for (int c = 0; c < kMaxCluster; ++c)
                        if (c < ctas) v[c] = cluster_ld4(h0 + 16 * at, (uint32_t)c);
                    h[i] = v[0];
#pragma unroll
                    for (int c = 1; c < kMaxCluster; ++c)
                        if (c < ctas) h[i].x += v[c].x, h[i].y += v[c].y, h[i].z += v[c].z, h[i].w += v[c].w;
                } else {
                    h[i] = sums[at];
                }
            }
            named_bar_sync(1, kWorkers);
            if (ctas > 1) {
                cluster_arrive();
                cluster_wait();
            }
#pragma unroll
            for (int i = 0; i < kAll; ++i) {
                const int at = tid + i * kWorkers, r = at / kQuads, j = ((at % kQuads) ^ (r & (kQuads - 1))) * 4;
                const float v[4] = {j < rank ? h[i].x * scale : 0.0f, j + 1 < rank ? h[i].y * scale : 0.0f,  // (x may hold NaN)
                                    j + 2 < rank ? h[i].z * scale : 0.0f, j + 3 < rank ? h[i].w * scale : 0.0f};
                __nv_bfloat16 p[4][W::kParts];
#pragma unroll
                for (int e = 0; e < 4; ++e) split<W::kParts>(v[e], p[e]);
#pragma unroll
                for (int q = 0; q < W::kParts; ++q) {
                    __nv_bfloat162 two[2] = {__halves2bfloat162(p[0][q], p[1][q]), __halves2bfloat162(p[2][q], p[3][q])};
                    *reinterpret_cast<uint2*>(h_parts + q * W::kPart + place<128>(r, j / 8) + j % 8 * 2) = *reinterpret_cast<const uint2*>(two);
                }
                if (L.h != nullptr && blockIdx.y == 0 && r % ctas == (int)cta && rows[r] >= 0)
#pragma unroll
                    for (int e = 0; e < 4; ++e)
                        if (j + e < L.r) L.h[(size_t)rows[r] * L.r + j + e] = v[e];
            }
            fence_proxy_async_smem();
            mbar_arrive(&have_h);
        }
        // out: this thread's row of every fourth item
        for (int i = nk + ((group - nk) & 3); i < total; i += kGroups) {
            wait(&come_y[i & 3][warp & 3], (i - nk) >> 2 & 1);
            if (rank > 0) products(i);
            tc_after();
            unsigned char* const mine_at = smem + (i & 3) * kSlotBytes + mine * kPitch;
            constexpr int kPer = 16 / (int)sizeof(TY);
            if (rank > 0) {
                for (int j0 = 0; j0 < W::kOutCols; j0 += 16) {
                    float v[16];
                    tc_ld8(t_out + (i & 1) * 128 + ((uint32_t)quarter << 16) + j0, v);
                    tc_ld8(t_out + (i & 1) * 128 + ((uint32_t)quarter << 16) + j0 + 8, v + 8);
                    uint4 had[16 / kPer];
#pragma unroll
                    for (int c = 0; c < 16 / kPer; ++c) had[c] = lds128(mine_at + (j0 / kPer + c) * 16);
                    tc_ld_wait(v);
                    if (j0 + 16 == W::kOutCols) {
                        tc_before();
                        __syncwarp();
                        if (lane == 0) mbar_arrive(&have_read[i & 1]);
                    }
#pragma unroll
                    for (int c = 0; c < 16 / kPer; ++c) {
                        float s[kPer];
                        Vec<TY>::unpack(had[c], s);
#pragma unroll
                        for (int e = 0; e < kPer; ++e) s[e] += v[c * kPer + e];
                        uint4 w;
                        if constexpr (sizeof(TY) == 2) {
                            uint32_t two[4];
#pragma unroll
                            for (int e = 0; e < 4; ++e) {
                                const __nv_bfloat162 t = __floats2bfloat162_rn(s[2 * e], s[2 * e + 1]);
                                two[e] = *reinterpret_cast<const uint32_t*>(&t);
                            }
                            w = make_uint4(two[0], two[1], two[2], two[3]);
                        } else {
                            w = make_uint4(__float_as_uint(s[0]), __float_as_uint(s[1]), __float_as_uint(s[2]), __float_as_uint(s[3]));
                        }
                        *reinterpret_cast<uint4*>(mine_at + (j0 / kPer + c) * 16) = w;
                    }
                }
            }
            __syncwarp();
            // the warp's 32 rows, two at a time
            const int piece_out = lane & 15, n_out = bytes(i);
            const unsigned char* const from = smem + (i & 3) * kSlotBytes + (quarter + (lane >> 4)) * kPitch + piece_out * 16;
            if (piece_out * 16 < n_out) {
#pragma unroll
                for (int j = 0; j < 16; ++j) {
                    char* const to = out_at[quarter + (lane >> 4) + 2 * j];
                    const uint4 w = *reinterpret_cast<const uint4*>(from + 2 * j * kPitch);
                    if (to != nullptr) *reinterpret_cast<uint4*>(to + at_col(i) + piece_out * 16) = w;
                }
            }
            fence_proxy_async_smem();
            __syncwarp();
            fetch(i + kGroups);
        }
    }
    copies_wait_all();
    if (failed) {  // copies may be in flight: give them time to land
        atomicAdd(&wide_timeouts, 1u);
        const unsigned long long t0 = global_ns();
        while (global_ns() - t0 < 2000000ull) __nanosleep(1000);
    }
    tc_before();
    __syncthreads();
    if (warp == 0 && rank > 0) {
        tc_after();
        tc_free<512>(tmem);
    }
}

template <int RP, typename TY>
cudaError_t launch(const AdaptLaunch& a, cudaStream_t stream) {
    using W = Wide<RP, TY>;
    const auto kernel = k_adapt_wide<RP, TY>;
    static std::atomic<int> known[kMaxCluster + 1];
    const cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, W::kSmem);
    if (e != cudaSuccess) return e;
    // The cluster, and the clusters that share a tile's columns (each with its own h), whose rounds take the least time for nearly
    // the most tiles that there can be (one too many for a round costs a second). Measured, in microseconds: an item of x takes
    // 0.6, one of y 1.2, or what the memory takes for those of all CTAs, and to begin and to join take 8.
    const long long tiles = most_tiles(a.rows, a.n_adapters, kTileRows), expect = tiles > 1 ? tiles - 1 : 1;
    const int k_items = (a.k + W::kCols - 1) / W::kCols, n_items = a.out != nullptr ? (a.n + W::kOutCols - 1) / W::kOutCols : 0;
    int ctas = 1;
    long long sharing = 1;
    double best = 1e30;
    for (int c = 1; c <= kMaxCluster; ++c) {
        const int fit = resident_clusters(kernel, c, kWideThreads, W::kSmem, known);
        const long long most = n_items / c < 1 ? 1 : n_items / c;
        for (long long s = 1; s <= most && s <= 16 && (s == 1 || expect * s <= fit); ++s) {
            const long long rounds = (expect * s + fit - 1) / fit;
            const double at_once = (double)(expect * s * c) / (double)rounds;
            const double x = at_once * 0.0056 > 0.6 ? at_once * 0.0056 : 0.6, y = at_once * 0.0113 > 1.2 ? at_once * 0.0113 : 1.2;
            const double time = (double)rounds * ((double)k_items / c * x + (double)n_items / (double)(c * s) * y + 8);
            if (time < best * 0.99) best = time, ctas = c, sharing = s;
        }
    }
    cudaLaunchConfig_t cfg = launch_shape(dim3((unsigned)(tiles * ctas), (unsigned)sharing), kWideThreads, stream);
    cfg.dynamicSmemBytes = W::kSmem;
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
cudaError_t launch_rank(const AdaptLaunch& a, cudaStream_t stream) {
    return a.r <= 16 ? launch<16, TY>(a, stream) : a.r <= 32 ? launch<32, TY>(a, stream) : launch<64, TY>(a, stream);
}

}  // namespace

cudaError_t launch_adapt_wide(const AdaptLaunch& a, bool y_f32, cudaStream_t stream) {
    return y_f32 ? launch_rank<float>(a, stream) : launch_rank<__nv_bfloat16>(a, stream);
}

cudaError_t adapt_wide_timeouts(unsigned* n, cudaStream_t stream) {
    return cudaMemcpyFromSymbolAsync(n, wide_timeouts, sizeof *n, 0, cudaMemcpyDeviceToHost, stream);
}

}  // namespace tsffn
