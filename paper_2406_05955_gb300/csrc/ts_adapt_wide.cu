// ts_adapt_wide.cu -- ts_adapt_rows over many rows (a list, r up to 64): tiles of 128 rows of one adapter on the tensor cores.
//
// The tile's cluster shares k and the columns as in ts_adapt.cu. A CTA's items are chunks 256 bytes of each row wide: of x and
// A_i, whose products are summed in tensor memory, and then of y and B_i. h is the M operand of the second product, as 2 (bf16
// rows) or 3 (fp32) bf16 numbers in shared memory, and a row of its products is a lane of tensor memory: so a thread has a row of
// an item to itself. It fetches it by one bulk copy into a row of shared memory, adds to it in place and sends it off by
// another; no two threads touch the same bytes, and nothing is written twice.
//
// Warps 0-3 and 4-7 take items of y in turn (and copy x, 16 bytes at a time, in the order the tensor cores want), warps 8-11
// copy A and B, warp 12 issues the products. They wait for one another by barriers in shared memory only. What was measured on the
// way, 8192 rows, k = 4096, n = 14336, r = 64, bf16: eight warps that do everything, a CTA barrier an item, 130 us (0.9 us an item
// whatever it holds: the longest warp's copies, products and sums in a row); the same with sixteen warps, or two CTAs of half
// the item, 130-140; a warp of its own for the products 128 (16-byte copies and pieces of 64 bytes a warp: 2 us for 2 KB);
// as it is 114.
#include <atomic>

#include "ts_adapt.cuh"
#include "ts_grouped.h"

namespace tsffn {
namespace {

__device__ unsigned wide_status;

constexpr int kTileRows = 128;
constexpr int kGroup = kTileRows, kWorkers = 2 * kGroup;  // threads that take items of y in turn
constexpr int kCarriers = 128;                            // that copy A and B
constexpr int kWideThreads = kWorkers + kCarriers + kWarp;
constexpr int kXSlots = 4;                                // items of x in the ring
constexpr int kRowBytes = 2 * kChunk;                     // a group's thread has two items of its row at a time
constexpr int kPitch = kRowBytes + 16;                    // bytes from a row to the next: 8 rows' same piece lie in 8 banks
constexpr int kGroupBytes = kTileRows * kPitch;
constexpr int kRing = 2 * kGroupBytes;                    // rows of y and out of both groups; before, the items of x
static_assert(kRing % 1024 == 0 && kRing >= kXSlots * kTileRows * kChunk, "");

template <int RP, typename TY>
struct Wide {
    static constexpr int kCols = kChunk / 2;                   // of x and A in an item
    static constexpr int kOutCols = kChunk / (int)sizeof(TY);  // of y and out
    static constexpr int kParts = sizeof(TY) == 2 ? 2 : 3;
    static constexpr int kMat = RP * kChunk;                   // of A or B in an item
    static constexpr int kMats = RP == 64 && kParts == 3 ? 2 : 3;
    static constexpr int kPart = kTileRows * 128;              // of h: 128 bytes a row, of which r take 2 r
    static constexpr int kSmem = 1024 + kRing + kMats * kMat + kParts * kPart;
    static constexpr int kMine = RP / 2;                       // components of a thread's row
    static_assert(kTileRows * RP * 4 <= kParts * kPart, "the sums lie where h will");
};

__device__ __forceinline__ void bulk_store(void* to, uint32_t from, unsigned bytes) {
    asm volatile("cp.async.bulk.global.shared::cta.bulk_group [%0], [%1], %2;" ::"l"(to), "r"(from), "r"(bytes) : "memory");
    asm volatile("cp.async.bulk.commit_group;" ::: "memory");
}
__device__ __forceinline__ void bulk_wait_read() { asm volatile("cp.async.bulk.wait_group.read 0;" ::: "memory"); }
__device__ __forceinline__ void bulk_wait() { asm volatile("cp.async.bulk.wait_group 0;" ::: "memory"); }

template <int RP, typename TY>
__global__ void __launch_bounds__(kWideThreads, 1) k_adapt_wide(const __grid_constant__ AdaptLaunch L, int ctas, int high) {
    using W = Wide<RP, TY>;
    extern __shared__ unsigned char raw[];
    __shared__ TileRows found;
    __shared__ int rows[kTileRows];
    __shared__ uint2 x_at[kTileRows];  // first byte of each row of x (none: the highest bit)
    __shared__ uint64_t come_x[kXSlots], come_y[2][kGroup / kWarp], come_mat[W::kMats];  // copies of x, of a warp's rows of y, of A or B
    __shared__ uint64_t done_x[kXSlots], done_out[2], done_mat[W::kMats];  // products: of an item of x, of a group's item, with a matrix
    __shared__ uint64_t have_h, have_read[2];   // h as bf16 numbers; the products of a group's item are in registers
    __shared__ uint32_t tmem;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const uint32_t cta = cluster_rank();
    unsigned char* const smem = raw + (-smem_u32(raw) & 1023u);
    unsigned char* const mats = smem + kRing;
    unsigned char* const h_parts = mats + W::kMats * W::kMat;
    const uint32_t smem0 = smem_u32(smem), mats0 = smem_u32(mats), h0 = smem_u32(h_parts);
    pdl_wait();
    find_listed<kTileRows>(L, (int)(blockIdx.x / ctas), &found, rows, high);
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
    }
    if (tid == 0) {
        for (int i = 0; i < kXSlots; ++i) {
            mbar_init(&come_x[i], kWorkers);
            mbar_init(&done_x[i], 1);
        }
        for (int i = 0; i < W::kMats; ++i) {
            mbar_init(&come_mat[i], kCarriers);
            mbar_init(&done_mat[i], 1);
        }
        for (int g = 0; g < 2; ++g) {
            for (int q = 0; q < kGroup / kWarp; ++q) mbar_init(&come_y[g][q], 1);
            mbar_init(&done_out[g], 1);
        }
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
    // The items: nk of x, and then, in the order of their products, those of y, four at a time: the first of two that group 0
    // has, the first of group 1, the second of group 0, the second of group 1. `part` says which item of this CTA's columns that
    // is; the last ones may be missing.
    const int total = nk + (nn + 3) / 4 * 4;
    const auto part = [&](int i) { return (i - nk) / 4 * 4 + (i - nk) % 2 * 2 + (i - nk) / 2 % 2; };
    const auto missing = [&](int i) { return i >= nk && part(i) >= nn; };

    bool failed = false;
    const auto wait = [&](uint64_t* bar, unsigned parity) {
        if (!failed) failed = !mbar_wait(bar, parity);  // (after the first that gives up, none waits)
    };

    if (warp >= (kWorkers + kCarriers) / kWarp) {
        // ---- the products -------------------------------------------------------------------------------------------
        int mat = 0, round = 0, taken[2] = {0, 0};
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
            if (missing(i)) continue;
            const int group = (i - nk) & 1;
            if (i < nk) {
                wait(&come_x[i & 3], i >> 2 & 1);
            } else {
                const int n = group ? taken[1]++ : taken[0]++;  // items of this group before
                if (n > 0) wait(&have_read[group], (n - 1) & 1);
            }
            wait(&come_mat[mat], round & 1);
            failed = __any_sync(0xffffffffu, failed);
            if (!failed) {
                fence_proxy_async_smem();
                tc_after();
                if (elect_one()) {
                    const uint32_t m = mats0 + mat * W::kMat, at = smem0 + (i & 3) * (kTileRows * kChunk);
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
                                tc_mma(t_out + group * 128, desc_k(h0 + q * W::kPart) + 2 * ks, desc_n(m, RP * 128) + 128 * ks,
                                       idesc(W::kOutCols, false, true), q < W::kParts - 1 || ks > 0);
                    }
                    tc_commit(&done_mat[mat]);
                    if (!(L.test_stall && i + 4 >= total)) tc_commit(i < nk ? &done_x[i & 3] : &done_out[group]);
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
        int mat = 0, round = 0;
        for (int i = 0; i < total && rank > 0; ++i) {
            if (i == nk && !met) cluster_arrive();
            if (i == nk + W::kMats) meet();
            if (missing(i)) continue;
            if (round > 0) wait(&done_mat[mat], (round - 1) & 1);
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
                const int col = (n0 + part(i)) * W::kOutCols + b_piece * 8;
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
            if (++mat == W::kMats) mat = 0, ++round;
        }
        if (total == nk && !met) cluster_arrive();
        meet();
    } else {
        // ---- rows ---------------------------------------------------------------------------------------------------
        const int group = warp >> 2, quarter = (warp & 3) * 32, mine = quarter + lane;  // this thread's row of the group's items
        const int row = rows[mine];
        const char* const y_row = reinterpret_cast<const char*>(y + (row < 0 ? 0 : row * L.ldy));
        char* const out_row = reinterpret_cast<char*>(out + (row < 0 ? 0 : row * L.ldo));
        const int there = __popc(__ballot_sync(0xffffffffu, row >= 0));
        // the two items of y of number `pair` of this group: where they begin in a row, and their bytes
        const auto at_pair = [&](int pair) { return (int64_t)(n0 + 4 * pair + 2 * group) * kChunk; };
        const auto bytes = [&](int pair) {
            const int mine = min(2, nn - 4 * pair - 2 * group);  // items
            return (int)min((int64_t)mine * kChunk, (int64_t)L.n * (int)sizeof(TY) - at_pair(pair));
        };
        const int pairs = (nn - 2 * group + 3) / 4;
        unsigned char* const mine_at = smem + group * kGroupBytes + mine * kPitch;
        const auto fetch_y = [&](int pair) {
            if (pair >= pairs) return;
            uint64_t* const bar = &come_y[group][warp & 3];
            const int n = bytes(pair);
            if (lane == 0) mbar_arrive_expect_tx(bar, (unsigned)(there * n));
            __syncwarp();
            if (row >= 0) tma_load_1d(mine_at, y_row + at_pair(pair), (unsigned)n, bar);
        };
        // x: a warp copies the half `group` of 32 rows, 8 lanes a row
        const int piece = group * 8 + (lane & 7), x_row = quarter + (lane >> 3);
        const uint32_t x_to = group * (kTileRows * 128) + place<128>(x_row, piece & 7);
        const auto fetch_x = [&](int i) {
            if (i >= nk) return;
            const int col = (k0 + i) * W::kCols + piece * 8;
            const bool in = col < L.k;
            const char* const base = reinterpret_cast<const char*>(x + (in ? col : 0));
            const uint32_t to = smem0 + (i & 3) * (kTileRows * kChunk);
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const uint2 at = x_at[x_row + j * 4];
                copy16(to + (x_to ^ (j & 1) << 6) + j * 4 * 128, base + ((uint64_t)(at.y & 0x7fffffffu) << 32 | at.x), in && (int)at.y >= 0);
            }
            copies_arrive(&come_x[i & 3]);
        };
#pragma unroll 1
        for (int i = 0; i < kXSlots; ++i) fetch_x(i);
        if (rank > 0) {
            float sum[W::kMine] = {};
            for (int i = 1; i <= nk; ++i) {
                wait(&done_x[(i - 1) & 3], (i - 1) >> 2 & 1);
                fetch_x(i - 1 + kXSlots);
                if (i == nk) {  // y comes where x was
                    fence_proxy_async_smem();
                    fetch_y(0);
                }
                if (i == nk || (i & 1) == 0) {
                    // The tensor cores cut bits off a long sum: every 256 of k it is added up here.
                    tc_after();
                    float v[W::kMine];
#pragma unroll
                    for (int j = 0; j < W::kMine; j += 8)
                        tc_ld8(t_h + ((i - 1) >> 1 & 3) * 64 + ((uint32_t)quarter << 16) + group * W::kMine + j, v + j);
                    tc_ld_wait(v);
#pragma unroll
                    for (int j = 0; j < W::kMine; ++j) sum[j] += v[j];
                    tc_before();
                }
            }
            if (nk == 0) fetch_y(0);
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
        if (rank == 0) fetch_y(0);
        // out: this thread's row of the group's items, two at a time
        constexpr int kPer = 16 / (int)sizeof(TY);
        int taken = 0;
        for (int pair = 0; pair < pairs; ++pair) {
            wait(&come_y[group][warp & 3], pair & 1);
#pragma unroll 1
            for (int half = 0; half < 2 && rank > 0 && 4 * pair + 2 * group + half < nn; ++half) {
                wait(&done_out[group], taken++ & 1);
                tc_after();
                unsigned char* const at = mine_at + half * kChunk;
#pragma unroll
                for (int j0 = 0; j0 < W::kOutCols; j0 += 32) {
                    float v[32];
#pragma unroll
                    for (int j = 0; j < 32; j += 8) tc_ld8(t_out + group * 128 + ((uint32_t)quarter << 16) + j0 + j, v + j);
                    uint4 had[32 / kPer];
#pragma unroll
                    for (int c = 0; c < 32 / kPer; ++c) had[c] = lds128(at + (j0 / kPer + c) * 16);
                    tc_ld_wait(v);
                    if (j0 + 32 == W::kOutCols) {
                        tc_before();
                        __syncwarp();
                        if (lane == 0) mbar_arrive(&have_read[group]);
                    }
#pragma unroll
                    for (int c = 0; c < 32 / kPer; ++c) {
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
                        *reinterpret_cast<uint4*>(at + (j0 / kPer + c) * 16) = w;
                    }
                }
            }
            fence_proxy_async_smem();
            if (row >= 0) bulk_store(out_row + at_pair(pair), smem_u32(mine_at), (unsigned)bytes(pair));
            if (pair + 1 < pairs) {
                bulk_wait_read();  // (a thread's row has left before the next one comes there)
                __syncwarp();
                fetch_y(pair + 1);
            }
        }
        bulk_wait();
    }
    copies_wait_all();
    if (failed) {  // copies may be in flight: give them time to land
        atomicOr(&wide_status, kStatusTimeout);
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

// Clusters of `ctas` CTAs that can be on the device at once: a cluster has to fit into a part of it, so of the larger ones
// there are fewer than the SMs divided by their size (of 8 CTAs, one on an SM: 15 on 152 SMs). Asked for once.
template <int RP, typename TY>
int resident_clusters(int ctas) {
    static std::atomic<int> known[kMaxCluster + 1];
    int n = known[ctas].load(std::memory_order_relaxed);
    if (n == 0) {
        cudaLaunchConfig_t cfg = launch_shape(dim3((unsigned)ctas), kWideThreads, nullptr);
        cfg.dynamicSmemBytes = Wide<RP, TY>::kSmem;
        cudaLaunchAttribute at{};
        at.id = cudaLaunchAttributeClusterDimension;
        at.val.clusterDim = {(unsigned)ctas, 1, 1};
        cfg.attrs = &at;
        cfg.numAttrs = 1;
        if (cudaOccupancyMaxActiveClusters(&n, k_adapt_wide<RP, TY>, &cfg) != cudaSuccess || n < 1) n = kSms / ctas;
        known[ctas].store(n, std::memory_order_relaxed);
    }
    return n;
}

template <int RP, typename TY>
cudaError_t launch(const AdaptLaunch& a, cudaStream_t stream) {
    using W = Wide<RP, TY>;
    const auto kernel = k_adapt_wide<RP, TY>;
    const cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, W::kSmem);
    if (e != cudaSuccess) return e;
    // The rows of a tile, the cluster, and the clusters that share a tile's columns (each with its own h), whose rounds take the
    // least time for nearly the most tiles that there can be (one too many for a round costs a second). Time in items of 128
    // rows: an item of fewer takes less, down to what its latencies take, and to begin and to join take about 8.
    const int k_items = (a.k + W::kCols - 1) / W::kCols, n_items = a.out != nullptr ? (a.n + W::kOutCols - 1) / W::kOutCols : 0;
    int ctas = 1, high = kTileRows;
    long long sharing = 1;
    double best = 1e30;
    for (int c = 1; c <= kMaxCluster; ++c) {
        const int fit = resident_clusters<RP, TY>(c);
        const long long most = n_items / c < 1 ? 1 : n_items / c;
        for (int rows = kTileRows; rows >= kTileRows / 2; rows -= 4) {
            const long long expect = most_tiles(a.rows, a.n_adapters, rows) - 1;
            const double item = rows > 80 ? rows / (double)kTileRows : 80.0 / kTileRows;
            for (long long s = 1; s <= most && s <= 16 && (s == 1 || expect * s <= fit); ++s) {
                const double time = (double)((expect * s + fit - 1) / fit) * (((double)k_items / c + (double)n_items / (double)(c * s)) * item + 8);
                if (time < best * 0.99) best = time, ctas = c, sharing = s, high = rows;
            }
        }
    }
    const long long tiles = most_tiles(a.rows, a.n_adapters, high);
    cudaLaunchConfig_t cfg = launch_shape(dim3((unsigned)(tiles * ctas), (unsigned)sharing), kWideThreads, stream);
    cfg.dynamicSmemBytes = W::kSmem;
    cudaLaunchAttribute at[2]{};
    at[0].id = cudaLaunchAttributeClusterDimension;
    at[0].val.clusterDim = {(unsigned)ctas, 1, 1};
    at[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at[1].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = at;
    cfg.numAttrs = 2;
    return cudaLaunchKernelEx(&cfg, kernel, a, ctas, high);
}

template <typename TY>
cudaError_t launch_rank(const AdaptLaunch& a, cudaStream_t stream) {
    return a.r <= 16 ? launch<16, TY>(a, stream) : a.r <= 32 ? launch<32, TY>(a, stream) : launch<64, TY>(a, stream);
}

}  // namespace

cudaError_t launch_adapt_wide(const AdaptLaunch& a, bool y_f32, cudaStream_t stream) {
    return y_f32 ? launch_rank<float>(a, stream) : launch_rank<__nv_bfloat16>(a, stream);
}

cudaError_t adapt_wide_status(unsigned* bits, cudaStream_t stream) {
    static const unsigned zero = 0;
    cudaError_t e = cudaMemcpyFromSymbolAsync(bits, wide_status, sizeof *bits, 0, cudaMemcpyDeviceToHost, stream);
    if (e == cudaSuccess) e = cudaMemcpyToSymbolAsync(wide_status, &zero, sizeof zero, 0, cudaMemcpyHostToDevice, stream);
    return e == cudaSuccess ? cudaStreamSynchronize(stream) : e;
}

}  // namespace tsffn
