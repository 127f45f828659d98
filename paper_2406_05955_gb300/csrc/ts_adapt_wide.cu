// ts_adapt_wide.cu -- ts_adapt_rows over many rows (a list, r up to 64): tiles of 128 rows of one adapter on the tensor cores.
//
// The tile's cluster shares k and the columns as in ts_adapt.cu. A CTA's items are chunks 256 bytes of each row wide: of x and
// A_i, whose products are summed in tensor memory, and then of y and B_i. h is the M operand of the second product, as 2 (bf16
// rows) or 3 (fp32) bf16 numbers in shared memory; a row of its sums is a lane of tensor memory, so a thread adds 16 bytes
// of its own row of y at a time, and its warp writes them as 64-byte pieces of rows.
//
// Eight warps copy items into a ring, add y and write; a ninth issues the products. They wait for one another by barriers in
// shared memory only (an item has come; its products are done; sums have been read), so no warp waits for another's copies to
// be issued, and the two CTAs of an SM fill each other's gaps. (With a CTA barrier an item, the products issued by one of
// the eight: 0.9 us an item whatever it held, 130 us where this takes XX.)
#include "ts_adapt.cuh"
#include "ts_grouped.h"

namespace tsffn {
namespace {

__device__ unsigned wide_status;

constexpr int kTileRows = 128;
constexpr int kWorkers = 256, kWideThreads = kWorkers + kWarp;
constexpr int kWideChunk = 128;                      // bytes of a row in an item
constexpr int kSides = kWorkers / kTileRows;  // warps that share 32 rows: each has a part of an item's columns

template <int RP, typename TY>
struct Wide {
    static constexpr int kCols = kWideChunk / 2;                   // of x and A in an item
    static constexpr int kOutCols = kWideChunk / (int)sizeof(TY);  // of y and out
    static constexpr int kParts = sizeof(TY) == 2 ? 2 : 3;
    static constexpr int kRowsBytes = kTileRows * kWideChunk, kSlot = kRowsBytes + RP * kWideChunk;
    static constexpr int kPart = kTileRows * 128;                  // of h: 128 bytes a row, of which r take 2 r
    static constexpr int kRoom = 108 * 1024 - kParts * kPart - 1024;  // two CTAs on an SM
    static constexpr int kSlots = kRoom / kSlot < 4 ? kRoom / kSlot : 4;
    static constexpr int kSmem = kSlots * kSlot + kParts * kPart + 1024;
    static constexpr int kMine = RP / kSides;                      // components of a thread's row
    static_assert(kSlots >= 2 && kTileRows * RP * 4 <= kParts * kPart, "the sums lie where h will");
};

template <int RP, typename TY>
__global__ void __launch_bounds__(kWideThreads, 2) k_adapt_wide(const __grid_constant__ AdaptLaunch L, int ctas) {
    using W = Wide<RP, TY>;
    extern __shared__ unsigned char raw[];
    __shared__ TileRows found;
    __shared__ int rows[kTileRows];
    __shared__ uint2 x_at[kTileRows], y_at[kTileRows];  // first byte of each row (none: the highest bit)
    __shared__ char* out_at[kTileRows];                 // and of out (nullptr)
    __shared__ uint64_t come[W::kSlots], done[W::kSlots];  // an item's copies, its products
    __shared__ uint64_t have_h, have_read[2];              // h as bf16 numbers, the products of an item, which alternate
    __shared__ uint32_t tmem;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const uint32_t cta = cluster_rank();
    unsigned char* const smem = raw + (-smem_u32(raw) & 1023u);
    unsigned char* const h_parts = smem + W::kSlots * W::kSlot;
    const uint32_t smem0 = smem_u32(smem), h0 = smem_u32(h_parts);
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
        const uint64_t none = 1ull << 63, xb = row < 0 ? none : (uint64_t)(row * L.ldx * 2), yb = row < 0 ? none : (uint64_t)(row * L.ldy * (int)sizeof(TY));
        x_at[tid] = make_uint2((uint32_t)xb, (uint32_t)(xb >> 32));
        y_at[tid] = make_uint2((uint32_t)yb, (uint32_t)(yb >> 32));
        out_at[tid] = row < 0 ? nullptr : reinterpret_cast<char*>(out + row * L.ldo);
    }
    if (tid == 0) {
        for (int i = 0; i < W::kSlots; ++i) {
            mbar_init(&come[i], kWorkers);
            mbar_init(&done[i], 1);
        }
        mbar_init(&have_h, kWorkers);
        for (int i = 0; i < 2; ++i) mbar_init(&have_read[i], kWorkers / kWarp);
        mbar_fence_init();
    }
    if (warp == 0 && rank > 0) tc_alloc<256>(&tmem);
    tc_before();
    __syncthreads();
    tc_after();
    // tensor memory: two sums of h, one of them being read, and two items' products
    const uint32_t t_h = rank > 0 ? tmem : 0, t_out = t_h + 128;

    const int k_chunks = rank > 0 ? (L.k + W::kCols - 1) / W::kCols : 0;
    const int n_chunks = out != nullptr ? (L.n + W::kOutCols - 1) / W::kOutCols : 0;
    const int k0 = (int)((long long)k_chunks * cta / ctas), nk = (int)((long long)k_chunks * (cta + 1) / ctas) - k0;
    const int all = ctas * (int)gridDim.y, me = (int)(blockIdx.y * ctas + cta);
    const int n0 = (int)((long long)n_chunks * me / all), nn = (int)((long long)n_chunks * (me + 1) / all) - n0;
    const int total = nk + nn;

    // A warp has 64 bytes of 32 rows of an item.
    const int quarter = (warp & 3) * 32, side = warp >> 2;
    const int piece = side * 4 + (lane & 3);  // the 16-byte piece of a row that this thread copies, of every 8th row
    const int my_row = quarter + (lane >> 2);
    const uint32_t to_rows = place<128>(my_row, piece);
    constexpr int kPer = 16 / (int)sizeof(TY), kAStep = kWorkers / 8, kBPieces = W::kOutCols / 8, kBStep = kWorkers / kBPieces;
    const int a_row = tid / 8, a_piece = tid % 8, b_row = tid / kBPieces, b_piece = tid % kBPieces;
    const uint32_t a_to = W::kRowsBytes + place<128>(a_row, a_piece), b_to = W::kRowsBytes + place<128>(b_row, b_piece);
    const int64_t a_step = (int64_t)kAStep * L.k * 2, b_step = (int64_t)kBStep * L.n * 2;
    const auto from = [](const char* base, const uint2& at) { return base + ((uint64_t)(at.y & 0x7fffffffu) << 32 | at.x); };
    const auto issue = [&](int i, int slot) {
        if (i >= total) return;
        const uint32_t to = smem0 + (uint32_t)slot * W::kSlot;
        if (i < nk) {
            const int col = (k0 + i) * W::kCols + piece * 8, a_col = (k0 + i) * W::kCols + a_piece * 8;
            const bool in = col < L.k, a_in = a_col < L.k;
            const char* const base = reinterpret_cast<const char*>(x + (in ? col : 0));
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const uint2 at = x_at[my_row + j * 8];
                copy16(to + to_rows + j * 8 * 128, from(base, at), in && (int)at.y >= 0);
            }
            const char* mat = reinterpret_cast<const char*>(a + (size_t)a_row * L.k + (a_in ? a_col : 0));
#pragma unroll
            for (int j = 0; j < (RP + kAStep - 1) / kAStep; ++j) {
                const bool take = a_in && a_row + j * kAStep < rank;
                if (RP >= kAStep || a_row < RP) copy16(to + a_to + j * kAStep * 128, take ? mat : reinterpret_cast<const char*>(a), take);
                mat += a_step;
            }
        } else {
            const int col0 = (n0 + i - nk) * W::kOutCols, col = col0 + piece * kPer, b_col = col0 + b_piece * 8;
            const bool in = col < L.n, b_in = b_col < L.n;
            const char* const base = reinterpret_cast<const char*>(y + (in ? col : 0));
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const uint2 at = y_at[my_row + j * 8];
                copy16(to + to_rows + j * 8 * 128, from(base, at), in && (int)at.y >= 0);
            }
            if (rank > 0) {
                const char* mat = reinterpret_cast<const char*>(b + (size_t)b_row * L.n + (b_in ? b_col : 0));
#pragma unroll
                for (int j = 0; j < (RP + kBStep - 1) / kBStep; ++j) {
                    const bool take = b_in && b_row + j * kBStep < rank;
                    if (RP >= kBStep || b_row < RP) copy16(to + b_to + j * kBStep * 128, take ? mat : reinterpret_cast<const char*>(b), take);
                    mat += b_step;
                }
            }
        }
        copies_arrive(&come[slot]);
    };

    const auto multiply = [&](int i, int slot) {  // by one thread
        const uint32_t at = smem0 + (uint32_t)slot * W::kSlot, mat = at + W::kRowsBytes;
        if (i < nk) {
            const uint32_t d = t_h + (i >> 2 & 1) * 64;
#pragma unroll
            for (int ks = 0; ks < W::kCols / 16; ++ks)
                tc_mma(d, desc_k(at) + 2 * ks, desc_k(mat) + 2 * ks, idesc(RP, false, false), (i & 3) != 0 || ks > 0);
        } else {
#pragma unroll
            for (int q = W::kParts - 1; q >= 0; --q)
#pragma unroll
                for (int ks = 0; ks < RP / 16; ++ks)
                    tc_mma(t_out + (i & 1) * 64, desc_k(h0 + q * W::kPart) + 2 * ks, desc_n(mat, 1024) + 128 * ks,
                           idesc(W::kOutCols, false, true), q < W::kParts - 1 || ks > 0);
        }
        if (!(L.test_stall && i == total - 1)) tc_commit(&done[slot]);
    };

    // The tensor cores cut bits off a long sum: every 256 of k it is added up here.
    const auto take_over = [&](int i, float (&sum)[W::kMine]) {
        float v[W::kMine];
#pragma unroll
        for (int j = 0; j < W::kMine; j += W::kMine < 8 ? 4 : 8) {
            const uint32_t at = t_h + (i >> 2 & 1) * 64 + ((uint32_t)quarter << 16) + side * W::kMine + j;
            if constexpr (W::kMine < 8) tc_ld4(at, v + j);
            else tc_ld8(at, v + j);
        }
        tc_ld_wait(v);
#pragma unroll
        for (int j = 0; j < W::kMine; ++j) sum[j] += v[j];
        tc_before();
    };

    // h of the whole tile, summed over the cluster, as bf16 numbers. The sums lie where those will.
    const auto join = [&](const float (&sum)[W::kMine]) {
        constexpr int kQuads = RP / 4, kAll = kTileRows * kQuads / kWorkers;
        float4* const sums = reinterpret_cast<float4*>(h_parts);
        const int mine = quarter + lane;
#pragma unroll
        for (int j = 0; j < W::kMine; j += 4)  // (a row's quads are permuted: whole rows would lie in the same banks)
            sums[mine * kQuads + (((side * W::kMine + j) / 4) ^ (mine & (kQuads - 1)))] = make_float4(sum[j], sum[j + 1], sum[j + 2], sum[j + 3]);
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
            const int at = tid + i * kWorkers, row = at / kQuads, j = ((at % kQuads) ^ (row & (kQuads - 1))) * 4;
            const float v[4] = {j < rank ? h[i].x * scale : 0.0f, j + 1 < rank ? h[i].y * scale : 0.0f,  // (x may hold NaN)
                                j + 2 < rank ? h[i].z * scale : 0.0f, j + 3 < rank ? h[i].w * scale : 0.0f};
            __nv_bfloat16 p[4][W::kParts];
#pragma unroll
            for (int e = 0; e < 4; ++e) split<W::kParts>(v[e], p[e]);
#pragma unroll
            for (int q = 0; q < W::kParts; ++q) {
                __nv_bfloat162 two[2] = {__halves2bfloat162(p[0][q], p[1][q]), __halves2bfloat162(p[2][q], p[3][q])};
                *reinterpret_cast<uint2*>(h_parts + q * W::kPart + place<128>(row, j / 8) + j % 8 * 2) = *reinterpret_cast<const uint2*>(two);
            }
            if (L.h != nullptr && blockIdx.y == 0 && row % ctas == (int)cta && rows[row] >= 0)
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    if (j + e < L.r) L.h[(size_t)rows[row] * L.r + j + e] = v[e];
        }
        fence_proxy_async_smem();
        mbar_arrive(&have_h);
    };

    // out of item i: this warp's part
    const auto add = [&](int i, int slot) {
        unsigned char* const tile = smem + slot * W::kSlot;
        const int mine = quarter + lane;
        constexpr int kCols = 4 * kPer;  // of this thread's row
        float v[kCols];
        if (rank > 0) {
#pragma unroll
            for (int j = 0; j < kCols; j += 8) tc_ld8(t_out + (i & 1) * 64 + ((uint32_t)quarter << 16) + side * kCols + j, v + j);
            tc_ld_wait(v);
            tc_before();
            __syncwarp();
            if (lane == 0) mbar_arrive(&have_read[i & 1]);
        } else {
#pragma unroll
            for (int j = 0; j < kCols; ++j) v[j] = 0.0f;
        }
#pragma unroll
        for (int c = 0; c < 4; ++c) {
            uint4* const p = reinterpret_cast<uint4*>(tile + place<128>(mine, side * 4 + c));
            const uint4 had = *p;
            float s[kPer];
            Vec<TY>::unpack(had, s);
#pragma unroll
            for (int e = 0; e < kPer; ++e) s[e] += v[c * kPer + e];
            if constexpr (sizeof(TY) == 2) {
                uint32_t w[4];
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const __nv_bfloat162 two = __floats2bfloat162_rn(s[2 * e], s[2 * e + 1]);
                    w[e] = *reinterpret_cast<const uint32_t*>(&two);
                }
                *p = make_uint4(w[0], w[1], w[2], w[3]);
            } else {
                *reinterpret_cast<float4*>(p) = make_float4(s[0], s[1], s[2], s[3]);
            }
        }
        __syncwarp();
        const int col = (n0 + i - nk) * W::kOutCols + piece * kPer;
        if (col < L.n)
#pragma unroll
            for (int j = 0; j < 4; ++j)
                if (char* const to = out_at[my_row + j * 8]; to != nullptr)
                    *reinterpret_cast<uint4*>(to + (int64_t)col * (int)sizeof(TY)) = *reinterpret_cast<const uint4*>(tile + to_rows + j * 8 * 128);
        __syncwarp();
    };

    bool failed = false;
    const auto wait = [&](uint64_t* bar, unsigned parity) {
        if (!failed) failed = !mbar_wait(bar, parity);  // (after the first that gives up, none waits)
    };
    if (warp == kWorkers / kWarp) {
        if (rank > 0) {
            int slot = 0, round = 0;
            for (int i = 0; i <= total; ++i) {
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
                // the n-th item of its kind's buffer: the one before that must have been read
                if (i >= nk + 2) wait(&have_read[i & 1], ((i - nk) / 2 - 1) & 1);
                wait(&come[slot], round & 1);
                failed = __any_sync(0xffffffffu, failed);
                if (!failed) {
                    fence_proxy_async_smem();
                    tc_after();
                    if (elect_one()) multiply(i, slot);
                    __syncwarp();
                }
                if (++slot == W::kSlots) slot = 0, ++round;
            }
        }
    } else {
#pragma unroll
        for (int i = 0; i < W::kSlots; ++i) issue(i, i);
        // Turn i: item i - 1 is finished and its place in the ring given to item i - 1 + kSlots.
        int slot = 0, round = 0;  // of item i - 1
        const auto await = [&] {
            wait(&come[slot], round & 1);
            if (rank > 0) wait(&done[slot], round & 1);
            tc_after();
        };
        const auto go_on = [&](int i) {
            issue(i - 1 + W::kSlots, slot);
            if (++slot == W::kSlots) slot = 0, ++round;
        };
        if (rank > 0) {
            float sum[W::kMine] = {};
            for (int i = 1; i <= nk; ++i) {
                await();
                if (i == nk || (i & 3) == 0) take_over(i - 1, sum);
                if (i < nk) go_on(i);
            }
            join(sum);
            if (nk > 0) go_on(nk);
        }
        for (int i = nk + 1; i <= total; ++i) {
            await();
            add(i - 1, slot);
            go_on(i);
        }
    }
    copies_wait_all();
    if (failed) atomicOr(&wide_status, kStatusTimeout);
    tc_before();
    __syncthreads();
    if (warp == 0 && rank > 0) {
        tc_after();
        tc_free<256>(tmem);
    }
}

template <int RP, typename TY>
cudaError_t launch(const AdaptLaunch& a, cudaStream_t stream) {
    using W = Wide<RP, TY>;
    const auto kernel = k_adapt_wide<RP, TY>;
    const cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, W::kSmem);
    if (e != cudaSuccess) return e;
    // Two CTAs an SM: the cluster whose rounds of CTAs take the least time, for as many tiles as whole ones and half a one an
    // adapter. Beside its items, a CTA takes the time of about 8 to begin and to join.
    const long long tiles = most_tiles(a.rows, a.n_adapters, kTileRows), expect = (2 * (a.rows / kTileRows) + tiles + 1) / 3;
    const double items = (double)(a.k / W::kCols) + (a.out != nullptr ? a.n / W::kOutCols : 0);
    int ctas = 1;
    double best = 1e30;
    for (int c = 1; c <= kMaxCluster; c *= 2) {
        const double time = (double)((expect * c + kResidentCtas - 1) / kResidentCtas) * (items / c + 8);
        if (time < best) best = time, ctas = c;
    }
    const long long chunks = (a.n + W::kOutCols - 1) / W::kOutCols;
    long long sharing = a.out != nullptr ? kResidentCtas / (tiles * ctas) : 1;
    if (sharing > chunks / (2 * ctas)) sharing = chunks / (2 * ctas);
    if (sharing < 1) sharing = 1;
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

cudaError_t adapt_wide_status(unsigned* bits, cudaStream_t stream) {
    static const unsigned zero = 0;
    cudaError_t e = cudaMemcpyFromSymbolAsync(bits, wide_status, sizeof *bits, 0, cudaMemcpyDeviceToHost, stream);
    if (e == cudaSuccess) e = cudaMemcpyToSymbolAsync(wide_status, &zero, sizeof zero, 0, cudaMemcpyHostToDevice, stream);
    return e == cudaSuccess ? cudaStreamSynchronize(stream) : e;
}

}  // namespace tsffn
