// ts_adapt_wide.cu -- ts_adapt_rows over many rows (a list, r up to 64): tiles of 128 rows of one adapter on the tensor cores.
//
// The tile's cluster shares k and the columns as in ts_adapt.cu. A CTA's items are chunks 256 bytes of each row wide: of x and
// A_i, whose products are summed in tensor memory, and then of y and B_i. h is the M operand of the second product, as 2 (bf16
// rows) or 3 (fp32) bf16 numbers in shared memory; a row of its sums is a lane of tensor memory, so a thread adds 16 bytes
// of its own row of y at a time, and its warp writes them as whole 128-byte lines. The warp that adds a part of y is also the
// one that copies it, so items are waited for by the thread's own copies and one CTA barrier each, and the copies of the ring's
// next items are always on their way: 80 to 96 KB, one CTA an SM.
#include "ts_adapt.cuh"
#include "ts_grouped.h"

namespace tsffn {
namespace {

__device__ unsigned wide_status;

constexpr int kTileRows = 128;

template <int RP, typename TY>
struct Wide {
    static constexpr int kCols = kChunk / 2;                   // of x and A in an item
    static constexpr int kOutCols = kChunk / (int)sizeof(TY);  // of y and out
    static constexpr int kParts = sizeof(TY) == 2 ? 2 : 3;
    static constexpr int kRowsBytes = kTileRows * kChunk, kSlot = kRowsBytes + RP * kChunk;
    static constexpr int kSlots = RP <= 32 ? 4 : 3;
    static constexpr int kPart = kTileRows * 128;              // of h: 128 bytes a row, of which r take 2 r
    static constexpr int kSmem = kSlots * kSlot + kParts * kPart + 1024;
    static constexpr int kMine = RP / 2;                       // components of a thread's row
    static_assert(kTileRows * RP * 4 <= kParts * kPart, "the sums lie where h will");
};

template <int RP, typename TY>
__global__ void __launch_bounds__(kThreads, 1) k_adapt_wide(const __grid_constant__ AdaptLaunch L, int ctas) {
    using W = Wide<RP, TY>;
    extern __shared__ unsigned char raw[];
    __shared__ TileRows found;
    __shared__ int rows[kTileRows];
    __shared__ long long x_at[kTileRows], y_at[kTileRows], out_at[kTileRows];  // first element of each row
    __shared__ uint64_t done[2];  // the products of an item, which alternate
    __shared__ uint32_t tmem;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const uint32_t cta = cluster_rank();
    unsigned char* const smem = reinterpret_cast<unsigned char*>((reinterpret_cast<uintptr_t>(raw) + 1023) & ~(uintptr_t)1023);
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
            for (int i = tid; i < count * L.r; i += kThreads)
                if (rows[i / L.r] >= 0) L.h[(size_t)rows[i / L.r] * L.r + i % L.r] = 0.0f;
        if (out == y) return;  // (of both nullptr too)
    }
    if (tid < kTileRows) {
        const int row = rows[tid];
        x_at[tid] = row < 0 ? -1 : row * L.ldx;
        y_at[tid] = row < 0 ? -1 : row * L.ldy;
        out_at[tid] = row * L.ldo;
    }
    if (tid == 0) {
        mbar_init(&done[0], 1);
        mbar_init(&done[1], 1);
        mbar_fence_init();
    }
    if (warp == 0 && rank > 0) tc_alloc<512>(&tmem);
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

    // A warp has 32 rows' left or right half of an item.
    const int quarter = (warp & 3) * 32, half = warp >> 2;
    const int piece = half * 8 + (lane & 7);  // the 16-byte piece of a row that this thread copies, of every 4th row
    const auto issue = [&](int i) {
        if (i < total) {
            const uint32_t to = smem0 + (uint32_t)(i % W::kSlots) * W::kSlot, mat = to + W::kRowsBytes;
            if (i < nk) {
                const int col = (k0 + i) * W::kCols + piece * 8;
                const bool in = col < L.k;
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    const int row = quarter + j * 4 + (lane >> 3);
                    const long long at = x_at[row];
                    const bool take = in && at >= 0;
                    copy16(to + half * (W::kRowsBytes / 2) + place<128>(row, piece & 7), take ? x + at + col : x, take);
                }
                const int c = tid % 16, a_col = (k0 + i) * W::kCols + c * 8;
#pragma unroll
                for (int j = 0; j < RP / 16; ++j) {
                    const int row = tid / 16 + j * 16;
                    const bool take = row < rank && a_col < L.k;
                    copy16(mat + (c >> 3) * (RP * 128) + place<128>(row, c & 7), take ? a + (size_t)row * L.k + a_col : a, take);
                }
            } else {
                constexpr int kPer = 16 / (int)sizeof(TY);
                const int col0 = (n0 + i - nk) * W::kOutCols, col = col0 + piece * kPer;
                const bool in = col < L.n;
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    const int row = quarter + j * 4 + (lane >> 3);
                    const long long at = y_at[row];
                    const bool take = in && at >= 0;
                    copy16(to + place<kChunk>(row, piece), take ? y + at + col : y, take);
                }
                constexpr int kBPieces = W::kOutCols / 8, kBStep = kThreads / kBPieces;
                const int c = tid % kBPieces, b_col = col0 + c * 8;
                if (rank > 0) {
#pragma unroll
                    for (int j = 0; j < (RP + kBStep - 1) / kBStep; ++j) {
                        const int row = tid / kBPieces + j * kBStep;
                        const bool take = row < rank && b_col < L.n;
                        if (RP >= kBStep || row < RP)
                            copy16(mat + (c >> 3) * (RP * 128) + place<128>(row, c & 7), take ? b + (size_t)row * L.n + b_col : b, take);
                    }
                }
            }
        }
        copies_commit();
    };

    const auto multiply = [&](int i) {  // by one thread
        const uint32_t at = smem0 + (uint32_t)(i % W::kSlots) * W::kSlot, mat = at + W::kRowsBytes;
        if (i < nk) {
            const uint32_t d = t_h + (i >> 1 & 1) * 64;
#pragma unroll
            for (int ks = 0; ks < W::kCols / 16; ++ks)
                tc_mma(d, desc_k(at + (ks >> 2) * (W::kRowsBytes / 2)) + 2 * (ks & 3), desc_k(mat + (ks >> 2) * (RP * 128)) + 2 * (ks & 3),
                       idesc(RP, false, false), (i & 1) != 0 || ks > 0);
        } else {
#pragma unroll
            for (int q = W::kParts - 1; q >= 0; --q)
#pragma unroll
                for (int ks = 0; ks < RP / 16; ++ks)
                    tc_mma(t_out + (i & 1) * 128, desc_k(h0 + q * W::kPart) + 2 * ks, desc_n(mat, RP * 128) + 128 * ks,
                           idesc(W::kOutCols, false, true), q < W::kParts - 1 || ks > 0);
        }
        if (!(L.test_stall && i == total - 1)) tc_commit(&done[i & 1]);
    };

    float sum[W::kMine] = {};
    // The tensor cores cut bits off a long sum: every 256 of k it is added up here.
    const auto take_over = [&](int i) {
        float v[W::kMine];
#pragma unroll
        for (int j = 0; j < W::kMine; j += 8) tc_ld8(t_h + (i >> 1 & 1) * 64 + ((uint32_t)quarter << 16) + half * W::kMine + j, v + j);
        tc_ld_wait(v);
#pragma unroll
        for (int j = 0; j < W::kMine; ++j) sum[j] += v[j];
        tc_before();
    };

    // h of the whole tile, summed over the cluster, as bf16 numbers. The sums lie where those will.
    const auto join = [&] {
        constexpr int kQuads = RP / 4, kAll = kTileRows * kQuads / kThreads;
        float4* const sums = reinterpret_cast<float4*>(h_parts);
        const int mine = quarter + lane;
#pragma unroll
        for (int j = 0; j < W::kMine; j += 4)  // (a row's quads are permuted: whole rows would lie in the same banks)
            sums[mine * kQuads + (((half * W::kMine + j) / 4) ^ (mine & (kQuads - 1)))] = make_float4(sum[j], sum[j + 1], sum[j + 2], sum[j + 3]);
        __syncthreads();
        if (ctas > 1) {
            cluster_arrive();
            cluster_wait();
        }
        float4 h[kAll];
#pragma unroll
        for (int i = 0; i < kAll; ++i) {
            const int at = tid + i * kThreads;
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
        __syncthreads();
        if (ctas > 1) {
            cluster_arrive();
            cluster_wait();
        }
#pragma unroll
        for (int i = 0; i < kAll; ++i) {
            const int at = tid + i * kThreads, row = at / kQuads, j = ((at % kQuads) ^ (row & (kQuads - 1))) * 4;
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
        __syncthreads();
    };

    // out of item i: this warp's rows and half
    const auto add = [&](int i) {
        constexpr int kPer = 16 / (int)sizeof(TY);
        unsigned char* const tile = smem + (i % W::kSlots) * W::kSlot;
        const int mine = quarter + lane;
#pragma unroll
        for (int j0 = 0; j0 < 8 * kPer; j0 += 32) {  // of the thread's 8 pieces, 32 columns' at a time
            float v[32];
            if (rank > 0) {
#pragma unroll
                for (int j = 0; j < 32; j += 8)
                    tc_ld8(t_out + (i & 1) * 128 + ((uint32_t)quarter << 16) + half * 8 * kPer + j0 + j, v + j);
                tc_ld_wait(v);
            } else {
#pragma unroll
                for (int j = 0; j < 32; ++j) v[j] = 0.0f;
            }
#pragma unroll
            for (int c = 0; c < 32 / kPer; ++c) {
                uint4* const p = reinterpret_cast<uint4*>(tile + place<kChunk>(mine, half * 8 + j0 / kPer + c));
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
        }
        tc_before();
        __syncwarp();
        const int col = (n0 + i - nk) * W::kOutCols + piece * kPer;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const int row = quarter + j * 4 + (lane >> 3);
            if (rows[row] >= 0 && col < L.n)
                *reinterpret_cast<uint4*>(out + out_at[row] + col) = *reinterpret_cast<const uint4*>(tile + place<kChunk>(row, piece));
        }
        __syncwarp();
    };

    bool failed = false, joined = false;
#pragma unroll
    for (int i = 0; i < W::kSlots; ++i) issue(i);
    // Turn i: item i has come and is multiplied, item i - 1 is finished and its place in the ring given to item i - 1 + kSlots.
    for (int i = 0; i <= total; ++i) {
        if (i == 0) copies_wait<W::kSlots - 1>();
        else copies_wait<W::kSlots - 2>();
        fence_proxy_async_smem();
        if (__syncthreads_or(failed)) break;
        tc_after();
        const bool now = i < total && rank > 0;
        if (now && i != nk && warp == 0 && elect_one()) multiply(i);  // (the first that needs h: below)
        if (i > 0 && rank > 0) {
            failed = !mbar_wait(&done[(i - 1) & 1], (i - 1) >> 1 & 1);
            tc_after();
        }
        if (i == nk && rank > 0 && __syncthreads_or(failed)) break;  // (as one, before the join's barriers)
        if (i > 0 && i <= nk && rank > 0 && (i == nk || (i & 1) == 0)) take_over(i - 1);
        if (i == nk && rank > 0) {
            join();
            joined = true;
            if (now && warp == 0 && elect_one()) multiply(i);
        }
        if (i > nk && !failed) add(i - 1);
        if (i > 0) issue(i - 1 + W::kSlots);
    }
    copies_wait<0>();
    if (failed) atomicOr(&wide_status, kStatusTimeout);
    if (rank > 0 && ctas > 1 && !joined) {  // the others of the cluster read this CTA's sums, whatever they are
        for (int i = 0; i < 2; ++i) {
            __syncthreads();
            cluster_arrive();
            cluster_wait();
        }
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
    const cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, W::kSmem);
    if (e != cudaSuccess) return e;
    // A CTA an SM: the cluster whose rounds of CTAs take the least time, for as many tiles as whole ones and half a one an
    // adapter
    const long long tiles = most_tiles(a.rows, a.n_adapters, kTileRows), expect = (2 * (a.rows / kTileRows) + tiles + 1) / 3;
    int ctas = 1;
    double best = 1e30;
    for (int c = 1; c <= kMaxCluster; c *= 2) {
        const double time = (double)((expect * c + kSms - 1) / kSms) / c;
        if (time < best * 0.95) best = time, ctas = c;
    }
    const long long chunks = (a.n + W::kOutCols - 1) / W::kOutCols;
    long long sharing = a.out != nullptr ? kSms / (tiles * ctas) : 1;
    if (sharing > chunks / (2 * ctas)) sharing = chunks / (2 * ctas);
    if (sharing < 1) sharing = 1;
    cudaLaunchConfig_t cfg = launch_shape(dim3((unsigned)(tiles * ctas), (unsigned)sharing), kThreads, stream);
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
