// ts_grouped.cu -- products of ragged groups of rows with each group's own weights: y = x W_e, or
// max(0, x W_e) max(0, x U_e) (Eq. 1 with the dReLU of Eq. 2), over bf16 weights or e4m3 ones with a scale for
// each 128 x 128 block (and one for each 128 elements of a row of x), on the 5th-generation tensor cores.
//
// A tile is D[i][t] = W[i] . x_t for 256 weight rows i (gated: 128 neurons, gate and up rows) and up to 256 rows t of
// one group. The weights are the MMA's M and the rows of x its N, which may be any multiple of 16: a group's rows are
// cut into equal tiles, so ragged groups waste at most 15 rows a tile, and one kernel serves one row and thousands.
// (e4m3 products of many rows are taken the other way round: XM below.)
//
// A tile belongs to a pair of CTAs (tcgen05 cta_group::2): each loads its 128 weight rows and half of the rows of x, and
// the MMA reads both halves of x, so that a pair moves 64 KB for 2 x 256 x 256 x 64 flop and not 96 (one CTA
// alone would have to fetch 96 bytes a clock from L2 to keep its tensor core busy, a pair 64 a CTA).
//
// Roles of a CTA's warps: 0 loads stages of 128 bytes of k by TMA, 1 (of the first CTA) issues the MMAs, 4-11 take the
// sums out of tensor memory, where two accumulators take turns. They keep running sums in fp32 registers and add an
// accumulator to them every few stages (Kind): the tensor cores truncate when they accumulate, and each 128 of k of
// e4m3 products has scales of its own, which enter there.
//
// What bounds it, and what it measured (d = 4096, m = 14336): few rows, reading the weights (gated bf16, 16 rows over
// 8 groups: 281 us, 6.7 TB/s); many rows of bf16, the tensor cores under the power cap (8192 rows: plain 500 us, 1.9 PFLOP/s,
// where a library's product takes 471-484; gated over 8 equal groups 1053-1165 us, 1.65-1.83 PFLOP/s, over ragged ones 1225-1310);
// many rows of e4m3, handing an accumulator to the summing warps and back at every 128 of k, 0.44 us where its MMAs take
// 0.27 (8192 rows: plain 345-374 us, gated over 8 equal groups 700 us, 2.75 PFLOP/s, over ragged ones 780; 2000 rows over 8
// equal groups 230-254 us, of which reading the weights is 139, over ragged ones 284-333); one row, latency (1 x 4096 x 14336
// e4m3: 23.8 us, of which reading the weights is 9: launch, set-up, the first load, the join of a tile's parts and the
// stores come one after another).
#include <cuda_fp8.h>

#include "ts_grouped.h"
#include "ts_kernels.cuh"

namespace tsffn {
namespace {

constexpr int kEpiWarp0 = 4;
constexpr int kCtaThreads = (kEpiWarp0 + kEpiWarps) * kWarp;
constexpr int kStageW = 16384;                  // weights of a stage: 128 rows of 128 bytes
constexpr int kMaxStages = 12;
constexpr int kStageMem = 192 * 1024;           // bytes of all stages
constexpr int kMaxBufs = 4;                     // accumulators in tensor memory
// Tiles of x that one sweep over the weights serves. One group, 14336 x 4096, 8192 rows, plain bf16: 8 tiles 506-511 us, 16
// 501, 32 527-535; 16384 rows, gated bf16: 2215, 2180, 2282; 8192 rows, gated e4m3: 700-740 with each.
constexpr int kBand = 16;
constexpr int kScaleWarps = 2, kScaleSlots = 4;
// Fewest stages of a part of a tile. A part costs its pair about 3 us (written, made visible, counted and read again): with
// 16 rows through a 4096 x 4096 bf16 matrix, 4 stages take 18.5 us, 16 16.8, 24 18.1; 300 rows, 1024 x 512, 18.2, 11.1, 16.2.
constexpr int kMinSteps = 16;

__device__ __forceinline__ void sts128(uint32_t to, uint32_t a, uint32_t b, uint32_t c, uint32_t d) {
    asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(to), "r"(a), "r"(b), "r"(c), "r"(d) : "memory");
}

// ---- tiles and their parts --------------------------------------------------
// The tiles [0, whole * pairs) go round the pairs whole. The steps of the others (as many tiles as one to two rounds)
// are dealt out evenly, in order, so that all pairs end together: a pair's share begins and ends anywhere in a tile.
struct Parts {
    int pairs, steps;   // CTA pairs, stages of a tile
    int whole;          // rounds of whole tiles
    int sharers;        // pairs that get some of the rest
    int base, more;     // steps of each of them; the first `more` have one more
    __device__ void set(int tiles, int pairs_, int steps_) {
        pairs = pairs_;
        steps = steps_;
        whole = tiles % pairs == 0 ? tiles / pairs : max(0, tiles / pairs - 1);
        const int total = (tiles - whole * pairs) * steps;  // fewer than two rounds of at most 2^22 steps: below 2^31
        sharers = max(1, min(pairs, total / kMinSteps));
        base = total / sharers;
        more = total % sharers;
    }
    __device__ int begin(int q) const { return q * base + min(q, more); }
    // the pair that has step s
    __device__ int owner(int s) const {
        const int first = more * (base + 1);  // steps of the pairs that have one more
        return s < first ? s / (base + 1) : more + (s - first) / base;
    }
    // The same by a call: in the kernels of wide tiles the join's loop then leaves registers to the sums (gated e4m3, 8192 rows
    // in 8 equal groups, 14336 x 4096: 766 -> 688 us); in those of narrow tiles it would cost 1 to 2 us.
    __device__ __noinline__ int begin_called(int q) const { return begin(q); }
};

struct Seg {
    int tile, k0, k1;       // stages [k0, k1) of a tile
    int rest;               // its number among the tiles that are shared, -1: a whole one
    int g, wt, row0, rows, cols;  // group, tile of weights, first row of x, rows, and their number rounded up to 16
};

struct Shared {
    uint64_t full[kMaxStages], empty[kMaxStages], tfull[kMaxBufs], tempty[kMaxBufs], sempty[kMaxBufs];
    uint64_t met[kEpiWarps / 2];                // gated: a gate and an up warp
    uint64_t never;                             // nothing arrives here (GroupedLaunch::test_stall)
    unsigned before[kEpiWarps / 2];
    uint32_t tmem;
    int fail;
    int max_cols;                               // widest tile
    Parts parts;
    Seg seg[kEpiWarps];
    int first[kMaxGroups + 1];                  // tiles before each group
    int row0[kMaxGroups], rows[kMaxGroups];
    alignas(16) float scale[2][512];            // e4m3, [gate, up]: row times weight, of each accumulator's columns
    float raw[kScaleSlots][kScaleWarps][6][kWarp];  // and what they are made of, as it was copied
    alignas(16) unsigned char turn[kEpiWarps][2048];
};

// ---- cluster and tcgen05 helpers (pairs of CTAs) ---------------------------
__device__ __forceinline__ uint32_t cta_rank() {
    uint32_t r;
    asm volatile("mov.u32 %0, %cluster_ctarank;" : "=r"(r));
    return r;
}
__device__ __forceinline__ void cluster_sync() {
    asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}
// address of this CTA's `p` in CTA `rank` of the cluster
__device__ __forceinline__ uint32_t in_cta(const void* p, uint32_t rank) {
    uint32_t a;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(a) : "r"(smem_u32(p)), "r"(rank));
    return a;
}
// (It passes on nothing that was written to memory, so the release needs no wider scope than the CTA.)
__device__ __forceinline__ void arrive_at(uint32_t cluster_addr) {
    asm volatile("mbarrier.arrive.shared::cluster.b64 _, [%0];" ::"r"(cluster_addr) : "memory");
}
// 2-D box into this CTA's shared memory, its bytes counted by the barrier at `bar` (a CTA of the pair)
__device__ __forceinline__ void tma_box(uint32_t dst, const CUtensorMap* map, int x, int y, uint32_t bar) {
    asm volatile(
        "cp.async.bulk.tensor.2d.cta_group::2.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];" ::"r"(
            dst),
        "l"(map), "r"(x), "r"(y), "r"(bar)
        : "memory");
}
// What the host has copied to a map in global memory is what this thread's later boxes go by, and no map that lay at the
// same address before. (A map that is a parameter needs no such fence.)
__device__ __forceinline__ void map_acquire(const CUtensorMap* map) {
    asm volatile("fence.proxy.tensormap::generic.acquire.sys [%0], 128;" ::"l"(map) : "memory");
}
// 4-byte copy global -> shared (bytes = 0: zero)
__device__ __forceinline__ void cp4(float* dst, const float* src, uint32_t bytes) {
    asm volatile("cp.async.ca.shared.global [%0], [%1], 4, %2;" ::"r"(smem_u32(dst)), "l"(src), "r"(bytes) : "memory");
}
__device__ __forceinline__ void cp_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void cp_wait() {
    asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory");
}
__device__ __forceinline__ bool elect_one() {
    uint32_t p;
    asm volatile("{\n\t.reg .pred p;\n\telect.sync _|p, 0xffffffff;\n\tselp.u32 %0, 1, 0, p;\n\t}" : "=r"(p));
    return p != 0;
}
__device__ __forceinline__ uint32_t uniform(uint32_t v) { return __shfl_sync(0xffffffffu, v, 0); }
__device__ __forceinline__ void tc_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tc_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }
template <bool E8>
__device__ __forceinline__ void pair_mma(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t accumulate) {
    if constexpr (E8)
        asm volatile(
            "{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\t"
            "tcgen05.mma.cta_group::2.kind::f8f6f4 [%0], %1, %2, %3, p;\n\t}" ::"r"(d),
            "l"(a), "l"(b), "r"(idesc), "r"(accumulate)
            : "memory");
    else
        asm volatile(
            "{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\t"
            "tcgen05.mma.cta_group::2.kind::f16 [%0], %1, %2, %3, p;\n\t}" ::"r"(d),
            "l"(a), "l"(b), "r"(idesc), "r"(accumulate)
            : "memory");
}
// arrive on `bar` of both CTAs when the MMAs issued so far have completed
__device__ __forceinline__ void pair_commit(uint64_t* bar) {
    asm volatile(
        "tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;" ::"r"(
            smem_u32(bar)),
        "h"((uint16_t)3)
        : "memory");
}
// 16 lanes x 64 columns: of each 8 columns, thread t gets columns 2 (t % 4) and + 1 of lanes t / 4 (v[4 j], v[4 j + 1])
// and t / 4 + 8 (v[4 j + 2], v[4 j + 3])
__device__ __forceinline__ void tc_ld64(uint32_t taddr, uint32_t (&r)[32]) {
    asm volatile(
        "tcgen05.ld.sync.aligned.16x256b.x8.b32 "
        "{%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31}, [%32];"
        : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]),
          "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]), "=r"(r[16]),
          "=r"(r[17]), "=r"(r[18]), "=r"(r[19]), "=r"(r[20]), "=r"(r[21]), "=r"(r[22]), "=r"(r[23]), "=r"(r[24]),
          "=r"(r[25]), "=r"(r[26]), "=r"(r[27]), "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), "=r"(r[31])
        : "r"(taddr)
        : "memory");
}
__device__ __forceinline__ void tc_ld16(uint32_t taddr, uint32_t (&r)[8]) {  // 16 columns
    asm volatile("tcgen05.ld.sync.aligned.16x256b.x2.b32 {%0,%1,%2,%3,%4,%5,%6,%7}, [%8];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7])
                 : "r"(taddr)
                 : "memory");
}
__device__ __forceinline__ void tc_ld_wait16(uint32_t (&a)[8], uint32_t (&b)[8]) {
    asm volatile("tcgen05.wait::ld.sync.aligned;"
                 : "+r"(a[0]), "+r"(a[1]), "+r"(a[2]), "+r"(a[3]), "+r"(a[4]), "+r"(a[5]), "+r"(a[6]), "+r"(a[7]),
                   "+r"(b[0]), "+r"(b[1]), "+r"(b[2]), "+r"(b[3]), "+r"(b[4]), "+r"(b[5]), "+r"(b[6]), "+r"(b[7])
                 :
                 : "memory");
}
__device__ __forceinline__ void tc_ld32(uint32_t taddr, uint32_t (&r)[32]) {  // 32 lanes x 32 columns, a lane a thread
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x32.b32 "
        "{%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31}, [%32];"
        : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]),
          "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]), "=r"(r[16]),
          "=r"(r[17]), "=r"(r[18]), "=r"(r[19]), "=r"(r[20]), "=r"(r[21]), "=r"(r[22]), "=r"(r[23]), "=r"(r[24]),
          "=r"(r[25]), "=r"(r[26]), "=r"(r[27]), "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), "=r"(r[31])
        : "r"(taddr)
        : "memory");
}
// the values of the loads before: not to be used earlier
__device__ __forceinline__ void tc_ld_wait(uint32_t (&r)[32]) {
    asm volatile("tcgen05.wait::ld.sync.aligned;"
                 : "+r"(r[0]), "+r"(r[1]), "+r"(r[2]), "+r"(r[3]), "+r"(r[4]), "+r"(r[5]), "+r"(r[6]), "+r"(r[7]),
                   "+r"(r[8]), "+r"(r[9]), "+r"(r[10]), "+r"(r[11]), "+r"(r[12]), "+r"(r[13]), "+r"(r[14]), "+r"(r[15]),
                   "+r"(r[16]), "+r"(r[17]), "+r"(r[18]), "+r"(r[19]), "+r"(r[20]), "+r"(r[21]), "+r"(r[22]), "+r"(r[23]),
                   "+r"(r[24]), "+r"(r[25]), "+r"(r[26]), "+r"(r[27]), "+r"(r[28]), "+r"(r[29]), "+r"(r[30]), "+r"(r[31])
                 :
                 : "memory");
}
// shared-memory descriptors with the 128-byte swizzle: k along the 128-byte rows (atoms of 8 rows, 1024 bytes apart) ...
__device__ __forceinline__ uint64_t desc_k(uint32_t saddr) {
    return (uint64_t)((saddr & 0x3FFFFu) >> 4) | (uint64_t)1 << 16 | (uint64_t)(1024 >> 4) << 32 | (uint64_t)1 << 46 |
           (uint64_t)2 << 61;
}
// ... or 64 weight rows along them (8 of k an atom, `lbo` bytes between blocks of 64 weight rows)
__device__ __forceinline__ uint64_t desc_mn(uint32_t saddr, uint32_t lbo) {
    return (uint64_t)((saddr & 0x3FFFFu) >> 4) | (uint64_t)(lbo >> 4) << 16 | (uint64_t)(1024 >> 4) << 32 |
           (uint64_t)1 << 46 | (uint64_t)2 << 61;
}

// pairs of fp32 in one instruction
using f32x2 = unsigned long long;
__device__ __forceinline__ f32x2 pack2(uint32_t a, uint32_t b) { return (f32x2)b << 32 | a; }
__device__ __forceinline__ float lo2(f32x2 v) { return __uint_as_float((uint32_t)v); }
__device__ __forceinline__ float hi2(f32x2 v) { return __uint_as_float((uint32_t)(v >> 32)); }
__device__ __forceinline__ f32x2 fma2(f32x2 a, f32x2 b, f32x2 c) {
    f32x2 d;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(d) : "l"(a), "l"(b), "l"(c));
    return d;
}
__device__ __forceinline__ f32x2 add2(f32x2 a, f32x2 b) {
    f32x2 d;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(a), "l"(b));
    return d;
}

// Registers: the warps that keep the sums get those that the others do not need. Of the block's 384 x 168 = 64512,
// 128 x 56 + 256 x 224 = 64512 are dealt out.
__device__ __forceinline__ void regs_shrink() { asm volatile("setmaxnreg.dec.sync.aligned.u32 56;"); }
__device__ __forceinline__ void regs_grow() { asm volatile("setmaxnreg.inc.sync.aligned.u32 224;"); }

__device__ __forceinline__ uint32_t bf16x2(f32x2 v) {
    const __nv_bfloat162 b = __floats2bfloat162_rn(lo2(v), hi2(v));
    return *reinterpret_cast<const uint32_t*>(&b);
}
// four 8 x 8 matrices, each turned round: lane i gives the place of row i % 8 of matrix i / 8
__device__ __forceinline__ void stmatrix(uint32_t to, uint32_t a, uint32_t b, uint32_t c, uint32_t d) {
    asm volatile("stmatrix.sync.aligned.m8n8.x4.trans.shared.b16 [%0], {%1, %2, %3, %4};" ::"r"(to), "r"(a), "r"(b), "r"(c),
                 "r"(d)
                 : "memory");
}

// Tiles of a group of n rows, and rows of each.
__device__ __forceinline__ int tiles_of(int n) { return (n + kMaxTileRows - 1) / kMaxTileRows; }
__device__ __forceinline__ int tile_rows(int n, int tiles) { return ((n + tiles - 1) / tiles + 15) / 16 * 16; }

// A pair's way through its tiles and parts of tiles.
struct Walk {
    int round = 0, at = -1;
    template <bool XM>
    __device__ bool next(const Shared& sh, int n_groups, int w_tiles, Seg& s) {
        const Parts& P = sh.parts;
        const int pair = blockIdx.x >> 1;
        if (round < P.whole) {
            s.tile = round * P.pairs + pair;
            s.rest = -1;
            s.k0 = 0;
            s.k1 = P.steps;
            ++round;
        } else {
            if (pair >= P.sharers) return false;
            if (at < 0) at = P.begin(pair);
            const int end = P.begin(pair + 1);
            if (at >= end) return false;
            s.rest = at / P.steps;
            s.tile = P.whole * P.pairs + s.rest;
            s.k0 = at - s.rest * P.steps;
            s.k1 = min(P.steps, s.k0 + (end - at));
            at += s.k1 - s.k0;
        }
        int lo = 0, hi = n_groups;  // the last group whose first tile is not behind
        while (hi - lo > 1) {
            const int mid = (lo + hi) / 2;
            if (sh.first[mid] <= s.tile) lo = mid;
            else hi = mid;
        }
        s.g = lo;
        int t = s.tile - sh.first[lo];
        const int n = sh.rows[lo], tiles = tiles_of(n);
        const int band = t / (kBand * w_tiles), width = min(kBand, tiles - band * kBand);
        t -= band * kBand * w_tiles;
        s.wt = t / width;
        const int j = band * kBand + t % width;
        const int high = XM ? kMaxTileRows : tile_rows(n, tiles);
        s.row0 = sh.row0[lo] + j * high;
        s.rows = max(0, min(high, n - j * high));
        s.cols = high;
        return true;
    }
};

// XM (e4m3): the rows of x are the MMA's M, always 256 of them, and the weights its N. What a lane of tensor memory holds
// then belongs to one row of x, with one scale, and 32 lanes can be read at a time: a load of 16 lanes (of columns that
// have scales of their own) takes as long, and for wide tiles that is what bound e4m3 products: 8192 rows, 4096 x 14336,
// 424 -> 346 us. Narrow tiles would be mostly zeros.
template <bool E8, bool GATED, bool KN, bool XM>
struct Kind {
    static constexpr int kStep = E8 ? 128 : 64;          // elements of k of a stage
    // Stages of an accumulator, for bf16 outputs and for fp32 ones. A step of 16 of k takes off up to 2^-24 of the bf16 sum,
    // always toward 0: Gaussian rows are off by 9.9e-7 (2-norm) after 16 stages, 64 steps, which an output rounded to
    // bf16 (1.7e-3) does not show; after 8, 4 and 2 by 4.8e-7, 2.4e-7 and 1.6e-7. More hand-overs cost time where the tensor cores
    // bound: 16, 8, 4 and 2 stages, 8192 rows, 14336 x 4096, bf16 outputs 496, 514, 541 and 592 us, fp32 ones 548, 608, 635
    // and 653; 4096 x 14336 by rows of k, fp32 ones 532, 547, 554 and 605; of 40 to 2400 rows the same within 2% down to 4.
    static constexpr int kChunk = E8 ? 1 : 16, kChunkF32 = E8 ? 1 : 4;
    static constexpr int kTileN = GATED ? 128 : 256;     // outputs of a tile
    static constexpr int kBoxes = GATED || KN ? 2 : 1;   // boxes of weights of a CTA's stage
    static constexpr int kOffW = XM ? kStageW : 0, kOffX = XM ? 0 : kStageW;  // in a stage: M's operand, then N's
    static constexpr uint32_t kIdesc = (1u << 4) | (E8 ? 0u : (1u << 7) | (1u << 10)) | (KN ? 1u << 15 : 0u) | (16u << 24);
};

// Bounded wait; the clock is read only now and then.
__device__ __forceinline__ bool wait_for(uint64_t* bar, unsigned parity, Shared& sh) {
    unsigned long long t0 = 0;
    for (int i = 1; !mbar_try_wait_sleep(bar, parity, 10000u); ++i) {
        if ((i & 255) != 0) continue;
        const unsigned long long t = global_ns();
        if (t0 == 0) t0 = t;
        else if (t - t0 > kWaitLimitNs) {
            sh.fail = 1;
            return false;
        }
    }
    return true;
}

template <bool E8, bool GATED, bool KN, bool XM>
__global__ void __cluster_dims__(2, 1, 1) __launch_bounds__(kCtaThreads, 1) k_grouped(const __grid_constant__ GroupedLaunch L) {
    using K = Kind<E8, GATED, KN, XM>;
    static_assert(!XM || (E8 && !KN), "");
    extern __shared__ __align__(1024) unsigned char sm_raw[];
    __shared__ Shared sh;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const uint32_t rank = cta_rank();
    const int chunk_stages = L.y_f32 ? K::kChunkF32 : K::kChunk;
    const int steps = (L.k + K::kStep - 1) / K::kStep, w_tiles = (L.n + K::kTileN - 1) / K::kTileN;

    // ---- set-up: barriers, tensor memory, the groups' tiles ----
    if (warp == 0) {
        pdl_wait();
        int tiles_before = 0, widest = 16;
        for (int e0 = 0; e0 < L.n_groups; e0 += kWarp) {
            const int e = e0 + lane;
            int a = 0, n = 0;
            if (e < L.n_groups) {
                a = L.offsets != nullptr ? L.offsets[e] : 0;
                const int b = L.offsets != nullptr ? L.offsets[e + 1] : L.rows;
                const bool ok = a >= 0 && b >= a && b <= L.rows;
                if (!ok && blockIdx.x == 0) atomicOr(L.status, kStatusBadIndex);
                n = ok ? b - a : 0;
                sh.row0[e] = a;
                sh.rows[e] = n;
            }
            const int tiles = tiles_of(n);
            if (n > 0) widest = XM ? kMaxTileRows : max(widest, tile_rows(n, tiles));
            int sum = tiles * w_tiles;
#pragma unroll
            for (int o = 1; o < kWarp; o <<= 1) {
                const int v = __shfl_up_sync(0xffffffffu, sum, o);
                if (lane >= o) sum += v;
            }
            if (e < L.n_groups) sh.first[e + 1] = tiles_before + sum;
            tiles_before += __shfl_sync(0xffffffffu, sum, kWarp - 1);
        }
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) widest = max(widest, __shfl_xor_sync(0xffffffffu, widest, o));
        if (lane == 0) {
            sh.first[0] = 0;
            sh.max_cols = widest;
            sh.parts.set(tiles_before, L.pairs, steps);
        }
    } else if (warp == 1 && lane == 0) {
        for (int s = 0; s < kMaxStages; ++s) {
            mbar_init(&sh.full[s], 1);
            mbar_init(&sh.empty[s], 1);
        }
        for (int b = 0; b < kMaxBufs; ++b) {
            mbar_init(&sh.tfull[b], E8 ? 1 + kScaleWarps : 1);
            mbar_init(&sh.sempty[b], kEpiWarps);
            mbar_init(&sh.tempty[b], 2 * kEpiWarps);
        }
        for (int b = 0; b < kEpiWarps / 2; ++b) mbar_init(&sh.met[b], 2);
        mbar_init(&sh.never, 1);
        sh.fail = 0;
        mbar_fence_init();
    } else if (warp == 2) {
        pdl_wait();  // (a CTA of the launch before may hold tensor memory)
        asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&sh.tmem)), "r"(512)
                     : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
    }
    pdl_wait();
    tc_before();
    __syncthreads();
    cluster_sync();
    tc_after();

    const uint32_t sm0 = (smem_u32(sm_raw) + 1023u) & ~1023u;
    // the smallest box of x that holds a CTA's half of the widest tile sets the size of a stage
    const int x_rows_max = max(8, 1 << (32 - __clz(sh.max_cols / 2 - 1)));
    const uint32_t stage_bytes = kStageW + x_rows_max * 128;
    const int stages = min(kMaxStages, kStageMem / (int)stage_bytes);
    // tensor memory holds two accumulators, or four where the widest tile has at most 128 columns (a warp's loads are of 64
    // columns from the first that it holds on, so that narrower accumulators would have to end before the last ones do)
    const int lg_bufs = sh.max_cols <= 128 ? 2 : 1, n_bufs = 1 << lg_bufs, buf_cols = 512 >> lg_bufs;
    Walk walk;

    if (warp < kEpiWarp0) {
        regs_shrink();
        if (warp == 0) {
            // ---- loads: lane i < kBoxes a box of weights, the next one the rows of x ----
            int st = 0, n_loaded = 0, group = -1;
            unsigned ph = 0;
            bool ok = true;
            Seg sg;
            while (ok && walk.next<XM>(sh, L.n_groups, w_tiles, sg)) {
                const GroupWeights* gw = L.weights + sg.g;
                const int x_rows = max(8, 1 << (32 - __clz(sg.cols / 2 - 1))), xi = __ffs(x_rows) - 4;
                const uint32_t bytes = 2u * (kStageW + x_rows * 128);
                const CUtensorMap* map = &L.x[xi];
                uint32_t off = K::kOffX;
                int cy = sg.row0 + (int)rank * (sg.cols / 2), cx = 0;  // coordinate of the box besides k's
                if (lane < K::kBoxes) {
                    if constexpr (GATED && XM) {  // 128 gate rows by one CTA, the same neurons' up rows by the other
                        map = rank ? &gw->u : &gw->w;
                        off = K::kOffW + lane * 8192;
                        cy = sg.wt * 128 + lane * 64;
                    } else if constexpr (GATED) {  // 64 gate rows, then the same neurons' up rows
                        map = lane ? &gw->u : &gw->w;
                        off = lane * 8192;
                        cy = sg.wt * 128 + (int)rank * 64;
                    } else if constexpr (KN) {
                        map = &gw->w;
                        off = lane * 8192;
                        cx = sg.wt * 256 + (int)rank * 128 + lane * 64;
                    } else {
                        map = &gw->w;
                        off = K::kOffW;
                        cy = sg.wt * 256 + (int)rank * 128;
                    }
                    if (sg.g != group) map_acquire(map);
                }
                group = sg.g;
                for (int k = sg.k0; k < sg.k1; ++k) {
                    if (n_loaded >= stages) ok = wait_for(&sh.empty[st], ph ^ 1u, sh);
                    ok = __all_sync(0xffffffffu, ok);
                    if (!ok) break;
                    if (rank == 0 && lane == 0) mbar_arrive_expect_tx(&sh.full[st], bytes);
                    __syncwarp();
                    const uint32_t dst = sm0 + st * stage_bytes + off, bar = in_cta(&sh.full[st], 0);
                    if (lane <= K::kBoxes) {
                        if (KN && lane < K::kBoxes) tma_box(dst, map, cx, k * K::kStep, bar);
                        else tma_box(dst, map, k * K::kStep, cy, bar);
                    }
                    ++n_loaded;
                    if (++st == stages) {
                        st = 0;
                        ph ^= 1u;
                    }
                }
            }
            // the last stages' releases come from the other CTA: wait for them before leaving
            if (n_loaded < stages) {
                st = 0;
                ph = 1;
            }
            for (int i = min(n_loaded, stages); ok && i > 0; --i) {
                ok = __all_sync(0xffffffffu, wait_for(&sh.empty[st], ph ^ 1u, sh));
                if (++st == stages) {
                    st = 0;
                    ph ^= 1u;
                }
            }
        } else if (warp == 1) {
            // ---- MMAs, by the first CTA. The whole warp runs the loop and one lane issues, so that what the MMAs take
            // is known to be the same for all lanes and stays in uniform registers. ----
            if (rank == 0) {
                const uint32_t tmem = uniform(sh.tmem), base = uniform(sm0), size = uniform(stage_bytes);
                const int n_st = (int)uniform((uint32_t)stages), lg = (int)uniform((uint32_t)lg_bufs), bufs = 1 << lg;
                int st = 0, chunk = 0;
                unsigned ph = 0;
                bool ok = true;
                Seg sg;
                while (ok && walk.next<XM>(sh, L.n_groups, w_tiles, sg)) {
                    const int half = (int)uniform((uint32_t)sg.cols) / 2;
                    const int k_end = (int)uniform((uint32_t)sg.k1);
                    int k = (int)uniform((uint32_t)sg.k0);
                    const uint32_t idesc = K::kIdesc | (uint32_t)(2 * half >> 3) << 17;
                    // A lane whose limit has passed goes on with the others to the tile's end, without waiting: the limit may
                    // pass for some lanes alone, and all of them have to take part in the election. (A vote at every
                    // stage instead: 8192 rows, 4096 x 14336 e4m3, 366 us for 360.)
                    for (; k < k_end; ++chunk) {
                        const int first = k, kc = min(k_end, k + chunk_stages), buf = chunk & (bufs - 1);
                        const uint32_t d = tmem + (buf << (9 - lg));
                        for (; k < kc; ++k) {
                            // the accumulator is what is waited for longest: its barrier last
                            if (ok) ok = wait_for(&sh.full[st], ph, sh);
                            if (ok && k == first && chunk >= bufs) ok = wait_for(&sh.tempty[buf], ((chunk >> lg) & 1) ^ 1u, sh);
                            tc_after();
                            const uint32_t a0 = base + st * size;
                            const uint64_t bd = desc_k(a0 + kStageW);
                            const uint64_t ad = KN ? desc_mn(a0, 8192) : desc_k(a0);
                            if (elect_one() && ok) {
#pragma unroll
                                for (int i = 0; i < 4; ++i)
                                    pair_mma<E8>(d, ad + (KN ? 128 : 2) * i, bd + 2 * i, idesc, k > first || i > 0);
                                if (k + 1 == kc) pair_commit(&sh.tfull[buf]);
                                pair_commit(&sh.empty[st]);
                            }
                            __syncwarp();
                            if (++st == n_st) {
                                st = 0;
                                ph ^= 1u;
                            }
                        }
                    }
                    ok = __all_sync(0xffffffffu, ok);
                }
            }
            __syncwarp();
        } else if constexpr (E8) {
            // ---- scales, by a warp for each CTA's half of the rows of x: those of an accumulator's columns times that of the
            // weights. They are copied kScaleSlots - 1 stages ahead: an L2 access takes longer than a stage's MMAs. ----
            const int half = warp - 2;
            int chunk = 0;
            bool ok = true;
            Seg sg;
            while (ok && walk.next<XM>(sh, L.n_groups, w_tiles, sg)) {
                // this warp's part: columns [c0, c0 + cols) of an accumulator, XM: lanes of it
                const int cols = XM ? 64 : sg.cols / 2, c0 = half * cols, first = XM ? (int)rank * 128 + c0 : c0;
                const int last_block = (L.n + kScaleBlock - 1) / kScaleBlock - 1;
                const GroupWeights* gw = L.weights + sg.g;
                // one scale of the weights (XM: two) for all outputs of a tile, and one for the up product
                const float* ws = gw->ws + (size_t)(GATED ? sg.wt : min(2 * sg.wt + (XM ? 0 : (int)rank), last_block)) * steps + sg.k0;
                const float* us = GATED ? gw->us + (size_t)sg.wt * steps + sg.k0
                                  : XM  ? gw->ws + (size_t)min(2 * sg.wt + 1, last_block) * steps + sg.k0
                                        : nullptr;
                const float* xs = L.x_scale + (size_t)sg.k0 * L.ld_scale + sg.row0 + first + lane;
                const int in = min(cols, sg.rows - first) - lane;  // this lane copies columns lane + 32 i, 32 i < in
                int ahead = sg.k0, slot = chunk;
                auto fetch = [&]() {
                    if (ahead < sg.k1) {
                        float* to = &sh.raw[slot & (kScaleSlots - 1)][half][0][lane];
#pragma unroll
                        for (int i = 0; i < 4; ++i) cp4(to + 32 * i, 32 * i < in ? xs + 32 * i : L.x_scale, 32 * i < in ? 4 : 0);
                        cp4(to + 128, ws++, 4);
                        if (GATED || XM) cp4(to + 160, us++, 4);
                        xs += L.ld_scale;
                    }
                    cp_commit();
                    ++ahead;
                    ++slot;
                };
                for (int i = 0; i < kScaleSlots - 1; ++i) fetch();
                for (int k = sg.k0; k < sg.k1; ++k, ++chunk) {
                    fetch();  // (what a lane copies it reads itself)
                    cp_wait<kScaleSlots - 1>();
                    const float* raw = &sh.raw[chunk & (kScaleSlots - 1)][half][0][lane];
                    const float g = raw[128], u = GATED || XM ? raw[160] : 0.0f;
                    const int buf = chunk & (n_bufs - 1);
                    if (chunk >= n_bufs)
                        ok = __all_sync(0xffffffffu, wait_for(&sh.sempty[buf], ((chunk >> lg_bufs) & 1) ^ 1u, sh));
                    if (!ok) break;
                    float* to = &sh.scale[0][buf * buf_cols + c0 + lane];
#pragma unroll
                    for (int i = 0; i < 4; ++i)
                        if (32 * i + lane < cols) {
                            to[32 * i] = raw[32 * i] * g;
                            if (GATED || XM) to[512 + 32 * i] = raw[32 * i] * u;
                        }
                    __syncwarp();
                    if (lane == 0) mbar_arrive(&sh.tfull[buf]);
                }
            }
        }
    } else {
        regs_grow();
        // ---- sums: a warp may read the 32 lanes of its number modulo 4; it holds those of half ew / 4 of a tile's columns ----
        const int ew = warp - kEpiWarp0, q = warp & 3, half = ew >> 2;
        const uint32_t lane_addr = sh.tmem + ((uint32_t)(32 * q) << 16);
        int chunk = 0;
        bool ok = true;
        // gated: a gate warp and the up warp of the same neurons wait for each other
        const int both = half * 2 + (q & 1);
        unsigned met = 0;
        auto meet = [&]() {
            __syncwarp();
            if (lane == 0) mbar_arrive(&sh.met[both]);
            const bool here = __all_sync(0xffffffffu, wait_for(&sh.met[both], met & 1u, sh));
            ++met;
            return here;
        };
        const Seg& sg = sh.seg[ew];
        while (ok) {
            {
                Seg now;
                if (!walk.next<XM>(sh, L.n_groups, w_tiles, now)) break;
                __syncwarp();
                if (lane == 0) sh.seg[ew] = now;
                __syncwarp();
            }
            const int cols = sg.cols / 2, c0 = half * cols;  // this warp's columns, a multiple of 8 ...
            const int w0 = min(cols, 64), w1 = cols - w0;  // ... in two chunks
            f32x2 acc[2][2][16];  // [16 lanes][64 columns][of 8 columns: lanes t / 4, lanes t / 4 + 8]
#pragma unroll
            for (int i = 0; i < 64; ++i) acc[i >> 5][(i >> 4) & 1][i & 15] = 0ull;
            auto release = [&](int buf) {
                tc_before();
                __syncwarp();
                if (elect_one()) {
                    arrive_at(in_cta(&sh.tempty[buf], 0));
                    if (E8) mbar_arrive(&sh.sempty[buf]);
                }
            };
            auto filled = [&](int buf) {
                ok = __all_sync(0xffffffffu, wait_for(&sh.tfull[buf], (chunk >> lg_bufs) & 1, sh));
                tc_after();
                return ok;
            };
            if constexpr (XM) {
                // lane = row of x; acc[b][c]: columns 32 b .. + 31 of chunk c. Plain: the two chunks follow on one another, from
                // column 128 half on; gated: chunk 0 gate values, chunk 1 the up values of the same 64 neurons.
                const float* scale = &sh.scale[GATED ? 0 : half][32 * q + lane];
                for (int left = sg.k1 - sg.k0; left > 0; --left, ++chunk) {
                    const int buf = chunk & 1;
                    if (!filled(buf)) break;
                    const uint32_t s0 = __float_as_uint(scale[buf * 256]), s1 = GATED ? __float_as_uint(scale[512 + buf * 256]) : s0;
#pragma unroll
                    for (int c = 0; c < 2; ++c) {
                        const f32x2 sc = c ? pack2(s1, s1) : pack2(s0, s0);
                        const uint32_t from = lane_addr + buf * 256 + (GATED ? 64 * half + 128 * c : 128 * half + 64 * c);
#pragma unroll
                        for (int b = 0; b < 2; ++b) {
                            uint32_t r[32];
                            tc_ld32(from + 32 * b, r);
                            tc_ld_wait(r);
                            if (b == 1 && c == 1) release(buf);
#pragma unroll
                            for (int j = 0; j < 16; ++j) acc[b][c][j] = fma2(pack2(r[2 * j], r[2 * j + 1]), sc, acc[b][c][j]);
                        }
                    }
                }
            } else if constexpr (E8) {
                const float* scale = &sh.scale[GATED ? q >> 1 : 0][c0 + 2 * (lane & 3)];
                for (int left = sg.k1 - sg.k0; left > 0; --left, ++chunk) {
                    const int buf = chunk & (n_bufs - 1);
                    if (!filled(buf)) break;
                    const uint32_t from = lane_addr + buf * buf_cols + c0;
                    const f32x2* s2 = reinterpret_cast<const f32x2*>(scale + buf * buf_cols);
                    if (cols <= 16) {  // both halves of the lanes at once
                        uint32_t r0[8], r1[8];
                        tc_ld16(from, r0);
                        tc_ld16(from + (16u << 16), r1);
                        const f32x2 sa = s2[0], sb = s2[4];
                        tc_ld_wait16(r0, r1);
                        release(buf);
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            acc[0][0][i] = fma2(pack2(r0[2 * i], r0[2 * i + 1]), i < 2 ? sa : sb, acc[0][0][i]);
                            acc[1][0][i] = fma2(pack2(r1[2 * i], r1[2 * i + 1]), i < 2 ? sa : sb, acc[1][0][i]);
                        }
                        continue;
                    }
#pragma unroll
                    for (int c = 0; c < 2; ++c) {
                        if (c == 1 && w1 == 0) break;
                        uint32_t r[32];
                        tc_ld64(from + 64 * c, r);
                        f32x2 sc[8];
#pragma unroll
                        for (int j = 0; j < 8; ++j) sc[j] = s2[32 * c + 4 * j];
#pragma unroll
                        for (int h = 0; h < 2; ++h) {
                            tc_ld_wait(r);
                            if (h == 1 && (c == 1 || w1 == 0)) release(buf);
#pragma unroll
                            for (int j = 0; j < 8; ++j) {
                                acc[h][c][2 * j] = fma2(pack2(r[4 * j], r[4 * j + 1]), sc[j], acc[h][c][2 * j]);
                                acc[h][c][2 * j + 1] = fma2(pack2(r[4 * j + 2], r[4 * j + 3]), sc[j], acc[h][c][2 * j + 1]);
                            }
                            if (h == 0) tc_ld64(from + 64 * c + (16u << 16), r);
                        }
                    }
                }
            } else {
                for (int left = sg.k1 - sg.k0; left > 0; left -= chunk_stages, ++chunk) {
                    const int buf = chunk & (n_bufs - 1);
                    if (!filled(buf)) break;
#pragma unroll
                    for (int c = 0; c < 2; ++c) {
                        if (c == 1 && w1 == 0) break;
#pragma unroll
                        for (int h = 0; h < 2; ++h) {
                            uint32_t r[32];
                            tc_ld64(lane_addr + ((uint32_t)(16 * h) << 16) + buf * buf_cols + c0 + 64 * c, r);
                            tc_ld_wait(r);
#pragma unroll
                            for (int j = 0; j < 8; ++j) {
                                acc[h][c][2 * j] = add2(acc[h][c][2 * j], pack2(r[4 * j], r[4 * j + 1]));
                                acc[h][c][2 * j + 1] = add2(acc[h][c][2 * j + 1], pack2(r[4 * j + 2], r[4 * j + 3]));
                            }
                        }
                    }
                    release(buf);
                }
            }
            if (!ok) break;
            if (sg.k1 - sg.k0 < steps) {
                // A part of a tile: left in global memory; the warp that comes last adds the parts in the order of k.
                const Parts& P = sh.parts;
                const int pair = blockIdx.x >> 1;
                const int s0 = sg.rest * steps;
                const int p0 = P.owner(s0), p1 = P.owner(s0 + steps - 1);
                auto part_of = [&](int p) {  // a pair's first tile is in its slot 0, its last one in slot 1
                    const int slot = (XM ? P.begin_called(p) : P.begin(p)) >= s0 ? 0 : 1;
                    return reinterpret_cast<f32x2*>(L.partial) +
                           ((size_t)((p * 2 + slot) * 2 + (int)rank) * kEpiWarps + ew) * (L.part_chunks * 1024) + lane;
                };
                // value i of a chunk of `width` columns: whether its 8 columns are any of the tile's
                auto in = [](int i, int width) { return 8 * ((i & 15) >> 1) < width; };
                f32x2* to = part_of(pair);
#pragma unroll
                for (int c = 0; c < 2; ++c)
#pragma unroll
                    for (int i = 0; i < 32; ++i)
                        if (in(i, c ? w1 : w0)) __stcg(to + (c * 32 + i) * kWarp, acc[i >> 4][c][i & 15]);
                __threadfence();
                __syncwarp();
                unsigned* count = L.arrived + ((size_t)sg.rest * 2 + rank) * kEpiWarps + ew;
                unsigned before = 0;
                if constexpr (GATED && !XM) {  // a gate and an up warp finish a tile together, so they are counted as one
                    ok = meet();
                    if (q < 2 && lane == 0) sh.before[both] = atomicAdd(count, 1u);
                    ok = ok && meet();
                    if (!ok) break;
                    before = sh.before[both];
                } else {
                    if (lane == 0) before = atomicAdd(count, 1u);
                    before = __shfl_sync(0xffffffffu, before, 0);
                }
                if ((int)before != p1 - p0) continue;
                __threadfence();
                if (lane == 0 && (!GATED || XM || q < 2)) *count = 0u;
#pragma unroll
                for (int i = 0; i < 64; ++i) acc[i >> 5][(i >> 4) & 1][i & 15] = 0ull;
                auto join_few = [&](auto groups) {  // of 8 columns
                    constexpr int kG = decltype(groups)::value;
                    for (int p = p0; p <= p1; ++p) {
                        const f32x2* from = part_of(p);
#pragma unroll
                        for (int i = 0; i < 4 * kG; ++i) {
                            f32x2& a = acc[i / (2 * kG)][0][i % (2 * kG)];
                            a = add2(a, __ldcg(from + (16 * (i / (2 * kG)) + i % (2 * kG)) * kWarp));
                        }
                    }
                };
                if (!XM && cols == 8) {
                    join_few(std::integral_constant<int, 1>());
                } else if (!XM && cols == 16) {
                    join_few(std::integral_constant<int, 2>());
                } else {
#pragma unroll 1
                    for (int p = p0; p <= p1; ++p) {
                        const f32x2* from = part_of(p);
#pragma unroll
                        for (int c = 0; c < 2; ++c) {
                            if (c == 1 && w1 == 0) break;
#pragma unroll
                            for (int h = 0; h < 2; ++h) {
                                f32x2 v[16];
#pragma unroll
                                for (int i = 0; i < 16; ++i) v[i] = __ldcg(from + (c * 32 + h * 16 + i) * kWarp);
#pragma unroll
                                for (int i = 0; i < 16; ++i) acc[h][c][i] = add2(acc[h][c][i], v[i]);
                                asm volatile("" ::: "memory");  // no more loads at once than there are registers for
                            }
                        }
                    }
                }
            }
            if constexpr (XM) {
                // a thread's row of y, `kOut` outputs from n0 on, in pieces of 64 bytes that are turned round in shared memory
                // so that 4 lanes write one row's, as whole sectors
                constexpr int kOut = GATED ? 64 : 128;
                const int row = (int)rank * 128 + 32 * q, n0 = GATED ? sg.wt * 128 + 64 * half : sg.wt * 256 + 128 * half;
                if constexpr (GATED) {
#pragma unroll
                    for (int i = 0; i < 32; ++i) {
                        f32x2& a = acc[i >> 4][0][i & 15];
                        const f32x2 u = acc[i >> 4][1][i & 15];
                        a = pack2(__float_as_uint(lo2(a) > 0.0f && lo2(u) > 0.0f ? lo2(a) * lo2(u) : 0.0f),
                                  __float_as_uint(hi2(a) > 0.0f && hi2(u) > 0.0f ? hi2(a) * hi2(u) : 0.0f));
                    }
                }
                const int rows = sg.rows - row;  // of this warp's 32
                if (L.y_vec && n0 + kOut <= L.n) {
                    unsigned char* turn = sh.turn[ew];
                    const int swz = (lane >> 1) & 3, r8 = lane >> 2;  // chunk c of row r lies at c ^ (r / 2 % 4)
                    const uint32_t at = smem_u32(turn) + lane * 64;
                    const size_t size = L.y_f32 ? 4 : 2;
                    char* y = static_cast<char*>(L.y) + ((size_t)(sg.row0 + row) * L.ldy + n0) * size + (lane & 3) * 16;
                    auto write_out = [&](int piece) {
                        __syncwarp();
#pragma unroll
                        for (int r0 = 0; r0 < 32; r0 += 8) {
                            const int r = r0 + r8;
                            const uint4 v = lds128(turn + r * 64 + (((lane & 3) ^ ((r >> 1) & 3)) << 4));
                            if (r < rows) *reinterpret_cast<uint4*>(y + (size_t)r * L.ldy * size + piece * 64) = v;
                        }
                        __syncwarp();
                    };
                    if (L.y_f32) {
#pragma unroll
                        for (int p = 0; p < kOut / 16; ++p) {
#pragma unroll
                            for (int c = 0; c < 4; ++c) {
                                const f32x2 a = acc[(p >> 1) & 1][p >> 2][(p & 1) * 8 + 2 * c], b = acc[(p >> 1) & 1][p >> 2][(p & 1) * 8 + 2 * c + 1];
                                sts128(at + ((c ^ swz) << 4), (uint32_t)a, (uint32_t)(a >> 32), (uint32_t)b, (uint32_t)(b >> 32));
                            }
                            write_out(p);
                        }
                    } else {
#pragma unroll
                        for (int p = 0; p < kOut / 32; ++p) {
#pragma unroll
                            for (int c = 0; c < 4; ++c) {
                                const f32x2* v = &acc[p & 1][p >> 1][4 * c];
                                sts128(at + ((c ^ swz) << 4), bf16x2(v[0]), bf16x2(v[1]), bf16x2(v[2]), bf16x2(v[3]));
                            }
                            write_out(p);
                        }
                    }
                } else if (lane < rows) {
#pragma unroll
                    for (int i = 0; i < kOut / 2; ++i) {
                        const f32x2 v = acc[(i >> 4) & 1][i >> 5][i & 15];
                        const int n = n0 + 2 * i;
                        const size_t at = (size_t)(sg.row0 + row + lane) * L.ldy + n;
                        if (L.y_f32) {
                            if (n < L.n) static_cast<float*>(L.y)[at] = lo2(v);
                            if (n + 1 < L.n) static_cast<float*>(L.y)[at + 1] = hi2(v);
                        } else {
                            if (n < L.n) static_cast<__nv_bfloat16*>(L.y)[at] = __float2bfloat16_rn(lo2(v));
                            if (n + 1 < L.n) static_cast<__nv_bfloat16*>(L.y)[at + 1] = __float2bfloat16_rn(hi2(v));
                        }
                    }
                }
                __syncwarp();
                continue;
            } else {
                // outputs: [16 lanes h][8 lanes r] of each 8 columns
                const int mlane = lane >> 2;
                int n0 = sg.wt * 256 + (int)rank * 128 + q * 32, cb = c0;  // the warp's first output and first column
                unsigned char* turn = sh.turn[ew];
                if constexpr (GATED) {
                    // Warp q < 2 holds the gate values and warp q + 2 the up values of the same neurons: the first finishes
                    // the first chunk of columns, the second the other, each with what the other sends it, 16 columns at a time.
                    n0 = sg.wt * 128 + (int)rank * 64 + (q & 1) * 32;
                    cb = q < 2 ? c0 : c0 + w0;
                    f32x2* mine = reinterpret_cast<f32x2*>(turn) + lane;
                    const f32x2* theirs = reinterpret_cast<const f32x2*>(sh.turn[ew ^ 2]) + lane;
    #pragma unroll
                    for (int p = 0; p < 4; ++p) {
                        if (16 * p >= w0) break;
    #pragma unroll
                        for (int i = 0; i < 8; ++i) mine[i * kWarp] = q < 2 ? acc[i >> 2][1][4 * p + (i & 3)] : acc[i >> 2][0][4 * p + (i & 3)];
                        ok = ok && meet();
    #pragma unroll
                        for (int i = 0; i < 8; ++i) {
                            const f32x2 a = q < 2 ? acc[i >> 2][0][4 * p + (i & 3)] : acc[i >> 2][1][4 * p + (i & 3)], b = theirs[i * kWarp];
                            acc[i >> 2][0][4 * p + (i & 3)] =
                                pack2(__float_as_uint(lo2(a) > 0.0f && lo2(b) > 0.0f ? lo2(a) * lo2(b) : 0.0f),
                                      __float_as_uint(hi2(a) > 0.0f && hi2(b) > 0.0f ? hi2(a) * hi2(b) : 0.0f));
                        }
                        ok = ok && meet();  // both have read before either writes there again
                    }
                    if (!ok) break;
                }
                constexpr int kC = GATED ? 1 : 2;
                const int width[2] = {GATED && q >= 2 ? w1 : w0, GATED ? 0 : w1};  // columns of chunk 0 and 1 that the warp finishes
                if (L.y_f32) {
                    float* y = static_cast<float*>(L.y) + (size_t)sg.row0 * L.ldy + n0 + mlane;
    #pragma unroll
                    for (int c = 0; c < kC; ++c)
    #pragma unroll
                        for (int i = 0; i < 16; ++i) {
                            if (8 * (i >> 1) >= width[c]) continue;
                            const int col = cb + c * w0 + 8 * (i >> 1) + 2 * (lane & 3);  // and + 1
                            float* at = y + (size_t)col * L.ldy + 8 * (i & 1);
    #pragma unroll
                            for (int h = 0; h < 2; ++h) {
                                const bool in = n0 + mlane + 8 * (i & 1) + 16 * h < L.n;
                                if (in && col < sg.rows) at[16 * h] = lo2(acc[h][c][i]);
                                if (in && col + 1 < sg.rows) at[16 * h + L.ldy] = hi2(acc[h][c][i]);
                            }
                        }
                } else if (L.y_vec && n0 + 32 <= L.n) {
                    // bf16: 16 rows of y at a time are turned round in shared memory, so that a store writes whole sectors, 64
                    // bytes of a row. (Two bytes of 16 rows each, straight from the registers, held the tiles up: 8192 rows
                    // through an 8192 x 4096 matrix took 323 us against 289.)
                    constexpr int kPitch = 80;
                    const uint32_t to = smem_u32(turn) + (lane & 7) * kPitch + (lane >> 3) * 16;
                    __nv_bfloat16* y = static_cast<__nv_bfloat16*>(L.y) + (size_t)(sg.row0 + cb) * L.ldy + n0;
    #pragma unroll
                    for (int c = 0; c < kC; ++c)
    #pragma unroll
                        for (int p = 0; p < 4; ++p) {  // 16 columns: lanes 0-7 and 8-15 of the first 8, of the next 8
                            if (16 * p >= width[c]) continue;
                            const f32x2* v0 = &acc[0][c][4 * p];
                            const f32x2* v1 = &acc[1][c][4 * p];
                            __syncwarp();
                            stmatrix(to, bf16x2(v0[0]), bf16x2(v0[1]), bf16x2(v1[0]), bf16x2(v1[1]));
                            stmatrix(to + 8 * kPitch, bf16x2(v0[2]), bf16x2(v0[3]), bf16x2(v1[2]), bf16x2(v1[3]));
                            __syncwarp();
    #pragma unroll
                            for (int r0 = 0; r0 < 16; r0 += 8) {
                                const int r = r0 + (lane >> 2), col = c * w0 + 16 * p + r;
                                const uint4 v = lds128(turn + r * kPitch + (lane & 3) * 16);
                                if (16 * p + r < width[c] && cb + col < sg.rows)
                                    *reinterpret_cast<uint4*>(y + (size_t)col * L.ldy + (lane & 3) * 8) = v;
                            }
                        }
                } else {
                    __nv_bfloat16* y = static_cast<__nv_bfloat16*>(L.y) + (size_t)sg.row0 * L.ldy + n0 + mlane;
    #pragma unroll
                    for (int c = 0; c < kC; ++c)
    #pragma unroll
                        for (int i = 0; i < 16; ++i) {
                            if (8 * (i >> 1) >= width[c]) continue;
                            const int col = cb + c * w0 + 8 * (i >> 1) + 2 * (lane & 3);  // and + 1
                            __nv_bfloat16* at = y + (size_t)col * L.ldy + 8 * (i & 1);
    #pragma unroll
                            for (int h = 0; h < 2; ++h) {
                                const bool in = n0 + mlane + 8 * (i & 1) + 16 * h < L.n;
                                if (in && col < sg.rows) at[16 * h] = __float2bfloat16_rn(lo2(acc[h][c][i]));
                                if (in && col + 1 < sg.rows) at[16 * h + L.ldy] = __float2bfloat16_rn(hi2(acc[h][c][i]));
                            }
                        }
                }
            }
        }
        if (L.test_stall && ew == 0) wait_for(&sh.never, 0u, sh);
    }

    // ---- the end: no CTA leaves while the other may still signal or read it ----
    __syncthreads();  // no wait of the CTA can give up after this
    if (sh.fail) {    // copies may be in flight: give them time to land
        if (tid == 0) atomicOr(L.status, kStatusTimeout);
        const unsigned long long t0 = global_ns();
        while (global_ns() - t0 < 2000000ull) __nanosleep(1000);
    }
    tc_before();
    __syncwarp();
    cluster_sync();
    if (warp == 2) {
        tc_after();
        asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(sh.tmem), "r"(512) : "memory");
    }
}

constexpr int kDynSmem = kStageMem + 1024;

using Kernel = void (*)(GroupedLaunch);

template <typename F>
cudaError_t each_kernel(F&& f) {
    for (Kernel k : {k_grouped<false, false, false, false>, k_grouped<false, false, true, false>,
                     k_grouped<false, true, false, false>, k_grouped<true, false, false, false>,
                     k_grouped<true, true, false, false>, k_grouped<true, false, false, true>, k_grouped<true, true, false, true>}) {
        const cudaError_t e = f(k);
        if (e != cudaSuccess) return e;
    }
    return cudaSuccess;
}

Kernel pick(bool e4m3, bool gated, bool kn, bool xm) {
    if (e4m3 && xm) return gated ? k_grouped<true, true, false, true> : k_grouped<true, false, false, true>;
    if (e4m3) return gated ? k_grouped<true, true, false, false> : k_grouped<true, false, false, false>;
    if (gated) return k_grouped<false, true, false, false>;
    return kn ? k_grouped<false, false, true, false> : k_grouped<false, false, false, false>;
}

using EncodeFn = CUresult (*)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*,
                              const cuuint32_t*, const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle,
                              CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

EncodeFn encoder() {
    static const EncodeFn fn = []() -> EncodeFn {
        void* p = nullptr;
        cudaDriverEntryPointQueryResult found;
        if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &p, 12000, cudaEnableDefault, &found) != cudaSuccess ||
            found != cudaDriverEntryPointSuccess)
            return nullptr;
        return reinterpret_cast<EncodeFn>(p);
    }();
    return fn;
}

}  // namespace

bool grouped_map(CUtensorMap* m, const void* p, bool e4m3, int64_t cols, int64_t rows, int64_t ld, int box_rows) {
    const EncodeFn fn = encoder();
    if (!fn) return false;
    const int size = e4m3 ? 1 : 2;
    const cuuint64_t dims[2] = {(cuuint64_t)cols, (cuuint64_t)rows}, strides[1] = {(cuuint64_t)(ld * size)};
    const cuuint32_t box[2] = {(cuuint32_t)(128 / size), (cuuint32_t)box_rows}, one[2] = {1, 1};
    return fn(m, e4m3 ? CU_TENSOR_MAP_DATA_TYPE_UINT8 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 2, const_cast<void*>(p), dims,
              strides, box, one, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
              CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

cudaError_t prepare_grouped() {
    return each_kernel(
        [](Kernel k) { return cudaFuncSetAttribute(k, cudaFuncAttributeMaxDynamicSharedMemorySize, kDynSmem); });
}

namespace {
cudaLaunchConfig_t configure(int pairs, cudaStream_t stream) {
    cudaLaunchConfig_t cfg = launch_shape(dim3(2 * pairs), kCtaThreads, stream);
    cfg.dynamicSmemBytes = kDynSmem;
    return cfg;
}
}  // namespace

int grouped_pairs() {
    cudaLaunchConfig_t cfg = configure(1, nullptr);
    cudaLaunchAttribute at{};
    at.id = cudaLaunchAttributeClusterDimension;
    at.val.clusterDim = {2, 1, 1};
    cfg.attrs = &at;
    cfg.numAttrs = 1;
    int n = 0;
    if (cudaOccupancyMaxActiveClusters(&n, pick(true, true, false, true), &cfg) != cudaSuccess) {
        cudaGetLastError();
        return 0;
    }
    return n;
}

cudaError_t launch_grouped(const GroupedLaunch& a, bool e4m3, bool gated, bool kn, cudaStream_t stream) {
    return launch_after(pick(e4m3, gated, kn, grouped_x_is_m(e4m3, gated, a.rows, a.n_groups)), configure(a.pairs, stream), a);
}

}  // namespace tsffn
