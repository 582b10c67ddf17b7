// Attention of a chunk of new tokens over the pot and, causally, over itself, on the 5th-generation tensor cores (bf16).
//
// The query heads of a KV head share its keys: a unit's rows are folded token by token, row t * G + g, and a query tile is the
// rows of floor(128 / G) tokens (TMA fetches it as a box of G heads x tokens, whatever the strides).  Keys come in tiles of KT,
// first the pot's, then the chunk's.  Per tile and stream
//   S = Q K^T   128 x KT fp32 in tensor memory (both operands in shared memory, K-major, 128-byte swizzle)
//   softmax     a thread owns half of a row (one warp per scheduler and stream would be a chain of latencies: 1900 cycles a tile, two 1500): p = 2^(s c - m - 40),
//               l += p in fp32, and p as bf16 over S in tensor memory.  No maximum is taken: fp32 and bf16 have the same exponents, so p is as exact far above 1
//               as below.  The reference m is 0 unless the sum of the row's first tile is far from 1, and only a later tile whose sum passes 2^24 moves it (the row's sums and output
//               are then scaled down).  The 40 orders are what a row's weights can sum up to so: all p together stay below 1, and no sum of p v on the way is larger than the largest value.  Tiles with columns that some row does not see, those two kinds, and those of a row whose reference is beyond 2^12, take a general form that does take the maximum.  All exponentials are the
//               special-function unit's: a quarter of them as a polynomial on the FMA pipe took 1016 us for 4 streams x 2048 tokens over 6144 rows instead of 950
//               (in long runs the power limit holds the clock at 1.6 GHz, and what is issued costs power).
//   O += P V    P from tensor memory, V as it lies (channels contiguous: the N-major operand layout), 128 x D fp32 in tensor memory
// A block runs two streams so that the tensor core works on one while the other's softmax runs: two query tiles that share the
// key tiles (kSplit = false), or one query tile whose key tiles take turns (kSplit, for calls of few rows; merged at the
// end).  More than 128 channels: one stream, tensor memory holds one output.  Calls with fewer query tiles than
// SMs spread a tile's keys over a cluster whose blocks merge their results through distributed shared memory: nothing is
// exchanged through global memory, and the result does not depend on timing.
//
// Registers: 18 warps leave 96 a thread; the kernel spills 40 to 56 bytes, the general form of a tile 56 to 68.
// Warps: 0 loads (TMA), 1 issues the products, 2-9 / 10-17 softmax of the two streams (2-5, 10-13 the left half of the columns).  Between two streams' products the issuing warp waits for nothing but
// the next P: every look at a barrier costs about 90 cycles even if it has long been passed, and the tensor core's queue is shorter than that.
// (A warp for each stream's products: 1140 us against 1020 for 4 streams x 2048 tokens over 6144 rows, their products then alternate one by one and both are late.)
// All waits are bounded (wait_ns): one that runs out
// raises the block's give-up flag and IPOT_E_TIMEOUT; from then on nothing more is put in flight, and what is in flight is
// waited for before tensor memory is released.
#pragma once
#include "cluster.cuh"
#include "k_chunk_fma.cuh"   // chunk_tokens, chunk_ex2
#include "ops.h"
#include "ptx.cuh"

namespace ipotk {

constexpr int kCtRows = 128;
constexpr unsigned long long kChunkLandNs = 200ull * 1000 * 1000;
// Half a tile's sum of a row up to 2^24 leaves the reference where it is, and half a first tile's from 2^-12 on lets it be 0; both carry 2^-lift like all p.  2^40: two halves of up to 2^15
// tiles.  (At the other end a product with a value keeps bf16's bits above 2^-117, so values below 2^-65 may begin to lose some.)
constexpr float kChunkLift = 40.f, kChunkLifted = 1099511627776.f;   // and 2^40
constexpr float kChunkMost = 1.52587890625e-05f;                     // 2^24 2^-40
constexpr float kChunkLeast = 2.220446049250313e-16f;                // 2^-12 2^-40
// The row's maximum is a rounded product, and s c, not rounded before the reference is subtracted, misses it by up to half its last place: 1 from 2^24 on, further out more than the exponential's
// range.  The general form rounds the product, so that the maximum comes out as what it was taken for.  Up to here that differs from a plain tile's weights by 2^-13 of an order at most, and references
// are whole numbers, which add up exactly.  From here on a row takes nothing but the general form: its reference then waits in its threads' shared memory and is NaN in their registers, so that a
// plain tile's sum is NaN and the check that there is fails.  (4 streams x 2048 tokens over 6144 rows 953.4 -> 954.4 us, 2048 tokens into an empty pot 45.0 -> 45.6; a compare per tile and a
// flag across them cost 4.5 %.)
constexpr float kChunkFar = 4096.f;

template <int D, bool kSplit> struct ChunkTc {
    static constexpr int kStreams = D > 128 ? 1 : 2;
    static constexpr int kQTiles = kSplit ? 1 : 2;
    static constexpr int kKeys = D > 128 ? 64 : 128;
    static constexpr int kHalves = D / 64;                                   // blocks of 64 channels
    static constexpr uint32_t kKeyBlk = kKeys * 128, kStageBytes = kHalves * kKeyBlk;
    static constexpr uint32_t kQBlk = kCtRows * 128, kQBytes = kHalves * kQBlk;
    static constexpr int kStages = D == 64 ? 8 : D == 128 && kSplit ? 6 : 5;
    static constexpr int kPitch = D + 4;                                     // of a row of a partial result
    static constexpr uint32_t kOffStage = 0, kOffQ = kStages * kStageBytes, kOffStat = kOffQ + kQTiles * kQBytes;   // [2][128] float2
    static constexpr uint32_t kOffBar = kOffStat + kStreams * kCtRows * 8, kOffFlag = kOffBar + 8 * 32, kSmemBytes = kOffFlag + 16;
    static constexpr uint32_t kOutCol = 256;                                 // tensor memory: S of stream i at 128 i, O at 256 + D i
    static constexpr int kThreads = 64 + 256 * kStreams;
    static constexpr int kCols = kKeys / 2;                                  // of a softmax thread
    static constexpr bool kPush = D <= 128;                                  // room for what the cluster's other blocks send
    static constexpr uint32_t kPartBytes = kCtRows * kPitch * 4;
    static_assert(kPartBytes <= kStages * kStageBytes && (!kPush || 2 * kPartBytes + 8 * kPitch * 4 <= kStages * kStageBytes), "partial results take the stages' place");
    static_assert(kSmemBytes <= 232448, "shared memory of a block");
};
enum { kCbQ = 0, kCbFull = 1, kCbEmpty = 9, kCbS = 17, kCbP = 19, kCbO = 21, kCbDrain = 23, kCbMerge = 24, kCbCount = 25 };

// D[M x N] += A B with A in tensor memory (a row per lane, two bf16 per column).
__device__ __forceinline__ void tc_mma_bf16_ts(uint32_t d_tmem, uint32_t a_tmem, uint64_t b_desc, uint32_t idesc, uint32_t accumulate)
{
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "setp.ne.b32 p, %4, 0;\n\t"
        "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}"
        ::"r"(d_tmem), "r"(a_tmem), "l"(b_desc), "r"(idesc), "r"(accumulate) : "memory");
}
// An N-major operand with 128-byte swizzle: blocks of 64 columns `blk` bytes apart, 8 rows of K 1024 bytes apart.
__device__ __forceinline__ uint64_t smem_desc_sw128_nmajor(uint32_t addr, uint32_t blk)
{
    return (uint64_t)((addr & 0x3FFFFu) >> 4) | ((uint64_t)(blk >> 4) << 16) | ((uint64_t)(1024 >> 4) << 32) | ((uint64_t)1 << 46) | ((uint64_t)2 << 61);
}
__device__ __forceinline__ void tma_load_5d(uint32_t dst, const CUtensorMap *map, int c0, int c1, int c2, int c3, int c4, uint32_t bar)
{
    asm volatile(
        "cp.async.bulk.tensor.5d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4, %5, %6}], [%7];"
        ::"r"(dst), "l"(map), "r"(c0), "r"(c1), "r"(c2), "r"(c3), "r"(c4), "r"(bar) : "memory");
}
__device__ __forceinline__ void tmem_st32(uint32_t taddr, const uint32_t (&v)[32])
{
    asm volatile(
        "tcgen05.st.sync.aligned.32x32b.x32.b32 [%32], "
        "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, "
        "%16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31};"
        ::"r"(v[0]), "r"(v[1]), "r"(v[2]), "r"(v[3]), "r"(v[4]), "r"(v[5]), "r"(v[6]), "r"(v[7]),
          "r"(v[8]), "r"(v[9]), "r"(v[10]), "r"(v[11]), "r"(v[12]), "r"(v[13]), "r"(v[14]), "r"(v[15]),
          "r"(v[16]), "r"(v[17]), "r"(v[18]), "r"(v[19]), "r"(v[20]), "r"(v[21]), "r"(v[22]), "r"(v[23]),
          "r"(v[24]), "r"(v[25]), "r"(v[26]), "r"(v[27]), "r"(v[28]), "r"(v[29]), "r"(v[30]), "r"(v[31]),
          "r"(taddr) : "memory");
}

// A wait of at most wait_ns from its start.  flag: the block's give-up flag; with heed_flag off it is a wait for what is in flight and will land, which the block must not end before (its
// limit is never less than 200 ms).
__device__ __forceinline__ bool chunk_wait(uint32_t bar, uint32_t parity, volatile int *flag, const ChunkTcParams &p, bool heed_flag = true)
{
    unsigned long long t0 = 0;
    for (uint32_t i = 0;; ++i) {
        if (mbar_try_wait(bar, parity)) return true;
        if ((i & 31u) == 31u) {
            if (heed_flag && *flag) return false;
            const unsigned long long now = global_timer_ns();
            if (!t0) t0 = now;
            if (now - t0 > (heed_flag ? p.wait_ns : max(p.wait_ns, kChunkLandNs))) {
                *flag = 1;
                set_status(p.status, kStatusTimeout);
                return false;
            }
        }
    }
}

// The two warps that share 32 rows of a stream.
__device__ __forceinline__ void chunk_pair_sync(int id) { asm volatile("bar.sync %0, 64;" ::"r"(id) : "memory"); }
__device__ __forceinline__ bool chunk_pair_any(int id, bool x)
{
    uint32_t r;
    asm volatile(
        "{\n\t.reg .pred p, q;\n\tsetp.ne.u32 p, %1, 0;\n\t"
        "barrier.cta.red.or.pred q, %2, 64, p;\n\tselp.u32 %0, 1, 0, q;\n\t}"
        : "=r"(r) : "r"((uint32_t)x), "r"(id) : "memory");
    return r != 0;
}

// A tile of a warp's rows in general: one with columns that some row does not see, a first one whose sum is far from 1, one that left the range, and every one of a row with a far
// reference: the row's maximum becomes the reference if it is above it.
// W columns from ts on, of which this row sees `cols`; the other warp of the pair has the other half and takes part.  seen: the row's two maxima and, between two tiles, a far reference, each
// thread's in its half.  scale: whether O holds something already (W2 columns of it from `to` on are this warp's).  m: the reference + kChunkLift, as a plain tile takes it (-inf: none yet).
// Leaves p over the first half of its columns; (reference + kChunkLift or NaN, sum).
template <int W, int W2>
__device__ __noinline__ float2 chunk_tile_general(uint32_t ts, uint32_t to, int cols, float c, float m, float sum, bool valid, bool scale, float2 *seen, int half, int pair)
{
    float *mine = half ? &seen->y : &seen->x;
    m = isnan(m) ? *mine : m - kChunkLift;
    uint32_t v[W / 32][32];
    float mx[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
    for (int a = 0; a < W / 32; ++a) tmem_ld32(ts + 32 * a, v[a]);
#pragma unroll
    for (int a = 0; a < W / 32; ++a) {
        tmem_wait_ld(v[a]);
#pragma unroll
        for (int e = 0; e < 32; ++e) {
            if (32 * a + e >= cols) v[a][e] = __float_as_uint(-INFINITY);
            mx[e & 3] = fmaxf(mx[e & 3], __uint_as_float(v[a][e]));
        }
    }
    float top = fmaxf(fmaxf(mx[0], mx[1]), fmaxf(mx[2], mx[3]));
    *mine = top;
    chunk_pair_sync(pair);
    top = ceilf(fmaxf(seen->x, seen->y) * c);
    const bool moves = valid && top > m;
    if (__any_sync(0xffffffffu, moves)) {   // (the same rows, the same answer in both warps)
        const float to_m = moves ? top : m, f = moves ? chunk_ex2(m - to_m) : 1.f;   // (m = -inf: 0)
        sum *= f;
        m = to_m;
        if (scale) {
            // the product that last added to O has finished: it was issued before the one that made this tile's logits
#pragma unroll 1
            for (int a = 0; a < W2; a += 32) {
                uint32_t o[32];
                tmem_ld32(to + a, o);
                tmem_wait_ld(o);
#pragma unroll
                for (int e = 0; e < 32; ++e) o[e] = __float_as_uint(__uint_as_float(o[e]) * f);
                tmem_st32(to + a, o);
            }
        }
    }
    const float ref = m == -INFINITY ? 0.f : m;
    const float2 r2 = make_float2(-ref, -ref), l2 = make_float2(-kChunkLift, -kChunkLift);
    float s[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int a = 0; a < W / 32; ++a) {
        uint32_t h[16];
#pragma unroll
        for (int e = 0; e < 32; e += 2) {
            const float2 z = __fadd2_rn(__fadd2_rn(make_float2(__fmul_rn(__uint_as_float(v[a][e]), c), __fmul_rn(__uint_as_float(v[a][e + 1]), c)), r2), l2);
            const float x = chunk_ex2(z.x), y = chunk_ex2(z.y);   // (-inf: 0)
            s[e & 2] += x;
            s[(e & 2) + 1] += y;
            const __nv_bfloat162 b = __floats2bfloat162_rn(x, y);
            h[e >> 1] = *reinterpret_cast<const uint32_t *>(&b);
        }
        tmem_st16(ts + 16 * a, h);
    }
    chunk_pair_sync(pair);   // both maxima have been read (every call has the same barriers, whatever the two warps have read: after a wait that ran out they no longer go in step)
    if (fabsf(ref) >= kChunkFar) {
        *mine = m;
        m = NAN;
    } else {
        m += kChunkLift;
    }
    return make_float2(m, sum + ((s[0] + s[1]) + (s[2] + s[3])));
}

// The same for a tile that every row sees, against the reference as it is: 32 columns at a time, the next ones on their way meanwhile.  h: p, two to a register.
template <int W>
__device__ __forceinline__ float chunk_tile(uint32_t ts, float c, float m, uint32_t (&h)[W / 32][16])
{
    const float2 c2 = make_float2(c, c), r2 = make_float2(-m, -m);
    float2 s[2] = {make_float2(0.f, 0.f), make_float2(0.f, 0.f)};
    uint32_t v[W > 32 ? 2 : 1][32];
    tmem_ld32(ts, v[0]);
#pragma unroll
    for (int a = 0; a < W / 32; ++a) {
        tmem_wait_ld(v[a & 1]);
        if (a + 1 < W / 32) tmem_ld32(ts + 32 * (a + 1), v[(a + 1) & 1]);
#pragma unroll
        for (int e = 0; e < 32; e += 2) {
            const float2 x = __ffma2_rn(make_float2(__uint_as_float(v[a & 1][e]), __uint_as_float(v[a & 1][e + 1])), c2, r2), w = make_float2(chunk_ex2(x.x), chunk_ex2(x.y));
            s[(e >> 1) & 1] = __fadd2_rn(s[(e >> 1) & 1], w);
            const __nv_bfloat162 b = __floats2bfloat162_rn(w.x, w.y);
            h[a][e >> 1] = *reinterpret_cast<const uint32_t *>(&b);
        }
    }
    const float2 t = __fadd2_rn(s[0], s[1]);
    return t.x + t.y;
}

// grid: cluster x (row tiles or pairs of them, the longest first) x units.
template <int D, bool kSplit>
__global__ void __launch_bounds__(ChunkTc<D, kSplit>::kThreads, 1)
chunk_tc_kernel(const __grid_constant__ CUtensorMap mapQ, const __grid_constant__ CUtensorMap mapK, const __grid_constant__ CUtensorMap mapV,
                const __grid_constant__ CUtensorMap mapKnew, const __grid_constant__ CUtensorMap mapVnew, const __grid_constant__ ChunkTcParams p)
{
    using L = ChunkTc<D, kSplit>;
    constexpr int S = L::kStreams, KT = L::kKeys;
    extern __shared__ __align__(1024) uint8_t ct_raw[];
    const uint32_t base = smem_u32(ct_raw);
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const uint32_t rank = cluster_rank(), ranks = cluster_size();
    auto bar = [&](int i) { return base + L::kOffBar + 8u * (uint32_t)i; };
    volatile int *flag = reinterpret_cast<volatile int *>(ct_raw + L::kOffFlag);
    uint32_t *tmem_slot = reinterpret_cast<uint32_t *>(ct_raw + L::kOffFlag + 8);
    if (base & 1023u) {   // the swizzled tiles need this alignment
        if (threadIdx.x == 0) set_status(p.c.status, kStatusBounds);
        return;
    }
    // ---- which rows and keys
    const int units = p.c.layers * p.c.streams * p.c.Hkv, item = blockIdx.x / ranks, unit = item % units;
    const int tile0 = (p.items_per_unit - 1 - item / units) * L::kQTiles;   // of kCtRows rows: p.tile_tokens tokens
    const int hkv = unit % p.c.Hkv, b = unit / p.c.Hkv % p.c.streams, l = unit / p.c.Hkv / p.c.streams;
    if (warp == 2 && lane < 5) {   // (the maps are parameters: they can be fetched before anything else is there)
        const CUtensorMap *maps[5] = {&mapQ, &mapK, &mapV, &mapKnew, &mapVnew};
        asm volatile("prefetch.tensormap [%0];" ::"l"(maps[lane]) : "memory");
    }
    if (threadIdx.x == 0) {
        *flag = 0;
        for (int i = 0; i < kCbCount; ++i) mbar_init(bar(i), i >= kCbP && i < kCbO ? 8 : 1);   // (P: a stream's eight warps)
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == 1) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(tmem_slot)), "r"(512u) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = *tmem_slot;
    pdl_wait();
    pdl_release();
    const int n = chunk_tokens(p.c, b), G = p.c.G, t0 = tile0 * p.tile_tokens;
    // tokens of the query tiles, and the key tiles they need: the pot's, then the chunk's up to the last token
    const int tokens[2] = {min(p.tile_tokens, n - t0), kSplit ? 0 : min(p.tile_tokens, n - t0 - p.tile_tokens)};
    const int seen = min(n, t0 + L::kQTiles * p.tile_tokens);   // chunk tokens that some row sees
    const int pot_tiles = (p.c.len + KT - 1) / KT, all_tiles = t0 < n ? pot_tiles + (seen + KT - 1) / KT : 0;
    const int first = (int)((long long)all_tiles * rank / ranks), tiles = (int)((long long)all_tiles * (rank + 1) / ranks) - first;
    const int pot_unit = p.c.unit0 + unit;

    if (warp == 0) {
        // ---------------------------------------------------------------- loads
        if (lane == 0 && tiles > 0) {
            mbar_expect_tx(bar(kCbQ), L::kQTiles * L::kHalves * (uint32_t)(p.tile_tokens * G * 128));
            for (int i = 0; i < L::kQTiles; ++i)
                for (int h = 0; h < L::kHalves; ++h)
                    tma_load_5d(base + L::kOffQ + i * L::kQBytes + h * L::kQBlk, &mapQ, 64 * h, hkv * G, t0 + i * p.tile_tokens, b, l, bar(kCbQ));
            uint32_t k = 0;   // loads so far
            bool ok = true;
            auto load = [&](int t, bool values) {
                const uint32_t slot = k % L::kStages, fill = k / L::kStages, dst = base + L::kOffStage + slot * L::kStageBytes;
                ok = ok && chunk_wait(bar(kCbEmpty + slot), (fill & 1) ^ 1, flag, p);
                if (!ok) return;
                mbar_expect_tx(bar(kCbFull + slot), L::kStageBytes);
                const int tile = first + t;
                if (tile < pot_tiles) {
                    for (int h = 0; h < L::kHalves; ++h) tma_load_3d(dst + h * L::kKeyBlk, values ? &mapV : &mapK, 64 * h, tile * KT, pot_unit, bar(kCbFull + slot));
                } else {
                    for (int h = 0; h < L::kHalves; ++h)
                        tma_load_5d(dst + h * L::kKeyBlk, values ? &mapVnew : &mapKnew, 64 * h, (tile - pot_tiles) * KT, hkv, b, l, bar(kCbFull + slot));
                }
                ++k;
            };
            constexpr int ahead = kSplit ? S : 1;   // tiles whose logits are under way before the first output product
            for (int t = 0; t < min(ahead, tiles); ++t) load(t, false);
            for (int t = 0; t < tiles && ok; ++t) {
                load(t, true);
                if (t + ahead < tiles) load(t + ahead, false);
            }
            // what was issued lands in this block's shared memory: the last load of every slot completes before the block ends
            chunk_wait(bar(kCbQ), 0, flag, p, false);
            for (uint32_t j = k > (uint32_t)L::kStages ? k - L::kStages : 0; j < k; ++j) chunk_wait(bar(kCbFull + j % L::kStages), (j / L::kStages) & 1, flag, p, false);
        }
        __syncwarp();
    } else if (warp == 1) {
        // ---------------------------------------------------------------- products
        const bool leader = elect_one();
        const uint32_t idesc_s = (1u << 4) | (1u << 7) | (1u << 10) | ((uint32_t)(KT >> 3) << 17) | ((128u >> 4) << 24);
        const uint32_t idesc_o = (1u << 4) | (1u << 7) | (1u << 10) | (1u << 16) | ((uint32_t)((p.c.d + 15) / 16 * 2) << 17) | ((128u >> 4) << 24);
        const int ksteps = (p.c.d + 15) / 16;
        bool ok = tiles > 0, any = false;
        auto wait = [&](int which, uint32_t parity) { ok = ok && __all_sync(0xffffffffu, chunk_wait(bar(which), parity, flag, p)); };
        auto wait_stage = [&](uint32_t at) { wait(kCbFull + at % L::kStages, (at / L::kStages) & 1); };
        const uint64_t q_desc = smem_desc_sw128(base + L::kOffQ), k_desc = smem_desc_sw128(base + L::kOffStage), v_desc = smem_desc_sw128_nmajor(base + L::kOffStage, L::kKeyBlk);
        // (the elected lane) S of stream i from stage `at`; O of stream i += P V
        auto logits = [&](int i, uint32_t at) {
            const uint64_t a = q_desc + (kSplit ? 0 : i) * (L::kQBytes >> 4), b = k_desc + at % L::kStages * (L::kStageBytes >> 4);
#pragma unroll
            for (int c = 0; c < D / 16; ++c)
                if (c < ksteps) tc_mma_bf16(tmem + 128 * i, a + (c >> 2) * (L::kQBlk >> 4) + 2 * (c & 3), b + (c >> 2) * (L::kKeyBlk >> 4) + 2 * (c & 3), idesc_s, c > 0);
            tc_commit(bar(kCbS + i));
        };
        auto output = [&](int i, uint32_t at, bool more) {
            const uint64_t b = v_desc + at % L::kStages * (L::kStageBytes >> 4);
#pragma unroll
            for (int c = 0; c < KT / 16; ++c)
                tc_mma_bf16_ts(tmem + L::kOutCol + D * i, tmem + 128 * i + (c >= KT / 32 ? L::kCols - 8 * (KT / 32) : 0) + 8 * c, b + c * (16 * 128 >> 4), idesc_o, more || c > 0);
        };
        auto release = [&](uint32_t at) { tc_commit(bar(kCbEmpty + at % L::kStages)); };
        // Values behind a stream's last token count for nothing but must be finite: 0 times what lies there is not 0 otherwise.
        const int ragged = n < p.c.n && n % KT ? pot_tiles + n / KT - first : -1;   // the tile that has some
        auto clear_padding = [&](uint32_t at) {
            uint8_t *v = ct_raw + L::kOffStage + at % L::kStages * L::kStageBytes;
            for (int h = 0; h < L::kHalves; ++h)
                for (int e = n % KT * 8 + lane; e < KT * 8; e += 32) *reinterpret_cast<uint4 *>(v + h * L::kKeyBlk + e * 16) = make_uint4(0, 0, 0, 0);
            asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
            __syncwarp();
        };
        // keys and values of tile t were the how-manyth load (see there)
        constexpr int ahead = kSplit ? S : 1;
        auto keys_at = [&](int t) { return (uint32_t)(t < ahead ? t : 2 * t - ahead + 1); };
        auto values_at = [&](int t) { return (uint32_t)(min(ahead, tiles) + t + min(t, max(0, tiles - ahead))); };
        const int live = kSplit ? S : tokens[1] > 0 ? 2 : 1;   // streams
        wait(kCbQ, 0);
        for (int t = 0; t < min(ahead, tiles); ++t) {
            wait_stage(keys_at(t));
            if (!ok) break;
            any = true;
            tc_fence_after();
            if (leader) {
                for (int i = kSplit ? t : 0; i < (kSplit ? t + 1 : live); ++i) logits(i, keys_at(t));
                release(keys_at(t));
            }
            __syncwarp();
        }
        for (int t = 0; t < tiles && ok; ++t) {
            const uint32_t at = values_at(t);
            const bool more = t + ahead < tiles;
            wait_stage(at);
            if (more) wait_stage(at + 1);   // the keys loaded next
            if (ok && t == ragged) clear_padding(at);
            for (int i = kSplit ? t % S : 0; i < (kSplit ? t % S + 1 : live); ++i) {
                wait(kCbP + i, (kSplit ? t / S : t) & 1);
                if (!ok) break;
                tc_fence_after();
                if (leader) {
                    output(i, at, t >= ahead);
                    if (more) logits(i, at + 1);
                    else tc_commit(bar(kCbO + i));
                }
                __syncwarp();
            }
            if (leader && ok) {
                release(at);
                if (more) release(at + 1);
            }
            __syncwarp();
        }
        if (any) {   // every product has finished before tensor memory is released
            if (leader) tc_commit(bar(kCbDrain));
            chunk_wait(bar(kCbDrain), 0, flag, p, false);
        }
        __syncwarp();
    } else {
        // ---------------------------------------------------------------- softmax
        const int i = (warp - 2) >> 3, half = ((warp - 2) >> 2) & 1, q = warp & 3, row = q * 32 + lane, pair = 1 + 4 * i + q;   // (a warp may touch the TMEM lanes of its quarter)
        constexpr int W = L::kCols, W2 = D / 2;   // columns of S and O
        const uint32_t lanes = tmem + ((uint32_t)(q * 32) << 16), ts = lanes + 128 * i + W * half, to = lanes + L::kOutCol + D * i + W2 * half;
        const int qt = kSplit ? 0 : i, ti = row / G, t = t0 + qt * p.tile_tokens + ti, g = row - ti * G;
        const bool valid = ti < tokens[qt], works = __any_sync(0xffffffffu, valid);
        const int mine = tiles <= 0 || tokens[qt] <= 0 ? 0 : kSplit ? (tiles - i + S - 1) / S : tiles;
        const float c = p.c.scale_log2e;
        float2 *stat = reinterpret_cast<float2 *>(ct_raw + L::kOffStat) + i * kCtRows + row;   // (what the row's two threads tell each other; at the end its statistics)
        float m = -INFINITY, sum = 0.f;   // the reference + kChunkLift; the sum is this half's
        for (int j = 0; j < mine; ++j) {
            const int tile = first + (kSplit ? j * S + i : j);
            // columns that this row sees
            const int cols = tile < pot_tiles ? min(KT, p.c.len - tile * KT) : min(KT, t + 1 - (tile - pot_tiles) * KT);
            const bool masked = __any_sync(0xffffffffu, valid && cols < KT);
            chunk_wait(bar(kCbS + i), j & 1, flag, p);
            __syncwarp();
            tc_fence_after();
            if (works) {
                bool general = masked;
                if (!general) {
                    uint32_t h[W / 32][16];
                    const float ref = j ? m : kChunkLift, s = chunk_tile<W>(ts, c, ref, h);
                    general = chunk_pair_any(pair, valid && !(s < kChunkMost && (j || s > kChunkLeast)));   // (the logits are still there)
                    if (!general) {
                        m = ref;
                        sum += s;
#pragma unroll
                        for (int a = 0; a < W / 32; ++a) tmem_st16(ts + 16 * a, h[a]);
                    }
                }
                if (general) {
                    const float2 r = chunk_tile_general<W, W2>(ts, to, cols - W * half, c, m, sum, valid, j > 0, stat, half, pair);
                    m = r.x;
                    sum = r.y;
                }
                tmem_wait_st();
            }
            tc_fence_before();
            __syncwarp();
            if (lane == 0 && p.withhold != i) mbar_arrive(bar(kCbP + i));
        }
        if (mine > 0) {
            chunk_wait(bar(kCbO + i), 0, flag, p);
            __syncwarp();
            tc_fence_after();
        }
        if (works) {   // the two halves' sums
            m = isnan(m) ? (half ? stat->y : stat->x) : m - kChunkLift;   // (NaN: a far reference)
            (half ? stat->y : stat->x) = sum;
            chunk_pair_sync(pair);
            sum = stat->x + stat->y;
            chunk_pair_sync(pair);
            if (kSplit && !half) *stat = make_float2(m, sum);   // (-inf, 0 where no key has been seen)
        }
        if (!kSplit && works && mine > 0) {   // (mine > 0 is uniform over the stream)
            const float inv = 1.f / sum;
            __nv_bfloat16 *o = (__nv_bfloat16 *)p.c.out + l * p.c.os.layer + b * p.c.os.stream + (long long)(hkv * G + g) * p.c.os.head + (long long)t * p.c.os.token + W2 * half;
#pragma unroll 1
            for (int a = 0; a < W2; a += 32) {
                uint32_t x[32];
                tmem_ld32(to + a, x);
                tmem_wait_ld(x);
#pragma unroll
                for (int e = 0; e < 32; e += 8) {
                    uint32_t w[4];
#pragma unroll
                    for (int f = 0; f < 4; ++f) {
                        const __nv_bfloat162 h = __floats2bfloat162_rn(__uint_as_float(x[e + 2 * f]) * inv, __uint_as_float(x[e + 2 * f + 1]) * inv);
                        w[f] = *reinterpret_cast<const uint32_t *>(&h);
                    }
                    if (valid && W2 * half + a + e < p.c.d) *reinterpret_cast<uint4 *>(o + a + e) = make_uint4(w[0], w[1], w[2], w[3]);
                }
            }
            if (valid && !half && p.c.lse) p.c.lse[(((size_t)l * p.c.streams + b) * p.c.Hkv * G + hkv * G + g) * p.c.n + t] = 0.6931471805599453f * (m + log2f(sum * kChunkLifted));
        }
    }
    if (kSplit) {
        // ---- the streams' results become one, and the cluster's blocks'
        tc_fence_before();
        __syncthreads();   // all products are done: the stages' memory is free
        tc_fence_after();
        float *part = reinterpret_cast<float *>(ct_raw + L::kOffStage);   // [128][pitch]
        float2 *stat = reinterpret_cast<float2 *>(ct_raw + L::kOffStat);
        const int i = warp < 2 ? -1 : (warp - 2) >> 3, half = ((warp - 2) >> 2) & 1, q = warp & 3, row = q * 32 + lane;
        const int ti = row / G, t = t0 + ti, g = row - ti * G;
        const bool valid = ti < tokens[0], works = __any_sync(0xffffffffu, valid), mine0 = tiles > 0, mine1 = S == 2 && tiles > 1;   // (which streams have had keys)
        const float2 s0 = stat[row], s1 = S == 2 ? stat[(S - 1) * kCtRows + row] : make_float2(-INFINITY, 0.f);
        const float ref = fmaxf(s0.x, s1.x), f0 = s0.x == -INFINITY ? 0.f : chunk_ex2(s0.x - ref), f1 = s1.x == -INFINITY ? 0.f : chunk_ex2(s1.x - ref), den = s0.y * f0 + s1.y * f1;
        float4 *at = reinterpret_cast<float4 *>(part + (size_t)row * L::kPitch + D / 2 * half);
        const uint32_t to = tmem + ((uint32_t)(q * 32) << 16) + L::kOutCol + D / 2 * half;
        if (i == 1 && works && mine1) {
#pragma unroll 1
            for (int a = 0; a < D / 64; ++a) {
                uint32_t x[32];
                tmem_ld32(to + D + 32 * a, x);
                tmem_wait_ld(x);
#pragma unroll
                for (int e = 0; e < 8; ++e)
                    at[a * 8 + e] = make_float4(__uint_as_float(x[4 * e]) * f1, __uint_as_float(x[4 * e + 1]) * f1, __uint_as_float(x[4 * e + 2]) * f1, __uint_as_float(x[4 * e + 3]) * f1);
            }
        }
        __syncthreads();
        if (i == 0 && works) {
            const float inv = 1.f / den;
            __nv_bfloat16 *o = (__nv_bfloat16 *)p.c.out + l * p.c.os.layer + b * p.c.os.stream + (long long)(hkv * G + g) * p.c.os.head + (long long)t * p.c.os.token + D / 2 * half;
#pragma unroll 1
            for (int a = 0; a < D / 64; ++a) {
                uint32_t x[32];
                if (mine0) {
                    tmem_ld32(to + 32 * a, x);
                    tmem_wait_ld(x);
                }
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const float4 y = mine1 ? at[a * 8 + e] : make_float4(0.f, 0.f, 0.f, 0.f);
                    const float z[4] = {y.x, y.y, y.z, y.w};
#pragma unroll
                    for (int k = 0; k < 4; ++k) x[4 * e + k] = __float_as_uint(mine0 ? fmaf(__uint_as_float(x[4 * e + k]), f0, z[k]) : 0.f);
                    if (ranks > 1) at[a * 8 + e] = make_float4(__uint_as_float(x[4 * e]), __uint_as_float(x[4 * e + 1]), __uint_as_float(x[4 * e + 2]), __uint_as_float(x[4 * e + 3]));
                }
                if (ranks == 1) {
#pragma unroll
                    for (int e = 0; e < 32; e += 8) {
                        uint32_t w[4];
#pragma unroll
                        for (int k = 0; k < 4; ++k) {
                            const __nv_bfloat162 h = __floats2bfloat162_rn(__uint_as_float(x[e + 2 * k]) * inv, __uint_as_float(x[e + 2 * k + 1]) * inv);
                            w[k] = *reinterpret_cast<const uint32_t *>(&h);
                        }
                        if (valid && D / 2 * half + 32 * a + e < p.c.d) *reinterpret_cast<uint4 *>(o + 32 * a + e) = make_uint4(w[0], w[1], w[2], w[3]);
                    }
                }
            }
            if (ranks > 1) {
                if (!half) stat[row] = make_float2(ref, den);   // (everyone has read what was there)
            } else if (valid && !half && p.c.lse) {
                p.c.lse[(((size_t)l * p.c.streams + b) * p.c.Hkv * G + hkv * G + g) * p.c.n + t] = 0.6931471805599453f * (ref + log2f(den * kChunkLifted));
            }
        }
        if (ranks > 1) {
            // Every block of the cluster owns some rows.  Their results come to it as one copy of shared memory from each of the others (L::kPush), or, where there is no room for
            // that, it reads them there (64 tokens over 8000 rows, clusters of 7: reading everything, statistics per vector, 33.6 us, now 26.7).
            const int vecs = p.c.d / 8, rows = max(tokens[0], 0) * G, per = (rows + (int)ranks - 1) / (int)ranks, mine_from = min(rows, (int)rank * per), mine_rows = min(rows, mine_from + per) - mine_from;
            float *got = part + L::kPartBytes / 4;
            float2 *stats = reinterpret_cast<float2 *>(ct_raw + L::kOffQ);   // [blocks][own rows]
            asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
            cluster_sync();   // all results are there, and nobody's stages are in use any more
            if (L::kPush && threadIdx.x == 0 && tiles > 0) {
                for (uint32_t o = 0; o < ranks; ++o) {
                    const int from = min(rows, (int)o * per), n_rows = min(rows, from + per) - from;
                    if (n_rows <= 0) continue;
                    asm volatile("cp.async.bulk.shared::cluster.shared::cta.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(cluster_addr(got + (size_t)rank * per * L::kPitch, o)),
                                 "r"(smem_u32(part + (size_t)from * L::kPitch)), "r"((uint32_t)n_rows * L::kPitch * 4u), "r"(cluster_addr(ct_raw + L::kOffBar + 8 * kCbMerge, o)) : "memory");
                }
            }
            for (int e = threadIdx.x; e < mine_rows * (int)ranks; e += L::kThreads) {
                const int k = e / mine_rows;
                stats[e] = cluster_ld2(cluster_addr(&stat[mine_from + e - k * mine_rows], k));
            }
            if (L::kPush && mine_rows > 0) {
                // (blocks that have had no key tile send nothing)
                if (threadIdx.x == 0) mbar_expect_tx(bar(kCbMerge), (uint32_t)min((int)ranks, all_tiles) * (uint32_t)mine_rows * L::kPitch * 4u);
                chunk_wait(bar(kCbMerge), 0, flag, p, false);
            }
            __syncthreads();
            // a thread has 8 channels of a row
            for (int e = threadIdx.x; e < mine_rows * vecs; e += L::kThreads) {
                const int r = e / vecs, v = e - r * vecs, row = mine_from + r;
                float ref = -INFINITY, den = 0.f, o[8];
#pragma unroll
                for (int k = 0; k < 8; ++k) o[k] = 0.f;
                for (uint32_t k = 0; k < ranks; ++k) ref = fmaxf(ref, stats[k * mine_rows + r].x);
                for (uint32_t k = 0; k < ranks; ++k) {
                    const float2 st = stats[k * mine_rows + r];
                    if (st.x == -INFINITY) continue;   // it has seen no key of this row: what it holds is not a number
                    float4 x, y;
                    if (L::kPush) {
                        const float4 *src = reinterpret_cast<const float4 *>(got + (size_t)(k * per + r) * L::kPitch + 8 * v);
                        x = src[0];
                        y = src[1];
                    } else {
                        const uint32_t src = cluster_addr(part + (size_t)row * L::kPitch + 8 * v, k);
                        x = cluster_ld4(src);
                        y = cluster_ld4(src + 16);
                    }
                    const float f = chunk_ex2(st.x - ref), z[8] = {x.x, x.y, x.z, x.w, y.x, y.y, y.z, y.w};
                    den = fmaf(st.y, f, den);
#pragma unroll
                    for (int c = 0; c < 8; ++c) o[c] = fmaf(z[c], f, o[c]);
                }
                const float inv = 1.f / den;
                uint32_t w[4];
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    const __nv_bfloat162 h = __floats2bfloat162_rn(o[2 * k] * inv, o[2 * k + 1] * inv);
                    w[k] = *reinterpret_cast<const uint32_t *>(&h);
                }
                const int ti = row / G, g = row - ti * G, t = t0 + ti;
                __nv_bfloat16 *out = (__nv_bfloat16 *)p.c.out + l * p.c.os.layer + b * p.c.os.stream + (long long)(hkv * G + g) * p.c.os.head + (long long)t * p.c.os.token;
                *reinterpret_cast<uint4 *>(out + 8 * v) = make_uint4(w[0], w[1], w[2], w[3]);
                if (v == 0 && p.c.lse) p.c.lse[(((size_t)l * p.c.streams + b) * p.c.Hkv * G + hkv * G + g) * p.c.n + t] = 0.6931471805599453f * (ref + log2f(den * kChunkLifted));
            }
            cluster_sync();   // no block ends while others read or send
        }
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    if (warp == 1) asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(512u) : "memory");
}

// ------------------------------------------------------------------ host side
// [layer][stream][head][token][d] bf16 as a map of five dimensions, whatever the strides; a box is 64 channels of `heads` heads x `tokens` tokens (heads inside)
// or, keys, of `tokens` tokens of one head.
inline bool chunk_map(TcEncodeFn encode, CUtensorMap *map, const void *ptr, const ChunkParams &p, const Strides &s, int heads_all, bool queries, int heads, int tokens)
{
    // a stride that no second element ever uses may be anything: one that is always allowed stands in
    auto bytes = [](long long stride, int extent, long long other) { return (cuuint64_t)(2 * (extent > 1 ? stride : other)); };
    const cuuint64_t st_h = bytes(s.head, heads_all, p.d), st_t = bytes(s.token, p.n, p.d), st_b = bytes(s.stream, p.streams, p.d), st_l = bytes(s.layer, p.layers, p.d);
    const cuuint64_t dims[5] = {(cuuint64_t)p.d, (cuuint64_t)(queries ? heads_all : p.n), (cuuint64_t)(queries ? p.n : heads_all), (cuuint64_t)p.streams, (cuuint64_t)p.layers};
    const cuuint64_t strides[4] = {queries ? st_h : st_t, queries ? st_t : st_h, st_b, st_l};
    const cuuint32_t box[5] = {64, (cuuint32_t)(queries ? heads : tokens), (cuuint32_t)(queries ? tokens : 1), 1, 1}, each[5] = {1, 1, 1, 1, 1};
    return encode(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 5, const_cast<void *>(ptr), dims, strides, box, each, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
                  CU_TENSOR_MAP_L2_PROMOTION_L2_128B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}
inline bool chunk_pot_map(TcEncodeFn encode, CUtensorMap *map, const void *ptr, const ChunkParams &p, int pot_units, int keys)
{
    const cuuint64_t dims[3] = {(cuuint64_t)p.d, (cuuint64_t)(p.len > 0 ? p.len : 1), (cuuint64_t)pot_units};
    const cuuint64_t strides[2] = {(cuuint64_t)p.d * 2, (cuuint64_t)p.unit_rows * p.d * 2};
    const cuuint32_t box[3] = {64, (cuuint32_t)keys, 1}, each[3] = {1, 1, 1};
    return encode(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 3, const_cast<void *>(ptr), dims, strides, box, each, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
                  CU_TENSOR_MAP_L2_PROMOTION_L2_128B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// *done: the call has been launched (or failed to be); false: its strides are none that a tensor map takes.
template <int D, bool kSplit>
inline cudaError_t launch_chunk_tc_t(const ChunkParams &c, const ChunkTcHost &host, int tile_tokens, int tiles, cudaStream_t stream, bool *done)
{
    using L = ChunkTc<D, kSplit>;
    *done = false;
    TcEncodeFn encode = (TcEncodeFn)host.encode;
    CUtensorMap q, K, V, k, v;
    if (!chunk_map(encode, &q, c.q, c, c.qs, c.Hkv * c.G, true, c.G, tile_tokens) || !chunk_map(encode, &k, c.k, c, c.ks, c.Hkv, false, 1, L::kKeys) ||
        !chunk_map(encode, &v, c.v, c, c.vs, c.Hkv, false, 1, L::kKeys) || !chunk_pot_map(encode, &K, c.potK, c, host.pot_units, L::kKeys) ||
        !chunk_pot_map(encode, &V, c.potV, c, host.pot_units, L::kKeys))
        return cudaSuccess;
    *done = true;
    auto kern = chunk_tc_kernel<D, kSplit>;
    const cudaError_t e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)L::kSmemBytes);
    if (e != cudaSuccess) return e;
    ChunkTcParams p;
    const long long items = (long long)c.layers * c.streams * c.Hkv * ((tiles + L::kQTiles - 1) / L::kQTiles);
    const int key_tiles = (c.len + L::kKeys - 1) / L::kKeys + (c.n + L::kKeys - 1) / L::kKeys;
    static ClusterFit fit;
    // few query tiles: a tile's keys over a cluster, two key tiles a block
    const int cluster = kSplit ? choose_cluster(fit, kern, dim3(L::kThreads), L::kSmemBytes, items, std::min(8, (key_tiles + 1) / 2)) : 1;
    if (items * cluster > 0x7fffffff) return cudaErrorInvalidValue;
    p.c = c;
    p.tile_tokens = tile_tokens;
    p.items_per_unit = (tiles + L::kQTiles - 1) / L::kQTiles;
    p.withhold = host.withhold;
    p.wait_ns = host.wait_ns;
    p.status = c.status;
    return launch_cluster(kern, dim3((unsigned)(cluster * items)), dim3(L::kThreads), L::kSmemBytes, cluster, stream, q, K, V, k, v, p);
}

inline cudaError_t launch_chunk_tc(const ChunkParams &c, const ChunkTcHost &host, cudaStream_t stream, bool *done)
{
    const int tile_tokens = kCtRows / c.G, tiles = (c.n + tile_tokens - 1) / tile_tokens;
    const long long units = (long long)c.layers * c.streams * c.Hkv;
    // Two query tiles a block share its key tiles, in half as many blocks that each take 1.45 times as long (two streams per key tile are then both busy); one goes faster where that saves no
    // round of blocks.  us, two / one: 12 units of 12 tiles over 2000 rows 43 / 30, 13 tiles 44 / 51, 22 tiles 49 / 58, 25 tiles 80 / 83; 32 units of 9 tiles 77 / 56, 10 tiles 80 / 83.
    // Streams of different lengths: how long the host does not know; a quarter of the tiles is taken to be padding.  3 streams of 180 tiles, with no padding, 15, 25 and 50 % of it: 46 / 54,
    // 45 / 52, 45 / 31, 44 / 30.  (Full streams lose a sixth by it between 149 and 197 tiles, padded ones gain a third; over 90 calls of 2 to 8 streams with 0 to 50 % padding and 150 to 350
    // tiles the choice costs 5 % on average, and without the quarter 12 %.)
    auto rounds = [&](long long blocks) { return ((c.tokens ? blocks - blocks / 4 : blocks) + host.sm_count - 1) / host.sm_count; };
    const bool pairs = c.d <= 128 && 4 * rounds(units * ((tiles + 1) / 2)) < 3 * rounds(units * tiles);
    if (c.d > 128) return launch_chunk_tc_t<256, true>(c, host, tile_tokens, tiles, stream, done);
    if (c.d > 64) return pairs ? launch_chunk_tc_t<128, false>(c, host, tile_tokens, tiles, stream, done)
                               : launch_chunk_tc_t<128, true>(c, host, tile_tokens, tiles, stream, done);
    return pairs ? launch_chunk_tc_t<64, false>(c, host, tile_tokens, tiles, stream, done)
                 : launch_chunk_tc_t<64, true>(c, host, tile_tokens, tiles, stream, done);
}

}  // namespace ipotk
