// Attention of at most 8 query rows of a KV head (or twice as many, in two groups) over many keys: generation.  Two calls come here:
//   a chunk of few tokens (kSparse = false): rows t * G + g over the pot's rows and the chunk's rows 0 .. t;
//   one token over selected blocks of the pot (kSparse = true; the query heads of a KV head in groups of 8).
// Either is a stream of keys and values through few rows, split over a thread-block cluster per unit: bound by HBM, or where there
// are few units by the latency of one chain - launch, (scores, selection,) first loads, merge.
//
// Selection (kSparse).  s_b = sum_h sum_c max(q_hc lo_bc, q_hc hi_bc) over the unit's query heads.  A channel takes hi where q is positive
//   and lo where it is negative, so the heads' positive and negative parts are added first: s_b = sum_c (q+_c hi_bc + q-_c lo_bc), two
//   products per channel whatever the number of heads.  In 64 bits: which block is in must not depend on the order of a sum.  The
//   cluster's blocks share the scoring and put every score into each other's shared memory; then each finds, for itself, the
//   (n - 1)-th largest of the order-preserving 64-bit keys by a search over its bits, and lists the chosen blocks in ascending order.
// few_mma_kernel (bf16): a warp owns tiles of 16 keys and a ring of cp.async stages of its own, rows XOR-swizzled for ldmatrix;
//   S^T = q K^T and O += P V are m16n8k16 tiles with fp32 accumulation.  Of the 16 rows 8 are queries: the other 8 of the output product hold the
//   second of three bf16 terms of the weights where the result is fp32 (kSparse: 24 bits, nothing is rounded to bf16); a
//   bf16 result takes the weights' first term.  tcgen05 does not fit: its smallest tile has 64 rows.
// few_fma_kernel (f32): a group of lanes owns a key (a 16-byte vector of the row or two per lane), four keys at a time.
// Merge: the block's warps in shared memory; then every block of the cluster owns a share of the result and is sent what the others have of it
// (stores into its shared memory: they are done by the time of the one barrier, which loads after it would not be).  No scratch, no atomics.
#pragma once
#include "common.cuh"
#include "cluster.cuh"
#include "ops.h"
#include "k_rotary.cuh"   // RowVec, to_float, from_float

namespace ipotk {

__device__ __forceinline__ float few_ex2(float x)
{
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
// 2^(m - ref), 0 where nothing has been seen (m = -inf) whatever ref is
__device__ __forceinline__ float few_scale(float m, float ref) { return m == -INFINITY ? 0.f : few_ex2(m - ref); }

// Weights enter the product with the values times this: at most 2^15 slots and 16 tokens of weights up to 1 then sum up to at most 1, and no sum on the way is larger than the largest value.
// (A power of two: nothing is rounded by it, down to values of 2^-80.)
constexpr float kFewShare = 1.f / 65536.f;

constexpr int kFewThreads = 128, kFewWarps = kFewThreads / 32, kFewMaxRanks = kMostRanks;
constexpr int kFewRows = 8;       // query rows of a block
constexpr int kFewBlocks = 2048;  // blocks of a unit: 32768 slots, 16 rows
constexpr int kScoreBytes = kFewBlocks * (int)sizeof(double);
constexpr int kFewFmaRoom = 64 * 1024;   // for bounds (few_fma_kernel; the others have their ring)

__device__ __forceinline__ void few_cp_async16(void *dst, const void *src, bool there)
{
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"((uint32_t)__cvta_generic_to_shared(dst)), "l"(src), "r"(there ? 16 : 0) : "memory");
}

// What a block works on, and what its threads know of it.
struct FewUnit {
    int l, b, hkv, unit;      // of the call, and of the pot
    int n;                    // tokens of the stream (kSparse: 1)
    int row0, rows;           // query rows of this block: row0 .. (kSparse: heads), folded t * G + g
    uint32_t rank, ranks;
    __device__ __forceinline__ FewUnit(const FewParams &p)
    {
        const int u = blockIdx.y;
        hkv = u % p.Hkv;
        b = u / p.Hkv % p.streams;
        l = u / p.Hkv / p.streams;
        unit = p.unit0 + u;
        n = p.tokens ? min(max(__ldg(p.tokens + b), 0), p.n) : p.n;
        row0 = blockIdx.z * kFewRows;
        rows = min(kFewRows, p.G * n - row0);
        rank = cluster_rank();
        ranks = cluster_size();
    }
    __device__ __forceinline__ long long q_at(const FewParams &p, int row) const
    {
        const int t = (row0 + row) / p.G, g = row0 + row - t * p.G;
        return l * p.qs.layer + b * p.qs.stream + (long long)(hkv * p.G + g) * p.qs.head + (long long)t * p.qs.token;
    }
};

// Shared memory besides the keys' ring.
struct FewShared {
    uint16_t list[kFewBlocks];                     // the chosen blocks
    uint2 reach[kFewWarps];
    unsigned long long count[2][kFewWarps];
    float2 warp_stat[kFewWarps][kFewRows];      // (reference in binary orders, sum) of the warps,
    float weight[kFewWarps][kFewRows];          // what their results are multiplied by,
    float2 stat[kFewMaxRanks][kFewRows];           // and of the cluster's blocks
};

// ------------------------------------------------------------------ scores and selection
// Monotone map double -> uint64; no finite number becomes 0.
__device__ __forceinline__ unsigned long long order_key64(double s)
{
    const unsigned long long b = (unsigned long long)__double_as_longlong(s + 0.0);   // (-0 counts as 0)
    return b ^ ((unsigned long long)((long long)b >> 63) | 0x8000000000000000ull);
}

// The ascending list of the `need` largest of `others` keys (ties: the lower block); a thread has up to KPT neighbouring blocks.  The keys are taken apart at
// the highest bit in which they differ: 32 bits from there decide nearly always, those below them where that leaves a tie.  Two bits a step: three counts
// in one sum over the warp, one barrier a step, and the search ends as soon as a count is right.  (One warp with 8 keys a lane and no barrier: 600 cycles
// a step, this 300.)
template <int KPT>
__device__ __forceinline__ void select_in_block(FewShared &sh, const double *score, int others, int need)
{
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, per = (others + kFewThreads - 1) / kFewThreads, first = threadIdx.x * per, here = max(0, min(per, others - first));
    uint32_t hi[KPT], lo[KPT];   // 0 where there is no block
    {
        unsigned long long key[KPT];
        uint32_t top = 0, low = 0xffffffffu;
#pragma unroll
        for (int i = 0; i < KPT; ++i) {
            key[i] = 0;
            if (i < here) {
                key[i] = order_key64(score[first + i]);
                top = max(top, (uint32_t)(key[i] >> 32));
                low = min(low, (uint32_t)(key[i] >> 32));
            }
        }
        top = __reduce_max_sync(0xffffffffu, top);
        low = __reduce_min_sync(0xffffffffu, low);
        if (lane == 0) sh.reach[warp] = make_uint2(top, low);
        __syncthreads();
#pragma unroll
        for (int v = 0; v < kFewWarps; ++v) {
            top = max(top, sh.reach[v].x);
            low = min(low, sh.reach[v].y);
        }
        // (where the upper halves agree the whole lower ones are compared)
        const int shift = top != low ? 32 - __clz(top ^ low) : 0;   // bits below the 32 that are looked at first
#pragma unroll
        for (int i = 0; i < KPT; ++i) {
            hi[i] = (uint32_t)(key[i] >> shift);
            lo[i] = shift ? (uint32_t)(key[i] << (32 - shift)) : 0u;
        }
    }
    int parity = 0;
    // the block's sum of three counts, 21 bits each
    auto block_sum = [&](uint32_t c) {   // (ten bits each: at most 512 in a warp)
        c = __reduce_add_sync(0xffffffffu, c);
        if (lane == 0) sh.count[parity][warp] = (c & 1023) | (unsigned long long)(c >> 10 & 1023) << 21 | (unsigned long long)(c >> 20) << 42;
        __syncthreads();
        unsigned long long all = 0;
#pragma unroll
        for (int v = 0; v < kFewWarps; ++v) all += sh.count[parity][v];
        parity ^= 1;
        return all;
    };
    uint32_t in = 0, group = here > 0 ? 0xffffffffu >> (32 - here) : 0u;   // bit i: block first + i is in; may still be
    int left = need;
#pragma unroll 1
    for (int level = 0; level < 2 && left > 0; ++level) {
        uint32_t k[KPT], at = 0;
#pragma unroll
        for (int i = 0; i < KPT; ++i) k[i] = group >> i & 1 ? (level ? lo[i] : hi[i]) : 0u;   // (`at` with a bit set is never 0)
        bool exact = false;
#pragma unroll 1
        for (int bit = 30; bit >= 0 && !exact; bit -= 2) {
            uint32_t c1 = 0, c2 = 0, c3 = 0;
#pragma unroll
            for (int i = 0; i < KPT; ++i) {
                c1 += k[i] >= (at | 1u << bit);
                c2 += k[i] >= (at | 2u << bit);
                c3 += k[i] >= (at | 3u << bit);
            }
            const unsigned long long all = block_sum(c1 | c2 << 10 | c3 << 20);
            const int n1 = (int)(all & 0x1fffff), n2 = (int)(all >> 21 & 0x1fffff), n3 = (int)(all >> 42);
            at |= (n3 >= left ? 3u : n2 >= left ? 2u : n1 >= left ? 1u : 0u) << bit;
            exact = n1 == left || n2 == left || n3 == left;
        }
        uint32_t above = 0, equal = 0;
#pragma unroll
        for (int i = 0; i < KPT; ++i)
            if (group >> i & 1) {
                above |= (uint32_t)(k[i] > at || (exact && k[i] == at)) << i;
                equal |= (uint32_t)(!exact && k[i] == at) << i;
            }
        in |= above;
        group = equal;
        left = exact ? 0 : left - (int)(block_sum(__popc(above)) & 0x1fffff);
    }
    // `left` of those that agree in all bits, the lower blocks, are in too.  Places by an exclusive sum over the threads, both counts in one number
    const int both = __popc(in) | __popc(group) << 16;
    int incl = both;
#pragma unroll
    for (int off = 1; off < 32; off <<= 1) {
        const int v = __shfl_up_sync(0xffffffffu, incl, off);
        if (lane >= off) incl += v;
    }
    if (lane == 31) sh.count[parity][warp] = (unsigned)incl;
    __syncthreads();
    int before = incl - both;
#pragma unroll
    for (int v = 0; v < kFewWarps; ++v)
        if (v < warp) before += (int)sh.count[parity][v];
    int equal_before = before >> 16, place = (before & 0xffff) + min(equal_before, left);
#pragma unroll
    for (int i = 0; i < KPT; ++i) {
        bool is = in >> i & 1;
        if (group >> i & 1) is = equal_before++ < left;
        if (is) sh.list[place++] = (uint16_t)(first + i);
    }
}

// All blocks of the cluster: sh.list becomes the ascending list of the chosen blocks, its length is returned.  free_bytes: shared memory that is free
// meanwhile, room_bytes behind kFewBlocks scores, at the same place in every block.  The cluster has arrived at its first barrier.
template <typename T>
__device__ __forceinline__ int select_blocks(FewShared &sh, uint8_t *free_bytes, int room_bytes, const FewParams &p, const FewUnit &u)
{
    double *score = reinterpret_cast<double *>(free_bytes);
    RowVec<T> *bounds = reinterpret_cast<RowVec<T> *>(score + kFewBlocks);
    constexpr int VE = RowVec<T>::kElems, NV = sizeof(T) == 2 ? 2 : 4, BF = 4;   // 256 channels: 64 vectors of bf16 bounds, 128 of f32
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, vecs = p.d / VE, pieces = 2 * vecs;
    const int total = (p.len + p.block_rows - 1) / p.block_rows, want = min(p.blocks, total), others = total - 1, need = want - 1;
    if (want == total || need == 0) {
        for (int b = threadIdx.x; b < want; b += kFewThreads) sh.list[b] = (uint16_t)(need == 0 ? others : b);
        __syncthreads();
        cluster_wait();
        return want;
    }
    // this block's share of the others: their bounds come into shared memory, as many at once as find room.  (Straight into registers, four blocks a warp and four more on their
    // way, the loads were a chain of latencies: 256 units x 127 blocks x 128 channels 41.0 us for the call, 38.4 so.)
    const T *lo = (const T *)p.lo + (size_t)u.unit * p.unit_blocks * p.d, *hi = (const T *)p.hi + (size_t)u.unit * p.unit_blocks * p.d;
    const int mine0 = (int)((long long)others * u.rank / u.ranks), mine = (int)((long long)others * (u.rank + 1) / u.ranks) - mine0, room = room_bytes / (2 * p.d * (int)sizeof(T));
    auto fetch = [&](int from) {
        const int n = min(room, mine - from) * vecs;
        const RowVec<T> *l = reinterpret_cast<const RowVec<T> *>(lo + (size_t)(mine0 + from) * p.d), *h = reinterpret_cast<const RowVec<T> *>(hi + (size_t)(mine0 + from) * p.d);
        for (int e = threadIdx.x; e < n; e += kFewThreads) {
            few_cp_async16(bounds + e, l + e, true);
            few_cp_async16(bounds + room * vecs + e, h + e, true);
        }
        asm volatile("cp.async.commit_group;" ::: "memory");
    };
    fetch(0);
    // what the heads' queries sum up to in those channels, above and below zero
    double w[NV * VE];
    const T *q = (const T *)p.q + u.l * p.qs.layer + u.b * p.qs.stream + (long long)u.hkv * p.G * p.qs.head;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        const int piece = lane + 32 * i;
#pragma unroll
        for (int e = 0; e < VE; ++e) w[i * VE + e] = 0.0;
        if (piece >= pieces) continue;
        const bool upper = piece >= vecs;
        constexpr int HB = 8;   // heads on their way at once
#pragma unroll 1
        for (int h0 = 0; h0 < p.G; h0 += HB) {
            RowVec<T> y[HB];
#pragma unroll
            for (int h = 0; h < HB; ++h) y[h] = *reinterpret_cast<const RowVec<T> *>(q + min(h0 + h, p.G - 1) * p.qs.head + (piece - (upper ? vecs : 0)) * VE);
#pragma unroll
            for (int h = 0; h < HB; ++h)
#pragma unroll
                for (int e = 0; e < VE; ++e) {
                    const float f = to_float(y[h].e[e]);
                    w[i * VE + e] += (double)(h0 + h < p.G ? (upper ? fmaxf(f, 0.f) : fminf(f, 0.f)) : 0.f);
                }
        }
    }
    cluster_wait();   // all of the cluster has started: its shared memory may be written
    for (int from = 0; from < mine; from += room) {
        if (from) {
            __syncthreads();
            fetch(from);
        }
        asm volatile("cp.async.wait_all;" ::: "memory");
        __syncthreads();
        const int n = min(room, mine - from);
        for (int i0 = warp; i0 < n; i0 += BF * kFewWarps) {
            double sum[BF];   // of four blocks side by side: the chains of 64-bit sums are long
#pragma unroll
            for (int f = 0; f < BF; ++f) sum[f] = 0.0;
#pragma unroll
            for (int i = 0; i < NV; ++i)
                if (lane + 32 * i < pieces) {
                    const int piece = lane + 32 * i;
                    const RowVec<T> *at = bounds + (piece >= vecs ? room * vecs + piece - vecs : piece);
                    RowVec<T> x[BF];
#pragma unroll
                    for (int f = 0; f < BF; ++f) x[f] = at[min(i0 + f * kFewWarps, n - 1) * vecs];
#pragma unroll
                    for (int e = 0; e < VE; ++e)
#pragma unroll
                        for (int f = 0; f < BF; ++f) sum[f] = fma(w[i * VE + e], (double)to_float(x[f].e[e]), sum[f]);
                }
            // sums over the lanes: a lane keeps half of what it has and sends the other half, so that lanes 8 f .. 8 f + 7 end with block f's
            static_assert(BF == 4, "two halvings");
            {
                const bool up = lane & 16;
                const double s0 = __shfl_xor_sync(0xffffffffu, up ? sum[0] : sum[2], 16), s1 = __shfl_xor_sync(0xffffffffu, up ? sum[1] : sum[3], 16);
                sum[0] = (up ? sum[2] : sum[0]) + s0;
                sum[1] = (up ? sum[3] : sum[1]) + s1;
            }
            {
                const bool up = lane & 8;
                const double s0 = __shfl_xor_sync(0xffffffffu, up ? sum[0] : sum[1], 8);
                sum[0] = (up ? sum[1] : sum[0]) + s0;
            }
#pragma unroll
            for (int off = 4; off >= 1; off >>= 1) sum[0] += __shfl_xor_sync(0xffffffffu, sum[0], off);
            const int i = i0 + (lane >> 3) * kFewWarps;
            if (i < n)
                for (uint32_t r = lane & 7; r < u.ranks; r += 8) cluster_st(cluster_addr(score + mine0 + from + i, r), sum[0]);
        }
    }
    cluster_sync();
    if (others <= 2 * kFewThreads) select_in_block<2>(sh, score, others, need);
    else select_in_block<kFewBlocks / kFewThreads>(sh, score, others, need);
    if (threadIdx.x == 0) sh.list[need] = (uint16_t)others;
    __syncthreads();
    return want;
}

// ------------------------------------------------------------------ the end of a block's work
// part: [warps][rows][d + 4] outputs against the references in sh.warp_stat, times kFewShare; got: room for the blocks' shares of the result.
// kAlone: with a way of its own for a block that is its own cluster, which has much for few threads (selected blocks of 256 units 38.4 -> 36.6 us).  Its code costs launches of few
// units, which never come there, 0.6 of 7.3 us: a single token's few microseconds are worth more than 2 of the 80 that many units take.
template <typename O, bool kAlone>
__device__ __forceinline__ void few_finish(float *part, float *got, FewShared &sh, const FewParams &p, const FewUnit &u)
{
    const int ds = p.d + 4, all = u.rows * p.d, share = ((all + (int)u.ranks - 1) / (int)u.ranks + 3) & ~3;
    __syncthreads();
    for (int e = threadIdx.x; e < u.rows * (int)u.ranks; e += kFewThreads) {   // a row's statistics to one block of the cluster
        const int r = e / u.rows, h = e - r * u.rows;
        float ref = -INFINITY, sum = 0.f;
#pragma unroll
        for (int w = 0; w < kFewWarps; ++w) ref = fmaxf(ref, sh.warp_stat[w][h].x);
#pragma unroll
        for (int w = 0; w < kFewWarps; ++w) {
            const float f = few_scale(sh.warp_stat[w][h].x, ref);
            sum = fmaf(sh.warp_stat[w][h].y, f, sum);
            if (r == 0) sh.weight[w][h] = f;
        }
        cluster_st(cluster_addr(&sh.stat[u.rank][h], r), make_float2(ref, sum));
    }
    __syncthreads();
    for (int e = threadIdx.x * 4; e < all; e += kFewThreads * 4) {
        const int h = e / p.d, c = e - h * p.d, owner = e / share;
        float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
        for (int w = 0; w < kFewWarps; ++w) {
            const float4 x = *reinterpret_cast<const float4 *>(part + (w * u.rows + h) * ds + c);
            const float f = sh.weight[w][h];
            v = make_float4(fmaf(x.x, f, v.x), fmaf(x.y, f, v.y), fmaf(x.z, f, v.z), fmaf(x.w, f, v.w));
        }
        cluster_st(cluster_addr(got + u.rank * share + e - owner * share, owner), v);
    }
    cluster_sync();   // from here on a block touches its own memory alone
    if (kAlone && u.ranks == 1) {
        for (int e = threadIdx.x * 4; e < all; e += kFewThreads * 4) {
            const int h = e / p.d, c = e - h * p.d, t = (u.row0 + h) / p.G, g = u.hkv * p.G + u.row0 + h - t * p.G;
            const float2 st = sh.stat[0][h];
            const float den = st.y * kFewShare;
            const float4 x = *reinterpret_cast<const float4 *>(got + e);
            struct alignas(4 * sizeof(O)) Four {
                O e[4];
            } out;
            out.e[0] = from_float<O>(x.x / den);
            out.e[1] = from_float<O>(x.y / den);
            out.e[2] = from_float<O>(x.z / den);
            out.e[3] = from_float<O>(x.w / den);
            *reinterpret_cast<Four *>((O *)p.out + u.l * p.os.layer + u.b * p.os.stream + g * p.os.head + (long long)t * p.os.token + c) = out;
            if (c == 0 && p.lse) p.lse[(((size_t)u.l * p.streams + u.b) * p.Hkv * p.G + g) * p.n + t] = 0.6931471805599453f * (st.x + log2f(st.y));
        }
        return;
    }
    for (int i = threadIdx.x; i < share; i += kFewThreads) {
        const int e = u.rank * share + i;
        if (e >= all) break;
        const int h = e / p.d, c = e - h * p.d;
        float ref = -INFINITY, o = 0.f, sum = 0.f;
        float2 st[kFewMaxRanks];
        float x[kFewMaxRanks];
#pragma unroll
        for (uint32_t r = 0; r < kFewMaxRanks; ++r) {   // all reads at once
            st[r] = make_float2(-INFINITY, 0.f);
            x[r] = 0.f;
            if (r < u.ranks) {
                st[r] = sh.stat[r][h];
                x[r] = got[r * share + i];
            }
            ref = fmaxf(ref, st[r].x);
        }
#pragma unroll
        for (uint32_t r = 0; r < kFewMaxRanks; ++r) {
            const float f = few_scale(st[r].x, ref);
            o = fmaf(x[r], f, o);
            sum = fmaf(st[r].y, f, sum);
        }
        const int t = (u.row0 + h) / p.G, g = u.hkv * p.G + u.row0 + h - t * p.G;
        ((O *)p.out)[u.l * p.os.layer + u.b * p.os.stream + g * p.os.head + (long long)t * p.os.token + c] = from_float<O>(o / (sum * kFewShare));
        if (c == 0 && p.lse) p.lse[(((size_t)u.l * p.streams + u.b) * p.Hkv * p.G + g) * p.n + t] = 0.6931471805599453f * (ref + log2f(sum));
    }
}

// Tiles of 16 keys: kSparse, of the selected blocks; else of the pot's rows and, the last one, of the chunk's.
template <bool kSparse> struct FewTiles {
    int pot, all;
    __device__ __forceinline__ FewTiles(const FewParams &p, const FewUnit &u, int selected)
    {
        pot = kSparse ? selected * (p.block_rows / 16) : (p.len + 15) / 16;
        all = kSparse ? pot : pot + 1;   // (at most 16 tokens)
    }
    // first row and number of rows (0: none are there); fresh: they are the chunk's
    __device__ __forceinline__ void locate(const FewParams &p, const FewUnit &u, const uint16_t *list, int tile, int &row, int &count, bool &fresh) const
    {
        fresh = false;
        if (kSparse) {
            const int per = p.block_rows / 16, i = tile / per;
            row = list[i] * p.block_rows + (tile - i * per) * 16;
            count = max(0, min(16, p.len - row));
        } else if (tile < pot) {
            row = tile * 16;
            count = min(16, p.len - row);
        } else {
            fresh = true;
            row = 0;
            count = u.n;
        }
    }
};

// ------------------------------------------------------------------ bf16: warp-level tensor cores
constexpr int kFewStages = 3;
template <int D> struct FewRing {
    static constexpr size_t kBytes = (size_t)kFewWarps * kFewStages * 2 * 16 * D * 2;
    static constexpr size_t kGot = (kFewRows * D + 4 * kFewMaxRanks) * sizeof(float);
    static_assert(kBytes >= kScoreBytes + 8 * 1024 && kBytes >= kFewWarps * kFewRows * (D + 4) * sizeof(float), "scores and the merge take its place");
};

__device__ __forceinline__ void few_ldmatrix(uint32_t (&r)[4], uint32_t addr)
{
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0, %1, %2, %3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr));
}
__device__ __forceinline__ void few_ldmatrix_t(uint32_t (&r)[4], uint32_t addr)
{
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0, %1, %2, %3}, [%4];" : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr));
}
__device__ __forceinline__ void few_mma(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1)
{
    asm volatile(
        "mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
        : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint32_t few_pack(float lo, float hi)
{
    const __nv_bfloat162 h = __floats2bfloat162_rn(lo, hi);
    return *reinterpret_cast<const uint32_t *>(&h);
}
__device__ __forceinline__ float few_bf16(float x) { return __bfloat162float(__float2bfloat16_rn(x)); }

// grid (cluster, units, groups of 8 query rows).  D: channels, rounded up to 64, 128 or 256.
template <int D, bool kSparse>
__global__ void __launch_bounds__(kFewThreads)
few_mma_kernel(const __grid_constant__ FewParams p)
{
    cluster_arrive();
    pdl_wait();
    pdl_release();
    using T = __nv_bfloat16;
    constexpr int VPR = D / 8, NT = D / 8, STAGE = 16 * VPR;   // 16-byte vectors of a row, output tiles of 8 channels, vectors of a stage's keys
    extern __shared__ __align__(16) uint8_t few_raw[];
    const FewUnit u(p);
    using Ring = FewRing<D>;
    FewShared &sh = *reinterpret_cast<FewShared *>(few_raw + Ring::kBytes);
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, quad = lane >> 2, tq = lane & 3, vecs = p.d / 8;
    if (!kSparse && u.rows <= 0) {   // (the whole cluster)
        cluster_wait();
        return;
    }
    // A fragments of the queries: row quad, rows 8 .. 15 are zero
    uint32_t qa[D / 16][2];
    {
        const T *qr = (const T *)p.q + u.q_at(p, min(quad, u.rows - 1));
#pragma unroll
        for (int ks = 0; ks < D / 16; ++ks)
#pragma unroll
            for (int x = 0; x < 2; ++x) {
                const int c = ks * 16 + x * 8 + 2 * tq;
                qa[ks][x] = quad < u.rows && c < p.d ? __ldg(reinterpret_cast<const uint32_t *>(qr + c)) : 0u;
            }
    }
    const int selected = kSparse ? select_blocks<T>(sh, few_raw, (int)Ring::kBytes - kScoreBytes, p, u) : 0;
    const FewTiles<kSparse> tiles(p, u, selected);
    const uint4 *K = reinterpret_cast<const uint4 *>((const T *)p.K + (size_t)u.unit * p.unit_rows * p.d);
    const uint4 *V = reinterpret_cast<const uint4 *>((const T *)p.V + (size_t)u.unit * p.unit_rows * p.d);
    uint4 *ring = reinterpret_cast<uint4 *>(few_raw) + (size_t)warp * kFewStages * 2 * STAGE;
    const int w0 = u.rank * kFewWarps + warp, step = u.ranks * kFewWarps, mine = tiles.all > w0 ? (tiles.all - w0 + step - 1) / step : 0;

    auto issue = [&](int i) {   // this warp's i-th tile into stage i % kFewStages
        if (i < mine) {
            int row, count;
            bool fresh;
            tiles.locate(p, u, sh.list, w0 + i * step, row, count, fresh);
            constexpr int RX = 32 / VPR;   // rows that the warp's lanes cover
            const int r0 = lane / VPR, c = lane - r0 * VPR;
            const uint4 *gk = K + (size_t)row * vecs, *gv = V + (size_t)row * vecs;
            long long pk = vecs, pv = vecs;   // of a row
            if (!kSparse && fresh) {
                gk = reinterpret_cast<const uint4 *>((const T *)p.k + u.l * p.ks.layer + u.b * p.ks.stream + u.hkv * p.ks.head);
                gv = reinterpret_cast<const uint4 *>((const T *)p.v + u.l * p.vs.layer + u.b * p.vs.stream + u.hkv * p.vs.head);
                pk = p.ks.token / 8;
                pv = p.vs.token / 8;
            }
            gk += r0 * pk + c;
            gv += r0 * pv + c;
            uint4 *sk = ring + (size_t)(i % kFewStages) * 2 * STAGE, *sv = sk + STAGE;
#pragma unroll
            for (int x = 0; x < 16 / RX; ++x, gk += RX * pk, gv += RX * pv) {
                const int r = x * RX + r0, at = r * VPR + (c ^ (r & 7));
                const bool there = r < count && c < vecs;   // what is not becomes zeros
                few_cp_async16(sk + at, there ? gk : K, there);
                few_cp_async16(sv + at, there ? gv : V, there);
            }
        }
        asm volatile("cp.async.commit_group;" ::: "memory");
    };
#pragma unroll
    for (int i = 0; i < kFewStages - 1; ++i) issue(i);

    if (kSparse && p.list && u.rank == 0 && u.row0 == 0)
        for (int i = threadIdx.x; i < p.blocks; i += kFewThreads) p.list[(size_t)blockIdx.y * p.blocks + i] = i < selected ? sh.list[i] : -1;
    const int seen = (u.row0 + quad) / p.G + 1;   // of the chunk's rows
    float o[NT][4];
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) o[nt][0] = o[nt][1] = o[nt][2] = o[nt][3] = 0.f;
    float m = -INFINITY, l = 0.f;   // of row quad; l is this lane's share of the sum

    for (int i = 0; i < mine; ++i) {
        asm volatile("cp.async.wait_group %0;" ::"n"(kFewStages - 2) : "memory");
        __syncwarp();   // every lane's copies of tile i are in; every lane is done with the stage refilled next
        issue(i + kFewStages - 1);
        int row, count;
        bool fresh;
        tiles.locate(p, u, sh.list, w0 + i * step, row, count, fresh);
        if (count <= 0) continue;
        if (!kSparse && fresh) count = min(count, seen);
        const uint32_t sk = (uint32_t)__cvta_generic_to_shared(ring + (size_t)(i % kFewStages) * 2 * STAGE), sv = sk + STAGE * 16;
        // ---- S^T = q K^T for 16 keys: two column tiles of 8
        float s0[4] = {0.f, 0.f, 0.f, 0.f}, s1[4] = {0.f, 0.f, 0.f, 0.f}, z0[4] = {0.f, 0.f, 0.f, 0.f}, z1[4] = {0.f, 0.f, 0.f, 0.f};   // (even and odd steps: shorter chains)
        {
            const int r = (lane & 7) + ((lane >> 4) & 1) * 8, cs = (lane >> 3) & 1;
#pragma unroll
            for (int ks = 0; ks < D / 16; ++ks) {
                uint32_t b[4];
                few_ldmatrix(b, sk + (uint32_t)(r * VPR + ((2 * ks + cs) ^ (r & 7))) * 16);
                few_mma(ks & 1 ? z0 : s0, qa[ks][0], 0u, qa[ks][1], 0u, b[0], b[1]);
                few_mma(ks & 1 ? z1 : s1, qa[ks][0], 0u, qa[ks][1], 0u, b[2], b[3]);
            }
        }
        s0[0] += z0[0];
        s0[1] += z0[1];
        s1[0] += z1[0];
        s1[1] += z1[1];
        // this lane: row quad, keys 2 tq, + 1 and 8 + 2 tq, + 1 of the tile; the first key is there for every row
        float sc[4] = {s0[0] * p.scale_log2e, s0[1] * p.scale_log2e, s1[0] * p.scale_log2e, s1[1] * p.scale_log2e}, mt = -INFINITY;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            if ((j >> 1) * 8 + 2 * tq + (j & 1) >= count) sc[j] = -INFINITY;
            mt = fmaxf(mt, sc[j]);
        }
        mt = fmaxf(mt, __shfl_xor_sync(0xffffffffu, mt, 1));
        mt = fmaxf(mt, __shfl_xor_sync(0xffffffffu, mt, 2));
        const float mn = fmaxf(m, mt);
        if (__any_sync(0xffffffffu, mn > m)) {
            const float corr = few_scale(m, mn);
            l *= corr;
#pragma unroll
            for (int nt = 0; nt < NT; ++nt) {
                o[nt][0] *= corr;
                o[nt][1] *= corr;
                if (kSparse) {
                    o[nt][2] *= corr;
                    o[nt][3] *= corr;
                }
            }
            m = mn;
        }
        float w[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            w[j] = few_ex2(sc[j] - m);   // -inf -> 0
            l += w[j];
            w[j] *= kFewShare;
        }
        // A fragments of the weights (columns: the tile's keys); kSparse: the first two of three terms in rows 0 .. 7 and 8 .. 15, then the third
        const uint32_t a0 = few_pack(w[0], w[1]), a2 = few_pack(w[2], w[3]);
        uint32_t a1 = 0u, a3 = 0u, b0 = 0u, b2 = 0u;
        if (kSparse) {
            float mid[4], rest[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const float r = w[j] - few_bf16(w[j]);
                mid[j] = r;
                rest[j] = r - few_bf16(r);
            }
            a1 = few_pack(mid[0], mid[1]);
            a3 = few_pack(mid[2], mid[3]);
            b0 = few_pack(rest[0], rest[1]);
            b2 = few_pack(rest[2], rest[3]);
        }
        // ---- O += P V, two output tiles per ldmatrix
        const int r = (lane & 7) + ((lane >> 3) & 1) * 8, cv = lane >> 4;
#pragma unroll
        for (int nt = 0; nt < NT; nt += 2) {
            uint32_t b[4];
            few_ldmatrix_t(b, sv + (uint32_t)(r * VPR + ((nt + cv) ^ (r & 7))) * 16);
            few_mma(o[nt], a0, a1, a2, a3, b[0], b[1]);
            few_mma(o[nt + 1], a0, a1, a2, a3, b[2], b[3]);
            if (kSparse) {
                few_mma(o[nt], b0, 0u, b2, 0u, b[0], b[1]);
                few_mma(o[nt + 1], b0, 0u, b2, 0u, b[2], b[3]);
            }
        }
    }
    asm volatile("cp.async.wait_group 0;" ::: "memory");
    l += __shfl_xor_sync(0xffffffffu, l, 1);
    l += __shfl_xor_sync(0xffffffffu, l, 2);
    __syncthreads();   // every warp has left its ring: the memory now carries the merge
    float *part = reinterpret_cast<float *>(few_raw), *got = reinterpret_cast<float *>(few_raw + Ring::kBytes + sizeof(FewShared));
    if (quad < u.rows) {
        float *out = part + ((size_t)warp * u.rows + quad) * (p.d + 4) + 2 * tq;
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
            if (nt * 8 < p.d) *reinterpret_cast<float2 *>(out + nt * 8) = kSparse ? make_float2(o[nt][0] + o[nt][2], o[nt][1] + o[nt][3]) : make_float2(o[nt][0], o[nt][1]);
        if (tq == 0) sh.warp_stat[warp][quad] = make_float2(m, l);
    }
    if (!kSparse) cluster_wait();   // all of the cluster has started: its shared memory may be written
    if (kSparse) few_finish<float, true>(part, got, sh, p, u);
    else few_finish<T, false>(part, got, sh, p, u);
}

// ------------------------------------------------------------------ f32
// grid as above.  A lane has VPL vectors of a key's row (groups of lpk lanes).
template <int R, int VPL, bool kSparse>
__global__ void __launch_bounds__(kFewThreads)
few_fma_kernel(const __grid_constant__ FewParams p, int lpk)
{
    cluster_arrive();
    pdl_wait();
    pdl_release();
    constexpr int VE = 4, KT = 4;
    extern __shared__ __align__(16) uint8_t few_raw[];   // FewShared, the blocks' shares of the result, the warps' results (and before them the scores)
    const FewUnit u(p);
    FewShared &sh = *reinterpret_cast<FewShared *>(few_raw);
    float *got = reinterpret_cast<float *>(few_raw + sizeof(FewShared)), *part = got + R * p.d + 4 * kFewMaxRanks;
    if (!kSparse && u.rows <= 0) {   // (the whole cluster)
        cluster_wait();
        return;
    }
    const int selected = kSparse ? select_blocks<float>(sh, reinterpret_cast<uint8_t *>(part), kFewFmaRoom, p, u) : 0;
    if (kSparse && p.list && u.rank == 0 && u.row0 == 0)
        for (int i = threadIdx.x; i < p.blocks; i += kFewThreads) p.list[(size_t)blockIdx.y * p.blocks + i] = i < selected ? sh.list[i] : -1;
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, vecs = p.d / VE;
    const int gpw = 32 / lpk, gq = lane / lpk, gl = lane - gq * lpk, ng = kFewWarps * gpw, grp = warp * gpw + gq;
    const float4 *K = reinterpret_cast<const float4 *>((const float *)p.K + (size_t)u.unit * p.unit_rows * p.d);
    const float4 *V = reinterpret_cast<const float4 *>((const float *)p.V + (size_t)u.unit * p.unit_rows * p.d);
    const float4 *Kn = nullptr, *Vn = nullptr;
    if (!kSparse) {
        Kn = reinterpret_cast<const float4 *>((const float *)p.k + u.l * p.ks.layer + u.b * p.ks.stream + u.hkv * p.ks.head);
        Vn = reinterpret_cast<const float4 *>((const float *)p.v + u.l * p.vs.layer + u.b * p.vs.stream + u.hkv * p.vs.head);
    }
    float4 qf[R][VPL], acc[R][VPL];
    float m[R], l[R];
#pragma unroll
    for (int h = 0; h < R; ++h) {
        m[h] = -INFINITY;
        l[h] = 0.f;
#pragma unroll
        for (int i = 0; i < VPL; ++i) {
            const int v = gl + i * lpk;
            qf[h][i] = acc[h][i] = make_float4(0.f, 0.f, 0.f, 0.f);
            if (h < u.rows && v < vecs) {
                qf[h][i] = *reinterpret_cast<const float4 *>((const float *)p.q + u.q_at(p, h) + v * VE);
                qf[h][i].x *= p.scale_log2e;
                qf[h][i].y *= p.scale_log2e;
                qf[h][i].z *= p.scale_log2e;
                qf[h][i].w *= p.scale_log2e;
            }
        }
    }
    // all keys numbered through; this block of the cluster has an even share, its lane groups take turns
    const int all = kSparse ? selected * p.block_rows : p.len + u.n, per = (all + u.ranks - 1) / u.ranks, first = u.rank * per, last = min(all, first + per);
    for (int base = first; base < last; base += KT * ng) {
        float s[KT][R];
        int seen_by[KT];   // the first row of the block that sees the key; R: none
        float4 vv[KT][VPL];
#pragma unroll
        for (int j = 0; j < KT; ++j) {
            const int i = base + j * ng + grp;
            seen_by[j] = R;
            const float4 *ka = K, *va = V;
            if (i < last) {
                if (kSparse) {
                    const int row = sh.list[i / p.block_rows] * p.block_rows + i % p.block_rows;
                    if (row < p.len) {
                        seen_by[j] = 0;
                        ka = K + (size_t)row * vecs;
                        va = V + (size_t)row * vecs;
                    }
                } else if (i < p.len) {
                    seen_by[j] = 0;
                    ka = K + (size_t)i * vecs;
                    va = V + (size_t)i * vecs;
                } else {
                    const int t = i - p.len;
                    seen_by[j] = min(t * p.G - u.row0, R);   // (below 0: all)
                    ka = Kn + t * (p.ks.token / VE);
                    va = Vn + t * (p.vs.token / VE);
                }
            }
#pragma unroll
            for (int h = 0; h < R; ++h) s[j][h] = 0.f;
#pragma unroll
            for (int x = 0; x < VPL; ++x) {
                const int v = gl + x * lpk;
                vv[j][x] = make_float4(0.f, 0.f, 0.f, 0.f);
                if (seen_by[j] < R && v < vecs) {
                    const float4 kk = ka[v];
                    vv[j][x] = va[v];
#pragma unroll
                    for (int h = 0; h < R; ++h)
                        s[j][h] = fmaf(kk.x, qf[h][x].x, fmaf(kk.y, qf[h][x].y, fmaf(kk.z, qf[h][x].z, fmaf(kk.w, qf[h][x].w, s[j][h]))));
                }
            }
        }
        for (int off = lpk >> 1; off >= 1; off >>= 1) {
#pragma unroll
            for (int j = 0; j < KT; ++j)
#pragma unroll
                for (int h = 0; h < R; ++h) s[j][h] += __shfl_xor_sync(0xffffffffu, s[j][h], off);
        }
#pragma unroll
        for (int h = 0; h < R; ++h) {
            float mn = m[h];
#pragma unroll
            for (int j = 0; j < KT; ++j) mn = fmaxf(mn, h >= seen_by[j] ? s[j][h] : -INFINITY);
            const float corr = few_scale(m[h], mn);
            m[h] = mn;
            l[h] *= corr;
#pragma unroll
            for (int x = 0; x < VPL; ++x) {
                acc[h][x].x *= corr;
                acc[h][x].y *= corr;
                acc[h][x].z *= corr;
                acc[h][x].w *= corr;
            }
#pragma unroll
            for (int j = 0; j < KT; ++j) {
                float w = h >= seen_by[j] ? few_ex2(s[j][h] - mn) : 0.f;
                l[h] += w;
                w *= kFewShare;
#pragma unroll
                for (int x = 0; x < VPL; ++x) {
                    acc[h][x].x = fmaf(w, vv[j][x].x, acc[h][x].x);
                    acc[h][x].y = fmaf(w, vv[j][x].y, acc[h][x].y);
                    acc[h][x].z = fmaf(w, vv[j][x].z, acc[h][x].z);
                    acc[h][x].w = fmaf(w, vv[j][x].w, acc[h][x].w);
                }
            }
        }
    }
    for (int off = lpk; off < 32; off <<= 1) {   // the groups of a warp
#pragma unroll
        for (int h = 0; h < R; ++h) {
            const float m2 = __shfl_xor_sync(0xffffffffu, m[h], off), l2 = __shfl_xor_sync(0xffffffffu, l[h], off), mn = fmaxf(m[h], m2);
            const float ca = few_scale(m[h], mn), cb = few_scale(m2, mn);
            l[h] = l[h] * ca + l2 * cb;
            m[h] = mn;
#pragma unroll
            for (int x = 0; x < VPL; ++x) {
                acc[h][x].x = acc[h][x].x * ca + __shfl_xor_sync(0xffffffffu, acc[h][x].x, off) * cb;
                acc[h][x].y = acc[h][x].y * ca + __shfl_xor_sync(0xffffffffu, acc[h][x].y, off) * cb;
                acc[h][x].z = acc[h][x].z * ca + __shfl_xor_sync(0xffffffffu, acc[h][x].z, off) * cb;
                acc[h][x].w = acc[h][x].w * ca + __shfl_xor_sync(0xffffffffu, acc[h][x].w, off) * cb;
            }
        }
    }
    __syncthreads();   // (the scores' place)
    if (gq == 0) {
#pragma unroll
        for (int h = 0; h < R; ++h) {
            if (h >= u.rows) break;
            float4 *row = reinterpret_cast<float4 *>(part + ((size_t)warp * u.rows + h) * (p.d + 4));
#pragma unroll
            for (int x = 0; x < VPL; ++x)
                if (gl + x * lpk < vecs) row[gl + x * lpk] = acc[h][x];
            if (gl == 0) sh.warp_stat[warp][h] = make_float2(m[h], l[h]);
        }
    }
    if (!kSparse) cluster_wait();   // all of the cluster has started: its shared memory may be written
    few_finish<float, kSparse>(part, got, sh, p, u);
}

// ------------------------------------------------------------------ host side
// blocks of a cluster: as many as find a place at once, and at least one tile of 16 keys for every warp.  (8 warps a block, one on an SM: a cluster of 16 then needs 16 SMs of one
// GPC to itself, and 8 of them do not run side by side: one token over 4095 rows, 8 units 13.8 us against 8.9.)
template <typename... A>
inline cudaError_t launch_few_t(ClusterFit &fit, void (*kern)(FewParams, A...), const FewParams &p, size_t smem, int keys, cudaStream_t stream, A... args)
{
    const cudaError_t e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
    if (e != cudaSuccess) return e;
    const dim3 block(kFewThreads);
    const int groups = (p.n * p.G + kFewRows - 1) / kFewRows, units = p.layers * p.streams * p.Hkv;
    const int cluster = choose_cluster(fit, kern, block, smem, (long long)units * groups, (keys + 16 * kFewWarps - 1) / (16 * kFewWarps));
    return launch_cluster(kern, dim3(cluster, units, groups), block, smem, cluster, stream, p, args...);
}

template <int R, int VPL, bool kSparse>
inline cudaError_t launch_few_fma(const FewParams &p, int lpk, int keys, cudaStream_t stream)
{
    static ClusterFit fit;
    size_t part = (size_t)kFewWarps * R * (p.d + 4) * sizeof(float);
    if (kSparse && part < kScoreBytes + kFewFmaRoom) part = kScoreBytes + kFewFmaRoom;
    return launch_few_t<int>(fit, few_fma_kernel<R, VPL, kSparse>, p, sizeof(FewShared) + (R * p.d + 4 * kFewMaxRanks) * sizeof(float) + part, keys, stream, lpk);
}

template <int D, bool kSparse>
inline cudaError_t launch_few_mma(const FewParams &p, int keys, cudaStream_t stream)
{
    static ClusterFit fit;
    using Ring = FewRing<D>;
    return launch_few_t<>(fit, few_mma_kernel<D, kSparse>, p, Ring::kBytes + sizeof(FewShared) + Ring::kGot, keys, stream);
}

template <bool kSparse>
inline cudaError_t launch_few(const FewParams &p, bool f32, cudaStream_t stream)
{
    const int keys = kSparse ? (p.len < p.blocks * p.block_rows ? p.len : p.blocks * p.block_rows) : p.len + p.n;
    if (!f32) {
        if (p.d <= 64) return launch_few_mma<64, kSparse>(p, keys, stream);
        return p.d <= 128 ? launch_few_mma<128, kSparse>(p, keys, stream) : launch_few_mma<256, kSparse>(p, keys, stream);
    }
    const int vecs = p.d / 4, rows = p.n * p.G;
    int lpk = 1;
    while (lpk < vecs && lpk < 32) lpk *= 2;
    if (vecs > 32) {
        if (rows == 1) return launch_few_fma<1, 2, kSparse>(p, lpk, keys, stream);
        return rows <= 4 ? launch_few_fma<4, 2, kSparse>(p, lpk, keys, stream) : launch_few_fma<8, 2, kSparse>(p, lpk, keys, stream);
    }
    if (rows == 1) return launch_few_fma<1, 1, kSparse>(p, lpk, keys, stream);
    if (rows == 2) return launch_few_fma<2, 1, kSparse>(p, lpk, keys, stream);
    return rows <= 4 ? launch_few_fma<4, 1, kSparse>(p, lpk, keys, stream) : launch_few_fma<8, 1, kSparse>(p, lpk, keys, stream);
}

}  // namespace ipotk
