// Attention of at most 8 query rows of a KV head over many keys: generation.  Two calls come here:
//   a chunk of few tokens (kSparse = false): rows t * G + g over the pot's rows and the chunk's rows 0 .. t;
//   one token over selected blocks of the pot (kSparse = true; the query heads of a KV head in groups of 8).
// Either is a stream of keys and values through few rows, split over a thread-block cluster per unit: bound by HBM, or where there
// are few units by the latency of one chain - launch, (scores, selection,) first loads, merge.
//
// Selection (kSparse).  s_b = sum_h sum_c max(q_hc lo_bc, q_hc hi_bc) over the unit's query heads.  A channel takes hi where q is positive
//   and lo where it is negative, so the heads' positive and negative parts are added first: s_b = sum_c (q+_c hi_bc + q-_c lo_bc), two
//   products per channel whatever the number of heads.  In 64 bits: which block is in must not depend on the order of a sum.  The
//   cluster's blocks share the scoring and put every score into each other's shared memory; then each finds, for itself, the
//   (n - 1)-th largest of the order-preserving 64-bit keys bit by bit from the highest bit in which they differ (a count over the
//   block per bit, and the search ends as soon as a count is right), and lists the chosen blocks in ascending order.
// few_mma_kernel (bf16): a warp owns tiles of 16 keys and a ring of cp.async stages of its own, rows XOR-swizzled for ldmatrix;
//   S^T = q K^T and O += P V are m16n8k16 tiles with fp32 accumulation.  Of the 16 rows 8 are queries: the other 8 of the output product hold the
//   second of three bf16 terms of the weights where the result is fp32 (kSparse: 24 bits, nothing is rounded to bf16); a
//   bf16 result takes the weights' first term.  tcgen05 does not fit: its smallest tile has 64 rows.
// few_fma_kernel (f32): a group of lanes owns a key (a 16-byte vector of the row or two per lane), four keys at a time.
// Merge: the block's warps in shared memory, the cluster's blocks through distributed shared memory: no scratch, no atomics.
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

constexpr int kFewThreads = 128, kFewWarps = kFewThreads / 32;
constexpr int kFewRows = 8;       // query rows of a block
constexpr int kFewBlocks = 2048;  // blocks of a unit: 32768 slots, 16 rows

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

// ------------------------------------------------------------------ scores and selection
struct BlockSelection {
    uint16_t list[kFewBlocks];
    unsigned long long reach[2][kFewWarps];
    int count[2][kFewWarps];
};

// Monotone map double -> uint64.
__device__ __forceinline__ unsigned long long order_key64(double s)
{
    const unsigned long long b = (unsigned long long)__double_as_longlong(s + 0.0);   // (-0 counts as 0)
    return b ^ ((unsigned long long)((long long)b >> 63) | 0x8000000000000000ull);
}

// All blocks of the cluster: sel.list becomes the ascending list of the chosen blocks, its length is returned.  score: kFewBlocks numbers of
// shared memory that is free meanwhile, at the same place in every block.
template <typename T>
__device__ __forceinline__ int select_blocks(BlockSelection &sel, double *score, const FewParams &p, const FewUnit &u)
{
    constexpr int VE = RowVec<T>::kElems, NV = sizeof(T) == 2 ? 2 : 4, KPT = kFewBlocks / kFewThreads;   // 256 channels: 64 vectors of bf16 bounds, 128 of f32
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, vecs = p.d / VE, pieces = 2 * vecs;
    const int total = (p.len + p.block_rows - 1) / p.block_rows, want = min(p.blocks, total);
    if (want == total) {
        for (int b = threadIdx.x; b < total; b += kFewThreads) sel.list[b] = b;
        __syncthreads();
        return want;
    }
    // this lane's channels: vector lane + 32 i of a block's lower, then upper bounds; what the heads' queries sum up to there
    double w[NV * VE];
    const T *q = (const T *)p.q + u.l * p.qs.layer + u.b * p.qs.stream + (long long)u.hkv * p.G * p.qs.head;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
        const int piece = lane + 32 * i;
#pragma unroll
        for (int e = 0; e < VE; ++e) w[i * VE + e] = 0.0;
        if (piece >= pieces) continue;
        const bool upper = piece >= vecs;
        for (int h = 0; h < p.G; ++h) {
            const RowVec<T> x = *reinterpret_cast<const RowVec<T> *>(q + h * p.qs.head + (piece - (upper ? vecs : 0)) * VE);
#pragma unroll
            for (int e = 0; e < VE; ++e) {
                const float f = to_float(x.e[e]);
                if (upper ? f > 0.f : f < 0.f) w[i * VE + e] += (double)f;
            }
        }
    }
    const T *lo = (const T *)p.lo + (size_t)u.unit * p.unit_blocks * p.d, *hi = (const T *)p.hi + (size_t)u.unit * p.unit_blocks * p.d;
    constexpr int BF = 4;   // blocks whose bounds are on their way at once
    const int stride = u.ranks * kFewWarps;
    for (int b0 = u.rank * kFewWarps + warp; b0 < total - 1; b0 += BF * stride) {
        RowVec<T> x[BF][NV];
#pragma unroll
        for (int f = 0; f < BF; ++f)
#pragma unroll
            for (int i = 0; i < NV; ++i) {
                const int piece = lane + 32 * i, b = b0 + f * stride;
                const bool upper = piece >= vecs;
                if (piece < pieces && b < total - 1) x[f][i] = *reinterpret_cast<const RowVec<T> *>((upper ? hi : lo) + (size_t)b * p.d + (piece - (upper ? vecs : 0)) * VE);
            }
#pragma unroll
        for (int f = 0; f < BF; ++f) {
            const int b = b0 + f * stride;
            if (b >= total - 1) break;
            double s = 0.0;
#pragma unroll
            for (int i = 0; i < NV; ++i)
                if (lane + 32 * i < pieces) {
#pragma unroll
                    for (int e = 0; e < VE; ++e) s = fma(w[i * VE + e], (double)to_float(x[f][i].e[e]), s);
                }
#pragma unroll
            for (int off = 16; off >= 1; off >>= 1) s += __shfl_xor_sync(0xffffffffu, s, off);
            if (lane < (int)u.ranks) cluster_st(cluster_addr(score + b, lane), s);
        }
    }
    cluster_sync();
    // a thread has the keys of `per` neighbouring blocks; the newest block is in and stands outside
    const int others = total - 1, per = (others + kFewThreads - 1) / kFewThreads, first = threadIdx.x * per, here = max(0, min(per, others - first));
    unsigned long long key[KPT], top = 0, low = ~0ull;
#pragma unroll
    for (int i = 0; i < KPT; ++i) {
        key[i] = 0;
        if (i < here) {
            key[i] = order_key64(score[first + i]);
            top = max(top, key[i]);
            low = min(low, key[i]);
        }
    }
#pragma unroll
    for (int off = 16; off >= 1; off >>= 1) {
        top = max(top, __shfl_xor_sync(0xffffffffu, top, off));
        low = min(low, __shfl_xor_sync(0xffffffffu, low, off));
    }
    if (lane == 0) {
        sel.reach[0][warp] = top;
        sel.reach[1][warp] = low;
    }
    __syncthreads();
#pragma unroll
    for (int w2 = 0; w2 < kFewWarps; ++w2) {
        top = max(top, sel.reach[0][w2]);
        low = min(low, sel.reach[1][w2]);
    }
    const int need = want - 1;
    auto block_sum = [&](int v, int parity) {
        v = __reduce_add_sync(0xffffffffu, v);
        if (lane == 0) sel.count[parity][warp] = v;
        __syncthreads();
        int s = 0;
#pragma unroll
        for (int w2 = 0; w2 < kFewWarps; ++w2) s += sel.count[parity][w2];
        return s;
    };
    // the largest `at` such that at least `need` keys are >= at (all bits of the common prefix are those of every key)
    unsigned long long at = 0;
    bool exact = false;   // exactly the keys >= at are in
    int parity = 0;
    if (need > 0) {
        const unsigned long long diff = top ^ low;
        int bit = diff ? 63 - __clzll((long long)diff) : -1;
        at = bit >= 0 ? top & ~((2ull << bit) - 1) : top;
        for (; bit >= 0 && !exact; --bit) {
            const unsigned long long cand = at | (1ull << bit);
            int c = 0;
#pragma unroll
            for (int i = 0; i < KPT; ++i) {
                if (i >= per) break;
                c += i < here && key[i] >= cand;
            }
            c = block_sum(c, parity);
            parity ^= 1;
            if (c >= need) at = cand;
            exact = c == need;
        }
    }
    // keys above `at` are in, and of those equal to it the first ones (all of them where the count was exact)
    int above = 0, equal = 0;
#pragma unroll
    for (int i = 0; i < KPT; ++i) {
        above += i < here && key[i] > at;
        equal += i < here && key[i] == at;
    }
    if (need == 0) above = equal = 0;
    // exclusive sums over the threads before this one: both counts in one number
    int both = above | equal << 16, incl = both;
#pragma unroll
    for (int off = 1; off < 32; off <<= 1) {
        const int v = __shfl_up_sync(0xffffffffu, incl, off);
        if (lane >= off) incl += v;
    }
    if (lane == 31) sel.count[parity][warp] = incl;
    __syncthreads();
    int before = incl - both, all = 0;
#pragma unroll
    for (int w2 = 0; w2 < kFewWarps; ++w2) {
        const int c = sel.count[parity][w2];
        if (w2 < warp) before += c;
        all += c;
    }
    const int take_equal = need - (all & 0xffff);
    int eq_before = before >> 16, place = (before & 0xffff) + min(eq_before, take_equal);
    if (need > 0) {
#pragma unroll
        for (int i = 0; i < KPT; ++i) {
            if (i >= here) continue;
            bool in = key[i] > at;
            if (key[i] == at) in = eq_before++ < take_equal;
            if (in) sel.list[place++] = first + i;
        }
    }
    if (threadIdx.x == 0) sel.list[need] = total - 1;
    __syncthreads();
    return want;
}

// ------------------------------------------------------------------ the end of a block's work
// part: [warps][rows][d + 2] (output against a reference, the reference in binary orders, the sum); mine: [rows][d + 2] of this block.
template <typename O>
__device__ __forceinline__ void few_finish(float *part, float *mine, const FewParams &p, const FewUnit &u)
{
    const int ds = p.d + 2;
    __syncthreads();
    for (int e = threadIdx.x; e < u.rows * ds; e += kFewThreads) {
        const int h = e / ds, c = e - h * ds;
        float ref = -INFINITY;
#pragma unroll
        for (int w = 0; w < kFewWarps; ++w) ref = fmaxf(ref, part[(w * u.rows + h) * ds + p.d]);
        float v = ref;
        if (c != p.d) {
            v = 0.f;
#pragma unroll
            for (int w = 0; w < kFewWarps; ++w) v = fmaf(part[(w * u.rows + h) * ds + c], few_scale(part[(w * u.rows + h) * ds + p.d], ref), v);
        }
        mine[e] = v;
    }
    cluster_sync();
    for (int e = u.rank * kFewThreads + threadIdx.x; e < u.rows * p.d; e += u.ranks * kFewThreads) {
        const int h = e / p.d, c = e - h * p.d;
        float ref = -INFINITY, o = 0.f, den = 0.f;
        constexpr int RB = 4;   // ranks whose values are on their way at once
        for (uint32_t r0 = 0; r0 < u.ranks; r0 += RB) {
            float m[RB], s[RB], x[RB];
#pragma unroll
            for (int i = 0; i < RB; ++i) {
                const uint32_t r = min(r0 + i, u.ranks - 1);
                m[i] = cluster_ld(cluster_addr(mine + h * ds + p.d, r));
                s[i] = cluster_ld(cluster_addr(mine + h * ds + p.d + 1, r));
                x[i] = cluster_ld(cluster_addr(mine + h * ds + c, r));
                if (r0 + i >= u.ranks) m[i] = -INFINITY;
            }
            float top = ref;
#pragma unroll
            for (int i = 0; i < RB; ++i) top = fmaxf(top, m[i]);
            const float f0 = few_scale(ref, top);
            o *= f0;
            den *= f0;
            ref = top;
#pragma unroll
            for (int i = 0; i < RB; ++i) {
                const float f = few_scale(m[i], ref);
                o = fmaf(x[i], f, o);
                den = fmaf(s[i], f, den);
            }
        }
        const int t = (u.row0 + h) / p.G, g = u.hkv * p.G + u.row0 + h - t * p.G;
        ((O *)p.out)[u.l * p.os.layer + u.b * p.os.stream + g * p.os.head + (long long)t * p.os.token + c] = from_float<O>(o / den);
        if (c == 0 && p.lse) p.lse[(((size_t)u.l * p.streams + u.b) * p.Hkv * p.G + g) * p.n + t] = 0.6931471805599453f * (ref + log2f(den));
    }
    cluster_sync();   // no block ends while others read its results
}

// Tiles of 16 keys: kSparse, of the selected blocks; else of the pot's rows and, the last one, of the chunk's.
template <bool kSparse> struct FewTiles {
    int pot, all;
    __device__ __forceinline__ FewTiles(const FewParams &p, const FewUnit &u, int selected)
    {
        pot = kSparse ? selected * (p.block_rows / 16) : (p.len + 15) / 16;
        all = kSparse ? pot : pot + 1;   // (at most 8 tokens)
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
    static_assert(kBytes >= kFewBlocks * sizeof(double) && kBytes >= (kFewWarps + 1) * kFewRows * (D + 2) * 4, "scores and the merge take its place");
};

__device__ __forceinline__ void few_cp_async16(void *dst, const void *src, bool there)
{
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"((uint32_t)__cvta_generic_to_shared(dst)), "l"(src), "r"(there ? 16 : 0) : "memory");
}
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
    pdl_wait();
    pdl_release();
    using T = __nv_bfloat16;
    constexpr int VPR = D / 8, NT = D / 8, STAGE = 16 * VPR;   // 16-byte vectors of a row, output tiles of 8 channels, vectors of a stage's keys
    extern __shared__ __align__(16) uint8_t few_raw[];
    const FewUnit u(p);
    BlockSelection *sel = reinterpret_cast<BlockSelection *>(few_raw + FewRing<D>::kBytes);
    int selected = 0;
    if (kSparse) {
        cluster_sync();   // all of the cluster has started: its shared memory may be written
        selected = select_blocks<T>(*sel, reinterpret_cast<double *>(few_raw), p, u);
        if (p.list && u.rank == 0 && u.row0 == 0)
            for (int i = threadIdx.x; i < p.blocks; i += kFewThreads) p.list[(size_t)blockIdx.y * p.blocks + i] = i < selected ? sel->list[i] : -1;
    } else if (u.rows <= 0) {
        return;   // (the whole cluster)
    }
    const FewTiles<kSparse> tiles(p, u, selected);
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, quad = lane >> 2, tq = lane & 3, vecs = p.d / 8;
    const uint4 *K = reinterpret_cast<const uint4 *>((const T *)p.K + (size_t)u.unit * p.unit_rows * p.d);
    const uint4 *V = reinterpret_cast<const uint4 *>((const T *)p.V + (size_t)u.unit * p.unit_rows * p.d);
    uint4 *ring = reinterpret_cast<uint4 *>(few_raw) + (size_t)warp * kFewStages * 2 * STAGE;
    const int w0 = u.rank * kFewWarps + warp, step = u.ranks * kFewWarps, mine = tiles.all > w0 ? (tiles.all - w0 + step - 1) / step : 0;

    auto issue = [&](int i) {   // this warp's i-th tile into stage i % kFewStages
        if (i < mine) {
            int row, count;
            bool fresh;
            tiles.locate(p, u, kSparse ? sel->list : nullptr, w0 + i * step, row, count, fresh);
            const uint4 *gk = K + (size_t)row * vecs, *gv = V + (size_t)row * vecs;
            long long pk = vecs, pv = vecs;   // of a row
            if (!kSparse && fresh) {
                gk = reinterpret_cast<const uint4 *>((const T *)p.k + u.l * p.ks.layer + u.b * p.ks.stream + u.hkv * p.ks.head);
                gv = reinterpret_cast<const uint4 *>((const T *)p.v + u.l * p.vs.layer + u.b * p.vs.stream + u.hkv * p.vs.head);
                pk = p.ks.token / 8;
                pv = p.vs.token / 8;
            }
            uint4 *sk = ring + (size_t)(i % kFewStages) * 2 * STAGE, *sv = sk + STAGE;
#pragma unroll
            for (int x = 0; x < STAGE / 32; ++x) {
                const int e = x * 32 + lane, r = e / VPR, c = e - r * VPR, at = r * VPR + (c ^ (r & 7));
                const bool there = r < count && c < vecs;   // what is not becomes zeros
                few_cp_async16(sk + at, there ? gk + r * pk + c : K, there);
                few_cp_async16(sv + at, there ? gv + r * pv + c : V, there);
            }
        }
        asm volatile("cp.async.commit_group;" ::: "memory");
    };
#pragma unroll
    for (int i = 0; i < kFewStages - 1; ++i) issue(i);

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
        tiles.locate(p, u, kSparse ? sel->list : nullptr, w0 + i * step, row, count, fresh);
        if (count <= 0) continue;
        if (!kSparse && fresh) count = min(count, seen);
        const uint32_t sk = (uint32_t)__cvta_generic_to_shared(ring + (size_t)(i % kFewStages) * 2 * STAGE), sv = sk + STAGE * 16;
        // ---- S^T = q K^T for 16 keys: two column tiles of 8
        float s0[4] = {0.f, 0.f, 0.f, 0.f}, s1[4] = {0.f, 0.f, 0.f, 0.f};
        {
            const int r = (lane & 7) + ((lane >> 4) & 1) * 8, cs = (lane >> 3) & 1;
#pragma unroll
            for (int ks = 0; ks < D / 16; ++ks) {
                uint32_t b[4];
                few_ldmatrix(b, sk + (uint32_t)(r * VPR + ((2 * ks + cs) ^ (r & 7))) * 16);
                few_mma(s0, qa[ks][0], 0u, qa[ks][1], 0u, b[0], b[1]);
                few_mma(s1, qa[ks][0], 0u, qa[ks][1], 0u, b[2], b[3]);
            }
        }
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
    float *part = reinterpret_cast<float *>(few_raw);
    const int ds = p.d + 2;
    if (quad < u.rows) {
        float *out = part + ((size_t)warp * u.rows + quad) * ds;
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
            if (nt * 8 < p.d) {
                out[nt * 8 + 2 * tq] = kSparse ? o[nt][0] + o[nt][2] : o[nt][0];
                out[nt * 8 + 2 * tq + 1] = kSparse ? o[nt][1] + o[nt][3] : o[nt][1];
            }
        if (tq == 0) {
            out[p.d] = m;
            out[p.d + 1] = l;
        }
    }
    if (kSparse) few_finish<float>(part, part + (size_t)kFewWarps * kFewRows * ds, p, u);
    else few_finish<T>(part, part + (size_t)kFewWarps * kFewRows * ds, p, u);
}

// ------------------------------------------------------------------ f32
// grid as above.  A lane has VPL vectors of a key's row (groups of lpk lanes).
template <int R, int VPL, bool kSparse>
__global__ void __launch_bounds__(kFewThreads)
few_fma_kernel(const __grid_constant__ FewParams p, int lpk)
{
    pdl_wait();
    pdl_release();
    constexpr int VE = 4, KT = 4;
    extern __shared__ __align__(16) uint8_t few_raw[];   // the selection, then [warps][R][d + 2] and [R][d + 2]
    const FewUnit u(p);
    BlockSelection *sel = reinterpret_cast<BlockSelection *>(few_raw);
    float *part = reinterpret_cast<float *>(few_raw + (kSparse ? sizeof(BlockSelection) : 0));
    int selected = 0;
    if (kSparse) {
        cluster_sync();
        selected = select_blocks<float>(*sel, reinterpret_cast<double *>(part), p, u);
        if (p.list && u.rank == 0 && u.row0 == 0)
            for (int i = threadIdx.x; i < p.blocks; i += kFewThreads) p.list[(size_t)blockIdx.y * p.blocks + i] = i < selected ? sel->list[i] : -1;
    } else if (u.rows <= 0) {
        return;
    }
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
                    const int row = sel->list[i / p.block_rows] * p.block_rows + i % p.block_rows;
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
                    seen_by[j] = t * p.G;   // (row0 is 0)
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
                const float w = h >= seen_by[j] ? few_ex2(s[j][h] - mn) : 0.f;
                l[h] += w;
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
    const int ds = p.d + 2;
    if (gq == 0) {
#pragma unroll
        for (int h = 0; h < R; ++h) {
            if (h >= u.rows) break;
            float *row = part + ((size_t)warp * u.rows + h) * ds;
#pragma unroll
            for (int x = 0; x < VPL; ++x) {
                const int v = gl + x * lpk;
                if (v < vecs) {
                    row[v * VE] = acc[h][x].x;
                    row[v * VE + 1] = acc[h][x].y;
                    row[v * VE + 2] = acc[h][x].z;
                    row[v * VE + 3] = acc[h][x].w;
                }
            }
            if (gl == 0) {
                row[p.d] = m[h];
                row[p.d + 1] = l[h];
            }
        }
    }
    few_finish<float>(part, part + (size_t)kFewWarps * R * ds, p, u);
}

// ------------------------------------------------------------------ host side
template <typename... A>
inline cudaError_t launch_few_t(void (*kern)(FewParams, A...), const FewParams &p, size_t smem, int cluster, cudaStream_t stream, A... args)
{
    const cudaError_t e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
    if (e != cudaSuccess) return e;
    return launch_cluster(kern, dim3(cluster, p.layers * p.streams * p.Hkv, (p.n * p.G + kFewRows - 1) / kFewRows), dim3(kFewThreads), smem, cluster, stream, p, args...);
}

template <int R, int VPL, bool kSparse>
inline cudaError_t launch_few_fma(const FewParams &p, int lpk, int cluster, cudaStream_t stream)
{
    size_t smem = (size_t)(kFewWarps + 1) * R * (p.d + 2) * sizeof(float);
    if (kSparse) smem = sizeof(BlockSelection) + (smem > kFewBlocks * sizeof(double) ? smem : kFewBlocks * sizeof(double));
    return launch_few_t<int>(few_fma_kernel<R, VPL, kSparse>, p, smem, cluster, stream, lpk);
}

template <int D, bool kSparse>
inline cudaError_t launch_few_mma(const FewParams &p, int cluster, cudaStream_t stream)
{
    return launch_few_t<>(few_mma_kernel<D, kSparse>, p, FewRing<D>::kBytes + (kSparse ? sizeof(BlockSelection) : 0), cluster, stream);
}

template <bool kSparse>
inline cudaError_t launch_few(const FewParams &p, bool f32, int sm_count, cudaStream_t stream)
{
    // blocks of a cluster: as many as find a place at once (two on an SM), and at least one tile of 16 keys for every warp
    const long long units = (long long)p.layers * p.streams * p.Hkv * ((p.n * p.G + kFewRows - 1) / kFewRows);
    const int keys = kSparse ? (p.len < p.blocks * p.block_rows ? p.len : p.blocks * p.block_rows) : p.len + p.n;
    int cluster = 1;
    while (cluster < 16 && units * cluster * 2 <= 2LL * sm_count && keys > cluster * 16 * kFewWarps) cluster *= 2;
    if (!f32) return p.d <= 64 ? launch_few_mma<64, kSparse>(p, cluster, stream) : p.d <= 128 ? launch_few_mma<128, kSparse>(p, cluster, stream) : launch_few_mma<256, kSparse>(p, cluster, stream);
    const int vecs = p.d / 4, rows = p.n * p.G;
    int lpk = 1;
    while (lpk < vecs && lpk < 32) lpk *= 2;
    if (vecs > 32)
        return rows == 1 ? launch_few_fma<1, 2, kSparse>(p, lpk, cluster, stream) : rows <= 4 ? launch_few_fma<4, 2, kSparse>(p, lpk, cluster, stream)
                                                                                             : launch_few_fma<8, 2, kSparse>(p, lpk, cluster, stream);
    return rows == 1 ? launch_few_fma<1, 1, kSparse>(p, lpk, cluster, stream) : rows == 2 ? launch_few_fma<2, 1, kSparse>(p, lpk, cluster, stream)
         : rows <= 4 ? launch_few_fma<4, 1, kSparse>(p, lpk, cluster, stream)
                                                                                         : launch_few_fma<8, 1, kSparse>(p, lpk, cluster, stream);
}

}  // namespace ipotk
