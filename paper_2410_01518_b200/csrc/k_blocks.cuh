// Generation over selected blocks of the pot.  Slots are taken in blocks of R; the smallest and largest value of every channel
// over a block's keys bound every logit in it:  q . k_j <= sum_c max(q_c lo_c, q_c hi_c)  for all j of the block.
//
// block_bounds_kernel: those bounds, for the blocks whose rows have changed.  Bound: HBM, every changed key once.
//
// blocks_attn_kernel: one unit per thread-block cluster.
//   score    s_b = sum_h sum_c max(q_hc lo_bc, q_hc hi_bc) over the unit's query heads.  A channel takes hi where q is positive and lo where it is
//            negative, so the heads' positive and negative parts are added first: s_b = sum_c (q+_c hi_bc + q-_c lo_bc), two products
//            per channel whatever the number of heads.  In 64 bits: which block is in must not depend on the order of a sum.  The
//            cluster's blocks share the scoring and put every score into each other's shared memory.
//   select   the block of the newest rows and the n - 1 others with the largest score (ties: the lower block), as an ascending list, in every
//            block of the cluster.
//   attend   softmax attention over the rows of the selected blocks: a group of lanes owns a key (a 16-byte vector of the row or two per lane), four keys at a
//            time; running maximum and sum per head, everything fp32.
//   merge    groups, warps, and the cluster's blocks through distributed shared memory.
#pragma once
#include "common.cuh"
#include "ops.h"
#include "k_rotary.cuh"   // RowVec, to_float

namespace ipotk {

// ------------------------------------------------------------------ bounds
constexpr int kBoundThreads = 128;

// grid (blocks from first_block on, units).  Threads: a vector of the row each, several rows side by side.
template <typename T>
__global__ void __launch_bounds__(kBoundThreads)
block_bounds_kernel(const T *__restrict__ K, T *__restrict__ lo, T *__restrict__ hi, int first_block, int rows_per_block, int len, int d, size_t unit_rows, int unit_blocks)
{
    pdl_wait();
    pdl_release();
    constexpr int VE = RowVec<T>::kElems;
    __shared__ RowVec<T> part[2][kBoundThreads];
    const int vecs = d / VE, side = kBoundThreads / vecs, r0 = threadIdx.x / vecs, v = threadIdx.x - r0 * vecs;
    const int block = first_block + blockIdx.x, n = min(rows_per_block, len - block * rows_per_block);
    const RowVec<T> *src = reinterpret_cast<const RowVec<T> *>(K + ((size_t)blockIdx.y * unit_rows + (size_t)block * rows_per_block) * d);
    RowVec<T> a, b;
    if (r0 < side && r0 < n) {
        a = b = src[(size_t)r0 * vecs + v];
        for (int r = r0 + side; r < n; r += side) {
            const RowVec<T> x = src[(size_t)r * vecs + v];
#pragma unroll
            for (int e = 0; e < VE; ++e) {
                if (to_float(x.e[e]) < to_float(a.e[e])) a.e[e] = x.e[e];
                if (to_float(x.e[e]) > to_float(b.e[e])) b.e[e] = x.e[e];
            }
        }
        part[0][threadIdx.x] = a;
        part[1][threadIdx.x] = b;
    }
    __syncthreads();
    if (r0 == 0) {
        for (int r = 1; r < min(side, n); ++r) {
            const RowVec<T> x = part[0][r * vecs + v], y = part[1][r * vecs + v];
#pragma unroll
            for (int e = 0; e < VE; ++e) {
                if (to_float(x.e[e]) < to_float(a.e[e])) a.e[e] = x.e[e];
                if (to_float(y.e[e]) > to_float(b.e[e])) b.e[e] = y.e[e];
            }
        }
        const size_t at = ((size_t)blockIdx.y * unit_blocks + block) * vecs + v;
        reinterpret_cast<RowVec<T> *>(lo)[at] = a;
        reinterpret_cast<RowVec<T> *>(hi)[at] = b;
    }
}

template <typename T>
inline cudaError_t launch_block_bounds_t(const void *K, void *lo, void *hi, int first_row, int len, int rows, int d, int units, size_t unit_rows, int unit_blocks, cudaStream_t stream)
{
    const int first = first_row / rows;
    const dim3 grid((len + rows - 1) / rows - first, units);
    return launch_pdl(block_bounds_kernel<T>, grid, dim3(kBoundThreads), 0, stream, (const T *)K, (T *)lo, (T *)hi, first, rows, len, d, unit_rows, unit_blocks);
}

// ------------------------------------------------------------------ the cluster
__device__ __forceinline__ uint32_t cluster_rank()
{
    uint32_t r;
    asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
    return r;
}
__device__ __forceinline__ uint32_t cluster_size()
{
    uint32_t r;
    asm volatile("mov.u32 %0, %%cluster_nctarank;" : "=r"(r));
    return r;
}
__device__ __forceinline__ void cluster_sync()
{
    __syncwarp();
    asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}
// The address of `p`, a pointer into this block's shared memory, in block `rank` of the cluster.
__device__ __forceinline__ uint32_t cluster_addr(const void *p, uint32_t rank)
{
    uint32_t a;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(a) : "r"((uint32_t)__cvta_generic_to_shared(p)), "r"(rank));
    return a;
}
__device__ __forceinline__ float cluster_ld(uint32_t addr)
{
    float v;
    asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(v) : "r"(addr) : "memory");
    return v;
}
__device__ __forceinline__ void cluster_st(uint32_t addr, double v) { asm volatile("st.shared::cluster.f64 [%0], %1;" ::"r"(addr), "d"(v) : "memory"); }

// ------------------------------------------------------------------ scores and selection
constexpr int kBlkThreads = 256, kBlkWarps = kBlkThreads / 32;
constexpr int kBlkMax = 2048;     // blocks of a unit: 32768 slots, 16 rows
constexpr int kBlkHeads = 8;      // query heads of a launch's block

struct BlockSelection {
    double score[kBlkMax];
    int list[kBlkMax];
    uint8_t in[kBlkMax];
};

// All blocks of the cluster: sel.list becomes the ascending list of the chosen blocks, its length is returned.
template <typename T>
__device__ __forceinline__ int select_blocks(BlockSelection &sel, const BlocksParams &p, int unit, uint32_t rank, uint32_t ranks)
{
    constexpr int VE = RowVec<T>::kElems, MAXV = 128 / 32;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, vecs = p.d / VE, pieces = 2 * vecs;
    const int total = (p.len + p.rows - 1) / p.rows, want = min(p.blocks, total);
    if (want < total) {
        // this lane's channels: vector (lane + 32 i) of a block's lower, then upper bounds; what the heads' queries sum up to there
        double w[MAXV * VE > 16 ? 16 : MAXV * VE];
        constexpr int NV = (MAXV * VE > 16 ? 16 : MAXV * VE) / VE;   // 256 channels: 2 vectors of bf16, 4 of f32
        const T *q = (const T *)p.q + (size_t)(unit - p.unit0) * p.G * p.d;
#pragma unroll
        for (int i = 0; i < NV; ++i) {
            const int piece = lane + 32 * i;
#pragma unroll
            for (int e = 0; e < VE; ++e) w[i * VE + e] = 0.0;
            if (piece >= pieces) continue;
            const bool upper = piece >= vecs;
            for (int h = 0; h < p.G; ++h) {
                const RowVec<T> x = *reinterpret_cast<const RowVec<T> *>(q + (size_t)h * p.d + (piece - (upper ? vecs : 0)) * VE);
#pragma unroll
                for (int e = 0; e < VE; ++e) {
                    const float f = to_float(x.e[e]);
                    if (upper ? f > 0.f : f < 0.f) w[i * VE + e] += (double)f;
                }
            }
        }
        const T *lo = (const T *)p.lo + (size_t)unit * p.unit_blocks * p.d, *hi = (const T *)p.hi + (size_t)unit * p.unit_blocks * p.d;
        for (int b = rank * kBlkWarps + warp; b < total - 1; b += ranks * kBlkWarps) {
            double s = 0.0;
#pragma unroll
            for (int i = 0; i < NV; ++i) {
                const int piece = lane + 32 * i;
                if (piece >= pieces) continue;
                const bool upper = piece >= vecs;
                const RowVec<T> x = *reinterpret_cast<const RowVec<T> *>((upper ? hi : lo) + (size_t)b * p.d + (piece - (upper ? vecs : 0)) * VE);
#pragma unroll
                for (int e = 0; e < VE; ++e) s = fma(w[i * VE + e], (double)to_float(x.e[e]), s);
            }
#pragma unroll
            for (int off = 16; off >= 1; off >>= 1) s += __shfl_xor_sync(0xffffffffu, s, off);
            if (lane < (int)ranks) cluster_st(cluster_addr(&sel.score[b], lane), s);
        }
        cluster_sync();
        for (int b = threadIdx.x; b < total; b += kBlkThreads) {
            bool in = b == total - 1;
            if (!in) {
                const double s = sel.score[b];
                int before = 0;
                for (int o = 0; o < total - 1; ++o) {
                    const double x = sel.score[o];
                    before += x > s || (x == s && o < b);
                }
                in = before < want - 1;
            }
            sel.in[b] = in;
        }
        __syncthreads();
        if (warp == 0) {
            int n = 0;
            for (int b0 = 0; b0 < total; b0 += 32) {
                const bool in = b0 + lane < total && sel.in[b0 + lane];
                const uint32_t m = __ballot_sync(0xffffffffu, in);
                if (in) sel.list[n + __popc(m & ((1u << lane) - 1))] = b0 + lane;
                n += __popc(m);
            }
        }
    } else {
        for (int b = threadIdx.x; b < total; b += kBlkThreads) sel.list[b] = b;
    }
    __syncthreads();
    return want;
}

__device__ __forceinline__ float blk_ex2(float x)
{
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
__device__ __forceinline__ float blk_scale(float m, float ref) { return m == -INFINITY ? 0.f : blk_ex2(m - ref); }

// The cluster's results: part holds [warps][G][d + 2] (output against a reference, the reference, the sum) of this block.
__device__ __forceinline__ void blocks_finish(float *part, float *mine, int G, int d, const BlocksParams &p, int out_row, uint32_t rank, uint32_t ranks)
{
    const int ds = d + 2;
    __syncthreads();
    for (int e = threadIdx.x; e < G * ds; e += kBlkThreads) {
        const int h = e / ds, c = e - h * ds;
        float ref = -INFINITY;
        for (int w = 0; w < kBlkWarps; ++w) ref = fmaxf(ref, part[(w * G + h) * ds + d]);
        float v = ref;
        if (c != d) {
            v = 0.f;
            for (int w = 0; w < kBlkWarps; ++w) v = fmaf(part[(w * G + h) * ds + c], blk_scale(part[(w * G + h) * ds + d], ref), v);
        }
        mine[e] = v;
    }
    cluster_sync();
    for (int e = rank * kBlkThreads + threadIdx.x; e < G * d; e += ranks * kBlkThreads) {
        const int h = e / d, c = e - h * d;
        float ref = -INFINITY, o = 0.f, den = 0.f;
        for (uint32_t r = 0; r < ranks; ++r) ref = fmaxf(ref, cluster_ld(cluster_addr(mine + h * ds + d, r)));
        for (uint32_t r = 0; r < ranks; ++r) {
            const float f = blk_scale(cluster_ld(cluster_addr(mine + h * ds + d, r)), ref);
            o = fmaf(cluster_ld(cluster_addr(mine + h * ds + c, r)), f, o);
            den = fmaf(cluster_ld(cluster_addr(mine + h * ds + d + 1, r)), f, den);
        }
        p.out[(size_t)(out_row + h) * d + c] = o / den;
        if (c == 0 && p.lse) p.lse[out_row + h] = 0.6931471805599453f * (ref + log2f(den));
    }
    cluster_sync();   // no block ends while others read its results
}

// grid (cluster, units, groups of kBlkHeads query heads).  A lane has VPL vectors of a key's row (lane group of lpk lanes).
template <typename T, int G, int VPL>
__global__ void __launch_bounds__(kBlkThreads)
blocks_attn_kernel(const __grid_constant__ BlocksParams p, int lpk)
{
    pdl_wait();
    pdl_release();
    constexpr int VE = RowVec<T>::kElems, KT = 4;
    __shared__ BlockSelection sel;
    extern __shared__ float blk_part[];   // [warps][heads][d + 2], then [heads][d + 2]
    const int unit = p.unit0 + blockIdx.y, h0 = blockIdx.z * kBlkHeads, heads = min(G, p.G - h0);
    const uint32_t rank = cluster_rank(), ranks = cluster_size();
    cluster_sync();   // all of the cluster has started: its shared memory may be written
    const int n = select_blocks<T>(sel, p, unit, rank, ranks);
    if (p.list && rank == 0 && h0 == 0)
        for (int i = threadIdx.x; i < p.blocks; i += kBlkThreads) p.list[(size_t)(unit - p.unit0) * p.blocks + i] = i < n ? sel.list[i] : -1;

    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, vecs = p.d / VE;
    const int gpw = 32 / lpk, gq = lane / lpk, gl = lane - gq * lpk, ng = kBlkWarps * gpw, grp = warp * gpw + gq;
    const RowVec<T> *K = reinterpret_cast<const RowVec<T> *>((const T *)p.K + (size_t)unit * p.unit_rows * p.d);
    const RowVec<T> *V = reinterpret_cast<const RowVec<T> *>((const T *)p.V + (size_t)unit * p.unit_rows * p.d);
    float qf[G][VPL * VE], acc[G][VPL * VE], m[G], l[G];
#pragma unroll
    for (int h = 0; h < G; ++h) {
        m[h] = -INFINITY;
        l[h] = 0.f;
#pragma unroll
        for (int i = 0; i < VPL; ++i) {
            const int v = gl + i * lpk;
            RowVec<T> x;
            const bool there = h < heads && v < vecs;
            if (there) x = *reinterpret_cast<const RowVec<T> *>((const T *)p.q + ((size_t)(unit - p.unit0) * p.G + h0 + h) * p.d + v * VE);
#pragma unroll
            for (int e = 0; e < VE; ++e) {
                qf[h][i * VE + e] = there ? to_float(x.e[e]) * p.scale_log2e : 0.f;
                acc[h][i * VE + e] = 0.f;
            }
        }
    }
    // the selected rows, numbered through the list; this block of the cluster has an even share, its lane groups take turns
    const int all = n * p.rows, per = (all + ranks - 1) / ranks, first = rank * per, last = min(all, first + per);
    for (int base = first; base < last; base += KT * ng) {
        float s[KT][G];
        bool valid[KT];
        RowVec<T> vv[KT][VPL];
#pragma unroll
        for (int j = 0; j < KT; ++j) {
            const int i = base + j * ng + grp;
            int row = 0;
            valid[j] = i < last;
            if (valid[j]) {
                row = sel.list[i / p.rows] * p.rows + i % p.rows;
                valid[j] = row < p.len;
            }
#pragma unroll
            for (int h = 0; h < G; ++h) s[j][h] = 0.f;
#pragma unroll
            for (int i2 = 0; i2 < VPL; ++i2) {
                const int v = gl + i2 * lpk;
                if (valid[j] && v < vecs) {
                    const RowVec<T> x = K[(size_t)row * vecs + v];
                    vv[j][i2] = V[(size_t)row * vecs + v];
#pragma unroll
                    for (int h = 0; h < G; ++h)
#pragma unroll
                        for (int e = 0; e < VE; ++e) s[j][h] = fmaf(to_float(x.e[e]), qf[h][i2 * VE + e], s[j][h]);
                } else {
#pragma unroll
                    for (int e = 0; e < VE; ++e) vv[j][i2].e[e] = from_float<T>(0.f);
                }
            }
        }
        for (int off = lpk >> 1; off >= 1; off >>= 1) {
#pragma unroll
            for (int j = 0; j < KT; ++j)
#pragma unroll
                for (int h = 0; h < G; ++h) s[j][h] += __shfl_xor_sync(0xffffffffu, s[j][h], off);
        }
#pragma unroll
        for (int h = 0; h < G; ++h) {
            float mn = m[h];
#pragma unroll
            for (int j = 0; j < KT; ++j) mn = fmaxf(mn, valid[j] ? s[j][h] : -INFINITY);
            const float corr = blk_scale(m[h], mn);
            m[h] = mn;
            l[h] *= corr;
#pragma unroll
            for (int e = 0; e < VPL * VE; ++e) acc[h][e] *= corr;
#pragma unroll
            for (int j = 0; j < KT; ++j) {
                const float w = valid[j] ? blk_ex2(s[j][h] - mn) : 0.f;
                l[h] += w;
#pragma unroll
                for (int i2 = 0; i2 < VPL; ++i2)
#pragma unroll
                    for (int e = 0; e < VE; ++e) acc[h][i2 * VE + e] = fmaf(w, to_float(vv[j][i2].e[e]), acc[h][i2 * VE + e]);
            }
        }
    }
    for (int off = lpk; off < 32; off <<= 1) {   // the groups of a warp
#pragma unroll
        for (int h = 0; h < G; ++h) {
            const float m2 = __shfl_xor_sync(0xffffffffu, m[h], off), l2 = __shfl_xor_sync(0xffffffffu, l[h], off), mn = fmaxf(m[h], m2);
            const float ca = blk_scale(m[h], mn), cb = blk_scale(m2, mn);
            l[h] = l[h] * ca + l2 * cb;
            m[h] = mn;
#pragma unroll
            for (int e = 0; e < VPL * VE; ++e) acc[h][e] = acc[h][e] * ca + __shfl_xor_sync(0xffffffffu, acc[h][e], off) * cb;
        }
    }
    const int ds = p.d + 2;
    if (gq == 0) {
#pragma unroll
        for (int h = 0; h < G; ++h) {
            if (h >= heads) break;
            float *row = blk_part + ((size_t)warp * heads + h) * ds;
#pragma unroll
            for (int i = 0; i < VPL; ++i)
                if (gl + i * lpk < vecs)
#pragma unroll
                    for (int e = 0; e < VE; ++e) row[(gl + i * lpk) * VE + e] = acc[h][i * VE + e];
            if (gl == 0) {
                row[p.d] = m[h];
                row[p.d + 1] = l[h];
            }
        }
    }
    float *mine = blk_part + (size_t)kBlkWarps * G * ds;
    blocks_finish(blk_part, mine, heads, p.d, p, (unit - p.unit0) * p.G + h0, rank, ranks);
}

template <typename T, int G, int VPL>
inline cudaError_t launch_blocks_t(const BlocksParams &p, int lpk, int cluster, cudaStream_t stream)
{
    const size_t smem = (size_t)(kBlkWarps + 1) * G * (p.d + 2) * sizeof(float);
    auto kern = blocks_attn_kernel<T, G, VPL>;
    const cudaError_t e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
    if (e != cudaSuccess) return e;
    cudaLaunchConfig_t lc = {};
    lc.gridDim = dim3(cluster, p.layers * p.streams * p.Hkv, (p.G + kBlkHeads - 1) / kBlkHeads);
    lc.blockDim = dim3(kBlkThreads);
    lc.dynamicSmemBytes = smem;
    lc.stream = stream;
    cudaLaunchAttribute at[2];
    at[0].id = cudaLaunchAttributeClusterDimension;
    at[0].val.clusterDim.x = cluster;
    at[0].val.clusterDim.y = at[0].val.clusterDim.z = 1;
    at[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    at[1].val.programmaticStreamSerializationAllowed = 1;
    lc.attrs = at;
    lc.numAttrs = 2;
    return cudaLaunchKernelEx(&lc, kern, p, lpk);
}

template <typename T>
inline cudaError_t launch_blocks(const BlocksParams &p, int cluster, cudaStream_t stream)
{
    const int vecs = p.d * (int)sizeof(T) / 16;
    int lpk = 1;
    while (lpk < vecs && lpk < 32) lpk *= 2;
    if constexpr (sizeof(T) == 4) {   // (256 channels of bf16 are 32 vectors)
        if (vecs > 32) {
            if (p.G == 1) return launch_blocks_t<T, 1, 2>(p, lpk, cluster, stream);
            if (p.G <= 4) return launch_blocks_t<T, 4, 2>(p, lpk, cluster, stream);
            return launch_blocks_t<T, 8, 2>(p, lpk, cluster, stream);
        }
    }
    if (p.G == 1) return launch_blocks_t<T, 1, 1>(p, lpk, cluster, stream);
    if (p.G == 2) return launch_blocks_t<T, 2, 1>(p, lpk, cluster, stream);
    if (p.G <= 4) return launch_blocks_t<T, 4, 1>(p, lpk, cluster, stream);
    return launch_blocks_t<T, 8, 1>(p, lpk, cluster, stream);
}

}  // namespace ipotk
