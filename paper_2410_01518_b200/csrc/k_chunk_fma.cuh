// Attention of a chunk of new tokens over the pot and, causally, over itself, with fp32 FMAs: f32 pots, and bf16 calls that the tensor-core
// kernel does not take.  out_h[t] = sum_j softmax_j(q_h[t] . k_j / sqrt(d)) v_j over the pot's rows [0, len) and the chunk's rows 0 .. t.
//
// The query heads of a KV head share its keys, so a unit's rows are folded token by token: row t * G + g.  A block has BM of
// them and goes over the keys they see in tiles of 64, with the running maximum and sum of the softmax.  A thread has 4 rows x 4 keys of S = Q K^T, summed over
// pairs of channels with packed FMAs from rows as they lie in memory (pitches keep the 16-byte reads free of bank conflicts), and 4 rows x
// d / 16 channels of O += P V in registers; P goes through shared memory.  Few row tiles spread their keys over a cluster, whose blocks merge through distributed shared
// memory.  The next tile's keys are on their way (cp.async) while this one's values are multiplied, the next values during the next logits: either has one buffer.
// (With loads that were waited for, 8 warps a block: 1000 tokens of 8 heads of 128 channels over 2048 rows 524 us, now 384.)  Bound: FMA issue and shared-memory reads (32 packed FMAs per eight 16-byte reads).
#pragma once
#include <algorithm>

#include "common.cuh"
#include "ops.h"
#include "cluster.cuh"
#include "k_rotary.cuh"   // RowVec, to_float, from_float

namespace ipotk {

constexpr int kCfKeys = 64;

template <int DP, int BM> struct ChunkFmaSmem {
    static constexpr int kThreads = 4 * BM, kPitch = DP + 4, kPPitch = kCfKeys + 16;
    float q[BM][kPitch];        // at the end the block's partial result
    float k[kCfKeys][kPitch];   // keys and values of a tile
    float v[kCfKeys][kPitch];
    float p[BM][kPPitch];
    float2 stat[BM];
};

__device__ __forceinline__ float chunk_ex2(float x)
{
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

// Tokens of stream b that are there.
__device__ __forceinline__ int chunk_tokens(const ChunkParams &p, int b) { return p.tokens ? min(max(__ldg(p.tokens + b), 0), p.n) : p.n; }

// grid: cluster x (row tiles, the longest first) x units.
template <typename T, int DP, int BM>
__global__ void __launch_bounds__(4 * BM)
chunk_fma_kernel(const __grid_constant__ ChunkParams p, int units)
{
    pdl_wait();
    pdl_release();
    using Smem = ChunkFmaSmem<DP, BM>;
    constexpr int VE = RowVec<T>::kElems, CV = DP / 64, NT = Smem::kThreads, RS = BM / 4;   // 4-channel vectors of a thread; threads; rows between a thread's
    extern __shared__ __align__(16) uint8_t chunk_raw[];
    Smem &sm = *reinterpret_cast<Smem *>(chunk_raw);
    const uint32_t rank = cluster_rank(), ranks = cluster_size();
    const int item = blockIdx.x / ranks, items = gridDim.x / ranks, unit = item % units, hkv = unit % p.Hkv, b = unit / p.Hkv % p.streams, l = unit / p.Hkv / p.streams;
    const int n = chunk_tokens(p, b), G = p.G, row0 = (items / units - 1 - item / units) * BM;
    if (row0 >= n * G) return;   // (the whole cluster)
    const int rows = min(BM, n * G - row0), all_keys = p.len + (row0 + rows - 1) / G + 1, tiles = (all_keys + kCfKeys - 1) / kCfKeys;
    const int first = (int)((long long)tiles * rank / ranks) * kCfKeys, keys = min(all_keys, (int)((long long)tiles * (rank + 1) / ranks) * kCfKeys);
    // weights enter the product with the values times this power of two: however many keys there are, their sum is at most 1, and no sum on the way is larger than the largest value
    const float share = __int_as_float((127 - (32 - __clz(all_keys))) << 23);
    const int tid = threadIdx.x, ty = tid >> 4, tx = tid & 15, vecs = p.d / VE;
    const T *potK = (const T *)p.potK + (size_t)(p.unit0 + unit) * p.unit_rows * p.d, *potV = (const T *)p.potV + (size_t)(p.unit0 + unit) * p.unit_rows * p.d;
    const T *newK = (const T *)p.k + l * p.ks.layer + b * p.ks.stream + hkv * p.ks.head, *newV = (const T *)p.v + l * p.vs.layer + b * p.vs.stream + hkv * p.vs.head;
    const T *q = (const T *)p.q + l * p.qs.layer + b * p.qs.stream + (long long)hkv * G * p.qs.head;

    // channels that are not there count as zeros
    for (int i = tid; i < BM * (DP - p.d); i += NT) {
        const int r = i / (DP - p.d), c = p.d + i - r * (DP - p.d);
        sm.q[r][c] = 0.f;
        if (r < kCfKeys) sm.k[r][c] = sm.v[r][c] = 0.f;
    }
    auto put = [&](float *dst, const T *src, bool there, float scale) {   // a vector, as floats; zeros where there is none
        RowVec<T> x;
        if (there) x = *reinterpret_cast<const RowVec<T> *>(src);
#pragma unroll
        for (int e = 0; e < VE; e += 4)
            *reinterpret_cast<float4 *>(dst + e) = there ? make_float4(to_float(x.e[e]) * scale, to_float(x.e[e + 1]) * scale, to_float(x.e[e + 2]) * scale, to_float(x.e[e + 3]) * scale)
                                                         : make_float4(0.f, 0.f, 0.f, 0.f);
    };
    for (int i = tid; i < BM * vecs; i += NT) {
        const int r = i / vecs, v = i - r * vecs, t = (row0 + r) / G, g = row0 + r - t * G;
        put(&sm.q[r][v * VE], q + (long long)t * p.qs.token + g * p.qs.head + v * VE, r < rows, p.scale_log2e);
    }
    // a tile's keys or values, in flight when this returns (f32) or there
    auto load = [&](float (*dst)[Smem::kPitch], const T *pot, const T *fresh, long long token, int k0) {
        for (int i = tid; i < kCfKeys * vecs; i += NT) {
            const int r = i / vecs, v = i - r * vecs, j = k0 + r;
            const T *src = j >= keys ? pot : (j < p.len ? pot + (size_t)j * p.d : fresh + (j - p.len) * token) + v * VE;
            if constexpr (sizeof(T) == 4)
                asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"((uint32_t)__cvta_generic_to_shared(&dst[r][v * VE])), "l"(src), "r"(j < keys ? 16 : 0) : "memory");
            else
                put(&dst[r][v * VE], src, j < keys, 1.f);
        }
        asm volatile("cp.async.commit_group;" ::: "memory");
    };
    if (first < keys) {
        load(sm.k, potK, newK, p.ks.token, first);
        load(sm.v, potV, newV, p.vs.token, first);
    }
    // a thread's rows are ty + RS i, its keys tx + 16 j of a tile, its channels 64 c + 4 tx ..
    float m[4], sum[4];
    float4 acc[4][CV];
    int limit[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        m[i] = -INFINITY;
        sum[i] = 0.f;
        limit[i] = p.len + (row0 + ty + RS * i) / G + 1;
#pragma unroll
        for (int c = 0; c < CV; ++c) acc[i][c] = make_float4(0.f, 0.f, 0.f, 0.f);
    }
    for (int k0 = first; k0 < keys; k0 += kCfKeys) {
        asm volatile("cp.async.wait_group 1;" ::: "memory");   // the keys (the values were asked for behind them)
        __syncthreads();
        float s[4][4];
        {
            float2 s2[4][4];
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int j = 0; j < 4; ++j) s2[i][j] = make_float2(0.f, 0.f);
#pragma unroll 4
            for (int c = 0; c < DP; c += 4) {
                float4 a[4], k4[4];
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    a[i] = *reinterpret_cast<const float4 *>(&sm.q[ty + RS * i][c]);
                    k4[i] = *reinterpret_cast<const float4 *>(&sm.k[tx + 16 * i][c]);
                }
#pragma unroll
                for (int i = 0; i < 4; ++i)
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        s2[i][j] = __ffma2_rn(make_float2(a[i].x, a[i].y), make_float2(k4[j].x, k4[j].y), s2[i][j]);
                        s2[i][j] = __ffma2_rn(make_float2(a[i].z, a[i].w), make_float2(k4[j].z, k4[j].w), s2[i][j]);
                    }
            }
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int j = 0; j < 4; ++j) s[i][j] = s2[i][j].x + s2[i][j].y;
        }
        __syncthreads();   // the keys have been read
        const bool more = k0 + kCfKeys < keys;
        if (more) load(sm.k, potK, newK, p.ks.token, k0 + kCfKeys);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            float mt = -INFINITY;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                if (k0 + tx + 16 * j >= limit[i]) s[i][j] = -INFINITY;
                mt = fmaxf(mt, s[i][j]);
            }
#pragma unroll
            for (int off = 8; off >= 1; off >>= 1) mt = fmaxf(mt, __shfl_xor_sync(0xffffffffu, mt, off));
            const float mn = fmaxf(m[i], mt), ref = mn == -INFINITY ? 0.f : mn, corr = chunk_ex2(m[i] - ref);
            float ps = 0.f;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                s[i][j] = chunk_ex2(s[i][j] - ref);
                ps += s[i][j];
                sm.p[ty + RS * i][tx + 16 * j] = s[i][j] * share;
            }
            m[i] = mn;
            sum[i] = sum[i] * corr + ps;   // this thread's share
#pragma unroll
            for (int c = 0; c < CV; ++c) acc[i][c] = make_float4(acc[i][c].x * corr, acc[i][c].y * corr, acc[i][c].z * corr, acc[i][c].w * corr);
        }
        if (more) asm volatile("cp.async.wait_group 1;" ::: "memory");   // the values
        else asm volatile("cp.async.wait_group 0;" ::: "memory");
        __syncthreads();   // (a row of P is its half warp's own)
#pragma unroll 2
        for (int j = 0; j < kCfKeys; j += 4) {   // (beyond the last key P and the values are zeros)
            float4 a[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) a[i] = *reinterpret_cast<const float4 *>(&sm.p[ty + RS * i][j]);
#pragma unroll
            for (int e = 0; e < 4; ++e)
#pragma unroll
                for (int c = 0; c < CV; ++c) {
                    const float4 v4 = *reinterpret_cast<const float4 *>(&sm.v[j + e][c * 64 + tx * 4]);
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const float w = e == 0 ? a[i].x : e == 1 ? a[i].y : e == 2 ? a[i].z : a[i].w;
                        const float2 lo = __ffma2_rn(make_float2(w, w), make_float2(v4.x, v4.y), make_float2(acc[i][c].x, acc[i][c].y));
                        const float2 hi = __ffma2_rn(make_float2(w, w), make_float2(v4.z, v4.w), make_float2(acc[i][c].z, acc[i][c].w));
                        acc[i][c] = make_float4(lo.x, lo.y, hi.x, hi.y);
                    }
                }
        }
        __syncthreads();   // the values have been read
        if (more) load(sm.v, potV, newV, p.vs.token, k0 + kCfKeys);
    }
    const long long lse0 = ((long long)l * p.streams + b) * p.Hkv * G + hkv * G;
    T *out = (T *)p.out + l * p.os.layer + b * p.os.stream + (long long)hkv * G * p.os.head;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
#pragma unroll
        for (int off = 8; off >= 1; off >>= 1) sum[i] += __shfl_xor_sync(0xffffffffu, sum[i], off);
    }
    if (ranks == 1) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int r = ty + RS * i, t = (row0 + r) / G, g = row0 + r - t * G;
            if (r >= rows) continue;
            T *o = out + g * p.os.head + (long long)t * p.os.token;
            const float inv = 1.f / (sum[i] * share);
#pragma unroll
            for (int c = 0; c < CV; ++c) {
                struct alignas(4 * sizeof(T)) Four {
                    T e[4];
                } x;
                x.e[0] = from_float<T>(acc[i][c].x * inv);
                x.e[1] = from_float<T>(acc[i][c].y * inv);
                x.e[2] = from_float<T>(acc[i][c].z * inv);
                x.e[3] = from_float<T>(acc[i][c].w * inv);
                if (c * 64 + tx * 4 < p.d) *reinterpret_cast<Four *>(o + c * 64 + tx * 4) = x;
            }
            if (tx == 0 && p.lse) p.lse[(lse0 + g) * p.n + t] = 0.6931471805599453f * (m[i] + log2f(sum[i]));
        }
        return;
    }
    // ---- the cluster: partial results in place of the queries, merged four channels of a row per thread
    __syncthreads();
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        const int r = ty + RS * i;
#pragma unroll
        for (int c = 0; c < CV; ++c) *reinterpret_cast<float4 *>(&sm.q[r][c * 64 + tx * 4]) = acc[i][c];
        if (tx == 0) sm.stat[r] = make_float2(m[i], sum[i]);
    }
    cluster_sync();
    for (int e = rank * NT + tid; e < rows * (p.d / 4); e += ranks * NT) {
        const int r = e / (p.d / 4), c = e - r * (p.d / 4), t = (row0 + r) / G, g = row0 + r - t * G;
        float ref = -INFINITY, den = 0.f, o[4] = {0.f, 0.f, 0.f, 0.f};
        for (uint32_t k = 0; k < ranks; ++k) ref = fmaxf(ref, cluster_ld(cluster_addr(&sm.stat[r].x, k)));
        for (uint32_t k = 0; k < ranks; ++k) {
            const uint32_t st = cluster_addr(&sm.stat[r], k), src = cluster_addr(&sm.q[r][4 * c], k);
            const float f = chunk_ex2(cluster_ld(st) - ref);   // (some rank has seen a key: ref is finite)
            const float4 x = cluster_ld4(src);
            den = fmaf(cluster_ld(st + 4), f, den);
            o[0] = fmaf(x.x, f, o[0]);
            o[1] = fmaf(x.y, f, o[1]);
            o[2] = fmaf(x.z, f, o[2]);
            o[3] = fmaf(x.w, f, o[3]);
        }
        T *dst = out + g * p.os.head + (long long)t * p.os.token + 4 * c;
#pragma unroll
        for (int x = 0; x < 4; ++x) dst[x] = from_float<T>(o[x] / (den * share));
        if (c == 0 && p.lse) p.lse[(lse0 + g) * p.n + t] = 0.6931471805599453f * (ref + log2f(den));
    }
    cluster_sync();   // no block ends while others read its results
}

template <typename T, int DP, int BM>
inline cudaError_t launch_chunk_fma_t(const ChunkParams &p, cudaStream_t stream)
{
    using Smem = ChunkFmaSmem<DP, BM>;
    static_assert(sizeof(Smem) <= 232448, "shared memory of a block");
    auto kern = chunk_fma_kernel<T, DP, BM>;
    const cudaError_t e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)sizeof(Smem));
    if (e != cudaSuccess) return e;
    const int units = p.layers * p.streams * p.Hkv;
    const long long items = ((long long)p.n * p.G + BM - 1) / BM * units;
    static ClusterFit fit;
    const int cluster = choose_cluster(fit, kern, dim3(Smem::kThreads), sizeof(Smem), items, std::min(8, (p.len + p.n + 2 * kCfKeys - 1) / (2 * kCfKeys)));   // two key tiles each
    if (items * cluster > 0x7fffffff) return cudaErrorInvalidValue;
    return launch_cluster(kern, dim3((unsigned)(items * cluster)), dim3(Smem::kThreads), sizeof(Smem), cluster, stream, p, units);
}

template <typename T>
inline cudaError_t launch_chunk_fma(const ChunkParams &p, cudaStream_t stream)
{
    // 64 rows: three blocks of them share an SM (64 channels: 4 streams x 1000 tokens of 8 heads over 2048 rows 659 us, 128 rows 702), nothing else fits (256), or
    // there are no more (few tokens); else 128 (128 channels: one stream of these 384 us, 64 rows 524)
    if (p.d > 128) return launch_chunk_fma_t<T, 256, 64>(p, stream);
    if (p.d <= 64) return launch_chunk_fma_t<T, 64, 64>(p, stream);
    return (long long)p.n * p.G <= 64 ? launch_chunk_fma_t<T, 128, 64>(p, stream) : launch_chunk_fma_t<T, 128, 128>(p, stream);
}

}  // namespace ipotk
