// Attention of a chunk of new tokens over the pot and, causally, over itself, with fp32 FMAs: every type, head dimension and
// group size.  out_h[t] = sum_j softmax_j(q_h[t] . k_j / sqrt(d)) v_j over the pot's rows [0, len) and the chunk's rows 0 .. t.
//
// The query heads of a KV head share its keys, so a unit's rows are folded token by token: row t * G + g.  A block has BM of
// them and goes over the keys they see in tiles of 64, with the running maximum and sum of the softmax: products S = Q K^T from
// transposed tiles in shared memory (a thread has BM / 16 rows x 4 keys), probabilities back into shared memory, O += P V with BM / 16 rows
// x d / 16 channels in a thread's registers.  Everything is fp32.  Bound: FMA issue and shared-memory reads (4 x 4 products
// per two 16-byte reads).
#pragma once
#include "common.cuh"
#include "ops.h"
#include "k_rotary.cuh"   // RowVec, to_float, from_float

namespace ipotk {

constexpr int kCfThreads = 256;
constexpr int kCfKeys = 64;

template <int DP, int BM> struct ChunkFmaSmem {
    static constexpr int kKeyPitch = kCfKeys + 4;   // (the transposing stores of a warp then fall into different banks)
    static constexpr int kRowPitch = BM + 4;
    float q[DP][kRowPitch];
    float k[DP][kKeyPitch];
    float v[kCfKeys][DP];
    float p[kCfKeys][kRowPitch];
};

__device__ __forceinline__ float chunk_ex2(float x)
{
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

// Tokens of stream b that are there.
__device__ __forceinline__ int chunk_tokens(const ChunkParams &p, int b) { return p.tokens ? min(max(__ldg(p.tokens + b), 0), p.n) : p.n; }

template <typename T, int DP, int BM>
__global__ void __launch_bounds__(kCfThreads)
chunk_fma_kernel(const __grid_constant__ ChunkParams p)
{
    pdl_wait();
    pdl_release();
    using Smem = ChunkFmaSmem<DP, BM>;
    constexpr int VE = RowVec<T>::kElems, RT = BM / 16, CV = DP / 64;   // rows and 4-channel vectors of a thread
    extern __shared__ __align__(16) uint8_t chunk_raw[];
    Smem &sm = *reinterpret_cast<Smem *>(chunk_raw);
    const int unit = blockIdx.y, hkv = unit % p.Hkv, b = unit / p.Hkv % p.streams, l = unit / p.Hkv / p.streams;
    const int n = chunk_tokens(p, b), G = p.G, row0 = ((int)gridDim.x - 1 - (int)blockIdx.x) * BM;   // the longest rows first
    if (row0 >= n * G) return;
    const int rows = min(BM, n * G - row0), keys = p.len + (row0 + rows - 1) / G + 1;
    const int tid = threadIdx.x, ty = tid >> 4, tx = tid & 15, vecs = p.d / VE;
    const T *potK = (const T *)p.potK + (size_t)(p.unit0 + unit) * p.unit_rows * p.d, *potV = (const T *)p.potV + (size_t)(p.unit0 + unit) * p.unit_rows * p.d;
    const T *newK = (const T *)p.k + l * p.ks.layer + b * p.ks.stream + hkv * p.ks.head, *newV = (const T *)p.v + l * p.vs.layer + b * p.vs.stream + hkv * p.vs.head;
    const T *q = (const T *)p.q + l * p.qs.layer + b * p.qs.stream + (long long)hkv * G * p.qs.head;

    if (DP > p.d) {   // channels that are not there count as zeros
        for (int i = tid; i < (DP - p.d) * Smem::kRowPitch; i += kCfThreads) sm.q[p.d][i] = 0.f;
        for (int i = tid; i < (DP - p.d) * Smem::kKeyPitch; i += kCfThreads) sm.k[p.d][i] = 0.f;
        for (int i = tid; i < kCfKeys * (DP - p.d); i += kCfThreads) sm.v[i / (DP - p.d)][p.d + i % (DP - p.d)] = 0.f;
    }
    for (int i = tid; i < BM * vecs; i += kCfThreads) {
        const int r = i % BM, v = i / BM, t = (row0 + r) / G, g = row0 + r - t * G;
        RowVec<T> x;
        if (r < rows) x = *reinterpret_cast<const RowVec<T> *>(q + (long long)t * p.qs.token + g * p.qs.head + v * VE);
#pragma unroll
        for (int e = 0; e < VE; ++e) sm.q[v * VE + e][r] = r < rows ? to_float(x.e[e]) * p.scale_log2e : 0.f;
    }
    float m[RT], sum[RT], acc[RT][CV][4];
    int limit[RT];
#pragma unroll
    for (int i = 0; i < RT; ++i) {
        m[i] = -INFINITY;
        sum[i] = 0.f;
        limit[i] = p.len + (row0 + ty * RT + i) / G + 1;
#pragma unroll
        for (int c = 0; c < CV; ++c) acc[i][c][0] = acc[i][c][1] = acc[i][c][2] = acc[i][c][3] = 0.f;
    }
    for (int k0 = 0; k0 < keys; k0 += kCfKeys) {
        __syncthreads();
        for (int i = tid; i < kCfKeys * vecs; i += kCfThreads) {
            const int r = i % kCfKeys, v = i / kCfKeys, j = k0 + r;
            RowVec<T> x;
            if (j < keys) x = *reinterpret_cast<const RowVec<T> *>((j < p.len ? potK + (size_t)j * p.d : newK + (j - p.len) * p.ks.token) + v * VE);
#pragma unroll
            for (int e = 0; e < VE; ++e) sm.k[v * VE + e][r] = j < keys ? to_float(x.e[e]) : 0.f;
        }
        for (int i = tid; i < kCfKeys * vecs; i += kCfThreads) {
            const int r = i / vecs, v = i - r * vecs, j = k0 + r;
            RowVec<T> x;
            if (j < keys) x = *reinterpret_cast<const RowVec<T> *>((j < p.len ? potV + (size_t)j * p.d : newV + (j - p.len) * p.vs.token) + v * VE);
#pragma unroll
            for (int e = 0; e < VE; ++e) sm.v[r][v * VE + e] = j < keys ? to_float(x.e[e]) : 0.f;
        }
        __syncthreads();
        float s[RT][4];
#pragma unroll
        for (int i = 0; i < RT; ++i) s[i][0] = s[i][1] = s[i][2] = s[i][3] = 0.f;
#pragma unroll 4
        for (int c = 0; c < DP; ++c) {
            float a[RT];
            if (RT == 4) *reinterpret_cast<float4 *>(a) = *reinterpret_cast<const float4 *>(&sm.q[c][ty * RT]);
            else a[0] = sm.q[c][ty];
            const float4 k4 = *reinterpret_cast<const float4 *>(&sm.k[c][tx * 4]);
#pragma unroll
            for (int i = 0; i < RT; ++i) {
                s[i][0] = fmaf(a[i], k4.x, s[i][0]);
                s[i][1] = fmaf(a[i], k4.y, s[i][1]);
                s[i][2] = fmaf(a[i], k4.z, s[i][2]);
                s[i][3] = fmaf(a[i], k4.w, s[i][3]);
            }
        }
#pragma unroll
        for (int i = 0; i < RT; ++i) {
            float mt = -INFINITY;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                if (k0 + tx * 4 + j >= limit[i]) s[i][j] = -INFINITY;
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
                sm.p[tx * 4 + j][ty * RT + i] = s[i][j];
            }
            m[i] = mn;
            sum[i] = sum[i] * corr + ps;   // this thread's share
#pragma unroll
            for (int c = 0; c < CV; ++c)
#pragma unroll
                for (int e = 0; e < 4; ++e) acc[i][c][e] *= corr;
        }
        __syncthreads();
        const int here = min(kCfKeys, keys - k0);
#pragma unroll 4
        for (int j = 0; j < here; ++j) {
            float a[RT];
            if (RT == 4) *reinterpret_cast<float4 *>(a) = *reinterpret_cast<const float4 *>(&sm.p[j][ty * RT]);
            else a[0] = sm.p[j][ty];
#pragma unroll
            for (int c = 0; c < CV; ++c) {
                const float4 v4 = *reinterpret_cast<const float4 *>(&sm.v[j][c * 64 + tx * 4]);
#pragma unroll
                for (int i = 0; i < RT; ++i) {
                    acc[i][c][0] = fmaf(a[i], v4.x, acc[i][c][0]);
                    acc[i][c][1] = fmaf(a[i], v4.y, acc[i][c][1]);
                    acc[i][c][2] = fmaf(a[i], v4.z, acc[i][c][2]);
                    acc[i][c][3] = fmaf(a[i], v4.w, acc[i][c][3]);
                }
            }
        }
    }
#pragma unroll
    for (int i = 0; i < RT; ++i) {
#pragma unroll
        for (int off = 8; off >= 1; off >>= 1) sum[i] += __shfl_xor_sync(0xffffffffu, sum[i], off);
        const int r = ty * RT + i, t = (row0 + r) / G, g = row0 + r - t * G;
        if (r >= rows) continue;
        T *o = (T *)p.out + l * p.os.layer + b * p.os.stream + (long long)(hkv * G + g) * p.os.head + (long long)t * p.os.token;
        const float inv = 1.f / sum[i];
#pragma unroll
        for (int c = 0; c < CV; ++c)
#pragma unroll
            for (int e = 0; e < 4; ++e)
                if (c * 64 + tx * 4 + e < p.d) o[c * 64 + tx * 4 + e] = from_float<T>(acc[i][c][e] * inv);
        if (tx == 0 && p.lse) p.lse[(((size_t)l * p.streams + b) * p.Hkv * G + hkv * G + g) * p.n + t] = 0.6931471805599453f * (m[i] + log2f(sum[i]));
    }
}

template <typename T, int DP, int BM>
inline cudaError_t launch_chunk_fma_t(const ChunkParams &p, cudaStream_t stream)
{
    const size_t smem = sizeof(ChunkFmaSmem<DP, BM>);
    auto kern = chunk_fma_kernel<T, DP, BM>;
    const cudaError_t e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
    if (e != cudaSuccess) return e;
    const int units = p.layers * p.streams * p.Hkv;
    return launch_pdl(kern, dim3((unsigned)(((long long)p.n * p.G + BM - 1) / BM), units), dim3(kCfThreads), smem, stream, p);
}

template <typename T>
inline cudaError_t launch_chunk_fma(const ChunkParams &p, cudaStream_t stream)
{
    if ((long long)p.n * p.G <= 16)
        return p.d <= 64 ? launch_chunk_fma_t<T, 64, 16>(p, stream) : p.d <= 128 ? launch_chunk_fma_t<T, 128, 16>(p, stream) : launch_chunk_fma_t<T, 256, 16>(p, stream);
    return p.d <= 64 ? launch_chunk_fma_t<T, 64, 64>(p, stream) : p.d <= 128 ? launch_chunk_fma_t<T, 128, 64>(p, stream) : launch_chunk_fma_t<T, 256, 64>(p, stream);
}

}  // namespace ipotk
