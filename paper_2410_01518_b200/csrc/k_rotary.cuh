// Rotary positions for the rows that are not in the pot (queries, a chunk's keys) and the tables of cosines and sines
// that these kernels and the pot's own movers (k_rope.cuh) read.
//
// rope_table_kernel: entry (p, i) is the cosine (sine) of p * f_i times a magnitude.  Far positions need more than fp32: the
//   angle is taken in turns, p * (f_i / 2 pi), in 64 bits, its whole turns are dropped there (exact), and cosine and sine of
//   what is left, at most half a turn, are fp32, rounded once more where the table is bf16.  Error of the angle: up to
//   (ln b + 8) 2^-53 of it, b the base - the exponent of b is rounded, and so are the power, the stretched base or the blend, 2 pi, the quotient and the product - + 2^-24 of half a turn.
// rope_rows_kernel: lo' = fma(lo, cos, -(hi * sin)), hi' = fma(hi, cos, lo * sin), as the movers have it, in fp32, rounded once to the
//   rows' type; channels behind the rotated part are copied.  A thread has one 16-byte vector (half pairing: a vector and its
//   partners) of kRowHeads heads of a token: the table's vectors are loaded once for them.  Bound: HBM, every row in and out.
#pragma once
#include "common.cuh"
#include "ops.h"

namespace ipotk {

constexpr int kRotThreads = 128;

template <typename T> __device__ __forceinline__ T from_float(float x);
template <> __device__ __forceinline__ float from_float<float>(float x) { return x; }
template <> __device__ __forceinline__ __nv_bfloat16 from_float<__nv_bfloat16>(float x) { return __float2bfloat16_rn(x); }
__device__ __forceinline__ float to_float(float x) { return x; }
__device__ __forceinline__ float to_float(__nv_bfloat16 x) { return __bfloat162float(x); }

template <typename T> struct alignas(16) RowVec {
    static constexpr int kElems = 16 / sizeof(T);
    T e[kElems];
};

// A thread: one vector of 16 bytes of the flat [positions][half] arrays.
template <typename T>
__global__ void __launch_bounds__(kRotThreads)
rope_table_kernel(const __grid_constant__ RopeTableParams p)
{
    constexpr int VE = RowVec<T>::kElems;
    __shared__ double turns[kRopeMaxPairs];
    for (int i = threadIdx.x; i < p.half; i += kRotThreads) turns[i] = p.turns[i];
    __syncthreads();
    pdl_wait();
    pdl_release();
    const long long e0 = ((long long)blockIdx.x * kRotThreads + threadIdx.x) * VE;
    if (e0 >= p.entries) return;
    long long row = e0 / p.half;
    int i = (int)(e0 - row * p.half);
    RowVec<T> c, s;
#pragma unroll
    for (int k = 0; k < VE; ++k) {
        const double a = (double)(p.first + row) * turns[i];
        float sn, cs;
        sincospif(2.f * (float)(a - rint(a)), &sn, &cs);
        c.e[k] = from_float<T>(cs * p.magnitude);
        s.e[k] = from_float<T>(sn * p.magnitude);
        if (++i == p.half) {
            i = 0;
            ++row;
        }
    }
    T *co = (T *)p.cos_t + e0, *so = (T *)p.sin_t + e0;
    if (e0 + VE <= p.entries) {
        *reinterpret_cast<RowVec<T> *>(co) = c;
        *reinterpret_cast<RowVec<T> *>(so) = s;
    } else {
#pragma unroll
        for (int k = 0; k < VE; ++k)
            if (e0 + k < p.entries) {
                co[k] = c.e[k];
                so[k] = s.e[k];
            }
    }
}

// The position of token t of stream b; negative: its rows are left alone.
__device__ __forceinline__ int rope_position(const RopeRowsParams &p, int b, int t)
{
    int pos = p.positions ? __ldg(p.positions + (size_t)b * p.n + t) : p.first + t;
    if (pos >= p.table_rows) {
        set_status(p.status, kStatusBounds);
        pos = -1;
    }
    return pos;
}

__device__ __forceinline__ void rotate_pair(float lo, float hi, float cs, float sn, float &lo_out, float &hi_out)
{
    lo_out = __fmaf_rn(lo, cs, -__fmul_rn(hi, sn));
    hi_out = __fmaf_rn(hi, cs, __fmul_rn(lo, sn));
}

constexpr int kRowHeads = 4;   // of a thread

// What a thread block has: a layer, a stream and up to kRowHeads neighbouring heads of the queries or of the keys; a thread has a token of
// them (everything but the token is the block's, so addresses cost a thread one multiplication each).
struct RowHeads {
    const char *src;
    char *dst;
    long long in_head, out_head, in_token, out_token;   // bytes
    int b, n;
    __device__ __forceinline__ RowHeads(const RopeRowsParams &p, int elem)
    {
        const int q_groups = (p.heads[0] + kRowHeads - 1) / kRowHeads, group = blockIdx.y, w = group >= q_groups, h = (group - (w ? q_groups : 0)) * kRowHeads, l = blockIdx.z / p.streams;
        b = blockIdx.z - l * p.streams;
        const Strides &in = p.in[w], &out = p.out[w];
        src = (const char *)p.src[w] + (l * in.layer + b * in.stream + h * in.head) * elem;
        dst = (char *)p.dst[w] + (l * out.layer + b * out.stream + h * out.head) * elem;
        in_head = in.head * elem;
        out_head = out.head * elem;
        in_token = in.token * elem;
        out_token = out.token * elem;
        n = min(kRowHeads, p.heads[w] - h);
    }
};

// grid (blocks over tokens x items, head groups, layers x streams).  Items of a row: half pairing, one per vector of the lower
// half (it brings its partner); interleaved, one per rotated vector; and one per vector, or two vectors, that are copied.  Both kinds load before
// and store behind the rotation: a warp has items of both.  16 streams x 2048 tokens x 40 heads x 128 channels (671 MB): 98.8 us, 6.8 TB/s, all or half of them rotated; streams of
// different lengths, half as many rows, 58.5 us, 6.1 TB/s.  (Stored as a struct of elements: 138 us.  Stores that are evicted first: no gain out of place, 84 MB in place 20 -> 24 us.)
template <typename T, typename TT, bool kInterleaved>
__global__ void __launch_bounds__(kRotThreads)
rope_rows_kernel(const __grid_constant__ RopeRowsParams p, int items)
{
    pdl_wait();
    pdl_release();
    constexpr int VE = RowVec<T>::kElems;
    const unsigned at = blockIdx.x * kRotThreads + threadIdx.x, t = at / (unsigned)items;
    if (t >= (unsigned)p.n) return;
    const int item = at - t * items;
    const RowHeads rows(p, sizeof(T));
    const int pos = rope_position(p, rows.b, t);
    if (pos < 0) return;
    const char *src = rows.src + t * rows.in_token;
    char *dst = rows.dst + t * rows.out_token;
    // its vector, and (half pairing) a second one: the partner, or where vectors are copied one more of them
    const int rv = p.rotary / VE, half = p.rotary / 2, turned = kInterleaved ? rv : rv / 2, vecs = p.d / VE;
    const bool turns = item < turned;
    const int v = turns ? item : rv + item - turned, v2 = turns ? item + turned : v + (vecs - rv + 1) / 2;
    const bool two = !kInterleaved && v2 < vecs;
    RowVec<T> x[kRowHeads], y[kRowHeads];
#pragma unroll
    for (int i = 0; i < kRowHeads; ++i)
        if (i < rows.n) {
            x[i] = reinterpret_cast<const RowVec<T> *>(src + i * rows.in_head)[v];
            if (two) y[i] = reinterpret_cast<const RowVec<T> *>(src + i * rows.in_head)[v2];
        }
    if (turns) {
        constexpr int TE = kInterleaved ? VE / 2 : VE;   // table entries
        struct alignas(TE * sizeof(TT) < 16 ? TE * sizeof(TT) : 16) Part {
            TT e[TE];
        };
        const Part pc = *reinterpret_cast<const Part *>((const TT *)p.cos_t + (size_t)pos * half + item * TE);
        const Part ps = *reinterpret_cast<const Part *>((const TT *)p.sin_t + (size_t)pos * half + item * TE);
#pragma unroll
        for (int k = 0; k < TE; ++k) {
            const float cs = to_float(pc.e[k]), sn = to_float(ps.e[k]);
            float a, c;
#pragma unroll
            for (int i = 0; i < kRowHeads; ++i) {
                T &lo = kInterleaved ? x[i].e[2 * k] : x[i].e[k], &hi = kInterleaved ? x[i].e[2 * k + 1] : y[i].e[k];
                rotate_pair(to_float(lo), to_float(hi), cs, sn, a, c);
                lo = from_float<T>(a);
                hi = from_float<T>(c);
            }
        }
    }
#pragma unroll
    for (int i = 0; i < kRowHeads; ++i)
        if (i < rows.n) reinterpret_cast<uint4 *>(dst + i * rows.out_head)[v] = *reinterpret_cast<const uint4 *>(x + i);
    if (two) {
#pragma unroll
        for (int i = 0; i < kRowHeads; ++i)
            if (i < rows.n) reinterpret_cast<uint4 *>(dst + i * rows.out_head)[v2] = *reinterpret_cast<const uint4 *>(y + i);
    }
}

// Rotated parts that do not split into whole vectors: a thread has one channel pair, or one channel that is copied.  Bound: 2-byte accesses (122 of 128 channels in the case above 295 us, 26 of
// them 423).
template <typename T, typename TT, bool kInterleaved>
__global__ void __launch_bounds__(kRotThreads)
rope_pairs_kernel(const __grid_constant__ RopeRowsParams p, int items)
{
    pdl_wait();
    pdl_release();
    const unsigned at = blockIdx.x * kRotThreads + threadIdx.x, t = at / (unsigned)items;
    if (t >= (unsigned)p.n) return;
    const int item = at - t * items;
    const RowHeads rows(p, sizeof(T));
    const int pos = rope_position(p, rows.b, t);
    if (pos < 0) return;
    const char *src = rows.src + t * rows.in_token;
    char *dst = rows.dst + t * rows.out_token;
    const int half = p.rotary / 2;
    if (item >= half) {
        const int c = p.rotary + item - half;
#pragma unroll
        for (int i = 0; i < kRowHeads; ++i)
            if (i < rows.n) ((T *)(dst + i * rows.out_head))[c] = ((const T *)(src + i * rows.in_head))[c];
        return;
    }
    const float cs = to_float(((const TT *)p.cos_t)[(size_t)pos * half + item]), sn = to_float(((const TT *)p.sin_t)[(size_t)pos * half + item]);
    const int lo = kInterleaved ? 2 * item : item, hi = kInterleaved ? lo + 1 : lo + half;
#pragma unroll
    for (int i = 0; i < kRowHeads; ++i)
        if (i < rows.n) {
            float a, c;
            rotate_pair(to_float(((const T *)(src + i * rows.in_head))[lo]), to_float(((const T *)(src + i * rows.in_head))[hi]), cs, sn, a, c);
            ((T *)(dst + i * rows.out_head))[lo] = from_float<T>(a);
            ((T *)(dst + i * rows.out_head))[hi] = from_float<T>(c);
        }
}

template <typename T, typename TT, bool kInterleaved>
inline cudaError_t launch_rope_rows_t(const RopeRowsParams &p, cudaStream_t stream)
{
    constexpr int VE = RowVec<T>::kElems;
    // whole vectors: of the rows, and (half pairing) of each half of the rotated part
    const bool vectors = p.rotary % (kInterleaved ? VE : 2 * VE) == 0;
    const int rest = p.d / VE - p.rotary / VE;   // vectors that are copied
    const int items = vectors ? (kInterleaved ? p.d / VE : p.rotary / VE / 2 + (rest + 1) / 2) : p.d - p.rotary / 2;
    const int groups = (p.heads[0] + kRowHeads - 1) / kRowHeads + (p.heads[1] + kRowHeads - 1) / kRowHeads;
    const long long threads = (long long)p.n * items;
    const dim3 grid((unsigned)((threads + kRotThreads - 1) / kRotThreads), groups, p.layers * p.streams);
    return launch_pdl(vectors ? rope_rows_kernel<T, TT, kInterleaved> : rope_pairs_kernel<T, TT, kInterleaved>, grid, dim3(kRotThreads), 0, stream, p, items);
}

}  // namespace ipotk
