// Rotary positions for the rows that are not in the pot (queries, a chunk's keys) and the tables of cosines and sines
// that these kernels and the pot's own movers (k_rope.cuh) read.
//
// rope_table_kernel: entry (p, i) is the cosine (sine) of p * f_i times a magnitude.  Far positions need more than fp32: the
//   angle is taken in turns, p * (f_i / 2 pi), in 64 bits, its whole turns are dropped there (exact), and cosine and sine of
//   what is left, at most half a turn, are fp32, rounded once more where the table is bf16.  Error of the angle: 2^-52 of it (the two roundings of
//   the product) + 2^-24 of half a turn.
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

// Heads are numbered through queries and keys; a thread has up to kRowHeads of them, those of its group.
struct RowHeads {
    const char *src[kRowHeads];
    char *dst[kRowHeads];
    int n;
    __device__ __forceinline__ RowHeads(const RopeRowsParams &p, int group, int l, int b, int t, int elem)
    {
        n = 0;
        const int all = p.heads[0] + p.heads[1];
#pragma unroll
        for (int i = 0; i < kRowHeads; ++i) {
            const int h = group * kRowHeads + i;
            if (h < all) {
                const int w = h >= p.heads[0], hh = h - (w ? p.heads[0] : 0);
                const Strides &in = p.in[w], &out = p.out[w];
                src[i] = (const char *)p.src[w] + (l * in.layer + b * in.stream + hh * in.head + t * in.token) * elem;
                dst[i] = (char *)p.dst[w] + (l * out.layer + b * out.stream + hh * out.head + t * out.token) * elem;
                n = i + 1;
            }
        }
    }
};

// grid (blocks over tokens x head groups x items, streams, layers).  Items of a row: half pairing, one per vector of the lower
// half (it brings its partner); interleaved, one per rotated vector; and one per vector that is copied.
template <typename T, typename TT, bool kInterleaved>
__global__ void __launch_bounds__(kRotThreads)
rope_rows_kernel(const __grid_constant__ RopeRowsParams p, int items, int groups)
{
    pdl_wait();
    pdl_release();
    constexpr int VE = RowVec<T>::kElems;
    const unsigned at = blockIdx.x * kRotThreads + threadIdx.x;
    const unsigned per_token = (unsigned)(items * groups), t = at / per_token, rest = at - t * per_token;
    if (t >= (unsigned)p.n) return;
    const int group = rest / items, item = rest - group * items, b = blockIdx.y, l = blockIdx.z;
    const int pos = rope_position(p, b, t);
    if (pos < 0) return;
    const int rv = p.rotary / VE, half = p.rotary / 2, turned = kInterleaved ? rv : rv / 2;
    const RowHeads rows(p, group, l, b, t, sizeof(T));
    RowVec<T> x[kRowHeads], y[kRowHeads];
    if (item >= turned) {   // a vector behind the rotated part
        const int v = rv + item - turned;
#pragma unroll
        for (int i = 0; i < kRowHeads; ++i)
            if (i < rows.n) x[i] = reinterpret_cast<const RowVec<T> *>(rows.src[i])[v];
#pragma unroll
        for (int i = 0; i < kRowHeads; ++i)
            if (i < rows.n) reinterpret_cast<RowVec<T> *>(rows.dst[i])[v] = x[i];
        return;
    }
    constexpr int TE = kInterleaved ? VE / 2 : VE;   // table entries
    float cs[TE], sn[TE];
    {
        const TT *c = (const TT *)p.cos_t + (size_t)pos * half + item * TE, *s = (const TT *)p.sin_t + (size_t)pos * half + item * TE;
        struct alignas(TE * sizeof(TT) < 16 ? TE * sizeof(TT) : 16) Part {
            TT e[TE];
        };
        const Part pc = *reinterpret_cast<const Part *>(c), ps = *reinterpret_cast<const Part *>(s);
#pragma unroll
        for (int k = 0; k < TE; ++k) {
            cs[k] = to_float(pc.e[k]);
            sn[k] = to_float(ps.e[k]);
        }
    }
#pragma unroll
    for (int i = 0; i < kRowHeads; ++i)
        if (i < rows.n) {
            x[i] = reinterpret_cast<const RowVec<T> *>(rows.src[i])[item];
            if (!kInterleaved) y[i] = reinterpret_cast<const RowVec<T> *>(rows.src[i])[item + turned];
        }
#pragma unroll
    for (int i = 0; i < kRowHeads; ++i)
        if (i < rows.n) {
            float a, c;
#pragma unroll
            for (int k = 0; k < TE; ++k) {
                if (kInterleaved) {
                    rotate_pair(to_float(x[i].e[2 * k]), to_float(x[i].e[2 * k + 1]), cs[k], sn[k], a, c);
                    x[i].e[2 * k] = from_float<T>(a);
                    x[i].e[2 * k + 1] = from_float<T>(c);
                } else {
                    rotate_pair(to_float(x[i].e[k]), to_float(y[i].e[k]), cs[k], sn[k], a, c);
                    x[i].e[k] = from_float<T>(a);
                    y[i].e[k] = from_float<T>(c);
                }
            }
            reinterpret_cast<RowVec<T> *>(rows.dst[i])[item] = x[i];
            if (!kInterleaved) reinterpret_cast<RowVec<T> *>(rows.dst[i])[item + turned] = y[i];
        }
}

// Rotated parts that do not split into whole vectors: a thread has one channel pair, or one channel that is copied.
template <typename T, typename TT, bool kInterleaved>
__global__ void __launch_bounds__(kRotThreads)
rope_pairs_kernel(const __grid_constant__ RopeRowsParams p, int items, int groups)
{
    pdl_wait();
    pdl_release();
    const unsigned at = blockIdx.x * kRotThreads + threadIdx.x;
    const unsigned per_token = (unsigned)(items * groups), t = at / per_token, rest = at - t * per_token;
    if (t >= (unsigned)p.n) return;
    const int group = rest / items, item = rest - group * items, b = blockIdx.y, l = blockIdx.z;
    const int pos = rope_position(p, b, t);
    if (pos < 0) return;
    const int half = p.rotary / 2;
    const RowHeads rows(p, group, l, b, t, sizeof(T));
    if (item >= half) {
        const int c = p.rotary + item - half;
#pragma unroll
        for (int i = 0; i < kRowHeads; ++i)
            if (i < rows.n) ((T *)rows.dst[i])[c] = ((const T *)rows.src[i])[c];
        return;
    }
    const float cs = to_float(((const TT *)p.cos_t)[(size_t)pos * half + item]), sn = to_float(((const TT *)p.sin_t)[(size_t)pos * half + item]);
    const int lo = kInterleaved ? 2 * item : item, hi = kInterleaved ? lo + 1 : lo + half;
#pragma unroll
    for (int i = 0; i < kRowHeads; ++i)
        if (i < rows.n) {
            float a, c;
            rotate_pair(to_float(((const T *)rows.src[i])[lo]), to_float(((const T *)rows.src[i])[hi]), cs, sn, a, c);
            ((T *)rows.dst[i])[lo] = from_float<T>(a);
            ((T *)rows.dst[i])[hi] = from_float<T>(c);
        }
}

template <typename T, typename TT, bool kInterleaved>
inline cudaError_t launch_rope_rows_t(const RopeRowsParams &p, cudaStream_t stream)
{
    constexpr int VE = RowVec<T>::kElems;
    // whole vectors: of the rows, and (half pairing) of each half of the rotated part
    const bool vectors = p.rotary % (kInterleaved ? VE : 2 * VE) == 0;
    const int items = vectors ? p.d / VE - (kInterleaved ? 0 : p.rotary / VE / 2) : p.d - p.rotary / 2;
    const int groups = (p.heads[0] + p.heads[1] + kRowHeads - 1) / kRowHeads;
    const long long threads = (long long)p.n * items * groups;
    const dim3 grid((unsigned)((threads + kRotThreads - 1) / kRotThreads), p.streams, p.layers);
    return launch_pdl(vectors ? rope_rows_kernel<T, TT, kInterleaved> : rope_pairs_kernel<T, TT, kInterleaved>, grid, dim3(kRotThreads), 0, stream, p, items,
                      groups);
}

}  // namespace ipotk
