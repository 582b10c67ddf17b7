// Generation over selected blocks of the pot: the bounds that the selection goes by (k_few.cuh has the rest).  Slots are taken in blocks
// of R; the smallest and largest value of every channel over a block's keys bound every logit in it:
// q . k_j <= sum_c max(q_c lo_c, q_c hi_c) for all j of the block.
//
// append_bounds_kernel: an append that keeps them; block_bounds_kernel: those of blocks whose rows something else has written (a cycle's gather, the rotated
// copy, a host copy).  Bound: HBM, every changed key once.
#pragma once
#include "common.cuh"
#include "ops.h"
#include "k_rotary.cuh"   // RowVec, to_float

namespace ipotk {

// ------------------------------------------------------------------ bounds
constexpr int kBoundThreads = 128;

// lo <- min(lo, x), hi <- max(hi, x), channel by channel
__device__ __forceinline__ void widen(RowVec<float> &lo, RowVec<float> &hi, const RowVec<float> &x, const RowVec<float> &y)
{
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        lo.e[e] = fminf(lo.e[e], x.e[e]);
        hi.e[e] = fmaxf(hi.e[e], y.e[e]);
    }
}
__device__ __forceinline__ void widen(RowVec<__nv_bfloat16> &lo, RowVec<__nv_bfloat16> &hi, const RowVec<__nv_bfloat16> &x, const RowVec<__nv_bfloat16> &y)
{
    __nv_bfloat162 *a = reinterpret_cast<__nv_bfloat162 *>(lo.e), *b = reinterpret_cast<__nv_bfloat162 *>(hi.e);
    const __nv_bfloat162 *c = reinterpret_cast<const __nv_bfloat162 *>(x.e), *d = reinterpret_cast<const __nv_bfloat162 *>(y.e);
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        a[e] = __hmin2(a[e], c[e]);
        b[e] = __hmax2(b[e], d[e]);
    }
}

// A thread has vector v of every `side`-th row.  Joins what the rows' threads have seen; the result is with the threads of row 0.
template <typename T>
__device__ __forceinline__ void join_bounds(RowVec<T> &a, RowVec<T> &b, RowVec<T> (*part)[kBoundThreads], int side, int vecs, int r0, int v)
{
    part[0][threadIdx.x] = a;
    part[1][threadIdx.x] = b;
    __syncthreads();
    if (r0 == 0)
        for (int r = 1; r < side; ++r) widen(a, b, part[0][r * vecs + v], part[1][r * vecs + v]);
}

// grid (blocks from first_block on, units).  Threads: a vector of the row each, several rows side by side.
template <typename T>
__global__ void __launch_bounds__(kBoundThreads)
block_bounds_kernel(const T *__restrict__ K, T *__restrict__ lo, T *__restrict__ hi, int first_block, int rows_per_block, int len, int d, size_t unit_rows, int unit_blocks)
{
    pdl_wait();
    pdl_release();
    __shared__ RowVec<T> part[2][kBoundThreads];
    const int vecs = d / RowVec<T>::kElems, r0 = threadIdx.x / vecs, v = threadIdx.x - r0 * vecs;
    const int block = first_block + blockIdx.x, n = min(rows_per_block, len - block * rows_per_block), side = min(kBoundThreads / vecs, n);
    const RowVec<T> *src = reinterpret_cast<const RowVec<T> *>(K + ((size_t)blockIdx.y * unit_rows + (size_t)block * rows_per_block) * d);
    RowVec<T> a, b;
    if (r0 < side) {
        a = b = src[(size_t)r0 * vecs + v];
        int r = r0 + side;
        for (; r + 3 * side < n; r += 4 * side) {
            RowVec<T> x[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) x[i] = src[(size_t)(r + i * side) * vecs + v];
#pragma unroll
            for (int i = 0; i < 4; ++i) widen(a, b, x[i], x[i]);
        }
        for (; r < n; r += side) {
            const RowVec<T> x = src[(size_t)r * vecs + v];
            widen(a, b, x, x);
        }
    }
    join_bounds(a, b, part, side, vecs, r0, v);
    if (r0 == 0) {
        const size_t at = ((size_t)blockIdx.y * unit_blocks + block) * vecs + v;
        reinterpret_cast<RowVec<T> *>(lo)[at] = a;
        reinterpret_cast<RowVec<T> *>(hi)[at] = b;
    }
}

// An append that takes the bounds along: a thread block copies a block's new rows, keys and values, and bounds them by the keys on their way through, and with them the rows that were
// there.  (Those are read again: their bounds may be those of an earlier replay of the same call, over rows that this one replaces.)  grid (blocks that rows [first_row, first_row + n) touch, units); srcK, srcV [units][n][d].  Bound: HBM, the copy.
// kEarly as in append_kernel.
template <typename T, bool kEarly>
__global__ void __launch_bounds__(kBoundThreads)
append_bounds_kernel(const T *__restrict__ srcK, const T *__restrict__ srcV, T *__restrict__ potK, T *__restrict__ potV, T *__restrict__ lo, T *__restrict__ hi,
                     int rows_per_block, int first_row, int n, int d, size_t unit_rows, int unit_blocks)
{
    if (kEarly) {
        pdl_wait();
        pdl_release();
    }
    using Vec = RowVec<T>;
    __shared__ Vec part[2][kBoundThreads];
    const int vecs = d / Vec::kElems, r0 = threadIdx.x / vecs, v = threadIdx.x - r0 * vecs;
    const int block = first_row / rows_per_block + blockIdx.x, from = max(first_row, block * rows_per_block), to = min(first_row + n, (block + 1) * rows_per_block);
    const int rows = to - from, old = from - block * rows_per_block, side = min(kBoundThreads / vecs, max(rows, old));
    const size_t s = ((size_t)blockIdx.y * n + from - first_row) * vecs, t = ((size_t)blockIdx.y * unit_rows + from) * vecs;
    const Vec *sk = reinterpret_cast<const Vec *>(srcK) + s, *sv = reinterpret_cast<const Vec *>(srcV) + s;
    Vec *tk = reinterpret_cast<Vec *>(potK) + t, *tv = reinterpret_cast<Vec *>(potV) + t;
    Vec a, b;
    if (r0 < side) {
        constexpr int RB = 4;   // rows of keys, and of values, on their way at once
        for (int r = r0; r < rows; r += RB * side) {
            Vec x[RB], y[RB];
#pragma unroll
            for (int i = 0; i < RB; ++i)
                if (r + i * side < rows) {
                    x[i] = sk[(size_t)(r + i * side) * vecs + v];
                    y[i] = sv[(size_t)(r + i * side) * vecs + v];
                }
            if (r == r0) a = b = x[0];
#pragma unroll
            for (int i = 0; i < RB; ++i)
                if (r + i * side < rows) {
                    tk[(size_t)(r + i * side) * vecs + v] = x[i];
                    tv[(size_t)(r + i * side) * vecs + v] = y[i];
                    widen(a, b, x[i], x[i]);
                }
        }
        const Vec *there = tk - (size_t)old * vecs;
        for (int r = r0; r < old; r += RB * side) {
            Vec x[RB];
#pragma unroll
            for (int i = 0; i < RB; ++i) x[i] = there[(size_t)min(r + i * side, old - 1) * vecs + v];   // (the last row again: it changes no bound)
            if (r == r0 && r0 >= rows) a = b = x[0];
#pragma unroll
            for (int i = 0; i < RB; ++i) widen(a, b, x[i], x[i]);
        }
    }
    join_bounds(a, b, part, side, vecs, r0, v);
    if (r0 == 0) {
        const size_t at = ((size_t)blockIdx.y * unit_blocks + block) * vecs + v;
        reinterpret_cast<Vec *>(lo)[at] = a;
        reinterpret_cast<Vec *>(hi)[at] = b;
    }
}

template <typename T>
inline cudaError_t launch_block_bounds_t(const void *K, void *lo, void *hi, int first_row, int len, int rows, int d, int units, size_t unit_rows, int unit_blocks, cudaStream_t stream)
{
    const int first = first_row / rows;
    const dim3 grid((len + rows - 1) / rows - first, units);
    return launch_pdl(block_bounds_kernel<T>, grid, dim3(kBoundThreads), 0, stream, (const T *)K, (T *)lo, (T *)hi, first, rows, len, d, unit_rows, unit_blocks);
}

template <typename T>
inline cudaError_t launch_append_bounds_t(const void *srcK, const void *srcV, void *potK, void *potV, void *lo, void *hi, int first_row, int n, int rows, int d, int units, size_t unit_rows,
                                          int unit_blocks, int sm_count, cudaStream_t stream)
{
    const dim3 grid((first_row + n + rows - 1) / rows - first_row / rows, units);
    if ((long long)grid.x * units <= 8LL * sm_count)
        return launch_pdl(append_bounds_kernel<T, true>, grid, dim3(kBoundThreads), 0, stream, (const T *)srcK, (const T *)srcV, (T *)potK, (T *)potV, (T *)lo, (T *)hi, rows, first_row, n, d,
                          unit_rows, unit_blocks);
    append_bounds_kernel<T, false><<<grid, kBoundThreads, 0, stream>>>((const T *)srcK, (const T *)srcV, (T *)potK, (T *)potV, (T *)lo, (T *)hi, rows, first_row, n, d, unit_rows, unit_blocks);
    return cudaGetLastError();
}

}  // namespace ipotk
