// Generation over selected blocks of the pot: the bounds that the selection goes by (k_few.cuh has the rest).  Slots are taken in blocks
// of R; the smallest and largest value of every channel over a block's keys bound every logit in it:
// q . k_j <= sum_c max(q_c lo_c, q_c hi_c) for all j of the block.
//
// block_bounds_kernel: those bounds, for the blocks whose rows have changed.  Bound: HBM, every changed key once.
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

}  // namespace ipotk
