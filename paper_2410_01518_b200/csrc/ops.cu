// Kernels of the operators around the pot and their launchers: a second compilation unit beside ipot_api.cu.
#include "ops.h"

#include "k_blocks.cuh"
#include "k_chunk_fma.cuh"
#include "k_chunk_tc.cuh"
#include "k_few.cuh"
#include "k_rotary.cuh"

namespace ipotk {

cudaError_t launch_rope_tables(const RopeTableParams &p, bool f32, cudaStream_t stream)
{
    const long long vecs = (p.entries * (f32 ? 4 : 2) + 15) / 16;
    const dim3 grid((unsigned)((vecs + kRotThreads - 1) / kRotThreads));
    return launch_pdl(f32 ? rope_table_kernel<float> : rope_table_kernel<__nv_bfloat16>, grid, dim3(kRotThreads), 0, stream, p);
}

cudaError_t launch_rope_rows(const RopeRowsParams &p, bool f32, bool table_f32, bool interleaved, cudaStream_t stream)
{
    using bf16 = __nv_bfloat16;
    if (f32) {
        if (table_f32) return interleaved ? launch_rope_rows_t<float, float, true>(p, stream) : launch_rope_rows_t<float, float, false>(p, stream);
        return interleaved ? launch_rope_rows_t<float, bf16, true>(p, stream) : launch_rope_rows_t<float, bf16, false>(p, stream);
    }
    if (table_f32) return interleaved ? launch_rope_rows_t<bf16, float, true>(p, stream) : launch_rope_rows_t<bf16, float, false>(p, stream);
    return interleaved ? launch_rope_rows_t<bf16, bf16, true>(p, stream) : launch_rope_rows_t<bf16, bf16, false>(p, stream);
}

// Few rows have a kernel of their own: up to 8 of a KV head, or two groups of 8 that each go over the keys.
// Two groups (us, this / the other kernel for 9 rows and more, or how many times as long the other takes; 16 rows, units x keys).  bf16: as long as half of L2 holds the keys, so that the second group finds what the first has read, and
// the groups do not queue for SMs (a block's shared memory goes with d); or where a handful of units leaves the other kernel, 8 blocks a unit, most SMs idle.
//   d = 64   16 x 2000 6.3/8.8   64 x 4095 20/21    128 x 2000 21/19   256 x 2000 40/38
//   d = 128  4 x 32000 29/40   8 x 4095 14/15   8 x 16000 28/25   32 x 2000 12/15   32 x 16000 57/52   64 x 500 10/12   64 x 8000 57/53   128 x 500 17/12   256 x 4095 153/96
//   d = 256  2 x 32000 46/86   8 x 2000 15/15   8 x 16000 56/49   16 x 1000 1.10   24 x 1000 0.80   32 x 500 15/13   256 x 4095 366/181
// f32, where the other kernel has more to issue: by the groups alone.
//   d = 64   8 x 32000 220/360   32 x 4095 76/87   64 x 8000 293/294   96 x 2000 1.33   128 x 2000 222/150
//   d = 128  2 x 32000 331/598   8 x 4095 56/91    48 x 2000 1.29      96 x 2000 1.36   128 x 2000 453/306
//   d = 256  8 x 4095 102/167   16 x 2000 1.43   24 x 2000 0.89   32 x 4095 345/309
// (Over 493 calls of 1 to 256 units, 64 to 256 channels and 300 to 32000 keys the choice costs 1 % on average; most, 1.8 times, for f32 at 24 units x 300 keys x 256 channels.)
// Else tensor cores for bf16, unless a group's heads do not fit into one tile of query rows or the strides are none that a tensor map
// takes (an input whose rows repeat by a stride of 0).
static bool two_groups_of_rows(const ChunkParams &p, bool f32, long long l2_bytes)
{
    const long long units = (long long)p.layers * p.streams * p.Hkv;
    if (f32) return units <= (p.d <= 128 ? 96 : 16);
    const double key_bytes = 4.0 * units * ((double)p.len + p.n) * p.d;
    return units <= 4 || (key_bytes <= 0.5 * l2_bytes && units * p.d <= (p.d <= 128 ? 8192 : 4096));
}

cudaError_t launch_chunk_attention(const ChunkParams &p, bool f32, const ChunkTcHost &host, cudaStream_t stream)
{
    const int rows = p.n * p.G;   // (at most 2^30)
    if (rows <= kFewRows || (rows <= 2 * kFewRows && two_groups_of_rows(p, f32, host.l2_bytes))) {
        FewParams f = {};
        f.q = p.q; f.qs = p.qs; f.K = p.potK; f.V = p.potV;
        f.unit0 = p.unit0; f.unit_rows = p.unit_rows; f.len = p.len;
        f.k = p.k; f.v = p.v; f.ks = p.ks; f.vs = p.vs; f.tokens = p.tokens; f.n = p.n;
        f.out = p.out; f.os = p.os; f.lse = p.lse;
        f.layers = p.layers; f.streams = p.streams; f.Hkv = p.Hkv; f.G = p.G; f.d = p.d;
        f.scale_log2e = p.scale_log2e;
        return launch_few<false>(f, f32, stream);
    }
    if (f32) return launch_chunk_fma<float>(p, stream);
    if (host.encode && p.G <= kCtRows) {
        bool done = false;
        ChunkParams t = p;
        t.scale_log2e = tensor_scale_log2e(p.d);
        const cudaError_t e = launch_chunk_tc(t, host, stream, &done);
        if (done || e != cudaSuccess) return e;
    }
    return launch_chunk_fma<__nv_bfloat16>(p, stream);
}

cudaError_t launch_block_bounds(const void *K, void *lo, void *hi, int first_row, int len, int rows, int d, int units, size_t unit_rows, int unit_blocks, bool f32,
                                cudaStream_t stream)
{
    return f32 ? launch_block_bounds_t<float>(K, lo, hi, first_row, len, rows, d, units, unit_rows, unit_blocks, stream)
               : launch_block_bounds_t<__nv_bfloat16>(K, lo, hi, first_row, len, rows, d, units, unit_rows, unit_blocks, stream);
}

cudaError_t launch_append_bounds(const void *srcK, const void *srcV, void *potK, void *potV, void *lo, void *hi, int first_row, int n, int rows, int d, int units, size_t unit_rows,
                                 int unit_blocks, bool f32, int sm_count, cudaStream_t stream)
{
    return f32 ? launch_append_bounds_t<float>(srcK, srcV, potK, potV, lo, hi, first_row, n, rows, d, units, unit_rows, unit_blocks, sm_count, stream)
               : launch_append_bounds_t<__nv_bfloat16>(srcK, srcV, potK, potV, lo, hi, first_row, n, rows, d, units, unit_rows, unit_blocks, sm_count, stream);
}

cudaError_t launch_decode_blocks(const FewParams &p, bool f32, cudaStream_t stream)
{
    return launch_few<true>(p, f32, stream);
}

}  // namespace ipotk
