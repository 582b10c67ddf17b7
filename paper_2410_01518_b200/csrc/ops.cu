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

// Few rows have a kernel of their own: up to 8 of a KV head, or two groups of 8 that each go over the keys, as long as the second finds them in L2 (bf16, 8 heads a
// KV head of 128 channels, us, this / tcgen05: 16 rows, 8 units x 4095 keys 11.6 / 15.8, 64 units 33.5 / 35.1, 256 units 152 / 117; 8 units x 16000 25.6 / 27.0, 64 units 103 / 91).
// Else tensor cores for bf16, unless a group's heads do not fit into one tile of query rows or the strides are none that a tensor map
// takes (an input whose rows repeat by a stride of 0).
cudaError_t launch_chunk_attention(const ChunkParams &p, bool f32, const ChunkTcHost &host, cudaStream_t stream)
{
    constexpr double kStaysInL2 = 134e6;
    const int rows = p.n * p.G;   // (at most 2^30)
    const double key_bytes = 2.0 * p.layers * p.streams * p.Hkv * ((double)p.len + p.n) * p.d * (f32 ? 4 : 2);
    if (rows <= kFewRows || (rows <= 2 * kFewRows && key_bytes <= kStaysInL2)) {
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
