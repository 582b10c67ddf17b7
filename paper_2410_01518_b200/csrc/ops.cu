// Kernels of the operators around the pot and their launchers: a second compilation unit beside ipot_api.cu.
#include "ops.h"

#include "k_chunk_fma.cuh"
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

cudaError_t launch_chunk_attention(const ChunkParams &p, bool f32, cudaStream_t stream)
{
    return f32 ? launch_chunk_fma<float>(p, stream) : launch_chunk_fma<__nv_bfloat16>(p, stream);
}

}  // namespace ipotk
