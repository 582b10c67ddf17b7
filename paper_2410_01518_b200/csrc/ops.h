// Host launchers of the operators around the pot (ops.cu): plain parameters, no pot object.  Arguments have been checked.
#pragma once
#include <cuda_runtime.h>
#include <stddef.h>
#include <stdint.h>

namespace ipotk {

// Elements between neighbours of a [layer][stream][head][token][d] array; the channels of a row are contiguous.
struct Strides {
    long long layer, stream, head, token;
};

// ------------------------------------------------------------------ rotary positions (k_rotary.cuh)
constexpr int kRopeMaxPairs = 128;
struct RopeTableParams {
    double turns[kRopeMaxPairs];   // of a channel pair per position, in whole turns
    float magnitude;
    int half;                      // pairs
    long long first;
    long long entries;             // positions * half
    void *cos_t, *sin_t;
};
cudaError_t launch_rope_tables(const RopeTableParams &p, bool f32, cudaStream_t stream);

struct RopeRowsParams {
    const void *src[2];            // queries, keys; NULL: none of them
    void *dst[2];
    Strides in[2], out[2];
    int heads[2];
    const void *cos_t, *sin_t;
    const int32_t *positions;      // [streams][n], or NULL: first + token
    int first, table_rows, rotary, d, n, streams, layers;
    int *status;
};
// interleaved: pairs (2c, 2c + 1), else (c, c + rotary / 2)
cudaError_t launch_rope_rows(const RopeRowsParams &p, bool f32, bool table_f32, bool interleaved, cudaStream_t stream);

// ------------------------------------------------------------------ a chunk's attention over pot and chunk (k_chunk_*.cuh)
struct ChunkParams {
    const void *q, *k, *v;         // of the layers asked for
    void *out;
    float *lse;                    // [layers][streams][heads][n], or NULL
    Strides qs, ks, vs, os;
    const int32_t *tokens;         // [streams], or NULL: all n
    const void *potK, *potV;       // [units][unit_rows][d], from the pot's first unit on
    int unit0;                     // the first unit asked for
    int unit_rows, len;
    int layers, streams, Hkv, G, d, n;
    float scale_log2e;
    int *status;
};
// What the choice of a kernel and the tensor-core kernel need besides.
struct ChunkTcHost {
    void *encode;                  // cuTensorMapEncodeTiled, or NULL: no tensor-core kernel
    int sm_count, l2_bytes, pot_units;
    int withhold;                  // -1; test hook: this stream's softmax never reports
    unsigned long long wait_ns;
};
struct ChunkTcParams {
    ChunkParams c;
    int tile_tokens, items_per_unit;
    int withhold;
    unsigned long long wait_ns;
    int *status;
};
cudaError_t launch_chunk_attention(const ChunkParams &p, bool f32, const ChunkTcHost &host, cudaStream_t stream);

// ------------------------------------------------------------------ few query rows, generation over selected blocks (k_few.cuh, k_blocks.cuh)
struct FewParams {
    const void *q;                 // of the layers asked for
    Strides qs;
    const void *K, *V;             // [units][unit_rows][d], from the pot's first unit on
    int unit0, unit_rows, len;
    // a chunk of few tokens (1 token and none of these over selected blocks)
    const void *k, *v;
    Strides ks, vs;
    const int32_t *tokens;
    int n;
    // selected blocks
    const void *lo, *hi;           // [units][unit_blocks][d]
    int32_t *list;                 // [layers][streams][Hkv][blocks], or NULL
    int unit_blocks, block_rows, blocks;
    void *out;
    Strides os;
    float *lse;                    // [layers][streams][heads][n], or NULL
    int layers, streams, Hkv, G, d;
    float scale_log2e;
};
cudaError_t launch_decode_blocks(const FewParams &p, bool f32, cudaStream_t stream);
// bounds of the blocks that hold rows [first_row, len) of every unit
cudaError_t launch_block_bounds(const void *K, void *lo, void *hi, int first_row, int len, int rows, int d, int units, size_t unit_rows, int unit_blocks, bool f32,
                                cudaStream_t stream);

// an append of n rows of keys and values [units][n][d] behind first_row, bounds included
cudaError_t launch_append_bounds(const void *srcK, const void *srcV, void *potK, void *potV, void *lo, void *hi, int first_row, int n, int rows, int d, int units, size_t unit_rows,
                                 int unit_blocks, bool f32, int sm_count, cudaStream_t stream);

}  // namespace ipotk
