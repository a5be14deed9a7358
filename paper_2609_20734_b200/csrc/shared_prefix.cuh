// What the two kernels of the shared-prefix Full pass have in common: parameters of the first (shared_prefix.cu) and
// the descriptor by which the second (splitkv_tma.cu, kInstFold) finds the partial results of a row.
#pragma once
#include <cuda_bf16.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include "oda_device.cuh"

namespace oda {

struct SharedRow {   // one request
    int32_t unit;    // first tile of its row block within one (layer, kv head)
    int32_t tiles;   // tiles of its prefix (0: it shares nothing)
    int32_t row;     // its first row within the row block
};

// Partial results of a row over its prefix: chunk 0 at row ((gated layer) * batch + b) * q_heads + head, chunk c > 0 at
// ext_row0 + (first span + c) * 256 + row + head within the group.
struct SharedDesc {
    int32_t t1, total, nseg;         // tiles of one (layer, kv head), of all, spans they are cut into
    int32_t gated_index[kMaxLayers]; // layer -> its place among the call's gated layers
    SharedRow rows[kMaxBatch];
};

struct SharedParams {
    const __nv_bfloat16* q;
    const int32_t* block_table;
    const int32_t* seq_lens;
    const uint8_t* flags;
    const int32_t* group_start;
    const int32_t* group_prefix;
    int32_t* status;
    SharedDesc* desc;
    int32_t* page_shift;             // [batch] pages that the second kernel skips
    int32_t* tail_lens;              // [batch] positions that it sees
    float* part_o;                   // [rows][D] unnormalised
    float2* part_ml;                 // [rows] (m in log2 units, l)
    size_t ext_row0;
    int32_t batch, num_groups, num_q_heads, num_kv_heads, group, max_blocks_per_seq, num_gated, blocks_per_layer;
    float scale_log2e;
    uint8_t layer[kMaxLayers];       // the call's gated layers
    uint16_t kv_index[kMaxLayers];   // and their cache slices
};

cudaError_t launch_shared_prefix(const SharedParams& p, const void* kmap, const void* vmap, int head_dim, bool out_bf16,
                                 int grid, cudaStream_t st, bool pdl);

}  // namespace oda
