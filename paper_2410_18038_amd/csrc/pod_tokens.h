// What happens to a batch's new tokens before their attention: blocks and slots from the request lengths, and their
// projections normalised, rotated and written to where the attention reads them.
#pragma once
#include <hip/hip_runtime_api.h>

#include <string>

#include "../../include/pod_attn.h"
#include "pod_common.h"

namespace pod {

// Division of a 31-bit token or slot number by `d` as a product: ceil(2^32 / d) is at most one too large a factor for the
// quotient (0 stands for d = 1).
inline uint32_t division_magic(int32_t d) { return d > 1 ? (uint32_t)(((uint64_t(1) << 32) + (uint64_t)d - 1) / (uint64_t)d) : 0u; }

struct TableArgs {
    const int32_t *seq_meta, *free_blocks;
    int32_t *block_table, *slots, *positions, *report;
    int32_t n_free, n_prefill, n_decode, n_rows;
    int32_t block_size;                    // tokens per block; 0: contiguous
    int32_t per_row;                       // tokens a cache row has room for
    uint32_t magic;                        // of block_size
    int32_t max_blocks, n_cache_rows, n_blocks;
    int32_t n_decode_wgs, wgs_per_prefill; // workgroups: the decode requests', then so many for each prefill request
};

struct AppendArgs {
    const void *q, *k, *v;
    const uint64_t *table;
    const void *q_weight, *k_weight;
    const int32_t *slots, *positions;
    void *q_out, *k_cache, *v_cache;
    int64_t q_stride, k_stride, v_stride;  // elements between rows
    int64_t block_elems, head_stride;      // elements between blocks (or cache rows), between the heads of one
    int32_t tok_stride;
    int32_t per_block;                     // slots per block (or cache row)
    uint32_t magic;                        // of per_block
    int32_t n_slots;                       // slots of the cache
    int32_t n_rows, n_q_heads, n_kv_heads;
    int32_t rot_dim;                       // 0: no rotation
    float cos_sin_scale, eps, weight_offset;
    int32_t norm_q, norm_k;
};

hipError_t launch_tables(const TableArgs &a, hipStream_t stream);
hipError_t launch_append(const AppendArgs &a, int dtype, int head_dim, int layout, hipStream_t stream);
// Heads that a wavefront of the append kernel works on at a time.
constexpr int append_heads(int head_dim) { return kWaveSize * 16 / head_dim; }

}  // namespace pod
