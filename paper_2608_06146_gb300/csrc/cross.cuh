// cross.cuh -- what the cross-attention kernels share: the packed rows of a block, and the arguments.
#pragma once

#include "common.cuh"
#include "cross_internal.h"

// Arguments of the forward and of both backward passes.
struct padoc_cross_args {
    const padoc_cross_unit *units;             // forward or dq items
    const int32_t *ctas;                       // first item of each CTA's list, and the end; null: an item a CTA
    const padoc_cross_merge *merges;
    const padoc_cross_key_tile *tiles;
    const padoc_cross_cover *covers;
    const void *q, *k, *v, *out, *dout;
    const float *lse_in;
    int64_t q_stride, k_stride, v_stride;      // elements
    int64_t query_rows, key_rows;
    int64_t dq_stride, dk_stride, dv_stride;
    void *o, *dq, *dk, *dv;
    float *lse;
    float *part, *part_lse;                    // partial results
    float *part_dkv;                           // of key tiles: [slot][128][dV | dK]
    const padoc_cross_dkv *dkv;                // dk/dv items (bf16), each CTA's list of them, and what joins parts
    const int32_t *dkv_ctas;
    const padoc_cross_dkv_sum *dkv_sums;
    int32_t num_dkv_ctas, num_dkv_sums, num_dkv_slots;
    int32_t gap_tile;                          // first of the tiles that no row sees (the last ones)
    float *neg_lse2, *dsum;                    // -lse * log2(e) and rowsum(dO * O) (bf16: 16 bytes of its negative): [Hkv][subs][64]
    int32_t unit_rows;                         // packed rows of a forward or dq item, and of its partial result
    int32_t num_units, num_ctas, num_merges, max_parts, num_tiles, num_subs;
    int32_t tail_begin, tail_tiles;            // key rows that the plan does not reach
    int32_t hq, hkv, group, block_tokens;      // block_tokens: 64 / group
    float scale, scale_log2;
    int *err;
};

// The (token, head) of packed row r (of a run of blocks) of a unit whose first token is tok: false past its rows.
__device__ __forceinline__ bool cross_row(const padoc_cross_args &a, int tok, int ntok, int r, int &token, int &head)
{
    const int rr = r % PADOC_CROSS_BLOCK, t = rr / a.group;
    const int i = r / PADOC_CROSS_BLOCK * a.block_tokens + t;
    token = tok + i;
    head = rr - t * a.group;
    return t < a.block_tokens && i < ntok;
}

// The forward's units on the tensor cores (cross_tc.cu).
padoc_status padoc_cross_launch_tc(const padoc_cross_args &args, int head_dim, cudaStream_t stream);
// The same for items of at most 32 rows, each by a cluster (cross_few.cu).
padoc_status padoc_cross_launch_few(const padoc_cross_args &args, int head_dim, int cluster, cudaStream_t stream);
// The backward's passes on the tensor cores (cross_bwd_tc.cu).
padoc_status padoc_cross_launch_bwd_tc(const padoc_cross_args &args, int head_dim, cudaStream_t stream);
