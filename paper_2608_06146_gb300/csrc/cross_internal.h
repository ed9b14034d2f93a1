// cross_internal.h -- layouts shared by the cross-attention planner and its kernels.
//
// Rows are packed for the tensor cores as (token, query head of the KV head's group): 64-row blocks of
// 64 / group tokens, so that every query head of a KV head reads a key tile together, whatever the group. A tile is
// two blocks, the M = 128 of the MMAs; the forward's unit is two tiles.
#pragma once

#include <stdint.h>

#include "padoc_attn.h"

#define PADOC_CROSS_BLOCK 64         // rows of a block
#define PADOC_CROSS_UNIT_BLOCKS 4    // blocks of the forward's unit
#define PADOC_CROSS_DQ_BLOCKS 2      // blocks of the dq pass's unit
#define PADOC_CROSS_KEY_TILE 128     // keys of a tile: of the forward's steps and of the dk/dv pass's units
#define PADOC_CROSS_DQ_STEP 64       // keys of a step of the dq pass
#define PADOC_CROSS_FEW_ROWS 32      // most rows of a unit of the kernel for few rows
#define PADOC_CROSS_FEW_STEP 64      // keys of its tiles

// Forward and dq work item: tokens of one segment, one KV head, a part of the segment's keys. 32 bytes.
struct padoc_cross_unit {
    int32_t tok, ntok;    // query rows
    int32_t k0, nk;       // key rows, nk >= 1
    int32_t g;            // KV head
    int32_t slot;         // partial result, -1: the rows' whole key range, written as the output
    int32_t sub;          // dq: index of the first block in the statistics, -1: another part writes them
    int32_t pad;
};
// Rows joined from parts slot .. slot + parts - 1 (none: a segment without keys). 32 bytes.
struct padoc_cross_merge {
    int32_t tok, ntok, slot, parts, g;
    int32_t pad[3];
};
// Keys of one or more overlapping ranges, with covers cover .. cover + ncover - 1, of `steps` blocks together. 32 bytes.
struct padoc_cross_key_tile {
    int32_t k0, nk;
    int32_t cover, ncover;
    int32_t steps;
    int32_t pad[3];
};
// A segment that sees keys k0 .. k0 + nk - 1 of the tile: its rows and blocks. 32 bytes.
struct padoc_cross_cover {
    int32_t tok, ntok, sub, nsub;
    int32_t k0, nk;
    int32_t pad[2];
};

// dk/dv work item (bf16): steps first .. first + steps - 1 of a key tile for one KV head. 32 bytes.
struct padoc_cross_dkv {
    int32_t k0, nk, cover;
    int32_t first, steps;
    int32_t g;
    int32_t slot;         // partial sums, -1: all of the tile's steps, written as the gradients
    int32_t pad;
};
// A key tile's sums joined from parts slot .. slot + parts - 1. 32 bytes.
struct padoc_cross_dkv_sum {
    int32_t k0, nk, g, slot, parts;
    int32_t pad[3];
};

// Blocks of the statistics, lse and D: [Hkv][num_subs][64] floats each.
