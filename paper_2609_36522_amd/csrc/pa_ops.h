// Declarations shared by the operators' host side (paraanya_ops.cpp) and their gfx950 kernels.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "paraanya_ops.h"

namespace pa {

// ------------------------------------------------------------------ launch parameters
struct NormDev {
    const void *x, *dy, *w, *b;
    void *y, *dx, *dw, *db;
    float *mean, *rstd;              // written by the forward pass (may be null), read by the backward
    float* part;                     // backward: [blocks][2][cols] partial sums of dweight, dbias
    int64_t rows, x_stride, y_stride, dx_stride;
    int cols, blocks;                // blocks: rows of `part`
    float eps;
};

struct CrossDev {
    const void *q, *k, *v, *d_o;
    void *o, *dq, *dk, *dv;
    float* stats;                    // [batch][q_heads][q_len][2]
    const int32_t* kv_lens;
    const void* mask;
    int mask_kind;
    int batch, q_heads, kv_heads, group;   // group: query heads per kv head
    int q_len, kv_len, dim;
    int rows;                        // q_len * group: rows that share a kv head, row = token * group + head in group
    int whole;                       // forward, dq: row tiles that one block takes over all keys; the others are
    int splits, split_keys;          // split into key ranges of split_keys keys (a multiple of the key tile)
    int row_splits, split_tiles;     // dk, dv: ranges of split_tiles tiles of 32 tokens of a query head
    float scale;
    int64_t mask_stride;
    int64_t qs[3], ks[3], vs[3], os[3], dos[3], dqs[3], dks[3], dvs[3];   // batch, token, head
    int tile_rows, tiles;            // rows of a row tile, row tiles of all samples and kv heads
    float* part;                     // partial o, or partial dq: [split tile][splits][tile_rows][dim]
    float* part_stats;               // [split tile][splits][tile_rows][2]
    float* row_stats;                // backward: [batch][q_heads][tiles of 32 tokens][3][32]
    float *part_dk, *part_dv;        // [row_splits][batch * kv_heads][kv_len][dim]
};

struct LoraDev {
    const void *x, *w, *bias, *a, *b;
    void* y;
    void* t;                         // [rows][rank_pad] x A^T, scaled, in the element type
    const int32_t *offsets, *ids;
    const float* scales;
    int rows, in, out, rank, rank_pad, adapters, requests;   // rank_pad: a multiple of 16
    int64_t x_stride, w_stride, y_stride;
};

// Launchers return the launch's hipError_t.
hipError_t norm_forward(const NormDev& d, int dtype, int param_dtype, hipStream_t st);
int norm_backward_blocks(int64_t rows, int64_t cols);
hipError_t norm_backward(const NormDev& d, int dtype, int param_dtype, hipStream_t st);

// How the forward pass (and dq) splits the keys, and dk, dv the rows: see cross_plan (k_cross_bwd.hip).
void cross_plan(CrossDev& d, bool backward);
hipError_t cross_forward(const CrossDev& d, int dtype, hipStream_t st);
hipError_t cross_backward(const CrossDev& d, int dtype, hipStream_t st);

hipError_t lora_linear(const LoraDev& d, int dtype, hipStream_t st);

}  // namespace pa
