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

struct GroupDev {
    const void *x, *dy, *w, *b;
    void *y, *dx, *dw, *db;
    float *mean, *rstd;              // [batch][groups]
    float* part;                     // forward: [batch][groups][chunks][2] mean, sum of squared differences;
                                     // backward: [batch][chunks][2][channels] sums of dz xh, dz
    float* sums;                     // backward: [batch][2][channels], the same over all chunks
    float* means;                    // backward: [batch][groups][2] mean(g), mean(g xh)
    int64_t xs[2], ys[2], dxs[2];    // batch, pixel
    int batch, pixels, channels, groups, width;   // width: channels of a group
    int sample0;                     // a launch's first sample
    int slab, slabs;                 // channels of a block (whole groups; the last has what is left), blocks over them
    int chunk, chunks;               // pixels of a block, blocks over them
    int spread;                      // pixels of a block in the second pass
    float per_width;                 // 1 / width
    int whole;                       // a block's registers hold a slab's pixels: no partial sums
    int param_dtype, act;
    float eps;
};

struct FeedDev {
    const void *x, *gate, *up, *down, *dy;      // as given, with their strides
    int64_t x_stride, gate_stride, up_stride, down_stride, y_stride;
    const void *gate_bias, *up_bias, *down_bias;
    void* y;
    void* h;                         // [rows][hidden_pad] the gated product
    uint16_t *by_z, *by_u, *last;    // [rows][hidden_pad] u act'(g) and act(g), by which dh gives dz and du, in 24 bits: their upper
                                     // halves, and the last byte of both (may be null)
    void *dx, *dgate, *dup, *ddown, *dgate_bias, *dup_bias, *ddown_bias;
    void *dz, *du;                   // backward: [rows][hidden_pad] gradients by the two projections
    void *x_pad, *gate_pad, *up_pad, *down_pad, *dy_pad;   // copies in whole pieces of 16 bytes (null: read in place)
    float* largest;                  // backward in fp16: kLargest partial maxima of |dy|
    float* part;                     // partial sums of y, or of dx and then of the weights' gradients
    int rows, in, hidden, out;
    int in_pad, hidden_pad, out_pad; // multiples of 8
    int down_splits, dx_splits, weight_splits;   // ranges of a product's reduction that are summed apart
};
constexpr int kLargest = 256;

struct Int8Dev {
    const int8_t *x, *w;
    const float *x_scale, *w_scale;
    const void* bias;
    void* y;
    int rows, in, out;
    int64_t x_stride, w_stride, y_stride;
};

struct QuantizeDev {
    const void* x;
    int8_t* q;
    float* scale;
    int64_t rows, x_stride, q_stride;
    int cols;
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

// Fills in width and slab .. whole from the sizes.
void group_plan(GroupDev& d, int dtype, bool backward);
hipError_t group_forward(const GroupDev& d, int dtype, hipStream_t st);
hipError_t group_backward(const GroupDev& d, int dtype, hipStream_t st);

// Whether rows are read straight from memory (no copies in whole pieces).
bool feed_few(int64_t rows);
// Fills in the splits from the sizes; bytes of `part`.
size_t feed_plan(FeedDev& d, bool backward);
hipError_t feed_forward(const FeedDev& d, int dtype, int act, hipStream_t st);
hipError_t feed_backward(const FeedDev& d, int dtype, hipStream_t st);

hipError_t quantize_rows(const QuantizeDev& d, int dtype, hipStream_t st);
hipError_t int8_linear(const Int8Dev& d, int dtype, hipStream_t st);

}  // namespace pa
