// Launchers of the training calls: a mask's transpose, attention's gradients, the layer norm.
#pragma once

#include <hip/hip_runtime_api.h>
#include <stdint.h>

namespace rt {

// The launchers below are declared weak so that a host-only build of api.cpp (the checks
// under a sanitizer) can leave out those that it has no stand-in for.

// Transpose of a block mask (index.hip): row kb of mask m lists the query blocks that keep kb.  The plan that follows
// says which workgroup of the gradients' call walks what: lists of more than `seg` entries are split.
//   {mask * n_blk + kb, first entry, entries, part or -1} of every row, the first part of a split one,
//   then max_more of the like for further parts (mask * n_blk + kb is -1: none),
//   then max_more of {mask * n_blk + kb, first part, parts, 0} of split lists (-1: none)
// A first entry of -1: the mask's entries did not fit.
struct TransposeArgs {
    const int32_t* row_ptr;  // [n_masks][n_blk + 1]
    const int32_t* col_idx;
    int32_t nnz, n_blk, n_masks;
    int32_t* t_row_ptr;
    int32_t* t_col_idx;
    int32_t t_nnz;           // room for entries in t_col_idx
    int32_t* plan;           // behind them
    int32_t seg, max_more;
};
__attribute__((weak)) hipError_t launch_index_transpose(const TransposeArgs& a, hipStream_t stream);

// Gradients of attention (attn_grad.hip).
constexpr int kDenseRows = 128;  // rows of a dense tile
struct GradArgs {
    const uint16_t* q;  // bf16 [B,H,T,D]
    const uint16_t* k;
    const uint16_t* v;
    const uint16_t* o;
    const uint16_t* d_o;
    const float* row_max;  // fp32 [B,H,T]
    const float* row_sum;
    const float* rho;   // or null
    float rho_delta;
    float* d_rho;       // or null
    uint16_t* dq;
    uint16_t* dk;
    uint16_t* dv;
    float* row_vals;    // workspace [B,H][2][T64]: log2 of the denominator over the row's factor, and -dO . O
    int32_t T64;        // T in whole 64
    int32_t split;      // dense: workgroups that share a tile's walk; more than 1: part is [tile][split][dK, dV, dQ][rows][D]
    float* part;        // workspace: fp32 dK and dV [place][2][block][D] of split lists, max_slots for each use of a mask
    const int32_t* plan;  // of the transposed mask
    int32_t t_nnz, seg, max_more;
    int32_t fold;       // parts of a split list that a workgroup takes together
    int32_t max_base, max_slots;  // part numbers of the plan; places in `part`
    const int32_t* t_row_ptr;
    const int32_t* row_ptr;  // null: dense
    const int32_t* col_idx;
    const int32_t* t_col_idx;
    int32_t nnz, n_masks, heads;
    int32_t T, n_blk, block;
    int32_t n_bh;
    float scale_log2;   // log2(e) / sqrt(D)
    float scale_nat;    // 1 / sqrt(D)
};
__attribute__((weak)) hipError_t launch_attention_backward(const GradArgs& a, int D, hipStream_t stream);

// Layer norm (norm.hip).
enum { kBf16 = 0, kF16 = 1, kF32 = 2 };
struct NormArgs {
    const void* x;
    const void* dy;      // backward
    const void* weight;  // or null
    const void* bias;
    void* y;             // forward
    void* dx;            // backward
    float* mean_out;     // forward, or null
    float* rstd_out;
    const float* mean;   // backward
    const float* rstd;
    float* dweight;      // backward, or null
    float* dbias;
    float* partial;      // backward: [sets][parts][2][width]
    int64_t xs[3], ys[3], dxs[3];  // elements between rows: of x, of y or dy, of dx
    int32_t n1, n2;
    int32_t flat;        // rows of every tensor are s[2] apart throughout
    uint32_t rows_per_set, sets;
    uint32_t turn0;      // forward: workgroups of earlier launches
    int32_t width, type;
    int32_t vec;         // rows start on 16 bytes and hold whole chunks of 8 elements
    int32_t weight_f32;
    float eps;
};
__attribute__((weak)) hipError_t launch_norm(const NormArgs& a, hipStream_t stream);
// parts: the most workgroups (partial sums) of a set
__attribute__((weak)) hipError_t launch_norm_backward(const NormArgs& a, int32_t parts, hipStream_t stream);

}  // namespace rt
