// Launchers of rotary positions (rope.hip) and differential attention (attn_diff.hip).
#pragma once

#include <hip/hip_runtime_api.h>
#include <stdint.h>

namespace rt {

// (weak, as train.h's)

struct RopeArgs {
    const void* x;
    void* y;
    const void* positions;  // [T][axes], or [B][T][axes]
    const double* freq;     // [pairs], radians a position
    const int32_t* axis;    // [pairs]
    int64_t xs[3], ys[3];   // elements between samples, heads, tokens
    int32_t B, H, T, D;
    int32_t pairs, axes;
    int32_t type, pos_type;   // as train.h's kBf16 ..; 0: int32, 1: int64, 2: fp32
    int32_t half, per_sample;
    int32_t vec;              // elements of an access: 8, 4, or 1 where rows do not fit them
    int32_t inverse;
    float amplitude;
    int32_t each, groups;     // heads of a thread, threads that share a token's heads
};
constexpr int kRopeAhead = 4;  // heads that a thread asks for at once
// threads of a token and group of heads: one for each piece of a row, or for each pair of pieces that are turned together
inline int64_t rope_places(const RopeArgs& a) {
    return a.half || a.vec == 1 ? a.pairs / a.vec + (a.D - 2 * a.pairs) / a.vec : a.D / a.vec;
}
inline int64_t rope_blocks(const RopeArgs& a) { return (int64_t)a.B * a.groups * (((int64_t)a.T * rope_places(a) + 255) / 256); }
__attribute__((weak)) hipError_t launch_rope(const RopeArgs& a, hipStream_t stream);

constexpr int kDiffRows = 128;  // rows of a tile of four waves
constexpr int kDiffShort = 128;  // most rows of queries whose values a workgroup forms
constexpr int kDiffParts = 32;  // parts of a tile's keys, at most
constexpr float kDiffMove = 24.0f;  // the running max moves where a probability against it would pass 2^24
struct DiffArgs {
    const uint16_t* q;  // bf16 [B, 2 H, Tq, D]
    const uint16_t* k;  // bf16 [B, 2 H, Tk, D]
    const uint16_t* v;  // bf16 [B, H, Tk, 2 D]
    const float* lam;   // [H], or one value (lam_step 0)
    int32_t lam_step;
    const int32_t* k_lens;  // [B], or null
    int32_t by_len;  // the samples with most keys first (B up to 64)
    int32_t B, H, Tq, Tk, n_bh;
    float scale_nat, scale_log2;
    float move;  // the running max moves where a score is this far above it
    // forward
    uint16_t* o;    // bf16 [B, H, Tq, 2 D]
    uint16_t* o2;   // or null, with the statistics
    float* row_max;  // fp32 [B, 2 H, Tq]
    float* row_sum;
    int32_t by_keys;  // a workgroup's waves share the keys of 32 queries; else they take 32 queries each
    int32_t split;  // workgroups that share a tile's keys
    float* part;    // workspace of split walks
    // backward
    const uint16_t* d_o;
    uint16_t* dq;
    uint16_t* dk;
    uint16_t* dv;
    float* d_lam;
    float* row_vals;  // workspace [B, H][4][T64]
    double* lam_part;  // workspace [B, H][T64 / 16]: sums of -delta_2
    int32_t T64;      // Tq in whole 64
    int32_t short_rows;  // the workgroups form the row values
    int32_t q_first;  // tiles of queries before those of keys
    int32_t two;      // eight waves to a tile, four of them for each half of a stage
    int32_t split_k, split_q;  // workgroups that share the walk of a tile of keys, of queries
    float* part_k;    // workspace of split walks
    float* part_q;
};
__attribute__((weak)) hipError_t launch_diff(const DiffArgs& a, int D, hipStream_t stream);
__attribute__((weak)) hipError_t launch_diff_backward(const DiffArgs& a, int D, hipStream_t stream);

}  // namespace rt
