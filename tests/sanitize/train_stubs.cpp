// Host-only stand-ins for the launchers of the training calls, beside launch_stubs.cpp.
#include <hip/hip_runtime_api.h>

#include <cstdio>
#include <cstdlib>

#include "train.h"

#define EXPECT(c)                                                                  \
    do {                                                                           \
        if (!(c)) {                                                                \
            std::fprintf(stderr, "launch stub: expectation failed: %s\n", #c);    \
            std::abort();                                                          \
        }                                                                          \
    } while (0)

namespace rt {

hipError_t launch_index_transpose(const TransposeArgs& a, hipStream_t) {
    EXPECT(a.row_ptr && a.col_idx && a.t_row_ptr && a.t_col_idx);
    EXPECT(a.n_blk > 0 && a.n_masks > 0 && a.nnz > 0 && a.t_nnz >= a.nnz);
    EXPECT(a.plan >= a.t_col_idx + a.t_nnz && a.seg >= 1 && a.max_more >= 0);
    return hipSuccess;
}

hipError_t launch_attention_backward(const GradArgs& a, int D, hipStream_t) {
    EXPECT(D == 64 || D == 72);
    EXPECT(a.q && a.k && a.v && a.o && a.d_o && a.row_max && a.row_sum && a.dq && a.dk && a.dv);
    EXPECT(a.row_vals && a.T64 >= a.T && a.T64 < a.T + 64 && a.T64 % 64 == 0);
    EXPECT(a.T > 0 && a.n_bh > 0 && (long long)a.T * D * 2 <= (1LL << 30));
    EXPECT(!a.d_rho || a.rho);
    if (!a.row_ptr) EXPECT(a.split >= 1 && a.split <= a.T64 / 64 && a.part >= a.row_vals + 2 * (size_t)a.n_bh * a.T64);
    if (a.row_ptr) {
        EXPECT(a.col_idx && a.t_col_idx && a.plan > a.t_col_idx && a.nnz > 0);
        EXPECT(a.n_blk == (a.T + a.block - 1) / a.block && a.n_bh % a.n_masks == 0);
        EXPECT(a.fold >= 1 && a.seg >= 1 && a.t_row_ptr && a.max_slots <= a.max_base);
        EXPECT(a.max_more ? a.max_slots >= 2 * a.max_more / a.fold : a.max_slots == 0);
        EXPECT((char*)a.part >= (char*)(a.row_vals + 2 * (size_t)a.n_bh * a.T64) && ((uintptr_t)a.part & 15) == 0);
        EXPECT((a.block == 32 || a.block == 64) && a.n_masks >= 1);
    }
    return hipSuccess;
}

static void check_norm(const NormArgs& a) {
    EXPECT(a.x && a.width >= 1 && a.width <= 16384 && a.type >= 0 && a.type <= 2);
    EXPECT(a.rows_per_set > 0 && a.sets > 0 && (uint64_t)a.rows_per_set * a.sets < (1ull << 31));
    EXPECT(!a.vec || a.width % 8 == 0);
    EXPECT(a.n1 > 0 && a.n2 > 0);
}

hipError_t launch_norm(const NormArgs& a, hipStream_t) {
    check_norm(a);
    EXPECT(a.y && a.eps >= 0);
    return hipSuccess;
}

hipError_t launch_norm_backward(const NormArgs& a, int32_t parts, hipStream_t) {
    if (a.rows_per_set == 0) {
        EXPECT((a.dweight || a.dbias) && a.sets > 0 && a.width >= 1);
        return hipSuccess;
    }
    check_norm(a);
    EXPECT(a.dy && a.dx && a.mean && a.rstd && a.partial && parts >= 1);
    return hipSuccess;
}

}  // namespace rt
