// Gradients of attention (gfx950, CDNA4): dQ, dK, dV of dense and block-sparse attention, with or without the
// reshape's factor, the probabilities recomputed from the forward call's row statistics.
//
//   grad_rows    per query row: -delta = -dO . O, and log2 of the denominator over the row's factor
//   grad_dense   dK and dV of 128 keys, or dQ of 128 queries, to a workgroup of four waves
//   grad_sparse  the same for one block, over the blocks its row of the (transposed) mask lists
//   grad_join    sums of the parts of key blocks whose lists were split
//   grad_sum     the same of dense tiles whose walks are shared, where there are few
//
// Seven products of T x T x D instead of the five that the gradients need: the scores and dP are formed for dK and dV
// and again for dQ, so that every sum stays in one wave's registers: no atomics, equal bits from equal calls.
// The wave's walk is attn_grad_tiles.h's.

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "attn_common.h"
#include "attn_grad_tiles.h"
#include "train.h"

namespace rt {
namespace {

// ---- rows ----------------------------------------------------------------------------------

// 8 lanes a row; rows are counted with each head's padded to whole 64, whose values are zeros
template <int D>
__global__ __launch_bounds__(256) void grad_rows(GradArgs a, int64_t rows) {
    const int64_t i = ((int64_t)blockIdx.x * 256 + threadIdx.x) >> 3;
    const int c = threadIdx.x & 7;
    if (i >= rows) return;
    const int64_t bh = i / a.T64;
    const int t = (int)(i - bh * a.T64);
    float* vals = a.row_vals + bh * 2 * a.T64 + t;
    if (t >= a.T) {
        if (c == 0) vals[0] = vals[a.T64] = 0.f;
        return;
    }
    const int64_t row = bh * a.T + t;
    const float s = row_delta<D>(a, row, c);
    if (c == 0) {
        float log = row_log(a, row);
        if (a.rho) {
            const float r = a.rho[row] + a.rho_delta;
            log -= log2f(fminf(1.0f, r));  // a factor of 0: +inf, no probability
            if (a.d_rho) a.d_rho[row] = r <= 1.0f ? s : 0.f;
        }
        vals[0] = log;
        vals[a.T64] = -s;
    }
}

// Stages of the ring.  Two: a longer lead cost more than it gave (three: dense CogVideoX 15.4 against 14.8 ms, all with
// two waves to a SIMD; its sparse call 785 us with four, 696 with two).
constexpr int kStages = 2;

// ---- dense ---------------------------------------------------------------------------------

// A head of up to kShort rows: its workgroups form the row values themselves (those of dK and dV all of them, in LDS),
// which saves the launch of grad_rows.
constexpr int kShort = 512;

// dK and dV (KV) or dQ of 32 W rows of a head against all of the other side: stages 0, 1, .. of 64 rows.  SPLIT: against
// one of a.split parts of it, whose fp32 sums grad_sum adds.
template <int D, bool KV, int W, bool SHORT, bool SPLIT>
__device__ __forceinline__ void dense_walk(const GradArgs& a, lds_u8* lds, int item, int part) {
    using R = GradRing<D, KV && !SHORT, W, 64, kStages>;
    const int T = a.T, n64 = (T + 63) >> 6, n_tile = (T + 32 * W - 1) / (32 * W);
    const int bh = item / n_tile;
    const int row0 = ((item - bh * n_tile) * W + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6)) * 32;
    const size_t head_off = (size_t)bh * (size_t)T * D;
    R ring;
    ring.init(lds, (KV ? a.q : a.k) + head_off, (KV ? a.d_o : a.v) + head_off, a.row_vals + (size_t)bh * 2 * a.T64, T,
              a.T64);
    const int s0 = SPLIT ? n64 * part / a.split : 0, s1 = SPLIT ? n64 * (part + 1) / a.split : n64;
    ring.load(0, s0 * 64);
    GradTile<D, KV, R::ZERO, R::TENSOR> t;
    t.init(lds, a.scale_log2);
    t.load_own(a, head_off, row0, T);
    constexpr int LOGS = R::LDS, MINUS = LOGS + kShort * 4;  // SHORT: LDS offsets of all rows' values
    if (KV && SHORT) {
        for (int i = threadIdx.x >> 3; i < a.T64; i += 8 * W) {
            const int c = threadIdx.x & 7;
            float log = 0.f, minus = 0.f;
            if (i < T) {
                const size_t row = (size_t)bh * T + i;
                minus = -row_delta<D>(a, row, c);
                log = row_log(a, row);
            }
            if (c == 0) {
                *(__attribute__((address_space(3))) float*)(lds + LOGS + 4 * i) = log;
                *(__attribute__((address_space(3))) float*)(lds + MINUS + 4 * i) = minus;
            }
        }
    }
    if (!KV) {
        if (SHORT)
            t.make_values(a, bh, row0, T);
        else
            t.load_values(a, bh, row0, T);
    }
    int st = 0;  // LDS offset of the stage in use
    for (int s = s0; s < s1; ++s) {
        ring.turn();
        ring.load(R::STAGE - st, (s + 1) * 64);
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int cx = st + 32 * h * R::ROWB, row = s * 64 + 32 * h;
            t.scores(cx, SHORT ? MINUS + 4 * row : st + R::STAT + 256 + 128 * h);
            if (!KV && row + 32 > T) t.mask(row, T);
            t.soft(SHORT ? LOGS + 4 * row : st + R::STAT + 128 * h);
            t.grads(cx);
        }
        st = R::STAGE - st;
    }
    wait_vm<0>();  // nothing may land in LDS after the workgroup has ended
    if (SPLIT) {
        float* to = a.part + ((size_t)item * a.split + part) * (3 * 32 * W * D) + (threadIdx.x >> 6) * 32 * D;
        t.store_part(0, to + (KV ? 0 : 2 * 32 * W * D), a.scale_nat);
        if (KV) t.store_part(KV ? 1 : 0, to + 32 * W * D, 1.0f);
        return;
    }
    t.store_all(a, head_off, row0, T);
}

template <int D, int W, int WAVES, bool SHORT, bool SPLIT>
__global__ __launch_bounds__(64 * W) __attribute__((amdgpu_waves_per_eu(WAVES, WAVES))) void grad_dense(GradArgs a,
                                                                                                      int n_items,
                                                                                                      int per_xcd) {
    __shared__ __attribute__((aligned(1024))) unsigned char smem[GradRing<D, true, W, 64, kStages>::LDS +
                                                                 (SHORT ? 2 * kShort * 4 : 0)];
    // the first half of the workgroups, which has more to do, takes dK and dV
    const bool kv = (int)blockIdx.x < 8 * per_xcd;
    const int g = kv ? blockIdx.x : blockIdx.x - 8 * per_xcd;
    int item = (g & 7) * per_xcd + (g >> 3), part = 0;
    if (item >= n_items) return;
    if (SPLIT) {
        part = item % a.split;
        item /= a.split;
    }
    if (kv)
        dense_walk<D, true, W, SHORT, SPLIT>(a, (lds_u8*)smem, item, part);
    else
        dense_walk<D, false, W, SHORT, SPLIT>(a, (lds_u8*)smem, item, part);
}

// out[j .. j + 3], below size, from n parts STRIDE apart, in order; four of them asked for at a time
template <int STRIDE>
__device__ __forceinline__ void sum_parts(const float* part, int n, uint16_t* out, int j, int size) {
    if (j >= size) return;
    f32x4 s = {};
#pragma unroll 4
    for (int k = 0; k < n; ++k) s += *reinterpret_cast<const f32x4*>(part + (size_t)k * STRIDE + j);
    reinterpret_cast<uint32_t*>(out + j)[0] = pack_bf16(s[0], s[1]);
    reinterpret_cast<uint32_t*>(out + j)[1] = pack_bf16(s[2], s[3]);
}

// dK, dV or dQ (blockIdx.y) of 32 W rows, 1024 values of them (blockIdx.z)
template <int D, int W>
__global__ __launch_bounds__(256) void grad_sum(GradArgs a) {
    constexpr int SIZE = 32 * W * D;
    const int n_tile = (a.T + 32 * W - 1) / (32 * W), bh = blockIdx.x / n_tile, row0 = (blockIdx.x - bh * n_tile) * 32 * W;
    const float* part = a.part + (size_t)blockIdx.x * a.split * (3 * SIZE) + blockIdx.y * SIZE;
    uint16_t* out = (blockIdx.y == 0 ? a.dk : blockIdx.y == 1 ? a.dv : a.dq) + ((size_t)bh * a.T + row0) * D;
    const int left = a.T - row0, size = (left < 32 * W ? left : 32 * W) * D;
    sum_parts<3 * SIZE>(part, a.split, out, blockIdx.z * 1024 + threadIdx.x * 4, size);
}

// ---- sparse --------------------------------------------------------------------------------

// dK and dV (KV) or dQ of one block of a head against the `count` blocks listed from `list` on.  part: null, or where
// the fp32 sums of a split list go.
template <int D, bool KV, int W>
__device__ __forceinline__ void sparse_walk(const GradArgs& a, lds_u8* lds, int bh, int blk, const int32_t* list, int count,
                                            float* part) {
    using R = GradRing<D, KV, W, 32, kStages>;
    const int T = a.T, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int row0 = blk * (32 * W) + 32 * wave;
    const size_t head_off = (size_t)bh * (size_t)T * D;
    const csr_ptr idx = (csr_ptr)list;
    const int n = count * W;
    R ring;
    ring.init(lds, (KV ? a.q : a.k) + head_off, (KV ? a.d_o : a.v) + head_off, a.row_vals + (size_t)bh * 2 * a.T64, T,
              a.T64);
    auto row_at = [&](int s) {  // first row of stage s; none past the list or for an index out of range
        if (s >= n) return -1;
        const int c = idx[s / W];
        return c < 0 || c >= a.n_blk ? -1 : c * (32 * W) + 32 * (s % W);
    };
    int rows[kStages];  // of the stages under way; the last one is the next to be asked for
#pragma unroll
    for (int i = 0; i < kStages; ++i) rows[i] = row_at(i);
#pragma unroll
    for (int i = 0; i < kStages - 1; ++i) ring.load(i * R::STAGE, rows[i]);
    GradTile<D, KV, R::ZERO, R::TENSOR> t;
    t.init(lds, a.scale_log2);
    t.load_own(a, head_off, row0, T);
    if (!KV) t.load_values(a, bh, row0, T);
    int st = 0;
    for (int s = 0; s < n; ++s) {
        ring.turn();
        ring.load(st == 0 ? (kStages - 1) * R::STAGE : st - R::STAGE, rows[kStages - 1]);
        const int at = rows[0];
#pragma unroll
        for (int i = 0; i < kStages - 1; ++i) rows[i] = rows[i + 1];
        rows[kStages - 1] = row_at(s + kStages);
        t.scores(st, st + R::STAT + 128);
        if (!KV && (at < 0 || at + 32 > T)) t.mask(at < 0 ? T : at, T);
        t.soft(st + R::STAT);
        t.grads(st);
        st = st == (kStages - 1) * R::STAGE ? 0 : st + R::STAGE;
    }
    wait_vm<0>();
    if (part) {
        if (KV) {
            t.store_part(0, part + 32 * wave * D, a.scale_nat);
            t.store_part(KV ? 1 : 0, part + 32 * (W + wave) * D, 1.0f);
        }
        return;
    }
    t.store_all(a, head_off, row0, T);
}

// Where the parts of a list whose numbers in the plan begin with `base` lie.  Taken `fold` at a time, n of them (more
// than fold) need n / fold places, rounded up: at most 2 n / fold, rounded down.
__device__ __forceinline__ int part_place(const GradArgs& a, int base) {
    base = base < a.max_base ? base : a.max_base;
    return a.fold > 1 ? 2 * base / a.fold : base;
}

// W: waves of a block (32 rows each).  Workgroups: the further parts of split lists, dK and dV of every block, then dQ,
// so that what takes longest begins first.  (A block's dK and dV next to its dQ, which reads the same rows, was no
// faster at the CogVideoX shape and 20 % slower where the lists are random.)
//
// Three waves to a SIMD where two share a ring (72 wide: 3 registers spilled, none read inside the walk).  A lone wave's ring leaves room for two by LDS; in the registers of three
// the 72-wide walk's sums go through the accumulator file (32 heads of 4096 tokens, 9 kept blocks of 32: 84 against 75
// us with all 512 registers for two; 1024 tokens 30.5 against 26.2; 64-wide ones equal).
template <int D, int W>
__global__ __launch_bounds__(64 * W) __attribute__((amdgpu_waves_per_eu(W == 1 ? 2 : 3, W == 1 ? 2 : 3))) void
grad_sparse(GradArgs a, int more, int n_items, int per_xcd) {
    __shared__ __attribute__((aligned(1024))) unsigned char smem[GradRing<D, true, W, 32, kStages>::LDS];
    lds_u8* const lds = (lds_u8*)smem;
    const csr_ptr plan = (csr_ptr)a.plan;
    int bh, blk, m, item;
    if ((int)blockIdx.x < more) {
        // every fold-th part of a list is one to begin with, so that of `fold` items in a row at most one is
        const int each = (a.max_more + a.fold - 1) / a.fold, rep = blockIdx.x / each;
        const int i0 = (blockIdx.x - rep * each) * a.fold, i1 = i0 + a.fold < a.max_more ? i0 + a.fold : a.max_more;
        int row = -1;
        item = a.n_masks * a.n_blk + i0 - 1;
        for (int i = i0; i < i1 && row < 0; ++i) {
            row = plan[4 * ++item];
            if (row < 0 || row >= a.n_masks * a.n_blk) return;  // no more items
            const int nth = plan[4 * item + 3] - plan[4 * row + 3];
            if (nth < 1 || nth % a.fold) row = -1;
        }
        if (row < 0) return;
        m = row / a.n_blk;
        blk = row - m * a.n_blk;
        bh = a.n_masks == 1 ? rep : (a.n_masks == a.heads ? rep * a.heads + m : m);
    } else {
        const int g = blockIdx.x - more, half = g < 8 * per_xcd ? 0 : 8 * per_xcd;
        const int i = ((g - half) & 7) * per_xcd + ((g - half) >> 3);
        if (i >= n_items) return;
        bh = i / a.n_blk;
        blk = i - bh * a.n_blk;
        m = a.n_masks == 1 ? 0 : (a.n_masks == a.heads ? bh % a.heads : bh);
        item = half ? -1 : m * a.n_blk + blk;
    }
    if (item < 0) {
        const csr_ptr p = (csr_ptr)a.row_ptr + (size_t)m * (a.n_blk + 1) + blk;
        int b = p[0], e = p[1];
        b = b < 0 ? 0 : (b > a.nnz ? a.nnz : b);
        e = e < b ? b : (e > a.nnz ? a.nnz : e);
        sparse_walk<D, false, W>(a, lds, bh, blk, a.col_idx + b, e - b, nullptr);
    } else if (plan[4 * item + 1] >= 0) {
        // (clamped to their arrays, as the CSR is: whatever t holds, nothing else is read or written)
        const csr_ptr p = plan + 4 * item;
        const int first = p[1] < a.t_nnz ? p[1] : a.t_nnz, base = plan[4 * (m * a.n_blk + blk) + 3];
        int slot = p[3] < 0 || base < 0 || p[3] < base ? -1 : part_place(a, base) + (p[3] - base) / a.fold, count = p[2];
        if (slot >= 0 && a.fold > 1) {
            const int left = a.t_row_ptr[m * (a.n_blk + 1) + blk + 1] - first;
            count = a.seg * a.fold;
            if (left <= count) {
                count = left;
                if (p[3] == base) slot = -1;  // all of the list
            }
        }
        slot = slot < a.max_slots ? slot : -1;
        count = count < 0 ? 0 : (count < a.t_nnz - first ? count : a.t_nnz - first);
        const int rep = a.n_masks == 1 ? bh : (a.n_masks == a.heads ? bh / a.heads : 0);
        sparse_walk<D, true, W>(a, lds, bh, blk, a.t_col_idx + first, count,
                                slot < 0 ? nullptr : a.part + ((size_t)rep * a.max_slots + slot) * (2 * 32 * W * D));
    } else {  // the transpose did not fit its array
        const size_t at = (size_t)bh * (size_t)a.T * D + (size_t)blk * 32 * W * D;
        const int left = a.T - blk * 32 * W, size = (left < 32 * W ? left : 32 * W) * D;
        for (int j = threadIdx.x; j < size; j += 64 * W) a.dk[at + j] = a.dv[at + j] = 0x7fc0;
    }
}

// dK (blockIdx.y 0) or dV of one split key block: its parts in order
template <int D, int W>
__device__ __forceinline__ void join_list(const GradArgs& a, int rep, int i) {
    const csr_ptr p = (csr_ptr)a.plan + 4 * (a.n_masks * a.n_blk + a.max_more + i);
    const int row = p[0];
    if (row < 0 || row >= a.n_masks * a.n_blk || p[1] < 0 || p[2] <= a.fold || p[2] > a.max_base) return;
    const int m = row / a.n_blk, blk = row - m * a.n_blk, first = part_place(a, p[1]), n = (p[2] + a.fold - 1) / a.fold;
    if (n > a.max_slots - first) return;
    const int bh = a.n_masks == 1 ? rep : (a.n_masks == a.heads ? rep * a.heads + m : m);
    constexpr int SIZE = 32 * W * D;
    const float* part = a.part + ((size_t)rep * a.max_slots + first) * (2 * SIZE) + blockIdx.y * SIZE;
    uint16_t* out = (blockIdx.y ? a.dv : a.dk) + (size_t)bh * (size_t)a.T * D + (size_t)blk * SIZE;
    const int left = a.T - blk * 32 * W, size = (left < 32 * W ? left : 32 * W) * D;
    for (int j = threadIdx.x * 4; j < size; j += 2048) sum_parts<2 * SIZE>(part, n, out, j, size);
}
template <int D, int W>
__global__ __launch_bounds__(512) void grad_join(GradArgs a) {
    const int each = (a.max_more + a.fold - 1) / a.fold, rep = blockIdx.x / each;
    for (int i = blockIdx.x - rep * each; i < a.max_more; i += each) join_list<D, W>(a, rep, i);
}

template <int D, int W>
hipError_t launch_sparse(const GradArgs& a, hipStream_t stream) {
    const int rep = a.n_bh / a.n_masks, more = rep * ((a.max_more + a.fold - 1) / a.fold), n = a.n_bh * a.n_blk, per = (n + 7) / 8;
    hipLaunchKernelGGL((grad_sparse<D, W>), dim3(more + 16 * per), dim3(64 * W), 0, stream, a, more, n, per);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess || more == 0) return e;
    hipLaunchKernelGGL((grad_join<D, W>), dim3(more, 2), dim3(512), 0, stream, a);
    return hipGetLastError();
}

template <int D>
hipError_t launch_d(const GradArgs& a, hipStream_t stream) {
    constexpr int W = kDenseRows / 32;
    const int n = a.n_bh * ((a.T + 32 * W - 1) / (32 * W)), per = (n + 7) / 8;
    const bool few = n < 256;  // 2 n workgroups over 256 CUs
    if (a.row_ptr || a.T > kShort || !few) {
        const int64_t rows = (int64_t)a.n_bh * a.T64;
        hipLaunchKernelGGL((grad_rows<D>), dim3((uint32_t)((rows * 8 + 255) / 256)), dim3(256), 0, stream, a, rows);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    if (a.row_ptr) return a.block == 64 ? launch_sparse<D, 2>(a, stream) : launch_sparse<D, 1>(a, stream);
    // Workgroups of four waves (eight: 15.6 against 15.4 ms at the CogVideoX shape, 11.4 against 8.4 us at 2 heads of 256
    // tokens).  64-wide heads run three waves to a SIMD where there are as many (14.5 against 14.8 ms, though the
    // compiler spills 6 registers, 4 of them read again at each stage of dK and dV; 9.0 against 7.9 us where there are
    // not: a wave with fewer registers waits more); 72-wide ones spill far more (819 against 533).
    if (!few)
        hipLaunchKernelGGL((grad_dense<D, W, D == 64 ? 3 : 2, false, false>), dim3(16 * per), dim3(64 * W), 0, stream, a, n, per);
    else if (a.split > 1) {
        const int all = n * a.split, each = (all + 7) / 8;
        hipLaunchKernelGGL((grad_dense<D, W, 2, false, true>), dim3(16 * each), dim3(64 * W), 0, stream, a, all, each);
        const hipError_t e = hipGetLastError();
        if (e != hipSuccess) return e;
        hipLaunchKernelGGL((grad_sum<D, W>), dim3(n, 3, kDenseRows * D / 1024), dim3(256), 0, stream, a);
    } else if (a.T > kShort)
        hipLaunchKernelGGL((grad_dense<D, W, 2, false, false>), dim3(16 * per), dim3(64 * W), 0, stream, a, n, per);
    else
        hipLaunchKernelGGL((grad_dense<D, W, 2, true, false>), dim3(16 * per), dim3(64 * W), 0, stream, a, n, per);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_attention_backward(const GradArgs& a, int D, hipStream_t stream) {
    return D == 64 ? launch_d<64>(a, stream) : launch_d<72>(a, stream);
}

}  // namespace rt
