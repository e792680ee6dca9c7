// Differential attention and its gradients (gfx950, CDNA4).
//
//   P_i = softmax(Q_i K_i^T / sqrt(D)), i = 1, 2, over the keys that a sample has;  O = P_1 V - lam P_2 V
//
//   dA = dO V^T,  delta_i = dO . (P_i V),  dS_1 = P_1 (dA - delta_1),  dS_2 = -lam P_2 (dA - delta_2)
//   dV = (P_1 - lam P_2)^T dO,  dQ_i = dS_i K_i / sqrt(D),  dK_i = dS_i^T Q_i / sqrt(D),  dlam = -sum of delta_2
//
//   diff_fwd    32 queries of both maps to a wave: one pass over the keys, V read once for both
//   diff_few    the same for up to 16 queries, the maps side by side in a product's columns
//   diff_join   the parts of split walks
//   diff_rows   per query row: log2 of both denominators, -delta_2, delta_2 - delta_1; per 16 rows the sum of -delta_2
//   diff_bwd    dK_1, dK_2 and dV of 128 keys, or dQ_1 and dQ_2 of 128 queries, to a workgroup of four waves; dlam
//   diff_sum    the parts of split walks
//
// The maps share V, dA and the product that forms dV: with D-wide maps and 2 D-wide values the gradient executes 28 D
// multiplications and additions a pair of query and key (scores and dA are formed for dK, dV and again for dQ, so that
// every sum stays in one wave's registers: no atomics, equal bits from equal calls); two calls of plain attention's
// gradients over 2 D-wide values would execute 40 D.
//
// The products are transposed as in attn_grad_tiles.h: a 32x32x16 accumulator hands each lane 16 rows of the side
// read from LDS for one own row, which is what the B operand of the next product takes, so that P and dS never leave
// registers; they are rounded to bf16 there, as the matrix products take them.  Scores, statistics and sums are fp32.
// That rounding puts 0.0020 of O's norm beside the 0.0017 of O's own (the maps' errors add up where what their outputs have
// in common cancels); a second product with what the rounding left would take a third to a half longer (2 samples of 15 heads
// 17776 tokens 6.56 -> 10.0 ms, one head of 4096 35 -> 49 us).  diff_few, which waits for memory, makes it.
//
// Bound by the matrix cores and vector issue under the power limit, as plain attention is: 2 samples of 15 heads, 17776
// tokens, D = 64 take 6.6 to 7.3 ms (1.00 to 1.11 PFLOP/s of 12 D; matrix cores busy 55 % at 1.64 to 1.73 GHz, 152 vector
// instructions and 24 matrix products a chunk of 32 x 32), their gradients 15.9 to 17.8 ms (0.96 to 1.07 PFLOP/s
// executed; 55 % at 1.70 to 1.80 GHz; waves wait 26 % of their time).  Two waves to a SIMD is what the registers
// allow: a wave holds 32 x 2 D sums for both maps (128 registers) forward, 32 x 4 D backward.  So the walk of dK and dV
// keeps its own values in LDS, and offsets packed; with spills of 90 registers it took twice the time.

#include <hip/hip_runtime.h>
#include <stdint.h>

#include <type_traits>

#include "attn_common.h"
#include "attn_grad_tiles.h"
#include "heads.h"

namespace rt {
namespace {

constexpr float kLog2e = 1.4426950408889634f;

// ---- rows in LDS ---------------------------------------------------------------------------

// 256-byte rows' 16 slots are swizzled by the row, so that 16 rows of a row read (one slot) and the four rows of half a
// transposed one (four slots) fall on different banks.
template <int D>
__device__ __forceinline__ int wide_swz(int r) {
    return Geo<D>::SWZ ? ((r & 3) << 2) | ((r >> 2) & 3) : 0;
}

// hides a lane constant's value, so that what derives from it is formed anew (one v_xad_u32 a read) instead of held in
// registers throughout a walk
__device__ __forceinline__ void fresh(int& x) { asm volatile("" : "+v"(x)); }

// A wave's reads of narrow rows (queries or keys, D wide) and of wide ones (values or output gradients, 2 D wide).
// 72-wide heads: narrow rows' last 8 elements are half a k-step of the scores; in the gradients those of both maps share
// the 16 rows of a 16x16x32 product, which wide rows' last 16 fill by themselves.
template <int D>
struct Reads {
    static constexpr int NB = 2 * D, WB = 4 * D;   // bytes of a row
    static constexpr int WS = 2 * D / 16;          // k-steps of a wide row
    static constexpr bool TAIL = D == 72, SWZ = Geo<D>::SWZ;

    lds_u8* lds;
    int lane, l32, hi;
    int n_rd, n_tr, n_t, w_rd, w_tr, w_t;

    __device__ __forceinline__ void init(lds_u8* smem) {
        lds = smem;
        lane = threadIdx.x & 63;
        l32 = lane & 31;
        hi = lane >> 5;
        // as in attn_grad_tiles.h: row l32, slot hi; transposed rows 4 hi + L / 4 (+ 8), which puts elements
        // 32 dt + 16 hi .. + 15 on a lane's 16 accumulators
        const int G4 = lane >> 4, L = lane & 15;
        const int r = 4 * hi + (L >> 2), d = 16 * (L & 1) + 8 * (G4 & 1) + 4 * ((L >> 1) & 1);
        n_rd = l32 * NB + ((hi ^ swz<D>(l32)) * 16);
        n_tr = r * NB + (((d >> 3) ^ swz<D>(r)) * 16) + (d & 7) * 2;
        w_rd = l32 * WB + ((hi ^ wide_swz<D>(l32)) * 16);
        w_tr = r * WB + (((d >> 3) ^ wide_swz<D>(r)) * 16) + (d & 7) * 2;
        const int tr = 16 * (G4 & 1) + 4 * (G4 >> 1) + (L >> 2);
        n_t = tr * NB + (64 + 4 * (L & 1)) * 2;
        w_t = tr * WB + (128 + 4 * (L & 3)) * 2;
    }
    // offsets two to a register, from which unpack() forms them anew: a walk that is short of registers holds three
    int pk[3];
    __device__ __forceinline__ void pack() {
        pk[0] = n_rd | n_tr << 16;
        pk[1] = w_rd | w_tr << 16;
        pk[2] = n_t | w_t << 16;
    }
    __device__ __forceinline__ void unpack() {
        fresh(pk[0]);
        fresh(pk[1]);
        fresh(pk[2]);
        n_rd = pk[0] & 0xffff;
        n_tr = pk[0] >> 16;
        w_rd = pk[1] & 0xffff;
        w_tr = pk[1] >> 16;
        n_t = pk[2] & 0xffff;
        w_t = pk[2] >> 16;
        fresh(lane);
        l32 = lane & 31;
        hi = lane >> 5;
    }
    __device__ __forceinline__ bf16x8 n_row(int base, int s) const {
        return *(const lds_bf16x8*)(lds + (SWZ ? (n_rd ^ (32 * s)) + base : n_rd + base + 32 * s));
    }
    __device__ __forceinline__ bf16x8 n_row_tail(int base, int zero) const {
        return *(const lds_bf16x8*)(lds + (hi ? zero : n_rd + base + 128));
    }
    __device__ __forceinline__ bf16x8 w_row(int base, int s) const {
        return *(const lds_bf16x8*)(lds + (SWZ ? (w_rd ^ (32 * s)) + base : w_rd + base + 32 * s));
    }
    static __device__ __forceinline__ bf16x8 tr_read(const lds_u8* p, const lds_u8* p8) {
        const bf16x4 v0 = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((lds_bf16x4*)p);
        const bf16x4 v1 = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((lds_bf16x4*)p8);
        return __builtin_shufflevector(v0, v1, 0, 1, 2, 3, 4, 5, 6, 7);
    }
    __device__ __forceinline__ bf16x8 n_col(int base, int dt, int ks) const {
        const lds_u8* p = lds + base + 16 * ks * NB;
        return SWZ ? tr_read(p + (n_tr ^ (64 * dt)), p + 8 * NB + (n_tr ^ (64 * dt) ^ 32))
                   : tr_read(p + n_tr + 64 * dt, p + 8 * NB + n_tr + 64 * dt);
    }
    __device__ __forceinline__ bf16x8 w_col(int base, int dt, int ks) const {
        const lds_u8* p = lds + base + 16 * ks * WB;
        return SWZ ? tr_read(p + (w_tr ^ (64 * dt)), p + 8 * WB + (w_tr ^ (64 * dt) ^ 32))
                   : tr_read(p + w_tr + 64 * dt, p + 8 * WB + w_tr + 64 * dt);
    }
    // narrow rows' last 8 elements, in rows 0 .. 7 of the product and again in 8 .. 15
    __device__ __forceinline__ bf16x8 n_col_tail(int base) const { return tr_read(lds + base + n_t, lds + base + n_t + 8 * NB); }
    __device__ __forceinline__ bf16x8 w_col_tail(int base) const { return tr_read(lds + base + w_t, lds + base + w_t + 8 * WB); }

    // rows row0 .. + 31 of x (zeros from row `end` on): lane holds row l32, elements 16 s + 8 hi ..
    template <int S>
    __device__ __forceinline__ void own_rows(const uint16_t* x, int bytes, int row0, int end, bf16x8 (&to)[S],
                                             bf16x8* tail) const {
        const __amdgpu_buffer_rsrc_t rs = __builtin_amdgcn_make_buffer_rsrc((void*)x, (short)0, end * bytes, 0x00020000);
        const int off = (row0 + l32) * bytes;
        auto load = [&](int o) { return __builtin_bit_cast(bf16x8, __builtin_amdgcn_raw_buffer_load_b128(rs, o, 0, 0)); };
#pragma unroll
        for (int s = 0; s < S; ++s) to[s] = load(off + 32 * s + 16 * hi);
        if (tail) *tail = load(hi ? kOob : off + 128);
    }
};

__device__ __forceinline__ bf16x8 op(const uint32_t (&p)[8], int ks) {
    return __builtin_bit_cast(bf16x8, u32x4{p[4 * ks], p[4 * ks + 1], p[4 * ks + 2], p[4 * ks + 3]});
}
// the two operands of 16 contraction rows become two of 32 for the halves of the own rows (attn_tiles.h)
__device__ __forceinline__ void halves(const uint32_t (&p)[8], uint32_t (&y)[8]) {
#pragma unroll
    for (int r = 0; r < 4; ++r) {
        auto s = __builtin_amdgcn_permlane16_swap(p[r], p[4 + r], false, false);
        y[r] = s[0];
        y[4 + r] = s[1];
    }
}
__device__ __forceinline__ f32x4 mma16(const bf16x8& x, const bf16x8& y, const f32x4& z) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(x, y, z, 0, 0, 0);
}

// Two stages of BS rows of both maps' narrow rows and of the wide ones (and, VALS, of four values a row), filled and
// read by W waves: the stage after the one in use is asked for when all waves are through the one before it.  Rows past
// the end read as zeros.
template <int D, int W, int BS, bool VALS>
struct DiffRing {
    static constexpr int NB = 2 * D, WB = 4 * D, NT = BS * NB, WT = BS * WB;
    static constexpr int WIDE = 2 * NT, VAL = WIDE + WT, STAGE = VAL + (VALS ? BS * 16 : 0);
    static constexpr int ZERO = 2 * STAGE, LDS = ZERO + 64;
    static_assert(W == 1 || W % 4 == 0, "whole fours of kilobytes");
    static_assert(!VALS || BS * 16 % 512 == 0, "values in one load");

    uint32_t lds0;
    int lane, w;
    int from_n[2], from_w, T64;
    i32x4 rs[3], vs;

    __device__ __forceinline__ void init(lds_u8* lds, const uint16_t* x1, const uint16_t* x2, const uint16_t* y, int rows) {
        lds0 = (uint32_t)(uintptr_t)lds;
        lane = threadIdx.x & 63;
        w = W == 1 ? 0 : __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
        rs[0] = buffer_rsrc(x1, rows * NB);
        rs[1] = buffer_rsrc(x2, rows * NB);
        rs[2] = buffer_rsrc(y, rows * WB);
        // (a wave of four or eight fills kilobytes of one place in four: the same offsets every time)
        from_n[0] = narrow_from(W > 1 ? w : 0);
        from_n[1] = W > 1 ? from_n[0] : narrow_from(1);
        from_w = wide_from(W > 1 ? w : 0);
        if (w == 0 && lane < 4) *(lds_u32x4*)(lds + ZERO + 16 * lane) = u32x4{};
    }
    __device__ __forceinline__ void init_values(const float* vals, int T64_) {
        T64 = T64_;
        vs = buffer_rsrc(vals, T64 * 16);
    }
    // a lane's source offset in kilobyte kb: 8 narrow rows, of odd and even ones, or 4 wide ones, of every fourth
    __device__ __forceinline__ int narrow_from(int kb) const {
        return Geo<D>::SWZ ? (lane >> 3) * NB + (((lane & 7) ^ swz<D>((lane >> 3) | ((kb & 1) << 3))) * 16) : lane * 16;
    }
    __device__ __forceinline__ int wide_from(int kb) const {
        return Geo<D>::SWZ ? (lane >> 4) * WB + (((lane & 15) ^ wide_swz<D>((lane >> 4) | ((kb & 3) << 2))) * 16) : lane * 16;
    }
    __device__ __forceinline__ int narrow_of(int n) const { return W > 1 ? from_n[0] : from_n[n & 1]; }
    __device__ __forceinline__ int wide_of(int n) const { return W > 1 || !Geo<D>::SWZ ? from_w : from_w ^ ((n & 3) * 16); }
    template <int SIZE, bool WD>
    __device__ __forceinline__ void fill(uint32_t dst, int at, const i32x4& r) const {
        constexpr int FULL = SIZE / (1024 * W), REST = (SIZE - FULL * 1024 * W) / (16 * W);
        static_assert(FULL * 1024 * W + REST * 16 * W == SIZE && (REST == 0 || !Geo<D>::SWZ), "even shares");
#pragma unroll
        for (int n = 0; n < FULL; ++n) {
            const int kb = n * W + w;
            dma16(__builtin_amdgcn_readfirstlane(dst + kb * 1024), (WD ? wide_of(n) : narrow_of(n)) + at + kb * 1024, r);
        }
        if (REST) {
            const int b = FULL * W * 1024 + w * REST * 16;
            if (lane < REST) dma16(__builtin_amdgcn_readfirstlane(dst + b), lane * 16 + at + b, r);
        }
    }
    __device__ __forceinline__ void load(int to, int row0) const {
        const uint32_t dst = lds0 + to;
        fill<NT, false>(dst, row0 * NB, rs[0]);
        fill<NT, false>(dst + NT, row0 * NB, rs[1]);
        fill<WT, true>(dst + WIDE, row0 * WB, rs[2]);
        if (VALS && w == 0 && lane < BS) {
            int l = lane;
            fresh(l);
            dma16(__builtin_amdgcn_readfirstlane(dst + VAL), (l / (BS / 4)) * T64 * 4 + (l % (BS / 4)) * 16 + row0 * 4, vs);
        }
    }
    // 32 rows from row0 on of the wave's own wide ones
    __device__ __forceinline__ void load_own(int to, int row0, const i32x4& r) const {
#pragma unroll
        for (int kb = 0; kb < 32 * WB / 1024; ++kb)
            dma16(__builtin_amdgcn_readfirstlane(lds0 + to + kb * 1024), wide_from(kb) + row0 * WB + kb * 1024, r);
    }
    // the stage asked for has landed, and every wave is through the one before it
    __device__ __forceinline__ void turn() const {
        wait_vm<0>();
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        if (W > 1) __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
    }
};

typedef __attribute__((address_space(3))) float lds_f32;
typedef __attribute__((address_space(3))) f32x4 lds_f32x4;

// Heads are taken in the order of head_of().  Where samples have numbers of keys of their own (a.by_len, for up to 64
// samples): those of the samples with most keys first, so that the longest walks begin first, and each XCD takes an eighth
// of every sample's tiles, in tiles that follow one another (9 heads of 7238 tokens and fewer keys 391 -> 264 us, gradients
// of 25 heads of 4789 760 -> 572).  Else heads of the samples in turn, an eighth of all tiles to an XCD.
__device__ __forceinline__ int keys_in(const DiffArgs& a, int n) { return n < 0 ? 0 : (n > a.Tk ? a.Tk : n); }
// by_len: the sample with the r-th most keys, and their number
__device__ __forceinline__ int sample_of(const DiffArgs& a, int r, int& keys) {
    const int lane = threadIdx.x & 63, mine = lane < a.B ? keys_in(a, a.k_lens[lane]) : 0;
    int rank = lane < a.B ? 0 : 64;
    for (int b = 0; b < a.B; ++b) {
        const int other = __builtin_amdgcn_readlane(mine, b);
        rank += other > mine || (other == mine && b < lane);
    }
    const int b = __builtin_ctzll(__builtin_amdgcn_ballot_w64(rank == r));
    keys = __builtin_amdgcn_readlane(mine, b);
    return b;
}
// The n-th head to be taken, b H + h, and its keys.
__device__ __forceinline__ int head_of(const DiffArgs& a, int n, int& keys) {
    if (a.by_len) {
        const int r = n / a.H;
        return sample_of(a, r, keys) * a.H + n - r * a.H;
    }
    const int h = n / a.B, b = n - h * a.B;
    keys = a.k_lens ? keys_in(a, a.k_lens[b]) : a.Tk;
    return b * a.H + h;
}
// Workgroups of an XCD for n items, and the item of workgroup g, or -1: an XCD has every eighth workgroup.
__host__ __device__ inline int per_xcd(const DiffArgs& a, int n) {
    return a.by_len ? a.B * ((n / a.B + 7) / 8) : (n + 7) / 8;
}
__device__ __forceinline__ int eighth(int x, int n) { return (int)((int64_t)x * n / 8); }
__device__ __forceinline__ int item_of(const DiffArgs& a, int g, int n) {
    int x = g & 7, j = g >> 3, m = n, before = 0;
    if (a.by_len) {
        m = n / a.B;
        const int per = (m + 7) / 8, r = j / per;
        x = (x + r) & 7;  // what a sample's tiles leave of eight is another XCD's each time
        j -= r * per;
        before = r * m;
    }
    j += eighth(x, m);
    return j < eighth(x + 1, m) ? before + j : -1;
}
// The same (by_len) for tiles of keys, n_tile a head in parts of `split`; also the item's head and keys.  Those past a
// sample's keys have no work: an XCD takes an eighth of the others and then an eighth of these, so that a head over many
// XCDs leaves none of them idle (gradients of a head of 4000 tokens and one of 1550 keys 126 -> 84 us, of 45 heads of 700
// 52 -> 46).
__host__ __device__ inline int per_xcd_k(const DiffArgs& a, int n) { return per_xcd(a, n) + (a.by_len ? a.B : 0); }
__device__ __forceinline__ int item_of_k(const DiffArgs& a, int g, int n, int n_tile, int split, int& bh, int& keys) {
    const int m = n / a.B, per = (m + 7) / 8 + 1, r = (g >> 3) / per, x = (g + r) & 7;
    int j = (g >> 3) - r * per;
    const int b = sample_of(a, r, keys);
    int first = 0, tiles = (keys + kDiffRows - 1) / kDiffRows, of = a.H * tiles * split;
    if (const int here = eighth(x + 1, of) - eighth(x, of); j >= here) {
        j -= here;
        first = tiles;
        tiles = n_tile - tiles;
        of = a.H * tiles * split;
    }
    j += eighth(x, of);
    if (j >= eighth(x + 1, of)) return -1;
    const int h = j / (tiles * split);
    bh = b * a.H + h;
    return r * m + (h * n_tile + first) * split + j - h * tiles * split;
}

// ---- forward -------------------------------------------------------------------------------

// A running max further out than this has a product with c2 whose rounding shows in an exponent (at 2^40 it makes 0 or
// infinity of the largest probability): these are then formed by differences of scores, exact where they matter.  In every
// chunk that would be an instruction more for each; the test takes 0 to 1.5 % (2 samples of 15 heads, 17776 tokens 6.56 ->
// 6.59 ms, one head of 4096 35.8 -> 36.3 us).  diff_few, which waits for memory, always forms them so (27.3 -> 27.7 us, 15
// tokens over 17776 keys).
constexpr float kFar = 65536.0f;
constexpr float kLowest = -3.402823466e38f;  // of a running max; finite: a chunk without keys gives p = 0, not NaN

// the part of a tile's rows for which a sample has no keys: its statistics alone, by which diff_join leaves the sums out
template <int D>
__device__ __forceinline__ void empty_part(const DiffArgs& a, int bh, int part, int row0, int rows) {
    const int map = threadIdx.x & 1, row = row0 + (threadIdx.x >> 1);
    if ((int)threadIdx.x >= 2 * rows || row >= a.Tq) return;
    float* x = a.part + (size_t)a.n_bh * a.split * 2 * a.Tq * (2 * D) + ((((size_t)bh * a.split + part) * 2 + map) * a.Tq + row) * 3;
    x[0] = kLowest;
    x[1] = 0.f;
    x[2] = -INFINITY;
}

// A workgroup of four waves takes 32 queries to a wave, which share a ring of keys and values; or (KEYS, where there are
// few tiles) 32 queries in all, the waves every fourth 32 keys each from rings of their own, and joins their sums in LDS.
// SPLIT: a part of the keys, whose sums against their own running max go to a.part ([tile's head][part][map][query][2 D],
// then [..][3] of the max in score units, the sum and the true max).
template <int D, bool KEYS, bool STATS, bool SPLIT>
__global__ __launch_bounds__(KEYS ? 512 : 256) __attribute__((amdgpu_waves_per_eu(2, 2))) void
diff_fwd(DiffArgs a, int n_items) {
    constexpr int BS = KEYS ? 32 : 64, STEP = KEYS ? 4 : 1;  // keys of a stage; stages from one of a wave to its next
    using R = DiffRing<D, KEYS ? 1 : 4, BS, false>;
    constexpr int NB = R::NB, WB = R::WB;
    constexpr bool TAIL = D == 72;
    constexpr int STAT = 4 * R::LDS;  // KEYS: [wave][map][query] of the running max, the sum and the true max
    __shared__ __attribute__((aligned(1024))) unsigned char smem[KEYS ? STAT + 4 * 2 * 32 * 12 : R::LDS];
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    lds_u8* const lds = (lds_u8*)smem + (KEYS ? wave * R::LDS : 0);

    int item = item_of(a, blockIdx.x, n_items), part = 0;
    if (item < 0) return;
    if (SPLIT) {
        part = item % a.split;
        item /= a.split;
    }
    constexpr int ROWS = KEYS ? 32 : kDiffRows;
    const int n_tile = (a.Tq + ROWS - 1) / ROWS, head = item / n_tile;
    int keys;
    const int bh = head_of(a, head, keys);
    const int row0 = (item - head * n_tile) * ROWS + (KEYS ? 0 : wave * 32);
    const int n_st = (keys + BS - 1) / BS;
    // parts are as long for every sample, so that those of short ones cost little
    const int per = SPLIT ? ((a.Tk + BS - 1) / BS + a.split - 1) / a.split : n_st;
    const int first_stage = part * per + (KEYS ? wave : 0), end_stage = SPLIT && part * per + per < n_st ? part * per + per : n_st;
    if (SPLIT && part * per >= n_st) {
        empty_part<D>(a, bh, part, (item - head * n_tile) * ROWS, ROWS);
        return;
    }

    R ring;
    ring.init(lds, a.k + (size_t)(2 * bh) * a.Tk * D, a.k + (size_t)(2 * bh + 1) * a.Tk * D, a.v + (size_t)bh * a.Tk * (2 * D), keys);
    ring.load(0, first_stage * BS);
    Reads<D> rd;
    rd.init(lds);
    rd.pack();
    bf16x8 q[2][4], q_tail[2];
#pragma unroll
    for (int i = 0; i < 2; ++i)
        rd.own_rows(a.q + (size_t)(2 * bh + i) * a.Tq * D, NB, row0, a.Tq, q[i], TAIL ? &q_tail[i] : nullptr);

    f32x16 acc[2][4];
    f32x4 tacc[2][2];
    float m_run[2], m_top[2], l_run[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
#pragma unroll
        for (int d = 0; d < 4; ++d) acc[i][d] = f32x16{};
        tacc[i][0] = tacc[i][1] = f32x4{};
        m_run[i] = kLowest;
        m_top[i] = -INFINITY;
        l_run[i] = 0.f;
    }
    // a value of each query as the tails' accumulators hold them: query 16 h + lane % 16
    auto tail_bcast = [&](float x, int h) {
        return __int_as_float(__builtin_amdgcn_ds_bpermute((16 * h + (rd.lane & 15)) << 2, __float_as_int(x)));
    };
    const float c2 = a.scale_log2;
    auto stage = [&](auto odd, int s) {
        constexpr int st = decltype(odd)::value ? R::STAGE : 0;
        ring.turn();
        ring.load(R::STAGE - st, (s + STEP) * BS);
        if (row0 < a.Tq) {
#pragma unroll
            for (int h = 0; h < BS / 32; ++h) {
                const int first = s * BS + 32 * h, cv = st + R::WIDE + 32 * h * WB;
                if (D == 72) rd.unpack();
                const int cx = st + 32 * h * NB;
                auto mask = [&](f32x16& sc) {
                    if (first + 32 > keys) {
                        const int lim = keys - first - 4 * rd.hi;
#pragma unroll
                        for (int x = 0; x < 16; ++x)
                            if (8 * (x >> 2) + (x & 3) >= lim) sc[x] = -INFINITY;
                    }
                };
                uint32_t pk[2][8];
                // Probabilities of a map against its running max, a matrix product of the other's between two pairs of
                // them; should one pass 2^24, the max moves and they are formed again, as where it lies far out.
                auto soft = [&](int i, const f32x16& sc, auto&& product) {
                    float top = -INFINITY;
                    auto form = [&](auto far, auto&& between) {
                        const float mc = m_run[i] * c2;
                        auto p = [&](float s) {
                            return __builtin_amdgcn_exp2f(decltype(far)::value ? (s - m_run[i]) * c2 : __builtin_fmaf(s, c2, -mc));
                        };
                        float sum[2] = {0.f, 0.f};
#pragma unroll
                        for (int x = 0; x < 16; x += 2) {
                            const float e0 = p(sc[x]), e1 = p(sc[x + 1]);
                            sum[(x >> 1) & 1] += e0 + e1;
                            pk[i][x / 2] = pack_bf16(e0, e1);
                            between(x);
                        }
                        return sum[0] + sum[1];
                    };
                    float sum = form(std::integral_constant<bool, false>{}, [&](int x) {
                        top = fmaxf(fmaxf(top, sc[x]), sc[x + 1]);
                        __builtin_amdgcn_sched_barrier(0);
                        product(x / 2);
                        __builtin_amdgcn_sched_barrier(0);
                    });
                    if (STATS) m_top[i] = fmaxf(m_top[i], top);
                    if (__builtin_amdgcn_ballot_w64(top - m_run[i] > a.move) | __builtin_amdgcn_ballot_w64(fabsf(m_run[i]) > kFar)) {
                        const float to = fmaxf(m_run[i], pair_max(top));
                        const float alpha = __builtin_amdgcn_exp2f((m_run[i] - to) * c2);
                        m_run[i] = to;
                        l_run[i] *= alpha;
#pragma unroll
                        for (int d = 0; d < 4; ++d) acc[i][d] *= alpha;
                        if (TAIL) {
                            tacc[i][0] *= tail_bcast(alpha, 0);
                            tacc[i][1] *= tail_bcast(alpha, 1);
                        }
                        sum = form(std::integral_constant<bool, true>{}, [](int) {});
                    }
                    l_run[i] += sum;
                };
                f32x16 s0 = {}, s1 = {};
                bf16x8 k1[4], v[8];
#pragma unroll
                for (int k = 0; k < 4; ++k) s0 = mma(rd.n_row(cx, k), q[0][k], s0);
#pragma unroll
                for (int k = 0; k < 4; ++k) k1[k] = rd.n_row(cx + R::NT, k);
                if (TAIL) s0 = mma(rd.n_row_tail(cx, R::ZERO), q_tail[0], s0);
                mask(s0);
                soft(0, s0, [&](int p) {
                    if (p % 2 == 0) s1 = mma(k1[p / 2], q[1][p / 2], s1);
                });
                if (TAIL) s1 = mma(rd.n_row_tail(cx + R::NT, R::ZERO), q_tail[1], s1);
                mask(s1);
                auto v_at = [&](int p) { return rd.w_col(cv, p & 3, p >> 2); };
#pragma unroll
                for (int p = 0; p < 8; ++p)
                    if (!TAIL || p < 2) v[p] = v_at(p);
                soft(1, s1, [&](int p) {
                    acc[0][p & 3] = mma(TAIL ? v[p & 1] : v[p], op(pk[0], p >> 2), acc[0][p & 3]);
                    if (TAIL && p < 6) v[p & 1] = v_at(p + 2);
                });
#pragma unroll
                for (int p = 0; p < 8; ++p) acc[1][p & 3] = mma(TAIL ? v_at(p) : v[p], op(pk[1], p >> 2), acc[1][p & 3]);
                if (TAIL) {
                    const bf16x8 v = rd.w_col_tail(cv);
#pragma unroll
                    for (int i = 0; i < 2; ++i) {
                        uint32_t y[8];
                        halves(pk[i], y);
                        tacc[i][0] = mma16(v, op(y, 0), tacc[i][0]);
                        tacc[i][1] = mma16(v, op(y, 1), tacc[i][1]);
                    }
                }
            }
        }
    };
    for (int s = first_stage; s < end_stage; s += 2 * STEP) {
        stage(std::integral_constant<bool, false>{}, s);
        if (s + STEP < end_stage) stage(std::integral_constant<bool, true>{}, s + STEP);
    }
    wait_vm<0>();  // nothing may land in LDS after the workgroup has ended
    if (row0 >= a.Tq) return;
    const int row = row0 + rd.l32;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        l_run[i] = pair_sum(l_run[i]);
        if (STATS) m_top[i] = pair_max(m_top[i]);
    }
    constexpr int TILES = KEYS ? 1 : 4;  // of 32 elements that a wave writes, from `col0` on
    const int col0 = KEYS ? 32 * wave : 0;
    const bool lead = !KEYS || wave == 0;
    if constexpr (KEYS) {
        lds_u8* const all = (lds_u8*)smem;
        auto stat = [&](int w, int i) { return (lds_f32*)(all + STAT) + ((w * 2 + i) * 32 + rd.l32) * 3; };
        if (rd.hi == 0) {
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                stat(wave, i)[0] = m_run[i];
                stat(wave, i)[1] = l_run[i];
                stat(wave, i)[2] = m_top[i];
            }
        }
        __syncthreads();
        // each wave's sums against the largest running max, in its own ring's place: [map][element tile][u][lane]
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            float m = -INFINITY, l = 0.f, top = -INFINITY;
#pragma unroll
            for (int w = 0; w < 4; ++w) {
                m = fmaxf(m, stat(w, i)[0]);
                top = fmaxf(top, stat(w, i)[2]);
            }
#pragma unroll
            for (int w = 0; w < 4; ++w) l = __builtin_fmaf(__builtin_amdgcn_exp2f((stat(w, i)[0] - m) * c2), stat(w, i)[1], l);
            const float f = __builtin_amdgcn_exp2f((m_run[i] - m) * c2);
#pragma unroll
            for (int d = 0; d < 4; ++d)
#pragma unroll
                for (int u = 0; u < 4; ++u)
                    *(lds_f32x4*)(lds + ((i * 4 + d) * 4 + u) * 1024 + rd.lane * 16) =
                        f32x4{acc[i][d][4 * u] * f, acc[i][d][4 * u + 1] * f, acc[i][d][4 * u + 2] * f, acc[i][d][4 * u + 3] * f};
            if (TAIL) {
#pragma unroll
                for (int h = 0; h < 2; ++h) *(lds_f32x4*)(lds + 32768 + (i * 2 + h) * 1024 + rd.lane * 16) = tacc[i][h] * tail_bcast(f, h);
            }
            m_run[i] = m;
            l_run[i] = l;
            m_top[i] = top;
        }
        __syncthreads();
#pragma unroll
        for (int i = 0; i < 2; ++i) {
#pragma unroll
            for (int u = 0; u < 4; ++u) {
                f32x4 x = {};
#pragma unroll
                for (int w = 0; w < 4; ++w) x += *(const lds_f32x4*)(all + w * R::LDS + ((i * 4 + wave) * 4 + u) * 1024 + rd.lane * 16);
#pragma unroll
                for (int e = 0; e < 4; ++e) acc[i][0][4 * u + e] = x[e];
            }
            if (TAIL && wave == 0) {
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    tacc[i][h] = f32x4{};
#pragma unroll
                    for (int w = 0; w < 4; ++w) tacc[i][h] += *(const lds_f32x4*)(all + w * R::LDS + 32768 + (i * 2 + h) * 1024 + rd.lane * 16);
                }
            }
        }
    }
    if (SPLIT) {
        const size_t n_part = (size_t)a.n_bh * a.split, at = (size_t)bh * a.split + part;
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            float* o = a.part + (at * 2 + i) * a.Tq * (2 * D);
            if (row < a.Tq) {
#pragma unroll
                for (int d = 0; d < TILES; ++d)
#pragma unroll
                    for (int u = 0; u < 4; ++u)
                        *reinterpret_cast<f32x4*>(o + (size_t)row * (2 * D) + col0 + 32 * d + 16 * rd.hi + 4 * u) =
                            f32x4{acc[i][d][4 * u], acc[i][d][4 * u + 1], acc[i][d][4 * u + 2], acc[i][d][4 * u + 3]};
                if (lead && rd.hi == 0) {
                    float* x = a.part + n_part * 2 * a.Tq * (2 * D) + ((at * 2 + i) * a.Tq + row) * 3;
                    x[0] = m_run[i];
                    x[1] = l_run[i];
                    x[2] = STATS ? m_top[i] : 0.f;
                }
            }
            if (TAIL && lead) {
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const int r = row0 + 16 * h + (rd.lane & 15);
                    if (r < a.Tq) *reinterpret_cast<f32x4*>(o + (size_t)r * (2 * D) + 128 + 4 * (rd.lane >> 4)) = tacc[i][h];
                }
            }
        }
        return;
    }
    float inv[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        inv[i] = l_run[i] == 0.f ? 0.f : 1.0f / l_run[i];  // no keys: 0
        if (STATS && lead && rd.hi == 0 && row < a.Tq) {
            const size_t at = (size_t)(2 * bh + i) * a.Tq + row;
            a.row_max[at] = m_top[i] * a.scale_nat;
            a.row_sum[at] = l_run[i] == 0.f ? 0.f : l_run[i] * __builtin_amdgcn_exp2f((m_run[i] - m_top[i]) * c2);
        }
    }
    const float lam = a.lam[(bh % a.H) * a.lam_step];
    uint16_t* const o = a.o + (size_t)bh * a.Tq * (2 * D);
    uint16_t* const o2 = STATS ? a.o2 + (size_t)bh * a.Tq * (2 * D) : nullptr;
    if (row < a.Tq) {
#pragma unroll
        for (int d = 0; d < TILES; ++d)
#pragma unroll
            for (int u = 0; u < 2; ++u) {
                uint32_t x[4], y[4];
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const int j = 8 * u + 2 * e;
                    const float b0 = acc[1][d][j] * inv[1], b1 = acc[1][d][j + 1] * inv[1];
                    x[e] = pack_bf16(__builtin_fmaf(-lam, b0, acc[0][d][j] * inv[0]), __builtin_fmaf(-lam, b1, acc[0][d][j + 1] * inv[0]));
                    y[e] = pack_bf16(b0, b1);
                }
                const size_t at = (size_t)row * (2 * D) + col0 + 32 * d + 16 * rd.hi + 8 * u;
                *reinterpret_cast<u32x4*>(o + at) = u32x4{x[0], x[1], x[2], x[3]};
                if (STATS) *reinterpret_cast<u32x4*>(o2 + at) = u32x4{y[0], y[1], y[2], y[3]};
            }
    }
    if (TAIL && lead) {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const float i0 = tail_bcast(inv[0], h), i1 = tail_bcast(inv[1], h);
            const int r = row0 + 16 * h + (rd.lane & 15);
            if (r < a.Tq) {
                const size_t at = (size_t)r * (2 * D) + 128 + 4 * (rd.lane >> 4);
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    const float b0 = tacc[1][h][2 * e] * i1, b1 = tacc[1][h][2 * e + 1] * i1;
                    reinterpret_cast<uint32_t*>(o + at)[e] = pack_bf16(__builtin_fmaf(-lam, b0, tacc[0][h][2 * e] * i0), __builtin_fmaf(-lam, b1, tacc[0][h][2 * e + 1] * i0));
                    if (STATS) reinterpret_cast<uint32_t*>(o2 + at)[e] = pack_bf16(b0, b1);
                }
            }
        }
    }
}

// Up to 16 queries of a head, as diff_fwd's KEYS: map 1's in columns 0 .. 15 of the 32x32 products, map 2's in the others,
// so that a chunk takes one softmax and V's products once (24 matrix products and 16 exponentials a lane, where two maps
// apart would make 40 and 32).  Probabilities go into the products in two bf16 pieces, which leaves the error to O's own
// rounding (8 x 15 tokens over up to 8192 keys 35.0 -> 36.2 us, 53.6 either way with keys and values cold).  The maps'
// scores come out of accumulators of their own, of which a lane takes its map's: one for both, with zeros for the other
// map's queries, would give 0 times a key that is not finite in one map to the other (36.3 us for 36.7).
template <int D, bool STATS, bool SPLIT>
__global__ __launch_bounds__(512) __attribute__((amdgpu_waves_per_eu(2, 2))) void diff_few(DiffArgs a, int n_items) {
    constexpr int BS = 32, STEP = 4;
    using R = DiffRing<D, 1, BS, false>;
    constexpr int NB = R::NB;
    constexpr bool TAIL = D == 72;
    constexpr int STAT = 4 * R::LDS;  // [wave][column] of the running max, the sum and the true max
    __shared__ __attribute__((aligned(1024))) unsigned char smem[STAT + 4 * 32 * 12];
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    lds_u8* const all = (lds_u8*)smem;
    lds_u8* const lds = all + wave * R::LDS;

    int item = item_of(a, blockIdx.x, n_items), part = 0;
    if (item < 0) return;
    if (SPLIT) {
        part = item % a.split;
        item /= a.split;
    }
    int keys;
    const int bh = head_of(a, item, keys);
    const int n_st = (keys + BS - 1) / BS;
    const int per = SPLIT ? ((a.Tk + BS - 1) / BS + a.split - 1) / a.split : n_st;
    const int first_stage = part * per + wave, end_stage = SPLIT && part * per + per < n_st ? part * per + per : n_st;
    if (SPLIT && part * per >= n_st) {
        empty_part<D>(a, bh, part, 0, 16);
        return;
    }

    R ring;
    ring.init(lds, a.k + (size_t)(2 * bh) * a.Tk * D, a.k + (size_t)(2 * bh + 1) * a.Tk * D, a.v + (size_t)bh * a.Tk * (2 * D), keys);
    ring.load(0, first_stage * BS);
    Reads<D> rd;
    rd.init(lds);
    const int map = rd.l32 >> 4, row = rd.l32 & 15;
    bf16x8 q[2][4], q_tail[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const __amdgpu_buffer_rsrc_t rs = __builtin_amdgcn_make_buffer_rsrc((void*)(a.q + (size_t)(2 * bh + i) * a.Tq * D), (short)0, a.Tq * NB, 0x00020000);
        const int off = map == i ? row * NB : kOob;
        auto load = [&](int o) { return __builtin_bit_cast(bf16x8, __builtin_amdgcn_raw_buffer_load_b128(rs, o, 0, 0)); };
#pragma unroll
        for (int k = 0; k < 4; ++k) q[i][k] = load(off + 32 * k + 16 * rd.hi);
        if (TAIL) q_tail[i] = load(rd.hi ? kOob : off + 128);
    }
    f32x16 acc[4];
    f32x4 tacc[2];  // of map 1 and of map 2
#pragma unroll
    for (int d = 0; d < 4; ++d) acc[d] = f32x16{};
    tacc[0] = tacc[1] = f32x4{};
    float m_run = kLowest, m_top = -INFINITY, l_run = 0.f;
    // a value of each column as the tails' accumulators hold them: query lane % 16 of map i
    auto tail_bcast = [&](float x, int i) { return __int_as_float(__builtin_amdgcn_ds_bpermute((16 * i + (rd.lane & 15)) << 2, __float_as_int(x))); };
    const float c2 = a.scale_log2;
    int st = 0;
    for (int s = first_stage; s < end_stage; s += STEP) {
        ring.turn();
        ring.load(R::STAGE - st, (s + STEP) * BS);
        const int cv = st + R::WIDE;
        f32x16 both[2] = {};
#pragma unroll
        for (int i = 0; i < 2; ++i) {
#pragma unroll
            for (int k = 0; k < 4; ++k) both[i] = mma(rd.n_row(st + i * R::NT, k), q[i][k], both[i]);
            if (TAIL) both[i] = mma(rd.n_row_tail(st + i * R::NT, R::ZERO), q_tail[i], both[i]);
        }
        f32x16 sc;
#pragma unroll
        for (int x = 0; x < 16; ++x) sc[x] = map ? both[1][x] : both[0][x];
        if ((s + 1) * BS > keys) {
            const int lim = keys - s * BS - 4 * rd.hi;
#pragma unroll
            for (int x = 0; x < 16; ++x)
                if (8 * (x >> 2) + (x & 3) >= lim) sc[x] = -INFINITY;
        }
        float top = fmaxf(fmaxf(sc[0], sc[1]), sc[2]);
#pragma unroll
        for (int x = 3; x < 15; x += 2) top = fmaxf(fmaxf(top, sc[x]), sc[x + 1]);
        top = fmaxf(top, sc[15]);
        if (STATS) m_top = fmaxf(m_top, top);
        if (__builtin_amdgcn_ballot_w64(top - m_run > a.move)) {
            const float to = fmaxf(m_run, pair_max(top));
            const float alpha = __builtin_amdgcn_exp2f((m_run - to) * c2);
            m_run = to;
            l_run *= alpha;
#pragma unroll
            for (int d = 0; d < 4; ++d) acc[d] *= alpha;
            if (TAIL) {
                tacc[0] *= tail_bcast(alpha, 0);
                tacc[1] *= tail_bcast(alpha, 1);
            }
        }
        float sum[2] = {0.f, 0.f};
        uint32_t pk[8], rest[8];
#pragma unroll
        for (int x = 0; x < 16; x += 2) {
            const float e0 = __builtin_amdgcn_exp2f((sc[x] - m_run) * c2), e1 = __builtin_amdgcn_exp2f((sc[x + 1] - m_run) * c2);
            sum[(x >> 1) & 1] += e0 + e1;
            pk[x / 2] = pack_bf16(e0, e1);
            rest[x / 2] = pack_bf16(e0 - lo_f(pk[x / 2]), e1 - hi_f(pk[x / 2]));
        }
        l_run += sum[0] + sum[1];
#pragma unroll
        for (int p = 0; p < 8; ++p) {
            const bf16x8 v = rd.w_col(cv, p & 3, p >> 2);
            acc[p & 3] = mma(v, op(pk, p >> 2), acc[p & 3]);
            acc[p & 3] = mma(v, op(rest, p >> 2), acc[p & 3]);
        }
        if (TAIL) {
            const bf16x8 v = rd.w_col_tail(cv);
            uint32_t y[8];
            halves(pk, y);
            tacc[0] = mma16(v, op(y, 0), tacc[0]);
            tacc[1] = mma16(v, op(y, 1), tacc[1]);
            halves(rest, y);
            tacc[0] = mma16(v, op(y, 0), tacc[0]);
            tacc[1] = mma16(v, op(y, 1), tacc[1]);
        }
        st = R::STAGE - st;
    }
    wait_vm<0>();  // nothing may land in LDS after the workgroup has ended

    // the waves' sums against the largest running max, each in its own ring's place, then a tile of 32 elements to a wave
    l_run = pair_sum(l_run);
    if (STATS) m_top = pair_max(m_top);
    auto stat = [&](int w) { return (lds_f32*)(all + STAT) + (w * 32 + rd.l32) * 3; };
    if (rd.hi == 0) {
        stat(wave)[0] = m_run;
        stat(wave)[1] = l_run;
        stat(wave)[2] = m_top;
    }
    __syncthreads();
    float m = -INFINITY, l = 0.f;
    m_top = -INFINITY;
#pragma unroll
    for (int w = 0; w < 4; ++w) {
        m = fmaxf(m, stat(w)[0]);
        m_top = fmaxf(m_top, stat(w)[2]);
    }
#pragma unroll
    for (int w = 0; w < 4; ++w) l = __builtin_fmaf(__builtin_amdgcn_exp2f((stat(w)[0] - m) * c2), stat(w)[1], l);
    const float f = __builtin_amdgcn_exp2f((m_run - m) * c2);
#pragma unroll
    for (int d = 0; d < 4; ++d)
#pragma unroll
        for (int u = 0; u < 4; ++u)
            *(lds_f32x4*)(lds + (d * 4 + u) * 1024 + rd.lane * 16) =
                f32x4{acc[d][4 * u] * f, acc[d][4 * u + 1] * f, acc[d][4 * u + 2] * f, acc[d][4 * u + 3] * f};
    if (TAIL) {
#pragma unroll
        for (int i = 0; i < 2; ++i) *(lds_f32x4*)(lds + 16384 + i * 1024 + rd.lane * 16) = tacc[i] * tail_bcast(f, i);
    }
    __syncthreads();
    float inv = l == 0.f ? 0.f : 1.0f / l;  // no keys: 0
    f32x4 x[4];
#pragma unroll
    for (int u = 0; u < 4; ++u) {
        x[u] = f32x4{};
#pragma unroll
        for (int w = 0; w < 4; ++w) x[u] += *(const lds_f32x4*)(all + w * R::LDS + (wave * 4 + u) * 1024 + rd.lane * 16);
    }
    if (TAIL && wave == 0) {
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            tacc[i] = f32x4{};
#pragma unroll
            for (int w = 0; w < 4; ++w) tacc[i] += *(const lds_f32x4*)(all + w * R::LDS + 16384 + i * 1024 + rd.lane * 16);
        }
    }
    const int col = 32 * wave + 16 * rd.hi;
    if (SPLIT) {
        if (row < a.Tq) {
            const size_t at = ((size_t)bh * a.split + part) * 2 + map;
#pragma unroll
            for (int u = 0; u < 4; ++u) *reinterpret_cast<f32x4*>(a.part + (at * a.Tq + row) * (2 * D) + col + 4 * u) = x[u];
            if (wave == 0 && rd.hi == 0) {
                float* y = a.part + (size_t)a.n_bh * a.split * 2 * a.Tq * (2 * D) + (at * a.Tq + row) * 3;
                y[0] = m;
                y[1] = l;
                y[2] = STATS ? m_top : 0.f;
            }
        }
        if (TAIL && wave == 0 && (rd.lane & 15) < a.Tq) {
#pragma unroll
            for (int i = 0; i < 2; ++i)
                *reinterpret_cast<f32x4*>(a.part + ((((size_t)bh * a.split + part) * 2 + i) * a.Tq + (rd.lane & 15)) * (2 * D) + 128 + 4 * (rd.lane >> 4)) = tacc[i];
        }
        return;
    }
    if (STATS && wave == 0 && rd.hi == 0 && row < a.Tq) {
        const size_t at = (size_t)(2 * bh + map) * a.Tq + row;
        a.row_max[at] = m_top * a.scale_nat;
        a.row_sum[at] = l == 0.f ? 0.f : l * __builtin_amdgcn_exp2f((m - m_top) * c2);
    }
    const float lam = a.lam[(bh % a.H) * a.lam_step];
    // the maps' values of a query from the lanes of both: map 1's lanes write o, map 2's o2
    uint32_t out[8];
#pragma unroll
    for (int u = 0; u < 4; ++u) {
        float y[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            const uint32_t v = __float_as_uint(x[u][e] * inv);
            auto r = __builtin_amdgcn_permlane16_swap(v, v, false, false);
            y[e] = map ? __uint_as_float(r[1]) : __builtin_fmaf(-lam, __uint_as_float(r[1]), __uint_as_float(r[0]));
        }
        out[2 * u] = pack_bf16(y[0], y[1]);
        out[2 * u + 1] = pack_bf16(y[2], y[3]);
    }
    if (row < a.Tq && (STATS || map == 0)) {
        uint16_t* const to = (map ? a.o2 : a.o) + ((size_t)bh * a.Tq + row) * (2 * D) + col;
        *reinterpret_cast<u32x4*>(to) = u32x4{out[0], out[1], out[2], out[3]};
        *reinterpret_cast<u32x4*>(to + 8) = u32x4{out[4], out[5], out[6], out[7]};
    }
    if (TAIL && wave == 0) {
        const float i0 = tail_bcast(inv, 0), i1 = tail_bcast(inv, 1);
        if ((rd.lane & 15) < a.Tq) {
            const size_t at = ((size_t)bh * a.Tq + (rd.lane & 15)) * (2 * D) + 128 + 4 * (rd.lane >> 4);
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                const float b0 = tacc[1][2 * e] * i1, b1 = tacc[1][2 * e + 1] * i1;
                reinterpret_cast<uint32_t*>(a.o + at)[e] = pack_bf16(__builtin_fmaf(-lam, b0, tacc[0][2 * e] * i0), __builtin_fmaf(-lam, b1, tacc[0][2 * e + 1] * i0));
                if (STATS) reinterpret_cast<uint32_t*>(a.o2 + at)[e] = pack_bf16(b0, b1);
            }
        }
    }
}

// A query row of split walks to a workgroup: D / 2 threads take 4 elements each of every EACH-th part
template <int D>
__global__ __launch_bounds__(256) void diff_join(DiffArgs a) {
    constexpr int LANES = D / 2, EACH = 256 / LANES;
    __shared__ float stat[2][kDiffParts][3];
    __shared__ f32x4 sums[2][EACH][LANES];
    const int64_t bh = blockIdx.x / a.Tq, row = blockIdx.x - bh * a.Tq;
    auto at = [&](int map, int p) { return ((bh * a.split + p) * 2 + map) * (size_t)a.Tq + row; };
    if ((int)threadIdx.x < 2 * a.split) {
        const int map = threadIdx.x & 1, p = threadIdx.x >> 1;
        const float* x = a.part + (size_t)a.n_bh * a.split * 2 * a.Tq * (2 * D) + at(map, p) * 3;
#pragma unroll
        for (int i = 0; i < 3; ++i) stat[map][p][i] = x[i];
    }
    __syncthreads();
    const int g = threadIdx.x / LANES, j = threadIdx.x - g * LANES;
    float m[2], top[2], l[2];
#pragma unroll
    for (int map = 0; map < 2; ++map) {
        m[map] = top[map] = -INFINITY;
        l[map] = 0.f;
        for (int p = 0; p < a.split; ++p) {
            m[map] = fmaxf(m[map], stat[map][p][0]);
            top[map] = fmaxf(top[map], stat[map][p][2]);
        }
        auto factor = [&](int p) { return __builtin_amdgcn_exp2f((stat[map][p][0] - m[map]) * a.scale_log2); };
        for (int p = 0; p < a.split; ++p) l[map] = __builtin_fmaf(factor(p), stat[map][p][1], l[map]);
        if (g < EACH) {
            f32x4 s = {};
#pragma unroll 4
            for (int p = g; p < a.split; p += EACH)
                if (stat[map][p][1] != 0.f) s += *reinterpret_cast<const f32x4*>(a.part + at(map, p) * (2 * D) + 4 * j) * factor(p);
            sums[map][g][j] = s;
        }
    }
    __syncthreads();
    if (g > 0) return;
    f32x4 o[2];
#pragma unroll
    for (int map = 0; map < 2; ++map) {
        o[map] = f32x4{};
#pragma unroll
        for (int i = 0; i < EACH; ++i) o[map] += sums[map][i][j];
        o[map] *= l[map] == 0.f ? 0.f : 1.0f / l[map];
        if (a.row_max && j == 0) {
            const size_t to = (size_t)(2 * bh + map) * a.Tq + row;
            a.row_max[to] = top[map] * a.scale_nat;
            a.row_sum[to] = l[map] == 0.f ? 0.f : l[map] * __builtin_amdgcn_exp2f((m[map] - top[map]) * a.scale_log2);
        }
    }
    const f32x4 d = o[0] - o[1] * a.lam[(bh % a.H) * a.lam_step];
    const size_t to = (size_t)blockIdx.x * (2 * D) + 4 * j;
    reinterpret_cast<uint32_t*>(a.o + to)[0] = pack_bf16(d[0], d[1]);
    reinterpret_cast<uint32_t*>(a.o + to)[1] = pack_bf16(d[2], d[3]);
    if (a.o2) {
        reinterpret_cast<uint32_t*>(a.o2 + to)[0] = pack_bf16(o[1][0], o[1][1]);
        reinterpret_cast<uint32_t*>(a.o2 + to)[1] = pack_bf16(o[1][2], o[1][3]);
    }
}

template <int D, bool STATS, bool SPLIT>
hipError_t launch_fwd(const DiffArgs& a, hipStream_t stream) {
    auto run = [&](auto kernel, int rows) {
        const int n = a.n_bh * ((a.Tq + rows - 1) / rows) * (SPLIT ? a.split : 1), per = per_xcd(a, n);
        hipLaunchKernelGGL(kernel, dim3(8 * per), dim3(256), 0, stream, a, n);
        return hipGetLastError();
    };
    const hipError_t e = !a.by_keys ? run(diff_fwd<D, false, STATS, SPLIT>, kDiffRows)
                                    : (a.Tq <= 16 ? run(diff_few<D, STATS, SPLIT>, 16) : run(diff_fwd<D, true, STATS, SPLIT>, 32));
    if (e != hipSuccess || !SPLIT) return e;
    hipLaunchKernelGGL((diff_join<D>), dim3(a.n_bh * a.Tq), dim3(256), 0, stream, a);
    return hipGetLastError();
}
template <int D>
hipError_t launch_fwd_d(const DiffArgs& a, hipStream_t stream) {
    if (a.split > 1) return a.o2 ? launch_fwd<D, true, true>(a, stream) : launch_fwd<D, false, true>(a, stream);
    return a.o2 ? launch_fwd<D, true, false>(a, stream) : launch_fwd<D, false, false>(a, stream);
}

// ---- backward ------------------------------------------------------------------------------

// By 16 lanes a row (lane c of them; the first two take a 72-wide head's last chunks too): dO . O and dO . O_2 of row `row`
// (counted over the heads), in all of them
template <int D>
__device__ __forceinline__ void row_products(const DiffArgs& a, int64_t row, int c, float& s, float& s2) {
    s = s2 = 0.f;
    auto add = [&](int ch) {
        const size_t at = row * (2 * D) + 8 * ch;
        const u32x4 x = *reinterpret_cast<const u32x4*>(a.o + at), x2 = *reinterpret_cast<const u32x4*>(a.o2 + at),
                    y = *reinterpret_cast<const u32x4*>(a.d_o + at);
#pragma unroll
        for (int w = 0; w < 4; ++w) {
            s = __builtin_fmaf(lo_f(x[w]), lo_f(y[w]), s);
            s = __builtin_fmaf(hi_f(x[w]), hi_f(y[w]), s);
            s2 = __builtin_fmaf(lo_f(x2[w]), lo_f(y[w]), s2);
            s2 = __builtin_fmaf(hi_f(x2[w]), hi_f(y[w]), s2);
        }
    };
    add(c);
    if (D == 72 && c < 2) add(16 + c);
    s += dpp<0xB1>(s);
    s2 += dpp<0xB1>(s2);
    s += dpp<0x4E>(s);
    s2 += dpp<0x4E>(s2);
    s += dpp<0x141>(s);
    s2 += dpp<0x141>(s2);
    s += dpp<0x140>(s);
    s2 += dpp<0x140>(s2);
}
// value c (0 .. 3) of row t of head bh from these products: log2 of a map's denominator, -delta_2, delta_2 - delta_1
__device__ __forceinline__ float row_value(const DiffArgs& a, int64_t bh, int t, int c, float s, float s2) {
    if (c < 2) {
        const size_t at = (size_t)(2 * bh + c) * a.Tq + t;
        const float l = a.row_sum[at];
        return l == 0.f ? INFINITY : __builtin_fmaf(a.row_max[at], kLog2e, log2f(l));
    }
    // delta_1 = dO . O + lam delta_2
    return c == 2 ? -s2 : s2 - __builtin_fmaf(a.lam[(bh % a.H) * a.lam_step], s2, s);
}

// Rows are counted with each head's padded to whole 64, whose values are zeros.  A workgroup's 16 rows, of one head, leave
// their sum of -delta_2 for dlam.
template <int D>
__global__ __launch_bounds__(256) void diff_rows(DiffArgs a) {
    __shared__ float lam_row[16];
    const int64_t i = ((int64_t)blockIdx.x * 256 + threadIdx.x) >> 4;
    const int c = threadIdx.x & 15;
    const int64_t bh = i / a.T64;
    const int t = (int)(i - bh * a.T64);
    float s = 0.f, s2 = 0.f;
    if (t < a.Tq) row_products<D>(a, bh * a.Tq + t, c, s, s2);
    if (c == 0) lam_row[threadIdx.x >> 4] = -s2;
    __syncthreads();
    if (threadIdx.x == 0) {
        double sum = 0.0;
#pragma unroll
        for (int r = 0; r < 16; ++r) sum += lam_row[r];
        a.lam_part[blockIdx.x] = sum;
    }
    if (c < 4) a.row_vals[bh * 4 * a.T64 + (size_t)c * a.T64 + t] = t < a.Tq ? row_value(a, bh, t, c, s, s2) : 0.f;
}

// SHORT: the values of rows t0 .. t0 + n - 1 of a head into LDS, [4][pitch]
template <int D>
__device__ __forceinline__ void rows_to_lds(const DiffArgs& a, lds_u8* to, int pitch, int bh, int t0, int n) {
    const int c = threadIdx.x & 15;
    for (int i = threadIdx.x >> 4; i < n; i += blockDim.x >> 4) {
        float s = 0.f, s2 = 0.f;
        const int t = t0 + i;
        if (t < a.Tq) row_products<D>(a, (int64_t)bh * a.Tq + t, c, s, s2);
        if (c < 4) *(lds_f32*)(to + (c * pitch + i) * 4) = t < a.Tq ? row_value(a, bh, t, c, s, s2) : 0.f;
    }
}

// dlam of head h (all heads where they share it), in 64 bits
template <int D, bool SHORT>
__device__ __forceinline__ void sum_lam(const DiffArgs& a, double* lds, int h) {
    double s = 0.0;
    const int step = a.lam_step ? a.H : 1;
    if (SHORT) {
        for (int bh = h; bh < a.n_bh; bh += step)
            for (int t = threadIdx.x >> 4; t < a.Tq; t += blockDim.x >> 4) {
                float x, x2;
                row_products<D>(a, (int64_t)bh * a.Tq + t, threadIdx.x & 15, x, x2);
                if ((threadIdx.x & 15) == 0) s -= x2;
            }
    } else {
        const int each = a.T64 / 16;  // sums of a head
        const int n = a.lam_step ? each : a.n_bh * each;
        for (int bh = h; bh < a.n_bh; bh += a.lam_step ? a.H : a.n_bh) {
            const double* x = a.lam_part + (size_t)bh * each;
#pragma unroll 4
            for (int t = threadIdx.x; t < n; t += blockDim.x) s += x[t];
        }
    }
    lds[threadIdx.x] = s;
    for (int m = blockDim.x / 2; m; m /= 2) {
        __syncthreads();
        if ((int)threadIdx.x < m) lds[threadIdx.x] += lds[threadIdx.x + m];
    }
    if (threadIdx.x == 0) a.d_lam[h] = (float)lds[0];
}

// Heads of up to kShortRows queries in few tiles: the workgroups form the row values themselves (those of dK and dV all of
// a head's, in LDS), which saves the launch of diff_rows: one head of 100 tokens 16.7 -> 13.9 us; of 256, in turns of 16
// rows, 17.6 -> 20.
constexpr int kShortRows = kDiffShort;

// 16-byte pieces of a lane's sums
template <int D, bool KV>
constexpr int SUMS = (KV ? 32 : 16) + (D == 72 ? (KV ? 4 : 2) : 0);

// Own rows K_1, K_2, V (KV) against X = Q_1, Q_2 and Y = dO of the queries, or own Q_1, Q_2, dO against K_1, K_2, V:
// 32 own rows to a wave, kDiffRows to a workgroup of four waves, against stages of BS rows; or (TWO) to one of eight, of
// which four take the first half of each stage and four the other, and join their sums in LDS.  SPLIT: against a part
// of the other side.
template <int D, bool KV, int BS, bool TWO, bool SPLIT, bool SHORT>
__device__ __forceinline__ void diff_walk(const DiffArgs& a, lds_u8* lds, int item, int part, int tile, int bh, int keys) {
    constexpr int W = kDiffRows / 32;
    static_assert(!TWO || BS == 64, "a half to each four waves");
    using R = DiffRing<D, TWO ? 2 * W : W, BS, KV && !SHORT>;
    constexpr int OWN = R::LDS + (SHORT ? kShortRows * 16 : 0);  // LDS offset of what the walk keeps of its own
    using Rd = Reads<D>;
    constexpr int NB = R::NB, WB = R::WB, NW = KV ? 4 : 1;
    constexpr bool TAIL = D == 72;
    const int T = KV ? a.Tk : a.Tq, Tx = KV ? a.Tq : a.Tk;  // rows of the own side and of the other
    const int w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), wave = TWO ? w % W : w, half = TWO ? w / W : 0;
    const int row0 = (tile * W + wave) * 32;
    const int own_end = KV ? keys : T, x_end = KV ? Tx : keys;
    const int tile0 = row0 - 32 * wave;
    int n_st = (x_end + BS - 1) / BS;
    if (KV && tile0 >= keys) n_st = 0;  // keys that the sample does not have
    const int split = KV ? a.split_k : a.split_q;
    const int per = SPLIT ? ((Tx + BS - 1) / BS + split - 1) / split : n_st;
    const int s0 = part * per, s1 = SPLIT && s0 + per < n_st ? s0 + per : n_st;
    if (SPLIT && split > 1 && s0 >= n_st) return;  // diff_sum leaves it out

    const size_t n_x = (size_t)(2 * bh) * Tx * D, n_own = (size_t)(2 * bh) * T * D;
    const size_t w_x = (size_t)bh * Tx * (2 * D), w_own = (size_t)bh * T * (2 * D);
    const uint16_t* x = (KV ? a.q : a.k) + n_x;
    const uint16_t* own = (KV ? a.k : a.q) + n_own;
    R ring;
    ring.init(lds, x, x + (size_t)Tx * D, (KV ? a.d_o : a.v) + w_x, x_end);
    const float* vals = a.row_vals + (size_t)bh * 4 * a.T64;
    if (KV && !SHORT) ring.init_values(vals, a.T64);
    ring.load(0, s0 * BS);
    Rd rd;
    rd.init(lds);
    rd.pack();
    bf16x8 n_op[2][4], n_tail[2], w_op[KV ? 1 : Rd::WS];
#pragma unroll
    for (int i = 0; i < 2; ++i) rd.own_rows(own + (size_t)i * T * D, NB, row0, own_end, n_op[i], TAIL ? &n_tail[i] : nullptr);
    const int own_v = OWN + 32 * wave * WB, own_t = OWN + 32 * W * WB + wave * 1024;
    if constexpr (KV) {
        if (half == 0) ring.load_own(own_v, row0, buffer_rsrc(a.v + w_own, own_end * WB));
        if (TAIL && half == 0 && !rd.hi) {
            *(lds_bf16x8*)(lds + own_t + rd.l32 * 16) = n_tail[0];
            *(lds_bf16x8*)(lds + own_t + 512 + rd.l32 * 16) = n_tail[1];
        }
    } else
        rd.own_rows(a.d_o + w_own, WB, row0, own_end, w_op, nullptr);
    float log[2] = {INFINITY, INFINITY}, minus = 0.f, more = 0.f;  // of the own query
    if (SHORT) {
        rows_to_lds<D>(a, lds + R::LDS, kShortRows, bh, KV ? 0 : tile0, KV ? a.T64 : 32 * W);
        __syncthreads();
    }
    if (!KV && row0 + rd.l32 < T) {
        auto value = [&](int n) { return SHORT ? *(lds_f32*)(lds + R::LDS + (n * kShortRows + 32 * wave + rd.l32) * 4) : vals[n * a.T64 + row0 + rd.l32]; };
        log[0] = value(0);
        log[1] = value(1);
        minus = value(2);
        more = value(3);
    }
    const float c2 = a.scale_log2, lam = a.lam[(bh % a.H) * a.lam_step];

    f32x16 acc[2][2], wacc[NW];  // dK or dQ of each map; dV
    f32x4 tacc[2], wtacc[2];  // 72 wide: both maps' last 8 elements, dV's last 16, of 16 own rows each
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        acc[i][0] = acc[i][1] = f32x16{};
        tacc[i] = wtacc[i] = f32x4{};
    }
#pragma unroll
    for (int d = 0; d < NW; ++d) wacc[d] = f32x16{};

    int st = 0;
    for (int s = s0; s < s1; ++s) {
        ring.turn();
        ring.load(R::STAGE - st, (s + 1) * BS);
        if (row0 < own_end) {
#pragma unroll
            for (int i = 0; i < (TWO ? 1 : BS / 32); ++i) {
                const int h = TWO ? half : i, cw = st + R::WIDE + 32 * h * WB, first = s * BS + 32 * h;
                if (KV) rd.unpack();
                // four values of a chunk's rows 8 j + 4 hi ..
                auto value = [&](int n, int j) {
                    const int at = SHORT ? R::LDS + (n * kShortRows + s * BS) * 4 : st + R::VAL + n * BS * 4;
                    return __builtin_bit_cast(f32x4, *(const lds_u32x4*)(lds + at + (32 * h + 8 * j + 4 * rd.hi) * 4));
                };
                f32x16 dp;  // dA - delta_2
                if (KV) {
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        const f32x4 v = value(2, j);
#pragma unroll
                        for (int e = 0; e < 4; ++e) dp[4 * j + e] = v[e];
                    }
                } else {
                    dp = f32x16{} + minus;
                }
                const int cx = st + 32 * h * NB;
                auto mask = [&](f32x16& sc) {
                    if (!KV && first + 32 > keys) {
                        const int lim = keys - first - 4 * rd.hi;
#pragma unroll
                        for (int x = 0; x < 16; ++x)
                            if (8 * (x >> 2) + (x & 3) >= lim) sc[x] = -INFINITY;
                    }
                };
                f32x16 p1;  // map 1's probabilities (KV)
                uint32_t pk[8], ds[2][8];
                // P and dS of a map, a matrix product after every four of them
                auto soft = [&](int i, const f32x16& sc, auto&& product) {
#pragma unroll
                    for (int j = 0; j < 4; ++j) {
                        f32x4 lg = {log[i], log[i], log[i], log[i]}, mo = {more, more, more, more};
                        if (KV) lg = value(i, j);
                        if (KV && i == 0) mo = value(3, j);
#pragma unroll
                        for (int e = 0; e < 4; e += 2) {
                            const int x = 4 * j + e;
                            const float e0 = __builtin_amdgcn_exp2f(__builtin_fmaf(sc[x], c2, -lg[e]));
                            const float e1 = __builtin_amdgcn_exp2f(__builtin_fmaf(sc[x + 1], c2, -lg[e + 1]));
                            if (i == 0) {
                                ds[0][x / 2] = pack_bf16(e0 * (dp[x] + mo[e]), e1 * (dp[x + 1] + mo[e + 1]));
                                p1[x] = e0;
                                p1[x + 1] = e1;
                            } else {
                                ds[1][x / 2] = pack_bf16(e0 * dp[x], e1 * dp[x + 1]);
                                if (KV) pk[x / 2] = pack_bf16(__builtin_fmaf(-lam, e0, p1[x]), __builtin_fmaf(-lam, e1, p1[x + 1]));
                            }
                        }
                        product(j);
                    }
                };
                auto grad = [&](int i, int k) { acc[i][k & 1] = mma(rd.n_col(cx + i * R::NT, k & 1, k >> 1), op(ds[i], k >> 1), acc[i][k & 1]); };
                f32x16 s0 = {}, s1 = {};
                auto score = [&](int i, int k, f32x16& sc) { sc = mma(rd.n_row(cx + i * R::NT, k), n_op[i][k], sc); };
                auto pull = [&](int k) { dp = mma(rd.w_row(cw, k), KV ? rd.w_row(own_v, k) : w_op[KV ? 0 : k], dp); };
                if constexpr (!TAIL) {
                    // what does not wait for what stands side by side: 16.2 to 15.9 ms at the CogVideoX shape
#pragma unroll
                    for (int k = 0; k < Rd::WS; ++k) {
                        pull(k);
                        if (k < 4) score(0, k, s0);
                    }
                    mask(s0);
                    soft(0, s0, [&](int k) { score(1, k, s1); });
                    mask(s1);
                    soft(1, s1, [&](int k) { grad(0, k); });
#pragma unroll
                    for (int k = 0; k < 4; ++k) grad(1, k);
                } else {
                    // 72-wide heads have no registers for that (8.6 to 9.2 ms, 16 heads of 16384 tokens): a map at a time
#pragma unroll
                    for (int k = 0; k < Rd::WS; ++k) pull(k);
#pragma unroll
                    for (int i = 0; i < 2; ++i) {
                        f32x16& sc = i ? s1 : s0;
#pragma unroll
                        for (int k = 0; k < 4; ++k) score(i, k, sc);
                        const bf16x8 y = KV ? *(const lds_bf16x8*)(lds + (rd.hi ? R::ZERO : own_t + 512 * i + rd.l32 * 16)) : n_tail[i];
                        sc = mma(rd.n_row_tail(cx + i * R::NT, R::ZERO), y, sc);
                        mask(sc);
                        soft(i, sc, [](int) {});
#pragma unroll
                        for (int k = 0; k < 4; ++k) grad(i, k);
                        // Map i's rows of the product are lanes 32 i .. + 31; the others keep theirs.  (Zeros for the other map's
                        // rows would need no choice, but make NaN of this map's NaN there: 9.00 ms for 8.87, 16 heads of 16384
                        // tokens.  Accumulators for each map, with 4 registers spilled: 8.99, 88 heads of 4 queries 522 us for 505.)
                        const bf16x8 c = rd.n_col_tail(cx + i * R::NT);
                        uint32_t z[8];
                        halves(ds[i], z);
#pragma unroll
                        for (int h = 0; h < 2; ++h) {
                            const f32x4 t = mma16(c, op(z, h), tacc[h]);
#pragma unroll
                            for (int e = 0; e < 4; ++e) tacc[h][e] = rd.hi == i ? t[e] : tacc[h][e];
                        }
                        if (KV) __builtin_amdgcn_sched_barrier(0);  // else registers spill
                    }
                }
                if (KV) {
#pragma unroll
                    for (int ks = 0; ks < 2; ++ks)
#pragma unroll
                        for (int d = 0; d < NW; ++d) wacc[d] = mma(rd.w_col(cw, d, ks), op(pk, ks), wacc[d]);
                    if (TAIL) {
                        const bf16x8 c = rd.w_col_tail(cw);
                        uint32_t y[8];
                        halves(pk, y);
                        wtacc[0] = mma16(c, op(y, 0), wtacc[0]);
                        wtacc[1] = mma16(c, op(y, 1), wtacc[1]);
                    }
                }
            }
        }
        st = R::STAGE - st;
    }
    wait_vm<0>();  // nothing may land in LDS after the workgroup has ended
    if constexpr (TWO) {
        // the second four waves' sums, in pieces of 16 bytes a lane
        lds_u8* const at = lds + wave * SUMS<D, KV> * 1024 + rd.lane * 16;
        auto each = [&](auto&& fn) {
            int n = 0;
            auto tile = [&](f32x16& c) {
#pragma unroll
                for (int u = 0; u < 4; ++u, ++n) {
                    f32x4 x = {c[4 * u], c[4 * u + 1], c[4 * u + 2], c[4 * u + 3]};
                    fn(x, (lds_f32x4*)(at + n * 1024));
#pragma unroll
                    for (int e = 0; e < 4; ++e) c[4 * u + e] = x[e];
                }
            };
#pragma unroll
            for (int i = 0; i < 4; ++i) tile(acc[i / 2][i % 2]);
#pragma unroll
            for (int d = 0; d < (KV ? 4 : 0); ++d) tile(wacc[d]);
            if (TAIL) {
#pragma unroll
                for (int i = 0; i < 2; ++i, ++n) fn(tacc[i], (lds_f32x4*)(at + n * 1024));
#pragma unroll
                for (int i = 0; i < (KV ? 2 : 0); ++i, ++n) fn(wtacc[i], (lds_f32x4*)(at + n * 1024));
            }
        };
        __syncthreads();
        if (half) each([](f32x4& x, lds_f32x4* p) { *p = x; });
        __syncthreads();
        if (half) return;
        each([](f32x4& x, lds_f32x4* p) { x += *p; });
    }

    // rows of a tile as fp32 [32][width] of a part, or rounded into the output (rows past the keys as zeros)
    const bool parts = SPLIT && split > 1;
    // lanes from t0 on: the rows of t that hold the last elements
    auto store = [&](const f32x16* c, int tiles, const f32x4* t, int t0, int t_n, int width, float f, float* to, uint16_t* out) {
        const int row = row0 + rd.l32;
        auto put = [&](int r, int col, float x0, float x1, float x2, float x3) {
            if (parts) {
                *reinterpret_cast<f32x4*>(to + (r - row0) * width + col) = f32x4{x0, x1, x2, x3};
            } else if (r < T) {
                uint32_t* p = reinterpret_cast<uint32_t*>(out + (size_t)r * width + col);
                p[0] = pack_bf16(x0, x1);
                p[1] = pack_bf16(x2, x3);
            }
        };
#pragma unroll
        for (int d = 0; d < 4; ++d) {
            if (d >= tiles) break;
#pragma unroll
            for (int u = 0; u < 4; ++u) {
                auto v = [&](int e) { return row >= own_end ? 0.f : c[d][4 * u + e] * f; };
                put(row, 32 * d + 16 * rd.hi + 4 * u, v(0), v(1), v(2), v(3));
            }
        }
        const int g = (rd.lane - t0) >> 4;  // group of four rows
        if (TAIL && g >= 0 && 4 * g < t_n) {
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const int r = row0 + 16 * h + (rd.lane & 15);
                auto v = [&](int e) { return r >= own_end ? 0.f : t[h][e] * f; };
                put(r, width - t_n + 4 * g, v(0), v(1), v(2), v(3));
            }
        }
    };
    const float f2 = -lam * a.scale_nat;
    constexpr int TILE = 32 * W * D;  // of one map
    float* to = parts ? (KV ? a.part_k : a.part_q) + ((size_t)item * split + part) * ((KV ? 4 : 2) * TILE) : nullptr;
    uint16_t* const out = (KV ? a.dk : a.dq) + n_own;
    store(acc[0], 2, tacc, 0, 8, D, a.scale_nat, to + 32 * wave * D, out);
    store(acc[1], 2, tacc, 32, 8, D, f2, to + TILE + 32 * wave * D, out + (size_t)T * D);
    if (KV) store(wacc, 4, wtacc, 0, 16, 2 * D, 1.0f, to + 2 * TILE + 32 * wave * (2 * D), a.dv + w_own);
}

constexpr int most(int x, int y) { return x > y ? x : y; }

template <int D, bool TWO, bool SPLIT, bool SHORT>
__global__ __launch_bounds__(TWO ? 512 : 256) __attribute__((amdgpu_waves_per_eu(2, 2))) void diff_bwd(DiffArgs a, int n_lam, int n_k,
                                                                                                     int per_k, int n_q, int per_q) {
    constexpr int W = TWO ? 8 : 4, BS_K = TWO ? 64 : 32;
    constexpr int LDS_K = DiffRing<D, W, BS_K, !SHORT>::LDS + kDiffRows * (4 * D + (D == 72 ? 32 : 0)), LDS_Q = DiffRing<D, W, 64, false>::LDS;
    constexpr int VALS = SHORT ? kShortRows * 16 : 0;
    __shared__ __attribute__((aligned(1024))) unsigned char smem[most(most(LDS_K, LDS_Q) + VALS, TWO ? 4 * SUMS<D, true> * 1024 : 0)];
    lds_u8* const lds = (lds_u8*)smem;
    int g = blockIdx.x;
    const int lam8 = (n_lam + 7) & ~7;  // (whole eights, so that a tile's XCD goes by its number)
    if (g < lam8) {
        if (g < n_lam) sum_lam<D, SHORT>(a, reinterpret_cast<double*>(smem), g);
        return;
    }
    g -= lam8;
    // what takes longer first
    const int ahead = 8 * (a.q_first ? per_q : per_k);
    const bool kv = (g < ahead) != (a.q_first != 0);
    if (g >= ahead) g -= ahead;
    auto walk = [&](auto side) {
        constexpr bool KV = decltype(side)::value;
        const int split = KV ? a.split_k : a.split_q, n_tile = ((KV ? a.Tk : a.Tq) + kDiffRows - 1) / kDiffRows;
        int bh = 0, keys = 0, part = 0;
        const bool some = KV && a.by_len;  // of a head's tiles have work
        int item = some ? item_of_k(a, g, n_k, n_tile, split, bh, keys) : item_of(a, g, KV ? n_k : n_q);
        if (item < 0) return;
        if (SPLIT) {
            part = item % split;
            item /= split;
        }
        const int head = item / n_tile, tile = item - head * n_tile;
        if (!some) bh = head_of(a, head, keys);
        diff_walk<D, KV, KV ? BS_K : 64, TWO, SPLIT, SHORT>(a, lds, item, part, tile, bh, keys);
    };
    if (kv)
        walk(std::integral_constant<bool, true>{});
    else
        walk(std::integral_constant<bool, false>{});
}

// Sums of a tile's parts: dK_1, dK_2, the halves of dV (kind 0 .. 3; `tiles_k` of them in x), then dQ_1, dQ_2 (4, 5);
// blockIdx.y counts from `kind0`; bs_k: rows of a stage of dK and dV's walks
template <int D>
__global__ __launch_bounds__(256) void diff_sum(DiffArgs a, int bs_k, int kind0, int tiles_k, int tiles_q) {
    constexpr int TILE = kDiffRows * D;
    const int kind = kind0 + blockIdx.y;
    const bool kv = kind < 4;
    if ((int)blockIdx.x >= (kv ? tiles_k : tiles_q)) return;
    const int T = kv ? a.Tk : a.Tq, n_tile = (T + kDiffRows - 1) / kDiffRows, n = kv ? a.split_k : a.split_q;
    int keys;
    const int head = blockIdx.x / n_tile, bh = head_of(a, head, keys), row0 = (blockIdx.x - head * n_tile) * kDiffRows;
    const int width = kv && kind >= 2 ? 2 * D : D, which = kv ? kind : kind - 4;
    const size_t stride = (kv ? 4 : 2) * (size_t)TILE;
    const float* part = (kv ? a.part_k : a.part_q) + (size_t)blockIdx.x * n * stride + (size_t)which * TILE;
    uint16_t* out;
    int skip = 0;  // elements of dV before this half
    if (width == D) {
        out = (kv ? a.dk : a.dq) + (size_t)(2 * bh + which) * T * D;
    } else {
        out = a.dv + (size_t)bh * T * (2 * D);
        skip = (which - 2) * TILE;
    }
    const int j = blockIdx.z * 1024 + threadIdx.x * 4;
    const int left = T - row0, size = (left < kDiffRows ? left : kDiffRows) * width;
    if (j >= TILE || skip + j >= size) return;
    // parts that hold rows of the other side, as diff_walk has them; none for keys that the sample does not have
    const int Tx = kv ? a.Tq : a.Tk, bs = kv ? bs_k : 64, per = ((Tx + bs - 1) / bs + n - 1) / n;
    const int stages = kv ? (row0 < keys ? (Tx + bs - 1) / bs : 0) : (keys + bs - 1) / bs, full = (stages + per - 1) / per;
    f32x4 s = {};
#pragma unroll 4
    for (int p = 0; p < full; ++p) s += *reinterpret_cast<const f32x4*>(part + p * stride + j);
    uint32_t* to = reinterpret_cast<uint32_t*>(out + (size_t)row0 * width + skip + j);
    to[0] = pack_bf16(s[0], s[1]);
    to[1] = pack_bf16(s[2], s[3]);
}

template <int D>
hipError_t launch_bwd_d(const DiffArgs& a, hipStream_t stream) {
    const int64_t rows = (int64_t)a.n_bh * a.T64;
    hipError_t e = hipSuccess;
    if (rows > 0 && !a.short_rows) {
        hipLaunchKernelGGL((diff_rows<D>), dim3((uint32_t)(rows / 16)), dim3(256), 0, stream, a);
        e = hipGetLastError();
        if (e != hipSuccess) return e;
    }
    const int tiles_k = a.n_bh * ((a.Tk + kDiffRows - 1) / kDiffRows), tiles_q = a.n_bh * ((a.Tq + kDiffRows - 1) / kDiffRows);
    const bool split = a.split_k > 1 || a.split_q > 1;
    const int n_k = tiles_k * a.split_k, n_q = tiles_q * a.split_q, per_k = per_xcd_k(a, n_k), per_q = per_xcd(a, n_q);
    const int n_lam = a.lam_step ? a.H : 1;
    const dim3 grid(((n_lam + 7) & ~7) + 8 * per_k + 8 * per_q);
    auto run = [&](auto kernel, int threads) {
        hipLaunchKernelGGL(kernel, grid, dim3(threads), 0, stream, a, n_lam, n_k, per_k, n_q, per_q);
        return hipGetLastError();
    };
    if (a.short_rows)
        e = a.two ? run(diff_bwd<D, true, false, true>, 512) : run(diff_bwd<D, false, false, true>, 256);
    else if (a.two)
        e = split ? run(diff_bwd<D, true, true, false>, 512) : run(diff_bwd<D, true, false, false>, 512);
    else
        e = split ? run(diff_bwd<D, false, true, false>, 256) : run(diff_bwd<D, false, false, false>, 256);
    if (e != hipSuccess || !split) return e;
    const int sums_k = a.split_k > 1 ? tiles_k : 0, sums_q = a.split_q > 1 ? tiles_q : 0, kind0 = sums_k ? 0 : 4;
    hipLaunchKernelGGL((diff_sum<D>), dim3(most(sums_k, sums_q), (sums_q ? 6 : 4) - kind0, kDiffRows * D / 1024), dim3(256), 0, stream, a,
                       a.two ? 64 : 32, kind0, sums_k, sums_q);
    return hipGetLastError();
}

}  // namespace

hipError_t launch_diff(const DiffArgs& a, int D, hipStream_t stream) {
    return D == 64 ? launch_fwd_d<64>(a, stream) : launch_fwd_d<72>(a, stream);
}
hipError_t launch_diff_backward(const DiffArgs& a, int D, hipStream_t stream) {
    return D == 64 ? launch_bwd_d<64>(a, stream) : launch_bwd_d<72>(a, stream);
}

}  // namespace rt
