// One wave's part of attention's gradients (attn_grad.hip).  It holds 32 rows of its own (keys and values for dK and
// dV, queries and output gradients for dQ) and takes 32-row chunks of the other side, X and Y, from LDS:
//
//   KV   own K, V;   X = Q, Y = dO    S = X K^T, dP = Y V^T - delta;  dV^T += Y^T P,  dK^T += X^T dS
//   !KV  own Q, dO;  X = K, Y = V     S^T = X Q^T, dP^T = Y dO^T - delta;  dQ^T += X^T dS^T
//
// with P = exp2(c S - log), dS = P dP.  The 32x32x16 accumulator of a score hands each lane 16 rows of X of one own
// row, which are exactly the 8 + 8 contraction values that the B operand of the gradients' products takes, so P and
// dS never leave registers.  They are rounded to bf16 there, as the matrix products take them (the same rounding
// that the forward call gives P); scores, dP, P times dP and all sums are fp32.
//
// delta enters as the accumulator that dP starts from, not by a subtraction for each element.
//
// 72-wide heads: the 8 dims past 64 take one k-step of the scores, half of it zeros in both operands, and one
// 16x16x32 product for 16 own rows of the gradients.
//
// 32 own rows, so that two or three waves share a SIMD and one's products run under another's exponentials.  Measured
// against one wave of 64 rows to a SIMD, half the LDS reads a product, whose tiles ran half a step apart as in
// attn_tiles.h (CogVideoX, two waves): dK and dV 10.1 -> 9.1 ms, dQ 7.2 -> 6.6 ms (that wave's 456 registers lie half in
// the accumulator file, from where the vector unit has to copy every score); 72-wide heads did not fit it.  The same
// half step within these waves: 8.9 and 6.6 ms, and spills for 72-wide heads; not kept.  64 queries a wave for dQ alone,
// whose sums take half the registers: 6.5 ms in a launch of its own, no less than its share of the common one.  The
// chunk's code once for chunks with rows past the end and once for the others: the compiler spills 49 registers of the
// 168 (26 ms for 15).
#pragma once

#include "attn_common.h"
#include "train.h"

namespace rt {
namespace {

typedef float f32x4 __attribute__((ext_vector_type(4)));

constexpr int kOff = 0x60000000;  // buffer offset past every record, also after small additions

__device__ __forceinline__ f32x16 mma(const bf16x8& x, const bf16x8& y, const f32x16& z) {
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(x, y, z, 0, 0, 0);
}

// 64-wide rows' 16-byte slots are swizzled by the row, for LDS that serves 256 bytes a cycle, two rows: the 16 rows
// of a quarter of a row read (one slot) and the 4 rows of half a transposed one (four slots) then fall on different
// banks.  (r >> 1) & 7 with bits 2, 1 and 3 of r for bits 0, 2 and 1, so that rows 16 apart agree and rows 8 apart
// differ in bit 1.  72-wide rows (144 bytes) do so by themselves, transposed reads two to a bank.
template <int D>
__device__ __forceinline__ int swz(int r) {
    return Geo<D>::SWZ ? ((r & 2) << 1) | ((r & 8) >> 2) | ((r & 4) >> 2) : 0;
}

// 8 lanes a row (lane c of them; of a 72-wide row the first takes the last 8 elements too): dO . O, in all of them
template <int CTRL>
__device__ __forceinline__ float dpp(float x) {
    return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(x), CTRL, 0xf, 0xf, true));
}
template <int D>
__device__ __forceinline__ float row_delta(const GradArgs& a, size_t row, int c) {
    float s = 0.f;
    auto add = [&](int ch) {
        const size_t at = row * D + 8 * ch;
        const u32x4 x = *reinterpret_cast<const u32x4*>(a.o + at), y = *reinterpret_cast<const u32x4*>(a.d_o + at);
#pragma unroll
        for (int w = 0; w < 4; ++w) {
            s = __builtin_fmaf(lo_f(x[w]), lo_f(y[w]), s);
            s = __builtin_fmaf(hi_f(x[w]), hi_f(y[w]), s);
        }
    };
    add(c);
    if (D == 72 && c == 0) add(8);
    s += dpp<0xB1>(s);
    s += dpp<0x4E>(s);
    return s + dpp<0x141>(s);
}
// log2 of a row's denominator
__device__ __forceinline__ float row_log(const GradArgs& a, size_t row) {
    return __builtin_fmaf(a.row_max[row], 1.44269504f, log2f(a.row_sum[row]));
}

// ZERO: LDS offset of 16 zero bytes.  A chunk's 32 rows of Y lie CHUNK_Y behind those of X.
template <int D, bool KV, int ZERO, int CHUNK_Y>
struct GradTile {
    using G = Geo<D>;
    static constexpr int ROWB = 2 * D;
    static constexpr bool TAIL = D == 72;
    static constexpr int NG = KV ? 2 : 1;  // gradients: 0 from X (dK or dQ), 1 from Y (dV)

    lds_u8* lds;
    int lane, l32, hi;
    int rd, tr, t_rd;
    float c2;
    bf16x8 own[2][4], own_tail[2];  // [K or Q, V or dO][k-step]
    f32x16 acc[NG][2];              // [gradient][dims 32 dt ..]
    f32x4 tacc[NG][2];              // [gradient][16 own rows]: dims 64 + 4 (lane / 16) .. in lanes below 32
    f32x16 sc, dp;                  // the chunk's scores and dP
    uint32_t pk[8], ds[8];          // bf16 P (KV) and dS
    float log, nd;                  // !KV: of the lane's own row: log2 of its denominator, -delta

    __device__ __forceinline__ void init(lds_u8* smem, float scale_log2) {
        lds = smem;
        lane = threadIdx.x & 63;
        l32 = lane & 31;
        hi = lane >> 5;
        c2 = scale_log2;
        // a lane's reads, see attn_tiles.h: row l32, chunk hi; rows 4 hi + L / 4 (+ 8) transposed, which puts dims
        // 32 dt + 16 hi .. + 15 on a lane's 16 accumulators
        rd = l32 * ROWB + ((hi ^ swz<D>(l32)) * 16);
        const int G4 = lane >> 4, L = lane & 15;
        const int r = 4 * hi + (L >> 2), d = 16 * (L & 1) + 8 * (G4 & 1) + 4 * ((L >> 1) & 1);
        tr = r * ROWB + (((d >> 3) ^ swz<D>(r)) * 16) + (d & 7) * 2;
        t_rd = (16 * (G4 & 1) + 4 * (G4 >> 1) + (L >> 2)) * ROWB + (64 + 4 * (L & 1)) * 2;
#pragma unroll
        for (int g = 0; g < NG; ++g) {
            acc[g][0] = acc[g][1] = f32x16{};
            tacc[g][0] = tacc[g][1] = f32x4{};
        }
    }

    // rows row0 .. + 31 of a head's x (zeros past its end): lane holds row l32, dims 16 s + 8 hi ..
    __device__ __forceinline__ void load_rows(const uint16_t* x, int row0, int T, bf16x8 (&to)[4], bf16x8& to_tail) {
        const __amdgpu_buffer_rsrc_t rs = __builtin_amdgcn_make_buffer_rsrc((void*)x, (short)0, T * ROWB, 0x00020000);
        const int off = (row0 + l32) * ROWB;
        auto load = [&](int o) { return __builtin_bit_cast(bf16x8, __builtin_amdgcn_raw_buffer_load_b128(rs, o, 0, 0)); };
#pragma unroll
        for (int s = 0; s < 4; ++s) to[s] = load(off + 32 * s + 16 * hi);
        if (TAIL) to_tail = load(hi ? kOob : off + 128);
    }
    __device__ __forceinline__ void load_own(const GradArgs& a, size_t head_off, int row0, int T) {
        load_rows((KV ? a.k : a.q) + head_off, row0, T, own[0], own_tail[0]);
        load_rows((KV ? a.v : a.d_o) + head_off, row0, T, own[1], own_tail[1]);
    }
    // !KV: the own row's log and -delta, as grad_rows left them
    __device__ __forceinline__ void load_values(const GradArgs& a, int bh, int row0, int T) {
        const float* vals = a.row_vals + (size_t)bh * 2 * a.T64;
        const int row = row0 + l32;
        log = row < T ? vals[row] : INFINITY;
        nd = row < T ? vals[a.T64 + row] : 0.f;
    }
    // or formed from the own rows
    __device__ __forceinline__ void make_values(const GradArgs& a, int bh, int row0, int T) {
        bf16x8 o[4], o_tail;
        load_rows(a.o + (size_t)bh * (size_t)T * D, row0, T, o, o_tail);
        const int row = row0 + l32;
        float s = 0.f;
        auto add = [&](const bf16x8& x, const bf16x8& y) {
#pragma unroll
            for (int e = 0; e < 8; ++e) s = __builtin_fmaf((float)x[e], (float)y[e], s);
        };
#pragma unroll
        for (int k = 0; k < 4; ++k) add(o[k], own[1][k]);
        if (TAIL) add(o_tail, own_tail[1]);
        log = row < T ? row_log(a, (size_t)bh * T + row) : INFINITY;
        nd = -pair_sum(s);
    }

    __device__ __forceinline__ bf16x8 row_read(int base, int s) const {
        return *(const lds_bf16x8*)(lds + (G::SWZ ? (rd ^ (32 * s)) + base : rd + base + 32 * s));
    }
    __device__ __forceinline__ bf16x8 row_tail(int base) const {
        return *(const lds_bf16x8*)(lds + (hi ? ZERO : rd + base + 128));
    }
    static __device__ __forceinline__ bf16x8 tr_read(const lds_u8* p, const lds_u8* p8) {
        const bf16x4 v0 = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((lds_bf16x4*)p);
        const bf16x4 v1 = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((lds_bf16x4*)(p8 + 8 * ROWB));
        return __builtin_shufflevector(v0, v1, 0, 1, 2, 3, 4, 5, 6, 7);
    }
    __device__ __forceinline__ bf16x8 col_read(int base, int k) const {
        const int at = base + 16 * (k >> 1) * ROWB, d = 64 * (k & 1);
        return G::SWZ ? tr_read(lds + (tr ^ d) + at, lds + (tr ^ d ^ 32) + at) : tr_read(lds + tr + d + at, lds + tr + d + at);
    }
    __device__ __forceinline__ bf16x8 col_tail(int base) const { return tr_read(lds + t_rd + base, lds + t_rd + base); }
    static __device__ __forceinline__ bf16x8 op(const uint32_t (&p)[8], int ks) {
        return __builtin_bit_cast(bf16x8, u32x4{p[4 * ks], p[4 * ks + 1], p[4 * ks + 2], p[4 * ks + 3]});
    }
    // four of a chunk's 32 row values: a lane's rows 8 j + 4 hi ..
    __device__ __forceinline__ f32x4 value_read(int base, int j) const {
        return __builtin_bit_cast(f32x4, *(const lds_u32x4*)(lds + base + (8 * j + 4 * hi) * 4));
    }
    // the tails' product of one gradient: the two operands of 16 contraction rows become two of 32 for the halves of
    // the own rows, see attn_tiles.h
    __device__ __forceinline__ void tail_mma(int g, int base, const uint32_t (&p)[8]) {
        const bf16x8 x = col_tail(base);
        uint32_t y[8];
#pragma unroll
        for (int r = 0; r < 4; ++r) {
            auto s = __builtin_amdgcn_permlane16_swap(p[r], p[4 + r], false, false);
            y[r] = s[0];
            y[4 + r] = s[1];
        }
#pragma unroll
        for (int h = 0; h < 2; ++h)
            tacc[g][h] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(x, op(y, h), tacc[g][h], 0, 0, 0);
    }

    // scores and dP of the chunk at LDS offset cx, its rows' -deltas at minus
    __device__ __forceinline__ void scores(int cx, int minus) {
        if (KV) {
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const f32x4 v = value_read(minus, j);
#pragma unroll
                for (int i = 0; i < 4; ++i) dp[4 * j + i] = v[i];
            }
        } else {
            dp = f32x16{} + nd;
        }
        sc = f32x16{};
#pragma unroll
        for (int s = 0; s < 4; ++s) {
            sc = mma(row_read(cx, s), own[0][s], sc);
            dp = mma(row_read(cx + CHUNK_Y, s), own[1][s], dp);
        }
        if (TAIL) {
            sc = mma(row_tail(cx), own_tail[0], sc);
            dp = mma(row_tail(cx + CHUNK_Y), own_tail[1], dp);
        }
    }
    // P and dS of it, its rows' logs at logs
    __device__ __forceinline__ void soft(int logs) {
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            f32x4 v = {log, log, log, log};
            if (KV) v = value_read(logs, j);
#pragma unroll
            for (int i = 0; i < 4; i += 2) {
                const int x = 4 * j + i;
                const float e0 = __builtin_amdgcn_exp2f(__builtin_fmaf(sc[x], c2, -v[i]));
                const float e1 = __builtin_amdgcn_exp2f(__builtin_fmaf(sc[x + 1], c2, -v[i + 1]));
                if (KV) pk[x / 2] = pack_bf16(e0, e1);
                ds[x / 2] = pack_bf16(e0 * dp[x], e1 * dp[x + 1]);
            }
        }
    }
    // its gradients
    __device__ __forceinline__ void grads(int cx) {
#pragma unroll
        for (int k = 0; k < 4; ++k)
#pragma unroll
            for (int g = 0; g < NG; ++g)
                acc[g][k & 1] = mma(col_read(cx + g * CHUNK_Y, k), op(g ? pk : ds, k >> 1), acc[g][k & 1]);
        if (TAIL) {
#pragma unroll
            for (int g = 0; g < NG; ++g) tail_mma(g, cx + g * CHUNK_Y, g ? pk : ds);
        }
    }
    // scores for rows of X from row0 on that lie past T have no probability (!KV)
    __device__ __forceinline__ void mask(int row0, int T) {
        const int lim = T - row0 - 4 * hi;
#pragma unroll
        for (int x = 0; x < 16; ++x)
            if (8 * (x >> 2) + (x & 3) >= lim) sc[x] = -INFINITY;
    }

    // gradient g of the own rows as fp32 [32][D], times f
    __device__ __forceinline__ void store_part(int g, float* x, float f) const {
#pragma unroll
        for (int dt = 0; dt < 2; ++dt)
#pragma unroll
            for (int u = 0; u < 4; ++u) {
                const f32x16& c = acc[g][dt];
                *reinterpret_cast<f32x4*>(x + l32 * D + 32 * dt + 16 * hi + 4 * u) =
                    f32x4{c[4 * u] * f, c[4 * u + 1] * f, c[4 * u + 2] * f, c[4 * u + 3] * f};
            }
        if (TAIL && lane < 32) {
#pragma unroll
            for (int h = 0; h < 2; ++h)
                *reinterpret_cast<f32x4*>(x + (16 * h + (lane & 15)) * D + 64 + 4 * (lane >> 4)) = tacc[g][h] * f;
        }
    }

    __device__ __forceinline__ void store_all(const GradArgs& a, size_t head_off, int row0, int T) const {
        store(0, (KV ? a.dk : a.dq) + head_off, row0, T, a.scale_nat);
        if (KV) store(NG - 1, a.dv + head_off, row0, T, 1.0f);
    }
    // gradient g of the own rows row0 .. (those below T), times f
    __device__ __forceinline__ void store(int g, uint16_t* x, int row0, int T, float f) const {
        const int row = row0 + l32;
        if (row < T) {
#pragma unroll
            for (int dt = 0; dt < 2; ++dt)
#pragma unroll
                for (int u = 0; u < 2; ++u) {
                    const f32x16& c = acc[g][dt];
                    *reinterpret_cast<u32x4*>(x + (size_t)row * D + 32 * dt + 16 * hi + 8 * u) = u32x4{
                        pack_bf16(c[8 * u] * f, c[8 * u + 1] * f), pack_bf16(c[8 * u + 2] * f, c[8 * u + 3] * f),
                        pack_bf16(c[8 * u + 4] * f, c[8 * u + 5] * f), pack_bf16(c[8 * u + 6] * f, c[8 * u + 7] * f)};
                }
        }
        if (TAIL && lane < 32) {
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const int r = row0 + 16 * h + (lane & 15);
                const f32x4& c = tacc[g][h];
                if (r < T) {
                    uint32_t* p = reinterpret_cast<uint32_t*>(x + (size_t)r * D + 64 + 4 * (lane >> 4));
                    p[0] = pack_bf16(c[0] * f, c[1] * f);
                    p[1] = pack_bf16(c[2] * f, c[3] * f);
                }
            }
        }
    }
};

// The ring of NS stages of BS rows of X and Y (and, VALS, of their logs and -deltas) that W waves fill and read: stage
// s + NS - 1 is asked for when all waves are through s - 1, whose place it takes.  The first half of the waves loads X,
// the other half Y (a lone wave both), the first wave the row values.  Rows past the head's end read as zeros.
template <int D, bool VALS, int W, int BS, int NS>
struct GradRing {
    static constexpr int ROWB = 2 * D, TENSOR = BS * ROWB, STAT = 2 * TENSOR, STAGE = STAT + BS * 8;
    static constexpr int ZERO = NS * STAGE, LDS = ZERO + 64;
    static constexpr int WT = W > 1 ? W / 2 : 1;                 // waves of a tensor
    static constexpr int SL = BS * Geo<D>::SLOTS;                // its 16-byte slots
    static constexpr int FULL = SL / (64 * WT);                  // whole loads of a wave
    static constexpr int REST = (SL - FULL * 64 * WT) / WT;      // lanes of one more
    static constexpr int LOADS = (W > 1 ? 1 : 2) * (FULL + (REST ? 1 : 0));  // (and one of the row values)
    static_assert(FULL * 64 * WT + REST * WT == SL && (WT == 1 || WT % 2 == 0), "even shares");

    uint32_t lds0;
    int lane, w, wt, first;
    int from[2];  // a lane's source offset in an even and in an odd kilobyte of a stage
    int from_st;
    i32x4 rs[2], st;

    __device__ __forceinline__ void init(lds_u8* lds, const uint16_t* x, const uint16_t* y, const float* vals,
                                         int T, int T64) {
        lds0 = (uint32_t)(uintptr_t)lds;
        lane = threadIdx.x & 63;
        w = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
        first = W > 1 ? w / WT : 0;
        wt = W > 1 ? w % WT : 0;
        rs[0] = buffer_rsrc(x, T * ROWB);
        rs[1] = buffer_rsrc(y, T * ROWB);
        // lanes of the first half of BS values take logs, the others -deltas
        if (VALS) {
            st = buffer_rsrc(vals, T64 * 8);
            from_st = lane < BS / 4 ? lane * 16 : T64 * 4 + (lane - BS / 4) * 16;
        }
#pragma unroll
        for (int p = 0; p < 2; ++p)
            from[p] = Geo<D>::SWZ ? (lane >> 3) * ROWB + (((lane & 7) ^ swz<D>((lane >> 3) | (p << 3))) * 16) : lane * 16;
        if (threadIdx.x < 4) *(lds_u32x4*)(lds + ZERO + 16 * threadIdx.x) = u32x4{};
    }
    // the stage of rows row0 .. (none for a negative one: zeros) into the ring's place at LDS offset `to`
    __device__ __forceinline__ void load(int to, int row0) {
        const int at = row0 < 0 ? kOff : row0 * ROWB, at4 = row0 < 0 ? kOff : row0 * 4;
#pragma unroll
        for (int i = 0; i < (W > 1 ? 1 : 2); ++i) {
            const int y = W > 1 ? first : i;
            const i32x4 r = y ? rs[1] : rs[0];
            const uint32_t dst = lds0 + to + y * TENSOR;
#pragma unroll
            for (int n = 0; n < FULL; ++n) {
                const int kb = n * WT + wt;
                dma16(__builtin_amdgcn_readfirstlane(dst + kb * 1024), (WT > 1 ? (wt & 1 ? from[1] : from[0]) : from[n & 1]) + at + kb * 1024, r);
            }
            if (REST) {
                const int b = FULL * WT * 1024 + wt * REST * 16;
                if (lane < REST) dma16(__builtin_amdgcn_readfirstlane(dst + b), from[0] + at + b, r);
            }
        }
        if (VALS && w == 0 && lane < BS / 2)
            dma16(__builtin_amdgcn_readfirstlane(lds0 + to + STAT), from_st + at4, st);
    }
    // the oldest of NS - 1 stages asked for has landed, and every wave is through the stage before it
    __device__ __forceinline__ void turn() {
        if (VALS && w == 0)
            wait_vm<(NS - 2) * (LOADS + 1)>();
        else
            wait_vm<(NS - 2) * LOADS>();
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        if (W > 1) __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
    }
};

}  // namespace
}  // namespace rt
