// Gradients of attention (gfx950, CDNA4): dQ, dK, dV of dense and block-sparse attention, with or without the
// reshape's factor, the probabilities recomputed from the forward call's row statistics.
//
//   grad_rows  per query row: delta = dO . O, and log2 of the denominator over the row's factor
//   grad_kv    a wave per 32 NT keys walks the queries:
//                S = Q K^T, P = exp2(c S - row_log), dP = dO V^T, dS = P (dP - delta)
//                dV^T += dO^T P,  dK^T += Q^T dS
//   grad_q     a wave per 32 NT queries walks the keys:
//                S^T = K Q^T, P^T, dP^T = V dO^T, dS^T;  dQ^T += K^T dS^T
//
// Seven products of T x T x D instead of the five that the gradients need: the scores and dP are formed twice, so
// that every sum stays in one wave's registers, with no atomics and equal bits from equal calls.
//
// Layouts.  The 32x32x16 accumulator of S hands each lane 16 rows of one column, which are exactly the 8 + 8
// contraction values that the B operand of the next product takes, so P and dS never leave registers; what the
// walk streams (Q and dO, or K and V) goes through LDS in 32-row chunks and is read twice, as rows for the scores
// and transposed for the gradients.

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "attn_common.h"
#include "kernels.h"

namespace rt {
namespace {

__device__ __forceinline__ f32x16 mma(const bf16x8& x, const bf16x8& y, const f32x16& z) {
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(x, y, z, 0, 0, 0);
}

// ---- rows ----------------------------------------------------------------------------------

template <int CTRL>
__device__ __forceinline__ float dpp(float x) {
    return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(x), CTRL, 0xf, 0xf, true));
}

// 8 lanes a row; of a 72-wide row the first takes the last 8 elements too
template <int D>
__global__ __launch_bounds__(256) void grad_rows(GradArgs a, int64_t rows) {
    const int64_t row = ((int64_t)blockIdx.x * 256 + threadIdx.x) >> 3;
    const int c = threadIdx.x & 7;
    if (row >= rows) return;
    float s = 0.f;
    auto add = [&](int ch) {
        const size_t at = (size_t)row * D + 8 * ch;
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
    s += dpp<0x141>(s);
    if (c == 0) {
        float log = __builtin_fmaf(a.row_max[row], 1.44269504f, log2f(a.row_sum[row]));
        if (a.rho) {
            const float r = a.rho[row] + a.rho_delta;
            log -= log2f(fminf(1.0f, r));  // a factor of 0: +inf, no probability
            if (a.d_rho) a.d_rho[row] = r <= 1.0f ? s : 0.f;
        }
        a.row_log[row] = log;
        a.row_delta[row] = s;
    }
}

// ---- the walks -----------------------------------------------------------------------------

// 16-byte slot of a row in LDS: both the 8 consecutive rows of a row read and the 4 of a transposed one, which
// touches slots s and s ^ 2, fall on different banks
template <int D>
__device__ __forceinline__ int swz(int r) {
    return Geo<D>::SWZ ? ((r & 2) << 1) | ((r & 4) >> 1) | (r & 1) : 0;
}

// Geometry of the streamed rows: 32-row chunks of two tensors, two buffers, W waves that share them.
template <int D, int W>
struct Walk {
    using G = Geo<D>;
    static constexpr int ROWB = 2 * D;
    static constexpr int SIZE = 32 * ROWB;                          // one tensor's chunk
    static constexpr int SLOTS = 32 * G::SLOTS;                     // its 16-byte slots
    static constexpr int PER = (2 * SLOTS + 64 * W - 1) / (64 * W); // a thread's slots of both tensors
    static constexpr int KS = (D + 15) / 16;                        // k-steps of a score
    static constexpr int DT = (D + 31) / 32;                        // 32-row tiles of a gradient
    static constexpr int ZERO = 4 * SIZE;                           // 16 zero bytes
    static constexpr int STAT = ZERO + 64;                          // grad_kv: [2][2][32] row values
    static constexpr int LDS = STAT + 512;                          // (reads of a tile past row 31 end in here)

    lds_u8* lds;
    int lane, l32, hi;
    int rd, tr;
    u32x4 next[PER];

    __device__ __forceinline__ void init(unsigned char* smem) {
        lds = (lds_u8*)smem;
        lane = threadIdx.x & 63;
        l32 = lane & 31;
        hi = lane >> 5;
        // a lane's reads, see attn_tiles.h: row l32, and rows 4 hi + L / 4 (+ 8) transposed
        rd = l32 * ROWB + ((hi ^ swz<D>(l32)) * 16);
        const int L = lane & 15;
        const int r = 4 * hi + (L >> 2), d = 16 * (L & 1) + 8 * ((lane >> 4) & 1) + 4 * ((L >> 1) & 1);
        tr = r * ROWB + (((d >> 3) ^ swz<D>(r)) * 16) + (d & 7) * 2;
        if (threadIdx.x < 4) *(lds_u32x4*)(lds + ZERO + 16 * threadIdx.x) = u32x4{};
    }
    // rows row0 .. + 31 of tensors x and y on their way into registers; rows past T read as zeros
    __device__ __forceinline__ void fetch(__amdgpu_buffer_rsrc_t x, __amdgpu_buffer_rsrc_t y, int row0) {
#pragma unroll
        for (int n = 0; n < PER; ++n) {
            const int i = threadIdx.x + n * 64 * W;
            const bool second = i >= SLOTS;
            const int off = row0 * ROWB + (second ? i - SLOTS : i) * 16;
            if (i < 2 * SLOTS) next[n] = __builtin_amdgcn_raw_buffer_load_b128(second ? y : x, off, 0, 0);
        }
    }
    // and from there into buffer b
    __device__ __forceinline__ void put(int b) {
#pragma unroll
        for (int n = 0; n < PER; ++n) {
            const int i = threadIdx.x + n * 64 * W;
            const bool second = i >= SLOTS;
            const int j = second ? i - SLOTS : i, r = j / G::SLOTS, slot = j - r * G::SLOTS;
            if (i < 2 * SLOTS)
                *(lds_u32x4*)(lds + (2 * b + second) * SIZE + r * ROWB + ((slot ^ swz<D>(r)) * 16)) = next[n];
        }
    }
    // rows operand of k-step s of buffer b's tensor x: row l32, dims 16 s + 8 hi ..; a 72-wide row's last step has
    // zeros in its upper half, in both operands
    __device__ __forceinline__ bf16x8 rows(int b, int x, int s) const {
        const lds_u8* p = lds + (2 * b + x) * SIZE;
        if (D == 72 && s == 4) return *(const lds_bf16x8*)(hi ? lds + ZERO : p + rd + 128);
        return *(const lds_bf16x8*)(p + (G::SWZ ? rd ^ (32 * s) : rd + 32 * s));
    }
    // transposed operand (dims of tile dt) x (rows 16 ks ..); a lane's 16 accumulators of a product with it are dims
    // 32 dt + 16 hi .. (of a 72-wide head's tile 2 the first 8 in lanes of the lower half, the others unused)
    __device__ __forceinline__ bf16x8 cols(int b, int x, int dt, int ks) const {
        const lds_u8* p = lds + (2 * b + x) * SIZE + 16 * ks * ROWB + (G::SWZ ? tr ^ (64 * dt) : tr + 64 * dt);
        const bf16x4 v0 = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((lds_bf16x4*)p);
        const bf16x4 v1 = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((lds_bf16x4*)(p + 8 * ROWB));
        return __builtin_shufflevector(v0, v1, 0, 1, 2, 3, 4, 5, 6, 7);
    }
};

// operand held by a wave throughout: row `row` (zeros past T), dims 16 s + 8 hi ..
template <int D>
__device__ __forceinline__ bf16x8 own_row(__amdgpu_buffer_rsrc_t x, int row, int s, int hi) {
    const int off = (D == 72 && s == 4 && hi) ? kOob : row * 2 * D + 32 * s + 16 * hi;
    return __builtin_bit_cast(bf16x8, __builtin_amdgcn_raw_buffer_load_b128(x, off, 0, 0));
}

template <int D>
__device__ __forceinline__ __amdgpu_buffer_rsrc_t head_of(const uint16_t* x, size_t head_off, int T) {
    return __builtin_amdgcn_make_buffer_rsrc((void*)(x + head_off), (short)0, T * D * 2, 0x00020000);
}

__device__ __forceinline__ bf16x8 operand(const uint32_t (&p)[8], int ks) {
    return __builtin_bit_cast(bf16x8, u32x4{p[4 * ks], p[4 * ks + 1], p[4 * ks + 2], p[4 * ks + 3]});
}

// 32 rows' gradients times f from accumulators: lane's row `row`, dims 32 dt + 16 hi ..
template <int D>
__device__ __forceinline__ void store_rows(uint16_t* x, int row, int T, int hi, const f32x16* acc, float f) {
    if (row >= T) return;
#pragma unroll
    for (int dt = 0; dt < (D + 31) / 32; ++dt)
#pragma unroll
        for (int u = 0; u < 2; ++u) {
            const int d = 32 * dt + 16 * hi + 8 * u;
            if (d >= D) continue;
            const f32x16& c = acc[dt];
            *reinterpret_cast<u32x4*>(x + (size_t)row * D + d) =
                u32x4{pack_bf16(c[8 * u] * f, c[8 * u + 1] * f), pack_bf16(c[8 * u + 2] * f, c[8 * u + 3] * f),
                      pack_bf16(c[8 * u + 4] * f, c[8 * u + 5] * f), pack_bf16(c[8 * u + 6] * f, c[8 * u + 7] * f)};
        }
}

// The blocks that a wave walks: all of them, or a CSR row's (offsets clamped to the array).
template <bool DENSE>
struct List {
    const int32_t* idx;
    int n, n_blk;
    bool bad;
    __device__ __forceinline__ void init(const GradArgs& a, const int32_t* ptr, const int32_t* col, int nnz, int bh,
                                         int blk) {
        n_blk = a.n_blk;
        bad = false;
        if (DENSE) {
            n = n_blk;
            return;
        }
        const int mid = a.n_masks <= 1 ? 0 : (a.n_masks == a.heads ? bh % a.heads : bh);
        const int32_t* p = ptr + (size_t)mid * (n_blk + 1) + blk;
        int b = p[0], e = p[1];
        bad = b < 0;
        b = b < 0 ? 0 : (b > nnz ? nnz : b);
        e = e < b ? b : (e > nnz ? nnz : e);
        idx = col + b;
        n = e - b;
    }
    __device__ __forceinline__ int operator[](int i) const {  // a block past the last one for an index out of range
        if (DENSE) return i;
        const int c = idx[i];
        return c < 0 || c > n_blk ? n_blk : c;
    }
};

// D, tiles of 32 keys a wave, waves of a workgroup (they share a dense walk)
template <int D, int NT, int W, bool DENSE>
__global__ __launch_bounds__(64 * W) void grad_kv(GradArgs a, int n_items, int per_xcd) {
    using Wk = Walk<D, W>;
    __shared__ __attribute__((aligned(128))) unsigned char smem[Wk::LDS];
    constexpr int BS = 32 * NT;
    const int item = (blockIdx.x & 7) * per_xcd + (blockIdx.x >> 3);
    if (item >= n_items) return;
    const int T = a.T, n_tile = (a.n_blk + W - 1) / W;
    const int bh = item / n_tile, w = threadIdx.x >> 6, blk = (item - bh * n_tile) * W + w;
    const size_t head_off = (size_t)bh * (size_t)T * D, stat_off = (size_t)bh * T;
    const auto q_rs = head_of<D>(a.q, head_off, T), do_rs = head_of<D>(a.d_o, head_off, T);
    const auto k_rs = head_of<D>(a.k, head_off, T), v_rs = head_of<D>(a.v, head_off, T);
    Wk wk;
    wk.init(smem);
    List<DENSE> list;
    list.init(a, a.t_row_ptr, a.t_col_idx, a.t_nnz, bh, blk);

    bf16x8 kop[NT][Wk::KS], vop[NT][Wk::KS];
    f32x16 dk[NT][Wk::DT], dv[NT][Wk::DT];
#pragma unroll
    for (int t = 0; t < NT; ++t) {
#pragma unroll
        for (int s = 0; s < Wk::KS; ++s) {
            kop[t][s] = own_row<D>(k_rs, blk * BS + 32 * t + wk.l32, s, wk.hi);
            vop[t][s] = own_row<D>(v_rs, blk * BS + 32 * t + wk.l32, s, wk.hi);
        }
#pragma unroll
        for (int d = 0; d < Wk::DT; ++d) dk[t][d] = dv[t][d] = f32x16{};
    }

    const int n_chunk = list.n * NT;
    auto row_of = [&](int c) { return list[c / NT] * BS + (c % NT) * 32; };
    // row values of a chunk: threads 0 .. 31 row_log (+inf past T: no probability), 32 .. 63 delta
    float stat = 0.f;
    auto fetch_stat = [&](int row0) {
        const int row = row0 + wk.l32;
        if (threadIdx.x < 32)
            stat = row < T ? a.row_log[stat_off + row] : INFINITY;
        else if (threadIdx.x < 64)
            stat = row < T ? a.row_delta[stat_off + row] : 0.f;
    };
    auto put_stat = [&](int b) {
        if (threadIdx.x < 64)
            *(__attribute__((address_space(3))) float*)(wk.lds + Wk::STAT + b * 256 + threadIdx.x * 4) = stat;
    };
    if (n_chunk > 0) {
        wk.fetch(q_rs, do_rs, row_of(0));
        fetch_stat(row_of(0));
        wk.put(0);
        put_stat(0);
    }
    __syncthreads();
    for (int c = 0; c < n_chunk; ++c) {
        const int b = c & 1;
        if (c + 1 < n_chunk) {
            wk.fetch(q_rs, do_rs, row_of(c + 1));
            fetch_stat(row_of(c + 1));
        }
        // a lane's rows 8 j + 4 hi + i
        float log[16], delta[16];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const u32x4 x = *(const lds_u32x4*)(wk.lds + Wk::STAT + b * 256 + (8 * j + 4 * wk.hi) * 4);
            const u32x4 y = *(const lds_u32x4*)(wk.lds + Wk::STAT + b * 256 + 128 + (8 * j + 4 * wk.hi) * 4);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                log[4 * j + i] = __uint_as_float(x[i]);
                delta[4 * j + i] = __uint_as_float(y[i]);
            }
        }
        uint32_t p[NT][8], ds[NT][8];
#pragma unroll
        for (int t = 0; t < NT; ++t) {
            f32x16 sc = {}, dp = {};
#pragma unroll
            for (int s = 0; s < Wk::KS; ++s) sc = mma(wk.rows(b, 0, s), kop[t][s], sc);
#pragma unroll
            for (int s = 0; s < Wk::KS; ++s) dp = mma(wk.rows(b, 1, s), vop[t][s], dp);
#pragma unroll
            for (int x = 0; x < 16; x += 2) {
                const float e0 = __builtin_amdgcn_exp2f(__builtin_fmaf(sc[x], a.scale_log2, -log[x]));
                const float e1 = __builtin_amdgcn_exp2f(__builtin_fmaf(sc[x + 1], a.scale_log2, -log[x + 1]));
                p[t][x / 2] = pack_bf16(e0, e1);
                ds[t][x / 2] = pack_bf16(e0 * (dp[x] - delta[x]), e1 * (dp[x + 1] - delta[x + 1]));
            }
        }
#pragma unroll
        for (int ks = 0; ks < 2; ++ks)
#pragma unroll
            for (int d = 0; d < Wk::DT; ++d) {
                const bf16x8 xo = wk.cols(b, 1, d, ks), xq = wk.cols(b, 0, d, ks);
#pragma unroll
                for (int t = 0; t < NT; ++t) {
                    dv[t][d] = mma(xo, operand(p[t], ks), dv[t][d]);
                    dk[t][d] = mma(xq, operand(ds[t], ks), dk[t][d]);
                }
            }
        if (c + 1 < n_chunk) {
            wk.put(b ^ 1);
            put_stat(b ^ 1);
        }
        __syncthreads();
    }
    const float f = list.bad ? NAN : 1.0f;  // a transpose that did not fit its array
#pragma unroll
    for (int t = 0; t < NT; ++t) {
        const int row = blk * BS + 32 * t + wk.l32;
        store_rows<D>(a.dk + head_off, row, T, wk.hi, dk[t], a.scale_nat * f);
        store_rows<D>(a.dv + head_off, row, T, wk.hi, dv[t], f);
    }
}

template <int D, int NT, int W, bool DENSE>
__global__ __launch_bounds__(64 * W) void grad_q(GradArgs a, int n_items, int per_xcd) {
    using Wk = Walk<D, W>;
    __shared__ __attribute__((aligned(128))) unsigned char smem[Wk::LDS];
    constexpr int BS = 32 * NT;
    const int item = (blockIdx.x & 7) * per_xcd + (blockIdx.x >> 3);
    if (item >= n_items) return;
    const int T = a.T, n_tile = (a.n_blk + W - 1) / W;
    const int bh = item / n_tile, w = threadIdx.x >> 6, blk = (item - bh * n_tile) * W + w;
    const size_t head_off = (size_t)bh * (size_t)T * D, stat_off = (size_t)bh * T;
    const auto q_rs = head_of<D>(a.q, head_off, T), do_rs = head_of<D>(a.d_o, head_off, T);
    const auto k_rs = head_of<D>(a.k, head_off, T), v_rs = head_of<D>(a.v, head_off, T);
    Wk wk;
    wk.init(smem);
    List<DENSE> list;
    list.init(a, a.row_ptr, a.col_idx, a.nnz, bh, blk);

    bf16x8 qop[NT][Wk::KS], oop[NT][Wk::KS];
    f32x16 dq[NT][Wk::DT];
    float log[NT], delta[NT];
#pragma unroll
    for (int t = 0; t < NT; ++t) {
        const int row = blk * BS + 32 * t + wk.l32;
        log[t] = row < T ? a.row_log[stat_off + row] : INFINITY;
        delta[t] = row < T ? a.row_delta[stat_off + row] : 0.f;
#pragma unroll
        for (int s = 0; s < Wk::KS; ++s) {
            qop[t][s] = own_row<D>(q_rs, row, s, wk.hi);
            oop[t][s] = own_row<D>(do_rs, row, s, wk.hi);
        }
#pragma unroll
        for (int d = 0; d < Wk::DT; ++d) dq[t][d] = f32x16{};
    }

    const int n_chunk = list.n * NT;
    auto row_of = [&](int c) { return list[c / NT] * BS + (c % NT) * 32; };
    if (n_chunk > 0) {
        wk.fetch(k_rs, v_rs, row_of(0));
        wk.put(0);
    }
    __syncthreads();
    for (int c = 0; c < n_chunk; ++c) {
        const int b = c & 1, row0 = row_of(c);
        if (c + 1 < n_chunk) wk.fetch(k_rs, v_rs, row_of(c + 1));
        uint32_t ds[NT][8];
#pragma unroll
        for (int t = 0; t < NT; ++t) {
            f32x16 sc = {}, dp = {};
#pragma unroll
            for (int s = 0; s < Wk::KS; ++s) sc = mma(wk.rows(b, 0, s), qop[t][s], sc);
#pragma unroll
            for (int s = 0; s < Wk::KS; ++s) dp = mma(wk.rows(b, 1, s), oop[t][s], dp);
            if (row0 + 32 > T) {  // keys past T have no probability
#pragma unroll
                for (int x = 0; x < 16; ++x)
                    if (row0 + 8 * (x >> 2) + 4 * wk.hi + (x & 3) >= T) {
                        sc[x] = -INFINITY;
                        dp[x] = 0.f;
                    }
            }
#pragma unroll
            for (int x = 0; x < 16; x += 2) {
                const float e0 = __builtin_amdgcn_exp2f(__builtin_fmaf(sc[x], a.scale_log2, -log[t]));
                const float e1 = __builtin_amdgcn_exp2f(__builtin_fmaf(sc[x + 1], a.scale_log2, -log[t]));
                ds[t][x / 2] = pack_bf16(e0 * (dp[x] - delta[t]), e1 * (dp[x + 1] - delta[t]));
            }
        }
#pragma unroll
        for (int ks = 0; ks < 2; ++ks)
#pragma unroll
            for (int d = 0; d < Wk::DT; ++d) {
                const bf16x8 xk = wk.cols(b, 0, d, ks);
#pragma unroll
                for (int t = 0; t < NT; ++t) dq[t][d] = mma(xk, operand(ds[t], ks), dq[t][d]);
            }
        if (c + 1 < n_chunk) wk.put(b ^ 1);
        __syncthreads();
    }
#pragma unroll
    for (int t = 0; t < NT; ++t)
        store_rows<D>(a.dq + head_off, blk * BS + 32 * t + wk.l32, T, wk.hi, dq[t], a.scale_nat);
}

template <int D, int NT, int W, bool DENSE>
hipError_t launch_walks(GradArgs a, hipStream_t stream) {
    a.n_blk = (a.T + 32 * NT - 1) / (32 * NT);
    const int n = a.n_bh * ((a.n_blk + W - 1) / W), per = (n + 7) / 8;
    hipLaunchKernelGGL((grad_kv<D, NT, W, DENSE>), dim3(8 * per), dim3(64 * W), 0, stream, a, n, per);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL((grad_q<D, NT, W, DENSE>), dim3(8 * per), dim3(64 * W), 0, stream, a, n, per);
    return hipGetLastError();
}

template <int D>
hipError_t launch_d(const GradArgs& a, hipStream_t stream) {
    const int64_t rows = (int64_t)a.n_bh * a.T;
    hipLaunchKernelGGL((grad_rows<D>), dim3((uint32_t)((rows * 8 + 255) / 256)), dim3(256), 0, stream, a, rows);
    hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
    if (!a.row_ptr) return launch_walks<D, 2, 4, true>(a, stream);
    return a.block == 64 ? launch_walks<D, 2, 1, false>(a, stream) : launch_walks<D, 1, 1, false>(a, stream);
}

}  // namespace

hipError_t launch_attention_backward(const GradArgs& a, int D, hipStream_t stream) {
    return D == 64 ? launch_d<64>(a, stream) : launch_d<72>(a, stream);
}

}  // namespace rt
