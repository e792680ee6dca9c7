// Layer norm of rows and its gradients (gfx950).
//
//   norm_fwd   mean, rstd = (var + eps)^-1/2, xh = (x - mean) rstd, y = xh w + b
//   norm_bwd   g = dy w,  dx = rstd (g - mean(g) - xh mean(g xh)), and for each column
//              dw = sum over rows of dy xh,  db = sum over rows of dy
//   norm_join  the columns' sums from the workgroups' partial ones
//
// Memory bound: a row is read once and held in registers (as 32-bit values; the variance is taken from the
// differences to the mean, not from a sum of squares) and its result written once.  LPR lanes share a row,
// VEC consecutive elements a lane and chunk (16-byte accesses of 16-bit types), NV chunks; short rows share
// a wave, so that its accesses stay wide, and several rows are in flight for each lane.
//
// The gradient's column sums: a workgroup walks its share of the rows with one sum a lane and column in
// registers, joins its lanes and waves in a fixed order and writes one partial sum; norm_join adds those in
// a fixed order.  No atomics: equal calls give equal bits.
//
// Measured (a large copy here moves 5.1 TB/s, read and written): heads of CogVideoX-2B out of a packed projection
// (1066560 rows of 64, bf16) 60 us, 4.7 TB/s, their gradients 86 + 4 us, 4.7 TB/s; gradients of 8192 tokens of 1152 with
// weights for each sample 15.4 + 3.8 us: two or three rows to a wave, so that starting, joining and the sums' second
// pass weigh as much as the rows.  Four rows in flight instead of two and two turns of loads ahead changed nothing.

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "train.h"

namespace rt {
namespace {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));

template <int TYPE>
struct Elem;
template <>
struct Elem<kBf16> {
    typedef __bf16 type;
    typedef bf16x8 vec8;
};
template <>
struct Elem<kF16> {
    typedef _Float16 type;
    typedef f16x8 vec8;
};
template <>
struct Elem<kF32> {
    typedef float type;
};

// VEC (8 or 1) consecutive elements as they lie in memory, and as 32-bit values
template <int TYPE, int VEC>
struct Raw {
    typedef typename Elem<TYPE>::type E;
    E v;
    __device__ __forceinline__ void load(const void* p, int64_t at) { v = static_cast<const E*>(p)[at]; }
    __device__ __forceinline__ void get(float (&x)[1]) const { x[0] = (float)v; }
};
template <int TYPE>
struct Raw<TYPE, 8> {
    typedef typename Elem<TYPE>::type E;
    typename Elem<TYPE>::vec8 v;
    __device__ __forceinline__ void load(const void* p, int64_t at) {
        v = *reinterpret_cast<const typename Elem<TYPE>::vec8*>(static_cast<const E*>(p) + at);
    }
    __device__ __forceinline__ void get(float (&x)[8]) const {
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = (float)v[i];
    }
};
template <>
struct Raw<kF32, 8> {
    f32x4 a, b;
    __device__ __forceinline__ void load(const void* p, int64_t at) {
        const f32x4* e = reinterpret_cast<const f32x4*>(static_cast<const float*>(p) + at);
        a = e[0];
        b = e[1];
    }
    __device__ __forceinline__ void get(float (&x)[8]) const {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            x[i] = a[i];
            x[4 + i] = b[i];
        }
    }
};
template <int TYPE, int VEC>
__device__ __forceinline__ void load(const void* p, int64_t at, float (&x)[VEC]) {
    Raw<TYPE, VEC> r;
    r.load(p, at);
    r.get(x);
}

template <int TYPE, int VEC>
__device__ __forceinline__ void store(void* p, int64_t at, const float (&x)[VEC]) {
    typedef typename Elem<TYPE>::type E;
    E* e = static_cast<E*>(p) + at;
    if constexpr (VEC == 1) {
        e[0] = (E)x[0];
    } else if constexpr (TYPE == kF32) {
        reinterpret_cast<f32x4*>(e)[0] = f32x4{x[0], x[1], x[2], x[3]};
        reinterpret_cast<f32x4*>(e)[1] = f32x4{x[4], x[5], x[6], x[7]};
    } else {
        typename Elem<TYPE>::vec8 v;
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = (E)x[i];
        *reinterpret_cast<typename Elem<TYPE>::vec8*>(e) = v;
    }
}

// the weight or bias of VEC columns: of the rows' type or 32-bit (the same for the whole launch)
template <int TYPE, int VEC>
__device__ __forceinline__ void load_weight(const void* p, bool f32, int64_t at, float (&x)[VEC]) {
    if (f32)
        load<kF32, VEC>(p, at, x);
    else
        load<TYPE, VEC>(p, at, x);
}

template <int CTRL>
__device__ __forceinline__ float dpp(float x) {
    return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(x), CTRL, 0xf, 0xf, true));
}

// sum over groups of N lanes (a power of two up to 64), in all of them
template <int N>
__device__ __forceinline__ float lane_sum(float x) {
    if (N > 1) x += dpp<0xB1>(x);   // quad_perm 1, 0, 3, 2
    if (N > 2) x += dpp<0x4E>(x);   // quad_perm 2, 3, 0, 1
    if (N > 4) x += dpp<0x141>(x);  // row_half_mirror
    if (N > 8) x += dpp<0x140>(x);  // row_mirror
    if (N > 16) {
        auto r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
        x = __uint_as_float(r[0]) + __uint_as_float(r[1]);
    }
    if (N > 32) {
        auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
        x = __uint_as_float(r[0]) + __uint_as_float(r[1]);
    }
    return x;
}

// sum over the LPR lanes of a row, in all of them; rows of more than a wave through LDS, `slot` another one each time
template <int LPR>
__device__ __forceinline__ float row_sum(float x, float* lds, int slot) {
    x = lane_sum<(LPR < 64 ? LPR : 64)>(x);
    if constexpr (LPR > 64) {
        constexpr int WAVES = LPR / 64;
        if ((threadIdx.x & 63) == 0) lds[slot * WAVES + (threadIdx.x >> 6)] = x;
        __syncthreads();
        x = lds[slot * WAVES];
#pragma unroll
        for (int w = 1; w < WAVES; ++w) x += lds[slot * WAVES + w];
    }
    return x;
}

constexpr int threads_of(int LPR) { return LPR > 256 ? LPR : 256; }
// rows in flight for each lane, with the next ones asked for ahead in the gradient
constexpr int rows_at_once(int VEC, int NV) { return VEC * NV <= 16 ? 2 : 1; }
constexpr int bwd_rows(int VEC, int NV) { return VEC * NV <= 8 ? 2 : 1; }

// element offset of row r of a sample set's rows (r counts n0, n1, n2, the last one fastest)
__device__ __forceinline__ int64_t row_at(const NormArgs& a, const int64_t (&s)[3], uint32_t r) {
    if (a.flat) return (int64_t)r * s[2];
    const uint32_t t = r / (uint32_t)a.n2, i2 = r - t * (uint32_t)a.n2;
    const uint32_t i0 = t / (uint32_t)a.n1, i1 = t - i0 * (uint32_t)a.n1;
    return i0 * s[0] + i1 * s[1] + i2 * s[2];
}

template <int TYPE, int VEC, int LPR, int NV>
__global__ __launch_bounds__(threads_of(LPR)) void norm_fwd(NormArgs a) {
    constexpr int NT = threads_of(LPR), RPW = NT / LPR, U = rows_at_once(VEC, NV);
    __shared__ float lds[LPR > 64 ? 2 * U * (LPR / 64) : 1];
    const int lane = threadIdx.x % LPR;
    const uint32_t first = a.rows_per_set * blockIdx.y, end = first + a.rows_per_set;
    const uint32_t row0 = first + (a.turn0 + blockIdx.x) * (RPW * U) + threadIdx.x / LPR;
    float x[U][NV][VEC];
    bool there[NV];
#pragma unroll
    for (int k = 0; k < NV; ++k) there[k] = (k * LPR + lane) * VEC < a.width;
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const uint32_t r = row0 + u * RPW;
        const int64_t at = row_at(a, a.xs, r < end ? r : end - 1);
#pragma unroll
        for (int k = 0; k < NV; ++k) {
#pragma unroll
            for (int e = 0; e < VEC; ++e) x[u][k][e] = 0.f;
            if (there[k]) load<TYPE, VEC>(a.x, at + (k * LPR + lane) * VEC, x[u][k]);
        }
    }
    float mean[U], rstd[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
        float s = 0.f;
#pragma unroll
        for (int k = 0; k < NV; ++k)
#pragma unroll
            for (int e = 0; e < VEC; ++e) s += x[u][k][e];
        mean[u] = row_sum<LPR>(s, lds, 2 * u) / a.width;
        s = 0.f;
#pragma unroll
        for (int k = 0; k < NV; ++k)
#pragma unroll
            for (int e = 0; e < VEC; ++e) {
                const float d = x[u][k][e] - mean[u];
                if (there[k]) s = __builtin_fmaf(d, d, s);
            }
        rstd[u] = 1.0f / sqrtf(row_sum<LPR>(s, lds, 2 * u + 1) / a.width + a.eps);
    }
    const int64_t wat = (int64_t)blockIdx.y * a.width;
#pragma unroll
    for (int k = 0; k < NV; ++k) {
        if (!there[k]) continue;
        const int col = (k * LPR + lane) * VEC;
        float w[VEC], b[VEC];
#pragma unroll
        for (int e = 0; e < VEC; ++e) {
            w[e] = 1.f;
            b[e] = 0.f;
        }
        if (a.weight) load_weight<TYPE, VEC>(a.weight, a.weight_f32, wat + col, w);
        if (a.bias) load_weight<TYPE, VEC>(a.bias, a.weight_f32, wat + col, b);
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const uint32_t r = row0 + u * RPW;
            if (r >= end) continue;
            float y[VEC];
#pragma unroll
            for (int e = 0; e < VEC; ++e) y[e] = __builtin_fmaf((x[u][k][e] - mean[u]) * rstd[u], w[e], b[e]);
            store<TYPE, VEC>(a.y, row_at(a, a.ys, r) + col, y);
        }
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
        const uint32_t r = row0 + u * RPW;
        if (lane == 0 && r < end) {
            if (a.mean_out) a.mean_out[r] = mean[u];
            if (a.rstd_out) a.rstd_out[r] = rstd[u];
        }
    }
}

// Each turn's rows are asked for a turn ahead.
template <int TYPE, int VEC, int LPR, int NV>
__global__ __launch_bounds__(threads_of(LPR)) void norm_bwd(NormArgs a) {
    constexpr int NT = threads_of(LPR), RPW = NT / LPR, U = bwd_rows(VEC, NV);
    constexpr int COLS = LPR * NV * VEC;
    constexpr int PITCH = COLS / VEC + 8;  // sums of equal places in a lane's chunks lie together: no bank conflicts
    __shared__ float lds[LPR > 64 ? 4 * U * (LPR / 64) : 2 * VEC * PITCH];
    const int lane = threadIdx.x % LPR;
    const uint32_t first = a.rows_per_set * blockIdx.y, end = first + a.rows_per_set;
    const float inv_width = 1.0f / a.width;
    bool there[NV];
    float w[NV][VEC], dw[NV][VEC], db[NV][VEC];
#pragma unroll
    for (int k = 0; k < NV; ++k) {
        const int col = (k * LPR + lane) * VEC;
        there[k] = col < a.width;
#pragma unroll
        for (int e = 0; e < VEC; ++e) {
            w[k][e] = 1.f;
            dw[k][e] = db[k][e] = 0.f;
        }
        if (there[k] && a.weight) load_weight<TYPE, VEC>(a.weight, a.weight_f32, (int64_t)blockIdx.y * a.width + col, w[k]);
    }
    Raw<TYPE, VEC> rx[U][NV], ry[U][NV];
    float rm[U], rr[U];
    auto ask = [&](uint32_t base) {
#pragma unroll
        for (int u = 0; u < U; ++u) {
            uint32_t r = first + base + threadIdx.x / LPR + u * RPW;
            r = r < end ? r : end - 1;
            const int64_t xat = row_at(a, a.xs, r), yat = row_at(a, a.ys, r);
            rm[u] = a.mean[r];
            rr[u] = a.rstd[r];
#pragma unroll
            for (int k = 0; k < NV; ++k) {
                const int col = there[k] ? (k * LPR + lane) * VEC : 0;
                rx[u][k].load(a.x, xat + col);
                ry[u][k].load(a.dy, yat + col);
            }
        }
    };
    int turn = 0;  // LDS slots of one turn stay untouched while the next one uses the others
    const uint32_t step = RPW * U * gridDim.x;
    ask(blockIdx.x * (RPW * U));
    // all threads of a workgroup take the same number of turns
    for (uint32_t base = blockIdx.x * (RPW * U); base < a.rows_per_set; base += step, turn ^= 1) {
        float x[U][NV][VEC], dy[U][NV][VEC], mean[U], rstd[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
            mean[u] = rm[u];
            rstd[u] = rr[u];
#pragma unroll
            for (int k = 0; k < NV; ++k) {
                rx[u][k].get(x[u][k]);
                ry[u][k].get(dy[u][k]);
            }
        }
        if (base + step < a.rows_per_set) ask(base + step);
#pragma unroll
        for (int u = 0; u < U; ++u) {
            const uint32_t r = first + base + threadIdx.x / LPR + u * RPW;
            float s1 = 0.f, s2 = 0.f;
#pragma unroll
            for (int k = 0; k < NV; ++k) {
                if (!there[k]) continue;
#pragma unroll
                for (int e = 0; e < VEC; ++e) {
                    const float xh = (x[u][k][e] - mean[u]) * rstd[u], g = dy[u][k][e] * w[k][e];
                    x[u][k][e] = xh;
                    s1 += g;
                    s2 = __builtin_fmaf(g, xh, s2);
                }
            }
            if (r < end) {
#pragma unroll
                for (int k = 0; k < NV; ++k) {
#pragma unroll
                    for (int e = 0; e < VEC; ++e) {
                        dw[k][e] = __builtin_fmaf(dy[u][k][e], x[u][k][e], dw[k][e]);
                        db[k][e] += dy[u][k][e];
                    }
                }
            }
            s1 = row_sum<LPR>(s1, lds, 2 * (turn * U + u)) * inv_width;
            s2 = row_sum<LPR>(s2, lds, 2 * (turn * U + u) + 1) * inv_width;
            if (r < end) {
                const int64_t at = row_at(a, a.dxs, r);
#pragma unroll
                for (int k = 0; k < NV; ++k) {
                    if (!there[k]) continue;
                    float dx[VEC];
#pragma unroll
                    for (int e = 0; e < VEC; ++e)
                        dx[e] = (__builtin_fmaf(dy[u][k][e], w[k][e], -s1) - x[u][k][e] * s2) * rstd[u];
                    store<TYPE, VEC>(a.dx, at + (k * LPR + lane) * VEC, dx);
                }
            }
        }
    }
    if (!a.dweight && !a.dbias) return;
    // one partial sum for each column of this workgroup: in the workspace, or the result where it is the only one
    const int64_t set = blockIdx.y;
    float* pw = a.dweight ? a.dweight + set * a.width : nullptr;
    float* pb = a.dbias ? a.dbias + set * a.width : nullptr;
    if (gridDim.x > 1) {
        pw = a.partial + (set * gridDim.x + blockIdx.x) * 2 * a.width;
        pb = pw + a.width;
    }
    if constexpr (LPR >= NT) {
#pragma unroll
        for (int k = 0; k < NV; ++k) {
            if (!there[k]) continue;
#pragma unroll
            for (int e = 0; e < VEC; ++e) {
                const int col = (k * LPR + lane) * VEC + e;
                if (pw) pw[col] = dw[k][e];
                if (pb) pb[col] = db[k][e];
            }
        }
    } else {
#pragma unroll
        for (int k = 0; k < NV; ++k)
#pragma unroll
            for (int e = 0; e < VEC; ++e)
#pragma unroll
                for (int d = LPR; d < 64; d *= 2) {
                    dw[k][e] += __shfl_xor(dw[k][e], d);
                    db[k][e] += __shfl_xor(db[k][e], d);
                }
        for (int wave = 0; wave < NT / 64; ++wave) {
            __syncthreads();
            if ((int)(threadIdx.x >> 6) == wave && (threadIdx.x & 63) < LPR) {
#pragma unroll
                for (int k = 0; k < NV; ++k)
#pragma unroll
                    for (int e = 0; e < VEC; ++e) {
                        const int at = e * PITCH + k * LPR + lane;
                        lds[at] = wave ? lds[at] + dw[k][e] : dw[k][e];
                        lds[VEC * PITCH + at] = wave ? lds[VEC * PITCH + at] + db[k][e] : db[k][e];
                    }
            }
        }
        __syncthreads();
        for (int col = threadIdx.x; col < a.width; col += NT) {
            const int at = col % VEC * PITCH + col / VEC;
            if (pw) pw[col] = lds[at];
            if (pb) pb[col] = lds[VEC * PITCH + at];
        }
    }
}

// sums of `parts` partial sums for each of a set's 2 * width columns (the weight's, then the bias's)
__global__ __launch_bounds__(1024) void norm_join(const float* partial, int32_t parts, int32_t width, float* dweight,
                                                  float* dbias) {
    __shared__ float lds[64][17];
    const int c = threadIdx.x & 15, slice = threadIdx.x >> 4;
    const int col = blockIdx.x * 16 + c;
    const int64_t set = blockIdx.y;
    float s = 0.f;
    if (col < 2 * width) {
        const float* p = partial + set * parts * 2 * width + col;
#pragma unroll 8
        for (int i = slice; i < parts; i += 64) s += p[(int64_t)i * 2 * width];
    }
    lds[slice][c] = s;
    __syncthreads();
    if (threadIdx.x < 16 && col < 2 * width) {
        s = 0.f;
#pragma unroll
        for (int i = 0; i < 64; ++i) s += lds[i][c];
        if (col < width) {
            if (dweight) dweight[set * width + col] = s;
        } else if (dbias) {
            dbias[set * width + col - width] = s;
        }
    }
}

// The gradients of rows in 1024 lanes spill (128 registers to a lane): 16 to 46 of them in chunks of 8, 52 to 133 one by
// one.
//
// Lanes and chunks of a row.  Rows of up to 512 elements (64 one by one) share a wave, so that its accesses stay
// full; longer ones take a wave with more chunks, and over 2048 (512) a workgroup, whose registers would else not
// hold a row and its column sums.
template <int TYPE, bool BWD, int VEC, int LPR, int NV>
hipError_t launch(NormArgs a, uint32_t parts, hipStream_t stream) {
    constexpr int NT = threads_of(LPR);
    constexpr uint32_t RPT = NT / LPR * (BWD ? bwd_rows(VEC, NV) : rows_at_once(VEC, NV));  // rows of a workgroup's turn
    const uint32_t turns = (a.rows_per_set + RPT - 1) / RPT;
    if (!BWD) {  // (a launch has less than 2^32 threads)
        constexpr uint32_t MOST = (1u << 31) / NT;
        for (a.turn0 = 0; a.turn0 < turns; a.turn0 += MOST) {
            const uint32_t n = turns - a.turn0 < MOST ? turns - a.turn0 : MOST;
            hipLaunchKernelGGL((norm_fwd<TYPE, VEC, LPR, NV>), dim3(n, a.sets), dim3(NT), 0, stream, a);
            const hipError_t e = hipGetLastError();
            if (e != hipSuccess) return e;
        }
        return hipSuccess;
    }
    hipLaunchKernelGGL((norm_bwd<TYPE, VEC, LPR, NV>), dim3(turns < parts ? turns : parts, a.sets), dim3(NT), 0, stream, a);
    hipError_t e = hipGetLastError();
    if (e == hipSuccess && turns > 1 && parts > 1 && (a.dweight || a.dbias)) {
        hipLaunchKernelGGL(norm_join, dim3((2 * a.width + 15) / 16, a.sets), dim3(1024), 0, stream, a.partial,
                           (int32_t)(turns < parts ? turns : parts), a.width, a.dweight, a.dbias);
        e = hipGetLastError();
    }
    return e;
}

template <int TYPE, bool BWD>
hipError_t launch_type(const NormArgs& a, uint32_t parts, hipStream_t s) {
    const int w = a.width;
    if (a.vec) {
        if (w <= 64) return launch<TYPE, BWD, 8, 8, 1>(a, parts, s);
        if (w <= 128) return launch<TYPE, BWD, 8, 16, 1>(a, parts, s);
        if (w <= 256) return launch<TYPE, BWD, 8, 32, 1>(a, parts, s);
        if (w <= 512) return launch<TYPE, BWD, 8, 64, 1>(a, parts, s);
        if (w <= 1024) return launch<TYPE, BWD, 8, 64, 2>(a, parts, s);
        if (w <= 1536) return launch<TYPE, BWD, 8, 64, 3>(a, parts, s);
        if (w <= 2048) return launch<TYPE, BWD, 8, 64, 4>(a, parts, s);
        if (w <= 4096) return launch<TYPE, BWD, 8, 256, 2>(a, parts, s);
        if (w <= 8192) return launch<TYPE, BWD, 8, 256, 4>(a, parts, s);
        return launch<TYPE, BWD, 8, 1024, 2>(a, parts, s);
    }
    if (w <= 16) return launch<TYPE, BWD, 1, 16, 1>(a, parts, s);
    if (w <= 64) return launch<TYPE, BWD, 1, 64, 1>(a, parts, s);
    if (w <= 128) return launch<TYPE, BWD, 1, 64, 2>(a, parts, s);
    if (w <= 256) return launch<TYPE, BWD, 1, 64, 4>(a, parts, s);
    if (w <= 512) return launch<TYPE, BWD, 1, 64, 8>(a, parts, s);
    if (w <= 2048) return launch<TYPE, BWD, 1, 256, 8>(a, parts, s);
    if (w <= 8192) return launch<TYPE, BWD, 1, 1024, 8>(a, parts, s);
    return launch<TYPE, BWD, 1, 1024, 16>(a, parts, s);
}

template <bool BWD>
hipError_t launch_any(const NormArgs& a, uint32_t parts, hipStream_t s) {
    if (a.type == kBf16) return launch_type<kBf16, BWD>(a, parts, s);
    if (a.type == kF16) return launch_type<kF16, BWD>(a, parts, s);
    return launch_type<kF32, BWD>(a, parts, s);
}

}  // namespace

hipError_t launch_norm(const NormArgs& a, hipStream_t stream) { return launch_any<false>(a, 0, stream); }

hipError_t launch_norm_backward(const NormArgs& a, int32_t parts, hipStream_t stream) {
    if (a.rows_per_set == 0) {  // sums over no rows
        hipLaunchKernelGGL(norm_join, dim3((2 * a.width + 15) / 16, a.sets), dim3(1024), 0, stream, a.partial, 0,
                           a.width, a.dweight, a.dbias);
        return hipGetLastError();
    }
    return launch_any<true>(a, (uint32_t)parts, stream);
}

}  // namespace rt
