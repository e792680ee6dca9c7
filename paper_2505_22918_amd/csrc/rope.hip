// Rotary positions (gfx950): pairs of a head's elements are rotated by the angle of their token's position.
//
//   theta = position[axis of the pair] * freq[pair]
//   (a, b) -> amplitude (a cos - b sin, a sin + b cos); the gradient rotates by -theta
//
// A pair is two neighbours (interleaved) or two elements half the rotated part apart; elements past it are copied.
// The angle is formed and taken off whole turns in 64 bits, so that far positions keep theirs (in 32 bits position
// 10^6 is off by 0.06 radians); its cosine and sine are Taylor polynomials on an eighth of a turn to either side.
// They are formed once for all heads of a token: a thread holds one place of a row, 8 or 4 elements or a single pair,
// and walks over the heads, four loads ahead.  No table of cosines is read.
//
// Memory bound: each element is read once and written once.  Queries and keys of 2 samples of 30 heads, 17776 tokens, out
// of a packed projection (bf16, D = 64) 114 us, 4.8 TB/s, as a large copy; 32 heads of 16384 tokens, two thirds of 72
// rotated in halves (fp16) 36 us, 4.1 TB/s.  The first heads are asked for before the angles are formed (41 us after).

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "heads.h"
#include "train.h"

namespace rt {
namespace {

template <int TYPE>
struct Elem;
template <>
struct Elem<kBf16> {
    typedef __bf16 type;
};
template <>
struct Elem<kF16> {
    typedef _Float16 type;
};
template <>
struct Elem<kF32> {
    typedef float type;
};

// VEC consecutive elements, at their size times VEC or 16 bytes
template <int TYPE, int VEC>
struct Piece {
    typedef typename Elem<TYPE>::type E;
    static constexpr int BYTES = VEC * (int)sizeof(E), ALIGN = BYTES < 16 ? BYTES : 16;
    struct __attribute__((aligned(ALIGN))) Mem {
        E e[VEC];
    };
    Mem m;
    __device__ __forceinline__ void load(const void* p, int64_t at) {
        m = *reinterpret_cast<const Mem*>(reinterpret_cast<const E*>(p) + at);
    }
    __device__ __forceinline__ void store(void* p, int64_t at) const {
        *reinterpret_cast<Mem*>(reinterpret_cast<E*>(p) + at) = m;
    }
};

// amplitude times cosine and sine of 2 pi * turns
__device__ __forceinline__ void cos_sin(double turns, float amplitude, float& c, float& s) {
    const double r = turns - rint(turns), k = rint(4.0 * r);
    const float x = (float)(4.0 * r - k) * 1.57079633f;  // within pi / 4 of quarter k
    const float z = x * x;
    const float sn = __builtin_fmaf(
        x * z, __builtin_fmaf(z, __builtin_fmaf(z, __builtin_fmaf(z, 2.75573192e-6f, -1.98412698e-4f), 8.33333333e-3f), -1.66666667e-1f), x);
    const float cs = __builtin_fmaf(
        z, __builtin_fmaf(z, __builtin_fmaf(z, __builtin_fmaf(z, __builtin_fmaf(z, -2.75573192e-7f, 2.48015873e-5f), -1.38888889e-3f), 4.16666667e-2f), -0.5f),
        1.0f);
    const int q = (int)k;
    const float c0 = q & 1 ? sn : cs, s0 = q & 1 ? cs : sn;
    c = amplitude * ((q + 1) & 2 ? -c0 : c0);
    s = amplitude * (q & 2 ? -s0 : s0);
}

// cosine and sine of pair p (below pairs) of token `row` (counted over the samples that have positions of their own)
__device__ __forceinline__ void turn_of(const RopeArgs& a, int64_t row, int p, float& c, float& s) {
    const uint32_t ax = a.axes > 1 ? (uint32_t)a.axis[p] : 0u;  // (clamped: whatever the plan holds, positions are read)
    const int64_t at = row * a.axes + (ax < (uint32_t)a.axes ? ax : 0u);
    const double pos = a.pos_type == 0   ? (double)reinterpret_cast<const int32_t*>(a.positions)[at]
                       : a.pos_type == 1 ? (double)reinterpret_cast<const int64_t*>(a.positions)[at]
                                         : (double)reinterpret_cast<const float*>(a.positions)[at];
    cos_sin(pos * (a.freq[p] * 0.15915494309189535), a.amplitude, c, s);
    if (a.inverse) s = -s;
}

// HALF: pairs half the rotated part apart.  VEC 1: a pair, or an element past the rotated part.
template <int TYPE, bool HALF, int VEC>
__global__ __launch_bounds__(256) void rope_rows(RopeArgs a) {
    typedef typename Elem<TYPE>::type E;
    constexpr bool TWO = HALF || VEC == 1;       // a thread's pairs lie in two pieces
    constexpr int NP = TWO ? VEC : VEC / 2;      // pairs of a thread
    const int rot = 2 * a.pairs;
    const int turned = TWO ? a.pairs / VEC : 0;  // threads of a row with two pieces; the others take one
    const int items = TWO ? turned + (a.D - rot) / VEC : a.D / VEC;
    const uint32_t all = (uint32_t)a.T * (uint32_t)items, blocks = (all + 255) / 256;
    const uint32_t part = blockIdx.x / blocks, i = (blockIdx.x - part * blocks) * 256 + threadIdx.x;
    if (i >= all) return;
    const int b = part / a.groups, g = part - b * a.groups;
    const int t = i / items, item = i - t * items;
    const int64_t row = (a.per_sample ? (int64_t)b * a.T : 0) + t;
    const bool two = TWO && item < turned;
    int at0, at1 = 0, p0;  // the pieces' first elements, the first pair
    if (TWO) {
        p0 = item * VEC;
        at0 = two ? (HALF ? p0 : 2 * p0) : rot + (item - turned) * VEC;
        at1 = HALF ? a.pairs + p0 : 2 * p0 + 1;
    } else {
        at0 = item * VEC;
        p0 = at0 / 2;
    }
    const int h0 = g * a.each, h1 = h0 + a.each < a.H ? h0 + a.each : a.H;
    const int64_t xat = b * a.xs[0] + t * a.xs[2], yat = b * a.ys[0] + t * a.ys[2];
    Piece<TYPE, VEC> x[kRopeAhead], x2[kRopeAhead];
    auto ask = [&](int h) {
#pragma unroll
        for (int u = 0; u < kRopeAhead; ++u) {
            const int64_t from = xat + (h + u < h1 ? h + u : h1 - 1) * a.xs[1];
            x[u].load(a.x, from + at0);
            if (two) x2[u].load(a.x, from + at1);
        }
    };
    ask(h0);
    float c[NP], s[NP];
    if (!TWO || two) {
#pragma unroll
        for (int p = 0; p < NP; ++p)
            if (TWO || p0 + p < a.pairs) turn_of(a, row, p0 + p, c[p], s[p]);
    }
    for (int h = h0; h < h1; h += kRopeAhead) {
#pragma unroll
        for (int u = 0; u < kRopeAhead; ++u) {
            if (h + u >= h1) break;
            const int64_t to = yat + (h + u) * a.ys[1];
            if (TWO) {
                if (two) {
#pragma unroll
                    for (int p = 0; p < NP; ++p) {
                        const float m = (float)x[u].m.e[p], n = (float)x2[u].m.e[p];
                        x[u].m.e[p] = (E)__builtin_fmaf(m, c[p], -(n * s[p]));
                        x2[u].m.e[p] = (E)__builtin_fmaf(m, s[p], n * c[p]);
                    }
                    x2[u].store(a.y, to + at1);
                }
            } else {
#pragma unroll
                for (int p = 0; p < NP; ++p) {
                    if (p0 + p < a.pairs) {
                        const float m = (float)x[u].m.e[2 * p], n = (float)x[u].m.e[2 * p + 1];
                        x[u].m.e[2 * p] = (E)__builtin_fmaf(m, c[p], -(n * s[p]));
                        x[u].m.e[2 * p + 1] = (E)__builtin_fmaf(m, s[p], n * c[p]);
                    }
                }
            }
            x[u].store(a.y, to + at0);
        }
        if (h + kRopeAhead < h1) ask(h + kRopeAhead);
    }
}

template <int TYPE, bool HALF>
hipError_t launch_layout(const RopeArgs& a, dim3 grid, hipStream_t stream) {
    if constexpr (TYPE != kF32) {
        if (a.vec == 8) {
            hipLaunchKernelGGL((rope_rows<TYPE, HALF, 8>), grid, dim3(256), 0, stream, a);
            return hipGetLastError();
        }
    }
    if (a.vec == 4)
        hipLaunchKernelGGL((rope_rows<TYPE, HALF, 4>), grid, dim3(256), 0, stream, a);
    else
        hipLaunchKernelGGL((rope_rows<TYPE, HALF, 1>), grid, dim3(256), 0, stream, a);
    return hipGetLastError();
}
template <int TYPE>
hipError_t launch_type(const RopeArgs& a, dim3 grid, hipStream_t stream) {
    return a.half ? launch_layout<TYPE, true>(a, grid, stream) : launch_layout<TYPE, false>(a, grid, stream);
}

}  // namespace

hipError_t launch_rope(const RopeArgs& a, hipStream_t stream) {
    const dim3 grid((uint32_t)rope_blocks(a));
    return a.type == kBf16 ? launch_type<kBf16>(a, grid, stream)
                           : (a.type == kF16 ? launch_type<kF16>(a, grid, stream) : launch_type<kF32>(a, grid, stream));
}

}  // namespace rt
