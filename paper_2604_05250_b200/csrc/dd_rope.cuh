// Norm and rotation of one head's row, shared by dd_qk_norm_rope and dd_cache_append.
//
//   y = x / sqrt(mean(x^2) + eps) * w            (no weight: y = x)
//   (y_i, y_j) <- (y_i cos - y_j sin, y_i sin + y_j cos) for the pairs (i, j) of the first `dims` entries:
//   (i, i + dims/2), or neighbours (2i, 2i + 1); the angle of pair i at a position is entry i of that position's row in the tables.
//
// D / 16 lanes hold a row, each two chunks of 8 entries (16 bytes of bf16): the two members of a pair are then always in one lane,
// whichever the pairing, and a lane's 8 pairs take 8 neighbouring entries of the tables.  All arithmetic is fp32, in the order and with the
// roundings written here (fused where it says so, each product by itself elsewhere; nothing is left to the compiler's contraction), so that
// a row's result does not depend on which kernel computes it.
#pragma once

#include <cuda_bf16.h>
#include <stdint.h>

#include "../../include/dualdiff.h"

namespace ddrope {

struct Rotation {
    const float *cos, *sin;     // [positions, dims / 2]; dims = 0: no rotation
    int positions, dims, interleaved;
};

template <int D>
struct Lane {
    static constexpr int kLanes = D / 16;
    int a, b;                   // the lane's chunks of 8 entries
    bool rotates;
    __device__ __forceinline__ Lane(int lane, const Rotation &r)
    {
        const int half = r.dims / 16;
        rotates = lane < half;
        if (r.interleaved || !rotates) { a = 2 * lane; b = a + 1; }
        else { a = lane; b = lane + half; }
    }
};

struct Angles {
    float c[8], s[8];
};

// The angles of a lane's pairs at `position`; NaN outside the tables (the result is then NaN, and nothing is read).
__device__ __forceinline__ void load_angles(Angles &t, const Rotation &r, long position, int lane, bool rotates)
{
    if (!rotates) return;
    if (position < 0 || position >= r.positions) {
#pragma unroll
        for (int i = 0; i < 8; ++i) t.c[i] = t.s[i] = __int_as_float(0x7fffffff);
        return;
    }
    const size_t at = (size_t)position * (r.dims / 2) + 8 * lane;
    const float4 *c = reinterpret_cast<const float4 *>(r.cos + at), *s = reinterpret_cast<const float4 *>(r.sin + at);
    *reinterpret_cast<float4 *>(&t.c[0]) = __ldg(c);
    *reinterpret_cast<float4 *>(&t.c[4]) = __ldg(c + 1);
    *reinterpret_cast<float4 *>(&t.s[0]) = __ldg(s);
    *reinterpret_cast<float4 *>(&t.s[4]) = __ldg(s + 1);
}

// kMixed: as x * 1 + (-0) (exact), for a kernel whose ALU has more to do than its multipliers.  Prompts into a cache 123 -> 115 us, with packed
// products; qk_norm_rope_kernel 47.7 -> 50.
template <bool kMixed = false>
__device__ __forceinline__ void unpack(float *x, const uint4 &v)
{
    const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        if constexpr (kMixed)
            asm("{\n\t.reg .b16 l, h, one;\n\tmov.b16 one, 0x3F80;\n\tmov.b32 {l, h}, %2;\n\tfma.rn.f32.bf16 %0, l, one, 0f80000000;\n\t"
                "fma.rn.f32.bf16 %1, h, one, 0f80000000;\n\t}"
                : "=f"(x[2 * i]), "=f"(x[2 * i + 1]) : "r"(w[i]));
        else {
            x[2 * i] = __uint_as_float(w[i] << 16);
            x[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u);
        }
    }
}

__device__ __forceinline__ uint4 pack(const float *x)
{
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        __nv_bfloat162 h = __floats2bfloat162_rn(x[2 * i], x[2 * i + 1]);
        w[i] = *reinterpret_cast<uint32_t *>(&h);
    }
    return make_uint4(w[0], w[1], w[2], w[3]);
}

// x[0..7], x[8..15]: the lane's chunks.  weight: bf16 [D], or null for a row that is not normed.  any (the same in all lanes): some row
// of the warp may be; every lane then takes part in the sums.
template <int D, bool kMixed = false>
__device__ __forceinline__ void norm_rows(float (&x)[16], const __nv_bfloat16 *weight, bool any, float eps, const Lane<D> &l)
{
    if (!any) return;
    float ss = 0.f;
#pragma unroll
    for (int i = 0; i < 16; ++i) ss = __fmaf_rn(x[i], x[i], ss);
#pragma unroll
    for (int o = Lane<D>::kLanes / 2; o > 0; o /= 2) ss = __fadd_rn(ss, __shfl_xor_sync(0xFFFFFFFFu, ss, o));
    if (!weight) return;
    const float r = rsqrtf(__fmaf_rn(ss, 1.f / D, eps));
    float w[16];
    unpack<kMixed>(w, __ldg(reinterpret_cast<const uint4 *>(weight) + l.a));
    unpack<kMixed>(w + 8, __ldg(reinterpret_cast<const uint4 *>(weight) + l.b));
#pragma unroll
    for (int i = 0; i < 16; ++i) x[i] = __fmul_rn(__fmul_rn(x[i], r), w[i]);
}

template <int D>
__device__ __forceinline__ void rotate_row(float (&x)[16], const Angles &t, bool rotates, bool interleaved)
{
    if (!rotates) return;
    if (interleaved) {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const float a = x[2 * i], b = x[2 * i + 1];
            x[2 * i] = __fsub_rn(__fmul_rn(a, t.c[i]), __fmul_rn(b, t.s[i]));
            x[2 * i + 1] = __fadd_rn(__fmul_rn(a, t.s[i]), __fmul_rn(b, t.c[i]));
        }
    } else {
        // two pairs at a time, by packed instructions; p - q as q * -1 + p, the same rounding
#pragma unroll
        for (int i = 0; i < 8; i += 2) {
            const float2 a = make_float2(x[i], x[i + 1]), b = make_float2(x[8 + i], x[9 + i]), c = make_float2(t.c[i], t.c[i + 1]),
                         s = make_float2(t.s[i], t.s[i + 1]);
            const float2 u = __ffma2_rn(__fmul2_rn(b, s), make_float2(-1.f, -1.f), __fmul2_rn(a, c)), v = __fadd2_rn(__fmul2_rn(a, s), __fmul2_rn(b, c));
            x[i] = u.x; x[i + 1] = u.y;
            x[8 + i] = v.x; x[9 + i] = v.y;
        }
    }
}

// Host side: the rotation as the kernels take it.
inline int check_rotation(const dd_rotation *given, int D, Rotation &r)
{
    r = Rotation{nullptr, nullptr, 0, 0, 0};
    if (!given || given->dims == 0) return DD_OK;
    if (!given->cos || !given->sin || given->positions <= 0 || given->dims < 0) return DD_ERR_INVALID_ARG;
    if (given->dims > D || given->dims % 16 != 0) return DD_ERR_UNSUPPORTED;
    if ((((uintptr_t)given->cos | (uintptr_t)given->sin) & 15) != 0) return DD_ERR_UNSUPPORTED;
    r = Rotation{given->cos, given->sin, given->positions, given->dims, given->interleaved ? 1 : 0};
    return DD_OK;
}

}  // namespace ddrope
