// A unit of work of the kernels that go over heads: 16 elements of one head of a token in a thread, eight of each half where halves are
// paired by the rotation, else 16 neighbours.
#pragma once

#include "peqa_device.h"

namespace peqa {

struct Eight {
    float x[8];
};

__device__ __forceinline__ Eight eight(u32x4 v)
{
    Eight e;
#pragma unroll
    for (int i = 0; i < 4; ++i) { e.x[2 * i] = bf16_lo(v[i]); e.x[2 * i + 1] = bf16_hi(v[i]); }
    return e;
}

__device__ __forceinline__ u32x4 to_bf16(const Eight &e)
{
    u32x4 v;
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = pack_bf16x2(e.x[2 * i], e.x[2 * i + 1]);
    return v;
}

// x / scale to 8-bit floats, nearest even, past the largest finite value to it; NaN stays NaN.  The quotient is the product with the
// reciprocal and one correction by its remainder, three instructions for the eleven of a division (half of the vector instructions of
// keys and values); a quotient that is infinite has no remainder.
__device__ __forceinline__ u32x2 to_fp8(const Eight &e, float scale, float inverse)
{
    float y[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const float first = e.x[i] * inverse, d = fabsf(first) < 1024.f ? fmaf(fmaf(-first, scale, e.x[i]), inverse, first) : first;
        y[i] = d != d ? d : fminf(fmaxf(d, -448.f), 448.f);
    }
    u32x2 v;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        int w = __builtin_amdgcn_cvt_pk_fp8_f32(y[4 * i], y[4 * i + 1], 0, false);
        v[i] = (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(y[4 * i + 2], y[4 * i + 3], w, true);
    }
    return v;
}

// Cosines and sines of the eight pairs of unit `part` at a position: rows of the tables have `units` units.
struct Angles {
    float c[8], s[8];
};
__device__ __forceinline__ Angles angles(const float *cos_table, const float *sin_table, int pos, int units, int part)
{
    const size_t row = (size_t)pos * (size_t)(units * 8) + (size_t)(part * 8);
    Angles a;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const f32x4 cv = *reinterpret_cast<const f32x4 *>(cos_table + row + 4 * i);
        const f32x4 sv = *reinterpret_cast<const f32x4 *>(sin_table + row + 4 * i);
#pragma unroll
        for (int j = 0; j < 4; ++j) { a.c[4 * i + j] = cv[j]; a.s[4 * i + j] = sv[j]; }
    }
    return a;
}

// The unit's pairs turned: (a, b) -> (a c - b s, a s + b c); BACK: by the transposed matrix.
template <bool INTERLEAVED, bool BACK = false> __device__ __forceinline__ void turn(Eight &e0, Eight &e1, const Angles &t)
{
    if (INTERLEAVED) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const float a0 = e0.x[2 * i], b0 = e0.x[2 * i + 1], a1 = e1.x[2 * i], b1 = e1.x[2 * i + 1];
            const float s0 = BACK ? -t.s[i] : t.s[i], s1 = BACK ? -t.s[4 + i] : t.s[4 + i];
            e0.x[2 * i] = fmaf(a0, t.c[i], -(b0 * s0));
            e0.x[2 * i + 1] = fmaf(a0, s0, b0 * t.c[i]);
            e1.x[2 * i] = fmaf(a1, t.c[4 + i], -(b1 * s1));
            e1.x[2 * i + 1] = fmaf(a1, s1, b1 * t.c[4 + i]);
        }
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const float p = e0.x[i], r = e1.x[i], s = BACK ? -t.s[i] : t.s[i];
            e0.x[i] = fmaf(p, t.c[i], -(r * s));
            e1.x[i] = fmaf(p, s, r * t.c[i]);
        }
    }
}

// The sum over the 2^shift lanes (4, 8 or 16 neighbours) that have a head's units, in all of them.
template <int CTRL> __device__ __forceinline__ float add_moved(float v)
{
    return v + __uint_as_float(__builtin_amdgcn_update_dpp(0, __float_as_uint(v), CTRL, 0xF, 0xF, true));
}
__device__ __forceinline__ float over_head(float v, int shift)
{
    v = add_moved<0xB1>(v);                                // quad_perm 1, 0, 3, 2
    v = add_moved<0x4E>(v);                                // quad_perm 2, 3, 0, 1
    if (shift > 2) v = add_moved<0x141>(v);                // row_half_mirror: the other four of eight
    if (shift > 3) v = add_moved<0x140>(v);                // row_mirror: the other eight of sixteen
    return v;
}

// One over the root mean square of a head, of which the unit has 16 elements.
__device__ __forceinline__ float inverse_rms(const Eight &e0, const Eight &e1, int shift, float eps)
{
    float sum = 0.f;
#pragma unroll
    for (int i = 0; i < 8; ++i) sum = fmaf(e0.x[i], e0.x[i], fmaf(e1.x[i], e1.x[i], sum));
    return rsqrtf(over_head(sum, shift) * (1.f / (float)(16 << shift)) + eps);
}

// Eight of a head's fp32 weights; none are ones.
__device__ __forceinline__ Eight weights_at(const float *w, int at)
{
    Eight e;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const f32x4 v = w ? *reinterpret_cast<const f32x4 *>(w + at + 4 * i) : f32x4{1.f, 1.f, 1.f, 1.f};
#pragma unroll
        for (int j = 0; j < 4; ++j) e.x[4 * i + j] = v[j];
    }
    return e;
}

}  // namespace peqa
