// Rotary positions: the angle, its sine and cosine, and a pair turned by them.
// Shared by rotary.hip (readme_rotary) and kv_append.hip, whose keys have to be
// the same bits, so every sum of products is written out as the fused operation
// that it is.
#pragma once

#include "common.hpp"
#include "internal.hpp"

namespace readme {

struct Turn {
    float c, s;  // amplitude times cosine and sine
};

// Sixteen dims of a head, the part of one thread, and the eight angles of their
// pairs: chunk ch of D / 16 has the pairs 8 ch .. 8 ch + 7 if ch < rot / 16 (in
// either layout), and no pair otherwise.  Its dims are two runs of eight.
struct Chunk {
    int a, b;   // first dims of the runs
    bool turns;
};
__device__ __forceinline__ Chunk chunk_of(int ch, int rot, int layout) {
    Chunk k;
    k.turns = ch < rot / 16;
    const bool half = layout == README_ROTARY_HALF && k.turns;
    k.a = half ? 8 * ch : 16 * ch;
    k.b = half ? rot / 2 + 8 * ch : 16 * ch + 8;
    return k;
}

// The angle pos * f in fp64, less the nearest multiple n pi / 2: adding 1.5 2^52
// rounds to an integer and leaves it in the low bits; pi / 2 in two parts keeps the
// remainder exact to 2^-53 of a turn up to angles of 2^50.  Then fp32: sine and
// cosine of [-pi/4, pi/4] by their Taylor series to x^9 and x^10, whose next terms
// are below 2e-9.  Together within 2^-23 of the exact sine and cosine.
__device__ __forceinline__ Turn turn_of(double pos, double f, float amplitude, float sign) {
    constexpr double kRound = 6755399441055744.0;
    const double angle = pos * f;
    const double m = fma(angle, 0.63661977236758134308, kRound);
    const int n = (int)(uint32_t)__double_as_longlong(m);
    const double k = m - kRound;
    double r = fma(-k, 1.5707963267948965580, angle);
    r = fma(-k, 6.1232339957367658860e-17, r);
    const float x = (float)r, z = x * x;
    float s = fmaf(z, 2.7557319e-6f, -1.9841270e-4f);
    s = fmaf(z, s, 8.3333333e-3f);
    s = fmaf(z, s, -1.6666667e-1f);
    s = fmaf(z * x, s, x);
    float c = fmaf(z, -2.7557319e-7f, 2.4801587e-5f);
    c = fmaf(z, c, -1.3888889e-3f);
    c = fmaf(z, c, 4.1666667e-2f);
    c = fmaf(z * z, c, fmaf(z, -0.5f, 1.0f));
    Turn t;
    t.c = amplitude * ((n & 1) ? s : c);
    t.s = amplitude * ((n & 1) ? c : s);
    if ((n + 1) & 2) t.c = -t.c;  // quadrants 1 and 2
    if (n & 2) t.s = -t.s;        // quadrants 2 and 3
    t.s *= sign;
    return t;
}
__device__ __forceinline__ void turn_pair(const Turn& t, float& a, float& b) {
    const float bs = b * t.s, as = a * t.s;
    const float a1 = fmaf(a, t.c, -bs), b1 = fmaf(b, t.c, as);
    a = a1;
    b = b1;
}

// The chunk's sixteen values, run a first, turned by its eight angles.
__device__ __forceinline__ void turn_chunk(const Turn (&t)[8], int layout, float (&x)[16]) {
    if (layout == README_ROTARY_HALF) {
#pragma unroll
        for (int e = 0; e < 8; ++e) turn_pair(t[e], x[e], x[8 + e]);
    } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) turn_pair(t[e], x[2 * e], x[2 * e + 1]);
    }
}

// Eight consecutive values of a row as fp32.
template <int DT>
__device__ __forceinline__ void load8(const void* base, int64_t at, uint4 (&raw)[DT == README_F32 ? 2 : 1]) {
    const uint4* p = reinterpret_cast<const uint4*>(reinterpret_cast<const char*>(base) +
                                                    at * (DT == README_F32 ? 4 : 2));
#pragma unroll
    for (auto& v : raw) v = *p++;
}
template <int DT>
__device__ __forceinline__ void widen8(const uint4 (&raw)[DT == README_F32 ? 2 : 1], float* x) {
    if constexpr (DT == README_F32) {
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            x[4 * i] = __uint_as_float(raw[i].x);
            x[4 * i + 1] = __uint_as_float(raw[i].y);
            x[4 * i + 2] = __uint_as_float(raw[i].z);
            x[4 * i + 3] = __uint_as_float(raw[i].w);
        }
    } else {
        const uint32_t w[4] = {raw[0].x, raw[0].y, raw[0].z, raw[0].w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            x[2 * i] = bf16_lo(w[i]);
            x[2 * i + 1] = bf16_hi(w[i]);
        }
    }
}

// Eight fp32 values to a row's type, bf16 by the hardware conversion (nearest even).
template <int DT>
__device__ __forceinline__ void narrow8(const float* x, uint4 (&raw)[DT == README_F32 ? 2 : 1]) {
    if constexpr (DT == README_F32) {
#pragma unroll
        for (int i = 0; i < 2; ++i)
            raw[i] = make_uint4(__float_as_uint(x[4 * i]), __float_as_uint(x[4 * i + 1]),
                                __float_as_uint(x[4 * i + 2]), __float_as_uint(x[4 * i + 3]));
    } else {
        typedef float f32x2 __attribute__((ext_vector_type(2)));
        typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
        uint32_t w[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const f32x2 p = {x[2 * i], x[2 * i + 1]};
            w[i] = __builtin_bit_cast(uint32_t, __builtin_convertvector(p, bf16x2));
        }
        raw[0] = make_uint4(w[0], w[1], w[2], w[3]);
    }
}
template <int DT>
__device__ __forceinline__ void store8(void* base, int64_t at, const uint4 (&raw)[DT == README_F32 ? 2 : 1]) {
    uint4* p = reinterpret_cast<uint4*>(reinterpret_cast<char*>(base) + at * (DT == README_F32 ? 4 : 2));
#pragma unroll
    for (auto& v : raw) *p++ = v;
}

// The rotation of a call as the kernels take it.
struct RotaryArgs {
    const int32_t* pos;  // append: NULL, the position a row is stored at
    const double* freqs;
    float amplitude;
    int rot, layout, inverse;
};

// The host checks of `rot` and its kin (rotary_abi.hip), sizes before pointers.
readme_status rotary_check_sizes(int32_t D, int32_t rot, readme_rotary_layout layout,
                                 int32_t inverse, float amplitude);

hipError_t launch_rotary(readme_dtype dt, int64_t T, int H, int D, const RotaryArgs& a, const void* x,
                         int64_t ld_x, void* y, int64_t ld_y, hipStream_t s);

}  // namespace readme
