// Norm and rotation of a head that DH / 16 lanes hold, sixteen channels each, for the kernels that store K/V in pages.
#pragma once
#include "common.h"

namespace odb {

namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
typedef float f32x8 __attribute__((ext_vector_type(8)));
template <class T> struct Vec;
template <> struct Vec<_Float16> { typedef f16x8 v8; };
template <> struct Vec<__bf16> { typedef bf16x8 v8; };
template <> struct Vec<float> { typedef f32x8 v8; };

template <class T>
__device__ __forceinline__ f32x8 load8(const T *p) {
    return __builtin_convertvector(*reinterpret_cast<const typename Vec<T>::v8 *>(p), f32x8);
}
// one rounding, to nearest even, of a value computed in 32 bits; beyond the type's range it becomes infinite
template <class T>
__device__ __forceinline__ void store8(T *p, f32x8 x) {
    *reinterpret_cast<typename Vec<T>::v8 *>(p) = __builtin_convertvector(x, typename Vec<T>::v8);
}

// First channels of a lane's two eights: in the half layout channel pair (j, j + rot / 2) sits in one lane as elements of its first and its
// second eight, in the interleaved layout (2j, 2j + 1) inside each eight.  Lanes behind the rotated part hold two neighbouring eights that
// pass through.
struct HeadLane { int c0, c1; bool turns; };
template <bool INTER>
__device__ __forceinline__ HeadLane head_lane(int l, int rot) {
    const int half = rot / 2, turning = rot / 16;               // lanes of a head that turn
    HeadLane h;
    h.turns = l < turning;
    if (INTER) { h.c0 = l * 16; h.c1 = h.c0 + 8; }
    else if (h.turns) { h.c0 = l * 8; h.c1 = h.c0 + half; }
    else { h.c0 = rot + (l - turning) * 16; h.c1 = h.c0 + 8; }
    return h;
}

__device__ __forceinline__ void load_angles(const float *t, float (&cs)[8], float (&sn)[8]) {       // eight (cos, sin)
#pragma unroll
    for (int i = 0; i < 4; i++) {
        const float4 x = *reinterpret_cast<const float4 *>(t + 4 * i);
        cs[2 * i] = x.x; sn[2 * i] = x.y; cs[2 * i + 1] = x.z; sn[2 * i + 1] = x.w;
    }
}

template <int DH>
__device__ __forceinline__ void norm_head(f32x8 &x, f32x8 &y, const float *gain, float eps, int c0, int c1) {
    constexpr int LANES = DH / 16;
    float ss = 0.f;
#pragma unroll
    for (int i = 0; i < 8; i++) ss += x[i] * x[i] + y[i] * y[i];
#pragma unroll
    for (int o = LANES / 2; o > 0; o >>= 1) ss += __shfl_xor(ss, o);
    const float r = 1.0f / sqrtf(ss / (float)DH + eps);
    const f32x8 g0 = load8(gain + c0), g1 = load8(gain + c1);
    x = x * r * g0;
    y = y * r * g1;
}

template <bool INTER>
__device__ __forceinline__ void turn_head(f32x8 &x, f32x8 &y, const float (&cs)[8], const float (&sn)[8]) {
    if (INTER) {
#pragma unroll
        for (int i = 0; i < 4; i++) {
            const float u = x[2 * i], v = x[2 * i + 1], p = y[2 * i], q = y[2 * i + 1];
            x[2 * i] = u * cs[i] - v * sn[i];
            x[2 * i + 1] = v * cs[i] + u * sn[i];
            y[2 * i] = p * cs[4 + i] - q * sn[4 + i];
            y[2 * i + 1] = q * cs[4 + i] + p * sn[4 + i];
        }
    } else {
#pragma unroll
        for (int i = 0; i < 8; i++) {
            const float u = x[i], v = y[i];
            x[i] = u * cs[i] - v * sn[i];
            y[i] = v * cs[i] + u * sn[i];
        }
    }
}

}  // namespace
}  // namespace odb
