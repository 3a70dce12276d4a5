// What the kernels on 4-bit weights share: the layout of an int4 handle, its decoding, vectors as pieces, activations.
//
// M[r][c] = s[r][g] (q[r][c] - z[r][g]), g = c / group, q and z from -8 to 7.  A handle keeps
//   codes   u = q + 8 in [row group of 16][tile of 256 columns][half][lane][4 dwords], one load of 16 bytes per lane
//           and half tile.  Lane l holds row l % 16; its dword d (0..3 in the first half, 4..7 in the second) holds the
//           columns 32 d + 8 (l / 16) .. + 7 of the tile: byte b column b in its low nibble and column b + 4 in its high
//           one.  Every 32-column step of the matrix cores lies in one group of columns.
//   scales  [row group][tile][row][groups of the tile], bf16 if every scale is one, else float32
//   zeros   the same, int8, if there are any
// Groups of columns are 32, 64 or 128 wide here (the widest that divides the caller's): 8, 4 or 2 per tile.
//
// A byte 0000uuuu is the 8-bit float (e4m3) u 2^-9, subnormal up to 7, so v_cvt_scalef32_pk_bf16_fp8 with scale 2^9
// makes two exact bf16 of two bytes: 7 instructions for the eight codes of a dword.  Only whole numbers and the
// elements of the vector are multiplied there, and a sum over a group is scaled afterwards, in float32, so nothing of
// a weight is rounded; sum (q - z) x = sum u x - (8 + z) sum x, with the vector's sum per group.
#pragma once

#include "rsr_internal.h"

namespace rsr {

constexpr int kInt4Tile = 256;       // columns of a tile
constexpr int kInt4Steps = 8;        // 32-column steps of a tile
constexpr int kInt4TileDwords = 512; // of 16 rows and 256 columns

// An int4 handle's arrays, as kernel arguments.
struct Int4 {
    const uint32_t *codes;
    const void *scales;
    const int8_t *zeros;  // may be null
    int wide;             // scales are float32
};

inline Int4 int4_of(const rsr_handle_s *h) {
    return {reinterpret_cast<const uint32_t *>(h->packed), h->scales, h->zeros, h->wide_scales};
}

namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
// vectors start anywhere: 16 bytes at the alignment of an element (the hardware takes any)
typedef uint32_t u32x4_any __attribute__((ext_vector_type(4), aligned(2)));

__device__ __forceinline__ float widen(float x) { return x; }
__device__ __forceinline__ float widen(uint16_t x) { return __uint_as_float((uint32_t)x << 16); }
__device__ __forceinline__ void put(float *at, float x) { *at = x; }
__device__ __forceinline__ void put(uint16_t *at, float x) { *at = __builtin_bit_cast(uint16_t, (__bf16)x); }

// Scale and zero point of (row, column): idx = ((row group * tiles + tile) * 16 + row % 16) * groups per tile + group.
__device__ __forceinline__ float scale_at(const Int4 &m, long long idx) {
    return m.wide ? static_cast<const float *>(m.scales)[idx] : widen(static_cast<const uint16_t *>(m.scales)[idx]);
}

// ---- activations --------------------------------------------------------------------------------
__device__ __forceinline__ float sigmoid(float x) { return __builtin_amdgcn_rcpf(1.0f + expf(-x)); }

constexpr float kGeluC = 0.7978845608028654f;  // sqrt(2 / pi)

// act(a).  gelu is the tanh form: 0.5 a (1 + tanh(z)) = a sigmoid(2 z).
__device__ __forceinline__ float activate(int act, float a) {
    if (act == RSR_SILU) return a * sigmoid(a);
    if (act == RSR_GELU) return a * sigmoid(2.0f * kGeluC * (a + 0.044715f * a * a * a));
    const float r = fmaxf(a, 0.0f);
    return a != a ? a : r * r;
}

// act(a) and its derivative.  1 - sigmoid(x) is sigmoid(-x), without the cancellation.
__device__ __forceinline__ float activate(int act, float a, float *slope) {
    if (act == RSR_SILU) {
        const float p = sigmoid(a);
        *slope = p * (1.0f + a * sigmoid(-a));
        return a * p;
    }
    if (act == RSR_GELU) {
        const float p = sigmoid(2.0f * kGeluC * (a + 0.044715f * a * a * a));
        // (beyond 16 the second term is zero, and a * a would overflow)
        const float b = fminf(fmaxf(a, -16.0f), 16.0f), z2 = 2.0f * kGeluC * (b + 0.044715f * b * b * b);
        *slope = p + b * sigmoid(z2) * sigmoid(-z2) * 2.0f * kGeluC * (1.0f + 0.134145f * b * b);
        return a * p;
    }
    const float r = a != a ? a : fmaxf(a, 0.0f);
    *slope = 2.0f * r;
    return r * r;
}

}  // namespace
}  // namespace rsr
