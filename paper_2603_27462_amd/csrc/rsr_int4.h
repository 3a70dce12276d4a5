// What the kernels on 4-bit weights share: the layout of an int4 handle, its decoding, vectors as pieces, activations.
//
// M[r][c] = s[r][g] (q[r][c] - z[r][g]), g = c / group, q and z from -8 to 7.  A handle keeps
//   codes   u = q + 8 in [row group of 16][tile of 256 columns][half][lane][4 dwords], one load of 16 bytes per lane
//           and half tile.  Lane l holds row l % 16; its dword d (0..3 in the first half, 4..7 in the second) holds the
//           columns 32 d + 8 (l / 16) .. + 7 of the tile: byte b column b in its low nibble and column b + 4 in its high
//           one.  Every 32-column step of the matrix cores lies in one group of columns.
//   scales  [row group][tile][row][groups of the tile], bf16 if every scale is one, else float32
//   zeros   the same, int8, if there are any
// Scales are followed by 64 bytes that are read and not used.  The index of a scale is ((row group * tiles + tile) * 16 + row % 16)
// * groups of a tile + group, less than the bytes of the codes.
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

// ---- vectors ---------------------------------------------------------------------------------------
// Eight consecutive elements, as loaded (columns past the end: zeros).
template <typename VT>
struct Piece {
    u32x4 q[sizeof(VT) / 2];
};

template <typename VT>
__device__ __forceinline__ Piece<VT> load_whole_piece(const VT *__restrict__ at) {
    Piece<VT> p;
#pragma unroll
    for (int i = 0; i < (int)sizeof(VT) / 2; ++i)
        p.q[i] = *reinterpret_cast<const u32x4_any *>(reinterpret_cast<const unsigned char *>(at) + 16 * i);
    return p;
}

// The piece of `row` at column `col`.
template <typename VT>
__device__ __forceinline__ Piece<VT> load_piece(const VT *__restrict__ row, int col, int end) {
    Piece<VT> p = {};
    if (col + 8 <= end) {
        p = load_whole_piece<VT>(row + col);
    } else if (col < end) {
        uint32_t e[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            e[i] = 0;
            if (col + i < end)
                e[i] = sizeof(VT) == 4 ? reinterpret_cast<const uint32_t *>(row)[col + i]
                                       : reinterpret_cast<const uint16_t *>(row)[col + i];
        }
        if (sizeof(VT) == 4) {
            p.q[0] = u32x4{e[0], e[1], e[2], e[3]};
            p.q[sizeof(VT) / 2 - 1] = u32x4{e[4], e[5], e[6], e[7]};
        } else {
            p.q[0] = u32x4{e[0] | e[1] << 16, e[2] | e[3] << 16, e[4] | e[5] << 16, e[6] | e[7] << 16};
        }
    }
    return p;
}

// low half: of a, high half: of b
__device__ __forceinline__ uint32_t high_halves(uint32_t a, uint32_t b) {
    return __builtin_amdgcn_perm(b, a, 0x07060302u);
}

// Writes the piece to LDS: one plane for bf16, three (`plane` bytes apart) for float32, x = top + middle + bottom 8 bits
// exactly.
__device__ __forceinline__ void store_piece(unsigned char *at, int, const Piece<uint16_t> &p) {
    *reinterpret_cast<u32x4 *>(at) = p.q[0];
}
__device__ __forceinline__ void store_piece(unsigned char *at, int plane, const Piece<float> &p) {
    uint32_t x[8] = {p.q[0].x, p.q[0].y, p.q[0].z, p.q[0].w, p.q[1].x, p.q[1].y, p.q[1].z, p.q[1].w};
#pragma unroll
    for (int pl = 0; pl < 3; ++pl) {
        *reinterpret_cast<u32x4 *>(at + pl * plane) = u32x4{high_halves(x[0], x[1]), high_halves(x[2], x[3]),
                                                            high_halves(x[4], x[5]), high_halves(x[6], x[7])};
        if (pl < 2) {
#pragma unroll
            for (int i = 0; i < 8; ++i)
                x[i] = __float_as_uint(__uint_as_float(x[i]) - __uint_as_float(x[i] & 0xffff0000u));
        }
    }
}

// Sum of the piece's elements.
__device__ __forceinline__ float piece_sum(const Piece<uint16_t> &p) {
    float sum = 0.0f;
#pragma unroll
    for (int i = 0; i < 4; ++i)
        sum = __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2, (uint32_t)p.q[0][i]),
                                              __builtin_bit_cast(bf16x2, 0x3f803f80u), sum, false);
    return sum;
}
__device__ __forceinline__ float piece_sum(const Piece<float> &p) {
    const u32x4 a = p.q[0], b = p.q[1];
    float sum = 0.0f;
#pragma unroll
    for (int i = 0; i < 4; ++i) sum += __uint_as_float(a[i]) + __uint_as_float(b[i]);
    return sum;
}

// Sum over aligned runs of LANES (4, 8 or 16) lanes, in each of them.
template <int CTRL>
__device__ __forceinline__ float plus_moved(float x) {
    return x + __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(x), CTRL, 0xf, 0xf, true));
}
template <int LANES>
__device__ __forceinline__ float run_sum(float x) {
    x = plus_moved<0xb1>(x);                    // the neighbour
    x = plus_moved<0x4e>(x);                    // the other pair
    if (LANES >= 8) x = plus_moved<0x141>(x);   // mirrored in eight: the other quad
    if (LANES >= 16) x = plus_moved<0x140>(x);  // mirrored in sixteen
    return x;
}

// ---- weights ------------------------------------------------------------------------------------------
// Two bf16 of two bytes 0000uuuu.
__device__ __forceinline__ uint32_t low_pair(uint32_t bytes) {
    return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(bytes, 512.0f, false));
}
__device__ __forceinline__ uint32_t high_pair(uint32_t bytes) {
    return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(bytes, 512.0f, true));
}
// The eight codes of a dword as an operand.
__device__ __forceinline__ bf16x8 decode(uint32_t d) {
    const uint32_t lo = d & 0x0f0f0f0fu, hi = (d >> 4) & 0x0f0f0f0fu;
    return __builtin_bit_cast(bf16x8, u32x4{low_pair(lo), high_pair(lo), low_pair(hi), high_pair(hi)});
}

__device__ __forceinline__ bf16x8 lds_operand(const unsigned char *at) {
    return __builtin_bit_cast(bf16x8, *reinterpret_cast<const u32x4 *>(at));
}

__device__ __forceinline__ f32x4 mfma16(bf16x8 a, bf16x8 b, f32x4 acc) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, acc, 0, 0, 0);
}
__device__ __forceinline__ f32x16 mfma32(bf16x8 a, bf16x8 b, f32x16 acc) {
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, acc, 0, 0, 0);
}
// Row of the 32 x 32 result of accumulator register i in lane half h; its column is lane % 32.
__device__ __forceinline__ int acc_row(int i, int h) { return 8 * (i >> 2) + 4 * h + (i & 3); }

// N neighbouring scales and zero points of one row, as loaded: a few words more than bf16 scales have, and some bytes of
// codes where there are no zero points, rather than a branch, behind which all loads would be waited for.
typedef uint32_t u32x4_words __attribute__((ext_vector_type(4), aligned(4)));
typedef uint32_t u32x2_words __attribute__((ext_vector_type(2), aligned(4)));
typedef uint32_t u32_any __attribute__((aligned(1)));
typedef uint16_t u16_any __attribute__((aligned(1)));

template <int N>
struct Scales {
    uint32_t s[N];   // wide: each a float32; else two bf16 in each of the first N / 2 (N = 1: in either half, odd)
    uint32_t z[(N + 3) / 4];
    uint32_t odd;
};
template <int N>
__device__ __forceinline__ Scales<N> load_scales(const Int4 &m, long long idx) {
    Scales<N> r;
    const unsigned char *base = static_cast<const unsigned char *>(m.scales) + (idx << (m.wide ? 2 : 1));
    const int8_t *z = (m.zeros ? m.zeros : reinterpret_cast<const int8_t *>(m.codes)) + idx;
    r.odd = 0;
    if constexpr (N == 1) {
        r.odd = m.wide ? 0u : (uint32_t)idx & 1u;
        r.s[0] = *reinterpret_cast<const uint32_t *>(base - 2 * r.odd);
        r.z[0] = (uint8_t)z[0];
    }
    if constexpr (N == 2) {
        const u32x2 x = *reinterpret_cast<const u32x2_words *>(base);
        r.s[0] = x.x; r.s[1] = x.y;
        r.z[0] = *reinterpret_cast<const u16_any *>(z);
    }
    if constexpr (N >= 4) {
#pragma unroll
        for (int i = 0; i < N; i += 4) {
            const u32x4 x = *reinterpret_cast<const u32x4_words *>(base + 4 * i);
            r.s[i] = x.x; r.s[i + 1] = x.y; r.s[i + 2] = x.z; r.s[i + 3] = x.w;
        }
#pragma unroll
        for (int i = 0; i < N / 4; ++i) r.z[i] = *reinterpret_cast<const u32_any *>(z + 4 * i);
    }
    return r;
}
template <int N>
__device__ __forceinline__ float scale_of(const Scales<N> &r, int wide, int i) {
    const uint32_t pair = r.s[i >> 1];
    const uint32_t narrow = N == 1 ? (r.odd ? pair & 0xffff0000u : pair << 16) : i & 1 ? pair & 0xffff0000u : pair << 16;
    return __uint_as_float(wide ? r.s[i] : narrow);
}
template <int N>
__device__ __forceinline__ int zero_of(const Scales<N> &r, const Int4 &m, int i) {
    const int z = (int)__builtin_amdgcn_sbfe((int)r.z[i >> 2], 8u * (i & 3), 8u);
    return m.zeros ? z : 0;
}
// (8 + z) / 8, what the sum of -8 x is multiplied with
template <int N>
__device__ __forceinline__ float zero_factor(const Scales<N> &r, const Int4 &m, int i) {
    return 1.0f + 0.125f * (float)zero_of(r, m, i);
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
