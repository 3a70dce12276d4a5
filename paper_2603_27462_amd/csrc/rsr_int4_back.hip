// Input gradients of products with 4-bit weights (gfx950): dx = scale M^T dy, the sum of two of them, and the gradient of the
// gated block's activation.
#include "rsr_int4.h"

#include <cstdio>
#include <type_traits>

namespace rsr {

namespace {

// (da, db) from (a, b) and dh, four elements of a vector per thread; dpre may be pre.  6912 x 1024, bf16 dh: 127 MB in 20 us, a large
// copy's rate.
typedef float f32x4_any __attribute__((ext_vector_type(4), aligned(4)));
typedef uint16_t u16x4_any __attribute__((ext_vector_type(4), aligned(2)));

template <typename VT>
__global__ __launch_bounds__(256) void k_gated_slopes(const float *pre, const VT *__restrict__ dh, long long ldd, int act,
                                                      int rows, float *dpre) {
    const int r = ((int)blockIdx.x * 256 + (int)threadIdx.x) * 4;
    if (r >= rows) return;
    const long long n = blockIdx.y, at = 2 * n * rows + r;
    const VT *from = dh + n * ldd + r;
    float a[4], b[4], d[4];
    const int live = min(4, rows - r);
    if (live == 4) {
        const f32x4_any x = *reinterpret_cast<const f32x4_any *>(pre + at), y = *reinterpret_cast<const f32x4_any *>(pre + at + rows);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            a[i] = x[i];
            b[i] = y[i];
        }
        if constexpr (sizeof(VT) == 4) {
            const f32x4_any z = *reinterpret_cast<const f32x4_any *>(from);
#pragma unroll
            for (int i = 0; i < 4; ++i) d[i] = z[i];
        } else {
            const u16x4_any z = *reinterpret_cast<const u16x4_any *>(from);
#pragma unroll
            for (int i = 0; i < 4; ++i) d[i] = widen((uint16_t)z[i]);
        }
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            a[i] = i < live ? pre[at + i] : 0.0f;
            b[i] = i < live ? pre[at + rows + i] : 0.0f;
            d[i] = i < live ? widen(from[i]) : 0.0f;
        }
    }
    f32x4_any da, db;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        float slope;
        const float f = activate(act, a[i], &slope);
        da[i] = d[i] * b[i] * slope;
        db[i] = d[i] * f;
    }
    if (live == 4) {
        *reinterpret_cast<f32x4_any *>(dpre + at) = da;
        *reinterpret_cast<f32x4_any *>(dpre + at + rows) = db;
    } else {
        for (int i = 0; i < live; ++i) {
            dpre[at + i] = da[i];
            dpre[at + rows + i] = db[i];
        }
    }
}

// ---- the transposed product ----------------------------------------------------------------------------
// out[n][c] = sum over r of (dy[n][r] s[r][g]) (u[r][c] - (8 + z[r][g])), g the group of c.  The sum runs over the rows, so it is dy
// that is scaled, once per group of columns, on its way into LDS: as three bf16 planes, which hold all of it, or as two where dy and
// out are both bf16 (one alone, dy s rounded to bf16, left results off by 0.0023 where rounding only them leaves 0.0017); the codes are whole numbers as ever, and sum dy s (8 + z), the same for all columns of a group, is taken off at the end.
//
// The matrix cores want eight consecutive rows of a column in a lane where the codes have eight columns of a row: they go
// through LDS, where ds_read_b64_tr_b4 turns 16 rows of 16 nibbles around within 16 lanes.  Rows are laid out there as
// 16 dwords of (32-column step, slice of 8 columns) and 8 bytes more, so that a lane's 8 bytes are 16 consecutive columns and
// 16 rows fall into different banks.  After it lane i of 16 holds column 8 (i / 8) + i % 8 / 2 + 4 (i % 2) of the 16, rows 0 to 7 in its
// first dword and 8 to 15 in its second; decoding a dword yields its rows in the order 0 2 4 6 1 3 5 7, and dy is staged in
// that order.  An MFMA takes 8 rows of each of two row groups.
typedef int i32x2 __attribute__((ext_vector_type(2)));
constexpr int kCodeRow = 72;                      // bytes of 128 columns of a row in LDS
constexpr int kCodeGroup = kDenseRows * kCodeRow; // and of a row group

__device__ __forceinline__ i32x2 turned(const unsigned char *at) {
    return __builtin_amdgcn_ds_read_tr4_b64_v2i32(
        (__attribute__((address_space(3))) i32x2 *)(reinterpret_cast<const i32x2 *>(at)));
}
// Column of lane i (of 32) within the 32 of an operand.
__device__ __forceinline__ int turned_column(int i) { return 8 * (i >> 3) + ((i & 7) >> 1) + 4 * (i & 1); }

__device__ __forceinline__ uint32_t rounded_pair(float a, float b) {
    return __builtin_bit_cast(uint32_t, bf16x2{(__bf16)a, (__bf16)b});
}

__device__ __forceinline__ void widen_piece(const Piece<uint16_t> &p, float (&x)[8]) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
        x[2 * i] = __uint_as_float(p.q[0][i] << 16);
        x[2 * i + 1] = __uint_as_float(p.q[0][i] & 0xffff0000u);
    }
}
__device__ __forceinline__ void widen_piece(const Piece<float> &p, float (&x)[8]) {
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = __uint_as_float(p.q[i >> 2][i & 3]);
}

// Eight rows of dy, scaled, to LDS as two or three planes of bf16; adds their sum times (8 + z), of what was written, to t: of three
// planes that of the top one to t[0], of the others to t[1].  zeros: 8 + z in bf16, in the order that the rows are written in.
// Two planes hold 16 bits: the product of a bf16 dy and a bf16 scale exactly, any other to 2^-16.
template <int PLANES>
__device__ __forceinline__ void stage_scaled(const float (&x)[8], const float (&scale)[8], u32x4 zeros, unsigned char *at,
                                             int plane, float (&t)[PLANES == 3 ? 2 : 1]) {
    uint32_t b[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
        const int r = i < 4 ? 2 * i : 2 * i - 7;
        b[i] = __float_as_uint(x[r] * scale[r]);
    }
    auto tops = [&] { return u32x4{high_halves(b[0], b[1]), high_halves(b[2], b[3]), high_halves(b[4], b[5]), high_halves(b[6], b[7])}; };
    if constexpr (PLANES == 2) {
        const u32x4 top = tops();
        u32x4 rest;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            float y[2];
#pragma unroll
            for (int e = 0; e < 2; ++e)
                y[e] = __uint_as_float(b[2 * i + e]) - __uint_as_float(b[2 * i + e] & 0xffff0000u);
            rest[i] = rounded_pair(y[0], y[1]);
        }
        *reinterpret_cast<u32x4 *>(at) = top;
        *reinterpret_cast<u32x4 *>(at + plane) = rest;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const bf16x2 z = __builtin_bit_cast(bf16x2, (uint32_t)zeros[i]);
            t[0] = __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2, (uint32_t)top[i]), z, t[0], false);
            t[0] = __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2, (uint32_t)rest[i]), z, t[0], false);
        }
    } else {
#pragma unroll
        for (int pl = 0; pl < 3; ++pl) {
            *reinterpret_cast<u32x4 *>(at + pl * plane) = tops();
            if (pl < 2) {
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const float z = __uint_as_float(i & 1 ? zeros[i >> 1] & 0xffff0000u : zeros[i >> 1] << 16);
                    const float top = __uint_as_float(b[i] & 0xffff0000u), rest = __uint_as_float(b[i]) - top;
                    if (pl == 0) {
                        t[0] += top * z;
                        t[1] += rest * z;
                    }
                    b[i] = __float_as_uint(rest);
                }
            }
        }
    }
}

// Scales of a run of rows in LDS: float32 [group][row], and 8 + z in bf16 [group][row in the order of the operands].
__device__ __forceinline__ void put_scale(float *scales, uint16_t *zeros, int at, float s, int z) {
    const int e = at & 7;
    scales[at] = s;
    zeros[(at & ~7) + (e >> 1) + 4 * (e & 1)] = (uint16_t)(__float_as_uint(8.0f + (float)z) >> 16);
}

// ---- tile: 128 columns --------------------------------------------------------------------------------
// Two waves beside each other in columns, 64 each, and two in vectors, 32 each; KW = 2: two such sets, one multiplies the
// first eight rows of every row group and one the others, and they add up at the end.  A stage is ROWS rows of one matrix: dy
// scaled for each of the NG groups of the 128 columns, and the codes.  One barrier per stage.
// Three planes: the top one has sums of its own, whose products have few bits and add up almost exactly.
// Scaling dy and splitting it into planes costs 49 vector instructions per eight elements and group of columns (two planes; one
// rounded plane took 25), about as long as the products of a group of 128; a tile of groups of 64 does it twice.  4096 x 14336, 2048 bf16
// vectors, groups of 128: 531 us (453 TFLOP/s, twice that on the matrix cores; one rounded plane took 317), of 64 760 us.  Groups of
// 32 have no tile: four scaled copies of a stage leave room for one workgroup per CU, 2151 us where split takes 1418.
// Measured against it, groups of 128, two planes, 4096 x 14336, 2048 / 256 / 64 vectors: 64 rows in four waves 531 / 90 / 76 us, 128
// rows in eight 664 / 100 / 53 (both are used), 64 rows in eight 635 / 93 / 63, 128 vectors with 32 rows in four 534 / 151 / 162, with 64
// rows in eight 597 / 89 / 102, 32 rows in four 609 / 114 / 107.
template <typename VT, int PLANES, int NG, int ROWS, int KW>
struct BackTile {
    static constexpr int threads = 256 * KW;
    static constexpr int vectors = 64;
    static constexpr int pieces = ROWS / 8;
    static constexpr int loads = vectors * pieces / threads;
    static constexpr int stride = ROWS * 2 + 16;  // bytes between vectors: an odd number of 16-byte units
    static constexpr int plane = vectors * stride;
    static constexpr int copy = PLANES * plane;   // of a group
    static constexpr int row_groups = ROWS / kDenseRows;
    static constexpr int codes = NG * copy;
    static constexpr int buffer = codes + row_groups * kCodeGroup;
    static constexpr int table = NG * ROWS * 6;   // scales and zero points
    static constexpr int sums = PLANES == 3 ? 2 : 1;
    static constexpr int staged = 2 * buffer + 2 * table;
    static constexpr int joined = KW == 2 ? 4 * 32 * 64 * 4 : 0;
    static constexpr int bytes = staged > joined ? staged : joined;
};

template <typename VT, typename OT, int PLANES, int NG, int ROWS, int KW>
__global__ __launch_bounds__(256 * KW, 2) void k_int4_back_tile(Int4 m0, Int4 m1, int both, int gpt,
                                                               const VT *__restrict__ dy, int ntiles, int n_rows,
                                                               int n_cols, long long ldv, int batch, float scale,
                                                               OT *__restrict__ out, long long ldo, int col_tiles,
                                                               int vec_tiles) {
    using S = BackTile<VT, PLANES, NG, ROWS, KW>;
    extern __shared__ __attribute__((aligned(16))) unsigned char smem[];
    const int tid = threadIdx.x, lane = tid & 63, half = lane >> 5;
    const int w = __builtin_amdgcn_readfirstlane(tid >> 6), wc = w & 1, wv = (w >> 1) & 1, kw = w >> 2;
    // each XCD gets a contiguous run of tiles, eight column tiles for every vector tile
    const int all = col_tiles * vec_tiles, per = (all + 7) / 8;
    const int lin = (blockIdx.x & 7) * per + (blockIdx.x >> 3);
    if ((int)(blockIdx.x >> 3) >= per || lin >= all) return;
    const int band = lin / (8 * vec_tiles), in_band = lin - band * 8 * vec_tiles;
    const int band_cols = min(8, col_tiles - band * 8);
    const int ct = band * 8 + in_band % band_cols, vec0 = in_band / band_cols * S::vectors;
    const int tile = ct >> 1, part = ct & 1;  // the half of a tile of codes
    const int ngroups = (n_rows + kDenseRows - 1) / kDenseRows;
    const int stages1 = (n_rows + ROWS - 1) / ROWS, stages = both ? 2 * stages1 : stages1;

    constexpr int kApart = S::threads / S::pieces;
    const int piece = tid % S::pieces, mine = tid / S::pieces;
    const VT *first = dy + (long long)min(vec0 + mine, batch - 1) * ldv + 8 * piece;
    const bool whole = vec0 + S::vectors <= batch;
    const int whole_stages = whole ? n_rows / ROWS : 0;  // of a matrix
    Piece<VT> p[S::loads];
    auto request_whole = [&](int k, int s) {
#pragma unroll
        for (int j = 0; j < S::loads; ++j)
            p[j] = load_whole_piece<VT>(first + j * (kApart * ldv) + (long long)k * n_rows + s * ROWS);
    };
    auto request_v = [&](int s) {
        const int k = s >= stages1, sk = s - k * stages1;
        if (sk < whole_stages) {
            request_whole(k, sk);
        } else {
#pragma unroll
            for (int j = 0; j < S::loads; ++j)
                p[j] = load_piece<VT>(dy + (long long)min(vec0 + mine + j * kApart, batch - 1) * ldv + (long long)k * n_rows,
                                      sk * ROWS + 8 * piece, n_rows);
        }
    };
    // codes: a thread per (row group, lane); a thread per (group, row) for the scales
    u32x4 c;
    constexpr int kScales = (NG * ROWS + S::threads - 1) / S::threads;
    Scales<1> sv[kScales];
    const int code_group = (tid >> 6) % S::row_groups;  // (further threads: the same again)
    auto request_codes = [&](int s) {
        const int k = s >= stages1;
        const long long rg = min((s - k * stages1) * S::row_groups + code_group, ngroups - 1);
        c = *reinterpret_cast<const u32x4 *>((k ? m1.codes : m0.codes) + ((rg * ntiles + tile) * 2 + part) * 256 + lane * 4);
    };
    auto put_codes = [&](int buf) {
        uint32_t *to = reinterpret_cast<uint32_t *>(smem + buf * S::buffer + S::codes + code_group * kCodeGroup + (lane & 15) * kCodeRow) + (lane >> 4);
#pragma unroll
        for (int d = 0; d < 4; ++d) to[4 * d] = c[d];
    };
    auto pick = [&](int k) {
        return Int4{k ? m1.codes : m0.codes, k ? m1.scales : m0.scales, k ? m1.zeros : m0.zeros, k ? m1.wide : m0.wide};
    };
    auto request_scales = [&](int s) {
        const int k = s >= stages1;
        const Int4 m = pick(k);
#pragma unroll
        for (int j = 0; j < kScales; ++j) {
            const int i = (j * S::threads + tid) % (NG * ROWS), r = (s - k * stages1) * ROWS + i % ROWS, g = i / ROWS;
            const long long rg = min(r / kDenseRows, ngroups - 1);
            const long long idx = ((rg * ntiles + tile) * kDenseRows + r % kDenseRows) * gpt + part * NG + g;
            sv[j] = load_scales<1>(m, idx);
        }
    };
    float *const table = reinterpret_cast<float *>(smem + 2 * S::buffer);
    auto put_scales = [&](int s, int buf) {
        const Int4 m = pick(s >= stages1);
        float *to = table + buf * (S::table / 4);
#pragma unroll
        for (int j = 0; j < kScales; ++j)
            put_scale(to, reinterpret_cast<uint16_t *>(to + NG * ROWS), (j * S::threads + tid) % (NG * ROWS),
                      scale_of(sv[j], m.wide, 0), zero_of(sv[j], m, 0));
    };
    float minus[NG][S::loads][S::sums] = {};
    auto stage = [&](int buf) {
        unsigned char *to = smem + buf * S::buffer + mine * S::stride + 16 * piece;
        const float *from = table + buf * (S::table / 4);
#pragma unroll
        for (int g = 0; g < NG; ++g) {
            float sc[8];
#pragma unroll
            for (int i = 0; i < 8; i += 4) {
                const f32x4 q = *reinterpret_cast<const f32x4 *>(from + g * ROWS + 8 * piece + i);
                sc[i] = q.x; sc[i + 1] = q.y; sc[i + 2] = q.z; sc[i + 3] = q.w;
            }
            const u32x4 z = *reinterpret_cast<const u32x4 *>(reinterpret_cast<const uint16_t *>(from + NG * ROWS) + g * ROWS + 8 * piece);
#pragma unroll
            for (int j = 0; j < S::loads; ++j) {
                float x[8];
                widen_piece(p[j], x);
                stage_scaled<PLANES>(x, sc, z, to + g * S::copy + j * kApart * S::stride, S::plane, minus[g][j]);
            }
        }
    };
    f32x16 acc[S::sums][2] = {};
    request_scales(0);
    put_scales(0, 0);
    if (stages > 1) {
        request_scales(1);
        put_scales(1, 1);
    }
    request_codes(0);
    request_v(0);
    __syncthreads();
    put_codes(0);
    stage(0);
    if (stages > 1) {
        request_codes(1);
        request_v(1);
    }
    if (stages > 2) request_scales(2);
    __syncthreads();
    auto step = [&](int s, auto steady) __attribute__((always_inline)) {
        // the next stage goes to the other buffer, which nobody reads any more
        if (steady || s + 1 < stages) {
            put_codes((s + 1) & 1);
            stage((s + 1) & 1);
        }
        if (steady || s + 2 < stages) {
            put_scales(s + 2, s & 1);
            request_codes(s + 2);
            if constexpr (steady)
                request_whole(s + 2 >= stages1, s + 2 - (s + 2 >= stages1) * stages1);
            else
                request_v(s + 2);
        }
        request_scales(min(s + 3, stages - 1));
        const unsigned char *buf = smem + (s & 1) * S::buffer;
        const unsigned char *operand = buf + (wv * 32 + (lane & 31)) * S::stride + 32 * half;
        // lanes 0..15 and 16..31: the halves of a 32-column step, lanes from 32 on: the second row group
        const unsigned char *code = buf + S::codes + half * kCodeGroup + (lane & 15) * kCodeRow + 16 * (2 * wc) + 8 * ((lane >> 4) & 1);
#pragma unroll
        for (int q = 0; q < S::row_groups / 2; ++q) {
            i32x2 y[2];
#pragma unroll
            for (int r = 0; r < 2; ++r) y[r] = turned(code + q * 2 * kCodeGroup + 16 * r);
#pragma unroll
            for (int mm = 0; mm < 2 / KW; ++mm) {
                bf16x8 x[2];
#pragma unroll
                for (int r = 0; r < 2; ++r) x[r] = decode((uint32_t)(KW == 1 ? y[r][mm] : kw ? y[r].y : y[r].x));
                const unsigned char *at_m = operand + 64 * q + 16 * (KW == 1 ? mm : kw);
#pragma unroll
                for (int pl = 0; pl < PLANES; ++pl) {
                    // (one group of all 128 columns, or one per wave)
                    const bf16x8 o = lds_operand(at_m + pl * S::plane + (NG == 1 ? 0 : wc) * S::copy);
#pragma unroll
                    for (int r = 0; r < 2; ++r) {
                        f32x16 &to = acc[pl ? S::sums - 1 : 0][r];
                        to = mfma32(o, x[r], to);
                    }
                }
            }
        }
        __syncthreads();
    };
    int s = 0;
    while (s < stages) {
        const int end = s < stages1 ? 0 : stages1, far = end + whole_stages - 2;  // steps whose next but one is whole and of the same matrix
        for (; s < far; ++s) step(s, std::true_type());
        for (const int last = end + stages1; s < last; ++s) step(s, std::false_type());
    }
    // (the scales requested last are not used; waited for here, so that no store below has to)
    __builtin_amdgcn_s_waitcnt(0x0f70);
    if constexpr (S::sums == 2) {
#pragma unroll
        for (int r = 0; r < 2; ++r) acc[0][r] += acc[1][r];
    }
    if constexpr (KW == 2) {
        // the second set hands over its sums (the last barrier is behind every read of the buffers)
        float *red = reinterpret_cast<float *>(smem) + (w & 3) * 2048 + lane;
        if (kw == 1) {
#pragma unroll
            for (int i = 0; i < 32; ++i) red[i * 64] = acc[0][i >> 4][i & 15];
        }
        __syncthreads();
        if (kw == 0) {
#pragma unroll
            for (int i = 0; i < 32; ++i) acc[0][i >> 4][i & 15] += red[i * 64];
        }
        __syncthreads();
    }
    // what is taken off, per group and vector
    float *off = reinterpret_cast<float *>(smem);
#pragma unroll
    for (int g = 0; g < NG; ++g)
#pragma unroll
        for (int j = 0; j < S::loads; ++j) {
            float t = run_sum<S::pieces>(minus[g][j][0]);
            if (S::sums == 2) t += run_sum<S::pieces>(minus[g][j][S::sums - 1]);
            if (piece == 0) off[g * S::vectors + mine + j * kApart] = t;
        }
    __syncthreads();
    if (kw == 1) return;
#pragma unroll
    for (int r = 0; r < 2; ++r) {
        const int col = ct * 128 + wc * 64 + r * 32 + turned_column(lane & 31);
        const float *o = off + (NG == 1 ? 0 : wc) * S::vectors;
#pragma unroll
        for (int i = 0; i < 16; ++i) {
            const int v = wv * 32 + acc_row(i, half);
            if (vec0 + v < batch && col < n_cols)
                put(out + (long long)(vec0 + v) * ldo + col, scale * (acc[0][r][i] - o[v]));
        }
    }
}

// ---- split: up to 32 vectors, and more where an estimate prefers it to tiles or there are none (launch_all) ------------
// WAVES waves share the rows of 64 columns; each stages 32 rows of dy, scaled, and their codes in LDS of its own.  Bound by the chain
// of a step (scales, dy, operands: three turns through LDS) and what is around it: 4096 x 14336, one bf16 vector 17.2 us (1.7 TB/s,
// a plain read of the codes 6.2; 13.7 with dy s rounded to one plane, and that 22.5 where branches around its requests had all loads
// waited for).
// Up to 16 vectors (VECS): the other 16 rows of the MFMA repeat them.
template <int PLANES, int NG, int VECS>
struct BackSplit {
    static constexpr int rows = 32, vectors = VECS;
    static constexpr int stride = rows * 2 + 16;
    static constexpr int plane = vectors * stride;
    static constexpr int copy = PLANES * plane;
    static constexpr int codes = NG * copy;
    static constexpr int row_bytes = 40;                      // 64 columns of a row, and 8 bytes more
    static constexpr int table = codes + rows * row_bytes;
    static constexpr int wave_bytes = table + NG * rows * 6;
};

template <typename VT, typename OT, int PLANES, int NG, int VECS, int WAVES>
__global__ __launch_bounds__(WAVES * 64, WAVES / 4) void k_int4_back_split(Int4 m0, Int4 m1, int both, int gpt,
                                                                       const VT *__restrict__ dy, int ntiles, int n_rows,
                                                                       int n_cols, long long ldv, int batch, float scale,
                                                                       OT *__restrict__ out, long long ldo, int col_tiles) {
    using S = BackSplit<PLANES, NG, VECS>;
    constexpr int kPieces = VECS / 16;
    constexpr int kAhead = PLANES == 3 && sizeof(VT) == 4 ? 1 : 2;  // steps whose loads are on their way
    extern __shared__ __attribute__((aligned(16))) unsigned char smem[];
    const int tid = threadIdx.x, lane = tid & 63, half = lane >> 5;
    const int w = __builtin_amdgcn_readfirstlane(tid >> 6);
    // neighbours, which share lines of the codes, on one XCD
    const int per = (col_tiles + 7) / 8, ct = (blockIdx.x & 7) * per + (blockIdx.x >> 3);
    if ((int)(blockIdx.x >> 3) >= per || ct >= col_tiles) return;
    const int vec0 = blockIdx.y * S::vectors;
    const int tile = ct >> 2, quarter = ct & 3;
    const int ngroups = (n_rows + kDenseRows - 1) / kDenseRows;
    const int steps1 = (n_rows + S::rows - 1) / S::rows, steps = both ? 2 * steps1 : steps1;
    const int s0 = (int)((long long)steps * w / WAVES), s1 = (int)((long long)steps * (w + 1) / WAVES);
    unsigned char *mine = smem + w * S::wave_bytes;
    float *table = reinterpret_cast<float *>(mine + S::table);
    uint16_t *table_z = reinterpret_cast<uint16_t *>(table + NG * S::rows);

    const int piece = lane & 3;  // eight rows, of vectors lane / 4 and 16 further on
    Piece<VT> p[kAhead][kPieces];
    u32x2 c[kAhead][2];          // of two row groups
    Scales<1> sv[kAhead];        // of row lane % 32, group lane / 32
    auto pick = [&](int k) {
        return Int4{k ? m1.codes : m0.codes, k ? m1.scales : m0.scales, k ? m1.zeros : m0.zeros, k ? m1.wide : m0.wide};
    };
    const VT *first[kPieces];
#pragma unroll
    for (int j = 0; j < kPieces; ++j) first[j] = dy + (long long)min(vec0 + 16 * j + (lane >> 2), batch - 1) * ldv;
    auto request = [&](int slot, int s, auto whole) {
        const int k = s >= steps1, row = (s - k * steps1) * S::rows;
        const Int4 m = pick(k);
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            const long long rg = min(row / kDenseRows + j, ngroups - 1);
            c[slot][j] = *reinterpret_cast<const u32x2 *>(m.codes + ((rg * ntiles + tile) * 2 + (quarter >> 1)) * 256 + lane * 4 + (quarter & 1) * 2);
        }
        const long long rg = min((row + (lane & 31)) / kDenseRows, ngroups - 1);
        const long long idx = ((rg * ntiles + tile) * kDenseRows + (lane & 15)) * gpt + (NG == 2 ? 2 * quarter + half : quarter * gpt / 4);
        sv[slot] = load_scales<1>(m, idx);
        if (whole || row + S::rows <= n_rows) {
#pragma unroll
            for (int j = 0; j < kPieces; ++j) p[slot][j] = load_whole_piece<VT>(first[j] + (long long)k * n_rows + row + 8 * piece);
        } else {
#pragma unroll
            for (int j = 0; j < kPieces; ++j) p[slot][j] = load_piece<VT>(first[j] + (long long)k * n_rows, row + 8 * piece, n_rows);
        }
    };
    constexpr int kSums = PLANES == 3 ? 2 : 1;  // the top plane, and the others
    f32x16 acc[kSums][2] = {};
    float minus[NG][kPieces][kSums] = {};
    auto step = [&](int d, int s, auto whole) __attribute__((always_inline)) {
        const Int4 m = pick(s >= steps1);
        // (one group: the upper half of the lanes writes the same again)
        put_scale(table, table_z, NG == 2 ? lane : lane & 31, scale_of(sv[d], m.wide, 0), zero_of(sv[d], m, 0));
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            uint32_t *to = reinterpret_cast<uint32_t *>(mine + S::codes + (j * kDenseRows + (lane & 15)) * S::row_bytes) + (lane >> 4);
            to[0] = c[d][j].x;
            to[4] = c[d][j].y;
        }
        float x[kPieces][8];
#pragma unroll
        for (int j = 0; j < kPieces; ++j) widen_piece(p[d][j], x[j]);
        request(d, min(s + kAhead, s1 - 1), whole);
        // the wave's LDS operations execute in order: no barrier inside a wave
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        __builtin_amdgcn_wave_barrier();
#pragma unroll
        for (int g = 0; g < NG; ++g) {
            float sc[8];
#pragma unroll
            for (int i = 0; i < 8; i += 4) {
                const f32x4 q = *reinterpret_cast<const f32x4 *>(table + g * S::rows + 8 * piece + i);
                sc[i] = q.x; sc[i + 1] = q.y; sc[i + 2] = q.z; sc[i + 3] = q.w;
            }
            const u32x4 z = *reinterpret_cast<const u32x4 *>(table_z + g * S::rows + 8 * piece);
#pragma unroll
            for (int j = 0; j < kPieces; ++j)
                stage_scaled<PLANES>(x[j], sc, z, mine + g * S::copy + (16 * j + (lane >> 2)) * S::stride + 16 * piece, S::plane,
                                     minus[g][j]);
        }
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        __builtin_amdgcn_wave_barrier();
        const unsigned char *operand = mine + (lane & (VECS - 1)) * S::stride + 32 * half;
        const unsigned char *code = mine + S::codes + (half * kDenseRows + (lane & 15)) * S::row_bytes + 8 * ((lane >> 4) & 1);
        i32x2 y[2];
#pragma unroll
        for (int r = 0; r < 2; ++r) y[r] = turned(code + 16 * r);
#pragma unroll
        for (int m = 0; m < 2; ++m)
#pragma unroll
            for (int pl = 0; pl < PLANES; ++pl) {
                bf16x8 o[2];
                o[0] = lds_operand(operand + pl * S::plane + 16 * m);
                o[1] = NG == 2 ? lds_operand(operand + S::copy + pl * S::plane + 16 * m) : o[0];
#pragma unroll
                for (int r = 0; r < 2; ++r) {
                    f32x16 &to = acc[pl ? kSums - 1 : 0][r];
                    to = mfma32(o[r], decode((uint32_t)y[r][m]), to);
                }
            }
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        __builtin_amdgcn_wave_barrier();
    };
    // Requests behind the last step ask for it again: a branch around them would have all loads waited for behind it.
    auto run = [&](auto whole) __attribute__((always_inline)) {
#pragma unroll
        for (int d = 0; d < kAhead; ++d) request(d, min(s0 + d, s1 - 1), whole);
        int s = s0;
        for (; s + kAhead <= s1; s += kAhead) {
#pragma unroll
            for (int d = 0; d < kAhead; ++d) step(d, s + d, whole);
        }
#pragma unroll
        for (int d = 0; d < kAhead - 1; ++d)
            if (s + d < s1) step(d, s + d, whole);
    };
    if (s0 < s1) {
        if (n_rows % S::rows == 0)
            run(std::true_type());
        else
            run(std::false_type());
    }
    __syncthreads();  // the staging areas become the partial results [wave][register][lane], and what is taken off
    float *red = reinterpret_cast<float *>(smem), *off = red + WAVES * 32 * 64;
#pragma unroll
    for (int i = 0; i < 32; ++i) {
        if (acc_row(i & 15, 0) >= VECS || vec0 + acc_row(i & 15, 0) >= batch) continue;
        float sum = acc[0][i >> 4][i & 15];
        if (kSums == 2) sum += acc[kSums - 1][i >> 4][i & 15];
        red[(w * 32 + i) * 64 + lane] = sum;
    }
#pragma unroll
    for (int g = 0; g < NG; ++g)
#pragma unroll
        for (int j = 0; j < kPieces; ++j) {
            float t = run_sum<4>(minus[g][j][0]);
            if (kSums == 2) t += run_sum<4>(minus[g][j][kSums - 1]);
            if (piece == 0) off[(w * NG + g) * S::vectors + 16 * j + (lane >> 2)] = t;
        }
    __syncthreads();
    for (int i = w; i < 32; i += WAVES) {
        if (acc_row(i & 15, 0) >= VECS || vec0 + acc_row(i & 15, 0) >= batch) continue;
        const int v = acc_row(i & 15, half), r = i >> 4, col = ct * 64 + r * 32 + turned_column(lane & 31);
        float sum = 0.0f, t = 0.0f;
#pragma unroll
        for (int u = 0; u < WAVES; ++u) {
            sum += red[(u * 32 + i) * 64 + lane];
            t += off[(u * NG + (NG == 2 ? r : 0)) * S::vectors + v];
        }
        if (vec0 + v < batch && col < n_cols) put(out + (long long)(vec0 + v) * ldo + col, scale * (sum - t));
    }
}

struct Args {
    Int4 m[2];
    int both, gpt, ntiles, n_rows, n_cols, batch, device;
    const void *dy;
    long long ldv, ldo;
    float scale;
    void *out;
    hipStream_t stream;
    char *name;  // not null: write the name of the kernel there (of several the first) instead of launching it
    size_t name_len;
};

template <typename VT, typename OT, typename... Number>
hipError_t put_name(const Args &x, const char *format, Number... n) {
    if (!x.name[0])
        std::snprintf(x.name, x.name_len, format, sizeof(VT) == 4 ? "float" : "unsigned short", sizeof(OT) == 4 ? "float" : "unsigned short", n...);
    return hipSuccess;
}

template <typename VT, typename OT, int PLANES, int NG, int ROWS, int KW>
hipError_t launch_tile(const Args &x) {
    using S = BackTile<VT, PLANES, NG, ROWS, KW>;
    if (x.name) return put_name<VT, OT>(x, "k_int4_back_tile<%s, %s, %d, %d, %d, %d>", PLANES, NG, ROWS, KW);
    static std::atomic<size_t> enabled[kMaxDevices];
    auto kern = k_int4_back_tile<VT, OT, PLANES, NG, ROWS, KW>;
    static_assert(S::bytes <= kLdsBytes && S::codes >= NG * S::vectors * 4, "two stages, and then what is taken off");
    if (hipError_t e = ensure_dynamic_lds(reinterpret_cast<const void *>(kern), S::bytes, x.device, enabled)) return e;
    const int col_tiles = (x.n_cols + 127) / 128, vec_tiles = (x.batch + S::vectors - 1) / S::vectors;
    const int per = (int)(((long long)col_tiles * vec_tiles + 7) / 8);
    hipLaunchKernelGGL(kern, dim3((unsigned)(per * 8)), dim3(S::threads), S::bytes, x.stream, x.m[0], x.m[1], x.both, x.gpt,
                       static_cast<const VT *>(x.dy), x.ntiles, x.n_rows, x.n_cols, x.ldv, x.batch, x.scale,
                       static_cast<OT *>(x.out), x.ldo, col_tiles, vec_tiles);
    return hipGetLastError();
}

template <typename VT, typename OT, int PLANES, int NG, int VECS, int WAVES>
hipError_t launch_split_waves(const Args &x) {
    using S = BackSplit<PLANES, NG, VECS>;
    if (x.name) return put_name<VT, OT>(x, "k_int4_back_split<%s, %s, %d, %d, %d, %d>", PLANES, NG, VECS, WAVES);
    static std::atomic<size_t> enabled[kMaxDevices];
    auto kern = k_int4_back_split<VT, OT, PLANES, NG, VECS, WAVES>;
    constexpr size_t staged = (size_t)WAVES * S::wave_bytes, joined = (size_t)WAVES * (32 * 64 + NG * S::vectors) * 4;
    constexpr size_t lds = staged > joined ? staged : joined;
    static_assert(lds <= (size_t)kLdsBytes, "staging, and then the partial results of all waves");
    if (hipError_t e = ensure_dynamic_lds(reinterpret_cast<const void *>(kern), lds, x.device, enabled)) return e;
    const int col_tiles = (x.n_cols + 63) / 64, per = (col_tiles + 7) / 8;
    hipLaunchKernelGGL(kern, dim3((unsigned)(per * 8), (unsigned)((x.batch + S::vectors - 1) / S::vectors)),
                       dim3(WAVES * 64), lds, x.stream, x.m[0], x.m[1], x.both, x.gpt, static_cast<const VT *>(x.dy),
                       x.ntiles, x.n_rows, x.n_cols, x.ldv, x.batch, x.scale, static_cast<OT *>(x.out), x.ldo, col_tiles);
    return hipGetLastError();
}

template <typename VT, typename OT, int PLANES, int NG>
hipError_t launch_split(const Args &x) {
    if (x.batch > 16) return launch_split_waves<VT, OT, PLANES, NG, 32, 8>(x);
    // sixteen waves where every one gets four steps, and the registers allow it.  Measured, one vector, sixteen / eight: 14336 x 4096
    // 38.5 / 47.2 us, 4096 x 14336 17.3 / 18.3, 2560 x 6912 in groups of 32 13.1 / 14.2 (with 40 bytes of scratch), 1024 x 1024 in groups
    // of 32 7.5 / 7.2
    if constexpr (PLANES == 2 && sizeof(VT) == 2)
        if (x.n_rows >= 2048) return launch_split_waves<VT, OT, PLANES, NG, 16, 16>(x);
    return launch_split_waves<VT, OT, PLANES, NG, 16, 8>(x);
}

// Estimates in microseconds for more than 32 vectors.  A round of split, one workgroup per CU, takes 1.12 us (three planes 1.4) per 256
// rows.  A workgroup of a tile takes 1.1 us per 64 rows and 1.46 per 128 (two planes), 1.15 per 64 (three); those of 128 rows, and of
// three planes, have a CU to themselves and go in rounds, the others share it, three at once, for 0.58 us more each.  Measured, split / 128 rows /
// 64 rows, groups of 128, two planes: 4096 x 14336, 64 vectors 43 / 53 / 76, 256 136 / 100 / 90, 2048 1040 / 664 / 531; 14336 x 4096, 256
// vectors 132 / 161 / 245, 2048 911 / 636 / 582; 6912 x 2560, 256 60 / 82 / 115, 512 91 / 80 / 114, 2048 299 / 230 / 199; 2560 x 6912, 64
// 15 / 35 / 47, 256 56 / 36 / 47; both matrices of 6912 x 2560, 1024 vectors 304 / 317 / 299.  Three planes, split / tile: 4096 x 14336,
// 64 54 / 80, 256 171 / 150; 14336 x 4096, 256 161 / 257, 512 304 / 257.
// Groups of 64, two planes, split / tile (32 rows): 4096 x 14336, 128 vectors 78 / 127, 512 264 / 257, 2048 1041 / 760; 14336 x 4096, 1024
// 494 / 465.  In groups of 64 tiles of three planes lose to split (4096 x 14336, 256 and 512 vectors 174 / 182 and 336 / 366; 6912 x 2560,
// 512 117 / 260), in groups of 32 all do (three planes: 230 / 414 and 451 / 826; two: 128 and 2048 vectors 103 / 170 and 1418 / 2151).
float per_cu(int columns, int vectors, const Args &x) {
    return (float)((((long long)x.n_cols + columns - 1) / columns * ((x.batch + vectors - 1) / vectors) + 255) / 256);
}

template <typename VT, typename OT, int PLANES>
hipError_t launch_all(const Args &x) {
    if (x.gpt == 8) return launch_split<VT, OT, PLANES, 2>(x);
    if (x.batch <= 32 || (x.gpt == 4 && PLANES == 3)) return launch_split<VT, OT, PLANES, 1>(x);
    const float rows = (float)x.n_rows * (x.both ? 2.0f : 1.0f), tiles = per_cu(128, 64, x);
    const float split = 4.0f + (PLANES == 3 ? 1.4f : 1.12f) * rows / 256.0f * per_cu(64, 32, x);
    auto shared = [&](int stage_rows, float alone, float more) {
        const float together = 0.2f + more * tiles;
        return 3.0f + rows / (float)stage_rows * (alone > together ? alone : together);
    };
    if constexpr (PLANES == 3) {
        if (split < 3.0f + 1.15f * rows / 64.0f * tiles) return launch_split<VT, OT, PLANES, 1>(x);
        return launch_tile<VT, OT, PLANES, 1, 64, 2>(x);
    } else {
        if (x.gpt == 4) {
            if (split < shared(32, 0.97f, 0.42f)) return launch_split<VT, OT, PLANES, 1>(x);
            return launch_tile<VT, OT, PLANES, 2, 32, 1>(x);
        }
        const float few = 3.0f + 1.46f * rows / 128.0f * tiles, many = shared(64, 1.1f, 0.58f);
        if (split < (few < many ? few : many)) return launch_split<VT, OT, PLANES, 1>(x);
        if (many < few) return launch_tile<VT, OT, PLANES, 1, 64, 1>(x);
        return launch_tile<VT, OT, PLANES, 1, 128, 2>(x);
    }
}

// (A launch holds fewer than 2^32 threads, at most 1024 per 64 columns and 32 vectors, and 65535 sets of vectors: so many at
// a time.)
template <typename VT, typename OT, int PLANES>
hipError_t launch(const Args &x) {
    const long long sets = (1LL << 31) / (1024LL * ((x.n_cols + 63) / 64));
    const int most = 32 * (int)(sets > 16384 ? 16384 : sets);
    if (x.batch <= most) return launch_all<VT, OT, PLANES>(x);
    Args y = x;
    for (int n = 0; n < x.batch; n += most) {
        y.batch = x.batch - n < most ? x.batch - n : most;
        y.dy = static_cast<const VT *>(x.dy) + n * x.ldv;
        y.out = static_cast<OT *>(x.out) + n * x.ldo;
        if (hipError_t e = launch_all<VT, OT, PLANES>(y)) return e;
    }
    return hipSuccess;
}

Args args_of(const rsr_handle_s *a, const rsr_handle_s *b, const void *dy, float scale, void *out, int batch, int64_t ldv,
             int64_t ldo, hipStream_t stream) {
    Args x = {};
    x.m[0] = int4_of(a);
    if (b) x.m[1] = int4_of(b);
    x.both = b != nullptr;
    x.gpt = kInt4Tile / a->group;
    x.ntiles = (int)((a->cols + kInt4Tile - 1) / kInt4Tile);
    x.n_rows = (int)a->rows;
    x.n_cols = (int)a->cols;
    x.batch = batch;
    x.device = a->device;
    x.dy = dy;
    x.ldv = ldv;
    x.ldo = ldo;
    x.scale = scale;
    x.out = out;
    x.stream = stream;
    return x;
}

hipError_t launch_types(const Args &x, int v_dtype, bool short_dy, int out_dtype) {
    if (v_dtype == RSR_BF16)
        return out_dtype != RSR_BF16 ? launch<uint16_t, float, 3>(x) : launch<uint16_t, uint16_t, 2>(x);
    if (out_dtype != RSR_BF16) return launch<float, float, 3>(x);
    return short_dy ? launch<float, uint16_t, 2>(x) : launch<float, uint16_t, 3>(x);
}

}  // namespace

hipError_t launch_int4_transposed(const rsr_handle_s *a, const rsr_handle_s *b, const void *dy, int v_dtype, bool short_dy,
                                  float scale, void *out, int out_dtype, int batch, int64_t ldv, int64_t ldo,
                                  hipStream_t stream) {
    return launch_types(args_of(a, b, dy, scale, out, batch, ldv, ldo, stream), v_dtype, short_dy, out_dtype);
}

void int4_transposed_kernel_name(const rsr_handle_s *a, const rsr_handle_s *b, int v_dtype, bool short_dy, int out_dtype,
                                 int batch, char *buf, size_t len) {
    Args x = args_of(a, b, nullptr, 1.0f, nullptr, batch, a->rows * (b ? 2 : 1), a->cols, nullptr);
    x.name = buf;
    x.name_len = len;
    buf[0] = 0;
    (void)launch_types(x, v_dtype, short_dy, out_dtype);
}

hipError_t launch_gated_slopes(const float *pre, const void *dh, int d_dtype, int64_t ldd, int act, int64_t rows,
                               int batch, float *dpre, hipStream_t stream) {
    // (a launch holds fewer than 2^32 threads, and 65535 vectors: so many at a time)
    const int64_t blocks = (rows + 1023) / 1024, fit = ((int64_t)1 << 31) / (256 * blocks);
    const int most = (int)(fit < 65535 ? fit : 65535);
    for (int n = 0; n < batch; n += most) {
        const dim3 grid((unsigned)blocks, (unsigned)(batch - n < most ? batch - n : most));
        const float *from = pre + 2LL * n * rows;
        float *to = dpre + 2LL * n * rows;
        if (d_dtype == RSR_BF16)
            hipLaunchKernelGGL(k_gated_slopes<uint16_t>, grid, dim3(256), 0, stream, from,
                               static_cast<const uint16_t *>(dh) + n * ldd, (long long)ldd, act, (int)rows, to);
        else
            hipLaunchKernelGGL(k_gated_slopes<float>, grid, dim3(256), 0, stream, from,
                               static_cast<const float *>(dh) + n * ldd, (long long)ldd, act, (int)rows, to);
        if (hipError_t e = hipGetLastError()) return e;
    }
    return hipSuccess;
}

}  // namespace rsr
