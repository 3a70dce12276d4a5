// Input gradients of products with 4-bit weights (gfx950): dx = scale M^T dy, the sum of two of them, and the gradient of the
// gated block's activation.
#include "rsr_int4.h"

namespace rsr {

namespace {

// (da, db) from (a, b) and dh, one thread per element; dpre may be pre.
template <typename VT>
__global__ __launch_bounds__(256) void k_gated_slopes(const float *pre, const VT *__restrict__ dh, long long ldd, int act,
                                                      int rows, long long count, float *dpre) {
    const long long i = (long long)blockIdx.x * 256 + threadIdx.x;
    if (i >= count) return;
    const long long n = i / rows, r = i - n * rows, at = 2 * n * rows + r;
    const float a = pre[at], b = pre[at + rows], d = widen(dh[n * ldd + r]);
    float slope;
    const float f = activate(act, a, &slope);
    dpre[at] = d * b * slope;
    dpre[at + rows] = d * f;
}

// ---- the transposed product ----------------------------------------------------------------------------
// out[n][c] = sum over r of (dy[n][r] s[r][g]) (u[r][c] - (8 + z[r][g])), g the group of c.  The sum runs over the rows, so it is dy
// that is scaled, once per group of columns, on its way into LDS (one bf16 plane, rounded, or three that hold all of
// it); the codes are whole numbers as ever, and sum dy s (8 + z), the same for all columns of a group, is taken off at the end.
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

// Eight rows of dy, scaled, to LDS; returns t + their sum times (8 + z), of what was written.  zeros: 8 + z in bf16, in the order
// that the rows are written in.
template <int PLANES>
__device__ __forceinline__ float stage_scaled(const float (&x)[8], const float (&scale)[8], u32x4 zeros, unsigned char *at,
                                              int plane, float t) {
    float y[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) y[i] = x[i] * scale[i];
    if constexpr (PLANES == 1) {
        const u32x4 w = {rounded_pair(y[0], y[2]), rounded_pair(y[4], y[6]), rounded_pair(y[1], y[3]), rounded_pair(y[5], y[7])};
        *reinterpret_cast<u32x4 *>(at) = w;
#pragma unroll
        for (int i = 0; i < 4; ++i)
            t = __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2, (uint32_t)w[i]), __builtin_bit_cast(bf16x2, (uint32_t)zeros[i]), t, false);
    } else {
        uint32_t b[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const int from = i < 4 ? 2 * i : 2 * i - 7;
            b[i] = __float_as_uint(y[from]);
            t += y[from] * __uint_as_float(i & 1 ? zeros[i >> 1] & 0xffff0000u : zeros[i >> 1] << 16);
        }
#pragma unroll
        for (int pl = 0; pl < 3; ++pl) {
            *reinterpret_cast<u32x4 *>(at + pl * plane) =
                u32x4{high_halves(b[0], b[1]), high_halves(b[2], b[3]), high_halves(b[4], b[5]), high_halves(b[6], b[7])};
            if (pl < 2) {
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    b[i] = __float_as_uint(__uint_as_float(b[i]) - __uint_as_float(b[i] & 0xffff0000u));
            }
        }
    }
    return t;
}

// Scales of a run of rows in LDS: float32 [group][row], and 8 + z in bf16 [group][row in the order of the operands].
__device__ __forceinline__ void put_scale(float *scales, uint16_t *zeros, int at, float s, int z) {
    const int e = at & 7;
    scales[at] = s;
    zeros[(at & ~7) + (e >> 1) + 4 * (e & 1)] = (uint16_t)(__float_as_uint(8.0f + (float)z) >> 16);
}

// ---- tile: 128 columns --------------------------------------------------------------------------------
// Two waves beside each other in columns, 64 each, and two in vectors, 32 VB each.  A stage is ROWS rows of one matrix: dy scaled
// for each of the NG groups of the 128 columns, and the codes.  One barrier per stage.
template <typename VT, int PLANES, int NG, int VB, int ROWS>
struct BackTile {
    static constexpr int vectors = 64 * VB;
    static constexpr int pieces = ROWS / 8;
    static constexpr int loads = vectors * pieces / 256;
    static constexpr int stride = ROWS * 2 + 16;  // bytes between vectors: an odd number of 16-byte units
    static constexpr int plane = vectors * stride;
    static constexpr int copy = PLANES * plane;   // of a group
    static constexpr int row_groups = ROWS / kDenseRows;
    static constexpr int codes = NG * copy;
    static constexpr int buffer = codes + row_groups * kCodeGroup;
    static constexpr int table = NG * ROWS * 6;   // scales and zero points
    static constexpr int bytes = 2 * buffer + 2 * table;
};

template <typename VT, typename OT, int PLANES, int NG, int VB, int ROWS>
__global__ __launch_bounds__(256, 2) void k_int4_back_tile(Int4 m0, Int4 m1, int both, int gpt, const VT *__restrict__ dy,
                                                          int ntiles, int n_rows, int n_cols, long long ldv, int batch,
                                                          float scale, OT *__restrict__ out, long long ldo, int col_tiles,
                                                          int vec_tiles) {
    using S = BackTile<VT, PLANES, NG, VB, ROWS>;
    extern __shared__ __attribute__((aligned(16))) unsigned char smem[];
    const int tid = threadIdx.x, lane = tid & 63, half = lane >> 5;
    const int w = __builtin_amdgcn_readfirstlane(tid >> 6), wc = w & 1, wv = w >> 1;
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

    constexpr int kApart = 256 / S::pieces;
    const int piece = tid % S::pieces, mine = tid / S::pieces;
    const VT *first = dy + (long long)min(vec0 + mine, batch - 1) * ldv + 8 * piece;
    const bool whole = vec0 + S::vectors <= batch;
    Piece<VT> p[S::loads];
    auto request_v = [&](int s) {
        const int k = s >= stages1, row = (s - k * stages1) * ROWS;
        if (whole && row + ROWS <= n_rows) {
#pragma unroll
            for (int j = 0; j < S::loads; ++j)
                p[j] = load_whole_piece<VT>(first + j * (kApart * ldv) + (long long)k * n_rows + row);
        } else {
#pragma unroll
            for (int j = 0; j < S::loads; ++j)
                p[j] = load_piece<VT>(dy + (long long)min(vec0 + mine + j * kApart, batch - 1) * ldv + (long long)k * n_rows,
                                      row + 8 * piece, n_rows);
        }
    };
    // codes: a thread per (row group, lane)
    u32x4 c;
    const bool has_codes = tid < S::row_groups * 64;
    auto request_codes = [&](int s) {
        if (!has_codes) return;
        const int k = s >= stages1;
        const long long rg = min((s - k * stages1) * S::row_groups + (tid >> 6), ngroups - 1);
        c = *reinterpret_cast<const u32x4 *>((k ? m1.codes : m0.codes) + ((rg * ntiles + tile) * 2 + part) * 256 + lane * 4);
    };
    auto put_codes = [&](int buf) {
        if (!has_codes) return;
        uint32_t *to = reinterpret_cast<uint32_t *>(smem + buf * S::buffer + S::codes + (tid >> 6) * kCodeGroup + (lane & 15) * kCodeRow) + (lane >> 4);
#pragma unroll
        for (int d = 0; d < 4; ++d) to[4 * d] = c[d];
    };
    // scales: a thread per (group, row)
    constexpr int kScales = (NG * ROWS + 255) / 256;
    float sv[kScales];
    int zv[kScales];
    auto request_scales = [&](int s) {
        const int k = s >= stages1;
        const Int4 &m = k ? m1 : m0;
#pragma unroll
        for (int j = 0; j < kScales; ++j) {
            const int i = j * 256 + tid, r = (s - k * stages1) * ROWS + i % ROWS, g = i / ROWS;
            if (i >= NG * ROWS) break;
            const long long rg = min(r / kDenseRows, ngroups - 1);
            const long long idx = ((rg * ntiles + tile) * kDenseRows + r % kDenseRows) * gpt + part * NG + g;
            sv[j] = scale_at(m, idx);
            zv[j] = m.zeros ? m.zeros[idx] : 0;
        }
    };
    float *const table = reinterpret_cast<float *>(smem + 2 * S::buffer);
    auto put_scales = [&](int buf) {
        float *to = table + buf * (S::table / 4);
#pragma unroll
        for (int j = 0; j < kScales; ++j) {
            const int i = j * 256 + tid;
            if (i < NG * ROWS) put_scale(to, reinterpret_cast<uint16_t *>(to + NG * ROWS), i, sv[j], zv[j]);
        }
    };
    float minus[NG][S::loads] = {};
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
                minus[g][j] = stage_scaled<PLANES>(x, sc, z, to + g * S::copy + j * kApart * S::stride, S::plane, minus[g][j]);
            }
        }
    };
    f32x16 acc[2][VB] = {};
    request_scales(0);
    put_scales(0);
    if (stages > 1) {
        request_scales(1);
        put_scales(1);
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
    for (int s = 0; s < stages; ++s) {
        const unsigned char *buf = smem + (s & 1) * S::buffer;
        const unsigned char *operand = buf + (wv * 32 * VB + (lane & 31)) * S::stride + 32 * half;
        // lanes 0..15 and 16..31: the halves of a 32-column step, lanes from 32 on: the second row group
        const unsigned char *code = buf + S::codes + half * kCodeGroup + (lane & 15) * kCodeRow + 16 * (2 * wc) + 8 * ((lane >> 4) & 1);
#pragma unroll
        for (int q = 0; q < S::row_groups / 2; ++q) {
            i32x2 y[2];
#pragma unroll
            for (int r = 0; r < 2; ++r) y[r] = turned(code + q * 2 * kCodeGroup + 16 * r);
#pragma unroll
            for (int m = 0; m < 2; ++m) {
                bf16x8 x[2];
#pragma unroll
                for (int r = 0; r < 2; ++r) x[r] = decode((uint32_t)y[r][m]);
#pragma unroll
                for (int n = 0; n < VB; ++n)
#pragma unroll
                    for (int pl = 0; pl < PLANES; ++pl) {
                        const unsigned char *at = operand + pl * S::plane + n * 32 * S::stride + 64 * q + 16 * m;
                        bf16x8 o[2];
                        // (groups of this wave's two 32-column steps: one of all 128 columns, one per 64, one per 32)
                        o[0] = lds_operand(at + (NG == 1 ? 0 : NG == 2 ? wc : 2 * wc) * S::copy);
                        o[1] = NG == 4 ? lds_operand(at + (2 * wc + 1) * S::copy) : o[0];
#pragma unroll
                        for (int r = 0; r < 2; ++r) acc[r][n] = mfma32(o[r], x[r], acc[r][n]);
                    }
            }
        }
        // the next stage goes to the other buffer, which nobody reads any more
        if (s + 1 < stages) {
            put_codes((s + 1) & 1);
            stage((s + 1) & 1);
        }
        if (s + 2 < stages) {
            put_scales(s & 1);
            request_codes(s + 2);
            request_v(s + 2);
        }
        if (s + 3 < stages) request_scales(s + 3);
        __syncthreads();
    }
    // what is taken off, per group and vector (the last barrier is behind every read of the buffers)
    float *off = reinterpret_cast<float *>(smem);
#pragma unroll
    for (int g = 0; g < NG; ++g)
#pragma unroll
        for (int j = 0; j < S::loads; ++j) {
            const float t = run_sum<S::pieces>(minus[g][j]);
            if (piece == 0) off[g * S::vectors + mine + j * kApart] = t;
        }
    __syncthreads();
#pragma unroll
    for (int r = 0; r < 2; ++r) {
        const int col = ct * 128 + wc * 64 + r * 32 + turned_column(lane & 31);
        const float *o = off + (NG == 1 ? 0 : NG == 2 ? wc : 2 * wc + r) * S::vectors;
#pragma unroll
        for (int n = 0; n < VB; ++n)
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                const int v = (wv * VB + n) * 32 + acc_row(i, half);
                if (vec0 + v < batch && col < n_cols) put(out + (long long)(vec0 + v) * ldo + col, scale * (acc[r][n][i] - o[v]));
            }
    }
}

// ---- split: up to 32 vectors -----------------------------------------------------------------------------
// Eight waves share the rows of 64 columns; each stages 32 rows of dy, scaled, and their codes in LDS of its own.
constexpr int kBackWaves = 8;

template <int PLANES, int NG>
struct BackSplit {
    static constexpr int rows = 32, vectors = 32;
    static constexpr int stride = rows * 2 + 16;
    static constexpr int plane = vectors * stride;
    static constexpr int copy = PLANES * plane;
    static constexpr int codes = NG * copy;
    static constexpr int row_bytes = 40;                      // 64 columns of a row, and 8 bytes more
    static constexpr int table = codes + rows * row_bytes;
    static constexpr int wave_bytes = table + NG * rows * 6;
};

template <typename VT, typename OT, int PLANES, int NG>
__global__ __launch_bounds__(kBackWaves * 64, 2) void k_int4_back_split(Int4 m0, Int4 m1, int both, int gpt,
                                                                       const VT *__restrict__ dy, int ntiles, int n_rows,
                                                                       int n_cols, long long ldv, int batch, float scale,
                                                                       OT *__restrict__ out, long long ldo, int col_tiles) {
    using S = BackSplit<PLANES, NG>;
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
    const int s0 = (int)((long long)steps * w / kBackWaves), s1 = (int)((long long)steps * (w + 1) / kBackWaves);
    unsigned char *mine = smem + w * S::wave_bytes;
    float *table = reinterpret_cast<float *>(mine + S::table);
    uint16_t *table_z = reinterpret_cast<uint16_t *>(table + NG * S::rows);

    const int piece = lane & 3;  // eight rows, of vectors lane / 4 and 16 further on
    Piece<VT> p[2];
    u32x2 c[2];                  // of two row groups
    float sv;                    // scale of row lane % 32, group lane / 32
    int zv;
    auto request = [&](int s) {
        const int k = s >= steps1, row = (s - k * steps1) * S::rows;
        const Int4 &m = k ? m1 : m0;
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            const long long rg = min(row / kDenseRows + j, ngroups - 1);
            c[j] = *reinterpret_cast<const u32x2 *>(m.codes + ((rg * ntiles + tile) * 2 + (quarter >> 1)) * 256 + lane * 4 + (quarter & 1) * 2);
        }
        const long long rg = min((row + (lane & 31)) / kDenseRows, ngroups - 1);
        const long long idx = ((rg * ntiles + tile) * kDenseRows + (lane & 15)) * gpt + (NG == 2 ? 2 * quarter + half : quarter * gpt / 4);
        sv = scale_at(m, idx);
        zv = m.zeros ? m.zeros[idx] : 0;
#pragma unroll
        for (int j = 0; j < 2; ++j)
            p[j] = load_piece<VT>(dy + (long long)min(vec0 + 16 * j + (lane >> 2), batch - 1) * ldv + (long long)k * n_rows,
                                  row + 8 * piece, n_rows);
    };
    f32x16 acc[2] = {};
    float minus[NG][2] = {};
    if (s0 < s1) request(s0);
    for (int s = s0; s < s1; ++s) {
        if (NG == 2 || half == 0) put_scale(table, table_z, lane, sv, zv);
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            uint32_t *to = reinterpret_cast<uint32_t *>(mine + S::codes + (j * kDenseRows + (lane & 15)) * S::row_bytes) + (lane >> 4);
            to[0] = c[j].x;
            to[4] = c[j].y;
        }
        float x[2][8];
        widen_piece(p[0], x[0]);
        widen_piece(p[1], x[1]);
        if (s + 1 < s1) request(s + 1);
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
            for (int j = 0; j < 2; ++j)
                minus[g][j] = stage_scaled<PLANES>(x[j], sc, z, mine + g * S::copy + (16 * j + (lane >> 2)) * S::stride + 16 * piece,
                                                   S::plane, minus[g][j]);
        }
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        __builtin_amdgcn_wave_barrier();
        const unsigned char *operand = mine + (lane & 31) * S::stride + 32 * half;
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
                for (int r = 0; r < 2; ++r) acc[r] = mfma32(o[r], decode((uint32_t)y[r][m]), acc[r]);
            }
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        __builtin_amdgcn_wave_barrier();
    }
    __syncthreads();  // the staging areas become the partial results [wave][register][lane], and what is taken off
    float *red = reinterpret_cast<float *>(smem), *off = red + kBackWaves * 32 * 64;
#pragma unroll
    for (int i = 0; i < 32; ++i) red[(w * 32 + i) * 64 + lane] = acc[i >> 4][i & 15];
#pragma unroll
    for (int g = 0; g < NG; ++g)
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            const float t = run_sum<4>(minus[g][j]);
            if (piece == 0) off[(w * NG + g) * S::vectors + 16 * j + (lane >> 2)] = t;
        }
    __syncthreads();
    for (int i = w; i < 32; i += kBackWaves) {
        const int v = acc_row(i & 15, half), r = i >> 4, col = ct * 64 + r * 32 + turned_column(lane & 31);
        float sum = 0.0f, t = 0.0f;
#pragma unroll
        for (int u = 0; u < kBackWaves; ++u) {
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
};

template <typename VT, typename OT, int PLANES, int NG, int VB, int ROWS>
hipError_t launch_tile(const Args &x) {
    using S = BackTile<VT, PLANES, NG, VB, ROWS>;
    static std::atomic<size_t> enabled[kMaxDevices];
    auto kern = k_int4_back_tile<VT, OT, PLANES, NG, VB, ROWS>;
    static_assert(S::bytes <= kLdsBytes && S::codes >= NG * S::vectors * 4, "two stages, and then what is taken off");
    if (hipError_t e = ensure_dynamic_lds(reinterpret_cast<const void *>(kern), S::bytes, x.device, enabled)) return e;
    const int col_tiles = (x.n_cols + 127) / 128, vec_tiles = (x.batch + S::vectors - 1) / S::vectors;
    const int per = (int)(((long long)col_tiles * vec_tiles + 7) / 8);
    hipLaunchKernelGGL(kern, dim3((unsigned)(per * 8)), dim3(256), S::bytes, x.stream, x.m[0], x.m[1], x.both, x.gpt,
                       static_cast<const VT *>(x.dy), x.ntiles, x.n_rows, x.n_cols, x.ldv, x.batch, x.scale,
                       static_cast<OT *>(x.out), x.ldo, col_tiles, vec_tiles);
    return hipGetLastError();
}

template <typename VT, typename OT, int PLANES, int NG>
hipError_t launch_split(const Args &x) {
    using S = BackSplit<PLANES, NG>;
    static std::atomic<size_t> enabled[kMaxDevices];
    auto kern = k_int4_back_split<VT, OT, PLANES, NG>;
    constexpr size_t staged = (size_t)kBackWaves * S::wave_bytes, joined = (size_t)kBackWaves * (32 * 64 + NG * S::vectors) * 4;
    constexpr size_t lds = staged > joined ? staged : joined;
    static_assert(lds <= (size_t)kLdsBytes, "staging, and then the partial results of all waves");
    if (hipError_t e = ensure_dynamic_lds(reinterpret_cast<const void *>(kern), lds, x.device, enabled)) return e;
    const int col_tiles = (x.n_cols + 63) / 64, per = (col_tiles + 7) / 8;
    hipLaunchKernelGGL(kern, dim3((unsigned)(per * 8), (unsigned)((x.batch + S::vectors - 1) / S::vectors)),
                       dim3(kBackWaves * 64), lds, x.stream, x.m[0], x.m[1], x.both, x.gpt, static_cast<const VT *>(x.dy),
                       x.ntiles, x.n_rows, x.n_cols, x.ldv, x.batch, x.scale, static_cast<OT *>(x.out), x.ldo, col_tiles);
    return hipGetLastError();
}

template <typename VT, typename OT, int PLANES>
hipError_t launch(const Args &x) {
    const long long tiles = (long long)((x.n_cols + 127) / 128) * ((x.batch + 127) / 128);
    if (x.batch <= 32 || tiles < 64) return x.gpt == 8 ? launch_split<VT, OT, PLANES, 2>(x) : launch_split<VT, OT, PLANES, 1>(x);
    if constexpr (PLANES == 3)
        return x.gpt == 8   ? launch_tile<VT, OT, 3, 4, 1, 32>(x)
               : x.gpt == 4 ? launch_tile<VT, OT, 3, 2, 2, 32>(x)
                            : launch_tile<VT, OT, 3, 1, 2, 32>(x);
    else
        return x.gpt == 8   ? launch_tile<VT, OT, 1, 4, 2, 32>(x)
               : x.gpt == 4 ? launch_tile<VT, OT, 1, 2, 2, 32>(x)
                            : launch_tile<VT, OT, 1, 1, 2, 64>(x);
}

}  // namespace

hipError_t launch_int4_transposed(const rsr_handle_s *a, const rsr_handle_s *b, const void *dy, int v_dtype, bool rounded,
                                  float scale, void *out, int out_dtype, int batch, int64_t ldv, int64_t ldo,
                                  hipStream_t stream) {
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
    if (v_dtype == RSR_BF16)
        return out_dtype != RSR_BF16 ? launch<uint16_t, float, 3>(x) : launch<uint16_t, uint16_t, 1>(x);
    if (out_dtype != RSR_BF16) return launch<float, float, 3>(x);
    return rounded ? launch<float, uint16_t, 1>(x) : launch<float, uint16_t, 3>(x);
}

hipError_t launch_gated_slopes(const float *pre, const void *dh, int d_dtype, int64_t ldd, int act, int64_t rows,
                               int batch, float *dpre, hipStream_t stream) {
    // (a launch holds fewer than 2^32 threads: so many vectors at a time)
    const int64_t most = ((int64_t)1 << 31) / rows;
    for (int64_t n = 0; n < batch; n += most) {
        const int64_t count = (batch - n < most ? batch - n : most) * rows;
        const dim3 grid((unsigned)((count + 255) / 256));
        if (d_dtype == RSR_BF16)
            hipLaunchKernelGGL(k_gated_slopes<uint16_t>, grid, dim3(256), 0, stream, pre + 2 * n * rows,
                               static_cast<const uint16_t *>(dh) + n * ldd, (long long)ldd, act, (int)rows, (long long)count,
                               dpre + 2 * n * rows);
        else
            hipLaunchKernelGGL(k_gated_slopes<float>, grid, dim3(256), 0, stream, pre + 2 * n * rows,
                               static_cast<const float *>(dh) + n * ldd, (long long)ldd, act, (int)rows, (long long)count,
                               dpre + 2 * n * rows);
        if (hipError_t e = hipGetLastError()) return e;
    }
    return hipSuccess;
}

}  // namespace rsr
