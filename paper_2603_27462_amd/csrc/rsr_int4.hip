// Products with 4-bit weights and group scales (gfx950): packing, and y = scale M x for one or many vectors; with two
// matrices of one shape, h = act(Mg x) * (Mu x).
#include "rsr_int4.h"

#include <cstdio>
#include <type_traits>

namespace rsr {

namespace {

// ---- packing --------------------------------------------------------------------------------------
typedef uint32_t u32x2_bytes __attribute__((ext_vector_type(2), aligned(1)));

// One thread per (row group, tile, lane): its eight dwords.
__global__ __launch_bounds__(256) void k_int4_pack(const int8_t *__restrict__ Q, int64_t rows, int64_t cols,
                                                   int64_t ntiles, int64_t threads, uint32_t *__restrict__ codes,
                                                   int *__restrict__ flags) {
    const int64_t gid = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (gid >= threads) return;
    const int lane = (int)(gid & 63);
    const int64_t gt = gid >> 6, G = gt / ntiles, t = gt - G * ntiles;
    const int64_t i = G * kDenseRows + (lane & 15);
    uint32_t bad = 0, word[kInt4Steps];
#pragma unroll
    for (int d = 0; d < kInt4Steps; ++d) {
        const int64_t j0 = t * kInt4Tile + 32 * d + 8 * (lane >> 4);
        uint32_t x[2] = {0, 0};
        if (i < rows) {
            const int8_t *from = Q + i * cols + j0;
            if (j0 + 8 <= cols) {
                const u32x2_bytes y = *reinterpret_cast<const u32x2_bytes *>(from);
                x[0] = y.x;
                x[1] = y.y;
            } else {
                for (int e = 0; e < 8 && j0 + e < cols; ++e) x[e >> 2] |= (uint32_t)(uint8_t)from[e] << (8 * (e & 3));
            }
        }
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            x[h] = ((x[h] & 0x7f7f7f7fu) + 0x08080808u) ^ (x[h] & 0x80808080u);  // 8 more, byte by byte
            bad |= x[h] & 0xf0f0f0f0u;
        }
        word[d] = (x[0] & 0x0f0f0f0fu) | (x[1] & 0x0f0f0f0fu) << 4;
    }
    u32x4 *to = reinterpret_cast<u32x4 *>(codes + gt * kInt4TileDwords) + lane;
    to[0] = u32x4{word[0], word[1], word[2], word[3]};
    to[64] = u32x4{word[4], word[5], word[6], word[7]};
    if (bad) atomicOr(flags, 1);
}

// flags[0] |= 1 for a scale that is not finite or a zero point out of range; flags[1] |= 1 for a scale that is no bf16.
__global__ __launch_bounds__(256) void k_int4_check_scales(const float *__restrict__ scales,
                                                           const int8_t *__restrict__ zeros, int64_t count,
                                                           int *__restrict__ flags) {
    uint32_t bad = 0, wide = 0;
    for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < count; i += (int64_t)gridDim.x * 256) {
        const uint32_t bits = __float_as_uint(scales[i]);
        bad |= (bits & 0x7f800000u) == 0x7f800000u;
        wide |= (bits & 0xffffu) != 0;
        if (zeros) bad |= zeros[i] < -8 || zeros[i] > 7;
    }
    if (bad) atomicOr(flags, 1);
    if (wide) atomicOr(flags + 1, 1);
}

// Scales and zero points in the handle's order, one thread per value; `group`: the caller's, `per`: columns of one of the handle's.
__global__ __launch_bounds__(256) void k_int4_pack_scales(const float *__restrict__ scales,
                                                          const int8_t *__restrict__ zeros, int64_t rows, int64_t cols,
                                                          int64_t group, int64_t ntiles, int per, int64_t count,
                                                          int wide, void *__restrict__ to, int8_t *__restrict__ zto) {
    const int64_t gid = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (gid >= count) return;
    const int gpt = kInt4Tile / per;
    const int64_t k = gid % gpt, r = gid / gpt % kDenseRows, gt = gid / (gpt * kDenseRows), G = gt / ntiles, t = gt - G * ntiles;
    const int64_t row = G * kDenseRows + r, col = t * kInt4Tile + k * per;
    const bool live = row < rows && col < cols;
    const int64_t from = row * ((cols + group - 1) / group) + col / group;
    const float s = live ? scales[from] : 0.0f;
    if (wide)
        static_cast<float *>(to)[gid] = s;
    else
        static_cast<uint16_t *>(to)[gid] = (uint16_t)(__float_as_uint(s) >> 16);
    if (zto) zto[gid] = live ? zeros[from] : 0;
}

// ---- few: up to four vectors ------------------------------------------------------------------------
// Bound by memory and the start-up of a launch: 4096 x 14336, one bf16 vector 8.4 us with the codes from HBM (3.6 TB/s; a plain
// read of them in one launch 6.2), gate and up of 6912 x 2560 6.7 us (4.6); 367 vector instructions and 28 MFMAs per wave.
// Requests beyond a wave's tiles instead of branches around them, as in the other kernels, lose here, where a wave has one
// to four tiles: 640 x 2560 3.5 -> 4.9 us.
// A wave takes 16 rows (of both matrices, if there are two) and a share of the columns; `wk` waves of a workgroup share
// the columns of a row group and add their partial results at the end, the only place where waves wait for each other.
// Every wave stages its own columns of v, and the sums of v over the groups, in LDS of its own.  The vectors are the rows of
// the MFMA: vector q sits in rows 4q.. (float32: its three planes in rows 4q, 4q+1, 4q+2), so that lane 16 q + r of
// the result holds everything about (vector q, row r), and one MFMA serves all planes.
// (Two matrices take twice the registers, so at most eight waves.)
constexpr int few_most_waves(int nm) { return nm == 2 ? 8 : 16; }

template <typename VT, int NV, int GPT>
struct Few {
    static constexpr int planes = sizeof(VT) == 4 ? 3 : 1;
    static constexpr int tiles = NV == 1 ? (planes == 3 && GPT == 8 ? 2 : 4) : planes == 3 ? 1 : 2;  // staged at a time
    static constexpr int cols = tiles * kInt4Tile;
    static constexpr int pieces = cols / 8;
    static constexpr int loads = NV * pieces / 64;
    static constexpr int stride = cols * 2 + 16;  // bytes between slots: an odd number of 16-byte units
    static constexpr int sums = NV * tiles * GPT;
    static constexpr int wave_bytes = NV * planes * stride + (sums * 4 + 15) / 16 * 16;
};

template <typename VT, int NV, int GPT, int NM>
__global__ __launch_bounds__(few_most_waves(NM) * 64) void k_int4_few(Int4 m0, Int4 m1, const VT *__restrict__ v, int ntiles, int ngroups,
                                                  int n_in, int n_out, long long ldv, int nv, int wk_log2, float scale,
                                                  void *__restrict__ out, int out_bf16, long long ldo, int act,
                                                  float *__restrict__ pre) {
    using S = Few<VT, NV, GPT>;
    constexpr int kSteps = kInt4Steps / GPT, kRun = kInt4Tile / GPT / 8;
    extern __shared__ __attribute__((aligned(16))) unsigned char smem[];
    const int tid = threadIdx.x, lane = tid & 63, waves = blockDim.x >> 6;
    const int w = __builtin_amdgcn_readfirstlane(tid >> 6), wr = w >> wk_log2, wk = w - (wr << wk_log2);
    const int g = min((int)(blockIdx.x * (waves >> wk_log2)) + wr, ngroups - 1);
    const int t0 = (int)((long long)ntiles * wk >> wk_log2), t1 = (int)((long long)ntiles * (wk + 1) >> wk_log2);
    const int m = lane & 15;
    const Int4 mat[2] = {m0, m1};
    const uint32_t *code[NM];
    long long scale_row[NM];
#pragma unroll
    for (int k = 0; k < NM; ++k) {
        code[k] = mat[k].codes + (long long)g * ntiles * kInt4TileDwords + lane * 4;
        scale_row[k] = ((long long)g * ntiles * kDenseRows + m) * GPT;
    }
    unsigned char *mine = smem + w * S::wave_bytes;
    float *sums = reinterpret_cast<float *>(mine + NV * S::planes * S::stride);

    Piece<VT> p[S::loads];
    auto request_v = [&](int t) {
#pragma unroll
        for (int j = 0; j < S::loads; ++j) {
            const int i = j * 64 + lane, n = NV == 1 ? 0 : min(i / S::pieces, nv - 1);
            p[j] = load_piece<VT>(v + n * ldv, t * kInt4Tile + 8 * (i % S::pieces), n_in);
        }
    };
    u32x4 c[NM][S::tiles][2];
    Scales<GPT> sc[NM][S::tiles];
    auto request_codes = [&](int t) {
#pragma unroll
        for (int i = 0; i < S::tiles; ++i)
            if (t + i < t1) {
#pragma unroll
                for (int k = 0; k < NM; ++k) {
                    const u32x4 *at = reinterpret_cast<const u32x4 *>(code[k] + (long long)(t + i) * kInt4TileDwords);
                    c[k][i][0] = __builtin_nontemporal_load(at);
                    c[k][i][1] = __builtin_nontemporal_load(at + 64);
                    sc[k][i] = load_scales<GPT>(mat[k], scale_row[k] + (long long)(t + i) * kDenseRows * GPT);
                }
            }
    };
    const int q = lane >> 4, slot = (NV == 1 ? 0 : m >> 2) * S::planes + (S::planes == 3 ? min(m & 3, 2) : 0);
    const unsigned char *operand = mine + slot * S::stride + q * 16;
    const float *sum_of = sums + (NV == 1 ? 0 : q) * S::tiles * GPT;
    float total[NM] = {};
    if (t0 < t1) {
        request_v(t0);
        request_codes(t0);
    }
    for (int t = t0; t < t1; t += S::tiles) {
#pragma unroll
        for (int j = 0; j < S::loads; ++j) {
            const int i = j * 64 + lane;
            store_piece(mine + (i / S::pieces) * S::planes * S::stride + 16 * (i % S::pieces), S::stride, p[j]);
            const float x = run_sum<kRun>(piece_sum(p[j]));
            if (i % kRun == 0) sums[i / kRun] = -8.0f * x;
        }
        if (t + S::tiles < t1) request_v(t + S::tiles);
        // the wave's LDS operations execute in order: no barrier inside a wave
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        __builtin_amdgcn_wave_barrier();
#pragma unroll
        for (int i = 0; i < S::tiles; ++i) {
            if (t + i >= t1) break;
#pragma unroll
            for (int gr = 0; gr < GPT; ++gr) {
                f32x4 acc[NM] = {};
#pragma unroll
                for (int st = gr * kSteps; st < (gr + 1) * kSteps; ++st) {
                    const bf16x8 x = lds_operand(operand + i * kInt4Tile * 2 + st * 64);
#pragma unroll
                    for (int k = 0; k < NM; ++k) acc[k] = mfma16(x, decode(c[k][i][st >> 2][st & 3]), acc[k]);
                }
                const float minus = sum_of[i * GPT + gr];
#pragma unroll
                for (int k = 0; k < NM; ++k) {
                    float part = acc[k].x;
                    if (S::planes == 3) part += acc[k].y + acc[k].z;
                    total[k] += scale_of(sc[k][i], mat[k].wide, gr) * (part + minus * zero_factor(sc[k][i], mat[k], gr));
                }
            }
        }
        if (t + S::tiles < t1) request_codes(t + S::tiles);
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        __builtin_amdgcn_wave_barrier();
    }
    int group = blockIdx.x * (waves >> wk_log2) + wr;
    if (wk_log2 > 0) {
        float *red = reinterpret_cast<float *>(smem + waves * S::wave_bytes);
#pragma unroll
        for (int k = 0; k < NM; ++k) red[(w * NM + k) * 64 + lane] = total[k];
        __syncthreads();
        if (w >= waves >> wk_log2) return;
#pragma unroll
        for (int k = 0; k < NM; ++k) total[k] = 0.0f;
        for (int i = 0; i < 1 << wk_log2; ++i)
#pragma unroll
            for (int k = 0; k < NM; ++k) total[k] += red[(((w << wk_log2) + i) * NM + k) * 64 + lane];
        group = blockIdx.x * (waves >> wk_log2) + w;
    }
    const long long row = (long long)group * kDenseRows + m;
    if (q >= nv || row >= n_out) return;
    float result;
    if constexpr (NM == 2) {
        if (pre) {
            pre[2 * q * (long long)n_out + row] = total[0];
            pre[(2 * q + 1) * (long long)n_out + row] = total[1];
        }
        result = activate(act, total[0]) * total[NM - 1];
    } else {
        result = scale * total[0];
    }
    if (out_bf16)
        put(static_cast<uint16_t *>(out) + q * ldo + row, result);
    else
        put(static_cast<float *>(out) + q * ldo + row, result);
}

// ---- split: five to 32 vectors, and more where an estimate prefers it to tiles (split_us, tile_us) -------------
// WAVES waves share the columns of G row groups (of each matrix); each stages its own columns of 16 NT vectors, half a tile at
// a time.  The vectors are the rows of the MFMA: lane l of the result holds row l % 16 of vectors 4 (l / 16) .. + 3.
// 14336 x 4096, 16 bf16 vectors, groups of 64: 14.8 us (a plain read of the codes 6.5); a step's staging, decoding and scaling are
// about 160 vector instructions per two row groups, and there are few steps to a wave.
template <typename VT, int NT, int GPT>
struct Split {
    static constexpr int planes = sizeof(VT) == 4 ? 3 : 1;
    static constexpr int vectors = 16 * NT;
    static constexpr int cols = kInt4Tile / 2;  // staged at a time
    static constexpr int groups = GPT / 2;      // of them
    static constexpr int pieces = cols / 8;
    static constexpr int loads = vectors * pieces / 64;
    static constexpr int stride = cols * 2 + 16;  // bytes between vectors: an odd number of 16-byte units
    static constexpr int plane = vectors * stride;
    static constexpr int wave_bytes = planes * plane + groups * vectors * 4;
};

template <typename VT, int NT, int GPT, int NM, int G, int WAVES>
__global__ __launch_bounds__(WAVES * 64, WAVES / 4) void k_int4_split(
    Int4 m0, Int4 m1, const VT *__restrict__ v, int ntiles, int ngroups, int n_in, int n_out, long long ldv, int batch,
    float scale, void *__restrict__ out, int out_bf16, long long ldo, int act, float *__restrict__ pre) {
    using S = Split<VT, NT, GPT>;
    constexpr int kSteps = kInt4Steps / GPT, kRun = kInt4Tile / GPT / 8, kAcc = NM * G * NT * 4;
    extern __shared__ __attribute__((aligned(16))) unsigned char smem[];
    const int tid = threadIdx.x, lane = tid & 63;
    const int w = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int vec0 = blockIdx.y * S::vectors, group0 = blockIdx.x * G;
    const int halves = (n_in + S::cols - 1) / S::cols;
    const int h0 = (int)((long long)halves * w / WAVES), h1 = (int)((long long)halves * (w + 1) / WAVES);
    const Int4 mat[2] = {m0, m1};
    unsigned char *mine = smem + w * S::wave_bytes;
    float *sums = reinterpret_cast<float *>(mine + S::planes * S::plane);  // [group][vector]

    const VT *row[S::loads];
#pragma unroll
    for (int j = 0; j < S::loads; ++j)
        row[j] = v + (long long)min(vec0 + (j * 64 + lane) / S::pieces, batch - 1) * ldv;
    const int piece = lane % S::pieces;
    const uint32_t *code[NM][G];
    long long scale_row[NM][G];
#pragma unroll
    for (int k = 0; k < NM; ++k)
#pragma unroll
        for (int g = 0; g < G; ++g) {
            const long long rg = min(group0 + g, ngroups - 1);
            code[k][g] = mat[k].codes + rg * ntiles * kInt4TileDwords + lane * 4;
            scale_row[k][g] = (rg * ntiles * kDenseRows + (lane & 15)) * GPT;
        }
    Piece<VT> p[S::loads];
    auto request_v = [&](int h, auto whole) {
        if (whole || (h + 1) * S::cols <= n_in) {
#pragma unroll
            for (int j = 0; j < S::loads; ++j) p[j] = load_whole_piece<VT>(row[j] + h * S::cols + 8 * piece);
        } else {
#pragma unroll
            for (int j = 0; j < S::loads; ++j) p[j] = load_piece<VT>(row[j], h * S::cols + 8 * piece, n_in);
        }
    };
    auto request_codes = [&](int h, u32x4 (&c)[NM][G], Scales<S::groups> (&sc)[NM][G]) {
#pragma unroll
        for (int k = 0; k < NM; ++k)
#pragma unroll
            for (int g = 0; g < G; ++g) {
                c[k][g] = __builtin_nontemporal_load(reinterpret_cast<const u32x4 *>(code[k][g] + (long long)h * 256));
                sc[k][g] = load_scales<S::groups>(mat[k], scale_row[k][g] + (long long)(h >> 1) * kDenseRows * GPT + (h & 1) * S::groups);
            }
    };
    constexpr int kAhead = NM * G * NT <= 4 ? 2 : 1;  // half tiles whose codes are on their way
    u32x4 codes[kAhead][NM][G];
    Scales<S::groups> scales[kAhead][NM][G];
    float total[NM][G][NT][4] = {};
    auto step = [&](int h, u32x4 (&c)[NM][G], Scales<S::groups> (&sc)[NM][G], auto whole) __attribute__((always_inline)) {
#pragma unroll
        for (int j = 0; j < S::loads; ++j) {
            const int n = (j * 64 + lane) / S::pieces;
            store_piece(mine + n * S::stride + 16 * piece, S::plane, p[j]);
            const float x = run_sum<kRun>(piece_sum(p[j]));
            if (piece % kRun == 0) sums[piece / kRun * S::vectors + n] = -8.0f * x;
        }
        request_v(min(h + 1, h1 - 1), whole);
        // the wave's LDS operations execute in order: no barrier inside a wave
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        __builtin_amdgcn_wave_barrier();
        const unsigned char *operand = mine + (lane & 15) * S::stride + (lane >> 4) * 16;
#pragma unroll
        for (int gr = 0; gr < S::groups; ++gr) {
            f32x4 acc[NM][G][NT] = {};
#pragma unroll
            for (int st = gr * kSteps; st < (gr + 1) * kSteps; ++st) {
                bf16x8 x[NT][S::planes];
#pragma unroll
                for (int n = 0; n < NT; ++n)
#pragma unroll
                    for (int pl = 0; pl < S::planes; ++pl)
                        x[n][pl] = lds_operand(operand + pl * S::plane + n * 16 * S::stride + st * 64);
#pragma unroll
                for (int k = 0; k < NM; ++k)
#pragma unroll
                    for (int g = 0; g < G; ++g) {
                        const bf16x8 y = decode(c[k][g][st]);
#pragma unroll
                        for (int pl = 0; pl < S::planes; ++pl)
#pragma unroll
                            for (int n = 0; n < NT; ++n) acc[k][g][n] = mfma16(x[n][pl], y, acc[k][g][n]);
                    }
            }
#pragma unroll
            for (int n = 0; n < NT; ++n) {
                const f32x4 minus = *reinterpret_cast<const f32x4 *>(sums + gr * S::vectors + n * 16 + 4 * (lane >> 4));
#pragma unroll
                for (int k = 0; k < NM; ++k)
#pragma unroll
                    for (int g = 0; g < G; ++g) {
                        const float a = scale_of(sc[k][g], mat[k].wide, gr), z = zero_factor(sc[k][g], mat[k], gr);
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            total[k][g][n][i] += a * (acc[k][g][n][i] + minus[i] * z);
                            asm volatile("" : "+v"(total[k][g][n][i]));  // (here: see k_int4_tile)
                        }
                    }
            }
        }
        __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
        __builtin_amdgcn_wave_barrier();
        request_codes(min(h + kAhead, h1 - 1), c, sc);
    };
    // Requests behind the last half tile ask for it again: a branch around them would have all loads waited for behind it.
    auto run = [&](auto whole) __attribute__((always_inline)) {
        request_v(h0, whole);
#pragma unroll
        for (int d = 0; d < kAhead; ++d) request_codes(min(h0 + d, h1 - 1), codes[d], scales[d]);
        int h = h0;
        for (; h + kAhead <= h1; h += kAhead) {
#pragma unroll
            for (int d = 0; d < kAhead; ++d) step(h + d, codes[d], scales[d], whole);
        }
#pragma unroll
        for (int d = 0; d < kAhead - 1; ++d)
            if (h + d < h1) step(h + d, codes[d], scales[d], whole);
    };
    if (h0 < h1) {
        if (h1 * S::cols <= n_in)
            run(std::true_type());
        else
            run(std::false_type());
    }
    __syncthreads();  // the staging areas become the partial results [wave][matrix][group, 16 vectors, register][lane]
    float *red = reinterpret_cast<float *>(smem);
#pragma unroll
    for (int k = 0; k < NM; ++k)
#pragma unroll
        for (int i = 0; i < kAcc / NM; ++i)
            red[((w * NM + k) * (kAcc / NM) + i) * 64 + lane] = total[k][i / (4 * NT)][i / 4 % NT][i & 3];
    __syncthreads();
    for (int i = w; i < kAcc / NM; i += WAVES) {
        float sum[NM] = {};
#pragma unroll
        for (int k = 0; k < NM; ++k)
#pragma unroll
            for (int u = 0; u < WAVES; ++u) sum[k] += red[((u * NM + k) * (kAcc / NM) + i) * 64 + lane];
        const long long r = (long long)(group0 + i / (4 * NT)) * kDenseRows + (lane & 15);
        const int n = vec0 + i / 4 % NT * 16 + 4 * (lane >> 4) + (i & 3);
        if (n >= batch || r >= n_out) continue;
        float result;
        if constexpr (NM == 2) {
            if (pre) {
                pre[2 * n * (long long)n_out + r] = sum[0];
                pre[(2 * n + 1) * (long long)n_out + r] = sum[1];
            }
            result = activate(act, sum[0]) * sum[NM - 1];
        } else {
            result = scale * sum[0];
        }
        if (out_bf16)
            put(static_cast<uint16_t *>(out) + n * ldo + r, result);
        else
            put(static_cast<float *>(out) + n * ldo + r, result);
    }
}

// ---- tile: large batches -----------------------------------------------------------------------------
// Four waves, each with 64 rows (one matrix) or 32 rows of both, and the same 64 vectors; the vectors are staged in LDS, double
// buffered, one barrier per stage, and their sums over the groups with them; the codes come straight from memory, every
// wave those of its own rows.  A stage's group is decoded once into registers for all of the wave's vectors; its sum starts at
// minus eight times the vector's, and is scaled and added to the result's.
// 4096 x 14336, 2048 bf16 vectors, groups of 128: 270 us (890 TFLOP/s, a library product 191); 284 vector instructions to 32 MFMAs
// per wave and stage, MFMA busy 44 %, vector issue 48 %, hardly at the same time.  Measured against it: 256 rows x 128 vectors in
// eight waves 299, 128 x 128 in four with stages of 64 columns 429, 32 rows x 128 vectors per wave 302, 64 x 128 per wave with all 512
// registers 358; the next stage written between or behind the products 277 to 303; sums scaled behind the branches of a stage
// (where the compiler moves them if it may) spill 700 bytes.  Groups of 32: 392 us, a sum of 32 columns is two MFMAs and 16
// multiplications.  With zero points and groups of 128 three registers do not fit (16 bytes of scratch).
constexpr int kTileWaves = 4, kTileVecs = 2;  // 64 rows each; blocks of 32 vectors

template <typename VT, int GPT>
struct Tile {
    static constexpr int planes = sizeof(VT) == 4 ? 3 : 1;
    static constexpr int threads = 64 * kTileWaves;
    static constexpr int vectors = 32 * kTileVecs;
    static constexpr int cols = sizeof(VT) == 4 ? 64 : 128;  // staged at a time
    static constexpr int group = kInt4Tile / GPT < cols ? kInt4Tile / GPT : cols;
    static constexpr int groups = cols / group;
    static constexpr int scales = cols * GPT / kInt4Tile ? cols * GPT / kInt4Tile : 1;
    static constexpr int pieces = cols / 8;
    static constexpr int loads = vectors * pieces / threads;
    static constexpr int stride = cols * 2 + 16;
    static constexpr int plane = vectors * stride;
    static constexpr int buffer = planes * plane + groups * vectors * 4;
    static constexpr int dwords = cols / 32;  // of a lane and row group
};

template <typename VT, int GPT, int NM, bool ZEROS>
__global__ __launch_bounds__(64 * kTileWaves, 2) void k_int4_tile(
    Int4 m0, Int4 m1, const VT *__restrict__ v, int ntiles, int ngroups, int n_in, int n_out, long long ldv, int batch,
    float scale, void *__restrict__ out, int out_bf16, long long ldo, int act, float *__restrict__ pre, int row_tiles,
    int vec_tiles) {
    using S = Tile<VT, GPT>;
    constexpr int kRows = kTileWaves * 64 / NM, kRun = S::group / 8;
    extern __shared__ __attribute__((aligned(16))) unsigned char smem[];
    const int tid = threadIdx.x, lane = tid & 63, half = lane >> 5;
    const int w = __builtin_amdgcn_readfirstlane(tid >> 6);
    // consecutive workgroups go to the eight XCDs in turn: each XCD gets a contiguous run of
    // tiles, eight row tiles for every vector tile, so that its L2 sees the same vectors again
    const int all = row_tiles * vec_tiles, per = (all + 7) / 8;
    const int lin = (blockIdx.x & 7) * per + (blockIdx.x >> 3);
    if ((int)(blockIdx.x >> 3) >= per || lin >= all) return;
    const int band = lin / (8 * vec_tiles), in_band = lin - band * 8 * vec_tiles;
    const int band_rows = min(8, row_tiles - band * 8);
    const int rt = band * 8 + in_band % band_rows, vec0 = in_band / band_rows * S::vectors;
    const Int4 mat[2] = {m0, NM == 2 ? m1 : m0};

    // piece j of this thread: of vector mine + j * kApart, a uniform distance further on (no vector there: the last one again, not stored)
    constexpr int kApart = S::threads / S::pieces;
    const int piece = tid % S::pieces, mine = tid / S::pieces;
    const VT *first = v + (long long)min(vec0 + mine, batch - 1) * ldv + 8 * piece;
    unsigned char *const to = smem + mine * S::stride + 16 * piece;
    float *const sum_to = reinterpret_cast<float *>(smem + S::planes * S::plane) + piece / kRun * S::vectors + mine;
    // row block r: matrix r of two, or the next 32 rows
    const int row0 = rt * kRows + w * (64 / NM);
    const uint32_t *code[2][2];
    long long scale_row[2];
#pragma unroll
    for (int r = 0; r < 2; ++r) {
        const int rg = row0 / kDenseRows + (NM == 2 ? 0 : 2 * r);
#pragma unroll
        for (int g = 0; g < 2; ++g)
            code[r][g] = mat[r].codes + (long long)min(rg + g, ngroups - 1) * ntiles * kInt4TileDwords + lane * 4;
        scale_row[r] = ((long long)min(rg + ((lane >> 4) & 1), ngroups - 1) * ntiles * kDenseRows + (lane & 15)) * GPT;
    }
    Piece<VT> p[S::loads];
    const bool whole = vec0 + S::vectors <= batch;
    const int whole_stages = whole ? n_in / S::cols : 0;
    auto request_v = [&](int s) {
        if (s < whole_stages) {
#pragma unroll
            for (int j = 0; j < S::loads; ++j)
                p[j] = load_whole_piece<VT>(first + j * (kApart * ldv) + s * S::cols);
        } else {
#pragma unroll
            for (int j = 0; j < S::loads; ++j)
                p[j] = load_piece<VT>(v + (long long)min(vec0 + mine + j * kApart, batch - 1) * ldv, s * S::cols + 8 * piece, n_in);
        }
    };
    auto stage = [&](int buf) {
#pragma unroll
        for (int j = 0; j < S::loads; ++j) {
            store_piece(to + buf * S::buffer + j * kApart * S::stride, S::plane, p[j]);
            const float x = run_sum<kRun>(piece_sum(p[j]));
            sum_to[buf * (S::buffer / 4) + j * kApart] = -8.0f * x;  // (every lane of the run, the same)
        }
    };
    auto request_codes = [&](int s, uint32_t (&c)[2][2][S::dwords], Scales<S::scales> (&sc)[2]) {
#pragma unroll
        for (int r = 0; r < 2; ++r) {
#pragma unroll
            for (int g = 0; g < 2; ++g) {
                if constexpr (S::dwords == 4) {
                    const u32x4 x = *reinterpret_cast<const u32x4 *>(code[r][g] + (long long)s * 256);
#pragma unroll
                    for (int d = 0; d < 4; ++d) c[r][g][d] = x[d];
                } else {
                    const u32x2 x = *reinterpret_cast<const u32x2 *>(code[r][g] + (long long)(s >> 1) * 256 + (s & 1) * 2);
                    c[r][g][0] = x.x;
                    c[r][g][1] = x.y;
                }
            }
            constexpr int kPerTile = kInt4Tile / S::cols;
            sc[r] = load_scales<S::scales>(mat[r], scale_row[r] + (long long)(s / kPerTile) * kDenseRows * GPT +
                                                       s % kPerTile * S::cols * GPT / kInt4Tile);
        }
    };
    float total[2][kTileVecs][16] = {};
    uint32_t c[2][2][S::dwords], cn[2][2][S::dwords];
    Scales<S::scales> sc[2], scn[2];
    const int stages = (n_in + S::cols - 1) / S::cols;
    request_codes(0, c, sc);
    request_v(0);
    stage(0);
    if (stages > 1) request_v(1);
    __syncthreads();
    auto step = [&](int s, auto steady) __attribute__((always_inline)) {
        request_codes(min(s + 1, stages - 1), cn, scn);
        // the next stage goes to the other buffer, which nobody reads any more
        if constexpr (steady) {
            stage((s + 1) & 1);
#pragma unroll
            for (int j = 0; j < S::loads; ++j)
                p[j] = load_whole_piece<VT>(first + j * (kApart * ldv) + (s + 2) * S::cols);
        } else {
            if (s + 1 < stages) stage((s + 1) & 1);
            if (s + 2 < stages) request_v(s + 2);
        }
#pragma unroll
        for (int r = 0; r < 2; ++r)
#pragma unroll
            for (int d = 0; d < S::dwords; ++d) {
                // lanes below 32: slice 0 (then 1) of both row groups, the others: slice 2 (3)
                const auto x = __builtin_amdgcn_permlane16_swap(c[r][0][d], c[r][1][d], false, false);
                c[r][0][d] = x[0];
                c[r][1][d] = x[1];
            }
        const unsigned char *buf = smem + (s & 1) * S::buffer;
        const float *sums = reinterpret_cast<const float *>(buf + S::planes * S::plane) + 4 * half;
        buf += (lane & 31) * S::stride + 32 * half;
#pragma unroll
        for (int gr = 0; gr < S::groups; ++gr) {
            bf16x8 x[2][S::group / 16];
            float a[2], z[2];
#pragma unroll
            for (int r = 0; r < 2; ++r) {
#pragma unroll
                for (int ks = 0; ks < S::group / 16; ++ks) x[r][ks] = decode(c[r][ks & 1][gr * (S::group / 32) + ks / 2]);
                a[r] = scale_of(sc[r], mat[r].wide, S::scales == 1 ? 0 : gr);
                z[r] = zero_factor(sc[r], mat[r], S::scales == 1 ? 0 : gr);
            }
#pragma unroll
            for (int n = 0; n < kTileVecs; ++n) {
                f32x16 minus;
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const f32x4 q = *reinterpret_cast<const f32x4 *>(sums + gr * S::vectors + n * 32 + 8 * i);
#pragma unroll
                    for (int e = 0; e < 4; ++e) minus[4 * i + e] = q[e];
                }
                f32x16 acc[2] = {minus, minus};
                if constexpr (ZEROS) {
#pragma unroll
                    for (int r = 0; r < 2; ++r)
#pragma unroll
                        for (int i = 0; i < 16; ++i) acc[r][i] *= z[r];
                }
#pragma unroll
                for (int ks = 0; ks < S::group / 16; ++ks)
#pragma unroll
                    for (int pl = 0; pl < S::planes; ++pl) {
                        const bf16x8 o = lds_operand(buf + pl * S::plane + n * 32 * S::stride + gr * S::group * 2 + (ks >> 1) * 64 + (ks & 1) * 16);
#pragma unroll
                        for (int r = 0; r < 2; ++r) acc[r] = mfma32(o, x[r][ks], acc[r]);
                    }
#pragma unroll
                for (int r = 0; r < 2; ++r)
#pragma unroll
                    for (int i = 0; i < 16; ++i) {
                        total[r][n][i] += a[r] * acc[r][i];
                        // (here, and not behind the branches below: all blocks' sums at once do not fit the registers)
                        asm volatile("" : "+v"(total[r][n][i]));
                    }
            }
        }
        __syncthreads();
#pragma unroll
        for (int r = 0; r < 2; ++r) {
#pragma unroll
            for (int g = 0; g < 2; ++g)
#pragma unroll
                for (int d = 0; d < S::dwords; ++d) c[r][g][d] = cn[r][g][d];
            sc[r] = scn[r];
        }
    };
    int s = 0;
    for (; s + 2 < whole_stages; ++s) step(s, std::true_type());
    for (; s < stages; ++s) step(s, std::false_type());
    // The codes requested last are not used.  They are waited for here (vmcnt = 0): if one of their
    // registers comes to hold an address or a result below, every store gets a wait for all that is on its way.
    __builtin_amdgcn_s_waitcnt(0x0f70);
#pragma unroll
    for (int r = 0; r < (NM == 2 ? 1 : 2); ++r) {
        const int row_out = row0 + r * 32 + (lane & 31);
#pragma unroll
        for (int b = 0; b < kTileVecs; ++b)
#pragma unroll
            for (int i = 0; i < 16; ++i) {
                const long long n = vec0 + b * 32 + acc_row(i, half);
                if (n >= batch || row_out >= n_out) continue;
                float result;
                if constexpr (NM == 2) {
                    if (pre) {
                        pre[2 * n * n_out + row_out] = total[0][b][i];
                        pre[(2 * n + 1) * n_out + row_out] = total[1][b][i];
                    }
                    result = activate(act, total[0][b][i]) * total[1][b][i];
                } else {
                    result = scale * total[r][b][i];
                }
                if (out_bf16)
                    put(static_cast<uint16_t *>(out) + n * ldo + row_out, result);
                else
                    put(static_cast<float *>(out) + n * ldo + row_out, result);
            }
    }
}

}  // namespace

int64_t int4_code_bytes(int64_t rows, int64_t cols) {
    return row_groups(rows) * ((cols + kInt4Tile - 1) / kInt4Tile) * kInt4TileDwords * 4;
}
int64_t int4_groups(int64_t rows, int64_t cols, int per) {
    return row_groups(rows) * ((cols + kInt4Tile - 1) / kInt4Tile) * kDenseRows * (kInt4Tile / per);
}

hipError_t launch_int4_check_scales(const float *scales, const int8_t *zeros, int64_t count, int *flags) {
    const int64_t blocks = (count + 255) / 256;
    hipLaunchKernelGGL(k_int4_check_scales, dim3((unsigned)(blocks < 4096 ? blocks : 4096)), dim3(256), 0, 0, scales, zeros,
                       count, flags);
    return hipGetLastError();
}

hipError_t launch_int4_pack(const rsr_handle_s *h, const int8_t *Q, const float *scales, const int8_t *zeros,
                            int64_t group, int *flags) {
    const int64_t ntiles = (h->cols + kInt4Tile - 1) / kInt4Tile;
    // (a launch holds fewer than 2^32 threads: so many row groups at a time)
    const int64_t band = (((int64_t)1 << 31) / (64 * ntiles)) * kDenseRows;
    uint32_t *to = reinterpret_cast<uint32_t *>(h->packed);
    for (int64_t r = 0; r < h->rows; r += band) {
        const int64_t n = h->rows - r < band ? h->rows - r : band, threads = row_groups(n) * ntiles * 64;
        hipLaunchKernelGGL(k_int4_pack, dim3((unsigned)((threads + 255) / 256)), dim3(256), 0, 0, Q + r * h->cols, n, h->cols,
                           ntiles, threads, to, flags);
        if (hipError_t e = hipGetLastError()) return e;
        to += threads * kInt4Steps;
    }
    const int64_t per_group = ntiles * kDenseRows * (kInt4Tile / h->group), most = ((int64_t)1 << 31) / per_group;
    const int64_t n_groups = (h->cols + group - 1) / group;
    for (int64_t G = 0; G < row_groups(h->rows); G += most) {
        const int64_t r = G * kDenseRows, left = row_groups(h->rows) - G, count = (left < most ? left : most) * per_group;
        void *at = static_cast<unsigned char *>(h->scales) + G * per_group * (h->wide_scales ? 4 : 2);
        hipLaunchKernelGGL(k_int4_pack_scales, dim3((unsigned)((count + 255) / 256)), dim3(256), 0, 0, scales + r * n_groups,
                           zeros ? zeros + r * n_groups : nullptr, h->rows - r, h->cols, group, ntiles, h->group, count,
                           h->wide_scales, at, zeros ? h->zeros + G * per_group : nullptr);
        if (hipError_t e = hipGetLastError()) return e;
    }
    return hipSuccess;
}

namespace {

struct Args {
    Int4 m[2];
    const void *v;
    int ntiles, ngroups, n_in, n_out, batch, device;
    long long ldv, ldo;
    float scale;
    void *out;
    int out_bf16, act;
    float *pre;
    hipStream_t stream;
    char *name;  // not null: write the name of the kernel there instead of launching it
    size_t name_len;
};

template <typename VT, typename... Number>
hipError_t put_name(const Args &x, const char *kernel, const char *numbers, Number... n) {
    if (x.name[0]) return hipSuccess;  // (of several launches the first)
    const int at = std::snprintf(x.name, x.name_len, "%s<%s, ", kernel, sizeof(VT) == 4 ? "float" : "unsigned short");
    if (at > 0 && (size_t)at < x.name_len) std::snprintf(x.name + at, x.name_len - at, numbers, n...);
    return hipSuccess;
}

// Waves that share the columns of a row group: as many as stage all of theirs at once, and more while the chip has fewer
// than four waves per CU.  Measured, one bf16 vector, 1 / 2 / 4 / 8 / 16 waves: 4096 x 14336 30.5 / 17.5 / 12.0 / 9.2 / 8.4 us, 14336 x 4096
// 12.0 / 9.1 / 8.4 / 9.1 / 12.4 (4 are taken), 2560 x 6912 16.4 / 10.1 / 6.4 / 5.2 / 5.1, 640 x 2560 7.2 / 4.9 / 3.4 / 3.4 / 3.6; four vectors on
// 4096 x 14336 41 / 23 / 13 / 11 / 10.
int few_wk_log2(int ntiles, int ngroups, int tiles, int most) {
    int log2 = 0;
    while (2 << log2 <= most && (ntiles + tiles - 1) / tiles > 1 << log2) ++log2;
    while (2 << log2 <= most && 1 << log2 < ntiles && (long long)ngroups << log2 < 1024) ++log2;
    return log2;
}

template <typename VT, int NV, int GPT, int NM>
hipError_t launch_few(const Args &x) {
    using S = Few<VT, NV, GPT>;
    if (x.name) return put_name<VT>(x, "k_int4_few", "%d, %d, %d>", NV, GPT, NM);
    static std::atomic<size_t> enabled[kMaxDevices];
    auto kern = k_int4_few<VT, NV, GPT, NM>;
    const int wk_log2 = few_wk_log2(x.ntiles, x.ngroups, S::tiles, few_most_waves(NM));
    int waves = wk_log2 < 2 ? 4 : 1 << wk_log2;
    const size_t lds = (size_t)waves * (S::wave_bytes + NM * 64 * 4);
    static_assert(few_most_waves(NM) * (S::wave_bytes + NM * 64 * 4) <= kLdsBytes, "every wave stages columns of its own");
    if (hipError_t e = ensure_dynamic_lds(reinterpret_cast<const void *>(kern), lds, x.device, enabled)) return e;
    const int groups = waves >> wk_log2;
    hipLaunchKernelGGL(kern, dim3((unsigned)((x.ngroups + groups - 1) / groups)), dim3(waves * 64), lds, x.stream, x.m[0],
                       x.m[1], static_cast<const VT *>(x.v), x.ntiles, x.ngroups, x.n_in, x.n_out, x.ldv, x.batch,
                       wk_log2, x.scale, x.out, x.out_bf16, x.ldo, x.act, x.pre);
    return hipGetLastError();
}

template <typename VT, int NT, int GPT, int NM, int G, int WAVES>
hipError_t launch_split_rows(const Args &x) {
    using S = Split<VT, NT, GPT>;
    if (x.name) return put_name<VT>(x, "k_int4_split", "%d, %d, %d, %d, %d>", NT, GPT, NM, G, WAVES);
    static std::atomic<size_t> enabled[kMaxDevices];
    auto kern = k_int4_split<VT, NT, GPT, NM, G, WAVES>;
    constexpr size_t staged = (size_t)WAVES * S::wave_bytes, joined = (size_t)WAVES * NM * G * NT * 4 * 64 * 4;
    constexpr size_t lds = staged > joined ? staged : joined;
    static_assert(lds <= (size_t)kLdsBytes, "staging, and then the partial results of all waves");
    if (hipError_t e = ensure_dynamic_lds(reinterpret_cast<const void *>(kern), lds, x.device, enabled)) return e;
    hipLaunchKernelGGL(kern, dim3((unsigned)((x.ngroups + G - 1) / G), (unsigned)((x.batch + S::vectors - 1) / S::vectors)),
                       dim3(WAVES * 64), lds, x.stream, x.m[0], x.m[1], static_cast<const VT *>(x.v), x.ntiles, x.ngroups,
                       x.n_in, x.n_out, x.ldv, x.batch, x.scale, x.out, x.out_bf16, x.ldo, x.act, x.pre);
    return hipGetLastError();
}

template <typename VT, int GPT, int NM>
hipError_t launch_split(const Args &x) {
    // one row group per workgroup while there are fewer than two workgroups per CU, and sixteen waves for it where each gets two
    // steps.  Measured, two row groups / one / one with sixteen waves: 4096 x 14336, 8 vectors 15.7 / 13.4 / 11.6 us, 16 vectors 16.5 /
    // 14.0 / 13.6, 32 23.6 / 20.1 / -, 64 23.8 / 37.0 / -; 14336 x 4096, 16 vectors 13.8 / 16.0 / 20.0, 32 19.7 / 26.1 / -; 2560 x 6912, 16
    // 9.5 / 8.0 / 8.1; 640 x 2560, 16 5.5 / 4.7 / 5.1.
    constexpr int kVectors = sizeof(VT) == 4 ? 16 : 32;
    const bool few_rows = (long long)x.ngroups * ((x.batch + kVectors - 1) / kVectors) < 512;
    if (x.batch <= 16 || sizeof(VT) == 4) {
        if constexpr (sizeof(VT) == 2)
            if (few_rows && x.n_in >= 4096) return launch_split_rows<VT, 1, GPT, NM, 1, 16>(x);
        return few_rows ? launch_split_rows<VT, 1, GPT, NM, 1, 8>(x) : launch_split_rows<VT, 1, GPT, NM, 2, 8>(x);
    }
    if constexpr (sizeof(VT) == 2)
        return few_rows ? launch_split_rows<VT, 2, GPT, NM, 1, 8>(x) : launch_split_rows<VT, 2, GPT, NM, 2, 8>(x);
    return hipErrorInvalidValue;
}

template <typename VT, int GPT, int NM, bool ZEROS>
hipError_t launch_tile_shape(const Args &x) {
    using S = Tile<VT, GPT>;
    if (x.name) return put_name<VT>(x, "k_int4_tile", "%d, %d, %s>", GPT, NM, ZEROS ? "true" : "false");
    static std::atomic<size_t> enabled[kMaxDevices];
    auto kern = k_int4_tile<VT, GPT, NM, ZEROS>;
    constexpr size_t lds = 2 * (size_t)S::buffer;
    static_assert(lds <= (size_t)kLdsBytes, "two stages");
    if (hipError_t e = ensure_dynamic_lds(reinterpret_cast<const void *>(kern), lds, x.device, enabled)) return e;
    constexpr int rows = kTileWaves * 64 / NM;
    const int row_tiles = (x.n_out + rows - 1) / rows, vec_tiles = (x.batch + S::vectors - 1) / S::vectors;
    const int per = (int)(((long long)row_tiles * vec_tiles + 7) / 8);
    hipLaunchKernelGGL(kern, dim3((unsigned)(per * 8)), dim3(S::threads), lds, x.stream, x.m[0], x.m[1],
                       static_cast<const VT *>(x.v), x.ntiles, x.ngroups, x.n_in, x.n_out, x.ldv, x.batch, x.scale, x.out,
                       x.out_bf16, x.ldo, x.act, x.pre, row_tiles, vec_tiles);
    return hipGetLastError();
}

// Estimates in microseconds that decide between the two for more than 32 vectors.  split goes by the half tiles that
// all workgroups together multiply; a tile's workgroup takes 1.45 us (float32 1.7) per stage of its columns, alone on its CU
// or not, two of them 1.65 times as long.  Measured, split / tile: bf16 14336 x 4096, 64 vectors 36 / 51, 128 62 / 51;
// 4096 x 14336, 256 vectors 143 / 157; 6912 x 2560, 256 68 / 35; 2560 x 6912, 256 48 / 79; 640 x 2560, 256 11 / 33; float32 14336 x
// 4096, 100 vectors 116 / 111; 4096 x 14336, 100 148 / 369.
template <bool WIDE>
float split_us(const Args &x, int nm) {
    const float halves = (float)((x.n_in + 127) / 128), sets = (float)(WIDE ? (x.batch + 15) / 16 : (x.batch + 31) / 32);
    return 4.0f + (WIDE ? 0.6e-3f : 0.5e-3f) * (float)nm * (float)x.ngroups * halves * sets;
}
template <bool WIDE>
float tile_us(const Args &x, int nm) {
    const int rows = kTileWaves * 64 / nm;
    const float groups = (float)(((long long)x.n_out + rows - 1) / rows) * (float)((x.batch + 63) / 64);
    const float rounds = groups <= 256.0f ? 1.0f : groups <= 512.0f ? 1.65f : 1.65f * groups / 512.0f;
    return 3.0f + (WIDE ? 1.7f * (float)((x.n_in + 63) / 64) : 1.45f * (float)((x.n_in + 127) / 128)) * rounds;
}

template <typename VT, int GPT, int NM>
hipError_t launch_any(const Args &x) {
    if (x.batch == 1) return launch_few<VT, 1, GPT, NM>(x);
    if (x.batch <= 4) return launch_few<VT, 4, GPT, NM>(x);
    if (x.batch <= 32 || split_us<sizeof(VT) == 4>(x, NM) < tile_us<sizeof(VT) == 4>(x, NM)) return launch_split<VT, GPT, NM>(x);
    return x.m[0].zeros || x.m[1].zeros ? launch_tile_shape<VT, GPT, NM, true>(x) : launch_tile_shape<VT, GPT, NM, false>(x);
}

template <typename VT, int NM>
hipError_t launch_all(const Args &x, int group) {
    return group == 32 ? launch_any<VT, 8, NM>(x) : group == 64 ? launch_any<VT, 4, NM>(x) : launch_any<VT, 2, NM>(x);
}

// (A launch holds fewer than 2^32 threads, at most 512 per row group and 16 vectors, and 65535 sets of vectors: so many at a time.  Split with
// sixteen waves has 1024 per row group, but fewer than 512 workgroups.)
template <typename VT, int NM>
hipError_t launch_groups(const Args &x, int group) {
    const long long sets = (1LL << 31) / (512LL * x.ngroups);
    const int most = 16 * (int)(sets < 4 ? 4 : sets > 32768 ? 32768 : sets);
    if (x.batch <= most) return launch_all<VT, NM>(x, group);
    Args y = x;
    for (int n = 0; n < x.batch; n += most) {
        y.batch = x.batch - n < most ? x.batch - n : most;
        y.v = static_cast<const VT *>(x.v) + n * x.ldv;
        y.out = static_cast<unsigned char *>(x.out) + n * x.ldo * (x.out_bf16 ? 2 : 4);
        if (x.pre) y.pre = x.pre + 2LL * n * x.n_out;
        if (hipError_t e = launch_all<VT, NM>(y, group)) return e;
    }
    return hipSuccess;
}

Args args_of(const rsr_handle_s *a, const rsr_handle_s *b, int act, const void *v, float scale, void *out, int out_dtype,
             float *pre, int batch, int64_t ldv, int64_t ldo, hipStream_t stream) {
    Args x = {};
    x.m[0] = int4_of(a);
    if (b) x.m[1] = int4_of(b);
    x.v = v;
    x.ntiles = (int)((a->cols + kInt4Tile - 1) / kInt4Tile);
    x.ngroups = (int)row_groups(a->rows);
    x.n_in = (int)a->cols;
    x.n_out = (int)a->rows;
    x.batch = batch;
    x.device = a->device;
    x.ldv = ldv;
    x.ldo = ldo;
    x.scale = scale;
    x.out = out;
    x.out_bf16 = out_dtype == RSR_BF16;
    x.act = act;
    x.pre = pre;
    x.stream = stream;
    return x;
}

}  // namespace

hipError_t launch_int4(const rsr_handle_s *h, const void *v, int v_dtype, float scale, void *out, int out_dtype,
                       int batch, int64_t ldv, int64_t ldo, hipStream_t stream) {
    const Args x = args_of(h, nullptr, 0, v, scale, out, out_dtype, nullptr, batch, ldv, ldo, stream);
    return v_dtype == RSR_BF16 ? launch_groups<uint16_t, 1>(x, h->group) : launch_groups<float, 1>(x, h->group);
}

void int4_kernel_name(const rsr_handle_s *h, const rsr_handle_s *up, int v_dtype, int batch, char *buf, size_t len) {
    Args x = args_of(h, up, 0, nullptr, 1.0f, nullptr, RSR_F32, nullptr, batch, h->cols, h->rows, nullptr);
    x.name = buf;
    x.name_len = len;
    buf[0] = 0;
    if (up)
        (void)(v_dtype == RSR_BF16 ? launch_groups<uint16_t, 2>(x, h->group) : launch_groups<float, 2>(x, h->group));
    else
        (void)(v_dtype == RSR_BF16 ? launch_groups<uint16_t, 1>(x, h->group) : launch_groups<float, 1>(x, h->group));
}

hipError_t launch_int4_gated(const rsr_handle_s *gate, const rsr_handle_s *up, const void *v, int v_dtype, int act,
                             void *out, int out_dtype, float *pre, int batch, int64_t ldv, int64_t ldo,
                             hipStream_t stream) {
    const Args x = args_of(gate, up, act, v, 1.0f, out, out_dtype, pre, batch, ldv, ldo, stream);
    return v_dtype == RSR_BF16 ? launch_groups<uint16_t, 2>(x, gate->group) : launch_groups<float, 2>(x, gate->group);
}

}  // namespace rsr
