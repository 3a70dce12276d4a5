// Products with 4-bit weights and group scales (gfx950): packing, and y = scale M x for one or many vectors; with two
// matrices of one shape, h = act(Mg x) * (Mu x).
#include "rsr_int4.h"

namespace rsr {

namespace {

// ---- packing --------------------------------------------------------------------------------------
// One thread per (row group, tile, lane): its eight dwords.
__global__ __launch_bounds__(256) void k_int4_pack(const int8_t *__restrict__ Q, int64_t rows, int64_t cols,
                                                   int64_t ntiles, int64_t threads, uint32_t *__restrict__ codes,
                                                   int *__restrict__ flags) {
    const int64_t gid = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (gid >= threads) return;
    const int lane = (int)(gid & 63);
    const int64_t gt = gid >> 6, G = gt / ntiles, t = gt - G * ntiles;
    const int64_t i = G * kDenseRows + (lane & 15);
    bool bad = false;
#pragma unroll
    for (int d = 0; d < kInt4Steps; ++d) {
        const int64_t j0 = t * kInt4Tile + 32 * d + 8 * (lane >> 4);
        uint32_t word = 0x88888888u;  // zero
        if (i < rows) {
            for (int e = 0; e < 8 && j0 + e < cols; ++e) {
                const int q = Q[i * cols + j0 + e];
                bad |= q < -8 || q > 7;
                const int at = 8 * (e & 3) + 4 * (e >> 2);
                word = (word & ~(15u << at)) | ((uint32_t)(q + 8) & 15u) << at;
            }
        }
        codes[gt * kInt4TileDwords + (d >> 2) * 256 + lane * 4 + (d & 3)] = word;
    }
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

// ---- a row of a vector per thread --------------------------------------------------------------------
template <typename VT>
__device__ float dot(const Int4 &m, int gpt, int ntiles, const VT *x, int n_in, long long row) {
    const long long G = row / kDenseRows;
    const int r = (int)(row % kDenseRows), steps = kInt4Steps / gpt;
    float sum = 0.0f, part = 0.0f, total = 0.0f;
    for (int t = 0; t < ntiles; ++t)
        for (int d = 0; d < kInt4Steps; ++d) {
            for (int slice = 0; slice < 4; ++slice) {
                const uint32_t w = m.codes[(G * ntiles + t) * kInt4TileDwords + (d >> 2) * 256 + (16 * slice + r) * 4 + (d & 3)];
                for (int e = 0; e < 8; ++e) {
                    const int j = t * kInt4Tile + 32 * d + 8 * slice + e;
                    if (j >= n_in) break;
                    const float v = widen(x[j]);
                    part += (float)((w >> (8 * (e & 3) + 4 * (e >> 2))) & 15u) * v;
                    total += v;
                }
            }
            if ((d + 1) % steps == 0) {
                const long long idx = ((G * ntiles + t) * kDenseRows + r) * gpt + d / steps;
                const float z = m.zeros ? (float)m.zeros[idx] : 0.0f;
                sum += scale_at(m, idx) * (part - (8.0f + z) * total);
                part = total = 0.0f;
            }
        }
    return sum;
}

template <typename VT, typename OT>
__global__ __launch_bounds__(256) void k_int4_rows(Int4 a, Int4 b, int gated, int act, int gpt, int ntiles,
                                                   const VT *__restrict__ v, int n_in, int n_out, long long ldv,
                                                   float scale, OT *__restrict__ out, long long ldo, float *__restrict__ pre) {
    const int row = blockIdx.x * 256 + threadIdx.x;
    const long long n = blockIdx.y + (long long)blockIdx.z * 32768;
    if (row >= n_out) return;
    const float x = dot(a, gpt, ntiles, v + n * ldv, n_in, row);
    if (!gated) {
        put(out + n * ldo + row, scale * x);
        return;
    }
    const float y = dot(b, gpt, ntiles, v + n * ldv, n_in, row);
    if (pre) {
        pre[2 * n * n_out + row] = x;
        pre[(2 * n + 1) * n_out + row] = y;
    }
    put(out + n * ldo + row, activate(act, x) * y);
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

template <typename VT, typename OT>
hipError_t launch(const rsr_handle_s *a, const rsr_handle_s *b, int act, const void *v, float scale, void *out,
                  float *pre, int batch, int64_t ldv, int64_t ldo, hipStream_t stream) {
    const int ntiles = (int)((a->cols + kInt4Tile - 1) / kInt4Tile);
    const dim3 grid((unsigned)((a->rows + 255) / 256), (unsigned)(batch < 32768 ? batch : 32768));
    for (int n = 0; n < batch; n += 32768) {
        const int some = batch - n < 32768 ? batch - n : 32768;
        hipLaunchKernelGGL((k_int4_rows<VT, OT>), dim3(grid.x, (unsigned)some), dim3(256), 0, stream, int4_of(a),
                           b ? int4_of(b) : Int4{}, b != nullptr, act, kInt4Tile / a->group, ntiles,
                           static_cast<const VT *>(v) + n * ldv, (int)a->cols, (int)a->rows, (long long)ldv, scale,
                           static_cast<OT *>(out) + n * ldo, (long long)ldo, pre ? pre + 2 * n * a->rows : nullptr);
        if (hipError_t e = hipGetLastError()) return e;
    }
    return hipSuccess;
}

template <typename VT>
hipError_t launch_to(const rsr_handle_s *a, const rsr_handle_s *b, int act, const void *v, float scale, void *out,
                     int out_dtype, float *pre, int batch, int64_t ldv, int64_t ldo, hipStream_t stream) {
    return out_dtype == RSR_BF16 ? launch<VT, uint16_t>(a, b, act, v, scale, out, pre, batch, ldv, ldo, stream)
                                 : launch<VT, float>(a, b, act, v, scale, out, pre, batch, ldv, ldo, stream);
}

}  // namespace

hipError_t launch_int4(const rsr_handle_s *h, const void *v, int v_dtype, float scale, void *out, int out_dtype,
                       int batch, int64_t ldv, int64_t ldo, hipStream_t stream) {
    return v_dtype == RSR_BF16
               ? launch_to<uint16_t>(h, nullptr, 0, v, scale, out, out_dtype, nullptr, batch, ldv, ldo, stream)
               : launch_to<float>(h, nullptr, 0, v, scale, out, out_dtype, nullptr, batch, ldv, ldo, stream);
}

hipError_t launch_int4_gated(const rsr_handle_s *gate, const rsr_handle_s *up, const void *v, int v_dtype, int act,
                             void *out, int out_dtype, float *pre, int batch, int64_t ldv, int64_t ldo,
                             hipStream_t stream) {
    return v_dtype == RSR_BF16
               ? launch_to<uint16_t>(gate, up, act, v, 1.0f, out, out_dtype, pre, batch, ldv, ldo, stream)
               : launch_to<float>(gate, up, act, v, 1.0f, out, out_dtype, pre, batch, ldv, ldo, stream);
}

}  // namespace rsr
