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

// ---- a column of a vector per thread -----------------------------------------------------------------
template <typename VT>
__device__ float column_dot(const Int4 &m, int gpt, int ntiles, const VT *dy, int n_rows, int col) {
    const int t = col / kInt4Tile, c = col % kInt4Tile, d = c / 32, slice = c % 32 / 8, e = c % 8;
    float sum = 0.0f;
    for (int row = 0; row < n_rows; ++row) {
        const long long G = row / kDenseRows;
        const int r = row % kDenseRows;
        const uint32_t w = m.codes[(G * ntiles + t) * kInt4TileDwords + (d >> 2) * 256 + (16 * slice + r) * 4 + (d & 3)];
        const long long idx = ((G * ntiles + t) * kDenseRows + r) * gpt + d / (kInt4Steps / gpt);
        const float z = m.zeros ? (float)m.zeros[idx] : 0.0f;
        const float u = (float)((w >> (8 * (e & 3) + 4 * (e >> 2))) & 15u);
        sum += scale_at(m, idx) * widen(dy[row]) * (u - (8.0f + z));
    }
    return sum;
}

template <typename VT, typename OT>
__global__ __launch_bounds__(256) void k_int4_columns(Int4 a, Int4 b, int both, int gpt, int ntiles,
                                                      const VT *__restrict__ dy, int n_rows, int n_cols, long long ldv,
                                                      float scale, OT *__restrict__ out, long long ldo) {
    const int col = blockIdx.x * 256 + threadIdx.x;
    const long long n = blockIdx.y;
    if (col >= n_cols) return;
    float x = column_dot(a, gpt, ntiles, dy + n * ldv, n_rows, col);
    if (both) x += column_dot(b, gpt, ntiles, dy + n * ldv + n_rows, n_rows, col);
    put(out + n * ldo + col, scale * x);
}

template <typename VT, typename OT>
hipError_t launch(const rsr_handle_s *a, const rsr_handle_s *b, const void *dy, float scale, void *out, int batch,
                  int64_t ldv, int64_t ldo, hipStream_t stream) {
    const int ntiles = (int)((a->cols + kInt4Tile - 1) / kInt4Tile);
    for (int n = 0; n < batch; n += 32768) {
        const int some = batch - n < 32768 ? batch - n : 32768;
        hipLaunchKernelGGL((k_int4_columns<VT, OT>), dim3((unsigned)((a->cols + 255) / 256), (unsigned)some), dim3(256), 0,
                           stream, int4_of(a), b ? int4_of(b) : Int4{}, b != nullptr, kInt4Tile / a->group, ntiles,
                           static_cast<const VT *>(dy) + n * ldv, (int)a->rows, (int)a->cols, (long long)ldv, scale,
                           static_cast<OT *>(out) + n * ldo, (long long)ldo);
        if (hipError_t e = hipGetLastError()) return e;
    }
    return hipSuccess;
}

}  // namespace

hipError_t launch_int4_transposed(const rsr_handle_s *a, const rsr_handle_s *b, const void *dy, int v_dtype, float scale,
                                  void *out, int out_dtype, int batch, int64_t ldv, int64_t ldo, hipStream_t stream) {
    if (v_dtype == RSR_BF16)
        return out_dtype == RSR_BF16 ? launch<uint16_t, uint16_t>(a, b, dy, scale, out, batch, ldv, ldo, stream)
                                     : launch<uint16_t, float>(a, b, dy, scale, out, batch, ldv, ldo, stream);
    return out_dtype == RSR_BF16 ? launch<float, uint16_t>(a, b, dy, scale, out, batch, ldv, ldo, stream)
                                 : launch<float, float>(a, b, dy, scale, out, batch, ldv, ldo, stream);
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
