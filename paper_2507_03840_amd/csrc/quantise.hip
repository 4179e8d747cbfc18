// Rows and matrices to 8-bit codes (codes8.h): a scale for every 128 columns of a row, or for every 128 x 128 values of a matrix, whose
// codes are also written transposed for the product of the way back.
#include "codes8.h"

namespace {

constexpr int QT_WAVES = 4;

// One wave for a block of 128 columns of a row
template <class T>
__global__ void __launch_bounds__(QT_WAVES * 64) qt_any_rows_kernel(const T* x, long x_stride, long n, int cols, uint8_t* q, long q_stride, uint8_t* scale) {
  const int lane = threadIdx.x & 63, blocks = (cols + C8_BLOCK - 1) / C8_BLOCK;
  const long item = (long)blockIdx.x * QT_WAVES + (threadIdx.x >> 6), row = item / blocks;
  if (row >= n) return;
  const int c0 = (int)(item % blocks) * C8_BLOCK, c = c0 + lane;
  const T* at = x + row * x_stride;
  const float v0 = c < cols ? (float)at[c] : 0.0f, v1 = c + 64 < cols ? (float)at[c + 64] : 0.0f;
  c8_store_block(v0, v1, c0, cols, lane, q + row * q_stride, scale + item);
}

struct QtMatrices {
  long rows, cols, qs, ts;      // row strides of q and qt
  uint8_t *q, *scale, *qt, *scale_t;   // qt, scale_t: both or neither
};

// A workgroup for 128 x 128 values: all in registers, codes through LDS
constexpr int QT_THREADS = 256, QT_EACH = C8_BLOCK * C8_BLOCK / QT_THREADS;
template <class T>
__global__ void __launch_bounds__(QT_THREADS) qt_matrix_kernel(QtMatrices p, const T* W) {
  __shared__ uint8_t code[C8_BLOCK][C8_BLOCK + 4];
  __shared__ unsigned most[QT_THREADS / 64];
  const int tid = threadIdx.x, lane = tid & 63;
  const long nr = (p.rows + C8_BLOCK - 1) / C8_BLOCK, nc = (p.cols + C8_BLOCK - 1) / C8_BLOCK;
  const long b = blockIdx.x / (nr * nc), at = blockIdx.x % (nr * nc), r0 = at / nc * C8_BLOCK, c0 = at % nc * C8_BLOCK;
  const int c = tid % C8_BLOCK, r = tid / C8_BLOCK;
  float v[QT_EACH];
  unsigned m = 0;
#pragma unroll
  for (int i = 0; i < QT_EACH; ++i) {
    const long row = r0 + r + 2 * i;
    v[i] = row < p.rows && c0 + c < p.cols ? (float)W[(b * p.rows + row) * p.cols + c0 + c] : 0.0f;
    m = max(m, c8_magnitude(v[i]));
  }
  m = c8_wave_max(m, 64);
  if (lane == 0) most[tid >> 6] = m;
  __syncthreads();
  for (int w = 0; w < QT_THREADS / 64; ++w) m = max(m, most[w]);
  const int byte = c8_scale_byte(m);
  const float inverse = c8_inverse(byte);
#pragma unroll
  for (int i = 0; i < QT_EACH; ++i) code[r + 2 * i][c] = (uint8_t)c8_pair(c8_scaled(v[i], inverse), 0.0f);
  __syncthreads();
  const long row_end = min(r0 + C8_BLOCK, p.rows), col_end = min(c0 + C8_BLOCK, p.cols);
  const long row_pad = min(r0 + C8_BLOCK, (p.rows + 15) / 16 * 16), col_pad = min(c0 + C8_BLOCK, (p.cols + 15) / 16 * 16);
  for (int i = tid; i < C8_BLOCK * C8_BLOCK; i += QT_THREADS) {
    const int k = i / C8_BLOCK, j = i % C8_BLOCK;
    if (r0 + k < row_end && c0 + j < col_pad) p.q[(b * p.rows + r0 + k) * p.qs + c0 + j] = code[k][j];
    if (p.qt && c0 + k < col_end && r0 + j < row_pad) p.qt[(b * p.cols + c0 + k) * p.ts + r0 + j] = code[j][k];
  }
  if (tid == 0) {
    p.scale[(b * nr + r0 / C8_BLOCK) * nc + c0 / C8_BLOCK] = (uint8_t)byte;
    if (p.qt) p.scale_t[(b * nc + c0 / C8_BLOCK) * nr + r0 / C8_BLOCK] = (uint8_t)byte;
  }
}

template <class T>
int qt_rows(egnn_ctx* ctx, const void* x, int64_t x_stride, int64_t n, int32_t cols, void* q, int64_t q_stride, void* scale, hipStream_t st) {
  const int64_t items = n * c8_blocks(cols);
  hipLaunchKernelGGL(qt_any_rows_kernel<T>, dim3((unsigned)((items + QT_WAVES - 1) / QT_WAVES)), dim3(QT_WAVES * 64), 0, st, (const T*)x, (long)x_stride,
                     (long)n, cols, (uint8_t*)q, (long)q_stride, (uint8_t*)scale);
  EGNN_LAUNCH_CHECK(ctx, "quantise_rows");
  return EGNN_OK;
}

}  // namespace

extern "C" int egnn_quantise_rows(egnn_ctx* ctx, int32_t dtype, const void* x, int64_t x_stride, int64_t n_rows, int32_t n_cols, void* q,
                                  int64_t q_stride, void* scale, void* stream) {
  if (!ctx) return EGNN_EINVAL;
  if (!rt_size(dtype)) return egnn_fail(ctx, EGNN_EINVAL, "quantise_rows: dtype must be EGNN_F32, EGNN_F16 or EGNN_BF16");
  if (n_rows < 0 || n_rows > 0x7fffffff) return egnn_fail(ctx, EGNN_EINVAL, "quantise_rows: n_rows must be in 0..2^31-1");
  if (n_cols < 1 || n_cols > 65536) return egnn_fail(ctx, EGNN_EINVAL, "quantise_rows: n_cols must be in 1..65536");
  if (n_rows > 0 && (!x || !q || !scale)) return egnn_fail(ctx, EGNN_EINVAL, "quantise_rows: null pointer");
  if (x_stride < n_cols) return egnn_fail(ctx, EGNN_EINVAL, "quantise_rows: a row stride below the row's length");
  if (q_stride < n_cols || q_stride % 16 || (uintptr_t)q % 16)
    return egnn_fail(ctx, EGNN_EINVAL, "quantise_rows: rows of codes begin at multiples of 16 bytes");
  if (n_rows == 0) return EGNN_OK;
  hipStream_t st = (hipStream_t)stream;
  if (dtype == EGNN_F32) return qt_rows<float>(ctx, x, x_stride, n_rows, n_cols, q, q_stride, scale, st);
  if (dtype == EGNN_F16) return qt_rows<_Float16>(ctx, x, x_stride, n_rows, n_cols, q, q_stride, scale, st);
  return qt_rows<__bf16>(ctx, x, x_stride, n_rows, n_cols, q, q_stride, scale, st);
}

extern "C" int egnn_quantise_matrices(egnn_ctx* ctx, int32_t dtype, const void* W, int32_t batch, int32_t rows, int32_t cols, void* q,
                                      int64_t q_stride, void* scale, void* qt, int64_t qt_stride, void* scale_t, void* stream) {
  if (!ctx) return EGNN_EINVAL;
  if (!rt_size(dtype)) return egnn_fail(ctx, EGNN_EINVAL, "quantise_matrices: dtype must be EGNN_F32, EGNN_F16 or EGNN_BF16");
  if (batch < 0 || batch > 65535) return egnn_fail(ctx, EGNN_EINVAL, "quantise_matrices: batch must be in 0..65535");
  if (rows < 1 || rows > 65536 || cols < 1 || cols > 65536) return egnn_fail(ctx, EGNN_EINVAL, "quantise_matrices: rows and cols must be in 1..65536");
  const int64_t blocks = (int64_t)batch * c8_blocks(rows) * c8_blocks(cols);
  if (blocks > 0x7fffffff) return egnn_fail(ctx, EGNN_EINVAL, "quantise_matrices: more than 2^31 - 1 blocks");
  if (batch > 0 && !qt != !scale_t) return egnn_fail(ctx, EGNN_EINVAL, "quantise_matrices: codes and scales go together");
  if (batch > 0 && (!W || !q || !scale)) return egnn_fail(ctx, EGNN_EINVAL, "quantise_matrices: null pointer");
  if (q_stride < cols || q_stride % 16 || (uintptr_t)q % 16 || (qt && (qt_stride < rows || qt_stride % 16 || (uintptr_t)qt % 16)))
    return egnn_fail(ctx, EGNN_EINVAL, "quantise_matrices: rows of codes begin at multiples of 16 bytes");
  if (batch == 0) return EGNN_OK;
  const QtMatrices p{rows, cols, q_stride, qt_stride, (uint8_t*)q, (uint8_t*)scale, (uint8_t*)qt, (uint8_t*)scale_t};
  hipStream_t st = (hipStream_t)stream;
#define QT_CALL(T) hipLaunchKernelGGL(qt_matrix_kernel<T>, dim3((unsigned)blocks), dim3(QT_THREADS), 0, st, p, (const T*)W)
  if (dtype == EGNN_F32) QT_CALL(float);
  else if (dtype == EGNN_F16) QT_CALL(_Float16);
  else QT_CALL(__bf16);
#undef QT_CALL
  EGNN_LAUNCH_CHECK(ctx, "quantise_matrices");
  return EGNN_OK;
}
