// Rows and matrices to 8-bit codes (codes8.h): a scale for every 128 columns of a row, or for every 128 x 128 values of a matrix, whose
// codes are also written transposed for the product of the way back.
//
// What bounds both is memory: everything is read once, into registers.  Measured: 300,000 x 64 fp32 rows 17.8 us (5.4 TB/s); 16 x 1024 x 512 fp32
// matrices, both orders, 10.8 (512 workgroups of 128 x 128 values, 4.7 TB/s).
#include "codes8.h"
#include "row_vectors.h"

namespace {

constexpr int QT_THREADS = 256, QT_AHEAD = 4;   // blocks of a row under way in a thread

// `lanes` lanes for a block of a row, a vector each; what bounds it is memory.
template <class T, bool EVEN>
__global__ void __launch_bounds__(QT_THREADS) qt_rows_kernel(const T* x, long x_stride, long n, int cols, int lanes, uint8_t* q, long q_stride, uint8_t* scale) {
  typedef Rv<T, EVEN> R;
  constexpr int V = R::V, BL = C8_BLOCK / V;
  const int blocks = (cols + C8_BLOCK - 1) / C8_BLOCK, vecs = (cols + V - 1) / V, lane = threadIdx.x & (lanes - 1), groups = QT_THREADS / lanes;
  const long items = n * blocks, item0 = ((long)blockIdx.y * gridDim.x + blockIdx.x) * groups * QT_AHEAD + threadIdx.x / lanes;
  typename R::vec x_in[QT_AHEAD];
  long row[QT_AHEAD];
  int j[QT_AHEAD];
#pragma unroll
  for (int u = 0; u < QT_AHEAD; ++u) {
    const long item = min(item0 + u * groups, items - 1);
    row[u] = blocks == 1 ? item : item <= 0xffffffffl ? (long)((unsigned)item / (unsigned)blocks) : item / blocks;
    j[u] = (int)(item - row[u] * blocks) * BL + lane;
    x_in[u] = R::load_any(x + row[u] * x_stride, j[u], cols);
  }
#pragma unroll
  for (int u = 0; u < QT_AHEAD; ++u) {
    float v[V];
#pragma unroll
    for (int i = 0; i < V; ++i) v[i] = (float)x_in[u][i];
    const int byte = c8_to_scale(v, lanes);
    if (item0 + u * groups >= items) continue;
    uint8_t* to = q + row[u] * q_stride;
    if (j[u] < vecs) c8_store(to + j[u] * V, v);
    if (lane == 0) scale[row[u] * blocks + j[u] / BL] = (uint8_t)byte;
    if (j[u] == vecs - 1) {
      const float none[V] = {};
      for (int c = vecs * V; c < ((cols + 15) & ~15); c += V) c8_store(to + c, none);
    }
  }
}

struct QtMatrices {
  long rows, cols, qs, ts;             // row strides of q and qt
  uint8_t *q, *scale, *qt, *scale_t;   // qt, scale_t: both or neither
};

// A workgroup for 128 x 128 values: all in registers, read once; transposed codes through LDS, four by four in a thread.
constexpr int QT_WORDS = C8_BLOCK / 4;
template <class T, bool EVEN>
__global__ void __launch_bounds__(QT_THREADS) qt_matrix_kernel(QtMatrices p, const T* W) {
  typedef Rv<T, EVEN> R;
  constexpr int V = R::V, LANES = C8_BLOCK / V, STEP = QT_THREADS / LANES, EACH = C8_BLOCK / STEP;      // of a row; rows at a time; turns
  __shared__ unsigned code[C8_BLOCK][QT_WORDS + 1];
  __shared__ unsigned most[QT_THREADS / 64];
  const int tid = threadIdx.x, lane = tid & 63, j = tid % LANES, r = tid / LANES;
  const long nr = (p.rows + C8_BLOCK - 1) / C8_BLOCK, nc = (p.cols + C8_BLOCK - 1) / C8_BLOCK;
  const long b = blockIdx.x / (nr * nc), at = blockIdx.x % (nr * nc), r0 = at / nc * C8_BLOCK, c0 = at % nc * C8_BLOCK;
  const int rows = (int)min((long)C8_BLOCK, p.rows - r0), cols = (int)min((long)C8_BLOCK, p.cols - c0);
  typename R::vec in[EACH];
#pragma unroll
  for (int i = 0; i < EACH; ++i) in[i] = R::load_any(W + (b * p.rows + r0 + min(r + i * STEP, rows - 1)) * p.cols + c0, j, cols);
  const bool whole = j * V < cols;          // (EVEN has the last vector again behind the end; it adds nothing to the largest magnitude)
  unsigned m = 0;
#pragma unroll
  for (int i = 0; i < EACH; ++i)
#pragma unroll
    for (int k = 0; k < V; ++k) m = max(m, c8_magnitude((float)in[i][k]));
  m = c8_wave_max(m, 64);
  if (lane == 0) most[tid >> 6] = m;
  __syncthreads();
#pragma unroll
  for (int w = 0; w < QT_THREADS / 64; ++w) m = max(m, most[w]);
  const int byte = c8_scale_byte(m);
  const float inverse = c8_inverse(byte);
  const int col_pad = (cols + 15) & ~15, row_pad = (rows + 15) & ~15;
#pragma unroll
  for (int i = 0; i < EACH; ++i) {
    const int row = r + i * STEP;
    float v[V];
#pragma unroll
    for (int k = 0; k < V; ++k) v[k] = whole && row < rows ? c8_scaled((float)in[i][k], inverse) : 0.0f;
    if (row < rows && j * V < col_pad) c8_store(p.q + (b * p.rows + r0 + row) * p.qs + c0 + j * V, v);
#pragma unroll
    for (int k = 0; k < V; k += 4) code[row][(j * V + k) / 4] = c8_four(v[k], v[k + 1], v[k + 2], v[k + 3]);
  }
  if (tid == 0) {
    p.scale[(b * nr + r0 / C8_BLOCK) * nc + c0 / C8_BLOCK] = (uint8_t)byte;
    if (p.qt) p.scale_t[(b * nc + c0 / C8_BLOCK) * nr + r0 / C8_BLOCK] = (uint8_t)byte;
  }
  if (!p.qt) return;
  __syncthreads();
#pragma unroll
  for (int i = 0; i < QT_WORDS * QT_WORDS / QT_THREADS; ++i) {
    const int four_rows = tid % QT_WORDS, four_cols = tid / QT_WORDS + i * (QT_THREADS / QT_WORDS);
    unsigned a[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) a[k] = code[4 * four_rows + k][four_cols];
    // bytes 0 and 1, or 2 and 3, of two words, then of pairs of those
    const unsigned x0 = __builtin_amdgcn_perm(a[1], a[0], 0x05010400u), x1 = __builtin_amdgcn_perm(a[3], a[2], 0x05010400u);
    const unsigned x2 = __builtin_amdgcn_perm(a[1], a[0], 0x07030602u), x3 = __builtin_amdgcn_perm(a[3], a[2], 0x07030602u);
    const unsigned t[4] = {__builtin_amdgcn_perm(x1, x0, 0x05040100u), __builtin_amdgcn_perm(x1, x0, 0x07060302u), __builtin_amdgcn_perm(x3, x2, 0x05040100u),
                           __builtin_amdgcn_perm(x3, x2, 0x07060302u)};
    if (4 * four_rows >= row_pad) continue;
#pragma unroll
    for (int k = 0; k < 4; ++k)
      if (4 * four_cols + k < cols) *(unsigned*)(p.qt + (b * p.cols + c0 + 4 * four_cols + k) * p.ts + r0 + 4 * four_rows) = t[k];
  }
}

template <class T>
int qt_rows(egnn_ctx* ctx, const void* x, int64_t x_stride, int64_t n, int32_t cols, void* q, int64_t q_stride, void* scale, hipStream_t st) {
  constexpr int V = RvWidth<T>::V;
  int lanes = 1;
  while (lanes * V < cols && lanes * V < C8_BLOCK) lanes *= 2;
  const long each = (long)QT_THREADS / lanes * QT_AHEAD, grid = (n * c8_blocks(cols) + each - 1) / each;
  // (folded where more than 2^32 threads would go along one axis)
  const dim3 blocks = grid < 1l << 23 ? dim3((unsigned)grid) : dim3(1u << 23, (unsigned)((grid + (1l << 23) - 1) >> 23));
  const bool even = cols % V == 0 && rv_aligned({x}, {x_stride * (int64_t)sizeof(T)});
#define QT_CALL(E) hipLaunchKernelGGL((qt_rows_kernel<T, E>), blocks, dim3(QT_THREADS), 0, st, (const T*)x, (long)x_stride, (long)n, cols, lanes, \
                                      (uint8_t*)q, (long)q_stride, (uint8_t*)scale)
  if (even) QT_CALL(true); else QT_CALL(false);
#undef QT_CALL
  EGNN_LAUNCH_CHECK(ctx, "quantise_rows");
  return EGNN_OK;
}

template <class T>
int qt_matrices(egnn_ctx* ctx, const QtMatrices& p, const void* W, int64_t blocks, hipStream_t st) {
  if (p.cols % RvWidth<T>::V == 0 && rv_aligned({W}, {}))
    hipLaunchKernelGGL((qt_matrix_kernel<T, true>), dim3((unsigned)blocks), dim3(QT_THREADS), 0, st, p, (const T*)W);
  else
    hipLaunchKernelGGL((qt_matrix_kernel<T, false>), dim3((unsigned)blocks), dim3(QT_THREADS), 0, st, p, (const T*)W);
  EGNN_LAUNCH_CHECK(ctx, "quantise_matrices");
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
  if (blocks * QT_THREADS > 0xffffffffl) return egnn_fail(ctx, EGNN_EINVAL, "quantise_matrices: more than 2^24 blocks");
  if (batch > 0 && !qt != !scale_t) return egnn_fail(ctx, EGNN_EINVAL, "quantise_matrices: codes and scales go together");
  if (batch > 0 && (!W || !q || !scale)) return egnn_fail(ctx, EGNN_EINVAL, "quantise_matrices: null pointer");
  if (q_stride < cols || q_stride % 16 || (uintptr_t)q % 16 || (qt && (qt_stride < rows || qt_stride % 16 || (uintptr_t)qt % 16)))
    return egnn_fail(ctx, EGNN_EINVAL, "quantise_matrices: rows of codes begin at multiples of 16 bytes");
  if (batch == 0) return EGNN_OK;
  const QtMatrices p{rows, cols, q_stride, qt_stride, (uint8_t*)q, (uint8_t*)scale, (uint8_t*)qt, (uint8_t*)scale_t};
  hipStream_t st = (hipStream_t)stream;
  if (dtype == EGNN_F32) return qt_matrices<float>(ctx, p, W, blocks, st);
  if (dtype == EGNN_F16) return qt_matrices<_Float16>(ctx, p, W, blocks, st);
  return qt_matrices<__bf16>(ctx, p, W, blocks, st);
}
