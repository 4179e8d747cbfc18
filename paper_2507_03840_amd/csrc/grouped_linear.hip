// Rows put in groups by a key, and rows times the matrix of their group with its adjoint.
//
//   group_rows:  a stable counting sort.  Row (i, (l, m)) of atom i with key s goes to group s (lmax + 1) + l; inside a group the
//                rows ascend.  Only the keys are sorted: (l, m) runs through fixed places of an atom's rows.
//   linear:      y_r = x_r W_g^T + b_g,   dx_r = dy_r W_g,   dW_g = sum_r dy_r^T x_r,   db_g = sum_r dy_r   (r in group g).
#include "row_types.h"

namespace {

constexpr int GR_THREADS = 256, GR_WAVES = GR_THREADS / 64;
constexpr int GR_CHUNKS = 512;         // workgroups of the sort; each reads the counts of all chunks
constexpr int GR_CHUNK_KEYS = 1024;    // a chunk holds at least this many keys
constexpr int GR_MAX_GROUPS = 1024;    // counts of a workgroup lie in LDS, once per wave

__device__ __forceinline__ int gr_key(const int* key, long i, int G) { return min(max(key[i], 0), G - 1); }

__global__ __launch_bounds__(GR_THREADS) void gr_count_kernel(const int* key, long n, int G, long chunk, int* counts) {
  __shared__ int s[GR_MAX_GROUPS];
  for (int g = threadIdx.x; g < G; g += GR_THREADS) s[g] = 0;
  __syncthreads();
  const long b = (long)blockIdx.x * chunk, e = min(b + chunk, n);
  for (long i = b + threadIdx.x; i < e; i += GR_THREADS) atomicAdd(&s[gr_key(key, i, G)], 1);   // whole numbers: any order
  __syncthreads();
  for (int g = threadIdx.x; g < G; g += GR_THREADS) counts[(size_t)blockIdx.x * G + g] = s[g];
}

__global__ __launch_bounds__(GR_THREADS) void gr_place_kernel(const int* key, long n, int G, int lmax, long chunk, const int* counts,
                                                              int* ptr, int* perm) {
  __shared__ int base[GR_MAX_GROUPS], total[GR_MAX_GROUPS], first[GR_MAX_GROUPS], wave_count[GR_WAVES][GR_MAX_GROUPS];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int degrees = lmax < 0 ? 1 : lmax + 1, D = degrees * degrees;
  for (int g = tid; g < G; g += GR_THREADS) {
    int before = 0, all = 0;
    for (int c = 0; c < (int)gridDim.x; ++c) {
      const int v = counts[(size_t)c * G + g];
      before += c < (int)blockIdx.x ? v : 0;
      all += v;
    }
    base[g] = before;
    total[g] = all;
    for (int w = 0; w < GR_WAVES; ++w) wave_count[w][g] = 0;
  }
  __syncthreads();
  if (tid == 0) {
    int at = 0;
    for (int g = 0; g < G; ++g) {
      first[g] = at;
      at += total[g];
    }
  }
  __syncthreads();
  if (blockIdx.x == 0)
    for (int g = tid; g <= G; g += GR_THREADS)
      for (int l = 0; l < degrees; ++l) {
        if (g < G) ptr[g * degrees + l] = first[g] * D + total[g] * l * l;
        else if (l == 0) ptr[G * degrees] = (int)(n * D);
      }
  const long b = (long)blockIdx.x * chunk, e = min(b + chunk, n);
  for (long i0 = b; i0 < e; i0 += GR_THREADS) {
    const long i = i0 + tid;
    const bool there = i < e;
    const int g = there ? gr_key(key, i, G) : -1;
    // lanes of this wave with the same key
    unsigned long long same = __ballot(there);
    for (int bit = 0; (G - 1) >> bit; ++bit) {
      const unsigned long long set = __ballot(there && (g >> bit & 1));
      same &= (g >> bit & 1) ? set : ~set;
    }
    const int rank = __popcll(same & ((1ull << lane) - 1));
    if (there && rank == 0) wave_count[wave][g] = __popcll(same);
    __syncthreads();
    if (there) {
      int r = base[g] + rank;
      for (int w = 0; w < wave; ++w) r += wave_count[w][g];
      for (int l = 0, k = 0; l < degrees; ++l) {
        const long at = (long)first[g] * D + (long)total[g] * l * l + (long)r * (2 * l + 1);
        for (int m = 0; m < 2 * l + 1; ++m, ++k) perm[at + m] = (int)(i * D) + k;
      }
    }
    __syncthreads();
    for (int h = tid; h < G; h += GR_THREADS)
      for (int w = 0; w < GR_WAVES; ++w) {
        base[h] += wave_count[w][h];
        wave_count[w][h] = 0;
      }
    __syncthreads();
  }
}

long gr_chunk(int64_t n) {
  long c = (n + GR_CHUNKS - 1) / GR_CHUNKS;
  if (c < GR_CHUNK_KEYS) c = GR_CHUNK_KEYS;
  return (c + GR_THREADS - 1) / GR_THREADS * GR_THREADS;
}
long gr_chunks(int64_t n) { return n ? (n + gr_chunk(n) - 1) / gr_chunk(n) : 1; }

// ---- products ----------------------------------------------------------------------------------------------------------
struct GlRows {
  long n;            // rows of x and y
  int G;
  const int *ptr, *perm;
};
__device__ __forceinline__ long gl_begin(const GlRows& p, int g) { return min(max((long)p.ptr[g], 0l), p.n); }
__device__ __forceinline__ long gl_row(const GlRows& p, long at) {
  return p.perm ? min(max((long)p.perm[at], 0l), p.n - 1) : at;
}

constexpr int GL_TILE = 64, GL_K = 16;

// y rows = x rows times W_g^T (BACK: W_g) + bias; 64 rows of one group by 64 columns
template <class T, bool BACK>
__global__ __launch_bounds__(256) void gl_rows_kernel(GlRows p, const T* x, long xs, const T* W, const float* bias, int K, int N, T* y,
                                                      long ys) {
  __shared__ float sx[GL_K][GL_TILE + 4], sw[GL_K][GL_TILE + 4];
  __shared__ int s_g, s_tile;
  const int tid = threadIdx.x;
  if (tid == 0) {
    int left = blockIdx.x, g = 0;
    for (; g < p.G; ++g) {
      const int tiles = (int)((max(gl_begin(p, g + 1) - gl_begin(p, g), 0l) + GL_TILE - 1) / GL_TILE);
      if (left < tiles) break;
      left -= tiles;
    }
    s_g = g;
    s_tile = left;
  }
  __syncthreads();
  const int g = s_g;
  if (g >= p.G) return;
  const long r0 = gl_begin(p, g) + (long)s_tile * GL_TILE, r1 = min(r0 + GL_TILE, gl_begin(p, g + 1));
  const int n0 = blockIdx.y * GL_TILE;
  const T* Wg = W + (size_t)g * K * N;
  float acc[4][4] = {};
  const int ti = (tid >> 4) * 4, tj = (tid & 15) * 4;
  const long row = r0 + (tid >> 2) < r1 ? gl_row(p, r0 + (tid >> 2)) : -1;
  for (int k0 = 0; k0 < K; k0 += GL_K) {
    for (int q = 0; q < 4; ++q) {
      const int k = (tid & 3) * 4 + q, n = tid >> 2;
      sx[k][tid >> 2] = row >= 0 && k0 + k < K ? (float)x[row * xs + k0 + k] : 0.0f;
      const bool in = n0 + n < N && k0 + k < K;
      sw[k][n] = !in ? 0.0f : BACK ? (float)Wg[(size_t)(k0 + k) * N + n0 + n] : (float)Wg[(size_t)(n0 + n) * K + k0 + k];
    }
    __syncthreads();
    for (int k = 0; k < GL_K; ++k)
      for (int a = 0; a < 4; ++a)
        for (int b = 0; b < 4; ++b) acc[a][b] += sx[k][ti + a] * sw[k][tj + b];
    __syncthreads();
  }
  for (int a = 0; a < 4; ++a) {
    if (r0 + ti + a >= r1) continue;
    const long r = gl_row(p, r0 + ti + a);
    for (int b = 0; b < 4; ++b)
      if (n0 + tj + b < N) y[r * ys + n0 + tj + b] = (T)(acc[a][b] + (bias ? bias[(size_t)g * N + n0 + tj + b] : 0.0f));
  }
}

// dW_g: 64 outputs by 64 inputs, over all rows of the group; db_g by the first column of workgroups
template <class T>
__global__ __launch_bounds__(256) void gl_weights_kernel(GlRows p, const T* x, long xs, const T* dy, long dys, int K, int N, float* dW,
                                                         float* db) {
  __shared__ float sx[GL_K][GL_TILE + 4], sd[GL_K][GL_TILE + 4];
  const int tid = threadIdx.x, g = blockIdx.z;
  const long r0 = gl_begin(p, g), r1 = gl_begin(p, g + 1);
  const int k0 = blockIdx.x * GL_TILE, n0 = blockIdx.y * GL_TILE;
  float acc[4][4] = {}, sum[4] = {};
  const int ti = (tid >> 4) * 4, tj = (tid & 15) * 4;
  for (long r = r0; r < r1; r += GL_K) {
    const int k = tid >> 4;
    const long row = r + k < r1 ? gl_row(p, r + k) : -1;
    for (int q = 0; q < 4; ++q) {
      const int c = (tid & 15) * 4 + q;
      sx[k][c] = row >= 0 && k0 + c < K ? (float)x[row * xs + k0 + c] : 0.0f;
      sd[k][c] = row >= 0 && n0 + c < N ? (float)dy[row * dys + n0 + c] : 0.0f;
    }
    __syncthreads();
    for (int j = 0; j < GL_K; ++j)
      for (int a = 0; a < 4; ++a) {
        sum[a] += sd[j][ti + a];
        for (int b = 0; b < 4; ++b) acc[a][b] += sd[j][ti + a] * sx[j][tj + b];
      }
    __syncthreads();
  }
  for (int a = 0; a < 4; ++a) {
    if (n0 + ti + a >= N) continue;
    for (int b = 0; b < 4; ++b)
      if (dW && k0 + tj + b < K) dW[((size_t)g * N + n0 + ti + a) * K + k0 + tj + b] = acc[a][b];
    if (db && k0 == 0 && tj == 0) db[(size_t)g * N + n0 + ti + a] = sum[a];
  }
}

int gl_check(egnn_ctx* ctx, const char* who, int32_t dtype, int64_t n, int32_t K, int32_t N, int32_t G, const int32_t* ptr) {
  const std::string at(who);
  if (!rt_size(dtype)) return egnn_fail(ctx, EGNN_EINVAL, at + ": dtype must be EGNN_F32, EGNN_F16 or EGNN_BF16");
  if (n < 0 || n > 0x7fffffff) return egnn_fail(ctx, EGNN_EINVAL, at + ": n_rows must be in 0..2^31-1");
  if (K < 1 || K > 65536 || N < 1 || N > 65536) return egnn_fail(ctx, EGNN_EINVAL, at + ": n_in and n_out must be in 1..65536");
  if (G < 1 || G > 65535) return egnn_fail(ctx, EGNN_EINVAL, at + ": n_groups must be in 1..65535");
  if (!ptr) return egnn_fail(ctx, EGNN_EINVAL, at + ": null pointer");
  return EGNN_OK;
}

template <class T>
int gl_forward(egnn_ctx* ctx, const GlRows& p, const void* x, int64_t xs, const void* W, const float* bias, int K, int N, void* y,
               int64_t ys, hipStream_t st) {
  const dim3 grid((unsigned)((p.n + GL_TILE - 1) / GL_TILE + p.G), (N + GL_TILE - 1) / GL_TILE);
  hipLaunchKernelGGL((gl_rows_kernel<T, false>), grid, dim3(256), 0, st, p, (const T*)x, (long)xs, (const T*)W, bias, K, N, (T*)y,
                     (long)ys);
  EGNN_LAUNCH_CHECK(ctx, "grouped_linear");
  return EGNN_OK;
}

template <class T>
int gl_backward(egnn_ctx* ctx, const GlRows& p, const void* x, int64_t xs, const void* W, const void* dy, int64_t dys, int K, int N,
                void* dx, int64_t dxs, float* dW, float* db, hipStream_t st) {
  if (dx && p.n) {
    const dim3 grid((unsigned)((p.n + GL_TILE - 1) / GL_TILE + p.G), (K + GL_TILE - 1) / GL_TILE);
    hipLaunchKernelGGL((gl_rows_kernel<T, true>), grid, dim3(256), 0, st, p, (const T*)dy, (long)dys, (const T*)W, (const float*)nullptr,
                       N, K, (T*)dx, (long)dxs);
    EGNN_LAUNCH_CHECK(ctx, "grouped_linear_backward");
  }
  if (dW || db) {
    const dim3 grid((K + GL_TILE - 1) / GL_TILE, (N + GL_TILE - 1) / GL_TILE, p.G);
    hipLaunchKernelGGL((gl_weights_kernel<T>), grid, dim3(256), 0, st, p, (const T*)x, (long)xs, (const T*)dy, (long)dys, K, N, dW, db);
    EGNN_LAUNCH_CHECK(ctx, "grouped_linear_backward");
  }
  return EGNN_OK;
}

}  // namespace

extern "C" int egnn_group_rows_workspace_bytes(const egnn_ctx* ctx, int64_t n, int32_t n_groups, size_t* bytes) {
  if (!ctx || !bytes || n < 0 || n > 0x7fffffff || n_groups < 1 || n_groups > GR_MAX_GROUPS)
    return egnn_fail(const_cast<egnn_ctx*>(ctx), EGNN_EINVAL, "group_rows_workspace_bytes: bad argument");
  *bytes = (size_t)gr_chunks(n) * n_groups * sizeof(int);
  return EGNN_OK;
}

extern "C" int egnn_group_rows(egnn_ctx* ctx, const int32_t* key, int64_t n, int32_t n_groups, int32_t lmax, int32_t* ptr,
                               int32_t* perm, void* ws, size_t ws_bytes, void* stream) {
  if (!ctx) return EGNN_EINVAL;
  if (n_groups < 1 || n_groups > GR_MAX_GROUPS) return egnn_fail(ctx, EGNN_EINVAL, "group_rows: n_groups must be in 1..1024");
  if (lmax < -1 || lmax > 15) return egnn_fail(ctx, EGNN_EINVAL, "group_rows: lmax must be in -1..15");
  const int64_t rows_per_key = lmax < 0 ? 1 : (int64_t)(lmax + 1) * (lmax + 1);
  if (n < 0 || n > 0x7fffffff / rows_per_key) return egnn_fail(ctx, EGNN_EINVAL, "group_rows: the rows must be in 0..2^31-1");
  if (!ptr || (n > 0 && (!key || !perm))) return egnn_fail(ctx, EGNN_EINVAL, "group_rows: null pointer");
  size_t need = 0;
  egnn_group_rows_workspace_bytes(ctx, n, n_groups, &need);
  if (!ws || (uintptr_t)ws % 256 || ws_bytes < need)
    return egnn_fail(ctx, EGNN_EWS, "group_rows: workspace too small or not 256-byte aligned");
  hipStream_t st = (hipStream_t)stream;
  const unsigned chunks = (unsigned)gr_chunks(n);
  hipLaunchKernelGGL(gr_count_kernel, dim3(chunks), dim3(GR_THREADS), 0, st, key, (long)n, n_groups, gr_chunk(n), (int*)ws);
  hipLaunchKernelGGL(gr_place_kernel, dim3(chunks), dim3(GR_THREADS), 0, st, key, (long)n, n_groups, lmax, gr_chunk(n), (const int*)ws,
                     ptr, perm);
  EGNN_LAUNCH_CHECK(ctx, "group_rows");
  return EGNN_OK;
}

extern "C" int egnn_grouped_linear_workspace_bytes(const egnn_ctx* ctx, int64_t n_rows, int32_t n_groups, int32_t n_in, int32_t n_out,
                                                   size_t* bytes) {
  if (!ctx || !bytes || n_rows < 0 || n_rows > 0x7fffffff || n_groups < 1 || n_groups > 65535 || n_in < 1 || n_in > 65536 || n_out < 1 ||
      n_out > 65536)
    return egnn_fail(const_cast<egnn_ctx*>(ctx), EGNN_EINVAL, "grouped_linear_workspace_bytes: bad argument");
  *bytes = 256;
  return EGNN_OK;
}

extern "C" int egnn_grouped_linear(egnn_ctx* ctx, int32_t dtype, const void* x, int64_t x_stride, int64_t n_rows, int32_t n_in,
                                   int32_t n_out, const void* W, const float* bias, const int32_t* ptr, const int32_t* perm,
                                   int32_t n_groups, void* y, int64_t y_stride, void* stream) {
  if (!ctx) return EGNN_EINVAL;
  if (int rc = gl_check(ctx, "grouped_linear", dtype, n_rows, n_in, n_out, n_groups, ptr)) return rc;
  if (!W || (n_rows > 0 && (!x || !y))) return egnn_fail(ctx, EGNN_EINVAL, "grouped_linear: null pointer");
  if (x_stride < n_in || y_stride < n_out) return egnn_fail(ctx, EGNN_EINVAL, "grouped_linear: a row stride below the row's length");
  if (n_rows == 0) return EGNN_OK;
  const GlRows p{n_rows, n_groups, ptr, perm};
  hipStream_t st = (hipStream_t)stream;
  if (dtype == EGNN_F32) return gl_forward<float>(ctx, p, x, x_stride, W, bias, n_in, n_out, y, y_stride, st);
  if (dtype == EGNN_F16) return gl_forward<_Float16>(ctx, p, x, x_stride, W, bias, n_in, n_out, y, y_stride, st);
  return gl_forward<__bf16>(ctx, p, x, x_stride, W, bias, n_in, n_out, y, y_stride, st);
}

extern "C" int egnn_grouped_linear_backward(egnn_ctx* ctx, int32_t dtype, const void* x, int64_t x_stride, const void* W,
                                            const void* dy, int64_t dy_stride, int64_t n_rows, int32_t n_in, int32_t n_out,
                                            const int32_t* ptr, const int32_t* perm, int32_t n_groups, void* dx, int64_t dx_stride,
                                            float* dW, float* db, void* ws, size_t ws_bytes, void* stream) {
  if (!ctx) return EGNN_EINVAL;
  if (int rc = gl_check(ctx, "grouped_linear_backward", dtype, n_rows, n_in, n_out, n_groups, ptr)) return rc;
  if (n_rows > 0 && (!dy || (dx && !W) || (dW && !x))) return egnn_fail(ctx, EGNN_EINVAL, "grouped_linear_backward: null pointer");
  if (x_stride < n_in || dy_stride < n_out || (dx && dx_stride < n_in))
    return egnn_fail(ctx, EGNN_EINVAL, "grouped_linear_backward: a row stride below the row's length");
  size_t need = 0;
  egnn_grouped_linear_workspace_bytes(ctx, n_rows, n_groups, n_in, n_out, &need);
  if (!ws || (uintptr_t)ws % 256 || ws_bytes < need)
    return egnn_fail(ctx, EGNN_EWS, "grouped_linear_backward: workspace too small or not 256-byte aligned");
  const GlRows p{n_rows, n_groups, ptr, perm};
  hipStream_t st = (hipStream_t)stream;
  if (dtype == EGNN_F32) return gl_backward<float>(ctx, p, x, x_stride, W, dy, dy_stride, n_in, n_out, dx, dx_stride, dW, db, st);
  if (dtype == EGNN_F16) return gl_backward<_Float16>(ctx, p, x, x_stride, W, dy, dy_stride, n_in, n_out, dx, dx_stride, dW, db, st);
  return gl_backward<__bf16>(ctx, p, x, x_stride, W, dy, dy_stride, n_in, n_out, dx, dx_stride, dW, db, st);
}
