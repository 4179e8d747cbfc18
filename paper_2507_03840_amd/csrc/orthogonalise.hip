// An update orthogonalised by Newton-Schulz products, and the optimiser's step around it.
//
//   x_0 = u / (|u|_F + 1e-7),   x_{k+1} = a x_k + (b g + c g^2) x_k,   g = x_k x_k^T  (from the side with fewer rows),
// with the published coefficients of the Muon optimiser: the singular values of u go to within about 0.7 .. 1.2.
// Step: m' = beta m + g, u = g + beta m', W' = (1 - lr weight_decay) W - lr sqrt(max(1, rows / cols)) orthogonalise(u).
#include "row_types.h"

namespace {

constexpr float OU_A = 3.4445f, OU_B = -4.7750f, OU_C = 2.0315f, OU_EPS = 1e-7f;

struct OuShape {
  int batch, rows, cols, n, m;   // n = the smaller side, m = the larger one
  bool tall;                     // rows > cols: x is the transpose of the caller's matrix
};

size_t ou_align(size_t n) { return (n + 255) & ~(size_t)255; }

struct OuStep { const float *g, *m; float beta; float* m_out; };

// x_0 of one matrix, [n][m]
template <class T>
__global__ __launch_bounds__(1024) void ou_first_kernel(OuShape p, const T* u, OuStep w, float* x) {
  __shared__ double s[1024];
  const size_t size = (size_t)p.rows * p.cols, at = (size_t)blockIdx.x * size;
  double t = 0.0;
  for (size_t i = threadIdx.x; i < size; i += 1024) {
    float v;
    if (w.m) {
      const float m = w.beta * w.m[at + i] + w.g[at + i];
      v = w.g[at + i] + w.beta * m;
    } else {
      v = (float)u[at + i];
    }
    t += (double)v * v;
  }
  s[threadIdx.x] = t;
  for (int h = 512; h; h >>= 1) {
    __syncthreads();
    if ((int)threadIdx.x < h) s[threadIdx.x] += s[threadIdx.x + h];
  }
  __syncthreads();
  const float inv = (float)(1.0 / (sqrt(s[0]) + (double)OU_EPS));
  for (size_t i = threadIdx.x; i < size; i += 1024) {
    float v;
    if (w.m) {
      const float m = w.beta * w.m[at + i] + w.g[at + i];
      v = w.g[at + i] + w.beta * m;
      w.m_out[at + i] = m;
    } else {
      v = (float)u[at + i];
    }
    const int r = (int)(i / p.cols), c = (int)(i % p.cols);
    x[at + (p.tall ? (size_t)c * p.m + r : (size_t)r * p.m + c)] = v * inv;
  }
}

// C = alpha A B' + beta D per matrix, B' = B^T (NT) or B; A [I][K], C and D [I][J]
template <bool NT>
__global__ __launch_bounds__(256) void ou_product_kernel(const float* A, const float* B, const float* D, float* C, int I, int J, int K,
                                                         float alpha, float beta) {
  __shared__ float sa[16][68], sb[16][68];
  const int tid = threadIdx.x, i0 = blockIdx.y * 64, j0 = blockIdx.x * 64;
  const size_t z = blockIdx.z;
  A += z * I * K;
  B += z * K * J;
  float acc[4][4] = {};
  const int ti = (tid >> 4) * 4, tj = (tid & 15) * 4;
  for (int k0 = 0; k0 < K; k0 += 16) {
    for (int q = 0; q < 4; ++q) {
      const int k = (tid & 3) * 4 + q, r = tid >> 2;
      const bool in = k0 + k < K;
      sa[k][r] = in && i0 + r < I ? A[(size_t)(i0 + r) * K + k0 + k] : 0.0f;
      sb[k][r] = !in || j0 + r >= J ? 0.0f : NT ? B[(size_t)(j0 + r) * K + k0 + k] : B[(size_t)(k0 + k) * J + j0 + r];
    }
    __syncthreads();
    for (int k = 0; k < 16; ++k)
      for (int a = 0; a < 4; ++a)
        for (int b = 0; b < 4; ++b) acc[a][b] += sa[k][ti + a] * sb[k][tj + b];
    __syncthreads();
  }
  for (int a = 0; a < 4; ++a)
    for (int b = 0; b < 4; ++b) {
      const int i = i0 + ti + a, j = j0 + tj + b;
      if (i >= I || j >= J) continue;
      const size_t at = z * I * J + (size_t)i * J + j;
      C[at] = alpha * acc[a][b] + (D ? beta * D[at] : 0.0f);
    }
}

template <class T>
__global__ __launch_bounds__(256) void ou_last_kernel(OuShape p, const float* x, T* y, const float* W, float keep, float scale) {
  const size_t size = (size_t)p.rows * p.cols, at = (size_t)blockIdx.y * size;
  const size_t i = (size_t)blockIdx.x * 256 + threadIdx.x;
  if (i >= size) return;
  const int r = (int)(i / p.cols), c = (int)(i % p.cols);
  const float v = x[at + (p.tall ? (size_t)c * p.m + r : (size_t)r * p.m + c)];
  y[at + i] = (T)(W ? keep * W[at + i] - scale * v : v);
}

int ou_check(egnn_ctx* ctx, const char* who, int32_t batch, int32_t rows, int32_t cols, int32_t steps) {
  const std::string at(who);
  if (batch < 0 || batch > 65535 || rows < 1 || rows > 65536 || cols < 1 || cols > 65536)
    return egnn_fail(ctx, EGNN_EINVAL, at + ": batch must be in 0..65535, rows and cols in 1..65536");
  if (steps < 1 || steps > 32) return egnn_fail(ctx, EGNN_EINVAL, at + ": steps must be in 1..32");
  return EGNN_OK;
}

OuShape ou_shape(int32_t batch, int32_t rows, int32_t cols) {
  return {batch, rows, cols, rows < cols ? rows : cols, rows < cols ? cols : rows, rows > cols};
}

size_t ou_bytes(const OuShape& p) {
  return 2 * ou_align((size_t)p.batch * p.n * p.m * 4) + 2 * ou_align((size_t)p.batch * p.n * p.n * 4);
}

template <class T>
int ou_run(egnn_ctx* ctx, const OuShape& p, const void* u, const OuStep& w, int steps, void* y, const float* W, float keep, float scale,
           void* ws, hipStream_t st) {
  float* x = (float*)ws;
  float* x2 = (float*)((char*)x + ou_align((size_t)p.batch * p.n * p.m * 4));
  float* g = (float*)((char*)x2 + ou_align((size_t)p.batch * p.n * p.m * 4));
  float* q = (float*)((char*)g + ou_align((size_t)p.batch * p.n * p.n * 4));
  hipLaunchKernelGGL((ou_first_kernel<T>), dim3(p.batch), dim3(1024), 0, st, p, (const T*)u, w, x);
  const int tn = (p.n + 63) / 64, tm = (p.m + 63) / 64;
  for (int k = 0; k < steps; ++k) {
    hipLaunchKernelGGL((ou_product_kernel<true>), dim3(tn, tn, p.batch), dim3(256), 0, st, x, x, (const float*)nullptr, g, p.n, p.n, p.m,
                       1.0f, 0.0f);
    hipLaunchKernelGGL((ou_product_kernel<true>), dim3(tn, tn, p.batch), dim3(256), 0, st, g, g, (const float*)g, q, p.n, p.n, p.n, OU_C,
                       OU_B);
    hipLaunchKernelGGL((ou_product_kernel<false>), dim3(tm, tn, p.batch), dim3(256), 0, st, q, x, (const float*)x, x2, p.n, p.m, p.n,
                       1.0f, OU_A);
    float* t = x; x = x2; x2 = t;
  }
  const size_t size = (size_t)p.rows * p.cols;
  hipLaunchKernelGGL((ou_last_kernel<T>), dim3((unsigned)((size + 255) / 256), p.batch), dim3(256), 0, st, p, x, (T*)y, W, keep, scale);
  EGNN_LAUNCH_CHECK(ctx, "orthogonalise");
  return EGNN_OK;
}

}  // namespace

extern "C" int egnn_orthogonalise_workspace_bytes(const egnn_ctx* ctx, int32_t batch, int32_t rows, int32_t cols, size_t* bytes) {
  if (!ctx || !bytes) return egnn_fail(const_cast<egnn_ctx*>(ctx), EGNN_EINVAL, "orthogonalise_workspace_bytes: null pointer");
  if (int rc = ou_check(const_cast<egnn_ctx*>(ctx), "orthogonalise_workspace_bytes", batch, rows, cols, 1)) return rc;
  *bytes = ou_bytes(ou_shape(batch, rows, cols));
  return EGNN_OK;
}

extern "C" int egnn_orthogonalise(egnn_ctx* ctx, int32_t dtype, const void* g, int32_t batch, int32_t rows, int32_t cols, int32_t steps,
                                  void* y, void* ws, size_t ws_bytes, void* stream) {
  if (!ctx) return EGNN_EINVAL;
  if (!rt_size(dtype)) return egnn_fail(ctx, EGNN_EINVAL, "orthogonalise: dtype must be EGNN_F32, EGNN_F16 or EGNN_BF16");
  if (int rc = ou_check(ctx, "orthogonalise", batch, rows, cols, steps)) return rc;
  if (batch == 0) return EGNN_OK;
  if (!g || !y) return egnn_fail(ctx, EGNN_EINVAL, "orthogonalise: null pointer");
  const OuShape p = ou_shape(batch, rows, cols);
  if (!ws || (uintptr_t)ws % 256 || ws_bytes < ou_bytes(p))
    return egnn_fail(ctx, EGNN_EWS, "orthogonalise: workspace too small or not 256-byte aligned");
  const OuStep w{};
  hipStream_t st = (hipStream_t)stream;
  if (dtype == EGNN_F32) return ou_run<float>(ctx, p, g, w, steps, y, nullptr, 0.0f, 0.0f, ws, st);
  if (dtype == EGNN_F16) return ou_run<_Float16>(ctx, p, g, w, steps, y, nullptr, 0.0f, 0.0f, ws, st);
  return ou_run<__bf16>(ctx, p, g, w, steps, y, nullptr, 0.0f, 0.0f, ws, st);
}

extern "C" int egnn_muon_step(egnn_ctx* ctx, const float* W, const float* g, const float* m, int32_t batch, int32_t rows, int32_t cols,
                              float lr, float beta, float weight_decay, int32_t steps, float* W_out, float* m_out, void* ws,
                              size_t ws_bytes, void* stream) {
  if (!ctx) return EGNN_EINVAL;
  if (int rc = ou_check(ctx, "muon_step", batch, rows, cols, steps)) return rc;
  if (batch == 0) return EGNN_OK;
  if (!W || !g || !m || !W_out || !m_out) return egnn_fail(ctx, EGNN_EINVAL, "muon_step: null pointer");
  const OuShape p = ou_shape(batch, rows, cols);
  if (!ws || (uintptr_t)ws % 256 || ws_bytes < ou_bytes(p))
    return egnn_fail(ctx, EGNN_EWS, "muon_step: workspace too small or not 256-byte aligned");
  const float scale = (float)((double)lr * sqrt(rows > cols ? (double)rows / cols : 1.0));
  const float keep = (float)(1.0 - (double)lr * (double)weight_decay);
  return ou_run<float>(ctx, p, nullptr, OuStep{g, m, beta, m_out}, steps, W_out, W, keep, scale, ws, (hipStream_t)stream);
}
