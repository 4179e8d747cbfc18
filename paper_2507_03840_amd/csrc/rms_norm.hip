// Root-mean-square norm by degree with the residual's addition, output also in 8 bits, and its adjoint.
//
// A row holds (lmax + 1)^2 planes of C channels, 2 l + 1 of them of degree l (lmax = 0: a plain row of C values).  For each row and degree,
// over its L = (2 l + 1) C values:
//   h = x + r rounded to the type,  rho = 1 / sqrt(sum h^2 / L + eps),  y = h rho gamma_{l,c}.
// No mean is subtracted and gamma is the same for all m of a degree, so the norm commutes with rotations.  y is that of the stored, rounded sum:
// the adjoint, which reads h, is then the adjoint of what was computed.  With d = gamma dy:
//   dx = dh + rho (d - h rho^2 sum(d h) / L),  dgamma_{l,c} = sum over rows and m of dy h rho.
// Sums over a row are fp64: squares of any fp32 value stay finite, and the two terms of dx, which cancel in short rows (for one value all but
// eps rho^2 of them), are subtracted in fp64 from a rho that is made again from h.
#include "codes8.h"

namespace {

struct RnShape {
  long n;               // rows
  int C, lmax;
  float eps;
};

template <class T>
struct RnForward {
  const T *x, *r;       // r may be NULL
  T *h, *y;             // either may be NULL
  uint8_t *q, *scale;   // both or neither
  long xs, rs, hs, ys, qs;
  const float* gamma;
};

constexpr int RN_WAVES = 4;   // a wave for each (row, degree), so many to a workgroup

template <class T>
__device__ __forceinline__ float rn_sum(const RnForward<T>& a, long row, int at) {
  float v = (float)a.x[row * a.xs + at];
  if (a.r) v = (float)(T)(v + (float)a.r[row * a.rs + at]);
  return v;
}

// One wave for a row and degree, of any sizes.  Both passes give a value to the same lane: where h overwrites x, the second pass
// reads what the lane itself has written.
template <class T>
__global__ void __launch_bounds__(RN_WAVES * 64) rn_any_kernel(RnShape p, RnForward<T> a) {
  const int lane = threadIdx.x & 63, degrees = p.lmax + 1;
  const long item = (long)blockIdx.x * RN_WAVES + (threadIdx.x >> 6);
  if (item >= p.n * degrees) return;
  const long row = item / degrees;
  const int l = (int)(item % degrees), first = l * l, last = (l + 1) * (l + 1), dim = degrees * degrees, C = p.C;
  const int blocks = (C + C8_BLOCK - 1) / C8_BLOCK;
  double sum = 0.0;
  for (int plane = first; plane < last; ++plane)
    for (int c = lane; c < C; c += 64) {
      const float v = rn_sum(a, row, plane * C + c);
      if (a.h) a.h[row * a.hs + plane * C + c] = (T)v;
      sum += (double)v * (double)v;
    }
  const double rho = 1.0 / sqrt(c8_wave_sum(sum, 64) / ((double)(last - first) * C) + (double)p.eps);
  for (int plane = first; plane < last; ++plane)
    for (int b = 0; b < blocks; ++b) {
      float v[2] = {0.0f, 0.0f};
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        const int c = b * C8_BLOCK + k * 64 + lane;
        if (c >= C) continue;
        const float h = a.h ? (float)a.h[row * a.hs + plane * C + c] : rn_sum(a, row, plane * C + c);
        v[k] = (float)((double)h * rho) * a.gamma[l * C + c];
        if (a.y) a.y[row * a.ys + plane * C + c] = (T)v[k];
      }
      if (a.q) {
        const long out = row * dim + plane;
        c8_store_block(v[0], v[1], b * C8_BLOCK, C, lane, a.q + out * a.qs, a.scale + out * blocks + b);
      }
    }
}

template <class T>
struct RnAdjoint {
  const T *h, *dy, *dh;   // dh may be NULL
  T* dx;
  float* part;            // [chunks][lmax + 1][C]
  long hs, dys, dhs, dxs, rows;   // rows of a chunk
  const float* gamma;
};

// A workgroup for a chunk of rows and a degree: its waves take the rows in turn.  The gradient of gamma is added in LDS a row after the other by
// the wave whose turn it is.
template <class T>
__global__ void __launch_bounds__(RN_WAVES * 64) rn_any_adjoint_kernel(RnShape p, RnAdjoint<T> a) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, degrees = p.lmax + 1, l = blockIdx.y, C = p.C;
  const int first = l * l, last = (l + 1) * (l + 1);
  const long begin = (long)blockIdx.x * a.rows, end = min(begin + a.rows, p.n);
  for (long r0 = begin; r0 < end; r0 += RN_WAVES) {
    const long row = r0 + wave;
    double sum = 0.0, along = 0.0;
    if (row < end)
      for (int plane = first; plane < last; ++plane)
        for (int c = lane; c < C; c += 64) {
          const double h = (double)(float)a.h[row * a.hs + plane * C + c];
          sum += h * h;
          along += h * (double)((float)a.dy[row * a.dys + plane * C + c] * a.gamma[l * C + c]);
        }
    const double L = (double)(last - first) * C, rho = 1.0 / sqrt(c8_wave_sum(sum, 64) / L + (double)p.eps);
    const double back = c8_wave_sum(along, 64) / L * rho * rho;
    for (int turn = 0; turn < RN_WAVES; ++turn) {
      __syncthreads();
      if (turn != wave || row >= end) continue;
      for (int c = lane; c < C; c += 64) {
        double dg = 0.0;
        for (int plane = first; plane < last; ++plane) {
          const double h = (double)(float)a.h[row * a.hs + plane * C + c];
          const float dy = (float)a.dy[row * a.dys + plane * C + c];
          dg += (double)dy * h * rho;
          double v = rho * ((double)(dy * a.gamma[l * C + c]) - h * back);
          if (a.dh) v += (double)(float)a.dh[row * a.dhs + plane * C + c];
          a.dx[row * a.dxs + plane * C + c] = (T)(float)v;
        }
        float* at = a.part + ((long)blockIdx.x * degrees + l) * C + c;
        *at = (row == begin ? 0.0f : *at) + (float)dg;
      }
    }
  }
}

__global__ void rn_join_kernel(const float* part, long chunks, long n, float* out) {
  const long i = (long)blockIdx.x * blockDim.x + threadIdx.x;
  if (i >= n) return;
  double sum = 0.0;
  for (long k = 0; k < chunks; ++k) sum += (double)part[k * n + i];
  out[i] = (float)sum;
}

struct RnSplit { long rows; int chunks; size_t bytes; };
RnSplit rn_split(int64_t n, int lmax, int C) {
  RnSplit s;
  s.rows = (n + 511) / 512;
  if (s.rows < RN_WAVES) s.rows = RN_WAVES;
  s.chunks = n ? (int)((n + s.rows - 1) / s.rows) : 1;
  s.bytes = (size_t)s.chunks * (lmax + 1) * C * sizeof(float);
  return s;
}

int rn_check(egnn_ctx* ctx, const char* who, int32_t dtype, int64_t n, int32_t lmax, int32_t C, float eps) {
  const std::string at(who);
  if (!rt_size(dtype)) return egnn_fail(ctx, EGNN_EINVAL, at + ": dtype must be EGNN_F32, EGNN_F16 or EGNN_BF16");
  if (n < 0 || n > 0x7fffffff) return egnn_fail(ctx, EGNN_EINVAL, at + ": n_rows must be in 0..2^31-1");
  if (lmax < 0 || lmax > 15) return egnn_fail(ctx, EGNN_EINVAL, at + ": lmax must be in 0..15");
  if (C < 1 || C > 65536) return egnn_fail(ctx, EGNN_EINVAL, at + ": channels must be in 1..65536");
  if (!(eps > 0.0f) || !(eps < 3.0e38f)) return egnn_fail(ctx, EGNN_EINVAL, at + ": eps must be > 0 and finite");
  return EGNN_OK;
}

template <class T>
int rn_forward(egnn_ctx* ctx, const RnShape& p, const RnForward<T>& a, hipStream_t st) {
  const long items = p.n * (p.lmax + 1);
  hipLaunchKernelGGL(rn_any_kernel<T>, dim3((unsigned)((items + RN_WAVES - 1) / RN_WAVES)), dim3(RN_WAVES * 64), 0, st, p, a);
  EGNN_LAUNCH_CHECK(ctx, "rms_norm");
  return EGNN_OK;
}

template <class T>
int rn_backward(egnn_ctx* ctx, const RnShape& p, const RnAdjoint<T>& a, const RnSplit& s, float* dgamma, hipStream_t st) {
  const long n = (long)(p.lmax + 1) * p.C;
  if (p.n) hipLaunchKernelGGL(rn_any_adjoint_kernel<T>, dim3((unsigned)s.chunks, p.lmax + 1), dim3(RN_WAVES * 64), 0, st, p, a);
  hipLaunchKernelGGL(rn_join_kernel, dim3((unsigned)((n + 255) / 256)), dim3(256), 0, st, (const float*)a.part, p.n ? (long)s.chunks : 0l, n, dgamma);
  EGNN_LAUNCH_CHECK(ctx, "rms_norm_backward");
  return EGNN_OK;
}

}  // namespace

extern "C" int egnn_rms_norm(egnn_ctx* ctx, int32_t dtype, const void* x, int64_t x_stride, const void* r, int64_t r_stride, int64_t n_rows,
                             int32_t lmax, int32_t channels, const float* gamma, float eps, void* h, int64_t h_stride, void* y,
                             int64_t y_stride, void* q, int64_t q_stride, void* scale, void* stream) {
  if (!ctx) return EGNN_EINVAL;
  if (int rc = rn_check(ctx, "rms_norm", dtype, n_rows, lmax, channels, eps)) return rc;
  const int64_t row = (int64_t)(lmax + 1) * (lmax + 1) * channels;
  if (!gamma || (n_rows > 0 && !x)) return egnn_fail(ctx, EGNN_EINVAL, "rms_norm: null pointer");
  if (n_rows > 0 && !y && !q) return egnn_fail(ctx, EGNN_EINVAL, "rms_norm: neither y nor q is asked for");
  if (n_rows > 0 && !q != !scale) return egnn_fail(ctx, EGNN_EINVAL, "rms_norm: codes and scales go together");
  if (n_rows > 0 && h && !r) return egnn_fail(ctx, EGNN_EINVAL, "rms_norm: h is the sum with a residual");
  if (n_rows > 0 && h && h == y) return egnn_fail(ctx, EGNN_EINVAL, "rms_norm: h and y are two outputs");
  if (x_stride < row || (r && r_stride < row) || (h && h_stride < row) || (y && y_stride < row))
    return egnn_fail(ctx, EGNN_EINVAL, "rms_norm: a row stride below the row's length");
  if (q && (q_stride < channels || q_stride % 16 || (uintptr_t)q % 16))
    return egnn_fail(ctx, EGNN_EINVAL, "rms_norm: rows of codes begin at multiples of 16 bytes");
  if (n_rows == 0) return EGNN_OK;
  const RnShape p{n_rows, channels, lmax, eps};
  hipStream_t st = (hipStream_t)stream;
#define RN_CALL(T) return rn_forward<T>(ctx, p, {(const T*)x, (const T*)r, (T*)h, (T*)y, (uint8_t*)q, (uint8_t*)scale, x_stride, r_stride, h_stride, y_stride, q_stride, gamma}, st)
  if (dtype == EGNN_F32) RN_CALL(float);
  if (dtype == EGNN_F16) RN_CALL(_Float16);
  RN_CALL(__bf16);
#undef RN_CALL
}

extern "C" int egnn_rms_norm_workspace_bytes(const egnn_ctx* ctx, int64_t n_rows, int32_t lmax, int32_t channels, size_t* bytes) {
  if (!ctx || !bytes || n_rows < 0 || n_rows > 0x7fffffff || lmax < 0 || lmax > 15 || channels < 1 || channels > 65536)
    return egnn_fail(const_cast<egnn_ctx*>(ctx), EGNN_EINVAL, "rms_norm_workspace_bytes: bad argument");
  *bytes = rn_split(n_rows, lmax, channels).bytes;
  return EGNN_OK;
}

extern "C" int egnn_rms_norm_backward(egnn_ctx* ctx, int32_t dtype, const void* h, int64_t h_stride, const void* dy, int64_t dy_stride,
                                      const void* dh, int64_t dh_stride, int64_t n_rows, int32_t lmax, int32_t channels, const float* gamma,
                                      float eps, void* dx, int64_t dx_stride, float* dgamma, void* ws, size_t ws_bytes, void* stream) {
  if (!ctx) return EGNN_EINVAL;
  if (int rc = rn_check(ctx, "rms_norm_backward", dtype, n_rows, lmax, channels, eps)) return rc;
  const int64_t row = (int64_t)(lmax + 1) * (lmax + 1) * channels;
  if (!gamma || !dgamma || (n_rows > 0 && (!h || !dy || !dx))) return egnn_fail(ctx, EGNN_EINVAL, "rms_norm_backward: null pointer");
  if (h_stride < row || dy_stride < row || (dh && dh_stride < row) || dx_stride < row)
    return egnn_fail(ctx, EGNN_EINVAL, "rms_norm_backward: a row stride below the row's length");
  const RnSplit s = rn_split(n_rows, lmax, channels);
  if (!ws || (uintptr_t)ws % 256 || ws_bytes < s.bytes)
    return egnn_fail(ctx, EGNN_EWS, "rms_norm_backward: workspace too small or not 256-byte aligned");
  const RnShape p{n_rows, channels, lmax, eps};
  hipStream_t st = (hipStream_t)stream;
#define RN_CALL(T) return rn_backward<T>(ctx, p, {(const T*)h, (const T*)dy, (const T*)dh, (T*)dx, (float*)ws, h_stride, dy_stride, dh_stride, dx_stride, s.rows, gamma}, s, dgamma, st)
  if (dtype == EGNN_F32) RN_CALL(float);
  if (dtype == EGNN_F16) RN_CALL(_Float16);
  RN_CALL(__bf16);
#undef RN_CALL
}
