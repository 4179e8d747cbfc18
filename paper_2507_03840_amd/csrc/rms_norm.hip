// Root-mean-square norm by degree with the residual's addition, output also in 8 bits, and its adjoint.
//
// A row holds (lmax + 1)^2 planes of C channels, 2 l + 1 of them of degree l (lmax = 0: a plain row of C values).  For each row and degree,
// over its L = (2 l + 1) C values:
//   h = x + r rounded to the type,  rho = 1 / sqrt(sum h^2 / L + eps),  y = h rho gamma_{l,c}.
// No mean is subtracted and gamma is the same for all m of a degree, so the norm commutes with rotations.  y is that of the stored, rounded sum:
// the adjoint, which reads h, is then the adjoint of what was computed.  With d = gamma dy:
//   dx = dh + rho (d - h rho^2 sum(d h) / L),  dgamma_{l,c} = sum over rows and m of dy h rho.
// Sums over a row are fp64: squares of any fp32 value stay finite.  The two terms of dx, which cancel in short rows (for one value all but
// eps rho^2 of them), are subtracted in fp64 in rows of up to 32 values, from a rho that is made again from h; in longer ones in fp32.
//
// What bounds it is memory: a row is read once, into registers, and written from there.  Short rows share a wave (a power of two of lanes each, four rows
// under way), long ones have a wave or a workgroup; a degree is a row of its own, with all its planes on their way together.
//
// Measured: 2,350,179 x 64 bf16 with the residual, sum and codes out, 189 us (5.6 TB/s); 20,000 x 25 x 64 fp32, sum and y out, 87 (5.9); 20,000 x 1024
// bf16 29 (5.6); 64 x 9 x 16 fp32 4.0.  The adjoint with the gradient from besides 113 (4.5 TB/s), and 37 (4.4), then 5 to join the chunks' gradients of
// gamma: reading three tensors and writing one, it stays there with 8 or 16 bytes a lane, two to five waves a SIMD, one turn or many a workgroup.
#include <algorithm>
#include "codes8.h"
#include "row_vectors.h"

namespace {

constexpr int RN_SHORT = 32;           // up to so many values the adjoint's differences are fp64
constexpr int RN_THREADS = 256, RN_WAVES = RN_THREADS / 64;

struct RnShape {
  long n;               // rows
  int C, lmax;
  float eps;
  int lanes;            // of a row, where a wave takes several
};

// 1 / sqrt(v) to fp64's last bits: the instruction's is off by up to 2^-24.2 (4e6 values each of 2^-140 to 2^250), one Newton step leaves 2^-47.8, of which
// short rows, where all but a small part of two terms cancels, would have up to three fp32 roundings.  With e = 1 - v r^2, 1 / sqrt(1 - e) = 1 + e / 2 + 3 e^2 / 8 + O(e^3).
__device__ __forceinline__ double rn_rsqrt(double v) {
  const double r = __builtin_amdgcn_rsq(v), e = fma(-(v * r), r, 1.0);
  return r > 0.0 ? fma(r * e, fma(0.375, e, 0.5), r) : r;      // (0 for an infinite v, where e is NaN; NaN stays)
}

template <class T>
struct RnForward {
  const T *x, *r;       // r may be NULL
  T *h, *y;             // either may be NULL
  uint8_t *q, *scale;   // both or neither
  long xs, rs, hs, ys, qs;
  const float* gamma;
};

// Sum over the `lanes` lanes of a row, to all of them
template <bool WIDE>
__device__ __forceinline__ double rn_row_sum(double v, int lanes, double* lds) {
  if constexpr (!WIDE) return c8_wave_sum(v, lanes);
  v = c8_wave_sum(v, 64);
  if ((threadIdx.x & 63) == 0) lds[threadIdx.x >> 6] = v;
  __syncthreads();
  v = lds[0];
#pragma unroll
  for (int w = 1; w < RN_WAVES; ++w) v += lds[w];
  return v;
}

// Number of a workgroup: a grid of more than 2^23 is folded, as no more than 2^32 threads go along one axis
__device__ __forceinline__ long rn_block() { return (long)blockIdx.y * gridDim.x + blockIdx.x; }
dim3 rn_grid(long blocks) { return blocks < 1l << 23 ? dim3((unsigned)blocks) : dim3(1u << 23, (unsigned)((blocks + (1l << 23) - 1) >> 23)); }

// Degree of a workgroup: workgroups go through the degrees of a run of rows, the longest first, before the next rows, so that short ones run beside long ones
__device__ __forceinline__ int rn_degree(const RnShape& p) { return p.lmax - (int)(rn_block() % (p.lmax + 1)); }

// U rows at a time of one degree, PL planes each, by `lanes` lanes with NV vectors of a plane each (WIDE: by the workgroup).  All of them are
// read before anything is written.
template <class T, bool EVEN, int PL, int U, int NV, bool WIDE>
__device__ __forceinline__ void rn_write(const RnShape& p, const RnForward<T>& a, int l) {
  typedef Rv<T, EVEN> R;
  constexpr int V = R::V, BL = C8_BLOCK / V;
  __shared__ double lds[RN_WAVES];
  const int lanes = WIDE ? RN_THREADS : p.lanes, lane = threadIdx.x & (lanes - 1), groups = RN_THREADS / lanes, C = p.C;
  const int dim = (p.lmax + 1) * (p.lmax + 1), vecs = (C + V - 1) / V, blocks = (C + C8_BLOCK - 1) / C8_BLOCK;
  const long row0 = rn_block() / (p.lmax + 1) * groups * U + threadIdx.x / lanes;
  typename R::vec h[U][PL][NV];
#pragma unroll
  for (int u = 0; u < U; ++u)
#pragma unroll
    for (int m = 0; m < PL; ++m)
#pragma unroll
      for (int k = 0; k < NV; ++k) h[u][m][k] = R::load(a.x + min(row0 + u * groups, p.n - 1) * a.xs + (l * l + m) * C, lane + k * lanes, C);
  if (a.r) {
    typename R::vec r[U][PL][NV];
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
      for (int m = 0; m < PL; ++m)
#pragma unroll
        for (int k = 0; k < NV; ++k) r[u][m][k] = R::load(a.r + min(row0 + u * groups, p.n - 1) * a.rs + (l * l + m) * C, lane + k * lanes, C);
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
      for (int m = 0; m < PL; ++m)
#pragma unroll
        for (int k = 0; k < NV; ++k)
#pragma unroll
          for (int i = 0; i < V; ++i) h[u][m][k][i] = (T)((float)h[u][m][k][i] + (float)r[u][m][k][i]);
  }
  float gain[NV][V];
#pragma unroll
  for (int k = 0; k < NV; ++k) R::load_floats(a.gamma + l * C, lane + k * lanes, C, gain[k]);
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const long row = row0 + u * groups;
    const bool there = row < p.n;
    double sum = 0.0;
#pragma unroll
    for (int m = 0; m < PL; ++m)
#pragma unroll
      for (int k = 0; k < NV; ++k) {
        if (a.h && there) R::store(a.h + row * a.hs + (l * l + m) * C, lane + k * lanes, C, h[u][m][k]);
        if (lane + k * lanes < vecs)
#pragma unroll
          for (int i = 0; i < V; ++i) sum += (double)(float)h[u][m][k][i] * (double)(float)h[u][m][k][i];
      }
    const double rho = rn_rsqrt(rn_row_sum<WIDE>(sum, lanes, lds) / ((double)PL * C) + (double)p.eps);
    // (a rho that fp32 holds with fewer bits: of rows of more than 2^64)
    const bool large = rho < 0x1p-64;
    const float by = (float)(large ? rho * 0x1p64 : rho), down = large ? 0x1p-64f : 1.0f;
#pragma unroll
    for (int m = 0; m < PL; ++m)
#pragma unroll
      for (int k = 0; k < NV; ++k) {
        const int j = lane + k * lanes;
        float v[V];
#pragma unroll
        for (int i = 0; i < V; ++i) v[i] = (float)h[u][m][k][i] * down * by * gain[k][i];
        if (!EVEN && !(rho >= 0.0)) {       // a NaN in the row: the zeros behind its last value stay zeros
#pragma unroll
          for (int i = 0; i < V; ++i) v[i] = j * V + i < C ? v[i] : 0.0f;
        }
        if (a.y && there) {
          typename R::vec y;
#pragma unroll
          for (int i = 0; i < V; ++i) y[i] = (T)v[i];
          R::store(a.y + row * a.ys + (l * l + m) * C, j, C, y);
        }
        if (!a.q) continue;
        const int byte = c8_to_scale(v, WIDE || lanes > BL ? BL : lanes);
        const long out = row * dim + l * l + m;
        if (!there) continue;
        if (j < vecs) c8_store(a.q + out * a.qs + j * V, v);
        if (j < vecs && j % BL == 0) a.scale[out * blocks + j / BL] = (uint8_t)byte;
        const float none[V] = {};
        if (j == 0)
          for (int c = vecs * V; c < ((C + 15) & ~15); c += V) c8_store(a.q + out * a.qs + c, none);
      }
  }
}

template <class T, bool EVEN, int NV>
__global__ void __launch_bounds__(RN_THREADS) rn_rows_kernel(RnShape p, RnForward<T> a) { rn_write<T, EVEN, 1, NV == 1 ? 4 : 1, NV, false>(p, a, 0); }
template <class T, bool EVEN, int NV>
__global__ void __launch_bounds__(RN_THREADS) rn_wide_kernel(RnShape p, RnForward<T> a) { rn_write<T, EVEN, 1, 1, NV, true>(p, a, 0); }
template <class T, bool EVEN>
__global__ void __launch_bounds__(RN_THREADS) rn_degrees_kernel(RnShape p, RnForward<T> a) {
  switch (rn_degree(p)) {
    case 0: rn_write<T, EVEN, 1, 1, 1, false>(p, a, 0); break;
    case 1: rn_write<T, EVEN, 3, 1, 1, false>(p, a, 1); break;
    case 2: rn_write<T, EVEN, 5, 1, 1, false>(p, a, 2); break;
    case 3: rn_write<T, EVEN, 7, 1, 1, false>(p, a, 3); break;
    default: rn_write<T, EVEN, 9, 1, 1, false>(p, a, 4);
  }
}

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
  const long item = rn_block() * RN_WAVES + (threadIdx.x >> 6);
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

// Chunks of rows of the adjoint, the same for every type and degree: as many workgroups as run at once (1,024, or 2,048 with degrees, whose workgroups are of
// unlike length), and no fewer than 1,024 values of a plane in each, so that the chunks' gradients of gamma are a small part of what is read (2,000 x 9 x 64
// fp32, in cache: 7.9 us, with 4,096 values 12.6; 50,000 x 64 bf16 is the same with both).
struct RnSplit { long rows; int chunks; };
RnSplit rn_split(int64_t n, int lmax, int C) {
  const long most = lmax ? 2048l / (lmax + 1) : 1024;
  RnSplit s;
  s.rows = std::max<long>(std::max<long>((n + most - 1) / most, 1024l / C), 1);
  const long whole = C >= 256 ? 4 : 16;          // rows that a workgroup takes at once, or a part of them
  if (s.rows > whole) s.rows = (s.rows + whole - 1) / whole * whole;
  s.chunks = n ? (int)((n + s.rows - 1) / s.rows) : 1;
  return s;
}

template <class T>
struct RnAdjoint {
  const T *h, *dy, *dh;   // dh may be NULL
  T* dx;
  float* part;            // [chunks][lmax + 1][C], the highest degree first; doubles where rows are added there one by one
  long hs, dys, dhs, dxs;
  const float* gamma;
};

// The rows of a chunk, in the layout of rn_write; the gradient of gamma stays in registers until the last of them.  Where a turn's rows are few registers,
// the next turn's are on their way meanwhile.
template <class T, bool EVEN, int PL, int U, int NV, bool WIDE, int V>
__device__ __forceinline__ void rn_adjoint(const RnShape& p, const RnSplit& s, const RnAdjoint<T>& a, int l, double* lds) {
  typedef Rv<T, EVEN, V> R;
  constexpr bool EARLY = PL * U * NV <= 2;
  const int lanes = WIDE ? RN_THREADS : p.lanes, lane = threadIdx.x & (lanes - 1), groups = RN_THREADS / lanes, C = p.C;
  const int vecs = (C + V - 1) / V;
  // the last rows first: what was written last, h by the forward call or dy by the call before, is the part that the caches still hold
  // (20,000 x 25 x 64 fp32, forward and back, 204 us; the first rows first 212)
  const long begin = (long)(s.chunks - 1 - blockIdx.x / (p.lmax + 1)) * s.rows, end = min(begin + s.rows, p.n);
  float gain[NV][V];
  double dg[NV][V];
#pragma unroll
  for (int k = 0; k < NV; ++k) {
    R::load_floats(a.gamma + l * C, lane + k * lanes, C, gain[k]);
#pragma unroll
    for (int i = 0; i < V; ++i) dg[k][i] = 0.0;
  }
  struct Rows { typename R::vec h[U][PL][NV], dy[U][PL][NV], dh[U][PL][NV]; };
  auto fetch = [&](long r0, Rows& o) {
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
      for (int m = 0; m < PL; ++m)
#pragma unroll
        for (int k = 0; k < NV; ++k) {
          const long row = min(r0 + u * groups, end - 1);
          o.h[u][m][k] = R::load(a.h + row * a.hs + (l * l + m) * C, lane + k * lanes, C);
          o.dy[u][m][k] = R::load(a.dy + row * a.dys + (l * l + m) * C, lane + k * lanes, C);
        }
    if (a.dh)
#pragma unroll
      for (int u = 0; u < U; ++u)
#pragma unroll
        for (int m = 0; m < PL; ++m)
#pragma unroll
          for (int k = 0; k < NV; ++k) o.dh[u][m][k] = R::load(a.dh + min(r0 + u * groups, end - 1) * a.dhs + (l * l + m) * C, lane + k * lanes, C);
  };
  Rows now, then;
  if constexpr (EARLY) fetch(begin + threadIdx.x / lanes, then);
  for (long r0 = begin + threadIdx.x / lanes, turn = begin; turn < end; r0 += groups * U, turn += groups * U) {
    if constexpr (EARLY) {
      now = then;
      fetch(r0 + groups * U, then);
    } else {
      fetch(r0, now);
    }
    auto &h = now.h, &dy = now.dy, &dh = now.dh;
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const long row = r0 + u * groups;
      const bool there = row < end;
      double sum = 0.0, along = 0.0;
#pragma unroll
      for (int m = 0; m < PL; ++m)
#pragma unroll
        for (int k = 0; k < NV; ++k)
          if (lane + k * lanes < vecs)
#pragma unroll
            for (int i = 0; i < V; ++i) {
              const double v = (double)(float)h[u][m][k][i];
              sum += v * v;
              along += v * (double)((float)dy[u][m][k][i] * gain[k][i]);
            }
      sum = rn_row_sum<WIDE>(sum, lanes, lds);
      if constexpr (WIDE) __syncthreads();
      along = rn_row_sum<WIDE>(along, lanes, lds);
      if constexpr (WIDE) __syncthreads();
      const double rho = rn_rsqrt(sum / ((double)PL * C) + (double)p.eps);
      along = along / ((double)PL * C) * rho;
      if (!there) continue;
      if (PL * C <= RN_SHORT) {
#pragma unroll
        for (int k = 0; k < NV; ++k)
#pragma unroll
          for (int m = 0; m < PL; ++m) {
            typename R::vec dx;
#pragma unroll
            for (int i = 0; i < V; ++i) {
              const double hat = (double)(float)h[u][m][k][i] * rho;
              const float d = (float)dy[u][m][k][i];
              dg[k][i] += (double)d * hat;
              double g = rho * ((double)(d * gain[k][i]) - hat * along);
              if (a.dh) g += (double)(float)dh[u][m][k][i];
              dx[i] = (T)(float)g;
            }
            R::store(a.dx + row * a.dxs + (l * l + m) * C, lane + k * lanes, C, dx);
          }
        continue;
      }
      // (as in rn_write: of rows of more than 2^64 rho is held times 2^64)
      const bool large = rho < 0x1p-64;
      const float by = (float)(large ? rho * 0x1p64 : rho), down = large ? 0x1p-64f : 1.0f, back = (float)along;
#pragma unroll
      for (int k = 0; k < NV; ++k) {
        float terms[V] = {};
#pragma unroll
        for (int m = 0; m < PL; ++m) {
          typename R::vec dx;
#pragma unroll
          for (int i = 0; i < V; ++i) {
            const float hat = (float)h[u][m][k][i] * down * by, d = (float)dy[u][m][k][i];
            terms[i] = fmaf(d, hat, terms[i]);
            float g = fmaf(-hat, back, d * gain[k][i]) * by * down;
            if (a.dh) g += (float)dh[u][m][k][i];
            dx[i] = (T)g;
          }
          R::store(a.dx + row * a.dxs + (l * l + m) * C, lane + k * lanes, C, dx);
        }
#pragma unroll
        for (int i = 0; i < V; ++i) dg[k][i] += (double)terms[i];
      }
    }
  }
  float* out = a.part + (long)blockIdx.x * C;
  if constexpr (WIDE) {
#pragma unroll
    for (int k = 0; k < NV; ++k)
#pragma unroll
      for (int i = 0; i < V; ++i)
        if ((lane + k * lanes) * V + i < C) out[(lane + k * lanes) * V + i] = (float)dg[k][i];
  } else {
    const int width = vecs * V;
#pragma unroll
    for (int k = 0; k < NV; ++k)
#pragma unroll
      for (int i = 0; i < V; ++i) {
        for (int at = lanes; at < 64; at <<= 1) dg[k][i] += __shfl_xor(dg[k][i], at);
        if ((threadIdx.x & 63) < lanes && lane + k * lanes < vecs) lds[(threadIdx.x >> 6) * width + (lane + k * lanes) * V + i] = dg[k][i];
      }
    __syncthreads();
    for (int c = threadIdx.x; c < C; c += RN_THREADS) {
      double sum = lds[c];
#pragma unroll
      for (int w = 1; w < RN_WAVES; ++w) sum += lds[w * width + c];
      out[c] = (float)sum;
    }
  }
}

template <class T, bool EVEN, int NV>
__global__ void __launch_bounds__(RN_THREADS) rn_rows_adjoint_kernel(RnShape p, RnSplit s, RnAdjoint<T> a) {
  extern __shared__ double rn_lds[];
  rn_adjoint<T, EVEN, 1, NV == 1 ? 2 : 1, NV, false, RvWidth<T>::V>(p, s, a, 0, rn_lds);
}
template <class T, bool EVEN, int NV>
__global__ void __launch_bounds__(RN_THREADS) rn_wide_adjoint_kernel(RnShape p, RnSplit s, RnAdjoint<T> a) {
  extern __shared__ double rn_lds[];
  rn_adjoint<T, EVEN, 1, 1, NV, true, RvWidth<T>::V>(p, s, a, 0, rn_lds);
}
template <class T, bool EVEN, int V>
__global__ void __launch_bounds__(RN_THREADS) rn_degrees_adjoint_kernel(RnShape p, RnSplit s, RnAdjoint<T> a) {
  extern __shared__ double rn_lds[];
  switch (rn_degree(p)) {
    case 0: rn_adjoint<T, EVEN, 1, 1, 1, false, V>(p, s, a, 0, rn_lds); break;
    case 1: rn_adjoint<T, EVEN, 3, 1, 1, false, V>(p, s, a, 1, rn_lds); break;
    case 2: rn_adjoint<T, EVEN, 5, 1, 1, false, V>(p, s, a, 2, rn_lds); break;
    case 3: rn_adjoint<T, EVEN, 7, 1, 1, false, V>(p, s, a, 3, rn_lds); break;
    default: rn_adjoint<T, EVEN, 9, 1, 1, false, V>(p, s, a, 4, rn_lds);
  }
}

// A workgroup for a chunk of rows and a degree, of any sizes: its waves take the rows in turn.  The gradient of gamma is added a row after the other by
// the wave whose turn it is.
template <class T>
__global__ void __launch_bounds__(RN_WAVES * 64) rn_any_adjoint_kernel(RnShape p, RnSplit s, RnAdjoint<T> a) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, l = rn_degree(p), C = p.C;
  const int first = l * l, last = (l + 1) * (l + 1);
  const long begin = (long)(blockIdx.x / (p.lmax + 1)) * s.rows, end = min(begin + s.rows, p.n);
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
        double* at = (double*)a.part + (long)blockIdx.x * C + c;
        *at = (row == begin ? 0.0 : *at) + dg;
      }
    }
  }
}

// Adds the chunks' gradients of gamma: 16 channels of a degree a workgroup, each by 32 threads that take the chunks in turn, four of them under way
constexpr int RN_JOIN = 512, RN_JOIN_TURNS = RN_JOIN / 16;
template <class P>
__global__ void __launch_bounds__(RN_JOIN) rn_join_kernel(RnShape p, RnSplit s, const P* part, float* dgamma) {
  __shared__ double lds[RN_JOIN_TURNS][17];
  const int l = blockIdx.y, c = min((int)blockIdx.x * 16 + (int)(threadIdx.x & 15), p.C - 1), turn = threadIdx.x >> 4;
  const int end = p.n ? s.chunks : 0;
  double sum = 0.0;
  for (int k = turn; k < end; k += 4 * RN_JOIN_TURNS) {
    P v[4];
#pragma unroll
    for (int u = 0; u < 4; ++u) v[u] = part[((long)min(k + u * RN_JOIN_TURNS, end - 1) * (p.lmax + 1) + p.lmax - l) * p.C + c];
#pragma unroll
    for (int u = 0; u < 4; ++u)
      if (k + u * RN_JOIN_TURNS < end) sum += (double)v[u];
  }
  lds[turn][threadIdx.x & 15] = sum;
  __syncthreads();
  if (threadIdx.x >= 16 || (int)(blockIdx.x * 16 + threadIdx.x) >= p.C) return;
  for (int k = 1; k < RN_JOIN_TURNS; ++k) sum += lds[k][threadIdx.x];
  dgamma[l * p.C + c] = (float)sum;
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

// Lanes of a row: the least power of two with a vector of a plane each, or a wave
int rn_lanes(int vecs) {
  int lanes = 1;
  while (lanes < vecs && lanes < 64) lanes *= 2;
  return lanes;
}

template <class T, bool EVEN>
bool rn_forward_vectors(const RnShape& p, const RnForward<T>& a, int vecs, hipStream_t st) {
  auto rows = [&](int groups) { return rn_grid((p.n + groups - 1) / groups * (p.lmax + 1)); };
  const dim3 block(RN_THREADS);
  const int groups = RN_THREADS / p.lanes;
  if (p.C < RvWidth<T>::V) return false;
  if (p.lmax) {
    if (p.lmax > 4 || vecs > 64) return false;
    hipLaunchKernelGGL((rn_degrees_kernel<T, EVEN>), rows(groups), block, 0, st, p, a);
  } else if (vecs <= 64) {
    hipLaunchKernelGGL((rn_rows_kernel<T, EVEN, 1>), rows(groups * 4), block, 0, st, p, a);
  // a wave up to 256 vectors, a workgroup above (20,000 rows bf16 with codes, wave : workgroup, 128 vectors 28 : 46 us, 256 56 : 59, 512 114 : 102;
  // 64 to 2,048 rows of 128 or 256 within 5 %)
  } else if (vecs <= 128) {
    hipLaunchKernelGGL((rn_rows_kernel<T, EVEN, 2>), rows(groups), block, 0, st, p, a);
  } else if (vecs <= 256) {
    hipLaunchKernelGGL((rn_rows_kernel<T, EVEN, 4>), rows(groups), block, 0, st, p, a);
  } else if (vecs <= 2 * RN_THREADS) {
    hipLaunchKernelGGL((rn_wide_kernel<T, EVEN, 2>), rows(1), block, 0, st, p, a);
  } else if (vecs <= 4 * RN_THREADS) {
    hipLaunchKernelGGL((rn_wide_kernel<T, EVEN, 4>), rows(1), block, 0, st, p, a);
  } else if (vecs <= 8 * RN_THREADS) {
    hipLaunchKernelGGL((rn_wide_kernel<T, EVEN, 8>), rows(1), block, 0, st, p, a);
  } else {
    return false;
  }
  return true;
}

template <class T>
int rn_forward(egnn_ctx* ctx, RnShape p, const RnForward<T>& a, hipStream_t st) {
  const int vecs = (p.C + RvWidth<T>::V - 1) / RvWidth<T>::V, size = sizeof(T);
  p.lanes = rn_lanes(vecs);
  const bool even = p.C % RvWidth<T>::V == 0 && rv_aligned({a.x, a.r, a.h, a.y, a.gamma}, {a.xs * size, a.r ? a.rs * size : 0, a.h ? a.hs * size : 0, a.y ? a.ys * size : 0});
  if (!(even ? rn_forward_vectors<T, true>(p, a, vecs, st) : rn_forward_vectors<T, false>(p, a, vecs, st))) {
    const long items = p.n * (p.lmax + 1);
    hipLaunchKernelGGL(rn_any_kernel<T>, rn_grid((items + RN_WAVES - 1) / RN_WAVES), dim3(RN_THREADS), 0, st, p, a);
  }
  EGNN_LAUNCH_CHECK(ctx, "rms_norm");
  return EGNN_OK;
}

template <class T, bool EVEN>
bool rn_backward_vectors(const RnShape& p, const RnSplit& s, const RnAdjoint<T>& a, int vecs, hipStream_t st) {
  constexpr int V = RvWidth<T>::V;
  const dim3 grid(s.chunks * (p.lmax + 1)), block(RN_THREADS);
  const size_t lds = (size_t)RN_WAVES * vecs * V * sizeof(double);
  if (p.C < V) return false;
  if (p.lmax) {
    if (p.lmax > 4 || vecs > 64) return false;
    // 16-bit values in vectors of 8 bytes, as long as a wave has lanes for them: half the registers (20,000 x 25 x 64 bf16 67 us, with 16 bytes 76; fp32
    // 119 and 113)
    if (V == 8 && p.C <= 256) {
      RnShape half = p;
      half.lanes = rn_lanes((p.C + 3) / 4);
      hipLaunchKernelGGL((rn_degrees_adjoint_kernel<T, EVEN, 4>), grid, block, lds, st, half, s, a);
    } else {
      hipLaunchKernelGGL((rn_degrees_adjoint_kernel<T, EVEN, V>), grid, block, lds, st, p, s, a);
    }
  } else if (vecs <= 64) {
    hipLaunchKernelGGL((rn_rows_adjoint_kernel<T, EVEN, 1>), grid, block, lds, st, p, s, a);
  } else if (vecs <= 128) {
    hipLaunchKernelGGL((rn_rows_adjoint_kernel<T, EVEN, 2>), grid, block, lds, st, p, s, a);
  } else if (vecs <= 2 * RN_THREADS) {
    hipLaunchKernelGGL((rn_wide_adjoint_kernel<T, EVEN, 2>), grid, block, RN_WAVES * sizeof(double), st, p, s, a);
  } else if (vecs <= 4 * RN_THREADS) {
    hipLaunchKernelGGL((rn_wide_adjoint_kernel<T, EVEN, 4>), grid, block, RN_WAVES * sizeof(double), st, p, s, a);
  } else if (V == 4 && vecs <= 8 * RN_THREADS) {
    if constexpr (V == 4) hipLaunchKernelGGL((rn_wide_adjoint_kernel<T, EVEN, 8>), grid, block, RN_WAVES * sizeof(double), st, p, s, a);
  } else {
    return false;
  }
  return true;
}

template <class T>
int rn_backward(egnn_ctx* ctx, RnShape p, RnAdjoint<T> a, float* dgamma, hipStream_t st) {
  const int vecs = (p.C + RvWidth<T>::V - 1) / RvWidth<T>::V, size = sizeof(T);
  const RnSplit s = rn_split(p.n, p.lmax, p.C);
  p.lanes = rn_lanes(vecs);
  const bool alone = p.n && s.chunks == 1 && p.lmax == 0;          // one chunk: its gradient of gamma is that of all
  const bool even = p.C % RvWidth<T>::V == 0 && rv_aligned({a.h, a.dy, a.dh, a.dx, a.gamma}, {a.hs * size, a.dys * size, a.dh ? a.dhs * size : 0, a.dxs * size});
  RnAdjoint<T> direct = a;
  if (alone) direct.part = dgamma;
  const dim3 join((p.C + 15) / 16, p.lmax + 1);
  if (!p.n || (even ? rn_backward_vectors<T, true>(p, s, direct, vecs, st) : rn_backward_vectors<T, false>(p, s, direct, vecs, st))) {
    if (!alone) hipLaunchKernelGGL(rn_join_kernel<float>, join, dim3(RN_JOIN), 0, st, p, s, (const float*)a.part, dgamma);
  } else {
    hipLaunchKernelGGL(rn_any_adjoint_kernel<T>, dim3(s.chunks * (p.lmax + 1)), dim3(RN_THREADS), 0, st, p, s, a);
    hipLaunchKernelGGL(rn_join_kernel<double>, join, dim3(RN_JOIN), 0, st, p, s, (const double*)a.part, dgamma);
  }
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
  if (n_rows > 1 && ((h && ((h == x && h_stride != x_stride) || (h == r && h_stride != r_stride))) ||
      (y && ((y == x && y_stride != x_stride) || (r && y == r && y_stride != r_stride)))))
    return egnn_fail(ctx, EGNN_EINVAL, "rms_norm: a result in the place of an operand has its row stride");
  if (q && (q_stride < channels || q_stride % 16 || (uintptr_t)q % 16))
    return egnn_fail(ctx, EGNN_EINVAL, "rms_norm: rows of codes begin at multiples of 16 bytes");
  if (n_rows == 0) return EGNN_OK;
  const RnShape p{n_rows, channels, lmax, eps, 1};
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
  *bytes = (size_t)rn_split(n_rows, lmax, channels).chunks * (lmax + 1) * channels * sizeof(double);
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
  if (n_rows > 1 && ((dx == h && dx_stride != h_stride) || (dx == dy && dx_stride != dy_stride) || (dh && dx == dh && dx_stride != dh_stride)))
    return egnn_fail(ctx, EGNN_EINVAL, "rms_norm_backward: a result in the place of an operand has its row stride");
  size_t need = 0;
  egnn_rms_norm_workspace_bytes(ctx, n_rows, lmax, channels, &need);
  if (!ws || (uintptr_t)ws % 256 || ws_bytes < need)
    return egnn_fail(ctx, EGNN_EWS, "rms_norm_backward: workspace too small or not 256-byte aligned");
  const RnShape p{n_rows, channels, lmax, eps, 1};
  hipStream_t st = (hipStream_t)stream;
#define RN_CALL(T) return rn_backward<T>(ctx, p, {(const T*)h, (const T*)dy, (const T*)dh, (T*)dx, (float*)ws, h_stride, dy_stride, dh_stride, dx_stride, gamma}, dgamma, st)
  if (dtype == EGNN_F32) RN_CALL(float);
  if (dtype == EGNN_F16) RN_CALL(_Float16);
  RN_CALL(__bf16);
#undef RN_CALL
}
