// Group norm with SiLU over the rows of a structure (or of each of several), channels last, and its adjoint.
//
// Rows of one segment s (a structure) and the channels of one group g are normalised together:
//   mean = sum x / n, var = sum (x - mean)^2 / n, rstd = 1 / sqrt(var + eps), n = rows of s times channels of g,
//   xhat = (x - mean) rstd, z = gamma_c xhat + beta_c, y = z / (1 + exp(-z)).
// Adjoint, with dz = dy sig (1 + z (1 - sig)), sig = 1 / (1 + exp(-z)):
//   dgamma_c = sum_rows dz xhat, dbeta_c = sum_rows dz, dx = rstd (gamma_c dz - mean_g(gamma dz) - xhat mean_g(gamma dz xhat)).
// (The three terms of dx cancel in small groups, and are all there is of it in groups of one or two values: they are subtracted in fp64.)
// Both directions are a pass that sums and a pass that writes, one launch each.  What bounds them is memory: x (and dy) are
// read twice, because the sums of all rows of a segment come before its first result.  The second pass goes through its rows from the last
// to the first, so that it begins with what the first pass left in the caches.  Where one workgroup takes all rows the two are one launch.
//
// Measured: 625,262 x 32 fp32 14 + 27 us forward, 27 + 39 adjoint (80 MB a tensor, read again from the 256 MB cache); 2,350,179 x 64 bf16 77 us (3.9
// TB/s) + 101 us (6.0 TB/s); 20,000 x 64 fp32 inside [20,000][25][64] in 37 segments 9 + 11 + 10 + 11; 64 x 16 in one launch 4.6.  Where
// tensors are small or segments many, it is not memory: a launch of ragged segments starts with a search of dependent loads for its first
// segment, and a workgroup takes its segments in turn, each with several barriers (300 structures of one row beside one of 100,000: 810 us).
//
// The rows are cut into equal chunks, one workgroup each; segments are ragged and may be shorter or longer than a chunk.
// A chunk c and a segment s that share rows own the slot c + s of the partial sums: walking along the rows either c or s
// goes up by one, so no two pairs share a slot, the slots of a segment are contiguous, and their number is at most chunks +
// segments.  The second pass adds the slots of its segments itself, in a fixed order (no atomics).
#include "row_types.h"

namespace {

constexpr int GN_CHUNKS = 512;        // two workgroups per compute unit; the second pass reads all partial sums of a segment (forward and
                                      // adjoint of 625,262 x 32 fp32 41 and 65 us, of 2,350,179 x 64 bf16 177 and 297 over and over on one
                                      // tensor; 256 chunks 41 and 63, 186 and 348; 1,024 47 and 70, 187 and 323)
constexpr int GN_CHUNK_BYTES = 16384; // a chunk holds at least this much of x, unless its segments are short: below it the launch is longer than
                                      // the reading
constexpr int GN_ALONE_BYTES = 131072; // up to this much of x, of two segments at most, one workgroup takes all rows (1,000 x 32 fp32
                                       // 9.8 us alone, 12.1 in two launches; 2,000 x 32 14.8 and 11.9)
constexpr int GN_THREADS = 512;       // 1,024 where a row has more than 512 pieces
constexpr int GN_ROWS = 4;            // rows of a thread under way at once

struct GnShape {
  long n;               // rows
  int C, G, S;          // channels, groups, segments
  int chunks;
  long rows;            // rows per chunk
  const int* ptr;       // [S + 1] or NULL: one segment of all rows
};

__host__ __device__ inline long gn_clamp(long v, long n) { return v < 0 ? 0 : v > n ? n : v; }
__device__ __forceinline__ long gn_begin(const GnShape& p, int s) { return p.ptr ? gn_clamp(p.ptr[s], p.n) : s ? p.n : 0; }

// first segment that ends behind `row`
__device__ __forceinline__ int gn_first_segment(const GnShape& p, long row) {
  int lo = 0, hi = p.S;
  while (lo < hi) {
    const int mid = lo + ((hi - lo) >> 1);
    if (gn_begin(p, mid + 1) > row) hi = mid; else lo = mid + 1;
  }
  return lo;
}

// ---- sums inside a workgroup -------------------------------------------------------------------------------------------------
// v[rows][width]: sums over the rows, to row 0
template <class P>
__device__ __forceinline__ void gn_sum_over_rows(P* v, int rows, int width) {
  while (rows > 1) {
    const int half = (rows + 1) >> 1;
    __syncthreads();
    for (int e = threadIdx.x; e < (rows - half) * width; e += blockDim.x) {
      v[e].x += v[e + half * width].x;
      v[e].y += v[e + half * width].y;
    }
    rows = half;
  }
  __syncthreads();
}
// v[n]: sums over runs of `size`, to the first of each
template <class P>
__device__ __forceinline__ void gn_sum_over_runs(P* v, int n, int size) {
  for (int left = size; left > 1;) {
    const int half = (left + 1) >> 1;
    for (int e = threadIdx.x; e < n; e += blockDim.x) {
      const int k = e % size;
      if (k < left - half) {
        v[e].x += v[e + half].x;
        v[e].y += v[e + half].y;
      }
    }
    left = half;
    __syncthreads();
  }
}

// calls f(row index of GN_ROWS rows, number of them that are there) for the rows of this thread, the last ones first
template <class F>
__device__ __forceinline__ void gn_rows_backwards(long b, long e, int rr, int slots, const F& f) {
  const long mine = e - b > rr ? (e - b - rr + slots - 1) / slots : 0;      // rows b + rr + k slots
  for (long k = (mine + GN_ROWS - 1) / GN_ROWS - 1; k >= 0; --k) f(b + rr + k * GN_ROWS * slots, (int)min((long)GN_ROWS, mine - k * GN_ROWS));
}

struct GnLanes { int L, slots, l, rr; };
template <int V>
__device__ __forceinline__ GnLanes gn_lanes(int C) {
  GnLanes t;
  t.L = C / V;
  t.slots = blockDim.x / t.L;
  t.l = threadIdx.x % t.L;
  t.rr = threadIdx.x / t.L;
  return t;
}

// ---- forward ---------------------------------------------------------------------------------------------------------
// Sums over the rows b .. e - 1 of one segment, per group, to s[g * run]; returns run.
// They are of x - x', x' the first value of the segment and group, and fp64: sum (x - x')^2 / n - (sum (x - x') / n)^2 then loses nothing to
// a mean far from zero, and a first value far from all others costs n 2^-53.
template <class T, int V>
__device__ __forceinline__ int gn_segment_rows(const GnShape& p, const T* x, long x_stride, const T* first, long b, long e, double2* s) {
  const GnLanes t = gn_lanes<V>(p.C);
  const int size = p.C / p.G;
  const bool whole = size % V == 0;            // all values of a thread are of one group
  double a1[V], a2[V], from[V];
#pragma unroll
  for (int q = 0; q < V; ++q) {
    a1[q] = a2[q] = 0.0;
    from[q] = (double)(float)first[(t.l * V + q) / size * size];
  }
  if (t.rr < t.slots) {
    for (long r = b + t.rr; r < e; r += GN_ROWS * t.slots) {
      float v[GN_ROWS][V];
#pragma unroll
      for (int k = 0; k < GN_ROWS; ++k) rt_load<T, V>(x + min(r + (long)k * t.slots, e - 1) * x_stride + t.l * V, v[k]);
#pragma unroll
      for (int k = 0; k < GN_ROWS; ++k)
        if (r + (long)k * t.slots < e)
#pragma unroll
          for (int q = 0; q < V; ++q) {
            const double d = (double)v[k][q] - from[q];
            a1[q] += d;
            a2[q] += d * d;
          }
    }
    if (whole) {
#pragma unroll
      for (int q = 1; q < V; ++q) {
        a1[0] += a1[q];
        a2[0] += a2[q];
      }
      s[t.rr * t.L + t.l] = make_double2(a1[0], a2[0]);
    } else {
#pragma unroll
      for (int q = 0; q < V; ++q) s[t.rr * p.C + t.l * V + q] = make_double2(a1[q], a2[q]);
    }
  }
  const int width = whole ? t.L : p.C, run = width / p.G;
  gn_sum_over_rows(s, t.slots, width);
  gn_sum_over_runs(s, width, run);
  return run;
}

template <class T, int V>
__global__ __launch_bounds__(V == 1 ? 1024 : GN_THREADS) void gn_sums_kernel(GnShape p, const T* x, long x_stride, double2* part, float* first_of) {
  extern __shared__ double2 smem[];
  const long r0 = (long)blockIdx.x * p.rows, r1 = min(r0 + p.rows, p.n);
  const int size = p.C / p.G;
  for (int s = gn_first_segment(p, r0); s < p.S; ++s) {
    const long sb = gn_begin(p, s), b = max(sb, r0), e = min(gn_begin(p, s + 1), r1);
    if (sb >= r1) break;
    if (b >= e) continue;
    const T* first = x + sb * x_stride;
    const int run = gn_segment_rows<T, V>(p, x, x_stride, first, b, e, smem);
    for (int g = threadIdx.x; g < p.G; g += blockDim.x) {
      part[((size_t)blockIdx.x + s) * p.G + g] = smem[g * run];
      if (b == sb) first_of[(size_t)s * p.G + g] = (float)first[g * size];   // (y may be x: kept apart)
    }
    __syncthreads();
  }
}

// sums of the slots of segment s, to v[G]; v has room for a value of every thread
__device__ __forceinline__ void gn_segment_sums(const GnShape& p, const double2* part, int s, double2* v) {
  const int c0 = (int)(gn_begin(p, s) / p.rows), c1 = (int)((gn_begin(p, s + 1) - 1) / p.rows);
  const int rows = max(1, (int)blockDim.x / p.G), k = threadIdx.x / p.G;
  if (k < rows)
    for (int g = threadIdx.x % p.G; g < p.G; g += blockDim.x) {
      double2 t = make_double2(0.0, 0.0);
#pragma unroll 4
      for (int c = c0 + k; c <= c1; c += rows) {
        const double2 u = part[((size_t)c + s) * p.G + g];
        t.x += u.x;
        t.y += u.y;
      }
      v[k * p.G + g] = t;
    }
  gn_sum_over_rows(v, min(rows, c1 - c0 + 1), p.G);
}

__device__ __forceinline__ float gn_sigmoid(float z) { return __builtin_amdgcn_rcpf(1.0f + __expf(-z)); }

// ALONE: the only workgroup, which makes the sums itself
template <class T, int V, bool ALONE>
__global__ __launch_bounds__(V == 1 ? 1024 : GN_THREADS) void gn_write_kernel(GnShape p, const T* x, long x_stride, const float* gamma, const float* beta,
                                                        float eps, T* y, long y_stride, float* mean, float* rstd,
                                                        const double2* part, const float* first) {
  extern __shared__ double2 smem[];
  __shared__ float s_mean[1024], s_rstd[1024];
  const GnLanes t = gn_lanes<V>(p.C);
  const long r0 = (long)blockIdx.x * p.rows, r1 = min(r0 + p.rows, p.n);
  const int size = p.C / p.G;
  // segments without rows: the first workgroup writes their zeros
  if (blockIdx.x == 0)
    for (long s = threadIdx.x; s < p.S; s += blockDim.x)
      if (gn_begin(p, (int)s) >= gn_begin(p, (int)s + 1))
        for (int g = 0; g < p.G; ++g) mean[s * p.G + g] = rstd[s * p.G + g] = 0.0f;
  float ga[V], be[V];
#pragma unroll
  for (int q = 0; q < V; ++q) {
    ga[q] = gamma[t.l * V + q];
    be[q] = beta[t.l * V + q];
  }
  for (int s = gn_first_segment(p, r0); s < p.S; ++s) {
    const long sb = gn_begin(p, s), se = gn_begin(p, s + 1);
    const long b = max(sb, r0), e = min(se, r1);
    if (sb >= r1) break;
    if (b >= e) continue;
    int run = 1;
    const T* head = x + sb * x_stride;
    if (ALONE) run = gn_segment_rows<T, V>(p, x, x_stride, head, b, e, smem);
    else gn_segment_sums(p, part, s, smem);
    for (int g = threadIdx.x; g < p.G; g += blockDim.x) {
      const double n = (double)(se - sb) * size, mu = smem[g * run].x / n;
      const double var = smem[g * run].y / n - mu * mu;
      const float from = ALONE ? (float)head[g * size] : first[(size_t)s * p.G + g];
      s_mean[g] = (float)((double)from + mu);
      s_rstd[g] = (float)(1.0 / sqrt((var < 0.0 ? 0.0 : var) + (double)eps));   // (a NaN stays one)
      if (b == sb) {
        mean[(size_t)s * p.G + g] = s_mean[g];
        rstd[(size_t)s * p.G + g] = s_rstd[g];
      }
    }
    __syncthreads();
    if (t.rr < t.slots) {
      float mu[V], rs[V];
#pragma unroll
      for (int q = 0; q < V; ++q) {
        const int g = (t.l * V + q) / size;
        mu[q] = s_mean[g];
        rs[q] = s_rstd[g];
      }
      gn_rows_backwards(b, e, t.rr, t.slots, [&](long r, int rows) {
        float v[GN_ROWS][V];
#pragma unroll
        for (int k = 0; k < GN_ROWS; ++k) rt_load<T, V>(x + (r + (long)min(k, rows - 1) * t.slots) * x_stride + t.l * V, v[k]);
#pragma unroll
        for (int k = 0; k < GN_ROWS; ++k) {
          if (k >= rows) break;
#pragma unroll
          for (int q = 0; q < V; ++q) {
            const float z = (v[k][q] - mu[q]) * rs[q] * ga[q] + be[q];
            v[k][q] = z * gn_sigmoid(z);
          }
          rt_store<T, V>(y + (r + (long)k * t.slots) * y_stride + t.l * V, v[k]);
        }
      });
    }
    __syncthreads();
  }
}

// ---- adjoint ---------------------------------------------------------------------------------------------------------
struct GnAdjoint {
  const float *mean, *rstd, *gamma, *beta;
};
// LDS of the sums: double2 [C] of the whole chunk, double2 [C] of groups, float2 [slots][C] (at most 64 KB)
__host__ __device__ inline size_t gn_adjoint_lds(int C, int slots) { return (size_t)C * (2 * sizeof(double2) + slots * sizeof(float2)); }

// Sums over the rows b .. e - 1 of segment s: per channel into rows[C] (and added to total[C]), per group with gamma into groups[g * size].
// GN_ROWS terms are added in fp32, those of a thread and of the chunk's segments in fp64, those of the threads in fp32 again, as a tree
// of at most nine levels (so that LDS holds them).
template <class T, int V>
__device__ __forceinline__ void gn_adjoint_rows(const GnShape& p, const GnAdjoint& w, const T* x, long x_stride, const T* dy, long dy_stride, int s, long b,
                                                long e, const float (&ga)[V], const float (&be)[V], float2* rows, double2* total,
                                                double2* groups) {
  const GnLanes t = gn_lanes<V>(p.C);
  const int size = p.C / p.G;
  if (t.rr < t.slots) {
    float mu[V], rs[V];
    double a1[V], a2[V];
#pragma unroll
    for (int q = 0; q < V; ++q) {
      const size_t at = (size_t)s * p.G + (t.l * V + q) / size;
      mu[q] = w.mean[at];
      rs[q] = w.rstd[at];
      a1[q] = a2[q] = 0.0;
    }
    for (long r = b + t.rr; r < e; r += GN_ROWS * t.slots) {
      float v[GN_ROWS][V], d[GN_ROWS][V];
#pragma unroll
      for (int k = 0; k < GN_ROWS; ++k) {
        const long at = min(r + (long)k * t.slots, e - 1);
        rt_load<T, V>(x + at * x_stride + t.l * V, v[k]);
        rt_load<T, V>(dy + at * dy_stride + t.l * V, d[k]);
      }
      float s1[V] = {}, s2[V] = {};
#pragma unroll
      for (int k = 0; k < GN_ROWS; ++k)
        if (r + (long)k * t.slots < e)
#pragma unroll
          for (int q = 0; q < V; ++q) {
            const float h = (v[k][q] - mu[q]) * rs[q], z = h * ga[q] + be[q], sig = gn_sigmoid(z);
            const float dz = d[k][q] * sig * (1.0f + z * (1.0f - sig));
            s1[q] += dz;
            s2[q] += dz * h;
          }
#pragma unroll
      for (int q = 0; q < V; ++q) {
        a1[q] += (double)s1[q];
        a2[q] += (double)s2[q];
      }
    }
#pragma unroll
    for (int q = 0; q < V; ++q) rows[t.rr * p.C + t.l * V + q] = make_float2((float)a1[q], (float)a2[q]);
  }
  gn_sum_over_rows(rows, t.slots, p.C);
  for (int c = threadIdx.x; c < p.C; c += blockDim.x) {
    total[c].x += (double)rows[c].x;
    total[c].y += (double)rows[c].y;
    groups[c] = make_double2((double)w.gamma[c] * rows[c].x, (double)w.gamma[c] * rows[c].y);
  }
  __syncthreads();
  gn_sum_over_runs(groups, p.C, size);
}

template <class T, int V>
__global__ __launch_bounds__(V == 1 ? 1024 : GN_THREADS) void gn_adjoint_sums_kernel(GnShape p, GnAdjoint w, const T* x, long x_stride, const T* dy,
                                                               long dy_stride, double2* part, float2* channel_part) {
  extern __shared__ double2 smem[];
  const GnLanes t = gn_lanes<V>(p.C);
  double2 *total = smem, *groups = smem + p.C;
  float2* srow = (float2*)(smem + 2 * p.C);
  const long r0 = (long)blockIdx.x * p.rows, r1 = min(r0 + p.rows, p.n);
  const int size = p.C / p.G;
  float ga[V], be[V];
#pragma unroll
  for (int q = 0; q < V; ++q) {
    ga[q] = w.gamma[t.l * V + q];
    be[q] = w.beta[t.l * V + q];
  }
  for (int c = threadIdx.x; c < p.C; c += blockDim.x) total[c] = make_double2(0.0, 0.0);
  for (int s = gn_first_segment(p, r0); s < p.S; ++s) {
    const long b = max(gn_begin(p, s), r0), e = min(gn_begin(p, s + 1), r1);
    if (gn_begin(p, s) >= r1) break;
    if (b >= e) continue;
    gn_adjoint_rows<T, V>(p, w, x, x_stride, dy, dy_stride, s, b, e, ga, be, srow, total, groups);
    for (int g = threadIdx.x; g < p.G; g += blockDim.x) part[((size_t)blockIdx.x + s) * p.G + g] = groups[g * size];
    __syncthreads();
  }
  for (int c = threadIdx.x; c < p.C; c += blockDim.x) channel_part[(size_t)blockIdx.x * p.C + c] = make_float2((float)total[c].x, (float)total[c].y);
}

template <class T, int V, bool ALONE>
__global__ __launch_bounds__(V == 1 ? 1024 : GN_THREADS) void gn_adjoint_write_kernel(GnShape p, GnAdjoint w, const T* x, long x_stride, const T* dy,
                                                                long dy_stride, T* dx, long dx_stride, float* dgamma,
                                                                float* dbeta, const double2* part, const float2* channel_part) {
  extern __shared__ double2 smem[];
  const GnLanes t = gn_lanes<V>(p.C);
  double2 *total = smem, *groups = ALONE ? smem + p.C : smem;             // ALONE: as in the sums
  float2* srow = (float2*)(smem + 2 * p.C);
  if (!ALONE && (int)blockIdx.x >= p.chunks) {   // the last workgroups add the channels' sums over the chunks, 16 channels each
    const int c = ((int)blockIdx.x - p.chunks) * 16 + threadIdx.x % 16, per = blockDim.x / 16;
    double2 u = make_double2(0.0, 0.0);
    if (c < p.C)
#pragma unroll 4
      for (int k = threadIdx.x / 16; k < p.chunks; k += per) {
        const float2 v = channel_part[(size_t)k * p.C + c];
        u.x += v.x;
        u.y += v.y;
      }
    smem[threadIdx.x] = u;
    gn_sum_over_rows(smem, per, 16);
    if (threadIdx.x < 16 && c < p.C) {
      dbeta[c] = (float)smem[threadIdx.x].x;
      dgamma[c] = (float)smem[threadIdx.x].y;
    }
    return;
  }
  const long r0 = (long)blockIdx.x * p.rows, r1 = min(r0 + p.rows, p.n);
  const int size = p.C / p.G;
  float ga[V], be[V];
#pragma unroll
  for (int q = 0; q < V; ++q) {
    ga[q] = w.gamma[t.l * V + q];
    be[q] = w.beta[t.l * V + q];
  }
  if (ALONE)
    for (int c = threadIdx.x; c < p.C; c += blockDim.x) total[c] = make_double2(0.0, 0.0);
  for (int s = gn_first_segment(p, r0); s < p.S; ++s) {
    const long sb = gn_begin(p, s), se = gn_begin(p, s + 1);
    const long b = max(sb, r0), e = min(se, r1);
    if (sb >= r1) break;
    if (b >= e) continue;
    if (ALONE) gn_adjoint_rows<T, V>(p, w, x, x_stride, dy, dy_stride, s, b, e, ga, be, srow, total, groups);
    else gn_segment_sums(p, part, s, groups);
    if (t.rr < t.slots) {
      float mu[V], rs[V];
      double m1[V], m2[V];
      const double inv = 1.0 / ((double)(se - sb) * size);
#pragma unroll
      for (int q = 0; q < V; ++q) {
        const int g = (t.l * V + q) / size;
        const size_t at = (size_t)s * p.G + g;
        mu[q] = w.mean[at];
        rs[q] = w.rstd[at];
        m1[q] = groups[ALONE ? g * size : g].x * inv;
        m2[q] = groups[ALONE ? g * size : g].y * inv;
      }
      gn_rows_backwards(b, e, t.rr, t.slots, [&](long r, int rows) {
        float v[GN_ROWS][V], d[GN_ROWS][V];
#pragma unroll
        for (int k = 0; k < GN_ROWS; ++k) {
          const long at = r + (long)min(k, rows - 1) * t.slots;
          rt_load<T, V>(x + at * x_stride + t.l * V, v[k]);
          rt_load<T, V>(dy + at * dy_stride + t.l * V, d[k]);
        }
#pragma unroll
        for (int k = 0; k < GN_ROWS; ++k) {
          if (k >= rows) break;
#pragma unroll
          for (int q = 0; q < V; ++q) {
            const float h = (v[k][q] - mu[q]) * rs[q], z = h * ga[q] + be[q], sig = gn_sigmoid(z);
            const float dz = d[k][q] * sig * (1.0f + z * (1.0f - sig));
            v[k][q] = rs[q] * (float)((double)ga[q] * dz - m1[q] - (double)h * m2[q]);
          }
          rt_store<T, V>(dx + (r + (long)k * t.slots) * dx_stride + t.l * V, v[k]);
        }
      });
    }
    __syncthreads();
  }
  if (ALONE) {
    __syncthreads();
    for (int c = threadIdx.x; c < p.C; c += blockDim.x) {
      dbeta[c] = (float)total[c].x;
      dgamma[c] = (float)total[c].y;
    }
  }
}

__global__ void gn_no_rows_kernel(float* a, long na, float* b, long nb) {
  for (long i = threadIdx.x; i < na; i += blockDim.x) a[i] = 0.0f;
  for (long i = threadIdx.x; i < nb; i += blockDim.x) b[i] = 0.0f;
}

size_t gn_align(size_t n) { return (n + 255) & ~(size_t)255; }

GnShape gn_shape(int64_t n, int32_t C, int32_t G, int32_t S, const int32_t* ptr, int element) {
  GnShape p;
  p.n = n; p.C = C; p.G = G; p.S = S; p.ptr = ptr;
  long least = (GN_CHUNK_BYTES + (long)C * element - 1) / ((long)C * element);
  // a workgroup takes its segments one after the other: about two of them each (forward of 1,000 x 32 fp32 in 100 segments 15 us, in one
  // workgroup 256; 5,000 x 64 in 300 20 us, in chunks of 16 KB 28)
  if (S > 1 && 2 * n / S < least) least = 2 * n / S > 0 ? 2 * n / S : 1;
  p.rows = (n + GN_CHUNKS - 1) / GN_CHUNKS;
  if (p.rows < least) p.rows = least;
  // groups of fewer than four channels keep a sum per value instead of one per thread (325 x 200 fp16 in 200 groups 13 us, alone 18)
  const double alone = C / G < 4 ? GN_ALONE_BYTES / 4 : GN_ALONE_BYTES;
  if (S <= 2 && (double)n * C * element <= alone) p.rows = n > 0 ? n : 1;
  p.chunks = (int)((n + p.rows - 1) / p.rows);
  return p;
}

// partial sums per slot, channel sums per chunk (element = 4: the most chunks any type gives)
size_t gn_part_bytes(const GnShape& p) { return gn_align(((size_t)p.chunks + p.S) * p.G * sizeof(double2)); }
size_t gn_first_bytes(const GnShape& p) { return gn_align((size_t)p.S * p.G * sizeof(float)); }
size_t gn_channel_bytes(const GnShape& p) { return gn_align((size_t)p.chunks * p.C * sizeof(float2)); }

int gn_check(egnn_ctx* ctx, const char* who, int32_t dtype, int64_t n, int32_t C, int32_t G, const int32_t* ptr, int32_t S) {
  const std::string at(who);
  if (!rt_size(dtype)) return egnn_fail(ctx, EGNN_EINVAL, at + ": dtype must be EGNN_F32, EGNN_F16 or EGNN_BF16");
  if (n < 0 || n > 0x7fffffff) return egnn_fail(ctx, EGNN_EINVAL, at + ": n_rows must be in 0..2^31-1");
  if (C < 1 || C > 1024) return egnn_fail(ctx, EGNN_EINVAL, at + ": channels must be in 1..1024");
  if (G < 1 || C % G) return egnn_fail(ctx, EGNN_EINVAL, at + ": groups must divide the channels");
  if (S < 1 || (!ptr && S != 1)) return egnn_fail(ctx, EGNN_EINVAL, at + ": n_segments must be at least 1, and 1 without ptr");
  return EGNN_OK;
}

// vector width for which all rows are aligned
template <class T>
int gn_width(int32_t C, std::initializer_list<const void*> at, std::initializer_list<int64_t> strides) {
  for (int v = 16 / (int)sizeof(T); v > 1; v /= 2) {
    if (v == 2) continue;
    bool fits = C % v == 0;
    for (const void* a : at) fits = fits && (uintptr_t)a % (v * sizeof(T)) == 0;
    for (int64_t s : strides) fits = fits && s % v == 0;
    if (fits) return v;
  }
  return 1;
}

struct GnLaunch { int threads, slots; };
GnLaunch gn_launch(int C, int V, bool halved = false) {
  const int L = C / V, threads = L > GN_THREADS ? 1024 : halved ? GN_THREADS / 2 : GN_THREADS;      // (V > 1: at most 256 pieces)
  return {threads, threads / L};
}

template <class T, int V>
int gn_forward(egnn_ctx* ctx, const GnShape& p, const void* x, int64_t xs, const float* gamma, const float* beta, float eps, void* y,
               int64_t ys, float* mean, float* rstd, void* ws, hipStream_t st) {
  // eight sums a thread, where a thread's values are of several groups: half the threads, for LDS
  const GnLaunch at = gn_launch(p.C, V, V == 8 && p.C / p.G % V != 0);
  double2* part = (double2*)ws;
  float* first = (float*)((char*)ws + gn_part_bytes(p));
  const size_t sums = (size_t)at.slots * (p.C / p.G % V ? p.C : p.C / V) * sizeof(double2);
  if (p.chunks == 1) {
    hipLaunchKernelGGL((gn_write_kernel<T, V, true>), dim3(1), dim3(at.threads), sums, st, p, (const T*)x, (long)xs, gamma, beta, eps, (T*)y,
                       (long)ys, mean, rstd, (const double2*)nullptr, (const float*)nullptr);
  } else {
    const size_t slots = (size_t)(p.G > at.threads ? p.G : at.threads) * sizeof(double2);
    hipLaunchKernelGGL((gn_sums_kernel<T, V>), dim3(p.chunks), dim3(at.threads), sums, st, p, (const T*)x, (long)xs, part, first);
    hipLaunchKernelGGL((gn_write_kernel<T, V, false>), dim3(p.chunks), dim3(at.threads), slots, st, p, (const T*)x, (long)xs, gamma, beta, eps,
                       (T*)y, (long)ys, mean, rstd, (const double2*)part, (const float*)first);
  }
  EGNN_LAUNCH_CHECK(ctx, "group_norm");
  return EGNN_OK;
}

template <class T, int V>
int gn_backward(egnn_ctx* ctx, const GnShape& p, const GnAdjoint& w, const void* x, int64_t xs, const void* dy, int64_t dys, void* dx,
                int64_t dxs, float* dgamma, float* dbeta, void* ws, hipStream_t st) {
  const GnLaunch at = gn_launch(p.C, V);
  double2* part = (double2*)ws;
  float2* channel_part = (float2*)((char*)ws + gn_part_bytes(p));
  if (p.chunks == 1) {
    hipLaunchKernelGGL((gn_adjoint_write_kernel<T, V, true>), dim3(1), dim3(at.threads), gn_adjoint_lds(p.C, at.slots), st, p, w, (const T*)x, (long)xs,
                       (const T*)dy, (long)dys, (T*)dx, (long)dxs, dgamma, dbeta, (const double2*)nullptr, (const float2*)nullptr);
  } else {
    const size_t slots = (size_t)(p.G > at.threads ? p.G : at.threads) * sizeof(double2);
    // (eight values a thread and their fp64 sums are 161 registers, for one workgroup per compute unit instead of two: adjoint of 300,000 x 64 bf16
    // 53.8 us, with four 48.2)
    constexpr int VS = V == 8 ? 4 : V;
    const GnLaunch first = gn_launch(p.C, VS);
    hipLaunchKernelGGL((gn_adjoint_sums_kernel<T, VS>), dim3(p.chunks), dim3(first.threads), gn_adjoint_lds(p.C, first.slots), st, p, w, (const T*)x,
                       (long)xs, (const T*)dy, (long)dys, part, channel_part);
    hipLaunchKernelGGL((gn_adjoint_write_kernel<T, V, false>), dim3(p.chunks + (p.C + 15) / 16), dim3(at.threads), slots, st, p, w, (const T*)x,
                       (long)xs, (const T*)dy, (long)dys, (T*)dx, (long)dxs, dgamma, dbeta, (const double2*)part,
                       (const float2*)channel_part);
  }
  EGNN_LAUNCH_CHECK(ctx, "group_norm_backward");
  return EGNN_OK;
}

}  // namespace

extern "C" int egnn_group_norm_workspace_bytes(const egnn_ctx* ctx, int64_t n_rows, int32_t n_segments, int32_t channels,
                                               int32_t groups, size_t* bytes) {
  if (!ctx || !bytes || n_rows < 0 || n_rows > 0x7fffffff || n_segments < 1 || channels < 1 || channels > 1024 || groups < 1 ||
      channels % groups)
    return egnn_fail(const_cast<egnn_ctx*>(ctx), EGNN_EINVAL, "group_norm_workspace_bytes: bad argument");
  const GnShape p = gn_shape(n_rows, channels, groups, n_segments, nullptr, 4);
  const size_t forward = gn_part_bytes(p) + gn_first_bytes(p), backward = gn_part_bytes(p) + gn_channel_bytes(p);
  *bytes = forward > backward ? forward : backward;
  return EGNN_OK;
}

extern "C" int egnn_group_norm(egnn_ctx* ctx, int32_t dtype, const void* x, int64_t x_stride, int64_t n_rows, int32_t channels,
                               int32_t groups, const int32_t* ptr, int32_t n_segments, const float* gamma, const float* beta,
                               float eps, void* y, int64_t y_stride, float* mean, float* rstd, void* ws, size_t ws_bytes,
                               void* stream) {
  if (!ctx) return EGNN_EINVAL;
  if (int rc = gn_check(ctx, "group_norm", dtype, n_rows, channels, groups, ptr, n_segments)) return rc;
  if (!gamma || !beta || !mean || !rstd || (n_rows > 0 && (!x || !y)))
    return egnn_fail(ctx, EGNN_EINVAL, "group_norm: null pointer");
  if (x_stride < channels || y_stride < channels) return egnn_fail(ctx, EGNN_EINVAL, "group_norm: a row stride below the channels");
  if (!(eps > 0.0f)) return egnn_fail(ctx, EGNN_EINVAL, "group_norm: eps must be > 0");
  hipStream_t st = (hipStream_t)stream;
  const GnShape p = gn_shape(n_rows, channels, groups, n_segments, ptr, rt_size(dtype));
  if (n_rows == 0) {
    const long k = (long)n_segments * groups;
    hipLaunchKernelGGL(gn_no_rows_kernel, dim3(1), dim3(256), 0, st, mean, k, rstd, k);
    EGNN_LAUNCH_CHECK(ctx, "group_norm");
    return EGNN_OK;
  }
  if (!ws || (uintptr_t)ws % 256 || ws_bytes < gn_part_bytes(p) + gn_first_bytes(p))
    return egnn_fail(ctx, EGNN_EWS, "group_norm: workspace too small or not 256-byte aligned");
#define GN_CALL(T, V) return gn_forward<T, V>(ctx, p, x, x_stride, gamma, beta, eps, y, y_stride, mean, rstd, ws, st)
  if (dtype == EGNN_F32) {
    if (gn_width<float>(channels, {x, y}, {x_stride, y_stride}) == 4) GN_CALL(float, 4);
    GN_CALL(float, 1);
  }
  const int v = gn_width<_Float16>(channels, {x, y}, {x_stride, y_stride});
  if (dtype == EGNN_F16) {
    if (v == 8) GN_CALL(_Float16, 8);
    if (v == 4) GN_CALL(_Float16, 4);
    GN_CALL(_Float16, 1);
  }
  if (v == 8) GN_CALL(__bf16, 8);
  if (v == 4) GN_CALL(__bf16, 4);
  GN_CALL(__bf16, 1);
#undef GN_CALL
}

extern "C" int egnn_group_norm_backward(egnn_ctx* ctx, int32_t dtype, const void* x, int64_t x_stride, const void* dy,
                                        int64_t dy_stride, const float* mean, const float* rstd, int64_t n_rows, int32_t channels,
                                        int32_t groups, const int32_t* ptr, int32_t n_segments, const float* gamma,
                                        const float* beta, void* dx, int64_t dx_stride, float* dgamma, float* dbeta, void* ws,
                                        size_t ws_bytes, void* stream) {
  if (!ctx) return EGNN_EINVAL;
  if (int rc = gn_check(ctx, "group_norm_backward", dtype, n_rows, channels, groups, ptr, n_segments)) return rc;
  if (!gamma || !beta || !mean || !rstd || !dgamma || !dbeta || (n_rows > 0 && (!x || !dy || !dx)))
    return egnn_fail(ctx, EGNN_EINVAL, "group_norm_backward: null pointer");
  if (x_stride < channels || dy_stride < channels || dx_stride < channels)
    return egnn_fail(ctx, EGNN_EINVAL, "group_norm_backward: a row stride below the channels");
  hipStream_t st = (hipStream_t)stream;
  const GnShape p = gn_shape(n_rows, channels, groups, n_segments, ptr, rt_size(dtype));
  if (n_rows == 0) {
    hipLaunchKernelGGL(gn_no_rows_kernel, dim3(1), dim3(256), 0, st, dgamma, (long)channels, dbeta, (long)channels);
    EGNN_LAUNCH_CHECK(ctx, "group_norm_backward");
    return EGNN_OK;
  }
  if (!ws || (uintptr_t)ws % 256 || ws_bytes < gn_part_bytes(p) + gn_channel_bytes(p))
    return egnn_fail(ctx, EGNN_EWS, "group_norm_backward: workspace too small or not 256-byte aligned");
  const GnAdjoint w{mean, rstd, gamma, beta};
#define GN_CALL(T, V) return gn_backward<T, V>(ctx, p, w, x, x_stride, dy, dy_stride, dx, dx_stride, dgamma, dbeta, ws, st)
  if (dtype == EGNN_F32) {
    if (gn_width<float>(channels, {x, dy, dx}, {x_stride, dy_stride, dx_stride}) == 4) GN_CALL(float, 4);
    GN_CALL(float, 1);
  }
  const int v = gn_width<_Float16>(channels, {x, dy, dx}, {x_stride, dy_stride, dx_stride});
  if (dtype == EGNN_F16) {
    if (v == 8) GN_CALL(_Float16, 8);
    if (v == 4) GN_CALL(_Float16, 4);
    GN_CALL(_Float16, 1);
  }
  if (v == 8) GN_CALL(__bf16, 8);
  if (v == 4) GN_CALL(__bf16, 4);
  GN_CALL(__bf16, 1);
#undef GN_CALL
}
