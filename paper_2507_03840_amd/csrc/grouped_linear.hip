// Rows put in groups by a key, and rows times the matrix of their group with its adjoint.
//
//   group_rows:  a stable counting sort.  Row (i, (l, m)) of atom i with key s goes to group s (lmax + 1) + l; inside a group the
//                rows ascend.  Only the keys are sorted: (l, m) runs through fixed places of an atom's rows.
//   linear:      y_r = x_r W_g^T + b_g,   dx_r = dy_r W_g,   dW_g = sum_r dy_r^T x_r,   db_g = sum_r dy_r   (r in group g).
#include "row_types.h"
#include "stream_gemm.h"

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

// counts NULL: the only workgroup, which counts itself
__global__ __launch_bounds__(GR_THREADS) void gr_place_kernel(const int* key, long n, int G, int lmax, long chunk, const int* counts,
                                                              int* ptr, int* perm) {
  __shared__ int base[GR_MAX_GROUPS], total[GR_MAX_GROUPS], first[GR_MAX_GROUPS], wave_count[GR_WAVES][GR_MAX_GROUPS];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int degrees = lmax < 0 ? 1 : lmax + 1, D = degrees * degrees;
  for (int g = tid; g < G; g += GR_THREADS) {
    int before = 0, all = 0;
    if (counts)
#pragma unroll 8
      for (int c = 0; c < (int)gridDim.x; ++c) {
        const int v = counts[(size_t)c * G + g];
        before += c < (int)blockIdx.x ? v : 0;
        all += v;
      }
    base[g] = before;
    total[g] = all;
    for (int w = 0; w < GR_WAVES; ++w) wave_count[w][g] = 0;
  }
  if (!counts) {
    __syncthreads();
    for (long i = tid; i < n; i += GR_THREADS) atomicAdd(&total[gr_key(key, i, G)], 1);   // whole numbers: any order
  }
  __syncthreads();
  if (wave == 0) {
    int at = 0;
    for (int g0 = 0; g0 < G; g0 += 64) {
      const int mine = g0 + lane < G ? total[g0 + lane] : 0;
      int sum = mine;
      for (int h = 1; h < 64; h <<= 1) {
        const int v = __shfl_up(sum, h);
        if (lane >= h) sum += v;
      }
      if (g0 + lane < G) first[g0 + lane] = at + sum - mine;
      at += __shfl(sum, 63);
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

// The types on the matrix cores: fp32 as three bf16 pieces, each the rest of the ones before rounded to nearest (8 bits and a sign each: exact, no
// scaling, so gradients of any size from 2^-112 on keep their accuracy; below, pieces underflow), whose six leading products are kept.  The dropped
// ones, mid lo and smaller, are at most 2^-24 of the product and of either sign (with pieces cut off instead of rounded they were up to
// 2^-21 and always of the product's sign).  Long contractions sum the five lesser products apart from hi hi: eight of them at a time are less than
// half a step of a sum of some thousand terms, and would be rounded away one after the other (rows of 4,096 values from 1 to 2: off by 1.2e-5 with
// pieces cut off and one sum, 6e-7 rounded and one sum, 3.4e-7 with two; torch in fp32 2.4e-7).
// half precision and bfloat16 as they are.  An infinite value leaves NaN behind its first piece, and so do finite values whose pieces or
// products overflow: fp32 results that are NaN are made again with the values themselves (gl_again), which leaves NaN only where it belongs.
typedef _Float16 gl_h8 __attribute__((ext_vector_type(8)));
typedef float gl_f16v __attribute__((ext_vector_type(16)));
template <class T> struct GlType {
  static constexpr int PIECES = 1;
  typedef uint4 Raw;                                     // eight values
};
template <> struct GlType<float> {
  static constexpr int PIECES = 3;
  struct Raw { uint4 a, b; };
};

__device__ __forceinline__ gl_f16v gl_mfma(uint4 a, uint4 b, gl_f16v c, __bf16) {
  return __builtin_amdgcn_mfma_f32_32x32x16_bf16(as_bf16x8(a), as_bf16x8(b), c, 0, 0, 0);
}
__device__ __forceinline__ gl_f16v gl_mfma(uint4 a, uint4 b, gl_f16v c, _Float16) {
  return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(gl_h8, a), __builtin_bit_cast(gl_h8, b), c, 0, 0, 0);
}
template <class T>
__device__ __forceinline__ gl_f16v gl_product(const uint4 (&a)[1], const uint4 (&b)[1], gl_f16v c) {
  return gl_mfma(a[0], b[0], c, T());
}
__device__ __forceinline__ gl_f16v gl_lesser(const uint4 (&a)[3], const uint4 (&b)[3], gl_f16v c) {
  const __bf16 t = {};
  c = gl_mfma(a[2], b[0], c, t);
  c = gl_mfma(a[0], b[2], c, t);
  c = gl_mfma(a[1], b[1], c, t);
  c = gl_mfma(a[1], b[0], c, t);
  return gl_mfma(a[0], b[1], c, t);
}
template <class T>
__device__ __forceinline__ gl_f16v gl_product(const uint4 (&a)[3], const uint4 (&b)[3], gl_f16v c) {
  return gl_mfma(a[0], b[0], gl_lesser(a, b, c), __bf16{});
}
__device__ __forceinline__ gl_f16v gl_zero() {
  gl_f16v v;
#pragma unroll
  for (int i = 0; i < 16; ++i) v[i] = 0.0f;
  return v;
}
// A sum over a long contraction: fp32's lesser products apart from hi hi
template <class T>
struct GlSum {
  gl_f16v sum = gl_zero();
  template <class P> __device__ __forceinline__ void add(const P& a, const P& b) { sum = gl_product<T>(a, b, sum); }
  __device__ __forceinline__ gl_f16v value() const { return sum; }
};
template <>
struct GlSum<float> {
  gl_f16v sum = gl_zero(), lesser = gl_zero();
  __device__ __forceinline__ void add(const uint4 (&a)[3], const uint4 (&b)[3]) {
    lesser = gl_lesser(a, b, lesser);
    sum = gl_mfma(a[0], b[0], sum, __bf16{});
  }
  __device__ __forceinline__ gl_f16v value() const {
    gl_f16v v;
#pragma unroll
    for (int i = 0; i < 16; ++i) v[i] = sum[i] + lesser[i];
    return v;
  }
};

// Eight values at p, aligned to one value.  Loads are never under a condition: a condition would end in a wait for the load.  At the end of
// a row the last eight values of the row are taken instead (it has that many, or the row is narrow) and moved down by the places too many.
typedef uint32_t gl_u4 __attribute__((ext_vector_type(4), aligned(2)));
__device__ __forceinline__ uint4 gl_load16(const void* p) {
  const gl_u4 v = *reinterpret_cast<const gl_u4*>(p);
  return make_uint4(v.x, v.y, v.z, v.w);
}
template <class T>
__device__ __forceinline__ void gl_load(const T* p, uint4& r) { r = gl_load16(p); }
__device__ __forceinline__ void gl_load(const float* p, GlType<float>::Raw& r) {
  r.a = gl_load16(p);
  r.b = gl_load16(p + 4);
}
// the first `valid` of eight values, zeros behind them (rows of fewer than eight)
template <class T>
__device__ __forceinline__ void gl_load_narrow(const T* p, int valid, uint4& r) {
  uint32_t w[4] = {};
#pragma unroll
  for (int q = 0; q < 8; ++q)
    if (q < valid) w[q >> 1] |= (uint32_t) reinterpret_cast<const uint16_t*>(p)[q] << (16 * (q & 1));
  r = make_uint4(w[0], w[1], w[2], w[3]);
}
__device__ __forceinline__ void gl_load_narrow(const float* p, int valid, GlType<float>::Raw& r) {
  uint32_t w[8] = {};
#pragma unroll
  for (int q = 0; q < 8; ++q)
    if (q < valid) w[q] = __float_as_uint(p[q]);
  r.a = make_uint4(w[0], w[1], w[2], w[3]);
  r.b = make_uint4(w[4], w[5], w[6], w[7]);
}
// moves the values down by n places, zeros behind them (n >= 8: nothing is left)
template <int N, int BY>
__device__ __forceinline__ void gl_down(uint32_t (&w)[N], bool yes) {
#pragma unroll
  for (int q = 0; q < N; ++q) w[q] = yes ? (q + BY < N ? w[q + BY] : 0u) : w[q];
}
__device__ __forceinline__ void gl_shift(uint4& r, int n) {
  uint32_t w[4] = {r.x, r.y, r.z, r.w};
#pragma unroll
  for (int q = 0; q < 4; ++q)
    if (n & 1) w[q] = w[q] >> 16 | (q < 3 ? w[q + 1] << 16 : 0u);
  gl_down<4, 1>(w, n & 2);
  gl_down<4, 2>(w, n & 4);
  gl_down<4, 4>(w, n >= 8);
  r = make_uint4(w[0], w[1], w[2], w[3]);
}
__device__ __forceinline__ void gl_shift(GlType<float>::Raw& r, int n) {
  uint32_t w[8] = {r.a.x, r.a.y, r.a.z, r.a.w, r.b.x, r.b.y, r.b.z, r.b.w};
  gl_down<8, 1>(w, n & 1);
  gl_down<8, 2>(w, n & 2);
  gl_down<8, 4>(w, n & 4);
  gl_down<8, 8>(w, n >= 8);
  r.a = make_uint4(w[0], w[1], w[2], w[3]);
  r.b = make_uint4(w[4], w[5], w[6], w[7]);
}
// two values rounded to bf16
__device__ __forceinline__ uint32_t gl_round2(float a, float b) {
  typedef __bf16 pair __attribute__((ext_vector_type(2)));
  const pair v = {(__bf16)a, (__bf16)b};
  return __builtin_bit_cast(uint32_t, v);
}
// -> pieces
__device__ __forceinline__ void gl_cut(uint4 r, uint4 (&to)[1]) { to[0] = r; }
__device__ __forceinline__ void gl_cut(const GlType<float>::Raw& r, uint4 (&to)[3]) {
  const uint32_t w[8] = {r.a.x, r.a.y, r.a.z, r.a.w, r.b.x, r.b.y, r.b.z, r.b.w};
  uint32_t h[4], m[4], l[4];
#pragma unroll
  for (int q = 0; q < 4; ++q) {
    float a = __uint_as_float(w[2 * q]), b = __uint_as_float(w[2 * q + 1]);
    h[q] = gl_round2(a, b);
    a -= __uint_as_float(h[q] << 16), b -= __uint_as_float(h[q] & 0xffff0000u);
    m[q] = gl_round2(a, b);
    a -= __uint_as_float(m[q] << 16), b -= __uint_as_float(m[q] & 0xffff0000u);
    l[q] = gl_round2(a, b);
  }
  to[0] = make_uint4(h[0], h[1], h[2], h[3]);
  to[1] = make_uint4(m[0], m[1], m[2], m[3]);
  to[2] = make_uint4(l[0], l[1], l[2], l[3]);
}
// sum of n products of values a_step and b_step apart
__device__ __forceinline__ float gl_again(const float* a, long a_step, const float* b, long b_step, long n) {
  float sum = 0.0f;
  for (long k = 0; k < n && sum == sum; ++k) sum = __builtin_fmaf(a[k * a_step], b[k * b_step], sum);
  return sum;
}
template <class T>
__device__ __forceinline__ void gl_add(uint4 r, float (&to)[8]) {
  typedef T vec __attribute__((ext_vector_type(8)));
  const vec v = __builtin_bit_cast(vec, r);
#pragma unroll
  for (int q = 0; q < 8; ++q) to[q] += (float)v[q];
}
template <class T>
__device__ __forceinline__ void gl_add(const GlType<float>::Raw& r, float (&to)[8]) {
  const uint32_t w[8] = {r.a.x, r.a.y, r.a.z, r.a.w, r.b.x, r.b.y, r.b.z, r.b.w};
#pragma unroll
  for (int q = 0; q < 8; ++q) to[q] += __uint_as_float(w[q]);
}

// One tile of a product in LDS, as pieces, 16 bits a value, in one of two layouts:
//   along the contraction  [SIDE][KS]: rows of 2 KS + 16 bytes, so that eight rows read at one place meet different banks;
//   across it              [KS][SIDE]: rows of 2 SIDE + 64 bytes; the operand's eight contraction indices come out of two transposing reads
//                          of four rows each (ds_read_b64_tr_b16: lane i of sixteen gets column i of the four rows that its lanes point to).
template <int SIDE, int KS, bool ACROSS>
struct GlTile {
  static constexpr int ROW = ACROSS ? 2 * SIDE + 64 : 2 * KS + 16;           // bytes
  static constexpr int ROWS = ACROSS ? KS : SIDE, PLANE = ROW * ROWS;
  static constexpr int EIGHTS = (ACROSS ? SIDE : KS) / 8;                     // of a row
  static constexpr int CHUNKS = ROWS * EIGHTS / 256;                          // a thread stages so many pieces of eight values
  static_assert(ROWS * EIGHTS % 256 == 0, "whole rounds");
  __device__ static int row(int c) { return (threadIdx.x + 256 * c) / EIGHTS; }
  __device__ static int col(int c) { return (threadIdx.x + 256 * c) % EIGHTS * 8; }
  __device__ static int at(int c) { return row(c) * ROW + col(c) * 2; }
  // operand of 32 rows from `side` on, contraction indices 16 s ..
  __device__ static uint4 operand(const char* plane, int side, int s) {
    const int lane = threadIdx.x & 63, hh = lane >> 5;
    if (!ACROSS) return *reinterpret_cast<const uint4*>(plane + (side + (lane & 31)) * ROW + (16 * s + 8 * hh) * 2);
    typedef short s4 __attribute__((ext_vector_type(4)));
    typedef __attribute__((address_space(3))) s4* lp;
    const char* p = plane + (16 * s + 8 * hh + ((lane & 15) >> 2)) * ROW + (side + (lane & 16) + 4 * (lane & 3)) * 2;
    const uint2 u = __builtin_bit_cast(uint2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lp)p));
    const uint2 v = __builtin_bit_cast(uint2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lp)(p + 4 * ROW)));
    return make_uint4(u.x, u.y, v.x, v.y);
  }
};

enum GlKind { GL_FORWARD, GL_INPUT, GL_WEIGHTS };      // y = x W^T + b;  dx = dy W;  dW = dy^T x, db

template <class T>
struct GlArgs {
  GlRows rows;
  const T *a, *b;                 // GL_FORWARD: x, W;  GL_INPUT: dy, W;  GL_WEIGHTS: dy, x
  long a_stride, b_stride;
  int I, J, K;                    // result columns n of the output (GL_WEIGHTS: n_out x n_in); K: contraction (unused by GL_WEIGHTS)
  T* y;
  long y_stride;
  const float* bias;
  float *dW, *db;                 // GL_WEIGHTS: per slot [I][J] and [I]
  int tiles_j;                    // column tiles
  long chunk;                     // GL_WEIGHTS: rows of a slot at most
};

// Result j of row `row` of y or dx, and value (i, j) of dW over the rows r0 .. r1 - 1
template <GlKind KIND>
__device__ __forceinline__ float gl_again_row(const GlArgs<float>& g, int group, long row, int j) {
  const float* W = g.b + (size_t)group * g.J * g.K;
  const float* a = g.a + row * g.a_stride;
  if (KIND == GL_INPUT) return gl_again(a, 1, W + j, g.J, g.K);
  return gl_again(a, 1, W + (size_t)j * g.K, 1, g.K) + (g.bias ? g.bias[(size_t)group * g.J + j] : 0.0f);
}
__device__ __forceinline__ float gl_again_weight(const GlArgs<float>& g, long r0, long r1, int i, int j) {
  float sum = 0.0f;
  for (long r = r0; r < r1 && sum == sum; ++r) {
    const long row = gl_row(g.rows, r);
    sum = __builtin_fmaf(g.a[row * g.a_stride + i], g.b[row * g.b_stride + j], sum);
  }
  return sum;
}

// Tile `t` of the rows: group and first row; false past the end.  The tiles of a group start at its first row.
__device__ __forceinline__ bool gl_find(const GlRows& p, long t, int size, int& group, long& r0, long& r1) {
  __shared__ long s_sum[4], s_found[3];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  if (tid == 0) s_found[0] = -1;
  for (int g0 = 0; g0 < p.G; g0 += 256) {
    const int g = g0 + tid;
    long b = 0, e = 0;
    if (g < p.G) {
      b = gl_begin(p, g);
      e = gl_begin(p, g + 1);
    }
    const long mine = e > b ? (e - b + size - 1) / size : 0;
    long sum = mine;
    for (int h = 1; h < 64; h <<= 1) {
      const long v = __shfl_up(sum, h);
      if (lane >= h) sum += v;
    }
    __syncthreads();
    if (lane == 63) s_sum[wave] = sum;
    __syncthreads();
    long before = 0, all = 0;
    for (int w = 0; w < 4; ++w) {
      before += w < wave ? s_sum[w] : 0;
      all += s_sum[w];
    }
    if (t < all) {
      const long first = before + sum - mine;
      if (t >= first && t < first + mine) {
        s_found[0] = g;
        s_found[1] = b + (t - first) * size;
        s_found[2] = min(b + (t - first + 1) * size, e);
      }
      __syncthreads();
      break;
    }
    t -= all;
  }
  if (s_found[0] < 0) return false;
  group = (int)s_found[0];
  r0 = s_found[1];
  r1 = s_found[2];
  return true;
}

// Slot `t` of the rows cut into equal chunks: chunk c and group g that share rows own slot c + g (either goes up by one from slot to slot, so
// no two pairs share one).  With one chunk the slot is the group.
__device__ __forceinline__ bool gl_slot(const GlRows& p, long chunk, int t, int& group, long& r0, long& r1) {
  int lo = 0, hi = p.G - 1;                       // the last group whose first slot is not behind t
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (gl_begin(p, mid) / chunk + mid <= t) lo = mid; else hi = mid - 1;
  }
  group = lo;
  const long b = gl_begin(p, lo), e = gl_begin(p, lo + 1), c = t - lo;
  r0 = max(b, c * chunk);
  r1 = min(e, (c + 1) * chunk);
  return c >= 0 && r0 < r1;
}

// Units (group, tile of its weight gradient) of one XCD where every slot is a group: consecutive ones, so that the tiles of a group share
// its rows in one L2, and so many that each XCD gets an eighth of the rows to be read (groups may differ in size by any factor).
// 256 threads; returns the units first .. last - 1.
__device__ __forceinline__ void gl_units(const GlRows& p, int tiles, int xcd, long& first, long& last) {
  constexpr long LEAST = 64;                      // a unit costs as much as so many rows, whatever its rows
  __shared__ long s_sum[4], s_unit[2];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  long total = (long)p.G * LEAST;
  {
    long rows = 0;
    for (int g = tid; g < p.G; g += 256) rows += max(gl_begin(p, g + 1) - gl_begin(p, g), 0l);
    for (int h = 32; h; h >>= 1) rows += __shfl_xor(rows, h);
    if (lane == 0) s_sum[wave] = rows;
    if (tid < 2) s_unit[tid] = (long)p.G * tiles;
    __syncthreads();
    total += s_sum[0] + s_sum[1] + s_sum[2] + s_sum[3];
  }
  long before = 0;
  for (int g0 = 0; g0 < p.G; g0 += 256) {
    const int g = g0 + tid;
    const long mine = g < p.G ? max(gl_begin(p, g + 1) - gl_begin(p, g), 0l) + LEAST : 0;
    long sum = mine;
    for (int h = 1; h < 64; h <<= 1) {
      const long v = __shfl_up(sum, h);
      if (lane >= h) sum += v;
    }
    __syncthreads();
    if (lane == 63) s_sum[wave] = sum;
    __syncthreads();
    long start = before + sum - mine;
    for (int w = 0; w < wave; ++w) start += s_sum[w];
    for (int x = 0; x < 2; ++x) {                 // the first unit whose work begins at or behind the XCD's share
      const long at = total * (xcd + x) / 8;
      if (mine && at >= start && at < start + mine) s_unit[x] = (long)g * tiles + ((at - start) * tiles + mine - 1) / mine;
    }
    before += s_sum[0] + s_sum[1] + s_sum[2] + s_sum[3];
  }
  __syncthreads();
  first = s_unit[0];
  last = xcd == 7 ? (long)p.G * tiles : s_unit[1];
}

// Measured: 20,000 rows 512 to 1,024 in 16 ragged groups, bf16, 21 GFLOP each: forward 54 us, dx 48, dW 64 (330 to 440 TFLOP/s; a tile has 8 to
// 16 turns, so that its start and end count as much as its products; LDS busy 37 %, without conflicts).
// 256 threads, four waves, each a quarter of the BM x BN tile in 32 x 32 blocks.  Tiles go from memory to registers DEPTH turns ahead, are cut
// into pieces on the way to one of two LDS buffers, and are contracted from the other.
// NARROW: a side that is read along has fewer than eight values.
constexpr int GL_PIECE = 2048;     // GL_WEIGHTS: row numbers kept in LDS (a row number loaded in turn would have to wait for the rows before it)
template <class T, GlKind KIND, int BM, int BN, int KS, bool NARROW>
__device__ __forceinline__ void gl_tile(const GlArgs<T>& g, long tile, char* smem) {
  constexpr int NP = GlType<T>::PIECES, MB = BM / 64, NB = BN / 64;
  typedef typename GlType<T>::Raw Raw;
  typedef GlTile<BM, KS, KIND == GL_WEIGHTS> TA;
  typedef GlTile<BN, KS, KIND != GL_FORWARD> TB;
  constexpr int STAGE = NP * (TA::PLANE + TB::PLANE);
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int r32 = lane & 31, hh = lane >> 5;

  int group;
  long r0, r1;
  const long rt = tile / g.tiles_j;
  const int ct = (int)(tile - rt * g.tiles_j);
  int i0 = 0, j0 = ct * BN;
  if (KIND == GL_WEIGHTS) {
    const int across = g.dW ? (g.J + BN - 1) / BN : 1;
    i0 = ct / across * BM;
    j0 = ct % across * BN;
    const bool there = rt < 0x7fffffff && gl_slot(g.rows, g.chunk, (int)rt, group, r0, r1);
    if (!there && (g.chunk < g.rows.n || rt >= g.rows.G)) return;
    if (!there) r0 = r1 = 0;                          // one chunk: a group without rows gets its zeros here
  } else if (!gl_find(g.rows, rt, BM, group, r0, r1)) {
    return;
  }

  // What this thread stages.  Rows of the result past its end, and columns past its last, may hold anything (the last ones again): they do
  // not reach others.  Only contraction indices past the end have to be zero, in both operands: they end in the last turn.
  const int turns = (int)(KIND == GL_WEIGHTS ? (r1 - r0 + KS - 1) / KS : (g.K + KS - 1) / KS);
  constexpr int DEPTH = KIND == GL_WEIGHTS ? 3 : 2;
  const T *pa[TA::CHUNKS], *pb[TB::CHUNKS];           // row, or column for rows that change with the turn
  int da[TA::CHUNKS], db[TB::CHUNKS];                 // across: places the columns are moved down at the end of a row
  bool edge_a = false, edge_b = false;
  __shared__ int s_rows[KIND == GL_WEIGHTS ? GL_PIECE : 1];
  const T* const W = KIND == GL_WEIGHTS ? nullptr : g.b + (long)group * g.J * g.K;
  if (turns > 0) {
#pragma unroll
    for (int c = 0; c < TA::CHUNKS; ++c) {
      if (KIND == GL_WEIGHTS) {
        const int col = i0 + TA::col(c), from = NARROW ? col : min(col, g.I - 8);
        pa[c] = g.a + min(from, g.I - 1);
        da[c] = col - from;
      } else {
        pa[c] = g.a + gl_row(g.rows, min(r0 + TA::row(c), r1 - 1)) * g.a_stride;
      }
    }
#pragma unroll
    for (int c = 0; c < TB::CHUNKS; ++c) {
      const int col = j0 + TB::col(c), from = NARROW ? col : min(col, g.J - 8);
      if (KIND == GL_FORWARD) {                       // W[j][k]
        pb[c] = W + (long)min(j0 + TB::row(c), g.J - 1) * g.K;
      } else {                                        // W[k][j], x[r][j]
        pb[c] = (KIND == GL_INPUT ? W : g.b) + min(from, g.J - 1);
        db[c] = col - from;
      }
    }
    edge_a = KIND == GL_WEIGHTS && i0 + BM > g.I && !NARROW;
    edge_b = KIND != GL_FORWARD && j0 + BN > g.J && !NARROW;
  }
  Raw a[DEPTH][TA::CHUNKS], b[DEPTH][TB::CHUNKS];
  long piece = r0;                                    // GL_WEIGHTS: first row in s_rows
  auto row_of = [&](int turn, int at) -> long { return s_rows[min((int)(r0 - piece) + turn * KS + at, min(GL_PIECE, (int)(r1 - piece)) - 1)]; };
  auto fetch = [&](int turn, int to) {
#pragma unroll
    for (int c = 0; c < TA::CHUNKS; ++c) {
      const int k = turn * KS + TA::col(c);
      const T* p = pa[c] + (KIND == GL_WEIGHTS ? row_of(turn, TA::row(c)) * g.a_stride : (long)min(k, NARROW ? g.K - 1 : g.K - 8));
      if (NARROW) gl_load_narrow(p, KIND == GL_WEIGHTS ? g.I - i0 - TA::col(c) : g.K - k, a[to][c]);
      else gl_load(p, a[to][c]);
    }
#pragma unroll
    for (int c = 0; c < TB::CHUNKS; ++c) {
      const int k = turn * KS + (KIND == GL_FORWARD ? TB::col(c) : TB::row(c));
      const T* p = pb[c] + (KIND == GL_WEIGHTS ? row_of(turn, TB::row(c)) * g.b_stride
                            : KIND == GL_INPUT ? (long)min(k, g.K - 1) * g.J : (long)min(k, NARROW ? g.K - 1 : g.K - 8));
      if (NARROW) gl_load_narrow(p, KIND == GL_FORWARD ? g.K - k : g.J - j0 - TB::col(c), b[to][c]);
      else gl_load(p, b[to][c]);
    }
  };
  float turn_sum[8];
  double col_sum[8] = {};
  const bool sums = KIND == GL_WEIGHTS && g.db && j0 == 0;
  auto stage = [&](int turn, int at) {
    char* to = smem + (turn & 1) * STAGE;
    const bool last = turn + 1 == turns;
    const long left = (KIND == GL_WEIGHTS ? r1 - r0 : (long)g.K) - (long)turn * KS;      // contraction indices from this turn on
    if (KIND == GL_WEIGHTS && edge_a) {
#pragma unroll
      for (int c = 0; c < TA::CHUNKS; ++c) gl_shift(a[at][c], da[c]);
    }
    if (KIND != GL_FORWARD && edge_b) {
#pragma unroll
      for (int c = 0; c < TB::CHUNKS; ++c) gl_shift(b[at][c], db[c]);
    }
    if (last && left < KS) {
#pragma unroll
      for (int c = 0; c < TA::CHUNKS; ++c) {
        if (KIND == GL_WEIGHTS) gl_shift(a[at][c], TA::row(c) < left ? 0 : 8);
        else if (!NARROW) gl_shift(a[at][c], max(0, TA::col(c) + 8 - (int)left));
      }
#pragma unroll
      for (int c = 0; c < TB::CHUNKS; ++c) {
        if (KIND != GL_FORWARD) gl_shift(b[at][c], TB::row(c) < left ? 0 : 8);
        else if (!NARROW) gl_shift(b[at][c], max(0, TB::col(c) + 8 - (int)left));
      }
    }
#pragma unroll
    for (int q = 0; q < 8; ++q) turn_sum[q] = 0.0f;
#pragma unroll
    for (int c = 0; c < TA::CHUNKS; ++c) {
      uint4 v[NP];
      gl_cut(a[at][c], v);
      if (sums) gl_add<T>(a[at][c], turn_sum);
#pragma unroll
      for (int q = 0; q < NP; ++q) *reinterpret_cast<uint4*>(to + q * TA::PLANE + TA::at(c)) = v[q];
    }
#pragma unroll
    for (int c = 0; c < TB::CHUNKS; ++c) {
      uint4 v[NP];
      gl_cut(b[at][c], v);
#pragma unroll
      for (int q = 0; q < NP; ++q) *reinterpret_cast<uint4*>(to + NP * TA::PLANE + q * TB::PLANE + TB::at(c)) = v[q];
    }
    if (sums)
#pragma unroll
      for (int q = 0; q < 8; ++q) col_sum[q] += (double)turn_sum[q];
  };

  GlSum<T> total[MB][NB];
  const int wi = (wave >> 1) * (BM / 2), wj = (wave & 1) * (BN / 2);
  auto contract = [&](int k) {
    rb_release_barrier();        // (only LDS is waited for: the next turns' loads stay under way)
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "workgroup", "local");
    const char* from = smem + (k & 1) * STAGE;
#pragma unroll
    for (int s = 0; s < KS / 16; ++s) {
      uint4 fa[MB][NP], fb[NB][NP];
#pragma unroll
      for (int x = 0; x < MB; ++x)
#pragma unroll
        for (int q = 0; q < NP; ++q) fa[x][q] = TA::operand(from + q * TA::PLANE, wi + 32 * x, s);
#pragma unroll
      for (int y = 0; y < NB; ++y)
#pragma unroll
        for (int q = 0; q < NP; ++q) fb[y][q] = TB::operand(from + NP * TA::PLANE + q * TB::PLANE, wj + 32 * y, s);
#pragma unroll
      for (int x = 0; x < MB; ++x)
#pragma unroll
        for (int y = 0; y < NB; ++y) total[x][y].add(fa[x], fb[y]);
    }
  };
  // turns k0 .. k1 - 1; their number of loads under way is the same in every turn of the first loop
  auto run = [&](int k0, int k1) {
#pragma unroll
    for (int d = 0; d < DEPTH; ++d) fetch(min(k0 + d, k1 - 1), d);
    stage(k0, 0);
    fetch(min(k0 + DEPTH, k1 - 1), 0);
    int k = k0;
    for (; k + 2 * DEPTH < k1; k += DEPTH)
#pragma unroll
      for (int d = 0; d < DEPTH; ++d) {
        contract(k + d);
        stage(k + d + 1, (d + 1) % DEPTH);
        fetch(k + d + 1 + DEPTH, (d + 1) % DEPTH);
      }
#pragma unroll
    for (int d = 0; d < 2 * DEPTH; ++d)
      if (k + d < k1) {
        contract(k + d);
        if (k + d + 1 < k1) {
          stage(k + d + 1, (d + 1) % DEPTH);
          if (d + 1 < DEPTH && k + d + 1 + DEPTH < k1) fetch(k + d + 1 + DEPTH, (d + 1) % DEPTH);
        }
      }
  };
  if (KIND == GL_WEIGHTS) {
    for (int k = 0; k < turns; k += GL_PIECE / KS) {
      piece = r0 + (long)k * KS;
      __syncthreads();
      for (int i = tid; i < GL_PIECE; i += 256) s_rows[i] = (int)gl_row(g.rows, min(piece + i, r1 - 1));
      __syncthreads();
      run(k, min(turns, k + GL_PIECE / KS));
    }
  } else {
    run(0, turns);
  }

  // a lane holds column j = lane & 31 of its blocks and four times four neighbouring rows i
  gl_f16v acc[MB][NB];
#pragma unroll
  for (int x = 0; x < MB; ++x)
#pragma unroll
    for (int y = 0; y < NB; ++y) acc[x][y] = total[x][y].value();
  if (KIND == GL_WEIGHTS) {
    float* to = g.dW ? g.dW + (size_t)rt * g.I * g.J : nullptr;
#pragma unroll
    for (int x = 0; x < MB; ++x)
#pragma unroll
      for (int y = 0; y < NB; ++y)
#pragma unroll
        for (int q = 0; q < 16; ++q) {
          const int i = i0 + wi + 32 * x + 8 * (q >> 2) + 4 * hh + (q & 3), j = j0 + wj + 32 * y + r32;
          if (to && i < g.I && j < g.J) to[(size_t)i * g.J + j] = acc[x][y][q];
        }
    if constexpr (NP == 3) {
      bool again = false;
#pragma unroll
      for (int x = 0; x < MB; ++x)
#pragma unroll
        for (int y = 0; y < NB; ++y)
#pragma unroll
          for (int q = 0; q < 16; ++q) again |= acc[x][y][q] != acc[x][y][q];
      if (to && again)
#pragma unroll 1
        for (int k = 0; k < MB * NB * 16; ++k) {
          const int x = k / (16 * NB), y = k / 16 % NB, q = k & 15;
          const int i = i0 + wi + 32 * x + 8 * (q >> 2) + 4 * hh + (q & 3), j = j0 + wj + 32 * y + r32;
          if (i >= g.I || j >= g.J) continue;
          float* at = to + (size_t)i * g.J + j;
          if (*at != *at) *at = gl_again_weight(g, r0, r1, i, j);
        }
    }
    if (sums) {                  // the threads of a column of pieces
      __syncthreads();
      double* s = reinterpret_cast<double*>(smem);
      constexpr int E = TA::EIGHTS, R = 256 / E;
#pragma unroll
      for (int q = 0; q < 8; ++q) s[(tid / E) * BM + tid % E * 8 + q] = col_sum[q];
      __syncthreads();
      if (tid < BM && i0 + tid < g.I) {
        double t = 0.0;
        for (int r = 0; r < R; ++r) t += s[r * BM + tid];
        g.db[(size_t)rt * g.I + i0 + tid] = (float)t;
      }
    }
    return;
  }
  // Rows of results go through LDS, to be written eight values a thread.  Whatever has to be loaded is loaded before the first of them is
  // stored: loads and stores return in order, and a load behind a store would wait for it.
  constexpr int LD = BN + 4, ACROSS = BN / 8, ITEMS = BM * ACROSS / 256;
  const int jl = tid % ACROSS * 8, j = j0 + jl, valid = g.J - j;
  long row[ITEMS];
  float bias[8];
#pragma unroll
  for (int e = 0; e < ITEMS; ++e) row[e] = gl_row(g.rows, min(r0 + tid / ACROSS + e * (256 / ACROSS), r1 - 1));
#pragma unroll
  for (int q = 0; q < 8; ++q) bias[q] = KIND == GL_FORWARD && g.bias ? g.bias[(size_t)group * g.J + min(j + q, g.J - 1)] : 0.0f;
  rb_release_barrier();
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "workgroup", "local");
  float* tile_out = reinterpret_cast<float*>(smem);
#pragma unroll
  for (int x = 0; x < MB; ++x)
#pragma unroll
    for (int y = 0; y < NB; ++y)
#pragma unroll
      for (int q = 0; q < 16; ++q) tile_out[(wi + 32 * x + 8 * (q >> 2) + 4 * hh + (q & 3)) * LD + wj + 32 * y + r32] = acc[x][y][q];
  rb_release_barrier();
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "workgroup", "local");
  const bool wide = ((uintptr_t)g.y | (g.y_stride * sizeof(T))) % 16 == 0;
#pragma unroll
  for (int e = 0; e < ITEMS; ++e) {
    const int i = tid / ACROSS + e * (256 / ACROSS);
    float v[8];
    *reinterpret_cast<float4*>(v) = *reinterpret_cast<const float4*>(tile_out + i * LD + jl);
    *reinterpret_cast<float4*>(v + 4) = *reinterpret_cast<const float4*>(tile_out + i * LD + jl + 4);
#pragma unroll
    for (int q = 0; q < 8; ++q) v[q] += bias[q];
    if (r0 + i >= r1 || valid <= 0) continue;
    T* to = g.y + row[e] * g.y_stride + j;
    if (wide && valid >= 8) {
      rt_store<T, 8>(to, v);
    } else {
#pragma unroll
      for (int q = 0; q < 8; ++q)
        if (q < valid) to[q] = (T)v[q];
    }
    if constexpr (NP == 3) {
      bool again = false;
#pragma unroll
      for (int q = 0; q < 8; ++q) again |= v[q] != v[q];
      if (again)
#pragma unroll 1
        for (int q = 0; q < min(8, valid); ++q)
          if (to[q] != to[q]) to[q] = gl_again_row<KIND>(g, group, row[e], j + q);
    }
  }
}

// Neighbouring tiles to the same XCD (workgroups go round the eight of them in turn), the columns of a tile of rows one after the other.
template <class T, GlKind KIND, int BM, int BN, int KS, bool NARROW>
__global__ __launch_bounds__(256) void gl_tile_kernel(GlArgs<T> g) {
  extern __shared__ __align__(16) char smem[];
  const long per = gridDim.x >> 3, place = blockIdx.x >> 3;
  if (KIND == GL_WEIGHTS && g.chunk >= g.rows.n) {
    long tile, end;
    gl_units(g.rows, g.tiles_j, blockIdx.x & 7, tile, end);
    for (tile += place; tile < end; tile += per) {
      gl_tile<T, KIND, BM, BN, KS, NARROW>(g, tile, smem);
      __syncthreads();
    }
  } else {
    gl_tile<T, KIND, BM, BN, KS, NARROW>(g, (blockIdx.x & 7) * per + place, smem);
  }
}

// ---- n_in and n_out of at most 64: the group's matrix stays in registers ------------------------------------------------------
// A wave takes an equal share of the rows, group by group, 32 at a time, and nothing is shared between waves: no LDS tile, no barrier.  The
// product is y^T = W x^T, so that a lane holds one row and writes its values four neighbouring ones at a time.  The next rows are under way
// while the matrix cores work on these: 300,000 rows of 64 fp32 by 15 groups take 46 us forward (154 MB, 3.3 TB/s), 56 with the
// transposed matrices of dx.  At 64 x 64 the three pieces of an fp32 matrix are 192 registers and do not all stay: 22 values a lane are spilled
// forward and 48 for dx (none of the 16-bit types, none at 32 x 32): half the rate of a copy.
// KB: contraction steps of 16, NB: output blocks of 32; 16 KB >= K, 32 NB >= J.
template <class T, GlKind KIND, int KB, int NB, bool NARROW>
__global__ __launch_bounds__(256, 2) void gl_lean_rows_kernel(GlArgs<T> g, long share) {
  constexpr int NP = GlType<T>::PIECES;
  typedef typename GlType<T>::Raw Raw;
  __shared__ __align__(16) float s_bias[4][32 * NB];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), r32 = lane & 31, hh = lane >> 5;
  const long first = ((long)blockIdx.x * 4 + wave) * share, end = min(first + share, g.rows.n);
  int lo = 0, hi = g.rows.G - 1;                     // the last group that does not begin behind the first row
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (gl_begin(g.rows, mid) <= first) lo = mid; else hi = mid - 1;
  }
  auto raw = [&](const T* row, int s, Raw& to) {      // eight values of a row from 16 s + 8 hh on, the row's last ones past its end
    const int k = 16 * s + 8 * hh;
    if (NARROW) gl_load_narrow(row + min(k, g.K - 1), g.K - k, to);
    else gl_load(row + min(k, g.K - 8), to);
  };
  auto edge = [&](int s, Raw& r) {
    if (!NARROW && 16 * KB > g.K) gl_shift(r, max(0, 16 * s + 8 * hh + 8 - g.K));
  };
  const bool wide = ((uintptr_t)g.y | (g.y_stride * sizeof(T))) % (4 * sizeof(T)) == 0;
  for (int group = lo; group < g.rows.G; ++group) {
    const long b = max(gl_begin(g.rows, group), first), e = min(gl_begin(g.rows, group + 1), end);
    if (b >= end) break;
    if (b >= e) continue;
    // rows of the next tile first: their way to memory passes while the matrix is prepared
    auto row_at = [&](long r) { return gl_row(g.rows, min(r + r32, e - 1)); };
    long here = row_at(b), next = row_at(b + 32);
    Raw x[KB];
#pragma unroll
    for (int s = 0; s < KB; ++s) raw(g.a + here * g.a_stride, s, x[s]);
    uint4 w[KB][NB][NP];
    const T* W = g.b + (size_t)group * g.J * g.K;
#pragma unroll
    for (int n = 0; n < NB; ++n) {
      const int j = 32 * n + r32;
#pragma unroll
      for (int s = 0; s < KB; ++s) {
        Raw r;
        if (KIND == GL_FORWARD) {                     // W[j][k]
          raw(W + (size_t)min(j, g.J - 1) * g.K, s, r);
          edge(s, r);
        } else {                                      // W[k][j]
          T v[8];
#pragma unroll
          for (int q = 0; q < 8; ++q) {
            const int k = 16 * s + 8 * hh + q;
            v[q] = W[(size_t)min(k, g.K - 1) * g.J + min(j, g.J - 1)];
            if (k >= g.K) v[q] = (T)0.0f;
          }
          __builtin_memcpy(&r, v, sizeof(Raw));
        }
        gl_cut(r, w[s][n]);
      }
    }
    if (KIND == GL_FORWARD) {
      if (lane < 32 * NB) s_bias[wave][lane] = g.bias ? g.bias[(size_t)group * g.J + min(lane, g.J - 1)] : 0.0f;
      __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront", "local");
      __builtin_amdgcn_wave_barrier();
      __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront", "local");
    }
    for (long r = b; r < e; r += 32) {
      uint4 v[KB][NP];
#pragma unroll
      for (int s = 0; s < KB; ++s) {
        edge(s, x[s]);
        gl_cut(x[s], v[s]);
      }
      const long mine = here;
      here = next;
      if (r + 32 < e) {
#pragma unroll
        for (int s = 0; s < KB; ++s) raw(g.a + here * g.a_stride, s, x[s]);
        next = row_at(r + 64);
      }
      gl_f16v acc[NB];
#pragma unroll
      for (int n = 0; n < NB; ++n)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          float4 t = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
          if (KIND == GL_FORWARD) t = *reinterpret_cast<const float4*>(&s_bias[wave][32 * n + 8 * i + 4 * hh]);
          acc[n][4 * i] = t.x; acc[n][4 * i + 1] = t.y; acc[n][4 * i + 2] = t.z; acc[n][4 * i + 3] = t.w;
        }
#pragma unroll
      for (int s = 0; s < KB; ++s)
#pragma unroll
        for (int n = 0; n < NB; ++n) acc[n] = gl_product<T>(w[s][n], v[s], acc[n]);
      if (r + r32 < e) {
        T* to = g.y + mine * g.y_stride;
#pragma unroll
        for (int n = 0; n < NB; ++n)
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const int j = 32 * n + 8 * i + 4 * hh;
            const float t[4] = {acc[n][4 * i], acc[n][4 * i + 1], acc[n][4 * i + 2], acc[n][4 * i + 3]};
            if (wide && j + 4 <= g.J) {
              rt_store<T, 4>(to + j, t);
            } else {
#pragma unroll
              for (int q = 0; q < 4; ++q)
                if (j + q < g.J) to[j + q] = (T)t[q];
            }
          }
        if constexpr (NP == 3) {
          bool again = false;
#pragma unroll
          for (int n = 0; n < NB; ++n)
#pragma unroll
            for (int i = 0; i < 16; ++i) again |= acc[n][i] != acc[n][i];
          if (again)
#pragma unroll 1
            for (int k = 0; k < NB * 16; ++k) {
              const int j = 8 * (k >> 2) + 4 * hh + (k & 3);
              if (j < g.J && to[j] != to[j]) to[j] = gl_again_row<KIND>(g, group, mine, j);
            }
        }
      }
    }
  }
}

// dW and db of a slot: each wave its own sixteen rows in turn, operands straight from memory (lane = column, eight rows), the waves' sums
// joined at the end (300,000 rows of 64 and 64 fp32: 51 us for 154 MB, and 6 to join the slots; its 248 registers allow 512 workgroups at a time,
// and the 767 slots take one and a half rounds).  MB, NB: blocks of 32 outputs and inputs.
template <class T, int MB, int NB>
__global__ __launch_bounds__(256, 2) void gl_lean_weights_kernel(GlArgs<T> g) {
  constexpr int NP = GlType<T>::PIECES, PART = MB * NB * 1024;
  typedef typename GlType<T>::Raw Raw;
  __shared__ float s_part[4][PART / 2];
  __shared__ double s_db[8][32 * MB];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), r32 = lane & 31, hh = lane >> 5;
  int group;
  long r0, r1;
  const int slot = blockIdx.x;
  const bool there = gl_slot(g.rows, g.chunk, slot, group, r0, r1);
  if (!there && (g.chunk < g.rows.n || slot >= g.rows.G)) return;
  if (!there) r0 = r1 = 0;                             // one chunk: a group without rows gets its zeros here
  GlSum<T> total[MB][NB];
  double col_sum[MB] = {};
  int ci[MB], cj[NB];
#pragma unroll
  for (int m = 0; m < MB; ++m) ci[m] = min(32 * m + r32, g.I - 1);
#pragma unroll
  for (int n = 0; n < NB; ++n) cj[n] = min(32 * n + r32, g.J - 1);
  T d[MB][8], x[NB][8];
  long row = 0;                                        // lane i of sixteen: row i of the unit to be fetched next
  auto rows_of = [&](long u) { return gl_row(g.rows, min(u + (lane & 15), r1 - 1)); };
  auto fetch = [&]() {
#pragma unroll
    for (int q = 0; q < 8; ++q) {
      const long r = __shfl(row, 8 * hh + q);
      const T* pd = g.a + r * g.a_stride;
      const T* px = g.b + r * g.b_stride;
#pragma unroll
      for (int m = 0; m < MB; ++m) d[m][q] = pd[ci[m]];
#pragma unroll
      for (int n = 0; n < NB; ++n) x[n][q] = g.dW ? px[cj[n]] : (T)0.0f;
    }
  };
  const long u0 = r0 + 16 * wave;
  if (u0 < r1) {
    row = rows_of(u0);
    fetch();
    row = rows_of(u0 + 64);
  }
  for (long u = u0; u < r1; u += 64) {
    uint4 a[MB][NP], b[NB][NP];
    const bool cut_off = u + 16 > r1;
#pragma unroll
    for (int m = 0; m < MB; ++m) {
      if (cut_off)
#pragma unroll
        for (int q = 0; q < 8; ++q)
          if (u + 8 * hh + q >= r1) d[m][q] = (T)0.0f;
      float t = 0.0f;
#pragma unroll
      for (int q = 0; q < 8; ++q) t += (float)d[m][q];
      col_sum[m] += (double)t;
      Raw r;
      __builtin_memcpy(&r, d[m], sizeof(Raw));
      gl_cut(r, a[m]);
    }
#pragma unroll
    for (int n = 0; n < NB; ++n) {
      if (cut_off)
#pragma unroll
        for (int q = 0; q < 8; ++q)
          if (u + 8 * hh + q >= r1) x[n][q] = (T)0.0f;
      Raw r;
      __builtin_memcpy(&r, x[n], sizeof(Raw));
      gl_cut(r, b[n]);
    }
    if (u + 64 < r1) {
      fetch();
      row = rows_of(u + 128);
    }
#pragma unroll
    for (int m = 0; m < MB; ++m)
#pragma unroll
      for (int n = 0; n < NB; ++n) total[m][n].add(a[m], b[n]);
  }
  if (g.db) {
#pragma unroll
    for (int m = 0; m < MB; ++m) s_db[wave * 2 + hh][32 * m + r32] = col_sum[m];
    __syncthreads();
    if (tid < g.I) {
      double t = 0.0;
      for (int i = 0; i < 8; ++i) t += s_db[i][tid];
      g.db[(size_t)slot * g.I + tid] = (float)t;
    }
  }
  if (!g.dW) return;
  gl_f16v acc[MB][NB];
#pragma unroll
  for (int m = 0; m < MB; ++m)
#pragma unroll
    for (int n = 0; n < NB; ++n) acc[m][n] = total[m][n].value();
  // half of the values at a time: [register][lane] of every wave
#pragma unroll
  for (int half = 0; half < 2; ++half) {
    __syncthreads();
#pragma unroll
    for (int m = 0; m < MB; ++m)
#pragma unroll
      for (int n = 0; n < NB; ++n)
#pragma unroll
        for (int q = 0; q < 8; ++q) s_part[wave][((m * NB + n) * 8 + q) * 64 + lane] = acc[m][n][8 * half + q];
    __syncthreads();
    for (int e = tid; e < PART / 2; e += 256) {
      const int l = e & 63, q = (e >> 6) & 7, n = (e >> 9) % NB, m = (e >> 9) / NB;
      const int i = 32 * m + 8 * (2 * half + (q >> 2)) + 4 * (l >> 5) + (q & 3), j = 32 * n + (l & 31);
      if (i >= g.I || j >= g.J) continue;
      float sum = (s_part[0][e] + s_part[1][e]) + (s_part[2][e] + s_part[3][e]);
      if constexpr (NP == 3)
        if (sum != sum) sum = gl_again_weight(g, r0, r1, i, j);
      g.dW[((size_t)slot * g.I + i) * g.J + j] = sum;
    }
  }
}

// Sums of the slots of every group, n values a slot for dW and m for db behind them: sixteen values a workgroup, sixteen slots at a time.
__global__ __launch_bounds__(256) void gl_join_kernel(GlRows p, long chunk, const float* dW_part, const float* db_part, float* dW, float* db,
                                                      long n, long m) {
  __shared__ float s[16][68];
  const int g = blockIdx.y, k = threadIdx.x >> 4;
  const long n4 = dW ? (n + 63) / 64 * 64 : 0;
  const long at = (long)blockIdx.x * 64 + (threadIdx.x & 15) * 4;
  const bool first = at < n4;
  const float* part = first ? dW_part : db_part;
  const long i = first ? at : at - n4, size = first ? n : m;
  const long b = gl_begin(p, g), e = gl_begin(p, g + 1);
  float t[4] = {};
  if (b < e)
#pragma unroll 4
    for (long c = b / chunk + k; c <= (e - 1) / chunk; c += 16)
#pragma unroll
      for (int q = 0; q < 4; ++q) t[q] += part[(size_t)(c + g) * size + min(i + q, size - 1)];
#pragma unroll
  for (int q = 0; q < 4; ++q) s[k][(threadIdx.x & 15) * 4 + q] = t[q];
  __syncthreads();
  if (threadIdx.x < 64) {
    const long v = (long)blockIdx.x * 64 + threadIdx.x, w = v < n4 ? v : v - n4;
    float sum = 0.0f;
    for (int r = 0; r < 16; ++r) sum += s[r][threadIdx.x];
    if (v < n4 && w < n) dW[(size_t)g * n + w] = sum;
    if (v >= n4 && w < m) db[(size_t)g * m + w] = sum;
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

size_t gl_align(size_t n) { return (n + 255) & ~(size_t)255; }

// Rows of one slot of the weight gradient: enough slots that the launch fills the compute units three times, of at least 256 rows
// (below that a slot's partial result is longer than what it reads).  Adjoint in us with one, three, six times: 20,000 rows 512 to 256 in 4
// groups bf16 77, 58, 50; 300,000 of 64 in 15 groups bf16 51, 47, 54, fp32 83, 88, 95; 50,000 of 128 in 15 fp32 64, 69, 80.  Three times is for
// the 16-bit types, where few groups of wide matrices need it most; fp32, which loses 5 to 8 % by it, follows the same rule, as the
// workspace is sized without the type.
struct GlSplit { long chunk; int slots; size_t weights, bytes; };
GlSplit gl_split(int64_t n, int G, int K, int N) {
  GlSplit s;
  const long tiles = (long)((N + 63) / 64) * ((K + 63) / 64);
  long chunks = (3 * EGNN_CUS + tiles - 1) / tiles - G;
  if (chunks > n / 256) chunks = n / 256;
  if (chunks < 1) chunks = 1;
  s.chunk = n ? (n + chunks - 1) / chunks : 1;
  s.slots = chunks > 1 ? (int)((n + s.chunk - 1) / s.chunk) + G : G;
  s.weights = gl_align((size_t)s.slots * N * K * sizeof(float));
  s.bytes = chunks > 1 ? s.weights + gl_align((size_t)s.slots * N * sizeof(float)) : 256;
  return s;
}

template <class T, GlKind KIND, int BM, int BN, int KS, bool NARROW = false>
int gl_launch(egnn_ctx* ctx, const GlArgs<T>& g, long tiles, hipStream_t st) {
  constexpr size_t stage = GlType<T>::PIECES * (GlTile<BM, KS, KIND == GL_WEIGHTS>::PLANE + GlTile<BN, KS, KIND != GL_FORWARD>::PLANE);
  constexpr size_t out = KIND == GL_WEIGHTS ? (size_t)256 * 8 * sizeof(double) : (size_t)BM * (BN + 4) * sizeof(float);
  constexpr size_t lds = 2 * stage > out ? 2 * stage : out;
  if (tiles > 0xfffff0) return egnn_fail(ctx, EGNN_EINVAL, "grouped_linear: more tiles than a launch holds");
  static bool ready[64];
  if (int rc = rt_allow_lds(ctx, (const void*)gl_tile_kernel<T, KIND, BM, BN, KS, NARROW>, lds, ready)) return rc;
  hipLaunchKernelGGL((gl_tile_kernel<T, KIND, BM, BN, KS, NARROW>), dim3((unsigned)((tiles + 7) / 8 * 8)), dim3(256), lds, st, g);
  EGNN_LAUNCH_CHECK(ctx, "grouped_linear");
  return EGNN_OK;
}

// Matrices of at most 32 x 32 (one register block) always go the lean way, those of at most 64 x 64 from GL_LEAN_ROWS rows on: with few rows
// the way to the first product counts (us forward + adjoint, lean against tiles, 15 groups of 64 x 64 in any order: 20,000 rows fp32 14 + 34 : 9 + 25,
// 80,000 24 + 48 : 18 + 48, 150,000 30 + 69 : 29 + 72, 300,000 42 + 96 : 52 + 109; bf16 40,000 10 + 26 : 8 + 19, 80,000 11 + 30 : 11 + 27,
// 150,000 16 + 38 : 16 + 40; 32 x 32: 40,000 fp32 8 + 19 : 9 + 27).  Around 80,000 to 150,000 rows the two are within a tenth of each other.
constexpr int GL_LEAN_ROWS = 80000;
bool gl_lean(int64_t n, int K, int N) { return K <= 64 && N <= 64 && ((K <= 32 && N <= 32) || K < 8 || N < 8 || n >= GL_LEAN_ROWS); }

// Tiles of 64 x 64, or of 128 x 128 for 16-bit values where there are enough of those for every compute unit: half the LDS traffic a product, but
// a quarter of the workgroups (us forward, 128 against 64: 2,000 rows 1,024 to 1,024 in 4 groups 14.6 : 15.8, 5,000 in 8 24.3 : 26.7,
// 20,000 512 to 1,024 in 16 42 : 49).  fp32 has six products a pair of operands and is not bound by LDS: 64 x 64 is faster at all sizes
// (128 x 64: 20,000 rows 512 to 1,024 221 : 190, 20,000 of 128 18.0 : 13.7).
template <class T, GlKind KIND>
int gl_rows(egnn_ctx* ctx, GlArgs<T> g, hipStream_t st) {
  constexpr int KS = GlType<T>::PIECES == 1 ? 64 : 32;
  auto tiles = [&](int side) {
    g.tiles_j = (g.J + side - 1) / side;
    return ((g.rows.n + side - 1) / side + g.rows.G) * (long)g.tiles_j;
  };
  if (gl_lean(g.rows.n, g.K, g.J)) {
    // 2,048 waves, two per SIMD, as long as each gets at least 32 rows (300,000 x 64 fp32: 42 us; 1,024 waves 44, 4,096 49)
    long share = (g.rows.n + 2047) / 2048;
    if (share < 32) share = 32;
    const unsigned grid = (unsigned)((g.rows.n + 4 * share - 1) / (4 * share));
    if (g.K < 8)
      hipLaunchKernelGGL((gl_lean_rows_kernel<T, KIND, 1, 2, true>), dim3(grid), dim3(256), 0, st, g, share);
    else if (g.J <= 32 && g.K <= 32)
      hipLaunchKernelGGL((gl_lean_rows_kernel<T, KIND, 2, 1, false>), dim3(grid), dim3(256), 0, st, g, share);
    else
      hipLaunchKernelGGL((gl_lean_rows_kernel<T, KIND, 4, 2, false>), dim3(grid), dim3(256), 0, st, g, share);
    EGNN_LAUNCH_CHECK(ctx, "grouped_linear");
    return EGNN_OK;
  }
  if (g.K < 8 || (KIND == GL_INPUT && g.J < 8)) return gl_launch<T, KIND, 64, 64, KS, true>(ctx, g, tiles(64), st);
  if constexpr (GlType<T>::PIECES == 1)
    if (g.J > 64 && tiles(128) >= EGNN_CUS) return gl_launch<T, KIND, 128, 128, KS>(ctx, g, tiles(128), st);
  return gl_launch<T, KIND, 64, 64, KS>(ctx, g, tiles(64), st);
}

template <class T>
int gl_forward(egnn_ctx* ctx, const GlRows& p, const void* x, int64_t xs, const void* W, const float* bias, int K, int N, void* y,
               int64_t ys, hipStream_t st) {
  GlArgs<T> g{p, (const T*)x, (const T*)W, xs, 0, 0, N, K, (T*)y, ys, bias, nullptr, nullptr, 0, 0};
  return gl_rows<T, GL_FORWARD>(ctx, g, st);
}

template <class T>
int gl_backward(egnn_ctx* ctx, const GlRows& p, const void* x, int64_t xs, const void* W, const void* dy, int64_t dys, int K, int N,
                void* dx, int64_t dxs, float* dW, float* db, void* ws, hipStream_t st) {
  if (dx && p.n) {
    GlArgs<T> g{p, (const T*)dy, (const T*)W, dys, 0, 0, K, N, (T*)dx, dxs, nullptr, nullptr, nullptr, 0, 0};
    if (int rc = gl_rows<T, GL_INPUT>(ctx, g, st)) return rc;
  }
  if (!dW && !db) return EGNN_OK;
  const GlSplit s = gl_split(p.n, p.G, K, N);
  const bool join = s.slots > p.G;
  float *pw = dW, *pb = db;
  if (join) {
    pw = dW ? (float*)ws : nullptr;
    pb = db ? (float*)((char*)ws + s.weights) : nullptr;
  }
  // (db alone: x may be NULL, and dy, whose rows have N values, takes its place in loads whose results nobody uses)
  GlArgs<T> g{p, (const T*)dy, (const T*)(dW ? x : dy), dys, dW ? xs : dys, N, dW ? K : N, 0, nullptr, 0, nullptr, pw, pb, 0, s.chunk};
  constexpr int KS = GlType<T>::PIECES == 1 ? 64 : 32;
  auto tiles = [&](int side) {
    g.tiles_j = ((N + side - 1) / side) * (dW ? (K + side - 1) / side : 1);      // db alone: the first column of tiles
    return (long)s.slots * g.tiles_j;
  };
  int rc = EGNN_OK;
  if (gl_lean(p.n, K, N)) {
    if (N <= 32 && K <= 32)
      hipLaunchKernelGGL((gl_lean_weights_kernel<T, 1, 1>), dim3(s.slots), dim3(256), 0, st, g);
    else
      hipLaunchKernelGGL((gl_lean_weights_kernel<T, 2, 2>), dim3(s.slots), dim3(256), 0, st, g);
    EGNN_LAUNCH_CHECK(ctx, "grouped_linear_backward");
  } else if (N < 8 || K < 8) {
    rc = gl_launch<T, GL_WEIGHTS, 64, 64, KS, true>(ctx, g, tiles(64), st);
  } else if (GlType<T>::PIECES == 1 && N > 64 && K > 64 && tiles(128) > EGNN_CUS) {
    // (as in gl_rows; half the contraction a turn, for three workgroups' worth of LDS: with 64 a turn 103 us instead of 64 at 20,000 rows)
    if constexpr (GlType<T>::PIECES == 1) rc = gl_launch<T, GL_WEIGHTS, 128, 128, KS / 2>(ctx, g, tiles(128), st);
  } else {
    rc = gl_launch<T, GL_WEIGHTS, 64, 64, KS>(ctx, g, tiles(64), st);
  }
  if (rc) return rc;
  if (join) {
    const long n = dW ? (long)N * K : 0, m = db ? N : 0;
    const long blocks = (n + 63) / 64 + (m + 63) / 64;
    hipLaunchKernelGGL(gl_join_kernel, dim3((unsigned)blocks, p.G), dim3(256), 0, st, p, s.chunk, pw, pb, dW, db, n, m);
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
  if (chunks > 1) hipLaunchKernelGGL(gr_count_kernel, dim3(chunks), dim3(GR_THREADS), 0, st, key, (long)n, n_groups, gr_chunk(n), (int*)ws);
  hipLaunchKernelGGL(gr_place_kernel, dim3(chunks), dim3(GR_THREADS), 0, st, key, (long)n, n_groups, lmax, gr_chunk(n),
                     chunks > 1 ? (const int*)ws : nullptr, ptr, perm);
  EGNN_LAUNCH_CHECK(ctx, "group_rows");
  return EGNN_OK;
}

extern "C" int egnn_grouped_linear_workspace_bytes(const egnn_ctx* ctx, int64_t n_rows, int32_t n_groups, int32_t n_in, int32_t n_out,
                                                   size_t* bytes) {
  if (!ctx || !bytes || n_rows < 0 || n_rows > 0x7fffffff || n_groups < 1 || n_groups > 65535 || n_in < 1 || n_in > 65536 || n_out < 1 ||
      n_out > 65536)
    return egnn_fail(const_cast<egnn_ctx*>(ctx), EGNN_EINVAL, "grouped_linear_workspace_bytes: bad argument");
  *bytes = gl_split(n_rows, n_groups, n_in, n_out).bytes;
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
  if ((dW && x_stride < n_in) || dy_stride < n_out || (dx && dx_stride < n_in))
    return egnn_fail(ctx, EGNN_EINVAL, "grouped_linear_backward: a row stride below the row's length");
  size_t need = 0;
  egnn_grouped_linear_workspace_bytes(ctx, n_rows, n_groups, n_in, n_out, &need);
  if (!ws || (uintptr_t)ws % 256 || ws_bytes < need)
    return egnn_fail(ctx, EGNN_EWS, "grouped_linear_backward: workspace too small or not 256-byte aligned");
  const GlRows p{n_rows, n_groups, ptr, perm};
  hipStream_t st = (hipStream_t)stream;
  if (dtype == EGNN_F32) return gl_backward<float>(ctx, p, x, x_stride, W, dy, dy_stride, n_in, n_out, dx, dx_stride, dW, db, ws, st);
  if (dtype == EGNN_F16) return gl_backward<_Float16>(ctx, p, x, x_stride, W, dy, dy_stride, n_in, n_out, dx, dx_stride, dW, db, ws, st);
  return gl_backward<__bf16>(ctx, p, x, x_stride, W, dy, dy_stride, n_in, n_out, dx, dx_stride, dW, db, ws, st);
}
