// Rows in 8-bit codes times the matrix of their group in 8-bit codes, with a scale for every 128 columns of a row and every 128 x 128 values
// of a matrix (codes8.h).
//
//   y_r = sum over blocks b of 128 columns of 2^(e_rb + e_nb) sum_{k in b} q_rk w_nk + bias_gn  for every row r of group g.
// Products of codes are exact in fp32 and sums are fp32, joined on two ways:
//   * bf16 results: the 8-bit matrix instruction with scales (16 x 16 results from 128 values of k, twice the rate of the 16-bit ones).  The
//     scales are powers of two in the form that the instruction takes beside its operands (a byte for the 32 values of k a lane holds), so
//     that a sum over k needs nothing between its blocks.  The instruction adds products eight at a time after cutting each off at 2^-13 of the largest
//     one's power of two (measured: 2^-13 of it beside it is kept, 2^-14 is not; with every 8-bit form), and then in fp32.  That is at most 7 * 2^-13 of the
//     terms' magnitudes and 1.5e-5 of the result's norm on normally distributed values, against 1.7e-3 for the rounding to bf16 that follows.
//   * fp32 and fp16 results: codes are taken to bf16, exactly, and multiplied by the 16-bit instruction, whose sums are fp32 throughout (no more than
//     3.7 2^-24 of the terms' magnitudes off where the 8-bit one was 2,300); the sum of a block is scaled by an exact ldexp and added.
//
// 16 x 16 results: lane l holds codes of row l % 16 of either operand, of a quarter l / 16 of the block (which codes of k are where does not matter,
// as long as it is the same for both).  W is the first operand and the rows the second, so that a lane's four results are neighbours in a row of y.
#include "codes8.h"

namespace {

typedef int sl_i8 __attribute__((ext_vector_type(8)));
typedef float sl_f4 __attribute__((ext_vector_type(4)));
typedef __bf16 sl_b8 __attribute__((ext_vector_type(8)));

struct SlArgs {
  long n;                       // rows
  int K, N, G, kb, nb;          // kb, nb: blocks of 128 along k and n
  const uint8_t *q, *qs, *w, *ws;
  long q_stride, w_stride, y_stride;
  const float* bias;
  const int *ptr, *perm;        // ptr NULL: one group of all rows
  void* y;
  int tiles_n;
};

__device__ __forceinline__ long sl_begin(const SlArgs& p, int g) { return p.ptr ? min(max((long)p.ptr[g], 0l), p.n) : g ? p.n : 0; }
__device__ __forceinline__ long sl_row(const SlArgs& p, long at) { return p.perm ? min(max((long)p.perm[at], 0l), p.n - 1) : at; }

struct SlTile { int g; long begin, end; };   // rows begin .. end - 1 of the order by group; g < 0: there is no such tile
// The tile-th of the row tiles of all groups, SIDE rows each: every wave adds up the groups' tiles, 64 groups at a time
template <int SIDE>
__device__ __forceinline__ SlTile sl_tile(const SlArgs& p, long tile) {
  const int lane = threadIdx.x & 63;
  if (!p.ptr) return {tile * SIDE < p.n ? 0 : -1, tile * SIDE, min((tile + 1) * SIDE, p.n)};
  long before = 0;
  for (int g0 = 0; g0 < p.G; g0 += 64) {
    const int g = min(g0 + lane, p.G - 1);
    const long b = sl_begin(p, g), e = sl_begin(p, g + 1);
    const int mine = g0 + lane < p.G && e > b ? (int)((e - b + SIDE - 1) / SIDE) : 0;
    int sum = mine;
    for (int d = 1; d < 64; d <<= 1) {
      const int v = __shfl_up(sum, d);
      if (lane >= d) sum += v;
    }
    const unsigned long long past = __ballot(before + sum > tile);
    if (past) {
      const int k = __ffsll((unsigned long long)past) - 1;
      const long from = __shfl(b, k) + (tile - before - __shfl(sum - mine, k)) * SIDE;
      return {g0 + k, from, min(from + SIDE, __shfl(e, k))};
    }
    before += __shfl(sum, 63);
  }
  return {-1, 0, 0};
}

// eight codes of two words as bf16, exactly: a code's value is the upper half of a float
__device__ __forceinline__ sl_b8 sl_bf16(int lo, int hi) {
  typedef float f2 __attribute__((ext_vector_type(2)));
  const f2 a = __builtin_amdgcn_cvt_pk_f32_fp8(lo, false), b = __builtin_amdgcn_cvt_pk_f32_fp8(lo, true);
  const f2 c = __builtin_amdgcn_cvt_pk_f32_fp8(hi, false), d = __builtin_amdgcn_cvt_pk_f32_fp8(hi, true);
  auto both = [](f2 v) { return __builtin_amdgcn_perm(__float_as_uint(v[1]), __float_as_uint(v[0]), 0x07060302u); };
  const uint4 u = make_uint4(both(a), both(b), both(c), both(d));
  return *reinterpret_cast<const sl_b8*>(&u);
}

// c + w q over a block of 128, scales as bytes
template <bool EXACT>
__device__ __forceinline__ sl_f4 sl_mma(const sl_i8& w, const sl_i8& q, sl_f4 c, int ew, int eq) {
  if constexpr (!EXACT) return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(w, q, c, 0, 0, 0, ew, 0, eq);
  sl_f4 sum = {};
#pragma unroll
  for (int s = 0; s < 4; ++s)
    sum = __builtin_amdgcn_mfma_f32_16x16x32_bf16(sl_bf16(w[2 * s], w[2 * s + 1]), sl_bf16(q[2 * s], q[2 * s + 1]), sum, 0, 0, 0);
#pragma unroll
  for (int i = 0; i < 4; ++i) c[i] += ldexpf(sum[i], ew + eq - 254);
  return c;
}

// 32 codes from column k of a row of K; columns from K rounded up to 16 on are not read
__device__ __forceinline__ sl_i8 sl_load(const uint8_t* row, int k, int K) {
  const uint4 zero = make_uint4(0, 0, 0, 0);
  const uint4 a = k < K ? *(const uint4*)(row + k) : zero, b = k + 16 < K ? *(const uint4*)(row + k + 16) : zero;
  return sl_i8{(int)a.x, (int)a.y, (int)a.z, (int)a.w, (int)b.x, (int)b.y, (int)b.z, (int)b.w};
}

// A wave for 32 rows by 32 columns of y, operands straight from memory
constexpr int SL_WAVES = 4;
template <class T>
__global__ void __launch_bounds__(SL_WAVES * 64) sl_direct_kernel(SlArgs p) {
  const int lane = threadIdx.x & 63, j = lane & 15, quarter = lane >> 4;
  const long item = (long)blockIdx.x * SL_WAVES + (threadIdx.x >> 6);
  const SlTile t = sl_tile<32>(p, item / p.tiles_n);
  if (t.g < 0) return;
  const int n0 = (int)(item % p.tiles_n) * 32;
  const uint8_t *w[2], *ws[2], *q[2], *qs[2];
  long row[2];
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const int n = min(n0 + 16 * i + j, p.N - 1);
    w[i] = p.w + ((long)t.g * p.N + n) * p.w_stride;
    ws[i] = p.ws + ((long)t.g * p.nb + n / C8_BLOCK) * p.kb;
    row[i] = sl_row(p, min(t.begin + 16 * i + j, t.end - 1));
    q[i] = p.q + row[i] * p.q_stride;
    qs[i] = p.qs + row[i] * p.kb;
  }
  sl_f4 sum[2][2] = {};
  for (int b = 0; b < p.kb; ++b) {
    const int k = b * C8_BLOCK + 32 * quarter;
    sl_i8 wv[2], qv[2];
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      wv[i] = sl_load(w[i], k, p.K);
      qv[i] = sl_load(q[i], k, p.K);
    }
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
      for (int r = 0; r < 2; ++r) sum[i][r] = sl_mma<!__is_same(T, __bf16)>(wv[i], qv[r], sum[i][r], ws[i][b], qs[r][b]);
  }
#pragma unroll
  for (int r = 0; r < 2; ++r) {
    if (t.begin + 16 * r + j >= t.end) continue;
    T* y = (T*)p.y + row[r] * p.y_stride;
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const int n = n0 + 16 * i + 4 * quarter + e;
        if (n < p.N) y[n] = (T)(sum[i][r][e] + (p.bias ? p.bias[(long)t.g * p.N + n] : 0.0f));
      }
  }
}

template <class T>
int sl_product(egnn_ctx* ctx, SlArgs p, hipStream_t st) {
  p.tiles_n = (p.N + 31) / 32;
  const long items = ((p.n + 31) / 32 + p.G) * p.tiles_n;
  hipLaunchKernelGGL(sl_direct_kernel<T>, dim3((unsigned)((items + SL_WAVES - 1) / SL_WAVES)), dim3(SL_WAVES * 64), 0, st, p);
  EGNN_LAUNCH_CHECK(ctx, "scaled_linear");
  return EGNN_OK;
}

}  // namespace

extern "C" int egnn_scaled_linear(egnn_ctx* ctx, const void* q, int64_t q_stride, const void* q_scale, int64_t n_rows, int32_t n_in,
                                  int32_t n_out, const void* w, int64_t w_stride, const void* w_scale, const float* bias, const int32_t* ptr,
                                  const int32_t* perm, int32_t n_groups, int32_t dtype, void* y, int64_t y_stride, void* stream) {
  if (!ctx) return EGNN_EINVAL;
  if (!rt_size(dtype)) return egnn_fail(ctx, EGNN_EINVAL, "scaled_linear: dtype must be EGNN_F32, EGNN_F16 or EGNN_BF16");
  if (n_rows < 0 || n_rows > 0x7fffffff) return egnn_fail(ctx, EGNN_EINVAL, "scaled_linear: n_rows must be in 0..2^31-1");
  if (n_in < 1 || n_in > 65536 || n_out < 1 || n_out > 65536) return egnn_fail(ctx, EGNN_EINVAL, "scaled_linear: n_in and n_out must be in 1..65536");
  if (n_groups < 1 || n_groups > 65535) return egnn_fail(ctx, EGNN_EINVAL, "scaled_linear: n_groups must be in 1..65535");
  if (!ptr && (n_groups != 1 || perm)) return egnn_fail(ctx, EGNN_EINVAL, "scaled_linear: without ptr there is one group of all rows, in their order");
  if (!w || !w_scale || (n_rows > 0 && (!q || !q_scale || !y))) return egnn_fail(ctx, EGNN_EINVAL, "scaled_linear: null pointer");
  if (q_stride < n_in || q_stride % 16 || (uintptr_t)q % 16 || w_stride < n_in || w_stride % 16 || (uintptr_t)w % 16)
    return egnn_fail(ctx, EGNN_EINVAL, "scaled_linear: rows of codes begin at multiples of 16 bytes");
  if (y_stride < n_out) return egnn_fail(ctx, EGNN_EINVAL, "scaled_linear: a row stride below the row's length");
  if (n_rows == 0) return EGNN_OK;
  const SlArgs p{n_rows, n_in, n_out, n_groups, c8_blocks(n_in), c8_blocks(n_out), (const uint8_t*)q, (const uint8_t*)q_scale, (const uint8_t*)w,
                 (const uint8_t*)w_scale, q_stride, w_stride, y_stride, bias, ptr, perm, y, 0};
  hipStream_t st = (hipStream_t)stream;
  if (dtype == EGNN_F32) return sl_product<float>(ctx, p, st);
  if (dtype == EGNN_F16) return sl_product<_Float16>(ctx, p, st);
  return sl_product<__bf16>(ctx, p, st);
}
