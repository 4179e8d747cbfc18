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
#include <algorithm>
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
  bool even;                    // rows of y begin at multiples of 16 bytes
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
      // (at least 0: groups that overlap, which is no order of the rows, may number more tiles than an int holds)
      const long from = max(__shfl(b, k) + (tile - before - __shfl(sum - mine, k)) * SIDE, 0l);
      return {g0 + k, from, min(from + SIDE, __shfl(e, k))};
    }
    before += __shfl(sum, 63);
  }
  return {-1, 0, 0};
}

// eight codes of two words as bf16, exactly
__device__ __forceinline__ sl_b8 sl_bf16(int lo, int hi) {
  typedef __bf16 b2 __attribute__((ext_vector_type(2)));
  const b2 a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, 1.0f, false), b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, 1.0f, true);
  const b2 c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, 1.0f, false), d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, 1.0f, true);
  return sl_b8{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
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

__device__ const uint4 sl_zeros = {0, 0, 0, 0};      // what is read for columns from K on (loads are never under a condition)

// 32 codes from column k of a row of K
__device__ __forceinline__ sl_i8 sl_load(const uint8_t* row, int k, int K) {
  const uint4 a = *(const uint4*)(k < K ? row + k : (const uint8_t*)&sl_zeros), b = *(const uint4*)(k + 16 < K ? row + k + 16 : (const uint8_t*)&sl_zeros);
  return sl_i8{(int)a.x, (int)a.y, (int)a.z, (int)a.w, (int)b.x, (int)b.y, (int)b.z, (int)b.w};
}

// What is read behind column K, up to a multiple of 16, is no part of a row, whatever lies there: zero.  (After the loads, so that none waits; kernels
// for K of no multiple of 16, ODD, are apart.  They take the last block behind all others where masks among these would cost registers: the tiles of 256
// spilled 87, 309 us instead of 120 for 8192 x 4090 by 4096 bf16; 4096 of k 115.)
__device__ __forceinline__ uint4 sl_first(const uint4& v, int count) {
  auto word = [](unsigned w, int bytes) { return bytes >= 4 ? w : bytes > 0 ? w & ((1u << 8 * bytes) - 1) : 0u; };
  return make_uint4(word(v.x, count), word(v.y, count - 4), word(v.z, count - 8), word(v.w, count - 12));
}
__device__ __forceinline__ void sl_trim(sl_i8& v, int k, int K) {
  const uint4 a = sl_first(make_uint4(v[0], v[1], v[2], v[3]), K - k), b = sl_first(make_uint4(v[4], v[5], v[6], v[7]), K - k - 16);
  v = sl_i8{(int)a.x, (int)a.y, (int)a.z, (int)a.w, (int)b.x, (int)b.y, (int)b.z, (int)b.w};
}

// 16 bytes of results to columns n .. of a row
template <class T>
__device__ __forceinline__ void sl_store_piece(const SlArgs& p, T* y, int n, const uint4& v) {
  constexpr int E = 16 / sizeof(T);
  if (p.even && n + E <= p.N) {
    *(uint4*)(y + n) = v;
  } else {
    typedef T all __attribute__((ext_vector_type(E)));
    const all u = *reinterpret_cast<const all*>(&v);
#pragma unroll
    for (int e = 0; e < E; ++e)
      if (n + e < p.N) y[n + e] = u[e];
  }
}
// LDS written by lanes of a wave is read by others of the same wave (its accesses go in order)
__device__ __forceinline__ void sl_wave_sync() {
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront", "local");
  __builtin_amdgcn_wave_barrier();
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront", "local");
}

// Tile of a workgroup: workgroups go round the eight XCDs, and each of those takes a run of tiles, for its L2; in the order of all tiles, `down` row tiles
// go through the columns together.
__device__ __forceinline__ void sl_item(long block, long items, int tiles_n, int down, long& row_tile, int& col_tile) {
  const long each = items / 8, more = items % 8, xcd = block % 8, at = xcd * each + min(xcd, more) + block / 8;
  const long rows = items / tiles_n, band = at / ((long)down * tiles_n), in = at - band * down * tiles_n, high = min((long)down, rows - band * down);
  row_tile = band * down + in % high;
  col_tile = (int)(in / high);
}

constexpr int SL_WAVES = 4, SL_DOWN = 4;

// ---- few rows -----------------------------------------------------------------------------------------------------------------
// What bounds it is reading W once (one row of 2048 by 4096 bf16 4.4 us for 8.4 MB: launch and a chain of two loads as much as memory).  A workgroup makes 16 columns of up to 16 R rows; its waves take the blocks of k in turn, SL_AHEAD of them under way
// in each, and add up through LDS in the order of the waves.
constexpr int SL_FEW = 8, SL_AHEAD = 4;
template <class T, int R, bool ODD>
__global__ void __launch_bounds__(SL_FEW * 64) sl_few_kernel(SlArgs p) {
  constexpr bool EXACT = !__is_same(T, __bf16);
  __shared__ sl_f4 lds[SL_FEW][R][64];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, j = lane & 15, quarter = lane >> 4;
  const SlTile t = sl_tile<16 * R>(p, blockIdx.x / p.tiles_n);
  if (t.g < 0) return;
  const int n0 = (int)(blockIdx.x % p.tiles_n) * 16, n = min(n0 + j, p.N - 1);
  const uint8_t *w = p.w + ((long)t.g * p.N + n) * p.w_stride, *ws = p.ws + ((long)t.g * p.nb + n / C8_BLOCK) * p.kb, *q[R], *qs[R];
#pragma unroll
  for (int r = 0; r < R; ++r) {
    const long row = sl_row(p, min(t.begin + 16 * r + j, t.end - 1));
    q[r] = p.q + row * p.q_stride;
    qs[r] = p.qs + row * p.kb;
  }
  sl_f4 sum[R] = {};
  const int whole = ODD ? p.kb - 1 : p.kb, K = ODD ? whole * C8_BLOCK : p.K;        // ODD: the last block is taken apart
  for (int b0 = wave; b0 < whole; b0 += SL_FEW * SL_AHEAD) {
    sl_i8 wv[SL_AHEAD], qv[SL_AHEAD][R];
    int ew[SL_AHEAD], eq[SL_AHEAD][R];
#pragma unroll
    for (int u = 0; u < SL_AHEAD; ++u) {
      const int b = b0 + u * SL_FEW, k = b * C8_BLOCK + 32 * quarter, at = min(b, p.kb - 1);
      wv[u] = sl_load(w, k, K);
      ew[u] = ws[at];
#pragma unroll
      for (int r = 0; r < R; ++r) {
        qv[u][r] = sl_load(q[r], k, K);
        eq[u][r] = qs[r][at];
      }
    }
#pragma unroll
    for (int u = 0; u < SL_AHEAD; ++u)
#pragma unroll
      for (int r = 0; r < R; ++r) sum[r] = sl_mma<EXACT>(wv[u], qv[u][r], sum[r], ew[u], eq[u][r]);
  }
  if (ODD && wave == whole % SL_FEW) {
    const int k = whole * C8_BLOCK + 32 * quarter;
    sl_i8 wv = sl_load(w, k, p.K), qv[R];
    int eq[R];
#pragma unroll
    for (int r = 0; r < R; ++r) {
      qv[r] = sl_load(q[r], k, p.K);
      eq[r] = qs[r][whole];
    }
    sl_trim(wv, k, p.K);
#pragma unroll
    for (int r = 0; r < R; ++r) {
      sl_trim(qv[r], k, p.K);
      lds[wave][r][lane] = sl_mma<EXACT>(wv, qv[r], sum[r], ws[whole], eq[r]);
    }
  } else {
#pragma unroll
    for (int r = 0; r < R; ++r) lds[wave][r][lane] = sum[r];
  }
  __syncthreads();
  for (int i = threadIdx.x; i < R * 256; i += SL_FEW * 64) {
    const int col = i & 15, row = i >> 4, at = (row & 15) + 16 * (col >> 2);        // lane and element that hold it
    float v = lds[0][row >> 4][at][col & 3];
#pragma unroll
    for (int k = 1; k < SL_FEW; ++k) v += lds[k][row >> 4][at][col & 3];
    if (t.begin + row < t.end && n0 + col < p.N)
      ((T*)p.y)[sl_row(p, t.begin + row) * p.y_stride + n0 + col] = (T)(v + (p.bias ? p.bias[(long)t.g * p.N + n0 + col] : 0.0f));
  }
}

// ---- many rows, one block of k ------------------------------------------------------------------------------------------------
// Up to 128 of k and 32 F columns: what bounds it is memory, the rows in and out.  W stays in registers (H turns of 64 of k) while a wave takes a run of
// 32-row tiles in the order by group, the next one's codes and the row numbers of the one after that under way.  Measured: 300,000 x 64 by 64 fp32 18.4 us
// (5.2 TB/s), in 15 groups of rows in any order 20 to 24 (rows of 64 bytes are half a line each).
struct SlWalk { int g; long at, end; };
__device__ __forceinline__ SlWalk sl_next(const SlArgs& p, SlWalk t) {
  t.at += 32;
  while (t.at >= t.end && t.g + 1 < p.G) {
    ++t.g;
    t.at = sl_begin(p, t.g);
    t.end = sl_begin(p, t.g + 1);
  }
  return t;
}

template <class T, int H, int F, bool ODD>
__global__ void __launch_bounds__(SL_WAVES * 64) sl_rows_kernel(SlArgs p, long share) {
  constexpr bool EXACT = !__is_same(T, __bf16);
  typedef float sl_f16 __attribute__((ext_vector_type(16)));
  const int lane = threadIdx.x & 63, j = lane & 31, half = lane >> 5;
  constexpr int n0 = 0;
  constexpr int PIECES = 2 * F * (int)sizeof(T);                 // of 16 bytes, of a row of the wave's results
  __shared__ __attribute__((aligned(16))) uint8_t lds[SL_WAVES][32 * PIECES * 16];
  __shared__ float4 bias_lds[SL_WAVES][8 * F];                  // (in LDS, not in 32 F registers)
  uint8_t* out = lds[threadIdx.x >> 6];
  float4* bias = bias_lds[threadIdx.x >> 6];
  const SlTile first = sl_tile<32>(p, ((long)blockIdx.x * SL_WAVES + (threadIdx.x >> 6)) * share);
  if (first.g < 0) return;
  SlWalk now{first.g, first.begin, sl_begin(p, first.g + 1)}, then = sl_next(p, now);
  auto row_of = [&](const SlWalk& t) { return sl_row(p, min(t.at + j, max(t.end, 1l) - 1)); };
  struct Rows { sl_i8 q[H]; int e; };
  auto fetch = [&](long row) {
    Rows o;
#pragma unroll
    for (int h = 0; h < H; ++h) o.q[h] = sl_load(p.q + row * p.q_stride, 64 * h + 32 * half, p.K);
    o.e = p.qs[row];
    return o;
  };
  // results go through LDS, so that rows are written whole; a row's pieces lie at (piece xor row), for the banks
  auto swizzle = [](int r) { return PIECES >= 16 ? r & 15 : PIECES == 8 ? r >> 1 & 7 : r >> 2 & 3; };
  sl_i8 keep[ODD ? H : 1];
#pragma unroll
  for (int h = 0; h < (ODD ? H : 0); ++h) {
    keep[h] = sl_i8{-1, -1, -1, -1, -1, -1, -1, -1};
    sl_trim(keep[h], 64 * h + 32 * half, p.K);
  }
  long row = row_of(now), row_then = row_of(then);
  Rows v = fetch(row);
  sl_i8 w[F][H];
  int ew[F], loaded = -1;
  for (long k = 0; k < share && now.at < now.end; ++k) {
    const SlWalk far = sl_next(p, then);
    const Rows v_then = fetch(row_then);
    const long row_far = row_of(far);
    if (now.g != loaded) {
      loaded = now.g;
#pragma unroll
      for (int i = 0; i < F; ++i) {
        const int n = min(n0 + 32 * i + j, p.N - 1);
#pragma unroll
        for (int h = 0; h < H; ++h) w[i][h] = sl_load(p.w + ((long)now.g * p.N + n) * p.w_stride, 64 * h + 32 * half, p.K);
        ew[i] = p.ws[(long)now.g * p.nb + min(n0 + 32 * i, p.N - 1) / C8_BLOCK];
      }
      if constexpr (ODD)
#pragma unroll
        for (int i = 0; i < F; ++i)
#pragma unroll
          for (int h = 0; h < H; ++h) w[i][h] &= keep[h];
      if (lane < 32 * F) ((float*)bias)[lane] = p.bias ? p.bias[(long)now.g * p.N + min(n0 + lane, p.N - 1)] : 0.0f;
      sl_wave_sync();
    }
    if constexpr (ODD)
#pragma unroll
      for (int h = 0; h < H; ++h) v.q[h] &= keep[h];
#pragma unroll
    for (int i = 0; i < F; ++i) {
      sl_f16 sum;
#pragma unroll
      for (int e = 0; e < 16; ++e) sum[e] = 0.0f;
#pragma unroll
      for (int h = 0; h < H; ++h) {
        if constexpr (EXACT) {
#pragma unroll
          for (int s = 0; s < 4; ++s)
            sum = __builtin_amdgcn_mfma_f32_32x32x16_bf16(sl_bf16(w[i][h][2 * s], w[i][h][2 * s + 1]), sl_bf16(v.q[h][2 * s], v.q[h][2 * s + 1]), sum, 0, 0, 0);
        } else {
          sum = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(w[i][h], v.q[h], sum, 0, 0, 0, ew[i], 0, v.e);
        }
      }
      if constexpr (EXACT)
#pragma unroll
        for (int e = 0; e < 16; ++e) sum[e] = ldexpf(sum[e], ew[i] + v.e - 254);
      typedef T four __attribute__((ext_vector_type(4)));
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const int col = 32 * i + 8 * e + 4 * half, byte = col * (int)sizeof(T);
        const float4 b = bias[col / 4];
        const four u = {(T)(sum[4 * e] + b.x), (T)(sum[4 * e + 1] + b.y), (T)(sum[4 * e + 2] + b.z), (T)(sum[4 * e + 3] + b.w)};
        *(four*)(out + j * PIECES * 16 + 16 * (byte / 16 ^ swizzle(j)) + byte % 16) = u;
      }
    }
    sl_wave_sync();
#pragma unroll
    for (int it = 0; it < PIECES / 2; ++it) {
      const int r = it * (64 / PIECES) + lane / PIECES, k = lane % PIECES;
      const long to = __shfl(row, r);
      if (now.at + r < now.end) sl_store_piece<T>(p, (T*)p.y + to * p.y_stride, n0 + k * 16 / (int)sizeof(T), *(const uint4*)(out + r * PIECES * 16 + 16 * (k ^ swizzle(r))));
    }
    sl_wave_sync();
    now = then;
    then = far;
    row = row_then;
    row_then = row_far;
    v = v_then;
  }
}

// ---- tiles through LDS -------------------------------------------------------------------------------------------------------
// A workgroup of four waves makes SIDE x SIDE results, a quarter each; a turn takes 64 of k, a block of 128 two turns.  Rows of both operands go
// straight from memory to LDS, a block's 128 bytes of a row at once (16 bytes a lane), into one of two buffers, and from there to registers one turn ahead:
// while a turn's products run, the next one's operands are read.  One barrier a block: behind it the next block is in LDS, and nobody reads this
// one's buffer any more, so that the block after the next can be asked for.  (Measured, 8192 x 4096 by 4096 bf16: 115 us, 2,390 TFLOP/s, matrix units 65 %
// busy; with 64 bytes of a row at a time, four buffers and three turns ahead 152, as L2 has twice the requests; without the order of instructions
// below 167; eight waves and no reading ahead 146.  With one buffer, three workgroups of 128 x 128 a compute unit: 20,000 x 512 by 1024 in 16 groups of rows in any order 28.)  A row's eight pieces of 16 bytes lie at (piece xor row / 2), so that 16 rows read
// at once lie in all 64 banks.
typedef __attribute__((address_space(3))) uint8_t sl_lds;
typedef const __attribute__((address_space(1))) uint8_t sl_global;
constexpr int SL_ARRIVED = 0xf70;                              // the operand of s_waitcnt that waits until no load is out

template <int LOADS>
__device__ __forceinline__ void sl_stage(const uint8_t* const (&row)[LOADS], uint8_t* to, int k, int K) {
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
#pragma unroll
  for (int i = 0; i < LOADS; ++i) {
    const uint8_t* from = k < K ? row[i] + k : (const uint8_t*)&sl_zeros;
    __builtin_amdgcn_global_load_lds((sl_global*)from, (sl_lds*)to + (i * SL_WAVES + wave) * 1024, 16, 0, 0);
  }
}

// a barrier that waits for LDS alone, not for loads that are on their way to other buffers
__device__ __forceinline__ void sl_barrier() {
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "workgroup", "local");
  __builtin_amdgcn_s_barrier();
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "workgroup", "local");
}

template <class T, int SIDE, bool TWO, bool ODD>
__global__ void __launch_bounds__(SL_WAVES * 64, SIDE == 256 ? 1 : TWO || !__is_same(T, __bf16) ? 2 : 3) sl_tile_kernel(SlArgs p, long tiles) {
  constexpr bool EXACT = !__is_same(T, __bf16);
  constexpr int F = SIDE / 64;                                        // fragments of 32 rows of a wave, of either operand
  constexpr int LOADS = SIDE * C8_BLOCK / (SL_WAVES * 1024);          // of a lane, of either operand, a block
  constexpr int COLS = 32 * F, PIECES = COLS * (int)sizeof(T) / 16;   // a wave's results: columns, and pieces of 16 bytes of a row
  constexpr int OUT = COLS * PIECES * 16, BUFFER = 2 * SIDE * C8_BLOCK, ROOM = !TWO && SL_WAVES * OUT > BUFFER ? SL_WAVES * OUT : BUFFER;
  static_assert(F <= 4 && COLS <= C8_BLOCK && SL_WAVES * OUT <= (TWO ? 2 : 1) * ROOM, "scales in a word, one scale of W a wave, room for the results of all");
  __shared__ __attribute__((aligned(1024))) uint8_t b0[ROOM], b1[TWO ? BUFFER : 16];
  __shared__ __attribute__((aligned(16))) uint8_t le0[SIDE], le1[SIDE];
  __shared__ int rows[SIDE];
  __shared__ __attribute__((aligned(16))) float bias[SIDE];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), j = lane & 31, half = lane >> 5, wr = wave >> 1, wn = wave & 1;
  long row_tile;
  int col_tile;
  sl_item(blockIdx.x, tiles, p.tiles_n, SL_DOWN, row_tile, col_tile);
  const SlTile t = sl_tile<SIDE>(p, row_tile);
  if (t.g < 0) return;
  const int n0 = col_tile * SIDE;
  const uint8_t *q_row[LOADS], *w_row[LOADS];
#pragma unroll
  for (int i = 0; i < LOADS; ++i) {
    const int r = (i * SL_WAVES + wave) * 8 + (lane >> 3);
    q_row[i] = p.q + sl_row(p, min(t.begin + r, t.end - 1)) * p.q_stride;
    w_row[i] = p.w + ((long)t.g * p.N + min(n0 + r, p.N - 1)) * p.w_stride;
  }
  // (a lane's rows are 32 apart, so that row / 2 has the same last three bits for all of them)
  const int piece = 16 * ((lane & 7) ^ ((wave * 8 + (lane >> 3)) >> 1 & 7));
  // scales of the rows: thread r brings that of row r to where lane r % 32 finds those of its fragments side by side
  const int mine = threadIdx.x % SIDE;
  const uint8_t* scale_at = p.qs + sl_row(p, min(t.begin + mine, t.end - 1)) * p.kb;
  const int scale_to = mine / (32 * F) * (32 * F) + (mine & 31) * F + (mine / 32) % F;
  const uint8_t* wscale_at = p.ws + ((long)t.g * p.nb + min((n0 + wn * COLS) / C8_BLOCK, p.nb - 1)) * p.kb;

  typedef float sl_f16 __attribute__((ext_vector_type(16)));
  sl_f16 sum[F][F], part[EXACT ? F : 1][EXACT ? F : 1];
#pragma unroll
  for (int i = 0; i < F; ++i)
#pragma unroll
    for (int r = 0; r < F; ++r)
#pragma unroll
      for (int e = 0; e < 16; ++e) sum[i][r][e] = 0.0f;
  const int from = (wr * COLS + j) * C8_BLOCK, wfrom = (SIDE + wn * COLS + j) * C8_BLOCK;
  const int at0 = 16 * ((2 * half) ^ (j >> 1 & 7)), at1 = 16 * ((2 * half + 1) ^ (j >> 1 & 7));
  struct Operands { sl_i8 q[F], w[F]; };
  auto fetch = [&](const uint8_t* buffer, int second, Operands& o) {
    auto one = [&](const uint8_t* row) {
      const uint4 a = *(const uint4*)(row + (at0 ^ 64 * second)), b = *(const uint4*)(row + (at1 ^ 64 * second));
      return sl_i8{(int)a.x, (int)a.y, (int)a.z, (int)a.w, (int)b.x, (int)b.y, (int)b.z, (int)b.w};
    };
#pragma unroll
    for (int i = 0; i < F; ++i) {
      o.w[i] = one(buffer + wfrom + i * 32 * C8_BLOCK);
      o.q[i] = one(buffer + from + i * 32 * C8_BLOCK);
    }
  };
  auto scales = [&](const uint8_t* le) {
    if constexpr (F == 4) return *(const unsigned*)(le + wr * COLS + j * F);
    else return (unsigned)*(const uint16_t*)(le + wr * COLS + j * F);
  };
  auto stage_up_to = [&](uint8_t* buffer, int b, int K) {
    sl_stage<LOADS>(q_row, buffer, b * C8_BLOCK + piece, K);
    sl_stage<LOADS>(w_row, buffer + SIDE * C8_BLOCK, b * C8_BLOCK + piece, K);
  };
  const int whole = ODD ? p.kb - 1 : p.kb, K = ODD && TWO ? whole * C8_BLOCK : p.K;       // ODD with two buffers: the last block is taken apart
  auto stage = [&](uint8_t* buffer, int b) { stage_up_to(buffer, b, K); };
  // ODD, the last block has arrived: the piece that K ends inside is trimmed where it lies, by the lane that asked for it
  auto trim = [&](uint8_t* buffer) {
    sl_wave_sync();
    const int left = p.K - whole * C8_BLOCK - piece;
    if (left <= 0 || left >= 16) return;
#pragma unroll 4
    for (int i = 0; i < 2 * LOADS; ++i) {
      uint4* at = (uint4*)(buffer + (i * SL_WAVES + wave) * 1024 + lane * 16);      // (rows of W behind those of the codes)
      *at = sl_first(*at, left);
    }
  };
  auto block_at = [&](int b) { return min(b, p.kb - 1); };

  // (of the blocks 0 and 1)
  const int scale0 = scale_at[0];
  const float bias0 = p.bias ? p.bias[(long)t.g * p.N + min(n0 + mine, p.N - 1)] : 0.0f;
  int scale = scale_at[block_at(1)], ew = wscale_at[0], ew_next = wscale_at[block_at(1)];
  stage(b0, 0);
  if constexpr (TWO) stage(b1, 1);
  rows[mine] = (int)sl_row(p, min(t.begin + mine, t.end - 1));
  le0[scale_to] = (uint8_t)scale0;
  bias[mine] = bias0;
  // (both blocks: the writes to LDS just above, of values that were loaded, wait for every load before them)
  __builtin_amdgcn_s_waitcnt(SL_ARRIVED);
  if (ODD && !TWO && whole == 0) trim(b0);
  sl_barrier();
  unsigned eq = scales(le0), eq_next = eq;

  Operands even, odd;
  auto products = [&](const Operands& now, bool second) {
#pragma unroll
    for (int r = 0; r < F; ++r)
#pragma unroll
      for (int i = 0; i < F; ++i) {
        const int e = (int)(eq >> (8 * r) & 0xff);
        if constexpr (!EXACT) {
          sum[i][r] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(now.w[i], now.q[r], sum[i][r], 0, 0, 0, ew, 0, e);
        } else {
          sl_f16 v;
#pragma unroll
          for (int k = 0; k < 16; ++k) v[k] = second ? part[i][r][k] : 0.0f;
#pragma unroll
          for (int k = 0; k < 4; ++k)
            v = __builtin_amdgcn_mfma_f32_32x32x16_bf16(sl_bf16(now.w[i][2 * k], now.w[i][2 * k + 1]), sl_bf16(now.q[r][2 * k], now.q[r][2 * k + 1]), v, 0, 0, 0);
          if (!second) {
            part[i][r] = v;
          } else {
#pragma unroll
            for (int k = 0; k < 16; ++k) sum[i][r][k] += ldexpf(v[k], ew + e - 254);
          }
        }
      }
  };
  // block b from `here`; the block after it lies, or arrives, in `next`
  auto block = [&](int b, uint8_t* here, const uint8_t* next, uint8_t* le) {
    le[scale_to] = (uint8_t)scale;                        // of the next block
    scale = scale_at[block_at(b + 2)];
    const int ew_far = wscale_at[block_at(b + 2)];
    fetch(here, 1, odd);
    products(even, false);
    if constexpr (!EXACT) {                               // a product and a read of LDS in turn
#pragma unroll
      for (int k = 0; k < F * F; ++k) {
        __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
        __builtin_amdgcn_sched_group_barrier(0x100, 4 / F, 0);
      }
    }
    __builtin_amdgcn_sched_barrier(0);
    __builtin_amdgcn_s_waitcnt(SL_ARRIVED);              // this wave's part of the next block is in LDS
    sl_barrier();
    __builtin_amdgcn_sched_barrier(0);
    eq_next = scales(le);
    stage(here, b + 2);
    fetch(next, 0, even);
    products(odd, true);
    if constexpr (!EXACT) {
#pragma unroll
      for (int k = 0; k < F * F; ++k) {
        __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
        __builtin_amdgcn_sched_group_barrier(0x020, 4 / F, 0);
        __builtin_amdgcn_sched_group_barrier(0x100, 4 / F, 0);
      }
    }
    __builtin_amdgcn_sched_barrier(0);
    eq = eq_next;
    ew = ew_next;
    ew_next = ew_far;
  };
  if constexpr (TWO) {
    fetch(b0, 0, even);
    for (int b = 0; b < whole; b += 2) {                  // (what lies behind K: zeros)
      block(b, b0, b1, le1);
      if constexpr (SIDE < 256)
        if (b + 1 >= whole) break;
      block(b + 1, b1, b0, le0);
    }
  } else {
    for (int b = 0;;) {
      fetch(b0, 0, even);
      products(even, false);
      fetch(b0, 1, even);
      products(even, true);
      if (++b == p.kb) break;
      sl_barrier();
      stage(b0, b);
      le0[scale_to] = (uint8_t)scale;
      scale = scale_at[block_at(b + 1)];
      ew = ew_next;
      ew_next = wscale_at[block_at(b + 1)];
      __builtin_amdgcn_s_waitcnt(SL_ARRIVED);
      if (ODD && b == whole) trim(b0);
      sl_barrier();
      eq = scales(le0);
    }
  }
  if constexpr (ODD && TWO) {                             // eq and ew are those of the last block
    __builtin_amdgcn_s_waitcnt(SL_ARRIVED);
    sl_barrier();                                         // nothing is on its way to the buffer any more, and nobody reads it
    stage_up_to(b0, whole, p.K);
    __builtin_amdgcn_s_waitcnt(SL_ARRIVED);
    trim(b0);
    sl_barrier();
    fetch(b0, 0, even);
    products(even, false);
    fetch(b0, 1, even);
    products(even, true);
  }

  // Results through LDS, a buffer for each wave, so that rows are written whole; a row's pieces of 16 bytes lie at (piece xor row), for the banks.
  __builtin_amdgcn_s_waitcnt(SL_ARRIVED);
  __syncthreads();
  uint8_t* out = TWO ? (wave & 1 ? b1 : b0) + (wave >> 1) * OUT : b0 + wave * OUT;
  auto swizzle = [](int row) { return PIECES == 16 ? row & 15 : row >> 1 & 7; };
  typedef T four __attribute__((ext_vector_type(4)));
#pragma unroll
  for (int i = 0; i < F; ++i)
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const int col = 32 * i + 8 * k + 4 * half;
      const float4 b4 = *(const float4*)(bias + wn * COLS + col);
      const float b[4] = {b4.x, b4.y, b4.z, b4.w};
#pragma unroll
      for (int r = 0; r < F; ++r) {
        four u;
#pragma unroll
        for (int e = 0; e < 4; ++e) u[e] = (T)(sum[i][r][4 * k + e] + b[e]);
        const int row = 32 * r + j, byte = col * (int)sizeof(T);
        *(four*)(out + row * PIECES * 16 + 16 * (byte / 16 ^ swizzle(row)) + byte % 16) = u;
      }
    }
  __syncthreads();
  const int k = lane % PIECES, n = n0 + wn * COLS + k * 16 / (int)sizeof(T);
#pragma unroll
  for (int it = 0; it < COLS * PIECES / 64; ++it) {
    const int row = it * (64 / PIECES) + lane / PIECES, at = wr * COLS + row;
    if (t.begin + at >= t.end) continue;
    sl_store_piece<T>(p, (T*)p.y + (long)rows[at] * p.y_stride, n, *(const uint4*)(out + row * PIECES * 16 + 16 * (k ^ swizzle(row))));
  }
}

// row tiles of SIDE rows of all groups at most: each group that has rows may end inside one
long sl_row_tiles(const SlArgs& p, int side) { return (p.n + side - 1) / side + (p.ptr ? std::min<long>(p.G, p.n) : 0); }

int sl_launched(egnn_ctx* ctx) {
  EGNN_LAUNCH_CHECK(ctx, "scaled_linear");
  return EGNN_OK;
}
int sl_too_many(egnn_ctx* ctx) { return egnn_fail(ctx, EGNN_EINVAL, "scaled_linear: more than 2^32 threads' worth of results"); }

template <class T, int SIDE, bool TWO, bool ODD>
int sl_tiles(egnn_ctx* ctx, SlArgs p, hipStream_t st) {
  p.tiles_n = (p.N + SIDE - 1) / SIDE;
  const long items = sl_row_tiles(p, SIDE) * p.tiles_n;
  if (items * SL_WAVES * 64 > 0xffffffffl) return sl_too_many(ctx);
  hipLaunchKernelGGL((sl_tile_kernel<T, SIDE, TWO, ODD>), dim3((unsigned)items), dim3(SL_WAVES * 64), 0, st, p, items);
  return sl_launched(ctx);
}

template <class T, int H, int F, bool ODD>
int sl_rows(egnn_ctx* ctx, const SlArgs& p, hipStream_t st) {
  // as many waves as run at once: two a SIMD with their 150 to 190 registers, four of the narrow ones (300,000 x 64 by 64 fp32 in 15 groups 24.3 us with
  // 2,048 waves, 29.4 with 4,096; 2,000,000 x 16 by 16 33.5 and 23.2)
  const long waves = F == 1 ? 4096 : 2048, tiles = sl_row_tiles(p, 32), share = (tiles + waves - 1) / waves;
  hipLaunchKernelGGL((sl_rows_kernel<T, H, F, ODD>), dim3((unsigned)((tiles + share * SL_WAVES - 1) / (share * SL_WAVES))), dim3(SL_WAVES * 64), 0, st, p, share);
  return sl_launched(ctx);
}

template <class T, int R, bool ODD>
int sl_few(egnn_ctx* ctx, SlArgs p, hipStream_t st) {
  p.tiles_n = (p.N + 15) / 16;
  hipLaunchKernelGGL((sl_few_kernel<T, R, ODD>), dim3((unsigned)(sl_row_tiles(p, 16 * R) * p.tiles_n)), dim3(SL_FEW * 64), 0, st, p);
  return sl_launched(ctx);
}

// Which kernel (times in us):
//   * up to 128 of k and 64 columns: W in registers (300,000 x 64 by 64 fp32 in 15 groups of rows in any order 23, tiles 45; 100,000 x 128
//     by 64 bf16 9.2 and 11.2);
//   * where 16 columns by the rows of an average group, 64 at most, make no more workgroups than 256 (512 for fp32 and fp16): k over the waves of a workgroup
//     (128 x 2048 by 1024 bf16, 128 workgroups, 10.7, tiles 13.1; by 4096, 512 of them, 18.5 and 13.3; fp32 21 and 28);
//   * bf16 tiles of 256, one workgroup per compute unit, where k is 2,048 at least and the last round of 256 of them is full enough that seven in ten places are
//     used on average (4096 x 4096 by 4096 60, tiles of 128 87; 10,000 rows, 640 tiles, 162 and 184; 5120 rows, 320 tiles, 102 and 93; with 1,024 of k
//     and 10,000 rows 66 and 57);
//   * else tiles of 128: bf16 with two buffers as long as there is about one for each compute unit (2048 x 4096 by 2048 32 and, with one buffer, 39), with
//     one buffer, three workgroups per compute unit, above that (20,000 x 512 by 1024 in one group 25.1 and 21.7, in 16 of rows in any order 33 and 28).  fp32 and fp16 have one buffer always: twice the products
//     and the sums of a block beside those of all leave no registers for more (20,000 x 512 by 1024 fp32 in one group 45 and 40, in 16 57 and 51).
template <class T, bool ODD>
int sl_product(egnn_ctx* ctx, SlArgs p, hipStream_t st) {
  constexpr bool EXACT = !__is_same(T, __bf16);
  p.even = (uintptr_t)p.y % 16 == 0 && p.y_stride * sizeof(T) % 16 == 0;
  if (p.K <= C8_BLOCK && p.N <= 64) {
    if (p.K <= 64) return p.N <= 32 ? sl_rows<T, 1, 1, ODD>(ctx, p, st) : sl_rows<T, 1, 2, ODD>(ctx, p, st);
    return p.N <= 32 ? sl_rows<T, 2, 1, ODD>(ctx, p, st) : sl_rows<T, 2, 2, ODD>(ctx, p, st);
  }
  const long each = p.n / p.G;
  const int R = each <= 16 ? 1 : each <= 32 ? 2 : 4;
  if (sl_row_tiles(p, 16 * R) * ((p.N + 15) / 16) <= (EXACT ? 512 : 256))
    return R == 1 ? sl_few<T, 1, ODD>(ctx, p, st) : R == 2 ? sl_few<T, 2, ODD>(ctx, p, st) : sl_few<T, 4, ODD>(ctx, p, st);
  if constexpr (!EXACT) {
    const long large = sl_row_tiles(p, 256) * ((p.N + 255) / 256), places = (large + EGNN_CUS - 1) / EGNN_CUS * EGNN_CUS;
    if (p.K >= 2048 && large * 10 >= places * 7) return sl_tiles<T, 256, true, ODD>(ctx, p, st);
    if (sl_row_tiles(p, 128) * ((p.N + 127) / 128) <= 3 * EGNN_CUS / 2) return sl_tiles<T, 128, true, ODD>(ctx, p, st);
  }
  return sl_tiles<T, 128, false, ODD>(ctx, p, st);
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
                 (const uint8_t*)w_scale, q_stride, w_stride, y_stride, bias, ptr, perm, y, 0, false};
  hipStream_t st = (hipStream_t)stream;
  if (dtype == EGNN_F32) return n_in % 16 ? sl_product<float, true>(ctx, p, st) : sl_product<float, false>(ctx, p, st);
  if (dtype == EGNN_F16) return n_in % 16 ? sl_product<_Float16, true>(ctx, p, st) : sl_product<_Float16, false>(ctx, p, st);
  return n_in % 16 ? sl_product<__bf16, true>(ctx, p, st) : sl_product<__bf16, false>(ctx, p, st);
}
