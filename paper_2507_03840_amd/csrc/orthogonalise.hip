// An update orthogonalised by Newton-Schulz products, and the optimiser's step around it.
//
//   x_0 = u / (|u|_F + 1e-7),   x_{k+1} = a x_k + p x_k,   p = b g + c g^2,   g = x_k x_k^T  (x from the side with fewer rows),
// with the published coefficients of the Muon optimiser: the singular values of u go to within about 0.7 .. 1.2.
// Step: m' = beta m + g, u = g + beta m', W' = (1 - lr weight_decay) W - lr sqrt(max(1, rows / cols)) orthogonalise(u).
//
// All products are C = A B^T of operands with the contraction along the rows: g = x x^T, g g (g is symmetric), p x with x^T kept
// beside x.  They run on the matrix cores on half-precision pieces: v s = hi + lo, hi = v s rounded to 11 bits, lo = the rest
// rounded to 11 bits, and hi hi + hi lo + lo hi (the dropped lo lo is 2^-24 of the product).  |x_0|_F <= 1 and the steps keep
// the singular values below 1.2025, so every entry of x, g and p is bounded whatever the input, and one fixed power of two as
// scale s leaves nothing to overflow.  Nothing above 2^-39 underflows, and that counts from the norm: what is kept is X, x = sigma X, from
// X_0 = u / |u|, sigma_0 = |u| / (|u| + 1e-7) on, sigma_{k+1} = min(1, a sigma_k): where |u| is far below 1e-7, x is too, and a few steps
// only multiply it by a.  With r = sigma_k / sigma_{k+1} = max(1 / a, sigma_k) a step is
//   X_{k+1} = r (a X + (b sigma^2 G + c sigma^4 G^2) X),   G = X X^T,
// whose factor of each singular value lies below that of sigma = 1, so the bounds hold for X as well.  Above |u| = 5e-8 sigma is 1 from the
// second step on.
// p stays without its a I, and a x is added to (b g + c g^2) x in fp32: pieces of 22 bits of a on the diagonal of p would take the same part
// of every singular value's last bits, again in every step (1536 x 2048 1.33e-5 off 64 bits with it in p, 5.4e-6 without; torch in fp32 8.3e-6).
// Every type of result comes from both pieces: with hi alone bfloat16 results of wide updates were 4e-4 to 6e-4 off beside their last rounding
// (1.7e-3).
#include "row_types.h"
#include "stream_gemm.h"
#include <math.h>
#include <type_traits>

namespace {

constexpr float OU_A = 3.4445f, OU_B = -4.7750f, OU_C = 2.0315f;
constexpr double OU_EPS = 1e-7;
// entries of x are at most 1.2025, of g 1.446, of p 2.81 (its eigenvalues lie between b^2 / 4c = -2.81 and 0): times these at most 47,400
constexpr float OU_SX = 32768.0f, OU_SG = 32768.0f, OU_SP = 16384.0f;
constexpr int OU_PARTS = 512;       // partial sums of squares per matrix, at most

typedef _Float16 ou_h8 __attribute__((ext_vector_type(8)));
typedef float ou_f16v __attribute__((ext_vector_type(16)));

struct OuShape {
  int batch, rows, cols, n, m;   // n = the smaller side, m = the larger one
  int np, mp;                    // rounded up to 64: the rest is zero
  bool tall;                     // rows > cols: x is the transpose of the caller's matrix
};

size_t ou_align(size_t n) { return (n + 255) & ~(size_t)255; }

// u: the caller's matrices, or g + beta m' of the optimiser's step (g = u, m = m')
template <class T>
struct OuInput { const T* u; const float* m; float beta; };

template <class T>
__device__ __forceinline__ float ou_value(const OuInput<T>& in, size_t i) {
  return in.m ? (float)in.u[i] + in.beta * in.m[i] : (float)in.u[i];
}

__device__ __forceinline__ void ou_cut(float v, _Float16& hi, _Float16& lo) {
  hi = (_Float16)v;
  lo = (_Float16)(v - (float)hi);
}

// ---- sums of squares (fp64: no overflow, no underflow), and the new momentum
// V values at a time (4 where every matrix begins and ends in aligned fours), sixteen a thread and round, all loaded before the first is used.
constexpr int OU_ROUND = 4096;      // values of a workgroup and round
template <class T, int V>
__global__ __launch_bounds__(256) void ou_square_kernel(OuInput<T> in, const float* m_old, float* m_new, size_t size, double* part) {
  __shared__ double s[256];
  constexpr int U = 16 / V;
  const size_t at = (size_t)blockIdx.y * size;
  double t = 0.0;
  for (size_t b = (size_t)blockIdx.x * OU_ROUND; b < size; b += (size_t)gridDim.x * OU_ROUND) {
    float v[U][V], mm[U][V];
#pragma unroll
    for (int k = 0; k < U; ++k) {
      const size_t i = b + (size_t)(k * 256 + threadIdx.x) * V, from = at + (i < size ? i : size - V);
      rt_load<T, V>(in.u + from, v[k]);
      if (m_old) rt_load<float, V>(m_old + from, mm[k]);
    }
#pragma unroll
    for (int k = 0; k < U; ++k) {
      const size_t i = b + (size_t)(k * 256 + threadIdx.x) * V;
      const bool there = i < size;
#pragma unroll
      for (int q = 0; q < V; ++q) {
        if (m_old) {
          mm[k][q] = in.beta * mm[k][q] + v[k][q];
          v[k][q] = v[k][q] + in.beta * mm[k][q];
        }
        if (there) t += (double)v[k][q] * (double)v[k][q];
      }
      if (m_old && there) rt_store<float, V>(m_new + at + i, mm[k]);
    }
  }
  s[threadIdx.x] = t;
  for (int h = 128; h; h >>= 1) {
    __syncthreads();
    if ((int)threadIdx.x < h) s[threadIdx.x] += s[threadIdx.x + h];
  }
  if (threadIdx.x == 0) part[(size_t)blockIdx.y * OU_PARTS + blockIdx.x] = s[0];
}

// sum of squares of one matrix from its parts, in every lane
__device__ __forceinline__ double ou_squares(const double* part, int parts) {
  double t = 0.0;
  for (int i = threadIdx.x & 63; i < parts; i += 64) t += part[i];
  for (int h = 32; h; h >>= 1) t += __shfl_xor(t, h);
  return t;
}

__device__ __forceinline__ double ou_inverse(double squares) { return squares == 0.0 ? 0.0 : 1.0 / sqrt(squares); }   // (a NaN stays one)
__device__ __forceinline__ double ou_sigma0(double squares) { return sqrt(squares) / (sqrt(squares) + OU_EPS); }

// Factors of step k (0, 1, ..) of a matrix: X_{k+1} = x X + (g G + gg G^2) X, and sigma_{k+1}
struct OuStep { float x, g, gg, sigma; };
__device__ __forceinline__ OuStep ou_step(double sigma, int k) {
  for (; k > 0 && sigma < 1.0; --k) sigma = fmin(1.0, (double)OU_A * sigma);
  const double next = fmin(1.0, (double)OU_A * sigma), r = next < 1.0 ? 1.0 / (double)OU_A : sigma, s2 = sigma * sigma;
  return {(float)(r * OU_A), (float)(r * OU_B * s2), (float)(r * OU_C * s2 * s2), (float)next};
}

// ---- x_0 in pieces, in both layouts: 64 x 64 tiles.  x [hi, lo][np][mp], xt [hi, lo][mp][np] per matrix
template <class T>
__global__ __launch_bounds__(256) void ou_pieces_kernel(OuShape p, OuInput<T> in, const double* part, int parts, double* sigma, _Float16* x,
                                                        _Float16* xt) {
  __shared__ float tile[64][65];    // [i][j] of x
  const size_t z = blockIdx.z;
  const int i0 = blockIdx.y * 64, j0 = blockIdx.x * 64, t = threadIdx.x;
  float v[16];
#pragma unroll
  for (int k = 0; k < 16; ++k) {                     // (never under a condition: all loads before the first is waited for)
    const int a = (t >> 6) + 4 * k, b = t & 63;       // b along the caller's rows
    const int i = min(i0 + (p.tall ? b : a), p.n - 1), j = min(j0 + (p.tall ? a : b), p.m - 1);
    v[k] = ou_value(in, z * p.rows * p.cols + (p.tall ? (size_t)j * p.cols + i : (size_t)i * p.cols + j));
  }
  const double squares = ou_squares(part + z * OU_PARTS, parts), inv = ou_inverse(squares) * (double)OU_SX;
  if (blockIdx.x == 0 && blockIdx.y == 0 && t == 0) sigma[z] = ou_sigma0(squares);
#pragma unroll
  for (int k = 0; k < 16; ++k) {
    const int a = (t >> 6) + 4 * k, b = t & 63;
    const bool there = i0 + (p.tall ? b : a) < p.n && j0 + (p.tall ? a : b) < p.m;
    const float x0 = there ? (float)((double)v[k] * inv) : 0.0f;
    if (p.tall) tile[b][a] = x0; else tile[a][b] = x0;
  }
  __syncthreads();
  const size_t plane = (size_t)p.np * p.mp;
  for (int k = 0; k < 2; ++k) {
    const int r = (t >> 3) + 32 * k, c = (t & 7) * 8;
    ou_h8 hi, lo, thi, tlo;
#pragma unroll
    for (int q = 0; q < 8; ++q) {
      _Float16 h, l;
      ou_cut(tile[r][c + q], h, l);
      hi[q] = h; lo[q] = l;
      ou_cut(tile[c + q][r], h, l);
      thi[q] = h; tlo[q] = l;
    }
    _Float16* to = x + z * 2 * plane + (size_t)(i0 + r) * p.mp + j0 + c;
    _Float16* tt = xt + z * 2 * plane + (size_t)(j0 + r) * p.np + i0 + c;
    *(ou_h8*)to = hi;
    *(ou_h8*)tt = thi;
    *(ou_h8*)(to + plane) = lo;
    *(ou_h8*)(tt + plane) = tlo;
  }
}

// ---- products ----------------------------------------------------------------------------------------------------------
enum OuProduct { OU_GRAM, OU_POLY, OU_UPDATE, OU_LAST };

template <class T>
struct OuOut {     // y = q, or keep W - scale q
  T* y;
  const float* W;
  float keep, scale;
  bool eights;        // rows of y in aligned eights
  bool fours;         // tall, and rows of all the caller's matrices in aligned fours
};

struct OuOperands {
  const _Float16 *A, *B;   // per matrix [hi, lo][I][K], [hi, lo][J][K]
  _Float16 *C, *Ct;        // results in pieces: C [hi, lo][J][I] (the transpose; g and p are symmetric), Ct [hi, lo][I][J]
  int I, J, K;             // multiples of 64
  const double* sigma;     // sigma_0 of every matrix
  int step;
};

typedef const __attribute__((address_space(1))) void* ou_gp;
typedef __attribute__((address_space(3))) void* ou_lp;

// waits until at most N loads of this wave are under way (loads return in order), then for the other waves
template <int N>
__device__ __forceinline__ void ou_loads_then_barrier() {
  static_assert(N < 64, "the counter of loads has six bits");
  asm volatile("" ::: "memory");
  __builtin_amdgcn_s_waitcnt((N & 15) | 7 << 4 | 15 << 8 | (N >> 4) << 14);
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
}

// waits for LDS alone, not for stores to memory
__device__ __forceinline__ void ou_lds_barrier() {
  rb_release_barrier();
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "workgroup", "local");
}

// C = A B^T of one tile TILE x TILE: four waves, each a quarter (TILE / 2 squared) in 32 x 32 blocks; for tiles of 64 twice four, each
// with half of a turn's contraction (the chain of dependent products of a turn is what a small tile waits for).  64 contraction indices a
// turn, brought straight into one of STAGES LDS buffers, STAGES - 1 turns ahead: with one wave per SIMD nothing else hides the way to
// memory.  A row of 128 bytes lies in LDS as eight pieces of 16 bytes, piece c at place c ^ (row / 2 & 7): the sixteen lanes whose
// 16-byte reads go together (0-3, 12-15, 20-23, 24-27 and the others) then meet all 64 banks (with c ^ (row & 7) half of the LDS cycles were
// conflicts).  The operands of a step of 16 are read from LDS while the products of the one before run.
template <int TILE>
struct OuTile {
  static constexpr int STAGES = TILE == 128 ? 2 : 4;
  static constexpr int SETS = TILE == 64 ? 2 : 1, THREADS = 256 * SETS;   // sets of four waves
  static constexpr int PLANE = TILE * 8, STAGE = 4 * PLANE;              // uint4
  static constexpr int LOADS = 4 * TILE / 32 / SETS;                      // of a wave per turn
  static constexpr size_t LDS = (size_t)STAGES * STAGE * 16;
};

template <class T, int TILE, OuProduct WHAT>
__global__ __launch_bounds__((OuTile<TILE>::THREADS)) void ou_product_kernel(OuShape p, OuOperands o, OuOut<T> out) {
  extern __shared__ uint4 smem[];                     // [STAGES][2 operands][hi, lo][TILE][8]
  typedef OuTile<TILE> Tile;
  constexpr int HALF = TILE / 2, B = HALF / 32, PLANE = Tile::PLANE, STAGE = Tile::STAGE, STAGES = Tile::STAGES;
  constexpr int SETS = Tile::SETS, THREADS = Tile::THREADS, ROUNDS = TILE / 32 / SETS;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const size_t z = blockIdx.z;
  const int i0 = blockIdx.y * TILE, j0 = blockIdx.x * TILE;
  const size_t plane_a = (size_t)o.I * o.K, plane_b = (size_t)o.J * o.K;
  const _Float16* A = o.A + z * 2 * plane_a;
  const _Float16* Bm = o.B + z * 2 * plane_b;
  const int wi = (wave >> 1 & 1) * HALF, wj = (wave & 1) * HALF, set = wave >> 2;

  // lane's place in a load of eight rows
  const int lrow = lane >> 3, lpiece = (lane & 7) ^ ((wave & 1) << 2 | lrow >> 1);
  const _Float16 *pa[ROUNDS], *pb[ROUNDS];
#pragma unroll
  for (int r = 0; r < ROUNDS; ++r) {
    const int row = (r * 4 * SETS + wave) * 8 + lrow;
    pa[r] = A + (size_t)min(i0 + row, o.I - 1) * o.K + lpiece * 8;
    pb[r] = Bm + (size_t)min(j0 + row, o.J - 1) * o.K + lpiece * 8;
  }
  auto fetch = [&](int turn, int stage) {
    uint4* to = smem + stage * STAGE + wave * 64;
#pragma unroll
    for (int q = 0; q < 2; ++q)
#pragma unroll
      for (int r = 0; r < ROUNDS; ++r) {
        __builtin_amdgcn_global_load_lds((ou_gp)(pa[r] + q * plane_a + turn * 64), (ou_lp)(to + q * PLANE + r * 256 * SETS), 16, 0, 0);
        __builtin_amdgcn_global_load_lds((ou_gp)(pb[r] + q * plane_b + turn * 64), (ou_lp)(to + (2 + q) * PLANE + r * 256 * SETS), 16, 0, 0);
      }
  };

  ou_f16v acc[B][B];
#pragma unroll
  for (int a = 0; a < B; ++a)
#pragma unroll
    for (int b = 0; b < B; ++b)
#pragma unroll
      for (int i = 0; i < 16; ++i) acc[a][b][i] = 0.0f;
  const int r32 = lane & 31, hh = lane >> 5;
  const int turns = o.K / 64;
#pragma unroll
  for (int k = 0; k < STAGES - 1; ++k) fetch(min(k, turns - 1), k);
  int stage = 0;
  for (int k = 0; k < turns; ++k) {
    ou_loads_then_barrier<(STAGES - 2) * Tile::LOADS>();   // this turn's operands are in LDS, the buffer of the turn before is free
    // (past the end the last turn is fetched again: the number of loads under way is the same in every turn)
    fetch(min(k + STAGES - 1, turns - 1), stage ? stage - 1 : STAGES - 1);
    const uint4* sa = smem + stage * STAGE + (wi + r32) * 8;
    const uint4* sb = smem + stage * STAGE + 2 * PLANE + (wj + r32) * 8;
    stage = stage + 1 == STAGES ? 0 : stage + 1;
    ou_h8 a[2][B][2], b[2][B][2];
    auto operands = [&](int s) {
      const int place = (2 * (s + set * (4 / SETS)) + hh) ^ (r32 >> 1 & 7);
#pragma unroll
      for (int x = 0; x < B; ++x)
#pragma unroll
        for (int q = 0; q < 2; ++q) {
          a[s & 1][x][q] = __builtin_bit_cast(ou_h8, sa[q * PLANE + x * 256 + place]);
          b[s & 1][x][q] = __builtin_bit_cast(ou_h8, sb[q * PLANE + x * 256 + place]);
        }
    };
    operands(0);
#pragma unroll
    for (int s = 0; s < 4 / SETS; ++s) {
      if (s + 1 < 4 / SETS) operands(s + 1);
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int t = 0; t < 3; ++t)     // lo hi, hi lo, hi hi
#pragma unroll
        for (int x = 0; x < B; ++x)
#pragma unroll
          for (int y = 0; y < B; ++y)
            acc[x][y] = __builtin_amdgcn_mfma_f32_32x32x16_f16(a[s & 1][x][t == 0], b[s & 1][y][t == 1], acc[x][y], 0, 0, 0);
      __builtin_amdgcn_sched_barrier(0);
    }
  }
  ou_loads_then_barrier<0>();      // (no load to LDS outlives the workgroup)

  // Results go through LDS, so that whole lines are read and written: a lane holds column j = lane & 31 of its blocks and four times
  // four neighbouring rows i; row j of the tile in LDS, its pieces of four values exchanged by j.
  constexpr float unscale = WHAT == OU_GRAM ? 1.0f / (OU_SX * OU_SX) : WHAT == OU_POLY ? 1.0f / (OU_SG * OU_SG) : 1.0f / (OU_SP * OU_SX);
  constexpr float scale = WHAT == OU_GRAM ? OU_SG : WHAT == OU_POLY ? OU_SP : OU_SX;
  constexpr int SLOTS = TILE / 4;
  float4* tile = (float4*)smem;                      // [j][SLOTS]
  auto slot = [](int j, int i4) { return j * SLOTS + (i4 ^ (j & (SLOTS - 1))); };
#pragma unroll
  for (int part = 0; part < SETS; ++part) {
    if (set == part)
#pragma unroll
      for (int x = 0; x < B; ++x)
#pragma unroll
        for (int y = 0; y < B; ++y)
#pragma unroll
          for (int r = 0; r < 4; ++r) {
            float4& t = tile[slot(wj + 32 * y + r32, (wi + 32 * x + 8 * r + 4 * hh) >> 2)];
            float4 v = make_float4(acc[x][y][4 * r], acc[x][y][4 * r + 1], acc[x][y][4 * r + 2], acc[x][y][4 * r + 3]);
            if (part) {
              v.x += t.x; v.y += t.y; v.z += t.z; v.w += t.w;
            }
            t = v;
          }
    if (part + 1 < SETS) ou_lds_barrier();
  }
  // Whatever has to be loaded is loaded before the first result is stored: loads and stores return in order, and a load behind a store
  // would wait for it (so did barriers that wait for stores).
  const size_t plane_c = (size_t)o.I * o.J;
  constexpr int ACROSS = TILE / 8, ITEMS = TILE * ACROSS / THREADS;   // threads along a row, eight values each
  constexpr bool STEP = WHAT == OU_UPDATE || WHAT == OU_LAST;   // p x
  constexpr bool OLD = WHAT == OU_POLY || STEP;                 // + b g, or + a x
  const int n = p.n, m = p.m, across = tid % ACROSS * 8;
  ou_h8 oh[OLD ? ITEMS : 1], ol[OLD ? ITEMS : 1];
  auto along_i = [&](int e, int& i, int& j, int& jl) {            // eight i of one j
    jl = tid / ACROSS + e * (THREADS / ACROSS);
    i = i0 + across;
    j = j0 + jl;
    return i < o.I && j < o.J;
  };
  if (OLD)
#pragma unroll
    for (int e = 0; e < ITEMS; ++e) {
      int i, j, jl;
      along_i(e, i, j, jl);
      const _Float16* old = (STEP ? Bm : A) + (size_t)min(j, o.J - 1) * o.I + min(i, o.I - 8);
      oh[e] = *(const ou_h8*)old;
      ol[e] = *(const ou_h8*)(old + plane_c);
    }
  const OuStep step = OLD ? ou_step(o.sigma[z], o.step) : OuStep{};
  const bool flip = WHAT == OU_UPDATE || (WHAT == OU_LAST && !p.tall);     // rows of (another) result run along j
  float keep[WHAT == OU_LAST ? ITEMS : 1][8];
  if (WHAT == OU_LAST && out.W)
#pragma unroll
    for (int e = 0; e < ITEMS; ++e) {
      const int r = (flip ? i0 : j0) + tid / ACROSS + e * (THREADS / ACROSS), c = (flip ? j0 : i0) + across;
      const float* w = out.W + z * n * m + (size_t)min(r, (flip ? n : m) - 1) * p.cols;
#pragma unroll
      for (int q = 0; q < 8; ++q) keep[e][q] = out.keep * w[min(c + q, p.cols - 1)];
    }
  // (r, c) of the caller's matrix
  auto write_last = [&](int e, int r, int c, float (&v)[8]) {
    if (r >= p.rows || c >= p.cols) return;
#pragma unroll
    for (int q = 0; q < 8; ++q)
      v[q] = out.W ? keep[e][q] - out.scale * step.sigma * v[q] : step.sigma * v[q];
    T* to = out.y + z * n * m + (size_t)r * p.cols + c;
    if (out.eights) {
      rt_store<T, 8>(to, v);
    } else {
#pragma unroll
      for (int q = 0; q < 8; ++q)
        if (c + q < p.cols) to[q] = (T)v[q];
    }
  };
  ou_lds_barrier();
#pragma unroll
  for (int e = 0; e < ITEMS; ++e) {
    int i, j, jl;
    if (!along_i(e, i, j, jl)) continue;
    const float4 lo4 = tile[slot(jl, across >> 2)], hi4 = tile[slot(jl, (across >> 2) + 1)];
    float v[8] = {lo4.x, lo4.y, lo4.z, lo4.w, hi4.x, hi4.y, hi4.z, hi4.w};
#pragma unroll
    for (int q = 0; q < 8; ++q) v[q] *= unscale;
    if (OLD)
#pragma unroll
      for (int q = 0; q < 8; ++q) {
        const float before = (float)oh[e][q] + (float)ol[e][q];
        v[q] = STEP ? v[q] + step.x * (1.0f / OU_SX) * before : step.gg * v[q] + step.g * (1.0f / OU_SG) * before;
      }
    if (flip) {
      tile[slot(jl, across >> 2)] = make_float4(v[0], v[1], v[2], v[3]);
      tile[slot(jl, (across >> 2) + 1)] = make_float4(v[4], v[5], v[6], v[7]);
    }
    if (WHAT == OU_LAST) {
      if (!flip) write_last(e, j, i, v);
      continue;
    }
    ou_h8 hi, lo;
#pragma unroll
    for (int q = 0; q < 8; ++q) {
      _Float16 h, l;
      ou_cut(v[q] * scale, h, l);
      hi[q] = h; lo[q] = l;
    }
    _Float16* c = o.C + z * 2 * plane_c + (size_t)j * o.I + i;
    *(ou_h8*)c = hi;
    *(ou_h8*)(c + plane_c) = lo;
  }
  if (!flip) return;
  ou_lds_barrier();
  const float* flat = (const float*)smem;
#pragma unroll
  for (int e = 0; e < ITEMS; ++e) {                                // eight j of one i
    const int il = tid / ACROSS + e * (THREADS / ACROSS), i = i0 + il, j = j0 + across;
    if (i >= o.I || j >= o.J) continue;
    float v[8];
#pragma unroll
    for (int q = 0; q < 8; ++q) v[q] = flat[4 * slot(across + q, il >> 2) + (il & 3)];
    if (WHAT == OU_LAST) {
      write_last(e, i, j, v);
      continue;
    }
    ou_h8 hi, lo;
#pragma unroll
    for (int q = 0; q < 8; ++q) {
      _Float16 h, l;
      ou_cut(v[q] * scale, h, l);
      hi[q] = h; lo[q] = l;
    }
    _Float16* ct = o.Ct + z * 2 * plane_c + (size_t)i * o.J + j;
    *(ou_h8*)ct = hi;
    *(ou_h8*)(ct + plane_c) = lo;
  }
}

// ---- n <= 64: all of g and p in one workgroup ----------------------------------------------------------------------------------
// The long side is cut into slabs of up to 256 columns of x (rows of x^T), 32 to a wave.  A launch takes the parts of g = x x^T of all
// slabs, and every workgroup adds them (always in the same order), makes p for itself, takes its slab one step further and leaves
// the slab's part of the next g.  So a step is one launch; where one slab holds everything (ALONE) all steps are one.
//
// Everything stays in the order in which 32 x 32 products land in the accumulators: a lane holds one column and sixteen rows, eight and
// eight (fragment t = 0, 1).  Read as an operand, the lane's column is the operand's row and the sixteen rows are contraction indices, in an
// order that does not matter as long as both operands share it.  So the fragments of g serve as both operands of g g (g and p are
// symmetric), those of x (lane = k, registers = i) with p's make the next x, and x^T (lane = column j, registers = rows k), both operands of g,
// is x times the identity: no value ever changes lanes but in the matrix cores.
// Until step 1 a slab is scaled by its own norm: the sums of squares of the others come with their parts of G, no pass for |u| alone.
//
// g g keeps lo lo as well: on its diagonal these are squares, which add up instead of averaging out (8 x 8 to 64 x 64 fp32, 30 matrices each, against
// 64 bits: 0.65 to 0.98e-6 off with it, 0.78 to 1.3e-6 without, torch in fp32 0.64 to 1.1e-6; 15 x 32 x 32 12.7 us against 12.8).
//
// What bounds it: the chain of dependent products, conversions and barriers of a step, and the reading of the parts (16 KB a slab from L2).
// Measured, a step of the optimiser: 15 x 32 x 32 15.7 us in one launch, 3 x 2688 x 64 65 us in six.
constexpr int OS_ROWS = 256, OS_WAVES = OS_ROWS / 32;
constexpr int OS_SLABS = 64;                 // more columns than this many slabs: a workgroup takes several turns

struct OsPlace {
  uint4* x;               // [batch][slabs * turns][8 waves][NB blocks][2 fragments][2 pieces][64 lanes] between two launches
  const float4* part_in;  // [batch][slabs][NB^2 blocks][4][64 lanes]: parts of g of this step
  float4* part_out;       // of the next one
  double* squares;        // [batch][slabs]: sums of squares of the slabs
  double* sigma;          // [batch], from step 1 on
  int slabs, turns;
};

template <int NB>
struct OsLds {
  static constexpr int FRAGMENTS = NB * NB * 2 * 2 * 64;                // uint4: g or p, [rows block][columns block][t][piece][lane]
  static constexpr int PARTS = NB * NB * 4 * 64;                        // float4: one wave's part of g
  static size_t bytes(int waves) { return (size_t)(2 * FRAGMENTS + waves * PARTS) * 16; }
};

// Eight values times `scale` -> hi and lo.  scale has to be a power of two: the compiler may round the product to 11 bits in one step or in
// two, hi and the remainder each in its own way, which is the same only where the product is exact.
__device__ __forceinline__ void os_cut(const float (&v)[8], float scale, ou_h8& hi, ou_h8& lo) {
#pragma unroll
  for (int q = 0; q < 8; ++q) {
    const _Float16 h = (_Float16)(v[q] * scale);
    hi[q] = h;
    lo[q] = (_Float16)__builtin_fmaf(v[q], scale, -(float)h);
  }
}

__device__ __forceinline__ ou_f16v os_product(const ou_h8 (&a)[2], const ou_h8 (&b)[2], ou_f16v acc) {   // [0] = hi, [1] = lo
  acc = __builtin_amdgcn_mfma_f32_32x32x16_f16(a[1], b[0], acc, 0, 0, 0);
  acc = __builtin_amdgcn_mfma_f32_32x32x16_f16(a[0], b[1], acc, 0, 0, 0);
  return __builtin_amdgcn_mfma_f32_32x32x16_f16(a[0], b[0], acc, 0, 0, 0);
}

__device__ __forceinline__ ou_f16v os_zero() {
  ou_f16v v;
#pragma unroll
  for (int i = 0; i < 16; ++i) v[i] = 0.0f;
  return v;
}

// sum over the workgroup, in every thread
__device__ __forceinline__ double os_sum(double t, double* s) {
  for (int h = 32; h; h >>= 1) t += __shfl_xor(t, h);
  if ((threadIdx.x & 63) == 0) s[threadIdx.x >> 6] = t;
  __syncthreads();
  t = 0.0;
  for (int w = 0; w < (int)blockDim.x >> 6; ++w) t += s[w];
  __syncthreads();
  return t;
}

template <class T, int NB, bool ALONE>
__global__ __launch_bounds__(512) void ou_slab_kernel(OuShape p, OuInput<T> in, const float* m_old, float* m_new, OsPlace w, int step,
                                                      int steps, OuOut<T> out) {
  extern __shared__ uint4 smem[];
  typedef OsLds<NB> Lds;
  uint4* sg = smem;
  uint4* sp = smem + Lds::FRAGMENTS;
  float4* sums = (float4*)(smem + 2 * Lds::FRAGMENTS);
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), waves = blockDim.x >> 6;
  const int r32 = lane & 31, hh = lane >> 5, slab = blockIdx.x, turns = ALONE ? 1 : w.turns;
  const size_t z = blockIdx.y, at0 = z * p.rows * p.cols;
  auto fragment = [&](const uint4* from, int a, int b, int t, ou_h8 (&v)[2]) {
    const uint4* f = from + ((a * NB + b) * 2 + t) * 128 + lane;
    v[0] = __builtin_bit_cast(ou_h8, f[0]);
    v[1] = __builtin_bit_cast(ou_h8, f[64]);
  };
  // First of the four elements of the caller's matrix (one apart, or a row) for registers 4 r .. 4 r + 3 of block b of fragments of x, and
  // how many of them there are.
  const size_t apart = p.tall ? 1 : p.cols;
  auto place = [&](int first, int b, int r, size_t& at) {
    const int i = 32 * b + 8 * r + 4 * hh, c = first + r32;
    at = at0 + (p.tall ? (size_t)c * p.cols + i : (size_t)i * p.cols + c);
    return c < p.m ? min(4, p.n - i) : 0;
  };
  auto load4 = [&](const auto* from, size_t at, int there, float (&v)[4]) {
#pragma unroll
    for (int q = 0; q < 4; ++q) v[q] = 0.0f;
    if (out.fours && there == 4) {
      rt_load(from + at, v);
    } else {
#pragma unroll
      for (int q = 0; q < 4; ++q)
        if (q < there) v[q] = (float)from[at + q * apart];
    }
  };
  auto store4 = [&](auto* to, size_t at, int there, const float (&v)[4]) {
    if (out.fours && there == 4) {
      rt_store(to + at, v);
    } else {
#pragma unroll
      for (int q = 0; q < 4; ++q)
        if (q < there) to[at + q * apart] = (std::remove_pointer_t<decltype(to)>)v[q];
    }
  };
  // u of one turn's rows; the new momentum on the way
  auto input = [&](int first, bool write, float (&u)[NB][16]) {
#pragma unroll
    for (int b = 0; b < NB; ++b)
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        size_t at;
        const int there = place(first, b, r, at);
        float v[4], mm[4];
        load4(in.u, at, there, v);
        if (m_old) {
          load4(write ? m_old : m_new, at, there, mm);
#pragma unroll
          for (int q = 0; q < 4; ++q) {
            if (write) mm[q] = in.beta * mm[q] + v[q];
            v[q] = v[q] + in.beta * mm[q];
          }
          if (write) store4(m_new, at, there, mm);
        }
#pragma unroll
        for (int q = 0; q < 4; ++q) u[b][4 * r + q] = v[q];
      }
  };

  ou_h8 x[NB][2][2];           // fragments of x: [block][t][piece]
  ou_f16v g[NB][NB];
  auto row_of = [&](int turn) { return (slab * turns + turn) * OS_ROWS + wave * 32; };      // first row of x^T of this wave
  auto kept = [&](int turn) { return w.x + (((z * w.slabs + slab) * turns + turn) * OS_WAVES + wave) * (NB * 256) + lane; };
  auto clear = [&]() {
#pragma unroll
    for (int a = 0; a < NB; ++a)
#pragma unroll
      for (int b = 0; b < NB; ++b) g[a][b] = os_zero();
  };
  auto load_x = [&](int turn) {
    const uint4* from = kept(turn);
#pragma unroll
    for (int b = 0; b < NB; ++b)
#pragma unroll
      for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int q = 0; q < 2; ++q) x[b][t][q] = __builtin_bit_cast(ou_h8, from[((b * 2 + t) * 2 + q) * 64]);
  };
  auto store_x = [&](int turn) {
    uint4* to = kept(turn);
#pragma unroll
    for (int b = 0; b < NB; ++b)
#pragma unroll
      for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int q = 0; q < 2; ++q) to[((b * 2 + t) * 2 + q) * 64] = __builtin_bit_cast(uint4, x[b][t][q]);
  };
  auto cut = [&](const ou_f16v& acc, float scale, ou_h8 (&to)[2][2]) {
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      float v[8];
#pragma unroll
      for (int q = 0; q < 8; ++q) v[q] = acc[8 * t + q];
      os_cut(v, scale, to[t][0], to[t][1]);
    }
  };
  auto add_g = [&](const ou_h8 (&xt)[NB][2][2]) {
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
      for (int a = 0; a < NB; ++a)
#pragma unroll
        for (int b = 0; b < NB; ++b) g[a][b] = os_product(xt[a][t], xt[b][t], g[a][b]);
  };

  // x^T of block b of x by a product with the identity: exact, as every value is two pieces.  (Made by a product with p of its own, as x
  // is, x^T would be rounded apart from x: twice the error of a result of full rank.)
  auto turned = [&](int b, ou_h8 (&to)[2][2]) {
    ou_f16v rows = os_zero();
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      ou_h8 one;
#pragma unroll
      for (int q = 0; q < 8; ++q) one[q] = (_Float16)(16 * t + 8 * (q >> 2) + 4 * hh + (q & 3) == r32 ? 1.0f : 0.0f);
      rows = __builtin_amdgcn_mfma_f32_32x32x16_f16(x[b][t][1], one, rows, 0, 0, 0);
      rows = __builtin_amdgcn_mfma_f32_32x32x16_f16(x[b][t][0], one, rows, 0, 0, 0);
    }
    cut(rows, 1.0f, to);
  };

  // step 0: X = u / |u| (of the slab) and its G
  double sigma0 = 0.0;
  auto begin = [&]() {
    float u[NB][16];
    double t = 0.0;
    for (int turn = 0; turn < turns; ++turn) {
      input(row_of(turn), true, u);
#pragma unroll
      for (int b = 0; b < NB; ++b)
#pragma unroll
        for (int q = 0; q < 16; ++q) t += (double)u[b][q] * (double)u[b][q];
    }
    t = os_sum(t, (double*)smem);
    const double inverse = ou_inverse(t);
    if (ALONE) sigma0 = ou_sigma0(t);
    if (!ALONE && tid == 0) w.squares[z * w.slabs + slab] = t;
    clear();
    for (int turn = 0; turn < turns; ++turn) {
      if (turns > 1) input(row_of(turn), false, u);
      ou_h8 xt[NB][2][2];
#pragma unroll
      for (int b = 0; b < NB; ++b) {
#pragma unroll
        for (int t = 0; t < 2; ++t) {
          float v[8];
#pragma unroll
          for (int q = 0; q < 8; ++q) v[q] = (float)((double)u[b][8 * t + q] * inverse);
          os_cut(v, OU_SX, x[b][t][0], x[b][t][1]);
        }
        turned(b, xt[b]);
      }
      if (!ALONE) store_x(turn);
      add_g(xt);
    }
  };

  // p of step k = 1, 2, .. in LDS, from the parts of G of all waves or of all slabs; in step 1 times the scale of this slab's X, as are the
  // factors that are returned
  auto make_p = [&](int k) {
    const bool first = k == 1;
    double norm = 1.0, factor = 1.0;
    if (!ALONE) {
      if (first) {
        const double t = ou_squares(w.squares + z * w.slabs, w.slabs);
        norm = ou_inverse(t);
        factor = sqrt(w.squares[z * w.slabs + slab]) * norm;
        sigma0 = ou_sigma0(t);
        if (slab == 0 && tid == 0) w.sigma[z] = sigma0;
      } else {
        sigma0 = w.sigma[z];
      }
    }
    OuStep at_step = ou_step(sigma0, k - 1);
    at_step.x *= (float)factor;
    at_step.g *= (float)factor;
    at_step.gg *= (float)factor;
    const int parts = ALONE ? waves : w.slabs;
    const float4* from = ALONE ? sums : w.part_in + z * w.slabs * Lds::PARTS;
    for (int e = tid; e < NB * NB * 128; e += blockDim.x) {        // the values of one fragment are two float4 of a lane
      const int at = (e >> 6) * 128 + (e & 63);
      float v[8] = {};
#pragma unroll 4
      for (int t = 0; t < parts; ++t) {
        const float4 lo = from[t * Lds::PARTS + at], hi = from[t * Lds::PARTS + at + 64];
        float f = 1.0f;
        if (!ALONE && first) f = (float)(w.squares[z * w.slabs + t] * norm * norm);
        v[0] += f * lo.x; v[1] += f * lo.y; v[2] += f * lo.z; v[3] += f * lo.w;
        v[4] += f * hi.x; v[5] += f * hi.y; v[6] += f * hi.z; v[7] += f * hi.w;
      }
      ou_h8 h, l;
      os_cut(v, OU_SG, h, l);
      sg[at] = __builtin_bit_cast(uint4, h);
      sg[at + 64] = __builtin_bit_cast(uint4, l);
    }
    __syncthreads();
    for (int e = wave; e < NB * NB; e += waves) {                  // a block a wave
      const int a = e / NB, b = e % NB;
      ou_f16v acc = os_zero();
#pragma unroll
      for (int c = 0; c < NB; ++c)
#pragma unroll
        for (int t = 0; t < 2; ++t) {
          ou_h8 ga[2], gb[2];
          fragment(sg, c, a, t, ga);
          fragment(sg, c, b, t, gb);
          acc = __builtin_amdgcn_mfma_f32_32x32x16_f16(ga[1], gb[1], acc, 0, 0, 0);
          acc = os_product(ga, gb, acc);
        }
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        ou_h8 ge[2], h, l;
        fragment(sg, a, b, t, ge);
        float v[8];
#pragma unroll
        for (int q = 0; q < 8; ++q) {
          v[q] = at_step.gg * (1.0f / (OU_SG * OU_SG)) * acc[8 * t + q] + at_step.g * (1.0f / OU_SG) * ((float)ge[0][q] + (float)ge[1][q]);
        }
        os_cut(v, OU_SP, h, l);
        uint4* to = sp + (e * 2 + t) * 128 + lane;
        to[0] = __builtin_bit_cast(uint4, h);
        to[64] = __builtin_bit_cast(uint4, l);
      }
    }
    __syncthreads();
    return at_step;
  };

  // the next X (times OU_SP OU_SX), row block b
  auto times_p = [&](int b, const OuStep& f) {
    ou_f16v acc = os_zero();
#pragma unroll
    for (int c = 0; c < NB; ++c)
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        ou_h8 pf[2];
        fragment(sp, c, b, t, pf);
        acc = os_product(pf, x[c][t], acc);
      }
    const float a = f.x * OU_SP;
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
      for (int q = 0; q < 8; ++q) acc[8 * t + q] += a * ((float)x[b][t][0][q] + (float)x[b][t][1][q]);
    return acc;
  };

  auto advance = [&](const OuStep& f) {
    clear();
    for (int turn = 0; turn < turns; ++turn) {
      if (!ALONE) load_x(turn);
      ou_h8 xt[NB][2][2];
      ou_f16v next[NB];
#pragma unroll
      for (int b = 0; b < NB; ++b) next[b] = times_p(b, f);
#pragma unroll
      for (int b = 0; b < NB; ++b) cut(next[b], 1.0f / OU_SP, x[b]);
      if (!ALONE) store_x(turn);
#pragma unroll
      for (int b = 0; b < NB; ++b) turned(b, xt[b]);
      add_g(xt);
    }
  };

  auto finish = [&](const OuStep& f) {
    for (int turn = 0; turn < turns; ++turn) {
      float old[NB][4][4];
      if (out.W)
#pragma unroll
        for (int b = 0; b < NB; ++b)
#pragma unroll
          for (int r = 0; r < 4; ++r) {
            size_t at;
            const int there = place(row_of(turn), b, r, at);
            load4(out.W, at, there, old[b][r]);
          }
      if (!ALONE) load_x(turn);
#pragma unroll
      for (int b = 0; b < NB; ++b) {
        const ou_f16v last = times_p(b, f);
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          size_t at;
          const int there = place(row_of(turn), b, r, at);
          float v[4];
#pragma unroll
          for (int q = 0; q < 4; ++q) {
            v[q] = last[4 * r + q] * (1.0f / (OU_SP * OU_SX)) * f.sigma;
            if (out.W) v[q] = out.keep * old[b][r][q] - out.scale * v[q];
          }
          store4(out.y, at, there, v);
        }
      }
    }
  };

  auto publish = [&]() {
#pragma unroll
    for (int a = 0; a < NB; ++a)
#pragma unroll
      for (int b = 0; b < NB; ++b)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          constexpr float v = 1.0f / (OU_SX * OU_SX);
          sums[wave * Lds::PARTS + ((a * NB + b) * 4 + r) * 64 + lane] =
              make_float4(g[a][b][4 * r] * v, g[a][b][4 * r + 1] * v, g[a][b][4 * r + 2] * v, g[a][b][4 * r + 3] * v);
        }
    __syncthreads();
    if (ALONE) return;
    for (int e = tid; e < Lds::PARTS; e += blockDim.x) {
      float4 t = sums[e];
      for (int i = 1; i < waves; ++i) {
        const float4 v = sums[i * Lds::PARTS + e];
        t.x += v.x; t.y += v.y; t.z += v.z; t.w += v.w;
      }
      w.part_out[(z * w.slabs + slab) * Lds::PARTS + e] = t;
    }
  };

  if (ALONE) {
    begin();
    publish();
    for (int k = 1; k < steps; ++k) {
      advance(make_p(k));
      publish();
    }
    finish(make_p(steps));
  } else if (step == 0) {
    begin();
    publish();
  } else {
    const OuStep f = make_p(step);
    if (step < steps) {
      advance(f);
      publish();
    } else {
      finish(f);
    }
  }
}

OuShape ou_shape(int32_t batch, int32_t rows, int32_t cols) {
  OuShape p;
  p.batch = batch; p.rows = rows; p.cols = cols;
  p.n = rows < cols ? rows : cols;
  p.m = rows < cols ? cols : rows;
  p.np = (p.n + 63) / 64 * 64;
  p.mp = (p.m + 63) / 64 * 64;
  p.tall = rows > cols;
  return p;
}

struct OsSpace { size_t squares, sigma, x, g, bytes; int slabs, turns, blocks; };
OsSpace os_space(const OuShape& p) {
  OsSpace s;
  const int slabs = (p.m + OS_ROWS - 1) / OS_ROWS;
  s.blocks = p.n <= 32 ? 1 : 2;
  s.turns = (slabs + OS_SLABS - 1) / OS_SLABS;
  s.slabs = (slabs + s.turns - 1) / s.turns;
  s.squares = 0;
  s.sigma = ou_align((size_t)p.batch * s.slabs * sizeof(double));
  s.x = s.sigma + ou_align((size_t)p.batch * sizeof(double));
  s.g = s.x + ou_align((size_t)p.batch * s.slabs * s.turns * OS_WAVES * s.blocks * 256 * sizeof(uint4));
  s.bytes = slabs == 1 ? 256 : s.g + 2 * ou_align((size_t)p.batch * s.slabs * s.blocks * s.blocks * 256 * sizeof(float4));
  return s;
}

int ou_parts(size_t size) { return (int)(size > (size_t)OU_PARTS * OU_ROUND ? OU_PARTS : (size + OU_ROUND - 1) / OU_ROUND); }

// Side of at most 32: one block of 32 x 32 holds g, otherwise four do (15 matrices 32 x 32: a step of the optimiser 15.7 us with one, 42 us
// with four; 3 of 2,000 x 32: 38 and 57).
template <class T, int NB>
int ou_run_slabs(egnn_ctx* ctx, const OuShape& p, const OuInput<T>& in, const float* m_old, float* m_new, int steps,
                 const OuOut<T>& out, void* ws, hipStream_t st) {
  const OsSpace s = os_space(p);
  const size_t most = OsLds<NB>::bytes(OS_WAVES);
  if (p.m <= OS_ROWS) {
    const int waves = (p.m + 31) / 32;
    static bool ready[64];
    if (int rc = rt_allow_lds(ctx, (const void*)ou_slab_kernel<T, NB, true>, most, ready)) return rc;
    hipLaunchKernelGGL((ou_slab_kernel<T, NB, true>), dim3(1, p.batch), dim3(64 * waves), OsLds<NB>::bytes(waves), st, p, in, m_old, m_new,
                       OsPlace{}, 0, steps, out);
    EGNN_LAUNCH_CHECK(ctx, "orthogonalise");
    return EGNN_OK;
  }
  static bool ready[64];
  if (int rc = rt_allow_lds(ctx, (const void*)ou_slab_kernel<T, NB, false>, most, ready)) return rc;
  float4* g[2] = {(float4*)((char*)ws + s.g), (float4*)((char*)ws + s.g + (s.bytes - s.g) / 2)};
  for (int k = 0; k <= steps; ++k) {
    const OsPlace w{(uint4*)((char*)ws + s.x), g[k & 1], g[(k + 1) & 1], (double*)((char*)ws + s.squares), (double*)((char*)ws + s.sigma), s.slabs, s.turns};
    hipLaunchKernelGGL((ou_slab_kernel<T, NB, false>), dim3(s.slabs, p.batch), dim3(64 * OS_WAVES), most, st, p, in, m_old, m_new, w, k, steps,
                       out);
  }
  EGNN_LAUNCH_CHECK(ctx, "orthogonalise");
  return EGNN_OK;
}

struct OuSpace { size_t part, sigma, x, xt, g, bytes; };
OuSpace ou_space(const OuShape& p) {
  if (p.n <= 64) return {0, 0, 0, 0, 0, os_space(p).bytes};
  OuSpace s;
  s.part = 0;
  s.sigma = ou_align((size_t)p.batch * OU_PARTS * sizeof(double));
  s.x = s.sigma + ou_align((size_t)p.batch * sizeof(double));
  const size_t x = ou_align((size_t)p.batch * 2 * p.np * p.mp * 2), g = ou_align((size_t)p.batch * 2 * p.np * p.np * 2);
  s.xt = s.x + x;             // twice: a product reads one and writes the other
  s.g = s.xt + 2 * x;         // g and p
  s.bytes = s.g + 2 * g;
  return s;
}

template <class T, int TILE, OuProduct WHAT>
int ou_product_tile(egnn_ctx* ctx, const OuShape& p, const OuOperands& o, const OuOut<T>& out, hipStream_t st) {
  constexpr size_t lds = OuTile<TILE>::LDS;
  static bool ready[64];
  if (int rc = rt_allow_lds(ctx, (const void*)ou_product_kernel<T, TILE, WHAT>, lds, ready)) return rc;
  const dim3 grid((o.J + TILE - 1) / TILE, (o.I + TILE - 1) / TILE, p.batch);
  hipLaunchKernelGGL((ou_product_kernel<T, TILE, WHAT>), grid, dim3(OuTile<TILE>::THREADS), lds, st, p, o, out);
  EGNN_LAUNCH_CHECK(ctx, "orthogonalise");
  return EGNN_OK;
}

// Tiles of 128 where half the compute units get one, else of 64: a wide tile takes half the LDS traffic a product, but four times as long
// (us a step of the optimiser, 128 against 64: 1 x 768 x 768 369 : 150, 1 x 1280 x 2048 637 : 516, 2 x 1310 x 1071 535 : 605, 1 x 1536 x 2048 689 : 738).
template <class T, OuProduct WHAT>
int ou_product(egnn_ctx* ctx, const OuShape& p, const OuOperands& o, const OuOut<T>& out, hipStream_t st) {
  const long wide = (long)((o.I + 127) / 128) * ((o.J + 127) / 128) * p.batch;
  if (wide >= 128) return ou_product_tile<T, 128, WHAT>(ctx, p, o, out, st);
  return ou_product_tile<T, 64, WHAT>(ctx, p, o, out, st);
}

template <class T>
int ou_run(egnn_ctx* ctx, const OuShape& p, const OuInput<T>& in, const float* m_old, float* m_new, int steps, const OuOut<T>& out,
           void* ws, hipStream_t st) {
  if (p.n <= 32) return ou_run_slabs<T, 1>(ctx, p, in, m_old, m_new, steps, out, ws, st);
  if (p.n <= 64) return ou_run_slabs<T, 2>(ctx, p, in, m_old, m_new, steps, out, ws, st);
  const OuSpace s = ou_space(p);
  double* part = (double*)((char*)ws + s.part);
  double* sigma = (double*)((char*)ws + s.sigma);
  _Float16* x = (_Float16*)((char*)ws + s.x);
  _Float16* xt = (_Float16*)((char*)ws + s.xt);
  _Float16* xt2 = (_Float16*)((char*)ws + s.xt + (s.g - s.xt) / 2);
  _Float16* g = (_Float16*)((char*)ws + s.g);
  _Float16* q = (_Float16*)((char*)ws + s.g + (s.bytes - s.g) / 2);
  const size_t size = (size_t)p.rows * p.cols;
  const int parts = ou_parts(size);
  const uintptr_t all = (uintptr_t)in.u | (uintptr_t)m_old | (uintptr_t)m_new;
  if (size % 4 == 0 && all % 16 == 0)
    hipLaunchKernelGGL((ou_square_kernel<T, 4>), dim3(parts, p.batch), dim3(256), 0, st, in, m_old, m_new, size, part);
  else
    hipLaunchKernelGGL((ou_square_kernel<T, 1>), dim3(parts, p.batch), dim3(256), 0, st, in, m_old, m_new, size, part);
  hipLaunchKernelGGL((ou_pieces_kernel<T>), dim3(p.mp / 64, p.np / 64, p.batch), dim3(256), 0, st, p, in, part, parts, sigma, x, xt);
  EGNN_LAUNCH_CHECK(ctx, "orthogonalise");
  const OuOut<float> none{};
  for (int k = 0; k < steps; ++k) {
    if (int rc = ou_product<float, OU_GRAM>(ctx, p, {x, x, g, nullptr, p.np, p.np, p.mp, sigma, k}, none, st)) return rc;
    if (int rc = ou_product<float, OU_POLY>(ctx, p, {g, g, q, nullptr, p.np, p.np, p.np, sigma, k}, none, st)) return rc;
    if (k + 1 == steps) return ou_product<T, OU_LAST>(ctx, p, {q, xt, nullptr, nullptr, p.np, p.mp, p.np, sigma, k}, out, st);
    if (int rc = ou_product<float, OU_UPDATE>(ctx, p, {q, xt, xt2, x, p.np, p.mp, p.np, sigma, k}, none, st)) return rc;
    _Float16* t = xt; xt = xt2; xt2 = t;
  }
  return EGNN_OK;
}

int ou_check(egnn_ctx* ctx, const char* who, int32_t batch, int32_t rows, int32_t cols, int32_t steps) {
  const std::string at(who);
  if (batch < 0 || batch > 65535 || rows < 1 || rows > 65536 || cols < 1 || cols > 65536)
    return egnn_fail(ctx, EGNN_EINVAL, at + ": batch must be in 0..65535, rows and cols in 1..65536");
  if (steps < 1 || steps > 32) return egnn_fail(ctx, EGNN_EINVAL, at + ": steps must be in 1..32");
  return EGNN_OK;
}

template <class T>
int ou_matrices(egnn_ctx* ctx, const OuShape& p, const void* g, int steps, void* y, void* ws, hipStream_t st) {
  const OuInput<T> in{(const T*)g, nullptr, 0.0f};
  const OuOut<T> out{(T*)y, nullptr, 0.0f, 0.0f, p.cols % 8 == 0 && (uintptr_t)y % 16 == 0,
                     p.tall && p.cols % 4 == 0 && ((uintptr_t)g | (uintptr_t)y) % (4 * sizeof(T)) == 0};
  return ou_run<T>(ctx, p, in, nullptr, nullptr, steps, out, ws, st);
}

}  // namespace

extern "C" int egnn_orthogonalise_workspace_bytes(const egnn_ctx* ctx, int32_t batch, int32_t rows, int32_t cols, size_t* bytes) {
  if (!ctx || !bytes) return egnn_fail(const_cast<egnn_ctx*>(ctx), EGNN_EINVAL, "orthogonalise_workspace_bytes: null pointer");
  if (int rc = ou_check(const_cast<egnn_ctx*>(ctx), "orthogonalise_workspace_bytes", batch, rows, cols, 1)) return rc;
  *bytes = ou_space(ou_shape(batch, rows, cols)).bytes;
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
  if (!ws || (uintptr_t)ws % 256 || ws_bytes < ou_space(p).bytes)
    return egnn_fail(ctx, EGNN_EWS, "orthogonalise: workspace too small or not 256-byte aligned");
  hipStream_t st = (hipStream_t)stream;
  if (dtype == EGNN_F32) return ou_matrices<float>(ctx, p, g, steps, y, ws, st);
  if (dtype == EGNN_F16) return ou_matrices<_Float16>(ctx, p, g, steps, y, ws, st);
  return ou_matrices<__bf16>(ctx, p, g, steps, y, ws, st);
}

extern "C" int egnn_muon_step(egnn_ctx* ctx, const float* W, const float* g, const float* m, int32_t batch, int32_t rows, int32_t cols,
                              float lr, float beta, float weight_decay, int32_t steps, float* W_out, float* m_out, void* ws,
                              size_t ws_bytes, void* stream) {
  if (!ctx) return EGNN_EINVAL;
  if (int rc = ou_check(ctx, "muon_step", batch, rows, cols, steps)) return rc;
  if (batch == 0) return EGNN_OK;
  if (!W || !g || !m || !W_out || !m_out) return egnn_fail(ctx, EGNN_EINVAL, "muon_step: null pointer");
  const OuShape p = ou_shape(batch, rows, cols);
  if (!ws || (uintptr_t)ws % 256 || ws_bytes < ou_space(p).bytes)
    return egnn_fail(ctx, EGNN_EWS, "muon_step: workspace too small or not 256-byte aligned");
  const float scale = (float)((double)lr * sqrt(rows > cols ? (double)rows / cols : 1.0));
  const float keep = (float)(1.0 - (double)lr * (double)weight_decay);
  const uintptr_t all = (uintptr_t)g | (uintptr_t)m | (uintptr_t)m_out | (uintptr_t)W | (uintptr_t)W_out;
  const OuOut<float> out{W_out, W, keep, scale, cols % 8 == 0 && (uintptr_t)W_out % 16 == 0, p.tall && cols % 4 == 0 && all % 16 == 0};
  return ou_run<float>(ctx, p, OuInput<float>{g, m_out, beta}, m, m_out, steps, out, ws, (hipStream_t)stream);
}
