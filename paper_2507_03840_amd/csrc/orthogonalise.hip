// An update orthogonalised by Newton-Schulz products, and the optimiser's step around it.
//
//   x_0 = u / (|u|_F + 1e-7),   x_{k+1} = p x_k,   p = a I + b g + c g^2,   g = x_k x_k^T  (x from the side with fewer rows),
// with the published coefficients of the Muon optimiser: the singular values of u go to within about 0.7 .. 1.2.
// Step: m' = beta m + g, u = g + beta m', W' = (1 - lr weight_decay) W - lr sqrt(max(1, rows / cols)) orthogonalise(u).
//
// All products are C = A B^T of operands with the contraction along the rows: g = x x^T, g g (g is symmetric), p x with x^T kept
// beside x.  They run on the matrix cores on half-precision pieces: v s = hi + lo, hi = v s rounded to 11 bits, lo = the rest
// rounded to 11 bits, and hi hi + hi lo + lo hi (the dropped lo lo is 2^-24 of the product).  |x_0|_F <= 1 and the steps keep
// the singular values below 1.2025, so every entry of x, g and p is bounded whatever the input, and one fixed power of two as
// scale s leaves nothing to overflow and nothing above 2^-39 to underflow.
// Results in bfloat16 of wide updates (both sides at least OU_ONE_PIECE) need no lo in the products: see ou_pieces().  The largest term
// of a step, a x, then stays out of them: x^T keeps both pieces, and p is b g + c g^2 alone.
#include "row_types.h"
#include <math.h>
#include <type_traits>

namespace {

constexpr float OU_A = 3.4445f, OU_B = -4.7750f, OU_C = 2.0315f;
constexpr double OU_EPS = 1e-7;
// entries of x are at most 1.2025, of g 1.446, of p 3.4445 (its eigenvalues lie between 0.6 and a): times these at most 56,500
constexpr float OU_SX = 32768.0f, OU_SG = 32768.0f, OU_SP = 16384.0f;
constexpr int OU_PARTS = 512;       // partial sums of squares per matrix, at most
constexpr int OU_ONE_PIECE = 256;

typedef _Float16 ou_h8 __attribute__((ext_vector_type(8)));
typedef _Float16 ou_h4 __attribute__((ext_vector_type(4)));
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
template <class T>
__global__ __launch_bounds__(256) void ou_square_kernel(OuInput<T> in, const float* m_old, float* m_new, size_t size, double* part) {
  __shared__ double s[256];
  const size_t at = (size_t)blockIdx.y * size;
  const size_t per = (size + gridDim.x - 1) / gridDim.x, b = blockIdx.x * per, e = min(b + per, size);
  double t = 0.0;
  for (size_t i = b + threadIdx.x; i < e; i += 256) {
    float v = (float)in.u[at + i];
    if (m_old) {
      const float mm = in.beta * m_old[at + i] + v;
      m_new[at + i] = mm;
      v = v + in.beta * mm;
    }
    t += (double)v * (double)v;
  }
  s[threadIdx.x] = t;
  for (int h = 128; h; h >>= 1) {
    __syncthreads();
    if ((int)threadIdx.x < h) s[threadIdx.x] += s[threadIdx.x + h];
  }
  if (threadIdx.x == 0) part[(size_t)blockIdx.y * OU_PARTS + blockIdx.x] = s[0];
}

// 1 / (|u| + eps) of one matrix, in every lane
__device__ __forceinline__ double ou_inverse_norm(const double* part, int parts) {
  double t = 0.0;
  for (int i = threadIdx.x & 63; i < parts; i += 64) t += part[i];
  for (int h = 32; h; h >>= 1) t += __shfl_xor(t, h);
  return 1.0 / (sqrt(t) + OU_EPS);
}

// ---- x_0 in pieces, in both layouts: 64 x 64 tiles.  x [P pieces][np][mp], xt [2 pieces][mp][np] per matrix
template <class T, int P>
__global__ __launch_bounds__(256) void ou_pieces_kernel(OuShape p, OuInput<T> in, const double* part, int parts, _Float16* x,
                                                        _Float16* xt) {
  __shared__ float tile[64][65];    // [i][j] of x
  const size_t z = blockIdx.z;
  const double inv = ou_inverse_norm(part + z * OU_PARTS, parts) * (double)OU_SX;
  const int i0 = blockIdx.y * 64, j0 = blockIdx.x * 64, t = threadIdx.x;
  for (int k = 0; k < 16; ++k) {
    const int a = (t >> 6) + 4 * k, b = t & 63;       // b along the caller's rows
    const int i = i0 + (p.tall ? b : a), j = j0 + (p.tall ? a : b);
    const bool there = i < p.n && j < p.m;
    const size_t at = z * p.rows * p.cols + (p.tall ? (size_t)j * p.cols + i : (size_t)i * p.cols + j);
    const float v = there ? (float)((double)ou_value(in, at) * inv) : 0.0f;
    if (p.tall) tile[b][a] = v; else tile[a][b] = v;
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
    _Float16* to = x + z * P * plane + (size_t)(i0 + r) * p.mp + j0 + c;
    _Float16* tt = xt + z * 2 * plane + (size_t)(j0 + r) * p.np + i0 + c;
    *(ou_h8*)to = hi;
    *(ou_h8*)tt = thi;
    if (P == 2) *(ou_h8*)(to + plane) = lo;
    *(ou_h8*)(tt + plane) = tlo;
  }
}

// ---- products ----------------------------------------------------------------------------------------------------------
enum OuProduct { OU_GRAM, OU_POLY, OU_UPDATE, OU_LAST };

template <class T>
struct OuOut { T* y; const float* W; float keep, scale; };   // of the last product: y = q, or keep W - scale q

struct OuOperands {
  const _Float16 *A, *B;   // per matrix [P pieces][I][K], [P pieces][J][K]; x^T always has two pieces
  _Float16 *C, *Ct;        // results in pieces: C [..][J][I] (the transpose; g and p are symmetric), Ct [P pieces][I][J]
  int I, J, K;             // multiples of 64
};

typedef const __attribute__((address_space(1))) void* ou_gp;
typedef __attribute__((address_space(3))) void* ou_lp;

// 4 x 4 halves across a quad of lanes: lane q holds column q of rows 0..3, and gets row q
__device__ __forceinline__ uint2 ou_turn(uint2 v, int lane) {
  const uint32_t pa = __builtin_amdgcn_mov_dpp(v.x, 0xB1, 0xf, 0xf, true), pb = __builtin_amdgcn_mov_dpp(v.y, 0xB1, 0xf, 0xf, true);
  const bool odd = lane & 1, upper = lane & 2;
  const uint32_t a = odd ? __builtin_amdgcn_perm(v.x, pa, 0x07060302) : __builtin_amdgcn_perm(pa, v.x, 0x05040100);
  const uint32_t b = odd ? __builtin_amdgcn_perm(v.y, pb, 0x07060302) : __builtin_amdgcn_perm(pb, v.y, 0x05040100);
  const uint32_t qa = __builtin_amdgcn_mov_dpp(a, 0x4E, 0xf, 0xf, true), qb = __builtin_amdgcn_mov_dpp(b, 0x4E, 0xf, 0xf, true);
  return upper ? make_uint2(qb, b) : make_uint2(a, qa);
}

// waits until at most N loads of this wave are under way (loads return in order), then for the other waves
template <int N>
__device__ __forceinline__ void ou_loads_then_barrier() {
  static_assert(N < 64, "the counter of loads has six bits");
  asm volatile("" ::: "memory");
  __builtin_amdgcn_s_waitcnt((N & 15) | 7 << 4 | 15 << 8 | (N >> 4) << 14);
  __builtin_amdgcn_s_barrier();
  asm volatile("" ::: "memory");
}

// C = A B^T of one tile TILE x TILE: four waves, each a quarter (TILE / 2 squared) in 32 x 32 blocks.  64 contraction indices a
// turn, brought straight into one of STAGES LDS buffers, STAGES - 1 turns ahead: with one wave per SIMD nothing else hides the way to
// memory.  A row of 128 bytes lies in LDS as eight pieces of 16 bytes, piece c at place c ^ (row & 7): eight lanes that read the same
// piece of eight rows meet all banks.  The operands of a step of 16 are read from LDS while the products of the one before run.
template <int P, int TILE>
struct OuTile {
  static constexpr int STAGES = P * TILE >= 256 ? 2 : 4;
  static constexpr int PLANE = TILE * 8, STAGE = 2 * P * PLANE;          // uint4
  static constexpr int LOADS = 2 * P * TILE / 32;                         // of a wave per turn
  static constexpr size_t LDS = (size_t)STAGES * STAGE * 16;
};

template <class T, int P, int TILE, OuProduct WHAT>
__global__ __launch_bounds__(256) void ou_product_kernel(OuShape p, OuOperands o, OuOut<T> out) {
  extern __shared__ uint4 smem[];                     // [STAGES][2 operands][P][TILE][8]
  constexpr bool STEP = WHAT == OU_UPDATE || WHAT == OU_LAST;   // p x
  constexpr int PB = STEP ? 2 : P;
  typedef OuTile<P, TILE> Tile;
  constexpr int HALF = TILE / 2, B = HALF / 32, PLANE = Tile::PLANE, STAGE = Tile::STAGE, STAGES = Tile::STAGES;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const size_t z = blockIdx.z;
  const int i0 = blockIdx.y * TILE, j0 = blockIdx.x * TILE;
  const size_t plane_a = (size_t)o.I * o.K, plane_b = (size_t)o.J * o.K;
  const _Float16* A = o.A + z * P * plane_a;
  const _Float16* Bm = o.B + z * PB * plane_b;
  const int wi = (wave >> 1) * HALF, wj = (wave & 1) * HALF;

  // lane's place in a load of eight rows
  const int lrow = lane >> 3, lpiece = (lane & 7) ^ lrow;
  const _Float16 *pa[TILE / 32], *pb[TILE / 32];
#pragma unroll
  for (int r = 0; r < TILE / 32; ++r) {
    const int row = (r * 4 + wave) * 8 + lrow;
    pa[r] = A + (size_t)min(i0 + row, o.I - 1) * o.K + lpiece * 8;
    pb[r] = Bm + (size_t)min(j0 + row, o.J - 1) * o.K + lpiece * 8;
  }
  auto fetch = [&](int turn, int stage) {
    uint4* to = smem + stage * STAGE + wave * 64;
#pragma unroll
    for (int q = 0; q < P; ++q)
#pragma unroll
      for (int r = 0; r < TILE / 32; ++r) {
        __builtin_amdgcn_global_load_lds((ou_gp)(pa[r] + q * plane_a + turn * 64), (ou_lp)(to + q * PLANE + r * 256), 16, 0, 0);
        __builtin_amdgcn_global_load_lds((ou_gp)(pb[r] + q * plane_b + turn * 64), (ou_lp)(to + (P + q) * PLANE + r * 256), 16, 0, 0);
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
    const uint4* sb = smem + stage * STAGE + P * PLANE + (wj + r32) * 8;
    stage = stage + 1 == STAGES ? 0 : stage + 1;
    ou_h8 a[2][B][P], b[2][B][P];
    auto operands = [&](int s) {
      const int place = (2 * s + hh) ^ (r32 & 7);
#pragma unroll
      for (int x = 0; x < B; ++x)
#pragma unroll
        for (int q = 0; q < P; ++q) {
          a[s & 1][x][q] = __builtin_bit_cast(ou_h8, sa[q * PLANE + x * 256 + place]);
          b[s & 1][x][q] = __builtin_bit_cast(ou_h8, sb[q * PLANE + x * 256 + place]);
        }
    };
    operands(0);
#pragma unroll
    for (int s = 0; s < 4; ++s) {
      if (s < 3) operands(s + 1);
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int t = P == 2 ? 0 : 2; t < 3; ++t)     // lo hi, hi lo, hi hi
#pragma unroll
        for (int x = 0; x < B; ++x)
#pragma unroll
          for (int y = 0; y < B; ++y)
            acc[x][y] = __builtin_amdgcn_mfma_f32_32x32x16_f16(a[s & 1][x][t == 0 ? P - 1 : 0], b[s & 1][y][t == 1 ? P - 1 : 0], acc[x][y], 0, 0, 0);
      __builtin_amdgcn_sched_barrier(0);
    }
  }
  ou_loads_then_barrier<0>();      // (no load to LDS outlives the workgroup)

  // a lane holds column j = lane & 31 of its blocks and four times four neighbouring rows i
  constexpr float unscale = WHAT == OU_GRAM ? 1.0f / (OU_SX * OU_SX) : WHAT == OU_POLY ? 1.0f / (OU_SG * OU_SG) : 1.0f / (OU_SP * OU_SX);
  constexpr float scale = WHAT == OU_GRAM ? OU_SG : WHAT == OU_POLY ? OU_SP : OU_SX;
  const size_t plane_c = (size_t)o.I * o.J;
#pragma unroll
  for (int x = 0; x < B; ++x)
#pragma unroll
    for (int y = 0; y < B; ++y)
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const int i = i0 + wi + 32 * x + 8 * r + 4 * hh, j = j0 + wj + 32 * y + r32;
        float v[4];
#pragma unroll
        for (int q = 0; q < 4; ++q) v[q] = acc[x][y][4 * r + q] * unscale;
        if (STEP && P == 1 && i < o.I && j < o.J) {
          const _Float16* old = Bm + (size_t)j * o.I + i;
          const ou_h4 xh = *(const ou_h4*)old, xl = *(const ou_h4*)(old + plane_b);
#pragma unroll
          for (int q = 0; q < 4; ++q) v[q] += OU_A * (((float)xh[q] + (float)xl[q]) * (1.0f / OU_SX));
        }
        if (WHAT == OU_LAST) {
          const int n = p.n, m = p.m;
#pragma unroll
          for (int q = 0; q < 4; ++q) {
            if (i + q >= n || j >= m) continue;
            const size_t at = z * n * m + (p.tall ? (size_t)j * n + i + q : (size_t)(i + q) * m + j);
            out.y[at] = (T)(out.W ? out.keep * out.W[at] - out.scale * v[q] : v[q]);
          }
          continue;
        }
        if (i >= o.I || j >= o.J) continue;           // (a tile of 128 over sides that are multiples of 64: whole quads of lanes)
        const size_t at = (size_t)j * o.I + i;
        if (WHAT == OU_POLY) {
          const _Float16* g = A + at;
          ou_h4 gh = *(const ou_h4*)g, gl;
          if (P == 2) gl = *(const ou_h4*)(g + plane_a);
#pragma unroll
          for (int q = 0; q < 4; ++q) {
            const float gv = ((float)gh[q] + (P == 2 ? (float)gl[q] : 0.0f)) * (1.0f / OU_SG);
            v[q] = OU_C * v[q] + OU_B * gv + (P == 2 && i + q == j && j < p.n ? OU_A : 0.0f);
          }
        }
        ou_h4 hi, lo;
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          _Float16 h, l;
          ou_cut(v[q] * scale, h, l);
          hi[q] = h; lo[q] = l;
        }
        _Float16* c = o.C + z * (STEP ? 2 : P) * plane_c + at;
        *(ou_h4*)c = hi;
        if (STEP || P == 2) *(ou_h4*)(c + plane_c) = lo;
        if (WHAT == OU_UPDATE) {
          _Float16* ct = o.Ct + z * P * plane_c + (size_t)(i + (lane & 3)) * o.J + (j & ~3);
          *(uint2*)ct = ou_turn(__builtin_bit_cast(uint2, hi), lane);
          if (P == 2) *(uint2*)(ct + plane_c) = ou_turn(__builtin_bit_cast(uint2, lo), lane);
        }
      }
}

// ---- n <= 64: all of g and p in one workgroup ----------------------------------------------------------------------------------
// The long side is cut into slabs of 128 columns of x (rows of x^T).  A launch takes the parts of g = x x^T of all slabs, and every
// workgroup adds them (16 KB a slab, always in the same order), makes p for itself, takes its slab one step further and leaves
// the slab's part of the next g.  So a step is one launch; with up to 128 columns in all (ALONE) everything is one.
//
// x^T p lands in the accumulators with a lane holding column j and rows k of x^T four by four; that is also how the next product, g =
// sum_k x^T[k][i] x^T[k][j], wants both its operands if the same order of k is taken for both, which any order may be.  Only the next
// step's x^T has to change lanes (through memory, each wave its own rows).  Step 0 takes p = I, which is exact in pieces.
constexpr int OS_ROWS = 128;                 // of a slab: 32 a wave
constexpr int OS_SLABS = 64;                 // more columns than this many slabs: a workgroup takes several
constexpr int OS_X = 2 * OS_ROWS * 8;        // LDS, in uint4: x^T pieces; then g and p pieces, and over them the waves' parts of g
constexpr size_t OS_LDS = (size_t)OS_X * 16 + 4 * 64 * 64 * 4;

struct OsPlace {
  _Float16* xt;           // [batch][slabs * turns * 128][2 pieces][64]
  const float* part_in;   // [batch][slabs][64 * 64]: parts of g of this step
  float* part_out;        // of the next one
  const double* squares;  // sums of squares (not ALONE)
  int n_squares, slabs, turns;
};

// place of element (r, c) of a 64-wide tile of halves: 16-byte pieces exchanged by row, as in the products above
__device__ __forceinline__ int os_at(int r, int c) { return r * 64 + (((c >> 3) ^ (r & 7)) << 3) + (c & 7); }

template <class T, bool ALONE>
__global__ __launch_bounds__(256) void ou_slab_kernel(OuShape p, OuInput<T> in, const float* m_old, float* m_new, OsPlace w, int step,
                                                      int steps, OuOut<T> out) {
  extern __shared__ uint4 smem[];
  _Float16* sx = (_Float16*)smem;                        // [2][128][64]
  _Float16* sg = (_Float16*)(smem + OS_X);               // [2][64][64]
  _Float16* sp = sg + 2 * 64 * 64;                       // [2][64][64]
  float4* sums = (float4*)(smem + OS_X);                 // [4 waves][64][16], over sg and sp
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int r32 = lane & 31, hh = lane >> 5, slab = blockIdx.x;
  const size_t z = blockIdx.y, size = (size_t)p.rows * p.cols, at0 = z * size;
  double inv;
  if (ALONE) {
    double t = 0.0;
    for (int i = tid; i < (int)size; i += 256) {
      float v = (float)in.u[at0 + i];
      if (m_old) {
        const float mm = in.beta * m_old[at0 + i] + v;
        m_new[at0 + i] = mm;
        v = v + in.beta * mm;
      }
      t += (double)v * (double)v;
    }
    for (int h = 32; h; h >>= 1) t += __shfl_xor(t, h);
    double* s = (double*)smem;
    if (lane == 0) s[wave] = t;
    __syncthreads();
    inv = (double)OU_SX / (sqrt((s[0] + s[1]) + (s[2] + s[3])) + OU_EPS);
    __syncthreads();
  } else if (step == 0) {
    inv = ou_inverse_norm(w.squares + z * OU_PARTS, w.n_squares) * (double)OU_SX;
  }

  ou_f16v g[2][2];
  for (int k = ALONE ? 0 : step; k <= (ALONE ? steps : step); ++k) {
    // p in pieces
    if (k == 0) {
      for (int e = tid; e < 64 * 64; e += 256) {
        const int r = e >> 6, c = e & 63;
        sp[os_at(r, c)] = (_Float16)(r == c ? OU_SP : 0.0f);
        sp[64 * 64 + os_at(r, c)] = (_Float16)0.0f;
      }
    } else {
      float4 v[4];
      if (ALONE) {
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          const int e = tid + 256 * q;
          const float4 a = sums[e], b = sums[1024 + e], c = sums[2048 + e], d = sums[3072 + e];
          v[q] = make_float4((a.x + b.x) + (c.x + d.x), (a.y + b.y) + (c.y + d.y), (a.z + b.z) + (c.z + d.z), (a.w + b.w) + (c.w + d.w));
        }
        __syncthreads();
      } else {
        const float4* from = (const float4*)w.part_in + z * w.slabs * 1024;
#pragma unroll
        for (int q = 0; q < 4; ++q) v[q] = from[tid + 256 * q];
#pragma unroll 4
        for (int t = 1; t < w.slabs; ++t)
#pragma unroll
          for (int q = 0; q < 4; ++q) {
            const float4 a = from[t * 1024 + tid + 256 * q];
            v[q].x += a.x; v[q].y += a.y; v[q].z += a.z; v[q].w += a.w;
          }
      }
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const int e = tid + 256 * q, r = e >> 4, c = 4 * ((e & 15) ^ (r & 15));
        const float f[4] = {v[q].x, v[q].y, v[q].z, v[q].w};
        ou_h4 hi, lo;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          _Float16 h, l;
          ou_cut(f[i] * OU_SG, h, l);
          hi[i] = h; lo[i] = l;
        }
        *(ou_h4*)(sg + os_at(r, c)) = hi;
        *(ou_h4*)(sg + 64 * 64 + os_at(r, c)) = lo;
      }
      __syncthreads();
      const int wi = (wave >> 1) * 32, wj = (wave & 1) * 32;
      ou_f16v acc;
#pragma unroll
      for (int i = 0; i < 16; ++i) acc[i] = 0.0f;
#pragma unroll
      for (int s = 0; s < 4; ++s) {
        const int c = 16 * s + 8 * hh;
        const ou_h8 ah = *(const ou_h8*)(sg + os_at(wi + r32, c)), al = *(const ou_h8*)(sg + 64 * 64 + os_at(wi + r32, c));
        const ou_h8 bh = *(const ou_h8*)(sg + os_at(wj + r32, c)), bl = *(const ou_h8*)(sg + 64 * 64 + os_at(wj + r32, c));
        acc = __builtin_amdgcn_mfma_f32_32x32x16_f16(al, bh, acc, 0, 0, 0);
        acc = __builtin_amdgcn_mfma_f32_32x32x16_f16(ah, bl, acc, 0, 0, 0);
        acc = __builtin_amdgcn_mfma_f32_32x32x16_f16(ah, bh, acc, 0, 0, 0);
      }
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const int i = wi + 8 * r + 4 * hh, j = wj + r32;
        const ou_h4 gh = *(const ou_h4*)(sg + os_at(j, i)), gl = *(const ou_h4*)(sg + 64 * 64 + os_at(j, i));
        ou_h4 hi, lo;
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          const float gv = ((float)gh[q] + (float)gl[q]) * (1.0f / OU_SG);
          const float v = OU_C * (acc[4 * r + q] * (1.0f / (OU_SG * OU_SG))) + OU_B * gv + (i + q == j ? OU_A : 0.0f);
          _Float16 h, l;
          ou_cut(v * OU_SP, h, l);
          hi[q] = h; lo[q] = l;
        }
        *(ou_h4*)(sp + os_at(j, i)) = hi;
        *(ou_h4*)(sp + 64 * 64 + os_at(j, i)) = lo;
      }
    }
#pragma unroll
    for (int a = 0; a < 2; ++a)
#pragma unroll
      for (int b = 0; b < 2; ++b)
#pragma unroll
        for (int i = 0; i < 16; ++i) g[a][b][i] = 0.0f;
    __syncthreads();       // p is there

    for (int turn = 0; turn < (ALONE ? 1 : w.turns); ++turn) {
      const int first = (slab * (ALONE ? 1 : w.turns) + turn) * OS_ROWS;      // row of x^T
      _Float16* mine = ALONE ? nullptr : w.xt + ((z * w.slabs * w.turns + slab * w.turns + turn) * OS_ROWS + wave * 32) * 128;
      if (k == 0) {       // x_0 = u / |u|, each wave its own rows
        for (int e = lane; e < 32 * 64; e += 64) {
          const int row = p.tall ? e >> 6 : e & 31, i = p.tall ? e & 63 : e >> 5;
          const int c = first + wave * 32 + row;
          const bool there = i < p.n && c < p.m;
          const size_t at = at0 + (p.tall ? (size_t)c * p.cols + i : (size_t)i * p.cols + c);
          const float v = there ? (float)((double)ou_value(in, at) * inv) : 0.0f;
          _Float16 h, l;
          ou_cut(v, h, l);
          sx[os_at(wave * 32 + row, i)] = h;
          sx[OS_ROWS * 64 + os_at(wave * 32 + row, i)] = l;
        }
        __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront", "local");
        __builtin_amdgcn_wave_barrier();
        __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront", "local");
      }
      ou_f16v acc[2];
#pragma unroll
      for (int i = 0; i < 16; ++i) acc[0][i] = acc[1][i] = 0.0f;
#pragma unroll
      for (int s = 0; s < 4; ++s) {
        const int c = 16 * s + 8 * hh;
        ou_h8 ah, al;
        if (ALONE || k == 0) {
          ah = *(const ou_h8*)(sx + os_at(wave * 32 + r32, c));
          al = *(const ou_h8*)(sx + OS_ROWS * 64 + os_at(wave * 32 + r32, c));
        } else {
          ah = *(const ou_h8*)(mine + r32 * 128 + c);
          al = *(const ou_h8*)(mine + r32 * 128 + 64 + c);
        }
#pragma unroll
        for (int b = 0; b < 2; ++b) {
          const ou_h8 bh = *(const ou_h8*)(sp + os_at(32 * b + r32, c)), bl = *(const ou_h8*)(sp + 64 * 64 + os_at(32 * b + r32, c));
          acc[b] = __builtin_amdgcn_mfma_f32_32x32x16_f16(al, bh, acc[b], 0, 0, 0);
          acc[b] = __builtin_amdgcn_mfma_f32_32x32x16_f16(ah, bl, acc[b], 0, 0, 0);
          acc[b] = __builtin_amdgcn_mfma_f32_32x32x16_f16(ah, bh, acc[b], 0, 0, 0);
        }
      }
      if (k == steps) {
#pragma unroll
        for (int b = 0; b < 2; ++b)
#pragma unroll
          for (int i = 0; i < 16; ++i) {
            const int j = 32 * b + r32, c = first + wave * 32 + 8 * (i >> 2) + 4 * hh + (i & 3);
            if (j >= p.n || c >= p.m) continue;
            const size_t at = at0 + (p.tall ? (size_t)c * p.cols + j : (size_t)j * p.cols + c);
            const float v = acc[b][i] * (1.0f / (OU_SP * OU_SX));
            out.y[at] = (T)(out.W ? out.keep * out.W[at] - out.scale * v : v);
          }
        continue;
      }
      ou_h8 xh[2][2], xl[2][2];        // [column block][16 rows]: the operands of g
#pragma unroll
      for (int b = 0; b < 2; ++b)
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          _Float16 h, l;
          ou_cut(acc[b][i] * (1.0f / OU_SP), h, l);
          xh[b][i >> 3][i & 7] = h;
          xl[b][i >> 3][i & 7] = l;
        }
#pragma unroll
      for (int b = 0; b < 2; ++b)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          ou_h4 h, l;
#pragma unroll
          for (int q = 0; q < 4; ++q) {
            h[q] = xh[b][r >> 1][4 * (r & 1) + q];
            l[q] = xl[b][r >> 1][4 * (r & 1) + q];
          }
          const uint2 th = ou_turn(__builtin_bit_cast(uint2, h), lane), tl = ou_turn(__builtin_bit_cast(uint2, l), lane);
          const int row = 8 * r + 4 * hh + (lane & 3), c = 32 * b + (r32 & ~3);
          if (ALONE) {
            *(uint2*)(sx + os_at(wave * 32 + row, c)) = th;
            *(uint2*)(sx + OS_ROWS * 64 + os_at(wave * 32 + row, c)) = tl;
          } else {
            *(uint2*)(mine + row * 128 + c) = th;
            *(uint2*)(mine + row * 128 + 64 + c) = tl;
          }
        }
#pragma unroll
      for (int t = 0; t < 2; ++t)
#pragma unroll
        for (int a = 0; a < 2; ++a)
#pragma unroll
          for (int b = 0; b < 2; ++b) {
            g[a][b] = __builtin_amdgcn_mfma_f32_32x32x16_f16(xl[a][t], xh[b][t], g[a][b], 0, 0, 0);
            g[a][b] = __builtin_amdgcn_mfma_f32_32x32x16_f16(xh[a][t], xl[b][t], g[a][b], 0, 0, 0);
            g[a][b] = __builtin_amdgcn_mfma_f32_32x32x16_f16(xh[a][t], xh[b][t], g[a][b], 0, 0, 0);
          }
    }
    if (k == steps) return;
    __syncthreads();       // p is no longer read: the waves' parts of g go over it
#pragma unroll
    for (int a = 0; a < 2; ++a)
#pragma unroll
      for (int b = 0; b < 2; ++b)
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          const int i = 32 * a + 8 * r + 4 * hh, j = 32 * b + r32;
          constexpr float u = 1.0f / (OU_SX * OU_SX);
          sums[wave * 1024 + j * 16 + ((i >> 2) ^ (j & 15))] =
              make_float4(g[a][b][4 * r] * u, g[a][b][4 * r + 1] * u, g[a][b][4 * r + 2] * u, g[a][b][4 * r + 3] * u);
        }
    __syncthreads();
    if (!ALONE) {
      float4* to = (float4*)w.part_out + (z * w.slabs + slab) * 1024;
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const int e = tid + 256 * q;
        const float4 a = sums[e], b = sums[1024 + e], c = sums[2048 + e], d = sums[3072 + e];
        to[e] = make_float4((a.x + b.x) + (c.x + d.x), (a.y + b.y) + (c.y + d.y), (a.z + b.z) + (c.z + d.z), (a.w + b.w) + (c.w + d.w));
      }
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

// Pieces per operand.  One piece of 11 bits adds its error to that of a bfloat16 result (8 bits): measured on updates with a few
// strong directions, 4e-4 to 6e-4 of the result beside the 1.7e-3 of the last rounding where both sides are at least 256, but 2e-3 at
// 64 x 900 and more below; half precision and fp32 results would lose 2 and 400 times their own accuracy.
int ou_pieces(const OuShape& p, int32_t dtype) { return dtype == EGNN_BF16 && p.n >= OU_ONE_PIECE ? 1 : 2; }

struct OsSpace { size_t part, xt, g, bytes; int slabs, turns; };
OsSpace os_space(const OuShape& p) {
  OsSpace s;
  const int pieces = (p.m + OS_ROWS - 1) / OS_ROWS;
  s.turns = (pieces + OS_SLABS - 1) / OS_SLABS;
  s.slabs = (pieces + s.turns - 1) / s.turns;
  s.part = 0;
  s.xt = ou_align((size_t)p.batch * OU_PARTS * sizeof(double));
  s.g = s.xt + ou_align((size_t)p.batch * s.slabs * s.turns * OS_ROWS * 128 * 2);
  s.bytes = s.slabs == 1 && s.turns == 1 ? 256 : s.g + 2 * ou_align((size_t)p.batch * s.slabs * 64 * 64 * 4);
  return s;
}

int ou_parts(size_t size) { return (int)(size > (size_t)OU_PARTS * 4096 ? OU_PARTS : (size + 4095) / 4096); }

template <class T>
int ou_run_slabs(egnn_ctx* ctx, const OuShape& p, const OuInput<T>& in, const float* m_old, float* m_new, int steps,
                 const OuOut<T>& out, void* ws, hipStream_t st) {
  const OsSpace s = os_space(p);
  static bool ready = false;      // (set again by two threads at once: to the same value)
  if (!ready) {
    EGNN_HIP(ctx, hipFuncSetAttribute((const void*)ou_slab_kernel<T, true>, hipFuncAttributeMaxDynamicSharedMemorySize, (int)OS_LDS));
    EGNN_HIP(ctx, hipFuncSetAttribute((const void*)ou_slab_kernel<T, false>, hipFuncAttributeMaxDynamicSharedMemorySize, (int)OS_LDS));
    ready = true;
  }
  if (s.slabs == 1 && s.turns == 1) {
    hipLaunchKernelGGL((ou_slab_kernel<T, true>), dim3(1, p.batch), dim3(256), OS_LDS, st, p, in, m_old, m_new, OsPlace{}, 0, steps, out);
    EGNN_LAUNCH_CHECK(ctx, "orthogonalise");
    return EGNN_OK;
  }
  double* part = (double*)((char*)ws + s.part);
  float* g[2] = {(float*)((char*)ws + s.g), (float*)((char*)ws + s.g + (s.bytes - s.g) / 2)};
  const size_t size = (size_t)p.rows * p.cols;
  hipLaunchKernelGGL((ou_square_kernel<T>), dim3(ou_parts(size), p.batch), dim3(256), 0, st, in, m_old, m_new, size, part);
  for (int k = 0; k <= steps; ++k) {
    const OsPlace w{(_Float16*)((char*)ws + s.xt), g[k & 1], g[(k + 1) & 1], part, ou_parts(size), s.slabs, s.turns};
    hipLaunchKernelGGL((ou_slab_kernel<T, false>), dim3(s.slabs, p.batch), dim3(256), OS_LDS, st, p, in, m_old, m_new, w, k, steps, out);
  }
  EGNN_LAUNCH_CHECK(ctx, "orthogonalise");
  return EGNN_OK;
}

struct OuSpace { size_t part, x, xt, g, bytes; };
OuSpace ou_space(const OuShape& p, int pieces) {
  if (p.n <= 64) return {0, 0, 0, 0, os_space(p).bytes};
  OuSpace s;
  s.part = 0;
  s.x = ou_align((size_t)p.batch * OU_PARTS * sizeof(double));
  const size_t x = ou_align((size_t)p.batch * 2 * p.np * p.mp * 2), g = ou_align((size_t)p.batch * pieces * p.np * p.np * 2);
  s.xt = s.x + x;             // twice: a product reads one and writes the other
  s.g = s.xt + 2 * x;         // g and p
  s.bytes = s.g + 2 * g;
  return s;
}

template <class T, int P, int TILE, OuProduct WHAT>
int ou_product_tile(egnn_ctx* ctx, const OuShape& p, const OuOperands& o, const OuOut<T>& out, hipStream_t st) {
  constexpr size_t lds = OuTile<P, TILE>::LDS;
  static bool ready = false;      // (set again by two threads at once: to the same value)
  if (!ready && lds > 65536) {
    EGNN_HIP(ctx, hipFuncSetAttribute((const void*)ou_product_kernel<T, P, TILE, WHAT>, hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds));
    ready = true;
  }
  const dim3 grid((o.J + TILE - 1) / TILE, (o.I + TILE - 1) / TILE, p.batch);
  hipLaunchKernelGGL((ou_product_kernel<T, P, TILE, WHAT>), grid, dim3(256), lds, st, p, o, out);
  EGNN_LAUNCH_CHECK(ctx, "orthogonalise");
  return EGNN_OK;
}

template <class T, int P, OuProduct WHAT>
int ou_product(egnn_ctx* ctx, const OuShape& p, const OuOperands& o, const OuOut<T>& out, hipStream_t st) {
  const long wide = (long)((o.I + 127) / 128) * ((o.J + 127) / 128) * p.batch;
  if (wide >= 128) return ou_product_tile<T, P, 128, WHAT>(ctx, p, o, out, st);
  return ou_product_tile<T, P, 64, WHAT>(ctx, p, o, out, st);
}

template <class T, int P>
int ou_run(egnn_ctx* ctx, const OuShape& p, const OuInput<T>& in, const float* m_old, float* m_new, int steps, const OuOut<T>& out,
           void* ws, hipStream_t st) {
  if (p.n <= 64) return ou_run_slabs<T>(ctx, p, in, m_old, m_new, steps, out, ws, st);
  const OuSpace s = ou_space(p, P);
  double* part = (double*)((char*)ws + s.part);
  _Float16* x = (_Float16*)((char*)ws + s.x);
  _Float16* xt = (_Float16*)((char*)ws + s.xt);
  _Float16* xt2 = (_Float16*)((char*)ws + s.xt + (s.xt - s.x));
  _Float16* g = (_Float16*)((char*)ws + s.g);
  _Float16* q = (_Float16*)((char*)ws + s.g + (s.bytes - s.g) / 2);
  const size_t size = (size_t)p.rows * p.cols;
  const int parts = ou_parts(size);
  hipLaunchKernelGGL((ou_square_kernel<T>), dim3(parts, p.batch), dim3(256), 0, st, in, m_old, m_new, size, part);
  hipLaunchKernelGGL((ou_pieces_kernel<T, P>), dim3(p.mp / 64, p.np / 64, p.batch), dim3(256), 0, st, p, in, part, parts, x, xt);
  EGNN_LAUNCH_CHECK(ctx, "orthogonalise");
  const OuOut<float> none{};
  for (int k = 0; k < steps; ++k) {
    if (int rc = ou_product<float, P, OU_GRAM>(ctx, p, {x, x, g, nullptr, p.np, p.np, p.mp}, none, st)) return rc;
    if (int rc = ou_product<float, P, OU_POLY>(ctx, p, {g, g, q, nullptr, p.np, p.np, p.np}, none, st)) return rc;
    if (k + 1 == steps) return ou_product<T, P, OU_LAST>(ctx, p, {q, xt, nullptr, nullptr, p.np, p.mp, p.np}, out, st);
    if (int rc = ou_product<float, P, OU_UPDATE>(ctx, p, {q, xt, xt2, x, p.np, p.mp, p.np}, none, st)) return rc;
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
int ou_matrices(egnn_ctx* ctx, int32_t dtype, const OuShape& p, const void* g, int steps, void* y, void* ws, hipStream_t st) {
  const OuInput<T> in{(const T*)g, nullptr, 0.0f};
  const OuOut<T> out{(T*)y, nullptr, 0.0f, 0.0f};
  if constexpr (std::is_same<T, __bf16>::value)
    if (ou_pieces(p, dtype) == 1) return ou_run<T, 1>(ctx, p, in, nullptr, nullptr, steps, out, ws, st);
  return ou_run<T, 2>(ctx, p, in, nullptr, nullptr, steps, out, ws, st);
}

}  // namespace

extern "C" int egnn_orthogonalise_workspace_bytes(const egnn_ctx* ctx, int32_t batch, int32_t rows, int32_t cols, size_t* bytes) {
  if (!ctx || !bytes) return egnn_fail(const_cast<egnn_ctx*>(ctx), EGNN_EINVAL, "orthogonalise_workspace_bytes: null pointer");
  if (int rc = ou_check(const_cast<egnn_ctx*>(ctx), "orthogonalise_workspace_bytes", batch, rows, cols, 1)) return rc;
  *bytes = ou_space(ou_shape(batch, rows, cols), 2).bytes;
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
  if (!ws || (uintptr_t)ws % 256 || ws_bytes < ou_space(p, ou_pieces(p, dtype)).bytes)
    return egnn_fail(ctx, EGNN_EWS, "orthogonalise: workspace too small or not 256-byte aligned");
  hipStream_t st = (hipStream_t)stream;
  if (dtype == EGNN_F32) return ou_matrices<float>(ctx, dtype, p, g, steps, y, ws, st);
  if (dtype == EGNN_F16) return ou_matrices<_Float16>(ctx, dtype, p, g, steps, y, ws, st);
  return ou_matrices<__bf16>(ctx, dtype, p, g, steps, y, ws, st);
}

extern "C" int egnn_muon_step(egnn_ctx* ctx, const float* W, const float* g, const float* m, int32_t batch, int32_t rows, int32_t cols,
                              float lr, float beta, float weight_decay, int32_t steps, float* W_out, float* m_out, void* ws,
                              size_t ws_bytes, void* stream) {
  if (!ctx) return EGNN_EINVAL;
  if (int rc = ou_check(ctx, "muon_step", batch, rows, cols, steps)) return rc;
  if (batch == 0) return EGNN_OK;
  if (!W || !g || !m || !W_out || !m_out) return egnn_fail(ctx, EGNN_EINVAL, "muon_step: null pointer");
  const OuShape p = ou_shape(batch, rows, cols);
  if (!ws || (uintptr_t)ws % 256 || ws_bytes < ou_space(p, 2).bytes)
    return egnn_fail(ctx, EGNN_EWS, "muon_step: workspace too small or not 256-byte aligned");
  const float scale = (float)((double)lr * sqrt(rows > cols ? (double)rows / cols : 1.0));
  const float keep = (float)(1.0 - (double)lr * (double)weight_decay);
  return ou_run<float, 2>(ctx, p, OuInput<float>{g, m_out, beta}, m, m_out, steps, OuOut<float>{W_out, W, keep, scale}, ws,
                          (hipStream_t)stream);
}
