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
constexpr int OU_PARTS = 64;        // partial sums of squares per matrix
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
  const int lane = threadIdx.x & 63;
  double t = lane < parts ? part[lane] : 0.0;
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

// C = A B^T of one tile TILE x TILE: four waves, each a quarter (TILE / 2 squared) in 32 x 32 blocks.  64 contraction indices a
// turn, brought straight into one of two LDS buffers while the other is contracted.  A row of 128 bytes lies in LDS as eight
// pieces of 16 bytes, piece c at place c ^ (row & 7): eight lanes that read the same piece of eight rows meet all banks.
template <class T, int P, int TILE, OuProduct WHAT>
__global__ __launch_bounds__(256) void ou_product_kernel(OuShape p, OuOperands o, OuOut<T> out) {
  extern __shared__ uint4 smem[];                     // [2][2 operands][P][TILE][8]
  constexpr bool STEP = WHAT == OU_UPDATE || WHAT == OU_LAST;   // p x
  constexpr int PB = STEP ? 2 : P;
  constexpr int HALF = TILE / 2, B = HALF / 32, PLANE = TILE * 8, STAGE = 2 * P * PLANE;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const size_t z = blockIdx.z;
  const int i0 = blockIdx.y * TILE, j0 = blockIdx.x * TILE;
  const size_t plane_a = (size_t)o.I * o.K, plane_b = (size_t)o.J * o.K;
  const _Float16* A = o.A + z * P * plane_a;
  const _Float16* Bm = o.B + z * PB * plane_b;
  const int wi = (wave >> 1) * HALF, wj = (wave & 1) * HALF;

  // lane's place in a load of eight rows
  const int lrow = lane >> 3, lpiece = (lane & 7) ^ lrow;
  auto fetch = [&](int k0, int stage) {
    uint4* to = smem + stage * STAGE;
#pragma unroll
    for (int q = 0; q < P; ++q)
#pragma unroll
      for (int r = 0; r < TILE / 32; ++r) {
        const int row = (r * 4 + wave) * 8;
        const _Float16* a = A + q * plane_a + (size_t)min(i0 + row + lrow, o.I - 1) * o.K + k0 + lpiece * 8;
        const _Float16* b = Bm + q * plane_b + (size_t)min(j0 + row + lrow, o.J - 1) * o.K + k0 + lpiece * 8;
        __builtin_amdgcn_global_load_lds((ou_gp)a, (ou_lp)(to + q * PLANE + row * 8), 16, 0, 0);
        __builtin_amdgcn_global_load_lds((ou_gp)b, (ou_lp)(to + (P + q) * PLANE + row * 8), 16, 0, 0);
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
  fetch(0, 0);
  for (int k = 0; k < turns; ++k) {
    __syncthreads();      // this turn's operands are in LDS, the other buffer is free
    if (k + 1 < turns) fetch((k + 1) * 64, (k + 1) & 1);
    const uint4* sa = smem + (k & 1) * STAGE;
    const uint4* sb = sa + P * PLANE;
#pragma unroll
    for (int s = 0; s < 4; ++s) {
      ou_h8 a[B][P], b[B][P];
      const int place = (2 * s + hh) ^ (r32 & 7);
#pragma unroll
      for (int x = 0; x < B; ++x)
#pragma unroll
        for (int q = 0; q < P; ++q) {
          a[x][q] = __builtin_bit_cast(ou_h8, sa[q * PLANE + (wi + 32 * x + r32) * 8 + place]);
          b[x][q] = __builtin_bit_cast(ou_h8, sb[q * PLANE + (wj + 32 * x + r32) * 8 + place]);
        }
      if (P == 2) {
#pragma unroll
        for (int x = 0; x < B; ++x)
#pragma unroll
          for (int y = 0; y < B; ++y) acc[x][y] = __builtin_amdgcn_mfma_f32_32x32x16_f16(a[x][P - 1], b[y][0], acc[x][y], 0, 0, 0);
#pragma unroll
        for (int x = 0; x < B; ++x)
#pragma unroll
          for (int y = 0; y < B; ++y) acc[x][y] = __builtin_amdgcn_mfma_f32_32x32x16_f16(a[x][0], b[y][P - 1], acc[x][y], 0, 0, 0);
      }
#pragma unroll
      for (int x = 0; x < B; ++x)
#pragma unroll
        for (int y = 0; y < B; ++y) acc[x][y] = __builtin_amdgcn_mfma_f32_32x32x16_f16(a[x][0], b[y][0], acc[x][y], 0, 0, 0);
    }
  }

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

struct OuSpace { size_t part, x, xt, g, bytes; };
OuSpace ou_space(const OuShape& p, int pieces) {
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
  constexpr size_t lds = (size_t)2 * 2 * P * TILE * 128;
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
  const OuSpace s = ou_space(p, P);
  double* part = (double*)((char*)ws + s.part);
  _Float16* x = (_Float16*)((char*)ws + s.x);
  _Float16* xt = (_Float16*)((char*)ws + s.xt);
  _Float16* xt2 = (_Float16*)((char*)ws + s.xt + (s.xt - s.x));
  _Float16* g = (_Float16*)((char*)ws + s.g);
  _Float16* q = (_Float16*)((char*)ws + s.g + (s.bytes - s.g) / 2);
  const size_t size = (size_t)p.rows * p.cols;
  int parts = (int)((size + 4095) / 4096);
  parts = parts > OU_PARTS ? OU_PARTS : parts;
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
