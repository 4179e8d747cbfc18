// The norm of many gradients together, and the gradients scaled by what keeps it below a bound.
//
//   norm = sqrt(sum over tensors and values of g^2),  factor = min(1, most / (norm + 1e-6)),  g' = g factor rounded to the type.
// Squares and sums are fp64: no finite fp32 value overflows or vanishes, and the sum does not depend on how it is cut.  A norm that is not finite
// leaves every gradient as it is and gives the factor 0: there is no step to take.
//
// Two launches: pieces of the tensors are summed, each workgroup to a slot of its own; then every workgroup adds all slots, in the
// same order, and scales its pieces.  No atomics: the same bits every time.  The tensors' addresses travel as kernel arguments, so that a call
// copies nothing from host memory and can be captured; CG_TENSORS of them at a time.
//
// What bounds it is memory: the bound needs all gradients before the first is scaled, so they are read twice.  Measured: 100 M fp32 values to another place
// 65 + 146 us (6.2 and 5.5 TB/s), 24 tensors of together 417,000 values 4.8 + 5.3.
#include <algorithm>
#include "row_vectors.h"

namespace {

constexpr int CG_TENSORS = 96;        // of 40 bytes each: kernel arguments of just under 4 KB
constexpr int CG_THREADS = 256;
constexpr int CG_SLOTS = 1024;        // workgroups of a launch at most
constexpr int64_t CG_CACHED = 128 << 20;   // more than this and its results do not stay in the 256 MB cache: results go past it, so that what the second pass
                                      // reads again stays (100 M fp32 values 252 us, past the cache 220)
constexpr int CG_AHEAD = 4;           // vectors of a thread under way at once

struct CgTensor {
  const void* data;
  void* out;
  long n, first;                      // values; pieces of the tensors before it
  int dtype;
};
struct CgTable {
  CgTensor t[CG_TENSORS];
  int count, piece;                   // piece: values of a piece
  long pieces;
};

// calls f(tensor, first value, values) for the run of pieces of workgroup `block`; backwards: the last first
template <class F>
__device__ __forceinline__ void cg_pieces(const CgTable& p, long block, bool backwards, const F& f) {
  const long each = (p.pieces + gridDim.x - 1) / gridDim.x, begin = block * each, end = min(begin + each, p.pieces);
  if (begin >= end) return;
  const long from = backwards ? end - 1 : begin;
  int at = 0;                         // the last tensor that begins at `from` or before (tensors of no values are not in the table)
  for (int step = 64; step; step >>= 1)
    if (at + step < p.count && p.t[at + step].first <= from) at += step;
  for (long k = from; k >= begin && k < end; k += backwards ? -1 : 1) {
    while (at + 1 < p.count && p.t[at + 1].first <= k) ++at;
    while (p.t[at].first > k) --at;
    const CgTensor& t = p.t[at];
    const long first = (k - t.first) * p.piece;
    f(t, first, (int)min((long)p.piece, t.n - first));
  }
}

// calls f(first value, vector) for the vectors of a thread among n values at `data`, CG_AHEAD of them loaded at a time, and g(value) for the last values
// of the n that make no vector
template <class T, class F, class G>
__device__ __forceinline__ void cg_vectors(const T* data, int n, const F& f, const G& g) {
  typedef Rv<T, false> R;
  constexpr int V = R::V;
  const int vecs = n / V;
  for (int i = threadIdx.x; i < vecs; i += CG_THREADS * CG_AHEAD) {
    typename R::vec v[CG_AHEAD];
#pragma unroll
    for (int u = 0; u < CG_AHEAD; ++u) v[u] = *(const typename R::loose*)(data + min(i + u * CG_THREADS, vecs - 1) * V);
#pragma unroll
    for (int u = 0; u < CG_AHEAD; ++u)
      if (i + u * CG_THREADS < vecs) f((i + u * CG_THREADS) * V, v[u]);
  }
  if ((int)threadIdx.x < n - vecs * V) g(vecs * V + threadIdx.x);
}

__device__ __forceinline__ double cg_block_sum(double v) {
  __shared__ double part[CG_THREADS / 64];
  for (int d = 32; d; d >>= 1) v += __shfl_xor(v, d);
  __syncthreads();
  if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = v;
  __syncthreads();
  v = part[0];
  for (int w = 1; w < CG_THREADS / 64; ++w) v += part[w];
  return v;
}

template <class T>
__device__ __forceinline__ double cg_square(const CgTensor& t, long at, int n) {
  const T* g = (const T*)t.data + at;
  double sum = 0.0;
  auto add = [&](T v) { sum += (double)(float)v * (double)(float)v; };
  cg_vectors(g, n, [&](int, const typename Rv<T, false>::vec& v) {
#pragma unroll
    for (int i = 0; i < Rv<T, false>::V; ++i) add(v[i]);
  }, [&](int i) { add(g[i]); });
  return sum;
}

__global__ void __launch_bounds__(CG_THREADS) cg_square_kernel(CgTable p, double* slot) {
  double sum = 0.0;
  cg_pieces(p, blockIdx.x, false, [&](const CgTensor& t, long at, int n) {
    sum += t.dtype == EGNN_F32 ? cg_square<float>(t, at, n) : t.dtype == EGNN_F16 ? cg_square<_Float16>(t, at, n) : cg_square<__bf16>(t, at, n);
  });
  sum = cg_block_sum(sum);
  if (threadIdx.x == 0) slot[blockIdx.x] = sum;
}

template <class T, bool PAST>
__device__ __forceinline__ void cg_scale(const CgTensor& t, long at, int n, float by) {
  typedef typename Rv<T, false>::loose vec;
  const T* g = (const T*)t.data + at;
  T* out = (T*)t.out + at;
  cg_vectors(g, n, [&](int i, typename Rv<T, false>::vec v) {
#pragma unroll
    for (int k = 0; k < Rv<T, false>::V; ++k) v[k] = (T)((float)v[k] * by);
    if constexpr (PAST) __builtin_nontemporal_store((vec)v, (vec*)(out + i));
    else *(vec*)(out + i) = v;
  }, [&](int i) { out[i] = (T)((float)g[i] * by); });
}

// The second pass begins with what the first one read last, which the caches still hold.
template <bool PAST>
__global__ void __launch_bounds__(CG_THREADS) cg_scale_kernel(CgTable p, const double* slot, int slots, float most, float* norm, bool tell) {
  double sum = 0.0;
  for (int i = threadIdx.x; i < slots; i += CG_THREADS) sum += slot[i];
  const double length = sqrt(cg_block_sum(sum));
  const bool finite = length < (double)__builtin_inff() && (float)length < __builtin_inff();
  const float factor = !finite ? 0.0f : (float)fmin(1.0, (double)most / (length + 1e-6));
  if (tell && blockIdx.x == 0 && threadIdx.x == 0) {
    norm[0] = (float)length;
    norm[1] = factor;
  }
  const float by = finite ? factor : 1.0f;
  cg_pieces(p, gridDim.x - 1 - blockIdx.x, true, [&](const CgTensor& t, long at, int n) {
    if (by == 1.0f && t.out == t.data) return;
    if (t.dtype == EGNN_F32) cg_scale<float, PAST>(t, at, n, by);
    else if (t.dtype == EGNN_F16) cg_scale<_Float16, PAST>(t, at, n, by);
    else cg_scale<__bf16, PAST>(t, at, n, by);
  });
}

int cg_blocks(long pieces) { return (int)std::min<long>(std::max<long>(pieces, 1), CG_SLOTS); }

int cg_check(egnn_ctx* ctx, const char* who, const egnn_tensor* t, int32_t count) {
  const std::string at(who);
  if (count < 0 || (count > 0 && !t)) return egnn_fail(ctx, EGNN_EINVAL, at + ": no list of tensors");
  for (int32_t i = 0; i < count; ++i) {
    if (!rt_size(t[i].dtype)) return egnn_fail(ctx, EGNN_EINVAL, at + ": dtype must be EGNN_F32, EGNN_F16 or EGNN_BF16");
    if (t[i].n < 0 || t[i].n > ((int64_t)1 << 40)) return egnn_fail(ctx, EGNN_EINVAL, at + ": the values of a tensor must be in 0..2^40");
    if (!t[i].n) continue;
    if (!t[i].data || !t[i].out) return egnn_fail(ctx, EGNN_EINVAL, at + ": null pointer");
    if ((uintptr_t)t[i].data % rt_size(t[i].dtype) || (uintptr_t)t[i].out % rt_size(t[i].dtype))
      return egnn_fail(ctx, EGNN_EINVAL, at + ": a tensor that is not aligned to its values");
  }
  return EGNN_OK;
}

// What is written must overlap nothing else of the list, and its own source only as a whole: else results would depend on the order of
// workgroups (a tensor that is in the list twice would be scaled twice).
bool cg_overlaps(const egnn_tensor* t, int32_t count) {
  struct Range { uintptr_t begin, end; int32_t tensor; bool written; };
  std::vector<Range> all;
  all.reserve(2 * (size_t)count);
  for (int32_t i = 0; i < count; ++i) {
    if (!t[i].n) continue;
    const uintptr_t size = (uintptr_t)t[i].n * rt_size(t[i].dtype);
    if (t[i].data != t[i].out) all.push_back({(uintptr_t)t[i].data, (uintptr_t)t[i].data + size, i, false});
    all.push_back({(uintptr_t)t[i].out, (uintptr_t)t[i].out + size, i, true});
  }
  std::sort(all.begin(), all.end(), [](const Range& a, const Range& b) { return a.begin < b.begin; });
  uintptr_t any = 0, written = 0;      // ends of what came before, of all and of what is written
  for (const Range& r : all) {
    if (r.begin < written || (r.written && r.begin < any)) return true;
    any = std::max(any, r.end);
    if (r.written) written = std::max(written, r.end);
  }
  return false;
}

// Tables of up to CG_TENSORS tensors that have values, one after the other.  A piece is what a workgroup reads at once, 4,096 to 16,384 values: fewer where all
// values make few workgroups.
struct CgWalk {
  const egnn_tensor* t;
  int32_t count, at = 0, piece = 0;
  bool past = false;
  bool next(CgTable& p) {
    if (!piece) {
      int64_t all = 0, bytes = 0;
      for (int32_t i = 0; i < count; ++i) {
        all += t[i].n;
        bytes += t[i].n * rt_size(t[i].dtype);
      }
      past = bytes > CG_CACHED;
      for (piece = 16384; piece > 4096 && all / piece < CG_SLOTS; piece /= 2) {}
    }
    p.count = 0;
    p.pieces = 0;
    p.piece = piece;
    for (; at < count && p.count < CG_TENSORS; ++at) {
      if (!t[at].n) continue;
      p.t[p.count++] = {t[at].data, t[at].out, (long)t[at].n, p.pieces, t[at].dtype};
      p.pieces += (long)((t[at].n + piece - 1) / piece);
    }
    return p.count > 0;
  }
};

}  // namespace

extern "C" int egnn_clip_gradients_workspace_bytes(const egnn_ctx* ctx, const egnn_tensor* tensors, int32_t n_tensors, size_t* bytes) {
  egnn_ctx* c = const_cast<egnn_ctx*>(ctx);
  if (!ctx || !bytes) return egnn_fail(c, EGNN_EINVAL, "clip_gradients_workspace_bytes: bad argument");
  if (int rc = cg_check(c, "clip_gradients_workspace_bytes", tensors, n_tensors)) return rc;
  CgTable p;
  size_t slots = 0;
  for (CgWalk w{tensors, n_tensors}; w.next(p);) slots += (size_t)cg_blocks(p.pieces);
  *bytes = slots * sizeof(double);
  return EGNN_OK;
}

extern "C" int egnn_clip_gradients(egnn_ctx* ctx, const egnn_tensor* tensors, int32_t n_tensors, float max_norm, float* norm, void* ws,
                                   size_t ws_bytes, void* stream) {
  if (!ctx) return EGNN_EINVAL;
  if (int rc = cg_check(ctx, "clip_gradients", tensors, n_tensors)) return rc;
  if (!(max_norm > 0.0f)) return egnn_fail(ctx, EGNN_EINVAL, "clip_gradients: max_norm must be > 0");
  if (!norm) return egnn_fail(ctx, EGNN_EINVAL, "clip_gradients: null pointer");
  try {
    if (cg_overlaps(tensors, n_tensors)) return egnn_fail(ctx, EGNN_EINVAL, "clip_gradients: what is written overlaps another tensor of the list");
  } catch (const std::exception&) {
    return egnn_fail(ctx, EGNN_EINVAL, "clip_gradients: no host memory for the list");
  }
  size_t need = 0;
  egnn_clip_gradients_workspace_bytes(ctx, tensors, n_tensors, &need);
  if (need && (!ws || (uintptr_t)ws % 256 || ws_bytes < need))
    return egnn_fail(ctx, EGNN_EWS, "clip_gradients: workspace too small or not 256-byte aligned");
  hipStream_t st = (hipStream_t)stream;
  double* slot = (double*)ws;
  CgTable p;
  int slots = 0;
  for (CgWalk w{tensors, n_tensors}; w.next(p);) {
    hipLaunchKernelGGL(cg_square_kernel, dim3(cg_blocks(p.pieces)), dim3(CG_THREADS), 0, st, p, slot + slots);
    slots += cg_blocks(p.pieces);
  }
  bool tell = true;
  CgWalk w{tensors, n_tensors};
  while (w.next(p) || tell) {
    hipLaunchKernelGGL(w.past ? cg_scale_kernel<true> : cg_scale_kernel<false>, dim3(cg_blocks(p.pieces)), dim3(CG_THREADS), 0, st, p, (const double*)slot, slots,
                       max_norm, norm, tell);
    tell = false;
  }
  EGNN_LAUNCH_CHECK(ctx, "clip_gradients");
  return EGNN_OK;
}
