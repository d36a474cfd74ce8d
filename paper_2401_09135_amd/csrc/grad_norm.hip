// The global norm of a gradient that lies in many tensors (als_k_grad_norm), and clipping by it (als_k_grad_clip).
//
// norm = sqrt(sum of all squares).  Memory bounds it: 4 or 2 bytes read an element, and read and written once more where it is clipped.  Squares are formed and
// added in double: no square of a finite fp32 value leaves its range, and the sum over 10^8 elements keeps all digits of the result; at 6 TB/s a CU
// gets 2.5 elements a clock and could add 64.  The tensors of a launch are a table in the kernel's arguments; each is cut into chunks, the chunks
// of a launch are dealt to its workgroups in equal runs, and every workgroup leaves one partial sum, which one workgroup adds in order.
#include "fp8.h"

#include <algorithm>
#include <vector>

namespace als {

namespace {

constexpr int GN_TENSORS = 96;              // of a launch (its arguments stay below 4 KB)
constexpr int GN_BLOCKS = 2048;             // workgroups of a launch at most: 8 on every CU
constexpr int64_t GN_CHUNK = 16384;         // bytes

struct GradTable {
  const void* in[GN_TENSORS];
  void* out[GN_TENSORS];
  int64_t numel[GN_TENSORS];     // times 2, + 1 for bf16
  int64_t chunk0[GN_TENSORS + 1];
  int n;
};

// A tensor in pieces of 16 bytes of memory, the first and last of which may be shared with others: piece p holds elements p E - lead .. + E - 1
template <typename T>
struct Pieces {
  static constexpr int E = 16 / sizeof(T);
  const T* base;   // of piece 0, at or before the tensor
  int lead;        // elements of piece 0 that belong to others
  int64_t numel, count;
  __device__ __forceinline__ Pieces(const void* p, int64_t n) {
    lead = (int)((uintptr_t)p % 16 / sizeof(T));
    base = (const T*)p - lead;
    numel = n;
    count = (n + lead + E - 1) / E;
  }
  __device__ __forceinline__ bool whole(int64_t p) const { return p * E >= lead && p * E + E <= numel + lead; }
  __device__ __forceinline__ bool has(int64_t p, int e) const { const int64_t i = p * E + e; return i >= lead && i < numel + lead; }
  __device__ __forceinline__ void load(int64_t p, float (&v)[E]) const {
    if (whole(p)) {
      if constexpr (sizeof(T) == 4) {
        const f32x4 x = reinterpret_cast<const f32x4*>(base)[p];
#pragma unroll
        for (int e = 0; e < E; e++) v[e] = x[e];
      } else {
        const bf16x8 x = reinterpret_cast<const bf16x8*>(base)[p];
#pragma unroll
        for (int e = 0; e < E; e++) v[e] = (float)x[e];
      }
    } else {
#pragma unroll
      for (int e = 0; e < E; e++) v[e] = has(p, e) ? (float)base[p * E + e] : 0.0f;
    }
  }
};

__host__ __device__ inline int64_t chunk_pieces() { return GN_CHUNK / 16; }
// chunks of a tensor: as many as it may take for any alignment of its first element
inline int64_t chunks_of(int64_t numel, bool bf) {
  const int E = bf ? 8 : 4;
  return numel ? (numel + E - 1 + E - 1) / E / chunk_pieces() + 1 : 0;
}

__device__ __forceinline__ double wave_sum_f64(double v) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o, 64);
  return v;
}

// calls f(in, out, numel, bf16, first piece, last piece + 1) for the chunks of this workgroup
template <typename F>
__device__ __forceinline__ void for_chunks(const GradTable& t, F f) {
  const int64_t total = t.chunk0[t.n];
  int64_t c = total * blockIdx.x / gridDim.x;
  const int64_t end = total * (blockIdx.x + 1) / gridDim.x;
  if (c >= end) return;
  int lo = 0, hi = t.n;
  while (hi - lo > 1) {
    const int mid = (lo + hi) / 2;
    if (t.chunk0[mid] <= c) lo = mid; else hi = mid;
  }
  while (c < end) {
    while (t.chunk0[lo + 1] <= c) lo++;   // tensors without elements have no chunks
    const int64_t stop = t.chunk0[lo + 1] < end ? t.chunk0[lo + 1] : end;
    f(t.in[lo], t.out[lo], t.numel[lo] >> 1, (t.numel[lo] & 1) != 0, (c - t.chunk0[lo]) * chunk_pieces(), (stop - t.chunk0[lo]) * chunk_pieces());
    c = stop;
  }
}

template <typename T>
__device__ __forceinline__ double squares(const void* in, int64_t numel, int64_t p0, int64_t p1) {
  const Pieces<T> x(in, numel);
  if (p1 > x.count) p1 = x.count;
  double s = 0.0;
  for (int64_t p = p0 + threadIdx.x; p < p1; p += 256) {
    float v[Pieces<T>::E];
    x.load(p, v);
#pragma unroll
    for (int e = 0; e < Pieces<T>::E; e++) s = fma((double)v[e], (double)v[e], s);
  }
  return s;
}

__global__ __launch_bounds__(256) void grad_squares_kernel(GradTable t, double* __restrict__ partial) {
  __shared__ double sh[4];
  double s = 0.0;
  for_chunks(t, [&](const void* in, void*, int64_t numel, bool bf, int64_t p0, int64_t p1) {
    s += bf ? squares<bf16>(in, numel, p0, p1) : squares<float>(in, numel, p0, p1);
  });
  s = wave_sum_f64(s);
  if ((threadIdx.x & 63) == 0) sh[threadIdx.x >> 6] = s;
  __syncthreads();
  if (threadIdx.x == 0) partial[blockIdx.x] = sh[0] + sh[1] + sh[2] + sh[3];
}

// also leaves the norm in double in partial[0], if there is one
__global__ __launch_bounds__(1024) void grad_norm_kernel(double* partial, int64_t n, float* __restrict__ norm, float* log, const StepState* ss, int64_t log_offset) {
  __shared__ double sh[16];
  double s = 0.0;
  for (int64_t i = threadIdx.x; i < n; i += 1024) s += partial[i];
  s = wave_sum_f64(s);
  if ((threadIdx.x & 63) == 0) sh[threadIdx.x >> 6] = s;
  __syncthreads();
  if (threadIdx.x == 0) {
    for (int i = 1; i < 16; i++) s += sh[i];
    s = sqrt(s);
    norm[0] = (float)s;
    if (n) partial[0] = s;   // every sum has been read
    if (ss) log = ss->loss_out + ss->step + log_offset;
    if (log) log[0] = (float)s;
  }
}

template <typename T>
__device__ __forceinline__ void scale_pieces(const void* in, void* out, int64_t numel, int64_t p0, int64_t p1, double k) {
  constexpr int E = Pieces<T>::E;
  const Pieces<T> x(in, numel);
  if (p1 > x.count) p1 = x.count;
  T* o = (T*)out - x.lead;   // element i of piece p goes to o[p E + i]
  const bool aligned = ((uintptr_t)o % 16) == 0;
  auto scaled = [k](float g) { return (float)((double)g * k); };
  for (int64_t p = p0 + threadIdx.x; p < p1; p += 256) {
    float v[E];
    x.load(p, v);
    if (aligned && x.whole(p)) {
      if constexpr (sizeof(T) == 4) {
        reinterpret_cast<f32x4*>(o)[p] = (f32x4){scaled(v[0]), scaled(v[1]), scaled(v[2]), scaled(v[3])};
      } else {
        bf16x8 y;
#pragma unroll
        for (int e = 0; e < E; e++) y[e] = (bf16)scaled(v[e]);
        reinterpret_cast<bf16x8*>(o)[p] = y;
      }
    } else {
#pragma unroll
      for (int e = 0; e < E; e++)
        if (x.has(p, e)) o[p * E + e] = (T)scaled(v[e]);
    }
  }
}

// count: partial sums that each workgroup adds itself, in the order of grad_norm_kernel, the first one leaving the norm; 0: the norm is in partial[0].  The coefficient and the
// products with it are in double: a norm of finite gradients can leave fp32's range, and an output is then what it is there, and rounded once (half a percent of 10^8
// elements).
__global__ __launch_bounds__(256) void grad_clip_kernel(GradTable t, float* norm, double max_norm, const double* __restrict__ partial, int count) {
  double root;
  if (count) {
    __shared__ double sh[4];
    const double s = wave_sum_f64((int)threadIdx.x < count ? partial[threadIdx.x] : 0.0);
    if ((threadIdx.x & 63) == 0) sh[threadIdx.x >> 6] = s;
    __syncthreads();
    root = sqrt(sh[0] + sh[1] + sh[2] + sh[3]);
    if (blockIdx.x == 0 && threadIdx.x == 0) norm[0] = (float)root;
  } else {
    root = partial[0];
  }
  const double k = root <= max_norm ? 1.0 : max_norm / root;
  for_chunks(t, [&](const void* in, void* out, int64_t numel, bool bf, int64_t p0, int64_t p1) {
    if (k == 1.0 && in == out) return;   // nothing changes
    if (bf) scale_pieces<bf16>(in, out, numel, p0, p1, k);
    else scale_pieces<float>(in, out, numel, p0, p1, k);
  });
}

bool is_bf16(const int32_t* dtypes, int i) { return dtypes && dtypes[i] == ALS_DTYPE_BF16; }

// the tables of a list, one launch after the other; f(table, blocks, index of the launch's first partial sum)
template <typename F>
int for_launches(int n, const void* const* in, void* const* out, const int64_t* numel, const int32_t* dtypes, F f) {
  int64_t partial0 = 0;
  for (int i0 = 0; i0 < n;) {
    GradTable t;
    t.n = 0;
    t.chunk0[0] = 0;
    for (; i0 < n && t.n < GN_TENSORS; i0++) {
      if (!numel[i0]) continue;
      t.in[t.n] = in[i0]; t.out[t.n] = out ? out[i0] : nullptr;
      t.numel[t.n] = numel[i0] * 2 + is_bf16(dtypes, i0);
      t.chunk0[t.n + 1] = t.chunk0[t.n] + chunks_of(numel[i0], is_bf16(dtypes, i0));
      t.n++;
    }
    if (!t.n) continue;
    const int blocks = (int)std::min<int64_t>(t.chunk0[t.n], GN_BLOCKS);
    const int rc = f(t, blocks, partial0);
    if (rc) return rc;
    partial0 += blocks;
  }
  return ALS_OK;
}

int check_list(int n, const void* const* grads, const int64_t* numel, const int32_t* dtypes, const float* norm_out, const char* what) {
  if (n < 0 || n > (1 << 20)) return set_error(ALS_ERR_INVALID, "%s: bad count %d", what, n);
  if (!norm_out || (uintptr_t)norm_out % 4 || (n && (!grads || !numel))) return set_error(ALS_ERR_INVALID, "%s: null argument", what);
  for (int i = 0; i < n; i++) {
    if (numel[i] < 0 || numel[i] > (int64_t)1 << 48) return set_error(ALS_ERR_INVALID, "%s: tensor %d: bad element count", what, i);
    if (dtypes && dtypes[i] != ALS_DTYPE_F32 && dtypes[i] != ALS_DTYPE_BF16) return set_error(ALS_ERR_INVALID, "%s: tensor %d: unknown dtype %d", what, i, dtypes[i]);
    if (numel[i] && (!grads[i] || (uintptr_t)grads[i] % (is_bf16(dtypes, i) ? 2 : 4)))
      return set_error(ALS_ERR_INVALID, "%s: tensor %d is null or not aligned to its type", what, i);
  }
  return ALS_OK;
}
int check_list_ws(int n, const int64_t* numel, const void* ws, size_t ws_bytes, const char* what) {
  const size_t need = als_k_grad_norm_ws_bytes(n, numel);
  if (need && (!ws || (uintptr_t)ws % 16)) return set_error(ALS_ERR_INVALID, "%s: workspace must be non-null and 16-byte aligned", what);
  if (ws_bytes < need) return set_error(ALS_ERR_INVALID, "%s: workspace too small: %zu bytes given, %zu needed", what, ws_bytes, need);
  return ALS_OK;
}

}  // namespace

// the partial sums of a list; count: how many
static int grad_squares(int n, const void* const* grads, const int64_t* numel, const int32_t* dtypes, double* partial, int64_t& count, hipStream_t st) {
  count = 0;
  return for_launches(n, grads, nullptr, numel, dtypes, [&](const GradTable& t, int blocks, int64_t p0) {
    hipLaunchKernelGGL(grad_squares_kernel, dim3(blocks), dim3(256), 0, st, t, partial + p0);
    ALS_CHECK_LAUNCH();
    count = p0 + blocks;
    return ALS_OK;
  });
}

int grad_norm(int n, const void* const* grads, const int64_t* numel, const int32_t* dtypes, float* norm_out, double* partial, hipStream_t st, float* log,
              const StepState* ss, int64_t log_offset) {
  int64_t count = 0;
  int rc = grad_squares(n, grads, numel, dtypes, partial, count, st);
  if (rc) return rc;
  hipLaunchKernelGGL(grad_norm_kernel, dim3(1), dim3(1024), 0, st, partial, count, norm_out, log, ss, log_offset);
  ALS_CHECK_LAUNCH();
  return ALS_OK;
}

}  // namespace als

using namespace als;

extern "C" size_t als_k_grad_norm_ws_bytes(int n, const int64_t* numel) {
  // a launch takes GN_TENSORS tensors with elements; the count of its workgroups is largest if all are fp32
  if (n <= 0 || !numel) return 0;
  size_t blocks = 0;
  int64_t chunks = 0;
  int in_launch = 0;
  for (int i = 0; i < n; i++) {
    if (numel[i] <= 0) continue;
    chunks += chunks_of(numel[i], false);
    if (++in_launch == GN_TENSORS) {
      blocks += (size_t)std::min<int64_t>(chunks, GN_BLOCKS);
      chunks = 0;
      in_launch = 0;
    }
  }
  blocks += (size_t)std::min<int64_t>(chunks, GN_BLOCKS);
  return blocks * sizeof(double);
}

extern "C" int als_k_grad_norm(int n, const void* const* grads, const int64_t* numel, const int32_t* dtypes, float* norm_out, void* ws_dev,
                               size_t ws_bytes, void* stream) {
  int rc = check_list(n, grads, numel, dtypes, norm_out, "als_k_grad_norm");
  if (!rc) rc = check_list_ws(n, numel, ws_dev, ws_bytes, "als_k_grad_norm");
  if (rc) return rc;
  return grad_norm(n, grads, numel, dtypes, norm_out, (double*)ws_dev, (hipStream_t)stream);
}

extern "C" int als_k_grad_clip(int n, const void* const* grads, void* const* outs, const int64_t* numel, const int32_t* dtypes, double max_norm,
                               float* norm_out, void* ws_dev, size_t ws_bytes, void* stream) {
  int rc = check_list(n, grads, numel, dtypes, norm_out, "als_k_grad_clip");
  if (rc) return rc;
  if (!((float)max_norm > 0) || max_norm > 3.4e38) return set_error(ALS_ERR_INVALID, "als_k_grad_clip: max_norm must be positive and finite");
  if (n && !outs) return set_error(ALS_ERR_INVALID, "als_k_grad_clip: null argument");
  // No output may overlap another tensor: sorted by address, the outputs and the inputs that are no output must lie one behind the other.
  // (Inputs may overlap each other.)
  struct Range { uintptr_t begin, end; bool out; };
  try {
    std::vector<Range> r;
    r.reserve(2 * (size_t)n);
    for (int i = 0; i < n; i++) {
      if (!numel[i]) continue;
      const size_t size = is_bf16(dtypes, i) ? 2 : 4;
      if (!outs[i] || (uintptr_t)outs[i] % size) return set_error(ALS_ERR_INVALID, "als_k_grad_clip: output %d is null or not aligned to its type", i);
      r.push_back(Range{(uintptr_t)outs[i], (uintptr_t)outs[i] + (size_t)numel[i] * size, true});
      if (outs[i] != grads[i]) r.push_back(Range{(uintptr_t)grads[i], (uintptr_t)grads[i] + (size_t)numel[i] * size, false});
    }
    auto less = [](const Range& a, const Range& b) { return a.begin < b.begin; };
    if (!std::is_sorted(r.begin(), r.end(), less)) std::sort(r.begin(), r.end(), less);
    uintptr_t out_end = 0, any_end = 0;   // of those before
    for (const Range& x : r) {
      if (x.begin < (x.out ? any_end : out_end)) return set_error(ALS_ERR_INVALID, "als_k_grad_clip: an output overlaps another tensor");
      any_end = std::max(any_end, x.end);
      if (x.out) out_end = std::max(out_end, x.end);
    }
  } catch (...) {
    return set_error(ALS_ERR_INVALID, "out of host memory");
  }
  rc = check_list_ws(n, numel, ws_dev, ws_bytes, "als_k_grad_clip");
  double* partial = (double*)ws_dev;
  hipStream_t st = (hipStream_t)stream;
  int64_t count = 0;
  if (!rc) rc = grad_squares(n, grads, numel, dtypes, partial, count, st);
  if (rc) return rc;
  // up to 256 partial sums, one a thread, are added again by every workgroup that clips: a launch less (16 tensors of 7187 elements 12.2 us to 9.5,
  // of 60000, 240 sums, 12.2 to 9.8; in one launch no more can be added without a loop)
  const int again = count <= 256 && n <= GN_TENSORS ? (int)count : 0;
  if (!again) {
    hipLaunchKernelGGL(grad_norm_kernel, dim3(1), dim3(1024), 0, st, partial, count, norm_out, nullptr, nullptr, 0);
    ALS_CHECK_LAUNCH();
  }
  return for_launches(n, grads, outs, numel, dtypes, [&](const GradTable& t, int blocks, int64_t) {
    hipLaunchKernelGGL(grad_clip_kernel, dim3(blocks), dim3(256), 0, st, t, norm_out, max_norm, partial, again);
    ALS_CHECK_LAUNCH();
    return ALS_OK;
  });
}
