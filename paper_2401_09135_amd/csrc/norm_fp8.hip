// Norm with the residual's addition and an output in 8 bits (als_k_norm_fwd), and its backward pass (als_k_norm_bwd), for rows of up to 16384 elements.
//
// Memory bounds both: every tensor is read or written once.  A row stays in the registers of a wavefront (d <= 1024), of 256 threads (d <= 4096) or of 1024; a thread
// has 2 or 4 runs of 4 consecutive elements of it, so that a load or store of fp32 is 1 KB without gaps for a wavefront, and a block of 128 is 32 neighbouring lanes', whose
// scale needs no LDS.  The backward pass loads a row while it works on the one before.  16384 x 896, forward (fp32 input, all outputs) 40.3 us, 5.5 TB/s; backward (bf16 dy, all
// outputs) 47 us, 5 TB/s with the second launch that adds the gain's gradient; LayerNorm 41 and 48.  16384 x 512 20.4 and 25; 16384 x 1023 52 and 58 to 60; 2000 x 8192 47 and 60
// (LayerNorm 49 and 67); 1000 x 16000 52 and 68 (57 and 76).  With runs of 8, loaded behind branches, and no row ahead 16384 x 896 takes 9 and 6 % longer, 16384 x 1023 backward 23 %,
// 16384 x 512 backward 12 %; with 4 runs where 2 reach 16384 x 512 backward 10 %, 2000 x 8192 forward 22 %.
#include "fp8.h"

#include <type_traits>

namespace als {

namespace {

constexpr int NORM_MAX_D = 16384;
constexpr int NORM_LAUNCH_ROWS = 1 << 21;   // of a launch of the forward pass: a grid has fewer than 2^32 threads

template <typename F>
__device__ __forceinline__ F norm_wave_sum(F v) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o, 64);
  return v;
}
// the sum over the NT threads that hold a row; sh: NT / 64 numbers of their own, U of which are read at once
template <int NT, int U = NT / 64, typename F>
__device__ __forceinline__ F row_sum(F v, F* sh) {
  v = norm_wave_sum(v);
  if (NT == 64) return v;
  __syncthreads();   // the last reading of sh is over
  if ((threadIdx.x & 63) == 0) sh[threadIdx.x >> 6] = v;
  __syncthreads();
  F s = sh[0];
#pragma unroll U
  for (int i = 1; i < NT / 64; i++) s += sh[i];
  return s;
}

// Element c of a row whose address all lanes share, by a 32-bit offset: a register a lane instead of two
template <typename P>
__device__ __forceinline__ P* element(P* row, int c) {
  typedef typename std::conditional<std::is_const<P>::value, const char, char>::type byte;
  return reinterpret_cast<P*>(reinterpret_cast<byte*>(row) + (unsigned)c * (unsigned)sizeof(P));
}

// A thread's elements of a row as they lie in memory, runs of 4, run s at 4 (t + NT s).  What is loaded is not used, and so not waited for, before settle() and
// at(), and loads have no branches: a run that the row ends in or before is the row's last 4 elements in its place.
template <typename T, int NT, int RUNS>
struct RowPart {
  typedef T run __attribute__((ext_vector_type(4)));
  run v[RUNS];
  __device__ __forceinline__ void load(const T* row, int d, int t) {
    if (d >= 4) {
#pragma unroll
      for (int s = 0; s < RUNS; s++) {
        const int c = 4 * (t + NT * s);
        __builtin_memcpy(&v[s], element(row, c < d - 4 ? c : d - 4), sizeof(run));
      }
    } else {
#pragma unroll
      for (int i = 0; i < 3; i++) v[0][i] = row[i < d ? i : 0];
    }
  }
  // moves the elements of a run that the row ends in to their places
  __device__ __forceinline__ void settle(int d, int t) {
    if (d % 4 == 0) return;
    const T z = (T)0.0f;
    if (d < 4) {
      if (d < 3) v[0][2] = z;
      if (d < 2) v[0][1] = z;
      v[0][3] = z;
      return;
    }
#pragma unroll
    for (int s = 0; s < RUNS; s++) {
      const int k = 4 * (t + NT * s) - (d - 4);   // 1, 2 or 3 in such a run
      const run x = v[s];
      v[s] = k == 1 ? (run){x[1], x[2], x[3], z} : k == 2 ? (run){x[2], x[3], z, z} : k == 3 ? (run){x[3], z, z, z} : x;
    }
  }
  // 0 outside the row
  __device__ __forceinline__ float at(int s, int i, int d, int t) const { return 4 * (t + NT * s) < d ? (float)v[s][i] : 0.0f; }
};

struct NormFwdArgs {
  const void* x; const float* resid; const float* gain; float* total; bf16* y;
  uint8_t* q; uint8_t* scale; int64_t ld, ld_scale; int format;
  float* rstd; int rows, d; double eps;
};

// NT threads a row; NT = 64: four rows a workgroup
template <typename T, int NT, int RUNS, bool CENTER>
__global__ __launch_bounds__(NT == 64 ? 256 : NT) void norm_fwd_kernel(NormFwdArgs a) {
  __shared__ double sh[NT / 64];
  const int t = NT == 64 ? threadIdx.x & 63 : threadIdx.x;
  const int row = NT == 64 ? blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6) : blockIdx.x;
  if (row >= a.rows) return;   // a whole wavefront, or nobody where the threads of a row meet
  const int64_t base = (int64_t)row * a.d;
  RowPart<T, NT, RUNS> x;
  RowPart<float, NT, RUNS> resid, gain;
  x.load((const T*)a.x + base, a.d, t);
  if (a.resid) resid.load(a.resid + base, a.d, t);
  gain.load(a.gain, a.d, t);
  x.settle(a.d, t);
  float v[RUNS][4];
#pragma unroll
  for (int s = 0; s < RUNS; s++)
#pragma unroll
    for (int i = 0; i < 4; i++) v[s][i] = x.at(s, i, a.d, t);
  if (a.resid) {
    resid.settle(a.d, t);
#pragma unroll
    for (int s = 0; s < RUNS; s++) {
#pragma unroll
      for (int i = 0; i < 4; i++) v[s][i] += resid.at(s, i, a.d, t);
      store4(element(a.total + base, 4 * (t + NT * s)), a.d - 4 * (t + NT * s), v[s]);
    }
  }
  // Sums of a row in double: what they are off by is the same for the whole row, and turns as many of its 8-bit values as lie that near to a border between two.
  // 5 of the wavefronts' sums are read at once: all 16 are 32 registers, with which a CU has one workgroup of 1024 threads instead of two (2000 x 8192 19 % longer).
  double mean = 0.0;
  if (CENTER) {
    double sum = 0.0;
#pragma unroll
    for (int s = 0; s < RUNS; s++)
#pragma unroll
      for (int i = 0; i < 4; i++) sum += (double)v[s][i];
    mean = row_sum<NT, 5>(sum, sh) / a.d;
  }
  double ss = 0.0;
#pragma unroll
  for (int s = 0; s < RUNS; s++)
#pragma unroll
    for (int i = 0; i < 4; i++) {
      const double e = CENTER ? (4 * (t + NT * s) + i < a.d ? (double)v[s][i] - mean : 0.0) : (double)v[s][i];
      ss = fma(e, e, ss);
    }
  ss = row_sum<NT, 5>(ss, sh);
  // An output in 8 bits turns an error of one rounding into a step of 1/16 where it falls on a border: what follows is in double too and rounded once, at the end, so that no
  // row that fp32 holds is too large or too small on the way.  (Up to 4096 elements a row that costs nothing, 1000 x 16000 3 %, with a mean 4; 2000 x 8192 with a mean 8.)
  gain.settle(a.d, t);
  const double rd = 1.0 / sqrt(ss / a.d + a.eps);
  if (t == 0) a.rstd[row] = (float)rd;
#pragma unroll
  for (int s = 0; s < RUNS; s++) {
    const int c = 4 * (t + NT * s), n = a.d - c;
#pragma unroll
    for (int i = 0; i < 4; i++) v[s][i] = (float)((CENTER ? (double)v[s][i] - mean : (double)v[s][i]) * rd * (double)gain.at(s, i, a.d, t));
    if (a.y) store4(element(a.y + base, c), n, v[s]);
    if (a.q) {
      unsigned m = 0;
#pragma unroll
      for (int i = 0; i < 4; i++) m = max(m, fp8_magnitude(v[s][i]));
      const int b = fp8_scale_byte(lanes32_max(m), a.format);
      const float sc = fp8_scale(b);
      if (n > 0) {
        if ((t & 31) == 0) a.scale[(int64_t)row * a.ld_scale + c / 128] = (uint8_t)b;
        store4_bytes(element(a.q + (int64_t)row * a.ld, c), n, fp8_pack4(v[s][0], v[s][1], v[s][2], v[s][3], sc, a.format));
      }
    }
  }
}

struct NormBwdArgs {
  const void* dy; const float* total; const float* rstd; const float* gain; const float* ds_in; float* ds; bf16* lp;
  float* partial;   // [blocks][d]
  int rows, d;
};
// Rows of a workgroup's threads at a time: 4 of 64 threads, or one.  At most 512 workgroups, each of which leaves a row of partial sums of the gain's gradient.
int norm_bwd_blocks(int rows, int d) {
  const int at_once = d <= 1024 ? 4 : 1;
  const int b = (rows + at_once - 1) / at_once;
  return b < 512 ? b : 512;
}

template <typename T, int NT, int RUNS, bool CENTER>
__global__ __launch_bounds__(NT == 64 ? 256 : NT) void norm_bwd_kernel(NormBwdArgs a) {
  constexpr int AT_ONCE = NT == 64 ? 4 : 1;
  __shared__ float sh[NT / 64];
  __shared__ double sh_mean[CENTER ? NT / 64 : 1];
  __shared__ float parts[NT == 64 ? 3 : 1][NT == 64 ? 1024 : 1];
  const int t = NT == 64 ? threadIdx.x & 63 : threadIdx.x, w = NT == 64 ? __builtin_amdgcn_readfirstlane(threadIdx.x >> 6) : 0;
  const float inv_d = 1.0f / (float)a.d;
  float dg[RUNS][4];
  // The next row is loaded while one is worked on.  1024 threads with 4 runs have 128 registers each and no room for that; their gain and its gradient are in LDS (with all in
  // registers, some of them in scratch memory, 1000 rows of 16000 take 148 us).
  constexpr bool AHEAD = NT * RUNS <= 2048;
  __shared__ f32x4 kept[2][AHEAD ? 1 : RUNS][AHEAD ? 1 : NT];
  RowPart<float, NT, RUNS> gain, total, in;
  RowPart<T, NT, RUNS> dy;
  float rstd = 0.0f;
  auto load = [&](int row) {
    if (row >= a.rows) return;
    const int64_t base = (int64_t)row * a.d;
    rstd = a.rstd[row];
    total.load(a.total + base, a.d, t);
    dy.load((const T*)a.dy + base, a.d, t);
    if (AHEAD && a.ds_in) in.load(a.ds_in + base, a.d, t);
  };
  gain.load(a.gain, a.d, t);
  const int stride = gridDim.x * AT_ONCE;
  int row = blockIdx.x * AT_ONCE + w;
  if (AHEAD) load(row);
  gain.settle(a.d, t);
#pragma unroll
  for (int s = 0; s < RUNS; s++) {
#pragma unroll
    for (int i = 0; i < 4; i++) dg[s][i] = 0.0f;
    if (!AHEAD) {
      kept[0][s][t] = gain.v[s];
      kept[1][s][t] = (f32x4){0.0f, 0.0f, 0.0f, 0.0f};
    }
  }
  for (; row < a.rows; row += stride) {
    const int64_t base = (int64_t)row * a.d;
    int d = a.d;
    asm volatile("" : "+s"(d));   // comparisons with it are made in every row: two registers each to keep them for all rows are too many
    if (!AHEAD) load(row);
    total.settle(d, t);
    dy.settle(d, t);
    const float r = rstd;
    float x[RUNS][4], h[RUNS][4];
    double sx = 0.0;
    float sh1 = 0.0f, dot = 0.0f;
#pragma unroll
    for (int s = 0; s < RUNS; s++)
#pragma unroll
      for (int i = 0; i < 4; i++) {
        x[s][i] = total.at(s, i, d, t);
        h[s][i] = dy.at(s, i, d, t);
        if (CENTER) sx += (double)x[s][i];
      }
    RowPart<float, NT, RUNS> add = in;
    if (AHEAD) load(row + stride);
    // The mean in double, as in the forward pass: what it is off by is the same for the whole row, adds up in the gain's gradient, and is in fp32 a rounding times the mean over
    // the spread (rows of 896 with a mean of 1000 spreads: xh off by 5e-5 in the mean, 1.5e-4 at most).  That costs 1 to 2 % up to 4096 elements a row and 5 % above.  The mean is
    // taken off in two parts, halved with the row where the difference could leave fp32's range.
    const double mean = CENTER ? row_sum<NT>(sx, sh_mean) / d : 0.0;
    const float whole = (float)mean, half = fabsf(whole) > 0x1p100f ? 0.5f : 1.0f, off = -whole * half, rest = (float)(mean - (double)whole) * half, rc = half < 1.0f ? r * 2.0f : r;
#pragma unroll
    for (int s = 0; s < RUNS; s++) {
      if (!AHEAD) gain.v[s] = kept[0][s][t];
      f32x4 sum = AHEAD ? (f32x4){dg[s][0], dg[s][1], dg[s][2], dg[s][3]} : kept[1][s][t];
#pragma unroll
      for (int i = 0; i < 4; i++) {
        x[s][i] = (CENTER ? fmaf(x[s][i], half, off) - rest : x[s][i]) * rc;   // xh; outside the row h is 0
        sum[i] += h[s][i] * x[s][i];
        h[s][i] *= gain.at(s, i, d, t);
        sh1 += h[s][i];
        dot += h[s][i] * x[s][i];
        if (AHEAD) dg[s][i] = sum[i];
      }
      if (!AHEAD) kept[1][s][t] = sum;
    }
    dot = row_sum<NT>(dot, sh) * inv_d;
    const float m1 = CENTER ? row_sum<NT>(sh1, sh) * inv_d : 0.0f;
#pragma unroll
    for (int s = 0; s < RUNS; s++) {
#pragma unroll
      for (int i = 0; i < 4; i++) h[s][i] = r * (h[s][i] - m1 - x[s][i] * dot);
    }
    if (a.ds_in) {
      if (!AHEAD) add.load(a.ds_in + base, d, t);
      add.settle(d, t);
#pragma unroll
      for (int s = 0; s < RUNS; s++)
#pragma unroll
        for (int i = 0; i < 4; i++) h[s][i] += (float)add.v[s][i];
    }
#pragma unroll
    for (int s = 0; s < RUNS; s++) {
      const int c = 4 * (t + NT * s);
      store4(element(a.ds + base, c), d - c, h[s]);
      if (a.lp) store4(element(a.lp + base, c), d - c, h[s]);
    }
  }
  if (!AHEAD) {
#pragma unroll
    for (int s = 0; s < RUNS; s++) __builtin_memcpy(dg[s], &kept[1][s][t], 16);
  }
  float* out = a.partial + (int64_t)blockIdx.x * a.d;
  if (NT == 64) {   // the four wavefronts' sums, in their order
    if (w)
#pragma unroll
      for (int s = 0; s < RUNS; s++) __builtin_memcpy(parts[w - 1] + 4 * (t + NT * s), dg[s], 16);
    __syncthreads();
    if (w) return;
#pragma unroll
    for (int s = 0; s < RUNS; s++)
#pragma unroll
      for (int j = 0; j < 3; j++) {
        float o[4];
        __builtin_memcpy(o, parts[j] + 4 * (t + NT * s), 16);
#pragma unroll
        for (int i = 0; i < 4; i++) dg[s][i] += o[i];
      }
  }
#pragma unroll
  for (int s = 0; s < RUNS; s++) store4(element(out, 4 * (t + NT * s)), a.d - 4 * (t + NT * s), dg[s]);
}

// dgain = the sum of the blocks' rows, in the order of the blocks: 16 columns a workgroup, 64 groups of lanes each with every 64th row
__global__ __launch_bounds__(1024) void norm_dgain_kernel(const float* __restrict__ partial, float* __restrict__ dgain, int blocks, int d) {
  __shared__ float sh[64][17];
  const int lc = threadIdx.x & 15, c = blockIdx.x * 16 + lc, g = threadIdx.x >> 4;
  float s = 0.0f;
  if (c < d) {
    float v[8];   // blocks <= 512
#pragma unroll
    for (int i = 0; i < 8; i++) v[i] = g + 64 * i < blocks ? partial[(int64_t)(g + 64 * i) * d + c] : 0.0f;
#pragma unroll
    for (int i = 0; i < 8; i++) s += v[i];
  }
  sh[g][lc] = s;
  __syncthreads();
  if (threadIdx.x < 64) {   // lane g2 * 16 + lc: groups 16 g2 .. + 15, and then the four sums
    const int g2 = threadIdx.x >> 4;
    float r = 0.0f;
#pragma unroll
    for (int i = 0; i < 16; i++) r += sh[16 * g2 + i][lc];
    r += __shfl_xor(r, 16, 64);
    r += __shfl_xor(r, 32, 64);
    if (threadIdx.x < 16 && c < d) dgain[c] = r;
  }
}

}  // namespace

}  // namespace als

using namespace als;

// Launches KERNEL<T, NT, RUNS, CENTER> for a row of d: as few threads as hold it, in half as many runs where those reach
#define ALS_NORM_C(KERNEL, T, NT, RUNS, GRID) \
  do { \
    const dim3 grid_(GRID), block_(NT == 64 ? 256 : NT); \
    if (center) hipLaunchKernelGGL((KERNEL<T, NT, RUNS, true>), grid_, block_, 0, st, a); \
    else hipLaunchKernelGGL((KERNEL<T, NT, RUNS, false>), grid_, block_, 0, st, a); \
  } while (0)
#define ALS_NORM(KERNEL, T, GRID64, GRID) \
  do { \
    if (d <= 512) ALS_NORM_C(KERNEL, T, 64, 2, GRID64); \
    else if (d <= 1024) ALS_NORM_C(KERNEL, T, 64, 4, GRID64); \
    else if (d <= 2048) ALS_NORM_C(KERNEL, T, 256, 2, GRID); \
    else if (d <= 4096) ALS_NORM_C(KERNEL, T, 256, 4, GRID); \
    else if (d <= 8192) ALS_NORM_C(KERNEL, T, 1024, 2, GRID); \
    else ALS_NORM_C(KERNEL, T, 1024, 4, GRID); \
  } while (0)

static int check_norm(int rows, int d, int norm_kind, const char* what) {
  if (rows < 0 || rows > 1 << 30 || d < 1 || d > NORM_MAX_D) return set_error(ALS_ERR_INVALID, "%s: rows must be in 0..2^30 and d in 1..%d", what, NORM_MAX_D);
  if (norm_kind != ALS_NORM_RMS && norm_kind != ALS_NORM_LAYER) return set_error(ALS_ERR_INVALID, "%s: unknown norm_kind", what);
  return ALS_OK;
}

extern "C" int als_k_norm_fwd(const void* x, int dtype, const float* resid, const float* gain, float* total, void* y, const als_fp8* q, float* rstd,
                              int rows, int d, double eps, int norm_kind, void* stream) {
  int rc = check_norm(rows, d, norm_kind, "als_k_norm_fwd");
  if (!rc) rc = check_dtype(dtype, "als_k_norm_fwd");
  if (!rc && q) rc = check_fp8(q, rows, d, "als_k_norm_fwd, q");
  if (rc) return rc;
  if (q && q->block_rows != 1) return set_error(ALS_ERR_INVALID, "als_k_norm_fwd: q must have block_rows 1");
  if (!(eps >= 0) || eps > 1e30) return set_error(ALS_ERR_INVALID, "als_k_norm_fwd: eps must be finite and >= 0");
  if (rows == 0) return ALS_OK;   // buffers without elements may be null
  if (!y && !q) return set_error(ALS_ERR_INVALID, "als_k_norm_fwd: no output");
  if (!resid != !total) return set_error(ALS_ERR_INVALID, "als_k_norm_fwd: resid and total are both null or neither");
  if (!x || !gain || !rstd) return set_error(ALS_ERR_INVALID, "als_k_norm_fwd: null argument");
  if ((uintptr_t)x % (dtype == ALS_DTYPE_BF16 ? 2 : 4) || ((uintptr_t)resid | (uintptr_t)gain | (uintptr_t)total | (uintptr_t)rstd) % 4 || (uintptr_t)y % 2)
    return set_error(ALS_ERR_INVALID, "als_k_norm_fwd: a tensor is not aligned to its type");
  const bool center = norm_kind == ALS_NORM_LAYER;
  hipStream_t st = (hipStream_t)stream;
  for (int row0 = 0; row0 < rows; row0 += NORM_LAUNCH_ROWS) {
    const int n = rows - row0 < NORM_LAUNCH_ROWS ? rows - row0 : NORM_LAUNCH_ROWS;
    const int64_t at = (int64_t)row0 * d;
    NormFwdArgs a;
    a.x = (const char*)x + at * (dtype == ALS_DTYPE_BF16 ? 2 : 4);
    a.resid = resid ? resid + at : nullptr; a.gain = gain; a.total = total ? total + at : nullptr; a.y = y ? (bf16*)y + at : nullptr;
    a.q = q ? (uint8_t*)q->data + row0 * q->ld : nullptr; a.scale = q ? q->scale + row0 * q->ld_scale : nullptr;
    a.ld = q ? q->ld : 0; a.ld_scale = q ? q->ld_scale : 0; a.format = q ? q->format : 0;
    a.rstd = rstd + row0; a.rows = n; a.d = d; a.eps = eps;
    if (dtype == ALS_DTYPE_BF16) ALS_NORM(norm_fwd_kernel, bf16, (n + 3) / 4, n);
    else ALS_NORM(norm_fwd_kernel, float, (n + 3) / 4, n);
    ALS_CHECK_LAUNCH();
  }
  return ALS_OK;
}

extern "C" size_t als_k_norm_bwd_ws_bytes(int rows, int d) {
  if (rows < 0 || rows > 1 << 30 || d < 1 || d > NORM_MAX_D) return 0;
  return (size_t)norm_bwd_blocks(rows, d) * d * sizeof(float);
}

extern "C" int als_k_norm_bwd(const void* dy, int dtype, const float* total, const float* rstd, const float* gain, const float* ds_in, float* ds,
                              void* ds_lp, float* dgain, int rows, int d, int norm_kind, void* ws_dev, size_t ws_bytes, void* stream) {
  int rc = check_norm(rows, d, norm_kind, "als_k_norm_bwd");
  if (!rc) rc = check_dtype(dtype, "als_k_norm_bwd");
  if (rc) return rc;
  if (!dgain || (uintptr_t)dgain % 4) return set_error(ALS_ERR_INVALID, "als_k_norm_bwd: dgain is null or not aligned to its type");
  if (rows && (!dy || !total || !rstd || !gain || !ds || !ws_dev)) return set_error(ALS_ERR_INVALID, "als_k_norm_bwd: null argument");
  if ((uintptr_t)dy % (dtype == ALS_DTYPE_BF16 ? 2 : 4) || ((uintptr_t)total | (uintptr_t)rstd | (uintptr_t)gain | (uintptr_t)ds_in | (uintptr_t)ds) % 4 || (uintptr_t)ds_lp % 2)
    return set_error(ALS_ERR_INVALID, "als_k_norm_bwd: a tensor is not aligned to its type");
  if (rows && (uintptr_t)ws_dev % 16) return set_error(ALS_ERR_INVALID, "als_k_norm_bwd: workspace must be 16-byte aligned");
  if (ws_bytes < als_k_norm_bwd_ws_bytes(rows, d))
    return set_error(ALS_ERR_INVALID, "als_k_norm_bwd: workspace too small: %zu bytes given, %zu needed", ws_bytes, als_k_norm_bwd_ws_bytes(rows, d));
  NormBwdArgs a;
  a.dy = dy; a.total = total; a.rstd = rstd; a.gain = gain; a.ds_in = ds_in; a.ds = ds; a.lp = (bf16*)ds_lp; a.partial = (float*)ws_dev;
  a.rows = rows; a.d = d;
  const bool center = norm_kind == ALS_NORM_LAYER;
  hipStream_t st = (hipStream_t)stream;
  const int blocks = norm_bwd_blocks(rows, d);
  if (rows) {
    if (dtype == ALS_DTYPE_BF16) ALS_NORM(norm_bwd_kernel, bf16, blocks, blocks);
    else ALS_NORM(norm_bwd_kernel, float, blocks, blocks);
    ALS_CHECK_LAUNCH();
  }
  hipLaunchKernelGGL(norm_dgain_kernel, dim3((d + 15) / 16), dim3(1024), 0, st, a.partial, dgain, blocks, d);
  ALS_CHECK_LAUNCH();
  return ALS_OK;
}
