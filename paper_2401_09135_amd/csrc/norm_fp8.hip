// Norm with the residual's addition and an output in 8 bits (als_k_norm_fwd), and its backward pass (als_k_norm_bwd), for rows of up to 16384 elements.
//
// Memory bounds both: every tensor is read or written once.  A row stays in the registers of a wavefront (d <= 1024), of 256 threads (d <= 4096) or of
// 1024; a thread has up to 2 runs of 8 consecutive elements of it, so that a block of 128 is 16 neighbouring lanes' and its scale needs no LDS.
#include "fp8.h"

namespace als {

namespace {

constexpr int NORM_MAX_D = 16384;
constexpr int NORM_LAUNCH_ROWS = 1 << 21;   // of a launch of the forward pass: a grid has fewer than 2^32 threads

__device__ __forceinline__ float norm_wave_sum(float v) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o, 64);
  return v;
}
// the sum over the NT threads that hold a row; sh: NT / 64 floats of their own
template <int NT>
__device__ __forceinline__ float row_sum(float v, float* sh) {
  v = norm_wave_sum(v);
  if (NT == 64) return v;
  __syncthreads();   // the last reading of sh is over
  if ((threadIdx.x & 63) == 0) sh[threadIdx.x >> 6] = v;
  __syncthreads();
  float s = sh[0];
#pragma unroll
  for (int i = 1; i < NT / 64; i++) s += sh[i];
  return s;
}

constexpr int NORM_RUNS = 2;   // runs of 8 elements of a thread

struct NormFwdArgs {
  const void* x; const float* resid; const float* gain; float* total; bf16* y;
  uint8_t* q; uint8_t* scale; int64_t ld, ld_scale; int format;
  float* rstd; int rows, d; float eps;
};

// NT threads a row; NT = 64: four rows a workgroup
template <typename T, int NT, bool CENTER>
__global__ __launch_bounds__(NT == 64 ? 256 : NT) void norm_fwd_kernel(NormFwdArgs a) {
  __shared__ float sh[NT / 64];
  const int t = NT == 64 ? threadIdx.x & 63 : threadIdx.x;
  const int row = NT == 64 ? blockIdx.x * 4 + (threadIdx.x >> 6) : blockIdx.x;
  if (row >= a.rows) return;   // a whole wavefront, or nobody where the threads of a row meet
  const int64_t base = (int64_t)row * a.d;
  float v[NORM_RUNS][8], e[NORM_RUNS][8];
  float sum = 0.0f;
#pragma unroll
  for (int s = 0; s < NORM_RUNS; s++) load8((const T*)a.x + base + 8 * (t + NT * s), a.d - 8 * (t + NT * s), v[s]);
  if (a.resid) {
#pragma unroll
    for (int s = 0; s < NORM_RUNS; s++) load8(a.resid + base + 8 * (t + NT * s), a.d - 8 * (t + NT * s), e[s]);
#pragma unroll
    for (int s = 0; s < NORM_RUNS; s++) {
#pragma unroll
      for (int i = 0; i < 8; i++) v[s][i] += e[s][i];
      store8(a.total + base + 8 * (t + NT * s), a.d - 8 * (t + NT * s), v[s]);
    }
  }
#pragma unroll
  for (int s = 0; s < NORM_RUNS; s++) load8(a.gain + 8 * (t + NT * s), a.d - 8 * (t + NT * s), e[s]);
  if (CENTER)
#pragma unroll
    for (int s = 0; s < NORM_RUNS; s++)
#pragma unroll
      for (int i = 0; i < 8; i++) sum += v[s][i];
  if (CENTER) {
    const float mean = row_sum<NT>(sum, sh) / (float)a.d;
#pragma unroll
    for (int s = 0; s < NORM_RUNS; s++)
#pragma unroll
      for (int i = 0; i < 8; i++)
        if (8 * (t + NT * s) + i < a.d) v[s][i] -= mean;
  }
  float ss = 0.0f;
#pragma unroll
  for (int s = 0; s < NORM_RUNS; s++)
#pragma unroll
    for (int i = 0; i < 8; i++) ss += v[s][i] * v[s][i];
  ss = row_sum<NT>(ss, sh);
  // rstd in two parts, and each product with what its rounding left: an output in 8 bits turns an error of one rounding into a step of 1/16 where it falls on a border,
  // and what follows is rounded once.  (0.5 us of 48.)
  const double rd = 1.0 / sqrt((double)ss / a.d + (double)a.eps);
  const float r = (float)rd, r_rest = (float)(rd - (double)r);
  if (t == 0) a.rstd[row] = r;
#pragma unroll
  for (int s = 0; s < NORM_RUNS; s++) {
    const int c = 8 * (t + NT * s), n = a.d - c;
#pragma unroll
    for (int i = 0; i < 8; i++) {
      const float p = v[s][i] * e[s][i], p_rest = fmaf(v[s][i], e[s][i], -p);
      v[s][i] = fmaf(p, r, fmaf(p, r_rest, p_rest * r));
    }
    if (a.y) store8(a.y + base + c, n, v[s]);
    if (a.q) {
      unsigned m = 0;
#pragma unroll
      for (int i = 0; i < 8; i++) m = max(m, fp8_magnitude(v[s][i]));
      const int b = fp8_scale_byte(lanes16_max(m), a.format);
      const float sc = fp8_scale(b);
      if (n > 0) {
        if ((t & 15) == 0) a.scale[(int64_t)row * a.ld_scale + c / 128] = (uint8_t)b;
        store8_bytes(a.q + (int64_t)row * a.ld + c, n, fp8_pack4(v[s][0], v[s][1], v[s][2], v[s][3], sc, a.format),
                     fp8_pack4(v[s][4], v[s][5], v[s][6], v[s][7], sc, a.format));
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

template <typename T, int NT, bool CENTER>
__global__ __launch_bounds__(NT == 64 ? 256 : NT) void norm_bwd_kernel(NormBwdArgs a) {
  constexpr int AT_ONCE = NT == 64 ? 4 : 1;
  __shared__ float sh[NT / 64];
  __shared__ float parts[NT == 64 ? 3 : 1][NT == 64 ? 1024 : 1];
  const int t = NT == 64 ? threadIdx.x & 63 : threadIdx.x, w = NT == 64 ? threadIdx.x >> 6 : 0;
  const float inv_d = 1.0f / (float)a.d;
  float dg[NORM_RUNS][8], g[NORM_RUNS][8];
#pragma unroll
  for (int s = 0; s < NORM_RUNS; s++) {
    load8(a.gain + 8 * (t + NT * s), a.d - 8 * (t + NT * s), g[s]);
#pragma unroll
    for (int i = 0; i < 8; i++) dg[s][i] = 0.0f;
  }
  for (int row = blockIdx.x * AT_ONCE + w; row < a.rows; row += gridDim.x * AT_ONCE) {
    const int64_t base = (int64_t)row * a.d;
    const float r = a.rstd[row];
    float x[NORM_RUNS][8], h[NORM_RUNS][8];
    float sx = 0.0f, sh1 = 0.0f, dot = 0.0f;
#pragma unroll
    for (int s = 0; s < NORM_RUNS; s++) {
      const int c = 8 * (t + NT * s), n = a.d - c;
      load8(a.total + base + c, n, x[s]);
      load8((const T*)a.dy + base + c, n, h[s]);
      if (CENTER)
#pragma unroll
        for (int i = 0; i < 8; i++) sx += x[s][i];
    }
    const float mean = CENTER ? row_sum<NT>(sx, sh) * inv_d : 0.0f;
#pragma unroll
    for (int s = 0; s < NORM_RUNS; s++)
#pragma unroll
      for (int i = 0; i < 8; i++) {
        const bool in = 8 * (t + NT * s) + i < a.d;
        x[s][i] = CENTER ? (in ? (x[s][i] - mean) * r : 0.0f) : x[s][i] * r;   // xh
        dg[s][i] += h[s][i] * x[s][i];
        h[s][i] *= g[s][i];
        sh1 += h[s][i];
        dot += h[s][i] * x[s][i];
      }
    dot = row_sum<NT>(dot, sh) * inv_d;
    const float m1 = CENTER ? row_sum<NT>(sh1, sh) * inv_d : 0.0f;
#pragma unroll
    for (int s = 0; s < NORM_RUNS; s++) {
      const int c = 8 * (t + NT * s), n = a.d - c;
      float o[8];
#pragma unroll
      for (int i = 0; i < 8; i++) o[i] = r * (h[s][i] - m1 - x[s][i] * dot);
      if (a.ds_in) {
        float in[8];
        load8(a.ds_in + base + c, n, in);
#pragma unroll
        for (int i = 0; i < 8; i++) o[i] += in[i];
      }
      store8(a.ds + base + c, n, o);
      if (a.lp) store8(a.lp + base + c, n, o);
    }
  }
  float* out = a.partial + (int64_t)blockIdx.x * a.d;
  if (NT == 64) {   // the four wavefronts' sums, in their order
    if (w)
#pragma unroll
      for (int s = 0; s < NORM_RUNS; s++) __builtin_memcpy(parts[w - 1] + 8 * (t + NT * s), dg[s], 32);
    __syncthreads();
    if (w) return;
#pragma unroll
    for (int s = 0; s < NORM_RUNS; s++)
#pragma unroll
      for (int j = 0; j < 3; j++) {
        float o[8];
        load8(parts[j] + 8 * (t + NT * s), 8, o);
#pragma unroll
        for (int i = 0; i < 8; i++) dg[s][i] += o[i];
      }
  }
#pragma unroll
  for (int s = 0; s < NORM_RUNS; s++) store8(out + 8 * (t + NT * s), a.d - 8 * (t + NT * s), dg[s]);
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

// Launches KERNEL<T, NT, CENTER> for a row of d
#define ALS_NORM_C(KERNEL, T, NT, GRID) \
  do { \
    const dim3 grid_(GRID), block_(NT == 64 ? 256 : NT); \
    if (center) hipLaunchKernelGGL((KERNEL<T, NT, true>), grid_, block_, 0, st, a); \
    else hipLaunchKernelGGL((KERNEL<T, NT, false>), grid_, block_, 0, st, a); \
  } while (0)
#define ALS_NORM(KERNEL, T, GRID64, GRID) \
  do { \
    if (d <= 1024) ALS_NORM_C(KERNEL, T, 64, GRID64); \
    else if (d <= 4096) ALS_NORM_C(KERNEL, T, 256, GRID); \
    else ALS_NORM_C(KERNEL, T, 1024, GRID); \
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
  if (!y && !q) return set_error(ALS_ERR_INVALID, "als_k_norm_fwd: no output");
  if (!resid != !total) return set_error(ALS_ERR_INVALID, "als_k_norm_fwd: resid and total are both null or neither");
  if (rows == 0) return ALS_OK;
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
    a.rstd = rstd + row0; a.rows = n; a.d = d; a.eps = (float)eps;
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
