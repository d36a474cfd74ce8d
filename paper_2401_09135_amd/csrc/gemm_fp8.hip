// Products of matrices in 8 bits: the entry point, which tile and how many shares of K it takes, and the sum of the shares (gemm_fp8_kernels.h has the kernels)
#include "gemm_fp8_kernels.h"

#include <algorithm>
#include <atomic>

namespace als {

extern template int gemm_fp8_launch<0, 0>(Fp8Args, int, Fp8Out, hipStream_t);
extern template int gemm_fp8_launch<0, 1>(Fp8Args, int, Fp8Out, hipStream_t);
extern template int gemm_fp8_launch<1, 0>(Fp8Args, int, Fp8Out, hipStream_t);
extern template int gemm_fp8_launch<1, 1>(Fp8Args, int, Fp8Out, hipStream_t);

namespace {

// C = R + the shares' partial sums, in their order
template <typename TO>
__global__ __launch_bounds__(256) void gemm_fp8_reduce_kernel(const float* __restrict__ partial, int nsplit, int64_t stride, TO* C, int64_t ldc, const float* R,
                                                              int64_t ldr, int M, int N) {
  // partial sums have rows of N4 floats, N rounded up to 4, so that four columns are aligned there
  const int n4 = (N + 3) / 4;
  const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (i >= (int64_t)M * n4) return;
  const int row = (int)(i / n4), col = (int)(i - (int64_t)row * n4) * 4;
  const f32x4* p = reinterpret_cast<const f32x4*>(partial) + i;
  f32x4 v = *p;
  for (int s = 1; s < nsplit; s++) v += p[s * (stride / 4)];
  TO* o = C + (int64_t)row * ldc + col;
  const float* r = R ? R + (int64_t)row * ldr + col : nullptr;
  if (col + 4 <= N && (((uintptr_t)o) & (4 * sizeof(TO) - 1)) == 0 && (((uintptr_t)r) & 15) == 0) {
    if (r) v += *reinterpret_cast<const f32x4*>(r);
    if constexpr (sizeof(TO) == 4) {
      *reinterpret_cast<f32x4*>(o) = v;
    } else {
      bf16x4 y;
#pragma unroll
      for (int e = 0; e < 4; e++) y[e] = (bf16)v[e];
      *reinterpret_cast<bf16x4*>(o) = y;
    }
  } else {
#pragma unroll
    for (int e = 0; e < 4; e++)
      if (col + e < N) o[e] = (TO)(r ? v[e] + r[e] : v[e]);
  }
}

// ---- which kernel ---------------------------------------------------------------------------------
// Tiles of 256, 128 or 64 and shares of K: the least of an estimate in us, whose constants were fitted to the times of 3 to 27 choices each for 150 products of 1 to
// 16384 rows, 16 to 8192 columns and K of 32 to 16384, both result types.  What it chooses takes 0.6 % longer than the best of them in the mean and 18 % at
// worst; tiles of 256 alone would take 2.6 times as long, of 128 1.5, of 64 1.2, the best tile without shares of K 1.14.
//   a slice of a tile takes its latency (1.55, 0.58 or 0.25 us; fp32 results 1.35 to 1.45 times that; two tiles of 64 share a CU and take 1.8), a tile 6.4, 2.5 or 1.9 us besides,
//   a CU gets 54 KB of operands a us at most; shares cost 1.4 us, 0.2 each and their partial sums, written and read at 5.2 TB/s.
// In us, tile / shares: 896 x 3584 x 15315 bf16 128/1 83, 256/4 92, 256/1 182, 64/1 156; fp32 256/4 102, 128/1 108, 256/1 263; 1024 x 896 x 3584 64/1 12, 128/1 18, 256/1 44;
// 2048 x 2048 x 2048 128/1 14, 64/1 20, 256/1 28; 1 x 4096 x 4096 64/4 8.9, 64/1 12.6, 128/4 11; 16384 x 896 x 896 256/1 20, 128/1 29, 64/1 36.
struct Fp8Plan { int tile, nsplit; };
std::atomic<int> g_fp8_tile{0}, g_fp8_shares{0};   // als_k_set_gemm_fp8

// tiles and shares that fp8_divide can number
bool fp8_numbered(int M, int N, int tile, int shares) { return gemm_tiles(M, N, tile, tile) * gemm_tiles(M, N, tile, tile) * shares < (int64_t)1 << 32; }

size_t fp8_ws_bytes(int M, int N, int nsplit) { return nsplit > 1 ? (size_t)nsplit * M * ((size_t)(N + 3) / 4 * 4) * 4 : 0; }

Fp8Plan fp8_plan(int M, int N, int K, bool wide, size_t ws_bytes) {
  const int nkt = (K + 127) / 128;
  Fp8Plan best{64, 1};
  if (nkt == 0) return best;
  const int tile_hook = g_fp8_tile.load(std::memory_order_relaxed), shares_hook = g_fp8_shares.load(std::memory_order_relaxed);
  if (tile_hook) {
    best.tile = tile_hook;
    best.nsplit = std::min(shares_hook, nkt);
    if (fp8_ws_bytes(M, N, best.nsplit) > ws_bytes || !fp8_numbered(M, N, best.tile, best.nsplit)) best.nsplit = 1;
    return best;
  }
  struct Kind { int tile; double slice, wide, tile_us; };
  static constexpr Kind kinds[] = {{256, 1.55, 1.35, 6.4}, {128, 0.58, 1.45, 2.5}, {64, 0.25, 1.4, 1.9}};
  static constexpr int shares[] = {1, 2, 3, 4, 6, 8, 12, 16, 24};
  double best_us = 1e30;
  for (const Kind& k : kinds)
    for (int s : shares) {
      if (s > 1 && (s > nkt / 2 || fp8_ws_bytes(M, N, s) > std::min(ws_bytes, (size_t)256 << 20) || !fp8_numbered(M, N, k.tile, s))) break;
      const int64_t tiles = gemm_tiles(M, N, k.tile, k.tile) * s, on_cu = (tiles + 255) / 256;
      const int slices = (nkt + s - 1) / s;
      const double slice = k.slice * (wide ? k.wide : 1.0);
      double us = k.tile == 64 ? (on_cu + 1) / 2 * (slices * slice * (on_cu > 1 ? 1.8 : 1.0) + k.tile_us) : on_cu * (slices * slice + k.tile_us);
      us = std::max(us, on_cu * slices * (256.0 * k.tile) / 54e3);
      if (s > 1) us += 1.4 + 0.2 * s + (double)M * N * (8.0 * s + (wide ? 4 : 2)) / 5.2e6;
      if (us < best_us) {
        best_us = us;
        best = Fp8Plan{k.tile, s};
      }
    }
  return best;
}

int launch_fp8(const Fp8Args& g, int fa, int fb, int tile, Fp8Out out, hipStream_t st) {
  if (fa == ALS_FP8_E4M3) return fb == ALS_FP8_E4M3 ? gemm_fp8_launch<0, 0>(g, tile, out, st) : gemm_fp8_launch<0, 1>(g, tile, out, st);
  return fb == ALS_FP8_E4M3 ? gemm_fp8_launch<1, 0>(g, tile, out, st) : gemm_fp8_launch<1, 1>(g, tile, out, st);
}

int run_fp8(const Fp8Args& g, int fa, int fb, void* ws, size_t ws_bytes, hipStream_t st) {
  const Fp8Plan plan = fp8_plan(g.M, g.N, g.K, !g.c_bf16, ws_bytes);
  if (plan.nsplit <= 1) return launch_fp8(g, fa, fb, plan.tile, g.c_bf16 ? FP8_BF16 : FP8_F32, st);
  Fp8Args p = g;   // partial sums: fp32, [nsplit][M][N rounded up to 4]
  p.nsplit = plan.nsplit;
  p.ldc = (g.N + 3) / 4 * 4;
  p.split_stride = g.M * p.ldc;
  p.c = ws; p.c_size = 4; p.r = nullptr;
  const int rc = launch_fp8(p, fa, fb, plan.tile, g.c_bf16 ? FP8_PARTIAL : FP8_F32, st);
  if (rc) return rc;
  const dim3 grid((unsigned)((g.M * (p.ldc / 4) + 255) / 256));
  if (g.c_bf16) hipLaunchKernelGGL(gemm_fp8_reduce_kernel<bf16>, grid, dim3(256), 0, st, (const float*)ws, p.nsplit, p.split_stride, (bf16*)g.c, g.ldc, g.r, g.ldr, g.M, g.N);
  else hipLaunchKernelGGL(gemm_fp8_reduce_kernel<float>, grid, dim3(256), 0, st, (const float*)ws, p.nsplit, p.split_stride, (float*)g.c, g.ldc, g.r, g.ldr, g.M, g.N);
  ALS_CHECK_LAUNCH();
  return ALS_OK;
}

int gemm_fp8(Fp8Args g, int fa, int fb, void* ws, size_t ws_bytes, hipStream_t st) {
  // tiles are numbered in 16 bits (fp8_divide); more take several launches, by rows
  const int rows = (int)((1 << 16) / gemm_tiles(1, g.N, 64, 64) * 64 / 256 * 256);
  if (g.M > rows) {
    for (int m = 0; m < g.M; m += rows) {
      Fp8Args p = g;
      p.a = g.a + (int64_t)m * g.lda;
      p.sa = g.sa + (int64_t)(m >> g.sha) * g.lda_s;
      p.c = (char*)g.c + (int64_t)m * g.ldc * (g.c_bf16 ? 2 : 4);
      p.r = g.r ? g.r + (int64_t)m * g.ldr : nullptr;
      p.M = g.M - m < rows ? g.M - m : rows;
      const int rc = gemm_fp8(p, fa, fb, ws, ws_bytes, st);
      if (rc) return rc;
    }
    return ALS_OK;
  }
  g.nsplit = 1; g.split_stride = 0;
  return run_fp8(g, fa, fb, ws, ws_bytes, st);
}

}  // namespace

}  // namespace als

using namespace als;

extern "C" size_t als_k_gemm_fp8_ws_bytes(int M, int N, int K) {
  if (M <= 0 || N <= 0 || K <= 0 || M > 1 << 30 || N > 1 << 20 || K > 1 << 30) return 0;
  return std::max(fp8_ws_bytes(M, N, fp8_plan(M, N, K, false, SIZE_MAX).nsplit), fp8_ws_bytes(M, N, fp8_plan(M, N, K, true, SIZE_MAX).nsplit));
}

extern "C" int als_k_set_gemm_fp8(int tile, int shares) {
  if (tile != 0 && tile != 64 && tile != 128 && tile != 256) return set_error(ALS_ERR_INVALID, "als_k_set_gemm_fp8: tile must be 0, 64, 128 or 256");
  if (shares < (tile ? 1 : 0) || shares > 64) return set_error(ALS_ERR_INVALID, "als_k_set_gemm_fp8: bad number of shares");
  g_fp8_shares = shares;
  g_fp8_tile = tile;
  return ALS_OK;
}

extern "C" int als_k_gemm_fp8_route(int M, int N, int K, int out_dtype, size_t ws_bytes, int* tile_out, int* shares_out) {
  if (M <= 0 || N <= 0 || K < 0 || M > 1 << 30 || N > 1 << 20 || K > 1 << 30 || !tile_out || !shares_out) return set_error(ALS_ERR_INVALID, "als_k_gemm_fp8_route: null argument or bad size");
  const Fp8Plan p = fp8_plan(M, N, K, out_dtype == ALS_DTYPE_F32, ws_bytes);
  *tile_out = p.tile; *shares_out = p.nsplit;
  return ALS_OK;
}

extern "C" int als_k_gemm_fp8(const als_fp8* A, const als_fp8* B, void* C, int64_t ldc, int out_dtype, const float* R, int64_t ldr, int M, int N,
                              int K, void* ws_dev, size_t ws_bytes, void* stream) {
  if (!A || !B) return set_error(ALS_ERR_INVALID, "als_k_gemm_fp8: null argument");
  if (M < 0 || N < 0 || K < 0 || M > 1 << 30 || N > 1 << 20 || K > 1 << 30) return set_error(ALS_ERR_INVALID, "als_k_gemm_fp8: M and K must be in 0..2^30, N in 0..2^20");
  int rc = check_dtype(out_dtype, "als_k_gemm_fp8");
  if (!rc) rc = check_fp8(A, M, K, "als_k_gemm_fp8, A");
  if (!rc) rc = check_fp8(B, N, K, "als_k_gemm_fp8, B");
  if (rc) return rc;
  if (M == 0 || N == 0) return ALS_OK;
  // a tile's rows are addressed with 32 bits
  if (A->ld > 1 << 23 || B->ld > 1 << 23 || A->ld_scale > 1 << 23 || B->ld_scale > 1 << 23) return set_error(ALS_ERR_INVALID, "als_k_gemm_fp8: ld beyond 2^23");
  if (!C || ldc < N || (uintptr_t)C % (out_dtype == ALS_DTYPE_BF16 ? 2 : 4)) return set_error(ALS_ERR_INVALID, "als_k_gemm_fp8: C is null or not aligned to its type, or ldc below N");
  if (ldc > 1 << 26 || ldr > 1 << 26) return set_error(ALS_ERR_INVALID, "als_k_gemm_fp8: ldc or ldr beyond 2^26");
  if (R && (ldr < N || (uintptr_t)R % 4)) return set_error(ALS_ERR_INVALID, "als_k_gemm_fp8: R is not aligned to its type, or ldr below N");
  if ((const void*)R == C && (out_dtype != ALS_DTYPE_F32 || ldr != ldc)) return set_error(ALS_ERR_INVALID, "als_k_gemm_fp8: R may be C in fp32 with the same ld only");
  if (ws_dev && (uintptr_t)ws_dev % 256) return set_error(ALS_ERR_INVALID, "als_k_gemm_fp8: workspace must be 256-byte aligned");
  Fp8Args g;
  g.a = (const uint8_t*)A->data; g.b = (const uint8_t*)B->data; g.sa = A->scale; g.sb = B->scale;
  g.lda = (int)A->ld; g.ldb = (int)B->ld; g.lda_s = (int)A->ld_scale; g.ldb_s = (int)B->ld_scale;
  g.sha = A->block_rows == 128 ? 7 : 0; g.shb = B->block_rows == 128 ? 7 : 0;
  g.M = M; g.N = N; g.K = K; g.tiles_m = g.tiles_n = 0; g.div_tiles = g.div_span = 0;
  g.c = C; g.ldc = ldc; g.c_bf16 = out_dtype == ALS_DTYPE_BF16; g.c_size = g.c_bf16 ? 2 : 4; g.r = R; g.ldr = ldr;
  return gemm_fp8(g, A->format, B->format, ws_dev, ws_dev ? ws_bytes : 0, (hipStream_t)stream);
}
