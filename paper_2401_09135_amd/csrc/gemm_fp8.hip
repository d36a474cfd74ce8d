// Products of matrices in 8 bits with a power-of-two scale for each block of 128 (als_k_gemm_fp8): C = A B^T (+ R), A [M, K], B [N, K].
//
// bf16 results: v_mfma_scale_f32_32x32x64_f8f6f4 takes a scale byte for each row and 32 elements of K of either operand and adds to fp32, so the
// scales cost no vector instruction.  It cuts each product to 2^-13 of the largest of the 8 neighbours in K that it adds first (measured: 2^16 + 4 is
// 2^16 where the two are among the same 8, and exact elsewhere), so that sums of random signs are off by 1.5e-5 of their size: far below a rounding to bf16
// (up to 2^-8), and more than fp32 results may be off.
// fp32 results: elements are turned into bf16 with their scale on the way to the matrix instruction (exactly: 4 bits and 8 of exponent), whose products are
// exact and whose sums are fp32, at half the rate.  Elements under 2^-126 have fewer bits there.
// A lane holds row lane & 31 and 32 bytes of K; which 32 of the 64 a half of the wavefront holds does not matter, as both operands are dealt alike and a
// block of 128 has one scale.  Products are formed transposed (B's rows are the result's rows), so that a lane has 4 consecutive columns of C.
#include "fp8.h"

namespace als {

namespace {

typedef int i32x8 __attribute__((ext_vector_type(8)));

struct Fp8Args {
  const uint8_t* a; const uint8_t* b; const uint8_t* sa; const uint8_t* sb;
  int64_t lda, ldb, lda_s, ldb_s;
  int sha, shb;            // log2 of block_rows
  int M, N, K, tiles_n;
  void* c; int64_t ldc; int c_bf16;
  const float* r; int64_t ldr;
};

// 16 bytes of row `row` from k on; bytes from K on are 0
__device__ __forceinline__ u32x4 load_k16(const uint8_t* p, int k, int K) {
  u32x4 v = {0, 0, 0, 0};
  if (k < K) v = *reinterpret_cast<const u32x4*>(p + k);
  const int n = K - k;
  if (n < 16) {
#pragma unroll
    for (int i = 0; i < 4; i++) {
      const int left = n - 4 * i;
      if (left < 4) v[i] = left > 0 ? v[i] & ((1u << (8 * left)) - 1) : 0u;
    }
  }
  return v;
}

// the elements of four bytes times 2^e as bf16
template <int F>
__device__ __forceinline__ void widen4(int bytes, float scale, bf16x8& out, int at) {
  typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
  bf16x2 lo, hi;
  if (F == ALS_FP8_E4M3) {
    lo = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(bytes, scale, false);
    hi = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(bytes, scale, true);
  } else {
    lo = __builtin_amdgcn_cvt_scalef32_pk_bf16_bf8(bytes, scale, false);
    hi = __builtin_amdgcn_cvt_scalef32_pk_bf16_bf8(bytes, scale, true);
  }
  out[at] = lo[0]; out[at + 1] = lo[1]; out[at + 2] = hi[0]; out[at + 3] = hi[1];
}
template <int F>
__device__ __forceinline__ bf16x8 widen8(int a, int b, int scale_byte) {
  // 2^-127 is no normal fp32 number, but the conversion takes the exponent alone
  const float s = __builtin_bit_cast(float, scale_byte << 23);
  bf16x8 out;
  widen4<F>(a, s, out, 0);
  widen4<F>(b, s, out, 4);
  return out;
}

template <int FA, int FB, bool WIDE>
__global__ __launch_bounds__(256) void gemm_fp8_kernel(Fp8Args g) {
  __shared__ __attribute__((aligned(16))) uint8_t As[64 * 128], Bs[64 * 128];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, hf = lane >> 5, wm = wave >> 1, wn = wave & 1;
  const int m0 = blockIdx.x / g.tiles_n * 64, n0 = blockIdx.x % g.tiles_n * 64;
  auto row_of = [](int r, int n) { return r < n ? r : n - 1; };   // rows beyond the matrix are its last one and not stored
  const int fx = hf ^ (((lane & 31) >> 1) & 7);
  const int am = row_of(m0 + wm * 32 + (lane & 31), g.M), bn = row_of(n0 + wn * 32 + (lane & 31), g.N);
  const uint8_t* sa = g.sa + (int64_t)(am >> g.sha) * g.lda_s;
  const uint8_t* sb = g.sb + (int64_t)(bn >> g.shb) * g.ldb_s;
  f32x16 acc;
#pragma unroll
  for (int i = 0; i < 16; i++) acc[i] = 0.0f;
  for (int k0 = 0, kb = 0; k0 < g.K; k0 += 128, kb++) {
    __syncthreads();
#pragma unroll
    for (int i = 0; i < 2; i++) {
      const int R = i * 32 + (threadIdx.x >> 3), c = threadIdx.x & 7, pos = R * 128 + (c ^ ((R >> 1) & 7)) * 16;
      *reinterpret_cast<u32x4*>(As + pos) = load_k16(g.a + (int64_t)row_of(m0 + R, g.M) * g.lda, k0 + 16 * c, g.K);
      *reinterpret_cast<u32x4*>(Bs + pos) = load_k16(g.b + (int64_t)row_of(n0 + R, g.N) * g.ldb, k0 + 16 * c, g.K);
    }
    const int xa = sa[kb], xb = sb[kb];
    __syncthreads();
#pragma unroll
    for (int s = 0; s < 2; s++) {
      i32x8 af, bf;
#pragma unroll
      for (int h = 0; h < 2; h++) {
        const int pos = (((2 * s + h) * 2) ^ fx) * 16;
        const u32x4 x = *reinterpret_cast<const u32x4*>(As + (wm * 32 + (lane & 31)) * 128 + pos);
        const u32x4 y = *reinterpret_cast<const u32x4*>(Bs + (wn * 32 + (lane & 31)) * 128 + pos);
#pragma unroll
        for (int i = 0; i < 4; i++) { af[4 * h + i] = (int)x[i]; bf[4 * h + i] = (int)y[i]; }
      }
      if constexpr (WIDE) {
#pragma unroll
        for (int j = 0; j < 8; j += 2)
          acc = __builtin_amdgcn_mfma_f32_32x32x16_bf16(widen8<FB>(bf[j], bf[j + 1], xb), widen8<FA>(af[j], af[j + 1], xa), acc, 0, 0, 0);
      } else {
        acc = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(bf, af, acc, FB, FA, 0, xb, 0, xa);
      }
    }
  }
  const int m = m0 + wm * 32 + (lane & 31);
  if (m >= g.M) return;
#pragma unroll
  for (int i = 0; i < 16; i++) {
    const int n = n0 + wn * 32 + 8 * (i >> 2) + 4 * hf + (i & 3);
    if (n >= g.N) continue;
    const float v = g.r ? acc[i] + g.r[(int64_t)m * g.ldr + n] : acc[i];
    if (g.c_bf16) ((bf16*)g.c)[(int64_t)m * g.ldc + n] = (bf16)v;
    else ((float*)g.c)[(int64_t)m * g.ldc + n] = v;
  }
}

int gemm_fp8(Fp8Args g, int fa, int fb, hipStream_t st) {
  const int64_t tiles = gemm_tiles(g.M, g.N, 64, 64);
  if (tiles > 0x7fffffff) return set_error(ALS_ERR_INVALID, "als_k_gemm_fp8: product too large");
  g.tiles_n = (g.N + 63) / 64;
#define ALS_FP8_GEMM(FA, FB)                                                                                        \
  do {                                                                                                              \
    if (g.c_bf16) hipLaunchKernelGGL((gemm_fp8_kernel<FA, FB, false>), dim3((unsigned)tiles), dim3(256), 0, st, g); \
    else hipLaunchKernelGGL((gemm_fp8_kernel<FA, FB, true>), dim3((unsigned)tiles), dim3(256), 0, st, g);           \
  } while (0)
  if (fa == ALS_FP8_E4M3) { if (fb == ALS_FP8_E4M3) ALS_FP8_GEMM(0, 0); else ALS_FP8_GEMM(0, 1); }
  else { if (fb == ALS_FP8_E4M3) ALS_FP8_GEMM(1, 0); else ALS_FP8_GEMM(1, 1); }
#undef ALS_FP8_GEMM
  ALS_CHECK_LAUNCH();
  return ALS_OK;
}

}  // namespace

}  // namespace als

using namespace als;

extern "C" size_t als_k_gemm_fp8_ws_bytes(int M, int N, int K) { return 0; }

extern "C" int als_k_gemm_fp8(const als_fp8* A, const als_fp8* B, void* C, int64_t ldc, int out_dtype, const float* R, int64_t ldr, int M, int N,
                              int K, void* ws_dev, size_t ws_bytes, void* stream) {
  if (!A || !B) return set_error(ALS_ERR_INVALID, "als_k_gemm_fp8: null argument");
  if (M < 0 || N < 0 || K < 0 || M > 1 << 30 || N > 1 << 30 || K > 1 << 30) return set_error(ALS_ERR_INVALID, "als_k_gemm_fp8: M, N, K must be in 0..2^30");
  int rc = check_dtype(out_dtype, "als_k_gemm_fp8");
  if (!rc) rc = check_fp8(A, M, K, "als_k_gemm_fp8, A");
  if (!rc) rc = check_fp8(B, N, K, "als_k_gemm_fp8, B");
  if (rc) return rc;
  if (M == 0 || N == 0) return ALS_OK;
  if (!C || ldc < N || (uintptr_t)C % (out_dtype == ALS_DTYPE_BF16 ? 2 : 4)) return set_error(ALS_ERR_INVALID, "als_k_gemm_fp8: C is null or not aligned to its type, or ldc below N");
  if (R && (ldr < N || (uintptr_t)R % 4)) return set_error(ALS_ERR_INVALID, "als_k_gemm_fp8: R is not aligned to its type, or ldr below N");
  if ((const void*)R == C && (out_dtype != ALS_DTYPE_F32 || ldr != ldc)) return set_error(ALS_ERR_INVALID, "als_k_gemm_fp8: R may be C in fp32 with the same ld only");
  if (ws_dev && (uintptr_t)ws_dev % 256) return set_error(ALS_ERR_INVALID, "als_k_gemm_fp8: workspace must be 256-byte aligned");
  Fp8Args g;
  g.a = (const uint8_t*)A->data; g.b = (const uint8_t*)B->data; g.sa = A->scale; g.sb = B->scale;
  g.lda = A->ld; g.ldb = B->ld; g.lda_s = A->ld_scale; g.ldb_s = B->ld_scale;
  g.sha = A->block_rows == 128 ? 7 : 0; g.shb = B->block_rows == 128 ? 7 : 0;
  g.M = M; g.N = N; g.K = K; g.tiles_n = 0;
  g.c = C; g.ldc = ldc; g.c_bf16 = out_dtype == ALS_DTYPE_BF16; g.r = R; g.ldr = ldr;
  return gemm_fp8(g, A->format, B->format, (hipStream_t)stream);
}
