// 8-bit matrices (als_fp8): scales and conversion on the device, checks on the host.
#pragma once
#include "common.h"

namespace als {

// Both formats' largest value is 1.75 * 2^t, t = 8 (e4m3) and 15 (e5m2).  amax = m 2^k with 1 <= m < 2 is at most that value times 2^e from
// e = k - t on if m <= 1.75, from k - t + 1 on else: the scale's byte e + 127 comes from the bits of amax alone.  0 is a block without finite magnitudes.
__device__ __forceinline__ int fp8_scale_byte(float amax, int format) {
  const unsigned u = __builtin_bit_cast(unsigned, amax);
  const int b = (int)(u >> 23) - (format == ALS_FP8_E4M3 ? 8 : 15) + ((u & 0x7fffff) > 0x600000);
  return u == 0 ? 127 : (b < 0 ? 0 : b);
}
// 1 / the scale: 2^(127 - s), s from 0 to 247 (e4m3's largest is 254 - 8 + 1), always a normal number
__device__ __forceinline__ float fp8_inv_scale(int byte) { return __builtin_bit_cast(float, (unsigned)(254 - byte) << 23); }
// |v| as the block's largest magnitude sees it
__device__ __forceinline__ float fp8_magnitude(float v) {
  const float a = fabsf(v);
  return a < __builtin_inff() ? a : 0.0f;   // false for NaN too
}
// four values, already divided by the scale, to four bytes
__device__ __forceinline__ unsigned fp8_pack4(float a, float b, float c, float d, int format) {
  int v;
  if (format == ALS_FP8_E4M3) {
    v = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
    v = __builtin_amdgcn_cvt_pk_fp8_f32(c, d, v, true);
  } else {
    v = __builtin_amdgcn_cvt_pk_bf8_f32(a, b, 0, false);
    v = __builtin_amdgcn_cvt_pk_bf8_f32(c, d, v, true);
  }
  return (unsigned)v;
}

// Eight consecutive elements from p; elements from n on are 0 and not read.  VEC: p is 16-byte aligned.
template <bool VEC>
__device__ __forceinline__ void load8(const float* p, int n, float (&v)[8]) {
  if (VEC && n >= 8) {
    const f32x4 a = reinterpret_cast<const f32x4*>(p)[0], b = reinterpret_cast<const f32x4*>(p)[1];
#pragma unroll
    for (int i = 0; i < 4; i++) { v[i] = a[i]; v[4 + i] = b[i]; }
  } else {
#pragma unroll
    for (int i = 0; i < 8; i++) v[i] = i < n ? p[i] : 0.0f;
  }
}
template <bool VEC>
__device__ __forceinline__ void load8(const bf16* p, int n, float (&v)[8]) {
  if (VEC && n >= 8) {
    const bf16x8 a = *reinterpret_cast<const bf16x8*>(p);
#pragma unroll
    for (int i = 0; i < 8; i++) v[i] = (float)a[i];
  } else {
#pragma unroll
    for (int i = 0; i < 8; i++) v[i] = i < n ? (float)p[i] : 0.0f;
  }
}
template <bool VEC>
__device__ __forceinline__ void store8(float* p, int n, const float (&v)[8]) {
  if (VEC && n >= 8) {
    reinterpret_cast<f32x4*>(p)[0] = (f32x4){v[0], v[1], v[2], v[3]};
    reinterpret_cast<f32x4*>(p)[1] = (f32x4){v[4], v[5], v[6], v[7]};
  } else {
#pragma unroll
    for (int i = 0; i < 8; i++)
      if (i < n) p[i] = v[i];
  }
}
template <bool VEC>
__device__ __forceinline__ void store8(bf16* p, int n, const float (&v)[8]) {
  if (VEC && n >= 8) {
    bf16x8 a;
#pragma unroll
    for (int i = 0; i < 8; i++) a[i] = (bf16)v[i];
    *reinterpret_cast<bf16x8*>(p) = a;
  } else {
#pragma unroll
    for (int i = 0; i < 8; i++)
      if (i < n) p[i] = (bf16)v[i];
  }
}
// eight bytes to p, which is 8-byte aligned; only the first n of them
__device__ __forceinline__ void store8_bytes(uint8_t* p, int n, unsigned lo, unsigned hi) {
  if (n >= 8) {
    *reinterpret_cast<uint2*>(p) = make_uint2(lo, hi);
  } else {
#pragma unroll
    for (int i = 0; i < 8; i++)
      if (i < n) p[i] = (uint8_t)((i < 4 ? lo : hi) >> (8 * (i & 3)));
  }
}

inline int64_t fp8_blocks(int64_t cols) { return (cols + 127) / 128; }
// what als.h asks of a matrix in 8 bits; `what` names it in the error
inline int check_fp8(const als_fp8* f, int64_t rows, int64_t cols, const char* what) {
  if (f->format != ALS_FP8_E4M3 && f->format != ALS_FP8_E5M2) return set_error(ALS_ERR_INVALID, "%s: unknown 8-bit format %d", what, f->format);
  if (f->block_rows != 1 && f->block_rows != 128) return set_error(ALS_ERR_INVALID, "%s: block_rows must be 1 or 128", what);
  if (rows == 0 || cols == 0) return ALS_OK;
  if (!f->data || !f->scale) return set_error(ALS_ERR_INVALID, "%s: null data or scale", what);
  if (f->ld < cols || f->ld % 16 || f->ld_scale < fp8_blocks(cols) || f->ld_scale % 4)
    return set_error(ALS_ERR_INVALID, "%s: ld must be a multiple of 16 and at least %lld, ld_scale of 4 and at least %lld", what, (long long)cols, (long long)fp8_blocks(cols));
  if ((uintptr_t)f->data % 16 || (uintptr_t)f->scale % 4) return set_error(ALS_ERR_INVALID, "%s: data must be 16-byte aligned, scale 4-byte", what);
  return ALS_OK;
}
inline int check_dtype(int dtype, const char* what) {
  if (dtype != ALS_DTYPE_F32 && dtype != ALS_DTYPE_BF16) return set_error(ALS_ERR_INVALID, "%s: unknown dtype %d", what, dtype);
  return ALS_OK;
}

}  // namespace als
