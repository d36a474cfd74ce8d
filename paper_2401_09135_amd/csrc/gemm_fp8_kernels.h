// Products of matrices in 8 bits with a power-of-two scale for each block of 128 (als_k_gemm_fp8): C = A B^T (+ R), A [M, K], B [N, K].
//
// bf16 results: v_mfma_scale_f32_32x32x64_f8f6f4 takes a scale byte for each row and 32 elements of K of either operand and adds to fp32, so the
// scales cost no vector instruction.  It cuts each product to 2^-13 of the largest of the 8 neighbours in K that it adds first (measured: 2^16 + 4 is
// 2^16 where the two are among the same 8, and exact elsewhere), towards zero: nothing is lost where these are within 2^6 of one another, as products of two e4m3 values have 6
// bits behind the point, and less than 7 2^-13 of the largest at worst.  Sums of K = 8192 are off by 1.5e-5 (normal numbers, random signs) to 7e-5 (outliers, magnitudes over five decades) of their size, and
// those of one sign too small by 3e-6 and 1e-4: far below a rounding to bf16 (up to 2^-8), of which 1 in 60 turns out otherwise, and more than fp32 results may be off.
// fp32 results: elements are turned into bf16 with their scale on the way to the matrix instruction (exactly: 4 bits and 8 of exponent), whose products are
// exact and whose sums are fp32, at half the rate.  Elements under 2^-126 have fewer bits there.
// A lane holds row lane & 31 and 32 bytes of K; which 32 of the 64 a half of the wavefront holds does not matter, as both operands are dealt alike and a
// block of 128 has one scale.  Products are formed transposed (B's rows are the result's rows), so that a lane has 4 consecutive columns of C.
#pragma once

#include "fp8.h"

namespace als {

struct Fp8Args {
  const uint8_t* a; const uint8_t* b; const uint8_t* sa; const uint8_t* sb;
  int lda, ldb, lda_s, ldb_s;
  int sha, shb;            // log2 of block_rows
  int M, N, K, tiles_m, tiles_n;
  int nsplit; int64_t split_stride;   // shares of K, and elements between their partial sums
  unsigned div_tiles, div_span;       // fp8_reciprocal of tiles_m tiles_n and of 8 tiles_m
  void* c; int64_t ldc; int c_bf16, c_size;   // c_size: bytes of what is written, 4 for partial sums
  const float* r; int64_t ldr;
};

// how the tiles' sums are made and left: bf16 or fp32 results, or partial sums (fp32) of bf16 results
enum Fp8Out { FP8_BF16, FP8_F32, FP8_PARTIAL };
template <int FA, int FB>
int gemm_fp8_launch(Fp8Args g, int tile, Fp8Out out, hipStream_t st);   // FA, FB: 0 is e4m3, 1 is e5m2; each pair is a source of its own

namespace {

typedef int i32x8 __attribute__((ext_vector_type(8)));

// n / d for n, d with n d < 2^32, by a multiplication: n (2^32 / d + e) / 2^32 with 0 < e <= 1 is less than 1 / d beyond n / d
inline unsigned fp8_reciprocal(unsigned d) { return d == 1 ? 0 : (unsigned)(((uint64_t)1 << 32) / d) + 1; }
__device__ __forceinline__ int fp8_divide(int n, unsigned reciprocal) { return reciprocal ? (int)__umulhi((unsigned)n, reciprocal) : n; }

// whether 16 bytes (four columns of bf16 where R is added) a lane can be written, and R read
__host__ __device__ inline bool fp8_aligned(const Fp8Args& g) {
  const uint64_t c = g.c_size == 2 ? ((uint64_t)(uintptr_t)g.c | (uint64_t)(g.ldc * 2)) : ((uint64_t)(uintptr_t)g.c | (uint64_t)(g.ldc * 4));
  return (c & 15) == 0 && (((uint64_t)(uintptr_t)g.r | (uint64_t)(g.r ? g.ldr * 4 : 0)) & 15) == 0;
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
// scale: 2^(s - 127) for a scale byte s, its bits being s << 23 (2^-127 is no normal fp32 number, but the conversion takes the exponent alone)
template <int F>
__device__ __forceinline__ bf16x8 widen8(int a, int b, int scale) {
  const float s = __builtin_bit_cast(float, scale);
  bf16x8 out;
  widen4<F>(a, s, out, 0);
  widen4<F>(b, s, out, 4);
  return out;
}

// ---- tiles of 256 x 256 ------------------------------------------------------------------------
// A K slice of 128 of a 256 x 256 tile is 64 KB of operands for as many matrix cycles (2048 at the 8-bit rate) as a slice of 64 of the bf16 kernels of
// gemm_pingpong.h, and the same form serves: one workgroup of 8 wavefronts a CU, in two groups of four that alternate between a MEMORY phase (fragments of one
// half of the slice from LDS into registers) and a COMPUTE phase (matrix instructions and nothing else), one phase apart, so that every matrix pipe has one
// wavefront at work while the other's reads and waits hide behind it.
//   group 0: M(kt, h) at barrier 4 kt + 2 h, C(kt, h) one later; group 1 all of it one later.
// Operands go straight to LDS, by group 0's wavefronts alone.  What a slice has to wait for is the latency of a load and then its bytes at about 40 a clock, so that two
// buffers of 64 KB, loaded in one piece, give 2400 clocks a slice (1890 TFLOP/s on an 8192-cube; 2900 without loads, 3250 with matrix instructions alone).
// All 160 KB of LDS are therefore a ring of five units of 32 KB, A_0 B_0 A_1 B_1 ..: while slice kt is read, B_kt+1 and A_kt+2 are under way, issued in this
// order, and only the first of them is awaited at the slice's end.  Unit u lies in slot u mod 5:
//   B_kt+1, issued in M(kt, 0), takes the slot of A_kt-1 and A_kt+2, in M(kt, 1), that of B_kt-1, whose last reading was group 1's M(kt - 1, 1), one barrier before M(kt, 0);
//   both of slice kt + 1 have landed before the barrier ahead of M(kt + 1, 0).
// Row R of a unit has 128 bytes, whose 16-byte piece c lies at piece c ^ ((R >> 1) & 7): the fragment reads are free of bank conflicts without padding.
// K that is no multiple of 128: the last slice's pieces behind it are loaded from its last piece and zeroed in LDS by the wavefront that loaded them.
__device__ __forceinline__ int fp8_uniform(int v) { return __builtin_amdgcn_readfirstlane(v); }

// 16 bytes of a row's piece `piece` (of 8) of the slice; left: bytes of the row that the slice holds (128 but for the last).  In LDS: bytes from `left` on to 0.
__device__ __forceinline__ void zero_behind(char* row, int swizzle, int left) {
  for (int c = left >> 4; c < 8; c++) {
    u32x4* p = reinterpret_cast<u32x4*>(row + (c ^ swizzle) * 16);
    u32x4 v = {0, 0, 0, 0};
    const int n = left - 16 * c;   // bytes of this piece that count
    if (n > 0) {
      v = *p;
#pragma unroll
      for (int i = 0; i < 4; i++) {
        const int l = n - 4 * i;
        if (l < 4) v[i] = l > 0 ? v[i] & ((1u << (8 * l)) - 1) : 0u;
      }
    }
    *p = v;
  }
}

// One wavefront's TM x 32 rows and TN x 32 columns of C from its accumulators, 32 rows at a time through 4 KB of LDS, so that a store instruction covers whole
// segments of rows: bf16 results are rounded first and go 64 columns at a time, others 32.  Row r of the staging has 128 bytes, its 16-byte piece c
// at piece c ^ (r & 7).  LDS serves a wavefront's instructions in their order, so nothing waits between writing, reading and writing again; the fences
// keep the compiler to that order.  16 bytes a lane where C (and R) are aligned for it and all rows and columns exist, else an element a lane.
// R is read a block of 32 x 32 ahead of the stores: a load behind a store is waited for with the store.
constexpr int F8_STAGING = 32 * 128;
__device__ __forceinline__ void fp8_order() { asm volatile("" ::: "memory"); }

// How the kernel's results are written: bit 0: R is added, bit 1: C or R is not aligned for 16 bytes a lane, bit 3: where R is added, parts of 128 x 64 may end outside of the matrix.  Kernels of
// their own, as one that could do all keeps too few registers for the products; tiles of 128 and 64 ask at run time (EPI_ASK).
// One kernel for all with R takes 4 % longer for 16384 x 896 x 3584 fp32, 6 % for 16384 x 3584 x 896 (now 169 us) and 11 % for 14638 x 6376 x 563 (362 us; 8 rows of R at once at the
// edges); one for all of bf16 36 % for 16384 x 896 x 3584 with R (66 us).  The kernels of the edges keep 25 to 77 registers in scratch memory, the others with fp32 results 5: R at a
// ragged edge is what costs most beside its floor (362 us, 224 without R).
constexpr int EPI_ADD = 1, EPI_ANY = 2, EPI_ASK = 4, EPI_EDGE = 8;
template <int HOW, int TM, int TN, typename TO>
__device__ __forceinline__ void fp8_epilogue(const f32x16 (&acc)[TM][TN], char* stg, const Fp8Args& g, TO* C, const float* R, int row0, int col0, int lane) {
  asm volatile("" : "+v"(lane));   // nothing of this is kept in registers from tile to tile
  const int r8 = lane >> 3, c8 = lane & 7, wr = lane & 31, hf = lane >> 5, ldc = (int)g.ldc, ldr = (int)g.ldr;
  const bool add_r = HOW & EPI_ASK ? R != nullptr : (HOW & EPI_ADD) != 0;
  C += (int64_t)row0 * g.ldc + col0;
  if (add_r) R += (int64_t)row0 * g.ldr + col0;
  const int rows = g.M - row0, cols = g.N - col0;   // that are left
  const bool full = (HOW & (EPI_ADD | EPI_EDGE)) == EPI_ADD || (rows >= TM * 32 && cols >= TN * 32);
  const bool vec = full && (HOW & EPI_ASK ? fp8_aligned(g) : !(HOW & EPI_ANY));
  if (sizeof(TO) == 2 && TN == 2 && !add_r) {
    const unsigned off = (unsigned)((r8 * ldc + c8 * 8) * (int)sizeof(TO));
#pragma unroll
    for (int i = 0; i < TM; i++) {
#pragma unroll
      for (int j = 0; j < TN; j++)
#pragma unroll
        for (int q = 0; q < 4; q++) {
          bf16x4 v;
#pragma unroll
          for (int e = 0; e < 4; e++) v[e] = (bf16)acc[i][j][4 * q + e];
          *reinterpret_cast<bf16x4*>(stg + wr * 128 + (((4 * j + q) ^ (wr & 7)) * 16) + hf * 8) = v;
        }
      fp8_order();
      TO* o = C + (int64_t)(i * 32) * g.ldc;
      if (vec) {
        u32x4 v[4];
#pragma unroll
        for (int p = 0; p < 4; p++) v[p] = *reinterpret_cast<const u32x4*>(stg + (p * 8 + r8) * 128 + (c8 ^ r8) * 16);
#pragma unroll
        for (int p = 0; p < 4; p++, o += 8 * g.ldc) __builtin_nontemporal_store(v[p], reinterpret_cast<u32x4*>(reinterpret_cast<char*>(o) + off));
      } else {
        const int n = rows - i * 32 < 32 ? rows - i * 32 : 32;
#pragma unroll 4
        for (int r = 0; r < n; r++, o += g.ldc) {
          const TO v = *reinterpret_cast<const TO*>(stg + r * 128 + ((lane >> 3) ^ (r & 7)) * 16 + c8 * 2);
          if (lane < cols) o[lane] = v;
        }
      }
      fp8_order();
    }
    return;
  }
  // a lane's place in the first rows of a block: four columns of row r8, or column wr of row hf
  const unsigned off = (unsigned)((vec ? r8 * ldc + c8 * 4 : hf * ldc + wr) * (int)sizeof(TO)), roff = (unsigned)((vec ? r8 * ldr + c8 * 4 : hf * ldr + wr) * 4);
  float add[2][16];   // of this block of 32 x 32 and of the next one (further ahead the registers do not reach)
  auto load_add = [&](int s) {
    const char* x = reinterpret_cast<const char*>(R + (int64_t)(s / TN * 32) * g.ldr + s % TN * 32);
    if (vec) {
#pragma unroll
      for (int p = 0; p < 4; p++, x += 32 * g.ldr) {
        const f32x4 v = *reinterpret_cast<const f32x4*>(x + roff);
#pragma unroll
        for (int e = 0; e < 4; e++) add[s & 1][4 * p + e] = v[e];
      }
    } else {
#pragma unroll
      for (int p = 0; p < 16; p++, x += 8 * g.ldr) add[s & 1][p] = *reinterpret_cast<const float*>(x + roff);
    }
  };
  if (add_r && full) load_add(0);
#pragma unroll
  for (int i = 0; i < TM; i++)
#pragma unroll
    for (int j = 0; j < TN; j++) {
      const int s = i * TN + j;
#pragma unroll
      for (int q = 0; q < 4; q++)
        *reinterpret_cast<f32x4*>(stg + wr * 128 + ((2 * q + hf) ^ (wr & 7)) * 16) =
            (f32x4){acc[i][j][4 * q], acc[i][j][4 * q + 1], acc[i][j][4 * q + 2], acc[i][j][4 * q + 3]};
      fp8_order();
      if (add_r && full && s + 1 < TM * TN) load_add(s + 1);
      TO* o = C + (int64_t)(i * 32) * g.ldc + j * 32;
      if (vec) {
        f32x4 v[4];
#pragma unroll
        for (int p = 0; p < 4; p++) v[p] = *reinterpret_cast<const f32x4*>(stg + (p * 8 + r8) * 128 + (c8 ^ r8) * 16);
#pragma unroll
        for (int p = 0; p < 4; p++, o += 8 * g.ldc) {
          if (add_r)
#pragma unroll
            for (int e = 0; e < 4; e++) v[p][e] += add[s & 1][4 * p + e];
          char* x = reinterpret_cast<char*>(o) + off;
          if constexpr (sizeof(TO) == 4) {
            __builtin_nontemporal_store(v[p], reinterpret_cast<f32x4*>(x));
          } else {
            bf16x4 y;
#pragma unroll
            for (int e = 0; e < 4; e++) y[e] = (bf16)v[p][e];
            __builtin_nontemporal_store(y, reinterpret_cast<bf16x4*>(x));
          }
        }
      } else if (full) {
#pragma unroll
        for (int p = 0; p < 16; p++, o += 2 * g.ldc) {
          const int r = 2 * p + hf;
          float v = *reinterpret_cast<const float*>(stg + r * 128 + ((wr >> 2) ^ (r & 7)) * 16 + (wr & 3) * 4);
          if (add_r) v += add[s & 1][p];
          *reinterpret_cast<TO*>(reinterpret_cast<char*>(o) + off) = (TO)v;
        }
      } else {
        const int n = rows - i * 32 < 32 ? rows - i * 32 : 32, m = cols - j * 32;   // rows and columns of the block
        if (m > 0) {
          constexpr int U = 8;   // rows of a half of the wavefront under way at once; those behind the last are the last, so that their loads need no branch
          const float* from = add_r ? R + (int64_t)(i * 32) * g.ldr + j * 32 + (wr < m ? wr : m - 1) : nullptr;
#pragma unroll 1
          for (int r0 = hf; r0 < n + hf; r0 += 2 * U) {
            float x[U];
#pragma unroll
            for (int u = 0; u < U; u++) x[u] = add_r ? from[(int64_t)(r0 + 2 * u < n ? r0 + 2 * u : n - 1) * g.ldr] : 0.0f;
#pragma unroll
            for (int u = 0; u < U; u++) {
              const int r = r0 + 2 * u;
              const float v = *reinterpret_cast<const float*>(stg + (r & 31) * 128 + ((wr >> 2) ^ (r & 7)) * 16 + (wr & 3) * 4);
              if (r < n && wr < m) o[(int64_t)r * g.ldc + wr] = (TO)(add_r ? v + x[u] : v);
            }
          }
        }
      }
      fp8_order();
    }
}

constexpr int F8_UNIT = 32 * 1024;   // bytes of a slice of A or B

template <int N>
__device__ __forceinline__ void wait_loads() {   // all but the N youngest loads of this wavefront have landed
  asm volatile("s_waitcnt vmcnt(%0)" ::"n"(N) : "memory");
}

// memory from p on, for loads with 32-bit offsets (and scalar ones) that stay inside it by themselves
__device__ __forceinline__ __amdgpu_buffer_rsrc_t fp8_buffer(const uint8_t* p) {
  const uint64_t u = (uint64_t)(uintptr_t)p;
  const uint64_t s = (uint64_t)(unsigned)fp8_uniform((int)(unsigned)u) | (uint64_t)(unsigned)fp8_uniform((int)(unsigned)(u >> 32)) << 32;
  return __builtin_amdgcn_make_buffer_rsrc((void*)(uintptr_t)s, 0, -1, 0x00027000);
}

// Tile `id` of the launch: its place in C, its K slices, and where its share's partial sums begin.  Workgroups are dealt to the XCDs in turn: each XCD gets
// a contiguous run of tiles, numbered down column blocks 8 wide, share after share.
struct Fp8Tile { int m0, n0, slice0, nk, z; };
__device__ __forceinline__ Fp8Tile fp8_tile(const Fp8Args& g, int id) {
  const int ntiles = g.tiles_m * g.tiles_n, total = ntiles * g.nsplit, base = total / 8, rem = total % 8, x = id & 7;
  const int p = x * base + (x < rem ? x : rem) + (id >> 3);
  const int z = fp8_divide(p, g.div_tiles), tile = p - z * ntiles;
  const int b = fp8_divide(tile, g.div_span), r = tile - b * 8 * g.tiles_m;
  const int width = g.tiles_n - b * 8 < 8 ? g.tiles_n - b * 8 : 8, row = width == 8 ? r >> 3 : r / width;
  const int nkt = (g.K + 127) / 128, q = g.nsplit == 1 ? nkt : nkt / g.nsplit, e = nkt - q * g.nsplit;
  Fp8Tile t;
  t.m0 = row * 256;
  t.n0 = (b * 8 + r - row * width) * 256;
  t.nk = q + (z < e ? 1 : 0);
  t.slice0 = z * q + (z < e ? z : e);
  t.z = z;
  return t;
}

template <int FA, int FB, bool WIDE, typename TO, int HOW>
__global__ __launch_bounds__(512, 1) void gemm_fp8_pp_kernel(Fp8Args g, int tiles) {
  __shared__ __attribute__((aligned(1024))) char smem[5 * F8_UNIT];
  constexpr int TM = 4, TN = 2;
  const int tid = threadIdx.x, lane = tid & 63, wave = fp8_uniform(tid >> 6), grp = wave >> 2, sub = wave & 3, hf = lane >> 5;
  const int nkt = (g.K + 127) / 128, tail = g.K & 127;   // slices of K, and the bytes that the last one has if it is not whole
  const unsigned lds0 = (unsigned)(uintptr_t)(__attribute__((address_space(3))) char*)(smem);

  // ---- loads: group 0's wavefronts issue the units of all tiles of the workgroup in one stream, A then B of a slice.  Wavefront w has rows 64 w .. + 63 of a
  // unit, 8 an instruction: lane l row l >> 3 of them, piece (l & 7) ^ ((R >> 1) & 7), which alternates between two.  Rows beyond the matrix are its last one.
  int p_id = blockIdx.x, p_kt = 0, p_slot = 0;   // of the next unit: its tile, its slice there, its slot
  Fp8Tile p_tile = fp8_tile(g, p_id);
  const int lrow = 64 * sub + (lane >> 3), piece0 = ((lane & 7) ^ (lane >> 4)) * 16, piece1 = piece0 ^ 64;
  auto issue_unit = [&](const uint8_t* op, unsigned ld, int rows) {   // op: the tile's first row; rows: of the matrix from there on
    const int kb = p_tile.slice0 + p_kt;
    const uint8_t* p = op + (int64_t)kb * 128;
    unsigned dst = lds0 + p_slot * F8_UNIT + 64 * sub * 128;
    int pc[2] = {piece0, piece1};
    if (tail && kb == nkt - 1) {
      const int last_piece = (tail - 1) & ~15;
      pc[0] = pc[0] < last_piece ? pc[0] : last_piece;
      pc[1] = pc[1] < last_piece ? pc[1] : last_piece;
    }
    if (rows >= 256) {
      const unsigned off = (unsigned)lrow * ld;
#pragma unroll
      for (int i = 0; i < 8; i++, p += 8 * ld, dst += 1024) global_to_lds_16(p, off + pc[i & 1], dst);
    } else {
#pragma unroll
      for (int i = 0; i < 8; i++, dst += 1024) {
        const int R = lrow + 8 * i;
        global_to_lds_16(p, (unsigned)(R < rows ? R : rows - 1) * ld + pc[i & 1], dst);
      }
    }
    p_slot = p_slot < 4 ? p_slot + 1 : 0;
  };
  // whether there was one
  auto issue_a = [&]() {
    if (p_id >= tiles) return false;
    issue_unit(g.a + (int64_t)p_tile.m0 * g.lda, g.lda, g.M - p_tile.m0);
    return true;
  };
  auto issue_b = [&]() {
    if (p_id >= tiles) return;
    issue_unit(g.b + (int64_t)p_tile.n0 * g.ldb, g.ldb, g.N - p_tile.n0);
    if (++p_kt == p_tile.nk) {
      p_kt = 0;
      p_id += gridDim.x;
      if (p_id < tiles) p_tile = fp8_tile(g, p_id);
    }
  };
  // slice kb in these slots, whose loads by this wavefront have landed, if K ends inside it: lane l has row l of the 64 of A and of B
  auto end_of_k = [&](int kb, int slot_a, int slot_b) {
    if (!tail || kb != nkt - 1) return;
    const int R = 64 * sub + lane;
    zero_behind(smem + slot_a * F8_UNIT + R * 128, (R >> 1) & 7, tail);
    zero_behind(smem + slot_b * F8_UNIT + R * 128, (R >> 1) & 7, tail);
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
  };

  // ---- the 128 x 64 of a wavefront: group g has columns 128 g .. + 127 of a tile, or rows if its lower half lies outside: the dead half is then one group
  auto row_half = [&](const Fp8Tile& t) { return t.m0 + 128 >= g.M && t.n0 + 128 < g.N ? grp : sub >> 1; };
  auto col_quarter = [&](const Fp8Tile& t) { return t.m0 + 128 >= g.M && t.n0 + 128 < g.N ? sub : grp * 2 + (sub & 1); };

  // ---- scale bytes: a lane's rows of A and of B, four slices a word.  The next four's, or the next tile's first, are loaded when the present ones' begin.  The
  // compiler waits for them with all loads under way, so the words change hands at a slice's end, with the next A not yet issued.
  unsigned sa[TM], sb[TN], na[TM], nb[TN];
  auto load_scales = [&](const Fp8Tile& t, int kb) {
    const __amdgpu_buffer_rsrc_t Sa = fp8_buffer(g.sa + (int64_t)(t.m0 >> g.sha) * g.lda_s), Sb = fp8_buffer(g.sb + (int64_t)(t.n0 >> g.shb) * g.ldb_s);
    const int ra = row_half(t) * 128 + (lane & 31), rb = col_quarter(t) * 64 + (lane & 31), la = g.M - 1 - t.m0, lb = g.N - 1 - t.n0;
#pragma unroll
    for (int i = 0; i < TM; i++) {
      const int r = ra + 32 * i < la ? ra + 32 * i : la;
      na[i] = __builtin_amdgcn_raw_buffer_load_b32(Sa, (unsigned)((r >> g.sha) * g.lda_s), kb & ~3, 0);
    }
#pragma unroll
    for (int j = 0; j < TN; j++) {
      const int r = rb + 32 * j < lb ? rb + 32 * j : lb;
      nb[j] = __builtin_amdgcn_raw_buffer_load_b32(Sb, (unsigned)((r >> g.shb) * g.ldb_s), kb & ~3, 0);
    }
  };
  auto take_scales = [&]() {   // the empty statements are uses: the wait is here, and not in every slice
#pragma unroll
    for (int i = 0; i < TM; i++) {
      sa[i] = na[i];
      asm volatile("" : "+v"(sa[i]));
    }
#pragma unroll
    for (int j = 0; j < TN; j++) {
      sb[j] = nb[j];
      asm volatile("" : "+v"(sb[j]));
    }
  };
  int xa[TM], xb[TN];   // a slice's (WIDE: as the bits of fp32)
  auto slice_scales = [&](int kb) {
    const int sh = 8 * (kb & 3);
#pragma unroll
    for (int i = 0; i < TM; i++) xa[i] = (int)((sa[i] >> sh) & 255u) << (WIDE ? 23 : 0);
#pragma unroll
    for (int j = 0; j < TN; j++) xb[j] = (int)((sb[j] >> sh) & 255u) << (WIDE ? 23 : 0);
  };

  // ---- products
  f32x16 acc[TM][TN];
  const int fx = hf ^ (((lane & 31) >> 1) & 7);
  i32x8 af[TM], bfr[TN];
  auto fragment = [&](const char* s, int h) {
    const u32x4 x = *reinterpret_cast<const u32x4*>(s + (((4 * h) ^ fx) * 16)), y = *reinterpret_cast<const u32x4*>(s + (((4 * h + 2) ^ fx) * 16));
    return (i32x8){(int)x[0], (int)x[1], (int)x[2], (int)x[3], (int)y[0], (int)y[1], (int)y[2], (int)y[3]};
  };
  auto read_fragments = [&](const char* a, const char* b, int h) {
#pragma unroll
    for (int j = 0; j < TN; j++) bfr[j] = fragment(b + j * 32 * 128, h);
#pragma unroll
    for (int i = 0; i < TM; i++) af[i] = fragment(a + i * 32 * 128, h);
  };
  // WIDE: the fragments of 16 of K are turned into bf16 while the matrix instructions of the 16 before run, those of a phase's first 16 before its barrier
  bf16x8 wa, wb[TN];
  auto widen_a = [&](int i, int k) { return widen8<FA>(af[i][2 * k], af[i][2 * k + 1], xa[i]); };
  auto widen_b = [&](int j, int k) { return widen8<FB>(bfr[j][2 * k], bfr[j][2 * k + 1], xb[j]); };
  auto widen_first = [&]() {
    if constexpr (WIDE) {
#pragma unroll
      for (int j = 0; j < TN; j++) wb[j] = widen_b(j, 0);
      wa = widen_a(0, 0);
    }
  };
  auto compute_phase = [&](bool live) {
    __builtin_amdgcn_sched_barrier(0);
    if (live) {
      __builtin_amdgcn_s_setprio(1);
      if constexpr (WIDE) {
#pragma unroll
        for (int k = 0; k < 4; k++) {
          bf16x8 nb8[TN];
#pragma unroll
          for (int i = 0; i < TM; i++) {
            acc[i][0] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(wb[0], wa, acc[i][0], 0, 0, 0);
            bf16x8 next = wa;
            if (i + 1 < TM) next = widen_a(i + 1, k);
            else if (k < 3) next = widen_a(0, k + 1);
            acc[i][1] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(wb[1], wa, acc[i][1], 0, 0, 0);
            if (k < 3 && i == 1) nb8[0] = widen_b(0, k + 1);
            if (k < 3 && i == 2) nb8[1] = widen_b(1, k + 1);
            wa = next;
          }
          if (k < 3) {
#pragma unroll
            for (int j = 0; j < TN; j++) wb[j] = nb8[j];
          }
        }
#pragma unroll
        for (int s = 0; s < 32; s++) {   // a matrix instruction, then three conversions
          __builtin_amdgcn_sched_group_barrier(0x8, 1, 0);
          __builtin_amdgcn_sched_group_barrier(0x2, 3, 0);
        }
      } else {
#pragma unroll
        for (int i = 0; i < TM; i++)
#pragma unroll
          for (int j = 0; j < TN; j++) acc[i][j] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(bfr[j], af[i], acc[i][j], FB, FA, 0, xb[j], 0, xa[i]);
      }
      __builtin_amdgcn_s_setprio(0);
    }
    __builtin_amdgcn_sched_barrier(0);
  };

  int id = blockIdx.x, slot = 0;   // slot: of the present slice's A
  Fp8Tile t = p_tile;
  auto next_slot = [](int s, int by) { return s + by < 5 ? s + by : s + by - 5; };
  load_scales(t, t.slice0);
  take_scales();
  if (grp == 0) {
    issue_a();
    issue_b();
    issue_a();
    if (t.nk > 1 || (int)gridDim.x + id < tiles) wait_loads<8>(); else wait_loads<0>();   // but for the last of the three, if there was one
    end_of_k(t.slice0, 0, 1);
  }
  __syncthreads();
  while (true) {
    const int mh = row_half(t), ncol0 = col_quarter(t) * 64, id2 = id + gridDim.x;
    const bool live = t.m0 + mh * 128 < g.M && t.n0 + ncol0 < g.N, more = id2 < tiles;
    const Fp8Tile t2 = more ? fp8_tile(g, id2) : t;
    const int a_lds = (mh * 128 + (lane & 31)) * 128, b_lds = (ncol0 + (lane & 31)) * 128;
#pragma unroll
    for (int i = 0; i < TM; i++)
#pragma unroll
      for (int j = 0; j < TN; j++)
#pragma unroll
        for (int v = 0; v < 16; v++) acc[i][j][v] = 0.0f;
    if (grp == 1) __builtin_amdgcn_s_barrier();   // one phase behind
    for (int kt = 0; kt < t.nk;) {
      const int end4 = ((t.slice0 + kt) | 3) + 1 - t.slice0, end = end4 < t.nk ? end4 : t.nk;
      if (end < t.nk) load_scales(t, t.slice0 + end);
      else load_scales(t2, t2.slice0);
      for (; kt < end; kt++) {
        const char* a = smem + slot * F8_UNIT + a_lds;
        const char* b = smem + next_slot(slot, 1) * F8_UNIT + b_lds;
        if (live) read_fragments(a, b, 0);
        slice_scales(t.slice0 + kt);
        if (grp == 0) issue_b();
        if (live) widen_first();
        __syncthreads();
        compute_phase(live);
        __builtin_amdgcn_s_barrier();
        if (live) read_fragments(a, b, 1);
        bool ahead = false;
        if (grp == 0 && kt + 1 < end) ahead = issue_a();
        if (live) widen_first();
        __syncthreads();
        compute_phase(live);
        slot = next_slot(slot, 2);
        if (grp == 0) {
          if (ahead) wait_loads<8>(); else wait_loads<0>();
          end_of_k(kt + 1 < t.nk ? t.slice0 + kt + 1 : more ? t2.slice0 : 0, slot, next_slot(slot, 1));
        }
        // both groups pass as many barriers: group 1 leaves its last one out, behind which nobody reads this tile any more
        if (!(grp == 1 && kt == t.nk - 1)) __builtin_amdgcn_s_barrier();
      }
      take_scales();
      if (grp == 0) issue_a();
    }
    if (live) {   // through the two slots that the last slice had
      TO* C = (TO*)g.c + (int64_t)t.z * g.split_stride;
      char* stg = smem + next_slot(slot, grp ? 4 : 3) * F8_UNIT + sub * F8_STAGING;
      fp8_epilogue<HOW, TM, TN, TO>(acc, stg, g, C, g.r, t.m0 + mh * 128, t.n0 + ncol0, lane);
    }
    if (!more) break;
    __syncthreads();   // the staging is free again
    t = t2;
    id = id2;
  }
}

// ---- tiles of 128 x 128 and 64 x 64 -------------------------------------------------------------
// For products whose tiles of 256 x 256 leave much of the chip idle, or that have fewer rows.  The latency of the operands bounds them, so a workgroup keeps
// NST - 1 slices under way (96 KB; 64 KB each for two workgroups a CU with 64 x 64) and waits for the oldest only, one barrier a slice, as in
// gemm_mfma_deep.hip.  Two wavefronts share a sub-tile of 64 rows, each with 64 of the 128 of a slice; their sums meet in LDS, and each writes half of the rows.
// Slice kt lies in buffer kt % NST: behind the barrier of slice kt, which every wavefront reaches with its reads of slice kt - 1 done and its loads of slice kt
// landed, slice kt + NST - 1 is loaded into the buffer of slice kt - 1.  Scale words (four slices of a row) are loaded to LDS with the first slice of the four, ahead of it;
// the waits count the operands' loads alone, so that one with scale words behind it waits for a little more than it has to.
__device__ __forceinline__ void global_to_lds_4(const void* base, unsigned voff, unsigned lds_addr) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tglobal_load_lds_dword %1, %2" ::"s"(lds_addr), "v"(voff), "s"(base) : "memory");
}
template <int LPW, int LEFT>
__device__ __forceinline__ void wait_slices(int younger) {   // younger: slices under way behind the awaited one, at most LEFT
  if constexpr (LEFT == 0) wait_loads<0>();
  else if (younger >= LEFT) wait_loads<LPW * LEFT>();
  else wait_slices<LPW, LEFT - 1>(younger);
}

template <int BM, int BN, int NST>
struct Fp8Deep {
  static constexpr int WM = BM / 64, WN = 2, NW = 2 * WM * WN, NT = 64 * NW, TM = 2, TN = BN / WN / 32;
  static constexpr int A_BYTES = BM * 128, B_BYTES = BN * 128, STAGE = A_BYTES + B_BYTES, SCALES = (BM + BN) * 4;
  static constexpr int LA = A_BYTES / 1024 / NW, LB = B_BYTES / 1024 / NW;   // loads of a wavefront a slice
  static constexpr int LDS = NST * STAGE + 2 * SCALES;
  static_assert(NT == 4 * BM && LA * 1024 * NW == A_BYTES && LB * 1024 * NW == B_BYTES && 8 * (LA + LB) <= 64 && (BM + BN) % 64 == 0 && (BM + BN) / 64 <= NW && LDS <= 160 * 1024, "whole loads");
  static_assert((NST - 2) * (LA + LB) < 63, "the wait counter has 6 bits");
  static_assert(NW * (TN * 4096 + F8_STAGING) <= NST * STAGE, "exchange and staging fit the operand buffers");
};

template <int FA, int FB, bool WIDE, typename TO, int BM, int BN, int NST>
__global__ __launch_bounds__(4 * BM) void gemm_fp8_deep_kernel(Fp8Args g) {
  typedef Fp8Deep<BM, BN, NST> D;
  constexpr int TM = D::TM, TN = D::TN, LA = D::LA, LB = D::LB;
  __shared__ __attribute__((aligned(1024))) char smem[D::LDS];
  const int lane = threadIdx.x & 63, wave = fp8_uniform(threadIdx.x >> 6), share = wave & 1, wn = (wave >> 1) & 1, wm = wave >> 2, hf = lane >> 5;
  // a contiguous run of tiles, columns fastest, for every XCD; share of K after share of K
  const int ntiles = g.tiles_m * g.tiles_n, total = ntiles * g.nsplit, base = total / 8, rem = total % 8, x8 = blockIdx.x & 7;
  const int p = x8 * base + (x8 < rem ? x8 : rem) + (blockIdx.x >> 3), z = p / ntiles, tile = p - z * ntiles;
  const int m0 = tile / g.tiles_n * BM, n0 = (tile - tile / g.tiles_n * g.tiles_n) * BN;
  const int nkt = (g.K + 127) / 128, tail = g.K & 127, q = nkt / g.nsplit, e = nkt - q * g.nsplit;
  const int nk = q + (z < e ? 1 : 0), slice0 = z * q + (z < e ? z : e);

  const uint8_t* Ag = g.a + (int64_t)m0 * g.lda;
  const uint8_t* Bg = g.b + (int64_t)n0 * g.ldb;
  const int rows_a = g.M - m0, rows_b = g.N - n0;   // rows beyond the matrix are its last one
  unsigned a_off[LA], b_off[LB];
  int a_piece[LA], b_piece[LB];
#pragma unroll
  for (int i = 0; i < LA; i++) {
    const int R = 8 * (LA * wave + i) + (lane >> 3);
    a_off[i] = (unsigned)(R < rows_a ? R : rows_a - 1) * (unsigned)g.lda;
    a_piece[i] = ((lane & 7) ^ ((R >> 1) & 7)) * 16;
  }
#pragma unroll
  for (int i = 0; i < LB; i++) {
    const int R = 8 * (LB * wave + i) + (lane >> 3);
    b_off[i] = (unsigned)(R < rows_b ? R : rows_b - 1) * (unsigned)g.ldb;
    b_piece[i] = ((lane & 7) ^ ((R >> 1) & 7)) * 16;
  }
  // wavefront w < (BM + BN) / 64 loads the scale words of rows 64 w .. of A's and then B's
  const int srow = 64 * wave + lane;
  const bool s_mine = wave < (BM + BN) / 64, s_of_a = 64 * wave < BM;
  const uint8_t* Sg = s_of_a ? g.sa + (int64_t)(m0 >> g.sha) * g.lda_s : g.sb + (int64_t)(n0 >> g.shb) * g.ldb_s;
  unsigned s_off;
  {
    const int r = s_of_a ? srow : srow - BM, rows = s_of_a ? rows_a : rows_b;
    s_off = (unsigned)(((r < rows ? r : rows - 1) >> (s_of_a ? g.sha : g.shb)) * (s_of_a ? g.lda_s : g.ldb_s));
  }
  const unsigned lds0 = (unsigned)(uintptr_t)(__attribute__((address_space(3))) char*)(smem);
  auto issue = [&](int kt, int buf) {
    const int kb = slice0 + kt;
    if (s_mine && (kt == 0 || (kb & 3) == 0)) global_to_lds_4(Sg + (kb & ~3), s_off, lds0 + NST * D::STAGE + ((kb >> 2) & 1) * D::SCALES + wave * 256);
    const uint8_t* ap = Ag + (int64_t)kb * 128;
    const uint8_t* bp = Bg + (int64_t)kb * 128;
    const unsigned dst = lds0 + buf * D::STAGE;
    const int most = tail && kb == nkt - 1 ? (tail - 1) & ~15 : 112;
#pragma unroll
    for (int i = 0; i < LA; i++) global_to_lds_16(ap, a_off[i] + (a_piece[i] < most ? a_piece[i] : most), dst + (LA * wave + i) * 1024);
#pragma unroll
    for (int i = 0; i < LB; i++) global_to_lds_16(bp, b_off[i] + (b_piece[i] < most ? b_piece[i] : most), dst + D::A_BYTES + (LB * wave + i) * 1024);
  };
  // the wavefront's own loads of a slice that K ends in: lane l has row l of its rows of A, then of B
  auto end_of_k = [&](int kt, int buf) {
    if (!tail || slice0 + kt != nkt - 1) return;
    if (lane < 8 * (LA + LB)) {
      const bool a = lane < 8 * LA;
      const int R = a ? 8 * LA * wave + lane : 8 * LB * wave + lane - 8 * LA;
      zero_behind(smem + buf * D::STAGE + (a ? 0 : D::A_BYTES) + R * 128, (R >> 1) & 7, tail);
    }
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
  };

  f32x16 acc[TM][TN];
#pragma unroll
  for (int i = 0; i < TM; i++)
#pragma unroll
    for (int j = 0; j < TN; j++)
#pragma unroll
      for (int v = 0; v < 16; v++) acc[i][j][v] = 0.0f;
  const int fx = hf ^ (((lane & 31) >> 1) & 7);
  const int a_lds = (wm * 64 + (lane & 31)) * 128, b_lds = D::A_BYTES + (wn * TN * 32 + (lane & 31)) * 128;
  const int sa_lds = NST * D::STAGE + (wm * 64 + (lane & 31)) * 4, sb_lds = NST * D::STAGE + (BM + wn * TN * 32 + (lane & 31)) * 4;
  auto compute = [&](const char* s, int kb) {
    auto fragment = [&](const char* r) {
      const u32x4 x = *reinterpret_cast<const u32x4*>(r + (((4 * share) ^ fx) * 16)), y = *reinterpret_cast<const u32x4*>(r + (((4 * share + 2) ^ fx) * 16));
      return (i32x8){(int)x[0], (int)x[1], (int)x[2], (int)x[3], (int)y[0], (int)y[1], (int)y[2], (int)y[3]};
    };
    const char* sc = smem + ((kb >> 2) & 1) * D::SCALES + (kb & 3);
    i32x8 af[TM], bfr[TN];
    int xa[TM], xb[TN];
#pragma unroll
    for (int j = 0; j < TN; j++) {
      bfr[j] = fragment(s + b_lds + j * 32 * 128);
      xb[j] = (int)*reinterpret_cast<const uint8_t*>(sc + sb_lds + j * 32 * 4) << (WIDE ? 23 : 0);
    }
#pragma unroll
    for (int i = 0; i < TM; i++) {
      af[i] = fragment(s + a_lds + i * 32 * 128);
      xa[i] = (int)*reinterpret_cast<const uint8_t*>(sc + sa_lds + i * 32 * 4) << (WIDE ? 23 : 0);
    }
    if constexpr (WIDE) {
#pragma unroll
      for (int k = 0; k < 8; k += 2) {
        bf16x8 a[TM], b[TN];
#pragma unroll
        for (int j = 0; j < TN; j++) b[j] = widen8<FB>(bfr[j][k], bfr[j][k + 1], xb[j]);
#pragma unroll
        for (int i = 0; i < TM; i++) a[i] = widen8<FA>(af[i][k], af[i][k + 1], xa[i]);
#pragma unroll
        for (int i = 0; i < TM; i++)
#pragma unroll
          for (int j = 0; j < TN; j++) acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(b[j], a[i], acc[i][j], 0, 0, 0);
      }
    } else {
#pragma unroll
      for (int i = 0; i < TM; i++)
#pragma unroll
        for (int j = 0; j < TN; j++) acc[i][j] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(bfr[j], af[i], acc[i][j], FB, FA, 0, xb[j], 0, xa[i]);
    }
  };

#pragma unroll
  for (int s = 0; s < NST - 1; s++)
    if (s < nk) issue(s, s);
  int cur = 0;   // kt % NST
  for (int kt = 0; kt < nk; kt++) {
    wait_slices<LA + LB, NST - 2>(nk - 1 - kt);
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    end_of_k(kt, cur);
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
    if (kt + NST - 1 < nk) issue(kt + NST - 1, cur == 0 ? NST - 1 : cur - 1);
    compute(smem + cur * D::STAGE, slice0 + kt);
    cur = cur == NST - 1 ? 0 : cur + 1;
  }

  __syncthreads();   // every wavefront is done with the operand buffers
  f32x16 own[1][TN];
  f32x4* give = reinterpret_cast<f32x4*>(smem + wave * (TN * 4096));
  const f32x4* take = reinterpret_cast<const f32x4*>(smem + (wave ^ 1) * (TN * 4096));
#pragma unroll
  for (int j = 0; j < TN; j++) {
    const f32x16 x = share ? acc[0][j] : acc[1][j];
    own[0][j] = share ? acc[1][j] : acc[0][j];
#pragma unroll
    for (int w = 0; w < 4; w++) give[(j * 4 + w) * 64 + lane] = (f32x4){x[4 * w], x[4 * w + 1], x[4 * w + 2], x[4 * w + 3]};
  }
  __syncthreads();
#pragma unroll
  for (int j = 0; j < TN; j++)
#pragma unroll
    for (int w = 0; w < 4; w++) {
      const f32x4 x = take[(j * 4 + w) * 64 + lane];
#pragma unroll
      for (int v = 0; v < 4; v++) own[0][j][4 * w + v] += x[v];
    }
  const int row0 = m0 + wm * 64 + share * 32, col0 = n0 + wn * TN * 32;
  if (row0 >= g.M || col0 >= g.N) return;
  fp8_epilogue<EPI_ASK, 1, TN, TO>(own, smem + D::NW * (TN * 4096) + wave * F8_STAGING, g, (TO*)g.c + (int64_t)z * g.split_stride, g.r, row0, col0, lane);
}

template <int FA, int FB, bool WIDE, typename TO>
inline int launch_fp8(Fp8Args g, int tile, hipStream_t st) {
  g.tiles_m = (g.M + tile - 1) / tile;
  g.tiles_n = (g.N + tile - 1) / tile;
  const int tiles = g.tiles_m * g.tiles_n * g.nsplit;
  g.div_tiles = fp8_reciprocal(g.tiles_m * g.tiles_n);
  g.div_span = fp8_reciprocal(8 * g.tiles_m);
  if (tile == 256) {
    const dim3 grid(tiles < 256 ? tiles : 256);   // one a CU
    if constexpr (!WIDE && sizeof(TO) == 4) {     // partial sums, aligned
      hipLaunchKernelGGL((gemm_fp8_pp_kernel<FA, FB, WIDE, TO, 0>), grid, dim3(512), 0, st, g, tiles);
    } else {
      const bool whole = g.M % 128 == 0 && g.N % 64 == 0;   // no wavefront's part of a tile ends outside
      const int how = (g.r ? EPI_ADD : 0) | (fp8_aligned(g) ? 0 : EPI_ANY) | (g.r && !(whole && fp8_aligned(g)) ? EPI_EDGE : 0);
      if (how == 0) hipLaunchKernelGGL((gemm_fp8_pp_kernel<FA, FB, WIDE, TO, 0>), grid, dim3(512), 0, st, g, tiles);
      else if (how == EPI_ADD) hipLaunchKernelGGL((gemm_fp8_pp_kernel<FA, FB, WIDE, TO, EPI_ADD>), grid, dim3(512), 0, st, g, tiles);
      else if (how == (EPI_ADD | EPI_EDGE)) hipLaunchKernelGGL((gemm_fp8_pp_kernel<FA, FB, WIDE, TO, EPI_ADD | EPI_EDGE>), grid, dim3(512), 0, st, g, tiles);
      else if (how == EPI_ANY) hipLaunchKernelGGL((gemm_fp8_pp_kernel<FA, FB, WIDE, TO, EPI_ANY>), grid, dim3(512), 0, st, g, tiles);
      else hipLaunchKernelGGL((gemm_fp8_pp_kernel<FA, FB, WIDE, TO, EPI_ADD | EPI_ANY | EPI_EDGE>), grid, dim3(512), 0, st, g, tiles);
    }
  } else if (tile == 128) hipLaunchKernelGGL((gemm_fp8_deep_kernel<FA, FB, WIDE, TO, 128, 128, 4>), dim3(tiles), dim3(Fp8Deep<128, 128, 4>::NT), 0, st, g);
  else hipLaunchKernelGGL((gemm_fp8_deep_kernel<FA, FB, WIDE, TO, 64, 64, 4>), dim3(tiles), dim3(Fp8Deep<64, 64, 4>::NT), 0, st, g);
  ALS_CHECK_LAUNCH();
  return ALS_OK;
}

}  // namespace

template <int FA, int FB>
int gemm_fp8_launch(Fp8Args g, int tile, Fp8Out out, hipStream_t st) {
  if (out == FP8_BF16) return launch_fp8<FA, FB, false, bf16>(g, tile, st);
  return out == FP8_F32 ? launch_fp8<FA, FB, true, float>(g, tile, st) : launch_fp8<FA, FB, false, float>(g, tile, st);
}

}  // namespace als
