// Microscaled 4-bit floating point: sizes of the layout that include/adadim.h defines, and the
// quantizer's arithmetic.  Internal header.
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include "common.cuh"

namespace adadim {
namespace fp4 {

constexpr int kSfRows = 128;                 // rows of a scale tile
constexpr int kSfTileBytes = 512;            // 128 rows x 4 blocks
constexpr int kMaxGroups = 1024;

__host__ __device__ constexpr int block_of(int format) { return format == ADADIM_MXFP4 ? 32 : 16; }
// columns of a scale tile, and scale tiles of one tile row
__host__ __device__ constexpr int sf_cols(int format) { return 4 * block_of(format); }
__host__ __device__ __forceinline__ int64_t sf_tiles(int format, int64_t cols) {
  return (cols + sf_cols(format) - 1) / sf_cols(format);
}
// Tile rows of a matrix; of rows in groups (group e starts at tile row offsets[e] / 128 + e, and
// floor(a / 128) + ceil(n / 128) <= floor((a + n) / 128) + 1, so groups never overlap).
// Inside the library activations may be laid out for token tiles of another height `lt`: the rows are
// cut every lt (in each group), and every cut starts a tile row (TMEM holds the scales of 32 rows per
// column, and a product's scales have to begin on a whole tile).  lt = 128 is the public layout.
__host__ __device__ __forceinline__ int64_t sf_tile_rows(int64_t rows, int n_groups, int lt = kSfRows) {
  return (n_groups > 0 ? rows / lt + n_groups : (rows + lt - 1) / lt) * ((lt + kSfRows - 1) / kSfRows);
}
inline size_t scale_bytes(int format, int64_t rows, int64_t cols, int n_groups) {
  return static_cast<size_t>(sf_tile_rows(rows, n_groups)) * sf_tiles(format, cols) * kSfTileBytes;
}
inline int64_t code_pitch(int64_t cols) { return static_cast<int64_t>(round_up((cols + 1) / 2, 16)); }

// ---- device --------------------------------------------------------------------------------------
// log2 of the tensor scale: max(ceil(log2(amax / 2688)), -100), 2688 = 1.3125 * 2^11
__device__ __forceinline__ int tensor_scale_log2(const float* amax) {
  if (amax == nullptr) return 0;
  const float a = *amax;
  if (!(a > 0.0f) || !(a < INFINITY)) return 0;
  const uint32_t bits = __float_as_uint(a);
  const int e = static_cast<int>(bits >> 23) - 127;                  // a subnormal gives -127: clamped below
  const int c = e - 11 + ((bits & 0x7fffffu) > 0x280000u ? 1 : 0);   // 0x280000 = 0.3125 * 2^23
  return c < -100 ? -100 : c;
}
__device__ __forceinline__ float exp2_int(int e) { return __uint_as_float(static_cast<uint32_t>(e + 127) << 23); }   // -126 .. 127

// Four bytes of E2M1 pairs from eight values; the even element of a pair in the low half.
__device__ __forceinline__ uint32_t e2m1_pack8(const float* v) {
  uint32_t r;
  asm("{\n\t.reg .b8 a, b, c, d;\n\t"
      "cvt.rn.satfinite.e2m1x2.f32 a, %2, %1;\n\t"
      "cvt.rn.satfinite.e2m1x2.f32 b, %4, %3;\n\t"
      "cvt.rn.satfinite.e2m1x2.f32 c, %6, %5;\n\t"
      "cvt.rn.satfinite.e2m1x2.f32 d, %8, %7;\n\t"
      "mov.b32 %0, {a, b, c, d};\n\t}"
      : "=r"(r) : "f"(v[0]), "f"(v[1]), "f"(v[2]), "f"(v[3]), "f"(v[4]), "f"(v[5]), "f"(v[6]), "f"(v[7]));
  return r;
}
// E4M3 byte nearest to v >= 0 (ties to even, at most 448), and its value
__device__ __forceinline__ uint32_t e4m3_of(float v) {
  uint16_t r;
  asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(r) : "f"(0.0f), "f"(v));
  return r & 0xffu;
}
__device__ __forceinline__ float e4m3_value(uint32_t byte) {
  uint32_t h2;
  asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(h2) : "h"(static_cast<uint16_t>(byte)));
  return __half2float(__ushort_as_half(static_cast<uint16_t>(h2 & 0xffffu)));
}

// The scale of a block with largest magnitude m (NaN if the block holds one).  What is returned:
// the byte, and the divisor of the elements as (s, 1 / s correctly rounded); s = 0 means all codes 0.
struct BlockScale {
  uint32_t byte;
  float s, rcp;
  bool finite;
  bool far;                // NVFP4: quotients of binary32 numbers may overflow (amax far below the block's m)
};
template <int FORMAT>
__device__ __forceinline__ BlockScale block_scale(float m, int t_log2) {
  BlockScale b;
  const bool finite = m < INFINITY;                                  // false for NaN too
  b.finite = finite;
  b.far = false;
  if (FORMAT == ADADIM_MXFP4) {
    const int e = static_cast<int>(__float_as_uint(m) >> 23) - 2;    // biased exponent of the scale
    const int byte = e < 0 ? 0 : e;
    b.byte = finite ? static_cast<uint32_t>(byte) : 0xffu;
    // 2^(byte - 127) and its reciprocal, both exact (byte is at most 252; 2^-127 is a subnormal number)
    b.s = byte == 0 ? __uint_as_float(0x00400000u) : __uint_as_float(static_cast<uint32_t>(byte) << 23);
    b.rcp = __uint_as_float(static_cast<uint32_t>(254 - byte) << 23);
  } else {
    // m / t is exact.  The binary32 quotient by 6 decides every comparison with a number of at most
    // 5 significant bits as the exact quotient does: a number that is not the midpoint c differs from
    // it by at least an ulp of the dividend 6 c, which is more than half an ulp of the quotient.
    const float u = __fdiv_rn(m * exp2_int(-t_log2), 6.0f);
    b.byte = finite ? e4m3_of(u) : 0x7fu;
    const float sf = finite ? e4m3_value(b.byte) : 0.0f;
    b.s = sf * exp2_int(t_log2);
    b.rcp = b.s > 0.0f ? __frcp_rn(b.s) : 0.0f;
    b.far = m * b.rcp > 1e30f;
  }
  return b;
}
// x / s as the quantizer needs it: something that lies on the same side of (or on) every midpoint c
// of two levels as the exact quotient, and keeps the sign of a zero.
//   MXFP4: exact (s is a power of two).
//   NVFP4, x of a 16-bit type: x * (1 / s) is within 2^-23 of the quotient; a quotient that is not c
//     differs from it by 2^-11 or more (x has at most 11 significant bits, c s at most 7), so rounding
//     the product to 17 significant bits restores exact midpoints and moves nothing across one.
//   NVFP4, x binary32: the correctly rounded quotient, by the argument given for the block scale.
template <int FORMAT, bool X16>
__device__ __forceinline__ float scaled(float x, const BlockScale& b) {
  if (FORMAT == ADADIM_MXFP4) return x * b.rcp;
  if (X16) return __uint_as_float((__float_as_uint(x * b.rcp) + 0x40u) & ~0x7fu);
  return copysignf(quotient(x, b.s, b.rcp), x);
}
// The eight codes of v[0..7], elements of one block
template <int FORMAT, bool X16>
__device__ __forceinline__ uint32_t codes8(const float* v, const BlockScale& b) {
  float q[8];
#pragma unroll
  for (int k = 0; k < 8; ++k) {
    float x = v[k];
    if (FORMAT == ADADIM_NVFP4 && !X16 && b.far) x = fminf(fmaxf(x, -8.0f * b.s), 8.0f * b.s);   // beyond 6 s all the same
    q[k] = scaled<FORMAT, X16>(x, b);
  }
  const uint32_t r = e2m1_pack8(q);
  return b.finite ? r : 0u;
}
// The values of eight packed codes, low half first.
__device__ __forceinline__ void e2m1_values8(uint32_t codes, float (&v)[8]) {
  uint32_t h[4];
  asm("{\n\t.reg .b8 a, b, c, d;\n\t"
      "mov.b32 {a, b, c, d}, %4;\n\t"
      "cvt.rn.f16x2.e2m1x2 %0, a;\n\t"
      "cvt.rn.f16x2.e2m1x2 %1, b;\n\t"
      "cvt.rn.f16x2.e2m1x2 %2, c;\n\t"
      "cvt.rn.f16x2.e2m1x2 %3, d;\n\t}"
      : "=r"(h[0]), "=r"(h[1]), "=r"(h[2]), "=r"(h[3]) : "r"(codes));
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    const float2 f = __half22float2(*reinterpret_cast<const __half2*>(&h[k]));
    v[2 * k] = f.x;
    v[2 * k + 1] = f.y;
  }
}

// The rows that scale tile row v holds (see sf_tile_rows): first and count, 0 if it holds none.  Groups are
// found by bisection over the clamped offsets.
__device__ __forceinline__ int clamped(int v, int rows) { return v < 0 ? 0 : v > rows ? rows : v; }
__device__ __forceinline__ void rows_of_tile_row(const int32_t* offsets, int n_groups, int rows, int lt, int v, int& first, int& count) {
  const int sub = (lt + kSfRows - 1) / kSfRows, cut = v / sub, part = v - cut * sub;
  int a = 0, z = rows, skip = cut * lt;
  if (offsets != nullptr) {
    int lo = 0, hi = n_groups - 1;                                   // last e with offsets[e] / lt + e <= cut
    while (lo < hi) {
      const int mid = (lo + hi + 1) >> 1;
      if (clamped(offsets[mid], rows) / lt + mid <= cut) lo = mid; else hi = mid - 1;
    }
    a = clamped(offsets[lo], rows);
    z = clamped(offsets[lo + 1], rows);
    skip = (cut - (a / lt + lo)) * lt;
  }
  first = a + skip + part * kSfRows;
  count = skip < 0 ? 0 : min(min(lt - part * kSfRows, kSfRows), z - first);
  if (count < 0) count = 0;
}

}  // namespace fp4

// implemented in fp4_quant.cu and fp4_matmul.cu
int absmax_launch(const void* X, int xdtype, int64_t rows, int64_t cols, int64_t ldx, float* amax, cudaStream_t st);
int quantize_fp4_launch(const void* X, int xdtype, int64_t rows, int64_t cols, int64_t ldx, int64_t x_rows, int format,
                        const int32_t* row_index, const int32_t* offsets, int n_groups, const adadim_fp4tensor& q,
                        int lt, void* values, int vdtype, int64_t ldv, cudaStream_t st);
// How a product is laid out on the SMs.
struct Fp4Plan {
  bool pair;               // which kernel
  int n_tile;              // tokens of a tile
  int splits, per_sm;      // split kernel: CTAs of a cluster, CTAs of an SM
};
// own_layout: the activations' scales are laid out as the plan likes best (lt = n_tile), otherwise lt = 128
Fp4Plan fp4_plan(int64_t rows, int64_t out, int64_t in, int n_experts, int format, bool own_layout);
int fp4_matmul_launch(const Fp4Plan& plan, const adadim_fp4tensor& A, int lt, int64_t n_rows, const int32_t* offsets,
                      int n_experts, const adadim_fp4tensor& B, int64_t out, int64_t in, int format, void* Y, int ydtype,
                      int64_t ldy, int* status_dev, bool chained, cudaStream_t st);
// the most scale tile rows that activations take in any plan's layout
int64_t fp4_most_tile_rows(int64_t rows, int n_experts);

}  // namespace adadim
