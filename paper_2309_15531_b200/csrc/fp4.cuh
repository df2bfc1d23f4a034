// Microscaled 4-bit floating point: sizes of the layout that include/adadim.h defines, and the
// quantizer's arithmetic.  Internal header.
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include <atomic>

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

// Two binary32 operations at once (the packed instructions of this architecture).
__device__ __forceinline__ uint64_t pack2(float a, float b) {
  uint64_t r;
  asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(a), "f"(b));
  return r;
}
__device__ __forceinline__ void unpack2(uint64_t v, float& a, float& b) { asm("mov.b64 {%0, %1}, %2;" : "=f"(a), "=f"(b) : "l"(v)); }
__device__ __forceinline__ uint64_t mul2(uint64_t a, uint64_t b) {
  uint64_t r;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}
__device__ __forceinline__ uint64_t add2(uint64_t a, uint64_t b) {
  uint64_t r;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}
__device__ __forceinline__ uint64_t fma2(uint64_t a, uint64_t b, uint64_t c) {
  uint64_t r;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
  return r;
}

// The scale of a block with largest magnitude m (NaN if the block holds one).  What is returned: the
// byte, and the divisor of the elements as s and 1 / s (exact for MXFP4; for NVFP4 correctly rounded, or
// with X16 within an ulp); s = 0 means that every value is 0.
struct BlockScale {
  uint32_t byte;
  float s, rcp;
  bool finite;
  bool far;                // NVFP4: quotients of binary32 numbers may overflow (amax far below the block's m)
};
template <int FORMAT, bool X16>
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
    // m / t is exact (and cut where it is far beyond the largest scale anyway).  The correctly rounded
    // quotient by 6 decides every comparison with a number of at most 5 significant bits as the exact
    // quotient does: a number that is not the midpoint c differs from it by at least an ulp of the dividend
    // 6 c, which is more than half an ulp of the quotient.
    const float u = quotient(fminf(m * exp2_int(-t_log2), 1e30f), 6.0f, 1.0f / 6.0f);
    b.byte = finite ? e4m3_of(u) : 0x7fu;
    const float sf = finite ? e4m3_value(b.byte) : 0.0f;
    b.s = sf * exp2_int(t_log2);
    if (X16) asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(b.rcp) : "f"(b.s));
    else b.rcp = __frcp_rn(b.s);
    if (!(b.s > 0.0f)) b.rcp = 0.0f;
    if (!X16) b.far = m * b.rcp > 1e30f;
  }
  return b;
}
// The eight codes of v[0..7], elements of one block, from x / s in a form that lies on the same side of
// (or on) every midpoint c of two levels as the exact quotient:
//   MXFP4: exact (s is a power of two).
//   NVFP4, x of a 16-bit type: x * (1 / s) is within 2^-22 of the quotient, relatively, and 5 is the largest c.
//     A quotient that is not c differs from it by 2^-11 c or more (x has at most 11 significant bits, c s at
//     most 7) and c is at least 1/4, so rounding to multiples of 2^-18, by adding 48 and taking it away,
//     restores exact midpoints and moves nothing across one.
//   NVFP4, x binary32: the correctly rounded quotient, by the argument given for the block scale.
// The sign of a zero is not kept.
template <int FORMAT, bool X16>
__device__ __forceinline__ uint32_t codes8(const float* v, const BlockScale& b) {
  float q[8];
  const uint64_t rcp = pack2(b.rcp, b.rcp);
#pragma unroll
  for (int k = 0; k < 8; k += 2) {
    float x0 = v[k], x1 = v[k + 1];
    if (FORMAT == ADADIM_NVFP4 && !X16 && b.far) {                   // beyond 6 s all the same
      x0 = fminf(fmaxf(x0, -8.0f * b.s), 8.0f * b.s);
      x1 = fminf(fmaxf(x1, -8.0f * b.s), 8.0f * b.s);
    }
    const uint64_t x = pack2(x0, x1);
    uint64_t y;
    if (FORMAT == ADADIM_MXFP4) {
      y = mul2(x, rcp);
    } else if (X16) {
      y = add2(fma2(x, rcp, pack2(48.0f, 48.0f)), pack2(-48.0f, -48.0f));
    } else {
      const uint64_t q0 = mul2(x, rcp);
      y = fma2(fma2(pack2(-b.s, -b.s), q0, x), rcp, q0);
    }
    unpack2(y, q[k], q[k + 1]);
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

// ---- a matrix to be quantized: 16 consecutive elements at a time -------------------------------------
constexpr int kPer = 16;
struct Source {
  const void* X;
  int64_t ldx, x_rows;
  const int32_t* row_index;   // row r is X[row_index[r]], zeros where that is outside; NULL: X[r]
  uintptr_t begin, end;       // the bytes of X: no 16-byte block that leaves them is loaded whole
  int wide;                   // every row (or the only one) starts on a 32-byte boundary
};
inline Source source_of(const void* X, int dtype, int64_t ldx, int64_t x_rows, int64_t cols, const int32_t* row_index) {
  const int64_t esz = dtype == ADADIM_F32 ? 4 : 2;
  const uintptr_t x0 = reinterpret_cast<uintptr_t>(X);
  Source s = {X, ldx, x_rows, row_index, x0, x0, x0 % 32 == 0 && (x_rows == 1 || (ldx * esz) % 32 == 0)};
  if (x_rows > 0) s.end = x0 + static_cast<uintptr_t>(((x_rows - 1) * ldx + cols) * esz);
  return s;
}
template <typename T> struct Elem;
template <> struct Elem<__half> {
  typedef __half2 Two;
  static __device__ __forceinline__ float to_f32(uint16_t b) { return __half2float(__ushort_as_half(b)); }
  static __device__ __forceinline__ Two abs2(uint32_t w) { return __habs2(*reinterpret_cast<const Two*>(&w)); }
  static __device__ __forceinline__ float2 widen2(uint32_t w) { return __half22float2(*reinterpret_cast<const Two*>(&w)); }
  static __device__ __forceinline__ float top_f32(Two t) { return __half2float(__hmax_nan(__low2half(t), __high2half(t))); }
};
template <> struct Elem<__nv_bfloat16> {
  typedef __nv_bfloat162 Two;
  static __device__ __forceinline__ float to_f32(uint16_t b) { return __uint_as_float(static_cast<uint32_t>(b) << 16); }
  static __device__ __forceinline__ Two abs2(uint32_t w) { return __habs2(*reinterpret_cast<const Two*>(&w)); }
  static __device__ __forceinline__ float2 widen2(uint32_t w) { return make_float2(__uint_as_float(w << 16), __uint_as_float(w & 0xffff0000u)); }
  static __device__ __forceinline__ float top_f32(Two t) { return __bfloat162float(__hmax_nan(__low2bfloat16(t), __high2bfloat16(t))); }
};

// The sixteen elements of a thread as they lie in memory, and their loads.
template <typename T> struct Raw { uint32_t w[kPer * sizeof(T) / 4]; };

__device__ __forceinline__ void load32(const void* p, uint32_t* w) {            // 32-byte aligned
  asm volatile("ld.global.nc.v8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
               : "=r"(w[0]), "=r"(w[1]), "=r"(w[2]), "=r"(w[3]), "=r"(w[4]), "=r"(w[5]), "=r"(w[6]), "=r"(w[7]) : "l"(p));
}
template <typename T>
__device__ __forceinline__ void load16_aligned(const T* p, Raw<T>& r) {
  load32(p, r.w);
  if constexpr (sizeof(T) == 4) load32(p + 8, r.w + 8);
}
// Any alignment: the 16-byte blocks that hold the elements, shifted into place.  The caller has checked
// that the blocks lie inside the matrix.
template <typename T>
__device__ __forceinline__ void load16_shifted(const T* p, Raw<T>& r) {
  constexpr int kW = kPer * sizeof(T) / 4;
  const uint32_t off = static_cast<uint32_t>(reinterpret_cast<uintptr_t>(p)) & 15u;
  const uint4* q = reinterpret_cast<const uint4*>(reinterpret_cast<uintptr_t>(p) - off);
  uint32_t w[kW + 4];
#pragma unroll
  for (int k = 0; k <= kW / 4; ++k) {
    const uint4 v = k < kW / 4 || off != 0 ? __ldg(q + k) : make_uint4(0, 0, 0, 0);
    w[4 * k] = v.x; w[4 * k + 1] = v.y; w[4 * k + 2] = v.z; w[4 * k + 3] = v.w;
  }
#pragma unroll
  for (int k = 0; k < kW + 2; ++k) if (off & 8u) w[k] = w[k + 2];
#pragma unroll
  for (int k = 0; k < kW + 1; ++k) if (off & 4u) w[k] = w[k + 1];
#pragma unroll
  for (int k = 0; k < kW; ++k) r.w[k] = sizeof(T) == 2 ? __funnelshift_r(w[k], w[k + 1], (off & 2u) * 8) : w[k];
}
// The first n elements one by one, zeros behind them.
template <typename T>
__device__ __forceinline__ void load16_narrow(const T* p, int n, Raw<T>& r) {
#pragma unroll
  for (int k = 0; k < kPer * static_cast<int>(sizeof(T)) / 4; ++k) {
    if constexpr (sizeof(T) == 2) {
      const uint16_t* h = reinterpret_cast<const uint16_t*>(p);
      const uint32_t lo = 2 * k < n ? h[2 * k] : 0u, hi = 2 * k + 1 < n ? h[2 * k + 1] : 0u;
      r.w[k] = lo | (hi << 16);
    } else {
      r.w[k] = k < n ? reinterpret_cast<const uint32_t*>(p)[k] : 0u;
    }
  }
}
// Widened to binary32; the largest magnitude as a binary32 pattern (patterns are ordered as integers)
template <typename T>
__device__ __forceinline__ uint32_t widen(const Raw<T>& r, float (&v)[kPer]) {
  if constexpr (sizeof(T) == 2) {
    typename Elem<T>::Two top = Elem<T>::abs2(r.w[0]);
#pragma unroll
    for (int k = 1; k < 8; ++k) top = __hmax2_nan(top, Elem<T>::abs2(r.w[k]));   // a NaN stays on top
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      const float2 f = Elem<T>::widen2(r.w[k]);
      v[2 * k] = f.x;
      v[2 * k + 1] = f.y;
    }
    return __float_as_uint(Elem<T>::top_f32(top)) & 0x7fffffffu;
  } else {
    uint32_t m = 0;
#pragma unroll
    for (int k = 0; k < kPer; ++k) {
      v[k] = __uint_as_float(r.w[k]);
      m = max(m, r.w[k] & 0x7fffffffu);
    }
    return m;
  }
}

// Row r of the matrix in X, or -1 for a row of zeros.
__device__ __forceinline__ int64_t source_row(const Source& s, int64_t r) {
  if (s.row_index == nullptr) return r;
  const int64_t src = s.row_index[r];
  return src < 0 || src >= s.x_rows ? -1 : src;
}
// Elements c0 .. c0 + n - 1 of row src of X (n = 0 or src = -1: none), zeros behind them.
template <typename T>
__device__ __forceinline__ void load16(const Source& s, int64_t src, int64_t c0, int n, Raw<T>& r) {
  const T* at = static_cast<const T*>(s.X) + src * s.ldx + c0;
  const uintptr_t a = reinterpret_cast<uintptr_t>(at);
  if (src < 0 || n == 0) load16_narrow(at, 0, r);
  else if (n == kPer && s.wide) load16_aligned(at, r);
  else if (n == kPer && (a & ~uintptr_t(15)) >= s.begin && a + kPer * sizeof(T) + 15 < s.end) load16_shifted(at, r);
  else load16_narrow(at, n, r);
}

// The rows that scale tile row v holds (see sf_tile_rows): first and count, 0 if it holds none.  For a whole
// converged warp: the group is found by counting over the clamped offsets, all of which are loaded at once.
__device__ __forceinline__ int clamped(int v, int rows) { return v < 0 ? 0 : v > rows ? rows : v; }
__device__ __forceinline__ void rows_of_tile_row(const int32_t* offsets, int n_groups, int rows, int lt, int v, int& first, int& count) {
  const int sub = (lt + kSfRows - 1) / kSfRows, cut = v / sub, part = v - cut * sub;
  int a = 0, z = rows, skip = cut * lt;
  if (offsets != nullptr) {
    const int lane = threadIdx.x & 31;
    int n = 0;                                                       // groups with offsets[e] / lt + e <= cut
    for (int e0 = 0; e0 < n_groups; e0 += 32) {
      const int e = e0 + lane;
      n += __popc(__ballot_sync(0xffffffffu, e < n_groups && clamped(offsets[e], rows) / lt + e <= cut));
    }
    const int e = n > 0 ? n - 1 : 0;
    a = clamped(offsets[e], rows);
    z = clamped(offsets[e + 1], rows);
    skip = (cut - (a / lt + e)) * lt;
  }
  first = a + skip + part * kSfRows;
  count = skip < 0 ? 0 : min(min(lt - part * kSfRows, kSfRows), z - first);
  if (count < 0) count = 0;
}

}  // namespace fp4

// Sets an attribute of a kernel the first time it is launched on a device (a kernel's attributes stay as they are
// set; asking again costs each call half a microsecond).
template <typename K>
int set_once(K kernel, cudaFuncAttribute attr, int value, std::atomic<uint64_t>& devices) {
  int dev = 0;
  ADADIM_CUDA_TRY(cudaGetDevice(&dev));
  const uint64_t bit = uint64_t{1} << (dev & 63);
  if (dev < 64 && (devices.load(std::memory_order_acquire) & bit) != 0) return ADADIM_OK;
  ADADIM_CUDA_TRY(cudaFuncSetAttribute(kernel, attr, value));
  if (dev < 64) devices.fetch_or(bit, std::memory_order_release);
  return ADADIM_OK;
}

// implemented in fp4_quant.cu and fp4_matmul.cu
int absmax_launch(const void* X, int xdtype, int64_t rows, int64_t cols, int64_t ldx, float* amax, cudaStream_t st);
// amax: where the tensor scale comes from and what q.amax is set to; NULL: it comes from q.amax
int quantize_fp4_launch(const fp4::Source& x, int xdtype, int64_t rows, int64_t cols, int format, const int32_t* offsets,
                        int n_groups, const adadim_fp4tensor& q, const float* amax, int lt, void* values, int vdtype, int64_t ldv,
                        cudaStream_t st);
// How a product is laid out on the SMs.
struct Fp4Plan {
  bool pair;               // which kernel
  int n_tile;              // tokens of a tile
  int splits, per_sm;      // split kernel: CTAs of a cluster, CTAs of an SM
  bool fused;              // it quantizes the activations itself
};
// The activations come quantized (lt = 128), or the library quantizes them: then their scales are laid out as
// the plan likes best (lt = n_tile), and `fuse` says that the product could do it
// (X and Y of one type, 32-byte aligned rows, whole sixteens of columns).
Fp4Plan fp4_plan(int64_t rows, int64_t out, int64_t in, int n_experts, int format, bool quantized, bool fuse);
// A: quantized activations, or with plan.fused only their amax, and x the matrix itself.
int fp4_matmul_launch(const Fp4Plan& plan, const adadim_fp4tensor& A, int lt, const fp4::Source& x, int64_t n_rows,
                      const int32_t* offsets, int n_experts, const adadim_fp4tensor& B, int64_t out, int64_t in, int format, void* Y, int ydtype,
                      int64_t ldy, int* status_dev, bool chained, cudaStream_t st);
// the most scale tile rows that activations take in any plan's layout
int64_t fp4_most_tile_rows(int64_t rows, int n_experts);

}  // namespace adadim
