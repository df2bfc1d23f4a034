// Microscaled 4-bit quantizer and the largest magnitude its tensor scale is taken from.
//
// Both are bound by memory.  Quantizer: a CTA owns one scale tile, 128 rows x 64 (NVFP4) or 128 (MXFP4)
// columns, so the scales leave as one contiguous run although a row's scales lie 512 bytes apart.  A
// thread takes 16 consecutive columns (one NVFP4 block, half an MXFP4 block: the halves meet in one
// shuffle) of 2 or 4 rows, all of whose loads are issued before the first is used; its codes are one
// 8-byte store.  Work per element is a few instructions: packed magnitude maximum on the integer
// patterns (an infinity or NaN stays on top), one quotient (three operations against the block's
// reciprocal; MXFP4 one multiplication by a power of two), and the hardware conversion of pairs to E2M1.
#include "fp4.cuh"
#include "umma.cuh"

namespace adadim {
namespace {

using namespace fp4;

constexpr int kThreads = 256;
constexpr int kPer = 16;                     // columns of a thread

// ---- loads: 16 elements widened to binary32, magnitudes' maximum as a binary32 pattern -----------------
template <typename T> struct Elem;
template <> struct Elem<__half> {
  static __device__ __forceinline__ float to_f32(uint16_t b) { return __half2float(__ushort_as_half(b)); }
};
template <> struct Elem<__nv_bfloat16> {
  static __device__ __forceinline__ float to_f32(uint16_t b) { return __uint_as_float(static_cast<uint32_t>(b) << 16); }
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
__device__ __forceinline__ void store32(void* p, const uint32_t* w) {           // 32-byte aligned
  asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};"
               ::"l"(p), "r"(w[0]), "r"(w[1]), "r"(w[2]), "r"(w[3]), "r"(w[4]), "r"(w[5]), "r"(w[6]), "r"(w[7]) : "memory");
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
  uint32_t m = 0;
  if constexpr (sizeof(T) == 2) {
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      m = __vmaxu2(m, r.w[k] & 0x7fff7fffu);
      v[2 * k] = Elem<T>::to_f32(static_cast<uint16_t>(r.w[k] & 0xffffu));
      v[2 * k + 1] = Elem<T>::to_f32(static_cast<uint16_t>(r.w[k] >> 16));
    }
    return __float_as_uint(Elem<T>::to_f32(static_cast<uint16_t>(max(m & 0xffffu, m >> 16)))) & 0x7fffffffu;
  } else {
#pragma unroll
    for (int k = 0; k < kPer; ++k) {
      v[k] = __uint_as_float(r.w[k]);
      m = max(m, r.w[k] & 0x7fffffffu);
    }
    return m;
  }
}

struct QuantParams {
  const void* X;
  int64_t cols, ldx, x_rows;
  int rows, lt;
  const int32_t* row_index;
  const int32_t* offsets;
  int n_groups;
  uint8_t* codes;
  uint8_t* scales;
  const float* amax;
  int64_t ld;
  void* values;
  int64_t ldv;
  int64_t n_sf;               // scale tiles of a tile row
  int wide_x, wide_v;         // X, values: every row starts on a 32-byte boundary
  uintptr_t x_begin, x_end;   // the bytes of X: no 16-byte block that leaves them is loaded whole
};

// VALUES: 0 none, 1 bf16, 2 fp32
template <typename T, int FORMAT, int VALUES>
__global__ void __launch_bounds__(kThreads)
quantize_kernel(const QuantParams p) {
  constexpr int kCols = sf_cols(FORMAT), kChunks = kCols / kPer;     // 4 or 8 threads to a row
  constexpr int kStep = kThreads / kChunks, kRows = kSfRows / kStep; // rows of one sweep, rows of a thread
  __shared__ __align__(16) uint8_t sf[kSfTileBytes];
  ptx::pdl_launch_dependents();                               // a product launched behind this may start on its weight
  const int n_sf = static_cast<int>(p.n_sf);
  const int v = blockIdx.x / n_sf;                            // tile row
  const int cx = blockIdx.x - v * n_sf;
  int first, count;
  rows_of_tile_row(p.offsets, p.n_groups, p.rows, p.lt, v, first, count);
  if (count <= 0) return;

  const int chunk = threadIdx.x % kChunks;
  const int64_t c0 = static_cast<int64_t>(cx) * kCols + chunk * kPer;
  const int n = static_cast<int>(p.cols - c0 < kPer ? (p.cols - c0 < 0 ? 0 : p.cols - c0) : kPer);   // columns here
  const T* X = static_cast<const T*>(p.X);
  Raw<T> raw[kRows];
#pragma unroll
  for (int i = 0; i < kRows; ++i) {
    const int r = i * kStep + threadIdx.x / kChunks;
    int64_t src = static_cast<int64_t>(first) + r;
    if (r < count && p.row_index != nullptr) {
      src = p.row_index[src];
      if (src < 0 || src >= p.x_rows) src = -1;
    }
    const T* at = X + src * p.ldx + c0;
    const uintptr_t a = reinterpret_cast<uintptr_t>(at);
    if (r >= count || src < 0 || n == 0) load16_narrow(at, 0, raw[i]);
    else if (n == kPer && p.wide_x) load16_aligned(at, raw[i]);
    else if (n == kPer && (a & ~uintptr_t(15)) >= p.x_begin && a + kPer * sizeof(T) + 15 < p.x_end) load16_shifted(at, raw[i]);
    else load16_narrow(at, n, raw[i]);
  }
  const int t_log2 = FORMAT == ADADIM_NVFP4 ? tensor_scale_log2(p.amax) : 0;
#pragma unroll
  for (int i = 0; i < kRows; ++i) {
    const int r = i * kStep + threadIdx.x / kChunks;
    const int64_t row = static_cast<int64_t>(first) + r;
    float x[kPer];
    uint32_t top = widen(raw[i], x);
    if (FORMAT == ADADIM_MXFP4) top = max(top, __shfl_xor_sync(0xffffffffu, top, 1));
    const BlockScale b = block_scale<FORMAT>(__uint_as_float(top), t_log2);
    uint2 c;
    c.x = codes8<FORMAT, sizeof(T) == 2>(x, b);
    c.y = codes8<FORMAT, sizeof(T) == 2>(x + 8, b);
    const bool live = r < count && n > 0;
    const int blk = chunk * kPer / block_of(FORMAT);
    if (FORMAT == ADADIM_NVFP4 || (chunk & 1) == 0)           // 0 behind the last row and column
      sf[(r % 32) * 16 + (r / 32) * 4 + blk] = static_cast<uint8_t>(live ? b.byte : 0u);
    if (!live) continue;
    *reinterpret_cast<uint2*>(p.codes + row * p.ld + c0 / 2) = c;
    if (VALUES != 0) {
      const float s = b.finite ? b.s : __uint_as_float(0x7fffffffu);
      float q[kPer];
      e2m1_values8(c.x, *reinterpret_cast<float(*)[8]>(q));
      e2m1_values8(c.y, *reinterpret_cast<float(*)[8]>(q + 8));
#pragma unroll
      for (int k = 0; k < kPer; ++k) q[k] *= s;
      if (VALUES == 1) {
        __nv_bfloat16* out = static_cast<__nv_bfloat16*>(p.values) + row * p.ldv + c0;
        if (n == kPer && p.wide_v) {
          uint32_t w[8];
#pragma unroll
          for (int k = 0; k < 8; ++k) {
            const __nv_bfloat162 h = __floats2bfloat162_rn(q[2 * k], q[2 * k + 1]);
            w[k] = *reinterpret_cast<const uint32_t*>(&h);
          }
          store32(out, w);
        } else {
#pragma unroll
          for (int k = 0; k < kPer; ++k) if (k < n) out[k] = __float2bfloat16_rn(q[k]);
        }
      } else {
        float* out = static_cast<float*>(p.values) + row * p.ldv + c0;
        if (n == kPer && p.wide_v) {
          store32(out, reinterpret_cast<const uint32_t*>(q));
          store32(out + 8, reinterpret_cast<const uint32_t*>(q) + 8);
        } else {
#pragma unroll
          for (int k = 0; k < kPer; ++k) if (k < n) out[k] = q[k];
        }
      }
    }
  }
  __syncthreads();
  if (threadIdx.x < kSfTileBytes / 16)
    reinterpret_cast<uint4*>(p.scales + static_cast<int64_t>(blockIdx.x) * kSfTileBytes)[threadIdx.x] =
        reinterpret_cast<const uint4*>(sf)[threadIdx.x];
}

template <typename T>
__global__ void __launch_bounds__(256)
absmax_kernel(const T* __restrict__ X, int64_t rows, int64_t cols, int64_t ldx, int wide, float* amax) {
  constexpr int kVec = 16 / sizeof(T);
  uint32_t top = 0;
  const int64_t per_row = (cols + kVec - 1) / kVec, total = rows * per_row;
  for (int64_t i = static_cast<int64_t>(blockIdx.x) * 256 + threadIdx.x; i < total; i += static_cast<int64_t>(gridDim.x) * 256) {
    const int64_t r = i / per_row, c = (i - r * per_row) * kVec;
    const T* p = X + r * ldx + c;
    if (wide && c + kVec <= cols) {
      const uint4 raw = __ldg(reinterpret_cast<const uint4*>(p));
      const uint32_t w[4] = {raw.x, raw.y, raw.z, raw.w};
      if constexpr (sizeof(T) == 2) {
        uint32_t m = 0;
#pragma unroll
        for (int k = 0; k < 4; ++k) m = __vmaxu2(m, w[k] & 0x7fff7fffu);
        top = max(top, __float_as_uint(Elem<T>::to_f32(static_cast<uint16_t>(max(m & 0xffffu, m >> 16)))) & 0x7fffffffu);
      } else {
#pragma unroll
        for (int k = 0; k < 4; ++k) top = max(top, w[k] & 0x7fffffffu);
      }
    } else {
      for (int k = 0; k < kVec && c + k < cols; ++k) {
        if constexpr (sizeof(T) == 2) {
          top = max(top, __float_as_uint(Elem<T>::to_f32(reinterpret_cast<const uint16_t*>(p)[k])) & 0x7fffffffu);
        } else {
          top = max(top, reinterpret_cast<const uint32_t*>(p)[k] & 0x7fffffffu);
        }
      }
    }
  }
  top = __reduce_max_sync(0xffffffffu, top);
  // patterns of non-negative floats are ordered as unsigned integers: the result has no order to depend on
  if ((threadIdx.x & 31) == 0 && top != 0) atomicMax(reinterpret_cast<unsigned int*>(amax), top);
}

template <typename T, int FORMAT>
void launch_values(const QuantParams& p, int vsel, dim3 grid, cudaStream_t st) {
  if (vsel == 0) quantize_kernel<T, FORMAT, 0><<<grid, kThreads, 0, st>>>(p);
  else if (vsel == 1) quantize_kernel<T, FORMAT, 1><<<grid, kThreads, 0, st>>>(p);
  else quantize_kernel<T, FORMAT, 2><<<grid, kThreads, 0, st>>>(p);
}
template <typename T>
void launch_format(const QuantParams& p, int format, int vsel, dim3 grid, cudaStream_t st) {
  if (format == ADADIM_MXFP4) launch_values<T, ADADIM_MXFP4>(p, vsel, grid, st);
  else launch_values<T, ADADIM_NVFP4>(p, vsel, grid, st);
}

}  // namespace

int absmax_launch(const void* X, int xdtype, int64_t rows, int64_t cols, int64_t ldx, float* amax, cudaStream_t st) {
  const int64_t esz = xdtype == ADADIM_F32 ? 4 : 2;
  const int wide = aligned16(X) && (ldx * esz) % 16 == 0;
  const int64_t vecs = rows * ((cols * esz + 15) / 16);
  const unsigned grid = static_cast<unsigned>(vecs / 256 + 1 < 148 * 8 ? vecs / 256 + 1 : 148 * 8);
  if (xdtype == ADADIM_F32) absmax_kernel<float><<<grid, 256, 0, st>>>(static_cast<const float*>(X), rows, cols, ldx, wide, amax);
  else if (xdtype == ADADIM_F16) absmax_kernel<__half><<<grid, 256, 0, st>>>(static_cast<const __half*>(X), rows, cols, ldx, wide, amax);
  else absmax_kernel<__nv_bfloat16><<<grid, 256, 0, st>>>(static_cast<const __nv_bfloat16*>(X), rows, cols, ldx, wide, amax);
  return cudaGetLastError() == cudaSuccess ? ADADIM_OK : ADADIM_ERR_CUDA;
}

int quantize_fp4_launch(const void* X, int xdtype, int64_t rows, int64_t cols, int64_t ldx, int64_t x_rows, int format,
                        const int32_t* row_index, const int32_t* offsets, int n_groups, const adadim_fp4tensor& q,
                        int lt, void* values, int vdtype, int64_t ldv, cudaStream_t st) {
  const int64_t esz = xdtype == ADADIM_F32 ? 4 : 2, vsz = vdtype == ADADIM_F32 ? 4 : 2;
  QuantParams p = {};
  p.X = X;
  p.cols = cols;
  p.ldx = ldx;
  p.x_rows = x_rows;
  p.rows = static_cast<int>(rows);
  p.lt = lt;
  p.row_index = row_index;
  p.offsets = offsets;
  p.n_groups = n_groups;
  p.codes = q.codes;
  p.scales = q.scales;
  p.amax = q.amax;
  p.ld = q.ld;
  p.values = values;
  p.ldv = ldv;
  p.n_sf = sf_tiles(format, cols);
  const uintptr_t x0 = reinterpret_cast<uintptr_t>(X);
  p.wide_x = x0 % 32 == 0 && (ldx * esz) % 32 == 0;
  p.wide_v = values != nullptr && reinterpret_cast<uintptr_t>(values) % 32 == 0 && (ldv * vsz) % 32 == 0;
  p.x_begin = x0;
  p.x_end = x0 + static_cast<uintptr_t>(((x_rows - 1) * ldx + cols) * esz);
  const dim3 grid(static_cast<unsigned>(p.n_sf * sf_tile_rows(rows, n_groups, lt)));
  const int vsel = values == nullptr ? 0 : vdtype == ADADIM_BF16 ? 1 : 2;
  if (xdtype == ADADIM_F32) launch_format<float>(p, format, vsel, grid, st);
  else if (xdtype == ADADIM_F16) launch_format<__half>(p, format, vsel, grid, st);
  else launch_format<__nv_bfloat16>(p, format, vsel, grid, st);
  return cudaGetLastError() == cudaSuccess ? ADADIM_OK : ADADIM_ERR_CUDA;
}

}  // namespace adadim
