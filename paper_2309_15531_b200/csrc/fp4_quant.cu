// Microscaled 4-bit quantizer and the largest magnitude its tensor scale is taken from.
//
// Both are bound by memory.  Quantizer: a CTA owns 128 rows x 256 columns, that is 4 (NVFP4) or 2
// (MXFP4) whole scale tiles, so the scales of a tile are gathered in shared memory and leave as one
// contiguous run although a row's scales lie 512 bytes apart; a thread takes 16 consecutive columns
// (one NVFP4 block, half an MXFP4 block: the halves meet in one shuffle), which makes its codes one
// 8-byte store.  Work per element is a few instructions: packed magnitude maximum on the integer
// patterns (an infinity or NaN stays on top), one correctly rounded quotient (three operations against
// the block's reciprocal; MXFP4 one multiplication by a power of two), and the hardware
// conversion of pairs to E2M1.
#include "fp4.cuh"
#include "umma.cuh"

namespace adadim {
namespace {

using namespace fp4;

constexpr int kThreads = 256;
constexpr int kCols = 256;                   // columns of a CTA
constexpr int kPer = 16;                     // columns of a thread
constexpr int kRowsAtOnce = kThreads / (kCols / kPer);

// ---- loads: 16 elements widened to binary32, magnitudes' maximum as a binary32 pattern -----------------
template <typename T> struct Elem;
template <> struct Elem<__half> {
  static __device__ __forceinline__ float to_f32(uint16_t b) { return __half2float(__ushort_as_half(b)); }
};
template <> struct Elem<__nv_bfloat16> {
  static __device__ __forceinline__ float to_f32(uint16_t b) { return __uint_as_float(static_cast<uint32_t>(b) << 16); }
};

template <typename T>
__device__ __forceinline__ void load16_wide(const T* p, float (&v)[kPer], uint32_t& top) {
  if constexpr (sizeof(T) == 2) {
    uint4 raw[2] = {__ldg(reinterpret_cast<const uint4*>(p)), __ldg(reinterpret_cast<const uint4*>(p) + 1)};
    const uint32_t* w = reinterpret_cast<const uint32_t*>(raw);
    uint32_t m = 0;
#pragma unroll
    for (int k = 0; k < 8; ++k) {
      m = __vmaxu2(m, w[k] & 0x7fff7fffu);
      v[2 * k] = Elem<T>::to_f32(static_cast<uint16_t>(w[k] & 0xffffu));
      v[2 * k + 1] = Elem<T>::to_f32(static_cast<uint16_t>(w[k] >> 16));
    }
    const uint32_t h = max(m & 0xffffu, m >> 16);
    top = __float_as_uint(Elem<T>::to_f32(static_cast<uint16_t>(h))) & 0x7fffffffu;
  } else {
    uint32_t m = 0;
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const float4 a = __ldg(reinterpret_cast<const float4*>(p) + k);
      v[4 * k] = a.x; v[4 * k + 1] = a.y; v[4 * k + 2] = a.z; v[4 * k + 3] = a.w;
    }
#pragma unroll
    for (int k = 0; k < kPer; ++k) m = max(m, __float_as_uint(v[k]) & 0x7fffffffu);
    top = m;
  }
}
template <typename T>
__device__ __forceinline__ float load1(const T* p) {
  if constexpr (sizeof(T) == 2) return Elem<T>::to_f32(*reinterpret_cast<const uint16_t*>(p));
  else return *p;
}
template <typename T>
__device__ __forceinline__ void load16_narrow(const T* p, int n, float (&v)[kPer], uint32_t& top) {
  top = 0;
#pragma unroll
  for (int k = 0; k < kPer; ++k) {
    v[k] = k < n ? load1(p + k) : 0.0f;
    top = max(top, __float_as_uint(v[k]) & 0x7fffffffu);
  }
}

struct QuantParams {
  const void* X;
  int64_t cols, ldx, x_rows;
  int rows;
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
  int wide_x, wide_v;         // X, values: every row starts on a 16-byte boundary
};

// VALUES: 0 none, 1 bf16, 2 fp32
template <typename T, int FORMAT, int VALUES>
__global__ void __launch_bounds__(kThreads)
quantize_kernel(const QuantParams p) {
  constexpr int kTiles = kCols / sf_cols(FORMAT);
  __shared__ __align__(16) uint8_t sf[kTiles * kSfTileBytes];
  ptx::pdl_launch_dependents();                               // a product launched behind this may start on its weight
  const int col_ctas = static_cast<int>((p.cols + kCols - 1) / kCols);
  const int v = blockIdx.x / col_ctas;                        // tile row
  const int cx = blockIdx.x - v * col_ctas;
  int first = v * kSfRows, count = min(kSfRows, p.rows - first);
  if (p.offsets != nullptr) rows_of_tile_row(p.offsets, p.n_groups, p.rows, v, first, count);
  if (count <= 0) return;
  for (int k = threadIdx.x; k < kTiles * kSfTileBytes / 4; k += kThreads) reinterpret_cast<uint32_t*>(sf)[k] = 0;
  __syncthreads();

  const int t_log2 = FORMAT == ADADIM_NVFP4 ? tensor_scale_log2(p.amax) : 0;
  const int chunk = threadIdx.x % (kCols / kPer);
  const int64_t c0 = static_cast<int64_t>(cx) * kCols + chunk * kPer;
  const int n = static_cast<int>(p.cols - c0 < kPer ? (p.cols - c0 < 0 ? 0 : p.cols - c0) : kPer);   // columns here
  const T* X = static_cast<const T*>(p.X);
  for (int r = threadIdx.x / (kCols / kPer); r < kSfRows; r += kRowsAtOnce) {
    // whole warps take the same two rows, so the shuffle below always finds its partner
    const bool live = r < count;
    if (__all_sync(0xffffffffu, !live)) break;
    float x[kPer];
    uint32_t top = 0;
    const int64_t row = static_cast<int64_t>(first) + r;
    int64_t src = row;
    if (live && p.row_index != nullptr) {
      src = p.row_index[row];
      if (src < 0 || src >= p.x_rows) src = -1;
    }
    if (live && n == kPer && p.wide_x && src >= 0) load16_wide(X + src * p.ldx + c0, x, top);
    else load16_narrow(X + src * p.ldx + c0, live && src >= 0 ? n : 0, x, top);
    if (FORMAT == ADADIM_MXFP4) top = max(top, __shfl_xor_sync(0xffffffffu, top, 1));
    const BlockScale b = block_scale<FORMAT>(__uint_as_float(top), t_log2);
    uint2 c;
    c.x = codes8<FORMAT, sizeof(T) == 2>(x, b);
    c.y = codes8<FORMAT, sizeof(T) == 2>(x + 8, b);
    if (!live || n == 0) continue;
    *reinterpret_cast<uint2*>(p.codes + row * p.ld + c0 / 2) = c;
    const int blk = chunk * kPer / block_of(FORMAT);
    if (FORMAT == ADADIM_NVFP4 || (chunk & 1) == 0)
      sf[(blk / 4) * kSfTileBytes + (r % 32) * 16 + (r / 32) * 4 + blk % 4] = static_cast<uint8_t>(b.byte);
    if (VALUES != 0) {
      const float s = b.finite ? b.s : __uint_as_float(0x7fffffffu);
      float q[kPer];
#pragma unroll
      for (int k = 0; k < kPer; ++k) q[k] = e2m1_value((k < 8 ? c.x : c.y) >> (4 * (k & 7)) & 15u) * s;
      if (VALUES == 1) {
        __nv_bfloat16* out = static_cast<__nv_bfloat16*>(p.values) + row * p.ldv + c0;
        if (n == kPer && p.wide_v) {
          uint32_t w[8];
#pragma unroll
          for (int k = 0; k < 8; ++k) {
            const __nv_bfloat162 h = __floats2bfloat162_rn(q[2 * k], q[2 * k + 1]);
            w[k] = *reinterpret_cast<const uint32_t*>(&h);
          }
          reinterpret_cast<uint4*>(out)[0] = make_uint4(w[0], w[1], w[2], w[3]);
          reinterpret_cast<uint4*>(out)[1] = make_uint4(w[4], w[5], w[6], w[7]);
        } else {
#pragma unroll
          for (int k = 0; k < kPer; ++k) if (k < n) out[k] = __float2bfloat16_rn(q[k]);
        }
      } else {
        float* out = static_cast<float*>(p.values) + row * p.ldv + c0;
        if (n == kPer && p.wide_v) {
#pragma unroll
          for (int k = 0; k < 4; ++k) reinterpret_cast<float4*>(out)[k] = make_float4(q[4 * k], q[4 * k + 1], q[4 * k + 2], q[4 * k + 3]);
        } else {
#pragma unroll
          for (int k = 0; k < kPer; ++k) if (k < n) out[k] = q[k];
        }
      }
    }
  }
  __syncthreads();
  // the tiles of this CTA's columns; the last CTA of a row may have fewer
  const int64_t t0 = static_cast<int64_t>(cx) * kTiles;
  const int nt = static_cast<int>(p.n_sf - t0 < kTiles ? p.n_sf - t0 : kTiles);
  uint4* dst = reinterpret_cast<uint4*>(p.scales + (v * p.n_sf + t0) * kSfTileBytes);
  for (int k = threadIdx.x; k < nt * (kSfTileBytes / 16); k += kThreads) dst[k] = reinterpret_cast<const uint4*>(sf)[k];
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
      for (int k = 0; k < kVec && c + k < cols; ++k) top = max(top, __float_as_uint(load1(p + k)) & 0x7fffffffu);
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
                        void* values, int vdtype, int64_t ldv, cudaStream_t st) {
  const int64_t esz = xdtype == ADADIM_F32 ? 4 : 2, vsz = vdtype == ADADIM_F32 ? 4 : 2;
  QuantParams p = {};
  p.X = X;
  p.cols = cols;
  p.ldx = ldx;
  p.x_rows = x_rows;
  p.rows = static_cast<int>(rows);
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
  p.wide_x = aligned16(X) && (ldx * esz) % 16 == 0;
  p.wide_v = values != nullptr && aligned16(values) && (ldv * vsz) % 16 == 0;
  const dim3 grid(static_cast<unsigned>((cols + kCols - 1) / kCols * sf_tile_rows(rows, n_groups)));
  const int vsel = values == nullptr ? 0 : vdtype == ADADIM_BF16 ? 1 : 2;
  if (xdtype == ADADIM_F32) launch_format<float>(p, format, vsel, grid, st);
  else if (xdtype == ADADIM_F16) launch_format<__half>(p, format, vsel, grid, st);
  else launch_format<__nv_bfloat16>(p, format, vsel, grid, st);
  return cudaGetLastError() == cudaSuccess ? ADADIM_OK : ADADIM_ERR_CUDA;
}

}  // namespace adadim
