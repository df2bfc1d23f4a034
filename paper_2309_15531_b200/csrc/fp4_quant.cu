// Microscaled 4-bit quantizer and the largest magnitude its tensor scale is taken from.
//
// Both are bound by memory.  Quantizer: a CTA owns one scale tile, 128 rows x 64 (NVFP4) or 128 (MXFP4)
// columns (for token tiles of 16, 32 or 64 rows up to 128 / rows tiles side by side), so the scales leave as
// one contiguous run although a row's scales lie 512 bytes apart.  A thread takes 16 consecutive columns (one
// NVFP4 block, half an MXFP4 block: the halves meet in one shuffle) of 4 or 8 rows, the loads of four of them
// issued before the first is used; its codes are one 8-byte store.  What it executes matters as much as what
// it moves (24 instructions an element were the limit at 39 us for W[11008,4096] with its values): packed
// magnitude maximum, packed binary32 for the quotients, hardware conversions to and from E2M1.
#include "fp4.cuh"
#include "umma_fp4.cuh"

namespace adadim {
namespace {

using namespace fp4;

// How the work is laid out, by the number of CTAs (one to a scale tile):
//   kMany  128 threads, a thread takes 4 or 8 rows, the loads of four in flight together (with 8, MXFP4 with few
//          CTAs makes two dependent round trips to memory)
//   kLow   the same for a product's low token tiles, which may lie side by side in a CTA, and for up to kLowCtas
//          CTAs in front of a product: with the SM's shared memory left to the product (see the launcher)
//   kFew   up to kFewCtas: 512 threads with one or two rows each, to have something to hide the latencies behind
// Measured on one size on each side of the bound, with the data in L2: 333 x 5003 fp32, 237 CTAs, 13.4 us as kMany and
// 7.4 us as kFew; 2048 x 4096 bf16 to MXFP4, 512 CTAs, 6.8 us as kMany and 7.8 us as kFew (from DRAM 9.7 us as kMany).
// Times are the best of a graph's replays; sustained from Python W[11008,4096] with its values takes 36.9 us (35.2), 333 x
// 5003 8.2 us (7.1).  Codes only: W[11008,4096] 23.2 us to NVFP4 (floor 17.6), 22.1 us to MXFP4; 2048 x 4096 7.5 and 8.4 us.
enum Mode { kMany, kLow, kFew };
constexpr int kFewCtas = 2 * 148, kLowCtas = 4 * 148;
template <Mode MODE>
constexpr int kThreadsOf = MODE == kFew ? 512 : 128;

__device__ __forceinline__ void store32(void* p, const uint32_t* w) {           // 32-byte aligned
  asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};"
               ::"l"(p), "r"(w[0]), "r"(w[1]), "r"(w[2]), "r"(w[3]), "r"(w[4]), "r"(w[5]), "r"(w[6]), "r"(w[7]) : "memory");
}

// Sixteen values to any address: up to the next 16-byte boundary one by one, then whole 16-byte blocks.
__device__ __forceinline__ void store16_shifted(float* out, const float (&q)[kPer]) {
  const int head = static_cast<int>((16u - (static_cast<uint32_t>(reinterpret_cast<uintptr_t>(out)) & 15u)) >> 2) & 3;
  float r[kPer + 2];                                          // q from `head` on
#pragma unroll
  for (int k = 0; k < kPer; ++k) r[k] = head & 1 ? q[k + 1 < kPer ? k + 1 : k] : q[k];
#pragma unroll
  for (int k = 0; k < kPer; ++k) if (head & 2) r[k] = r[k + 2 < kPer ? k + 2 : k];
#pragma unroll
  for (int k = 0; k < 3; ++k) if (k < head) out[k] = q[k];
  float4* block = reinterpret_cast<float4*>(out + head);
#pragma unroll
  for (int k = 0; k < 3; ++k) block[k] = make_float4(r[4 * k], r[4 * k + 1], r[4 * k + 2], r[4 * k + 3]);
  if (head == 0) {
    block[3] = make_float4(q[12], q[13], q[14], q[15]);
  } else {
#pragma unroll
    for (int k = 0; k < 3; ++k) if (k < 4 - head) out[head + 12 + k] = r[12 + k];
  }
}
// The same for bf16 patterns, with 4-byte blocks.
__device__ __forceinline__ void store16_shifted(__nv_bfloat16* out, const uint16_t (&h)[kPer]) {
  uint16_t* o = reinterpret_cast<uint16_t*>(out);
  if (reinterpret_cast<uintptr_t>(out) & 2u) {
    o[0] = h[0];
#pragma unroll
    for (int k = 1; k < kPer - 1; k += 2) *reinterpret_cast<uint32_t*>(o + k) = h[k] | static_cast<uint32_t>(h[k + 1]) << 16;
    o[kPer - 1] = h[kPer - 1];
  } else {
#pragma unroll
    for (int k = 0; k < kPer; k += 2) *reinterpret_cast<uint32_t*>(o + k) = h[k] | static_cast<uint32_t>(h[k + 1]) << 16;
  }
}

// 160 bytes: with 168 a launch took the host 0.25 us longer.
struct QuantParams {
  Source x;
  int64_t cols;
  int rows, lt;
  int side;                   // tiles side by side in a CTA, a power of two, at most 128 / lt
  int n_groups;
  const int32_t* offsets;
  uint8_t* codes;
  uint8_t* scales;
  const float* amax;
  float* kept;                // a copy of it that stays with the codes, NULL: none
  int64_t ld;
  void* values;
  int64_t ldv;
  int64_t n_sf;               // scale tiles of a tile row
  int wide_v;                 // values: every row starts on a 32-byte boundary
};

// CTAs of an SM that the registers must leave room for: the loads in flight are what hides the memory's latency
template <typename T, Mode MODE>
constexpr int kResident = MODE == kFew ? 2 : sizeof(T) == 4 ? 5 : 8;

// VALUES: 0 none, 1 bf16, 2 fp32
template <typename T, int FORMAT, int VALUES, Mode MODE>
__global__ void __launch_bounds__(kThreadsOf<MODE>, kResident<T, MODE>)
quantize_kernel(const QuantParams p) {
  constexpr int kThreads = kThreadsOf<MODE>;
  constexpr int kChunks = sf_cols(FORMAT) / kPer;             // threads to a row of a tile: 4 or 8
  constexpr int kRows = kSfRows * kChunks / kThreads;         // rows of a thread: 4 or 8, kFew 1 or 2
  constexpr int kBatch = kRows < 4 ? kRows : 4;
  extern __shared__ __align__(16) uint8_t sf[];               // [side][kSfTileBytes]
  ptx::pdl_launch_dependents();                               // a product launched behind this may start on its weight
  if (FORMAT == ADADIM_NVFP4 && p.kept != nullptr && blockIdx.x == 0 && threadIdx.x == 0) *p.kept = *p.amax;
  const int side = MODE == kLow ? p.side : 1;
  const int n_sf = static_cast<int>(p.n_sf), ctas = MODE == kLow ? (n_sf + side - 1) / side : n_sf;
  const int v = blockIdx.x / ctas;                            // tile row
  const int tile0 = (blockIdx.x - v * ctas) * side;           // first of the tiles side by side
  int first, count;
  rows_of_tile_row(p.offsets, p.n_groups, p.rows, p.lt, v, first, count);
  if (count <= 0) return;

  const int wide = kChunks * side, shift = __ffs(wide) - 1;   // threads to a row, a power of two
  const int chunk = threadIdx.x & (wide - 1), row0 = threadIdx.x >> shift, row_step = kThreads >> shift;
  const int64_t c0 = (static_cast<int64_t>(tile0) * kChunks + chunk) * kPer;
  const int n = static_cast<int>(p.cols - c0 < kPer ? (p.cols - c0 < 0 ? 0 : p.cols - c0) : kPer);   // columns here
  const int t_log2 = FORMAT == ADADIM_NVFP4 ? tensor_scale_log2(p.amax) : 0;
  const int blk = chunk * kPer / block_of(FORMAT);
  uint8_t* sf_at = sf + (blk / 4) * kSfTileBytes + blk % 4;
  uint8_t* codes = p.codes + static_cast<int64_t>(first) * p.ld + c0 / 2;
#pragma unroll 1
  for (int r1 = row0; r1 - row0 < kRows * row_step && r1 - row0 < count; r1 += kBatch * row_step) {
    Raw<T> raw[kBatch];
#pragma unroll
    for (int i = 0; i < kBatch; ++i) {
      const int r = r1 + i * row_step;
      const int64_t src = r < count ? source_row(p.x, static_cast<int64_t>(first) + r) : -1;
      load16(p.x, src, c0, n, raw[i]);
    }
#pragma unroll
    for (int i = 0; i < kBatch; ++i) {
      const int r = r1 + i * row_step;
      float x[kPer];
      uint32_t top = widen(raw[i], x);
      if (FORMAT == ADADIM_MXFP4) top = max(top, __shfl_xor_sync(0xffffffffu, top, 1));
      const BlockScale b = block_scale<FORMAT, sizeof(T) == 2>(__uint_as_float(top), t_log2);
      uint2 c;
      c.x = codes8<FORMAT, sizeof(T) == 2>(x, b);
      c.y = codes8<FORMAT, sizeof(T) == 2>(x + 8, b);
      const bool live = r < count && n > 0;
      if (FORMAT == ADADIM_NVFP4 || (chunk & 1) == 0)         // 0 behind the last row and column
        sf_at[(r & 31) * 16 + (r >> 5) * 4] = static_cast<uint8_t>(live ? b.byte : 0u);
      if (!live) continue;
      *reinterpret_cast<uint2*>(codes + r * p.ld) = c;
      if (VALUES != 0) {
        const int64_t row = static_cast<int64_t>(first) + r;
        const float s = b.finite ? b.s : __uint_as_float(0x7fffffffu);
        float q[kPer];
        e2m1_values8(c.x, *reinterpret_cast<float(*)[8]>(q));
        e2m1_values8(c.y, *reinterpret_cast<float(*)[8]>(q + 8));
        const uint64_t s2 = pack2(s, s);
#pragma unroll
        for (int k = 0; k < kPer; k += 2) unpack2(mul2(pack2(q[k], q[k + 1]), s2), q[k], q[k + 1]);
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
          } else if (n == kPer) {
            uint16_t h[kPer];
#pragma unroll
            for (int k = 0; k < kPer; ++k) h[k] = __bfloat16_as_ushort(__float2bfloat16_rn(q[k]));
            store16_shifted(out, h);
          } else {
#pragma unroll
            for (int k = 0; k < kPer; ++k) if (k < n) out[k] = __float2bfloat16_rn(q[k]);
          }
        } else {
          float* out = static_cast<float*>(p.values) + row * p.ldv + c0;
          if (n == kPer && p.wide_v) {
            store32(out, reinterpret_cast<const uint32_t*>(q));
            store32(out + 8, reinterpret_cast<const uint32_t*>(q) + 8);
          } else if (n == kPer) {
            store16_shifted(out, q);
          } else {
#pragma unroll
            for (int k = 0; k < kPer; ++k) if (k < n) out[k] = q[k];
          }
        }
      }
    }
  }
  // rows of a public (128-row) tile that no sweep reached
  if (p.lt % kSfRows == 0)
    for (int r = row0; r < kSfRows; r += row_step)
      if (r >= count && (FORMAT == ADADIM_NVFP4 || (chunk & 1) == 0)) sf_at[(r & 31) * 16 + (r >> 5) * 4] = 0;
  __syncthreads();
  // (in a token tile lower than 128 the places of the rows it does not have hold anything: nobody reads them)
  const int tiles = min(p.side, n_sf - tile0);
  uint4* dst = reinterpret_cast<uint4*>(p.scales + (static_cast<int64_t>(v) * n_sf + tile0) * kSfTileBytes);
  for (int k = threadIdx.x; k < tiles * (kSfTileBytes / 16); k += kThreads) dst[k] = reinterpret_cast<const uint4*>(sf)[k];
}

// Segments of a row (of the whole matrix where its rows follow one another), four 16-byte loads of a thread in flight;
// one atomic per CTA.  Bound by memory: 8192 x 8192 bf16 21.6 us, 6220 GB/s (with a division for every load: 31.4 us).
// Rows that do not start on 16-byte boundaries are read element by element (3333 x 5003 fp32 13.7 us, 4870 GB/s, 0.74 of
// the copy rate), and of a row shorter than a segment the other threads are idle (200000 x 50 bf16 119 us).
constexpr int kMaxThreads = 256, kMaxLoads = 4;
template <typename T>
constexpr int kSegment = kMaxThreads * kMaxLoads * 16 / static_cast<int>(sizeof(T));
template <typename T>
__device__ __forceinline__ uint32_t magnitude(const uint4& raw) {
  const uint32_t w[4] = {raw.x, raw.y, raw.z, raw.w};
  if constexpr (sizeof(T) == 2) {
    typename Elem<T>::Two m = Elem<T>::abs2(w[0]);
#pragma unroll
    for (int k = 1; k < 4; ++k) m = __hmax2_nan(m, Elem<T>::abs2(w[k]));
    return __float_as_uint(Elem<T>::top_f32(m)) & 0x7fffffffu;
  } else {
    return max(max(w[0] & 0x7fffffffu, w[1] & 0x7fffffffu), max(w[2] & 0x7fffffffu, w[3] & 0x7fffffffu));
  }
}
template <typename T>
__device__ __forceinline__ uint32_t magnitude(const T* p) {
  if constexpr (sizeof(T) == 2) return __float_as_uint(Elem<T>::to_f32(*reinterpret_cast<const uint16_t*>(p))) & 0x7fffffffu;
  else return *reinterpret_cast<const uint32_t*>(p) & 0x7fffffffu;
}
template <typename T>
__global__ void __launch_bounds__(kMaxThreads)
absmax_kernel(const T* __restrict__ X, int64_t rows, int64_t cols, int64_t ldx, int wide, float* amax) {
  constexpr int kVec = 16 / sizeof(T);
  __shared__ uint32_t tops[kMaxThreads / 32];
  const int64_t segments = (cols + kSegment<T> - 1) / kSegment<T>, total = rows * segments;
  uint32_t top = 0;
  for (int64_t i = blockIdx.x; i < total; i += gridDim.x) {
    const int64_t r = segments == 1 ? i : i / segments, c0 = (i - r * segments) * kSegment<T>;
    const int n = static_cast<int>(cols - c0 < kSegment<T> ? cols - c0 : kSegment<T>);
    const T* p = X + r * ldx + c0;
    int done = 0;
    if (wide) {
      uint4 raw[kMaxLoads];
#pragma unroll
      for (int k = 0; k < kMaxLoads; ++k) {
        const int at = (k * kMaxThreads + threadIdx.x) * kVec;
        raw[k] = at + kVec <= n ? __ldg(reinterpret_cast<const uint4*>(p + at)) : make_uint4(0, 0, 0, 0);
      }
#pragma unroll
      for (int k = 0; k < kMaxLoads; ++k) top = max(top, magnitude<T>(raw[k]));
      done = n / kVec * kVec;
    }
#pragma unroll 4
    for (int at = done + threadIdx.x; at < n; at += kMaxThreads) top = max(top, magnitude<T>(p + at));
  }
  top = __reduce_max_sync(0xffffffffu, top);
  if ((threadIdx.x & 31) == 0) tops[threadIdx.x / 32] = top;
  __syncthreads();
  if (threadIdx.x < 32) {
    top = __reduce_max_sync(0xffffffffu, threadIdx.x < kMaxThreads / 32 ? tops[threadIdx.x] : 0u);
    // patterns of non-negative floats are ordered as unsigned integers: the result has no order to depend on
    if (threadIdx.x == 0 && top != 0) atomicMax(reinterpret_cast<unsigned int*>(amax), top);
  }
}

template <typename T, int FORMAT, int VALUES, Mode MODE>
int launch(const QuantParams& p, dim3 grid, cudaStream_t st) {
  // A product behind this kernel starts while this one runs and needs nearly all of an SM's shared memory:
  // if this kernel left the SM with a small share, the product would wait until the SM is empty.  Except with
  // many CTAs, where it would cost the cache that the loads in flight need, the share is therefore set to the most.
  if (VALUES == 0 && MODE != kMany) {
    static std::atomic<uint64_t> done{0};
    const int rc = set_once(quantize_kernel<T, FORMAT, VALUES, MODE>, cudaFuncAttributePreferredSharedMemoryCarveout,
                            cudaSharedmemCarveoutMaxShared, done);
    if (rc != ADADIM_OK) return rc;
  }
  quantize_kernel<T, FORMAT, VALUES, MODE><<<grid, kThreadsOf<MODE>, static_cast<size_t>(p.side) * kSfTileBytes, st>>>(p);
  return cudaGetLastError() == cudaSuccess ? ADADIM_OK : ADADIM_ERR_CUDA;
}
template <typename T, int FORMAT, int VALUES>
int launch_mode(const QuantParams& p, dim3 grid, cudaStream_t st) {
  if (VALUES == 0 && (p.side > 1 || (grid.x > kFewCtas && (p.lt < kSfRows || grid.x <= kLowCtas)))) return launch<T, FORMAT, VALUES, VALUES == 0 ? kLow : kMany>(p, grid, st);
  return grid.x <= kFewCtas ? launch<T, FORMAT, VALUES, kFew>(p, grid, st) : launch<T, FORMAT, VALUES, kMany>(p, grid, st);
}
template <typename T, int FORMAT>
int launch_values(const QuantParams& p, int vsel, dim3 grid, cudaStream_t st) {
  if (vsel == 0) return launch_mode<T, FORMAT, 0>(p, grid, st);
  return vsel == 1 ? launch_mode<T, FORMAT, 1>(p, grid, st) : launch_mode<T, FORMAT, 2>(p, grid, st);
}
template <typename T>
int launch_format(const QuantParams& p, int format, int vsel, dim3 grid, cudaStream_t st) {
  return format == ADADIM_MXFP4 ? launch_values<T, ADADIM_MXFP4>(p, vsel, grid, st) : launch_values<T, ADADIM_NVFP4>(p, vsel, grid, st);
}

}  // namespace

int absmax_launch(const void* X, int xdtype, int64_t rows, int64_t cols, int64_t ldx, float* amax, cudaStream_t st) {
  const int64_t esz = xdtype == ADADIM_F32 ? 4 : 2;
  if (ldx == cols || rows == 1) { cols *= rows; ldx = cols; rows = 1; }
  const int wide = aligned16(X) && (rows == 1 || (ldx * esz) % 16 == 0);
  const int64_t segment = esz == 4 ? kSegment<float> : kSegment<__half>;
  const int64_t segments = rows * ((cols + segment - 1) / segment);
  const unsigned grid = static_cast<unsigned>(segments < 148 * 8 ? segments : 148 * 8);
  if (xdtype == ADADIM_F32) absmax_kernel<float><<<grid, kMaxThreads, 0, st>>>(static_cast<const float*>(X), rows, cols, ldx, wide, amax);
  else if (xdtype == ADADIM_F16) absmax_kernel<__half><<<grid, kMaxThreads, 0, st>>>(static_cast<const __half*>(X), rows, cols, ldx, wide, amax);
  else absmax_kernel<__nv_bfloat16><<<grid, kMaxThreads, 0, st>>>(static_cast<const __nv_bfloat16*>(X), rows, cols, ldx, wide, amax);
  return cudaGetLastError() == cudaSuccess ? ADADIM_OK : ADADIM_ERR_CUDA;
}

int quantize_fp4_launch(const fp4::Source& x, int xdtype, int64_t rows, int64_t cols, int format, const int32_t* offsets,
                        int n_groups, const adadim_fp4tensor& q, const float* amax, int lt, void* values, int vdtype, int64_t ldv,
                        cudaStream_t st) {
  const int64_t vsz = vdtype == ADADIM_F32 ? 4 : 2;
  QuantParams p = {};
  p.x = x;
  p.cols = cols;
  p.rows = static_cast<int>(rows);
  p.lt = lt;
  p.offsets = offsets;
  p.n_groups = n_groups;
  p.codes = q.codes;
  p.scales = q.scales;
  p.amax = amax != nullptr ? amax : q.amax;
  p.kept = amax != nullptr && amax != q.amax ? const_cast<float*>(q.amax) : nullptr;
  p.ld = q.ld;
  p.values = values;
  p.ldv = ldv;
  p.n_sf = sf_tiles(format, cols);
  p.wide_v = values != nullptr && reinterpret_cast<uintptr_t>(values) % 32 == 0 && (ldv * vsz) % 32 == 0;
  // lt is 16, 32, 64 or a multiple of 128; low tiles go side by side as long as every SM still has a CTA
  const int64_t tile_rows = sf_tile_rows(rows, n_groups, lt);
  p.side = 1;
  while (p.side * 2 * lt <= kSfRows && tile_rows * (p.n_sf / (2 * p.side)) >= 148) p.side *= 2;
  const dim3 grid(static_cast<unsigned>((p.n_sf + p.side - 1) / p.side * tile_rows));
  const int vsel = values == nullptr ? 0 : vdtype == ADADIM_BF16 ? 1 : 2;
  if (xdtype == ADADIM_F32) return launch_format<float>(p, format, vsel, grid, st);
  return xdtype == ADADIM_F16 ? launch_format<__half>(p, format, vsel, grid, st) : launch_format<__nv_bfloat16>(p, format, vsel, grid, st);
}

}  // namespace adadim
