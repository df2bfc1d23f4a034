// Product of two microscaled 4-bit matrices on the block-scaled tensor-core path, plain and grouped
// by expert:  Y[t, o] = 2^(ta + tb) sum_k A[t, k] B[o, k],  scales applied by the matrix instruction.
//
// The weight is the instruction's M side (128 of its rows per tile) and the tokens its N side, in
// every case: N may be any multiple of 16, so one token, the ragged end of an expert's rows and a
// full tile all run without multiplying padding, and the accumulator of one weight row sits in one
// TMEM lane.  Both operands arrive by TMA as 256-column stages (128 bytes of codes per row,
// 128-byte swizzle) together with their scale tiles, which the issuing thread copies from shared
// memory to TMEM in front of the MMAs that use them.
#include "fp4.cuh"
#include "umma.cuh"

namespace adadim {
namespace {

using namespace fp4;

constexpr int kKT = 256;                               // columns of a stage
constexpr int kThreads = 192;                          // TMA warp, MMA warp, four epilogue warps
constexpr int kMaxStages = 8;
constexpr uint32_t kWBytes = 128 * 128;
constexpr int kBand = 8;                               // weight tiles that share a sweep over the tokens

struct MmParams {
  int64_t out, in;
  int rows;                                            // of A and Y
  int n_experts;                                       // 0: dense
  const int32_t* offsets;
  int m_tiles;                                         // 128-row tiles of one weight
  int n_tile;                                          // tokens of a tile (box height of A)
  int num_k;                                           // stages of a tile
  int n_stages;
  int64_t n_sf;                                        // scale tiles of a tile row
  int64_t w_sf_rows;                                   // scale tile rows of one weight
  void* Y;
  int ydtype;
  int64_t ldy;
  const float* a_amax;
  const float* b_amax;
  int* status_dev;
};

__host__ __device__ constexpr uint32_t sf_stage_bytes(int format) { return kKT / sf_cols(format) * kSfTileBytes; }
__host__ __device__ __forceinline__ uint32_t stage_bytes(int format, int n_tile) {
  return kWBytes + static_cast<uint32_t>(n_tile) * 128 + 2 * sf_stage_bytes(format);
}

// One output tile: 128 weight rows from `m` on, the `count` (<= n_tile) rows of A from `row` on.
struct Tile {
  int e, m, row, count;
  int64_t a_sf_row;                                    // scale tile row of A, and where in it the tile
  int a_sf_col;                                        // begins, in 32-row columns
};

// Tiles are numbered expert by expert; inside one, bands of kBand weight tiles sweep over the tokens,
// so that the CTAs at work at one time share both operands in L2.
__device__ __forceinline__ Tile tile_of(int t, const MmParams& p, const int* prefix) {
  Tile x;
  x.e = 0;
  int first = 0, n = p.rows;
  if (p.n_experts > 0) {
    int lo = 0, hi = p.n_experts - 1;                  // last e with prefix[e] <= t
    while (lo < hi) {
      const int mid = (lo + hi + 1) >> 1;
      if (prefix[mid] <= t) lo = mid; else hi = mid - 1;
    }
    x.e = lo;
    t -= prefix[lo];
    first = clamped(p.offsets[lo], p.rows);
    n = clamped(p.offsets[lo + 1], p.rows) - first;
  }
  const int n_tiles = (n + p.n_tile - 1) / p.n_tile;
  const int band = t / (kBand * n_tiles);
  const int in_band = t - band * kBand * n_tiles;
  const int width = min(kBand, p.m_tiles - band * kBand);
  const int j = in_band / width;
  x.m = (band * kBand + in_band - j * width) * 128;
  x.row = first + j * p.n_tile;
  x.count = min(p.n_tile, n - j * p.n_tile);
  x.a_sf_row = (p.n_experts > 0 ? first / kSfRows + x.e : 0) + j * p.n_tile / kSfRows;
  x.a_sf_col = j * p.n_tile % kSfRows / 32;            // several tiles only where n_tile is a multiple of 32
  return x;
}

__device__ __forceinline__ void store_y(void* Y, int ydtype, int64_t at, float v) {
  if (ydtype == ADADIM_BF16) static_cast<__nv_bfloat16*>(Y)[at] = __float2bfloat16_rn(v);
  else if (ydtype == ADADIM_F16) static_cast<__half*>(Y)[at] = __float2half_rn(v);
  else static_cast<float*>(Y)[at] = v;
}

template <int FORMAT>
__global__ void __launch_bounds__(kThreads, 1)
fp4_matmul_kernel(const __grid_constant__ CUtensorMap tmW, const __grid_constant__ CUtensorMap tmA,
                  const __grid_constant__ CUtensorMap tmWs, const __grid_constant__ CUtensorMap tmAs, const MmParams p) {
  constexpr bool NV = FORMAT == ADADIM_NVFP4;
  constexpr uint32_t kSf = sf_stage_bytes(FORMAT);
  constexpr int kSfTiles = kSf / kSfTileBytes;         // scale tiles of a stage: 4 or 2
  constexpr uint32_t kSfCol = 256;                     // TMEM: two accumulators of 128 columns, then scales

  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
  __shared__ uint64_t full[kMaxStages], empty[kMaxStages], acc_full[2], acc_empty[2], drain;
  __shared__ uint32_t tmem_slot;
  __shared__ int dead_word;
  __shared__ int prefix[kMaxGroups + 1];
  volatile int* dead = &dead_word;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  const uint32_t stage_size = stage_bytes(FORMAT, p.n_tile);

  if (threadIdx.x == 0) {
    for (int s = 0; s < p.n_stages; ++s) { ptx::mbar_init(&full[s], 1); ptx::mbar_init(&empty[s], 1); }
    for (int b = 0; b < 2; ++b) { ptx::mbar_init(&acc_full[b], 1); ptx::mbar_init(&acc_empty[b], 4); }
    ptx::mbar_init(&drain, 1);
    dead_word = 0;
    ptx::fence_mbar_init();
    ptx::tma_prefetch_desc(&tmW);
    ptx::tma_prefetch_desc(&tmA);
    ptx::tma_prefetch_desc(&tmWs);
    ptx::tma_prefetch_desc(&tmAs);
  }
  if (warp == 1) {
    ptx::tmem_alloc(&tmem_slot, 512);
    ptx::tmem_relinquish();
  }
  // tiles of each expert, then their running sum
  if (warp == 2 && p.n_experts > 0) {
    int sum = 0;
    for (int e0 = 0; e0 < p.n_experts; e0 += 32) {
      const int e = e0 + lane;
      int c = 0;
      if (e < p.n_experts) {
        const int a = p.offsets[e], z = p.offsets[e + 1];
        if (blockIdx.x == 0 && (a < 0 || z > p.rows || z < a)) report(p.status_dev, ADADIM_ERR_SHAPE);
        const int n = clamped(z, p.rows) - clamped(a, p.rows);
        c = n > 0 ? (n + p.n_tile - 1) / p.n_tile * p.m_tiles : 0;
      }
      int s = c;
#pragma unroll
      for (int d = 1; d < 32; d <<= 1) {
        const int o = __shfl_up_sync(0xffffffffu, s, d);
        if (lane >= d) s += o;
      }
      if (e < p.n_experts) prefix[e] = sum + s - c;
      sum += __shfl_sync(0xffffffffu, s, 31);
    }
    if (lane == 0) prefix[p.n_experts] = sum;
  }
  ptx::tc_fence_before_sync();
  __syncthreads();
  ptx::tc_fence_after_sync();
  const uint32_t tmem = tmem_slot;
  const int num_tiles = p.n_experts > 0 ? prefix[p.n_experts] : (p.rows + p.n_tile - 1) / p.n_tile * p.m_tiles;

  if (warp == 0) {
    // ------------------------------------------------------------------ TMA producer
    if (lane == 0) {
      int stage = 0;
      uint32_t phase = 0;
      int last_phase[kMaxStages];
      for (int s = 0; s < kMaxStages; ++s) last_phase[s] = -1;
      for (int t = blockIdx.x; t < num_tiles && !*dead; t += gridDim.x) {
        const Tile x = tile_of(t, p, prefix);
        const int w_row = static_cast<int>(x.e * p.out + x.m);
        const int64_t w_sf = (x.e * p.w_sf_rows + x.m / kSfRows) * p.n_sf, a_sf = x.a_sf_row * p.n_sf;
        for (int k = 0; k < p.num_k; ++k) {
          if (!ptx::mbar_wait(&empty[stage], phase ^ 1u, dead, p.status_dev)) break;
          uint8_t* w_dst = smem + stage * stage_size;
          uint8_t* a_dst = w_dst + kWBytes;
          uint8_t* ws_dst = a_dst + p.n_tile * 128;
          ptx::mbar_arrive_expect_tx(&full[stage], stage_size);
          last_phase[stage] = static_cast<int>(phase);
          ptx::tma_load_2d(w_dst, &tmW, k * (kKT / 2), w_row, &full[stage]);
          ptx::tma_load_2d(a_dst, &tmA, k * (kKT / 2), x.row, &full[stage]);
          ptx::tma_load_2d(ws_dst, &tmWs, 0, static_cast<int>((w_sf + k * kSfTiles) * 4), &full[stage]);
          ptx::tma_load_2d(ws_dst + kSf, &tmAs, 0, static_cast<int>((a_sf + k * kSfTiles) * 4), &full[stage]);
          if (++stage == p.n_stages) { stage = 0; phase ^= 1u; }
        }
      }
      if (*dead) {
        // a wait ran out somewhere: let the copies already issued land before shared memory goes away
        for (int s = 0; s < p.n_stages; ++s) {
          if (last_phase[s] < 0) continue;
          const long long t0 = clock64();
          while (!ptx::mbar_try_wait(&full[s], static_cast<uint32_t>(last_phase[s])) && clock64() - t0 < ptx::kWaitLimit) {}
        }
      }
    }
  } else if (warp == 1) {
    // ------------------------------------------------------------------ MMA issuer
    if (lane == 0) {
      constexpr uint64_t desc = ptx::smem_desc_sw128(16, 1024);        // K-major: 8-row groups 1024 bytes apart
      constexpr uint64_t sf_desc = ptx::smem_desc_plain(16, 128);
      int stage = 0, buf = 0;
      uint32_t phase = 0, acc_phase = 0;
      bool ok = true;
      for (int t = blockIdx.x; t < num_tiles && ok; t += gridDim.x) {
        const Tile x = tile_of(t, p, prefix);
        const int n = (x.count + 15) & ~15;
        const uint32_t id0 = ptx::idesc_fp4(128, n, !NV, 0), id1 = ptx::idesc_fp4(128, n, !NV, NV ? 0 : 2);
        ok = ptx::mbar_wait(&acc_empty[buf], acc_phase ^ 1u, dead, p.status_dev);
        if (!ok) break;
        ptx::tc_fence_after_sync();
        const uint32_t d = tmem + buf * 128;
        for (int k = 0; k < p.num_k; ++k) {
          ok = ptx::mbar_wait(&full[stage], phase, dead, p.status_dev);
          if (!ok) break;
          ptx::tc_fence_after_sync();
          const uint32_t w_addr = ptx::smem_addr(smem + stage * stage_size);
          const uint32_t a_addr = w_addr + kWBytes;
          const uint32_t ws_addr = a_addr + p.n_tile * 128, as_addr = ws_addr + kSf;
#pragma unroll
          for (int j = 0; j < kSfTiles; ++j) {
            ptx::tmem_cp_scales(tmem + kSfCol + j * 4, ptx::with_start(sf_desc, ws_addr + j * kSfTileBytes));
            ptx::tmem_cp_scales(tmem + kSfCol + 16 + j * 4, ptx::with_start(sf_desc, as_addr + j * kSfTileBytes));
          }
          // 64-column steps that hold columns of the matrix; beyond them scales need not exist
          const int64_t left = p.in - static_cast<int64_t>(k) * kKT;
          const int steps = left >= kKT ? 4 : static_cast<int>((left + 63) / 64);
          for (int j = 0; j < steps; ++j) {
            const uint32_t sf = NV ? j * 4 : j / 2 * 4;
            ptx::mma_fp4<NV>(d, ptx::with_start(desc, w_addr + j * 32), ptx::with_start(desc, a_addr + j * 32),
                             (j & 1) ? id1 : id0, tmem + kSfCol + sf, tmem + kSfCol + 16 + sf + x.a_sf_col, (k | j) != 0);
          }
          ptx::mma_commit(&empty[stage]);
          if (++stage == p.n_stages) { stage = 0; phase ^= 1u; }
        }
        if (!ok) break;
        ptx::mma_commit(&acc_full[buf]);
        buf ^= 1;
        if (buf == 0) acc_phase ^= 1u;
      }
      if (*dead) {
        ptx::mma_commit(&drain);
        const long long t0 = clock64();
        while (!ptx::mbar_try_wait(&drain, 0) && clock64() - t0 < ptx::kWaitLimit) {}
      }
    }
  } else {
    // ------------------------------------------------------------------ epilogue (warps 2..5)
    const int q = warp & 3;                            // TMEM lane quadrant this warp may read
    int buf = 0;
    uint32_t acc_phase = 0;
    const int ta = NV ? tensor_scale_log2(p.a_amax) : 0, tb = NV ? tensor_scale_log2(p.b_amax) : 0;
    const float sa = exp2_int(ta), sb = exp2_int(tb);
    for (int t = blockIdx.x; t < num_tiles; t += gridDim.x) {
      const Tile x = tile_of(t, p, prefix);
      if (!ptx::mbar_wait(&acc_full[buf], acc_phase, dead, p.status_dev)) break;
      ptx::tc_fence_after_sync();
      const int64_t o = x.m + q * 32 + lane;
      const int64_t base = static_cast<int64_t>(x.row) * p.ldy + o;
#pragma unroll 1
      for (int c = 0; c < x.count; c += 32) {
        float v[32];
        ptx::tmem_ld32(tmem + (static_cast<uint32_t>(q * 32) << 16) + buf * 128 + c, v);
        if (o < p.out) {
#pragma unroll
          for (int j = 0; j < 32; ++j)
            if (c + j < x.count) store_y(p.Y, p.ydtype, base + (c + j) * p.ldy, v[j] * sa * sb);
        }
      }
      ptx::tc_fence_before_sync();
      __syncwarp();
      if (lane == 0) ptx::mbar_arrive(&acc_empty[buf]);
      buf ^= 1;
      if (buf == 0) acc_phase ^= 1u;
    }
  }

  ptx::tc_fence_before_sync();
  __syncthreads();
  if (warp == 1) {
    ptx::tc_fence_after_sync();
    ptx::tmem_dealloc(tmem, 512);
  }
}

template <int FORMAT>
int launch(const CUtensorMap (&tm)[4], const MmParams& p, unsigned grid, size_t smem, cudaStream_t st) {
  ADADIM_CUDA_TRY(cudaFuncSetAttribute(fp4_matmul_kernel<FORMAT>, cudaFuncAttributeMaxDynamicSharedMemorySize, 226 * 1024 - 6144));
  fp4_matmul_kernel<FORMAT><<<grid, kThreads, smem, st>>>(tm[0], tm[1], tm[2], tm[3], p);
  return cudaGetLastError() == cudaSuccess ? ADADIM_OK : ADADIM_ERR_CUDA;
}

}  // namespace

int fp4_matmul_launch(const adadim_fp4tensor& A, int64_t n_rows, const int32_t* offsets, int n_experts,
                      const adadim_fp4tensor& B, int64_t out, int64_t in, int format, void* Y, int ydtype, int64_t ldy,
                      int* status_dev, cudaStream_t st) {
  static int sm_count = 0;
  if (sm_count == 0) {
    int dev = 0;
    ADADIM_CUDA_TRY(cudaGetDevice(&dev));
    ADADIM_CUDA_TRY(cudaDeviceGetAttribute(&sm_count, cudaDevAttrMultiProcessorCount, dev));
  }
  MmParams p = {};
  p.out = out;
  p.in = in;
  p.rows = static_cast<int>(n_rows);
  p.n_experts = n_experts;
  p.offsets = offsets;
  p.m_tiles = static_cast<int>((out + 127) / 128);
  p.n_tile = n_rows <= 16 ? 16 : n_rows <= 32 ? 32 : n_rows <= 64 ? 64 : 128;
  p.num_k = static_cast<int>((in + kKT - 1) / kKT);
  p.n_sf = sf_tiles(format, in);
  p.w_sf_rows = sf_tile_rows(out, 0);
  p.Y = Y;
  p.ydtype = ydtype;
  p.ldy = ldy;
  p.a_amax = A.amax;
  p.b_amax = B.amax;
  p.status_dev = status_dev;
  const size_t per = stage_bytes(format, p.n_tile);
  p.n_stages = static_cast<int>((220 * 1024 - 6144) / per);
  if (p.n_stages > kMaxStages) p.n_stages = kMaxStages;
  const int64_t weights = n_experts > 0 ? n_experts : 1;
  const uint64_t inner = static_cast<uint64_t>((in + 1) / 2);
  const uint32_t sf_box = sf_stage_bytes(format) / 128;
  CUtensorMap tm[4];
  int rc;
  if ((rc = make_tmap_u8(&tm[0], B.codes, inner, static_cast<uint64_t>(weights * out), static_cast<uint64_t>(B.ld), 128, true)) != ADADIM_OK) return rc;
  if ((rc = make_tmap_u8(&tm[1], A.codes, inner, static_cast<uint64_t>(n_rows), static_cast<uint64_t>(A.ld), static_cast<uint32_t>(p.n_tile), true)) != ADADIM_OK) return rc;
  if ((rc = make_tmap_u8(&tm[2], B.scales, 128, weights * scale_bytes(format, out, in, 0) / 128, 128, sf_box, false)) != ADADIM_OK) return rc;
  if ((rc = make_tmap_u8(&tm[3], A.scales, 128, scale_bytes(format, n_rows, in, n_experts) / 128, 128, sf_box, false)) != ADADIM_OK) return rc;
  // dense: the tiles are known here; grouped: at most one partial tile for every expert on top
  int64_t tiles = (n_rows + p.n_tile - 1) / p.n_tile;
  if (n_experts > 0) tiles += n_experts;
  tiles *= p.m_tiles;
  const unsigned grid = static_cast<unsigned>(tiles < sm_count ? tiles : sm_count);
  const size_t smem = p.n_stages * per + 1024;
  return format == ADADIM_MXFP4 ? launch<ADADIM_MXFP4>(tm, p, grid, smem, st) : launch<ADADIM_NVFP4>(tm, p, grid, smem, st);
}

}  // namespace adadim
