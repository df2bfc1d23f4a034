// Product of two microscaled 4-bit matrices on the block-scaled tensor-core path, plain and grouped
// by expert:  Y[t, o] = 2^(ta + tb) sum_k A[t, k] B[o, k],  scales applied by the matrix instruction.
//
// The weight is the instruction's M side and the tokens its N side, in every case: N may be any
// multiple of 16, so one token, the ragged end of an expert's rows and a full tile all run without
// multiplying padding, and the accumulator of one weight row sits in one TMEM lane.  Both operands
// arrive by TMA as 256-column stages (128 bytes of codes per row, 128-byte swizzle) together with
// their scale tiles, which the issuing thread copies from shared memory to TMEM in front of the MMAs
// that use them.  Two kernels:
//   pair   many tokens, bound by the tensor pipe: a cluster of two CTAs works on one 256 x 256 tile
//          (each CTA loads half of either operand, so a step's bytes per CTA are half of what one CTA
//          on a 128 x 256 tile would need), persistent over the tiles, with two accumulators that
//          share 64 of their 256 TMEM columns (512 columns hold two of them and the scales only that
//          way): the epilogue drains the shared columns first, and the next tile's MMAs wait for
//          those alone.
//   split  few tokens, bound by the weight's bytes: 128 weight rows x up to 128 tokens per cluster, the
//          columns split over the cluster's 1 .. 8 CTAs, partial sums exchanged through distributed
//          shared memory and added in the order of the columns; two CTAs to an SM.  Launched behind
//          the quantizer it starts streaming the weight at once and waits only before it reads the
//          activations.
#include "fp4.cuh"
#include "umma.cuh"

namespace adadim {
namespace {

using namespace fp4;

constexpr int kKT = 256;                               // columns of a stage
constexpr int kThreads = 192;                          // TMA warp, MMA warp, four epilogue warps
constexpr int kPairThreads = 320;                      // pair kernel: eight
constexpr int kMaxStages = 8;
constexpr uint32_t kWBytes = 128 * 128;
constexpr int kBand = 8;                               // weight tiles that share a sweep over the tokens

struct MmParams {
  int64_t out, in;
  int rows;                                            // of A and Y
  int n_experts;                                       // 0: dense
  const int32_t* offsets;
  int m_tiles;                                         // tiles of one weight's rows
  int n_tile;                                          // tokens of a tile
  int num_k;                                           // stages of a tile
  int n_stages;
  int splits;                                          // split kernel: CTAs of a cluster
  int64_t n_sf;                                        // scale tiles of a tile row
  int64_t w_sf_rows;                                   // scale tile rows of one weight
  void* Y;
  int64_t ldy;
  const float* a_amax;
  const float* b_amax;
  int* status_dev;
};

__host__ __device__ constexpr uint32_t sf_stage_bytes(int format) { return kKT / sf_cols(format) * kSfTileBytes; }
// bytes one CTA loads for a stage: 128 weight rows, its share of the tokens, their scales (of all tokens)
__host__ __device__ __forceinline__ uint32_t stage_bytes(int format, bool pair, int n_tile) {
  return kWBytes + static_cast<uint32_t>(pair ? n_tile / 2 : n_tile) * 128 + (pair ? 3 : 2) * sf_stage_bytes(format);
}

// One output tile: weight rows from `m` on, the `count` (<= n_tile) rows of A from `row` on.
struct Tile {
  int e, m, row, count;
  int64_t a_sf_row;                                    // scale tile row of A, and where in it the tile
  int a_sf_col;                                        // begins, in 32-row columns
};

// Tiles are numbered expert by expert; inside one, bands of kBand weight tiles sweep over the tokens,
// so that the CTAs at work at one time share both operands in L2.
template <int TILE_M>
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
  x.m = (band * kBand + in_band - j * width) * TILE_M;
  x.row = first + j * p.n_tile;
  x.count = min(p.n_tile, n - j * p.n_tile);
  x.a_sf_row = (p.n_experts > 0 ? first / kSfRows + x.e : 0) + j * p.n_tile / kSfRows;
  x.a_sf_col = j * p.n_tile % kSfRows / 32;            // several tiles only where n_tile is a multiple of 32
  return x;
}
// Tiles of each expert as a running sum, by one warp; prefix[n_experts] is their number.
__device__ __forceinline__ void tile_prefix(const MmParams& p, int lane, int* prefix) {
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

__device__ __forceinline__ void put(__nv_bfloat16* y, float v) { *y = __float2bfloat16_rn(v); }
__device__ __forceinline__ void put(__half* y, float v) { *y = __float2half_rn(v); }
__device__ __forceinline__ void put(float* y, float v) { *y = v; }
// 32 tokens of one weight row: y + j * ldy receives v[j] * scale, j < n
template <typename T>
__device__ __forceinline__ void store_tokens(T* y, int64_t ldy, int n, float scale, const float (&v)[32]) {
  if (n >= 32) {
#pragma unroll
    for (int j = 0; j < 32; ++j) { put(y, v[j] * scale); y += ldy; }
  } else {
#pragma unroll
    for (int j = 0; j < 32; ++j) { if (j < n) put(y, v[j] * scale); y += ldy; }
  }
}
// 2^(ta + tb).  Each lies between 2^-100 and 2^117: the product is 0 or infinite only where |amax| of both
// matrices are so far out that every result is.
template <bool NV>
__device__ __forceinline__ float product_scale(const MmParams& p) {
  return NV ? exp2_int(tensor_scale_log2(p.a_amax)) * exp2_int(tensor_scale_log2(p.b_amax)) : 1.0f;
}
// After a wait that ran out: time for the copies already issued to land before shared memory goes away
// (they take microseconds).
__device__ __forceinline__ void let_copies_land() {
  const long long t0 = clock64();
  while (clock64() - t0 < (1 << 20)) {}
}

// The MMAs of one stage: scale tiles to TMEM, then the 64-column steps that hold columns of the matrix
// (beyond them scales need not exist).  SFT: TMEM columns of one scale tile of the tokens.
template <int FORMAT, bool PAIR>
__device__ __forceinline__ void issue_stage(uint32_t d, uint32_t sf_tmem, int a_sf_col, uint32_t w_addr, uint32_t a_addr,
                                            uint32_t ws_addr, uint32_t id0, uint32_t id1, int steps, bool first) {
  constexpr bool NV = FORMAT == ADADIM_NVFP4;
  constexpr uint32_t kSf = sf_stage_bytes(FORMAT);
  constexpr int kSfTiles = kSf / kSfTileBytes;                       // scale tiles of a stage: 4 or 2
  constexpr uint64_t desc = ptx::smem_desc_sw128(16, 1024);          // K-major: 8-row groups 1024 bytes apart
  constexpr uint64_t sf_desc = ptx::smem_desc_plain(16, 128);
  constexpr int kTok = PAIR ? 8 : 4;                                 // TMEM columns of one step's token scales
#pragma unroll
  for (int j = 0; j < kSfTiles; ++j) {
    ptx::tmem_cp_scales<PAIR>(sf_tmem + j * 4, ptx::with_start(sf_desc, ws_addr + j * kSfTileBytes));
    ptx::tmem_cp_scales<PAIR>(sf_tmem + 16 + j * kTok, ptx::with_start(sf_desc, ws_addr + kSf + j * kSfTileBytes));
    if (PAIR) ptx::tmem_cp_scales<PAIR>(sf_tmem + 16 + j * kTok + 4, ptx::with_start(sf_desc, ws_addr + 2 * kSf + j * kSfTileBytes));
  }
  auto step = [&](int j) {
    const int tile = NV ? j : j / 2;
    ptx::mma_fp4<NV, PAIR>(d, ptx::with_start(desc, w_addr + j * 32), ptx::with_start(desc, a_addr + j * 32),
                           (j & 1) ? id1 : id0, sf_tmem + tile * 4, sf_tmem + 16 + tile * kTok + a_sf_col, !(first && j == 0));
  };
  if (steps == 4) {
#pragma unroll
    for (int j = 0; j < 4; ++j) step(j);
  } else {
#pragma unroll 1
    for (int j = 0; j < steps; ++j) step(j);
  }
}
__device__ __forceinline__ int steps_of(int64_t in, int k) {
  const int64_t left = in - static_cast<int64_t>(k) * kKT;
  return left >= kKT ? 4 : static_cast<int>((left + 63) / 64);
}

// ---- pair -----------------------------------------------------------------------------------------
template <int FORMAT, typename T>
__global__ void __launch_bounds__(kPairThreads, 1)
fp4_pair_kernel(const __grid_constant__ CUtensorMap tmW, const __grid_constant__ CUtensorMap tmA,
                const __grid_constant__ CUtensorMap tmWs, const __grid_constant__ CUtensorMap tmAs, const MmParams p) {
  constexpr bool NV = FORMAT == ADADIM_NVFP4;
  constexpr uint32_t kSf = sf_stage_bytes(FORMAT);
  constexpr int kSfTiles = kSf / kSfTileBytes;
  constexpr uint32_t kAccStep = 192, kSfCol = 448;     // accumulators at 0 and 192, scales at 448

  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
  __shared__ uint64_t full[kMaxStages], empty[kMaxStages], acc_full[2], acc_empty[2], part_empty;
  __shared__ uint32_t tmem_slot;
  __shared__ int dead_word;
  __shared__ int prefix[kMaxGroups + 1];
  volatile int* dead = &dead_word;
  const int warp = ptx::uniform_warp(), lane = threadIdx.x & 31;
  const uint32_t rank = ptx::cluster_ctarank();
  const uint32_t stage_size = stage_bytes(FORMAT, true, p.n_tile);
  const uint32_t a_bytes = static_cast<uint32_t>(p.n_tile) * 64;
  const int pair0 = blockIdx.x >> 1, pairs = gridDim.x >> 1;

  if (threadIdx.x == 0) {
    for (int s = 0; s < p.n_stages; ++s) { ptx::mbar_init(&full[s], 1); ptx::mbar_init(&empty[s], 1); }
    for (int b = 0; b < 2; ++b) { ptx::mbar_init(&acc_full[b], 1); ptx::mbar_init(&acc_empty[b], 16); }
    ptx::mbar_init(&part_empty, 16);
    dead_word = 0;
    ptx::fence_mbar_init();
    ptx::tma_prefetch_desc(&tmW);
    ptx::tma_prefetch_desc(&tmA);
    ptx::tma_prefetch_desc(&tmWs);
    ptx::tma_prefetch_desc(&tmAs);
  }
  if (warp == 1) {
    ptx::tmem_alloc_pair(&tmem_slot, 512);
    ptx::tmem_relinquish_pair();
  }
  if (warp == 2 && p.n_experts > 0) tile_prefix(p, lane, prefix);
  ptx::tc_fence_before_sync();
  __syncthreads();
  ptx::cluster_sync();                                 // both CTAs' barriers exist before either signals the other's
  ptx::tc_fence_after_sync();
  const uint32_t tmem = tmem_slot;
  const int num_tiles = p.n_experts > 0 ? prefix[p.n_experts] : (p.rows + p.n_tile - 1) / p.n_tile * p.m_tiles;

  if (warp == 0) {
    // ------------------------------------------------------------------ TMA producer (both CTAs)
    int stage = 0;
    uint32_t phase = 0;
    bool ok = true;
    ptx::pdl_wait();
    for (int t = pair0; t < num_tiles && ok; t += pairs) {
      const Tile x = tile_of<256>(t, p, prefix);
      const int half = ((x.count + 15) & ~15) >> 1;    // tokens of this CTA
      const int w_row = static_cast<int>(x.e * p.out + x.m) + static_cast<int>(rank) * 128;
      const int a_row = x.row + static_cast<int>(rank) * half;
      int w_sf = static_cast<int>((x.e * p.w_sf_rows + x.m / kSfRows + rank) * p.n_sf * 4);
      int a_sf0 = static_cast<int>(x.a_sf_row * p.n_sf * 4), a_sf1 = static_cast<int>((x.a_sf_row + 1) * p.n_sf * 4);
      for (int k = 0; k < p.num_k; ++k) {
        ok = ptx::mbar_wait_warp(&empty[stage], phase ^ 1u, dead, p.status_dev);
        if (!ok) break;
        uint8_t* w_dst = smem + stage * stage_size;
        uint8_t* a_dst = w_dst + kWBytes;
        uint8_t* ws_dst = a_dst + a_bytes;
        const uint32_t bar = ptx::map_to_cta(ptx::smem_addr(&full[stage]), 0);
        if (ptx::elect_one()) {
          // one barrier, the leader's, counts both CTAs' bytes
          if (rank == 0) ptx::mbar_arrive_expect_tx(&full[stage], 2 * stage_size);
          ptx::tma_load_2d_pair(w_dst, &tmW, k * (kKT / 2), w_row, bar);
          ptx::tma_load_2d_pair(a_dst, &tmA, k * (kKT / 2), a_row, bar);
          ptx::tma_load_2d_pair(ws_dst, &tmWs, 0, w_sf, bar);
          ptx::tma_load_2d_pair(ws_dst + kSf, &tmAs, 0, a_sf0, bar);
          ptx::tma_load_2d_pair(ws_dst + 2 * kSf, &tmAs, 0, a_sf1, bar);
        }
        __syncwarp();
        w_sf += kSfTiles * 4;
        a_sf0 += kSfTiles * 4;
        a_sf1 += kSfTiles * 4;
        if (++stage == p.n_stages) { stage = 0; phase ^= 1u; }
      }
    }
    if (!ok) let_copies_land();
  } else if (warp == 1) {
    // ------------------------------------------------------------------ MMA issuer (leader)
    if (rank == 0) {
      int stage = 0, buf = 0;
      uint32_t phase = 0, acc_phase = 0, part_phase = 0;
      bool ok = true, ready = false;
      for (int t = pair0; t < num_tiles && ok; t += pairs) {
        const Tile x = tile_of<256>(t, p, prefix);
        const int n = (x.count + 15) & ~15;
        const uint32_t id0 = ptx::idesc_fp4(256, n, !NV, 0), id1 = ptx::idesc_fp4(256, n, !NV, NV ? 0 : 2);
        ok = ptx::mbar_wait_warp(&acc_empty[buf], acc_phase ^ 1u, dead, p.status_dev);
        if (ok && t != pair0) {                        // the tile before has left the shared columns
          ok = ptx::mbar_wait_warp(&part_empty, part_phase, dead, p.status_dev);
          part_phase ^= 1u;
        }
        if (!ok) break;
        ptx::tc_fence_after_sync();
        for (int k = 0; k < p.num_k; ++k) {
          if (!ready) ok = ptx::mbar_wait_warp(&full[stage], phase, dead, p.status_dev);
          if (!ok) break;
          ptx::tc_fence_after_sync();
          const int cur = stage;
          if (++stage == p.n_stages) { stage = 0; phase ^= 1u; }
          // asked before this stage's instructions are issued: the answer is there when they are
          const bool next = ptx::mbar_try_wait(&full[stage], phase);
          const uint32_t w_addr = ptx::smem_addr(smem + cur * stage_size);
          const int steps = steps_of(p.in, k);
          if (ptx::elect_one()) {
            issue_stage<FORMAT, true>(tmem + buf * kAccStep, tmem + kSfCol, 0, w_addr, w_addr + kWBytes,
                                      w_addr + kWBytes + a_bytes, id0, id1, steps, k == 0);
            ptx::mma_commit_pair(&empty[cur]);
            if (k == p.num_k - 1) ptx::mma_commit_pair(&acc_full[buf]);
          }
          ready = __all_sync(0xffffffffu, next) != 0;
        }
        buf ^= 1;
        if (buf == 0) acc_phase ^= 1u;
      }
      if (!ok) let_copies_land();
    }
  } else {
    // ------------------------------------------------------------------ epilogue (warps 2..9 of both CTAs)
    const int q = warp & 3;                            // TMEM lane quadrant this warp may read
    const int side = (warp - 2) >> 2;                  // of each 64 columns, which 32 this warp takes
    int buf = 0;
    uint32_t acc_phase = 0;
    const float scale = product_scale<NV>(p);
    const uint32_t part_bar = ptx::map_to_cta(ptx::smem_addr(&part_empty), 0);
    for (int t = pair0; t < num_tiles; t += pairs) {
      const Tile x = tile_of<256>(t, p, prefix);
      if (!ptx::mbar_wait_warp(&acc_full[buf], acc_phase, dead, p.status_dev)) break;
      ptx::tc_fence_after_sync();
      const int64_t o = x.m + static_cast<int>(rank) * 128 + q * 32 + lane;
      T* y = static_cast<T*>(p.Y) + static_cast<int64_t>(x.row) * p.ldy + o;
      const uint32_t acc = tmem + (static_cast<uint32_t>(q * 32) << 16) + buf * kAccStep;
      // the shared columns first: the last 64 of accumulator 0, the first 64 of accumulator 1
      const int s0 = (buf == 0 ? static_cast<int>(kAccStep) : 0) + side * 32;
      {
        float v[32];
        if (s0 < x.count) ptx::tmem_ld32(acc + s0, v);
        ptx::tc_fence_before_sync();
        __syncwarp();
        if (lane == 0) ptx::mbar_arrive_cluster(part_bar);
        if (s0 < x.count && o < p.out) store_tokens(y + s0 * p.ldy, p.ldy, x.count - s0, scale, v);
      }
#pragma unroll 1
      for (int c = (buf == 0 ? 0 : 64) + side * 32; c < min(x.count, buf == 0 ? 192 : 256); c += 64) {
        float v[32];
        ptx::tmem_ld32(acc + c, v);
        if (o < p.out) store_tokens(y + c * p.ldy, p.ldy, x.count - c, scale, v);
      }
      ptx::tc_fence_before_sync();
      __syncwarp();
      if (lane == 0) ptx::mbar_arrive_cluster(ptx::map_to_cta(ptx::smem_addr(&acc_empty[buf]), 0));
      buf ^= 1;
      if (buf == 0) acc_phase ^= 1u;
    }
  }

  ptx::tc_fence_before_sync();
  __syncthreads();
  ptx::cluster_sync();                                 // no CTA leaves while the other may still signal it
  if (warp == 1) {
    ptx::tc_fence_after_sync();
    ptx::tmem_dealloc_pair(tmem, 512);
  }
}

// ---- split ----------------------------------------------------------------------------------------
template <int FORMAT, typename T>
__global__ void __launch_bounds__(kThreads, 2)
fp4_split_kernel(const __grid_constant__ CUtensorMap tmW, const __grid_constant__ CUtensorMap tmA,
                 const __grid_constant__ CUtensorMap tmWs, const __grid_constant__ CUtensorMap tmAs, const MmParams p) {
  constexpr bool NV = FORMAT == ADADIM_NVFP4;
  constexpr uint32_t kSf = sf_stage_bytes(FORMAT);
  constexpr int kSfTiles = kSf / kSfTileBytes;
  constexpr uint32_t kSfCol = 128;                     // TMEM: one accumulator of 128 columns, then scales

  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
  __shared__ uint64_t full[kMaxStages], empty[kMaxStages], acc_full, red_full;
  __shared__ uint32_t tmem_slot;
  __shared__ int dead_word;
  __shared__ int prefix[kMaxGroups + 1];
  volatile int* dead = &dead_word;
  const int warp = ptx::uniform_warp(), lane = threadIdx.x & 31;
  const uint32_t stage_size = stage_bytes(FORMAT, false, p.n_tile);
  const uint32_t a_bytes = static_cast<uint32_t>(p.n_tile) * 128;
  float* red = reinterpret_cast<float*>(smem + p.n_stages * stage_size);     // [tokens of this CTA][splits][128 rows]
  const int rank = blockIdx.x % p.splits, t = blockIdx.x / p.splits;
  const int k0 = static_cast<int>(static_cast<int64_t>(p.num_k) * rank / p.splits);
  const int k1 = static_cast<int>(static_cast<int64_t>(p.num_k) * (rank + 1) / p.splits);

  if (threadIdx.x == 0) {
    for (int s = 0; s < p.n_stages; ++s) { ptx::mbar_init(&full[s], 1); ptx::mbar_init(&empty[s], 1); }
    ptx::mbar_init(&acc_full, 1);
    ptx::mbar_init(&red_full, 4 * p.splits);
    dead_word = 0;
    ptx::fence_mbar_init();
    ptx::tma_prefetch_desc(&tmW);
    ptx::tma_prefetch_desc(&tmA);
    ptx::tma_prefetch_desc(&tmWs);
    ptx::tma_prefetch_desc(&tmAs);
  }
  if (warp == 1) {
    ptx::tmem_alloc(&tmem_slot, 256);
    ptx::tmem_relinquish();
  }
  if (warp == 2 && p.n_experts > 0) tile_prefix(p, lane, prefix);
  ptx::tc_fence_before_sync();
  __syncthreads();
  if (p.splits > 1) ptx::cluster_sync();
  ptx::tc_fence_after_sync();
  const uint32_t tmem = tmem_slot;
  const int num_tiles = p.n_experts > 0 ? prefix[p.n_experts] : (p.rows + p.n_tile - 1) / p.n_tile * p.m_tiles;
  const bool work = t < num_tiles;                     // the grid is an upper bound where experts are ragged
  Tile x = {};
  if (work) x = tile_of<128>(t, p, prefix);

  if (warp == 0) {
    // ------------------------------------------------------------------ TMA producer
    if (work) {
      const int w_row = static_cast<int>(x.e * p.out + x.m);
      const int w_sf = static_cast<int>((x.e * p.w_sf_rows + x.m / kSfRows) * p.n_sf * 4);
      const int a_sf = static_cast<int>(x.a_sf_row * p.n_sf * 4);
      auto load_w = [&](int k, int stage) {
        uint8_t* w_dst = smem + stage * stage_size;
        if (ptx::elect_one()) {
          ptx::mbar_arrive_expect_tx(&full[stage], stage_size);
          ptx::tma_load_2d(w_dst, &tmW, k * (kKT / 2), w_row, &full[stage]);
          ptx::tma_load_2d(w_dst + kWBytes + a_bytes, &tmWs, 0, w_sf + k * kSfTiles * 4, &full[stage]);
        }
        __syncwarp();
      };
      auto load_a = [&](int k, int stage) {
        uint8_t* a_dst = smem + stage * stage_size + kWBytes;
        if (ptx::elect_one()) {
          ptx::tma_load_2d(a_dst, &tmA, k * (kKT / 2), x.row, &full[stage]);
          ptx::tma_load_2d(a_dst + a_bytes + kSf, &tmAs, 0, a_sf + k * kSfTiles * 4, &full[stage]);
        }
        __syncwarp();
      };
      // the ring's first fill: the weight does not depend on the launch before this one
      const int ahead = min(k1 - k0, p.n_stages);
      for (int i = 0; i < ahead; ++i) load_w(k0 + i, i);
      ptx::pdl_wait();
      for (int i = 0; i < ahead; ++i) load_a(k0 + i, i);
      int stage = 0;
      uint32_t phase = 0;
      bool ok = true;
      for (int k = k0 + ahead; k < k1 && ok; ++k) {
        ok = ptx::mbar_wait_warp(&empty[stage], phase, dead, p.status_dev);
        if (!ok) break;
        load_w(k, stage);
        load_a(k, stage);
        if (++stage == p.n_stages) { stage = 0; phase ^= 1u; }
      }
      if (!ok) let_copies_land();
    }
  } else if (warp == 1) {
    // ------------------------------------------------------------------ MMA issuer
    if (work) {
      const int n = (x.count + 15) & ~15;
      const uint32_t id0 = ptx::idesc_fp4(128, n, !NV, 0), id1 = ptx::idesc_fp4(128, n, !NV, NV ? 0 : 2);
      int stage = 0;
      uint32_t phase = 0;
      bool ok = true;
      for (int k = k0; k < k1; ++k) {
        ok = ptx::mbar_wait_warp(&full[stage], phase, dead, p.status_dev);
        if (!ok) break;
        ptx::tc_fence_after_sync();
        const uint32_t w_addr = ptx::smem_addr(smem + stage * stage_size);
        const int steps = steps_of(p.in, k);
        if (ptx::elect_one()) {
          issue_stage<FORMAT, false>(tmem, tmem + kSfCol, x.a_sf_col, w_addr, w_addr + kWBytes, w_addr + kWBytes + a_bytes,
                                     id0, id1, steps, k == k0);
          ptx::mma_commit(&empty[stage]);
          if (k == k1 - 1) ptx::mma_commit(&acc_full);
        }
        __syncwarp();
        if (++stage == p.n_stages) { stage = 0; phase ^= 1u; }
      }
      if (!ok) let_copies_land();
    }
  } else if (work) {
    // ------------------------------------------------------------------ epilogue (warps 2..5)
    const int q = warp & 3;                            // TMEM lane quadrant this warp may read
    const float scale = product_scale<NV>(p);
    const int row = q * 32 + lane;
    const int64_t o = x.m + row;
    T* y = static_cast<T*>(p.Y) + static_cast<int64_t>(x.row) * p.ldy + o;
    const uint32_t acc = tmem + (static_cast<uint32_t>(q * 32) << 16);
    bool ok = ptx::mbar_wait_warp(&acc_full, 0, dead, p.status_dev);
    ptx::tc_fence_after_sync();
    if (p.splits == 1) {
#pragma unroll 1
      for (int c = 0; c < x.count && ok; c += 32) {
        float v[32];
        ptx::tmem_ld32(acc + c, v);
        if (o < p.out) store_tokens(y + c * p.ldy, p.ldy, x.count - c, scale, v);
      }
    } else {
      // token c of the tile is finished by CTA c % splits: every CTA sends it its partial sums
#pragma unroll 1
      for (int c = 0; c < x.count && ok; c += 32) {
        float v[32];
        ptx::tmem_ld32(acc + c, v);
#pragma unroll
        for (int j = 0; j < 32; ++j) {
          if (c + j < x.count) {
            const int dst = (c + j) % p.splits, slot = (c + j) / p.splits;
            ptx::st_cluster_f32(ptx::map_to_cta(ptx::smem_addr(red + (slot * p.splits + rank) * 128 + row), dst), v[j]);
          }
        }
      }
      __syncwarp();
      if (lane < p.splits) ptx::mbar_arrive_release_cluster(ptx::map_to_cta(ptx::smem_addr(&red_full), lane));
      ok = ptx::mbar_wait_warp(&red_full, 0, dead, p.status_dev) && ok;
      ptx::fence_acquire_cluster();
      for (int c = rank, slot = 0; c < x.count && ok; c += p.splits, ++slot) {
        float s = 0.0f;
        for (int k = 0; k < p.splits; ++k) s += red[(slot * p.splits + k) * 128 + row];
        if (o < p.out) put(y + c * p.ldy, s * scale);
      }
    }
  }

  ptx::tc_fence_before_sync();
  __syncthreads();
  if (p.splits > 1) ptx::cluster_sync();               // no CTA leaves while another may still write to it
  if (warp == 1) {
    ptx::tc_fence_after_sync();
    ptx::tmem_dealloc(tmem, 256);
  }
}

constexpr size_t kSmemOne = 220 * 1024, kSmemTwo = 106 * 1024;       // dynamic shared memory at one and two CTAs per SM

template <typename K>
int launch(K kernel, const CUtensorMap (&tm)[4], const MmParams& p, unsigned grid, int threads, int cluster, size_t smem,
           bool chained, cudaStream_t st) {
  ADADIM_CUDA_TRY(cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, static_cast<int>(kSmemOne)));
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(grid);
  cfg.blockDim = dim3(static_cast<unsigned>(threads));
  cfg.dynamicSmemBytes = smem;
  cfg.stream = st;
  cudaLaunchAttribute attr[2];
  int n = 0;
  if (cluster > 1) {
    attr[n].id = cudaLaunchAttributeClusterDimension;
    attr[n].val.clusterDim.x = static_cast<unsigned>(cluster);
    attr[n].val.clusterDim.y = 1;
    attr[n].val.clusterDim.z = 1;
    ++n;
  }
  if (chained) {                                       // may start while the quantizer before it in the stream runs
    attr[n].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[n].val.programmaticStreamSerializationAllowed = 1;
    ++n;
  }
  cfg.attrs = attr;
  cfg.numAttrs = static_cast<unsigned>(n);
  ADADIM_CUDA_TRY(cudaLaunchKernelEx(&cfg, kernel, tm[0], tm[1], tm[2], tm[3], p));
  return ADADIM_OK;
}

template <typename T>
int launch_format(bool pair, int format, const CUtensorMap (&tm)[4], const MmParams& p, unsigned grid, size_t smem, bool chained,
                  cudaStream_t st) {
  if (pair) return format == ADADIM_MXFP4 ? launch(fp4_pair_kernel<ADADIM_MXFP4, T>, tm, p, grid, kPairThreads, 2, smem, chained, st)
                                          : launch(fp4_pair_kernel<ADADIM_NVFP4, T>, tm, p, grid, kPairThreads, 2, smem, chained, st);
  return format == ADADIM_MXFP4 ? launch(fp4_split_kernel<ADADIM_MXFP4, T>, tm, p, grid, kThreads, p.splits, smem, chained, st)
                                : launch(fp4_split_kernel<ADADIM_NVFP4, T>, tm, p, grid, kThreads, p.splits, smem, chained, st);
}

}  // namespace

int fp4_matmul_launch(const adadim_fp4tensor& A, int64_t n_rows, const int32_t* offsets, int n_experts,
                      const adadim_fp4tensor& B, int64_t out, int64_t in, int format, void* Y, int ydtype, int64_t ldy,
                      int* status_dev, bool chained, cudaStream_t st) {
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
  p.num_k = static_cast<int>((in + kKT - 1) / kKT);
  p.n_sf = sf_tiles(format, in);
  p.w_sf_rows = sf_tile_rows(out, 0);
  p.Y = Y;
  p.ldy = ldy;
  p.a_amax = A.amax;
  p.b_amax = B.amax;
  p.status_dev = status_dev;
  const int64_t weights = n_experts > 0 ? n_experts : 1;
  const int64_t typical = (n_rows + weights - 1) / weights;          // rows of one expert if they were equal
  const bool pair = typical > 128;
  if (pair) {
    p.n_tile = 256;
  } else {
    // several tiles of one expert begin at multiples of 32 rows (the scale tiles' columns)
    const int64_t want = n_experts > 0 ? (2 * typical < n_rows ? 2 * typical : n_rows) : n_rows;
    p.n_tile = want <= 16 && want == n_rows ? 16 : want <= 32 ? 32 : want <= 64 ? 64 : 128;
  }
  p.m_tiles = static_cast<int>((out + (pair ? 255 : 127)) / (pair ? 256 : 128));
  // dense: the tiles are known here; grouped: at most one partial tile for every expert on top
  int64_t tiles = (n_rows + p.n_tile - 1) / p.n_tile;
  if (n_experts > 0) tiles += n_experts < n_rows ? n_experts : n_rows;
  tiles *= p.m_tiles;

  const uint64_t inner = static_cast<uint64_t>((in + 1) / 2);
  const uint32_t sf_box = sf_stage_bytes(format) / 128;
  CUtensorMap tm[4];
  int rc;
  if ((rc = make_tmap_u8(&tm[0], B.codes, inner, static_cast<uint64_t>(weights * out), static_cast<uint64_t>(B.ld), 128, true)) != ADADIM_OK) return rc;
  if ((rc = make_tmap_u8(&tm[1], A.codes, inner, static_cast<uint64_t>(n_rows), static_cast<uint64_t>(A.ld),
                         static_cast<uint32_t>(pair ? p.n_tile / 2 : p.n_tile), true)) != ADADIM_OK) return rc;
  if ((rc = make_tmap_u8(&tm[2], B.scales, 128, weights * scale_bytes(format, out, in, 0) / 128, 128, sf_box, false)) != ADADIM_OK) return rc;
  if ((rc = make_tmap_u8(&tm[3], A.scales, 128, scale_bytes(format, n_rows, in, n_experts) / 128, 128, sf_box, false)) != ADADIM_OK) return rc;

  const size_t per = stage_bytes(format, pair, p.n_tile);
  unsigned grid;
  size_t smem;
  if (pair) {
    p.n_stages = static_cast<int>((kSmemOne - 1024) / per);
    if (p.n_stages > kMaxStages) p.n_stages = kMaxStages;
    grid = static_cast<unsigned>(2 * (tiles < sm_count / 2 ? tiles : sm_count / 2));
    smem = p.n_stages * per + 1024;
  } else {
    // split the columns until there are two CTAs for every SM
    p.splits = 1;
    while (p.splits < 8 && tiles * p.splits * 2 <= 2 * sm_count && p.splits * 2 <= p.num_k) p.splits *= 2;
    const size_t red = p.splits > 1 ? static_cast<size_t>((p.n_tile + p.splits - 1) / p.splits) * p.splits * 512 : 0;
    p.n_stages = static_cast<int>((kSmemTwo - 1024 - red) / per);
    if (p.n_stages > kMaxStages) p.n_stages = kMaxStages;
    if (p.n_stages < 2) p.n_stages = 2;
    grid = static_cast<unsigned>(tiles * p.splits);
    smem = p.n_stages * per + red + 1024;
  }
  if (ydtype == ADADIM_F32) return launch_format<float>(pair, format, tm, p, grid, smem, chained, st);
  if (ydtype == ADADIM_F16) return launch_format<__half>(pair, format, tm, p, grid, smem, chained, st);
  return launch_format<__nv_bfloat16>(pair, format, tm, p, grid, smem, chained, st);
}

}  // namespace adadim
