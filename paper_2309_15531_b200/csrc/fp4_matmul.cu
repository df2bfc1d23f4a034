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
//          on a 128 x 256 tile would need), persistent over the tiles, with two accumulators in TMEM,
//          so that one is drained while the other is filled.
//   split  few tokens, bound by the weight's bytes: 128 weight rows x up to 128 tokens per cluster, the
//          columns split over the cluster's 1 .. 8 CTAs, partial sums exchanged through distributed
//          shared memory and added in the order of the columns; up to four CTAs to an SM, so that all
//          tiles are under way at once and share the memory's bandwidth evenly.  Launched behind the
//          quantizer it starts streaming the weight at once and waits only before it reads the
//          activations.
// Times in the comments below are the best of a graph's replays at 1.9 GHz.  In a run of seconds the power cap (1.3 to 1.6
// GHz) lengthens the many-token cases (2048 x W[11008,4096] 41-44 -> 53 us, 8 experts x 8192 rows 163-173 -> 196-201 us),
// and a caller in Python the shortest ones (1 x W[4096,4096] 6.3 -> 8.2 us).
#include "fp4.cuh"
#include "umma_fp4.cuh"

namespace adadim {
namespace {

using namespace fp4;

constexpr int kKT = 256;                               // columns of a stage
constexpr int kThreads = 192;                          // TMA warp, MMA warp, four epilogue warps
constexpr int kPairThreads = 320;                      // pair kernel: eight
constexpr int kMaxStages = 8;
constexpr uint32_t kWBytes = 128 * 128;
constexpr uint32_t kOutBytes = 8 * 4096;               // pair kernel: tiles of Y on their way out
constexpr int kFusedThreads = 320;                     // split kernel that quantizes: four warps more,
constexpr int kFusedPerSm = 3;                         // CTAs of an SM (by its registers)
constexpr int kFusedTile = 16;                         // the tokens of a tile, of which it has
constexpr int kFusedTokens = 8;                        // up to so many: see plan_of
constexpr int kBand = 8;                               // weight tiles that share a sweep over the tokens

struct MmParams {
  int64_t out, in;
  int rows;                                            // of A and Y
  int n_experts;                                       // 0: dense
  const int32_t* offsets;
  int m_tiles;                                         // tiles of one weight's rows
  int n_tile;                                          // tokens of a tile
  int lt;                                              // of the layout of A's scales: n_tile is a multiple of it
                                                       // (or there is one tile)
  int lt_per_tile, sub;                                // n_tile / lt; scale tile rows of lt rows
  int num_k;                                           // stages of a tile
  int n_stages;
  int splits;                                          // split kernel: CTAs of a cluster
  int tmem_cols;                                       // and TMEM columns
  Source x;                                            // and, where it quantizes the activations, those
  int64_t n_sf;                                        // scale tiles of a tile row
  int64_t w_sf_rows;                                   // scale tile rows of one weight
  void* Y;
  int64_t ldy;
  int bulk_y;                                          // pair kernel: Y can be stored by TMA
  unsigned pace_ns;                                    // and the pause between two stores of 32 tokens
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
  int a_sf_row;                                        // scale tile row of A
};

// a / b for a, b > 0.  In binary32 below 2^21, where (a + 1/2) / b is off by less than its distance 1 / (2 b) from
// a whole number: a sixth of an integer division's latency, which a tile's first stage would wait for.
__device__ __forceinline__ int quick_div(int a, int b) {
  if (a >= (1 << 21)) return a / b;
  return static_cast<int>((static_cast<float>(a) + 0.5f) * __frcp_rn(static_cast<float>(b)));
}
// Tiles are numbered expert by expert; inside one, bands of kBand weight tiles sweep over the tokens,
// so that the CTAs at work at one time share both operands in L2.
__device__ __forceinline__ Tile tile_of(int t, const MmParams& p, const int* prefix) {
  constexpr int TILE_M = 256;
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
  const int n_tiles = quick_div(n + p.n_tile - 1, p.n_tile);
  const int band = quick_div(t, kBand * n_tiles);
  const int in_band = t - band * kBand * n_tiles;
  const int width = min(kBand, p.m_tiles - band * kBand);
  const int j = quick_div(in_band, width);
  x.m = (band * kBand + in_band - j * width) * TILE_M;
  x.row = first + j * p.n_tile;
  x.count = min(p.n_tile, n - j * p.n_tile);
  x.a_sf_row = ((p.n_experts > 0 ? quick_div(first, p.lt) + x.e : 0) + j * p.lt_per_tile) * p.sub;
  return x;
}
// The tiles of a persistent warp, first, first + step, ..: worked out for 32 of them at a time, one by each lane
// (a tile takes several hundred cycles of dependent divisions, which would stall the loads at its start).
struct TileWalk {
  Tile mine;
  int n;
  __device__ __forceinline__ Tile next(int t, int step, int num_tiles, const MmParams& p, const int* prefix) {
    const int lane = threadIdx.x & 31;
    if ((n & 31) == 0) mine = t + lane * step < num_tiles ? tile_of(t + lane * step, p, prefix) : Tile{};
    const int from = n++ & 31;
    Tile x;
    x.e = __shfl_sync(0xffffffffu, mine.e, from);
    x.m = __shfl_sync(0xffffffffu, mine.m, from);
    x.row = __shfl_sync(0xffffffffu, mine.row, from);
    x.count = __shfl_sync(0xffffffffu, mine.count, from);
    x.a_sf_row = __shfl_sync(0xffffffffu, mine.a_sf_row, from);
    return x;
  }
};
// The split kernel's order: the token tiles of one weight tile next to each other.  Dense: from the grid.
__device__ __forceinline__ Tile tile_at(int j, int m, int e, int first, int n, const MmParams& p) {
  Tile x;
  x.e = e;
  x.m = m * 128;
  x.row = first + j * p.n_tile;
  x.count = min(p.n_tile, n - j * p.n_tile);
  x.a_sf_row = ((p.n_experts > 0 ? quick_div(first, p.lt) + e : 0) + j * p.lt_per_tile) * p.sub;
  return x;
}
__device__ __forceinline__ Tile tile_of_group(int t, const MmParams& p, const int* prefix) {
  int lo = 0, hi = p.n_experts - 1;                    // last e with prefix[e] <= t
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (prefix[mid] <= t) lo = mid; else hi = mid - 1;
  }
  const int first = clamped(p.offsets[lo], p.rows), n = clamped(p.offsets[lo + 1], p.rows) - first;
  const int n_tiles = quick_div(n + p.n_tile - 1, p.n_tile), m = quick_div(t - prefix[lo], n_tiles);
  return tile_at(t - prefix[lo] - m * n_tiles, m, lo, first, n, p);
}
// Tiles of each expert as a running sum, by one warp; prefix[n_experts] is their number.
__device__ __forceinline__ void tile_prefix(const MmParams& p, int lane, int* prefix) {
  int sum = 0;
  for (int e0 = 0; e0 < p.n_experts; e0 += 32) {
    const int e = e0 + lane;
    int c = 0;
    if (e < p.n_experts) {
      const int a = p.offsets[e], z = p.offsets[e + 1];
      if (blockIdx.x + blockIdx.y == 0 && (a < 0 || z > p.rows || z < a)) report(p.status_dev, ADADIM_ERR_SHAPE);
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
template <typename T>
__device__ __forceinline__ uint32_t packed(float a, float b) {       // a in the low half
  if constexpr (sizeof(T) == 4) return 0;
  else if constexpr (__is_same(T, __half)) { const __half2 h = __floats2half2_rn(a, b); return *reinterpret_cast<const uint32_t*>(&h); }
  else { const __nv_bfloat162 h = __floats2bfloat162_rn(a, b); return *reinterpret_cast<const uint32_t*>(&h); }
}
// 2^(ta + tb), which lies between 2^-200 and 2^234, as two factors that binary32 holds (one could be 0 or infinite where
// the result is neither).  Multiplied one after the other they round once at most: a sum is 0, or between 2^-20 (the
// smallest product of two codes and their scales) and 2^43, so that v * a is exact, or infinite where v * a * b is too.
struct ProductScale { float a, b; };
__device__ __forceinline__ float operator*(float v, const ProductScale& s) { return v * s.a * s.b; }
template <bool NV>
__device__ __forceinline__ ProductScale product_scale(const MmParams& p) {
  if (!NV) return {1.0f, 1.0f};
  const int e = tensor_scale_log2(p.a_amax) + tensor_scale_log2(p.b_amax), half = e / 2;
  return {exp2_int(half), exp2_int(e - half)};
}
// The same for two sums at once, rounded to a pair of 16-bit results.
template <typename T>
__device__ __forceinline__ uint32_t packed(float x, float y, const ProductScale& s) {
  unpack2(mul2(mul2(pack2(x, y), pack2(s.a, s.a)), pack2(s.b, s.b)), x, y);
  return packed<T>(x, y);
}
// 32 tokens of one weight row: y + j * ldy receives v[j] * scale, j < n
template <typename T>
__device__ __forceinline__ void store_tokens(T* y, int64_t ldy, int n, const ProductScale& scale, const float (&v)[32]) {
  if (n >= 32) {
#pragma unroll
    for (int j = 0; j < 32; ++j) { put(y, v[j] * scale); y += ldy; }
  } else {
#pragma unroll
    for (int j = 0; j < 32; ++j) { if (j < n) put(y, v[j] * scale); y += ldy; }
  }
}
// After a wait that ran out: time for the copies already issued to land before shared memory goes away
// (they take microseconds).
__device__ __forceinline__ void let_copies_land() {
  const long long t0 = clock64();
  while (clock64() - t0 < (1 << 20)) {}
}

// The MMAs of one stage: scale tiles to TMEM, then the 64-column steps that hold columns of the matrix
// (beyond them scales need not exist).  Addresses are shared-memory addresses in units of 16 bytes, added to
// constant descriptors.  PAIR and NVFP4: in two halves that use the same TMEM columns in turn (the copies and
// MMAs of one thread execute in order), so that a stage's scales fit into 32 columns.
template <int FORMAT, bool PAIR>
__device__ __forceinline__ void issue_stage(uint32_t d, uint32_t sf_tmem, uint32_t w, uint32_t a, uint32_t ws, uint32_t id0,
                                            uint32_t id1, int steps, bool first) {
  constexpr bool NV = FORMAT == ADADIM_NVFP4;
  constexpr uint32_t kSf16 = sf_stage_bytes(FORMAT) / 16, kTile16 = kSfTileBytes / 16;
  constexpr int kSfTiles = sf_stage_bytes(FORMAT) / kSfTileBytes;    // scale tiles of a stage: 4 or 2
  constexpr uint64_t desc = ptx::smem_desc_sw128(16, 1024);          // K-major: 8-row groups 1024 bytes apart
  constexpr uint64_t sf_desc = ptx::smem_desc_plain(16, 128);
  constexpr int kTok = PAIR ? 8 : 4;                                 // TMEM columns of one step's token scales
  constexpr int kHalves = PAIR && NV ? 2 : 1, kTilesPer = kSfTiles / kHalves, kTokAt = 4 * kTilesPer;
  auto copy = [&](int j) {                                           // scale tile j of the stage
    const int at = j % kTilesPer;
    ptx::tmem_cp_scales<PAIR>(sf_tmem + at * 4, sf_desc + ws + j * kTile16);
    ptx::tmem_cp_scales<PAIR>(sf_tmem + kTokAt + at * kTok, sf_desc + ws + kSf16 + j * kTile16);
    if (PAIR) ptx::tmem_cp_scales<PAIR>(sf_tmem + kTokAt + at * kTok + 4, sf_desc + ws + 2 * kSf16 + j * kTile16);
  };
  auto step = [&](int j) {
    const int at = (NV ? j : j / 2) % kTilesPer;
    ptx::mma_fp4<NV, PAIR>(d, desc + w + j * 2, desc + a + j * 2, (j & 1) ? id1 : id0, sf_tmem + at * 4,
                           sf_tmem + kTokAt + at * kTok, !(first && j == 0));
  };
#pragma unroll
  for (int h = 0; h < kHalves; ++h) {
#pragma unroll
    for (int j = 0; j < kTilesPer; ++j) copy(h * kTilesPer + j);
#pragma unroll
    for (int j = h * 4 / kHalves; j < (h + 1) * 4 / kHalves; ++j)
      if (j < steps) step(j);
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
                const __grid_constant__ CUtensorMap tmWs, const __grid_constant__ CUtensorMap tmAs,
                const __grid_constant__ CUtensorMap tmY, const MmParams p) {
  constexpr bool NV = FORMAT == ADADIM_NVFP4;
  constexpr uint32_t kSf = sf_stage_bytes(FORMAT);
  constexpr int kSfTiles = kSf / kSfTileBytes;
  // TMEM: two accumulators and 32 columns of scales.  240 tokens: side by side.  256 tokens: they share 32
  // columns, which the epilogue drains first and the next tile's MMAs wait for.
  constexpr uint32_t kSfCol = 480;
  const bool sharing = p.n_tile > 240;
  const uint32_t acc_step = sharing ? 224 : 240;

  extern __shared__ uint8_t smem_raw[];
  const uint32_t smem_at = (ptx::smem_addr(smem_raw) + 1023u) & ~1023u;      // shared-memory address of the ring
  uint8_t* smem = smem_raw + (smem_at - ptx::smem_addr(smem_raw));
  __shared__ uint64_t full[kMaxStages], empty[kMaxStages], acc_full[2], acc_empty[2], part_empty;
  __shared__ int stage_n[kMaxStages];                  // tokens of the tile a stage belongs to, from the producer
  __shared__ uint32_t tmem_slot;
  __shared__ int dead_word;
  volatile int* dead = &dead_word;
  const int warp = ptx::uniform_warp(), lane = threadIdx.x & 31;
  const uint32_t rank = ptx::cluster_ctarank();
  const uint32_t stage_size = stage_bytes(FORMAT, true, p.n_tile);
  const uint32_t a_bytes = static_cast<uint32_t>(p.n_tile) * 64;
  const uint32_t out_at = smem_at + p.n_stages * stage_size;                  // [4 warp pairs][2][32 tokens][128 bytes]
  int* prefix = reinterpret_cast<int*>(smem + p.n_stages * stage_size + kOutBytes);      // [n_experts + 1], grouped only
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
    TileWalk walk = {};
    for (int t = pair0; t < num_tiles && ok; t += pairs) {
      const Tile x = walk.next(t, pairs, num_tiles, p, prefix);
      const int half = ((x.count + 15) & ~15) >> 1;    // tokens of this CTA
      const int w_row = static_cast<int>(x.e * p.out + x.m) + static_cast<int>(rank) * 128;
      const int a_row = x.row + static_cast<int>(rank) * half;
      int w_sf = static_cast<int>((x.e * p.w_sf_rows + x.m / kSfRows + rank) * p.n_sf * 4);
      int a_sf0 = static_cast<int>(x.a_sf_row * p.n_sf * 4), a_sf1 = a_sf0 + static_cast<int>(p.n_sf * 4);
      for (int k = 0; k < p.num_k; ++k) {
        ok = ptx::mbar_wait_warp(&empty[stage], phase ^ 1u, dead, p.status_dev);
        if (!ok) break;
        uint8_t* w_dst = smem + stage * stage_size;
        uint8_t* a_dst = w_dst + kWBytes;
        uint8_t* ws_dst = a_dst + a_bytes;
        const uint32_t bar = ptx::map_to_cta(ptx::smem_addr(&full[stage]), 0);
        if (ptx::elect_one()) {
          // one barrier, the leader's, counts both CTAs' bytes
          if (rank == 0) {
            stage_n[stage] = 2 * half;
            ptx::mbar_arrive_expect_tx(&full[stage], 2 * stage_size);
          }
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
        uint32_t id0 = 0, id1 = 0;
        ok = ptx::mbar_wait_warp(&acc_empty[buf], acc_phase ^ 1u, dead, p.status_dev);
        if (ok && sharing && t != pair0) {             // the tile before has left the shared columns
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
          const bool next = ptx::mbar_test(&full[stage], phase);
          if (k == 0) {
            const int n = __shfl_sync(0xffffffffu, stage_n[cur], 0);
            id0 = ptx::idesc_fp4(256, n, !NV, 0);
            id1 = ptx::idesc_fp4(256, n, !NV, NV ? 0 : 2);
          }
          const uint32_t w16 = (smem_at + cur * stage_size) >> 4;
          const int steps = steps_of(p.in, k);
          if (ptx::elect_one()) {
            issue_stage<FORMAT, true>(tmem + buf * acc_step, tmem + kSfCol, w16, w16 + kWBytes / 16,
                                      w16 + (kWBytes + a_bytes) / 16, id0, id1, steps, k == 0);
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
    const int side = (warp - 2) >> 2;                  // of each 64 columns, the 32 that this warp takes
    int buf = 0;
    uint32_t acc_phase = 0;
    const ProductScale scale = product_scale<NV>(p);
    const uint32_t part_bar = ptx::map_to_cta(ptx::smem_addr(&part_empty), 0);
    auto give_back = [&]() {
      ptx::tc_fence_before_sync();
      __syncwarp();
      if (lane == 0) ptx::mbar_arrive_cluster(part_bar);
    };
    const bool bulk_y = sizeof(T) == 2 && p.bulk_y;
    int out_buf = 0;
    const int out_id = 1 + side * 2 + (q >> 1);        // named barrier of the warp pair
    TileWalk walk = {};
    for (int t = pair0; t < num_tiles; t += pairs) {
      const Tile x = walk.next(t, pairs, num_tiles, p, prefix);
      bool ok = ptx::mbar_wait_warp(&acc_full[buf], acc_phase, dead, p.status_dev);
      if (bulk_y) ok = ptx::named_all(out_id, 64, ok);                        // both warps of a pair go on, or neither
      if (!ok) break;
      ptx::tc_fence_after_sync();
      const int64_t o = x.m + static_cast<int>(rank) * 128 + q * 32 + lane;
      T* y = static_cast<T*>(p.Y) + static_cast<int64_t>(x.row) * p.ldy + o;
      const uint32_t acc = tmem + (static_cast<uint32_t>(q * 32) << 16) + buf * acc_step;
      // Columns c .. c + 31 of the accumulator.  Results of 16 bits leave through shared memory, 64 weight rows of
      // 16 tokens by a pair of warps as a bulk store: 64-byte stores from registers held up the loads of the
      // next tile's operands (2048 tokens x W[11008,4096]: a tile of 7700 cycles took 9200).
      auto drain = [&](int c, bool hand_back) {
        const int left = x.count - c;
        // the matrix's last tile may be cut anywhere (what lies behind the matrix is not written), others at 16
        if (left > 0 && bulk_y && (left >= 32 || left == 16 || (p.n_experts == 0 && x.row + x.count == p.rows))) {
          float lo[16], hi[16];
          ptx::tmem_ld_fragments(acc + c, lo, hi);
          if (hand_back) give_back();
          if (lane == 0 && (q & 1) == 0) ptx::bulk_wait_read_but_one();       // this buffer's last store has read it
          ptx::named_sync(out_id, 64);
          const uint32_t tile = out_at + (side * 4 + (q >> 1) * 2 + out_buf) * 4096;
          const uint32_t unit = (q & 1) * 4 + (lane >> 3);                    // 16 bytes: eight weight rows
#pragma unroll
          for (int u = 0; u < 4; ++u) {
            const int token = u * 8 + (lane & 7);
            ptx::stmatrix_trans(tile + token * 128 + ((unit ^ (token & 7)) << 4), packed<T>(lo[4 * u], lo[4 * u + 1], scale),
                                packed<T>(lo[4 * u + 2], lo[4 * u + 3], scale),
                                packed<T>(hi[4 * u], hi[4 * u + 1], scale),
                                packed<T>(hi[4 * u + 2], hi[4 * u + 3], scale));
          }
          ptx::fence_proxy_async();
          ptx::named_sync(out_id, 64);
          const int y_col = x.m + static_cast<int>(rank) * 128 + (q >> 1) * 64;
          if (lane == 0 && (q & 1) == 0) {
            if (y_col < p.out) {
              ptx::tma_store_2d(&tmY, y_col, x.row + c, tile);
              if (left > 16) ptx::tma_store_2d(&tmY, y_col, x.row + c + 16, tile + 16 * 128);
            }
            ptx::bulk_commit();
          }
          out_buf ^= 1;
        } else {
          float v[32];
          if (left > 0) ptx::tmem_ld32(acc + c, v);
          if (hand_back) give_back();
          if (left > 0 && o < p.out) store_tokens(y + c * p.ldy, p.ldy, left, scale, v);
        }
      };
      int done = -1;                                   // the shared columns, taken first by half of the warps
      if (sharing) {
        const int c = buf == 0 ? 224 : 0;
        if (side == (c >> 5 & 1)) {
          done = c;
          drain(c, true);
        } else {
          give_back();
        }
      }
#pragma unroll 1
      for (int c = side * 32; c < x.count; c += 64)
        if (c != done) {
          drain(c, false);
          if (p.pace_ns > 0 && t + pairs < num_tiles) __nanosleep(p.pace_ns);
        }
      ptx::tc_fence_before_sync();
      __syncwarp();
      if (lane == 0) ptx::mbar_arrive_cluster(ptx::map_to_cta(ptx::smem_addr(&acc_empty[buf]), 0));
      buf ^= 1;
      if (buf == 0) acc_phase ^= 1u;
    }
    if (bulk_y && lane == 0) ptx::bulk_wait_all();     // every store is complete before the CTA ends
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
// Tokens that one CTA of a cluster of `splits` finishes: a multiple of four, the last CTAs may have none.
__host__ __device__ __forceinline__ int tokens_of_cta(int count, int splits) {
  return ((count + splits - 1) / splits + 3) & ~3;
}
// floats that a CTA receives: for each of its tokens and each CTA, 128 rows
__host__ __device__ __forceinline__ int exchange_floats(int n_tile, int splits) {
  return splits > 1 ? tokens_of_cta(n_tile, splits) * splits * 128 : 0;
}

// FUSED: the activations are p.x, of type T, and eight warps (the epilogue's four among them) quantize
// them into the ring; there is one tile of up to kFusedTokens tokens, dense, and a warp takes two of them.
template <int FORMAT, typename T, bool FUSED>
__global__ void __launch_bounds__(FUSED ? kFusedThreads : kThreads, FUSED ? kFusedPerSm : 4)
fp4_split_kernel(const __grid_constant__ CUtensorMap tmW, const __grid_constant__ CUtensorMap tmA,
                 const __grid_constant__ CUtensorMap tmWs, const __grid_constant__ CUtensorMap tmAs,
                 const __grid_constant__ CUtensorMap, const MmParams p) {
  constexpr bool NV = FORMAT == ADADIM_NVFP4;
  constexpr uint32_t kSf = sf_stage_bytes(FORMAT);
  constexpr int kSfTiles = kSf / kSfTileBytes;

  extern __shared__ uint8_t smem_raw[];
  const uint32_t smem_at = (ptx::smem_addr(smem_raw) + 1023u) & ~1023u;      // shared-memory address of the ring
  uint8_t* smem = smem_raw + (smem_at - ptx::smem_addr(smem_raw));
  __shared__ uint64_t full[kMaxStages], empty[kMaxStages], acc_full, red_full;
  __shared__ uint32_t tmem_slot;
  __shared__ int dead_word;
  volatile int* dead = &dead_word;
  const int warp = ptx::uniform_warp(), lane = threadIdx.x & 31;
  const uint32_t stage_size = stage_bytes(FORMAT, false, p.n_tile);
  const uint32_t a_bytes = static_cast<uint32_t>(p.n_tile) * 128;
  float4* red = reinterpret_cast<float4*>(smem + p.n_stages * stage_size);   // [CTA][4 tokens][128 rows]
  int* prefix = reinterpret_cast<int*>(red + exchange_floats(p.n_tile, p.splits) / 4);      // [n_experts + 1], grouped only
  // grid: x / splits is the token tile and y the weight tile (grouped: x / splits numbers both); splits is a power of two
  const int rank = blockIdx.x & (p.splits - 1), t = static_cast<int>(blockIdx.x) >> (__ffs(p.splits) - 1);
  const int k0 = p.num_k * rank / p.splits, k1 = p.num_k * (rank + 1) / p.splits;
  const uint32_t sf_col = p.n_tile;                    // TMEM: an accumulator of n_tile columns, then scales of two stages

  Tile x = {};
  bool work = true;
  if (!FUSED && p.n_experts > 0) {
    if (warp == 2) tile_prefix(p, lane, prefix);
    __syncthreads();
    work = t < prefix[p.n_experts];       // the grid is an upper bound
    if (work) x = tile_of_group(t, p, prefix);
  } else {
    x = tile_at(t, blockIdx.y, 0, 0, p.rows, p);
  }
  const int mine = tokens_of_cta(x.count, p.splits);   // tokens finished here: [rank * mine, + tokens)
  const int tokens = max(0, min(mine, x.count - rank * mine));

  const int w_row = static_cast<int>(x.e * p.out + x.m);
  const int w_sf = static_cast<int>((x.e * p.w_sf_rows + x.m / kSfRows) * p.n_sf * 4);
  const int a_sf = static_cast<int>(x.a_sf_row * p.n_sf * 4);
  auto load_w = [&](int k, int stage) {
    uint8_t* w_dst = smem + stage * stage_size;
    if (ptx::elect_one()) {
      ptx::mbar_arrive_expect_tx(&full[stage], FUSED ? kWBytes + kSf : stage_size);
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
  const int ahead = work ? min(k1 - k0, p.n_stages) : 0;
  // FUSED: warps that share a stage (two tokens each), and stages under way at once.  Not more than the ring
  // has: a warp's wait for its next place would otherwise be two phases of that barrier ahead.
  const int sharing = x.count > 4 ? 4 : x.count > 2 ? 2 : 1;
  const int in_turn = min(8 / sharing, p.n_stages);
  if (warp == 0) {
    // the ring's first fill starts before anything else: the weight does not depend on the launch ahead
    if (ptx::elect_one()) {
      for (int s = 0; s < p.n_stages; ++s) { ptx::mbar_init(&full[s], FUSED ? 1 + sharing : 1); ptx::mbar_init(&empty[s], 1); }
      ptx::mbar_init(&acc_full, 1);
      ptx::mbar_init(&red_full, 1);
      dead_word = 0;
      ptx::fence_mbar_init();
      if (p.splits > 1) ptx::mbar_arrive_expect_tx(&red_full, static_cast<uint32_t>(p.splits * ((tokens + 3) / 4) * 128 * 16));
    }
    __syncwarp();
    for (int i = 0; i < ahead; ++i) load_w(k0 + i, i);
  }
  if (p.splits > 1) ptx::cluster_arrive();             // waited for before the first word goes to another CTA
  if (warp == 1) {
    ptx::tmem_alloc(&tmem_slot, p.tmem_cols);
    ptx::tmem_relinquish();
  }
  ptx::tc_fence_before_sync();
  __syncthreads();
  ptx::tc_fence_after_sync();
  const uint32_t tmem = tmem_slot;

  if (warp == 0) {
    // ------------------------------------------------------------------ TMA producer
    if (!FUSED) {
      ptx::pdl_wait();
      for (int i = 0; i < ahead; ++i) load_a(k0 + i, i);
    }
    int stage = 0;
    uint32_t phase = 0;
    bool ok = true;
    for (int k = k0 + ahead; k < k1 && work; ++k) {
      ok = ptx::mbar_wait_warp(&empty[stage], phase, dead, p.status_dev);
      if (!ok) break;
      load_w(k, stage);
      if (!FUSED) load_a(k, stage);
      if (++stage == p.n_stages) { stage = 0; phase ^= 1u; }
    }
    if (!ok) let_copies_land();
  } else if (warp == 1) {
    // ------------------------------------------------------------------ MMA issuer
    if (work) {
      const int n = (x.count + 15) & ~15;
      const uint32_t id0 = ptx::idesc_fp4(128, n, !NV, 0), id1 = ptx::idesc_fp4(128, n, !NV, NV ? 0 : 2);
      int stage = 0;
      uint32_t phase = 0;
      bool ok = true, ready = false;
      for (int k = k0; k < k1; ++k) {
        if (!ready) ok = ptx::mbar_wait_warp(&full[stage], phase, dead, p.status_dev);
        if (!ok) break;
        ptx::tc_fence_after_sync();
        const int cur = stage;
        if (++stage == p.n_stages) { stage = 0; phase ^= 1u; }
        // asked before this stage's instructions are issued: the answer is there when they are
        const bool next = ptx::mbar_test(&full[stage], phase);
        const uint32_t w16 = (smem_at + cur * stage_size) >> 4;
        const int steps = steps_of(p.in, k);
        if (ptx::elect_one()) {
          issue_stage<FORMAT, false>(tmem, tmem + sf_col + (k & 1) * 32, w16, w16 + kWBytes / 16,
                                     w16 + (kWBytes + a_bytes) / 16, id0, id1, steps, k == k0);
          ptx::mma_commit(&empty[cur]);
          if (k == k1 - 1) ptx::mma_commit(&acc_full);
        }
        ready = __all_sync(0xffffffffu, next) != 0;
      }
      if (!ok) let_copies_land();
    }
  } else if (work) {
    if (FUSED) {
      // ---------------------------------------------------------------- quantizer (warps 2..9)
      // 16 columns of a token per lane, two tokens across the lanes; the next stage's are loaded while this
      // one's are worked on.  Rows behind `count` are left as they are in the ring: what they give lands in
      // columns of the accumulator that nobody reads.
      const int group = (warp - 2) / sharing, chunk = lane & 15;
      const int r = ((warp - 2) - group * sharing) * 2 + (lane >> 4);
      const T* at = static_cast<const T*>(p.x.X) + static_cast<int64_t>(r < x.count ? x.row + r : 0) * p.x.ldx;
      const int t_log2 = NV ? tensor_scale_log2(p.a_amax) : 0;
      const uint32_t a_at = r * 128 + (((chunk >> 1) ^ (r & 7)) << 4) + (chunk & 1) * 8;
      const int blk = NV ? chunk : chunk >> 1;
      const uint32_t s_at = (blk >> 2) * kSfTileBytes + r * 16 + (blk & 3);
      Raw<T> next;
      auto load = [&](int i) {
        const int64_t c0 = static_cast<int64_t>(k0 + i) * kKT + chunk * kPer;
        if (r < x.count && c0 < p.in) load16_aligned(at + c0, next);
        else
#pragma unroll
          for (uint32_t& w : next.w) w = 0;
      };
      if (group < in_turn) load(group);
      int slot = group;
      uint32_t phase = 0;
      for (int i = group; group < in_turn && i < k1 - k0; i += in_turn) {
        float v[kPer];
        uint32_t top = widen(next, v);
        load(i + in_turn);
        if (!NV) top = max(top, __shfl_xor_sync(0xffffffffu, top, 1));
        const BlockScale b = block_scale<FORMAT, sizeof(T) == 2>(__uint_as_float(top), t_log2);
        uint2 c;
        c.x = codes8<FORMAT, sizeof(T) == 2>(v, b);
        c.y = codes8<FORMAT, sizeof(T) == 2>(v + 8, b);
        if (!ptx::mbar_wait_warp(&empty[slot], phase ^ 1u, dead, p.status_dev)) break;
        uint8_t* a_dst = smem + slot * stage_size + kWBytes;
        if (r < x.count) {
          *reinterpret_cast<uint2*>(a_dst + a_at) = c;
          if (NV || (chunk & 1) == 0) (a_dst + a_bytes + kSf)[s_at] = static_cast<uint8_t>(b.byte);
        }
        ptx::fence_proxy_async();
        __syncwarp();
        if (lane == 0) ptx::mbar_arrive(&full[slot]);
        slot += in_turn;
        if (slot >= p.n_stages) { slot -= p.n_stages; phase ^= 1u; }
      }
    }
    if (warp < 6) {
    // ------------------------------------------------------------------ epilogue (warps 2..5)
    const int q = warp & 3;                            // TMEM lane quadrant this warp may read
    const ProductScale scale = product_scale<NV>(p);
    const int row = q * 32 + lane;
    const int64_t o = x.m + row;
    T* y = static_cast<T*>(p.Y) + static_cast<int64_t>(x.row) * p.ldy + o;
    const uint32_t acc = tmem + (static_cast<uint32_t>(q * 32) << 16);
    if (p.splits > 1) ptx::cluster_wait();             // the other CTAs have set up their barriers
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
      // tokens in fours: CTA c / mine finishes token c, and every CTA sends it its partial sums
      const uint32_t red_addr = ptx::smem_addr(red), bar_addr = ptx::smem_addr(&red_full);
      const int fours = mine / 4;
#pragma unroll 1
      for (int c = 0; c < x.count && ok; c += 32) {
        float v[32];
        ptx::tmem_ld32(acc + c, v);
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          const int four = c / 4 + j;
          if (four * 4 < x.count) {
            const int dst = four / fours, slot = four - dst * fours;
            ptx::st_async_v4(ptx::map_to_cta(red_addr + ((rank * fours + slot) * 128 + row) * 16, dst), v[4 * j], v[4 * j + 1],
                             v[4 * j + 2], v[4 * j + 3], ptx::map_to_cta(bar_addr, dst));
          }
        }
      }
      ok = ptx::mbar_wait_warp_cluster(&red_full, 0, dead, p.status_dev) && ok;
      y += rank * mine * p.ldy;
      for (int f = 0; f * 4 < tokens && ok; ++f) {
        float4 s = red[f * 128 + row];
        for (int k = 1; k < p.splits; ++k) {
          const float4 v = red[(k * fours + f) * 128 + row];
          s.x += v.x; s.y += v.y; s.z += v.z; s.w += v.w;
        }
        if (o < p.out) {
          put(y, s.x * scale);
          if (f * 4 + 1 < tokens) put(y + p.ldy, s.y * scale);
          if (f * 4 + 2 < tokens) put(y + 2 * p.ldy, s.z * scale);
          if (f * 4 + 3 < tokens) put(y + 3 * p.ldy, s.w * scale);
        }
        y += 4 * p.ldy;
      }
    }
    }
  }

  if (p.splits > 1) {
    if (warp < 2 || warp >= 6 || !work) ptx::cluster_wait();
    ptx::cluster_arrive();                             // no CTA leaves while another may still write to it
    ptx::cluster_wait();
  }
  ptx::tc_fence_before_sync();
  __syncthreads();
  if (warp == 1) {
    ptx::tc_fence_after_sync();
    ptx::tmem_dealloc(tmem, p.tmem_cols);
  }
}

constexpr size_t kSmem = 220 * 1024;                   // dynamic shared memory of one SM's split CTAs
constexpr size_t kSmemPair = 226 * 1024 - 512;         // and of a pair CTA
// A split CTA takes at least so much shared memory for each TMEM column: an SM's shared memory (228 KB) then runs
// out before its 512 columns do.  A CTA that had to wait for columns could keep its cluster waiting, whose other
// CTAs hold columns that another cluster needs, of this kernel or of one on another stream.
constexpr size_t kSmemPerTmemColumn = 368;
static_assert(kSmemPerTmemColumn * (512 + 128) > 228 * 1024, "one CTA more than the columns allow must not fit");

// ---- host: tensor maps ----------------------------------------------------------------------------
// A 2-D tensor of `inner` elements per row with boxes of {box_inner, box_rows}, outside of which 0 is read.
int encode(CUtensorMap* map, CUtensorMapDataType type, const void* base, uint64_t inner, uint64_t rows, uint64_t pitch_bytes,
           uint32_t box_inner, uint32_t box_rows, CUtensorMapSwizzle swizzle, CUtensorMapL2promotion promotion) {
  typedef decltype(&cuTensorMapEncodeTiled) Fn;
  static const Fn fn = []() -> Fn {
    void* p = nullptr;
    cudaDriverEntryPointQueryResult q;
    if (cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &p, cudaEnableDefault, &q) != cudaSuccess) return nullptr;
    return q == cudaDriverEntryPointSuccess ? reinterpret_cast<Fn>(p) : nullptr;
  }();
  if (fn == nullptr) return ADADIM_ERR_CUDA;
  const cuuint64_t dims[2] = {inner, rows}, strides[1] = {pitch_bytes};
  const cuuint32_t box[2] = {box_inner, box_rows}, step[2] = {1, 1};
  return fn(map, type, 2, const_cast<void*>(base), dims, strides, box, step, CU_TENSOR_MAP_INTERLEAVE_NONE, swizzle, promotion,
            CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS ? ADADIM_OK : ADADIM_ERR_CUDA;
}
// 16-bit elements with 128-byte swizzle, for stores.
int make_tmap_u16(CUtensorMap* map, const void* base, uint64_t inner, uint64_t rows, uint64_t pitch_bytes, uint32_t box_rows) {
  return encode(map, CU_TENSOR_MAP_DATA_TYPE_UINT16, base, inner, rows, pitch_bytes, 64, box_rows, CU_TENSOR_MAP_SWIZZLE_128B,
                CU_TENSOR_MAP_L2_PROMOTION_NONE);
}
// Bytes with 128-byte swizzle (packed codes) or without (scale tiles as 128-byte rows).
int make_tmap_u8(CUtensorMap* map, const void* base, uint64_t inner, uint64_t rows, uint64_t pitch_bytes, uint32_t box_rows,
                 bool swizzle) {
  return encode(map, CU_TENSOR_MAP_DATA_TYPE_UINT8, base, inner, rows, pitch_bytes, 128, box_rows,
                swizzle ? CU_TENSOR_MAP_SWIZZLE_128B : CU_TENSOR_MAP_SWIZZLE_NONE, CU_TENSOR_MAP_L2_PROMOTION_L2_256B);
}

template <auto KERNEL>
int launch(const CUtensorMap (&tm)[5], const MmParams& p, dim3 grid, int threads, int cluster, size_t smem, bool chained,
           cudaStream_t st) {
  static std::atomic<uint64_t> done{0};
  const int rc = set_once(KERNEL, cudaFuncAttributeMaxDynamicSharedMemorySize, static_cast<int>(kSmemPair), done);
  if (rc != ADADIM_OK) return rc;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = grid;
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
  ADADIM_CUDA_TRY(cudaLaunchKernelEx(&cfg, KERNEL, tm[0], tm[1], tm[2], tm[3], tm[4], p));
  return ADADIM_OK;
}

template <typename T>
int launch_format(bool pair, bool fused, int format, const CUtensorMap (&tm)[5], const MmParams& p, dim3 grid, size_t smem, bool chained,
                  cudaStream_t st) {
  if (pair) return format == ADADIM_MXFP4 ? launch<fp4_pair_kernel<ADADIM_MXFP4, T>>(tm, p, grid, kPairThreads, 2, smem, chained, st)
                                          : launch<fp4_pair_kernel<ADADIM_NVFP4, T>>(tm, p, grid, kPairThreads, 2, smem, chained, st);
  if (fused) return format == ADADIM_MXFP4 ? launch<fp4_split_kernel<ADADIM_MXFP4, T, true>>(tm, p, grid, kFusedThreads, p.splits, smem, false, st)
                                           : launch<fp4_split_kernel<ADADIM_NVFP4, T, true>>(tm, p, grid, kFusedThreads, p.splits, smem, false, st);
  return format == ADADIM_MXFP4 ? launch<fp4_split_kernel<ADADIM_MXFP4, T, false>>(tm, p, grid, kThreads, p.splits, smem, chained, st)
                                : launch<fp4_split_kernel<ADADIM_NVFP4, T, false>>(tm, p, grid, kThreads, p.splits, smem, chained, st);
}

// Tiles of fewer tokens than 128 are cut no lower than this, and only up to so many rows (of a typical
// expert), which bounds the scale tiles of the activations.
constexpr int kMinCut = 32, kMaxCutRows = 512;
constexpr int kMinPairTile = 160;                      // the pair kernel's lowest token tile, two scale tile rows
// kFusedTokens, the rows up to which a dense product quantizes them itself: every weight tile's CTA repeats the work, which at
// 8 rows hides behind the weight's bytes and at 16 does not (16 x W[28672,8192]: 35.3 us fused, 24.5 us behind
// the quantizer; 8 x W[4096,4096]: 6.7 and 7.4 us).  Where the weight is in L2 it does not quite at 8 either (8 x
// W[11008,4096]: 11.6 us, 16 behind the quantizer 10.3 us).  Not with experts, some of which have more rows than the
// typical one (128 rows over 32: 27.4 us fused, 25.0 us behind the quantizer).
static_assert(kFusedTokens <= 8, "the quantizing warps take two tokens each, up to four warps to a stage");

// The plan of least estimated time, in nanoseconds.  What the estimate is made of was measured on the
// kernels (1.9 GHz, 148 SMs); over a sweep of 25 shapes its choice was within a tenth of the best plan's time.
//   pair   a 256-column stage of a 256 x n tile takes 270 n / 256, and a CTA takes in no more than 130 bytes
//          a nanosecond; a tile 1000 on top, 1500 where its accumulators share columns; start and end 5000;
//          it streams a weight no faster than 1 / 1.7 of the split kernel.
//   split  a CTA's stage takes no less than 300 whatever its size, an SM takes in 80 bytes a nanosecond; start
//          and end 4000, an exchange between the CTAs of a cluster 1500 + 15 a token; and in all no less than
//          the weights' bytes at 6000 a nanosecond.
//   The result's bytes leave at 5000 (pair) or 2500 (split) a nanosecond, hardly beside the rest.
Fp4Plan plan_of(int64_t rows, int64_t out, int64_t in, int n_experts, int format, bool quantized, bool fuse, int sms) {
  const int64_t weights = n_experts > 0 ? (n_experts < rows ? n_experts : rows) : 1;
  const int64_t typical = (rows + weights - 1) / weights;            // rows of one expert if they were equal
  const int64_t num_k = (in + kKT - 1) / kKT;
  // tiles of an expert's rows: experts are not equal, which costs half a tile each, or with few rows takes some of
  // them a tile further
  auto token_tiles = [&](int64_t n) {
    if (n_experts == 0) return (rows + n - 1) / n;
    return typical > 2 * n ? (weights * typical + weights * n / 2) / n : weights * ((typical + typical / 2 + n - 1) / n);
  };
  Fp4Plan best = {true, 256, 1, 1, false};
  double best_ns = 1e300;
  const double floor_ns = static_cast<double>(weights * out) * static_cast<double>(in) * (format == ADADIM_MXFP4 ? 0.53125 : 0.5625) / 6000.0;
  const double y_bytes = 2.0 * static_cast<double>(rows) * static_cast<double>(out);
  for (int n_tile = 256; n_tile >= (quantized ? 256 : kMinPairTile); n_tile -= 16) {
    const int64_t tiles = (out + 255) / 256 * token_tiles(n_tile), waves = (tiles + sms / 2 - 1) / (sms / 2);
    const double n = typical < n_tile ? static_cast<double>((typical + 15) / 16 * 16) : n_tile;
    const double bytes = stage_bytes(format, true, n_tile) / 130.0, stage = 1.055 * n < bytes ? bytes : 1.055 * n;
    double ns = static_cast<double>(waves) * (static_cast<double>(num_k) * stage + (n_tile > 240 ? 1500.0 : 1000.0));
    if (ns < 1.7 * floor_ns) ns = 1.7 * floor_ns;
    ns += 5000.0 + y_bytes / 5000.0;
    if (ns < best_ns) { best_ns = ns; best.n_tile = n_tile; }
  }
  for (int n_tile = 16; n_tile <= 128; n_tile *= 2) {
    // lower tiles than 128 rows: only where they are the only ones, or the scales are laid out for them
    const bool fused = fuse && n_experts == 0 && n_tile <= kFusedTile && rows <= kFusedTokens;
    if (n_tile < 128 && rows > n_tile && (quantized || (n_tile < kMinCut && !fused) || typical > kMaxCutRows)) continue;
    if (n_tile > 16 && n_tile / 2 >= rows) break;
    const int64_t tiles = (out + 127) / 128 * token_tiles(n_tile);
    const size_t per = stage_bytes(format, false, n_tile);
    for (int splits = 1; splits <= 8 && splits <= num_k; splits *= 2) {
      const int64_t ctas = tiles * splits, k = (num_k + splits - 1) / splits;
      const size_t fixed = exchange_floats(n_tile, splits) * 4 + 1024 + static_cast<size_t>(n_experts + 1) * 4;
      const int stages = static_cast<int>(k < 3 ? k : 3);
      const int most = fused ? kFusedPerSm : 4;
      int per_sm = static_cast<int>((ctas + sms - 1) / sms < most ? (ctas + sms - 1) / sms : most);
      // clusters find their SMs more easily when they need not be empty (64 x W[1024,12288] over 8: 12.8 -> 8.5 us)
      if (splits > 1 && per_sm < 2) per_sm = 2;
      while (per_sm > 1 && (per_sm * (stages * per + fixed + 1024) > kSmem || per_sm * (n_tile <= 64 ? 128 : 256) > 512)) --per_sm;
      if (stages * per + fixed + 1024 > kSmem) continue;
      const int64_t waves = (ctas + static_cast<int64_t>(per_sm) * sms - 1) / (static_cast<int64_t>(per_sm) * sms);
      const double latency = static_cast<double>(waves) * static_cast<double>(k) * 300.0;
      const double bytes = static_cast<double>(ctas) / sms * static_cast<double>(k) * static_cast<double>(per) / 80.0;
      double ns = latency > bytes ? latency : bytes;
      if (ns < floor_ns) ns = floor_ns;
      ns += 4000.0 + y_bytes / 2500.0 + (splits > 1 ? 1500.0 + 15.0 * n_tile : 0.0);
      if (ns < best_ns) { best_ns = ns; best = {false, n_tile, splits, per_sm, fused}; }
    }
  }
  return best;
}

constexpr int kSms = 148;

}  // namespace

Fp4Plan fp4_plan(int64_t rows, int64_t out, int64_t in, int n_experts, int format, bool quantized, bool fuse) {
  return plan_of(rows, out, in, n_experts, format, quantized, fuse, kSms);
}

int64_t fp4_most_tile_rows(int64_t rows, int n_experts) {
  const int64_t groups = n_experts > 0 ? n_experts : 1;
  if (rows == 0) return 0;
  const int lowest = rows <= kMaxCutRows * groups ? kMinCut : kMinPairTile / 2;      // rows a tile row has at least, but for ends
  return rows / lowest + 2 * groups + 2;
}

int fp4_matmul_launch(const Fp4Plan& plan, const adadim_fp4tensor& A, int lt, const fp4::Source& x, int64_t n_rows,
                      const int32_t* offsets, int n_experts, const adadim_fp4tensor& B, int64_t out, int64_t in, int format, void* Y, int ydtype,
                      int64_t ldy, int* status_dev, bool chained, cudaStream_t st) {
  const bool pair = plan.pair;
  MmParams p = {};
  p.out = out;
  p.in = in;
  p.rows = static_cast<int>(n_rows);
  p.n_experts = n_experts;
  p.offsets = offsets;
  p.n_tile = plan.n_tile;
  p.lt = lt;
  p.lt_per_tile = plan.n_tile / lt;
  p.sub = static_cast<int>((lt + kSfRows - 1) / kSfRows);
  p.x = x;
  p.splits = plan.splits;
  p.num_k = static_cast<int>((in + kKT - 1) / kKT);
  p.n_sf = sf_tiles(format, in);
  p.w_sf_rows = sf_tile_rows(out, 0);
  p.Y = Y;
  p.ldy = ldy;
  p.a_amax = A.amax;
  p.b_amax = B.amax;
  p.status_dev = status_dev;
  p.m_tiles = static_cast<int>((out + (pair ? 255 : 127)) / (pair ? 256 : 128));
  // dense: the tiles are known here; grouped: at most one partial tile for every expert on top
  int64_t token_tiles = (n_rows + p.n_tile - 1) / p.n_tile;
  if (n_experts > 0) token_tiles += n_experts < n_rows ? n_experts : n_rows;
  const int64_t tiles = token_tiles * p.m_tiles;

  const int64_t weights = n_experts > 0 ? n_experts : 1;
  const uint64_t inner = static_cast<uint64_t>((in + 1) / 2);
  const uint32_t sf_box = sf_stage_bytes(format) / 128;
  CUtensorMap tm[5];
  int rc;
  if ((rc = make_tmap_u8(&tm[0], B.codes, inner, static_cast<uint64_t>(weights * out), static_cast<uint64_t>(B.ld), 128, true)) != ADADIM_OK) return rc;
  if ((rc = make_tmap_u8(&tm[2], B.scales, 128, weights * scale_bytes(format, out, in, 0) / 128, 128, sf_box, false)) != ADADIM_OK) return rc;
  if (plan.fused) {
    tm[1] = tm[0];                                     // not used
    tm[3] = tm[2];
  } else {
    if ((rc = make_tmap_u8(&tm[1], A.codes, inner, static_cast<uint64_t>(n_rows), static_cast<uint64_t>(A.ld),
                           static_cast<uint32_t>(pair ? p.n_tile / 2 : p.n_tile), true)) != ADADIM_OK) return rc;
    if ((rc = make_tmap_u8(&tm[3], A.scales, 128, static_cast<uint64_t>(sf_tile_rows(n_rows, n_experts, lt) * p.n_sf * 4), 128, sf_box, false)) != ADADIM_OK) return rc;
  }

  tm[4] = tm[0];                                       // used by the pair kernel only
  const size_t per = stage_bytes(format, pair, p.n_tile);
  size_t fixed = 1024;                                 // alignment, and what lies behind the ring
  dim3 grid;
  if (pair) {
    grid = dim3(static_cast<unsigned>(2 * (tiles < kSms / 2 ? tiles : kSms / 2)));
    fixed += kOutBytes + static_cast<size_t>(n_experts > 0 ? n_experts + 1 : 0) * 4;
    p.n_stages = static_cast<int>((kSmemPair - fixed) / per);
    const int64_t ysz = ydtype == ADADIM_F32 ? 4 : 2;
    // All CTAs drain at the same time, and their stores hold up each other's loads: pauses spread the stores over
    // the next tile's time (270 ns a stage, four stores of a warp pair) where that is long enough.  2048 tokens x
    // W[11008,4096] 42.3 -> 40.7 us, experts 177 -> 170 us (16 stages a tile); with four stages (in = 1024) it lost 7 %.
    // Between those two the bound at 16 is not measured.
    p.pace_ns = p.num_k < 16 ? 0u : p.num_k < 32 ? 30u * static_cast<unsigned>(p.num_k) : 960u;
    p.bulk_y = ysz == 2 && aligned16(Y) && (ldy * ysz) % 16 == 0;
    if (p.bulk_y && (rc = make_tmap_u16(&tm[4], Y, static_cast<uint64_t>(out), static_cast<uint64_t>(n_rows),
                                        static_cast<uint64_t>(ldy * ysz), 16)) != ADADIM_OK) return rc;
  } else {
    grid = n_experts > 0 ? dim3(static_cast<unsigned>(tiles * p.splits))
                         : dim3(static_cast<unsigned>(token_tiles * p.splits), static_cast<unsigned>(p.m_tiles));
    p.tmem_cols = p.n_tile <= 64 ? 128 : 256;
    fixed += exchange_floats(p.n_tile, p.splits) * 4 + static_cast<size_t>(n_experts > 0 ? n_experts + 1 : 0) * 4;
    p.n_stages = static_cast<int>((kSmem / plan.per_sm - 1024 - fixed) / per);     // 1024: a CTA's share kept by the system
    const int k = (p.num_k + p.splits - 1) / p.splits;
    if (p.n_stages > k) p.n_stages = k;
  }
  if (p.n_stages > kMaxStages) p.n_stages = kMaxStages;
  size_t smem = p.n_stages * per + fixed;
  if (!pair && smem < kSmemPerTmemColumn * p.tmem_cols) smem = kSmemPerTmemColumn * p.tmem_cols;
  if (ydtype == ADADIM_F32) return launch_format<float>(pair, plan.fused, format, tm, p, grid, smem, chained, st);
  if (ydtype == ADADIM_F16) return launch_format<__half>(pair, plan.fused, format, tm, p, grid, smem, chained, st);
  return launch_format<__nv_bfloat16>(pair, plan.fused, format, tm, p, grid, smem, chained, st);
}

}  // namespace adadim
