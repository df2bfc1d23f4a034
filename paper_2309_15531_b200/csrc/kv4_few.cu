// Attention over the 4-bit key-value cache for few query rows a key head: one token of each request, a few drafted ones.
//
//   o = softmax(scale q K^T) V,  K and V = code * scale * 2^t
//
// Bound by the cache's bytes, 9/16 of a byte an element; what it executes comes next (a byte holds two elements, each of which
// has to become an fp16 number times its block's scale).  So a warp has 32 tokens' codes at a time in a ring of three steps in shared memory,
// as they lie in the cache, brought by bulk copies (fragments loaded straight from memory: 394 us where this takes 140), and
// takes them from there into the registers of the matrix instruction (m16n8k16), each byte once: tokens are the M side of
// S^T = K Q^T and channels that of O^T = V^T P^T, so that eight query rows (a group of heads, a few tokens) fill the N side, which
// a tile of tcgen05 with 128 rows of queries would leave empty.  The order of the channels inside a product is free: lane
// (g, c) = (lane / 4, lane % 4) takes held / 4 neighbouring channels of a key and uses them over all steps, and of a value held / 8
// neighbouring channels of four tokens; q and o follow that order.  S^T comes out with tokens down and is turned
// into the B side of the second product by movmatrix.
//
// code * scale has six significant bits and is exact in fp16; 2^t goes into the factor of the scores and of the result.
// Running maximum and sum per row, the maximum taken anew only where a score passes it by more than 2^8, which fp16 weights
// bear (see kLift); the sums are those of the rounded weights.
//
// The work of all requests, key heads and row tiles is laid out on one line and cut into equal parts, one a CTA, whatever the requests'
// lengths; the four warps of a CTA take 32 tokens each of a chunk of 128.  What is cut is joined by a second kernel in the order of
// the tokens, so that results do not depend on timing.  Small calls go to clusters instead (see kv4_few_kernel).
//
// 64 requests of up to 16384 tokens, 8 key heads of 128 channels with 8 query heads each: 141 us in replays of a graph, 649 MB, 4.6 TB/s, 0.70 of
// a copy's rate (passes launched one after another 145 to 155 us, 0.64 to 0.68); two thirds of the issue slots are taken, half of the ALU's, and
// a CTA's last piece and the join come on top.  One token over 4096: 11.3 us.
#include "kv4_line.cuh"

namespace adadim {
namespace {

using namespace kv4;
using fp4::exp2_int;

constexpr int kFewThreads = 128, kFewWarps = 4, kStep = 32, kChunk = kStep * kFewWarps;
// What a unit costs beside its tokens, in tokens: the least mean time over 43 sets of 24 to 200 requests with lengths up to 3000 .. 30000 and
// heads of 64, 128 and 256 channels: with 300, 500, 640, 750, 850, 1000 and 1500, 93.9, 88.5, 88.3, 88.6, 89.5, 90.6 and 93.8 us; the slowest of them,
// 64 requests of up to 16384 tokens, 167, 154, 147, 138, 139, 139 and 146.
constexpr int kFewCost = 750;
constexpr int kLeastPart = 256;                  // a CTA's part is no smaller
constexpr int kStages = 3;                       // steps of a warp on their way or being worked on (2 and 4: the same time within 2 us of 150)
// CTAs of an SM: what registers (a thread's 128, 168 or 255) and the ring of steps leave room for
constexpr int few_per_sm(int held, int nt) { return held == 256 ? 2 : held == 128 && nt == 2 ? 3 : 4; }
constexpr int few_ctas(int held, int nt) { return kSms * few_per_sm(held, nt); }

__device__ __forceinline__ void mma16816(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
  asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
      : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint32_t transposed(uint32_t v) {
  uint32_t r;
  asm("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(r) : "r"(v));
  return r;
}
template <int BYTES>
__device__ __forceinline__ void lds(const char* p, uint32_t* w) {
  if constexpr (BYTES >= 16) {
#pragma unroll
    for (int k = 0; k < BYTES / 16; ++k) {
      const uint4 v = reinterpret_cast<const uint4*>(p)[k];
      w[4 * k] = v.x; w[4 * k + 1] = v.y; w[4 * k + 2] = v.z; w[4 * k + 3] = v.w;
    }
  } else if constexpr (BYTES == 8) {
    const uint2 v = *reinterpret_cast<const uint2*>(p);
    w[0] = v.x; w[1] = v.y;
  } else {
    w[0] = *reinterpret_cast<const uint32_t*>(p);
  }
}
template <int BYTES>
__device__ __forceinline__ uint32_t lds_scales(const char* p) {
  if constexpr (BYTES == 4) return *reinterpret_cast<const uint32_t*>(p);
  else if constexpr (BYTES == 2) return *reinterpret_cast<const uint16_t*>(p);
  else return *reinterpret_cast<const uint8_t*>(p);
}
__device__ __forceinline__ float ld_cluster_f32(uint32_t addr) {
  float v;
  asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(v) : "r"(addr) : "memory");
  return v;
}

// 32 tokens in shared memory as they lie in the cache: keys' codes, values' codes, keys' scales, values' scales.
template <int HELD> struct Stage {
  static constexpr int kCodes = kStep * HELD / 2, kScales = kStep * HELD / 16, kV = kCodes, kKs = 2 * kCodes, kVs = 2 * kCodes + kScales;
  static constexpr int kBytes = 2 * (kCodes + kScales);
};

__host__ __device__ constexpr size_t few_ring(int held, int nt) {
  const size_t ring = static_cast<size_t>(kFewWarps) * kStages * (kStep * (held + held / 8)), results = sizeof(float) * kFewWarps * 8 * nt * (held + 4);
  return whole256(ring > results ? ring : results);
}

// The queries of lane (g, c): row g's channels c * HELD / 4 .., two to a word, in the order of the products' steps.
template <int HELD, typename T>
__device__ __forceinline__ void load_queries(const T* q, bool there, bool wide, int dim, int c, uint32_t (&raw)[HELD / 8]) {
#pragma unroll
  for (int k = 0; k < HELD / 16; ++k) {
    const int d = c * (HELD / 4) + 4 * k;                            // dim is a multiple of 16
    raw[2 * k] = raw[2 * k + 1] = 0;
    if (there && d < dim) {
      if (wide) {
        const uint2 v = *reinterpret_cast<const uint2*>(q + d);
        raw[2 * k] = v.x;
        raw[2 * k + 1] = v.y;
      } else {
        const uint16_t* u = reinterpret_cast<const uint16_t*>(q + d);
        raw[2 * k] = u[0] | static_cast<uint32_t>(u[1]) << 16;
        raw[2 * k + 1] = u[2] | static_cast<uint32_t>(u[3]) << 16;
      }
    }
  }
}

// LINE: the CTAs have equal parts of the line of work.  Otherwise a cluster of p.cluster CTAs has a unit: its CTAs take every p.cluster-th chunk
// and join their results through distributed shared memory, so that a small call is one launch without a look at all requests.
template <int HELD, int NT, typename T, bool LINE>
__global__ void __launch_bounds__(kFewThreads, few_per_sm(HELD, NT)) kv4_few_kernel(Kv4Attention p) {
  constexpr int kRows = 8 * NT, kSteps = HELD / 16, kK = HELD / 8, kV = HELD / 16;   // kK, kV: bytes of a key, a value in a lane
  constexpr int kPitch = HELD + 4;
  typedef Stage<HELD> St;
  static_assert(St::kBytes == kStep * (HELD + HELD / 8), "as few_ring has it");
  extern __shared__ __align__(128) char smem[];
  float* so = reinterpret_cast<float*>(smem);                                        // [warp][row][pitch], over the ring
  int64_t* line = reinterpret_cast<int64_t*>(smem + few_ring(HELD, NT));             // LINE: work in front of each request
  float* mine = reinterpret_cast<float*>(smem + few_ring(HELD, NT));                 // otherwise: the CTA's results [row][HELD]
  __shared__ float2 mine_stats[LINE ? 1 : kRows];                                    // .. and their maxima and sums
  __shared__ float sm_m[kFewWarps][kRows], sm_l[kFewWarps][kRows];
  __shared__ int64_t sums[kFewWarps];
  __shared__ uint64_t bars[kFewWarps][kStages];
  __shared__ int dead_flag;
  volatile int* dead = &dead_flag;
  const int tid = threadIdx.x, lane = tid & 31, warp = ptx::uniform_warp(), g = lane >> 2, c = lane & 3;
  const Cache& cache = p.cache;
  const Partials part = partials_of(p.workspace, gridDim.x, kRows);
  if (tid == 0) {
    dead_flag = 0;
    for (int k = 0; k < kFewWarps * kStages; ++k) ptx::mbar_init(&bars[0][0] + k, 1);
    ptx::fence_mbar_init();
  }
  int64_t at = 0, end = 0;
  int4 desc = make_int4(0, 0, 0, 0);
  const int size = LINE ? 1 : p.cluster, rank = LINE ? 0 : static_cast<int>(blockIdx.x) % size, stride = kChunk * size;
  int request = 0, unit_head = 0, unit_tile = 0, unit_tiles = 0;
  Request unit_request = {0, 0, 0};
  if constexpr (LINE) {
    sum_line(p, kRows, kFewCost, line, sums);
    const int64_t total = line[p.n_requests];
    const int64_t parts = max(int64_t{1}, min(static_cast<int64_t>(gridDim.x), quick_div(total, kLeastPart)));
    at = blockIdx.x < parts ? quick_div(total * blockIdx.x, parts) : total;
    end = blockIdx.x < parts ? quick_div(total * (blockIdx.x + 1), parts) : total;
  } else {
    const int u = static_cast<int>(blockIdx.x) / size, of_request = cache.kv_heads * p.tiles;
    request = u / of_request;
    unit_head = (u - request * of_request) / p.tiles;
    unit_tile = u - request * of_request - unit_head * p.tiles;
    bool good;
    unit_request = request_of(p.offsets, p.lengths, request, p.n_rows, p.width << cache.page_log2, good);
    if (!good && tid == 0) report(p.status_dev, ADADIM_ERR_SHAPE);
    const int64_t rows = static_cast<int64_t>(unit_request.rows) * p.group;
    unit_tiles = rows < p.least_rows || rows > p.most_rows ? 0 : static_cast<int>((rows + kRows - 1) / kRows);
    __syncthreads();                                                 // the barriers are set up
  }

  const int t_k = kv4::cache_scale_log2(cache, 0), t_v = kv4::cache_scale_log2(cache, 1);
  char* const ring = smem + warp * (kStages * St::kBytes);
  uint64_t* const bar = bars[warp];
  int stage = 0;
  uint32_t parity = 0;
  bool paged = true;
  while (LINE ? at < end : unit_tile < unit_tiles) {                 // p.tiles holds for the longest request, unless the caller was wrong
    const Piece x = LINE ? next_piece(p, line, at, end, request, kRows, kFewCost, kChunk)
                         : whole_unit(p, unit_request, request, unit_head, unit_tile, kRows, kChunk);
    if constexpr (LINE) request = x.request; else unit_tile += p.tiles;
    const Request& r = x.r;
    const int head = x.head, tile = x.tile, rows = x.rows, own = r.length - r.rows, row0 = tile * kRows;
    const int t0 = token_of(p, row0), t1 = token_of(p, row0 + rows - 1), key_hi = key_end(p, x, row0 + rows - 1);
    // positions that every row sees
    const int all_hi = p.causal ? min(r.length, own + t0 + 1) : r.length, all_lo = p.window > 0 ? own + t1 - p.window + 1 : 0;

    // queries are asked for first, their words are needed when the cache's first bytes are on their way
    uint32_t raw[NT][HELD / 8];
#pragma unroll
    for (int u = 0; u < NT; ++u) {
      const int row = row0 + u * 8 + g;
      const bool there = row < r.rows * p.group;
      const int tok = there ? token_of(p, row) : 0, h = there ? head * p.group + row - tok * p.group : 0;
      load_queries<HELD>(static_cast<const T*>(p.q.p) + (r.first + tok) * p.q.ld + h * p.q.lh, there, p.wide_q != 0, cache.dim, c, raw[u]);
    }

    // the warp's steps: 32 tokens of every chunk, in a ring
    const int first = x.key_lo + (x.c0 + rank) * kChunk + warp * kStep;
    const bool stopped = __any_sync(0xffffffffu, *dead != 0);
    const int steps = first >= key_hi || stopped ? 0 : min(x.c1 - x.c0, (key_hi - first + stride - 1) / stride);
    int pages = -1;                                                  // of the sixteens of tokens of the next 16 steps, one a lane
    uint32_t usable = 0;                                             // two bits a stage: whether its sixteens lie in the cache
    auto fetch = [&](int it, int to) {
      if ((it & 15) == 0) {
        const int64_t tok = first + static_cast<int64_t>(it + (lane >> 1)) * stride + (lane & 1) * 16;
        // a page whose last token lies behind every row's window is not looked at
        pages = tok < key_hi && (tok | ((1 << cache.page_log2) - 1)) >= x.seen_lo ? p.table[request * p.ldt + (tok >> cache.page_log2)] : -2;
        if (pages != -2 && (pages < 0 || pages >= cache.n_pages)) { pages = -2; paged = false; }
      }
      const int pg0 = __shfl_sync(0xffffffffu, pages, (it & 15) * 2), pg1 = __shfl_sync(0xffffffffu, pages, (it & 15) * 2 + 1);
      usable = (usable & ~(3u << 2 * to)) | (pg0 >= 0 ? 1u : 0u) << 2 * to | (pg1 >= 0 ? 2u : 0u) << 2 * to;
      if (ptx::elect_one()) {
        const int place = (first + it * stride) & ((1 << cache.page_log2) - 1);
        char* const at_stage = ring + to * St::kBytes;
        const int64_t gap = static_cast<int64_t>(cache.kv_heads) << cache.page_log2;   // rows from a page's keys to its values
        if (cache.page_log2 >= 5) {
          if (pg0 >= 0) {
            ptx::mbar_arrive_expect_tx(&bar[to], St::kBytes);
            const int64_t row = kv4::cache_row(cache, pg0, 0, head, place);
            const uint8_t *codes = cache.codes + row * (HELD / 2), *scales = cache.scales + row * (HELD / 16);
            ptx::bulk_load(at_stage, codes, St::kCodes, &bar[to]);
            ptx::bulk_load(at_stage + St::kKs, scales, St::kScales, &bar[to]);
            ptx::bulk_load(at_stage + St::kV, codes + gap * (HELD / 2), St::kCodes, &bar[to]);
            ptx::bulk_load(at_stage + St::kVs, scales + gap * (HELD / 16), St::kScales, &bar[to]);
          } else {
            ptx::mbar_arrive(&bar[to]);
          }
        } else {
          const uint32_t bytes = ((pg0 >= 0) + (pg1 >= 0)) * (St::kBytes / 2);
          if (bytes > 0) ptx::mbar_arrive_expect_tx(&bar[to], bytes); else ptx::mbar_arrive(&bar[to]);
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            const int pg = h == 0 ? pg0 : pg1;
            if (pg < 0) continue;
            const int64_t row = kv4::cache_row(cache, pg, 0, head, 0);                 // a page is one sixteen
            const uint8_t *codes = cache.codes + row * (HELD / 2), *scales = cache.scales + row * (HELD / 16);
            ptx::bulk_load(at_stage + h * (St::kCodes / 2), codes, St::kCodes / 2, &bar[to]);
            ptx::bulk_load(at_stage + St::kKs + h * (St::kScales / 2), scales, St::kScales / 2, &bar[to]);
            ptx::bulk_load(at_stage + St::kV + h * (St::kCodes / 2), codes + gap * (HELD / 2), St::kCodes / 2, &bar[to]);
            ptx::bulk_load(at_stage + St::kVs + h * (St::kScales / 2), scales + gap * (HELD / 16), St::kScales / 2, &bar[to]);
          }
        }
      }
      __syncwarp();
    };
    {
      int to = stage;
      for (int it = 0; it < min(steps, kStages); ++it) {
        fetch(it, to);
        to = to + 1 == kStages ? 0 : to + 1;
      }
    }

    // queries as fp16, and what their scores are multiplied by
    uint32_t qb[NT][kSteps][2];
    float factor[NT][2];
    int lim[NT][2], low[NT][2];
#pragma unroll
    for (int u = 0; u < NT; ++u) {
      uint32_t most = 0;                                             // magnitudes are ordered as whole numbers
#pragma unroll
      for (int k = 0; k < HELD / 8; ++k) most = __vmaxu2(most, raw[u][k] & 0x7fff7fffu);
      most = max(most & 0xffffu, most >> 16);
      most = max(most, __shfl_xor_sync(0xffffffffu, most, 1));
      most = max(most, __shfl_xor_sync(0xffffffffu, most, 2));
      const int e = query_exponent<T>(most);
      const float scaled = exp2_int(e);
#pragma unroll
      for (int k = 0; k < HELD / 8; ++k) qb[u][k >> 1][k & 1] = query_bits<T>(raw[u][k], scaled);
      // a query that is not finite makes every score it has with a key NaN
      const float f = query_fine<T>(most) ? ldexpf(p.scale * kLog2e, t_k - e) : __int_as_float(0x7fffffff);
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        const int n = 2 * c + k;
        factor[u][k] = __shfl_sync(0xffffffffu, f, n * 4);
        const int t = token_of(p, row0 + u * 8 + n);
        lim[u][k] = p.causal ? min(r.length, own + t + 1) : r.length;
        low[u][k] = p.window > 0 ? own + t - p.window + 1 : 0;
      }
    }
    float o[NT][kSteps][4] = {};
    float m[NT][2], l[NT][4] = {};                                   // l: every row of channels has the same sums
#pragma unroll
    for (int u = 0; u < NT; ++u) m[u][0] = m[u][1] = -INFINITY;

    // tokens of a sixteen in the order of the products: n even n / 2, n odd (n / 2 ^ 1) + 4, the upper eight the same.  Lane (g, c) then has the
    // scores of places pk and pk + 8, and of values the places pv[0] = c, pv[1] and those + 8; neighbouring
    // lanes' reads of a row of 64 bytes fall into different banks for keys, into two at a time for values.
    const int pk = (g & 1) ? ((g >> 1) ^ 1) + 4 : g >> 1, pv1 = (c ^ 1) + 4;

#pragma unroll 1
    for (int it = 0; it < steps; ++it) {
      const char* const from = ring + stage * St::kBytes;
      if (!ptx::mbar_wait_warp(&bar[stage], parity, dead, p.status_dev)) break;       // (one answer for all lanes: they work together behind it)
      const uint32_t use = usable >> 2 * stage & 3u;
      const int tok = first + it * stride;
      // scores of tokens tok + place and rows 2 c, 2 c + 1 of every eight
      float sc[2][NT][4] = {};
#pragma unroll
      for (int hh = 0; hh < 2; ++hh) {
        const char* const codes = from + (hh * 16 + pk) * (HELD / 2) + c * kK;
        const char* const scales = from + St::kKs + (hh * 16 + pk) * (HELD / 16) + c * (HELD / 64);
        uint32_t k0[kK / 4], k1[kK / 4];
        lds<kK>(codes, k0);
        lds<kK>(codes + 8 * (HELD / 2), k1);
        const uint32_t s0 = lds_scales<HELD / 64>(scales), s1 = lds_scales<HELD / 64>(scales + 8 * (HELD / 16));
        __half2 ks0[HELD / 64], ks1[HELD / 64];
#pragma unroll
        for (int b = 0; b < HELD / 64; ++b) {
          const __half2 two0 = scales_of(s0 >> (b & ~1) * 8), two1 = scales_of(s1 >> (b & ~1) * 8);
          ks0[b] = (b & 1) ? __high2half2(two0) : __low2half2(two0);
          ks1[b] = (b & 1) ? __high2half2(two1) : __low2half2(two1);
        }
#pragma unroll
        for (int j = 0; j < kSteps; j += 2) {
          __half2 x0[4], x1[4];
          values8(k0[j / 2], x0);
          values8(k1[j / 2], x1);
#pragma unroll
          for (int k = 0; k < 4; ++k) { x0[k] = __hmul2(x0[k], ks0[j / 4]); x1[k] = __hmul2(x1[k], ks1[j / 4]); }
#pragma unroll
          for (int u = 0; u < NT; ++u) {
            mma16816(sc[hh][u], half2_bits(x0[0]), half2_bits(x1[0]), half2_bits(x0[1]), half2_bits(x1[1]), qb[u][j][0], qb[u][j][1]);
            mma16816(sc[hh][u], half2_bits(x0[2]), half2_bits(x1[2]), half2_bits(x0[3]), half2_bits(x1[3]), qb[u][j + 1][0], qb[u][j + 1][1]);
          }
        }
      }
      const bool edge = tok < all_lo || tok + kStep > all_hi || use != 3u;
#pragma unroll
      for (int hh = 0; hh < 2; ++hh)
#pragma unroll
        for (int u = 0; u < NT; ++u)
#pragma unroll
          for (int k = 0; k < 4; ++k) sc[hh][u][k] *= factor[u][k & 1];
      if (edge) {
#pragma unroll
        for (int hh = 0; hh < 2; ++hh)
#pragma unroll
          for (int u = 0; u < NT; ++u)
#pragma unroll
            for (int k = 0; k < 4; ++k) {
              const int t = tok + hh * 16 + pk + 8 * (k >> 1);
              if (t >= lim[u][k & 1] || t < low[u][k & 1] || (use >> hh & 1u) == 0) sc[hh][u][k] = -INFINITY;
            }
      }
      float top[NT][2];
      bool grows = false;
#pragma unroll
      for (int u = 0; u < NT; ++u)
#pragma unroll
        for (int k = 0; k < 2; ++k) {
          top[u][k] = fmaxf(fmaxf(sc[0][u][k], sc[0][u][k + 2]), fmaxf(sc[1][u][k], sc[1][u][k + 2]));
          grows |= top[u][k] - m[u][k] > kGrowth;
        }
      if (__any_sync(0xffffffffu, grows)) {
#pragma unroll
        for (int u = 0; u < NT; ++u)
#pragma unroll
          for (int k = 0; k < 2; ++k) {
            float t = top[u][k];
#pragma unroll
            for (int d = 4; d < 32; d <<= 1) t = fmaxf(t, __shfl_xor_sync(0xffffffffu, t, d));
            if (t > m[u][k]) {
              const float f = exp2_fast(m[u][k] - t);               // 0 at the first
              m[u][k] = t;
              l[u][k] *= f;
#pragma unroll
              for (int j = 0; j < kSteps; ++j) { o[u][j][k] *= f; o[u][j][k + 2] *= f; }
            }
          }
      }
      uint32_t pb[2][NT][2];
#pragma unroll
      for (int u = 0; u < NT; ++u) {
        const float base0 = lifted(m[u][0]), base1 = lifted(m[u][1]);
#pragma unroll
        for (int hh = 0; hh < 2; ++hh) {
          pb[hh][u][0] = transposed(half2_bits(__floats2half2_rn(exp2_fast(sc[hh][u][0] - base0), exp2_fast(sc[hh][u][1] - base1))));
          pb[hh][u][1] = transposed(half2_bits(__floats2half2_rn(exp2_fast(sc[hh][u][2] - base0), exp2_fast(sc[hh][u][3] - base1))));
          mma16816(l[u], 0x3c003c00u, 0x3c003c00u, 0x3c003c00u, 0x3c003c00u, pb[hh][u][0], pb[hh][u][1]);
        }
      }
      // values: of four tokens a sixteen, two channels at a time
      uint32_t v[2][4][kV / 4], vs[2][4];
#pragma unroll
      for (int hh = 0; hh < 2; ++hh)
#pragma unroll
        for (int h = 0; h < 4; ++h) {
          const int place = hh * 16 + ((h & 1) ? pv1 : c) + 8 * (h >> 1);
          lds<kV>(from + St::kV + place * (HELD / 2) + g * kV, v[hh][h]);
          vs[hh][h] = lds_scales<(HELD == 256 ? 2 : 1)>(from + St::kVs + place * (HELD / 16) + (HELD == 256 ? 2 * g : HELD == 128 ? g : g >> 1));
        }
      __syncwarp();
      if (it + kStages < steps) fetch(it + kStages, stage);
      if (++stage == kStages) { stage = 0; parity ^= 1u; }
      if (tok + kStep > key_hi || use != 3u) {
#pragma unroll
        for (int hh = 0; hh < 2; ++hh)
#pragma unroll
          for (int h = 0; h < 4; ++h)
            if (tok + hh * 16 + ((h & 1) ? pv1 : c) + 8 * (h >> 1) >= key_hi || (use >> hh & 1u) == 0) vs[hh][h] = 0;
      }
      __half2 w[2][2][HELD == 256 ? 2 : 1];
      uint32_t any_nan = 0;
#pragma unroll
      for (int hh = 0; hh < 2; ++hh)
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const uint32_t two = (vs[hh][2 * h] & 0xffu) | (vs[hh][2 * h + 1] & 0xffu) << 8;
          w[hh][h][0] = scales_of(two);
          any_nan |= (two & 0x7f7fu) + 0x0101u;
          if constexpr (HELD == 256) {
            const uint32_t up = (vs[hh][2 * h] >> 8) | (vs[hh][2 * h + 1] & 0xff00u);
            w[hh][h][1] = scales_of(up);
            any_nan |= (up & 0x7f7fu) + 0x0101u;
          }
        }
      if (__any_sync(0xffffffffu, (any_nan & 0x8080u) != 0)) {
        // values that are NaN reach the rows that see their token and no other
#pragma unroll
        for (int hh = 0; hh < 2; ++hh)
#pragma unroll
          for (int h = 0; h < 4; ++h) {
#pragma unroll 1
            for (int src = 0; src < 4; ++src) {
              const uint32_t nan = __shfl_sync(0xffffffffu, ((vs[hh][h] & 0x7f7fu) + 0x0101u) & 0x8080u, (lane & ~3) + src);
              const int t = tok + hh * 16 + ((h & 1) ? (src ^ 1) + 4 : src) + 8 * (h >> 1);
#pragma unroll
              for (int u = 0; u < NT; ++u)
#pragma unroll
                for (int k = 0; k < 2; ++k)
                  if (t < lim[u][k] && t >= low[u][k]) {
#pragma unroll
                    for (int j = 0; j < kSteps; ++j)
                      if (nan & (HELD == 256 && j >= kSteps / 2 ? 0x8000u : 0x80u)) o[u][j][k] = o[u][j][k + 2] = __int_as_float(0x7fffffff);
                  }
            }
          }
        const __half2 none = __float2half2_rn(0.0f);
#pragma unroll
        for (int hh = 0; hh < 2; ++hh)
#pragma unroll
          for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int b = 0; b < (HELD == 256 ? 2 : 1); ++b) {
              const __half2 x = w[hh][h][b];
              w[hh][h][b] = __halves2half2(__hisnan(__low2half(x)) ? __low2half(none) : __low2half(x), __hisnan(__high2half(x)) ? __low2half(none) : __high2half(x));
            }
      }
      // a lane's byte j holds its channels 2 j and 2 j + 1: rows g and g + 8 of the product's j-th step of channels
#pragma unroll
      for (int hh = 0; hh < 2; ++hh)
#pragma unroll
        for (int q = 0; q < kV / 4; ++q) {
          __half2 lo0[4], hi0[4], lo1[4], hi1[4];
          const uint32_t a = v[hh][0][q], b = v[hh][1][q], d = v[hh][2][q], f = v[hh][3][q];
          values8((a & 0x0f0f0f0fu) | (b << 4 & 0xf0f0f0f0u), lo0);
          values8((a >> 4 & 0x0f0f0f0fu) | (b & 0xf0f0f0f0u), hi0);
          values8((d & 0x0f0f0f0fu) | (f << 4 & 0xf0f0f0f0u), lo1);
          values8((d >> 4 & 0x0f0f0f0fu) | (f & 0xf0f0f0f0u), hi1);
#pragma unroll
          for (int k = 0; k < 4; ++k) {
            const int j = 4 * q + k, blk = HELD == 256 && j >= 8 ? 1 : 0;
            const __half2 s0 = w[hh][0][blk], s1 = w[hh][1][blk];
            const uint32_t a0 = half2_bits(__hmul2(lo0[k], s0)), a1 = half2_bits(__hmul2(hi0[k], s0));
            const uint32_t a2 = half2_bits(__hmul2(lo1[k], s1)), a3 = half2_bits(__hmul2(hi1[k], s1));
#pragma unroll
            for (int u = 0; u < NT; ++u) mma16816(o[u][j], a0, a1, a2, a3, pb[hh][u][0], pb[hh][u][1]);
          }
        }
    }
    __syncthreads();
    if (LINE && *dead) break;                                        // (a cluster goes through its barriers all the same)

    // the warps' parts together
#pragma unroll
    for (int u = 0; u < NT; ++u)
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        const int row = u * 8 + 2 * c + k;
        if (g == 0) { sm_m[warp][row] = m[u][k]; sm_l[warp][row] = l[u][k]; }
        float* to = so + (warp * kRows + row) * kPitch + g * (HELD / 8);
#pragma unroll
        for (int j = 0; j < kSteps; ++j) *reinterpret_cast<float2*>(to + 2 * j) = make_float2(o[u][j][k], o[u][j][k + 2]);
      }
    __syncthreads();
    const bool whole = LINE ? x.starts && x.ends : size == 1;
    const int slot = x.starts ? 1 : 0;
    for (int e = tid; e < rows * HELD; e += kFewThreads) {
      const int row = e / HELD, d = e - row * HELD;
      float top = sm_m[0][row];
#pragma unroll
      for (int w = 1; w < kFewWarps; ++w) top = fmaxf(top, sm_m[w][row]);
      float sum = 0.0f, v = 0.0f;
#pragma unroll
      for (int w = 0; w < kFewWarps; ++w) {
        // a warp that saw nothing holds zeros; one that saw a NaN holds NaN
        const float f = sm_m[w][row] == -INFINITY ? 1.0f : exp2_fast(sm_m[w][row] - top);
        sum += sm_l[w][row] * f;
        v += so[(w * kRows + row) * kPitch + d] * f;
      }
      if (whole) {
        if (d < cache.dim) {
          const int rr = row0 + row, tok = token_of(p, rr), h = head * p.group + rr - tok * p.group;
          T* out = static_cast<T*>(p.o.p) + (r.first + tok) * p.o.ld + h * p.o.lh;
          out[d] = static_cast<T>(sum == 0.0f ? v : ldexpf(v / sum, t_v));
        }
      } else if constexpr (LINE) {
        const int64_t at_row = (static_cast<int64_t>(blockIdx.x) * 2 + slot) * kRows + row;
        part.o[at_row * HELD + d] = v;
        if (d == 0) part.stats[at_row] = make_float2(top, sum);
      } else {
        mine[e] = v;
        if (d == 0) mine_stats[row] = make_float2(top, sum);
      }
    }
    if (LINE && !whole) note_piece(desc, x);
    if (!LINE && size > 1) {
      ptx::cluster_sync();
      const uint32_t mine_at = ptx::smem_addr(mine), stats_at = ptx::smem_addr(mine_stats);
      for (int e = rank * kFewThreads + tid; e < rows * HELD; e += size * kFewThreads) {
        const int row = e / HELD, d = e - row * HELD;
        if (d >= cache.dim) continue;
        float v[8], sm[8], sl[8], top = -INFINITY;
#pragma unroll
        for (int k = 0; k < 8; ++k)
          if (k < size) {
            v[k] = ld_cluster_f32(ptx::map_to_cta(mine_at + e * 4, k));
            const uint32_t st = ptx::map_to_cta(stats_at + row * 8, k);
            sm[k] = ld_cluster_f32(st);
            sl[k] = ld_cluster_f32(st + 4);
          }
#pragma unroll
        for (int k = 0; k < 8; ++k) if (k < size) top = fmaxf(top, sm[k]);
        float sum = 0.0f, o1 = 0.0f;
#pragma unroll
        for (int k = 0; k < 8; ++k)
          if (k < size) {
            const float f = sm[k] == -INFINITY ? 1.0f : exp2_fast(sm[k] - top);
            sum += sl[k] * f;
            o1 += v[k] * f;
          }
        const int rr = row0 + row, tok = token_of(p, rr), h = head * p.group + rr - tok * p.group;
        T* out = static_cast<T*>(p.o.p) + (r.first + tok) * p.o.ld + h * p.o.lh;
        out[d] = static_cast<T>(sum == 0.0f ? o1 : ldexpf(o1 / sum, t_v));
      }
      ptx::cluster_sync();                                           // the others have read what is here
    }
    ptx::fence_proxy_async();                                        // the ring is written by bulk copies again
    __syncthreads();
  }
  ptx::pdl_launch_dependents();
  if (*dead) {                                                       // a wait ran out: no copy may be in flight when the CTA ends
    const long long t = clock64();
    for (int k = 0; k < kStages; ++k)
      while (!ptx::mbar_try_wait(&bar[k], parity ^ (k < stage ? 1u : 0u)) && clock64() - t < ptx::kWaitLimit / 4) {}
    desc = make_int4(0, 0, 0, 0);
  }
  if (LINE && tid == 0) part.desc[blockIdx.x] = desc;
  if (__any_sync(0xffffffffu, !paged) && lane == 0) report(p.status_dev, ADADIM_ERR_PAGES);
  ptx::pdl_wait();                                                   // no earlier than the kernel before it
}

// A call's units, and the tokens that the table and the window allow each.
int64_t units_of(const Kv4Attention& a, int tile_rows, int64_t max_new) {
  return (max_new * a.group + tile_rows - 1) / tile_rows * a.n_requests * a.cache.kv_heads;
}
int64_t span_of(const Kv4Attention& a, int64_t max_new) {
  const int64_t span = a.width << a.cache.page_log2;
  return a.causal && a.window > 0 && a.window + max_new + kStep < span ? a.window + max_new + kStep : span;
}
// Whether a call's units go to clusters, and of how many CTAs: where there is little to read altogether (2^20 tokens of key heads are
// 25 us), so that unequal lengths cost less than the second launch that joins cut units, and enough units, or short ones, that clusters of
// up to eight CTAs find the SMs enough to do.  (One token of a request with 8 key heads, line against clusters: 8256 tokens 16.1 and 14.2 us,
// 16384 19.7 and 21.2, 32768 24 and 36, 131072 46 and 129; with one key head 8256 11.7 and 13.8, 16384 13.4 and 21.)
int cluster_of(const Kv4Attention& a, int tile_rows, int ctas, int64_t max_new, int& tiles) {
  const int64_t units = units_of(a, tile_rows, max_new), span = span_of(a, max_new);
  if (units > 4 * ctas || units * span > (int64_t{1} << 20) || (units < 16 && span > 8192)) return 0;
  tiles = static_cast<int>((max_new * a.group + tile_rows - 1) / tile_rows);
  int size = 1;
  while (size < 8 && units * size * 2 <= ctas && span > kChunk * size) size *= 2;
  return size;
}

template <int HELD, int NT, typename T, bool LINE>
int few_start(const Kv4Attention& a, int ctas, size_t more, bool chained, cudaStream_t st) {
  static std::atomic<uint64_t> done{0};
  const int rc = set_once(kv4_few_kernel<HELD, NT, T, LINE>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                          static_cast<int>(few_ring(HELD, NT) + sizeof(int64_t) * (kMaxRequests + 1)), done);
  if (rc != ADADIM_OK) return rc;
  return chained_launch(kv4_few_kernel<HELD, NT, T, LINE>, dim3(static_cast<unsigned>(ctas)), kFewThreads, few_ring(HELD, NT) + more, chained, st, a, LINE ? 1 : a.cluster);
}
template <int HELD, int NT, typename T>
int few_launch(Kv4Attention a, int64_t max_new, bool chained, int& ctas, int& tile_rows, cudaStream_t st) {
  tile_rows = 8 * NT;
  a.cluster = chained ? 0 : cluster_of(a, tile_rows, few_ctas(HELD, NT), max_new, a.tiles);
  if (a.cluster > 0) {
    ctas = 0;                                                        // nothing to join
    return few_start<HELD, NT, T, false>(a, a.tiles * a.n_requests * a.cache.kv_heads * a.cluster, sizeof(float) * tile_rows * HELD, false, st);
  }
  ctas = few_ctas(HELD, NT);
  return few_start<HELD, NT, T, true>(a, ctas, sizeof(int64_t) * (static_cast<size_t>(a.n_requests) + 1), chained, st);
}
template <int HELD, typename T>
int few_held(const Kv4Attention& a, int64_t max_new, bool chained, int& ctas, int& tile_rows, cudaStream_t st) {
  // behind the kernel for many rows this one has requests of one token, or of a few
  if (HELD < 256 && (chained ? 1 : max_new) * a.group > 8) return few_launch<HELD, HELD < 256 ? 2 : 1, T>(a, max_new, chained, ctas, tile_rows, st);
  return few_launch<HELD, 1, T>(a, max_new, chained, ctas, tile_rows, st);
}
template <typename T>
int few_type(const Kv4Attention& a, int64_t max_new, bool chained, int& ctas, int& tile_rows, cudaStream_t st) {
  if (a.cache.held == 64) return few_held<64, T>(a, max_new, chained, ctas, tile_rows, st);
  return a.cache.held == 128 ? few_held<128, T>(a, max_new, chained, ctas, tile_rows, st) : few_held<256, T>(a, max_new, chained, ctas, tile_rows, st);
}

}  // namespace

// Many rows, but few units of this kernel over few tokens, which clusters are done with before the other kernel's tiles are set up: 40
// tokens of 32 heads over themselves 9.7 us against 38, eight such prompts 22 against 38, 128 rows of 8 key heads over 8192 (2^19 tokens) 38
// against 46, four times 64 rows over as many (2^20) 55 against 47.
bool kv4_few_suits(const Kv4Attention& a, int64_t max_new) {
  int tiles;
  return units_of(a, 16, max_new) * span_of(a, max_new) <= (int64_t{1} << 19) && cluster_of(a, 16, few_ctas(a.cache.held, 2), max_new, tiles) > 0;
}
size_t kv4_few_workspace(int held) {
  const size_t one = partials_bytes(few_ctas(held, 1), 8, held), two = held < 256 ? partials_bytes(few_ctas(held, 2), 16, held) : 0;
  return one > two ? one : two;
}

int kv4_few_launch(const Kv4Attention& a, int dtype, int64_t max_new, bool chained, int& ctas, int& tile_rows, cudaStream_t st) {
  return dtype == ADADIM_F16 ? few_type<__half>(a, max_new, chained, ctas, tile_rows, st) : few_type<__nv_bfloat16>(a, max_new, chained, ctas, tile_rows, st);
}

}  // namespace adadim
