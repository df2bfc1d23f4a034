// Attention over the 4-bit key-value cache for few query rows a key head: one token of each request, a few drafted ones.
//
//   o = softmax(scale q K^T) V,  K and V = code * scale * 2^t
//
// Bound by the cache's bytes, 9/16 of a byte an element; what it executes comes next (a byte holds two elements, each of which
// has to become an fp16 number times its block's scale).  So codes go from memory into the registers that the matrix instruction
// (m16n8k16) takes, with no shared memory between: tokens are the M side of S^T = K Q^T and channels that of O^T = V^T P^T, so that eight
// query rows (a group of heads, a few tokens) fill the N side.  The order of the channels inside a product is free: lane
// (g, c) = (lane / 4, lane % 4) takes held / 4 neighbouring channels of a key and uses them over all steps, and of a value held / 8
// neighbouring channels of four tokens; q and o follow that order.  S^T comes out with tokens down and is turned
// into the B side of the second product by movmatrix.
//
// code * scale has six significant bits and is exact in fp16; 2^t goes into the factor of the scores and of the result.
// Running maximum and sum per row, the maximum taken anew only where a score passes it by more than 2^8, which fp16 weights
// bear (they are rounded to 11 bits and lie below 2^8).
//
// The work of all requests, key heads and row tiles is laid out on one line in chunks of 64 tokens and cut into equal parts,
// one a CTA, whatever the requests' lengths; the four warps of a CTA take 16 tokens each of a chunk.  What is cut is joined by
// a second kernel in the order of the tokens, so that results do not depend on timing.
#include "kv4.cuh"

namespace adadim {
namespace {

using kv4::Cache;
using kv4::Request;

constexpr int kFewThreads = 128, kFewWarps = 4, kStep = 16, kChunk = kStep * kFewWarps;
constexpr int kUnitCost = 1;                     // what a unit costs beside its chunks, in chunks
constexpr int kLeastChunks = 4;                  // a CTA's part is no smaller
constexpr int kFewPerSm = 4, kFewCtas = 148 * kFewPerSm;
constexpr float kLog2e = 1.4426950408889634f;

enum : int { kBegins = 1, kEnds = 2 };           // a cut unit begins in this CTA's part (and goes on) / one from before ends in it

// Where the parts of cut units are kept: slot 0 of a CTA for the one that began before, 1 for the one that goes on.
struct Partials {
  int4* desc;              // request, head, tile of the unit that begins; kBegins, kEnds
  float2* stats;           // [cta][2][rows] maximum and sum
  float* o;                // [cta][2][rows][held]
};
__host__ __device__ constexpr size_t whole256(size_t bytes) { return (bytes + 255) / 256 * 256; }
__host__ __device__ inline Partials partials_of(char* ws, int ctas, int rows) {
  Partials p;
  p.desc = reinterpret_cast<int4*>(ws);
  p.stats = reinterpret_cast<float2*>(ws + whole256(sizeof(int4) * ctas));
  p.o = reinterpret_cast<float*>(reinterpret_cast<char*>(p.stats) + whole256(sizeof(float2) * 2 * ctas * rows));
  return p;
}
size_t partials_bytes(int ctas, int rows, int held) {
  return whole256(sizeof(int4) * ctas) + whole256(sizeof(float2) * 2 * ctas * rows) + sizeof(float) * 2 * ctas * rows * held;
}

__device__ __forceinline__ uint32_t half2_bits(__half2 h) { return *reinterpret_cast<uint32_t*>(&h); }
__device__ __forceinline__ __half2 bits_half2(uint32_t b) { return *reinterpret_cast<__half2*>(&b); }
// eight codes as fp16, two to a register
__device__ __forceinline__ void values8(uint32_t w, __half2 (&v)[4]) {
  uint32_t h[4];
  asm("{\n\t.reg .b8 a, b, c, d;\n\t"
      "mov.b32 {a, b, c, d}, %4;\n\t"
      "cvt.rn.f16x2.e2m1x2 %0, a;\n\t"
      "cvt.rn.f16x2.e2m1x2 %1, b;\n\t"
      "cvt.rn.f16x2.e2m1x2 %2, c;\n\t"
      "cvt.rn.f16x2.e2m1x2 %3, d;\n\t}"
      : "=r"(h[0]), "=r"(h[1]), "=r"(h[2]), "=r"(h[3]) : "r"(w));
#pragma unroll
  for (int k = 0; k < 4; ++k) v[k] = bits_half2(h[k]);
}
// two E4M3 bytes as fp16
__device__ __forceinline__ __half2 scales_of(uint32_t two) {
  uint32_t r;
  asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(r) : "h"(static_cast<uint16_t>(two)));
  return bits_half2(r);
}
__device__ __forceinline__ void mma16816(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
  asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};"
      : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint32_t transposed(uint32_t v) {
  uint32_t r;
  asm("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(r) : "r"(v));
  return r;
}
__device__ __forceinline__ float exp2_fast(float x) {
  float r;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
  return r;
}
template <int BYTES>
__device__ __forceinline__ void load_stream(const uint8_t* p, uint32_t* w) {
  if constexpr (BYTES == 32) {
    asm volatile("ld.global.nc.L1::no_allocate.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(w[0]), "=r"(w[1]), "=r"(w[2]), "=r"(w[3]) : "l"(p));
    asm volatile("ld.global.nc.L1::no_allocate.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(w[4]), "=r"(w[5]), "=r"(w[6]), "=r"(w[7]) : "l"(p + 16));
  } else if constexpr (BYTES == 16) {
    asm volatile("ld.global.nc.L1::no_allocate.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(w[0]), "=r"(w[1]), "=r"(w[2]), "=r"(w[3]) : "l"(p));
  } else if constexpr (BYTES == 8) {
    asm volatile("ld.global.nc.L1::no_allocate.v2.b32 {%0, %1}, [%2];" : "=r"(w[0]), "=r"(w[1]) : "l"(p));
  } else {
    asm volatile("ld.global.nc.L1::no_allocate.b32 %0, [%1];" : "=r"(w[0]) : "l"(p));
  }
}
template <int BYTES>
__device__ __forceinline__ uint32_t load_scales(const uint8_t* p) {
  if constexpr (BYTES == 4) return __ldg(reinterpret_cast<const uint32_t*>(p));
  else if constexpr (BYTES == 2) return __ldg(reinterpret_cast<const uint16_t*>(p));
  else return __ldg(p);
}

// ---- the line of work ------------------------------------------------------------------------------
// A unit: the query rows row0 .. of one tile (row r of a request is token r / group, head r % group of the key head's), and the
// tokens lo .. hi - 1 of the cache that some of them sees, lo a multiple of 16.
struct Shape {
  int tiles;               // of a key head
  int64_t unit;            // what a unit takes of the line
};
__device__ __forceinline__ Shape shape_of(const Kv4Attention& p, const Request& r, int tile_rows) {
  Shape s = {0, 0};
  const int64_t rows = static_cast<int64_t>(r.rows) * p.group;
  if (rows == 0 || rows > p.few_rows) return s;
  s.tiles = static_cast<int>((rows + tile_rows - 1) / tile_rows);
  int64_t chunks = (r.length + kChunk - 1) / kChunk;
  if (p.window > 0 && p.causal) {
    const int64_t tokens = min(r.rows, (tile_rows + p.group - 2) / p.group + 1);
    chunks = min(chunks, (static_cast<int64_t>(p.window) + tokens + 14) / kChunk + 2);
  }
  s.unit = chunks + kUnitCost;
  return s;
}

template <int HELD, int NT, typename T>
__global__ void __launch_bounds__(kFewThreads) kv4_few_kernel(Kv4Attention p) {
  constexpr int kRows = 8 * NT, kSteps = HELD / 16, kK = HELD / 8, kV = HELD / 16;   // kK, kV: bytes of a key, a value in a lane
  constexpr int kPitch = HELD + 4;
  extern __shared__ __align__(16) char smem[];
  float* so = reinterpret_cast<float*>(smem);                                        // [warp][row][pitch]
  int64_t* line = reinterpret_cast<int64_t*>(smem + sizeof(float) * kFewWarps * kRows * kPitch);   // work in front of each request
  __shared__ float sm_m[kFewWarps][kRows], sm_l[kFewWarps][kRows];
  __shared__ int64_t sums[kFewWarps];
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, g = lane >> 2, c = lane & 3;
  const Cache& cache = p.cache;
  const Partials part = partials_of(p.workspace, gridDim.x, kRows);
  const int64_t most = p.width << cache.page_log2;

  // the line: every CTA sums it up for itself
  {
    int64_t carry = 0;
    bool good = true;
    for (int i0 = 0; i0 < p.n_requests; i0 += kFewThreads) {
      const int i = i0 + tid;
      int64_t w = 0;
      if (i < p.n_requests) {
        bool ok;
        const Request r = kv4::request_of(p.offsets, p.lengths, i, p.n_rows, most, ok);
        good &= ok;
        const Shape s = shape_of(p, r, kRows);
        w = s.unit * s.tiles * cache.kv_heads;
      }
      int64_t sum = w;
#pragma unroll
      for (int d = 1; d < 32; d <<= 1) {
        const int64_t u = __shfl_up_sync(0xffffffffu, sum, d);
        if (lane >= d) sum += u;
      }
      if (lane == 31) sums[warp] = sum;
      __syncthreads();
      int64_t before = carry;
#pragma unroll
      for (int k = 0; k < kFewWarps; ++k) {
        if (k < warp) before += sums[k];
        carry += sums[k];
      }
      if (i < p.n_requests) line[i] = before + sum - w;
      __syncthreads();
    }
    if (tid == 0) line[p.n_requests] = carry;
    if (!good && blockIdx.x == 0) report(p.status_dev, ADADIM_ERR_SHAPE);
    __syncthreads();
  }
  const int64_t total = line[p.n_requests];
  const int64_t parts = max(int64_t{1}, min(static_cast<int64_t>(gridDim.x), total / kLeastChunks));
  int64_t at = blockIdx.x < parts ? total * blockIdx.x / parts : total;
  const int64_t end = blockIdx.x < parts ? total * (blockIdx.x + 1) / parts : total;
  int4 desc = make_int4(0, 0, 0, 0);

  const int t_k = kv4::cache_scale_log2(cache, 0), t_v = kv4::cache_scale_log2(cache, 1);
  bool paged = true;
  int request = 0;
  while (at < end) {
    // the request and unit that `at` lies in
    {
      int lo = request, hi = p.n_requests;
      while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (line[mid] <= at) lo = mid; else hi = mid;
      }
      request = lo;
    }
    bool ok;
    const Request r = kv4::request_of(p.offsets, p.lengths, request, p.n_rows, most, ok);
    const Shape s = shape_of(p, r, kRows);
    const int64_t within = at - line[request], number = within / s.unit, begin = within - number * s.unit;
    const int64_t stop = min(s.unit, begin + end - at);
    const int head = static_cast<int>(number / s.tiles), tile = static_cast<int>(number - static_cast<int64_t>(head) * s.tiles);
    at += stop - begin;
    const bool starts = begin == 0, ends = stop == s.unit;

    const int rows = min(kRows, r.rows * p.group - tile * kRows);
    const int t0 = tile * kRows / p.group, t1 = (tile * kRows + rows - 1) / p.group, own = r.length - r.rows;
    int key_hi = p.causal ? min(r.length, own + t1 + 1) : r.length;
    int key_lo = p.window > 0 ? max(0, own + t0 - p.window + 1) & ~(kStep - 1) : 0;
    // positions that every row sees
    const int all_hi = p.causal ? min(r.length, own + t0 + 1) : r.length, all_lo = p.window > 0 ? own + t1 - p.window + 1 : 0;
    const int chunks = key_hi > key_lo ? (key_hi - key_lo + kChunk - 1) / kChunk : 0;
    const int ch0 = min(chunks, max(0, static_cast<int>(begin) - kUnitCost)), ch1 = ends ? chunks : min(chunks, max(0, static_cast<int>(stop) - kUnitCost));

    // queries: lane (g, c) holds of row g the channels c * held / 4 ..; what its scores are multiplied by
    uint32_t qb[NT][kSteps][2];
    float factor[NT][2];
    int lim[NT][2], low[NT][2];
#pragma unroll
    for (int u = 0; u < NT; ++u) {
      const int row = tile * kRows + u * 8 + g;
      const bool there = row < r.rows * p.group;
      const int tok = there ? row / p.group : 0, h = there ? head * p.group + row - tok * p.group : 0;
      const T* q = static_cast<const T*>(p.q.p) + (r.first + tok) * p.q.ld + h * p.q.lh;
      float x[HELD / 4];
#pragma unroll
      for (int k = 0; k < HELD / 4; ++k) {
        const int d = c * (HELD / 4) + k;
        x[k] = there && d < cache.dim ? static_cast<float>(q[d]) : 0.0f;
      }
      float top = 0.0f;
      bool fine = true;
#pragma unroll
      for (int k = 0; k < HELD / 4; ++k) { top = fmaxf(top, fabsf(x[k])); fine &= fabsf(x[k]) < INFINITY; }
      top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 1));
      top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 2));
      const uint32_t bad = __ballot_sync(0xffffffffu, !fine);
      // a power of two takes the row's largest to 2^14 .. 2^15: a bf16 number keeps all its bits, unless it lies 2^30 below
      const int e = top > 0.0f ? 14 - (static_cast<int>(__float_as_uint(top) >> 23) - 127) : 0;
#pragma unroll
      for (int j = 0; j < kSteps; ++j)
#pragma unroll
        for (int k = 0; k < 2; ++k)
          qb[u][j][k] = half2_bits(__floats2half2_rn(ldexpf(x[4 * j + 2 * k], e), ldexpf(x[4 * j + 2 * k + 1], e)));
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        const int n = 2 * c + k, other = tile * kRows + u * 8 + n;
        const int oe = __shfl_sync(0xffffffffu, e, n * 4);
        // a query that is not finite makes every score it has with a key NaN
        factor[u][k] = (bad >> (n * 4) & 15u) != 0 ? __int_as_float(0x7fffffff) : ldexpf(p.scale * kLog2e, t_k - oe);
        const int t = other / p.group;
        lim[u][k] = p.causal ? min(r.length, own + t + 1) : r.length;
        low[u][k] = p.window > 0 ? own + t - p.window + 1 : 0;
      }
    }
    float o[NT][kSteps][4] = {};
    float m[NT][2], l[NT][2];
#pragma unroll
    for (int u = 0; u < NT; ++u)
#pragma unroll
      for (int k = 0; k < 2; ++k) { m[u][k] = -INFINITY; l[u][k] = 0.0f; }

    // the warp's steps: 16 tokens of every chunk, the next step's bytes on their way while one is worked on
    struct Raw {
      uint32_t k[2][kK / 4], v[4][kV / 4], ks[2], vs[4];
    };
    const int first = key_lo + ch0 * kChunk + warp * kStep, steps = ch1 - ch0;
    int pages = -1;                                                // of the next 32 steps, one a lane
    auto fetch = [&](int it, Raw& raw) -> bool {
      if ((it & 31) == 0) {
        const int64_t tok = first + static_cast<int64_t>(it + lane) * kChunk;
        pages = it + lane < steps && tok < key_hi ? p.table[request * p.ldt + (tok >> cache.page_log2)] : -2;
      }
      const int page = __shfl_sync(0xffffffffu, pages, it & 31);
      if (page < 0 || page >= cache.n_pages) { paged &= page == -2; return false; }
      const int tok = first + it * kChunk, place = tok & ((1 << cache.page_log2) - 1);
      const int64_t kr = kv4::cache_row(cache, page, 0, head, place), vr = kv4::cache_row(cache, page, 1, head, place);
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const int64_t row = kr + (g >> 1) + 4 * (g & 1) + 8 * h;
        load_stream<kK>(cache.codes + row * (HELD / 2) + c * kK, raw.k[h]);
        raw.ks[h] = load_scales<HELD / 64>(cache.scales + row * (HELD / 16) + c * (HELD / 64));
      }
#pragma unroll
      for (int h = 0; h < 4; ++h) {
        const int64_t row = vr + c + 4 * h;
        load_stream<kV>(cache.codes + row * (HELD / 2) + g * kV, raw.v[h]);
        raw.vs[h] = load_scales<(HELD == 256 ? 2 : 1)>(cache.scales + row * (HELD / 16) + (HELD == 256 ? 2 * g : HELD == 128 ? g : g >> 1));
      }
      return true;
    };
    Raw cur, next;
    bool have = steps > 0 && fetch(0, cur);
#pragma unroll 1
    for (int it = 0; it < steps; ++it) {
      bool more = false;
      if (it + 1 < steps) more = fetch(it + 1, next);
      if (have) {
        const int tok = first + it * kChunk;
        // scores of tokens tok + place(g) and + 8, rows 2 c and 2 c + 1 of every eight
        float sc[NT][4] = {};
        {
          __half2 ks[2][HELD / 64];
#pragma unroll
          for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int b = 0; b < HELD / 64; ++b) {
              const __half2 two = scales_of(cur.ks[h] >> (b & ~1) * 8);
              ks[h][b] = (b & 1) ? __high2half2(two) : __low2half2(two);
            }
#pragma unroll
          for (int j = 0; j < kSteps; j += 2) {
            __half2 x0[4], x1[4];
            values8(cur.k[0][j / 2], x0);
            values8(cur.k[1][j / 2], x1);
#pragma unroll
            for (int k = 0; k < 4; ++k) { x0[k] = __hmul2(x0[k], ks[0][j / 4]); x1[k] = __hmul2(x1[k], ks[1][j / 4]); }
#pragma unroll
            for (int u = 0; u < NT; ++u) {
              mma16816(sc[u], half2_bits(x0[0]), half2_bits(x1[0]), half2_bits(x0[1]), half2_bits(x1[1]), qb[u][j][0], qb[u][j][1]);
              mma16816(sc[u], half2_bits(x0[2]), half2_bits(x1[2]), half2_bits(x0[3]), half2_bits(x1[3]), qb[u][j + 1][0], qb[u][j + 1][1]);
            }
          }
        }
        const bool edge = tok < all_lo || tok + kStep > all_hi;
        bool grows = false;
#pragma unroll
        for (int u = 0; u < NT; ++u)
#pragma unroll
          for (int k = 0; k < 4; ++k) {
            sc[u][k] *= factor[u][k & 1];
            if (edge) {
              const int t = tok + (g >> 1) + 4 * (g & 1) + 8 * (k >> 1);
              if (t >= lim[u][k & 1] || t < low[u][k & 1]) sc[u][k] = -INFINITY;
            }
            grows |= sc[u][k] > m[u][k & 1] + 8.0f;
          }
        if (__any_sync(0xffffffffu, grows)) {
#pragma unroll
          for (int u = 0; u < NT; ++u)
#pragma unroll
            for (int k = 0; k < 2; ++k) {
              float top = fmaxf(sc[u][k], sc[u][k + 2]);
#pragma unroll
              for (int d = 4; d < 32; d <<= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, d));
              if (top > m[u][k]) {
                const float f = exp2_fast(m[u][k] - top);           // 0 at the first
                m[u][k] = top;
                l[u][k] *= f;
#pragma unroll
                for (int j = 0; j < kSteps; ++j) { o[u][j][k] *= f; o[u][j][k + 2] *= f; }
              }
            }
        }
        uint32_t pb[NT][2];
#pragma unroll
        for (int u = 0; u < NT; ++u) {
          float w[4];
#pragma unroll
          for (int k = 0; k < 4; ++k) {
            const float base = m[u][k & 1] == -INFINITY ? 0.0f : m[u][k & 1];
            w[k] = exp2_fast(sc[u][k] - base);
            l[u][k & 1] += w[k];
          }
          pb[u][0] = transposed(half2_bits(__floats2half2_rn(w[0], w[1])));
          pb[u][1] = transposed(half2_bits(__floats2half2_rn(w[2], w[3])));
        }
        // values: of tokens c and c + 4 (the upper half: + 8) two channels at a time
        if (tok + kStep > key_hi) {
#pragma unroll
          for (int h = 0; h < 4; ++h)
            if (tok + c + 4 * h >= key_hi) cur.vs[h] = 0;
        }
        uint32_t any_nan = 0;
#pragma unroll
        for (int h = 0; h < 4; ++h) any_nan |= ((cur.vs[h] & 0x7f7fu) + 0x0101u) & 0x8080u;
        if (__any_sync(0xffffffffu, any_nan != 0)) {
          // values that are NaN reach the rows that see their token and no other
#pragma unroll 1
          for (int src = 0; src < 4; ++src)
#pragma unroll
            for (int h = 0; h < 4; ++h) {
              const uint32_t nan = __shfl_sync(0xffffffffu, ((cur.vs[h] & 0x7f7fu) + 0x0101u) & 0x8080u, (lane & ~3) + src);
              const int t = tok + src + 4 * h;
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
#pragma unroll
          for (int h = 0; h < 4; ++h) {
            if ((cur.vs[h] & 0x7fu) == 0x7fu) cur.vs[h] &= 0xff00u;
            if ((cur.vs[h] & 0x7f00u) == 0x7f00u) cur.vs[h] &= 0xffu;
          }
        }
        __half2 vs[2][HELD == 256 ? 2 : 1];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          vs[h][0] = scales_of((cur.vs[2 * h] & 0xffu) | (cur.vs[2 * h + 1] & 0xffu) << 8);
          if constexpr (HELD == 256) vs[h][1] = scales_of((cur.vs[2 * h] >> 8) | (cur.vs[2 * h + 1] & 0xff00u));
        }
        // a lane's byte j holds its channels 2 j and 2 j + 1: rows g and g + 8 of the product's j-th step of channels
#pragma unroll
        for (int w = 0; w < kV / 4; ++w) {
          __half2 lo0[4], hi0[4], lo1[4], hi1[4];
          const uint32_t a = cur.v[0][w], b = cur.v[1][w], d = cur.v[2][w], f = cur.v[3][w];
          values8((a & 0x0f0f0f0fu) | (b << 4 & 0xf0f0f0f0u), lo0);
          values8((a >> 4 & 0x0f0f0f0fu) | (b & 0xf0f0f0f0u), hi0);
          values8((d & 0x0f0f0f0fu) | (f << 4 & 0xf0f0f0f0u), lo1);
          values8((d >> 4 & 0x0f0f0f0fu) | (f & 0xf0f0f0f0u), hi1);
#pragma unroll
          for (int k = 0; k < 4; ++k) {
            const int j = 4 * w + k;
            const __half2 s0 = vs[0][HELD == 256 && j >= 8 ? 1 : 0], s1 = vs[1][HELD == 256 && j >= 8 ? 1 : 0];
            const uint32_t a0 = half2_bits(__hmul2(lo0[k], s0)), a1 = half2_bits(__hmul2(hi0[k], s0));
            const uint32_t a2 = half2_bits(__hmul2(lo1[k], s1)), a3 = half2_bits(__hmul2(hi1[k], s1));
#pragma unroll
            for (int u = 0; u < NT; ++u) mma16816(o[u][j], a0, a1, a2, a3, pb[u][0], pb[u][1]);
          }
        }
      }
      cur = next;
      have = more;
    }

    // the warps' parts together
#pragma unroll
    for (int u = 0; u < NT; ++u)
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        float sum = l[u][k];
#pragma unroll
        for (int d = 4; d < 32; d <<= 1) sum += __shfl_xor_sync(0xffffffffu, sum, d);
        const int row = u * 8 + 2 * c + k;
        if (g == 0) { sm_m[warp][row] = m[u][k]; sm_l[warp][row] = sum; }
        float* to = so + (warp * kRows + row) * kPitch + g * (HELD / 8);
#pragma unroll
        for (int j = 0; j < kSteps; ++j) *reinterpret_cast<float2*>(to + 2 * j) = make_float2(o[u][j][k], o[u][j][k + 2]);
      }
    __syncthreads();
    const bool whole = starts && ends;
    const int slot = starts ? 1 : 0;
    for (int e = tid; e < rows * HELD; e += kFewThreads) {
      const int row = e / HELD, d = e - row * HELD;
      float top = sm_m[0][row];
#pragma unroll
      for (int w = 1; w < kFewWarps; ++w) top = fmaxf(top, sm_m[w][row]);
      float sum = 0.0f, v = 0.0f;
#pragma unroll
      for (int w = 0; w < kFewWarps; ++w) {
        const float f = sm_m[w][row] == -INFINITY && top != -INFINITY ? 0.0f : top == -INFINITY ? 1.0f : exp2_fast(sm_m[w][row] - top);
        sum += sm_l[w][row] * f;
        // a warp that saw nothing adds nothing; one that saw a NaN adds it
        v += so[(w * kRows + row) * kPitch + d] * f;
      }
      if (whole) {
        if (d < cache.dim) {
          const int rr = tile * kRows + row, tok = rr / p.group, h = head * p.group + rr - tok * p.group;
          T* out = static_cast<T*>(p.o.p) + (r.first + tok) * p.o.ld + h * p.o.lh;
          out[d] = static_cast<T>(sum == 0.0f ? v : ldexpf(v / sum, t_v));
        }
      } else {
        const int64_t at_row = (static_cast<int64_t>(blockIdx.x) * 2 + slot) * kRows + row;
        part.o[at_row * HELD + d] = v;
        if (d == 0) part.stats[at_row] = make_float2(top, sum);
      }
    }
    if (!whole) {
      if (starts) { desc.x = request; desc.y = head; desc.z = tile; desc.w |= kBegins; }
      if (!starts && ends) desc.w |= kEnds;
    }
    __syncthreads();
  }
  if (tid == 0) part.desc[blockIdx.x] = desc;
  if (__any_sync(0xffffffffu, !paged) && lane == 0) report(p.status_dev, ADADIM_ERR_PAGES);
}

// ---- joining what was cut ---------------------------------------------------------------------------
// CTA (b, row): the unit that began in part b and went on.  Its parts are those of b, b + 1, .. up to the one it ends in, the
// warps take every eighth of them; the sums are formed in that order.
constexpr int kJoinThreads = 256, kJoinWarps = 8;

template <int HELD, int NT, typename T>
__global__ void __launch_bounds__(kJoinThreads) kv4_join_kernel(Kv4Attention p, int ctas) {
  constexpr int kRows = 8 * NT, kEach = HELD / 32;
  __shared__ float acc[kJoinWarps][HELD];
  __shared__ float sm_m[kJoinWarps], sm_l[kJoinWarps];
  const int b = blockIdx.x, row = blockIdx.y, tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  ptx::pdl_wait();
  const Partials part = partials_of(p.workspace, ctas, kRows);
  const int4 desc = part.desc[b];
  if ((desc.w & kBegins) == 0) return;
  int last = b + 1;                                                  // the part it ends in
  for (int k = b + 1; k < ctas; k += 32) {
    const uint32_t found = __ballot_sync(0xffffffffu, k + lane < ctas && (part.desc[k + lane].w & kEnds) != 0);
    if (found != 0) { last = k + __ffs(static_cast<int>(found)) - 1; break; }
  }
  bool ok;
  const Request r = kv4::request_of(p.offsets, p.lengths, desc.x, p.n_rows, p.width << p.cache.page_log2, ok);
  const int rr = desc.z * kRows + row;
  if (rr >= r.rows * p.group) return;
  float m = -INFINITY, l = 0.0f, v[kEach] = {};
  for (int k = b + warp; k <= last; k += kJoinWarps) {
    const int64_t at = (static_cast<int64_t>(k) * 2 + (k == b ? 1 : 0)) * kRows + row;
    const float2 s = part.stats[at];
    const float top = fmaxf(m, s.x);
    const float f = m == -INFINITY ? 1.0f : exp2_fast(m - top), h = s.x == -INFINITY ? 1.0f : exp2_fast(s.x - top);
    // (a part without a maximum holds zeros, or NaN)
    m = top;
    l = l * f + s.y * h;
#pragma unroll
    for (int e = 0; e < kEach; ++e) v[e] = v[e] * f + part.o[at * HELD + e * 32 + lane] * h;
  }
#pragma unroll
  for (int e = 0; e < kEach; ++e) acc[warp][e * 32 + lane] = v[e];
  if (lane == 0) { sm_m[warp] = m; sm_l[warp] = l; }
  __syncthreads();
  float top = sm_m[0];
#pragma unroll
  for (int w = 1; w < kJoinWarps; ++w) top = fmaxf(top, sm_m[w]);
  const int tok = rr / p.group, h = desc.y * p.group + rr - tok * p.group;
  T* out = static_cast<T*>(p.o.p) + (r.first + tok) * p.o.ld + h * p.o.lh;
  const int t_v = kv4::cache_scale_log2(p.cache, 1);
  for (int d = tid; d < p.cache.dim; d += kJoinThreads) {
    float sum = 0.0f, x = 0.0f;
#pragma unroll
    for (int w = 0; w < kJoinWarps; ++w) {
      const float f = sm_m[w] == -INFINITY ? 1.0f : exp2_fast(sm_m[w] - top);
      sum += sm_l[w] * f;
      x += acc[w][d] * f;
    }
    out[d] = static_cast<T>(sum == 0.0f ? x : ldexpf(x / sum, t_v));
  }
}

template <int HELD, int NT, typename T>
int few_launch(const Kv4Attention& a, cudaStream_t st) {
  constexpr size_t kFixed = sizeof(float) * kFewWarps * 8 * NT * (HELD + 4);
  static std::atomic<uint64_t> done{0};
  const int rc = set_once(kv4_few_kernel<HELD, NT, T>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                          static_cast<int>(kFixed + sizeof(int64_t) * (kv4::kMaxRequests + 1)), done);
  if (rc != ADADIM_OK) return rc;
  const size_t smem = kFixed + sizeof(int64_t) * (static_cast<size_t>(a.n_requests) + 1);
  kv4_few_kernel<HELD, NT, T><<<kFewCtas, kFewThreads, smem, st>>>(a);
  ADADIM_CUDA_TRY(cudaGetLastError());
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(kFewCtas, 8 * NT);
  cfg.blockDim = dim3(kJoinThreads);
  cfg.stream = st;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  ADADIM_CUDA_TRY(cudaLaunchKernelEx(&cfg, kv4_join_kernel<HELD, NT, T>, a, static_cast<int>(kFewCtas)));
  return ADADIM_OK;
}
template <int HELD, typename T>
int few_held(const Kv4Attention& a, int64_t max_new, cudaStream_t st) {
  if (HELD < 256 && max_new * a.group > 8) return few_launch<HELD, HELD < 256 ? 2 : 1, T>(a, st);
  return few_launch<HELD, 1, T>(a, st);
}
template <typename T>
int few_type(const Kv4Attention& a, int64_t max_new, cudaStream_t st) {
  if (a.cache.held == 64) return few_held<64, T>(a, max_new, st);
  return a.cache.held == 128 ? few_held<128, T>(a, max_new, st) : few_held<256, T>(a, max_new, st);
}

}  // namespace

size_t kv4_workspace(int64_t n_requests, int64_t n_rows, int q_heads, int kv_heads, int head_dim) {
  const int held = kv4::held_dim(head_dim);
  return partials_bytes(kFewCtas, held < 256 ? 16 : 8, held);
}

int kv4_attention_launch(const Kv4Attention& a, int dtype, int64_t max_new, cudaStream_t st) {
  Kv4Attention few = a;
  few.few_rows = 0x7fffffff;
  return dtype == ADADIM_F16 ? few_type<__half>(few, max_new, st) : few_type<__nv_bfloat16>(few, max_new, st);
}

}  // namespace adadim
