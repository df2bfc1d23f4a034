// Attention over the 4-bit key-value cache: what the kernels for few and for many query rows share.  The line of work that is cut
// into equal parts, where the parts of cut units are kept, numbers out of codes.  Internal header.
#pragma once

#include "kv4.cuh"

namespace adadim {
namespace kv4 {

constexpr int kSms = 148;
// Rows a key head up to which the kernel for few rows has a call (a cache of 16 requests of up to 8192 tokens: 24 rows 68 us against 79, 32 rows
// 69 against 83, 40 rows 88 against 83), and those that it takes, in eights, of a call with both kernels.
constexpr int kFewRows = 32, kFewBeside = 16;
constexpr int kManyRequests = 3500;              // of a call, for the many-row kernel
constexpr float kLog2e = 1.4426950408889634f;
// Weights are fp16, 2^7 times what they are to the row's reference: its largest score when it was last taken, which is done where a score
// passes it by more than 2^8, so that they end at 2^15.  So they have their 11 bits down to 2^-21 of the reference's, below that
// fp16's least step, 2^-31 of it, and a reference's own weight is in every row's sum.  (Without the 2^7, 2^-14 and 2^-24.)
constexpr float kGrowth = 8.0f, kLift = 7.0f;
// What is subtracted from scores whose reference is m: rounded up, so that no weight passes 2^15 where binary32 holds scores in steps of two
// and more (how far a score passes m is asked for by their difference, which such steps do not change).
__device__ __forceinline__ float lifted(float m) { return m == -INFINITY ? 0.0f : __fsub_ru(m, kLift); }

__host__ __device__ constexpr size_t whole256(size_t bytes) { return (bytes + 255) / 256 * 256; }

// ---- arithmetic --------------------------------------------------------------------------------------
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
__device__ __forceinline__ float exp2_fast(float x) {
  float r;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(r) : "f"(x));
  return r;
}
// a / b where both mostly fit 32 bits
__device__ __forceinline__ int64_t quick_div(int64_t a, int64_t b) {
  if (((a | b) >> 32) == 0) return static_cast<uint32_t>(a) / static_cast<uint32_t>(b);
  return a / b;
}
// A word of 16-bit queries as fp16 times f = 2^e (fp16 queries: as they are).
template <typename T>
__device__ __forceinline__ uint32_t query_bits(uint32_t raw, float f) {
  if constexpr (std::is_same<T, __half>::value) return raw;
  else return half2_bits(__floats2half2_rn(__uint_as_float(raw << 16) * f, __uint_as_float(raw & 0xffff0000u) * f));
}
// bf16 rows are multiplied by the power of two that takes their largest to 2^14 .. 2^15 (2^127 at most, where it is below 2^-113): a
// number keeps all its bits unless it lies 2^16 below the largest, and then is off by 2^-25 of the largest or less.
// top: the row's largest magnitude as a pattern (patterns are ordered).
template <typename T>
__device__ __forceinline__ int query_exponent(uint32_t top) { return std::is_same<T, __half>::value ? 0 : min(127, 141 - static_cast<int>(top >> 7)); }
template <typename T>
__device__ __forceinline__ bool query_fine(uint32_t top) { return top < (std::is_same<T, __half>::value ? 0x7c00u : 0x7f80u); }

// ---- the line of work --------------------------------------------------------------------------------
// A unit: the query rows of one tile (row r of a request is token r / group, head r % group of the key head's) and the
// tokens of the cache that some of them sees.  All units lie on one line, request after request, key head after key head, tile after tile,
// each as long as it has tokens and a fixed cost, and the line is cut into equal parts, one a CTA, whatever the
// requests' lengths.  A tile's length is an estimate that is the same for every reader.
struct Shape {
  int tiles;               // of a key head
  int64_t first, step;     // tile t takes first + t step of the line
  __device__ __forceinline__ int64_t before(int64_t t) const { return t * first + step * (t * (t - 1) / 2); }
};
__device__ __forceinline__ Shape shape_of(const Kv4Attention& p, const Request& r, int tile_rows, int cost) {
  Shape s = {0, 0, 0};
  const int64_t rows = static_cast<int64_t>(r.rows) * p.group;
  if (rows < p.least_rows || rows > p.most_rows || rows == 0) return s;
  s.tiles = static_cast<int>((rows + tile_rows - 1) / tile_rows);
  const int64_t each = min(r.rows, (tile_rows + p.group - 1) / p.group), own = r.length - r.rows;
  if (!p.causal) s.first = r.length;
  else if (p.window > 0) s.first = min(static_cast<int64_t>(r.length), p.window + each);
  else {
    s.first = max(int64_t{0}, min(static_cast<int64_t>(r.length), own + each));
    s.step = s.tiles > 1 ? each : 0;
  }
  s.first += cost;
  return s;
}
// token of a row: row / group by a reciprocal that the host has formed
__device__ __forceinline__ int token_of(const Kv4Attention& p, int row) {
  if (p.group == 1) return row;
  const uint32_t t = __umulhi(static_cast<uint32_t>(row), p.group_rcp);      // the quotient or one more
  return static_cast<int>(t - (t * static_cast<uint32_t>(p.group) > static_cast<uint32_t>(row) ? 1u : 0u));
}
// Work in front of each request into line[0 .. n_requests]; for all threads of a CTA, the first 128 of which sum up.
__device__ __forceinline__ void sum_line(const Kv4Attention& p, int tile_rows, int cost, int64_t* line, int64_t (&sums)[4]) {
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int64_t most = p.width << p.cache.page_log2;
  int64_t carry = 0;
  bool good = true;
  for (int i0 = 0; i0 < p.n_requests; i0 += 128) {
    const int i = i0 + tid;
    int64_t w = 0, sum = 0;
    if (tid < 128) {
      if (i < p.n_requests) {
        bool ok;
        const Request r = request_of(p.offsets, p.lengths, i, p.n_rows, most, ok);
        good &= ok;
        const Shape s = shape_of(p, r, tile_rows, cost);
        w = s.before(s.tiles) * p.cache.kv_heads;
      }
      sum = w;
#pragma unroll
      for (int d = 1; d < 32; d <<= 1) {
        const int64_t u = __shfl_up_sync(0xffffffffu, sum, d);
        if (lane >= d) sum += u;
      }
      if (lane == 31) sums[warp] = sum;
    }
    __syncthreads();
    int64_t before = carry;
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      if (k < warp) before += sums[k];
      carry += sums[k];
    }
    if (tid < 128 && i < p.n_requests) line[i] = before + sum - w;
    __syncthreads();
  }
  if (tid == 0) line[p.n_requests] = carry;
  if (!good && blockIdx.x == 0) report(p.status_dev, ADADIM_ERR_SHAPE);
  __syncthreads();
}

// One CTA's part of a unit.
struct Piece {
  Request r;
  int request, head, tile, rows;       // rows of the tile
  int seen_lo, key_lo, chunks;         // first token that some row sees, that rounded down to a multiple of 32, chunks of all of them
  int c0, c1;                          // this piece's chunks
  bool starts, ends;                   // the unit begins, ends in it
};
// The piece that begins at `at`, which is moved to the next one's begin.
__device__ __forceinline__ Piece next_piece(const Kv4Attention& p, const int64_t* line, int64_t& at, int64_t end, int request, int tile_rows, int cost,
                                            int chunk) {
  Piece x;
  int lo = request, hi = p.n_requests;
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (line[mid] <= at) lo = mid; else hi = mid;
  }
  x.request = lo;
  bool ok;
  x.r = request_of(p.offsets, p.lengths, lo, p.n_rows, p.width << p.cache.page_log2, ok);
  const Shape s = shape_of(p, x.r, tile_rows, cost);
  const int64_t of_head = s.before(s.tiles), within = at - line[lo];
  x.head = static_cast<int>(quick_div(within, of_head));
  const int64_t rest = within - x.head * of_head;
  int t = 0, above = s.tiles;
  while (above - t > 1) {
    const int mid = (t + above) >> 1;
    if (s.before(mid) <= rest) t = mid; else above = mid;
  }
  x.tile = t;
  const int64_t unit = s.first + t * s.step, begin = rest - s.before(t), stop = min(unit, begin + end - at);
  at += stop - begin;
  x.starts = begin == 0;
  x.ends = stop == unit;
  x.rows = static_cast<int>(min(static_cast<int64_t>(tile_rows), static_cast<int64_t>(x.r.rows) * p.group - static_cast<int64_t>(t) * tile_rows));
  const int t0 = token_of(p, t * tile_rows), t1 = token_of(p, t * tile_rows + x.rows - 1), own = x.r.length - x.r.rows;
  const int key_hi = p.causal ? max(0, min(x.r.length, own + t1 + 1)) : x.r.length;
  x.seen_lo = p.window > 0 ? max(0, own + t0 - p.window + 1) : 0;
  x.key_lo = x.seen_lo & ~31;
  x.chunks = key_hi > x.key_lo ? (key_hi - x.key_lo + chunk - 1) / chunk : 0;
  const int from = begin <= cost ? 0 : static_cast<int>(min(static_cast<int64_t>(x.chunks), (begin - cost + chunk - 1) / chunk));
  const int to = stop <= cost ? 0 : static_cast<int>(min(static_cast<int64_t>(x.chunks), (stop - cost + chunk - 1) / chunk));
  x.c0 = x.starts ? 0 : from;
  x.c1 = x.ends ? x.chunks : to;
  return x;
}
__device__ __forceinline__ int key_end(const Kv4Attention& p, const Piece& x, int last_row);
// A whole unit, of a request that has the tile.
__device__ __forceinline__ Piece whole_unit(const Kv4Attention& p, const Request& r, int request, int head, int tile, int tile_rows, int chunk) {
  Piece x;
  x.r = r;
  x.request = request;
  x.head = head;
  x.tile = tile;
  x.rows = static_cast<int>(min(static_cast<int64_t>(tile_rows), static_cast<int64_t>(r.rows) * p.group - static_cast<int64_t>(tile) * tile_rows));
  x.seen_lo = p.window > 0 ? max(0, r.length - r.rows + token_of(p, tile * tile_rows) - p.window + 1) : 0;
  x.key_lo = x.seen_lo & ~31;
  const int hi = key_end(p, x, tile * tile_rows + x.rows - 1);
  x.chunks = hi > x.key_lo ? (hi - x.key_lo + chunk - 1) / chunk : 0;
  x.c0 = 0;
  x.c1 = x.chunks;
  x.starts = x.ends = true;
  return x;
}
__device__ __forceinline__ int key_end(const Kv4Attention& p, const Piece& x, int last_row) {      // behind the last token that a row up to last_row of the request sees
  return p.causal ? max(0, min(x.r.length, x.r.length - x.r.rows + token_of(p, last_row) + 1)) : x.r.length;
}

// ---- parts of cut units --------------------------------------------------------------------------------
enum : int { kBegins = 1, kEnds = 2 };           // a cut unit begins in this CTA's part (and goes on) / one from before ends in it

// Slot 0 of a CTA is for the unit that began before, slot 1 for the one that goes on.
struct Partials {
  int4* desc;              // request, head, tile of the unit that begins; kBegins, kEnds
  float2* stats;           // [cta][2][rows] maximum and sum
  float* o;                // [cta][2][rows][held]
};
__host__ __device__ inline Partials partials_of(char* ws, int ctas, int rows) {
  Partials p;
  p.desc = reinterpret_cast<int4*>(ws);
  p.stats = reinterpret_cast<float2*>(ws + whole256(sizeof(int4) * ctas));
  p.o = reinterpret_cast<float*>(reinterpret_cast<char*>(p.stats) + whole256(sizeof(float2) * 2 * ctas * rows));
  return p;
}
__host__ __device__ constexpr size_t partials_bytes(int ctas, int rows, int held) {
  return whole256(sizeof(int4) * ctas) + whole256(sizeof(float2) * 2 * ctas * rows) + whole256(sizeof(float) * 2 * ctas * rows * held);
}
// What a CTA writes down of a piece that is not a whole unit.
__device__ __forceinline__ void note_piece(int4& desc, const Piece& x) {
  if (x.starts) { desc.x = x.request; desc.y = x.head; desc.z = x.tile; desc.w |= kBegins; }
  else if (x.ends) desc.w |= kEnds;
}

}  // namespace kv4
}  // namespace adadim
