// Attention over the 4-bit key-value cache: which kernels a call takes, and the joining of what they cut.
#include "kv4_line.cuh"

namespace adadim {
namespace {

using namespace kv4;

// ---- joining what was cut ---------------------------------------------------------------------------
// The unit that began in part b and went on: its parts are those of b, b + 1, .. up to the one it ends in.  A warp has a row and goes
// through them in that order; with SPLIT, where few units are cut into many parts, the eight warps of a CTA have one row of the few-row
// kernel's and take every eighth part.  Either way the order of the sums is fixed.  One launch joins both kernels' units: the first
// few_blocks CTAs those of the kernel for few rows.
constexpr int kJoinThreads = 256, kJoinWarps = 8;
constexpr int kManyBlocks = 8;                   // CTAs that share a unit of the kernel for many rows, whose warps have several rows each

struct Joined {
  char* workspace;
  int ctas, tile_rows;
};

template <int HELD, bool SPLIT, typename T>
__global__ void __launch_bounds__(kJoinThreads) kv4_join_kernel(Kv4Attention p, Joined few, Joined many, int few_blocks) {
  constexpr int kEach = HELD / 32;
  __shared__ float acc[SPLIT ? kJoinWarps : 1][HELD];
  __shared__ float2 stats[kJoinWarps];
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const bool of_few = static_cast<int>(blockIdx.x) < few_blocks, split = SPLIT && of_few;
  const Joined& from = of_few ? few : many;
  const int at_block = of_few ? blockIdx.x : blockIdx.x - few_blocks, ys = split ? from.tile_rows : of_few ? from.tile_rows / kJoinWarps : kManyBlocks;
  const int b = at_block / ys, y = at_block - b * ys;
  ptx::pdl_wait();
  const Partials part = partials_of(from.workspace, from.ctas, from.tile_rows);
  const int4 desc = part.desc[b];
  if ((desc.w & kBegins) == 0) return;
  int last = b + 1;                                                  // the part it ends in
  for (int k = b + 1; k < from.ctas; k += 32) {
    const uint32_t found = __ballot_sync(0xffffffffu, k + lane < from.ctas && (part.desc[k + lane].w & kEnds) != 0);
    if (found != 0) { last = k + __ffs(static_cast<int>(found)) - 1; break; }
  }
  bool ok;
  const Request r = request_of(p.offsets, p.lengths, desc.x, p.n_rows, p.width << p.cache.page_log2, ok);
  const int t_v = cache_scale_log2(p.cache, 1), rows = r.rows * p.group - desc.z * from.tile_rows;
  for (int row = split ? y : y * kJoinWarps + warp; row < min(rows, from.tile_rows); row += split ? from.tile_rows : ys * kJoinWarps) {
  const int rr = desc.z * from.tile_rows + row;
  float m = -INFINITY, l = 0.0f, v[kEach] = {};
#pragma unroll 4
  for (int k = b + (split ? warp : 0); k <= last; k += split ? kJoinWarps : 1) {
    const int64_t at = (static_cast<int64_t>(k) * 2 + (k == b ? 1 : 0)) * from.tile_rows + row;
    const float2 s = part.stats[at];
    float o[kEach];
#pragma unroll
    for (int e = 0; e < kEach; ++e) o[e] = part.o[at * HELD + e * 32 + lane];
    // a part without a maximum holds zeros, or NaN
    const float top = fmaxf(m, s.x), f = m == -INFINITY ? 1.0f : exp2_fast(m - top), h = s.x == -INFINITY ? 1.0f : exp2_fast(s.x - top);
    m = top;
    l = l * f + s.y * h;
#pragma unroll
    for (int e = 0; e < kEach; ++e) v[e] = v[e] * f + o[e] * h;
  }
  const int tok = token_of(p, rr), head = desc.y * p.group + rr - tok * p.group;
  T* out = static_cast<T*>(p.o.p) + (r.first + tok) * p.o.ld + head * p.o.lh;
  if (split) {
    if constexpr (SPLIT) {
#pragma unroll
      for (int e = 0; e < kEach; ++e) acc[warp][e * 32 + lane] = v[e];
      if (lane == 0) stats[warp] = make_float2(m, l);
      __syncthreads();
      float top = stats[0].x;
#pragma unroll
      for (int w = 1; w < kJoinWarps; ++w) top = fmaxf(top, stats[w].x);
      for (int d = tid; d < p.cache.dim; d += kJoinThreads) {
        float sum = 0.0f, x = 0.0f;
#pragma unroll
        for (int w = 0; w < kJoinWarps; ++w) {
          const float f = stats[w].x == -INFINITY ? 1.0f : exp2_fast(stats[w].x - top);
          sum += stats[w].y * f;
          x += acc[w][d] * f;
        }
        out[d] = static_cast<T>(sum == 0.0f ? x : ldexpf(x / sum, t_v));
      }
    }
  } else {
#pragma unroll
    for (int e = 0; e < kEach; ++e) {
      const int d = e * 32 + lane;
      if (d < p.cache.dim) out[d] = static_cast<T>(l == 0.0f ? v[e] : ldexpf(v[e] / l, t_v));
    }
  }
  }
}

template <int HELD, bool SPLIT, typename T>
int join(const Kv4Attention& a, const Joined& few, const Joined& many, cudaStream_t st) {
  const int few_blocks = few.ctas * (SPLIT ? few.tile_rows : few.tile_rows / kJoinWarps), many_blocks = many.ctas * kManyBlocks;
  return chained_launch(kv4_join_kernel<HELD, SPLIT, T>, dim3(static_cast<unsigned>(few_blocks + many_blocks)), kJoinThreads, 0, true, st, a, 1, few, many,
                        few_blocks);
}
template <bool SPLIT, typename T>
int join_held(const Kv4Attention& a, const Joined& few, const Joined& many, cudaStream_t st) {
  if (a.cache.held == 64) return join<64, SPLIT, T>(a, few, many, st);
  return a.cache.held == 128 ? join<128, SPLIT, T>(a, few, many, st) : join<256, SPLIT, T>(a, few, many, st);
}

// The kernel for many rows holds its line of work beside 192 KB of tiles, and TMEM has no room for heads of 256 channels (a prompt of 4096
// tokens of 16 such heads takes 1.2 ms in the other one, where 32 heads of 128 take 0.21 here).
bool many_possible(int64_t n_requests, int held) { return n_requests <= kManyRequests && held <= 128; }

}  // namespace

size_t kv4_workspace(int64_t n_requests, int64_t n_rows, int q_heads, int kv_heads, int head_dim) {
  const int held = held_dim(head_dim);
  const bool many = many_possible(n_requests, held) && n_rows * (q_heads / kv_heads) > kFewRows;
  return kv4_few_workspace(held) + (many ? kv4_many_workspace(held) : 0);
}

// The kernels follow one another by programmatic launches: each may begin when the one before it has begun everywhere, and ends
// no earlier than that one, so that what comes behind the last one comes behind them all.
int kv4_attention_launch(const Kv4Attention& given, int dtype, int64_t max_new, cudaStream_t st) {
  Kv4Attention a = given;
  a.group_rcp = a.group == 1 ? 0 : static_cast<uint32_t>((uint64_t{1} << 32) / a.group + 1);
  a.wide_q = reinterpret_cast<uintptr_t>(a.q.p) % 8 == 0 && a.q.ld % 4 == 0 && a.q.lh % 4 == 0;
  a.wide16_q = reinterpret_cast<uintptr_t>(a.q.p) % 16 == 0 && a.q.ld % 8 == 0 && a.q.lh % 8 == 0;
  a.wide16_o = reinterpret_cast<uintptr_t>(a.o.p) % 16 == 0 && a.o.ld % 8 == 0 && a.o.lh % 8 == 0;
  a.least_rows = 1;
  a.most_rows = int64_t{1} << 40;
  Joined few = {a.workspace, 0, 0}, many = {a.workspace + kv4_few_workspace(a.cache.held), 0, kJoinWarps};
  int rc;
  if (max_new * a.group > kFewRows && many_possible(a.n_requests, a.cache.held) && !kv4_few_suits(a, max_new)) {
    a.least_rows = kFewBeside + 1;
    a.workspace = many.workspace;
    rc = kv4_many_launch(a, dtype, many.ctas, many.tile_rows, st);
    if (rc != ADADIM_OK) return rc;
    a.least_rows = 1;
    a.most_rows = kFewBeside;
    a.workspace = few.workspace;
  }
  rc = kv4_few_launch(a, dtype, max_new, many.ctas > 0, few.ctas, few.tile_rows, st);
  if (rc != ADADIM_OK) return rc;
  if (few.ctas + many.ctas == 0) return ADADIM_OK;
  // few units are cut into many parts each: one of 100000 tokens takes 103 us with a CTA a row, 111 with a warp; 512 of 16384 take 148 and 140
  const bool split = static_cast<int64_t>(a.n_requests) * a.cache.kv_heads < 64;
  if (dtype == ADADIM_F16) return split ? join_held<true, __half>(a, few, many, st) : join_held<false, __half>(a, few, many, st);
  return split ? join_held<true, __nv_bfloat16>(a, few, many, st) : join_held<false, __nv_bfloat16>(a, few, many, st);
}

}  // namespace adadim
