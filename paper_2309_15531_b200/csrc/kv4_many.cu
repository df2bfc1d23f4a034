// Attention over the 4-bit key-value cache for many query rows a key head: prompts, pieces of prompts, many drafted tokens.
//
// Bound by arithmetic: 4 dim operations for every pair of a query and a key, on the tensor cores (tcgen05, fp16 operands, binary32
// accumulators in TMEM), and as much by the exponentials between the two products: 128 x 128 pairs are 1024 cycles of either
// unit.  A CTA has 256 query rows in two tiles of 128 (a group of heads of one key head, tokens outer), so that
// one tile's softmax runs while the other one's products do:
//   warps 0-3, 4-7   a tile each: a thread has a row, takes its scores from TMEM and puts the weights back as fp16 where the scores
//                    were, from where the second product takes them; 64 tokens at a time, so that the products for one half of
//                    128 tokens run while the weights of the other are formed
//   warps 8-11       turn 128 tokens' codes into fp16 tiles in shared memory (128-byte swizzle; keys and values alike: a token
//                    is a row, which is K-major for keys and MN-major for values), two stages of each, keys a chunk ahead of
//                    values; the codes of the next two turns are loaded into registers meanwhile, so that 4-bit bytes are all
//                    that is read of the cache
//   warp 12          issues the products
//   warp 13          finds the CTA's next pieces of the line, and brings their queries into L2
// Loops that the warps are in all the time are kept short (32 scores a turn): a warp that runs through a thousand instructions
// waits for them more than it executes.
// The largest score is taken anew only where a row passes it by more than 2^8; then the accumulator in TMEM is rescaled.
// A unit of at most 128 rows has both tiles for itself: each takes every other 128 tokens, and the first tile's threads put
// the two results together from TMEM.
// The line of work is cut into one part a CTA as for few rows.
//
// Heads of 128 channels.  1024 rows of each of 64 heads over 32768 tokens: 1.10 ms, 1.02 PFLOP/s, 0.61 of cuBLAS's rate; 4096 tokens of 32
// heads over themselves: 210 us, of which 27 are the join's and about 15 the start and the ends of units.  What bounds the loop is a
// tile's chain of scores, softmax and weights: a chunk takes both tiles 2.2 us, of which 1.1 are exponentials; the tensor pipe is busy for
// half of the time, issue slots for 45 %.  16 requests of five drafted tokens (40 rows a unit) over up to 8192: 81 us, there bound by the unpacking
// warps.  These are replays of a graph; passes launched one after another take 2 to 3 % more.
#include "kv4_line.cuh"

namespace adadim {
namespace {

using namespace kv4;
using fp4::exp2_int;

constexpr int kTile = 128, kRows = 2 * kTile, kChunk = 128, kHalf = kChunk / 2;
constexpr int kUnpackWarp = 8, kUnpackWarps = 4, kIssueWarp = 12, kJobWarp = 13, kThreads = 16 * 32;   // two warps only fill up
// What a unit costs beside its tokens, in tokens: with 300, 640 and 1000 five drafted tokens of 16 requests take 113, 83 and 86 us, a prompt
// of 300 tokens 48, 33 and 40, one of 4096 204, 208 and 218.
constexpr int kCost = 640;
constexpr int kLeastPart = 1024;                 // a CTA's part is no smaller (256: the prompt of 300 tokens 41 us)
constexpr int kRing = 8;                         // chunks whose notes about tokens are kept

template <int HELD> struct Many {
  static constexpr int kBox = kTile * 128;                           // 64 channels of 128 rows
  static constexpr int kBytes = HELD / 64 * kBox;                    // a tile of queries, keys or values
  static constexpr int kQ = 0, kK = 2 * kBytes, kV = 4 * kBytes, kLine = 6 * kBytes;
  static constexpr size_t kSmem = kLine + 1024;                      // and the alignment to 1024 bytes
};

__host__ __device__ constexpr uint32_t idesc_f16(int M, int N, bool b_mn) {
  return (1u << 4) | (static_cast<uint32_t>(b_mn) << 16) | (static_cast<uint32_t>(N >> 3) << 17) | (static_cast<uint32_t>(M >> 4) << 24);
}
// D[tmem] (+)= A[tmem] * B[smem], fp16
__device__ __forceinline__ void mma_f16_ts(uint32_t d_tmem, uint32_t a_tmem, uint64_t bdesc, uint32_t idesc, bool accumulate) {
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "setp.ne.b32 p, %4, 0;\n\t"
      "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}"
      ::"r"(d_tmem), "r"(a_tmem), "l"(bdesc), "r"(idesc), "r"(static_cast<uint32_t>(accumulate))
      : "memory");
}
#define ADADIM_R32(r) "+r"(r[0]), "+r"(r[1]), "+r"(r[2]), "+r"(r[3]), "+r"(r[4]), "+r"(r[5]), "+r"(r[6]), "+r"(r[7]), "+r"(r[8]), "+r"(r[9]), \
  "+r"(r[10]), "+r"(r[11]), "+r"(r[12]), "+r"(r[13]), "+r"(r[14]), "+r"(r[15]), "+r"(r[16]), "+r"(r[17]), "+r"(r[18]), "+r"(r[19]), "+r"(r[20]), \
  "+r"(r[21]), "+r"(r[22]), "+r"(r[23]), "+r"(r[24]), "+r"(r[25]), "+r"(r[26]), "+r"(r[27]), "+r"(r[28]), "+r"(r[29]), "+r"(r[30]), "+r"(r[31])
// 32 columns of this thread's TMEM lane, there after ld32_wait of the same registers
__device__ __forceinline__ void ld32(uint32_t taddr, uint32_t (&r)[32]) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x32.b32 "
      "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, "
      "%16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31}, [%32];"
      : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]),
        "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]),
        "=r"(r[16]), "=r"(r[17]), "=r"(r[18]), "=r"(r[19]), "=r"(r[20]), "=r"(r[21]), "=r"(r[22]), "=r"(r[23]),
        "=r"(r[24]), "=r"(r[25]), "=r"(r[26]), "=r"(r[27]), "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), "=r"(r[31])
      : "r"(taddr) : "memory");
}
__device__ __forceinline__ void ld32_wait(uint32_t (&r)[32]) { asm volatile("tcgen05.wait::ld.sync.aligned;" : ADADIM_R32(r) : : "memory"); }
__device__ __forceinline__ void st16(uint32_t taddr, const uint32_t (&r)[16]) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], "
      "{%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16};"
      ::"r"(taddr), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]),
        "r"(r[8]), "r"(r[9]), "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15])
      : "memory");
}
__device__ __forceinline__ void ld16(uint32_t taddr, uint32_t (&r)[16]) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x16.b32 "
      "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];"
      : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]),
        "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
      : "r"(taddr) : "memory");
}
__device__ __forceinline__ void ld16_wait(uint32_t (&r)[16]) {
  asm volatile("tcgen05.wait::ld.sync.aligned;"
               : "+r"(r[0]), "+r"(r[1]), "+r"(r[2]), "+r"(r[3]), "+r"(r[4]), "+r"(r[5]), "+r"(r[6]), "+r"(r[7]),
                 "+r"(r[8]), "+r"(r[9]), "+r"(r[10]), "+r"(r[11]), "+r"(r[12]), "+r"(r[13]), "+r"(r[14]), "+r"(r[15]) : : "memory");
}
__device__ __forceinline__ void st_wait() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }

__device__ __forceinline__ float max3(float a, float b, float c) {
  float r;
  asm("max.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
  return r;
}

// The same value in all lanes of a converged warp, which the compiler then knows: what the products' instructions are given stays
// in uniform registers (60 cycles an instruction where it had to be brought there from every lane's).
__device__ __forceinline__ int same(int v) { return __reduce_max_sync(0xffffffffu, v); }

// A piece as all warps of the CTA take it.  Chunks of tile i: [c0, c1_of[i]), or of those every other one from c0 + i on where both
// tiles have the same rows; they begin at token key_lo, chunk 0's first.
struct __align__(16) Job {
  int first, rows_all, length, request, head, tile, rows, seen_lo, c0, c1, c1_of[2], key_hi, starts, ends, none;
  __device__ __forceinline__ int key_lo() const { return seen_lo & ~31; }
};
constexpr int kJobs = 4;                         // that lie ready

template <typename T>
__device__ __forceinline__ uint32_t two_of(float a, float b) {       // rounded, side by side
  if constexpr (std::is_same<T, __half>::value) return half2_bits(__floats2half2_rn(a, b));
  const __nv_bfloat162 h = __floats2bfloat162_rn(a, b);
  return *reinterpret_cast<const uint32_t*>(&h);
}
template <typename T>
__device__ __forceinline__ T* of_lane(T* p, int lane) { return reinterpret_cast<T*>(__shfl_sync(0xffffffffu, reinterpret_cast<unsigned long long>(p), lane)); }

struct __align__(16) Shared {
  Job jobs[kJobs];
  uint64_t job_full[kJobs], job_empty[kJobs];

  uint64_t k_full[2], k_empty[2], v_full[2], v_empty[2], q_ready[2][kJobs], s_full[2][2], p_ready[2][2], o_done[2][2],   // [tile][half of the tokens]
           twin_full, twin_free, drain;
  uint32_t tmem;
  int dead;
  uint32_t hidden[kRing][kTile / 32];            // tokens whose page lies outside the cache, a bit each
  uint32_t nan_any[kRing][kUnpackWarps];         // whether a warp's tokens have values that are NaN; which:
  uint8_t nan_of[kRing][kTile];                  // a bit for each of a token's blocks
  float twin_m[kTile], twin_l[kTile];            // the second tile's maxima, sums and NaN blocks of the rows that both have
  uint32_t twin_nans[kTile];
};

__device__ __forceinline__ bool is_twin(int rows) { return rows <= kTile; }   // both tiles have the same rows (prompts beside single tokens: 130 -> 125 us)
__device__ __forceinline__ Job job_of(const Kv4Attention& p, const Piece& x) {
  const int row0 = x.tile * kRows;
  Job j;
  j.first = x.r.first;
  j.rows_all = x.r.rows;
  j.length = x.r.length;
  j.request = x.request;
  j.head = x.head;
  j.tile = x.tile;
  j.rows = x.rows;
  j.seen_lo = x.seen_lo;
  j.c0 = x.c0;
  j.c1 = x.c1;
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const int hi = key_end(p, x, row0 + min(x.rows, (i + 1) * kTile) - 1);
    j.c1_of[i] = is_twin(x.rows) ? x.c1 : max(x.c0, min(x.c1, hi > x.key_lo ? (hi - x.key_lo + kChunk - 1) / kChunk : 0));
  }
  j.key_hi = key_end(p, x, row0 + x.rows - 1);
  j.starts = x.starts;
  j.ends = x.ends;
  j.none = 0;
  return j;
}

template <int HELD, typename T>
__global__ void __launch_bounds__(kThreads, 1) kv4_many_kernel(Kv4Attention p) {
  typedef Many<HELD> Mm;
  extern __shared__ char smem_raw[];
  char* const smem = smem_raw + (1024 - (ptx::smem_addr(smem_raw) & 1023)) % 1024;
  int64_t* line = reinterpret_cast<int64_t*>(smem + Mm::kLine);
  __shared__ Shared sh;
  __shared__ int64_t sums[4];
  volatile int* dead = &sh.dead;
  int* const status = p.status_dev;
  const int tid = threadIdx.x, lane = tid & 31, warp = ptx::uniform_warp();
  const Cache& cache = p.cache;
  if (warp == kIssueWarp) {
    if (lane == 0) {
      sh.dead = 0;
      for (int k = 0; k < kJobs; ++k) {
        ptx::mbar_init(&sh.job_full[k], 1);
        ptx::mbar_init(&sh.job_empty[k], kIssueWarp + 1);           // warps that take it
        for (int i = 0; i < 2; ++i) ptx::mbar_init(&sh.q_ready[i][k], 4);
      }
      for (int k = 0; k < 2; ++k) {
        ptx::mbar_init(&sh.k_full[k], kUnpackWarps);
        ptx::mbar_init(&sh.v_full[k], kUnpackWarps);
        ptx::mbar_init(&sh.k_empty[k], 1);
        ptx::mbar_init(&sh.v_empty[k], 1);
          for (int h = 0; h < 2; ++h) {
          ptx::mbar_init(&sh.s_full[k][h], 1);
          ptx::mbar_init(&sh.p_ready[k][h], 4);
          ptx::mbar_init(&sh.o_done[k][h], 1);
        }
      }
      ptx::mbar_init(&sh.twin_full, 4);
      ptx::mbar_init(&sh.twin_free, 4);
      ptx::mbar_init(&sh.drain, 1);
      ptx::fence_mbar_init();
    }
    __syncwarp();
    ptx::tmem_alloc(&sh.tmem, 512);
    ptx::tmem_relinquish();
  }
  ptx::tc_fence_before_sync();
  ptx::pdl_launch_dependents();
  sum_line(p, kRows, kCost, line, sums);                             // ends with a barrier
  ptx::tc_fence_after_sync();
  const uint32_t tmem = sh.tmem;
  const Partials part = partials_of(p.workspace, gridDim.x, kRows);
  uint32_t jobs = 0;
  // The next piece, for a whole warp; false after the last one.  taken() gives its place in the ring back: a tile without tokens in a
  // piece goes on at once, and may write and announce the queries of later ones, so a place carries its own barriers of queries, and
  // is given back after they have been arrived at and waited for.
  auto take = [&](Job& x) -> bool {
    const uint32_t slot = jobs % kJobs;
    if (!ptx::mbar_wait_warp(&sh.job_full[slot], jobs / kJobs & 1u, dead, status)) return false;
    x = sh.jobs[slot];
    __syncwarp();
    return x.none == 0;
  };
  auto taken = [&]() {
    if (lane == 0) ptx::mbar_arrive(&sh.job_empty[jobs % kJobs]);
    ++jobs;
  };

  if (warp < 8) {
    // ---- softmax: a thread has a row of tile i
    const int i = warp >> 2, row_in = tid & 127;
    const uint32_t quad = static_cast<uint32_t>(warp & 3) << 21;     // this warp's 32 TMEM lanes
    const uint32_t s_at = tmem + quad + i * 128, o_at = tmem + quad + 256 + i * HELD;
    char* const q_smem = smem + Mm::kQ + i * Mm::kBytes + row_in * 128;
    const int t_k = cache_scale_log2(cache, 0), t_v = cache_scale_log2(cache, 1);
    constexpr int kLanes = HELD / 8, kAtOnce = 32 / kLanes;          // a row's 16-byte pieces are copied by so many lanes, so many rows at once
    const int in_row = lane % kLanes, rows0 = (warp & 3) * 32;
    // this lane's 16-byte piece of row r of the warp's: at q_tile + r * 128 + (r % 8 * 16 ^ swizzled)
    char* const q_tile = smem + Mm::kQ + i * Mm::kBytes + (in_row >> 3) * Mm::kBox;
    const int swizzled = (in_row & 7) << 4;
    auto piece_of_row = [&](int k) { return reinterpret_cast<uint4*>(q_smem + (k >> 3) * Mm::kBox + (((k & 7) ^ (row_in & 7)) << 4)); };
    int64_t seen = 0;                                                // chunks of all pieces so far, of both tiles
    uint32_t turn = 0;                                               // .. of this tile
    uint32_t twins = 0;                                              // pieces so far that both tiles had for themselves
    Job x;
    while (take(x)) {
      const int64_t first_seen = seen;
      seen += x.c1 - x.c0;
      const bool twin = is_twin(x.rows);
      const int tile_row = twin ? 0 : i * kTile, rows = min(x.rows - tile_row, kTile), by = twin ? 2 : 1;
      const int row = x.tile * kRows + tile_row + row_in, own = x.length - x.rows_all;
      const bool there = row_in < rows;
      const int tok_of = token_of(p, min(row, x.rows_all * p.group - 1)), head = x.head * p.group + (there ? row - tok_of * p.group : 0);
      const int lim = p.causal ? min(x.length, own + tok_of + 1) : x.length, low = p.window > 0 ? own + tok_of - p.window + 1 : 0;
      const int first_row = x.tile * kRows + tile_row, ta = token_of(p, first_row), tb = token_of(p, first_row + rows - 1);
      const int all_hi = p.causal ? min(x.length, own + ta + 1) : x.length, all_lo = p.window > 0 ? own + tb - p.window + 1 : 0;
      // the row of queries as fp16 into shared memory
      float factor, most_score;                                      // no score of the row is larger
      bool fine;                                                     // the row's query and the scale are finite
      {
        // A warp copies its 32 rows to shared memory as they are, neighbouring lanes a row's neighbouring channels; then each thread
        // goes through its own row there.  Short loops: what is gone through once costs what it takes to fetch the instructions.
        const T* const q_row = static_cast<const T*>(p.q.p) + (x.first + tok_of) * p.q.ld + head * p.q.lh;
        const bool in_head = 8 * in_row < cache.dim;
#pragma unroll 4
        for (int n = 0; n < kLanes; ++n) {
          const int r = rows0 + n * kAtOnce + lane / kLanes;
          const T* const src = of_lane(q_row, r & 31) + (in_head ? 8 * in_row : 0);
          const bool valid = r < rows && in_head;
          char* const dst = q_tile + r * 128 + ((r & 7) << 4 ^ swizzled);
          if (p.wide16_q) {
            asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(ptx::smem_addr(dst)), "l"(src), "r"(valid ? 16 : 0) : "memory");
          } else {
            const uint16_t* u = reinterpret_cast<const uint16_t*>(src);
            uint16_t w[8] = {};
#pragma unroll
            for (int k = 0; k < 8; ++k) if (valid) w[k] = u[k];
            *reinterpret_cast<uint4*>(dst) = make_uint4(w[0] | static_cast<uint32_t>(w[1]) << 16, w[2] | static_cast<uint32_t>(w[3]) << 16,
                                                        w[4] | static_cast<uint32_t>(w[5]) << 16, w[6] | static_cast<uint32_t>(w[7]) << 16);
          }
        }
        asm volatile("cp.async.wait_all;" ::: "memory");
        __syncwarp();
        uint32_t most = 0;
#pragma unroll 4
        for (int k = 0; k < HELD / 8; ++k) {
          const uint4 v = *piece_of_row(k);
          most = __vmaxu2(most, __vmaxu2(__vmaxu2(v.x & 0x7fff7fffu, v.y & 0x7fff7fffu), __vmaxu2(v.z & 0x7fff7fffu, v.w & 0x7fff7fffu)));
        }
        most = max(most & 0xffffu, most >> 16);
        const int e = query_exponent<T>(most);
        const float f = exp2_int(e);
        // a negative scale turns the queries' signs, so that the factor of the scores is not negative
        const uint32_t sign = p.scale < 0.0f ? 0x80008000u : 0u;
        fine = query_fine<T>(most) && p.scale == p.scale;
        if (!std::is_same<T, __half>::value || sign != 0 || !fine) {
#pragma unroll 4
          for (int k = 0; k < HELD / 8; ++k) {
            const uint4 v = *piece_of_row(k);
            *piece_of_row(k) = !fine ? make_uint4(0u, 0u, 0u, 0u)
                                     : make_uint4(query_bits<T>(v.x, f) ^ sign, query_bits<T>(v.y, f) ^ sign, query_bits<T>(v.z, f) ^ sign,
                                                  query_bits<T>(v.w, f) ^ sign);
          }
        }
        // Neither zero nor NaN, so that what is hidden stays at minus infinity.  A row that is not fine has scores of zero, and so a maximum if
        // it sees anything; then it is NaN.
        factor = fine ? fmaxf(ldexpf(fabsf(p.scale) * kLog2e, t_k - e), 1.2e-38f) : 1.2e-38f;
        const float most_q = std::is_same<T, __half>::value ? __half2float(__ushort_as_half(static_cast<unsigned short>(most))) : __uint_as_float(most << 16) * f;
        most_score = fine ? most_q * (2688.0f * cache.dim) * factor : 0.0f;
      }
      // Where scores may lie beyond 2^24, in steps of two and more, the weights come from the rounded product that the reference is one of, and
      // not from the one that a fused operation keeps: it may be half a step larger.
      const float score_factor = factor;
      const bool large = __any_sync(0xffffffffu, most_score >= 16777216.0f);
      if (large) factor = 1.0f;
      // the second tile's last result has been taken in
      if (i == 1 && twins > 0 && !ptx::mbar_wait_warp(&sh.twin_free, (twins - 1) & 1u, dead, status)) break;
      ptx::fence_proxy_async();
      __syncwarp();
      if (lane == 0) ptx::mbar_arrive(&sh.q_ready[i][jobs % kJobs]);
      taken();

      float m = -INFINITY, l = 0.0f, base = 0.0f;
      uint32_t nans = 0;                                             // blocks of the row's result that are NaN
      const int c1 = i == 0 ? x.c1_of[0] : x.c1_of[1];
      // what was noted about the values of chunk ch: a row has the NaN of the tokens that it sees
      auto note_nans = [&](int ch) {
        const int slot = static_cast<int>((first_seen + ch - x.c0) & (kRing - 1));
        const uint4 any = *reinterpret_cast<const uint4*>(sh.nan_any[slot]);
        if ((any.x | any.y | any.z | any.w) == 0) return;
        const int tok = x.key_lo() + ch * kChunk;
        for (int k = 0; k < kUnpackWarps; ++k) {
          if (sh.nan_any[slot][k] == 0) continue;
          for (int t = k * 32; t < k * 32 + 32; ++t)
            if (tok + t < lim && tok + t >= low) nans |= sh.nan_of[slot][t];
        }
      };
      bool ok = true;
      const int from = twin ? x.c0 + i : x.c0;
      int last = -1;                                                 // chunk
      for (int ch = from; ok && ch < c1; last = ch, ch += by, ++turn) {
        const int slot = static_cast<int>((first_seen + ch - x.c0) & (kRing - 1));
#pragma unroll 1
        for (int h = 0; h < 2; ++h) {
          ok = ptx::mbar_wait_warp(&sh.s_full[i][h], turn & 1u, dead, status);
          if (!ok) break;
          ptx::tc_fence_after_sync();
          const uint32_t at_half = s_at + h * kHalf;
          uint32_t va[32], vb[32];
          if (large) {                                               // scores times their factor, in place
#pragma unroll 1
            for (int k = 0; k < kHalf / 16; ++k) {
              uint32_t v[16];
              ld16(at_half + 16 * k, v);
              ld16_wait(v);
#pragma unroll
              for (int e = 0; e < 16; ++e) v[e] = __float_as_uint(__uint_as_float(v[e]) * score_factor);
              st16(at_half + 16 * k, v);
            }
            st_wait();
          }
          ld32(at_half, va);
          ld32(at_half + 32, vb);
          const int tok = x.key_lo() + ch * kChunk + h * kHalf;
          const uint2 hid = *reinterpret_cast<const uint2*>(&sh.hidden[slot][2 * h]);
          const bool edge = tok < all_lo || tok + kHalf > all_hi || (hid.x | hid.y) != 0;
          if (h == 0 && last >= 0) note_nans(last);
          ld32_wait(va);
          ld32_wait(vb);
          if (edge) {
            // 32 tokens' bits: which this row sees.  What it does not see is taken away before it is looked at.
            auto hide = [&](uint32_t (&v)[32], int first, uint32_t hidden) {
              const int a = low - first, z = lim - first;            // from a on, up to z
              const uint32_t up = z >= 32 ? 0xffffffffu : z <= 0 ? 0u : (1u << z) - 1u;
              const uint32_t from = a <= 0 ? 0xffffffffu : a >= 32 ? 0u : ~((1u << a) - 1u);
              const uint32_t see = up & from & ~hidden;
#pragma unroll
              for (int k = 0; k < 32; ++k) if ((see >> k & 1u) == 0) v[k] = 0xff800000u;
            };
            hide(va, tok, hid.x);
            hide(vb, tok + 32, hid.y);
          }
          float top;
          {
            float t0 = -INFINITY, t1 = -INFINITY, t2 = -INFINITY, t3 = -INFINITY;
#pragma unroll
            for (int k = 0; k < 32; k += 4) {
              t0 = max3(t0, __uint_as_float(va[k]), __uint_as_float(va[k + 1]));
              t1 = max3(t1, __uint_as_float(va[k + 2]), __uint_as_float(va[k + 3]));
              t2 = max3(t2, __uint_as_float(vb[k]), __uint_as_float(vb[k + 1]));
              t3 = max3(t3, __uint_as_float(vb[k + 2]), __uint_as_float(vb[k + 3]));
            }
            top = fmaxf(max3(t0, t1, t2), t3);
          }
          const float high = top == -INFINITY ? -INFINITY : top * factor;
          if (__any_sync(0xffffffffu, high - m > kGrowth)) {
            const float now = high > m ? high : m, g = m == -INFINITY || now == m ? 1.0f : exp2_fast(m - now);
            m = now;
            l *= g;
            base = lifted(m);
            if (last >= 0 || h > 0) {
              // once the last product of values is done, that of the other half
              ok = ptx::mbar_wait_warp(&sh.o_done[i][h ^ 1], (turn + h + 1) & 1u, dead, status);
              if (!ok) break;
              ptx::tc_fence_after_sync();
#pragma unroll 1
              for (int k = 0; k < HELD / 16; ++k) {
                uint32_t o[16];
                ld16(o_at + 16 * k, o);
                ld16_wait(o);
#pragma unroll
                for (int e = 0; e < 16; ++e) o[e] = __float_as_uint(__uint_as_float(o[e]) * g);
                st16(o_at + 16 * k, o);
              }
              st_wait();
            }
          }
          uint64_t sum[2] = {0, 0};                                  // pairs of binary32 zeros
          const uint64_t mul = fp4::pack2(factor, factor), sub = fp4::pack2(-base, -base);
          // the sum is that of the weights before they are rounded (of the rounded ones: the prompt 227 us against 208, errors the same)
          auto weigh = [&](const uint32_t (&v)[32], uint32_t to) {
            uint32_t w[16];
#pragma unroll
            for (int k = 0; k < 16; ++k) {
              float a, b;
              fp4::unpack2(fp4::fma2(fp4::pack2(__uint_as_float(v[2 * k]), __uint_as_float(v[2 * k + 1])), mul, sub), a, b);
              a = exp2_fast(a);
              b = exp2_fast(b);
              sum[k & 1] = fp4::add2(sum[k & 1], fp4::pack2(a, b));
              w[k] = half2_bits(__floats2half2_rn(a, b));
            }
            st16(to, w);
          };
          weigh(va, at_half);
          weigh(vb, at_half + 16);
          st_wait();
          ptx::tc_fence_before_sync();
          __syncwarp();
          if (lane == 0) ptx::mbar_arrive(&sh.p_ready[i][h]);
          float a, b;
          fp4::unpack2(fp4::add2(sum[0], sum[1]), a, b);
          l += a + b;
        }
      }
      if (!ok) break;
      if (!fine && m != -INFINITY) l = __int_as_float(0x7fffffff);
      // the row's result
      const bool some = last >= 0;
      if (some) {
        if (!ptx::mbar_wait_warp(&sh.o_done[i][1], (turn - 1) & 1u, dead, status)) break;
        ptx::tc_fence_after_sync();
        note_nans(last);
      }
      // rows that both tiles have: what the first tile's threads have to know of the second's, and the factors of the two results
      float mine = 1.0f, others = 0.0f;
      bool both = false;
      if (twin) {
        if (i == 1) {
          sh.twin_m[row_in] = m;
          sh.twin_l[row_in] = l;
          sh.twin_nans[row_in] = nans;
          ptx::tc_fence_before_sync();
          __syncwarp();
          if (lane == 0) ptx::mbar_arrive(&sh.twin_full);
          ++twins;
          continue;
        }
        if (!ptx::mbar_wait_warp(&sh.twin_full, twins & 1u, dead, status)) break;
        ptx::tc_fence_after_sync();
        ++twins;
        const float om = sh.twin_m[row_in], ol = sh.twin_l[row_in], top = fmaxf(m, om);
        nans |= sh.twin_nans[row_in];
        both = x.c1 - x.c0 > 1;                                      // the second tile had chunks
        mine = m == -INFINITY ? 1.0f : exp2_fast(m - top);
        others = om == -INFINITY ? 1.0f : exp2_fast(om - top);       // (without a maximum there are zeros, or NaN)
        l = l * mine + (both ? ol * others : 0.0f);
        m = top;
      }
      const bool whole = x.starts && x.ends;
      const int slot = x.starts ? 1 : 0;
      const int64_t slot_row = (static_cast<int64_t>(blockIdx.x) * 2 + slot) * kRows + tile_row;
      const float inv = l == 0.0f ? 1.0f : exp2_int(t_v) / l;
      T* const o_row = static_cast<T*>(p.o.p) + (x.first + tok_of) * p.o.ld + head * p.o.lh;
      if (!whole && there) part.stats[slot_row + row_in] = make_float2(m, l);
      // Through the queries' place in shared memory, which no product reads any more: a row's numbers leave side by side.  A part of
      // a unit is binary32 and takes two turns.
      const int columns = whole ? HELD : HELD / 2;
      for (int from_column = 0; from_column < HELD; from_column += columns) {
#pragma unroll 1
        for (int k = 0; k < columns / 32; ++k) {
          uint32_t v[32];
          const int column = from_column + 32 * k;
          if (some) {
            ld32(o_at + column, v);
            ld32_wait(v);
            if (both) {                                              // the same for the whole CTA
              uint32_t w[32];
              ld32(o_at + HELD + column, w);
              ld32_wait(w);
#pragma unroll
              for (int e = 0; e < 32; ++e) v[e] = __float_as_uint(__uint_as_float(v[e]) * mine + __uint_as_float(w[e]) * others);
            }
          } else {
#pragma unroll
            for (int e = 0; e < 32; ++e) v[e] = 0u;
          }
          if (nans != 0) {
#pragma unroll
            for (int e = 0; e < 32; ++e)
              if (nans >> ((column >> 4) + (e >> 4)) & 1u) v[e] = 0x7fffffffu;
          }
          if (whole) {
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              uint32_t h[4];
#pragma unroll
              for (int n = 0; n < 4; ++n) h[n] = two_of<T>(__uint_as_float(v[8 * e + 2 * n]) * inv, __uint_as_float(v[8 * e + 2 * n + 1]) * inv);
              *piece_of_row(4 * k + e) = make_uint4(h[0], h[1], h[2], h[3]);
            }
          } else {
#pragma unroll
            for (int e = 0; e < 8; ++e) *piece_of_row(8 * k + e) = make_uint4(v[4 * e], v[4 * e + 1], v[4 * e + 2], v[4 * e + 3]);
          }
        }
        __syncwarp();
#pragma unroll 4
        for (int n = 0; n < kLanes; ++n) {
          const int r = rows0 + n * kAtOnce + lane / kLanes;
          const uint4 v = *reinterpret_cast<const uint4*>(q_tile + r * 128 + ((r & 7) << 4 ^ swizzled));
          T* const out = of_lane(o_row, r & 31) + 8 * in_row;
          if (r >= rows) continue;
          if (!whole) {
            *reinterpret_cast<uint4*>(part.o + (slot_row + r) * HELD + from_column + 4 * in_row) = v;
          } else if (8 * in_row < cache.dim) {
            if (p.wide16_o) {
              *reinterpret_cast<uint4*>(out) = v;
            } else {
              const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
              for (int e = 0; e < 8; ++e) reinterpret_cast<uint16_t*>(out)[e] = static_cast<uint16_t>(w[e >> 1] >> (e & 1) * 16);
            }
          }
        }
        __syncwarp();
      }
      ptx::tc_fence_before_sync();                                   // the next piece's products write over what was read here
      if (twin) {
        __syncwarp();
        if (lane == 0) ptx::mbar_arrive(&sh.twin_free);
      }
    }
  } else if (warp < kUnpackWarp + kUnpackWarps) {
    // ---- codes to fp16 tiles: a thread has a token, all of its channels
    constexpr int kWords = HELD / 8;                                 // words of codes of a thread's token
    const int t = tid - kUnpackWarp * 32, sub = warp - kUnpackWarp;
    char* const row_at = smem + t * 128;
    const int64_t gap = static_cast<int64_t>(cache.kv_heads) << cache.page_log2;   // rows from a page's keys to its values
    int64_t seen = 0;
    bool paged = true;
    Job x;
    while (take(x)) {
      taken();
      const int key_hi = x.key_hi, steps = x.c1 - x.c0;
      const int tok0 = x.key_lo() + x.c0 * kChunk + t;                 // this thread's token of the first chunk
      const int32_t* const table = p.table + x.request * p.ldt;
      // its page: -1 outside the cache, -2 none
      auto page_of = [&](int it) -> int {
        const int64_t tok = tok0 + static_cast<int64_t>(it) * kChunk;
        if (it >= steps || tok >= key_hi) return -2;
        const int page = table[tok >> cache.page_log2];
        return page < 0 || page >= cache.n_pages ? -1 : page;
      };
      // Turns: keys of chunk 0, of 1, values of 0, keys of 2, values of 1, ..: keys run a chunk ahead, so that the scores of the next
      // tokens never wait behind the values of these.  Every turn is the same short loop; the codes of the next two are on their way.
      struct Turn { int chunk; bool values; };
      struct Codes { uint32_t w[kWords], s[kWords / 8]; int page; };
      auto after = [&](const Turn& a) {
        if (a.values) return a.chunk + 2 < steps ? Turn{a.chunk + 2, false} : Turn{a.chunk + 1, true};
        return a.chunk > 0 ? Turn{a.chunk - 1, true} : steps > 1 ? Turn{1, false} : Turn{0, true};
      };
      // (tokens behind every row's window lie in chunk 0 only; their pages are not looked at)
      int soon = tok0 < x.seen_lo ? -2 : page_of(0), page = -2, before = -2, keys = -1;      // pages of the next keys' chunk, of the last one's, of the one's before; which the last one is
      auto fetch = [&](const Turn& a, Codes& to) {
        to.page = -2;
        if (a.chunk < steps) {
          if (!a.values) {
            before = page;
            page = soon;
            keys = a.chunk;
            soon = page_of(a.chunk + 1);
          }
          to.page = keys == a.chunk ? page : before;
        }
        if (to.page >= 0) {
          const int64_t row = cache_row(cache, to.page, 0, x.head, (tok0 + a.chunk * kChunk) & ((1 << cache.page_log2) - 1)) + (a.values ? gap : 0);
          const uint4* c = reinterpret_cast<const uint4*>(cache.codes + row * (HELD / 2));
#pragma unroll
          for (int k = 0; k < kWords / 4; ++k) {
            const uint4 u = __ldg(c + k);
            to.w[4 * k] = u.x; to.w[4 * k + 1] = u.y; to.w[4 * k + 2] = u.z; to.w[4 * k + 3] = u.w;
          }
          const uint32_t* f = reinterpret_cast<const uint32_t*>(cache.scales + row * (HELD / 16));
#pragma unroll
          for (int k = 0; k < kWords / 8; ++k) to.s[k] = __ldg(f + k);
        } else {                                                     // a token that is not there
#pragma unroll
          for (int k = 0; k < kWords; ++k) to.w[k] = 0;
#pragma unroll
          for (int k = 0; k < kWords / 8; ++k) to.s[k] = 0;
        }
      };
      Turn ta = {0, false}, tb = after(ta), tc = after(tb);
      Codes a, b, c;
      fetch(ta, a);
      fetch(tb, b);
      bool ok = true;
#pragma unroll 1
      for (int turn = 0; turn < 2 * steps; ++turn) {
        fetch(tc, c);
        const int64_t n = seen + ta.chunk;                           // of all
        const int stage = static_cast<int>(n & 1), slot = static_cast<int>(n & (kRing - 1));
        if (!ta.values) {
          const uint32_t out = __ballot_sync(0xffffffffu, a.page == -1);
          paged &= a.page != -1;
          if (lane == 0) sh.hidden[slot][sub] = out;
        } else {
          // blocks of values that are NaN: noted, and zero in the product
          uint32_t bits = 0;
#pragma unroll
          for (int k = 0; k < kWords / 8; ++k) {
            const uint32_t bad = (((a.s[k] & 0x7f7f7f7fu) + 0x01010101u) & 0x80808080u) >> 7;
            a.s[k] &= ~(bad * 0xffu);
            bits |= ((bad & 1u) | (bad >> 7 & 2u) | (bad >> 14 & 4u) | (bad >> 21 & 8u)) << 4 * k;
          }
          const bool any = __any_sync(0xffffffffu, bits != 0);
          if (any) sh.nan_of[slot][t] = static_cast<uint8_t>(bits);
          if (lane == 0) sh.nan_any[slot][sub] = any;
        }
        ok = ptx::mbar_wait_warp(ta.values ? &sh.v_empty[stage] : &sh.k_empty[stage], (static_cast<uint32_t>(n >> 1) & 1u) ^ 1u, dead, status);
        if (!ok) break;
        char* const to = row_at + (ta.values ? Mm::kV : Mm::kK) + stage * Mm::kBytes;
#pragma unroll
        for (int k = 0; k < kWords; k += 4) {
          const __half2 two = scales_of(a.s[k >> 3] >> (k & 4) * 4);             // two blocks, four words
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const __half2 s = e < 2 ? __low2half2(two) : __high2half2(two);
            __half2 v[4];
            values8(a.w[k + e], v);
            const uint4 w = make_uint4(half2_bits(__hmul2(v[0], s)), half2_bits(__hmul2(v[1], s)), half2_bits(__hmul2(v[2], s)), half2_bits(__hmul2(v[3], s)));
            *reinterpret_cast<uint4*>(to + ((k + e) >> 3) * Mm::kBox + ((((k + e) & 7) ^ (t & 7)) << 4)) = w;
          }
        }
        ptx::fence_proxy_async();
        __syncwarp();
        if (lane == 0) ptx::mbar_arrive(ta.values ? &sh.v_full[stage] : &sh.k_full[stage]);
        a = b;
        b = c;
        ta = tb;
        tb = tc;
        tc = after(tc);
      }
      seen += steps;
      if (!ok) break;
    }
    if (__any_sync(0xffffffffu, !paged) && lane == 0) report(status, ADADIM_ERR_PAGES);
  } else if (warp == kIssueWarp) {
    // ---- products
    constexpr uint32_t kScores = idesc_f16(128, kHalf, false), kValues = idesc_f16(128, HELD, true);
    constexpr uint64_t kmajor = ptx::smem_desc_sw128(16, 1024), mnmajor = ptx::smem_desc_sw128(Mm::kBox, 1024);
    const uint32_t base = ptx::smem_addr(smem), tm = static_cast<uint32_t>(same(static_cast<int>(tmem)));
    uint32_t seen = 0;                                               // chunks of all pieces so far
    uint32_t turn[2] = {0, 0};                                       // .. of each tile
    bool ok = true;
    Job x;
    while (ok && take(x)) {
      const int steps = same(x.c1 - x.c0), twin = same(is_twin(x.rows));
      const int n[2] = {same(x.c1_of[0] - x.c0), same(x.c1_of[1] - x.c0)};    // chunks of each tile
      for (int i = 0; i < 2; ++i) ok = ok && ptx::mbar_wait_warp(&sh.q_ready[i][jobs % kJobs], jobs / kJobs & 1u, dead, status);
      taken();
      auto scores = [&](int i, int h, uint32_t stage) {
        const uint32_t d = tm + i * 128 + h * kHalf;
        const uint64_t a = ptx::with_start(kmajor, base + Mm::kQ + i * Mm::kBytes);
        const uint64_t b = ptx::with_start(kmajor, base + Mm::kK + stage * Mm::kBytes + h * (kHalf * 128));
        if (ptx::elect_one()) {
#pragma unroll
          for (int k = 0; k < HELD / 16; ++k) {
            const uint64_t step = ((k >> 2) * Mm::kBox + (k & 3) * 32) >> 4;
            ptx::mma_f16(d, a + step, b + step, kScores, k != 0);
          }
          ptx::mma_commit(&sh.s_full[i][h]);
        }
        __syncwarp();
      };
      auto wait_keys = [&](uint32_t at_chunk) {
        const bool got = ptx::mbar_wait_warp(&sh.k_full[at_chunk & 1u], at_chunk >> 1 & 1u, dead, status);
        ptx::tc_fence_after_sync();
        return got;
      };
      // The scores of the first chunk, both tiles'; of the first two where each tile has its own.
      for (int it = 0; ok && it < min(steps, twin ? 2 : 1); ++it) {
        const uint32_t stage = (seen + it) & 1u;
        ok = wait_keys(seen + it);
        if (!ok) break;
        for (int h = 0; h < 2; ++h)
          for (int i = 0; i < 2; ++i)
            if (twin ? i == it : n[i] > 0) scores(i, h, stage);
        if (ptx::elect_one()) ptx::mma_commit(&sh.k_empty[stage]);
        __syncwarp();
      }
      for (int it = 0; ok && it < steps; ++it, ++seen) {
        const uint32_t stage = seen & 1u;
        const int next = it + (twin ? 2 : 1);                        // the chunk whose scores follow these weights' products
        const uint32_t ahead = (seen + next - it) & 1u;
        ok = ptx::mbar_wait_warp(&sh.v_full[stage], seen >> 1 & 1u, dead, status);
        bool keys = false;
#pragma unroll 1
        for (int hi = 0; hi < 4; ++hi) {                             // halves of the tokens, tiles in turn
          const int h = hi >> 1, i = hi & 1, mine = i == 0 ? n[0] : n[1];
          if (!ok || it >= mine || (twin && i != (it & 1))) continue;
          ok = ptx::mbar_wait_warp(&sh.p_ready[i][h], (i == 0 ? turn[0] : turn[1]) & 1u, dead, status);
          if (!ok) continue;
          if (i == 0) turn[0] += h; else turn[1] += h;
          ptx::tc_fence_after_sync();
          {
            const uint32_t d = tm + 256 + i * HELD, a = tm + i * 128 + h * kHalf;
            const uint64_t b = ptx::with_start(mnmajor, base + Mm::kV + stage * Mm::kBytes + h * (kHalf * 128));
            const bool onto = it > (twin ? i : 0) || h != 0;
            if (ptx::elect_one()) {
#pragma unroll
              for (int k = 0; k < kHalf / 16; ++k) mma_f16_ts(d, a + k * 8, b + ((k * 16 * 128) >> 4), kValues, onto || k != 0);
              ptx::mma_commit(&sh.o_done[i][h]);
            }
            __syncwarp();
          }
          if (next < mine) {
            if (!keys) { ok = wait_keys(seen + next - it); keys = true; }
            if (ok) scores(i, h, ahead);
          }
        }
        if (ok && next < steps && !keys) ok = wait_keys(seen + next - it);       // a chunk that no tile takes any more
        if (ok && ptx::elect_one()) {
          ptx::mma_commit(&sh.v_empty[stage]);
          if (next < steps) ptx::mma_commit(&sh.k_empty[ahead]);
        }
        __syncwarp();
      }
    }
    if (__any_sync(0xffffffffu, *dead != 0)) {
      if (ptx::elect_one()) ptx::mma_commit(&sh.drain);
      __syncwarp();
      const long long t = clock64();
      while (!ptx::mbar_try_wait(&sh.drain, 0) && clock64() - t < ptx::kWaitLimit / 4) {}
    }
  } else if (warp == kJobWarp) {
    // ---- pieces
    const int64_t total = line[p.n_requests];
    const int64_t parts = max(int64_t{1}, min(static_cast<int64_t>(gridDim.x), quick_div(total, kLeastPart)));
    int64_t at = blockIdx.x < parts ? quick_div(total * blockIdx.x, parts) : total;
    const int64_t end = blockIdx.x < parts ? quick_div(total * (blockIdx.x + 1), parts) : total;
    int4 desc = make_int4(0, 0, 0, 0);
    int request = 0;
    for (bool more = true; more;) {
      Job j = {};
      more = at < end;
      j.none = !more;
      if (more) {
        const Piece x = next_piece(p, line, at, end, request, kRows, kCost, kChunk);
        request = x.request;
        if (!(x.starts && x.ends)) note_piece(desc, x);
        j = job_of(p, x);
      }
      const uint32_t slot = jobs % kJobs;
      if (!ptx::mbar_wait_warp(&sh.job_empty[slot], (jobs / kJobs & 1u) ^ 1u, dead, status)) break;
      if (lane == 0) {
        sh.jobs[slot] = j;
        ptx::mbar_arrive(&sh.job_full[slot]);
      }
      __syncwarp();
      ++jobs;
      for (int row = lane; row < j.rows; row += 32) {
        const int of = j.tile * kRows + row, tk = token_of(p, of), hd = j.head * p.group + of - tk * p.group;
        const char* q = reinterpret_cast<const char*>(static_cast<const T*>(p.q.p) + (j.first + tk) * p.q.ld + hd * p.q.lh);
        for (int b = 0; b < cache.dim * 2; b += 128) asm volatile("prefetch.global.L2 [%0];" ::"l"(q + b));
      }
    }
    if (lane == 0) part.desc[blockIdx.x] = desc;
  }
  ptx::tc_fence_before_sync();
  __syncthreads();
  if (*dead && tid == 0) part.desc[blockIdx.x] = make_int4(0, 0, 0, 0);
  if (warp == kIssueWarp) {
    ptx::tc_fence_after_sync();
    ptx::tmem_dealloc(tmem, 512);
  }
}

template <int HELD, typename T>
int many_launch(const Kv4Attention& a, cudaStream_t st) {
  const size_t smem = Many<HELD>::kSmem + sizeof(int64_t) * (static_cast<size_t>(a.n_requests) + 1);
  static std::atomic<uint64_t> done{0};
  const int rc = set_once(kv4_many_kernel<HELD, T>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                          static_cast<int>(Many<HELD>::kSmem + sizeof(int64_t) * (kManyRequests + 1)), done);
  if (rc != ADADIM_OK) return rc;
  return chained_launch(kv4_many_kernel<HELD, T>, dim3(kSms), kThreads, smem, false, st, a, 1);
}

}  // namespace

size_t kv4_many_workspace(int held) { return partials_bytes(kSms, kRows, held); }

int kv4_many_launch(const Kv4Attention& a, int dtype, int& ctas, int& tile_rows, cudaStream_t st) {
  ctas = kSms;
  tile_rows = kRows;
  if (a.cache.held == 64) return dtype == ADADIM_F16 ? many_launch<64, __half>(a, st) : many_launch<64, __nv_bfloat16>(a, st);
  return dtype == ADADIM_F16 ? many_launch<128, __half>(a, st) : many_launch<128, __nv_bfloat16>(a, st);
}

}  // namespace adadim
