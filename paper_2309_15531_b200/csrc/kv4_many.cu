// Attention over the 4-bit key-value cache for many query rows a key head: prompts, pieces of prompts, many drafted tokens.
//
// Bound by arithmetic: 4 dim operations for every pair of a query and a key, on the tensor cores (tcgen05, fp16 operands, binary32
// accumulators in TMEM), and as much by the exponentials between the two products: 128 x 128 pairs are 1024 cycles of either
// unit.  A CTA has 256 query rows in two tiles of 128 (a group of heads of one key head, tokens outer), so that
// one tile's softmax runs while the other one's products do:
//   warps 0-3, 4-7   a tile each: a thread has a row, reads its 128 scores from TMEM twice (largest, then weights) and puts the
//                    weights back as fp16 where the scores were, from where the second product takes them
//   warps 8-11       turn 128 tokens' codes into fp16 tiles in shared memory (128-byte swizzle; keys and values alike: a token
//                    is a row, which is K-major for keys and MN-major for values), two stages of each; the next
//                    tokens' codes are loaded into registers meanwhile, so that 4-bit bytes are all that is read of the cache
//   warp 12          issues the products
// Loops that the warps are in all the time are kept short (32 scores a turn): a warp that runs through a thousand instructions
// waits for them more than it executes.
// The largest score is taken anew only where a row passes it by more than 2^8; then the accumulator in TMEM is rescaled.
// The line of work is cut into one part a CTA as for few rows.
#include "kv4_line.cuh"

namespace adadim {
namespace {

using namespace kv4;
using fp4::exp2_int;

constexpr int kTile = 128, kRows = 2 * kTile, kChunk = 128;
constexpr int kUnpackWarp = 8, kUnpackWarps = 4, kIssueWarp = 12, kThreads = 16 * 32;   // three warps only fill up
constexpr int kCost = 512;                       // what a unit costs beside its tokens, in tokens
constexpr int kLeastPart = 1024;                 // a CTA's part is no smaller
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
__device__ __forceinline__ void st32(uint32_t taddr, const uint32_t (&r)[32]) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x32.b32 [%0], "
      "{%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16, "
      "%17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31, %32};"
      ::"r"(taddr), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]),
        "r"(r[8]), "r"(r[9]), "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15]),
        "r"(r[16]), "r"(r[17]), "r"(r[18]), "r"(r[19]), "r"(r[20]), "r"(r[21]), "r"(r[22]), "r"(r[23]),
        "r"(r[24]), "r"(r[25]), "r"(r[26]), "r"(r[27]), "r"(r[28]), "r"(r[29]), "r"(r[30]), "r"(r[31])
      : "memory");
}
__device__ __forceinline__ void st16(uint32_t taddr, const uint32_t (&r)[16]) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], "
      "{%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, %16};"
      ::"r"(taddr), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]),
        "r"(r[8]), "r"(r[9]), "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15])
      : "memory");
}
__device__ __forceinline__ void st_wait() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }

__device__ __forceinline__ float max3(float a, float b, float c) {
  float r;
  asm("max.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
  return r;
}

struct __align__(16) Shared {
  uint64_t k_full[2], k_empty[2], v_full[2], v_empty[2], q_ready[2], s_full[2], p_ready[2], o_done[2], drain;
  uint32_t tmem;
  int dead;
  uint32_t hidden[kRing][kTile / 32];            // tokens whose page lies outside the cache, a bit each
  uint32_t nan_any[kRing][kUnpackWarps];         // whether a warp's tokens have values that are NaN; which:
  uint8_t nan_of[kRing][kTile];                  // a bit for each of a token's blocks
};

// chunks of a tile of the piece: [c0, this)
__device__ __forceinline__ int chunks_of_tile(const Kv4Attention& p, const Piece& x, int i) {
  if (x.rows <= i * kTile) return x.c0;
  const int hi = key_end(p, x, x.tile * kRows + min(x.rows, (i + 1) * kTile) - 1);
  return max(x.c0, min(x.c1, hi > x.key_lo ? (hi - x.key_lo + kChunk - 1) / kChunk : 0));
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
      for (int k = 0; k < 2; ++k) {
        ptx::mbar_init(&sh.k_full[k], kUnpackWarps);
        ptx::mbar_init(&sh.v_full[k], kUnpackWarps);
        ptx::mbar_init(&sh.k_empty[k], 1);
        ptx::mbar_init(&sh.v_empty[k], 1);
        ptx::mbar_init(&sh.q_ready[k], 4);
        ptx::mbar_init(&sh.s_full[k], 1);
        ptx::mbar_init(&sh.p_ready[k], 4);
        ptx::mbar_init(&sh.o_done[k], 1);
      }
      ptx::mbar_init(&sh.drain, 1);
      ptx::fence_mbar_init();
    }
    __syncwarp();
    ptx::tmem_alloc(&sh.tmem, 512);
    ptx::tmem_relinquish();
  }
  ptx::tc_fence_before_sync();
  sum_line(p, kRows, kCost, line, sums);                             // ends with a barrier
  ptx::tc_fence_after_sync();
  const uint32_t tmem = sh.tmem;
  const Partials part = partials_of(p.workspace, gridDim.x, kRows);
  const int64_t total = line[p.n_requests];
  const int64_t parts = max(int64_t{1}, min(static_cast<int64_t>(gridDim.x), quick_div(total, kLeastPart)));
  int64_t at = blockIdx.x < parts ? quick_div(total * blockIdx.x, parts) : total;
  const int64_t end = blockIdx.x < parts ? quick_div(total * (blockIdx.x + 1), parts) : total;
  int request = 0;

  if (warp < 8) {
    // ---- softmax: a thread has a row of tile i
    const int i = warp >> 2, row_in = tid & 127;
    const uint32_t quad = static_cast<uint32_t>(warp & 3) << 21;     // this warp's 32 TMEM lanes
    const uint32_t s_at = tmem + quad + i * 128, o_at = tmem + quad + 256 + i * HELD;
    char* const q_smem = smem + Mm::kQ + i * Mm::kBytes + row_in * 128;
    const int t_k = cache_scale_log2(cache, 0), t_v = cache_scale_log2(cache, 1);
    int64_t seen = 0;                                                // chunks of all pieces so far, of both tiles
    uint32_t done = 0;                                               // .. of this tile
    while (at < end && !*dead) {
      const Piece x = next_piece(p, line, at, end, request, kRows, kCost, kChunk);
      request = x.request;
      const int64_t first_seen = seen;
      seen += x.c1 - x.c0;
      const int rows = min(x.rows - i * kTile, kTile);
      if (rows <= 0) continue;
      const int row = x.tile * kRows + i * kTile + row_in, own = x.r.length - x.r.rows;
      const bool there = row_in < rows;
      const int tok_of = token_of(p, min(row, x.r.rows * p.group - 1)), head = x.head * p.group + (there ? row - tok_of * p.group : 0);
      const int lim = p.causal ? min(x.r.length, own + tok_of + 1) : x.r.length, low = p.window > 0 ? own + tok_of - p.window + 1 : 0;
      const int first_row = x.tile * kRows + i * kTile, ta = token_of(p, first_row), tb = token_of(p, first_row + rows - 1);
      const int all_hi = p.causal ? min(x.r.length, own + ta + 1) : x.r.length, all_lo = p.window > 0 ? own + tb - p.window + 1 : 0;
      // the row of queries as fp16 into shared memory
      float factor;
      {
        const T* q = static_cast<const T*>(p.q.p) + (x.r.first + tok_of) * p.q.ld + head * p.q.lh;
        uint32_t raw[HELD / 2], most = 0;
#pragma unroll
        for (int k = 0; k < HELD / 8; ++k) {
          uint4 v = make_uint4(0, 0, 0, 0);
          if (there && 8 * k < cache.dim) {
            if (p.wide16_q) {
              v = *reinterpret_cast<const uint4*>(q + 8 * k);
            } else {
              const uint16_t* u = reinterpret_cast<const uint16_t*>(q + 8 * k);
              v.x = u[0] | static_cast<uint32_t>(u[1]) << 16; v.y = u[2] | static_cast<uint32_t>(u[3]) << 16;
              v.z = u[4] | static_cast<uint32_t>(u[5]) << 16; v.w = u[6] | static_cast<uint32_t>(u[7]) << 16;
            }
          }
          raw[4 * k] = v.x; raw[4 * k + 1] = v.y; raw[4 * k + 2] = v.z; raw[4 * k + 3] = v.w;
        }
#pragma unroll
        for (int k = 0; k < HELD / 2; ++k) most = __vmaxu2(most, raw[k] & 0x7fff7fffu);
        most = max(most & 0xffffu, most >> 16);
        const int e = query_exponent<T>(most), e1 = e >> 1;
        const float f1 = exp2_int(e1), f2 = exp2_int(e - e1);
        // a negative scale turns the queries' signs, so that the factor of the scores is not negative
        const uint32_t sign = p.scale < 0.0f ? 0x80008000u : 0u;
#pragma unroll
        for (int k = 0; k < HELD / 8; ++k) {
          const uint4 v = make_uint4(query_bits<T>(raw[4 * k], f1, f2) ^ sign, query_bits<T>(raw[4 * k + 1], f1, f2) ^ sign,
                                     query_bits<T>(raw[4 * k + 2], f1, f2) ^ sign, query_bits<T>(raw[4 * k + 3], f1, f2) ^ sign);
          *reinterpret_cast<uint4*>(q_smem + (k >> 3) * Mm::kBox + (((k & 7) ^ (row_in & 7)) << 4)) = v;
        }
        // (not zero, so that what is hidden stays at minus infinity)
        factor = query_fine<T>(most) && p.scale == p.scale ? fmaxf(ldexpf(fabsf(p.scale) * kLog2e, t_k - e), 1.2e-38f) : __int_as_float(0x7fffffff);
      }
      ptx::fence_proxy_async();
      __syncwarp();
      if (lane == 0) ptx::mbar_arrive(&sh.q_ready[i]);

      float m = -INFINITY, l = 0.0f;
      uint32_t nans = 0;                                             // blocks of the row's result that are NaN
      const int c1 = chunks_of_tile(p, x, i);
      // what was noted about the values of chunk ch: a row has the NaN of the tokens that it sees
      auto note_nans = [&](int ch) {
        const int slot = static_cast<int>((first_seen + ch - x.c0) & (kRing - 1));
        const uint4 any = *reinterpret_cast<const uint4*>(sh.nan_any[slot]);
        if ((any.x | any.y | any.z | any.w) == 0) return;
        const int tok = x.key_lo + ch * kChunk;
        for (int k = 0; k < kUnpackWarps; ++k) {
          if (sh.nan_any[slot][k] == 0) continue;
          for (int t = k * 32; t < k * 32 + 32; ++t)
            if (tok + t < lim && tok + t >= low) nans |= sh.nan_of[slot][t];
        }
      };
      for (int ch = x.c0; ch < c1; ++ch) {
        if (!ptx::mbar_wait_warp(&sh.s_full[i], done & 1u, dead, status)) break;
        ptx::tc_fence_after_sync();
        const int tok = x.key_lo + ch * kChunk, slot = static_cast<int>((first_seen + ch - x.c0) & (kRing - 1));
        const uint4 hid = *reinterpret_cast<const uint4*>(sh.hidden[slot]);
        const bool edge = tok < all_lo || tok + kChunk > all_hi || (hid.x | hid.y | hid.z | hid.w) != 0;
        if (ch > x.c0) note_nans(ch - 1);
        // 32 tokens' bits: which this row sees.  What it does not see is taken away before it is looked at.
        auto hide = [&](uint32_t (&v)[32], int q) {
          const int a = low - (tok + 32 * q), z = lim - (tok + 32 * q);          // from a on, up to z
          const uint32_t up = z >= 32 ? 0xffffffffu : z <= 0 ? 0u : (1u << z) - 1u;
          const uint32_t from = a <= 0 ? 0xffffffffu : a >= 32 ? 0u : ~((1u << a) - 1u);
          const uint32_t see = up & from & ~sh.hidden[slot][q];
#pragma unroll
          for (int k = 0; k < 32; ++k) if ((see >> k & 1u) == 0) v[k] = 0xff800000u;
        };
        uint32_t va[32], vb[32];
        float top = -INFINITY;
#pragma unroll 1
        for (int q = 0; q < 4; q += 2) {
          ld32(s_at + 32 * q, va);
          ld32(s_at + 32 * q + 32, vb);
          ld32_wait(va);
          ld32_wait(vb);
          if (edge) {
            hide(va, q);
            hide(vb, q + 1);
          }
          float t0 = -INFINITY, t1 = -INFINITY, t2 = -INFINITY, t3 = -INFINITY;
#pragma unroll
          for (int k = 0; k < 32; k += 4) {
            t0 = max3(t0, __uint_as_float(va[k]), __uint_as_float(va[k + 1]));
            t1 = max3(t1, __uint_as_float(va[k + 2]), __uint_as_float(va[k + 3]));
            t2 = max3(t2, __uint_as_float(vb[k]), __uint_as_float(vb[k + 1]));
            t3 = max3(t3, __uint_as_float(vb[k + 2]), __uint_as_float(vb[k + 3]));
          }
          top = max3(top, max3(t0, t1, t2), t3);
        }
        const float high = top == -INFINITY ? -INFINITY : top * factor;
        if (__any_sync(0xffffffffu, high > m + 8.0f)) {
          const float now = fmaxf(m, high), f = exp2_fast((m == -INFINITY ? now : m) - (now == -INFINITY ? 0.0f : now));
          if (now > m) {
            l = m == -INFINITY ? l : l * f;
          }
          const float g = now > m && m != -INFINITY ? f : 1.0f;
          m = now;
          if (ch > x.c0) {
            if (!ptx::mbar_wait_warp(&sh.o_done[i], (done - 1) & 1u, dead, status)) break;
            ptx::tc_fence_after_sync();
#pragma unroll 1
            for (int k = 0; k < HELD / 32; ++k) {
              ld32(o_at + 32 * k, vb);
              ld32_wait(vb);
#pragma unroll
              for (int e = 0; e < 32; ++e) vb[e] = __float_as_uint(__uint_as_float(vb[e]) * g);
              st32(o_at + 32 * k, vb);
            }
            st_wait();
          }
        }
        const float base = m == -INFINITY ? 0.0f : m;
        uint64_t sum[2] = {0, 0};                                    // pairs of binary32 zeros
        const uint64_t mul = fp4::pack2(factor, factor), sub = fp4::pack2(-base, -base);
        ld32(s_at, va);
#pragma unroll 1
        for (int q = 0; q < 4; ++q) {
          ld32_wait(va);
          if (edge) hide(va, q);
          uint32_t w[16];
#pragma unroll
          for (int k = 0; k < 16; ++k) {
            float a, b;
            fp4::unpack2(fp4::fma2(fp4::pack2(__uint_as_float(va[2 * k]), __uint_as_float(va[2 * k + 1])), mul, sub), a, b);
            a = exp2_fast(a);
            b = exp2_fast(b);
            sum[k & 1] = fp4::add2(sum[k & 1], fp4::pack2(a, b));
            w[k] = half2_bits(__floats2half2_rn(a, b));
          }
          if (q < 3) ld32(s_at + 32 * q + 32, va);
          st16(s_at + 16 * q, w);
        }
        {
          float a, b;
          fp4::unpack2(fp4::add2(sum[0], sum[1]), a, b);
          l += a + b;
        }
        st_wait();
        ptx::tc_fence_before_sync();
        __syncwarp();
        if (lane == 0) ptx::mbar_arrive(&sh.p_ready[i]);
        ++done;
      }
      // the row's result
      const bool some = c1 > x.c0;
      if (some) {
        if (!ptx::mbar_wait_warp(&sh.o_done[i], (done - 1) & 1u, dead, status)) break;
        ptx::tc_fence_after_sync();
        note_nans(c1 - 1);
      }
      const bool whole = x.starts && x.ends;
      const int slot = x.starts ? 1 : 0;
      const int64_t at_row = (static_cast<int64_t>(blockIdx.x) * 2 + slot) * kRows + i * kTile + row_in;
      const float inv = l == 0.0f ? 1.0f : exp2_int(t_v) / l;
      T* out = static_cast<T*>(p.o.p) + (x.r.first + tok_of) * p.o.ld + head * p.o.lh;
      if (!whole && there) part.stats[at_row] = make_float2(m, l);
#pragma unroll 1
      for (int k = 0; k < HELD / 32; ++k) {
        uint32_t v[32];
        if (some) {
          ld32(o_at + 32 * k, v);
          ld32_wait(v);
        } else {
#pragma unroll
          for (int e = 0; e < 32; ++e) v[e] = 0u;
        }
#pragma unroll
        for (int e = 0; e < 32; ++e) {
          float f = __uint_as_float(v[e]);
          if (nans >> (2 * k + (e >> 4)) & 1u) f = __int_as_float(0x7fffffff);
          if (whole) f *= inv;
          v[e] = __float_as_uint(f);
        }
        if (!there) continue;
        if (!whole) {
          float4* to = reinterpret_cast<float4*>(part.o + at_row * HELD + 32 * k);
#pragma unroll
          for (int e = 0; e < 8; ++e)
            to[e] = make_float4(__uint_as_float(v[4 * e]), __uint_as_float(v[4 * e + 1]), __uint_as_float(v[4 * e + 2]), __uint_as_float(v[4 * e + 3]));
        } else {
          __align__(16) T h[32];
#pragma unroll
          for (int e = 0; e < 32; ++e) h[e] = static_cast<T>(__uint_as_float(v[e]));
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const int d = 32 * k + 8 * e;
            if (d >= cache.dim) continue;
            if (p.wide16_o) {
              *reinterpret_cast<uint4*>(out + d) = reinterpret_cast<uint4*>(h)[e];
            } else {
#pragma unroll
              for (int n = 0; n < 8; ++n) out[d + n] = h[8 * e + n];
            }
          }
        }
      }
      ptx::tc_fence_before_sync();                                   // the next piece's products write over what was read here
    }
  } else if (warp < kUnpackWarp + kUnpackWarps) {
    // ---- codes to fp16 tiles: a thread has half of a token's channels
    constexpr int kWords = HELD / 8;                                 // words of codes of a thread's token
    const int t = tid - kUnpackWarp * 32, sub = warp - kUnpackWarp;
    char* const row_at = smem + t * 128;
    const int64_t gap = static_cast<int64_t>(cache.kv_heads) << cache.page_log2;   // rows from a page's keys to its values
    int64_t seen = 0;
    bool paged = true;
    while (at < end && !*dead) {
      const Piece x = next_piece(p, line, at, end, request, kRows, kCost, kChunk);
      request = x.request;
      const int key_hi = key_end(p, x, x.tile * kRows + x.rows - 1), steps = x.c1 - x.c0;
      const int tok0 = x.key_lo + x.c0 * kChunk + t;                 // this thread's token of the first chunk
      const int32_t* const table = p.table + x.request * p.ldt;
      // its page: -1 outside the cache, -2 none
      auto page_of = [&](int it) -> int {
        const int64_t tok = tok0 + static_cast<int64_t>(it) * kChunk;
        if (it >= steps || tok >= key_hi) return -2;
        const int page = table[tok >> cache.page_log2];
        return page < 0 || page >= cache.n_pages ? -1 : page;
      };
      uint32_t kc[kWords], vc[kWords], ks[kWords / 8], vs[kWords / 8];
      auto load = [&](int64_t row, uint32_t (&codes)[kWords], uint32_t (&scales)[kWords / 8]) {
        const uint4* c = reinterpret_cast<const uint4*>(cache.codes + row * (HELD / 2));
#pragma unroll
        for (int k = 0; k < kWords / 4; ++k) {
          const uint4 a = __ldg(c + k);
          codes[4 * k] = a.x; codes[4 * k + 1] = a.y; codes[4 * k + 2] = a.z; codes[4 * k + 3] = a.w;
        }
        const uint32_t* f = reinterpret_cast<const uint32_t*>(cache.scales + row * (HELD / 16));
#pragma unroll
        for (int k = 0; k < kWords / 8; ++k) scales[k] = __ldg(f + k);
      };
      auto row_of = [&](int page, int it) { return cache_row(cache, page, 0, x.head, (tok0 + it * kChunk) & ((1 << cache.page_log2) - 1)); };
      auto put = [&](const uint32_t (&codes)[kWords], const uint32_t (&scales)[kWords / 8], char* to) {
#pragma unroll
        for (int k = 0; k < kWords; k += 4) {
          const __half2 two = scales_of(scales[k >> 3] >> (k & 4) * 4);          // two blocks, four words
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const __half2 s = e < 2 ? __low2half2(two) : __high2half2(two);
            __half2 v[4];
            values8(codes[k + e], v);
            const uint4 w = make_uint4(half2_bits(__hmul2(v[0], s)), half2_bits(__hmul2(v[1], s)), half2_bits(__hmul2(v[2], s)), half2_bits(__hmul2(v[3], s)));
            *reinterpret_cast<uint4*>(to + ((k + e) >> 3) * Mm::kBox + ((((k + e) & 7) ^ (t & 7)) << 4)) = w;
          }
        }
      };
#pragma unroll
      for (int k = 0; k < kWords; ++k) kc[k] = vc[k] = 0;
#pragma unroll
      for (int k = 0; k < kWords / 8; ++k) ks[k] = vs[k] = 0;
      int page = page_of(0), after = page_of(1);
      if (page >= 0) {
        const int64_t row = row_of(page, 0);
        load(row, kc, ks);
        load(row + gap, vc, vs);
      }
#pragma unroll 1
      for (int it = 0; it < steps; ++it, ++seen) {
        const int stage = static_cast<int>(seen & 1), slot = static_cast<int>(seen & (kRing - 1));
        const uint32_t empty = (static_cast<uint32_t>(seen >> 1) & 1u) ^ 1u;
        const int now = page;
        page = after;
        after = page_of(it + 2);
        const uint32_t out = __ballot_sync(0xffffffffu, now == -1);
        paged &= now != -1;
        if (now < 0) {                                               // a token that is not there: zeros
#pragma unroll
          for (int k = 0; k < kWords / 8; ++k) ks[k] = vs[k] = 0;
        }
        // blocks of values that are NaN: noted, and zero in the product
        uint32_t bits = 0;
#pragma unroll
        for (int k = 0; k < kWords / 8; ++k) {
          const uint32_t bad = (((vs[k] & 0x7f7f7f7fu) + 0x01010101u) & 0x80808080u) >> 7;
          vs[k] &= ~(bad * 0xffu);
          bits |= ((bad & 1u) | (bad >> 7 & 2u) | (bad >> 14 & 4u) | (bad >> 21 & 8u)) << 4 * k;
        }
        const bool any = __any_sync(0xffffffffu, bits != 0);
        if (any) sh.nan_of[slot][t] = static_cast<uint8_t>(bits);
        if (lane == 0) {
          sh.nan_any[slot][sub] = any;
          sh.hidden[slot][sub] = out;
        }
        const int64_t row = page >= 0 ? row_of(page, it + 1) : 0;
        if (!ptx::mbar_wait_warp(&sh.k_empty[stage], empty, dead, status)) break;
        put(kc, ks, row_at + Mm::kK + stage * Mm::kBytes);
        if (page >= 0) load(row, kc, ks);
        ptx::fence_proxy_async();
        __syncwarp();
        if (lane == 0) ptx::mbar_arrive(&sh.k_full[stage]);
        if (!ptx::mbar_wait_warp(&sh.v_empty[stage], empty, dead, status)) break;
        put(vc, vs, row_at + Mm::kV + stage * Mm::kBytes);
        if (page >= 0) load(row + gap, vc, vs);
        ptx::fence_proxy_async();
        __syncwarp();
        if (lane == 0) ptx::mbar_arrive(&sh.v_full[stage]);
      }
    }
    if (__any_sync(0xffffffffu, !paged) && lane == 0) report(status, ADADIM_ERR_PAGES);
  } else if (warp == kIssueWarp) {
    // ---- products
    constexpr uint32_t kScores = idesc_f16(128, kChunk, false), kValues = idesc_f16(128, HELD, true);
    constexpr uint64_t kmajor = ptx::smem_desc_sw128(16, 1024), mnmajor = ptx::smem_desc_sw128(Mm::kBox, 1024);
    const uint32_t base = ptx::smem_addr(smem);
    int64_t seen = 0;
    uint32_t pieces[2] = {0, 0}, done[2] = {0, 0};
    int4 desc = make_int4(0, 0, 0, 0);
    bool ok = true;
    while (ok && at < end && !*dead) {
      const Piece x = next_piece(p, line, at, end, request, kRows, kCost, kChunk);
      request = x.request;
      if (!(x.starts && x.ends)) note_piece(desc, x);
      const int c1[2] = {chunks_of_tile(p, x, 0), chunks_of_tile(p, x, 1)};
      const int64_t first_seen = seen;
      seen += x.c1 - x.c0;
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        if (x.rows <= i * kTile) continue;
        ok = ok && ptx::mbar_wait_warp(&sh.q_ready[i], pieces[i] & 1u, dead, status);
        ++pieces[i];
      }
      auto scores = [&](int i, int stage) {
        if (ptx::elect_one()) {
#pragma unroll
          for (int k = 0; k < HELD / 16; ++k)
            ptx::mma_f16(tmem + i * 128, ptx::with_start(kmajor, base + Mm::kQ + i * Mm::kBytes + (k >> 2) * Mm::kBox + (k & 3) * 32),
                         ptx::with_start(kmajor, base + Mm::kK + stage * Mm::kBytes + (k >> 2) * Mm::kBox + (k & 3) * 32), kScores, k != 0);
          ptx::mma_commit(&sh.s_full[i]);
        }
        __syncwarp();
      };
      auto wait_keys = [&](int ch) {
        const int64_t n = first_seen + ch - x.c0;
        const bool got = ptx::mbar_wait_warp(&sh.k_full[n & 1], static_cast<uint32_t>(n >> 1) & 1u, dead, status);
        ptx::tc_fence_after_sync();
        return got;
      };
      if (ok && x.c0 < x.c1) {
        const int stage = static_cast<int>(first_seen & 1);
        ok = wait_keys(x.c0);
        if (ok) {
          if (x.c0 < c1[0]) scores(0, stage);
          if (x.c0 < c1[1]) scores(1, stage);
          if (ptx::elect_one()) ptx::mma_commit(&sh.k_empty[stage]);
          __syncwarp();
        }
      }
      for (int ch = x.c0; ok && ch < x.c1; ++ch) {
        const int64_t n = first_seen + ch - x.c0;
        const int stage = static_cast<int>(n & 1), ahead = stage ^ 1;
        ok = ptx::mbar_wait_warp(&sh.v_full[stage], static_cast<uint32_t>(n >> 1) & 1u, dead, status);
        bool keys = false;
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          if (!ok || ch >= c1[i]) continue;
          ok = ptx::mbar_wait_warp(&sh.p_ready[i], done[i] & 1u, dead, status);
          if (!ok) continue;
          ++done[i];
          ptx::tc_fence_after_sync();
          if (ptx::elect_one()) {
#pragma unroll
            for (int k = 0; k < kChunk / 16; ++k)
              mma_f16_ts(tmem + 256 + i * HELD, tmem + i * 128 + k * 8, ptx::with_start(mnmajor, base + Mm::kV + stage * Mm::kBytes + k * (16 * 128)), kValues,
                         ch != x.c0 || k != 0);
            ptx::mma_commit(&sh.o_done[i]);
          }
          __syncwarp();
          if (ch + 1 < c1[i]) {
            if (!keys) { ok = wait_keys(ch + 1); keys = true; }
            if (ok) scores(i, ahead);
          }
        }
        if (ok && ptx::elect_one()) {
          ptx::mma_commit(&sh.v_empty[stage]);
          if (ch + 1 < x.c1) ptx::mma_commit(&sh.k_empty[ahead]);
        }
        __syncwarp();
        // a chunk that no tile takes any more has its keys handed back all the same
        if (ok && ch + 1 < x.c1 && !keys) ok = wait_keys(ch + 1);
      }
    }
    if (*dead) {
      desc = make_int4(0, 0, 0, 0);
      if (ptx::elect_one()) ptx::mma_commit(&sh.drain);
      __syncwarp();
      const long long t = clock64();
      while (!ptx::mbar_try_wait(&sh.drain, 0) && clock64() - t < ptx::kWaitLimit / 4) {}
    }
    if (lane == 0) part.desc[blockIdx.x] = desc;
  }
  ptx::tc_fence_before_sync();
  __syncthreads();
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
  kv4_many_kernel<HELD, T><<<kSms, kThreads, smem, st>>>(a);
  ADADIM_CUDA_TRY(cudaGetLastError());
  return kv4_join_launch(a, std::is_same<T, __half>::value ? ADADIM_F16 : ADADIM_BF16, kSms, kRows, false, st);
}

}  // namespace

size_t kv4_many_workspace(int held) { return partials_bytes(kSms, kRows, held); }

int kv4_many_launch(const Kv4Attention& a, int dtype, cudaStream_t st) {
  if (a.cache.held == 64) return dtype == ADADIM_F16 ? many_launch<64, __half>(a, st) : many_launch<64, __nv_bfloat16>(a, st);
  return dtype == ADADIM_F16 ? many_launch<128, __half>(a, st) : many_launch<128, __nv_bfloat16>(a, st);
}

}  // namespace adadim
