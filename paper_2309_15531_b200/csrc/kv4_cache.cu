// Block tables and slot maps, and the rotating, quantizing append to the 4-bit key-value cache.
#include "kv4.cuh"

namespace adadim {
namespace {

using namespace fp4;
using kv4::Cache;

// ---- block tables and slot maps --------------------------------------------------------------------
// A few kilobytes: bound by latency. Every CTA forms the sums over all requests for itself (8192 requests: 32 a thread) and
// then looks its new tokens up in them, so that one launch does it all and no CTA waits for another. A new token's page is
// taken from the list of free pages, not from the table another CTA may be writing.  64 requests 3.7 us, 1000 requests with prompts 7.1 us.
constexpr int kTableThreads = 256, kTableRows = 1024;

struct TableParams {
  const int32_t *past, *fresh;
  int n, page_log2;
  int32_t* table;
  int64_t ldt, width;
  const int32_t* free_pages;
  int n_free;
  const int32_t* cursor;
  int rows;
  int32_t *lengths, *offsets, *requests, *positions, *slots, *next;
  int* status_dev;
};

__device__ __forceinline__ bool counts_of(const TableParams& p, int i, int& past, int& fresh) {
  past = p.past[i];
  fresh = p.fresh[i];
  const bool good = past >= 0 && fresh >= 0 && static_cast<int64_t>(past) + fresh <= 0x7fffffff;
  if (!good) past = fresh = 0;
  return good;
}
__device__ __forceinline__ int pages_of(int64_t tokens, int page_log2) {
  return static_cast<int>((tokens + (int64_t{1} << page_log2) - 1) >> page_log2);
}

__global__ void __launch_bounds__(kTableThreads) page_tables_kernel(TableParams p) {
  extern __shared__ int64_t sums[];                                  // new tokens and pages in front of each request
  __shared__ int64_t part[2][kTableThreads / 32];
  int64_t* before = sums;
  int64_t* taken = sums + p.n + 1;
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int each = (p.n + kTableThreads - 1) / kTableThreads;
  const int i0 = min(tid * each, p.n), i1 = min(i0 + each, p.n);
  bool good = true, paged = true;
  int64_t a = 0, b = 0;
  for (int i = i0; i < i1; ++i) {
    int past, fresh;
    good &= counts_of(p, i, past, fresh);
    before[i] = a;
    taken[i] = b;
    a += fresh;
    b += pages_of(static_cast<int64_t>(past) + fresh, p.page_log2) - pages_of(past, p.page_log2);
  }
  int64_t sa = a, sb = b;                                            // sums up to this thread's end
#pragma unroll
  for (int d = 1; d < 32; d <<= 1) {
    const int64_t ua = __shfl_up_sync(0xffffffffu, sa, d), ub = __shfl_up_sync(0xffffffffu, sb, d);
    if (lane >= d) { sa += ua; sb += ub; }
  }
  if (lane == 31) { part[0][warp] = sa; part[1][warp] = sb; }
  __syncthreads();
  int64_t all_a = 0, all_b = 0;
#pragma unroll
  for (int w = 0; w < kTableThreads / 32; ++w) {
    if (w < warp) { sa += part[0][w]; sb += part[1][w]; }
    all_a += part[0][w];
    all_b += part[1][w];
  }
  for (int i = i0; i < i1; ++i) { before[i] += sa - a; taken[i] += sb - b; }
  if (tid == 0) { before[p.n] = all_a; taken[p.n] = all_b; }
  __syncthreads();
  int64_t cursor = p.cursor == nullptr ? 0 : *p.cursor;
  if (cursor < 0) { good = false; cursor = 0; }
  good &= all_a <= p.rows;

  if (blockIdx.x == 0) {
    for (int i = tid; i <= p.n; i += kTableThreads) {
      p.offsets[i] = static_cast<int32_t>(min(before[i], static_cast<int64_t>(p.rows)));
      if (i < p.n) {
        int past, fresh;
        counts_of(p, i, past, fresh);
        p.lengths[i] = past + fresh;
      }
    }
    if (tid == 0) *p.next = static_cast<int32_t>(min(cursor + all_b, static_cast<int64_t>(0x7fffffff)));
  }
  // the new pages of a request: a warp
  for (int i = blockIdx.x * (kTableThreads / 32) + warp; i < p.n; i += gridDim.x * (kTableThreads / 32)) {
    const int need = static_cast<int>(taken[i + 1] - taken[i]);
    if (need == 0) continue;
    int past, fresh;
    counts_of(p, i, past, fresh);
    const int64_t had = pages_of(past, p.page_log2);
    for (int k = lane; k < need; k += 32) {
      const int64_t at = cursor + taken[i] + k;
      const int page = at < p.n_free ? p.free_pages[at] : -1;
      if (had + k < p.width) p.table[i * p.ldt + had + k] = page;
      paged &= had + k < p.width && page >= 0;
    }
  }
  for (int64_t r = int64_t{blockIdx.x} * kTableRows + tid; r < min(static_cast<int64_t>(p.rows), (blockIdx.x + int64_t{1}) * kTableRows); r += kTableThreads) {
    int request = -1, position = 0, slot = -1;
    if (r < all_a) {
      int lo = 0, hi = p.n;                                          // before[lo] <= r < before[hi]
      while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (before[mid] <= r) lo = mid; else hi = mid;
      }
      int past, fresh;
      counts_of(p, lo, past, fresh);
      request = lo;
      position = past + static_cast<int>(r - before[lo]);
      const int64_t q = position >> p.page_log2, had = pages_of(past, p.page_log2);
      int page = -1;
      if (q < p.width) {
        const int64_t at = cursor + taken[lo] + q - had;
        page = q < had ? p.table[lo * p.ldt + q] : at < p.n_free ? p.free_pages[at] : -1;
      }
      const int64_t s = (static_cast<int64_t>(page) << p.page_log2) + (position & ((1 << p.page_log2) - 1));
      if (page >= 0 && s <= 0x7fffffff) slot = static_cast<int>(s);
      paged &= slot >= 0;
    }
    p.requests[r] = request;
    p.positions[r] = position;
    p.slots[r] = slot;
  }
  if (!good) report(p.status_dev, ADADIM_ERR_SHAPE);
  if (!paged) report(p.status_dev, ADADIM_ERR_PAGES);
}

// ---- append ------------------------------------------------------------------------------------------
// Bound by memory in long prompts, by latency for few tokens (then a token's heads are shared by several CTAs). A CTA has one
// token, or four one after the other: their angles are formed once, in binary64 (positions times frequencies lose a far position's
// angle in binary32), by all its threads, and used by all heads. A thread takes eight channels of a key or value (the two halves of a block meet in one shuffle), or
// eight pairs of a query. Keys are rotated in binary64, so that a block's scale and codes are those of the exact rotation:
// binary32 would decide otherwise for values next to the middle of two codes, and the cache would depend on the kernel.  16-bit queries,
// most of a prompt's bytes, are rotated in binary32, by the same kernel and with its registers.
// 8192 tokens of 80 heads of 128 channels: 85 us, 4.0 TB/s, 0.62 of a copy's rate, waiting for loads with 56 % of the issue slots taken; one token 3.8 us.
constexpr int kAppendThreads = 256, kMaxPairs = 128, kMostTokens = 4;

struct AppendParams {
  Kv4Heads q, qr, k, v, k_values, v_values;
  int q_heads;
  const int32_t* slots;
  Kv4Rotary rotary;
  Cache cache;
  int wide_q, wide_qr, wide_k, wide_v, wide_kv, wide_vv;             // 16-byte loads and stores
  int q_chunks;                                                      // tasks of a query head
  uint32_t q_rcp;                                                    // 2^32 / q_chunks + 1
  int chunk_log2;                                                    // of the eights of channels of a held head
  int each;                                                          // tokens of a CTA
  int64_t n_tokens;
};

template <typename T> __device__ __forceinline__ float widened(T x);
template <> __device__ __forceinline__ float widened(float x) { return x; }
template <> __device__ __forceinline__ float widened(__half x) { return __half2float(x); }
template <> __device__ __forceinline__ float widened(__nv_bfloat16 x) { return __bfloat162float(x); }
template <typename T> __device__ __forceinline__ T narrowed(float x);
template <> __device__ __forceinline__ float narrowed(float x) { return x; }
template <> __device__ __forceinline__ __half narrowed(float x) { return __float2half_rn(x); }
template <> __device__ __forceinline__ __nv_bfloat16 narrowed(float x) { return __float2bfloat16_rn(x); }

template <typename T>
__device__ __forceinline__ void load_chunk(const T* p, bool wide, float (&v)[8]) {
  __align__(16) T e[8];
  if (wide) {
#pragma unroll
    for (int k = 0; k < static_cast<int>(sizeof(T)) / 2; ++k) reinterpret_cast<uint4*>(e)[k] = reinterpret_cast<const uint4*>(p)[k];
  } else {
#pragma unroll
    for (int k = 0; k < 8; ++k) e[k] = p[k];
  }
#pragma unroll
  for (int k = 0; k < 8; ++k) v[k] = widened(e[k]);
}
template <typename T>
__device__ __forceinline__ void store_chunk(T* p, bool wide, const float (&v)[8]) {
  __align__(16) T e[8];
#pragma unroll
  for (int k = 0; k < 8; ++k) e[k] = narrowed<T>(v[k]);
  if (wide) {
#pragma unroll
    for (int k = 0; k < static_cast<int>(sizeof(T)) / 2; ++k) reinterpret_cast<uint4*>(p)[k] = reinterpret_cast<uint4*>(e)[k];
  } else {
#pragma unroll
    for (int k = 0; k < 8; ++k) p[k] = e[k];
  }
}

// Pair j of a query: 16-bit ones in binary32 with the rounded sine and cosine (off by 2^-22 of the pair, far below half of their step); binary32
// ones in binary64, rounded once.
template <typename T>
__device__ __forceinline__ void turn_query(float& a, float& b, int j, const float2* turn, const double* turn_c, const double* turn_s) {
  if constexpr (sizeof(T) == 4) {
    const double c = turn_c[j], s = turn_s[j], u = a, w = b;
    a = static_cast<float>(u * c - w * s);
    b = static_cast<float>(w * c + u * s);
  } else {
    const float2 cs = turn[j];
    const float u = a, w = b;
    a = u * cs.x - w * cs.y;
    b = w * cs.x + u * cs.y;
  }
}

// Scale byte and codes of eight channels of a block, from binary64; `m`: bits of the block's largest magnitude.
__device__ __forceinline__ uint32_t quantize_exact(const double (&z)[8], uint64_t m_bits, int t_log2, uint32_t& byte, float& s) {
  s = 0.0f;
  if (m_bits >= 0x7ff0000000000000ull) { byte = 0x7f; return 0; }
  const double unit = __longlong_as_double(static_cast<int64_t>(t_log2 + 1023) << 52);
  const double m = __longlong_as_double(static_cast<int64_t>(m_bits));
  // nearest by binary32, then put right by the two middles, which binary64 holds exactly
  byte = e4m3_of(fminf(static_cast<float>(m * __longlong_as_double(static_cast<int64_t>(1023 - t_log2) << 52)) * (1.0f / 6.0f), 1000.0f));
  const double here = e4m3_value(byte);
  if (byte > 0) {
    const double edge = (here + e4m3_value(byte - 1)) * 3.0 * unit;
    if (m < edge || (m == edge && (byte & 1))) --byte;
  }
  if (byte < 0x7e) {
    const double edge = (static_cast<double>(e4m3_value(byte)) + e4m3_value(byte + 1)) * 3.0 * unit;
    if (m > edge || (m == edge && (byte & 1))) ++byte;
  }
  s = e4m3_value(byte);
  if (byte == 0) return 0;
  const double step = s * unit, rcp = 1.0 / step;
  float y[8];
  bool close = false;
#pragma unroll
  for (int k = 0; k < 8; ++k) {
    y[k] = static_cast<float>(z[k] * rcp);
    // every middle of two levels is a multiple of 1/4; y (up to 7.1, beyond 6 it does not matter) is within 2^-21.9 of the quotient
    const float f = 4.0f * y[k];
    close |= fabsf(f - rintf(f)) < 1.0f / (1 << 18);
  }
  if (!close) return e2m1_pack8(y);
  uint32_t codes = 0;
#pragma unroll 1
  for (int k = 0; k < 8; ++k) {
    const double x = fabs(z[k]);
    uint32_t c = x > 0.25 * step;
    c += x >= 0.75 * step;
    c += x > 1.25 * step;
    c += x >= 1.75 * step;
    c += x > 2.5 * step;
    c += x >= 3.5 * step;
    c += x > 5.0 * step;
    codes |= (c | (z[k] < 0.0 ? 8u : 0u)) << (4 * k);
  }
  return codes;
}

// ODD: a half of the rotated part is an odd number of fours of channels, so that an eight may lie in both halves and
// its partners are loaded one by one.
template <typename T, typename V, bool ODD>
__global__ void __launch_bounds__(kAppendThreads) kv4_append_kernel(AppendParams p) {
  __shared__ double turns_c[kMostTokens][kMaxPairs], turns_s[kMostTokens][kMaxPairs];
  __shared__ float2 turns[kMostTokens][kMaxPairs];
  const int64_t first = blockIdx.x * static_cast<int64_t>(p.each);
  const int tid = threadIdx.x, half = p.rotary.dim >> 1, tokens = static_cast<int>(min(static_cast<int64_t>(p.each), p.n_tokens - first));
  const bool adjacent = p.rotary.adjacent != 0;
  for (int at = tid; at < tokens * kMaxPairs; at += kAppendThreads) {
    const int k = at / kMaxPairs, j = at % kMaxPairs;
    if (j >= half) continue;
    const int ax = p.rotary.axis == nullptr ? 0 : min(static_cast<int>(p.rotary.axis[j]), p.rotary.axes - 1);
    const double angle = static_cast<double>(p.rotary.positions[ax * p.rotary.ld + first + k]) * p.rotary.freq[j];
    // the angle without whole turns, 2 pi as two numbers, so that sincos finds it small
    const double whole = rint(angle * 0.15915494309189535);
    const double rest = fma(-whole, 2.4492935982947064e-16, fma(-whole, 6.283185307179586, angle));
    double s, c;
    sincos(rest, &s, &c);
    turns_c[k][j] = c;
    turns_s[k][j] = s;
    turns[k][j] = make_float2(static_cast<float>(c), static_cast<float>(s));
  }
  __syncthreads();
  const Cache& cache = p.cache;
  const int chunks = 1 << p.chunk_log2, kv_tasks = cache.kv_heads << p.chunk_log2, tasks = 2 * kv_tasks + p.q_heads * p.q_chunks;
  const int lane = tid & 31;
  const uint32_t pair = 3u << (lane & ~1);

  for (int n = 0; n < tokens; ++n) {
  const int64_t t = first + n, slot = p.slots[t];
  const double *const turn_c = turns_c[n], *const turn_s = turns_s[n];
  const float2* const turn = turns[n];
  const bool stored = slot >= 0 && slot >> cache.page_log2 < cache.n_pages;
  for (int task = blockIdx.y * kAppendThreads + tid; task < tasks; task += gridDim.y * kAppendThreads) {
    if (task < 2 * kv_tasks) {
      // kv_tasks and chunks are even, so that the two lanes of a pair have the halves of one block
      const int value = task >= kv_tasks, at = value ? task - kv_tasks : task, head = at >> p.chunk_log2, chunk = at & (chunks - 1), c0 = chunk * 8;
      const Kv4Heads& src = value ? p.v : p.k;
      const bool wide = value ? p.wide_v : p.wide_k, inside = c0 < cache.dim;
      const T* row = static_cast<const T*>(src.p) + t * src.ld + head * src.lh;
      float x[8] = {};
      if (inside) load_chunk(row + c0, wide, x);
      const int t_log2 = kv4::cache_scale_log2(cache, value);
      uint32_t byte, codes;
      float s;
      if (!value && half > 0) {
        double z[8];
        if (inside && c0 < 2 * half) {
          if (adjacent) {
#pragma unroll
            for (int k = 0; k < 8; k += 2) {
              const double c = turn_c[(c0 + k) >> 1], sn = turn_s[(c0 + k) >> 1], a = x[k], b = x[k + 1];
              z[k] = a * c - b * sn;
              z[k + 1] = b * c + a * sn;
            }
          } else if constexpr (ODD) {
#pragma unroll
            for (int k = 0; k < 8; ++k) {
              const bool second = c0 + k >= half;
              const int j = second ? c0 + k - half : c0 + k;
              const double c = turn_c[j], sn = second ? turn_s[j] : -turn_s[j];
              z[k] = static_cast<double>(x[k]) * c + static_cast<double>(widened(row[second ? j : j + half])) * sn;
            }
          } else {
            const bool second = c0 >= half;
            const int j0 = second ? c0 - half : c0;
            float other[8];
            load_chunk(row + (second ? j0 : c0 + half), wide, other);
#pragma unroll
            for (int k = 0; k < 8; ++k) {
              const double c = turn_c[j0 + k], sn = second ? turn_s[j0 + k] : -turn_s[j0 + k];
              z[k] = static_cast<double>(x[k]) * c + static_cast<double>(other[k]) * sn;
            }
          }
        } else {
#pragma unroll
          for (int k = 0; k < 8; ++k) z[k] = x[k];
        }
        uint64_t m = 0;
#pragma unroll
        for (int k = 0; k < 8; ++k) {
          const uint64_t b = static_cast<uint64_t>(__double_as_longlong(z[k])) & 0x7fffffffffffffffull;
          m = b > m ? b : m;                                         // a NaN is above everything
        }
        const uint64_t o = __shfl_xor_sync(pair, m, 1);
        codes = quantize_exact(z, o > m ? o : m, t_log2, byte, s);
      } else {
        uint32_t m = 0;
#pragma unroll
        for (int k = 0; k < 8; ++k) m = max(m, __float_as_uint(x[k]) & 0x7fffffffu);
        m = max(m, __shfl_xor_sync(pair, m, 1));
        const BlockScale b = block_scale<ADADIM_NVFP4, sizeof(T) == 2>(__uint_as_float(m), t_log2);
        codes = codes8<ADADIM_NVFP4, sizeof(T) == 2>(x, b);
        byte = b.byte;
        s = byte == 0x7f ? 0.0f : e4m3_value(byte);
      }
      if (stored) {
        const int64_t r = kv4::cache_row(cache, slot >> cache.page_log2, value, head, static_cast<int>(slot & ((1 << cache.page_log2) - 1)));
        reinterpret_cast<uint32_t*>(cache.codes)[r * chunks + chunk] = codes;
        if ((lane & 1) == 0) cache.scales[r * (chunks >> 1) + (chunk >> 1)] = static_cast<uint8_t>(byte);
      }
      const Kv4Heads& dst = value ? p.v_values : p.k_values;
      if (dst.p != nullptr && inside) {
        float w[8];
        e2m1_values8(codes, w);
        const float f = byte == 0x7f ? __uint_as_float(0x7fffffffu) : s * exp2_int(t_log2);
#pragma unroll
        for (int k = 0; k < 8; ++k) w[k] *= f;
        store_chunk(static_cast<V*>(dst.p) + t * dst.ld + head * dst.lh + c0, value ? p.wide_vv : p.wide_kv, w);
      }
    } else {
      const int at = task - 2 * kv_tasks, head = p.q_chunks == 1 ? at : static_cast<int>(__umulhi(static_cast<uint32_t>(at), p.q_rcp)), chunk = at - head * p.q_chunks;   // at * q_chunks < 2^32
      const T* row = static_cast<const T*>(p.q.p) + t * p.q.ld + head * p.q.lh;
      T* out = static_cast<T*>(p.qr.p) + t * p.qr.ld + head * p.qr.lh;
      float a[8], b[8];
      if (adjacent) {
        const int c0 = chunk * 8;
        load_chunk(row + c0, p.wide_q, a);
        if (c0 < 2 * half) {
#pragma unroll
          for (int k = 0; k < 8; k += 2) turn_query<T>(a[k], a[k + 1], (c0 + k) >> 1, turn, turn_c, turn_s);
        }
        store_chunk(out + c0, p.wide_qr, a);
      } else if (ODD && chunk * 8 < half) {                        // pairs whose second channels lie at odd fours; four of them at the end
        const int j0 = chunk * 8, n = min(8, half - j0);
#pragma unroll
        for (int k = 0; k < 8; ++k) {
          a[k] = k < n ? widened(row[j0 + k]) : 0.0f;
          b[k] = k < n ? widened(row[j0 + half + k]) : 0.0f;
        }
#pragma unroll
        for (int k = 0; k < 8; ++k) {
          if (k >= n) continue;
          turn_query<T>(a[k], b[k], j0 + k, turn, turn_c, turn_s);
          out[j0 + k] = narrowed<T>(a[k]);
          out[j0 + half + k] = narrowed<T>(b[k]);
        }
      } else if (!ODD && chunk * 8 < half) {
        const int j0 = chunk * 8;
        load_chunk(row + j0, p.wide_q, a);
        load_chunk(row + j0 + half, p.wide_q, b);
#pragma unroll
        for (int k = 0; k < 8; ++k) turn_query<T>(a[k], b[k], j0 + k, turn, turn_c, turn_s);
        store_chunk(out + j0, p.wide_qr, a);
        store_chunk(out + j0 + half, p.wide_qr, b);
      } else {
        const int c0 = chunk * 8 + (ODD ? half - 4 : half);          // behind the rotated channels
        load_chunk(row + c0, p.wide_q, a);
        store_chunk(out + c0, p.wide_qr, a);
      }
    }
  }
  }
}

int wide_heads(const Kv4Heads& h, int64_t esz) {
  return reinterpret_cast<uintptr_t>(h.p) % 16 == 0 && (h.ld * esz) % 16 == 0 && (h.lh * esz) % 16 == 0;
}

template <typename T>
int append_types(const AppendParams& p, int vdtype, dim3 grid, cudaStream_t st) {
  const bool odd = !p.rotary.adjacent && p.rotary.dim % 16 != 0;
  if (vdtype == ADADIM_F32 && odd) kv4_append_kernel<T, float, true><<<grid, kAppendThreads, 0, st>>>(p);
  else if (vdtype == ADADIM_F32) kv4_append_kernel<T, float, false><<<grid, kAppendThreads, 0, st>>>(p);
  else if (odd) kv4_append_kernel<T, __nv_bfloat16, true><<<grid, kAppendThreads, 0, st>>>(p);
  else kv4_append_kernel<T, __nv_bfloat16, false><<<grid, kAppendThreads, 0, st>>>(p);
  return cudaGetLastError() == cudaSuccess ? ADADIM_OK : ADADIM_ERR_CUDA;
}

}  // namespace

int page_tables_launch(const int32_t* past, const int32_t* fresh, int n_requests, int page, int32_t* table, int64_t ldt,
                       int64_t width, const int32_t* free_pages, int n_free, const int32_t* cursor, int rows, int32_t* lengths,
                       int32_t* offsets, int32_t* requests, int32_t* positions, int32_t* slots, int32_t* next, int* status_dev,
                       cudaStream_t st) {
  const TableParams p = {past, fresh, n_requests, kv4::log2_of(page), table, ldt, width, free_pages, n_free, cursor, rows,
                         lengths, offsets, requests, positions, slots, next, status_dev};
  const size_t smem = 2 * sizeof(int64_t) * (static_cast<size_t>(n_requests) + 1);
  static std::atomic<uint64_t> done{0};
  const int rc = set_once(page_tables_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize,
                          static_cast<int>(2 * sizeof(int64_t) * (kv4::kMaxRequests + 1)), done);
  if (rc != ADADIM_OK) return rc;
  const int64_t by_rows = (static_cast<int64_t>(rows) + kTableRows - 1) / kTableRows, by_requests = (n_requests + 63) / 64;
  const int64_t grid = by_rows > by_requests ? by_rows : by_requests;
  page_tables_kernel<<<static_cast<unsigned>(grid < 1 ? 1 : grid), kTableThreads, smem, st>>>(p);
  return cudaGetLastError() == cudaSuccess ? ADADIM_OK : ADADIM_ERR_CUDA;
}

int kv4_append_launch(const Kv4Heads& q, const Kv4Heads& qr, int q_heads, const Kv4Heads& k, const Kv4Heads& v, int dtype,
                      int64_t n_tokens, const int32_t* slots, const Kv4Rotary& rotary, const Cache& cache,
                      const Kv4Heads& k_values, const Kv4Heads& v_values, int vdtype, cudaStream_t st) {
  const int64_t esz = dtype == ADADIM_F32 ? 4 : 2, vsz = vdtype == ADADIM_F32 ? 4 : 2;
  AppendParams p = {};
  p.q = q; p.qr = qr; p.k = k; p.v = v; p.k_values = k_values; p.v_values = v_values;
  p.q_heads = q_heads;
  p.slots = slots;
  p.rotary = rotary;
  p.cache = cache;
  p.wide_q = wide_heads(q, esz);
  p.wide_qr = wide_heads(qr, esz);
  p.wide_k = wide_heads(k, esz);
  p.wide_v = wide_heads(v, esz);
  p.wide_kv = wide_heads(k_values, vsz);
  p.wide_vv = wide_heads(v_values, vsz);
  p.q_chunks = rotary.adjacent ? cache.dim / 8 : (rotary.dim + 15) / 16 + (cache.dim - rotary.dim) / 8;
  const int64_t tasks = static_cast<int64_t>(cache.kv_heads) * (cache.held / 8) * 2 + static_cast<int64_t>(q_heads) * p.q_chunks;
  p.q_rcp = static_cast<uint32_t>((uint64_t{1} << 32) / p.q_chunks + 1);
  p.chunk_log2 = kv4::log2_of(cache.held / 8);
  p.n_tokens = n_tokens;
  // Four tokens a CTA from three waves of such CTAs on; fewer leave SMs idle in the last one.  Four against one, in us, 64 + 8 + 8 heads of 128
  // (12 + 3 + 3 of 80): 3000 tokens 46 and 37 (19.4 and 15.7), 4096 47.8 and 43 (19.9 and 19.1), 7104 79 and 78 (29.3 and 30.1), 8192 85 and
  // 89 (29.5 and 33.8), 12000 128 and 126 (41 and 45), 16384 164 and 170.
  p.each = n_tokens >= 3 * 148 * 4 * kMostTokens ? kMostTokens : 1;
  const int64_t most = (tasks + kAppendThreads - 1) / kAppendThreads, wanted = 148 * 4 / n_tokens;
  const dim3 grid(static_cast<unsigned>((n_tokens + p.each - 1) / p.each), static_cast<unsigned>(wanted < 1 ? 1 : wanted > most ? most : wanted));
  if (dtype == ADADIM_F32) return append_types<float>(p, vdtype, grid, st);
  return dtype == ADADIM_F16 ? append_types<__half>(p, vdtype, grid, st) : append_types<__nv_bfloat16>(p, vdtype, grid, st);
}

}  // namespace adadim
