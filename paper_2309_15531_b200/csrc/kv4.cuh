// Key-value cache in 4 bits: the layout that include/adadim.h defines, and what its kernels share.  Internal header.
#pragma once

#include <type_traits>

#include "fp4.cuh"
#include "umma_fp4.cuh"

namespace adadim {
namespace kv4 {

constexpr int kMaxRequests = 8192;
constexpr int kMinPage = 16, kMaxPage = 1024;

__host__ __device__ constexpr int held_dim(int head_dim) { return head_dim <= 64 ? 64 : head_dim <= 128 ? 128 : 256; }

struct Cache {
  uint8_t* codes;
  uint8_t* scales;
  const float* amax;       // keys, values; or NULL
  int64_t n_pages;
  int page_log2, kv_heads, dim, held;
};
inline int log2_of(int v) {
  int n = 0;
  while ((1 << n) < v) ++n;
  return n;
}
inline Cache cache_of(const adadim_kv4cache& c) {
  return {c.codes, c.scales, c.amax, c.n_pages, log2_of(c.page), c.kv_heads, c.head_dim, held_dim(c.head_dim)};
}
// Token rows in front of (page, keys or values, head, place): its codes are `held / 2` times that, its scales held / 16 times.
__device__ __forceinline__ int64_t cache_row(const Cache& c, int64_t page, int value, int head, int place) {
  return (((page * 2 + value) * c.kv_heads + head) << c.page_log2) + place;
}
__device__ __forceinline__ int cache_scale_log2(const Cache& c, int value) {
  return fp4::tensor_scale_log2(c.amax == nullptr ? nullptr : c.amax + value);
}

// A request of a batch as every kernel reads it: its query rows and its tokens, clamped to what there is.
struct Request {
  int first, rows, length;
};
__device__ __forceinline__ Request request_of(const int32_t* offsets, const int32_t* lengths, int i, int n_rows, int64_t most, bool& good) {
  const int a = offsets[i], z = offsets[i + 1], n = lengths[i];
  Request r;
  r.first = fp4::clamped(a, n_rows);
  r.rows = max(fp4::clamped(z, n_rows) - r.first, 0);
  r.length = static_cast<int>(n < 0 ? 0 : n > most ? most : n);
  good = a >= 0 && z >= a && z <= n_rows && n >= 0 && n <= most;
  return r;
}

}  // namespace kv4

struct Kv4Heads {
  void* p;
  int64_t ld, lh;
};
struct Kv4Rotary {
  const int32_t* positions;
  const double* freq;
  const uint8_t* axis;
  int64_t ld;
  int axes, dim, adjacent;
};
struct Kv4Attention {
  Kv4Heads q, o;
  int n_rows, q_heads, group;
  uint32_t group_rcp;      // 2^32 / group + 1, 0 for 1
  int wide_q, wide16_q, wide16_o;  // four, eight channels of a query (a result) are one load (store)
  const int32_t *offsets, *lengths, *table;
  int n_requests;
  int64_t ldt, width;
  kv4::Cache cache;
  float scale;
  int causal;
  int window;              // 0: none
  int64_t least_rows, most_rows;   // a kernel takes the requests with so many rows a key head
  int cluster, tiles;      // few rows without the line: CTAs of a unit; tiles of a key head that the grid has
  int* status_dev;
  char* workspace;
};

// chained: may begin while the kernel before it runs.  cluster: CTAs of a cluster
template <typename... P, typename... A>
int chained_launch(void (*kernel)(P...), dim3 grid, int threads, size_t smem, bool chained, cudaStream_t st, const Kv4Attention& a, int cluster, const A&... args) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = grid;
  cfg.blockDim = dim3(static_cast<unsigned>(threads));
  cfg.dynamicSmemBytes = smem;
  cfg.stream = st;
  cudaLaunchAttribute attr[2];
  int n = 0;
  if (chained) {
    attr[n].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[n++].val.programmaticStreamSerializationAllowed = 1;
  }
  if (cluster > 1) {
    attr[n].id = cudaLaunchAttributeClusterDimension;
    attr[n].val.clusterDim.x = static_cast<unsigned>(cluster);
    attr[n].val.clusterDim.y = attr[n].val.clusterDim.z = 1;
    ++n;
  }
  cfg.attrs = attr;
  cfg.numAttrs = static_cast<unsigned>(n);
  return cudaLaunchKernelEx(&cfg, kernel, a, args...) == cudaSuccess ? ADADIM_OK : ADADIM_ERR_CUDA;
}

// implemented in kv4_cache.cu, kv4_attention.cu, kv4_few.cu, kv4_many.cu
int page_tables_launch(const int32_t* past, const int32_t* fresh, int n_requests, int page, int32_t* table, int64_t ldt,
                       int64_t width, const int32_t* free_pages, int n_free, const int32_t* cursor, int rows, int32_t* lengths,
                       int32_t* offsets, int32_t* requests, int32_t* positions, int32_t* slots, int32_t* next, int* status_dev,
                       cudaStream_t st);
int kv4_append_launch(const Kv4Heads& q, const Kv4Heads& qr, int q_heads, const Kv4Heads& k, const Kv4Heads& v, int dtype,
                      int64_t n_tokens, const int32_t* slots, const Kv4Rotary& rotary, const kv4::Cache& cache,
                      const Kv4Heads& k_values, const Kv4Heads& v_values, int vdtype, cudaStream_t st);
int kv4_attention_launch(const Kv4Attention& a, int dtype, int64_t max_new, cudaStream_t st);
// ctas, tile_rows: what the joining kernel has to know.  chained: behind the kernel for many rows
int kv4_few_launch(const Kv4Attention& a, int dtype, int64_t max_new, bool chained, int& ctas, int& tile_rows, cudaStream_t st);
bool kv4_few_suits(const Kv4Attention& a, int64_t max_new);
size_t kv4_few_workspace(int held);
int kv4_many_launch(const Kv4Attention& a, int dtype, int& ctas, int& tile_rows, cudaStream_t st);
size_t kv4_many_workspace(int held);
size_t kv4_workspace(int64_t n_requests, int64_t n_rows, int q_heads, int kv_heads, int head_dim);

}  // namespace adadim
