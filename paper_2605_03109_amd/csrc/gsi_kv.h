// The paged cache of keys and values in 4 bits: what gsi_kv.hip and the attention over it share.
#pragma once
#include "gsi_internal.h"

namespace gsi {

// Elements that share one scale, and the shape of a page: codes [heads, page, dim / 2], scales [heads, dim / 32, page]
constexpr int kKvBlock = 32;
constexpr int kKvMaxDim = 256;
constexpr int kKvMaxPage = 4096;
constexpr int64_t kKvMaxRequests = 16384;  // of one table call: two prefix sums of them lie in LDS

struct KvView {
  uint8_t *K, *Ks, *V, *Vs;
  int64_t n_pages;
  int heads, dim, page_shift;
  __host__ __device__ int page() const { return 1 << page_shift; }
  // first byte of a head's rows in a page, and of a head's scales
  __host__ __device__ int64_t code_at(int64_t page_id, int head) const { return ((page_id * heads + head) << page_shift) * (dim / 2); }
  __host__ __device__ int64_t scale_at(int64_t page_id, int head) const { return ((page_id * heads + head) * (dim / kKvBlock)) << page_shift; }
};

hipError_t kv_tables(const int32_t* kv_len, const int32_t* n_new, int64_t B, const int32_t* free_pages, const int32_t* n_free,
                     int64_t free_cap, int32_t* table, int64_t width, int page_shift, int64_t T, int32_t* kv_len_out,
                     int32_t* q_start, int32_t* slots, int32_t* positions, int32_t* status, hipStream_t s);
hipError_t kv_append(const KvView& c, const void* K, const void* V, int64_t T, int64_t k_stride, int64_t v_stride, int dtype,
                     const int32_t* slots, hipStream_t s);
hipError_t kv_expand(const KvView& c, const int32_t* slots, int64_t T, void* K, void* V, int dtype, hipStream_t s);

struct KvAttend {
  KvView c;
  const void* Q;
  int64_t T, q_stride;
  int heads, dtype;
  const int32_t *q_start, *kv_len;  // q_start NULL: token t is the only one of request t
  int64_t B;
  const int32_t* table;
  int64_t width;
  int64_t max_q, max_len;           // what the caller expects: they choose kernels, tiles and launches, never which keys are seen
  float scale;
  void* O;
  float* lse;                       // NULL: not written
};
size_t kv_attention_workspace(const KvAttend& a);
hipError_t kv_attention(const KvAttend& a, void* ws, hipStream_t s);

}  // namespace gsi
