// The paged cache of keys and values in 4 bits: its tables, its rows written and read back.
//
// E2M1: sign, then 0 .5 1 1.5 2 3 4 6.  Of 32 elements along a head the scale is the smallest 2^e (byte e + 127, in
// 2 .. 254) with max|x| / 2^e <= 6, so that nothing saturates and every value is a normal number or zero (but those of elements from 3.5 * 2^126 on,
// which round to 2^128: infinite); an element's code is the nearest to x / 2^e, ties to the even code (the division is exact).  A block with an element that is not
// finite gets the byte 255: every value of it reads as NaN.  The conversions are the card's own (the formats of its
// matrix instructions); they round as written here for every scale.
#include <algorithm>

#include "gsi_device.h"
#include "gsi_kv.h"

namespace gsi {
namespace {

constexpr int kScanThreads = 512;

// Sums that stop at `most` (both below 2^30): associative, so a scan of them is exact however it is cut.
__device__ __forceinline__ int add_to(int a, int b, int most) { return min(a + b, most); }

// Exclusive scan over the workgroup of one value per thread on top of `carry`, which becomes the total.
__device__ __forceinline__ int block_scan(int v, int most, int& carry, int* wave_sums) {
  const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave;
  int incl = v;
#pragma unroll
  for (int o = 1; o < kWave; o <<= 1) {
    const int up = __shfl_up(incl, o, kWave);
    if (lane >= o) incl = add_to(incl, up, most);
  }
  __syncthreads();  // the sums of the round before are read
  if (lane == kWave - 1) wave_sums[wave] = incl;
  __syncthreads();
  int before = carry, total = carry;
#pragma unroll
  for (int w = 0; w < kScanThreads / kWave; ++w) {
    if (w == wave) before = total;
    total = add_to(total, wave_sums[w], most);
  }
  carry = total;
  const int excl = __shfl_up(incl, 1, kWave);
  return lane == 0 ? before : add_to(before, excl, most);
}

// the last i with start[i] <= x, start[0] = 0 <= x < start[n]
__device__ __forceinline__ int owner(const int* start, int n, int x) {
  int lo = 0, hi = n;
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (start[mid] <= x) lo = mid;
    else hi = mid;
  }
  return lo;
}

// Every workgroup scans the lengths of all requests (they are few bytes, and a second launch would cost more than the
// scan) and then takes its share of the tokens, the new pages and the requests.  Latency bounds it: lengths, scans in LDS, a search, one
// read of the table or the free list.  32 requests 4.5 us, 300 requests of 27000 new tokens 6.0 us.
__global__ __launch_bounds__(kScanThreads) void tables_kernel(const int32_t* __restrict__ kv_len, const int32_t* __restrict__ n_new, int B,
                                                              const int32_t* __restrict__ free_pages,
                                                              const int32_t* __restrict__ n_free, int free_cap,
                                                              int32_t* table, int64_t width, int page_shift, int T,
                                                              int32_t* __restrict__ kv_len_out, int32_t* __restrict__ q_start,
                                                              int32_t* __restrict__ slots, int32_t* __restrict__ positions,
                                                              int32_t* __restrict__ status) {
  extern __shared__ int lds[];
  __shared__ int wave_sums[kScanThreads / kWave];
  constexpr int kMost = 1 << 30;
  int* const tok = lds;            // [B + 1] first new token of a request
  int* const first = lds + B + 1;  // [B + 1] first new page of a request, in the order of the free list
  const int page = 1 << page_shift;
  const auto len_of = [&](int b) { return min(max(kv_len[b], 0), kMost); };
  const auto pages = [&](int len) { return (len + page - 1) >> page_shift; };  // len <= 2^31 - 4096
  const auto held = [&](int n) { return (int)min((int64_t)n, width); };
  const auto names_page = [&](int entry) { return entry >= 0 && entry <= (0x7fffffff >> page_shift); };  // one whose slots are numbers
  int carry = 0;
  for (int b0 = 0; b0 < B; b0 += kScanThreads) {
    const int b = b0 + threadIdx.x;
    const int at = block_scan(b < B ? min(max(n_new[b], 0), T) : 0, T, carry, wave_sums);
    if (b < B) tok[b] = at;
  }
  if (threadIdx.x == 0) tok[B] = carry;
  __syncthreads();
  int carry_pages = 0, carry_all = 0;
  for (int b0 = 0; b0 < B; b0 += kScanThreads) {
    const int b = b0 + threadIdx.x;
    int in_table = 0, all = 0;
    if (b < B) {
      const int len = len_of(b), have = pages(len), need = pages(len + (tok[b + 1] - tok[b]));
      all = need - have;
      in_table = held(need) - held(have);
      // new tokens on a page that was begun before: it may be one that was not there then (the entries of this call lie behind it)
      if (blockIdx.x == 0 && tok[b + 1] > tok[b] && (len & (page - 1)) && !(have <= width && names_page(table[b * width + have - 1]))) ++all;
    }
    const int at = block_scan(in_table, kMost, carry_pages, wave_sums);
    block_scan(all, kMost, carry_all, wave_sums);
    if (b < B) first[b] = at;
  }
  if (threadIdx.x == 0) first[B] = carry_pages;
  __syncthreads();
  const int tokens = tok[B], wanted = first[B];
  const int avail = min(max(n_free[0], 0), free_cap);
  const int me = blockIdx.x * kScanThreads + threadIdx.x, all_threads = gridDim.x * kScanThreads;
  const auto fresh = [&](int i) { return i < avail ? free_pages[i] : -1; };
  if (me == 0) {
    status[0] = min(wanted, avail);
    status[1] = carry_all - min(wanted, avail);
  }
  for (int b = me; b <= B; b += all_threads) {
    q_start[b] = tok[b];
    if (b < B) kv_len_out[b] = len_of(b) + (tok[b + 1] - tok[b]);
  }
  for (int i = me; i < wanted; i += all_threads) {
    const int b = owner(first, B, i);
    table[b * width + held(pages(len_of(b))) + (i - first[b])] = fresh(i);
  }
  for (int t = me; t < T; t += all_threads) {
    int slot = -1, pos = -1;
    if (t < tokens) {
      const int b = owner(tok, B, t), len = len_of(b), have = pages(len);
      pos = len + (t - tok[b]);
      const int j = pos >> page_shift;
      // entries of this call are not read back: another workgroup may not have written them yet
      const int entry = j >= width ? -1 : (j < have ? table[b * width + j] : fresh(first[b] + j - have));
      if (names_page(entry)) slot = (entry << page_shift) + (pos & (page - 1));
    }
    slots[t] = slot;
    positions[t] = pos;
  }
}

// ---- rows ------------------------------------------------------------------------------------------------
// A workgroup takes 16 tokens by 128 elements, 8 elements a thread: four threads hold the block of a scale, and the scale bytes of
// consecutive tokens, which lie side by side, come from one workgroup.  Memory bounds both directions: 8192 tokens x 32 heads x 128 in bf16, 170 MB,
// are written in 34 us (5.0 TB/s, a copy's rate) and read back in 26 us (6.5 TB/s); 8 tokens x 12 x 64 take 2.9 us each.
constexpr int kRowTokens = 16, kRowThreads = 256, kRowElems = 128;

struct RowPlace {
  int64_t t;
  int e, head, d;  // element of the token's row; its head and place there
  int64_t page;
  int off;
  bool ok;
};
__device__ __forceinline__ RowPlace place_of(const KvView& c, const int32_t* slots, int64_t T) {
  RowPlace r;
  const int cols = (c.heads * c.dim + kRowElems - 1) / kRowElems;
  r.t = (int64_t)(blockIdx.x / cols) * kRowTokens + threadIdx.x / 16;
  r.e = (int)(blockIdx.x % cols) * kRowElems + threadIdx.x % 16 * 8;
  r.ok = r.t < T && r.e < c.heads * c.dim;
  const int slot = r.ok ? slots[r.t] : -1;
  r.head = r.e / c.dim;
  r.d = r.e - r.head * c.dim;
  r.page = slot >> c.page_shift;
  r.off = slot & (c.page() - 1);
  if (slot < 0 || r.page >= c.n_pages) r.page = -1;
  return r;
}

// four code bytes and the scale byte of the block that four neighbouring threads hold
__device__ __forceinline__ void quantise8(const float (&x)[8], uint32_t& codes, int& scale) {
  float most = 0.f;
#pragma unroll
  for (int i = 0; i < 8; ++i) most = fmaxf(most, fabsf(x[i]));
  // NaN anywhere: 0 * x is NaN for infinities and NaN alike, and a sum keeps it
  float odd = 0.f;
#pragma unroll
  for (int i = 0; i < 8; ++i) odd = fmaf(0.f, x[i], odd);
  most = fmaxf(most, dpp_move<0xB1>(most));
  most = fmaxf(most, dpp_move<0x4E>(most));
  odd += dpp_move<0xB1>(odd);
  odd += dpp_move<0x4E>(odd);
  const int e = ((int)((__float_as_uint(most) + 0x3fffffu) >> 23)) - 2;  // one more where the significand is above 1.5
  const bool fine = odd == 0.f;
  scale = fine ? min(max(e, 2), 254) : 255;
  codes = 0;
  if (fine) {
    const float s = __uint_as_float((uint32_t)scale << 23);
    codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(codes, x[0], x[1], s, 0);
    codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(codes, x[2], x[3], s, 1);
    codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(codes, x[4], x[5], s, 2);
    codes = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(codes, x[6], x[7], s, 3);
  }
}

// Rows are read once: past the caches, 8192 tokens x 32 heads x 128 are written and read back in 60 us, through them in 66.
template <class X>
__device__ __forceinline__ void load8(const typename X::storage* p, bool wide, float (&x)[8]) {
  if (wide) {
#pragma unroll
    for (int i = 0; i < 8; i += X::kVec) {
      typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
      const u32x4 w = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(p + i));
      X::widen(make_uint4(w[0], w[1], w[2], w[3]), reinterpret_cast<float(&)[X::kVec]>(x[i]));
    }
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = X::load(p, i);
  }
}

template <class X>
__global__ __launch_bounds__(kRowThreads) void append_kernel(KvView c, const typename X::storage* __restrict__ K,
                                                             const typename X::storage* __restrict__ V, int64_t T, int64_t k_stride,
                                                             int64_t v_stride, bool wide, const int32_t* __restrict__ slots) {
  const RowPlace r = place_of(c, slots, T);
  if (!r.ok || r.page < 0) return;  // groups of four threads leave together
  float k[8], v[8];
  load8<X>(K + r.t * k_stride + r.e, wide, k);
  load8<X>(V + r.t * v_stride + r.e, wide, v);
  uint32_t kc, vc;
  int ks, vs;
  quantise8(k, kc, ks);
  quantise8(v, vc, vs);
  const int64_t code = c.code_at(r.page, r.head) + (int64_t)r.off * (c.dim / 2) + r.d / 2;
  *reinterpret_cast<uint32_t*>(c.K + code) = kc;
  *reinterpret_cast<uint32_t*>(c.V + code) = vc;
  if (r.d % kKvBlock == 0) {
    const int64_t scale = c.scale_at(r.page, r.head) + ((int64_t)(r.d / kKvBlock) << c.page_shift) + r.off;
    c.Ks[scale] = (uint8_t)ks;
    c.Vs[scale] = (uint8_t)vs;
  }
}

template <class X>
__device__ __forceinline__ void expand8(uint32_t codes, int scale, typename X::storage* out) {
  const float s = __uint_as_float((uint32_t)scale << 23);
  typedef float f32x2 __attribute__((ext_vector_type(2)));
  f32x2 v[4];
  v[0] = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes, s, 0);
  v[1] = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes, s, 1);
  v[2] = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes, s, 2);
  v[3] = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes, s, 3);
  if constexpr (sizeof(*out) == 4) {
    reinterpret_cast<float4*>(out)[0] = make_float4(v[0][0], v[0][1], v[1][0], v[1][1]);
    reinterpret_cast<float4*>(out)[1] = make_float4(v[2][0], v[2][1], v[3][0], v[3][1]);
  } else {  // two significand bits: exact in bf16
    uint32_t w[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) w[i] = (__float_as_uint(v[i][0]) >> 16) | (__float_as_uint(v[i][1]) & 0xffff0000u);
    *reinterpret_cast<uint4*>(out) = make_uint4(w[0], w[1], w[2], w[3]);
  }
}

template <class X>
__global__ __launch_bounds__(kRowThreads) void expand_kernel(KvView c, const int32_t* __restrict__ slots, int64_t T,
                                                             typename X::storage* __restrict__ K, typename X::storage* __restrict__ V) {
  const RowPlace r = place_of(c, slots, T);
  if (!r.ok) return;
  uint32_t kc = 0, vc = 0;
  int ks = 127, vs = 127;
  if (r.page >= 0) {
    const int64_t code = c.code_at(r.page, r.head) + (int64_t)r.off * (c.dim / 2) + r.d / 2;
    const int64_t scale = c.scale_at(r.page, r.head) + ((int64_t)(r.d / kKvBlock) << c.page_shift) + r.off;
    kc = *reinterpret_cast<const uint32_t*>(c.K + code);
    vc = *reinterpret_cast<const uint32_t*>(c.V + code);
    ks = c.Ks[scale];
    vs = c.Vs[scale];
  }
  const int64_t at = r.t * c.heads * c.dim + r.e;
  expand8<X>(kc, ks, K + at);
  expand8<X>(vc, vs, V + at);
}

unsigned row_blocks(const KvView& c, int64_t T) {
  return (unsigned)(ceil_div(T, kRowTokens) * ceil_div((int64_t)c.heads * c.dim, kRowElems));
}

}  // namespace

hipError_t kv_tables(const int32_t* kv_len, const int32_t* n_new, int64_t B, const int32_t* free_pages, const int32_t* n_free,
                     int64_t free_cap, int32_t* table, int64_t width, int page_shift, int64_t T, int32_t* kv_len_out,
                     int32_t* q_start, int32_t* slots, int32_t* positions, int32_t* status, hipStream_t s) {
  const size_t lds = 2 * (size_t)(B + 1) * sizeof(int);
  static LdsLimit limit;
  if (lds > 60 * 1024)
    if (hipError_t e = limit.allow((const void*)tables_kernel, 2 * (kKvMaxRequests + 1) * sizeof(int)); e != hipSuccess) return e;
  const unsigned blocks = (unsigned)std::min<int64_t>(ceil_div(std::max(T, B), kScanThreads), 256);
  tables_kernel<<<std::max(blocks, 1u), kScanThreads, lds, s>>>(kv_len, n_new, (int)B, free_pages, n_free, (int)free_cap, table, width,
                                                               page_shift, (int)T, kv_len_out, q_start, slots, positions, status);
  return hipGetLastError();
}

hipError_t kv_append(const KvView& c, const void* K, const void* V, int64_t T, int64_t k_stride, int64_t v_stride, int dtype,
                     const int32_t* slots, hipStream_t s) {
  const size_t es = elem_size(dtype);
  const auto whole = [&](const void* p, int64_t stride) { return reinterpret_cast<uintptr_t>(p) % 16 == 0 && (size_t)stride * es % 16 == 0; };
  const bool wide = whole(K, k_stride) && whole(V, v_stride);
  if (dtype == GSI_BF16)
    append_kernel<BF16><<<row_blocks(c, T), kRowThreads, 0, s>>>(c, reinterpret_cast<const uint16_t*>(K), reinterpret_cast<const uint16_t*>(V), T,
                                                                 k_stride, v_stride, wide, slots);
  else
    append_kernel<F32><<<row_blocks(c, T), kRowThreads, 0, s>>>(c, reinterpret_cast<const float*>(K), reinterpret_cast<const float*>(V), T,
                                                                k_stride, v_stride, wide, slots);
  return hipGetLastError();
}

hipError_t kv_expand(const KvView& c, const int32_t* slots, int64_t T, void* K, void* V, int dtype, hipStream_t s) {
  if (dtype == GSI_BF16)
    expand_kernel<BF16><<<row_blocks(c, T), kRowThreads, 0, s>>>(c, slots, T, reinterpret_cast<uint16_t*>(K), reinterpret_cast<uint16_t*>(V));
  else
    expand_kernel<F32><<<row_blocks(c, T), kRowThreads, 0, s>>>(c, slots, T, reinterpret_cast<float*>(K), reinterpret_cast<float*>(V));
  return hipGetLastError();
}

}  // namespace gsi
