// Device code that the attention kernels over the 4-bit cache share (gsi_attend.hip, gsi_prompt.hip).
#pragma once
#include "gsi_device.h"
#include "gsi_kv.h"

namespace gsi {

// Launches of the two kernels, each for its own requests: those of at most `few` rows of a head of keys (tokens times the heads
// that share it) and those of more.
hipError_t attend_few(const KvAttend& a, int64_t few, void* ws, hipStream_t s);
size_t attend_few_workspace(const KvAttend& a, int64_t few);
hipError_t attend_prompt(const KvAttend& a, int64_t few, bool zero, void* ws, hipStream_t s);  // zero: it clears the rows of no request
size_t attend_prompt_workspace(const KvAttend& a);

namespace {

typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef __attribute__((__vector_size__(8 * sizeof(__bf16)))) __bf16 bf16x8;

constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;
// The running maximum of a row moves only when a score passes it by more than 2^kSlack in the exponential: weights stay below
// 2^kSlack, which costs fp32 sums and bf16 weights nothing, and almost no step rescales what is summed so far.
constexpr float kSlack = 8.f;

// A score's factor in the exponential, above 0: the largest score is then the largest product, whose factor enters one fused operation with the
// maximum's subtraction.  A negative scale turns the queries' sign; one of 0 becomes the smallest number, 2^-149, which takes the largest products to
// 2^-21 at most.
__device__ __forceinline__ float exponent_scale(float scale) { return fmaxf(fabsf(scale) * kLog2e, 1.40129846e-45f); }

struct Span {  // a request's tokens of the call and its keys
  int t0, n;
  int len;   // keys that its row of the table has places for
  int past;  // keys in front of its first token of the call, whether there are places for them or not (below 0: so many tokens see none)
  // the last key that token i sees
  __device__ __forceinline__ int last_key(int i) const { return min(past + i, len - 1); }
};
__device__ __forceinline__ int places(const KvAttend& a, const Span& s) { return (int)min((int64_t)s.past + s.n, a.width << a.c.page_shift); }
__device__ __forceinline__ Span span_of(const KvAttend& a, int b) {
  Span s;
  const int T = (int)a.T;
  s.t0 = a.q_start ? min(max(a.q_start[b], 0), T) : min(b, T);
  const int t1 = a.q_start ? min(max(a.q_start[b + 1], s.t0), T) : min(b + 1, T);
  s.n = t1 - s.t0;
  s.past = max(a.kv_len[b], 0) - s.n;
  s.len = places(a, s);
  return s;
}

// Codes as pairs of bf16, exact: pair SEL of a word, and its four.
__device__ __forceinline__ float scale_value(int byte) { return __uint_as_float((uint32_t)byte << 23); }
template <int SEL>
__device__ __forceinline__ uint32_t two_values(uint32_t w, float scale) {
  return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, SEL));
}
__device__ __forceinline__ u32x4 eight_values(uint32_t w, float scale) {
  return u32x4{two_values<0>(w, scale), two_values<1>(w, scale), two_values<2>(w, scale), two_values<3>(w, scale)};
}

__device__ __forceinline__ int64_t divide(int64_t a, int64_t b) {  // both at least 0; the quotient of 64 bits takes a hundred instructions
  return ((a | b) >> 32) == 0 ? (int64_t)((uint32_t)a / (uint32_t)b) : a / b;
}

// Quotients of numbers from 0 to below 2^31 by a divisor that the host knows.  m = floor(2^(31 + s) / d) + 1 with 2^s >= d is off by less than 2^s / d from
// 2^(31 + s) / d, and the quotient by less than 1 / d.
struct Divisor {
  uint32_t m;
  int shift;
  Divisor() : Divisor(1) {}
  explicit Divisor(uint32_t d) : shift(31) {
    while ((1ull << (shift - 31)) < d) ++shift;
    m = (uint32_t)((1ull << shift) / d + 1);
  }
  __device__ __forceinline__ int operator()(int x) const { return (int)(((uint64_t)(uint32_t)x * m) >> shift); }
};

// Work in units, by request: `units` says how many a span has.  The spans of 256 requests at a time and prefix sums of their units lie in LDS; all
// threads of a workgroup of 256 call these functions together.
constexpr int kScan = 256;
struct Prefix {
  int64_t incl[kScan];
  int64_t sums[kScan / kWave];
  int t0[kScan], n[kScan], past[kScan];
};
template <class U>
__device__ __forceinline__ int64_t scan_requests(const KvAttend& a, int64_t b0, Prefix& x, U units) {
  const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave;
  const int64_t b = b0 + threadIdx.x;
  int64_t v = 0;
  Span sp{0, 0, 0, 0};
  if (b < a.B) {
    sp = span_of(a, (int)b);
    v = units(sp);
  }
#pragma unroll
  for (int o = 1; o < kWave; o <<= 1) {
    if (o >= a.B) break;  // (what a lane behind the last request has then is not used)
    const int64_t up = __shfl_up(v, o, kWave);
    if (lane >= o) v += up;
  }
  __syncthreads();
  if (lane == max((int)min(a.B - b0 - wave * kWave, (int64_t)kWave), 1) - 1) x.sums[wave] = v;
  __syncthreads();
  int64_t total = 0;
#pragma unroll
  for (int w = 0; w < kScan / kWave; ++w) {
    if (w < wave) v += x.sums[w];
    total += x.sums[w];
  }
  x.incl[threadIdx.x] = v;
  x.t0[threadIdx.x] = sp.t0;
  x.n[threadIdx.x] = sp.n;
  x.past[threadIdx.x] = sp.past;
  __syncthreads();
  return total;
}
template <class U>
__device__ __forceinline__ int64_t total_units(const KvAttend& a, Prefix& x, U units) {
  int64_t total = scan_requests(a, 0, x, units);
  for (int64_t b0 = kScan; b0 < a.B; b0 += kScan) total += scan_requests(a, b0, x, units);
  return total;
}
// (the first 256 requests' spans stay in LDS unless there are more requests)
__device__ __forceinline__ Span span_at(const KvAttend& a, const Prefix& x, int b) {
  if (a.B > kScan) return span_of(a, b);
  Span s{x.t0[b], x.n[b], 0, x.past[b]};
  s.len = places(a, s);
  return s;
}

// The request of unit u (a wave's own) after total_units, and the units before it; the first one where u is past the end.
struct Place {
  int b;
  int64_t before;
};
template <class U>
__device__ __forceinline__ Place place_of(const KvAttend& a, Prefix& x, int64_t total, int64_t u, U units) {
  Place p{0, 0};
  int64_t carry = 0;
  bool found = false;
  for (int64_t b0 = 0; b0 < a.B && carry < total; b0 += kScan) {
    const int64_t here = a.B <= kScan ? total : scan_requests(a, b0, x, units);
    if (!found && u < carry + here) {
      int lo = 0;  // the first request whose inclusive sum is above u - carry: behind all whose sums are not
      for (int i = threadIdx.x % kWave; b0 + i - i % kWave < a.B && i < kScan; i += kWave)
        lo += __popcll(__ballot(b0 + i < a.B && x.incl[i] <= u - carry));
      p.b = (int)b0 + lo;
      p.before = carry + (lo ? x.incl[lo - 1] : 0);
      found = true;
    }
    carry += here;
  }
  p.b = __builtin_amdgcn_readfirstlane(p.b);
  return p;
}

// Equal shares of the units for the workgroups, `least` units at least each.
struct Shares {
  int64_t total, groups, each, more;  // each: units of a workgroup; the first `more` have one more
  __device__ __forceinline__ int64_t of_group(int64_t g) const { return each * g + min(g, more); }
  __device__ __forceinline__ int64_t units_of_group(int64_t g) const { return each + (g < more ? 1 : 0); }
  __device__ __forceinline__ int64_t group_of(int64_t u) const {
    const int64_t big = more * (each + 1);
    return u < big ? divide(u, each + 1) : more + divide(u - big, each);
  }
};
__device__ __forceinline__ Shares shares_of(int64_t total, int64_t groups, int64_t least) {
  groups = max((int64_t)1, min(groups, divide(total, least)));
  const int64_t each = divide(total, groups);
  return Shares{total, groups, each, total - each * groups};
}

// N elements (8 or 16) of a query row from element d on, as they are stored (minus: with the other sign); zero for no row
template <class X, int N>
struct QueryPart {
  static constexpr int kSize = sizeof(typename X::storage), kVectors = N * kSize / 16;
  u32x4 w[kVectors];
  __device__ __forceinline__ void load(const typename X::storage* row, int d, bool ok, bool wide, bool minus) {
#pragma unroll
    for (int i = 0; i < kVectors; ++i) w[i] = u32x4{0, 0, 0, 0};
    if (!ok) return;
    if (wide) {
#pragma unroll
      for (int i = 0; i < kVectors; ++i) w[i] = *reinterpret_cast<const u32x4*>(row + d + 16 / kSize * i);
    } else {
#pragma unroll
      for (int i = 0; i < N; ++i) {
        if constexpr (kSize == 4) w[i / 4][i % 4] = __float_as_uint(row[d + i]);
        else w[i / 8][i / 2 % 4] |= (uint32_t)row[d + i] << (16 * (i & 1));
      }
    }
    if (minus) {
#pragma unroll
      for (int i = 0; i < kVectors; ++i) w[i] ^= kSize == 4 ? 0x80000000u : 0x80008000u;
    }
  }
  // term t of CH: eight elements as an operand
  template <int CH>
  __device__ __forceinline__ void terms(int eight, bf16x8 (&out)[CH]) const {
    if constexpr (kSize == 2) {
      out[0] = __builtin_bit_cast(bf16x8, w[eight]);
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        float e = __uint_as_float(w[2 * eight + i / 4][i % 4]);
#pragma unroll
        for (int t = 0; t < CH; ++t) {
          const __bf16 v = (__bf16)e;
          out[t][i] = v;
          e -= (float)v;
        }
      }
    }
  }
};

__device__ __forceinline__ float row16_max(float v) {  // over aligned groups of 16 lanes
  v = fmaxf(v, dpp_move<0xB1>(v));
  v = fmaxf(v, dpp_move<0x4E>(v));
  v = fmaxf(v, dpp_move<0x141>(v));
  return fmaxf(v, dpp_move<0x140>(v));
}
__device__ __forceinline__ float row16_sum(float v) {
  v += dpp_move<0xB1>(v);
  v += dpp_move<0x4E>(v);
  v += dpp_move<0x141>(v);
  return v + dpp_move<0x140>(v);
}

// Rows of tokens that belong to no request, in front of the first one's and behind the last one's: zero.
template <class X>
__device__ __forceinline__ void clear_idle_rows(const KvAttend& a) {
  if (!a.q_start) return;
  const int T = (int)a.T;
  const int front = a.B > 0 ? min(max(a.q_start[0], 0), T) : 0, back = a.B > 0 ? min(max(a.q_start[a.B], front), T) : 0;
  if (front == 0 && back == T) return;
  typename X::storage* const O = reinterpret_cast<typename X::storage*>(a.O);
  const int64_t row = (int64_t)a.heads * a.c.dim, all = (int64_t)gridDim.x * gridDim.y * blockDim.x;
  const int64_t me = ((int64_t)blockIdx.y * gridDim.x + blockIdx.x) * blockDim.x + threadIdx.x;
  const int64_t idle = front + (T - back), skip = back - front;
  for (int64_t i = me; i < idle * row; i += all) X::store(O, i < front * row ? i : i + skip * row, 0.f);
  if (a.lse)
    for (int64_t i = me; i < idle * a.heads; i += all) a.lse[i < (int64_t)front * a.heads ? i : i + skip * a.heads] = -INFINITY;
}

// A rare path that is to stay a branch: the compiler would compute both sides for every element.  The condition is the same in every lane.
__device__ __forceinline__ bool rarely(bool x) { return __builtin_expect(__builtin_amdgcn_readfirstlane((int)x), 0); }
__device__ __forceinline__ void keep_branch() { asm volatile(""); }

// Reads of LDS stay in front of this point: the compiler would request each right before its use and wait for all of its latency.
__device__ __forceinline__ void hold_lds() { __builtin_amdgcn_sched_barrier(0x41f); }

// Nothing is moved across this point.
__device__ __forceinline__ void hold_all() { __builtin_amdgcn_sched_barrier(0); }

// Ends the wait for an operand that was loaded before a loop: the compiler would wait for all loads there, in every step.
__device__ __forceinline__ void arrive(bf16x8& x) { asm volatile("" : "+v"(x)); }

__device__ __forceinline__ void order_lds() { asm volatile("" ::: "memory"); }  // a wave's LDS accesses run in program order

}  // namespace
}  // namespace gsi
