// Attention over the paged cache in 4 bits, many rows: prompts and their chunks.
//
// A workgroup of four waves takes 128 rows (tokens times the heads that share a head of keys), 32 a wave, and 64 keys a step.  Scores and
// outputs are kept transposed, tokens by rows and elements by rows: a row's scores then lie in two lanes, its maximum and its sum
// need no exchange but one, and the weights are the second product's operand as they come out of the first (the tokens of its
// contraction taken in the order of the accumulator's registers).  Keys lie in LDS as they are held, 16 bytes a block, and every wave converts
// what it reads; values are converted once, on their way to LDS, and read there with the transposing reads.
#include <algorithm>

#include "gsi_attend.h"

namespace gsi {
namespace {

constexpr int kWaves = 4, kThreads = kWaves * kWave;
constexpr int kTile = 32 * kWaves;  // rows of a workgroup
constexpr int kStep = 64;           // keys of a step

typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef short s16x8 __attribute__((ext_vector_type(8)));
typedef __attribute__((address_space(3))) s16x4 lds_s16x4;

struct Prompt {
  KvAttend a;
  int64_t few;   // requests of at most so many rows are another kernel's
  int group;
  int q_wide;
  int splits;    // parts of a tile's keys
  int zero;      // whether this launch writes the tokens of no request
  float* parts;  // [splits][T * heads][dim + 2]: sums, maximum, sum of weights
};

template <int ND>
struct Lds {  // of one step
  static constexpr int kStride = 64 * (ND | 1);  // bytes of a token's values: four tokens lie in distinct banks
  static constexpr int kKeys = 0, kScales = ND * kStep * 16, kValues = kScales + ND * kStep, kSize = kValues + kStep * kStride;
};

__device__ __forceinline__ int64_t tiles_of(const Prompt& f, const Span& s) {
  const int64_t rows = (int64_t)s.n * f.group;
  return rows > f.few ? (rows + kTile - 1) / kTile : 0;
}

// the request of tile `slot` and the tiles before it; -1: there are not so many
__device__ __forceinline__ int owner_of(const Prompt& f, int64_t slot, int64_t& before, int64_t* lds) {
  const int lane = threadIdx.x % kWave;
  if (threadIdx.x == 0) lds[4] = -1;
  int64_t carry = 0;
  for (int64_t b0 = 0; b0 < f.a.B; b0 += kThreads) {
    const int64_t b = b0 + threadIdx.x;
    const int64_t mine = b < f.a.B ? tiles_of(f, span_of(f.a, (int)b)) : 0;
    int64_t incl = mine;
#pragma unroll
    for (int o = 1; o < kWave; o <<= 1) {
      const int64_t up = __shfl_up(incl, o, kWave);
      if (lane >= o) incl += up;
    }
    __syncthreads();
    if (lane == kWave - 1) lds[threadIdx.x / kWave] = incl;
    __syncthreads();
    int64_t at = carry;
    for (int w = 0; w < (int)threadIdx.x / kWave; ++w) at += lds[w];
    at += incl - mine;
    if (slot >= at && slot < at + mine) {
      lds[4] = b;
      lds[5] = at;
    }
    carry += lds[0] + lds[1] + lds[2] + lds[3];
    if (slot < carry) break;
  }
  __syncthreads();
  before = lds[5];
  return (int)lds[4];
}

__device__ __forceinline__ uint32_t bf16_pair(float a, float b) {
  const bf16x2 v = {(__bf16)a, (__bf16)b};
  return __builtin_bit_cast(uint32_t, v);
}
template <int SEL>
__device__ __forceinline__ uint32_t two_values(uint32_t w, float scale) {
  return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, SEL));
}
__device__ __forceinline__ u32x4 eight_values(uint32_t w, float scale) {
  return u32x4{two_values<0>(w, scale), two_values<1>(w, scale), two_values<2>(w, scale), two_values<3>(w, scale)};
}

template <class X, int ND>
__global__ __launch_bounds__(kThreads, ND <= 4 ? 2 : 1) void prompt_kernel(Prompt f) {
  constexpr bool F = sizeof(typename X::storage) == 4;
  constexpr int QT = F ? 3 : 1, PT = F ? 3 : 1, NP = (ND + 1) / 2, KU = (ND + 3) / 4;
  using M = Lds<ND>;
  extern __shared__ __align__(16) char lds[];
  __shared__ int64_t scan[6];
  __shared__ int spoiled[3][ND];  // first token of a step whose value is NaN, by block: three steps' worth, one of them being cleared
  const KvAttend& a = f.a;
  const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave, c = lane & 31, h = lane >> 5;
  constexpr int D = 32 * ND, half = D / 2;

  // heads of keys run fastest: with eight of them and more, an XCD's cache holds the same ones throughout
  const int kvh = blockIdx.x % a.c.heads;
  int64_t before;
  const int b = __builtin_amdgcn_readfirstlane(owner_of(f, blockIdx.x / a.c.heads, before, scan));
  if (f.zero) clear_idle_rows<X>(a);
  if (b < 0) return;
  const Span sp = span_of(a, b);
  // the last tile, which sees the most keys, first
  const int tile = (int)(tiles_of(f, sp) - 1 - (blockIdx.x / a.c.heads - before));
  const int all_rows = sp.n * f.group, row0 = tile * kTile, shift0 = sp.len - sp.n;

  const int rid = row0 + 32 * wave + c;
  const bool real = rid < all_rows;
  const int tok = real ? rid / f.group : 0, head = kvh * f.group + (real ? rid % f.group : 0);
  const int lim = real ? shift0 + tok : -1;  // the last key that this lane's row sees
  // of the wave's rows, and of the workgroup's: the last key that any sees, and the last that all see (idle rows aside)
  const int wave_first = row0 + 32 * wave, wave_last = min(wave_first + 31, all_rows - 1);
  const int wave_high = wave_first < all_rows ? shift0 + wave_last / f.group : -1;
  const int wave_low = wave_first < all_rows ? shift0 + wave_first / f.group : -1;
  const int high = shift0 + min(row0 + kTile - 1, all_rows - 1) / f.group, low = shift0 + row0 / f.group;

  // query rows: the operand's elements 8 h + u of product (p, w) are elements 32 (2 p + h) + 8 w + u
  bf16x8 q[NP][4][QT];
  {
    const typename X::storage* const Q = reinterpret_cast<const typename X::storage*>(a.Q) + (int64_t)(sp.t0 + tok) * a.q_stride + (int64_t)head * D;
#pragma unroll
    for (int p = 0; p < NP; ++p)
#pragma unroll
      for (int y = 0; y < 2; ++y) {
        Query16<X> raw;
        const int d = 32 * (2 * p + h) + 16 * y;
        raw.load(Q, d, real && d < D, f.q_wide, a.scale < 0.f);
        raw.template terms<QT>(0, q[p][2 * y]);
        raw.template terms<QT>(1, q[p][2 * y + 1]);
      }
  }

  f32x16 o[ND];
#pragma unroll
  for (int d = 0; d < ND; ++d)
#pragma unroll
    for (int i = 0; i < 16; ++i) o[d][i] = 0.f;
  float m = -INFINITY, l = 0.f;
  const float zscale = exponent_scale(a.scale);

  const int steps = high < 0 ? 0 : high / kStep + 1;
  const int step0 = (int)((int64_t)steps * blockIdx.y / f.splits), step1 = (int)((int64_t)steps * (blockIdx.y + 1) / f.splits);
  const int32_t* const trow = a.table + (int64_t)b * a.width;
  const int last = (int)a.width - 1, mask = a.c.page() - 1;

  // what a thread brings of a step: blocks of keys (one token's 32 codes), scale bytes of four keys, words of values (8 codes) with their scale
  struct Bring {
    u32x4 k[KU];
    uint32_t ks;
    uint32_t v[ND];
    uint32_t vs[ND];
    int there;  // a bit for each 16 tokens whose page is there
  };
  struct Entries {
    int e[4];
  };
  const auto entries = [&](int step) {
    Entries r;
#pragma unroll
    for (int g = 0; g < 4; ++g) r.e[g] = trow[min((step * kStep + 16 * g) >> a.c.page_shift, last)];
    return r;
  };
  const int uwave = __builtin_amdgcn_readfirstlane(wave);
  const int64_t code0 = a.c.code_at(0, kvh), scale0 = a.c.scale_at(0, kvh);
  const uint32_t code_stride = (uint32_t)a.c.code_at(1, 0), scale_stride = (uint32_t)a.c.scale_at(1, 0);
  struct Four {
    uint64_t a, b, c, d;
  };
  const auto pick = [](Four x, int g) {
    const uint64_t a = x.a, b = x.b, c = x.c, d = x.d;
    const uint64_t low = (g & 1) ? b : a, high = (g & 1) ? d : c;
    return (g & 2) ? high : low;
  };
  // the same in every lane of a wave
  const auto uniform = [](uint64_t x) {
    return (uint64_t)(uint32_t)__builtin_amdgcn_readfirstlane((int)(uint32_t)(x >> 32)) << 32 | (uint32_t)__builtin_amdgcn_readfirstlane((int)(uint32_t)x);
  };
  // token and block of the i-th block of keys: where the blocks of 16 tokens fill waves, a wave's lie on one page
  struct TokenBlock {
    int t, blk;
  };
  const auto key_block = [](int i) {
    const int u = i * kThreads + threadIdx.x;
    if constexpr (ND % 4 == 0) return TokenBlock{u / (16 * ND) * 16 + u % 16, u % (16 * ND) / 16};
    else return TokenBlock{u % kStep, u / kStep};
  };
  // word u of the values: 64 ND words to 16 tokens, so that a wave's lie on one page; token u / (4 ND), word u % (4 ND) of it
  const auto bring = [&](int step, const Entries& en) {
    Bring r;
    r.there = 0;
    const auto place = [&](int g, uint64_t base, uint32_t stride, int each) {
      const uint32_t page = __builtin_amdgcn_readfirstlane(en.e[g]);  // (here, a step later: its load is not waited for where it is requested)
      const bool ok = page < (uint32_t)a.c.n_pages;
      r.there |= ok ? 1 << g : 0;
      return base + (uint64_t)(ok ? page : 0u) * stride + ((step * kStep + 16 * g) & mask) * each;
    };
    const Four code{place(0, code0, code_stride, half), place(1, code0, code_stride, half), place(2, code0, code_stride, half), place(3, code0, code_stride, half)};
    const Four scale{place(0, scale0, scale_stride, 1), place(1, scale0, scale_stride, 1), place(2, scale0, scale_stride, 1), place(3, scale0, scale_stride, 1)};
#pragma unroll
    for (int i = 0; i < KU; ++i) {
      const auto [t, blk] = key_block(i);
      if constexpr (ND % 4 == 0) r.k[i] = *reinterpret_cast<const u32x4*>(a.c.K + uniform(pick(code, (i * kWaves + uwave) / (ND / 4))) + (uint32_t)((t % 16) * half + blk * 16));
      else if (blk < ND) r.k[i] = *reinterpret_cast<const u32x4*>(a.c.K + pick(code, t / 16) + ((t % 16) * half + blk * 16));
    }
    if ((int)threadIdx.x < ND * 16) {
      const int t = threadIdx.x % 16 * 4, blk = threadIdx.x / 16;
      r.ks = *reinterpret_cast<const uint32_t*>(a.c.Ks + pick(scale, t / 16) + ((blk << a.c.page_shift) + t % 16));
    }
#pragma unroll
    for (int i = 0; i < ND; ++i) {
      const int g = ND % 4 == 0 ? i / (ND / 4) : (i * kWaves + uwave) / ND, u = i * kThreads + threadIdx.x, t = u / (4 * ND), w = u % (4 * ND);
      r.v[i] = *reinterpret_cast<const uint32_t*>(a.c.V + uniform(pick(code, g)) + (uint32_t)((t % 16) * half + w * 4));
      r.vs[i] = (a.c.Vs + uniform(pick(scale, g)))[(uint32_t)(((w / 4) << a.c.page_shift) + t % 16)];
    }
    return r;
  };
  const auto stage = [&](int step, const Bring& r) {
    char* const at = lds + (step & 1) * M::kSize;
    const bool special = rarely(step * kStep + kStep - 1 > low || r.there != 15);
#pragma unroll
    for (int i = 0; i < KU; ++i) {
      const auto [t, blk] = key_block(i);
      if (ND % 4 == 0 || blk < ND) *reinterpret_cast<u32x4*>(at + M::kKeys + (blk * kStep + t) * 16) = r.k[i];
    }
    if ((int)threadIdx.x < ND * 16) *reinterpret_cast<uint32_t*>(at + M::kScales + threadIdx.x * 4) = r.ks;
#pragma unroll
    for (int i = 0; i < ND; ++i) {
      const int u = i * kThreads + threadIdx.x, t = u / (4 * ND), w = u % (4 * ND);
      uint32_t word = r.v[i], vs = r.vs[i];
      if (special) {
        keep_branch();
        // 0 times what is not seen, or seen by some rows only, has to be 0: NaN goes to its rows by `spoiled`
        const bool seen = step * kStep + t < sp.len && (r.there >> (t / 16) & 1);
        if (seen && vs == 255u) atomicMin(&spoiled[step % 3][w / 4], step * kStep + t);
        if (!seen || vs == 255u) {
          word = 0;
          vs = 127;
        }
      }
      *reinterpret_cast<u32x4*>(at + M::kValues + t * M::kStride + w * 16) = eight_values(word, scale_value(vs));
    }
  };

  if ((int)threadIdx.x < 3 * ND) spoiled[threadIdx.x / ND][threadIdx.x % ND] = 0x7fffffff;
  __syncthreads();
  int there = 15;
  Entries en{};
  if (step0 < step1) {
    const Bring r = bring(step0, entries(step0));
    en = entries(step0 + 1);
    there = r.there;
    stage(step0, r);
  }
#pragma unroll
  for (int p = 0; p < NP; ++p)
#pragma unroll
    for (int w = 0; w < 4; ++w)
#pragma unroll
      for (int t = 0; t < QT; ++t) arrive(q[p][w][t]);
  __syncthreads();
  const int vlane = (4 * h + ((lane & 15) >> 2)) * M::kStride + 32 * ((lane >> 4) & 1) + 8 * (lane & 3);
  for (int step = step0; step < step1; ++step) {
    Bring next;
    const bool more = step + 1 < step1;
    if (more) {
      next = bring(step + 1, en);
      en = entries(step + 2);
    }
    if ((int)threadIdx.x < ND) spoiled[(step + 2) % 3][threadIdx.x] = 0x7fffffff;
    const char* const at = lds + (step & 1) * M::kSize;
    const int key = step * kStep;
    if (key <= wave_high) {  // else no row of this wave sees the step
      f32x16 s[2];
#pragma unroll
      for (int y = 0; y < 2; ++y)
#pragma unroll
        for (int i = 0; i < 16; ++i) s[y][i] = 0.f;
#pragma unroll
      for (int p = 0; p < NP; ++p) {
        const bool in = ND % 2 == 0 || 2 * p + h < ND;
        const int blk = in ? 2 * p + h : ND - 1;
        u32x4 code[2];
        float sc[2];
#pragma unroll
        for (int y = 0; y < 2; ++y) {
          code[y] = *reinterpret_cast<const u32x4*>(at + M::kKeys + (blk * kStep + 32 * y + c) * 16);
          const uint32_t byte = reinterpret_cast<const uint8_t*>(at + M::kScales)[blk * kStep + 32 * y + c];
          sc[y] = in ? scale_value(byte) : 1.f;
        }
#pragma unroll
        for (int w = 0; w < 4; ++w)
#pragma unroll
          for (int y = 0; y < 2; ++y) {
            const bf16x8 k = __builtin_bit_cast(bf16x8, eight_values(code[y][w], sc[y]));
#pragma unroll
            for (int t = 0; t < QT; ++t) s[y] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(k, q[p][w][t], s[y], 0, 0, 0);
          }
      }
      if (rarely(key + kStep - 1 > wave_low || there != 15)) {
        keep_branch();
#pragma unroll
        for (int y = 0; y < 2; ++y)
#pragma unroll
          for (int i = 0; i < 16; ++i) {
            const int t = 32 * y + 8 * (i / 4) + 4 * h + i % 4;
            s[y][i] = key + t <= lim && (there >> (2 * y + i / 8) & 1) ? s[y][i] : -INFINITY;
          }
      }
      if (rarely(key + kStep - 1 > low || there != 15)) {  // as stage() has it
        keep_branch();
#pragma unroll
        for (int d = 0; d < ND; ++d)
          if (spoiled[step % 3][d] <= lim) {
#pragma unroll
            for (int i = 0; i < 16; ++i) o[d][i] = NAN;
          }
      }
      float top = s[0][0];
#pragma unroll
      for (int y = 0; y < 2; ++y)
#pragma unroll
        for (int i = 0; i < 16; ++i) top = fmaxf(top, s[y][i]);
      if (__any(top * zscale > m + kSlack)) {
        top = fmaxf(top, __shfl_xor(top, 32, kWave));
        const float next_m = fmaxf(m, top * zscale);
        const float keep = next_m == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(m - next_m);
        m = next_m;
        l *= keep;
#pragma unroll
        for (int d = 0; d < ND; ++d)
#pragma unroll
          for (int i = 0; i < 16; ++i) o[d][i] *= keep;
      }
      const float base = m == -INFINITY ? 0.f : m;
#pragma unroll
      for (int y = 0; y < 2; ++y)
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          s[y][i] = __builtin_amdgcn_exp2f(fmaf(s[y][i], zscale, -base));
          l += s[y][i];
        }
#pragma unroll
      for (int y = 0; y < 2; ++y)
#pragma unroll
        for (int x = 0; x < 2; ++x) {
          bf16x8 pf[PT];
#pragma unroll
          for (int t = 0; t < PT; ++t) {
            u32x4 w;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              float& lo = reinterpret_cast<float*>(&s[y])[8 * x + 2 * i];
              float& hi = reinterpret_cast<float*>(&s[y])[8 * x + 2 * i + 1];
              w[i] = bf16_pair(lo, hi);
              if (t + 1 < PT) {
                lo -= bf16_lo(w[i]);
                hi -= bf16_hi(w[i]);
              }
            }
            pf[t] = __builtin_bit_cast(bf16x8, w);
          }
          const char* const va = at + M::kValues + vlane + (32 * y + 16 * x) * M::kStride;
#pragma unroll
          for (int d = 0; d < ND; ++d) {
            const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(va + 64 * d));
            const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(va + 64 * d + 8 * M::kStride));
            const bf16x8 v = __builtin_bit_cast(bf16x8, (s16x8)__builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
#pragma unroll
            for (int t = 0; t < PT; ++t) o[d] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(v, pf[t], o[d], 0, 0, 0);
          }
        }
    }
    if (more) {
      stage(step + 1, next);
      there = next.there;
    }
    __syncthreads();
  }

  l += __shfl_xor(l, 32, kWave);
  if (!real) return;
  const int64_t orow = (int64_t)(sp.t0 + tok) * a.heads + head;
  if (f.splits == 1) {
    const float inv = l == 0.f ? 0.f : 1.f / l;
    typename X::storage* const out = reinterpret_cast<typename X::storage*>(a.O) + orow * D;
#pragma unroll
    for (int d = 0; d < ND; ++d)
#pragma unroll
      for (int i = 0; i < 16; i += 4) {
        typename X::storage* const p = out + 32 * d + 2 * i + 4 * h;
        if constexpr (F) *reinterpret_cast<f32x4*>(p) = f32x4{o[d][i] * inv, o[d][i + 1] * inv, o[d][i + 2] * inv, o[d][i + 3] * inv};
        else *reinterpret_cast<u32x2*>(p) = u32x2{bf16_pair(o[d][i] * inv, o[d][i + 1] * inv), bf16_pair(o[d][i + 2] * inv, o[d][i + 3] * inv)};
      }
    if (a.lse && h == 0) a.lse[orow] = l == 0.f ? -INFINITY : (m == -INFINITY ? l : (m + log2f(l)) * kLn2);
  } else {
    float* const out = f.parts + ((int64_t)blockIdx.y * a.T * a.heads + orow) * (D + 2);
#pragma unroll
    for (int d = 0; d < ND; ++d)
#pragma unroll
      for (int i = 0; i < 16; i += 2) *reinterpret_cast<f32x2*>(out + 32 * d + 8 * (i / 4) + 4 * h + i % 4) = f32x2{o[d][i], o[d][i + 1]};
    if (h == 0) {
      out[D] = m;
      out[D + 1] = l;
    }
  }
}

// Joins the parts of a tile's keys, a workgroup per token and head, in their order.
template <class X>
__global__ __launch_bounds__(kKvMaxDim) void join_parts(Prompt f) {
  const KvAttend& a = f.a;
  const int t = blockIdx.x, head = blockIdx.y, D = a.c.dim, d = threadIdx.x;
  int lo = 0, hi = (int)a.B;  // the request with q_start[lo] <= t < q_start[lo + 1]
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if ((a.q_start ? a.q_start[mid] : mid) <= t) lo = mid;
    else hi = mid;
  }
  const Span sp = span_of(a, lo);
  if (t < sp.t0 || t >= sp.t0 + sp.n || tiles_of(f, sp) == 0) return;
  const int64_t orow = (int64_t)t * a.heads + head;
  const float* const p0 = f.parts + orow * (D + 2);
  const int64_t next = a.T * a.heads * (int64_t)(D + 2);
  float top = -INFINITY;
  for (int i = 0; i < f.splits; ++i) top = fmaxf(top, p0[i * next + D]);
  float sum = 0.f, o = 0.f;
  for (int i = 0; i < f.splits; ++i) {
    const float* const p = p0 + i * next;
    const float k = p[D] == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(p[D] - top);
    sum += p[D + 1] * k;
    if (d < D) o += p[d] * k;
  }
  if (d < D) X::store(reinterpret_cast<typename X::storage*>(a.O), orow * D + d, sum == 0.f ? 0.f : o / sum);
  if (a.lse && d == 0) a.lse[orow] = sum == 0.f ? -INFINITY : (top == -INFINITY ? sum : (top + log2f(sum)) * kLn2);
}

int64_t prompt_slots(const KvAttend& a) { return ceil_div(a.T * (a.heads / a.c.heads), kTile) + a.B; }

// Parts of the keys of every tile: where the tiles leave the chip idle (two workgroups a unit), as many as fill it, of 256 keys at least.
int prompt_splits(const KvAttend& a) {
  const int64_t rows = a.T * (a.heads / a.c.heads);
  const int64_t tiles = std::max<int64_t>(1, rows / kTile) * a.c.heads;
  return (int)std::max<int64_t>(1, std::min<int64_t>(512 / tiles, a.max_len / 256));
}

template <class X, int ND>
hipError_t launch_prompt(const Prompt& f, hipStream_t s) {
  const int bytes = 2 * Lds<ND>::kSize;
  static LdsLimit limit;
  if (bytes > 60 * 1024)
    if (hipError_t e = limit.allow((const void*)prompt_kernel<X, ND>, bytes); e != hipSuccess) return e;
  prompt_kernel<X, ND><<<dim3((unsigned)(prompt_slots(f.a) * f.a.c.heads), f.splits), kThreads, bytes, s>>>(f);
  if (f.splits > 1) join_parts<X><<<dim3((unsigned)f.a.T, f.a.heads), kKvMaxDim, 0, s>>>(f);
  return hipGetLastError();
}
template <class X>
hipError_t launch_prompt(const Prompt& f, hipStream_t s) {
  switch (f.a.c.dim / 32) {
    case 1: return launch_prompt<X, 1>(f, s);
    case 2: return launch_prompt<X, 2>(f, s);
    case 3: return launch_prompt<X, 3>(f, s);
    case 4: return launch_prompt<X, 4>(f, s);
    case 5: return launch_prompt<X, 5>(f, s);
    case 6: return launch_prompt<X, 6>(f, s);
    case 7: return launch_prompt<X, 7>(f, s);
    default: return launch_prompt<X, 8>(f, s);
  }
}

}  // namespace

size_t attend_prompt_workspace(const KvAttend& a) {
  const int n = prompt_splits(a);
  return n > 1 ? align_up((size_t)n * a.T * a.heads * (a.c.dim + 2) * sizeof(float), 256) : 0;
}

hipError_t attend_prompt(const KvAttend& a, int64_t few, bool zero, void* ws, hipStream_t s) {
  Prompt f{};
  f.a = a;
  f.few = few;
  f.group = a.heads / a.c.heads;
  const size_t es = elem_size(a.dtype);
  f.q_wide = reinterpret_cast<uintptr_t>(a.Q) % 16 == 0 && (size_t)a.q_stride * es % 16 == 0;
  f.splits = prompt_splits(a);
  f.zero = zero;
  f.parts = reinterpret_cast<float*>(ws);
  return a.dtype == GSI_BF16 ? launch_prompt<BF16>(f, s) : launch_prompt<F32>(f, s);
}

}  // namespace gsi
