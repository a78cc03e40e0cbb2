// Attention over the paged cache in 4 bits, few rows: single tokens, and a few tokens of a request.
//
// For a row (a token and a head) with query q: s_j = scale q.k_j over the keys that it sees, o = sum_j 2^(s_j' - m) v_j / sum_j 2^(s_j' - m),
// s' = s log2 e, m a running maximum.  A workgroup takes up to 16 rows that share a head of keys and 256 keys at a time, 64 a
// wave.  Both products are bf16 matrix products of codes times scales (exact in bf16).  A lane loads 32 consecutive codes of a key, which
// are its operands of four products over 8 elements each, and 4, 8 or 16 elements of eight consecutive values, which
// are the rows of as many products over 32 tokens: neither keys nor values need a transposition through LDS.
#include <algorithm>

#include "gsi_attend.h"

namespace gsi {
namespace {

constexpr int kWaves = 4, kThreads = kWaves * kWave;
constexpr int kStep = 64;               // keys of a wave and step
constexpr int kUnit = kWaves * kStep;   // keys of a workgroup and step: the unit in which the work is dealt out
constexpr int kRows = 16;               // rows of the products
constexpr int kPStride = kStep + 8;     // bf16 elements of a row of weights in LDS

struct Few {
  KvAttend a;
  int64_t few;    // requests of more rows are another kernel's
  int group;      // heads that share a head of keys
  int tile_rows;  // rows of a tile: 4, 8 or 16
  int q_wide;     // 16-byte loads of queries
  float* parts;   // [2 * workgroups][tile_rows][dim + 2]: sums, maximum, sum of weights of a cut tile
  int* heads;     // [workgroups][4]: the tile that a workgroup begins and does not end, and the workgroup that ends it
};

__device__ __forceinline__ int rows_of(const Few& f, const Span& s) {
  const int64_t rows = (int64_t)s.n * f.group;
  return rows <= f.few ? (int)rows : 0;
}
// Units of a request: tiles of rows, times heads of keys, times units of keys (one where there are rows but no keys)
__device__ __forceinline__ int64_t units_of(const Few& f, const Span& s, int& per_tile, int& tiles) {
  tiles = (rows_of(f, s) + f.tile_rows - 1) / f.tile_rows;
  per_tile = max(1, (s.len + kUnit - 1) / kUnit);
  return (int64_t)tiles * f.a.c.heads * per_tile;
}

// The units of all requests, and the request that unit `u` lies in with the units before it.  One round of loads up to 256 requests.
struct Place {
  int64_t total, before;
  int b;
};
__device__ __forceinline__ int64_t wave_scan(int64_t v) {
  const int lane = threadIdx.x % kWave;
#pragma unroll
  for (int o = 1; o < kWave; o <<= 1) {
    const int64_t up = __shfl_up(v, o, kWave);
    if (lane >= o) v += up;
  }
  return v;
}
__device__ __forceinline__ int64_t total_units(const Few& f, int64_t* lds) {
  int64_t sum = 0;
  int per, tiles;
  for (int64_t b = threadIdx.x; b < f.a.B; b += kThreads) sum += units_of(f, span_of(f.a, (int)b), per, tiles);
  sum = wave_scan(sum);
  __syncthreads();
  if (threadIdx.x % kWave == kWave - 1) lds[threadIdx.x / kWave] = sum;
  __syncthreads();
  return lds[0] + lds[1] + lds[2] + lds[3];
}
__device__ __forceinline__ Place place_of_unit(const Few& f, int64_t u, int64_t* lds) {
  // lds: [0..3] sums of the waves, [4] request, [5] units before it
  Place p{0, 0, 0};
  int64_t carry = 0;
  for (int64_t b0 = 0; b0 < f.a.B; b0 += kThreads) {
    const int64_t b = b0 + threadIdx.x;
    int per, tiles;
    const int64_t mine = b < f.a.B ? units_of(f, span_of(f.a, (int)b), per, tiles) : 0;
    const int64_t incl = wave_scan(mine);
    __syncthreads();
    if (threadIdx.x % kWave == kWave - 1) lds[threadIdx.x / kWave] = incl;
    __syncthreads();
    int64_t at = carry;
    for (int w = 0; w < (int)threadIdx.x / kWave; ++w) at += lds[w];
    const int64_t before = at + incl - mine;
    if (u >= before && u < before + mine) {
      lds[4] = b;
      lds[5] = before;
    }
    carry += lds[0] + lds[1] + lds[2] + lds[3];
    if (u < carry) break;  // the same for every thread
  }
  __syncthreads();
  p.b = (int)lds[4];
  p.before = lds[5];
  __syncthreads();
  return p;
}

// ---- a step's operands: 64 keys and values ------------------------------------------------------------------
template <int DPL>
struct VWord;  // the codes of a lane's DPL elements of a token
template <> struct VWord<4> { using type = uint16_t; };
template <> struct VWord<8> { using type = uint32_t; };
template <> struct VWord<16> { using type = u32x2; };

template <int DPL>
struct Step {
  static constexpr int DC = DPL == 16 ? 2 : 1;  // products of 128 elements of a key
  u32x4 k[DC][4];     // token 4 c + j of lane c's block
  uint32_t ks[DC];    // its four scale bytes
  typename VWord<DPL>::type v[2][8];
  u32x2 vs[2];
};

struct Pages {  // page ids of a lane's keys and of its two groups of eight values; as the table has them
  int k, v[2];
};

template <int DPL>
struct Lane {  // where a lane's operands lie
  int c, g;         // lane % 16, lane / 16
  int kblk[2];      // blocks of 32 elements of a key (held in range)
  bool kreal[2];
  int vd;           // first element of its values (held in range)
  __device__ __forceinline__ Lane(int dim) {
    const int lane = threadIdx.x % kWave;
    c = lane % 16;
    g = lane / 16;
#pragma unroll
    for (int x = 0; x < 2; ++x) {
      kreal[x] = (g + 4 * x) * kKvBlock < dim;
      kblk[x] = kreal[x] ? g + 4 * x : 0;
    }
    vd = c * DPL < dim ? c * DPL : 0;
  }
};

template <int DPL>
__device__ __forceinline__ Pages load_pages(const int32_t* row, int64_t width, int shift, const Lane<DPL>& L, int key) {
  // entries past the row's end are not needed: no key lies there
  const int last = (int)width - 1;
  Pages p;
  p.k = row[min((key + 4 * L.c) >> shift, last)];
#pragma unroll
  for (int h = 0; h < 2; ++h) p.v[h] = row[min((key + 32 * h + 8 * L.g) >> shift, last)];
  return p;
}

template <int DPL>
__device__ __forceinline__ void load_step(Step<DPL>& s, const KvView& c, int kvh, const Pages& p, const Lane<DPL>& L, int key) {
  const int mask = c.page() - 1, half = c.dim / 2;
  const int64_t n = c.n_pages;
  {
    const int64_t page = (uint32_t)p.k < (uint32_t)n ? p.k : 0;  // another page's keys are not seen
    const int off = (key + 4 * L.c) & mask;
    const uint8_t* const codes = c.K + c.code_at(page, kvh) + (int64_t)off * half;
    const uint8_t* const scales = c.Ks + c.scale_at(page, kvh) + off;
#pragma unroll
    for (int x = 0; x < Step<DPL>::DC; ++x) {
      const uint8_t* const at = codes + L.kblk[x] * 16;
#pragma unroll
      for (int j = 0; j < 4; ++j) s.k[x][j] = *reinterpret_cast<const u32x4*>(at + j * half);
      s.ks[x] = *reinterpret_cast<const uint32_t*>(scales + ((int64_t)L.kblk[x] << c.page_shift));
    }
  }
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const int64_t page = (uint32_t)p.v[h] < (uint32_t)n ? p.v[h] : 0;
    const int off = (key + 32 * h + 8 * L.g) & mask;
    const uint8_t* const at = c.V + c.code_at(page, kvh) + (int64_t)off * half + L.vd / 2;
#pragma unroll
    for (int u = 0; u < 8; ++u) s.v[h][u] = *reinterpret_cast<const typename VWord<DPL>::type*>(at + u * half);
    s.vs[h] = *reinterpret_cast<const u32x2*>(c.Vs + c.scale_at(page, kvh) + ((int64_t)(L.vd / kKvBlock) << c.page_shift) + off);
  }
}

template <int SEL>
__device__ __forceinline__ uint32_t two_values(uint32_t w, float scale) {
  return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(w, scale, SEL));
}

// Elements 2 B, 2 B + 1 of eight tokens as two operands of eight bf16 values each
template <int B>
__device__ __forceinline__ void two_operands(const uint32_t (&w)[8], const float (&scale)[8], bf16x8& even, bf16x8& odd) {
  u32x4 e, o;
#pragma unroll
  for (int u = 0; u < 4; ++u) {
    const uint32_t a = two_values<B>(w[2 * u], scale[2 * u]), b = two_values<B>(w[2 * u + 1], scale[2 * u + 1]);
    e[u] = __builtin_amdgcn_perm(b, a, 0x05040100u);
    o[u] = __builtin_amdgcn_perm(b, a, 0x07060302u);
  }
  even = __builtin_bit_cast(bf16x8, e);
  odd = __builtin_bit_cast(bf16x8, o);
}

template <int DPL>
__device__ __forceinline__ uint32_t word_of(const typename VWord<DPL>::type& v, int i) {
  if constexpr (DPL == 16) return v[i];
  else return v;
}

// Queries as the first operand of the scores, in QT bf16 terms: one is a bf16 query itself, three leave 2^-24 of an fp32 element.
// Keys are converted to bf16 (exact).  The matrix unit would take them as they are held, against 8-bit terms of the
// queries, at the same rate; but its sums of 8-bit products keep only 2^-17 of their terms at worst (7e-7 on the average), these 2^-23.
template <int QT, int DC>
struct Query {
  bf16x8 q[DC][QT][4];
  template <class X>
  __device__ __forceinline__ void load(const typename X::storage* row, int D, bool real, bool wide, int g) {
#pragma unroll
    for (int x = 0; x < DC; ++x)
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const int d = 128 * x + 32 * g + 16 * h;
        float e[16];
        load_q16<X>(row, d, real && d < D, wide, e);
#pragma unroll
        for (int t = 0; t < QT; ++t)
#pragma unroll
          for (int i = 0; i < 16; ++i) {
            const __bf16 v = (__bf16)e[i];
            q[x][t][2 * h + i / 8][i % 8] = v;
            if (t + 1 < QT) e[i] -= (float)v;
          }
      }
  }
  // s[j] += scores of tokens 4 c + j over the x-th 128 elements
  __device__ __forceinline__ void times(int x, const u32x4 (&k)[4], uint32_t ks, f32x4 (&s)[4]) const {
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const float sc = scale_value((ks >> (8 * j)) & 255u);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const u32x4 w = {two_values<0>(k[j][i], sc), two_values<1>(k[j][i], sc), two_values<2>(k[j][i], sc), two_values<3>(k[j][i], sc)};
#pragma unroll
        for (int t = 0; t < QT; ++t) s[j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(q[x][t][i], __builtin_bit_cast(bf16x8, w), s[j], 0, 0, 0);
      }
    }
  }
};

// One launch for every cut of the work: a workgroup takes an equal share of the units, whichever tiles they belong to.
template <class X, int NR, int DPL>
__global__ __launch_bounds__(kThreads, DPL == 16 ? 1 : 2) void few_kernel(Few f) {
  constexpr bool F = sizeof(typename X::storage) == 4;
  constexpr int QT = F ? 3 : 1, PT = F ? 3 : 1, DC = Step<DPL>::DC, TR = 4 * NR;
  __shared__ int64_t scan[8];
  __shared__ alignas(16) uint16_t weights[kWaves][PT][kRows][kPStride];
  __shared__ alignas(16) float sums[2][4 * NR][16 * DPL];
  __shared__ float stats[kWaves][2][4 * NR];
  const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave;
  const KvAttend& a = f.a;
  const int D = a.c.dim;
  const Lane<DPL> L(D);

  // tokens of no request
  {
    const int64_t t0 = !a.q_start ? a.T : a.B > 0 ? min(max(a.q_start[a.B], 0), (int)a.T) : 0;
    typename X::storage* const O = reinterpret_cast<typename X::storage*>(a.O);
    const int64_t row = (int64_t)a.heads * D, me = (int64_t)blockIdx.x * kThreads + threadIdx.x, all = (int64_t)gridDim.x * kThreads;
    for (int64_t i = t0 * row + me; i < a.T * row; i += all) X::store(O, i, 0.f);
    if (a.lse)
      for (int64_t i = t0 * a.heads + me; i < a.T * a.heads; i += all) a.lse[i] = -INFINITY;
  }

  const int64_t total = total_units(f, scan);
  const int64_t W = min((int64_t)gridDim.x, total), w = blockIdx.x;  // every workgroup that takes part has a unit
  if (threadIdx.x == 0) f.heads[4 * w] = -1;
  if (w >= W) return;
  int64_t u = total * w / W;
  const int64_t u_end = total * (w + 1) / W;
  Place at = place_of_unit(f, u, scan);
  int b = at.b;
  int64_t before = at.before;

  for (int i = threadIdx.x; i < kWaves * PT * kRows * kPStride / 2; i += kThreads) reinterpret_cast<uint32_t*>(weights)[i] = 0;
  __syncthreads();

  const float zscale = a.scale * kLog2e;
  while (u < u_end) {
    Span sp = span_of(a, b);
    int per, tiles;
    int64_t mine = units_of(f, sp, per, tiles);
    while (u >= before + mine) {  // the next request with rows
      before += mine;
      ++b;
      sp = span_of(a, b);
      mine = units_of(f, sp, per, tiles);
    }
    const int seg = (int)((u - before) / per), first = (int)(u - before - (int64_t)seg * per);
    const int64_t seg_begin = before + (int64_t)seg * per, seg_end = seg_begin + per;
    const int last = (int)(min(u_end, seg_end) - seg_begin);
    const int kvh = seg % a.c.heads, tile = seg / a.c.heads;
    const int rows = min(TR, sp.n * f.group - tile * TR);

    // row r of the tile is row 4 (r % 4) + r / 4 of the products: up to four rows lie in one accumulator register of the four lane groups
    Query<QT, DC> q;
    {
      const int r = (L.c >> 2) + 4 * (L.c & 3), rid = tile * TR + r;
      const bool real = r < rows;
      const int tok = real ? rid / f.group : 0, head = kvh * f.group + (real ? rid % f.group : 0);
      q.template load<X>(reinterpret_cast<const typename X::storage*>(a.Q) + (int64_t)(sp.t0 + tok) * a.q_stride + (int64_t)head * D, D, real, f.q_wide, L.g);
    }
    // the last key that a row sees: rows r = g + 4 i of this lane
    int lim[NR];
    int lim_low = sp.len - 1;
#pragma unroll
    for (int i = 0; i < NR; ++i) {
      const int r = L.g + 4 * i, tok = (tile * TR + r) / f.group;
      lim[i] = r < rows ? sp.len - sp.n + tok : -1;
    }
    lim_low = sp.len - sp.n + (tile * TR) / f.group;  // what every row of the tile sees

    f32x4 o[DPL];
    float m[NR], l[NR];
#pragma unroll
    for (int j = 0; j < DPL; ++j) o[j] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int i = 0; i < NR; ++i) {
      m[i] = -INFINITY;
      l[i] = 0.f;
    }

    const int32_t* const trow = a.table + (int64_t)b * a.width;
    const int key_end = min(sp.len, last * kUnit);
    int key = first * kUnit + wave * kStep;
    Step<DPL> cur, nxt;
    Pages pc, pn;
    if (key < key_end) {
      pc = load_pages<DPL>(trow, a.width, a.c.page_shift, L, key);
      pn = load_pages<DPL>(trow, a.width, a.c.page_shift, L, key + kUnit);
      load_step<DPL>(cur, a.c, kvh, pc, L, key);
    }
    while (key < key_end) {
      const bool more = key + kUnit < key_end;
      Pages p2 = pn;
      if (more) {
        load_step<DPL>(nxt, a.c, kvh, pn, L, key + kUnit);
        p2 = load_pages<DPL>(trow, a.width, a.c.page_shift, L, key + 2 * kUnit);
      }
      // scores: rows by tokens 4 c + j
      f32x4 s[4];
#pragma unroll
      for (int j = 0; j < 4; ++j) s[j] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int x = 0; x < DC; ++x) q.times(x, cur.k[x], L.kreal[x] ? cur.ks[x] : 0x7f7f7f7fu, s);  // (queries are zero past the head's end)
      float z[NR][4];
#pragma unroll
      for (int i = 0; i < NR; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) z[i][j] = s[j][i] * zscale;
      const uint32_t np = (uint32_t)a.c.n_pages;
      const bool k_there = (uint32_t)pc.k < np;
      bool v_there[2];
#pragma unroll
      for (int h = 0; h < 2; ++h) v_there[h] = (uint32_t)pc.v[h] < np;
      if (key + kStep - 1 > lim_low || __any(!k_there || !v_there[0] || !v_there[1])) {
        // the end of the keys, keys that only some rows see, or pages that are not there
        int bad = 0x7fffffff;
#pragma unroll
        for (int i = 0; i < NR; ++i)
#pragma unroll
          for (int j = 0; j < 4; ++j) z[i][j] = k_there && key + 4 * L.c + j <= lim[i] ? z[i][j] : -INFINITY;
#pragma unroll
        for (int h = 0; h < 2; ++h)
#pragma unroll
          for (int x = 0; x < 8; ++x) {
            // a value that no row sees, or that is NaN, does not enter the product: 0 times it would not be 0
            const int k = key + 32 * h + 8 * L.g + x, sh = 8 * (x & 3);
            const bool seen = v_there[h] && k < sp.len, nan = ((cur.vs[h][x / 4] >> sh) & 255u) == 255u;
            if (seen && nan) bad = min(bad, k);
            if (!seen || nan) {
              cur.v[h][x] = typename VWord<DPL>::type{};
              cur.vs[h][x / 4] = (cur.vs[h][x / 4] & ~(255u << sh)) | (127u << sh);
            }
          }
        // ... it goes to the rows that see it, in the elements of its block
        bad = min(bad, __shfl_xor(bad, 16, kWave));
        bad = min(bad, __shfl_xor(bad, 32, kWave));
#pragma unroll
        for (int i = 0; i < NR; ++i)
          if (bad <= lim[i]) {
#pragma unroll
            for (int j = 0; j < DPL; ++j) o[j][i] = NAN;
          }
      }
      // the maximum
      bool moves = false;
#pragma unroll
      for (int i = 0; i < NR; ++i) moves |= fmaxf(fmaxf(z[i][0], z[i][1]), fmaxf(z[i][2], z[i][3])) > m[i] + kSlack;
      if (__any(moves)) {
#pragma unroll
        for (int i = 0; i < NR; ++i) {
          const float top = row16_max(fmaxf(fmaxf(z[i][0], z[i][1]), fmaxf(z[i][2], z[i][3])));
          const float next = fmaxf(m[i], top);
          const float keep = next == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(m[i] - next);
          m[i] = next;
          l[i] *= keep;
#pragma unroll
          for (int j = 0; j < DPL; ++j) o[j][i] *= keep;
        }
      }
      // weights, through LDS into the layout of the second product
#pragma unroll
      for (int i = 0; i < NR; ++i) {
        const float base = m[i] == -INFINITY ? 0.f : m[i];
        float p[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          p[j] = __builtin_amdgcn_exp2f(z[i][j] - base);
          l[i] += p[j];
        }
#pragma unroll
        for (int t = 0; t < PT; ++t) {
          u32x2 pk;
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            const bf16x2 v = {(__bf16)p[2 * h], (__bf16)p[2 * h + 1]};
            pk[h] = __builtin_bit_cast(uint32_t, v);
            if (t + 1 < PT) {
              p[2 * h] -= bf16_lo(pk[h]);
              p[2 * h + 1] -= bf16_hi(pk[h]);
            }
          }
          *reinterpret_cast<u32x2*>(&weights[wave][t][4 * L.g + i][4 * L.c]) = pk;
        }
      }
      order_lds();
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        bf16x8 pa[PT];
#pragma unroll
        for (int t = 0; t < PT; ++t) pa[t] = *reinterpret_cast<const bf16x8*>(&weights[wave][t][L.c][32 * h + 8 * L.g]);
        float vsc[8];
#pragma unroll
        for (int x = 0; x < 8; ++x) vsc[x] = scale_value((cur.vs[h][x / 4] >> (8 * (x & 3))) & 255u);
#pragma unroll
        for (int i = 0; i < (DPL + 7) / 8; ++i) {
          uint32_t word[8];
#pragma unroll
          for (int x = 0; x < 8; ++x) word[x] = word_of<DPL>(cur.v[h][x], i);
#define GSI_VALUES(B)                                                                                          \
  {                                                                                                            \
    bf16x8 even, odd;                                                                                          \
    two_operands<B>(word, vsc, even, odd);                                                                     \
    _Pragma("unroll") for (int t = 0; t < PT; ++t) {                                                           \
      o[8 * i + 2 * B] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(pa[t], even, o[8 * i + 2 * B], 0, 0, 0);      \
      o[8 * i + 2 * B + 1] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(pa[t], odd, o[8 * i + 2 * B + 1], 0, 0, 0); \
    }                                                                                                          \
  }
          GSI_VALUES(0)
          GSI_VALUES(1)
          if constexpr (DPL >= 8) {
            GSI_VALUES(2)
            GSI_VALUES(3)
          }
#undef GSI_VALUES
        }
      }
      order_lds();
      cur = nxt;
      pc = pn;
      pn = p2;
      key += kUnit;
    }

    // the four waves' sums, in a fixed order: 2 onto 0 and 3 onto 1, then 1 onto 0
    float scale_o[NR], top[NR], sum[NR];
#pragma unroll
    for (int i = 0; i < NR; ++i) {
      l[i] = row16_sum(l[i]);
      if (L.c == 0) {
        stats[wave][0][4 * i + L.g] = m[i];
        stats[wave][1][4 * i + L.g] = l[i];
      }
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < NR; ++i) {
      const int r = 4 * i + L.g;
      top[i] = -INFINITY;
      sum[i] = 0.f;
#pragma unroll
      for (int v = 0; v < kWaves; ++v) top[i] = fmaxf(top[i], stats[v][0][r]);
#pragma unroll
      for (int v = 0; v < kWaves; ++v) {
        const float mv = stats[v][0][r];
        sum[i] += stats[v][1][r] * (mv == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(mv - top[i]));  // (sums of such a wave: 0, or NaN)
      }
      scale_o[i] = m[i] == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(m[i] - top[i]);
    }
#pragma unroll
    for (int j = 0; j < DPL; ++j)
#pragma unroll
      for (int i = 0; i < NR; ++i) o[j][i] *= scale_o[i];
    const auto put = [&](int slot) {
#pragma unroll
      for (int i = 0; i < NR; ++i)
#pragma unroll
        for (int j = 0; j < DPL; j += 4)
          *reinterpret_cast<f32x4*>(&sums[slot][4 * i + L.g][DPL * L.c + j]) = f32x4{o[j][i], o[j + 1][i], o[j + 2][i], o[j + 3][i]};
    };
    const auto add = [&](int slot) {
#pragma unroll
      for (int i = 0; i < NR; ++i)
#pragma unroll
        for (int j = 0; j < DPL; j += 4) {
          const f32x4 v = *reinterpret_cast<const f32x4*>(&sums[slot][4 * i + L.g][DPL * L.c + j]);
#pragma unroll
          for (int e = 0; e < 4; ++e) o[j + e][i] += v[e];
        }
    };
    if (wave >= 2) put(wave - 2);
    __syncthreads();
    if (wave < 2) add(wave);
    if (wave == 1) put(1);
    __syncthreads();
    if (wave == 0) {
      add(1);
      const bool whole = first == 0 && last == per;
      float* part = nullptr;
      if (!whole) {
        // the first tile of a workgroup, if another began it: slot 2 w; else the tile is cut at this workgroup's end
        const int64_t slot = first != 0 ? 2 * w : 2 * w + 1;
        part = f.parts + slot * TR * (D + 2);
        if (first == 0 && lane == 0) {
          // the workgroup with unit seg_end - 1: the largest v with total * v / W <= seg_end - 1
          int64_t v = (seg_end * W - 1) / total;
          while (total * (v + 1) / W <= seg_end - 1) ++v;
          while (total * v / W > seg_end - 1) --v;
          f.heads[4 * w + 1] = tile;
          f.heads[4 * w + 2] = kvh;
          f.heads[4 * w + 3] = (int)v;
          f.heads[4 * w] = b;
        }
      }
#pragma unroll
      for (int i = 0; i < NR; ++i) {
        const int r = 4 * i + L.g;
        if (r >= rows) continue;
        const int rid = tile * TR + r;
        const int64_t orow = (int64_t)(sp.t0 + rid / f.group) * a.heads + kvh * f.group + rid % f.group;
        if (whole) {
          const float inv = sum[i] == 0.f ? 0.f : 1.f / sum[i];
          typename X::storage* const out = reinterpret_cast<typename X::storage*>(a.O) + orow * D + DPL * L.c;
          if (DPL * L.c < D)
#pragma unroll
            for (int j = 0; j < DPL; j += 4) {
              if constexpr (F) {
                *reinterpret_cast<f32x4*>(out + j) = f32x4{o[j][i] * inv, o[j + 1][i] * inv, o[j + 2][i] * inv, o[j + 3][i] * inv};
              } else {
                const bf16x2 lo = {(__bf16)(o[j][i] * inv), (__bf16)(o[j + 1][i] * inv)}, hi = {(__bf16)(o[j + 2][i] * inv), (__bf16)(o[j + 3][i] * inv)};
                *reinterpret_cast<u32x2*>(out + j) = u32x2{__builtin_bit_cast(uint32_t, lo), __builtin_bit_cast(uint32_t, hi)};
              }
            }
          if (a.lse && L.c == 0) a.lse[orow] = sum[i] == 0.f ? -INFINITY : (top[i] == -INFINITY ? sum[i] : (top[i] + log2f(sum[i])) * kLn2);
        } else {
          float* const row = part + r * (D + 2);
          if (DPL * L.c < D)
#pragma unroll
            for (int j = 0; j < DPL; j += 2) *reinterpret_cast<f32x2*>(row + DPL * L.c + j) = f32x2{o[j][i], o[j + 1][i]};
          if (L.c == 0) {
            row[D] = top[i];
            row[D + 1] = sum[i];
          }
        }
      }
    }
    u = min(u_end, seg_end);
    __syncthreads();  // stats and sums are read before the next tile writes them
  }
}

// Joins the parts of the tiles that a cut went through: a workgroup per possible cut and row, in the order of the parts.
template <class X>
__global__ __launch_bounds__(kKvMaxDim) void join_kernel(Few f) {
  const KvAttend& a = f.a;
  const int w = blockIdx.x, r = blockIdx.y, D = a.c.dim;
  const int b = f.heads[4 * w];
  if (b < 0) return;
  const int tile = f.heads[4 * w + 1], kvh = f.heads[4 * w + 2], end = f.heads[4 * w + 3];
  const Span sp = span_of(a, b);
  const int rid = tile * f.tile_rows + r;
  if (rid >= sp.n * f.group) return;
  const auto part = [&](int i) { return f.parts + (int64_t)(i == w ? 2 * w + 1 : 2 * i) * f.tile_rows * (D + 2) + r * (D + 2); };
  float top = -INFINITY;
  for (int i = w; i <= end; ++i) top = fmaxf(top, part(i)[D]);
  const int d = threadIdx.x;
  float sum = 0.f, o = 0.f;
  for (int i = w; i <= end; ++i) {
    const float* const p = part(i);
    const float mv = p[D], k = mv == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(mv - top);
    sum += p[D + 1] * k;
    if (d < D) o += p[d] * k;
  }
  const int64_t orow = (int64_t)(sp.t0 + rid / f.group) * a.heads + kvh * f.group + rid % f.group;
  if (d < D) X::store(reinterpret_cast<typename X::storage*>(a.O), orow * D + d, sum == 0.f ? 0.f : o / sum);
  if (a.lse && d == 0) a.lse[orow] = sum == 0.f ? -INFINITY : (top == -INFINITY ? sum : (top + log2f(sum)) * kLn2);
}

// The smallest tile that holds the rows of the longest request that is expected.
int few_tile(const KvAttend& a, int64_t few) {
  const int64_t rows = std::min(std::min(a.max_q, a.T) * (a.heads / a.c.heads), few);
  return rows <= 4 ? 4 : rows <= 8 ? 8 : 16;
}
int few_workgroups(const KvAttend& a, int tile_rows) {
  const int64_t tiles = ceil_div(std::min(a.max_q, a.T) * (a.heads / a.c.heads), tile_rows);
  const double units = (double)a.B * tiles * a.c.heads * (double)ceil_div(a.max_len, kUnit);
  return (int)std::max(1.0, std::min(units, 768.0));
}

template <class X, int NR>
void launch_few(const Few& f, int W, hipStream_t s) {
  const int D = f.a.c.dim;
  if (D <= 64) few_kernel<X, NR, 4><<<W, kThreads, 0, s>>>(f);
  else if (D <= 128) few_kernel<X, NR, 8><<<W, kThreads, 0, s>>>(f);
  else few_kernel<X, NR, 16><<<W, kThreads, 0, s>>>(f);
}
template <class X>
void launch_few(const Few& f, int W, hipStream_t s) {
  if (f.tile_rows == 4) launch_few<X, 1>(f, W, s);
  else if (f.tile_rows == 8) launch_few<X, 2>(f, W, s);
  else launch_few<X, 4>(f, W, s);
  join_kernel<X><<<dim3(W, f.tile_rows), kKvMaxDim, 0, s>>>(f);
}

}  // namespace

size_t attend_few_workspace(const KvAttend& a, int64_t few) {
  const int tile = few_tile(a, few);
  const size_t W = (size_t)few_workgroups(a, tile);
  return align_up(W * 16, 256) + align_up(2 * W * tile * (a.c.dim + 2) * sizeof(float), 256);
}

hipError_t attend_few(const KvAttend& a, int64_t few, void* ws, hipStream_t s) {
  Few f{};
  f.a = a;
  f.few = few;
  f.group = a.heads / a.c.heads;
  f.tile_rows = few_tile(a, few);
  const size_t es = elem_size(a.dtype);
  f.q_wide = reinterpret_cast<uintptr_t>(a.Q) % 16 == 0 && (size_t)a.q_stride * es % 16 == 0;
  const int W = few_workgroups(a, f.tile_rows);
  f.heads = reinterpret_cast<int*>(ws);
  f.parts = reinterpret_cast<float*>(static_cast<char*>(ws) + align_up((size_t)W * 16, 256));
  if (a.dtype == GSI_BF16) launch_few<BF16>(f, W, s);
  else launch_few<F32>(f, W, s);
  return hipGetLastError();
}

// Which kernels a call takes.  Requests of at most kFewRows rows of a head of keys are cheaper where a workgroup has 16 rows; where no
// request is expected to have more, those take all of them, and where the requests are about of one length, or few rows are
// not expected at all, the others do.
constexpr int64_t kFewRows = 32;
enum Kernels { kFewOnly, kPromptOnly, kBoth };
static Kernels kernels_of(const KvAttend& a) {
  const int64_t most = std::min(a.max_q, a.T);
  if (most * (a.heads / a.c.heads) <= kFewRows || a.B == 0) return kFewOnly;
  return 2 * a.T >= a.B * most ? kPromptOnly : kBoth;
}

size_t kv_attention_workspace(const KvAttend& a) {
  switch (kernels_of(a)) {
    case kFewOnly: return attend_few_workspace(a, INT64_MAX);
    case kPromptOnly: return attend_prompt_workspace(a);
    default: return attend_few_workspace(a, kFewRows) + attend_prompt_workspace(a);
  }
}

hipError_t kv_attention(const KvAttend& a, void* ws, hipStream_t s) {
  switch (kernels_of(a)) {
    case kFewOnly: return attend_few(a, INT64_MAX, ws, s);
    case kPromptOnly: return attend_prompt(a, 0, true, ws, s);
    default: break;
  }
  if (hipError_t e = attend_few(a, kFewRows, ws, s); e != hipSuccess) return e;
  return attend_prompt(a, kFewRows, false, static_cast<char*>(ws) + attend_few_workspace(a, kFewRows), s);
}

}  // namespace gsi
