// Attention over the paged cache in 4 bits, few rows: single tokens, and a few tokens of a request.
//
// For a row (a token and a head) with query q: s_j = scale q.k_j over the keys that it sees, o = sum_j 2^(s_j' - m) v_j / sum_j 2^(s_j' - m),
// s' = s log2 e, m a running maximum.  A wave takes up to 16 rows that share a head of keys and 64 keys a step.  Both products are
// bf16 matrix products of codes times scales (exact in bf16), and neither operand is transposed: a lane loads 16, 32 or 64 consecutive
// codes of a key, its operands of products over 8 elements each, and 4, 8 or 16 elements of 16 consecutive values.  A pair
// of those as it is converted, two elements of one token, is a pair of the contraction: the weights of a row are given twice,
// once with zeros against the odd elements and once with zeros against the even ones, as two rows of the product.
//
// Memory bounds it where contexts are long: every code and scale is read once, by eight waves a unit that request a step's keys and values while they
// work on the step before.  8 contexts of 131000 keys x 8 heads x 128 are read at 5.3 TB/s, two of 60000 and 131000 (208 MB) at 4.6 in 45.5 us, 64
// fp32 tokens x 32 heads over 287 MB at 4.4 in 64 us (streaming reads reach 6.5 TB/s); 5 to 8 us of join_kernel come on top.  In those the matrix units are busy
// for 11 % of the time, and the conversions of codes, exponentials and sums take about half of the issue slots of a SIMD's two waves.  Short
// contexts are bound by the chain of loads in front of the first product: one token of 12 heads over 210 keys 8.4 us.
#include <algorithm>

#include "gsi_attend.h"

namespace gsi {
namespace {

constexpr int kWaves = 4, kThreads = kWaves * kWave;
constexpr int kStep = 64;             // keys of a wave and step: the unit in which the work is dealt out
constexpr int kPStride = kStep + 4;   // bf16 weights of a row in LDS
// Parts of a tile that one wave joins by itself: two contexts of 60000 and 131000 keys x 8 heads x 128, whose tiles have about 100 parts, take 55 us
// with the four waves of a workgroup at them, 61 without; tiles of two or three parts do as well by single waves.
constexpr int kManyParts = 12;

struct Few {
  KvAttend a;
  int64_t few;    // requests of more rows are another kernel's
  int group;      // heads that share a head of keys
  int tile_rows;  // rows of a tile
  Divisor by_group, by_heads, by_tile;  // by the heads of a group, the heads of keys, the rows of a tile
  int q_wide;     // 16-byte loads of queries
  int whole;      // a workgroup takes whole tiles, its waves parts of their keys; else every wave an equal share of all steps
  float* parts;   // [2 * waves][tile_rows][dim]: sums of a cut tile
  float2* stats;  // [2 * waves][tile_rows]: their maxima and sums of weights; a maximum of NaN: no part (another wave's place has it)
  int* cuts;      // [waves][4]: the tile that a wave begins and does not end, and the wave that ends it
};

// Tiles of a request and the steps of each (one where there are rows but no keys).  A tile counts as kTileCost units and one for every step: its
// queries, first loads and output cost a wave about as much as so many steps (64 fp32 tokens x 32 heads over 287 MB: 70 us; counted as none 86, as
// four 71; the other calls here lie within 3 % of their best with two).
constexpr int kTileCost = 2;
struct Steps {
  int tiles, per_tile;
};
__device__ __forceinline__ Steps steps_of(const Few& f, const Span& s) {
  const int64_t rows = (int64_t)s.n * f.group;
  return Steps{rows <= f.few ? f.by_tile((int)rows + f.tile_rows - 1) : 0, max(1, (s.len + kStep - 1) / kStep)};
}
__device__ __forceinline__ int tile_units(const Few& f, const Steps& st) { return f.whole ? 1 : st.per_tile + kTileCost; }

// Wave i of the launch takes the units [first_unit(i), first_unit(i + 1)): a quarter of its workgroup's.  No wave before the last that has any is
// without one.
__device__ __forceinline__ int64_t first_unit(const Shares& s, int64_t i) {
  const int64_t g = i / kWaves, k = i % kWaves;
  if (s.total < kWaves) return min(i, s.total);
  return s.of_group(g) + s.units_of_group(g) * k / kWaves;
}
__device__ __forceinline__ int64_t owner(const Shares& s, int64_t u) {  // the wave that has unit u
  int64_t i = (s.total < kWaves ? 0 : s.group_of(u)) * kWaves + kWaves - 1;
  while (first_unit(s, i) > u) --i;
  return i;
}

// ---- operands -------------------------------------------------------------------------------------------------
template <int DPL>
struct VWord;  // the codes of a lane's DPL elements of a value
template <> struct VWord<4> { using type = uint16_t; };
template <> struct VWord<8> { using type = uint32_t; };
template <> struct VWord<16> { using type = u32x2; };
template <int DPL>
__device__ __forceinline__ uint32_t word_of(const typename VWord<DPL>::type& v, int i) {
  if constexpr (DPL == 16) return v[i];
  else return v;
}

// Lane (c, g) of a wave: of a key, the 8 KW elements from 8 KW g on, of token 4 c + j; of a value, the DPL elements from DPL c on, of the tokens 16 g ..
template <int DPL>
struct Lane {
  static constexpr int KW = DPL / 2, KB = KW == 8 ? 2 : 1;  // words of a key; blocks that they lie in
  int c, g;
  int kd[KB];  // first element of its block's part (in range: what lies past the head's end meets queries of zero)
  bool kin[KB];
  int vd;      // first element of its values (in range: such columns are not stored)
  __device__ __forceinline__ Lane(int dim) {
    const int lane = threadIdx.x % kWave;
    c = lane % 16;
    g = lane / 16;
#pragma unroll
    for (int x = 0; x < KB; ++x) {
      const int d = 8 * KW * g + kKvBlock * x;
      kin[x] = d < dim;
      kd[x] = kin[x] ? d : 0;
    }
    vd = c * DPL < dim ? c * DPL : 0;
  }
};

template <int DPL>
struct Keys {
  uint32_t w[4][Lane<DPL>::KW];
  uint32_t scale[Lane<DPL>::KB];  // of the four tokens, a byte each
};
template <int DPL>
struct Values {
  typename VWord<DPL>::type w[16];
  u32x4 scale;
};

// a request's row of the table, and the head's rows in page 0 with the bytes from page to page (below 2^32: 4096 heads of 128 bytes, 4096 tokens)
struct Where {
  const int32_t* row;
  const uint8_t *K, *Ks, *V, *Vs;
  uint32_t code_stride, scale_stride;
};
__device__ __forceinline__ int page_of(const KvAttend& a, const Where& at, int key) {
  return at.row[min(key >> a.c.page_shift, (int)a.width - 1)];  // (entries past the row's end: no key lies there)
}
__device__ __forceinline__ bool is_page(const KvAttend& a, int page) { return (uint32_t)page < (uint32_t)a.c.n_pages; }

template <int DPL>
__device__ __forceinline__ void load_keys(Keys<DPL>& k, const KvAttend& a, const Where& at, int page, const Lane<DPL>& L, int key, int half) {
  const KvView& c = a.c;
  const uint32_t p = is_page(a, page) ? page : 0;  // another page's keys: they are not seen
  const int off = (key + 4 * L.c) & (c.page() - 1);
  const uint8_t* const codes = at.K + (uint64_t)p * at.code_stride + off * half;
  const uint8_t* const scales = at.Ks + (uint64_t)p * at.scale_stride + off;
#pragma unroll
  for (int x = 0; x < Lane<DPL>::KB; ++x) {
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const uint8_t* const from = codes + j * half + L.kd[x] / 2;
      if constexpr (DPL == 4) {
        const u32x2 v = *reinterpret_cast<const u32x2*>(from);
        k.w[j][0] = v[0];
        k.w[j][1] = v[1];
      } else {
        const u32x4 v = *reinterpret_cast<const u32x4*>(from);
#pragma unroll
        for (int i = 0; i < 4; ++i) k.w[j][4 * x + i] = v[i];
      }
    }
    k.scale[x] = *reinterpret_cast<const uint32_t*>(scales + ((L.kd[x] / kKvBlock) << c.page_shift));
  }
}
template <int DPL>
__device__ __forceinline__ void load_values(Values<DPL>& v, const KvAttend& a, const Where& at, int page, const Lane<DPL>& L, int key, int half) {
  const KvView& c = a.c;
  const uint32_t p = is_page(a, page) ? page : 0;
  const int off = (key + 16 * L.g) & (c.page() - 1);
  const uint8_t* const from = at.V + (uint64_t)p * at.code_stride + (off * half + L.vd / 2);
#pragma unroll
  for (int u = 0; u < 16; ++u) v.w[u] = *reinterpret_cast<const typename VWord<DPL>::type*>(from + u * half);
  v.scale = *reinterpret_cast<const u32x4*>(at.Vs + (uint64_t)p * at.scale_stride + (((L.vd / kKvBlock) << c.page_shift) + off));
}

// Rows of the products.  Rows r of a tile lie in lane group r % 4 and register r / 4 of the scores.  FOLD: two rows of fp32, whose three terms (of a
// query, of a weight) are rows of one product instead of three products: row r's terms are the registers of lane group r of the scores,
// which are added, and the registers of lane groups 2 r and 2 r + 1 (even, odd elements) of the output, which are added at the end.  TWO: four rows of
// bf16, whose weights have a second term in the rows of the second product that would be idle: the output is then off by its own rounding alone
// (to 64 bits 0.0017 of it; with one term 0.0024).  More rows of bf16 have one term: a second takes products of its own (8 rows x 256 51 us, with one 49; 16
// rows x 128 84, with one 75).
template <bool F, int NR>
struct Rows {
  static constexpr bool kFold = F && NR == 0;
  static constexpr int kTile = kFold ? 2 : 4 * NR;      // rows of a tile
  static constexpr int kRegs = kFold ? 1 : NR;          // registers of scores
  static constexpr int kChain = F && !kFold ? 3 : 1;    // products that add up terms
  static constexpr bool kTwo = !F && NR == 1;
  static constexpr int kImages = F ? 3 : kTwo ? 2 : 1;  // of the weights in LDS
  static constexpr int kOut = kRegs > 2 ? 2 : 1;        // products that share converted values
  // row of the tile, and term, that row x of the first product has (-1: none)
  __device__ static __forceinline__ int row(int x) { return kFold ? (x / 4 < 2 && x % 4 < 3 ? x / 4 : -1) : (x % 4 < NR ? x / 4 + 4 * (x % 4) : -1); }
  __device__ static __forceinline__ int term(int x) { return kFold ? min(x % 4, 2) : 0; }
};

// Workgroups a unit that the registers leave.  (One where two would spill: 64 requests of 3 tokens behind up to 4000 keys x 256, 8 heads to one of keys,
// bf16 149 us, with two and spills 204; fp32 210, 425.)
__host__ __device__ constexpr int few_resident(bool f32, int tile_rows, int width) {
  if (width > 128 && (tile_rows == 16 || (tile_rows == 8 && f32))) return 1;
  return width > 128 || tile_rows > 4 ? 2 : 3;
}

template <class X, int NR, int DPL, bool EXACT>
__global__ __launch_bounds__(kThreads, few_resident(sizeof(typename X::storage) == 4, 4 * NR, 16 * DPL)) void few_kernel(Few f) {
  constexpr bool F = sizeof(typename X::storage) == 4;
  using R = Rows<F, NR>;
  using Ln = Lane<DPL>;
  constexpr int KW = Ln::KW, KB = Ln::KB, TR = R::kTile, NS = R::kRegs, CH = R::kChain, NO = R::kOut, JP = DPL / 2;
  __shared__ Prefix prefix;
  __shared__ alignas(16) uint16_t weights[kWaves][R::kImages][TR][kPStride];
  __shared__ alignas(16) float sums[2][TR][16 * DPL];
  __shared__ float stats[kWaves][2][TR];
  const int lane = threadIdx.x % kWave, wave = __builtin_amdgcn_readfirstlane(threadIdx.x / kWave);
  const KvAttend& a = f.a;
  const int D = EXACT ? 16 * DPL : a.c.dim;
  const Ln L(D);

  // this wave's units
  const int64_t me = (int64_t)blockIdx.x * kWaves + wave;
  if (!f.whole && threadIdx.x < kWaves) f.cuts[4 * (blockIdx.x * kWaves + threadIdx.x)] = -1;
  const auto units = [&](const Span& sp) {
    const Steps st = steps_of(f, sp);
    return (int64_t)st.tiles * a.c.heads * tile_units(f, st);
  };
  const int64_t total = total_units(a, prefix, units);
  if (total == 0) {
    clear_idle_rows<X>(a);
    return;
  }
  Shares sh{};
  int64_t u, u_end;
  if (f.whole) {
    u = blockIdx.x;
    u_end = total;
  } else {
    sh = shares_of(total, gridDim.x, kWaves);
    if (blockIdx.x >= sh.groups) {
      clear_idle_rows<X>(a);
      return;
    }
    u = first_unit(sh, me);
    u_end = first_unit(sh, me + 1);
  }
  const Place place = place_of(a, prefix, total, u, units);
  int b = place.b;
  int64_t before = place.before;
  // whether the workgroup's units are all steps of one tile: its waves' parts are then joined here
  bool together = f.whole;
  if (!f.whole) {
    if (threadIdx.x == 0) {
      const Steps st = steps_of(f, span_at(a, prefix, b));
      const int64_t per = tile_units(f, st), g0 = sh.of_group(blockIdx.x) - before, g1 = sh.of_group(blockIdx.x + 1) - before;
      const int64_t tile = divide(g0, per);
      stats[0][0][0] = total >= kWaves && g0 >= tile * per + (g0 > tile * per ? kTileCost : 0) && g1 <= (tile + 1) * per && g1 - g0 >= kWaves * (kTileCost + 1) ? 1.f : 0.f;
    }
    __syncthreads();
    together = stats[0][0][0] != 0.f;
    __syncthreads();
  }

  const float zscale = exponent_scale(a.scale);
  // row of the output product: the weights' image and row that lane c's row has, and whether it is the one of the odd elements
  int p_row[NO];
  bool p_odd;
  if constexpr (R::kFold) {
    p_row[0] = (min(L.c % 4, 2) * TR + L.c / 8) * kPStride;
    p_odd = (L.c / 4) & 1;
  } else {
#pragma unroll
    for (int y = 0; y < NO; ++y) p_row[y] = R::kTwo ? (L.c % 4 / 2 * TR + L.c / 4) * kPStride : (L.c / 4 + 4 * min(2 * y + (L.c % 4) / 2, NS - 1)) * kPStride;
    p_odd = L.c & 1;
  }
  const uint32_t sel0 = p_odd ? 0x01000c0cu : 0x0c0c0100u, sel1 = p_odd ? 0x03020c0cu : 0x0c0c0302u;
  uint16_t* const my_weights = &weights[wave][0][0][0];
  constexpr int kImage = TR * kPStride;

  while (u < u_end) {
    Span sp = span_at(a, prefix, b);
    Steps st = steps_of(f, sp);
    int per = tile_units(f, st);
    int64_t mine = (int64_t)st.tiles * a.c.heads * per;
    while (u >= before + mine) {  // the next request with rows
      before += mine;
      ++b;
      sp = span_at(a, prefix, b);
      st = steps_of(f, sp);
      per = tile_units(f, st);
      mine = (int64_t)st.tiles * a.c.heads * per;
    }
    sp.t0 = __builtin_amdgcn_readfirstlane(sp.t0);
    sp.n = __builtin_amdgcn_readfirstlane(sp.n);
    sp.len = __builtin_amdgcn_readfirstlane(sp.len);
    sp.past = __builtin_amdgcn_readfirstlane(sp.past);
    const int seg = __builtin_amdgcn_readfirstlane(f.whole ? (int)(u - before) : (int)divide(u - before, per));
    const int64_t seg_begin = before + (int64_t)seg * per;
    const int tile = f.by_heads(seg), kvh = seg - tile * a.c.heads;
    const int rows = min(TR, sp.n * f.group - tile * TR);
    int first, last;  // steps
    if (f.whole) {
      first = st.per_tile * wave / kWaves;
      last = st.per_tile * (wave + 1) / kWaves;
    } else {
      first = max(0, (int)(u - seg_begin) - kTileCost);
      last = (int)(min(u_end, seg_begin + per) - seg_begin) - kTileCost;
      if (last <= 0 && !together) {  // the tile begins with the next wave
        u = u_end;
        break;
      }
    }
    first = __builtin_amdgcn_readfirstlane(first);
    last = __builtin_amdgcn_readfirstlane(last);

    const int64_t code0 = a.c.code_at(0, kvh), scale0 = a.c.scale_at(0, kvh);
    const Where at{a.table + (int64_t)b * a.width, a.c.K + code0, a.c.Ks + scale0, a.c.V + code0, a.c.Vs + scale0,
                   (uint32_t)a.c.code_at(1, 0), (uint32_t)a.c.scale_at(1, 0)};
    // query rows are requested first: they are converted while keys and values are on their way
    QueryPart<X, 16> raw[KW / 2];
    {
      const int r = R::row(L.c), rid = tile * TR + r;
      const bool real = r >= 0 && r < rows;
      const int tok = real ? f.by_group(rid) : 0, head = kvh * f.group + (real ? rid - tok * f.group : 0);
      const typename X::storage* const Q = reinterpret_cast<const typename X::storage*>(a.Q) + (int64_t)(sp.t0 + tok) * a.q_stride + (int64_t)head * D;
#pragma unroll
      for (int x = 0; x < KW / 2; ++x) {
        const int d = 8 * KW * L.g + 16 * x;
        raw[x].load(Q, d, real && d < D, f.q_wide, a.scale < 0.f);
      }
    }
    const int key_end = min(sp.len, last * kStep);
    int key = first * kStep;
    Keys<DPL> K;
    Values<DPL> V;
    int pk = 0, pv = 0, pk1 = 0, pv1 = 0;  // page ids of the lane's keys and values: of this step and the next
    if (key < key_end) {
      pk = page_of(a, at, key + 4 * L.c);
      pv = page_of(a, at, key + 16 * L.g);
      pk1 = page_of(a, at, key + kStep + 4 * L.c);
      pv1 = page_of(a, at, key + kStep + 16 * L.g);
      load_keys<DPL>(K, a, at, pk, L, key, D / 2);
      load_values<DPL>(V, a, at, pv, L, key, D / 2);
    }

    bf16x8 q[KW][CH];
#pragma unroll
    for (int x = 0; x < KW; ++x) {
      if constexpr (R::kFold) {
        bf16x8 all[3];
        raw[x / 2].template terms<3>(x % 2, all);
        const int t = R::term(L.c);
        q[x][0] = t == 0 ? all[0] : t == 1 ? all[1] : all[2];
      } else {
        raw[x / 2].template terms<CH>(x % 2, q[x]);
      }
#pragma unroll
      for (int t = 0; t < CH; ++t) arrive(q[x][t]);
    }
    // the last key that a row sees: by the layout of the scores, and of the output (the same but where terms are folded)
    int lim[NS], lim_o[NS];
    const auto last_key = [&](int r) { return r < rows ? sp.last_key(f.by_group(tile * TR + r)) : -1; };
#pragma unroll
    for (int i = 0; i < NS; ++i) {
      lim[i] = last_key(L.g + 4 * i);
      lim_o[i] = R::kFold ? last_key(L.g / 2) : lim[i];
    }
    const int lim_low = sp.last_key(f.by_group(tile * TR));  // what every row of the tile sees

    f32x4 o[NO][JP];
    float m[NS], l[NS];
#pragma unroll
    for (int y = 0; y < NO; ++y)
#pragma unroll
      for (int j = 0; j < JP; ++j) o[y][j] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int i = 0; i < NS; ++i) {
      m[i] = -INFINITY;
      l[i] = 0.f;
    }
    const auto scale_out = [&](const float (&by)[NS]) {  // by: of the lane's rows of scores
      if constexpr (R::kFold || R::kTwo) {
        const float k = R::kFold ? __shfl(by[0], (L.g / 2) * 16 + L.c, kWave) : by[0];
#pragma unroll
        for (int j = 0; j < JP; ++j) o[0][j] *= k;
      } else {
#pragma unroll
        for (int i = 0; i < NS; ++i)
#pragma unroll
          for (int j = 0; j < JP; ++j) {
            o[i / 2][j][2 * (i % 2)] *= by[i];
            o[i / 2][j][2 * (i % 2) + 1] *= by[i];
          }
      }
    };

    while (key < key_end) {
      const bool more = key + kStep < key_end;
      // scores: rows by tokens 4 c + j
      f32x4 s[4];
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        s[j] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int w = 0; w < KW; ++w) {
          const int x = w / 4 < KB ? w / 4 : 0;
          const float sc = L.kin[x] ? scale_value((K.scale[x] >> (8 * j)) & 255u) : 1.f;
          const bf16x8 k = __builtin_bit_cast(bf16x8, eight_values(K.w[j][w], sc));
#pragma unroll
          for (int t = 0; t < CH; ++t) s[j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(q[w][t], k, s[j], 0, 0, 0);
        }
      }
      const bool k_there = is_page(a, pk), v_there = is_page(a, pv);
      if (more) {
        pk = pk1;
        load_keys<DPL>(K, a, at, pk, L, key + kStep, D / 2);
        pk1 = page_of(a, at, key + 2 * kStep + 4 * L.c);
      }
      float z[NS][4];
#pragma unroll
      for (int i = 0; i < NS; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) z[i][j] = R::kFold ? s[j][0] + s[j][1] + s[j][2] : s[j][i];
      if (rarely(key + kStep - 1 > lim_low || __any(!k_there || !v_there))) {
        keep_branch();
        // the end of the keys, keys that only some rows see, or pages that are not there
        int bad = 0x7fffffff;
#pragma unroll
        for (int i = 0; i < NS; ++i)
#pragma unroll
          for (int j = 0; j < 4; ++j) z[i][j] = k_there && key + 4 * L.c + j <= lim[i] ? z[i][j] : -INFINITY;
#pragma unroll
        for (int x = 0; x < 16; ++x) {
          // a value that no row sees, or that is NaN, does not enter the product: 0 times it would not be 0
          const int k = key + 16 * L.g + x, shift = 8 * (x & 3);
          const bool seen = v_there && k < sp.len, nan = ((V.scale[x / 4] >> shift) & 255u) == 255u;
          if (seen && nan) bad = min(bad, k);
          if (!seen || nan) {
            V.w[x] = typename VWord<DPL>::type{};
            V.scale[x / 4] = (V.scale[x / 4] & ~(255u << shift)) | (127u << shift);
          }
        }
        // ... it goes to the rows that see it, in the elements of its block
        bad = min(bad, __shfl_xor(bad, 16, kWave));
        bad = min(bad, __shfl_xor(bad, 32, kWave));
#pragma unroll
        for (int i = 0; i < NS; ++i)
          if (bad <= lim_o[i]) {
#pragma unroll
            for (int j = 0; j < JP; ++j) {
              if constexpr (R::kFold) o[0][j][0] = NAN;
              else o[i / 2][j][2 * (i % 2)] = o[i / 2][j][2 * (i % 2) + 1] = NAN;
            }
          }
      }
      // the maximum
      bool moves = false;
      float top[NS];
#pragma unroll
      for (int i = 0; i < NS; ++i) {
        top[i] = fmaxf(fmaxf(z[i][0], z[i][1]), fmaxf(z[i][2], z[i][3]));
        moves |= top[i] * zscale > m[i] + kSlack;
      }
      if (__any(moves)) {
        float keep[NS];
#pragma unroll
        for (int i = 0; i < NS; ++i) {
          const float next = fmaxf(m[i], row16_max(top[i]) * zscale);
          keep[i] = next == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(m[i] - next);
          m[i] = next;
          l[i] *= keep[i];
        }
        scale_out(keep);
      }
      // weights, through LDS into the layout of the second product
#pragma unroll
      for (int i = 0; i < NS; ++i) {
        const float base = m[i] == -INFINITY ? 0.f : m[i];
        float p[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          p[j] = __builtin_amdgcn_exp2f(fmaf(z[i][j], zscale, -base));
          l[i] += p[j];
        }
#pragma unroll
        for (int t = 0; t < R::kImages; ++t) {
          u32x2 pair;
#pragma unroll
          for (int y = 0; y < 2; ++y) {
            const bf16x2 v = {(__bf16)p[2 * y], (__bf16)p[2 * y + 1]};
            pair[y] = __builtin_bit_cast(uint32_t, v);
            if (t + 1 < R::kImages) {
              p[2 * y] -= bf16_lo(pair[y]);
              p[2 * y + 1] -= bf16_hi(pair[y]);
            }
          }
          if (!R::kFold || L.g < TR) *reinterpret_cast<u32x2*>(my_weights + t * kImage + (L.g + 4 * i) * kPStride + 4 * L.c) = pair;
        }
      }
      order_lds();
#pragma unroll
      for (int y4 = 0; y4 < 4; ++y4) {  // tokens 16 g + 4 y4 ..
        bf16x8 p[NO][CH];
#pragma unroll
        for (int y = 0; y < NO; ++y)
#pragma unroll
          for (int t = 0; t < CH; ++t) {
            const u32x2 w = *reinterpret_cast<const u32x2*>(my_weights + t * kImage + p_row[y] + 16 * L.g + 4 * y4);
            p[y][t] = __builtin_bit_cast(bf16x8, u32x4{__builtin_amdgcn_perm(w[0], w[0], sel0), __builtin_amdgcn_perm(w[0], w[0], sel1),
                                                       __builtin_amdgcn_perm(w[1], w[1], sel0), __builtin_amdgcn_perm(w[1], w[1], sel1)});
          }
        float sc[4];
#pragma unroll
        for (int x = 0; x < 4; ++x) sc[x] = scale_value((V.scale[y4] >> (8 * x)) & 255u);
#pragma unroll
        for (int i = 0; i < (DPL + 7) / 8; ++i) {
          uint32_t w[4];
#pragma unroll
          for (int x = 0; x < 4; ++x) w[x] = word_of<DPL>(V.w[4 * y4 + x], i);
#define GSI_VALUES(B)                                                                                                                   \
  {                                                                                                                                     \
    const bf16x8 v = __builtin_bit_cast(bf16x8, u32x4{two_values<B>(w[0], sc[0]), two_values<B>(w[1], sc[1]), two_values<B>(w[2], sc[2]), \
                                                      two_values<B>(w[3], sc[3])});                                                     \
    _Pragma("unroll") for (int y = 0; y < NO; ++y) _Pragma("unroll") for (int t = 0; t < CH; ++t)                                       \
        o[y][4 * i + B] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(p[y][t], v, o[y][4 * i + B], 0, 0, 0);                                \
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
      if (more) {
        pv = pv1;
        load_values<DPL>(V, a, at, pv, L, key + kStep, D / 2);
        pv1 = page_of(a, at, key + 2 * kStep + 16 * L.g);
      }
      key += kStep;
    }

    // the row's sums: o of element pairs (2 j, 2 j + 1) of the lane's DPL elements, from here on element by element in `out`
    float out[NS][DPL];
#pragma unroll
    for (int i = 0; i < NS; ++i) l[i] = row16_sum(l[i]);
    if constexpr (R::kFold) {
      // even elements lie in lane group 2 r, odd ones in 2 r + 1; lane group r takes both (groups 2 and 3: nothing)
      const int even = (2 * (L.g & 1)) * 16 + L.c;
#pragma unroll
      for (int j = 0; j < JP; ++j) {
        const float x = o[0][j][0] + o[0][j][1] + o[0][j][2];
        out[0][2 * j] = __shfl(x, even, kWave);
        out[0][2 * j + 1] = __shfl(x, even + 16, kWave);
      }
    } else {
#pragma unroll
      for (int i = 0; i < NS; ++i)
#pragma unroll
        for (int j = 0; j < JP; ++j) {
          out[i][2 * j] = R::kTwo ? o[0][j][0] + o[0][j][2] : o[i / 2][j][2 * (i % 2)];
          out[i][2 * j + 1] = R::kTwo ? o[0][j][1] + o[0][j][3] : o[i / 2][j][2 * (i % 2) + 1];
        }
    }
    const bool holds = !R::kFold || L.g < TR;  // lane groups with rows
    if (together) {
      // four waves' sums, in a fixed order: 2 onto 0 and 3 onto 1, then 1 onto 0
      __syncthreads();
      if (holds && L.c == 0) {
#pragma unroll
        for (int i = 0; i < NS; ++i) {
          stats[wave][0][4 * i + L.g] = m[i];
          stats[wave][1][4 * i + L.g] = l[i];
        }
      }
      __syncthreads();
      const auto put = [&](int slot) {
        if (holds) {
#pragma unroll
          for (int i = 0; i < NS; ++i)
#pragma unroll
            for (int j = 0; j < DPL; j += 4)
              *reinterpret_cast<f32x4*>(&sums[slot][4 * i + L.g][DPL * L.c + j]) = f32x4{out[i][j], out[i][j + 1], out[i][j + 2], out[i][j + 3]};
        }
      };
      const auto add = [&](int slot) {
        if (holds) {
#pragma unroll
          for (int i = 0; i < NS; ++i)
#pragma unroll
            for (int j = 0; j < DPL; j += 4) {
              const f32x4 v = *reinterpret_cast<const f32x4*>(&sums[slot][4 * i + L.g][DPL * L.c + j]);
#pragma unroll
              for (int e = 0; e < 4; ++e) out[i][j + e] += v[e];
            }
        }
      };
#pragma unroll
      for (int i = 0; i < NS; ++i) {
        const int r = holds ? 4 * i + L.g : 0;
        float top = -INFINITY, sum = 0.f;
#pragma unroll
        for (int v = 0; v < kWaves; ++v) top = fmaxf(top, stats[v][0][r]);
#pragma unroll
        for (int v = 0; v < kWaves; ++v) {
          const float mv = stats[v][0][r];
          sum += stats[v][1][r] * (mv == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(mv - top));  // (the sum of such a wave: 0, or NaN)
        }
        const float k = m[i] == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(m[i] - top);
#pragma unroll
        for (int j = 0; j < DPL; ++j) out[i][j] *= k;
        m[i] = top;
        l[i] = sum;
      }
      if (wave >= 2) put(wave - 2);
      __syncthreads();
      if (wave < 2) add(wave);
      if (wave == 1) put(1);
      __syncthreads();
      if (wave == 0) add(1);
    }
    if (together && !f.whole && wave != 0 && lane < TR) f.stats[2 * me * TR + lane] = make_float2(NAN, 0.f);
    if (!together || wave == 0) {
      const int64_t to = together && !f.whole ? sh.of_group(blockIdx.x + 1) : u_end;  // where this part ends
      const bool complete = f.whole || (first == 0 && to >= seg_begin + per);
      float* part = nullptr;
      if (!complete) {
        // place 2 i: a tile that an earlier wave began; place 2 i + 1: one that begins here and ends elsewhere
        part = f.parts + (2 * me + (first == 0)) * TR * D;
        if (first == 0 && lane == 0) {
          int* const cut = f.cuts + 4 * me;
          cut[1] = tile;
          cut[2] = kvh;
          cut[3] = (int)owner(sh, seg_begin + per - 1);
          cut[0] = b;
        }
      }
#pragma unroll
      for (int i = 0; i < NS; ++i) {
        const int r = 4 * i + L.g;
        if (!holds || r >= rows) continue;
        const int rid = tile * TR + r;
        const int tok = f.by_group(rid);
        const int64_t orow = (int64_t)(sp.t0 + tok) * a.heads + kvh * f.group + rid - tok * f.group;
        if (complete) {
          const float inv = l[i] == 0.f ? 0.f : 1.f / l[i];
          typename X::storage* const to_o = reinterpret_cast<typename X::storage*>(a.O) + orow * D + DPL * L.c;
          if (DPL * L.c < D)
#pragma unroll
            for (int j = 0; j < DPL; j += 4) {
              if constexpr (F) {
                *reinterpret_cast<f32x4*>(to_o + j) = f32x4{out[i][j] * inv, out[i][j + 1] * inv, out[i][j + 2] * inv, out[i][j + 3] * inv};
              } else {
                const bf16x2 lo = {(__bf16)(out[i][j] * inv), (__bf16)(out[i][j + 1] * inv)}, hi = {(__bf16)(out[i][j + 2] * inv), (__bf16)(out[i][j + 3] * inv)};
                *reinterpret_cast<u32x2*>(to_o + j) = u32x2{__builtin_bit_cast(uint32_t, lo), __builtin_bit_cast(uint32_t, hi)};
              }
            }
          if (a.lse && L.c == 0) a.lse[orow] = l[i] == 0.f ? -INFINITY : (m[i] == -INFINITY ? l[i] : (m[i] + log2f(l[i])) * kLn2);
        } else {
          if (DPL * L.c < D)
#pragma unroll
            for (int j = 0; j < DPL; j += 4)
              *reinterpret_cast<f32x4*>(part + r * D + DPL * L.c + j) = f32x4{out[i][j], out[i][j + 1], out[i][j + 2], out[i][j + 3]};
          if (L.c == 0) f.stats[(2 * me + (first == 0)) * TR + r] = make_float2(m[i], l[i]);
        }
      }
    }
    u = f.whole ? u + gridDim.x : min(u_end, seg_begin + per);
  }
  clear_idle_rows<X>(a);
}

// Joins the parts of the tiles that a cut went through, in their order: a workgroup for the cuts that begin in one of few_kernel's and a row, a wave for
// each of them; one of many parts is taken by the four waves together.  How much each part counts is worked out first, so that the loads
// of the parts themselves wait for nothing.  Latency bounds it: 5 us for tiles of two or three parts, 8 us for 16 of 128 parts.
constexpr int kListed = 512;
template <class X>
__global__ __launch_bounds__(kThreads) void join_kernel(Few f) {
  __shared__ float weight[kWaves][kListed], total[kWaves][kListed];
  __shared__ int place[kWaves][kListed];
  __shared__ float lds[kThreads][5];
  const KvAttend& a = f.a;
  const int D = a.c.dim, lane = threadIdx.x % kWave, wave = threadIdx.x / kWave;
  const int lanes = D <= 64 ? 16 : D <= 128 ? 32 : 64;  // four elements each
  typedef int i32x4 __attribute__((ext_vector_type(4)));
  i32x4 cuts[kWaves];
#pragma unroll
  for (int k = 0; k < kWaves; ++k) cuts[k] = *reinterpret_cast<const i32x4*>(f.cuts + 4 * (blockIdx.x * kWaves + k));
#pragma unroll
  for (int k = 0; k < kWaves; ++k) {
    const int w = blockIdx.x * kWaves + k, b = cuts[k][0];
    if (b < 0) continue;
    const int tile = cuts[k][1], kvh = cuts[k][2], end = cuts[k][3];
    const bool many = end - w >= kManyParts;
    if (!many && wave != k) continue;
    const Span sp = span_of(a, b);
    const int rows = min(f.tile_rows, sp.n * f.group - tile * f.tile_rows);
    const int each = kWave / lanes, ways = many ? each * kWaves : each;     // parts at a time
    const int way = many ? threadIdx.x / lanes : lane / lanes, d = 4 * ((many ? threadIdx.x : lane) % lanes);
    // where wave i's part lies (none where its workgroup's first wave has it for the four)
    const auto slot = [&](int i) { return i == w ? 2 * i + 1 : 2 * i; };
    for (int r = blockIdx.y; r < rows; r += gridDim.y) {
      const auto row_of = [&](int s) { return (int64_t)s * f.tile_rows + r; };
      float top = -INFINITY, sum = 0.f;
      f32x4 o = {0.f, 0.f, 0.f, 0.f};
      // kListed parts at a time; a wave works out the list by itself, the same one in each where four work together
      for (int i0 = w; i0 <= end; i0 += kListed) {
        const int i1 = min(end + 1, i0 + kListed);
        float mine = -INFINITY;
        int n = 0;
        for (int i = i0 + lane; i - lane < i1; i += kWave) {
          const float2 ml = f.stats[row_of(slot(min(i, end)))];
          const float m = ml.x;
          const bool has = i < i1 && m == m;
          const uint64_t ballot = __ballot(has);
          if (has) {
            const int at = n + __popcll(ballot & ((1ull << lane) - 1));
            place[wave][at] = slot(i);
            weight[wave][at] = m;
            total[wave][at] = ml.y;
          }
          n += __popcll(ballot);
          mine = has ? fmaxf(mine, m) : mine;
        }
#pragma unroll
        for (int x = kWave / 2; x; x >>= 1) mine = fmaxf(mine, __shfl_xor(mine, x, kWave));
        const float next = fmaxf(top, mine), keep = next == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(top - next);
        top = next;
        sum *= keep;
        o *= keep;
        order_lds();
#pragma unroll 8
        for (int y = way; y < n; y += ways) {
          const f32x4 v = *reinterpret_cast<const f32x4*>(f.parts + row_of(place[wave][y]) * D + min(d, D - 4));
          const float mv = weight[wave][y], x = mv == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(mv - top);
          sum += total[wave][y] * x;
#pragma unroll
          for (int e = 0; e < 4; ++e) o[e] += v[e] * x;
        }
        order_lds();
      }
      // the ways' sums, in their order
      if (many) {
        float* const mine = lds[threadIdx.x];
        __syncthreads();
#pragma unroll
        for (int e = 0; e < 4; ++e) mine[e] = o[e];
        mine[4] = sum;
        __syncthreads();
        if ((int)threadIdx.x < lanes)
          for (int y = 1; y < ways; ++y) {
            const float* const other = lds[threadIdx.x + y * lanes];
#pragma unroll
            for (int e = 0; e < 4; ++e) o[e] += other[e];
            sum += other[4];
          }
      } else {
        for (int y = lanes; y < kWave; y <<= 1) {
#pragma unroll
          for (int e = 0; e < 4; ++e) o[e] += __shfl_xor(o[e], y, kWave);
          sum += __shfl_xor(sum, y, kWave);
        }
      }
      if ((many ? (int)threadIdx.x : lane) < lanes) {
        const int rid = tile * f.tile_rows + r;
        const int tok = f.by_group(rid);
        const int64_t orow = (int64_t)(sp.t0 + tok) * a.heads + kvh * f.group + rid - tok * f.group;
        const float inv = sum == 0.f ? 0.f : 1.f / sum;
        typename X::storage* const to = reinterpret_cast<typename X::storage*>(a.O) + orow * D + d;
        if (d < D)
#pragma unroll
          for (int e = 0; e < 4; ++e) X::store(to, e, o[e] * inv);
        if (a.lse && d == 0) a.lse[orow] = sum == 0.f ? -INFINITY : (top == -INFINITY ? sum : (top + log2f(sum)) * kLn2);
      }
    }
  }
}

// The smallest tile that holds the rows of the longest request that is expected: 2 (fp32), 4 (bf16), 8 or 16.
// Products and exponentials grow with it: single fp32 tokens of 64 requests x 32 heads, 100 to 4000 keys x 128, in tiles of 2 70 us, of 16 96 us; 3 to 5 bf16
// tokens of 16 requests x 16 heads, up to 6000 keys x 256, in tiles of 8 49 us, of 16 71 us.
int few_tile(const KvAttend& a, int64_t few) {
  const int64_t rows = std::min(std::min(a.max_q, a.T) * (a.heads / a.c.heads), few);
  if (a.dtype == GSI_F32 && rows <= 2) return 2;
  if (a.dtype == GSI_BF16 && rows <= 4) return 4;
  return rows <= 8 ? 8 : 16;
}
int64_t few_tiles(const KvAttend& a, int tile_rows) {
  return a.B * ceil_div(std::min(a.max_q, a.T) * (a.heads / a.c.heads), tile_rows) * a.c.heads;
}
// Workgroups of a launch: two a unit, or one where no more are resident.  64 fp32 tokens x 32 heads over 287 MB 70.5 us, with 768 72.6 and with 1024 82 (more
// waves at work on the memory at once, but more cut tiles and first loads); one a unit: those 3 tokens x 256 of bf16 128 us, with 512 149.
int few_groups(const KvAttend& a, int tile_rows) { return 256 * std::min(few_resident(a.dtype == GSI_F32, tile_rows, a.c.dim), 2); }
// Whether a workgroup takes a whole tile, its waves a part of the keys each, and nothing is cut or joined: where there is one tile at most for each, and the
// keys are so few that sharing them out saves less than the joining costs.  us a call, whole tiles / shares, bf16 single tokens, two heads to one of
// keys: 8 tiles of up to 1024 keys x 128 14 / 18, 2048 17 / 19, 4096 24 / 20; 512 tiles of 1024 18 / 23, 2048 24 / 27, 4096 43 / 43;
// 64 tiles x 256 of 1024 18 / 19, 2048 26 / 22; 1024 tiles of 1024 29 / 28, 8192 tiles of up to 512 261 / 80.
bool few_whole(const KvAttend& a, int tile_rows) { return few_tiles(a, tile_rows) <= few_groups(a, tile_rows) && a.max_len <= (a.c.dim > 128 ? 1024 : 2048); }
int few_workgroups(const KvAttend& a, int tile_rows) {
  const double tiles = (double)few_tiles(a, tile_rows), steps = few_whole(a, tile_rows) ? 1.0 : (double)ceil_div(a.max_len, kStep) / kWaves;
  return (int)std::max(1.0, std::min(tiles * steps, (double)few_groups(a, tile_rows)));
}

template <class X, int NR>
void launch_few(const Few& f, int W, hipStream_t s) {
  const int D = f.a.c.dim;
  if (D == 64) few_kernel<X, NR, 4, true><<<W, kThreads, 0, s>>>(f);
  else if (D == 128) few_kernel<X, NR, 8, true><<<W, kThreads, 0, s>>>(f);
  else if (D == 256) few_kernel<X, NR, 16, true><<<W, kThreads, 0, s>>>(f);
  else if (D < 64) few_kernel<X, NR, 4, false><<<W, kThreads, 0, s>>>(f);
  else if (D < 128) few_kernel<X, NR, 8, false><<<W, kThreads, 0, s>>>(f);
  else few_kernel<X, NR, 16, false><<<W, kThreads, 0, s>>>(f);
}
template <class X>
void launch_few(const Few& f, int W, hipStream_t s) {
  constexpr int kSmall = sizeof(typename X::storage) == 4 ? 0 : 1;
  if (f.tile_rows <= 4) launch_few<X, kSmall>(f, W, s);
  else if (f.tile_rows == 8) launch_few<X, 2>(f, W, s);
  else launch_few<X, 4>(f, W, s);
  if (!f.whole) {
    const int64_t rows = std::min<int64_t>(std::min(f.a.max_q, f.a.T) * f.group, f.tile_rows);
    join_kernel<X><<<dim3(W, (unsigned)std::max<int64_t>(rows, 1)), kThreads, 0, s>>>(f);
  }
}

}  // namespace

static size_t cuts_bytes(size_t W) { return align_up(W * kWaves * 16, 256); }
static size_t stats_bytes(size_t W, int tile) { return align_up(2 * W * kWaves * tile * sizeof(float2), 256); }
size_t attend_few_workspace(const KvAttend& a, int64_t few) {
  const int tile = few_tile(a, few);
  if (few_whole(a, tile)) return 0;
  const size_t W = (size_t)few_workgroups(a, tile);
  return cuts_bytes(W) + stats_bytes(W, tile) + align_up(2 * W * kWaves * tile * a.c.dim * sizeof(float), 256);
}

hipError_t attend_few(const KvAttend& a, int64_t few, void* ws, hipStream_t s) {
  Few f{};
  f.a = a;
  f.few = few;
  f.group = a.heads / a.c.heads;
  f.tile_rows = few_tile(a, few);
  f.by_group = Divisor(f.group);
  f.by_heads = Divisor(a.c.heads);
  f.by_tile = Divisor(f.tile_rows);
  f.whole = few_whole(a, f.tile_rows);
  const size_t es = elem_size(a.dtype);
  f.q_wide = reinterpret_cast<uintptr_t>(a.Q) % 16 == 0 && (size_t)a.q_stride * es % 16 == 0;
  const int W = few_workgroups(a, f.tile_rows);
  f.cuts = reinterpret_cast<int*>(ws);
  f.stats = reinterpret_cast<float2*>(static_cast<char*>(ws) + cuts_bytes(W));
  f.parts = reinterpret_cast<float*>(static_cast<char*>(ws) + cuts_bytes(W) + stats_bytes(W, f.tile_rows));
  if (a.dtype == GSI_BF16) launch_few<BF16>(f, W, s);
  else launch_few<F32>(f, W, s);
  return hipGetLastError();
}

// Which kernels a call takes, by the rows that its longest request has to a head of keys (tokens times heads that share it).  The workgroups of few rows
// read the keys once for 16 rows, those of many rows once for 128 but with a step that costs them as much for 20 rows as for 128.
// us a call, few / many rows, 8 heads of keys:
//   up to 16 rows: few.  16 rows, 16 requests of up to 4000 keys x 128: bf16 34 / 46, fp32 42 / 78.
//   up to 32: few, but for bf16 over short contexts of many requests, where few rows are cut and joined and many are not.  32 rows, 64 requests of up to
//     4000 keys: x 64 60 / 77, x 128 75 / 80, x 256 128 / 235, fp32 x 128 105 / 215; of up to 700: bf16 x 128 47 / 26.
//   up to 64: few where that makes a tile for each workgroup at most (64 rows, 8 requests of up to 4000 keys x 128: bf16 39 / 44, fp32 51 / 79), and for fp32
//     rows of 128 and more, whose products are three, and the widest heads (64 requests: fp32 x 128 170 / 231, x 256 322 / 505; bf16 x 256 213 /
//     245; not so x 128 113 / 91, fp32 x 64 123 / 106).
//   more: many (128 rows, 64 requests of up to 700: bf16 78 / 36, fp32 111 / 79; fp32 x 256 of up to 4000 589 / 589).
// A call of single tokens and prompts takes both kernels, each for its requests, where the mean request has few rows.  both / many rows: 63 single tokens
// behind 100 to 4000 keys and a prompt of 128, 32 heads of keys, bf16 115 / 192, fp32 166 / 492; requests of 1 to 64 tokens, four heads to
// one of keys (60 rows in the mean), bf16 87 / 61.  The few are then single tokens and others of up to 8 rows, whose tiles are small.  us with 8 / with
// 32 rows (tiles of 16): 250 single tokens and a prompt of 1024, 32 heads of keys, bf16 205 / 212, fp32 260 / 307, 8 heads of keys fp32 145 /
// 163; 60 requests of 3 tokens and a prompt of 512, 32 heads of keys, fp32 156 / 177, but 8 heads of keys (12 rows) 158 / 130.
constexpr int64_t kFewRows = 16;
static int64_t both_rows(const KvAttend& a) { return std::max(a.heads / a.c.heads, 8); }
enum Kernels { kFewOnly, kPromptOnly, kBoth };
static Kernels kernels_of(const KvAttend& a) {
  const int64_t group = a.heads / a.c.heads, rows = std::min(a.max_q, a.T) * group;
  const bool f32 = a.dtype == GSI_F32, fit = few_tiles(a, kFewRows) <= few_groups(a, kFewRows);
  const bool few = rows <= kFewRows || (rows <= 2 * kFewRows && (fit || f32 || a.c.dim > 128 || a.max_len > 1024)) ||
                   (rows <= 4 * kFewRows && (fit || (f32 && a.c.dim >= 128) || a.c.dim > 192));
  if (few || a.B == 0) return kFewOnly;
  return a.T * group < (f32 ? 3 : 1) * kFewRows * a.B ? kBoth : kPromptOnly;
}

size_t kv_attention_workspace(const KvAttend& a) {
  switch (kernels_of(a)) {
    case kFewOnly: return attend_few_workspace(a, INT64_MAX);
    case kPromptOnly: return attend_prompt_workspace(a);
    default: return attend_few_workspace(a, both_rows(a)) + attend_prompt_workspace(a);
  }
}

hipError_t kv_attention(const KvAttend& a, void* ws, hipStream_t s) {
  switch (kernels_of(a)) {
    case kFewOnly: return attend_few(a, INT64_MAX, ws, s);
    case kPromptOnly: return attend_prompt(a, 0, true, ws, s);
    default: break;
  }
  if (hipError_t e = attend_few(a, both_rows(a), ws, s); e != hipSuccess) return e;
  return attend_prompt(a, both_rows(a), false, static_cast<char*>(ws) + attend_few_workspace(a, both_rows(a)), s);
}

}  // namespace gsi
