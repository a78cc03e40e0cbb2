// Attention over the paged cache in 4 bits, many rows: prompts and their chunks.
//
// A workgroup of four waves takes 128 rows (tokens times the heads that share a head of keys), 32 a wave, and 64 keys a step.  Scores and
// outputs are kept transposed, tokens by rows and elements by rows: a row's scores then lie in two lanes, its maximum and its sum
// need no exchange but one, and the weights are the second product's operand as they come out of the first (the tokens of its
// contraction taken in the order of the accumulator's registers).  Keys and values are converted once, on their way to LDS; values are read
// there with the transposing reads.  (By each wave for itself, chunks of 512 tokens behind 6000 to 15000 keys took 410 us; this way 379.)
//
// Issue bounds it: those chunks, 346 GFLOP, run at 0.92 PFLOP/s (a plain loop of matrix instructions on random data at 1.47), with the matrix units busy for a third of the time;
// exponentials, sums, the conversion of the next step and the reads of LDS take the slots of a SIMD's two waves beside them.  2048 tokens from the
// first on x 32 heads x 128, 34 GFLOP, take 58 us: tiles of one round, of which the longest, alone on its unit towards the end, sets the time.
// fp32 rows have three products in place of one: six prompts of 90 to 700 tokens, 24 heads over 8 of 96, 33 GFLOP as bf16, 61 us.
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
  Divisor by_group, by_heads;  // by the heads of a group, the heads of keys
  int q_wide;
  int zero;       // whether this launch clears the rows of tokens of no request
  int fold;       // whole tiles: of a request, the one half from the last on, then the other from the first on
  // shares (null: a workgroup takes a whole tile)
  f32x4* parts;   // [2 * workgroups][dim / 8][256]: a thread's sums of a cut tile
  float2* stats;  // [2 * workgroups][128]: a row's maximum and sum of weights; a maximum of NaN: no part
  int* cuts;      // [workgroups][4]: the tile that a workgroup begins and does not end, and the one that ends it
};

// Waves a SIMD (workgroups a unit) that the registers leave.  (Three, with spills: 692 us on long contexts where two take 385.)
__host__ __device__ constexpr int prompt_waves(int nd) { return nd > 4 ? 1 : 2; }

template <int ND>
struct Lds {  // of one step
  static constexpr int kStride = 64 * (ND | 1);  // bytes of a token's values: four tokens lie in distinct banks
  // keys: pieces of eight elements, of all tokens one after another; then the values
  static constexpr int kKeys = 0, kValues = 4 * ND * kStep * 16, kSize = kValues + kStep * kStride;
};

__device__ __forceinline__ int64_t tiles_of(const Prompt& f, const Span& s) {
  const int64_t rows = (int64_t)s.n * f.group;
  return rows > f.few ? (rows + kTile - 1) / kTile : 0;
}

__device__ __forceinline__ int high_of(const Prompt& f, const Span& s, int tile) {  // the last key that a row of the tile sees
  return s.last_key(f.by_group(min(tile * kTile + kTile - 1, s.n * f.group - 1)));
}
__device__ __forceinline__ int steps_of(const Prompt& f, const Span& s, int tile) { return max(0, high_of(f, s, tile)) / kStep + 1; }

// What a tile costs, in keys times the heads of a group: the keys that its rows see, which grow by 128 from tile to tile (past the table's last place they
// do not: such tiles count for more than they are), and two steps for its queries and its output.  A closed form: the cost of a request's first t tiles is 64 t^2 + (a - 64) t.
struct Cost {
  int64_t a;  // of the first tile
  int64_t tiles;
  __device__ __forceinline__ Cost(const Prompt& f, const Span& s)
      : a((int64_t)f.group * (max(0, min(s.past, s.len)) + 2 * kStep) + kTile), tiles(tiles_of(f, s)) {}
  __device__ __forceinline__ int64_t of_tile(int64_t t) const { return a + kTile * t; }
  __device__ __forceinline__ int64_t before(int64_t t) const { return (kTile / 2 * t + a - kTile / 2) * t; }
  __device__ __forceinline__ int64_t all() const { return before(tiles); }
  __device__ __forceinline__ int64_t tile_at(int64_t u) const {  // the tile with before(t) <= u < before(t + 1)
    const double half = 0.5 * (double)(a - kTile / 2);
    int64_t t = (int64_t)((sqrt(half * half + kTile / 2 * (double)u) - half) / (kTile / 2));
    t = min(max(t, (int64_t)0), tiles - 1);
    while (t > 0 && before(t) > u) --t;
    while (t + 1 < tiles && before(t + 1) <= u) ++t;
    return t;
  }
};

__device__ __forceinline__ uint32_t bf16_pair(float a, float b) {
  const bf16x2 v = {(__bf16)a, (__bf16)b};
  return __builtin_bit_cast(uint32_t, v);
}

// A lane's elements of a row of the output: 32 d + 8 i + 4 h .. of its ND blocks from block d0 on.
template <class X, int ND>
__device__ __forceinline__ void store_rows(const KvAttend& a, const f32x16 (&o)[ND], float m, float l, int64_t orow, int h, int d0 = 0) {
  const float inv = l == 0.f ? 0.f : 1.f / l;
  typename X::storage* const out = reinterpret_cast<typename X::storage*>(a.O) + orow * a.c.dim + 32 * d0 + 4 * h;
#pragma unroll
  for (int d = 0; d < ND; ++d)
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      typename X::storage* const p = out + 32 * d + 8 * i;
      const float x[4] = {o[d][4 * i] * inv, o[d][4 * i + 1] * inv, o[d][4 * i + 2] * inv, o[d][4 * i + 3] * inv};
      if constexpr (sizeof(*p) == 4) *reinterpret_cast<f32x4*>(p) = f32x4{x[0], x[1], x[2], x[3]};
      else *reinterpret_cast<u32x2*>(p) = u32x2{bf16_pair(x[0], x[1]), bf16_pair(x[2], x[3])};
    }
  if (a.lse && h == 0 && d0 == 0) a.lse[orow] = l == 0.f ? -INFINITY : (m == -INFINITY ? l : (m + log2f(l)) * kLn2);
}

template <class X, int ND>
__global__ __launch_bounds__(kThreads, prompt_waves(ND)) void prompt_kernel(Prompt f) {
  constexpr bool F = sizeof(typename X::storage) == 4;
  constexpr int QT = F ? 3 : 1, PT = F ? 3 : 1, NP = 2 * ND, KU = (ND + 3) / 4;
  using M = Lds<ND>;
  // bf16 weights in one term, rounded to 2^-8: their second one would be a product more for every two.  (An output is then off by 0.0022 to 0.0025 of itself
  // in the mean, with two by 0.0017, its own rounding; four chunks of 512 behind 6000 to 15000 keys 381 us, with two 490; 2048 tokens x 32 heads x
  // 128 61.5 and 72, x 16 x 256 102 and 111.)
  // fp32 queries of 224 elements and more are read again in every step: their three terms and the output would take all registers.  (2048 tokens x 16
  // heads x 256 182 us, kept with spills 381; x 192, where they fit, 118, read again 152; x 128 at two workgroups a unit 91, 90 and in chunks
  // behind long contexts 276, 318.)
  constexpr bool kStream = F && ND > 6;
  // 32 keys' scores at a time where the registers of 64 do not fit: fp32 rows that keep their queries (2048 tokens x 32 heads x 128: 139 us, in one
  // piece 180), and wide heads (bf16, 2048 x 16 x 256: 103 us, in one piece 111)
  constexpr int NY = (F && !kStream) || (!F && ND > 6) ? 1 : 2;
  // Values are requested ahead where registers are left for it
  constexpr bool kAhead = !F || ND == 5;
  extern __shared__ __align__(16) char lds[];
  __shared__ Prefix prefix;
  __shared__ int spoiled[3][ND];  // first token of a step whose value is NaN, by block: three steps' worth, one of them being cleared
  const KvAttend& a = f.a;
  const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave, c = lane & 31, h = lane >> 5;
  constexpr int D = 32 * ND, half = D / 2;

  int kvh, b, tile;
  int64_t u = 0, u_end = 1, before = 0;  // shares: this workgroup's units, and those before request b
  // workgroups run round the eight caches of the chip: those of consecutive shares are taken to one
  const int64_t me = !f.parts ? blockIdx.x : gridDim.x % 8 == 0 ? blockIdx.x % 8 * (gridDim.x / 8) + blockIdx.x / 8 : blockIdx.x;
  Shares sh{};
  if (!f.parts) {
    // heads of keys run fastest: with eight of them and more, a cache holds the same ones throughout
    const auto units = [&](const Span& s) { return tiles_of(f, s); };
    const int64_t total = total_units(a, prefix, units), slot = f.by_heads(blockIdx.x);
    const Place p = place_of(a, prefix, total, slot, units);
    if (f.zero) clear_idle_rows<X>(a);
    if (slot >= total) return;
    b = p.b;
    kvh = (int)blockIdx.x - (int)slot * a.c.heads;
    const int64_t n = tiles_of(f, span_at(a, prefix, b)), i = slot - p.before;
    // The last tiles see the most keys and come first.  Where all workgroups are resident at once, a unit has the i-th and the i-th of the second
    // half: that half runs the other way, and what two workgroups of a unit do together is about the same everywhere.
    tile = (int)(!f.fold || i < (n + 1) / 2 ? n - 1 - i : i - (n + 1) / 2);
  } else {
    const auto units = [&](const Span& s) { return a.c.heads * Cost(f, s).all(); };
    const int64_t total = total_units(a, prefix, units);
    sh = shares_of(total, gridDim.x, 8 * kStep * f.group);
    u = sh.of_group(me);
    u_end = total == 0 || me >= sh.groups ? u : sh.of_group(me + 1);
    const Place p = place_of(a, prefix, total, u, units);
    b = p.b;
    before = p.before;
    if (f.zero) clear_idle_rows<X>(a);
    if (threadIdx.x == 0) f.cuts[4 * me] = -1;
  }
  const int uwave = __builtin_amdgcn_readfirstlane(wave);
  const float zscale = exponent_scale(a.scale);
  const int last = (int)a.width - 1, mask = a.c.page() - 1;
  const uint32_t code_stride = (uint32_t)a.c.code_at(1, 0), scale_stride = (uint32_t)a.c.scale_at(1, 0);

  while (u < u_end) {
  Span sp = span_at(a, prefix, b);
  int step0 = 0, step1;
  int64_t stop = u_end;
  if (!f.parts) {
    step1 = steps_of(f, sp, tile);
  } else {
    Cost cost(f, sp);
    while (u >= before + a.c.heads * cost.all()) {  // the next request with tiles
      before += a.c.heads * cost.all();
      ++b;
      sp = span_at(a, prefix, b);
      cost = Cost(f, sp);
    }
    const int64_t all = cost.all();
    kvh = (int)divide(u - before, all);
    const int64_t at = u - before - kvh * all, t = cost.tile_at(at), own = cost.of_tile(t), off = at - cost.before(t);
    tile = (int)t;
    const int64_t end = u - off + own;
    stop = min(u_end, end);
    const int steps = steps_of(f, sp, tile);
    // a boundary lies in front of the step that has its share of the tile's cost: the same for the workgroups on both its sides
    const auto step_at = [&](int64_t x) { return (int)((double)steps * (double)x / (double)own); };
    step0 = step_at(off);
    step1 = stop == end ? steps : step_at(stop - (u - off));
  }
  b = __builtin_amdgcn_readfirstlane(b);
  tile = __builtin_amdgcn_readfirstlane(tile);
  kvh = __builtin_amdgcn_readfirstlane(kvh);
  step0 = __builtin_amdgcn_readfirstlane(step0);
  step1 = __builtin_amdgcn_readfirstlane(step1);
  sp.t0 = __builtin_amdgcn_readfirstlane(sp.t0);
  sp.n = __builtin_amdgcn_readfirstlane(sp.n);
  sp.len = __builtin_amdgcn_readfirstlane(sp.len);
  sp.past = __builtin_amdgcn_readfirstlane(sp.past);
  const bool ends = !f.parts || step1 == steps_of(f, sp, tile), complete = step0 == 0 && ends;
  if (step0 >= step1) {
    // the boundaries on both sides lie in front of one step: no part of the tile
    if (step0 > 0 && threadIdx.x < kTile) f.stats[2 * me * kTile + threadIdx.x] = make_float2(NAN, 0.f);
    u = stop;
    continue;
  }
  const int all_rows = sp.n * f.group, row0 = tile * kTile;

  const int rid = row0 + 32 * wave + c;
  const bool real = rid < all_rows;
  const int tok = real ? f.by_group(rid) : 0, head = kvh * f.group + (real ? rid - tok * f.group : 0);
  const int lim = real ? sp.last_key(tok) : -1;  // the last key that this lane's row sees
  // of the wave's rows, and of the workgroup's: the last key that any sees, and the last that all see (idle rows aside)
  const int wave_first = row0 + 32 * wave, wave_last = min(wave_first + 31, all_rows - 1);
  const int wave_high = wave_first < all_rows ? sp.last_key(f.by_group(wave_last)) : -1;
  const int wave_low = wave_first < all_rows ? sp.last_key(f.by_group(wave_first)) : -1;
  const int low = sp.last_key(f.by_group(row0));

  // query rows: the operand's elements 8 h + u of product p are elements 16 p + 8 h + u
  const typename X::storage* Q = reinterpret_cast<const typename X::storage*>(a.Q) + (int64_t)(sp.t0 + tok) * a.q_stride + (int64_t)head * D;
  bf16x8 q[kStream ? 2 : NP][QT];
  if constexpr (!kStream) {
#pragma unroll
    for (int p = 0; p < NP; ++p) {
      QueryPart<X, 8> raw;
      raw.load(Q, 16 * p + 8 * h, real, f.q_wide, a.scale < 0.f);
      raw.template terms<QT>(0, q[p]);
    }
  }

  f32x16 o[ND];
#pragma unroll
  for (int d = 0; d < ND; ++d)
#pragma unroll
    for (int i = 0; i < 16; ++i) o[d][i] = 0.f;
  float m = -INFINITY, l = 0.f;
  const int32_t* const trow = a.table + (int64_t)b * a.width;

  // A wave brings 16 tokens of a step, which lie on one page: a thread blocks of keys (one token's 32 codes) and words of values (8 codes), each with its
  // scale byte.
  struct Bring {
    u32x4 k[KU];
    uint32_t ks[KU];
    uint32_t v[ND];
    uint32_t vs[ND];
    int there;  // a bit for each 16 tokens whose page is there
  };
  const int64_t code0 = a.c.code_at(0, kvh), scale0 = a.c.scale_at(0, kvh);
  const auto entry = [&](int step) { return trow[min((step * kStep + 16 * (lane & 3)) >> a.c.page_shift, last)]; };  // lane i: of the step's 16 (i % 4) .. tokens
  const auto bring = [&](int step, int en) {
    Bring r;
    r.there = (int)__ballot((uint32_t)en < (uint32_t)a.c.n_pages) & 15;
    const uint32_t page = r.there >> uwave & 1 ? __builtin_amdgcn_readlane(en, uwave) : 0;  // another page's keys: they are not seen
    const int off = (step * kStep + 16 * uwave) & mask;
    const uint64_t code = code0 + (uint64_t)page * code_stride + off * half, scale = scale0 + (uint64_t)page * scale_stride + off;
#pragma unroll
    for (int i = 0; i < KU; ++i) {
      const int u = i * kWave + lane, t = u % 16, blk = u / 16;
      if (ND % 4 == 0 || blk < ND) {
        r.k[i] = *reinterpret_cast<const u32x4*>(a.c.K + code + (uint32_t)(t * half + blk * 16));
        r.ks[i] = (a.c.Ks + scale)[(uint32_t)((blk << a.c.page_shift) + t)];
      }
    }
#pragma unroll
    for (int i = 0; i < ND; ++i) {
      const int u = i * kWave + lane, t = u / (4 * ND), w = u % (4 * ND);
      r.v[i] = *reinterpret_cast<const uint32_t*>(a.c.V + code + (uint32_t)(t * half + w * 4));
      r.vs[i] = (a.c.Vs + scale)[(uint32_t)(((w / 4) << a.c.page_shift) + t)];
    }
    return r;
  };
  const auto stage = [&](int step, const Bring& r) {
    char* const at = lds + (step & 1) * M::kSize;
    const bool special = rarely(step * kStep + kStep - 1 > low || r.there != 15);
#pragma unroll
    for (int i = 0; i < KU; ++i) {
      const int u = i * kWave + lane, t = 16 * uwave + u % 16, blk = u / 16;
      if (ND % 4 == 0 || blk < ND) {
        const float scale = scale_value(r.ks[i]);
#pragma unroll
        for (int w = 0; w < 4; ++w) *reinterpret_cast<u32x4*>(at + M::kKeys + ((4 * blk + w) * kStep + t) * 16) = eight_values(r.k[i][w], scale);
      }
    }
#pragma unroll
    for (int i = 0; i < ND; ++i) {
      const int u = i * kWave + lane, t = 16 * uwave + u / (4 * ND), w = u % (4 * ND);
      uint32_t word = r.v[i], vs = r.vs[i];
      if (special) {
        keep_branch();
        // 0 times what is not seen, or seen by some rows only, has to be 0: NaN goes to its rows by `spoiled`
        const bool seen = step * kStep + t < sp.len && (r.there >> uwave & 1);
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
  int en;
  {
    const Bring r = bring(step0, entry(step0));
    en = entry(step0 + 1);
    there = r.there;
    stage(step0, r);
  }
  if constexpr (!kStream) {
#pragma unroll
    for (int p = 0; p < NP; ++p)
#pragma unroll
      for (int t = 0; t < QT; ++t) arrive(q[p][t]);
  }
  __syncthreads();
  const int vlane = (4 * h + ((lane & 15) >> 2)) * M::kStride + 32 * ((lane >> 4) & 1) + 8 * (lane & 3);
  for (int step = step0; step < step1; ++step) {
    Bring next;
    const bool more = step + 1 < step1;
    if (more) {
      next = bring(step + 1, en);
      en = entry(step + 2);  // (taken a step later: it is not waited for here)
    }
    if ((int)threadIdx.x < ND) spoiled[(step + 2) % 3][threadIdx.x] = 0x7fffffff;
    const char* const at = lds + (step & 1) * M::kSize;
    const int key = step * kStep;
#pragma unroll
    for (int y0 = 0; y0 < 2; y0 += NY) {
      if (key + 32 * y0 > wave_high) continue;  // no row of this wave sees these keys
      f32x16 s[NY];
#pragma unroll
      for (int y = 0; y < NY; ++y)
#pragma unroll
        for (int i = 0; i < 16; ++i) s[y][i] = 0.f;
      // keys of two products at a time, requested while the ones before are multiplied
      bf16x8 k[2][2][NY];
      QueryPart<X, 8> raw[2][2];
      if constexpr (kStream) asm volatile("" : "+v"(Q));  // (not read once in front of all steps)
      const auto read_keys = [&](int n) {
        if constexpr (kStream) {
#pragma unroll
          for (int p = 0; p < 2; ++p) raw[n & 1][p].load(Q, 16 * (2 * n + p) + 8 * h, real, f.q_wide, a.scale < 0.f);
        }
#pragma unroll
        for (int p = 0; p < 2; ++p)
#pragma unroll
          for (int y = 0; y < NY; ++y)
            k[n & 1][p][y] = *reinterpret_cast<const bf16x8*>(at + M::kKeys + ((2 * (2 * n + p) + h) * kStep + 32 * (y0 + y) + c) * 16);
        hold_all();
      };
      read_keys(0);
#pragma unroll
      for (int n = 0; n < NP / 2; ++n) {
        if (n + 1 < NP / 2) read_keys(n + 1);
#pragma unroll
        for (int p = 0; p < 2; ++p) {
          if constexpr (kStream) raw[n & 1][p].template terms<QT>(0, q[p]);
#pragma unroll
          for (int t = 0; t < QT; ++t)
#pragma unroll
            for (int y = 0; y < NY; ++y) s[y] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(k[n & 1][p][y], q[kStream ? p : 2 * n + p][t], s[y], 0, 0, 0);
        }
      }
      // values of 16 tokens at a time, requested while the ones before are multiplied: the first ones before the exponentials
      bf16x8 v[2][ND];
      const auto read_values = [&](int n) {
        const char* const va = at + M::kValues + vlane + (32 * y0 + 16 * n) * M::kStride;
#pragma unroll
        for (int d = 0; d < ND; ++d) {
          const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(va + 64 * d));
          const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(va + 64 * d + 8 * M::kStride));
          v[n & 1][d] = __builtin_bit_cast(bf16x8, (s16x8)__builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
        }
        if constexpr (kAhead) hold_lds();
      };
      if constexpr (kAhead) read_values(0);
      if (rarely(key + 32 * (y0 + NY) - 1 > wave_low || there != 15)) {
        keep_branch();
#pragma unroll
        for (int y = 0; y < NY; ++y)
#pragma unroll
          for (int i = 0; i < 16; ++i) {
            const int t = 32 * (y0 + y) + 8 * (i / 4) + 4 * h + i % 4;
            s[y][i] = key + t <= lim && (there >> (2 * (y0 + y) + i / 8) & 1) ? s[y][i] : -INFINITY;
          }
      }
      if (y0 == 0 && rarely(key + kStep - 1 > low || there != 15)) {  // as stage() has it
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
      for (int y = 0; y < NY; ++y)
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
      for (int y = 0; y < NY; ++y)
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          s[y][i] = __builtin_amdgcn_exp2f(fmaf(s[y][i], zscale, -base));
          l += s[y][i];
        }
#pragma unroll
      for (int n = 0; n < 2 * NY; ++n) {
        if constexpr (!kAhead) read_values(n);
        else if (n + 1 < 2 * NY) read_values(n + 1);
        float e[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) e[i] = s[n / 2][8 * (n & 1) + i];
        bf16x8 pf[PT];
#pragma unroll
        for (int t = 0; t < PT; ++t) {
          u32x4 w;
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            w[i] = bf16_pair(e[2 * i], e[2 * i + 1]);
            if (t + 1 < PT) {
              e[2 * i] -= bf16_lo(w[i]);
              e[2 * i + 1] -= bf16_hi(w[i]);
            }
          }
          pf[t] = __builtin_bit_cast(bf16x8, w);
        }
#pragma unroll
        for (int d = 0; d < ND; ++d)
#pragma unroll
          for (int t = 0; t < PT; ++t) o[d] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(v[n & 1][d], pf[t], o[d], 0, 0, 0);
      }
    }
    if (more) {
      stage(step + 1, next);
      there = next.there;
    }
    __syncthreads();
  }

  l += __shfl_xor(l, 32, kWave);
  if (complete) {
    if (real) store_rows<X, ND>(a, o, m, l, (int64_t)(sp.t0 + tok) * a.heads + head, h);
  } else {
    // place 2 i: a tile that an earlier workgroup began; place 2 i + 1: one that begins here and ends elsewhere
    const int64_t place = 2 * me + (step0 == 0);
    f32x4* const part = f.parts + place * (D / 8) * kThreads + threadIdx.x;
#pragma unroll
    for (int d = 0; d < ND; ++d)
#pragma unroll
      for (int i = 0; i < 4; ++i) part[(4 * d + i) * kThreads] = f32x4{o[d][4 * i], o[d][4 * i + 1], o[d][4 * i + 2], o[d][4 * i + 3]};
    if (h == 0) f.stats[place * kTile + 32 * wave + c] = make_float2(m, l);
    if (step0 == 0 && threadIdx.x == 0) {
      int* const cut = f.cuts + 4 * me;
      cut[1] = tile;
      cut[2] = kvh;
      const Cost cost(f, sp);
      cut[3] = (int)sh.group_of(before + kvh * cost.all() + cost.before(tile + 1) - 1);
      cut[0] = b;
    }
  }
  u = stop;
  }
}

// Joins the parts of a cut tile in their order: a workgroup for each 32 elements of the tile that another has begun and not ended, whose threads
// have the rows and elements that those of prompt_kernel had.  Memory bounds it: 512 workgroups' parts of 128 x 128, 64 MB, 17 us; of 128 x 96 14 us.
template <class X>
__global__ __launch_bounds__(kThreads) void join_tiles(Prompt f) {
  const KvAttend& a = f.a;
  const int w = blockIdx.x, d = blockIdx.y;
  typedef int i32x4 __attribute__((ext_vector_type(4)));
  const i32x4 cut = *reinterpret_cast<const i32x4*>(f.cuts + 4 * w);
  const int b = cut[0], tile = cut[1], kvh = cut[2], end = cut[3];
  if (b < 0) return;
  const int lane = threadIdx.x % kWave, wave = threadIdx.x / kWave, c = lane & 31, h = lane >> 5;
  const Span sp = span_of(a, b);
  const int rid = tile * kTile + 32 * wave + c;
  float top = -INFINITY, sum = 0.f;
  f32x16 o[1];
#pragma unroll
  for (int i = 0; i < 16; ++i) o[0][i] = 0.f;
  // two parts are requested at a time, with their maxima
  for (int i0 = w; i0 <= end; i0 += 2) {
    float2 ml[2];
    f32x4 v[2][4];
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      const int i = min(i0 + k, end);
      const int64_t place = i == w ? 2 * i + 1 : 2 * i;
      ml[k] = f.stats[place * kTile + 32 * wave + c];
      const f32x4* const part = f.parts + (place * (a.c.dim / 8) + 4 * d) * kThreads + threadIdx.x;
#pragma unroll
      for (int y = 0; y < 4; ++y) v[k][y] = part[y * kThreads];
    }
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      const float m = ml[k].x;
      if (i0 + k > end || m != m) continue;  // (a maximum of NaN: no part; the same for all threads)
      const float next = fmaxf(top, m), keep = next == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(top - next);
      const float x = m == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(m - next);
      top = next;
      sum = fmaf(sum, keep, ml[k].y * x);
#pragma unroll
      for (int e = 0; e < 16; ++e) o[0][e] = fmaf(o[0][e], keep, v[k][e / 4][e % 4] * x);
    }
  }
  if (rid >= sp.n * f.group) return;
  const int tok = f.by_group(rid);
  const int64_t orow = (int64_t)(sp.t0 + tok) * a.heads + kvh * f.group + rid - tok * f.group;
  store_rows<X, 1>(a, o, top, sum, orow, h, d);
}

int64_t prompt_slots(const KvAttend& a) { return ceil_div(a.T * (a.heads / a.c.heads), kTile) + a.B; }

// Workgroups that are resident at once: two a unit, one where a wave has more than half the registers.
int prompt_resident(const KvAttend& a) { return 256 * prompt_waves(a.c.dim / 32); }
// Whether the keys of all tiles are dealt out in equal shares.  That writes, reads and joins two parts a workgroup, about 15 us; whole tiles leave units idle: by
// far the most where there are fewer tiles than workgroups fit, some where the tiles of about one round differ in length, little
// after two rounds, whose last tiles are the shortest of a request.  Steps are weighted by what one costs (elements of a head, the three products of fp32).
// us a call, shares / whole tiles, 8 heads of keys x 128, four heads to one, unless said:
//   load below 0.75: 512 tokens after 3000, bf16 66 / 89, fp32 115 / 196; 256 after 2000 47 / 63; 60 after 15000 72 / 352; 1024 from the first on 49 / 34
//   below 1.75: 8192 x 8 heads from the first on 175 / 199, 2048 x 32 heads 77 / 61 (its fp32 139 / 143); 2048 after 2000, tiles of about one
//     length, 138 / 121; six of 300 after 100 to 3000 80 / 99; four of 512 after 6000 to 15000 383 / 432
//   above: 4096 x 32 181 / 164; two of 8192 x 16 625 / 582; eight of 512 after 6000 to 15000 734 / 803, after 1500 to 4000 236 / 247, fp32 546 / 583; eight
//     of 500 to 1000 after 500 to 3000 230 / 213
bool prompt_shares(const KvAttend& a) {
  const double tiles = (double)a.c.heads * (double)ceil_div(a.T * (a.heads / a.c.heads), kTile), resident = prompt_resident(a);
  const double load = tiles / resident, steps = (double)ceil_div(a.max_len, kStep) * (a.dtype == GSI_F32 ? 2 : 1) * a.c.dim / 128;
  const double least = a.B == 1 ? steps * (double)std::max<int64_t>(a.max_len - a.T, 0) / (double)a.max_len : 0.0;  // of the shortest tile
  return load < 0.75 ? steps >= 32.0 : load < 1.75 ? steps - least >= 48.0 : a.B > 1 && steps >= 64.0 * load;
}
size_t parts_bytes(const KvAttend& a, size_t W) { return 2 * W * kTile * a.c.dim * sizeof(float); }
size_t stats_bytes(size_t W) { return 2 * W * kTile * sizeof(float2); }

template <class X, int ND>
hipError_t launch_prompt(const Prompt& f, hipStream_t s) {
  const int bytes = 2 * Lds<ND>::kSize;
  static LdsLimit limit;
  if (bytes > 60 * 1024)
    if (hipError_t e = limit.allow((const void*)prompt_kernel<X, ND>, bytes); e != hipSuccess) return e;
  if (!f.parts) {
    prompt_kernel<X, ND><<<(unsigned)(prompt_slots(f.a) * f.a.c.heads), kThreads, bytes, s>>>(f);
  } else {
    const int W = prompt_resident(f.a);
    prompt_kernel<X, ND><<<W, kThreads, bytes, s>>>(f);
    join_tiles<X><<<dim3(W, ND), kThreads, 0, s>>>(f);
  }
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
  if (!prompt_shares(a)) return 0;
  const size_t W = prompt_resident(a);
  return parts_bytes(a, W) + stats_bytes(W) + align_up(W * 16, 256);
}

hipError_t attend_prompt(const KvAttend& a, int64_t few, bool zero, void* ws, hipStream_t s) {
  Prompt f{};
  f.a = a;
  f.few = few;
  f.group = a.heads / a.c.heads;
  f.by_group = Divisor(f.group);
  f.by_heads = Divisor(a.c.heads);
  const size_t es = elem_size(a.dtype);
  f.q_wide = reinterpret_cast<uintptr_t>(a.Q) % 16 == 0 && (size_t)a.q_stride * es % 16 == 0;
  f.zero = zero;
  // (2048 tokens x 32 heads x 128 61 us, without 64; two of 1500 x 32 heads x 64, whose workgroups are not all resident, 53 us, without 47)
  f.fold = prompt_slots(a) * a.c.heads <= prompt_resident(a) + a.B * a.c.heads;
  if (prompt_shares(a)) {
    const size_t W = prompt_resident(a);
    char* const p = static_cast<char*>(ws);
    f.parts = reinterpret_cast<f32x4*>(p);
    f.stats = reinterpret_cast<float2*>(p + parts_bytes(a, W));
    f.cuts = reinterpret_cast<int*>(p + parts_bytes(a, W) + stats_bytes(W));
  }
  return a.dtype == GSI_BF16 ? launch_prompt<BF16>(f, s) : launch_prompt<F32>(f, s);
}

}  // namespace gsi
