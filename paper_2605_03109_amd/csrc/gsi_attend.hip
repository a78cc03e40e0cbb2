// Attention over the paged cache in 4 bits.
#include "gsi_device.h"
#include "gsi_kv.h"

namespace gsi {
namespace {

struct Span {  // a request's tokens of the call and its keys
  int t0, n, len;
};
__device__ __forceinline__ Span span_of(const KvAttend& a, int b) {
  Span s;
  const int T = (int)a.T;
  s.t0 = a.q_start ? min(max(a.q_start[b], 0), T) : min(b, T);
  const int t1 = a.q_start ? min(max(a.q_start[b + 1], s.t0), T) : min(b + 1, T);
  s.n = t1 - s.t0;
  s.len = (int)min((int64_t)max(a.kv_len[b], 0), a.width << a.c.page_shift);
  return s;
}

// A wave per token and head: a lane takes a key for the scores and every 64th element for the output.
template <class X>
__global__ __launch_bounds__(kWave) void attend_token(KvAttend a) {
  __shared__ float q[kKvMaxDim], p[kWave];
  const int lane = threadIdx.x, t = blockIdx.x, h = blockIdx.y, D = a.c.dim;
  const int kvh = h / (a.heads / a.c.heads);
  typename X::storage* const out = reinterpret_cast<typename X::storage*>(a.O) + ((int64_t)t * a.heads + h) * D;
  int b = 0;
  Span s{0, 0, 0};
  for (b = 0; b < a.B; ++b) {
    s = span_of(a, b);
    if (t >= s.t0 && t < s.t0 + s.n) break;
  }
  const int keys = b < a.B ? s.len - s.n + (t - s.t0) + 1 : 0;
  const typename X::storage* const Q = reinterpret_cast<const typename X::storage*>(a.Q) + t * a.q_stride + (int64_t)h * D;
  for (int d = lane; d < D; d += kWave) q[d] = X::load(Q, d);
  __syncthreads();
  float m = -INFINITY, l = 0.f, o[kKvMaxDim / kWave] = {};
  for (int k0 = 0; k0 < keys; k0 += kWave) {
    const int key = k0 + lane;
    int64_t page = key < keys ? a.table[b * a.width + (key >> a.c.page_shift)] : -1;
    if (page >= a.c.n_pages) page = -1;
    float z = -INFINITY;
    if (page >= 0) {
      z = 0.f;
      const int off = key & (a.c.page() - 1);
      const uint8_t* codes = a.c.K + a.c.code_at(page, kvh) + (int64_t)off * (D / 2);
      const uint8_t* scales = a.c.Ks + a.c.scale_at(page, kvh) + off;
      for (int d = 0; d < D; d += 2) {
        const float sc = __uint_as_float((uint32_t)scales[(d / kKvBlock) << a.c.page_shift] << 23);
        const auto v = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(codes[d / 2], sc, 0);
        z = fmaf(q[d], v[0], fmaf(q[d + 1], v[1], z));
      }
      z *= a.scale;
    }
    float top = z;
    for (int i = kWave / 2; i; i >>= 1) top = fmaxf(top, __shfl_xor(top, i, kWave));
    const float next = fmaxf(m, top);
    if (next == -INFINITY && !__any(z != z)) continue;
    const float keep = expf(m - next), e = expf(z - next);
    m = next;
    float sum = e;
    for (int i = kWave / 2; i; i >>= 1) sum += __shfl_xor(sum, i, kWave);
    l = l * keep + sum;
    for (float& x : o) x *= keep;
    for (int j = 0; j < kWave && k0 + j < keys; ++j) {
      const float pj = __shfl(e, j, kWave);
      const int64_t pg = a.table[b * a.width + ((k0 + j) >> a.c.page_shift)];
      if (pg < 0 || pg >= a.c.n_pages) continue;
      const int off = (k0 + j) & (a.c.page() - 1);
      for (int i = 0; i * kWave + lane < D; ++i) {
        const int d = i * kWave + lane;
        const uint8_t code = a.c.V[a.c.code_at(pg, kvh) + (int64_t)off * (D / 2) + d / 2];
        const float sc = __uint_as_float((uint32_t)a.c.Vs[a.c.scale_at(pg, kvh) + ((int64_t)(d / kKvBlock) << a.c.page_shift) + off] << 23);
        const auto v = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(code, sc, 0);
        o[i] = fmaf(pj, v[d & 1], o[i]);
      }
    }
  }
  for (int i = 0; i * kWave + lane < D; ++i) X::store(out, i * kWave + lane, l != 0.f ? o[i] / l : 0.f);
  if (a.lse && lane == 0) a.lse[(int64_t)t * a.heads + h] = l != 0.f ? m + logf(l) : -INFINITY;
}

}  // namespace

size_t kv_attention_workspace(const KvAttend&) { return 0; }

hipError_t kv_attention(const KvAttend& a, void*, hipStream_t s) {
  const dim3 grid((unsigned)a.T, (unsigned)a.heads);
  if (a.dtype == GSI_BF16) attend_token<BF16><<<grid, kWave, 0, s>>>(a);
  else attend_token<F32><<<grid, kWave, 0, s>>>(a);
  return hipGetLastError();
}

}  // namespace gsi
