// attend.hip — attention of a step's tokens over the paged cache
// (atp_kv_attend).
#include "kvdev.h"

namespace atp {
namespace {

constexpr int kWaves = 4;

// One wave per (row, query head), one token per lane at a time: dot product,
// running maximum and sum, then the weights times V with the lanes over the
// dimensions.
template <typename T, typename CT>
__global__ void __launch_bounds__(kWaves * 64) k_attend(AttendArgs a) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  __shared__ float qs[kWaves][256];
  const int64_t item = blockIdx.x * int64_t(kWaves) + wave, n = int64_t(a.n_seq) * a.max_fresh * a.h.n_q;
  if (item >= n) return;
  const int32_t h = int32_t(item % a.h.n_q), i = int32_t(item / a.h.n_q % a.max_fresh), s = int32_t(item / a.h.n_q / a.max_fresh);
  const int32_t r0 = a.starts[s], r1 = a.starts[s + 1], cached = a.cached[s];
  const int64_t ctx = int64_t(cached) + r1 - r0;
  if (r0 < 0 || r1 < r0 || r1 > a.max_tokens || r1 - r0 > a.max_fresh || cached < 0 || ctx > a.max_ctx ||
      ctx > int64_t(a.max_blocks) * a.c.bt) {
    flag(a.status, ATP_EINVAL);
    return;
  }
  if (i >= r1 - r0) return;
  const int32_t j = (h + a.h.cut) / a.h.group + a.h.kv0, hd = a.c.hd;
  const T *q = static_cast<const T *>(a.q) + (r0 + i) * a.q_stride + int64_t(h) * hd;
  for (int d = lane; d < hd; d += 64) qs[wave][d] = as_f32(q[d]);
  __builtin_amdgcn_wave_barrier();
  const int32_t pos = cached + i, lo = a.window > 0 ? max(0, pos - a.window + 1) : 0;
  const float ks = a.c.scales ? a.c.scales[j] : 1.0f, vs = a.c.scales ? a.c.scales[a.c.n_kv + j] : 1.0f;
  float m = -INFINITY, l = 0, o[4] = {0, 0, 0, 0};
  for (int32_t t0 = lo; t0 <= pos; t0 += 64) {
    const int32_t t = t0 + lane;
    float score = -INFINITY;
    const char *row = nullptr;
    if (t <= pos) {
      const int32_t p = a.table[int64_t(s) * a.max_blocks + t / a.c.bt];
      if (p < -1 || p >= a.c.num_blocks) flag(a.status, ATP_EINVAL);
      if (p >= 0 && p < a.c.num_blocks) {
        row = a.c.base + p * a.c.block_stride + int64_t(j) * a.c.head_stride + int64_t(t % a.c.bt) * a.c.tok_stride;
        const CT *k = reinterpret_cast<const CT *>(row);
        float dot = 0;
        for (int d = 0; d < hd; ++d) dot += qs[wave][d] * as_f32(k[d]);
        score = dot * ks * a.scale;
        if (a.softcap > 0) score = a.softcap * tanhf(score / a.softcap);
        if (a.slopes) score += a.slopes[h] * float(t - pos);
      }
    }
    float top = score;
    for (int d = 32; d; d >>= 1) top = fmaxf(top, __shfl_xor(top, d));
    top = fmaxf(top, m);
    if (top == -INFINITY && __ballot(row != nullptr && score != score) == 0) continue;  // nothing seen yet
    const float keep = expf(m - top), p = row ? expf(score - top) : 0.0f;
    m = top;
    l = l * keep + p;
    for (int e = 0; e < 4; ++e) o[e] *= keep;
    for (int x = 0; x < 64; ++x) {
      const uint64_t rx = __shfl(reinterpret_cast<uint64_t>(row), x);
      if (!rx) continue;
      const float px = __shfl(p, x);
      const CT *v = reinterpret_cast<const CT *>(rx + a.c.v_off);
      for (int e = 0; e < 4; ++e)
        if (e * 64 + lane < hd) o[e] += px * as_f32(v[e * 64 + lane]);
    }
  }
  for (int d = 32; d; d >>= 1) l += __shfl_xor(l, d);
  const float inv = l == 0 ? 0 : vs / l;
  T *out = static_cast<T *>(a.out) + (r0 + i) * a.out_stride + int64_t(h) * hd;
  for (int e = 0; e < 4; ++e)
    if (e * 64 + lane < hd) out[e * 64 + lane] = rounded<T>(o[e] * inv);
  if (a.lse && lane == 0) a.lse[int64_t(r0 + i) * a.h.n_q + h] = l == 0 ? -INFINITY : m + logf(l);
}

}  // namespace

uint64_t attend_workspace(const AttendArgs &a) { return 0; }

void attend_launch(const AttendArgs &a, void *ws, void *stream) {
  const hipStream_t st = kv_stream(stream);
  const int64_t n = int64_t(a.n_seq) * a.max_fresh * a.h.n_q;
  const dim3 grid(uint32_t((n + kWaves - 1) / kWaves)), block(kWaves * 64);
  const bool b = a.dtype == ATP_BF16, e = a.cache_dtype == ATP_E4M3;
  if (b && e)
    hipLaunchKernelGGL((k_attend<__bf16, E4M3>), grid, block, 0, st, a);
  else if (b)
    hipLaunchKernelGGL((k_attend<__bf16, __bf16>), grid, block, 0, st, a);
  else if (e)
    hipLaunchKernelGGL((k_attend<_Float16, E4M3>), grid, block, 0, st, a);
  else
    hipLaunchKernelGGL((k_attend<_Float16, _Float16>), grid, block, 0, st, a);
  kv_hip(hipGetLastError(), "atp_kv_attend");
}

}  // namespace atp
