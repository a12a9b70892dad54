// attend.hip — attention of a step's tokens over the paged cache
// (atp_kv_attend).
#include <algorithm>

#include "attend.h"

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

// Joins a row's chunks: out = sum 2^(lse_c - max) out_c / sum 2^(lse_c - max),
// each chunk's out_c being its own weighted mean.  One workgroup per row and
// head; 16, 32 or 64 lanes hold its dimensions, 4 each, and as many groups of
// lanes take chunks in turn; their sums are added in a fixed order.
constexpr int kJoinThreads = 256;
template <typename T>
__global__ void __launch_bounds__(kJoinThreads) k_join(AttendKernel a, int32_t align, int32_t lanes) {
  __shared__ float red[kJoinThreads / 64], red2[kJoinThreads / 64];
  __shared__ float4 acc[kJoinThreads];
  const int32_t item = blockIdx.x, h = item % a.h.n_q, i = item / a.h.n_q % a.max_fresh, s = item / a.h.n_q / a.max_fresh;
  const Seq q = sequence(a, s);
  if (!q.ok || i >= q.n) return;
  const int tid = threadIdx.x, groups = blockDim.x / lanes, waves = blockDim.x / 64;
  const int32_t span = q.ctx - first_seen(a, q.cached, align);
  const int32_t chunks = min(a.split.n_split, max(1, (span + a.split.chunk - 1) / a.split.chunk));
  const int64_t row = int64_t(q.r0 + i) * a.h.n_q + h;
  const float *lse = a.split.part_lse + row * a.split.n_split;
  float most = -INFINITY, total = 0;
  for (int c = tid; c < chunks; c += blockDim.x) most = fmaxf(most, lse[c]);
  for (int d = 32; d; d >>= 1) most = fmaxf(most, __shfl_xor(most, d));
  if ((tid & 63) == 0) red[tid >> 6] = most;
  __syncthreads();
  for (int w = 0; w < waves; ++w) most = fmaxf(most, red[w]);
  const float base = most == -INFINITY ? 0.0f : most;
  for (int c = tid; c < chunks; c += blockDim.x) total += __builtin_amdgcn_exp2f(lse[c] - base);
  for (int d = 32; d; d >>= 1) total += __shfl_xor(total, d);
  if ((tid & 63) == 0) red2[tid >> 6] = total;
  __syncthreads();
  total = 0;
  for (int w = 0; w < waves; ++w) total += red2[w];
  const int at = tid % lanes, group = tid / lanes, d = at * 4, hd = a.c.hd;
  float4 x = {0, 0, 0, 0};
  if (d < hd) {
    const float *part = a.split.part + row * a.split.n_split * hd + d;
#pragma unroll 4
    for (int c = group; c < chunks; c += groups) {
      const float w = __builtin_amdgcn_exp2f(lse[c] - base);
      const float4 y = *reinterpret_cast<const float4 *>(part + int64_t(c) * hd);
      x.x += w * y.x;
      x.y += w * y.y;
      x.z += w * y.z;
      x.w += w * y.w;
    }
  }
  acc[tid] = x;
  __syncthreads();
  if (group == 0 && d < hd) {
    for (int g = 1; g < groups; ++g) {
      const float4 y = acc[g * lanes + at];
      x.x += y.x;
      x.y += y.y;
      x.z += y.z;
      x.w += y.w;
    }
    const float inv = total == 0 ? 0.0f : 1.0f / total;
    T *dst = static_cast<T *>(a.out) + (q.r0 + i) * a.out_stride + int64_t(h) * hd + d;
    *reinterpret_cast<u32x2_t *>(dst) = u32x2_t{pack2<T>(x.x * inv, x.y * inv), pack2<T>(x.z * inv, x.w * inv)};
  }
  if (tid == 0 && a.lse) a.lse[row] = total == 0 ? -INFINITY : (base + __builtin_amdgcn_logf(total)) * kLn2;
}

uint64_t magic_of(uint32_t d) { return d <= 1 ? 0 : ~uint64_t(0) / d + 1; }  // ceil(2^64 / d)

// Rows of a KV head that one sequence brings, at most.
int64_t rows_per_head(const AttendArgs &a) { return int64_t(a.max_fresh) * std::min(a.h.group, a.h.n_q); }

constexpr int64_t kFewRows = 32;
constexpr int32_t kFewAlign = 32;         // chunks of the context begin at multiples of it
constexpr int32_t kFewGroups = 1024;      // workgroups that fill the chip twice over
constexpr int32_t kFewLeast = 256;        // tokens of the shortest chunk

// `most`: chunks that no call with these bounds exceeds, whatever its window.
AttendSplit cut(const AttendArgs &a, int64_t *most) {
  AttendSplit s{0, 1, nullptr, nullptr};
  const int64_t full = int64_t(a.max_ctx) + kFewAlign;
  const int64_t span = a.window > 0 ? std::min<int64_t>(full, int64_t(a.window) + a.max_fresh + kFewAlign) : full;
  s.chunk = int32_t(std::min<int64_t>(span / kFewAlign * kFewAlign + kFewAlign, INT32_MAX / kFewAlign * kFewAlign));
  *most = 1;
  if (rows_per_head(a) > kFewRows) return s;
  const int64_t base = std::max<int64_t>(1, int64_t(a.n_seq) * a.h.n_run), fill = (kFewGroups + base - 1) / base;
  const int64_t parts = std::min(fill, (span + kFewLeast - 1) / kFewLeast);
  *most = std::min(fill, (full + kFewLeast - 1) / kFewLeast);
  s.chunk = int32_t(std::min<int64_t>(((span + parts - 1) / parts + kFewAlign - 1) / kFewAlign * kFewAlign, s.chunk));
  s.n_split = int32_t((span + s.chunk - 1) / s.chunk);
  return s;
}

uint64_t lay_out(const AttendArgs &a, void *ws, AttendSplit *s) {
  int64_t most;
  *s = cut(a, &most);
  if (most == 1) return 0;
  const uint64_t rows = uint64_t(a.max_tokens) * a.h.n_q * uint64_t(most), part = (rows * a.c.hd * 4 + 255) / 256 * 256;
  s->part = static_cast<float *>(ws);
  s->part_lse = reinterpret_cast<float *>(static_cast<char *>(ws) + part);
  return part + (rows * 4 + 255) / 256 * 256;
}

// HIP counts a launch's threads in 32 bits.
dim3 grid_of(int64_t groups, int threads) {
  if (groups * threads >= (int64_t(1) << 32)) throw Error(ATP_EINVAL, "step too large for one launch: n_seq * max_fresh * heads");
  return dim3(uint32_t(groups));
}

}  // namespace

uint64_t attend_workspace(const AttendArgs &a) {
  AttendSplit s;
  return lay_out(a, nullptr, &s);
}

void attend_launch(const AttendArgs &args, void *ws, void *stream) {
  AttendKernel a;
  static_cast<AttendArgs &>(a) = args;
  lay_out(args, ws, &a.split);
  a.bt_magic = magic_of(uint32_t(a.c.bt));
  const bool b = a.dtype == ATP_BF16, e = a.cache_dtype == ATP_E4M3;
  const int64_t n = int64_t(a.n_seq) * a.max_fresh * a.h.n_q;
  const dim3 rows = grid_of(n, kJoinThreads);
  if (rows_per_head(a) <= kFewRows) {
    const dim3 work = grid_of(int64_t(a.n_seq) * a.h.n_run * a.split.n_split, 256);
    const hipStream_t st = kv_stream(stream);
    attend_few(a, work, st);
    kv_hip(hipGetLastError(), "atp_kv_attend");
    if (a.split.n_split > 1) {
      const int32_t lanes = a.c.hd <= 64 ? 16 : a.c.hd <= 128 ? 32 : 64;
      const dim3 grid = rows, block(a.split.n_split <= 64 / lanes * 4 ? 64 : kJoinThreads);
      if (b)
        hipLaunchKernelGGL((k_join<__bf16>), grid, block, 0, st, a, kFewAlign, lanes);
      else
        hipLaunchKernelGGL((k_join<_Float16>), grid, block, 0, st, a, kFewAlign, lanes);
    }
    kv_hip(hipGetLastError(), "atp_kv_attend");
    return;
  }
  const hipStream_t st = kv_stream(stream);
  const dim3 grid(uint32_t((n + kWaves - 1) / kWaves)), block(kWaves * 64);
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
