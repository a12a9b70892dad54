// attend.hip — attention of a step's tokens over the paged cache
// (atp_kv_attend): which kernel takes the call, how the context is cut over
// workgroups, and the join of the chunks.
#include <algorithm>

#include "attend.h"

namespace atp {
namespace {

// Joins a row's chunks: out = sum 2^(lse_c - max) out_c / sum 2^(lse_c - max),
// each chunk's out_c being its own weighted mean.  One workgroup per row and
// head; 16, 32 or 64 lanes hold its dimensions, 4 each, and as many groups of
// lanes take chunks in turn; their sums are added in a fixed order.
constexpr int kJoinThreads = 256;
constexpr int kMostSplit = 512;
template <typename T>
__global__ void __launch_bounds__(kJoinThreads) k_join(AttendKernel a, int32_t align, int32_t lanes, bool few_rows) {
  __shared__ float weight[kMostSplit];
  __shared__ float red[kJoinThreads / 64], red2[kJoinThreads / 64];
  __shared__ f32x4 acc[kJoinThreads];
  const int32_t item = blockIdx.x, h = item % a.h.n_q, at_row = item / a.h.n_q;
  int32_t s, i;
  if (few_rows) {  // a place for each sequence's most rows
    s = at_row / a.max_fresh;
    i = at_row % a.max_fresh;
  } else {  // the rows as they lie: the last sequence that starts at or before this one
    s = 0;
    for (int32_t hi = a.n_seq - 1; s < hi;) {
      const int32_t mid = (s + hi + 1) >> 1;
      if (a.starts[mid] <= at_row)
        s = mid;
      else
        hi = mid - 1;
    }
    i = at_row - a.starts[s];
  }
  const Seq q = sequence(a, s);
  if (!q.ok || i < 0 || i >= q.n) return;
  const int tid = threadIdx.x, groups = blockDim.x / lanes, waves = blockDim.x / 64;
  const int32_t span = q.ctx - first_seen(a, q.cached, align);
  const int32_t chunks = min(a.split.n_split, max(1, (span + a.split.chunk - 1) / a.split.chunk));
  const int64_t row = int64_t(q.r0 + i) * a.h.n_q + h;
  const float *lse = a.split.part_lse + row * a.split.n_split;
  float most = -INFINITY, total = 0;
  for (int c = tid; c < chunks; c += blockDim.x) {
    weight[c] = lse[c];
    most = fmaxf(most, weight[c]);
  }
  for (int d = 32; d; d >>= 1) most = fmaxf(most, __shfl_xor(most, d));
  if ((tid & 63) == 0) red[tid >> 6] = most;
  __syncthreads();
  for (int w = 0; w < waves; ++w) most = fmaxf(most, red[w]);
  const float base = most == -INFINITY ? 0.0f : most;
  for (int c = tid; c < chunks; c += blockDim.x) {
    weight[c] = __builtin_amdgcn_exp2f(weight[c] - base);
    total += weight[c];
  }
  for (int d = 32; d; d >>= 1) total += __shfl_xor(total, d);
  if ((tid & 63) == 0) red2[tid >> 6] = total;
  __syncthreads();
  total = 0;
  for (int w = 0; w < waves; ++w) total += red2[w];
  const int at = tid % lanes, group = tid / lanes, d = at * 4, hd = a.c.hd;
  f32x4 x = {0, 0, 0, 0};
  if (d < hd) {
    const float *part = a.split.part + row * a.split.n_split * hd + d;
    constexpr int kAhead = 4;
    for (int c0 = group; c0 < chunks; c0 += kAhead * groups) {
      f32x4 y[kAhead];
      float w[kAhead];
#pragma unroll
      for (int j = 0; j < kAhead; ++j) {
        const int c = c0 + j * groups;
        w[j] = c < chunks ? weight[c] : 0.0f;
        y[j] = f32x4{0, 0, 0, 0};
        if (w[j] != 0) y[j] = *reinterpret_cast<const f32x4 *>(part + int64_t(c) * hd);  // of 0: nothing may have been written
      }
#pragma unroll
      for (int j = 0; j < kAhead; ++j) x += w[j] * y[j];
    }
  }
  acc[tid] = x;
  __syncthreads();
  if (group == 0 && d < hd) {
    for (int g = 1; g < groups; ++g) x += acc[g * lanes + at];
    const float inv = total == 0 ? 0.0f : 1.0f / total;
    T *dst = static_cast<T *>(a.out) + (q.r0 + i) * a.out_stride + int64_t(h) * hd + d;
    *reinterpret_cast<u32x2_t *>(dst) = u32x2_t{pack2<T>(x[0] * inv, x[1] * inv), pack2<T>(x[2] * inv, x[3] * inv)};
  }
  if (tid == 0 && a.lse) a.lse[row] = total == 0 ? -INFINITY : (base + __builtin_amdgcn_logf(total)) * kLn2;
}

uint64_t magic_of(uint32_t d) { return d <= 1 ? 0 : ~uint64_t(0) / d + 1; }  // ceil(2^64 / d)

// Rows of a KV head that one sequence brings, at most.
int64_t rows_per_head(const AttendArgs &a) { return int64_t(a.max_fresh) * std::min(a.h.group, a.h.n_q); }

constexpr int32_t kFewGroups = 512, kTileGroups = 1024;  // workgroups that fill the chip
constexpr int32_t kFewLeast = 256, kTileLeast = 512;     // tokens of the shortest chunk

// The kernel of few rows holds two tiles of 16, one of more than 128 dimensions.
bool few(const AttendArgs &a) { return rows_per_head(a) <= (a.c.hd <= 128 ? 32 : 16); }

// Workgroups of one chunk that a call takes.
int64_t groups_of(const AttendArgs &a) {
  if (few(a)) return int64_t(a.n_seq) * a.h.n_run;
  int64_t n = 0;
  for (int32_t j = 0; j < a.h.n_run; ++j) {
    int32_t h0;
    n += tile_slots(a, run_heads(a.h, j, &h0));
  }
  return n;
}

// `most`: chunks that no call with these bounds exceeds, whatever its window.
AttendSplit cut(const AttendArgs &a, int64_t *most) {
  AttendSplit s{0, 1, nullptr, nullptr};
  const int32_t align = few(a) ? kFewAlign : kTileAlign, least = few(a) ? kFewLeast : kTileLeast;
  const int64_t groups = groups_of(a), wanted = few(a) ? kFewGroups : kTileGroups;
  const int64_t full = int64_t(a.max_ctx) + align;
  const int64_t span = a.window > 0 ? std::min<int64_t>(full, int64_t(a.window) + a.max_fresh + align) : full;
  const int64_t base = std::max<int64_t>(1, groups), fill = (wanted + base - 1) / base;  // at most kMostSplit
  const int64_t parts = std::min(fill, (span + least - 1) / least);
  *most = std::min(fill, (full + least - 1) / least);
  s.chunk = int32_t(((span + parts - 1) / parts + align - 1) / align * align);
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
  const dim3 work = grid_of(groups_of(a) * a.split.n_split, 256);
  const int64_t rows_each = few(a) ? int64_t(a.n_seq) * a.max_fresh : a.max_tokens;
  const dim3 rows = a.split.n_split > 1 ? grid_of(rows_each * a.h.n_q, kJoinThreads) : dim3(1);
  const hipStream_t st = kv_stream(stream);
  if (few(a))
    attend_few(a, work, st);
  else
    attend_tiles(a, work, st);
  kv_hip(hipGetLastError(), "atp_kv_attend");
  if (a.split.n_split > 1) {
    const int32_t lanes = a.c.hd <= 64 ? 16 : a.c.hd <= 128 ? 32 : 64, align = few(a) ? kFewAlign : kTileAlign;
    const dim3 block(a.split.n_split <= 64 / lanes * 4 ? 64 : kJoinThreads);
    if (a.dtype == ATP_BF16)
      hipLaunchKernelGGL((k_join<__bf16>), rows, block, 0, st, a, align, lanes, few(a));
    else
      hipLaunchKernelGGL((k_join<_Float16>), rows, block, 0, st, a, align, lanes, few(a));
    kv_hip(hipGetLastError(), "atp_kv_attend");
  }
}

}  // namespace atp
