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
constexpr int kMostSplit = 1024;
template <typename T>
__global__ void __launch_bounds__(kJoinThreads) k_join(AttendKernel a, int32_t lanes, bool few_rows) {
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
  const int64_t row = int64_t(q.r0 + i) * a.h.n_q + h;
  int32_t chunks;
  int64_t first, step;  // places of the row's chunks
  if (few_rows) {
    chunks = a.split.shares[2 * s + 1];
    if (chunks <= 1) return;  // written already
    const int32_t run = (h + a.h.cut) / a.h.group;
    int32_t h0;
    const int32_t gh = run_heads(a.h, run, &h0);
    step = int64_t(a.h.n_run) * a.split.n_split;
    first = (int64_t(a.split.shares[2 * s]) * a.h.n_run + run) * a.split.n_split + i * gh + h - h0;
  } else {
    const int32_t span = q.ctx - first_seen(a, q.cached, kTileAlign);
    chunks = min(a.split.n_split, max(1, (span + a.split.chunk - 1) / a.split.chunk));
    step = 1;
    first = row * a.split.n_split;
  }
  const float *lse = a.split.part_lse + first;
  float most = -INFINITY, total = 0;
  for (int c = tid; c < chunks; c += blockDim.x) {
    weight[c] = lse[c * step];
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
    const float *part = a.split.part + first * hd + d;
    constexpr int kAhead = 4;
    for (int c0 = group; c0 < chunks; c0 += kAhead * groups) {
      f32x4 y[kAhead];
      float w[kAhead];
#pragma unroll
      for (int j = 0; j < kAhead; ++j) {
        const int c = c0 + j * groups;
        w[j] = c < chunks ? weight[c] : 0.0f;
        y[j] = f32x4{0, 0, 0, 0};
        if (w[j] != 0) y[j] = *reinterpret_cast<const f32x4 *>(part + c * step * hd);  // of 0: nothing may have been written
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

constexpr int32_t kTileGroups = 1024;  // workgroups of many rows that fill the chip
constexpr int32_t kTileLeast = 512;                       // tokens of the shortest chunk of many rows

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

uint64_t padded(uint64_t bytes) { return (bytes + 255) / 256 * 256; }

// Where the call's chunks are kept, and how many workgroups it takes.
struct AttendPlan {
  AttendSplit split;
  int64_t workgroups;
  uint64_t bytes;
};

// Workgroups of few rows that the chip holds at once: one round of long chunks
// beat two of half the length (8192 tokens of 128 sessions: 192 against 197 us).
int32_t few_groups(const AttendArgs &a) {
  if (a.c.hd > 128 || (a.c.hd > 64 && rows_per_head(a) > 16)) return 256;
  return a.c.hd > 64 ? 512 : 768;
}

AttendPlan plan_few(const AttendArgs &a, char *ws) {
  AttendPlan p{};
  p.split.groups = few_groups(a);
  p.split.n_split = rows_per_head(a) > 16 ? 32 : 16;  // rows of a workgroup's place
  p.workgroups = groups_of(a);
  if (a.max_ctx <= kFewLeast) {  // no sequence takes two chunks
    p.split.n_split = 0;
    return p;
  }
  p.workgroups += p.split.groups;  // each sequence's last chunk may be short
  const uint64_t rows = uint64_t(p.workgroups) * uint64_t(p.split.n_split);
  p.split.part = reinterpret_cast<float *>(ws);
  p.split.part_lse = reinterpret_cast<float *>(ws + padded(rows * a.c.hd * 4));
  p.split.shares = reinterpret_cast<int32_t *>(ws + padded(rows * a.c.hd * 4) + padded(rows * 4));
  p.bytes = padded(rows * a.c.hd * 4) + padded(rows * 4) + padded(uint64_t(a.n_seq) * 8);
  return p;
}

// The workspace holds what no call with these bounds exceeds, whatever its window.
AttendPlan plan_tiles(const AttendArgs &a, char *ws) {
  AttendPlan p{};
  AttendSplit &s = p.split;
  const int64_t full = int64_t(a.max_ctx) + kTileAlign;
  const int64_t span = a.window > 0 ? std::min<int64_t>(full, int64_t(a.window) + a.max_fresh + kTileAlign) : full;
  const int64_t base = std::max<int64_t>(1, groups_of(a)), fill = (kTileGroups + base - 1) / base;
  const int64_t parts = std::min(fill, (span + kTileLeast - 1) / kTileLeast), most = std::min(fill, (full + kTileLeast - 1) / kTileLeast);
  s.chunk = int32_t(((span + parts - 1) / parts + kTileAlign - 1) / kTileAlign * kTileAlign);
  s.n_split = int32_t((span + s.chunk - 1) / s.chunk);
  p.workgroups = base * s.n_split;
  if (most == 1) return p;
  const uint64_t rows = uint64_t(a.max_tokens) * a.h.n_q * uint64_t(most);
  s.part = reinterpret_cast<float *>(ws);
  s.part_lse = reinterpret_cast<float *>(ws + padded(rows * a.c.hd * 4));
  p.bytes = padded(rows * a.c.hd * 4) + padded(rows * 4);
  return p;
}

AttendPlan plan(const AttendArgs &a, void *ws) {
  return few(a) ? plan_few(a, static_cast<char *>(ws)) : plan_tiles(a, static_cast<char *>(ws));
}

// HIP counts a launch's threads in 32 bits.
dim3 grid_of(int64_t groups, int threads) {
  if (groups * threads >= (int64_t(1) << 32)) throw Error(ATP_EINVAL, "step too large for one launch: n_seq * max_fresh * heads");
  return dim3(uint32_t(groups));
}

}  // namespace

uint64_t attend_workspace(const AttendArgs &a) { return plan(a, nullptr).bytes; }

void attend_launch(const AttendArgs &args, void *ws, void *stream) {
  AttendKernel a;
  static_cast<AttendArgs &>(a) = args;
  const AttendPlan p = plan(args, ws);
  a.split = p.split;
  a.bt_magic = magic_of(uint32_t(a.c.bt));
  const dim3 work = grid_of(p.workgroups, 256);
  const bool joined = few(a) ? a.split.n_split > 0 : a.split.n_split > 1;
  const int64_t rows_each = few(a) ? int64_t(a.n_seq) * a.max_fresh : a.max_tokens;
  const dim3 rows = joined ? grid_of(rows_each * a.h.n_q, kJoinThreads) : dim3(1);
  const hipStream_t st = kv_stream(stream);
  if (few(a))
    attend_few(a, work, st);
  else
    attend_tiles(a, work, st);
  kv_hip(hipGetLastError(), "atp_kv_attend");
  if (joined) {
    const int32_t lanes = a.c.hd <= 64 ? 16 : a.c.hd <= 128 ? 32 : 64;
    // chunks of a sequence, about
    const int64_t chunks = few(a) ? a.split.groups / groups_of(a) : a.split.n_split;
    const dim3 block(chunks > 64 / lanes * 4 ? kJoinThreads : 64);
    if (a.dtype == ATP_BF16)
      hipLaunchKernelGGL((k_join<__bf16>), rows, block, 0, st, a, lanes, few(a));
    else
      hipLaunchKernelGGL((k_join<_Float16>), rows, block, 0, st, a, lanes, few(a));
    kv_hip(hipGetLastError(), "atp_kv_attend");
  }
}

}  // namespace atp
