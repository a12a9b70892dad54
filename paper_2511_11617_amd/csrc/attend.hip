// attend.hip — attention of a step's tokens over the paged cache
// (atp_kv_attend): which kernel takes the call, how the context is cut over
// workgroups, and the join of the chunks.
#include <algorithm>

#include "attend.h"

namespace atp {
namespace {

// Joins a row's chunks: out = sum 2^(lse_c - max) out_c / sum 2^(lse_c - max),
// each chunk's out_c being its own weighted mean, in a fixed order.  An infinity
// or NaN of V that a chunk's rows saw stays one whatever the chunk's weight.

// Few rows: one workgroup per row and head; 16, 32 or 64 lanes hold its
// dimensions, 4 each, and as many groups of lanes take chunks in turn.
constexpr int kJoinThreads = 256;
constexpr int kMostSplit = 2048;  // at most two rounds of 768 chunks, and one, are one sequence's
template <typename T>
__global__ void __launch_bounds__(kJoinThreads) k_join(AttendKernel a, int32_t lanes) {
  __shared__ float weight[kMostSplit];
  __shared__ float red[kJoinThreads / 64], red2[kJoinThreads / 64];
  __shared__ f32x4 acc[kJoinThreads];
  const int32_t item = blockIdx.x, h = item % a.h.n_q, i = item / a.h.n_q % a.max_fresh, s = item / a.h.n_q / a.max_fresh;
  const Seq q = sequence(a, s);
  if (!q.ok || i >= q.n) return;
  const int tid = threadIdx.x, groups = blockDim.x / lanes, waves = blockDim.x / 64;
  const int64_t row = int64_t(q.r0 + i) * a.h.n_q + h;
  const int32_t chunks = a.split.shares[2 * s + 1];
  if (chunks <= 1) return;  // written already
  const int32_t run = (h + a.h.cut) / a.h.group;
  int32_t h0;
  const int32_t gh = run_heads(a.h, run, &h0);
  const int64_t step = int64_t(a.h.n_run) * a.split.n_split;  // from chunk to chunk
  const int64_t first = (int64_t(a.split.shares[2 * s]) * a.h.n_run + run) * a.split.n_split + i * gh + h - h0;
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
        if (c < chunks) y[j] = *reinterpret_cast<const f32x4 *>(part + c * step * hd);
      }
#pragma unroll
      for (int j = 0; j < kAhead; ++j) add_share(x, y[j], w[j]);
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

// Many rows: a workgroup takes 4 rows of a cut tile, `lanes` lanes each (a tile
// cut into hundreds of parts needs many workgroups on them).
constexpr int kJoinRows = 4;
template <typename T>
__global__ void __launch_bounds__(kJoinThreads) k_join_tiles(AttendKernel a, int32_t lanes) {
  const int32_t item = blockIdx.x / (kTileRows / kJoinRows), part = blockIdx.x % (kTileRows / kJoinRows);
  const int32_t place = a.split.cuts[2 * item], parts = a.split.cuts[2 * item + 1];
  if (parts <= 1) return;
  const TileItem t = tile_of(a, item);
  int32_t h0;
  const int32_t gh = run_heads(a.h, t.run, &h0), rows = t.n * gh, hd = a.c.hd;
  const int at = threadIdx.x % lanes, d = at * 4;
  const int32_t in = part * kJoinRows + threadIdx.x / lanes, r = t.tile * kTileRows + in;
  if (r < rows) {
    const float *lse = a.split.part_lse + int64_t(place) * kTileRows + in;
    float most = -INFINITY, total = 0;
    for (int c = at; c < parts; c += lanes) most = fmaxf(most, lse[int64_t(c) * kTileRows]);
    for (int e = lanes / 2; e; e >>= 1) most = fmaxf(most, __shfl_xor(most, e));
    const float base = most == -INFINITY ? 0.0f : most;
    f32x4 o = {0, 0, 0, 0};
    constexpr int kAhead = 4;
    for (int c0 = 0; c0 < parts; c0 += kAhead) {
      f32x4 y[kAhead];
      float w[kAhead];
#pragma unroll
      for (int j = 0; j < kAhead; ++j) {
        const int64_t from = (int64_t(place) + c0 + j) * kTileRows + in;
        w[j] = c0 + j < parts ? a.split.part_lse[from] : -INFINITY;
        y[j] = f32x4{0, 0, 0, 0};
        if (c0 + j < parts && d < hd) y[j] = *reinterpret_cast<const f32x4 *>(a.split.part + from * hd + d);
      }
#pragma unroll
      for (int j = 0; j < kAhead; ++j) {
        const float v = __builtin_amdgcn_exp2f(w[j] - base);
        total += v;
        add_share(o, y[j], v);
      }
    }
    const float inv = total == 0 ? 0.0f : 1.0f / total;
    const int32_t i = r / gh, h = h0 + r % gh;
    if (d < hd) {
      T *dst = static_cast<T *>(a.out) + (t.r0 + i) * a.out_stride + int64_t(h) * hd + d;
      *reinterpret_cast<u32x2_t *>(dst) = u32x2_t{pack2<T>(o[0] * inv, o[1] * inv), pack2<T>(o[2] * inv, o[3] * inv)};
    }
    if (at == 0 && a.lse) a.lse[int64_t(t.r0 + i) * a.h.n_q + h] = total == 0 ? -INFINITY : (base + __builtin_amdgcn_logf(total)) * kLn2;
  }
}

// The list of many rows' work, by one workgroup: tiles longer than the chip's
// share (their tokens over kTileParts) are cut into equal parts, and all go
// into the list longest first (32 classes of length), so that the last ones to
// begin are short.  (One prompt of 8192 behind 8192, 576 tiles: cut to shares of
// 1/640 535 to 557 us, of 1/1024 554, of 1/512 574, not cut 639; 1222 tiles of ragged
// prompts: not cut 158, cut to 1/640 172, not cut and in no order of length 212.
// At 256 dimensions, where the chip holds 256 tiles, 4096 behind 4096: 1/640 432,
// 1/256 490, 1/320 460, 1/1024 484.)
constexpr int kListThreads = 1024, kListTiles = 4096, kClasses = 32;
constexpr int32_t kTileParts = 640, kTileLeast = 512;
__global__ void __launch_bounds__(kListThreads) k_list_tiles(AttendKernel a, bool cut) {
  constexpr int kEach = kListTiles / kListThreads;
  __shared__ int64_t sums[kListThreads / 64];
  __shared__ int32_t spans[kListThreads / 64];
  __shared__ int32_t count[kClasses], from[kClasses], places, n;
  const int tid = threadIdx.x;
  for (int32_t s = tid; s < a.n_seq; s += kListThreads)
    if (!sequence(a, s).ok) flag(a.status, ATP_EINVAL);
  TileItem t[kEach];
  int64_t total = 0;
  int32_t longest = 0;
#pragma unroll
  for (int j = 0; j < kEach; ++j) {
    const int32_t item = j * kListThreads + tid;
    t[j].s = -1;
    if (item < a.split.tiles) t[j] = tile_of(a, item);
    if (t[j].s < 0) continue;
    total += t[j].hi - t[j].lo;
    longest = max(longest, t[j].hi - t[j].lo);
  }
  for (int d = 32; d; d >>= 1) {
    total += __shfl_xor(total, d);
    longest = max(longest, __shfl_xor(longest, d));
  }
  if ((tid & 63) == 0) {
    sums[tid >> 6] = total;
    spans[tid >> 6] = longest;
  }
  if (tid < kClasses) count[tid] = 0;
  if (tid == 0) places = n = 0;
  __syncthreads();
  total = 0;
  for (int w = 0; w < kListThreads / 64; ++w) {
    total += sums[w];
    longest = max(longest, spans[w]);
  }
  int32_t most = int32_t(min(max((total + kTileParts - 1) / kTileParts, int64_t(kTileLeast)), int64_t(1) << 30));
  if (!cut) most = 1 << 30;
  const int32_t scale = min(most, longest);  // of the classes; the host's bounds may be far above it
  int32_t parts[kEach], length[kEach], at[kEach];
#pragma unroll
  for (int j = 0; j < kEach; ++j) {
    parts[j] = 0;
    if (t[j].s < 0) continue;
    const int32_t span = t[j].hi - t[j].lo, want = (span + most - 1) / most;
    length[j] = ((span + want - 1) / want + kTileAlign - 1) / kTileAlign * kTileAlign;
    parts[j] = (span + length[j] - 1) / length[j];
    // class 0 is the longest
    const int32_t cls = kClasses - 1 - int32_t(min(int64_t(length[j]) * kClasses / (int64_t(scale) + 1), int64_t(kClasses - 1)));
    at[j] = cls << 24 | atomicAdd(&count[cls], parts[j]);
  }
  __syncthreads();
  if (tid == 0) {
    int32_t sum = 0;
    for (int c = 0; c < kClasses; ++c) {
      from[c] = sum;
      sum += count[c];
    }
    n = sum;
  }
  __syncthreads();
  for (int32_t i = n + tid; i < a.split.n_items; i += kListThreads) a.split.items[i].s = -1;
#pragma unroll
  for (int j = 0; j < kEach; ++j) {
    const int32_t item = j * kListThreads + tid;
    if (item >= a.split.tiles) continue;
    const int32_t place = parts[j] > 1 ? atomicAdd(&places, parts[j]) : -1;
    a.split.cuts[2 * item] = place;
    a.split.cuts[2 * item + 1] = parts[j];
    if (!parts[j]) continue;
    const int32_t first = from[at[j] >> 24] + (at[j] & 0xffffff);
    for (int k = 0; k < parts[j]; ++k) {
      TileItem one = t[j];
      one.lo = t[j].lo + k * length[j];
      one.hi = min(t[j].hi, one.lo + length[j]);
      one.place = parts[j] > 1 ? place + k : -1;
      a.split.items[first + k] = one;
    }
  }
}

uint64_t magic_of(uint32_t d) { return d <= 1 ? 0 : ~uint64_t(0) / d + 1; }  // ceil(2^64 / d)

// Rows of a KV head that one sequence brings, at most.
int64_t rows_per_head(const AttendArgs &a) { return int64_t(a.max_fresh) * std::min(a.h.group, a.h.n_q); }

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
  bool cut;  // many rows: tiles may be cut
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
  p.workgroups += (p.workgroups > p.split.groups ? 2 : 1) * p.split.groups;  // as few_rounds(); each sequence's last chunk may be short
  const uint64_t rows = uint64_t(p.workgroups) * uint64_t(p.split.n_split);
  p.split.part = reinterpret_cast<float *>(ws);
  p.split.part_lse = reinterpret_cast<float *>(ws + padded(rows * a.c.hd * 4));
  p.split.shares = reinterpret_cast<int32_t *>(ws + padded(rows * a.c.hd * 4) + padded(rows * 4));
  p.bytes = padded(rows * a.c.hd * 4) + padded(rows * 4) + padded(uint64_t(a.n_seq) * 8);
  return p;
}

// A call that fits the chip at once with short contexts needs no list, and one
// of more tiles than a list takes is even enough without.
AttendPlan plan_tiles(const AttendArgs &a, char *ws) {
  AttendPlan p{};
  AttendSplit &s = p.split;
  p.workgroups = groups_of(a);
  const int64_t fits = a.c.hd > 128 ? 256 : 512;
  if (p.workgroups > kListTiles || (p.workgroups <= fits && a.max_ctx <= kTileLeast)) return p;
  s.tiles = int32_t(p.workgroups);
  // cut where some of a step's tiles may be longer than the chip's share
  const int64_t each = (int64_t(a.max_ctx) + kTileAlign + kTileLeast - 1) / kTileLeast;  // parts of a tile, at most
  p.cut = p.workgroups < 2 * fits && each > 1;
  const int64_t places = p.cut ? std::min<int64_t>(2 * kTileParts, p.workgroups * each) : 0;
  if (p.cut) p.workgroups += std::min<int64_t>(kTileParts, p.workgroups * each);
  const uint64_t rows = uint64_t(places) * kTileRows;
  uint64_t at = 0;
  auto take = [&](uint64_t bytes) {
    char *q = ws + at;
    at += padded(bytes);
    return q;
  };
  s.n_items = int32_t(p.workgroups);
  s.items = reinterpret_cast<TileItem *>(take(uint64_t(p.workgroups) * sizeof(TileItem)));
  s.cuts = reinterpret_cast<int32_t *>(take(uint64_t(s.tiles) * 8));
  s.part = reinterpret_cast<float *>(take(rows * a.c.hd * 4));
  s.part_lse = reinterpret_cast<float *>(take(rows * 4));
  p.bytes = at;
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
  const bool joined = few(a) ? a.split.n_split > 0 : p.cut;
  const int64_t join_groups = few(a) ? int64_t(a.n_seq) * a.max_fresh * a.h.n_q : int64_t(a.split.tiles) * (kTileRows / kJoinRows);
  const dim3 rows = joined ? grid_of(join_groups, kJoinThreads) : dim3(1);
  const hipStream_t st = kv_stream(stream);
  const int32_t lanes = a.c.hd <= 64 ? 16 : a.c.hd <= 128 ? 32 : 64;
  const bool b = a.dtype == ATP_BF16;
  if (few(a)) {
    attend_few(a, work, st);
    kv_hip(hipGetLastError(), "atp_kv_attend");
    if (!joined) return;
    const dim3 block(a.split.groups / groups_of(a) > 64 / lanes * 4 ? kJoinThreads : 64);  // by a sequence's chunks, about
    if (b)
      hipLaunchKernelGGL((k_join<__bf16>), rows, block, 0, st, a, lanes);
    else
      hipLaunchKernelGGL((k_join<_Float16>), rows, block, 0, st, a, lanes);
  } else {
    if (a.split.tiles) {
      hipLaunchKernelGGL(k_list_tiles, dim3(1), dim3(kListThreads), 0, st, a, p.cut);
      kv_hip(hipGetLastError(), "atp_kv_attend");
    }
    attend_tiles(a, work, st);
    kv_hip(hipGetLastError(), "atp_kv_attend");
    if (!joined) return;
    if (b)
      hipLaunchKernelGGL((k_join_tiles<__bf16>), rows, dim3(kJoinRows * lanes), 0, st, a, lanes);
    else
      hipLaunchKernelGGL((k_join_tiles<_Float16>), rows, dim3(kJoinRows * lanes), 0, st, a, lanes);
  }
  kv_hip(hipGetLastError(), "atp_kv_attend");
}

}  // namespace atp
