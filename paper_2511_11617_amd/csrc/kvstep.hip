// kvstep.hip — a serving step's bookkeeping and writes: places for the new
// tokens (atp_kv_extend), rotary positions and the write of k and v into the
// cache (atp_kv_append).
#include "kvdev.h"

namespace atp {
namespace {

// ---- atp_kv_extend ----------------------------------------------------------
// Mathematics: the free ids are the zeros of a bitmap in which every table
// entry sets its bit; the k-th wanted entry, in (sequence, block) order,
// takes the k-th zero.  Both orders are exclusive prefix sums (of wanted
// entries over sequences, of zeros over bitmap words).  A second bitmap holds
// the ids that two entries name.

constexpr int kStepThreads = 256;
constexpr int kScanThreads = 1024;

// Workspace: the two bitmaps, free ids' rank before each word, wanted
// entries before each sequence, the free ids that are given out (ascending),
// and what k_scan found.
struct ExtendWs {
  uint32_t *used, *shared;
  int32_t *rank;    // [words]
  int32_t *before;  // [n_seq]
  int32_t *list;    // [num_blocks]
  int32_t *found;   // [0] a bad id was seen, [1] blocks taken (-1: the step failed)
};

__host__ __device__ inline int32_t words_of(int32_t num_blocks) { return int32_t((uint32_t(num_blocks) + 31) / 32); }

__device__ inline int32_t wave_sum(int32_t x) {
  for (int d = 32; d; d >>= 1) x += __shfl_xor(x, d);
  return x;
}

// Exclusive sum over the workgroup's threads; *total gets the whole sum.
__device__ inline int64_t block_scan(int64_t x, int64_t *total, int64_t *lds) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, waves = blockDim.x >> 6;
  int64_t inc = x;
  for (int d = 1; d < 64; d <<= 1) {
    const int64_t y = __shfl_up(inc, d);
    if (lane >= d) inc += y;
  }
  __syncthreads();
  if (lane == 63) lds[wave] = inc;
  __syncthreads();
  int64_t base = 0, all = 0;
  for (int w = 0; w < waves; ++w) {
    if (w < wave) base += lds[w];
    all += lds[w];
  }
  *total = all;
  return base + inc - x;
}

// The blocks [b, e) that sequence s's new tokens lie in (empty for none).
__device__ inline void new_range(const ExtendArgs &a, int32_t s, int32_t *b, int32_t *e) {
  const int32_t c = a.cached[s], f = a.fresh[s];
  *b = c / a.bt;
  *e = f ? int32_t((int64_t(c) + f + a.bt - 1) / a.bt) : *b;
}

__global__ void __launch_bounds__(kStepThreads) k_clear(uint32_t *p, int32_t n) {
  for (int64_t i = blockIdx.x * int64_t(kStepThreads) + threadIdx.x; i < n; i += int64_t(gridDim.x) * kStepThreads) p[i] = 0;
}

__global__ void __launch_bounds__(kStepThreads) k_mark(ExtendArgs a, ExtendWs w) {
  const int64_t n = int64_t(a.n_seq) * a.max_blocks;
  for (int64_t i = blockIdx.x * int64_t(kStepThreads) + threadIdx.x; i < n; i += int64_t(gridDim.x) * kStepThreads) {
    const int32_t p = a.table[i];
    if (a.new_table != a.table) a.new_table[i] = p;
    if (p < -1 || p >= a.num_blocks) {
      w.found[0] = 1;
    } else if (p >= 0) {
      const uint32_t bit = 1u << (p & 31);
      if (atomicOr(&w.used[p >> 5], bit) & bit) atomicOr(&w.shared[p >> 5], bit);
    }
  }
}

// One workgroup: lengths, starts, wanted entries, free ids and the verdict.
__global__ void __launch_bounds__(kScanThreads) k_scan(ExtendArgs a, ExtendWs w) {
  __shared__ int64_t lds[kScanThreads / 64];
  __shared__ int32_t bad;
  const int tid = threadIdx.x;
  if (tid == 0) bad = w.found[0];
  __syncthreads();
  const int64_t room = int64_t(a.max_blocks) * a.bt;
  int64_t tokens = 0;
  for (int32_t s0 = 0; s0 < a.n_seq; s0 += kScanThreads) {
    const int32_t s = s0 + tid;
    int64_t f = 0;
    if (s < a.n_seq) {
      const int32_t c = a.cached[s];
      f = a.fresh[s];
      if (c < 0 || f < 0 || int64_t(c) + f > room) bad = 1;
    }
    int64_t sum;
    const int64_t at = tokens + block_scan(f, &sum, lds);
    if (s < a.n_seq) a.starts[s] = int32_t(at);
    tokens += sum;
  }
  if (tid == 0 && tokens > a.max_tokens) bad = 1;
  __syncthreads();
  const bool in_range = !bad;  // read by every thread before one sets it again
  __syncthreads();
  int64_t wanted = 0, free_ids = 0;
  if (in_range) {  // every length is: the table may be indexed by it
    const int lane = tid & 63, wave = tid >> 6;
    for (int32_t s = wave; s < a.n_seq; s += kScanThreads / 64) {
      int32_t b, e, n = 0;
      new_range(a, s, &b, &e);
      for (int32_t i = b + lane; i < e; i += 64) {
        const int32_t p = a.table[int64_t(s) * a.max_blocks + i];
        if (p < 0)
          ++n;
        else if (w.shared[p >> 5] >> (p & 31) & 1)
          bad = 1;
      }
      n = wave_sum(n);
      if (lane == 0) w.before[s] = n;
    }
    __syncthreads();
    for (int32_t s0 = 0; s0 < a.n_seq; s0 += kScanThreads) {
      const int32_t s = s0 + tid;
      int64_t sum = 0;
      const int64_t at = wanted + block_scan(s < a.n_seq ? w.before[s] : 0, &sum, lds);
      if (s < a.n_seq) w.before[s] = int32_t(at);
      wanted += sum;
    }
    const int32_t words = words_of(a.num_blocks);
    for (int32_t i0 = 0; i0 < words; i0 += kScanThreads) {
      const int32_t i = i0 + tid;
      int64_t n = 0, sum;
      if (i < words) n = min(32, a.num_blocks - i * 32) - __popc(w.used[i]);
      const int64_t at = free_ids + block_scan(n, &sum, lds);
      if (i < words) w.rank[i] = int32_t(at);
      free_ids += sum;
    }
  }
  __syncthreads();
  const int32_t code = bad ? ATP_EINVAL : wanted > free_ids ? ATP_ECAPACITY : ATP_OK;
  if (code != ATP_OK)
    for (int32_t s = tid; s < a.n_seq; s += kScanThreads) a.starts[s] = 0;
  if (tid == 0) {
    a.starts[a.n_seq] = code == ATP_OK ? int32_t(tokens) : 0;
    a.status[0] = code;
    a.status[1] = code == ATP_OK ? int32_t(tokens) : 0;
    a.status[2] = bad ? 0 : int32_t(wanted);
    a.status[3] = bad ? 0 : int32_t(code == ATP_OK ? free_ids - wanted : free_ids);
    w.found[1] = code == ATP_OK ? int32_t(wanted) : -1;
  }
}

__global__ void __launch_bounds__(kStepThreads) k_list(ExtendArgs a, ExtendWs w) {
  const int32_t taken = w.found[1], words = words_of(a.num_blocks);
  if (taken <= 0) return;  // after a refusal, rank holds nothing
  for (int32_t i = blockIdx.x * kStepThreads + threadIdx.x; i < words; i += gridDim.x * kStepThreads) {
    int32_t r = w.rank[i];
    if (r >= taken) continue;
    const int32_t n = min(32, a.num_blocks - i * 32);
    uint32_t left = ~w.used[i] & (n == 32 ? ~0u : (1u << n) - 1);
    for (; left && r < taken; left &= left - 1) w.list[r++] = i * 32 + __ffs(left) - 1;
  }
}

// One wave per sequence.
__global__ void __launch_bounds__(kStepThreads) k_fill(ExtendArgs a, ExtendWs w) {
  if (w.found[1] < 0) return;
  const int lane = threadIdx.x & 63, waves = gridDim.x * (kStepThreads / 64);
  for (int32_t s = blockIdx.x * (kStepThreads / 64) + (threadIdx.x >> 6); s < a.n_seq; s += waves) {
    int32_t b, e, at = w.before[s];
    new_range(a, s, &b, &e);
    for (int32_t i0 = b; i0 < e; i0 += 64) {
      const int32_t i = i0 + lane;
      const int64_t cell = int64_t(s) * a.max_blocks + i;
      const bool want = i < e && a.table[cell] < 0;
      const uint64_t who = __ballot(want);
      if (want) a.new_table[cell] = w.list[at + __popcll(who & ((1ull << lane) - 1))];
      at += __popcll(who);
    }
  }
}

__global__ void __launch_bounds__(kStepThreads) k_slots(ExtendArgs a) {
  const int32_t tokens = a.starts[a.n_seq];
  for (int64_t t = blockIdx.x * int64_t(kStepThreads) + threadIdx.x; t < a.max_tokens; t += int64_t(gridDim.x) * kStepThreads) {
    int64_t slot = -1;
    int32_t pos = 0;
    if (t < tokens) {
      int32_t lo = 0, hi = a.n_seq - 1;  // the last sequence that starts at or before t
      while (lo < hi) {
        const int32_t mid = (lo + hi + 1) >> 1;
        if (a.starts[mid] <= t)
          lo = mid;
        else
          hi = mid - 1;
      }
      pos = a.cached[lo] + int32_t(t - a.starts[lo]);
      slot = int64_t(a.new_table[int64_t(lo) * a.max_blocks + pos / a.bt]) * a.bt + pos % a.bt;
    }
    a.slots[t] = slot;
    a.positions[t] = pos;
  }
}

uint64_t lay_out(const ExtendArgs &a, void *ws, ExtendWs *w) {
  char *p = static_cast<char *>(ws);
  uint64_t at = 0;
  auto take = [&](uint64_t bytes) {
    char *q = p + at;
    at += (bytes + 255) / 256 * 256;
    return q;
  };
  const uint64_t words = uint64_t(words_of(a.num_blocks));
  w->found = reinterpret_cast<int32_t *>(take(256));  // cleared with the bitmaps that follow it
  w->used = reinterpret_cast<uint32_t *>(take(words * 4));
  w->shared = reinterpret_cast<uint32_t *>(take(words * 4));
  w->rank = reinterpret_cast<int32_t *>(take(words * 4));
  w->before = reinterpret_cast<int32_t *>(take(uint64_t(a.n_seq) * 4));
  w->list = reinterpret_cast<int32_t *>(take(uint64_t(a.num_blocks) * 4));
  return at;
}

int grid_for(int64_t n, int per, int most) { return int(std::max<int64_t>(1, std::min<int64_t>((n + per - 1) / per, most))); }

// ---- atp_kv_append ------------------------------------------------------------
// (x, y) -> amplitude (x cos - y sin, y cos + x sin) per pair; the angle is
// position * turns[i] revolutions, reduced to a fraction in 64 bits.

template <typename T, typename CT>
__global__ void __launch_bounds__(kStepThreads) k_append(AppendArgs a) {
  const int32_t heads = a.n_q + 2 * a.c.n_kv, half = a.c.hd / 2;
  const int64_t n = int64_t(a.max_tokens) * heads * half, room = int64_t(a.c.num_blocks) * a.c.bt;
  for (int64_t i = blockIdx.x * int64_t(kStepThreads) + threadIdx.x; i < n; i += int64_t(gridDim.x) * kStepThreads) {
    const int32_t u = int32_t(i % half), h = int32_t(i / half % heads);
    const int64_t t = i / half / heads, slot = a.slots[t];
    if (slot < 0) continue;
    const bool is_q = h < a.n_q, is_v = h >= a.n_q + a.c.n_kv;
    if (!is_q && slot >= room) {
      flag(a.status, ATP_EINVAL);
      continue;
    }
    const int32_t j = is_q ? h : (h - a.n_q) % a.c.n_kv;
    const T *src = is_q ? static_cast<const T *>(a.q) + t * a.q_stride
                        : is_v ? static_cast<const T *>(a.v) + t * a.v_stride : static_cast<const T *>(a.k) + t * a.k_stride;
    src += int64_t(j) * a.c.hd;
    int32_t d0 = 2 * u, d1 = d0 + 1;
    const bool turn = !is_v && u < a.r.pairs;
    if (turn && !a.r.interleaved) d0 = u, d1 = u + a.r.pairs;
    float x = as_f32(src[d0]), y = as_f32(src[d1]);
    if (turn) {
      double r = double(a.positions[t]) * a.r.turns[u];
      r -= rint(r);
      float sn, cs;
      sincospif(2.0f * float(r), &sn, &cs);
      sn *= a.r.amplitude;
      cs *= a.r.amplitude;
      const float x2 = x * cs - y * sn, y2 = y * cs + x * sn;
      x = x2;
      y = y2;
    }
    if (is_q) {
      T *dst = static_cast<T *>(a.q_out) + t * a.q_out_stride + int64_t(j) * a.c.hd;
      dst[d0] = rounded<T>(x);
      dst[d1] = rounded<T>(y);
    } else {
      if (a.c.scales) {
        const float s = a.c.scales[is_v * a.c.n_kv + j];
        x /= s;
        y /= s;
      }
      CT *dst = reinterpret_cast<CT *>(a.c.base + is_v * a.c.v_off + slot / a.c.bt * a.c.block_stride +
                                       int64_t(j) * a.c.head_stride + slot % a.c.bt * a.c.tok_stride);
      dst[d0] = rounded<CT>(x);
      dst[d1] = rounded<CT>(y);
    }
  }
}

}  // namespace

uint64_t extend_workspace(const ExtendArgs &a) {
  ExtendWs w;
  return lay_out(a, nullptr, &w);
}

void extend_launch(const ExtendArgs &a, void *ws, void *stream) {
  const hipStream_t st = kv_stream(stream);
  ExtendWs w;
  lay_out(a, ws, &w);
  const int32_t words = words_of(a.num_blocks), clear = int32_t(w.shared - reinterpret_cast<uint32_t *>(w.found)) + words;
  hipLaunchKernelGGL(k_clear, dim3(grid_for(clear, kStepThreads, 1024)), dim3(kStepThreads), 0, st,
                     reinterpret_cast<uint32_t *>(w.found), clear);
  hipLaunchKernelGGL(k_mark, dim3(grid_for(int64_t(a.n_seq) * a.max_blocks, kStepThreads, 2048)), dim3(kStepThreads), 0, st, a, w);
  hipLaunchKernelGGL(k_scan, dim3(1), dim3(kScanThreads), 0, st, a, w);
  hipLaunchKernelGGL(k_list, dim3(grid_for(words, kStepThreads, 1024)), dim3(kStepThreads), 0, st, a, w);
  hipLaunchKernelGGL(k_fill, dim3(grid_for(a.n_seq, kStepThreads / 64, 1024)), dim3(kStepThreads), 0, st, a, w);
  hipLaunchKernelGGL(k_slots, dim3(grid_for(a.max_tokens, kStepThreads, 1024)), dim3(kStepThreads), 0, st, a);
  kv_hip(hipGetLastError(), "atp_kv_extend");
}

void append_launch(const AppendArgs &a, void *stream) {
  const hipStream_t st = kv_stream(stream);
  const int64_t n = int64_t(a.max_tokens) * (a.n_q + 2 * a.c.n_kv) * (a.c.hd / 2);
  const dim3 grid(grid_for(n, kStepThreads, 65536)), block(kStepThreads);
  const bool b = a.dtype == ATP_BF16, e = a.cache_dtype == ATP_E4M3;
  if (b && e)
    hipLaunchKernelGGL((k_append<__bf16, E4M3>), grid, block, 0, st, a);
  else if (b)
    hipLaunchKernelGGL((k_append<__bf16, __bf16>), grid, block, 0, st, a);
  else if (e)
    hipLaunchKernelGGL((k_append<_Float16, E4M3>), grid, block, 0, st, a);
  else
    hipLaunchKernelGGL((k_append<_Float16, _Float16>), grid, block, 0, st, a);
  kv_hip(hipGetLastError(), "atp_kv_append");
}

}  // namespace atp
