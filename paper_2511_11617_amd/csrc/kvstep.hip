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
constexpr int kScanWaves = kScanThreads / 64;
constexpr int kGroupWords = 256;   // bitmap words whose zeros are counted together
constexpr int kShortRange = 4;     // blocks of a sequence that one thread looks through

// A pool and a step that one workgroup serves alone, bitmaps in shared memory
// (one launch; k_extend_one below): the launches cost most of a small step.
// Against the seven launches below, which spread over the chip, 8 sessions
// take 7.5 against 15.5 us, 128 of 513 blocks 14.7 against 24.6, 250 of 513
// 22.7 against 25.5, and two prompts of 8000 tokens 22.8 against 21.1.
constexpr int32_t kOneWords = 16384;
constexpr int64_t kOneEntries = 1 << 17, kOneTokens = 1 << 13;

struct ExtendWs {
  uint32_t *used, *shared;
  int32_t *zeros;   // free ids of each group of words, then before it
  int32_t *before;  // wanted entries of each sequence, then before it
  int32_t *list;    // the free ids, ascending, as far as they are given out
  int32_t *found;   // [0] something refused was seen, [1] blocks taken (-1: the step failed)
};

__host__ __device__ inline int32_t words_of(int32_t num_blocks) { return int32_t((uint32_t(num_blocks) + 31) / 32); }
__host__ __device__ inline int32_t groups_of(int32_t words) { return (words + kGroupWords - 1) / kGroupWords; }

__device__ inline int32_t wave_sum(int32_t x) {
  for (int d = 32; d; d >>= 1) x += __shfl_xor(x, d);
  return x;
}

// Exclusive sum over the workgroup's threads; *total gets the whole sum.
template <typename I>
__device__ inline I block_scan(I x, I *total, I *lds) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  I inc = x;
  for (int d = 1; d < 64; d <<= 1) {
    const I y = __shfl_up(inc, d);
    if (lane >= d) inc += y;
  }
  __syncthreads();
  if (lane == 63) lds[wave] = inc;
  __syncthreads();
  I base = 0, all = 0;
  for (int w = 0; w < kScanWaves; ++w) {
    if (w < wave) base += lds[w];
    all += lds[w];
  }
  *total = all;
  return base + inc - x;
}

// The blocks [b, e) that sequence s's new tokens lie in (empty for none); its lengths are in range.
__device__ inline void new_range(const ExtendArgs &a, int32_t s, int32_t *b, int32_t *e) {
  const int32_t c = a.cached[s], f = a.fresh[s];
  *b = c / a.bt;
  *e = f ? int32_t((int64_t(c) + f + a.bt - 1) / a.bt) : *b;
}

__device__ inline bool lengths_fit(const ExtendArgs &a, int32_t s) {
  const int64_t c = a.cached[s], f = a.fresh[s];
  return c >= 0 && f >= 0 && c + f <= min(int64_t(a.max_blocks) * a.bt, int64_t(INT32_MAX));
}

__device__ inline uint32_t free_bits(const ExtendArgs &a, const uint32_t *used, int32_t word) {
  const int32_t n = min(32, a.num_blocks - word * 32);
  return ~used[word] & (n == 32 ? ~0u : (1u << n) - 1);
}

// Marks one table entry; false for an id that is none.
__device__ inline bool mark(int32_t p, int32_t num_blocks, uint32_t *used, uint32_t *shared) {
  if (p < -1 || p >= num_blocks) return false;
  if (p >= 0) {
    const uint32_t bit = 1u << (p & 31);
    if (atomicOr(&used[p >> 5], bit) & bit) atomicOr(&shared[p >> 5], bit);
  }
  return true;
}

// One entry of a sequence's new range: 1 where a block is wanted, 0 where one
// is there, -1 where that one is shared.
__device__ inline int32_t wants(const ExtendArgs &a, const uint32_t *shared, int32_t s, int32_t i) {
  const int32_t p = a.table[int64_t(s) * a.max_blocks + i];
  return p < 0 ? 1 : shared[p >> 5] >> (p & 31) & 1 ? -1 : 0;
}

// Wanted blocks of a sequence, by one wave; a shared block sets *bad.
__device__ inline int32_t wanted_by_wave(const ExtendArgs &a, const uint32_t *shared, int32_t s, int32_t b, int32_t e, bool *bad) {
  int32_t n = 0;
  for (int32_t i = b + (threadIdx.x & 63); i < e; i += 64) {
    const int32_t w = wants(a, shared, s, i);
    n += w > 0;
    *bad |= w < 0;
  }
  return wave_sum(n);
}

// Gives a sequence its blocks list[at...], by one wave.
__device__ inline void fill_by_wave(const ExtendArgs &a, const int32_t *list, int32_t at, int32_t s, int32_t b, int32_t e) {
  const int lane = threadIdx.x & 63;
  for (int32_t i0 = b; i0 < e; i0 += 64) {
    const int32_t i = i0 + lane;
    const int64_t cell = int64_t(s) * a.max_blocks + i;
    const bool want = i < e && a.table[cell] < 0;
    const uint64_t who = __ballot(want);
    if (want) a.new_table[cell] = list[at + __popcll(who & ((1ull << lane) - 1))];
    at += __popcll(who);
  }
}

// The place of row t, of `tokens` rows that are tokens.
__device__ inline void place(const ExtendArgs &a, const int32_t *starts, int32_t t, int32_t tokens) {
  int64_t slot = -1;
  int32_t pos = 0;
  if (t < tokens) {
    int32_t lo = 0, hi = a.n_seq - 1;  // the last sequence that starts at or before t
    while (lo < hi) {
      const int32_t mid = (lo + hi + 1) >> 1;
      if (starts[mid] <= t)
        lo = mid;
      else
        hi = mid - 1;
    }
    pos = a.cached[lo] + (t - starts[lo]);
    slot = int64_t(a.new_table[int64_t(lo) * a.max_blocks + pos / a.bt]) * a.bt + pos % a.bt;
  }
  a.slots[t] = slot;
  a.positions[t] = pos;
}

__device__ inline void verdict(const ExtendArgs &a, int32_t code, int32_t tokens, int32_t wanted, int32_t free_ids) {
  const bool ok = code == ATP_OK, bad = code == ATP_EINVAL;
  a.starts[a.n_seq] = ok ? tokens : 0;
  a.status[0] = code;
  a.status[1] = ok ? tokens : 0;
  a.status[2] = bad ? 0 : wanted;
  a.status[3] = bad ? 0 : ok ? free_ids - wanted : free_ids;
}

// ---- one workgroup
__global__ void __launch_bounds__(kScanThreads) k_extend_one(ExtendArgs a, ExtendWs w) {
  __shared__ uint32_t used[kOneWords], shared[kOneWords];
  __shared__ int64_t sums[kScanWaves];
  __shared__ int32_t sums32[kScanWaves], bad, longs;  // longs: some sequence's range is not short
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int32_t words = words_of(a.num_blocks);
  for (int32_t i = tid; i < words; i += kScanThreads) used[i] = shared[i] = 0;
  if (tid == 0) bad = longs = 0;
  __syncthreads();
  const int32_t entries = a.n_seq * a.max_blocks;
  bool wrong = false;
  const bool same = a.new_table == a.table;
  int32_t done = 0;  // entries that the 16-byte reads took
  if ((reinterpret_cast<uintptr_t>(a.table) | reinterpret_cast<uintptr_t>(a.new_table)) % 16 == 0) {
    constexpr int kAhead = 4;  // reads in flight in each thread
    const int32_t quads = entries / 4;
    for (int32_t q0 = tid; q0 < quads; q0 += kAhead * kScanThreads) {
      int4 p[kAhead];
#pragma unroll
      for (int j = 0; j < kAhead; ++j) {
        const int32_t q = q0 + j * kScanThreads;
        p[j] = q < quads ? reinterpret_cast<const int4 *>(a.table)[q] : int4{-1, -1, -1, -1};
      }
#pragma unroll
      for (int j = 0; j < kAhead; ++j) {
        const int32_t q = q0 + j * kScanThreads;
        if (!same && q < quads) reinterpret_cast<int4 *>(a.new_table)[q] = p[j];
        const int32_t id[4] = {p[j].x, p[j].y, p[j].z, p[j].w};
        uint32_t old[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const bool in = uint32_t(id[e]) < uint32_t(a.num_blocks);
          wrong |= !in && id[e] != -1;
          old[e] = in ? atomicOr(&used[id[e] >> 5], 1u << (id[e] & 31)) : 0;
        }
#pragma unroll
        for (int e = 0; e < 4; ++e)
          if (old[e] >> (id[e] & 31) & 1) atomicOr(&shared[id[e] >> 5], 1u << (id[e] & 31));
      }
    }
    done = quads * 4;
  }
  for (int32_t i = done + tid; i < entries; i += kScanThreads) {
    const int32_t p = a.table[i];
    if (!same) a.new_table[i] = p;
    wrong |= !mark(p, a.num_blocks, used, shared);
  }
  int64_t tokens = 0;
  for (int32_t s0 = 0; s0 < a.n_seq; s0 += kScanThreads) {
    const int32_t s = s0 + tid;
    if (s < a.n_seq) {
      if (lengths_fit(a, s)) {
        int32_t b, e;
        new_range(a, s, &b, &e);
        if (e - b > kShortRange) longs = 1;
      } else {
        wrong = true;
      }
    }
    int64_t sum;
    const int64_t start = tokens + block_scan(s < a.n_seq ? int64_t(a.fresh[s]) : 0, &sum, sums);
    if (s < a.n_seq) a.starts[s] = int32_t(start);
    tokens += sum;
  }
  if (wrong || tokens > a.max_tokens) bad = 1;
  __syncthreads();
  const bool in_range = !bad;  // read by every thread before one sets it again
  __syncthreads();
  int32_t wanted = 0, free_ids = 0, first = 0;
  const int32_t per = (words + kScanThreads - 1) / kScanThreads, from = min(words, tid * per), to = min(words, from + per);
  if (in_range) {
    wrong = false;
    for (int32_t s = longs ? wave : a.n_seq; s < a.n_seq; s += kScanWaves) {  // sequences with long ranges
      int32_t b, e;
      new_range(a, s, &b, &e);
      if (e - b <= kShortRange) continue;
      const int32_t n = wanted_by_wave(a, shared, s, b, e, &wrong);
      if (lane == 0) w.before[s] = n;
    }
    __syncthreads();
    for (int32_t s0 = 0; s0 < a.n_seq; s0 += kScanThreads) {
      const int32_t s = s0 + tid;
      int32_t n = 0, sum;
      if (s < a.n_seq) {
        int32_t b, e;
        new_range(a, s, &b, &e);
        if (e - b > kShortRange) n = w.before[s];
        if (e - b <= kShortRange)
          for (int32_t i = b; i < e; ++i) {
            const int32_t x = wants(a, shared, s, i);
            n += x > 0;
            wrong |= x < 0;
          }
      }
      const int32_t before = wanted + block_scan(n, &sum, sums32);
      if (s < a.n_seq) w.before[s] = before;
      wanted += sum;
    }
    if (wrong) bad = 1;
    int32_t n = 0;
    for (int32_t i = from; i < to; ++i) n += __popc(free_bits(a, used, i));
    first = block_scan(n, &free_ids, sums32);
  }
  __syncthreads();
  const int32_t code = bad ? ATP_EINVAL : wanted > free_ids ? ATP_ECAPACITY : ATP_OK;
  if (code != ATP_OK)
    for (int32_t s = tid; s < a.n_seq; s += kScanThreads) a.starts[s] = 0;
  if (tid == 0) verdict(a, code, int32_t(tokens), wanted, free_ids);
  if (code == ATP_OK && wanted) {
    for (int32_t i = from; i < to && first < wanted; ++i)
      for (uint32_t left = free_bits(a, used, i); left && first < wanted; left &= left - 1) w.list[first++] = i * 32 + __ffs(left) - 1;
    __syncthreads();
    for (int32_t s = longs ? wave : a.n_seq; s < a.n_seq; s += kScanWaves) {
      int32_t b, e;
      new_range(a, s, &b, &e);
      if (e - b > kShortRange) fill_by_wave(a, w.list, w.before[s], s, b, e);
    }
    for (int32_t s = tid; s < a.n_seq; s += kScanThreads) {
      int32_t b, e, k = w.before[s];
      new_range(a, s, &b, &e);
      if (e - b > kShortRange) continue;
      for (int32_t i = b; i < e; ++i) {
        const int64_t cell = int64_t(s) * a.max_blocks + i;
        if (a.table[cell] < 0) a.new_table[cell] = w.list[k++];
      }
    }
  }
  __syncthreads();
  const int32_t rows = code == ATP_OK ? int32_t(tokens) : 0;
  for (int32_t t = tid; t < a.max_tokens; t += kScanThreads) place(a, a.starts, t, rows);
}

// ---- many workgroups
__global__ void __launch_bounds__(kStepThreads) k_clear(uint32_t *p, int32_t n) {
  for (int64_t i = blockIdx.x * int64_t(kStepThreads) + threadIdx.x; i < n; i += int64_t(gridDim.x) * kStepThreads) p[i] = 0;
}

__global__ void __launch_bounds__(kStepThreads) k_mark(ExtendArgs a, ExtendWs w) {
  const int64_t n = int64_t(a.n_seq) * a.max_blocks;
  bool wrong = false;
  for (int64_t i = blockIdx.x * int64_t(kStepThreads) + threadIdx.x; i < n; i += int64_t(gridDim.x) * kStepThreads) {
    const int32_t p = a.table[i];
    if (a.new_table != a.table) a.new_table[i] = p;
    wrong |= !mark(p, a.num_blocks, w.used, w.shared);
  }
  if (wrong) w.found[0] = 1;
}

// Wanted blocks of each sequence (a wave each), free ids of each group of words.
__global__ void __launch_bounds__(kStepThreads) k_count(ExtendArgs a, ExtendWs w) {
  const int lane = threadIdx.x & 63, waves = gridDim.x * (kStepThreads / 64), wave = blockIdx.x * (kStepThreads / 64) + (threadIdx.x >> 6);
  const int32_t words = words_of(a.num_blocks);
  const bool known = w.found[0] == 0;  // every id may be followed into the bitmaps
  bool wrong = false;
  for (int32_t s = wave; s < a.n_seq; s += waves) {
    if (!lengths_fit(a, s)) {
      wrong = true;
      continue;
    }
    int32_t b, e;
    new_range(a, s, &b, &e);
    const int32_t n = known ? wanted_by_wave(a, w.shared, s, b, e, &wrong) : 0;
    if (lane == 0) w.before[s] = n;
  }
  for (int32_t g = wave; g < groups_of(words); g += waves) {
    int32_t n = 0;
    for (int32_t i = g * kGroupWords + lane; i < min(words, (g + 1) * kGroupWords); i += 64) n += __popc(free_bits(a, w.used, i));
    n = wave_sum(n);
    if (lane == 0) w.zeros[g] = n;
  }
  if (wrong) w.found[0] = 1;
}

// Exclusive sums and the verdict, by one workgroup.
__global__ void __launch_bounds__(kScanThreads) k_scan(ExtendArgs a, ExtendWs w) {
  __shared__ int64_t sums[kScanWaves];
  __shared__ int32_t sums32[kScanWaves];
  const int tid = threadIdx.x;
  const int32_t groups = groups_of(words_of(a.num_blocks));
  const bool known = w.found[0] == 0;  // else before[] may hold nothing
  int64_t tokens = 0;
  int32_t wanted = 0, free_ids = 0;
  for (int32_t s0 = 0; known && s0 < a.n_seq; s0 += kScanThreads) {
    const int32_t s = s0 + tid;
    int64_t sum;
    int32_t sum32;
    const int64_t start = tokens + block_scan(s < a.n_seq ? int64_t(a.fresh[s]) : 0, &sum, sums);
    const int32_t before = wanted + block_scan(s < a.n_seq ? w.before[s] : 0, &sum32, sums32);
    if (s < a.n_seq) {
      a.starts[s] = int32_t(start);
      w.before[s] = before;
    }
    tokens += sum;
    wanted += sum32;
  }
  for (int32_t g0 = 0; known && g0 < groups; g0 += kScanThreads) {
    const int32_t g = g0 + tid;
    int32_t sum;
    const int32_t at = free_ids + block_scan(g < groups ? w.zeros[g] : 0, &sum, sums32);
    if (g < groups) w.zeros[g] = at;
    free_ids += sum;
  }
  const int32_t code = !known || tokens > a.max_tokens ? ATP_EINVAL : wanted > free_ids ? ATP_ECAPACITY : ATP_OK;
  __syncthreads();
  if (code != ATP_OK)
    for (int32_t s = tid; s < a.n_seq; s += kScanThreads) a.starts[s] = 0;
  if (tid == 0) {
    verdict(a, code, int32_t(tokens), wanted, free_ids);
    w.found[1] = code == ATP_OK ? wanted : -1;
  }
}

// The free ids in order, a wave to a group of words.
__global__ void __launch_bounds__(kStepThreads) k_list(ExtendArgs a, ExtendWs w) {
  const int32_t taken = w.found[1], words = words_of(a.num_blocks);
  if (taken <= 0) return;  // after a refusal, zeros holds nothing
  const int lane = threadIdx.x & 63, waves = gridDim.x * (kStepThreads / 64);
  for (int32_t g = blockIdx.x * (kStepThreads / 64) + (threadIdx.x >> 6); g < groups_of(words); g += waves) {
    int32_t at = w.zeros[g];
    for (int32_t i0 = g * kGroupWords; i0 < (g + 1) * kGroupWords && at < taken; i0 += 64) {
      const int32_t i = i0 + lane;
      uint32_t left = i < words ? free_bits(a, w.used, i) : 0;
      int32_t inc = __popc(left);
      const int32_t n = inc;
      for (int d = 1; d < 64; d <<= 1) {
        const int32_t y = __shfl_up(inc, d);
        if (lane >= d) inc += y;
      }
      for (int32_t r = at + inc - n; left && r < taken; left &= left - 1) w.list[r++] = i * 32 + __ffs(left) - 1;
      at += __shfl(inc, 63);
    }
  }
}

__global__ void __launch_bounds__(kStepThreads) k_fill(ExtendArgs a, ExtendWs w) {
  if (w.found[1] <= 0) return;
  const int waves = gridDim.x * (kStepThreads / 64);
  for (int32_t s = blockIdx.x * (kStepThreads / 64) + (threadIdx.x >> 6); s < a.n_seq; s += waves) {
    int32_t b, e;
    new_range(a, s, &b, &e);
    fill_by_wave(a, w.list, w.before[s], s, b, e);
  }
}

__global__ void __launch_bounds__(kStepThreads) k_slots(ExtendArgs a) {
  const int32_t tokens = a.starts[a.n_seq];
  for (int64_t t = blockIdx.x * int64_t(kStepThreads) + threadIdx.x; t < a.max_tokens; t += int64_t(gridDim.x) * kStepThreads)
    place(a, a.starts, int32_t(t), tokens);
}

bool one_workgroup(const ExtendArgs &a) {
  return words_of(a.num_blocks) <= kOneWords && int64_t(a.n_seq) * a.max_blocks <= kOneEntries && a.max_tokens <= kOneTokens;
}

uint64_t lay_out(const ExtendArgs &a, void *ws, ExtendWs *w) {
  char *p = static_cast<char *>(ws);
  uint64_t at = 0;
  auto take = [&](uint64_t bytes) {
    char *q = p + at;
    at += (bytes + 255) / 256 * 256;
    return q;
  };
  *w = {};
  w->before = reinterpret_cast<int32_t *>(take(uint64_t(a.n_seq) * 4));
  w->list = reinterpret_cast<int32_t *>(take(uint64_t(a.num_blocks) * 4));
  if (one_workgroup(a)) return at;
  const uint64_t words = uint64_t(words_of(a.num_blocks));
  w->found = reinterpret_cast<int32_t *>(take(256));  // cleared with the bitmaps that follow it
  w->used = reinterpret_cast<uint32_t *>(take(words * 4));
  w->shared = reinterpret_cast<uint32_t *>(take(words * 4));
  w->zeros = reinterpret_cast<int32_t *>(take(uint64_t(groups_of(int32_t(words))) * 4));
  return at;
}

int grid_for(int64_t n, int per, int most) { return int(std::max<int64_t>(1, std::min<int64_t>((n + per - 1) / per, most))); }

// ---- atp_kv_append ------------------------------------------------------------
// (x, y) -> amplitude (x cos - y sin, y cos + x sin) per pair; the angle is
// position * turns[i] revolutions, reduced to a fraction in 64 bits.  Bound by
// the bytes: every input is read once and every output written once.

__device__ inline float2 turned(const RopeArgs &r, int32_t pos, int pair) {  // amplitude * (cos, sin)
  double x = double(pos) * r.turns[pair];
  x -= rint(x);
  float sn, cs;
  sincospif(2.0f * float(x), &sn, &cs);
  return {r.amplitude * cs, r.amplitude * sn};
}

// 8 elements as one read or write.
template <typename T>
__device__ inline void read8(const T *p, float *x) {
  const u32x4_t w = *reinterpret_cast<const u32x4_t *>(p);
  using v2 = T __attribute__((ext_vector_type(2)));
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const uint32_t one = w[i];
    const v2 y = __builtin_bit_cast(v2, one);
    x[2 * i] = float(y[0]);
    x[2 * i + 1] = float(y[1]);
  }
}
template <typename T>
__device__ inline void write8(T *p, const float *x) {
  using v2 = T __attribute__((ext_vector_type(2)));
  u32x4_t w;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const v2 y = {T(x[2 * i]), T(x[2 * i + 1])};
    w[i] = __builtin_bit_cast(uint32_t, y);
  }
  *reinterpret_cast<u32x4_t *>(p) = w;
}
template <>
__device__ inline void write8<E4M3>(E4M3 *p, const float *x) {
  u32x2_t w;
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    float y[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const float z = x[4 * i + j];
      y[j] = z > 448.0f ? 448.0f : z < -448.0f ? -448.0f : z;
    }
    int v = __builtin_amdgcn_cvt_pk_fp8_f32(y[0], y[1], 0, false);
    w[i] = uint32_t(__builtin_amdgcn_cvt_pk_fp8_f32(y[2], y[3], v, true));
  }
  *reinterpret_cast<u32x2_t *>(p) = w;
}

// Where rot_dim is a multiple of 16: 65536 tokens of 13 + 8 heads of 128 in 135
// us, 5.2 TB/s, 8192 in 16.4 (88 MB, which stay in the last-level cache from call
// to call; 20 with other inputs each time; a pair at a time 59).  A workgroup
// takes up to 4 tokens: its threads work out the tokens' cosines and sines into
// shared memory (once for all heads), then take units of 16 elements, the two 8s
// that turn together (or lie together, where nothing turns), as 16-byte reads
// and writes.
constexpr int kAppendTokens = 4;
template <typename T, typename CT>
__global__ void __launch_bounds__(kStepThreads) k_append16(AppendArgs a, int32_t tokens) {
  __shared__ float cosine[kAppendTokens][kMaxPairs], sine[kAppendTokens][kMaxPairs];
  __shared__ int64_t where[kAppendTokens];  // of the token's first head in the cache; -1 padding, -2 past the arena
  const int tid = threadIdx.x;
  const int64_t t0 = int64_t(blockIdx.x) * tokens;
  const int32_t n = int32_t(min(int64_t(tokens), a.max_tokens - t0)), pairs = a.r.pairs;
  if (tid < n) {
    const int64_t slot = a.slots[t0 + tid];
    int64_t at = -1;
    if (slot >= int64_t(a.c.num_blocks) * a.c.bt) {
      at = -2;
      if (a.c.n_kv) flag(a.status, ATP_EINVAL);
    } else if (slot >= 0) {
      const int64_t block = slot / a.c.bt;
      at = block * a.c.block_stride + (slot - block * a.c.bt) * a.c.tok_stride;
    }
    where[tid] = at;
  }
  for (int i = tid; i < n * pairs; i += kStepThreads) {
    const int t = i / pairs, p = i - t * pairs;
    const float2 x = turned(a.r, a.positions[t0 + t], p);
    cosine[t][p] = x.x;
    sine[t][p] = x.y;
  }
  __syncthreads();
  const int32_t hd = a.c.hd, per_head = (hd + 15) / 16, per_token = (a.n_q + 2 * a.c.n_kv) * per_head;
  for (int i = tid; i < n * per_token; i += kStepThreads) {
    const int t = i / per_token, in = i - t * per_token, h = in / per_head, u = in - h * per_head;
    const int64_t at = where[t], row = t0 + t;
    if (at == -1) continue;
    const bool is_q = h < a.n_q, is_v = h >= a.n_q + a.c.n_kv;
    if (!is_q && at < 0) continue;
    const int32_t j = is_q ? h : is_v ? h - a.n_q - a.c.n_kv : h - a.n_q;
    const T *src = (is_q ? static_cast<const T *>(a.q) + row * a.q_stride
                         : is_v ? static_cast<const T *>(a.v) + row * a.v_stride : static_cast<const T *>(a.k) + row * a.k_stride) +
                   int64_t(j) * hd;
    const bool turn = !is_v && u * 8 < pairs;
    const int32_t d0 = turn && !a.r.interleaved ? 8 * u : 16 * u, d1 = turn && !a.r.interleaved ? pairs + 8 * u : d0 + 8;
    const bool both = d1 < hd;  // head_dim is a multiple of 8: the last unit may be half of one
    float x[8], y[8];
    read8(src + d0, x);
    if (both) read8(src + d1, y);
    if (turn && a.r.interleaved) {
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        float *const z = e < 4 ? x : y;
        const int k = 2 * e % 8;
        const float c = cosine[t][8 * u + e], s = sine[t][8 * u + e], p = z[k], q = z[k + 1];
        z[k] = p * c - q * s;
        z[k + 1] = q * c + p * s;
      }
    } else if (turn) {
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const float c = cosine[t][8 * u + e], s = sine[t][8 * u + e], p = x[e], q = y[e];
        x[e] = p * c - q * s;
        y[e] = q * c + p * s;
      }
    }
    if (is_q) {
      T *dst = static_cast<T *>(a.q_out) + row * a.q_out_stride + int64_t(j) * hd;
      write8(dst + d0, x);
      if (both) write8(dst + d1, y);
    } else {
      if (a.c.scales) {
        const float s = a.c.scales[is_v * a.c.n_kv + j];
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          x[e] /= s;
          y[e] /= s;
        }
      }
      CT *dst = reinterpret_cast<CT *>(a.c.base + is_v * a.c.v_off + at + int64_t(j) * a.c.head_stride);
      write8(dst + d0, x);
      if (both) write8(dst + d1, y);
    }
  }
}

// Any even rot_dim: a thread takes a pair at a time (8192 tokens of 13 + 8 heads
// of 128, 124 of them turned: 59 us, by its 2-byte accesses and an angle for each
// head; of 80, 40 turned: 40 us).
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
      const float2 cs = turned(a.r, a.positions[t], u);
      const float x2 = x * cs.x - y * cs.y, y2 = y * cs.x + x * cs.y;
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
  if (one_workgroup(a)) {
    hipLaunchKernelGGL(k_extend_one, dim3(1), dim3(kScanThreads), 0, st, a, w);
  } else {
    constexpr int kWaves = kStepThreads / 64;
    const dim3 block(kStepThreads);
    const int32_t words = words_of(a.num_blocks), clear = int32_t(w.shared - reinterpret_cast<uint32_t *>(w.found)) + words;
    hipLaunchKernelGGL(k_clear, dim3(grid_for(clear, kStepThreads, 1024)), block, 0, st, reinterpret_cast<uint32_t *>(w.found), clear);
    hipLaunchKernelGGL(k_mark, dim3(grid_for(int64_t(a.n_seq) * a.max_blocks, kStepThreads, 2048)), block, 0, st, a, w);
    hipLaunchKernelGGL(k_count, dim3(grid_for(std::max(a.n_seq, groups_of(words)), kWaves, 1024)), block, 0, st, a, w);
    hipLaunchKernelGGL(k_scan, dim3(1), dim3(kScanThreads), 0, st, a, w);
    hipLaunchKernelGGL(k_list, dim3(grid_for(groups_of(words), kWaves, 1024)), block, 0, st, a, w);
    hipLaunchKernelGGL(k_fill, dim3(grid_for(a.n_seq, kWaves, 1024)), block, 0, st, a, w);
    hipLaunchKernelGGL(k_slots, dim3(grid_for(a.max_tokens, kStepThreads, 1024)), block, 0, st, a);
  }
  kv_hip(hipGetLastError(), "atp_kv_extend");
}

template <typename T, typename CT>
static void append_as(const AppendArgs &a, hipStream_t st) {
  if (a.r.pairs % 8 == 0) {
    // one token a workgroup until the chip is full of them
    const int32_t tokens = a.max_tokens < 2048 ? 1 : kAppendTokens;
    hipLaunchKernelGGL((k_append16<T, CT>), dim3((a.max_tokens + tokens - 1) / tokens), dim3(kStepThreads), 0, st, a, tokens);
  } else {
    const int64_t n = int64_t(a.max_tokens) * (a.n_q + 2 * a.c.n_kv) * (a.c.hd / 2);
    hipLaunchKernelGGL((k_append<T, CT>), dim3(grid_for(n, kStepThreads, 65536)), dim3(kStepThreads), 0, st, a);
  }
}

void append_launch(const AppendArgs &a, void *stream) {
  const hipStream_t st = kv_stream(stream);
  const bool b = a.dtype == ATP_BF16, e = a.cache_dtype == ATP_E4M3;
  if (b && e)
    append_as<__bf16, E4M3>(a, st);
  else if (b)
    append_as<__bf16, __bf16>(a, st);
  else if (e)
    append_as<_Float16, E4M3>(a, st);
  else
    append_as<_Float16, _Float16>(a, st);
  kv_hip(hipGetLastError(), "atp_kv_append");
}

}  // namespace atp
