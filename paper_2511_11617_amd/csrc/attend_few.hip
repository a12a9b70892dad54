// attend_few.hip — attention where few rows share a KV head's tokens: one
// token per sequence, or drafts.  Bound by reading K and V once.
//
// One workgroup takes (sequence, run of query heads with one KV head, chunk
// of the context); its four waves take steps of 32 tokens in turn.  K and V
// go from memory straight into the operands of the matrix instructions, with
// no shared memory between:
//   S^T = K Q^T   operand A: 16 tokens x 32 dimensions, a lane holds 8
//                 dimensions of one token as they lie in memory
//   O^T = V^T P^T operand B: the weights, which the lanes hold after the
//                 first product already: the result's tokens 4 j + i of lane
//                 group j are taken as the second product's inner index
//                 (two tiles of 16 tokens side by side), and V is read in the
//                 same order: a lane reads 8 tokens' values of its dimensions
//                 and exchanges halves of registers (one permute a dword)
// A row (token, query head) is a column of both products, so its maximum,
// sum and scale stay in its lanes.  The maximum moves only when a score
// passes it by 2^8, so a step has no cross-lane work in general.  The weights
// enter the second product as a sum of two 16-bit parts (the matrix units
// idle here): they lose nothing of note.
//
// Measured: 128 sessions of 8192 tokens, 2 KV heads of 128 in 16 bits, 190 us
// in this kernel = 5.6 TB/s, where a plain sum over 4 GiB reads 6.1; 3 sessions
// of up to 131000 in 8 bits, 31 us = 4.9 TB/s.
#include "attend.h"

namespace atp {
namespace {

constexpr int kFewWaves = 4;
// Tokens of a wave's step: 16 KB of K and V at 128 dimensions, in flight while
// the step before is computed (8-bit steps of 32 tokens were half of that).
template <typename CT, int HD>
constexpr int kStep = sizeof(CT) == 1 && HD <= 128 ? 64 : 32;

// A lane's 8 dimensions of a K row as an operand.
template <typename T, typename CT>
struct KChunk {
  using raw = u32x4_t;
  static __device__ typename Half16<T>::v8 operand(raw x) { return __builtin_bit_cast(typename Half16<T>::v8, x); }
};
template <typename T>
struct KChunk<T, E4M3> {
  using raw = u32x2_t;
  static __device__ typename Half16<T>::v8 operand(raw x) {
    const u32x4_t y = {Half16<T>::fp8_lo(x[0]), Half16<T>::fp8_hi(x[0]), Half16<T>::fp8_lo(x[1]), Half16<T>::fp8_hi(x[1])};
    return __builtin_bit_cast(typename Half16<T>::v8, y);
  }
};

template <int BYTES>
struct Bytes;
template <>
struct Bytes<4> { using t = uint32_t; };
template <>
struct Bytes<8> { using t = u32x2_t; };
template <>
struct Bytes<16> { using t = u32x4_t; };

// N values of a V row (N * sizeof(CT) bytes) as N / 2 dwords of pairs.
template <typename T, typename CT, int N>
struct VChunk {
  using raw = typename Bytes<N * int(sizeof(CT))>::t;
  static __device__ uint32_t pair(const raw &x, int i) {
    if constexpr (sizeof(CT) == 2) {
      return x[i];
    } else {
      uint32_t w;
      if constexpr (sizeof(raw) == 4)
        w = x;
      else
        w = x[i / 2];
      return i % 2 ? Half16<T>::fp8_hi(w) : Half16<T>::fp8_lo(w);
    }
  }
};

// The token of a lane's e-th score of a step, from its group's first on.
__device__ constexpr int token_of(int e) { return 16 * (e / 4) + e % 4; }

// Infinities and NaN of a chunk become 0; whether there were any.
template <typename T, typename CT>
__device__ inline bool clean_word(uint32_t &x) {
  if constexpr (sizeof(CT) == 2) {
    const uint32_t y = finite_only<T>(x);
    const bool found = not_finite<T>(x);
    x = y;
    return found;
  } else {
    const uint32_t nan = nan_bytes(x);
    x &= ~((nan >> 7) * 0xffu);
    return nan != 0;
  }
}
template <typename T, typename CT, typename V>
__device__ inline bool clean(V &x) {
  bool found = false;
  if constexpr (sizeof(V) == 4) {
    found = clean_word<T, CT>(x);
  } else {
#pragma unroll
    for (int i = 0; i < int(sizeof(V) / 4); ++i) {
      uint32_t w = x[i];
      found |= clean_word<T, CT>(w);
      x[i] = w;
    }
  }
  return found;
}

// The chunk of a workgroup.  Every workgroup sums the sequences' spans, which
// gives the chunks' length (groups of them over all, none shorter than
// kFewLeast), counts the chunks before each sequence and finds its own: the
// work is even whatever the lengths, and the host need not know them.
// Workgroup w takes run w % n_run of chunk w / n_run.
struct Share {
  int32_t s, lo, hi, count;  // count: chunks of the sequence; s < 0: none
};
__device__ inline Share share_of(const AttendKernel &a) {
  constexpr int T = kFewWaves * 64;
  __shared__ int64_t total64[kFewWaves];
  __shared__ int32_t sums[kFewWaves], mine[4];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  int64_t total = 0;
  int32_t span0 = 0, from0 = 0;  // of this thread's first sequence: most steps have no more than threads
  for (int32_t s = tid; s < a.n_seq; s += T) {
    const Seq q = sequence(a, s);
    if (!q.ok && blockIdx.x == 0) flag(a.status, ATP_EINVAL);
    const int32_t from = q.ok ? first_seen(a, q.cached, kFewAlign) : 0, span = q.ok && q.n ? q.ctx - from : 0;
    if (s == tid) {
      span0 = span;
      from0 = from;
    }
    total += span;
  }
  for (int d = 32; d; d >>= 1) total += __shfl_xor(total, d);
  if (lane == 0) total64[wave] = total;
  if (tid == 0) mine[0] = -1;
  __syncthreads();
  total = 0;
  for (int w = 0; w < kFewWaves; ++w) total += total64[w];
  // Sequences' last chunks may be short, which makes more workgroups than the
  // chip holds at once.  More sequences than that: two rounds' chunks (300 of up
  // to 3000 tokens: 108 against 116 us); else, where they are over an eighth
  // more, longer chunks (128 ragged ones of up to 8192: 113 against 134 us).
  const int64_t groups = few_rounds(a) * a.split.groups;
  const int64_t each = (total * a.h.n_run + groups - 1) / groups;
  const auto chunk_of = [](int64_t x) { return int32_t((min(max(x, int64_t(kFewLeast)), int64_t(1) << 30) + kFewAlign - 1) / kFewAlign * kFewAlign); };
  int32_t chunk = chunk_of(each);
  if (a.n_seq <= T && chunk > kFewLeast) {
    int32_t n = (span0 + chunk - 1) / chunk;
    for (int d = 32; d; d >>= 1) n += __shfl_xor(n, d);
    if (lane == 0) sums[wave] = n;
    __syncthreads();
    n = 0;
    for (int w = 0; w < kFewWaves; ++w) n += sums[w];
    if (int64_t(n) * a.h.n_run > groups + groups / 8) chunk = chunk_of(each + each / 3);
    __syncthreads();
  }
  const int32_t want = blockIdx.x / a.h.n_run;
  int32_t before = 0;
  for (int32_t s0 = 0; s0 < a.n_seq && (before <= want || blockIdx.x == 0); s0 += T) {
    const int32_t s = s0 + tid;
    int32_t span = span0, from = from0;
    if (s0 && s < a.n_seq) {
      const Seq q = sequence(a, s);
      from = q.ok ? first_seen(a, q.cached, kFewAlign) : 0;
      span = q.ok && q.n ? q.ctx - from : 0;
    }
    const int32_t n = s < a.n_seq ? (span + chunk - 1) / chunk : 0;
    int32_t inc = n;
    for (int d = 1; d < 64; d <<= 1) {
      const int32_t y = __shfl_up(inc, d);
      if (lane >= d) inc += y;
    }
    if (s0) __syncthreads();
    if (lane == 63) sums[wave] = inc;
    __syncthreads();
    int32_t at = before + inc - n;
    for (int w = 0; w < kFewWaves; ++w) {
      if (w < wave) at += sums[w];
      before += sums[w];
    }
    if (want >= at && want < at + n) {
      mine[0] = s;
      mine[1] = from + (want - at) * chunk;
      mine[2] = int32_t(min(int64_t(from) + span, int64_t(mine[1]) + chunk));
      mine[3] = n;
    }
    if (blockIdx.x == 0 && s < a.n_seq && a.split.shares) {  // for the join
      a.split.shares[2 * s] = at;
      a.split.shares[2 * s + 1] = n;
    }
  }
  __syncthreads();
  return {__builtin_amdgcn_readfirstlane(mine[0]), __builtin_amdgcn_readfirstlane(mine[1]), __builtin_amdgcn_readfirstlane(mine[2]),
          __builtin_amdgcn_readfirstlane(mine[3])};
}

// HD: dimensions the registers hold (head_dim is at most HD).  How rows lie:
//   WHOLE   head_dim is HD and block_tokens a multiple of 16, so that a tile of
//           16 tokens lies in one block and its id is the wave's (scalar)
//   EVEN    block_tokens a multiple of 16
//   ANY     each lane looks its tokens' blocks up
// Where head_dim is less than HD, dimensions beyond it are read from the row's
// begin; K's are made 0, V's end in results that nobody takes.
// MT: tiles of 16 rows.
enum { WHOLE = 0, EVEN = 1, ANY = 2 };
template <typename T, typename CT, int HD, int LIE, int MT>
__global__ void __launch_bounds__(kFewWaves * 64, HD == 256 || (HD == 128 && MT == 2) ? 1 : 2) k_few(AttendKernel a) {
  using H = Half16<T>;
  using v8 = typename H::v8;
  constexpr int TS = kStep<CT, HD>, U = TS / 16, KK = HD / 32, ND = HD / 16, NV = ND < 8 ? ND : 8, VP = ND / NV;
  using KC = KChunk<T, CT>;
  using VC = VChunk<T, CT, NV>;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), col = lane & 15, grp = lane >> 4;
  const Share sh = share_of(a);
  if (sh.s < 0) return;
  const int32_t run = blockIdx.x % a.h.n_run, s = sh.s;
  const Seq q = sequence(a, s);
  int32_t h0;
  const int32_t gh = run_heads(a.h, run, &h0), rows = q.n * gh;
  const int32_t lo = sh.lo, hi = sh.hi;
  const int32_t kv = a.h.kv0 + run, hd = a.c.hd;
  const char *const kbase = a.c.base + int64_t(kv) * a.c.head_stride;
  const char *const vbase = kbase + a.c.v_off;
  const int32_t *const table = a.table + int64_t(s) * a.max_blocks;
  const float ks = a.c.scales ? a.c.scales[kv] : 1.0f, vs = a.c.scales ? a.c.scales[a.c.n_kv + kv] : 1.0f;
  const float unit = a.scale * ks * (a.softcap > 0 ? 1.0f / a.softcap : kLog2e), cap2 = a.softcap * kLog2e;

  // The 8 dimensions that a lane brings to the k-th inner step of the first
  // product, of K and of q alike; in an 8-bit row, two steps' are side by side,
  // one 16-byte read.
  constexpr bool PAIRED = LIE == WHOLE && sizeof(CT) == 1;
  const auto dim_of = [&](int k) { return PAIRED ? 64 * (k / 2) + 16 * grp + 8 * (k % 2) : 32 * k + 8 * grp; };

  // rows of this lane: column `col` of each tile
  int32_t pos[MT];
  float slope[MT];
  v8 qf[MT][KK];
#pragma unroll
  for (int m = 0; m < MT; ++m) {
    const int32_t r = min(m * 16 + col, rows - 1), i = r / gh, h = h0 + r % gh;
    pos[m] = q.cached + i;
    slope[m] = a.slopes ? a.slopes[h] * kLog2e : 0.0f;
    const T *src = static_cast<const T *>(a.q) + (q.r0 + i) * a.q_stride + int64_t(h) * hd;
#pragma unroll
    for (int k = 0; k < KK; ++k) {
      const int d = dim_of(k);
      u32x4_t x = {0, 0, 0, 0};
      if (m * 16 + col < rows && (LIE == WHOLE || d < hd)) x = *reinterpret_cast<const u32x4_t *>(src + d);
      qf[m][k] = __builtin_bit_cast(v8, x);
    }
  }
  float top[MT], sum[MT];
  f32x4 o[MT][ND];
#pragma unroll
  for (int m = 0; m < MT; ++m) {
    top[m] = -INFINITY;
    sum[m] = 0;
#pragma unroll
    for (int e = 0; e < ND; ++e) o[m][e] = f32x4{0, 0, 0, 0};
  }

  // What a step reads, and which of its tokens are there (bit per token of
  // the lane: 4 of each tile).
  struct Step {
    typename KC::raw k[U][KK];
    typename VC::raw v[U][4][VP];
    uint32_t there;
  };
  const bool quads = a.c.bt % 4 == 0;  // 4 tokens from a multiple of 4 on lie in one block
  const int32_t row_step = a.c.tok_stride;
  int32_t left_lo = INT32_MAX, left_hi = 0;  // the wave's steps with infinities or NaN to be looked for again
  bool bad = false;
  auto block_of = [&](int32_t t) __attribute__((always_inline)) -> int32_t {  // t's block id, -1 for none
    if (t >= hi) return -1;
    const int32_t p = table[divided(t, a.bt_magic)];
    if (p < -1 || p >= a.c.num_blocks) bad = true;
    return uint32_t(p) < uint32_t(a.c.num_blocks) ? p : -1;
  };
  // bytes of a lane's chunks in a row; beyond head_dim: the row's begin
  uint32_t kd[KK], vd[VP];
#pragma unroll
  for (int k = 0; k < KK; ++k) kd[k] = (LIE == WHOLE || dim_of(k) < hd ? dim_of(k) : 0) * int(sizeof(CT));
#pragma unroll
  for (int c = 0; c < VP; ++c) vd[c] = (LIE == WHOLE || col * ND + c * NV < hd ? col * ND + c * NV : 0) * int(sizeof(CT));
  auto offset_of = [&](int32_t t, int32_t p) __attribute__((always_inline)) -> int64_t {  // of token t's row; an absent one is read from block 0 and masked
    return p < 0 ? 0 : p * a.c.block_stride + int64_t(t - int32_t(divided(t, a.bt_magic)) * a.c.bt) * a.c.tok_stride;
  };
  auto load = [&](int32_t t0, Step &x) __attribute__((always_inline)) {
    x.there = 0;
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const char *kt, *vt;  // of the lane's token of K, of its first of V
      if constexpr (LIE != ANY) {
        const int32_t t = t0 + 16 * u, p = block_of(t);
        const int64_t off = offset_of(t, p);
        if (p >= 0) x.there |= 0xfu << (4 * u);
        kt = kbase + off + uint32_t(col * a.c.tok_stride);
        vt = vbase + off + uint32_t(4 * grp * a.c.tok_stride);
      } else {
        const int32_t t = t0 + 16 * u + col, tv = t0 + 16 * u + 4 * grp;
        kt = kbase + offset_of(t, block_of(t));
        const int32_t p = block_of(tv);
        vt = vbase + offset_of(tv, p);
        if (quads && p >= 0) x.there |= 0xfu << (4 * u);
      }
#pragma unroll
      for (int k = 0; k < KK; k += PAIRED ? 2 : 1) {
        if constexpr (PAIRED) {
          const u32x4_t w = *reinterpret_cast<const u32x4_t *>(kt + kd[k]);
          x.k[u][k] = typename KC::raw{w[0], w[1]};
          x.k[u][k + 1] = typename KC::raw{w[2], w[3]};
        } else {
          x.k[u][k] = *reinterpret_cast<const typename KC::raw *>(kt + kd[k]);
        }
      }
      if (LIE != ANY || quads) {
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
          for (int c = 0; c < VP; ++c)
            x.v[u][i][c] = *reinterpret_cast<const typename VC::raw *>(vt + uint32_t(i * row_step) + vd[c]);
      } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const int32_t t = t0 + 16 * u + 4 * grp + i, p = block_of(t);
          if (p >= 0) x.there |= 1u << (4 * u + i);
#pragma unroll
          for (int c = 0; c < VP; ++c) x.v[u][i][c] = *reinterpret_cast<const typename VC::raw *>(vbase + offset_of(t, p) + vd[c]);
        }
      }
    }
  };

  auto compute = [&](int32_t t0, Step &x) __attribute__((always_inline)) {
    // every row sees every token of the step: the general case
    const bool whole = t0 + TS - 1 <= q.cached && t0 + TS <= hi && __ballot(x.there != (1u << 4 * U) - 1) == 0 &&
                       (a.window <= 0 || t0 > q.ctx - 1 - a.window);
    if (!whole) {
      // 0 times an unseen infinity or NaN would be NaN: they become 0 here, and
      // what of them is seen is put in behind the last step
      bool found = false;
#pragma unroll
      for (int u = 0; u < U; ++u)
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
          for (int c = 0; c < VP; ++c) found |= clean<T, CT>(x.v[u][i][c]);
      if (__ballot(found)) {
        left_lo = min(left_lo, t0);
        left_hi = t0 + TS;
      }
    }
    v8 ph[MT][U / 2], pl[MT][U / 2];
#pragma unroll
    for (int m = 0; m < MT; ++m) {
      f32x4 sc[U];
#pragma unroll
      for (int u = 0; u < U; ++u) {
        sc[u] = f32x4{0, 0, 0, 0};
#pragma unroll
        for (int k = 0; k < KK; ++k) {
          typename KC::raw kx = x.k[u][k];
          if (LIE != WHOLE && dim_of(k) >= hd) kx = typename KC::raw{};
          sc[u] = H::mfma16(KC::operand(kx), qf[m][k], sc[u]);
        }
      }
      // the lane's tokens are t0 + 4 grp + token_of(e)
      float z[4 * U];
#pragma unroll
      for (int e = 0; e < 4 * U; ++e) z[e] = sc[e / 4][e % 4] * unit;
      if (a.softcap > 0) {
#pragma unroll
        for (int e = 0; e < 4 * U; ++e) z[e] = cap2 * tanh_any(z[e]);
      }
      if (a.slopes) {
        const float from = float(t0 + 4 * grp - pos[m]);
#pragma unroll
        for (int e = 0; e < 4 * U; ++e) z[e] = __builtin_fmaf(slope[m], from + float(token_of(e)), z[e]);
      }
      if (!whole) {
        const int last = pos[m] - t0 - 4 * grp, first = a.window > 0 ? last - a.window : -1;
#pragma unroll
        for (int e = 0; e < 4 * U; ++e) {
          const bool seen = bool(token_of(e) <= last) & bool(token_of(e) > first) & bool(x.there >> e & 1);
          z[e] = seen ? z[e] : -INFINITY;
        }
      }
      float most = z[0];
#pragma unroll
      for (int e = 1; e < 4 * U; ++e) most = fmaxf(most, z[e]);
      if (__ballot(most - H::kLift > top[m] + 8.0f)) {
        most = fmaxf(most, __shfl_xor(most, 16));
        most = fmaxf(most, __shfl_xor(most, 32));
        const float now = fmaxf(top[m], most - H::kLift);
        const float keep = now == top[m] ? 1.0f : __builtin_amdgcn_exp2f(top[m] - now);
        top[m] = now;
        sum[m] *= keep;
#pragma unroll
        for (int e = 0; e < ND; ++e) o[m][e] *= keep;
      }
      // below any score but not -infinity, so that -infinity - it stays -infinity
      const float ref = top[m] == -INFINITY ? -3.0e38f : top[m];
      float p[4 * U];
#pragma unroll
      for (int e = 0; e < 4 * U; ++e) {
        p[e] = __builtin_amdgcn_exp2f(z[e] - ref);
        sum[m] += p[e];
      }
#pragma unroll
      for (int g = 0; g < U / 2; ++g) {
        u32x4_t hw, lw;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const float p0 = p[8 * g + 2 * e], p1 = p[8 * g + 2 * e + 1];
          const typename H::v2 first = {T(p0), T(p1)};
          hw[e] = __builtin_bit_cast(uint32_t, first);
          lw[e] = pack2<T>(p0 - float(first[0]), p1 - float(first[1]));
        }
        ph[m][g] = __builtin_bit_cast(v8, hw);
        pl[m][g] = __builtin_bit_cast(v8, lw);
      }
    }
#pragma unroll
    for (int g = 0; g < U / 2; ++g)
#pragma unroll
      for (int e = 0; e < ND; ++e) {
        u32x4_t f;
#pragma unroll
        for (int d = 0; d < 4; ++d) {  // tokens 2 d, 2 d + 1 of the lane's 8
          const uint32_t x0 = VC::pair(x.v[2 * g + d / 2][2 * (d % 2)][e / NV], e % NV / 2);
          const uint32_t x1 = VC::pair(x.v[2 * g + d / 2][2 * (d % 2) + 1][e / NV], e % NV / 2);
          f[d] = e % 2 ? high_halves(x0, x1) : low_halves(x0, x1);
        }
        const v8 vf = __builtin_bit_cast(v8, f);
#pragma unroll
        for (int m = 0; m < MT; ++m) {
          o[m][e] = H::mfma16(vf, ph[m][g], o[m][e]);
          o[m][e] = H::mfma16(vf, pl[m][g], o[m][e]);
        }
      }
  };

  // The next step's reads are in flight while one is computed: two sets of
  // registers in turn, as moving them would wait for the reads.
  {
    Step x, y;
    int32_t t0 = lo + wave * TS;
    if (t0 < hi) load(t0, x);
    while (t0 < hi) {
      const int32_t t1 = t0 + kFewWaves * TS, t2 = t1 + kFewWaves * TS;
      if (t1 < hi) load(t1, y);
      compute(t0, x);
      if (t1 >= hi) break;
      if (t2 < hi) load(t2, x);
      compute(t1, y);
      t0 = t2;
    }
  }
  // A seen infinity or NaN of V makes its dimension one, whatever its weight:
  // those cleaned out of a step are still to be added, and in a step that all
  // rows saw the two parts of a weight (0, or of unlike signs) may have made an
  // infinity a NaN.  Where such a step left a result that is not finite, the
  // wave's steps are gone through again (rarely; a score of NaN makes the whole
  // row one and needs nothing).
  bool odd = false;
#pragma unroll
  for (int m = 0; m < MT; ++m) {
    sum[m] += __shfl_xor(sum[m], 16);
    sum[m] += __shfl_xor(sum[m], 32);
    f32x4 z = {0, 0, 0, 0};  // 0, or NaN
#pragma unroll
    for (int e = 0; e < ND; ++e) z += o[m][e] * 0.0f;
    odd |= fabsf(sum[m]) <= FLT_MAX && !all_finite(z);
  }
  if (__ballot(odd)) {
    left_lo = lo + wave * TS;
    left_hi = hi;
  }
  if (left_lo < left_hi) {
    f32x4 wild[MT][ND];  // the sums of what is seen and not finite
#pragma unroll
    for (int m = 0; m < MT; ++m)
#pragma unroll
      for (int e = 0; e < ND; ++e) wild[m][e] = f32x4{0, 0, 0, 0};
#pragma unroll 1
    for (int32_t t1 = left_lo; t1 < left_hi; t1 += kFewWaves * TS) {
      const int32_t mine = lane < TS ? block_of(t1 + lane) : -1;  // a token a lane
      uint64_t which = __ballot(mine >= 0 && not_finite_row<T, CT>(vbase + offset_of(t1 + lane, mine), hd));
#pragma unroll 1
      for (; which; which &= which - 1) {
        const int32_t t = t1 + __builtin_ctzll(which);
        const CT *const v = reinterpret_cast<const CT *>(vbase + offset_of(t, block_of(t)));
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
          for (int e = 0; e < ND; ++e) {
            const int d = (4 * grp + i) * ND + e;
            const float y = LIE == WHOLE || d < hd ? as_f32(v[d]) : 0.0f;
#pragma unroll
            for (int m = 0; m < MT; ++m) {
              const bool sees = t <= pos[m] && (a.window <= 0 || pos[m] - t < a.window);
              if (sees && !(fabsf(y) <= FLT_MAX)) wild[m][e][i] += y;
            }
          }
      }
    }
#pragma unroll
    for (int m = 0; m < MT; ++m)
#pragma unroll
      for (int e = 0; e < ND; ++e)
#pragma unroll
        for (int i = 0; i < 4; ++i)
          if (wild[m][e][i] != 0) o[m][e][i] = wild[m][e][i];  // NaN is not 0 either
  }
  if (__ballot(bad) && lane == 0) flag(a.status, ATP_EINVAL);

  // join the four waves through shared memory, then write the rows
  __shared__ float so[kFewWaves][16][HD + 4];
  __shared__ float stop[kFewWaves][16], ssum[kFewWaves][16];
#pragma unroll
  for (int m = 0; m < MT; ++m) {
    if (m * 16 >= rows) break;
    if (m) __syncthreads();
    if (grp == 0) {
      stop[wave][col] = top[m];
      ssum[wave][col] = sum[m];
    }
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int e = 0; e < ND; e += 4)  // ND dimensions from (4 grp + i) * ND on
        *reinterpret_cast<f32x4 *>(&so[wave][col][(4 * grp + i) * ND + e]) = f32x4{o[m][e][i], o[m][e + 1][i], o[m][e + 2][i], o[m][e + 3][i]};
    __syncthreads();
    // 16 threads a row, 4 dimensions at a time
    const int r = threadIdx.x >> 4, part = threadIdx.x & 15;
    if (m * 16 + r < rows) {
      float all = -INFINITY, total = 0, f[kFewWaves];
#pragma unroll
      for (int w = 0; w < kFewWaves; ++w) all = fmaxf(all, stop[w][r]);
#pragma unroll
      for (int w = 0; w < kFewWaves; ++w) {
        f[w] = stop[w][r] == all ? 1.0f : __builtin_amdgcn_exp2f(stop[w][r] - all);
        total += f[w] * ssum[w][r];
      }
      const float inv = total == 0 ? 0.0f : vs / total;
      const float lse2 = total == 0 ? -INFINITY : all + __builtin_amdgcn_logf(total);
      const int32_t i = (m * 16 + r) / gh, h = h0 + (m * 16 + r) % gh;
      const int64_t row = int64_t(q.r0 + i) * a.h.n_q + h;
#pragma unroll
      for (int d = part * 4; d < HD; d += 64) {
        if (LIE != WHOLE && d >= hd) break;
        f32x4 x = {0, 0, 0, 0};
#pragma unroll
        for (int w = 0; w < kFewWaves; ++w) x += *reinterpret_cast<const f32x4 *>(&so[w][r][d]) * f[w];
        if (!all_finite(x)) {
          x = f32x4{0, 0, 0, 0};
          for (int w = 0; w < kFewWaves; ++w) add_share(x, *reinterpret_cast<const f32x4 *>(&so[w][r][d]), f[w]);
        }
        x *= inv;
        if (sh.count > 1) {
          *reinterpret_cast<f32x4 *>(a.split.part + (int64_t(blockIdx.x) * a.split.n_split + m * 16 + r) * hd + d) = x;
        } else {
          T *dst = static_cast<T *>(a.out) + (q.r0 + i) * a.out_stride + int64_t(h) * hd + d;
          *reinterpret_cast<u32x2_t *>(dst) = u32x2_t{pack2<T>(x[0], x[1]), pack2<T>(x[2], x[3])};
        }
      }
      if (part == 0) {
        if (sh.count > 1)
          a.split.part_lse[int64_t(blockIdx.x) * a.split.n_split + m * 16 + r] = lse2;
        else if (a.lse)
          a.lse[row] = lse2 * kLn2;
      }
    }
  }
}

template <typename T, typename CT, int HD, int LIE>
void launch(const AttendKernel &a, dim3 grid, hipStream_t st) {
  const dim3 block(kFewWaves * 64);
  const int64_t rows = int64_t(a.max_fresh) * std::min(a.h.group, a.h.n_q);
  if constexpr (HD <= 128) {  // two tiles of 256 dimensions do not fit the registers
    if (rows > 16) {
      hipLaunchKernelGGL((k_few<T, CT, HD, LIE, 2>), grid, block, 0, st, a);
      return;
    }
  }
  hipLaunchKernelGGL((k_few<T, CT, HD, LIE, 1>), grid, block, 0, st, a);
}

template <typename T, typename CT, int HD>
void by_rows(const AttendKernel &a, dim3 grid, hipStream_t st) {
  if (a.c.bt % 16)
    launch<T, CT, HD, ANY>(a, grid, st);
  else if (a.c.hd < HD)
    launch<T, CT, HD, EVEN>(a, grid, st);
  else
    launch<T, CT, HD, WHOLE>(a, grid, st);
}

template <typename T, typename CT>
void by_shape(const AttendKernel &a, dim3 grid, hipStream_t st) {
  if (a.c.hd <= 64)
    by_rows<T, CT, 64>(a, grid, st);
  else if (a.c.hd <= 128)
    by_rows<T, CT, 128>(a, grid, st);
  else
    by_rows<T, CT, 256>(a, grid, st);
}

}  // namespace

void attend_few(const AttendKernel &a, dim3 grid, hipStream_t st) {
  const bool b = a.dtype == ATP_BF16, e = a.cache_dtype == ATP_E4M3;
  if (b && e)
    by_shape<__bf16, E4M3>(a, grid, st);
  else if (b)
    by_shape<__bf16, __bf16>(a, grid, st);
  else if (e)
    by_shape<_Float16, E4M3>(a, grid, st);
  else
    by_shape<_Float16, _Float16>(a, grid, st);
}

}  // namespace atp
