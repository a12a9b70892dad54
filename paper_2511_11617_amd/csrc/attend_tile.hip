// attend_tile.hip — attention of prompts: many rows share a KV head's
// tokens.  Bound by the matrix units (4 dim operations per visible pair).
//
// One workgroup takes 128 rows of one (sequence, run of query heads with one
// KV head): row r is token r / heads, head r % heads, so that every row of
// the tile uses the same K and V.  Four waves hold 32 rows each; tiles of 64
// tokens of K and V pass through shared memory, two buffers deep, one barrier
// a tile.  Both products are taken transposed:
//   S^T = K Q^T (operand A: 32 tokens of K), O^T = V^T P^T (A: 32 dimensions)
// so a row is a column of both results: its maximum and sum stay in two lanes,
// and the weights are operand B of the second product where the first left
// them (the result's token order is the second product's inner order; V is
// read with the transposing LDS read in that same order).  The maximum moves
// only when a score passes it by 2^8.
// K rows are stored with their 16-byte chunks exchanged by the token (chunk
// ^ token), V rows with their 64-byte parts exchanged by it, so that neither
// read meets a bank twice; where the cache's elements are the products' own
// and fill the row, the loads go straight to shared memory (the lane picks
// the chunk that belongs at its place).
//
// Measured (128 dimensions, bf16): 900 TFLOP/s where the chip is full (8 prompts
// of 8192 behind 8192; 700 from an 8-bit cache), 860 for one such prompt, where
// a library product of 8192^3 reaches 1270.  In the latter a SIMD unit ends a
// wave's tile every 2670 clocks (of 2.2 GHz), 1024 of them in its matrix unit,
// with 1.65 waves on it on average: two workgroups a CU, so that one's softmax
// runs beside the other's products (a lone wave takes 4200 clocks a tile).
#include "attend.h"

namespace atp {
namespace {

constexpr int kTileThreads = 256, kTileTokens = 64;

using lds_ptr = __attribute__((address_space(3))) void *;
using glb_ptr = const __attribute__((address_space(1))) void *;
using i16x4 = short __attribute__((ext_vector_type(4)));

template <int HD>
struct Swizzle {
  static constexpr int kChunks = HD / 8;  // of 16 bytes, in a row
  // 16 tokens' equal chunks on 16 places; two rows of 64 dimensions share 256 bytes of banks
  static __device__ int k(int token) { return HD >= 128 ? token & 15 : (token >> 1) & 7; }
  static __device__ int v(int token) { return HD >= 128 ? (token & 3) << 2 : ((token >> 1) & 1) << 2; }
};

// The token of a lane's e-th score of a tile (two results of 16), for the lower half of the lanes; 4 more for the upper.
__device__ constexpr int token_of(int e) { return 32 * (e / 16) + 8 * (e % 16 / 4) + e % 4; }

template <typename T, typename CT, int HD, bool WHOLE, bool EXTRAS>
__global__ void __launch_bounds__(kTileThreads, HD == 256 ? 1 : 2) k_tile(AttendKernel a) {
  using H = Half16<T>;
  using v8 = typename H::v8;
  using SW = Swizzle<HD>;
  constexpr int KK = HD / 16, DT = HD / 32, ROW = HD * 2;
  constexpr bool DIRECT = WHOLE && sizeof(CT) == 2;
  constexpr int NCH = kTileTokens * SW::kChunks / kTileThreads;  // chunks a thread stages, of K and of V
  __shared__ __attribute__((aligned(256))) char lds[2][2][kTileTokens * ROW];
  __shared__ uint8_t there[2][kTileTokens];
  __shared__ int dirty[2];

  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), col = lane & 31, half = lane >> 5;
  TileItem it;
  if (a.split.items) {
    it = a.split.items[blockIdx.x];
  } else {
    if (int32_t(blockIdx.x) < a.n_seq && tid == 0 && !sequence(a, blockIdx.x).ok) flag(a.status, ATP_EINVAL);
    it = tile_of(a, blockIdx.x);
  }
  const auto uniform = [](int32_t x) { return __builtin_amdgcn_readfirstlane(x); };
  const int32_t s = uniform(it.s), run = uniform(it.run), tile = uniform(it.tile), lo = uniform(it.lo), hi = uniform(it.hi);
  if (s < 0) return;
  const Seq q = {uniform(it.r0), uniform(it.n), uniform(it.cached), uniform(it.cached) + uniform(it.n), true};
  int32_t h0;
  const int32_t gh = run_heads(a.h, run, &h0), rows = q.n * gh;

  const int32_t kv = a.h.kv0 + run, hd = a.c.hd;
  const int32_t row0 = tile * kTileRows, rowe = min(rows, row0 + kTileRows) - 1;
  const int32_t first_pos = q.cached + row0 / gh, last_pos = q.cached + rowe / gh;  // of the workgroup
  const int32_t *const table = a.table + int64_t(s) * a.max_blocks;
  const char *const kbase = a.c.base + int64_t(kv) * a.c.head_stride;
  const float ks = a.c.scales ? a.c.scales[kv] : 1.0f, vs = a.c.scales ? a.c.scales[a.c.n_kv + kv] : 1.0f;
  // the scale's sign goes with q, so that the largest product has the largest score
  // (a scale of 0 makes q 0, so that the unit is positive)
  const float unit = a.scale == 0 ? 1.0f : fabsf(a.scale) * ks * (EXTRAS && a.softcap > 0 ? 1.0f / a.softcap : kLog2e);
  const uint32_t sign = a.scale < 0 ? 0x80008000u : 0;

  const int32_t r = min(row0 + wave * 32 + col, rows - 1), tok = r / gh, head = h0 + r % gh, pos = q.cached + tok;
  const bool mine = row0 + wave * 32 + col < rows;
  const float slope = a.slopes ? a.slopes[head] * kLog2e : 0.0f;
  // the wave's first and last position
  const int32_t wfirst = q.cached + min(row0 + wave * 32, rows - 1) / gh, wlast = q.cached + min(row0 + wave * 32 + 31, rows - 1) / gh;
  const bool idle = row0 + wave * 32 >= rows;  // it only loads
  float top = -INFINITY, sum = 0;
  f32x16 o[DT];
#pragma unroll
  for (int d = 0; d < DT; ++d) o[d] = f32x16{};

  int32_t left_lo = INT32_MAX, left_hi = 0;  // tokens whose infinities and NaN are to be looked for again
  bool bad = false;
  auto block_of = [&](int32_t t) -> int32_t {
    if (t >= hi) return -1;
    const int32_t p = table[divided(t, a.bt_magic)];
    if (p < -1 || p >= a.c.num_blocks) bad = true;
    return uint32_t(p) < uint32_t(a.c.num_blocks) ? p : -1;
  };
  auto offset_of = [&](int32_t t, int32_t p) -> int64_t {
    return p < 0 ? 0 : p * a.c.block_stride + int64_t(t - int32_t(divided(t, a.bt_magic)) * a.c.bt) * a.c.tok_stride;
  };

  // Reads a tile of 64 tokens: to shared memory (DIRECT), or to registers that
  // store() converts and writes.  An absent token is read from block 0.
  struct Regs {
    uint32_t x[DIRECT ? 1 : NCH][2][sizeof(CT) == 2 ? 4 : 2];
    bool here[DIRECT ? 1 : NCH];
  };
  auto load = [&](int32_t t0, int buf, Regs &g) __attribute__((always_inline)) {
    if constexpr (DIRECT) {
      const int32_t t = t0 + 16 * wave, p = block_of(t);
      const char *const from = kbase + offset_of(t, p);
      constexpr int RPI = 1024 / ROW;  // rows of one instruction
      const int at = lane % SW::kChunks, sub = lane / SW::kChunks;
#pragma unroll
      for (int i = 0; i < 16 / RPI; ++i) {
        const int row = i * RPI + sub;
        const uint32_t line = row * a.c.tok_stride;
        char *const to = &lds[buf][0][(16 * wave + i * RPI) * ROW];
        __builtin_amdgcn_global_load_lds((glb_ptr)(from + line + ((at ^ SW::k(row)) << 4)), (lds_ptr)to, 16, 0, 0);
        __builtin_amdgcn_global_load_lds((glb_ptr)(from + a.c.v_off + line + ((at ^ SW::v(row)) << 4)),
                                         (lds_ptr)(to + kTileTokens * ROW), 16, 0, 0);
      }
      if (lane < 16) there[buf][16 * wave + lane] = p >= 0;
    } else {
#pragma unroll
      for (int i = 0; i < NCH; ++i) {
        const int idx = i * kTileThreads + tid, row = idx / SW::kChunks, c = idx % SW::kChunks;
        const int32_t t = t0 + row, p = block_of(t);
        const char *const from = kbase + offset_of(t, p) + c * 8 * int(sizeof(CT));
        const bool in = WHOLE || c * 8 < hd;
        using raw = typename std::conditional<sizeof(CT) == 2, u32x4_t, u32x2_t>::type;
        raw k = raw{}, v = raw{};
        if (in) {
          k = *reinterpret_cast<const raw *>(from);
          v = *reinterpret_cast<const raw *>(from + a.c.v_off);
        }
#pragma unroll
        for (int j = 0; j < int(sizeof(raw) / 4); ++j) {
          g.x[i][0][j] = k[j];
          g.x[i][1][j] = v[j];
        }
        g.here[i] = p >= 0;
      }
    }
  };
  auto store = [&](int buf, const Regs &g) __attribute__((always_inline)) {
    if constexpr (!DIRECT) {
#pragma unroll
      for (int i = 0; i < NCH; ++i) {
        const int idx = i * kTileThreads + tid, row = idx / SW::kChunks, c = idx % SW::kChunks;
#pragma unroll
        for (int w = 0; w < 2; ++w) {
          u32x4_t y;
          if constexpr (sizeof(CT) == 2)
            y = u32x4_t{g.x[i][w][0], g.x[i][w][1], g.x[i][w][2], g.x[i][w][3]};
          else
            y = u32x4_t{H::fp8_lo(g.x[i][w][0]), H::fp8_hi(g.x[i][w][0]), H::fp8_lo(g.x[i][w][1]), H::fp8_hi(g.x[i][w][1])};
          *reinterpret_cast<u32x4_t *>(&lds[buf][w][row * ROW + ((c ^ (w ? SW::v(row) : SW::k(row))) << 4)]) = y;
        }
        if (c == 0) there[buf][row] = g.here[i];
      }
    }
  };

  // the first tile is on its way while q comes in
  Regs first_tile;
  load(lo, 0, first_tile);
  v8 qf[KK];
  {
    const T *src = static_cast<const T *>(a.q) + (q.r0 + tok) * a.q_stride + int64_t(head) * hd;
#pragma unroll
    for (int k = 0; k < KK; ++k) {
      u32x4_t x = {0, 0, 0, 0};
      const int d = 16 * k + 8 * half;
      if (mine && a.scale != 0 && (WHOLE || d < hd)) x = *reinterpret_cast<const u32x4_t *>(src + d) ^ sign;
      qf[k] = __builtin_bit_cast(v8, x);
    }
  }

  // Operand A of the second product: of dimension 32 d + lane % 32, the tokens
  // 16 k + 4 half + (0..3) and those 8 further on.
  auto v_operand = [&](const char *vl, int d, int k) __attribute__((always_inline)) {
    const int token = 16 * k + 4 * half + (lane & 15) / 4, c = 4 * d + 2 * ((lane >> 4) & 1) + (lane & 3) / 2;
    const char *const p = vl + token * ROW + ((c ^ SW::v(token)) << 4) + (lane & 1) * 8;
    const i16x4 x0 = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) i16x4 *)(lds_ptr)p);
    const i16x4 x1 = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) i16x4 *)(lds_ptr)(p + 8 * ROW));
    const u32x2_t y0 = __builtin_bit_cast(u32x2_t, x0), y1 = __builtin_bit_cast(u32x2_t, x1);
    return u32x4_t{y0[0], y0[1], y1[0], y1[1]};
  };

  auto compute = [&](int32_t t0, int buf, uint64_t seen) __attribute__((always_inline)) {
    // some row of the wave does not see some token of the tile: few tiles of a long context
    const bool mixed = t0 + kTileTokens - 1 > wfirst || seen != ~0ull || (a.window > 0 && t0 <= wlast - a.window);
    const char *const kl = lds[buf][0], *const vl = lds[buf][1];
    f32x16 sc[2];
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      sc[u] = f32x16{};
#pragma unroll
      for (int k = 0; k < KK; ++k) {
        const u32x4_t x = *reinterpret_cast<const u32x4_t *>(kl + (32 * u + col) * ROW + (((2 * k + half) ^ SW::k(col)) << 4));
        sc[u] = H::mfma32(__builtin_bit_cast(v8, x), qf[k], sc[u]);
      }
    }
    // scores in base 2; without extras, still without their unit
    if (EXTRAS) {
      if (a.softcap > 0) {
        float x = 0;
#pragma unroll
        for (int e = 0; e < 32; ++e) x = fmaxf(x, fabsf(sc[e / 16][e % 16]));
        const float cap2 = a.softcap * kLog2e;
        if (__ballot(!(x * unit <= kTanhSmall)) == 0) {  // most tiles of a cap that is there for outliers
#pragma unroll
          for (int e = 0; e < 32; ++e) sc[e / 16][e % 16] = cap2 * tanh_small(sc[e / 16][e % 16] * unit);
        } else {
#pragma unroll
          for (int e = 0; e < 32; ++e) sc[e / 16][e % 16] = cap2 * tanh_any(sc[e / 16][e % 16] * unit);
        }
      }
      if (a.slopes) {  // without a cap, the scores have their unit still to come
        const float from = slope * float(t0 + 4 * half - pos), u = a.softcap > 0 ? 1.0f : unit;
#pragma unroll
        for (int e = 0; e < 32; ++e) sc[e / 16][e % 16] = __builtin_fmaf(sc[e / 16][e % 16], u, __builtin_fmaf(slope, float(token_of(e)), from));
      }
    }
    if (mixed) {  // a lane's tokens are t0 + 4 half + token_of(e): seen from the window's begin to its own position
      const int last = pos - t0 - 4 * half, first = a.window > 0 ? last - a.window : -1;
#pragma unroll
      for (int e = 0; e < 32; ++e) sc[e / 16][e % 16] = token_of(e) <= last ? sc[e / 16][e % 16] : -INFINITY;
      if (a.window > 0) {
#pragma unroll
        for (int e = 0; e < 32; ++e) sc[e / 16][e % 16] = token_of(e) > first ? sc[e / 16][e % 16] : -INFINITY;
      }
      if (seen != ~0ull) {
        const uint64_t mine64 = seen >> (4 * half);
#pragma unroll
        for (int e = 0; e < 32; ++e)
          sc[e / 16][e % 16] = uint32_t(mine64 >> (token_of(e) & 32)) & (1u << (token_of(e) & 31)) ? sc[e / 16][e % 16] : -INFINITY;
      }
    }
    float most = sc[0][0];
#pragma unroll
    for (int e = 1; e < 32; ++e) most = fmaxf(most, sc[e / 16][e % 16]);
    if (!EXTRAS) most *= unit;
    if (__ballot(most - H::kLift > top + 8.0f)) {
      most = fmaxf(most, __shfl_xor(most, 32));
      const float now = fmaxf(top, most - H::kLift);
      const float keep = now == top ? 1.0f : __builtin_amdgcn_exp2f(top - now);
      top = now;
      sum *= keep;
#pragma unroll
      for (int d = 0; d < DT; ++d) o[d] *= keep;
    }
    // below any score but not -infinity, so that -infinity - it stays -infinity
    const float ref = top == -INFINITY ? -3.0e38f : top;
    // The weights are rounded to 16 bits for the second product, their sum is
    // not: over many tokens that is an error like the output's own rounding (1.4
    // times in all).  Two parts, as with few rows, would double the product that
    // bounds this kernel.
    u32x4_t pw[4];
#pragma unroll
    for (int e = 0; e < 32; e += 2) {
      const float z0 = sc[e / 16][e % 16], z1 = sc[e / 16][e % 16 + 1];
      const float p0 = __builtin_amdgcn_exp2f(EXTRAS ? z0 - ref : __builtin_fmaf(z0, unit, -ref));
      const float p1 = __builtin_amdgcn_exp2f(EXTRAS ? z1 - ref : __builtin_fmaf(z1, unit, -ref));
      sum += p0 + p1;
      pw[e / 8][e % 8 / 2] = pack2<T>(p0, p1);
    }
#pragma unroll
    for (int k = 0; k < 4; ++k)
#pragma unroll
      for (int d = 0; d < DT; ++d)
        o[d] = H::mfma32(__builtin_bit_cast(v8, v_operand(vl, d, k)), __builtin_bit_cast(v8, pw[k]), o[d]);
  };

  // 0 times an unseen infinity or NaN would be NaN: in a tile with something
  // unseen, V's values that are not finite become 0, and what of them is seen
  // is put in behind the last tile.
  auto clean = [&](int buf) __attribute__((always_inline)) {
    constexpr int kMine = kTileTokens * ROW / 16 / kTileThreads;
    u32x4_t x[kMine];
    uint32_t found = 0;
#pragma unroll
    for (int i = 0; i < kMine; ++i) x[i] = *reinterpret_cast<u32x4_t *>(&lds[buf][1][(i * kTileThreads + tid) * 16]);
#pragma unroll
    for (int i = 0; i < kMine; ++i)
#pragma unroll
      for (int j = 0; j < 4; ++j) found |= not_finite<T>(x[i][j]);
    if (found) {
#pragma unroll
      for (int i = 0; i < kMine; ++i)
        *reinterpret_cast<u32x4_t *>(&lds[buf][1][(i * kTileThreads + tid) * 16]) =
            u32x4_t{finite_only<T>(x[i][0]), finite_only<T>(x[i][1]), finite_only<T>(x[i][2]), finite_only<T>(x[i][3])};
      dirty[buf] = 1;
    }
    __syncthreads();
    return dirty[buf] != 0;
  };

  {
    Regs &g = first_tile;
    store(0, g);
    if (tid == 0) dirty[0] = 0;
    int buf = 0;
    for (int32_t t0 = lo; t0 < hi; t0 += kTileTokens, buf ^= 1) {
      // this tile has come in for every wave, and none reads the other buffer any more
      asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
      __syncthreads();
      if (tid == 0) dirty[buf ^ 1] = 0;  // for the next tile
      const uint64_t seen = __ballot(there[buf][lane] != 0);
      if (t0 + kTileTokens - 1 > first_pos || seen != ~0ull || (a.window > 0 && t0 <= last_pos - a.window)) {
        if (clean(buf)) {
          left_lo = min(left_lo, t0);
          left_hi = min(t0 + kTileTokens, hi);
        }
      }
      const bool more = t0 + kTileTokens < hi;
      if (more) load(t0 + kTileTokens, buf ^ 1, g);
      if (!idle && t0 <= wlast && (a.window <= 0 || t0 + kTileTokens > wfirst - a.window + 1)) compute(t0, buf, seen);
      if (more) store(buf ^ 1, g);
    }
  }
  // A seen infinity or NaN of V makes its dimension one, whatever its weight:
  // those cleaned out of a tile are still to be added, and in a tile that all
  // rows saw a weight (or a later scale) of 0 may have made one a NaN.  Where
  // such a tile left a result that is not finite, all tiles are gone through
  // again (rarely; a score of NaN makes the whole row one and needs nothing).
  sum += __shfl_xor(sum, 32);
  f32x4 z = {0, 0, 0, 0};  // 0, or NaN
#pragma unroll
  for (int d = 0; d < DT; ++d)
#pragma unroll
    for (int i = 0; i < 16; i += 4) z += f32x4{o[d][i], o[d][i + 1], o[d][i + 2], o[d][i + 3]} * 0.0f;
  if (__ballot(mine && fabsf(sum) <= FLT_MAX && !all_finite(z))) {
    left_lo = lo;
    left_hi = hi;
  }
  if (left_lo < left_hi) {
    f32x16 wild[DT];  // the sums of what is seen and not finite
#pragma unroll
    for (int d = 0; d < DT; ++d) wild[d] = f32x16{};
    const char *const vbase = kbase + a.c.v_off;
#pragma unroll 1
    for (int32_t t0 = left_lo; t0 < left_hi; t0 += kTileTokens) {
      const int32_t p = block_of(t0 + lane);  // a token a lane
      uint64_t which = __ballot(p >= 0 && not_finite_row<T, CT>(vbase + offset_of(t0 + lane, p), hd));
#pragma unroll 1
      for (; which; which &= which - 1) {
        const int32_t t = t0 + __builtin_ctzll(which);
        if (t > pos || (a.window > 0 && pos - t >= a.window)) continue;
        const CT *const v = reinterpret_cast<const CT *>(vbase + offset_of(t, block_of(t)));
#pragma unroll
        for (int d = 0; d < DT; ++d)
#pragma unroll
          for (int i = 0; i < 16; i += 4) {
            const int at = 32 * d + 2 * i + 4 * half;
            if (!WHOLE && at >= hd) continue;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
              const float x = as_f32(v[at + j]);
              wild[d][i + j] += fabsf(x) <= FLT_MAX ? 0.0f : x;
            }
          }
      }
    }
#pragma unroll
    for (int d = 0; d < DT; ++d)
#pragma unroll
      for (int i = 0; i < 16; ++i)
        if (wild[d][i] != 0) o[d][i] = wild[d][i];  // NaN is not 0 either
  }
  if (__ballot(bad) && lane == 0) flag(a.status, ATP_EINVAL);
  if (!mine) return;
  const float inv = sum == 0 ? 0.0f : vs / sum;
  const float lse2 = sum == 0 ? -INFINITY : top + __builtin_amdgcn_logf(sum);
  const int64_t row = int64_t(q.r0 + tok) * a.h.n_q + head;
  const bool parts = it.place >= 0;
  const int64_t at_part = int64_t(it.place) * kTileRows + wave * 32 + col;
  if (half == 0) {
    if (parts)
      a.split.part_lse[at_part] = lse2;
    else if (a.lse)
      a.lse[row] = lse2 * kLn2;
  }
  T *const dst = static_cast<T *>(a.out) + (q.r0 + tok) * a.out_stride + int64_t(head) * hd;
  float *const part = parts ? a.split.part + at_part * hd : nullptr;
#pragma unroll
  for (int d = 0; d < DT; ++d)
#pragma unroll
    for (int i = 0; i < 16; i += 4) {
      const int at = 32 * d + 2 * i + 4 * half;
      if (!WHOLE && at >= hd) continue;
      const f32x4 x = {o[d][i] * inv, o[d][i + 1] * inv, o[d][i + 2] * inv, o[d][i + 3] * inv};
      if (parts)
        *reinterpret_cast<f32x4 *>(part + at) = x;
      else
        *reinterpret_cast<u32x2_t *>(dst + at) = u32x2_t{pack2<T>(x[0], x[1]), pack2<T>(x[2], x[3])};
    }
}

template <typename T, typename CT, int HD, bool WHOLE>
void launch(const AttendKernel &a, dim3 grid, hipStream_t st) {
  if (a.softcap > 0 || a.slopes)
    hipLaunchKernelGGL((k_tile<T, CT, HD, WHOLE, true>), grid, dim3(kTileThreads), 0, st, a);
  else
    hipLaunchKernelGGL((k_tile<T, CT, HD, WHOLE, false>), grid, dim3(kTileThreads), 0, st, a);
}

template <typename T, typename CT>
void by_shape(const AttendKernel &a, dim3 grid, hipStream_t st) {
  const int hd = a.c.hd;
  const bool even = a.c.bt % 16 == 0;
  if (hd == 64 && even)
    launch<T, CT, 64, true>(a, grid, st);
  else if (hd == 128 && even)
    launch<T, CT, 128, true>(a, grid, st);
  else if (hd == 256 && even)
    launch<T, CT, 256, true>(a, grid, st);
  else if (hd <= 64)
    launch<T, CT, 64, false>(a, grid, st);
  else if (hd <= 128)
    launch<T, CT, 128, false>(a, grid, st);
  else
    launch<T, CT, 256, false>(a, grid, st);
}

}  // namespace

void attend_tiles(const AttendKernel &a, dim3 grid, hipStream_t st) {
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
