// attend.h — what the attention kernels share: matrix instructions and their
// operands, a sequence's range of tokens, the score's extras and mask, and
// the places of tokens in the paged cache.
#pragma once
#include <cfloat>

#include "kvdev.h"

namespace atp {

using bf16x8 = __bf16 __attribute__((ext_vector_type(8)));
using f16x8 = _Float16 __attribute__((ext_vector_type(8)));
using f32x4 = float __attribute__((ext_vector_type(4)));
using f32x16 = float __attribute__((ext_vector_type(16)));

constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;

// What depends on the 16-bit type.  The softmax weights are taken as 2^(s - m
// + kLift) with m at most 8 below the largest score, so that in fp16 the
// largest, 2^15, does not overflow.  The lift keeps weights of 2^-21 of the
// largest normal there (2^-29 where that has risen by 2^8 since m was set); a
// smaller one is off by the type's least half step, 2^-25 / 2^7 = 2^-32 of the
// largest: over 131072 tokens, 2^-15 of the result in all at most, a sixteenth
// of its rounding.
template <typename T>
struct Half16;
template <>
struct Half16<__bf16> {
  using v8 = bf16x8;
  using v2 = bf16x2;
  static constexpr float kLift = 0;
  static constexpr uint32_t kExp = 0x7f80;  // exponent bits: all set = infinity or NaN
  static __device__ f32x4 mfma16(v8 a, v8 b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0); }
  static __device__ f32x16 mfma32(v8 a, v8 b, f32x16 c) { return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0); }
  static __device__ uint32_t fp8_lo(uint32_t x) { return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(x, 1.0f, false)); }
  static __device__ uint32_t fp8_hi(uint32_t x) { return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(x, 1.0f, true)); }
};
template <>
struct Half16<_Float16> {
  using v8 = f16x8;
  using v2 = f16x2;
  static constexpr float kLift = 7;
  static constexpr uint32_t kExp = 0x7c00;
  static __device__ f32x4 mfma16(v8 a, v8 b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0); }
  static __device__ f32x16 mfma32(v8 a, v8 b, f32x16 c) { return __builtin_amdgcn_mfma_f32_32x32x16_f16(a, b, c, 0, 0, 0); }
  static __device__ uint32_t fp8_lo(uint32_t x) { return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(x, 1.0f, false)); }
  static __device__ uint32_t fp8_hi(uint32_t x) { return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(x, 1.0f, true)); }
};

template <typename T>
__device__ inline uint32_t pack2(float a, float b) {
  typename Half16<T>::v2 v = {T(a), T(b)};
  return __builtin_bit_cast(uint32_t, v);
}

// Two dwords of 16-bit pairs -> their low halves, their high halves.
__device__ inline uint32_t low_halves(uint32_t a, uint32_t b) { return __builtin_amdgcn_perm(b, a, 0x05040100); }
__device__ inline uint32_t high_halves(uint32_t a, uint32_t b) { return __builtin_amdgcn_perm(b, a, 0x07060302); }

// x / d for x < 2^31 with magic = ceil(2^64 / d) (0 for d = 1).
__device__ inline uint32_t divided(uint32_t x, uint64_t magic) { return magic ? uint32_t(__umul64hi(x, magic)) : x; }

struct AttendKernel : AttendArgs {
  AttendSplit split;
  uint64_t bt_magic;
};

// Sequence s of the step, checked; `ok` false: nothing may be read for it.
struct Seq {
  int32_t r0, n, cached, ctx;  // first row, new tokens, tokens before, all tokens
  bool ok;
};
__device__ inline Seq sequence(const AttendArgs &a, int32_t s) {
  Seq q;
  q.r0 = a.starts[s];
  const int32_t r1 = a.starts[s + 1];
  q.cached = a.cached[s];
  q.n = r1 - q.r0;
  const int64_t ctx = int64_t(q.cached) + q.n;
  q.ok = q.r0 >= 0 && r1 >= q.r0 && r1 <= a.max_tokens && q.n <= a.max_fresh && q.cached >= 0 && ctx <= a.max_ctx &&
         ctx <= int64_t(a.max_blocks) * a.c.bt;
  q.ctx = int32_t(ctx);
  return q;
}

// The first token that any of the sequence's rows from position `pos` on
// sees, down to a multiple of `align`.
__device__ inline int32_t first_seen(const AttendArgs &a, int32_t pos, int32_t align) {
  const int32_t lo = a.window > 0 && pos >= a.window ? pos - a.window + 1 : 0;
  return lo / align * align;
}

// Local query heads [*h0, *h0 + count) of run j.
__host__ __device__ inline int32_t run_heads(const HeadRuns &h, int32_t j, int32_t *h0) {
  const int32_t b = j ? j * h.group - h.cut : 0, e = (j + 1) * h.group - h.cut;
  *h0 = b;
  return (e < h.n_q ? e : h.n_q) - b;
}

// tanh(x) where |x| is at most 0.4: its series to x^11, off by 2^-24 of itself.
__device__ inline float tanh_small(float x) {
  const float y = x * x;
  float p = -1382.0f / 155925.0f;
  p = __builtin_fmaf(p, y, 62.0f / 2835.0f);
  p = __builtin_fmaf(p, y, -17.0f / 315.0f);
  p = __builtin_fmaf(p, y, 2.0f / 15.0f);
  p = __builtin_fmaf(p, y, -1.0f / 3.0f);
  return __builtin_fmaf(p * y, x, x);
}
constexpr float kTanhSmall = 0.4f;
// tanh(x) = 1 - 2 / (e^2x + 1), off by a few units of 2^-24 of 1: too much near 0, where the series stands in.
__device__ inline float tanh_any(float x) {
  const float t = 1.0f - 2.0f * __builtin_amdgcn_rcpf(__builtin_amdgcn_exp2f(x * (2 * kLog2e)) + 1.0f);
  return fabsf(x) <= kTanhSmall ? tanh_small(x) : t;
}

// Two values of a 16-bit type with an infinity or NaN among them.
template <typename T>
__device__ inline bool not_finite(uint32_t x) {
  constexpr uint32_t lo = Half16<T>::kExp, hi = Half16<T>::kExp << 16;
  return (x & lo) == lo || (x & hi) == hi;
}
// x with 0 in the place of each half that is no number or no finite one.
template <typename T>
__device__ inline uint32_t finite_only(uint32_t x) {
  constexpr uint32_t e = Half16<T>::kExp;
  if ((x & e) == e) x &= 0xffff0000u;
  if ((x & e << 16) == e << 16) x &= 0xffffu;
  return x;
}
// The bytes of four e4m3 values that are NaN (0x7f, 0xff), as their highest bits.
__device__ inline uint32_t nan_bytes(uint32_t x) { return ((x & 0x7f7f7f7fu) + 0x01010101u) & 0x80808080u; }

// Whether a row of V (hd elements, a multiple of 8) holds an infinity or NaN.
template <typename T, typename CT>
__device__ inline bool not_finite_row(const char *row, int32_t hd) {
  bool found = false;
#pragma unroll 4
  for (int32_t d = 0; d < hd; d += 8) {
    if constexpr (sizeof(CT) == 2) {
      const u32x4_t x = *reinterpret_cast<const u32x4_t *>(row + 2 * d);
#pragma unroll
      for (int j = 0; j < 4; ++j) found |= not_finite<T>(x[j]);
    } else {
      const u32x2_t x = *reinterpret_cast<const u32x2_t *>(row + d);
      found |= (nan_bytes(x[0]) | nan_bytes(x[1])) != 0;
    }
  }
  return found;
}

// Whether all four are finite: 0 times anything else is NaN.
__device__ inline bool all_finite(f32x4 x) {
  const f32x4 z = x * 0.0f;
  return (z[0] + z[1]) + (z[2] + z[3]) == 0;
}

// Adds a part's result by its share of the whole; one that is not finite stays so even by 0.
__device__ inline void add_share(f32x4 &sum, f32x4 x, float share) {
#pragma unroll
  for (int i = 0; i < 4; ++i) sum[i] = fabsf(x[i]) <= FLT_MAX ? __builtin_fmaf(x[i], share, sum[i]) : sum[i] + x[i];
}

// The context's chunks begin at multiples of these.
constexpr int kFewAlign = 64, kTileAlign = 64;
constexpr int kFewLeast = 256;  // tokens of the shortest chunk of few rows
constexpr int kTileRows = 128;  // rows of a workgroup of attend_tile.hip

// Places for the tiles of rows of a run of gh heads: sequence s has those
// from starts[s] * gh / 128 + s on.
__host__ __device__ inline int64_t tile_slots(const AttendArgs &a, int32_t gh) {
  return int64_t(a.max_tokens) * gh / kTileRows + a.n_seq;
}

// Rounds of workgroups that few rows' chunks make: two where there are more
// sequences (times runs of heads) than the chip holds workgroups.
__host__ __device__ inline int64_t few_rounds(const AttendKernel &a) { return int64_t(a.n_seq) * a.h.n_run > a.split.groups ? 2 : 1; }

// The tile of rows that is number `item` of a call's, run by run (so that
// neighbours, which go to different dies, have alike work), and in a run from
// the last slot to the first; s < 0: none.
__device__ inline TileItem tile_of(const AttendArgs &a, int32_t item) {
  int32_t run = 0, slot = item, h0;
  int32_t n_slots = int32_t(tile_slots(a, run_heads(a.h, 0, &h0)));
  if (item >= n_slots) {
    const int32_t each = int32_t(tile_slots(a, a.h.group)), past = item - n_slots;
    run = min(1 + past / each, a.h.n_run - 1);
    slot = past - (run - 1) * each;
    n_slots = int32_t(tile_slots(a, run_heads(a.h, run, &h0)));
  }
  slot = n_slots - 1 - slot;
  const int32_t gh = run_heads(a.h, run, &h0);
  int32_t s = 0, hi_s = a.n_seq - 1;  // the last sequence whose slots begin at or before this one
  while (s < hi_s) {
    const int32_t mid = (s + hi_s + 1) >> 1;
    if (int64_t(a.starts[mid]) * gh / kTileRows + mid <= slot)
      s = mid;
    else
      hi_s = mid - 1;
  }
  const Seq q = sequence(a, s);
  const int32_t tile = slot - s - int32_t(int64_t(q.r0) * gh / kTileRows), rows = q.n * gh;
  if (!q.ok || tile < 0 || int64_t(tile) * kTileRows >= rows) return {-1, 0, 0, 0, 0, -1};
  const int32_t row0 = tile * kTileRows, rowe = min(rows, row0 + kTileRows) - 1;
  return {s, run, tile, first_seen(a, q.cached + row0 / gh, kTileAlign), q.cached + rowe / gh + 1, -1, q.r0, q.n, q.cached};
}

void attend_few(const AttendKernel &a, dim3 grid, hipStream_t st);
void attend_tiles(const AttendKernel &a, dim3 grid, hipStream_t st);

}  // namespace atp
