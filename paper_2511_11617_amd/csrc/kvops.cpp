// kvops.cpp — argument checks of the KV cache operators (host only): shapes,
// head ranges, alignment, overlaps and workspace sizes, all before the first
// HIP call; then the launchers of kvstep.hip and attend.hip.
#include "kvops.h"

#include <algorithm>
#include <cmath>
#include <initializer_list>
#include <string>

#include "plan.h"

namespace atp {
namespace {

[[noreturn]] void bad(int code, const std::string &m) { throw Error(code, m); }
void want(bool ok, const char *m) {
  if (!ok) bad(ATP_EINVAL, m);
}

uintptr_t at(const void *p) { return reinterpret_cast<uintptr_t>(p); }

bool meet(uintptr_t a, uint64_t an, uintptr_t b, uint64_t bn) { return an && bn && a < b + bn && b < a + an; }

// 16-bit rows: `rows` of them, `width` elements each, `stride` apart.
struct Rows {
  uintptr_t p;
  uint64_t stride, width, rows;  // bytes, bytes, count
  uint64_t bytes() const { return rows ? (rows - 1) * stride + width : 0; }
};

// Whether two sets of rows share a byte: with one stride, rows that keep to
// different parts of a wider row (q, k and v of one projection) do not.
bool meet(const Rows &a, const Rows &b) {
  if (!meet(a.p, a.bytes(), b.p, b.bytes())) return false;
  if (a.stride != b.stride || a.stride == 0) return true;
  const uint64_t d = a.p <= b.p ? (b.p - a.p) % a.stride : (a.stride - (a.p - b.p) % a.stride) % a.stride;
  return !(d >= a.width && a.stride - d >= b.width);
}

Rows rows_of(const void *p, int64_t stride, int64_t heads, int32_t hd, int32_t rows, const char *what) {
  const std::string w = what;
  if (!p) bad(ATP_EINVAL, w + " is NULL");
  if (stride < heads * hd) bad(ATP_EINVAL, w + ": stride below a row's width");
  if (stride >= (int64_t(1) << 40)) bad(ATP_EINVAL, w + ": stride too large");
  if (at(p) % 16 || stride % 8) bad(ATP_EALIGN, w + ": rows must be 16-byte aligned");
  return {at(p), uint64_t(stride) * 2, uint64_t(heads * hd) * 2, uint64_t(rows)};
}

// A buffer of the call, by its name in a refusal.
struct Buffer {
  const char *name;
  uintptr_t p;
  uint64_t n;
};

// Nothing that the kernels write may lie on what they read.
void check_apart(std::initializer_list<Buffer> written, std::initializer_list<Buffer> read) {
  for (const Buffer &w : written)
    for (const Buffer &r : read)
      if (meet(w.p, w.n, r.p, r.n)) bad(ATP_EINVAL, std::string(w.name) + " overlaps " + r.name);
}

int elem_bytes(int32_t t) { return t == ATP_E4M3 ? 1 : 2; }

void check_blocks(const atp_kv_cache &c) {
  want(c.block_tokens > 0, "cache: block_tokens must be positive");
  want(c.num_blocks > 0 && c.num_blocks < (int64_t(1) << 31), "cache: num_blocks must be positive and fit int32");
}

void check_table(const atp_kv_step &s) {
  want(s.n_seq >= 0 && s.max_blocks >= 0 && s.max_tokens >= 0, "step: negative size");
  want(s.max_blocks > 0 || s.n_seq == 0, "step: max_blocks must be positive");
}

int64_t n_kv(const atp_kv_cache &c) { return c.kv_heads.end - c.kv_heads.begin; }

// Types, heads and shape: everything but the arena's address.
HeadRuns check_shape(const atp_kv_cache &c) {
  check_blocks(c);
  want(c.num_layers > 0, "cache: num_layers must be positive");
  want(c.head_dim > 0 && c.head_dim <= 256 && c.head_dim % 8 == 0, "cache: head_dim must be a multiple of 8, at most 256");
  want(c.layout == ATP_KV_HEAD_MAJOR || c.layout == ATP_KV_TOKEN_MAJOR, "cache: bad layout");
  want(c.dtype == ATP_BF16 || c.dtype == ATP_FP16, "cache: dtype must be ATP_BF16 or ATP_FP16");
  want(c.cache_dtype == c.dtype || c.cache_dtype == ATP_E4M3, "cache: cache_dtype must be dtype or ATP_E4M3");
  want((c.cache_dtype == ATP_E4M3) == (c.scales != nullptr), "cache: scales go with ATP_E4M3, and only with it");
  const atp_range q = c.q_heads, k = c.kv_heads;
  want(q.begin >= 0 && q.begin <= q.end && k.begin >= 0 && k.begin <= k.end, "cache: bad head range");
  want(q.end <= (1 << 20) && k.end <= (1 << 20), "cache: head range too large");
  want(c.group > 0 && c.group <= (1 << 20), "cache: group must be positive");
  HeadRuns h{int32_t(q.end - q.begin), 0, 0, c.group, 0};
  if (h.n_q) {
    const int64_t first = q.begin / c.group, last = (q.end - 1) / c.group;
    want(first >= k.begin && last < k.end, "cache: a query head's KV head is not in kv_heads");
    h.n_run = int32_t(last - first + 1);
    h.kv0 = int32_t(first - k.begin);
    h.cut = int32_t(q.begin - first * c.group);
  }
  const unsigned __int128 block = (unsigned __int128)n_kv(c) * c.block_tokens * c.head_dim * elem_bytes(c.cache_dtype);
  want(block < (1u << 31), "cache: a block of one layer must be below 2 GiB");
  return h;
}

CacheView check_arena(const atp_kv_cache &c, int32_t layer) {
  want(layer >= 0 && layer < c.num_layers, "layer out of range");
  const int64_t eb = elem_bytes(c.cache_dtype), line = int64_t(c.head_dim) * eb, heads = n_kv(c);
  const int64_t block = heads * c.block_tokens * line;
  const unsigned __int128 plane = (unsigned __int128)block * uint64_t(c.num_blocks);
  if (plane * 2 * unsigned(c.num_layers) > c.arena_bytes) bad(ATP_ECAPACITY, "cache: arena_bytes below the arena's size");
  if (heads) want(c.arena != nullptr, "cache: arena is NULL");
  if (at(c.arena) % 256) bad(ATP_EALIGN, "cache: arena must be 256-byte aligned");
  if (at(c.scales) % 4) bad(ATP_EALIGN, "cache: scales must be 4-byte aligned");
  CacheView v;
  v.base = static_cast<char *>(c.arena) + uint64_t(plane) * 2 * unsigned(layer);
  v.v_off = int64_t(plane);
  v.block_stride = block;
  const bool head = c.layout == ATP_KV_HEAD_MAJOR;
  v.head_stride = int32_t(head ? c.block_tokens * line : line);
  v.tok_stride = int32_t(head ? line : heads * line);
  v.bt = c.block_tokens;
  v.hd = c.head_dim;
  v.num_blocks = int32_t(c.num_blocks);
  v.n_kv = int32_t(heads);
  v.scales = c.scales ? c.scales + int64_t(layer) * 2 * heads : nullptr;
  return v;
}

// The arena as far as the cache fills it.
Buffer arena_of(const atp_kv_cache &c, const CacheView &v) {
  return {"the arena", at(c.arena), uint64_t(v.v_off) * 2 * uint64_t(c.num_layers)};
}
Buffer scales_of(const atp_kv_cache &c) {
  return {"scales", at(c.scales), c.scales ? uint64_t(c.num_layers) * 2 * uint64_t(n_kv(c)) * 4 : 0};
}

void check_workspace(const void *ws, uint64_t have, uint64_t need) {
  if (have < need) bad(ATP_ECAPACITY, "workspace too small: " + std::to_string(need) + " bytes are needed");
  if (!need) return;
  want(ws != nullptr, "workspace is NULL");
  if (at(ws) % 256) bad(ATP_EALIGN, "workspace must be 256-byte aligned");
}

void check_words(const void *p, int align, const char *what, bool may_be_null = false) {
  if (!p && !may_be_null) bad(ATP_EINVAL, std::string(what) + " is NULL");
  if (at(p) % uintptr_t(align)) bad(ATP_EALIGN, std::string(what) + " is not aligned to its elements");
}

AttendArgs attend_args(const atp_kv_cache *cache, const atp_kv_step *step) {
  want(cache && step, "cache or step is NULL");
  AttendArgs a{};
  a.h = check_shape(*cache);
  check_table(*step);
  want(step->max_fresh >= 0 && step->max_ctx >= 0, "step: negative bound");
  want(step->max_ctx <= (1 << 30), "step: max_ctx above 2^30");
  want(step->max_fresh <= step->max_ctx || step->n_seq == 0, "step: max_ctx below max_fresh");
  want(int64_t(step->max_tokens) * a.h.n_q < (int64_t(1) << 31), "step: max_tokens times query heads must fit int32");
  a.c.hd = cache->head_dim;
  a.c.bt = cache->block_tokens;
  a.dtype = cache->dtype;
  a.cache_dtype = cache->cache_dtype;
  a.n_seq = step->n_seq;
  a.max_blocks = step->max_blocks;
  a.max_tokens = step->max_tokens;
  a.max_fresh = step->max_fresh;
  a.max_ctx = step->max_ctx;
  return a;
}

}  // namespace

void extend_args(const atp_kv_cache *cache, const atp_kv_step *step, ExtendArgs *a) {
  want(cache && step, "cache or step is NULL");
  check_blocks(*cache);
  check_table(*step);
  *a = {};
  a->n_seq = step->n_seq;
  a->max_blocks = step->max_blocks;
  a->bt = cache->block_tokens;
  a->num_blocks = int32_t(cache->num_blocks);
  a->max_tokens = step->max_tokens;
}

void kv_extend(const atp_kv_cache *cache, const atp_kv_step *step, const int32_t *table, void *workspace,
               uint64_t workspace_bytes, atp_stream stream) {
  ExtendArgs a;
  extend_args(cache, step, &a);
  const bool seqs = a.n_seq > 0, rows = a.max_tokens > 0;
  check_words(table, 4, "table", !seqs);
  check_words(step->block_table, 4, "step: block_table", !seqs);
  check_words(step->cached, 4, "step: cached", !seqs);
  check_words(step->fresh, 4, "step: fresh", !seqs);
  check_words(step->starts, 4, "step: starts");
  check_words(step->slots, 8, "step: slots", !rows);
  check_words(step->positions, 4, "step: positions", !rows);
  check_words(step->status, 4, "step: status");
  const uint64_t cells = uint64_t(a.n_seq) * uint64_t(a.max_blocks) * 4, lens = uint64_t(a.n_seq) * 4;
  struct Part {
    const void *p;
    uint64_t n;
  };
  const uint64_t ws_need = extend_workspace(a);
  check_workspace(workspace, workspace_bytes, ws_need);
  const Part out[] = {{step->block_table, cells}, {step->starts, lens + 4}, {step->slots, uint64_t(a.max_tokens) * 8},
                      {step->positions, uint64_t(a.max_tokens) * 4}, {step->status, 16}, {workspace, ws_need}};
  const Part in[] = {{step->cached, lens}, {step->fresh, lens}, {table, cells}};
  for (const Part &o : out)
    for (const Part &i : in)
      want((&o == out && i.p == o.p && i.p == table) || !meet(at(o.p), o.n, at(i.p), i.n),
           "an output overlaps an input (block_table may only be `table` itself)");
  for (const Part &o : out)
    for (const Part &p : out) want(&o == &p || !meet(at(o.p), o.n, at(p.p), p.n), "two outputs overlap");
  a.table = table;
  a.new_table = step->block_table;
  a.cached = step->cached;
  a.fresh = step->fresh;
  a.starts = step->starts;
  a.slots = step->slots;
  a.positions = step->positions;
  a.status = step->status;
  extend_launch(a, workspace, stream);
}

void kv_append(const atp_kv_cache *cache, const atp_kv_step *step, int32_t layer, const atp_rope *rope, const void *q,
               int64_t q_stride, const void *k, int64_t k_stride, const void *v, int64_t v_stride, void *q_out,
               int64_t q_out_stride, atp_stream stream) {
  want(cache && step, "cache or step is NULL");
  const HeadRuns h = check_shape(*cache);
  AppendArgs a{};
  a.c = check_arena(*cache, layer);
  want(step->max_tokens >= 0, "step: negative size");
  // HIP counts a launch's threads in 32 bits: 2^24 - 1 workgroups of 256, 4 rows each
  want(step->max_tokens <= (1 << 26) - 4, "step: max_tokens must be at most 2^26 - 4");
  a.n_q = h.n_q;
  a.dtype = cache->dtype;
  a.cache_dtype = cache->cache_dtype;
  a.max_tokens = step->max_tokens;
  a.r.amplitude = 1;
  if (rope) {
    const atp_rope &r = *rope;
    want(r.rot_dim >= 0 && r.rot_dim % 2 == 0 && r.rot_dim <= cache->head_dim, "rope: rot_dim must be even, 0 to head_dim");
    want(std::isfinite(r.base) && r.base > 0, "rope: base must be positive");
    want(std::isfinite(r.amplitude), "rope: amplitude must be finite");
    want(r.scaling >= ATP_ROPE_PLAIN && r.scaling <= ATP_ROPE_PARTS, "rope: unknown scaling");
    if (r.scaling != ATP_ROPE_PLAIN) want(std::isfinite(r.factor) && r.factor > 0, "rope: factor must be positive");
    if (r.scaling == ATP_ROPE_PARTS) {
      want(std::isfinite(r.low) && std::isfinite(r.high) && r.low < r.high, "rope: low must be below high");
      want(std::isfinite(r.original) && r.original > 0, "rope: original must be positive");
    }
    a.r.pairs = r.rot_dim / 2;
    a.r.interleaved = r.interleaved != 0;
    a.r.amplitude = float(r.amplitude);
    for (int i = 0; i < a.r.pairs; ++i) {
      double f = std::pow(r.base, -2.0 * i / r.rot_dim);
      if (r.scaling == ATP_ROPE_LINEAR) f /= r.factor;
      if (r.scaling == ATP_ROPE_PARTS) {
        double keep = (r.original * f / (2 * M_PI) - r.low) / (r.high - r.low);
        keep = keep < 0 ? 0 : keep > 1 ? 1 : keep;
        f = f * keep + f / r.factor * (1 - keep);
      }
      a.r.turns[i] = f / (2 * M_PI);
      want(std::isfinite(a.r.turns[i]), "rope: a frequency is not finite");
    }
  }
  check_words(step->status, 4, "step: status", true);
  if (!a.max_tokens || (!a.n_q && !a.c.n_kv)) return;
  check_words(step->slots, 8, "step: slots");
  check_words(step->positions, 4, "step: positions");
  const int32_t hd = cache->head_dim;
  Rows out{}, in[3] = {};
  if (a.n_q) {
    in[0] = rows_of(q, q_stride, a.n_q, hd, a.max_tokens, "q");
    out = rows_of(q_out, q_out_stride, a.n_q, hd, a.max_tokens, "q_out");
  }
  if (a.c.n_kv) {
    in[1] = rows_of(k, k_stride, a.c.n_kv, hd, a.max_tokens, "k");
    in[2] = rows_of(v, v_stride, a.c.n_kv, hd, a.max_tokens, "v");
  }
  const Buffer arena = arena_of(*cache, a.c), turned{"q_out", out.p, out.bytes()},
      status{"status", at(step->status), step->status ? 4u : 0u};
  const Buffer slots{"slots", at(step->slots), uint64_t(a.max_tokens) * 8},
      positions{"positions", at(step->positions), uint64_t(a.max_tokens) * 4}, scales = scales_of(*cache);
  check_apart({status}, {slots, positions, scales, turned, arena, Buffer{"q", in[0].p, in[0].bytes()},
                         Buffer{"k", in[1].p, in[1].bytes()}, Buffer{"v", in[2].p, in[2].bytes()}});
  check_apart({turned, arena}, {slots, positions, scales});
  for (const Rows &r : in) {
    want((&r == in && r.p == out.p && r.stride == out.stride) || !meet(r, out), "q_out overlaps an input");
    want(!meet(r.p, r.bytes(), at(cache->arena), cache->arena_bytes), "the arena overlaps an input");
  }
  want(!meet(out.p, out.bytes(), at(cache->arena), cache->arena_bytes), "q_out overlaps the arena");
  a.slots = step->slots;
  a.positions = step->positions;
  a.q = q;
  a.k = k;
  a.v = v;
  a.q_out = q_out;
  a.q_stride = q_stride;
  a.k_stride = k_stride;
  a.v_stride = v_stride;
  a.q_out_stride = q_out_stride;
  a.status = step->status;
  append_launch(a, stream);
}

uint64_t kv_attend_workspace(const atp_kv_cache *cache, const atp_kv_step *step) {
  return attend_workspace(attend_args(cache, step));
}

void kv_attend(const atp_kv_cache *cache, const atp_kv_step *step, int32_t layer, const atp_kv_mask *mask, const void *q,
               int64_t q_stride, void *out, int64_t out_stride, float *lse, void *workspace, uint64_t workspace_bytes,
               atp_stream stream) {
  AttendArgs a = attend_args(cache, step);
  a.c = check_arena(*cache, layer);
  want(mask != nullptr, "mask is NULL");
  want(std::isfinite(mask->scale), "mask: scale must be finite");
  want(std::isfinite(mask->softcap) && (mask->softcap == 0 || mask->softcap >= 1e-6f), "mask: softcap must be 0 or at least 1e-6");
  want(mask->window >= 0, "mask: negative window");
  check_words(mask->slopes, 4, "mask: slopes", true);
  check_words(step->status, 4, "step: status", true);
  check_words(lse, 4, "lse", true);
  if (!a.n_seq || !a.max_tokens || !a.h.n_q || !a.max_fresh) return;
  check_words(step->block_table, 4, "step: block_table");
  check_words(step->cached, 4, "step: cached");
  check_words(step->starts, 4, "step: starts");
  const Rows in = rows_of(q, q_stride, a.h.n_q, cache->head_dim, a.max_tokens, "q");
  const Rows to = rows_of(out, out_stride, a.h.n_q, cache->head_dim, a.max_tokens, "out");
  const uint64_t ws_need = attend_workspace(a), lse_bytes = lse ? uint64_t(a.max_tokens) * a.h.n_q * 4 : 0;
  check_workspace(workspace, workspace_bytes, ws_need);
  const Buffer arena = arena_of(*cache, a.c), outs{"out", to.p, to.bytes()}, sums{"lse", at(lse), lse_bytes},
      work{"workspace", at(workspace), ws_need}, status{"status", at(step->status), step->status ? 4u : 0u};
  const uint64_t seqs = uint64_t(a.n_seq);
  const Buffer table{"block_table", at(step->block_table), seqs * uint64_t(a.max_blocks) * 4}, cached{"cached", at(step->cached), seqs * 4},
      starts{"starts", at(step->starts), seqs * 4 + 4}, slopes{"slopes", at(mask->slopes), mask->slopes ? uint64_t(a.h.n_q) * 4 : 0},
      scales = scales_of(*cache);
  check_apart({status}, {table, cached, starts, slopes, scales, outs, sums, work, arena, Buffer{"q", in.p, in.bytes()}});
  check_apart({outs, sums, work}, {table, cached, starts, slopes, scales});
  want(!meet(in, to), "out overlaps q");
  want(!meet(to.p, to.bytes(), at(cache->arena), cache->arena_bytes), "out overlaps the arena");
  want(!meet(at(lse), lse_bytes, to.p, to.bytes()) && !meet(at(lse), lse_bytes, in.p, in.bytes()) &&
           !meet(at(lse), lse_bytes, at(cache->arena), cache->arena_bytes),
       "lse overlaps another buffer");
  for (const Rows &r : {in, to}) want(!meet(at(workspace), ws_need, r.p, r.bytes()), "workspace overlaps another buffer");
  want(!meet(at(workspace), ws_need, at(lse), lse_bytes) &&
           !meet(at(workspace), ws_need, at(cache->arena), cache->arena_bytes),
       "workspace overlaps another buffer");
  a.table = step->block_table;
  a.starts = step->starts;
  a.cached = step->cached;
  a.scale = mask->scale;
  a.softcap = mask->softcap;
  a.window = std::min(mask->window, 1 << 30);  // no context is longer, and differences with it stay in 32 bits
  a.slopes = mask->slopes;
  a.q = q;
  a.out = out;
  a.q_stride = q_stride;
  a.out_stride = out_stride;
  a.lse = lse;
  a.status = step->status;
  attend_launch(a, workspace, stream);
}

}  // namespace atp
