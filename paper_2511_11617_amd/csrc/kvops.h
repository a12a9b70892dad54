// kvops.h — KV cache operators of a serving step: what the host has checked
// and resolved (kvops.cpp, no HIP), handed to the kernels' launchers
// (kvstep.hip, attend.hip).
#pragma once

#include <stdint.h>

#include "../../include/atp.h"

namespace atp {

// The cache of one layer as a kernel addresses it: element (K|V, block p,
// head j, token o, dimension 0) lies v * v_off + p * block_stride +
// j * head_stride + o * tok_stride bytes behind base.  head_stride and
// tok_stride are below 2^31 (a block is), offsets in the arena are 64-bit.
struct CacheView {
  char *base;
  int64_t v_off, block_stride;
  int32_t head_stride, tok_stride;
  int32_t bt, hd;
  int32_t num_blocks;
  int32_t n_kv;         // KV heads of the arena
  const float *scales;  // this layer's [2][n_kv], E4M3 only
};

// Local query heads [0, n_q) in runs that share a KV head: run j of n_run
// reads KV head kv0 + j and holds the heads [max(0, j * group - cut),
// min(n_q, (j + 1) * group - cut)); the first and the last run may be short.
struct HeadRuns {
  int32_t n_q, n_run, kv0, group, cut;
};

struct ExtendArgs {
  const int32_t *table;
  int32_t *new_table;
  int32_t n_seq, max_blocks, bt, num_blocks;
  const int32_t *cached, *fresh;
  int32_t *starts;
  int64_t *slots;
  int32_t *positions;
  int32_t max_tokens;
  int32_t *status;
};
uint64_t extend_workspace(const ExtendArgs &a);
void extend_launch(const ExtendArgs &a, void *ws, void *stream);

constexpr int kMaxPairs = 128;  // head_dim is at most 256
struct RopeArgs {
  int32_t pairs;  // rot_dim / 2
  int32_t interleaved;
  float amplitude;
  double turns[kMaxPairs];  // revolutions per position
};
struct AppendArgs {
  CacheView c;
  RopeArgs r;
  int32_t n_q, dtype, cache_dtype, max_tokens;
  const int64_t *slots;
  const int32_t *positions;
  const void *q, *k, *v;
  void *q_out;
  int64_t q_stride, k_stride, v_stride, q_out_stride;  // elements
  int32_t *status;
};
void append_launch(const AppendArgs &a, void *stream);

struct AttendArgs {
  CacheView c;
  HeadRuns h;
  int32_t dtype, cache_dtype;
  const int32_t *table, *starts, *cached;
  int32_t n_seq, max_blocks, max_tokens, max_fresh, max_ctx;
  float scale, softcap;
  int32_t window;
  const float *slopes;
  const void *q;
  void *out;
  int64_t q_stride, out_stride;
  float *lse;
  int32_t *status;
};
uint64_t attend_workspace(const AttendArgs &a);
void attend_launch(const AttendArgs &a, void *ws, void *stream);

// How a call's context is cut over workgroups whose results are joined.
//   few rows   chunks of one length, found on the device, for about `groups`
//              workgroups over all sequences; workgroup w has the results'
//              place w, of n_split rows
//   many rows  a tile of 128 rows and a part of the tokens it sees is an item
//              of a list made on the device, longest first; each part of a
//              cut tile has a place of 128 rows.  Without a list, workgroup w
//              takes the whole tile w.
struct alignas(16) TileItem {
  int32_t s, run, tile, lo, hi;  // tokens [lo, hi); s < 0: none
  int32_t place;                 // of its results; -1: it writes the rows themselves
  int32_t r0, n, cached;         // the sequence's first row, new tokens and tokens before
  int32_t pad[3];
};
struct AttendSplit {
  int32_t groups, n_split;
  float *part, *part_lse;  // [place][rows][dim], [place][rows] (base 2)
  int32_t *shares;         // few: [n_seq][2], a sequence's first chunk and their number
  TileItem *items;
  int32_t *cuts;           // [tiles][2], a tile's first place and the number of its parts (0, 1: not cut)
  int32_t tiles, n_items;
};

// The checks of the entry points (Error on a refusal), before any HIP call.
void extend_args(const atp_kv_cache *cache, const atp_kv_step *step, ExtendArgs *a);
void kv_extend(const atp_kv_cache *cache, const atp_kv_step *step, const int32_t *table, void *workspace,
               uint64_t workspace_bytes, atp_stream stream);
void kv_append(const atp_kv_cache *cache, const atp_kv_step *step, int32_t layer, const atp_rope *rope, const void *q,
               int64_t q_stride, const void *k, int64_t k_stride, const void *v, int64_t v_stride, void *q_out,
               int64_t q_out_stride, atp_stream stream);
uint64_t kv_attend_workspace(const atp_kv_cache *cache, const atp_kv_step *step);
void kv_attend(const atp_kv_cache *cache, const atp_kv_step *step, int32_t layer, const atp_kv_mask *mask, const void *q,
               int64_t q_stride, void *out, int64_t out_stride, float *lse, void *workspace, uint64_t workspace_bytes,
               atp_stream stream);

}  // namespace atp
