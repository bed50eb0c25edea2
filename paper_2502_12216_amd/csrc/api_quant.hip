// Host side of the quantised cache: rows in and out, chosen blocks, single-token decode.
#include <hip/hip_runtime.h>
#include <math.h>
#include <string.h>

#include <algorithm>
#include <initializer_list>

#include "host.hpp"
#include "plan.hpp"

using namespace tactic_host;
using tactic::kHeadDim;

namespace {

constexpr int64_t kMaxInt = ((int64_t)1 << 31) - 1;
// Scoring workgroups aimed at.  1024, 1536, 2048, 4096 of them, us for 65536 blocks: four heads, scores and
// choice 18.6, 18.2, 18.6, 19.6; eight heads, with the decode 49.3, 50.6, 50.9, 53.6; 8192 blocks of 8 heads
// 40.7, 40.7, 41.5, 43.6 (the choice reads a maximum of each); 256 and 512 were 4 and 1 slower than 1024.
constexpr int64_t kScoreGroups = 1024;
constexpr int32_t kMaxBudget = 1 << 27;  // the blocks of 2^31 rows

tactic_status check_aligned(std::initializer_list<const void*> arrays, int bytes) {
  for (const void* p : arrays)
    if (reinterpret_cast<uintptr_t>(p) % bytes) return fail(TACTIC_ERR_INVALID_ARG, "an array is not %d-byte aligned", bytes);
  return TACTIC_OK;
}

// Checks of the cache; `rows`: whether its rows are used, and not its bounds alone.
tactic_status quant_args(const tactic_quant_kv* kv, const tactic_kv_shape* s, bool rows, tactic::QuantKV* out) {
  if (!kv) return fail(TACTIC_ERR_INVALID_ARG, "kv is null");
  if (kv->bits != 8 && kv->bits != 4) return fail(TACTIC_ERR_INVALID_ARG, "bits must be 8 or 4 (got %d)", kv->bits);
  if (kv->block != 0 && kv->block != 16 && kv->block != 32 && kv->block != 64 && kv->block != 128)
    return fail(TACTIC_ERR_INVALID_ARG, "block must be 16, 32, 64 or 128, or 0 without bounds (got %d)", kv->block);
  if (kv->bounds && kv->block == 0) return fail(TACTIC_ERR_INVALID_ARG, "bounds need a block");
  if (rows && s->total_tokens > 0 && (!kv->K || !kv->K_scale || !kv->V || !kv->V_scale))
    return fail(TACTIC_ERR_INVALID_ARG, "null cache array");
  tactic_status st;
  if ((st = check_aligned({kv->K, kv->V, kv->bounds}, 16)) != TACTIC_OK || (st = check_aligned({kv->K_scale, kv->V_scale}, 4)) != TACTIC_OK)
    return st;
  *out = tactic::QuantKV{};
  out->K = kv->K;
  out->K_scale = kv->K_scale;
  out->V = kv->V;
  out->V_scale = kv->V_scale;
  out->bounds = kv->bounds;
  out->bits = kv->bits;
  out->block = kv->block;
  if (kv->page_table && rows) {
    const tactic_paged_kv pages{reinterpret_cast<const uint16_t*>(kv->K), reinterpret_cast<const uint16_t*>(kv->V),
                                kv->page_table, nullptr, kv->page_size, kv->max_pages, kv->num_pages};
    if ((st = paged_args(&pages, s, &out->pk)) != TACTIC_OK) return st;
    out->paged = 1;
  }
  return TACTIC_OK;
}

tactic_status check_new_rows(const tactic_query_shape* q, const tactic_kv_shape* s) {
  if (!q) return fail(TACTIC_ERR_INVALID_ARG, "rows is null");
  if (!q->q_indptr) return fail(TACTIC_ERR_INVALID_ARG, "q_indptr is null");
  if (q->total_queries > kMaxInt / s->n_kv_heads) return fail(TACTIC_ERR_UNSUPPORTED, "total_queries * n_kv_heads >= 2^31");
  if (q->total_queries < 0 || q->max_queries < 0 || q->max_queries > q->total_queries || q->total_queries > q->max_queries * s->batch)
    return fail(TACTIC_ERR_INVALID_ARG, "inconsistent total_queries / max_queries");
  return TACTIC_OK;
}

tactic::QuantRowsArgs rows_args(const tactic_kv_shape* s, const tactic_query_shape* rows, const tactic::QuantKV& kv) {
  tactic::QuantRowsArgs a{};
  a.kv_indptr = s->kv_indptr;
  a.seq_len = s->seq_len;
  a.row_indptr = rows->q_indptr;
  a.B = s->batch;
  a.Hkv = s->n_kv_heads;
  a.total = s->total_tokens;
  a.n_rows = rows->total_queries;
  a.kv = kv;
  return a;
}

// The arrays of a cache
struct CacheSpans {
  Span s[5];
};
CacheSpans spans_of(const tactic::QuantKV& c, const tactic_kv_shape* s) {
  const int64_t rows = c.paged ? c.pk.num_pages * s->n_kv_heads * c.pk.page_size : s->total_tokens * s->n_kv_heads;
  const int64_t bounds = c.bounds ? (s->total_tokens / c.block + s->batch) * s->n_kv_heads * (4 * kHeadDim) : 0;
  return {{{c.K, rows * 16 * c.bits}, {c.V, rows * 16 * c.bits}, {c.K_scale, rows * 4}, {c.V_scale, rows * 4}, {c.bounds, bounds}}};
}
// Workgroups write some arrays while others read and write theirs: no two may overlap.
tactic_status check_apart(const CacheSpans& cache, bool cache_written, const Span& x, const Span& y, bool written) {
  for (const Span& c : cache.s) {
    if (overlap(c, x) || overlap(c, y)) return fail(TACTIC_ERR_INVALID_ARG, "rows must not overlap the cache");
    for (const Span& d : cache.s)
      if (cache_written && &c < &d && overlap(c, d)) return fail(TACTIC_ERR_INVALID_ARG, "the cache's arrays must not overlap one another");
  }
  if (written && overlap(x, y)) return fail(TACTIC_ERR_INVALID_ARG, "the outputs must not overlap one another");
  return TACTIC_OK;
}

struct SelectLayout {
  int64_t max_blocks, per, tops, scores, top, keys, bytes;
};
SelectLayout select_layout(const tactic_kv_shape* s, int block) {
  SelectLayout l{};
  l.max_blocks = std::max<int64_t>(1, (s->max_seq_len + block - 1) / block);
  // scoring workgroups of whole 16 blocks, about four for each compute unit if the sequences are as long as the longest
  const int64_t all = l.max_blocks * s->batch * s->n_kv_heads;
  l.per = std::min<int64_t>(1024, std::max<int64_t>(16, (all / kScoreGroups + 15) / 16 * 16));
  l.tops = (l.max_blocks + l.per - 1) / l.per;
  Layout L;
  const int64_t heads = (int64_t)s->batch * s->n_q_heads;
  l.scores = L.take(heads * l.max_blocks * 8);
  l.top = L.take(heads * l.tops * 8);
  l.keys = l.max_blocks > tactic::kSelectHeld ? L.take((int64_t)s->batch * s->n_kv_heads * l.max_blocks * 8) : 0;
  l.bytes = L.cur;
  return l;
}

// Whether the decode gives every KV head one workgroup, which joins its own waves and writes the
// outputs, or splits all rows evenly and joins the parts in a second launch.  One workgroup takes 4 us
// (eight query heads: 5) and `step` us for 128 rows of its four waves, the longer the more of them
// share the memory, or what memory gives it; the split 10 to 12 us (eight heads: 12 to 18; a start that
// looks at every group, the second launch) and the bytes at 6 TB/s.  Measured, one against split, us
// a call, rows of 8 KV heads, 8 bits and 4 heads each: one sequence of 512 rows 7.7, 10.5; 768 9.2,
// 10.5; 1024 10.7, 10.5; 4 of 768 10.2, 10.8; 1024 12.0, 10.9; 16 of 1536 18.5, 19.6; 2048 24.2, 21.8; 32 of 2048 26.5,
// 34.2; 4 bits: one of 1024 9.0, 10.0; 1536 12.1, 10.0; 16 of 2048 15.8, 17.1; eight heads at 8 bits: one of
// 512 9.2, 12.0; 768 12.3, 12.1; 4 of 1024 13.4, 12.6; 16 of 2048 26.2, 26.8.  One workgroup is as slow
// as its longest sequence, so that it is not used from 2048 rows on.
bool one_workgroup(const tactic_kv_shape* s, int bits, int64_t most) {
  if (most > 2048) return false;
  const bool eight = s->n_q_heads / s->n_kv_heads == 8;
  const double groups = (double)s->batch * s->n_kv_heads, row = 2 * (16.0 * bits + 4) / 6e6;
  const double shared = std::min(groups, 256.0) / 256, doublings = std::max(0.0, log2(std::min(groups, 256.0) / 8));
  const double step = (bits == 8 ? 0.81 + 0.118 * doublings : 0.66 + 0.03 * doublings) + (eight ? 0.2 : 0.0);
  const double rounds = std::max(1.0, ceil(groups / 512));
  const double all = std::min((double)s->total_tokens * s->n_kv_heads, groups * (double)most);
  const double one = (eight ? 5.0 : 4.0) + (double)most * rounds * std::max(step / 128, std::min(groups, 512.0) * row);
  return one <= (eight ? 11.7 + 6.5 * shared : 10.0 + 2.0 * shared) + all * row;
}

bool is_block(int block) { return block == 16 || block == 32 || block == 64 || block == 128; }

}  // namespace

extern "C" {

tactic_status tactic_quant_write(const uint16_t* k, const uint16_t* v, const tactic_kv_shape* shape,
                                 const tactic_query_shape* rows, const tactic_quant_kv* kv, hipStream_t stream) {
  tactic_status st;
  tactic::QuantKV c;
  if ((st = check_shape(shape)) != TACTIC_OK || (st = check_new_rows(rows, shape)) != TACTIC_OK ||
      (st = quant_args(kv, shape, true, &c)) != TACTIC_OK)
    return st;
  if (rows->total_queries == 0 || shape->total_tokens == 0) return TACTIC_OK;
  if (!k || !v) return fail(TACTIC_ERR_INVALID_ARG, "null argument");
  const int64_t bytes = rows->total_queries * shape->n_kv_heads * kHeadDim * 2;
  if ((st = check_aligned({k, v}, 16)) != TACTIC_OK || (st = check_apart(spans_of(c, shape), true, {k, bytes}, {v, bytes}, false)) != TACTIC_OK)
    return st;
  tactic::QuantRowsArgs a = rows_args(shape, rows, c);
  a.k = k;
  a.v = v;
  const hipError_t e = tactic::launch_quant_write(a, stream);
  return e == hipSuccess ? TACTIC_OK : hip_fail(e, "quantised write launch");
}

tactic_status tactic_quant_read(const tactic_quant_kv* kv, const tactic_kv_shape* shape,
                                const tactic_query_shape* rows, uint16_t* K_out, uint16_t* V_out,
                                hipStream_t stream) {
  tactic_status st;
  tactic::QuantKV c;
  if ((st = check_shape(shape)) != TACTIC_OK || (st = check_new_rows(rows, shape)) != TACTIC_OK ||
      (st = quant_args(kv, shape, true, &c)) != TACTIC_OK)
    return st;
  if (rows->total_queries == 0) return TACTIC_OK;
  if (!K_out || !V_out) return fail(TACTIC_ERR_INVALID_ARG, "null argument");
  const int64_t bytes = rows->total_queries * shape->n_kv_heads * kHeadDim * 2;
  if ((st = check_aligned({K_out, V_out}, 16)) != TACTIC_OK ||
      (st = check_apart(spans_of(c, shape), false, {K_out, bytes}, {V_out, bytes}, true)) != TACTIC_OK)
    return st;
  tactic::QuantRowsArgs a = rows_args(shape, rows, c);
  a.K_out = K_out;
  a.V_out = V_out;
  const hipError_t e = tactic::launch_quant_read(a, stream);
  return e == hipSuccess ? TACTIC_OK : hip_fail(e, "quantised read launch");
}

size_t tactic_block_select_workspace_size(const tactic_kv_shape* shape, int32_t block) {
  if (check_shape(shape) != TACTIC_OK) return 0;
  if (!is_block(block)) {
    fail(TACTIC_ERR_INVALID_ARG, "block must be 16, 32, 64 or 128 (got %d)", block);
    return 0;
  }
  return (size_t)select_layout(shape, block).bytes;
}

tactic_status tactic_block_select(const uint16_t* q, const tactic_quant_kv* kv, const tactic_kv_shape* shape,
                                  const tactic_block_params* params, int32_t* blocks, int32_t* counts,
                                  void* workspace, size_t workspace_bytes, hipStream_t stream) {
  tactic_status st;
  tactic::QuantKV c;
  if ((st = check_shape(shape)) != TACTIC_OK || (st = quant_args(kv, shape, false, &c)) != TACTIC_OK) return st;
  if (!params) return fail(TACTIC_ERR_INVALID_ARG, "params is null");
  if (params->budget < 1 || params->first < 0 || params->last < 0 || (int64_t)params->first + params->last > params->budget)
    return fail(TACTIC_ERR_INVALID_ARG, "budget must be >= 1 and at least first + last");
  if (params->budget > kMaxBudget) return fail(TACTIC_ERR_UNSUPPORTED, "budget > 2^27 blocks");
  if (!q || !blocks || !counts || !c.bounds) return fail(TACTIC_ERR_INVALID_ARG, "null argument");
  if ((st = check_aligned({q, workspace}, 16)) != TACTIC_OK || (st = check_aligned({blocks, counts}, 4)) != TACTIC_OK) return st;
  const SelectLayout l = select_layout(shape, c.block);
  if (!workspace || (int64_t)workspace_bytes < l.bytes)
    return fail(TACTIC_ERR_WORKSPACE, "workspace has %zu bytes, needs %lld", workspace_bytes, (long long)l.bytes);
  char* ws = static_cast<char*>(workspace);
  tactic::SelectArgs a{};
  a.q = q;
  a.bounds = c.bounds;
  a.kv_indptr = shape->kv_indptr;
  a.seq_len = shape->seq_len;
  a.B = shape->batch;
  a.Hq = shape->n_q_heads;
  a.Hkv = shape->n_kv_heads;
  a.G = a.Hq / a.Hkv;
  a.block = c.block;
  a.budget = params->budget;
  a.first = params->first;
  a.last = params->last;
  a.total = shape->total_tokens;
  a.max_blocks = l.max_blocks;
  a.per = (int)l.per;
  a.tops = l.tops;
  a.scores = reinterpret_cast<double*>(ws + l.scores);
  a.top = reinterpret_cast<double*>(ws + l.top);
  a.keys = reinterpret_cast<double*>(ws + l.keys);
  a.blocks = blocks;
  a.counts = counts;
  hipError_t e = hipSuccess;
  if (l.max_blocks > a.budget && !tactic::blocks_scored_by_select(a)) e = tactic::launch_block_scores(a, stream);  // (else every block is chosen)
  if (e == hipSuccess) e = tactic::launch_block_select(a, stream);
  return e == hipSuccess ? TACTIC_OK : hip_fail(e, "block selection launch");
}

tactic_status tactic_quant_decode(const uint16_t* q, const tactic_quant_kv* kv, const tactic_kv_shape* shape,
                                  const tactic_score_mod* mod, const int32_t* blocks, const int32_t* counts,
                                  int32_t budget, float* out, float* lse, void* workspace,
                                  size_t workspace_bytes, hipStream_t stream) {
  tactic_status st;
  tactic::QuantAttnArgs x{};
  if ((st = check_shape(shape)) != TACTIC_OK || (st = quant_args(kv, shape, true, &x.kv)) != TACTIC_OK || (st = check_mod(mod)) != TACTIC_OK)
    return st;
  if (mod && (mod->documents || mod->prefix_len)) return fail(TACTIC_ERR_UNSUPPORTED, "a quantised cache takes a cap and slopes only");
  if (!q || !out) return fail(TACTIC_ERR_INVALID_ARG, "null argument");
  if (!blocks != !counts) return fail(TACTIC_ERR_INVALID_ARG, "blocks and counts go together");
  if (blocks && (!is_block(x.kv.block) || budget < 1)) return fail(TACTIC_ERR_INVALID_ARG, "blocks need a block size and a budget >= 1");
  if ((st = check_aligned({q, out, workspace}, 16)) != TACTIC_OK || (st = check_aligned({blocks, counts, lse}, 4)) != TACTIC_OK) return st;
  const int64_t need = (int64_t)dense_workspace_bytes(shape, tactic::kMaxAttnGrid);
  if (!workspace || (int64_t)workspace_bytes < need)
    return fail(TACTIC_ERR_WORKSPACE, "workspace has %zu bytes, needs %lld", workspace_bytes, (long long)need);
  char* ws = static_cast<char*>(workspace);
  const int G = shape->n_q_heads / shape->n_kv_heads;
  const int64_t groups = (int64_t)shape->batch * shape->n_kv_heads;
  x.a.q = q;
  x.a.kv_indptr = shape->kv_indptr;
  x.a.seq_len = shape->seq_len;
  x.a.B = shape->batch;
  x.a.Hq = shape->n_q_heads;
  x.a.Hkv = shape->n_kv_heads;
  x.a.dense = 1;
  x.a.NV = shape->n_kv_heads;
  x.a.kv_div = 1;
  x.a.total = shape->total_tokens;
  Layout L;  // as in dense_workspace_bytes
  x.a.partials = reinterpret_cast<float*>(ws + L.take((groups + tactic::kMaxAttnGrid) * G * (kHeadDim + 2) * 4));
  x.a.ameta = reinterpret_cast<int64_t*>(ws + L.take((groups + 2) * 8));
  x.a.out = out;
  x.blocks = blocks;
  x.counts = counts;
  x.budget = budget;
  x.block = x.kv.block;
  if (mod) {
    x.cap = mod->cap;
    x.slopes = mod->slopes;
  }
  tactic::JoinArgs j{};
  j.lse = lse;
  j.rows = (int64_t)shape->batch * shape->n_q_heads;
  const int64_t most = blocks ? std::min<int64_t>(shape->max_seq_len, (int64_t)budget * x.block) : shape->max_seq_len;
  x.direct = one_workgroup(shape, x.kv.bits, most);
  x.lse = lse;
  hipError_t e = hipSuccess;
  if (x.direct) {
    e = tactic::launch_quant_attn(x, G, (int)groups, stream);
  } else {
    int grid = 0;
    e = tactic::quant_resident_grid(x, G, &grid);
    grid = std::min(grid, tactic::kMaxAttnGrid);
    x.per_grid = 1.0 / std::max(grid, 1);
    if (e == hipSuccess) e = tactic::launch_quant_attn(x, G, grid, stream);
    if (e == hipSuccess) e = tactic::launch_join(x.a, j, G, stream);
  }
  return e == hipSuccess ? TACTIC_OK : hip_fail(e, "quantised decode launch");
}

}  // extern "C"
