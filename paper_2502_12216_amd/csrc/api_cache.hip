// Host side of the calls beside the sparse decode: prompt attention, scored and
// shared-prefix decode, accumulated weights, eviction and insertion.
#include <hip/hip_runtime.h>
#include <math.h>
#include <string.h>

#include <algorithm>
#include <initializer_list>

#include "host.hpp"
#include "plan.hpp"

using namespace tactic_host;
using tactic::kHeadDim;
using tactic::kMaxSplits;

namespace {

constexpr int64_t kMaxInt = ((int64_t)1 << 31) - 1;
constexpr int kMaxRecent = 1 << 22;

// The kernels read and write rows 16 bytes at a time.
tactic_status check_rows(std::initializer_list<const void*> arrays) {
  for (const void* p : arrays)
    if (reinterpret_cast<uintptr_t>(p) % 16) return fail(TACTIC_ERR_INVALID_ARG, "q, k, v, caches, outputs and workspace must be 16-byte aligned");
  return TACTIC_OK;
}

tactic_status check_queries(const tactic_query_shape* q, const tactic_kv_shape* s) {
  if (!q) return fail(TACTIC_ERR_INVALID_ARG, "queries is null");
  if (!q->q_indptr) return fail(TACTIC_ERR_INVALID_ARG, "q_indptr is null");
  if (q->total_queries < 0 || q->max_queries < 0 || q->max_queries > q->total_queries)
    return fail(TACTIC_ERR_INVALID_ARG, "inconsistent total_queries / max_queries");
  if (q->total_queries > (int64_t)q->max_queries * s->batch)
    return fail(TACTIC_ERR_INVALID_ARG, "total_queries > batch * max_queries");
  if (q->total_queries * s->n_q_heads > kMaxInt)
    return fail(TACTIC_ERR_UNSUPPORTED, "total_queries * n_q_heads >= 2^31");
  return TACTIC_OK;
}

// Row tiles, their size and the splits of their keys for sources whose rows are at
// most max_rows each and total_rows together.
struct RowsPlan {
  int variant, splits;
  int64_t tiles;  // row tiles of one KV head, at most
};

// The row tile and the splits with the least estimated time.  A workgroup takes
// `item` us and `step` us for each round of its waves' tiles (`keys` keys); a compute
// unit runs one at a time (two of the smallest, at half the pace); the keys come once
// from memory, half of the shorter of the two hidden behind the longer.  Splits are
// joined by a second kernel: 4 us, and their sums written and read.  Every sequence counts as
// the longest, and documents as all seen.  Measured with 32 /
// 8 and 8 / 2 heads (us a call, tiles of 32, 64, 128, 256 rows with the best splits of
// each): prompts of 211 tokens 11, 12, 14, 15; 1000 tokens, 2 KV heads 16, 21, 24, 24;
// 2048 tokens 74, 85, 56, 65; 4096 tokens 245, 263, 180, 151; one token on 32768 34,
// 36, 38, 46; 20 on 131072 160, 131, 112, 157; 512 on 32768 444, 397, 308, 279.  Shared
// prefixes of 32768 tokens: 4 sequences 42, 44, 53, 75; 12 50, 45, 56, 77; 64 113, 104,
// 101, 101.  The choice is within a tenth of the best in all of these.
struct RowsCost {
  double item, step;
  int keys;
};
constexpr RowsCost kPromptCost[4] = {{1.3, 0.88, 128}, {2.0, 1.9, 128}, {2.5, 2.3, 128}, {2.0, 1.85, 64}};
constexpr RowsCost kSharedCost[4] = {{1.3, 1.05, 128}, {2.0, 1.9, 128}, {2.5, 1.7, 64}, {2.0, 1.8, 32}};

RowsPlan plan_rows(int64_t total_rows, int n_src, int Hkv, double mean_keys, int64_t max_keys, int64_t total_keys,
                   bool shared) {
  constexpr int kTry[] = {1, 2, 3, 4, 5, 6, 7, 8, 10, 12, 14, 16, 20, 24, 28, 32, 40, 48, 56, 64};
  static_assert(kMaxSplits == 64, "the splits tried");
  const double mem = (double)total_keys * Hkv * 512 / 6e6;  // 6 TB/s
  double best = INFINITY;
  RowsPlan p{3, 1, 0};
  for (int v = 0; v < 4; ++v) {
    const RowsCost& c = (shared ? kSharedCost : kPromptCost)[v];
    const int64_t per = tactic::rows_per_item(v);
    const double items = (double)std::max<int64_t>(n_src, (total_rows + per - 1) / per) * Hkv;
    for (const int s : kTry) {
      if (s > 1 && (int64_t)s * c.keys > max_keys) break;
      const double longest = ceil((double)max_keys / ((double)s * c.keys)), mean = mean_keys / ((double)s * c.keys);
      const double rounds = ceil(items * s / 256);
      const double run = std::max(longest * c.step + c.item, rounds * (mean * c.step + c.item));
      double t = std::max(run, mem) + 0.5 * std::min(run, mem);
      if (shared) t += 0.1 * s;
      else if (s > 1) t += 4 + 0.15 * s + (double)total_rows * Hkv * s * (2 * 520) / 4.5e6;
      if (t < best) {
        best = t;
        p.variant = v;
        p.splits = s;
      }
    }
  }
  p.tiles = total_rows / tactic::rows_per_item(p.variant) + n_src;
  return p;
}

struct PromptLayout {
  RowsPlan plan;
  int64_t part_o, part_ml, ranges, range_stride, items, counts, order, bytes;
  int wsplits;  // splits of tactic_prompt_weights
  int64_t wpart;
};

// Splits of the query rows of tactic_prompt_weights, of which a sequence has at most
// `rows` for a KV head.  Key tiles have 256 rows: the queries are split until there are
// eight workgroups for each of the 512 places (an early key is seen by more queries than
// a late one, so that they are of many lengths), of at least eight tiles of 64 rows each;
// or of two such tiles until there is one for each place.
int weight_splits(const tactic_kv_shape* s, int64_t rows) {
  const int64_t items = std::max<int64_t>(1, (s->total_tokens + 255) / 256) * s->n_kv_heads;
  const int64_t many = std::min<int64_t>(4096 / items, rows / 512), few = std::min<int64_t>(512 / items, rows / 128);
  return (int)std::max<int64_t>(1, std::min<int64_t>(std::max(many, few), kMaxSplits));
}

PromptLayout prompt_layout(const tactic_kv_shape* s, const tactic_query_shape* q) {
  PromptLayout p;
  const int G = s->n_q_heads / s->n_kv_heads;
  // a query sees its own position's keys: on average half its prompt's fewer than all
  const double mean = std::max(1.0, (double)s->max_seq_len - 0.5 * (double)std::min(q->max_queries, s->max_seq_len));
  p.plan = plan_rows(q->total_queries * G, s->batch, s->n_kv_heads, mean, s->max_seq_len, s->total_tokens, false);
  const int64_t rows = q->total_queries * s->n_q_heads;
  p.range_stride = (s->max_seq_len + 63) / 64;
  Layout L;
  p.ranges = L.take(p.range_stride * s->batch * 8);
  const int64_t behind = L.cur;
  p.part_o = p.plan.splits > 1 ? L.take(rows * p.plan.splits * kHeadDim * 4) : 0;
  p.part_ml = p.plan.splits > 1 ? L.take(rows * p.plan.splits * 8) : 0;
  p.items = L.take(p.plan.tiles * 16);
  p.counts = L.take(p.plan.tiles * 4);
  p.order = L.take(p.plan.tiles * 16);
  Layout W;
  W.cur = behind;
  p.wsplits = weight_splits(s, q->max_queries * G);
  p.wpart = p.wsplits > 1 ? W.take((int64_t)p.wsplits * s->n_kv_heads * s->total_tokens * 4) : 0;
  p.bytes = std::max<int64_t>(256, std::max(L.cur, W.cur));
  return p;
}

tactic_status check_workspace(const void* ws, size_t have, int64_t need) {
  if (!ws || (int64_t)have < need)
    return fail(TACTIC_ERR_WORKSPACE, "workspace has %zu bytes, needs %lld", have, (long long)need);
  return TACTIC_OK;
}

tactic_status prompt_impl(const uint16_t* q, const uint16_t* K, const uint16_t* V, const tactic::PagedKV* pk,
                          const tactic_kv_shape* shape, const tactic_query_shape* queries,
                          const tactic_score_mod* mod, uint16_t* out, float* lse, void* workspace,
                          size_t workspace_bytes, hipStream_t stream) {
  tactic_status st;
  if ((st = check_mod(mod)) != TACTIC_OK || (st = check_queries(queries, shape)) != TACTIC_OK) return st;
  if (queries->total_queries == 0) return TACTIC_OK;
  if (!q || !out || ((!K || !V) && shape->total_tokens > 0)) return fail(TACTIC_ERR_INVALID_ARG, "null argument");
  if ((st = check_rows({q, K, V, out, workspace})) != TACTIC_OK) return st;
  const PromptLayout p = prompt_layout(shape, queries);
  if ((st = check_workspace(workspace, workspace_bytes, p.bytes)) != TACTIC_OK) return st;
  if (p.plan.tiles * shape->n_kv_heads * p.plan.splits > kMaxInt) return fail(TACTIC_ERR_UNSUPPORTED, "more than 2^31 workgroups");
  char* ws = static_cast<char*>(workspace);
  tactic::RowsArgs a{};
  a.q = q;
  a.K = K;
  a.V = V;
  a.kv_indptr = shape->kv_indptr;
  a.seq_len = shape->seq_len;
  a.mode = 0;
  a.n_src = shape->batch;
  a.Hq = shape->n_q_heads;
  a.Hkv = shape->n_kv_heads;
  a.G = a.Hq / a.Hkv;
  a.splits = p.plan.splits;
  a.direct = p.plan.splits == 1;
  a.total = shape->total_tokens;
  a.n_queries = queries->total_queries;
  a.q_indptr = queries->q_indptr;
  if (mod) {
    a.cap = mod->cap;
    a.poly = tactic::cap_poly(mod->cap);
    a.slopes = mod->slopes;
    a.documents = mod->documents;
    a.prefix_len = mod->prefix_len;
  }
  a.doc_range = reinterpret_cast<const int2*>(ws + p.ranges);
  a.range_stride = p.range_stride;
  if (pk) {
    a.paged = 1;
    a.pk = *pk;
  }
  a.part_o = reinterpret_cast<float*>(ws + p.part_o);
  a.part_ml = reinterpret_cast<float*>(ws + p.part_ml);
  a.out = out;
  a.lse = lse;
  hipError_t e = hipSuccess;
  if (a.documents)
    e = tactic::launch_doc_range(a.documents, a.kv_indptr, a.seq_len, a.n_src, p.range_stride, reinterpret_cast<int2*>(ws + p.ranges), stream);
  // Documents give row tiles of any length in any order.  Where the form that skips what
  // they leave out (256 rows to an item, keys not split) has more than one and a half
  // items for each compute unit, and sequences of more than four key tiles, the long ones
  // are started first: two small kernels, 14 us, part of them beside the attention.
  // Without and with, us a call, cap, 32 heads on 8: 16000 + 8192 + 5001 tokens, documents of 1100 on
  // average 840, 808; of 300 484, 444; 3 x 2500 (of 500) 147, 121; 5000 (of 500) 114, 97;
  // 4096 (of 300) 85, 84; 3 x 1200 (of 300) 72, 57; 6 x 800 (of 200) 67, 69; 8 x 800 (of 100) 87, 79;
  // 30 x 250 84, 90; 20 x 120 36, 40; one item a unit: 2000 on 12000 79, 86.  The other forms go
  // through every tile and lose by it: 12000 tokens in three, 8 heads on 2, 234, 287; 8192 267, 416.
  const bool in_order = a.documents && p.plan.variant == 3 && a.splits == 1 && p.plan.tiles * a.Hkv > 384 && shape->max_seq_len > 256;
  if (e == hipSuccess && in_order) {
    int4* order = reinterpret_cast<int4*>(ws + p.order);
    e = tactic::launch_item_order(a, (int)p.plan.tiles, reinterpret_cast<int4*>(ws + p.items),
                                  reinterpret_cast<int32_t*>(ws + p.counts), order, stream);
    a.order = order;
  }
  if (e == hipSuccess) e = tactic::launch_rows_attn(a, p.plan.variant, false, p.plan.tiles * a.Hkv * a.splits, stream);
  if (e == hipSuccess && !a.direct) e = tactic::launch_rows_combine(a, stream);
  if (e != hipSuccess) return hip_fail(e, "prompt attention launch");
  return TACTIC_OK;
}

// Fills the arguments of a single-token launch over `shape` with a dense workspace.
void token_args(tactic::AttnArgs* aa, const uint16_t* q, const uint16_t* K, const uint16_t* V,
                const tactic::PagedKV* pk, const tactic_kv_shape* shape, float* out, char* ws) {
  memset(aa, 0, sizeof(*aa));
  const int64_t BG = (int64_t)shape->batch * shape->n_kv_heads;
  const int G = shape->n_q_heads / shape->n_kv_heads;
  aa->q = q;
  aa->K = K;
  aa->V = V;
  aa->kv_indptr = shape->kv_indptr;
  aa->seq_len = shape->seq_len;
  aa->B = shape->batch;
  aa->Hq = shape->n_q_heads;
  aa->Hkv = shape->n_kv_heads;
  aa->dense = 1;
  aa->NV = shape->n_kv_heads;
  aa->kv_div = 1;
  aa->total = shape->total_tokens;
  Layout L;  // as in dense_workspace_bytes
  aa->partials = reinterpret_cast<float*>(ws + L.take((BG + tactic::kMaxAttnGrid) * G * (kHeadDim + 2) * 4));
  aa->ameta = reinterpret_cast<int64_t*>(ws + L.take((BG + 2) * 8));
  if (pk) {
    aa->pk = *pk;
    aa->pk.perm = nullptr;
  }
  aa->out = out;
}

hipError_t launch_tokens(tactic::AttnArgs& aa, const tactic::TokenMod& m, bool paged, hipStream_t stream) {
  const int G = aa.Hq / aa.Hkv;
  int resident = 0, cus = 1;
  const hipError_t e = tactic::attn_resident_grid(G, aa.B * aa.Hkv, paged, &resident, &cus, m.positions || m.documents ? 2 : 1);
  if (e != hipSuccess) return e;
  aa.cus = cus;
  return tactic::launch_attn_mod(aa, m, G, std::min(resident, tactic::kMaxAttnGrid), paged, stream);
}

struct ScoredLayout {
  int64_t scores, bytes;
};
ScoredLayout scored_layout(const tactic_kv_shape* s, bool weights) {
  ScoredLayout p;
  Layout L;
  L.take((int64_t)dense_workspace_bytes(s, tactic::kMaxAttnGrid));
  p.scores = weights ? L.take(s->total_tokens * s->n_q_heads * 4) : 0;
  p.bytes = L.cur;
  return p;
}

tactic_status scored_impl(const uint16_t* q, const uint16_t* K, const uint16_t* V, const tactic::PagedKV* pk,
                          const tactic_kv_shape* shape, const tactic_score_mod* mod, const tactic_token_rows* rows,
                          float* out, float* lse, float* weights, void* workspace, size_t workspace_bytes,
                          hipStream_t stream) {
  tactic_status st;
  if ((st = check_mod(mod)) != TACTIC_OK) return st;
  if (!q || !out || ((!K || !V) && shape->total_tokens > 0)) return fail(TACTIC_ERR_INVALID_ARG, "null argument");
  if (mod && mod->prefix_len) return fail(TACTIC_ERR_INVALID_ARG, "prefix_len is for prompts");
  const bool docs = mod && mod->documents;
  if (docs != (rows && rows->q_documents)) return fail(TACTIC_ERR_INVALID_ARG, "documents and q_documents go together");
  if (mod && mod->slopes && rows && rows->positions && !rows->q_pos)
    return fail(TACTIC_ERR_INVALID_ARG, "slopes with positions need q_pos");
  if ((st = check_rows({q, K, V, out, workspace})) != TACTIC_OK) return st;
  const ScoredLayout p = scored_layout(shape, weights != nullptr);
  if ((st = check_workspace(workspace, workspace_bytes, p.bytes)) != TACTIC_OK) return st;
  char* ws = static_cast<char*>(workspace);
  tactic::AttnArgs aa;
  token_args(&aa, q, K, V, pk, shape, out, ws);
  tactic::TokenMod m{};
  if (mod) {
    m.cap = mod->cap;
    m.slopes = mod->slopes;
    m.documents = mod->documents;
  }
  if (rows) {
    m.positions = m.slopes ? rows->positions : nullptr;  // (only a bias by distance reads them)
    m.q_pos = rows->q_pos;
    m.q_documents = rows->q_documents;
  }
  m.scores = weights ? reinterpret_cast<float*>(ws + p.scores) : nullptr;
  tactic::JoinArgs j{};
  j.lse = lse;
  if (weights && shape->max_seq_len > 0) {
    j.scores = m.scores;
    j.weights = weights;
    j.chunks = (int)std::min<int64_t>((shape->max_seq_len + 2047) / 2048, 4096);
  }
  j.rows = (int64_t)shape->batch * shape->n_q_heads;
  const int G = aa.Hq / aa.Hkv;
  hipError_t e = launch_tokens(aa, m, pk != nullptr, stream);
  if (e == hipSuccess) e = tactic::launch_join(aa, j, G, stream);
  if (e != hipSuccess) return hip_fail(e, "scored decode launch");
  return TACTIC_OK;
}

tactic_status check_prefixes(const tactic_prefixes* p, const tactic_kv_shape* s) {
  if (!p) return fail(TACTIC_ERR_INVALID_ARG, "prefixes is null");
  if (p->n_prefixes < 1 || p->max_members < 0 || p->total_members < p->max_members || p->total_members > s->batch)
    return fail(TACTIC_ERR_INVALID_ARG, "inconsistent prefix counts");
  if (p->total_tokens < 0 || p->max_len < 0 || p->max_len > p->total_tokens)
    return fail(TACTIC_ERR_INVALID_ARG, "inconsistent prefix lengths");
  if (p->max_len + s->max_seq_len > kMaxInt) return fail(TACTIC_ERR_UNSUPPORTED, "prefix and sequence >= 2^31 tokens");
  if (!p->prefix_indptr || !p->prefix_of || !p->member_indptr || (!p->members && p->total_members > 0))
    return fail(TACTIC_ERR_INVALID_ARG, "null prefix pointer");
  return TACTIC_OK;
}

struct SharedLayout {
  RowsPlan plan;
  int64_t part_o, part_ml, bytes;
};
SharedLayout shared_layout(const tactic_kv_shape* s, const tactic_prefixes* p) {
  SharedLayout l;
  const int G = s->n_q_heads / s->n_kv_heads;
  l.plan = plan_rows((int64_t)p->total_members * G, p->n_prefixes, s->n_kv_heads, (double)p->max_len, p->max_len,
                     p->total_tokens, true);
  const int64_t rows = (int64_t)s->batch * s->n_q_heads;
  Layout L;
  L.take((int64_t)dense_workspace_bytes(s, tactic::kMaxAttnGrid));
  l.part_o = L.take(rows * l.plan.splits * kHeadDim * 4);
  l.part_ml = L.take(rows * l.plan.splits * 8);
  l.bytes = L.cur;
  return l;
}

// Sequences' rows are ranked by one workgroup for each KV head, or by 16 in four launches,
// which add up each other's counts: that pays where the one works long and few units are
// busy otherwise.  One against 16, us a call, 8 KV heads, an eighth kept, weights by a power law
// (three values): 24000 rows 29 (40) and 29 (31); 4 x 24000 40 (52) and 50 (53); 65536 + 30011
// 72 (99) and 63 (66); 4 x 65536 84 (114) and 89 (93); past 65536 rows the one makes
// its keys again in every pass: 131072 122 and 42; 4 x 131072 232 and 162; 8 x 348 and 315.
bool evict_sliced(int64_t max_len, int64_t groups) { return groups <= (max_len > 65536 ? 64 : 16) && max_len > 16384; }

struct EvictLayout {
  bool sliced;
  int64_t counts, chosen, ahead, bytes;
};
EvictLayout evict_layout(const tactic_kv_shape* s, int64_t out_total) {
  EvictLayout l{};
  const int64_t groups = (int64_t)s->batch * s->n_kv_heads;
  l.sliced = evict_sliced(s->max_seq_len, groups);
  Layout L;
  L.take(out_total * s->n_kv_heads * 4);
  if (l.sliced) {
    l.counts = L.take(3 * groups * tactic::kEvictSlices * tactic::kEvictBins * 4);
    l.chosen = L.take(2 * groups * 8);
    l.ahead = L.take(2 * groups * tactic::kEvictSlices * 4);
  }
  l.bytes = std::max<int64_t>(256, L.cur);
  return l;
}

tactic_status shared_impl(const uint16_t* q, const uint16_t* Kp, const uint16_t* Vp, const tactic::PagedKV* pkp,
                          const uint16_t* K, const uint16_t* V, const tactic::PagedKV* pk,
                          const tactic_kv_shape* shape, const tactic_prefixes* pre, const tactic_score_mod* mod,
                          float* out, float* lse, void* workspace, size_t workspace_bytes, hipStream_t stream) {
  tactic_status st;
  if ((st = check_mod(mod)) != TACTIC_OK) return st;
  if (mod && (mod->documents || mod->prefix_len))
    return fail(TACTIC_ERR_UNSUPPORTED, "a shared prefix takes a cap and slopes only");
  if (!q || !out || ((!K || !V) && shape->total_tokens > 0) || ((!Kp || !Vp) && pre->total_tokens > 0))
    return fail(TACTIC_ERR_INVALID_ARG, "null argument");
  if ((st = check_rows({q, Kp, Vp, K, V, out, workspace})) != TACTIC_OK) return st;
  const SharedLayout l = shared_layout(shape, pre);
  if ((st = check_workspace(workspace, workspace_bytes, l.bytes)) != TACTIC_OK) return st;
  if (l.plan.tiles * shape->n_kv_heads * l.plan.splits > kMaxInt) return fail(TACTIC_ERR_UNSUPPORTED, "more than 2^31 workgroups");
  char* ws = static_cast<char*>(workspace);
  tactic::RowsArgs a{};
  a.q = q;
  a.K = Kp;
  a.V = Vp;
  a.kv_indptr = pre->prefix_indptr;
  a.mode = 1;
  a.n_src = pre->n_prefixes;
  a.Hq = shape->n_q_heads;
  a.Hkv = shape->n_kv_heads;
  a.G = a.Hq / a.Hkv;
  a.splits = l.plan.splits;
  a.total = pre->total_tokens;
  a.n_queries = shape->batch;
  a.members = pre->members;
  a.member_indptr = pre->member_indptr;
  a.own_indptr = shape->kv_indptr;
  a.own_len = shape->seq_len;
  if (mod) {
    a.cap = mod->cap;
    a.poly = tactic::cap_poly(mod->cap);
    a.slopes = mod->slopes;
  }
  if (pkp) {
    a.paged = 1;
    a.pk = *pkp;
  }
  a.part_o = reinterpret_cast<float*>(ws + l.part_o);
  a.part_ml = reinterpret_cast<float*>(ws + l.part_ml);
  tactic::AttnArgs aa;
  token_args(&aa, q, K, V, pk, shape, out, ws);
  tactic::TokenMod m{};
  m.cap = a.cap;
  m.slopes = a.slopes;
  m.pos_base = pre->prefix_indptr;
  m.base_of = pre->prefix_of;
  tactic::JoinArgs j{};
  j.lse = lse;
  j.pre_o = a.part_o;
  j.pre_ml = a.part_ml;
  j.prefix_of = pre->prefix_of;
  j.pre_splits = l.plan.splits;
  j.rows = (int64_t)shape->batch * shape->n_q_heads;
  hipError_t e = hipSuccess;
  if (pre->total_members > 0)
    e = tactic::launch_rows_attn(a, l.plan.variant, true, l.plan.tiles * a.Hkv * a.splits, stream);
  if (e == hipSuccess) e = launch_tokens(aa, m, pk != nullptr, stream);
  if (e == hipSuccess) e = tactic::launch_join(aa, j, a.G, stream);
  if (e != hipSuccess) return hip_fail(e, "shared decode launch");
  return TACTIC_OK;
}

}  // namespace

tactic_status tactic_host::check_mod(const tactic_score_mod* m) {
  // (outside, the cap's reciprocal or its value in base 2 would leave the normal numbers)
  if (m && m->cap != 0.f && !(m->cap >= 0x1p-120f && m->cap <= 0x1p120f))
    return fail(TACTIC_ERR_INVALID_ARG, "cap must be 0 or in [2^-120, 2^120]");
  return TACTIC_OK;
}

extern "C" {

size_t tactic_prompt_attention_workspace_size(const tactic_kv_shape* shape, const tactic_query_shape* queries) {
  if (check_shape(shape) != TACTIC_OK || check_queries(queries, shape) != TACTIC_OK) return 0;
  return (size_t)prompt_layout(shape, queries).bytes;
}

tactic_status tactic_prompt_attention(const uint16_t* q, const uint16_t* K, const uint16_t* V,
                                      const tactic_kv_shape* shape, const tactic_query_shape* queries,
                                      const tactic_score_mod* mod, uint16_t* out, float* lse, void* workspace,
                                      size_t workspace_bytes, hipStream_t stream) {
  const tactic_status st = check_shape(shape);
  if (st != TACTIC_OK) return st;
  return prompt_impl(q, K, V, nullptr, shape, queries, mod, out, lse, workspace, workspace_bytes, stream);
}

tactic_status tactic_prompt_attention_paged(const uint16_t* q, const tactic_paged_kv* kv,
                                            const tactic_kv_shape* shape, const tactic_query_shape* queries,
                                            const tactic_score_mod* mod, uint16_t* out, float* lse,
                                            void* workspace, size_t workspace_bytes, hipStream_t stream) {
  tactic_status st = check_shape(shape);
  if (st != TACTIC_OK) return st;
  tactic::PagedKV pk;
  if ((st = paged_args(kv, shape, &pk)) != TACTIC_OK) return st;
  return prompt_impl(q, kv->K_pages, kv->V_pages, &pk, shape, queries, mod, out, lse, workspace, workspace_bytes,
                     stream);
}

tactic_status tactic_prompt_weights(const uint16_t* q, const uint16_t* K, const tactic_kv_shape* shape,
                                    const tactic_query_shape* queries, const tactic_score_mod* mod,
                                    const float* lse, int64_t window, float* weights, void* workspace,
                                    size_t workspace_bytes, hipStream_t stream) {
  tactic_status st = check_shape(shape);
  if (st != TACTIC_OK) return st;
  if ((st = check_mod(mod)) != TACTIC_OK || (st = check_queries(queries, shape)) != TACTIC_OK) return st;
  if (window < 0) return fail(TACTIC_ERR_INVALID_ARG, "window must be >= 0");
  if (queries->total_queries == 0 || shape->total_tokens == 0) return TACTIC_OK;
  if (!q || !K || !lse || !weights) return fail(TACTIC_ERR_INVALID_ARG, "null argument");
  if ((st = check_rows({q, K, workspace})) != TACTIC_OK) return st;
  const PromptLayout p = prompt_layout(shape, queries);
  if ((st = check_workspace(workspace, workspace_bytes, p.bytes)) != TACTIC_OK) return st;
  tactic::WeightArgs a{};
  a.q = q;
  a.K = K;
  a.kv_indptr = shape->kv_indptr;
  a.seq_len = shape->seq_len;
  a.q_indptr = queries->q_indptr;
  a.lse = lse;
  a.B = shape->batch;
  a.Hq = shape->n_q_heads;
  a.Hkv = shape->n_kv_heads;
  a.G = a.Hq / a.Hkv;
  a.splits = weight_splits(shape, (window > 0 ? std::min(window, (int64_t)queries->max_queries) : queries->max_queries) * a.G);
  a.total = shape->total_tokens;
  a.n_queries = queries->total_queries;
  a.window = window;
  if (mod) {
    a.cap = mod->cap;
    a.poly = tactic::cap_poly(mod->cap);
    a.slopes = mod->slopes;
    a.documents = mod->documents;
    a.prefix_len = mod->prefix_len;
  }
  char* ws = static_cast<char*>(workspace);
  a.doc_range = reinterpret_cast<const int2*>(ws + p.ranges);
  a.range_stride = p.range_stride;
  a.part = reinterpret_cast<float*>(ws + p.wpart);
  a.weights = weights;
  hipError_t e = hipSuccess;
  if (a.documents)
    e = tactic::launch_doc_range(a.documents, a.kv_indptr, a.seq_len, a.B, p.range_stride, reinterpret_cast<int2*>(ws + p.ranges), stream);
  if (e == hipSuccess) e = tactic::launch_prompt_weights(a, shape->max_seq_len, stream);
  if (e != hipSuccess) return hip_fail(e, "prompt weights launch");
  return TACTIC_OK;
}

size_t tactic_scored_decode_workspace_size(const tactic_kv_shape* shape, int32_t with_weights) {
  if (check_shape(shape) != TACTIC_OK) return 0;
  return (size_t)scored_layout(shape, with_weights != 0).bytes;
}

tactic_status tactic_scored_decode(const uint16_t* q, const uint16_t* K, const uint16_t* V,
                                   const tactic_kv_shape* shape, const tactic_score_mod* mod,
                                   const tactic_token_rows* rows, float* out, float* lse, float* weights,
                                   void* workspace, size_t workspace_bytes, hipStream_t stream) {
  const tactic_status st = check_shape(shape);
  if (st != TACTIC_OK) return st;
  return scored_impl(q, K, V, nullptr, shape, mod, rows, out, lse, weights, workspace, workspace_bytes, stream);
}

tactic_status tactic_scored_decode_paged(const uint16_t* q, const tactic_paged_kv* kv,
                                         const tactic_kv_shape* shape, const tactic_score_mod* mod,
                                         const tactic_token_rows* rows, float* out, float* lse, float* weights,
                                         void* workspace, size_t workspace_bytes, hipStream_t stream) {
  tactic_status st = check_shape(shape);
  if (st != TACTIC_OK) return st;
  tactic::PagedKV pk;
  if ((st = paged_args(kv, shape, &pk)) != TACTIC_OK) return st;
  return scored_impl(q, kv->K_pages, kv->V_pages, &pk, shape, mod, rows, out, lse, weights, workspace,
                     workspace_bytes, stream);
}

size_t tactic_shared_decode_workspace_size(const tactic_kv_shape* shape, const tactic_prefixes* prefixes) {
  if (check_shape(shape) != TACTIC_OK || check_prefixes(prefixes, shape) != TACTIC_OK) return 0;
  return (size_t)shared_layout(shape, prefixes).bytes;
}

tactic_status tactic_shared_decode(const uint16_t* q, const uint16_t* K_prefix, const uint16_t* V_prefix,
                                   const uint16_t* K, const uint16_t* V, const tactic_kv_shape* shape,
                                   const tactic_prefixes* prefixes, const tactic_score_mod* mod, float* out,
                                   float* lse, void* workspace, size_t workspace_bytes, hipStream_t stream) {
  tactic_status st = check_shape(shape);
  if (st != TACTIC_OK || (st = check_prefixes(prefixes, shape)) != TACTIC_OK) return st;
  return shared_impl(q, K_prefix, V_prefix, nullptr, K, V, nullptr, shape, prefixes, mod, out, lse, workspace,
                     workspace_bytes, stream);
}

tactic_status tactic_shared_decode_paged(const uint16_t* q, const tactic_paged_kv* kv_prefix,
                                         const tactic_paged_kv* kv, const tactic_kv_shape* shape,
                                         const tactic_prefixes* prefixes, const tactic_score_mod* mod, float* out,
                                         float* lse, void* workspace, size_t workspace_bytes, hipStream_t stream) {
  tactic_status st = check_shape(shape);
  if (st != TACTIC_OK || (st = check_prefixes(prefixes, shape)) != TACTIC_OK) return st;
  tactic::PagedKV pk, pkp;
  if ((st = paged_args(kv, shape, &pk)) != TACTIC_OK) return st;
  tactic_kv_shape ps = *shape;  // what paged_args compares the prefixes' pages with
  ps.max_seq_len = prefixes->max_len;
  if ((st = paged_args(kv_prefix, &ps, &pkp)) != TACTIC_OK) return st;
  return shared_impl(q, kv_prefix->K_pages, kv_prefix->V_pages, &pkp, kv->K_pages, kv->V_pages, &pk, shape, prefixes,
                     mod, out, lse, workspace, workspace_bytes, stream);
}

size_t tactic_evict_workspace_size(const tactic_kv_shape* shape, int64_t out_total) {
  if (check_shape(shape) != TACTIC_OK || out_total < 0) return 0;
  return (size_t)evict_layout(shape, out_total).bytes;
}

tactic_status tactic_evict(const uint16_t* K, const uint16_t* V, const tactic_kv_shape* shape, const float* weights,
                           const int32_t* positions, const int32_t* keep, const int32_t* newest, int32_t recent,
                           const int64_t* out_indptr, int64_t out_total, int64_t out_max, uint16_t* K_out,
                           uint16_t* V_out, float* weights_out, int32_t* positions_out, int64_t* out_len,
                           void* workspace, size_t workspace_bytes, hipStream_t stream) {
  tactic_status st = check_shape(shape);
  if (st != TACTIC_OK) return st;
  if (!keep || !out_indptr || !out_len) return fail(TACTIC_ERR_INVALID_ARG, "null argument");
  if ((!K || !V || !weights) && shape->total_tokens > 0) return fail(TACTIC_ERR_INVALID_ARG, "null argument");
  if ((!K_out || !V_out || !weights_out || !positions_out) && out_total > 0)
    return fail(TACTIC_ERR_INVALID_ARG, "null argument");
  if ((st = check_rows({K, V, K_out, V_out, workspace})) != TACTIC_OK) return st;
  if (out_len == shape->seq_len) return fail(TACTIC_ERR_INVALID_ARG, "out_len must not be the shape's seq_len");
  if (recent < 0 || recent > kMaxRecent) return fail(TACTIC_ERR_INVALID_ARG, "recent must be in [0, 2^22]");
  if (out_total < 0 || out_max < 0 || out_max > out_total)
    return fail(TACTIC_ERR_INVALID_ARG, "inconsistent out_total / out_max");
  if (out_max > kMaxInt) return fail(TACTIC_ERR_UNSUPPORTED, "a span >= 2^31");
  if ((st = check_workspace(workspace, workspace_bytes, (int64_t)tactic_evict_workspace_size(shape, out_total))) != TACTIC_OK)
    return st;
  // workgroups write rows while others read theirs: no output may lie in an input or in another output
  const int64_t rows_in = shape->total_tokens * shape->n_kv_heads, rows_out = out_total * shape->n_kv_heads;
  const Span in[] = {{K, rows_in * kHeadDim * 2}, {V, rows_in * kHeadDim * 2}, {weights, rows_in * 4}, {positions, rows_in * 4}};
  const Span outs[] = {{K_out, rows_out * kHeadDim * 2}, {V_out, rows_out * kHeadDim * 2}, {weights_out, rows_out * 4},
                       {positions_out, rows_out * 4}};
  for (const Span& o : outs) {
    for (const Span& i : in)
      if (overlap(o, i)) return fail(TACTIC_ERR_INVALID_ARG, "the outputs must not overlap the inputs");
    for (const Span& p : outs)
      if (&o < &p && overlap(o, p)) return fail(TACTIC_ERR_INVALID_ARG, "the outputs must not overlap one another");
  }
  tactic::EvictArgs a{};
  a.K = K;
  a.V = V;
  a.weights = weights;
  a.positions = positions;
  a.kv_indptr = shape->kv_indptr;
  a.seq_len = shape->seq_len;
  a.keep = keep;
  a.newest = newest;
  a.out_indptr = out_indptr;
  a.B = shape->batch;
  a.Hkv = shape->n_kv_heads;
  a.recent = recent;
  a.total = shape->total_tokens;
  a.out_total = out_total;
  a.K_out = K_out;
  a.V_out = V_out;
  a.weights_out = weights_out;
  a.positions_out = positions_out;
  a.out_len = out_len;
  const EvictLayout l = evict_layout(shape, out_total);
  char* ws = static_cast<char*>(workspace);
  a.rows = reinterpret_cast<int32_t*>(ws);
  if (l.sliced) {
    a.counts = reinterpret_cast<uint32_t*>(ws + l.counts);
    a.chosen = reinterpret_cast<uint2*>(ws + l.chosen);
    a.ahead = reinterpret_cast<uint32_t*>(ws + l.ahead);
  }
  const hipError_t e = tactic::launch_evict(a, shape->max_seq_len, std::min(out_max, shape->max_seq_len), stream);
  if (e != hipSuccess) return hip_fail(e, "evict launch");
  return TACTIC_OK;
}

tactic_status tactic_insert_token(const uint16_t* k, const uint16_t* v, const int32_t* newest, int32_t recent,
                                  const tactic_kv_shape* shape, int64_t* seq_len, uint16_t* K, uint16_t* V,
                                  float* weights, int32_t* positions, int32_t* rows, hipStream_t stream) {
  tactic_status st = check_shape(shape);
  if (st != TACTIC_OK) return st;
  if (!k || !v || !newest || !seq_len || !rows) return fail(TACTIC_ERR_INVALID_ARG, "null argument");
  if ((!K || !V || !weights || !positions) && shape->total_tokens > 0) return fail(TACTIC_ERR_INVALID_ARG, "null argument");
  if ((st = check_rows({k, v, K, V})) != TACTIC_OK) return st;
  if (seq_len != shape->seq_len) return fail(TACTIC_ERR_INVALID_ARG, "seq_len must be the shape's own array");
  if (recent < 0 || recent > kMaxRecent) return fail(TACTIC_ERR_INVALID_ARG, "recent must be in [0, 2^22]");
  tactic::InsertArgs a{};
  a.k = k;
  a.v = v;
  a.K = K;
  a.V = V;
  a.weights = weights;
  a.positions = positions;
  a.newest = newest;
  a.kv_indptr = shape->kv_indptr;
  a.seq_len = seq_len;
  a.B = shape->batch;
  a.Hkv = shape->n_kv_heads;
  a.recent = recent;
  a.total = shape->total_tokens;
  a.rows = rows;
  const hipError_t e = tactic::launch_insert(a, shape->max_seq_len, stream);
  if (e != hipSuccess) return hip_fail(e, "insert launch");
  return TACTIC_OK;
}

}  // extern "C"
