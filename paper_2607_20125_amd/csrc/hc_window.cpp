// Entry points of the operators of a model with a sliding window: norm with rotary positions, the cache in
// pages with its attention, attention over packed sequences with a window, and the gradients.
#include "hc_window.h"

#include "hc_args.h"

using namespace hc;

namespace {

// --- norm and rotary positions ---------------------------------------------------------------
hc_status check_norm(hc_ctx *c, const hc_norm_args *p, const void *tensors, int n_tensors, NormArgs &a) {
  if (!p || !tensors) return fail(c, HC_E_INVAL, "args or tensors is NULL");
  if (n_tensors != 1 && n_tensors != 2) return fail(c, HC_E_INVAL, "n_tensors must be 1 or 2");
  const hc_rotate_args &r = p->rotate;
  if (r.n_tokens < 0) return fail(c, HC_E_INVAL, "n_tokens must not be negative");
  if (p->weight_type != HC_BF16 && p->weight_type != HC_F32)
    return fail(c, HC_E_INVAL, "weight_type must be HC_BF16 or HC_F32");
  if (!(p->eps >= 0.f) || !std::isfinite(p->eps)) return fail(c, HC_E_INVAL, "eps must be finite and not negative");
  a = NormArgs{};
  const hc_status st = check_rotation(c, &r, true, a.rotate);
  if (st != HC_OK) return st;
  a.rotate.n_tokens = r.n_tokens;
  a.rotate.head_dim = r.head_dim;
  a.n_tensors = n_tensors;
  a.weight_type = p->weight_type;
  a.eps = p->eps;
  return HC_OK;
}

hc_status check_norm_size(hc_ctx *c, const NormArgs &a) {
  int64_t heads = 0;
  for (int i = 0; i < a.n_tensors; ++i) {
    if (a.t[i].n_heads < 1) return fail(c, HC_E_INVAL, "tensor %d: n_heads must be at least 1", i);
    heads += a.t[i].n_heads;
  }
  if (heads > 65535 || !good_grid((int64_t)a.rotate.n_tokens * (kRotMaxDim / 8) / kNormThreads + 1))
    return fail(c, HC_E_INVAL, "too many heads or tokens for one call");
  return HC_OK;
}

void plan_norm(NormArgs &a, bool halves, bool backward) {
  const int items = norm_items(a.rotate, halves);
  a.lane_bits = 0;
  while ((1 << a.lane_bits) < items) ++a.lane_bits;
  const int64_t per_group = kNormThreads >> a.lane_bits;
  const int64_t blocks = (a.rotate.n_tokens + per_group - 1) / per_group;
  // heads per thread: as many as leave 2048 work groups (8 for each CU), so that angles are
  // shared where there is work enough and few tokens still fill the card
  int64_t cuts = 0;
  for (int i = 0; i < a.n_tensors; ++i) {
    NormTensor &t = a.t[i];
    t.cuts = (int)std::min<int64_t>((t.n_heads + kNormInFlight - 1) / kNormInFlight,
                                    std::max<int64_t>(1, 2048 / a.n_tensors / std::max<int64_t>(1, blocks)));
    cuts += t.cuts;
  }
  a.groups = (int)blocks;
  if (backward && blocks > 0) {
    // work groups walk the tokens, 8 for each CU, all as often, and leave a row of sums each.  (4 for each CU: the
    // gradients of 10800 tokens of 12 + 12 heads 59 us instead of 49.)
    const int64_t most = std::max<int64_t>(1, 2048 / cuts), times = (blocks + most - 1) / most;
    a.groups = (int)((blocks + times - 1) / times);
  }
}

hc_status check_weight(hc_ctx *c, const char *name, const void *p) {
  if (p && !aligned16(p)) return fail(c, HC_E_INVAL, "%s must be 16-byte aligned", name);
  return HC_OK;
}

// Whether a tensor may take another's place: the same type and strides.
bool same_rows(int type_a, int type_b, const Rows &a, const Rows &b) {
  return type_a == type_b && (a.n_tokens <= 1 || a.token == b.token) && (a.n_heads <= 1 || a.head == b.head);
}

hc_status norm_grad_plan(hc_ctx *c, const hc_norm_args *p, const hc_norm_grad_tensor *t, int n_tensors, NormArgs &a) {
  hc_status st = check_norm(c, p, t, n_tensors, a);
  if (st != HC_OK) return st;
  for (int i = 0; i < n_tensors; ++i)
    a.t[i] = {t[i].x, t[i].weight, const_cast<void *>(t[i].dout), t[i].dx, t[i].dweight, t[i].x_token, t[i].x_head,
              t[i].dout_token, t[i].dout_head, t[i].dx_token, t[i].dx_head, t[i].n_heads, 0};
  if ((st = check_norm_size(c, a)) != HC_OK) return st;
  plan_norm(a, p->rotate.halves != 0, true);
  return HC_OK;
}
int64_t norm_grad_bytes(const NormArgs &a) {
  int64_t rows = 0;
  for (int i = 0; i < a.n_tensors; ++i) rows += norm_parts(a, i);
  return rows * a.rotate.head_dim * 4;
}

// --- the mask ---------------------------------------------------------------------------------
hc_status check_mask(hc_ctx *c, int block, int window, int sinks) {
  if (block < 0 || window < 0 || sinks < 0)
    return fail(c, HC_E_INVAL, "causal_block, window and sinks must not be negative");
  if (block == 0 && window > 0) return fail(c, HC_E_INVAL, "a window needs causal_block");
  return HC_OK;
}
// Keys that the units of a call see at most, of `keys`: R rows of them see a window, the blocks at its ends, and the first tokens.
int64_t seen_at_most(const SeqArgs &a, int64_t keys, int R) {
  if (a.window == 0) return keys;
  return std::min(keys, (int64_t)a.window + a.block + R / a.group + a.sinks);
}

// --- pages ----------------------------------------------------------------------------------------
hc_status check_pages(hc_ctx *c, const hc_pages *p, const hc_page_table *t, bool data, int &shift) {
  if (!p || !t) return fail(c, HC_E_INVAL, "pages or table is NULL");
  if (p->n_pages < 1 || p->n_heads < 1) return fail(c, HC_E_INVAL, "the pages' n_pages and n_heads must be at least 1");
  if (p->head_dim != 64 && p->head_dim != 128) return fail(c, HC_E_INVAL, "the pages' head_dim must be 64 or 128");
  if (p->page_tokens < 16 || p->page_tokens > 65536 || (p->page_tokens & (p->page_tokens - 1)) != 0)
    return fail(c, HC_E_INVAL, "page_tokens must be a power of two, 16 to 65536");
  for (shift = 4; 1 << shift < p->page_tokens;) ++shift;
  if (t->n_seqs < 1 || t->max_pages < 1) return fail(c, HC_E_INVAL, "the table's n_seqs and max_pages must be at least 1");
  if ((int64_t)t->max_pages << shift > INT32_MAX - kSeqKeys) return fail(c, HC_E_INVAL, "the table has too many slots");
  if (t->n_seqs > 1 && t->stride < t->max_pages) return fail(c, HC_E_INVAL, "the table's rows overlap");
  auto good = [](int64_t stride, int64_t n) { return n <= 1 || (stride >= 0 && stride % 8 == 0); };
  if (!good(p->k_page, p->n_pages) || !good(p->v_page, p->n_pages) || !good(p->k_token, 2) || !good(p->v_token, 2) ||
      !good(p->k_head, p->n_heads) || !good(p->v_head, p->n_heads))
    return fail(c, HC_E_INVAL, "pages: strides must be multiples of 8 and not negative");
  if (!data) return HC_OK;
  if (!p->k || !p->v || !aligned16(p->k) || !aligned16(p->v))
    return fail(c, HC_E_INVAL, "the pages' k and v must be 16-byte aligned device pointers");
  if (!t->table || !aligned4(t->table)) return fail(c, HC_E_INVAL, "table must be a 4-byte aligned device pointer");
  return HC_OK;
}
// Pages that are written: no two rows of them overlap, whatever the order of their axes.
hc_status check_written(hc_ctx *c, const char *name, const hc_pages *p, int64_t page, int64_t token, int64_t head) {
  struct { int64_t stride, n; } axes[3] = {{page, p->n_pages}, {token, p->page_tokens}, {head, p->n_heads}};
  std::sort(axes, axes + 3, [](const auto &x, const auto &y) { return x.stride < y.stride; });
  int64_t end = p->head_dim;
  for (const auto &x : axes) {
    if (x.n <= 1) continue;
    if (x.stride < end) return fail(c, HC_E_INVAL, "%s: rows of the pages overlap", name);
    end += x.stride > (INT64_MAX - end) / x.n ? INT64_MAX - end : (x.n - 1) * x.stride;
  }
  return HC_OK;
}

void use_pages(SeqArgs &a, const hc_pages *p, const hc_page_table *t, int shift) {
  a.k = (const uint16_t *)p->k; a.v = (const uint16_t *)p->v;
  a.k_page = p->k_page; a.k_token = p->k_token; a.k_head = p->k_head;
  a.v_page = p->v_page; a.v_token = p->v_token; a.v_head = p->v_head;
  a.table = t->table; a.table_seq = t->stride;
  a.n_pages = p->n_pages; a.page_shift = shift;
  a.capacity = t->max_pages << shift;
}

hc_status paged_plan(hc_ctx *c, const hc_pages *pages, const hc_page_table *table, const hc_paged_args *p, bool data,
                     SeqArgs &a, bool &few_rows) {
  int shift;
  hc_status st = check_pages(c, pages, table, data, shift);
  if (st != HC_OK) return st;
  if (!p) return fail(c, HC_E_INVAL, "args is NULL");
  if (p->n_tokens < 0) return fail(c, HC_E_INVAL, "n_tokens must not be negative");
  if (p->n_heads < 1 || p->n_heads % pages->n_heads != 0)
    return fail(c, HC_E_INVAL, "n_heads must be a multiple of the pages'");
  if (p->max_kv < 0) return fail(c, HC_E_INVAL, "max_kv must not be negative");
  if ((st = check_mask(c, p->causal_block, p->window, p->sinks)) != HC_OK) return st;
  if ((st = check_scale(c, p->softmax_scale)) != HC_OK) return st;
  if ((st = check_parts(c, "cu_seqlens", p->cu_seqlens, p->n_tokens, table->n_seqs)) != HC_OK) return st;
  a = SeqArgs{};
  a.q = (const uint16_t *)p->q; a.o = (uint16_t *)p->out;
  a.q_token = p->q_token; a.q_head = p->q_head; a.o_token = p->out_token; a.o_head = p->out_head;
  use_pages(a, pages, table, shift);
  a.cu_q = p->cu_seqlens; a.kv_len = p->kv_len;
  a.n_seqs = table->n_seqs; a.n_tokens = p->n_tokens;
  a.kv_heads = pages->n_heads; a.group = p->n_heads / pages->n_heads;
  a.block = p->causal_block; a.window = p->window; a.sinks = p->sinks;
  a.scale_log2 = scale_log2(p->softmax_scale, pages->head_dim);
  a.n_split = 1;
  const int64_t rows = (int64_t)p->n_tokens * a.group;
  // (the kernel for few rows reads the cache once per 16 rows: see cached_plan in hc_ops.cpp)
  few_rows = rows <= (int64_t)a.n_seqs * 2 * kDecodeRows;
  const int R = few_rows ? kDecodeRows : kSeqRows;
  // (a token adds ceil(group / R) units at most: no more are made room for where each sequence has one)
  const int64_t tiles = std::min(unit_room(p->n_tokens, a.n_seqs, a.group, R, p->cu_seqlens == nullptr),
                                 (int64_t)p->n_tokens * ((a.group + R - 1) / R));
  if (rows > INT32_MAX - kSeqRows || !good_grid(tiles * a.kv_heads))
    return fail(c, HC_E_INVAL, "too many query rows for one call");
  a.tiles = (int)tiles;
  const int64_t keys = seen_at_most(a, p->max_kv > 0 ? std::min(p->max_kv, a.capacity) : a.capacity, R);
  const int64_t units = seq_units(a);
  // Work groups wanted for few rows: 1024 against 1536, single tokens: 48 sequences of up to 8192 keys, 4 x 7 heads of 64 dims (192
  // units) 24.3 and 27.7 us; 32 of up to 4096, 8 x 4 heads of 128 dims (256) 64 and 67; 24 of up to 5000, 12 heads (288) 91.8 and 89.7.
  if (few_rows) choose_split(a, keys, units < 64 || units >= 512 ? 512 : units <= 256 ? 1024 : 1536, 4, kDecodeMaxSplit);
  else choose_split(a, keys, 512, 8, kSeqMaxSplit);
  // (the wide kernel's copies hold offsets of a run of 16 rows in 32 bits)
  a.wide = pages->head_dim == 128 && !few_rows && a.k_token < 1 << 24 && a.v_token < 1 << 24 && wide_rows(a, keys);
  cut_last_round(a, keys, a.window > 0 || (a.n_seqs == 1 && a.block == 0));
  return HC_OK;
}

// --- packed sequences -------------------------------------------------------------------------------
hc_status window_plan(hc_ctx *c, const hc_window_args *p, SeqArgs &a) {
  if (!p) return fail(c, HC_E_INVAL, "args is NULL");
  if (p->n_tokens < 0 || p->n_keys < 0 || p->n_seqs < 1)
    return fail(c, HC_E_INVAL, "n_tokens and n_keys must not be negative, n_seqs not below 1");
  if (p->n_kv_heads < 1 || p->n_heads < 1 || p->n_heads % p->n_kv_heads != 0)
    return fail(c, HC_E_INVAL, "n_heads must be a multiple of n_kv_heads");
  if (p->head_dim != 64 && p->head_dim != 128) return fail(c, HC_E_INVAL, "head_dim must be 64 or 128");
  if (p->n_keys > INT32_MAX - kSeqKeys) return fail(c, HC_E_INVAL, "too many keys for one call");
  if (!p->cu_k && p->n_keys != p->n_tokens)
    return fail(c, HC_E_INVAL, "cu_k is NULL, so n_keys must be n_tokens");
  if (p->cu_k && !aligned4(p->cu_k)) return fail(c, HC_E_INVAL, "cu_k must be 4-byte aligned");
  if (p->lse && !aligned4(p->lse)) return fail(c, HC_E_INVAL, "lse must be 4-byte aligned");
  hc_status st = check_mask(c, p->causal_block, p->window, p->sinks);
  if (st == HC_OK) st = check_scale(c, p->softmax_scale);
  if (st == HC_OK) st = check_parts(c, "cu_q", p->cu_q, p->n_tokens, p->n_seqs);
  if (st != HC_OK) return st;
  a = SeqArgs{};
  a.q = (const uint16_t *)p->q; a.o = (uint16_t *)p->out; a.lse = p->lse;
  a.q_token = p->q_token; a.q_head = p->q_head; a.o_token = p->out_token; a.o_head = p->out_head;
  a.k = (const uint16_t *)p->k; a.v = (const uint16_t *)p->v;
  a.k_token = p->k_token; a.k_head = p->k_head; a.v_token = p->v_token; a.v_head = p->v_head;
  a.cu_q = p->cu_q; a.cu_k = p->cu_k;
  a.n_seqs = p->n_seqs; a.n_tokens = p->n_tokens; a.n_keys = p->n_keys;
  a.kv_heads = p->n_kv_heads; a.group = p->n_heads / p->n_kv_heads;
  a.block = p->causal_block; a.window = p->window; a.sinks = p->sinks;
  a.scale_log2 = scale_log2(p->softmax_scale, p->head_dim);
  a.n_split = 1;
  const int64_t rows = (int64_t)p->n_tokens * a.group;
  const int64_t tiles = unit_room(p->n_tokens, p->n_seqs, a.group, kSeqRows, p->cu_q == nullptr);
  if (rows > INT32_MAX - kSeqRows || !good_grid(tiles * a.kv_heads))
    return fail(c, HC_E_INVAL, "too many query rows for one call");
  a.tiles = (int)tiles;
  // (the host knows how many keys the sequences have together, not how they are shared: the longest
  // of several, which ends last, is taken for twice the average)
  const int64_t keys = (int64_t)p->n_keys / p->n_seqs * (p->cu_q && p->n_seqs > 1 ? 2 : 1);
  choose_split(a, seen_at_most(a, keys, kSeqRows), 512, 8, kSeqMaxSplit);
  // (the wide kernel's copies hold offsets of 63 rows in 32 bits)
  a.wide = p->head_dim == 128 && p->k_token < 1 << 24 && p->v_token < 1 << 24 &&
           wide_rows(a, seen_at_most(a, p->n_keys / p->n_seqs, kSeqRows));
  cut_last_round(a, seen_at_most(a, keys, kSeqRows), a.window > 0 || (a.n_seqs == 1 && a.block == 0));
  return HC_OK;
}

hc_status check_window_tensors(hc_ctx *c, const hc_window_args *p, bool writes) {
  const Rows out{"out", p->out, p->out_token, p->out_head, p->n_tokens, p->n_heads};
  hc_status st = check_tensor(c, {"q", p->q, p->q_token, p->q_head, p->n_tokens, p->n_heads});
  if (st == HC_OK) st = writes ? check_output(c, out, p->head_dim) : check_tensor(c, out);
  if (st == HC_OK && p->n_keys > 0)
    st = check_tensor(c, {"k", p->k, p->k_token, p->k_head, p->n_keys, p->n_kv_heads});
  if (st == HC_OK && p->n_keys > 0)
    st = check_tensor(c, {"v", p->v, p->v_token, p->v_head, p->n_keys, p->n_kv_heads});
  return st;
}

// --- gradients --------------------------------------------------------------------------------------
hc_status grad_plan(hc_ctx *c, const hc_window_grad_args *g, GradArgs &a) {
  if (!g) return fail(c, HC_E_INVAL, "args is NULL");
  const hc_window_args *p = &g->forward;
  a = GradArgs{};
  const hc_status st = window_plan(c, p, a.seq);
  if (st != HC_OK) return st;
  a.lse = p->lse;
  a.dout = (const uint16_t *)g->dout;
  a.dq = (uint16_t *)g->dq; a.dk = (uint16_t *)g->dk; a.dv = (uint16_t *)g->dv;
  a.do_token = g->dout_token; a.do_head = g->dout_head; a.dq_token = g->dq_token; a.dq_head = g->dq_head;
  a.dk_token = g->dk_token; a.dk_head = g->dk_head; a.dv_token = g->dv_token; a.dv_head = g->dv_head;
  a.scale = p->softmax_scale > 0.f ? p->softmax_scale : 1.0f / std::sqrt((float)p->head_dim);
  // units: runs of 128 queries of a query head, and of 128 keys of a key head
  const int64_t q_tiles = unit_room(p->n_tokens, p->n_seqs, 1, kSeqRows, p->cu_q == nullptr);
  const bool alike = (p->cu_k ? p->cu_k : p->cu_q) == nullptr;
  const int64_t k_tiles = unit_room(p->n_keys, p->n_seqs, 1, kGradKeys, alike);
  const int64_t units = k_tiles * p->n_kv_heads;
  // Key units are cut into pieces of rows until 512 work groups run (two for each CU with 64-dim heads, two rounds with 128), but
  // no piece is shorter than 4 tiles of rows: a partial gradient costs two writes, two reads and a launch.  Forward and gradients
  // with 256, 384, 512 and 768: one sequence of 2048, 4 x 4 heads of 128 dims 152, 154, 159 and 175 us; two heads of 4096, 64 dims
  // 104, 100, 106 and 114; six prompts of up to 1450, window 512, 4 x 3 heads of 64 dims 126, 94, 85 and 90; ten of up to 2000,
  // window 1000, 2 x 4 heads 139, 117, 119 and 120.
  int64_t queries = (int64_t)p->n_tokens / p->n_seqs;            // that see a key, about
  if (p->window > 0) queries = std::min(queries, (int64_t)p->window + p->causal_block + kGradKeys);
  const int64_t tiles = queries * a.seq.group / 64;
  a.n_split = (int)std::max<int64_t>(1, std::min<int64_t>({512 / std::max<int64_t>(units, 1), tiles / 4, 16}));
  if (!good_grid(q_tiles * p->n_heads + units * std::max(a.n_split, 16)) ||
      !good_grid((int64_t)p->n_tokens * p->n_heads / (256 / 16) + 1))
    return fail(c, HC_E_INVAL, "too many rows for one call");
  a.seq.tiles = (int)q_tiles;
  a.key_tiles = (int)k_tiles;
  return HC_OK;
}
int64_t grad_stat_bytes(const hc_window_args &p) { return ((int64_t)p.n_tokens * p.n_heads * 8 + 15) / 16 * 16; }
int64_t grad_bytes(const hc_window_args &p, const GradArgs &a) {
  const int64_t parts = a.n_split > 1 ? (int64_t)a.key_tiles * p.n_kv_heads * a.n_split * 2 * kGradKeys * p.head_dim * 4 : 0;
  return grad_stat_bytes(p) + parts;
}

}  // namespace

extern "C" {

hc_status hc_norm_rotate(hc_ctx *c, const hc_norm_args *p, const hc_norm_tensor *t, int n_tensors, hc_stream stream) try {
  if (!c) return HC_E_INVAL;
  NormArgs a;
  hc_status st = check_norm(c, p, t, n_tensors, a);
  if (st != HC_OK) return st;
  const hc_rotate_args &r = p->rotate;
  for (int i = 0; i < n_tensors; ++i) {
    a.t[i] = {t[i].x, t[i].weight, t[i].out, nullptr, nullptr, t[i].x_token, t[i].x_head, t[i].out_token, t[i].out_head,
              0, 0, t[i].n_heads, 0};
    if (t[i].n_heads < 1 || r.n_tokens == 0) continue;
    const Rows x{"x", t[i].x, t[i].x_token, t[i].x_head, r.n_tokens, t[i].n_heads};
    const Rows out{"out", t[i].out, t[i].out_token, t[i].out_head, r.n_tokens, t[i].n_heads};
    st = check_tensor(c, x);
    if (st == HC_OK) st = check_output(c, out, r.head_dim);
    if (st == HC_OK) st = check_weight(c, "weight", t[i].weight);
    if (st != HC_OK) return st;
    if (x.p == out.p && !same_rows(r.x_type, r.out_type, x, out))
      return fail(c, HC_E_INVAL, "tensor %d: in place needs the same type and strides", i);
  }
  if ((st = check_norm_size(c, a)) != HC_OK) return st;
  if (r.n_tokens == 0) return HC_OK;
  if ((st = plan_rotation(c, &r, a.rotate)) != HC_OK) return st;
  plan_norm(a, r.halves != 0, false);
  OnDevice on(c->device);
  HC_HIP(c, on.status);
  return timed_launch(c, (hipStream_t)stream, HC_K_ROTATE, [&] {
    return launch_norm(a, r.x_type, r.out_type, r.halves != 0, (hipStream_t)stream);
  });
} HC_NO_HOST_MEMORY(c)

hc_status hc_norm_rotate_workspace(hc_ctx *c, const hc_norm_args *p, const hc_norm_grad_tensor *t, int n_tensors,
                                   int64_t *bytes) {
  if (!c) return HC_E_INVAL;
  if (!bytes) return fail(c, HC_E_INVAL, "bytes is NULL");
  NormArgs a;
  const hc_status st = norm_grad_plan(c, p, t, n_tensors, a);
  if (st != HC_OK) return st;
  *bytes = norm_grad_bytes(a);
  return HC_OK;
}

hc_status hc_norm_rotate_backward(hc_ctx *c, const hc_norm_args *p, const hc_norm_grad_tensor *t, int n_tensors,
                                  void *workspace, int64_t workspace_bytes, hc_stream stream) try {
  if (!c) return HC_E_INVAL;
  NormArgs a;
  hc_status st = norm_grad_plan(c, p, t, n_tensors, a);
  if (st != HC_OK) return st;
  const hc_rotate_args &r = p->rotate;
  for (int i = 0; i < n_tensors; ++i) {
    if ((st = check_weight(c, "weight", t[i].weight)) == HC_OK) st = check_weight(c, "dweight", t[i].dweight);
    if (st != HC_OK) return st;
    if (r.n_tokens == 0) continue;
    const Rows x{"x", t[i].x, t[i].x_token, t[i].x_head, r.n_tokens, t[i].n_heads};
    const Rows dout{"dout", t[i].dout, t[i].dout_token, t[i].dout_head, r.n_tokens, t[i].n_heads};
    const Rows dx{"dx", t[i].dx, t[i].dx_token, t[i].dx_head, r.n_tokens, t[i].n_heads};
    st = check_tensor(c, x);
    if (st == HC_OK) st = check_tensor(c, dout);
    if (st == HC_OK) st = check_output(c, dx, r.head_dim);
    if (st != HC_OK) return st;
    if ((dx.p == x.p && !same_rows(r.x_type, r.x_type, dx, x)) || (dx.p == dout.p && !same_rows(r.x_type, r.out_type, dx, dout)))
      return fail(c, HC_E_INVAL, "tensor %d: in place needs the same type and strides", i);
  }
  if ((st = check_workspace(c, workspace, workspace_bytes, norm_grad_bytes(a))) != HC_OK) return st;
  a.part = (float *)workspace;
  // (no tokens: the weights' gradients are zero, which the second launch writes)
  if ((st = plan_rotation(c, &r, a.rotate)) != HC_OK) return st;
  OnDevice on(c->device);
  HC_HIP(c, on.status);
  return timed_launch(c, (hipStream_t)stream, HC_K_ROTATE, [&] {
    return launch_norm_backward(a, r.x_type, r.out_type, r.halves != 0, (hipStream_t)stream);
  });
} HC_NO_HOST_MEMORY(c)

hc_status hc_paged_append(hc_ctx *c, const hc_pages *pages, const hc_page_table *table, const hc_qcache_rows *r,
                          hc_stream stream) try {
  if (!c) return HC_E_INVAL;
  int shift;
  hc_status st = check_pages(c, pages, table, true, shift);
  if (st == HC_OK) st = check_written(c, "k", pages, pages->k_page, pages->k_token, pages->k_head);
  if (st == HC_OK) st = check_written(c, "v", pages, pages->v_page, pages->v_token, pages->v_head);
  if (st != HC_OK) return st;
  if (!r) return fail(c, HC_E_INVAL, "rows is NULL");
  if (r->n_tokens < 0) return fail(c, HC_E_INVAL, "n_tokens must not be negative");
  if ((st = check_parts(c, "cu_seqlens", r->cu_seqlens, r->n_tokens, table->n_seqs)) != HC_OK) return st;
  if (r->n_tokens == 0) return HC_OK;
  st = check_tensor(c, {"k", r->k, r->k_token, r->k_head, r->n_tokens, pages->n_heads});
  if (st == HC_OK) st = check_tensor(c, {"v", r->v, r->v_token, r->v_head, r->n_tokens, pages->n_heads});
  if (st != HC_OK) return st;
  if (!r->start || !aligned4(r->start)) return fail(c, HC_E_INVAL, "start must be a 4-byte aligned device pointer");
  // (a work group's pieces are counted in 32 bits)
  if (pages->n_heads > 1 << 20 || !good_grid((int64_t)r->n_tokens / 4 + 1)) return fail(c, HC_E_INVAL, "too many rows for one call");
  OnDevice on(c->device);
  HC_HIP(c, on.status);
  const PagedRowsArgs a{*pages, *table, *r, shift};
  return timed_launch(c, (hipStream_t)stream, HC_K_CACHE, [&] { return launch_paged_append(a, (hipStream_t)stream); });
} HC_NO_HOST_MEMORY(c)

hc_status hc_paged_workspace(hc_ctx *c, const hc_pages *pages, const hc_page_table *table, const hc_paged_args *p,
                             int64_t *bytes) {
  if (!c) return HC_E_INVAL;
  if (!bytes) return fail(c, HC_E_INVAL, "bytes is NULL");
  SeqArgs a;
  bool few_rows;
  const hc_status st = paged_plan(c, pages, table, p, false, a, few_rows);
  if (st != HC_OK) return st;
  *bytes = part_bytes(a, pages->head_dim, few_rows ? kDecodeRows : kSeqRows);
  return HC_OK;
}

hc_status hc_paged_attention(hc_ctx *c, const hc_pages *pages, const hc_page_table *table, const hc_paged_args *p,
                             hc_stream stream) try {
  if (!c) return HC_E_INVAL;
  SeqArgs a;
  bool few_rows;
  hc_status st = paged_plan(c, pages, table, p, true, a, few_rows);
  if (st != HC_OK) return st;
  if (p->n_tokens == 0) return HC_OK;
  st = check_tensor(c, {"q", p->q, p->q_token, p->q_head, p->n_tokens, p->n_heads});
  if (st == HC_OK)
    st = check_output(c, {"out", p->out, p->out_token, p->out_head, p->n_tokens, p->n_heads}, pages->head_dim);
  if (st != HC_OK) return st;
  if (!p->kv_len || !aligned4(p->kv_len)) return fail(c, HC_E_INVAL, "kv_len must be a 4-byte aligned device pointer");
  const int R = few_rows ? kDecodeRows : kSeqRows;
  if ((st = check_workspace(c, p->workspace, p->workspace_bytes, part_bytes(a, pages->head_dim, R))) != HC_OK) return st;
  if (a.n_split > 1) use_workspace(a, p->workspace);
  OnDevice on(c->device);
  HC_HIP(c, on.status);
  return timed_launch(c, (hipStream_t)stream, HC_K_SEQUENCE, [&] {
    hipError_t e = few_rows ? launch_paged_decode(a, pages->head_dim, (hipStream_t)stream)
                            : launch_window(a, pages->head_dim, (hipStream_t)stream);
    if (e == hipSuccess && a.n_split > 1) e = launch_seq_merge(a, pages->head_dim, R, (hipStream_t)stream);
    return e;
  });
} HC_NO_HOST_MEMORY(c)

hc_status hc_window_workspace(hc_ctx *c, const hc_window_args *p, int64_t *bytes) {
  if (!c) return HC_E_INVAL;
  if (!bytes) return fail(c, HC_E_INVAL, "bytes is NULL");
  SeqArgs a;
  const hc_status st = window_plan(c, p, a);
  if (st != HC_OK) return st;
  *bytes = part_bytes(a, p->head_dim, kSeqRows, true);       // (with or without lse)
  return HC_OK;
}

hc_status hc_window_attention(hc_ctx *c, const hc_window_args *p, hc_stream stream) try {
  if (!c) return HC_E_INVAL;
  SeqArgs a;
  hc_status st = window_plan(c, p, a);
  if (st != HC_OK) return st;
  if (p->n_tokens == 0) return HC_OK;
  if ((st = check_window_tensors(c, p, true)) != HC_OK) return st;
  if ((st = check_workspace(c, p->workspace, p->workspace_bytes, part_bytes(a, p->head_dim, kSeqRows, true))) != HC_OK)
    return st;
  if (a.n_split > 1) use_workspace(a, p->workspace);
  OnDevice on(c->device);
  HC_HIP(c, on.status);
  return timed_launch(c, (hipStream_t)stream, HC_K_SEQUENCE, [&] {
    hipError_t e = launch_window(a, p->head_dim, (hipStream_t)stream);
    if (e == hipSuccess && a.n_split > 1) e = launch_seq_merge(a, p->head_dim, kSeqRows, (hipStream_t)stream);
    return e;
  });
} HC_NO_HOST_MEMORY(c)

hc_status hc_window_backward_workspace(hc_ctx *c, const hc_window_grad_args *g, int64_t *bytes) {
  if (!c) return HC_E_INVAL;
  if (!bytes) return fail(c, HC_E_INVAL, "bytes is NULL");
  GradArgs a;
  const hc_status st = grad_plan(c, g, a);
  if (st != HC_OK) return st;
  *bytes = grad_bytes(g->forward, a);
  return HC_OK;
}

hc_status hc_window_attention_backward(hc_ctx *c, const hc_window_grad_args *g, hc_stream stream) try {
  if (!c) return HC_E_INVAL;
  GradArgs a;
  hc_status st = grad_plan(c, g, a);
  if (st != HC_OK) return st;
  const hc_window_args &p = g->forward;
  if (p.n_tokens == 0 && p.n_keys == 0) return HC_OK;
  if (p.n_tokens > 0) {
    st = check_window_tensors(c, &p, false);
    if (st == HC_OK) st = check_tensor(c, {"dout", g->dout, g->dout_token, g->dout_head, p.n_tokens, p.n_heads});
    if (st == HC_OK) st = check_output(c, {"dq", g->dq, g->dq_token, g->dq_head, p.n_tokens, p.n_heads}, p.head_dim);
    if (st == HC_OK && !p.lse) st = fail(c, HC_E_INVAL, "lse is NULL");
    if (st == HC_OK && p.q == p.out) st = fail(c, HC_E_INVAL, "the forward call's out has overwritten q");
  }
  if (st == HC_OK && p.n_keys > 0) {
    st = check_tensor(c, {"k", p.k, p.k_token, p.k_head, p.n_keys, p.n_kv_heads});
    if (st == HC_OK) st = check_tensor(c, {"v", p.v, p.v_token, p.v_head, p.n_keys, p.n_kv_heads});
    if (st == HC_OK) st = check_output(c, {"dk", g->dk, g->dk_token, g->dk_head, p.n_keys, p.n_kv_heads}, p.head_dim);
    if (st == HC_OK) st = check_output(c, {"dv", g->dv, g->dv_token, g->dv_head, p.n_keys, p.n_kv_heads}, p.head_dim);
  }
  if (st != HC_OK) return st;
  // (logarithms of the rows' sums are divided by it)
  if (a.scale < 0x1p-100f) return fail(c, HC_E_INVAL, "softmax_scale must not be below 2^-100");
  // (the copies of 64 rows hold their offsets in 32 bits)
  for (int64_t stride : {p.n_tokens > 1 ? std::max(p.q_token, g->dout_token) : 0, p.n_keys > 1 ? std::max(p.k_token, p.v_token) : 0})
    if (stride >= 1 << 24) return fail(c, HC_E_INVAL, "token strides must be below 2^24");
  if ((st = check_workspace(c, g->workspace, g->workspace_bytes, grad_bytes(p, a))) != HC_OK) return st;
  a.stats = (float *)g->workspace;
  a.part = (float *)((char *)g->workspace + grad_stat_bytes(p));
  OnDevice on(c->device);
  HC_HIP(c, on.status);
  return timed_launch(c, (hipStream_t)stream, HC_K_GRADIENT, [&] {
    return p.head_dim == 128 ? launch_grad128(a, (hipStream_t)stream) : launch_grad64(a, (hipStream_t)stream);
  });
} HC_NO_HOST_MEMORY(c)

}  // extern "C"
