// Entry points of the operators beside the routed attention: rotary positions,
// attention over packed sequences, and the 4-bit cache with its attention.
#include "hc_args.h"

using namespace hc;

namespace {

hc_status run_seq(hc_ctx *c, const SeqArgs &a, int head_dim, bool few_rows, hipStream_t s) {
  return timed_launch(c, s, HC_K_SEQUENCE, [&] {
    hipError_t e = few_rows ? launch_decode(a, head_dim, s) : launch_seq(a, head_dim, s);
    if (e == hipSuccess && a.n_split > 1)
      e = launch_seq_merge(a, head_dim, few_rows ? kDecodeRows : kSeqRows, s);
    return e;
  });
}

// --- packed attention -----------------------------------------------------------------
hc_status packed_plan(hc_ctx *c, const hc_packed_args *p, SeqArgs &a) {
  if (!p) return fail(c, HC_E_INVAL, "args is NULL");
  if (p->n_tokens < 0 || p->n_keys < 0 || p->n_seqs < 1)
    return fail(c, HC_E_INVAL, "n_tokens and n_keys must not be negative, n_seqs not below 1");
  if (p->n_kv_heads < 1 || p->n_heads < 1 || p->n_heads % p->n_kv_heads != 0)
    return fail(c, HC_E_INVAL, "n_heads must be a multiple of n_kv_heads");
  if (p->head_dim != 64 && p->head_dim != 128) return fail(c, HC_E_INVAL, "head_dim must be 64 or 128");
  if (p->causal_block < 0) return fail(c, HC_E_INVAL, "causal_block must not be negative");
  // (the kernels round key counts up to whole tiles in 32 bits; keys of stride 0 take no memory)
  if (p->n_keys > INT32_MAX - kSeqKeys) return fail(c, HC_E_INVAL, "too many keys for one call");
  if (!p->cu_k && p->n_keys != p->n_tokens)
    return fail(c, HC_E_INVAL, "cu_k is NULL, so n_keys must be n_tokens");
  if (p->cu_k && !aligned4(p->cu_k)) return fail(c, HC_E_INVAL, "cu_k must be 4-byte aligned");
  hc_status st = check_scale(c, p->softmax_scale);
  if (st == HC_OK) st = check_parts(c, "cu_q", p->cu_q, p->n_tokens, p->n_seqs);
  if (st != HC_OK) return st;
  a = SeqArgs{};
  a.q = (const uint16_t *)p->q; a.o = (uint16_t *)p->out;
  a.q_token = p->q_token; a.q_head = p->q_head; a.o_token = p->out_token; a.o_head = p->out_head;
  a.k = (const uint16_t *)p->k; a.v = (const uint16_t *)p->v;
  a.k_token = p->k_token; a.k_head = p->k_head; a.v_token = p->v_token; a.v_head = p->v_head;
  a.cu_q = p->cu_q; a.cu_k = p->cu_k;
  a.n_seqs = p->n_seqs; a.n_tokens = p->n_tokens; a.n_keys = p->n_keys;
  a.kv_heads = p->n_kv_heads; a.group = p->n_heads / p->n_kv_heads;
  a.block = p->causal_block;
  a.scale_log2 = scale_log2(p->softmax_scale, p->head_dim);
  a.n_split = 1;
  const int64_t rows = (int64_t)p->n_tokens * a.group;
  const int64_t tiles = unit_room(p->n_tokens, p->n_seqs, a.group, kSeqRows, p->cu_q == nullptr);
  if (rows > INT32_MAX - kSeqRows || !good_grid(tiles * a.kv_heads))
    return fail(c, HC_E_INVAL, "too many query rows for one call");
  a.tiles = (int)tiles;
  // (the host knows how many keys the sequences have together, not how they are shared: the longest
  // of several, which ends last, is taken for twice the average)
  choose_split(a, (int64_t)p->n_keys / p->n_seqs * (p->cu_q && p->n_seqs > 1 ? 2 : 1), 512, 8, kSeqMaxSplit);
  // (the wide kernel's copies hold offsets of 63 rows in 32 bits)
  a.wide = p->head_dim == 128 && p->k_token < 1 << 24 && p->v_token < 1 << 24 &&
           wide_rows(a, p->n_keys / p->n_seqs);
  cut_last_round(a, p->n_keys, a.n_seqs == 1 && a.block == 0);
  return HC_OK;
}

// --- the 4-bit cache --------------------------------------------------------------------
hc_status check_cache(hc_ctx *c, const hc_qcache *k, bool data) {
  if (!k) return fail(c, HC_E_INVAL, "cache is NULL");
  if (k->n_seqs < 1 || k->n_heads < 1 || k->capacity < 1)
    return fail(c, HC_E_INVAL, "the cache's n_seqs, n_heads and capacity must be at least 1");
  if (k->head_dim != 64 && k->head_dim != 128)
    return fail(c, HC_E_INVAL, "the cache's head_dim must be 64 or 128");
  if (k->capacity > INT32_MAX - kQTokens) return fail(c, HC_E_INVAL, "the cache's capacity is too large");
  // (the product of three 31-bit numbers and a tile fits 128 bits only)
  if ((__int128)k->n_seqs * k->n_heads * qcache_head_bytes(k->capacity, k->head_dim) > INT64_MAX)
    return fail(c, HC_E_INVAL, "the cache is too large");
  if (data && (!k->data || !aligned16(k->data)))
    return fail(c, HC_E_INVAL, "the cache's data must be a 16-byte aligned device pointer");
  return HC_OK;
}

hc_status cache_rows(hc_ctx *c, const hc_qcache *k, const hc_qcache_rows *r, bool writes, hipStream_t s,
                     hipError_t (*launch)(const QCacheArgs &, hipStream_t)) {
  if (!c) return HC_E_INVAL;
  hc_status st = check_cache(c, k, true);
  if (st != HC_OK) return st;
  if (!r) return fail(c, HC_E_INVAL, "rows is NULL");
  if (r->n_tokens < 0) return fail(c, HC_E_INVAL, "n_tokens must not be negative");
  if ((st = check_parts(c, "cu_seqlens", r->cu_seqlens, r->n_tokens, k->n_seqs)) != HC_OK) return st;
  if (r->n_tokens == 0) return HC_OK;
  for (const Rows &t : {Rows{"k", r->k, r->k_token, r->k_head, r->n_tokens, k->n_heads},
                        Rows{"v", r->v, r->v_token, r->v_head, r->n_tokens, k->n_heads}}) {
    st = writes ? check_output(c, t, k->head_dim) : check_tensor(c, t);
    if (st != HC_OK) return st;
  }
  if (!r->start || !aligned4(r->start)) return fail(c, HC_E_INVAL, "start must be a 4-byte aligned device pointer");
  if (!good_grid(((int64_t)r->n_tokens + 7) / 8 * 8 * k->n_heads / 256 * 2 * (k->head_dim / 8) + 1))
    return fail(c, HC_E_INVAL, "too many rows for one call");
  OnDevice on(c->device);
  HC_HIP(c, on.status);
  const QCacheArgs a{*k, *r};
  return timed_launch(c, s, HC_K_CACHE, [&] { return launch(a, s); });
}

hc_status cached_plan(hc_ctx *c, const hc_qcache *k, const hc_qcache_attention_args *p, SeqArgs &a,
                      bool &few_rows) {
  hc_status st = check_cache(c, k, false);
  if (st != HC_OK) return st;
  if (!p) return fail(c, HC_E_INVAL, "args is NULL");
  if (p->n_tokens < 0) return fail(c, HC_E_INVAL, "n_tokens must not be negative");
  if (p->n_heads < 1 || p->n_heads % k->n_heads != 0)
    return fail(c, HC_E_INVAL, "n_heads must be a multiple of the cache's");
  if (p->causal_block < 0 || p->max_kv < 0)
    return fail(c, HC_E_INVAL, "causal_block and max_kv must not be negative");
  if ((st = check_scale(c, p->softmax_scale)) != HC_OK) return st;
  if ((st = check_parts(c, "cu_seqlens", p->cu_seqlens, p->n_tokens, k->n_seqs)) != HC_OK) return st;
  a = SeqArgs{};
  a.q = (const uint16_t *)p->q; a.o = (uint16_t *)p->out;
  a.q_token = p->q_token; a.q_head = p->q_head; a.o_token = p->out_token; a.o_head = p->out_head;
  a.cache = (const uint8_t *)k->data;
  a.cache_head = qcache_head_bytes(k->capacity, k->head_dim);
  a.capacity = k->capacity;
  a.cu_q = p->cu_seqlens; a.kv_len = p->kv_len;
  a.n_seqs = k->n_seqs; a.n_tokens = p->n_tokens;
  a.kv_heads = k->n_heads; a.group = p->n_heads / k->n_heads;
  a.block = p->causal_block;
  a.scale_log2 = scale_log2(p->softmax_scale, k->head_dim);
  a.n_split = 1;
  const int64_t rows = (int64_t)p->n_tokens * a.group;
  // The kernel for few rows reads the cache once per 16 rows and needs no LDS; up to two such
  // units per sequence it reads no more than the other kernel could hide.  (By the rows of the whole batch, which
  // is all that the host knows: a prompt of some hundred tokens beside many single ones runs by 16 rows too.)
  few_rows = rows <= (int64_t)k->n_seqs * 2 * kDecodeRows;
  const int R = few_rows ? kDecodeRows : kSeqRows;
  const int64_t tiles = unit_room(p->n_tokens, k->n_seqs, a.group, R, p->cu_seqlens == nullptr);
  if (rows > INT32_MAX - kSeqRows || !good_grid(tiles * a.kv_heads))
    return fail(c, HC_E_INVAL, "too many query rows for one call");
  a.tiles = (int)tiles;
  const int64_t keys = p->max_kv > 0 ? std::min(p->max_kv, k->capacity) : k->capacity;
  // Single tokens.  Two work groups per CU read a few long sequences fastest (131072 tokens of 8 heads: 26 us,
  // 30 with four, 33 with eight; two sequences of 65536: 31, 33 with four, 37 with six).  More sequences are
  // usually of different lengths and end unevenly, so their ranges are shorter: 48 of up to 8192 tokens, 4 heads,
  // 31 us with 512 groups, 23 with 1024, 19 with 1536; 8 of up to 32768, 8 heads, 47, 44 and 43.
  // (Equal ones lose by it: 32 of 8192, 8 heads, 32 and 36 us.)  512 units fill the card by themselves: 64
  // sequences of up to 1000 tokens, 8 heads, 13 us uncut, 20 in three ranges.
  // The borders are on the units that the launch has room for.  Where offsets are given those are more than can have
  // rows: the 48 sequences with 7 query heads to a key head are planned as 276 units and have 192, so
  // they are cut into 5 ranges, and into 8 where the same single tokens come without offsets.
  const int64_t units = seq_units(a);
  if (few_rows) choose_split(a, keys, units < 64 || units >= 512 ? 512 : units < 192 ? 1024 : 1536, 4, kDecodeMaxSplit);
  else choose_split(a, keys, 512, 8, kSeqMaxSplit);
  a.wide = k->head_dim == 128 && !few_rows && wide_rows(a, keys);
  cut_last_round(a, keys, a.n_seqs == 1 && a.block == 0);
  return HC_OK;
}

}  // namespace

extern "C" {

hc_status hc_rotate(hc_ctx *c, const hc_rotate_args *p, const hc_rotate_tensor *t, int n_tensors,
                    hc_stream stream) try {
  if (!c) return HC_E_INVAL;
  if (!p || !t) return fail(c, HC_E_INVAL, "args or tensors is NULL");
  if (n_tensors != 1 && n_tensors != 2) return fail(c, HC_E_INVAL, "n_tensors must be 1 or 2");
  if (p->n_tokens < 0) return fail(c, HC_E_INVAL, "n_tokens must not be negative");
  RotateArgs a;
  hc_status st = check_rotation(c, p, false, a);
  if (st != HC_OK) return st;
  int64_t heads = 0;
  for (int i = 0; i < n_tensors; ++i) {
    if (t[i].n_heads < 1) return fail(c, HC_E_INVAL, "tensor %d: n_heads must be at least 1", i);
    heads += t[i].n_heads;
    if (p->n_tokens == 0) continue;
    st = check_tensor(c, {"x", t[i].x, t[i].x_token, t[i].x_head, p->n_tokens, t[i].n_heads});
    if (st == HC_OK)
      st = check_output(c, {"out", t[i].out, t[i].out_token, t[i].out_head, p->n_tokens, t[i].n_heads}, p->head_dim);
    if (st != HC_OK) return st;
    if (t[i].x == t[i].out && (p->x_type != p->out_type || (p->n_tokens > 1 && t[i].x_token != t[i].out_token) ||
                               (t[i].n_heads > 1 && t[i].x_head != t[i].out_head)))
      return fail(c, HC_E_INVAL, "tensor %d: in place needs the same type and strides", i);
    a.t[i] = t[i];
  }
  if (heads > 65535 || !good_grid((int64_t)p->n_tokens * (p->head_dim / 8) / 256 + 1))
    return fail(c, HC_E_INVAL, "too many heads or tokens for one call");
  if (p->n_tokens == 0) return HC_OK;
  a.heads = (int)heads;
  if ((st = plan_rotation(c, p, a)) != HC_OK) return st;
  OnDevice on(c->device);
  HC_HIP(c, on.status);
  return timed_launch(c, (hipStream_t)stream, HC_K_ROTATE, [&] {
    return launch_rotate(a, p->x_type, p->out_type, p->halves != 0, (hipStream_t)stream);
  });
} HC_NO_HOST_MEMORY(c)

hc_status hc_packed_workspace(hc_ctx *c, const hc_packed_args *p, int64_t *bytes) {
  if (!c) return HC_E_INVAL;
  if (!bytes) return fail(c, HC_E_INVAL, "bytes is NULL");
  SeqArgs a;
  const hc_status st = packed_plan(c, p, a);
  if (st != HC_OK) return st;
  *bytes = part_bytes(a, p->head_dim, kSeqRows);
  return HC_OK;
}

hc_status hc_packed_attention(hc_ctx *c, const hc_packed_args *p, hc_stream stream) try {
  if (!c) return HC_E_INVAL;
  SeqArgs a;
  hc_status st = packed_plan(c, p, a);
  if (st != HC_OK) return st;
  if (p->n_tokens == 0) return HC_OK;
  st = check_tensor(c, {"q", p->q, p->q_token, p->q_head, p->n_tokens, p->n_heads});
  if (st == HC_OK) st = check_output(c, {"out", p->out, p->out_token, p->out_head, p->n_tokens, p->n_heads}, p->head_dim);
  if (st == HC_OK && p->n_keys > 0)
    st = check_tensor(c, {"k", p->k, p->k_token, p->k_head, p->n_keys, p->n_kv_heads});
  if (st == HC_OK && p->n_keys > 0)
    st = check_tensor(c, {"v", p->v, p->v_token, p->v_head, p->n_keys, p->n_kv_heads});
  if (st != HC_OK) return st;
  if ((st = check_workspace(c, p->workspace, p->workspace_bytes, part_bytes(a, p->head_dim, kSeqRows))) != HC_OK)
    return st;
  if (a.n_split > 1) use_workspace(a, p->workspace);
  OnDevice on(c->device);
  HC_HIP(c, on.status);
  return run_seq(c, a, p->head_dim, false, (hipStream_t)stream);
} HC_NO_HOST_MEMORY(c)

hc_status hc_qcache_bytes(const hc_qcache *k, int64_t *bytes) {
  if (!bytes || check_cache(nullptr, k, false) != HC_OK) return HC_E_INVAL;
  *bytes = (int64_t)k->n_seqs * k->n_heads * qcache_head_bytes(k->capacity, k->head_dim);
  return HC_OK;
}

hc_status hc_qcache_append(hc_ctx *c, const hc_qcache *k, const hc_qcache_rows *r, hc_stream stream) try {
  return cache_rows(c, k, r, false, (hipStream_t)stream, launch_qcache_append);
} HC_NO_HOST_MEMORY(c)

hc_status hc_qcache_read(hc_ctx *c, const hc_qcache *k, const hc_qcache_rows *r, hc_stream stream) try {
  return cache_rows(c, k, r, true, (hipStream_t)stream, launch_qcache_read);
} HC_NO_HOST_MEMORY(c)

hc_status hc_qcache_workspace(hc_ctx *c, const hc_qcache *k, const hc_qcache_attention_args *p,
                              int64_t *bytes) {
  if (!c) return HC_E_INVAL;
  if (!bytes) return fail(c, HC_E_INVAL, "bytes is NULL");
  SeqArgs a;
  bool few_rows;
  const hc_status st = cached_plan(c, k, p, a, few_rows);
  if (st != HC_OK) return st;
  *bytes = part_bytes(a, k->head_dim, few_rows ? kDecodeRows : kSeqRows);
  return HC_OK;
}

hc_status hc_qcache_attention(hc_ctx *c, const hc_qcache *k, const hc_qcache_attention_args *p,
                              hc_stream stream) try {
  if (!c) return HC_E_INVAL;
  SeqArgs a;
  bool few_rows;
  hc_status st = check_cache(c, k, true);
  if (st == HC_OK) st = cached_plan(c, k, p, a, few_rows);
  if (st != HC_OK) return st;
  if (p->n_tokens == 0) return HC_OK;
  st = check_tensor(c, {"q", p->q, p->q_token, p->q_head, p->n_tokens, p->n_heads});
  if (st == HC_OK) st = check_output(c, {"out", p->out, p->out_token, p->out_head, p->n_tokens, p->n_heads}, k->head_dim);
  if (st != HC_OK) return st;
  if (!p->kv_len || !aligned4(p->kv_len)) return fail(c, HC_E_INVAL, "kv_len must be a 4-byte aligned device pointer");
  if ((st = check_workspace(c, p->workspace, p->workspace_bytes,
                            part_bytes(a, k->head_dim, few_rows ? kDecodeRows : kSeqRows))) != HC_OK)
    return st;
  if (a.n_split > 1) use_workspace(a, p->workspace);
  OnDevice on(c->device);
  HC_HIP(c, on.status);
  return run_seq(c, a, k->head_dim, few_rows, (hipStream_t)stream);
} HC_NO_HOST_MEMORY(c)

}  // extern "C"
