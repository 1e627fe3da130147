// operators.cu -- host side of the operators on pages and state slots: argument
// checks, kernel parameters and launches.  Each entry checks everything it can
// before it enqueues anything, enqueues on the caller's stream only, and
// allocates nothing.

#include <algorithm>
#include <cmath>
#include <initializer_list>
#include <string.h>
#include <utility>

#include "operators.cuh"

using namespace kvx;

namespace {

constexpr int32_t kMaxSeqs = 65535, kMaxHeads = 4096;
constexpr int64_t kMaxRows = 1ll << 30;

kvx_status refuse(kvx_status st, const char* why) {
  set_error_text(why);
  return st;
}

// Bytes from the first to behind the last element of [n][strides] x [inner] elements.
bool extent(int64_t n0, int64_t s0, int64_t n1, int64_t s1, int64_t inner, int64_t size, int64_t* bytes) {
  if (n0 < 1 || n1 < 1 || s0 < 0 || s1 < 0) return false;
  const __int128 e = ((__int128)(n0 - 1) * s0 + (__int128)(n1 - 1) * s1 + inner) * size;
  if (e > INT64_MAX / 2) return false;
  *bytes = (int64_t)e;
  return true;
}

// Rows of `inner` elements that are written must not lie over one another: every dimension (its size and stride) has to
// step over all that those of smaller strides take.  At most three; extents are checked before.
bool disjoint(std::initializer_list<std::pair<int64_t, int64_t>> dims, int64_t inner) {
  std::pair<int64_t, int64_t> by_stride[3];
  int n = 0;
  for (const auto& d : dims)
    if (d.first > 1) by_stride[n++] = {d.second, d.first};
  std::sort(by_stride, by_stride + n);
  for (int i = 0; i < n; ++i) {
    if (by_stride[i].first < inner) return false;
    inner += (by_stride[i].second - 1) * by_stride[i].first;
  }
  return true;
}

bool vectors(const void* p, int64_t s0, int64_t s1) {  // 16-byte vectors of 2-byte elements
  return ((uintptr_t)p & 15) == 0 && s0 % 8 == 0 && s1 % 8 == 0;
}

struct Rows {  // a tensor of rows that a call reads or writes
  const void* p;
  int64_t n0, s0, n1, s1, inner;
  const char* what;
};

kvx_status check_rows(DeviceMemory& mem, const Rows& r, bool written) {
  int64_t bytes;
  if (!r.p) return refuse(KVX_EINVAL, r.what);
  if (!extent(r.n0, r.s0, r.n1, r.s1, r.inner, 2, &bytes)) return refuse(KVX_EINVAL, r.what);
  if (!vectors(r.p, r.n0 > 1 ? r.s0 : 0, r.n1 > 1 ? r.s1 : 0)) return refuse(KVX_EALIGN, r.what);
  if (written && !disjoint({{r.n0, r.s0}, {r.n1, r.s1}}, r.inner)) return refuse(KVX_EINVAL, r.what);
  const kvx_status st = mem.check(r.p, bytes);
  return st == KVX_OK ? st : refuse(st, r.what);
}

// n 4-byte values, 4-byte aligned.
kvx_status check_words(DeviceMemory& mem, const void* p, int64_t n, const char* what) {
  if (!p) return refuse(KVX_EINVAL, what);
  if ((uintptr_t)p & 3) return refuse(KVX_EALIGN, what);
  const kvx_status st = n > 0 ? mem.check(p, n * 4) : KVX_OK;
  return st == KVX_OK ? st : refuse(st, what);
}

bool check_types(int32_t type, int32_t cache_type, int32_t elem_bytes) {
  if (type != KVX_TYPE_BF16 && type != KVX_TYPE_FP16) return false;
  if (cache_type == KVX_TYPE_E4M3) return elem_bytes == 1;
  return cache_type == type && elem_bytes == 2;
}

// Checks what needs no device and fills the view but for its layer.
kvx_status view_pages(const CtxView& ctx, const kvx_pool* pool, const kvx_batch* b, Geometry* g, PagesView* v) {
  kvx_status st = check_shape(pool, g);
  if (st != KVX_OK) return refuse(st, "pool description");
  if (b->num_seqs < 0 || b->num_seqs > kMaxSeqs) return refuse(KVX_EINVAL, "num_seqs");
  if (pool->num_heads > kMaxHeads || pool->head_dim > 256) return refuse(KVX_EINVAL, "heads or head_dim");
  if (b->table_len < 1 || (b->num_seqs > 1 && b->table_stride < b->table_len))
    return refuse(KVX_EINVAL, "table_len or table_stride");
  const int64_t pack = pool->pages_per_block > 1 ? pool->pages_per_block : 1;
  if (b->table_len > INT32_MAX) return refuse(KVX_EINVAL, "table_len");
  const __int128 room = (__int128)b->table_len * pool->block_tokens * pack;
  const int64_t all = (int64_t)std::min<__int128>(room, (1ll << 30));
  if (b->max_length < 0 || b->max_length > room) return refuse(KVX_ERANGE, "max_length is more than the tables hold");
  const int64_t longest = b->max_length ? b->max_length : all;
  if (longest > (1ll << 30)) return refuse(KVX_EINVAL, "max_length");
  v->base = nullptr;
  v->tables = b->block_tables;
  v->lengths = b->lengths;
  v->err = ctx.err;
  v->table_stride = b->table_stride;
  v->half_bytes = g->page_bytes / 2;
  const bool hnd = pool->layout == KVX_LAYOUT_HND;
  // rows are counted in 32 bits (of which the last number means none)
  if (g->layer_bytes / g->row >= (1ll << 32) - 1) return refuse(KVX_ERANGE, "a layer of 2^32 rows or more");
  v->row_bytes = g->row;
  v->page_rows = (uint32_t)(g->page_bytes / g->row);
  v->token_rows = hnd ? 1 : (uint32_t)pool->num_heads;
  v->head_bytes = hnd ? g->row * pool->block_tokens : g->row;
  v->by_block = div31((uint32_t)pool->block_tokens);
  v->by_pack = div31((uint32_t)pack);
  v->entries = (uint32_t)std::min<int64_t>(pool->num_blocks / pack, INT32_MAX);
  v->table_len = (uint32_t)b->table_len;
  v->heads = pool->num_heads;
  v->head_dim = pool->head_dim;
  v->num_seqs = b->num_seqs;
  v->max_length = (int32_t)longest;
  return KVX_OK;
}

kvx_status check_tables(DeviceMemory& mem, const int32_t* p, int64_t n, int64_t stride, int64_t len, const char* what) {
  int64_t bytes;
  if (!extent(n, n > 1 ? stride : 0, 1, 0, len, 4, &bytes)) return refuse(KVX_EINVAL, what);
  return check_words(mem, p, bytes / 4, what);
}

kvx_status check_batch_memory(DeviceMemory& mem, const kvx_batch* b) {
  kvx_status st = check_tables(mem, b->block_tables, b->num_seqs, b->table_stride, b->table_len, "block_tables");
  return st != KVX_OK ? st : check_words(mem, b->lengths, b->num_seqs, "lengths");
}

kvx_status layer_of(DeviceMemory& mem, const kvx_pool* pool, int32_t layer, const Geometry& g, uint8_t** base) {
  if (layer < 0 || layer >= pool->num_layers) return refuse(KVX_ERANGE, "layer");
  uint8_t* p = (uint8_t*)pool->layer_base[layer];
  if (!p) return refuse(KVX_EINVAL, "layer_base");
  if ((uintptr_t)p & 15) return refuse(KVX_EALIGN, "layer_base");
  const kvx_status st = mem.check(p, g.layer_bytes);
  if (st != KVX_OK) return refuse(st, "layer_base");
  *base = p;
  return KVX_OK;
}

kvx_status launched(kvx_ctx* ctx, cudaError_t e, const char* what, int line, int n) {
  if (e != cudaSuccess) {
    record_cuda_error((int)e, what, line);
    return KVX_ECUDA;
  }
  count_launches(ctx, n);
  return KVX_OK;
}
#define KVX_LAUNCHED(ctx, call, n) launched(ctx, fault_point("launch") ? cudaErrorUnknown : call, #call, __LINE__, n)

kvx_status view_state(const CtxView& ctx, const kvx_state* s, const kvx_state_batch* b, int64_t offset, int64_t bytes,
                      DeviceMemory& mem, StateView* v) {
  if (s->num_slots < 1 || s->slot_bytes < 16) return refuse(KVX_EINVAL, "num_slots or slot_bytes");
  if (s->num_slots > INT32_MAX || s->slot_bytes > INT64_MAX / 2 / s->num_slots)
    return refuse(KVX_EINVAL, "num_slots or slot_bytes");
  if (offset < 0) return refuse(KVX_EINVAL, "offset in the slot");
  if (s->slot_bytes % 16 || offset % 16 || ((uintptr_t)s->base & 15)) return refuse(KVX_EALIGN, "state slots");
  if (offset > s->slot_bytes || bytes > s->slot_bytes - offset) return refuse(KVX_ERANGE, "the state does not fit its slot");
  if (b->tokens > INT32_MAX || (!b->starts && b->tokens != b->num_seqs)) return refuse(KVX_EINVAL, "tokens");
  kvx_status st = mem.check(s->base, s->num_slots * s->slot_bytes);
  if (st != KVX_OK) return refuse(st, "state slots");
  if ((st = check_words(mem, b->slots_in, b->num_seqs, "slots_in")) != KVX_OK) return st;
  if ((st = check_words(mem, b->slots_out, b->num_seqs, "slots_out")) != KVX_OK) return st;
  if (b->fresh && (st = check_words(mem, b->fresh, b->num_seqs, "fresh")) != KVX_OK) return st;
  if (b->starts && (st = check_words(mem, b->starts, b->num_seqs + 1, "starts")) != KVX_OK) return st;
  *v = {(uint8_t*)s->base, b->slots_in, b->slots_out, b->fresh, b->starts, ctx.err,
        s->num_slots, s->slot_bytes, offset, b->tokens, b->num_seqs};
  return KVX_OK;
}

// kv_attend's workspace.  The most CTAs a launch has are two an SM.
struct AttendSpace {
  int64_t items, parts, row_lse2, scores, bytes;  // offsets, and all of it
  int64_t score_stride;
  int32_t score_rows;
};
AttendSpace attend_space(const CtxView& ctx, const PagesView& v, const kvx_attention* a) {
  auto up = [](int64_t n) { return (n + 255) / 256 * 256; };
  const int64_t rows = (int64_t)a->q_heads / v.heads * a->new_tokens;
  const int64_t block = 8 * attend_tiles(v.head_dim, (int32_t)rows);
  const int64_t items = (int64_t)v.num_seqs * v.heads * ((rows + block - 1) / block);
  AttendSpace w;
  w.items = 0;
  w.parts = up(items * 8);
  w.row_lse2 = w.parts + up((int64_t)ctx.num_sms * 2 * 2 * block * (attend_pad(v.head_dim) + 2) * 4);
  w.scores = w.row_lse2;
  w.bytes = w.row_lse2;
  w.score_stride = ((int64_t)v.max_length + 47) / 16 * 16;  // steps of 32 keys may begin at any multiple of 16
  w.score_rows = (int32_t)((rows + 1) / 2 * 2);
  if (a->weights) {
    w.scores += up((int64_t)v.num_seqs * v.heads * rows * 4);
    w.bytes = w.scores + up((int64_t)v.num_seqs * v.heads * w.score_rows * w.score_stride * 4);
  }
  return w;
}

// Checks of an attention that need no device.
kvx_status check_attention(const kvx_pool* pool, const kvx_batch* batch, const kvx_attention* a) {
  if (!check_types(a->type, a->cache_type, pool->elem_bytes)) return refuse(KVX_EINVAL, "type, cache_type or elem_bytes");
  if (a->q_heads < 1 || a->q_heads > kMaxHeads || a->q_heads % pool->num_heads)
    return refuse(KVX_EINVAL, "q_heads is no multiple of the pool's heads");
  if (a->new_tokens < 1 || a->new_tokens > KVX_ATTEND_MAX_NEW_TOKENS) return refuse(KVX_EINVAL, "new_tokens");
  if (!std::isfinite(a->scale) || !(a->softcap >= 0.f) || !std::isfinite(a->softcap) || !std::isfinite(a->k_scale) ||
      !std::isfinite(a->v_scale) || a->window < 0)
    return refuse(KVX_EINVAL, "scale, softcap or window");
  if ((int64_t)batch->num_seqs * a->new_tokens * a->q_heads > kMaxRows)  // a CTA each where parts are joined
    return refuse(KVX_ERANGE, "more than 2^30 rows of queries");
  return KVX_OK;
}

// Over selected pages: what an attention may not have there.
kvx_status check_selected(const kvx_attention* a, int32_t budget) {
  if (budget < 1 || budget > kMaxRows) return refuse(KVX_EINVAL, "budget");
  if (a->window || a->slopes || a->weights) return refuse(KVX_EINVAL, "window, slopes or weights over selected pages");
  return KVX_OK;
}

bool check_cache_type(int32_t type, int32_t elem_bytes) {
  return type == KVX_TYPE_E4M3 ? elem_bytes == 1 : (type == KVX_TYPE_BF16 || type == KVX_TYPE_FP16) && elem_bytes == 2;
}

int64_t most_pages(const kvx_pool* pool, const PagesView& v) {
  return ((int64_t)v.max_length + pool->block_tokens - 1) / pool->block_tokens;
}

kvx_status check_selection(const kvx_pool* pool, const kvx_batch* batch, const PagesView& v, const kvx_selection* s) {
  if (s->type != KVX_TYPE_BF16 && s->type != KVX_TYPE_FP16) return refuse(KVX_EINVAL, "type");
  if (s->q_heads < 1 || s->q_heads > kMaxHeads || s->q_heads % pool->num_heads)
    return refuse(KVX_EINVAL, "q_heads is no multiple of the pool's heads");
  if (s->q_heads / pool->num_heads > kMaxScoreGroup) return refuse(KVX_EINVAL, "more than 128 query heads a KV head");
  if (s->new_tokens < 1 || s->new_tokens > KVX_ATTEND_MAX_NEW_TOKENS) return refuse(KVX_EINVAL, "new_tokens");
  if (s->budget < 1 || s->budget > kMaxRows || s->sinks < 0 || s->recent < 1 || (int64_t)s->sinks + s->recent > s->budget)
    return refuse(KVX_EINVAL, "budget, sinks or recent");
  const int64_t tokens = (int64_t)batch->num_seqs * s->new_tokens;
  if (tokens * s->q_heads > kMaxRows) return refuse(KVX_ERANGE, "more than 2^30 rows of queries");
  // a CTA a tile of pages and part of the new tokens, whatever its size
  if ((int64_t)batch->num_seqs * s->new_tokens * ((most_pages(pool, v) + kScorePages - 1) / kScorePages) > kMaxRows)
    return refuse(KVX_ERANGE, "more than 2^30 tiles of pages");
  return KVX_OK;
}

// kv_select's workspace: the scores, where there are more pages than are picked.
int64_t select_bytes(const kvx_pool* pool, const kvx_batch* batch, const PagesView& v, const kvx_selection* s) {
  const int64_t pages = most_pages(pool, v);
  return pages > s->budget ? (int64_t)batch->num_seqs * s->new_tokens * pool->num_heads * pages * 4 : 0;
}

kvx_status check_bounds(DeviceMemory& mem, const kvx_pool* pool, const kvx_bounds* b) {
  const int64_t rows = pool->num_blocks * (int64_t)pool->num_heads;
  if (!b->boxes) return refuse(KVX_EINVAL, "boxes");
  if ((uintptr_t)b->boxes & 15) return refuse(KVX_EALIGN, "boxes");
  const kvx_status st = mem.check(b->boxes, rows * 2 * pool->head_dim);
  return st != KVX_OK ? refuse(st, "boxes") : check_words(mem, b->sizes, rows, "sizes");
}

// What kv_append and kv_append_rotary check alike, in two parts: what needs no device, and the memory.
kvx_status view_append(const CtxView& ctx, const kvx_pool* pool, const kvx_batch* batch, const kvx_new_rows* rows, Geometry* g,
                       AppendParams* p) {
  kvx_status st = view_pages(ctx, pool, batch, g, &p->pages);
  if (st != KVX_OK) return st;
  if (!check_types(rows->type, rows->cache_type, pool->elem_bytes))
    return refuse(KVX_EINVAL, "type, cache_type or elem_bytes");
  if (rows->tokens < 0 || rows->tokens > INT32_MAX) return refuse(KVX_EINVAL, "tokens");
  if (!rows->starts && (rows->new_tokens < 1 || rows->tokens != (int64_t)rows->new_tokens * batch->num_seqs))
    return refuse(KVX_EINVAL, "tokens is not new_tokens of every sequence");
  for (float scale : {rows->k_scale, rows->v_scale})  // a subnormal one has no reciprocal: its zeros would be NaN
    if (!(scale == 0.f || (std::isnormal(scale) && scale > 0.f))) return refuse(KVX_EINVAL, "k_scale or v_scale");
  return KVX_OK;
}

kvx_status fill_append(DeviceMemory& mem, const kvx_pool* pool, int32_t layer, const kvx_batch* batch, const kvx_new_rows* rows,
                       const void* key, const void* value, const Geometry& g, AppendParams* p) {
  kvx_status st;
  if ((st = layer_of(mem, pool, layer, g, &p->pages.base)) != KVX_OK) return st;
  if ((st = check_batch_memory(mem, batch)) != KVX_OK) return st;
  if (rows->starts && (st = check_words(mem, rows->starts, batch->num_seqs + 1, "starts")) != KVX_OK) return st;
  const int64_t h = pool->num_heads, d = pool->head_dim;
  if ((st = check_rows(mem, {key, rows->tokens, rows->key_token_stride, h, rows->key_head_stride, d, "key"}, false)) != KVX_OK ||
      (st = check_rows(mem, {value, rows->tokens, rows->value_token_stride, h, rows->value_head_stride, d, "value"},
                       false)) != KVX_OK)
    return st;
  p->key = (const uint8_t*)key;
  p->value = (const uint8_t*)value;
  p->starts = rows->starts;
  p->tokens = rows->tokens;
  p->key_token = 2 * rows->key_token_stride;
  p->key_head = 2 * rows->key_head_stride;
  p->value_token = 2 * rows->value_token_stride;
  p->value_head = 2 * rows->value_head_stride;
  p->new_tokens = rows->new_tokens;
  p->num_seqs = batch->num_seqs;
  p->row_vecs = div31((uint32_t)(g.row / 16));
  p->k_scale = rows->k_scale ? rows->k_scale : 1.f;
  p->v_scale = rows->v_scale ? rows->v_scale : 1.f;
  return KVX_OK;
}

}  // namespace

kvx_status kv_append(kvx_ctx* c, const kvx_pool* pool, int32_t layer, const kvx_batch* batch, const kvx_new_rows* rows,
                     const void* key, const void* value, kvx_stream_t stream) {
  return guarded([&]() -> kvx_status {
    if (!c || !pool || !batch || !rows) return KVX_EINVAL;
    const CtxView ctx = view_of(c);
    AppendParams p;
    Geometry g;
    kvx_status st = view_append(ctx, pool, batch, rows, &g, &p);
    if (st != KVX_OK) return st;
    CurrentDevice guard(ctx.device);
    if (!guard.ok) return KVX_ECUDA;
    if ((st = check_stream(stream, ctx.device)) != KVX_OK) return refuse(st, "stream");
    if (rows->tokens == 0 || batch->num_seqs == 0) return KVX_OK;
    DeviceMemory mem(ctx.device);
    if ((st = fill_append(mem, pool, layer, batch, rows, key, value, g, &p)) != KVX_OK) return st;
    return KVX_LAUNCHED(c, launch_append(p, rows->type, rows->cache_type, ctx.num_sms, stream), 1);
  });
}

kvx_status kv_append_rotary(kvx_ctx* c, const kvx_pool* pool, int32_t layer, const kvx_batch* batch, const kvx_new_rows* rows,
                            const kvx_rotary* r, const void* q, const void* key, const void* value, void* q_out,
                            kvx_stream_t stream) {
  return guarded([&]() -> kvx_status {
    if (!c || !pool || !batch || !rows || !r) return KVX_EINVAL;
    const CtxView ctx = view_of(c);
    RotaryParams p;
    Geometry g;
    kvx_status st = view_append(ctx, pool, batch, rows, &g, &p.append);
    if (st != KVX_OK) return st;
    if (r->q_heads < 1 || r->q_heads > kMaxHeads) return refuse(KVX_EINVAL, "q_heads");
    if (r->rotary_dim < 0 || r->rotary_dim % 2 || r->rotary_dim > pool->head_dim) return refuse(KVX_EINVAL, "rotary_dim");
    if (!std::isfinite(r->rotary_scale) || !std::isfinite(r->eps) || r->eps < 0.f || !std::isfinite(r->weight_offset))
      return refuse(KVX_EINVAL, "rotary_scale, eps or weight_offset");
    CurrentDevice guard(ctx.device);
    if (!guard.ok) return KVX_ECUDA;
    if ((st = check_stream(stream, ctx.device)) != KVX_OK) return refuse(st, "stream");
    if (rows->tokens == 0 || batch->num_seqs == 0) return KVX_OK;
    DeviceMemory mem(ctx.device);
    if ((st = fill_append(mem, pool, layer, batch, rows, key, value, g, &p.append)) != KVX_OK) return st;
    const int64_t d = pool->head_dim, n = rows->tokens, hq = r->q_heads;
    if ((st = check_rows(mem, {q, n, r->q_token_stride, hq, r->q_head_stride, d, "q"}, false)) != KVX_OK ||
        (st = check_rows(mem, {q_out, n, r->out_token_stride, hq, r->out_head_stride, d, "q_out"}, true)) != KVX_OK)
      return st;
    if (q_out == q && ((n > 1 && r->q_token_stride != r->out_token_stride) || (hq > 1 && r->q_head_stride != r->out_head_stride)))
      return refuse(KVX_EINVAL, "q_out is q, with other strides");
    if (r->rotary_dim > 0 && (st = check_words(mem, r->inv_freq, r->rotary_dim / 2, "inv_freq")) != KVX_OK) return st;
    if (r->positions && (st = check_words(mem, r->positions, n, "positions")) != KVX_OK) return st;
    if (r->q_weight && (st = check_rows(mem, {r->q_weight, 1, 0, 1, 0, d, "q_weight"}, false)) != KVX_OK) return st;
    if (r->k_weight && (st = check_rows(mem, {r->k_weight, 1, 0, 1, 0, d, "k_weight"}, false)) != KVX_OK) return st;
    p.q = (const uint8_t*)q;
    p.q_out = (uint8_t*)q_out;
    p.q_weight = (const uint8_t*)r->q_weight;
    p.k_weight = (const uint8_t*)r->k_weight;
    p.inv_freq = r->inv_freq;
    p.positions = r->positions;
    p.q_token = 2 * r->q_token_stride;
    p.q_head = 2 * r->q_head_stride;
    p.out_token = 2 * r->out_token_stride;
    p.out_head = 2 * r->out_head_stride;
    p.q_heads = r->q_heads;
    p.rotary_dim = r->rotary_dim;
    p.interleaved = r->interleaved;
    p.rotary_scale = r->rotary_scale ? r->rotary_scale : 1.f;
    p.eps = r->eps;
    p.weight_offset = r->weight_offset;
    return KVX_LAUNCHED(c, launch_rotary(p, rows->type, rows->cache_type, ctx.num_sms, stream), 1);
  });
}

kvx_status kv_attend_workspace(kvx_ctx* c, const kvx_pool* pool, const kvx_batch* batch, const kvx_attention* a,
                               int64_t* bytes) {
  return guarded([&]() -> kvx_status {
    if (!c || !pool || !batch || !a || !bytes) return KVX_EINVAL;
    Geometry g;
    PagesView v;
    kvx_status st = view_pages(view_of(c), pool, batch, &g, &v);
    if (st == KVX_OK) st = check_attention(pool, batch, a);
    if (st != KVX_OK) return st;
    *bytes = attend_space(view_of(c), v, a).bytes;
    return KVX_OK;
  });
}

namespace {

// Attention over all pages, or over those selected ones alone.
kvx_status attend(kvx_ctx* c, const kvx_pool* pool, int32_t layer, const kvx_batch* batch, const kvx_attention* a, bool some,
                  int32_t budget, const int32_t* selected, const void* q, void* out, void* workspace, int64_t workspace_bytes,
                  kvx_stream_t stream) {
  const CtxView ctx = view_of(c);
  AttendParams p;
  Geometry g;
  kvx_status st = view_pages(ctx, pool, batch, &g, &p.pages);
  if (st == KVX_OK) st = check_attention(pool, batch, a);
  if (st == KVX_OK && some) st = check_selected(a, budget);
  if (st != KVX_OK) return st;
  CurrentDevice guard(ctx.device);
  if (!guard.ok) return KVX_ECUDA;
  if ((st = check_stream(stream, ctx.device)) != KVX_OK) return refuse(st, "stream");
  if (batch->num_seqs == 0) return KVX_OK;
  DeviceMemory mem(ctx.device);
  if ((st = layer_of(mem, pool, layer, g, &p.pages.base)) != KVX_OK) return st;
  if ((st = check_batch_memory(mem, batch)) != KVX_OK) return st;
  const int64_t tokens = (int64_t)batch->num_seqs * a->new_tokens, d = pool->head_dim;
  if ((st = check_rows(mem, {q, tokens, a->q_token_stride, a->q_heads, a->q_head_stride, d, "q"}, false)) != KVX_OK ||
      (st = check_rows(mem, {out, tokens, a->out_token_stride, a->q_heads, a->out_head_stride, d, "out"}, true)) != KVX_OK)
    return st;
  if (a->slopes && (st = check_words(mem, a->slopes, a->q_heads, "slopes")) != KVX_OK) return st;
  if (a->lse && (st = check_words(mem, a->lse, tokens * a->q_heads, "lse")) != KVX_OK) return st;
  if (a->weights) {
    int64_t bytes;
    if (!extent(batch->num_seqs, a->weights_seq_stride, pool->num_heads, a->weights_head_stride, p.pages.max_length, 4,
                  &bytes) ||
        !disjoint({{batch->num_seqs, a->weights_seq_stride}, {pool->num_heads, a->weights_head_stride}}, p.pages.max_length))
      return refuse(KVX_EINVAL, "strides of weights");
    if ((st = check_words(mem, a->weights, bytes / 4, "weights")) != KVX_OK) return st;
  }
  if (some && (st = check_words(mem, selected, tokens * pool->num_heads * budget, "selected")) != KVX_OK) return st;
  // over selected pages a query is a sequence of its own
  kvx_attention each = *a;
  if (some) p.pages.num_seqs = (int32_t)tokens, each.new_tokens = 1;
  const AttendSpace space = attend_space(ctx, p.pages, &each);
  if (workspace_bytes < space.bytes)
    return refuse(KVX_ERANGE, some ? "workspace is smaller than kv_attend_selected_workspace says"
                                   : "workspace is smaller than kv_attend_workspace says");
  if (!workspace || ((uintptr_t)workspace & 15)) return refuse(workspace ? KVX_EALIGN : KVX_EINVAL, "workspace");
  if ((st = mem.check(workspace, space.bytes)) != KVX_OK) return refuse(st, "workspace");
  uint8_t* ws = (uint8_t*)workspace;
  p.items = (int2*)(ws + space.items);
  p.parts = (float*)(ws + space.parts);
  p.row_lse2 = (float*)(ws + space.row_lse2);
  p.scores = (float*)(ws + space.scores);
  p.score_stride = space.score_stride;
  p.score_rows = space.score_rows;
  p.q = (const uint8_t*)q;
  p.out = (uint8_t*)out;
  p.lse = a->lse;
  p.weights = a->weights;
  p.slopes = a->slopes;
  p.q_token = 2 * a->q_token_stride;
  p.q_head = 2 * a->q_head_stride;
  p.out_token = 2 * a->out_token_stride;
  p.out_head = 2 * a->out_head_stride;
  p.weights_seq = a->weights_seq_stride;
  p.weights_head = a->weights_head_stride;
  p.q_heads = a->q_heads;
  p.group = a->q_heads / pool->num_heads;
  p.new_tokens = each.new_tokens;
  p.selected = some ? selected : nullptr;
  p.budget = budget;
  p.by_query = div31((uint32_t)a->new_tokens);
  // one that reaches past every key is none; smaller ones leave the kernels' 32-bit positions room
  p.window = a->window < p.pages.max_length ? a->window : 0;
  p.scale = a->scale ? a->scale : 1.f / std::sqrt((float)d);
  p.softcap = a->softcap;
  const bool e4m3 = a->cache_type == KVX_TYPE_E4M3;
  p.k_scale = e4m3 && a->k_scale ? a->k_scale : 1.f;
  p.v_scale = e4m3 && a->v_scale ? a->v_scale : 1.f;
  p.type = a->type;
  const int32_t rows = p.group * p.new_tokens, block = 8 * attend_tiles(p.pages.head_dim, rows);
  const int64_t blocks = (rows + block - 1) / block;
  p.part_rows = block;
  p.part_dim = attend_pad(p.pages.head_dim);
  const int32_t step = 16 * attend_blocks(p.part_dim, pool->elem_bytes, block / 8);
  int64_t longest = p.pages.max_length;
  if (some) longest = std::min<int64_t>(longest + pool->block_tokens - 1, (int64_t)budget * pool->block_tokens);
  p.most_steps = (int64_t)p.pages.num_seqs * p.pages.heads * blocks * ((longest + step - 1) / step + kItemSteps);
  p.min_steps = 6;  // one sequence of 1.8k tokens, 8 heads: 12.6 us, as with 3, and 14.5 with 12
  return KVX_LAUNCHED(c, launch_attend(p, a->cache_type, ctx.num_sms, stream), 2);
}

}  // namespace

kvx_status kv_attend(kvx_ctx* c, const kvx_pool* pool, int32_t layer, const kvx_batch* batch, const kvx_attention* a,
                     const void* q, void* out, void* workspace, int64_t workspace_bytes, kvx_stream_t stream) {
  return guarded([&]() -> kvx_status {
    if (!c || !pool || !batch || !a) return KVX_EINVAL;
    return attend(c, pool, layer, batch, a, false, 0, nullptr, q, out, workspace, workspace_bytes, stream);
  });
}

kvx_status kv_attend_selected_workspace(kvx_ctx* c, const kvx_pool* pool, const kvx_batch* batch, const kvx_attention* a,
                                        int32_t budget, int64_t* bytes) {
  return guarded([&]() -> kvx_status {
    if (!c || !pool || !batch || !a || !bytes) return KVX_EINVAL;
    Geometry g;
    PagesView v;
    kvx_status st = view_pages(view_of(c), pool, batch, &g, &v);
    if (st == KVX_OK) st = check_attention(pool, batch, a);
    if (st == KVX_OK) st = check_selected(a, budget);
    if (st != KVX_OK) return st;
    kvx_attention each = *a;
    v.num_seqs *= a->new_tokens;
    each.new_tokens = 1;
    *bytes = attend_space(view_of(c), v, &each).bytes;
    return KVX_OK;
  });
}

kvx_status kv_attend_selected(kvx_ctx* c, const kvx_pool* pool, int32_t layer, const kvx_batch* batch, const kvx_attention* a,
                              int32_t budget, const int32_t* selected, const void* q, void* out, void* workspace,
                              int64_t workspace_bytes, kvx_stream_t stream) {
  return guarded([&]() -> kvx_status {
    if (!c || !pool || !batch || !a) return KVX_EINVAL;
    return attend(c, pool, layer, batch, a, true, budget, selected, q, out, workspace, workspace_bytes, stream);
  });
}

kvx_status kv_bounds(kvx_ctx* c, const kvx_pool* pool, int32_t layer, const kvx_batch* batch, int32_t cache_type,
                     int64_t new_tokens, const kvx_bounds* bounds, kvx_stream_t stream) {
  return guarded([&]() -> kvx_status {
    if (!c || !pool || !batch || !bounds) return KVX_EINVAL;
    const CtxView ctx = view_of(c);
    BoundsParams p;
    Geometry g;
    kvx_status st = view_pages(ctx, pool, batch, &g, &p.pages);
    if (st != KVX_OK) return st;
    if (!check_cache_type(cache_type, pool->elem_bytes)) return refuse(KVX_EINVAL, "cache_type or elem_bytes");
    if (new_tokens < 1) return refuse(KVX_EINVAL, "new_tokens");
    CurrentDevice guard(ctx.device);
    if (!guard.ok) return KVX_ECUDA;
    if ((st = check_stream(stream, ctx.device)) != KVX_OK) return refuse(st, "stream");
    if (batch->num_seqs == 0) return KVX_OK;
    p.new_tokens = (int32_t)std::min<int64_t>(new_tokens, p.pages.max_length);
    const int64_t block = pool->block_tokens, most = (p.pages.max_length + block - 1) / block;
    p.pages_each = (int32_t)std::min(most, (p.new_tokens + block - 2) / block + 1);
    if ((int64_t)batch->num_seqs * p.pages_each * pool->num_heads > kMaxRows) return refuse(KVX_ERANGE, "more than 2^30 pages and heads");
    DeviceMemory mem(ctx.device);
    if ((st = layer_of(mem, pool, layer, g, &p.pages.base)) != KVX_OK) return st;
    if ((st = check_batch_memory(mem, batch)) != KVX_OK) return st;
    if ((st = check_bounds(mem, pool, bounds)) != KVX_OK) return st;
    p.boxes = bounds->boxes;
    p.sizes = bounds->sizes;
    p.by_heads = div31((uint32_t)pool->num_heads);
    return KVX_LAUNCHED(c, launch_bounds(p, cache_type, stream), 1);
  });
}

kvx_status kv_select_workspace(kvx_ctx* c, const kvx_pool* pool, const kvx_batch* batch, const kvx_selection* sel, int64_t* bytes) {
  return guarded([&]() -> kvx_status {
    if (!c || !pool || !batch || !sel || !bytes) return KVX_EINVAL;
    Geometry g;
    PagesView v;
    kvx_status st = view_pages(view_of(c), pool, batch, &g, &v);
    if (st == KVX_OK) st = check_selection(pool, batch, v, sel);
    if (st != KVX_OK) return st;
    *bytes = select_bytes(pool, batch, v, sel);
    return KVX_OK;
  });
}

kvx_status kv_select(kvx_ctx* c, const kvx_pool* pool, const kvx_batch* batch, const kvx_bounds* bounds, const kvx_selection* sel,
                     const void* q, int32_t* selected, void* workspace, int64_t workspace_bytes, kvx_stream_t stream) {
  return guarded([&]() -> kvx_status {
    if (!c || !pool || !batch || !bounds || !sel) return KVX_EINVAL;
    const CtxView ctx = view_of(c);
    SelectParams p;
    Geometry g;
    kvx_status st = view_pages(ctx, pool, batch, &g, &p.pages);
    if (st == KVX_OK) st = check_selection(pool, batch, p.pages, sel);
    if (st != KVX_OK) return st;
    CurrentDevice guard(ctx.device);
    if (!guard.ok) return KVX_ECUDA;
    if ((st = check_stream(stream, ctx.device)) != KVX_OK) return refuse(st, "stream");
    if (batch->num_seqs == 0) return KVX_OK;
    DeviceMemory mem(ctx.device);
    if ((st = check_batch_memory(mem, batch)) != KVX_OK) return st;
    if ((st = check_bounds(mem, pool, bounds)) != KVX_OK) return st;
    const int64_t tokens = (int64_t)batch->num_seqs * sel->new_tokens;
    if ((st = check_rows(mem, {q, tokens, sel->q_token_stride, sel->q_heads, sel->q_head_stride, pool->head_dim, "q"}, false)) != KVX_OK)
      return st;
    if ((st = check_words(mem, selected, tokens * pool->num_heads * sel->budget, "selected")) != KVX_OK) return st;
    const int64_t bytes = select_bytes(pool, batch, p.pages, sel);
    if (bytes > 0) {
      if (workspace_bytes < bytes) return refuse(KVX_ERANGE, "workspace is smaller than kv_select_workspace says");
      if (!workspace || ((uintptr_t)workspace & 15)) return refuse(workspace ? KVX_EALIGN : KVX_EINVAL, "workspace");
      if ((st = mem.check(workspace, bytes)) != KVX_OK) return refuse(st, "workspace");
    }
    p.boxes = bounds->boxes;
    p.sizes = bounds->sizes;
    p.q = (const uint8_t*)q;
    p.selected = selected;
    p.q_token = 2 * sel->q_token_stride;
    p.q_head = 2 * sel->q_head_stride;
    p.q_heads = sel->q_heads;
    p.group = sel->q_heads / pool->num_heads;
    p.new_tokens = sel->new_tokens;
    p.budget = sel->budget;
    p.sinks = sel->sinks;
    p.recent = sel->recent;
    p.scores = (float*)workspace;
    p.score_stride = most_pages(pool, p.pages);
    p.tokens_each = score_tokens(p.group, p.new_tokens);
    p.score_tiles = bytes > 0 ? (int32_t)((p.score_stride + kScorePages - 1) / kScorePages) : 0;
    p.score_parts = (p.new_tokens + p.tokens_each - 1) / p.tokens_each;
    return KVX_LAUNCHED(c, launch_select(p, sel->type, stream), 1 + (p.score_tiles > 0));
  });
}

kvx_status kv_evict(kvx_ctx* c, const kvx_pool* pool, const kvx_batch* batch, const kvx_eviction* e,
                    kvx_stream_t stream) {
  return guarded([&]() -> kvx_status {
    if (!c || !pool || !batch || !e) return KVX_EINVAL;
    const CtxView ctx = view_of(c);
    EvictParams p;
    Geometry g;
    kvx_status st = view_pages(ctx, pool, batch, &g, &p.pages);
    if (st != KVX_OK) return st;
    if (e->budget < 1 || e->budget > (1 << 30) || e->sinks < 0 || e->recent < 0 ||
        (int64_t)e->sinks + e->recent > e->budget)
      return refuse(KVX_EINVAL, "budget, sinks or recent");
    const int64_t pack = pool->pages_per_block > 1 ? pool->pages_per_block : 1;
    if (e->new_table_len < 1 || e->new_table_len > INT32_MAX ||
        (batch->num_seqs > 1 && e->new_table_stride < e->new_table_len))
      return refuse(KVX_EINVAL, "new_table_len or new_table_stride");
    const int64_t most = std::min<int64_t>(e->budget, p.pages.max_length);
    if ((__int128)e->new_table_len * pool->block_tokens * pack < most)
      return refuse(KVX_ERANGE, "new_tables hold fewer tokens than are kept");
    CurrentDevice guard(ctx.device);
    if (!guard.ok) return KVX_ECUDA;
    if ((st = check_stream(stream, ctx.device)) != KVX_OK) return refuse(st, "stream");
    const int64_t s = batch->num_seqs, h = pool->num_heads, layers = pool->num_layers;
    if (s == 0) return KVX_OK;
    if (layers * s * h * ((most + 31) / 32) > kMaxRows) return refuse(KVX_ERANGE, "more than 2^30 groups of 32 kept tokens");
    DeviceMemory mem(ctx.device);
    for (int32_t l = 0; l < layers; ++l)
      if ((st = layer_of(mem, pool, l, g, &p.layer_base[l])) != KVX_OK) return st;
    if ((st = check_batch_memory(mem, batch)) != KVX_OK) return st;
    if ((st = check_tables(mem, e->new_tables, s, e->new_table_stride, e->new_table_len, "new_tables")) != KVX_OK ||
        (st = check_words(mem, e->kept, layers * s * h * e->budget, "kept")) != KVX_OK ||
        (st = check_words(mem, e->new_lengths, s, "new_lengths")) != KVX_OK)
      return st;
    if (e->new_lengths < batch->lengths + s && batch->lengths < e->new_lengths + s)
      return refuse(KVX_EINVAL, "new_lengths overlaps the lengths that are read");
    int64_t bytes, upper;
    if (!extent(layers, e->weights_layer_stride, s, e->weights_seq_stride, 0, 4, &upper) ||
        !extent(h, e->weights_head_stride, 1, 0, p.pages.max_length, 4, &bytes))
      return refuse(KVX_EINVAL, "strides of weights");
    if ((st = check_words(mem, e->weights, (upper + bytes) / 4, "weights")) != KVX_OK) return st;
    if (e->new_weights) {
      if (!extent(layers, e->new_weights_layer_stride, s, e->new_weights_seq_stride, 0, 4, &upper) ||
          !extent(h, e->new_weights_head_stride, 1, 0, most, 4, &bytes) ||
          !disjoint({{layers, e->new_weights_layer_stride}, {s, e->new_weights_seq_stride}, {h, e->new_weights_head_stride}}, most))
        return refuse(KVX_EINVAL, "strides of new_weights");
      if ((st = check_words(mem, e->new_weights, (upper + bytes) / 4, "new_weights")) != KVX_OK) return st;
    }
    p.weights = e->weights;
    p.new_tables = e->new_tables;
    p.kept = e->kept;
    p.new_lengths = e->new_lengths;
    p.new_weights = e->new_weights;
    p.weights_layer = e->weights_layer_stride;
    p.weights_seq = e->weights_seq_stride;
    p.weights_head = e->weights_head_stride;
    p.new_weights_layer = e->new_weights_layer_stride;
    p.new_weights_seq = e->new_weights_seq_stride;
    p.new_weights_head = e->new_weights_head_stride;
    p.new_table_stride = e->new_table_stride;
    p.new_table_len = (uint32_t)e->new_table_len;
    p.budget = e->budget;
    p.sinks = e->sinks;
    p.recent = e->recent;
    p.num_layers = (int32_t)layers;
    p.row_vecs = div31((uint32_t)(g.row / 16));
    p.units = (int32_t)((most + 31) / 32);
    return KVX_LAUNCHED(c, launch_evict(p, stream), 2);
  });
}

kvx_status kv_state_conv(kvx_ctx* c, const kvx_state* state, const kvx_state_batch* batch, const kvx_conv* conv,
                         const void* x, void* out, kvx_stream_t stream) {
  return guarded([&]() -> kvx_status {
    if (!c || !state || !batch || !conv) return KVX_EINVAL;
    const CtxView ctx = view_of(c);
    if (conv->type != KVX_TYPE_BF16 && conv->type != KVX_TYPE_FP16) return refuse(KVX_EINVAL, "type");
    if (conv->channels < 8 || conv->channels > (1 << 24) || conv->width < 2 || conv->width > 4)
      return refuse(KVX_EINVAL, "channels or width");
    if (conv->channels % 8) return refuse(KVX_EALIGN, "channels");
    if (batch->num_seqs < 0 || batch->num_seqs > kMaxSeqs || batch->tokens < 0) return refuse(KVX_EINVAL, "num_seqs or tokens");
    CurrentDevice guard(ctx.device);
    if (!guard.ok) return KVX_ECUDA;
    kvx_status st = check_stream(stream, ctx.device);
    if (st != KVX_OK) return refuse(st, "stream");
    if (batch->num_seqs == 0) return KVX_OK;
    DeviceMemory mem(ctx.device);
    ConvParams p;
    const int64_t ch = conv->channels;
    if ((st = view_state(ctx, state, batch, state->conv_offset, (conv->width - 1) * ch * 2, mem, &p.state)) != KVX_OK)
      return st;
    if (batch->tokens > 0 &&
        ((st = check_rows(mem, {x, batch->tokens, conv->x_stride, 1, 0, ch, "x"}, false)) != KVX_OK ||
         (st = check_rows(mem, {out, batch->tokens, conv->out_stride, 1, 0, ch, "out"}, true)) != KVX_OK))
      return st;
    if ((st = check_rows(mem, {conv->weight, 1, 0, 1, 0, ch * conv->width, "weight"}, false)) != KVX_OK) return st;
    if (conv->bias && (st = check_rows(mem, {conv->bias, 1, 0, 1, 0, ch, "bias"}, false)) != KVX_OK) return st;
    p.x = (const uint8_t*)x;
    p.weight = (const uint8_t*)conv->weight;
    p.bias = (const uint8_t*)conv->bias;
    p.out = (uint8_t*)out;
    p.x_stride = conv->x_stride;
    p.out_stride = conv->out_stride;
    p.channels = conv->channels;
    p.width = conv->width;
    p.silu = conv->silu;
    return KVX_LAUNCHED(c, launch_conv(p, conv->type, stream), 1);
  });
}

namespace {

kvx_status check_scan(const kvx_state_batch* b, const kvx_scan* s) {
  if (s->type != KVX_TYPE_BF16 && s->type != KVX_TYPE_FP16) return refuse(KVX_EINVAL, "type");
  if (s->heads < 1 || s->heads > kMaxHeads || s->groups < 1 || s->heads % s->groups)
    return refuse(KVX_EINVAL, "heads or groups");
  const int32_t n = s->state_dim;
  if (n != 16 && n != 32 && n != 64 && n != 128 && n != 256) return refuse(KVX_EINVAL, "state_dim");
  if (s->head_dim < 8 || s->head_dim > 256) return refuse(KVX_EINVAL, "head_dim");
  if (s->head_dim % 8) return refuse(KVX_EALIGN, "head_dim");
  if (b->num_seqs < 0 || b->num_seqs > kMaxSeqs || b->tokens < 0) return refuse(KVX_EINVAL, "num_seqs or tokens");
  return KVX_OK;
}

// kv_state_scan's workspace: the segments' states and exponents, where sequences are cut.
struct ScanSpace {
  int32_t segment, by_token;
  int64_t exponents, bytes;
};
ScanSpace scan_space(const CtxView& ctx, const kvx_state_batch* b, const kvx_scan* a) {
  StateView v = {};
  v.starts = b->starts;
  v.tokens = b->tokens;
  v.num_seqs = b->num_seqs;
  bool cut;
  ScanSpace w = {};
  w.by_token = INT32_MAX;
  if (!ctx.scan_matrix) return w;
  w.segment = scan_segment(v, a->heads, a->head_dim, a->state_dim, ctx.num_sms, &cut, &w.by_token);
  if (cut) {
    const int64_t pieces = scan_pieces(v, w.segment);
    w.exponents = pieces * a->heads * a->head_dim * a->state_dim * 4;
    w.bytes = w.exponents + pieces * a->heads * 4;
  }
  return w;
}

}  // namespace

kvx_status kv_state_scan_workspace(kvx_ctx* c, const kvx_state_batch* batch, const kvx_scan* scan, int64_t* bytes) {
  return guarded([&]() -> kvx_status {
    if (!c || !batch || !scan || !bytes) return KVX_EINVAL;
    const kvx_status st = check_scan(batch, scan);
    if (st != KVX_OK) return st;
    *bytes = scan_space(view_of(c), batch, scan).bytes;
    return KVX_OK;
  });
}

kvx_status kv_state_scan(kvx_ctx* c, const kvx_state* state, const kvx_state_batch* batch, const kvx_scan* a,
                         const void* x, const void* dt, const void* B, const void* C, void* out, void* workspace,
                         int64_t workspace_bytes, kvx_stream_t stream) {
  return guarded([&]() -> kvx_status {
    if (!c || !state || !batch || !a) return KVX_EINVAL;
    const CtxView ctx = view_of(c);
    kvx_status st = check_scan(batch, a);
    if (st != KVX_OK) return st;
    CurrentDevice guard(ctx.device);
    if (!guard.ok) return KVX_ECUDA;
    if ((st = check_stream(stream, ctx.device)) != KVX_OK) return refuse(st, "stream");
    if (batch->num_seqs == 0) return KVX_OK;
    DeviceMemory mem(ctx.device);
    ScanParams p;
    const int64_t h = a->heads, d = a->head_dim, n = a->state_dim, rows = batch->tokens;
    if ((st = view_state(ctx, state, batch, state->recurrent_offset, h * d * n * 4, mem, &p.state)) != KVX_OK) return st;
    if (rows > 0) {
      if ((st = check_rows(mem, {x, rows, a->x_token_stride, h, a->x_head_stride, d, "x"}, false)) != KVX_OK ||
          (st = check_rows(mem, {B, rows, a->b_token_stride, a->groups, a->b_group_stride, n, "B"}, false)) != KVX_OK ||
          (st = check_rows(mem, {C, rows, a->c_token_stride, a->groups, a->c_group_stride, n, "C"}, false)) != KVX_OK ||
          (st = check_rows(mem, {out, rows, a->out_token_stride, h, a->out_head_stride, d, "out"}, true)) != KVX_OK)
        return st;
      int64_t bytes;
      if (!dt || !extent(rows, a->dt_token_stride, 1, 0, h, 2, &bytes)) return refuse(KVX_EINVAL, "dt");
      if ((uintptr_t)dt & 1) return refuse(KVX_EALIGN, "dt");
      if ((st = mem.check(dt, bytes)) != KVX_OK) return refuse(st, "dt");
    }
    if ((st = check_words(mem, a->A, h, "A")) != KVX_OK) return st;
    if (a->D && (st = check_words(mem, a->D, h, "D")) != KVX_OK) return st;
    if (a->dt_bias && (st = check_words(mem, a->dt_bias, h, "dt_bias")) != KVX_OK) return st;
    const ScanSpace space = scan_space(ctx, batch, a);
    if (space.bytes > 0) {
      if (workspace_bytes < space.bytes) return refuse(KVX_ERANGE, "workspace is smaller than kv_state_scan_workspace says");
      if (!workspace || ((uintptr_t)workspace & 15)) return refuse(workspace ? KVX_EALIGN : KVX_EINVAL, "workspace");
      if ((st = mem.check(workspace, space.bytes)) != KVX_OK) return refuse(st, "workspace");
    }
    p.segment = space.segment;
    p.pieces = space.segment ? (int32_t)scan_pieces(p.state, space.segment) : 0;
    p.by_token = space.by_token;
    p.segment_states = space.bytes > 0 ? (float*)workspace : nullptr;
    p.segment_exponents = space.bytes > 0 ? (float*)((uint8_t*)workspace + space.exponents) : nullptr;
    p.x = (const uint8_t*)x;
    p.dt = (const uint8_t*)dt;
    p.b = (const uint8_t*)B;
    p.c = (const uint8_t*)C;
    p.out = (uint8_t*)out;
    p.A = a->A;
    p.D = a->D;
    p.dt_bias = a->dt_bias;
    p.x_token = a->x_token_stride;
    p.x_head = a->x_head_stride;
    p.dt_token = a->dt_token_stride;
    p.b_token = a->b_token_stride;
    p.b_group = a->b_group_stride;
    p.c_token = a->c_token_stride;
    p.c_group = a->c_group_stride;
    p.out_token = a->out_token_stride;
    p.out_head = a->out_head_stride;
    p.heads = a->heads;
    p.head_dim = a->head_dim;
    p.state_dim = a->state_dim;
    p.heads_per_group = a->heads / a->groups;
    p.softplus = a->softplus;
    p.wait_cycles = ctx.wait_cycles;
    p.timeout = ctx.timeout;
    p.stall = p.segment && fault_point("scan_wait");
    return KVX_LAUNCHED(c, launch_scan(p, a->type, ctx.num_sms, stream),
                        (space.by_token >= 0) + (space.segment ? space.bytes > 0 ? 3 : 1 : 0));
  });
}

namespace {

kvx_status check_delta(const kvx_state_batch* b, const kvx_delta* d) {
  if (d->type != KVX_TYPE_BF16 && d->type != KVX_TYPE_FP16) return refuse(KVX_EINVAL, "type");
  if (d->heads < 1 || d->heads > kMaxHeads || d->groups < 1 || d->heads % d->groups) return refuse(KVX_EINVAL, "heads or groups");
  const int32_t n = d->state_dim;
  if (n != 16 && n != 32 && n != 64 && n != 128 && n != 256) return refuse(KVX_EINVAL, "state_dim");
  if (d->head_dim < 8 || d->head_dim > 256) return refuse(KVX_EINVAL, "head_dim");
  if (d->head_dim % 8) return refuse(KVX_EALIGN, "head_dim");
  if (!std::isfinite(d->scale) || !std::isfinite(d->eps) || d->eps < 0.f) return refuse(KVX_EINVAL, "scale or eps");
  if (b->num_seqs < 0 || b->num_seqs > kMaxSeqs || b->tokens < 0) return refuse(KVX_EINVAL, "num_seqs or tokens");
  return KVX_OK;
}

// kv_state_delta's workspace: what the chunks of 64 tokens are worked on with, where there are any.
struct DeltaSpace {
  int32_t by_token, long_seqs, pieces;
  int64_t heads, bytes;  // heads: the offset of head_space
};
kvx_status delta_space(const kvx_state_batch* b, const kvx_delta* d, DeltaSpace* w) {
  *w = {};
  if (!delta_by_chunks(b->tokens, b->num_seqs, b->starts, d->state_dim, &w->by_token)) return KVX_OK;
  // as many as sequences whose rows do not overlap can have
  w->long_seqs = (int32_t)std::min<int64_t>(b->num_seqs, w->by_token < 0 ? b->num_seqs : b->tokens / (w->by_token + 1));
  const int64_t pieces = b->tokens / kDeltaChunk + w->long_seqs;
  if (pieces > kMaxRows / d->heads) return refuse(KVX_ERANGE, "more than 2^30 chunks and heads");
  w->pieces = (int32_t)pieces;
  w->heads = pieces * d->groups * 2 * kDeltaChunk * d->state_dim * 2;
  w->bytes = w->heads + pieces * d->heads * kDeltaHeadBytes;
  return KVX_OK;
}

// A value a token and head, 2 bytes each.
kvx_status check_gate(DeviceMemory& mem, const void* p, int64_t tokens, int64_t stride, int64_t heads, const char* what) {
  int64_t bytes;
  if (!p || !extent(tokens, stride, 1, 0, heads, 2, &bytes)) return refuse(KVX_EINVAL, what);
  if ((uintptr_t)p & 1) return refuse(KVX_EALIGN, what);
  const kvx_status st = mem.check(p, bytes);
  return st == KVX_OK ? st : refuse(st, what);
}

}  // namespace

kvx_status kv_state_delta_workspace(kvx_ctx* c, const kvx_state_batch* batch, const kvx_delta* d, int64_t* bytes) {
  return guarded([&]() -> kvx_status {
    if (!c || !batch || !d || !bytes) return KVX_EINVAL;
    DeltaSpace space;
    kvx_status st = check_delta(batch, d);
    if (st == KVX_OK) st = delta_space(batch, d, &space);
    if (st != KVX_OK) return st;
    *bytes = space.bytes;
    return KVX_OK;
  });
}

kvx_status kv_state_delta(kvx_ctx* c, const kvx_state* state, const kvx_state_batch* batch, const kvx_delta* a, const void* q,
                          const void* k, const void* v, const void* dt, const void* beta, void* out, void* workspace,
                          int64_t workspace_bytes, kvx_stream_t stream) {
  return guarded([&]() -> kvx_status {
    if (!c || !state || !batch || !a) return KVX_EINVAL;
    const CtxView ctx = view_of(c);
    DeltaSpace space;
    kvx_status st = check_delta(batch, a);
    if (st == KVX_OK) st = delta_space(batch, a, &space);
    if (st != KVX_OK) return st;
    CurrentDevice guard(ctx.device);
    if (!guard.ok) return KVX_ECUDA;
    if ((st = check_stream(stream, ctx.device)) != KVX_OK) return refuse(st, "stream");
    if (batch->num_seqs == 0) return KVX_OK;
    DeviceMemory mem(ctx.device);
    DeltaParams p;
    const int64_t h = a->heads, d = a->head_dim, n = a->state_dim, rows = batch->tokens;
    if ((st = view_state(ctx, state, batch, state->recurrent_offset, h * d * n * 4, mem, &p.state)) != KVX_OK) return st;
    if (rows > 0) {
      if ((st = check_rows(mem, {q, rows, a->q_token_stride, a->groups, a->q_head_stride, n, "q"}, false)) != KVX_OK ||
          (st = check_rows(mem, {k, rows, a->k_token_stride, a->groups, a->k_head_stride, n, "k"}, false)) != KVX_OK ||
          (st = check_rows(mem, {v, rows, a->v_token_stride, h, a->v_head_stride, d, "v"}, false)) != KVX_OK ||
          (st = check_rows(mem, {out, rows, a->out_token_stride, h, a->out_head_stride, d, "out"}, true)) != KVX_OK)
        return st;
      if (out == q || out == k || out == v) return refuse(KVX_EINVAL, "out is q, k or v");
      if (dt && (st = check_gate(mem, dt, rows, a->dt_token_stride, h, "dt")) != KVX_OK) return st;
      if ((st = check_gate(mem, beta, rows, a->beta_token_stride, h, "beta")) != KVX_OK) return st;
    }
    if (dt && (st = check_words(mem, a->A, h, "A")) != KVX_OK) return st;
    if (dt && a->dt_bias && (st = check_words(mem, a->dt_bias, h, "dt_bias")) != KVX_OK) return st;
    if (space.bytes > 0) {
      if (workspace_bytes < space.bytes) return refuse(KVX_ERANGE, "workspace is smaller than kv_state_delta_workspace says");
      if (!workspace || ((uintptr_t)workspace & 15)) return refuse(workspace ? KVX_EALIGN : KVX_EINVAL, "workspace");
      if ((st = mem.check(workspace, space.bytes)) != KVX_OK) return refuse(st, "workspace");
    }
    p.by_token = space.by_token;
    p.long_seqs = space.long_seqs;
    p.pieces = space.pieces;
    p.rows_space = (uint8_t*)workspace;
    p.head_space = (uint8_t*)workspace + space.heads;
    p.wait_cycles = ctx.wait_cycles;
    p.timeout = ctx.timeout;
    p.stall = !p.pieces ? 0 : fault_point("delta_wait") ? 1 : fault_point("delta_wait_m") ? 2 : 0;
    p.q = (const uint8_t*)q;
    p.k = (const uint8_t*)k;
    p.v = (const uint8_t*)v;
    p.dt = (const uint8_t*)dt;
    p.beta = (const uint8_t*)beta;
    p.out = (uint8_t*)out;
    p.A = a->A;
    p.dt_bias = a->dt_bias;
    p.q_token = a->q_token_stride;
    p.q_head = a->q_head_stride;
    p.k_token = a->k_token_stride;
    p.k_head = a->k_head_stride;
    p.v_token = a->v_token_stride;
    p.v_head = a->v_head_stride;
    p.dt_token = a->dt_token_stride;
    p.beta_token = a->beta_token_stride;
    p.out_token = a->out_token_stride;
    p.out_head = a->out_head_stride;
    p.heads = a->heads;
    p.head_dim = a->head_dim;
    p.state_dim = a->state_dim;
    p.heads_per_group = a->heads / a->groups;
    p.groups = a->groups;
    p.softplus = a->softplus;
    p.sigmoid = a->sigmoid;
    p.normalize = a->normalize;
    p.scale = a->scale ? a->scale : 1.f / std::sqrt((float)n);
    p.eps = a->eps;
    return KVX_LAUNCHED(c, launch_delta(p, a->type, ctx.num_sms, stream), p.pieces ? 2 : 1);
  });
}
