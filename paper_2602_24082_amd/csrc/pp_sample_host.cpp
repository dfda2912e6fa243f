// Host entry points of the sampling operators declared in pp_attn.h: the paged cache,
// attention of drafted trees over it, draft verification.  Arguments are validated here
// before anything is enqueued; what lies in device arrays the kernels check themselves.
// Nothing here allocates or throws.

#include <hip/hip_runtime.h>

#include <cmath>
#include <initializer_list>

#include "../../include/pp_attn.h"
#include "pp_sample.h"

namespace pp {
namespace {

constexpr size_t kAlign = 256;

bool aligned(const void* p, uintptr_t to) { return (reinterpret_cast<uintptr_t>(p) & (to - 1)) == 0; }

// Regions of a workspace, one after the other.
struct Carve {
  char* base;
  size_t used = 0;
  explicit Carve(void* ws) : base((char*)ws) {}
  template <typename T>
  T* take(int64_t n) {
    T* p = base ? (T*)(base + used) : nullptr;
    used += ((size_t)n * sizeof(T) + kAlign - 1) / kAlign * kAlign;
    return p;
  }
};

pp_status check_cache(const pp_cache* c, CacheView* v) {
  if (!c) return report_error(PP_ERR_INVALID_ARGUMENT, "cache is NULL");
  if (c->num_slots < 1 || c->max_pages < 1 || c->num_pages < 1)
    return report_error(PP_ERR_INVALID_ARGUMENT, "num_slots, max_pages and num_pages must be >= 1");
  if ((int64_t)c->num_slots * c->max_pages > INT32_MAX)
    return report_error(PP_ERR_UNSUPPORTED, "a page table of %d x %d entries is too large", c->num_slots, c->max_pages);
  const int ps = c->page_size;
  if (ps < 16 || ps > 256 || (ps & (ps - 1)))
    return report_error(PP_ERR_UNSUPPORTED, "page_size %d not supported (16, 32, 64, 128 or 256)", ps);
  // places of tokens are counted in 32 bits, up to two blocks of keys past a sequence's last
  if ((int64_t)c->max_pages * ps > INT32_MAX - 1024 || (int64_t)c->num_pages * ps > INT32_MAX)
    return report_error(PP_ERR_UNSUPPORTED, "a sequence or pool of 2^31 tokens or more is too large");
  if (!c->page_table || !c->seq_len || !c->held || !c->refs)
    return report_error(PP_ERR_INVALID_ARGUMENT, "page_table, seq_len, held and refs must be non-NULL");
  if (!aligned(c->page_table, 4) || !aligned(c->seq_len, 4) || !aligned(c->held, 4) || !aligned(c->refs, 4))
    return report_error(PP_ERR_INVALID_ARGUMENT, "page_table, seq_len, held and refs must be 4-byte aligned");
  v->table = c->page_table;
  v->seq_len = c->seq_len;
  v->held = c->held;
  v->refs = c->refs;
  v->num_slots = c->num_slots;
  v->max_pages = c->max_pages;
  v->num_pages = c->num_pages;
  v->page_size = ps;
  v->page_log2 = __builtin_ctz((unsigned)ps);
  return PP_OK;
}

constexpr int kMostSeqs = 65535;  // a launch's second dimension
// query rows of the attention: the join takes 8 a workgroup of 256 threads at head size 128, and a launch
// has fewer than 2^32 threads
constexpr int64_t kMostRows = 8 * ((int64_t)UINT32_MAX / 256);
constexpr int kMostNew = 1 << 24;  // tokens a sequence and call: a launch's first, in threads

pp_status check_n(int n) {
  if (n < 0) return report_error(PP_ERR_INVALID_ARGUMENT, "n must be >= 0 (got %d)", n);
  if (n > kMostSeqs) return report_error(PP_ERR_UNSUPPORTED, "a call takes at most %d sequences (got %d)", kMostSeqs, n);
  return PP_OK;
}

pp_status check_dtype(pp_dtype t) {
  if (t != PP_BF16 && t != PP_FP32) return report_error(PP_ERR_INVALID_ARGUMENT, "unknown dtype %d", (int)t);
  return PP_OK;
}

pp_status check_head_dim(int hkv, int d) {
  if (hkv < 1) return report_error(PP_ERR_INVALID_ARGUMENT, "hkv must be >= 1");
  if (hkv > 4096) return report_error(PP_ERR_UNSUPPORTED, "at most 4096 kv-heads (got %d)", hkv);
  if (d != 64 && d != 128) return report_error(PP_ERR_UNSUPPORTED, "head_dim %d not supported (64 or 128)", d);
  return PP_OK;
}

pp_status check_q_heads(int hq, int hkv, int d) {
  if (hq < 1 || hkv < 1) return report_error(PP_ERR_INVALID_ARGUMENT, "hq and hkv must be >= 1");
  if (hq % hkv) return report_error(PP_ERR_INVALID_ARGUMENT, "hq (%d) must be a multiple of hkv (%d)", hq, hkv);
  if (hq > 4096) return report_error(PP_ERR_UNSUPPORTED, "at most 4096 query heads (got %d)", hq);
  return check_head_dim(hkv, d);
}

pp_status check_pools(const CacheView& c, pp_dtype dtype, int layers, int hkv, int d, void* k, void* v, CachePools* p) {
  pp_status st = check_dtype(dtype);
  if (st != PP_OK) return st;
  if ((st = check_head_dim(hkv, d)) != PP_OK) return st;
  if (layers < 0) return report_error(PP_ERR_INVALID_ARGUMENT, "layers must be >= 0");
  if (layers > 16384) return report_error(PP_ERR_UNSUPPORTED, "at most 16384 layers (got %d)", layers);
  if (layers && (!k || !v)) return report_error(PP_ERR_INVALID_ARGUMENT, "k_pages and v_pages must be non-NULL");
  if (!aligned(k, 16) || !aligned(v, 16)) return report_error(PP_ERR_INVALID_ARGUMENT, "k_pages and v_pages must be 16-byte aligned");
  p->k = (char*)k;
  p->v = (char*)v;
  p->layers = layers;
  p->hkv = hkv;
  p->row_bytes = d * (dtype == PP_BF16 ? 2 : 4);
  p->head_bytes = p->row_bytes * c.page_size;
  p->page_bytes = (int64_t)p->head_bytes * hkv;
  p->layer_bytes = p->page_bytes * c.num_pages;
  return PP_OK;
}

size_t carve_cache(const CacheView& c, int n, void* ws, CacheScratch* w) {
  Carve at(ws);
  w->mark = at.take<int32_t>(c.num_slots);
  w->first = at.take<int32_t>(n);
  w->list = at.take<int32_t>(c.num_pages);
  w->list2 = at.take<int32_t>(c.num_pages);
  w->renum = at.take<int32_t>(c.num_pages);
  w->moves = at.take<int32_t>(2);
  w->entries = at.take<ForkEntry>(n);
  return at.used;
}

pp_status check_ws(const void* ws, size_t ws_bytes, size_t need, const char* what) {
  if (ws_bytes < need) return report_error(PP_ERR_WORKSPACE_TOO_SMALL, "%s needs %zu workspace bytes, got %zu", what, need, ws_bytes);
  if (need && !ws) return report_error(PP_ERR_INVALID_ARGUMENT, "ws is NULL");
  if (!aligned(ws, kAlign)) return report_error(PP_ERR_INVALID_ARGUMENT, "ws must be 256-byte aligned");
  return PP_OK;
}

pp_status check_ints(std::initializer_list<const void*> ptrs) {
  for (const void* p : ptrs) {
    if (!p) return report_error(PP_ERR_INVALID_ARGUMENT, "a required int32 or float array is NULL");
    if (!aligned(p, 4)) return report_error(PP_ERR_INVALID_ARGUMENT, "int32 and float arrays must be 4-byte aligned");
  }
  return PP_OK;
}
pp_status check_optional(std::initializer_list<const void*> ptrs) {
  for (const void* p : ptrs)
    if (!aligned(p, 4)) return report_error(PP_ERR_INVALID_ARGUMENT, "int32 and float arrays must be 4-byte aligned");
  return PP_OK;
}

pp_status launched(hipError_t e, const char* what) { return e == hipSuccess ? PP_OK : report_hip_error(e, what); }

// What a call over the cache and n of its sequences has in common.
pp_status check_call(const pp_cache* cache, int n, const void* ws, size_t ws_bytes, const char* what, CacheView* c, CacheScratch* w) {
  pp_status st = check_cache(cache, c);
  if (st != PP_OK) return st;
  if ((st = check_n(n)) != PP_OK) return st;
  return check_ws(ws, ws_bytes, carve_cache(*c, n, const_cast<void*>(ws), w), what);
}

bool shape_tree(int n, int group, int nodes, int hq, int hkv, pp_dtype dtype, int d, bool shared, TreeShape* t) {
  t->n = n;
  t->nodes = nodes;
  t->group = group;
  t->groups = n / group;
  t->hq = hq;
  t->hkv = hkv;
  t->G = hq / hkv;
  const bool bf16 = dtype == PP_BF16;
  if ((int64_t)n * nodes * hq > kMostRows) return false;
  t->workers[0] = kCus * (bf16 ? (d == 128 ? kTreeSolo<128, uint16_t> : kTreeSolo<64, uint16_t>)
                               : (d == 128 ? kTreeSolo<128, float> : kTreeSolo<64, float>));
  t->workers[1] = kCus * (bf16 ? (d == 128 ? kTreeTeam<128, uint16_t> : kTreeTeam<64, uint16_t>)
                               : (d == 128 ? kTreeTeam<128, float> : kTreeTeam<64, float>));
  int64_t parts = 0;
  for (int k = 0; k < 2; ++k) {
    const int64_t rows = (int64_t)nodes * t->G * (k == 0 ? group : 1);
    if (rows > INT32_MAX / 2) return false;
    TreeKind& x = t->kind[k];
    x = TreeKind{};
    x.rows = k == 0 && (group == 1 || !shared) ? 0 : (int)rows;
    x.team = x.rows > kSoloRows;
    x.keys = !x.team ? kSoloKeys : bf16 ? kTeamKeys<128, uint16_t> : kTeamKeys<128, float>;
    const int tile = x.team ? kTeamRows : kSoloRows;
    x.tiles = (x.rows + tile - 1) / tile;
    x.part_rows = x.rows < tile ? x.rows : tile;
    x.part0 = parts;
    const int64_t results = (int64_t)(k == 0 ? t->groups : n) * x.tiles * hkv + t->workers[x.team];
    if (results > INT32_MAX) return false;  // tiles and partial results are counted in 32 bits
    parts += results * x.part_rows;
  }
  return true;
}

size_t carve_tree(const TreeShape& t, int d, void* ws, TreeLaunch* a) {
  Carve at(ws);
  const int items = t.n + t.groups;
  a->plan.items = at.take<TreeItem>(items);
  a->plan.nodes = at.take<int32_t>((int64_t)t.n * t.nodes);
  a->plan.head = at.take<int64_t>(5);
  for (int c = 0; c < 2; ++c) a->plan.start_item[c] = at.take<int32_t>(t.workers[c]);
  const TreeKind& last = t.kind[1];
  const int64_t parts = last.part0 + ((int64_t)t.n * last.tiles * t.hkv + t.workers[last.team]) * last.part_rows;
  a->part_ml = at.take<float>(2 * parts);
  a->part = at.take<float>(parts * d);
  return at.used;
}

// Names the calls that can go by a plan: those of its sizes.
uint64_t key_of(const TreeShape& t, const CacheView& c, int d, int dtype) {
  uint64_t k = 0x9e3779b97f4a7c15ull;
  for (const int x : {t.n, t.nodes, t.group, t.hq, t.hkv, t.kind[0].tiles, d, dtype, c.num_slots, c.max_pages, c.num_pages, c.page_size}) {
    k = (k ^ (uint32_t)x) * 0xd6e8feb86659fd93ull;
    k ^= k >> 32;
  }
  return k;
}

pp_status check_tree(int n, int group, int nodes, pp_dtype dtype, int hq, int hkv, int d) {
  pp_status st = check_dtype(dtype);
  if (st != PP_OK) return st;
  if ((st = check_q_heads(hq, hkv, d)) != PP_OK) return st;
  if (n < 0) return report_error(PP_ERR_INVALID_ARGUMENT, "n must be >= 0 (got %d)", n);
  if (n > kTreeSeqs) return report_error(PP_ERR_UNSUPPORTED, "a call takes at most %d sequences (got %d)", kTreeSeqs, n);
  if (group < 1 || n % group) return report_error(PP_ERR_INVALID_ARGUMENT, "n (%d) must be a multiple of group (%d)", n, group);
  if (nodes < 1) return report_error(PP_ERR_INVALID_ARGUMENT, "max_new must be >= 1");
  if (nodes > kTreeNodes)
    return report_error(PP_ERR_UNSUPPORTED, "a sequence's tree has at most %d nodes (got %d)", kTreeNodes, nodes);
  return PP_OK;
}

size_t carve_draft(DraftParams* p, void* ws) {
  Carve at(ws);
  const DraftShape& d = p->shape;
  const int64_t rows = (int64_t)d.n * d.nodes;
  p->part = at.take<DraftPart>(2 * rows * d.chunks);
  p->left = at.take<double>(rows * d.chunks);
  p->ends = at.take<double>((int64_t)d.n * d.chunks);
  p->row = at.take<DraftRow>(2 * rows);
  p->edge = at.take<DraftEdge>(rows);
  p->arrived = at.take<int32_t>((int64_t)d.n * kOwnLine);
  return at.used;
}

pp_status shape_draft(int n, int nodes, int vocab, int max_children, pp_dtype dtype, DraftShape* d) {
  pp_status st = check_dtype(dtype);
  if (st != PP_OK) return st;
  if (n < 0) return report_error(PP_ERR_INVALID_ARGUMENT, "n must be >= 0 (got %d)", n);
  if (nodes < 1) return report_error(PP_ERR_INVALID_ARGUMENT, "max_new must be >= 1");
  if (nodes > kTreeNodes)
    return report_error(PP_ERR_UNSUPPORTED, "a sequence's tree has at most %d nodes (got %d)", kTreeNodes, nodes);
  if ((int64_t)n * nodes > kMostSeqs) return report_error(PP_ERR_UNSUPPORTED, "a call takes at most %d rows of logits", kMostSeqs);
  if (vocab < 1) return report_error(PP_ERR_INVALID_ARGUMENT, "vocab must be >= 1");
  if (vocab > INT32_MAX - 2 * kDraftChunk) return report_error(PP_ERR_UNSUPPORTED, "vocab %d is too large", vocab);
  if (max_children < 1) return report_error(PP_ERR_INVALID_ARGUMENT, "max_children must be >= 1");
  d->n = n;
  d->nodes = nodes;
  d->vocab = vocab;
  const int reach = vocab + 16 / (dtype == PP_BF16 ? 2 : 4) - 1;  // from a 16-byte boundary on
  d->chunks = (reach + kDraftChunk - 1) / kDraftChunk;
  d->max_children = max_children < nodes ? max_children : nodes;
  return PP_OK;
}

}  // namespace
}  // namespace pp

using namespace pp;

extern "C" {

pp_status pp_cache_workspace_size(const pp_cache* cache, int n, size_t* bytes) {
  CacheView c;
  pp_status st = check_cache(cache, &c);
  if (st != PP_OK) return st;
  if ((st = check_n(n)) != PP_OK) return st;
  if (!bytes) return report_error(PP_ERR_INVALID_ARGUMENT, "bytes is NULL");
  CacheScratch w;
  *bytes = carve_cache(c, n, nullptr, &w);
  return PP_OK;
}

pp_status pp_cache_reserve(const pp_cache* cache, int n, const int32_t* slots, const int32_t* add, int32_t* status, void* ws,
                           size_t ws_bytes, void* hip_stream) {
  CacheView c;
  CacheScratch w;
  pp_status st = check_call(cache, n, ws, ws_bytes, "the cache", &c, &w);
  if (st != PP_OK) return st;
  if ((st = n ? check_ints({slots, add, status}) : check_ints({status})) != PP_OK) return st;
  return launched(launch_cache_reserve(c, n, slots, add, status, w, (hipStream_t)hip_stream), "cache reserve launch");
}

pp_status pp_cache_fork(const pp_cache* cache, int n, const int32_t* src, const int32_t* dst, pp_dtype dtype, int layers, int hkv,
                        int head_dim, void* k_pages, void* v_pages, int32_t* status, void* ws, size_t ws_bytes, void* hip_stream) {
  CacheView c;
  CacheScratch w;
  CachePools p;
  pp_status st = check_call(cache, n, ws, ws_bytes, "the cache", &c, &w);
  if (st != PP_OK) return st;
  if ((st = check_pools(c, dtype, layers, hkv, head_dim, k_pages, v_pages, &p)) != PP_OK) return st;
  if ((st = n ? check_ints({src, dst, status}) : check_ints({status})) != PP_OK) return st;
  return launched(launch_cache_fork(c, p, n, src, dst, status, w, (hipStream_t)hip_stream), "cache fork launch");
}

pp_status pp_cache_free(const pp_cache* cache, int n, const int32_t* slots, void* hip_stream) {
  CacheView c;
  pp_status st = check_cache(cache, &c);
  if (st != PP_OK) return st;
  if ((st = check_n(n)) != PP_OK) return st;
  if (n == 0) return PP_OK;
  if ((st = check_ints({slots})) != PP_OK) return st;
  return launched(launch_cache_free(c, n, slots, (hipStream_t)hip_stream), "cache free launch");
}

pp_status pp_cache_compact(const pp_cache* cache, pp_dtype dtype, int layers, int hkv, int head_dim, void* k_pages, void* v_pages,
                           int32_t* live, void* ws, size_t ws_bytes, void* hip_stream) {
  CacheView c;
  CacheScratch w;
  CachePools p;
  pp_status st = check_call(cache, 0, ws, ws_bytes, "the cache", &c, &w);
  if (st != PP_OK) return st;
  if ((st = check_pools(c, dtype, layers, hkv, head_dim, k_pages, v_pages, &p)) != PP_OK) return st;
  if ((st = check_ints({live})) != PP_OK) return st;
  return launched(launch_cache_compact(c, p, live, w, (hipStream_t)hip_stream), "cache compact launch");
}

pp_status pp_cache_accept(const pp_cache* cache, int n, const int32_t* slots, int max_new, const int32_t* count, const int32_t* path,
                          pp_dtype dtype, int layers, int hkv, int head_dim, void* k_pages, void* v_pages, int32_t* status, void* ws,
                          size_t ws_bytes, void* hip_stream) {
  CacheView c;
  CacheScratch w;
  CachePools p;
  pp_status st = check_call(cache, n, ws, ws_bytes, "the cache", &c, &w);
  if (st != PP_OK) return st;
  if ((st = check_pools(c, dtype, path ? layers : 0, hkv, head_dim, k_pages, v_pages, &p)) != PP_OK) return st;
  if (max_new < 1) return report_error(PP_ERR_INVALID_ARGUMENT, "max_new must be >= 1");
  if (path && max_new > kAcceptNodes)
    return report_error(PP_ERR_UNSUPPORTED, "a sequence's tree has at most %d nodes (got %d)", kAcceptNodes, max_new);
  if ((st = n ? check_ints({slots, count, status}) : check_ints({status})) != PP_OK) return st;
  if ((st = check_optional({path})) != PP_OK) return st;
  return launched(launch_cache_accept(c, p, n, slots, max_new, count, path, status, w, (hipStream_t)hip_stream),
                  "cache accept launch");
}

pp_status pp_cache_shared(const pp_cache* cache, int n, const int32_t* slots, int group, int32_t* shared, void* hip_stream) {
  CacheView c;
  pp_status st = check_cache(cache, &c);
  if (st != PP_OK) return st;
  if ((st = check_n(n)) != PP_OK) return st;
  if (group < 1 || n % group) return report_error(PP_ERR_INVALID_ARGUMENT, "n (%d) must be a multiple of group (%d)", n, group);
  if (n == 0) return PP_OK;
  if ((st = check_ints({slots, shared})) != PP_OK) return st;
  return launched(launch_cache_shared(c, n / group, slots, group, shared, (hipStream_t)hip_stream), "cache shared launch");
}

pp_status pp_cache_append(const pp_cache* cache, int n, const int32_t* slots, int max_new, const int32_t* count, const int32_t* start,
                          int64_t rows, const int32_t* parents, pp_dtype dtype, int hq, int hkv, int head_dim, float rope_base,
                          const void* q, const void* k, const void* v, void* q_rot, void* k_pages, void* v_pages,
                          void* hip_stream) {
  CacheView c;
  CachePools p;
  pp_status st = check_cache(cache, &c);
  if (st != PP_OK) return st;
  if ((st = check_n(n)) != PP_OK) return st;
  if ((st = check_pools(c, dtype, 1, hkv, head_dim, k_pages, v_pages, &p)) != PP_OK) return st;
  if (max_new < 1) return report_error(PP_ERR_INVALID_ARGUMENT, "max_new must be >= 1");
  if (max_new > kMostNew)
    return report_error(PP_ERR_UNSUPPORTED, "a call appends at most %d tokens to a sequence (got %d)", kMostNew, max_new);
  if (q && (hq < 1 || hq % hkv || hq > 4096))
    return report_error(PP_ERR_INVALID_ARGUMENT, "hq (%d) must be a multiple of hkv (%d), at most 4096", hq, hkv);
  if (!q != !q_rot) return report_error(PP_ERR_INVALID_ARGUMENT, "q and q_rot must be given together");
  if (parents && max_new > kTreeNodes)
    return report_error(PP_ERR_UNSUPPORTED, "a sequence's tree has at most %d nodes (got %d)", kTreeNodes, max_new);
  if (!(rope_base >= 0) || !std::isfinite(rope_base)) return report_error(PP_ERR_INVALID_ARGUMENT, "rope_base must be finite and >= 0");
  if (rows < 0 || (!start && rows < (int64_t)n * max_new))
    return report_error(PP_ERR_INVALID_ARGUMENT, "rows must be >= 0, and n * max_new without start");
  if (n == 0) return PP_OK;
  if (rows && (!k || !v)) return report_error(PP_ERR_INVALID_ARGUMENT, "k and v must be non-NULL");
  for (const void* x : {q, k, v, (const void*)q_rot})
    if (!aligned(x, 16)) return report_error(PP_ERR_INVALID_ARGUMENT, "q, k, v and q_rot must be 16-byte aligned");
  if ((st = check_ints({slots})) != PP_OK) return st;
  if ((st = check_optional({count, start, parents})) != PP_OK) return st;
  AppendParams a{};
  a.slots = slots;
  a.count = count;
  a.start = start;
  a.parents = parents;
  a.q = q;
  a.k = k;
  a.v = v;
  a.q_rot = q_rot;
  a.k_pages = k_pages;
  a.v_pages = v_pages;
  a.rows = rows;
  a.max_new = max_new;
  a.hq = q ? hq : 0;
  a.hkv = hkv;
  a.turns = rope_base > 0;
  if (a.turns)
    for (int j = 0; j < head_dim / 2; ++j) a.inv_freq[j] = std::pow((double)rope_base, -2.0 * j / head_dim);
  return launched(launch_cache_append(c, a, n, head_dim, dtype == PP_BF16 ? kBF16 : kFP32, (hipStream_t)hip_stream),
                  "cache append launch");
}

pp_status pp_tree_workspace_size(const pp_cache* cache, int n, int group, int max_new, pp_dtype dtype, int hq, int hkv, int head_dim,
                                 size_t* bytes) {
  CacheView c;
  pp_status st = check_cache(cache, &c);
  if (st != PP_OK) return st;
  if ((st = check_tree(n, group, max_new, dtype, hq, hkv, head_dim)) != PP_OK) return st;
  if (!bytes) return report_error(PP_ERR_INVALID_ARGUMENT, "bytes is NULL");
  TreeLaunch a{};
  if (!shape_tree(n, group, max_new, hq, hkv, dtype, head_dim, true, &a.shape))
    return report_error(PP_ERR_UNSUPPORTED, "the call has too many rows");
  *bytes = carve_tree(a.shape, head_dim, nullptr, &a);
  return PP_OK;
}

pp_status pp_tree_attn_fwd(const pp_cache* cache, int n, const int32_t* slots, int group, const int32_t* shared, int max_new,
                           const int32_t* count, const int32_t* parents, pp_dtype dtype, int hq, int hkv, int head_dim, float scale,
                           const void* q, const void* k_pages, const void* v_pages, void* o, float* lse, int planned, void* ws,
                           size_t ws_bytes, void* hip_stream) {
  CacheView c;
  pp_status st = check_cache(cache, &c);
  if (st != PP_OK) return st;
  if ((st = check_tree(n, group, max_new, dtype, hq, hkv, head_dim)) != PP_OK) return st;
  TreeLaunch a{};
  if (!shape_tree(n, group, max_new, hq, hkv, dtype, head_dim, true, &a.shape))
    return report_error(PP_ERR_UNSUPPORTED, "the call has too many rows");
  if ((st = check_ws(ws, ws_bytes, carve_tree(a.shape, head_dim, ws, &a), "tree attention")) != PP_OK) return st;
  if (!shared) shape_tree(n, group, max_new, hq, hkv, dtype, head_dim, false, &a.shape);
  if (n == 0) return PP_OK;
  if (!q || !k_pages || !v_pages || !o || !lse)
    return report_error(PP_ERR_INVALID_ARGUMENT, "q, k_pages, v_pages, o and lse must be non-NULL");
  if (!aligned(q, 16) || !aligned(k_pages, 16) || !aligned(v_pages, 16) || !aligned(o, 16) || !aligned(lse, 4))
    return report_error(PP_ERR_INVALID_ARGUMENT, "q, k_pages, v_pages and o must be 16-byte aligned, lse 4-byte aligned");
  if ((st = check_ints({slots})) != PP_OK) return st;
  if ((st = check_optional({shared, count, parents})) != PP_OK) return st;
  a.planned = planned != 0;
  a.slots = slots;
  a.count = count;
  a.shared = shared;
  a.parents = parents;
  a.q = q;
  a.k = k_pages;
  a.v = v_pages;
  a.o = o;
  a.lse = lse;
  a.scale = scale > 0.f ? scale : 1.0f / std::sqrt((float)head_dim);
  a.head_dim = head_dim;
  a.dtype = dtype == PP_BF16 ? kBF16 : kFP32;
  a.shape.key = key_of(a.shape, c, head_dim, a.dtype);
  return launched(launch_tree_attn(c, a, (hipStream_t)hip_stream), "tree attention launch");
}

pp_status pp_verify_workspace_size(int n, int max_new, int vocab, pp_dtype dtype, size_t* bytes) {
  DraftParams p{};
  const pp_status st = shape_draft(n, max_new, vocab, 1, dtype, &p.shape);
  if (st != PP_OK) return st;
  if (!bytes) return report_error(PP_ERR_INVALID_ARGUMENT, "bytes is NULL");
  *bytes = carve_draft(&p, nullptr);
  return PP_OK;
}

pp_status pp_verify_draft(int n, int max_new, int vocab, pp_dtype dtype, int max_children, const int32_t* count,
                          const int32_t* parents, const int32_t* tokens, const void* target, const void* draft,
                          const float* temperature, const float* u, int32_t* out_count, int32_t* out_tokens, int32_t* out_path,
                          float* out_logp, void* ws, size_t ws_bytes, void* hip_stream) {
  DraftParams p{};
  pp_status st = shape_draft(n, max_new, vocab, max_children, dtype, &p.shape);
  if (st != PP_OK) return st;
  if ((st = check_ws(ws, ws_bytes, carve_draft(&p, ws), "draft verification")) != PP_OK) return st;
  if (n == 0) return PP_OK;
  const uintptr_t esz = dtype == PP_BF16 ? 2 : 4;
  if (!target) return report_error(PP_ERR_INVALID_ARGUMENT, "target is NULL");
  if (!aligned(target, esz) || !aligned(draft, esz))
    return report_error(PP_ERR_INVALID_ARGUMENT, "target and draft must be aligned to their elements");
  if ((st = check_ints({tokens, u, out_count, out_tokens, out_path, out_logp})) != PP_OK) return st;
  if ((st = check_optional({count, parents, temperature})) != PP_OK) return st;
  p.target = target;
  p.draft = draft;
  p.tokens = tokens;
  p.parents = parents;
  p.count = count;
  p.temperature = temperature;
  p.u = u;
  p.out_count = out_count;
  p.out_tokens = out_tokens;
  p.out_path = out_path;
  p.out_logp = out_logp;
  return launched(launch_verify_draft(p, dtype == PP_BF16 ? kBF16 : kFP32, (hipStream_t)hip_stream), "draft verification launch");
}

}  // extern "C"
