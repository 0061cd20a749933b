// Host layer of the calls on the paged key/value cache: argument checks, launch geometry, workspace, entry points.
#include <algorithm>
#include <cmath>
#include <cstring>

#include "paged.h"

namespace tkphi {
namespace {

// Bytes of the workspace's parts, in order
struct PagedSpace {
  size_t arrived, joins, partial, plan_end, plan_item, keys, list, list_head, total;
};

size_t padded(size_t x) { return (x + 255) / 256 * 256; }
int64_t up(int64_t a, int64_t b) { return (a + b - 1) / b; }

tkphi_status hip_status(hipError_t e, const char* what) {
  if (e == hipSuccess) return TKPHI_OK;
  set_error("%s: %s", what, hipGetErrorString(e));
  return TKPHI_EHIP;
}

// Config and step: everything a call and the workspace's size have in common
// (codes: strides of the pool are those of a cache in 8 bits)
tkphi_status check_config(const tkphi_paged_config* c, const tkphi_step* st, PagedGeom* g, bool codes = false) {
  if (!c || !st) { set_error("cfg or step is null"); return TKPHI_EINVAL; }
  if (c->kv_dtype != TKPHI_F32 && c->kv_dtype != TKPHI_BF16) { set_error("kv_dtype=%d is not a tkphi_dtype", c->kv_dtype); return TKPHI_EINVAL; }
  if (c->n_kv_heads < 1 || c->n_kv_heads > 1024 || c->n_q_heads < 1 || c->n_q_heads % c->n_kv_heads != 0 || c->n_q_heads / c->n_kv_heads > kMaxGroup) {
    set_error("head counts %d/%d unsupported (need Hq %% Hkv == 0, ratio <= %d, Hkv <= 1024)", c->n_q_heads, c->n_kv_heads, kMaxGroup);
    return TKPHI_ESHAPE;
  }
  if (c->d_head != 64 && c->d_head != 128) { set_error("d_head=%d unsupported (64 or 128)", c->d_head); return TKPHI_ESHAPE; }
  if (!(c->score_scale > 0.f) || !std::isfinite(c->score_scale)) { set_error("score_scale=%g has to be positive and finite", c->score_scale); return TKPHI_EINVAL; }
  if (c->page_tokens < 1) { set_error("page_tokens=%d has to be positive", c->page_tokens); return TKPHI_ESHAPE; }
  if (codes && c->kv_dtype != TKPHI_BF16) { set_error("the calls on the cache in 8 bits take bf16 rows (kv_dtype=%d)", c->kv_dtype); return TKPHI_EUNSUPPORTED; }
  const int64_t es = codes ? 1 : c->kv_dtype == TKPHI_BF16 ? 2 : 4;
  for (const int64_t s : {c->stride_page, c->stride_head, c->stride_tok})
    if (s < 0 || s > (1ll << 48) || s * es % 16 != 0) { set_error("pool stride of %lld elements (need >= 0, 16-byte multiple)", (long long)s); return TKPHI_EALIGN; }
  if ((c->page_tokens > 1 && c->stride_tok < c->d_head) || (c->n_kv_heads > 1 && c->stride_head < c->d_head)) {
    set_error("pool strides %lld (heads), %lld (tokens) below d_head", (long long)c->stride_head, (long long)c->stride_tok);
    return TKPHI_EALIGN;
  }
  if (c->window < 0) { set_error("window=%d has to be >= 0", c->window); return TKPHI_EINVAL; }
  if (c->rot_dim < 0 || c->rot_dim > c->d_head || c->rot_dim % 16 != 0 || c->rot_adjacent < 0 || c->rot_adjacent > 1) {
    set_error("rot_dim=%d (a multiple of 16 up to d_head) or rot_adjacent=%d unsupported", c->rot_dim, c->rot_adjacent);
    return TKPHI_ESHAPE;
  }
  if (c->block != 0 && ((c->block != 16 && c->block != 32 && c->block != 64) || c->page_tokens % c->block != 0)) {
    set_error("block=%d unsupported (0, 16, 32 or 64, a divisor of page_tokens=%d)", c->block, c->page_tokens);
    return TKPHI_ESHAPE;
  }
  if (c->first_blocks < 0 || c->last_blocks < 0 || c->top_blocks < 0 || (int64_t)c->first_blocks + c->last_blocks + c->top_blocks > kMaxKept) {
    set_error("first_blocks=%d last_blocks=%d top_blocks=%d out of range (sum <= %d)", c->first_blocks, c->last_blocks, c->top_blocks, kMaxKept);
    return TKPHI_EINVAL;
  }
  if (c->workgroups < 0 || c->workgroups > kMaxSplit) { set_error("workgroups=%d outside [0, %d]", c->workgroups, kMaxSplit); return TKPHI_EINVAL; }
  if (c->block > 0 && c->stride_tok * es >= (1ll << 28)) { set_error("stride_tok=%lld too large for blocks", (long long)c->stride_tok); return TKPHI_ESHAPE; }
  for (const int32_t r : c->reserved)
    if (r != 0) { set_error("reserved words of the config must be 0"); return TKPHI_EINVAL; }
  if (st->n_seqs < 0 || st->rows < 0 || st->max_new < 0 || st->max_len < 0 || st->max_pages < 0 || st->reserved != 0) {
    set_error("step: n_seqs=%d rows=%d max_new=%d max_len=%d max_pages=%d reserved=%d", st->n_seqs, st->rows, st->max_new, st->max_len, st->max_pages,
              st->reserved);
    return TKPHI_EINVAL;
  }
  if (st->n_seqs > 65535 || st->rows > (1 << 27) || st->max_len > (1 << 30) || (int64_t)st->n_seqs * (st->max_len / 16 + 2) >= (1ll << 31)) {
    set_error("step: n_seqs=%d rows=%d max_len=%d too large", st->n_seqs, st->rows, st->max_len);
    return TKPHI_ESHAPE;
  }
  memset(g, 0, sizeof(*g));
  g->Hq = c->n_q_heads; g->Hkv = c->n_kv_heads; g->G = g->Hq / g->Hkv;
  g->d = c->d_head; g->dtype = c->kv_dtype;
  g->by_page.set(c->page_tokens);
  g->by_group.set(g->G);
  g->st_page = c->stride_page * es; g->st_head = c->stride_head * es; g->st_tok = c->stride_tok * es;
  g->window = c->window; g->rot = c->rot_dim; g->adjacent = c->rot_adjacent;
  g->block = c->block; g->first = c->first_blocks; g->last = c->last_blocks; g->top = c->top_blocks;
  g->n_seqs = st->n_seqs; g->max_pages = st->max_pages; g->rows = st->rows;
  g->max_new = std::min(st->max_new, st->rows); g->max_len = st->max_len;
  g->seqs = (const int4*)st->seqs; g->pages = st->pages;
  const double s2 = (double)c->score_scale * 1.4426950408889634074;
  g->scale2 = (float)s2;
  g->scale2_lo = (float)(s2 - (double)g->scale2);
  return TKPHI_OK;
}

// Items of the attention call: query rows per item, most items per sequence and KV head, workgroups.
// Up to 32 query rows per KV head (bf16) go to the split kernel, more to the chunk kernel, the whole call by the sequence with the most: 8 sequences of a 3B
// layer with 1000 to 16000 cached tokens and 30 rows each take 88 us there and 100 in the chunk kernel, with 33 rows 127 (two items) and 87. (One sequence over
// 4000: 33 and 30 us with 30 rows, 29 and 30 with 33.)  A plan, a launch of one workgroup and one that joins, is made where items have to be numbered: more than
// one per sequence and KV head, or more than 64 sequences, a lane each (64 sequences of up to 8000 tokens: 201 us without, 203 with; of up to 1000: 40 and 43).
void plan_attention(const tkphi_paged_config* c, PagedGeom* g) {
  const int64_t rows = (int64_t)g->max_new * g->G;
  const bool chunk = g->dtype == TKPHI_BF16 && rows > kPagedRows;
  g->tile_rows = chunk ? chunk_rows(g->d) : rows <= 16 ? 16 : kPagedRows;
  const int64_t tiles = std::max<int64_t>(1, up(rows, g->tile_rows));
  g->unit_shift = g->dtype == TKPHI_BF16 && !chunk ? 7 : 6;
  // Codes of 64 channels whose heads adjoin (tokens outermost): half a cache line per row and head, which two workgroups would fetch twice.  Where the rows of two heads
  // fit one tile, an item has both: one token each of 32 sequences of 16000 to 32000 tokens 141 instead of 237 us.
  g->pairs = g->S && g->d == 64 && rows <= 8 && g->n_seqs <= 64 && g->Hkv % 2 == 0 && g->st_head == 64 && g->st_tok >= 128 && g->by_page.d % 8 == 0 && g->st_tok < (1ll << 28);
  g->item_heads = g->pairs ? g->Hkv / 2 : g->Hkv;
  // at most (what counts is whether it passes 2^31: the product of all four bounds need not fit 64 bits)
  int64_t units = std::min<int64_t>((int64_t)g->n_seqs * tiles * up(std::max(g->max_len, 1), 1 << g->unit_shift), 1ll << 31) * g->item_heads;
  if (g->pairs && units >= (1ll << 31)) { g->pairs = 0; g->item_heads = g->Hkv; units *= 2; }
  g->least = 2;      // (1 or 4: 16 and 29 instead of 20 us for 16 tokens of a 3B layer alone, 51 and 47 instead of 43 for four chunks of up to 100)
  if (chunk || tiles > 1 || g->n_seqs > 64 || units >= (1ll << 31))
    g->plan_room = (int)std::min<int64_t>((int64_t)g->rows * g->G / g->tile_rows + g->n_seqs, (int64_t)g->n_seqs * tiles);
  g->splits = c->workgroups ? c->workgroups : (int)std::max<int64_t>(1, std::min<int64_t>(units, chunk ? 256 * chunk_per_simd(g->d) / (chunk_rows(g->d) / 128) : 256 * attend_per_cu(g->d, g->tile_rows / 16)));
  // Codes of 64 channels, where 32 tokens are 2 KB and a wavefront waits for them most of the time: with 64 at a time one token of each of 32 sequences of 1000,
  // 6000 and 24000 takes 23, 46 and 135 us instead of 22, 56 and 176; one of 32000, 65000 and 131000 tokens 22.4, 23.8 and 31.9 instead of 19.3, 26.4 and 37.9.
  // (128 channels: 234 and 235 for 32 sequences, 9.2 instead of 8.2 for the small ones.)
  g->wide = g->S && g->d == 64 && !g->pairs && g->tile_rows == 16 && units >= 8ll * g->splits;
}

// Query tokens whose scores and pieces the workspace holds at once: where several workgroups share a KV head of one of them it has a
// counter, and there are kMaxSplit of those at the same place whatever the step (they are zero between calls, and what follows them is not)
constexpr int kBlockSplitHeads = 512;     // without config.workgroups: KV heads of query tokens from which on each has one workgroup
static_assert(kBlockSplitHeads <= kMaxSplit, "the heads that several workgroups share have a counter each");
int block_row_group(const tkphi_paged_config* c) { return c->workgroups > 1 ? std::min(kBlockRowGroup, kMaxSplit / c->n_kv_heads) : kBlockRowGroup; }

void plan_blocks(const tkphi_paged_config* c, PagedGeom* g) {
  if (!g->block) return;
  g->max_blocks = (int)up(g->max_len, g->block);
  g->kept = std::max(1, std::min(g->first + g->last + g->top, std::max(g->max_blocks, 1)));
  const int64_t tiles = up((int64_t)g->kept * g->block, kPagedThreads / 64 * (g->dtype == TKPHI_BF16 ? 32 : 16));
  const int64_t heads = std::max<int64_t>(1, (int64_t)g->Hkv * g->row_group);
  g->splits = c->workgroups ? std::min(c->workgroups, 64) : (int)std::max<int64_t>(1, std::min(tiles, up(kBlockSplitHeads, heads)));
}

// Rows of partials that the attention of any step within these bounds needs: two per workgroup, of as many rows as an item of its kernel has.  Fewer new
// tokens may take another kernel with shorter items and more workgroups; within one kernel all grows with all bounds.
size_t partial_rows(const tkphi_paged_config* c, const PagedGeom& bound) {
  size_t most = 0;
  for (const int tokens : {16 / bound.G, kPagedRows / bound.G, bound.max_new}) {
    PagedGeom g = bound;
    g.max_new = std::min(g.max_new, tokens);
    plan_attention(c, &g);
    most = std::max(most, (size_t)g.splits * 2 * g.tile_rows);
  }
  return most;
}

// The largest need of any step within these bounds: every part grows with every bound, but for the block attention's partials, whose number of
// workgroups per head shrinks with the rows (their product stays below that of the heads, and 512, together)
PagedSpace space_of(const tkphi_paged_config* c, const PagedGeom& g0) {
  PagedGeom g = g0;
  PagedSpace s;
  const size_t row_bytes = (size_t)(g.d + 2) * sizeof(float);
  const int rg = std::min(g.rows, block_row_group(c));
  const int64_t heads = (int64_t)rg * g.Hkv;
  const int64_t items = (int64_t)g.rows * g.G / 16 + g.n_seqs;        // (a plan is at most that long, whichever kernel runs)
  int64_t block_slots = 0;
  if (g.block) {
    g.row_group = 1;                                                  // as many workgroups per head as there may be
    plan_blocks(c, &g);
    block_slots = c->workgroups ? heads * g.splits : std::min(heads * g.splits, heads + kBlockSplitHeads);
  }
  s.arrived = 256;
  s.joins = s.arrived + padded(kMaxSplit * sizeof(uint32_t));
  s.partial = s.joins + padded(kMaxSplit * 2 * sizeof(int4));
  s.plan_end = s.partial + padded(std::max<size_t>(partial_rows(c, g0), (size_t)block_slots * 16) * row_bytes);
  s.plan_item = s.plan_end + padded((size_t)items * sizeof(int64_t));
  s.keys = s.plan_item + padded((size_t)items * sizeof(int2) + 256);
  s.list = s.keys + padded(g.block ? (size_t)heads * g.max_blocks * sizeof(uint64_t) : 0);
  s.list_head = s.list + padded(g.block ? (size_t)heads * g.kept * sizeof(int2) : 0);
  s.total = s.list_head + padded(g.block ? (size_t)heads * sizeof(int4) : 0);
  return s;
}

tkphi_status check_pointer(const void* p, const char* name, size_t align) {
  if (!p) { set_error("%s is null", name); return TKPHI_EINVAL; }
  if ((uintptr_t)p % align != 0) { set_error("%s not %zu-byte aligned", name, align); return TKPHI_EALIGN; }
  return TKPHI_OK;
}

// strides of rows that are read or written (elements -> bytes)
tkphi_status check_rows(const PagedGeom& g, const void* p, const char* name, int heads, int64_t row, int64_t head, int64_t* row_bytes, int64_t* head_bytes) {
  const int64_t es = g.dtype == TKPHI_BF16 ? 2 : 4;
  const tkphi_status st = check_pointer(p, name, 16);
  if (st != TKPHI_OK) return st;
  if (row < 0 || head < 0 || row > (1ll << 40) || head > (1ll << 40) || row * es % 16 != 0 || head * es % 16 != 0 || (heads > 1 && head < g.d) ||
      (g.rows > 1 && row < g.d)) {
    set_error("%s: strides %lld (rows), %lld (heads) invalid (>= d_head, 16-byte multiples)", name, (long long)row, (long long)head);
    return TKPHI_EALIGN;
  }
  *row_bytes = row * es;
  *head_bytes = head * es;
  return TKPHI_OK;
}

// A pool of either kind: scales null for one of the rows' type
struct Pool {
  bool codes, given;
  void *K, *V, *S, *M;
  int32_t n_pages, reserved;
};
Pool pool_of(const tkphi_kv_pool* p) { return p ? Pool{false, true, p->K, p->V, nullptr, p->M, p->n_pages, p->reserved} : Pool{}; }
Pool pool_of(const tkphi_quant_pool* p) { return p ? Pool{true, true, p->K, p->V, p->scales, p->M, p->n_pages, p->reserved} : Pool{true}; }

// What all calls check after the config; nothing is left to do where *empty
tkphi_status check_call(const tkphi_paged_config* c, const tkphi_step* st, const Pool& pool, const void* io, void* ws, size_t ws_bytes,
                        PagedGeom* g, bool* empty) {
  tkphi_status r = check_config(c, st, g, pool.codes);
  if (r != TKPHI_OK) return r;
  if (!pool.given || !io) { set_error("pool or io is null"); return TKPHI_EINVAL; }
  if (!ws) { set_error("workspace is null"); return TKPHI_EWORKSPACE; }
  if ((uintptr_t)ws % 256 != 0) { set_error("workspace must be 256-byte aligned"); return TKPHI_EWORKSPACE; }
  *empty = st->n_seqs == 0 || st->rows == 0 || st->max_new == 0 || st->max_len == 0;
  const PagedSpace s = space_of(c, *g);
  if (ws_bytes < s.total) { set_error("workspace too small: %zu < %zu bytes", ws_bytes, s.total); return TKPHI_EWORKSPACE; }
  if (pool.n_pages < 0 || pool.reserved != 0) { set_error("pool: n_pages=%d reserved=%d", pool.n_pages, pool.reserved); return TKPHI_EINVAL; }
  if (*empty) return TKPHI_OK;
  if (pool.n_pages < 1) { set_error("pool without pages"); return TKPHI_EINVAL; }
  if ((r = check_pointer(st->seqs, "seqs", 16)) != TKPHI_OK) return r;
  if (st->max_pages < 1) { set_error("page table without entries"); return TKPHI_EINVAL; }
  if ((r = check_pointer(st->pages, "pages", 4)) != TKPHI_OK) return r;
  if ((r = check_pointer(pool.K, "K", 16)) != TKPHI_OK) return r;
  if ((r = check_pointer(pool.V, "V", 16)) != TKPHI_OK) return r;
  if (pool.codes && (r = check_pointer(pool.S, "scales", 16)) != TKPHI_OK) return r;
  g->n_pages = pool.n_pages;
  g->S = (uint16_t*)pool.S;
  g->K = (char*)pool.K; g->V = (char*)pool.V; g->M = (char*)pool.M;
  char* w = (char*)ws;
  g->status = (uint32_t*)w;
  g->plan_count = (int*)(w + s.keys - 256);
  g->arrived = (uint32_t*)(w + s.arrived);
  g->joins = (int4*)(w + s.joins);
  g->partial = (float*)(w + s.partial);
  g->plan_end = (int64_t*)(w + s.plan_end);
  g->plan_item = (int2*)(w + s.plan_item);
  g->keys = (uint64_t*)(w + s.keys);
  g->list = (int2*)(w + s.list);
  g->list_head = (int4*)(w + s.list_head);
  return TKPHI_OK;
}

tkphi_status check_attention_rows(const tkphi_attention_rows* io, PagedGeom* g) {
  tkphi_status r = check_rows(*g, io->q, "q", g->Hq, io->q_row, io->q_head, &g->q_row, &g->q_head);
  if (r == TKPHI_OK) r = check_rows(*g, io->out, "out", g->Hq, io->out_row, io->out_head, &g->out_row, &g->out_head);
  if (r != TKPHI_OK) return r;
  if ((uintptr_t)io->lse % 4 != 0) { set_error("lse misaligned"); return TKPHI_EALIGN; }
  g->q = (const char*)io->q;
  g->out = (char*)io->out;
  g->lse = io->lse;
  return TKPHI_OK;
}

tkphi_status check_norms(const tkphi_head_norms* n, PagedGeom* g) {
  if (!(n->eps >= 1.17549435e-38f) || !std::isfinite(n->eps)) { set_error("eps=%g has to be positive and finite", n->eps); return TKPHI_EINVAL; }
  if (!std::isfinite(n->weight_offset)) { set_error("weight_offset=%g has to be finite", n->weight_offset); return TKPHI_EINVAL; }
  const int64_t es = g->dtype == TKPHI_BF16 ? 2 : 4;
  const struct { const void* w; int64_t head; const char* name; } both[] = {{n->q_weight, n->q_weight_head, "q_weight"}, {n->k_weight, n->k_weight_head, "k_weight"}};
  for (const auto& x : both) {
    if ((uintptr_t)x.w % 16 != 0 || x.head < 0 || x.head > (1ll << 40) || x.head * es % 16 != 0 || (x.head > 0 && x.head < g->d)) {
      set_error("%s: misaligned, or stride %lld between heads (0 or >= d_head, 16-byte multiples)", x.name, (long long)x.head);
      return TKPHI_EALIGN;
    }
  }
  g->normed = 1;
  g->eps = n->eps;
  g->w_offset = n->weight_offset;
  g->qw = (const char*)n->q_weight; g->kw = (const char*)n->k_weight;
  g->qw_head = n->q_weight_head * es; g->kw_head = n->k_weight_head * es;
  return TKPHI_OK;
}

tkphi_status append(const tkphi_paged_config* cfg, const tkphi_step* step, const Pool& pool, const tkphi_new_rows* io, const tkphi_head_norms* norms,
                    void* workspace, size_t workspace_bytes, void* hip_stream, const char* what) {
  PagedGeom g;
  bool empty = false;
  tkphi_status st = check_call(cfg, step, pool, io, workspace, workspace_bytes, &g, &empty);
  if (st != TKPHI_OK || empty) return st;
  if ((st = check_rows(g, io->k, "k", g.Hkv, io->k_row, io->k_head, &g.k_row, &g.k_head)) != TKPHI_OK) return st;
  if ((st = check_rows(g, io->v, "v", g.Hkv, io->v_row, io->v_head, &g.v_row, &g.v_head)) != TKPHI_OK) return st;
  if (!io->q != !io->q_rot) { set_error("q and q_rot: both or neither"); return TKPHI_EINVAL; }
  if (io->q) {
    if ((st = check_rows(g, io->q, "q", g.Hq, io->q_row, io->q_head, &g.q_row, &g.q_head)) != TKPHI_OK) return st;
    if ((st = check_rows(g, io->q_rot, "q_rot", g.Hq, io->q_rot_row, io->q_rot_head, &g.out_row, &g.out_head)) != TKPHI_OK) return st;
  }
  if (g.rot > 0 && (st = check_pointer(io->inv_freq, "inv_freq", 8)) != TKPHI_OK) return st;
  if (g.block > 0 && (st = check_pointer(g.M, "M", 16)) != TKPHI_OK) return st;
  g.q = (const char*)io->q; g.k = (const char*)io->k; g.v = (const char*)io->v;
  g.out = (char*)io->q_rot;
  g.inv_freq = io->inv_freq;
  if (norms && (st = check_norms(norms, &g)) != TKPHI_OK) return st;
  g.by_half.set(g.rot / 2);
  g.by_lines.set((g.q ? g.G : 0) + 2);
  (void)hipGetLastError();
  launch_paged_append(g, (hipStream_t)hip_stream);
  return hip_status(hipGetLastError(), what);
}

tkphi_status attend(const tkphi_paged_config* cfg, const tkphi_step* step, const Pool& pool, const tkphi_attention_rows* io, void* workspace,
                    size_t workspace_bytes, void* hip_stream, const char* what) {
  PagedGeom g;
  bool empty = false;
  tkphi_status st = check_call(cfg, step, pool, io, workspace, workspace_bytes, &g, &empty);
  if (st != TKPHI_OK || empty) return st;
  if ((st = check_attention_rows(io, &g)) != TKPHI_OK) return st;
  plan_attention(cfg, &g);
  (void)hipGetLastError();
  launch_paged_attention(g, (hipStream_t)hip_stream);
  return hip_status(hipGetLastError(), what);
}

tkphi_status attend_blocks(const tkphi_paged_config* cfg, const tkphi_step* step, const Pool& pool, const tkphi_attention_rows* io, void* workspace,
                           size_t workspace_bytes, void* hip_stream, const char* name) {
  PagedGeom g;
  bool empty = false;
  tkphi_status st = check_call(cfg, step, pool, io, workspace, workspace_bytes, &g, &empty);
  if (st != TKPHI_OK) return st;
  if (g.block == 0) { set_error("%s needs cfg.block", name); return TKPHI_EINVAL; }
  if (g.last < 1) { set_error("last_blocks=%d: a query sees its own block", g.last); return TKPHI_EINVAL; }
  if (g.window != 0) { set_error("%s takes no window", name); return TKPHI_EUNSUPPORTED; }
  if (empty) return TKPHI_OK;
  if ((st = check_attention_rows(io, &g)) != TKPHI_OK) return st;
  if ((st = check_pointer(g.M, "M", 16)) != TKPHI_OK) return st;
  g.lse = nullptr;
  (void)hipGetLastError();
  const int group = block_row_group(cfg);
  for (g.row0 = 0; g.row0 < g.rows; g.row0 += group) {
    g.row_group = std::min(group, g.rows - g.row0);
    plan_blocks(cfg, &g);
    launch_block_select(g, (hipStream_t)hip_stream);
    launch_block_attention(g, (hipStream_t)hip_stream);
  }
  return hip_status(hipGetLastError(), name);
}

}  // namespace
}  // namespace tkphi

using namespace tkphi;

extern "C" {

size_t tkphi_paged_workspace_bytes(const tkphi_paged_config* cfg, const tkphi_step* step) {
  PagedGeom g;
  // (strides of codes pass as strides of bf16 rows, but for tokens of 2^27 and more that are taken by blocks)
  if (check_config(cfg, step, &g) != TKPHI_OK && (!cfg || cfg->kv_dtype != TKPHI_BF16 || check_config(cfg, step, &g, true) != TKPHI_OK)) return 0;
  return space_of(cfg, g).total;
}

tkphi_status tkphi_kv_append(const tkphi_paged_config* cfg, const tkphi_step* step, const tkphi_kv_pool* pool, const tkphi_new_rows* io,
                             void* workspace, size_t workspace_bytes, void* hip_stream) {
  return append(cfg, step, pool_of(pool), io, nullptr, workspace, workspace_bytes, hip_stream, "tkphi_kv_append launch");
}

tkphi_status tkphi_norm_append(const tkphi_paged_config* cfg, const tkphi_step* step, const tkphi_kv_pool* pool, const tkphi_new_rows* io,
                               const tkphi_head_norms* norms, void* workspace, size_t workspace_bytes, void* hip_stream) {
  if (!norms) { set_error("norms is null"); return TKPHI_EINVAL; }
  return append(cfg, step, pool_of(pool), io, norms, workspace, workspace_bytes, hip_stream, "tkphi_norm_append launch");
}

tkphi_status tkphi_quant_append(const tkphi_paged_config* cfg, const tkphi_step* step, const tkphi_quant_pool* pool, const tkphi_new_rows* io,
                                const tkphi_head_norms* norms, void* workspace, size_t workspace_bytes, void* hip_stream) {
  return append(cfg, step, pool_of(pool), io, norms, workspace, workspace_bytes, hip_stream, "tkphi_quant_append launch");
}

tkphi_status tkphi_paged_attention(const tkphi_paged_config* cfg, const tkphi_step* step, const tkphi_kv_pool* pool,
                                   const tkphi_attention_rows* io, void* workspace, size_t workspace_bytes, void* hip_stream) {
  return attend(cfg, step, pool_of(pool), io, workspace, workspace_bytes, hip_stream, "tkphi_paged_attention launch");
}

tkphi_status tkphi_quant_attention(const tkphi_paged_config* cfg, const tkphi_step* step, const tkphi_quant_pool* pool,
                                   const tkphi_attention_rows* io, void* workspace, size_t workspace_bytes, void* hip_stream) {
  return attend(cfg, step, pool_of(pool), io, workspace, workspace_bytes, hip_stream, "tkphi_quant_attention launch");
}

tkphi_status tkphi_block_attention(const tkphi_paged_config* cfg, const tkphi_step* step, const tkphi_kv_pool* pool,
                                   const tkphi_attention_rows* io, void* workspace, size_t workspace_bytes, void* hip_stream) {
  return attend_blocks(cfg, step, pool_of(pool), io, workspace, workspace_bytes, hip_stream, "tkphi_block_attention");
}

tkphi_status tkphi_quant_block_attention(const tkphi_paged_config* cfg, const tkphi_step* step, const tkphi_quant_pool* pool,
                                         const tkphi_attention_rows* io, void* workspace, size_t workspace_bytes, void* hip_stream) {
  return attend_blocks(cfg, step, pool_of(pool), io, workspace, workspace_bytes, hip_stream, "tkphi_quant_block_attention");
}

tkphi_status tkphi_quant_read(const tkphi_paged_config* cfg, const tkphi_step* step, const tkphi_quant_pool* pool, const tkphi_read_rows* io,
                              void* workspace, size_t workspace_bytes, void* hip_stream) {
  PagedGeom g;
  bool empty = false;
  tkphi_status st = check_call(cfg, step, pool_of(pool), io, workspace, workspace_bytes, &g, &empty);
  if (st != TKPHI_OK || empty) return st;
  if (!io->k && !io->v) { set_error("k and v are null"); return TKPHI_EINVAL; }
  if (io->k && (st = check_rows(g, io->k, "k", g.Hkv, io->k_row, io->k_head, &g.k_row, &g.k_head)) != TKPHI_OK) return st;
  if (io->v && (st = check_rows(g, io->v, "v", g.Hkv, io->v_row, io->v_head, &g.v_row, &g.v_head)) != TKPHI_OK) return st;
  g.k_out = (char*)io->k;
  g.v_out = (char*)io->v;
  (void)hipGetLastError();
  launch_paged_read(g, (hipStream_t)hip_stream);
  return hip_status(hipGetLastError(), "tkphi_quant_read launch");
}

}  // extern "C"
