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
tkphi_status check_config(const tkphi_paged_config* c, const tkphi_step* st, PagedGeom* g) {
  if (!c || !st) { set_error("cfg or step is null"); return TKPHI_EINVAL; }
  if (c->kv_dtype != TKPHI_F32 && c->kv_dtype != TKPHI_BF16) { set_error("kv_dtype=%d is not a tkphi_dtype", c->kv_dtype); return TKPHI_EINVAL; }
  if (c->n_kv_heads < 1 || c->n_kv_heads > 1024 || c->n_q_heads < 1 || c->n_q_heads % c->n_kv_heads != 0 || c->n_q_heads / c->n_kv_heads > kMaxGroup) {
    set_error("head counts %d/%d unsupported (need Hq %% Hkv == 0, ratio <= %d, Hkv <= 1024)", c->n_q_heads, c->n_kv_heads, kMaxGroup);
    return TKPHI_ESHAPE;
  }
  if (c->d_head != 64 && c->d_head != 128) { set_error("d_head=%d unsupported (64 or 128)", c->d_head); return TKPHI_ESHAPE; }
  if (!(c->score_scale > 0.f) || !std::isfinite(c->score_scale)) { set_error("score_scale=%g has to be positive and finite", c->score_scale); return TKPHI_EINVAL; }
  if (c->page_tokens < 1) { set_error("page_tokens=%d has to be positive", c->page_tokens); return TKPHI_ESHAPE; }
  const int64_t es = c->kv_dtype == TKPHI_BF16 ? 2 : 4;
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
// one per sequence and KV head, or more than 64 sequences, a lane each (64 sequences of up to 8000 tokens: 206 us without, 239 with; of up to 1000: 43 and 49).
void plan_attention(const tkphi_paged_config* c, PagedGeom* g) {
  const int64_t rows = (int64_t)g->max_new * g->G;
  const bool chunk = g->dtype == TKPHI_BF16 && rows > kPagedRows;
  g->tile_rows = chunk ? chunk_rows(g->d) : rows <= 16 ? 16 : kPagedRows;
  const int64_t tiles = std::max<int64_t>(1, up(rows, g->tile_rows));
  g->unit_shift = g->dtype == TKPHI_BF16 && !chunk ? 7 : 6;
  // at most (what counts is whether it passes 2^31: the product of all four bounds need not fit 64 bits)
  const int64_t units = std::min<int64_t>((int64_t)g->n_seqs * tiles * up(std::max(g->max_len, 1), 1 << g->unit_shift), 1ll << 31) * g->Hkv;
  g->least = 2;      // (1 or 4: 16 and 29 instead of 20 us for 16 tokens of a 3B layer alone, 51 and 47 instead of 43 for four chunks of up to 100)
  if (chunk || tiles > 1 || g->n_seqs > 64 || units >= (1ll << 31))
    g->plan_room = (int)std::min<int64_t>((int64_t)g->rows * g->G / g->tile_rows + g->n_seqs, (int64_t)g->n_seqs * tiles);
  g->splits = c->workgroups ? c->workgroups : (int)std::max<int64_t>(1, std::min<int64_t>(units, chunk ? 256 * chunk_per_simd(g->d) / (chunk_rows(g->d) / 128) : 256 * attend_per_cu(g->d, g->tile_rows / 16)));
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

// What all three calls check after the config; nothing is left to do where *empty
tkphi_status check_call(const tkphi_paged_config* c, const tkphi_step* st, const tkphi_kv_pool* pool, const void* io, void* ws, size_t ws_bytes,
                        PagedGeom* g, bool* empty) {
  tkphi_status r = check_config(c, st, g);
  if (r != TKPHI_OK) return r;
  if (!pool || !io) { set_error("pool or io is null"); return TKPHI_EINVAL; }
  if (!ws) { set_error("workspace is null"); return TKPHI_EWORKSPACE; }
  if ((uintptr_t)ws % 256 != 0) { set_error("workspace must be 256-byte aligned"); return TKPHI_EWORKSPACE; }
  *empty = st->n_seqs == 0 || st->rows == 0 || st->max_new == 0 || st->max_len == 0;
  const PagedSpace s = space_of(c, *g);
  if (ws_bytes < s.total) { set_error("workspace too small: %zu < %zu bytes", ws_bytes, s.total); return TKPHI_EWORKSPACE; }
  if (pool->n_pages < 0 || pool->reserved != 0) { set_error("pool: n_pages=%d reserved=%d", pool->n_pages, pool->reserved); return TKPHI_EINVAL; }
  if (*empty) return TKPHI_OK;
  if (pool->n_pages < 1) { set_error("pool without pages"); return TKPHI_EINVAL; }
  if ((r = check_pointer(st->seqs, "seqs", 16)) != TKPHI_OK) return r;
  if (st->max_pages < 1) { set_error("page table without entries"); return TKPHI_EINVAL; }
  if ((r = check_pointer(st->pages, "pages", 4)) != TKPHI_OK) return r;
  if ((r = check_pointer(pool->K, "K", 16)) != TKPHI_OK) return r;
  if ((r = check_pointer(pool->V, "V", 16)) != TKPHI_OK) return r;
  g->n_pages = pool->n_pages;
  g->K = (char*)pool->K; g->V = (char*)pool->V; g->M = (char*)pool->M;
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

}  // namespace
}  // namespace tkphi

using namespace tkphi;

extern "C" {

size_t tkphi_paged_workspace_bytes(const tkphi_paged_config* cfg, const tkphi_step* step) {
  PagedGeom g;
  if (check_config(cfg, step, &g) != TKPHI_OK) return 0;
  return space_of(cfg, g).total;
}

tkphi_status tkphi_kv_append(const tkphi_paged_config* cfg, const tkphi_step* step, const tkphi_kv_pool* pool, const tkphi_new_rows* io,
                             void* workspace, size_t workspace_bytes, void* hip_stream) {
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
  g.by_half.set(g.rot / 2);
  g.by_lines.set((g.q ? g.G : 0) + 2);
  (void)hipGetLastError();
  launch_paged_append(g, (hipStream_t)hip_stream);
  return hip_status(hipGetLastError(), "tkphi_kv_append launch");
}

tkphi_status tkphi_paged_attention(const tkphi_paged_config* cfg, const tkphi_step* step, const tkphi_kv_pool* pool,
                                   const tkphi_attention_rows* io, void* workspace, size_t workspace_bytes, void* hip_stream) {
  PagedGeom g;
  bool empty = false;
  tkphi_status st = check_call(cfg, step, pool, io, workspace, workspace_bytes, &g, &empty);
  if (st != TKPHI_OK || empty) return st;
  if ((st = check_attention_rows(io, &g)) != TKPHI_OK) return st;
  plan_attention(cfg, &g);
  (void)hipGetLastError();
  launch_paged_attention(g, (hipStream_t)hip_stream);
  return hip_status(hipGetLastError(), "tkphi_paged_attention launch");
}

tkphi_status tkphi_block_attention(const tkphi_paged_config* cfg, const tkphi_step* step, const tkphi_kv_pool* pool,
                                   const tkphi_attention_rows* io, void* workspace, size_t workspace_bytes, void* hip_stream) {
  PagedGeom g;
  bool empty = false;
  tkphi_status st = check_call(cfg, step, pool, io, workspace, workspace_bytes, &g, &empty);
  if (st != TKPHI_OK) return st;
  if (g.block == 0) { set_error("tkphi_block_attention needs cfg.block"); return TKPHI_EINVAL; }
  if (g.last < 1) { set_error("last_blocks=%d: a query sees its own block", g.last); return TKPHI_EINVAL; }
  if (g.window != 0) { set_error("tkphi_block_attention takes no window"); return TKPHI_EUNSUPPORTED; }
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
  return hip_status(hipGetLastError(), "tkphi_block_attention launch");
}

}  // extern "C"
