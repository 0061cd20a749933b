// Shared by the kernels on the paged key/value cache (paged_append, paged_attention, paged_blocks) and their host layer (paged_api).
#pragma once

#include "tkphi_internal.h"

namespace tkphi {

constexpr int kPagedThreads = 256;
constexpr int kPagedRows = 32;            // query rows (token x query head of one KV head) of a split item at most: two tiles of 16
// and of an item of the chunk kernel.  d = 128: one workgroup of 256 rows per CU; two of half the rows read every cached row twice as often (1.02
// against 0.95 ms for 2048 tokens over 30000).  d = 64, where the products are half as long and everything between them is not: three of
// 128 rows per CU, which fill each other's gaps (a prompt of 16000 tokens of a 1B layer 1.54 ms; two per CU 1.78; one of 256 rows about the same
// as three for prompts of 4000, but 65 instead of 40 us for 300 tokens over 2000: all without the sum of the rounded weights, which takes 5 %).
constexpr int chunk_rows(int d) { return d == 64 ? 128 : 256; }
constexpr int chunk_per_simd(int d) { return d == 64 ? 3 : 2; }      // wavefronts
constexpr int kMaxSplit = 1024;           // workgroups that the work of one attention call is spread over, at most
constexpr int kBlockRowGroup = 512;       // query tokens whose block scores the workspace holds at once, at most
constexpr int kMaxKept = 1024;            // blocks a query sees, at most

// Workgroups of the split kernel that a CU holds (by their registers); the work is cut into as many pieces as the GPU's 256 CUs hold, so that
// none waits for another to end: with 768 pieces where 256 ran at once the last ones ended three times later.
constexpr int attend_per_cu(int d, int row_tiles) { return d == 128 && row_tiles == 2 ? 1 : 2; }

// n / d by a multiplication, for 0 <= n < 2^31: with 2^(l-1) < d <= 2^l, ceil(2^(31 + l) / d) fits 32 bits and is exact there
struct Divisor {
  int d;
  uint32_t mul, shift;
  void set(int value) {
    int l = 0;
    value = value < 1 ? 1 : value;
    while ((1ll << l) < value) ++l;
    d = value;
    mul = (uint32_t)((((uint64_t)1 << (31 + l)) + value - 1) / value);
    shift = 31 + l;
  }
#ifdef __HIPCC__
  __host__ __device__ __forceinline__ int operator()(int n) const { return (int)(((uint64_t)(uint32_t)n * mul) >> shift); }
#endif
};

// Everything a kernel needs to know of one call, passed by value.
struct PagedGeom {
  const int4* seqs;
  const int32_t* pages;
  char *K, *V;
  const char* q;
  char* out;                              // q_rot or out
  int64_t st_page, st_head, st_tok;       // bytes
  int64_t q_row, q_head, out_row, out_head;
  uint32_t* status;
  float* lse;
  // attention: the work of all items (sequence x tile of query rows x KV head) in units of a fixed number of tokens is
  // cut into `splits` equal shares, one per workgroup
  uint32_t* arrived;                      // [kMaxSplit], of which [splits] or [row group][Hkv] are used: pieces of a split item that are done; zero between calls
  float* partial;                         // [splits][2][tile_rows][d + 2]
  int n_pages, n_seqs, max_pages, rows, max_new, max_len;
  int Hkv, G, Hq, d;
  Divisor by_page, by_group;              // tokens per page; G
  int window, splits;
  int unit_shift;                         // log2 of the tokens
  int tile_rows;                          // query rows per item
  float scale2, scale2_lo;                // score scale times log2(e), as the sum of two floats
  // the plan: items in order, where there are more than one per sequence and KV head, or many sequences
  int64_t* plan_end;                      // [items]: units up to and with this item
  int2* plan_item;                        // (sequence, tile)
  int* plan_count;
  int4* joins;                            // [splits][2] what paged_join_kernel has to know of the item that starts in a share and ends in another
  int plan_room;                          // items the plan has room for; 0: none needed
  int least;                              // units that a workgroup gets at least, with a plan
  // append
  int dtype, rot, adjacent;
  Divisor by_half, by_lines;              // rot / 2; rows per token and KV head: query heads, key, value
  const char *k, *v;
  const double* inv_freq;
  int64_t k_row, k_head, v_row, v_head;
  // blocks
  char* M;
  int block, first, last, top;
  int row0, row_group;                    // query tokens of this launch
  int max_blocks, kept;                   // bounds
  uint64_t* keys;                         // [row group][Hkv][max_blocks] order-preserving keys of the block scores; 0: not to be retrieved
  int2* list;                             // [row group][Hkv][kept] (page, block), ascending
  int4* list_head;                        // [row group][Hkv] entries, position of the query, its sequence, 0
};

void launch_paged_append(const PagedGeom& g, hipStream_t s);
void launch_paged_attention(const PagedGeom& g, hipStream_t s);
void launch_paged_chunk(const PagedGeom& g, hipStream_t s);
void launch_block_select(const PagedGeom& g, hipStream_t s);
void launch_block_attention(const PagedGeom& g, hipStream_t s);

#ifdef __HIPCC__
__device__ __forceinline__ int page_of(const PagedGeom& g, int t) { return g.by_page(t); }

// A sequence as the kernels take it: new_tokens 0 if its description is out of bounds.
struct PagedSeq {
  int cached, fresh, row;                 // tokens in the cache, new ones, first row
};
__device__ __forceinline__ PagedSeq check_seq(const PagedGeom& g, int4 w) {
  PagedSeq s{w.x, w.y, w.z};
  const bool bad = w.x < 0 || w.y < 0 || w.y > g.max_new || (int64_t)w.x + w.y > g.max_len || w.z < 0 || (int64_t)w.z + w.y > g.rows;
  if (bad) {
    s.fresh = 0;
    atomicOr(g.status, TKPHI_DEV_BAD_LENGTH);
  }
  return s;
}
// Page id of entry p of sequence i, -1 if absent (also behind the table's end); *bad: whether it is no page id
__device__ __forceinline__ int page_id(const PagedGeom& g, int i, int p, bool* bad) {
  const int id = g.pages[(int64_t)i * g.max_pages + min(p, g.max_pages - 1)];
  const bool there = p < g.max_pages, valid = (uint32_t)id < (uint32_t)g.n_pages;
  *bad = *bad || (there && !valid && id != -1);
  return there && valid ? id : -1;
}
__device__ __forceinline__ void report_pages(const PagedGeom& g, bool bad) {
  if (__any(bad) && (threadIdx.x & 63) == 0) atomicOr(g.status, TKPHI_DEV_BAD_PAGE);
}
__device__ __forceinline__ int page_id(const PagedGeom& g, int i, int p) {
  bool bad = false;
  const int id = page_id(g, i, p, &bad);
  if (bad) atomicOr(g.status, TKPHI_DEV_BAD_PAGE);
  return id;
}

// The sequence that owns unit x when sequence i has count(seq) units and they are numbered in order; wave-uniform, every wavefront by
// itself.  index: -1 if x is past the end; before: units of the sequences ahead of it.
struct FoundSeq {
  PagedSeq s;
  int index, before;
};
template <typename Count>
__device__ __forceinline__ FoundSeq find_seq(const PagedGeom& g, int x, Count&& count) {
  const int lane = threadIdx.x & 63;
  FoundSeq f;
  f.index = -1;
  int base = 0;
  for (int i0 = 0; i0 < g.n_seqs; i0 += 64) {
    PagedSeq s{0, 0, 0};
    int c = 0;
    if (i0 + lane < g.n_seqs) {
      s = check_seq(g, g.seqs[i0 + lane]);
      c = s.fresh > 0 ? count(s) : 0;
    }
    const int incl = wave_scan_incl(c);
    const int total = __builtin_amdgcn_readlane(incl, 63);
    if (x < base + total) {
      const int at = __builtin_ctzll(__ballot(base + incl > x));
      f.index = i0 + at;
      f.s.cached = __builtin_amdgcn_readlane(s.cached, at);
      f.s.fresh = __builtin_amdgcn_readlane(s.fresh, at);
      f.s.row = __builtin_amdgcn_readlane(s.row, at);
      f.before = base + __builtin_amdgcn_readlane(incl - c, at);
      return f;
    }
    base += total;
  }
  f.before = base;
  f.s = PagedSeq{0, 0, 0};
  return f;
}
// The sequence whose new tokens row x belongs to (index -1: none), wave-uniform
__device__ __forceinline__ FoundSeq find_row(const PagedGeom& g, int x) {
  const int lane = threadIdx.x & 63;
  FoundSeq f;
  f.index = -1;
  f.before = 0;
  f.s = PagedSeq{0, 0, 0};
  for (int i0 = 0; i0 < g.n_seqs; i0 += 64) {
    PagedSeq s{0, 0, 0};
    if (i0 + lane < g.n_seqs) s = check_seq(g, g.seqs[i0 + lane]);
    const uint64_t has = __ballot(s.fresh > 0 && s.row <= x && x - s.row < s.fresh);
    if (has) {
      const int at = __builtin_ctzll(has);
      f.index = i0 + at;
      f.s.cached = __builtin_amdgcn_readlane(s.cached, at);
      f.s.fresh = __builtin_amdgcn_readlane(s.fresh, at);
      f.s.row = __builtin_amdgcn_readlane(s.row, at);
      break;
    }
  }
  return f;
}
#endif

}  // namespace tkphi
