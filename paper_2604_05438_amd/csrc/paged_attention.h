// What the attention kernels on the paged cache share: items and their cut into pieces, outputs, partials and their joining.
#pragma once

#include "paged.h"

namespace tkphi {

constexpr float kLn2 = 0.69314718055994530942f;
constexpr int kJoinPairs = 2048;          // (m, l) of pieces x rows in LDS at once
constexpr int join_lds(int threads, int rows) { return (kJoinPairs + threads + rows) * 8; }

template <typename T>
__device__ __forceinline__ void store_out(const PagedGeom& g, int token_row, int head, int c, float o, float m, float l) {
  const float y = l == 0.f ? 0.f : o / l;                          // (l = 0: the row sees nothing)
  char* dst = g.out + (int64_t)token_row * g.out_row + (int64_t)head * g.out_head;
  if constexpr (sizeof(T) == 2) ((__bf16*)dst)[c] = (__bf16)y;
  else ((float*)dst)[c] = y;
  if (c == 0 && g.lse) g.lse[(int64_t)token_row * g.Hq + head] = l == 0.f ? -INFINITY : (m + log2f(l)) * kLn2;
}

// A partial in memory: O [rows][D], then (m, l) [rows]; GPU-coherent accesses of 8 bytes
__device__ __forceinline__ void store_pair(float* p, float a, float b) {
  store_agent((uint64_t*)p, (uint64_t)__float_as_uint(b) << 32 | __float_as_uint(a));
}
__device__ __forceinline__ float2 load_pair(const float* p) {
  const uint64_t v = load_agent((const uint64_t*)p);
  return make_float2(__uint_as_float((uint32_t)v), __uint_as_float((uint32_t)(v >> 32)));
}

static_assert(kJoinPairs >= kMaxSplit, "one row of the most pieces has to fit");

// Joins `pieces` partials of `rows` x D of an item, piece p at slot(p) with (m, l) behind `stride` rows; called by the last workgroup to
// arrive.  What a thread needs is requested before it waits: one load after another, each to memory and back, a join of 64 pieces
// of one row took 30 us, and one of 2 pieces of 256 rows as much.
template <typename T, int D, int NT, typename Slot, typename RowOf>
__device__ void join_pieces(const PagedGeom& g, int pieces, int rows, int stride, char* lds, Slot&& slot, RowOf&& row_of) {
  constexpr int HALF = D / 2, BATCH = 8, WIDE = 16;
  float2* ml = (float2*)lds;                                       // [rows][pieces]: (m, l), then (weight, -)
  float2* part = ml + kJoinPairs;                                  // [threads]
  float2* sums = part + NT;                                        // [rows]: m, l of the whole
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int group = min(rows, kJoinPairs / pieces);
  for (int r0 = 0; r0 < rows; r0 += group) {
    const int n = min(group, rows - r0);
    const int items = n * HALF;
    // few elements: the pieces are shared by several threads, and the first loads go out at once
    const int share = max(1, NT / items), first = tid / items;
    const bool few = items <= NT && first < share;
    float2 fv[WIDE];
    if (few) {
#pragma unroll
      for (int k = 0; k < WIDE; ++k) fv[k] = load_pair(slot(min(first + k * share, pieces - 1)) + r0 * D + tid % items * 2);
    }
    __syncthreads();
    for (int x = tid; x < n * pieces; x += NT) ml[x] = load_pair(slot(x % pieces) + stride * D + (r0 + x / pieces) * 2);
    __syncthreads();
    if (pieces <= 8) {
      for (int r = tid; r < n; r += NT) {
        float2* row = ml + r * pieces;
        float m = -INFINITY, l = 0.f;
        for (int p = 0; p < pieces; ++p) m = fmaxf(m, row[p].x);
        const float ref = m == -INFINITY ? 0.f : m;
        for (int p = 0; p < pieces; ++p) {
          const float f = __builtin_amdgcn_exp2f(row[p].x - ref);
          l = fmaf(row[p].y, f, l);
          row[p].x = f;
        }
        sums[r] = make_float2(m, l);
      }
    } else {
      for (int r = wave; r < n; r += NT / 64) {
        float2* row = ml + r * pieces;
        float m = -INFINITY, l = 0.f;
        for (int p = lane; p < pieces; p += 64) m = fmaxf(m, row[p].x);
        m = wave_max(m);
        const float ref = m == -INFINITY ? 0.f : m;
        for (int p = lane; p < pieces; p += 64) {
          const float f = __builtin_amdgcn_exp2f(row[p].x - ref);
          l = fmaf(row[p].y, f, l);
          row[p].x = f;
        }
        l = wave_sum(l);
        if (lane == 0) sums[r] = make_float2(m, l);
      }
    }
    __syncthreads();
    const auto finish = [&](int x, float2 o) {                     // element x: a row and a pair of its channels
      const int r = x / HALF, c = x % HALF;
      int token, head;
      row_of(r0 + r, &token, &head);
      store_out<T>(g, token, head, 2 * c, o.x, sums[r].x, sums[r].y);
      store_out<T>(g, token, head, 2 * c + 1, o.y, sums[r].x, sums[r].y);
    };
    if (items <= NT) {
      const int x = tid % items, r = x / HALF;
      float2 o = make_float2(0.f, 0.f);
      if (few)
        for (int p0 = first;;) {
#pragma unroll
          for (int k = 0; k < WIDE; ++k) {
            if (p0 + k * share >= pieces) continue;
            const float f = ml[r * pieces + p0 + k * share].x;
            o.x = fmaf(fv[k].x, f, o.x);
            o.y = fmaf(fv[k].y, f, o.y);
          }
          p0 += share * WIDE;
          if (p0 >= pieces) break;
#pragma unroll
          for (int k = 0; k < WIDE; ++k) fv[k] = load_pair(slot(min(p0 + k * share, pieces - 1)) + r0 * D + x * 2);
        }
      part[tid] = o;
      __syncthreads();
      if (first == 0) {
        for (int k = 1; k < share; ++k) {
          o.x += part[k * items + x].x;
          o.y += part[k * items + x].y;
        }
        finish(x, o);
      }
    } else {                                                       // many: several elements of two pieces at a time
      for (int x0 = tid; x0 < items; x0 += NT * BATCH) {
        float2 o[BATCH];
#pragma unroll
        for (int k = 0; k < BATCH; ++k) o[k] = make_float2(0.f, 0.f);
        for (int p = 0; p < pieces; p += 2) {
          const int p1 = min(p + 1, pieces - 1);
          float2 a[BATCH], b[BATCH];
#pragma unroll
          for (int k = 0; k < BATCH; ++k) {
            const int x = min(x0 + k * NT, items - 1);
            a[k] = load_pair(slot(p) + r0 * D + x * 2);
            b[k] = load_pair(slot(p1) + r0 * D + x * 2);
          }
#pragma unroll
          for (int k = 0; k < BATCH; ++k) {
            const int r = min(x0 + k * NT, items - 1) / HALF;
            const float f = ml[r * pieces + p].x, h = ml[r * pieces + p1].x;
            o[k].x = fmaf(a[k].x, f, o[k].x);
            o[k].y = fmaf(a[k].y, f, o[k].y);
            if (p1 == p) continue;
            o[k].x = fmaf(b[k].x, h, o[k].x);
            o[k].y = fmaf(b[k].y, h, o[k].y);
          }
        }
#pragma unroll
        for (int k = 0; k < BATCH; ++k)
          if (x0 + k * NT < items) finish(x0 + k * NT, o[k]);
      }
    }
  }
}

// Counts the workgroup in at *arrived (its partial is stored); true in the last of `pieces`, which leaves the count at zero.
__device__ __forceinline__ bool last_to_arrive(uint32_t* arrived, int pieces, int* sh) {
  wait_stores();                                                   // (every wavefront for its own GPU-coherent stores)
  __syncthreads();
  if (threadIdx.x == 0) {
    const bool last = atomicAdd(arrived, 1u) == (uint32_t)pieces - 1u;
    if (last) __hip_atomic_store(arrived, 0u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);      // for the next call
    *sh = last;
  }
  __syncthreads();
  return *sh != 0;
}

// units of one item (tile j of the query rows of sequence s): the tokens any of its rows can see, from a multiple of the unit on
struct ItemRange {
  int begin, low, end, rows;                                       // first token of the units, first and last one seen, query rows
};
__device__ __forceinline__ ItemRange item_range(const PagedGeom& g, const PagedSeq& s, int j) {
  ItemRange it;
  const int r0 = j * g.tile_rows;
  it.rows = min(g.tile_rows, s.fresh * g.G - r0);
  const int i0 = r0 / g.G, i1 = (r0 + it.rows - 1) / g.G;
  it.end = s.cached + i1 + 1;
  it.low = g.window > 0 ? max(0, s.cached + i0 + 1 - g.window) : 0;
  it.begin = it.low / g.unit * g.unit;
  return it;
}
__device__ __forceinline__ int item_units(const PagedGeom& g, const ItemRange& it) { return (it.end - it.begin + g.unit - 1) / g.unit; }

// Workgroup b of n -> its share's number: consecutive shares, which pass over the same KV head, on one XCD (workgroup b runs on XCD b % 8)
__device__ __forceinline__ int share_number(int b, int n) { return n % 8 == 0 ? b % 8 * (n / 8) + b / 8 : b; }

// The work of a call in order: KV heads outermost, then items, then units of an item.  Workgroup w of W takes the units
// [all w / W, all (w + 1) / W).  (Divisions of 64-bit numbers take 0.3 us each, and here they are all in a row: none where the numbers are small.)
struct Share {
  int64_t per_head, all, begin, end;       // units of a KV head, of all; this workgroup's
  int64_t each;                            // all / W
  int W, rest;                             // workgroups; all % W
  int count;                               // planned items
  PagedSeq s;                              // without a plan, for up to 64 sequences: the lane's, its units, and up to with it
  int units, units_incl;
  __device__ __forceinline__ int64_t first_of(int w) const { return each * w + (int64_t)((uint32_t)(rest * w) / (uint32_t)W); }
  // the workgroup of a unit: the last w with first_of(w) <= unit
  __device__ __forceinline__ int owner(int64_t unit) const {
    int w = min((int)((float)unit * ((float)W / (float)all)), W - 1);
    while (w > 0 && first_of(w) > unit) --w;
    while (w + 1 < W && first_of(w + 1) <= unit) ++w;
    return w;
  }
};
__device__ __forceinline__ int64_t quotient(int64_t a, int64_t b) {
  return a >> 32 ? a / b : (int64_t)((uint32_t)a / (uint32_t)b);   // (0 <= a, 0 < b; b > a if b is the larger)
}
__device__ __forceinline__ int first_item_units(const PagedGeom& g, const PagedSeq& s) { return s.fresh > 0 ? item_units(g, item_range(g, s, 0)) : 0; }
// least: units that a workgroup gets at least where there are more workgroups than that
__device__ __forceinline__ Share share_of(const PagedGeom& g, int w, int least) {
  Share r;
  r.count = 0;
  r.s = PagedSeq{0, 0, 0};
  r.units = r.units_incl = 0;
  if (g.tiles > 1) {
    r.count = *g.plan_count;
    r.per_head = r.count > 0 ? g.plan_end[r.count - 1] : 0;
  } else if (g.n_seqs <= 64) {
    const int lane = threadIdx.x & 63;
    if (lane < g.n_seqs) {
      r.s = check_seq(g, g.seqs[lane]);
      r.units = first_item_units(g, r.s);
    }
    r.units_incl = wave_scan_incl(r.units);
    r.per_head = __builtin_amdgcn_readlane(r.units_incl, 63);
  } else {
    r.per_head = find_seq(g, 0x7fffffff, [&](const PagedSeq& s) { return first_item_units(g, s); }).total;
  }
  r.all = r.per_head * g.Hkv;
  r.W = (int)min((int64_t)g.splits, (r.all + least - 1) / least);
  r.begin = r.end = r.each = 0;
  r.rest = 0;
  if (w < r.W) {
    r.each = quotient(r.all, r.W);
    r.rest = (int)(r.all - r.each * r.W);
    r.begin = r.first_of(w);
    r.end = r.first_of(w + 1);
  }
  return r;
}

// The part of an item that unit x and those after it, up to the end of the share, belong to
struct Piece {
  PagedSeq s;
  ItemRange it;
  int seq, tile, h;
  int u0, u1, units;                       // this piece's units of the item's
  int64_t item0, item1;                    // the item's units among all
  __device__ __forceinline__ bool whole() const { return u0 == 0 && u1 == units; }
  __device__ __forceinline__ void place(const PagedGeom& g, int row, int* token, int* head) const {
    const int r = tile * g.tile_rows + row, i = r / g.G;
    *token = s.row + i;
    *head = h * g.G + r - i * g.G;
  }
};
// hint: the planned item before (-1: none); set to this one
__device__ __forceinline__ Piece piece_at(const PagedGeom& g, const Share& sh, int64_t x, int* hint) {
  Piece p;
  p.h = __builtin_amdgcn_readfirstlane((int)quotient(x, sh.per_head));
  const int64_t y = x - p.h * sh.per_head;
  int64_t before;
  if (g.tiles > 1) {
    int a = y == 0 ? 0 : *hint + 1;        // the next one; to begin with, 64 ends at a time, the first item whose end is past y
    if (*hint < 0 && y > 0) {
      int n = sh.count, step = 1;          // among items [a, a + n)
      a = 0;
      while (n > 1) {
        step = (n + 63) / 64;
        const int at = a + min(((int)(threadIdx.x & 63) + 1) * step, n) - 1;
        const uint64_t past = __ballot(g.plan_end[at] > y);
        const int k = __builtin_ctzll(past);
        n = min(step, n - k * step);
        a += k * step;
      }
    }
    *hint = a;
    const int2 it = g.plan_item[a];
    p.seq = it.x; p.tile = it.y;
    before = a > 0 ? g.plan_end[a - 1] : 0;
    p.s = check_seq(g, g.seqs[p.seq]);
  } else if (g.n_seqs <= 64) {
    p.seq = __builtin_ctzll(__ballot((int64_t)sh.units_incl > y));
    p.tile = 0;
    p.s.cached = __builtin_amdgcn_readlane(sh.s.cached, p.seq);
    p.s.fresh = __builtin_amdgcn_readlane(sh.s.fresh, p.seq);
    p.s.row = __builtin_amdgcn_readlane(sh.s.row, p.seq);
    before = __builtin_amdgcn_readlane(sh.units_incl - sh.units, p.seq);
  } else {
    const FoundSeq f = find_seq(g, (int)y, [&](const PagedSeq& s) { return first_item_units(g, s); });
    p.s = f.s; p.seq = f.index; p.tile = 0;
    before = f.before;
  }
  p.it = item_range(g, p.s, p.tile);
  p.units = item_units(g, p.it);
  p.u0 = (int)(y - before);
  p.item0 = p.h * sh.per_head + before;
  p.item1 = p.item0 + p.units;
  p.u1 = (int)(min(sh.end, p.item1) - p.item0);
  return p;
}
// where workgroup w keeps its partial of the piece that starts at unit x: of its first piece, or of its last
__device__ __forceinline__ float* partial_slot(const PagedGeom& g, int w, bool first) {
  return g.partial + ((int64_t)w * 2 + (first ? 0 : 1)) * g.tile_rows * (g.d + 2);
}
// After this workgroup's partial of an item that is not whole is stored: the last one to arrive joins the item's pieces.
template <typename T, int D, int NT>
__device__ __forceinline__ void finish_item(const PagedGeom& g, const Share& sh, const Piece& p, char* lds, int* sh_last) {
  const int w0 = sh.owner(p.item0), w1 = sh.owner(p.item1 - 1);
  if (!last_to_arrive(g.arrived + w0, w1 - w0 + 1, sh_last)) return;
  const bool first = sh.first_of(w0) == p.item0;          // the first workgroup's share starts with this item
  join_pieces<T, D, NT>(g, w1 - w0 + 1, p.it.rows, g.tile_rows, lds, [&](int k) { return partial_slot(g, w0 + k, k > 0 || first); },
                    [&](int row, int* token, int* head) { p.place(g, row, token, head); });
}

}  // namespace tkphi
