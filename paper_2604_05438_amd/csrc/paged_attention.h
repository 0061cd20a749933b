// What the attention kernels on the paged cache share: items and their cut into pieces, outputs, partials and their joining.
#pragma once

#include <type_traits>

#include "paged.h"

namespace tkphi {

constexpr float kLn2 = 0.69314718055994530942f;
constexpr int kJoinPairs = 2048;          // (m, l) of pieces x rows in LDS at once
constexpr int join_lds(int threads, int rows) { return (kJoinPairs + rows) * 8 > threads * 16 ? (kJoinPairs + rows) * 8 : threads * 16; }

// The weights of bf16 values are rounded to bf16 for the product O = P V, and O is divided by the sum of the weights as rounded: what a weight's rounding
// adds to the product it adds to the divisor, the output is a mean of the values it sees, off by at most 2^-8 sum p |v - y| / sum p.  (Divided by
// the sum of the weights themselves, which lse takes, a peak whose weight is no round number had its half step of 2^-8 in the output.)  A partial's O is
// multiplied by l over that sum, and goes with l from there on.
__device__ __forceinline__ float to_sum(float l, float l_rounded) { return l == 0.f ? 0.f : l * __builtin_amdgcn_rcpf(l_rounded); }

template <typename T>
__device__ __forceinline__ void store_out(const PagedGeom& g, int token_row, int head, int c, float2 o, float m, float l) {
  const float inv = l == 0.f ? 0.f : 1.f / l;                      // (l = 0: the row sees nothing, and o is 0)
  char* dst = g.out + (int64_t)token_row * g.out_row + (int64_t)head * g.out_head + c * sizeof(T);
  if constexpr (sizeof(T) == 2) *(__attribute__((address_space(1))) uint32_t*)dst = __builtin_bit_cast(uint32_t, (bf16x2_t){(__bf16)(o.x * inv), (__bf16)(o.y * inv)});
  else *(__attribute__((address_space(1))) uint64_t*)dst = (uint64_t)__float_as_uint(o.y * inv) << 32 | __float_as_uint(o.x * inv);
  if (c == 0 && g.lse) g.lse[(int64_t)token_row * g.Hq + head] = l == 0.f ? -INFINITY : (m + __builtin_amdgcn_logf(l)) * kLn2;
}

// A partial in memory: O [rows][D], then (m, l) [rows]; GPU-coherent accesses of 8 bytes
__device__ __forceinline__ void store_pair(float* p, float a, float b) {
  store_agent((uint64_t*)p, (uint64_t)__float_as_uint(b) << 32 | __float_as_uint(a));
}
// SAME: within the launch that stored it (GPU-coherent); otherwise after a kernel boundary
template <bool SAME>
__device__ __forceinline__ float2 load_pair(const float* p) {
  uint64_t v;
  if constexpr (SAME) v = load_agent((const uint64_t*)p);
  else v = *(const __attribute__((address_space(1))) uint64_t*)p;
  return make_float2(__uint_as_float((uint32_t)v), __uint_as_float((uint32_t)(v >> 32)));
}

static_assert(kJoinPairs >= kMaxSplit, "one row of the most pieces has to fit");

// Joins `pieces` partials of the rows [row0, row0 + rows) of an item, piece p at slot(p) with (m, l) behind `stride` rows.  What a thread needs
// is requested before it waits: one load after another, each to memory and back, a join of 64 pieces of one row took 30 us.
template <typename T, int D, int NT, bool SAME, typename Slot, typename RowOf>
__device__ void join_pieces(const PagedGeom& g, int pieces, int row0, int rows, int stride, char* lds, Slot&& slot, RowOf&& row_of) {
  constexpr int HALF = D / 2;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const auto finish = [&](int r, int c, float2 o, float m, float l) {          // channels c, c + 1 of row row0 + r
    int token, head;
    row_of(row0 + r, &token, &head);
    store_out<T>(g, token, head, c, o, m, l);
  };
  // Few elements (pairs of channels) of many pieces: several threads share the pieces of one; each of them gets along with one round of loads, (m, l) among them
  if (rows * HALF <= NT && pieces > 4) {
    constexpr int WIDE = 16;
    const int items = rows * HALF, share = NT / items, x = tid % items, mine = tid / items, r = x / HALF, c = x % HALF * 2;
    float4* part = (float4*)lds;
    __syncthreads();
    float m = -INFINITY, l = 0.f;
    float2 o = make_float2(0.f, 0.f);
    if (mine < share)
      for (int p0 = mine; p0 < pieces; p0 += share * WIDE) {
        float2 v[WIDE], ml[WIDE];
#pragma unroll
        for (int k = 0; k < WIDE; ++k) {
          const float* at = slot(min(p0 + k * share, pieces - 1));
          v[k] = load_pair<SAME>(at + (row0 + r) * D + c);
          ml[k] = load_pair<SAME>(at + stride * D + (row0 + r) * 2);
        }
        float mb = m;
#pragma unroll
        for (int k = 0; k < WIDE; ++k) mb = fmaxf(mb, ml[k].x);      // (the last one again past the end)
        const float ref = mb == -INFINITY ? 0.f : mb, fix = __builtin_amdgcn_exp2f(m - ref);
        m = mb;
        l *= fix; o.x *= fix; o.y *= fix;
#pragma unroll
        for (int k = 0; k < WIDE; ++k) {
          const bool in = p0 + k * share < pieces;
          const float f = __builtin_amdgcn_exp2f(ml[k].x - ref);
          l = fmaf(in ? ml[k].y : 0.f, f, l);
          o.x = fmaf(in ? v[k].x : 0.f, f, o.x);
          o.y = fmaf(in ? v[k].y : 0.f, f, o.y);
        }
      }
    part[tid] = make_float4(m, l, o.x, o.y);
    __syncthreads();
    if (mine == 0) {
      for (int k = 1; k < share; ++k) {
        const float4 other = part[k * items + x];
        const float mb = fmaxf(m, other.x), ref = mb == -INFINITY ? 0.f : mb;
        const float f = __builtin_amdgcn_exp2f(m - ref), h = __builtin_amdgcn_exp2f(other.x - ref);
        m = mb;
        l = fmaf(other.y, h, l * f);
        o.x = fmaf(other.z, h, o.x * f);
        o.y = fmaf(other.w, h, o.y * f);
      }
      finish(r, c, o, m, l);
    }
    return;
  }
  float2* ml = (float2*)lds;                                       // [rows][pieces]: (m, l), then (weight, -)
  float2* sums = ml + kJoinPairs;                                  // [rows]: m, l of the whole
  const int group = min(rows, kJoinPairs / pieces);
  for (int r0 = 0; r0 < rows; r0 += group) {
    const int n = min(group, rows - r0);
    const int items = n * HALF;
    __syncthreads();
    for (int x = tid; x < n * pieces; x += NT) ml[x] = load_pair<SAME>(slot(x % pieces) + stride * D + (row0 + r0 + x / pieces) * 2);
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
    // E elements of 16 / E pieces at a time
    const auto sum_up = [&](auto elements) {
      constexpr int E = decltype(elements)::value, P = 16 / E;
      for (int x0 = tid; x0 < items; x0 += NT * E) {
        float2 o[E];
#pragma unroll
        for (int k = 0; k < E; ++k) o[k] = make_float2(0.f, 0.f);
        for (int p0 = 0; p0 < pieces; p0 += P) {
          float2 v[P][E];
#pragma unroll
          for (int y = 0; y < P; ++y) {
            const float* at = slot(min(p0 + y, pieces - 1)) + (row0 + r0) * D;
#pragma unroll
            for (int k = 0; k < E; ++k) v[y][k] = load_pair<SAME>(at + min(x0 + k * NT, items - 1) * 2);
          }
#pragma unroll
          for (int k = 0; k < E; ++k) {
            const float2* f = ml + min(x0 + k * NT, items - 1) / HALF * pieces;
#pragma unroll
            for (int y = 0; y < P; ++y) {
              const bool in = p0 + y < pieces;
              const float weight = f[min(p0 + y, pieces - 1)].x;
              o[k].x = fmaf(in ? v[y][k].x : 0.f, weight, o[k].x);
              o[k].y = fmaf(in ? v[y][k].y : 0.f, weight, o[k].y);
            }
          }
        }
#pragma unroll
        for (int k = 0; k < E; ++k)
          if (x0 + k * NT < items) {
            const int x = x0 + k * NT, r = x / HALF;
            finish(r0 + r, x % HALF * 2, o[k], sums[r].x, sums[r].y);
          }
      }
    };
    if (pieces <= 2) sum_up(std::integral_constant<int, 8>());
    else if (pieces > 4 && items <= 2 * NT) sum_up(std::integral_constant<int, 2>());
    else sum_up(std::integral_constant<int, 4>());
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
  const int i0 = g.by_group(r0), i1 = g.by_group(r0 + it.rows - 1);
  it.end = s.cached + i1 + 1;
  it.low = g.window > 0 ? max(0, s.cached + i0 + 1 - g.window) : 0;
  it.begin = it.low >> g.unit_shift << g.unit_shift;
  return it;
}
__device__ __forceinline__ int item_units(const PagedGeom& g, const ItemRange& it) { return (it.end - it.begin + (1 << g.unit_shift) - 1) >> g.unit_shift; }

// Workgroup b of n -> its share's number: consecutive shares, which pass over the same KV head, on one XCD (workgroup b runs on XCD b % 8)
__device__ __forceinline__ int share_number(int b, int n) { return n % 8 == 0 ? b % 8 * (n / 8) + b / 8 : b; }

// A value that is the same in every lane, in scalar registers (what is loaded arrives in vector registers, and would stay there)
__device__ __forceinline__ int uniform(int x) { return __builtin_amdgcn_readfirstlane(x); }
__device__ __forceinline__ int64_t uniform(int64_t x) {
  return (int64_t)(uint32_t)__builtin_amdgcn_readfirstlane((int)(uint32_t)x) | (int64_t)__builtin_amdgcn_readfirstlane((int)(x >> 32)) << 32;
}

// The work of a call in order: KV heads outermost, then items, then units of an item, in W equal shares (the first ones one unit longer).
// PLAN: the items have been listed by paged_plan_kernel.  Otherwise there are at most 64 sequences of one item per KV head, a lane holds each,
// and the numbers fit 32 bits: a launch over short contexts lasts as long as its longest chain of instructions and loads, and 64-bit divisions, searches
// and loads one after another made 3 us of it.
template <bool PLAN>
struct Share {
  using Int = std::conditional_t<PLAN, int64_t, int>;
  Int per_head, all, begin, end, each;     // units of a KV head, of all; this workgroup's; all / W
  int W, rest;                             // workgroups; all % W
  int count;                               // planned items
  PagedSeq s;                              // (no plan) the lane's sequence, its units, and up to with it
  int units, units_incl;
  static __device__ __forceinline__ Int quotient(Int a, Int b) {
    if constexpr (PLAN) {
      if (a >> 32 || b >> 32) return a / b;
    }
    return (Int)((uint32_t)a / (uint32_t)b);
  }
  __device__ __forceinline__ Int first_of(int w) const { return each * w + min(w, rest); }
  __device__ __forceinline__ int owner(Int unit) const {                // the workgroup whose share has this unit
    const Int longer = (each + 1) * rest;
    return __builtin_amdgcn_readfirstlane((int)(unit < longer ? quotient(unit, each + 1) : rest + quotient(unit - longer, each)));
  }
};
template <bool PLAN>
__device__ __forceinline__ Share<PLAN> share_of(const PagedGeom& g, int w) {
  using Int = typename Share<PLAN>::Int;
  Share<PLAN> r;
  r.count = 0;
  r.s = PagedSeq{0, 0, 0};
  r.units = r.units_incl = 0;
  if constexpr (PLAN) {
    r.count = uniform(*g.plan_count);
    r.per_head = r.count > 0 ? uniform(g.plan_end[r.count - 1]) : 0;
  } else {
    const int lane = threadIdx.x & 63;
    if (lane < g.n_seqs) {
      r.s = check_seq(g, g.seqs[lane]);
      r.units = r.s.fresh > 0 ? item_units(g, item_range(g, r.s, 0)) : 0;
    }
    r.units_incl = wave_scan_incl(r.units);
    r.per_head = __builtin_amdgcn_readlane(r.units_incl, 63);
  }
  r.all = r.per_head * g.Hkv;
  r.W = (int)min((Int)g.splits, PLAN ? (r.all + g.least - 1) / g.least : r.all);
  r.begin = r.end = r.each = 0;
  r.rest = 0;
  if (w < r.W) {
    r.each = uniform(Share<PLAN>::quotient(r.all, r.W));
    r.rest = (int)(r.all - r.each * r.W);
    r.begin = r.first_of(w);
    r.end = r.first_of(w + 1);
  }
  return r;
}

// The part of an item that unit x and those after it, up to the end of the share, belong to
template <bool PLAN>
struct Piece {
  using Int = typename Share<PLAN>::Int;
  PagedSeq s;
  ItemRange it;
  int seq, tile, h;
  int u0, u1, units;                       // this piece's units of the item's
  Int item0, item1;                        // the item's units among all
  __device__ __forceinline__ bool whole() const { return u0 == 0 && u1 == units; }
  __device__ __forceinline__ void place(const PagedGeom& g, int row, int* token, int* head) const {
    const int r = (PLAN ? tile * g.tile_rows : 0) + row, i = g.by_group(r);
    *token = s.row + i;
    *head = h * g.G + r - i * g.G;
  }
};
// hint: the planned item before (-1: none); set to this one
template <bool PLAN>
__device__ __forceinline__ Piece<PLAN> piece_at(const PagedGeom& g, const Share<PLAN>& sh, typename Share<PLAN>::Int x, int* hint) {
  using Int = typename Share<PLAN>::Int;
  Piece<PLAN> p;
  p.h = __builtin_amdgcn_readfirstlane((int)Share<PLAN>::quotient(x, sh.per_head));
  const Int y = x - p.h * sh.per_head;
  Int before;
  if constexpr (PLAN) {
    int a = uniform(y == 0 ? 0 : *hint + 1);        // the next one; to begin with, 64 ends at a time, the first item whose end is past y
    if (*hint < 0 && y > 0) {
      int n = sh.count, step = 1;          // among items [a, a + n)
      a = 0;
      while (n > 1) {
        step = (n + 63) / 64;
        const int at = a + min(((int)(threadIdx.x & 63) + 1) * step, n) - 1;
        const uint64_t past = __ballot(g.plan_end[at] > y);
        const int k = uniform(__builtin_ctzll(past));
        n = min(step, n - k * step);
        a += k * step;
      }
    }
    *hint = a;
    const int2 it = g.plan_item[a];
    p.seq = uniform(it.x);
    p.tile = uniform(it.y);
    before = a > 0 ? uniform(g.plan_end[a - 1]) : 0;
    p.s = check_seq(g, g.seqs[p.seq]);
    p.s = PagedSeq{uniform(p.s.cached), uniform(p.s.fresh), uniform(p.s.row)};
  } else {
    p.seq = __builtin_ctzll(__ballot(sh.units_incl > y));
    p.tile = 0;
    p.s.cached = __builtin_amdgcn_readlane(sh.s.cached, p.seq);
    p.s.fresh = __builtin_amdgcn_readlane(sh.s.fresh, p.seq);
    p.s.row = __builtin_amdgcn_readlane(sh.s.row, p.seq);
    before = __builtin_amdgcn_readlane(sh.units_incl - sh.units, p.seq);
  }
  p.it = item_range(g, p.s, p.tile);
  p.units = item_units(g, p.it);
  p.u0 = __builtin_amdgcn_readfirstlane((int)(y - before));
  p.item0 = p.h * sh.per_head + before;
  p.item1 = p.item0 + p.units;
  p.u1 = (int)(min(sh.end, p.item1) - p.item0);
  return p;
}
// where workgroup w keeps its partial of the piece that starts at unit x: of its first piece, or of its last
__device__ __forceinline__ float* partial_slot(const PagedGeom& g, int w, bool first) {
  return g.partial + ((int64_t)w * 2 + (first ? 0 : 1)) * g.tile_rows * (g.d + 2);
}
// With a plan: which item, if any, paged_join_kernel joins for share w, the one that starts in it and ends in another
struct JoinRecord {
  int4 a{0, 0, 0, 0}, b{0, 0, 0, 0};       // pieces (0: none), rows, KV head, first row among the sequence's; first row of q and out, whether the share starts with it
  __device__ __forceinline__ void note(const PagedGeom& g, const Share<true>& sh, const Piece<true>& p, int w, bool first) {
    if (p.u0 > 0 || p.item1 <= sh.end) return;
    a = make_int4(sh.owner(p.item1 - 1) - w + 1, p.it.rows, p.h, p.tile * g.tile_rows);
    b = make_int4(p.s.row, first, 0, 0);
  }
  __device__ __forceinline__ void store(const PagedGeom& g, int w) const {       // by every workgroup of the launch
    if (threadIdx.x == 0) { g.joins[2 * w] = a; g.joins[2 * w + 1] = b; }
  }
};

// After this workgroup's partial of an item that is not whole is stored: the last one to arrive joins the item's pieces.  (With a plan a
// kernel of its own does, in which many workgroups share the rows of an item: paged_join_kernel.)
template <typename T, int D, int NT>
__device__ __forceinline__ void finish_item(const PagedGeom& g, const Share<false>& sh, const Piece<false>& p, char* lds, int* sh_last) {
  const int w0 = sh.owner(p.item0), w1 = sh.owner(p.item1 - 1);
  if (!last_to_arrive(g.arrived + w0, w1 - w0 + 1, sh_last)) return;
  const bool first = sh.first_of(w0) == p.item0;          // the first workgroup's share starts with this item
  join_pieces<T, D, NT, true>(g, w1 - w0 + 1, 0, p.it.rows, g.tile_rows, lds, [&](int k) { return partial_slot(g, w0 + k, k > 0 || first); },
                              [&](int row, int* token, int* head) { p.place(g, row, token, head); });
}

}  // namespace tkphi
