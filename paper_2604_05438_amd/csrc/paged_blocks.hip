// Selection of tkphi_block_attention: per query token and KV head the blocks whose mean keys score highest.
//
// score(b) = max over the KV head's query heads of q . M_b.  Which blocks a query sees is a yes or no, so the scores are sums in 64 bits (products of two
// bf16 are exact there, of two fp32 too), compared as order-preserving 64-bit keys, equal ones by the lower block.
#include <type_traits>

#include "paged.h"
#include "select_utils.h"

namespace tkphi {

// Order-preserving key of a score, 0 for what is not retrieved (NaN, -inf)
__device__ __forceinline__ uint64_t score_key64(double x) {
  if (!(x > -INFINITY)) return 0ull;
  const uint64_t b = __builtin_bit_cast(uint64_t, x + 0.0);        // (-0 and 0 are equal)
  return b >> 63 ? ~b : b | 0x8000000000000000ull;
}

__device__ __forceinline__ double quad_sum(double x) {             // over 4 neighbouring lanes, in every one
  const auto move = [](double y, auto ctrl) {
    const uint64_t b = __builtin_bit_cast(uint64_t, y);
    return __builtin_bit_cast(double, (uint64_t)dpp_move<decltype(ctrl)::value>((uint32_t)b) | (uint64_t)dpp_move<decltype(ctrl)::value>((uint32_t)(b >> 32)) << 32);
  };
  x += move(x, std::integral_constant<int, 0xB1>());               // quad_perm [1, 0, 3, 2]
  return x + move(x, std::integral_constant<int, 0x4E>());         // quad_perm [2, 3, 0, 1]
}

// A lane takes a quarter of the channels of two blocks; the queries, 64-bit numbers in LDS, are read once for both.  Bound by the 64-bit
// arithmetic, the sums over lanes among it (an eighth of the channels of four blocks per lane: 15 us for the 16 sequences of a 1B layer, over 38000 blocks;
// a quarter of two: 11), and by the means' rows of 128 bytes.
constexpr int kScoreLanes = 4, kScoreEach = 2;
constexpr int kScoreBlocks = kPagedThreads / kScoreLanes * kScoreEach;         // per pass of a workgroup
template <typename T, int D>
__global__ __launch_bounds__(kPagedThreads) void block_score_kernel(PagedGeom g, int blocks_per_wg) {
  constexpr int EPL = Elem<T>::per16, C = D / kScoreLanes, PAD = 2;            // channels per lane
  __shared__ __align__(16) double q[kMaxGroup][kScoreLanes * (C + PAD)];
  const int h = blockIdx.y, local = blockIdx.z, token = g.row0 + local, tid = threadIdx.x;
  const FoundSeq f = find_row(g, token);
  if (f.index < 0) return;
  const int pos = f.s.cached + token - f.s.row, have = pos / g.block + 1;
  if (have <= g.kept) return;                                      // it sees all of them
  const int lo = max(g.first, (int)blockIdx.x * blocks_per_wg), hi = min(have - g.last, ((int)blockIdx.x + 1) * blocks_per_wg);
  if (lo >= hi) return;
  const int part = tid % kScoreLanes, per = g.by_page.d / g.block;
  uint64_t* keys = g.keys + ((int64_t)local * g.Hkv + h) * g.max_blocks;
  bool staged = false;
  for (int b0 = lo; b0 < hi; b0 += kScoreBlocks) {
    // blocks b0 + tid / 4 + 64 k
    int id[kScoreEach];
    u32x4 u[kScoreEach][C / EPL];
#pragma unroll
    for (int k = 0; k < kScoreEach; ++k) {
      const int b = b0 + tid / kScoreLanes + k * (kPagedThreads / kScoreLanes);
      id[k] = b < hi ? page_id(g, f.index, b / per) : -1;
    }
#pragma unroll
    for (int k = 0; k < kScoreEach; ++k) {
      const int b = b0 + tid / kScoreLanes + k * (kPagedThreads / kScoreLanes);
      const char* src = g.M + ((((int64_t)max(id[k], 0) * g.Hkv + h) * per + b % per) * D + part * C) * sizeof(T);
#pragma unroll
      for (int j = 0; j < C / EPL; ++j) u[k][j] = gload128(src + j * 16);
    }
    if (!staged) {
      for (int i = tid; i < g.G * D; i += kPagedThreads) {
        const int a = i / D, c = i % D;
        q[a][c / C * (C + PAD) + c % C] = (double)Elem<T>::load1(g.q + (int64_t)token * g.q_row + (int64_t)(h * g.G + a) * g.q_head, c);
      }
      __syncthreads();
      staged = true;
    }
    double best[kScoreEach];
    bool nan[kScoreEach];
#pragma unroll
    for (int k = 0; k < kScoreEach; ++k) { best[k] = -INFINITY; nan[k] = false; }
#pragma unroll
    for (int a = 0; a < kMaxGroup; ++a) {
      if (a >= g.G) break;
      double sum[kScoreEach];
#pragma unroll
      for (int k = 0; k < kScoreEach; ++k) sum[k] = 0.0;
#pragma unroll
      for (int j = 0; j < C / EPL; ++j) {
        double y[EPL];
#pragma unroll
        for (int e = 0; e < EPL; ++e) y[e] = q[a][part * (C + PAD) + j * EPL + e];
#pragma unroll
        for (int k = 0; k < kScoreEach; ++k) {
          float x[EPL];
          Elem<T>::unpack(make_uint4(u[k][j].x, u[k][j].y, u[k][j].z, u[k][j].w), x);
#pragma unroll
          for (int e = 0; e < EPL; ++e) sum[k] = fma((double)x[e], y[e], sum[k]);
        }
      }
#pragma unroll
      for (int k = 0; k < kScoreEach; ++k) {
        const double s = quad_sum(sum[k]);
        nan[k] = nan[k] || s != s;
        best[k] = s > best[k] ? s : best[k];
      }
    }
#pragma unroll
    for (int k = 0; k < kScoreEach; ++k) {
      const int b = b0 + tid / kScoreLanes + k * (kPagedThreads / kScoreLanes);
      if (part == 0 && b < hi) keys[b] = nan[k] || id[k] < 0 ? 0ull : score_key64(best[k]);
    }
  }
}

// The edge of a selection: taken are keys > edge and, of those equal to it, the first `ties`
struct Edge {
  uint64_t key;
  int ties;
};

// Up to kHeld keys per thread, thread t's k-th being number t + k kSelThreads: a histogram over 32 octaves of the score by sign and five
// bits each (of a leading digit nearly all would share a few bins), then the exact order within the bin of the edge.
// false: that bin holds more than fits (the caller sorts digit by digit).
constexpr int kHeld = 8, kScoreBins = 2048;
struct HeldScratch {
  uint32_t hist[kScoreBins];
  uint64_t cand[kSelThreads];
  int cand_at[kSelThreads];
  int scan[16];
  int bin, need, n_cand;
  Edge edge;
};
__device__ __forceinline__ int score_bin(uint64_t key) {           // monotone in the key
  const bool pos = key >> 63;
  const uint64_t mag = (pos ? key : ~key) & 0x7fffffffffffffffull;
  const int e = (int)(mag >> 52) - (1023 - 16), m = (int)(mag >> 47) & 31;
  const int b = e < 0 ? 0 : e > 31 ? 1023 : e * 32 + m;
  return pos ? 1024 + b : 1023 - b;
}
// rounds: how many of the kHeld are in use
__device__ __forceinline__ bool find_edge(const uint64_t (&key)[kHeld], int rounds, int want, HeldScratch& sh, Edge* edge) {
  const int tid = threadIdx.x;
#pragma unroll
  for (int k = 0; k < kScoreBins / kSelThreads; ++k) sh.hist[tid + k * kSelThreads] = 0;
  if (tid == 0) sh.n_cand = 0;
  lds_barrier();
  int bin[kHeld];
#pragma unroll
  for (int k = 0; k < kHeld; ++k) {
    if (k >= rounds) break;
    bin[k] = score_bin(key[k]);
    if (key[k]) atomicAdd(&sh.hist[bin[k]], 1u);
  }
  lds_barrier();
  // thread t looks at the two bins from the top: number of keys in the bins above
  const int b1 = kScoreBins - 1 - 2 * tid;
  const int c1 = (int)sh.hist[b1], c0 = (int)sh.hist[b1 - 1];
  const int incl = sel_scan_incl(c0 + c1, sh.scan), above = incl - c0 - c1;
  if (above < want && want <= incl) {
    const bool first = want <= above + c1;
    sh.bin = first ? b1 : b1 - 1;
    sh.need = want - above - (first ? 0 : c1);
  }
  if (tid == kSelThreads - 1 && incl < want) sh.bin = -1;          // all of them (where exactly `want` compete, the edge is the last of them)
  lds_barrier();
  const int edge_bin = sh.bin, need = sh.need;
  if (edge_bin < 0) return true;
  const int count = (int)sh.hist[edge_bin];
  if (count > kSelThreads) return false;
#pragma unroll
  for (int k = 0; k < kHeld; ++k) {
    if (k >= rounds) break;
    if (key[k] && bin[k] == edge_bin) {
      const int at = atomicAdd(&sh.n_cand, 1);
      sh.cand[at] = key[k];
      sh.cand_at[at] = tid + k * kSelThreads;
    }
  }
  lds_barrier();
  if (tid < count) {                                               // the need-th of the bin, equal keys by number
    const uint64_t mine = sh.cand[tid];
    const int at = sh.cand_at[tid];
    int ahead = 0, same = 0;
    for (int j = 0; j < count; ++j) {
      const uint64_t other = sh.cand[j];
      ahead += other > mine;
      same += other == mine && sh.cand_at[j] < at;
    }
    if (ahead + same == need - 1) sh.edge = Edge{mine, same + 1};
  }
  lds_barrier();
  *edge = sh.edge;
  return true;
}

// One workgroup per query token and KV head: the blocks it sees, ascending
__global__ __launch_bounds__(kSelThreads) void block_select_kernel(PagedGeom g) {
  __shared__ HeldScratch sh;
  __shared__ int want_sh, counted[kHeld * 16];
  __shared__ uint64_t prefix;
  const int h = blockIdx.x, local = blockIdx.y, token = g.row0 + local, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int64_t at = (int64_t)local * g.Hkv + h;
  const FoundSeq f = find_row(g, token);
  if (f.index < 0) {
    if (tid == 0) g.list_head[at] = make_int4(0, 0, 0, 0);
    return;
  }
  const int pos = f.s.cached + token - f.s.row, have = pos / g.block + 1, per = g.by_page.d / g.block;
  const int lo = g.first, hi = have - g.last, n = hi - lo;         // blocks [lo, hi) compete
  const bool all = have <= g.kept;
  const uint64_t* keys = g.keys + at * g.max_blocks + lo;
  int2* list = g.list + at * g.kept;
  Edge edge{1ull, 0x7fffffff};                                     // (all that are eligible)
  uint64_t key[kHeld];
  int page[kHeld];
  const bool held = n <= kHeld * kSelThreads;
  const int rounds = held ? (n + kSelThreads - 1) / kSelThreads : kHeld;
  if (!all) {
    if (held) {
#pragma unroll
      for (int k = 0; k < kHeld; ++k) {
        if (k >= rounds) break;
        const int j = tid + k * kSelThreads;
        key[k] = j < n && g.top > 0 ? keys[j] : 0ull;
        page[k] = j < n ? page_id(g, f.index, (lo + j) / per) : -1;
      }
    }
    if (g.top == 0) {
      edge = Edge{~0ull, 0};
    } else if (!(held && find_edge(key, rounds, g.top, sh, &edge))) {
      int eligible = 0;
      for (int j = tid; j < n; j += kSelThreads) eligible += keys[j] != 0ull;
      eligible = wave_sum(eligible);
      if (lane == 0) counted[wave] = eligible;
      lds_barrier();
      eligible = wave_sum(lane < 16 ? counted[lane] : 0);
      lds_barrier();
      if (eligible > g.top) {
        edge.key = radix_select_desc(n, g.top, [&](int j, uint64_t* v) { *v = keys[j]; return *v != 0ull; }, sh.hist, sh.scan, &prefix, &want_sh);
        edge.ties = want_sh;
      }
    }
  }
  // Ascending list: first blocks, taken ones of [lo, hi), last blocks.  All blocks in order where it sees all.
  const int front = all ? have : lo;
  for (int b = tid; b < front; b += kSelThreads) list[b] = make_int2(page_id(g, f.index, b / per), b);
  int count = front, equal = 0;
  if (!all) {
    for (int j0 = 0; j0 < n; j0 += kHeld * kSelThreads) {          // (once where the keys are held)
      if (!held) {
#pragma unroll
        for (int k = 0; k < kHeld; ++k) {
          const int j = j0 + tid + k * kSelThreads;
          key[k] = j < n ? keys[j] : 0ull;
          page[k] = j < n ? page_id(g, f.index, (lo + j) / per) : -1;
        }
      }
      // how many wavefront w takes of its 64 k-th keys, and how many ties there are ahead
      uint64_t over[kHeld], tie[kHeld];
#pragma unroll
      for (int k = 0; k < kHeld; ++k) {
        if (k >= rounds) break;
        over[k] = __ballot(key[k] > edge.key);
        tie[k] = __ballot(key[k] == edge.key && key[k] != 0ull);
        if (lane == 0) counted[k * 16 + wave] = __builtin_popcountll(over[k]) | __builtin_popcountll(tie[k]) << 16;
      }
      lds_barrier();
      // prefix sums over the counts (k, wavefront), two per lane; the ties' limit applies in order
      const bool used = 2 * lane < 16 * rounds;
      const int a = used ? counted[2 * lane] : 0, b = used ? counted[2 * lane + 1] : 0;
      const int o_incl = wave_scan_incl((a & 0xffff) + (b & 0xffff)), t_incl = wave_scan_incl((a >> 16) + (b >> 16));
#pragma unroll
      for (int k = 0; k < kHeld; ++k) {
        if (k >= rounds) break;
        const int c = k * 16 + wave, from = c >> 1;                // counts before c: of the lanes before, and of this lane's first
        const int pa = __builtin_amdgcn_readlane(a, from), pb = __builtin_amdgcn_readlane(b, from);
        const int o_before = __builtin_amdgcn_readlane(o_incl, from) - (pa & 0xffff) - (pb & 0xffff) + (c & 1 ? pa & 0xffff : 0);
        const int t_before = equal + __builtin_amdgcn_readlane(t_incl, from) - (pa >> 16) - (pb >> 16) + (c & 1 ? pa >> 16 : 0);
        const uint64_t below = (1ull << lane) - 1ull;
        const int my_t = t_before + __builtin_popcountll(tie[k] & below);
        const bool is_over = (over[k] >> lane) & 1, take = is_over || (((tie[k] >> lane) & 1) && my_t < edge.ties);
        // taken ties ahead of this key: min(ties ahead, limit) less those before this sweep, which `count` has
        const int place = count + o_before + __builtin_popcountll(over[k] & below) + min(my_t, edge.ties) - min(equal, edge.ties);
        const int blk = lo + j0 + tid + k * kSelThreads;
        if (take) list[place] = make_int2(page[k], blk);
      }
      const int o_all = __builtin_amdgcn_readlane(o_incl, 63), t_all = __builtin_amdgcn_readlane(t_incl, 63);
      count += o_all + min(equal + t_all, edge.ties) - min(equal, edge.ties);
      equal += t_all;
      lds_barrier();
    }
    for (int b = tid; b < g.last; b += kSelThreads) list[count + b] = make_int2(page_id(g, f.index, (hi + b) / per), hi + b);
    count += g.last;
  }
  if (tid == 0) g.list_head[at] = make_int4(count, pos, f.index, 0);
}

void launch_block_select(const PagedGeom& g, hipStream_t s) {
  // about a thousand workgroups at most
  const int64_t passes = (g.max_blocks + kScoreBlocks - 1) / kScoreBlocks, heads = (int64_t)g.Hkv * g.row_group;
  const int per_wg = (int)((passes * heads + 1023) / 1024) * kScoreBlocks;
  const dim3 grid((g.max_blocks + per_wg - 1) / per_wg, g.Hkv, g.row_group);
  if (g.max_blocks > g.kept && g.top > 0) {
    if (g.dtype == TKPHI_BF16) {
      if (g.d == 64) hipLaunchKernelGGL((block_score_kernel<uint16_t, 64>), grid, dim3(kPagedThreads), 0, s, g, per_wg);
      else hipLaunchKernelGGL((block_score_kernel<uint16_t, 128>), grid, dim3(kPagedThreads), 0, s, g, per_wg);
    } else {
      if (g.d == 64) hipLaunchKernelGGL((block_score_kernel<float, 64>), grid, dim3(kPagedThreads), 0, s, g, per_wg);
      else hipLaunchKernelGGL((block_score_kernel<float, 128>), grid, dim3(kPagedThreads), 0, s, g, per_wg);
    }
  }
  hipLaunchKernelGGL(block_select_kernel, dim3(g.Hkv, g.row_group), dim3(kSelThreads), 0, s, g);
}

}  // namespace tkphi
