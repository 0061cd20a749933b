// Selection of tkphi_block_attention: per query token and KV head the blocks whose mean keys score highest.
//
// score(b) = max over the KV head's query heads of q . M_b.  Which blocks a query sees is a yes or no, so the scores are sums in 64 bits (products of two
// bf16 are exact there, of two fp32 too), compared as order-preserving 64-bit keys, equal ones by the lower block.
#include "paged.h"
#include "select_utils.h"

namespace tkphi {

// Order-preserving key of a score, 0 for what is not retrieved (NaN, -inf)
__device__ __forceinline__ uint64_t score_key64(double x) {
  if (!(x > -INFINITY)) return 0ull;
  const uint64_t b = __builtin_bit_cast(uint64_t, x + 0.0);        // (-0 and 0 are equal)
  return b >> 63 ? ~b : b | 0x8000000000000000ull;
}

__device__ __forceinline__ double quad_sum(double x) {             // over 4 neighbouring lanes
  for (int k = 1; k < 4; k *= 2) x += __shfl_xor(x, k);
  return x;
}

constexpr int kScoreBlocks = 64;          // blocks per pass of a workgroup: 4 lanes each
template <typename T, int D>
__global__ __launch_bounds__(kPagedThreads) void block_score_kernel(PagedGeom g, int blocks_per_wg) {
  constexpr int EPL = Elem<T>::per16, C = D / 4, PAD = 2;          // channels per lane
  __shared__ __align__(16) double q[kMaxGroup][4 * (C + PAD)];
  const int h = blockIdx.y, local = blockIdx.z, token = g.row0 + local, tid = threadIdx.x;
  const FoundSeq f = find_row(g, token);
  if (f.index < 0) return;
  const int pos = f.s.cached + token - f.s.row, have = pos / g.block + 1;
  if (have <= g.kept) return;                                      // it sees all of them
  const int lo = max(g.first, (int)blockIdx.x * blocks_per_wg), hi = min(have - g.last, ((int)blockIdx.x + 1) * blocks_per_wg);
  if (lo >= hi) return;
  for (int i = tid; i < g.G * D; i += kPagedThreads) {
    const int a = i / D, c = i % D;
    q[a][c / C * (C + PAD) + c % C] = (double)Elem<T>::load1(g.q + (int64_t)token * g.q_row + (int64_t)(h * g.G + a) * g.q_head, c);
  }
  __syncthreads();
  const int part = tid & 3, per = g.page / g.block;
  uint64_t* keys = g.keys + ((int64_t)local * g.Hkv + h) * g.max_blocks;
  for (int b0 = lo; b0 < hi; b0 += kScoreBlocks) {
    const int b = b0 + (tid >> 2), page = b / per;
    const int id = b < hi ? page_id(g, f.index, page) : -1;
    const char* src = g.M + ((((int64_t)max(id, 0) * g.Hkv + h) * per + b % per) * D + part * C) * sizeof(T);
    double sum[kMaxGroup];
#pragma unroll
    for (int a = 0; a < kMaxGroup; ++a) sum[a] = 0.0;
#pragma unroll
    for (int j = 0; j < C / EPL; ++j) {
      const u32x4 u = gload128(src + j * 16);
      float x[EPL];
      Elem<T>::unpack(make_uint4(u.x, u.y, u.z, u.w), x);
#pragma unroll
      for (int a = 0; a < kMaxGroup; ++a)
        if (a < g.G) {
#pragma unroll
          for (int e = 0; e < EPL; ++e) sum[a] = fma((double)x[e], q[a][part * (C + PAD) + j * EPL + e], sum[a]);
        }
    }
    double best = -INFINITY;
    bool nan = false;
#pragma unroll
    for (int a = 0; a < kMaxGroup; ++a)
      if (a < g.G) {
        const double s = quad_sum(sum[a]);
        nan = nan || s != s;
        best = s > best ? s : best;
      }
    if (part == 0 && b < hi) keys[b] = nan || id < 0 ? 0ull : score_key64(best);
  }
}

// One workgroup per query token and KV head: the blocks it sees, ascending
__global__ __launch_bounds__(kSelThreads) void block_select_kernel(PagedGeom g) {
  __shared__ uint32_t hist[256];
  __shared__ int scan[16], want_sh, eligible;
  __shared__ uint64_t prefix;
  const int h = blockIdx.x, local = blockIdx.y, token = g.row0 + local, tid = threadIdx.x;
  const int64_t at = (int64_t)local * g.Hkv + h;
  const FoundSeq f = find_row(g, token);
  if (f.index < 0) {
    if (tid == 0) g.list_head[at] = make_int4(0, 0, 0, 0);
    return;
  }
  const int pos = f.s.cached + token - f.s.row, have = pos / g.block + 1, per = g.page / g.block;
  const int lo = g.first, hi = have - g.last;                      // blocks [lo, hi) compete
  const bool all = have <= g.kept;
  const uint64_t* keys = g.keys + at * g.max_blocks;
  uint64_t edge = 1ull;                                            // taken: key > edge, and the first `ties` of those equal to it
  int ties = 0x7fffffff;
  if (!all) {
    if (tid == 0) eligible = 0;
    __syncthreads();
    int n = 0;
    for (int b = lo + tid; b < hi; b += kSelThreads) n += keys[b] != 0ull;
    n = wave_sum(n);
    if ((tid & 63) == 0) atomicAdd(&eligible, n);
    __syncthreads();
    if (g.top == 0) {
      edge = ~0ull;
      ties = 0;
    } else if (eligible > g.top) {
      edge = radix_select_desc(hi - lo, g.top, [&](int j, uint64_t* v) { *v = keys[lo + j]; return *v != 0ull; }, hist, scan, &prefix, &want_sh);
      ties = want_sh;
    }
  }
  int2* list = g.list + at * g.kept;
  int count = 0, equal = 0;
  for (int b0 = 0; b0 < have; b0 += kSelThreads) {
    const int b = b0 + tid;
    const bool competes = !all && b >= lo && b < hi;
    const uint64_t key = competes ? keys[b] : 0ull;
    const bool tie = competes && key == edge;
    const int tie_incl = sel_scan_incl(tie ? 1 : 0, scan);
    const bool take = b < have && (!competes || key > edge || (tie && equal + tie_incl <= ties));
    if (tid == kSelThreads - 1) want_sh = tie_incl;
    const int incl = sel_scan_incl(take ? 1 : 0, scan);
    if (take) list[count + incl - 1] = make_int2(page_id(g, f.index, b / per), b);
    if (tid == kSelThreads - 1) eligible = incl;
    __syncthreads();
    equal += want_sh;
    count += eligible;
    __syncthreads();
  }
  if (tid == 0) g.list_head[at] = make_int4(count, pos, f.index, 0);
}

void launch_block_select(const PagedGeom& g, hipStream_t s) {
  // passes of 64 blocks per workgroup: about a thousand workgroups
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
