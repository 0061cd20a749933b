// Launches of the attention calls on the paged cache: the plan, the kernels, the joins of a plan's pieces.
#include "paged_split.h"

namespace tkphi {

// The items in order with the running sum of their units, by one workgroup.  (Items past the plan's room, as there are if sequences share
// rows, are left out.)
__global__ __launch_bounds__(1024) void paged_plan_kernel(PagedGeom g) {
  __shared__ int first[1025];
  __shared__ uint32_t sums[16];
  __shared__ int64_t sums64[16];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  int items = 0;
  for (int i0 = 0; i0 < g.n_seqs; i0 += 1024) {                    // 1024 sequences: where their items start, then all items at once
    int tiles = 0;
    if (i0 + tid < g.n_seqs) {
      const PagedSeq s = check_seq(g, g.seqs[i0 + tid]);
      tiles = s.fresh > 0 ? (s.fresh * g.G + g.tile_rows - 1) / g.tile_rows : 0;
    }
    // (up to 2^27 rows, 8 heads and 32 rows per item: 2^31 items of 64 sequences that share rows)
    const uint32_t x = (uint32_t)wave_scan_incl(tiles);
    if (lane == 63) sums[wave] = x;
    __syncthreads();
    int64_t ahead = 0, all = 0;
    for (int k = 0; k < 16; ++k) {
      if (k < wave) ahead += sums[k];
      all += sums[k];
    }
    first[tid + 1] = (int)min(ahead + (int64_t)x, (int64_t)(g.plan_room - items));
    if (tid == 0) first[0] = 0;
    __syncthreads();
    if (items + all > g.plan_room) {
      if (tid == 0) atomicOr(g.status, TKPHI_DEV_BAD_LENGTH);
      all = g.plan_room - items;
    }
    for (int j = tid; j < (int)all; j += 1024) {
      int a = 0, b = min(1024, g.n_seqs - i0) - 1;                 // last sequence that starts at or before j (and has items)
      while (a < b) {
        const int c = (a + b + 1) / 2;
        if (first[c] <= j) a = c;
        else b = c - 1;
      }
      g.plan_item[items + j] = make_int2(i0 + a, j - first[a]);
    }
    items += (int)all;
    __syncthreads();
  }
  __threadfence_block();
  __syncthreads();
  int64_t base = 0;
  for (int j0 = 0; j0 < items; j0 += 1024) {
    const int j = j0 + tid;
    int64_t x = 0;
    if (j < items) {
      const int2 it = g.plan_item[j];
      x = item_units(g, item_range(g, check_seq(g, g.seqs[it.x]), it.y));
    }
    for (int k = 1; k < 64; k *= 2) {
      const int64_t y = __shfl_up(x, k);
      if (lane >= k) x += y;
    }
    if (lane == 63) sums64[wave] = x;
    __syncthreads();
    int64_t ahead = 0, all = 0;
    for (int k = 0; k < 16; ++k) {
      if (k < wave) ahead += sums64[k];
      all += sums64[k];
    }
    __syncthreads();
    if (j < items) g.plan_end[j] = base + ahead + x;
    base += all;
  }
  if (tid == 0) *g.plan_count = items;
}

// After the kernels with a plan: the item that starts in share w and ends in another is joined, 32 rows per workgroup at a time, 8 of many pieces (one workgroup for
// a whole item: 250 us for 64 rows in 125 pieces)
constexpr int kJoinRows = 32, kJoinGroups = 8;
template <typename T, int D>
__global__ __launch_bounds__(kPagedThreads) void paged_join_kernel(PagedGeom g) {
  __shared__ __align__(16) char lds[join_lds(kPagedThreads, kJoinRows)];
  const int w = blockIdx.x;
  const int4 a = g.joins[2 * w], b = g.joins[2 * w + 1];
  const int pieces = uniform(a.x), rows = uniform(a.y), h = uniform(a.z), row0 = uniform(a.w), q0 = uniform(b.x), first = uniform(b.y);
  if (pieces == 0) return;
  const int step = pieces <= 4 ? kJoinRows : 8;
  for (int r0 = blockIdx.y * step; r0 < rows; r0 += step * kJoinGroups)
    join_pieces<T, D, kPagedThreads, false>(g, pieces, r0, min(step, rows - r0), g.tile_rows, lds,
                                            [&](int k) { return partial_slot(g, w + k, k > 0 || first); },
                                            [&](int row, int* token, int* head) {
                                              const int r = row0 + row, i = g.by_group(r);
                                              *token = q0 + i;
                                              *head = h * g.G + r - i * g.G;
                                            });
}

template <typename T, int D>
static void launch_attend(const PagedGeom& g, hipStream_t s) {
  if (g.plan_room) hipLaunchKernelGGL(paged_plan_kernel, dim3(1), dim3(1024), 0, s, g);
  if (g.tile_rows > kPagedRows) launch_paged_chunk(g, s);
  else if (g.S) launch_split_codes(g, s);
  else launch_split_rows<T, D>(g, s);
  if (g.plan_room) hipLaunchKernelGGL((paged_join_kernel<T, D>), dim3(g.splits, kJoinGroups), dim3(kPagedThreads), 0, s, g);
}
void launch_paged_attention(const PagedGeom& g, hipStream_t s) {
  if (g.dtype == TKPHI_BF16) {
    if (g.d == 64) launch_attend<uint16_t, 64>(g, s);
    else launch_attend<uint16_t, 128>(g, s);
  } else {
    if (g.d == 64) launch_attend<float, 64>(g, s);
    else launch_attend<float, 128>(g, s);
  }
}

void launch_block_attention(const PagedGeom& g, hipStream_t s) {
  if (g.S) {
    launch_blocks_codes(g, s);
  } else if (g.dtype == TKPHI_BF16) {
    if (g.d == 64) launch_blocks<uint16_t, 64>(g, s);
    else launch_blocks<uint16_t, 128>(g, s);
  } else {
    if (g.d == 64) launch_blocks<float, 64>(g, s);
    else launch_blocks<float, 128>(g, s);
  }
}

}  // namespace tkphi
