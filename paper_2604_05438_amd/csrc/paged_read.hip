// tkphi_quant_read: tokens of a cache in 8 bits as bf16 rows, in any layout (for the calls on contiguous caches).
//
// Codes times their row's power of two: one conversion per pair.  A workgroup takes 64 consecutive positions of one sequence and KV head; a lane has
// 8 codes of up to 8 rows on their way before it converts the first.  Bound by memory: a prefix of 131072 tokens of a 3B layer (807 MB) 147 us = 5.5 TB/s, a large
// copy runs at 5.1.  (16 codes per lane, whose two stores each leave gaps for the other's: 182 us; loads that stay in the caches 158.  Stores that do not: 142, but what
// reads the rows comes next.)  Keys alone take 97 us, values 91: their codes are read in both cases.
#include "paged.h"

namespace tkphi {

constexpr int kReadTile = 64;

template <int D>
__global__ __launch_bounds__(kPagedThreads) void paged_read_kernel(PagedGeom g) {
  constexpr int PIECES = D / 8, EACH = kReadTile * 2 * PIECES / kPagedThreads;       // 8 codes, 16 bytes of a row; per thread
  const int h = blockIdx.y, tid = threadIdx.x;
  const FoundSeq f = find_seq(g, blockIdx.x, [&](const PagedSeq& s) { return (s.cached + s.fresh - 1) / kReadTile - s.cached / kReadTile + 1; });
  if (f.index < 0) return;
  if (blockIdx.x == gridDim.x - 1) {                             // past what the rows allow for: sequences share some (tiles from here on are left out)
    if (h == 0 && tid == 0) atomicOr(g.status, TKPHI_DEV_BAD_LENGTH);
    return;
  }
  const int t0 = (f.s.cached / kReadTile + ((int)blockIdx.x - f.before)) * kReadTile;
  const int lo = max(t0, f.s.cached), hi = min(t0 + kReadTile, f.s.cached + f.s.fresh);
  const int first_row = f.s.row + (lo - f.s.cached), p = tid % PIECES;
  bool lost = false;
  uint64_t w[EACH];
  uint32_t scale[EACH];
#pragma unroll
  for (int k = 0; k < EACH; ++k) {                               // keys, then values; absent tokens read page 0
    const int i = (tid + k * kPagedThreads) / PIECES, is_v = i / kReadTile, t = min(lo + i % kReadTile, hi - 1);
    const int pt = page_of(g, t), id = page_id(g, f.index, pt, &lost), in = t - pt * g.by_page.d;
    lost = lost || id < 0;
    w[k] = __builtin_nontemporal_load((const __attribute__((address_space(1))) uint64_t*)((is_v ? g.V : g.K) + (int64_t)max(id, 0) * g.st_page + h * g.st_head +
                                                                                          (int64_t)in * g.st_tok + p * 8));
    scale[k] = ((const __attribute__((address_space(1))) uint8_t*)(g.S + scale_at(g, max(id, 0), h, in)))[is_v];
    if (id < 0) scale[k] = 0x100;
  }
#pragma unroll
  for (int k = 0; k < EACH; ++k) {
    const int i = (tid + k * kPagedThreads) / PIECES, is_v = i / kReadTile, t = lo + i % kReadTile;
    char* const base = is_v ? g.v_out : g.k_out;
    if (t >= hi || !base) continue;
    char* dst = base + (int64_t)(first_row + t - lo) * (is_v ? g.v_row : g.k_row) + h * (is_v ? g.v_head : g.k_head) + p * 16;
    u32x4 a = decode8((uint32_t)w[k], (uint32_t)(w[k] >> 32), __uint_as_float((scale[k] & 0xffu) << 23));
    if (scale[k] & 0x100u) a = (u32x4){0u, 0u, 0u, 0u};
    *(__attribute__((address_space(1))) u32x4*)dst = a;
  }
  report_pages(g, lost);
}

void launch_paged_read(const PagedGeom& g, hipStream_t s) {
  // sequence by sequence a tile at either end may be cut
  const int64_t by_rows = g.rows / kReadTile + 2ll * g.n_seqs, by_seqs = (int64_t)g.n_seqs * ((g.max_new - 2 + kReadTile) / kReadTile + 1);
  const dim3 grid((unsigned)(by_rows < by_seqs ? by_rows : by_seqs) + 1, g.Hkv);          // (the last one has a tile only where sequences share rows)
  if (g.d == 64) hipLaunchKernelGGL(paged_read_kernel<64>, grid, dim3(kPagedThreads), 0, s, g);
  else hipLaunchKernelGGL(paged_read_kernel<128>, grid, dim3(kPagedThreads), 0, s, g);
}

}  // namespace tkphi
