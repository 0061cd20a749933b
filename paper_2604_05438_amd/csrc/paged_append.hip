// tkphi_kv_append: new queries and keys turned to their positions, keys and values to their pages, mean keys of filled blocks.
//
// A pair of channels (a, b) of the token at position p becomes (a cos - b sin, a sin + b cos) at the angle p inv_freq[j].
// A workgroup takes a tile of consecutive cache positions of one sequence (a whole block where means are kept, so that the mean has one
// writer and a fixed order) and one KV head with its query heads.  Bound by memory: every row is read once and written
// once, 16 bytes per lane; the angles (64 bits: at position 10^6 a 32-bit product is off by 0.06 rad) are taken once per
// token, pair and workgroup and shared through LDS.  A chunk of 16001 tokens of a 3B layer (24 / 8 heads of 128): 77 us = 4.3 TB/s, where a large copy
// runs at 4.85; 64 single tokens 5 us.  Several KV heads per workgroup, which share the angles: 76 us, but 21 instead of 11 us for 3000 tokens of
// a 1B layer; non-temporal loads: 14 instead of 11 us there; two or four tasks per thread at a time: no faster.
#include "paged.h"

namespace tkphi {

// cos and sin of the angle x, in revolutions of a quarter turn: reduced in 64 bits, then the Taylor series on [-pi/4, pi/4], whose first
// dropped terms are below 2e-9
__device__ __forceinline__ float2 cos_sin(double x) {
  const double quarters = x * 0.63661977236758134308;            // 2 / pi
  const double whole = rint(quarters);
  const float y = (float)((quarters - whole) * 1.57079632679489661923);
  const float z = y * y;
  float s = fmaf(z, 1.f / 362880.f, -1.f / 5040.f);
  s = fmaf(z, s, 1.f / 120.f);
  s = fmaf(z, s, -1.f / 6.f);
  s = fmaf(z * y, s, y);
  float c = fmaf(z, -1.f / 3628800.f, 1.f / 40320.f);
  c = fmaf(z, c, -1.f / 720.f);
  c = fmaf(z, c, 1.f / 24.f);
  c = fmaf(z, c, -0.5f);
  c = fmaf(z, c, 1.f);
  const int k = (int)((long long)whole & 3);
  const float cc = k & 1 ? s : c, ss = k & 1 ? c : s;
  return make_float2(k == 1 || k == 2 ? -cc : cc, k >= 2 ? -ss : ss);
}

template <typename T> __device__ __forceinline__ u32x4 pack16(const float* x);
template <> __device__ __forceinline__ u32x4 pack16<float>(const float* x) {
  return (u32x4){__float_as_uint(x[0]), __float_as_uint(x[1]), __float_as_uint(x[2]), __float_as_uint(x[3])};
}
template <> __device__ __forceinline__ u32x4 pack16<uint16_t>(const float* x) {
  u32x4 r;
#pragma unroll
  for (int i = 0; i < 4; ++i) r[i] = __builtin_bit_cast(uint32_t, (bf16x2_t){(__bf16)x[2 * i], (__bf16)x[2 * i + 1]});
  return r;
}
typedef __attribute__((address_space(1))) u32x4* gout128;
__device__ __forceinline__ void gstore128(void* p, u32x4 v) { *(gout128)p = v; }

template <typename T, int D>
__global__ __launch_bounds__(kPagedThreads) void paged_append_kernel(PagedGeom g, int tile) {
  constexpr int EPL = Elem<T>::per16, PAIRS = D / (2 * EPL);     // pairs of 16-byte pieces per row
  extern __shared__ __align__(16) char lds[];
  const int h = blockIdx.y, tid = threadIdx.x;
  const FoundSeq f = find_seq(g, blockIdx.x, [&](const PagedSeq& s) { return (s.cached + s.fresh - 1) / tile - s.cached / tile + 1; });
  if (f.index < 0) return;
  if (blockIdx.x == gridDim.x - 1) {                             // past what the rows allow for: sequences share some (tiles from here on are left out)
    if (h == 0 && tid == 0) atomicOr(g.status, TKPHI_DEV_BAD_LENGTH);
    return;
  }
  const int t0 = (f.s.cached / tile + ((int)blockIdx.x - f.before)) * tile;
  const int lo = max(t0, f.s.cached), hi = min(t0 + tile, f.s.cached + f.s.fresh);      // new tokens of this tile
  const int n = hi - lo, half = g.rot / 2;
  float2* turn = (float2*)lds;                                   // [tile][rot / 2]
  T* kept = (T*)(lds + (size_t)tile * half * sizeof(float2));    // [tile][D] keys as stored, for the mean
  const bool fills = g.block > 0 && hi == t0 + tile;
  const int first_row = f.s.row + (lo - f.s.cached);
  const int block_entry = page_of(g, t0), block_row = t0 - block_entry * g.by_page.d;   // (a block lies in one page)
  bool lost = false;

  if (fills && lo > t0) {                                      // older keys of the block
    const char* src = g.K + (int64_t)max(page_id(g, f.index, block_entry), 0) * g.st_page + h * g.st_head + (int64_t)block_row * g.st_tok;
    constexpr int PIECES = D / EPL;
    for (int i = tid; i < (lo - t0) * PIECES; i += kPagedThreads)
      *(u32x4*)(kept + (i / PIECES) * D + (i % PIECES) * EPL) = gload128(src + (int64_t)(i / PIECES) * g.st_tok + (i % PIECES) * 16);
  }
  for (int i = tid; i < n * half; i += kPagedThreads) {
    const int t = g.by_half(i), j = i - t * half;
    turn[i] = cos_sin((double)(lo + t) * g.inv_freq[j]);
  }
  __syncthreads();
  const int lines = g.by_lines.d;                                // query heads, the key, the value
  const int rotated = g.rot / (2 * EPL);                         // pairs of pieces that turn
  for (int i = tid; i < n * lines * PAIRS; i += kPagedThreads) {
    const int p = i % PAIRS, t = g.by_lines(i / PAIRS), line = i / PAIRS - t * lines;
    const bool is_v = line == lines - 1, is_k = line == lines - 2;
    const char* src = is_v   ? g.v + (int64_t)(first_row + t) * g.v_row + h * g.v_head
                      : is_k ? g.k + (int64_t)(first_row + t) * g.k_row + h * g.k_head
                             : g.q + (int64_t)(first_row + t) * g.q_row + (int64_t)(h * g.G + line) * g.q_head;
    const bool turns = !is_v && p < rotated;
    // the two pieces: first and second halves of the pairs, or neighbours
    const int pa = turns && !g.adjacent ? p : 2 * p, pb = turns && !g.adjacent ? p + rotated : 2 * p + 1;
    u32x4 ua = gload128(src + pa * 16), ub = gload128(src + pb * 16);
    char* dst;
    if (line < lines - 2) {
      dst = g.out + (int64_t)(first_row + t) * g.out_row + (int64_t)(h * g.G + line) * g.out_head;
    } else {
      const int pt = page_of(g, lo + t), id = page_id(g, f.index, pt, &lost);
      dst = id < 0 ? nullptr : (is_v ? g.V : g.K) + (int64_t)id * g.st_page + h * g.st_head + (int64_t)(lo + t - pt * g.by_page.d) * g.st_tok;
      lost = lost || id < 0;
    }
    if (turns) {
      float a[EPL], b[EPL], x[EPL], y[EPL];
      Elem<T>::unpack(make_uint4(ua.x, ua.y, ua.z, ua.w), a);
      Elem<T>::unpack(make_uint4(ub.x, ub.y, ub.z, ub.w), b);
      const float2* cs = turn + t * half + p * EPL;
      if (g.adjacent) {
#pragma unroll
        for (int e = 0; e < EPL; e += 2) {
          const float2 c = cs[e / 2], c2 = cs[EPL / 2 + e / 2];
          x[e] = a[e] * c.x - a[e + 1] * c.y;
          x[e + 1] = a[e] * c.y + a[e + 1] * c.x;
          y[e] = b[e] * c2.x - b[e + 1] * c2.y;
          y[e + 1] = b[e] * c2.y + b[e + 1] * c2.x;
        }
      } else {
#pragma unroll
        for (int e = 0; e < EPL; ++e) {
          const float2 c = cs[e];
          x[e] = a[e] * c.x - b[e] * c.y;
          y[e] = a[e] * c.y + b[e] * c.x;
        }
      }
      ua = pack16<T>(x);
      ub = pack16<T>(y);
    }
    if (dst) {
      gstore128(dst + pa * 16, ua);
      gstore128(dst + pb * 16, ub);
    }
    if (is_k && fills) {
      T* key = kept + (lo + t - t0) * D;
      *(u32x4*)(key + pa * EPL) = ua;
      *(u32x4*)(key + pb * EPL) = ub;
    }
  }
  report_pages(g, lost);
  if (!fills) return;
  __syncthreads();
  const int id = page_id(g, f.index, block_entry);
  const int per = g.by_page.d / g.block, b = block_row / g.block;
  for (int c = tid; c < D && id >= 0; c += kPagedThreads) {
    float sum = 0.f;
    for (int t = 0; t < tile; ++t) sum += Elem<T>::load1(kept, t * D + c);
    sum *= 1.f / (float)g.block;                               // (a power of two)
    const int64_t at = (((int64_t)id * g.Hkv + h) * per + b) * D + c;
    if constexpr (sizeof(T) == 2) ((__bf16*)g.M)[at] = (__bf16)sum;
    else ((float*)g.M)[at] = sum;
  }
}

void launch_paged_append(const PagedGeom& g, hipStream_t s) {
  const int tile = g.block ? g.block : 16;
  // sequence by sequence a tile at either end may be cut
  const int64_t by_rows = g.rows / tile + 2ll * g.n_seqs, by_seqs = (int64_t)g.n_seqs * ((g.max_new - 2 + tile) / tile + 1);
  const unsigned tiles = (unsigned)(by_rows < by_seqs ? by_rows : by_seqs);
  const dim3 grid(tiles + 1, g.Hkv);                             // (the last one has a tile only where sequences share rows)
  const size_t lds = (size_t)tile * (g.rot / 2) * sizeof(float2) + (g.block ? (size_t)tile * g.d * (g.dtype == TKPHI_BF16 ? 2 : 4) : 0);
  if (g.dtype == TKPHI_BF16) {
    if (g.d == 64) hipLaunchKernelGGL((paged_append_kernel<uint16_t, 64>), grid, dim3(kPagedThreads), lds, s, g, tile);
    else hipLaunchKernelGGL((paged_append_kernel<uint16_t, 128>), grid, dim3(kPagedThreads), lds, s, g, tile);
  } else {
    if (g.d == 64) hipLaunchKernelGGL((paged_append_kernel<float, 64>), grid, dim3(kPagedThreads), lds, s, g, tile);
    else hipLaunchKernelGGL((paged_append_kernel<float, 128>), grid, dim3(kPagedThreads), lds, s, g, tile);
  }
}

}  // namespace tkphi
