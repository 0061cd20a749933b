// tkphi_kv_append, tkphi_norm_append, tkphi_quant_append: new queries and keys, normed by head where asked for, turned to their positions, keys and values
// to their pages, in the rows' own type or in 8 bits, mean keys of filled blocks.
//
// Norm: y = x / sqrt(mean x^2 + eps) (w + offset), in 32 bits with the rotation behind it, rounded once.  8 bits: see Code8; the scale is that of the
// row as it would be stored in 32 bits.
// A pair of channels (a, b) of the token at position p becomes (a cos - b sin, a sin + b cos) at the angle p inv_freq[j].
// A workgroup takes a tile of consecutive cache positions of one sequence (a whole block where means are kept, so that the mean has one
// writer and a fixed order) and one KV head with its query heads.  Bound by memory: every row is read once and written
// once, 16 bytes per lane; the angles (64 bits: at position 10^6 a 32-bit product is off by 0.06 rad) are taken once per
// token, pair and workgroup and shared through LDS.  A chunk of 16001 tokens of a 3B layer (24 / 8 heads of 128): 77 us = 4.3 TB/s, normed 79 (74 with
// angles that cost nothing); 12946 tokens of nine sequences of a 1B layer into codes, normed, 43 us = 3.4 TB/s (neither normed nor turned, without means: 37).  Line by
// line, so that a wavefront's lanes do the same, the last one took 44 us, before 50; with the next task's rows requested ahead 54.  A large copy
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

// A row of the cache in 8 bits out of the two pieces of it that a lane holds (the row's `lanes` lanes ask together): codes of both, and the scale byte.
// The scale goes by the largest finite element; what is not finite becomes NaN by the conversion.
struct Coded {
  uint32_t x[2], y[2];
  uint32_t scale;
};
// top: bits of the row's largest size, f 2^k with 1 <= f < 2; the largest code is 1.75 x 2^8
__device__ __forceinline__ uint32_t scale_byte(uint32_t top) {
  return (uint32_t)min(max((int)(top >> 23) - 8 + ((top & 0x7fffffu) > 0x600000u), kLeastScale), kMostScale);
}
typedef short pp_short2 __attribute__((ext_vector_type(2)));
typedef unsigned short pp_ushort2 __attribute__((ext_vector_type(2)));
// (the conversions divide by the scale, exactly: the code is the only rounding)
__device__ __forceinline__ uint32_t codes_of(const float* v, float scale) {
  pp_short2 r = {0, 0};
  r = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(r, v[0], v[1], scale, false);
  r = __builtin_amdgcn_cvt_scalef32_pk_fp8_f32(r, v[2], v[3], scale, true);
  return __builtin_bit_cast(uint32_t, r);
}
__device__ __forceinline__ uint32_t codes_of(uint32_t a, uint32_t b, float scale) {
  pp_short2 r = {0, 0};
  r = __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(r, __builtin_bit_cast(bf16x2_t, a), scale, false);
  r = __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(r, __builtin_bit_cast(bf16x2_t, b), scale, true);
  return __builtin_bit_cast(uint32_t, r);
}
// Code 256 (0x78) of the largest power of two would be 2^128, no bf16 number: elements that round to it, from 1.9375 x 2^127 on, take the code before, 240, which is
// still within 2^-4 of them (by the size x: x - 240 2^120 < 2^-4 x up to 2^128)
__device__ __forceinline__ uint32_t below_256(uint32_t codes) {
  const uint32_t other = ((codes & 0x7f7f7f7fu) ^ 0x78787878u) + 0x7f7f7f7fu;        // highest bit of a byte: it is another code
  return codes - ((~other & 0x80808080u) >> 7);
}
__device__ __forceinline__ void keep_finite(Coded& c) {
  if (c.scale != kMostScale) return;
#pragma unroll
  for (int i = 0; i < 2; ++i) { c.x[i] = below_256(c.x[i]); c.y[i] = below_256(c.y[i]); }
}
// of 32-bit numbers; their sizes compare as integers
__device__ __forceinline__ Coded encode(const float* x, const float* y, int lanes) {
  const auto size = [](float v) { return __float_as_uint(v) & 0x7fffffffu; };
  uint32_t top = 0;
#pragma unroll
  for (int e = 0; e < 8; ++e) top = max(top, max(size(x[e]), size(y[e])));
  if (__any(top >= 0x7f800000u)) {
    const auto finite = [&](float v) { return size(v) < 0x7f800000u ? size(v) : 0u; };
    top = 0;
#pragma unroll
    for (int e = 0; e < 8; ++e) top = max(top, max(finite(x[e]), finite(y[e])));
  }
  Coded c;
  c.scale = scale_byte(lanes_reduce(top, lanes, MaxOp()));
  const float scale = __uint_as_float(c.scale << 23);
  c.x[0] = codes_of(x, scale); c.x[1] = codes_of(x + 4, scale);
  c.y[0] = codes_of(y, scale); c.y[1] = codes_of(y + 4, scale);
  keep_finite(c);
  return c;
}
// of bf16 pairs as they are
__device__ __forceinline__ Coded encode(u32x4 x, u32x4 y, int lanes) {
  const auto sizes = [](uint32_t w) { return __builtin_bit_cast(pp_ushort2, w & 0x7fff7fffu); };
  pp_ushort2 both = {0, 0};
#pragma unroll
  for (int e = 0; e < 4; ++e) both = __builtin_elementwise_max(both, __builtin_elementwise_max(sizes(x[e]), sizes(y[e])));
  if (__any(max((uint32_t)both.x, (uint32_t)both.y) >= 0x7f80u)) {
    const auto finite = [&](uint32_t w) {
      const pp_ushort2 s = sizes(w);
      return (pp_ushort2){s.x < 0x7f80 ? s.x : (unsigned short)0, s.y < 0x7f80 ? s.y : (unsigned short)0};
    };
    both = (pp_ushort2){0, 0};
#pragma unroll
    for (int e = 0; e < 4; ++e) both = __builtin_elementwise_max(both, __builtin_elementwise_max(finite(x[e]), finite(y[e])));
  }
  Coded c;
  c.scale = scale_byte(lanes_reduce(max((uint32_t)both.x, (uint32_t)both.y) << 16, lanes, MaxOp()));
  const float scale = __uint_as_float(c.scale << 23);
  c.x[0] = codes_of(x.x, x.y, scale); c.x[1] = codes_of(x.z, x.w, scale);
  c.y[0] = codes_of(y.x, y.y, scale); c.y[1] = codes_of(y.z, y.w, scale);
  keep_finite(c);
  return c;
}

// C: the cache's type; NORM: heads of q and k are normed first
template <typename C, int D, bool NORM>
__global__ __launch_bounds__(kPagedThreads) void paged_append_kernel(PagedGeom g, int tile) {
  using T = typename Cached<C>::Row;
  constexpr bool CODES = Cached<C>::codes;
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
    if constexpr (CODES) {
      const uint16_t* scales = g.S + scale_at(g, max(page_id(g, f.index, block_entry), 0), h, block_row);
      for (int i = tid; i < (lo - t0) * PIECES; i += kPagedThreads) {
        const uint64_t w = *(const __attribute__((address_space(1))) uint64_t*)(src + (int64_t)(i / PIECES) * g.st_tok + (i % PIECES) * 8);
        *(u32x4*)(kept + (i / PIECES) * D + (i % PIECES) * EPL) = decode8((uint32_t)w, (uint32_t)(w >> 32), key_scale(scales[i / PIECES]));
      }
    } else {
      for (int i = tid; i < (lo - t0) * PIECES; i += kPagedThreads)
        *(u32x4*)(kept + (i / PIECES) * D + (i % PIECES) * EPL) = gload128(src + (int64_t)(i / PIECES) * g.st_tok + (i % PIECES) * 16);
    }
  }
  for (int i = tid; i < n * half; i += kPagedThreads) {
    const int t = g.by_half(i), j = i - t * half;
    turn[i] = cos_sin((double)(lo + t) * g.inv_freq[j]);
  }
  __syncthreads();
  const int lines = g.by_lines.d;                                // query heads, the key, the value
  const int rotated = g.rot / (2 * EPL);                         // pairs of pieces that turn
  // line by line (query heads, key, value), so that the lanes of a wavefront do the same; (i + 1/2) / m in 32 bits is off by less than 2^-11 below 2^14
  const int m = n * PAIRS;
  const float each = 1.f / (float)m;
  for (int i = tid; i < lines * m; i += kPagedThreads) {
    const int line = (int)(((float)i + 0.5f) * each), j = i - line * m, p = j % PAIRS, t = j / PAIRS;
    const bool is_v = line == lines - 1, is_k = line == lines - 2;
    const char* src = is_v   ? g.v + (int64_t)(first_row + t) * g.v_row + h * g.v_head
                      : is_k ? g.k + (int64_t)(first_row + t) * g.k_row + h * g.k_head
                             : g.q + (int64_t)(first_row + t) * g.q_row + (int64_t)(h * g.G + line) * g.q_head;
    const bool turns = !is_v && p < rotated;
    // the two pieces: first and second halves of the pairs; of the row, which a row's lanes then read and write without gaps; or neighbours
    const bool whole = is_v || rotated == PAIRS || rotated == 0, first = whole || (turns && !g.adjacent);
    const int pa = first ? p : 2 * p, pb = whole ? p + PAIRS : first ? p + rotated : 2 * p + 1;
    u32x4 ua = gload128(src + pa * 16), ub = gload128(src + pb * 16);
    u32x4 wa, wb;
    const char* weights = nullptr;
    if constexpr (NORM) {
      weights = is_v ? nullptr : is_k ? g.kw : g.qw;
      if (weights) {
        weights += is_k ? h * g.kw_head : (int64_t)(h * g.G + line) * g.qw_head;
        wa = gload128(weights + pa * 16);
        wb = gload128(weights + pb * 16);
      }
    }
    char* dst;
    uint8_t* scale_dst = nullptr;
    if (line < lines - 2) {
      dst = g.out + (int64_t)(first_row + t) * g.out_row + (int64_t)(h * g.G + line) * g.out_head;
    } else {
      const int pt = page_of(g, lo + t), id = page_id(g, f.index, pt, &lost);
      dst = id < 0 ? nullptr : (is_v ? g.V : g.K) + (int64_t)id * g.st_page + h * g.st_head + (int64_t)(lo + t - pt * g.by_page.d) * g.st_tok;
      lost = lost || id < 0;
      if constexpr (CODES) scale_dst = (uint8_t*)(g.S + scale_at(g, max(id, 0), h, lo + t - pt * g.by_page.d)) + is_v;
    }
    Coded c;
    if (turns || (!is_v && (NORM || (CODES && is_k)))) {
      float a[EPL], b[EPL], x[EPL], y[EPL];
      Elem<T>::unpack(make_uint4(ua.x, ua.y, ua.z, ua.w), a);
      Elem<T>::unpack(make_uint4(ub.x, ub.y, ub.z, ub.w), b);
      if constexpr (NORM) {                                      // (a row's lanes are PAIRS neighbours)
        float sum = 0.f;
#pragma unroll
        for (int e = 0; e < EPL; ++e) sum = fmaf(a[e], a[e], fmaf(b[e], b[e], sum));
        const float by = __builtin_amdgcn_rsqf(fmaf(lanes_sum(sum, PAIRS), 1.f / D, g.eps));
#pragma unroll
        for (int e = 0; e < EPL; ++e) { a[e] *= by; b[e] *= by; }
        if (weights) {
          float fa[EPL], fb[EPL];
          Elem<T>::unpack(make_uint4(wa.x, wa.y, wa.z, wa.w), fa);
          Elem<T>::unpack(make_uint4(wb.x, wb.y, wb.z, wb.w), fb);
#pragma unroll
          for (int e = 0; e < EPL; ++e) { a[e] *= fa[e] + g.w_offset; b[e] *= fb[e] + g.w_offset; }
        }
      }
      const float2* cs = turn + t * half + (g.adjacent ? pa * (EPL / 2) : p * EPL);
      if ((CODES || NORM) && !turns) {
#pragma unroll
        for (int e = 0; e < EPL; ++e) { x[e] = a[e]; y[e] = b[e]; }
      } else if (g.adjacent) {
#pragma unroll
        for (int e = 0; e < EPL; e += 2) {
          const float2 c0 = cs[e / 2], c2 = cs[(pb - pa) * (EPL / 2) + e / 2];
          x[e] = a[e] * c0.x - a[e + 1] * c0.y;
          x[e + 1] = a[e] * c0.y + a[e + 1] * c0.x;
          y[e] = b[e] * c2.x - b[e + 1] * c2.y;
          y[e + 1] = b[e] * c2.y + b[e + 1] * c2.x;
        }
      } else {
#pragma unroll
        for (int e = 0; e < EPL; ++e) {
          const float2 c0 = cs[e];
          x[e] = a[e] * c0.x - b[e] * c0.y;
          y[e] = a[e] * c0.y + b[e] * c0.x;
        }
      }
      bool packed = true;
      if constexpr (CODES) {
        packed = !is_k;
        if (is_k) c = encode(x, y, PAIRS);
      }
      if (packed) {
        ua = pack16<T>(x);
        ub = pack16<T>(y);
      }
    }
    if constexpr (CODES)
      if (is_k || is_v) {
        if (is_v) c = encode(ua, ub, PAIRS);
        if (dst) {
          typedef __attribute__((address_space(1))) uint64_t* gout64;
          *(gout64)(dst + pa * 8) = (uint64_t)c.x[1] << 32 | c.x[0];
          *(gout64)(dst + pb * 8) = (uint64_t)c.y[1] << 32 | c.y[0];
          if (p == 0) *scale_dst = (uint8_t)c.scale;
          dst = nullptr;
        }
        if (is_k && fills) {                                     // the key as stored, for the mean
          const float scale = __uint_as_float(c.scale << 23);
          ua = decode8(c.x[0], c.x[1], scale);
          ub = decode8(c.y[0], c.y[1], scale);
        }
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

template <typename C, int D>
static void launch_append(const PagedGeom& g, dim3 grid, size_t lds, int tile, hipStream_t s) {
  if (g.normed) hipLaunchKernelGGL((paged_append_kernel<C, D, true>), grid, dim3(kPagedThreads), lds, s, g, tile);
  else hipLaunchKernelGGL((paged_append_kernel<C, D, false>), grid, dim3(kPagedThreads), lds, s, g, tile);
}
void launch_paged_append(const PagedGeom& g, hipStream_t s) {
  const int tile = g.block ? g.block : 16;
  // sequence by sequence a tile at either end may be cut
  const int64_t by_rows = g.rows / tile + 2ll * g.n_seqs, by_seqs = (int64_t)g.n_seqs * ((g.max_new - 2 + tile) / tile + 1);
  const unsigned tiles = (unsigned)(by_rows < by_seqs ? by_rows : by_seqs);
  const dim3 grid(tiles + 1, g.Hkv);                             // (the last one has a tile only where sequences share rows)
  const size_t lds = (size_t)tile * (g.rot / 2) * sizeof(float2) + (g.block ? (size_t)tile * g.d * (g.dtype == TKPHI_BF16 ? 2 : 4) : 0);
  if (g.S) {
    if (g.d == 64) launch_append<Code8, 64>(g, grid, lds, tile, s);
    else launch_append<Code8, 128>(g, grid, lds, tile, s);
  } else if (g.dtype == TKPHI_BF16) {
    if (g.d == 64) launch_append<uint16_t, 64>(g, grid, lds, tile, s);
    else launch_append<uint16_t, 128>(g, grid, lds, tile, s);
  } else {
    if (g.d == 64) launch_append<float, 64>(g, grid, lds, tile, s);
    else launch_append<float, 128>(g, grid, lds, tile, s);
  }
}

}  // namespace tkphi
