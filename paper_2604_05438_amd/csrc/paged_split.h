// The split kernel: attention of up to 32 query rows per KV head over the paged cache, and over listed blocks of it (bf16 and fp32 caches in
// paged_attention.hip, codes in paged_attention_codes.hip).
//
// One pass over the keys and values with the running maximum and sum of the softmax, on the matrix cores: a wavefront takes tiles
// of tokens against 16 (or 32) query rows, S^T = K Q^T, then O^T += V^T P^T.  The rows of S^T that a lane holds are exactly the inner
// indices it has to deliver of P^T, so P never leaves its lane; V passes through LDS, where the bf16 form reads it transposed.
// The query rows of an item are the new tokens times the query heads of one KV head (every cached row is read once for all of
// them); the work of all items is cut into equal pieces along the tokens, and the workgroup that finishes an item last joins its pieces (with a plan,
// paged_join_kernel does).
//
// Bound by the read stream where there is much of it: a step of 32 sequences of a 3B layer, 720000 cached tokens (2.96 GB), 450 us = 6.6 TB/s, as codes (1.49 GB)
// 235 us = 6.3 TB/s; five tokens each of 8 sequences (283 MB) 61 us.  Short calls are a chain of round trips: a 1B layer over 4002 tokens 8.5 us (as codes 8.2), of which, by the
// clock in the workgroup that ends last, sequences 1.3 (1.1), queries 0.2, page ids and rows 2.6 (2.0), the join of the wavefronts with the wait for them 0.6 (1.3),
// partials and their count 0.7, the join of 32 pieces 2.4 (2.3).
#pragma once

#include "paged_attention.h"

namespace tkphi {

typedef __attribute__((__vector_size__(8 * sizeof(__bf16)))) __bf16 pa_bf16x8;
typedef __attribute__((__vector_size__(4 * sizeof(short)))) short pa_s16x4;
typedef __attribute__((__vector_size__(4 * sizeof(float)))) float pa_floatx4;
typedef unsigned int pa_u32x2 __attribute__((ext_vector_type(2)));
union PagedFrag {
  u32x4 u;
  pa_bf16x8 v;
  pa_u32x2 h[2];
};

// 4 values of one channel out of 4 rows of LDS: the 16 lanes of a group point at 4 rows x 16 channels of bf16 (lane i at row i / 4, channels
// 4 (i % 4) ..) and lane i gets channel i of the four rows
__device__ __forceinline__ pa_u32x2 lds_read_transposed(const char* p) {
  return __builtin_bit_cast(pa_u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) pa_s16x4*)p));
}

__device__ __forceinline__ int64_t of_lane(int64_t x, int lane) {
  return (int64_t)(uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)x, lane) | (int64_t)__builtin_amdgcn_readlane((int)(x >> 32), lane) << 32;
}

// One wavefront's share of an item piece.
// T, D: storage, head dimension; RT: tiles of 16 query rows; STREAM: the cache is read once (non-temporal loads); UNIFORM: 8 tokens always lie in one page
// A load instruction covers 8 rows x 128 bytes, whole cache lines: lane (r, kg) takes 16 bytes of row r mod 8, in the first half of its line for
// r < 8, in the second for r >= 8.  Keys of 16 rows then change places between two registers to make plain operands; values go to LDS anyway.
// (Half lines at a time: 5.8 TB/s for a step of 32 sequences instead of 6.5.)
// WIDE: twice as many tokens at a time (codes of 64 channels, whose tiles are otherwise half as large as all others; see paged_api)
// PAIR: rows of codes of two KV heads of 64 channels that adjoin, as one of D = 128: query rows 0 .. 7 are of the first, 8 .. 15 of the second; a score takes the
// head's half of the channels, and of an output row only that half counts
template <typename T, int D, int RT, bool STREAM, bool UNIFORM, bool WIDE = false, bool PAIR = false>
struct WaveAttend {
  using Row = typename Cached<T>::Row;
  static constexpr bool BF = Cached<T>::bf16, CODES = Cached<T>::codes;
  static constexpr int RB = D * (int)sizeof(Row);                 // bytes of a row, as it is contracted
  static constexpr int SUB = WIDE ? 4 : BF ? 2 : 1;                          // subtiles of 16 tokens that are loaded and contracted together
  static constexpr int TOK = 16 * SUB;
  static constexpr int NP = (SUB + 1) / 2;                        // operands of weights: of 32 tokens each (fp32: 16)
  static constexpr int NF = RB / 64;                              // 16-byte pieces of a row per lane
  static constexpr int NL = D * Cached<T>::bytes / 64;            // of the row in the cache: fewer for codes (one, a whole row by 4 lanes, at D = 64)
  static constexpr int VROW = RB + 32;                            // LDS row of V
  static constexpr int LDS = TOK * VROW;                          // LDS bytes per wavefront
  static constexpr int CT = D / 16;

  PagedFrag q[RT][NF];
  pa_floatx4 o[RT][CT];                                           // O^T: channels 16 ct + 4 kg + i of query row (lane & 15)
  float m[RT], l[RT];                                             // running maximum (of the row) and sum (of this lane's tokens), base 2
  pa_floatx4 lr[RT];                                              // bf16: sum of the row's weights as rounded, as one more channel of 1 (in every element)
  int lim[RT], low[RT];                                           // tokens [low, lim] are seen by this lane's row

  __device__ __forceinline__ void reset() {
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
      m[rt] = -INFINITY;
      l[rt] = 0.f;
      lr[rt] = (pa_floatx4){0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int ct = 0; ct < CT; ++ct) o[rt][ct] = (pa_floatx4){0.f, 0.f, 0.f, 0.f};
    }
  }

  static constexpr int GR = TOK / 8;                              // groups of 8 tokens per tile

  // The cached rows of a tile, in groups of 8 tokens; lanes 8 u .. 8 u + 7 (of GR x 8) hold what is said of group u, in vector registers (as scalars they would be
  // spilled to those): the byte offset of the group's first row (not UNIFORM: of its row lane % 8), the position of its first token,
  // and which of its tokens anyone may see (the rows of the others are readable all the same).
  struct Rows {
    int64_t off;
    int pos, mask;
    int64_t scale;                                                 // codes: where the scales of token lane % TOK of the tile are
    __device__ __forceinline__ int64_t offset(int u) const {
      if constexpr (UNIFORM) {
        return of_lane(off, 8 * u);
      } else {                                                     // (looked up by every lane for all its rows, the lookups took longer than all else)
        const int from = (8 * u + (threadIdx.x & 7)) * 4;
        return (int64_t)(uint32_t)__builtin_amdgcn_ds_bpermute(from, (int)(uint32_t)off) | (int64_t)__builtin_amdgcn_ds_bpermute(from, (int)(off >> 32)) << 32;
      }
    }
    __device__ __forceinline__ int pos_of(int u) const { return __builtin_amdgcn_readlane(pos, 8 * u); }
    __device__ __forceinline__ int mask_of(int u) const { return __builtin_amdgcn_readlane(mask, 8 * u); }
  };
  static __device__ __forceinline__ int lane_offset() { return (NL > 1 ? ((threadIdx.x >> 3) & 1) * 64 : 0) + ((threadIdx.x >> 4) & 3) * 16; }
  // where query piece f of a lane lies in its row: the channels that piece f of a key has
  static __device__ __forceinline__ int query_offset(int f) {
    const int kg = (threadIdx.x >> 4) & 3;
    if constexpr (PAIR) return kg * 32 + (f & 1) * 16;             // (of the row's own head)
    return CODES ? (f >> 1) * 128 + kg * 32 + (f & 1) * 16 : f * 64 + kg * 16;
  }
  // `at`: what the lane adds to the groups' offsets
  __device__ __forceinline__ void load(const char* base, uint32_t at, const Rows& r, PagedFrag (&f)[SUB][NL]) {
#pragma unroll
    for (int s = 0; s < SUB; ++s) {
      if constexpr (NL == 1) {
        const int64_t first = r.offset(2 * s), second = r.offset(2 * s + 1);
        const char* p = base + (threadIdx.x & 8 ? second : first) + at;
        f[s][0].u = STREAM ? gload128_stream(p) : gload128(p);
      } else {
#pragma unroll
        for (int u = 0; u < 2; ++u)
#pragma unroll
          for (int j = 0; j < NL / 2; ++j) {
            const char* p = base + r.offset(2 * s + u) + at + j * 128;
            f[s][2 * j + u].u = STREAM ? gload128_stream(p) : gload128(p);
          }
      }
    }
  }
  static __device__ __forceinline__ uint32_t load_scales(const PagedGeom& g, const Rows& r) {
    typedef const __attribute__((address_space(1))) uint16_t* scales_ptr;
    if constexpr (PAIR) return *(scales_ptr)(g.S + r.scale) | (uint32_t)*(scales_ptr)(g.S + r.scale + g.by_page.d) << 16;
    else if constexpr (CODES) return *(scales_ptr)(g.S + r.scale);
    else return 0;
  }
  // of the scales that load_scales brought, those of token t of the tile
  static __device__ __forceinline__ uint32_t scales_of(uint32_t mine, int t) { return (uint32_t)__builtin_amdgcn_ds_bpermute(t * 4, (int)mine); }

  // the operands of 16 rows out of what two groups loaded: lanes 8 .. 15 of each row of 16 of the one <-> lanes 0 .. 7 of the other
  static __device__ __forceinline__ void to_operands(PagedFrag (&f)[NL]) {
#pragma unroll
    for (int j = 0; j + 1 < NL; j += 2) {
      const PagedFrag a = f[j], b = f[j + 1];
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        f[j].u[e] = (uint32_t)__builtin_amdgcn_update_dpp((int)a.u[e], (int)b.u[e], 0x128, 0xf, 0xc, false);
        f[j + 1].u[e] = (uint32_t)__builtin_amdgcn_update_dpp((int)b.u[e], (int)a.u[e], 0x128, 0xf, 0x3, false);
      }
    }
  }

  // pieces of a row of codes as they are contracted
  static __device__ __forceinline__ void decode(const PagedFrag (&c)[NL], uint32_t scales, PagedFrag (&k)[NF]) {
#pragma unroll
    for (int j = 0; j < NF; ++j) k[j].u = decode8(c[j / 2].u[2 * (j & 1)], c[j / 2].u[2 * (j & 1) + 1], key_scale(PAIR && j >= NF / 2 ? scales >> 16 : scales));
  }

  __device__ __forceinline__ pa_floatx4 score(const PagedFrag (&k)[NF], const PagedFrag (&qq)[NF]) {
    pa_floatx4 p = (pa_floatx4){0.f, 0.f, 0.f, 0.f};
    if constexpr (PAIR) {                                          // (each half by itself: a key of the one head may be no number)
      pa_floatx4 p1 = p;
#pragma unroll
      for (int j = 0; j < NF / 2; ++j) {
        p = __builtin_amdgcn_mfma_f32_16x16x32_bf16(k[j].v, qq[j].v, p, 0, 0, 0);
        p1 = __builtin_amdgcn_mfma_f32_16x16x32_bf16(k[NF / 2 + j].v, qq[NF / 2 + j].v, p1, 0, 0, 0);
      }
#pragma unroll
      for (int e = 0; e < 4; ++e) p[e] = threadIdx.x & 8 ? p1[e] : p[e];
    } else if constexpr (BF) {
#pragma unroll
      for (int j = 0; j < NF; ++j) p = __builtin_amdgcn_mfma_f32_16x16x32_bf16(k[j].v, qq[j].v, p, 0, 0, 0);
    } else {
      pa_floatx4 p1 = p;
#pragma unroll
      for (int j = 0; j < NF; ++j)
#pragma unroll
        for (int e = 0; e < 4; e += 2) {
          p = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(k[j].u[e]), __uint_as_float(qq[j].u[e]), p, 0, 0, 0);
          p1 = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(k[j].u[e + 1]), __uint_as_float(qq[j].u[e + 1]), p1, 0, 0, 0);
        }
      p += p1;
    }
    return p;
  }

  static __device__ __forceinline__ bool not_finite(const u32x4 w) {
    bool odd = false;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      if constexpr (BF) odd = odd || (w[e] & 0x7f80u) == 0x7f80u || (w[e] & 0x7f800000u) == 0x7f800000u;
      else odd = odd || (w[e] & 0x7f800000u) == 0x7f800000u;
    }
    return odd;
  }

  // O^T += V^T P^T of a tile, token by token for the rows that see it
  __device__ __forceinline__ void add_seen(const PagedFrag (&p)[RT][NP], const Rows& rows, const char* vlds) {
    const int lane = threadIdx.x & 63, r = lane & 15, kg = lane >> 4;
#pragma unroll
    for (int u = 0; u < SUB; ++u)
#pragma unroll
      for (int e = 0; e < 4; ++e)
        for (int k = 0; k < 4; ++k) {
          const int slot = 4 * k + e, in = slot & 7;
          const int pos = (k >> 1 ? rows.pos_of(2 * u + 1) : rows.pos_of(2 * u)) + in;
          const bool there = ((k >> 1 ? rows.mask_of(2 * u + 1) : rows.mask_of(2 * u)) >> in) & 1;
          const char* v = vlds + (u * 16 + slot) * VROW;
#pragma unroll
          for (int rt = 0; rt < RT; ++rt) {
            const uint32_t word = __shfl(p[rt][u / 2].u[BF ? 2 * (u & 1) + e / 2 : e], 16 * k + r);
            const float weight = __uint_as_float(!BF ? word : e & 1 ? word & 0xffff0000u : word << 16);
            if (!there || pos < low[rt] || pos > lim[rt]) continue;
#pragma unroll
            for (int ct = 0; ct < CT; ++ct)
#pragma unroll
              for (int i = 0; i < 4; ++i) o[rt][ct][i] = fmaf(weight, Elem<Row>::load1(v, ct * 16 + kg * 4 + i), o[rt][ct][i]);
          }
        }
  }

  // rows_of(i): the rows of its tile i; tiles 0 .. n - 1.  clean(i): every row sees every token of tile i.  at: see load().
  template <typename RowsOf, typename Clean>
  __device__ __forceinline__ void run(const PagedGeom& g, int h, char* vlds, int n, uint32_t lane_at, RowsOf&& rows_of, Clean&& clean) {
    if (n <= 0) return;
    const int lane = threadIdx.x & 63, r = lane & 15, kg = lane >> 4, r7 = lane & 7;
    const char* Kb = g.K + h * g.st_head;
    const char* Vb = g.V + h * g.st_head;
    char* const vw = vlds + (NL > 1 ? r7 : r) * VROW + lane_offset() * (CODES ? 2 : 1);
    PagedFrag kf[SUB][NL], vf[SUB][NL];
    Rows cur = rows_of(0);
    load(Kb, lane_at, cur, kf);
    uint32_t scales = load_scales(g, cur), scales_next = 0;
    load(Vb, lane_at, cur, vf);
    Rows nxt = rows_of(min(1, n - 1));
    for (int i = 0; i < n; ++i) {
      const Rows here = cur;
      cur = nxt;
      // ---- scores
      pa_floatx4 s[SUB][RT];
#pragma unroll
      for (int u = 0; u < SUB; ++u) {
        to_operands(kf[u]);
        if constexpr (CODES) {
          PagedFrag k[NF];
          decode(kf[u], scales_of(scales, 16 * u + r), k);
#pragma unroll
          for (int rt = 0; rt < RT; ++rt) s[u][rt] = score(k, q[rt]);
        } else {
#pragma unroll
          for (int rt = 0; rt < RT; ++rt) s[u][rt] = score(kf[u], q[rt]);
        }
      }
      if (i + 1 < n) {
        load(Kb, lane_at, cur, kf);
        scales_next = load_scales(g, cur);
      }
      nxt = rows_of(min(i + 2, n - 1));
      // ---- what nobody may see
      const bool all = clean(i) && __all(here.mask == 0xff);
      if (!all) {
#pragma unroll
        for (int u = 0; u < SUB; ++u) {
          const int pos0 = (kg < 2 ? here.pos_of(2 * u) : here.pos_of(2 * u + 1)) + 4 * (kg & 1);
          const int bits = (kg < 2 ? here.mask_of(2 * u) : here.mask_of(2 * u + 1)) >> (4 * (kg & 1));
#pragma unroll
          for (int e = 0; e < 4; ++e)
#pragma unroll
            for (int rt = 0; rt < RT; ++rt)
              if (!((bits >> e) & 1) || pos0 + e < low[rt] || pos0 + e > lim[rt]) s[u][rt][e] = -INFINITY;
        }
      }
      // ---- running maximum and sum
      PagedFrag p[RT][NP];
#pragma unroll
      for (int rt = 0; rt < RT; ++rt) {
        float x[SUB][4], mx = -INFINITY;
#pragma unroll
        for (int u = 0; u < SUB; ++u)
#pragma unroll
          for (int e = 0; e < 4; ++e) mx = fmaxf(mx, s[u][rt][e]);
        mx = across_32(across_16(mx, MaxOp()), MaxOp()) * g.scale2;
        const float mn = fmaxf(m[rt], mx);
        const float ref = mn == -INFINITY ? 0.f : mn;              // (nothing seen yet: exp2(-inf - 0) = 0)
        const float fix = __builtin_amdgcn_exp2f(m[rt] - ref);
        m[rt] = mn;
        float sum = 0.f;
#pragma unroll
        for (int u = 0; u < SUB; ++u)
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            if constexpr (BF) x[u][e] = __builtin_amdgcn_exp2f(fmaf(s[u][rt][e], g.scale2, -ref));
            else x[u][e] = __builtin_amdgcn_exp2f(s[u][rt][e] == -INFINITY ? -INFINITY : fmaf(s[u][rt][e], g.scale2, fmaf(s[u][rt][e], g.scale2_lo, -ref)));
            sum += x[u][e];
          }
        l[rt] = fmaf(l[rt], fix, sum);
        if (__any(fix != 1.f)) {                                   // (a maximum is rarely passed after the first tiles)
#pragma unroll
          for (int ct = 0; ct < CT; ++ct) o[rt][ct] *= fix;
          if constexpr (BF) lr[rt] *= fix;
        }
        if constexpr (BF) {                                        // (the weights enter the product in the cache's own type)
#pragma unroll
          for (int u = 0; u < SUB; ++u)
#pragma unroll
            for (int e = 0; e < 2; ++e)
              p[rt][u / 2].u[2 * (u & 1) + e] = __builtin_bit_cast(uint32_t, (bf16x2_t){(__bf16)x[u][2 * e], (__bf16)x[u][2 * e + 1]});
        } else {
#pragma unroll
          for (int e = 0; e < 4; ++e) p[rt][0].u[e] = __float_as_uint(x[0][e]);
        }
      }
      // ---- V through LDS; rows that nobody sees as zeros, whatever they hold
      bool odd = false;                                            // a value that is no number, or infinite, which some rows may not see
      if constexpr (CODES) {
        constexpr int PER = NL > 1 ? 1 : 2;                        // groups of 8 rows per load
#pragma unroll
        for (int u = 0; u < GR; u += PER) {
          const int first = here.mask_of(u), second = here.mask_of(u + PER - 1), mask = lane & 8 && PER == 2 ? second : first;
          const uint32_t both = scales_of(scales, 8 * u + (PER == 1 ? r7 : r));
          const float scale = value_scale(PAIR ? (lane & 8 ? both >> 16 : both & 0xffffu) : both);
          const u32x4 c = vf[u / 2][PER == 1 ? u % 2 : 0].u;
#pragma unroll
          for (int x = 0; x < 2; ++x) {
            u32x4 w = decode8(c[2 * x], c[2 * x + 1], scale);
            if (!all) {
              if (!((mask >> r7) & 1)) w = (u32x4){0u, 0u, 0u, 0u};
              odd = odd || not_finite(w);
            }
            *(u32x4*)(vw + u * 8 * VROW + x * 16) = w;
          }
        }
        scales = scales_next;
      } else {
#pragma unroll
        for (int u = 0; u < GR; ++u)
#pragma unroll
          for (int j = 0; j < NF / 2; ++j) {
            u32x4 w = vf[u / 2][2 * j + u % 2].u;
            if (!all) {
              if (!((here.mask_of(u) >> r7) & 1)) w = (u32x4){0u, 0u, 0u, 0u};
              odd = odd || not_finite(w);
            }
            *(u32x4*)(vw + u * 8 * VROW + j * 128) = w;
          }
      }
      if (i + 1 < n) load(Vb, lane_at, cur, vf);
      if constexpr (BF) {
        PagedFrag ones;
        ones.u = (u32x4){0x3f803f80u, 0x3f803f80u, 0x3f803f80u, 0x3f803f80u};
#pragma unroll
        for (int rt = 0; rt < RT; ++rt)
#pragma unroll
          for (int x = 0; x < NP; ++x) lr[rt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(ones.v, p[rt][x].v, lr[rt], 0, 0, 0);
      }
      if (!all && __ballot(odd)) {                                 // (0 times such a value is not 0: row by row, without what they do not see)
        add_seen(p, here, vlds);
        continue;
      }
      if constexpr (BF) {
#pragma unroll
        for (int x = 0; x < NP; ++x)
#pragma unroll
          for (int ct = 0; ct < CT; ++ct) {
            PagedFrag a;
            const char* at = vlds + (x * 32 + kg * 4 + (r >> 2)) * VROW + ct * 32 + (r & 3) * 8;
            a.h[0] = lds_read_transposed(at);
            a.h[1] = lds_read_transposed(at + 16 * VROW);
#pragma unroll
            for (int rt = 0; rt < RT; ++rt) o[rt][ct] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a.v, p[rt][x].v, o[rt][ct], 0, 0, 0);
          }
      } else {
#pragma unroll
        for (int e = 0; e < 4; ++e)
#pragma unroll
          for (int ct = 0; ct < CT; ++ct) {
            const float a = *(const float*)(vlds + (kg * 4 + e) * VROW + ct * 64 + r * 4);
#pragma unroll
            for (int rt = 0; rt < RT; ++rt) o[rt][ct] = __builtin_amdgcn_mfma_f32_16x16x4f32(a, __uint_as_float(p[rt][0].u[e]), o[rt][ct], 0, 0, 0);
          }
      }
    }
  }
};

constexpr int pmax(int a, int b) { return a > b ? a : b; }
template <typename T, int D, int RT, bool WIDE = false>
constexpr int attend_lds() { return pmax(pmax(WaveAttend<T, D, RT, true, true, WIDE>::LDS, 16 * RT * (D + 2) * 4) * (kPagedThreads / 64), join_lds(kPagedThreads, 16 * RT)); }

// Joins the wavefronts of the workgroup through LDS, [waves][rows][D + 2] (O, m, l); emit(row, channel, O of it and the next one, m, l).
template <typename T, int D, int RT, bool STREAM, bool UNIFORM, bool WIDE, bool PAIR, typename Emit>
__device__ __forceinline__ void join_waves(WaveAttend<T, D, RT, STREAM, UNIFORM, WIDE, PAIR>& w, char* lds, int rows, Emit&& emit) {
  constexpr int W = kPagedThreads / 64, R = 16 * RT, STR = D + 2;
  const int lane = threadIdx.x & 63, r = lane & 15, kg = lane >> 4, wave = threadIdx.x >> 6;
  float* mine = (float*)lds + (size_t)wave * R * STR;
  __syncthreads();                                                 // (every wavefront is done with its V rows)
#pragma unroll
  for (int rt = 0; rt < RT; ++rt) {
    const float l = across_32(across_16(w.l[rt], AddOp()), AddOp());
    float f = 1.f;
    if constexpr (Cached<T>::bf16) f = to_sum(l, w.lr[rt][0]);
    float* row = mine + (rt * 16 + r) * STR;
#pragma unroll
    for (int ct = 0; ct < D / 16; ++ct)
#pragma unroll
      for (int i = 0; i < 4; ++i) row[ct * 16 + kg * 4 + i] = w.o[rt][ct][i] * f;
    if (kg == 0) { row[D] = w.m[rt]; row[D + 1] = l; }
  }
  __syncthreads();
  for (int x = threadIdx.x; x < rows * (D / 2); x += kPagedThreads) {
    const int row = x / (D / 2), c = x % (D / 2) * 2;
    const float* at = (const float*)lds + row * STR;
    float m = -INFINITY, l = 0.f;
    float2 o = make_float2(0.f, 0.f);
#pragma unroll
    for (int k = 0; k < W; ++k) m = fmaxf(m, at[k * R * STR + D]);
    const float ref = m == -INFINITY ? 0.f : m;
#pragma unroll
    for (int k = 0; k < W; ++k) {
      const float f = __builtin_amdgcn_exp2f(at[k * R * STR + D] - ref);
      l = fmaf(at[k * R * STR + D + 1], f, l);
      o.x = fmaf(at[k * R * STR + c], f, o.x);
      o.y = fmaf(at[k * R * STR + c + 1], f, o.y);
    }
    emit(row, c, o, m, l);
  }
}

// UNIFORM: 8 tokens always lie in one page
// STREAM: non-temporal loads, where a workgroup is the only one that reads a line: every sequence has one item per KV head, whose rows are whole lines.  (With several items of a sequence they read the same
// rows.  128 single tokens over up to 8000, which have a plan for their number: 378 us, with plain loads 416.)  WIDE, PAIR: see WaveAttend
template <typename T, int D, int RT, bool PLAN, bool UNIFORM, bool STREAM, bool WIDE = false, bool PAIR = false>
__global__ __launch_bounds__(kPagedThreads, attend_per_cu(D, RT)) void paged_attend_kernel(PagedGeom g) {
  using Wave = WaveAttend<T, D, RT, STREAM, UNIFORM, WIDE, PAIR>;
  constexpr int WAVES = kPagedThreads / 64, HD = PAIR ? D / 2 : D;
  __shared__ __align__(16) char lds[attend_lds<T, D, RT, WIDE>()];
  __shared__ int sh_last;
  const int lane = threadIdx.x & 63, r = lane & 15, wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));

  const int w = blockIdx.x;
  const auto sh = share_of<PLAN>(g, w);
  Wave at;
  int hint = -1;
  JoinRecord join;
  for (auto x = sh.begin; x < sh.end;) {
    const auto p = piece_at<PLAN>(g, sh, x, &hint);
    const PagedSeq s = p.s;
    const ItemRange it = p.it;
    const int h = PAIR ? 2 * p.h : p.h, seq = p.seq;
    const int rows = PAIR ? 2 * it.rows : it.rows;                 // (PAIR: those of the second head behind those of the first)
    const auto place = [&](int row, int* token, int* head) {
      if constexpr (PAIR) {
        const int second = row >= it.rows, x = row - (second ? it.rows : 0), i = g.by_group(x);
        *token = s.row + i;
        *head = (h + second) * g.G + x - i * g.G;
      } else {
        p.place(g, row, token, head);
      }
    };
    const int t0 = it.begin + (p.u0 << g.unit_shift), t1 = min(it.begin + (p.u1 << g.unit_shift), it.end);
    bool bad = false;

    // ---- this piece: tokens [t0, t1)
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
      const bool live = PAIR ? (r & 7) < it.rows : rt * 16 + r < it.rows;
      int token, head;
      place(PAIR ? (r & 7) + (r >> 3) * it.rows : rt * 16 + r, &token, &head);
      const int i = token - s.row;
      at.lim[rt] = live ? s.cached + i : -1;
      at.low[rt] = live ? (g.window > 0 ? max(0, s.cached + i + 1 - g.window) : 0) : 1;
      const char* src = g.q + (int64_t)token * g.q_row + (int64_t)head * g.q_head;
#pragma unroll
      for (int f = 0; f < Wave::NF; ++f) {
        at.q[rt][f].u = (u32x4){0u, 0u, 0u, 0u};
        if (live && (!PAIR || f / (Wave::NF / 2) == r >> 3)) at.q[rt][f].u = gload128(src + Wave::query_offset(f));
      }
    }
    const int seen_all = s.cached + (PLAN ? g.by_group(p.tile * g.tile_rows) : 0);         // last token that every row sees
    const int low_all = g.window > 0 ? it.end - g.window : 0;      // first one (rows of no query may come out as they like)
    at.reset();
    const int tiles = (t1 - t0 + Wave::TOK - 1) / Wave::TOK, mine = (tiles - wave + WAVES - 1) / WAVES;
    const auto tile0 = [&](int i) { return t0 + (wave + i * WAVES) * Wave::TOK; };
    const uint32_t lane_at = Wave::lane_offset() + (UNIFORM ? (uint32_t)(lane & 7) * (uint32_t)g.st_tok : 0u);
    at.run(g, h, lds + wave * Wave::LDS, mine, lane_at,
           [&](int i) {
             typename Wave::Rows rows{};
             const int tb = tile0(i);
             if constexpr (UNIFORM) {                              // lanes 8 u .. 8 u + 7 look up the page of group u (scalar code took twice as long as all else)
               const int t = tb + (lane >> 3) % Wave::GR * 8, pt = page_of(g, t), in = t - pt * g.by_page.d;
               const int from = max(it.low - t, 0), to = min(t1 - t, 8);                        // tokens [from, to) of the group
               bool odd = false;
               const int id = page_id(g, seq, pt, &odd), there = from < to ? id : -1;
               bad = bad || (odd && from < to);
               rows.off = (int64_t)max(there, 0) * g.st_page + (int64_t)in * g.st_tok;
               rows.pos = t;
               rows.mask = there < 0 ? 0 : ((1 << to) - 1) & ~((1 << from) - 1);
               if constexpr (Wave::CODES) rows.scale = scale_at(g, max(there, 0), h, in) + (lane & 7);
             } else {                                              // every lane its token
               const int mine = (lane >> 3) % Wave::GR, t = tb + lane % Wave::TOK, pt = page_of(g, t), in = t - pt * g.by_page.d;
               const int id = t >= it.low && t < t1 ? page_id(g, seq, pt, &bad) : -1;
               rows.off = (int64_t)max(id, 0) * g.st_page + (int64_t)in * g.st_tok;
               rows.pos = tb + mine * 8;
               rows.mask = (int)(__ballot(id >= 0) >> (8 * mine) & 0xff);
               if constexpr (Wave::CODES) rows.scale = scale_at(g, max(id, 0), h, in);
             }
             return rows;
           },
           [&](int i) { return tile0(i) >= low_all && tile0(i) + Wave::TOK - 1 <= seen_all; });

    // ---- out, or a partial
    const bool whole = p.whole();
    float* slot = partial_slot(g, w, x == sh.begin);
    join_waves<T, D, RT, STREAM, UNIFORM, WIDE, PAIR>(at, lds, PAIR ? 8 + it.rows : it.rows, [&](int row, int c, float2 o, float m, float l) {
      if constexpr (PAIR) {
        const int second = row >> 3;
        if ((row & 7) >= it.rows || (c >= HD) != (second != 0)) return;
        row = (row & 7) + (second ? it.rows : 0);
        c -= second ? HD : 0;
      }
      if (whole) {
        int token, head;
        place(row, &token, &head);
        store_out<typename Wave::Row>(g, token, head, c, o, m, l);
      } else if constexpr (PLAN) {
        *(float2*)(slot + row * HD + c) = o;
        if (c == 0) *(float2*)(slot + g.tile_rows * HD + row * 2) = make_float2(m, l);
      } else {
        store_pair(slot + row * HD + c, o.x, o.y);
        if (c == 0) store_pair(slot + g.tile_rows * HD + row * 2, m, l);
      }
    });
    report_pages(g, bad);
    if constexpr (!PLAN) {
      if (!whole) finish_item<typename Wave::Row, HD, kPagedThreads>(g, sh, p, rows, place, lds, &sh_last);
    }
    if constexpr (PLAN) join.note(g, sh, p, w, x == sh.begin);
    __syncthreads();
    x = min(sh.end, p.item1);
  }
  if constexpr (PLAN) join.store(g, w);
}

// ---- over blocks: `splits` workgroups per query token and KV head, each with an equal share of the listed blocks' tokens.  Non-temporal loads: of one token each of 64
// sequences, 128 blocks of codes of 64 channels, 118 us (plain loads 121), tokens outermost 141 (146), over bf16 139 (152).  Tokens of one sequence read the same blocks in
// part: 512 of them, d = 128, 479 us over codes and 648 over bf16 (plain loads 441, 637).
template <typename T, int D>
__global__ __launch_bounds__(kPagedThreads) void block_attend_kernel(PagedGeom g) {
  using Wave = WaveAttend<T, D, 1, true, true>;
  constexpr int WAVES = kPagedThreads / 64;
  __shared__ __align__(16) char lds[attend_lds<T, D, 1>()];
  __shared__ int sh_last;
  const int lane = threadIdx.x & 63, r = lane & 15, wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));
  const int h = blockIdx.y, local = blockIdx.z, token = g.row0 + local, split = blockIdx.x;
  const int64_t at_list = (int64_t)local * g.Hkv + h;
  const int4 head = g.list_head[at_list];                          // entries, position of the query, its sequence; 0 entries: a row of no sequence
  if (head.x <= 0) return;
  const int2* list = g.list + at_list * g.kept;
  const int slots = head.x * g.block;                              // listed blocks times tokens
  const int tiles = (slots + Wave::TOK - 1) / Wave::TOK;
  const int a = (int)((int64_t)tiles * split / g.splits), b = (int)((int64_t)tiles * (split + 1) / g.splits);

  Wave at;
  at.lim[0] = r < g.G ? head.y : -1;
  at.low[0] = r < g.G ? 0 : 1;
  const char* src = g.q + (int64_t)token * g.q_row + (int64_t)(h * g.G + min(r, g.G - 1)) * g.q_head;
#pragma unroll
  for (int f = 0; f < Wave::NF; ++f) {
    at.q[0][f].u = (u32x4){0u, 0u, 0u, 0u};
    if (r < g.G) at.q[0][f].u = gload128(src + Wave::query_offset(f));
  }
  at.reset();
  const int per = g.by_page.d / g.block, shift = 31 - __builtin_clz(g.block);          // (a power of two of at least 16 tokens, in one page)
  const auto tile_slot = [&](int i) { return (a + wave + i * WAVES) * Wave::TOK; };
  at.run(g, h, lds + wave * Wave::LDS, (b - a - wave + WAVES - 1) / WAVES, Wave::lane_offset() + (uint32_t)(lane & 7) * (uint32_t)g.st_tok,
         [&](int i) {
           typename Wave::Rows rows{};
           const int t0 = tile_slot(i), t = t0 + (lane >> 3) % Wave::GR * 8, in = t & (g.block - 1);      // lanes 8 u .. 8 u + 7: group u
           const int2 blk = list[min(t >> shift, head.x - 1)];
           const int page_row = (blk.y % per << shift) + in, pos = (blk.y << shift) + in, n = head.y + 1 - pos;          // tokens up to the query's own
           rows.off = (int64_t)max(blk.x, 0) * g.st_page + (int64_t)page_row * g.st_tok;
           rows.pos = pos;
           rows.mask = blk.x < 0 || n <= 0 || t >= slots ? 0 : n >= 8 ? 0xff : (1 << n) - 1;
           if constexpr (Wave::CODES) rows.scale = scale_at(g, max(blk.x, 0), h, page_row) + (lane & 7);
           return rows;
         },
         [&](int) { return true; });                               // (all rows are the same token's)
  const int pieces = min(g.splits, tiles);
  const bool whole = pieces == 1;
  float* part = g.partial + at_list * g.splits * 16 * (D + 2);
  // (with fewer tiles than workgroups some have none: piece p belongs to the p-th workgroup with one)
  if (a == b) return;
  const int piece = tiles < g.splits ? a : split;
  float* slot = part + (int64_t)piece * 16 * (D + 2);
  join_waves<T, D, 1, true, true, false, false>(at, lds, g.G, [&](int row, int c, float2 o, float m, float l) {
    if (whole) {
      store_out<typename Wave::Row>(g, token, h * g.G + row, c, o, m, l);
    } else {
      store_pair(slot + row * D + c, o.x, o.y);
      if (c == 0) store_pair(slot + 16 * D + row * 2, m, l);
    }
  });
  if (!whole && last_to_arrive(g.arrived + at_list, pieces, &sh_last))
    join_pieces<typename Wave::Row, D, kPagedThreads, true>(g, pieces, 0, g.G, 16, lds, [&](int p) { return part + (int64_t)p * 16 * (D + 2); },
                      [&](int row, int* t, int* hd) { *t = token; *hd = h * g.G + row; });
}

static inline bool groups_in_pages(const PagedGeom& g) { return g.by_page.d % 8 == 0 && g.st_tok < (1ll << 28); }       // (offsets of 32 bits within 8 tokens)
template <typename T, int D, int RT, bool PLAN, bool STREAM>
static void launch_split(const PagedGeom& g, hipStream_t s) {
  const bool uniform = groups_in_pages(g);
  const dim3 grid(g.splits), block(kPagedThreads);
  if constexpr (Cached<T>::codes && D == 64 && RT == 1) {
    if constexpr (!PLAN && STREAM)
      if (g.pairs) {
        hipLaunchKernelGGL((paged_attend_kernel<T, 128, RT, PLAN, true, STREAM, false, true>), grid, block, 0, s, g);
        return;
      }
    if (g.wide && uniform) {
      hipLaunchKernelGGL((paged_attend_kernel<T, D, RT, PLAN, true, STREAM, true>), grid, block, 0, s, g);
      return;
    }
  }
  if constexpr (PLAN || STREAM)
    if (!uniform) {
      hipLaunchKernelGGL((paged_attend_kernel<T, D, RT, PLAN, false, STREAM>), grid, block, 0, s, g);
      return;
    }
  hipLaunchKernelGGL((paged_attend_kernel<T, D, RT, PLAN, true, STREAM>), grid, block, 0, s, g);
}
template <typename T, int D, int RT>
static void launch_split(const PagedGeom& g, hipStream_t s) {
  // Codes of 64 channels, tokens outermost: the other half of a line is another workgroup's.  128 single tokens over 4000 to 8000 253 us with STREAM, 219 without, on pages
  // of 100 tokens 254 and 232; without a plan 3 tokens each of 32 sequences of 2000 to 65000 334 and 251, of 500 to 2000 27.1 and 26.6, one token of three heads
  // 93 and 91; but on pages of 100 tokens, without a plan, 234 and 259.
  const bool half_lines = Cached<T>::codes && D == 64 && g.st_tok != 64;
  if constexpr (Cached<T>::codes && D == 64)
    if (!g.plan_room && half_lines && !g.pairs && groups_in_pages(g)) {
      launch_split<T, D, RT, false, false>(g, s);
      return;
    }
  if (!g.plan_room) launch_split<T, D, RT, false, true>(g, s);
  else if ((int64_t)g.max_new * g.G <= g.tile_rows && !half_lines) launch_split<T, D, RT, true, true>(g, s);
  else launch_split<T, D, RT, true, false>(g, s);
}
// the items of a call of at most 32 rows per KV head, one token's blocks
template <typename T, int D>
static void launch_split_rows(const PagedGeom& g, hipStream_t s) {
  if (g.tile_rows <= 16) launch_split<T, D, 1>(g, s);
  else launch_split<T, D, 2>(g, s);
}
template <typename T, int D>
static void launch_blocks(const PagedGeom& g, hipStream_t s) {
  hipLaunchKernelGGL((block_attend_kernel<T, D>), dim3(g.splits, g.Hkv, g.row_group), dim3(kPagedThreads), 0, s, g);
}

}  // namespace tkphi
