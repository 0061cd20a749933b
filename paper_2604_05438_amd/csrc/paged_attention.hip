// Attention of new tokens over the paged cache: tkphi_paged_attention, and the attention part of tkphi_block_attention.
//
// One pass over the keys and values with the running maximum and sum of the softmax, on the matrix cores: a wavefront takes tiles
// of tokens against 16 (or 32) query rows, S^T = K Q^T, then O^T += V^T P^T.  The rows of S^T that a lane holds are exactly the inner
// indices it has to deliver of P^T, so P never leaves its lane; V passes through LDS, where the bf16 form reads it transposed.
// The query rows of an item are the new tokens times the query heads of one KV head (every cached row is read once for all of
// them); the work of all items is cut into equal pieces along the tokens, and the workgroup that finishes an item last joins its pieces (with a plan,
// paged_join_kernel does).
//
// Bound by the read stream where there is much of it: a step of 32 sequences of a 3B layer, 720000 cached tokens (2.96 GB), 455 us = 6.5 TB/s; five tokens
// each of 8 sequences (283 MB) 62 us.  Short calls are a chain of round trips: a 1B layer over 4002 tokens 9.4 us, of which sequences 0.7, page ids and
// rows 2.5, the join of the wavefronts 0.6, partials and their count 1.5, the join of 32 pieces 2.5.
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

// One wavefront's share of an item piece.
// T, D: storage, head dimension; RT: tiles of 16 query rows; STREAM: the cache is read once (non-temporal loads)
// A load instruction covers 8 rows x 128 bytes, whole cache lines: lane (r, kg) takes 16 bytes of row r mod 8, in the first half of its line for
// r < 8, in the second for r >= 8.  Keys of 16 rows then change places between two registers to make plain operands; values go to LDS anyway.
// (Half lines at a time: 5.8 TB/s for a step of 32 sequences instead of 6.5.)
template <typename T, int D, int RT, bool STREAM>
struct WaveAttend {
  static constexpr bool BF = sizeof(T) == 2;
  static constexpr int RB = D * (int)sizeof(T);                   // bytes of a row
  static constexpr int SUB = BF ? 2 : 1;                          // subtiles of 16 tokens that are loaded and contracted together
  static constexpr int TOK = 16 * SUB;
  static constexpr int NF = RB / 64;                              // 16-byte pieces of a row per lane
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

  // The cached rows of a tile: byte offset of the lane's row of each group of 8, the position of the group's first token, and which of
  // its tokens anyone may see (the rows of the others are readable all the same).
  struct Rows {
    int64_t off[GR];
    int pos[GR], mask[GR];
  };
  static __device__ __forceinline__ int lane_offset() { return ((threadIdx.x >> 3) & 1) * 64 + ((threadIdx.x >> 4) & 3) * 16; }

  // `at`: what the lane adds to the groups' offsets
  __device__ __forceinline__ void load(const char* base, uint32_t at, const Rows& r, PagedFrag (&f)[SUB][NF]) {
#pragma unroll
    for (int s = 0; s < SUB; ++s)
#pragma unroll
      for (int u = 0; u < 2; ++u)
#pragma unroll
        for (int j = 0; j < NF / 2; ++j) {
          const char* p = base + r.off[2 * s + u] + at + j * 128;
          f[s][2 * j + u].u = STREAM ? gload128_stream(p) : gload128(p);
        }
  }

  // the operands of 16 rows out of what two groups loaded: lanes 8 .. 15 of each row of 16 of the one <-> lanes 0 .. 7 of the other
  static __device__ __forceinline__ void to_operands(PagedFrag (&f)[NF]) {
#pragma unroll
    for (int j = 0; j < NF; j += 2) {
      const PagedFrag a = f[j], b = f[j + 1];
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        f[j].u[e] = (uint32_t)__builtin_amdgcn_update_dpp((int)a.u[e], (int)b.u[e], 0x128, 0xf, 0xc, false);
        f[j + 1].u[e] = (uint32_t)__builtin_amdgcn_update_dpp((int)b.u[e], (int)a.u[e], 0x128, 0xf, 0x3, false);
      }
    }
  }

  __device__ __forceinline__ pa_floatx4 score(const PagedFrag (&k)[NF], const PagedFrag (&qq)[NF]) {
    pa_floatx4 p = (pa_floatx4){0.f, 0.f, 0.f, 0.f};
    if constexpr (BF) {
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
  __device__ __forceinline__ void add_seen(const PagedFrag (&p)[RT][(SUB + 1) / 2], const Rows& rows, const char* vlds) {
    const int lane = threadIdx.x & 63, r = lane & 15, kg = lane >> 4;
#pragma unroll
    for (int u = 0; u < SUB; ++u)
#pragma unroll
      for (int e = 0; e < 4; ++e)
        for (int k = 0; k < 4; ++k) {
          const int slot = 4 * k + e, in = slot & 7;
          const int pos = (k >> 1 ? rows.pos[2 * u + 1] : rows.pos[2 * u]) + in;
          const bool there = ((k >> 1 ? rows.mask[2 * u + 1] : rows.mask[2 * u]) >> in) & 1;
          const char* v = vlds + (u * 16 + slot) * VROW;
#pragma unroll
          for (int rt = 0; rt < RT; ++rt) {
            const uint32_t word = __shfl(p[rt][0].u[BF ? 2 * u + e / 2 : e], 16 * k + r);
            const float weight = __uint_as_float(!BF ? word : e & 1 ? word & 0xffff0000u : word << 16);
            if (!there || pos < low[rt] || pos > lim[rt]) continue;
#pragma unroll
            for (int ct = 0; ct < CT; ++ct)
#pragma unroll
              for (int i = 0; i < 4; ++i) o[rt][ct][i] = fmaf(weight, Elem<T>::load1(v, ct * 16 + kg * 4 + i), o[rt][ct][i]);
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
    char* const vw = vlds + r7 * VROW + lane_offset();
    PagedFrag kf[SUB][NF], vf[SUB][NF];
    Rows cur = rows_of(0);
    load(Kb, lane_at, cur, kf);
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
#pragma unroll
        for (int rt = 0; rt < RT; ++rt) s[u][rt] = score(kf[u], q[rt]);
      }
      if (i + 1 < n) load(Kb, lane_at, cur, kf);
      nxt = rows_of(min(i + 2, n - 1));
      // ---- what nobody may see
      bool all = clean(i);
#pragma unroll
      for (int u = 0; u < GR; ++u) all = all && here.mask[u] == 0xff;
      if (!all) {
#pragma unroll
        for (int u = 0; u < SUB; ++u) {
          const int pos0 = (kg < 2 ? here.pos[2 * u] : here.pos[2 * u + 1]) + 4 * (kg & 1);
          const int bits = (kg < 2 ? here.mask[2 * u] : here.mask[2 * u + 1]) >> (4 * (kg & 1));
#pragma unroll
          for (int e = 0; e < 4; ++e)
#pragma unroll
            for (int rt = 0; rt < RT; ++rt)
              if (!((bits >> e) & 1) || pos0 + e < low[rt] || pos0 + e > lim[rt]) s[u][rt][e] = -INFINITY;
        }
      }
      // ---- running maximum and sum
      PagedFrag p[RT][(SUB + 1) / 2];
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
#pragma unroll
        for (int ct = 0; ct < CT; ++ct) o[rt][ct] *= fix;
        if constexpr (BF) {                                        // (the weights enter the product in the cache's own type)
          lr[rt] *= fix;
#pragma unroll
          for (int u = 0; u < SUB; ++u)
#pragma unroll
            for (int e = 0; e < 2; ++e)
              p[rt][0].u[2 * u + e] = __builtin_bit_cast(uint32_t, (bf16x2_t){(__bf16)x[u][2 * e], (__bf16)x[u][2 * e + 1]});
        } else {
#pragma unroll
          for (int e = 0; e < 4; ++e) p[rt][0].u[e] = __float_as_uint(x[0][e]);
        }
      }
      // ---- V through LDS; rows that nobody sees as zeros, whatever they hold
      bool odd = false;                                            // a value that is no number, or infinite, which some rows may not see
#pragma unroll
      for (int u = 0; u < GR; ++u)
#pragma unroll
        for (int j = 0; j < NF / 2; ++j) {
          u32x4 w = vf[u / 2][2 * j + u % 2].u;
          if (!all) {
            if (!((here.mask[u] >> r7) & 1)) w = (u32x4){0u, 0u, 0u, 0u};
            odd = odd || not_finite(w);
          }
          *(u32x4*)(vw + u * 8 * VROW + j * 128) = w;
        }
      if (i + 1 < n) load(Vb, lane_at, cur, vf);
      if constexpr (BF) {
        PagedFrag ones;
        ones.u = (u32x4){0x3f803f80u, 0x3f803f80u, 0x3f803f80u, 0x3f803f80u};
#pragma unroll
        for (int rt = 0; rt < RT; ++rt) lr[rt] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(ones.v, p[rt][0].v, lr[rt], 0, 0, 0);
      }
      if (!all && __ballot(odd)) {                                 // (0 times such a value is not 0: row by row, without what they do not see)
        add_seen(p, here, vlds);
        continue;
      }
      if constexpr (BF) {
#pragma unroll
        for (int ct = 0; ct < CT; ++ct) {
          PagedFrag a;
          const char* at = vlds + (kg * 4 + (r >> 2)) * VROW + ct * 32 + (r & 3) * 8;
          a.h[0] = lds_read_transposed(at);
          a.h[1] = lds_read_transposed(at + 16 * VROW);
#pragma unroll
          for (int rt = 0; rt < RT; ++rt) o[rt][ct] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(a.v, p[rt][0].v, o[rt][ct], 0, 0, 0);
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
template <typename T, int D, int RT, bool STREAM>
constexpr int attend_lds() { return pmax(pmax(WaveAttend<T, D, RT, STREAM>::LDS, 16 * RT * (D + 2) * 4) * (kPagedThreads / 64), join_lds(kPagedThreads, 16 * RT)); }

// Joins the wavefronts of the workgroup through LDS, [waves][rows][D + 2] (O, m, l); emit(row, channel, O of it and the next one, m, l).
template <typename T, int D, int RT, bool STREAM, typename Emit>
__device__ __forceinline__ void join_waves(WaveAttend<T, D, RT, STREAM>& w, char* lds, int rows, Emit&& emit) {
  constexpr int W = kPagedThreads / 64, R = 16 * RT, STR = D + 2;
  const int lane = threadIdx.x & 63, r = lane & 15, kg = lane >> 4, wave = threadIdx.x >> 6;
  float* mine = (float*)lds + (size_t)wave * R * STR;
  __syncthreads();                                                 // (every wavefront is done with its V rows)
#pragma unroll
  for (int rt = 0; rt < RT; ++rt) {
    const float l = across_32(across_16(w.l[rt], AddOp()), AddOp());
    float f = 1.f;
    if constexpr (sizeof(T) == 2) f = to_sum(l, w.lr[rt][0]);
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

// UNIFORM: 8 tokens always lie in one page
template <typename T, int D, int RT, bool PLAN, bool UNIFORM>
__global__ __launch_bounds__(kPagedThreads, attend_per_cu(D, RT)) void paged_attend_kernel(PagedGeom g) {
  // Non-temporal loads where the cache is read once for sure; with a plan several items of a sequence may read the same rows.  (128 sequences of one token have a
  // plan too: 420 us; 375 with non-temporal loads.)
  constexpr bool STREAM = !PLAN;
  using Wave = WaveAttend<T, D, RT, STREAM>;
  constexpr int WAVES = kPagedThreads / 64;
  __shared__ __align__(16) char lds[attend_lds<T, D, RT, STREAM>()];
  __shared__ int sh_last;
  const int lane = threadIdx.x & 63, r = lane & 15, kg = lane >> 4, wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));

  const int w = blockIdx.x;
  const auto sh = share_of<PLAN>(g, w);
  Wave at;
  int hint = -1;
  JoinRecord join;
  for (auto x = sh.begin; x < sh.end;) {
    const auto p = piece_at<PLAN>(g, sh, x, &hint);
    const PagedSeq s = p.s;
    const ItemRange it = p.it;
    const int h = p.h, seq = p.seq;
    const int t0 = it.begin + (p.u0 << g.unit_shift), t1 = min(it.begin + (p.u1 << g.unit_shift), it.end);
    bool bad = false;

    // ---- this piece: tokens [t0, t1)
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
      const bool live = rt * 16 + r < it.rows;
      int token, head;
      p.place(g, rt * 16 + r, &token, &head);
      const int i = token - s.row;
      at.lim[rt] = live ? s.cached + i : -1;
      at.low[rt] = live ? (g.window > 0 ? max(0, s.cached + i + 1 - g.window) : 0) : 1;
      const char* src = g.q + (int64_t)token * g.q_row + (int64_t)head * g.q_head;
#pragma unroll
      for (int f = 0; f < Wave::NF; ++f) {
        at.q[rt][f].u = (u32x4){0u, 0u, 0u, 0u};
        if (live) at.q[rt][f].u = gload128(src + f * 64 + kg * 16);
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
             typename Wave::Rows rows;
             const int tb = tile0(i);
             if constexpr (UNIFORM) {                              // lane u < GR looks up the page of group u
               const int t = tb + min(lane, Wave::GR - 1) * 8, pt = page_of(g, t);
               const int id = t + 7 >= it.low && t < t1 ? page_id(g, seq, pt, &bad) : -1;
#pragma unroll
               for (int u = 0; u < Wave::GR; ++u) {
                 const int tu = tb + u * 8, gid = __builtin_amdgcn_readlane(id, u), gp = __builtin_amdgcn_readlane(pt, u);
                 const int from = max(it.low - tu, 0), to = min(t1 - tu, 8);                    // tokens [from, to) of the group
                 rows.off[u] = (int64_t)max(gid, 0) * g.st_page + (int64_t)(tu - gp * g.by_page.d) * g.st_tok;
                 rows.pos[u] = tu;
                 rows.mask[u] = gid < 0 || from >= to ? 0 : ((1 << to) - 1) & ~((1 << from) - 1);
               }
             } else {
#pragma unroll
               for (int u = 0; u < Wave::GR; ++u) {
                 const int t = tb + u * 8 + (lane & 7), pt = page_of(g, t);
                 const int id = t >= it.low && t < t1 ? page_id(g, seq, pt, &bad) : -1;
                 rows.off[u] = (int64_t)max(id, 0) * g.st_page + (int64_t)(t - pt * g.by_page.d) * g.st_tok;
                 rows.pos[u] = tb + u * 8;
                 rows.mask[u] = (int)(__ballot(id >= 0) & 0xff);
               }
             }
             return rows;
           },
           [&](int i) { return tile0(i) >= low_all && tile0(i) + Wave::TOK - 1 <= seen_all; });

    // ---- out, or a partial
    const bool whole = p.whole();
    float* slot = partial_slot(g, w, x == sh.begin);
    join_waves<T, D, RT, STREAM>(at, lds, it.rows, [&](int row, int c, float2 o, float m, float l) {
      if (whole) {
        int token, head;
        p.place(g, row, &token, &head);
        store_out<T>(g, token, head, c, o, m, l);
      } else if constexpr (PLAN) {
        *(float2*)(slot + row * D + c) = o;
        if (c == 0) *(float2*)(slot + g.tile_rows * D + row * 2) = make_float2(m, l);
      } else {
        store_pair(slot + row * D + c, o.x, o.y);
        if (c == 0) store_pair(slot + g.tile_rows * D + row * 2, m, l);
      }
    });
    report_pages(g, bad);
    if constexpr (!PLAN) {
      if (!whole) finish_item<T, D, kPagedThreads>(g, sh, p, lds, &sh_last);
    }
    if constexpr (PLAN) join.note(g, sh, p, w, x == sh.begin);
    __syncthreads();
    x = min(sh.end, p.item1);
  }
  if constexpr (PLAN) join.store(g, w);
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

// ---- over blocks: `splits` workgroups per query token and KV head, each with an equal share of the listed blocks' tokens
template <typename T, int D>
__global__ __launch_bounds__(kPagedThreads) void block_attend_kernel(PagedGeom g) {
  using Wave = WaveAttend<T, D, 1, true>;
  constexpr int WAVES = kPagedThreads / 64;
  __shared__ __align__(16) char lds[attend_lds<T, D, 1, true>()];
  __shared__ int sh_last;
  const int lane = threadIdx.x & 63, r = lane & 15, kg = lane >> 4, wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x >> 6));
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
    if (r < g.G) at.q[0][f].u = gload128(src + f * 64 + kg * 16);
  }
  at.reset();
  const int per = g.by_page.d / g.block, shift = 31 - __builtin_clz(g.block);          // (a power of two of at least 16 tokens, in one page)
  const auto tile_slot = [&](int i) { return (a + wave + i * WAVES) * Wave::TOK; };
  at.run(g, h, lds + wave * Wave::LDS, (b - a - wave + WAVES - 1) / WAVES, Wave::lane_offset() + (uint32_t)(lane & 7) * (uint32_t)g.st_tok,
         [&](int i) {
           typename Wave::Rows rows;
           const int t0 = tile_slot(i), e = (t0 + min(lane, Wave::GR - 1) * 8) >> shift;
           const int2 blk = list[min(e, head.x - 1)];              // lane u < GR: the block of group u
           const int first = blk.y % per << shift;
#pragma unroll
           for (int u = 0; u < Wave::GR; ++u) {
             const int in = (t0 + u * 8) & (g.block - 1), id = __builtin_amdgcn_readlane(blk.x, u);
             const int pos = (__builtin_amdgcn_readlane(blk.y, u) << shift) + in, n = head.y + 1 - pos;         // tokens up to the query's own
             rows.off[u] = (int64_t)max(id, 0) * g.st_page + (int64_t)(__builtin_amdgcn_readlane(first, u) + in) * g.st_tok;
             rows.pos[u] = pos;
             rows.mask[u] = id < 0 || n <= 0 || t0 + u * 8 >= slots ? 0 : n >= 8 ? 0xff : (1 << n) - 1;
           }
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
  join_waves<T, D, 1, true>(at, lds, g.G, [&](int row, int c, float2 o, float m, float l) {
    if (whole) {
      store_out<T>(g, token, h * g.G + row, c, o, m, l);
    } else {
      store_pair(slot + row * D + c, o.x, o.y);
      if (c == 0) store_pair(slot + 16 * D + row * 2, m, l);
    }
  });
  if (!whole && last_to_arrive(g.arrived + at_list, pieces, &sh_last))
    join_pieces<T, D, kPagedThreads, true>(g, pieces, 0, g.G, 16, lds, [&](int p) { return part + (int64_t)p * 16 * (D + 2); },
                      [&](int row, int* t, int* hd) { *t = token; *hd = h * g.G + row; });
}

template <typename T, int D, int RT>
static void launch_split(const PagedGeom& g, hipStream_t s) {
  const bool uniform = g.by_page.d % 8 == 0 && g.st_tok < (1ll << 28);           // (offsets of 32 bits within 8 tokens)
  const auto kernel = g.plan_room ? uniform ? paged_attend_kernel<T, D, RT, true, true> : paged_attend_kernel<T, D, RT, true, false>
                                  : uniform ? paged_attend_kernel<T, D, RT, false, true> : paged_attend_kernel<T, D, RT, false, false>;
  hipLaunchKernelGGL(kernel, dim3(g.splits), dim3(kPagedThreads), 0, s, g);
}
template <typename T, int D>
static void launch_attend(const PagedGeom& g, hipStream_t s) {
  if (g.plan_room) hipLaunchKernelGGL(paged_plan_kernel, dim3(1), dim3(1024), 0, s, g);
  if (g.tile_rows > kPagedRows) launch_paged_chunk(g, s);
  else if (g.tile_rows <= 16) launch_split<T, D, 1>(g, s);
  else launch_split<T, D, 2>(g, s);
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
  const dim3 grid(g.splits, g.Hkv, g.row_group);
  if (g.dtype == TKPHI_BF16) {
    if (g.d == 64) hipLaunchKernelGGL((block_attend_kernel<uint16_t, 64>), grid, dim3(kPagedThreads), 0, s, g);
    else hipLaunchKernelGGL((block_attend_kernel<uint16_t, 128>), grid, dim3(kPagedThreads), 0, s, g);
  } else {
    if (g.d == 64) hipLaunchKernelGGL((block_attend_kernel<float, 64>), grid, dim3(kPagedThreads), 0, s, g);
    else hipLaunchKernelGGL((block_attend_kernel<float, 128>), grid, dim3(kPagedThreads), 0, s, g);
  }
}

}  // namespace tkphi
