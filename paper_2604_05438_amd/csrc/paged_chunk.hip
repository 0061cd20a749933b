// tkphi_paged_attention for many query rows per KV head (chunks, prompts), bf16.
//
// One pass over the keys and values with the running maximum and sum of the softmax.  A workgroup holds 256 query rows (d = 64: 128; new
// tokens times the query heads of one KV head, a wavefront 32 of them in registers) and passes over tiles of 128 (64) cached tokens, which go from memory
// straight to LDS a tile ahead, 64 of them at a time; S^T = K Q^T and O^T += V^T P^T on v_mfma_f32_32x32x16_bf16.  A lane holds all of S^T for one query row but the half
// its partner lane 32 further has, and exactly what it has to deliver of P^T: maximum and sum take one exchange, P none.
//
// 2048 tokens over 30000 cached ones (24 / 8 heads of 128) 0.84 to 0.96 ms, by the card: 810 to 930 TFLOP/s, two thirds to three quarters of what a large
// library product reaches; four prompts of 1762 to 3604 tokens (32 / 8 heads of 64) 0.33 to 0.36 ms.  The matrix cores are busy 39 % of the time (19 % at d = 64);
// without loads from memory the former takes 6 % less, without exponentials 7, without the reads of K from LDS 11, in another order of instructions the same:
// what is left are the dependencies of two wavefronts per SIMD (a wavefront alone with 64 rows and 512 registers: 1.65 ms).
#include "paged_attention.h"

namespace tkphi {

typedef __attribute__((__vector_size__(8 * sizeof(__bf16)))) __bf16 pc_bf16x8;
typedef __attribute__((__vector_size__(4 * sizeof(short)))) short pc_s16x4;
typedef __attribute__((__vector_size__(16 * sizeof(float)))) float pc_floatx16;
typedef unsigned int pc_u32x2 __attribute__((ext_vector_type(2)));
typedef __attribute__((address_space(3))) char* lds_ptr;
union ChunkFrag {
  u32x4 u;
  pc_bf16x8 v;
  pc_u32x2 h[2];
};

constexpr int kChunkTokens = 64;                                   // that a wavefront takes at a time
constexpr int kPageCache = 2048;                                   // entries of the page table in LDS
constexpr float kSlack = 8.f;             // the reference of the exponentials is raised when a score passes it by 2^8 (sums stay far from overflow)

// LDS of one tile: rows of D bf16 in 16-byte pieces, piece c of row r at place c ^ key_swap(r) or c ^ value_swap(r).  Keys are read as 16 bytes of 32
// rows, values as 64 bytes of 8 rows: either way the rows spread over the banks.
template <int D> __device__ __forceinline__ int key_swap(int r) { return r & (D / 8 - 1); }
template <int D> __device__ __forceinline__ int value_swap(int r) {
  return D == 128 ? (r & 3) << 2 | ((r >> 2) & 3) : ((r >> 1) & 1) << 2 | ((r >> 2) & 3);
}

template <int D>
struct ChunkTile {
  static constexpr int RB = D * 2, PIECES = RB / 16;
  static constexpr int TOKENS = D == 64 ? 64 : 128, HALVES = TOKENS / kChunkTokens;      // that go to LDS at a time
  static constexpr int BYTES = TOKENS * RB;
  static constexpr int BUFS = 2;                                   // tiles in LDS: one that is worked on, the others on their way
  static constexpr int ROWS = 1024 / RB;                           // rows that one load of a wavefront covers
  static constexpr int WAVES = chunk_rows(D) / 32, THREADS = 64 * WAVES;
  static constexpr int WAVE_TOKENS = TOKENS / WAVES, GROUPS = WAVE_TOKENS / 16;     // rows of a tile that a wavefront loads, 16 at a time
  static constexpr int LOADS = WAVE_TOKENS / ROWS, EACH = LOADS / GROUPS;                // loads per wavefront of K, and of V; and per 16 rows
};
static_assert(ChunkTile<128>::LOADS == 2 * ChunkTile<128>::HALVES && ChunkTile<64>::LOADS == 2 * ChunkTile<64>::HALVES, "");

// Adds the two weights of a register, as they were rounded.  (2048 tokens over 30000 / four prompts / a prompt of 16000 tokens of a 1B layer, us: 868 / 327 / 1542; without
// this sum 849 / 314 / 1461; unpacked and added 3 and 9 % more; as 4 x 4 products with ones on the matrix cores 876 / 327 / 1498, but 45.5 instead of 43.9 for 300
// tokens over 2000, by registers spilled; as one more channel, as in the split kernel, it would take 16 registers that are not there.)
__device__ __forceinline__ float add_rounded(uint32_t pair, float sum) {
  return __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2_t, pair), __builtin_bit_cast(bf16x2_t, 0x3f803f80u), sum, false);
}

// UNIFORM: 16 tokens always lie in one page
template <int D, bool UNIFORM>
__global__ __launch_bounds__(ChunkTile<D>::THREADS) __attribute__((amdgpu_waves_per_eu(chunk_per_simd(D), chunk_per_simd(D)))) void paged_chunk_kernel(PagedGeom g) {
  using Tile = ChunkTile<D>;
  constexpr int THREADS = Tile::THREADS, RB = Tile::RB, NF = D / 16, CT = D / 32, BUFS = Tile::BUFS;
  // tiles of K and V each
  __shared__ __align__(8192) char lds[BUFS * 2 * Tile::BYTES];
  __shared__ int sh_page[kPageCache];
  __shared__ __align__(8) uint16_t sh_present[BUFS][Tile::TOKENS / 16];      // which tokens of the tile anyone may see
  __shared__ int sh_odd[4];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int col = lane & 31, hi = lane >> 5, i16 = lane & 15, grp = (lane >> 4) & 1;
  const uint32_t lds0 = (uint32_t)(size_t)(lds_ptr)lds;
  if (tid < 4) sh_odd[tid] = 0;

  // Where this lane reads: keys of row col, channels 16 f + 8 hi .., at kbase ^ 32 f; values of row 4 hi + i16 / 4 (and + 8), transposed
  // by the read (lane i of 16 points at row i / 4, channels 4 (i % 4) .. and gets channel i of the four), channels 32 ct + 16 grp .., at
  // vbase ^ (64 ct + 32 x) and x times 8 rows on.  (The swaps are exclusive ors, so are the steps; registers are what this kernel is short of.)
  const int kbase = col * RB + (hi ^ key_swap<D>(col)) * 16;
  const int vrow = 4 * hi + (i16 >> 2), vbase = vrow * RB + ((2 * grp + ((i16 & 3) >> 1)) ^ value_swap<D>(vrow)) * 16 + (i16 & 1) * 8;
  // And what it loads: places lane % PIECES of rows WAVE_TOKENS wave + ROWS k + lane / PIECES of the tile
  const int lrow = lane / Tile::PIECES, lplace = lane % Tile::PIECES;
  const uint32_t kplace = (lplace ^ key_swap<D>(lrow)) * 16, vplace = (lplace ^ value_swap<D>(lrow)) * 16;        // of k = 0
  const uint32_t lrow_at = UNIFORM ? (uint32_t)(lrow * (int)g.st_tok) : 0u;
  const auto kat = [&](int k) { return lrow_at + (kplace ^ (D == 128 ? 64u * k : 0u)); };
  const auto vat = [&](int k) { return lrow_at + (vplace ^ (D == 128 ? 16u * k : 32u * (k & 1))); };
  const int64_t step = UNIFORM ? Tile::ROWS * g.st_tok : 0;        // from the rows of load k to those of k + 1

  const int w = share_number(blockIdx.x, gridDim.x);
  const Share<true> sh = share_of<true>(g, w);
  int hint = -1;
  JoinRecord join;
  for (int64_t x = sh.begin; x < sh.end;) {
    const Piece<true> p = piece_at<true>(g, sh, x, &hint);
    const PagedSeq s = p.s;
    const ItemRange it = p.it;
    const int t0 = it.begin + p.u0 * kChunkTokens, t1 = min(it.begin + p.u1 * kChunkTokens, it.end);

    // ---- query rows
    ChunkFrag q[NF];
    const int row = wave * 32 + col;
    const bool live = row < it.rows;
    int token, head;
    p.place(g, min(row, it.rows - 1), &token, &head);
    const int lim = s.cached + token - s.row, low = g.window > 0 ? max(0, lim + 1 - g.window) : 0;      // tokens [low, lim] are seen
    const char* qsrc = g.q + (int64_t)token * g.q_row + (int64_t)head * g.q_head;
#pragma unroll
    for (int f = 0; f < NF; ++f) q[f].u = gload128(qsrc + f * 32 + hi * 16);
    const int lim_lo = __builtin_amdgcn_readlane(lim, 0), lim_hi = __builtin_amdgcn_readlane(lim, 31);   // rows ascend by token
    const int low_lo = __builtin_amdgcn_readlane(low, 0), low_hi = __builtin_amdgcn_readlane(low, 31);
    const bool idle = wave * 32 >= it.rows;

    pc_floatx16 o[CT];
    float m = -INFINITY, l = 0.f, lr = 0.f;                         // maximum, sum of the weights, and of the weights as rounded
#pragma unroll
    for (int ct = 0; ct < CT; ++ct)
#pragma unroll
      for (int e = 0; e < 16; ++e) o[ct][e] = 0.f;

    const char* const Kh = g.K + p.h * g.st_head;
    const char* const Vh = g.V + p.h * g.st_head;
    const int seen_first = s.cached + g.by_group(p.tile * g.tile_rows);  // limit of the workgroup's first row
    const int low_last = g.window > 0 ? it.end - g.window : 0;     // first token that its last row sees

    // Stretches of the piece whose part of the page table fits LDS
    const int stretch = (int)min((int64_t)16384, (int64_t)(kPageCache - 2) * g.by_page.d / kChunkTokens * kChunkTokens);
    for (int ts = t0; ts < t1; ts += stretch) {
    const int te = min(ts + stretch, t1), n = (te - ts + Tile::TOKENS - 1) / Tile::TOKENS;
    const int page0 = page_of(g, ts), page_lo = page_of(g, max(ts, it.low)), page_hi = page_of(g, te - 1);
    __syncthreads();                                               // (the stretch, or the item, before is done with LDS)
    for (int e = page_lo + tid; e <= page_hi; e += THREADS) sh_page[e - page0] = page_id(g, p.seq, e);
    __syncthreads();

    // UNIFORM: where the tile that is being loaded comes from, and goes to; its loads are spread over the work on the tile before the last
    // (all at once right after the barrier they kept every wavefront from its products for 1900 of a tile's 11600 cycles)
    int64_t coming[Tile::GROUPS] = {};
    uint32_t coming_lds = 0;
    const auto request = [&](int i, bool at_once) {
      const int buf = i % BUFS, tw = ts + i * Tile::TOKENS + wave * Tile::WAVE_TOKENS;
      const uint32_t kdst = lds0 + buf * 2 * Tile::BYTES + wave * Tile::WAVE_TOKENS * RB, vdst = kdst + Tile::BYTES;
      if constexpr (UNIFORM) {
        uint32_t present = 0;
#pragma unroll
        for (int y = 0; y < Tile::GROUPS; ++y) {
          const int t = tw + 16 * y, pt = page_of(g, t), a = max(it.low - t, 0), z = min(te - t, 16);        // tokens [a, z) of the 16
          const int id = a < z ? __builtin_amdgcn_readfirstlane(sh_page[pt - page0]) : -1;
          if (id >= 0) present |= (((1u << z) - 1u) & ~((1u << a) - 1u)) << (16 * y);
          coming[y] = (int64_t)max(id, 0) * g.st_page + (int64_t)(t - pt * g.by_page.d) * g.st_tok;
        }
        coming_lds = kdst;
        if (at_once) {
#pragma unroll
          for (int k = 0; k < Tile::LOADS; ++k) {
            const int64_t at = coming[k / Tile::EACH] + k % Tile::EACH * step;
            load_to_lds16(Kh + at, kat(k), kdst + k * 1024);
            load_to_lds16(Vh + at, vat(k), vdst + k * 1024);
          }
        }
        if (lane < Tile::GROUPS) sh_present[buf][wave * Tile::GROUPS + lane] = (uint16_t)(present >> (16 * lane));
      } else {
        uint32_t present = 0;
#pragma unroll
        for (int k = 0; k < Tile::LOADS; ++k) {
          const int r = k * Tile::ROWS + lrow, t = tw + r, pt = page_of(g, t);
          const int id = t >= it.low && t < te ? sh_page[pt - page0] : -1;
          const int64_t at = (int64_t)max(id, 0) * g.st_page + (int64_t)(t - pt * g.by_page.d) * g.st_tok;
          load_to_lds16(Kh + at + kat(k), kdst + k * 1024);
          load_to_lds16(Vh + at + vat(k), vdst + k * 1024);
          const uint64_t there = __ballot(id >= 0);
#pragma unroll
          for (int y = 0; y < Tile::ROWS; ++y) present |= (uint32_t)((there >> (y * Tile::PIECES)) & 1) << (k * Tile::ROWS + y);
        }
        if (lane < Tile::GROUPS) sh_present[buf][wave * Tile::GROUPS + lane] = (uint16_t)(present >> (16 * lane));
      }
    };

    request(0, true);
    for (int i = 0; i < n; ++i) {
      // tile i is there, tile i - 1 is done with
      wait_vm_loads<0>();
      lds_barrier();
      if (tid < 2) sh_odd[2 * (1 - (i & 1)) + tid] = 0;
      const int buf = i % BUFS;
      const bool more = i + 1 < n;
      if (more) request(i + 1, false);
      // one load at each of four places per 64 tokens: first those of K, then those of V
      const auto spread = [&](int half, int y) {
        if constexpr (UNIFORM) {
          if (!more) return;
          const bool v = Tile::HALVES == 2 ? half == 1 : y >= Tile::LOADS;
          const int k = y % Tile::LOADS;
          load_to_lds16((v ? Vh : Kh) + coming[k / Tile::EACH] + k % Tile::EACH * step, v ? vat(k) : kat(k), coming_lds + (v ? Tile::BYTES : 0) + k * 1024);
        }
      };
#pragma unroll 1
      for (int half = 0; half < Tile::HALVES; ++half) {
      const int tb = ts + i * Tile::TOKENS + half * kChunkTokens;
      if (tb < te) {
      const bool skip = idle || tb > lim_hi || tb + kChunkTokens <= low_lo;        // (nothing here for this wavefront)
      const int half_at = buf * 2 * Tile::BYTES + half * kChunkTokens * RB;        // a multiple of 8 KB
      char* const vt = lds + half_at + Tile::BYTES;
      const uint64_t in_lds = *(const uint64_t*)(sh_present[buf] + half * 4);

      // ---- S^T: token 32 u + 8 a + 4 hi + b in element 4 a + b of sc[u]
      spread(half, 0);
      pc_floatx16 sc[2];
      if (!skip) {
#pragma unroll
      for (int e = 0; e < 16; ++e) sc[0][e] = sc[1][e] = 0.f;
#pragma unroll
      for (int f = 0; f < NF; ++f)
#pragma unroll
        for (int u = 0; u < 2; ++u) {
          ChunkFrag k;
          k.u = *(const u32x4*)(lds + (((half_at + kbase) ^ (32 * f)) + u * 32 * RB));
          sc[u] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(k.v, q[f].v, sc[u], 0, 0, 0);
        }
      // the LDS reads run four ahead of the products that take them
      __builtin_amdgcn_sched_group_barrier(0x100, 4, 0);
#pragma unroll
      for (int k = 0; k < 2 * NF; ++k) {
        __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
        if (k < 2 * NF - 4) __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
      }
      }
      spread(half, 1);
      const uint64_t present = (uint64_t)(uint32_t)__builtin_amdgcn_readfirstlane((int)(uint32_t)in_lds) |
                               (uint64_t)(uint32_t)__builtin_amdgcn_readfirstlane((int)(in_lds >> 32)) << 32;

      // ---- a tile that some row of the workgroup does not see all of: values that nobody sees become zeros, whatever they hold, and so do those
      // that are no numbers, or infinite, lest they meet the zero weights of rows that do not see them (add_odd puts them back)
      bool odd = false;
      if (present != ~0ull || tb + kChunkTokens - 1 > seen_first || tb < low_last) {
        bool mine = false;
        for (int k = tid; k < kChunkTokens * Tile::PIECES; k += THREADS) {
          const int r = k / Tile::PIECES;
          u32x4* at = (u32x4*)(vt + k * 16);
          if (!((present >> r) & 1)) {
            *at = (u32x4){0u, 0u, 0u, 0u};
          } else {
            u32x4 v = *at;
            bool bad = false;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              const bool a = (v[e] & 0x7f80u) == 0x7f80u, c = (v[e] & 0x7f800000u) == 0x7f800000u;
              if (a) v[e] &= 0xffff0000u;
              if (c) v[e] &= 0xffffu;
              bad = bad || a || c;
            }
            if (bad) *at = v;
            mine = mine || bad;
          }
        }
        if (mine) sh_odd[2 * (i & 1) + half] = 1;
        lds_barrier();
        odd = __builtin_amdgcn_readfirstlane(sh_odd[2 * (i & 1) + half]) != 0;
      }
      spread(half, 2);
      spread(half, 3);
      if (!skip) {

      if (present != ~0ull || tb + kChunkTokens - 1 > lim_lo || tb < low_hi) {
        // which of the 64 tokens the row sees, those 4 hi on at the bottom; a bit widened to a word picks the score or -inf
        const int last = lim - tb, first = max(low - tb, 0);
        uint64_t sees = last < 0 ? 0ull : last > 62 ? ~0ull : (2ull << last) - 1ull;
        sees &= first > 63 ? 0ull : ~0ull << first;
        sees = (sees & present) >> (4 * hi);
#pragma unroll
        for (int u = 0; u < 2; ++u)
#pragma unroll
          for (int e = 0; e < 16; ++e) {
            const int pick = __builtin_amdgcn_sbfe((int)(uint32_t)(sees >> (32 * u)), 8 * (e / 4) + e % 4, 1);
            sc[u][e] = __uint_as_float((__float_as_uint(sc[u][e]) & (uint32_t)pick) | (0xff800000u & ~(uint32_t)pick));
          }
      }
      // ---- running maximum and sum
      float mx = sc[0][0];
#pragma unroll
      for (int e = 1; e < 32; ++e) mx = fmaxf(mx, sc[e / 16][e % 16]);
      mx = across_32(mx, MaxOp()) * g.scale2;
      if (__any(mx > m + kSlack || (m == -INFINITY && mx > -INFINITY))) {
        const float mn = fmaxf(m, mx), fix = mn == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(m - mn);
        m = mn;
        l *= fix;
        lr *= fix;
#pragma unroll
        for (int ct = 0; ct < CT; ++ct)
#pragma unroll
          for (int e = 0; e < 16; ++e) o[ct][e] *= fix;
      }
      const float ref = m == -INFINITY ? 0.f : m;
      // ---- P^T of 16 tokens at a time, in the cache's own type, and O^T: the inner indices of step k are the tokens
      // 16 k + 4 hi + {0 .. 3} and 16 k + 8 + 4 hi + {0 .. 3}
      ChunkFrag pr[4];
      float sum[4];
      const auto weigh = [&](int k) {
        float e[8];
#pragma unroll
        for (int y = 0; y < 8; ++y) e[y] = __builtin_amdgcn_exp2f(fmaf(sc[k / 2][8 * (k & 1) + y], g.scale2, -ref));
#pragma unroll
        for (int y = 0; y < 4; ++y) pr[k].u[y] = __builtin_bit_cast(uint32_t, (bf16x2_t){(__bf16)e[2 * y], (__bf16)e[2 * y + 1]});
#pragma unroll
        for (int y = 0; y < 4; ++y) lr = add_rounded(pr[k].u[y], lr);
        sum[k] = ((e[0] + e[1]) + (e[2] + e[3])) + ((e[4] + e[5]) + (e[6] + e[7]));
      };
      __builtin_amdgcn_s_setprio(1);                               // (the wavefront next door, between its products, yields: 1 to 3 %)
      weigh(0);
#pragma unroll
      for (int k = 0; k < 4; ++k) {
#pragma unroll
        for (int ct = 0; ct < CT; ++ct) {
          ChunkFrag v;
#pragma unroll
          for (int y = 0; y < 2; ++y)
            v.h[y] = __builtin_bit_cast(pc_u32x2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) pc_s16x4*)(lds + (((half_at + vbase) ^ (64 * ct + 32 * y)) + Tile::BYTES + (8 * y + 16 * k) * RB))));
          o[ct] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(v.v, pr[k].v, o[ct], 0, 0, 0);
        }
        if (k < 3) weigh(k + 1);
      }
      __builtin_amdgcn_s_setprio(0);
      l += (sum[0] + sum[1]) + (sum[2] + sum[3]);
      // the next step's weights between this one's products
      __builtin_amdgcn_sched_group_barrier(0x100, 4, 0);
      __builtin_amdgcn_sched_group_barrier(0x002, 20, 0);
#pragma unroll
      for (int k = 0; k < 4 * CT; ++k) {
        __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
        if (k < 4 * CT - 2) __builtin_amdgcn_sched_group_barrier(0x100, 2, 0);
        if (k < 3 * CT) __builtin_amdgcn_sched_group_barrier(0x002, 28 / CT, 0);
      }
      if (odd) {                                                   // token by token: what was taken out of the values, for the rows that see it
#pragma unroll 1
        for (int slot = 0; slot < kChunkTokens; ++slot) {
          const int t = tb + slot;
          uint32_t word = 0;
#pragma unroll
          for (int k = 0; k < 16; ++k)
            if (k == (slot >> 5) * 8 + ((slot >> 3) & 3) * 2 + ((slot >> 1) & 1)) word = pr[k / 4].u[k % 4];
          word = (uint32_t)__shfl((int)word, (slot >> 2 & 1) * 32 + col);
          const float weight = __uint_as_float(slot & 1 ? word & 0xffff0000u : word << 16);
          if (!((present >> slot) & 1)) continue;
          const int pt = page_of(g, t), id = max(page_id(g, p.seq, pt), 0);
          const uint16_t* v = (const uint16_t*)(g.V + (int64_t)id * g.st_page + p.h * g.st_head + (int64_t)(t - pt * g.by_page.d) * g.st_tok);
          const bool sees = t <= lim && t >= low;
#pragma unroll
          for (int ct = 0; ct < CT; ++ct)
#pragma unroll
            for (int e = 0; e < 16; ++e) {
              const uint16_t bits = v[32 * ct + 8 * (e / 4) + 4 * hi + e % 4];
              if (sees && (bits & 0x7f80) == 0x7f80) o[ct][e] = fmaf(weight, bf16_bits_to_float(bits), o[ct][e]);
            }
        }
      }
      }
      }
      }
    }
    }
    // ---- out, or a partial
    l = across_32(l, AddOp());
    lr = across_32(lr, AddOp());
    const bool whole = p.whole();
    if (live) {
      if (whole) {
        const float inv = l == 0.f ? 0.f : 1.f / lr;
        char* dst = g.out + (int64_t)token * g.out_row + (int64_t)head * g.out_head;
#pragma unroll
        for (int ct = 0; ct < CT; ++ct)
#pragma unroll
          for (int a = 0; a < 4; ++a) {
            float y[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) y[e] = l == 0.f ? 0.f : o[ct][4 * a + e] * inv;
            pc_u32x2 v;
            v[0] = __builtin_bit_cast(uint32_t, (bf16x2_t){(__bf16)y[0], (__bf16)y[1]});
            v[1] = __builtin_bit_cast(uint32_t, (bf16x2_t){(__bf16)y[2], (__bf16)y[3]});
            *(__attribute__((address_space(1))) pc_u32x2*)(dst + (32 * ct + 8 * a + 4 * hi) * 2) = v;
          }
        if (hi == 0 && g.lse) g.lse[(int64_t)token * g.Hq + head] = l == 0.f ? -INFINITY : (m + __builtin_amdgcn_logf(l)) * kLn2;
      } else {
        float* slot = partial_slot(g, w, x == sh.begin);
        const float f = to_sum(l, lr);
#pragma unroll
        for (int ct = 0; ct < CT; ++ct)
#pragma unroll
          for (int a = 0; a < 4; ++a)
            *(__attribute__((address_space(1))) u32x4*)(slot + row * D + 32 * ct + 8 * a + 4 * hi) =
                (u32x4){__float_as_uint(o[ct][4 * a] * f), __float_as_uint(o[ct][4 * a + 1] * f), __float_as_uint(o[ct][4 * a + 2] * f), __float_as_uint(o[ct][4 * a + 3] * f)};
        if (hi == 0) *(float2*)(slot + g.tile_rows * D + row * 2) = make_float2(m, l);
      }
    }
    join.note(g, sh, p, w, x == sh.begin);
    x = min(sh.end, p.item1);
  }
  join.store(g, w);
}

void launch_paged_chunk(const PagedGeom& g, hipStream_t s) {
  const bool uniform = g.by_page.d % 16 == 0 && g.st_tok < (1ll << 27);       // (offsets of 32 bits within 8 tokens)
  if (g.d == 64) hipLaunchKernelGGL((uniform ? paged_chunk_kernel<64, true> : paged_chunk_kernel<64, false>), dim3(g.splits), dim3(ChunkTile<64>::THREADS), 0, s, g);
  else hipLaunchKernelGGL((uniform ? paged_chunk_kernel<128, true> : paged_chunk_kernel<128, false>), dim3(g.splits), dim3(ChunkTile<128>::THREADS), 0, s, g);
}

}  // namespace tkphi
