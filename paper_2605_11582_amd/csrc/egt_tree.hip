// Attention of drafted trees over a paged cache.
//
// Of one request and one key head, all query rows - its drafted tokens times the query heads that share the key head - meet
// the same keys: the cache is read once for all of them.  A workgroup has W waves, WR of them side by side over the rows
// (16 NR rows each) and W / WR groups of them over the keys; a group takes 32 keys at a time, and the grid cuts the keys into spans
// where requests and heads alone do not fill the chip (a second kernel joins them).  A step of a group:
//
//   stage          K and V of 32 keys through registers into LDS, each wave its share, in whole lines of the cache; the tiles
//                  behind them are on their way.  Groups of several waves have two buffers and meet in one barrier a step.
//   S^T = K Q^T    a lane: one key, 8 values of d; Q^T is held in registers.  Lane (g, n) gets scores of row n and keys
//                  4 g .. 4 g + 3 of either half of the 32.
//   p = exp2       against a reference per row that is raised only where a score passes it by 2^5: sums and O are rescaled
//                  rarely, and the maximum is joined over lanes only then.
//   O^T += V^T P^T the scores' layout is the B operand's if the 32 keys are counted 4 g + i, 16 + 4 g + i, so p goes on in its lane;
//                  V^T comes out of LDS by the transposing read; the sum of p is one more product, with ones.
//
// What bounds it: with up to 64 rows a key head the cache's bytes (16 rows over 131072 keys, 8 heads of 128: 107 us, 5.0 TB/s;
// 64 rows 116 us), above that the steps themselves, of which one wave a SIMD can hide little: 256 rows 187 us (184 to 193 from card to
// card, the join's 10 among them), 2.9 TB/s and 0.74 PFLOP/s, matrix units busy 40 % of the first kernel's time and vector units 45 %; its
// kernel keeps 68 bytes a lane in scratch.  A wave of two row tiles spends, of 2500 cycles a step,
// 345 on staging, 500 on addresses and requests, 610 on scores (256 of them products), 390 on weights and 555 on sums (288).  Short
// contexts are bound by a launch and the chain lengths - page numbers - keys, 8 to 10 us, and a launch more where there are several spans.
#include "egt_mfma_common.h"
#include "egt_serve.h"

#include <algorithm>

namespace egt {
namespace {

constexpr int TILE = 32;             // keys a wave takes at a time
// p is held as 2^SHIFT p against its reference, and may pass it by 2^SLACK: 2^15 at most in FP16, and whole
// precision down to 2^-24 of the largest weight.
constexpr float SHIFT = 10.f, SLACK = 5.f, EXP2_LIMIT = 32768.f;
// From here on the sum of an exponent and SHIFT is too coarse for one multiply-add against the reference (its steps pass what FP16 holds,
// from 2^24 on, and then SHIFT itself): the difference of the scores is taken first.
constexpr float FAR_SCORE = 0x1p20f;

struct TreeArgs {
  egt_tree_batch b;
  egt_kv_cache c;
  float *part;                       // [splits][tokens * heads][dim]: weighted sums of a span
  float2 *ml;                        // [splits][tokens * heads]: its reference and sum
  int32_t shift, group, splits, row_blocks, min_tiles, whole;
  float scale2;                      // |scale| log2(e)
  uint32_t flip;                     // sign of the scale, on pairs of q
};

typedef __attribute__((address_space(1))) u4 global_u4;
typedef short s4v __attribute__((ext_vector_type(4)));
typedef __attribute__((address_space(3))) s4v lds_s4v;

// All ones in the halves of a pair that are infinite or NaN.
__device__ __forceinline__ uint32_t odd_halves(uint32_t x) {
  const uint32_t lo = (x & 0x7c00u) == 0x7c00u ? 0xffffu : 0u, hi = (x & 0x7c000000u) == 0x7c000000u ? 0xffff0000u : 0u;
  return lo | hi;
}

// Units of 32 bytes of a key trade places by the key's number, so that the 16 keys of an operand read lie on different banks.
// (Rows of an odd number of 64 bytes do so by themselves.)
template <int DC>
constexpr int SWIZZLE = DC == 4 || DC == 8 ? 7 : DC == 2 || DC == 6 ? 3 : 0;

// How a request's keys are cut: the same answer in both kernels.
struct Spans { int ctx_tiles, tiles, per, count; };
__device__ __forceinline__ Spans spans_of(int len, int n, int splits, int min_tiles, int whole) {
  Spans s;
  s.ctx_tiles = (len + TILE - 1) / TILE;
  s.tiles = s.ctx_tiles + (n + TILE - 1) / TILE;
  s.per = s.tiles <= whole ? s.tiles : max((s.tiles + splits - 1) / splits, min_tiles);
  s.count = (s.tiles + s.per - 1) / s.per;
  return s;
}
enum { ROWS_NONE, ROWS_BAD, ROWS_FINE };
__device__ __forceinline__ int request_state(const TreeArgs &a, int t0, int t1, int len) {
  if (t0 < 0 || t1 <= t0 || t1 > a.b.tokens) return ROWS_NONE;
  return t1 - t0 > a.b.max_tokens || len < 0 || len > (int64_t)a.b.table_blocks << a.shift || (len > 0 && a.c.blocks == 0) ? ROWS_BAD : ROWS_FINE;
}

// Waves of a workgroup, and how many tiles ahead of their use a wave requests its share of them.  Eight waves where few rows leave most
// of them to the keys (us, eight against four: one token over 8000 keys of 8 heads 21.5 / 34.7, 32 requests over up to 2000 31.9 / 35.5),
// four where barriers tie them together; wide heads have no LDS for eight groups.
constexpr int waves_of(int dc, int wr) { return (dc <= 4 && wr <= 2) || wr > 4 ? 8 : 4; }
constexpr int ahead_of(int wr) { return wr >= 8 ? 3 : wr >= 4 ? 2 : 1; }

template <int DC, int NR, int WR>
__global__ __launch_bounds__(64 * waves_of(DC, WR), DC > 4 && WR < 8 ? 1 : 2) void k_tree(TreeArgs a) {
  // a key in LDS: ROW bytes, PIECES pieces of 16; a tile of K and one of V: KV bytes each; a wave stages LJ x 64 pieces of either
  constexpr int W = waves_of(DC, WR), WK = W / WR, ROW = 64 * DC, PIECES = 4 * DC, LJ = (2 * DC + WR - 1) / WR, BUFS = WR > 1 ? 2 : 1, KV = TILE * ROW;
  constexpr int AHEAD = ahead_of(WR);
  extern __shared__ __align__(16) uint8_t lds[];
  __shared__ int odd_seen[W];
  __shared__ uint64_t masks[EGT_MAX_TREE];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), n16 = lane & 15, g4 = lane >> 4;
  const int wr = wave % WR, wk = wave / WR, dim = a.c.dim;
  const int r = blockIdx.z, kh = blockIdx.y / a.row_blocks, rb = blockIdx.y % a.row_blocks;
  const int t0 = a.b.cu_tokens[r], t1 = a.b.cu_tokens[r + 1], len = a.b.lens[r];
  // The arguments are five lines of memory: asked for together, not one behind the other as they come up (us, so against left to
  // the compiler: seven requests of up to 31 tokens and 3000 keys, heads of 80, 22.8 / 24.1; one token over 777 keys, heads of 64, 128 and 192,
  // 10.4 / 10.5, 14.2 / 14.4 and 17.0 / 17.3; 256 rows over 32768 keys, heads of 96, 59.0 / 60.5; 80 rows of them, eight requests, 37.4 / 36.2).
  // Not where registers are short (heads of 128: 256 rows over 131072 keys 204 / 196, 80 rows, sixteen requests, 52.4 / 51.5; heads
  // of 200 to 256, one wave a SIMD: no difference).
  if constexpr (NR * DC < 8)
    asm volatile("" ::"s"(a.b.q), "s"(a.b.k_row), "s"(a.b.mask), "s"(a.b.requests), "s"(a.c.k), "s"(a.c.k_head), "s"(a.part), "s"(a.scale2));
  const int state = request_state(a, t0, t1, len);
  if (state == ROWS_NONE) return;
  const int n = t1 - t0;
  if (state == ROWS_BAD) {                            // (any number of tokens)
    if (blockIdx.x == 0 && rb == 0)
      for (int64_t e = threadIdx.x; e < (int64_t)n * a.group * dim; e += 64 * W) {
        const int64_t row = e / dim, tok = row / a.group;
        a.b.out[(t0 + tok) * a.b.out_row + (kh * a.group + row - tok * a.group) * a.b.out_head + e - row * dim] = 0x7e00;
      }
    return;
  }
  const int rows = n * a.group;
  const Spans sp = spans_of(len, n, a.splits, a.min_tiles, a.whole);
  const int row0 = rb * (16 * NR * WR);
  if ((int)blockIdx.x >= sp.count || row0 >= rows) return;
  const int base = row0 + wr * 16 * NR, begin = blockIdx.x * sp.per, end = min(begin + sp.per, sp.tiles);
  const bool busy = base < rows;                      // (a wave without rows still stages its share)
  // This wave's tiles are begin + wk + i WK, i < mine; all waves go `steps` steps, for they meet in barriers.  Steps and requests
  // past the last tile take that one again, with every key masked.
  const int steps = (end - begin + WK - 1) / WK, mine = (end - begin - wk + WK - 1) / WK;
  auto tile_of = [&](int i) { return min(begin + wk + i * WK, end - 1); };
  auto limit_of = [&](int i) {                        // keys that there are
    const int t = tile_of(i);
    return i >= mine ? 0 : t >= sp.ctx_tiles ? n - (t - sp.ctx_tiles) * TILE : len - t * TILE;
  };

  auto there = [&](int x) { return 2 * DC % WR == 0 || x * WR + wr < 2 * DC; };
  auto key_of = [&](int x) { return (64 * (x * WR + wr) + lane) / PIECES; };
  auto piece_of = [&](int x) { return (64 * (x * WR + wr) + lane) % PIECES; };
  auto turn = [](int key) { return SWIZZLE<DC> == 7 ? key & 7 : SWIZZLE<DC> == 3 ? (key >> 1) & 3 : 0; };

  // What a lane requests of a tile: piece `piece_of(x)` of key `key_of(x)`, LJ times.  Cached and drafted keys differ in numbers alone:
  // a drafted one is place i of a page 0 that begins at the request's first row.
  const int32_t *table = len > 0 ? a.b.block_table + (int64_t)r * a.b.ld_table : a.b.lens;
  const int pmask = (1 << a.shift) - 1;
  struct Pages { int at[LJ]; };
  auto pages_of = [&](int i) {
    const int t = tile_of(i);
    Pages p;
#pragma unroll
    for (int x = 0; x < LJ; ++x) p.at[x] = table[max(min(t * TILE + key_of(x), len - 1), 0) >> a.shift];
    return p;                                         // (not looked at here: a look would wait for it)
  };
  uint32_t worst = 0;                                 // the largest page number met
  struct Share { u4 at[LJ]; };
  auto request = [&](int i, const Pages &page, const uint16_t *cached, int64_t block_step, int64_t token_step, const uint16_t *drafts, int64_t row_step) {
    const int t = tile_of(i);
    const bool drafted = t >= sp.ctx_tiles;
    const uint16_t *from = drafted ? drafts : cached;
    const uint32_t ts = 2 * (uint32_t)(drafted ? row_step : token_step), bs = 2 * (uint32_t)block_step;
    const int first = (drafted ? t - sp.ctx_tiles : t) * TILE, within = drafted ? -1 : pmask, most = drafted ? n - 1 : INT32_MAX;
    Share s;
#pragma unroll
    for (int x = 0; x < LJ; ++x) {
      if (!there(x)) break;
      const uint32_t number = drafted ? 0u : (uint32_t)page.at[x];
      worst = max(worst, number);                     // (one that is not the cache's: NaN in the end, and the last one meanwhile)
      const uint32_t block = min(number, (uint32_t)max(a.c.blocks - 1, 0)), place = min((first + key_of(x)) & within, most);
      const int d = 8 * piece_of(x) < dim ? 8 * piece_of(x) : 0;
      s.at[x] = *(const global_u4 *)((uint64_t)block * bs + ((uint64_t)place * ts + (uint64_t)(from + d)));
    }
    return s;
  };
  auto request_k = [&](int i, const Pages &p) {
    return request(i, p, a.c.k + kh * a.c.k_head, a.c.k_block, a.c.k_token, a.b.k + t0 * a.b.k_row + kh * a.b.k_head, a.b.k_row);
  };
  auto request_v = [&](int i, const Pages &p) {
    return request(i, p, a.c.v + kh * a.c.v_head, a.c.v_block, a.c.v_token, a.b.v + t0 * a.b.v_row + kh * a.b.v_head, a.b.v_row);
  };

  // ... and where it goes in LDS
  uint8_t *group = lds + wk * (BUFS * 2 * KV);
  auto k_area = [&](int i) { return group + (BUFS > 1 ? (i & 1) * KV : 0); };
  auto v_area = [&](int i) { return group + BUFS * KV + (BUFS > 1 ? (i & 1) * KV : 0); };
  auto put = [&](const Share &s, uint8_t *to) {
#pragma unroll
    for (int x = 0; x < LJ; ++x) {
      if (!there(x)) break;
      const int key = key_of(x), pc = piece_of(x);
      *(u4 *)(to + key * ROW + 32 * ((pc >> 1) ^ turn(key)) + 16 * (pc & 1)) = s.at[x];
    }
  };
  auto stage_k = [&](int i, Share s) {                // columns past dim are zeros
    if (dim != 32 * DC)
#pragma unroll
      for (int x = 0; x < LJ; ++x)
        if (8 * piece_of(x) >= dim) s.at[x] = u4{0, 0, 0, 0};
    put(s, k_area(i));
  };
  // values of keys that there are not become zeros, and so, for now, does what is not finite in drafted tokens: rows
  // that do not see it must not meet it (0 times infinity)
  auto stage_v = [&](int i, Share s) {
    const bool drafted = tile_of(i) >= sp.ctx_tiles;
    const int limit = limit_of(i);
    if (drafted || limit < TILE) {
      bool odd = false;
#pragma unroll
      for (int x = 0; x < LJ; ++x) {
        if (!there(x)) break;
        if (key_of(x) >= limit) s.at[x] = u4{0, 0, 0, 0};
        if (drafted) {
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const uint32_t m = odd_halves(s.at[x][e]);
            odd |= m != 0;
            s.at[x][e] &= ~m;
          }
        }
      }
      if (odd) odd_seen[wk] = 1;
    }
    put(s, v_area(i));
  };

  // AHEAD tiles are on their way, and the page numbers of AHEAD more.  Which registers they come into is fixed (the loop goes AHEAD
  // tiles a round): a copy of a register that is still being loaded would wait for it.
  Share kring[AHEAD], vring[AHEAD];
  Pages pages[AHEAD];
#pragma unroll
  for (int j = 0; j < AHEAD; ++j) pages[j] = pages_of(j);
  // Q^T as the B operand: lane (g, n) holds d = 32 c + 8 g .. + 7 of row n (a row past the last: the last one again, which nobody
  // stores).  Requested behind the first page numbers, without a branch and looked at last: with a wait each sixteen
  // requests of up to 80 rows took 52 us and take 51.
  u4 q[NR][DC];
#pragma unroll
  for (int x = 0; x < NR; ++x) {
    const int row = min(base + 16 * x + n16, rows - 1), tok = row / a.group;
    const uint16_t *qp = a.b.q + (int64_t)(t0 + tok) * a.b.q_row + (int64_t)(kh * a.group + row - tok * a.group) * a.b.q_head;
#pragma unroll
    for (int c = 0; c < DC; ++c) q[x][c] = *(const u4 *)(qp + (32 * c + 8 * g4 < dim ? 32 * c + 8 * g4 : 0));
  }
  const uint64_t mask = a.b.mask[t0 + min((int)threadIdx.x, n - 1)];
#pragma unroll
  for (int j = 0; j < AHEAD; ++j) {
    kring[j] = request_k(j, pages[j]);
    vring[j] = request_v(j, pages[j]);
    pages[j] = pages_of(j + AHEAD);
  }
  if (threadIdx.x < W) odd_seen[threadIdx.x] = 0;
  if (threadIdx.x < EGT_MAX_TREE) masks[threadIdx.x] = mask;
#pragma unroll
  for (int x = 0; x < NR; ++x)
#pragma unroll
    for (int c = 0; c < DC; ++c)
#pragma unroll
      for (int e = 0; e < 4; ++e) q[x][c][e] = 32 * c + 8 * g4 < dim ? q[x][c][e] ^ a.flip : 0;
  f4 o[NR][2 * DC], l[NR];                            // weighted sums; sums
  float ref[NR], off[NR];                             // reference (a score); SHIFT - the reference as an exponent of 2, or infinite
  const _Float16 one = 1;
  const h8 ones = {one, one, one, one, one, one, one, one};
#pragma unroll
  for (int x = 0; x < NR; ++x) {
    ref[x] = -INFINITY;
    off[x] = INFINITY;
    l[x] = f4{0, 0, 0, 0};
#pragma unroll
    for (int d = 0; d < 2 * DC; ++d) o[x][d] = f4{0, 0, 0, 0};
  }

  lds_barrier();                                      // (odd_seen, masks)

  auto compute = [&](int i) {
      const int t = tile_of(i), limit = limit_of(i);
      const bool drafted = t >= sp.ctx_tiles;
      // Reads ahead of the products that use them, and kept there: left alone, the compiler waits for them two by two (a step of
      // two row tiles: scores 650 cycles and weighted sums 940, of 256 and 288 that the products take).
      f4 s[NR][2];
      u4 k[2][DC];
#pragma unroll
      for (int c = 0; c < DC; ++c)
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const int key = 16 * h + n16;
          k[h][c] = *(const u4 *)(k_area(i) + key * ROW + 32 * ((2 * c + (g4 >> 1)) ^ turn(key)) + 16 * (g4 & 1));
        }
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int x = 0; x < NR; ++x) s[x][0] = s[x][1] = f4{0, 0, 0, 0};
#pragma unroll
      for (int c = 0; c < DC; ++c)
#pragma unroll
        for (int x = 0; x < NR; ++x)
#pragma unroll
          for (int h = 0; h < 2; ++h) s[x][h] = __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(h8, k[h][c]), __builtin_bit_cast(h8, q[x][c]), s[x][h], 0, 0, 0);
      // V^T as the A operand: lane j of a group of 16 addresses 8 bytes of key 4 g + j / 4, and gets d = 16 dt + n of keys 4 g .. 4 g + 3
      constexpr int FAR = 4;
      u4 v[FAR];
      auto read_v = [&](int d) {
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const int key = 16 * h + 4 * g4 + (n16 >> 2);
          const u2 both = __builtin_bit_cast(u2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s4v *)(v_area(i) + key * ROW + 32 * (d ^ turn(key)) + 8 * (n16 & 3))));
          v[d % FAR][2 * h] = both.x;
          v[d % FAR][2 * h + 1] = both.y;
        }
      };
#pragma unroll
      for (int d = 0; d < FAR; ++d) read_v(d);
      __builtin_amdgcn_sched_barrier(0);
      if (drafted || limit < TILE) {
#pragma unroll
        for (int x = 0; x < NR; ++x) {
          const int row = base + 16 * x + n16;
          const uint32_t word = !drafted ? ~0u : row < rows ? (uint32_t)(masks[row / a.group] >> ((t - sp.ctx_tiles) * TILE)) : 0u;
#pragma unroll
          for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              const int key = 16 * h + 4 * g4 + e;
              if (key >= limit || !(word >> key & 1)) s[x][h][e] = -INFINITY;
            }
        }
      }
      // Scores that pass the reference too far show in p itself, whose bits order as whole numbers do (no reference yet, or one whose
      // exponent is FAR_SCORE or more: off is infinite, and so is p, or NaN).
      float e[NR][8];
      uint32_t most = 0;
#pragma unroll
      for (int x = 0; x < NR; ++x)
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          e[x][j] = __builtin_amdgcn_exp2f(fmaf(s[x][j >> 2][j & 3], a.scale2, off[x]));
          most = max(most, __builtin_bit_cast(uint32_t, e[x][j]));
        }
      if (__any(most > __builtin_bit_cast(uint32_t, EXP2_LIMIT))) {
#pragma unroll
        for (int x = 0; x < NR; ++x) {
          float top = fmaxf(fmaxf(fmaxf(s[x][0][0], s[x][0][1]), fmaxf(s[x][0][2], s[x][0][3])), fmaxf(fmaxf(s[x][1][0], s[x][1][1]), fmaxf(s[x][1][2], s[x][1][3])));
          top = fmaxf(top, __shfl_xor(top, 16, 64));
          top = fmaxf(top, __shfl_xor(top, 32, 64));
          const float to = (top - ref[x]) * a.scale2 > SLACK ? top : ref[x], was2 = ref[x] * a.scale2, to2 = to * a.scale2;
          const bool none = to2 == -INFINITY, far = !none && fabsf(to2) >= FAR_SCORE;
          // (nothing is there yet: 1)
          const float f = was2 == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(far ? (ref[x] - to) * a.scale2 : was2 - to2);
          ref[x] = to;
          off[x] = none || far ? INFINITY : SHIFT - to2;
          const float from = far ? to : 0.f, now = none || far ? SHIFT : off[x];
#pragma unroll
          for (int j = 0; j < 4; ++j) l[x][j] *= f;
#pragma unroll
          for (int d = 0; d < 2 * DC; ++d)
#pragma unroll
            for (int j = 0; j < 4; ++j) o[x][d][j] *= f;
#pragma unroll
          for (int j = 0; j < 8; ++j) e[x][j] = __builtin_amdgcn_exp2f(fmaf(s[x][j >> 2][j & 3] - from, a.scale2, now));
        }
      }
      h8 p[NR];
#pragma unroll
      for (int x = 0; x < NR; ++x)
#pragma unroll
        for (int j = 0; j < 8; ++j) p[x][j] = (_Float16)e[x][j];
#pragma unroll
      for (int x = 0; x < NR; ++x) l[x] = __builtin_amdgcn_mfma_f32_16x16x32_f16(ones, p[x], l[x], 0, 0, 0);      // (every entry of a row: its sum)
#pragma unroll
      for (int d = 0; d < 2 * DC; ++d) {
        const u4 now = v[d % FAR];
        if (d + FAR < 2 * DC) read_v(d + FAR);
#pragma unroll
        for (int x = 0; x < NR; ++x) o[x][d] = __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(h8, now), p[x], o[x][d], 0, 0, 0);
        __builtin_amdgcn_sched_barrier(0);
      }
  };
#pragma unroll 1
  for (int i = 0; i < steps; i += AHEAD)
#pragma unroll
    for (int j = 0; j < AHEAD; ++j) {
      if (i + j >= steps) break;
      stage_k(i + j, kring[j]);
      stage_v(i + j, vring[j]);
      kring[j] = request_k(i + j + AHEAD, pages[j]);
      vring[j] = request_v(i + j + AHEAD, pages[j]);
      pages[j] = pages_of(i + j + 2 * AHEAD);
      if (WR > 1) lds_barrier();                      // (two buffers: who writes the other one has passed this barrier, and so has every reader)
      if (busy) compute(i + j);
    }

  // the waves over the keys join: references and sums, then the weighted sums a row tile at a time through the V areas
  __shared__ float refs[W][16 * NR], sums[W][16 * NR];
#pragma unroll
  for (int x = 0; x < NR; ++x) {
    if (g4 == 0) {
      refs[wave][16 * x + n16] = ref[x] * a.scale2;   // (base 2)
      sums[wave][16 * x + n16] = l[x][0];
    }
  }
  const bool bad = __syncthreads_or(a.c.blocks > 0 && worst >= (uint32_t)a.c.blocks);
  if (odd_seen[wk] && base < rows) {                  // (rare) what is not finite in drafted tokens, to the rows that see it
    const int first = max(begin, sp.ctx_tiles);
    for (int key = 0; key < min((end - sp.ctx_tiles) * TILE, n); ++key) {
      const int of = sp.ctx_tiles + key / TILE;
      if (of < first || (of - begin) % WK != wk) continue;
      const uint16_t *vp = a.b.v + (int64_t)(t0 + key) * a.b.v_row + kh * a.b.v_head;
#pragma unroll
      for (int x = 0; x < NR; ++x) {
        const int row = base + 16 * x + n16;
        if (row >= rows || !(masks[row / a.group] >> key & 1)) continue;
#pragma unroll
        for (int d = 0; d < 2 * DC; ++d) {
          const int at = 16 * d + 4 * g4;
          if (at >= dim) continue;
          const u2 four = *(const u2 *)(vp + at);
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const uint16_t raw = (uint16_t)(four[i >> 1] >> 16 * (i & 1));
            if ((raw & 0x7c00) == 0x7c00) o[x][d][i] += (float)__builtin_bit_cast(_Float16, raw);
          }
        }
      }
    }
  }
#pragma unroll
  for (int x = 0; x < NR; ++x) {
    float top = -INFINITY, total = 0.f;
#pragma unroll
    for (int w = 0; w < WK; ++w) top = fmaxf(top, refs[WR * w + wr][16 * x + n16]);
    const float safe_top = top == -INFINITY ? 0.f : top;
#pragma unroll
    for (int w = 0; w < WK; ++w) {
      const float rw = refs[WR * w + wr][16 * x + n16];
      // (a wave without a reference has no weight, or only NaN: it keeps what it has)
      total += (rw == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(rw - safe_top)) * sums[WR * w + wr][16 * x + n16];
    }
    const float ref2 = ref[x] * a.scale2, f = ref2 == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(ref2 - safe_top);
    if (WK > 1) {
      float *area = (float *)(lds + wave * KV);
      // row n of 16, d back to back; rows are shifted by their number so that a store of 16 rows spreads over the banks
#pragma unroll
      for (int d = 0; d < 2 * DC; ++d) {
        f4 v = o[x][d];
#pragma unroll
        for (int i = 0; i < 4; ++i) v[i] *= f;
        *(f4 *)(area + n16 * (32 * DC) + 4 * ((4 * d + g4) ^ (n16 & 7))) = v;
      }
      __syncthreads();
      // wave w of the WK takes a WK-th of the d tiles
#pragma unroll
      for (int d = 0; d < 2 * DC; ++d) {
        if (d % WK != wk) continue;
        f4 v = {0, 0, 0, 0};
#pragma unroll
        for (int w = 0; w < WK; ++w) {
          const float *from = (const float *)(lds + (WR * w + wr) * KV);
          const f4 u = *(const f4 *)(from + n16 * (32 * DC) + 4 * ((4 * d + g4) ^ (n16 & 7)));
#pragma unroll
          for (int i = 0; i < 4; ++i) v[i] += u[i];
        }
        o[x][d] = v;
      }
    }
    const int row = base + 16 * x + n16, tok = row / a.group, h = kh * a.group + row - tok * a.group;
    if (row < rows) {
      if (sp.count == 1) {
        uint16_t *out = a.b.out + (int64_t)(t0 + tok) * a.b.out_row + (int64_t)h * a.b.out_head;
        const float inv = total == 0.f ? 0.f : 1.f / total;
#pragma unroll
        for (int d = 0; d < 2 * DC; ++d) {
          if (WK > 1 && d % WK != wk) continue;
          const int at = 16 * d + 4 * g4;
          if (at < dim) {
            u2 w;
#pragma unroll
            for (int i = 0; i < 2; ++i) {
              const h2 y = {(_Float16)(o[x][d][2 * i] * inv), (_Float16)(o[x][d][2 * i + 1] * inv)};
              w[i] = bad ? 0x7e007e00u : __builtin_bit_cast(uint32_t, y);
            }
            *(u2 *)(out + at) = w;
          }
        }
      } else {
        const int64_t to = ((int64_t)blockIdx.x * a.b.tokens + t0 + tok) * a.b.heads + h;
        if (wk == 0 && g4 == 0) a.ml[to] = float2{top, bad ? __builtin_nanf("") : total};
#pragma unroll
        for (int d = 0; d < 2 * DC; ++d) {
          if (WK > 1 && d % WK != wk) continue;
          const int at = 16 * d + 4 * g4;
          if (at < dim) *(f4 *)(a.part + to * dim + at) = o[x][d];
        }
      }
    }
    if (WK > 1) __syncthreads();
  }
}

// The spans of a row join: one wave a row, in the order of the spans.
__global__ __launch_bounds__(256) void k_tree_join(TreeArgs a) {
  const int r = blockIdx.z, lane = threadIdx.x & 63, h = blockIdx.x * 4 + (threadIdx.x >> 6);
  const int t0 = a.b.cu_tokens[r], t1 = a.b.cu_tokens[r + 1], len = a.b.lens[r], i = t0 + blockIdx.y;
  if (request_state(a, t0, t1, len) != ROWS_FINE || i >= t1 || h >= a.b.heads) return;
  const Spans sp = spans_of(len, t1 - t0, a.splits, a.min_tiles, a.whole);
  if (sp.count == 1) return;
  const int64_t row = (int64_t)i * a.b.heads + h, step = (int64_t)a.b.tokens * a.b.heads;
  float2 mine = lane < sp.count ? a.ml[lane * step + row] : float2{-INFINITY, 0.f};     // (64 spans at most)
  float top = mine.x;
#pragma unroll
  for (int x = 32; x > 0; x >>= 1) top = fmaxf(top, __shfl_xor(top, x, 64));
  const float w = mine.x == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(mine.x - (top == -INFINITY ? 0.f : top));
  float total = w * mine.y;
#pragma unroll
  for (int x = 32; x > 0; x >>= 1) total += __shfl_xor(total, x, 64);
  // lanes that the row's values leave over take spans of their own: `teams` of 1 << tshift lanes, joined at the end
  const int tshift = a.c.dim > 128 ? 6 : a.c.dim > 64 ? 5 : a.c.dim > 32 ? 4 : 3, teams = 64 >> tshift, d = 4 * (lane & ((1 << tshift) - 1));
  f4 v = {0, 0, 0, 0};
  const float *p = a.part + row * a.c.dim + (d < a.c.dim ? d : 0);
#pragma unroll 8
  for (int s = lane >> tshift; s < 64; s += teams) {
    if (s - (lane >> tshift) >= sp.count) break;      // (all teams leave together)
    const float f = __shfl(w, s, 64);                 // (every lane is here: lane s may have no part of the row)
    const f4 u = *(const f4 *)(p + min(s, sp.count - 1) * step * a.c.dim);
#pragma unroll
    for (int e = 0; e < 4; ++e) v[e] = s < sp.count ? fmaf(f, u[e], v[e]) : v[e];
  }
  for (int x = 32; x >= 1 << tshift; x >>= 1)
#pragma unroll
    for (int e = 0; e < 4; ++e) v[e] += __shfl_xor(v[e], x, 64);
  if (lane < 1 << tshift && d < a.c.dim) {
    const float inv = total == 0.f ? 0.f : 1.f / total;
    const h2 lo = {(_Float16)(v[0] * inv), (_Float16)(v[1] * inv)}, hi = {(_Float16)(v[2] * inv), (_Float16)(v[3] * inv)};
    *(u2 *)(a.b.out + i * a.b.out_row + h * a.b.out_head + d) = u2{__builtin_bit_cast(uint32_t, lo), __builtin_bit_cast(uint32_t, hi)};
  }
}

egt_status check_sizes(const egt_tree_batch *b, const egt_kv_cache *c) {
  if (!b) return EGT_ERR_NULL;
  const egt_status st = check_cache(c, false);
  if (st != EGT_OK) return st;
  if (b->requests < 0 || b->tokens < 0 || b->heads < 1 || b->heads % c->heads != 0 || b->max_tokens < 1 || b->max_tokens > EGT_MAX_TREE || b->table_blocks < 0 ||
      (int64_t)b->table_blocks * c->page > (1ll << 30))
    return EGT_ERR_SHAPE;
  return b->requests > EGT_MAX_REQUESTS || b->heads > 4096 ? EGT_ERR_UNSUPPORTED : EGT_OK;
}

constexpr int MAX_SPLITS = 64;
struct Shape { int nr, wr, row_blocks, splits, min_tiles, whole; };
Shape shape_of(const egt_tree_batch &b, const egt_kv_cache &c) {
  Shape s;
  const int rows = b.max_tokens * (b.heads / c.heads);
  // Two row tiles a wave from 65 rows on (up to 128 rows, us, two tiles of four waves against one of eight: sixteen requests of up to 80 rows
  // 52.8 / 53.9, 128 rows over 131072 keys 151 / 185 when both were there, 130 to 140 now); wider heads have no registers for them.
  s.nr = rows <= 64 || c.dim > 128 ? 1 : 2;
  s.wr = 1;
  while (s.wr < 8 && rows > 16 * s.nr * s.wr) s.wr *= 2;
  s.row_blocks = (rows + 16 * s.nr * s.wr - 1) / (16 * s.nr * s.wr);
  // A span is a tile a wave at least, and four tiles; up to two tiles a wave, and eight tiles, stay whole, for joining costs a launch (us,
  // one token over 777 keys of 32 heads: four spans and a join 13.7, one span of 3.4 tiles a wave 15.2; over 300 keys: three spans 12.8, one 11.8).
  const int waves = waves_of((c.dim + 31) / 32, s.wr);
  s.min_tiles = std::max(waves / s.wr, 4);
  s.whole = 2 * s.min_tiles;
  const int64_t groups = (int64_t)std::max(b.requests, 1) * c.heads * s.row_blocks, tiles = ((int64_t)b.table_blocks * c.page + TILE - 1) / TILE + 2;
  s.splits = (int)std::min<int64_t>({std::max<int64_t>((waves == 8 ? 256 : 512) / groups, 1), (tiles + s.min_tiles - 1) / s.min_tiles, MAX_SPLITS});
  if (tiles <= s.whole) s.splits = 1;
  return s;
}
size_t rows_of(const egt_tree_batch &b) { return (size_t)b.tokens * b.heads; }
size_t workspace_of(const egt_tree_batch &b, const egt_kv_cache &c) {
  const Shape s = shape_of(b, c);
  if (s.splits == 1) return 16;
  return ((rows_of(b) * s.splits * 4 * (c.dim + 2) + 15) & ~(size_t)15) + 16;
}

template <int DC, int NR, int WR>
hipError_t launch_tree(const TreeArgs &a, hipStream_t stream) {
  constexpr size_t bytes = (size_t)(waves_of(DC, WR) / WR) * (WR > 1 ? 2 : 1) * 2 * TILE * 64 * DC;
  if (bytes > 60 * 1024) {
    const hipError_t e = hipFuncSetAttribute((const void *)k_tree<DC, NR, WR>, hipFuncAttributeMaxDynamicSharedMemorySize, (int)bytes);
    if (e != hipSuccess) return e;
  }
  return launch(k_tree<DC, NR, WR>, dim3(a.splits, a.c.heads * a.row_blocks, a.b.requests), dim3(64 * waves_of(DC, WR)), bytes, stream, a);
}
template <int DC>
hipError_t launch_dim(const TreeArgs &a, const Shape &s, hipStream_t stream) {
  if constexpr (DC <= 4)
    if (s.nr == 2) return s.wr == 4 ? launch_tree<DC, 2, 4>(a, stream) : launch_tree<DC, 2, 8>(a, stream);
  switch (s.wr) {
    case 1: return launch_tree<DC, 1, 1>(a, stream);
    case 2: return launch_tree<DC, 1, 2>(a, stream);
    case 4: return launch_tree<DC, 1, 4>(a, stream);
    default: break;
  }
  if constexpr (DC > 4) return launch_tree<DC, 1, 8>(a, stream);
  return hipErrorInvalidValue;                        // (not reached: shape_of takes no other)
}

}  // namespace
}  // namespace egt

extern "C" {

egt_status egt_tree_attention_ws_bytes(const egt_tree_batch *b, const egt_kv_cache *cache, size_t *bytes) {
  if (!bytes) return EGT_ERR_NULL;
  const egt_status st = egt::check_sizes(b, cache);
  if (st == EGT_OK) *bytes = egt::workspace_of(*b, *cache);
  return st;
}

egt_status egt_tree_attention(const egt_tree_batch *b, const egt_kv_cache *cache, void *workspace, size_t workspace_bytes, void *stream) {
  egt_status st = egt::check_sizes(b, cache);
  if (st != EGT_OK) return st;
  st = egt::check_cache(cache, true);
  if (st != EGT_OK) return st;
  if (b->ld_table < b->table_blocks || !(__builtin_fabsf(b->scale) <= 0x1p126f)) return EGT_ERR_SHAPE;
  if (std::max({cache->k_block, cache->v_block, cache->k_token, cache->v_token, b->k_row, b->v_row}) >= 1ll << 31) return EGT_ERR_UNSUPPORTED;
  if (b->requests == 0 || b->tokens == 0) return EGT_OK;
  if (!b->q || !b->k || !b->v || !b->out || !b->lens || !b->cu_tokens || !b->mask || (b->table_blocks && !b->block_table) || !workspace) return EGT_ERR_NULL;
  if (workspace_bytes < egt::workspace_of(*b, *cache)) return EGT_ERR_SHAPE;
  if (!egt::whole16(b->q) || !egt::whole16(b->k) || !egt::whole16(b->v) || !egt::whole16(b->out) || !egt::whole16(workspace) ||
      !egt::whole8(b->q_row, b->q_head, b->k_row, b->k_head, b->v_row, b->v_head, b->out_row, b->out_head) || ((uintptr_t)b->mask & 7) ||
      ((uintptr_t)b->lens & 3) || ((uintptr_t)b->cu_tokens & 3) || ((uintptr_t)b->block_table & 3))
    return EGT_ERR_BUFFER;
  const egt::Shape s = egt::shape_of(*b, *cache);
  egt::TreeArgs a;
  a.b = *b;
  a.c = *cache;
  a.part = (float *)workspace;
  a.ml = (float2 *)(a.part + (egt::rows_of(*b) * s.splits * cache->dim + 3) / 4 * 4);
  a.shift = egt::log2_of(cache->page);
  a.group = b->heads / cache->heads;
  a.splits = s.splits;
  a.row_blocks = s.row_blocks;
  a.min_tiles = s.min_tiles;
  a.whole = s.whole;
  a.scale2 = std::max(__builtin_fabsf(b->scale) * 1.44269504088896340736f, 0x1p-126f);      // (zero times a masked score would be NaN)
  a.flip = __builtin_signbit(b->scale) ? 0x80008000u : 0u;
  const hipStream_t to = (hipStream_t)stream;
  hipError_t e;
  switch ((cache->dim + 31) / 32) {
    case 1: case 2: e = egt::launch_dim<2>(a, s, to); break;
    case 3: e = egt::launch_dim<3>(a, s, to); break;
    case 4: e = egt::launch_dim<4>(a, s, to); break;
    case 5: case 6: e = egt::launch_dim<6>(a, s, to); break;
    default: e = egt::launch_dim<8>(a, s, to); break;
  }
  if (e == hipSuccess && s.splits > 1) e = egt::launch(egt::k_tree_join, dim3((b->heads + 3) / 4, b->max_tokens, b->requests), dim3(256), 0, to, a);
  return egt::answer(e);
}

}  // extern "C"
