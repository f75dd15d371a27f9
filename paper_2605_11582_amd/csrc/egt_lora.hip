// Low-rank adapters of many requests beside a shared projection.
//
// Y[m] = base[m] + s B (A x[m]) for a few tokens an adapter and many adapters: every adapter in use is read once, and that is what
// bounds it (rank 32 beside 11008 x 4096: 0.95 MB an adapter).  Two kernels, for all of h = A x has to be there before any of B h:
//  - k_lora_shrink: a workgroup is one adapter and SLICE columns of A; its four waves take K-steps of 32 columns in turn, join
//    through LDS and leave FP32 partial sums in the workspace;
//  - k_lora_expand: a workgroup is one adapter and some rows of B; it adds the slices up, in order, and multiplies.
// Which tokens an adapter has is found by the workgroup itself: up to 64 tokens are one ballot.  The first of them speaks for the
// adapter, the workgroups of the others end at once.  Weights come straight from memory into operands: nothing is used twice.
// h goes into the second product as two FP16 numbers, each summed by itself: the first scaled by a power of two so that the token's
// largest is 2^14 .. 2^15, the second what the first leaves, 2^12 times as large.  That is 22 bits of every entry down to 2^-28 of
// the largest.  A token whose entries lie further apart, or are not finite, takes the result of the matrix instruction for FP32
// (for all tokens that costs 4 us of 64 tokens, 40 adapters of rank 32 beside 11008 x 4096: 15.5 -> 19.3).
#include "egt_mfma_common.h"
#include "egt_serve.h"

#include <algorithm>

namespace egt {
namespace {

constexpr int MAX_RANK = 128, SLICE = 512;

// The tokens that have token m's adapter (all without one, and all past the last one, count as one adapter each); `a`: that adapter,
// -1 or b.adapters.  0 where another token speaks for them.
__device__ __forceinline__ uint64_t members_of(const egt_lora_batch &b, int m, int &a) {
  const int lane = threadIdx.x & 63;
  int mine = lane < b.M ? b.index[lane] : 0;
  mine = mine < 0 ? -1 : min(mine, b.adapters);
  a = __builtin_amdgcn_readlane(mine, m);
  const uint64_t all = __ballot(lane < b.M && mine == a);
  return __builtin_ctzll(all) == m ? all : 0;
}
// ... one after the other (every wave writes the same)
__device__ __forceinline__ void list_members(uint64_t all, uint8_t *list) {
  const int lane = threadIdx.x & 63;
  if (all >> lane & 1) list[__builtin_popcountll(all & ((1ull << lane) - 1))] = (uint8_t)lane;
  __syncthreads();
}

template <int NT>      // tiles of 16 tokens
__device__ __forceinline__ void shrink(const egt_lora_batch &b, float *part, int a, int count, const uint8_t *list, f4 (*join)[NT][64]) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, n16 = lane & 15, g4 = lane >> 4;
  const int first = blockIdx.x * SLICE, width = min(SLICE, b.cols - first);
  const uint16_t *x[NT];
#pragma unroll
  for (int t = 0; t < NT; ++t) x[t] = b.X + list[min(16 * t + n16, count - 1)] * b.ldx + first;
  for (int j0 = 0; j0 < b.rank; j0 += 16) {
    const uint16_t *w = b.A + a * b.a_stride + (int64_t)min(j0 + n16, b.rank - 1) * b.cols + first;
    constexpr int STEPS = SLICE / 128;
    u4 wr[STEPS], xr[STEPS][NT];
#pragma unroll
    for (int s = 0; s < STEPS; ++s) {
      const int c = 128 * s + 32 * wave + 8 * g4, at = c < width ? c : 0;
      wr[s] = *(const u4 *)(w + at);
#pragma unroll
      for (int t = 0; t < NT; ++t) xr[s][t] = *(const u4 *)(x[t] + at);
    }
    f4 acc[NT];
#pragma unroll
    for (int t = 0; t < NT; ++t) acc[t] = f4{0, 0, 0, 0};
#pragma unroll
    for (int s = 0; s < STEPS; ++s) {
      const bool fine = 128 * s + 32 * wave + 8 * g4 < width;
      const u4 v = fine ? wr[s] : u4{0, 0, 0, 0};
#pragma unroll
      for (int t = 0; t < NT; ++t) {
        const u4 y = fine ? xr[s][t] : u4{0, 0, 0, 0};
        acc[t] = __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(h8, v), __builtin_bit_cast(h8, y), acc[t], 0, 0, 0);
      }
    }
    // lane (g, n): ranks j0 + 4 g .. + 3 of token n
#pragma unroll
    for (int t = 0; t < NT; ++t) join[wave][t][lane] = acc[t];
    __syncthreads();
    for (int t = wave; t < NT; t += 4) {
      f4 sum = join[0][t][lane];
#pragma unroll
      for (int v = 1; v < 4; ++v)
#pragma unroll
        for (int i = 0; i < 4; ++i) sum[i] += join[v][t][lane][i];
      const int n = 16 * t + n16, j = j0 + 4 * g4;
      if (n < count && j < b.rank) *(f4 *)(part + ((int64_t)blockIdx.x * b.M + list[n]) * b.rank + j) = sum;
    }
    __syncthreads();
  }
}

__global__ __launch_bounds__(256) void k_lora_shrink(egt_lora_batch b, float *part) {
  __shared__ uint8_t list[64];
  __shared__ f4 join[4][4][64];
  int a;
  const uint64_t all = members_of(b, blockIdx.y, a);
  if (!all || a < 0 || a >= b.adapters) return;
  list_members(all, list);
  const int count = __builtin_popcountll(all);
  if (count <= 16)
    shrink<1>(b, part, a, count, list, (f4(*)[1][64])join);
  else
    shrink<4>(b, part, a, count, list, join);
}

// Four values of a token from row `at` on, of `rows`: 8 bytes at once (WHOLE) or one by one.  A load takes rows that there are.
template <bool WHOLE>
__device__ __forceinline__ u2 get4(const uint16_t *p, int at, int rows) {
  if (WHOLE) return *(const u2 *)(p + min(at, rows - 4));
  uint32_t v[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) v[i] = p[min(at + i, rows - 1)];
  return u2{v[0] | v[1] << 16, v[2] | v[3] << 16};
}
template <bool WHOLE>
__device__ __forceinline__ void put4(uint16_t *p, int at, int rows, u2 v) {
  if (WHOLE) {
    if (at < rows) *(u2 *)(p + at) = v;
  } else {
    const uint32_t x = v.x, y = v.y;
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (at + i < rows) p[at + i] = (uint16_t)((i < 2 ? x : y) >> 16 * (i & 1));
  }
}

// Chunks of 32 ranks; tiles of 16 rows a wave; WHOLE: four rows of base and Y are 8 bytes of memory that can be asked for at once.
// All that a token needs is requested together: B before anything that has to be waited for, then base and the partial sums
// (64 tokens, 40 adapters of rank 32 beside 11008 x 4096, both kernels: 15.5 us; with a wait for each tile's base, and three waves a SIMD, 18.7).
template <int RC, int TILES, bool WHOLE>
__global__ __launch_bounds__(256, 2) void k_lora_expand(egt_lora_batch b, const float *part, int slices) {
  __shared__ uint8_t list[64];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, n16 = lane & 15, g4 = lane >> 4;
  int a;
  const uint64_t all = members_of(b, blockIdx.y, a);
  if (!all) return;
  const int count = __builtin_popcountll(all), row0 = (blockIdx.x * 4 + wave) * 16 * TILES;
  const bool based = b.base != nullptr;
  const uint16_t *base = based ? b.base : b.B;        // (any memory: read and not looked at)
  const int64_t ldbase = based ? b.ldbase : 0;
  if (a < 0 || a >= b.adapters) {                     // no adapter, or none that there is
    list_members(all, list);
    for (int n0 = 0; n0 < count; n0 += 16) {
      const int m = list[min(n0 + n16, count - 1)];
      u2 y[TILES];
#pragma unroll
      for (int t = 0; t < TILES; ++t) y[t] = get4<WHOLE>(base + m * ldbase, row0 + 16 * t + 4 * g4, b.rows);
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int t = 0; t < TILES; ++t) {
        const u2 nan = {0x7e007e00u, 0x7e007e00u}, none = {0, 0};
        if (n0 + n16 < count) put4<WHOLE>(b.Y + m * b.ldy, row0 + 16 * t + 4 * g4, b.rows, a >= 0 ? nan : based ? y[t] : none);
      }
    }
    return;
  }
  // the rows of B, as the A operand
  u4 w[TILES][RC];
#pragma unroll
  for (int t = 0; t < TILES; ++t)
#pragma unroll
    for (int c = 0; c < RC; ++c) {
      const int j = 32 * c + 8 * g4;
      w[t][c] = *(const u4 *)(b.B + a * b.b_stride + (int64_t)min(row0 + 16 * t + n16, b.rows - 1) * b.rank + (j < b.rank ? j : 0));
    }
  list_members(all, list);
  if (row0 >= b.rows) return;
  const float scale = b.scale ? b.scale[a] : 1.f;
  constexpr int FAR = (TILES > 4 ? 4 : 8) / RC;                         // slices at once (rank 32, eight tiles: few enough for four waves a SIMD; 17.7 us with three)
  auto tokens = [&](int n0) {                         // (16 of them)
    const int m = list[min(n0 + n16, count - 1)];
    u2 y[TILES];
#pragma unroll
    for (int t = 0; t < TILES; ++t) y[t] = get4<WHOLE>(base + m * ldbase, row0 + 16 * t + 4 * g4, b.rows);
    // h of this lane's token, as the B operand: ranks 32 c + 8 g .. + 7
    f4 h[RC][2];
#pragma unroll
    for (int c = 0; c < RC; ++c) h[c][0] = h[c][1] = f4{0, 0, 0, 0};
    for (int s0 = 0; s0 < slices; s0 += FAR) {
      f4 u[FAR][RC][2];
#pragma unroll
      for (int s = 0; s < FAR; ++s)
#pragma unroll
        for (int c = 0; c < RC; ++c) {
          const int j = 32 * c + 8 * g4;
          const float *p = part + ((int64_t)min(s0 + s, slices - 1) * b.M + m) * b.rank + (j < b.rank ? j : 0);
          u[s][c][0] = *(const f4 *)p;
          u[s][c][1] = *(const f4 *)(p + 4);
        }
      __builtin_amdgcn_sched_barrier(0);              // (left alone, the compiler asks for one slice after the other)
#pragma unroll
      for (int s = 0; s < FAR; ++s)
#pragma unroll
        for (int c = 0; c < RC; ++c)
#pragma unroll
          for (int i = 0; i < 8; ++i) h[c][i >> 2][i & 3] += s0 + s < slices ? u[s][c][i >> 2][i & 3] : 0.f;
    }
    // (sizes as whole numbers, which order as they do; `least`: one less than the smallest that is not zero)
    uint32_t most = 0, least = ~0u;
#pragma unroll
    for (int c = 0; c < RC; ++c)
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        if (32 * c + 8 * g4 >= b.rank) h[c][i >> 2][i & 3] = 0.f;
        const uint32_t size = __builtin_bit_cast(uint32_t, fabsf(h[c][i >> 2][i & 3]));
        most = max(most, size);
        least = min(least, size - 1);
      }
#pragma unroll
    for (int x = 16; x < 64; x *= 2) {
      most = max(most, (uint32_t)__shfl_xor((int)most, x, 64));
      least = min(least, (uint32_t)__shfl_xor((int)least, x, 64));
    }
    // `product(t)`: lane (g, n) gets rows 4 g .. + 3 of tile t, of token n.  (Past the rank: weights of rank 0 .. 7 times zeros.)
    auto finish = [&](auto product) {
#pragma unroll
      for (int t = 0; t < TILES; ++t) {
        const f4 sum = product(t);
        const uint32_t y01 = based ? y[t].x : 0u, y23 = based ? y[t].y : 0u;
        const h2 u01 = __builtin_bit_cast(h2, y01), u23 = __builtin_bit_cast(h2, y23);
        const h2 z01 = {(_Float16)((float)u01[0] + sum[0] * scale), (_Float16)((float)u01[1] + sum[1] * scale)};
        const h2 z23 = {(_Float16)((float)u23[0] + sum[2] * scale), (_Float16)((float)u23[1] + sum[3] * scale)};
        if (n0 + n16 < count) put4<WHOLE>(b.Y + m * b.ldy, row0 + 16 * t + 4 * g4, b.rows, u2{__builtin_bit_cast(uint32_t, z01), __builtin_bit_cast(uint32_t, z23)});
      }
    };
    constexpr uint32_t LARGE = (127 + 90) << 23, SMALL = (127 - 90) << 23, REACH = 28 << 23;      // 2^90, 2^-90, a ratio of 2^28
    const bool apart = most > LARGE || (most != 0 && (most < SMALL || least + 1 < most - REACH));
    const int e = max((int)(most >> 23) - 127, -90);
    const float up = __builtin_bit_cast(float, (uint32_t)(127 + 14 - e) << 23), back = __builtin_bit_cast(float, (uint32_t)(127 - 14 + e) << 23);
    h8 hi[RC], lo[RC];
#pragma unroll
    for (int c = 0; c < RC; ++c)
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const float v = h[c][i >> 2][i & 3] * up;
        hi[c][i] = (_Float16)v;
        lo[c][i] = (_Float16)((v - (float)hi[c][i]) * 4096.f);
      }
    auto halves = [&](int t) {
      f4 acc = {0, 0, 0, 0}, fine = {0, 0, 0, 0};
#pragma unroll
      for (int c = 0; c < RC; ++c) {
        acc = __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(h8, w[t][c]), hi[c], acc, 0, 0, 0);
        fine = __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(h8, w[t][c]), lo[c], fine, 0, 0, 0);
      }
#pragma unroll
      for (int i = 0; i < 4; ++i) acc[i] = fmaf(fine[i], 0x1p-12f, acc[i]) * back;
      return acc;
    };
    if (!__any(apart)) {
      finish(halves);
    } else {                                          // (a token's form is its own, whoever is beside it)
      finish([&](int t) {
        const f4 narrow = halves(t);
        f4 acc = {0, 0, 0, 0};
#pragma unroll
        for (int c = 0; c < RC; ++c) {
          u4 here = w[t][c];
          asm volatile("" : "+v"(here));              // (widened here and now: ahead of the loop over tokens it would cost eight registers)
          const h8 v = __builtin_bit_cast(h8, here);
#pragma unroll
          for (int i = 0; i < 8; ++i) acc = __builtin_amdgcn_mfma_f32_16x16x4f32((float)v[i], h[c][i >> 2][i & 3], acc, 0, 0, 0);      // (ranks 8 g + i)
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) acc[i] = apart ? acc[i] : narrow[i];
        return acc;
      });
    }
  };
  tokens(0);                                          // (by itself: a loop would wait for B at its start)
  for (int n0 = 16; n0 < count; n0 += 16) tokens(n0);
}

template <int RC>
hipError_t launch_expand(const egt_lora_batch &b, const float *part, int slices, hipStream_t stream) {
  // Row tiles a wave: more where there are plenty of rows if every token has an adapter of its own (the workgroups of tokens that
  // another one speaks for are launched too).  us of both kernels, 1024 columns, ranks 32 / 64 / 128, one tile against four: 512 groups
  // 8.0 / 10.0 / 16.2 against 8.4 / 10.3 / 16.2, 1024 groups 9.2 / 12.8 / 20.2 against 8.5 / 11.4 / 18.0, 2048 groups 13.1 / 17.8 / 26.8
  // against 9.8 / 14.2 / 21.3; four against eight, ranks 32 / 64: 3008 groups 11.9 / 16.0 against 11.5 / 16.2, 4096 groups 12.6 / 19.5
  // against 11.9 / 16.9, 11008 groups 20.6 / 33.3 against 17.7 / 30.2 (rank 128 has no registers for eight).
  const int64_t groups = (int64_t)((b.rows + 63) / 64) * std::min(b.M, b.adapters);
  const bool whole = b.rows % 4 == 0 && b.ldy % 4 == 0 && ((uintptr_t)b.Y & 7) == 0 && (!b.base || (b.ldbase % 4 == 0 && ((uintptr_t)b.base & 7) == 0));
  if (!whole) return launch(k_lora_expand<RC, 1, false>, dim3((b.rows + 63) / 64, b.M), dim3(256), 0, stream, b, part, slices);
  if constexpr (RC < 4)
    if (groups >= 4096) return launch(k_lora_expand<RC, 8, true>, dim3((b.rows + 511) / 512, b.M), dim3(256), 0, stream, b, part, slices);
  if (groups >= 2048) return launch(k_lora_expand<RC, 4, true>, dim3((b.rows + 255) / 256, b.M), dim3(256), 0, stream, b, part, slices);
  return launch(k_lora_expand<RC, 1, true>, dim3((b.rows + 63) / 64, b.M), dim3(256), 0, stream, b, part, slices);
}

egt_status check_sizes(int M, int cols, int rank) {
  if (M < 1 || M > 64 || cols < 8 || cols % 8 != 0 || rank < 8 || rank % 8 != 0) return EGT_ERR_SHAPE;
  return rank > MAX_RANK || cols > 1 << 30 ? EGT_ERR_UNSUPPORTED : EGT_OK;
}
int slices_of(int cols) { return (cols + SLICE - 1) / SLICE; }
size_t workspace_of(int M, int cols, int rank) { return 4 * (size_t)slices_of(cols) * M * rank; }

}  // namespace
}  // namespace egt

extern "C" {

egt_status egt_lora_smallm_ws_bytes(int M, int cols, int rank, size_t *bytes) {
  if (!bytes) return EGT_ERR_NULL;
  const egt_status st = egt::check_sizes(M, cols, rank);
  if (st == EGT_OK) *bytes = egt::workspace_of(M, cols, rank);
  return st;
}

egt_status egt_lora_smallm(const egt_lora_batch *b, void *workspace, size_t workspace_bytes, void *stream) {
  if (!b) return EGT_ERR_NULL;
  const egt_status st = egt::check_sizes(b->M, b->cols, b->rank);
  if (st != EGT_OK) return st;
  if (b->rows < 0 || b->adapters < 1 || b->ldx < b->cols || b->ldy < b->rows || (b->base && b->ldbase < b->rows) ||
      (b->base == b->Y && b->base && b->ldbase != b->ldy) || b->a_stride < 0 || b->b_stride < 0)
    return EGT_ERR_SHAPE;
  if (b->rows > (1 << 30) - 64) return EGT_ERR_UNSUPPORTED;      // (a launch has less than 2^32 threads)
  if (b->rows == 0) return EGT_OK;                    // nothing to compute, pointers not examined
  if (!b->X || !b->A || !b->B || !b->Y || !b->index || !workspace) return EGT_ERR_NULL;
  if (workspace_bytes < egt::workspace_of(b->M, b->cols, b->rank)) return EGT_ERR_SHAPE;
  if (!egt::whole16(b->X) || !egt::whole16(b->A) || !egt::whole16(b->B) || !egt::whole16(workspace) || !egt::whole8(b->ldx, b->a_stride, b->b_stride) ||
      ((uintptr_t)b->index & 3) || ((uintptr_t)b->scale & 3) || ((uintptr_t)b->base & 1) || ((uintptr_t)b->Y & 1))
    return EGT_ERR_BUFFER;
  const int slices = egt::slices_of(b->cols);
  hipError_t e = egt::launch(egt::k_lora_shrink, dim3(slices, b->M), dim3(256), 0, (hipStream_t)stream, *b, (float *)workspace);
  if (e != hipSuccess) return egt::answer(e);
  const hipStream_t to = (hipStream_t)stream;
  const float *part = (const float *)workspace;
  return egt::answer(b->rank <= 32 ? egt::launch_expand<1>(*b, part, slices, to) : b->rank <= 64 ? egt::launch_expand<2>(*b, part, slices, to)
                                                                                                 : egt::launch_expand<4>(*b, part, slices, to));
}

}  // extern "C"
