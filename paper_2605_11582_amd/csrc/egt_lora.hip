// Low-rank adapters of many requests beside a shared projection.
//
// Y[m] = base[m] + s B (A x[m]) for a few tokens an adapter and many adapters: every adapter in use is read once, and that is what
// bounds it (rank 32 beside 11008 x 4096: 0.95 MB an adapter).  Two kernels, for all of h = A x has to be there before any of B h:
//  - k_lora_shrink: a workgroup is one adapter and SLICE columns of A; its four waves take K-steps of 32 columns in turn, join
//    through LDS and leave FP32 partial sums in the workspace;
//  - k_lora_expand: a workgroup is one adapter and some rows of B; it adds the slices up, in order, and multiplies.
// Which tokens an adapter has is found by the workgroup itself: up to 64 tokens are one ballot.  The first of them speaks for the
// adapter, the workgroups of the others end at once.  Weights come straight from memory into operands: nothing is used twice.
// h goes into the second product as two FP16 numbers, scaled by a power of two so that the token's largest is 1 .. 2: 22 bits, and no overflow.
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

// 4 rows of Y, or of base, of one token: whole 8 bytes where memory and rows allow it
__device__ __forceinline__ void put4(uint16_t *p, int left, bool whole, const float (&v)[4]) {
  if (whole && left >= 4) {
    const h2 lo = {(_Float16)v[0], (_Float16)v[1]}, hi = {(_Float16)v[2], (_Float16)v[3]};
    *(u2 *)p = u2{__builtin_bit_cast(uint32_t, lo), __builtin_bit_cast(uint32_t, hi)};
  } else {
    for (int i = 0; i < 4; ++i)
      if (i < left) p[i] = __builtin_bit_cast(uint16_t, (_Float16)v[i]);
  }
}
__device__ __forceinline__ void get4(const uint16_t *p, int left, bool whole, float (&v)[4]) {
  if (whole && left >= 4) {
    const u2 w = *(const u2 *)p;
    const uint32_t x = w.x, y = w.y;                  // (a bit cast of a vector's element takes its first one here)
    const h2 lo = __builtin_bit_cast(h2, x), hi = __builtin_bit_cast(h2, y);
    v[0] = lo[0], v[1] = lo[1], v[2] = hi[0], v[3] = hi[1];
  } else {
    for (int i = 0; i < 4; ++i) v[i] = i < left ? (float)__builtin_bit_cast(_Float16, p[i]) : 0.f;
  }
}

template <int RC, int TILES>      // chunks of 32 ranks; tiles of 16 rows a wave
__global__ __launch_bounds__(256) void k_lora_expand(egt_lora_batch b, const float *part, int slices) {
  __shared__ uint8_t list[64];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, n16 = lane & 15, g4 = lane >> 4;
  int a;
  const uint64_t all = members_of(b, blockIdx.y, a);
  if (!all) return;
  const int count = __builtin_popcountll(all), row0 = (blockIdx.x * 4 + wave) * 16 * TILES;
  const bool some = a >= 0 && a < b.adapters;
  // the rows of B, as the A operand: requested before anything that has to be waited for
  u4 w[TILES][RC];
  if (some) {
#pragma unroll
    for (int t = 0; t < TILES; ++t)
#pragma unroll
      for (int c = 0; c < RC; ++c) {
        const int j = 32 * c + 8 * g4;
        w[t][c] = ld_stream<u4>(b.B + a * b.b_stride + (int64_t)min(row0 + 16 * t + n16, b.rows - 1) * b.rank + (j < b.rank ? j : 0));
      }
  }
  list_members(all, list);
  if (row0 >= b.rows) return;
  const bool base8 = ((uintptr_t)b.base & 7) == 0 && b.ldbase % 4 == 0, y8 = ((uintptr_t)b.Y & 7) == 0 && b.ldy % 4 == 0;
  const float scale = some && b.scale ? b.scale[a] : 1.f;
  for (int n0 = 0; n0 < count; n0 += 16) {
    const bool mine = n0 + n16 < count;
    const int m = list[min(n0 + n16, count - 1)];
    float y[TILES][4];
#pragma unroll
    for (int t = 0; t < TILES; ++t) {
      const int at = row0 + 16 * t + 4 * g4;
#pragma unroll
      for (int i = 0; i < 4; ++i) y[t][i] = 0.f;
      if (b.base && mine && at < b.rows) get4(b.base + m * b.ldbase + at, b.rows - at, base8, y[t]);
    }
    // h of this lane's token, as the B operand: ranks 32 c + 8 g .. + 7
    h8 hi[RC], lo[RC];
    float back = 1.f;
    if (some) {
      float h[RC][8], most = 0.f;
#pragma unroll
      for (int c = 0; c < RC; ++c) {
        const int j = 32 * c + 8 * g4;
        const float *p = part + (int64_t)m * b.rank + (j < b.rank ? j : 0);
        f4 s0 = {0, 0, 0, 0}, s1 = {0, 0, 0, 0};
#pragma unroll 8
        for (int s = 0; s < slices; ++s) {
          const f4 u0 = *(const f4 *)(p + (int64_t)s * b.M * b.rank), u1 = *(const f4 *)(p + (int64_t)s * b.M * b.rank + 4);
#pragma unroll
          for (int i = 0; i < 4; ++i) s0[i] += u0[i], s1[i] += u1[i];
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          h[c][i] = j < b.rank ? (i < 4 ? s0[i & 3] : s1[i & 3]) : 0.f;
          most = fmaxf(most, fabsf(h[c][i]));
        }
      }
      most = fmaxf(most, __shfl_xor(most, 16, 64));
      most = fmaxf(most, __shfl_xor(most, 32, 64));
      const int e = min(max((int)(__builtin_bit_cast(uint32_t, most) >> 23) - 127, -126), 126);
      const float down = __builtin_bit_cast(float, (uint32_t)(127 - e) << 23);
      back = __builtin_bit_cast(float, (uint32_t)(127 + e) << 23);
#pragma unroll
      for (int c = 0; c < RC; ++c)
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const float v = h[c][i] * down;
          hi[c][i] = (_Float16)v;
          lo[c][i] = fabsf(v) < 4.f ? (_Float16)(v - (float)hi[c][i]) : (_Float16)0.f;      // (infinite or NaN: as it is)
        }
    }
#pragma unroll
    for (int t = 0; t < TILES; ++t) {
      const int at = row0 + 16 * t + 4 * g4;
      f4 acc = {0, 0, 0, 0};
      if (some) {
#pragma unroll
        for (int c = 0; c < RC; ++c) {
          const u4 v = 32 * c + 8 * g4 < b.rank ? w[t][c] : u4{0, 0, 0, 0};
          acc = __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(h8, v), hi[c], acc, 0, 0, 0);
          acc = __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(h8, v), lo[c], acc, 0, 0, 0);
        }
      }
      // lane (g, n): rows `at` .. + 3 of token n
      if (mine && at < b.rows) {
#pragma unroll
        for (int i = 0; i < 4; ++i) y[t][i] = some ? y[t][i] + (acc[i] * scale) * back : a < 0 ? y[t][i] : __builtin_nanf("");
        put4(b.Y + m * b.ldy + at, b.rows - at, y8, y[t]);
      }
    }
  }
}

template <int RC>
hipError_t launch_expand(const egt_lora_batch &b, const float *part, int slices, hipStream_t stream) {
  // row tiles a wave: more where there are plenty of rows if every token has an adapter of its own (the workgroups of tokens that
  // another one speaks for are launched too)
  const int64_t groups = (int64_t)((b.rows + 63) / 64) * std::min(b.M, b.adapters);
  if constexpr (RC < 4)
    if (groups >= 4096) return launch(k_lora_expand<RC, 8>, dim3((b.rows + 511) / 512, b.M), dim3(256), 0, stream, b, part, slices);
  if (groups >= 2048) return launch(k_lora_expand<RC, 4>, dim3((b.rows + 255) / 256, b.M), dim3(256), 0, stream, b, part, slices);
  return launch(k_lora_expand<RC, 1>, dim3((b.rows + 63) / 64, b.M), dim3(256), 0, stream, b, part, slices);
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
  if (b->rows > 1 << 30) return EGT_ERR_UNSUPPORTED;
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
