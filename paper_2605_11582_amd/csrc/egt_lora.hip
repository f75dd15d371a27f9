// Low-rank adapters of many requests beside a shared projection.
#include "egt_serve.h"

namespace egt {
namespace {

constexpr int MAX_RANK = 128;

// h[m][j] = A[a][j] . x[m], a wave a row of A
__global__ __launch_bounds__(256) void k_lora_shrink(egt_lora_batch b, float *h) {
  const int m = blockIdx.x, a = b.index[m], lane = threadIdx.x & 63;
  if (a < 0 || a >= b.adapters) return;
  const __half *x = (const __half *)b.X + m * b.ldx;
  for (int j = threadIdx.x >> 6; j < b.rank; j += 4) {
    const __half *w = (const __half *)b.A + a * b.a_stride + (int64_t)j * b.cols;
    float s = 0.f;
    for (int c = lane; c < b.cols; c += 64) s = fmaf((float)w[c], (float)x[c], s);
    for (int o = 32; o > 0; o >>= 1) s += __shfl_xor(s, o, 64);
    if (lane == 0) h[m * b.rank + j] = s;
  }
}

__global__ __launch_bounds__(256) void k_lora_expand(egt_lora_batch b, const float *h) {
  const int m = blockIdx.y, a = b.index[m], r = blockIdx.x * 256 + threadIdx.x;
  if (r >= b.rows) return;
  float y = b.base ? (float)((const __half *)b.base)[m * b.ldbase + r] : 0.f;
  if (a >= b.adapters) {
    y = __builtin_nanf("");
  } else if (a >= 0) {
    const __half *w = (const __half *)b.B + a * b.b_stride + (int64_t)r * b.rank;
    float s = 0.f;
    for (int j = 0; j < b.rank; ++j) s = fmaf((float)w[j], h[m * b.rank + j], s);
    y += (b.scale ? b.scale[a] : 1.f) * s;
  }
  ((__half *)b.Y)[m * b.ldy + r] = __float2half(y);
}

egt_status check_sizes(int M, int cols, int rank) {
  if (M < 1 || M > 64 || cols < 8 || cols % 8 != 0 || rank < 8 || rank % 8 != 0) return EGT_ERR_SHAPE;
  return rank > MAX_RANK ? EGT_ERR_UNSUPPORTED : EGT_OK;
}
size_t workspace_of(int M, int, int rank) { return 4 * (size_t)M * rank; }

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
  if (b->rows == 0) return EGT_OK;                    // nothing to compute, pointers not examined
  if (!b->X || !b->A || !b->B || !b->Y || !b->index || !workspace) return EGT_ERR_NULL;
  if (workspace_bytes < egt::workspace_of(b->M, b->cols, b->rank)) return EGT_ERR_SHAPE;
  if (!egt::whole16(b->X) || !egt::whole16(b->A) || !egt::whole16(b->B) || !egt::whole16(workspace) || !egt::whole8(b->ldx, b->a_stride, b->b_stride) ||
      ((uintptr_t)b->index & 3) || ((uintptr_t)b->scale & 3))
    return EGT_ERR_BUFFER;
  hipError_t e = egt::launch(egt::k_lora_shrink, dim3(b->M), dim3(256), 0, (hipStream_t)stream, *b, (float *)workspace);
  if (e == hipSuccess) e = egt::launch(egt::k_lora_expand, dim3((b->rows + 255) / 256, b->M), dim3(256), 0, (hipStream_t)stream, *b, (const float *)workspace);
  return egt::answer(e);
}

}  // extern "C"
