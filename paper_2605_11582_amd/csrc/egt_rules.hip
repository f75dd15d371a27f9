// Penalties for repeated tokens, biases and grammar masks on logits.
#include "egt_serve.h"

namespace egt {
namespace {

constexpr int SLICE = 4096;              // ids a workgroup looks at
constexpr uint32_t PROMPT = 1u << 31;    // in a counter: the id is in the prompt

template <typename T>
__device__ __forceinline__ void put(T *p, float v);
template <>
__device__ __forceinline__ void put(float *p, float v) { *p = v; }
template <>
__device__ __forceinline__ void put(__half *p, float v) { *p = __float2half(v); }

// The request of a row: the last one that starts at the row or before; -1 where the row is nobody's.
__device__ __forceinline__ int request_of(const int32_t *cu, int n, int rows, int row) {
  int r = -1;
  for (int lo = 0, hi = n; lo < hi;) {
    const int mid = (lo + hi) >> 1;
    if (cu[mid] <= row) { r = mid; lo = mid + 1; } else { hi = mid; }
  }
  if (r < 0 || cu[r] < 0 || cu[r + 1] <= row || cu[r + 1] > rows) return -1;
  return r;
}

// A workgroup is one row and SLICE ids: it counts the row's history that falls among them in LDS - whole numbers, so that the
// order of the atomics does not show - and then passes over the logits once.
template <typename T>
__global__ __launch_bounds__(256) void k_logits_rules(egt_rules_batch b) {
  __shared__ uint32_t count[SLICE], named[SLICE];
  const int row = blockIdx.y, tid = threadIdx.x, first = blockIdx.x * SLICE, ids = min(SLICE, b.vocab - first);
  const int r = request_of(b.cu_tokens, b.requests, b.tokens, row);
  if (r < 0) return;
  for (int t = tid; t < SLICE; t += 256) count[t] = named[t] = 0;
  __syncthreads();
  if (b.history) {
    const int32_t *h = b.history + r * b.ld_history;
    const int n = min(max(b.history_len[r], 0), b.history_width), told = b.prompt_len ? min(max(b.prompt_len[r], 0), n) : 0;
    for (int i = tid; i < n; i += 256) {
      const uint32_t t = (uint32_t)(h[i] - first);
      if (t < (uint32_t)ids && h[i] >= 0) {
        if (i < told) atomicOr(&count[t], PROMPT); else atomicAdd(&count[t], 1u);
      }
    }
  }
  if (b.draft) {
    const int t0 = b.cu_tokens[r], n = min(b.cu_tokens[r + 1] - t0, 64);
    if (tid < n && (b.mask[row] >> tid & 1)) {
      const int id = b.draft[t0 + tid];
      if (id >= first && id < first + ids) atomicAdd(&count[id - first], 1u);
    }
  }
  if (b.bias_ids)
    for (int i = tid; i < b.n_bias; i += 256) {
      const int id = b.bias_ids[(int64_t)r * b.n_bias + i];
      if (id >= first && id < first + ids) atomicMax(&named[id - first], (uint32_t)i + 1);
    }
  __syncthreads();
  const float rep = b.repetition ? b.repetition[r] : 1.f, freq = b.frequency ? b.frequency[r] : 0.f, pres = b.presence ? b.presence[r] : 0.f;
  const int which = b.allowed ? b.allowed_row[row] : -1;
  const T *x = (const T *)b.logits + row * b.ld_logits + first;
  T *y = (T *)b.out + row * b.ld_out + first;
  for (int t = tid; t < ids; t += 256) {
    float v = (float)x[t];
    const uint32_t n = count[t];
    if (n && b.repetition) v = v > 0.f ? v / rep : v * rep;
    if (n & ~PROMPT) {
      v = v - freq * (float)(n & ~PROMPT);
      v = v - pres;
    }
    if (named[t]) v = v + b.bias[(int64_t)r * b.n_bias + named[t] - 1];
    if (which >= b.n_allowed && b.allowed) v = __builtin_nanf("");
    else if (which >= 0 && !(b.allowed[which * b.ld_allowed + ((first + t) >> 5)] >> ((first + t) & 31) & 1)) v = -INFINITY;
    put(y + t, v);
  }
}

}  // namespace
}  // namespace egt

extern "C" {

egt_status egt_logits_rules(const egt_rules_batch *b, void *stream) {
  if (!b) return EGT_ERR_NULL;
  if ((b->kind != EGT_LOGITS_FP16 && b->kind != EGT_LOGITS_FP32) || b->requests < 0 || b->tokens < 0 || b->vocab < 0 || b->n_bias < 0 || b->n_allowed < 0 ||
      b->ld_logits < b->vocab || b->ld_out < b->vocab || b->history_width < 0 || (b->history && b->ld_history < b->history_width) || b->ld_allowed < 0 || (b->allowed && b->ld_allowed < ((int64_t)b->vocab + 31) / 32) ||
      (b->logits == b->out && b->ld_logits != b->ld_out))
    return EGT_ERR_SHAPE;
  if (b->requests > EGT_MAX_REQUESTS || b->tokens > 65535) return EGT_ERR_UNSUPPORTED;
  if (b->requests == 0 || b->tokens == 0 || b->vocab == 0) return EGT_OK;
  if (!b->logits || !b->out || !b->cu_tokens || (b->history && !b->history_len) || (b->draft && !b->mask) || (b->bias_ids && !b->bias) ||
      (b->allowed && !b->allowed_row))
    return EGT_ERR_NULL;
  const uintptr_t size = b->kind == EGT_LOGITS_FP16 ? 1 : 3;
  if (((uintptr_t)b->logits & size) || ((uintptr_t)b->out & size) || ((uintptr_t)b->mask & 7)) return EGT_ERR_BUFFER;
  for (const void *p : {(const void *)b->cu_tokens, (const void *)b->history, (const void *)b->history_len, (const void *)b->prompt_len, (const void *)b->draft,
                        (const void *)b->repetition, (const void *)b->frequency, (const void *)b->presence, (const void *)b->bias_ids, (const void *)b->bias,
                        (const void *)b->allowed, (const void *)b->allowed_row})
    if ((uintptr_t)p & 3) return EGT_ERR_BUFFER;
  const dim3 grid((unsigned)((b->vocab + egt::SLICE - 1) / egt::SLICE), (unsigned)b->tokens);
  auto *kernel = b->kind == EGT_LOGITS_FP16 ? egt::k_logits_rules<__half> : egt::k_logits_rules<float>;
  return egt::answer(egt::launch(kernel, grid, dim3(256), 0, (hipStream_t)stream, *b));
}

}  // extern "C"
