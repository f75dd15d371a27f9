// Penalties for repeated tokens, biases and grammar masks on logits.
//
// One pass over the logits; what makes it more than a copy is that a row's history says something about a few thousand of a hundred
// thousand ids.  A workgroup takes a slice of the vocabulary and some rows: for every request among them it counts the history's ids that
// fall into the slice in LDS - whole numbers, so that the order of the atomics does not show - and its waves then pass over the
// rows, 8 ids a lane, each with its count at hand, the next row's logits on their way.  The drafted tokens that a row sees differ
// from row to row: their ids, few in a slice, are done again after the pass by the lanes that stand for them.  Bound by the logits' bytes, and for a single row by a
// launch and the chain cu_tokens - lengths - history - logits.
#include "egt_mfma_common.h"
#include "egt_serve.h"

#include <algorithm>

namespace egt {
namespace {

// A counter: how often the id is written, whether it is in the prompt, whether a bias names it.
constexpr uint32_t PROMPT = 1u << 31, NAMED = 1u << 30, COUNT = NAMED - 1;

// 8 logits, at any address that suits one
template <typename T>
struct __attribute__((packed, aligned(sizeof(T)))) Eight { T v[8]; };

__device__ __forceinline__ float wide(__half v) { return (float)v; }
__device__ __forceinline__ float wide(float v) { return v; }
__device__ __forceinline__ void narrow(__half &o, float v) { o = __float2half(v); }
__device__ __forceinline__ void narrow(float &o, float v) { o = v; }

// The request of a row: the last one that starts at the row or before; -1 where the row is nobody's.  All lanes look at once,
// 64 places a round.
__device__ __forceinline__ int request_of(const int32_t *cu, int n, int rows, int row) {
  const int lane = threadIdx.x & 63;
  int lo = 0;
  while (n > 1) {
    const int step = (n + 63) / 64, at = lane * step;
    const uint64_t before = __ballot(at < n && cu[lo + min(at, n - 1)] <= row);
    if (!before) return -1;
    const int k = 63 - __builtin_clzll(before);
    lo += k * step;
    n = min(step, n - k * step);
  }
  const int t0 = cu[lo], t1 = cu[lo + 1];
  return t0 >= 0 && t0 <= row && row < t1 && t1 <= rows ? lo : -1;
}

// What a request has the rules say.
struct Rules {
  float repetition, back, frequency, presence;        // back: 1 / repetition (a quotient is a product with it: one rounding more)
  const int32_t *bias_ids;
  const float *bias;
  int n_bias;
};
// The penalties, in their order, of an id with the counter `n`.
__device__ __forceinline__ float penalised(const Rules &u, float x, uint32_t n) {
  const float f = (float)(n & COUNT);
  float y = n & ~NAMED ? x * (x > 0.f ? u.back : u.repetition) : x;
  const float z = (y - u.frequency * f) - u.presence;
  return n & COUNT ? z : y;
}
template <typename T, int SLICE>
__global__ __launch_bounds__(256) void k_logits_rules(egt_rules_batch b, int rows_each) {
  // a wave takes a quarter of the slice: VL times 8 ids a lane
  constexpr int PART = SLICE / 4, VL = PART / 512 > 0 ? PART / 512 : 1;
  __shared__ uint32_t count[SLICE], named[SLICE];     // a counter for each id; one more than the last entry of the bias list that names it
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int first = blockIdx.x * SLICE, ids = min(SLICE, b.vocab - first), stop = min((int)(blockIdx.y + 1) * rows_each, b.tokens);
  const int from = wave * PART, to = min(from + PART, ids);      // (nothing where from >= to)

  // What is there of a row before anything is known of its request: its logits, and what its grammar allows.
  struct Row { Eight<T> v[VL]; uint32_t bits[VL]; bool broken; };
  auto fetch = [&](int row) {
    Row w;
    const int i = min(row, stop - 1);
    const int which = b.allowed ? b.allowed_row[i] : -1;
    w.broken = b.allowed && which >= b.n_allowed;
    const uint32_t *allowed = which >= 0 && !w.broken ? b.allowed + which * b.ld_allowed + first / 32 : nullptr;
    const T *x = (const T *)b.logits + i * b.ld_logits + first;
#pragma unroll
    for (int q = 0; q < VL; ++q) {
      const int t = from + 512 * q + 8 * lane;
      w.bits[q] = ~0u;
      if (t < to) {
        if (allowed) w.bits[q] = allowed[t >> 5];
        if (t + 8 <= to) {
          w.v[q] = *(const Eight<T> *)(x + t);
        } else {
#pragma unroll
          for (int e = 0; e < 8; ++e)
            if (t + e < to) w.v[q].v[e] = x[t + e];
        }
      }
    }
    return w;
  };

  int r = -1, t0 = 0, end = blockIdx.y * rows_each, draft = -1;      // the request at hand ends before row `end`
  Rules u;
  auto turn_to = [&](int row) {
    __syncthreads();                                  // (the counters of the last request are read no more)
    r = request_of(b.cu_tokens, b.requests, b.tokens, row);
    end = row + 1;
    if (r < 0) return;
    t0 = b.cu_tokens[r];
    end = b.cu_tokens[r + 1];
    const int mates = min(end - t0, 64);
    for (int t = 4 * tid; t < SLICE; t += 1024) {
      *(uint4 *)(count + t) = uint4{0, 0, 0, 0};
      if (b.bias_ids) *(uint4 *)(named + t) = uint4{0, 0, 0, 0};
    }
    u.bias_ids = b.bias_ids ? b.bias_ids + (int64_t)r * b.n_bias : nullptr;
    u.bias = b.bias_ids ? b.bias + (int64_t)r * b.n_bias : nullptr;
    u.n_bias = b.bias_ids ? b.n_bias : 0;
    u.repetition = b.repetition ? b.repetition[r] : 1.f;
    u.back = b.repetition ? 1.f / u.repetition : 1.f;
    u.frequency = b.frequency ? b.frequency[r] : 0.f;
    u.presence = b.presence ? b.presence[r] : 0.f;
    draft = b.draft && lane < mates ? b.draft[t0 + lane] : -1;      // the drafted token that this lane stands for
    __syncthreads();
    if (b.history) {
      const int32_t *h = b.history + r * b.ld_history;
      const int n = min(max(b.history_len[r], 0), b.history_width), told = b.prompt_len ? min(max(b.prompt_len[r], 0), n) : 0;
      auto take = [&](int i, int id) {
        const uint32_t t = (uint32_t)id - (uint32_t)first;
        if (t < (uint32_t)ids) {
          if (i < told) atomicOr(&count[t], PROMPT); else atomicAdd(&count[t], 1u);
        }
      };
      const int whole = ((uintptr_t)h & 15) == 0 ? n & ~3 : 0;
#pragma unroll 4
      for (int i = 4 * tid; i < whole; i += 1024) {
        const int4 v = *(const int4 *)(h + i);
        take(i, v.x), take(i + 1, v.y), take(i + 2, v.z), take(i + 3, v.w);
      }
      for (int i = whole + tid; i < n; i += 256) take(i, h[i]);
    }
    for (int i = tid; i < u.n_bias; i += 256) {
      const uint32_t t = (uint32_t)u.bias_ids[i] - (uint32_t)first;
      if (t < (uint32_t)ids) {
        atomicOr(&count[t], NAMED);
        atomicMax(&named[t], (uint32_t)i + 1);
      }
    }
    __syncthreads();
  };
  auto pass = [&](int row, Row &w) {
    if (row >= stop) return;
    if (row >= end) turn_to(row);
    if (r < 0 || from >= to) return;
    const T *x = (const T *)b.logits + row * b.ld_logits + first;
    T *y = (T *)b.out + row * b.ld_out + first;
    // the ids of drafted tokens that this row sees, again, by the lanes that stand for them: read before the pass, which may
    // be in place
    const bool seen = draft >= first + from && draft < first + to && (b.mask[row] >> lane & 1);
    const uint64_t some = __ballot(seen);
    float again = 0.f;
    if (some) {
      uint32_t times = 0;
      for (uint64_t left = some; left; left &= left - 1) times += __builtin_amdgcn_readlane(draft, __builtin_ctzll(left)) == draft;
      if (seen) {
        const int t = draft - first;
        const uint32_t n = count[t] + times;
        again = penalised(u, wide(x[t]), n);
        if (n & NAMED) again = again + u.bias[named[t] - 1];
        const int which = b.allowed ? b.allowed_row[row] : -1;
        if (w.broken) again = __builtin_nanf("");
        else if (which >= 0 && !(b.allowed[which * b.ld_allowed + (draft >> 5)] >> (draft & 31) & 1)) again = -INFINITY;
      }
    }
#pragma unroll
    for (int q = 0; q < VL; ++q) {
      const int t = from + 512 * q + 8 * lane;
      if (t >= to) continue;
      const uint4 c0 = *(const uint4 *)(count + t), c1 = *(const uint4 *)(count + t + 4);
      const uint32_t c[8] = {c0.x, c0.y, c0.z, c0.w, c1.x, c1.y, c1.z, c1.w}, any = (c0.x | c0.y | c0.z | c0.w) | (c1.x | c1.y | c1.z | c1.w);
      if (any) {
        float z[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) z[e] = penalised(u, wide(w.v[q].v[e]), c[e]);
        if (any & NAMED) {
#pragma unroll
          for (int e = 0; e < 8; ++e)
            if (c[e] & NAMED) z[e] = z[e] + u.bias[named[t + e] - 1];
        }
#pragma unroll
        for (int e = 0; e < 8; ++e)
          if (c[e]) narrow(w.v[q].v[e], z[e]);        // (ids that nothing is said of stay as they are)
      }
      const uint32_t bits = w.bits[q] >> (t & 31);
#pragma unroll
      for (int e = 0; e < 8; ++e)
        if (w.broken || !(bits >> e & 1)) narrow(w.v[q].v[e], w.broken ? __builtin_nanf("") : -INFINITY);
      if (t + 8 <= to) {
        *(Eight<T> *)(y + t) = w.v[q];
      } else {
#pragma unroll
        for (int e = 0; e < 8; ++e)
          if (t + e < to) y[t + e] = w.v[q].v[e];
      }
    }
    if (some) {
      wait_vmem<0>();                                 // (the pass has written these ids too)
      if (seen) narrow(y[draft - first], again);      // (tokens of one id write the same number)
    }
  };
  if (end >= b.cu_tokens[b.requests]) return;         // (rows behind the last request)
  // (one row's logits are on their way while the other is done; in place, no row is another's)
  Row even = fetch(end);
  for (int row = end; row < stop; row += 2) {
    Row odd = fetch(row + 1);
    pass(row, even);
    if (row + 2 < stop) even = fetch(row + 2);
    pass(row + 1, odd);
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
  if (b->requests > EGT_MAX_REQUESTS || b->tokens > 65535 || b->vocab > (1 << 30) || b->history_width > (1 << 29) || b->n_bias > (1 << 29)) return EGT_ERR_UNSUPPORTED;
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
  // Slices of 4096 ids count a history in fewer workgroups; where rows are few, slices of 1024 have the whole chip at work.  Rows of one
  // request share a count: as many together as a request has on average, as long as there are 2048 workgroups (128 rows of
  // 128000 ids, 72 of them used: 1024 workgroups 23.5 us, 2048 19.8, 4096 26.3; slices of 2048 21.2; of 8192 with 8 waves 22.5).
  const bool large = (int64_t)b->tokens * ((b->vocab + 4095) / 4096) >= 512;
  const int slices = large ? (b->vocab + 4095) / 4096 : (b->vocab + 1023) / 1024;
  const int64_t each = std::min<int64_t>((int64_t)b->tokens * slices / 2048, (b->tokens + b->requests - 1) / b->requests);
  const int rows_each = (int)std::min<int64_t>(std::max<int64_t>(each, 1), 64);
  const dim3 grid((unsigned)slices, (unsigned)((b->tokens + rows_each - 1) / rows_each)), block(256);
  const hipStream_t to = (hipStream_t)stream;
  if (b->kind == EGT_LOGITS_FP16)
    return egt::answer(large ? egt::launch(egt::k_logits_rules<__half, 4096>, grid, block, 0, to, *b, rows_each)
                             : egt::launch(egt::k_logits_rules<__half, 1024>, grid, block, 0, to, *b, rows_each));
  return egt::answer(large ? egt::launch(egt::k_logits_rules<float, 4096>, grid, block, 0, to, *b, rows_each)
                           : egt::launch(egt::k_logits_rules<float, 1024>, grid, block, 0, to, *b, rows_each));
}

}  // extern "C"
