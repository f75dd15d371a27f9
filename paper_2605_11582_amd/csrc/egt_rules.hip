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

// 16 bytes at any address that suits a logit
typedef u4 __attribute__((aligned(2))) loose_u4;

__device__ __forceinline__ float wide(__half v) { return (float)v; }
__device__ __forceinline__ float wide(float v) { return v; }
__device__ __forceinline__ void narrow(__half &o, float v) { o = __float2half(v); }
__device__ __forceinline__ void narrow(float &o, float v) { o = v; }

// 8 logits as they lie in memory
template <typename T>
struct Eight {
  static constexpr int N = sizeof(T) / 2;
  u4 w[N];
  __device__ __forceinline__ void load(const T *p) {
#pragma unroll
    for (int i = 0; i < N; ++i) w[i] = *(const loose_u4 *)((const uint8_t *)p + 16 * i);
  }
  __device__ __forceinline__ void store(T *p) const {
#pragma unroll
    for (int i = 0; i < N; ++i) *(loose_u4 *)((uint8_t *)p + 16 * i) = w[i];
  }
  __device__ __forceinline__ float get(int e) const {
    if constexpr (sizeof(T) == 4) {
      const uint32_t x = w[e >> 2][e & 3];
      return __builtin_bit_cast(float, x);
    } else {
      const uint32_t x = w[0][e >> 1];
      return (float)__builtin_bit_cast(_Float16, (uint16_t)(x >> 16 * (e & 1)));
    }
  }
  __device__ __forceinline__ void put(int e, float v) {
    if constexpr (sizeof(T) == 4) {
      w[e >> 2][e & 3] = __builtin_bit_cast(uint32_t, v);
    } else {
      const uint32_t x = __builtin_bit_cast(uint16_t, (_Float16)v);
      w[0][e >> 1] = e & 1 ? (w[0][e >> 1] & 0xffffu) | x << 16 : (w[0][e >> 1] & 0xffff0000u) | x;
    }
  }
};

// The request of a row: the last one that starts at the row or before; -1 where the row is nobody's.  All lanes look at once,
// 64 places a round; the first round's places, `mine` (64 or fewer requests: all there are), and the end of the last request are at hand.
struct Found { int r, t0, t1; };
__device__ __forceinline__ Found request_of(const int32_t *cu, int mine, int last, int n, int rows, int row) {
  const int lane = threadIdx.x & 63;
  int lo = 0, step = (n + 63) / 64;
  Found f = {-1, 0, 0};
  const uint64_t before = __ballot(lane * step < n && mine <= row);
  if (!before) return f;
  const int k = 63 - __builtin_clzll(before);
  if (step == 1) {
    lo = k;
    f.t0 = __builtin_amdgcn_readlane(mine, k);
    f.t1 = k + 1 < n ? __builtin_amdgcn_readlane(mine, k + 1) : last;
  } else {
    lo = k * step;
    n = min(step, n - lo);
    while (n > 1) {
      step = (n + 63) / 64;
      const uint64_t here = __ballot(lane * step < n && cu[lo + min(lane * step, n - 1)] <= row);      // (lane 0 says so: it did in the round before)
      const int j = here ? 63 - __builtin_clzll(here) : 0;
      lo += j * step;
      n = min(step, n - j * step);
    }
    f.t0 = cu[lo];
    f.t1 = cu[lo + 1];
  }
  if (f.t0 >= 0 && f.t0 <= row && row < f.t1 && f.t1 <= rows) f.r = lo;
  return f;
}

// What a request has the rules say.
struct Rules { float repetition, back, frequency, presence; };      // back: 1 / repetition (a quotient is a product with it: one rounding more)
// The penalties, in their order, of an id with the counter `n`; `bias` is the list's, where it names the id.
__device__ __forceinline__ float ruled(const Rules &u, float x, uint32_t n, float bias) {
  const float f = (float)(n & COUNT);
  const float y = n & ~NAMED ? x * (x > 0.f ? u.back : u.repetition) : x;
  const float z = (y - u.frequency * f) - u.presence, w = n & COUNT ? z : y;
  return n & NAMED ? w + bias : w;
}

// Loads that do not depend on each other are asked for together, also where a rule is left out or a place is not there (then from
// a place that is): a branch around a load, or a look at one, would wait for all that were asked for before.
template <typename T, int SLICE>
__global__ __launch_bounds__(256) void k_logits_rules(egt_rules_batch b, int rows_each) {
  // a wave takes a quarter of the slice: VL times 8 ids a lane
  constexpr int PART = SLICE / 4, VL = PART / 512 > 0 ? PART / 512 : 1;
  __shared__ uint32_t count[SLICE], named[SLICE];     // a counter for each id; one more than the last entry of the bias list that names it, then its bias
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int first = blockIdx.x * SLICE, ids = min(SLICE, b.vocab - first), row0 = blockIdx.y * rows_each, stop = min(row0 + rows_each, b.tokens);
  // (nothing where from >= to); whole pieces of 8 ids, and the ids behind them, one a lane
  const int from = wave * PART, to = min(from + PART, ids), wholes = max(to - from, 0) / 8, rest = from < to ? (to - from) % 8 : 0;

  // rows_each <= 64: a lane has what is said of one row
  const int last = b.cu_tokens[b.requests], step = (b.requests + 63) / 64, cu = b.cu_tokens[min(lane * step, b.requests)];
  const int own = min(row0 + lane, stop - 1);
  const int which_all = (b.allowed ? b.allowed_row : b.cu_tokens)[b.allowed ? own : 0];
  const uint64_t seen_all = b.draft ? b.mask[own] : 0;
  if (row0 >= last) return;                           // (rows behind the last request)

  // What is there of a row before anything is known of its request: its logits, and what its grammar allows.
  struct Row { Eight<T> v[VL]; uint32_t bits[VL], rest_bits; T rest; int which; };
  auto fetch = [&](int row) {
    Row w;
    const int i = min(row, stop - 1);
    const T *x = (const T *)b.logits + i * b.ld_logits + first;
    if (wholes) {
#pragma unroll
      for (int q = 0; q < VL; ++q) w.v[q].load(x + from + 8 * min(64 * q + lane, wholes - 1));
    }
    if (rest) w.rest = x[to - rest + min(lane, rest - 1)];
    const int which = __builtin_amdgcn_readlane(which_all, i - row0);
    w.which = b.allowed ? which : -1;
    const bool some = w.which >= 0 && w.which < b.n_allowed;
    const uint32_t *allowed = some ? b.allowed + which * b.ld_allowed + first / 32 : (const uint32_t *)b.cu_tokens;
#pragma unroll
    for (int q = 0; q < VL; ++q) w.bits[q] = allowed[some ? min(from + 512 * q + 8 * lane, ids - 1) >> 5 : 0];
    w.rest_bits = allowed[some ? (ids - 1) >> 5 : 0];
    return w;
  };

  int r = -1, end = row0, draft = -1;                 // the request at hand ends before row `end`
  Rules u;
  auto turn_to = [&](int row) {
    __syncthreads();                                  // (the counters of the last request are read no more)
    const Found f = request_of(b.cu_tokens, cu, last, b.requests, b.tokens, row);
    r = f.r;
    end = row + 1;
    if (r < 0) return;
    end = f.t1;
    const int mates = min(end - f.t0, 64);
    const float *none = (const float *)b.cu_tokens;   // (a place to read where a rule is left out)
    const float repetition = *(b.repetition ? b.repetition + r : none), frequency = *(b.frequency ? b.frequency + r : none), presence = *(b.presence ? b.presence + r : none);
    const int length = *(b.history ? b.history_len + r : b.cu_tokens), prompt = *(b.history && b.prompt_len ? b.prompt_len + r : b.cu_tokens);
    const int drafted = *(b.draft ? b.draft + f.t0 + min(lane, mates - 1) : b.cu_tokens);
    const int32_t *h = b.history ? b.history + r * b.ld_history : nullptr, *bias_ids = b.bias_ids ? b.bias_ids + (int64_t)r * b.n_bias : nullptr;
    const float *bias = b.bias_ids ? b.bias + (int64_t)r * b.n_bias : nullptr;
    // the history, 4096 ids at a time: four a thread in a piece of 16 bytes, the first ones before its length is known
    const int pieces = b.history && ((uintptr_t)h & 15) == 0 ? b.history_width / 4 : 0;
    int4 v[4];
    auto ask = [&](int p0) {
#pragma unroll
      for (int j = 0; j < 4; ++j) v[j] = *(const int4 *)(h + 4 * (int64_t)min(p0 + 256 * j + tid, pieces - 1));
    };
    if (pieces) ask(0);
    for (int t = 4 * tid; t < SLICE; t += 1024) {
      *(uint4 *)(count + t) = uint4{0, 0, 0, 0};
      if (b.bias_ids) *(uint4 *)(named + t) = uint4{0, 0, 0, 0};
    }
    u.repetition = b.repetition ? repetition : 1.f;
    u.back = b.repetition ? 1.f / repetition : 1.f;
    u.frequency = b.frequency ? frequency : 0.f;
    u.presence = b.presence ? presence : 0.f;
    draft = b.draft && lane < mates ? drafted : -1;   // the drafted token that this lane stands for
    const int n = b.history ? min(max(length, 0), b.history_width) : 0, told = b.history && b.prompt_len ? min(max(prompt, 0), n) : 0;
    lds_barrier();
    auto take = [&](int i, int id) {
      const uint32_t t = (uint32_t)id - (uint32_t)first;
      if (i < n && t < (uint32_t)ids) {
        if (i < told) atomicOr(&count[t], PROMPT); else atomicAdd(&count[t], 1u);
      }
    };
    for (int p0 = 0; p0 < pieces && 4 * p0 < n; p0 += 1024) {
      if (p0) ask(p0);
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const int p = p0 + 256 * j + tid;
        if (p < pieces) take(4 * p, v[j].x), take(4 * p + 1, v[j].y), take(4 * p + 2, v[j].z), take(4 * p + 3, v[j].w);
      }
    }
    for (int i = 4 * pieces + tid; i < n; i += 256) take(i, h[i]);
    if (b.bias_ids) {
      for (int i = tid; i < b.n_bias; i += 256) {
        const uint32_t t = (uint32_t)bias_ids[i] - (uint32_t)first;
        if (t < (uint32_t)ids) {
          atomicOr(&count[t], NAMED);
          atomicMax(&named[t], (uint32_t)i + 1);
        }
      }
    }
    lds_barrier();
    if (b.bias_ids) {                                 // every lane puts the biases of its own ids in the place of their numbers
#pragma unroll
      for (int q = 0; q < VL; ++q) {
        const int t = from + 512 * q + 8 * lane;
        if (t >= to) continue;
        uint32_t any = 0, c[8], value[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) any |= c[e] = named[t + e];      // (ids past the slice's last are in no list)
        if (!any) continue;
#pragma unroll
        for (int e = 0; e < 8; ++e) value[e] = ((const uint32_t *)bias)[c[e] ? c[e] - 1 : 0];
#pragma unroll
        for (int e = 0; e < 8; ++e) named[t + e] = c[e] ? value[e] : 0;
      }
    }
  };
  auto bias_of = [&](int t) { return __builtin_bit_cast(float, named[t]); };
  auto pass = [&](int row, Row &w) {
    if (row >= stop) return;
    if (row >= end) turn_to(row);
    if (r < 0 || from >= to) return;
    const T *x = (const T *)b.logits + row * b.ld_logits + first;
    T *y = (T *)b.out + row * b.ld_out + first;
    const bool broken = w.which >= b.n_allowed && b.allowed, some_allowed = w.which >= 0;
    // the ids of drafted tokens that this row sees, again, by the lanes that stand for them: read before the pass, which may
    // be in place
    const uint32_t seen_lo = (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)seen_all, row - row0);
    const uint32_t seen_hi = (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)(seen_all >> 32), row - row0);
    const bool seen = draft >= first + from && draft < first + to && ((lane < 32 ? seen_lo : seen_hi) >> (lane & 31) & 1);
    const uint64_t some = __ballot(seen);
    float again = 0.f;
    if (some) {
      uint32_t times = 0;
      for (uint64_t left = some; left; left &= left - 1) times += __builtin_amdgcn_readlane(draft, __builtin_ctzll(left)) == draft;
      if (seen) {
        const int t = draft - first;
        again = ruled(u, wide(x[t]), count[t] + times, b.bias_ids ? bias_of(t) : 0.f);
        if (broken) again = __builtin_nanf("");
        else if (some_allowed && !(b.allowed[w.which * b.ld_allowed + (draft >> 5)] >> (draft & 31) & 1)) again = -INFINITY;
      }
    }
#pragma unroll
    for (int q = 0; q < VL; ++q) {
      const int t = from + 512 * q + 8 * lane;
      if (64 * q + lane >= wholes) continue;
      const uint4 c0 = *(const uint4 *)(count + t), c1 = *(const uint4 *)(count + t + 4);
      const uint32_t c[8] = {c0.x, c0.y, c0.z, c0.w, c1.x, c1.y, c1.z, c1.w}, any = (c0.x | c0.y | c0.z | c0.w) | (c1.x | c1.y | c1.z | c1.w);
      if (any) {
        float add[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
        if (any & NAMED) {
#pragma unroll
          for (int e = 0; e < 8; ++e) add[e] = bias_of(t + e);
        }
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const float z = ruled(u, w.v[q].get(e), c[e], add[e]);
          if (c[e]) w.v[q].put(e, z);                 // (ids that nothing is said of stay as they are)
        }
      }
      const uint32_t bits = broken ? 0u : some_allowed ? w.bits[q] >> (t & 31) : ~0u;
      const float instead = broken ? __builtin_nanf("") : -INFINITY;
#pragma unroll
      for (int e = 0; e < 8; ++e)
        if (!(bits >> e & 1)) w.v[q].put(e, instead);
      w.v[q].store(y + t);
    }
    if (lane < rest) {
      const int t = to - rest + lane;
      T z = w.rest;
      if (count[t]) narrow(z, ruled(u, wide(z), count[t], b.bias_ids ? bias_of(t) : 0.f));
      if (broken) narrow(z, __builtin_nanf(""));
      else if (some_allowed && !(w.rest_bits >> (t & 31) & 1)) narrow(z, -INFINITY);
      y[t] = z;
    }
    if (some) {
      wait_vmem<0>();                                 // (the pass has written these ids too)
      if (seen) narrow(y[draft - first], again);      // (tokens of one id write the same number)
    }
  };
  // (one row's logits are on their way while the other is done; in place, no row is another's)
  Row even = fetch(row0);
  for (int row = row0; row < stop; row += 2) {
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
      !b->allowed != !b->allowed_row)
    return EGT_ERR_NULL;
  const uintptr_t size = b->kind == EGT_LOGITS_FP16 ? 1 : 3;
  if (((uintptr_t)b->logits & size) || ((uintptr_t)b->out & size) || ((uintptr_t)b->mask & 7)) return EGT_ERR_BUFFER;
  for (const void *p : {(const void *)b->cu_tokens, (const void *)b->history, (const void *)b->history_len, (const void *)b->prompt_len, (const void *)b->draft,
                        (const void *)b->repetition, (const void *)b->frequency, (const void *)b->presence, (const void *)b->bias_ids, (const void *)b->bias,
                        (const void *)b->allowed, (const void *)b->allowed_row})
    if ((uintptr_t)p & 3) return EGT_ERR_BUFFER;
  // Slices of 4096 ids count a history in fewer workgroups; where rows are few, slices of 1024 have the whole chip at work (us, slices of
  // 1024 against 4096, FP16, histories of 2048 ids, a token a request: 128 workgroups of 4096 ids 6.3 / 6.8, 256 7.9 / 7.0,
  // 512 12.3 / 7.8, 1024 21.0 / 10.4; FP32 6.7 / 7.0, 8.1 / 7.2, 13.0 / 9.0, 23.0 / 14.8).  Rows of one request share a count: as many
  // together as a request has on average, as long as there are 2048 workgroups (us with 1024, 2048 and 4096: sixteen requests, 72 of 128
  // rows used, 128000 ids 20.6, 19.9, 21.7; all 128 rows 22.3, 24.8, 31.6; 512 rows of eight requests 77, 75, 80; 256 rows of 64
  // requests, 32003 ids 16.7, 20.2, 20.1).
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
