// Attention of drafted trees over a paged cache.
#include "egt_serve.h"

namespace egt {
namespace {

// One workgroup of four waves a (token, head): a wave takes 64 keys at a time, a lane one of them.
__global__ __launch_bounds__(256) void k_tree_simple(egt_tree_batch b, egt_kv_cache c, int shift) {
  __shared__ float q[256], w[4][64], o[4][256], ml[4][2];
  const int r = blockIdx.z, h = blockIdx.y, kh = h / (b.heads / c.heads), tid = threadIdx.x, wave = tid >> 6, lane = tid & 63;
  const int t0 = b.cu_tokens[r], t1 = b.cu_tokens[r + 1], i = t0 + blockIdx.x;
  if (t0 < 0 || t1 > b.tokens || i >= t1) return;
  __half *out = (__half *)b.out + i * b.out_row + h * b.out_head;
  const int len = b.lens[r], n = t1 - t0;
  bool bad = n > b.max_tokens || len < 0 || len > (int64_t)b.table_blocks << shift;
  if (bad) {
    if (tid < c.dim) out[tid] = __float2half(__builtin_nanf(""));
    if (n > b.max_tokens && blockIdx.x == 0)          // (the rows that the grid does not reach)
      for (int j = b.max_tokens; j < n; ++j)
        if (tid < c.dim) ((__half *)b.out + (int64_t)(t0 + j) * b.out_row + h * b.out_head)[tid] = __float2half(__builtin_nanf(""));
    return;
  }
  if (tid < c.dim) q[tid] = (float)((const __half *)b.q)[i * b.q_row + h * b.q_head + tid] * b.scale;
  __syncthreads();
  const uint64_t mask = b.mask[i];
  float m = -INFINITY, l = 0.f, acc[4] = {0.f, 0.f, 0.f, 0.f};
  for (int k0 = 64 * wave; k0 < len + n; k0 += 256) {
    const int j = k0 + lane;
    bool seen = false;
    const __half *kp = nullptr;
    if (j < len) {
      const int block = b.block_table[(int64_t)r * b.ld_table + (j >> shift)];
      seen = block >= 0 && block < c.blocks;
      bad |= !seen;
      kp = (const __half *)c.k + block * c.k_block + kh * c.k_head + (j & ((1 << shift) - 1)) * c.k_token;
    } else if (j < len + n) {
      seen = mask >> (j - len) & 1;
      kp = (const __half *)b.k + (int64_t)(t0 + j - len) * b.k_row + kh * b.k_head;
    }
    float s = -INFINITY;
    if (seen) {
      s = 0.f;
      for (int d = 0; d < c.dim; ++d) s = fmaf(q[d], (float)kp[d], s);
    }
    // (a NaN score has to stay one: fmaxf would drop it)
    float top = s;
    for (int x = 32; x > 0; x >>= 1) top = fmaxf(top, __shfl_xor(top, x, 64));
    const float mn = fmaxf(m, top), ref = mn == -INFINITY ? 0.f : mn, f = m == -INFINITY ? 0.f : expf(m - ref);
    const float p = seen ? expf(s - ref) : 0.f;
    float sum = p;
    for (int x = 32; x > 0; x >>= 1) sum += __shfl_xor(sum, x, 64);
    l = l * f + sum;
    m = mn;
    w[wave][lane] = p;
    const uint64_t on = __ballot(seen);
    for (int x = 0; x < 4; ++x) acc[x] *= f;
    for (int x = 0; x < 64; ++x) {
      if (!(on >> x & 1)) continue;
      const int y = k0 + x;
      const __half *vp;
      if (y < len)
        vp = (const __half *)c.v + b.block_table[(int64_t)r * b.ld_table + (y >> shift)] * c.v_block + kh * c.v_head + (y & ((1 << shift) - 1)) * c.v_token;
      else
        vp = (const __half *)b.v + (int64_t)(t0 + y - len) * b.v_row + kh * b.v_head;
      for (int e = 0; e < 4; ++e)
        if (lane + 64 * e < c.dim) acc[e] = fmaf(w[wave][x], (float)vp[lane + 64 * e], acc[e]);
    }
  }
  if (lane == 0) { ml[wave][0] = m; ml[wave][1] = l; }
  for (int e = 0; e < 4; ++e) o[wave][lane + 64 * e] = acc[e];
  bad = __syncthreads_or(bad);
  float top = -INFINITY, total = 0.f, v = 0.f;
  for (int x = 0; x < 4; ++x) top = fmaxf(top, ml[x][0]);
  for (int x = 0; x < 4; ++x) {
    const float f = ml[x][0] == -INFINITY ? (ml[x][1] == 0.f ? 0.f : 1.f) : expf(ml[x][0] - top);
    total += f * ml[x][1];
    v += f * o[x][tid & 255];
  }
  if (tid < c.dim) out[tid] = __float2half(bad ? __builtin_nanf("") : total == 0.f ? 0.f : v / total);
}

egt_status check_sizes(const egt_tree_batch *b, const egt_kv_cache *c) {
  if (!b) return EGT_ERR_NULL;
  const egt_status st = check_cache(c, false);
  if (st != EGT_OK) return st;
  if (b->requests < 0 || b->tokens < 0 || b->heads < 1 || b->heads % c->heads != 0 || b->max_tokens < 1 || b->max_tokens > EGT_MAX_TREE || b->table_blocks < 0 ||
      (int64_t)b->table_blocks * c->page >= (1ll << 31))
    return EGT_ERR_SHAPE;
  return b->requests > EGT_MAX_REQUESTS || b->heads > 65535 ? EGT_ERR_UNSUPPORTED : EGT_OK;
}
size_t workspace_of(const egt_tree_batch *, const egt_kv_cache *) { return 16; }

}  // namespace
}  // namespace egt

extern "C" {

egt_status egt_tree_attention_ws_bytes(const egt_tree_batch *b, const egt_kv_cache *cache, size_t *bytes) {
  if (!bytes) return EGT_ERR_NULL;
  const egt_status st = egt::check_sizes(b, cache);
  if (st == EGT_OK) *bytes = egt::workspace_of(b, cache);
  return st;
}

egt_status egt_tree_attention(const egt_tree_batch *b, const egt_kv_cache *cache, void *workspace, size_t workspace_bytes, void *stream) {
  egt_status st = egt::check_sizes(b, cache);
  if (st != EGT_OK) return st;
  st = egt::check_cache(cache, true);
  if (st != EGT_OK) return st;
  if (b->ld_table < b->table_blocks || !(b->scale == b->scale)) return EGT_ERR_SHAPE;
  if (b->requests == 0 || b->tokens == 0) return EGT_OK;
  if (!b->q || !b->k || !b->v || !b->out || !b->lens || !b->cu_tokens || !b->mask || (b->table_blocks && !b->block_table) || !workspace) return EGT_ERR_NULL;
  if (workspace_bytes < egt::workspace_of(b, cache)) return EGT_ERR_SHAPE;
  if (!egt::whole16(b->q) || !egt::whole16(b->k) || !egt::whole16(b->v) || !egt::whole16(b->out) || !egt::whole16(workspace) ||
      !egt::whole8(b->q_row, b->q_head, b->k_row, b->k_head, b->v_row, b->v_head, b->out_row, b->out_head) || ((uintptr_t)b->mask & 7) ||
      ((uintptr_t)b->lens & 3) || ((uintptr_t)b->cu_tokens & 3) || ((uintptr_t)b->block_table & 3))
    return EGT_ERR_BUFFER;
  return egt::answer(egt::launch(egt::k_tree_simple, dim3(b->max_tokens, b->heads, b->requests), dim3(256), 0, (hipStream_t)stream, *b, *cache,
                                 egt::log2_of(cache->page)));
}

}  // extern "C"
