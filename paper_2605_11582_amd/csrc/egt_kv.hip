// The cache of a verification step: block tables and slot maps from request lengths, and the rows of new
// tokens into their slots.
#include "egt_serve.h"

#include <algorithm>

namespace egt {
namespace {

constexpr int SLOT_THREADS = 256;

// Sums are held to what fits 31 bits: the order of additions does not matter to them, and a sum that is held is too large for
// anything it is compared with.
constexpr uint32_t MOST = INT32_MAX;
__device__ __forceinline__ uint32_t held(uint32_t a, uint32_t b) { return min(a + b, MOST); }

// Sum over the lanes up to this one, within a row of 16 and then across rows.
__device__ __forceinline__ uint32_t sum_upto(uint32_t v) {
  v = held(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x111, 0xf, 0xf, false));      // row_shr:1, 2, 4, 8
  v = held(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x112, 0xf, 0xf, false));
  v = held(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x114, 0xf, 0xf, false));
  v = held(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x118, 0xf, 0xf, false));
  v = held(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x142, 0xa, 0xf, false));      // row_bcast:15 into rows 1 and 3
  v = held(v, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)v, 0x143, 0xc, 0xf, false));      // row_bcast:31 into rows 2 and 3
  return v;
}
// Sum over the threads before this one, or, for one wave's requests, over its lanes: then every wave has all of them and nobody waits.
template <bool ONE>
__device__ __forceinline__ uint32_t sum_before(uint32_t v, uint32_t *part) {
  const uint32_t upto = sum_upto(v);
  uint32_t before = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)upto, 0x138, 0xf, 0xf, false);      // wave_shr:1
  if (ONE) return before;
  const int wave = threadIdx.x >> 6;
  if ((threadIdx.x & 63) == 63) part[wave] = upto;
  __syncthreads();
  uint32_t waves = 0;
  for (int w = 0; w < wave; ++w) waves = held(waves, part[w]);
  __syncthreads();                                    // (part is used again)
  return held(waves, before);
}

// Two running sums over the requests - tokens, then pages - decide everything, and a few thousand lengths are 16 KB: every
// workgroup computes both for itself (each thread a run of requests, then one scan over the threads; up to 64 requests every wave
// for itself, a lane a request, in LDS of its own) and keeps them in LDS, so that the token slots, which are the bytes, are written
// by the whole chip without a second launch and without one workgroup waiting for another.  What binds it is that chain: lengths,
// two scans, a search, a page number, behind a launch.
template <bool ONE>
__global__ __launch_bounds__(SLOT_THREADS) void k_kv_slots(egt_slots_batch b, int shift) {
  extern __shared__ int32_t lds[];
  __shared__ uint32_t part[SLOT_THREADS / 64];
  const int n = b.requests, tid = threadIdx.x;
  int32_t *cu = lds + (ONE ? (tid >> 6) * (3 * n + 1) : 0), *first = cu + n + 1, *old = first + n;
  // (first token; first free page, -1: the request gets nothing; ONE: length)
  const int per = ONE ? 1 : (n + SLOT_THREADS - 1) / SLOT_THREADS;
  const int r0 = min((ONE ? tid & 63 : tid) * per, n), r1 = min(r0 + per, n);
  const int head = *b.free_head;
  // the first requests of a thread are in registers, asked for together
  constexpr int KEEP = ONE ? 1 : 4;
  int lens[KEEP], counts[KEEP];
#pragma unroll
  for (int j = 0; j < KEEP; ++j) {
    lens[j] = b.lens[min(r0 + j, n - 1)];
    counts[j] = b.counts[min(r0 + j, n - 1)];
  }
  auto each = [&](auto f) {
#pragma unroll
    for (int j = 0; j < KEEP; ++j)
      if (r0 + j < r1) f(r0 + j, lens[j], counts[j]);
    for (int r = r0 + KEEP; r < r1; ++r) f(r, b.lens[r], b.counts[r]);
  };
  uint32_t tokens = 0, pages = 0;
  each([&](int, int, int c) { tokens = held(tokens, (uint32_t)max(c, 0)); });
  uint32_t at = sum_before<ONE>(tokens, part);
  int need0 = -1;
  each([&](int r, int64_t len, int64_t c) {
    const uint32_t end = held(at, (uint32_t)max(c, (int64_t)0));
    const bool room = len >= 0 && c >= 0 && len + c <= (int64_t)b.table_blocks << shift && end <= (uint32_t)b.n_slots && end < MOST;
    const int64_t up = (1 << shift) - 1, need = room ? ((len + c + up) >> shift) - ((len + up) >> shift) : 0;
    cu[r] = (int32_t)min(at, (uint32_t)b.n_slots);
    need0 = room ? (int32_t)need : -1;
    if (ONE) old[r] = (int32_t)len;
    else first[r] = need0;                            // (kept there until the second scan is done)
    at = end;
    pages = held(pages, (uint32_t)need);
  });
  if (r0 < r1 && r1 == n) cu[n] = (int32_t)min(at, (uint32_t)b.n_slots);
  const uint32_t left = head >= 0 ? (uint32_t)max(b.n_free - head, 0) : 0;
  uint32_t start = sum_before<ONE>(pages, part), top = 0;
  const bool tells = blockIdx.x == 0 && (!ONE || tid < 64);
  each([&](int r, int len, int c) {
    const int need = ONE ? need0 : first[r];
    start = held(start, (uint32_t)max(need, 0));
    const bool fits = start <= left && start < MOST;
    const int free = need <= 0 ? need : fits ? (int32_t)(start - need) : -1;      // (no page needed: 0; refused already: -1)
    first[r] = free;
    if (need > 0 && fits) top = start;
    if (tells) {
      b.cu_tokens[r] = cu[r];
      b.new_lens[r] = len + (free >= 0 ? c : 0);
    }
  });
  if (tells && r0 < r1 && r1 == n) b.cu_tokens[n] = cu[n];
  if (ONE) {                                          // (the lanes of a wave read each other's entries)
    __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
    __builtin_amdgcn_wave_barrier();
    __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
  } else {
    __syncthreads();
  }

  if (blockIdx.x == 0) {
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) top = max(top, (uint32_t)__shfl_xor((int)top, o, 64));
    if (!ONE) {
      if ((tid & 63) == 0) part[tid >> 6] = top;
      __syncthreads();
      if (tid == 0)
        for (int w = 1; w < SLOT_THREADS / 64; ++w) top = max(top, part[w]);
    }
    if (tid == 0) *b.new_head = head + (int32_t)top;
  }
  // The slots: four in a row a thread, lengths and page numbers of the four asked for together.  A page that is taken begins with
  // a new token, which enters it in the table.
  const bool whole = ((uintptr_t)b.slots & 15u) == 0;
  const int mask = (1 << shift) - 1;
  for (int64_t i0 = 4 * ((int64_t)blockIdx.x * SLOT_THREADS + tid); i0 < b.n_slots; i0 += 4 * (int64_t)SLOT_THREADS * gridDim.x) {
    int r = 0;                                        // the last request that starts at i0 or before (n: no request's)
    for (int lo = 0, hi = n + 1; lo < hi;) {
      const int mid = (lo + hi) >> 1;
      if (cu[mid] <= i0) { r = mid; lo = mid + 1; } else { hi = mid; }
    }
    int of[4], len[4], block[4], s[4];
    bool there[4], taken[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      while (r < n && i0 + j >= cu[r + 1]) ++r;
      of[j] = min(r, n - 1);
      there[j] = r < n && first[of[j]] >= 0;
      len[j] = ONE ? old[of[j]] : b.lens[of[j]];
    }
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int p = (len[j] + (int)(i0 + j - cu[of[j]])) >> shift, have = (int)(((int64_t)len[j] + mask) >> shift);
      taken[j] = p >= have;
      const int32_t *from = taken[j] ? b.free_blocks + (head + first[of[j]] + p - have) : b.block_table + ((int64_t)of[j] * b.ld_table + p);
      block[j] = *(there[j] ? from : b.lens);         // (no slot: any memory, not looked at)
    }
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int pos = len[j] + (int)(i0 + j - cu[of[j]]);
      s[j] = there[j] && block[j] >= 0 && block[j] < b.blocks ? (block[j] << shift) + (pos & mask) : -1;
      if (there[j] && taken[j] && (pos & mask) == 0) b.block_table[(int64_t)of[j] * b.ld_table + (pos >> shift)] = block[j];
    }
    if (whole && i0 + 4 <= b.n_slots) {
      *(int4 *)(b.slots + i0) = int4{s[0], s[1], s[2], s[3]};
    } else {
      for (int j = 0; j < 4 && i0 + j < b.n_slots; ++j) b.slots[i0 + j] = s[j];
    }
  }
}

// A copy: bound by memory, or, for the tokens of a step, by the latency of a slot number and a row behind it.  2^tshift threads
// walk a token's 16-byte pieces, keys and values together (two requests in flight a piece); short rows share a workgroup.
__global__ __launch_bounds__(256) void k_kv_append(egt_append_batch b, egt_kv_cache c, int shift, int tshift) {
  const int t = threadIdx.x & ((1 << tshift) - 1);
  const int64_t i = ((int64_t)blockIdx.x << (8 - tshift)) + (threadIdx.x >> tshift);
  if (i >= b.n) return;
  const int slot = b.slots[i], row = b.rows ? b.rows[i] : (int)i;
  if (slot < 0 || (slot >> shift) >= c.blocks || row < 0 || row >= b.n_rows) return;
  const int64_t block = slot >> shift, place = slot & ((1 << shift) - 1);
  const uint16_t *ks = b.k + row * b.k_row, *vs = b.v + row * b.v_row;
  uint16_t *kd = c.k + block * c.k_block + place * c.k_token, *vd = c.v + block * c.v_block + place * c.v_token;
  const int per = c.dim / 8;
  for (int p = t; p < c.heads * per; p += 1 << tshift) {
    const int h = p / per, d = 8 * (p - h * per);
    const uint4 kk = *(const uint4 *)(ks + h * b.k_head + d), vv = *(const uint4 *)(vs + h * b.v_head + d);
    *(uint4 *)(kd + h * c.k_head + d) = kk;
    *(uint4 *)(vd + h * c.v_head + d) = vv;
  }
}

inline bool whole4(const void *p) { return ((uintptr_t)p & 3u) == 0; }

}  // namespace
}  // namespace egt

extern "C" {

egt_status egt_kv_slots(const egt_slots_batch *b, void *stream) {
  if (!b) return EGT_ERR_NULL;
  if (b->requests < 1 || b->table_blocks < 0 || b->ld_table < b->table_blocks || b->page < 1 || (b->page & (b->page - 1)) != 0 || b->blocks < 0 ||
      (int64_t)b->blocks * b->page >= (1ll << 31) || (int64_t)b->table_blocks * b->page >= (1ll << 31) || b->n_free < 0 || b->n_slots < 0)
    return EGT_ERR_SHAPE;
  if (b->requests > EGT_MAX_REQUESTS) return EGT_ERR_UNSUPPORTED;
  if (!b->lens || !b->counts || (b->table_blocks && !b->block_table) || (b->n_free && !b->free_blocks) || !b->free_head || (b->n_slots && !b->slots) ||
      !b->cu_tokens || !b->new_lens || !b->new_head)
    return EGT_ERR_NULL;
  for (const void *p : {(const void *)b->lens, (const void *)b->counts, (const void *)b->block_table, (const void *)b->free_blocks, (const void *)b->free_head,
                        (const void *)b->slots, (const void *)b->cu_tokens, (const void *)b->new_lens, (const void *)b->new_head})
    if (!egt::whole4(p)) return EGT_ERR_BUFFER;
  if (b->lens == b->new_lens || b->counts == b->new_lens || b->free_head == b->new_head) return EGT_ERR_BUFFER;
  // (a million slots: 1024 workgroups, each once through its chain, 6.7 us; 512, twice through the last part, 7.7)
  const int64_t want = ((int64_t)b->n_slots + 4 * egt::SLOT_THREADS - 1) / (4 * egt::SLOT_THREADS);
  const dim3 grid((unsigned)std::min<int64_t>(std::max<int64_t>(want, 1), 1024)), block(egt::SLOT_THREADS);
  const size_t lds = 4 * (size_t)(b->requests <= 64 ? egt::SLOT_THREADS / 64 * (3 * b->requests + 1) : 2 * b->requests + 1);
  return egt::answer(b->requests <= 64 ? egt::launch(egt::k_kv_slots<true>, grid, block, lds, (hipStream_t)stream, *b, egt::log2_of(b->page))
                                       : egt::launch(egt::k_kv_slots<false>, grid, block, lds, (hipStream_t)stream, *b, egt::log2_of(b->page)));
}

egt_status egt_kv_append(const egt_append_batch *b, const egt_kv_cache *cache, void *stream) {
  if (!b) return EGT_ERR_NULL;
  const egt_status st = egt::check_cache(cache, true);
  if (st != EGT_OK) return st;
  if (b->n < 0 || b->n_rows < 0) return EGT_ERR_SHAPE;
  if (b->n == 0 || b->n_rows == 0 || cache->blocks == 0) return EGT_OK;          // nothing to write
  if (!b->k || !b->v || !b->slots) return EGT_ERR_NULL;
  if (!egt::whole16(b->k) || !egt::whole16(b->v) || !egt::whole8(b->k_row, b->k_head, b->v_row, b->v_head) || !egt::whole4(b->slots) || !egt::whole4(b->rows))
    return EGT_ERR_BUFFER;
  const int64_t pieces = (int64_t)cache->heads * (cache->dim / 8);
  if (b->n >= 1 << 24 || pieces > 1 << 30) return EGT_ERR_UNSUPPORTED;     // (a launch has less than 2^32 threads; pieces are counted in 31 bits)
  int tshift = 2;
  while (tshift < 8 && (1 << tshift) < pieces) ++tshift;
  const int64_t groups = ((int64_t)b->n + (256 >> tshift) - 1) >> (8 - tshift);
  return egt::answer(egt::launch(egt::k_kv_append, dim3((unsigned)groups), dim3(256), 0, (hipStream_t)stream, *b, *cache, egt::log2_of(cache->page), tshift));
}

}  // extern "C"
