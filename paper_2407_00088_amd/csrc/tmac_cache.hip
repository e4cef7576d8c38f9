// Caches that keep the heaviest keys (tmac_attn.h): filling one from prompts or from another cache, and taking in one token.
//
// Eviction orders tokens by (recent or not, weight, slot).  As whole numbers: a weight's bits, mapped so that they ascend with
// its value (NaN as -inf), all ones for a recent token, which is above +inf; equal keys go by the slot.  Recent tokens leave only where
// positions repeat or lie ahead of what the cache has seen; the search is then made again over their weights.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cstdint>

#include "tmac_attn.h"
#include "tmac_attn_host.h"
#include "tmac_internal.h"

namespace tmac {
namespace cache {

typedef uint32_t u2 __attribute__((ext_vector_type(2)));
typedef uint32_t u4 __attribute__((ext_vector_type(4)));

__device__ __forceinline__ uint32_t order_key(float weight, bool recent) {
  const uint32_t u = __builtin_bit_cast(uint32_t, weight != weight ? -INFINITY : weight + 0.0f);  // (-0 becomes 0)
  return recent ? 0xffffffffu : (u >> 31) ? ~u : u | 0x80000000u;
}

__device__ __forceinline__ int clamp_to(int x, int most) { return x < 0 ? 0 : x > most ? most : x; }

struct FillArgs {
  const char *k_src, *v_src;
  const float* w_src;
  const int32_t *pos_src, *cu, *src_lens, *src_seen;
  char *k, *v;
  float* weight;
  int32_t *pos, *lens, *seen, *index;
  int64_t ks_seq, ks_token, ks_head, vs_seq, vs_token, vs_head;  // bytes
  int64_t ws_seq, ws_token, ws_head, ps_seq, ps_token, ps_head;  // elements
  int64_t k_seq, k_token, k_head, v_seq, v_token, v_head;        // bytes
  int B, Hkv, D, C, recent, total, blocks;
};

// Tokens of a sequence and head in the source: how many, and the first one's token index.
__device__ __forceinline__ int source_tokens(const FillArgs& a, int b, int h, int& first) {
  if (!a.cu) {
    first = 0;
    return clamp_to(a.src_lens[b * a.Hkv + h], a.total);
  }
  first = clamp_to(a.cu[b], a.total);
  return max(0, clamp_to(a.cu[b + 1], a.total) - first);
}

constexpr int WAVES = 16, DIGIT = 2048;
constexpr int COPIED = 1024;  // slots whose rows the selecting workgroup copies itself

// Number of set bits of `mask` below the lane.
__device__ __forceinline__ int below(uint64_t mask) {
  return __builtin_amdgcn_mbcnt_hi((uint32_t)(mask >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)mask, 0));
}

// Keys, values, weights and positions into slots [lo, lo + rows), rows Unit by Unit and past the caches: every byte is read once and
// written once.  index: their tokens.
template <typename Unit, int THREADS>
__device__ __forceinline__ void copy_rows(const FillArgs& a, int b, int h, int first, const int32_t* index, int lo, int rows) {
  const int per_row = a.D * 2 / (int)sizeof(Unit);
  const char* ks = a.k_src + b * a.ks_seq + h * a.ks_head + first * a.ks_token;
  const char* vs = a.v_src + b * a.vs_seq + h * a.vs_head + first * a.vs_token;
  char* kd = a.k + b * a.k_seq + h * a.k_head + lo * a.k_token;
  char* vd = a.v + b * a.v_seq + h * a.v_head + lo * a.v_token;
  const float* w = a.w_src + b * a.ws_seq + h * a.ws_head + first * a.ws_token;
  const int32_t* p = a.pos_src ? a.pos_src + b * a.ps_seq + h * a.ps_head + first * a.ps_token : nullptr;
  const int64_t slot0 = ((int64_t)b * a.Hkv + h) * a.C + lo;
  for (int x = threadIdx.x; x < rows; x += THREADS) {
    const int i = index[x];
    a.weight[slot0 + x] = w[i * a.ws_token];
    a.pos[slot0 + x] = p ? p[i * a.ps_token] : i;
  }
#pragma unroll 4
  for (int x = threadIdx.x; x < rows * per_row; x += THREADS) {
    const int row = x / per_row, at = (x - row * per_row) * (int)sizeof(Unit);
    const int64_t i = index[row];
    const Unit k = __builtin_nontemporal_load(reinterpret_cast<const Unit*>(ks + i * a.ks_token + at));
    const Unit v = __builtin_nontemporal_load(reinterpret_cast<const Unit*>(vs + i * a.vs_token + at));
    __builtin_nontemporal_store(k, reinterpret_cast<Unit*>(kd + row * a.k_token + at));
    __builtin_nontemporal_store(v, reinterpret_cast<Unit*>(vd + row * a.v_token + at));
  }
}

// What the selection shares: counters of a digit, and sums and counts of wavefronts.
struct Selecting {
  uint32_t count[DIGIT], wave_sum[2][WAVES], chosen[2];
};

// The places of the n - leave tokens that stay, in order: of keys read_key(i), i < n, the `leave` smallest go (equal ones by i).
// The leave-th smallest key is found digit by digit (11, 11 and 10 bits, counted in LDS), then every wavefront numbers the
// staying tokens of its run.  PER: tokens of a lane, which stay in registers from the first look on; 0: any number, read again by
// every step.  False: the leave-th is a recent token, nothing is written.  (128 caches, 4096 of 16384 tokens each: 24 us, the instructions of
// 16 wavefronts on one CU; with the keys in LDS it was 30, with four counters a digit still 24.)
template <int PER, typename ReadKey>
__device__ __forceinline__ bool select(ReadKey read_key, int n, uint32_t leave, int32_t* index, Selecting& sh) {
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int turns = (n + 64 * WAVES - 1) / (64 * WAVES), lo = wave * turns * 64;  // a wavefront's run: `turns` times 64 tokens
  uint32_t mine[PER ? PER : 1];
#pragma unroll
  for (int y = 0; y < PER; ++y)
    if (y < turns) mine[y] = lo + y * 64 + lane < n ? read_key(lo + y * 64 + lane) : 0u;
  auto each = [&](auto&& f) {
    if constexpr (PER != 0) {
#pragma unroll
      for (int y = 0; y < PER; ++y)
        if (y < turns) f(lo + y * 64 + lane, mine[y]);
    } else {
      for (int y = 0; y < turns; ++y) {
        const int i = lo + y * 64 + lane;
        f(i, i < n ? read_key(i) : 0u);
      }
    }
  };
  uint32_t prefix = 0, rank = leave - 1;  // of the key that is looked for, among those with its digits so far
#pragma unroll
  for (int pass = 0; pass < 3; ++pass) {
    const int shift = pass == 0 ? 21 : pass == 1 ? 10 : 0, bits = pass == 2 ? 10 : 11, above = shift + bits;
#pragma unroll
    for (int i = 0; i < DIGIT / (64 * WAVES); ++i) sh.count[tid + i * 64 * WAVES] = 0;
    __syncthreads();
    each([&](int i, uint32_t x) {
      const bool counts = i < n && (pass == 0 || x >> (above & 31) == prefix >> (above & 31));
      // (recent tokens lie side by side and would all meet in one counter: a wavefront's are counted together)
      const bool recent = counts && x == 0xffffffffu;
      const uint64_t together = __ballot(recent);
      if (counts && !recent) atomicAdd(&sh.count[(x >> shift) & ((1u << bits) - 1)], 1u);
      if (recent && below(together) == 0) atomicAdd(&sh.count[(1u << bits) - 1], (uint32_t)__builtin_popcountll(together));
    });
    __syncthreads();
    // two digits a thread
    const uint32_t c0 = sh.count[2 * tid], c1 = sh.count[2 * tid + 1];
    uint32_t incl = c0 + c1;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
      const uint32_t x = __shfl_up(incl, o);
      if (lane >= o) incl += x;
    }
    if (lane == 63) sh.wave_sum[0][wave] = incl;
    __syncthreads();
    uint32_t before = incl - c0 - c1;
#pragma unroll
    for (int i = 0; i < WAVES; ++i) before += i < wave ? sh.wave_sum[0][i] : 0;
    if (rank >= before && rank < before + c0) sh.chosen[0] = 2 * tid, sh.chosen[1] = before;
    if (rank >= before + c0 && rank < before + c0 + c1) sh.chosen[0] = 2 * tid + 1, sh.chosen[1] = before + c0;
    __syncthreads();
    prefix |= sh.chosen[0] << shift;
    rank -= sh.chosen[1];
  }
  if (__builtin_expect(__builtin_amdgcn_readfirstlane(prefix) == 0xffffffffu, 0)) return false;
  // of the tokens whose key is `prefix`, the first rank + 1 leave
  const uint32_t go = rank + 1;
  uint32_t greater = 0, equal = 0;
  each([&](int i, uint32_t x) {
    greater += __builtin_popcountll(__ballot(i < n && x > prefix));
    equal += __builtin_popcountll(__ballot(i < n && x == prefix));
  });
  __syncthreads();
  if (lane == 0) sh.wave_sum[0][wave] = greater, sh.wave_sum[1][wave] = equal;
  __syncthreads();
  greater = equal = 0;
#pragma unroll
  for (int i = 0; i < WAVES; ++i) greater += i < wave ? sh.wave_sum[0][i] : 0, equal += i < wave ? sh.wave_sum[1][i] : 0;
  uint32_t at = greater + (equal > go ? equal - go : 0);
  each([&](int i, uint32_t x) {
    const uint64_t same = __ballot(i < n && x == prefix);
    const bool stays = i < n && (x > prefix || (x == prefix && equal + below(same) >= go));
    const uint64_t mask = __ballot(stays);
    if (stays) index[at + below(mask)] = i;
    equal += __builtin_popcountll(same);
    at += __builtin_popcountll(mask);
  });
  return true;
}

// One workgroup a sequence and key head.  COPIES: it copies the rows too, else it leaves the tokens' places for the copying launch.
template <bool COPIES, typename Unit>
__global__ __launch_bounds__(64 * WAVES) void cache_select_kernel(const FillArgs a) {
  __shared__ Selecting sh;
  __shared__ int32_t kept[COPIES ? COPIED : 1];
  const int tid = threadIdx.x, bh = blockIdx.x, b = bh / a.Hkv, h = bh % a.Hkv;
  int first;
  const int n = source_tokens(a, b, h, first), keep = min(n, a.C);
  const int seen = a.src_seen ? a.src_seen[bh] : n;
  const float* w = a.w_src + b * a.ws_seq + h * a.ws_head + first * a.ws_token;
  const int32_t* p = a.pos_src ? a.pos_src + b * a.ps_seq + h * a.ps_head + first * a.ps_token : nullptr;
  int32_t* index = COPIES ? kept : a.index + (int64_t)bh * a.C;
  if (tid == 0) {
    a.lens[bh] = keep;
    a.seen[bh] = seen;
  }
  auto recent = [&](int i) { return (int64_t)(p ? p[i * a.ps_token] : i) >= (int64_t)seen - a.recent; };
  auto read_key = [&](int i) { return order_key(w[i * a.ws_token], recent(i)); };
  // (more leave than are not recent: those all, below any weight's key, then the lightest recent ones; no key is a recent token's then)
  auto read_again = [&](int i) { return recent(i) ? order_key(w[i * a.ws_token], false) : 0u; };
  if (n <= a.C) {
    for (int i = tid; i < n; i += 64 * WAVES) index[i] = i;
  } else if (n <= 4 * 64 * WAVES) {
    if (__builtin_expect(!select<4>(read_key, n, n - a.C, index, sh), 0)) select<4>(read_again, n, n - a.C, index, sh);
  } else if (n <= 16 * 64 * WAVES) {
    if (__builtin_expect(!select<16>(read_key, n, n - a.C, index, sh), 0)) select<0>(read_again, n, n - a.C, index, sh);
  } else {
    if (__builtin_expect(!select<0>(read_key, n, n - a.C, index, sh), 0)) select<0>(read_again, n, n - a.C, index, sh);
  }
  if constexpr (COPIES) {
    __syncthreads();
    copy_rows<Unit, 64 * WAVES>(a, b, h, first, kept, 0, keep);
  }
}

// 64 slots of a sequence and key head a workgroup: memory's rate bounds it (128 caches of 4096 slots of 128 elements, 550 MB read and
// written with the weights and positions: 106 us, 5.2 TB/s, what a large copy reaches).
template <typename Unit>
__global__ __launch_bounds__(256) void cache_copy_kernel(const FillArgs a) {
  const int bh = blockIdx.x / a.blocks, block = blockIdx.x % a.blocks, b = bh / a.Hkv, h = bh % a.Hkv;
  const int n = clamp_to(a.lens[bh], a.C), lo = block * 64, rows = min(64, n - lo);
  if (rows <= 0) return;
  int first;
  source_tokens(a, b, h, first);
  copy_rows<Unit, 256>(a, b, h, first, a.index + (int64_t)bh * a.C + lo, lo, rows);
}

struct AppendArgs {
  const char *k_new, *v_new;
  char *k, *v;
  float* weight;
  int32_t *pos, *lens, *seen;
  int64_t kn_seq, kn_head, vn_seq, vn_head, k_seq, k_token, k_head, v_seq, v_token, v_head;  // bytes
  int Hkv, D, C, recent;
};

// One workgroup a sequence and key head, of 256 threads or, for more than 1024 slots, 1024 (192 caches of 4095 slots: 14.3 us with 256, most
// of it waiting for one load after another, 4.8 with 1024; 32 of 256 slots 3.1).  Latency binds: lengths, slots, minimum, rows.
template <int THREADS>
__global__ __launch_bounds__(THREADS) void cache_append_kernel(const AppendArgs a) {
  __shared__ uint64_t least[THREADS / 64];
  const int tid = threadIdx.x, bh = blockIdx.x, b = bh / a.Hkv, h = bh % a.Hkv;
  const int n = clamp_to(a.lens[bh], a.C), seen = a.seen[bh];
  float* weight = a.weight + (int64_t)bh * a.C;
  int32_t* pos = a.pos + (int64_t)bh * a.C;
  // the new rows, 8 bytes a thread: keys, then values
  const int per_row = a.D / 4, at = (tid < per_row ? tid : tid - per_row) * 8;
  u2 row = {0u, 0u};
  if (tid < 2 * per_row)
    row = *reinterpret_cast<const u2*>((tid < per_row ? a.k_new + b * a.kn_seq + h * a.kn_head : a.v_new + b * a.vn_seq + h * a.vn_head) + at);
  // four slots a thread are on their way before it is known whether the cache is full
  float w4[4];
  int32_t p4[4];
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const int i = min(tid + j * THREADS, a.C - 1);
    w4[j] = weight[i], p4[j] = pos[i];
  }
  int slot = n;
  if (n == a.C) {
    const int64_t recent_from = (int64_t)seen + 1 - a.recent;
    uint64_t best = ~0ull;
    auto consider = [&](int i, float w, bool recent) {
      const uint64_t x = (uint64_t)order_key(w, recent) << 32 | (uint32_t)i;
      best = x < best ? x : best;
    };
#pragma unroll
    for (int j = 0; j < 4; ++j)
      if (tid + j * THREADS < n) consider(tid + j * THREADS, w4[j], p4[j] >= recent_from);
#pragma unroll 4
    for (int i = tid + 4 * THREADS; i < n; i += THREADS) consider(i, weight[i], pos[i] >= recent_from);
    auto meet = [&] {
#pragma unroll
      for (int o = 32; o > 0; o >>= 1) {
        const uint64_t x = __shfl_xor((unsigned long long)best, o);
        best = x < best ? x : best;
      }
      if ((tid & 63) == 0) least[tid >> 6] = best;
      __syncthreads();
#pragma unroll
      for (int i = 0; i < THREADS / 64; ++i) best = least[i] < best ? least[i] : best;
    };
    meet();
    if (best >> 32 == 0xffffffffu) {  // all are recent: by their weights
      best = ~0ull;
      for (int i = tid; i < n; i += THREADS) consider(i, weight[i], false);
      __syncthreads();
      meet();
    }
    slot = (int)(uint32_t)best;
  }
  // (every thread has read the lengths and the slots before any of them is changed)
  __syncthreads();
  if (tid == 0) {
    weight[slot] = 0.0f;
    pos[slot] = seen;
    a.seen[bh] = seen + 1;
    if (n < a.C) a.lens[bh] = n + 1;
  }
  if (tid < 2 * per_row)
    *reinterpret_cast<u2*>((tid < per_row ? a.k + b * a.k_seq + h * a.k_head + slot * a.k_token : a.v + b * a.v_seq + h * a.v_head + slot * a.v_token) + at) = row;
}

static bool cache_ok(const tmac_cache* c) {
  return c && c->B >= 0 && c->Hkv > 0 && c->D > 0 && c->D % 4 == 0 && c->capacity > 0 && c->recent >= 0 && c->recent <= c->capacity &&
         (c->elem == TMAC_ELEM_F16 || c->elem == TMAC_ELEM_BF16) && !c->reserved[0] && !c->reserved[1];
}
static bool cache_set(const tmac_cache* c) {
  return attn::rows_ok(&c->k, true, true, true) && attn::rows_ok(&c->v, true, true, true) && c->weight_dev && c->pos_dev && c->lens_dev &&
         c->seen_dev;
}
static tmac_status launch(const void* kernel, int64_t grid, int threads, void* args, void* stream) {
  if (!attn::launchable(grid, threads)) return TMAC_EUNSUPPORTED;
  void* ptrs[] = {args};
  const hipError_t e = hipLaunchKernel(kernel, dim3((unsigned)grid), dim3((unsigned)threads), ptrs, 0, static_cast<hipStream_t>(stream));
  if (e == hipSuccess) return TMAC_OK;
  note_hip_error((int)e);
  return TMAC_EHIP;
}

}  // namespace cache
}  // namespace tmac

using namespace tmac;
using namespace tmac::cache;

extern "C" size_t tmac_cache_fill_workspace_bytes(const tmac_cache* cache) {
  return cache_ok(cache) ? (size_t)cache->B * cache->Hkv * cache->capacity * 4 : 0;
}

extern "C" tmac_status tmac_cache_fill(const tmac_cache* cache, const tmac_cache_source* src, void* workspace_dev, size_t workspace_bytes,
                                       void* stream) {
  if (!cache_ok(cache) || !src || src->total < 0 || src->reserved) return TMAC_EINVAL;
  const int B = cache->B;
  if (B == 0) return TMAC_OK;
  if (!cache_set(cache) || !!src->cu_dev == !!src->lens_dev) return TMAC_EINVAL;
  const bool packed = src->cu_dev != nullptr;
  if (src->total > 0) {
    if (!attn::rows_ok(&src->k, !packed, true, true) || !attn::rows_ok(&src->v, !packed, true, true) || !src->weight.data) return TMAC_EINVAL;
    for (const tmac_view* x : {&src->weight, &src->pos})
      if (x->data && ((!packed && x->seq < 0) || x->token < 0 || x->head < 0 || (reinterpret_cast<uintptr_t>(x->data) & 3))) return TMAC_EINVAL;
  }
  if (cache->D > 128 || (int64_t)B * cache->Hkv > 0x7fffffff || attn::long_axis(cache->capacity) || attn::long_axis(src->total)) return TMAC_EUNSUPPORTED;
  if (!workspace_dev || (reinterpret_cast<uintptr_t>(workspace_dev) & 15)) return TMAC_EINVAL;
  if (workspace_bytes < tmac_cache_fill_workspace_bytes(cache)) return TMAC_ESIZE;
  FillArgs a = {};
  a.k_src = static_cast<const char*>(src->k.data), a.v_src = static_cast<const char*>(src->v.data);
  a.w_src = static_cast<const float*>(src->weight.data), a.pos_src = static_cast<const int32_t*>(src->pos.data);
  a.cu = src->cu_dev, a.src_lens = src->lens_dev, a.src_seen = src->seen_dev;
  a.k = static_cast<char*>(cache->k.data), a.v = static_cast<char*>(cache->v.data);
  a.weight = cache->weight_dev, a.pos = cache->pos_dev, a.lens = cache->lens_dev, a.seen = cache->seen_dev;
  a.index = static_cast<int32_t*>(workspace_dev);
  a.ks_seq = packed ? 0 : src->k.seq * 2, a.ks_token = src->k.token * 2, a.ks_head = src->k.head * 2;
  a.vs_seq = packed ? 0 : src->v.seq * 2, a.vs_token = src->v.token * 2, a.vs_head = src->v.head * 2;
  a.ws_seq = packed ? 0 : src->weight.seq, a.ws_token = src->weight.token, a.ws_head = src->weight.head;
  a.ps_seq = packed ? 0 : src->pos.seq, a.ps_token = src->pos.token, a.ps_head = src->pos.head;
  a.k_seq = cache->k.seq * 2, a.k_token = cache->k.token * 2, a.k_head = cache->k.head * 2;
  a.v_seq = cache->v.seq * 2, a.v_token = cache->v.token * 2, a.v_head = cache->v.head * 2;
  a.B = B, a.Hkv = cache->Hkv, a.D = cache->D, a.C = cache->capacity, a.recent = cache->recent, a.total = src->total;
  a.blocks = (cache->capacity + 63) / 64;
  const int64_t bh = (int64_t)B * cache->Hkv;
  const bool wide = attn::wide_rows(&src->k, a.D) && attn::wide_rows(&src->v, a.D) && attn::wide_rows(&cache->k, a.D) && attn::wide_rows(&cache->v, a.D);
  // Small caches are copied by the workgroup that selects, which saves a launch and what is between two (rows of 128 elements, 256 slots:
  // 8 caches 10.0 us, 11.2 in two launches; 96 of 100 elements 12.3, 13.6); beyond 128 KB of keys and values one workgroup's
  // copy takes longer than that (512 slots: 8 caches 15.7, 13.1; 96 caches 21.5, 18.8).
  if (cache->capacity <= COPIED && (int64_t)cache->capacity * a.D * 4 <= 131072)
    return cache::launch(wide ? (const void*)cache_select_kernel<true, u4> : (const void*)cache_select_kernel<true, u2>, bh, 64 * WAVES, &a, stream);
  if (!attn::launchable(bh * a.blocks, 256)) return TMAC_EUNSUPPORTED;
  const tmac_status st = cache::launch((const void*)cache_select_kernel<false, u2>, bh, 64 * WAVES, &a, stream);
  if (st != TMAC_OK) return st;
  return cache::launch(wide ? (const void*)cache_copy_kernel<u4> : (const void*)cache_copy_kernel<u2>, bh * a.blocks, 256, &a, stream);
}

extern "C" tmac_status tmac_cache_append(const tmac_cache* cache, const tmac_view* k, const tmac_view* v, void* stream) {
  if (!cache_ok(cache)) return TMAC_EINVAL;
  if (cache->B == 0) return TMAC_OK;
  if (!cache_set(cache) || !attn::rows_ok(k, true, false, true) || !attn::rows_ok(v, true, false, true)) return TMAC_EINVAL;
  if (cache->D > 128 || (int64_t)cache->B * cache->Hkv > 0x7fffffff || attn::long_axis(cache->capacity)) return TMAC_EUNSUPPORTED;
  AppendArgs a = {};
  a.k_new = static_cast<const char*>(k->data), a.v_new = static_cast<const char*>(v->data);
  a.k = static_cast<char*>(cache->k.data), a.v = static_cast<char*>(cache->v.data);
  a.weight = cache->weight_dev, a.pos = cache->pos_dev, a.lens = cache->lens_dev, a.seen = cache->seen_dev;
  a.kn_seq = k->seq * 2, a.kn_head = k->head * 2, a.vn_seq = v->seq * 2, a.vn_head = v->head * 2;
  a.k_seq = cache->k.seq * 2, a.k_token = cache->k.token * 2, a.k_head = cache->k.head * 2;
  a.v_seq = cache->v.seq * 2, a.v_token = cache->v.token * 2, a.v_head = cache->v.head * 2;
  a.Hkv = cache->Hkv, a.D = cache->D, a.C = cache->capacity, a.recent = cache->recent;
  const bool many = cache->capacity > 1024;
  return cache::launch(many ? (const void*)cache_append_kernel<1024> : (const void*)cache_append_kernel<256>, (int64_t)cache->B * cache->Hkv,
                       many ? 1024 : 256, &a, stream);
}
