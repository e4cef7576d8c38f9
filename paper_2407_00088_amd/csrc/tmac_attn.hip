// Attention over packed prompts and over shared prefixes and caches (tmac_attn.h): kernels on the core of tmac_attn_core.h,
// the kernel that joins parts of a row, the kernel of the keys' weights, and their host entry points.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstdint>
#include <type_traits>

#include "tmac_attn.h"
#include "tmac_attn_core.h"
#include "tmac_attn_host.h"
#include "tmac_internal.h"

namespace tmac {
namespace attn {

constexpr float LOG2E = 1.4426950408889634f, LN2 = 0.6931471805599453f;

// --- epilogue ------------------------------------------------------------------------------------------------------------

// Where a row's result goes: the finished row, or a part of it (sums against a number of its own, which ml holds in units of
// log 2, with the sum of exponentials).
struct Target {
  char* out;     // the row's D elements; null: the lane's row does not exist
  float* lse;    // or null
  float* part;   // parts: the row's D sums
  float* ml;     // parts: what the sums are taken against, and the sum
};

template <typename T>
__device__ __forceinline__ void store4(char* to, f4 x) {
  *reinterpret_cast<typename T::v4*>(to) = __builtin_convertvector(x, typename T::v4);
}

// row_lse (BLOCKS = 1 only, or null): 32 numbers in LDS beyond those that the sums meet in, the rows' lse in units of log 2, there for all
// wavefronts when it returns.
template <typename T, int DP, int BLOCKS>
__device__ __forceinline__ void finish(Rows<T, DP>& w, const Target& to, bool parts, int D, char* lds, float* row_lse = nullptr) {
  constexpr int ND = DP / 32;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, half = lane >> 5;
  w.l = add_halves(w.l);
  if constexpr (BLOCKS != 1) {
    if (!to.out) return;
    const float scale = parts ? 1.0f : w.l == 0.0f ? 0.0f : 1.0f / w.l;
#pragma unroll
    for (int d = 0; d < ND; ++d)
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const int at = d * 32 + r * 8 + half * 4;
        if (at >= D) continue;
        const f4 x = f4{w.o[d][4 * r], w.o[d][4 * r + 1], w.o[d][4 * r + 2], w.o[d][4 * r + 3]};
        if (parts) *reinterpret_cast<f4*>(to.part + at) = x;
        else store4<T>(to.out + at * 2, x * scale);
      }
    if (half != 0) return;
    if (parts) *reinterpret_cast<f2*>(to.ml) = f2{w.m, w.l};
    else if (to.lse) *to.lse = w.l == 0.0f ? -INFINITY : log2_sum<T>(w.m, w.l) * LN2;
  } else {
    // the wavefronts that share rows meet in LDS: [wave][32 rows][DP + 4] sums, then [wave][32] maximum and sum
    constexpr int KW = 4, W = DP + 4;
    float* sums = reinterpret_cast<float*>(lds);
    f2* ml = reinterpret_cast<f2*>(lds + 4 * 32 * W * 4);
    __syncthreads();
    if (half == 0) ml[wave * 32 + lane] = f2{w.m, w.l};
    __syncthreads();
    float m = -INFINITY;
#pragma unroll
    for (int i = 0; i < KW; ++i) m = fmaxf(m, ml[i * 32 + (lane & 31)][0]);
    const float a = w.m == m ? 1.0f : __builtin_amdgcn_exp2f(w.m - m);
    float* mine = sums + (wave * 32 + (lane & 31)) * W + half * 4;
#pragma unroll
    for (int d = 0; d < ND; ++d)
#pragma unroll
      for (int r = 0; r < 4; ++r)
        *reinterpret_cast<f4*>(mine + d * 32 + r * 8) =
            f4{w.o[d][4 * r], w.o[d][4 * r + 1], w.o[d][4 * r + 2], w.o[d][4 * r + 3]} * a;
    float l = 0.0f;
#pragma unroll
    for (int i = 0; i < KW; ++i) {
      const f2 x = ml[i * 32 + (lane & 31)];
      l += x[0] == m ? x[1] : x[1] * __builtin_amdgcn_exp2f(x[0] - m);
    }
    // (before the last barrier: the caller's wavefronts read it without another)
    if (row_lse && half == 0 && wave == 0) row_lse[lane] = l == 0.0f ? INFINITY : log2_sum<T>(m, l);
    __syncthreads();
    // every lane keeps its row's scale and target for the lanes that store the row
    const float inv = l == 0.0f ? 0.0f : 1.0f / l;
    if (to.out && half == 0 && wave == 0) {
      if (parts) *reinterpret_cast<f2*>(to.ml) = f2{m, l};
      else if (to.lse) *to.lse = l == 0.0f ? -INFINITY : log2_sum<T>(m, l) * LN2;
    }
    // the rows, dealt over the wavefronts: 16 lanes a row where DP = 64, 32 where it is 128
    constexpr int LPR = DP / 4, RPW = 64 / LPR, N = 32 / KW / RPW;
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int row = (wave * N + i) * RPW + lane / LPR, at = (lane % LPR) * 4;
      f4 x = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
      for (int j = 0; j < KW; ++j) x += *reinterpret_cast<const f4*>(sums + (j * 32 + row) * W + at);
      char* out = reinterpret_cast<char*>(__shfl((unsigned long long)to.out, row));
      float* part = reinterpret_cast<float*>(__shfl((unsigned long long)to.part, row));
      const float iv = __shfl(inv, row);
      if (out && at < D) {
        if (parts) *reinterpret_cast<f4*>(part + at) = x;
        else store4<T>(out + at * 2, x * iv);
      }
    }
  }
}

// The lane's row as the first product's operand; rows that do not exist and columns from D on are zeros.  wide: 16 bytes at a time.
template <typename T, int DP>
__device__ __forceinline__ void load_q(Rows<T, DP>& w, const char* row, bool exists, int D, int lane, bool wide) {
  const int half = lane >> 5;
  if (wide) {
#pragma unroll
    for (int t = 0; t < DP / 16; ++t) {
      const int at = 16 * t + 8 * half;
      u4 x = {0u, 0u, 0u, 0u};
      if (exists && at < D) x = *reinterpret_cast<const u4*>(row + at * 2);
      w.q[t] = __builtin_bit_cast(typename T::v8, x);
    }
    return;
  }
#pragma unroll
  for (int t = 0; t < DP / 16; ++t) {
    u2 x[2] = {{0u, 0u}, {0u, 0u}};
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      const int at = 16 * t + 8 * half + 4 * j;
      if (exists && at < D) x[j] = *reinterpret_cast<const u2*>(row + at * 2);
    }
    w.q[t] = __builtin_bit_cast(typename T::v8, u4{x[0][0], x[0][1], x[1][0], x[1][1]});
  }
}

// --- prompts --------------------------------------------------------------------------------------------------------------

struct PromptArgs {
  const char *q, *k, *v;
  char* out;
  const int32_t *cu_q, *cu_k;
  float *lse, *part, *ml;
  int64_t q_token, q_head, k_token, k_head, v_token, v_head, o_token, o_head;  // bytes
  int S, Tq, Tk, Hq, Hkv, G, D, causal, tiles, slices;
  int q_wide;  // rows of q that are read 16 bytes at a time
  float scale;
};

__device__ __forceinline__ int clamp_to(int x, int most) { return x < 0 ? 0 : x > most ? most : x; }

// Sum, and largest, of a number over the wavefront, in all lanes.
template <bool MAX>
__device__ __forceinline__ int over_wave(int x) {
  auto with = [](int a, int b) { return MAX ? max(a, b) : a + b; };
  // (lanes without a source keep 0, so the largest is of numbers that are not negative)
  x = with(x, __builtin_amdgcn_update_dpp(0, x, 0x111, 0xf, 0xf, false));  // from 1, 2, 4, 8 lanes below in the row of 16
  x = with(x, __builtin_amdgcn_update_dpp(0, x, 0x112, 0xf, 0xf, false));
  x = with(x, __builtin_amdgcn_update_dpp(0, x, 0x114, 0xf, 0xf, false));
  x = with(x, __builtin_amdgcn_update_dpp(0, x, 0x118, 0xf, 0xf, false));
  x = with(x, __builtin_amdgcn_update_dpp(0, x, 0x142, 0xa, 0xf, false));  // the last lane of the row below
  x = with(x, __builtin_amdgcn_update_dpp(0, x, 0x143, 0xc, 0xf, false));  // lane 31
  return __builtin_amdgcn_readlane(x, 63);
}

// Sequence, and place in it, of unit t of all sequences' tiles, heaviest first: sequence s has as many tiles as its rows (`n` rows of `cu`,
// G times) fill, tile i of which weighs i + (its keys before the first row) / (rows of a tile) / G or so.  Workgroups start in the order of their
// units, and a heavy one that starts last is what all others wait for.
// by_keys: the tiles are of keys, of which the first are the heaviest.  False: there is no such tile.
struct Place {
  int seq, tile, q0, nq, k0, nk;
};
__device__ __forceinline__ bool find_tile(const int32_t* cu_q, const int32_t* cu_k, int S, int Tq, int Tk, bool by_keys, int G, int per_tile, int t,
                                          Place& p) {
  auto extent = [](const int32_t* cu, int s, int T, int& at) {
    at = clamp_to(cu[s], T);
    return max(0, clamp_to(cu[s + 1], T) - at);
  };
  auto tiles_of = [&](int nq, int nk) { return (int)(((int64_t)(by_keys ? nk : nq) * G + per_tile - 1) / per_tile); };
  if (S == 1) {
    p.seq = 0;
    p.nq = extent(cu_q, 0, Tq, p.q0);
    p.nk = extent(cu_k, 0, Tk, p.k0);
    const int n = tiles_of(p.nq, p.nk);
    p.tile = by_keys ? t : n - 1 - t;
    return t < n;
  }
  const int lane = threadIdx.x & 63;
  for (int s0 = 0; s0 < S; s0 += 64) {  // (heaviest first among each 64 sequences)
    int q0 = 0, nq = 0, k0 = 0, nk = 0;
    if (s0 + lane < S) {
      nq = extent(cu_q, s0 + lane, Tq, q0);
      nk = extent(cu_k, s0 + lane, Tk, k0);
    }
    const int n = tiles_of(nq, nk), base = by_keys ? 0 : (int)((int64_t)max(0, nk - nq) * G / per_tile);
    const int total = over_wave<false>(n);
    if (t >= total) {
      t -= total;
      continue;
    }
    // the least level x of which at most t tiles lie above: count(x) = tiles of level x or more
    auto count = [&](int x) { return over_wave<false>(min(n, max(0, n + base - x))); };
    int lo = 0, hi = over_wave<true>(n ? n + base : 0);  // count(lo) > t, count(hi) = 0 <= t
    int above = 0;
    while (hi - lo > 1) {
      const int mid = (lo + hi) / 2, c = count(mid);
      if (c > t) lo = mid;
      else hi = mid, above = c;
    }
    const uint64_t there = __ballot(lo >= base && lo < n + base);
    const int rank = __builtin_amdgcn_mbcnt_hi((uint32_t)(there >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)there, 0));
    const int at = __builtin_ctzll(__ballot((there >> lane & 1) && rank == t - above));
    p.seq = s0 + at;
    p.q0 = __builtin_amdgcn_readlane(q0, at), p.nq = __builtin_amdgcn_readlane(nq, at);
    p.k0 = __builtin_amdgcn_readlane(k0, at), p.nk = __builtin_amdgcn_readlane(nk, at);
    const int level = lo - __builtin_amdgcn_readlane(base, at);
    p.tile = by_keys ? __builtin_amdgcn_readlane(n, at) - 1 - level : level;
    return true;
  }
  return false;
}

// Unit of a grid of heads and units: a head's units on one XCD where the heads divide among the eight (workgroups go round the XCDs
// by their number), so that a head's keys stay in that XCD's L2.  Neighbouring heads, whose rows share lines of memory, are on the
// same one, and every unit's turn comes for all of them before the next unit's, so that the heaviest units of all heads start
// first (prompts of 860, 2003, 564, 158, 369, 68, 104, 242 and 1312 tokens, 32 heads of 100 elements: 109.8 us one head after the other,
// 99.6 all heads in turn, 98.8 neighbours on one XCD too; one of 8192, 32 heads of 128: 567, 547, 548).
__device__ __forceinline__ void head_and_unit(int id, int heads, int& head, int& unit) {
  if (heads % 8 == 0) {
    const int j = id / 8, of_xcd = heads / 8;
    head = id % 8 * of_xcd + j % of_xcd;
    unit = j / of_xcd;
  } else {
    head = id % heads;
    unit = id / heads;
  }
}

// A wavefront's rows of a workgroup's tile, (query, head of the group) in that order, so that the keys they see do not fall with the
// row: 32 side by side (BLOCKS = 1: all wavefronts have the same).
struct Tile {
  int first, last;  // first > last: none
  int row;          // the lane's, or -1
  __device__ __forceinline__ Tile(int tile, int blocks, int wave, int lane, int rows) {
    first = tile * 32 * blocks + (blocks == 1 ? 0 : wave * 32);
    last = min(first + 32, rows) - 1;
    row = first + (lane & 31) < rows ? first + (lane & 31) : -1;
  }
};

// One workgroup: 32 BLOCKS rows of one sequence and key head over the keys they see, or one slice of those; queries are read once,
// keys once a tile, from the XCD's L2.  Long sequences are bound by power: 8192 tokens, 64 heads in groups of 8 of 128 elements take 1.10 to 1.15 ms, 1.0
// PFLOP/s of the pairs that rows see (a large matrix product reaches 1.37), at 1.7 of 2.4 GHz with the matrix units busy for 53 % of the
// cycles and the vector ALUs, mostly with exponentials, for 49 %; LDS has no bank conflicts.  Short ones are bound by latency: 33 tokens, 32
// heads 6.2 us, one wavefront's chain of loads, products and exchanges.
template <typename T, int DP, int BLOCKS>
__global__ __launch_bounds__(256, 2) void attn_prompt_kernel(const PromptArgs a) {
  typedef Shape<DP, BLOCKS> Sh;
  __shared__ __align__(1024) char lds[Sh::LDS];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  int h, unit;
  head_and_unit(blockIdx.x, a.Hkv, h, unit);
  const int z = unit % a.slices;
  Place p;
  if (!find_tile(a.cu_q, a.cu_k, a.S, a.Tq, a.Tk, false, a.G, 32 * BLOCKS, unit / a.slices, p)) return;
  const int k0 = p.k0, nk = p.nk;
  const int row0 = p.tile * 32 * BLOCKS, rows = p.nq * a.G, off = nk - p.nq;
  const Tile tile(p.tile, BLOCKS, wave, lane, rows);
  // the keys that any row of the tile sees, and this slice of them
  auto sees = [&](int row) { return a.causal ? max(0, min(nk, row / a.G + off + 1)) : nk; };
  constexpr int SK = BLOCKS == 1 ? 128 : 32 * Sh::KB;
  const int seen = sees(min(row0 + 32 * BLOCKS, rows) - 1), stages = (seen + SK - 1) / SK, per = (stages + a.slices - 1) / a.slices;
  Keys keys;
  keys.k_stride = a.k_token;
  keys.v_stride = a.v_token;
  keys.k = a.k + k0 * a.k_token + h * a.k_head;
  keys.v = a.v + k0 * a.v_token + h * a.v_head;
  keys.begin = min(seen, z * per * SK);
  keys.end = min(seen, (z + 1) * per * SK);
  Rows<T, DP> w;
  Target to = {};
  Limits lim;
  const bool any = tile.first <= tile.last, exists = tile.row >= 0;
  lim.least_wg = min(keys.end, sees(row0));
  lim.least = any ? min(keys.end, sees(tile.first)) : keys.end;
  lim.most = any ? min(keys.end, sees(tile.last)) : 0;
  lim.row = exists ? min(keys.end, sees(tile.row)) : keys.end;
  const int i = exists ? tile.row / a.G : 0, head = h * a.G + (exists ? tile.row - i * a.G : 0);
  load_q(w, a.q + (int64_t)(p.q0 + i) * a.q_token + head * a.q_head, exists, a.D, lane, a.q_wide);
  if (exists) {
    const int64_t token = p.q0 + i, slot = ((int64_t)z * a.Tq + token) * a.Hq + head;
    to.out = a.out + token * a.o_token + head * a.o_head;
    to.lse = a.lse ? a.lse + (int64_t)head * a.Tq + token : nullptr;
    to.part = a.part + slot * a.D;
    to.ml = a.ml + slot * 2;
  }
  const float c = a.scale * LOG2E;
  if constexpr (BLOCKS == 1) {
    run_streams<T, DP, false, false>(w, keys, a.D, c, lim, lds, Scores{});
    if (a.causal && has_odd_sums(w)) run_streams<T, DP, false, true>(w, keys, a.D, c, lim, lds, Scores{});
  } else {
    run_shared<T, DP, Sh::KB, false>(w, keys, a.D, c, lim, lds);
    if (a.causal && __syncthreads_or(has_odd_sums(w))) run_shared<T, DP, Sh::KB, true>(w, keys, a.D, c, lim, lds);
  }
  finish<T, DP, BLOCKS>(w, to, a.slices > 1, a.D, lds);
}

// --- decode -----------------------------------------------------------------------------------------------------------------

struct DecodeArgs {
  const char *q, *k0, *v0, *k, *v;
  char* out;
  const int32_t* lens;
  float *lse, *part, *ml, *scores, *weight;
  int64_t q_seq, q_head, k0_token, k0_head, v0_token, v0_head, k_seq, k_token, k_head, v_seq, v_token, v_head, o_seq, o_head;  // bytes
  int64_t score_stride;  // floats from row to row of the scores
  int B, Hq, Hkv, G, D, P, C;
  int prefix_tiles, prefix_slices, slice_keys;  // row tiles and slices of the prefix, keys of a slice
  int chunks, chunk_keys, row_blocks;           // of the caches: chunks of a whole one, keys of a chunk, blocks of 32 heads of a group
  int q_wide;                                   // rows of q that are read 16 bytes at a time
  int once;                                     // the caches are more than the chip's own caches hold
  int weight_blocks;                            // of the joining kernel: blocks of 1024 slots
  float scale;
};

__device__ __forceinline__ int slots_in_use(const DecodeArgs& a, int b, int h) { return clamp_to(a.lens[b * a.Hkv + h], a.C); }

// Weights of a workgroup's slots: what the scores of `heads` rows come to now that the rows' sums are known; 4 slots a thread.
// x: the first rows' scores, requested before the sums were known.
constexpr int AHEAD = 8;
__device__ __forceinline__ void request_scores(const float* scores, int64_t stride, int heads, f4 (&x)[AHEAD]) {
#pragma unroll
  for (int g = 0; g < AHEAD; ++g) x[g] = g < heads ? *reinterpret_cast<const f4*>(scores + g * stride) : f4{0.0f, 0.0f, 0.0f, 0.0f};
}
__device__ __forceinline__ f4 sum_weights(const float* scores, int64_t stride, int heads, const f4 (&x)[AHEAD], const float* row_lse, float c) {
  f4 sum = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
  for (int g = 0; g < AHEAD; ++g)
    if (g < heads) {
#pragma unroll
      for (int j = 0; j < 4; ++j) sum[j] += __builtin_amdgcn_exp2f(__builtin_fmaf(x[g][j], c, -row_lse[g]));
    }
#pragma unroll 4
  for (int g = AHEAD; g < heads; ++g) {
    const f4 y = *reinterpret_cast<const f4*>(scores + g * stride);
#pragma unroll
    for (int j = 0; j < 4; ++j) sum[j] += __builtin_amdgcn_exp2f(__builtin_fmaf(y[j], c, -row_lse[g]));
  }
  return sum;
}

// A short prefix and a whole cache in one chunk: at most so many slots, and the scores of at most so many rows in LDS.
constexpr int SHORT = 512, LDS_ROWS = 4;

// One decode step.  Workgroups of the prefix (all rows of a key head, 32 BLOCKS at a time, over one slice of its keys) and of the caches (one sequence
// and key head, one chunk of its slots), the former, longer ones first (mixed, 4 rows over 2047 keys took 13.9 instead of 11.7 us).  Every one
// leaves a part of its rows.  WHOLE: workgroups of the caches only, which take a short prefix first and leave finished rows and, with
// accumulate, the slots' weights.  A tile of 32 rows is
// mostly empty for a group of 8 heads, but caches are bound by memory (24 of 4095 slots, 8 key heads of 128 elements, 403 MB: 78 us,
// 5.2 TB/s, what a large copy reaches), and a prefix fills its tiles (64 rows of 64 heads in groups of 8 over 16384 keys: 46 us, 750 TFLOP/s
// before the parts are joined; a row alone would read 67 MB for itself).
template <typename T, int DP, int BLOCKS, bool WHOLE>
__global__ __launch_bounds__(256, 2) void attn_decode_kernel(const DecodeArgs a) {
  typedef Shape<DP, BLOCKS> ShP;
  typedef Shape<DP, 1> ShO;
  constexpr int LDS = ShP::LDS > ShO::LDS ? ShP::LDS : ShO::LDS;
  __shared__ __align__(1024) char lds[LDS];
  __shared__ float row_lse[WHOLE ? 32 : 1];
  __shared__ __align__(16) float row_scores[WHOLE ? LDS_ROWS * SHORT : 4];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const float c = a.scale * LOG2E;
  Keys keys;
  const int prefix = WHOLE ? 0 : a.Hkv * a.prefix_tiles * a.prefix_slices;
  int id = (int)blockIdx.x - prefix;
  if (!WHOLE && id < 0) {
    id += prefix;
    int h, unit;
    head_and_unit(id, a.Hkv, h, unit);
    const int z = unit / a.prefix_tiles;  // (a slice's tiles side by side: the same keys)
    const int rows = a.B * a.G;
    const Tile tile(unit % a.prefix_tiles, BLOCKS, wave, lane, rows);
    const bool exists = tile.row >= 0;
    const int b = exists ? tile.row / a.G : 0, head = h * a.G + (exists ? tile.row - b * a.G : 0);
    keys.k_stride = a.k0_token;
    keys.v_stride = a.v0_token;
    keys.k = a.k0 + h * a.k0_head;
    keys.v = a.v0 + h * a.v0_head;
    keys.begin = z * a.slice_keys;
    keys.end = min(a.P, keys.begin + a.slice_keys);
    Rows<T, DP> w;
    load_q(w, a.q + b * a.q_seq + head * a.q_head, exists, a.D, lane, a.q_wide);
    Target to = {};
    if (exists) {
      const int64_t row = (int64_t)b * a.Hq + head, slot = (int64_t)z * a.B * a.Hq + row;
      to.out = a.out;
      to.part = a.part + slot * a.D;
      to.ml = a.ml + slot * 2;
    }
    const Limits lim{keys.end, keys.end, keys.end, tile.first <= tile.last ? keys.end : 0};
    if constexpr (BLOCKS == 1) run_streams<T, DP, false, false>(w, keys, a.D, c, lim, lds, Scores{});
    else run_shared<T, DP, ShP::KB, false>(w, keys, a.D, c, lim, lds);
    finish<T, DP, BLOCKS>(w, to, true, a.D, lds);
    return;
  }
  const int h = id % a.Hkv;
  id /= a.Hkv;
  const int b = id % a.B;
  id /= a.B;
  const int block = id % a.row_blocks, chunk = id / a.row_blocks;
  const int g = block * 32 + (lane & 31);
  const bool exists = g < a.G;
  const int head = h * a.G + (exists ? g : 0);
  const int64_t row = (int64_t)b * a.Hq + head;
  Rows<T, DP> w;
  load_q(w, a.q + b * a.q_seq + head * a.q_head, exists, a.D, lane, a.q_wide);  // (on its way while the length is)
  const int n = slots_in_use(a, b, h);
  keys.begin = chunk * a.chunk_keys;
  keys.end = min(n, keys.begin + a.chunk_keys);
  if (!WHOLE && keys.begin >= keys.end) return;
  keys.k_stride = a.k_token;
  keys.v_stride = a.v_token;
  keys.k = a.k + b * a.k_seq + h * a.k_head;
  keys.v = a.v + b * a.v_seq + h * a.v_head;
  keys.once = a.once;
  // the group's rows of scores from this chunk on, in one range (the entry point keeps it below 2^31 bytes)
  Scores scores{};
  const bool in_lds_rows = WHOLE && a.G <= LDS_ROWS;
  if (a.scores && in_lds_rows) {
    if (exists) scores.lds = (uint32_t)(uintptr_t)(TMAC_LDS char*)(char*)(row_scores + g * SHORT);
  } else if (a.scores) {
    const int64_t from = ((int64_t)b * a.Hq + h * a.G + block * 32) * a.score_stride + keys.begin;
    const int rows = min(32, a.G - block * 32);
    scores.base = a.scores + from;
    scores.range = (int)(((rows - 1) * a.score_stride + a.chunk_keys) * 4);
    scores.offset = exists ? (uint32_t)((lane & 31) * a.score_stride * 4) : 0x7fff0000u;
  }
  // (whole rows with weights: the old ones are on their way early; a thread has four slots of at most 512)
  const int slot0 = threadIdx.x * 4;
  float* weight = WHOLE && a.scores ? a.weight + ((int64_t)b * a.Hkv + h) * a.C + slot0 : nullptr;
  float old[4];
#pragma unroll
  for (int j = 0; j < 4; ++j) old[j] = weight && slot0 + j < n ? weight[j] : 0.0f;
  if constexpr (WHOLE) {
    clear(w);
    const Keys shared{a.k0 + h * a.k0_head, a.v0 + h * a.v0_head, a.k0_token, a.v0_token, 0, a.P, false};
    if (a.P) run_streams<T, DP, false, false, true>(w, shared, a.D, c, Limits{a.P, a.P, a.P, a.P}, lds, Scores{});
  }
  run_streams<T, DP, true, false, WHOLE>(w, keys, a.D, c, Limits{keys.end, keys.end, keys.end, keys.end}, lds, scores);
  Target to = {};
  if (exists) {
    const int64_t slot = (int64_t)(a.prefix_slices + chunk) * a.B * a.Hq + row;
    to.out = a.out + b * a.o_seq + head * a.o_head;
    to.lse = a.lse ? a.lse + row : nullptr;
    to.part = a.part + slot * a.D;
    to.ml = a.ml + slot * 2;
  }
  finish<T, DP, 1>(w, to, !WHOLE, a.D, lds, WHOLE ? row_lse : nullptr);
  if (!WHOLE || !weight || slot0 >= n) return;
  // (the scores and row_lse have been written by this workgroup, before the last barrier of `finish`)
  f4 sum = {0.0f, 0.0f, 0.0f, 0.0f};
  if (in_lds_rows) {
    for (int y = 0; y < a.G; ++y) {
      const f4 x = *reinterpret_cast<const f4*>(row_scores + y * SHORT + slot0);
#pragma unroll
      for (int j = 0; j < 4; ++j) sum[j] += __builtin_amdgcn_exp2f(__builtin_fmaf(x[j], c, -row_lse[y]));
    }
  } else {
    const float* s = a.scores + ((int64_t)b * a.Hq + h * a.G) * a.score_stride + slot0;
    f4 x[AHEAD];
    request_scores(s, a.score_stride, a.G, x);
    sum = sum_weights(s, a.score_stride, a.G, x, row_lse, c);
  }
#pragma unroll
  for (int j = 0; j < 4; ++j)
    if (slot0 + j < n) weight[j] = old[j] + sum[j];
}

// --- parts of rows ------------------------------------------------------------------------------------------------------------

struct Joined {
  float top, sum;  // largest of what the parts' sums are taken against, sum of exponentials against it
};

// Of a row's n parts, one wavefront.
__device__ __forceinline__ Joined join(const float* ml, int64_t stride, int n, int lane) {
  float top = -INFINITY;
  for (int i = lane; i < n; i += 64) top = fmaxf(top, ml[i * stride]);
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor(top, o));
  float sum = 0.0f;
  for (int i = lane; i < n; i += 64) {
    const f2 x = *reinterpret_cast<const f2*>(ml + i * stride);
    sum += x[0] == top ? x[1] : x[1] * __builtin_amdgcn_exp2f(x[0] - top);
  }
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) sum += __shfl_xor(sum, o);
  return {top, sum};
}

template <typename T>
__device__ __forceinline__ void join_row(const float* part, const float* ml, int64_t rows, int64_t row, int n, int D, char* out, float* lse,
                                         int lane) {
  const Joined j = join(ml + row * 2, rows * 2, n, lane);
  f2 x = {0.0f, 0.0f};
  const int at = lane * 2;
  if (at < D) {
#pragma unroll 4
    for (int i = 0; i < n; ++i) {
      const float m = ml[(i * rows + row) * 2];
      const float a = m == j.top ? 1.0f : __builtin_amdgcn_exp2f(m - j.top);
      x += *reinterpret_cast<const f2*>(part + (i * rows + row) * D + at) * a;
    }
    const float inv = j.sum == 0.0f ? 0.0f : 1.0f / j.sum;
    typedef typename T::elem e2 __attribute__((ext_vector_type(2)));
    *reinterpret_cast<e2*>(out + at * 2) = __builtin_convertvector(x * inv, e2);
  }
  if (lane == 0 && lse) *lse = j.sum == 0.0f ? -INFINITY : log2_sum<T>(j.top, j.sum) * LN2;
}

// One wavefront a row: about 4 us, what a launch with a chain of two loads takes (128 rows after 8192 keys, 32 heads).
template <typename T>
__global__ __launch_bounds__(256) void join_prompt_kernel(const PromptArgs a) {
  const int64_t rows = (int64_t)a.Tq * a.Hq, row = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
  if (row >= rows) return;
  const int64_t token = row / a.Hq, head = row % a.Hq;
  join_row<T>(a.part, a.ml, rows, row, a.slices, a.D, a.out + token * a.o_token + head * a.o_head,
              a.lse ? a.lse + head * a.Tq + token : nullptr, threadIdx.x & 63);
}

// Rows, then (where weights are wanted) 1024 slots of a sequence and key head a workgroup: the scores that the decode kernel
// left become weights now that the rows' sums are known.  (24 caches of 4095 slots, 64 heads: 25 MB of scores, 6 MB of parts and 3 MB of
// weights 10 us, of which the first 4 are what a launch with a chain of loads takes.)
template <typename T>
__global__ __launch_bounds__(256) void join_decode_kernel(const DecodeArgs a) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int64_t rows = (int64_t)a.B * a.Hq;
  const int row_wgs = (int)((rows + 3) / 4);
  if ((int)blockIdx.x < row_wgs) {
    const int64_t row = (int64_t)blockIdx.x * 4 + wave;
    if (row >= rows) return;
    const int64_t b = row / a.Hq, head = row % a.Hq;
    const int n = a.C ? (slots_in_use(a, (int)b, (int)head / a.G) + a.chunk_keys - 1) / a.chunk_keys : 0;
    join_row<T>(a.part, a.ml, rows, row, a.prefix_slices + n, a.D, a.out + b * a.o_seq + head * a.o_head, a.lse ? a.lse + row : nullptr,
                lane);
    return;
  }
  const int id = blockIdx.x - row_wgs, bh = id % (a.B * a.Hkv), block = id / (a.B * a.Hkv);
  const int b = bh / a.Hkv, h = bh % a.Hkv, n = slots_in_use(a, b, h);
  if (block * 1024 >= n) return;
  const float c = a.scale * LOG2E;
  __shared__ float row_lse[128];
  const int at = block * 1024 + threadIdx.x * 4;
  float* weight = a.weight + (int64_t)bh * a.C + at;
  float old[4];
#pragma unroll
  for (int j = 0; j < 4; ++j) old[j] = at + j < n ? weight[j] : 0.0f;
  f4 sum = {0.0f, 0.0f, 0.0f, 0.0f};
  for (int g0 = 0; g0 < a.G; g0 += 128) {
    const int heads = min(128, a.G - g0);
    const float* s = a.scores + ((int64_t)b * a.Hq + h * a.G + g0) * a.score_stride + at;
    f4 x[AHEAD];
    request_scores(s, a.score_stride, at < n ? heads : 0, x);
    if (g0) __syncthreads();
    for (int g = wave; g < heads; g += 4) {
      const int64_t row = (int64_t)b * a.Hq + h * a.G + g0 + g;
      const Joined j = join(a.ml + row * 2, rows * 2, a.prefix_slices + (n + a.chunk_keys - 1) / a.chunk_keys, lane);
      // (a row without a score above -inf gives no weights)
      if (lane == 0) row_lse[g] = j.sum == 0.0f ? INFINITY : log2_sum<T>(j.top, j.sum);
    }
    __syncthreads();
    if (at < n) sum += sum_weights(s, a.score_stride, heads, x, row_lse, c);
  }
#pragma unroll
  for (int j = 0; j < 4; ++j)
    if (at + j < n) weight[j] = old[j] + sum[j];
}

// --- weights of a prompt's keys -----------------------------------------------------------------------------------------------

struct WeightArgs {
  const char *q, *k;
  const float* lse;
  const int32_t *cu_q, *cu_k;
  float *weight, *part;
  int64_t q_token, q_head, k_token, k_head;  // bytes
  int S, Tq, Tk, Hq, Hkv, G, D, causal, tiles, slices;
  float scale;
};

// One workgroup: 128 KB keys of one sequence and key head, 32 KB a wavefront, which stay in registers as the second operand of
// S = Q K^T; a lane owns a key (of each 32) and adds up exp(s - lse) over the queries that pass through LDS, 64 of one head at a time.
// Products and exponentials (16 a lane for 8 products of 32 x 32 x 16) take turns within a wavefront, and the two wavefronts of a SIMD overlap
// them only in part: 6144 tokens, 64 heads in groups of 8 of 128 elements take 322 to 338 us, 0.95 PFLOP/s of the pairs that are seen, matrix
// units 49 % busy and vector ALUs 62 % at 1.8 of 2.4 GHz.  What is not either is kept away from the vector ALUs: with two blocks of keys
// a wavefront the reads of q and of lse serve twice.  Nothing is added up atomically: a unit's sums go to memory once, those of its slices
// to a part each.
template <typename T, int DP, int KB>
__global__ __launch_bounds__(256, 2) void attn_weights_kernel(const WeightArgs a) {
  constexpr int SQ = 64, TILE = Layout<DP>::k_bytes(SQ), NT = DP / 16, KEYS = 128 * KB;
  __shared__ __align__(1024) char lds[2 * TILE];
  __shared__ __align__(16) float lse2[2][SQ];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), half = lane >> 5;
  int h, unit;
  head_and_unit(blockIdx.x, a.Hkv, h, unit);
  const int z = unit % a.slices;
  Place p;
  if (!find_tile(a.cu_q, a.cu_k, a.S, a.Tq, a.Tk, true, 1, KEYS, unit / a.slices, p)) return;
  const int k0 = p.k0, nk = p.nk, q0 = p.q0, nq = p.nq;
  const int off = nk - nq;                       // query i sees keys up to i + off
  const int j0 = p.tile * KEYS + wave * 32 * KB;  // the wavefront's first key
  // queries that see the tile's first key, in stages of 64, head after head; this slice's share of the stages
  const int first = a.causal ? min(nq, max(0, p.tile * KEYS - off)) / SQ * SQ : 0;
  const int stages = (nq - first + SQ - 1) / SQ;
  const int total = stages * a.G, from = (int)((int64_t)total * z / a.slices), to = (int)((int64_t)total * (z + 1) / a.slices);
  const float c = a.scale * LOG2E;
  const uint32_t lds0 = (uint32_t)(uintptr_t)(TMAC_LDS char*)lds;
  // The keys pass through the room of the queries, a wavefront's 32 at a time in a quarter of it: as rows, which memory gives whole (read
  // 8 bytes here and there by the lanes that need them they took 10 of a small call's 19 us).
  typename T::v8 kf[KB][NT];
  {
    const Stage<DP, 32, 1, false> ks(a.k_token, a.D, wave, lane);
    const uint32_t mine = lds0 + wave * Layout<DP>::k_bytes(32);
    const Reads<DP> reads(mine, 0, lane);
#pragma unroll
    for (int y = 0; y < KB; ++y) {
      const char* base = a.k + (int64_t)(k0 + min(nk, j0 + y * 32)) * a.k_token + h * a.k_head;
      const int there = nk - j0 - y * 32;
      ks.load(base, a.k_token, there, a.D, mine, wave);
      const u2 tail = load_tail<32>(base, a.k_token, there, a.D, lane);
      asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
      store_tail<DP, 32>(tail, a.D, mine, lane);
#pragma unroll
      for (int t = 0; t < NT; ++t) kf[y][t] = read_k<T>(reads.k_at(t));
      asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    }
  }
  __syncthreads();
  clear_pads<DP>(a.D, lds0, 2 * TILE, tid);
  const Stage<DP, SQ, 4, false> qs(a.q_token, a.D, wave, lane);
  const Reads<DP> reads(lds0, 0, lane);
  float next_lse = 0.0f;
  u2 next_tail = {0u, 0u};
  auto load = [&](int g, int i0, int buf) {
    const int head = h * a.G + g;
    const char* base = a.q + (int64_t)(q0 + i0) * a.q_token + head * a.q_head;
    qs.load(base, a.q_token, nq - i0, a.D, lds0 + buf * TILE, wave);
    next_tail = load_tail<SQ>(base, a.q_token, nq - i0, a.D, tid);
    if (tid < SQ) next_lse = i0 + tid < nq ? a.lse[(int64_t)head * a.Tq + q0 + i0 + tid] : -INFINITY;
  };
  // rows that are not there, or see nothing, give exp(s - inf) = 0
  auto settle = [&](int buf) {
    store_tail<DP, SQ>(next_tail, a.D, lds0 + buf * TILE, tid);
    if (tid < SQ) lse2[buf][tid] = next_lse == -INFINITY ? INFINITY : next_lse * LOG2E;
  };
  float sum[KB];
#pragma unroll
  for (int y = 0; y < KB; ++y) sum[y] = 0.0f;
  int g = 0, i0 = 0;  // head and first query of the stage
  if (from < to) {
    g = from / stages;
    i0 = first + (from - g * stages) * SQ;
    load(g, i0, 0);
    settle(0);
  }
  for (int s = from; s < to; ++s) {
    const int buf = (s - from) & 1;
    const int now = i0;
    wait_stage();
    i0 += SQ;
    if (i0 >= nq) i0 = first, ++g;
    if (s + 1 < to) load(g, i0, buf ^ 1);
    // some query does not see some key, or is not there (zeros times an infinite key would be NaN)
    const bool mask = (a.causal && j0 + 32 * KB - 1 > now + off) || now + SQ > nq;
    // the stage's part of the sums; masked: as a stage of its own, which the others are not to pay for
    auto add = [&](auto masked) {
#pragma unroll
      for (int b = 0; b < SQ / 32; ++b) {
        f16x x[KB];
#pragma unroll
        for (int y = 0; y < KB; ++y) x[y] = (f16x)(0.0f);
#pragma unroll
        for (int t = 0; t < NT; ++t) {
          const auto q = read_k<T>(reads.k_at(t) + buf * TILE + b * (TILE / 2));
#pragma unroll
          for (int y = 0; y < KB; ++y) x[y] = T::mfma(q, kf[y][t], x[y]);
        }
        f4 l[4];
#pragma unroll
        for (int r = 0; r < 4; ++r) l[r] = *reinterpret_cast<const f4*>(&lse2[buf][b * 32 + r * 8 + half * 4]);
#pragma unroll
        for (int y = 0; y < KB; ++y) {
          f4 part = {0.0f, 0.0f, 0.0f, 0.0f};
          // (the lane's key is seen by the queries from one row of the block on, up to the last)
          const int row0 = now + b * 32 + half * 4, seen_from = a.causal ? j0 + y * 32 + (lane & 31) - off - row0 : 0, last = nq - row0;
#pragma unroll
          for (int r = 0; r < 4; ++r)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              float e = __builtin_amdgcn_exp2f(__builtin_fmaf(x[y][4 * r + i], c, -l[r][i]));
              if constexpr (masked) e = r * 8 + i >= seen_from && r * 8 + i < last ? e : 0.0f;
              part[i] += e;
            }
          sum[y] += (part[0] + part[1]) + (part[2] + part[3]);
        }
      }
    };
    if (mask) {
      if (!(a.causal && j0 > now + SQ - 1 + off)) add(std::true_type{});  // (else no query of the stage sees a key of the wavefront)
    } else {
      add(std::false_type{});
    }
    if (s + 1 < to) settle(buf ^ 1);
  }
#pragma unroll
  for (int y = 0; y < KB; ++y) {
    const int j = j0 + y * 32 + (lane & 31);
    const float x = add_halves(sum[y]);
    if (half == 0 && j < nk) (a.slices > 1 ? a.part + ((int64_t)z * a.Hkv + h) * a.Tk : a.weight + (int64_t)h * a.Tk)[k0 + j] = x;
  }
}

// Slices' parts, in their order (4 us, a launch with one chain of loads).
__global__ __launch_bounds__(256) void sum_weights_kernel(const float* part, float* weight, int64_t n, int slices) {
  const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (i >= n) return;
  float x = 0.0f;
  for (int z = 0; z < slices; ++z) x += part[z * n + i];
  weight[i] = x;
}

// --- host -----------------------------------------------------------------------------------------------------------------------

static bool desc_ok(const tmac_attn_desc* d) {
  return d && d->Hq > 0 && d->Hkv > 0 && d->Hq % d->Hkv == 0 && d->D > 0 && d->D % 4 == 0 && std::isfinite(d->scale) && d->scale > 0.0f &&
         (d->elem == TMAC_ELEM_F16 || d->elem == TMAC_ELEM_BF16) && (d->causal == 0 || d->causal == 1) && !d->reserved[0] && !d->reserved[1];
}

constexpr int WGS = 512;  // workgroups that the chip holds at once, two on a CU

// Rows of a workgroup: 128 share each stage of keys, 32 let the wavefronts share the keys instead, for sequences of at most 32 rows (32
// of 8 rows after 1000 keys, 8 key heads: 24.7 us with 32, 28.6 with 128; 32 of 64 rows, 32 heads: 32.0 and 21.7) and where the last row's
// walk over its keys, four times as long with 128 rows, would take longer than the four times as many workgroups of 32: those take about
// (6 + seen keys / 80) us for each 128 of 128 rows' number, the walk (5 + keys / 46) us; where half of the chip would stay idle, always (8 heads, 4096 tokens: 61.8 us with 32, 86.8 with 128, 6000
// 120 and 134, 8192 209 and 208; 32 heads, 1024 tokens 26.8 and 27.9, 1600 50.6 and 42.8; 64 in groups of 8, 512 tokens 20.5 and 18.2; 2 key heads with
// 3 each, 3026, 1400, 700, 300 and 90 tokens 39.2 and 62.6; 40 heads, 256 tokens 10.0 and 13.1).
// Slices: as many as it takes to fill the chip, none shorter than 256 keys, if that saves the walk over 768 keys or more, since the
// parts are joined by another launch (16 rows after 4096 keys: 14.1 us in 16 slices, 15.0 in 8; 1000 rows, 8 heads in groups of 4:
// 18.2 us in two, 14.3 in one).
struct PromptPlan {
  int blocks, tiles, slices;
  size_t part, ml, bytes;
};
static PromptPlan prompt_plan(const tmac_attn_desc* d, int S, int Tq, int Tk) {
  PromptPlan p;
  const int64_t G = d->Hq / d->Hkv, rows = Tq * G;
  auto tiles_of = [&](int per) { return (int)std::min<int64_t>(rows / per + S, rows); };
  const int64_t keys = Tk / S, seen = d->causal ? std::max(keys / 2, keys - Tq / S / 2) : keys;
  const int64_t wide = (int64_t)tiles_of(128) * d->Hkv;
  // (wide / 128 (6 + seen / 80) against 5 + keys / 46, both 128 * 80 times)
  p.blocks = rows / S <= 32 || wide < WGS / 2 || wide * (480 + seen) <= 51200 + 224 * keys ? 1 : 4;
  p.tiles = tiles_of(32 * p.blocks);
  const int64_t wgs = (int64_t)p.tiles * d->Hkv;
  p.slices = (int)std::max<int64_t>(1, std::min<int64_t>({WGS / wgs, (Tk / S) / 256, 64}));
  if (Tk / S - Tk / S / p.slices < 768) p.slices = 1;
  p.part = p.slices > 1 ? (size_t)p.slices * Tq * d->Hq * d->D * 4 : 0;
  p.ml = p.slices > 1 ? (size_t)p.slices * Tq * d->Hq * 8 : 0;
  p.bytes = p.part + p.ml;
  return p;
}

// Blocks of 32 keys a wavefront: two, once that leaves enough units (each key tile's stages) for the chip; the reads of q then serve twice
// (6144 tokens, 64 heads in groups of 8: 379 us with one, 337 with two; five prompts of up to 777 tokens 17.5 and 20.2).  Slices of a tile's
// stages: twice the workgroups that the chip holds, up to four times while eight stages are left to each, because tiles weigh unlike but a
// workgroup's start costs as much as four stages or more (6144 tokens: 605 us at one time, 351 at two, 331 at four, 332 at eight; 12 of 327 tokens, 16
// heads of one key head 27.1 at four times, 19.4 so; 2000 tokens, 32 heads in groups of 4 38.6 and 32.1; 1024 tokens, 32 heads 17.0 and 14.1; three of
// 1000 27.6 and 28.3), none shorter than two stages (five of up to 777 17.5 us; four 21.6, one 20.2).
struct WeightsPlan {
  int blocks, tiles, slices;
  size_t bytes;
};
static WeightsPlan weights_plan(const tmac_attn_desc* d, int S, int Tq, int Tk) {
  WeightsPlan p;
  const int64_t stages = (int64_t)(Tq / S + 63) / 64 * (d->Hq / d->Hkv);
  auto tiles_of = [&](int per) { return (int)std::min<int64_t>(Tk / per + S, Tk); };
  p.blocks = (int64_t)tiles_of(256) * d->Hkv * stages >= 8192 ? 2 : 1;
  p.tiles = tiles_of(128 * p.blocks);
  const int64_t wgs = (int64_t)p.tiles * d->Hkv;
  p.slices = (int)std::max<int64_t>(1, std::min<int64_t>({4 * WGS / wgs, std::max<int64_t>(2 * WGS / wgs, stages / 8), stages / 2, 64}));
  p.bytes = p.slices > 1 ? (size_t)p.slices * d->Hkv * Tk * 4 : 0;
  return p;
}

struct DecodePlan {
  int blocks, tiles, slices, slice_keys, chunks, chunk_keys, row_blocks;
  bool whole_rows;
  int64_t score_stride;
  size_t part, ml, scores, bytes;
};
static DecodePlan decode_plan(const tmac_attn_desc* d, int B, int C, int P, bool accumulate) {
  DecodePlan p = {};
  const int64_t G = d->Hq / d->Hkv, rows = B * G;
  p.row_blocks = (int)((G + 31) / 32);
  if (C) {
    // Chunks of 128 to 512 slots, so that a long cache beside short ones is shared by many workgroups, by the rounds that full
    // caches take times what a round costs: its slots and about 96 more for the start, the meeting and the parts.
    const int64_t units = (int64_t)B * d->Hkv * p.row_blocks;
    int64_t best = INT64_MAX;
    for (int keys = 128; keys <= 512; keys += 128) {
      const int64_t cost = (units * ((C + keys - 1) / keys) + WGS - 1) / WGS * (keys + 96);
      if (cost < best) best = cost, p.chunk_keys = keys;
    }
    // A short cache in one chunk, after a short prefix, has nothing to join, which saves a launch (about 4 us, and what is between two).  Where
    // caches fill half of the chip, up to 512 keys of prefix in all rounds of workgroups (64 caches of 60 and of 500 slots, 8 key heads, 100 keys:
    // 12.0 and 20.7 us instead of 18.8 and 26.5; 512 keys 16.1 and 24.2 instead of 18.9 and 26.4; 1000 keys 21.6 and 29.2 instead of 21.0 and
    // 26.9); elsewhere, where the chip has room to walk them side by side, up to 512 of prefix and cache (4 caches of 60 slots, 8 key heads, 100
    // keys 10.0 instead of 12.5, 400 keys 13.4 instead of 14.5; of 500 slots, 200 keys 14.5 instead of 12.9).
    const int64_t rounds = (units + WGS - 1) / WGS;
    p.whole_rows = C <= SHORT && p.row_blocks == 1 && (2 * units >= WGS ? rounds * P : (int64_t)P + C) <= 512;
    if (p.whole_rows) p.chunk_keys = (C + 127) / 128 * 128;
    p.chunks = (C + p.chunk_keys - 1) / p.chunk_keys;
  }
  // Rows of the prefix's workgroups: 32, whose wavefronts share the keys, while that makes no more than 768 keys for each of the
  // workgroups that the chip holds, else 128 (8 key heads, 128 rows over 4000 keys: 15.7 us with 32, 19.2 with 128; over 16000 28.2 both; 512
  // rows over 16000 76.9 and 59.0; 32 key heads, 64 rows over 4000 23.7 and 27.9, over 16000 57.4 and 54.7).
  p.blocks = rows <= 32 || (rows + 31) / 32 * d->Hkv * P <= WGS * 768 ? 1 : 4;
  if (P && !p.whole_rows) {
    p.tiles = (int)((rows + 32 * p.blocks - 1) / (32 * p.blocks));
    // Slices until the prefix fills the chip, or beside caches half of it (64 rows over 16384 keys, 8 key heads of 128 elements, 64 caches
    // of 1024 slots: 84 us with all of it, 73 with half; without caches 50.6 and 52.7), none shorter than 256 keys.
    const int64_t slices = std::max<int64_t>(1, std::min<int64_t>({(C ? WGS / 2 : WGS) / ((int64_t)p.tiles * d->Hkv), P / 256, 64}));
    p.slice_keys = (int)((P + slices - 1) / slices + 127) / 128 * 128;
    p.slices = (P + p.slice_keys - 1) / p.slice_keys;
  }
  const size_t R = (size_t)B * d->Hq, parts = (size_t)p.slices + p.chunks;
  p.part = parts * R * d->D * 4;
  p.ml = parts * R * 8;
  p.score_stride = (int64_t)p.chunks * p.chunk_keys;
  p.scores = accumulate ? R * p.score_stride * 4 : 0;
  p.bytes = p.part + p.ml + p.scores + 32;
  return p;
}

template <typename Args>
static tmac_status launch(const void* kernel, int64_t grid, const Args& args, void* stream) {
  if (grid <= 0) return TMAC_OK;
  if (!launchable(grid, 256)) return TMAC_EUNSUPPORTED;
  Args a = args;
  void* ptrs[] = {&a};
  const hipError_t e = hipLaunchKernel(kernel, dim3((unsigned)grid), dim3(256), ptrs, 0, static_cast<hipStream_t>(stream));
  if (e == hipSuccess) return TMAC_OK;
  note_hip_error((int)e);
  return TMAC_EHIP;
}

template <typename T, int DP>
static const void* prompt_kernel(int blocks) {
  return blocks == 4 ? (const void*)attn_prompt_kernel<T, DP, 4> : (const void*)attn_prompt_kernel<T, DP, 1>;
}
template <typename T, int DP>
static const void* decode_kernel(int blocks) {  // 0: whole rows
  return blocks == 4   ? (const void*)attn_decode_kernel<T, DP, 4, false>
         : blocks == 1 ? (const void*)attn_decode_kernel<T, DP, 1, false>
                       : (const void*)attn_decode_kernel<T, DP, 1, true>;
}
template <typename T, int DP>
static const void* weights_kernel(int blocks) {
  return blocks == 2 ? (const void*)attn_weights_kernel<T, DP, 2> : (const void*)attn_weights_kernel<T, DP, 1>;
}
// Kernel for the type and the row length of a call, rows being padded to 64 or 128 elements in LDS.
#define TMAC_PICK(f, d, blocks)                                                              \
  ((d)->elem == TMAC_ELEM_F16 ? ((d)->D <= 64 ? f<F16, 64>(blocks) : f<F16, 128>(blocks))       \
                              : ((d)->D <= 64 ? f<BF16, 64>(blocks) : f<BF16, 128>(blocks)))

static bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15) == 0; }

}  // namespace attn
}  // namespace tmac

using namespace tmac;
using namespace tmac::attn;

extern "C" size_t tmac_attn_prompt_workspace_bytes(const tmac_attn_desc* desc, int32_t S, int32_t Tq, int32_t Tk) {
  if (!desc_ok(desc) || desc->D > 128 || S <= 0 || Tq <= 0 || Tk <= 0 || long_axis(S) || long_axis(Tq) || long_axis(Tk)) return 0;
  return prompt_plan(desc, S, Tq, Tk).bytes;
}

extern "C" tmac_status tmac_attn_prompt(const tmac_attn_desc* desc, const tmac_view* q, const tmac_view* k, const tmac_view* v, int32_t S,
                                        int32_t Tq, int32_t Tk, const int32_t* cu_q_dev, const int32_t* cu_k_dev, const tmac_view* out,
                                        float* lse_dev, void* workspace_dev, size_t workspace_bytes, void* stream) {
  if (!desc_ok(desc) || S < 0 || Tq < 0 || Tk < 0) return TMAC_EINVAL;
  if (S == 0 || Tq == 0) return TMAC_OK;
  if (!rows_ok(q, false, true, true) || !rows_ok(out, false, true, true) || !cu_q_dev || !cu_k_dev) return TMAC_EINVAL;
  if (Tk > 0 && (!rows_ok(k, false, true, true) || !rows_ok(v, false, true, true))) return TMAC_EINVAL;
  if (desc->D > 128 || (int64_t)Tq * desc->Hq > 0x7fffffff || long_axis(S) || long_axis(Tq) || long_axis(Tk)) return TMAC_EUNSUPPORTED;
  const tmac_view none = {};
  if (Tk == 0) k = v = &none;
  if (far_rows(k) || far_rows(v)) return TMAC_EUNSUPPORTED;
  PromptPlan p = prompt_plan(desc, S, Tq, std::max(Tk, 1));
  if (p.bytes) {
    if (!workspace_dev || !aligned16(workspace_dev)) return TMAC_EINVAL;
    if (workspace_bytes < p.bytes) return TMAC_ESIZE;
  }
  PromptArgs a = {};
  a.q = static_cast<const char*>(q->data), a.k = static_cast<const char*>(k->data), a.v = static_cast<const char*>(v->data);
  a.out = static_cast<char*>(out->data);
  a.cu_q = cu_q_dev, a.cu_k = cu_k_dev, a.lse = lse_dev;
  a.part = static_cast<float*>(workspace_dev);
  a.ml = a.part ? a.part + p.part / 4 : nullptr;
  a.q_token = q->token * 2, a.q_head = q->head * 2, a.k_token = k->token * 2, a.k_head = k->head * 2;
  a.v_token = v->token * 2, a.v_head = v->head * 2, a.o_token = out->token * 2, a.o_head = out->head * 2;
  a.S = S, a.Tq = Tq, a.Tk = Tk, a.Hq = desc->Hq, a.Hkv = desc->Hkv, a.G = desc->Hq / desc->Hkv, a.D = desc->D;
  a.causal = desc->causal, a.tiles = p.tiles, a.slices = p.slices, a.scale = desc->scale;
  a.q_wide = wide_rows(q, desc->D);
  const int64_t join_grid = p.slices > 1 ? ((int64_t)Tq * desc->Hq + 3) / 4 : 0;
  if (!launchable(join_grid, 256)) return TMAC_EUNSUPPORTED;
  const tmac_status st = launch(TMAC_PICK(prompt_kernel, desc, p.blocks), (int64_t)p.tiles * p.slices * desc->Hkv, a, stream);
  if (st != TMAC_OK) return st;
  return launch(desc->elem == TMAC_ELEM_F16 ? (const void*)join_prompt_kernel<F16> : (const void*)join_prompt_kernel<BF16>, join_grid, a, stream);
}

extern "C" size_t tmac_attn_weights_workspace_bytes(const tmac_attn_desc* desc, int32_t S, int32_t Tq, int32_t Tk) {
  if (!desc_ok(desc) || desc->D > 128 || S <= 0 || Tq <= 0 || Tk <= 0 || long_axis(S) || long_axis(Tq) || long_axis(Tk)) return 0;
  return weights_plan(desc, S, Tq, Tk).bytes;
}

extern "C" tmac_status tmac_attn_weights(const tmac_attn_desc* desc, const tmac_view* q, const tmac_view* k, const float* lse_dev,
                                         int32_t S, int32_t Tq, int32_t Tk, const int32_t* cu_q_dev, const int32_t* cu_k_dev,
                                         float* weight_dev, void* workspace_dev, size_t workspace_bytes, void* stream) {
  if (!desc_ok(desc) || S < 0 || Tq < 0 || Tk < 0) return TMAC_EINVAL;
  if (S == 0 || Tk == 0) return TMAC_OK;
  if (!rows_ok(k, false, true, true) || !cu_q_dev || !cu_k_dev || !weight_dev) return TMAC_EINVAL;
  if (Tq > 0 && (!rows_ok(q, false, true, true) || !lse_dev)) return TMAC_EINVAL;
  if (desc->D > 128 || (int64_t)Tq * desc->Hq > 0x7fffffff || long_axis(S) || long_axis(Tq) || long_axis(Tk)) return TMAC_EUNSUPPORTED;
  const tmac_view none = {};
  if (Tq == 0) q = &none;
  if (far_rows(q) || far_rows(k)) return TMAC_EUNSUPPORTED;
  const WeightsPlan p = weights_plan(desc, S, Tq, Tk);
  if (p.bytes) {
    if (!workspace_dev || !aligned16(workspace_dev)) return TMAC_EINVAL;
    if (workspace_bytes < p.bytes) return TMAC_ESIZE;
  }
  WeightArgs a = {};
  a.q = static_cast<const char*>(q->data), a.k = static_cast<const char*>(k->data);
  a.lse = lse_dev, a.cu_q = cu_q_dev, a.cu_k = cu_k_dev, a.weight = weight_dev, a.part = static_cast<float*>(workspace_dev);
  a.q_token = q->token * 2, a.q_head = q->head * 2, a.k_token = k->token * 2, a.k_head = k->head * 2;
  a.S = S, a.Tq = Tq, a.Tk = Tk, a.Hq = desc->Hq, a.Hkv = desc->Hkv, a.G = desc->Hq / desc->Hkv, a.D = desc->D;
  a.causal = desc->causal, a.tiles = p.tiles, a.slices = p.slices, a.scale = desc->scale;
  const int64_t n = (int64_t)desc->Hkv * Tk;
  if (p.slices > 1 && !launchable((n + 255) / 256, 256)) return TMAC_EUNSUPPORTED;
  const tmac_status st =
      launch(TMAC_PICK(weights_kernel, desc, p.blocks), (int64_t)p.tiles * p.slices * desc->Hkv, a, stream);
  if (st != TMAC_OK || p.slices == 1) return st;
  int64_t n_arg = n;
  int slices = p.slices;
  void* ptrs[] = {&a.part, &a.weight, &n_arg, &slices};
  const hipError_t e = hipLaunchKernel((const void*)sum_weights_kernel, dim3((unsigned)((n + 255) / 256)), dim3(256), ptrs, 0,
                                       static_cast<hipStream_t>(stream));
  if (e == hipSuccess) return TMAC_OK;
  note_hip_error((int)e);
  return TMAC_EHIP;
}

static bool decode_sizes_ok(const tmac_attn_desc* d, const tmac_cache* c, int32_t P, int32_t accumulate) {
  return desc_ok(d) && c && c->B >= 0 && c->capacity >= 0 && P >= 0 && (accumulate == 0 || accumulate == 1) && c->Hkv == d->Hkv &&
         c->D == d->D && c->elem == d->elem && !c->reserved[0] && !c->reserved[1];
}

extern "C" size_t tmac_attn_decode_workspace_bytes(const tmac_attn_desc* desc, const tmac_cache* cache, int32_t P, int32_t accumulate) {
  if (!decode_sizes_ok(desc, cache, P, accumulate) || desc->D > 128 || cache->B == 0 || long_axis(cache->capacity) || long_axis(P)) return 0;
  return decode_plan(desc, cache->B, cache->capacity, P, accumulate).bytes;
}

extern "C" tmac_status tmac_attn_decode(const tmac_attn_desc* desc, const tmac_view* q, const tmac_view* k0, const tmac_view* v0, int32_t P,
                                        const tmac_cache* cache, int32_t accumulate, const tmac_view* out, float* lse_dev,
                                        void* workspace_dev, size_t workspace_bytes, void* stream) {
  if (!decode_sizes_ok(desc, cache, P, accumulate)) return TMAC_EINVAL;
  const int B = cache->B, C = cache->capacity;
  if (B == 0) return TMAC_OK;
  if (!rows_ok(q, true, false, true) || !rows_ok(out, true, false, true)) return TMAC_EINVAL;
  if (P > 0 && (!rows_ok(k0, false, true, true) || !rows_ok(v0, false, true, true))) return TMAC_EINVAL;
  if (C > 0 && (!rows_ok(&cache->k, true, true, true) || !rows_ok(&cache->v, true, true, true) || !cache->lens_dev)) return TMAC_EINVAL;
  if (C > 0 && accumulate && !cache->weight_dev) return TMAC_EINVAL;
  if (desc->D > 128 || (int64_t)B * desc->Hq > 0x7fffffff || long_axis(C) || long_axis(P)) return TMAC_EUNSUPPORTED;
  const tmac_view none = {};
  if (P == 0) k0 = v0 = &none;
  const tmac_view* k = C ? &cache->k : &none;
  const tmac_view* v = C ? &cache->v : &none;
  if (far_rows(k0) || far_rows(v0) || far_rows(k) || far_rows(v)) return TMAC_EUNSUPPORTED;
  const DecodePlan p = decode_plan(desc, B, C, P, accumulate);
  if (accumulate && std::min(32, desc->Hq / desc->Hkv) * p.score_stride >= 0x1fff0000) return TMAC_EUNSUPPORTED;
  if (!workspace_dev || !aligned16(workspace_dev)) return TMAC_EINVAL;
  if (workspace_bytes < p.bytes) return TMAC_ESIZE;
  DecodeArgs a = {};
  a.q = static_cast<const char*>(q->data), a.k0 = static_cast<const char*>(k0->data), a.v0 = static_cast<const char*>(v0->data);
  a.k = static_cast<const char*>(k->data), a.v = static_cast<const char*>(v->data), a.out = static_cast<char*>(out->data);
  a.lens = cache->lens_dev, a.lse = lse_dev, a.weight = cache->weight_dev;
  a.scores = accumulate && C ? static_cast<float*>(workspace_dev) : nullptr;
  a.part = reinterpret_cast<float*>(static_cast<char*>(workspace_dev) + p.scores);
  a.ml = a.part + p.part / 4;
  a.q_seq = q->seq * 2, a.q_head = q->head * 2, a.o_seq = out->seq * 2, a.o_head = out->head * 2;
  a.k0_token = k0->token * 2, a.k0_head = k0->head * 2, a.v0_token = v0->token * 2, a.v0_head = v0->head * 2;
  a.k_seq = k->seq * 2, a.k_token = k->token * 2, a.k_head = k->head * 2;
  a.v_seq = v->seq * 2, a.v_token = v->token * 2, a.v_head = v->head * 2;
  a.score_stride = p.score_stride;
  a.B = B, a.Hq = desc->Hq, a.Hkv = desc->Hkv, a.G = desc->Hq / desc->Hkv, a.D = desc->D, a.P = P, a.C = C;
  a.prefix_tiles = p.tiles, a.prefix_slices = p.slices, a.slice_keys = p.slice_keys;
  a.chunks = p.chunks, a.chunk_keys = std::max(1, p.chunk_keys), a.row_blocks = p.row_blocks;
  a.q_wide = wide_rows(q, desc->D);
  // (24 caches of 4095 slots, 400 MB: 107 us a step where they are kept, 99.6 where they are not; a prefix of 42 MB 11.6 and 14.3)
  a.once = (int64_t)B * desc->Hkv * C * desc->D * 4 > (256 << 20);
  a.weight_blocks = a.scores ? (C + 1023) / 1024 : 0;
  a.scale = desc->scale;
  const int64_t grid = (int64_t)p.tiles * p.slices * desc->Hkv + (int64_t)B * desc->Hkv * p.row_blocks * p.chunks;
  const int64_t join_grid = p.whole_rows ? 0 : ((int64_t)B * desc->Hq + 3) / 4 + (int64_t)a.weight_blocks * B * desc->Hkv;
  if (!launchable(join_grid, 256)) return TMAC_EUNSUPPORTED;
  const tmac_status st = launch(TMAC_PICK(decode_kernel, desc, p.whole_rows ? 0 : p.blocks), grid, a, stream);
  if (st != TMAC_OK) return st;
  return launch(desc->elem == TMAC_ELEM_F16 ? (const void*)join_decode_kernel<F16> : (const void*)join_decode_kernel<BF16>, join_grid, a, stream);
}
