// Rotary positions, and filling and reading pages of keys and values in 8 bits (tmac_pages.h).
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstdint>
#include <type_traits>

#include "tmac_attn_host.h"
#include "tmac_internal.h"
#include "tmac_pages_core.h"
#include "tmac_pages_host.h"

namespace tmac {
namespace pages {

// --- rotation -----------------------------------------------------------------------------------------------------------------------

// Cosine and sine of an angle, times magnitude, rounded to 32 bits once.  The quarter turns are taken off (a position of 2^20 leaves 2^-35 of a turn), what
// is left, |x| <= pi / 4, has Taylor's polynomials up to x^13 and x^14, off by at most 2e-14.  All in 64 bits, whose products are as fast here: in 32 the last
// digit was off by one or two, and keys near the middle between two codes took the other one more often.
__device__ __forceinline__ f2 cos_sin(double angle, double magnitude) {
  const double quarters = angle * 0.63661977236758134308;  // 2 / pi
  const double whole = __builtin_rint(quarters);
  const double x = (quarters - whole) * 1.57079632679489661923, y = x * x;
  const double s = x * (1.0 + y * (-1.0 / 6 + y * (1.0 / 120 + y * (-1.0 / 5040 + y * (1.0 / 362880 + y * (-1.0 / 39916800 + y * (1.0 / 6227020800.0)))))));
  const double c = 1.0 + y * (-0.5 + y * (1.0 / 24 + y * (-1.0 / 720 + y * (1.0 / 40320 + y * (-1.0 / 3628800 + y * (1.0 / 479001600 + y * (-1.0 / 87178291200.0)))))));
  const int turn = (int)(whole - 4.0 * __builtin_floor(whole * 0.25));
  const float cc = (float)((turn & 1 ? s : c) * magnitude), ss = (float)((turn & 1 ? c : s) * magnitude);
  return f2{turn == 1 || turn == 2 ? -cc : cc, turn >= 2 ? -ss : ss};
}

struct RopeArgs {
  struct Item {
    const char* x;
    char* out;
    int64_t x_token, x_head, out_token, out_head;  // bytes
    int slice, H;                                  // its first slice, its heads
  } item[TMAC_ROPE_MAX];
  const double* freq;
  const int64_t* positions;  // null: from the batch
  Batch batch;
  double magnitude;
  int pairs, D, T, count;
  int slots, turning, slices, per_slice;   // vectors of a row, those that turn; wavefronts of a token, rows (heads of one item) of each
  uint32_t by_slots;                       // ceil(2^32 / slots), exact for what a slice has; 0: one slot
};

__device__ __forceinline__ int64_t position_of(const int64_t* positions, const Batch& b, int token) {
  if (positions) return positions[token];
  const Sequence seq(b, sequence_of(b, token));
  return (int64_t)seq.first + token - seq.row0;
}

template <int N>
struct Vec { typedef uint16_t type __attribute__((ext_vector_type(N))); };
template <>
struct Vec<1> { typedef uint16_t type; };
template <int N>
__device__ __forceinline__ uint16_t elem_of(const typename Vec<N>::type& x, int i) {
  if constexpr (N == 1) return x;
  else return x[i];
}

// The rows of one slice of one token, by one wavefront: its lanes take a pair each for the cosines and sines, then vectors of N
// elements, four at once.  Memory bounds it: 16384 tokens of 72 heads of 128 elements, 604 MB, 115 us = 5.2 TB/s, a copy's rate; 2003 tokens of 64 heads of
// 100, 51 MB, 13.8 us.  (A slice is of one tensor: with rows of several, every vector chose its tensor's strides, 23 us.)
template <bool BF16, bool INTERLEAVED, int N>
__device__ __forceinline__ void rotate_rows(const RopeArgs& a, int token, int slice, f2* turn) {
  typedef typename Vec<N>::type V;
  constexpr int PAIRS = INTERLEAVED ? N / 2 : N, AT_ONCE = 4;
  const int lane = threadIdx.x & 63;
  const int64_t position = position_of(a.positions, a.batch, token);
  const double freq = lane < a.pairs ? a.freq[lane] : 0.0;
  int k = 0;
#pragma unroll
  for (int j = 1; j < TMAC_ROPE_MAX; ++j) k += j < a.count && slice >= a.item[j].slice;
  const RopeArgs::Item& it = a.item[k];
  const int row0 = (slice - it.slice) * a.per_slice, n = (min(it.H, row0 + a.per_slice) - row0) * a.slots;
  const int64_t x_head = it.x_head, out_head = it.out_head;
  const char* const x0 = it.x + token * it.x_token + row0 * x_head;
  char* const out0 = it.out + token * it.out_token + row0 * out_head;
  for (int i0 = 0; i0 < n; i0 += 64 * AT_ONCE) {
    V first[AT_ONCE], second[AT_ONCE];
    char* to[AT_ONCE];
    int slot[AT_ONCE];
#pragma unroll
    for (int u = 0; u < AT_ONCE; ++u) {
      const int i = i0 + u * 64 + lane;
      slot[u] = -1;
      if (i >= n) continue;
      const int row = a.by_slots ? (int)__umulhi((uint32_t)i, a.by_slots) : i;
      slot[u] = i - row * a.slots;
      // a vector that turns, or one of those after the pairs
      const int d = slot[u] < a.turning ? slot[u] * N : 2 * a.pairs + (slot[u] - a.turning) * N;
      const char* x = x0 + row * x_head + d * 2;
      to[u] = out0 + row * out_head + d * 2;
      first[u] = *reinterpret_cast<const V*>(x);
      if (!INTERLEAVED && slot[u] < a.turning) second[u] = *reinterpret_cast<const V*>(x + a.pairs * 2);
    }
    if (i0 == 0) {
      // (the first rows are on their way)
      if (lane < a.pairs) turn[lane] = cos_sin((double)position * freq, a.magnitude);
      __builtin_amdgcn_wave_barrier();
    }
#pragma unroll
    for (int u = 0; u < AT_ONCE; ++u) {
      if (slot[u] < 0) continue;
      if (slot[u] >= a.turning) {
        *reinterpret_cast<V*>(to[u]) = first[u];
        continue;
      }
      uint16_t lo[N], hi[N];
#pragma unroll
      for (int p = 0; p < PAIRS; ++p) {
        const f2 cs = turn[slot[u] * PAIRS + p];
        const float x = to_float(elem_of<N>(first[u], INTERLEAVED ? 2 * p : p), BF16);
        const float y = to_float(INTERLEAVED ? elem_of<N>(first[u], 2 * p + (N > 1)) : elem_of<N>(second[u], p), BF16);
        const uint16_t x1 = from_float(x * cs[0] - y * cs[1], BF16), y1 = from_float(x * cs[1] + y * cs[0], BF16);
        if (INTERLEAVED) lo[2 * p] = x1, lo[2 * p + (N > 1)] = y1;
        else lo[p] = x1, hi[p] = y1;
      }
      V v;
      if constexpr (N == 1) v = lo[0];
      else
#pragma unroll
        for (int j = 0; j < N; ++j) v[j] = lo[j];
      *reinterpret_cast<V*>(to[u]) = v;
      if (!INTERLEAVED) {
        if constexpr (N == 1) v = hi[0];
        else
#pragma unroll
          for (int j = 0; j < N; ++j) v[j] = hi[j];
        *reinterpret_cast<V*>(to[u] + a.pairs * 2) = v;
      }
    }
  }
}

template <bool BF16, bool INTERLEAVED, int N>
__global__ __launch_bounds__(256) void rotate_kernel(const RopeArgs a) {
  __shared__ f2 turn[4][64];
  const int64_t w = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
  const int token = __builtin_amdgcn_readfirstlane((int)(w / a.slices)), slice = __builtin_amdgcn_readfirstlane((int)(w % a.slices));
  if (token < a.T) rotate_rows<BF16, INTERLEAVED, N>(a, token, slice, turn[threadIdx.x >> 6]);
}

// --- filling pages --------------------------------------------------------------------------------------------------------------------

struct StoreArgs {
  Pages pages;
  Batch batch;
  const char *k, *v;
  int64_t k_token, k_head, v_token, v_head;  // bytes
  const double* freq;                        // null: keys as they are
  const int64_t* positions;
  double magnitude;
  int pairs, turning, vectors;               // vectors of a row of keys, those that turn
  uint32_t by_vectors, by_pairs, by_values;  // ceil(2^32 / n); 0: n is 1
  int slots;                                 // blocks of a sequence that have workgroups; 0: starts[s] / 32 + 2 s on
  int heads, groups, workgroups;             // key heads of a workgroup, workgroups of a block, of all blocks; those behind turn queries
  RopeArgs q;
};

// The sequence and the block of the w-th place of a call, or false.
__device__ __forceinline__ bool block_of(const Batch& b, int slots, int w, int& s, int& j) {
  if (slots) {
    s = w / slots, j = w - s * slots;
  } else {
    // (sequence s has at most n / 32 + 2 of them, rounded down; both terms ascend)
    auto from = [&](int i) { return (int64_t)(clamp_to(b.cu[i], b.T) / BT) + 2 * (int64_t)i; };
    s = count_up_to(b.S, from, w);
    if (s >= b.S) return false;
    j = w - (int)from(s);
    if (j < 0) return false;  // (starts that fall, or do not begin at zero)
  }
  return true;
}
__device__ __forceinline__ int divided(int i, uint32_t by) { return by ? (int)__umulhi((uint32_t)i, by) : i; }

// A block of 32 tokens of a sequence that the call's tokens touch, for some key heads one after the other: rows come in vectors of N elements, the
// next head's while this one is worked on; keys turn on their way to LDS, by cosines and sines that are worked out once; with the scales
// known, a thread makes 16 codes of either plane.  A step's few tokens wait for memory one time after the other (lengths, table and rows, what the block
// holds: 24 sequences with their 64 query heads 6.6 us); prompts are bound by memory (16384 tokens, 8 key heads, 64 query heads, 637 MB: 129 us = 4.9 TB/s) or, with
// few bytes a workgroup, by the vector ALUs beside it (1790 tokens in seven prompts, 32 + 32 heads of 100: 24 us, 58 MB).
template <typename Code, bool BF16, bool INTERLEAVED, int N>
__global__ __launch_bounds__(256) void store_kernel(const StoreArgs a) {
  typedef typename Vec<N>::type V;
  constexpr int NV = N == 8 ? 8 : 4, KI = N == 8 ? 2 : 16 / N, VI = 32 / NV / 2, PAIRS = INTERLEAVED ? N / 2 : N;
  typedef typename Vec<NV>::type VV;
  __shared__ __attribute__((aligned(16))) f2 turn[BT * 64];
  __shared__ __attribute__((aligned(16))) float keys[BT][132];
  __shared__ __attribute__((aligned(16))) uint16_t values[BT][136];
  __shared__ float most[3][2][4];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  if ((int)blockIdx.x >= a.workgroups) {
    const int64_t w = (int64_t)(blockIdx.x - a.workgroups) * 4 + wave;
    const int token = __builtin_amdgcn_readfirstlane((int)(w / a.q.slices)), slice = __builtin_amdgcn_readfirstlane((int)(w % a.q.slices));
    if (token < (a.batch.cu ? a.batch.start(a.batch.S) : a.q.T)) rotate_rows<BF16, INTERLEAVED, N>(a.q, token, slice, turn + wave * 64);
    return;
  }
  const int h0 = blockIdx.x % a.groups * a.heads, h1 = min(a.pages.Hkv, h0 + a.heads);
  int s, j;
  if (!block_of(a.batch, a.slots, blockIdx.x / a.groups, s, j)) return;
  const Sequence seq(a.batch, s);
  if (j > (seq.n + BT - 2) / BT) return;  // (so that what follows stays below 2^31)
  const int block = max(seq.first, 0) / BT + j;
  // tokens [t0, t1) of the block are the call's
  const int t0 = max(0, seq.first - block * BT), t1 = min(BT, seq.len - block * BT), nt = t1 - t0;
  if (seq.n == 0 || nt <= 0) return;
  const int D = a.pages.D, chunks = a.pages.chunks, row0 = seq.row0 + block * BT - seq.first + t0;  // the row of token t0
  const int k_count = nt * a.vectors, v_count = nt * (D / NV);
  V k_lo[KI], k_hi[KI];
  VV v_in[VI];
  auto load = [&](int head) {
    const char* k = a.k + head * a.k_head + row0 * a.k_token;
    const char* v = a.v + head * a.v_head + row0 * a.v_token;
#pragma unroll
    for (int u = 0; u < KI; ++u) {
      const int i = tid + u * 256;
      if (i >= k_count) break;
      const int t = divided(i, a.by_vectors), slot = i - t * a.vectors;
      const int d = slot < a.turning ? slot * N : 2 * a.pairs + (slot - a.turning) * N;
      const char* at = k + t * a.k_token + d * 2;
      k_lo[u] = *reinterpret_cast<const V*>(at);
      if (!INTERLEAVED && slot < a.turning) k_hi[u] = *reinterpret_cast<const V*>(at + a.pairs * 2);
    }
#pragma unroll
    for (int u = 0; u < VI; ++u) {
      const int i = tid + u * 256;
      if (i >= v_count) break;
      const int t = divided(i, a.by_values);
      v_in[u] = *reinterpret_cast<const VV*>(v + t * a.v_token + (i - t * (D / NV)) * NV * 2);
    }
  };
  load(h0);
  const int64_t unit0 = a.pages.unit_of(a.batch.row(s), a.batch.width, block, h0);
  const int codes = chunks * BT;  // 16 of them a thread, in either plane
  // what a block that was begun before holds: its scales, the thread's values
  f2 was = {0.0f, 0.0f};
  u4 old = {0u, 0u, 0u, 0u};
  auto load_old = [&](int64_t unit) {
    if (t0 == 0 || unit0 < 0) return;
    was = *reinterpret_cast<const f2*>(a.pages.scales + unit * 2);
    if (tid < codes) old = *(reinterpret_cast<const u4*>(a.pages.values(unit)) + tid);
  };
  load_old(unit0);
  for (int i = tid; i < nt * a.pairs; i += 256) {
    const int t = divided(i, a.by_pairs), p = i - t * a.pairs;
    const int64_t position = a.positions ? a.positions[row0 + t] : (int64_t)block * BT + t0 + t;
    turn[i] = cos_sin((double)position * a.freq[p], a.magnitude);
  }
  if (unit0 < 0) return;
  __syncthreads();
  for (int head = h0; head < h1; ++head) {
    const int64_t unit = unit0 + ((int64_t)(head - h0) << a.pages.shift);
    float* scales = a.pages.scales + unit * 2;
    u4* const v_to = reinterpret_cast<u4*>(a.pages.values(unit)) + tid;
    // the largest, and zero where all are finite
    float mk = 0.0f, mv = 0.0f, odd_k = 0.0f, odd_v = 0.0f;
    auto take = [](float& most, float& odd, float x) { most = fmaxf(most, fabsf(x)), odd = __builtin_fmaf(x, 0.0f, odd); };
#pragma unroll
    for (int u = 0; u < KI; ++u) {
      const int i = tid + u * 256;
      if (i >= k_count) break;
      const int t = divided(i, a.by_vectors), slot = i - t * a.vectors;
      float lo[N], hi[N];
#pragma unroll
      for (int x = 0; x < N; ++x) lo[x] = to_float(elem_of<N>(k_lo[u], x), BF16);
      if (slot < a.turning) {
        if (!INTERLEAVED) {
#pragma unroll
          for (int x = 0; x < N; ++x) hi[x] = to_float(elem_of<N>(k_hi[u], x), BF16);
        }
#pragma unroll
        for (int p = 0; p < PAIRS; ++p) {
          const f2 cs = turn[t * a.pairs + slot * PAIRS + p];
          float& x = lo[INTERLEAVED ? 2 * p : p];
          float& y = INTERLEAVED ? lo[2 * p + (N > 1)] : hi[p];
          const float x1 = x * cs[0] - y * cs[1], y1 = x * cs[1] + y * cs[0];
          x = x1, y = y1;
          take(mk, odd_k, x1), take(mk, odd_k, y1);
        }
        if (!INTERLEAVED) {
#pragma unroll
          for (int x = 0; x < N; ++x) keys[t0 + t][slot * N + a.pairs + x] = hi[x];
        }
      } else {
#pragma unroll
        for (int x = 0; x < N; ++x) take(mk, odd_k, lo[x]);
      }
      const int d = slot < a.turning ? slot * N : 2 * a.pairs + (slot - a.turning) * N;
#pragma unroll
      for (int x = 0; x < N; ++x) keys[t0 + t][d + x] = lo[x];
    }
#pragma unroll
    for (int u = 0; u < VI; ++u) {
      const int i = tid + u * 256;
      if (i >= v_count) break;
      const int t = divided(i, a.by_values);
#pragma unroll
      for (int x = 0; x < NV; ++x) take(mv, odd_v, to_float(v_in[u][x], BF16));
      *reinterpret_cast<VV*>(&values[t0 + t][(i - t * (D / NV)) * NV]) = v_in[u];
    }
    if (head + 1 < h1) load(head + 1);
    float m[2];
    auto meet = [&](int place) {
#pragma unroll
      for (int o = 32; o > 0; o >>= 1) mk = fmaxf(mk, __shfl_xor(mk, o)), mv = fmaxf(mv, __shfl_xor(mv, o));
      if (lane == 0) most[place][0][wave] = mk, most[place][1][wave] = mv;
      __syncthreads();
#pragma unroll
      for (int x = 0; x < 2; ++x) m[x] = fmaxf(fmaxf(most[place][x][0], most[place][x][1]), fmaxf(most[place][x][2], most[place][x][3]));
    };
    mk = odd_k == 0.0f ? mk : INFINITY, mv = odd_v == 0.0f ? mv : INFINITY;
    meet((head - h0) & 1);
    const bool odd = m[0] == INFINITY || m[1] == INFINITY;
    if (__builtin_expect(odd, 0)) {  // some are infinite or no numbers: the largest of the others
      mk = mv = 0.0f;
      for (int i = tid; i < nt * D; i += 256) {
        const float x = fabsf(keys[t0 + i / D][i % D]), y = fabsf(to_float(values[t0 + i / D][i % D], BF16));
        mk = x <= 3.402823466e38f ? fmaxf(mk, x) : mk, mv = y <= 3.402823466e38f ? fmaxf(mv, y) : mv;
      }
      meet(2);
    }
    const float scale[2] = {fmaxf(was[0], Code::scale_for(m[0])), fmaxf(was[1], Code::scale_for(m[1]))};
    if (tid == 0) scales[0] = scale[0], scales[1] = scale[1];
    // New codes, old ones rounded again where the scale has grown, zeros in a block that is begun.  careful: of any numbers
    auto make = [&](auto careful) {
      auto encode = [](float a, float b, float c, float d) {
        if constexpr (decltype(careful)::value) return Code::encode(a == a ? a : 0.0f, b == b ? b : 0.0f, c == c ? c : 0.0f, d == d ? d : 0.0f);
        else return Code::encode_within(a, b, c, d);
      };
      // keys: token t, elements 16 c ..
      const int t = tid % BT, c = tid / BT;
      u4* const k_to = reinterpret_cast<u4*>(a.pages.keys(unit)) + tid;
      if (t >= t0 && t < t1) {
        const float inv = 1.0f / scale[0];
        u4 got;
#pragma unroll
        for (int w = 0; w < 4; ++w) {
          const int d = c * 16 + 4 * w;
          const f4 x = (d < D ? *reinterpret_cast<const f4*>(&keys[t][d]) : f4{0.0f, 0.0f, 0.0f, 0.0f}) * inv;
          got[w] = encode(x[0], x[1], x[2], x[3]);
        }
        *k_to = got;
      } else if (t0 == 0) {
        *k_to = u4{0u, 0u, 0u, 0u};
      } else if (was[0] != scale[0]) {
        u4 x = *k_to;
        const float ratio = was[0] / scale[0];
#pragma unroll
        for (int w = 0; w < 4; ++w) {
          float y[4];
          Code::decode(x[w], y);
          x[w] = Code::encode(y[0] * ratio, y[1] * ratio, y[2] * ratio, y[3] * ratio);
        }
        *k_to = x;
      }
      // values: element d, 16 tokens
      const int run = tid / 64, n = value_run(chunks, run * 32), half = (tid - run * 64) / n, d = run * 32 + (tid - run * 64) % n;
      const float inv = 1.0f / scale[1], ratio = was[1] / scale[1];
      u4 got;
#pragma unroll
      for (int w = 0; w < 4; ++w) {
        float y[4];
#pragma unroll
        for (int b = 0; b < 4; ++b) y[b] = to_float(values[value_token(half, 4 * w + b)][d], BF16) * inv;
        if (nt < BT) {
          float before[4] = {0.0f, 0.0f, 0.0f, 0.0f};
          if (t0) Code::decode(old[w], before);
#pragma unroll
          for (int b = 0; b < 4; ++b) {
            const int t = value_token(half, 4 * w + b);
            y[b] = t >= t0 && t < t1 ? y[b] : t0 ? before[b] * ratio : 0.0f;
          }
        }
        got[w] = d < D ? encode(y[0], y[1], y[2], y[3]) : 0u;
      }
      *v_to = got;
    };
    if (tid < codes) {
      if (__builtin_expect(odd, 0)) make(std::true_type{});
      else make(std::false_type{});
    }
    if (head + 1 < h1) {
      load_old(unit + ((int64_t)1 << a.pages.shift));
      __syncthreads();  // (the rows have been read)
    }
  }
}

// --- reading pages -----------------------------------------------------------------------------------------------------------------------

struct ReadArgs {
  Pages pages;
  Batch batch;
  char *k, *v;
  int64_t k_token, k_head, v_token, v_head;  // bytes
  int bf16, slots;
};

// A block of a sequence and key head, through LDS, since values lie by elements.  (16384 tokens of 8 heads: 28 us, 100 MB at 3.6 TB/s; who reads pages back
// copies or looks at them, so it was left there.)
template <typename Code>
__global__ __launch_bounds__(256) void read_kernel(const ReadArgs a) {
  __shared__ uint32_t rows[2][BT][33];
  const int tid = threadIdx.x, head = blockIdx.x % a.pages.Hkv;
  int s, j;
  if (!block_of(a.batch, a.slots, blockIdx.x / a.pages.Hkv, s, j)) return;
  const Sequence seq(a.batch, s);
  if (seq.n == 0 || j > (seq.n + BT - 2) / BT) return;
  // (rows before the first token: blocks count from the first row's, which may be below zero)
  const int block = (seq.first >= 0 ? seq.first / BT : -((-(int64_t)seq.first + BT - 1) / BT)) + j;
  const int t0 = max(0, seq.first - block * BT), t1 = min(BT, seq.len - block * BT);
  if (t1 <= t0) return;
  const int64_t unit = block < 0 ? -1 : a.pages.unit_of(a.batch.row(s), a.batch.width, block, head);
  const int chunks = a.pages.chunks, D = a.pages.D, row0 = seq.row0 + block * BT - seq.first;
  float scale[2] = {0.0f, 0.0f};
  if (unit >= 0) {
    scale[0] = a.pages.scales[unit * 2], scale[1] = a.pages.scales[unit * 2 + 1];
    for (int i = tid; i < chunks * BT; i += 256) {
      const u4 x = *reinterpret_cast<const u4*>(a.pages.keys(unit) + i * 16);
#pragma unroll
      for (int w = 0; w < 4; ++w) rows[0][i % BT][i / BT * 4 + w] = x[w];
      const u4 y = *reinterpret_cast<const u4*>(a.pages.values(unit) + i * 16);
      const int run = i / 64, n = value_run(chunks, run * 32), half = (i - run * 64) / n, d = run * 32 + (i - run * 64) % n;
#pragma unroll
      for (int b = 0; b < 16; ++b) reinterpret_cast<uint8_t*>(rows[1][value_token(half, b)])[d] = (uint8_t)(y[b >> 2] >> (8 * (b & 3)));
    }
  }
  __syncthreads();
  const int fours = D / 4;
  for (int i = tid; i < 2 * (t1 - t0) * fours; i += 256) {
    const int x = i >= (t1 - t0) * fours, r = i - (x ? (t1 - t0) * fours : 0), t = t0 + r / fours, w = r % fours;
    float y[4] = {0.0f, 0.0f, 0.0f, 0.0f};
    if (unit >= 0) Code::decode(rows[x][t][w], y);
    uint16_t got[4];
#pragma unroll
    for (int b = 0; b < 4; ++b) got[b] = from_float(y[b] * scale[x], a.bf16);
    char* to = x ? a.v + head * a.v_head + (row0 + t) * a.v_token : a.k + head * a.k_head + (row0 + t) * a.k_token;
    *reinterpret_cast<u2*>(to + w * 8) = u2{got[0] | (uint32_t)got[1] << 16, got[2] | (uint32_t)got[3] << 16};
  }
}

// --- host --------------------------------------------------------------------------------------------------------------------------------

static bool rope_ok(const tmac_rope* r) {
  return r && r->freq_dev && (reinterpret_cast<uintptr_t>(r->freq_dev) & 7) == 0 && r->D > 0 && r->D % 4 == 0 && r->rot >= 2 && r->rot % 2 == 0 &&
         r->rot <= r->D && (r->interleaved == 0 || r->interleaved == 1) && (r->elem == TMAC_ELEM_F16 || r->elem == TMAC_ELEM_BF16) &&
         std::isfinite(r->magnitude) && !r->reserved[0] && !r->reserved[1];
}

static uint32_t by(int n) { return n == 1 ? 0 : (uint32_t)((((uint64_t)1 << 32) + n - 1) / n); }

// Elements of a vector: side by side, whole pairs that end at rot; in halves, as many as end at rot / 2; eight where rows are aligned for it.
static int vector_of(const tmac_rope* r, bool wide) {
  const int half = r->rot / 2;
  const int n = r->interleaved ? (r->rot % 8 == 0 ? 8 : r->rot % 4 == 0 ? 4 : 2) : (half % 8 == 0 ? 8 : half % 4 == 0 ? 4 : half % 2 == 0 ? 2 : 1);
  return n == 8 && !wide ? 4 : n;
}
static int turning_of(const tmac_rope* r, int n) { return r->interleaved ? r->rot / n : r->rot / 2 / n; }
static bool wide_rows(const tmac_view& v, int D) { return D % 8 == 0 && (reinterpret_cast<uintptr_t>(v.data) & 15) == 0 && v.token % 8 == 0 && v.head % 8 == 0; }

// How the rows are dealt out.  n: elements of a vector.  Wavefronts of a token: until the chip has some thousands, or a wavefront one vector a lane left;
// of one item and at most 256 rows each.
static void plan_rope(RopeArgs& a, const tmac_rope* r, const tmac_rope_item* items, int count, int T, int n) {
  bool in_place = true;
  a.freq = r->freq_dev, a.magnitude = r->magnitude, a.pairs = r->rot / 2, a.D = r->D, a.T = T, a.count = count;
  int64_t rows = 0;
  for (int i = 0; i < count; ++i) {
    in_place = in_place && items[i].x.data == items[i].out.data;
    rows += items[i].H;
  }
  a.turning = turning_of(r, n);
  a.slots = a.turning + (in_place ? 0 : (r->D - r->rot) / n);
  a.by_slots = by(a.slots);
  const int64_t slices = std::max<int64_t>(1, std::min((rows * a.slots + 63) / 64, ((int64_t)8192 + T - 1) / T));
  a.per_slice = (int)std::min<int64_t>(256, (rows + slices - 1) / slices);
  a.slices = 0;
  for (int i = 0; i < count; ++i) {
    const tmac_rope_item& it = items[i];
    a.item[i] = {static_cast<const char*>(it.x.data), static_cast<char*>(it.out.data), it.x.token * 2, it.x.head * 2, it.out.token * 2, it.out.head * 2, a.slices, it.H};
    a.slices += (it.H + a.per_slice - 1) / a.per_slice;
  }
}

template <bool BF16, bool INTERLEAVED>
static const void* rotate_of(int n) {
  if (n == 8) return (const void*)rotate_kernel<BF16, INTERLEAVED, 8>;
  if (n == 4) return (const void*)rotate_kernel<BF16, INTERLEAVED, 4>;
  if (n == 2 || INTERLEAVED) return (const void*)rotate_kernel<BF16, INTERLEAVED, 2>;
  return (const void*)rotate_kernel<BF16, false, 1>;
}
template <typename Code, bool BF16, bool INTERLEAVED>
static const void* store_of(int n) {
  if (n == 8) return (const void*)store_kernel<Code, BF16, INTERLEAVED, 8>;
  if (n == 4) return (const void*)store_kernel<Code, BF16, INTERLEAVED, 4>;
  if (n == 2 || INTERLEAVED) return (const void*)store_kernel<Code, BF16, INTERLEAVED, 2>;
  return (const void*)store_kernel<Code, BF16, false, 1>;
}
template <typename Code>
static const void* store_of(bool bf16, bool interleaved, int n) {
  return bf16 ? (interleaved ? store_of<Code, true, true>(n) : store_of<Code, true, false>(n))
              : (interleaved ? store_of<Code, false, true>(n) : store_of<Code, false, false>(n));
}

}  // namespace pages
}  // namespace tmac

using namespace tmac;
using namespace tmac::pages;

extern "C" tmac_status tmac_rotate(const tmac_rope* rope, const tmac_rope_item* items, int32_t count, const int64_t* positions_dev, int32_t T,
                                   void* stream) {
  if (!rope_ok(rope) || !items || count < 1 || count > TMAC_ROPE_MAX || T < 0) return TMAC_EINVAL;
  if (T == 0) return TMAC_OK;
  if (!positions_dev || (reinterpret_cast<uintptr_t>(positions_dev) & 7)) return TMAC_EINVAL;
  int64_t rows = 0;
  for (int i = 0; i < count; ++i) {
    const tmac_rope_item& it = items[i];
    if (!item_ok(it)) return TMAC_EINVAL;
    rows += it.H;
  }
  if (rope->D > 128 || rows > (1 << 24) || attn::long_axis(T)) return TMAC_EUNSUPPORTED;
  bool wide = true;
  for (int i = 0; i < count; ++i) wide = wide && pages::wide_rows(items[i].x, rope->D) && pages::wide_rows(items[i].out, rope->D);
  const int n = vector_of(rope, wide);
  RopeArgs a = {};
  a.positions = positions_dev;
  plan_rope(a, rope, items, count, T, n);
  const void* kernel = rope->elem == TMAC_ELEM_BF16 ? (rope->interleaved ? rotate_of<true, true>(n) : rotate_of<true, false>(n))
                                                    : (rope->interleaved ? rotate_of<false, true>(n) : rotate_of<false, false>(n));
  return launch(kernel, ((int64_t)T * a.slices + 3) / 4, 256, &a, stream);
}

static bool sized(const tmac_pages* p) { return pages_ok(p) && p->D <= 128 && units_of(p) <= MOST_UNITS; }
extern "C" size_t tmac_pages_code_bytes(const tmac_pages* p) { return sized(p) ? (size_t)units_of(p) * chunks_of(p) * 1024 : 0; }
extern "C" size_t tmac_pages_scale_bytes(const tmac_pages* p) { return sized(p) ? (size_t)units_of(p) * 8 : 0; }

extern "C" tmac_status tmac_pages_append(const tmac_pages* p, const tmac_pages_batch* batch, int32_t elem, const tmac_view* k, const tmac_view* v,
                                         const tmac_rope* rope, const int64_t* positions_dev, const tmac_view* q, const tmac_view* q_out, int32_t Hq,
                                         void* stream) {
  if (!pages_ok(p) || !batch_ok(batch) || (elem != TMAC_ELEM_F16 && elem != TMAC_ELEM_BF16)) return TMAC_EINVAL;
  if (rope && (!rope_ok(rope) || rope->D != p->D || rope->elem != elem)) return TMAC_EINVAL;
  if (!!q != !!q_out || (q && !rope) || (positions_dev && (!rope || (reinterpret_cast<uintptr_t>(positions_dev) & 7)))) return TMAC_EINVAL;
  if (batch->S == 0 || batch->T == 0) return TMAC_OK;
  if (!pages_set(p) || !batch_set(batch) || !attn::rows_ok(k, false, true, true) || !attn::rows_ok(v, false, true, true)) return TMAC_EINVAL;
  tmac_rope_item item = {};
  if (q) {
    item = {*q, *q_out, Hq, 0};
    if (!item_ok(item)) return TMAC_EINVAL;
  }
  if (!supported(p, batch) || (q && Hq > (1 << 24))) return TMAC_EUNSUPPORTED;
  StoreArgs a = {};
  a.pages = view_of(p), a.batch = view_of(batch);
  a.k = static_cast<const char*>(k->data), a.v = static_cast<const char*>(v->data);
  a.k_token = k->token * 2, a.k_head = k->head * 2, a.v_token = v->token * 2, a.v_head = v->head * 2;
  const int D = p->D;
  const bool wide = pages::wide_rows(*k, D) && pages::wide_rows(*v, D) && (!q || (pages::wide_rows(*q, D) && pages::wide_rows(*q_out, D)));
  int n = wide ? 8 : 4;
  if (rope) {
    n = vector_of(rope, wide);
    a.freq = rope->freq_dev, a.pairs = rope->rot / 2, a.turning = turning_of(rope, n), a.magnitude = rope->magnitude;
  }
  a.positions = positions_dev;
  a.vectors = a.turning + (D - 2 * a.pairs) / n;
  a.by_vectors = by(a.vectors), a.by_pairs = by(std::max(1, a.pairs)), a.by_values = by(D / (n == 8 ? 8 : 4));
  const int64_t blocks = block_slots(batch, a.slots);
  // Key heads of a workgroup, which share cosines and sines: as many as leave the chip two workgroups a CU (seven prompts of 32 heads: 26.7 us, 30 with four
  // a CU, 36 with one head each)
  a.heads = (int)std::max<int64_t>(1, std::min<int64_t>(p->Hkv, blocks * p->Hkv / 512));
  a.groups = (p->Hkv + a.heads - 1) / a.heads;
  int64_t workgroups = blocks * a.groups;
  if (!attn::launchable(workgroups, 256)) return TMAC_EUNSUPPORTED;
  a.workgroups = (int)workgroups;
  if (q) {
    a.q.positions = positions_dev, a.q.batch = a.batch;
    plan_rope(a.q, rope, &item, 1, batch->T, n);
    workgroups += ((int64_t)batch->T * a.q.slices + 3) / 4;
  }
  const bool bf16 = elem == TMAC_ELEM_BF16, interleaved = rope && rope->interleaved;
  return launch(p->code == TMAC_CODE_I8 ? store_of<I8>(bf16, interleaved, n) : store_of<E4M3>(bf16, interleaved, n), workgroups, 256, &a, stream);
}

extern "C" tmac_status tmac_pages_read(const tmac_pages* p, const tmac_pages_batch* batch, int32_t elem, const tmac_view* k, const tmac_view* v,
                                       void* stream) {
  if (!pages_ok(p) || !batch_ok(batch) || (elem != TMAC_ELEM_F16 && elem != TMAC_ELEM_BF16)) return TMAC_EINVAL;
  if (batch->S == 0 || batch->T == 0) return TMAC_OK;
  if (!pages_set(p) || !batch_set(batch) || !attn::rows_ok(k, false, true, true) || !attn::rows_ok(v, false, true, true)) return TMAC_EINVAL;
  if (!supported(p, batch)) return TMAC_EUNSUPPORTED;
  ReadArgs a = {};
  a.pages = view_of(p), a.batch = view_of(batch);
  a.k = static_cast<char*>(k->data), a.v = static_cast<char*>(v->data);
  a.k_token = k->token * 2, a.k_head = k->head * 2, a.v_token = v->token * 2, a.v_head = v->head * 2;
  a.bf16 = elem == TMAC_ELEM_BF16;
  const int64_t blocks = block_slots(batch, a.slots);
  return launch(p->code == TMAC_CODE_I8 ? (const void*)read_kernel<I8> : (const void*)read_kernel<E4M3>, blocks * p->Hkv, 256, &a, stream);
}
