// Rotary positions, and filling and reading pages of keys and values in 8 bits (tmac_pages.h).
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstdint>

#include "tmac_attn_host.h"
#include "tmac_internal.h"
#include "tmac_pages_core.h"
#include "tmac_pages_host.h"

namespace tmac {
namespace pages {

// --- rotation -----------------------------------------------------------------------------------------------------------------------

// Cosine and sine of an angle.  The quarter turns are taken off in 64 bits (a position of 2^20 leaves 2^-35 of a turn), what is left,
// |x| <= pi / 4, has Taylor's polynomials up to x^9 and x^10: off by at most 2e-9, below the last digit of 32 bits.
__device__ __forceinline__ f2 cos_sin(double angle) {
  const double quarters = angle * 0.63661977236758134308;  // 2 / pi
  const double whole = __builtin_rint(quarters);
  const float x = (float)(quarters - whole) * 1.57079632679489661923f, y = x * x;
  const float s = x * (1.0f + y * (-1.0f / 6 + y * (1.0f / 120 + y * (-1.0f / 5040 + y * (1.0f / 362880)))));
  const float c = 1.0f + y * (-0.5f + y * (1.0f / 24 + y * (-1.0f / 720 + y * (1.0f / 40320 + y * (-1.0f / 3628800)))));
  const int turn = (int)(whole - 4.0 * __builtin_floor(whole * 0.25));
  const float cc = turn & 1 ? s : c, ss = turn & 1 ? c : s;
  return f2{turn == 1 || turn == 2 ? -cc : cc, turn >= 2 ? -ss : ss};
}

struct RopeArgs {
  struct Item {
    const char* x;
    char* out;
    int64_t x_token, x_head, out_token, out_head;  // bytes
    int row;                                       // the first of its heads among all items' heads
  } item[TMAC_ROPE_MAX];
  const double* freq;
  const int64_t* positions;  // null: from the batch
  Batch batch;
  float magnitude;
  int pairs, D, T, count, rows;            // rows: heads of all items
  int slots, turning, slices, per_slice;   // vectors of a row, those that turn; wavefronts of a token, rows of one
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
// elements.  Memory bounds it (16384 tokens of 72 heads of 128 elements, 604 MB: see the launch).
template <bool BF16, bool INTERLEAVED, int N>
__device__ __forceinline__ void rotate_rows(const RopeArgs& a, int token, int slice, f2* turn) {
  typedef typename Vec<N>::type V;
  constexpr int PAIRS = INTERLEAVED ? N / 2 : N, AT_ONCE = 4;
  const int lane = threadIdx.x & 63;
  const int64_t position = position_of(a.positions, a.batch, token);
  if (lane < a.pairs) turn[lane] = cos_sin((double)position * a.freq[lane]) * a.magnitude;
  __builtin_amdgcn_wave_barrier();
  const int row0 = slice * a.per_slice, n = (min(a.rows, row0 + a.per_slice) - row0) * a.slots;
  for (int i0 = 0; i0 < n; i0 += 64 * AT_ONCE) {
    V first[AT_ONCE], second[AT_ONCE];
    char* to[AT_ONCE];
    int slot[AT_ONCE];
#pragma unroll
    for (int u = 0; u < AT_ONCE; ++u) {
      const int i = i0 + u * 64 + lane;
      slot[u] = -1;
      if (i >= n) continue;
      const int r = a.by_slots ? (int)__umulhi((uint32_t)i, a.by_slots) : i, row = row0 + r;
      slot[u] = i - r * a.slots;
      int k = 0;
#pragma unroll
      for (int j = 1; j < TMAC_ROPE_MAX; ++j) k += j < a.count && row >= a.item[j].row;
      const RopeArgs::Item& it = a.item[k];
      // a vector that turns, or one of those after the pairs
      const int d = slot[u] < a.turning ? slot[u] * N : 2 * a.pairs + (slot[u] - a.turning) * N;
      const char* x = it.x + token * it.x_token + (row - it.row) * it.x_head + d * 2;
      to[u] = it.out + token * it.out_token + (row - it.row) * it.out_head + d * 2;
      first[u] = *reinterpret_cast<const V*>(x);
      if (!INTERLEAVED && slot[u] < a.turning) second[u] = *reinterpret_cast<const V*>(x + a.pairs * 2);
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
  float magnitude;
  int pairs, interleaved, bf16;
  int slots;  // blocks of a sequence that have workgroups; 0: starts[s] / 32 + 2 s on
};

// The sequence and the block of the j-th workgroup of a call, or false.
__device__ __forceinline__ bool block_of(const Batch& b, int slots, int w, int& s, int& j) {
  if (slots) {
    s = w / slots, j = w - s * slots;
  } else {
    // (sequence s has at most n / 32 + 2 of them, rounded down; both terms ascend)
    auto from = [&](int i) { return (int64_t)(clamp_to(b.cu[i], b.T) / BT) + 2 * (int64_t)i; };
    s = count_up_to(b.S, from, w);
    if (s >= b.S) return false;
    j = w - (int)from(s);
  }
  return true;
}

// A block of 32 tokens of a sequence and key head that the call's tokens touch.
template <typename Code>
__global__ __launch_bounds__(256) void store_kernel(const StoreArgs a) {
  __shared__ float rows[2][BT][132];
  __shared__ float most[2][4];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int head = blockIdx.x % a.pages.Hkv;
  int s, j;
  if (!block_of(a.batch, a.slots, blockIdx.x / a.pages.Hkv, s, j)) return;
  const Sequence seq(a.batch, s);
  const int block = max(seq.first, 0) / BT + j;
  // tokens [t0, t1) of the block are the call's
  const int t0 = max(0, seq.first - block * BT), t1 = min(BT, seq.len - block * BT);
  if (seq.n == 0 || t1 <= t0) return;
  const int64_t unit = a.pages.unit_of(a.batch.row(s), a.batch.width, block, head);
  if (unit < 0) return;
  const int D = a.pages.D, pairs = a.freq ? a.pairs : 0, plain = D - 2 * pairs;
  const int row0 = seq.row0 + block * BT - seq.first;  // the row of the block's first token, if it were the call's
  float mk = 0.0f, mv = 0.0f;
  auto take = [](float& most, float x) {
    if (fabsf(x) <= 3.402823466e38f) most = fmaxf(most, fabsf(x));
  };
  const char* k = a.k + head * a.k_head;
  const char* v = a.v + head * a.v_head;
  for (int i = tid; i < (t1 - t0) * pairs; i += 256) {
    const int t = t0 + i / pairs, p = i % pairs;
    const int64_t position = a.positions ? a.positions[row0 + t] : (int64_t)block * BT + t;
    const f2 cs = cos_sin((double)position * a.freq[p]) * a.magnitude;
    const int d0 = a.interleaved ? 2 * p : p, d1 = a.interleaved ? 2 * p + 1 : p + pairs;
    const uint16_t* row = reinterpret_cast<const uint16_t*>(k + (row0 + t) * a.k_token);
    const float x = to_float(row[d0], a.bf16), y = to_float(row[d1], a.bf16);
    const float x1 = x * cs[0] - y * cs[1], y1 = x * cs[1] + y * cs[0];
    rows[0][t][d0] = x1, rows[0][t][d1] = y1;
    take(mk, x1), take(mk, y1);
  }
  for (int i = tid; i < (t1 - t0) * plain; i += 256) {
    const int t = t0 + i / plain, d = 2 * pairs + i % plain;
    const float x = to_float(reinterpret_cast<const uint16_t*>(k + (row0 + t) * a.k_token)[d], a.bf16);
    rows[0][t][d] = x;
    take(mk, x);
  }
  for (int i = tid; i < (t1 - t0) * D; i += 256) {
    const int t = t0 + i / D, d = i % D;
    const float x = to_float(reinterpret_cast<const uint16_t*>(v + (row0 + t) * a.v_token)[d], a.bf16);
    rows[1][t][d] = x;
    take(mv, x);
  }
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) mk = fmaxf(mk, __shfl_xor(mk, o)), mv = fmaxf(mv, __shfl_xor(mv, o));
  if (lane == 0) most[0][wave] = mk, most[1][wave] = mv;
  float* scales = a.pages.scales + unit * 2;
  const float was[2] = {t0 ? scales[0] : 0.0f, t0 ? scales[1] : 0.0f};
  __syncthreads();
  float scale[2];
#pragma unroll
  for (int x = 0; x < 2; ++x) {
    float m = fmaxf(fmaxf(most[x][0], most[x][1]), fmaxf(most[x][2], most[x][3]));
    scale[x] = fmaxf(was[x], Code::scale_for(m));
  }
  if (tid == 0) scales[0] = scale[0], scales[1] = scale[1];
  // Sixteen codes of either plane at a time: new ones, old ones (rounded again where the scale has grown), zeros
  auto codes_of = [&](const float (*src)[132], float was, float scale, u4* at, auto&& token_of, auto&& d_of, bool some) {
    const float inv = 1.0f / scale, ratio = was / scale;
    u4 old = {0u, 0u, 0u, 0u};
    if (t0) old = *at;
    else if (!some) { *at = old; return; }
    u4 got;
#pragma unroll
    for (int w = 0; w < 4; ++w) {
      float y[4];
      Code::decode(old[w], y);
#pragma unroll
      for (int b = 0; b < 4; ++b) {
        const int t = token_of(4 * w + b), d = d_of(4 * w + b);
        y[b] *= ratio;
        if (t >= t0 && t < t1 && d < D) {
          const float x = src[t][d];
          y[b] = x == x ? x * inv : 0.0f;
        }
      }
      got[w] = Code::encode(y[0], y[1], y[2], y[3]);
    }
    *at = got;
  };
  for (int i = tid; i < a.pages.chunks * BT; i += 256) {
    const int t = i % BT, c = i / BT;
    const bool is_new = t >= t0 && t < t1;
    if (t0 && !is_new && was[0] == scale[0]) continue;
    codes_of(rows[0], was[0], scale[0], reinterpret_cast<u4*>(a.pages.keys(unit) + i * 16), [&](int) { return t; },
             [&](int b) { return c * 16 + b; }, is_new);
  }
  for (int i = tid; i < a.pages.chunks * BT; i += 256) {
    const int run = i / 64, n = value_run(a.pages.chunks, run * 32), half = (i - run * 64) / n, d = run * 32 + (i - run * 64) % n;
    codes_of(rows[1], was[1], scale[1], reinterpret_cast<u4*>(a.pages.values(unit) + i * 16), [&](int b) { return value_token(half, b); },
             [&](int) { return d; }, true);
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

// A block of a sequence and key head.
template <typename Code>
__global__ __launch_bounds__(256) void read_kernel(const ReadArgs a) {
  __shared__ uint32_t rows[2][BT][33];
  const int tid = threadIdx.x, head = blockIdx.x % a.pages.Hkv;
  int s, j;
  if (!block_of(a.batch, a.slots, blockIdx.x / a.pages.Hkv, s, j)) return;
  const Sequence seq(a.batch, s);
  if (seq.n == 0) return;
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
         std::isfinite(r->magnitude) && !r->reserved[0] && !r->reserved[1] && !r->reserved[2];
}

// The widest vectors that the rows' alignment allows, and how the rows are dealt out.
static int rope_plan(RopeArgs& a, const tmac_rope* r, const tmac_rope_item* items, int count, int T) {
  const int half = r->rot / 2;
  bool wide = r->D % 8 == 0, in_place = true;
  a.freq = r->freq_dev, a.magnitude = r->magnitude, a.pairs = half, a.D = r->D, a.T = T, a.count = count, a.rows = 0;
  for (int i = 0; i < count; ++i) {
    const tmac_rope_item& it = items[i];
    for (const tmac_view* v : {&it.x, &it.out}) wide = wide && (reinterpret_cast<uintptr_t>(v->data) & 15) == 0 && v->token % 8 == 0 && v->head % 8 == 0;
    in_place = in_place && it.x.data == it.out.data;
    a.item[i] = {static_cast<const char*>(it.x.data), static_cast<char*>(it.out.data), it.x.token * 2, it.x.head * 2, it.out.token * 2, it.out.head * 2, a.rows};
    a.rows += it.H;
  }
  // side by side: vectors of whole pairs that end at rot; in halves: that end at rot / 2
  int n = r->interleaved ? (r->rot % 8 == 0 ? 8 : r->rot % 4 == 0 ? 4 : 2) : (half % 8 == 0 ? 8 : half % 4 == 0 ? 4 : half % 2 == 0 ? 2 : 1);
  if (n == 8 && !wide) n = 4;
  a.turning = r->interleaved ? r->rot / n : half / n;
  a.slots = a.turning + (in_place ? 0 : (r->D - r->rot) / n);
  a.by_slots = a.slots == 1 ? 0 : (uint32_t)((((uint64_t)1 << 32) + a.slots - 1) / a.slots);
  return n;
}

template <bool BF16, bool INTERLEAVED>
static const void* rotate_of(int n) {
  if (n == 8) return (const void*)rotate_kernel<BF16, INTERLEAVED, 8>;
  if (n == 4) return (const void*)rotate_kernel<BF16, INTERLEAVED, 4>;
  if (n == 2 || INTERLEAVED) return (const void*)rotate_kernel<BF16, INTERLEAVED, 2>;
  return (const void*)rotate_kernel<BF16, false, 1>;
}

static tmac_status rotate(RopeArgs& a, const tmac_rope* r, const tmac_rope_item* items, int count, int T, void* stream) {
  const int n = rope_plan(a, r, items, count, T);
  // Wavefronts of a token: until the chip has some thousands, or a wavefront one vector a lane left; at most 256 rows each
  const int64_t vectors = (int64_t)a.rows * a.slots;
  const int64_t most = (vectors + 63) / 64, least = (a.rows + 255) / 256;
  a.slices = (int)std::max<int64_t>(least, std::min<int64_t>(most, (4096 + T - 1) / T));
  a.per_slice = (a.rows + a.slices - 1) / a.slices;
  a.slices = (a.rows + a.per_slice - 1) / a.per_slice;
  const void* kernel = r->elem == TMAC_ELEM_BF16 ? (r->interleaved ? rotate_of<true, true>(n) : rotate_of<true, false>(n))
                                                 : (r->interleaved ? rotate_of<false, true>(n) : rotate_of<false, false>(n));
  return launch(kernel, ((int64_t)T * a.slices + 3) / 4, 256, &a, stream);
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
  RopeArgs a = {};
  a.positions = positions_dev;
  return rotate(a, rope, items, count, T, stream);
}

extern "C" size_t tmac_pages_code_bytes(const tmac_pages* p) { return pages_ok(p) && p->D <= 128 ? (size_t)units_of(p) * chunks_of(p) * 1024 : 0; }
extern "C" size_t tmac_pages_scale_bytes(const tmac_pages* p) { return pages_ok(p) && p->D <= 128 ? (size_t)units_of(p) * 8 : 0; }

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
  if (rope) a.freq = rope->freq_dev, a.pairs = rope->rot / 2, a.interleaved = rope->interleaved, a.magnitude = rope->magnitude;
  a.positions = positions_dev;
  a.bf16 = elem == TMAC_ELEM_BF16;
  const int64_t blocks = block_slots(batch, a.slots);
  if (!attn::launchable(blocks * p->Hkv, 256)) return TMAC_EUNSUPPORTED;
  if (q) {
    RopeArgs r = {};
    r.positions = positions_dev, r.batch = a.batch;
    const tmac_status st = rotate(r, rope, &item, 1, batch->T, stream);
    if (st != TMAC_OK) return st;
  }
  return launch(p->code == TMAC_CODE_I8 ? (const void*)store_kernel<I8> : (const void*)store_kernel<E4M3>, blocks * p->Hkv, 256, &a, stream);
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
