// Attention over pages of keys and values in 8 bits (tmac_pages.h).
//
// Rows of a unit of work are (query token, head of the group) of one sequence and key head.  Products run on v_mfma_f32_32x32x16 in
// transposed form, S^T = K Q^T and O^T = V^T P^T, so that a lane owns a row (lane & 31): maximum and sum need one exchange between a
// wavefront's halves, and the exponentials are the second product's operand as they stand.  Codes are whole numbers or e4m3 values,
// which fp16 holds exactly; a block's scales are the same for all its products, so they are taken out of them:
//   x_j = s_j a + log2 sv,  a = sk scale log2 e,  p_j = 2^(x_j - m),  O += sum p_j code_j,  l += (sum p_j) / sv
// with m against the rows' largest x, and o = O / l.
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

typedef float f16x __attribute__((ext_vector_type(16)));

constexpr int ROWS = 32;
// The sums are taken against the row's maximum less this (in units of log 2): exponentials then reach 2^7, and 2^15 before the maximum is
// moved, and keep all fp16 bits down to 2^-20 of the largest.
constexpr float HEADROOM = 7.0f, KEPT = 15.0f;

struct AttendArgs {
  Pages pages;
  Batch batch;
  const char* q;
  char* out;
  int64_t q_token, q_head, out_token, out_head;  // bytes
  float* lse;
  int64_t* bases;  // [S + 1] units before each sequence, then the number of workgroups that have some
  float* parts;    // sums of pieces
  float c;         // scale log2 e
  int Hq, G, bf16, workgroups, least;
};

__device__ __forceinline__ float max_halves(float x) {
  const auto r = __builtin_amdgcn_permlane32_swap(__builtin_bit_cast(unsigned, x), __builtin_bit_cast(unsigned, x), false, false);
  return fmaxf(__builtin_bit_cast(float, (unsigned)r[0]), __builtin_bit_cast(float, (unsigned)r[1]));
}
__device__ __forceinline__ float add_halves(float x) {
  const auto r = __builtin_amdgcn_permlane32_swap(__builtin_bit_cast(unsigned, x), __builtin_bit_cast(unsigned, x), false, false);
  return __builtin_bit_cast(float, (unsigned)r[0]) + __builtin_bit_cast(float, (unsigned)r[1]);
}

// Eight codes as fp16.
template <typename Code>
__device__ __forceinline__ h8 halves_of(uint32_t a, uint32_t b);
template <>
__device__ __forceinline__ h8 halves_of<E4M3>(uint32_t a, uint32_t b) {
  const h2 x0 = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(a, 1.0f, false), x1 = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(a, 1.0f, true);
  const h2 x2 = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(b, 1.0f, false), x3 = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(b, 1.0f, true);
  return h8{x0[0], x0[1], x1[0], x1[1], x2[0], x2[1], x3[0], x3[1]};
}
// (a byte u = code + 128 below 0x64 is the fp16 number 1024 + u)
template <>
__device__ __forceinline__ h8 halves_of<I8>(uint32_t a, uint32_t b) {
  a ^= 0x80808080u, b ^= 0x80808080u;
  const h2 off = {(_Float16)1152.0f, (_Float16)1152.0f};
  h2 x[4];
  x[0] = __builtin_bit_cast(h2, __builtin_amdgcn_perm(0x64646464u, a, 0x07010700u)) - off;
  x[1] = __builtin_bit_cast(h2, __builtin_amdgcn_perm(0x64646464u, a, 0x07030702u)) - off;
  x[2] = __builtin_bit_cast(h2, __builtin_amdgcn_perm(0x64646464u, b, 0x07010700u)) - off;
  x[3] = __builtin_bit_cast(h2, __builtin_amdgcn_perm(0x64646464u, b, 0x07030702u)) - off;
  return h8{x[0][0], x[0][1], x[1][0], x[1][1], x[2][0], x[2][1], x[3][0], x[3][1]};
}

// --- which work is whose --------------------------------------------------------------------------------------------------------------
//
// A sequence of r rows (a key head) has tiles = ceil(r / 32), for each of them the blocks of its tokens: units (head, tile, block) in
// this order, sequence after sequence.  The workgroups share all units evenly, in order: a segment (sequence, head, tile) that several of them
// meet is joined afterwards.

struct Work {
  int rows, tiles, blocks;
  int64_t units;
  __device__ __forceinline__ Work(const AttendArgs& a, int s) {
    const Sequence seq(a.batch, s);
    rows = min(seq.n, a.batch.most) * a.G;
    tiles = (rows + ROWS - 1) / ROWS;
    const int64_t held = (int64_t)a.batch.width * BT << a.pages.shift;
    blocks = max(1, (int)((min((int64_t)seq.len, held) + BT - 1) / BT));
    units = (int64_t)a.pages.Hkv * tiles * blocks;
  }
};
__device__ __forceinline__ int64_t units_of_lane(const AttendArgs& a, int s) { return s < a.batch.S ? Work(a, s).units : 0; }

__device__ __forceinline__ int64_t shfl64(int64_t x, int from) {
  return (int64_t)((uint64_t)(uint32_t)__shfl((int)(x >> 32), from) << 32 | (uint32_t)__shfl((int)x, from));
}
__device__ __forceinline__ int64_t inclusive(int64_t x) {
  const int lane = threadIdx.x & 63;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const int64_t y = shfl64(x, max(lane - o, 0));
    if (lane >= o) x += y;
  }
  return x;
}

// Workgroups that have units: all, or as many as get `least` each.
__device__ __forceinline__ int64_t sharing(const AttendArgs& a, int64_t units) {
  return max((int64_t)1, min((int64_t)a.workgroups, (units + a.least - 1) / a.least));
}
__device__ __forceinline__ int64_t share_from(int64_t units, int64_t sharers, int64_t w) { return units * w / sharers; }
__device__ __forceinline__ int64_t owner_of(int64_t units, int64_t sharers, int64_t u) { return ((u + 1) * sharers - 1) / units; }

// Sums of pieces, of 32 rows: maximum and sum, then D values each.  A workgroup leaves at most two: of a segment that began before it
// (slot 0) and of one that goes on after it (slot 1).
template <int NI>
struct Part {
  static constexpr int W = NI * 32, FLOATS = ROWS * (W + 2);
};

// --- one wavefront's rows ---------------------------------------------------------------------------------------------------------------

template <typename Code, int NI>
struct Rows {
  h8 q[NI][2];
  f16x o[NI];
  float m, l, c;  // c: the row's scale log2 e
  int sees;       // tokens before this one

  __device__ __forceinline__ void clear() {
#pragma unroll
    for (int i = 0; i < NI; ++i) o[i] = (f16x)(0.0f);
    m = -INFINITY, l = 0.0f;
  }

  // Queries as fp16, the lane's half of every 32 elements.
  __device__ __forceinline__ void load_q(const AttendArgs& a, const char* q, bool valid, int half) {
    const int D = a.pages.D;
    float most = 0.0f;
    uint16_t raw[NI][16];
#pragma unroll
    for (int i = 0; i < NI; ++i)
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const int d = 32 * i + 16 * half + 4 * j;
        const u2 x = valid && d < D ? *reinterpret_cast<const u2*>(q + d * 2) : u2{0u, 0u};
#pragma unroll
        for (int y = 0; y < 4; ++y) raw[i][4 * j + y] = (uint16_t)(x[y >> 1] >> (16 * (y & 1)));
      }
    c = a.c;
    if (!a.bf16) {
#pragma unroll
      for (int i = 0; i < NI; ++i)
#pragma unroll
        for (int j = 0; j < 16; ++j) q_at(i, j) = __builtin_bit_cast(_Float16, raw[i][j]);
      return;
    }
#pragma unroll
    for (int i = 0; i < NI; ++i)
#pragma unroll
      for (int j = 0; j < 16; ++j) {
        const float x = fabsf(to_float(raw[i][j], true));
        most = fmaxf(most, x <= 3.4028235e38f ? x : 0.0f);
      }
    most = max_halves(most);
    // the largest to [2^14, 2^15)
    const int e = most > 0.0f ? (int)(__builtin_bit_cast(uint32_t, most) >> 23) - 127 - 14 : 0;
    c = __builtin_ldexpf(a.c, e);
#pragma unroll
    for (int i = 0; i < NI; ++i)
#pragma unroll
      for (int j = 0; j < 16; ++j) q_at(i, j) = (_Float16)__builtin_ldexpf(to_float(raw[i][j], true), -e);
  }
  struct At {
    h8& v;
    int j;
    __device__ __forceinline__ void operator=(_Float16 x) { v[j] = x; }
  };
  __device__ __forceinline__ At q_at(int i, int j) { return At{q[i][j >> 3], j & 7}; }

  __device__ __forceinline__ f16x scores(const u4 (&k)[NI]) const {
    f16x s = (f16x)(0.0f);
#pragma unroll
    for (int i = 0; i < NI; ++i) {
      s = __builtin_amdgcn_mfma_f32_32x32x16_f16(halves_of<Code>(k[i][0], k[i][1]), q[i][0], s, 0, 0, 0);
      s = __builtin_amdgcn_mfma_f32_32x32x16_f16(halves_of<Code>(k[i][2], k[i][3]), q[i][1], s, 0, 0, 0);
    }
    return s;
  }
  // The scores' exponentials, times the scale of the values; p[0]: tokens 0-3 and 16-19 of each half's, p[1]: 8-11 and 24-27.
  __device__ __forceinline__ void weigh(f16x s, int begin, bool masked, float sk, float sv, int half, h8 (&p)[2]) {
    if (masked) {
      const int x = sees - begin - 4 * half;
#pragma unroll
      for (int r = 0; r < 16; ++r) s[r] = (r >> 2) * 8 + (r & 3) < x ? s[r] : -INFINITY;
    }
    float mx = s[0];
#pragma unroll
    for (int r = 1; r < 16; ++r) mx = fmaxf(mx, s[r]);
    mx = max_halves(mx);
    const float a = sk * c, log_sv = __builtin_amdgcn_logf(sv), x = __builtin_fmaf(mx, a, log_sv);
    const bool grows = x - m > KEPT;
    if (__any(grows)) {
      const float to = grows ? __builtin_ceilf(x) - HEADROOM : m, alpha = grows ? __builtin_amdgcn_exp2f(m - to) : 1.0f;
#pragma unroll
      for (int i = 0; i < NI; ++i) o[i] *= alpha;
      l *= alpha;
      m = to;
    }
    const float base = log_sv - (m == -INFINITY ? 0.0f : m);
    float sum[2] = {0.0f, 0.0f};
#pragma unroll
    for (int r = 0; r < 16; ++r) {
      s[r] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[r], a, base));
      sum[r & 1] += s[r];
    }
    l = __builtin_fmaf(sum[0] + sum[1], 1.0f / sv, l);
#pragma unroll
    for (int r = 0; r < 16; ++r) p[r >> 2 & 1][(r >> 3) * 4 + (r & 3)] = (_Float16)s[r];
  }
  __device__ __forceinline__ void multiply(const u4 (&v)[NI], const h8 (&p)[2]) {
#pragma unroll
    for (int i = 0; i < NI; ++i) {
      o[i] = __builtin_amdgcn_mfma_f32_32x32x16_f16(halves_of<Code>(v[i][0], v[i][1]), p[0], o[i], 0, 0, 0);
      o[i] = __builtin_amdgcn_mfma_f32_32x32x16_f16(halves_of<Code>(v[i][2], v[i][3]), p[1], o[i], 0, 0, 0);
    }
  }
};

__device__ __forceinline__ int lane_value(int x, int lane) { return __builtin_amdgcn_readlane(x, lane); }

// Blocks [begin, end), every `step`-th from begin on, for one wavefront's rows.
template <typename Code, int NI>
__device__ __forceinline__ void run_blocks(const AttendArgs& a, Rows<Code, NI>& w, const int32_t* table, int head, int begin, int end, int step, int least) {
  const int lane = threadIdx.x & 63, half = lane >> 5, chunks = a.pages.chunks;
  // where the lane's 16 bytes of each run of 32 elements lie
  uint32_t v_at[NI];
  bool k_is[NI], v_is[NI];
#pragma unroll
  for (int i = 0; i < NI; ++i) {
    const int n = value_run(chunks, 32 * i);
    k_is[i] = 2 * i + half < chunks;
    v_is[i] = (lane & 31) < n && 2 * i < chunks;
    v_at[i] = i * 1024 + (half * n + (lane & 31)) * 16;
  }
  u4 k[NI], v[NI];
  for (int first = begin; first < end; first += 64 * step) {
    // 64 blocks' places and scales, one a lane
    const int mine = first + lane * step;
    const int64_t unit = mine < end ? a.pages.unit_of(table, a.batch.width, mine, head) : -1;
    float sk = 0.0f, sv = 0.0f;
    if (unit >= 0) {
      const f2 x = *reinterpret_cast<const f2*>(a.pages.scales + unit * 2);
      sk = x[0], sv = x[1];
    }
    uint64_t left = __ballot(unit >= 0);
    if (!left) continue;
    auto take = [&] {
      const int n = __builtin_ctzll(left);
      left &= left - 1;
      return n;
    };
    auto base_of = [&](int n) {
      return a.pages.keys((int64_t)((uint64_t)(uint32_t)lane_value((int)(unit >> 32), n) << 32 | (uint32_t)lane_value((int)unit, n)));
    };
    auto load_k = [&](int n) {
      const char* at = base_of(n);
#pragma unroll
      for (int i = 0; i < NI; ++i) k[i] = k_is[i] ? __builtin_nontemporal_load(reinterpret_cast<const u4*>(at + i * 1024 + lane * 16)) : u4{0u, 0u, 0u, 0u};
    };
    auto load_v = [&](int n) {
      const char* at = base_of(n) + a.pages.plane_bytes();
#pragma unroll
      for (int i = 0; i < NI; ++i) v[i] = v_is[i] ? __builtin_nontemporal_load(reinterpret_cast<const u4*>(at + v_at[i])) : u4{0u, 0u, 0u, 0u};
    };
    int n = take();
    load_k(n), load_v(n);
    while (true) {
      const int next = left ? take() : -1, at = (first + n * step) * BT;
      const f16x s = w.scores(k);
      if (next >= 0) load_k(next);
      h8 p[2];
      w.weigh(s, at, at + BT > least, __builtin_bit_cast(float, lane_value(__builtin_bit_cast(int, sk), n)),
              __builtin_bit_cast(float, lane_value(__builtin_bit_cast(int, sv), n)), half, p);
      w.multiply(v, p);
      if (next < 0) break;
      load_v(next);
      n = next;
    }
  }
}

// What becomes of a row's sums.
__device__ __forceinline__ float log_sum(float m, float l) {
  return (m + HEADROOM + __builtin_log2f(l * __builtin_exp2f(-HEADROOM))) * 0.69314718055994530942f;
}

// One workgroup's share of the units.  WAVES wavefronts take every WAVES-th block of a piece, their sums meet in LDS.
template <typename Code, int NI, int WAVES>
__global__ __launch_bounds__(64 * WAVES, 2) void attend_kernel(const AttendArgs a) {
  typedef Part<NI> P;
  constexpr int PITCH = P::W + 4;
  __shared__ float shared[WAVES == 1 ? 1 : WAVES * ROWS * (PITCH + 2)];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), half = lane >> 5;
  const int S = a.batch.S, D = a.pages.D;
  // all units, then the sequence of the share's first
  int64_t units = 0;
  for (int s = 0; s < S; s += 64) units += shfl64(inclusive(units_of_lane(a, s + lane)), 63);
  const int64_t sharers = sharing(a, units), w = blockIdx.x;
  if (blockIdx.x == 0 && wave == 0) {
    int64_t before = 0;
    for (int s = 0; s < S; s += 64) {
      const int64_t x = units_of_lane(a, s + lane), upto = inclusive(x);
      if (s + lane < S) a.bases[s + lane] = before + upto - x;
      before += shfl64(upto, 63);
    }
    if (lane == 0) a.bases[S] = units, a.bases[S + 1] = sharers;
  }
  if (w >= sharers) return;
  int64_t u = share_from(units, sharers, w);
  const int64_t end = share_from(units, sharers, w + 1);
  if (u >= end) return;
  int s = 0;
  int64_t local = 0, before = 0;
  for (int s0 = 0; s0 < S; s0 += 64) {
    const int64_t x = units_of_lane(a, s0 + lane), upto = before + inclusive(x), last = shfl64(upto, 63);
    if (u < last) {
      const int at = __builtin_ctzll(__ballot(upto > u));
      s = s0 + at;
      local = u - shfl64(upto - x, at);
      break;
    }
    before = last;
  }
  s = __builtin_amdgcn_readfirstlane(s);
  bool first_piece = true;
  while (u < end && s < S) {
    const Work work(a, s);
    if (local >= work.units) {
      ++s, local = 0;
      continue;
    }
    const Sequence seq(a.batch, s);
    const int64_t segment = local / work.blocks;
    const int begin = (int)(local - segment * work.blocks), stop = (int)min((int64_t)work.blocks, begin + (end - u));
    const int head = (int)(segment / work.tiles), tile = (int)(segment % work.tiles);
    // the lane's row
    const int r = tile * ROWS + (lane & 31), i = r / a.G, g = r - i * a.G;
    const bool valid = r < work.rows;
    const int row = seq.row0 + i, hq = head * a.G + g;
    Rows<Code, NI> x;
    const int most = (int)min((int64_t)seq.len, (int64_t)a.batch.width * BT << a.pages.shift);
    x.sees = valid ? clamp_to(seq.first + i + 1, most) : 0x7fffffff;
    x.clear();
    x.load_q(a, a.q + row * a.q_token + hq * a.q_head, valid, half);
    // (the first row of a tile sees least)
    const int least = clamp_to(seq.first + (tile * ROWS) / a.G + 1, most);
    const int mine = WAVES == 1 ? begin : begin + wave;
    run_blocks<Code, NI>(a, x, a.batch.row(s), head, mine, stop, WAVES, least);
    x.l = add_halves(x.l);
    const bool whole = begin == 0 && stop == work.blocks;
    float* part = a.parts + (2 * w + (begin == 0)) * P::FLOATS;
    auto put = [&](bool is, int row, int hq, int in_tile, int d, f4 o, float m, float l) {
      if (!is) return;
      if (whole) {
        const float inv = l > 0.0f || l != l ? 1.0f / l : 0.0f;
        uint16_t e[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) e[j] = from_float(o[j] * inv, a.bf16);
        if (d < D) *reinterpret_cast<u2*>(a.out + row * a.out_token + hq * a.out_head + d * 2) = u2{e[0] | (uint32_t)e[1] << 16, e[2] | (uint32_t)e[3] << 16};
        if (d == 0 && a.lse) a.lse[(int64_t)hq * a.batch.T + row] = log_sum(m, l);
      } else {
        *reinterpret_cast<f4*>(part + 2 * ROWS + in_tile * P::W + d) = o;
        if (d == 0) part[in_tile * 2] = m, part[in_tile * 2 + 1] = l;
      }
    };
    if constexpr (WAVES == 1) {
#pragma unroll
      for (int y = 0; y < NI; ++y)
#pragma unroll
        for (int z = 0; z < 4; ++z)
          put(valid, row, hq, lane & 31, 32 * y + 8 * z + 4 * half, f4{x.o[y][4 * z], x.o[y][4 * z + 1], x.o[y][4 * z + 2], x.o[y][4 * z + 3]}, x.m, x.l);
    } else {
      float* ml = shared + WAVES * ROWS * PITCH;
      if (!first_piece) __syncthreads();  // (the sums before have been read)
      if (half == 0) ml[(wave * ROWS + lane) * 2] = x.m, ml[(wave * ROWS + lane) * 2 + 1] = x.l;
#pragma unroll
      for (int y = 0; y < NI; ++y)
#pragma unroll
        for (int z = 0; z < 4; ++z)
          *reinterpret_cast<f4*>(shared + (wave * ROWS + (lane & 31)) * PITCH + 32 * y + 8 * z + 4 * half) =
              f4{x.o[y][4 * z], x.o[y][4 * z + 1], x.o[y][4 * z + 2], x.o[y][4 * z + 3]};
      __syncthreads();
      const int rows = min(ROWS, work.rows - tile * ROWS);
      for (int k = tid; k < rows * (P::W / 4); k += 64 * WAVES) {
        const int in_tile = k / (P::W / 4), d = k % (P::W / 4) * 4;
        float m = -INFINITY, l = 0.0f;
        f4 o = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
        for (int y = 0; y < WAVES; ++y) m = fmaxf(m, ml[(y * ROWS + in_tile) * 2]);
#pragma unroll
        for (int y = 0; y < WAVES; ++y) {
          const float my = ml[(y * ROWS + in_tile) * 2], f = my == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(my - m);
          l = __builtin_fmaf(ml[(y * ROWS + in_tile) * 2 + 1], f, l);
          o += *reinterpret_cast<const f4*>(shared + (y * ROWS + in_tile) * PITCH + d) * f;
        }
        const int rr = tile * ROWS + in_tile, ii = rr / a.G;
        put(true, seq.row0 + ii, head * a.G + rr - ii * a.G, in_tile, d, o, m, l);
      }
    }
    first_piece = false;
    u += stop - begin;
    local += stop - begin;
  }
}

// Rows of segments that several workgroups met: a wavefront a row, two elements a lane.
template <int NI>
__global__ __launch_bounds__(256) void join_kernel(const AttendArgs a) {
  typedef Part<NI> P;
  const int lane = threadIdx.x & 63;
  const int64_t id = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
  if (id >= (int64_t)a.batch.T * a.Hq) return;
  const int row = __builtin_amdgcn_readfirstlane((int)(id / a.Hq)), hq = __builtin_amdgcn_readfirstlane((int)(id % a.Hq));
  const int s = __builtin_amdgcn_readfirstlane(sequence_of(a.batch, row));
  const Sequence seq(a.batch, s);
  const Work work(a, s);
  const int head = hq / a.G, r = (row - seq.row0) * a.G + hq - head * a.G;
  if (row < seq.row0 || r >= work.rows) return;
  const int64_t units = a.bases[a.batch.S], sharers = a.bases[a.batch.S + 1];
  const int64_t from = a.bases[s] + ((int64_t)head * work.tiles + r / ROWS) * work.blocks;
  const int64_t w0 = owner_of(units, sharers, from), w1 = owner_of(units, sharers, from + work.blocks - 1);
  if (w0 == w1) return;
  const int in_tile = r % ROWS, d = lane * 2;
  auto part_of = [&](int64_t w) { return a.parts + (2 * w + (w == w0)) * P::FLOATS; };
  float m = -INFINITY;
  for (int64_t w = w0 + lane; w <= w1; w += 64) m = fmaxf(m, part_of(w)[in_tile * 2]);
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor(m, o));
  // (fmaxf leaves NaN aside: the sums have it)
  float l = 0.0f;
  f2 sum = {0.0f, 0.0f};
#pragma unroll 4
  for (int64_t w = w0; w <= w1; ++w) {
    const float* p = part_of(w);
    const float my = p[in_tile * 2], f = my == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(my - m);
    l = __builtin_fmaf(p[in_tile * 2 + 1], f, l);
    if (d < P::W) {
      const f2 o = *reinterpret_cast<const f2*>(p + 2 * ROWS + in_tile * P::W + d);
      sum[0] = __builtin_fmaf(o[0], f, sum[0]), sum[1] = __builtin_fmaf(o[1], f, sum[1]);
    }
  }
  const float inv = l > 0.0f || l != l ? 1.0f / l : 0.0f;
  if (d < a.pages.D)
    *reinterpret_cast<uint32_t*>(a.out + row * a.out_token + hq * a.out_head + d * 2) = from_float(sum[0] * inv, a.bf16) | (uint32_t)from_float(sum[1] * inv, a.bf16) << 16;
  if (lane == 0 && a.lse) a.lse[(int64_t)hq * a.batch.T + row] = log_sum(m, l);
}

// --- host ----------------------------------------------------------------------------------------------------------------------------------

static bool desc_ok(const tmac_attn_desc* d, const tmac_pages* p) {
  return d && d->Hq > 0 && d->Hkv == p->Hkv && d->Hq % d->Hkv == 0 && d->D == p->D && (d->elem == TMAC_ELEM_F16 || d->elem == TMAC_ELEM_BF16) &&
         std::isfinite(d->scale) && d->scale > 0 && d->causal == 1 && !d->reserved[0] && !d->reserved[1];
}

struct Plan {
  int workgroups, waves;
  size_t bases, parts;  // bytes
};
static Plan plan_of(const tmac_pages* p, const tmac_pages_batch* b) {
  Plan plan;
  plan.waves = 4;
  plan.workgroups = 512;
  plan.bases = (((size_t)b->S + 2) * 8 + 15) / 16 * 16;
  plan.parts = (size_t)plan.workgroups * 2 * ROWS * ((p->D + 31) / 32 * 32 + 2) * 4;
  return plan;
}

template <typename Code, int WAVES>
static const void* attend_of(int ni) {
  switch (ni) {
    case 1: return (const void*)attend_kernel<Code, 1, WAVES>;
    case 2: return (const void*)attend_kernel<Code, 2, WAVES>;
    case 3: return (const void*)attend_kernel<Code, 3, WAVES>;
    default: return (const void*)attend_kernel<Code, 4, WAVES>;
  }
}
static const void* join_of(int ni) {
  switch (ni) {
    case 1: return (const void*)join_kernel<1>;
    case 2: return (const void*)join_kernel<2>;
    case 3: return (const void*)join_kernel<3>;
    default: return (const void*)join_kernel<4>;
  }
}

}  // namespace pages
}  // namespace tmac

using namespace tmac;
using namespace tmac::pages;

extern "C" size_t tmac_pages_attend_workspace_bytes(const tmac_attn_desc* desc, const tmac_pages* p, const tmac_pages_batch* batch) {
  if (!pages_ok(p) || !batch_ok(batch) || !desc_ok(desc, p) || !supported(p, batch)) return 0;
  const Plan plan = plan_of(p, batch);
  return plan.bases + plan.parts;
}

extern "C" tmac_status tmac_pages_attend(const tmac_attn_desc* desc, const tmac_pages* p, const tmac_pages_batch* batch, const tmac_view* q,
                                         const tmac_view* out, float* lse_dev, void* workspace_dev, size_t workspace_bytes, void* stream) {
  if (!pages_ok(p) || !batch_ok(batch) || !desc_ok(desc, p)) return TMAC_EINVAL;
  if (batch->S == 0 || batch->T == 0) return TMAC_OK;
  if (!pages_set(p) || !batch_set(batch) || !attn::rows_ok(q, false, true, true) || !attn::rows_ok(out, false, true, true)) return TMAC_EINVAL;
  if (!supported(p, batch) || (int64_t)batch->T * desc->Hq > (1 << 30)) return TMAC_EUNSUPPORTED;
  if (!workspace_dev || (reinterpret_cast<uintptr_t>(workspace_dev) & 15)) return TMAC_EINVAL;
  const Plan plan = plan_of(p, batch);
  if (workspace_bytes < plan.bases + plan.parts) return TMAC_ESIZE;
  AttendArgs a = {};
  a.pages = view_of(p), a.batch = view_of(batch);
  a.q = static_cast<const char*>(q->data), a.out = static_cast<char*>(out->data);
  a.q_token = q->token * 2, a.q_head = q->head * 2, a.out_token = out->token * 2, a.out_head = out->head * 2;
  a.lse = lse_dev;
  a.bases = static_cast<int64_t*>(workspace_dev);
  a.parts = reinterpret_cast<float*>(static_cast<char*>(workspace_dev) + plan.bases);
  a.c = desc->scale * 1.44269504088896340736f;
  a.Hq = desc->Hq, a.G = desc->Hq / desc->Hkv, a.bf16 = desc->elem == TMAC_ELEM_BF16;
  a.workgroups = plan.workgroups, a.least = 8;
  const int ni = (p->D + 31) / 32;
  const void* kernel = p->code == TMAC_CODE_I8 ? attend_of<I8, 4>(ni) : attend_of<E4M3, 4>(ni);
  const tmac_status st = launch(kernel, plan.workgroups, 64 * plan.waves, &a, stream);
  if (st != TMAC_OK) return st;
  return launch(join_of(ni), ((int64_t)batch->T * desc->Hq + 3) / 4, 256, &a, stream);
}
