// Attention over pages of keys and values in 8 bits (tmac_pages.h).
//
// Rows of a unit of work are (query token, head of the group) of one sequence and key head.  Products run on the matrix units in
// transposed form, S^T = K Q^T and O^T = V^T P^T, so that a lane owns a row: maximum and sum need one or two exchanges within a
// wavefront, and the exponentials are the second product's operand as they stand.  Codes are whole numbers or e4m3 values,
// which fp16 holds exactly; a block's scales are the same for all its products, so they are taken out of them:
//   x_j = s_j a + log2 sv,  a = sk scale log2 e,  p_j = 2^(x_j - m),  O += sum p_j code_j,  l += (sum p_j) / sv
// with m against the row's largest x, and o = O / l.  m is a whole number.  x has the values' scale, which spans 2^179 (blocks of zeros have 2^-60), so what is far from the largest x may
// still be a part of l like any other: sums l move by whole powers of two, and blocks of small x are lifted (base_of).
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
  float c;  // scale log2 e
  int G, bf16;
  // The sequences of one kind, and how their work is dealt out
  struct Side {
    int rows_from, rows_to;  // sequences of so many rows (a key head)
    int workgroups, least;   // that share the units, and how many at least each
    int spare;               // units that a segment counts more than it has
    int tiles;               // that a sequence may have (many rows: all sequences), where every segment has a workgroup
    struct Note* notes;      // of each of the workgroups that share: the segment that goes on from the share before to this one
    float* parts;            // sums of pieces
  } few, many;
};

// A segment that shares w0 to w1 have pieces of: its rows are rows r = tile_row .. of sequence and head, `rows` in all.  w1 < w0: none.
struct Note {
  int w0, w1, row0, rows, tile_row, head;
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
// A sequence of r rows (a key head) has tiles = ceil(r / ROWS), for each of them the blocks of its tokens (of 32; of 64 where a tile has 128
// rows): units (head, tile, block) in this order, sequence after sequence.  A segment is one (sequence, head, tile).  What a segment costs
// beside its blocks (its queries, first loads, the meeting of its sums) counts as `spare` units before the first.

struct Work {
  Sequence seq;
  int rows, tiles, blocks, held;  // held: tokens that can be seen
  int64_t units;
  template <int ROWS>
  static __device__ __forceinline__ Work of(const AttendArgs& a, const AttendArgs::Side& side, const Sequence& seq) {
    Work w{seq};
    w.rows = min(seq.n, a.batch.most) * a.G;
    if (w.rows < side.rows_from || w.rows > side.rows_to) w.rows = 0;
    w.tiles = (w.rows + ROWS - 1) / ROWS;
    w.held = (int)min((int64_t)seq.len, (int64_t)a.batch.width * BT << a.pages.shift);
    constexpr int TOKENS = ROWS == 128 ? 2 * BT : BT;
    w.blocks = max(1, (w.held + TOKENS - 1) / TOKENS);
    w.units = (int64_t)a.pages.Hkv * w.tiles * (w.blocks + side.spare);
    return w;
  }
};

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
__device__ __forceinline__ int lane_value(int x, int lane) { return __builtin_amdgcn_readlane(x, lane); }
__device__ __forceinline__ float lane_value(float x, int lane) { return __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, x), lane)); }

// Workgroup w has the units from w times the share on.
__device__ __forceinline__ int64_t share_of(const AttendArgs::Side& x, int64_t units) {
  return max((int64_t)x.least, (units + x.workgroups - 1) / x.workgroups);
}

// Sums of pieces: maximum and sum of every row, then W values each.  A workgroup leaves at most two: of a segment that began before it
// (slot 0) and of one that goes on after it (slot 1).
__host__ __device__ __forceinline__ int part_floats(int rows, int width) { return rows * (width + 2); }

// --- one wavefront's rows ---------------------------------------------------------------------------------------------------------------

// What the two shapes have in common: queries as fp16 of a row's elements d_of(i, y) .. + 7.
template <int NQ>
struct Queries {
  h8 q[NQ][2];
  int e;     // they are the row's times 2^-e
  int sees;  // tokens before this one

  // What products with keys of this scale, times scale log2 e, are multiplied with.  Above zero and finite: a token that is not seen has the score -infinity, and
  // products may be zero.  (2^e by itself may be below the smallest number where the whole is not: queries of 2^-120 beside keys of 2^120.)
  __device__ __forceinline__ float factor(float scale) const { return __builtin_amdgcn_fmed3f(__builtin_ldexpf(scale, e), 0x1p-126f, 0x1.fffffep127f); }

  template <typename DOf>
  __device__ __forceinline__ void load(const AttendArgs& a, const char* at, bool valid, DOf&& d_of) {
    u2 raw[NQ][4];
#pragma unroll
    for (int i = 0; i < NQ; ++i)
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const int d = d_of(i) + 4 * j;
        raw[i][j] = valid && d < a.pages.D ? *reinterpret_cast<const u2*>(at + d * 2) : u2{0u, 0u};
      }
    e = 0;
    if (!a.bf16) {
#pragma unroll
      for (int i = 0; i < NQ; ++i)
#pragma unroll
        for (int y = 0; y < 2; ++y) q[i][y] = __builtin_bit_cast(h8, u4{raw[i][2 * y][0], raw[i][2 * y][1], raw[i][2 * y + 1][0], raw[i][2 * y + 1][1]});
      return;
    }
    float most = 0.0f;
    auto bf = [](const u2& x, int y) { return __builtin_bit_cast(float, y & 1 ? x[y >> 1] & 0xffff0000u : x[y >> 1] << 16); };
#pragma unroll
    for (int i = 0; i < NQ; ++i)
#pragma unroll
      for (int j = 0; j < 16; ++j) {
        const float x = fabsf(bf(raw[i][j >> 2], j & 3));
        most = fmaxf(most, x <= 3.4028235e38f ? x : 0.0f);
      }
    // the row's largest (its lanes lie `apart`) to [2^14, 2^15): a power of two, which goes into the factor
    most = over_row(most);
    e = most > 0.0f ? (int)(__builtin_bit_cast(uint32_t, most) >> 23) - 127 - 14 : 0;
#pragma unroll
    for (int i = 0; i < NQ; ++i)
#pragma unroll
      for (int j = 0; j < 16; ++j) q[i][j >> 3][j & 7] = (_Float16)__builtin_ldexpf(bf(raw[i][j >> 2], j & 3), -e);
  }
  int apart;
  __device__ __forceinline__ float over_row(float x) const {
    if (apart == 16) x = fmaxf(x, __shfl_xor(x, 16));
    return fmaxf(x, __shfl_xor(x, 32));
  }
};

// Sums against the maximum m times this power of two are against `to`.  (Whole numbers; -infinity: nothing has been summed.  A factor 2^(m - to) would be zero from 2^-127 on, where l may
// still be a number.)
__device__ __forceinline__ int places(float m, float to) { return (int)fmaxf(m - to, -1000.0f); }

// The running maximum.  x: the largest exponent of the block; returns whether any row's moved, and by what power of two the row's sums are multiplied.
__device__ __forceinline__ bool outgrown(float x, float& m, int& by) {
  const bool grows = x - m > KEPT;
  const float to = grows ? __builtin_ceilf(x) - HEADROOM : m;
  by = grows ? places(m, to) : 0;
  m = to;
  return __any(grows);
}
// What is added to a block's scores, the largest of which is `most`: log2 of the values' scale, less m0.  Where exponentials stay below 2^-30, fp16 holds none of them and the
// products get nothing; they are then lifted to 2^-30, by what their sum is divided by again, since they could be below 2^-126, which is zero too.
__device__ __forceinline__ float base_of(float log_sv, float m0, float most) {
  const float base = log_sv - m0;
  return most == -INFINITY ? base : fmaxf(base, __builtin_ceilf(-30.0f - most));
}

// A block's keys or values.
struct Plane {
  __amdgpu_buffer_rsrc_t rsrc;
  __device__ __forceinline__ Plane(const char* at, int bytes) : rsrc(__builtin_amdgcn_make_buffer_rsrc(const_cast<char*>(at), (short)0, bytes, 0x00020000)) {}
  // (read once: past the caches)
  __device__ __forceinline__ u4 load16(const At& at) const { return __builtin_bit_cast(u4, __builtin_amdgcn_raw_buffer_load_b128(rsrc, at.lane + at.fixed, 0, 2)); }
  // (the others of the head's tiles read it too)
  __device__ __forceinline__ u4 load16_kept(int lane) const { return __builtin_bit_cast(u4, __builtin_amdgcn_raw_buffer_load_b128(rsrc, lane, 0, 0)); }
  __device__ __forceinline__ u2 load8(const At& at) const { return __builtin_bit_cast(u2, __builtin_amdgcn_raw_buffer_load_b64(rsrc, at.lane + at.fixed, 0, 2)); }
};

template <typename Code, int NI, int ROWS>
struct Rows;

// 32 rows: v_mfma_f32_32x32x16, row lane & 31.  One block on its way: its registers hold no more at two wavefronts a SIMD.
template <typename Code, int NI>
struct Rows<Code, NI, 32> {
  static constexpr int NK = NI, NV = NI, DEPTH = 1;
  typedef u4 KRaw;
  typedef u4 VRaw;
  Queries<NI> q;
  f16x o[NI];
  float m, l;
  int lane;

  static __device__ __forceinline__ int row(int lane) { return lane & 31; }
  static __device__ __forceinline__ void load_k(u4 (&k)[NK], const Plane& p, int lane) {
#pragma unroll
    for (int i = 0; i < NK; ++i) k[i] = p.load16(Reads32::k(i, lane));
  }
  static __device__ __forceinline__ void load_v(u4 (&v)[NV], const Plane& p, int lane, bool odd) {
#pragma unroll
    for (int i = 0; i < NV; ++i) v[i] = p.load16(Reads32::v(i, lane, i == NV - 1, odd));
  }
  __device__ __forceinline__ void begin(const AttendArgs& a, const char* at, bool valid, int sees) {
    const int half = lane >> 5;
    q.apart = 32, q.sees = sees;
    q.load(a, at, valid, [&](int i) { return 32 * i + 16 * half; });
#pragma unroll
    for (int i = 0; i < NI; ++i) o[i] = (f16x)(0.0f);
    m = -INFINITY, l = 0.0f;
  }
  typedef f16x Scores;
  __device__ __forceinline__ f16x scores(const u4 (&k)[NK]) const {
    f16x s = (f16x)(0.0f);
#pragma unroll
    for (int i = 0; i < NI; ++i) {
      s = __builtin_amdgcn_mfma_f32_32x32x16_f16(halves_of<Code>(k[i][0], k[i][1]), q.q[i][0], s, 0, 0, 0);
      s = __builtin_amdgcn_mfma_f32_32x32x16_f16(halves_of<Code>(k[i][2], k[i][3]), q.q[i][1], s, 0, 0, 0);
    }
    return s;
  }
  // [0]: tokens 0-3 and 16-19 of the half's, [1]: 8-11 and 24-27, as two fp16 numbers each: the result is off by its own rounding only
  struct Weights { h8 p[2], rest[2]; };
  // sk: of the block's keys, times scale log2 e
  __device__ __forceinline__ Weights weigh(f16x s, int begin, bool masked, float sk, float sv) {
    if (masked) {
      const int x = q.sees - begin - 4 * (lane >> 5);
#pragma unroll
      for (int r = 0; r < 16; ++r) s[r] = (r >> 2) * 8 + (r & 3) < x ? s[r] : -INFINITY;
    }
    float mx = s[0];
#pragma unroll
    for (int r = 1; r < 16; ++r) mx = fmaxf(mx, s[r]);
    mx = max_halves(mx);
    const float a = q.factor(sk), log_sv = __builtin_amdgcn_logf(sv);
    int by;
    if (outgrown(__builtin_fmaf(mx, a, log_sv), m, by)) {
#pragma unroll
      for (int i = 0; i < NI; ++i) o[i] *= __builtin_ldexpf(1.0f, by);
      l = __builtin_ldexpf(l, by);
    }
    const float m0 = m == -INFINITY ? 0.0f : m, base = base_of(log_sv, m0, mx * a);
    float sum[2] = {0.0f, 0.0f};
#pragma unroll
    for (int r = 0; r < 16; ++r) {
      s[r] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[r], a, base));
      sum[r & 1] += s[r];
    }
    // (without the scale, or what stands for it, again by what the exponents really had of it: base is rounded, base + m0 is not)
    l = __builtin_fmaf(sum[0] + sum[1], __builtin_amdgcn_exp2f(-(base + m0)), l);
    Weights w;
#pragma unroll
    for (int r = 0; r < 16; ++r) w.p[r >> 2 & 1][(r >> 3) * 4 + (r & 3)] = (_Float16)s[r];
#pragma unroll
    for (int r = 0; r < 16; ++r) w.rest[r >> 2 & 1][(r >> 3) * 4 + (r & 3)] = (_Float16)(s[r] - (float)w.p[r >> 2 & 1][(r >> 3) * 4 + (r & 3)]);
    return w;
  }
  __device__ __forceinline__ void multiply(const u4 (&v)[NV], const Weights& w) {
#pragma unroll
    for (int i = 0; i < NI; ++i) {
#pragma unroll
      for (int y = 0; y < 2; ++y) {
        const h8 x = halves_of<Code>(v[i][2 * y], v[i][2 * y + 1]);
        o[i] = __builtin_amdgcn_mfma_f32_32x32x16_f16(x, w.p[y], o[i], 0, 0, 0);
        o[i] = __builtin_amdgcn_mfma_f32_32x32x16_f16(x, w.rest[y], o[i], 0, 0, 0);
      }
    }
  }
  __device__ __forceinline__ float sum() const { return add_halves(l); }
  // f(d, four sums from there on)
  template <typename F>
  __device__ __forceinline__ void each(F&& f) const {
    const int half = lane >> 5;
#pragma unroll
    for (int i = 0; i < NI; ++i)
#pragma unroll
      for (int z = 0; z < 4; ++z) f(32 * i + 8 * z + 4 * half, f4{o[i][4 * z], o[i][4 * z + 1], o[i][4 * z + 2], o[i][4 * z + 3]});
  }
};

// 16 rows: v_mfma_f32_16x16x32, row lane & 15.  Half the work of 32 for what is read, and half the registers, which take a second block on its way
// (32 sequences of 16384 tokens, 1.08 GB: 162 us = 6.7 TB/s, with one block and three wavefronts a SIMD 171).
template <typename Code, int NI>
struct Rows<Code, NI, 16> {
  static constexpr int NQ = (NI + 1) / 2, NK = 2 * NQ, NV = 2 * NI, DEPTH = 2;
  typedef u4 KRaw;
  typedef u2 VRaw;
  Queries<NQ> q;
  f4 o[NV];
  float m, l;
  int lane;

  static __device__ __forceinline__ int row(int lane) { return lane & 15; }
  static __device__ __forceinline__ void load_k(u4 (&k)[NK], const Plane& p, int lane) {
#pragma unroll
    for (int i = 0; i < NK; ++i) k[i] = p.load16(Reads16::k(i, lane));
  }
  static __device__ __forceinline__ void load_v(u2 (&v)[NV], const Plane& p, int lane, bool odd) {
#pragma unroll
    for (int i = 0; i < NV; ++i) v[i] = p.load8(Reads16::v(i, lane, i >= NV - 2, odd));
  }
  __device__ __forceinline__ void begin(const AttendArgs& a, const char* at, bool valid, int sees) {
    const int quarter = lane >> 4;
    q.apart = 16, q.sees = sees;
    q.load(a, at, valid, [&](int i) { return 16 * (4 * i + quarter); });
#pragma unroll
    for (int i = 0; i < NV; ++i) o[i] = (f4)(0.0f);
    m = -INFINITY, l = 0.0f;
  }
  struct Scores { f4 s[2]; };
  __device__ __forceinline__ Scores scores(const u4 (&k)[NK]) const {
    Scores s = {{(f4)(0.0f), (f4)(0.0f)}};
#pragma unroll
    for (int i = 0; i < NQ; ++i)
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        s.s[t] = __builtin_amdgcn_mfma_f32_16x16x32_f16(halves_of<Code>(k[2 * i + t][0], k[2 * i + t][1]), q.q[i][0], s.s[t], 0, 0, 0);
        s.s[t] = __builtin_amdgcn_mfma_f32_16x16x32_f16(halves_of<Code>(k[2 * i + t][2], k[2 * i + t][3]), q.q[i][1], s.s[t], 0, 0, 0);
      }
    return s;
  }
  // Tokens 0-3 of the quarter's four and 16 on.  As two fp16 numbers each, as above: eight more of the short matrix instructions a block, which memory's
  // time hides (a batch's step 46 us with and without).
  struct Weights { h8 p, rest; };
  static __device__ __forceinline__ float over_row(float x, bool adds) {
    const auto r = __builtin_amdgcn_permlane16_swap(__builtin_bit_cast(unsigned, x), __builtin_bit_cast(unsigned, x), false, false);
    const float a = __builtin_bit_cast(float, (unsigned)r[0]), b = __builtin_bit_cast(float, (unsigned)r[1]);
    return adds ? add_halves(a + b) : max_halves(fmaxf(a, b));
  }
  __device__ __forceinline__ Weights weigh(Scores x, int begin, bool masked, float sk, float sv) {
    float s[8];
#pragma unroll
    for (int r = 0; r < 8; ++r) s[r] = x.s[r >> 2][r & 3];
    if (masked) {
      const int upto = q.sees - begin - 4 * (lane >> 4);
#pragma unroll
      for (int r = 0; r < 8; ++r) s[r] = (r >> 2) * 16 + (r & 3) < upto ? s[r] : -INFINITY;
    }
    float mx = s[0];
#pragma unroll
    for (int r = 1; r < 8; ++r) mx = fmaxf(mx, s[r]);
    mx = over_row(mx, false);
    const float a = q.factor(sk), log_sv = __builtin_amdgcn_logf(sv);
    int by;
    if (outgrown(__builtin_fmaf(mx, a, log_sv), m, by)) {
#pragma unroll
      for (int i = 0; i < NV; ++i) o[i] *= __builtin_ldexpf(1.0f, by);
      l = __builtin_ldexpf(l, by);
    }
    const float m0 = m == -INFINITY ? 0.0f : m, base = base_of(log_sv, m0, mx * a);
    float sum[2] = {0.0f, 0.0f};
#pragma unroll
    for (int r = 0; r < 8; ++r) {
      s[r] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[r], a, base));
      sum[r & 1] += s[r];
    }
    l = __builtin_fmaf(sum[0] + sum[1], __builtin_amdgcn_exp2f(-(base + m0)), l);  // (as with 32 rows)
    Weights w;
#pragma unroll
    for (int r = 0; r < 8; ++r) w.p[r] = (_Float16)s[r];
#pragma unroll
    for (int r = 0; r < 8; ++r) w.rest[r] = (_Float16)(s[r] - (float)w.p[r]);
    return w;
  }
  __device__ __forceinline__ void multiply(const u2 (&v)[NV], const Weights& w) {
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const h8 x = halves_of<Code>(v[i][0], v[i][1]);
      o[i] = __builtin_amdgcn_mfma_f32_16x16x32_f16(x, w.p, o[i], 0, 0, 0);
      o[i] = __builtin_amdgcn_mfma_f32_16x16x32_f16(x, w.rest, o[i], 0, 0, 0);
    }
  }
  __device__ __forceinline__ float sum() const { return over_row(l, true); }
  template <typename F>
  __device__ __forceinline__ void each(F&& f) const {
    const int quarter = lane >> 4;
#pragma unroll
    for (int i = 0; i < NV; ++i) f(16 * i + 4 * quarter, o[i]);
  }
};

// Places and scales of up to 64 blocks, one a lane: blocks first, first + step, ... before end.
struct Blocks {
  int64_t unit;
  float sk, sv;
  // The page of the lane's block (which may be asked for before it is known where the blocks end).
  static __device__ __forceinline__ int page_of(const AttendArgs& a, const int32_t* table, int first, int step, int lane) {
    const int at = (first + lane * step) >> a.pages.shift;
    return at < a.batch.width ? table[at] : -1;
  }
  __device__ __forceinline__ Blocks(const AttendArgs& a, int page, int head, int first, int end, int step, int lane) : sk(0.0f), sv(0.0f) {
    const int mine = first + lane * step;
    unit = mine < end && (unsigned)page < (unsigned)a.pages.pages ? a.pages.unit(page, mine & ((1 << a.pages.shift) - 1), head) : -1;
  }
  __device__ __forceinline__ void scales(const AttendArgs& a) {
    if (unit >= 0) {
      const f2 x = *reinterpret_cast<const f2*>(a.pages.scales + unit * 2);
      sk = x[0], sv = x[1];
    }
  }
  __device__ __forceinline__ const char* at(const AttendArgs& a, int n) const {
    return a.pages.keys((int64_t)((uint64_t)(uint32_t)lane_value((int)(unit >> 32), n) << 32 | (uint32_t)lane_value((int)unit, n)));
  }
};

// Blocks first, first + step, ... before end for one wavefront's rows, whose queries q() loads.  least: tokens that every row sees.
// page: of the lane's first block.  R::DEPTH blocks are on their way: a block's keys are requested as soon as the ones in their registers have met the queries, its values as soon as
// those have met the exponentials.
template <typename R, typename Q>
__device__ __forceinline__ void run_blocks(const AttendArgs& a, R& w, const int32_t* table, int page, int head, int first, int end, int step, int least, Q&& q) {
  const int lane = w.lane, plane = a.pages.plane_bytes();
  const bool odd = a.pages.chunks & 1;
  typename R::KRaw k[R::DEPTH][R::NK];
  typename R::VRaw v[R::DEPTH][R::NV];
  bool loaded = false;
  for (; first < end; first += 64 * step) {
    if (loaded) page = Blocks::page_of(a, table, first, step, lane);
    Blocks blocks(a, page, head, first, end, step, lane);
    if (!loaded) q();
    loaded = true;
    uint64_t left = __ballot(blocks.unit >= 0);
    if (!left) continue;
    auto take = [&] {
      if (!left) return -1;
      const int n = __builtin_ctzll(left);
      left &= left - 1;
      return n;
    };
    auto load_k = [&](int j, int n) { R::load_k(k[j], Plane(blocks.at(a, n), plane), lane); };
    auto load_v = [&](int j, int n) { R::load_v(v[j], Plane(blocks.at(a, n) + plane, plane), lane, odd); };
    int n[R::DEPTH];
#pragma unroll
    for (int j = 0; j < R::DEPTH; ++j) {
      n[j] = take();
      if (n[j] >= 0) load_k(j, n[j]);
      if (j == 0) blocks.scales(a);
      if (n[j] >= 0) load_v(j, n[j]);
    }
    while (n[0] >= 0) {
#pragma unroll
      for (int j = 0; j < R::DEPTH; ++j) {
        if (j && n[j] < 0) break;
        const int next = take(), at = (first + n[j] * step) * BT;
        const typename R::Scores s = w.scores(k[j]);
        if (next >= 0) load_k(j, next);
        const typename R::Weights p = w.weigh(s, at, at + BT > least, lane_value(blocks.sk, n[j]) * a.c, lane_value(blocks.sv, n[j]));
        w.multiply(v[j], p);
        if (next >= 0) load_v(j, next);
        n[j] = next;
      }
    }
  }
  if (!loaded) q();
}

// What becomes of a row's sums.
__device__ __forceinline__ float log_sum(float m, float l) {
  return (m + HEADROOM + __builtin_log2f(l * __builtin_exp2f(-HEADROOM))) * 0.69314718055994530942f;
}

// A row's result: sums from d on, or its lse.
__device__ __forceinline__ void put_out(const AttendArgs& a, int row, int hq, int d, const f4& o, float m, float l) {
  const float inv = l > 0.0f || l != l ? 1.0f / l : 0.0f;
  uint16_t e[4];
#pragma unroll
  for (int j = 0; j < 4; ++j) e[j] = from_float(o[j] * inv, a.bf16);
  if (d < a.pages.D)
    *reinterpret_cast<u2*>(a.out + row * a.out_token + hq * a.out_head + d * 2) = u2{e[0] | (uint32_t)e[1] << 16, e[2] | (uint32_t)e[3] << 16};
  if (d == 0 && a.lse) a.lse[(int64_t)hq * a.batch.T + row] = log_sum(m, l);
}

// A piece of a segment: blocks [begin, stop).  Four wavefronts take every fourth, their sums meet in LDS.  part: where the piece's sums
// go, null: it is the whole segment, whose results go out.
constexpr int WAVES = 4;
template <int NI, int ROWS>
struct Meeting {
  static constexpr int W = NI * 32, PITCH = W + 4, FLOATS = WAVES * ROWS * (PITCH + 2);
};
template <typename Code, int NI, int ROWS>
__device__ __forceinline__ void run_piece(const AttendArgs& a, const Work& work, int s, int head, int tile, int begin, int stop, float* part, float* shared,
                                          bool again, int page) {
  typedef Meeting<NI, ROWS> M;
  constexpr int W = M::W, PITCH = M::PITCH;
  // (named anew for every piece: else what follows from it is worked out before the first and kept in 40 registers)
  int tid = threadIdx.x;
  asm volatile("" : "+v"(tid));
  const int lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  Rows<Code, NI, ROWS> x;
  x.lane = lane;
  const Sequence& seq = work.seq;
  // the lane's row
  const int in = x.row(lane), r = tile * ROWS + in, i = r / a.G, row = seq.row0 + i, hq = head * a.G + r - i * a.G;
  const bool valid = r < work.rows;
  // (the first row of a tile sees least)
  const int least = clamp_to(seq.first + (tile * ROWS) / a.G + 1, work.held);
  run_blocks(a, x, a.batch.row(s), page, head, begin + wave, stop, WAVES, least,
             [&] { x.begin(a, a.q + row * a.q_token + hq * a.q_head, valid, valid ? clamp_to(seq.first + i + 1, work.held) : 0x7fffffff); });
  const float l = x.sum();
  auto put = [&](int row, int hq, int in, int d, const f4& o, float m, float l) {
    if (!part) {
      put_out(a, row, hq, d, o, m, l);
    } else {
      *reinterpret_cast<f4*>(part + 2 * ROWS + in * W + d) = o;
      if (d == 0) part[in * 2] = m, part[in * 2 + 1] = l;
    }
  };
  float* ml = shared + WAVES * ROWS * PITCH;
  if (again) __syncthreads();  // (the sums before have been read)
  if (lane < ROWS) ml[(wave * ROWS + lane) * 2] = x.m, ml[(wave * ROWS + lane) * 2 + 1] = l;
  x.each([&](int d, const f4& o) { *reinterpret_cast<f4*>(shared + (wave * ROWS + in) * PITCH + d) = o; });
  __syncthreads();
  const int rows = min(ROWS, work.rows - tile * ROWS);
  for (int k = tid; k < rows * (W / 4); k += 64 * WAVES) {
    const int in = k / (W / 4), d = k % (W / 4) * 4;
    float m = -INFINITY, l = 0.0f;
    f4 o = {0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
    for (int y = 0; y < WAVES; ++y) m = fmaxf(m, ml[(y * ROWS + in) * 2]);
#pragma unroll
    for (int y = 0; y < WAVES; ++y) {
      const int by = places(ml[(y * ROWS + in) * 2], m);
      l += __builtin_ldexpf(ml[(y * ROWS + in) * 2 + 1], by);
      o += *reinterpret_cast<const f4*>(shared + (y * ROWS + in) * PITCH + d) * __builtin_ldexpf(1.0f, by);
    }
    const int r = tile * ROWS + in, i = r / a.G;
    put(seq.row0 + i, head * a.G + r - i * a.G, in, d, o, m, l);
  }
}

// A workgroup a segment: for short caches, where the launch that joins pieces would cost more (32 segments of 300 tokens 5.6 us: lengths and pages, scales
// and first keys, values, the meeting of four wavefronts, one wait after the other).
template <typename Code, int NI, int ROWS>
__global__ __launch_bounds__(64 * WAVES, 2) void attend_whole_kernel(const AttendArgs a) {
  __shared__ float shared[Meeting<NI, ROWS>::FLOATS];
  const int head = blockIdx.x % a.pages.Hkv, x = blockIdx.x / a.pages.Hkv, tile = x % a.few.tiles, s = x / a.few.tiles;
  const int page = Blocks::page_of(a, a.batch.row(s), threadIdx.x >> 6, WAVES, threadIdx.x & 63);  // (beside the lengths)
  const Work work = Work::of<ROWS>(a, a.few, Sequence(a.batch, s));
  if (tile >= work.tiles) return;
  run_piece<Code, NI, ROWS>(a, work, s, head, tile, 0, work.blocks, nullptr, shared, false, page);
}

// A workgroup's equal share of all units, in order: piece(work, sequence, head, tile, first and last block, whether that is the whole segment, whether there
// was a piece before).  A segment that several workgroups meet is joined afterwards.  numbers: of 64 sequences, Sequence's row0, n, len.
template <int ROWS, typename Piece>
__device__ __forceinline__ void walk_share(const AttendArgs& a, const AttendArgs::Side& side, int w, int (*numbers)[64], Piece&& piece) {
  const int lane = threadIdx.x & 63, S = a.batch.S;
  auto units_of = [&](int s0, bool keep) {
    Sequence seq;
    if (s0 + lane < S) seq = Sequence(a.batch, s0 + lane);
    if (keep) numbers[0][lane] = seq.row0, numbers[1][lane] = seq.n, numbers[2][lane] = seq.len;
    return Work::of<ROWS>(a, side, seq).units;
  };
  int64_t u, end, local, length;
  int s0 = 0, at;
  {
    int64_t x = units_of(0, true), upto = inclusive(x), units = shfl64(upto, 63);
    for (int i = 64; i < S; i += 64) units += shfl64(inclusive(units_of(i, false)), 63);
    const int64_t share = share_of(side, units);
    if (threadIdx.x == 0) side.notes[w] = Note{0, -1, 0, 0, 0, 0};
    u = share * w, end = min(units, u + share);
    if (u >= end) return;
    length = share;
    // the share's first sequence
    int64_t before = 0;
    while (u >= before + shfl64(upto, 63) && s0 + 64 < S) {
      before += shfl64(upto, 63);
      s0 += 64;
      x = units_of(s0, true);
      upto = inclusive(x);
    }
    at = __builtin_ctzll(__ballot(before + upto > u) | (uint64_t)1 << 63);
    local = u - (before + shfl64(upto - x, at));
  }
  bool again = false;
  while (u < end && s0 + at < S) {
    Sequence seq;
    seq.row0 = __builtin_amdgcn_readfirstlane(numbers[0][at]), seq.n = __builtin_amdgcn_readfirstlane(numbers[1][at]);
    seq.len = __builtin_amdgcn_readfirstlane(numbers[2][at]), seq.first = seq.len - seq.n;
    const Work work = Work::of<ROWS>(a, side, seq);
    if (local >= work.units) {
      local = 0;
      if (++at == 64) {
        at = 0, s0 += 64;
        units_of(s0, true);
      }
      continue;
    }
    const int whole = work.blocks + side.spare, segment = (int)(local / whole);
    const int from = (int)(local - (int64_t)segment * whole), to = (int)min((int64_t)whole, from + (end - u));
    if (to > side.spare) {
      const int begin = max(0, from - side.spare), stop = to - side.spare;
      if (begin > 0) {  // (the share's first piece: the first border within the segment has the note)
        const int64_t first = u - begin;
        const int w0 = (int)(first / length);
        if (w0 == w - 1 && threadIdx.x == 0)
          side.notes[w] = Note{w0, (int)((first + work.blocks - 1) / length), work.seq.row0, work.rows, segment % work.tiles * ROWS, segment / work.tiles};
      }
      piece(work, s0 + at, segment / work.tiles, segment % work.tiles, begin, stop, begin == 0 && stop == work.blocks, again);
      again = true;
    }
    u += to - from;
    local += to - from;
  }
}

// Where the sums of a share's piece go: slot 0 of a segment that began before the share, slot 1 of one that goes on after it.
__device__ __forceinline__ float* part_at(const AttendArgs::Side& side, int w, int begin, int floats) { return side.parts + (2 * (int64_t)w + (begin == 0)) * floats; }

template <typename Code, int NI, int ROWS>
__device__ __forceinline__ void run_share(const AttendArgs& a, int w, float* shared, int (*numbers)[64]) {
  walk_share<ROWS>(a, a.few, w, numbers, [&](const Work& work, int s, int head, int tile, int begin, int stop, bool whole, bool again) {
    const int page = Blocks::page_of(a, a.batch.row(s), begin + (int)(threadIdx.x >> 6), WAVES, threadIdx.x & 63);
    run_piece<Code, NI, ROWS>(a, work, s, head, tile, begin, stop, whole ? nullptr : part_at(a.few, w, begin, part_floats(ROWS, NI * 32)), shared, again, page);
  });
}
template <typename Code, int NI, int ROWS>
__global__ __launch_bounds__(256, 2) void attend_kernel(const AttendArgs a) {
  __shared__ float shared[Meeting<NI, ROWS>::FLOATS];
  __shared__ int numbers[4][3][64];
  run_share<Code, NI, ROWS>(a, blockIdx.x, shared, numbers[threadIdx.x >> 6]);
}

// --- many rows ------------------------------------------------------------------------------------------------------------------------------
//
// 128 rows a workgroup, 32 a wavefront: stages of 64 tokens are brought to fp16 once for all four, on their way from registers to LDS, two
// stages there: one is multiplied while the next is made and the one after that is on its way from memory.  Bound by products and exponentials that mostly take
// turns (1024 rows after 7168 tokens, 64 heads in groups of 8: 293 to 312 us by the machine, 0.82 to 0.88 PFLOP/s; matrix units 37 % busy, vector ALUs 54 %, LDS without conflicts, 2.0
// of 2.4 GHz; codes to fp16 are about a fifth of the vector instructions).
//
// Exponentials are one fp16 number each here, as in the prompts' attention (off by 2^-11 of themselves, the size of the result's own rounding; two for all rows: 400 us).  Sequences of up to
// EXACT_ROWS rows come here when others have more, and to smaller tiles when they are alone: they get two numbers in both, so that how exact a sequence's results are does not
// depend on the others.

constexpr int TILE = 128, STAGE = 64, EXACT_ROWS = 64;

template <int NI>
struct Staged {
  // Bytes: keys of a block [2 NI chunks][2][32 tokens] of 16 bytes, values [NI runs][2][2 halves][32 elements]
  static constexpr int PLANE = NI * 2048, BLOCK = 2 * PLANE, BYTES = 2 * BLOCK;
};

// TWO: exponentials as two fp16 numbers
template <typename Code, int NI, bool TWO>
__device__ __forceinline__ void run_tile(const AttendArgs& a, const Work& work, int s, int head, int tile, int begin, int stop, float* part, char* shared, bool again) {
  typedef Staged<NI> L;
  int tid = threadIdx.x;
  asm volatile("" : "+v"(tid));  // (as in run_piece)
  const int lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), half = lane >> 5;
  const Sequence& seq = work.seq;
  const int in = wave * 32 + (lane & 31), r = tile * TILE + in, i = r / a.G, row = seq.row0 + i, hq = head * a.G + r - i * a.G;
  const bool valid = r < work.rows;
  // tokens that the wavefront's first and last rows see
  const int first = tile * TILE + wave * 32, last = min(first + 31, work.rows - 1);
  const int least = clamp_to(seq.first + first / a.G + 1, work.held), most = first < work.rows ? clamp_to(seq.first + last / a.G + 1, work.held) : 0;
  const int32_t* table = a.batch.row(s);
  const int plane = a.pages.plane_bytes(), chunks = a.pages.chunks;
  // (stages that no row of the tile sees: shares count them)
  stop = max(begin, min(stop, (clamp_to(seq.first + (min((tile + 1) * TILE, work.rows) - 1) / a.G + 1, work.held) + STAGE - 1) / STAGE));
  // places and scales of 32 stages' blocks, one a lane; a stage's raw codes, 16 bytes of each plane a thread
  const int held_blocks = (work.held + BT - 1) / BT;
  int placed = begin;
  auto places = [&] {
    Blocks x(a, Blocks::page_of(a, table, placed * 2, 1, lane), head, placed * 2, held_blocks, 1, lane);
    x.scales(a);
    if (x.unit < 0) x.sk = 1.0f, x.sv = -1.0f;  // (a block that is not there: no token of it is seen)
    return x;
  };
  Blocks blocks = places();
  u4 raw[2][2];
  float scales[2][2], next_scales[2][2];
  auto fetch = [&](int stage) {
    if (stage == placed + 32) {
      placed = stage;
      blocks = places();
    }
#pragma unroll
    for (int b = 0; b < 2; ++b) {
      const int n = (stage - placed) * 2 + b;
      next_scales[b][0] = lane_value(blocks.sk, n), next_scales[b][1] = lane_value(blocks.sv, n);
      const bool there = lane_value((int)(blocks.unit >> 32), n) >= 0;
      const char* at = there ? blocks.at(a, n) : a.pages.codes;
      raw[b][0] = Plane(at, there ? plane : 0).load16_kept(tid * 16);
      raw[b][1] = Plane(at + plane, there ? plane : 0).load16_kept(tid * 16);
    }
  };
  // where this thread's 16 codes of either plane go
  const int run = tid >> 6, n = value_run(chunks, run * 32), in_run = tid & 63;
  const uint32_t k_to = ((tid >> 5) * 64 + (tid & 31)) * 16, v_to = (run * 128 + (in_run / n) * 32 + in_run % n) * 16;
  const bool k_is = tid < NI * 64, v_is = tid < chunks * 32;
  auto make = [&](int place) {
#pragma unroll
    for (int b = 0; b < 2; ++b) {
      char* to = shared + place * L::BYTES + b * L::BLOCK;
      if (k_is) {
        *reinterpret_cast<h8*>(to + k_to) = halves_of<Code>(raw[b][0][0], raw[b][0][1]);
        *reinterpret_cast<h8*>(to + k_to + 512) = halves_of<Code>(raw[b][0][2], raw[b][0][3]);
      }
      if (v_is) {
        *reinterpret_cast<h8*>(to + L::PLANE + v_to) = halves_of<Code>(raw[b][1][0], raw[b][1][1]);
        *reinterpret_cast<h8*>(to + L::PLANE + v_to + 1024) = halves_of<Code>(raw[b][1][2], raw[b][1][3]);
      }
      scales[b][0] = next_scales[b][0], scales[b][1] = next_scales[b][1];
    }
  };
  Rows<Code, NI, 32> x;
  x.lane = lane;
  fetch(begin);
  x.begin(a, a.q + row * a.q_token + hq * a.q_head, valid, valid ? clamp_to(seq.first + i + 1, work.held) : 0x7fffffff);
  if (again) __syncthreads();  // (the stages before have been read)
  make(0);
  if (begin + 1 < stop) fetch(begin + 1);
  __syncthreads();
  int place = 0;
  const char* const k_from = shared + (half * 64 + (lane & 31)) * 16;
  const char* const v_from = shared + L::PLANE + (half * 32 + (lane & 31)) * 16;
  for (int stage = begin; stage < stop; ++stage) {
    const int at = stage * STAGE;
    if (at < most) {
      const char* k = k_from + place * L::BYTES;
      const char* v = v_from + place * L::BYTES;
      f16x sc[2] = {(f16x)(0.0f), (f16x)(0.0f)};
#pragma unroll
      for (int t = 0; t < NI; ++t)
#pragma unroll
        for (int y = 0; y < 2; ++y)
#pragma unroll
          for (int b = 0; b < 2; ++b)
            sc[b] = __builtin_amdgcn_mfma_f32_32x32x16_f16(*reinterpret_cast<const h8*>(k + b * L::BLOCK + t * 2048 + y * 512), x.q.q[t][y], sc[b], 0, 0, 0);
      if (at + STAGE > least || scales[0][1] < 0.0f || scales[1][1] < 0.0f) {
#pragma unroll
        for (int b = 0; b < 2; ++b) {
          const int upto = scales[b][1] < 0.0f ? -1 : x.q.sees - at - b * BT - 4 * half;
#pragma unroll
          for (int r = 0; r < 16; ++r) sc[b][r] = (r >> 2) * 8 + (r & 3) < upto ? sc[b][r] : -INFINITY;
        }
      }
      float scale[2], base[2], largest[2], top = -INFINITY;
#pragma unroll
      for (int b = 0; b < 2; ++b) {
        float mx = sc[b][0];
#pragma unroll
        for (int r = 1; r < 16; ++r) mx = fmaxf(mx, sc[b][r]);
        scale[b] = x.q.factor(scales[b][0] * a.c), base[b] = __builtin_amdgcn_logf(fabsf(scales[b][1]));
        top = fmaxf(top, __builtin_fmaf(mx, scale[b], base[b]));
        largest[b] = mx * scale[b];  // (of the lane's tokens, whose sum is its own)
      }
      top = max_halves(top);
      int by;
      if (outgrown(top, x.m, by)) {
#pragma unroll
        for (int d = 0; d < NI; ++d) x.o[d] *= __builtin_ldexpf(1.0f, by);
        x.l = __builtin_ldexpf(x.l, by);
      }
      const float m0 = x.m == -INFINITY ? 0.0f : x.m;
      h8 p[2][2], rest[2][2];
#pragma unroll
      for (int b = 0; b < 2; ++b) {
        base[b] = base_of(base[b], m0, largest[b]);
        float sum[2] = {0.0f, 0.0f};
#pragma unroll
        for (int r = 0; r < 16; ++r) {
          const float e = __builtin_amdgcn_exp2f(__builtin_fmaf(sc[b][r], scale[b], base[b]));
          sum[r & 1] += e;
          const int y = r >> 2 & 1, j = (r >> 3) * 4 + (r & 3);
          p[b][y][j] = (_Float16)e;
          if constexpr (TWO) rest[b][y][j] = (_Float16)(e - (float)p[b][y][j]);
        }
        x.l = __builtin_fmaf(sum[0] + sum[1], __builtin_amdgcn_exp2f(-(base[b] + m0)), x.l);
      }
#pragma unroll
      for (int b = 0; b < 2; ++b)
#pragma unroll
        for (int y = 0; y < 2; ++y)
#pragma unroll
          for (int d = 0; d < NI; ++d) {
            const h8 codes = *reinterpret_cast<const h8*>(v + b * L::BLOCK + d * 2048 + y * 1024);
            x.o[d] = __builtin_amdgcn_mfma_f32_32x32x16_f16(codes, p[b][y], x.o[d], 0, 0, 0);
            if constexpr (TWO) x.o[d] = __builtin_amdgcn_mfma_f32_32x32x16_f16(codes, rest[b][y], x.o[d], 0, 0, 0);
          }
    }
    if (stage + 1 < stop) {
      place ^= 1;
      make(place);
      if (stage + 2 < stop) fetch(stage + 2);
      __syncthreads();
    }
  }
  const float l = x.sum();
  x.each([&](int d, const f4& o) {
    if (!valid) return;
    if (!part) {
      put_out(a, row, hq, d, o, x.m, l);
    } else {
      *reinterpret_cast<f4*>(part + 2 * TILE + in * (NI * 32) + d) = o;
      if (d == 0) part[in * 2] = x.m, part[in * 2 + 1] = l;
    }
  });
}

// SHARED: equal shares of all stages.  Else a workgroup a tile: of sequences in the order of their starts, tiles' slots from
// starts[s] G / 128 + s on; neighbouring workgroups, which go to neighbouring XCDs, take different key heads, so that a head's pages are in one XCD's
// cache; last tiles, which see most, first.  FEW: the first workgroups deal with the sequences of few rows.
template <typename Code, int NI, bool SHARED, bool FEW>
__global__ __launch_bounds__(256, 2) void attend_tiles_kernel(const AttendArgs a) {
  constexpr int FLOATS = Meeting<NI, 16>::FLOATS, BYTES = 2 * Staged<NI>::BYTES;
  __shared__ __attribute__((aligned(16))) char shared[FEW && FLOATS * 4 > BYTES ? FLOATS * 4 : BYTES];
  __shared__ int numbers[SHARED || FEW ? 4 : 1][3][64];
  int w = blockIdx.x;
  if constexpr (FEW) {
    if (w < a.few.workgroups) {
      run_share<Code, NI, 16>(a, w, reinterpret_cast<float*>(shared), numbers[threadIdx.x >> 6]);
      return;
    }
    w -= a.few.workgroups;
  }
  if constexpr (SHARED) {
    walk_share<TILE>(a, a.many, w, numbers[threadIdx.x >> 6], [&](const Work& work, int s, int head, int tile, int begin, int stop, bool whole, bool again) {
      float* const part = whole ? nullptr : part_at(a.many, w, begin, part_floats(TILE, NI * 32));
      if (work.rows <= EXACT_ROWS) run_tile<Code, NI, true>(a, work, s, head, tile, begin, stop, part, shared, again);
      else run_tile<Code, NI, false>(a, work, s, head, tile, begin, stop, part, shared, again);
    });
  } else {
    const int head = w % a.pages.Hkv, slot = a.many.tiles - 1 - w / a.pages.Hkv;
    auto from = [&](int i) { return (int64_t)a.batch.start(i) * a.G / TILE + i; };
    const int s = count_up_to(a.batch.S, from, slot);
    if (s >= a.batch.S) return;
    const int tile = slot - (int)from(s);
    const Work work = Work::of<TILE>(a, a.many, Sequence(a.batch, s));
    if (tile < 0 || tile >= work.tiles) return;  // (below 0: starts that fall, or do not begin at zero)
    if (work.rows <= EXACT_ROWS) run_tile<Code, NI, true>(a, work, s, head, tile, 0, work.blocks, nullptr, shared, false);
    else run_tile<Code, NI, false>(a, work, s, head, tile, 0, work.blocks, nullptr, shared, false);
  }
}

// --- joining ----------------------------------------------------------------------------------------------------------------------------------
//
// A segment that several workgroups met is joined by the workgroups of its first border: border w lies between shares w - 1 and w.  A thread has four
// elements of up to four rows, all of whose parts, or some of them at a time, are on their way at once.
constexpr int JOINING = 256;
template <int NI, int ROWS>
struct Joining {
  static constexpr int T = NI * 8, AT_ONCE = JOINING / T, MINE = (ROWS + AT_ONCE - 1) / AT_ONCE < 4 ? (ROWS + AT_ONCE - 1) / AT_ONCE : 4;
  static constexpr int GROUPS = (ROWS + AT_ONCE * MINE - 1) / (AT_ONCE * MINE);  // workgroups of a border
};
template <int NI, int ROWS>
__device__ __forceinline__ void join(const AttendArgs& a, const AttendArgs::Side& side, int border, int group) {
  typedef Joining<NI, ROWS> J;
  constexpr int W = NI * 32, T = J::T, AT_ONCE = J::AT_ONCE, MINE = J::MINE, PARTS = 8 / MINE;
  const Note note = side.notes[border];
  const int w0 = note.w0, w1 = note.w1;
  if (w1 <= w0) return;
  const int d = (int)threadIdx.x % T * 4, first = group * AT_ONCE * MINE + (int)threadIdx.x / T, rows = min(ROWS, note.rows - note.tile_row);
  if ((int)threadIdx.x >= AT_ONCE * T || first >= rows) return;
  float m[MINE], l[MINE];
  f4 sum[MINE];
#pragma unroll
  for (int y = 0; y < MINE; ++y) m[y] = -INFINITY, l[y] = 0.0f, sum[y] = (f4)(0.0f);
  for (int w = w0; w <= w1; w += PARTS) {
    f2 ml[MINE][PARTS];
    f4 o[MINE][PARTS];
#pragma unroll
    for (int x = 0; x < PARTS; ++x) {
      const float* p = part_at(side, min(w + x, w1), w + x == w0 ? 0 : 1, part_floats(ROWS, W));
#pragma unroll
      for (int y = 0; y < MINE; ++y) {
        const int in = min(first + y * AT_ONCE, rows - 1);
        ml[y][x] = *reinterpret_cast<const f2*>(p + in * 2);
        o[y][x] = *reinterpret_cast<const f4*>(p + 2 * ROWS + in * W + d);
      }
    }
#pragma unroll
    for (int y = 0; y < MINE; ++y) {
      float top = m[y];
#pragma unroll
      for (int x = 0; x < PARTS; ++x) top = fmaxf(top, w + x <= w1 ? ml[y][x][0] : -INFINITY);
      const int by = places(m[y], top);
      l[y] = __builtin_ldexpf(l[y], by), sum[y] *= __builtin_ldexpf(1.0f, by), m[y] = top;
#pragma unroll
      for (int x = 0; x < PARTS; ++x) {
        if (w + x > w1) continue;
        const int by = places(ml[y][x][0], top);
        l[y] += __builtin_ldexpf(ml[y][x][1], by);
        sum[y] += o[y][x] * __builtin_ldexpf(1.0f, by);
      }
    }
  }
#pragma unroll
  for (int y = 0; y < MINE; ++y) {
    const int in = first + y * AT_ONCE, r = note.tile_row + in, i = r / a.G;
    if (in < rows) put_out(a, note.row0 + i, note.head * a.G + r - i * a.G, d, sum[y], m[y], l[y]);
  }
}
template <int NI>
__global__ __launch_bounds__(JOINING) void join_kernel(const AttendArgs a, int few_rows, int few_borders) {
  int w = blockIdx.x;
  constexpr int G16 = Joining<NI, 16>::GROUPS, G32 = Joining<NI, 32>::GROUPS, G128 = Joining<NI, TILE>::GROUPS;
  const int few = few_borders * (few_rows == 16 ? G16 : G32);
  if (w >= few) join<NI, TILE>(a, a.many, (w - few) / G128 + 1, (w - few) % G128);
  else if (few_rows == 16) join<NI, 16>(a, a.few, w / G16 + 1, w % G16);
  else join<NI, 32>(a, a.few, w / G32 + 1, w % G32);
}
template <int NI>
static int64_t join_groups(int few_rows, int few_borders, int many_borders) {
  return (int64_t)few_borders * (few_rows == 16 ? Joining<NI, 16>::GROUPS : Joining<NI, 32>::GROUPS) + (int64_t)many_borders * Joining<NI, TILE>::GROUPS;
}

// --- host ----------------------------------------------------------------------------------------------------------------------------------

static bool desc_ok(const tmac_attn_desc* d, const tmac_pages* p) {
  return d && d->Hq > 0 && d->Hkv == p->Hkv && d->Hq % d->Hkv == 0 && d->D == p->D && (d->elem == TMAC_ELEM_F16 || d->elem == TMAC_ELEM_BF16) &&
         std::isfinite(d->scale) && d->scale > 0 && d->causal == 1 && !d->reserved[0] && !d->reserved[1];
}

// How the sequences of few and of many rows are dealt with.
struct Side {
  bool on, whole;  // whole: every segment by a workgroup of its own, nothing to join
  int rows, workgroups, least, spare, tiles, rows_from, rows_to;
  size_t notes, parts;  // bytes
  size_t bytes() const { return notes + parts; }
  void share(const tmac_pages* p) {
    notes = (size_t)workgroups * sizeof(Note);
    parts = (size_t)workgroups * 2 * part_floats(rows, (p->D + 31) / 32 * 32) * 4;
  }
  AttendArgs::Side args(char* workspace) const {
    return {rows_from, rows_to, workgroups, least, spare, tiles, reinterpret_cast<Note*>(workspace), reinterpret_cast<float*>(workspace + notes)};
  }
};
struct Plan {
  Side few, many;
};
// By the rows that a sequence and key head may have at most, the blocks that its table has room for, and the number of segments; what lengths there are is not
// known here (one sequence of 300 tokens and 32 key heads: 6 where the table has room for 1536 tokens, in shares 10 to 11 where it has more).  (us of one launch and its joining one.)
static Plan plan_of(const tmac_attn_desc* d, const tmac_pages* p, const tmac_pages_batch* b) {
  Plan plan = {};
  Side &few = plan.few, &many = plan.many;
  const int G = d->Hq / d->Hkv;
  const int64_t most = (int64_t)view_of(b).most * G;
  const int64_t blocks = (int64_t)b->width * p->page / BT, heads = (int64_t)b->S * p->Hkv;
  // Up to 64 rows in tiles of 32, which read a block twice, but have no wavefronts without rows: 40 rows of 32 sequences of up to 16384 tokens 107, in tiles of 128 rows 119; 64 rows 126
  // and 121; 64 rows of 16 sequences of 4200 tokens 56 and 79; of one of 7000 26 and 35.
  many.on = most > EXACT_ROWS;
  few.on = !many.on || (b->S > 1 && G <= 16);
  if (few.on) {
    few.rows = most > 16 && !many.on ? 32 : 16;
    few.rows_from = 1, few.rows_to = few.rows == 32 ? EXACT_ROWS : 16;
    few.tiles = few.rows == 32 ? (int)((most + 31) / 32) : 1;
    const int64_t segments = heads * few.tiles;
    // A workgroup a segment, without a joining launch, while that is not much longer than the others' share: 32 segments of 1000 tokens 8.3 against 12.5 in
    // shares, of 2000 tokens 18 against 14; 256 segments of 2000 tokens 24 against 37.
    few.whole = !many.on && blocks <= (segments < 256 ? 48 : 128) && segments * 256 <= 0xffffffff;
    if (few.whole) {
      few.workgroups = (int)segments;
    } else {
      // Shares: four wavefronts a CU with two blocks each on their way read 6.7 TB/s; twice as many gain nothing and leave twice as many pieces (32 sequences
      // of 128 to 16384 tokens 49 with 256 workgroups, 53 with 512, 62 with 768).  A segment costs as much as 16 blocks (none counted: 83, 8: 59, 16: 49).
      few.workgroups = 256, few.least = 8, few.spare = 16;
      few.share(p);
    }
  }
  if (many.on) {
    many.rows = TILE;
    many.rows_from = few.on ? 17 : 1, many.rows_to = 0x7fffffff;
    const int64_t slots = (int64_t)b->T * G / TILE + b->S, least = std::max<int64_t>(0, ((int64_t)b->T * G - (few.on ? 16 * (int64_t)b->S : 0)) / TILE) * p->Hkv;
    // A workgroup a tile where there are nearly two a CU, or few stages; else shares of all stages (344 tiles of up to 40 stages: 66 in shares, 76 whole;
    // 512 of 120: 371 and 319).
    many.whole = (least >= 448 || blocks <= 32) && (slots * p->Hkv + 1024) * 256 <= 0xffffffff;
    many.tiles = (int)slots;
    many.workgroups = many.whole ? (int)(slots * p->Hkv) : 512;
    if (!many.whole) {
      many.least = 4, many.spare = 2;
      many.share(p);
    }
  }
  return plan;
}

template <typename Code, int NI>
static const void* attend_of(const Plan& x) {
  if (x.many.on) {
    if (x.many.whole) return x.few.on ? (const void*)attend_tiles_kernel<Code, NI, false, true> : (const void*)attend_tiles_kernel<Code, NI, false, false>;
    return x.few.on ? (const void*)attend_tiles_kernel<Code, NI, true, true> : (const void*)attend_tiles_kernel<Code, NI, true, false>;
  }
  if (x.few.whole) {
    if (x.few.rows == 32) return (const void*)attend_whole_kernel<Code, NI, 32>;
    return (const void*)attend_whole_kernel<Code, NI, 16>;
  }
  return x.few.rows == 16 ? (const void*)attend_kernel<Code, NI, 16> : (const void*)attend_kernel<Code, NI, 32>;
}
template <typename Code>
static const void* attend_of(int ni, const Plan& x) {
  return ni == 1 ? attend_of<Code, 1>(x) : ni == 2 ? attend_of<Code, 2>(x) : ni == 3 ? attend_of<Code, 3>(x) : attend_of<Code, 4>(x);
}

}  // namespace pages
}  // namespace tmac

using namespace tmac;
using namespace tmac::pages;

extern "C" size_t tmac_pages_attend_workspace_bytes(const tmac_attn_desc* desc, const tmac_pages* p, const tmac_pages_batch* batch) {
  if (!pages_ok(p) || !batch_ok(batch) || !desc_ok(desc, p) || !supported(p, batch)) return 0;
  const Plan plan = plan_of(desc, p, batch);
  return plan.few.bytes() + plan.many.bytes();
}

extern "C" tmac_status tmac_pages_attend(const tmac_attn_desc* desc, const tmac_pages* p, const tmac_pages_batch* batch, const tmac_view* q,
                                         const tmac_view* out, float* lse_dev, void* workspace_dev, size_t workspace_bytes, void* stream) {
  if (!pages_ok(p) || !batch_ok(batch) || !desc_ok(desc, p)) return TMAC_EINVAL;
  if (batch->S == 0 || batch->T == 0) return TMAC_OK;
  if (!pages_set(p) || !batch_set(batch) || !attn::rows_ok(q, false, true, true) || !attn::rows_ok(out, false, true, true)) return TMAC_EINVAL;
  if (!supported(p, batch) || (int64_t)batch->T * desc->Hq > (1 << 30)) return TMAC_EUNSUPPORTED;
  const Plan plan = plan_of(desc, p, batch);
  const size_t need = plan.few.bytes() + plan.many.bytes();
  if (need && (!workspace_dev || (reinterpret_cast<uintptr_t>(workspace_dev) & 15))) return TMAC_EINVAL;
  if (workspace_bytes < need) return TMAC_ESIZE;
  AttendArgs a = {};
  a.pages = view_of(p), a.batch = view_of(batch);
  a.q = static_cast<const char*>(q->data), a.out = static_cast<char*>(out->data);
  a.q_token = q->token * 2, a.q_head = q->head * 2, a.out_token = out->token * 2, a.out_head = out->head * 2;
  a.lse = lse_dev;
  a.c = desc->scale * 1.44269504088896340736f;
  a.G = desc->Hq / desc->Hkv, a.bf16 = desc->elem == TMAC_ELEM_BF16;
  char* const workspace = static_cast<char*>(workspace_dev);
  a.few = plan.few.args(workspace), a.many = plan.many.args(workspace + plan.few.bytes());
  const int ni = (p->D + 31) / 32, workgroups = (plan.few.on ? plan.few.workgroups : 0) + (plan.many.on ? plan.many.workgroups : 0);
  const tmac_status st = launch(p->code == TMAC_CODE_I8 ? attend_of<I8>(ni, plan) : attend_of<E4M3>(ni, plan), workgroups, 64 * WAVES, &a, stream);
  if (st != TMAC_OK || need == 0) return st;
  int few_rows = plan.few.rows, few_borders = plan.few.on && !plan.few.whole ? plan.few.workgroups - 1 : 0;
  const int many_borders = plan.many.on && !plan.many.whole ? plan.many.workgroups - 1 : 0;
  const void* join = ni == 1 ? (const void*)join_kernel<1> : ni == 2 ? (const void*)join_kernel<2> : ni == 3 ? (const void*)join_kernel<3> : (const void*)join_kernel<4>;
  void* args[] = {&a, &few_rows, &few_borders};
  const int64_t groups = ni == 1 ? join_groups<1>(few_rows, few_borders, many_borders) : ni == 2 ? join_groups<2>(few_rows, few_borders, many_borders)
                       : ni == 3 ? join_groups<3>(few_rows, few_borders, many_borders) : join_groups<4>(few_rows, few_borders, many_borders);
  return launch_with(join, groups, JOINING, args, stream);
}
