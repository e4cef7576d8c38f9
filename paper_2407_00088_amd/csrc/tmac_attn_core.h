// Device core of the attention kernels: one workgroup of four wavefronts takes up to 128 query rows over a run of keys.
//
// For a row i: s_ij = scale q_i . k_j, running maximum m and sum l of exp(s - m), O_i = sum_j exp(s_ij - m) v_j, rescaled
// when the maximum has grown.  Products run on v_mfma_f32_32x32x16 in transposed form, S^T = K Q^T and O^T = V^T P^T, so
// that a lane owns one query row (lane & 31) and its scores sit in its own registers: maximum and sum need one exchange
// between the wavefront's halves, and the exponentials, rounded to the inputs' type, are the second product's operand as
// they stand.  (That operand's k order is then 0-3, 8-11 in the lower half and 4-7, 12-15 in the upper; the transposed
// reads of V, ds_read_b64_tr_b16, take the same order.)
#ifndef TMAC_ATTN_CORE_H_
#define TMAC_ATTN_CORE_H_

#include <hip/hip_runtime.h>

#include <cstdint>

namespace tmac {
namespace attn {

typedef _Float16 h2 __attribute__((ext_vector_type(2)));
typedef _Float16 h4 __attribute__((ext_vector_type(4)));
typedef _Float16 h8 __attribute__((ext_vector_type(8)));
typedef __bf16 b2 __attribute__((ext_vector_type(2)));
typedef __bf16 b4 __attribute__((ext_vector_type(4)));
typedef __bf16 b8 __attribute__((ext_vector_type(8)));
typedef float f2 __attribute__((ext_vector_type(2)));
typedef float f4 __attribute__((ext_vector_type(4)));
typedef float f8 __attribute__((ext_vector_type(8)));
typedef float f16x __attribute__((ext_vector_type(16)));
typedef short s4 __attribute__((ext_vector_type(4)));
typedef uint32_t u2 __attribute__((ext_vector_type(2)));
typedef uint32_t u4 __attribute__((ext_vector_type(4)));

#define TMAC_LDS __attribute__((address_space(3)))

struct F16 {
  typedef _Float16 elem;
  typedef h4 v4;
  typedef h8 v8;
  static constexpr uint32_t EXP = 0x7C00u, NEG_INF = 0xFC00u, POS_INF = 0x7C00u, ONE = 0x3C00u;
  static __device__ __forceinline__ f16x mfma(v8 a, v8 b, f16x c) { return __builtin_amdgcn_mfma_f32_32x32x16_f16(a, b, c, 0, 0, 0); }
};
struct BF16 {
  typedef __bf16 elem;
  typedef b4 v4;
  typedef b8 v8;
  static constexpr uint32_t EXP = 0x7F80u, NEG_INF = 0xFF80u, POS_INF = 0x7F80u, ONE = 0x3F80u;
  static __device__ __forceinline__ f16x mfma(v8 a, v8 b, f16x c) { return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0); }
};

// Larger of the two halves' values for the same row, in both.
__device__ __forceinline__ float max_halves(float x) {
  const auto r = __builtin_amdgcn_permlane32_swap(__builtin_bit_cast(unsigned, x), __builtin_bit_cast(unsigned, x), false, false);
  return fmaxf(__builtin_bit_cast(float, (unsigned)r[0]), __builtin_bit_cast(float, (unsigned)r[1]));
}
__device__ __forceinline__ float add_halves(float x) {
  const auto r = __builtin_amdgcn_permlane32_swap(__builtin_bit_cast(unsigned, x), __builtin_bit_cast(unsigned, x), false, false);
  return __builtin_bit_cast(float, (unsigned)r[0]) + __builtin_bit_cast(float, (unsigned)r[1]);
}

// Tiles of 16-bit rows of DP elements in LDS, unpadded, their 16-byte chunks permuted by the row so that a wavefront's
// reads meet all banks: K tiles are read 16 bytes of 32 rows at a time, V tiles 64 bytes of four rows.
template <int DP>
__device__ __forceinline__ int k_swizzle(int row) {
  return DP == 128 ? row & 15 : (row >> 1) & 7;
}
template <int DP>
__device__ __forceinline__ int v_swizzle(int row) {
  return DP == 128 ? (row & 3) << 2 : ((row >> 1) & 1) << 2;
}

// What a workgroup reads: keys [begin, end) of one sequence and key head.
struct Keys {
  const char* k;       // row 0 of the sequence and head
  const char* v;
  int64_t k_stride, v_stride;  // bytes from row to row
  int begin, end;      // the unit's keys; begin a multiple of the stage from the sequence's start or not, as the caller likes
};

// One stage of ROWS rows, straight into LDS: 1024 bytes an instruction, lane after lane.  Rows from `rows` on and columns
// from D on read as zeros (the descriptor's range).
template <int DP, int ROWS, bool IS_V>
__device__ __forceinline__ void stage_dma(const char* base, int64_t stride, int rows, int D, char* lds, int wave, int lane) {
  constexpr int CH = DP / 8, RPI = 64 / CH;
  const int row = wave * RPI + lane / CH;
  const int phys = lane % CH;
  const int chunk = phys ^ (IS_V ? v_swizzle<DP>(row) : k_swizzle<DP>(row));
  const int n = rows < ROWS ? rows : ROWS;
  const uint32_t range = n > 0 ? (uint32_t)((n - 1) * (int)stride + D * 2) : 0u;
  const auto rsrc = __builtin_amdgcn_make_buffer_rsrc((void*)base, (short)0, (int)range, 0x00020000);
  const uint32_t voff = chunk * 8 < D ? row * (uint32_t)stride + chunk * 16 : 0x7ffffff0u;
#pragma unroll
  for (int i = 0; i < ROWS / (4 * RPI); ++i)
    // (rows go into the offset that the range is checked against; far_rows keeps it below 2^32)
    __builtin_amdgcn_raw_ptr_buffer_load_lds(rsrc, (TMAC_LDS void*)(lds + (i * 4 + wave) * 1024), 16,
                                             voff + (uint32_t)(i * 4 * RPI) * (uint32_t)stride, 0, 0, 0);
}

// The same through registers, 8 bytes at a time, for rows that are not 16-byte aligned or whose length is no multiple of 8.
template <int DP, int ROWS, bool IS_V>
__device__ __forceinline__ void stage_copy(const char* base, int64_t stride, int rows, int D, char* lds, int tid) {
  constexpr int CH = DP / 4, N = ROWS * CH / 256;
#pragma unroll 8
  for (int i = 0; i < N; ++i) {
    const int at = i * 256 + tid, row = at / CH, c8 = at % CH;
    u2 x = {0u, 0u};
    if (row < rows && c8 * 4 < D) x = *reinterpret_cast<const u2*>(base + row * stride + c8 * 8);
    const int phys = (c8 >> 1) ^ (IS_V ? v_swizzle<DP>(row) : k_swizzle<DP>(row));
    *reinterpret_cast<u2*>(lds + row * DP * 2 + phys * 16 + (c8 & 1) * 8) = x;
  }
}

// Shape of a workgroup: RW wavefronts side by side over the rows, 32 each, 4 / RW over the keys of a stage.
template <int DP, bool DMA, int RW>
struct Shape {
  static constexpr int KW = 4 / RW, KT = RW == 4 ? 64 : 32, SK = KW * KT;
  static constexpr int TILE = SK * DP * 2, STAGE = 2 * TILE;
  // two stages where they leave room for two workgroups on a CU
  static constexpr int STAGES = DMA && 2 * STAGE <= 65536 ? 2 : 1;
  static constexpr int MERGE = KW > 1 ? 4 * 32 * (DP + 4) * 4 + 4 * 32 * 8 : 0;
  static constexpr int LDS = STAGES * STAGE > MERGE ? STAGES * STAGE : MERGE;
};

// The running softmax and sums of one wavefront's 32 rows.
template <typename T, int DP>
struct Rows {
  typename T::v8 q[DP / 16];
  f16x o[DP / 32];
  float m, l;      // largest score that the sums are taken against (as the product gives it), sum of this half's exponentials
};

// NaN and infinities of V in places that some row's mask hides: the tile's finite values have been multiplied; adds the
// others for the rows that see them.  c1 counts +inf or NaN, c2 -inf or NaN: NaN comes out as inf - inf.
template <typename T, int DP, int KT>
__device__ __forceinline__ typename T::v8 v_fragment(const char* const (&vaddr)[DP / 32], int dblk, int u) {
  const s4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((TMAC_LDS s4*)(vaddr[dblk] + (16 * u) * DP * 2));
  const s4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((TMAC_LDS s4*)(vaddr[dblk] + (16 * u + 8) * DP * 2));
  return __builtin_bit_cast(typename T::v8, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
}

// One tile of KT keys for one wavefront.  x: how many of the tile's keys, counted from its first key, the lane's row may see,
// less four in the upper half (only read where MASK).  hidden: some of those it may not see are there all the same.
template <typename T, int DP, int KT>
__device__ __forceinline__ void tile_step(Rows<T, DP>& w, const char* ktile, const char* vtile, float c, bool mask, bool hidden, int x,
                                          int lane, float* scores) {
  constexpr int NT = DP / 16, ND = DP / 32, NB = KT / 32;
  const int half = lane >> 5;
  f16x s[NB];
#pragma unroll
  for (int b = 0; b < NB; ++b) {
    s[b] = (f16x)(0.0f);
    const char* row = ktile + (b * 32 + (lane & 31)) * DP * 2;
#pragma unroll
    for (int t = 0; t < NT; ++t) {
      const auto a = *reinterpret_cast<const typename T::v8*>(row + ((2 * t + half) ^ k_swizzle<DP>(lane & 31)) * 16);
      s[b] = T::mfma(a, w.q[t], s[b]);
    }
  }
  if (scores) {
    // a decode step keeps its scores: the weights need the whole row's sum
#pragma unroll
    for (int b = 0; b < NB; ++b)
#pragma unroll
      for (int r = 0; r < 4; ++r)
        *reinterpret_cast<f4*>(scores + b * 32 + r * 8 + half * 4) = f4{s[b][4 * r], s[b][4 * r + 1], s[b][4 * r + 2], s[b][4 * r + 3]};
  }
  if (mask) {
#pragma unroll
    for (int b = 0; b < NB; ++b)
#pragma unroll
      for (int r = 0; r < 16; ++r) s[b][r] = b * 32 + (r >> 2) * 8 + (r & 3) < x ? s[b][r] : -INFINITY;
  }
  float mx = s[0][0];
#pragma unroll
  for (int b = 0; b < NB; ++b)
#pragma unroll
    for (int r = 0; r < 16; ++r) mx = fmaxf(mx, s[b][r]);
  mx = max_halves(mx);
  // The sums keep the maximum they have until a row's is 2^8 times larger: exponentials up to 256 are as exact in 16
  // bits, and most tiles then need no rescaling.  (Row by row: a row's bits do not depend on its neighbours.)
  const bool grows = mx * c > w.m * c + 8.0f;
  if (__any(grows)) {
    const float m = grows ? mx : w.m;
    const float alpha = grows ? __builtin_amdgcn_exp2f((w.m - m) * c) : 1.0f;
#pragma unroll
    for (int d = 0; d < ND; ++d) w.o[d] *= alpha;
    w.l *= alpha;
    w.m = m;
  }
  const float mc = w.m == -INFINITY ? 0.0f : w.m * c;
  typename T::v8 p[KT / 16];
  float sum = 0.0f;
#pragma unroll
  for (int b = 0; b < NB; ++b) {
    f16x e;
#pragma unroll
    for (int r = 0; r < 16; ++r) {
      e[r] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[b][r], c, -mc));
      sum += e[r];
    }
    p[2 * b] = __builtin_convertvector(__builtin_shufflevector(e, e, 0, 1, 2, 3, 4, 5, 6, 7), typename T::v8);
    p[2 * b + 1] = __builtin_convertvector(__builtin_shufflevector(e, e, 8, 9, 10, 11, 12, 13, 14, 15), typename T::v8);
  }
  w.l += sum;
  // V^T: lane i of sixteen takes row i / 4, columns 4 (i % 4) .. +3 and gets column i, rows 0..3
  const int i16 = lane & 15, key = 4 * half + (i16 >> 2);
  const char* vaddr[ND];
#pragma unroll
  for (int d = 0; d < ND; ++d) {
    const int chunk = (d * 4 + 2 * ((lane >> 4) & 1) + ((i16 & 3) >> 1)) ^ v_swizzle<DP>(i16 >> 2);
    vaddr[d] = vtile + key * DP * 2 + chunk * 16 + (i16 & 1) * 8;
  }
  bool odd = false;
  if (hidden) {
    // (rare: the diagonal's tiles; rarer still that there is anything to find)
    bool found = false;
#pragma unroll 4
    for (int i = 0; i < KT * DP * 2 / 1024; ++i) {
      const u4 q = *reinterpret_cast<const u4*>(vtile + (i * 64 + lane) * 16);
#pragma unroll
      for (int j = 0; j < 4; ++j) found |= (q[j] & T::EXP) == T::EXP || (q[j] & (T::EXP << 16)) == (T::EXP << 16);
    }
    odd = __any(found);
  }
  if (!odd) {
#pragma unroll
    for (int u = 0; u < KT / 16; ++u)
#pragma unroll
      for (int d = 0; d < ND; ++d) w.o[d] = T::mfma(v_fragment<T, DP, KT>(vaddr, d, u), p[u], w.o[d]);
    return;
  }
#pragma unroll 1
  for (int u = 0; u < KT / 16; ++u) {
    // which of the sixteen keys the lane's row sees, as ones and zeros
    uint32_t see[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int k0 = 16 * u + (j >> 1) * 8 + (j & 1) * 2;
      see[j] = (k0 < x ? T::ONE : 0u) | (k0 + 1 < x ? T::ONE << 16 : 0u);
    }
    const auto sees = __builtin_bit_cast(typename T::v8, u4{see[0], see[1], see[2], see[3]});
    typename T::v8 pu = p[0];
#pragma unroll
    for (int j = 1; j < KT / 16; ++j)
      if (u == j) pu = p[j];
#pragma unroll
    for (int d = 0; d < ND; ++d) {
      const u4 a = __builtin_bit_cast(u4, v_fragment<T, DP, KT>(vaddr, d, u));
      u4 fin, up, down;
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        uint32_t f = 0, p1 = 0, p2 = 0;
#pragma unroll
        for (int y = 0; y < 32; y += 16) {
          const uint32_t e = (a[j] >> y) & 0xffffu;
          const bool finite = (e & T::EXP) != T::EXP;
          f |= finite ? e << y : 0u;
          p1 |= !finite && e != T::NEG_INF ? T::ONE << y : 0u;
          p2 |= !finite && e != T::POS_INF ? T::ONE << y : 0u;
        }
        fin[j] = f, up[j] = p1, down[j] = p2;
      }
      w.o[d] = T::mfma(__builtin_bit_cast(typename T::v8, fin), pu, w.o[d]);
      const f16x n1 = T::mfma(__builtin_bit_cast(typename T::v8, up), sees, (f16x)(0.0f));
      const f16x n2 = T::mfma(__builtin_bit_cast(typename T::v8, down), sees, (f16x)(0.0f));
#pragma unroll
      for (int r = 0; r < 16; ++r) w.o[d][r] += (n1[r] > 0.0f ? INFINITY : 0.0f) + (n2[r] > 0.0f ? -INFINITY : 0.0f);
    }
  }
}

// Whether a wavefront's loads into LDS have landed, then the workgroup's.
__device__ __forceinline__ void wait_stage() { asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory"); }

// All keys of a unit for the workgroup's rows.  lim: keys that the lane's row sees, counted from the sequence's start (its
// own, and the least and the most of the wavefront); scores: where the lane's row keeps its scores (index 0 = keys.begin), or null.
template <typename T, int DP, bool DMA, int RW>
__device__ __forceinline__ void run_keys(Rows<T, DP>& w, const Keys& keys, int D, float c, int lim, int lim_least, int lim_most, char* lds,
                                         float* scores) {
  typedef Shape<DP, DMA, RW> Sh;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int kw = wave / RW;  // which part of a stage's keys
#pragma unroll
  for (int d = 0; d < DP / 32; ++d) w.o[d] = (f16x)(0.0f);
  w.m = -INFINITY;
  w.l = 0.0f;
  if (keys.begin >= keys.end) return;
  auto load = [&](int at, char* to) {
    const char* kb = keys.k + (int64_t)at * keys.k_stride;
    const char* vb = keys.v + (int64_t)at * keys.v_stride;
    if constexpr (DMA) {
      stage_dma<DP, Sh::SK, false>(kb, keys.k_stride, keys.end - at, D, to, wave, lane);
      stage_dma<DP, Sh::SK, true>(vb, keys.v_stride, keys.end - at, D, to + Sh::TILE, wave, lane);
    } else {
      stage_copy<DP, Sh::SK, false>(kb, keys.k_stride, keys.end - at, D, to, tid);
      stage_copy<DP, Sh::SK, true>(vb, keys.v_stride, keys.end - at, D, to + Sh::TILE, tid);
    }
  };
  auto compute = [&](int at, const char* from) {
    const int first = at + kw * Sh::KT;  // the wavefront's first key
    if (first >= lim_most) return;
    const bool mask = lim_least < first + Sh::KT;
    const int there = keys.end < first + Sh::KT ? keys.end : first + Sh::KT;
    tile_step<T, DP, Sh::KT>(w, from + kw * Sh::KT * DP * 2, from + Sh::TILE + kw * Sh::KT * DP * 2, c, mask, lim_least < there,
                             lim - first - 4 * (lane >> 5), lane, scores ? scores + (first - keys.begin) : nullptr);
  };
  if constexpr (Sh::STAGES == 2) {
    load(keys.begin, lds);
    int at = keys.begin;
    while (true) {
      wait_stage();
      if (at + Sh::SK < keys.end) load(at + Sh::SK, lds + Sh::STAGE);
      compute(at, lds);
      at += Sh::SK;
      if (at >= keys.end) break;
      wait_stage();
      if (at + Sh::SK < keys.end) load(at + Sh::SK, lds);
      compute(at, lds + Sh::STAGE);
      at += Sh::SK;
      if (at >= keys.end) break;
    }
  } else {
    for (int at = keys.begin; at < keys.end; at += Sh::SK) {
      if (at != keys.begin) __syncthreads();
      load(at, lds);
      wait_stage();
      compute(at, lds);
    }
  }
}

}  // namespace attn
}  // namespace tmac
#endif
