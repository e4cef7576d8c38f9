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

// LDS by its address there.
template <typename X>
__device__ __forceinline__ TMAC_LDS X* in_lds(uint32_t at) {
  return (TMAC_LDS X*)(uintptr_t)at;
}

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
  const char* k;               // row 0 of the sequence and head
  const char* v;
  int64_t k_stride, v_stride;  // bytes from row to row
  int begin, end;
};

// Rows of 16-bit elements on their way from memory to LDS: 1024 bytes a load of one wavefront, lane after lane, without passing
// through registers.  Memory need only be 8-byte aligned.  Chunks of 16 bytes that lie within the row's D elements are loaded;
// a half chunk at the row's end (D % 8 == 4) comes with its neighbour's elements, which is fine for V, whose columns from D on give
// results that nobody reads, but not for K, where they would meet the products' sums: there the half chunk goes through a
// register (load_tail, store_tail).  Chunks beyond are cleared once (clear_pads).
//
// The load is written out: of the builtin the compiler knows only that it writes LDS, and makes every transposed read wait
// for it, although that is another stage.  It has no result register; wait_stage waits for it.
__device__ __forceinline__ void load_to_lds(u4 rsrc, uint32_t lds, uint32_t offset, uint32_t scalar_offset) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, %3 offen lds"
               :
               : "s"(lds), "v"(offset), "s"(rsrc), "s"(scalar_offset)
               : "memory");
}
__device__ __forceinline__ u4 buffer_of(const char* base, int range) {
  const uint64_t at = (uint64_t)base;
  return u4{(uint32_t)at, (uint32_t)(at >> 32) & 0xffffu, (uint32_t)range, 0x00020000u};
}
template <int DP, int ROWS, bool IS_V>
struct Stage {
  static constexpr int CH = DP / 8, RPI = 64 / CH, N = ROWS / (4 * RPI);
  uint32_t offset;  // of the lane's chunk in the wavefront's first load
  bool wanted;

  __device__ __forceinline__ Stage(int64_t stride, int D, int wave, int lane) {
    // (a lane's row modulo the swizzle's period is the same in all its loads)
    const int row = wave * RPI + lane / CH, chunk = (lane % CH) ^ (IS_V ? v_swizzle<DP>(row) : k_swizzle<DP>(row));
    offset = row * (uint32_t)stride + chunk * 16;
    wanted = IS_V ? chunk * 8 < D : chunk * 8 + 8 <= D;
  }
  // Rows from `rows` on read as zeros: the descriptor's range ends there.  (What a scalar register adds to the address is not
  // checked against the range, so it is used for whole stages only.)
  __device__ __forceinline__ void load(const char* base, int64_t stride, int rows, int D, uint32_t lds, int wave) const {
    const int step = 4 * RPI * (int)stride;
    if (!wanted) return;
    if (rows >= ROWS) {
      const u4 rsrc = buffer_of(base, (ROWS - 1) * (int)stride + D * 2);
#pragma unroll
      for (int i = 0; i < N; ++i) load_to_lds(rsrc, lds + (i * 4 + wave) * 1024, offset, i * step);
    } else {
      const int range = rows > 0 ? (rows - 1) * (int)stride + D * 2 : 0;
#pragma unroll
      for (int i = 0; i < N; ++i)
        load_to_lds(buffer_of(base + i * (int64_t)step, max(0, range - i * step)), lds + (i * 4 + wave) * 1024, offset, 0);
    }
  }
};
template <int ROWS>
__device__ __forceinline__ u2 load_tail(const char* base, int64_t stride, int rows, int D, int tid) {
  u2 x = {0u, 0u};
  if (D % 8 && tid < ROWS && tid < rows) x = *reinterpret_cast<const u2*>(base + tid * stride + (D - 4) * 2);
  return x;
}
template <int DP, int ROWS>
__device__ __forceinline__ void store_tail(u2 x, int D, uint32_t lds, int tid) {
  if (D % 8 && tid < ROWS)
    *in_lds<u4>(lds + tid * DP * 2 + (((D - 4) / 8) ^ k_swizzle<DP>(tid)) * 16) = u4{x[0], x[1], 0u, 0u};
}
template <int DP>
__device__ __forceinline__ void clear_pads(int D, uint32_t lds, int bytes, int tid) {
  if (D == DP) return;
  for (int i = tid * 16; i < bytes; i += 4096) *in_lds<u4>(lds + i) = u4{0u, 0u, 0u, 0u};
  __syncthreads();
}

// Shape of a workgroup: RW wavefronts side by side over the rows, 32 each, 4 / RW over the keys of a stage.
template <int DP, int RW>
struct Shape {
  static constexpr int KW = 4 / RW, KT = RW == 4 ? 64 : 32, SK = KW * KT;
  static constexpr int TILE = SK * DP * 2, STAGE = 2 * TILE;
  // two stages where they leave room for two workgroups on a CU
  static constexpr int STAGES = 2 * STAGE <= 65536 ? 2 : 1;
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

// Where a lane reads its operands, in the first stage.  K: row lane % 32, 16 bytes at 16 (2 t + its half).  V^T: lane i of sixteen
// takes row i / 4, columns 4 (i % 4) .. +3 and gets column i, rows 0..3.
template <int DP>
struct Reads {
  uint32_t k[DP / 16], v[DP / 32];
  __device__ __forceinline__ Reads(uint32_t ktile, uint32_t vtile, int lane) {
    const int half = lane >> 5, row = lane & 31, i = lane & 15;
#pragma unroll
    for (int t = 0; t < DP / 16; ++t) k[t] = ktile + row * DP * 2 + ((2 * t + half) ^ k_swizzle<DP>(row)) * 16;
#pragma unroll
    for (int d = 0; d < DP / 32; ++d)
      v[d] = vtile + (4 * half + (i >> 2)) * DP * 2 + ((d * 4 + 2 * ((lane >> 4) & 1) + ((i & 3) >> 1)) ^ v_swizzle<DP>(i >> 2)) * 16 + (i & 1) * 8;
  }
};
template <typename T>
__device__ __forceinline__ typename T::v8 read_k(uint32_t at) {
  return *in_lds<const typename T::v8>(at);
}
template <typename T, int DP>
__device__ __forceinline__ typename T::v8 read_v(uint32_t at) {
  const s4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16(in_lds<s4>(at));
  const s4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16(in_lds<s4>(at + 8 * DP * 2));
  return __builtin_bit_cast(typename T::v8, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
}

// NaN and infinities of V in a tile some of whose places are hidden from some rows: a hidden place must not give 0 * NaN.  The finite
// values are multiplied as ever, the others counted for the rows that see them: n1 +inf or NaN, n2 -inf or NaN, so that NaN comes
// out as inf - inf.  Rare, and the only loop over it that is not unrolled.
template <typename T, int DP, int KT>
__device__ __forceinline__ void multiply_odd_values(Rows<T, DP>& w, typename T::v8 (&p)[KT / 16], const uint32_t (&v)[DP / 32], int x) {
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
    const typename T::v8 pu = p[0];
#pragma unroll
    for (int j = 1; j < KT / 16; ++j) p[j - 1] = p[j];
#pragma unroll
    for (int d = 0; d < DP / 32; ++d) {
      const u4 a = __builtin_bit_cast(u4, read_v<T, DP>(v[d] + 16 * u * DP * 2));
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

// Whether a wavefront's tile of V, KT rows from `vtile`, has anything but finite values.
template <typename T, int BYTES>
__device__ __forceinline__ bool has_odd_values(uint32_t vtile, int lane) {
  bool found = false;
#pragma unroll 4
  for (int i = 0; i < BYTES / 1024; ++i) {
    const u4 q = *in_lds<const u4>(vtile + (i * 64 + lane) * 16);
#pragma unroll
    for (int j = 0; j < 4; ++j) found |= (q[j] & T::EXP) == T::EXP || (q[j] & (T::EXP << 16)) == (T::EXP << 16);
  }
  return __any(found);
}

// One tile of KT keys for one wavefront, `at` bytes after the places of `reads`.  MASKED: the lane's row sees x of the tile's
// keys (less four in the upper half), and where `hidden`, some of those it does not see are there all the same.
template <typename T, int DP, int KT, bool MASKED, bool SCORES>
__device__ __forceinline__ void tile_step(Rows<T, DP>& w, const Reads<DP>& reads, uint32_t at, float c, bool hidden, int x, uint32_t vtile, int lane,
                                          float* scores) {
  constexpr int NT = DP / 16, ND = DP / 32, NB = KT / 32;
  f16x s[NB];
#pragma unroll
  for (int b = 0; b < NB; ++b) s[b] = (f16x)(0.0f);
#pragma unroll
  for (int t = 0; t < NT; ++t)
#pragma unroll
    for (int b = 0; b < NB; ++b) s[b] = T::mfma(read_k<T>(reads.k[t] + at + b * 32 * DP * 2), w.q[t], s[b]);
  if constexpr (SCORES) {
    // a decode step keeps its scores: the weights need the whole row's sum
    if (scores) {
      const int half = lane >> 5;
#pragma unroll
      for (int b = 0; b < NB; ++b)
#pragma unroll
        for (int r = 0; r < 4; ++r)
          *reinterpret_cast<f4*>(scores + b * 32 + r * 8 + half * 4) = f4{s[b][4 * r], s[b][4 * r + 1], s[b][4 * r + 2], s[b][4 * r + 3]};
    }
  }
  if constexpr (MASKED) {
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
  if constexpr (MASKED) {
    if (hidden && has_odd_values<T, KT * DP * 2>(vtile + at, lane)) {
      uint32_t v[ND];
#pragma unroll
      for (int d = 0; d < ND; ++d) v[d] = reads.v[d] + at;
      multiply_odd_values<T, DP, KT>(w, p, v, x);
      return;
    }
  }
#pragma unroll
  for (int u = 0; u < KT / 16; ++u)
#pragma unroll
    for (int d = 0; d < ND; ++d) w.o[d] = T::mfma(read_v<T, DP>(reads.v[d] + at + 16 * u * DP * 2), p[u], w.o[d]);
}

// Whether a wavefront's loads into LDS have landed, then the workgroup's.
__device__ __forceinline__ void wait_stage() { asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory"); }

// Keys that the rows see, counted from the sequence's start and at most keys.end: the lane's own row, the least of the
// workgroup's and of the wavefront's rows, the most of the wavefront's.
struct Limits {
  int row, least_wg, least, most;
};

// All keys of a unit for the workgroup's rows.  scores: where the lane's row keeps its scores (index 0 = keys.begin), or null.
template <typename T, int DP, int RW, bool SCORES>
__device__ __forceinline__ void run_keys(Rows<T, DP>& w, const Keys& keys, int D, float c, const Limits& lim, char* shared, float* scores) {
  typedef Shape<DP, RW> Sh;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int kw = RW == 4 ? 0 : wave / RW;  // which part of a stage's keys
  const uint32_t lds = (uint32_t)(uintptr_t)(TMAC_LDS char*)shared;
#pragma unroll
  for (int d = 0; d < DP / 32; ++d) w.o[d] = (f16x)(0.0f);
  w.m = -INFINITY;
  w.l = 0.0f;
  if (keys.begin >= keys.end) return;
  clear_pads<DP>(D, lds, Sh::STAGES * Sh::STAGE, tid);
  const Stage<DP, Sh::SK, false> ks(keys.k_stride, D, wave, lane);
  const Stage<DP, Sh::SK, true> vs(keys.v_stride, D, wave, lane);
  const Reads<DP> reads(lds + kw * Sh::KT * DP * 2, lds + Sh::TILE + kw * Sh::KT * DP * 2, lane);
  auto load = [&](int at, uint32_t to) {
    const char* kb = keys.k + (int64_t)at * keys.k_stride;
    ks.load(kb, keys.k_stride, keys.end - at, D, lds + to, wave);
    vs.load(keys.v + (int64_t)at * keys.v_stride, keys.v_stride, keys.end - at, D, lds + to + Sh::TILE, wave);
    return load_tail<Sh::SK>(kb, keys.k_stride, keys.end - at, D, tid);
  };
  auto whole = [&](int at, uint32_t from) {
    tile_step<T, DP, Sh::KT, false, SCORES>(w, reads, from, c, false, 0, 0, lane, SCORES && scores ? scores + (at + kw * Sh::KT - keys.begin) : nullptr);
  };
  auto masked = [&](int at, uint32_t from) {
    const int first = at + kw * Sh::KT;  // the wavefront's first key
    if (first >= lim.most) return;
    tile_step<T, DP, Sh::KT, true, SCORES>(w, reads, from, c, lim.least < min(keys.end, first + Sh::KT), lim.row - first - 4 * (lane >> 5),
                                           lds + Sh::TILE + kw * Sh::KT * DP * 2, lane, SCORES && scores ? scores + (first - keys.begin) : nullptr);
  };
  int at = keys.begin;
  if constexpr (Sh::STAGES == 2) {
    store_tail<DP, Sh::SK>(load(at, 0), D, lds, tid);
    // stages that every row sees whole, two at a time, so that their places are constants
    while (at + 2 * Sh::SK <= lim.least_wg) {
      wait_stage();
      u2 tail = load(at + Sh::SK, Sh::STAGE);
      whole(at, 0);
      store_tail<DP, Sh::SK>(tail, D, lds + Sh::STAGE, tid);
      at += Sh::SK;
      wait_stage();
      if (at + Sh::SK < keys.end) tail = load(at + Sh::SK, 0);
      whole(at, Sh::STAGE);
      store_tail<DP, Sh::SK>(tail, D, lds, tid);
      at += Sh::SK;
    }
    uint32_t from = 0;
#pragma unroll 1
    for (; at < keys.end; at += Sh::SK) {
      wait_stage();
      u2 tail = {0u, 0u};
      if (at + Sh::SK < keys.end) tail = load(at + Sh::SK, from ^ Sh::STAGE);
      masked(at, from);
      from ^= Sh::STAGE;
      store_tail<DP, Sh::SK>(tail, D, lds + from, tid);
    }
  } else {
    bool again = false;
    for (; at + Sh::SK <= lim.least_wg; at += Sh::SK) {
      if (again) __syncthreads();
      again = true;
      store_tail<DP, Sh::SK>(load(at, 0), D, lds, tid);
      wait_stage();
      whole(at, 0);
    }
#pragma unroll 1
    for (; at < keys.end; at += Sh::SK) {
      if (again) __syncthreads();
      again = true;
      store_tail<DP, Sh::SK>(load(at, 0), D, lds, tid);
      wait_stage();
      masked(at, 0);
    }
  }
}

}  // namespace attn
}  // namespace tmac
#endif
