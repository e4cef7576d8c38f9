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
#include <type_traits>

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

// HEADROOM: the sums are taken against the row's maximum less this (in units of log 2).  Exponentials of fp16 then reach 2^7, and 2^15
// before the maximum is moved (outgrows), and keep all their bits down to 2^-20 of the row's largest; below that they are off by at most
// 2^-31 of it.  (Against the maximum itself a flat tail of 10^5 keys beside a heavy one lost what lay below 2^-25.)  bf16 has the range anyway.
struct F16 {
  static constexpr float HEADROOM = 7.0f;
  typedef _Float16 elem;
  typedef h4 v4;
  typedef h8 v8;
  static constexpr uint32_t EXP = 0x7C00u, NEG_INF = 0xFC00u, POS_INF = 0x7C00u, ONE = 0x3C00u;
  static __device__ __forceinline__ f16x mfma(v8 a, v8 b, f16x c) { return __builtin_amdgcn_mfma_f32_32x32x16_f16(a, b, c, 0, 0, 0); }
};
struct BF16 {
  static constexpr float HEADROOM = 0.0f;
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

// Tiles of 16-bit rows, padded to DP elements, in LDS.  A load of one wavefront fills 1024 bytes, 16 a lane, in whole rows (pieces
// of rows would come slower from memory), within which the lanes' order is free.  K (and q for the weights) is read 16 bytes of 32 rows
// at a time: chunks of 16 bytes are permuted within fours by the row, and each 1024 bytes are followed by 64 unused ones; sixteen
// rows' chunks then meet all banks, and the products' steps along a row differ by constants.  V is read 64 bytes of four rows at a
// time: its 64-byte pieces are permuted by the row.
template <int DP>
struct Layout {
  static constexpr int CH = DP / 8, RPI = 64 / CH;  // chunks of a row, rows of a load
  static constexpr int k_bytes(int rows) { return rows / RPI * 1088; }
  static constexpr int v_bytes(int rows) { return rows * DP * 2; }
  static __host__ __device__ __forceinline__ int k_swizzle(int row) { return (DP == 128 ? row : row >> 1) & 3; }
  static __host__ __device__ __forceinline__ int v_swizzle(int row) { return (DP == 128 ? row & 3 : row >> 1 & 1) << 2; }
  static __device__ __forceinline__ int k_row(int row) { return row / RPI * 1088 + row % RPI * DP * 2; }
};

// What a workgroup reads: keys [begin, end) of one sequence and key head.
struct Keys {
  const char* k;               // row 0 of the sequence and head
  const char* v;
  int64_t k_stride, v_stride;  // bytes from row to row
  int begin, end;
  bool once;                   // read once, and more of them in a call than the caches hold (run_streams with SCORES only)
};

// Rows of 16-bit elements on their way from memory to LDS: 1024 bytes a load of one wavefront, lane after lane, without passing
// through registers.  Memory need only be 8-byte aligned.  Chunks of 16 bytes that lie within the row's D elements are loaded;
// a half chunk at the row's end (D % 8 == 4) comes with its neighbour's elements, or with zeros after the last row, which is fine for V,
// whose columns from D on give results that nobody reads, but not for K, where they would meet the products' sums: there the half chunk goes through a
// register (load_tail, store_tail).  Chunks beyond are cleared once (clear_pads).
//
// The load is written out: of the builtin the compiler knows only that it writes LDS, and makes every transposed read wait
// for it, although that is another stage.  It has no result register; wait_stage waits for it.
__device__ __forceinline__ void load_to_lds(u4 rsrc, uint32_t lds, uint32_t offset, uint32_t scalar_offset) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, %3 offen lds"
               :
               : "s"(__builtin_amdgcn_readfirstlane(lds)), "v"(offset), "s"(rsrc), "s"(__builtin_amdgcn_readfirstlane(scalar_offset))
               : "memory");
}
// The same for bytes that nobody reads again soon.
__device__ __forceinline__ void load_to_lds_once(u4 rsrc, uint32_t lds, uint32_t offset, uint32_t scalar_offset) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, %3 offen nt lds"
               :
               : "s"(__builtin_amdgcn_readfirstlane(lds)), "v"(offset), "s"(rsrc), "s"(__builtin_amdgcn_readfirstlane(scalar_offset))
               : "memory");
}
__device__ __forceinline__ u4 buffer_of(const char* base, int range) {
  const uint64_t at = (uint64_t)base;
  return u4{(uint32_t)__builtin_amdgcn_readfirstlane((int)at), (uint32_t)__builtin_amdgcn_readfirstlane((int)(at >> 32)) & 0xffffu,
            (uint32_t)__builtin_amdgcn_readfirstlane(range), 0x00020000u};
}
// WAVES wavefronts share the ROWS rows, or each loads rows of its own (WAVES = 1).
template <int DP, int ROWS, int WAVES, bool IS_V>
struct Stage {
  typedef Layout<DP> L;
  static constexpr int N = ROWS / (WAVES * L::RPI), APART = IS_V ? 1024 : 1088;
  uint32_t at;   // bytes from the first row to the lane's chunk in the wavefront's first load
  bool wanted;   // its elements lie within the row (K: all of them)

  __host__ __device__ __forceinline__ Stage(int64_t stride, int D, int wave, int lane) {
    const int row = lane / L::CH, chunk = (lane % L::CH) ^ (IS_V ? L::v_swizzle(row) : L::k_swizzle(row));
    at = (row + (WAVES == 1 ? 0 : wave * L::RPI)) * (uint32_t)stride + chunk * 16;
    wanted = IS_V ? chunk * 8 < D : chunk * 8 + 8 <= D;
  }
  // Bytes from the first row to the end of the last of n.
  static __host__ __device__ __forceinline__ int span(int64_t stride, int n, int D) { return n > 0 ? (n - 1) * (int)stride + D * 2 : 0; }
  // Whether scalar offsets may take the loads from row to row of a stage of which `rows` are there.  They are not checked against the
  // range, so all rows have to be there, and for V's half chunks, which come with the eight bytes after the row, one more.
  static __host__ __device__ __forceinline__ bool unchecked(int rows, int D) { return rows >= ROWS + (IS_V && D % 8 ? 1 : 0); }
  // Rows from `rows` on read as zeros: the descriptor's range ends there.  Unwanted chunks stay as they are where wavefronts share a
  // stage, and become zeros where they do not: such a load is always issued, so that loads can be counted.
  __device__ __forceinline__ void load(const char* base, int64_t stride, int rows, int D, uint32_t lds, int wave, bool once = false) const {
    if (WAVES != 1 && !wanted) return;
    const uint32_t offset = wanted ? at : 0x7fffff00u;
    const int step = WAVES * L::RPI * (int)stride;
    if (WAVES != 1) lds += wave * APART;
    if (unchecked(rows, D)) {
      const u4 rsrc = buffer_of(base, span(stride, ROWS, D));
      if (once) {
#pragma unroll
        for (int i = 0; i < N; ++i) load_to_lds_once(rsrc, lds + i * WAVES * APART, offset, i * step);
        return;
      }
#pragma unroll
      for (int i = 0; i < N; ++i) load_to_lds(rsrc, lds + i * WAVES * APART, offset, i * step);
    } else {
      const int range = span(stride, min(rows, ROWS), D);
#pragma unroll
      for (int i = 0; i < N; ++i) load_to_lds(buffer_of(base + i * (int64_t)step, max(0, range - i * step)), lds + i * WAVES * APART, offset, 0);
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
    *in_lds<u4>(lds + Layout<DP>::k_row(tid) + (((D - 4) / 8) ^ Layout<DP>::k_swizzle(tid)) * 16) = u4{x[0], x[1], 0u, 0u};
}
// (four wavefronts that share a stage)
template <int DP>
__device__ __forceinline__ void clear_pads(int D, uint32_t lds, int bytes, int tid) {
  if (D == DP) return;
  for (int i = tid * 16; i < bytes; i += 4096) *in_lds<u4>(lds + i) = u4{0u, 0u, 0u, 0u};
  __syncthreads();
}

// Shape of a workgroup, by the blocks of 32 rows that it serves.  4: its wavefronts have one each and share every stage of 32 KB
// keys, of which there are two.  1: all have the same block and stream tiles of 32 keys of their own, every fourth; their sums meet in
// LDS at the end.
template <int DP, int BLOCKS>
struct Shape {
  static constexpr int KB = 2;
  static constexpr int MERGE = BLOCKS == 1 ? 4 * 32 * (DP + 4) * 4 + 4 * 32 * 8 : 0;
  static constexpr int STAGES = (BLOCKS == 4 ? 2 * KB : 4) * (Layout<DP>::k_bytes(32) + Layout<DP>::v_bytes(32));
  static constexpr int LDS = STAGES > MERGE ? STAGES : MERGE;
};

// The running softmax and sums of one wavefront's 32 rows.
template <typename T, int DP>
struct Rows {
  typename T::v8 q[DP / 16];
  f16x o[DP / 32];
  float m, l;  // what the sums are taken against, in units of log 2, a whole number or infinite; sum of this half's exponentials
};

// Where a lane reads its operands.  K: row lane % 32, for step t of the product the chunk 2 t + the lane's half.  V^T: lane i of sixteen
// takes row i / 4, columns 4 (i % 4) .. +3 and gets column i, rows 0..3.
template <int DP>
struct Reads {
  uint32_t k[2], v[DP / 32], tile;  // tile: that of V itself
  __device__ __forceinline__ Reads(uint32_t ktile, uint32_t vtile, int lane) : tile(vtile) {
    const int half = lane >> 5, row = lane & 31, i = lane & 15;
#pragma unroll
    for (int y = 0; y < 2; ++y) k[y] = ktile + Layout<DP>::k_row(row) + ((2 * y + half) ^ Layout<DP>::k_swizzle(row)) * 16;
#pragma unroll
    for (int d = 0; d < DP / 32; ++d)
      v[d] = vtile + (4 * half + (i >> 2)) * DP * 2 + ((d * 4 + 2 * (lane >> 4 & 1) + ((i & 3) >> 1)) ^ Layout<DP>::v_swizzle(i >> 2)) * 16 + (i & 1) * 8;
  }
  __device__ __forceinline__ uint32_t k_at(int t) const { return k[t & 1] + (t >> 1) * 64; }
  __device__ __forceinline__ uint32_t v_at(int u, int d) const { return v[d] + u * DP * 32; }
  __device__ __forceinline__ void turn_k(int by) { k[0] += by, k[1] += by; }
  __device__ __forceinline__ void turn_v(int by) {
    tile += by;
#pragma unroll
    for (int d = 0; d < DP / 32; ++d) v[d] += by;
  }
};
template <typename T>
__device__ __forceinline__ typename T::v8 read_k(uint32_t at) {
  return *in_lds<const typename T::v8>(at);
}
template <typename T, int DP>
__device__ __forceinline__ typename T::v8 read_v(uint32_t at) {
  const s4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16(in_lds<s4>(at));
  const s4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16(in_lds<s4>(at + DP * 16));
  return __builtin_bit_cast(typename T::v8, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
}

// NaN and infinities of V in a tile some of whose places are hidden from some rows: a hidden place must not give 0 * NaN.  The finite
// values are multiplied as ever, the others counted for the rows that see them: n1 +inf or NaN, n2 -inf or NaN, so that NaN comes
// out as inf - inf.  Rare, and the only loop over it that is not unrolled.  x: keys of the tile that the lane's row sees (less four
// in the upper half).
template <typename T, int DP, int KT>
__device__ __forceinline__ void multiply_odd_values(Rows<T, DP>& w, typename T::v8 (&p)[KT / 16], const Reads<DP>& reads, int x) {
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
      const u4 a = __builtin_bit_cast(u4, read_v<T, DP>(reads.v_at(u, d)));
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
      __builtin_amdgcn_sched_barrier(0);  // (one count at a time in registers)
      const f16x n1 = T::mfma(__builtin_bit_cast(typename T::v8, up), sees, (f16x)(0.0f));
#pragma unroll
      for (int r = 0; r < 16; ++r) w.o[d][r] += n1[r] > 0.0f ? INFINITY : 0.0f;
      __builtin_amdgcn_sched_barrier(0);
      const f16x n2 = T::mfma(__builtin_bit_cast(typename T::v8, down), sees, (f16x)(0.0f));
#pragma unroll
      for (int r = 0; r < 16; ++r) w.o[d][r] += n2[r] > 0.0f ? -INFINITY : 0.0f;
      __builtin_amdgcn_sched_barrier(0);
    }
  }
}

// Whether a wavefront's tile of V has anything but finite values.
template <typename T, int BYTES>
__device__ __forceinline__ bool has_odd_values(uint32_t vtile, int lane) {
  bool found = false;
#pragma unroll 1
  for (int i = 0; i < BYTES / 1024; ++i) {
    const u4 q = *in_lds<const u4>(vtile + (i * 64 + lane) * 16);
#pragma unroll
    for (int j = 0; j < 4; ++j) found |= (q[j] & T::EXP) == T::EXP || (q[j] & (T::EXP << 16)) == (T::EXP << 16);
  }
  return __any(found);
}

// Whether any row of the wavefront has sums that are not finite.
template <typename T, int DP>
__device__ __forceinline__ bool has_odd_sums(const Rows<T, DP>& w) {
  float x = 0.0f;
#pragma unroll
  for (int d = 0; d < DP / 32; ++d)
#pragma unroll
    for (int r = 0; r < 16; ++r) x = __builtin_fmaf(w.o[d][r], 0.0f, x);
  return __any(x != x);
}

// Scores of 32 keys for the lane's row.
template <typename T, int DP>
__device__ __forceinline__ f16x scores_of(const Rows<T, DP>& w, const Reads<DP>& reads, int bytes) {
  f16x s = (f16x)(0.0f);
#pragma unroll
  for (int t = 0; t < DP / 16; ++t) s = T::mfma(read_k<T>(reads.k_at(t) + bytes), w.q[t], s);
  return s;
}

__device__ __forceinline__ float largest(const f16x& s) {
  float mx = s[0];
#pragma unroll
  for (int r = 1; r < 16; ++r) mx = fmaxf(mx, s[r]);
  return mx;
}

// Whether the row's sums have to be taken against a larger number.  They keep theirs until a score is 2^8 times larger:
// exponentials 256 times as large are as exact in 16 bits, and most tiles then need no rescaling.  (Row by row: a row's bits do not
// depend on its neighbours.)  A whole number in units of log 2, so that what is rescaled keeps its bits.  Compared is the exponent
// itself, so that it stays within the type also where m is too large for its last digits.
template <typename T>
__device__ __forceinline__ bool outgrows(float mx, float c, float m) {
  return __builtin_fmaf(mx, c, -m) > T::HEADROOM + 8.0f;
}
// log 2 of the sum of exp of a row's scores; l: of its exponentials against m.
template <typename T>
__device__ __forceinline__ float log2_sum(float m, float l) {
  return m + T::HEADROOM + __builtin_log2f(l * __builtin_exp2f(-T::HEADROOM));
}
template <typename T, int DP>
__device__ __forceinline__ void rescale(Rows<T, DP>& w, float mx, float c, bool grows) {
  const float m = grows ? __builtin_ceilf(mx * c) - T::HEADROOM : w.m;
  const float alpha = grows ? __builtin_amdgcn_exp2f(w.m - m) : 1.0f;
#pragma unroll
  for (int d = 0; d < DP / 32; ++d) w.o[d] *= alpha;
  w.l *= alpha;
  w.m = m;
}

// exp(s - m) of 32 keys, rounded to the type for the second product; returns their sum before rounding.
template <typename T>
__device__ __forceinline__ float exponentials(const f16x& s, float c, float m, typename T::v8& p0, typename T::v8& p1) {
  f16x e;
  float sum[2] = {0.0f, 0.0f};
#pragma unroll
  for (int r = 0; r < 16; ++r) {
    e[r] = __builtin_amdgcn_exp2f(__builtin_fmaf(s[r], c, -m));
    sum[r & 1] += e[r];
  }
  p0 = __builtin_convertvector(__builtin_shufflevector(e, e, 0, 1, 2, 3, 4, 5, 6, 7), typename T::v8);
  p1 = __builtin_convertvector(__builtin_shufflevector(e, e, 8, 9, 10, 11, 12, 13, 14, 15), typename T::v8);
  return sum[0] + sum[1];
}

// What exponents are taken against: a row without a score above -inf keeps exponentials of zero.
__device__ __forceinline__ float base_of(float m) { return m == -INFINITY ? 0.0f : m; }

template <typename T, int DP, int KT>
__device__ __forceinline__ void multiply_v(Rows<T, DP>& w, const Reads<DP>& reads, const typename T::v8 (&p)[KT / 16]) {
#pragma unroll
  for (int u = 0; u < KT / 16; ++u)
#pragma unroll
    for (int d = 0; d < DP / 32; ++d) w.o[d] = T::mfma(read_v<T, DP>(reads.v_at(u, d)), p[u], w.o[d]);
}

// Scores beyond the x keys of 32 that the lane's row sees (less four in the upper half).
__device__ __forceinline__ void hide(f16x& s, int x) {
#pragma unroll
  for (int r = 0; r < 16; ++r) s[r] = (r >> 2) * 8 + (r & 3) < x ? s[r] : -INFINITY;
}

// Keys that the rows see, counted from the sequence's start and at most keys.end: the lane's own row, the least of the
// workgroup's and of the wavefront's rows, the most of the wavefront's.
struct Limits {
  int row, least_wg, least, most;
};

// Where a decode step keeps its scores (the weights need the whole row's sum): one row of floats per lane's row, index 0 =
// keys.begin, in memory (rows that do not exist have an offset out of the range) or in LDS.
struct Scores {
  float* base;      // null: not in memory
  int range;        // bytes
  uint32_t offset;  // the lane's, in bytes
  static constexpr uint32_t NOWHERE = ~0u;  // (0 is a place)
  uint32_t lds = NOWHERE;                   // the lane's row there
};

template <typename T, int DP>
__device__ __forceinline__ void clear(Rows<T, DP>& w) {
#pragma unroll
  for (int d = 0; d < DP / 32; ++d) w.o[d] = (f16x)(0.0f);
  w.m = -INFINITY;
  w.l = 0.0f;
}

// Whether a wavefront's loads into LDS have landed, then the workgroup's.
__device__ __forceinline__ void wait_stage() { asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory"); }

// All keys of a unit where four wavefronts share the stages, of 32 KB keys each.
//
// A hidden place has an exponential of zero, and 0 * NaN is NaN: values of V that are not finite would show in rows that do not
// see them.  They are not looked for (that cost 15 % where sequences are short): the sums then hold something that is not finite
// at the end, and the unit is run again, CAREFUL, with the same bits for the rows that such values do not concern.
template <typename T, int DP, int KB, bool CAREFUL>
__device__ __forceinline__ void run_shared(Rows<T, DP>& w, const Keys& keys, int D, float c, const Limits& lim, char* shared) {
  constexpr int SK = 32 * KB, KS = Layout<DP>::k_bytes(SK), VS = Layout<DP>::v_bytes(SK);  // a stage's keys, its bytes
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const uint32_t lds = (uint32_t)(uintptr_t)(TMAC_LDS char*)shared, lds_v = lds + 2 * KS;  // two stages of K, two of V
  clear(w);
  if (keys.begin >= keys.end) return;
  clear_pads<DP>(D, lds, 2 * (KS + VS), tid);
  const Stage<DP, SK, 4, false> ks(keys.k_stride, D, wave, lane);
  const Stage<DP, SK, 4, true> vs(keys.v_stride, D, wave, lane);
  Reads<DP> reads(lds, lds_v, lane);
  // the stage from key `at` on goes to `place` (0 or 1); what a row's last half chunk needs of a register is stored after the
  // computation that the load runs beside
  auto load = [&](int at, int place) {
    const char* base = keys.k + (int64_t)at * keys.k_stride;
    ks.load(base, keys.k_stride, keys.end - at, D, lds + place * KS, wave);
    vs.load(keys.v + (int64_t)at * keys.v_stride, keys.v_stride, keys.end - at, D, lds_v + place * VS, wave);
    return load_tail<SK>(base, keys.k_stride, keys.end - at, D, tid);
  };
  store_tail<DP, SK>(load(keys.begin, 0), D, lds, tid);
  int place = 0, at = keys.begin;
  auto turn = [&](u2 tail) {
    reads.turn_k(place ? -KS : KS);
    reads.turn_v(place ? -VS : VS);
    place ^= 1;
    at += SK;
    store_tail<DP, SK>(tail, D, lds + place * KS, tid);
  };
  auto step = [&](auto masked) {
    f16x s[KB];
    typename T::v8 p[2 * KB];
#pragma unroll
    for (int b = 0; b < KB; ++b) s[b] = (f16x)(0.0f);
#pragma unroll
    for (int t = 0; t < DP / 16; ++t)
#pragma unroll
      for (int b = 0; b < KB; ++b) s[b] = T::mfma(read_k<T>(reads.k_at(t) + b * Layout<DP>::k_bytes(32)), w.q[t], s[b]);
    const int x = lim.row - at - 4 * (lane >> 5);
    if constexpr (masked) {
#pragma unroll
      for (int b = 0; b < KB; ++b) hide(s[b], x - 32 * b);
    }
    float mx = largest(s[0]);
#pragma unroll
    for (int b = 1; b < KB; ++b) mx = fmaxf(mx, largest(s[b]));
    mx = max_halves(mx);
    const bool grows = outgrows<T>(mx, c, w.m);
    if (__any(grows)) rescale(w, mx, c, grows);
    const float m = base_of(w.m);
#pragma unroll
    for (int b = 0; b < KB; ++b) w.l += exponentials<T>(s[b], c, m, p[2 * b], p[2 * b + 1]);
    if constexpr (CAREFUL) {
      if (has_odd_values<T, VS>(reads.tile, lane)) {
        multiply_odd_values<T, DP, SK>(w, p, reads, x);
        return;
      }
    }
    multiply_v<T, DP, SK>(w, reads, p);
  };
  auto next_stage = [&] {
    wait_stage();
    return at + SK < keys.end ? load(at + SK, place ^ 1) : u2{0u, 0u};
  };
  if constexpr (!CAREFUL) {
    while (at + SK <= lim.least_wg) {  // stages that every row sees whole
      const u2 tail = next_stage();
      step(std::false_type{});
      turn(tail);
    }
  }
#pragma unroll 1
  while (at < keys.end) {
    const u2 tail = next_stage();
    if (at < lim.most) step(std::true_type{});
    turn(tail);
  }
}

// All keys of a unit where every wavefront streams tiles of its own, 32 keys each, every fourth: a tile of K is requested as soon as
// the one before has met q, one of V as soon as the one before has met the exponentials, and nobody waits for anybody.
// SCORES: a cache, which keeps its scores where `scores` says.  ON: the rows have met other keys before.
template <typename T, int DP, bool SCORES, bool CAREFUL, bool ON = false>
__device__ __forceinline__ void run_streams(Rows<T, DP>& w, const Keys& keys, int D, float c, const Limits& lim, char* shared, const Scores& scores) {
  constexpr int KT = 32, KB = Layout<DP>::k_bytes(KT), VB = Layout<DP>::v_bytes(KT);
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const uint32_t lds = (uint32_t)(uintptr_t)(TMAC_LDS char*)shared + wave * (KB + VB), lds_v = lds + KB;
  if constexpr (!ON) clear(w);
  const Stage<DP, KT, 1, false> ks(keys.k_stride, D, wave, lane);
  const Stage<DP, KT, 1, true> vs(keys.v_stride, D, wave, lane);
  constexpr int LOADS = Stage<DP, KT, 1, false>::N;
  const Reads<DP> reads(lds, lds_v, lane);
  const int end = min(keys.end, lim.most);
  int at = keys.begin + wave * KT;
  if (at >= end) return;
  u2 tail;
  auto load_k = [&](int i) {
    const char* base = keys.k + (int64_t)i * keys.k_stride;
    ks.load(base, keys.k_stride, keys.end - i, D, lds, wave, SCORES && keys.once);
    tail = load_tail<KT>(base, keys.k_stride, keys.end - i, D, lane);
  };
  auto load_v = [&](int i) { vs.load(keys.v + (int64_t)i * keys.v_stride, keys.v_stride, keys.end - i, D, lds_v, wave, SCORES && keys.once); };
  load_k(at);
  load_v(at);
  bool stored = false;  // the tile before left scores, four stores after V's loads
  while (true) {
    // K has landed: V's loads, and stores of scores, are younger
    if (SCORES && stored) asm volatile("s_waitcnt vmcnt(%0)" ::"n"(LOADS + 4) : "memory");
    else asm volatile("s_waitcnt vmcnt(%0)" ::"n"(LOADS) : "memory");
    store_tail<DP, KT>(tail, D, lds, lane);
    f16x s = scores_of(w, reads, 0);
    const int next = at + 4 * KT;
    // (the products have read all of K)
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    if (next < end) load_k(next);
    const f16x raw = s;
    const int x = lim.row - at - 4 * (lane >> 5);
    if (lim.least < at + KT) hide(s, x);
    const float mx = max_halves(largest(s));
    const bool grows = outgrows<T>(mx, c, w.m);
    if (__any(grows)) rescale(w, mx, c, grows);
    typename T::v8 p[2];
    w.l += exponentials<T>(s, c, base_of(w.m), p[0], p[1]);
    if (next < end) asm volatile("s_waitcnt vmcnt(%0)" ::"n"(LOADS) : "memory");
    else asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    bool odd = false;
    if constexpr (CAREFUL) odd = has_odd_values<T, VB>(lds_v, lane);
    if (odd) multiply_odd_values<T, DP, 32>(w, p, reads, x);
    else multiply_v<T, DP, 32>(w, reads, p);
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    if (next < end) load_v(next);
    if (SCORES && scores.base) {
      const auto rsrc = __builtin_amdgcn_make_buffer_rsrc(scores.base, (short)0, scores.range, 0x00020000);
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const f4 x4 = {raw[4 * r], raw[4 * r + 1], raw[4 * r + 2], raw[4 * r + 3]};
        __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(u4, x4), rsrc, (int)(scores.offset + (uint32_t)(at - keys.begin + r * 8 + (lane >> 5) * 4) * 4u), 0, 0);
      }
      stored = true;
    }
    if (SCORES && scores.lds != Scores::NOWHERE) {
#pragma unroll
      for (int r = 0; r < 4; ++r)
        *in_lds<f4>(scores.lds + (at - keys.begin + r * 8 + (lane >> 5) * 4) * 4) = f4{raw[4 * r], raw[4 * r + 1], raw[4 * r + 2], raw[4 * r + 3]};
    }
    if (next >= end) break;
    at = next;
  }
}

}  // namespace attn
}  // namespace tmac
#endif
