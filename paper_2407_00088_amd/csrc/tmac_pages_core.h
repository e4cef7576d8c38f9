// Pages of keys and values in 8 bits (tmac_pages.h): where things lie, codes and their values, sequences of a call.
#ifndef TMAC_PAGES_CORE_H_
#define TMAC_PAGES_CORE_H_

#include <hip/hip_runtime.h>

#include <cstdint>

#include "tmac_pages.h"

namespace tmac {
namespace pages {

typedef _Float16 h2 __attribute__((ext_vector_type(2)));
typedef _Float16 h8 __attribute__((ext_vector_type(8)));
typedef float f2 __attribute__((ext_vector_type(2)));
typedef float f4 __attribute__((ext_vector_type(4)));
typedef uint32_t u2 __attribute__((ext_vector_type(2)));
typedef uint32_t u4 __attribute__((ext_vector_type(4)));

constexpr int BT = TMAC_BLOCK_TOKENS;
constexpr float LEAST_SCALE = 0x1p-60f;

__host__ __device__ __forceinline__ int clamp_to(int x, int most) { return x < 0 ? 0 : x > most ? most : x; }

// --- where things lie ---------------------------------------------------------------------------------------------------------

struct Pages {
  char* codes;
  float* scales;
  int pages, shift, Hkv, D, chunks;  // a page has 2^shift blocks; chunks of 16 elements of a row

  __host__ __device__ __forceinline__ int plane_bytes() const { return chunks * 512; }  // a block's keys, or its values
  // The unit of block `part` of a page that there is.
  __host__ __device__ __forceinline__ int64_t unit(int page, int part, int head) const {
    return (((int64_t)page * Hkv + head) << shift) + part;
  }
  // Of a sequence's block; -1 where the table has no page for it.
  __host__ __device__ __forceinline__ int64_t unit_of(const int32_t* table, int width, int block, int head) const {
    const int at = block >> shift;
    if (at >= width) return -1;
    const int page = table[at];
    return (unsigned)page < (unsigned)pages ? unit(page, block & ((1 << shift) - 1), head) : -1;
  }
  __host__ __device__ __forceinline__ char* keys(int64_t u) const { return codes + u * (2 * plane_bytes()); }
  __host__ __device__ __forceinline__ char* values(int64_t u) const { return codes + u * (2 * plane_bytes()) + plane_bytes(); }
};
// Bytes within a block's keys and values.
__host__ __device__ __forceinline__ int key_at(int token, int d) { return (d >> 4) * 512 + token * 16 + (d & 15); }
__host__ __device__ __forceinline__ int value_run(int chunks, int d) { return chunks * 16 - (d & ~31) < 32 ? 16 : 32; }
__host__ __device__ __forceinline__ int value_at(int chunks, int token, int d) {
  return (d >> 5) * 1024 + ((token >> 2 & 1) * value_run(chunks, d) + (d & 31)) * 16 + (token >> 3 & 1) * 8 + (token >> 4) * 4 + (token & 3);
}
// The token of byte j of a half's 16.
__host__ __device__ __forceinline__ int value_token(int half, int j) { return (j >> 3) * 8 + (j >> 2 & 1) * 16 + half * 4 + (j & 3); }

// What a lane reads of a block's keys and values as operands of 32 or 16 rows (tmac_pages_attn.hip): bytes, of which `fixed` are the
// same for all lanes.  Chunks and runs that are not there lie past the plane's end or NOWHERE, and read as zeros.
struct At {
  int lane, fixed;
};
constexpr int NOWHERE = 1 << 20;
struct Reads32 {  // v_mfma_f32_32x32x16: load i has 32 elements; keys: token lane & 31, 16 elements; values: element lane & 31, a half's 16 tokens
  static __host__ __device__ __forceinline__ At k(int i, int lane) { return {lane * 16, i * 1024}; }
  // last: of a row's runs of 32; odd: that has 16 elements only
  static __host__ __device__ __forceinline__ At v(int i, int lane, bool last, bool odd) {
    const int half = lane >> 5, d = lane & 31;
    return {last && odd ? (d < 16 ? half * 256 + d * 16 : NOWHERE) : lane * 16, i * 1024};
  }
};
struct Reads16 {  // v_mfma_f32_16x16x32: keys: load i has tokens 0-15 or 16-31 of 64 elements, a quarter's 16; values: 16 elements, a quarter's 8 tokens
  static __host__ __device__ __forceinline__ At k(int i, int lane) { return {(lane >> 4) * 512 + (lane & 15) * 16, (i >> 1) * 2048 + (i & 1) * 256}; }
  static __host__ __device__ __forceinline__ At v(int i, int lane, bool last, bool odd) {
    return {(lane & 15) * 16 + (lane >> 5) * 8 + (lane >> 4 & 1) * (last && odd ? 256 : 512), (i >> 1) * 1024 + (i & 1) * 256};
  }
};

// --- sequences of a call -----------------------------------------------------------------------------------------------------

struct Batch {
  const int32_t *table, *lens, *cu;
  int64_t table_stride;
  int S, width, T, most;  // most: of a sequence's rows, T where it is not known

  __device__ __forceinline__ int start(int s) const { return cu ? clamp_to(cu[s], T) : s; }
  __device__ __forceinline__ const int32_t* row(int s) const { return table + s * table_stride; }
};
// One sequence: rows [row0, row0 + n) are tokens [first, len), where a token below 0 is none.
struct Sequence {
  int row0 = 0, n = 0, len = 0, first = 0;
  Sequence() = default;
  __device__ __forceinline__ Sequence(const Batch& b, int s) {
    row0 = b.start(s);
    n = max(0, b.start(s + 1) - row0);
    len = clamp_to(b.lens[s], 1 << 30);
    first = len - n;
  }
};

// How many of i = 1 .. n have at(i) <= x, where at() does not fall: all lanes of a wavefront look at once.
template <typename At>
__device__ __forceinline__ int count_up_to(int n, At&& at, int64_t x) {
  const int lane = threadIdx.x & 63;
  int found = 0;
  for (int i = 0; i < n; i += 64) {
    const bool is = i + lane < n && at(i + lane + 1) <= x;
    const int here = __builtin_popcountll(__ballot(is));
    found += here;
    if (here < 64) break;
  }
  return found;
}
// The sequence of a row of the call.
__device__ __forceinline__ int sequence_of(const Batch& b, int row) {
  return b.cu ? min(count_up_to(b.S, [&](int i) { return (int64_t)b.cu[i]; }, row), b.S - 1) : row;
}

// --- codes ----------------------------------------------------------------------------------------------------------------------

struct I8 {
  static constexpr float MOST = 127.0f;
  static __device__ __forceinline__ float scale_for(float most) { return fmaxf(most * (1.0f / MOST), LEAST_SCALE); }
  // Four numbers, already multiplied by 1 / scale, as codes: any, or such as the scale was made for.
  static __device__ __forceinline__ uint32_t encode(float a, float b, float c, float d) {
    auto one = [](float x) { return (uint32_t)(int)fminf(fmaxf(__builtin_rintf(x), -MOST), MOST) & 0xffu; };
    return one(a) | one(b) << 8 | one(c) << 16 | one(d) << 24;
  }
  // Of numbers up to 127.4: 1.5 * 2^23 more, they have no places after the point, and their low byte is the code.  (Not as one operation with the
  // product that they come from, which is rounded by itself.)
  static __device__ __forceinline__ uint32_t encode_within(float a, float b, float c, float d) {
    auto one = [](float x) {
#pragma clang fp contract(off)
      return __builtin_bit_cast(uint32_t, x + 12582912.0f);
    };
    return __builtin_amdgcn_perm(__builtin_amdgcn_perm(one(d), one(c), 0x0c0c0400u), __builtin_amdgcn_perm(one(b), one(a), 0x0c0c0400u), 0x05040100u);
  }
  static __device__ __forceinline__ void decode(uint32_t x, float (&y)[4]) {
#pragma unroll
    for (int i = 0; i < 4; ++i) y[i] = (float)((int)(x << (24 - 8 * i)) >> 24);
  }
};
struct E4M3 {
  static constexpr float MOST = 448.0f;
  // most / 448 rounded up to a power of two: 448 is 1.75 * 2^8.
  static __device__ __forceinline__ float scale_for(float most) {
    const uint32_t bits = __builtin_bit_cast(uint32_t, most);
    const int e = (int)(bits >> 23) - 8 + ((bits & 0x7fffffu) > 0x600000u);
    return e < 127 - 60 ? LEAST_SCALE : __builtin_bit_cast(float, (uint32_t)e << 23);
  }
  static __device__ __forceinline__ uint32_t encode(float a, float b, float c, float d) {
    auto in = [](float x) { return fminf(fmaxf(x, -MOST), MOST); };
    int x = __builtin_amdgcn_cvt_pk_fp8_f32(in(a), in(b), 0, false);
    return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(in(c), in(d), x, true);
  }
  static __device__ __forceinline__ uint32_t encode_within(float a, float b, float c, float d) {
    const int x = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
    return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(c, d, x, true);
  }
  static __device__ __forceinline__ void decode(uint32_t x, float (&y)[4]) {
    const f2 lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)x, false), hi = __builtin_amdgcn_cvt_pk_f32_fp8((int)x, true);
    y[0] = lo[0], y[1] = lo[1], y[2] = hi[0], y[3] = hi[1];
  }
};

// --- 16-bit elements ---------------------------------------------------------------------------------------------------------------

__device__ __forceinline__ float to_float(uint16_t x, bool bf16) {
  return bf16 ? __builtin_bit_cast(float, (uint32_t)x << 16) : (float)__builtin_bit_cast(_Float16, x);
}
__device__ __forceinline__ uint16_t from_float(float x, bool bf16) {
  return bf16 ? __builtin_bit_cast(uint16_t, (__bf16)x) : __builtin_bit_cast(uint16_t, (_Float16)x);
}

}  // namespace pages
}  // namespace tmac
#endif
