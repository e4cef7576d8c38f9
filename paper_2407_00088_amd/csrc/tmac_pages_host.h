// Checks of what the entry points of tmac_pages.h are given (host code).
#ifndef TMAC_PAGES_HOST_H_
#define TMAC_PAGES_HOST_H_

#include <algorithm>
#include <cstdint>

#include "tmac_attn_host.h"
#include "tmac_internal.h"
#include "tmac_pages_core.h"

namespace tmac {
namespace pages {

inline tmac_status launch_with(const void* kernel, int64_t grid, int threads, void** args, void* stream) {
  if (!attn::launchable(grid, threads)) return TMAC_EUNSUPPORTED;
  const hipError_t e = hipLaunchKernel(kernel, dim3((unsigned)grid), dim3((unsigned)threads), args, 0, static_cast<hipStream_t>(stream));
  if (e == hipSuccess) return TMAC_OK;
  note_hip_error((int)e);
  return TMAC_EHIP;
}
inline tmac_status launch(const void* kernel, int64_t grid, int threads, void* args, void* stream) {
  void* ptrs[] = {args};
  return launch_with(kernel, grid, threads, ptrs, stream);
}

// In place, or apart (rows of a result that overlap each other are the caller's to avoid, as in the other entry points).
inline bool item_ok(const tmac_rope_item& it) {
  if (it.H <= 0 || it.reserved || !attn::rows_ok(&it.x, false, true, true) || !attn::rows_ok(&it.out, false, true, true)) return false;
  return it.x.data != it.out.data || (it.x.token == it.out.token && it.x.head == it.out.head);
}

inline bool pages_ok(const tmac_pages* p) {
  return p && p->pages >= 0 && p->page >= BT && p->page <= 4096 && (p->page & (p->page - 1)) == 0 && p->Hkv > 0 && p->D > 0 && p->D % 4 == 0 &&
         (p->code == TMAC_CODE_I8 || p->code == TMAC_CODE_E4M3) && !p->reserved[0] && !p->reserved[1] && !p->reserved[2];
}
inline bool pages_set(const tmac_pages* p) {
  return p->pages == 0 || (p->codes_dev && (reinterpret_cast<uintptr_t>(p->codes_dev) & 15) == 0 && p->scales_dev &&
                           (reinterpret_cast<uintptr_t>(p->scales_dev) & 7) == 0);
}
constexpr int64_t MOST_UNITS = (int64_t)1 << 40;
// (more than MOST_UNITS where there are: the product of all three may pass 64 bits)
inline int64_t units_of(const tmac_pages* p) {
  const int64_t heads = (int64_t)p->pages * p->Hkv;
  return heads > MOST_UNITS ? heads : heads * (p->page / BT);
}
inline int chunks_of(const tmac_pages* p) { return (p->D + 15) / 16; }

inline bool batch_ok(const tmac_pages_batch* b) {
  return b && b->S >= 0 && b->T >= 0 && b->width >= 0 && b->most >= 0 && b->table_stride >= b->width && (b->cu_dev || b->T == b->S);
}
inline bool batch_set(const tmac_pages_batch* b) { return (b->table_dev || b->width == 0) && b->lens_dev; }
inline bool supported(const tmac_pages* p, const tmac_pages_batch* b) {
  return p->D <= 128 && !attn::long_axis(b->S) && !attn::long_axis(b->T) && !attn::long_axis((int64_t)b->width * p->page) &&
         units_of(p) <= MOST_UNITS;
}

inline Pages view_of(const tmac_pages* p) {
  int shift = 0;
  while (BT << shift < p->page) ++shift;
  return Pages{static_cast<char*>(p->codes_dev), p->scales_dev, p->pages, shift, p->Hkv, p->D, chunks_of(p)};
}
inline Batch view_of(const tmac_pages_batch* b) {
  return Batch{b->table_dev, b->lens_dev, b->cu_dev, b->table_stride, b->S, b->width, b->T, !b->cu_dev ? 1 : b->most ? std::min(b->most, b->T) : b->T};
}

// Workgroups (a key head) for the blocks that the rows of a call touch: as many for every sequence as the longest can have, or, where that is
// fewer, n / 32 + 2 for each by the starts (slots 0).
inline int64_t block_slots(const tmac_pages_batch* b, int& slots) {
  const int most = view_of(b).most;
  slots = (int)(((int64_t)most + BT - 2) / BT + 1);
  const int64_t alike = (int64_t)b->S * slots, packed = b->T / BT + 2 * (int64_t)b->S;
  if (!b->cu_dev || alike <= packed) return alike;
  slots = 0;
  return packed;
}

}  // namespace pages
}  // namespace tmac
#endif
