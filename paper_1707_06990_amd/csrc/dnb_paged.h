// The layout of a paged cache, for the kernels that read or write it (dnb_paged_attn.hip, dnb_qk.hip).
#pragma once

#include <stdint.h>

#include <utility>

#include "../../include/dnb.h"

namespace dnb {
namespace paged {

// Checks a layout and fills in its strides.
inline int check_layout(const dnb_paged_layout& in, dnb_paged_layout* out) {
  dnb_paged_layout c = in;
  if (c.pages < 0 || c.page_size < 1 || c.kv_heads < 1 || c.head_dim < 1 || c.sequences < 1 || c.max_pages < 1 ||
      (c.dtype != DNB_F32 && c.dtype != DNB_BF16) || c.page_stride < 0 || c.row_stride < 0 || c.head_stride < 0)
    return DNB_E_BADDESC;
  if ((c.page_size & (c.page_size - 1)) != 0 || c.page_size > 65536 || c.head_dim % 8 != 0 || c.head_dim > 128) return DNB_E_UNSUPPORTED;
  const int64_t most = 0x7fffffff;
  if (c.pages > most || c.kv_heads > 65536 || c.sequences > (1 << 20) || (int64_t)c.max_pages * c.page_size > most) return DNB_E_RANGE;
  if (c.head_stride == 0) c.head_stride = c.head_dim;
  if (c.row_stride == 0) c.row_stride = (int64_t)c.kv_heads * c.head_dim;
  if (c.page_stride == 0) c.page_stride = c.page_size * c.row_stride;
  const int vec = c.dtype == DNB_BF16 ? 8 : 4;
  // rows are read and written in 16-byte pieces
  for (const int64_t s : {c.page_stride, c.row_stride, c.head_stride})
    if (s % vec != 0 || s > (1 << 30)) return DNB_E_RANGE;
  if (c.row_stride < c.head_dim || c.head_stride < c.head_dim) return DNB_E_RANGE;
  // No two of (page, row, head) may share memory, in whichever order they lie: by stride, each is at least as long as all below it.
  struct Way {
    int64_t stride, count;
  } ways[3] = {{c.page_stride, c.pages}, {c.row_stride, c.page_size}, {c.head_stride, c.kv_heads}};
  for (const int i : {0, 1, 0})
    if (ways[i].stride > ways[i + 1].stride) std::swap(ways[i], ways[i + 1]);
  int64_t extent = c.head_dim;
  for (const Way& w : ways) {
    if (w.count <= 1) continue;
    if (w.stride < extent) return DNB_E_RANGE;
    extent += (w.count - 1) * w.stride;
  }
  *out = c;
  return DNB_OK;
}

inline int log2_of(int32_t page_size) {
  int s = 0;
  while ((1 << s) < page_size) ++s;
  return s;
}

}  // namespace paged
}  // namespace dnb
