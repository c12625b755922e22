// view.h -- host checks of the tensors [rows][heads][head_dim] that the attention and rotation calls take.
#pragma once

#include <cstdint>

#include "attn.h"
#include "dsv.h"

namespace dsv {

constexpr int64_t kMaxRowStride = 1 << 23, kMaxHeadStride = (int64_t)1 << 40;

// The view with dense strides filled in; out: its vectors must be apart.
inline int view(const dsv_attn_view* v, int64_t rows, int32_t heads, int32_t d, bool out, AttnView* to) {
  if (!v) return DSV_ERR_ARG;
  to->ptr = v->ptr;
  to->row = v->row == 0 ? (int64_t)heads * d : v->row;
  to->head = v->head == 0 ? d : v->head;
  if (reinterpret_cast<uintptr_t>(v->ptr) & 15) return DSV_ERR_ARG;
  if (rows > 0 && !v->ptr) return DSV_ERR_ARG;
  if (to->row < d || to->head < d || (to->row & 7) || (to->head & 7) || to->row > kMaxRowStride ||
      to->head > kMaxHeadStride)
    return DSV_ERR_SIZE;
  if (out && rows > 0 && to->row < (heads - 1) * to->head + d && to->head < (rows - 1) * to->row + d) return DSV_ERR_SIZE;
  return DSV_OK;
}

}  // namespace dsv
