// Argument checks of rotary positions, and the kernels' arguments from the caller's.
#pragma once

#include "paged_checks.h"

namespace {

inline int64_t per16(int dtype) { return dtype == LVSPEC_F32 ? 4 : 8; }      // values of 16 bytes

inline int fill_rotation(const lvspec_rotation& r, int D, lvspec::RotaryKernelArgs& k) {
  if (r.dim < 2 || r.dim % 2 != 0 || r.dim > D || r.n_axes < 1 || r.n_axes > 4 || (r.interleaved != 0 && r.interleaved != 1) ||
      (r.transpose != 0 && r.transpose != 1))
    return LVSPEC_EINVAL;
  if (!(r.factor >= 0.f) || r.factor > 1.0e6f || r.pos_sa < 0) return LVSPEC_EINVAL;
  if (!r.inv_freq || !aligned(r.inv_freq, 4) || !aligned(r.pos, 4)) return LVSPEC_EINVAL;
  k.inv_freq = r.inv_freq; k.axis = r.axis; k.pos = r.pos; k.pos_sa = r.pos_sa;
  k.half = r.dim / 2; k.interleaved = r.interleaved; k.n_axes = r.n_axes;
  k.factor = r.factor > 0.f ? r.factor : 1.f;
  k.sine = r.transpose ? -k.factor : k.factor;
  return LVSPEC_OK;
}

// [n_rows, H, D] in and out
inline int fill_rows(int H, int D, int dtype, const void* x, int64_t x_sr, int64_t x_sh, void* y, int64_t y_sr,
                     int64_t y_sh, lvspec::RotaryRows& k) {
  const int64_t n = per16(dtype), s[] = {x_sr, x_sh, y_sr, y_sh};
  if (!x || !y || !aligned(x, 16) || !aligned(y, 16)) return LVSPEC_EINVAL;
  for (int64_t v : s)
    if (v < D || v % n != 0) return LVSPEC_EINVAL;
  if (x == y && (x_sr != y_sr || x_sh != y_sh)) return LVSPEC_EINVAL;
  k.x = x; k.y = y; k.x_sr = x_sr; k.x_sh = x_sh; k.y_sr = y_sr; k.y_sh = y_sh;
  k.H = H;
  return LVSPEC_OK;
}

// Rotation and queries of an append.
template <class Args>
int fill_append_rotation(const Args* a, const lvspec::AppendKernelArgs& rows, lvspec::AppendRotaryKernelArgs& k) {
  int rc = fill_rotation(a->rot, LVSPEC_HEAD_DIM, k.rot);
  if (rc != LVSPEC_OK) return rc;
  const bool any = rows.n_rows > 0;          // (without rows there are no positions and no queries to point at)
  if (a->rot.transpose != 0 || a->Hq < 0 || (any && a->rot.pos == nullptr && a->rot.n_axes != 1)) return LVSPEC_EINVAL;
  if (a->rot.dim % 16 != 0 || a->Hq > 65535) return LVSPEC_EUNSUPPORTED;
  if (any && a->Hq > 0) {
    rc = fill_rows(a->Hq, LVSPEC_HEAD_DIM, LVSPEC_BF16, a->q, a->q_sr, a->q_sh, a->q_out, a->qo_sr, a->qo_sh, k.q);
    if (rc != LVSPEC_OK) return rc;
  }
  const int64_t tiles = ((int64_t)rows.n_rows + 63) / 64;
  if (tiles * 2 * rows.Hkv + tiles * 2 + a->Hq + 1024 > (1 << 24)) return LVSPEC_EUNSUPPORTED;
  k.rows = rows;
  if (k.rot.pos == nullptr) k.rot.pos = rows.row_pos;
  return LVSPEC_OK;
}

}  // namespace
