// C ABI of rotary positions: argument validation, frequencies, and launches on the caller's stream.
#include <cmath>

#include "rotary_checks.h"

using lvspec::hip_fail;

extern "C" {

int lvspec_rotary(const lvspec_rotary_args* a, void* stream) {
  if (a == nullptr) return LVSPEC_EINVAL;
  if (a->n_rows < 0 || a->Hq < 1 || a->Hkv < 0 || a->D < 1 || a->dtype < LVSPEC_BF16 || a->dtype > LVSPEC_F32)
    return LVSPEC_EINVAL;
  lvspec::RotaryCallArgs k{};
  int rc = fill_rotation(a->rot, a->D, k.rot);
  if (rc != LVSPEC_OK) return rc;
  if (a->D > 512 || (int64_t)a->Hq + a->Hkv > 65535 || (int64_t)a->n_rows * a->D > (int64_t)1 << 32)
    return LVSPEC_EUNSUPPORTED;
  if (a->n_rows == 0) return LVSPEC_OK;
  if (!a->rot.pos) return LVSPEC_EINVAL;
  rc = fill_rows(a->Hq, a->D, a->dtype, a->q, a->q_sr, a->q_sh, a->q_out, a->qo_sr, a->qo_sh, k.q);
  if (rc == LVSPEC_OK && a->Hkv > 0)
    rc = fill_rows(a->Hkv, a->D, a->dtype, a->k, a->k_sr, a->k_sh, a->k_out, a->ko_sr, a->ko_sh, k.k);
  if (rc != LVSPEC_OK) return rc;
  k.n_rows = a->n_rows; k.D = a->D;
  k.in_place = a->q == a->q_out && (a->Hkv == 0 || a->k == a->k_out);
  const hipError_t e = lvspec::launch_rotary(k, a->dtype, static_cast<hipStream_t>(stream));
  return e == hipSuccess ? LVSPEC_OK : hip_fail(e);
}

int lvspec_rotary_frequencies(const lvspec_rotary_freq_args* a, float* inv_freq, float* factor) {
  if (a == nullptr || inv_freq == nullptr || factor == nullptr) return LVSPEC_EINVAL;
  if (a->dim < 2 || a->dim > 512 || a->dim % 2 != 0 || !(a->base > 1.0) || !std::isfinite(a->base)) return LVSPEC_EINVAL;
  if (a->scaling < LVSPEC_SCALING_NONE || a->scaling > LVSPEC_SCALING_YARN) return LVSPEC_EINVAL;
  if (a->scaling != LVSPEC_SCALING_NONE && (!(a->scale > 0.0) || !std::isfinite(a->scale))) return LVSPEC_EINVAL;
  if (a->scaling == LVSPEC_SCALING_NTK && a->dim == 2) return LVSPEC_EINVAL;
  const double dim = a->dim;
  double base = a->base, low = 0.0, high = 0.0;
  if (a->scaling == LVSPEC_SCALING_NTK) base *= std::pow(a->scale, dim / (dim - 2.0));
  *factor = 1.f;
  if (a->scaling == LVSPEC_SCALING_YARN) {
    const double fast = a->beta_fast == 0.0 ? 32.0 : a->beta_fast, slow = a->beta_slow == 0.0 ? 1.0 : a->beta_slow;
    if (!(a->original_len > 0.0) || !std::isfinite(a->original_len) || !(slow > 0.0) || !(fast >= slow) || !std::isfinite(fast))
      return LVSPEC_EINVAL;
    // the frequency (a real number) that turns so many times: base^(-2 i / dim) original_len = 2 pi times
    auto turns = [&](double times) { return dim * std::log(a->original_len / (2.0 * M_PI * times)) / (2.0 * std::log(base)); };
    low = std::fmax(std::floor(turns(fast)), 0.0);
    high = std::fmin(std::ceil(turns(slow)), dim - 1.0);
    if (a->scale > 1.0) *factor = (float)(0.1 * std::log(a->scale) + 1.0);
  }
  for (int i = 0; i < a->dim / 2; ++i) {
    double f = std::pow(base, -2.0 * i / dim);
    if (a->scaling == LVSPEC_SCALING_LINEAR) f /= a->scale;
    if (a->scaling == LVSPEC_SCALING_YARN) {
      // (ends that meet: a step)
      const double r = high > low ? std::fmin(std::fmax((i - low) / (high - low), 0.0), 1.0) : i > low ? 1.0 : 0.0;
      f = f * (1.0 - r) + f / a->scale * r;
    }
    inv_freq[i] = (float)f;
  }
  return LVSPEC_OK;
}

int lvspec_paged_append_rotary(const lvspec_paged_append_rotary_args* a, void* stream) {
  if (a == nullptr) return LVSPEC_EINVAL;
  lvspec::AppendKernelArgs rows{};
  int rc = fill_append(&a->rows, rows);
  if (rc != LVSPEC_OK) return rc;
  lvspec::AppendRotaryKernelArgs k{};
  rc = fill_append_rotation(a, rows, k);
  if (rc != LVSPEC_OK || rows.n_rows == 0) return rc;
  const hipError_t e = lvspec::launch_paged_append_rotary(k, false, static_cast<hipStream_t>(stream));
  return e == hipSuccess ? LVSPEC_OK : hip_fail(e);
}

}  // extern "C"
