// C ABI of the paged cache in 4 bits: argument validation and launches on the caller's stream.
#include "rotary_checks.h"

using lvspec::hip_fail;

extern "C" {

int lvspec_paged_mx_append(const lvspec_paged_mx_append_args* a, void* stream) {
  lvspec::AppendKernelArgs rows{};
  int rc = fill_append(a, rows);
  if (rc != LVSPEC_OK) return rc;
  hipError_t e;
  if (a->rot.dim != 0) {
    lvspec::AppendRotaryKernelArgs k{};
    rc = fill_append_rotation(a, rows, k);
    if (rc != LVSPEC_OK || rows.n_rows == 0) return rc;
    e = lvspec::launch_paged_append_rotary(k, true, static_cast<hipStream_t>(stream));
  } else {
    if (a->Hq != 0) return LVSPEC_EINVAL;
    if (rows.n_rows == 0) return LVSPEC_OK;
    e = lvspec::launch_paged_mx_append(rows, static_cast<hipStream_t>(stream));
  }
  return e == hipSuccess ? LVSPEC_OK : hip_fail(e);
}

int lvspec_paged_mx_read(const lvspec_paged_mx_read_args* a, void* stream) {
  if (a == nullptr) return LVSPEC_EINVAL;
  int rc = check_cache(&a->cache);
  if (rc != LVSPEC_OK) return rc;
  const lvspec_paged_mx_cache& c = a->cache;
  if (a->n_rows < 0) return LVSPEC_EINVAL;
  if (a->n_rows > (1 << 28)) return LVSPEC_EUNSUPPORTED;
  rc = check_cache_pointers(&c);
  if (rc != LVSPEC_OK) return rc;
  if (a->n_rows > 0 && (!a->slots || !a->k || !a->v)) return LVSPEC_EINVAL;
  const int64_t s[] = {a->k_sr, a->k_sh, a->v_sr, a->v_sh};
  for (int64_t v : s)
    if (!stride_ok(v) || v < c.D) return LVSPEC_EINVAL;
  if (!aligned(a->k, 16) || !aligned(a->v, 16)) return LVSPEC_EINVAL;
  if (a->n_rows == 0) return LVSPEC_OK;
  lvspec::ReadKernelArgs k{};
  k.k4 = static_cast<const uint8_t*>(c.k_pool); k.v4 = static_cast<const uint8_t*>(c.v_pool);
  k.k_scale = c.k_scale; k.v_scale = c.v_scale;
  k.k_tail = static_cast<const uint8_t*>(c.k_tail); k.v_tail = static_cast<const uint8_t*>(c.v_tail);
  k.slots = a->slots;
  k.k = static_cast<uint8_t*>(a->k); k.v = static_cast<uint8_t*>(a->v);
  k.k_sr = a->k_sr * 2; k.k_sh = a->k_sh * 2; k.v_sr = a->v_sr * 2; k.v_sh = a->v_sh * 2;
  k.n_rows = a->n_rows; k.B = c.B; k.Hkv = c.Hkv; k.n_blocks = c.n_blocks;
  const hipError_t e = lvspec::launch_paged_mx_read(k, static_cast<hipStream_t>(stream));
  return e == hipSuccess ? LVSPEC_OK : hip_fail(e);
}

size_t lvspec_verify_attn_paged_mx_workspace(const lvspec_paged_mx_attn_args* args) {
  PagedPlan pl;
  return plan_paged_attn(args, &pl) == LVSPEC_OK ? pl.ws_bytes : 0;
}

int lvspec_verify_attn_paged_mx(const lvspec_paged_mx_attn_args* a, void* stream) {
  lvspec::PagedAttnKernelArgs k{};
  const int rc = fill_attn(a, k);
  if (rc != LVSPEC_OK) return rc;
  const hipError_t e = lvspec::launch_paged_mx_attn(k, static_cast<hipStream_t>(stream));
  return e == hipSuccess ? LVSPEC_OK : hip_fail(e);
}

int lvspec_paged_mx_commit(const lvspec_paged_mx_commit_args* a, void* stream) {
  lvspec::PagedCommitKernelArgs k{};
  const int rc = fill_commit(a, k);
  if (rc != LVSPEC_OK) return rc;
  const hipError_t e = lvspec::launch_paged_mx_commit(k, static_cast<hipStream_t>(stream));
  return e == hipSuccess ? LVSPEC_OK : hip_fail(e);
}

}  // extern "C"
