// C ABI of the paged cache in 8 bits: argument validation and launches on the caller's stream.
#include "paged_checks.h"

using lvspec::hip_fail;

extern "C" {

int lvspec_paged_plan(const lvspec_paged_plan_args* a, void* stream) {
  if (a == nullptr) return LVSPEC_EINVAL;
  if (a->B < 1 || a->table_cols < 1 || a->n_blocks < 1 || a->max_rows < 0 || a->reserve < 0 ||
      (a->draft != 0 && a->draft != 1))
    return LVSPEC_EINVAL;
  if (a->B > LVSPEC_PAGED_MAX_B || a->n_blocks > LVSPEC_PAGED_MAX_BLOCKS || a->table_cols > LVSPEC_PAGED_MAX_BLOCKS ||
      a->max_rows > (1 << 28) || a->reserve > (1 << 20))
    return LVSPEC_EUNSUPPORTED;
  if (!a->kv_len || !a->n_new || !a->held || !a->state || !a->queue || !a->table || !a->granted || !a->new_held ||
      !a->new_state || !a->cu_rows || (a->max_rows > 0 && (!a->slots || !a->row_seq || !a->row_pos)))
    return LVSPEC_EINVAL;
  if (a->new_held == a->held || a->new_state == a->state) return LVSPEC_EINVAL;
  lvspec::PlanKernelArgs k{};
  k.kv_len = a->kv_len; k.n_new = a->n_new; k.held = a->held; k.state = a->state;
  k.queue = a->queue; k.table = a->table;
  k.granted = a->granted; k.new_held = a->new_held; k.new_state = a->new_state;
  k.cu_rows = a->cu_rows; k.slots = a->slots; k.row_seq = a->row_seq; k.row_pos = a->row_pos;
  k.B = a->B; k.cols = a->table_cols; k.n_blocks = a->n_blocks;
  k.max_rows = a->max_rows; k.reserve = a->reserve; k.draft = a->draft;
  const hipError_t e = lvspec::launch_paged_plan(k, static_cast<hipStream_t>(stream));
  return e == hipSuccess ? LVSPEC_OK : hip_fail(e);
}

int lvspec_paged_append(const lvspec_paged_append_args* a, void* stream) {
  lvspec::AppendKernelArgs k{};
  const int rc = fill_append(a, k);
  if (rc != LVSPEC_OK || k.n_rows == 0) return rc;
  const hipError_t e = lvspec::launch_paged_append(k, static_cast<hipStream_t>(stream));
  return e == hipSuccess ? LVSPEC_OK : hip_fail(e);
}

size_t lvspec_verify_attn_paged_workspace(const lvspec_paged_attn_args* args) {
  PagedPlan pl;
  return plan_paged_attn(args, &pl) == LVSPEC_OK ? pl.ws_bytes : 0;
}

int lvspec_verify_attn_paged(const lvspec_paged_attn_args* a, void* stream) {
  lvspec::PagedAttnKernelArgs k{};
  const int rc = fill_attn(a, k);
  if (rc != LVSPEC_OK) return rc;
  const hipError_t e = lvspec::launch_paged_attn(k, static_cast<hipStream_t>(stream));
  return e == hipSuccess ? LVSPEC_OK : hip_fail(e);
}

int lvspec_paged_commit(const lvspec_paged_commit_args* a, void* stream) {
  lvspec::PagedCommitKernelArgs k{};
  const int rc = fill_commit(a, k);
  if (rc != LVSPEC_OK) return rc;
  const hipError_t e = lvspec::launch_paged_commit(k, static_cast<hipStream_t>(stream));
  return e == hipSuccess ? LVSPEC_OK : hip_fail(e);
}

}  // extern "C"
