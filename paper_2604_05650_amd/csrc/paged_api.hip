// C ABI of the paged cache in 8 bits: argument validation and launches on the caller's stream.
#include <hip/hip_runtime.h>

#include <algorithm>

#include "../../include/lvspec.h"
#include "lvspec_kernels.h"

namespace {

using lvspec::hip_fail;

bool aligned(const void* p, uintptr_t n) { return (reinterpret_cast<uintptr_t>(p) & (n - 1)) == 0; }
bool stride_ok(int64_t s) { return s >= 0 && s % 8 == 0; }

int check_cache(const lvspec_paged_cache* c) {
  if (c->B < 1 || c->Hkv < 1 || c->D < 1 || c->n_blocks < 1) return LVSPEC_EINVAL;
  if (c->D != LVSPEC_HEAD_DIM) return LVSPEC_EUNSUPPORTED;
  if (c->B > LVSPEC_PAGED_MAX_B || c->Hkv > 4096 || c->n_blocks > LVSPEC_PAGED_MAX_BLOCKS) return LVSPEC_EUNSUPPORTED;
  return LVSPEC_OK;
}

int check_cache_pointers(const lvspec_paged_cache* c) {
  const void* p[] = {c->k_pool, c->v_pool, c->k_tail, c->v_tail};
  for (const void* x : p)
    if (x == nullptr || !aligned(x, 16)) return LVSPEC_EINVAL;
  if (!c->k_scale || !c->v_scale || !aligned(c->k_scale, 4) || !aligned(c->v_scale, 4)) return LVSPEC_EINVAL;
  return LVSPEC_OK;
}

struct PagedPlan {
  int G, R, n_rc, rpad, limit, spare;
  size_t ws_bytes;
};

int plan_paged_attn(const lvspec_paged_attn_args* a, PagedPlan* pl) {
  if (a == nullptr) return LVSPEC_EINVAL;
  const int rc = check_cache(&a->cache);
  if (rc != LVSPEC_OK) return rc;
  const lvspec_paged_cache& c = a->cache;
  if (a->gamma < 1 || a->gamma > LVSPEC_MAX_DRAFT_ROWS || a->Hq < 1 || a->Hq % c.Hkv != 0 || a->table_cols < 0)
    return LVSPEC_EINVAL;
  if (!(a->scale >= 0.f) || a->scale > 1.0e6f) return LVSPEC_EINVAL;
  if (a->Hq > 65536 || a->table_cols > LVSPEC_PAGED_MAX_BLOCKS) return LVSPEC_EUNSUPPORTED;
  pl->G = a->Hq / c.Hkv;
  pl->R = pl->G * a->gamma;
  pl->n_rc = (pl->R + 31) / 32;
  pl->rpad = ((pl->R + pl->n_rc - 1) / pl->n_rc + 3) / 4 * 4;
  // places of all units (eight for open rows each), parts and output rows are 32-bit numbers in the kernels, and
  // so are the threads of a launch
  const int64_t units = (int64_t)c.B * c.Hkv * pl->n_rc;
  if (units > 1 << 21 || units * ((int64_t)a->table_cols + 8) > (int64_t)1 << 30 || (int64_t)c.B * c.Hkv * pl->R > (int64_t)1 << 30)
    return LVSPEC_EUNSUPPORTED;
  const int cus = lvspec::num_compute_units();
  pl->limit = (int)units + cus - 1;
  pl->spare = pl->limit - std::max((int)units, cus);
  pl->ws_bytes = (size_t)pl->limit * pl->rpad * 131 * sizeof(float) + (size_t)units * 8;
  return LVSPEC_OK;
}

}  // namespace

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
  if (a == nullptr) return LVSPEC_EINVAL;
  int rc = check_cache(&a->cache);
  if (rc != LVSPEC_OK) return rc;
  const lvspec_paged_cache& c = a->cache;
  if (a->n_rows < 0) return LVSPEC_EINVAL;
  if (a->n_rows > (1 << 28)) return LVSPEC_EUNSUPPORTED;
  rc = check_cache_pointers(&c);
  if (rc != LVSPEC_OK) return rc;
  if (!a->cu_rows || (a->n_rows > 0 && (!a->k || !a->v || !a->slots || !a->row_seq || !a->row_pos)))
    return LVSPEC_EINVAL;
  if (!aligned(a->k, 16) || !aligned(a->v, 16) || !stride_ok(a->k_sr) || !stride_ok(a->k_sh) || !stride_ok(a->v_sr) ||
      !stride_ok(a->v_sh) || a->k_sr < c.D || a->v_sr < c.D || a->k_sh < c.D || a->v_sh < c.D)
    return LVSPEC_EINVAL;
  if (a->n_rows == 0) return LVSPEC_OK;
  lvspec::AppendKernelArgs k{};
  k.k = static_cast<const uint8_t*>(a->k); k.v = static_cast<const uint8_t*>(a->v);
  k.k_sr = a->k_sr * 2; k.k_sh = a->k_sh * 2; k.v_sr = a->v_sr * 2; k.v_sh = a->v_sh * 2;
  k.slots = a->slots; k.row_seq = a->row_seq; k.row_pos = a->row_pos; k.cu_rows = a->cu_rows;
  k.k8 = static_cast<uint8_t*>(c.k_pool); k.v8 = static_cast<uint8_t*>(c.v_pool);
  k.k_scale = c.k_scale; k.v_scale = c.v_scale;
  k.k_tail = static_cast<uint8_t*>(c.k_tail); k.v_tail = static_cast<uint8_t*>(c.v_tail);
  k.n_rows = a->n_rows; k.B = c.B; k.Hkv = c.Hkv; k.n_blocks = c.n_blocks;
  const hipError_t e = lvspec::launch_paged_append(k, static_cast<hipStream_t>(stream));
  return e == hipSuccess ? LVSPEC_OK : hip_fail(e);
}

size_t lvspec_verify_attn_paged_workspace(const lvspec_paged_attn_args* args) {
  PagedPlan pl;
  return plan_paged_attn(args, &pl) == LVSPEC_OK ? pl.ws_bytes : 0;
}

int lvspec_verify_attn_paged(const lvspec_paged_attn_args* a, void* stream) {
  PagedPlan pl;
  int rc = plan_paged_attn(a, &pl);
  if (rc != LVSPEC_OK) return rc;
  const lvspec_paged_cache& c = a->cache;
  rc = check_cache_pointers(&c);
  if (rc != LVSPEC_OK) return rc;
  if (!a->q || !a->out || !a->kv_len || (a->table_cols > 0 && !a->table)) return LVSPEC_EINVAL;
  if (!aligned(a->q, 16) || !aligned(a->out, 16)) return LVSPEC_EINVAL;
  if (!stride_ok(a->q_sb) || !stride_ok(a->q_sg) || !stride_ok(a->q_sh) || !stride_ok(a->o_sb) ||
      !stride_ok(a->o_sg) || !stride_ok(a->o_sh) || a->q_sh < c.D || a->o_sh < c.D)
    return LVSPEC_EINVAL;
  if ((a->vis_begin == nullptr) != (a->vis_end == nullptr)) return LVSPEC_EINVAL;
  if (a->vis_mass != nullptr && a->vis_begin == nullptr) return LVSPEC_EINVAL;
  if (a->draft_mask != nullptr) {
    for (int i = 0; i < a->gamma; ++i) {
      if (!((a->draft_mask[i] >> i) & 1u)) return LVSPEC_EINVAL;   // a row always sees itself
      if (a->gamma < 32 && (a->draft_mask[i] >> a->gamma) != 0u) return LVSPEC_EINVAL;
    }
  }
  if (a->workspace == nullptr || !aligned(a->workspace, 256) || a->workspace_bytes < pl.ws_bytes)
    return LVSPEC_EWORKSPACE;
  lvspec::PagedAttnKernelArgs k{};
  k.q = static_cast<const uint16_t*>(a->q);
  k.q_sb = a->q_sb; k.q_sg = a->q_sg; k.q_sh = a->q_sh;
  k.k8 = static_cast<const uint8_t*>(c.k_pool); k.v8 = static_cast<const uint8_t*>(c.v_pool);
  k.k_scale = c.k_scale; k.v_scale = c.v_scale;
  k.k_tail = static_cast<const uint8_t*>(c.k_tail); k.v_tail = static_cast<const uint8_t*>(c.v_tail);
  k.table = a->table; k.kv_len = a->kv_len;
  k.B = c.B; k.gamma = a->gamma; k.Hq = a->Hq; k.Hkv = c.Hkv; k.G = pl.G; k.R = pl.R;
  k.div_g = lvspec::make_fast_div((uint32_t)pl.G);
  k.rpad = pl.rpad; k.n_rc = pl.n_rc; k.n_blocks = c.n_blocks; k.cols = a->table_cols; k.limit = pl.limit; k.spare = pl.spare;
  const float scale = a->scale > 0.f ? a->scale : 1.0f / __builtin_sqrtf((float)c.D);
  k.scale_log2e = scale * 1.4426950408889634f;
  k.vis_begin = a->vis_begin; k.vis_end = a->vis_end;
  k.out = static_cast<uint16_t*>(a->out);
  k.o_sb = a->o_sb; k.o_sg = a->o_sg; k.o_sh = a->o_sh;
  k.lse = a->lse; k.vis_mass = a->vis_mass;
  k.ws = static_cast<float*>(a->workspace);
  for (int i = 0; i < 32; ++i)
    k.draft_mask[i] = a->draft_mask ? (i < a->gamma ? a->draft_mask[i] : 0u) : (0xffffffffu >> (31 - i));
  const hipError_t e = lvspec::launch_paged_attn(k, static_cast<hipStream_t>(stream));
  return e == hipSuccess ? LVSPEC_OK : hip_fail(e);
}

int lvspec_paged_commit(const lvspec_paged_commit_args* a, void* stream) {
  if (a == nullptr) return LVSPEC_EINVAL;
  int rc = check_cache(&a->cache);
  if (rc != LVSPEC_OK) return rc;
  const lvspec_paged_cache& c = a->cache;
  const int nbr = a->n_branches > 1 ? a->n_branches : 1;
  if (a->n_layers < 1 || a->n_layers > 65535 || a->n_branches < 0 || a->n_branches > LVSPEC_MAX_BRANCHES ||
      a->chain_len < 1 || a->chain_len > LVSPEC_MAX_GAMMA || nbr * a->chain_len > LVSPEC_MAX_DRAFT_ROWS ||
      a->table_cols < 1)
    return LVSPEC_EINVAL;
  if (a->table_cols > LVSPEC_PAGED_MAX_BLOCKS) return LVSPEC_EUNSUPPORTED;
  rc = check_cache_pointers(&c);
  if (rc != LVSPEC_OK) return rc;
  if (!a->table || !a->kv_len || !a->accept_len || !a->new_len || a->new_len == a->kv_len) return LVSPEC_EINVAL;
  if ((a->granted == nullptr) != (a->held == nullptr) || (a->granted == nullptr) != (a->cu_rows == nullptr))
    return LVSPEC_EINVAL;
  lvspec::PagedCommitKernelArgs k{};
  k.k8 = static_cast<uint8_t*>(c.k_pool); k.v8 = static_cast<uint8_t*>(c.v_pool);
  k.k_scale = c.k_scale; k.v_scale = c.v_scale;
  k.k_tail = static_cast<uint8_t*>(c.k_tail); k.v_tail = static_cast<uint8_t*>(c.v_tail);
  k.table = a->table; k.kv_len = a->kv_len; k.accept_len = a->accept_len;
  k.best_branch = nbr > 1 ? a->best_branch : nullptr;
  k.granted = a->granted; k.held = a->held; k.cu_rows = a->cu_rows;
  k.new_len = a->new_len;
  k.B = c.B; k.Hkv = c.Hkv; k.n_layers = a->n_layers; k.n_branches = nbr; k.chain_len = a->chain_len;
  k.n_blocks = c.n_blocks; k.cols = a->table_cols;
  const hipError_t e = lvspec::launch_paged_commit(k, static_cast<hipStream_t>(stream));
  return e == hipSuccess ? LVSPEC_OK : hip_fail(e);
}

}  // extern "C"
