// Argument checks of the calls on paged caches, in 8 and in 4 bits (the two structures name their fields alike), and
// the kernels' arguments from the caller's.
#pragma once

#include <hip/hip_runtime.h>

#include <algorithm>

#include "../../include/lvspec.h"
#include "lvspec_kernels.h"

namespace {

inline bool aligned(const void* p, uintptr_t n) { return (reinterpret_cast<uintptr_t>(p) & (n - 1)) == 0; }
inline bool stride_ok(int64_t s) { return s >= 0 && s % 8 == 0; }

template <class Cache>
int check_cache(const Cache* c) {
  if (c->B < 1 || c->Hkv < 1 || c->D < 1 || c->n_blocks < 1) return LVSPEC_EINVAL;
  if (c->D != LVSPEC_HEAD_DIM) return LVSPEC_EUNSUPPORTED;
  if (c->B > LVSPEC_PAGED_MAX_B || c->Hkv > 4096 || c->n_blocks > LVSPEC_PAGED_MAX_BLOCKS) return LVSPEC_EUNSUPPORTED;
  return LVSPEC_OK;
}

template <class Cache>
int check_cache_pointers(const Cache* c) {
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

template <class Args>
int plan_paged_attn(const Args* a, PagedPlan* pl) {
  if (a == nullptr) return LVSPEC_EINVAL;
  const int rc = check_cache(&a->cache);
  if (rc != LVSPEC_OK) return rc;
  const auto& c = a->cache;
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

template <class Args>
int fill_append(const Args* a, lvspec::AppendKernelArgs& k) {
  if (a == nullptr) return LVSPEC_EINVAL;
  int rc = check_cache(&a->cache);
  if (rc != LVSPEC_OK) return rc;
  const auto& c = a->cache;
  if (a->n_rows < 0) return LVSPEC_EINVAL;
  if (a->n_rows > (1 << 28)) return LVSPEC_EUNSUPPORTED;
  rc = check_cache_pointers(&c);
  if (rc != LVSPEC_OK) return rc;
  if (!a->cu_rows || (a->n_rows > 0 && (!a->k || !a->v || !a->slots || !a->row_seq || !a->row_pos)))
    return LVSPEC_EINVAL;
  if (!aligned(a->k, 16) || !aligned(a->v, 16) || !stride_ok(a->k_sr) || !stride_ok(a->k_sh) || !stride_ok(a->v_sr) ||
      !stride_ok(a->v_sh) || a->k_sr < c.D || a->v_sr < c.D || a->k_sh < c.D || a->v_sh < c.D)
    return LVSPEC_EINVAL;
  k.k = static_cast<const uint8_t*>(a->k); k.v = static_cast<const uint8_t*>(a->v);
  k.k_sr = a->k_sr * 2; k.k_sh = a->k_sh * 2; k.v_sr = a->v_sr * 2; k.v_sh = a->v_sh * 2;
  k.slots = a->slots; k.row_seq = a->row_seq; k.row_pos = a->row_pos; k.cu_rows = a->cu_rows;
  k.k8 = static_cast<uint8_t*>(c.k_pool); k.v8 = static_cast<uint8_t*>(c.v_pool);
  k.k_scale = c.k_scale; k.v_scale = c.v_scale;
  k.k_tail = static_cast<uint8_t*>(c.k_tail); k.v_tail = static_cast<uint8_t*>(c.v_tail);
  k.n_rows = a->n_rows; k.B = c.B; k.Hkv = c.Hkv; k.n_blocks = c.n_blocks;
  return LVSPEC_OK;
}

template <class Args>
int fill_attn(const Args* a, lvspec::PagedAttnKernelArgs& k) {
  PagedPlan pl;
  int rc = plan_paged_attn(a, &pl);
  if (rc != LVSPEC_OK) return rc;
  const auto& c = a->cache;
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
  return LVSPEC_OK;
}

template <class Args>
int fill_commit(const Args* a, lvspec::PagedCommitKernelArgs& k) {
  if (a == nullptr) return LVSPEC_EINVAL;
  int rc = check_cache(&a->cache);
  if (rc != LVSPEC_OK) return rc;
  const auto& c = a->cache;
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
  k.k8 = static_cast<uint8_t*>(c.k_pool); k.v8 = static_cast<uint8_t*>(c.v_pool);
  k.k_scale = c.k_scale; k.v_scale = c.v_scale;
  k.k_tail = static_cast<uint8_t*>(c.k_tail); k.v_tail = static_cast<uint8_t*>(c.v_tail);
  k.table = a->table; k.kv_len = a->kv_len; k.accept_len = a->accept_len;
  k.best_branch = nbr > 1 ? a->best_branch : nullptr;
  k.granted = a->granted; k.held = a->held; k.cu_rows = a->cu_rows;
  k.new_len = a->new_len;
  k.B = c.B; k.Hkv = c.Hkv; k.n_layers = a->n_layers; k.n_branches = nbr; k.chain_len = a->chain_len;
  k.n_blocks = c.n_blocks; k.cols = a->table_cols;
  return LVSPEC_OK;
}

}  // namespace
