// New rows into the paged caches with the keys, and the queries beside them, rotated on the way.
#include "paged_mx_store.h"
#include "rotary_dev.h"

namespace lvspec {

namespace {

// Keys of a tile of 64 packed rows, heads first .. last-1.  Rotated rows are rounded to bf16, which is what the ring
// holds, and go there or through LDS into their block: so a row's codes do not depend on the call it came in.
// Thread (r, p) = (tid / 8, tid % 8) turns piece p, eight pairs, of rows r and r + 32; its cosines and sines serve all
// the heads.
template <class Pool>
struct RotatedKeys {
  const AppendKernelArgs& a;
  const RotaryKernelArgs& rot;
  typename Pool::Scratch& scratch;
  uint8_t* s_rows;         // [64][256]
  const int r, p;
  const Piece e;
  Turn<8> turn[2];

  LVS_DEV RotatedKeys(const AppendKernelArgs& args, const RotaryKernelArgs& ro, typename Pool::Scratch& s, uint8_t* rows)
      : a(args), rot(ro), scratch(s), s_rows(rows), r(threadIdx.x >> 3), p(threadIdx.x & 7),
        e(piece_of(threadIdx.x & 7, 8, ro.half, 128, ro.interleaved != 0)) {}

  LVS_DEV void angles(int i, int64_t t) {
    if (e.turned) turn[i].at(rot, t, 8 * p);
  }
  // the thread's piece of a row, rotated where it is new
  LVS_DEV void piece(Packed<__bf16, 8>& u, Packed<__bf16, 8>& v, int i, const uint8_t* row, bool is_new) const {
    u.load(reinterpret_cast<const __bf16*>(row) + e.a);
    v.load(reinterpret_cast<const __bf16*>(row) + e.b);
    if (!is_new || !e.turned) return;
    float x[8], y[8];
    u.get(x);
    v.get(y);
    turn[i].apply(x, y, rot.interleaved != 0);
    u.put(x);
    v.put(y);
  }
  LVS_DEV void put(const Packed<__bf16, 8>& u, const Packed<__bf16, 8>& v, uint8_t* row) const {
    u.store(reinterpret_cast<__bf16*>(row) + e.a);
    v.store(reinterpret_cast<__bf16*>(row) + e.b);
  }
  // packed rows t[i] to ring rows code[i] (-1: not), in all the heads
  LVS_DEV void to_ring(const int64_t (&t)[2], const int (&code)[2], int first, int last) {
#pragma unroll
    for (int i = 0; i < 2; ++i)
      if (code[i] >= 0) angles(i, t[i]);
    for (int h = first; h < last; ++h)
#pragma unroll
      for (int i = 0; i < 2; ++i)
        if (code[i] >= 0) {
          Packed<__bf16, 8> u, v;
          piece(u, v, i, a.k + t[i] * a.k_sr + h * a.k_sh, true);
          put(u, v, a.k_tail + (((int64_t)(code[i] / kTailRows) * a.Hkv + h) * kTailRows + code[i] % kTailRows) * kRowBytes);
        }
  }
  LVS_DEV void tile(int number, int first, int last) {
    const int tid = threadIdx.x, lane = tid & 63, q = tid >> 4, c = tid & 15;
    const int t0 = number * kPageTokens, t = t0 + lane;
    const RowPlace row(a, t);
    const int my_tail = row.to_tail && !row.later ? LVSPEC_SLOT_TAIL - row.slot : -1;
    if (__ballot(my_tail >= 0) != 0ull) {
      const int64_t at[2] = {t0 + r, t0 + r + 32};
      const int code[2] = {__shfl(my_tail, r, 64), __shfl(my_tail, r + 32, 64)};
      to_ring(at, code, first, last);
    }
    unsigned long long todo = __ballot(row.slot >= 0 && (row.slot & (kPageTokens - 1)) == kPageTokens - 1);
    while (todo != 0ull) {
      const int l = __builtin_ctzll(todo);
      todo &= todo - 1;
      const int at = t0 + l;                               // last row of the block
      const int id = __builtin_amdgcn_readlane(row.slot, l) >> kPageShift;
      const int p0 = __builtin_amdgcn_readlane(row.pos, l) - (kPageTokens - 1);
      const int b = a.row_seq[at];
      if (id >= a.n_blocks || (uint32_t)b >= (uint32_t)a.B) continue;
      const int begin = a.cu_rows[b];
      if (begin < 0 || begin > at) continue;
      const int row0 = at - (kPageTokens - 1);
      bool is_new[2];
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        is_new[i] = row0 + r + 32 * i >= begin;
        if (is_new[i]) angles(i, row0 + r + 32 * i);
      }
      for (int h = first; h < last; ++h) {
        const uint8_t* ring = a.k_tail + ((int64_t)b * a.Hkv + h) * (kTailRows * kRowBytes);
        Packed<__bf16, 8> u[2], v[2];
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          const int k = r + 32 * i;
          piece(u[i], v[i], i, is_new[i] ? a.k + (int64_t)(row0 + k) * a.k_sr + h * a.k_sh
                                         : ring + ((p0 + k) & (kTailRows - 1)) * kRowBytes, is_new[i]);
        }
        __syncthreads();                                   // (the rows of the head before this one have been read)
#pragma unroll
        for (int i = 0; i < 2; ++i) put(u[i], v[i], s_rows + (r + 32 * i) * kRowBytes);
        __syncthreads();
        u32x4 x[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) x[i] = *reinterpret_cast<const u32x4*>(s_rows + (4 * q + i) * kRowBytes + c * 16);
        const int64_t to = (int64_t)id * a.Hkv + h;
        if (Pool::store(x, false, a.k8, a.k_scale, to, scratch)) Pool::mend(a.k8, to);
      }
      if (row0 < begin) {                                  // (the reads of the ring are behind a barrier)
        int end = a.cu_rows[b + 1];
        end = end < a.n_rows ? end : a.n_rows;
        const int from = max(at + 1, end - (kPageTokens - 1));
        int64_t rows[2];
        int code[2];
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          rows[i] = from + r + 32 * i;
          const int s = rows[i] < end ? a.slots[rows[i]] : LVSPEC_SLOT_NONE;
          code[i] = s <= LVSPEC_SLOT_TAIL && (LVSPEC_SLOT_TAIL - s) / kTailRows == b ? LVSPEC_SLOT_TAIL - s : -1;
        }
        to_ring(rows, code, first, last);
      }
    }
  }
};

// Workgroups: keys by tile and group of heads, values by tile and head, queries by 256 pieces and group of heads.
template <class Pool>
__global__ __launch_bounds__(kCacheThreads) void paged_append_rotary_kernel(AppendRotaryKernelArgs a) {
  __shared__ typename Pool::Scratch scratch;
  __shared__ __align__(16) uint8_t s_rows[kPageTokens * kRowBytes];
  const int tiles = (a.rows.n_rows + kPageTokens - 1) / kPageTokens;
  int w = blockIdx.x;
  if (w < tiles * a.k_groups) {
    const int group = w / tiles, first = group * a.k_heads;
    RotatedKeys<Pool> keys(a.rows, a.rot, scratch, s_rows);
    keys.tile(w - group * tiles, first, min(first + a.k_heads, a.rows.Hkv));
    return;
  }
  w -= tiles * a.k_groups;
  if (w < tiles * a.rows.Hkv) {
    const int h = w / tiles;
    append_rows<Pool>(a.rows, scratch, w - h * tiles, h, true);
    return;
  }
  w -= tiles * a.rows.Hkv;
  const int group = w / a.q_wgs;
  const int64_t i = (int64_t)(w - group * a.q_wgs) * kCacheThreads + threadIdx.x, t = i >> 3;
  if (t >= a.rows.n_rows || a.rows.row_seq[t] < 0) return;
  const bool pairs = a.rot.interleaved != 0;
  const Piece e = piece_of((int)i & 7, 8, a.rot.half, 128, pairs);
  if (!e.turned && a.q.x == a.q.y) return;
  Turn<8> turn;
  if (e.turned) turn.at(a.rot, t, 8 * ((int)i & 7));
  rotate_heads<__bf16, 8>(a.q, turn, e, pairs, t, group * a.q_heads, min((group + 1) * a.q_heads, a.q.H));
}

template <class Pool>
hipError_t launch(AppendRotaryKernelArgs a, hipStream_t stream) {
  const int64_t tiles = (a.rows.n_rows + kPageTokens - 1) / kPageTokens, cus = num_compute_units();
  // keys: heads that share a row's angles, as many as leave two workgroups for a compute unit
  int64_t k_groups = (2 * cus + tiles - 1) / tiles;
  k_groups = k_groups > a.rows.Hkv ? a.rows.Hkv : k_groups;
  a.k_heads = (int)((a.rows.Hkv + k_groups - 1) / k_groups);
  a.k_groups = (a.rows.Hkv + a.k_heads - 1) / a.k_heads;
  int64_t wgs = tiles * (a.k_groups + a.rows.Hkv);
  if (a.q.H > 0) {
    const int64_t threads = (int64_t)a.rows.n_rows * 8;
    a.q_wgs = (int)((threads + kCacheThreads - 1) / kCacheThreads);
    int64_t groups = (kRotaryEnough + threads - 1) / threads;
    groups = groups > a.q.H ? a.q.H : groups;
    a.q_heads = (int)((a.q.H + groups - 1) / groups);
    groups = (a.q.H + a.q_heads - 1) / a.q_heads;
    wgs += a.q_wgs * groups;
  }
  paged_append_rotary_kernel<Pool><<<dim3((unsigned)wgs), dim3(kCacheThreads), 0, stream>>>(a);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_paged_append_rotary(const AppendRotaryKernelArgs& a, bool four, hipStream_t stream) {
  return four ? launch<Pool4>(a, stream) : launch<Pool8>(a, stream);
}

}  // namespace lvspec
