// New rows into the paged caches with the keys, and the queries beside them, rotated on the way.
//
// One launch in place of a rotation and an append: keys cross memory once.  Bound by memory where rows are many: into the cache
// in 8 bits 16384 rows of 8 heads take 27.0 us, 101 MB at 3.8 TB/s (20.3 without the rotation, whose sums and angles in 64 bits
// hide behind the loads in part: vector instructions take 47 % of the time), 12 x (300 to 9000) rows of 4 heads with 28 of
// queries 114 us, 535 MB at 4.7; into the one in 4 bits 12 x (300 to 9000) rows of 8 heads 52 us, 161 MB at 3.1.  By what
// follows what where they are few: 16 x 5 rows 7.1 us (4.3 without the rotation), 2048 rows into 4 bits 12: places,
// requests, rows and positions one behind the other, then 16 angles of a thread.  Where rows are many, two workgroups a
// compute unit are all that 213 (8 bits) and 219 (4 bits) registers leave room for, 64 of them the cosines and sines of a
// thread's two rows.
#include "paged_mx_store.h"
#include "rotary_dev.h"

namespace lvspec {

namespace {

// The packed rows of a tile and the blocks that end in it, as append_rows (paged_store.h) finds them for one head, with the
// requests' first rows asked for by all lanes at once.  Both go by RowPlace for which ring rows are left to who reads the
// request's open block (`later`), and write those behind its reads: a change to one is a change to both.
struct Tile {
  const AppendKernelArgs& a;
  const int t0, lane;
  const int seq;               // request of the lane's row
  const RowPlace row;
  int begin, end;              // its packed rows; begin < 0: none
  unsigned long long todo;     // last rows of blocks
  int my_tail;                 // the ring's row for the lane's, -1: not, or later

  LVS_DEV Tile(const AppendKernelArgs& args, int number)
      : a(args), t0(number * kPageTokens), lane(threadIdx.x & 63),
        seq(number * kPageTokens + lane < args.n_rows ? args.row_seq[number * kPageTokens + lane] : -1),
        row(args, number * kPageTokens + lane) {
    my_tail = row.to_tail && !row.later ? LVSPEC_SLOT_TAIL - row.slot : -1;
    const bool last = row.slot >= 0 && (row.slot & (kPageTokens - 1)) == kPageTokens - 1 &&
                      (row.slot >> kPageShift) < a.n_blocks;
    todo = __ballot(last);
    if (todo == 0ull) return;
    const bool ok = (uint32_t)seq < (uint32_t)a.B;
    begin = ok ? a.cu_rows[seq] : -1;
    end = ok ? a.cu_rows[seq + 1] : -1;
    end = end < a.n_rows ? end : a.n_rows;
    todo = __ballot(last && begin >= 0 && begin <= t0 + lane);
  }
  struct Block {
    int at, id, p0, b, begin, end, row0;     // last row; place in the pool; position of its first row; request; rows
  };
  LVS_DEV bool next(Block& x) {
    if (todo == 0ull) return false;
    const int l = __builtin_ctzll(todo);
    todo &= todo - 1;
    x.at = t0 + l;
    x.id = __builtin_amdgcn_readlane(row.slot, l) >> kPageShift;
    x.p0 = __builtin_amdgcn_readlane(row.pos, l) - (kPageTokens - 1);
    x.b = __builtin_amdgcn_readlane(seq, l);
    x.begin = __builtin_amdgcn_readlane(begin, l);
    x.end = __builtin_amdgcn_readlane(end, l);
    x.row0 = x.at - (kPageTokens - 1);
    return true;
  }
  // Ring rows of a block's request behind the block that are left to who reads its open rows: the first, and the i-th's
  // ring row.
  LVS_DEV int later_from(const Block& x) const { return max(x.at + 1, x.end - (kPageTokens - 1)); }
  LVS_DEV int later_code(const Block& x, int64_t t) const {
    const int s = t < x.end ? a.slots[t] : LVSPEC_SLOT_NONE;
    return s <= LVSPEC_SLOT_TAIL && (LVSPEC_SLOT_TAIL - s) / kTailRows == x.b ? LVSPEC_SLOT_TAIL - s : -1;
  }
};

// Values of a tile, heads first .. last-1, a head's rows asked for before the one before it is stored.
template <class Pool>
LVS_DEV void append_values(const AppendKernelArgs& a, typename Pool::Scratch& scratch, int number, int first, int last) {
  Tile tile(a, number);
  const int tid = threadIdx.x, q = tid >> 4, c = tid & 15;
  auto ring = [&](int b, int h) { return a.v_tail + ((int64_t)b * a.Hkv + h) * (kTailRows * kRowBytes); };
  auto to_ring = [&](int64_t t, int code) {
    for (int h = first; h < last; ++h)
      *reinterpret_cast<u32x4*>(ring(code / kTailRows, h) + code % kTailRows * kRowBytes + c * 16) =
          *reinterpret_cast<const u32x4*>(a.v + t * a.v_sr + h * a.v_sh + c * 16);
  };
  if (__ballot(tile.my_tail >= 0) != 0ull) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int code = __shfl(tile.my_tail, 16 * i + q, 64);
      if (code >= 0) to_ring(tile.t0 + 16 * i + q, code);
    }
  }
  Tile::Block x;
  while (tile.next(x)) {
    u32x4 v[4];
    auto load = [&](int h) {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int r = 4 * q + i;
        const uint8_t* from = x.row0 + r >= x.begin ? a.v + (int64_t)(x.row0 + r) * a.v_sr + h * a.v_sh
                                                    : ring(x.b, h) + ((x.p0 + r) & (kTailRows - 1)) * kRowBytes;
        v[i] = *reinterpret_cast<const u32x4*>(from + c * 16);
      }
    };
    load(first);
    for (int h = first; h < last; ++h) {
      const u32x4 now[4] = {v[0], v[1], v[2], v[3]};
      if (h + 1 < last) load(h + 1);
      const int64_t to = (int64_t)x.id * a.Hkv + h;
      if (Pool::store(now, true, a.v8, a.v_scale, to, scratch)) Pool::mend(a.v8, to);
    }
    if (x.row0 < x.begin)                                  // (the reads of the ring are behind a barrier)
      for (int64_t t = tile.later_from(x) + q; t < x.end; t += kCacheThreads / 16) {
        const int code = tile.later_code(x, t);
        if (code >= 0) to_ring(t, code);
      }
  }
}

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
    if (e.turned) turn[i].at(rot, t, e.f);
  }
  typedef Packed<__bf16, 8> Eight;
  LVS_DEV void take(Eight& u, Eight& v, const uint8_t* row) const {
    u.load(reinterpret_cast<const __bf16*>(row) + e.a);
    v.load(reinterpret_cast<const __bf16*>(row) + e.b);
  }
  LVS_DEV void rotate(Eight& u, Eight& v, int i) const {
    if (!e.turned) return;
    float x[8], y[8];
    u.get(x);
    v.get(y);
    turn[i].apply(x, y, rot.interleaved != 0);
    u.put(x);
    v.put(y);
  }
  LVS_DEV void put(const Eight& u, const Eight& v, uint8_t* row) const {
    u.store(reinterpret_cast<__bf16*>(row) + e.a);
    v.store(reinterpret_cast<__bf16*>(row) + e.b);
  }
  // packed rows t[i] to ring rows code[i] (-1: not), in all the heads; a head's rows are asked for before the one before
  // it, or the angles, are done
  LVS_DEV void to_ring(const int64_t (&t)[2], const int (&code)[2], int first, int last) {
    Eight u[2], v[2];
    auto load = [&](int h) {
#pragma unroll
      for (int i = 0; i < 2; ++i)
        if (code[i] >= 0) take(u[i], v[i], a.k + t[i] * a.k_sr + h * a.k_sh);
    };
    load(first);
#pragma unroll
    for (int i = 0; i < 2; ++i)
      if (code[i] >= 0) angles(i, t[i]);
    for (int h = first; h < last; ++h) {
      Eight x[2] = {u[0], u[1]}, y[2] = {v[0], v[1]};
      if (h + 1 < last) load(h + 1);
#pragma unroll
      for (int i = 0; i < 2; ++i)
        if (code[i] >= 0) {
          rotate(x[i], y[i], i);
          put(x[i], y[i], a.k_tail + (((int64_t)(code[i] / kTailRows) * a.Hkv + h) * kTailRows + code[i] % kTailRows) * kRowBytes);
        }
    }
  }
  LVS_DEV void tile(int number, int first, int last) {
    Tile tile(a, number);
    const int tid = threadIdx.x, q = tid >> 4, c = tid & 15;
    if (__ballot(tile.my_tail >= 0) != 0ull) {
      const int64_t at[2] = {tile.t0 + r, tile.t0 + r + 32};
      const int code[2] = {__shfl(tile.my_tail, r, 64), __shfl(tile.my_tail, r + 32, 64)};
      to_ring(at, code, first, last);
    }
    Tile::Block b;
    while (tile.next(b)) {
      Eight u[2], v[2];
      bool is_new[2];
      auto load = [&](int h) {
        const uint8_t* ring = a.k_tail + ((int64_t)b.b * a.Hkv + h) * (kTailRows * kRowBytes);
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          const int k = r + 32 * i;
          take(u[i], v[i], is_new[i] ? a.k + (int64_t)(b.row0 + k) * a.k_sr + h * a.k_sh
                                     : ring + ((b.p0 + k) & (kTailRows - 1)) * kRowBytes);
        }
      };
#pragma unroll
      for (int i = 0; i < 2; ++i) is_new[i] = b.row0 + r + 32 * i >= b.begin;
      load(first);
#pragma unroll
      for (int i = 0; i < 2; ++i)
        if (is_new[i]) angles(i, b.row0 + r + 32 * i);
      for (int h = first; h < last; ++h) {
        // (the rows of the head before this one have been read: there are barriers behind that in store)
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          if (is_new[i]) rotate(u[i], v[i], i);
          put(u[i], v[i], s_rows + (r + 32 * i) * kRowBytes);
        }
        if (h + 1 < last) load(h + 1);
        lds_barrier();
        u32x4 x[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) x[i] = *reinterpret_cast<const u32x4*>(s_rows + (4 * q + i) * kRowBytes + c * 16);
        const int64_t to = (int64_t)b.id * a.Hkv + h;
        if (Pool::store(x, false, a.k8, a.k_scale, to, scratch)) Pool::mend(a.k8, to);
      }
      if (b.row0 < b.begin) {                              // (the reads of the ring are behind a barrier)
        const int from = tile.later_from(b);
        const int64_t rows[2] = {from + r, from + r + 32};
        const int code[2] = {tile.later_code(b, rows[0]), tile.later_code(b, rows[1])};
        to_ring(rows, code, first, last);
      }
    }
  }
};

// Workgroups: keys, and values, by tile and group of heads, queries by 256 pieces and group of heads.
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
  if (w < tiles * a.v_groups) {
    const int group = w / tiles, first = group * a.v_heads;
    append_values<Pool>(a.rows, scratch, w - group * tiles, first, min(first + a.v_heads, a.rows.Hkv));
    return;
  }
  w -= tiles * a.v_groups;
  const int group = w / a.q_wgs;
  const int64_t i = (int64_t)(w - group * a.q_wgs) * kCacheThreads + threadIdx.x, t = i >> 3;
  if (t >= a.rows.n_rows || a.rows.row_seq[t] < 0) return;
  const Piece e = piece_of((int)i & 7, 8, a.rot.half, 128, a.rot.interleaved != 0);
  if (!e.turned && a.q.x == a.q.y) return;
  // (eight pairs, as keys: with four 12 x (300 to 9000) rows take 114.9 us, with eight 113.9, five drafts no less)
  Turn<8> turn;
  bool ready = false;
  rotate_heads<__bf16, 8>(a.q, a.rot, turn, ready, e, t, group * a.q_heads, min((group + 1) * a.q_heads, a.q.H));
}

template <class Pool>
hipError_t launch(AppendRotaryKernelArgs a, hipStream_t stream) {
  const int64_t tiles = (a.rows.n_rows + kPageTokens - 1) / kPageTokens, cus = num_compute_units();
  // Heads that share a row's angles: as many as leave a workgroup of keys for each compute unit.  16384 rows, 8 heads,
  // 256 tiles: one group 28.0 us, two 31.9, four 39.9.
  int64_t k_groups = (cus + tiles - 1) / tiles;
  k_groups = k_groups > a.rows.Hkv ? a.rows.Hkv : k_groups;
  a.k_heads = (int)((a.rows.Hkv + k_groups - 1) / k_groups);
  a.k_groups = (a.rows.Hkv + a.k_heads - 1) / a.k_heads;
  // Values have no angles to share, but two workgroups are all that a compute unit has room for: four heads.  16384 rows,
  // 8 heads eight 27.8 us, four 27.0, two 28.9, one 31.3; 12 x (300 to 9000) rows in 4 bits, read back too, eight 89.1,
  // four 81.1, two 80.1, one 85.4.
  a.v_heads = a.k_heads < 4 ? a.k_heads : 4;
  a.v_groups = (a.rows.Hkv + a.v_heads - 1) / a.v_heads;
  int64_t wgs = tiles * (a.k_groups + a.v_groups);
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
