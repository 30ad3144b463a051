// Bookkeeping of the paged cache in 8 bits: block tables and slot maps from request lengths, new rows into
// the cache, and a verified step into the caches of all layers.
#include "paged_dev.h"

namespace lvspec {

namespace {

// ------------------------------------------------------------------------------ plan
// Which request gets which blocks is a pair of prefix sums over the requests (rows, blocks).  Every
// workgroup takes them by itself, 16 requests per thread at most, and then fills its share of the rows and
// of the table: one launch, no state changed in place, so that a second call on the same input gives the
// same answer.  Sums saturate just above what is compared with.
// Bound by latency: lengths, three sums one behind the other, a search for the row's request, the queue.  16
// requests with 5 drafts each 4.8 us, 64 prompts of 1000 to 16384 rows 9.0 us, of which the 4.2 MB written
// are 1.
constexpr int kPlanThreads = 256;
constexpr int kPlanMaxB = 4096;
constexpr int kPlanRows = 4;       // rows per thread and turn

struct PlanRequest {
  int len, rows, held, done, need;   // done: blocks that are complete behind the new rows; need: blocks wanted
};

LVS_DEV PlanRequest plan_request(const PlanKernelArgs& a, int b) {
  PlanRequest r;
  const int len = a.kv_len[b], rows = a.n_new[b], held = a.held[b];
  r.len = min(max(len, 0), 1 << 30);
  r.rows = min(max(rows, 0), a.max_rows + 1);
  r.held = min(max(held, 0), a.cols);
  r.done = (a.draft ? r.len : r.len + r.rows) >> kPageShift;
  r.need = len <= 0 && rows < 0 ? 0 : (r.len + r.rows + a.reserve) >> kPageShift;      // (finished: no reserve)
  return r;
}

// Sum over the threads before this one (returned) and over all of them (`all`) of x <= top, saturating at
// top; `part` is scratch of one value per wave.
LVS_DEV uint32_t sum_before(uint32_t x, uint32_t top, uint32_t* part, uint32_t& all) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    const uint32_t y = __shfl_up(x, d, 64);
    if (lane >= d) x = min(x + y, top);
  }
  __syncthreads();
  if (lane == 63) part[wave] = x;
  __syncthreads();
  uint32_t before = __shfl_up(x, 1, 64);
  before = lane == 0 ? 0u : before;
  all = 0;
#pragma unroll
  for (int w = 0; w < kPlanThreads / 64; ++w) {
    if (w < wave) before = min(before + part[w], top);
    all = min(all + part[w], top);
  }
  return before;
}

__global__ __launch_bounds__(kPlanThreads) void paged_plan_kernel(PlanKernelArgs a) {
  __shared__ int s_cu[kPlanMaxB + 1];       // first row of a request
  __shared__ int s_base[kPlanMaxB];         // its first block among those granted; -1: refused
  __shared__ int s_back[kPlanMaxB];         // first place of its surplus behind the queue's end
  __shared__ uint32_t s_part[kPlanThreads / 64];
  const int tid = threadIdx.x;
  const int per = (a.B + kPlanThreads - 1) / kPlanThreads;
  const int b0 = min(tid * per, a.B), b1 = min(b0 + per, a.B);
  const uint32_t row_top = (uint32_t)a.max_rows + 1, blk_top = (uint32_t)a.n_blocks + 1;
  int head = a.state[0] % a.n_blocks;
  head = head < 0 ? head + a.n_blocks : head;
  const int count = min(max(a.state[1], 0), a.n_blocks);

  uint32_t sum = 0, total, wanted, surplus;      // (wanted: only who fits is granted, see given)
  for (int b = b0; b < b1; ++b) sum = min(sum + (uint32_t)plan_request(a, b).rows, row_top);
  uint32_t at = sum_before(sum, row_top, s_part, total);
  total = min(total, (uint32_t)a.max_rows);
  uint32_t grow = 0, drop = 0;
  for (int b = b0; b < b1; ++b) {
    const PlanRequest r = plan_request(a, b);
    s_cu[b] = (int)min(at, (uint32_t)a.max_rows);
    at = min(at + (uint32_t)r.rows, row_top);
    // rows that fit the maps, a table that fits the sequence, open rows that fit the ring
    const bool may = r.need <= a.cols && (r.rows == 0 || at <= (uint32_t)a.max_rows) &&
                     r.len + r.rows - (r.done << kPageShift) <= kTailRows;
    s_base[b] = may ? 0 : -1;
    if (may) grow = min(grow + (uint32_t)max(r.need - r.held, 0), blk_top);
  }
  if (tid == 0) s_cu[a.B] = (int)total;
  at = sum_before(grow, blk_top, s_part, wanted);
  uint32_t given = 0;                       // blocks granted up to and with this thread's requests
  for (int b = b0; b < b1; ++b) {
    if (s_base[b] < 0) continue;
    const PlanRequest r = plan_request(a, b);
    const uint32_t want = (uint32_t)max(r.need - r.held, 0);
    const uint32_t end = min(at + want, blk_top);
    // first come, first served: who grows past the queue's count is refused, and so is everybody behind
    // them who grows
    if (want > 0 && end > (uint32_t)count) {
      s_base[b] = -1;
    } else {
      s_base[b] = (int)at;
      if (want > 0) given = max(given, end);
      drop = min(drop + (uint32_t)max(r.held - r.need, 0), blk_top);
    }
    at = end;
  }
  at = sum_before(drop, blk_top, s_part, surplus);
  for (int b = b0; b < b1; ++b) {
    s_back[b] = (int)at;
    if (s_base[b] < 0) continue;
    const PlanRequest r = plan_request(a, b);
    at = min(at + (uint32_t)max(r.held - r.need, 0), blk_top);
  }
  if (blockIdx.x == 0) {
    uint32_t all = wave_max_u32(given);
    __syncthreads();
    if ((tid & 63) == 0) s_part[tid >> 6] = all;
    __syncthreads();
    for (int w = 0; w < kPlanThreads / 64; ++w) all = max(all, s_part[w]);
    if (tid == 0) {
      const int left = count - (int)all;
      // (a queue that says it holds more than the pool has room for takes nothing back)
      a.new_state[0] = (int)(((uint32_t)head + all) % (uint32_t)a.n_blocks);
      a.new_state[1] = left + (int)min(surplus, (uint32_t)(a.n_blocks - count));
    }
    for (int b = b0; b < b1; ++b) {
      const PlanRequest r = plan_request(a, b);
      a.granted[b] = s_base[b] >= 0 ? 1 : 0;
      a.new_held[b] = s_base[b] >= 0 ? r.need : r.held;
      a.cu_rows[b] = s_cu[b];
    }
    if (tid == 0) a.cu_rows[a.B] = (int)total;
  }
  __syncthreads();

  // ---- table entries of the blocks to come, and surplus blocks back into the queue
  auto queued = [&](uint32_t i) { return a.queue[((uint32_t)head + i) % (uint32_t)a.n_blocks]; };
  for (int b = blockIdx.x; b < a.B; b += gridDim.x) {
    const int base = s_base[b];
    if (base < 0) continue;
    const PlanRequest r = plan_request(a, b);
    int32_t* row = a.table + (int64_t)b * a.cols;
    for (int i = r.held + tid; i < r.need; i += kPlanThreads) row[i] = queued((uint32_t)(base + i - r.held));
    for (int i = r.need + tid; i < r.held; i += kPlanThreads) {
      const int64_t to = (int64_t)count + s_back[b] + (i - r.need);
      if (to < a.n_blocks) a.queue[((int64_t)head + to) % a.n_blocks] = row[i];
    }
  }
  // ---- places of the rows
  for (int64_t t0 = (int64_t)blockIdx.x * (kPlanThreads * kPlanRows); t0 < a.max_rows;
       t0 += (int64_t)gridDim.x * (kPlanThreads * kPlanRows)) {
#pragma unroll
    for (int k = 0; k < kPlanRows; ++k) {
      const int64_t t = t0 + k * kPlanThreads + tid;
      if (t >= a.max_rows) break;
      int slot = LVSPEC_SLOT_NONE, seq = -1, pos = -1;
      if (t < (int64_t)total) {
        int lo = 0, hi = a.B - 1;            // the last request that starts at or before t
        while (lo < hi) {
          const int mid = (lo + hi + 1) >> 1;
          if (s_cu[mid] <= (int)t) lo = mid; else hi = mid - 1;
        }
        seq = lo;
        const PlanRequest r = plan_request(a, lo);
        pos = r.len + ((int)t - s_cu[lo]);
        const int base = s_base[lo], col = pos >> kPageShift;
        if (base >= 0) {
          if (col < r.done) {
            const int id = col < r.held ? a.table[(int64_t)lo * a.cols + col]
                                        : queued((uint32_t)(base + col - r.held));
            if ((uint32_t)id < (uint32_t)a.n_blocks) slot = id * kPageTokens + (pos & (kPageTokens - 1));
          } else {
            slot = LVSPEC_SLOT_TAIL - (lo * kTailRows + (pos & (kTailRows - 1)));
          }
        }
      }
      a.slots[t] = slot;
      a.row_seq[t] = seq;
      a.row_pos[t] = pos;
    }
  }
}

// ------------------------------------------------------------------------------ rounding to 8 bits
// A block of 64 rows x 128 bf16 in 256 threads: thread (q, c) = (tid / 16, tid % 16) holds the 16 bytes of
// chunk c of rows 4q .. 4q+3, so that four rows of one channel, a dword of the transposed block, are its own.
constexpr int kCacheThreads = 256;
constexpr int kTurnDwords = 16 * 132;      // transposed block, four dwords of padding per eight channels

// 2^e, e the smallest with max |x| <= 448 * 2^e and e >= -60, from the largest finite magnitude's bits.
LVS_DEV int scale_exponent(uint32_t amax) {
  const int e = (int)(amax >> 7) - 127 - 8 + ((amax & 0x7fu) > 0x60u ? 1 : 0);     // 448 = 1.75 * 2^8
  return e < -60 ? -60 : e;
}

LVS_DEV float bf16_lo(uint32_t x) { return __builtin_bit_cast(float, x << 16); }
LVS_DEV float bf16_hi(uint32_t x) { return __builtin_bit_cast(float, x & 0xffff0000u); }

// four floats to e4m3, nearest even; what is not finite becomes NaN (all finite ones are within 448)
LVS_DEV uint32_t pack_fp8(float a, float b, float c, float d) {
  const float nan = __builtin_nanf("");
  a = fabsf(a) <= 448.f ? a : nan;
  b = fabsf(b) <= 448.f ? b : nan;
  c = fabsf(c) <= 448.f ? c : nan;
  d = fabsf(d) <= 448.f ? d : nan;
  int r = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
  r = __builtin_amdgcn_cvt_pk_fp8_f32(c, d, r, true);
  return (uint32_t)r;
}

// x[i]: this thread's chunk of row 4q + i.  The scale is a power of two: x * 2^-e is exact, the conversion
// is the only rounding.  Every thread of the workgroup takes part.  Returned: keep_finite is to follow.
constexpr uint32_t kBeyond = 0x7f78;       // bits of 248 * 2^120
LVS_DEV bool store_block(const u32x4 (&x)[4], bool turned, uint8_t* dst, float* scale, uint32_t* s_turn,
                         uint32_t* s_max) {
  const int tid = threadIdx.x, q = tid >> 4, c = tid & 15;
  uint32_t amax = 0;
#pragma unroll
  for (int i = 0; i < 4; ++i)
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const uint32_t lo = x[i][j] & 0x7fffu, hi = (x[i][j] >> 16) & 0x7fffu;
      amax = max(amax, max(lo < 0x7f80u ? lo : 0u, hi < 0x7f80u ? hi : 0u));
    }
  amax = wave_max_u32(amax);
  __syncthreads();                           // (the scratch of a block before this one has been read)
  if ((tid & 63) == 0) s_max[tid >> 6] = amax;
  __syncthreads();
  amax = max(max(s_max[0], s_max[1]), max(s_max[2], s_max[3]));
  const bool beyond = __builtin_amdgcn_readfirstlane(amax) >= kBeyond;
  const int e = scale_exponent(amax);
  const float inv = __builtin_bit_cast(float, (uint32_t)(127 - e) << 23);
  if (tid == 0) *scale = __builtin_bit_cast(float, (uint32_t)(127 + e) << 23);
  if (!turned) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      uint2 y;
      y.x = pack_fp8(bf16_lo(x[i][0]) * inv, bf16_hi(x[i][0]) * inv, bf16_lo(x[i][1]) * inv, bf16_hi(x[i][1]) * inv);
      y.y = pack_fp8(bf16_lo(x[i][2]) * inv, bf16_hi(x[i][2]) * inv, bf16_lo(x[i][3]) * inv, bf16_hi(x[i][3]) * inv);
      *reinterpret_cast<uint2*>(dst + (4 * q + i) * 128 + c * 8) = y;
    }
    return beyond;
  }
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    s_turn[c * 132 + (2 * j) * 16 + q] = pack_fp8(bf16_lo(x[0][j]) * inv, bf16_lo(x[1][j]) * inv,
                                                  bf16_lo(x[2][j]) * inv, bf16_lo(x[3][j]) * inv);
    s_turn[c * 132 + (2 * j + 1) * 16 + q] = pack_fp8(bf16_hi(x[0][j]) * inv, bf16_hi(x[1][j]) * inv,
                                                      bf16_hi(x[2][j]) * inv, bf16_hi(x[3][j]) * inv);
  }
  __syncthreads();
#pragma unroll
  for (int k = 0; k < 2; ++k) {
    const int idx = tid + k * kCacheThreads, d = idx >> 2, g = idx & 3;
    *reinterpret_cast<u32x4*>(dst + idx * 16) =
        *reinterpret_cast<const u32x4*>(s_turn + (d >> 3) * 132 + (d & 7) * 16 + g * 4);
  }
  return beyond;
}

// Magnitudes from 248 * 2^120 on, the last ones of bf16, are rounded to 256 at the scale of 2^120, whose value 2^128
// is beyond bf16 and binary32: 240 (code 0x77) in the place of 256 (0x78), in a block that was just stored.  A
// second pass over such blocks only: in registers, before the store, it would take every block 1 to 5 % longer
// (16384 rows, 8 heads 20.8 us, so 21.0 to 21.9).
LVS_DEV void keep_finite(uint8_t* dst) {
  __syncthreads();
  for (int i = threadIdx.x; i < kPageBytes / 4; i += kCacheThreads) {
    uint32_t* at = reinterpret_cast<uint32_t*>(dst) + i;
    const uint32_t codes = *at, x = (codes & 0x7f7f7f7fu) ^ 0x78787878u;     // bytes of 256 are 0 in x
    *at = codes - (((0x80808080u - x) >> 7) & 0x01010101u);                 // (no byte borrows from the next)
  }
}

// ------------------------------------------------------------------------------ append
// One workgroup per 64 packed rows, kv head and tensor.  A block belongs to the workgroup that finds its
// last row; its first rows may be the packed rows of the tiles before or, where they came in an earlier
// call, rows of the ring.  Every row is read once and every block written once: bound by memory, 4.6 to 5.3 TB/s
// of reads and writes (16384 rows, 8 heads 19 to 22 us, 12 x (300 to 9000) rows 41), where a torch copy reaches
// 4.9; the turn of the values through LDS, a third of whose cycles are bank conflicts, hides behind that.
__global__ __launch_bounds__(kCacheThreads) void paged_append_kernel(AppendKernelArgs a) {
  __shared__ __align__(16) uint32_t s_turn[kTurnDwords];
  __shared__ uint32_t s_max[4];
  const int tid = threadIdx.x, lane = tid & 63, q = tid >> 4, c = tid & 15;
  const int h = blockIdx.y;
  const bool values = blockIdx.z != 0;
  const uint8_t* src = values ? a.v : a.k;
  const int64_t row_b = values ? a.v_sr : a.k_sr;
  src += (int64_t)h * (values ? a.v_sh : a.k_sh);
  uint8_t* tail = values ? a.v_tail : a.k_tail;
  const int t0 = blockIdx.x * kPageTokens;
  const int t = t0 + lane;
  const bool there = t < a.n_rows;
  const int slot = there ? a.slots[t] : LVSPEC_SLOT_NONE;
  const int pos = there ? a.row_pos[t] : 0;
  const bool to_tail = slot <= LVSPEC_SLOT_TAIL && LVSPEC_SLOT_TAIL - slot < a.B * kTailRows;
  // Rows of a request whose open block is completed by this call may share the ring's half with that
  // block (two blocks further on): the workgroup that reads the open block writes them, behind its reads.
  bool later = false;
  if (to_tail) {
    const int b = (LVSPEC_SLOT_TAIL - slot) / kTailRows;
    const int first = a.cu_rows[b];
    const int open = (pos - (t - first)) & (kPageTokens - 1);
    const int full = first + kPageTokens - 1 - open;
    if (open != 0 && first >= 0 && full < t && full >= 0) later = a.slots[full] >= 0;
  }
  const int my_tail = to_tail && !later ? LVSPEC_SLOT_TAIL - slot : -1;
  if (__ballot(my_tail >= 0) != 0ull) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int r = 16 * i + q;
      const int code = __shfl(my_tail, r, 64);
      if (code >= 0) {
        const int b = code / kTailRows, row = code % kTailRows;
        const u32x4 x = *reinterpret_cast<const u32x4*>(src + (int64_t)(t0 + r) * row_b + c * 16);
        *reinterpret_cast<u32x4*>(tail + (((int64_t)b * a.Hkv + h) * kTailRows + row) * kRowBytes + c * 16) = x;
      }
    }
  }
  unsigned long long todo = __ballot(slot >= 0 && (slot & (kPageTokens - 1)) == kPageTokens - 1), large = 0;
  while (todo != 0ull) {
    const int l = __builtin_ctzll(todo);
    todo &= todo - 1;
    const int at = t0 + l;                               // last row of the block
    const int id = __builtin_amdgcn_readlane(slot, l) >> kPageShift;
    const int p0 = __builtin_amdgcn_readlane(pos, l) - (kPageTokens - 1);
    const int b = a.row_seq[at];
    if (id >= a.n_blocks || (uint32_t)b >= (uint32_t)a.B) continue;
    const int first = a.cu_rows[b];
    if (first < 0 || first > at) continue;
    const int row0 = at - (kPageTokens - 1);             // packed row of the block's first token
    const uint8_t* ring = tail + ((int64_t)b * a.Hkv + h) * (kTailRows * kRowBytes);
    u32x4 x[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int r = 4 * q + i;
      const uint8_t* from = row0 + r >= first ? src + (int64_t)(row0 + r) * row_b
                                              : ring + ((p0 + r) & (kTailRows - 1)) * kRowBytes;
      x[i] = *reinterpret_cast<const u32x4*>(from + c * 16);
    }
    uint8_t* dst = (values ? a.v8 : a.k8) + ((int64_t)id * a.Hkv + h) * kPageBytes;
    if (store_block(x, values, dst, (values ? a.v_scale : a.k_scale) + (int64_t)id * a.Hkv + h, s_turn, s_max))
      large |= 1ull << l;
    if (row0 < first) {                                  // (the reads of the ring are behind a barrier)
      int end = a.cu_rows[b + 1];
      end = end < a.n_rows ? end : a.n_rows;
      const int from = max(at + 1, end - (kPageTokens - 1));
      for (int r = from + q; r < end; r += kCacheThreads / 16) {
        const int s = a.slots[r];
        const int code = LVSPEC_SLOT_TAIL - s;
        if (s <= LVSPEC_SLOT_TAIL && code / kTailRows == b) {
          const u32x4 y = *reinterpret_cast<const u32x4*>(src + (int64_t)r * row_b + c * 16);
          *reinterpret_cast<u32x4*>(tail + (((int64_t)b * a.Hkv + h) * kTailRows + code % kTailRows) * kRowBytes +
                                    c * 16) = y;
        }
      }
    }
  }
  for (; large != 0ull; large &= large - 1) {
    const int id = __builtin_amdgcn_readlane(slot, __builtin_ctzll(large)) >> kPageShift;
    keep_finite((values ? a.v8 : a.k8) + ((int64_t)id * a.Hkv + h) * kPageBytes);
  }
}

// ------------------------------------------------------------------------------ commit
// One workgroup per (sequence, kv head), tensor and layer: the kept chain's accepted rows move to the front
// of the draft area, and the block that they complete goes into the pool.  Both read the rows where the step
// left them; what is written (rows L .. L+tau-1, and the pool) is read by neither.
// All layers in one launch: a layer alone would be mostly launch.  Bound by memory where blocks become complete:
// 64 layers, 8 heads, 1 sequence 7.2 us for 25 MB, of which 3 are launch and lengths; 16 sequences with two
// chains of 10, a quarter of them with a block, 27 us for 126 MB, 4.6 TB/s.
// PLANNED: with what the step's plan granted, in a kernel of its own, whose loads go out with the lengths': 7.3 and
// 27.6 us per call, without a plan 7.2 and 27.3; chosen in one kernel 8.0 and 28.4.
template <bool PLANNED>
__global__ __launch_bounds__(kCacheThreads) void paged_commit_kernel(PagedCommitKernelArgs a) {
  __shared__ __align__(16) uint32_t s_turn[kTurnDwords];
  __shared__ uint32_t s_max[4];
  const int tid = threadIdx.x, q = tid >> 4, c = tid & 15;
  const int b = blockIdx.x / a.Hkv, h = blockIdx.x - b * a.Hkv;
  const bool values = blockIdx.y != 0;
  const int64_t layer = blockIdx.z;
  const int L = a.kv_len[b];
  // The table keeps entries of blocks that were given back, so what a sequence has is told by the plan: rows that
  // were not granted are not in the ring, and a block behind the held ones is another sequence's.
  int granted = 1, held = a.cols, rows = 0;
  if constexpr (PLANNED) {
    granted = a.granted[b];
    held = min(a.held[b], a.cols);
    rows = a.cu_rows[b + 1] - a.cu_rows[b];
  }
  int kept = a.best_branch != nullptr ? a.best_branch[b] : 0;
  kept = kept < 0 || kept >= a.n_branches ? 0 : kept;
  int tau = a.accept_len[b * a.n_branches + kept];
  tau = tau < 0 ? 0 : tau > a.chain_len ? a.chain_len : tau;
  if constexpr (PLANNED) tau = max(min(tau, rows - kept * a.chain_len), 0);
  const int col = L >> kPageShift;
  const bool in_range = L >= 0 && L <= a.cols * kPageTokens + kPageTokens - 1;
  const bool fills = in_range && ((L + tau) >> kPageShift) > col;
  int id = -1;
  if (fills && col < held) id = a.table[(int64_t)b * a.cols + col];
  // refused, no place for a block that becomes complete, or a length out of range: nothing is committed
  const bool ok = granted != 0 && in_range && (!fills || (uint32_t)id < (uint32_t)a.n_blocks);
  if (h == 0 && !values && layer == 0 && tid == 0) a.new_len[b] = ok ? L + tau : L;
  if (!ok) return;
  const int shift = kept * a.chain_len;
  uint8_t* ring = (values ? a.v_tail : a.k_tail) +
                  (layer * a.B * a.Hkv + (int64_t)b * a.Hkv + h) * (kTailRows * kRowBytes);
  if (fills) {
    u32x4 x[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int p = (col << kPageShift) + 4 * q + i;
      x[i] = *reinterpret_cast<const u32x4*>(ring + ((p < L ? p : p + shift) & (kTailRows - 1)) * kRowBytes + c * 16);
    }
    const int64_t at = (layer * a.n_blocks + id) * a.Hkv + h;
    uint8_t* dst = (values ? a.v8 : a.k8) + at * kPageBytes;
    if (store_block(x, values, dst, (values ? a.v_scale : a.k_scale) + at, s_turn, s_max)) keep_finite(dst);
  }
  if (shift > 0 && q < tau) {               // (at most 16 rows)
    const u32x4 y = *reinterpret_cast<const u32x4*>(ring + ((L + shift + q) & (kTailRows - 1)) * kRowBytes + c * 16);
    *reinterpret_cast<u32x4*>(ring + ((L + q) & (kTailRows - 1)) * kRowBytes + c * 16) = y;
  }
}

}  // namespace

hipError_t launch_paged_plan(const PlanKernelArgs& a, hipStream_t stream) {
  int64_t wgs = ((int64_t)a.max_rows + kPlanThreads * kPlanRows - 1) / (kPlanThreads * kPlanRows);
  const int64_t requests = a.B < 64 ? a.B : 64;
  if (wgs < requests) wgs = requests;
  if (wgs > 512) wgs = 512;
  paged_plan_kernel<<<dim3((unsigned)wgs), dim3(kPlanThreads), 0, stream>>>(a);
  return hipGetLastError();
}

hipError_t launch_paged_append(const AppendKernelArgs& a, hipStream_t stream) {
  const dim3 grid((unsigned)((a.n_rows + kPageTokens - 1) / kPageTokens), (unsigned)a.Hkv, 2);
  paged_append_kernel<<<grid, dim3(kCacheThreads), 0, stream>>>(a);
  return hipGetLastError();
}

hipError_t launch_paged_commit(const PagedCommitKernelArgs& a, hipStream_t stream) {
  const dim3 grid((unsigned)(a.B * a.Hkv), 2, (unsigned)a.n_layers);
  if (a.granted != nullptr)
    paged_commit_kernel<true><<<grid, dim3(kCacheThreads), 0, stream>>>(a);
  else
    paged_commit_kernel<false><<<grid, dim3(kCacheThreads), 0, stream>>>(a);
  return hipGetLastError();
}

}  // namespace lvspec
