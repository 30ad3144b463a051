// Bookkeeping of the paged cache in 8 bits: block tables and slot maps from request lengths, new rows into
// the cache, and a verified step into the caches of all layers.
#include "paged_store.h"

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

__global__ __launch_bounds__(kCacheThreads) void paged_append_kernel(AppendKernelArgs a) {
  __shared__ Pool8::Scratch scratch;
  append_rows<Pool8>(a, scratch, blockIdx.x, blockIdx.y, blockIdx.z != 0);
}

template <bool PLANNED>
__global__ __launch_bounds__(kCacheThreads) void paged_commit_kernel(PagedCommitKernelArgs a) {
  __shared__ Pool8::Scratch scratch;
  commit_rows<Pool8, PLANNED>(a, scratch);
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
