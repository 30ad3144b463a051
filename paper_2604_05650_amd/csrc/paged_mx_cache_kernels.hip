// Bookkeeping of the paged cache in 4 bits: new rows, a verified step, and rows read back.  (Plans are those of the
// cache in 8 bits.)
#include "paged_mx_store.h"

namespace lvspec {

namespace {

// 16384 rows of 8 heads 18.1 us, 85 MB at 4.7 TB/s (in 8 bits 20.4, 101 MB); 16 x 5 rows 3.0.
__global__ __launch_bounds__(kCacheThreads) void paged_mx_append_kernel(AppendKernelArgs a) {
  __shared__ Pool4::Scratch scratch;
  append_rows<Pool4>(a, scratch, blockIdx.x, blockIdx.y, blockIdx.z != 0);
}

// 64 layers of 8 heads: one sequence's block completed in each 7.8 us, mostly launch and lengths; 16 sequences' second
// chain of ten kept, four of whose blocks it completes, 38.7 (in 8 bits 8.4 and 41.9).
template <bool PLANNED>
__global__ __launch_bounds__(kCacheThreads) void paged_mx_commit_kernel(PagedCommitKernelArgs a) {
  __shared__ Pool4::Scratch scratch;
  commit_rows<Pool4, PLANNED>(a, scratch);
}

// ------------------------------------------------------------------------------ read
// One workgroup per 64 packed rows, kv head and tensor.  A key's eight channels are a dword of its block; the values,
// which lie by channel, go through LDS block by block.  Bound by memory, most of it writes: 16384 rows of 8 heads 16.0 us,
// 85 MB at 5.3 TB/s, 12 x (300 to 9000) rows 29.8 us, 179 MB at 6.0.
__global__ __launch_bounds__(kCacheThreads) void paged_mx_read_kernel(ReadKernelArgs a) {
  __shared__ __align__(16) uint8_t s_codes[16 * 272];
  __shared__ __align__(16) uint8_t s_scale[kScale4Bytes];
  const int tid = threadIdx.x, lane = tid & 63, q = tid >> 4, c = tid & 15;
  const int h = blockIdx.y;
  const bool values = blockIdx.z != 0;
  uint8_t* out = (values ? a.v : a.k) + (int64_t)h * (values ? a.v_sh : a.k_sh);
  const int64_t row_b = values ? a.v_sr : a.k_sr;
  const int t0 = blockIdx.x * kPageTokens;
  const int slot = t0 + lane < a.n_rows ? a.slots[t0 + lane] : LVSPEC_SLOT_NONE;
  const bool pooled = slot >= 0 && (slot >> kPageShift) < a.n_blocks;
  const int ring = slot <= LVSPEC_SLOT_TAIL && LVSPEC_SLOT_TAIL - slot < a.B * kTailRows ? LVSPEC_SLOT_TAIL - slot : -1;
  const u32x4 nan = {0x7fc07fc0u, 0x7fc07fc0u, 0x7fc07fc0u, 0x7fc07fc0u};
  const int place = pooled ? slot : -1;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int r = 16 * i + q;
    const int code = __shfl(ring, r, 64), at = __shfl(place, r, 64);
    u32x4 x;
    if (code >= 0) {
      const uint8_t* tail = values ? a.v_tail : a.k_tail;
      x = *reinterpret_cast<const u32x4*>(tail + (((int64_t)(code / kTailRows) * a.Hkv + h) * kTailRows + code % kTailRows) * kRowBytes + c * 16);
    } else if (at >= 0 && !values) {
      const int64_t block = (int64_t)(at >> kPageShift) * a.Hkv + h;
      const int token = at & (kPageTokens - 1);
      const uint32_t codes = *reinterpret_cast<const uint32_t*>(a.k4 + block * kPage4Bytes + (c >> 3) * 2048 + token * 32 + (c & 7) * 4);
      const uint32_t e = a.k_scale[block * kScale4Bytes + ((c >> 2) & 1) * 128 + (token & 31) * 4 + 2 * (token >> 5) + (c >> 3)];
      x = widen4(codes, __builtin_bit_cast(float, e << 23));
      if (e == 255u) x = nan;
    }
    if (code >= 0 || (at >= 0 && !values)) *reinterpret_cast<u32x4*>(out + (int64_t)(t0 + r) * row_b + c * 16) = x;
  }
  if (!values) return;
  unsigned long long todo = __ballot(pooled);
  while (todo != 0ull) {
    const int id = __builtin_amdgcn_readlane(slot, __builtin_ctzll(todo)) >> kPageShift;
    const unsigned long long same = __ballot(pooled && (slot >> kPageShift) == id);      // (the same in every wave)
    todo &= ~same;
    const int64_t block = (int64_t)id * a.Hkv + h;
    __syncthreads();
    *reinterpret_cast<u32x4*>(s_codes + (tid >> 4) * 272 + (tid & 15) * 16) =
        *reinterpret_cast<const u32x4*>(a.v4 + block * kPage4Bytes + tid * 16);
    if (tid < kScale4Bytes / 4)
      reinterpret_cast<uint32_t*>(s_scale)[tid] = reinterpret_cast<const uint32_t*>(a.v_scale + block * kScale4Bytes)[tid];
    __syncthreads();
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int r = 16 * i + q;
      const int token = __shfl(slot, r, 64) & (kPageTokens - 1);
      if (((same >> r) & 1ull) == 0ull) continue;
      const int half = (token >> 2) & 1, nth = (token >> 3) * 4 + (token & 3);
      uint32_t codes = 0;
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const uint32_t y = s_codes[c * 272 + j * 32 + half * 16 + (nth >> 1)];
        codes |= ((nth & 1 ? y >> 4 : y) & 15u) << (4 * j);
      }
      u32x4 x = widen4(codes, 1.f);
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const int ch = 8 * c + 2 * j;
        const uint32_t e0 = s_scale[half * 128 + (ch & 31) * 4 + (ch >> 5)];
        const uint32_t e1 = s_scale[half * 128 + ((ch + 1) & 31) * 4 + (ch >> 5)];
        const uint32_t lo = e0 == 255u ? 0x7fc0u : __builtin_bit_cast(uint32_t, bf16_lo(x[j]) * __builtin_bit_cast(float, e0 << 23)) >> 16;
        const uint32_t hi = e1 == 255u ? 0x7fc00000u : __builtin_bit_cast(uint32_t, bf16_hi(x[j]) * __builtin_bit_cast(float, e1 << 23)) & 0xffff0000u;
        x[j] = lo | hi;
      }
      *reinterpret_cast<u32x4*>(out + (int64_t)(t0 + r) * row_b + c * 16) = x;
    }
  }
}

}  // namespace

hipError_t launch_paged_mx_append(const AppendKernelArgs& a, hipStream_t stream) {
  const dim3 grid((unsigned)((a.n_rows + kPageTokens - 1) / kPageTokens), (unsigned)a.Hkv, 2);
  paged_mx_append_kernel<<<grid, dim3(kCacheThreads), 0, stream>>>(a);
  return hipGetLastError();
}

hipError_t launch_paged_mx_commit(const PagedCommitKernelArgs& a, hipStream_t stream) {
  const dim3 grid((unsigned)(a.B * a.Hkv), 2, (unsigned)a.n_layers);
  if (a.granted != nullptr)
    paged_mx_commit_kernel<true><<<grid, dim3(kCacheThreads), 0, stream>>>(a);
  else
    paged_mx_commit_kernel<false><<<grid, dim3(kCacheThreads), 0, stream>>>(a);
  return hipGetLastError();
}

hipError_t launch_paged_mx_read(const ReadKernelArgs& a, hipStream_t stream) {
  const dim3 grid((unsigned)((a.n_rows + kPageTokens - 1) / kPageTokens), (unsigned)a.Hkv, 2);
  paged_mx_read_kernel<<<grid, dim3(kCacheThreads), 0, stream>>>(a);
  return hipGetLastError();
}

}  // namespace lvspec
