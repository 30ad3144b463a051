// Attention of the draft rows over the paged cache in 8 bits (paged_dev.h), the same contract as
// verification attention over a bf16 cache.
//
// Kernel 1 (split):   a unit (sequence, kv head, row chunk of at most 32 rows) is cut into parts along its keys; a
//   workgroup takes one part, its streams (waves) every KS-th tile of 64 keys.  A wave fetches its tiles itself,
//   straight into its own 16 KiB of LDS, and waits for nobody else:
//     keys:   an operand of S^T = K Q^T is made of 16 bytes of a token, converted to bf16; which channels a
//             lane's operand holds is a permutation that K and Q share;
//     values: 16 bytes of a channel are 16 tokens.  The tokens of a lane's scores are those of its value
//             operand, and probabilities stay in their lane.
//   The conversion multiplies by the block's scale (a power of two): exact, and nothing is left to scale.
//   Softmax in base 2 with a running maximum, sums in 32 bits; probabilities are rounded to bf16 for the
//   second product (each by at most 2^-8 of itself, 2^-9 on average, which averages out over the keys; it is what the
//   matrix instructions take).  Open rows, at most 95 in bf16, are taken 32 at a time by the streams of a unit's first
//   part.  The streams merge through LDS in fixed order into one record per part.
// Kernel 2 (combine): merge of a row's records in fixed order, bf16 output.
// Small tables: one workgroup per unit writes the output itself, and there is no second kernel.
// Bound: the streaming read of K and V from memory, 16 x (2048 to 32768) keys, 8 heads, 5 rows of 5 heads 70 us for
// 367 MB, 5.2 TB/s; of short ones the start, the merge and the second launch, 16384 keys 13.2 + 4.0 us for
// 34 MB; of 33 and more rows the vector instructions, which every chunk of 32 has for itself (16384 keys, 100
// rows: 19 to 20 us, vector unit 37 % busy, matrix unit 18 %, start and merge among them; 4 x 65536 keys,
// 64 rows 110 us for 540 MB, 4.9 TB/s, matrix unit 25 %).
#include "paged_segment.h"

namespace lvspec {

namespace {

template <class Rows, int KS, bool ONCE>
__global__ __launch_bounds__(64 * KS, 2) void paged_attn_kernel(PagedAttnKernelArgs p) {
  extern __shared__ __align__(256) uint8_t smem[];
  Segment<Rows, KS, ONCE> sg(p, smem);
  ask_for_arguments(p);
  Part o;
  if (!find_part<ONCE>(p, o)) return;
  if (o.part == 0 && threadIdx.x == 0) records_of(p)[o.b * (p.Hkv * p.n_rc) + o.hr] = int2{o.w, o.n};
  const int L = o.p0 == 0 ? paged_len(p.kv_len[o.b], p.cols) : 0;      // (for the open rows)
  sg.begin(o.b, o.h, o.rc);
  if (o.p0 == 0) sg.open_rows(o.b, o.h, o.rc, L);
  sg.blocks(o.b, o.h, o.t0, o.t1);
  const uint32_t on = sg.active(o.t1 - o.t0, o.p0 == 0, L);
  if (o.n == 1)
    sg.finish(on, o.b, o.h, o.rc);
  else
    sg.end(on, o.rc, record_at(p, o.w));
}

// One workgroup per unit, straight to the output: for tables so narrow that cutting a unit does not pay.  Bound
// by latencies one behind the other (lengths, table, tiles, open rows, merge): 777 keys, 2 heads 7.8 us.
template <class Rows, int KS, bool ONCE>
__global__ __launch_bounds__(64 * KS, 2) void paged_attn_unit_kernel(PagedAttnKernelArgs p) {
  extern __shared__ __align__(256) uint8_t smem[];
  Segment<Rows, KS, ONCE> sg(p, smem);
  ask_for_arguments(p);
  const int bh = (int)((uint32_t)blockIdx.x / (uint32_t)p.n_rc), rc = blockIdx.x - bh * p.n_rc;
  const int b = (int)((uint32_t)bh / (uint32_t)p.Hkv), h = bh - b * p.Hkv;
  const int L = paged_len(p.kv_len[b], p.cols);
  sg.begin(b, h, rc);
  sg.blocks(b, h, 0, L >> kPageShift);
  sg.open_rows(b, h, rc, L);
  sg.finish(sg.active(L >> kPageShift, true, L), b, h, rc);
}

// ------------------------------------------------------------------------------ combine
// Groups of 32 lanes, a lane four channels.  SPLIT groups share an output row and take every SPLIT-th record each:
// all eight of a workgroup where a unit has many records, or one group per row.  4.0 to 4.8 us, a launch and two
// loads one behind the other; what is read, 2 to 5 MB, is the first kernel's and lies in the caches.
constexpr int kCombineThreads = 256;

template <int SPLIT>
__global__ __launch_bounds__(kCombineThreads) void paged_combine_kernel(PagedAttnKernelArgs p) {
  constexpr int kRows = 8 / SPLIT;               // output rows of a workgroup, all of one unit
  constexpr int kAhead = 8;
  __shared__ float s_m[8], s_l[8], s_v[8];
  __shared__ f32x4 s_o[SPLIT > 1 ? 8 : 1][32];
  const int tid = threadIdx.x, g = tid >> 5, l32 = tid & 31;
  const int HR = p.Hkv * p.n_rc;
  const int per_unit = (p.rpad + kRows - 1) / kRows;
  const int unit = (int)((uint32_t)blockIdx.x / (uint32_t)per_unit);
  const int b = (int)((uint32_t)unit / (uint32_t)HR), hr = unit - b * HR;
  const int h = (int)((uint32_t)hr / (uint32_t)p.n_rc), rc = hr - h * p.n_rc;
  const int in = (blockIdx.x - unit * per_unit) * kRows + g / SPLIT, r = rc * p.rpad + in;
  const bool row = in < p.rpad && r < p.R;
  const int2 own = records_of(p)[unit];
  if (own.y == 1) return;                        // (one part: it has written the output)
  const int n = own.y;
  const int64_t step = (int64_t)p.rpad * 131;
  const float* rec = record_at(p, own.x) + (row ? in : 0);
  // every group for itself: maximum, sums and output of its records, eight at a time
  float mm = kNegBig, l = 0.f, lv = 0.f;
  f32x4 o = {0.f, 0.f, 0.f, 0.f};
  const float* orec = rec + 3 * p.rpad + (row ? in : 0) * 127 + l32 * 4;
  for (int k0 = g % SPLIT; k0 < n; k0 += SPLIT * kAhead) {
    f32x4 x[kAhead];
    float m8[kAhead], l8[kAhead], v8[kAhead];
#pragma unroll
    for (int k = 0; k < kAhead; ++k) {
      const int at = k0 + SPLIT * k < n ? k0 + SPLIT * k : k0;
      const int64_t off = at * step;
      x[k] = *reinterpret_cast<const f32x4*>(orec + off);
      m8[k] = rec[off];
      l8[k] = rec[off + p.rpad];
      v8[k] = rec[off + 2 * p.rpad];
    }
    float top = mm;
#pragma unroll
    for (int k = 0; k < kAhead; ++k) top = fmaxf(top, m8[k]);
    const float old = fast_exp2(mm - top);
    mm = top;
    o *= old;
    l *= old;
    lv *= old;
#pragma unroll
    for (int k = 0; k < kAhead; ++k) {
      if (k0 + SPLIT * k < n) {
        const float f = fast_exp2(m8[k] - top);
        o += x[k] * f;
        l += l8[k] * f;
        lv += v8[k] * f;
      }
    }
  }
  if constexpr (SPLIT > 1) {
    if (l32 == 0) {
      s_m[g] = mm;
      s_l[g] = l;
      s_v[g] = lv;
    }
    s_o[g][l32] = o;
    __syncthreads();
    if (g % SPLIT != 0) return;
    float top = mm;
#pragma unroll
    for (int k = 1; k < SPLIT; ++k) top = fmaxf(top, s_m[g + k]);
    const float f = fast_exp2(mm - top);
    o *= f;
    l *= f;
    lv *= f;
#pragma unroll
    for (int k = 1; k < SPLIT; ++k) {
      const float f2 = fast_exp2(s_m[g + k] - top);
      o += s_o[g + k][l32] * f2;
      l += s_l[g + k] * f2;
      lv += s_v[g + k] * f2;
    }
    mm = top;
  }
  if (row) write_row(p, b, h, r, l32, o, mm, l, lv);
}

template <class Rows, int KS, bool ONCE>
hipError_t launch_parts(const PagedAttnKernelArgs& a, hipStream_t stream) {
  static LdsLimitOnce limit;
  constexpr size_t lds = segment_lds<Rows, KS>();
  hipError_t e = limit.ensure(reinterpret_cast<const void*>(&paged_attn_kernel<Rows, KS, ONCE>), lds);
  if (e != hipSuccess) return e;
  paged_attn_kernel<Rows, KS, ONCE><<<dim3((unsigned)(a.limit + 7) / 8 * 8), dim3(64 * KS), lds, stream>>>(a);
  e = hipGetLastError();
  return e != hipSuccess ? e : launch_paged_combine(a, stream);
}

template <class Rows, int KS, bool ONCE>
hipError_t launch_units(const PagedAttnKernelArgs& a, hipStream_t stream) {
  static LdsLimitOnce limit;
  constexpr size_t lds = segment_lds<Rows, KS>();
  hipError_t e = limit.ensure(reinterpret_cast<const void*>(&paged_attn_unit_kernel<Rows, KS, ONCE>), lds);
  if (e != hipSuccess) return e;
  const unsigned units = (unsigned)(a.B * a.Hkv * a.n_rc);
  paged_attn_unit_kernel<Rows, KS, ONCE><<<dim3(units), dim3(64 * KS), lds, stream>>>(a);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_paged_combine(const PagedAttnKernelArgs& a, hipStream_t stream) {
  const unsigned units = (unsigned)(a.B * a.Hkv * a.n_rc);
  // few units have many records each: all groups of a workgroup to one row.  8 units, 32 records each: 16.4 us
  // so and 17.7 with a group per row; 64 units, 4 each: 23.9 and 20.9.
  if ((int64_t)units * 16 > a.limit - a.spare)
    paged_combine_kernel<1><<<dim3(units * (unsigned)((a.rpad + 7) / 8)), dim3(kCombineThreads), 0, stream>>>(a);
  else
    paged_combine_kernel<8><<<dim3(units * (unsigned)a.rpad), dim3(kCombineThreads), 0, stream>>>(a);
  return hipGetLastError();
}

hipError_t launch_paged_attn(const PagedAttnKernelArgs& a, hipStream_t stream) {
  const bool once = a.n_rc == 1;
  const int64_t units = (int64_t)a.B * a.Hkv * a.n_rc;
  const int64_t cus = a.limit - units + 1;
  if (a.cols <= unit_columns(a.B, units, cus, 18)) {
    if (a.rpad <= 16) return launch_units<Rows16, 8, true>(a, stream);      // (one chunk: two have 17 rows each and more)
    return once ? launch_units<WideRows, 8, true>(a, stream) : launch_units<WideRows, 8, false>(a, stream);
  }
  // More than 64 rows are bound by vector instructions, beside which the matrix unit has more to do with two waves on a
  // SIMD.  But then one workgroup fills a CU, and parts beyond the compute units wait for a second turn: that
  // is for few units only.  Four and eight streams, us: 16384 keys, 100 rows 22.5 and 22.2 (24.5 both from memory rather
  // than the cache before it); 32000 keys, 100 rows 32.7 and 31.8; 60000 keys, 150 rows 68 and 63; 2 x 16000, 150 rows
  // 40.6 and 38.4; 5 x (1000 to 20000), 100 rows, 160 units 37.8 and 36.7; 6 of them, 192 units 47.7 and 54.3; 64 rows
  // 12 x (1000 to 20000) 54.4 and 59.7; 25 rows, 16384 keys 16.0 and 16.9.
  if (a.n_rc >= 3 && units * 8 <= cus * 5) return launch_parts<WideRows, 8, false>(a, stream);
  if (a.rpad <= 16) return launch_parts<Rows16, 4, true>(a, stream);
  return once ? launch_parts<WideRows, 4, true>(a, stream) : launch_parts<WideRows, 4, false>(a, stream);
}

}  // namespace lvspec
