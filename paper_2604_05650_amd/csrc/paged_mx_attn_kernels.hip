// Attention of the draft rows over the paged cache in 4 bits (paged_mx_dev.h); parts, open rows and merges are those of
// the cache in 8 bits (paged_segment.h).
//
// A wave takes every KS-th tile of 64 keys of its workgroup's part.  A tile's codes lie in memory as the lanes take
// them: they are loaded straight into registers, 1 KiB in one piece per instruction.
//   S^T = K Q^T: keys go into the matrix instructions as they are, with their scales.  What they meet are sums of three
//     numbers of 6 bits (e2m3, 1 to 7.5 in steps of an eighth to a half, and down to an eighth) with a power of two per
//     row and 32 channels: a bf16 number of 1/64 of the largest of its 32 and above loses nothing, a smaller one at
//     most 2^-14.9 of that largest (split6).  12 instructions of half the time instead of 16 of bf16, and no keys to widen.
//   O^T = V^T P^T: scores are left in the lanes that hold the values of their tokens, so probabilities, rounded to bf16
//     (each by at most 2^-8 of itself), go into the second product where they are; values are widened to bf16 with
//     their scales (exact).  In numbers of 6 bits probabilities take three as well, whose making costs what the
//     widening does, and what is far below the largest of its 32 loses its last bits.
//
// What bounds it: 16 x (2048 to 32768) keys of 8 heads, 25 rows take 46.4 us with the second kernel, 197 MB: memory, parts of
// unequal length (121 tiles where 90 would be even), start and merge (when it took 51, it took 41.8 without products and
// softmax).  4 x 65536 keys, 64 rows take 77.7 us: vector instructions, about 310 a tile of which 96 are exponentials or
// widen values, keep their unit busy for 48 % and the matrix unit is busy for 34 % of the time; two waves a SIMD, all that
// the registers hold, hide one behind the other in part (when it took 87, 62 without products and softmax).  One sequence of
// 16384 keys takes 15.0 us, 4 of them the second kernel and 11 what follows what in the first (lengths, queries, open rows,
// their split, two or three tiles a wave, merge 2.2); 777 keys 8.1.  The cache in 8 bits takes 72.5, 121, 15.7 and 7.6.
#include "paged_mx_dev.h"
#include "paged_segment.h"

namespace lvspec {

namespace {

// 32 numbers of 6 bits.
typedef uint32_t Six __attribute__((ext_vector_type(6)));
typedef float f32x32 __attribute__((ext_vector_type(32)));
typedef int i32x8 __attribute__((ext_vector_type(8)));

// x[0] y[0] x[1] y[1] .. / scale to the nearest numbers of 6 bits, and back.  (In assembly: the instructions write their
// result before they have read all they take, which this compiler does not know; the waits are those between
// instructions of this kind and what the compiler puts around them.)
LVS_DEV Six to_six(const f32x16& x, const f32x16& y, float scale) {
  Six r;
  asm("s_nop 1\n\tv_cvt_scalef32_2xpk16_fp6_f32 %0, %1, %2, %3\n\ts_nop 1" : "=&v"(r) : "v"(x), "v"(y), "v"(scale));
  return r;
}
LVS_DEV f32x32 from_six(const Six& x, float scale) {
  f32x32 r;
  asm("s_nop 1\n\tv_cvt_scalef32_pk32_f32_fp6 %0, %1, %2\n\ts_nop 1" : "=&v"(r) : "v"(x), "v"(scale));
  return r;
}

// Three terms, at scales of 1, 2^-4 and 2^-9, of numbers up to 7.5: what a term leaves, at most a quarter of its scale, is
// at most 4 of the second's, and what that leaves, an eighth, at most 4 of the third's.  Of a bf16 number the first two leave
// no more than 2^-8, 2 of the third's scale, where its step is 2^-12: numbers from 2^-5 on, whose last bit that is, are exact,
// and smaller ones off by 2^-13 at most.  The largest of the 32 is above 3.75, so that is 2^-14.9 of it.
template <class Put>
LVS_DEV void split6(f32x16 x, f32x16 y, Put&& put) {
  constexpr float kScale[3] = {1.f, 0x1p-4f, 0x1p-9f};
#pragma unroll
  for (int term = 0; term < 3; ++term) {
    const Six v = to_six(x, y, kScale[term]);
    put(term, v);
    if (term < 2) {
      const f32x32 z = from_six(v, kScale[term]);
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        x[i] -= z[2 * i];
        y[i] -= z[2 * i + 1];
      }
    }
  }
}

// D += A B, 32x32, 64 deep: A 32 codes of e2m1 a lane, scale in byte KS of ks; B 32 numbers of 6 bits, byte QS of qs.
template <int KS, int QS>
LVS_DEV f32x16 mfma_mx(const u32x4& a, uint32_t ks, const Six& b, uint32_t qs, const f32x16& c) {
  const i32x8 x = {(int)a[0], (int)a[1], (int)a[2], (int)a[3], 0, 0, 0, 0};
  const i32x8 y = {(int)b[0], (int)b[1], (int)b[2], (int)b[3], (int)b[4], (int)b[5], 0, 0};
  return __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(x, y, c, 4, 2, KS, (int)ks, QS, (int)qs);
}

// 32 query rows on 32x32 tiles: the tokens of a lane's scores are those of its values, element 16 t + r is token
// 32 t + 8 (r / 4) + 4 h + r % 4.
struct FourRows : WideRows {
  // A row of 32 tiles meets a new maximum in most of them, if only by a little, and a rescaling is a fifth of a tile's
  // vector instructions: 4 x 65536 keys, 64 rows 87.4 -> 81.6 us, 16 x (2048 to 32768) keys 51.0 -> 48.5.  The exact 1
  // that the largest probability often is otherwise is lost, and its rounding is one more: error against 64 bits 2.1e-3 and
  // 2.0e-3 -> 2.3e-3 (every probability is within 2^-8 of itself either way).
  static constexpr int kSlack = 8;
  static LVS_DEV int key_of(int lane, int e) { return 32 * (e >> 4) + 8 * ((e >> 2) & 3) + 4 * (lane >> 5) + (e & 3); }
  // channels 64 a + 32 h + 8 y .. +7 at 4 a + y, of queries and of open keys
  static LVS_DEV int channel(int x, int lane) { return 64 * (x >> 2) + 32 * (lane >> 5) + 8 * (x & 3); }
  LVS_DEV void load_q(const uint16_t* qp, int lane) {
#pragma unroll
    for (int x = 0; x < 8; ++x) q[x] = *reinterpret_cast<const u32x4*>(qp + channel(x, lane));
  }
  LVS_DEV void open_load(u32x4 (&k)[8], const uint8_t* kt, int p0, int lane) const {
#pragma unroll
    for (int x = 0; x < 8; ++x)
      k[x] = *reinterpret_cast<const u32x4*>(kt + ((p0 + (lane & 31)) & (kTailRows - 1)) * kRowBytes + 2 * channel(x, lane));
  }
  static constexpr int kSplitChunks = 5;      // of 16 bytes a lane: three terms and scales of half of q
  Six q6[3][2];            // term, channels 64 a + 32 h .. + 31
  uint32_t qs[2];          // their scales' exponents, byte by term

  // Half A of q to LDS, as lanes take it.  A row's 32 channels of which one is not finite are NaN.
  template <int A>
  LVS_DEV void split_q(uint32_t to, int lane) const {
    uint32_t m = 0;
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      const uint32_t w = q[4 * A + (i >> 2)][i & 3];
      m = max(m, max(w & 0x7fffu, (w >> 16) & 0x7fffu));
    }
    const bool nan = m >= 0x7f80u;
    const int e = max((int)(m >> 7) - 127 - 2 + ((m & 0x7fu) > 0x70u ? 1 : 0), -118);      // max |q| <= 7.5 * 2^e; 2^(e-9) is a scale
    const float inv = __builtin_bit_cast(float, (uint32_t)(127 - e) << 23);
    f32x16 x, y;
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      const uint32_t w = nan ? 0u : q[4 * A + (i >> 2)][i & 3];
      x[i] = __builtin_bit_cast(float, w << 16) * inv;      // (at 2^126 the nearest of 6 bits may be 2^128)
      y[i] = __builtin_bit_cast(float, w & 0xffff0000u) * inv;
    }
    const uint32_t byte = (uint32_t)(e + 127);
    uint32_t all[kSplitChunks * 4];
    all[18] = nan ? 0xffffffffu : byte | ((byte - 4) << 8) | ((byte - 9) << 16);
    all[19] = 0;
    split6(x, y, [&](int term, const Six& v) {
#pragma unroll
      for (int i = 0; i < 6; ++i) all[6 * term + i] = v[i];
    });
#pragma unroll
    for (int i = 0; i < kSplitChunks; ++i)
      *(__attribute__((address_space(3))) u32x4*)(uintptr_t)(to + i * 1024 + lane * 16) =
          u32x4{all[4 * i], all[4 * i + 1], all[4 * i + 2], all[4 * i + 3]};
  }
  template <int A>
  LVS_DEV void take_q(uint32_t from, int lane) {
    uint32_t all[kSplitChunks * 4];
#pragma unroll
    for (int i = 0; i < kSplitChunks; ++i) {
      const u32x4 x = lds_load16(from + i * 1024 + lane * 16);
#pragma unroll
      for (int j = 0; j < 4; ++j) all[4 * i + j] = x[j];
    }
#pragma unroll
    for (int term = 0; term < 3; ++term) q6[term][A] = Six{all[6 * term], all[6 * term + 1], all[6 * term + 2],
                                                           all[6 * term + 3], all[6 * term + 4], all[6 * term + 5]};
    qs[A] = all[18];
  }

  LVS_DEV void scores4(float (&s)[32], const u32x4 (&k)[4], uint32_t scales) const {
    auto tile = [&](auto t) {
      f32x16 z;
#pragma unroll
      for (int r = 0; r < 16; ++r) z[r] = 0.f;
      auto half = [&](auto a) {
        constexpr int ks = 2 * t.value + a.value;
        z = mfma_mx<ks, 0>(k[2 * a.value + t.value], scales, q6[0][a.value], qs[a.value], z);
        z = mfma_mx<ks, 1>(k[2 * a.value + t.value], scales, q6[1][a.value], qs[a.value], z);
        z = mfma_mx<ks, 2>(k[2 * a.value + t.value], scales, q6[2][a.value], qs[a.value], z);
      };
      half(std::integral_constant<int, 0>{});
      half(std::integral_constant<int, 1>{});
#pragma unroll
      for (int r = 0; r < 16; ++r) s[16 * t.value + r] = z[r];
    };
    tile(std::integral_constant<int, 0>{});
    tile(std::integral_constant<int, 1>{});
  }
  LVS_DEV void output4(const u32x4 (&pr)[4], const u32x4 (&v)[4], uint32_t scales) {
    const float f[4] = {scale4<0>(scales), scale4<1>(scales), scale4<2>(scales), scale4<3>(scales)};
#pragma unroll
    for (int y = 0; y < 4; ++y)
#pragma unroll
      for (int c = 0; c < 4; ++c) acc[c] = mfma32(widen4(v[c][y], f[c]), pr[y], acc[c]);
  }
};

// What a call reads once is not left in the caches, which pays where it comes from memory, as over a model's layers, and costs
// where the cache before the memory has it: 16384 keys, 25 rows over 30 sets 15.2 us and 15.9 without, over three 15.0 and
// 14.5; 16 x (2048 to 32768) keys 47.6 and 51.2, 64 x 4000 57.0 and 61.5.
template <bool ONCE, class T>
LVS_DEV T load_once(const uint8_t* at) {
  const T* p = reinterpret_cast<const T*>(at);
  if constexpr (ONCE) return __builtin_nontemporal_load(p);
  return *p;
}

template <int KS, bool ONCE>
struct Segment4 : Segment<FourRows, KS, ONCE> {
  using Base = Segment<FourRows, KS, ONCE>;
  using Base::p;
  using Base::st;
  using Base::stream;
  LVS_DEV Segment4(const PagedAttnKernelArgs& a, uint8_t* lds) : Base(a, lds) {}

  static_assert(KS >= 5, "the three streams that may have open rows, once, do not split queries");
  const int32_t* row;                  // of the table
  int h, t0, t1, mine;                 // kv head; tiles of the part; of the wave
  int ids;                             // blocks of 64 of them, one per lane; -1: no block of the pool
  int id;                              // of the tile that is on its way
  int64_t at;                          // its place in the pools; where there is no block, the first's
  u32x4 k[4];                          // its keys
  uint32_t ks;

  LVS_DEV void fetch(int j0, int lane) {
    const int t = t0 + stream + KS * (j0 + lane);
    ids = t < t1 ? row[t] : -1;
    ids = (uint32_t)ids < (uint32_t)p.n_blocks ? ids : -1;
  }
  LVS_DEV void next(int j, int lane) {
    if ((j & 63) == 0) fetch(j, lane);
    id = __builtin_amdgcn_readlane(ids, j & 63);
    at = (int64_t)max(id, 0) * p.Hkv + h;
    load(k, ks, p.k8, p.k_scale, at, lane);
  }
  LVS_DEV void load(u32x4 (&x)[4], uint32_t& scales, const uint8_t* pool, const void* scale, int64_t at, int lane) const {
    const uint8_t* from = pool + at * kPage4Bytes + (lane & 31) * 32 + (lane >> 5) * 16;
    scales = load_once<ONCE, uint32_t>(static_cast<const uint8_t*>(scale) + at * kScale4Bytes + lane * 4);
#pragma unroll
    for (int i = 0; i < 4; ++i) x[i] = load_once<ONCE, u32x4>(from + i * 1024);
  }

  // Open rows, where the segment has them (`open`), and tiles `from` .. to - 1 of a unit.  Two waves split the queries for all
  // (for every wave by itself it is half a microsecond of each SIMD).  In a WHOLE unit waves without open rows do not wait
  // for those that have them: 777 keys, 2 heads 8.1 -> 8.0 us, four sequences of 200 keys 8.0 -> 7.3.  In parts, of which
  // one in a few has any, it takes 1 % longer (4 x 65536 keys, 64 rows 82.5 -> 83.6).
  template <bool WHOLE>
  LVS_DEV void run4(int b, int head, int rc, int from, int to, bool open, int L) {
    row = p.table + (int64_t)b * p.cols;
    h = head;
    t0 = from;
    t1 = to;
    mine = (t1 - t0 - stream + KS - 1) / KS;
    const uint32_t at0 = lds_addr(this->smem) + kPageBytes, at1 = at0 + kRingBytes;      // (behind open rows)
    auto split = [&](int lane) {
      if (stream == 0) st.template split_q<0>(at0, lane);
      if (stream == 1) st.template split_q<1>(at1, lane);
      lds_barrier();
    };
    if (WHOLE && this->has_open(L)) {
      this->open_rows(b, head, rc, L, [&] {
        if (t1 > t0) lds_barrier();
      });
      if (mine > 0) next(0, Base::lane_now());
    } else {
      if (!WHOLE && open) this->open_rows(b, head, rc, L);
      if (mine > 0) next(0, Base::lane_now());
      if (t1 > t0) split(Base::lane_now());
    }
    if (t1 <= t0) return;
    const int lane = Base::lane_now();
    st.template take_q<0>(at0, lane);
    st.template take_q<1>(at1, lane);
    for (int j = 0; j < mine; ++j) {
      const bool there = id >= 0;        // (an entry that names no block of the pool: no key)
      u32x4 v[4];
      uint32_t vs;
      load(v, vs, p.v8, p.v_scale, at, lane);
      float s[32];
      st.scores4(s, k, ks);
      if (j + 1 < mine) next(j + 1, lane);
      if (!there) continue;
      this->softmax(s, (t0 + stream + KS * j) * kPageTokens, kPageTokens, [&](int e) { return FourRows::key_of(lane, e); });
      u32x4 pr[4];
#pragma unroll
      for (int y = 0; y < 4; ++y)
        pr[y] = pack8(s[8 * y], s[8 * y + 1], s[8 * y + 2], s[8 * y + 3], s[8 * y + 4], s[8 * y + 5], s[8 * y + 6],
                      s[8 * y + 7]);
      st.output4(pr, v, vs);
    }
  }
};

template <int KS, bool ONCE>
__global__ __launch_bounds__(64 * KS, 2) void paged_mx_attn_kernel(PagedAttnKernelArgs p) {
  extern __shared__ __align__(256) uint8_t smem[];
  Segment4<KS, ONCE> sg(p, smem);
  ask_for_arguments(p);
  Part o;
  if (!find_part<ONCE>(p, o)) return;
  if (o.part == 0 && threadIdx.x == 0) records_of(p)[o.b * (p.Hkv * p.n_rc) + o.hr] = int2{o.w, o.n};
  const int L = o.p0 == 0 ? paged_len(p.kv_len[o.b], p.cols) : 0;      // (for the open rows)
  sg.begin(o.b, o.h, o.rc);
  sg.template run4<false>(o.b, o.h, o.rc, o.t0, o.t1, o.p0 == 0, L);
  const uint32_t on = sg.active(o.t1 - o.t0, o.p0 == 0, L);
  if (o.n == 1)
    sg.finish(on, o.b, o.h, o.rc);
  else
    sg.end(on, o.rc, record_at(p, o.w));
}

// One workgroup per unit, straight to the output.
template <int KS, bool ONCE>
__global__ __launch_bounds__(64 * KS, 2) void paged_mx_attn_unit_kernel(PagedAttnKernelArgs p) {
  extern __shared__ __align__(256) uint8_t smem[];
  Segment4<KS, ONCE> sg(p, smem);
  ask_for_arguments(p);
  const int bh = (int)((uint32_t)blockIdx.x / (uint32_t)p.n_rc), rc = blockIdx.x - bh * p.n_rc;
  const int b = (int)((uint32_t)bh / (uint32_t)p.Hkv), h = bh - b * p.Hkv;
  const int L = paged_len(p.kv_len[b], p.cols);
  sg.begin(b, h, rc);
  sg.template run4<true>(b, h, rc, 0, L >> kPageShift, true, L);
  sg.finish(sg.active(L >> kPageShift, true, L), b, h, rc);
}

template <int KS, bool ONCE>
hipError_t launch_parts4(const PagedAttnKernelArgs& a, hipStream_t stream) {
  static LdsLimitOnce limit;
  constexpr size_t lds = segment_lds<FourRows, KS>();
  hipError_t e = limit.ensure(reinterpret_cast<const void*>(&paged_mx_attn_kernel<KS, ONCE>), lds);
  if (e != hipSuccess) return e;
  paged_mx_attn_kernel<KS, ONCE><<<dim3((unsigned)(a.limit + 7) / 8 * 8), dim3(64 * KS), lds, stream>>>(a);
  e = hipGetLastError();
  return e != hipSuccess ? e : launch_paged_combine(a, stream);
}

template <int KS, bool ONCE>
hipError_t launch_units4(const PagedAttnKernelArgs& a, hipStream_t stream) {
  static LdsLimitOnce limit;
  constexpr size_t lds = segment_lds<FourRows, KS>();
  hipError_t e = limit.ensure(reinterpret_cast<const void*>(&paged_mx_attn_unit_kernel<KS, ONCE>), lds);
  if (e != hipSuccess) return e;
  const unsigned units = (unsigned)(a.B * a.Hkv * a.n_rc);
  paged_mx_attn_unit_kernel<KS, ONCE><<<dim3(units), dim3(64 * KS), lds, stream>>>(a);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_paged_mx_attn(const PagedAttnKernelArgs& a, hipStream_t stream) {
  const bool once = a.n_rc == 1;
  const int64_t units = (int64_t)a.B * a.Hkv * a.n_rc;
  const int64_t cus = a.limit - units + 1;
  // One workgroup per unit and parts, us: 8 units 800 keys 10.2 and 11.9, 1400 11.4 and 12.1, 2000 12.7 and 12.3; 64 units 1500
  // keys 13.1 and 14.1, 2500 15.1 and 15.4, 4000 20.2 and 18.0; 128 units 2000 keys 14.2 and 18.6, 4000 21.1 and 22.9, 6000 27.7
  // and 28.0; 256 units 4000 keys 29.2 and 32.4, 512 units 56.7 and 62.1.
  if (a.cols <= unit_columns(a.B, units, cus, 26))
    return once ? launch_units4<8, true>(a, stream) : launch_units4<8, false>(a, stream);
  return once ? launch_parts4<8, true>(a, stream) : launch_parts4<8, false>(a, stream);
}

}  // namespace lvspec
