// Attention of the draft rows over the paged cache in 4 bits (paged_mx_dev.h); parts, open rows and merges are those of
// the cache in 8 bits (paged_segment.h).
//
// A wave takes every KS-th tile of 64 keys of its workgroup's part.  A tile's codes lie in memory as the lanes take
// them: they are loaded straight into registers, 1 KiB in one piece per instruction, and widened to bf16 with their
// scales (exact).  S^T = K Q^T leaves a row's scores in the lanes that hold the values of their tokens, so
// probabilities (rounded to bf16, each by at most 2^-8 of itself) go into the second product where they are.
#include "paged_mx_dev.h"
#include "paged_segment.h"

namespace lvspec {

namespace {

// 32 query rows on 32x32 tiles: the tokens of a lane's scores are those of its values, element 16 t + r is token
// 32 t + 8 (r / 4) + 4 h + r % 4.
struct FourRows : WideRows {
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
  LVS_DEV void scores4(float (&s)[32], const u32x4 (&k)[4], uint32_t scales) const {
    const float f[4] = {scale4<0>(scales), scale4<1>(scales), scale4<2>(scales), scale4<3>(scales)};
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      f32x16 z;
#pragma unroll
      for (int r = 0; r < 16; ++r) z[r] = 0.f;
#pragma unroll
      for (int x = 0; x < 8; ++x) z = mfma32(widen4(k[2 * (x >> 2) + t][x & 3], f[2 * t + (x >> 2)]), q[x], z);
#pragma unroll
      for (int r = 0; r < 16; ++r) s[16 * t + r] = z[r];
    }
  }
  LVS_DEV void output4(const u32x4 (&pr)[4], const u32x4 (&v)[4], uint32_t scales) {
    const float f[4] = {scale4<0>(scales), scale4<1>(scales), scale4<2>(scales), scale4<3>(scales)};
#pragma unroll
    for (int y = 0; y < 4; ++y)
#pragma unroll
      for (int c = 0; c < 4; ++c) acc[c] = mfma32(widen4(v[c][y], f[c]), pr[y], acc[c]);
  }
};

// A tile in registers.
struct Tile {
  u32x4 k[4], v[4];
  uint32_t ks, vs;
  int id;
};

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

  LVS_DEV void load(Tile& x, int id, int h, int lane) const {
    x.id = id;
    const int64_t at = (int64_t)max(id, 0) * p.Hkv + h;
    const uint8_t* k = p.k8 + at * kPage4Bytes;
    const uint8_t* v = p.v8 + at * kPage4Bytes;
    const int off = (lane & 31) * 32 + (lane >> 5) * 16;
    x.ks = load_once<ONCE, uint32_t>(static_cast<const uint8_t*>(p.k_scale) + at * kScale4Bytes + lane * 4);
#pragma unroll
    for (int i = 0; i < 4; ++i) x.k[i] = load_once<ONCE, u32x4>(k + i * 1024 + off);
    x.vs = load_once<ONCE, uint32_t>(static_cast<const uint8_t*>(p.v_scale) + at * kScale4Bytes + lane * 4);
#pragma unroll
    for (int i = 0; i < 4; ++i) x.v[i] = load_once<ONCE, u32x4>(v + i * 1024 + off);
  }

  LVS_DEV void take(const Tile& x, int tile, int lane) {
    if (x.id < 0) return;                // (an entry that names no block of the pool: no key)
    float s[32];
    st.scores4(s, x.k, x.ks);
    this->softmax(s, tile * kPageTokens, kPageTokens, [&](int e) { return FourRows::key_of(lane, e); });
    u32x4 pr[4];
#pragma unroll
    for (int y = 0; y < 4; ++y)
      pr[y] = pack8(s[8 * y], s[8 * y + 1], s[8 * y + 2], s[8 * y + 3], s[8 * y + 4], s[8 * y + 5], s[8 * y + 6],
                    s[8 * y + 7]);
    st.output4(pr, x.v, x.vs);
  }

  // tiles t0 .. t1-1 of a unit
  LVS_DEV void blocks4(int b, int h, int t0, int t1) {
    const int mine = (t1 - t0 - stream + KS - 1) / KS;
    if (mine <= 0) return;
    const int lane = Base::lane_now();
    const int32_t* row = p.table + (int64_t)b * p.cols;
    int ids;                             // blocks of 64 tiles, one per lane; -1: no block of the pool
    auto fetch = [&](int j0) {
      const int t = t0 + stream + KS * (j0 + lane);
      ids = t < t1 ? row[t] : -1;
      ids = (uint32_t)ids < (uint32_t)p.n_blocks ? ids : -1;
    };
    auto next = [&](Tile& x, int j) {
      if (j >= mine) return;
      if ((j & 63) == 0) fetch(j);
      load(x, __builtin_amdgcn_readlane(ids, j & 63), h, lane);
    };
    Tile x, y;
    next(x, 0);
    for (int j = 0; j < mine; j += 2) {
      next(y, j + 1);
      take(x, t0 + stream + KS * j, lane);
      next(x, j + 2);
      if (j + 1 < mine) take(y, t0 + stream + KS * (j + 1), lane);
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
  if (o.p0 == 0) sg.open_rows(o.b, o.h, o.rc, L);
  sg.blocks4(o.b, o.h, o.t0, o.t1);
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
  sg.blocks4(b, h, 0, L >> kPageShift);
  sg.open_rows(b, h, rc, L);
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
  if (a.cols <= unit_columns(a.B, units, cus))
    return once ? launch_units4<8, true>(a, stream) : launch_units4<8, false>(a, stream);
  return once ? launch_parts4<8, true>(a, stream) : launch_parts4<8, false>(a, stream);
}

}  // namespace lvspec
