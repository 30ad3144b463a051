// Attention of the draft rows over the paged cache in 8 bits (paged_dev.h), the same contract as
// verification attention over a bf16 cache.
//
// Kernel 1 (split):   the complete blocks of all sequences and kv heads form one line of 64-key tiles, cut
//   into equal stretches; a workgroup takes one stretch, its streams of waves every KS-th tile of it.  The
//   open rows of a unit (sequence, kv head, row chunk), at most 95 in bf16, are taken by a workgroup of
//   their own.  A tile goes from memory into registers and from there into the matrix instructions:
//     keys:   16 bytes per lane are two operands of S^T = K Q^T after their conversion to bf16; which
//             channels a lane's operand holds is a permutation that K and Q share;
//     values: 16 bytes per lane are 16 tokens of one channel.  The tokens of a lane's scores, row block b
//             of S^T being tokens 16 (m/4) + 4 b + m%4, are then the tokens of its value operand, and
//             probabilities stay in their lane.
//   The conversion multiplies by the block's scale (a power of two): exact, and nothing is left to scale.
//   Softmax in base 2 with a running maximum, sums in 32 bits; probabilities are rounded to bf16 for the
//   second product (relative 2^-9 each, which averages out over the keys; it is what the matrix
//   instructions take).  The streams merge through LDS in fixed order into one record per segment.
// Kernel 2 (combine): merge of a row's records in fixed order, bf16 output.
#include "attn_rows32.h"
#include "paged_dev.h"

namespace lvspec {

namespace {

typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef uint16_t u16x2 __attribute__((ext_vector_type(2)));

constexpr int kMergeStride = 132;      // floats per row in the merge buffer: output and two sums
constexpr float kNegBig = -1.0e30f;
constexpr uint32_t kBufferWord = 0x00020000;      // last word of a buffer resource: raw, 32-bit data

// eight e4m3 times 2^e as bf16 (exact)
LVS_DEV u32x4 widen(uint32_t lo, uint32_t hi, float scale) {
  auto two = [&](uint32_t x, auto upper) {
    return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((int)x, scale, decltype(upper)::value));
  };
  return u32x4{two(lo, std::false_type{}), two(lo, std::true_type{}), two(hi, std::false_type{}), two(hi, std::true_type{})};
}

// ------------------------------------------------------------------------------ tiles to LDS
// A wave's ring: one slot of keys, one of values.  Sixteen lanes of an operand read hold sixteen tokens (or
// channels) and would ask memory for sixteen rows at a time, a cache line each; copies go row by row instead,
// and LDS has the 16-byte chunks of a row in an order in which the operand reads meet no bank twice: with
// the four passes of 16 lanes of such a read (lds_load16), chunk c of token t at c ^ (t>>1 & 1 | t>>4 << 1), chunk c
// of channel d at c ^ v_place(d >> 2).
constexpr int kRingBytes = 2 * kPageBytes;

LVS_DEV int v_place(int q) { return ((q >> 1) & 1) | (((q ^ (q >> 1)) & 1) << 1); }    // 0 2 3 1

// Eight copies of 1 KiB of a block of the pool to a slot, lane l of copy y from offset y * 1024 + o[y / 2].  No
// block: a buffer of no bytes, nothing is fetched and zeros are written.  (The compiler does not know them as
// LDS writes or loads: waits are wait_copies, and m0 is as before.)
template <bool ONCE>
LVS_DEV void copy_page(const uint8_t* pool, int id, int64_t head, uint32_t slot, int o0, int o1, int o2, int o3,
                       int n_heads) {
  const uint64_t at = (uint64_t)(pool + ((int64_t)max(id, 0) * n_heads + head) * kPageBytes);
  u32x4 from = {(uint32_t)at, (uint32_t)(at >> 32) & 0xffffu, id >= 0 ? (uint32_t)kPageBytes : 0u, kBufferWord};
#pragma unroll
  for (int i = 0; i < 4; ++i) from[i] = __builtin_amdgcn_readfirstlane(from[i]);      // (in scalar registers)
  const uint32_t to = __builtin_amdgcn_readfirstlane(slot);
  uint32_t keep, far;
#define LVS_COPY_1(O, POLICY) "buffer_load_dwordx4 " O ", %7, %1 offen" POLICY " lds\n\t"
#define LVS_COPY_NEXT "s_add_u32 m0, m0, 0x400\n\ts_add_u32 %1, %1, 0x400\n\ts_nop 0\n\t"
#define LVS_COPY(P)                                                                                   \
  asm volatile("s_mov_b32 %0, m0\n\ts_mov_b32 m0, %6\n\ts_mov_b32 %1, 0\n\ts_nop 0\n\t"                 \
               LVS_COPY_1("%2", P) LVS_COPY_NEXT LVS_COPY_1("%2", P) LVS_COPY_NEXT                    \
               LVS_COPY_1("%3", P) LVS_COPY_NEXT LVS_COPY_1("%3", P) LVS_COPY_NEXT                    \
               LVS_COPY_1("%4", P) LVS_COPY_NEXT LVS_COPY_1("%4", P) LVS_COPY_NEXT                    \
               LVS_COPY_1("%5", P) LVS_COPY_NEXT LVS_COPY_1("%5", P) "s_mov_b32 m0, %0"               \
               : "=&s"(keep), "=&s"(far) : "v"(o0), "v"(o1), "v"(o2), "v"(o3), "s"(to), "s"(from) : "memory", "scc")
  if constexpr (ONCE)
    LVS_COPY(" nt");
  else
    LVS_COPY("");
#undef LVS_COPY
#undef LVS_COPY_NEXT
#undef LVS_COPY_1
}

// ------------------------------------------------------------------------------ the line of tiles
// A unit (sequence, kv head, row chunk) has kOpenTiles places for its open rows, which take about as long as
// so many tiles, and a place per tile of 64 keys.  Two ways to divide them:
//   the line: all units one behind the other, sequence by sequence (HR = Hkv * n_rc units each), cut into
//     equal stretches, one per workgroup.  Nobody waits for anybody, but a stretch over the end of a unit is two
//     segments, and a segment has 5 us of its own (first loads, merge);
//   parts: every unit in equal parts of at most so many places that there are no more parts than workgroups.
// The line is taken where a stretch is long (kLineLeast).  Who has the first of a unit's places does its open rows.
// Every wave finds its place by itself.
constexpr int kOpenTiles = 8;
constexpr int kLineLeast = 32;
constexpr int kPartRounds = 5;

LVS_DEV int wave_scan(int x) {               // inclusive sum over the lanes
  auto add = [&](uint32_t y) { x += (int)y; };
  add(dpp_move<0x111, 0xf>(0u, (uint32_t)x));    // row_shr 1, 2, 4, 8
  add(dpp_move<0x112, 0xf>(0u, (uint32_t)x));
  add(dpp_move<0x114, 0xf>(0u, (uint32_t)x));
  add(dpp_move<0x118, 0xf>(0u, (uint32_t)x));
  add(dpp_move<0x142, 0xa>(0u, (uint32_t)x));    // row_bcast 15, 31
  add(dpp_move<0x143, 0xc>(0u, (uint32_t)x));
  return x;
}
LVS_DEV int last_lane(int x) { return __builtin_amdgcn_readlane(x, 63); }

LVS_DEV int full_blocks(const PagedAttnKernelArgs& p, int b) { return paged_len(p.kv_len[b], p.cols) >> kPageShift; }

struct Cut {
  int total;           // places of all units (line), or parts of all units
  int len;             // places of a stretch; 0: parts
  uint32_t inv;        // parts: about 2^32 / most places of a part
  // a sequence's share of the line, or the parts of one of its units
  LVS_DEV int share(int places) const { return places == 0 || len > 0 ? places : 1 + (int)__umulhi((uint32_t)(places - 1), inv); }
};

// Exact, but some thirty instructions one behind the other, a tenth of a microsecond; and about.
LVS_DEV int divide(int x, int d) { return (int)((uint32_t)x / (uint32_t)d); }
LVS_DEV int about(int x, int d) { return (int)((float)x * __builtin_amdgcn_rcpf((float)d)); }

// places of the units of sequences b0 .. b0+63, one per lane; 0 behind the last one
LVS_DEV int places_of(const PagedAttnKernelArgs& p, int b) { return b < p.B ? full_blocks(p, b) + kOpenTiles : 0; }

// places0: those of the first 64 sequences
template <int KS>
LVS_DEV Cut cut_units(const PagedAttnKernelArgs& p, int lane, int places0) {
  int sum = last_lane(wave_scan(places0)), most = (int)wave_max_u32((uint32_t)places0);
  for (int b0 = 64; b0 < p.B; b0 += 64) {
    const int x = places_of(p, b0 + lane);
    sum += last_lane(wave_scan(x));
    most = max(most, (int)wave_max_u32((uint32_t)x));
  }
  const int HR = p.Hkv * p.n_rc, units = p.B * HR, cus = p.n_wg >> 1;
  Cut c;
  const int total = sum * HR, stretch = (total + p.n_wg - 1) >> p.wg_shift;
  c.total = total;
  c.len = stretch;
  if (stretch >= kLineLeast) return c;
  // Parts for one workgroup per CU (and some more of open rows only), or, where those take many rounds of
  // the streams, for two.
  c.len = 0;
  int limit = max(cus, units) + min(units, cus >> 3), part = 0;
  for (int wide = 0; wide < 2; ++wide) {
    part = max((about(total, limit) + KS - 1) / KS * KS, kOpenTiles);
    while (true) {
      c.inv = (uint32_t)(4294967040.f * __builtin_amdgcn_rcpf((float)part));
      int n = last_lane(wave_scan(c.share(places0)));
      for (int b0 = 64; b0 < p.B; b0 += 64) n += last_lane(wave_scan(c.share(places_of(p, b0 + lane))));
      c.total = n * HR;
      if (c.total <= limit || part >= most) break;
      part += max(part >> 3, KS) / KS * KS;
    }
    if (part <= kPartRounds * KS || limit >= p.n_wg) break;
    limit = p.n_wg;
  }
  // lengths so unequal that the longest part is well above the average
  const int even = about(total, limit);
  if (stretch >= kLineLeast / 2 && min(part, most) > even + (even >> 1) + kOpenTiles) {
    c.total = total;
    c.len = stretch;
  }
  return c;
}

// ------------------------------------------------------------------------------ split
// NB blocks of 16 rows by KS streams of tiles, a wave each.
template <int NB, int KS>
struct Shape {
  static constexpr int kRows = 16 * NB;
  static constexpr int kMergeBytes = (int)sizeof(float) * KS * kRows * (1 + kMergeStride);
  static constexpr int kLds = kMergeBytes > KS * kRingBytes ? kMergeBytes : KS * kRingBytes;
};

template <int NB>
struct RowState {
  f32x4 acc[NB][8];        // O^T: channels 16 db + 4 g4 + i of row n16
  float m[NB], l[NB], lv[NB];
};

// Scores of NK blocks of 16 keys to probabilities (in place); the running maximum and the sums follow.
// `first`: there is nothing to rescale yet.  The maximum is exact: a reference that is taken anew only for
// scores 2^8 above it saves 1 to 4 % of the time and costs the exact 1 of the largest probability (error
// against 64 bits 2.2e-3 -> 2.5e-3).
template <int NB, int NK>
LVS_DEV void softmax_tile(RowState<NB>& st, f32x4 (&s)[NB][NK], float c, bool first) {
  bool grow = false;
  float top[NB];
#pragma unroll
  for (int nb = 0; nb < NB; ++nb) {
    float t = s[nb][0][0];
#pragma unroll
    for (int k = 0; k < NK; ++k)
#pragma unroll
      for (int i = 0; i < 4; ++i) t = fmaxf(t, s[nb][k][i]);
    top[nb] = t * c;
    grow |= top[nb] > st.m[nb];
  }
  if (__any(grow)) {
#pragma unroll
    for (int nb = 0; nb < NB; ++nb) {
      const float x = max_rows(max_halves(fmaxf(st.m[nb], top[nb])));
      const float alpha = fast_exp2(st.m[nb] - x);
      st.m[nb] = x;
      if (!first) {
        st.l[nb] *= alpha;
        st.lv[nb] *= alpha;
#pragma unroll
        for (int db = 0; db < 8; ++db) st.acc[nb][db] *= alpha;
      }
    }
  }
#pragma unroll
  for (int nb = 0; nb < NB; ++nb) {
    float sum = 0.f;
#pragma unroll
    for (int k = 0; k < NK; ++k) {
#pragma unroll
      for (int i = 0; i < 4; ++i) s[nb][k][i] = fast_exp2(__builtin_fmaf(s[nb][k][i], c, -st.m[nb]));
      sum += (s[nb][k][0] + s[nb][k][1]) + (s[nb][k][2] + s[nb][k][3]);
    }
    st.l[nb] += sum;
  }
}

// softmax mass on the video span; key_of(k, i): cache row of score i of block k
template <int NB, int NK, class KeyOf>
LVS_DEV void span_mass(RowState<NB>& st, const f32x4 (&s)[NB][NK], int key0, int keys, int vis_b, int vis_e,
                       KeyOf&& key_of) {
  if (!(key0 < vis_e && key0 + keys > vis_b)) return;
#pragma unroll
  for (int nb = 0; nb < NB; ++nb) {
    float sum = 0.f;
#pragma unroll
    for (int k = 0; k < NK; ++k)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int key = key_of(k, i);
        sum += key >= vis_b && key < vis_e ? s[nb][k][i] : 0.f;
      }
    st.lv[nb] += sum;
  }
}

LVS_DEV u32x4 pack8(const f32x4& a, const f32x4& b) {
  return u32x4{pack_bf16(a[0], a[1]), pack_bf16(a[2], a[3]), pack_bf16(b[0], b[1]), pack_bf16(b[2], b[3])};
}

// four channels of an output row; lane 0 of 32 its log-sum-exp and mass
LVS_DEV void write_row(const PagedAttnKernelArgs& p, int b, int h, int r, int l32, const f32x4& o, float m, float l,
                       float lv) {
  const int i = (int)fast_div((uint32_t)r, p.div_g), head = h * p.G + (r - i * p.G);
  const float inv = 1.f / l;
  uint2 y;
  y.x = pack_bf16(o[0] * inv, o[1] * inv);
  y.y = pack_bf16(o[2] * inv, o[3] * inv);
  *reinterpret_cast<uint2*>(p.out + (int64_t)b * p.o_sb + (int64_t)i * p.o_sg + (int64_t)head * p.o_sh + l32 * 4) = y;
  if (l32 == 0) {
    const int64_t at = ((int64_t)b * p.Hq + head) * p.gamma + i;
    // ln(sum of exp) from base 2: ln 2 * (m + log2 l)
    if (p.lse != nullptr) p.lse[at] = 0.69314718055994531f * (m + __log2f(l));
    if (p.vis_mass != nullptr) p.vis_mass[at] = lv / l;
  }
}

template <int NB, int KS, bool ONCE>
struct Segment {
  using W = Shape<NB, KS>;
  const PagedAttnKernelArgs& p;
  uint8_t* smem;
  int stream;
  u32x4 q[NB][4];          // channels 64 (c/2) + 16 g4 + 8 (c%2) .. +7 of row n16
  RowState<NB> st;
  int vis_b, vis_e;
  bool fresh;              // nothing in the state yet

  LVS_DEV Segment(const PagedAttnKernelArgs& a, uint8_t* lds) : p(a), smem(lds) {
    stream = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  }

  // The lane's number, row or token (n16) and quarter (g4).  Every part of a segment takes them anew: what
  // follows from them would else be held in registers through the loop over the tiles.
  struct Lane {
    int lane, n16, g4;
    LVS_DEV Lane() {
      lane = threadIdx.x & 63;
      asm volatile("" : "+v"(lane));
      n16 = lane & 15;
      g4 = lane >> 4;
    }
  };

  LVS_DEV void begin(int b, int h, int rc) {
    const Lane me;
    const int n16 = me.n16, g4 = me.g4;
#pragma unroll
    for (int nb = 0; nb < NB; ++nb) {
      const int r = rc * p.rpad + nb * 16 + n16;
      const int rcl = r < p.R ? r : p.R - 1;     // (rows past the last one: that row again, to no output)
      const int qi = (int)fast_div((uint32_t)rcl, p.div_g);
      const uint16_t* qp = p.q + (int64_t)b * p.q_sb + (int64_t)qi * p.q_sg +
                           (int64_t)(h * p.G + (rcl - qi * p.G)) * p.q_sh;
#pragma unroll
      for (int c = 0; c < 4; ++c)
        q[nb][c] = *reinterpret_cast<const u32x4*>(qp + 64 * (c >> 1) + 16 * g4 + 8 * (c & 1));
#pragma unroll
      for (int db = 0; db < 8; ++db) st.acc[nb][db] = f32x4{0.f, 0.f, 0.f, 0.f};
      st.m[nb] = kNegBig;
      st.l[nb] = st.lv[nb] = 0.f;
    }
    fresh = true;
    vis_b = vis_e = 0;
    if (p.vis_begin != nullptr) {
      vis_b = __builtin_amdgcn_readfirstlane(p.vis_begin[b]);
      vis_e = __builtin_amdgcn_readfirstlane(p.vis_end[b]);
    }
  }

  // tiles t0 .. t1-1 of a unit
  LVS_DEV void blocks(int b, int h, int t0, int t1) {
    const int mine = (t1 - t0 - stream + KS - 1) / KS;
    if (mine <= 0) return;
    const Lane me;
    const int lane = me.lane, n16 = me.n16, g4 = me.g4;
    const int32_t* row = p.table + (int64_t)b * p.cols;
    // blocks of 64 tiles, one per lane.  An entry that names no block of the pool is -1.
    int ids;
    auto fetch = [&](int j0) {
      const int t = t0 + stream + KS * (j0 + lane);
      ids = t < t1 ? row[t] : -1;
      ids = (uint32_t)ids < (uint32_t)p.n_blocks ? ids : -1;
      asm volatile("" : "+v"(ids));      // (waited for here: the loop has no loads but its copies)
    };
    // scales by scalar loads, which do not count among the copies
    auto scale_of = [&](const float* scale, int id) {
      return *(const __attribute__((address_space(4))) float*)(uintptr_t)(scale + ((int64_t)max(id, 0) * p.Hkv + h));
    };
    const uint32_t k_slot = lds_addr(smem) + stream * kRingBytes, v_slot = k_slot + kPageBytes;
    // global side of the copies: row and chunk that belong at lane's place (see k_place, v_place)
    const int k_from = (lane >> 3) * 128, k_chunk = (lane & 7) ^ ((lane >> 4) & 1);
    int k_off[4];
#pragma unroll
    for (int y = 0; y < 4; ++y) k_off[y] = k_from + ((k_chunk ^ (y << 1)) << 4);
    const int v_off = (lane >> 2) * kPageTokens + (((lane & 3) ^ v_place(lane >> 4)) << 4);
    auto copy_k = [&](int id) { copy_page<ONCE>(p.k8, id, h, k_slot, k_off[0], k_off[1], k_off[2], k_off[3], p.Hkv); };
    auto copy_v = [&](int id) { copy_page<ONCE>(p.v8, id, h, v_slot, v_off, v_off, v_off, v_off, p.Hkv); };
    // LDS side of the operands: token 16 (n16/4) + 4 kb + n16%4, chunk 4 half + g4; channel 16 x + n16, chunk g4
    const uint32_t k_at = k_slot + (16 * (n16 >> 2) + (n16 & 3)) * 128;
    const int k_key = ((n16 >> 1) & 1) | ((n16 >> 2) << 1);
    const uint32_t k_at0 = k_at + ((g4 ^ k_key) << 4), k_at1 = k_at + (((4 + g4) ^ k_key) << 4);
    const uint32_t v_at = v_slot + n16 * kPageTokens + ((g4 ^ v_place(n16 >> 2)) << 4);
    fetch(0);
    int id = __builtin_amdgcn_readlane(ids, 0);
    copy_k(id);
    copy_v(id);
    float k_scale = scale_of(p.k_scale, id), v_scale = scale_of(p.v_scale, id);
    const float c = p.scale_log2e;
    for (int j = 0; j < mine; ++j) {
      const bool more = j + 1 < mine;
      if (((j + 1) & 63) == 0) fetch(j + 1);
      const int next = more ? __builtin_amdgcn_readlane(ids, (j + 1) & 63) : -1;
      u32x4 k[8];
      wait_copies<8>();                // all but V's
#pragma unroll
      for (int kb = 0; kb < 4; ++kb) {
        k[2 * kb] = lds_load16(k_at0 + kb * 512);
        k[2 * kb + 1] = lds_load16(k_at1 + kb * 512);
      }
      asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
      if (more) copy_k(next);
      const float k_next = scale_of(p.k_scale, next), v_next = scale_of(p.v_scale, next);
      f32x4 s[NB][4];
#pragma unroll
      for (int kb = 0; kb < 4; ++kb) {
#pragma unroll
        for (int nb = 0; nb < NB; ++nb) s[nb][kb] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int x = 0; x < 4; ++x) {
          const u32x4& raw = k[kb * 2 + (x >> 1)];
          const u32x4 a = widen(raw[(x & 1) * 2], raw[(x & 1) * 2 + 1], k_scale);
#pragma unroll
          for (int nb = 0; nb < NB; ++nb) s[nb][kb] = mfma16(a, q[nb][x], s[nb][kb]);
        }
      }
      u32x4 pr[NB][2];
      if (id >= 0) {
        softmax_tile<NB, 4>(st, s, c, fresh);
        fresh = false;
        const int key0 = (t0 + stream + KS * j) * kPageTokens;
        span_mass<NB, 4>(st, s, key0, kPageTokens, vis_b, vis_e,
                         [&](int kb, int i) { return key0 + 16 * g4 + 4 * kb + i; });
#pragma unroll
        for (int nb = 0; nb < NB; ++nb) {
          pr[nb][0] = pack8(s[nb][0], s[nb][1]);
          pr[nb][1] = pack8(s[nb][2], s[nb][3]);
        }
      }
      u32x4 v[8];
      if (more)
        wait_copies<8>();              // all but the next K's
      else
        wait_copies<0>();
#pragma unroll
      for (int x = 0; x < 8; ++x) v[x] = lds_load16(v_at + x * 1024);
      asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
      if (more) copy_v(next);
      if (id >= 0) {
#pragma unroll
        for (int db = 0; db < 8; ++db)
#pragma unroll
          for (int y = 0; y < 2; ++y) {
            const u32x4 a = widen(v[db][2 * y], v[db][2 * y + 1], v_scale);
#pragma unroll
            for (int nb = 0; nb < NB; ++nb) st.acc[nb][db] = mfma16(a, pr[nb][y], st.acc[nb][db]);
          }
      }
      id = next;
      k_scale = k_next;
      v_scale = v_next;
    }
  }

  // Makes values that are not finite zero; bit r: row r of the 32 has some.
  LVS_DEV uint32_t take_out(u32x4 (&v)[8]) {
    uint32_t rows = 0;
#pragma unroll
    for (int x = 0; x < 8; ++x) {
      bool bad = false;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const bool lo = (v[x][i] & 0x7f80u) == 0x7f80u, hi = (v[x][i] & 0x7f800000u) == 0x7f800000u;
        bad |= lo || hi;
        v[x][i] = (lo ? 0u : v[x][i] & 0xffffu) | (hi ? 0u : v[x][i] & 0xffff0000u);
      }
      const unsigned long long at = __ballot(bad);
#pragma unroll
      for (int i = 0; i < 4; ++i) rows |= ((at >> (16 * i)) & 0xffffull) != 0ull ? 1u << (4 * x + i) : 0u;
    }
    return rows;
  }

  // open rows: positions L / 64 * 64 .. L + gamma - 1, in pieces of 32 keys, one stream each
  LVS_DEV void open_rows(int b, int h, int rc, int L) {
    const Lane me;
    const int n16 = me.n16, g4 = me.g4;
    const int base = L & ~(kPageTokens - 1);
    const int n = L - base + p.gamma;
    uint32_t rowmask[NB];            // draft rows that row n16 sees
#pragma unroll
    for (int nb = 0; nb < NB; ++nb) {
      const int r = rc * p.rpad + nb * 16 + n16;
      rowmask[nb] = p.draft_mask[fast_div((uint32_t)(r < p.R ? r : p.R - 1), p.div_g)] & (0xffffffffu >> (32 - p.gamma));
    }
    const int64_t unit = ((int64_t)b * p.Hkv + h) * (kTailRows * kRowBytes);
    const uint8_t* kt = p.k_tail + unit;
    const uint8_t* vt = p.v_tail + unit;
    const uint32_t turn = lds_addr(smem) + stream * kRingBytes;
    const float c = p.scale_log2e;
    // (from the last stream on: the first ones have the odd tiles)
    for (int piece = KS - 1 - stream; piece * 32 < n; piece += KS) {
      const int p0 = base + piece * 32;
      u32x4 k[2][4], v[8];
#pragma unroll
      for (int kb = 0; kb < 2; ++kb)
#pragma unroll
        for (int x = 0; x < 4; ++x)
          k[kb][x] = *reinterpret_cast<const u32x4*>(kt + ((p0 + 16 * kb + n16) & (kTailRows - 1)) * kRowBytes +
                                                     2 * (64 * (x >> 1) + 16 * g4 + 8 * (x & 1)));
#pragma unroll
      for (int x = 0; x < 8; ++x)
        v[x] = *reinterpret_cast<const u32x4*>(vt + ((p0 + 4 * x + g4) & (kTailRows - 1)) * kRowBytes + n16 * 16);
      // Rows behind the last draft are nobody's: zero.  A value that is not finite would reach rows that do
      // not see its key, as 0 * inf: it is zero here as well, and its rows are remembered for below.
      uint32_t odd = 0;
      u16x2 top = {0, 0};
#pragma unroll
      for (int x = 0; x < 8; ++x) {
        v[x] = p0 + 4 * x + g4 < L + p.gamma ? v[x] : u32x4{0u, 0u, 0u, 0u};
#pragma unroll
        for (int i = 0; i < 4; ++i) top = __builtin_elementwise_max(top, __builtin_bit_cast(u16x2, v[x][i] & 0x7fff7fffu));
      }
      if (__any(top[0] >= 0x7f80 || top[1] >= 0x7f80)) odd = take_out(v);
#pragma unroll
      for (int x = 0; x < 8; ++x) {
        const int r = 4 * x + g4;
        *(__attribute__((address_space(3))) u32x4*)(uintptr_t)(turn + r * kRowBytes +
                                                               ((n16 ^ rows32_swz(r & 15)) << 4)) = v[x];
      }
      f32x4 s[NB][2];
#pragma unroll
      for (int nb = 0; nb < NB; ++nb)
#pragma unroll
        for (int kb = 0; kb < 2; ++kb) {
          f32x4 z = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
          for (int x = 0; x < 4; ++x) z = mfma16(k[kb][x], q[nb][x], z);
          // bit k: row n16 sees key k of the piece; committed keys first, then the draft rows
          const int old = L - p0;
          const uint32_t sees = old >= 32 ? 0xffffffffu
                                : old >= 0 ? ((1u << old) - 1u) | (rowmask[nb] << old) : rowmask[nb] >> min(-old, 31);
#pragma unroll
          for (int i = 0; i < 4; ++i) z[i] = (sees >> (4 * g4)) & (1u << (16 * kb + i)) ? z[i] : -INFINITY;
          s[nb][kb] = z;
        }
      softmax_tile<NB, 2>(st, s, c, fresh);
      fresh = false;
      span_mass<NB, 2>(st, s, p0, 32, vis_b, vis_e, [&](int kb, int i) { return p0 + 16 * kb + 4 * g4 + i; });
      u32x4 pr[NB];
#pragma unroll
      for (int nb = 0; nb < NB; ++nb) pr[nb] = pack8(s[nb][0], s[nb][1]);
      asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
      const int tr = 4 * g4 + (n16 >> 2);                      // row and chunk this lane hands in
#pragma unroll
      for (int db = 0; db < 8; ++db) {
        const uint32_t at = turn + ((((2 * db + ((n16 & 3) >> 1)) ^ rows32_swz(tr)) << 4) | ((n16 & 1) << 3));
        const u32x2 lo = lds_load_tr(at + tr * kRowBytes);
        const u32x2 hi = lds_load_tr(at + (16 + tr) * kRowBytes);
        const u32x4 a = u32x4{lo[0], lo[1], hi[0], hi[1]};
#pragma unroll
        for (int nb = 0; nb < NB; ++nb) st.acc[nb][db] = mfma16(a, pr[nb], st.acc[nb][db]);
      }
      // (any weight times a value that is not finite is that value: it is added as it is)
      while (odd != 0u) {
        const int key = __builtin_ctz(odd);
        odd &= odd - 1;
        const int j = p0 + key - L;
        const uint8_t* vr = vt + ((p0 + key) & (kTailRows - 1)) * kRowBytes;
#pragma unroll
        for (int db = 0; db < 8; ++db) {
          const uint2 x = *reinterpret_cast<const uint2*>(vr + 2 * (16 * db + 4 * g4));
          const f32x4 y = {__builtin_bit_cast(float, x.x << 16), __builtin_bit_cast(float, x.x & 0xffff0000u),
                           __builtin_bit_cast(float, x.y << 16), __builtin_bit_cast(float, x.y & 0xffff0000u)};
#pragma unroll
          for (int nb = 0; nb < NB; ++nb) {
            const bool sees = j < 0 || ((rowmask[nb] >> (j < 0 ? 0 : j)) & 1u) != 0u;
#pragma unroll
            for (int i = 0; i < 4; ++i)
              st.acc[nb][db][i] += sees && !(fabsf(y[i]) <= 3.4028234663852886e38f) ? y[i] : 0.f;
          }
        }
      }
    }
  }

  // streams that have something of a segment of n tiles, and of the open rows or not
  LVS_DEV uint32_t active(int n, bool open, int L) {
    uint32_t on = n >= KS ? (1u << KS) - 1u : (1u << max(n, 0)) - 1u;
    if (open) {
      const int pieces = ((L & (kPageTokens - 1)) + p.gamma + 31) >> 5;      // at most 3
      on |= ((1u << KS) - 1u) & ~((1u << max(KS - pieces, 0)) - 1u);
    }
    return on;
  }

  // The active streams' states to LDS, each brought to the row's common maximum first, so that what is left is
  // sums: [KS][kRows] maxima, then per stream and row 132 floats, the output, the denominator and its share
  // on the video span.
  LVS_DEV void gather(uint32_t on) {
    const Lane me;
    const int n16 = me.n16, g4 = me.g4;
    float* sm_m = reinterpret_cast<float*>(smem);
    __syncthreads();
    if (g4 == 0) {
#pragma unroll
      for (int nb = 0; nb < NB; ++nb) sm_m[stream * W::kRows + nb * 16 + n16] = st.m[nb];
    }
    __syncthreads();
    if (((on >> stream) & 1u) == 0u) return;
#pragma unroll
    for (int nb = 0; nb < NB; ++nb) {
      const int row = nb * 16 + n16;
      float mm = sm_m[row];
#pragma unroll
      for (int k = 1; k < KS; ++k) mm = fmaxf(mm, sm_m[k * W::kRows + row]);
      const float f = fast_exp2(st.m[nb] - mm);
      float* o = sm_m + KS * W::kRows + (stream * W::kRows + row) * kMergeStride;
#pragma unroll
      for (int db = 0; db < 8; ++db) *reinterpret_cast<f32x4*>(o + 16 * db + 4 * g4) = st.acc[nb][db] * f;
      float l = st.l[nb] * f, lv = st.lv[nb] * f;
      l += xor_shuffle(l, 16);
      l += xor_shuffle(l, 32);
      lv += xor_shuffle(lv, 16);
      lv += xor_shuffle(lv, 32);
      if (g4 == 0) *reinterpret_cast<float2*>(o + 128) = float2{l, lv};
    }
  }

  // sums over the active streams of four floats of a row
  LVS_DEV f32x4 merged(uint32_t on, int row, int c4) {
    const float* o = reinterpret_cast<const float*>(smem) + KS * W::kRows + row * kMergeStride + c4;
    f32x4 sum = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int k = 0; k < KS; ++k)
      if ((on >> k) & 1u) sum += *reinterpret_cast<const f32x4*>(o + k * W::kRows * kMergeStride);
    return sum;
  }
  LVS_DEV float merged_max(int row) {
    const float* sm_m = reinterpret_cast<const float*>(smem);
    float mm = sm_m[row];
#pragma unroll
    for (int k = 1; k < KS; ++k) mm = fmaxf(mm, sm_m[k * W::kRows + row]);
    return mm;
  }

  // the merged state into a record
  LVS_DEV void end(uint32_t on, int rc, float* rec) {
    gather(on);
    __syncthreads();
    const int rows = min(p.R - rc * p.rpad, p.rpad);
    for (int idx = threadIdx.x; idx < rows * 32; idx += 64 * KS) {
      const int row = idx >> 5, l32 = idx & 31;
      *reinterpret_cast<f32x4*>(rec + 3 * p.rpad + row * 128 + l32 * 4) = merged(on, row, l32 * 4);
    }
    for (int row = threadIdx.x; row < rows; row += 64 * KS) {
      const f32x4 l = merged(on, row, 128);
      rec[row] = merged_max(row);
      rec[p.rpad + row] = l[0];
      rec[2 * p.rpad + row] = l[1];
    }
  }

  // the merged state of a whole unit into the outputs
  LVS_DEV void finish(uint32_t on, int b, int h, int rc) {
    gather(on);
    __syncthreads();
    const int rows = min(p.R - rc * p.rpad, p.rpad);
    for (int idx = threadIdx.x; idx < rows * 32; idx += 64 * KS) {
      const int row = idx >> 5, l32 = idx & 31;
      const f32x4 l = merged(on, row, 128);
      write_row(p, b, h, rc * p.rpad + row, l32, merged(on, row, l32 * 4), merged_max(row), l[0], l[1]);
    }
  }
};

LVS_DEV float* record_at(const PagedAttnKernelArgs& p, int64_t i) { return p.ws + i * ((int64_t)p.rpad * 131); }

template <int NB, int KS, bool ONCE>
__global__ __launch_bounds__(64 * KS, 2) void paged_attn_kernel(PagedAttnKernelArgs p) {
  extern __shared__ __align__(256) uint8_t smem[];
  Segment<NB, KS, ONCE> sg(p, smem);
  const int HR = p.Hkv * p.n_rc, lane = threadIdx.x & 63;
  const int places0 = places_of(p, lane);
  const Cut cut = cut_units<KS>(p, lane, places0);
  const int len = max(cut.len, 1);
  const int used = cut.len > 0 ? divide(cut.total + len - 1, len) : cut.total;       // workgroups with work
  // work that follows each other goes to one XCD, which has the records of a unit in its L2
  const int each = (used + 7) >> 3;
  const int w = (blockIdx.x & 7) * each + (blockIdx.x >> 3);
  if ((int)(blockIdx.x >> 3) >= each || w >= used) return;
  int at = w * len;
  const int end = min(at + len, cut.total);
  bool again = false;
  int b0 = 0, before = 0;                        // sequences b0 .. b0+63 at hand, shares before them
  int places = places0, upto = wave_scan(cut.share(places));
  while (at < end) {
    int all = last_lane(upto);
    while (at >= all * HR) {                     // (ends: at < total)
      b0 += 64;
      before = all;
      places = places_of(p, b0 + lane);
      upto = before + wave_scan(cut.share(places));
      all = last_lane(upto);
    }
    const int in = __popcll(__ballot(at >= upto * HR));
    const int unit_places = __builtin_amdgcn_readlane(places, in);
    const int mine = cut.share(unit_places);
    const int y = at - (__builtin_amdgcn_readlane(upto, in) - mine) * HR;
    const int hr = divide(y, mine), x = y - hr * mine;
    const int b = b0 + in, h = ONCE ? hr : divide(hr, p.n_rc), rc = hr - h * p.n_rc;
    int p0 = x, p1 = min(mine, x + end - at);    // places of the unit
    at += p1 - p0;
    if (cut.len == 0) {
      const int q = divide(unit_places, mine), r = unit_places - q * mine;      // the first r have one more
      p0 = x * q + min(x, r);
      p1 = p0 + q + (x < r ? 1 : 0);
    }
    if (p0 > 0 && p1 <= kOpenTiles) continue;    // (only places of open rows, not the first)
    const int t0 = max(p0 - kOpenTiles, 0), t1 = p1 - kOpenTiles;
    if (again) __syncthreads();                  // (the segment before this one has been read from LDS)
    again = true;
    const int L = p0 == 0 ? paged_len(p.kv_len[b], p.cols) : 0;      // (for the open rows)
    sg.begin(b, h, rc);
    if (p0 == 0) sg.open_rows(b, h, rc, L);
    sg.blocks(b, h, t0, t1);
    const uint32_t on = sg.active(t1 - t0, p0 == 0, L);
    if (cut.len == 0 && mine == 1)
      sg.finish(on, b, h, rc);
    else
      sg.end(on, rc, record_at(p, cut.len > 0 ? (int64_t)w + (int64_t)b * HR + hr : w));
  }
}

// One workgroup per unit, straight to the output: for tables so narrow that cutting a unit does not pay.
template <int NB, int KS, bool ONCE>
__global__ __launch_bounds__(64 * KS, 2) void paged_attn_unit_kernel(PagedAttnKernelArgs p) {
  extern __shared__ __align__(256) uint8_t smem[];
  Segment<NB, KS, ONCE> sg(p, smem);
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
// all eight of a workgroup where a unit has many records, or one group per row.
constexpr int kCombineThreads = 256;

template <int SPLIT, int KS>
__global__ __launch_bounds__(kCombineThreads) void paged_combine_kernel(PagedAttnKernelArgs p) {
  constexpr int kRows = 8 / SPLIT;               // output rows of a workgroup, all of one unit
  constexpr int kAhead = 8;
  __shared__ float s_m[8], s_l[8], s_v[8];
  __shared__ f32x4 s_o[SPLIT > 1 ? 8 : 1][32];
  const int tid = threadIdx.x, lane = tid & 63, g = tid >> 5, l32 = tid & 31;
  const int HR = p.Hkv * p.n_rc;
  const int per_unit = (p.rpad + kRows - 1) / kRows;
  const int unit = (int)((uint32_t)blockIdx.x / (uint32_t)per_unit);
  const int b = (int)((uint32_t)unit / (uint32_t)HR), hr = unit - b * HR;
  const int h = (int)((uint32_t)hr / (uint32_t)p.n_rc), rc = hr - h * p.n_rc;
  const int in = (blockIdx.x - unit * per_unit) * kRows + g / SPLIT, r = rc * p.rpad + in;
  const bool row = in < p.rpad && r < p.R;
  // where the unit lies, and whose records are its own
  int places = places_of(p, lane);
  const Cut cut = cut_units<KS>(p, lane, places);
  int before = 0, share = 0;
  for (int b0 = 0; b0 <= b; b0 += 64) {
    if (b0 > 0) places = places_of(p, b0 + lane);
    const int f = cut.share(places);
    const int upto = wave_scan(f);
    if (b < b0 + 64) {
      share = __builtin_amdgcn_readlane(f, b - b0);
      before += __builtin_amdgcn_readlane(upto, b - b0) - share;
    } else {
      before += last_lane(upto);
    }
  }
  if (cut.len == 0 && share == 1) return;        // (one part: it has written the output)
  const int from = before * HR + hr * share;
  const int64_t step = (int64_t)p.rpad * 131;
  int64_t at0 = from, skip = 0;                  // first record, and records between it and the others
  int n = share;
  if (cut.len > 0) {
    // the stretch of the first place, and those from the first tile's to the last one's
    const int first = divide(from, cut.len), full = share - kOpenTiles;
    const int next = full > 0 ? max(divide(from + kOpenTiles, cut.len), first + 1) : first + 1;
    n = full > 0 ? max(divide(from + share - 1, cut.len) - next + 2, 1) : 1;
    at0 = (int64_t)first + unit;
    skip = (next - first - 1) * step;
  }
  const float* rec = record_at(p, at0) + (row ? in : 0);
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
      const int64_t off = at * step + (at > 0 ? skip : 0);
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

// Columns of a table up to which every unit is one workgroup's.  The longest sequence may have as many blocks, so the
// more units there are, the more of them pay: they fill the chip anyway.
int64_t unit_columns(int64_t units, int64_t cus) {
  if (units >= 2 * cus) return (int64_t)1 << 30;
  return units >= cus ? 64 : units >= cus / 4 ? 32 : 20;
}

template <int NB, int KS, bool ONCE>
hipError_t launch_line(const PagedAttnKernelArgs& a, hipStream_t stream) {
  static LdsLimitOnce limit;
  constexpr size_t lds = Shape<NB, KS>::kLds;
  hipError_t e = limit.ensure(reinterpret_cast<const void*>(&paged_attn_kernel<NB, KS, ONCE>), lds);
  if (e != hipSuccess) return e;
  const unsigned units = (unsigned)(a.B * a.Hkv * a.n_rc);
  // (a part for every unit at least; the grid is a multiple of 8)
  const unsigned wgs = ((units > (unsigned)a.n_wg ? units : (unsigned)a.n_wg) + 7) / 8 * 8;
  paged_attn_kernel<NB, KS, ONCE><<<dim3(wgs), dim3(64 * KS), lds, stream>>>(a);
  e = hipGetLastError();
  if (e != hipSuccess) return e;
  // records of a unit, about: n_wg / units + 1
  if ((int64_t)units * 8 > a.n_wg)
    paged_combine_kernel<1, KS><<<dim3(units * (unsigned)((a.rpad + 7) / 8)), dim3(kCombineThreads), 0, stream>>>(a);
  else
    paged_combine_kernel<8, KS><<<dim3(units * (unsigned)a.rpad), dim3(kCombineThreads), 0, stream>>>(a);
  return hipGetLastError();
}

template <int NB, int KS, bool ONCE>
hipError_t launch_units(const PagedAttnKernelArgs& a, hipStream_t stream) {
  static LdsLimitOnce limit;
  constexpr size_t lds = Shape<NB, KS>::kLds;
  hipError_t e = limit.ensure(reinterpret_cast<const void*>(&paged_attn_unit_kernel<NB, KS, ONCE>), lds);
  if (e != hipSuccess) return e;
  const unsigned units = (unsigned)(a.B * a.Hkv * a.n_rc);
  paged_attn_unit_kernel<NB, KS, ONCE><<<dim3(units), dim3(64 * KS), lds, stream>>>(a);
  return hipGetLastError();
}

}  // namespace

int paged_attn_workgroups(int num_cu) {
  int n = 8;
  while (2 * n <= 2 * num_cu && n < 1024) n *= 2;
  return n;
}

hipError_t launch_paged_attn(const PagedAttnKernelArgs& a, hipStream_t stream) {
  const bool once = a.n_rc == 1;
  const int64_t units = (int64_t)a.B * a.Hkv * a.n_rc, cus = a.n_wg / 2;
  if (a.cols <= unit_columns(units, cus)) {
    if (a.rpad <= 16) return once ? launch_units<1, 8, true>(a, stream) : launch_units<1, 8, false>(a, stream);
    return once ? launch_units<2, 8, true>(a, stream) : launch_units<2, 8, false>(a, stream);
  }
  if (a.rpad <= 16) return once ? launch_line<1, 4, true>(a, stream) : launch_line<1, 4, false>(a, stream);
  return once ? launch_line<2, 4, true>(a, stream) : launch_line<2, 4, false>(a, stream);
}

}  // namespace lvspec
