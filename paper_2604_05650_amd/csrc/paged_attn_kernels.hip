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
#include "attn_rows32.h"
#include "paged_dev.h"

namespace lvspec {

namespace {

typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef uint16_t u16x2 __attribute__((ext_vector_type(2)));

constexpr int kMergeStride = 132;      // floats per row in the merge buffer: output and two sums
constexpr float kNegBig = -3.4028234663852886e38f;      // below every finite score: a maximum of nothing, with no inf - inf
constexpr uint32_t kBufferWord = 0x00020000;      // last word of a buffer resource: raw, 32-bit data

// eight e4m3 times 2^e as bf16 (exact)
LVS_DEV u32x4 widen(uint32_t lo, uint32_t hi, float scale) {
  auto two = [&](uint32_t x, auto upper) {
    return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((int)x, scale, decltype(upper)::value));
  };
  return u32x4{two(lo, std::false_type{}), two(lo, std::true_type{}), two(hi, std::false_type{}), two(hi, std::true_type{})};
}

// ------------------------------------------------------------------------------ tiles to LDS
// A wave's ring: one slot of keys, one of values.  An operand read has as many tokens (or channels) as lanes and
// would ask memory for as many rows at a time, a cache line each; copies go row by row instead, and LDS has the
// 16-byte chunks of a row in an order in which the operand reads meet no bank twice: chunk c of token t at
// c ^ k_place(t), chunk c of channel d at c ^ v_place(d / 4), functions of the core (Rows16, WideRows).
constexpr int kRingBytes = 2 * kPageBytes;

// Eight copies of 1 KiB of a block of the pool to a slot, lane l of copy y from offset y * 1024 + o[y].  No
// block: a buffer of no bytes, nothing is fetched.  (The compiler does not know them as LDS writes or loads:
// waits are wait_copies, and m0 is as before.)
template <bool ONCE>
LVS_DEV void copy_page(const uint8_t* pool, int id, int64_t head, int n_heads, uint32_t slot, const int (&o)[8]) {
  const uint64_t at = (uint64_t)(pool + ((int64_t)max(id, 0) * n_heads + head) * kPageBytes);
  u32x4 from = {(uint32_t)at, (uint32_t)(at >> 32) & 0xffffu, id >= 0 ? (uint32_t)kPageBytes : 0u, kBufferWord};
#pragma unroll
  for (int i = 0; i < 4; ++i) from[i] = __builtin_amdgcn_readfirstlane(from[i]);      // (in scalar registers)
  const uint32_t to = __builtin_amdgcn_readfirstlane(slot);
  uint32_t keep, far;
#define LVS_COPY_1(O, P) "buffer_load_dwordx4 " O ", %11, %1 offen" P " lds\n\t"
#define LVS_COPY_NEXT "s_add_u32 m0, m0, 0x400\n\ts_add_u32 %1, %1, 0x400\n\ts_nop 0\n\t"
#define LVS_COPY(P)                                                                                   \
  asm volatile("s_mov_b32 %0, m0\n\ts_mov_b32 m0, %10\n\ts_mov_b32 %1, 0\n\ts_nop 0\n\t"                \
               LVS_COPY_1("%2", P) LVS_COPY_NEXT LVS_COPY_1("%3", P) LVS_COPY_NEXT                    \
               LVS_COPY_1("%4", P) LVS_COPY_NEXT LVS_COPY_1("%5", P) LVS_COPY_NEXT                    \
               LVS_COPY_1("%6", P) LVS_COPY_NEXT LVS_COPY_1("%7", P) LVS_COPY_NEXT                    \
               LVS_COPY_1("%8", P) LVS_COPY_NEXT LVS_COPY_1("%9", P) "s_mov_b32 m0, %0"               \
               : "=&s"(keep), "=&s"(far)                                                             \
               : "v"(o[0]), "v"(o[1]), "v"(o[2]), "v"(o[3]), "v"(o[4]), "v"(o[5]), "v"(o[6]), "v"(o[7]), "s"(to), \
                 "s"(from)                                                                           \
               : "memory", "scc")
  if constexpr (ONCE)
    LVS_COPY(" nt");
  else
    LVS_COPY("");
#undef LVS_COPY
#undef LVS_COPY_NEXT
#undef LVS_COPY_1
}

// ------------------------------------------------------------------------------ parts
// A unit has kOpenTiles places for its open rows, which take about as long as so many tiles, and a place per
// tile of 64 keys.  Every unit is cut into equal parts of at most so many places that there are no more parts
// than compute units (or units, if they are more); who has the first of a unit's places does its open rows.
// The lengths are on the device, so every wave finds the cut and its place by itself; a unit's first part
// leaves a note of its records for the merge.
// One workgroup of four waves per CU draws the 27 GB/s that are the CU's share of the memory's rate, and each
// part has 5 us of its own (first loads, merge, record).  For two per CU: 8 x 8000 keys, 40/8 heads, 8 rows
// 46.2 us against 38.5 here, 2 x 16000, 30 rows 50.4 and 44.8, 32 x 6000, 5 rows 84 and 69; equal
// stretches of one line of all units, whatever their ends: 16 x (2048 to 32768) keys 79 and 74.
// Where lengths are so ragged that whole parts leave the longest half as long again as an even share, there
// may be more: 32 x (500 to 60000) keys, 256 units, 298 us without this and 155 with it, 48 x (100 to 20000)
// 125 and 89.  Everywhere, it costs: 24 x 5000, 7 rows 26.8 and 33.9, 16 x (2048 to 32768) keys 74 and 80.
constexpr int kOpenTiles = 8;
constexpr int kRound = 4;          // tiles that four streams take at a time; any number: 16384 keys 16.7, so 16.0

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

// Exact, but some thirty instructions one behind the other, a tenth of a microsecond; and about.
LVS_DEV int divide(int x, int d) { return (int)((uint32_t)x / (uint32_t)d); }
LVS_DEV int about(int x, int d) { return (int)((float)x * __builtin_amdgcn_rcpf((float)d)); }

// Places of the units of sequences `per` lane .. `per` lane + `per` - 1; 0 behind the last one.
constexpr int kPer = 4;
struct Places {
  int per, of[kPer];
  LVS_DEV Places(const PagedAttnKernelArgs& p, int lane) : per((p.B + 63) >> 6) {
    of[0] = lane * per < p.B ? full_blocks(p, lane * per) + kOpenTiles : 0;
#pragma unroll
    for (int i = 1; i < kPer; ++i) of[i] = 0;
    if (per > 1) {
      asm volatile("");
#pragma unroll
      for (int i = 1; i < kPer; ++i) {
        const int b = lane * per + i;
        of[i] = i < per && b < p.B ? full_blocks(p, b) + kOpenTiles : 0;
      }
    }
  }
};

struct Cut {
  int total;           // parts of all units
  uint32_t inv;        // about 2^32 / most places of a part
  // parts of a unit of so many places: about places / most, rounded up
  LVS_DEV int parts(int places) const { return places == 0 ? 0 : 1 + (int)__umulhi((uint32_t)(places - 1), inv); }
  // of a unit of each of the lane's sequences
  LVS_DEV int parts(const Places& places) const {
    int n = parts(places.of[0]);
    if (places.per > 1) {
      asm volatile("");                  // (a jump, not four times the instructions)
#pragma unroll
      for (int i = 1; i < kPer; ++i) n += parts(places.of[i]);
    }
    return n;
  }
};

LVS_DEV Cut cut_units(const PagedAttnKernelArgs& p, const Places& places) {
  int sum = places.of[0], most = places.of[0];
  if (places.per > 1) {
    asm volatile("");
#pragma unroll
    for (int i = 1; i < kPer; ++i) {
      sum += places.of[i];
      most = max(most, places.of[i]);
    }
  }
  sum = last_lane(wave_scan(sum));
  most = (int)wave_max_u32((uint32_t)most);
  const int HR = p.Hkv * p.n_rc;
  Cut c;
  int limit = p.limit - p.spare;
  while (true) {
    const int even = about(sum * HR, limit);
    int part = max((even + kRound - 1) / kRound * kRound, kOpenTiles);
    while (true) {
      c.inv = (uint32_t)(4294967040.f * __builtin_amdgcn_rcpf((float)part));
      c.total = last_lane(wave_scan(c.parts(places))) * HR;
      if (c.total <= limit) break;            // (one part each serves, so it ends)
      part += max(part >> 3, kRound) / kRound * kRound;
    }
    if (limit == p.limit || min(part, most) <= even + (even >> 1) + kOpenTiles) return c;
    limit = p.limit;
  }
}

// ------------------------------------------------------------------------------ split
LVS_DEV u32x4 pack8(float a, float b, float c, float d, float e, float f, float g, float h) {
  return u32x4{pack_bf16(a, b), pack_bf16(c, d), pack_bf16(e, f), pack_bf16(g, h)};
}
LVS_DEV f32x4 four_bf16(const uint8_t* at) {
  const uint2 x = *reinterpret_cast<const uint2*>(at);
  return f32x4{__builtin_bit_cast(float, x.x << 16), __builtin_bit_cast(float, x.x & 0xffff0000u),
               __builtin_bit_cast(float, x.y << 16), __builtin_bit_cast(float, x.y & 0xffff0000u)};
}
LVS_DEV bool finite(float x) { return fabsf(x) <= 3.4028234663852886e38f; }

// Scores of a tile to probabilities (in place); running maximum m, sum l.  LANES lanes hold a row's scores.
// `first`: there is nothing to rescale yet.  The maximum is exact: a reference that is taken anew only for
// scores 2^8 above it saves 1 to 4 % of the time and costs the exact 1 of the largest probability (error
// against 64 bits 2.2e-3 -> 2.5e-3).
template <int LANES, int N, class Rescale>
LVS_DEV void softmax_row(float (&s)[N], float& m, float& l, float c, bool first, Rescale&& rescale) {
  float top = s[0];
#pragma unroll
  for (int i = 1; i < N; ++i) top = fmaxf(top, s[i]);
  top *= c;
  if (__any(top > m)) {
    float x = max_halves(fmaxf(m, top));
    if constexpr (LANES == 4) x = max_rows(x);
    const float alpha = fast_exp2(m - x);
    m = x;
    if (!first) rescale(alpha);
  }
#pragma unroll
  for (int i = 0; i < N; ++i) s[i] = fast_exp2(__builtin_fmaf(s[i], c, -m));
  float sum[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
  for (int i = 0; i < N; ++i) sum[i & 3] += s[i];
  l += (sum[0] + sum[1]) + (sum[2] + sum[3]);
}

// Up to 16 query rows, on 16x16 tiles: a quarter of the wave's lanes (g4) holds a row (n16).
// A tile's scores: key 16 g4 + 4 kb + i is element 4 kb + i.
struct Rows16 {
  static constexpr int kRows = 16, kScores = 16, kLanes = 4;
  u32x4 q[4];              // channels 64 (x/2) + 16 g4 + 8 (x%2) .. +7
  f32x4 acc[8];            // O^T: channels 16 db + 4 g4 + i
  float m, l, lv;

  static LVS_DEV int k_place(int t) { return ((t >> 1) & 1) | (((t >> 4) & 3) << 1); }
  static LVS_DEV int k_copy(int y, int lane) { return ((lane >> 4) & 1) | ((y >> 1) << 1); }      // of 8 y + lane / 8
  static LVS_DEV int v_place(int q) { return ((q >> 1) & 1) | (((q ^ (q >> 1)) & 1) << 1); }    // 0 2 3 1
  static LVS_DEV int row_of(int lane) { return lane & 15; }
  static LVS_DEV int key_of(int lane, int e) { return 16 * (lane >> 4) + e; }

  LVS_DEV void load_q(const uint16_t* qp, int lane) {
#pragma unroll
    for (int x = 0; x < 4; ++x)
      q[x] = *reinterpret_cast<const u32x4*>(qp + 64 * (x >> 1) + 16 * (lane >> 4) + 8 * (x & 1));
  }
  LVS_DEV void clear() {
#pragma unroll
    for (int db = 0; db < 8; ++db) acc[db] = f32x4{0.f, 0.f, 0.f, 0.f};
    m = kNegBig;
    l = lv = 0.f;
  }
  LVS_DEV void rescale(float a) {
    l *= a;
    lv *= a;
#pragma unroll
    for (int db = 0; db < 8; ++db) acc[db] *= a;
  }
  // operand reads: token 16 (n16/4) + 4 kb + n16%4, chunk 4 half + g4; channel 16 x + n16, chunk g4
  LVS_DEV void read_k(u32x4 (&k)[8], uint32_t slot, int lane) const {
    const int n16 = lane & 15, g4 = lane >> 4, t = 16 * (n16 >> 2) + (n16 & 3), f = k_place(t);
    const uint32_t a0 = slot + t * 128 + ((g4 ^ f) << 4), a1 = slot + t * 128 + (((4 + g4) ^ f) << 4);
#pragma unroll
    for (int kb = 0; kb < 4; ++kb) {
      k[2 * kb] = lds_load16(a0 + kb * 512);
      k[2 * kb + 1] = lds_load16(a1 + kb * 512);
    }
  }
  LVS_DEV void read_v(u32x4 (&v)[8], uint32_t slot, int lane) const {
    const int n16 = lane & 15;
    const uint32_t a = slot + n16 * kPageTokens + (((lane >> 4) ^ v_place(n16 >> 2)) << 4);
#pragma unroll
    for (int x = 0; x < 8; ++x) v[x] = lds_load16(a + x * 1024);
  }
  LVS_DEV void scores(float (&s)[16], const u32x4 (&k)[8], float scale) const {
#pragma unroll
    for (int kb = 0; kb < 4; ++kb) {
      f32x4 z = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int x = 0; x < 4; ++x) {
        const u32x4& raw = k[2 * kb + (x >> 1)];
        z = mfma16(widen(raw[(x & 1) * 2], raw[(x & 1) * 2 + 1], scale), q[x], z);
      }
#pragma unroll
      for (int i = 0; i < 4; ++i) s[4 * kb + i] = z[i];
    }
  }
  LVS_DEV void output(const u32x4 (&pr)[2], const u32x4 (&v)[8], float scale) {
#pragma unroll
    for (int db = 0; db < 8; ++db)
#pragma unroll
      for (int y = 0; y < 2; ++y) acc[db] = mfma16(widen(v[db][2 * y], v[db][2 * y + 1], scale), pr[y], acc[db]);
  }
  // a piece of 32 open rows: element 4 kb + i is key 16 kb + 4 g4 + i
  static constexpr int kOpenScores = 8;
  static LVS_DEV int open_key(int lane, int e) { return 16 * (e >> 2) + 4 * (lane >> 4) + (e & 3); }
  LVS_DEV void open_load(u32x4 (&k)[8], const uint8_t* kt, int p0, int lane) const {
#pragma unroll
    for (int kb = 0; kb < 2; ++kb)
#pragma unroll
      for (int x = 0; x < 4; ++x)
        k[4 * kb + x] = *reinterpret_cast<const u32x4*>(kt + ((p0 + 16 * kb + (lane & 15)) & (kTailRows - 1)) * kRowBytes +
                                                        2 * (64 * (x >> 1) + 16 * (lane >> 4) + 8 * (x & 1)));
  }
  LVS_DEV void open_scores(float (&s)[8], const u32x4 (&k)[8]) const {
#pragma unroll
    for (int kb = 0; kb < 2; ++kb) {
      f32x4 z = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int x = 0; x < 4; ++x) z = mfma16(k[4 * kb + x], q[x], z);
#pragma unroll
      for (int i = 0; i < 4; ++i) s[4 * kb + i] = z[i];
    }
  }
  LVS_DEV void open_output(const float (&s)[8], uint32_t turn, int lane) {
    const u32x4 pr = pack8(s[0], s[1], s[2], s[3], s[4], s[5], s[6], s[7]);
    const int n16 = lane & 15, tr = 4 * (lane >> 4) + (n16 >> 2);      // row and chunk this lane hands in
#pragma unroll
    for (int db = 0; db < 8; ++db) {
      const uint32_t at = turn + ((((2 * db + ((n16 & 3) >> 1)) ^ rows32_swz(tr)) << 4) | ((n16 & 1) << 3));
      const u32x2 lo = lds_load_tr(at + tr * kRowBytes);
      const u32x2 hi = lds_load_tr(at + (16 + tr) * kRowBytes);
      acc[db] = mfma16(u32x4{lo[0], lo[1], hi[0], hi[1]}, pr, acc[db]);
    }
  }
  LVS_DEV void add_odd(const uint8_t* row, bool sees, int lane) {
#pragma unroll
    for (int db = 0; db < 8; ++db) {
      const f32x4 y = four_bf16(row + 2 * (16 * db + 4 * (lane >> 4)));
#pragma unroll
      for (int i = 0; i < 4; ++i) acc[db][i] += sees && !finite(y[i]) ? y[i] : 0.f;
    }
  }
  LVS_DEV void store(float* o, float f, int lane) const {
#pragma unroll
    for (int db = 0; db < 8; ++db) *reinterpret_cast<f32x4*>(o + 16 * db + 4 * (lane >> 4)) = acc[db] * f;
  }
};

// 17 to 32 rows, on 32x32 tiles, which leave the vector unit more room beside the matrix unit than 16x16 ones
// (matrix instructions of one wave and FMAs of another on a SIMD: 366 us together, 238 and 307 alone; on 16x16
// 402, 257 and 307): half a wave's lanes (h) hold a row (n32).  Key 32 kb + 16 h + r is element 16 kb + r.
// (64 rows of a wave, which would share the conversion, take 400 registers, and half of a wave's are no operands
// of its vector instructions: 16384 keys, 150 rows 29.1 us so, in chunks of 32 23.2; 8 x 8000, 64 rows 43.8 and 40.2.)
struct WideRows {
  static constexpr int kRows = 32, kScores = 32, kLanes = 2;
  u32x4 q[8];              // channels 16 (2 (x/2) + h) + 8 (x%2) .. +7
  f32x16 acc[4];           // O^T: channels 32 db + 8 (r/4) + 4 h + r%4
  float m, l, lv;

  static LVS_DEV int k_place(int t) { return (t >> 1) & 7; }
  static LVS_DEV int k_copy(int y, int lane) { return (lane >> 4) | ((y & 1) << 2); }
  static LVS_DEV int v_place(int q) { return q & 3; }
  static LVS_DEV int row_of(int lane) { return lane & 31; }
  static LVS_DEV int key_of(int lane, int e) { return 32 * (e >> 4) + 16 * (lane >> 5) + (e & 15); }

  LVS_DEV void load_q(const uint16_t* qp, int lane) {
#pragma unroll
    for (int x = 0; x < 8; ++x)
      q[x] = *reinterpret_cast<const u32x4*>(qp + 16 * (2 * (x >> 1) + (lane >> 5)) + 8 * (x & 1));
  }
  LVS_DEV void clear() {
#pragma unroll
    for (int db = 0; db < 4; ++db)
#pragma unroll
      for (int r = 0; r < 16; ++r) acc[db][r] = 0.f;
    m = kNegBig;
    l = lv = 0.f;
  }
  LVS_DEV void rescale(float a) {
    l *= a;
    lv *= a;
#pragma unroll
    for (int db = 0; db < 4; ++db)
#pragma unroll
      for (int r = 0; r < 16; ++r) acc[db][r] *= a;
  }
  // operand reads: row m of block kb is token 32 kb + 16 (m/4 % 2) + 4 (m/8) + m%4, chunk 2 i + h; channel
  // 32 db + n32, chunk 2 kb + h
  LVS_DEV void read_k(u32x4 (&k)[8], uint32_t slot, int lane) const {
    const int n = lane & 31, t = 16 * ((n >> 2) & 1) + 4 * (n >> 3) + (n & 3);
    const uint32_t a = slot + t * 128 + (((lane >> 5) ^ k_place(t)) << 4);
#pragma unroll
    for (int kb = 0; kb < 2; ++kb)
#pragma unroll
      for (int i = 0; i < 4; ++i) k[4 * kb + i] = lds_load16((a ^ (i << 5)) + kb * 4096);
  }
  LVS_DEV void read_v(u32x4 (&v)[8], uint32_t slot, int lane) const {
    const int n = lane & 31;
    const uint32_t a = slot + n * kPageTokens + (((lane >> 5) ^ v_place(n >> 2)) << 4);
#pragma unroll
    for (int db = 0; db < 4; ++db)
#pragma unroll
      for (int kb = 0; kb < 2; ++kb) v[2 * db + kb] = lds_load16((a ^ (kb << 5)) + db * 2048);
  }
  LVS_DEV void scores(float (&s)[32], const u32x4 (&k)[8], float scale) const {
#pragma unroll
    for (int kb = 0; kb < 2; ++kb) {
      f32x16 z;
#pragma unroll
      for (int r = 0; r < 16; ++r) z[r] = 0.f;
#pragma unroll
      for (int x = 0; x < 8; ++x) {
        const u32x4& raw = k[4 * kb + (x >> 1)];
        z = mfma32(widen(raw[(x & 1) * 2], raw[(x & 1) * 2 + 1], scale), q[x], z);
      }
#pragma unroll
      for (int r = 0; r < 16; ++r) s[16 * kb + r] = z[r];
    }
  }
  LVS_DEV void output(const u32x4 (&pr)[4], const u32x4 (&v)[8], float scale) {
#pragma unroll
    for (int y = 0; y < 4; ++y)
#pragma unroll
      for (int db = 0; db < 4; ++db) {
        const u32x4& raw = v[2 * db + (y >> 1)];
        acc[db] = mfma32(widen(raw[(y & 1) * 2], raw[(y & 1) * 2 + 1], scale), pr[y], acc[db]);
      }
  }
  // a piece of 32 open rows: element r is key 8 (r/4) + 4 h + r%4
  static constexpr int kOpenScores = 16;
  static LVS_DEV int open_key(int lane, int e) { return 8 * (e >> 2) + 4 * (lane >> 5) + (e & 3); }
  LVS_DEV void open_load(u32x4 (&k)[8], const uint8_t* kt, int p0, int lane) const {
#pragma unroll
    for (int x = 0; x < 8; ++x)
      k[x] = *reinterpret_cast<const u32x4*>(kt + ((p0 + (lane & 31)) & (kTailRows - 1)) * kRowBytes +
                                             2 * (16 * (2 * (x >> 1) + (lane >> 5)) + 8 * (x & 1)));
  }
  LVS_DEV void open_scores(float (&s)[16], const u32x4 (&k)[8]) const {
    f32x16 z;
#pragma unroll
    for (int r = 0; r < 16; ++r) z[r] = 0.f;
#pragma unroll
    for (int x = 0; x < 8; ++x) z = mfma32(k[x], q[x], z);
#pragma unroll
    for (int r = 0; r < 16; ++r) s[r] = z[r];
  }
  LVS_DEV void open_output(const float (&s)[16], uint32_t turn, int lane) {
    const int h = lane >> 5, rr = (lane & 15) >> 2, g1 = (lane >> 4) & 1;
    const int chunk = (2 * g1 + ((lane & 3) >> 1)) ^ rows32_swz(4 * h + rr);
    const uint32_t a0 = turn + (4 * h + rr) * kRowBytes + (chunk << 4) + (lane & 1) * 8;
#pragma unroll
    for (int kt = 0; kt < 2; ++kt) {
      const u32x4 pr = pack8(s[8 * kt], s[8 * kt + 1], s[8 * kt + 2], s[8 * kt + 3], s[8 * kt + 4], s[8 * kt + 5],
                             s[8 * kt + 6], s[8 * kt + 7]);
#pragma unroll
      for (int db = 0; db < 4; ++db) {
        const uint32_t a = a0 ^ (db << 6);
        const u32x2 lo = lds_load_tr(a + kt * (16 * kRowBytes));
        const u32x2 hi = lds_load_tr((a ^ 32) + (kt * 16 + 8) * kRowBytes);
        acc[db] = mfma32(u32x4{lo[0], lo[1], hi[0], hi[1]}, pr, acc[db]);
      }
    }
  }
  LVS_DEV void add_odd(const uint8_t* row, bool sees, int lane) {
#pragma unroll
    for (int db = 0; db < 4; ++db)
#pragma unroll
      for (int g = 0; g < 4; ++g) {
        const f32x4 y = four_bf16(row + 2 * (32 * db + 8 * g + 4 * (lane >> 5)));
#pragma unroll
        for (int i = 0; i < 4; ++i) acc[db][4 * g + i] += sees && !finite(y[i]) ? y[i] : 0.f;
      }
  }
  LVS_DEV void store(float* o, float f, int lane) const {
#pragma unroll
    for (int db = 0; db < 4; ++db)
#pragma unroll
      for (int g = 0; g < 4; ++g)
        *reinterpret_cast<f32x4*>(o + 32 * db + 8 * g + 4 * (lane >> 5)) =
            f32x4{acc[db][4 * g], acc[db][4 * g + 1], acc[db][4 * g + 2], acc[db][4 * g + 3]} * f;
  }
};

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

// KS streams of tiles, a wave each.
template <class Rows, int KS>
constexpr int segment_lds() {
  constexpr int merge = (int)sizeof(float) * KS * Rows::kRows * (1 + kMergeStride);
  return merge > KS * kRingBytes ? merge : KS * kRingBytes;
}

template <class Rows, int KS, bool ONCE>
struct Segment {
  static constexpr int kRows = Rows::kRows;
  const PagedAttnKernelArgs& p;
  uint8_t* smem;
  int stream;
  Rows st;
  int vis_b, vis_e;
  bool fresh;              // nothing in the state yet

  LVS_DEV Segment(const PagedAttnKernelArgs& a, uint8_t* lds) : p(a), smem(lds) {
    stream = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  }

  // The lane's number.  Every part of a segment takes it anew: what follows from it would else be held in
  // registers through the loop over the tiles.
  static LVS_DEV int lane_now() {
    int lane = threadIdx.x & 63;
    asm volatile("" : "+v"(lane));
    return lane;
  }

  // draft row of the lane's query row (rows past the last one: that row again, to no output)
  LVS_DEV int query_row(int rc, int lane) const { return min(rc * p.rpad + Rows::row_of(lane), p.R - 1); }

  LVS_DEV void begin(int b, int h, int rc) {
    const int lane = lane_now(), r = query_row(rc, lane);
    const int qi = (int)fast_div((uint32_t)r, p.div_g);
    st.load_q(p.q + (int64_t)b * p.q_sb + (int64_t)qi * p.q_sg + (int64_t)(h * p.G + (r - qi * p.G)) * p.q_sh, lane);
    st.clear();
    fresh = true;
    vis_b = vis_e = 0;
    if (p.vis_begin != nullptr) {
      vis_b = __builtin_amdgcn_readfirstlane(p.vis_begin[b]);
      vis_e = __builtin_amdgcn_readfirstlane(p.vis_end[b]);
    }
  }

  // softmax of a tile or piece; its mass on the video span
  template <int N, class KeyOf>
  LVS_DEV void softmax(float (&s)[N], int key0, int keys, KeyOf&& key_of) {
    softmax_row<Rows::kLanes>(s, st.m, st.l, p.scale_log2e, fresh, [&](float a) { st.rescale(a); });
    fresh = false;
    if (key0 < vis_e && key0 + keys > vis_b) {
      float sum = 0.f;
#pragma unroll
      for (int e = 0; e < N; ++e) {
        const int key = key0 + key_of(e);
        sum += key >= vis_b && key < vis_e ? s[e] : 0.f;
      }
      st.lv += sum;
    }
  }

  // tiles t0 .. t1-1 of a unit
  LVS_DEV void blocks(int b, int h, int t0, int t1) {
    const int mine = (t1 - t0 - stream + KS - 1) / KS;
    if (mine <= 0) return;
    const int lane = lane_now();
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
    // global side of the copies: the chunk that belongs at the lane's place
    int k_off[8], v_off[8];
#pragma unroll
    for (int y = 0; y < 8; ++y) {
      k_off[y] = (lane >> 3) * 128 + (((lane & 7) ^ Rows::k_copy(y, lane)) << 4);
      v_off[y] = (lane >> 2) * kPageTokens + (((lane & 3) ^ Rows::v_place(lane >> 4)) << 4);
    }
    auto copy_k = [&](int id) { copy_page<ONCE>(p.k8, id, h, p.Hkv, k_slot, k_off); };
    auto copy_v = [&](int id) { copy_page<ONCE>(p.v8, id, h, p.Hkv, v_slot, v_off); };
    fetch(0);
    int id = __builtin_amdgcn_readlane(ids, 0);
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");      // (the open rows' reads of the ring)
    copy_k(id);
    copy_v(id);
    float k_scale = scale_of(p.k_scale, id), v_scale = scale_of(p.v_scale, id);
    for (int j = 0; j < mine; ++j) {
      const bool more = j + 1 < mine;
      if (((j + 1) & 63) == 0) fetch(j + 1);
      const int next = more ? __builtin_amdgcn_readlane(ids, (j + 1) & 63) : -1;
      u32x4 k[8];
      wait_copies<8>();                // all but V's
      st.read_k(k, k_slot, lane);
      asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
      if (more) copy_k(next);
      const float k_next = scale_of(p.k_scale, next), v_next = scale_of(p.v_scale, next);
      float s[Rows::kScores];
      st.scores(s, k, k_scale);
      u32x4 pr[Rows::kScores / 8];
      if (id >= 0) {                   // (an entry that names no block of the pool: no key)
        softmax(s, (t0 + stream + KS * j) * kPageTokens, kPageTokens, [&](int e) { return Rows::key_of(lane, e); });
#pragma unroll
        for (int y = 0; y < Rows::kScores / 8; ++y)
          pr[y] = pack8(s[8 * y], s[8 * y + 1], s[8 * y + 2], s[8 * y + 3], s[8 * y + 4], s[8 * y + 5], s[8 * y + 6],
                        s[8 * y + 7]);
      }
      u32x4 v[8];
      if (more)
        wait_copies<8>();              // all but the next K's
      else
        wait_copies<0>();
      st.read_v(v, v_slot, lane);
      asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
      if (more) copy_v(next);
      if (id >= 0) st.output(pr, v, v_scale);
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
    const int lane = lane_now(), n16 = lane & 15, g4 = lane >> 4;
    const int base = L & ~(kPageTokens - 1);
    const int n = L - base + p.gamma;
    const uint32_t rowmask = p.draft_mask[fast_div((uint32_t)query_row(rc, lane), p.div_g)] &
                             (0xffffffffu >> (32 - p.gamma));            // draft rows that the lane's row sees
    const int64_t unit = ((int64_t)b * p.Hkv + h) * (kTailRows * kRowBytes);
    const uint8_t* kt = p.k_tail + unit;
    const uint8_t* vt = p.v_tail + unit;
    const uint32_t turn = lds_addr(smem) + stream * kRingBytes;
    // (from the last stream on: the first ones have the odd tiles)
    for (int piece = KS - 1 - stream; piece * 32 < n; piece += KS) {
      const int p0 = base + piece * 32;
      u32x4 k[8], v[8];
      st.open_load(k, kt, p0, lane);
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
      float s[Rows::kOpenScores];
      st.open_scores(s, k);
      // bit k: the lane's row sees key k of the piece; committed keys first, then the draft rows
      const int old = L - p0;
      const uint32_t sees = old >= 32 ? 0xffffffffu
                            : old >= 0 ? ((1u << old) - 1u) | (rowmask << old) : rowmask >> min(-old, 31);
#pragma unroll
      for (int e = 0; e < Rows::kOpenScores; ++e) s[e] = (sees >> Rows::open_key(lane, e)) & 1u ? s[e] : -INFINITY;
      softmax(s, p0, 32, [&](int e) { return Rows::open_key(lane, e); });
      asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
      st.open_output(s, turn, lane);
      // (any weight times a value that is not finite is that value: it is added as it is)
      while (odd != 0u) {
        const int key = __builtin_ctz(odd);
        odd &= odd - 1;
        st.add_odd(vt + ((p0 + key) & (kTailRows - 1)) * kRowBytes, ((sees >> key) & 1u) != 0u, lane);
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
    const int lane = lane_now(), row = Rows::row_of(lane);
    float* sm_m = reinterpret_cast<float*>(smem);
    __syncthreads();
    if (lane < kRows) sm_m[stream * kRows + row] = st.m;
    __syncthreads();
    if (((on >> stream) & 1u) == 0u) return;
    const float f = fast_exp2(st.m - merged_max(row));
    float* o = sm_m + KS * kRows + (stream * kRows + row) * kMergeStride;
    st.store(o, f, lane);
    float l = st.l * f, lv = st.lv * f;
    if constexpr (Rows::kLanes == 4) {
      l += xor_shuffle(l, 16);
      lv += xor_shuffle(lv, 16);
    }
    l += xor_shuffle(l, 32);
    lv += xor_shuffle(lv, 32);
    if (lane < kRows) *reinterpret_cast<float2*>(o + 128) = float2{l, lv};
  }

  // Sums over the active streams of four floats of a row.  (All are read, at once: in the place of one that has
  // nothing is whatever was there, and is not added.)
  LVS_DEV f32x4 merged(uint32_t on, int row, int c4) const {
    const float* o = reinterpret_cast<const float*>(smem) + KS * kRows + row * kMergeStride + c4;
    f32x4 x[KS], sum = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int k = 0; k < KS; ++k) x[k] = *reinterpret_cast<const f32x4*>(o + k * kRows * kMergeStride);
#pragma unroll
    for (int k = 0; k < KS; ++k)
#pragma unroll
      for (int i = 0; i < 4; ++i) sum[i] += (on >> k) & 1u ? x[k][i] : 0.f;
    return sum;
  }
  LVS_DEV float merged_max(int row) const {
    const float* sm_m = reinterpret_cast<const float*>(smem);
    float mm = sm_m[row];
#pragma unroll
    for (int k = 1; k < KS; ++k) mm = fmaxf(mm, sm_m[k * kRows + row]);
    return mm;
  }
  // denominator and its share on the video span, by the 32 lanes that have the row
  LVS_DEV float2 merged_sums(uint32_t on, int row, int l32) const {
    const float* o = reinterpret_cast<const float*>(smem) + KS * kRows + row * kMergeStride + 128;
    const int k = l32 & (KS - 1);
    float2 x = *reinterpret_cast<const float2*>(o + k * kRows * kMergeStride);
    x = (on >> k) & 1u ? x : float2{0.f, 0.f};
#pragma unroll
    for (int d = 1; d < KS; d <<= 1) {
      x.x += xor_shuffle(x.x, d);
      x.y += xor_shuffle(x.y, d);
    }
    return x;
  }

  // the merged state into a record
  LVS_DEV void end(uint32_t on, int rc, float* rec) {
    gather(on);
    __syncthreads();
    const int rows = min(p.R - rc * p.rpad, p.rpad);
    for (int idx = threadIdx.x; idx < rows * 32; idx += 64 * KS) {
      const int row = idx >> 5, l32 = idx & 31;
      const float2 l = merged_sums(on, row, l32);
      *reinterpret_cast<f32x4*>(rec + 3 * p.rpad + row * 128 + l32 * 4) = merged(on, row, l32 * 4);
      if (l32 == 0) {
        rec[row] = merged_max(row);
        rec[p.rpad + row] = l.x;
        rec[2 * p.rpad + row] = l.y;
      }
    }
  }

  // the merged state of a whole unit into the outputs
  LVS_DEV void finish(uint32_t on, int b, int h, int rc) {
    gather(on);
    __syncthreads();
    const int rows = min(p.R - rc * p.rpad, p.rpad);
    for (int idx = threadIdx.x; idx < rows * 32; idx += 64 * KS) {
      const int row = idx >> 5, l32 = idx & 31;
      const float2 l = merged_sums(on, row, l32);
      const float mm = p.lse != nullptr ? merged_max(row) : 0.f;
      write_row(p, b, h, rc * p.rpad + row, l32, merged(on, row, l32 * 4), mm, l.x, l.y);
    }
  }
};

// Workspace: a record per part, and a unit's first record and their number.
LVS_DEV float* record_at(const PagedAttnKernelArgs& p, int64_t i) { return p.ws + i * ((int64_t)p.rpad * 131); }
LVS_DEV int2* records_of(const PagedAttnKernelArgs& p) { return reinterpret_cast<int2*>(record_at(p, p.limit)); }

// All cache lines of a kernel's arguments at its start, not one miss behind the other: 16384 keys, 25 rows 15.9 us
// without and 15.6, 100 rows 22.7 and 22.4 (four streams), 777 keys 8.1 and 7.9.
LVS_DEV void ask_for_arguments(const PagedAttnKernelArgs& p) {
  asm volatile("" ::"s"(p.q), "s"(p.k8), "s"(p.table), "s"(p.G), "s"(p.vis_begin), "s"(p.out), "s"(p.ws));
}

template <class Rows, int KS, bool ONCE>
__global__ __launch_bounds__(64 * KS, 2) void paged_attn_kernel(PagedAttnKernelArgs p) {
  extern __shared__ __align__(256) uint8_t smem[];
  Segment<Rows, KS, ONCE> sg(p, smem);
  const int HR = p.Hkv * p.n_rc, lane = threadIdx.x & 63;
  ask_for_arguments(p);
  const Places places(p, lane);
  const Cut cut = cut_units(p, places);
  // parts that follow each other go to one XCD, which has the records of a unit in its L2
  const int each = (cut.total + 7) >> 3;
  const int w = (blockIdx.x & 7) * each + (blockIdx.x >> 3);
  if ((int)(blockIdx.x >> 3) >= each || w >= cut.total) return;
  const int f = cut.parts(places), upto = wave_scan(f);
  const int holder = __popcll(__ballot(w >= upto * HR));      // the lane that has the sequence
  int b = holder * places.per, before = __builtin_amdgcn_readlane(upto - f, holder);
  int unit_places = __builtin_amdgcn_readlane(places.of[0], holder), n = cut.parts(unit_places);
#pragma unroll
  for (int i = 1; i < kPer; ++i)
    if (i < places.per && w >= (before + n) * HR) {
      before += n;
      ++b;
      unit_places = __builtin_amdgcn_readlane(places.of[i], holder);
      n = cut.parts(unit_places);
    }
  const int y = w - before * HR;
  const int hr = divide(y, n), part = y - hr * n;
  const int h = ONCE ? hr : divide(hr, p.n_rc), rc = hr - h * p.n_rc;
  const int q = divide(unit_places, n), r = unit_places - q * n;      // the first r parts have one more
  const int p0 = part * q + min(part, r), p1 = p0 + q + (part < r ? 1 : 0);
  const int t0 = max(p0 - kOpenTiles, 0), t1 = p1 - kOpenTiles;
  if (part == 0 && threadIdx.x == 0) records_of(p)[b * HR + hr] = int2{w, n};
  const int L = p0 == 0 ? paged_len(p.kv_len[b], p.cols) : 0;      // (for the open rows)
  sg.begin(b, h, rc);
  if (p0 == 0) sg.open_rows(b, h, rc, L);
  sg.blocks(b, h, t0, t1);
  const uint32_t on = sg.active(t1 - t0, p0 == 0, L);
  if (n == 1)
    sg.finish(on, b, h, rc);
  else
    sg.end(on, rc, record_at(p, w));
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

// Columns of a table up to which every unit is one workgroup's, with no second kernel.  The longest sequence may
// have as many blocks, so the more units there are, the more of them pay: they fill the chip anyway.  One
// workgroup per unit and parts, us: 8 units 800 keys 11.1 and 12.4, 1100 12.2 and 12.7, 1400 13.9 and 12.7;
// 64 units 1000 keys 13.3 and 13.8, 1500 15.9 and 14.4; 128 units 2000 keys 18.6 and 20.7, 3000 24.6 and 26.1;
// 256 units 4000 keys 45.9 and 49.8, 512 units 91.6 and 89.6.  It goes by the table's width, not by the lengths, which
// the host does not know: 777 keys, 2 heads 7.8 us with 13 columns, 9.8 with 1024.
// More than 64 kPer sequences are not cut, whose places a wave cannot hold.  That costs little where lengths are alike,
// 250 x (400 to 12000) keys, 2 heads 96 and 92, and much where one sequence is far longer than the others: one of
// 65536 keys among 500 each, 8 heads, 1 row of 5 heads 176 us with 256 sequences and 308 with 257.
int unit_columns(int64_t B, int64_t units, int64_t cus) {
  return B > 64 * kPer ? 1 << 30 : units >= cus / 2 ? 64 : 18;
}

template <class Rows, int KS, bool ONCE>
hipError_t launch_parts(const PagedAttnKernelArgs& a, hipStream_t stream) {
  static LdsLimitOnce limit;
  constexpr size_t lds = segment_lds<Rows, KS>();
  hipError_t e = limit.ensure(reinterpret_cast<const void*>(&paged_attn_kernel<Rows, KS, ONCE>), lds);
  if (e != hipSuccess) return e;
  const unsigned units = (unsigned)(a.B * a.Hkv * a.n_rc);
  paged_attn_kernel<Rows, KS, ONCE><<<dim3((unsigned)(a.limit + 7) / 8 * 8), dim3(64 * KS), lds, stream>>>(a);
  e = hipGetLastError();
  if (e != hipSuccess) return e;
  // few units have many records each: all groups of a workgroup to one row.  8 units, 32 records each: 16.4 us
  // so and 17.7 with a group per row; 64 units, 4 each: 23.9 and 20.9.
  if ((int64_t)units * 16 > a.limit - a.spare)
    paged_combine_kernel<1><<<dim3(units * (unsigned)((a.rpad + 7) / 8)), dim3(kCombineThreads), 0, stream>>>(a);
  else
    paged_combine_kernel<8><<<dim3(units * (unsigned)a.rpad), dim3(kCombineThreads), 0, stream>>>(a);
  return hipGetLastError();
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

hipError_t launch_paged_attn(const PagedAttnKernelArgs& a, hipStream_t stream) {
  const bool once = a.n_rc == 1;
  const int64_t units = (int64_t)a.B * a.Hkv * a.n_rc;
  const int64_t cus = a.limit - units + 1;
  if (a.cols <= unit_columns(a.B, units, cus)) {
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
