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

constexpr int kMergeStride = 132;      // floats per row in the merge buffer (pad)
constexpr float kNegBig = -1.0e30f;

// eight e4m3 times 2^e as bf16 (exact)
LVS_DEV u32x4 widen(uint32_t lo, uint32_t hi, float scale) {
  auto two = [&](uint32_t x, auto upper) {
    return __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8((int)x, scale, decltype(upper)::value));
  };
  return u32x4{two(lo, std::false_type{}), two(lo, std::true_type{}), two(hi, std::false_type{}), two(hi, std::true_type{})};
}

// ------------------------------------------------------------------------------ the line of tiles
// Sequence b's tiles start at HR * (complete blocks of the sequences before it), HR = Hkv * n_rc units
// each of full(b) tiles.  Every wave finds its place by itself: sequences in groups of 64, one per lane.
struct Line {
  int total;           // tiles of the line
  int per;             // tiles of a stretch
};

LVS_DEV int wave_scan(int x, int lane) {
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    const int y = __shfl_up(x, d, 64);
    x += lane >= d ? y : 0;
  }
  return x;
}

LVS_DEV int full_blocks(const PagedAttnKernelArgs& p, int b) {
  return b < p.B ? paged_len(p.kv_len[b], p.cols) >> kPageShift : 0;
}

template <int KS>
LVS_DEV Line line_of(const PagedAttnKernelArgs& p, int lane) {
  int sum = 0;
  for (int b0 = 0; b0 < p.B; b0 += 64) sum += full_blocks(p, b0 + lane);
#pragma unroll
  for (int d = 32; d > 0; d >>= 1) sum += __shfl_xor(sum, d, 64);
  Line l;
  l.total = __builtin_amdgcn_readfirstlane(sum) * p.Hkv * p.n_rc;
  // whole rounds of the streams: a stretch of 4 k + 1 tiles takes as long as one of 4 (k + 1)
  const int rounds = (l.total + p.n_wg * KS - 1) / (p.n_wg * KS);
  l.per = (rounds > 0 ? rounds : 1) * KS;
  return l;
}

// ------------------------------------------------------------------------------ split
template <int NB, int RG, int KS>
struct Shape {
  static constexpr int kWaves = RG * KS;
  static constexpr int kRows = 16 * NB * RG;
  static constexpr int kMergeBytes = (int)sizeof(float) * KS * kRows * (3 + kMergeStride);
  static constexpr int kTurnBytes = kWaves * 32 * kRowBytes;      // values of 32 open rows per wave
  static constexpr int kLds = kMergeBytes > kTurnBytes ? kMergeBytes : kTurnBytes;
};

template <int NB>
struct RowState {
  f32x4 acc[NB][8];        // O^T: channels 16 db + 4 g4 + i of row n16
  float m[NB], l[NB], lv[NB];
};

// scores of NK blocks of 16 keys to probabilities (in place); the running maximum and the sums follow
template <int NB, int NK>
LVS_DEV void softmax_tile(RowState<NB>& st, f32x4 (&s)[NB][NK], float c) {
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
      st.l[nb] *= alpha;
      st.lv[nb] *= alpha;
#pragma unroll
      for (int db = 0; db < 8; ++db) st.acc[nb][db] *= alpha;
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

template <int NB, int RG, int KS>
struct Segment {
  using W = Shape<NB, RG, KS>;
  const PagedAttnKernelArgs& p;
  uint8_t* smem;
  int lane, wave, stream, rg, n16, g4;
  u32x4 q[NB][4];          // channels 64 (c/2) + 16 g4 + 8 (c%2) .. +7 of row n16
  int draft_row[NB];       // -1: no row
  RowState<NB> st;
  int vis_b, vis_e;

  LVS_DEV Segment(const PagedAttnKernelArgs& a, uint8_t* lds) : p(a), smem(lds) {
    lane = threadIdx.x & 63;
    wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    stream = wave % KS;
    rg = wave / KS;
    n16 = lane & 15;
    g4 = lane >> 4;
  }

  LVS_DEV void begin(int b, int h, int rc) {
#pragma unroll
    for (int nb = 0; nb < NB; ++nb) {
      const int in = (rg * NB + nb) * 16 + n16, r = rc * p.rpad + in;
      const bool valid = in < p.rpad && r < p.R;
      const int rcl = r < p.R ? r : p.R - 1;
      const int qi = rcl / p.G;
      draft_row[nb] = valid ? qi : -1;
      const uint16_t* qp = p.q + (int64_t)b * p.q_sb + (int64_t)qi * p.q_sg +
                           (int64_t)(h * p.G + (rcl - qi * p.G)) * p.q_sh;
#pragma unroll
      for (int c = 0; c < 4; ++c) {
        const u32x4 x = *reinterpret_cast<const u32x4*>(qp + 64 * (c >> 1) + 16 * g4 + 8 * (c & 1));
        q[nb][c] = valid ? x : u32x4{0u, 0u, 0u, 0u};
      }
#pragma unroll
      for (int db = 0; db < 8; ++db) st.acc[nb][db] = f32x4{0.f, 0.f, 0.f, 0.f};
      st.m[nb] = kNegBig;
      st.l[nb] = st.lv[nb] = 0.f;
    }
    vis_b = p.vis_begin != nullptr ? p.vis_begin[b] : 0;
    vis_e = p.vis_begin != nullptr ? p.vis_end[b] : 0;
  }

  // tiles t0 .. t1-1 of a unit
  LVS_DEV void blocks(int b, int h, int t0, int t1) {
    const int mine = (t1 - t0 - stream + KS - 1) / KS;
    if (mine <= 0) return;
    const int32_t* row = p.table + (int64_t)b * p.cols;
    const int lane_at = (16 * (n16 >> 2) + (n16 & 3)) * 128 + 16 * g4;      // K: token, channel
    const int turn_at = n16 * kPageTokens + 16 * g4;                          // V: channel, token
    u32x4 k[8], v[8];
    int ids = 0;
    float ks = 0.f, vs = 0.f;
    auto fetch = [&](int j0) {          // blocks and scales of the next 64 tiles, one per lane
      const int t = t0 + stream + KS * (j0 + lane);
      ids = t < t1 ? row[t] : -1;
      const bool there = (uint32_t)ids < (uint32_t)p.n_blocks;
      const int64_t at = (int64_t)(there ? ids : 0) * p.Hkv + h;
      ks = p.k_scale[at];
      vs = p.v_scale[at];
      ids = there ? ids : -1;
    };
    auto load_k = [&](int id) {
      const uint8_t* kp = p.k8 + ((int64_t)(id < 0 ? 0 : id) * p.Hkv + h) * kPageBytes + lane_at;
#pragma unroll
      for (int x = 0; x < 8; ++x)       // block x / 2 of 16 keys, channels 64 (x%2) ..
        k[x] = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(kp + (x >> 1) * 512 + (x & 1) * 64));
    };
    auto load_v = [&](int id) {
      const uint8_t* vp = p.v8 + ((int64_t)(id < 0 ? 0 : id) * p.Hkv + h) * kPageBytes + turn_at;
#pragma unroll
      for (int db = 0; db < 8; ++db)
        v[db] = __builtin_nontemporal_load(reinterpret_cast<const u32x4*>(vp + db * 1024));
    };
    fetch(0);
    int id = __builtin_amdgcn_readlane(ids, 0);
    load_k(id);
    load_v(id);
    const float c = p.scale_log2e;
    for (int j = 0; j < mine; ++j) {
      const float k_scale = __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, ks), j & 63));
      const float v_scale = __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, vs), j & 63));
      const bool there = id >= 0;
      const bool more = j + 1 < mine;
      if (more && ((j + 1) & 63) == 0) fetch(j + 1);
      const int next = more ? __builtin_amdgcn_readlane(ids, (j + 1) & 63) : id;
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
      if (more) load_k(next);
      if (there) {                      // (an entry that names no block of the pool: no key)
        softmax_tile<NB, 4>(st, s, c);
        const int key0 = (t0 + stream + KS * j) * kPageTokens;
        span_mass<NB, 4>(st, s, key0, kPageTokens, vis_b, vis_e,
                         [&](int kb, int i) { return key0 + 16 * g4 + 4 * kb + i; });
        u32x4 pr[NB][2];
#pragma unroll
        for (int nb = 0; nb < NB; ++nb) {
          pr[nb][0] = pack8(s[nb][0], s[nb][1]);
          pr[nb][1] = pack8(s[nb][2], s[nb][3]);
        }
#pragma unroll
        for (int db = 0; db < 8; ++db)
#pragma unroll
          for (int y = 0; y < 2; ++y) {
            const u32x4 a = widen(v[db][2 * y], v[db][2 * y + 1], v_scale);
#pragma unroll
            for (int nb = 0; nb < NB; ++nb) st.acc[nb][db] = mfma16(a, pr[nb][y], st.acc[nb][db]);
          }
      }
      if (more) load_v(next);
      id = next;
    }
  }

  // open rows: positions L / 64 * 64 .. L + gamma - 1, in pieces of 32 keys, one stream each
  LVS_DEV void open_rows(int b, int h, int L) {
    const int base = L & ~(kPageTokens - 1);
    const int n = L - base + p.gamma;
    uint32_t rowmask[NB];
#pragma unroll
    for (int nb = 0; nb < NB; ++nb) {
      rowmask[nb] = 0u;
#pragma unroll
      for (int j = 0; j < 32; ++j) rowmask[nb] = draft_row[nb] == j ? p.draft_mask[j] : rowmask[nb];
      rowmask[nb] &= 0xffffffffu >> (32 - p.gamma);
    }
    const int64_t unit = ((int64_t)b * p.Hkv + h) * (kTailRows * kRowBytes);
    const uint8_t* kt = p.k_tail + unit;
    const uint8_t* vt = p.v_tail + unit;
    const uint32_t turn = lds_addr(smem) + wave * (32 * kRowBytes);
    const float c = p.scale_log2e;
    for (int piece = stream; piece * 32 < n; piece += KS) {
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
#pragma unroll
      for (int x = 0; x < 8; ++x) {
        const bool there = p0 + 4 * x + g4 < L + p.gamma;
        bool bad = false;
#pragma unroll
        for (int i = 0; i < 4; ++i) bad |= (v[x][i] & 0x7f80u) == 0x7f80u || (v[x][i] & 0x7f800000u) == 0x7f800000u;
        const unsigned long long at = __ballot(there && bad);
        if (at != 0ull) {
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            odd |= ((at >> (16 * i)) & 0xffffull) != 0ull ? 1u << (4 * x + i) : 0u;
            v[x][i] = (v[x][i] & 0x7f80u) == 0x7f80u ? v[x][i] & 0xffff0000u : v[x][i];
            v[x][i] = (v[x][i] & 0x7f800000u) == 0x7f800000u ? v[x][i] & 0xffffu : v[x][i];
          }
        }
        v[x] = there ? v[x] : u32x4{0u, 0u, 0u, 0u};
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
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const int j = p0 + 16 * kb + 4 * g4 + i - L;       // draft row of the key
            const int jc = j < 0 ? 0 : j > 31 ? 31 : j;
            const bool sees = j < 0 || (j < 32 && ((rowmask[nb] >> jc) & 1u) != 0u);
            z[i] = sees ? z[i] : -INFINITY;
          }
          s[nb][kb] = z;
        }
      softmax_tile<NB, 2>(st, s, c);
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

  // the streams' states into one record
  LVS_DEV void end(int rc, float* rec) {
    float* sm_m = reinterpret_cast<float*>(smem);          // [KS][kRows]
    float* sm_l = sm_m + KS * W::kRows;
    float* sm_v = sm_l + KS * W::kRows;
    float* sm_o = sm_v + KS * W::kRows;                    // [KS][kRows][kMergeStride]
    __syncthreads();
#pragma unroll
    for (int nb = 0; nb < NB; ++nb) {
      float l = st.l[nb], lv = st.lv[nb];
      l += xor_shuffle(l, 16);
      l += xor_shuffle(l, 32);
      lv += xor_shuffle(lv, 16);
      lv += xor_shuffle(lv, 32);
      const int r = stream * W::kRows + (rg * NB + nb) * 16 + n16;
      if (g4 == 0) {
        sm_m[r] = st.m[nb];
        sm_l[r] = l;
        sm_v[r] = lv;
      }
#pragma unroll
      for (int db = 0; db < 8; ++db)
        *reinterpret_cast<f32x4*>(sm_o + (size_t)r * kMergeStride + 16 * db + 4 * g4) = st.acc[nb][db];
    }
    __syncthreads();
    int rows = p.R - rc * p.rpad;
    rows = rows < p.rpad ? rows : p.rpad;
    for (int row = threadIdx.x; row < rows; row += 64 * W::kWaves) {
      float mm = sm_m[row];
#pragma unroll
      for (int k = 1; k < KS; ++k) mm = fmaxf(mm, sm_m[k * W::kRows + row]);
      float l = 0.f, lv = 0.f;
#pragma unroll
      for (int k = 0; k < KS; ++k) {
        const float f = fast_exp2(sm_m[k * W::kRows + row] - mm);
        l += sm_l[k * W::kRows + row] * f;
        lv += sm_v[k * W::kRows + row] * f;
      }
      rec[row] = mm;
      rec[p.rpad + row] = l;
      rec[2 * p.rpad + row] = lv;
    }
    for (int idx = threadIdx.x; idx < rows * 32; idx += 64 * W::kWaves) {
      const int row = idx >> 5, c4 = (idx & 31) * 4;
      float mm = sm_m[row];
#pragma unroll
      for (int k = 1; k < KS; ++k) mm = fmaxf(mm, sm_m[k * W::kRows + row]);
      f32x4 o = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int k = 0; k < KS; ++k)
        o += *reinterpret_cast<const f32x4*>(sm_o + (size_t)(k * W::kRows + row) * kMergeStride + c4) *
             fast_exp2(sm_m[k * W::kRows + row] - mm);
      *reinterpret_cast<f32x4*>(rec + 3 * p.rpad + row * 128 + c4) = o;
    }
  }
};

LVS_DEV float* record_at(const PagedAttnKernelArgs& p, int64_t i) { return p.ws + i * ((int64_t)p.rpad * 131); }

template <int NB, int RG, int KS>
__global__ __launch_bounds__(64 * RG * KS, 2) void paged_attn_kernel(PagedAttnKernelArgs p) {
  extern __shared__ __align__(256) uint8_t smem[];
  Segment<NB, RG, KS> sg(p, smem);
  const int HR = p.Hkv * p.n_rc;
  const int units = p.B * HR;
  if ((int)blockIdx.x < units) {                 // open rows first: they take the longest chain of steps
    const int u = blockIdx.x, b = u / HR, hr = u - b * HR, h = hr / p.n_rc, rc = hr - h * p.n_rc;
    const int L = paged_len(p.kv_len[b], p.cols);
    sg.begin(b, h, rc);
    sg.open_rows(b, h, L);
    sg.end(rc, record_at(p, (int64_t)p.n_wg + units + u));
    return;
  }
  const int i = blockIdx.x - units;
  // stretches that follow each other go to one XCD, which has the records of a unit in its L2
  const int w = (i & 7) * (p.n_wg >> 3) + (i >> 3);
  const Line line = line_of<KS>(p, sg.lane);
  int at = w * line.per;
  const int end = min(at + line.per, line.total);
  int b0 = 0, before = 0;                        // sequences b0 .. b0+63 at hand, tiles / HR before them
  while (at < end) {
    int full = full_blocks(p, b0 + sg.lane);
    int upto = before + wave_scan(full, sg.lane);
    int all = __builtin_amdgcn_readlane(upto, 63);
    while (at >= all * HR) {                     // (ends: at < total)
      b0 += 64;
      before = all;
      full = full_blocks(p, b0 + sg.lane);
      upto = before + wave_scan(full, sg.lane);
      all = __builtin_amdgcn_readlane(upto, 63);
    }
    const int in = __popcll(__ballot(at >= upto * HR));
    full = __builtin_amdgcn_readlane(full, in);
    const int x = at - (__builtin_amdgcn_readlane(upto, in) - full) * HR;
    const int hr = x / full, t0 = x - hr * full;
    const int t1 = min(full, t0 + end - at);
    const int b = b0 + in, h = hr / p.n_rc, rc = hr - h * p.n_rc;
    sg.begin(b, h, rc);
    sg.blocks(b, h, t0, t1);
    sg.end(rc, record_at(p, (int64_t)w + (int64_t)b * HR + hr));
    at += t1 - t0;
  }
}

// ------------------------------------------------------------------------------ combine
// One workgroup per output row: eight groups of 32 lanes take every eighth record, a lane four channels.
constexpr int kCombineThreads = 256;
constexpr int kCombineMax = 1024;      // records of a row: stretches of the line and its open rows

__global__ __launch_bounds__(kCombineThreads) void paged_combine_kernel(PagedAttnKernelArgs p, int ks) {
  __shared__ float s_w[kCombineMax + 1];
  __shared__ float s_red[3][4];
  __shared__ f32x4 s_o[8][32];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int row = blockIdx.x;                    // (b, kv head, row of its R)
  const int R = p.R, HR = p.Hkv * p.n_rc;
  const int bh = row / R, r = row - bh * R;
  const int b = bh / p.Hkv, h = bh - b * p.Hkv;
  const int rc = r / p.rpad, in = r - rc * p.rpad;
  const int hr = h * p.n_rc + rc;
  const int64_t unit = (int64_t)b * HR + hr;
  // where the unit lies on the line
  int sum = 0, mine = 0;
  for (int b0 = 0; b0 < p.B; b0 += 64) {
    const int f = full_blocks(p, b0 + lane);
    sum += f;
    mine += b0 + lane < b ? f : 0;
  }
#pragma unroll
  for (int d = 32; d > 0; d >>= 1) {
    sum += __shfl_xor(sum, d, 64);
    mine += __shfl_xor(mine, d, 64);
  }
  const int total = __builtin_amdgcn_readfirstlane(sum) * HR;
  const int rounds = (total + p.n_wg * ks - 1) / (p.n_wg * ks);
  const int per = (rounds > 0 ? rounds : 1) * ks;
  const int full = full_blocks(p, b);
  const int from = __builtin_amdgcn_readfirstlane(mine) * HR + hr * full;
  const int w0 = from / per;
  const int n = full > 0 ? (from + full - 1) / per - w0 + 1 : 0;      // records of blocks; one more of open rows
  auto rec = [&](int k) { return record_at(p, k < n ? w0 + k + unit : (int64_t)p.n_wg + p.B * HR + unit); };
  float mm = kNegBig;
  for (int k = tid; k <= n; k += kCombineThreads) {
    const float m = rec(k)[in];
    s_w[k] = m;
    mm = fmaxf(mm, m);
  }
  mm = wave_max(mm);
  if (lane == 0) s_red[0][wave] = mm;
  __syncthreads();
  mm = fmaxf(fmaxf(s_red[0][0], s_red[0][1]), fmaxf(s_red[0][2], s_red[0][3]));
  float l = 0.f, lv = 0.f;
  for (int k = tid; k <= n; k += kCombineThreads) {
    const float f = fast_exp2(s_w[k] - mm);
    const float* x = rec(k);
    l += x[p.rpad + in] * f;
    lv += x[2 * p.rpad + in] * f;
    s_w[k] = f;
  }
  l = wave_sum(l);
  lv = wave_sum(lv);
  if (lane == 0) {
    s_red[1][wave] = l;
    s_red[2][wave] = lv;
  }
  __syncthreads();
  l = (s_red[1][0] + s_red[1][1]) + (s_red[1][2] + s_red[1][3]);
  lv = (s_red[2][0] + s_red[2][1]) + (s_red[2][2] + s_red[2][3]);
  const int g = tid >> 5, c4 = (tid & 31) * 4;
  f32x4 o = {0.f, 0.f, 0.f, 0.f};
  for (int k = g; k <= n; k += 8)
    o += *reinterpret_cast<const f32x4*>(rec(k) + 3 * p.rpad + in * 128 + c4) * s_w[k];
  s_o[g][tid & 31] = o;
  __syncthreads();
  const int i = r / p.G, head = h * p.G + (r - i * p.G);
  if (tid < 32) {
#pragma unroll
    for (int k = 1; k < 8; ++k) o += s_o[k][tid];
    const float inv = 1.f / l;
    uint2 y;
    y.x = pack_bf16(o[0] * inv, o[1] * inv);
    y.y = pack_bf16(o[2] * inv, o[3] * inv);
    *reinterpret_cast<uint2*>(p.out + (int64_t)b * p.o_sb + (int64_t)i * p.o_sg + (int64_t)head * p.o_sh + c4) = y;
  }
  if (tid == 0) {
    const int64_t at = ((int64_t)b * p.Hq + head) * p.gamma + i;
    // ln(sum of exp) from base 2: ln 2 * (m + log2 l)
    if (p.lse != nullptr) p.lse[at] = 0.69314718055994531f * (mm + __log2f(l));
    if (p.vis_mass != nullptr) p.vis_mass[at] = lv / l;
  }
}

template <int NB, int RG, int KS>
hipError_t launch_shape(const PagedAttnKernelArgs& a, hipStream_t stream) {
  static LdsLimitOnce limit;
  const void* fn = reinterpret_cast<const void*>(&paged_attn_kernel<NB, RG, KS>);
  constexpr size_t lds = Shape<NB, RG, KS>::kLds;
  hipError_t e = limit.ensure(fn, lds);
  if (e != hipSuccess) return e;
  const int units = a.B * a.Hkv * a.n_rc;
  paged_attn_kernel<NB, RG, KS><<<dim3((unsigned)(units + a.n_wg)), dim3(64 * RG * KS), lds, stream>>>(a);
  e = hipGetLastError();
  if (e != hipSuccess) return e;
  paged_combine_kernel<<<dim3((unsigned)(a.B * a.Hkv * a.R)), dim3(kCombineThreads), 0, stream>>>(a, KS);
  return hipGetLastError();
}

}  // namespace

int paged_attn_workgroups(int rows, int num_cu) {
  (void)rows;
  const int n = 2 * num_cu / 8 * 8;
  return n < 8 ? 8 : n > kCombineMax ? kCombineMax : n;
}

hipError_t launch_paged_attn(const PagedAttnKernelArgs& a, hipStream_t stream) {
  if (a.rpad <= 16) return launch_shape<1, 1, 4>(a, stream);
  if (a.rpad <= 32) return launch_shape<2, 1, 4>(a, stream);
  return launch_shape<2, 2, 2>(a, stream);
}

}  // namespace lvspec
