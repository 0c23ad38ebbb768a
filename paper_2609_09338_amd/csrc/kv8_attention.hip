// Attention over the 8-bit cache (kv8.h) for few query vectors per kv head: single tokens, the
// rows of a verification, draft trees.
//
//   o_r = sum_t softmax_t(scale q_r . k_t) v_t over the positions t that row r sees
//
// Bound by the codes' bytes.  A block owns one kv head, one tile of 16 NT query vectors (rows x
// heads of the group) and one split of the context; its four wavefronts take the split's page
// pairs in turn, straight from memory into registers, the next pair requested while this one is
// computed.  Per pair (32 tokens) a wavefront computes
//   S^T[token][query] = K Q^T     (16x16x32, K steps over dims, codes converted to f16: exact)
//   O^T[dim][query] += V^T P^T    (16x16x32, the K index runs over 4 q .. 4 q + 3 of both pages)
// where lane (l % 16, q = l / 16) of the score tile holds exactly the four tokens of each page that
// the second product's B operand wants there: nothing moves between lanes in the loop.
//   * Queries are scaled by a power of two per vector into f16's range: bf16 queries are then
//     exact (f16 keeps 11 bits), fp32 ones go in as hi + lo (22 bits, two products).
//   * A key block's scale and the softmax scale are one factor of the exponent's fma.  A value
//     block's scale, relative to the largest of the wavefront's pages, multiplies P as it is
//     rounded to f16.  P is held with 2^6 .. 2^14 as its largest value: 11 bits down to 2^-20 of it
//     and an absolute 2^-30 below, where bf16's 8 bits would add an error of the output's own
//     rounding.  fp32 rows take P as hi + lo as well.  Maxima, sums and outputs are fp32.
//   * The running maximum only moves when a score passes it by 2^8 (one ballot a pair, no
//     cross-lane traffic otherwise); sums stay per lane until the end.
#include <algorithm>

#include "kv8.h"

namespace osp {
namespace {

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));

constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;
constexpr float kNoMax = -1.0e30f;   // below any score: a row that has seen nothing
constexpr float kLift = 6.f;         // P's largest value is 2^kLift, 2^(kLift + kSlack) before the maximum moves
constexpr float kSlack = 8.f;

OSP_DEV uint32_t h2(f16x2 v) { return __builtin_bit_cast(uint32_t, v); }
OSP_DEV uint32_t codes_f16(uint32_t u, bool hi) {
  return hi ? h2(__builtin_amdgcn_cvt_scalef32_pk_f16_fp8(u, 1.f, true)) : h2(__builtin_amdgcn_cvt_scalef32_pk_f16_fp8(u, 1.f, false));
}
OSP_DEV f16x8 frag(uint32_t a, uint32_t b, uint32_t c, uint32_t d) { return __builtin_bit_cast(f16x8, make_uint4(a, b, c, d)); }
// Eight codes (two dwords) as f16.
OSP_DEV f16x8 frag8(uint32_t a, uint32_t b) {
  return frag(codes_f16(a, false), codes_f16(a, true), codes_f16(b, false), codes_f16(b, true));
}
OSP_DEV f32x4 mfma(f16x8 a, f16x8 b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0); }

template <bool STREAM>
OSP_DEV uint4 load16(const uint8_t* p) {
  typedef uint32_t u4 __attribute__((ext_vector_type(4)));
  if constexpr (STREAM) {
    const u4 v = __builtin_nontemporal_load(reinterpret_cast<const u4*>(p));
    return make_uint4(v[0], v[1], v[2], v[3]);
  } else {
    return *reinterpret_cast<const uint4*>(p);
  }
}

// A lane's share of one page's keys and values: HD / 4 bytes of each.
template <int HD> struct Page {
  uint4 k[HD / 64], v[HD / 64];
  template <bool STREAM> OSP_DEV void load(const uint8_t* kp, const uint8_t* vp) {
#pragma unroll
    for (int i = 0; i < HD / 64; ++i) k[i] = load16<STREAM>(kp + 16 * i);
#pragma unroll
    for (int i = 0; i < HD / 64; ++i) v[i] = load16<STREAM>(vp + 16 * i);
  }
  OSP_DEV uint32_t kd(int i) const { return reinterpret_cast<const uint32_t*>(k)[i]; }
  OSP_DEV uint32_t vd(int i) const { return reinterpret_cast<const uint32_t*>(v)[i]; }
};

// What a block works on.
struct Item {
  Kv8Seq s;
  int b, tile, split, ns;
};

// Rows of sequence b and what they can see: no more than its table holds.
OSP_DEV Kv8Seq attn_seq(const Kv8AttnArgs& a, int b) {
  Kv8Seq s = kv8_seq(a.r, b);
  s.ctx = min(s.ctx, a.pool.max_pages * kKv8Page);
  return s;
}

// Splits of a pass.  split_len: the caller's, or an even deal of the tiles' positions over the
// items that the launch aims at, no finer than the quantum and no more than n_split a sequence.
OSP_DEV int plan_len(const Kv8AttnArgs& a, int cols, int group, int quantum, int lane) {
  if (a.split_len > 0) return a.split_len;
  float work = 0.f;
  int longest = 1;
  for (int b0 = 0; b0 < a.r.B; b0 += 64) {
    const int b = b0 + lane;
    if (b < a.r.B) {
      const Kv8Seq s = attn_seq(a, b);
      work += (float)(((s.end - s.beg) * group + cols - 1) / cols) * (float)s.ctx;
      longest = max(longest, s.ctx);
    }
  }
  if (a.r.B > 1) {
    work = wave_sum(work);
    longest = wave_max_i(longest);
  } else {
    work = lane_f(work, 0);
    longest = lane_i(longest, 0);
  }
  const float even = work / (float)a.items;
  int len = even < 1.0e9f ? (int)even + 1 : 1000000000;
  len = max(len, (longest + a.n_split - 1) / a.n_split);
  return (len + quantum - 1) / quantum * quantum;
}

// Item `it` of the pass: sequences in order, their tiles last to first (the last rows of a prompt
// see most), a tile's splits in order.  False: there are fewer.
OSP_DEV bool find_item(const Kv8AttnArgs& a, int it, int len, int cols, int group, int lane, Item& x) {
  int before = 0;
  for (int b0 = 0; b0 < a.r.B; b0 += 64) {
    const int b = b0 + lane;
    int tiles = 0, ns = 0;
    if (b < a.r.B) {
      const Kv8Seq s = attn_seq(a, b);
      tiles = ((s.end - s.beg) * group + cols - 1) / cols;
      ns = (s.ctx + len - 1) / len;
    }
    const int n = tiles * ns;
    const int incl = a.r.B > 1 ? wave_incl_scan<int>(n) : n;
    const uint64_t past = __builtin_amdgcn_ballot_w64(b < a.r.B && before + incl > it);
    if (past) {
      const int l = __builtin_ctzll(past);
      x.b = b0 + l;
      x.ns = lane_i(ns, l);
      const int at = it - before - (lane_i(incl, l) - lane_i(n, l));
      x.tile = lane_i(tiles, l) - 1 - at / x.ns;
      x.split = at % x.ns;
      x.s = attn_seq(a, x.b);
      return true;
    }
    before += lane_i(incl, 63);
    if (a.r.B <= 64) break;
  }
  return false;
}

// What a row sees: the positions before `lim`; with a tree those before `base` (the sequence's
// first new position) and base + i for the set bits i of w.
struct Sight {
  int lim;
  uint64_t w0, w1;
};
// Bit i: the row sees position t0 + i (i < 32).
OSP_DEV uint32_t sight32(const Sight& s, bool tree, int base, int t0) {
  const int n = s.lim - t0;
  uint32_t v = n >= 32 ? 0xffffffffu : n <= 0 ? 0u : (1u << n) - 1u;
  if (tree) {
    const int r = t0 - base;
    if (r >= 128) v = 0u;
    else if (r >= 64) v &= (uint32_t)(s.w1 >> (r - 64));
    else if (r > 32) v &= (uint32_t)(s.w0 >> r | s.w1 << (64 - r));
    else if (r >= 0) v &= (uint32_t)(s.w0 >> r);
    else if (r > -32) v &= (uint32_t)s.w0 << -r | ((1u << -r) - 1u);
  }
  return v;
}

template <int HD, int NT, bool F32, bool STREAM>
__global__ void __launch_bounds__(256) k_kv8_attn(Kv8AttnArgs a) {
  constexpr int KC = HD / 32;         // K steps of the score product
  constexpr int DT = HD / 16;         // 16-row tiles of dims
  constexpr int NP = F32 ? 2 : 1;     // parts of Q and P
  constexpr int COLS = 16 * NT;
  __shared__ float sm_o[4][16][HD + 4];
  __shared__ float sm_m[4][COLS], sm_l[4][COLS];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int g = blockIdx.x, group = a.nq / a.pool.nkv;
  const int n16 = lane & 15, qr = lane >> 4;
  const int len = plan_len(a, COLS, group, 128, lane);

  for (int it = blockIdx.y;; it += gridDim.y) {
    Item x;
    if (!find_item(a, it, len, COLS, group, lane, x)) return;
    const int nvec = (x.s.end - x.s.beg) * group, c0 = x.tile * COLS;

    // ---- queries and what they see --------------------------------------------------
    f16x8 qf[NT][NP][KC];
    float colc[NT], m[NT], l[NT];
    Sight see[NT];
    int lim_lo = 0x7fffffff, lim_hi = 0;
    bool missing = false;   // a visible position has no page
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
      const int c = c0 + 16 * nt + n16;
      const bool on = c < nvec;
      const int row = x.s.beg + (on ? c / group : 0), h = g * group + (on ? c % group : 0);
      float q[HD / 4];
      if (F32) {
        const float* p = reinterpret_cast<const float*>(a.q) + (long)row * a.ldq + (long)h * HD + qr * (HD / 4);
#pragma unroll
        for (int i = 0; i < HD / 4; i += 4) load_vec<float>(p + i, q + i);
      } else {
        const bf16_t* p = reinterpret_cast<const bf16_t*>(a.q) + (long)row * a.ldq + (long)h * HD + qr * (HD / 4);
#pragma unroll
        for (int i = 0; i < HD / 4; i += 8) load_vec<bf16_t>(p + i, q + i);
      }
      float big = 0.f;
#pragma unroll
      for (int i = 0; i < HD / 4; ++i) big = fmaxf(big, fabsf(q[i]));
      big = fmaxf(big, xor_lane_c(big, 16));
      big = fmaxf(big, xor_lane_c(big, 32));
      // 2^up takes the vector's largest magnitude into [2^13, 2^14)
      const int e = (int)((__float_as_uint(big) >> 23) & 255) - 127;
      const int up = big > 0.f && big < INFINITY ? min(max(13 - e, -114), 120) : 0;
      const float f = kv8_pow2(up);
      colc[nt] = kv8_pow2(-up) * (a.scale * kLog2e);
#pragma unroll
      for (int c8 = 0; c8 < KC; ++c8) {
        f16x8 hi, lo;
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          const float v = q[c8 * 8 + j] * f;
          hi[j] = (_Float16)v;
          lo[j] = (_Float16)(v - (float)hi[j]);
        }
        qf[nt][0][c8] = hi;
        if constexpr (F32) qf[nt][NP - 1][c8] = lo;
      }
      see[nt].lim = 0;
      see[nt].w0 = see[nt].w1 = 0;
      if (on) {
        see[nt].lim = a.r.cached ? x.s.first + row - x.s.beg + 1 : max(a.r.pos[row], 0) + 1;
        if (a.tree) {
          see[nt].lim = x.s.ctx;
          see[nt].w0 = a.tree[2 * (long)row];
          see[nt].w1 = a.tree[2 * (long)row + 1];
        }
        missing |= see[nt].lim > x.s.ctx;
        see[nt].lim = min(see[nt].lim, x.s.ctx);
        lim_lo = min(lim_lo, a.tree ? min(x.s.first, x.s.ctx) : see[nt].lim);
        lim_hi = max(lim_hi, see[nt].lim);
      }
      m[nt] = kNoMax;
      l[nt] = 0.f;
    }
    lim_lo = wave_min_i(lim_lo);
    lim_hi = wave_max_i(lim_hi);

    f32x4 acc[NT][DT];
#pragma unroll
    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
      for (int d = 0; d < DT; ++d) acc[nt][d] = f32x4{0.f, 0.f, 0.f, 0.f};

    // ---- the split's page pairs: wave, wave + 4, ... ---------------------------------
    const int p_lo = x.split * len, p_hi = min(p_lo + len, lim_hi);
    const int n_pairs = p_hi > p_lo ? (p_hi - p_lo + 31) / 32 : 0;
    const int mine = n_pairs > wave ? (n_pairs - wave + 3) / 4 : 0;
    const long k_off = (long)g * (kKv8Page * HD) + lane % 16 * HD + qr * (HD / 4);
    const long v_off = (long)(a.pool.nkv + g) * (kKv8Page * HD) + qr * 4 * HD + n16 * (HD / 4);
    float eref = 0.f;     // largest value scale so far (0: none)
    // 32 pairs at a time: a page and its scales a lane
    for (int i0 = 0; i0 < mine; i0 += 32) {
      const int todo = min(32, mine - i0);
      const int t_lane = p_lo + (wave + 4 * (i0 + (lane >> 1))) * 32 + (lane & 1) * 16;
      int id = 0;
      float sk = 0.f, sv = 0.f;
      const bool has = (lane >> 1) < todo && t_lane < p_hi;
      if (has) {
        id = kv8_page(a.pool, x.b, t_lane / kKv8Page);
        missing |= id < 0;
        if (id >= 0) {
          const float* s = a.pool.scales + (long)id * a.pool.scale_stride + 2 * g;
          sk = s[0];
          sv = s[1];
        }
      }
      const int ok = id >= 0 && has;
      id = max(id, 0);
      // values relative to the largest scale: P times it stays within f16
      const float top = fmaxf(eref, wave_max(fabsf(sv)));
      if (top > eref) {
        if (eref > 0.f) {
          const float f = eref / top;
#pragma unroll
          for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int d = 0; d < DT; ++d) acc[nt][d] *= f;
        }
        eref = top;
      }
      const float rel = eref > 0.f ? sv / eref : 0.f;

      Page<HD> buf[2][2];
      auto request = [&](Page<HD>(&pg)[2], int i) {
#pragma unroll
        for (int k = 0; k < 2; ++k) {
          const uint8_t* base = a.pool.codes + (long)lane_i(id, min(2 * i + k, 63)) * a.pool.page_stride;
          pg[k].template load<STREAM>(base + k_off, base + v_off);
        }
      };
      auto step = [&](Page<HD>(&pg)[2], int i) {
        const int t0 = p_lo + (wave + 4 * (i0 + i)) * 32;
        const float ska = lane_f(sk, 2 * i), skb = lane_f(sk, 2 * i + 1);
        const float rva = lane_f(rel, 2 * i), rvb = lane_f(rel, 2 * i + 1);
        const bool oka = lane_i(ok, 2 * i) != 0, okb = lane_i(ok, 2 * i + 1) != 0;
        const bool whole = t0 + 32 <= min(lim_lo, p_hi) && oka && okb;
        f16x8 kf[2][KC];
#pragma unroll
        for (int k = 0; k < 2; ++k)
#pragma unroll
          for (int c = 0; c < KC; ++c) kf[k][c] = frag8(pg[k].kd(2 * c), pg[k].kd(2 * c + 1));
        if (!whole) {
          // value codes past the context may be anything: 0 * NaN
#pragma unroll
          for (int k = 0; k < 2; ++k) {
            const int left = (k ? okb : oka) ? x.s.ctx - (t0 + 16 * k + 4 * qr) : 0;
            const uint32_t keep = left >= 4 ? 0xffffffffu : left <= 0 ? 0u : (1u << 8 * left) - 1u;
#pragma unroll
            for (int d = 0; d < HD / 64; ++d) {
              pg[k].v[d].x &= keep;
              pg[k].v[d].y &= keep;
              pg[k].v[d].z &= keep;
              pg[k].v[d].w &= keep;
            }
          }
        }
        f16x8 pf[NT][NP];
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
          f32x4 s[2] = {f32x4{0.f, 0.f, 0.f, 0.f}, f32x4{0.f, 0.f, 0.f, 0.f}};
#pragma unroll
          for (int k = 0; k < 2; ++k)
#pragma unroll
            for (int c = 0; c < KC; ++c)
#pragma unroll
              for (int p = 0; p < NP; ++p) s[k] = mfma(kf[k][c], qf[nt][p][c], s[k]);
          const float fa = ska * colc[nt], fb = skb * colc[nt];
          float y[8];
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            y[e] = s[0][e] * fa;
            y[4 + e] = s[1][e] * fb;
          }
          if (!whole) {
            const int end = p_hi - t0;
            const uint32_t in = (end >= 32 ? 0xffffffffu : (1u << end) - 1u) & (oka ? 0xffffffffu : 0xffff0000u) & (okb ? 0xffffffffu : 0xffffu);
            const uint32_t sight = (sight32(see[nt], a.tree != nullptr, x.s.first, t0) & in) >> (4 * qr);
#pragma unroll
            for (int e = 0; e < 8; ++e) {
              if (!(sight >> ((e >> 2) * 16 + (e & 3)) & 1)) y[e] = -INFINITY;
            }
          }
          const float mx = fmaxf(fmaxf(fmaxf(y[0], y[1]), fmaxf(y[2], y[3])), fmaxf(fmaxf(y[4], y[5]), fmaxf(y[6], y[7])));
          if (__builtin_amdgcn_ballot_w64(mx > m[nt] + kSlack)) {
            float cm = fmaxf(mx, xor_lane_c(mx, 16));
            cm = fmaxf(cm, xor_lane_c(cm, 32));
            const float mn = fmaxf(m[nt], cm);
            const float f = exp2f(m[nt] - mn);
            m[nt] = mn;
            l[nt] *= f;
#pragma unroll
            for (int d = 0; d < DT; ++d) acc[nt][d] *= f;
          }
          const float off = kLift - m[nt];
          float p[8];
#pragma unroll
          for (int e = 0; e < 8; ++e) p[e] = __builtin_amdgcn_exp2f(y[e] + off);
          l[nt] += ((p[0] + p[1]) + (p[2] + p[3])) + ((p[4] + p[5]) + (p[6] + p[7]));
          f16x8 hi, lo;
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            const float w = p[e] * (e < 4 ? rva : rvb);
            hi[e] = (_Float16)w;
            if constexpr (F32) lo[e] = (_Float16)(w - (float)hi[e]);
          }
          pf[nt][0] = hi;
          if constexpr (F32) pf[nt][NP - 1] = lo;
        }
#pragma unroll
        for (int d = 0; d < DT; ++d) {
          const f16x8 vf = frag8(pg[0].vd(d), pg[1].vd(d));
#pragma unroll
          for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int p = 0; p < NP; ++p) acc[nt][d] = mfma(vf, pf[nt][p], acc[nt][d]);
        }
      };
      request(buf[0], 0);
      for (int i = 0; i < todo; i += 2) {
        request(buf[1], i + 1);   // (past the last: page 0 of the pool or the last one's neighbour, unused)
        step(buf[0], i);
        if (i + 1 < todo) {
          request(buf[0], i + 2);
          step(buf[1], i + 1);
        }
      }
    }
    if (missing && a.err) atomicOr(a.err, 1u << 2);

    // ---- merge the wavefronts --------------------------------------------------------
    const bool direct = x.ns == 1 && a.out != nullptr;   // one split: no join
    const float vs = eref > 0.f ? eref : 0.f;
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
      l[nt] += xor_lane_c(l[nt], 16);
      l[nt] += xor_lane_c(l[nt], 32);
      if (qr == 0) {
        sm_m[wave][16 * nt + n16] = m[nt];
        sm_l[wave][16 * nt + n16] = l[nt];
      }
    }
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
      __syncthreads();   // (the tile before has been read)
#pragma unroll
      for (int d = 0; d < DT; ++d)
        *reinterpret_cast<float4*>(&sm_o[wave][n16][16 * d + 4 * qr]) =
            make_float4(acc[nt][d][0] * vs, acc[nt][d][1] * vs, acc[nt][d][2] * vs, acc[nt][d][3] * vs);
      __syncthreads();
      for (int i = threadIdx.x; i < 16 * HD / 4; i += 256) {
        const int j = i / (HD / 4), e = i % (HD / 4) * 4, c = c0 + 16 * nt + j;
        if (c >= nvec) continue;
        float M = kNoMax;
#pragma unroll
        for (int w = 0; w < 4; ++w) M = fmaxf(M, sm_m[w][16 * nt + j]);
        float L = 0.f, o[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int w = 0; w < 4; ++w) {
          const float f = exp2f(sm_m[w][16 * nt + j] - M);
          L += sm_l[w][16 * nt + j] * f;
          const float4 v = *reinterpret_cast<const float4*>(&sm_o[w][j][e]);
          o[0] += v.x * f;
          o[1] += v.y * f;
          o[2] += v.z * f;
          o[3] += v.w * f;
        }
        const int row = x.s.beg + c / group, h = g * group + c % group;
        if (e == 0 && h == 0 && x.split == 0 && a.row_ns) a.row_ns[row] = x.ns;
        if (direct) {
          const float inv = L > 0.f || L != L ? 1.f / L : 0.f;
          const long at = (long)row * a.ldo + (long)h * HD + e;
          if (a.x_bf16)
            *reinterpret_cast<uint2*>(reinterpret_cast<bf16_t*>(a.out) + at) =
                make_uint2(f32x2_to_bf16x2(o[0] * inv, o[1] * inv), f32x2_to_bf16x2(o[2] * inv, o[3] * inv));
          else
            *reinterpret_cast<float4*>(reinterpret_cast<float*>(a.out) + at) = make_float4(o[0] * inv, o[1] * inv, o[2] * inv, o[3] * inv);
        } else {
          float* pp = a.part + (((long)row * a.nq + h) * a.n_split + x.split) * (HD + 2);
          *reinterpret_cast<float2*>(pp + 2 + e) = make_float2(o[0], o[1]);
          *reinterpret_cast<float2*>(pp + 4 + e) = make_float2(o[2], o[3]);
          if (e == 0) {
            // (P was lifted by 2^kLift)
            pp[0] = a.natural ? (M > kNoMax ? (M - kLift) * kLn2 : -INFINITY) : M;
            pp[1] = L;
          }
        }
      }
    }
    __syncthreads();   // (sm_m, sm_l and sm_o are free for the next item)
  }
}

// One wavefront per (row, head): the splits' outputs, each with weight 2^(m_s - M).
template <int HD>
__global__ void __launch_bounds__(256) k_kv8_join(Kv8AttnArgs a) {
  constexpr int E = HD / 64;
  const int lane = threadIdx.x & 63;
  const int w = __builtin_amdgcn_readfirstlane(blockIdx.x * 4 + (threadIdx.x >> 6));
  const int row = w / a.nq, h = w % a.nq;
  const int total = a.r.count ? min(*a.r.count, a.r.rows) : a.r.rows;
  if (row >= total || (a.r.cu && row >= a.r.cu[a.r.B])) return;
  const int ns = min(a.row_ns[row], a.n_split);
  if (ns <= 1) return;   // (written by the attention itself)
  const float* pp = a.part + ((long)row * a.nq + h) * a.n_split * (HD + 2);
  const float m = lane < ns ? pp[(long)lane * (HD + 2)] : kNoMax;
  const float ls = lane < ns ? pp[(long)lane * (HD + 2) + 1] : 0.f;
  const float M = wave_max(m);
  const float f = exp2f(m - M);
  const float L = wave_sum(ls * f);
  float o[E] = {};
  for (int s = 0; s < ns; ++s) {
    const float ws = lane_f(f, s);
#pragma unroll
    for (int e = 0; e < E; ++e) o[e] += ws * pp[(long)s * (HD + 2) + 2 + lane * E + e];
  }
  const float inv = L > 0.f || L != L ? 1.f / L : 0.f;
  const long at = (long)row * a.ldo + (long)h * HD + lane * E;
#pragma unroll
  for (int e = 0; e < E; ++e) {
    if (a.x_bf16) reinterpret_cast<bf16_t*>(a.out)[at + e] = f32_to_bf16(o[e] * inv);
    else reinterpret_cast<float*>(a.out)[at + e] = o[e] * inv;
  }
}

template <int HD, int NT>
void launch_cols(const Kv8AttnArgs& a, dim3 grid, hipStream_t st) {
  if (a.x_bf16) {
    if (a.stream) hipLaunchKernelGGL((k_kv8_attn<HD, NT, false, true>), grid, dim3(256), 0, st, a);
    else hipLaunchKernelGGL((k_kv8_attn<HD, NT, false, false>), grid, dim3(256), 0, st, a);
  } else {
    if (a.stream) hipLaunchKernelGGL((k_kv8_attn<HD, NT, true, true>), grid, dim3(256), 0, st, a);
    else hipLaunchKernelGGL((k_kv8_attn<HD, NT, true, false>), grid, dim3(256), 0, st, a);
  }
}

// 16-column tiles of a launch: enough for a sequence's query vectors, at most four.
int cols_nt(int group, int max_rows) {
  const long c = (long)group * max_rows;
  return c <= 16 ? 1 : c <= 32 ? 2 : 4;
}

}  // namespace

int kv8_attention_tiles(int rows, int B, int group, int max_rows) {
  const int cols = 16 * cols_nt(group, max_rows);
  return (int)((long)rows * group / cols) + B;
}

void launch_kv8_attention(const Kv8AttnArgs& a, int max_rows, hipStream_t st) {
  const int nt = cols_nt(a.nq / a.pool.nkv, max_rows);
  long y = (long)a.tiles * a.n_split;
  if (a.split_len == 0 && a.n_split > 1) y = std::min<long>(y, (long)a.items + a.tiles);
  const dim3 grid(a.pool.nkv, (unsigned)std::min<long>(std::max<long>(y, 1), 65535));
  if (a.hd == 128) {
    if (nt == 1) launch_cols<128, 1>(a, grid, st);
    else if (nt == 2) launch_cols<128, 2>(a, grid, st);
    else launch_cols<128, 4>(a, grid, st);
  } else {
    if (nt == 1) launch_cols<64, 1>(a, grid, st);
    else if (nt == 2) launch_cols<64, 2>(a, grid, st);
    else launch_cols<64, 4>(a, grid, st);
  }
}

void launch_kv8_join(const Kv8AttnArgs& a, hipStream_t st) {
  const dim3 grid((unsigned)(((long)a.r.rows * a.nq + 3) / 4));
  if (a.hd == 128) hipLaunchKernelGGL(k_kv8_join<128>, grid, dim3(256), 0, st, a);
  else hipLaunchKernelGGL(k_kv8_join<64>, grid, dim3(256), 0, st, a);
}

}  // namespace osp
