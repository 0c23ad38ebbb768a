// Device code that the attention kernels over the 8-bit cache share: conversions, the deal of
// the work, what a row sees.
#pragma once

#include "kv8.h"

namespace osp {
namespace {

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));

constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;
constexpr float kNoMax = -INFINITY;  // the maximum of a row that has seen nothing
constexpr float kLift = 6.f;         // P's largest value is 2^kLift, 2^(kLift + kSlack) before the maximum moves
constexpr float kSlack = 8.f;
constexpr float kFar = 16777216.f;   // 2^24: from here on neighbouring floats are 2 and more apart
// Sums and outputs leave a wavefront at 2^-kDown: P reaches 2^14, and a sum of 2^18 such of the largest
// values fits.  Nothing that counts falls below: a row's sum is 2^5 at least, and the largest value of a
// block of the smallest scale, 2^-91, is 2^31 of the smallest floats there.
constexpr float kDown = 32.f, kDownBy = 0x1p-32f;

OSP_DEV uint32_t h2(f16x2 v) { return __builtin_bit_cast(uint32_t, v); }
// Two of a dword's codes as f16, times a power of two.
OSP_DEV uint32_t codes_f16(uint32_t u, bool hi, float r) {
  return hi ? h2(__builtin_amdgcn_cvt_scalef32_pk_f16_fp8(u, r, true)) : h2(__builtin_amdgcn_cvt_scalef32_pk_f16_fp8(u, r, false));
}
OSP_DEV f16x8 frag(uint32_t a, uint32_t b, uint32_t c, uint32_t d) { return __builtin_bit_cast(f16x8, make_uint4(a, b, c, d)); }
// Dword i of a lane's 16-byte pieces (i a constant once loops are unrolled: the pieces stay in registers).
OSP_DEV uint32_t word(const uint4* r, int i) {
  const uint4& v = r[i >> 2];
  switch (i & 3) {
    case 0: return v.x;
    case 1: return v.y;
    case 2: return v.z;
    default: return v.w;
  }
}
// Eight codes (two dwords) as f16, times ra and rb.
OSP_DEV f16x8 frag8(uint32_t a, uint32_t b, float ra = 1.f, float rb = 1.f) {
  return frag(codes_f16(a, false, ra), codes_f16(a, true, ra), codes_f16(b, false, rb), codes_f16(b, true, rb));
}
// Eight codes as bf16: the key operand beside bf16 queries, which go in as they are.
OSP_DEV uint32_t codes_bf16(uint32_t u, bool hi) {
  return hi ? __builtin_bit_cast(uint32_t, (bf16x2)__builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(u, 1.f, true))
            : __builtin_bit_cast(uint32_t, (bf16x2)__builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(u, 1.f, false));
}
OSP_DEV bf16x8 frag8_bf16(uint32_t a, uint32_t b) {
  return __builtin_bit_cast(bf16x8, make_uint4(codes_bf16(a, false), codes_bf16(a, true), codes_bf16(b, false), codes_bf16(b, true)));
}
OSP_DEV f32x4 mfma(bf16x8 a, bf16x8 b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0); }
OSP_DEV f32x4 mfma(f16x8 a, f16x8 b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0); }

// What a block works on.
struct Item {
  Kv8Seq s;
  int b, tile, split, ns;
  int lo, hi;     // positions
};

// Rows of sequence b and what they can see: no more than its table holds.
OSP_DEV Kv8Seq attn_seq(const Kv8AttnArgs& a, int b) {
  Kv8Seq s = kv8_seq(a.r, b);
  s.ctx = min(s.ctx, a.pool.max_pages * kKv8Page);
  return s;
}

// The deal of a pass.  Up to 64 sequences are read once, one a lane.
//   by splits  an item is one split of `len` positions of one tile
//   by units   (where a.by_units allows it) the tiles' contexts lie end to end in units of kUnit positions, and every
//              block takes the same number of them, whichever sequences they fall in: a block that is
//              left with a whole split of a long sequence reads alone at the end (64 sequences of 512
//              to 4095 positions by splits: 80 us)
constexpr int kUnit = 128;
struct Deal {
  Kv8Seq mine;    // sequence `lane`
  int len;        // positions of a split, or units of a block
  int units;      // by units: all of them (else 0)
};
OSP_DEV Kv8Seq seq_or_none(const Kv8AttnArgs& a, int b) {
  Kv8Seq s{0, 0, 0, 0};
  if (b < a.r.B) s = attn_seq(a, b);
  return s;
}
OSP_DEV int tiles_of(const Kv8Seq& s, int cols, int group) { return ((s.end - s.beg) * group + cols - 1) / cols; }
OSP_DEV int units_of(const Kv8Seq& s) { return (s.ctx + kUnit - 1) / kUnit; }

// split_len: the caller's, or an even deal of the tiles' positions over the items that the launch
// aims at, no finer than the quantum (a unit) and no more than n_split a sequence.
OSP_DEV Deal deal_of(const Kv8AttnArgs& a, int cols, int group, int quantum, int lane) {
  Deal d;
  d.mine = seq_or_none(a, lane);
  d.len = a.split_len;
  d.units = 0;
  if (d.len > 0) return d;
  float work = 0.f;
  int longest = 1, units = 0;
  for (int b0 = 0; b0 < a.r.B; b0 += 64) {
    const Kv8Seq s = b0 == 0 ? d.mine : seq_or_none(a, b0 + lane);
    if (a.by_units) units += tiles_of(s, cols, group) * units_of(s);
    else work += (float)tiles_of(s, cols, group) * (float)s.ctx;
    longest = max(longest, s.ctx);
  }
  longest = wave_max_i(longest);
  if (a.by_units) {
    units = lane_i(wave_incl_scan<int>(units), 63);
    d.len = kUnit;
    if (units == 0) return d;   // no row, no item
    const int even = (units + a.items - 1) / a.items;
    // By splits where they come out even: a split a block, at most a quarter longer than the even deal
    // (a second piece costs a block about as much as two or three units).
#pragma unroll 1
    for (int k = 0; k < 3; ++k) {
      const int len = even * (8 + k) / 8, whole = (longest + kUnit - 1) / kUnit;
      if ((whole + len - 1) / len > a.n_split) continue;
      int n = 0;
      for (int b0 = 0; b0 < a.r.B; b0 += 64) {
        const Kv8Seq s = b0 == 0 ? d.mine : seq_or_none(a, b0 + lane);
        n += tiles_of(s, cols, group) * ((units_of(s) + len - 1) / len);
      }
      if (lane_i(wave_incl_scan<int>(n), 63) <= a.items) {
        d.len = len * kUnit;
        return d;
      }
    }
    d.units = units;
    d.len = even;
    // (a tile may begin and end inside a block's range: one split more)
    d.len = max(d.len, ((longest + kUnit - 1) / kUnit + a.n_split - 2) / (a.n_split - 1));
    return d;
  }
  work = wave_sum(work);
  const float even = work / (float)a.items;
  d.len = even < 1.0e9f ? (int)even + 1 : 1000000000;
  d.len = max(d.len, (longest + a.n_split - 1) / a.n_split);
  d.len = (d.len + quantum - 1) / quantum * quantum;
  return d;
}

// By units: what lies at unit p of a block's range [.., end): a piece of one tile, positions
// [x.lo, x.hi), `used` units long.
OSP_DEV void find_piece(const Kv8AttnArgs& a, const Deal& d, int p, int end, int cols, int group, int lane, Item& x, int& used) {
  int before = 0;
  for (int b0 = 0; b0 < a.r.B; b0 += 64) {
    const Kv8Seq s = b0 == 0 ? d.mine : seq_or_none(a, b0 + lane);
    const int tiles = tiles_of(s, cols, group), u = units_of(s), n = tiles * u;
    const int incl = wave_incl_scan<int>(n);
    const uint64_t past = __builtin_amdgcn_ballot_w64(before + incl > p);
    if (past) {
      const int l = __builtin_ctzll(past), ul = lane_i(u, l);
      const int at = p - before - (lane_i(incl, l) - lane_i(n, l)), t = at / ul, o = at % ul;
      const int begin = p - o;                      // where the tile begins
      used = min(ul - o, end - p);
      x.b = b0 + l;
      x.tile = lane_i(tiles, l) - 1 - t;
      x.split = p / d.len - begin / d.len;
      x.ns = (begin + ul - 1) / d.len - begin / d.len + 1;
      x.s = Kv8Seq{lane_i(s.beg, l), lane_i(s.end, l), lane_i(s.first, l), lane_i(s.ctx, l)};
      x.lo = o * kUnit;
      x.hi = min((o + used) * kUnit, x.s.ctx);
      return;
    }
    before += lane_i(incl, 63);
  }
  used = end - p;   // (not reached: p < units)
  x.lo = x.hi = 0;
  x.tile = x.split = x.b = 0;
  x.ns = 1;
  x.s = Kv8Seq{0, 0, 0, 0};
}

// Item `it` of the pass: sequences in order, their tiles last to first (the last rows of a prompt
// see most), a tile's splits in order.  False: there are fewer.
OSP_DEV bool find_item(const Kv8AttnArgs& a, const Deal& d, int it, int cols, int group, int lane, Item& x) {
  int before = 0;
  for (int b0 = 0; b0 < a.r.B; b0 += 64) {
    const Kv8Seq s = b0 == 0 ? d.mine : seq_or_none(a, b0 + lane);
    const int tiles = tiles_of(s, cols, group), ns = min((s.ctx + d.len - 1) / d.len, a.n_split);
    const int n = tiles * ns;
    const int incl = wave_incl_scan<int>(n);
    const uint64_t past = __builtin_amdgcn_ballot_w64(before + incl > it);
    if (past) {
      const int l = __builtin_ctzll(past);
      x.b = b0 + l;
      x.ns = lane_i(ns, l);
      const int at = it - before - (lane_i(incl, l) - lane_i(n, l));
      x.tile = lane_i(tiles, l) - 1 - at / x.ns;
      x.split = at % x.ns;
      x.s = Kv8Seq{lane_i(s.beg, l), lane_i(s.end, l), lane_i(s.first, l), lane_i(s.ctx, l)};
      x.lo = x.split * d.len;
      x.hi = min(x.lo + d.len, x.s.ctx);
      return true;
    }
    before += lane_i(incl, 63);
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

// A row's place in the pass: what it sees, the tile's shortest and longest view, and whether
// some of it lies past the table.
OSP_DEV void sight_of(const Kv8AttnArgs& a, const Item& x, int row, bool on, Sight& s, int& lo, int& hi, bool& missing) {
  s.lim = 0;
  s.w0 = s.w1 = 0;
  if (!on) return;
  s.lim = a.r.cached ? x.s.first + row - x.s.beg + 1 : max(a.r.pos[row], 0) + 1;
  if (a.tree) {
    s.lim = x.s.ctx;
    s.w0 = a.tree[2 * (long)row];
    s.w1 = a.tree[2 * (long)row + 1];
  }
  missing |= s.lim > x.s.ctx;
  s.lim = min(s.lim, x.s.ctx);
  lo = min(lo, a.tree ? min(x.s.first, x.s.ctx) : s.lim);
  hi = max(hi, s.lim);
}

// sight32 of vector c of the item's sequence, its tree words read now: few tokens need them.
OSP_DEV uint32_t sight_now(const Kv8AttnArgs& a, const Item& x, int c, int group, int lim, int t0) {
  Sight s{lim, 0, 0};
  if (a.tree && lim > 0 && t0 + 32 > x.s.first) {
    const long row = x.s.beg + c / group;
    s.w0 = a.tree[2 * row];
    s.w1 = a.tree[2 * row + 1];
  }
  return sight32(s, a.tree != nullptr, x.s.first, t0);
}

// The tokens of a pair (bit i: the i-th) that lie in the split (`end`: its positions from the
// pair's first one on) and on a page.
OSP_DEV uint32_t in_pair(int end, bool oka, bool okb) {
  return (end >= 32 ? 0xffffffffu : end <= 0 ? 0u : (1u << end) - 1u) & (oka ? 0xffffffffu : 0xffff0000u) & (okb ? 0xffffffffu : 0xffffu);
}
// The lane's four scores of a page's tokens 4 qr + e: -inf where bit 4 qr + e of `sight` is clear.
OSP_DEV void mask_scores(f32x4& s, uint32_t sight, int qr) {
  const uint32_t v = sight >> (4 * qr);
#pragma unroll
  for (int e = 0; e < 4; ++e)
    if (!(v >> e & 1)) s[e] = -INFINITY;
}
// The factor of a page's scores: never zero, so that a masked one stays -inf (a large query over small keys
// has a use for the smallest).
OSP_DEV float score_factor(float sk, float colc) { return fmaxf(sk * colc, 1.4e-45f); }
OSP_DEV float max4(f32x4 s) { return fmaxf(fmaxf(s[0], s[1]), fmaxf(s[2], s[3])); }

// The power of two that takes a query vector's largest magnitude into [2^13, 2^14).
OSP_DEV int query_exp(float big) {
  const int e = (int)((__float_as_uint(big) >> 23) & 255) - 127;
  return big > 0.f && big < INFINITY ? min(max(13 - e, -114), 120) : 0;
}

// The lane's HD / 4 dims of an fp32 query vector as f16 parts hi + lo at a power of two of their own;
// returns the factor that undoes it.
template <int HD>
OSP_DEV float query_parts(const float* p, f16x8* hi, f16x8* lo) {
  float q[HD / 4], big = 0.f;
#pragma unroll
  for (int i = 0; i < HD / 4; i += 4) load_vec<float>(p + i, q + i);
#pragma unroll
  for (int i = 0; i < HD / 4; ++i) big = fmaxf(big, fabsf(q[i]));
  big = fmaxf(big, xor_lane_c(big, 16));
  big = fmaxf(big, xor_lane_c(big, 32));
  const int up = query_exp(big);
  const float f = kv8_pow2(up);
#pragma unroll
  for (int i = 0; i < HD / 4; ++i) {
    const float v = q[i] * f;
    hi[i / 8][i % 8] = (_Float16)v;
    lo[i / 8][i % 8] = (_Float16)(v - (float)hi[i / 8][i % 8]);
  }
  return kv8_pow2(-up);
}

// The unit of a wavefront's outputs.  Value codes go into the product relative to the largest value scale
// so far, as f16: exact down to 2^-15 of it (a code is a multiple of 2^-9, an f16 of 2^-24).  But scales of
// one pass may span 2^220, and the largest may belong to positions that a row does not see.  A wavefront
// that meets a scale below 2^-15 of its unit (a page of zeros has one), or whose unit has grown by more
// than 2^60 (up to there fp32 outputs hold what they had), goes on in a fixed unit, 2^kDown: codes
// unscaled, a product for each page, which joins the outputs at the page's scale (add_apart).
struct ValueUnit {
  float at = 0.f;       // the unit (0: no page yet)
  float first = 0.f;    // what it was at first
  bool apart = false;   // it is fixed
};
// A chunk's pages with value scales sv (0: none) join.  rel: the factor of a page's codes, or (apart) of
// its product.  Returns the factor for the outputs so far.
OSP_DEV float enter_scales(ValueUnit& u, float sv, float& rel) {
  rel = sv * kDownBy;
  if (u.apart) return 1.f;
  const float was = u.at, top = fmaxf(was, wave_max(sv));
  if (was == 0.f) u.first = top;
  const float r = top > 0.f ? sv / top : 0.f;
  u.at = top;
  u.apart = __builtin_amdgcn_ballot_w64((sv > 0.f && r < 0x1p-15f) || top * 0x1p-60f > u.first) != 0;
  if (u.apart) {
    u.at = 1.f / kDownBy;
    return was > 0.f ? was * kDownBy : 1.f;
  }
  rel = r;
  return was > 0.f ? was / top : 1.f;
}
// A lane's share of P for a pair's first (second) page alone.
OSP_DEV f16x8 page_of_pair(f16x8 p, int second) {
  const uint4 v = __builtin_bit_cast(uint4, p);
  return second ? frag(0u, 0u, v.z, v.w) : frag(v.x, v.y, 0u, 0u);
}
// acc[] += V P of a pair, a page at a time at its own factor; codes(d): its unscaled codes, dims 16 d ..
template <int NT, int NP, int DT, typename Codes>
OSP_DEV void add_apart(f32x4 (&acc)[NT][DT], const f16x8 (&p)[NT][NP], float fa, float fb, Codes codes) {
#pragma unroll 1
  for (int k = 0; k < 2; ++k) {
    const float f = k ? fb : fa;
    f16x8 one[NT][NP];
#pragma unroll
    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
      for (int i = 0; i < NP; ++i) one[nt][i] = page_of_pair(p[nt][i], k);
#pragma unroll
    for (int d = 0; d < DT; ++d) {
      const f16x8 vf = codes(d);
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) {
        f32x4 t = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int i = 0; i < NP; ++i) t = mfma(vf, one[nt][i], t);
#pragma unroll
        for (int e = 0; e < 4; ++e) acc[nt][d][e] = __builtin_fmaf(t[e], f, acc[nt][d][e]);
      }
    }
  }
}

// P = 2^z of a lane's eight exponents as f16 parts hi + lo; its sum joins l.
OSP_DEV void probability_parts(const float* z, float& l, f16x8& hi, f16x8& lo) {
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    const float p = __builtin_amdgcn_exp2f(z[e]);
    l += p;
    hi[e] = (_Float16)p;
    lo[e] = (_Float16)(p - (float)hi[e]);
  }
}

// P = 2^z of a lane's four exponents as f16; its sum (of the rounded values) joins l.
OSP_DEV void probabilities(const float* z, float& l, uint32_t* u) {
  const f16x2 one = {(_Float16)1.f, (_Float16)1.f};
#pragma unroll
  for (int e = 0; e < 2; ++e) {
    const f16x2 h = {(_Float16)__builtin_amdgcn_exp2f(z[2 * e]), (_Float16)__builtin_amdgcn_exp2f(z[2 * e + 1])};
    l = __builtin_amdgcn_fdot2(h, one, l, false);
    u[e] = h2(h);
  }
}
// z = s f + up of a pair's eight scores; their maximum joins top.
OSP_DEV void exponents(const f32x4* s, float fa, float fb, float up, float* z, float& top) {
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    z[e] = __builtin_fmaf(s[e >> 2][e & 3], e < 4 ? fa : fb, up);
    top = fmaxf(top, z[e]);
  }
}

// A maximum m takes in the largest of a pair's scores; returns the factor of sums and outputs so far.  (By
// differences: they are exact where they matter, m + kSlack is not.  Nothing seen yet, -inf: any score moves
// it, and none leaves it, by NaN.)
OSP_DEV float move_max(float& m, float cm) {
  const float was = m;
  if (cm - m > kSlack) m = ceilf(cm);
  return m > was ? exp2f(was - m) : 1.f;
}
OSP_DEV bool is_far(float m) { return fabsf(m) >= kFar && fabsf(m) < INFINITY; }
OSP_DEV bool any_far(float m) { return __builtin_amdgcn_ballot_w64(is_far(m)) != 0; }
// The exponents of a pair that may be masked, or (far) where some vector's maximum lies kFar or more from
// zero.  There a score's product must be rounded as its maximum's was: what the fma keeps below that rounding
// is as large as P's whole range, and the largest P would be 0 or infinite.
OSP_DEV void exponents_masked(const f32x4* s, float fa, float fb, float m, bool far, float* z, float& top) {
  const float at = m > kNoMax ? m : 0.f;   // (nothing seen: every score is -inf)
  exponents(s, fa, fb, kLift - at, z, top);
  if (!far) return;
#pragma unroll
  for (int e = 0; e < 8; ++e) {
#pragma clang fp contract(off)
    const float t = s[e >> 2][e & 3] * (e < 4 ? fa : fb);
    z[e] = is_far(m) ? (t - at) + kLift : z[e];
  }
}

}  // namespace
}  // namespace osp
