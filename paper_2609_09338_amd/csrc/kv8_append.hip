// Writing the 8-bit cache (kv8.h): new rows' queries and keys are normalised per head and
// rotated, and keys and values appended to the pages; the accepted path of a draft tree is
// moved to the positions after its context.
//
//   x' = R(pos) (x * gain / sqrt(mean(x^2) + eps)),  R: (a, b) -> (a cos - b sin, b cos + a sin)
//   scale of a block: the smallest 2^E >= amax / 448 over its new tokens, and not below the old
//   one while it holds older tokens; code = rne8(x' / 2^E)
//
// Bound by memory: every projection is read once, every query and code written once.  The
// scale of a block needs all of its new tokens, so a wavefront owns one block (page, kv head,
// keys or values) and holds its 16 hd values in registers: one pass, no LDS, no atomics on
// data, and the same codes whatever else is in the batch.
// A code is a rounding to 4 bits: a key that is off by 2^-24 next to a border changes by a
// sixteenth of itself.  Keys are therefore normalised and rotated in double (half of the fp32
// rate here), and rounded once: codes are those of the definition, not of a summation order.  fp32
// queries are formed so too (6.3e-8 of their size off in fp32, a rounding's 2.5e-8 so; 6000 rows of
// 32 heads 60 and 62 us); bf16 queries, whose rounding is 2^-8, in fp32 (8000 rows of 32 heads of 64
// 31 us, in double 38; 33 since rows outside the sequences are not read), times a power of two where
// their squares would not be fp32; and values need no more.
#include <type_traits>

#include "kv8.h"
#include "kv8_rows.h"

namespace osp {
namespace {

typedef float f32x2 __attribute__((ext_vector_type(2)));

template <typename T> OSP_DEV float gain_at(const void* g, int i) { return load_f32(reinterpret_cast<const T*>(g), i); }
OSP_DEV float gain(const void* g, int bf16, int i) { return bf16 ? gain_at<bf16_t>(g, i) : gain_at<float>(g, i); }

// N consecutive values of row r (N * sizeof(T) a multiple of 8), summed over K-split partials.
template <typename T, int N>
OSP_DEV void load_n(const void* base, long at, int ks, long split, float* x) {
  const T* p = reinterpret_cast<const T*>(base) + at;
  if constexpr (sizeof(T) == 2) {
    if constexpr (N % 8 == 0) {
#pragma unroll
      for (int i = 0; i < N; i += 8) load_vec<bf16_t>(p + i, x + i);
    } else {
      static_assert(N == 2, "");
      const uint32_t u = *reinterpret_cast<const uint32_t*>(p);
      x[0] = bf16_lo(u);
      x[1] = bf16_hi(u);
    }
  } else {
    auto piece = [&](const float* s, float* y, bool add) {
      if constexpr (N % 4 == 0) {
#pragma unroll
        for (int i = 0; i < N; i += 4) {
          const float4 v = *reinterpret_cast<const float4*>(s + i);
          y[i] = add ? y[i] + v.x : v.x;
          y[i + 1] = add ? y[i + 1] + v.y : v.y;
          y[i + 2] = add ? y[i + 2] + v.z : v.z;
          y[i + 3] = add ? y[i + 3] + v.w : v.w;
        }
      } else {
        static_assert(N == 2, "");
        const float2 v = *reinterpret_cast<const float2*>(s);
        y[0] = add ? y[0] + v.x : v.x;
        y[1] = add ? y[1] + v.y : v.y;
      }
    };
    piece(p, x, false);
    for (int k = 1; k < ks; ++k) piece(p + k * split, x, true);
  }
}

// x with its last bit set where the conversion dropped something: rounding the result again to
// fewer bits equals rounding x once.
OSP_DEV float to_float_odd(double x) {
  const float f = (float)x;
  int i = __float_as_int(f);
  if ((double)f != x) {
    if (fabs((double)f) > fabs(x)) --i;   // towards zero
    i |= 1;
  }
  return __int_as_float(i);
}

constexpr double kFloatMax = 3.4028234663852886e38;   // (below 448 2^kKv8MaxExp)

// Smallest E in [kKv8MinExp, kKv8MaxExp] with amax <= 448 2^E.
OSP_DEV int scale_exp(double amax) {
  int e = kKv8MinExp;
  if (amax > 0.0) {
    const long long b = __double_as_longlong(amax);
    // amax in [2^x, 2^(x + 1)); 448 = 1.75 2^8
    const int x = (int)((b >> 52) & 2047) - 1023;
    e = x - 8 + ((b & 0xfffffffffffffll) > 0xc000000000000ll ? 1 : 0);
  }
  return min(max(e, kKv8MinExp), kKv8MaxExp);
}
OSP_DEV int exp_of(float scale) { return min(max((int)((__float_as_uint(scale) >> 23) & 255) - 127, kKv8MinExp), kKv8MaxExp); }

OSP_DEV uint32_t pack4(float a, float b, float c, float d) {
  int u = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
  u = __builtin_amdgcn_cvt_pk_fp8_f32(c, d, u, true);
  return (uint32_t)u;
}
OSP_DEV void unpack4(uint32_t u, float* x) {
  const f32x2 a = __builtin_amdgcn_cvt_pk_f32_fp8((int)u, false), b = __builtin_amdgcn_cvt_pk_f32_fp8((int)u, true);
  x[0] = a[0];
  x[1] = a[1];
  x[2] = b[0];
  x[3] = b[1];
}
OSP_DEV uint32_t shift4(uint32_t u, float f) {
  float x[4];
  unpack4(u, x);
  return pack4(x[0] * f, x[1] * f, x[2] * f, x[3] * f);
}

OSP_DEV double wave_max_d(double v) {
  v = fmax(v, dpp_d<kDppXor1>(v));
  v = fmax(v, dpp_d<kDppXor2>(v));
  v = fmax(v, dpp_d<kDppHalfMirror>(v));
  v = fmax(v, dpp_d<kDppMirror>(v));
  return fmax(fmax(lane_d(v, 0), lane_d(v, 16)), fmax(lane_d(v, 32), lane_d(v, 48)));
}

// A wavefront's lanes over a block.  Keys: token l / 4, dims NE (l % 4) .. + NE of either half.
// Values: tokens 4 (l / 16) .. + 4, dims 16 d + 2 a and the one after, for the ND d's of its half.
template <int HD> struct Lanes {
  static constexpr int NE = HD / 8, ND = HD / 32;
  int t, j;                // keys
  int q, a, dh;            // values
  OSP_DEV explicit Lanes(int lane) : t(lane >> 2), j(lane & 3), q(lane >> 4), a(lane & 7), dh((lane >> 3) & 1) {}
  OSP_DEV int key_at(int half) const { return t * HD + half * (HD / 2) + j * NE; }
  OSP_DEV int value_at(int odd) const { return q * 4 * HD + (2 * a + odd) * (HD / 4) + dh * ND * 4; }
};

// Key codes of lane's 2 NE values at 1 / scale; HD / 8 bytes per half.
template <int HD>
OSP_DEV void store_keys(uint8_t* blk, const Lanes<HD>& L, const float* x) {
  constexpr int NE = HD / 8;
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    uint32_t u[NE / 4];
#pragma unroll
    for (int i = 0; i < NE / 4; ++i) u[i] = pack4(x[h * NE + 4 * i], x[h * NE + 4 * i + 1], x[h * NE + 4 * i + 2], x[h * NE + 4 * i + 3]);
    if constexpr (NE == 16) *reinterpret_cast<uint4*>(blk + L.key_at(h)) = make_uint4(u[0], u[1], u[2], u[3]);
    else *reinterpret_cast<uint2*>(blk + L.key_at(h)) = make_uint2(u[0], u[1]);
  }
}

// Older key codes (tokens before `off`) at a scale 1 / f times theirs.
template <int HD>
OSP_DEV void shift_keys(uint8_t* blk, const Lanes<HD>& L, int off, float f) {
  if (L.t >= off) return;
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    uint32_t* p = reinterpret_cast<uint32_t*>(blk + L.key_at(h));
#pragma unroll
    for (int i = 0; i < HD / 32; ++i) p[i] = shift4(p[i], f);
  }
}

// Value codes of tokens [lo, hi) (x[i][odd][d], token 4 q + i) at 1 / scale; the older ones
// (before lo) at f times their value.  Four tokens share a dword, so a partly new one is merged.
template <int HD>
OSP_DEV void store_values(uint8_t* blk, const Lanes<HD>& L, int lo, int hi, float f, bool shift, const float (*x)[2][HD / 32]) {
  constexpr int ND = HD / 32;
  const int t0 = 4 * L.q;
  const int a = min(max(lo - t0, 0), 4), b = min(max(hi - t0, 0), 4);   // new tokens [a, b) of the four
  if (a >= b && !(shift && a > 0)) return;
  // bytes [a, b): new; [0, a): older; [b, 4): as they are
  const uint32_t below_a = a >= 4 ? 0xffffffffu : (1u << 8 * a) - 1u;
  const uint32_t below_b = b >= 4 ? 0xffffffffu : (1u << 8 * b) - 1u;
  const uint32_t is_new = a < b ? below_b & ~below_a : 0u;
#pragma unroll
  for (int odd = 0; odd < 2; ++odd) {
    uint32_t* p = reinterpret_cast<uint32_t*>(blk + L.value_at(odd));
    uint32_t u[ND];
#pragma unroll
    for (int d = 0; d < ND; ++d) u[d] = pack4(x[0][odd][d], x[1][odd][d], x[2][odd][d], x[3][odd][d]);
    if (is_new != 0xffffffffu) {
#pragma unroll
      for (int d = 0; d < ND; ++d) {
        const uint32_t old = p[d];
        const uint32_t older = shift ? (shift4(old, f) & below_a) | (old & ~below_a) : old;
        u[d] = (u[d] & is_new) | (older & ~is_new);
      }
    }
    if constexpr (ND == 4) *reinterpret_cast<uint4*>(p) = make_uint4(u[0], u[1], u[2], u[3]);
    else *reinterpret_cast<uint2*>(p) = make_uint2(u[0], u[1]);
  }
}

// The sequence of page unit u: sequence b's units begin at cu[b] / 16 + 2 b, which leaves room
// for the pages that its rows touch (at most n / 16 + 2); with a row each, unit b is sequence b's; a single
// sequence has them all.
OSP_DEV int unit_seq(const Kv8Rows& r, int u) {
  if (!r.cu) return r.B == 1 ? 0 : u;
  int lo = 0, hi = r.B - 1;
  while (lo < hi) {
    const int mid = (lo + hi + 1) / 2;
    if (r.cu[mid] / 16 + 2 * mid <= u) lo = mid;
    else hi = mid - 1;
  }
  return lo;
}

template <typename T, int HD>
OSP_DEV void append_keys(const Kv8AppendArgs& a, int b, const Kv8Seq& s, int r0, int off, int n, int g, uint8_t* blk,
                         float* scale, int lane) {
  constexpr int NE = HD / 8;
  const Lanes<HD> L(lane);
  const bool mine = L.t >= off && L.t < off + n;
  const int row = r0 + L.t - off;
  double x[2 * NE];
  bool bad = false;
  if (mine) {
    float f[2 * NE];
#pragma unroll
    for (int h = 0; h < 2; ++h)
      load_n<T, NE>(a.k, (long)row * a.ldk + (long)g * HD + h * (HD / 2) + L.j * NE, a.ks, a.split, f + h * NE);
#pragma unroll
    for (int i = 0; i < 2 * NE; ++i) x[i] = f[i];
  } else {
#pragma unroll
    for (int i = 0; i < 2 * NE; ++i) x[i] = 0.0;
  }
  if (a.k_norm) {
    double ss = 0.0;
#pragma unroll
    for (int i = 0; i < 2 * NE; ++i) ss += x[i] * x[i];
    ss += dpp_d<kDppXor1>(ss);
    ss += dpp_d<kDppXor2>(ss);
    const double inv = 1.0 / sqrt(ss / HD + (double)a.eps);
#pragma unroll
    for (int i = 0; i < 2 * NE; ++i)
      x[i] *= inv * (double)gain(a.k_norm, a.g_bf16, (i / NE) * (HD / 2) + L.j * NE + i % NE);
  }
  if (a.rope_cos && mine) {
    const int p = a.rope_pos ? a.rope_pos[row] : s.first + row - s.beg;
    if ((p < 0 || p >= a.max_pos) && a.err) atomicOr(a.err, 1u << 7);
    const long c = (long)min(max(p, 0), a.max_pos - 1) * (HD / 2) + L.j * NE;
#pragma unroll
    for (int i = 0; i < NE; ++i) {
      const double co = a.rope_cos[c + i], si = a.rope_sin[c + i], u = x[i], w = x[NE + i];
      x[i] = u * co - w * si;
      x[NE + i] = w * co + u * si;
    }
  }
  double amax = 0.0;
#pragma unroll
  for (int i = 0; i < 2 * NE; ++i) {
    if (!(fabs(x[i]) <= kFloatMax)) {   // not finite, or not so once its gain has been applied
      x[i] = 0.0;
      bad = true;
    }
    amax = fmax(amax, fabs(x[i]));
  }
  if (bad && a.err) atomicOr(a.err, 1u << 6);
  amax = wave_max_d(amax);
  const int was = off > 0 ? exp_of(*scale) : kKv8MinExp;
  const int e = max(scale_exp(amax), was);
  if (off > 0 && e > was) shift_keys<HD>(blk, L, off, kv8_pow2(max(was - e, -126)));
  if (mine) {
    const double f = __longlong_as_double((long long)(1023 - e) << 52);
    float y[2 * NE];
#pragma unroll
    for (int i = 0; i < 2 * NE; ++i) y[i] = to_float_odd(x[i] * f);
    store_keys<HD>(blk, L, y);
  }
  if (lane == 0) *scale = kv8_pow2(e);
}

template <typename T, int HD>
OSP_DEV void append_values(const Kv8AppendArgs& a, int r0, int off, int n, int g, uint8_t* blk, float* scale, int lane) {
  constexpr int ND = HD / 32;
  const Lanes<HD> L(lane);
  float x[4][2][ND];
  float amax = 0.f;
  bool bad = false;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int t = 4 * L.q + i;
    const bool mine = t >= off && t < off + n;
#pragma unroll
    for (int d = 0; d < ND; ++d) {
      float f[2] = {0.f, 0.f};
      if (mine) load_n<T, 2>(a.v, (long)(r0 + t - off) * a.ldv + (long)g * HD + 16 * (L.dh * ND + d) + 2 * L.a, a.ks, a.split, f);
#pragma unroll
      for (int o = 0; o < 2; ++o) {
        if (!(fabsf(f[o]) < INFINITY)) {
          f[o] = 0.f;
          bad = true;
        }
        x[i][o][d] = f[o];
        amax = fmaxf(amax, fabsf(f[o]));
      }
    }
  }
  if (bad && a.err) atomicOr(a.err, 1u << 6);
  amax = wave_max(amax);
  const int was = off > 0 ? exp_of(*scale) : kKv8MinExp;
  const int e = max(scale_exp((double)amax), was);
  // 2^-e in two factors: either may lie outside the floats
  const float f0 = kv8_pow2(-e / 2), f1 = kv8_pow2(-e - (-e / 2));
#pragma unroll
  for (int i = 0; i < 4; ++i)
#pragma unroll
    for (int o = 0; o < 2; ++o)
#pragma unroll
      for (int d = 0; d < ND; ++d) x[i][o][d] = x[i][o][d] * f0 * f1;
  store_values<HD>(blk, L, off, off + n, kv8_pow2(max(was - e, -126)), off > 0 && e > was, x);
  if (lane == 0) *scale = kv8_pow2(e);
}

// Position of a row, for its rotation.
OSP_DEV int rope_row(const Kv8AppendArgs& a, int row) {
  if (!a.rope_cos) return 0;
  if (a.rope_pos) return a.rope_pos[row];
  if (a.r.pos) return a.r.pos[row];
  if (!a.r.cu) return a.r.B == 1 ? a.r.cached[0] + row : a.r.cached[row];
  int lo = 0, hi = a.r.B - 1;   // the last sequence that begins at or before the row
  while (lo < hi) {
    const int mid = (lo + hi + 1) / 2;
    if (a.r.cu[mid] <= row) lo = mid;
    else hi = mid - 1;
  }
  return a.r.cached[lo] + row - a.r.cu[lo];
}

template <int C> OSP_DEV float dpp(float v) { return dpp_f<C>(v); }
template <int C> OSP_DEV double dpp(double v) { return dpp_d<C>(v); }

// The sum over a head's LPH lanes.
template <int LPH, typename S> OSP_DEV S head_sum(S v) {
  v += dpp<kDppXor1>(v);
  v += dpp<kDppXor2>(v);
  if constexpr (LPH >= 8) v += dpp<kDppHalfMirror>(v);
  if constexpr (LPH >= 16) v += dpp<kDppMirror>(v);
  return v;
}

// Queries of RQ rows of q from row0 on: HD / (2 V) lanes a head, V values of either half a lane; every
// row's values are requested before the first is used.
template <typename T, int HD, int RQ>
OSP_DEV void do_queries(const Kv8AppendArgs& a, int row0, QueryRows q, int h0, int lane) {
  constexpr int V = Vec<T>::N, LPH = HD / (2 * V);
  const int h = h0 + lane / LPH, j = lane % LPH;
  if (h >= a.nq) return;   // (whole groups of lanes that reduce together)
  float xs[RQ][2 * V];
  int pos[RQ];
#pragma unroll
  for (int r = 0; r < RQ; ++r) {
    const int row = row_read(q, row0 + r);
#pragma unroll
    for (int k = 0; k < 2; ++k)
      load_n<T, V>(a.q, (long)row * a.ldq + (long)h * HD + k * (HD / 2) + j * V, a.ks, a.split, xs[r] + k * V);
  }
#pragma unroll
  for (int r = 0; r < RQ; ++r) pos[r] = rope_row(a, row_read(q, row0 + r));
#pragma unroll
  for (int r = 0; r < RQ; ++r) {
    const int row = row0 + r;
    if (!has_row(q, row)) continue;
    typedef typename std::conditional<sizeof(T) == 4, double, float>::type acc_t;
    acc_t x[2 * V];
#pragma unroll
    for (int i = 0; i < 2 * V; ++i) x[i] = xs[r][i];
    if (a.q_norm) {
      acc_t ss = 0;
#pragma unroll
      for (int i = 0; i < 2 * V; ++i) ss += x[i] * x[i];
      ss = head_sum<LPH>(ss);
      acc_t inv;
      if constexpr (sizeof(T) == 4) {
        inv = 1.0 / sqrt(ss / HD + (double)a.eps);
      } else {
        float eps = a.eps;
        // (not so for NaN) squares near the ends of fp32: the same of the head times a power of two
        if (!(ss < 0x1p120f && ss / HD + eps > 0x1p-90f)) {
          const float by = ss < 1.f ? 0x1p60f : 0x1p-70f;
          eps = eps * by * by;
          ss = 0.f;
#pragma unroll
          for (int i = 0; i < 2 * V; ++i) {
            x[i] *= by;
            ss += x[i] * x[i];
          }
          ss = head_sum<LPH>(ss);
        }
        inv = 1.0f / sqrtf(ss / HD + eps);
      }
#pragma unroll
      for (int i = 0; i < 2 * V; ++i) x[i] *= inv * (acc_t)gain(a.q_norm, a.g_bf16, (i / V) * (HD / 2) + j * V + i % V);
    }
    if (a.rope_cos) {
      const long c = (long)min(max(pos[r], 0), a.max_pos - 1) * (HD / 2) + j * V;
#pragma unroll
      for (int i = 0; i < V; ++i) {
        const acc_t co = a.rope_cos[c + i], si = a.rope_sin[c + i], u = x[i], w = x[V + i];
        x[i] = u * co - w * si;
        x[V + i] = w * co + u * si;
      }
    }
    float z[2 * V];
#pragma unroll
    for (int i = 0; i < 2 * V; ++i) z[i] = (float)x[i];
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      const long at = (long)row * a.ldo + (long)h * HD + k * (HD / 2) + j * V;
      T* o = reinterpret_cast<T*>(a.q_out) + at;
      const float* y = z + k * V;
      if constexpr (sizeof(T) == 2) {
        *reinterpret_cast<uint4*>(o) = make_uint4(f32x2_to_bf16x2(y[0] * a.q_scale, y[1] * a.q_scale), f32x2_to_bf16x2(y[2] * a.q_scale, y[3] * a.q_scale),
                                                  f32x2_to_bf16x2(y[4] * a.q_scale, y[5] * a.q_scale), f32x2_to_bf16x2(y[6] * a.q_scale, y[7] * a.q_scale));
      } else if (a.q_bf16) {
        *reinterpret_cast<uint2*>(reinterpret_cast<bf16_t*>(a.q_out) + at) =
            make_uint2(f32x2_to_bf16x2(y[0] * a.q_scale, y[1] * a.q_scale), f32x2_to_bf16x2(y[2] * a.q_scale, y[3] * a.q_scale));
      } else {
        *reinterpret_cast<float4*>(o) = make_float4(y[0] * a.q_scale, y[1] * a.q_scale, y[2] * a.q_scale, y[3] * a.q_scale);
      }
    }
  }
}
// Queries of group i of RQ rows, heads from h0 on.
template <typename T, int HD, int RQ>
OSP_DEV void query_group(const Kv8AppendArgs& a, int i, int h0, int lane) {
  const int total = a.r.count ? min(*a.r.count, a.r.rows) : a.r.rows;
  const QueryRows q = query_rows(total, a.r.cu ? a.r.cu[0] : 0, a.r.cu ? a.r.cu[a.r.B] : total);
  if (group_has_rows(q, i, RQ)) do_queries<T, HD, RQ>(a, i * RQ, q, h0, lane);
}

// One new token a sequence: a wavefront owns the token's key and value of one kv head, a rotation
// pair of dims (l, l + hd / 2) a lane.  (k_kv8_append holds a page's sixteen tokens; for one it runs
// 16 KB of code once.)  Older codes are touched where the scale grows.
template <typename T, int HD>
__global__ void __launch_bounds__(256) k_kv8_append_one(Kv8AppendArgs a, int units, int q_per_row) {
  constexpr int H = HD / 2, ND = HD / 32;
  const int lane = threadIdx.x & 63;
  const int w = __builtin_amdgcn_readfirstlane(blockIdx.x * 4 + (threadIdx.x >> 6));
  if (w >= units) {
    query_group<T, HD, 1>(a, (w - units) / q_per_row, ((w - units) % q_per_row) * (64 / (HD / (2 * Vec<T>::N))), lane);
    return;
  }
  const int g = w % a.pool.nkv, b = w / a.pool.nkv;
  const Kv8Seq s = kv8_seq(a.r, b);
  if (s.end <= s.beg) return;
  const int row = s.beg, e0 = lane % H, pg = s.first / kKv8Page, off = s.first % kKv8Page;
  const T *kp = reinterpret_cast<const T*>(a.k) + (long)row * a.ldk + (long)g * HD, *vp = reinterpret_cast<const T*>(a.v) + (long)row * a.ldv + (long)g * HD;
  float f[4] = {load_f32(kp, e0), load_f32(kp, e0 + H), load_f32(vp, e0), load_f32(vp, e0 + H)};
  for (int k = 1; k < a.ks; ++k) {
    f[0] += load_f32(kp, e0 + k * a.split);
    f[1] += load_f32(kp, e0 + H + k * a.split);
    f[2] += load_f32(vp, e0 + k * a.split);
    f[3] += load_f32(vp, e0 + H + k * a.split);
  }
  float co = 1.f, si = 0.f;
  if (a.rope_cos) {
    const int p = a.rope_pos ? a.rope_pos[row] : s.first;
    if ((p < 0 || p >= a.max_pos) && a.err) atomicOr(a.err, 1u << 7);
    const long c = (long)min(max(p, 0), a.max_pos - 1) * H + e0;
    co = a.rope_cos[c];
    si = a.rope_sin[c];
  }
  const int id = kv8_page(a.pool, b, pg);
  if (id < 0) {
    if (lane == 0 && a.err) atomicOr(a.err, 1u << 3);
    return;
  }
  uint8_t* kb = a.pool.codes + (long)id * a.pool.page_stride + (long)g * (kKv8Page * HD);
  uint8_t* vb = kb + (long)a.pool.nkv * (kKv8Page * HD);
  float* sc = a.pool.scales + (long)id * a.pool.scale_stride + 2 * g;
  const float was_k = sc[0], was_v = sc[1];
  double x0 = f[0], x1 = f[1];
  if (a.k_norm) {
    double ss = lane < H ? x0 * x0 + x1 * x1 : 0.0;
    ss = wave_sum_d(ss);
    const double inv = 1.0 / sqrt(ss / HD + (double)a.eps);
    x0 *= inv * (double)gain(a.k_norm, a.g_bf16, e0);
    x1 *= inv * (double)gain(a.k_norm, a.g_bf16, e0 + H);
  }
  const double y0 = x0 * (double)co - x1 * (double)si, y1 = x1 * (double)co + x0 * (double)si;
  double kv[2] = {y0, y1};
  bool bad = false;
  double kmax = 0.0;
  float vmax = 0.f;
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    if (!(fabs(kv[i]) <= kFloatMax)) { kv[i] = 0.0; bad = true; }
    if (!(fabsf(f[2 + i]) < INFINITY)) { f[2 + i] = 0.f; bad = true; }
    kmax = fmax(kmax, fabs(kv[i]));
    vmax = fmaxf(vmax, fabsf(f[2 + i]));
  }
  if (bad && a.err) atomicOr(a.err, 1u << 6);
  kmax = wave_max_d(kmax);
  vmax = wave_max(vmax);
  const int wk = off > 0 ? exp_of(was_k) : kKv8MinExp, wv = off > 0 ? exp_of(was_v) : kKv8MinExp;
  const int ek = max(scale_exp(kmax), wk), ev = max(scale_exp((double)vmax), wv);
  if (off > 0 && ek > wk) shift_keys<HD>(kb, Lanes<HD>(lane), off, kv8_pow2(max(wk - ek, -126)));
  if (off > 0 && ev > wv) {
    // (the new token's byte too: written below)
    const float r = kv8_pow2(max(wv - ev, -126));
    uint32_t* p = reinterpret_cast<uint32_t*>(vb);
    for (int i = lane; i < 4 * HD; i += 64) {
      const int live = min(max(off - 4 * (i / HD), 0), 4);   // older tokens of the four
      const uint32_t old = p[i], below = live >= 4 ? 0xffffffffu : (1u << 8 * live) - 1u;
      if (live > 0) p[i] = (shift4(old, r) & below) | (old & ~below);
    }
  }
  if (lane < H) {
    const double rk = __longlong_as_double((long long)(1023 - ek) << 52);
    const float r0 = kv8_pow2(-ev / 2), r1 = kv8_pow2(-ev - (-ev / 2));
    const uint32_t ku = pack4(to_float_odd(kv[0] * rk), to_float_odd(kv[1] * rk), 0.f, 0.f);
    const uint32_t vu = pack4(f[2] * r0 * r1, f[3] * r0 * r1, 0.f, 0.f);
    kb[off * HD + e0] = (uint8_t)ku;
    kb[off * HD + e0 + H] = (uint8_t)(ku >> 8);
    // the dword store above and this byte may come from different lanes
    __builtin_amdgcn_s_waitcnt(0);
    uint8_t* vt = vb + (off / 4) * 4 * HD + off % 4;
    vt[(e0 % 16) * (HD / 4) + (e0 / 16) * 4] = (uint8_t)vu;
    vt[(e0 % 16) * (HD / 4) + (e0 / 16 + ND) * 4] = (uint8_t)(vu >> 8);
  }
  if (lane == 0) {
    sc[0] = kv8_pow2(ek);
    sc[1] = kv8_pow2(ev);
  }
}

// Wavefronts [0, units): blocks of the cache; the rest: queries, one row each or (many) four.
constexpr int kQueryRows = 4;
constexpr long kManyQueries = 4 * 256 * 16;
template <typename T, int HD>
__global__ void __launch_bounds__(256) k_kv8_append(Kv8AppendArgs a, int units, int q_per_row, int many) {
  const int lane = threadIdx.x & 63;
  const int w = __builtin_amdgcn_readfirstlane(blockIdx.x * 4 + (threadIdx.x >> 6));
  if (w < units) {
    // kind and head innermost: the wavefronts of a page's rows run together
    const int kind = w & 1, g = (w >> 1) % a.pool.nkv, u = (w >> 1) / a.pool.nkv;
    const int b = unit_seq(a.r, u);
    const Kv8Seq s = kv8_seq(a.r, b);
    if (s.end <= s.beg) return;
    const int pg = s.first / kKv8Page + u - (a.r.cu ? a.r.cu[b] / 16 + 2 * b : b);   // (b = 0: all of u)
    const int lo = max(s.first, pg * kKv8Page), hi = min(s.first + (s.end - s.beg), (pg + 1) * kKv8Page);
    if (lo >= hi) return;
    const int id = kv8_page(a.pool, b, pg);
    if (id < 0) {
      if (lane == 0 && a.err) atomicOr(a.err, 1u << 3);
      return;
    }
    uint8_t* blk = a.pool.codes + (long)id * a.pool.page_stride + ((long)kind * a.pool.nkv + g) * (kKv8Page * HD);
    float* sc = a.pool.scales + (long)id * a.pool.scale_stride + 2 * g + kind;
    const int off = lo - pg * kKv8Page, r0 = s.beg + lo - s.first;
    if (kind == 0) append_keys<T, HD>(a, b, s, r0, off, hi - lo, g, blk, sc, lane);
    else append_values<T, HD>(a, r0, off, hi - lo, g, blk, sc, lane);
    return;
  }
  const int v = w - units, h0 = (v % q_per_row) * (64 / (HD / (2 * Vec<T>::N)));
  if (many) query_group<T, HD, kQueryRows>(a, v / q_per_row, h0, lane);
  else query_group<T, HD, 1>(a, v / q_per_row, h0, lane);
}

// One block per (sequence, kv head, keys or values): the positions base .. base + n - 1 take the
// codes of base + path[i], a page a wavefront.  path ascends, so a position's source lies at or behind
// it: no page's write reaches the sources of a later page, and once the block has read the sources
// of its pages it may write them in place.
// Bound by the round trips of a page (path, page table, scale and codes, older codes): paths of up to
// 9 positions of 64 sequences, cold pages, 13.5 us (page after page 15.4); one path 5 us.
// Values are carried at 2^-16 of theirs: 256 2^120, to which the largest floats round, is none.
constexpr float kKeepDown = 1.f / 65536.f;
template <int HD>
__global__ void __launch_bounds__(256) k_kv8_keep(Kv8KeepArgs a) {
  constexpr int NE = HD / 8, ND = HD / 32;
  __shared__ int sm_bad;   // the first page that ends the move
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int b = blockIdx.x, g = blockIdx.y >> 1, kind = blockIdx.y & 1;
  const Lanes<HD> L(lane);
  const int base = a.base[b], n = min(a.n[b], a.ld);
  const int32_t* path = a.path + (long)b * a.ld;
  if (n <= 0) return;
  if (base < 0 || base > kKv8MaxPos - n) {
    if (threadIdx.x == 0 && a.err) atomicOr(a.err, 1u << 3);
    return;
  }
  auto block = [&](int id) { return a.pool.codes + (long)id * a.pool.page_stride + ((long)kind * a.pool.nkv + g) * (kKv8Page * HD); };
  auto scale = [&](int id) { return a.pool.scales + (long)id * a.pool.scale_stride + 2 * g + kind; };
  if (threadIdx.x == 0) sm_bad = 0x7fffffff;
  __syncthreads();
  for (int pg0 = base / kKv8Page; pg0 * kKv8Page < base + n; pg0 += 4) {
    const int pg = pg0 + wave;
    const bool on = pg * kKv8Page < base + n;
    const int lo = max(base, pg * kKv8Page), hi = min(base + n, (pg + 1) * kKv8Page), off = lo - pg * kKv8Page;
    const int id = on ? kv8_page(a.pool, b, pg) : -1;
    // source of position pg * 16 + t: its page, token there, and whether it is one
    auto source = [&](int t, int& tok) {
      const int i = pg * kKv8Page + t - base;
      if (i < 0 || i >= n) return -2;
      const int at = path[i];
      if (at < i || (i > 0 && path[i - 1] >= at)) return -1;
      tok = (base + at) % kKv8Page;
      return kv8_page(a.pool, b, (base + at) / kKv8Page);
    };
    bool bad = on && id < 0;
    const float old = id >= 0 && off > 0 ? *scale(id) : 0.f;
    double amax = 0.0;
    float x[2 * NE];                 // keys
    float y[4][2][ND];               // values
    if (kind == 0) {
      int tok = 0;
      const int src = source(L.t, tok);
      bad |= src == -1;
#pragma unroll
      for (int i = 0; i < 2 * NE; ++i) x[i] = 0.f;
      if (src >= 0) {
        const float f = *scale(src) * kKeepDown;
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const uint32_t* p = reinterpret_cast<const uint32_t*>(block(src) + tok * HD + h * (HD / 2) + L.j * NE);
#pragma unroll
          for (int i = 0; i < NE / 4; ++i) unpack4(p[i], x + h * NE + 4 * i);
        }
#pragma unroll
        for (int i = 0; i < 2 * NE; ++i) {
          x[i] *= f;
          amax = fmax(amax, (double)fabsf(x[i]));
        }
      }
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        int tok = 0;
        const int src = source(4 * L.q + i, tok);
        bad |= src == -1;
        const float f = src >= 0 ? *scale(src) * kKeepDown : 0.f;
        const uint8_t* p = block(max(src, 0)) + (tok / 4) * 4 * HD + tok % 4;
#pragma unroll
        for (int o = 0; o < 2; ++o)
#pragma unroll
          for (int d = 0; d < ND; ++d) {
            float v = 0.f;
            if (src >= 0) v = __builtin_amdgcn_cvt_f32_fp8((int)p[(2 * L.a + o) * (HD / 4) + (L.dh * ND + d) * 4], 0) * f;
            y[i][o][d] = v;
            amax = fmax(amax, (double)fabsf(v));
          }
      }
    }
    // (a page without a place, or a path that does not ascend: this sequence's move ends here)
    if (__builtin_amdgcn_ballot_w64(bad) && lane == 0) atomicMin(&sm_bad, pg);
    amax = wave_max_d(amax);
    __syncthreads();   // the sources are read
    const int end = sm_bad;   // (or a page of the next round, which a faster wavefront has found)
    if (pg == end && lane == 0 && a.err) atomicOr(a.err, 1u << 3);
    if (on && pg < end) {
      const int was = off > 0 ? exp_of(old) : kKv8MinExp;
      const int e = max(scale_exp(amax / kKeepDown), was), up = 16 - e;
      const float f0 = kv8_pow2(up / 2), f1 = kv8_pow2(up - up / 2), older = kv8_pow2(max(was - e, -126));
      if (kind == 0) {
        if (off > 0 && e > was) shift_keys<HD>(block(id), L, off, older);
#pragma unroll
        for (int i = 0; i < 2 * NE; ++i) x[i] = x[i] * f0 * f1;
        if (L.t >= off && L.t < off + hi - lo) store_keys<HD>(block(id), L, x);
      } else {
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
          for (int o = 0; o < 2; ++o)
#pragma unroll
            for (int d = 0; d < ND; ++d) y[i][o][d] = y[i][o][d] * f0 * f1;
        store_values<HD>(block(id), L, off, off + hi - lo, older, off > 0 && e > was, y);
      }
      if (lane == 0) *scale(id) = kv8_pow2(e);
    }
    if (end < pg0 + 4) return;
  }
}

}  // namespace

// (a grid holds fewer than 2^32 threads)
constexpr long kMaxWaves = (1L << 26) - 4;
template <typename T, int HD>
bool launch_append(const Kv8AppendArgs& a, hipStream_t st) {
  constexpr int hpw = 64 / (HD / (2 * Vec<T>::N));   // heads a wavefront
  const int q_per_row = a.q ? (a.nq + hpw - 1) / hpw : 1;
  const long q_waves = a.q ? (long)a.r.rows * q_per_row : 0;
  const bool one = !a.r.cu && (a.r.B > 1 || a.r.rows == 1);
  const long units = one ? (long)a.r.B * a.pool.nkv : (a.r.rows / 16 + 2L * a.r.B) * a.pool.nkv * 2;
  // Four rows a wavefront where that still fills the chip (256 CUs of 16 such wavefronts).
  const int many = !one && q_waves >= kManyQueries;
  const long waves = units + (many ? (long)((a.r.rows + kQueryRows - 1) / kQueryRows) * q_per_row : q_waves);
  if (waves > kMaxWaves) return false;
  const dim3 grid((unsigned)((waves + 3) / 4));
  if (one) hipLaunchKernelGGL((k_kv8_append_one<T, HD>), grid, dim3(256), 0, st, a, (int)units, q_per_row);
  else hipLaunchKernelGGL((k_kv8_append<T, HD>), grid, dim3(256), 0, st, a, (int)units, q_per_row, many);
  return true;
}

bool launch_kv8_append(const Kv8AppendArgs& a, hipStream_t st) {
  if (a.x_bf16) return a.hd == 128 ? launch_append<bf16_t, 128>(a, st) : launch_append<bf16_t, 64>(a, st);
  return a.hd == 128 ? launch_append<float, 128>(a, st) : launch_append<float, 64>(a, st);
}

void launch_kv8_keep(const Kv8KeepArgs& a, hipStream_t st) {
  const dim3 grid(a.B, 2 * a.pool.nkv);
  if (a.hd == 128) hipLaunchKernelGGL(k_kv8_keep<128>, grid, dim3(256), 0, st, a);
  else hipLaunchKernelGGL(k_kv8_keep<64>, grid, dim3(256), 0, st, a);
}

}  // namespace osp
