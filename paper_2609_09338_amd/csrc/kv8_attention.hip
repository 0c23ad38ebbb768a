// Attention over the 8-bit cache (kv8.h) for few query vectors per kv head: single tokens, the
// rows of a verification, draft trees.
//
//   o_r = sum_t softmax_t(scale q_r . k_t) v_t over the positions t that row r sees
//
// Bound by the codes' bytes.  A block owns one kv head, one tile of 16 NT CT query vectors (rows x
// heads of the group) and one split of the context; its four wavefronts (CT = 2: twice four, each
// four for half of the vectors) take the split's page pairs in turn, straight from memory into
// registers, the next pair requested while this one is computed.  Per pair (32 tokens) a wavefront
// computes
//   S^T[token][query] = K Q^T     (16x16x32, K steps over dims; codes convert exactly)
//   O^T[dim][query] += V^T P^T    (16x16x32, the K index runs over 4 q .. 4 q + 3 of both pages)
// where lane (l % 16, q = l / 16) of the score tile holds exactly the four tokens of each page that
// the second product's B operand wants there: nothing moves between lanes in the loop.
//   * bf16 queries go in as they are, beside codes converted to bf16 (exact).  fp32 queries are
//     scaled by a power of two per vector into f16's range and go in as hi + lo (22 bits, two
//     products) beside f16 codes.
//   * A key block's scale and the softmax scale are one factor of the exponent's fma.  A value
//     block's scale, relative to the largest of the wavefront's pages so far, is an operand of its
//     codes' conversion (scales that lie too far apart for f16: ValueUnit).  P is held in f16 with 2^6 .. 2^14 as its largest value: 11 bits down to
//     2^-20 of it and an absolute 2^-31 below, where bf16's 8 bits would add an error of the output's
//     own rounding.  fp32 rows take P as hi + lo as well.  Maxima, sums and outputs are fp32.
//   * The running maximum only moves when a score passes it by 2^8 (one ballot a pair, no
//     cross-lane traffic otherwise), and then to a whole number: outputs are rescaled by powers of
//     two, exactly.  Scores may have any size that fp32 holds (exponents_masked).  Sums stay per lane
//     until the end.
// Measured, with the join: one token over 131002 positions (8 kv heads of 128) 57 us, 4.7 TB/s; the
// next token of 64 requests of 512 to 4095 positions 68 us, 4.2 TB/s (a copy reaches 4.8); 8 chains of 8
// rows over 4000 positions 23.3 us, 2.8 TB/s; one token over 2048 positions 7 + 3 us of latency.  What
// runs once a wavefront costs its instruction fetches: the code before and after the loop is kept
// short (converting the queries there and unrolled merges took 16 rows over 136 positions 26 us, 13 so).
#include <algorithm>
#include <type_traits>

#include "kv8_attn.h"

namespace osp {
namespace {

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
  OSP_DEV uint32_t kd(int i) const { return word(k, i); }
  OSP_DEV uint32_t vd(int i) const { return word(v, i); }
};

template <int HD, int NT, int CT, bool F32, bool STREAM>
__global__ void __launch_bounds__(256 * CT, NT == 1 || !F32 ? 2 : 1) k_kv8_attn(Kv8AttnArgs a) {
  constexpr int KC = HD / 32;         // K steps of the score product
  constexpr int DT = HD / 16;         // 16-row tiles of dims
  constexpr int NP = F32 ? 2 : 1;     // parts of Q and P
  constexpr int DEPTH = 2;            // pairs in registers
  constexpr int COLS = 16 * NT * CT;
  __shared__ float sm_o[4][COLS][HD + 4];
  __shared__ float sm_m[4][COLS], sm_l[4][COLS];
  const int lane = threadIdx.x & 63, w8 = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int wave = w8 & 3, v0 = (w8 >> 2) * 16 * NT;   // its share of the pages, its first vector
  const int g = blockIdx.x, group = a.nq / a.pool.nkv;
  const int n16 = lane & 15, qr = lane >> 4;
  const Deal deal = deal_of(a, COLS, group, kUnit, lane);
  int at = deal.units ? blockIdx.y * deal.len : blockIdx.y;      // a unit, or an item
  const int at_end = deal.units ? min(at + deal.len, deal.units) : 0;

  for (;;) {
    Item x;
    if (deal.units) {
      if (at >= at_end) return;
      int used;
      find_piece(a, deal, at, at_end, COLS, group, lane, x, used);
      at += used;
    } else {
      if (!find_item(a, deal, at, COLS, group, lane, x)) return;
      at += gridDim.y;
    }
    const int nvec = (x.s.end - x.s.beg) * group, c0 = x.tile * COLS;

    // ---- the split's page pairs: wave, wave + 4, ... ---------------------------------
    // Requested before anything else: the first pages, then the queries, then the scales.
    const int p_lo = x.lo, s_hi = x.hi;
    const long k_off = (long)g * (kKv8Page * HD) + n16 * HD + qr * (HD / 4);
    const long v_off = (long)(a.pool.nkv + g) * (kKv8Page * HD) + qr * 4 * HD + n16 * (HD / 4);
    // 32 of the wavefront's pairs at a time, a page a lane (-1: none, -2: not in the split)
    const int n_pairs = (s_hi - p_lo + 31) / 32, mine = n_pairs > wave ? (n_pairs - wave + 3) / 4 : 0;
    auto pair_at = [&](int i) { return p_lo + (wave + 4 * i) * 32; };
    auto pages_at = [&](int i0) {
      const int i = lane >> 1, t = pair_at(i0 + i) + (lane & 1) * 16;
      return i < mine - i0 && t < s_hi ? kv8_page(a.pool, x.b, t / kKv8Page) : -2;
    };
    int id = pages_at(0);
    Page<HD> buf[DEPTH][2];
    auto request = [&](Page<HD>(&pg)[2], int i) {   // (past the last: any page of the pool, unused)
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        const uint8_t* base = a.pool.codes + (long)max(lane_i(id, min(2 * i + k, 63)), 0) * a.pool.page_stride;
        pg[k].template load<STREAM>(base + k_off, base + v_off);
      }
    };
#pragma unroll
    for (int i = 0; i + 1 < DEPTH; ++i) request(buf[i], i);

    // ---- queries and what they see --------------------------------------------------
    typedef typename std::conditional<F32, f16x8, bf16x8>::type qk_t;
    qk_t qf[NT][NP][KC];
    float colc[NT], m[NT], l[NT];
    int lim[NT];
    int lim_lo = 0x7fffffff, lim_hi = 0;
    bool missing = false;   // a visible position has no page
    bool far = false;       // some vector's maximum is (kFar)
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
      const int c = c0 + v0 + 16 * nt + n16;
      const bool on = c < nvec;
      const int row = x.s.beg + (on ? c / group : 0), h = g * group + (on ? c % group : 0);
      const long at = (long)row * a.ldq + (long)h * HD + qr * (HD / 4);
      colc[nt] = a.scale * kLog2e;
      if constexpr (F32) {
        colc[nt] *= query_parts<HD>(reinterpret_cast<const float*>(a.q) + at, qf[nt][0], qf[nt][NP - 1]);
      } else {
        const uint4* p = reinterpret_cast<const uint4*>(reinterpret_cast<const bf16_t*>(a.q) + at);
#pragma unroll
        for (int i = 0; i < KC; ++i) qf[nt][0][i] = __builtin_bit_cast(bf16x8, p[i]);
      }
      Sight see;
      sight_of(a, x, row, on, see, lim_lo, lim_hi, missing);
      lim[nt] = see.lim;
      m[nt] = kNoMax;
      l[nt] = 0.f;
    }
    lim_lo = wave_min_i(lim_lo);

    f32x4 acc[NT][DT];
#pragma unroll
    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
      for (int d = 0; d < DT; ++d) acc[nt][d] = f32x4{0.f, 0.f, 0.f, 0.f};

    ValueUnit unit;
    float sk = 0.f, rel = 0.f;   // scales of the chunk's pages (keys; values: enter_scales)
    auto enter = [&]() {
      float sv = 0.f;
      sk = 0.f;
      if (id >= 0) {
        const float* s = a.pool.scales + (long)id * a.pool.scale_stride + 2 * g;
        sk = s[0];
        sv = s[1];
      }
      missing |= id == -1;
      const float f = enter_scales(unit, sv, rel);
      if (f != 1.f) {
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
          for (int d = 0; d < DT; ++d) acc[nt][d] *= f;
      }
    };
    auto step = [&](Page<HD>(&pg)[2], int i0, int i, auto apart) {
      const int t0 = pair_at(i0 + i);
      const float ska = lane_f(sk, 2 * i), skb = lane_f(sk, 2 * i + 1);
      const float rva = lane_f(rel, 2 * i), rvb = lane_f(rel, 2 * i + 1);
      const bool oka = lane_i(id, 2 * i) >= 0, okb = lane_i(id, 2 * i + 1) >= 0;
      const bool whole = t0 + 32 <= min(lim_lo, s_hi) && oka && okb && !far;
      f32x4 sc[NT][2];
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) sc[nt][0] = sc[nt][1] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int k = 0; k < 2; ++k)
#pragma unroll
        for (int c = 0; c < KC; ++c) {
          qk_t kf;
          if constexpr (F32) kf = frag8(pg[k].kd(2 * c), pg[k].kd(2 * c + 1));
          else kf = frag8_bf16(pg[k].kd(2 * c), pg[k].kd(2 * c + 1));
#pragma unroll
          for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int p = 0; p < NP; ++p) sc[nt][k] = mfma(kf, qf[nt][p][c], sc[nt][k]);
        }
      float z[NT][8], top = -INFINITY;
#pragma unroll
      for (int nt = 0; nt < NT; ++nt)
        exponents(sc[nt], score_factor(ska, colc[nt]), score_factor(skb, colc[nt]), kLift - m[nt], z[nt], top);
      // One branch for all that is rare: pairs that some vector sees in part, maxima that move or are far.
      if (!whole || __builtin_amdgcn_ballot_w64(top > kLift + kSlack)) {
        if (!whole) {
          // value codes past the context may be anything: 0 * NaN
#pragma unroll
          for (int k = 0; k < 2; ++k) {
            const int left = (k ? okb : oka) ? x.s.ctx - (t0 + 16 * k + 4 * qr) : 0;
            const uint32_t keep = left >= 4 ? 0xffffffffu : left <= 0 ? 0u : (1u << 8 * left) - 1u;
#pragma unroll
            for (int d = 0; d < HD / 64; ++d) {
              uint4& v = pg[k].v[d];
              v = make_uint4(v.x & keep, v.y & keep, v.z & keep, v.w & keep);
            }
          }
        }
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) {
          if (!whole) {
            const uint32_t v = sight_now(a, x, c0 + v0 + 16 * nt + n16, group, lim[nt], t0) & in_pair(s_hi - t0, oka, okb);
            mask_scores(sc[nt][0], v, qr);
            mask_scores(sc[nt][1], v >> 16, qr);
          }
          const float fa = score_factor(ska, colc[nt]), fb = score_factor(skb, colc[nt]);
          float cm = fmaxf(max4(sc[nt][0]) * fa, max4(sc[nt][1]) * fb);
          cm = fmaxf(cm, xor_lane_c(cm, 16));
          cm = fmaxf(cm, xor_lane_c(cm, 32));
          const float w = move_max(m[nt], cm);
          far |= any_far(m[nt]);
          l[nt] *= w;
#pragma unroll
          for (int d = 0; d < DT; ++d) acc[nt][d] *= w;
          exponents_masked(sc[nt], fa, fb, m[nt], far, z[nt], top);
        }
      }
      f16x8 pf[NT][NP];
#pragma unroll
      for (int nt = 0; nt < NT; ++nt) {
        if constexpr (F32) {
          probability_parts(z[nt], l[nt], pf[nt][0], pf[nt][NP - 1]);
        } else {
          uint32_t u[4];
          probabilities(z[nt], l[nt], u);
          probabilities(z[nt] + 4, l[nt], u + 2);
          pf[nt][0] = frag(u[0], u[1], u[2], u[3]);
        }
      }
      if constexpr (apart.value) {
        add_apart<NT, NP, DT>(acc, pf, rva, rvb, [&](int d) { return frag8(pg[0].vd(d), pg[1].vd(d)); });
      } else {
#pragma unroll
        for (int d = 0; d < DT; ++d) {
          const f16x8 vf = frag8(pg[0].vd(d), pg[1].vd(d), rva, rvb);
#pragma unroll
          for (int nt = 0; nt < NT; ++nt)
#pragma unroll
            for (int p = 0; p < NP; ++p) acc[nt][d] = mfma(vf, pf[nt][p], acc[nt][d]);
        }
      }
    };
    int i0 = 0;
    for (; i0 < mine; i0 += 32) {
      const int todo = min(32, mine - i0);
      if (i0 > 0) {
        id = pages_at(i0);
#pragma unroll
        for (int i = 0; i + 1 < DEPTH; ++i) request(buf[i], i);
      }
      enter();
      if (unit.apart) break;
      // (a ring without copies: a copy would wait for its load)
      for (int i = 0; i < todo; i += DEPTH) {
#pragma unroll
        for (int u = 0; u < DEPTH; ++u)
          if (i + u < todo) {
            request(buf[(u + DEPTH - 1) % DEPTH], i + u + DEPTH - 1);
            step(buf[u], i0, i + u, std::false_type{});
          }
      }
    }
    // (a loop of its own: with both sums in one, 64 chains of 8 rows over 2300 positions take 102 us, 74 so)
#pragma unroll 1
    for (; i0 < mine; i0 += 32) {
      id = pages_at(i0);
      enter();
      const int todo = min(32, mine - i0);
#pragma unroll 1
      for (int i = 0; i < todo; ++i) {
        Page<HD> one[2];
        request(one, i);
        step(one, i0, i, std::true_type{});
      }
    }
    if (missing && a.err) atomicOr(a.err, 1u << 2);

    // ---- merge the wavefronts --------------------------------------------------------
    const bool direct = x.ns == 1 && a.out != nullptr;   // one split: no join
    const float back = unit.at * kDownBy;
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
      l[nt] += xor_lane_c(l[nt], 16);
      l[nt] += xor_lane_c(l[nt], 32);
      if (qr == 0) {
        sm_m[wave][v0 + 16 * nt + n16] = m[nt];
        sm_l[wave][v0 + 16 * nt + n16] = l[nt] * kDownBy;
      }
#pragma unroll
      for (int d = 0; d < DT; ++d)
        *reinterpret_cast<float4*>(&sm_o[wave][v0 + 16 * nt + n16][16 * d + 4 * qr]) =
            make_float4(acc[nt][d][0] * back, acc[nt][d][1] * back, acc[nt][d][2] * back, acc[nt][d][3] * back);
    }
    __syncthreads();
#pragma unroll 1
    for (int i = threadIdx.x; i < COLS * HD / 4; i += 256 * CT) {
      const int j = i / (HD / 4), e = i % (HD / 4) * 4, c = c0 + j;
      if (c >= nvec) break;   // (j ascends)
      float M = kNoMax;
#pragma unroll
      for (int w = 0; w < 4; ++w) M = fmaxf(M, sm_m[w][j]);
      float L = 0.f, o[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int w = 0; w < 4; ++w) {
        const float f = M > kNoMax ? exp2f(sm_m[w][j] - M) : 0.f;
        L += sm_l[w][j] * f;
        const float4 v = *reinterpret_cast<const float4*>(&sm_o[w][j][e]);
        o[0] += v.x * f;
        o[1] += v.y * f;
        o[2] += v.z * f;
        o[3] += v.w * f;
      }
      const int row = x.s.beg + c / group, h = g * group + c % group;
      if (e == 0 && x.split == 0 && a.row_ns) a.row_ns[(long)row * a.nq + h] = x.ns;
      if (direct) {
        const float inv = L > 0.f || L != L ? 1.f / L : 0.f;
        const long at = (long)row * a.ldo + (long)h * HD + e;
        if constexpr (F32)
          *reinterpret_cast<float4*>(reinterpret_cast<float*>(a.out) + at) = make_float4(o[0] * inv, o[1] * inv, o[2] * inv, o[3] * inv);
        else
          *reinterpret_cast<uint2*>(reinterpret_cast<bf16_t*>(a.out) + at) =
              make_uint2(f32x2_to_bf16x2(o[0] * inv, o[1] * inv), f32x2_to_bf16x2(o[2] * inv, o[3] * inv));
      } else {
        float* pp = a.part + (((long)row * a.nq + h) * a.n_split + x.split) * (HD + 2);
        *reinterpret_cast<float2*>(pp + 2 + e) = make_float2(o[0], o[1]);
        *reinterpret_cast<float2*>(pp + 4 + e) = make_float2(o[2], o[3]);
        if (e == 0) {
          // (P was lifted by 2^kLift)
          pp[0] = a.natural ? (M > kNoMax ? (M - kLift + kDown) * kLn2 : -INFINITY) : M;
          pp[1] = L;
        }
      }
    }
    __syncthreads();   // (sm_m, sm_l and sm_o are free for the next item)
  }
}

// The splits' outputs, each with weight 2^(m_s - M).  W wavefronts per (row, head) take the splits in
// turn, every one of theirs requested at once: a join is two dependent loads long.
template <int HD, int W>
__global__ void __launch_bounds__(256) k_kv8_join(Kv8AttnArgs a) {
  constexpr int E = HD / 64, PER = 16, G = 4 / W;   // G (row, head) pairs a block
  __shared__ float sm[4][HD];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int i = blockIdx.x * G + wave / W, part = wave % W;
  const int row = i / a.nq, h = i % a.nq;
  const int total = a.r.count ? min(*a.r.count, a.r.rows) : a.r.rows;
  const bool on = row < total && !(a.r.cu && (row < a.r.cu[0] || row >= a.r.cu[a.r.B]));
  const int ns = on ? min(a.row_ns[i], a.n_split) : 0;
  float o[E] = {}, L = 0.f;
  if (ns > 1) {   // (else written by the attention itself)
    const float* pp = a.part + ((long)row * a.nq + h) * a.n_split * (HD + 2);
    const float m = lane < ns ? pp[(long)lane * (HD + 2)] : kNoMax;
    const float ls = lane < ns ? pp[(long)lane * (HD + 2) + 1] : 0.f;
    float f = 0.f;
    for (int s0 = 0; s0 < ns; s0 += PER * W) {
      float v[PER][E];
#pragma unroll
      for (int k = 0; k < PER; ++k) {
        const long s = min(s0 + part + k * W, ns - 1);   // (past the last: read again, weight 0)
#pragma unroll
        for (int e = 0; e < E; ++e) v[k][e] = pp[s * (HD + 2) + 2 + lane * E + e];
      }
      if (s0 == 0) {
        const float M = wave_max(m);
        f = M > kNoMax ? exp2f(m - M) : 0.f;
        L = wave_sum(ls * f);
      }
#pragma unroll
      for (int k = 0; k < PER; ++k) {
        const int s = s0 + part + k * W;
        const float w = s < ns ? lane_f(f, s) : 0.f;
#pragma unroll
        for (int e = 0; e < E; ++e) o[e] += s < ns ? w * v[k][e] : 0.f;
      }
    }
  }
  if constexpr (W > 1) {
#pragma unroll
    for (int e = 0; e < E; ++e) sm[wave][lane * E + e] = o[e];
    __syncthreads();
    if (part > 0) return;
#pragma unroll
    for (int w = 1; w < W; ++w)
#pragma unroll
      for (int e = 0; e < E; ++e) o[e] += sm[wave + w][lane * E + e];
  }
  if (ns <= 1) return;
  const float inv = L > 0.f || L != L ? 1.f / L : 0.f;
  const long at = (long)row * a.ldo + (long)h * HD + lane * E;
#pragma unroll
  for (int e = 0; e < E; ++e) {
    if (a.x_bf16) reinterpret_cast<bf16_t*>(a.out)[at + e] = f32_to_bf16(o[e] * inv);
    else reinterpret_cast<float*>(a.out)[at + e] = o[e] * inv;
  }
}

template <int HD, int NT, int CT>
void launch_cols(const Kv8AttnArgs& a, dim3 grid, hipStream_t st) {
  const dim3 block(256 * CT);
  if (a.x_bf16) {
    if (a.stream) hipLaunchKernelGGL((k_kv8_attn<HD, NT, CT, false, true>), grid, block, 0, st, a);
    else hipLaunchKernelGGL((k_kv8_attn<HD, NT, CT, false, false>), grid, block, 0, st, a);
  } else {
    if (a.stream) hipLaunchKernelGGL((k_kv8_attn<HD, NT, CT, true, true>), grid, block, 0, st, a);
    else hipLaunchKernelGGL((k_kv8_attn<HD, NT, CT, true, false>), grid, block, 0, st, a);
  }
}
template <int HD>
void launch_form(const Kv8AttnArgs& a, int form, dim3 grid, hipStream_t st) {
  if (form == kKv8Narrow) launch_cols<HD, 1, 1>(a, grid, st);
  else if (form == kKv8Shared) launch_cols<HD, 1, 2>(a, grid, st);
  else launch_cols<HD, 2, 1>(a, grid, st);
}

}  // namespace

// Up to 16 query vectors a kv head and sequence: one 16-column tile.  17 to 32: two tiles, either a
// wavefront each over the same pages (8 wavefronts a block: less code and no registers spilled, but
// every page converted twice and half as many pages in flight) or both in one wavefront.  Which, goes by
// the (kv head, position) pairs of the pass.  8 rows of 4 heads, us, each / both, with 128-wide heads:
// 8 sequences of 2000 positions and 8 kv heads 19 / 25, 8 of 3950 24 / 28, 10 of 3950 29 / 33, 12 of 3950
// 37 / 37, 64 of 2300 124 / 74, 32 of 3950 and 2 kv heads 25 / 29, 64 so 41 / 44; 64-wide: 8 of 3950 and
// 8 kv heads 16.4 / 16.9, 32 of 3950 34 / 36.  fp32, where both in one leave one wavefront a SIMD: 8 of
// 3950 27 / 37, 16 of 3950 43 / 51, 64 of 2300 127 / 82.  (The bound dates from slower kernels of the
// first kind; up to twice the pairs the two differ by 4 us at most.)  More vectors: kv8_prompt.hip.
int kv8_attention_form(int x_bf16, int group, int max_rows, long positions, int nkv) {
  const long c = (long)group * max_rows;
  if (c <= 16) return kKv8Narrow;
  if (c > 32) return kKv8Prompt;
  return positions * nkv <= (x_bf16 ? 1 << 18 : 1 << 19) ? kKv8Shared : kKv8Both;
}

void launch_kv8_attention(const Kv8AttnArgs& a, hipStream_t st) {
  long y = (long)a.tiles * a.n_split;
  if (a.by_units) y = a.items;
  else if (a.split_len == 0 && a.n_split > 1) y = std::min<long>(y, (long)a.items + a.tiles);
  const dim3 grid(a.pool.nkv, (unsigned)std::min<long>(std::max<long>(y, 1), 65535));
  if (a.form == kKv8Prompt) return launch_kv8_prompt(a, grid, st);
  if (a.hd == 128) launch_form<128>(a, a.form, grid, st);
  else launch_form<64>(a, a.form, grid, st);
}

void launch_kv8_join(const Kv8AttnArgs& a, hipStream_t st) {
  // few outputs: the latency of a wavefront's loads is the time; many: fewer wavefronts read more each
  const long n = (long)a.r.rows * a.nq;
  if (n <= 1024) {
    const dim3 grid((unsigned)n);
    if (a.hd == 128) hipLaunchKernelGGL((k_kv8_join<128, 4>), grid, dim3(256), 0, st, a);
    else hipLaunchKernelGGL((k_kv8_join<64, 4>), grid, dim3(256), 0, st, a);
  } else {
    const dim3 grid((unsigned)((n + 3) / 4));
    if (a.hd == 128) hipLaunchKernelGGL((k_kv8_join<128, 1>), grid, dim3(256), 0, st, a);
    else hipLaunchKernelGGL((k_kv8_join<64, 1>), grid, dim3(256), 0, st, a);
  }
}

}  // namespace osp
