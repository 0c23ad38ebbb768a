// Attention over the 8-bit cache (kv8.h) for many query vectors per kv head: prompts and chunks
// of them, large trees.
//
// Bound by the matrix cores and, as closely, by the vector ALUs that the softmax and the
// conversion of the codes need.  A block owns one kv head and 32 NW query vectors (rows x heads
// of the group), 32 to a wavefront, and walks the split's pages NW / 2 pairs a step:
//   * Each wavefront reads one pair's keys or values (as kv8_attention.hip does), converts them to
//     bf16 (keys) or f16 (values) once for the whole block and writes them to LDS in the order in
//     which the products' A operands are read: fragment (K step or dim tile), lane, 8 values.  Reads
//     and writes are 1 KB contiguous per instruction, without bank conflicts.  Two buffers, one
//     barrier a step; the next step's codes are requested before this one's products.
//   * S^T = K Q^T and O^T += V^T P^T as there, 16x16x32, with the queries and outputs of 32 vectors
//     in registers, two wavefronts a SIMD (three with 64-wide heads: 115 -> 97 us for a prompt of
//     4000 rows, 32 heads): one's softmax runs beside the other's products.  (64 vectors would halve
//     the reads of LDS, and need every register of a SIMD for one wavefront: 500 TFLOP/s.)
//   * A operands are read four ahead of the products that take them: with one read in flight at a
//     time, as the compiler orders them, the wavefronts wait for LDS (620 TFLOP/s).
//   * The softmax is kept to what a vector ALU must do a score: one fma, half a maximum, an exp2, half
//     a conversion and half a dot product with ones (the sum, of the rounded P).  All that is rare
//     (masks, maxima that move) sits behind one branch a pair of pages.
// 4 x 1000 rows over 6000 to 9000 positions, 32 heads of 128 over 8: 565 us, 948 TFLOP/s (a large
// bf16 matrix product reaches 1250 here); a prompt of 4099 rows 168 us, 820 TFLOP/s.  The same with
// one wavefront a token range and no LDS (kv8_attention.hip at 64 vectors) took 1010 and 373 us.
// fp32 rows take two products each (hi + lo), so 16 vectors a wavefront: a prompt of 4000 rows 267 us
// (128-wide heads), 163 us (64-wide).
#include <algorithm>
#include <type_traits>

#include "kv8_attn.h"

namespace osp {
namespace {

template <int HD, int NW, bool F32>
__global__ void __launch_bounds__(64 * NW, HD == 64 ? 3 : 2) k_kv8_prompt(Kv8AttnArgs a) {
  constexpr int KC = HD / 32, DT = HD / 16, NT = F32 ? 1 : 2, NP = F32 ? 2 : 1, COLS = 16 * NT * NW, PAIRS = NW / 2;
  typedef typename std::conditional<F32, f16x8, bf16x8>::type qk_t;
  constexpr int RAW = HD / 32;        // 16-byte pieces a lane reads of a pair's keys (values)
  __shared__ uint4 sm_k[2][PAIRS][2][KC][64];
  __shared__ uint4 sm_v[2][PAIRS][DT][64];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int g = blockIdx.x, group = a.nq / a.pool.nkv;
  const int n16 = lane & 15, qr = lane >> 4;
  const Deal deal = deal_of(a, COLS, group, 32 * PAIRS, lane);

  for (int it = blockIdx.y;; it += gridDim.y) {
    Item x;
    if (!find_item(a, deal, it, COLS, group, lane, x)) return;
    const int nvec = (x.s.end - x.s.beg) * group, c0 = x.tile * COLS + wave * (16 * NT);

    // ---- queries and what they see --------------------------------------------------
    qk_t qf[NT][NP][KC];
    float colc[NT], m[NT], l[NT];
    int lim[NT];
    int lim_lo = 0x7fffffff, lim_hi = 0;
    bool missing = false, far = false;   // far: some vector's maximum is (kFar)
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
      const int c = c0 + 16 * nt + n16;
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
    // (the block walks together: to the end of what any of its vectors sees)
    lim_lo = wave_min_i(lim_lo);
    lim_hi = wave_max_i(lim_hi);
    const int last = min((x.tile + 1) * COLS, nvec) - 1;
    const int t_hi = a.tree ? x.s.ctx : min(x.s.ctx, a.r.cached ? x.s.first + last / group + 1 : max(a.r.pos[x.s.beg + last / group], 0) + 1);

    f32x4 acc[NT][DT];
#pragma unroll
    for (int nt = 0; nt < NT; ++nt)
#pragma unroll
      for (int d = 0; d < DT; ++d) acc[nt][d] = f32x4{0.f, 0.f, 0.f, 0.f};

    const int p_lo = x.lo, p_hi = min(x.hi, t_hi);
    const int n_pairs = p_hi > p_lo ? (p_hi - p_lo + 31) / 32 : 0;
    const int n_steps = (n_pairs + PAIRS - 1) / PAIRS;
    // this wavefront's part of a step: keys or values of pair `wave % PAIRS`
    const bool is_v = wave >= PAIRS;
    const int my_pair = wave % PAIRS;
    const long off = is_v ? (long)(a.pool.nkv + g) * (kKv8Page * HD) + qr * 4 * HD + n16 * (HD / 4)
                          : (long)g * (kKv8Page * HD) + n16 * HD + qr * (HD / 4);
    ValueUnit unit;
    float rel = 0.f;   // of the chunk's pages
    uint4 raw[RAW];

    // pages p_lo / 16 + 64 c + lane of chunk c: id (-1: none), scales
    auto page_of = [&](int c) {
      const int t = p_lo + (64 * c + lane) * kKv8Page;
      return t < p_hi ? kv8_page(a.pool, x.b, t / kKv8Page) : -2;
    };
    auto scales_of = [&](int id, float& sk, float& sv) {
      sk = sv = 0.f;
      if (id >= 0) {
        const float* s = a.pool.scales + (long)id * a.pool.scale_stride + 2 * g;
        sk = s[0];
        sv = s[1];
      }
    };
    int id = page_of(0), id_next = page_of(1);
    float sk, sv, sk_next, sv_next;
    scales_of(id, sk, sv);
    // The codes of step s (its pages are in chunk `ids`).
    auto request = [&](int s, int ids) {
      const int at = (s * PAIRS + my_pair) * 2 & 63;
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        const uint8_t* base = a.pool.codes + (long)max(lane_i(ids, at + k), 0) * a.pool.page_stride + off;
#pragma unroll
        for (int i = 0; i < HD / 64; ++i) raw[k * (HD / 64) + i] = *reinterpret_cast<const uint4*>(base + 16 * i);
      }
    };
    auto stage = [&](int s, int buf, int ids) {
      if (is_v) {
        const int t0 = p_lo + (s * PAIRS + my_pair) * 32, at = (s * PAIRS + my_pair) * 2 & 63;
        const bool ok[2] = {lane_i(ids, at) >= 0, lane_i(ids, at + 1) >= 0};
        const float ra = unit.apart ? 1.f : lane_f(rel, at), rb = unit.apart ? 1.f : lane_f(rel, at + 1);
        if (t0 + 32 > p_hi || !ok[0] || !ok[1]) {
          // codes past the split, or of a missing page, may be anything: 0 * NaN
#pragma unroll
          for (int k = 0; k < 2; ++k) {
            const int left = ok[k] ? p_hi - (t0 + 16 * k + 4 * qr) : 0;
            const uint32_t keep = left >= 4 ? 0xffffffffu : left <= 0 ? 0u : (1u << 8 * left) - 1u;
#pragma unroll
            for (int i = 0; i < HD / 64; ++i) {
              uint4& v = raw[k * (HD / 64) + i];
              v = make_uint4(v.x & keep, v.y & keep, v.z & keep, v.w & keep);
            }
          }
        }
#pragma unroll
        for (int d = 0; d < DT; ++d) sm_v[buf][my_pair][d][lane] = __builtin_bit_cast(uint4, frag8(word(raw, d), word(raw, DT + d), ra, rb));
      } else {
#pragma unroll
        for (int k = 0; k < 2; ++k)
#pragma unroll
          for (int c = 0; c < KC; ++c)
          {
            const uint32_t u = word(raw, k * DT + 2 * c), w = word(raw, k * DT + 2 * c + 1);
            if constexpr (F32) sm_k[buf][my_pair][k][c][lane] = __builtin_bit_cast(uint4, frag8(u, w));
            else sm_k[buf][my_pair][k][c][lane] = __builtin_bit_cast(uint4, frag8_bf16(u, w));
          }
      }
    };

    // A new chunk's pages: values go into LDS relative to the largest scale so far (ValueUnit).
    auto enter = [&]() {
      missing |= id == -1;
      const float f = enter_scales(unit, sv, rel);   // (the same in every wavefront)
      if (f != 1.f) {
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
#pragma unroll
          for (int d = 0; d < DT; ++d) acc[nt][d] *= f;
      }
      scales_of(id_next, sk_next, sv_next);
    };
    enter();
    float sk_now = sk;   // scales and pages of the chunk that is computed (the loads are a step ahead)
    int id_now = id;
    if (n_steps > 0) {
      request(0, id);
      stage(0, 0, id);
    }
    __syncthreads();
    auto step = [&](int s, auto apart) {
      const int buf = s & 1, in_chunk = s * PAIRS * 2 & 63;
      if (in_chunk == 0) {
        sk_now = sk;
        id_now = id;
      }
#pragma unroll
      for (int pr = 0; pr < PAIRS; ++pr) {
        const int at = in_chunk + 2 * pr, t0 = p_lo + (s * PAIRS + pr) * 32;
        if (pr == 0 && s + 1 < n_steps) request(s + 1, ((s + 1) * PAIRS * 2 & 63) == 0 ? id_next : id_now);
        if (t0 >= lim_hi) continue;   // (none of this wavefront's vectors sees the pair, or it has none)
        const bool oka = lane_i(id_now, at) >= 0, okb = lane_i(id_now, at + 1) >= 0;
        const float ska = lane_f(sk_now, at), skb = lane_f(sk_now, at + 1);
        const bool whole = t0 + 32 <= min(lim_lo, p_hi) && oka && okb && !far;
        // A operands are read four ahead of the products that take them (left to itself the compiler
        // reads one, waits for it and uses it).
        f32x4 sc[NT][2];
        uint4 fr[2][4];
        const uint4* kp = &sm_k[buf][pr][0][0][lane];
        const uint4* vp = &sm_v[buf][pr][0][lane];
        auto read4 = [&](uint4* f, const uint4* p, int at) {
#pragma unroll
          for (int i = 0; i < 4; ++i) f[i] = p[(at + i) * 64];
        };
        read4(fr[0], kp, 0);
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int nt = 0; nt < NT; ++nt) sc[nt][0] = sc[nt][1] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int i = 0; i < 2 * KC; i += 4) {
          if (i + 4 < 2 * KC) read4(fr[(i / 4 + 1) & 1], kp, i + 4);
          else read4(fr[(i / 4 + 1) & 1], vp, 0);
          __builtin_amdgcn_sched_barrier(0);
#pragma unroll
          for (int j = 0; j < 4; ++j)
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
              for (int p = 0; p < NP; ++p)
                sc[nt][(i + j) / KC] = mfma(__builtin_bit_cast(qk_t, fr[i / 4 & 1][j]), qf[nt][p][(i + j) % KC], sc[nt][(i + j) / KC]);
          __builtin_amdgcn_sched_barrier(0);
        }
        float z[NT][8], top = -INFINITY;
#pragma unroll
        for (int nt = 0; nt < NT; ++nt)
          exponents(sc[nt], score_factor(ska, colc[nt]), score_factor(skb, colc[nt]), kLift - m[nt], z[nt], top);
        // One branch for all that is rare: pairs that some vector sees in part, maxima that move or are far.
        if (!whole || __builtin_amdgcn_ballot_w64(top > kLift + kSlack)) {
#pragma unroll
          for (int nt = 0; nt < NT; ++nt) {
            if (!whole) {
              const uint32_t v = sight_now(a, x, c0 + 16 * nt + n16, group, lim[nt], t0) & in_pair(p_hi - t0, oka, okb);
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
          add_apart<NT, NP, DT>(acc, pf, lane_f(rel, at), lane_f(rel, at + 1), [&](int d) { return __builtin_bit_cast(f16x8, vp[d * 64]); });
          continue;
        }
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int i = 0; i < DT; i += 4) {
          const int f = (2 * KC / 4 + i / 4) & 1;
          if (i + 4 < DT) read4(fr[f ^ 1], vp, i + 4);
          __builtin_amdgcn_sched_barrier(0);
#pragma unroll
          for (int j = 0; j < 4; ++j)
#pragma unroll
            for (int nt = 0; nt < NT; ++nt)
#pragma unroll
              for (int p = 0; p < NP; ++p) acc[nt][i + j] = mfma(__builtin_bit_cast(f16x8, fr[f][j]), pf[nt][p], acc[nt][i + j]);
          __builtin_amdgcn_sched_barrier(0);
        }
      }
      if (s + 1 < n_steps) {
        if (((s + 1) * PAIRS * 2 & 63) == 0) {
          id = id_next;
          sk = sk_next;
          sv = sv_next;
          id_next = page_of((s + 1) * PAIRS * 2 / 64 + 1);
          enter();
        }
        stage(s + 1, buf ^ 1, id);
      }
      __syncthreads();
    };
    // (two loops: with both sums in one, a prompt takes a tenth longer)
    int s0 = 0;
    for (; s0 < n_steps && !unit.apart; ++s0) step(s0, std::false_type{});
    for (; s0 < n_steps; ++s0) step(s0, std::true_type{});
    if (missing && a.err) atomicOr(a.err, 1u << 2);

    // ---- outputs: lane holds dims 16 d + 4 qr .. + 4 of vector n16 of each tile --------
    const bool direct = x.ns == 1 && (a.out || (a.o_hi && !F32));   // one split: no join
#pragma unroll
    for (int nt = 0; nt < NT; ++nt) {
      l[nt] += xor_lane_c(l[nt], 16);
      l[nt] += xor_lane_c(l[nt], 32);
      const int c = c0 + 16 * nt + n16;
      if (c >= nvec) continue;
      const int row = x.s.beg + c / group, h = g * group + c % group;
      if (qr == 0 && x.split == 0 && a.row_ns) a.row_ns[(long)row * a.nq + h] = x.ns;
      if (direct) {
        const float inv = l[nt] > 0.f || l[nt] != l[nt] ? unit.at / l[nt] : 0.f;
        const long at = (long)row * a.ldo + (long)h * HD + 4 * qr;
        if constexpr (F32) {
          float* o = reinterpret_cast<float*>(a.out) + at;
#pragma unroll
          for (int d = 0; d < DT; ++d)
            *reinterpret_cast<float4*>(o + 16 * d) = make_float4(acc[nt][d][0] * inv, acc[nt][d][1] * inv, acc[nt][d][2] * inv, acc[nt][d][3] * inv);
          continue;
        }
        if (a.o_hi) {
#pragma unroll
          for (int d = 0; d < DT; ++d) {
            uint2 hi, lo;
            split_bf16x2(acc[nt][d][0] * inv, acc[nt][d][1] * inv, hi.x, lo.x);
            split_bf16x2(acc[nt][d][2] * inv, acc[nt][d][3] * inv, hi.y, lo.y);
            *reinterpret_cast<uint2*>(a.o_hi + at + 16 * d) = hi;
            *reinterpret_cast<uint2*>(a.o_lo + at + 16 * d) = lo;
          }
          continue;
        }
        bf16_t* o = reinterpret_cast<bf16_t*>(a.out) + at;
#pragma unroll
        for (int d = 0; d < DT; ++d)
          *reinterpret_cast<uint2*>(o + 16 * d) = make_uint2(f32x2_to_bf16x2(acc[nt][d][0] * inv, acc[nt][d][1] * inv),
                                                             f32x2_to_bf16x2(acc[nt][d][2] * inv, acc[nt][d][3] * inv));
      } else {
        float* pp = a.part + (((long)row * a.nq + h) * a.n_split + x.split) * (HD + 2);
        const float back = unit.at * kDownBy;
        if (qr == 0) {
          pp[0] = a.natural ? (m[nt] > kNoMax ? (m[nt] - kLift + kDown) * kLn2 : -INFINITY) : m[nt];
          pp[1] = l[nt] * kDownBy;
        }
#pragma unroll
        for (int d = 0; d < DT; ++d) {
          *reinterpret_cast<float2*>(pp + 2 + 16 * d + 4 * qr) = make_float2(acc[nt][d][0] * back, acc[nt][d][1] * back);
          *reinterpret_cast<float2*>(pp + 4 + 16 * d + 4 * qr) = make_float2(acc[nt][d][2] * back, acc[nt][d][3] * back);
        }
      }
    }
  }
}

}  // namespace

template <int HD>
static void launch_prompt(const Kv8AttnArgs& a, dim3 grid, hipStream_t st) {
  constexpr int NW = kKv8PromptWaves;
  if (a.x_bf16) hipLaunchKernelGGL((k_kv8_prompt<HD, NW, false>), grid, dim3(64 * NW), 0, st, a);
  else hipLaunchKernelGGL((k_kv8_prompt<HD, NW, true>), grid, dim3(64 * NW), 0, st, a);
}

void launch_kv8_prompt(const Kv8AttnArgs& a, dim3 grid, hipStream_t st) {
  if (a.hd == 128) launch_prompt<128>(a, grid, st);
  else launch_prompt<64>(a, grid, st);
}

}  // namespace osp
