// The paged key/value cache held in 8 bits: layout, arguments and the device code that its
// kernels share (kv8_append.hip, kv8_attention.hip).  Not part of the public C ABI.
//
// A page holds 16 positions.  Per page and kv head there is a block of 16 hd key codes and
// one of 16 hd value codes, e4m3 (OCP; finite, magnitudes up to 448), each with one scale, a
// power of two: value = code * scale.  With scales that are powers of two a code moves from
// one scale to a larger one by its exponent alone: exact until it falls below 2^-6 of the
// scale, where e4m3 steps are even.  There a block whose scale grew while tokens were appended
// has been rounded twice, and a code may be a step from what a single pass would have kept (the
// first rounding can land on a tie).  A scale never shrinks while older tokens stay.
//
// Layout of a block.  Keys are token-major [16][hd]: lane (token l % 16, quarter l / 16) of a
// wavefront reads hd / 4 contiguous bytes, its share of every K step of S^T = K Q^T.  Values
// are [4][16][hd / 16][4] (token t, dim e at [t / 4][e % 16][e / 16][t % 4]): lane (e % 16 =
// l % 16, t / 4 = l / 16) reads hd / 4 contiguous bytes, the four tokens of its K index in
// O^T += V^T P^T for every 16-row tile of dims.  Either way a wavefront reads a block as one
// contiguous piece, 16 bytes a lane, and no code moves between lanes.
#pragma once

#include "common.h"
#include "internal.h"

namespace osp {

constexpr int kKv8Page = 16;
constexpr int kKv8MinExp = -100;   // smallest scale 2^-100 (an all-zero block)
constexpr int kKv8MaxExp = 120;    // 448 * 2^120 holds every finite float
constexpr int kKv8MaxSplits = 64;  // splits of a context: a lane each in a join
constexpr int kKv8MaxPos = 1 << 30;

struct Kv8Pool {
  const int32_t* table;     // [rows][max_pages] physical pages
  int max_pages;
  int num_pages;
  const int32_t* slot;      // table row of sequence b (nullable: b)
  const int32_t* nblocks;   // pages of a table row (nullable: max_pages)
  uint8_t* codes;           // page p at codes + p * page_stride: [2 (k, v)][nkv][16 hd]
  long page_stride;         // bytes
  float* scales;            // page p at scales + p * scale_stride: [nkv][2 (k, v)]
  long scale_stride;        // floats
  int nkv;
};

// The rows of a pass: sequence b has rows [cu[b], cu[b + 1]) (cu nullable: row b; a single
// sequence: every row), at positions
// cached[b] + j, or pos[row] where cached is null (ascending within a sequence; or all alike,
// rows that see the same context).
struct Kv8Rows {
  int B;
  int rows;                 // host bound on the rows
  const int32_t* count;     // device row count (nullable: rows)
  const int32_t* cu;
  const int32_t* cached;
  const int32_t* pos;
};

struct Kv8AppendArgs {
  Kv8Pool pool;
  Kv8Rows r;
  const int32_t* rope_pos;  // [rows] (nullable: the row's position)
  int x_bf16;               // q, k, v and q_out: bf16 (else fp32; q_out by q_bf16)
  int g_bf16;               // gains: bf16 (else fp32)
  const void *q, *k, *v;    // row r at + r * ld (elements); heads contiguous (q nullable)
  long ldq, ldk, ldv;
  int ks;                   // fp32 partial sums to add, `split` elements apart (1: plain)
  long split;
  int nq, hd;
  const void *q_norm, *k_norm;   // [hd] (nullable: no norm)
  float eps;
  const float *rope_cos, *rope_sin;   // [max_pos][hd / 2] (nullable: no rotation)
  int max_pos;
  void* q_out;              // row r at + r * ldo: [nq][hd]
  long ldo;
  int q_bf16;               // fp32 rows: q_out is bf16
  float q_scale;
  uint32_t* err;            // (nullable)
};
// False, and nothing enqueued: more blocks and rows than a grid holds.
bool launch_kv8_append(const Kv8AppendArgs& a, hipStream_t st);

struct Kv8KeepArgs {
  Kv8Pool pool;
  int B, hd;
  const int32_t* base;      // [B]
  const int32_t* path;      // [B][ld]
  int ld;
  const int32_t* n;         // [B]
  uint32_t* err;
};
void launch_kv8_keep(const Kv8KeepArgs& a, hipStream_t st);

struct Kv8AttnArgs {
  Kv8Pool pool;
  Kv8Rows r;
  int x_bf16;               // q and out: bf16 (else fp32)
  const void* q;            // row r at + r * ldq: [nq][hd]
  long ldq;
  int nq, hd;
  float scale;
  const uint64_t* tree;     // [rows][2] bit i: the row sees position cached + i (nullable: causal)
  int form;                 // kKv8Narrow ..
  int n_split;              // partials per row and head
  int split_len;            // positions per split (0: planned on the device from the lengths)
  int by_units;             // the work is dealt by units of positions across sequences (kv8_attn.h)
  int items;                // blocks per kv head that the plan aims at
  int tiles;                // host bound on the column tiles of all sequences
  int stream;               // pages are read once: non-temporal loads
  float* part;              // [rows][nq][n_split][hd + 2]: max, sum, unnormalised output
  int natural;              // part's maxima in natural units (else log2)
  int32_t* row_ns;          // [rows][nq] splits of each output (written by the attention, read by the merge)
  void* out;                // row r at + r * ldo: [nq][hd]
  long ldo;
  uint16_t *o_hi, *o_lo;    // or bf16 pairs [rows][nq hd] (kv8_prompt.hip, one split; nullable)
  uint32_t* err;
};
// The kernel of a pass of at most max_rows rows a sequence whose contexts are `positions` in all, and
// the query vectors of one of its tiles.
enum { kKv8Narrow = 0, kKv8Shared = 1, kKv8Both = 2, kKv8Prompt = 3 };
int kv8_attention_form(int x_bf16, int group, int max_rows, long positions, int nkv);
// (kv8_prompt.hip: four wavefronts of 32 bf16 vectors, or of 16 fp32 ones, which take two products each)
constexpr int kKv8PromptWaves = 4;
inline int kv8_form_cols(int form, int x_bf16) {
  return form == kKv8Narrow ? 16 : form != kKv8Prompt ? 32 : kKv8PromptWaves * (x_bf16 ? 32 : 16);
}
void launch_kv8_prompt(const Kv8AttnArgs& a, dim3 grid, hipStream_t st);
void launch_kv8_attention(const Kv8AttnArgs& a, hipStream_t st);
// out = the splits' joined outputs (a.n_split > 1)
void launch_kv8_join(const Kv8AttnArgs& a, hipStream_t st);


// -- shared by the kernels -----------------------------------------------------------------

// Rows and first position of sequence b (positions are bounded so that sums of them stay ints).
struct Kv8Seq {
  int beg, end;             // rows
  int first;                // position of the first row (pos: of the row)
  int ctx;                  // positions that its last row sees
};
OSP_DEV Kv8Seq kv8_seq(const Kv8Rows& r, int b) {
  const int total = r.count ? min(*r.count, r.rows) : r.rows;
  Kv8Seq s;
  s.beg = r.cu ? r.cu[b] : b;
  s.end = r.cu ? r.cu[b + 1] : r.B == 1 ? total : b + 1;
  s.beg = min(max(s.beg, 0), total);
  s.end = min(max(s.end, s.beg), total);
  if (r.cached) {
    s.first = min(max(r.cached[b], 0), kKv8MaxPos);
    s.ctx = s.end > s.beg ? s.first + (s.end - s.beg) : 0;
  } else {
    s.first = s.end > s.beg ? min(max(r.pos[s.beg], 0), kKv8MaxPos) : 0;
    s.ctx = s.end > s.beg ? min(max(r.pos[s.end - 1], 0), kKv8MaxPos) + 1 : 0;
  }
  return s;
}

// Physical page `page` of sequence b, or -1 where it has none.
OSP_DEV int kv8_page(const Kv8Pool& p, int b, int page) {
  const int row = p.slot ? p.slot[b] : b;
  const int n = p.nblocks ? min(p.nblocks[row], p.max_pages) : p.max_pages;
  if (page < 0 || page >= n) return -1;
  const int id = p.table[(long)row * p.max_pages + page];
  return id >= 0 && id < p.num_pages ? id : -1;
}

OSP_DEV float kv8_pow2(int e) { return __int_as_float((e + 127) << 23); }   // -126 <= e <= 127

}  // namespace osp
