// Attention over the cache.
//
// o_i = sum_j p_ij v_j with p = softmax over the positions j that row i sees, in one pass over the cache with a running
// maximum: nothing of size rows x positions is written.  A code of either format is exact in fp16, so both products run
// on the fp16 matrix cores on the codes themselves and the page scales are applied outside:
//
//   t_ij = c_i ks_j <q'_i, kcode_j> + log2 vs_j   c_i = scale log2(e) 2^e_i, q'_i = q_i 2^-e_i in fp16
//   w_ij = 2^(t_ij - M_i + 15)                    M_i = the running maximum of t_ij
//   o_i  = (sum_j w_ij vcode_j) / l_i             l_i = sum_j w_ij / vs_j  (in units of 2^18, see kUnit)
//
// q'_i is the row times the power of two that brings its largest value to [2^13, 2^14): a 16-bit value stays exact down
// to 2^-27 of the row's largest.  Taking the maximum of the weight with its value scale keeps w in fp16's range for
// whatever scales the pages have; w is rounded to fp16 for the second product (at most 2^-11 relative, down to 2^-29 of the largest
// weight, below that steps of 2^-39 of it; where the maximum lags, in kv_prompt_kernel, 2^-22 and 2^-32), l and every sum are
// fp32.  The rounding leaves fp16 results 2.4e-4 to 2.9e-4 from the exact ones (root mean square, relative; their own rounding
// alone 2.1e-4), bf16 ones where they are; a second half of w would take half as many products again.  fp32 queries take two
// halves of q' and of w and twice the products.
//
// Layout.  One wave takes 64 positions and 16 rows at a time, without LDS.  The scores are computed transposed (keys are
// the matrix instruction's rows, queries its columns), and the keys of the four 16-key products are chosen so that lane
// group g = lane / 16 ends with the scores of positions 16 g .. 16 g + 15 of its query: exactly the operand of the second
// product, whose other operand is 16 contiguous bytes of one dim of the value page.  A page is 16 tokens or more, so
// a lane's 16 positions share one page and its scales.
//
// Measured (8 cache heads of 128, bf16): one sequence of 131071 tokens 45 us for 268 MB and 4 to join; 64 sequences of 1 to
// 16384 tokens 176 us for 1028 MB, 5.8 TB/s, where a read alone reaches 6.3.  A chunk of a wave is about 540 vector
// instructions, 320 of them the widening of int8 codes (five per four codes, e4m3 two), and 32 products.  16 rows of 128 dims take 208
// registers, two waves to a SIMD; 32 rows take all 256 and spill 8 to 14 (36 to 60 bytes of scratch).
//
// 4-bit codes have a scale for each token: the factor ks_j and the logarithm of vs_j are brought to the lane of a position by a
// broadcast within its sixteen, and widening takes nine instructions for eight codes.  A chunk's codes take half the registers, so
// four-wave workgroups run three waves to a SIMD: 64 sequences of 1 to 16384 tokens 128 us for 619 MB, 4.8 TB/s (two waves, workgroups of eight:
// 150 us), one of 131071 of 96 dims in pages of 16 30 us for 109 MB.
#pragma once

#include <type_traits>
#include <utility>

#include "kv.hpp"

namespace kmq {
namespace {

constexpr int kChunk = 64;    // positions per step of a wave
constexpr float kLog2e = 1.44269504088896340736f;
constexpr float kUp = 15.0f;  // weights are at most 2^15
// l is kept in units of 2^18.  kv_write gives scales from 2^-100 (a page of zeros) to 2^121, so a position of the
// largest weight, 2^8 to 2^15, adds 2^97 to 2^-131 to it: sums of 2^30 positions stay below 2^128.
constexpr float kUnit = 0x1p-18f;

struct AttendArgs {
  KvCache C;
  KvSeqs S;
  KvAttend A;
  int rtiles;   // row tiles per sequence and head
  int deal;     // tiles are dealt out (kv_attend_kernel)
  int splits;   // the most that a tile is split into; if dealt out, workgroups
  int per;      // chunks of a split or, at least, of a workgroup
  float *part;  // blocks of accumulators, then M and l: [tile][split], or if dealt out two for each workgroup
  uint32_t block0;  // the launch's first workgroup (kv_prompt_kernel; see kv_piece)
};

__device__ __forceinline__ f32x4 mfma16(f16x8 a, f16x8 b, f32x4 c) {
  return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0);
}

__device__ __forceinline__ float max_groups(float x) {  // over the four lanes of one query
  x = fmaxf(x, __shfl_xor(x, 16));
  return fmaxf(x, __shfl_xor(x, 32));
}
__device__ __forceinline__ float sum_groups(float x) {
  x += __shfl_xor(x, 16);
  return x + __shfl_xor(x, 32);
}

// What brings l and the accumulators from maximum M to Mn: h * h, and where that is below the least normal number l, multiplied
// twice, keeps its size.  A page of tiny values adds up to 2^100 times its weight to l.
__device__ __forceinline__ float half_step(float M, float Mn) { return __builtin_amdgcn_exp2f(0.5f * (M - Mn)); }

// A lane's largest weight in a chunk is 2^(t - M + up), without its page's scale 2^(z - M + up).  True: the weights are below
// what fp16 holds and run into the least normal number, but over their page's scale they may count in l (zero pages beside
// values of 2^48 and more), so what they add is taken from the scores alone, down to the least number there is.
__device__ __forceinline__ bool far_below(float t, float z, float M) { return t < M - 100.0f && z > M - 146.0f; }
__device__ __forceinline__ float far_add(float l, float x) { return fmaf(__builtin_amdgcn_exp2f(x + 24.0f), 0x1p-24f, l); }

// Sixteen codes, the first (k = 0) or last eight of them for an operand, and where code i of eight lies in it.
template <int FMT>
using Codes16 = std::conditional_t<FMT == KM_KV_I4, u32x2, u32x4>;
template <int FMT>
__device__ __forceinline__ f16x8 widen8(const Codes16<FMT> &w, int k, const KvNibbles &nib) {
  if constexpr (FMT == KM_KV_I4) return kv_widen4x8(w[k], nib);
  else return kv_widen8<FMT>(w[2 * k], w[2 * k + 1]);
}
template <int FMT>
__device__ __forceinline__ constexpr int place8(int i) { return FMT == KM_KV_I4 ? kv_place4(i) : i; }

// 4-bit codes: a score times its token's key scale, from the lane that holds it, in base 2 with the log of its value scale.  The
// key scale is at least 2^-30 and c is not 0, so -infinity stays -infinity.
template <int L>
__device__ __forceinline__ float token_score(float s, float c, float ks, float lv) {
  return fmaf(s * kv_row_bcast<L>(ks), c, kv_row_bcast<L>(lv));
}
// Calls f with 0 .. N - 1 as constants.
template <typename F, int... I>
__device__ __forceinline__ void each_of(F &&f, std::integer_sequence<int, I...>) {
  (f(std::integral_constant<int, I>{}), ...);
}
template <int N, typename F>
__device__ __forceinline__ void each(F &&f) {
  each_of(f, std::make_integer_sequence<int, N>{});
}

// Floats of one (tile, split) block of partial results: NT x 4 accumulators of 64 lanes per 16 rows, then M and l of
// the 16 rows.
__host__ __device__ constexpr int part_floats(int nt) { return nt * 256 + 32; }

// 16 values of a row as fp32: N = 2 * NS groups of 16 bytes, fp32 ones (NS = 2) or of the type.
template <int NS>
__device__ __forceinline__ void values16(const u32x4 *raw, int type, float *x) {
  if constexpr (NS == 2) {
#pragma unroll
    for (int i = 0; i < 16; ++i) x[i] = __uint_as_float(raw[i / 4][i % 4]);
  } else if (type == KM_T_BF16) {
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      const uint32_t w = raw[i / 8][i / 2 % 4];
      x[i] = __uint_as_float(i % 2 ? w & 0xffff0000u : w << 16);
    }
  } else {
#pragma unroll
    for (int i = 0; i < 16; ++i) {
      const uint32_t w = raw[i / 8][i / 2 % 4];
      x[i] = (float)__builtin_bit_cast(f16x2, w)[i % 2];
    }
  }
}
template <int NS>
__device__ __forceinline__ float top16(const u32x4 *raw, int type) {
  float v[16], top = 0.0f;
  values16<NS>(raw, type, v);
#pragma unroll
  for (int i = 0; i < 16; ++i) top = fmaxf(top, fabsf(v[i]));
  return top;
}

__device__ __forceinline__ void store_o4(const KvAttend &A, int64_t o, const float *x) {
  if (A.type == KM_T_F32) kv_store<KM_T_F32, 4>(A.out.p, o, x);
  else if (A.type == KM_T_BF16) kv_store<KM_T_BF16, 4>(A.out.p, o, x);
  else kv_store<KM_T_F16, 4>(A.out.p, o, x);
}

// The power of two that takes a row whose largest magnitude is top to [2^13, 2^14), and what the products of the scaled
// row are multiplied by.  Exponents stay where the inverse is a normal number too.  A row with an infinity has no finite score,
// and a softmax over those is NaN; its products could all be -infinity, which counts as not seen, so it becomes NaN here.
__device__ __forceinline__ void q_scale(float top, float scale, float *f, float *c) {
  const int up = min(max(140 - (int)(__float_as_uint(top) >> 23), -126), 126);
  *f = top == INFINITY ? NAN : __uint_as_float((uint32_t)(127 + up) << 23);
  *c = scale * kLog2e * __uint_as_float((uint32_t)(127 - up) << 23);
}

// The log of a row's sum of exp, its weights up to 2^up, and what its accumulators are multiplied by, one after the other.
// l = 0: the row saw no position.
struct RowSum {
  float lse, a, b;
};
__device__ __forceinline__ RowSum row_sum(float M, float l, float up) {
  const bool low = l < 0x1p-100f;  // its inverse and the logarithm want a normal number
  const float z = low ? l * 0x1p24f : l;
  RowSum s;
  s.lse = l > 0.0f ? (M - up + (low ? -6.0f : 18.0f) + __builtin_amdgcn_logf(z)) * 0.69314718055994530942f
                   : (l == 0.0f ? -INFINITY : NAN);
  s.a = low ? 0x1p24f * kUnit : kUnit;
  s.b = l == 0.0f ? 0.0f : 1.0f / z;
  return s;
}

// Row r of a sequence's rows of one cache head: token-major, so that a tile's positions lie close together.
struct RowAt {
  int64_t q, o;  // element offsets
  int64_t lse;
};
__device__ __forceinline__ RowAt row_at(const KvAttend &A, const KvCache &C, const KvSeq &q, int h, int r) {
  const int tok = r / A.group, hq = h * A.group + r % A.group;
  const int64_t row = q.row0 + tok;
  return {row * A.q.row + hq * A.q.head, row * A.out.row + hq * A.out.head, row * C.heads * A.group + hq};
}

// Positions [lo, hi) that row r sees.
__device__ __forceinline__ void row_span(const KvAttend &A, const KvSeq &q, int r, int *lo, int *hi) {
  const int pos = q.len - q.n + r / A.group;
  *hi = A.causal ? max(pos + 1, 0) : q.len;
  *lo = A.window ? max(pos + 1 - A.window, 0) : 0;
}

// Chunks [cb, ce) of a split of rows [r0, r1), and how many splits these rows have: as many as their positions need,
// P.per chunks each, one if they see none.  False: no such split.
__device__ __forceinline__ bool tile_span(const AttendArgs &P, const KvSeq &q, int r0, int r1, int split, int *cb, int *ce,
                                          int *splits) {
  int lo, hi, any;
  row_span(P.A, q, r0, &lo, &any);      // the first row's first position
  row_span(P.A, q, r1 - 1, &any, &hi);  // the last row's last
  const int c0 = lo / kChunk, n = hi > lo ? (hi + kChunk - 1) / kChunk - c0 : 0;
  *splits = min(max((n + P.per - 1) / P.per, 1), P.splits);
  const int per = (n + *splits - 1) / *splits;
  *cb = c0 + split * per;
  *ce = min(*cb + per, c0 + n);
  return split < *splits;
}

// Dealing out.  The chunks of all tiles of a call, one sequence after the other, are cut into equal runs, a run for each
// workgroup, so that every workgroup streams as many bytes as the others whatever the lengths are.  A tile counts kTileCost
// chunks more than it has, about what a workgroup loses at its beginning and end.
constexpr int kTileCost = 8;

// The chunks that a sequence's rows see, in all of its tiles alike: [c0, c0 + n).
struct SeqChunks {
  int c0, n, tiles;
  int cost;  // of all its tiles
};
__device__ __forceinline__ SeqChunks seq_chunks(const AttendArgs &P, int b, int trows, KvSeq *q) {
  SeqChunks s{0, 0, 0, 0};
  if (!kv_seq(P.S, P.C.page, b, q) || q->n == 0) return s;
  int lo, hi, any;
  const int rows = q->n * P.A.group;
  row_span(P.A, *q, 0, &lo, &any);
  row_span(P.A, *q, rows - 1, &any, &hi);
  s.c0 = lo / kChunk;
  s.n = max(hi > lo ? (hi + kChunk - 1) / kChunk - s.c0 : 0, 1);  // rows that see nothing take a chunk all the same
  s.tiles = P.C.heads * ((rows + trows - 1) / trows);
  s.cost = s.tiles * (s.n + kTileCost);
  return s;
}

// Every wave goes through the sequences by itself, one per lane (the host deals only calls whose cost fits).
struct DealScan {
  int all;           // cost up to and including these 64 sequences
  int before, cost;  // of this lane's sequence
};
__device__ __forceinline__ DealScan deal_scan(const AttendArgs &P, int trows, int b0, int all) {
  const int lane = threadIdx.x & 63;
  KvSeq q;
  const int w = b0 + lane < P.S.n ? seq_chunks(P, b0 + lane, trows, &q).cost : 0;
  int sum = w;  // of the lanes up to this one
#pragma unroll
  for (int o = 1; o < 64; o *= 2) {
    const int y = __shfl_up(sum, o);
    if (lane >= o) sum += y;
  }
  return {all + __builtin_amdgcn_readlane(sum, 63), all + sum - w, w};
}
// the cost of the call; the scan of its last 64 sequences
__device__ __forceinline__ DealScan deal_all(const AttendArgs &P, int trows) {
  DealScan s{0, 0, 0};
  for (int b0 = 0; b0 < P.S.n; b0 += 64) s = deal_scan(P, trows, b0, s.all);
  return s;
}
// the cost of the sequences before b
__device__ __forceinline__ int deal_before(const AttendArgs &P, int trows, DealScan s, int b) {
  const int last = (P.S.n - 1) & ~63;
  if (b < last) {
    s.all = 0;
    for (int b0 = 0; b0 <= b; b0 += 64) s = deal_scan(P, trows, b0, s.all);
  }
  return __builtin_amdgcn_readlane(s.before, b & 63);
}
// the sequence that holds place `at`, and the cost of those before it
__device__ __forceinline__ int deal_find(const AttendArgs &P, int trows, DealScan s, int at, int *before) {
  int b0 = (P.S.n - 1) & ~63;
  uint64_t hit = __ballot(at >= s.before && at < s.before + s.cost);
  if (!hit) {
    s.all = 0;
    for (b0 = -64; !hit && b0 + 64 < P.S.n;) {
      b0 += 64;
      s = deal_scan(P, trows, b0, s.all);
      hit = __ballot(at >= s.before && at < s.before + s.cost);
    }
  }
  const int y = __ffsll((long long)hit) - 1;
  *before = __builtin_amdgcn_readlane(s.before, y);
  return b0 + y;
}
// the cost that a workgroup takes
__device__ __forceinline__ int deal_run(const AttendArgs &P, int all) {
  return max((int)(((uint32_t)all + P.splits - 1) / (uint32_t)P.splits), P.per);
}

constexpr int kAttendWaves = 4, kWideWaves = 8;  // of a workgroup (see plan)

// LDS of a workgroup: maxima and sums of each wave's rows, then each wave's accumulators.
template <int RT, int NT>
struct AttendWave {
  float m[RT][16], l[RT][16];
  f32x4 o[RT * NT][64];
};

// Chunks [cb, ce) of rows [r0, ...) of a sequence's head; the results, or where part is given the sums for the join.
template <int FMT, int NT, int RT, int NS, bool ONE, int W>
__device__ __forceinline__ void attend_tile(const AttendArgs &P, const KvSeq &q, int b, int h, int r0, int cb, int ce,
                                            float *part, AttendWave<RT, NT> *sh) {
  constexpr int NP = (NT + 3) / 4;  // groups of 64 dims
  const KvCache &C = P.C;
  const KvAttend &A = P.A;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), m = lane & 15, g = lane >> 4;
  const int d = C.d, rows = q.n * A.group;
  const KvNibbles nib = kv_nibbles();

  // Codes of a chunk.  Its page (ONE), or the pages of this lane's runs of 16: keys of run kr, values of run g.  Behind the
  // end and where a page is not there something of the cache is read that counts for nothing.
  const int64_t hb = kv_bytes<FMT>((int64_t)C.page * d);  // bytes of a page's head
  const int db = (int)kv_bytes<FMT>(d);                   // of a key
  const int pmask = C.page - 1, last = max(q.len - 1, 0);
  const int *table = P.S.table + (int64_t)b * P.S.table_ld;
  const int kr = m >> 2, ktok = m & 3;
  // This lane's 16 dims of group p, whose products another lane has already where they are past d.  4-bit codes: groups of 128
  // dims, 32 to a lane, as long as there are two groups of 64.
  auto own_dims = [&](int p) { return FMT == KM_KV_I4 && (p | 1) < NP ? 64 * (p & ~1) + 32 * g + 16 * (p & 1) : 64 * p + 16 * g; };
  auto dims_at = [&](int p) {
    return FMT == KM_KV_I4 && (p | 1) < NP ? min(64 * (p & ~1) + 32 * g, d - 32) + 16 * (p & 1) : min(64 * p + 16 * g, d - 16);
  };
  auto page_of = [&](int j) {
    const int pg = table[min(j, last) >> C.shift];
    return ONE ? __builtin_amdgcn_readfirstlane(pg) : pg;
  };
  auto page_at = [&](int pg) { return (int64_t)(pg >= 0 && pg < C.pages ? pg : 0) * C.heads + h; };
  int pk, pv;
  auto pages = [&](int c) {
    pv = page_of(c * kChunk + (ONE ? 0 : 16 * g));
    pk = ONE ? pv : page_of(c * kChunk + 16 * kr);
  };
  Codes16<FMT> kw[4][NP], vw[NT];
  float ks, vs;  // 4-bit codes: of position m of run g
  bool there;
  auto load_keys = [&](int c) {
    const int tk = c * kChunk + (ONE ? 0 : 16 * kr);
    const uint8_t *kp = C.k + page_at(pk) * hb + (tk & pmask) * db;
#pragma unroll
    for (int st = 0; st < 4; ++st)
#pragma unroll
      for (int p = 0; p < NP; ++p) {
        const uint8_t *at = kp + 4 * st * db + (uint32_t)(((ONE ? 16 * kr : 0) + ktok) * db + (int)kv_bytes<FMT>(dims_at(p)));
        if (FMT == KM_KV_I4 && (p | 1) < NP) {
          if (p & 1) continue;
          const u32x4 w = *reinterpret_cast<const u32x4 *>(at);
#pragma unroll
          for (int i = 0; i < 4; ++i) kw[st][p | (i / 2)][i % 2] = w[i];
        } else {
          kw[st][p] = *reinterpret_cast<const Codes16<FMT> *>(at);
        }
      }
  };
  auto load_values = [&](int c) {
    const int tv = c * kChunk + (ONE ? 0 : 16 * g);
    const int64_t at = page_at(pv);
    there = c * kChunk + 16 * g < q.len && pv >= 0 && pv < C.pages;
    const uint8_t *vp = C.v + at * hb + kv_bytes<FMT>(tv & pmask);
#pragma unroll
    for (int n = 0; n < NT; ++n)
      vw[n] = *reinterpret_cast<const Codes16<FMT> *>(vp + (int)kv_bytes<FMT>(min(16 * n, d - 16) * C.page) +
                                                      (uint32_t)kv_bytes<FMT>(m * C.page + (ONE ? 16 * g : 0)));
    if constexpr (FMT == KM_KV_I4) {
      const int64_t tok = at * C.page + (tv & pmask) + (ONE ? 16 * g : 0) + m;
      const bool in = there && c * kChunk + 16 * g + m < q.len;
      ks = in ? C.ks[tok] : 1.0f;
      vs = in ? C.vs[tok] : 1.0f;
    } else {
      ks = C.ks[at];
      vs = C.vs[at];
    }
  };
  int c = cb + wave;
  if (c < ce) {
    pages(c);
    load_keys(c);
    load_values(c);
    if (c + W < ce) pages(c + W);
  }

  // the rows of this lane (rows past the last repeat it and are not stored), their scale and their spans; dims past d are 0
  f16x8 qf[RT][NP][2][NS];
  float cs[RT];
  int lo[RT], hi[RT];
  u32x4 raw[RT][NP][2 * NS];  // 16 values each
#pragma unroll
  for (int u = 0; u < RT; ++u) {
    const int r = min(r0 + 16 * u + m, rows - 1);
    row_span(A, q, r, &lo[u], &hi[u]);
    const char *at = static_cast<const char *>(A.q.p) + row_at(A, C, q, h, r).q * (2 * NS);
#pragma unroll
    for (int p = 0; p < NP; ++p)
#pragma unroll
      for (int i = 0; i < 2 * NS; ++i)
        raw[u][p][i] = reinterpret_cast<const u32x4 *>(at + dims_at(p) * (2 * NS))[i];
  }
#pragma unroll
  for (int u = 0; u < RT; ++u) {
    float top = 0.0f;
#pragma unroll
    for (int p = 0; p < NP; ++p) top = fmaxf(top, top16<NS>(raw[u][p], A.type));
    float f;
    q_scale(max_groups(top), A.scale, &f, &cs[u]);
#pragma unroll
    for (int p = 0; p < NP; ++p) {
      const float fp = own_dims(p) < d ? f : 0.0f;
      float v[16];
      values16<NS>(raw[u][p], A.type, v);
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        const float y = fp == 0.0f ? 0.0f : v[i] * fp;
        const _Float16 y16 = (_Float16)y;
        qf[u][p][i / 8][0][place8<FMT>(i % 8)] = y16;
        if constexpr (NS == 2) qf[u][p][i / 8][1][place8<FMT>(i % 8)] = (_Float16)(y - (float)y16);
      }
    }
  }

  f32x4 acc[RT][NT];
  float M[RT], l[RT];
#pragma unroll
  for (int u = 0; u < RT; ++u) {
    M[u] = -INFINITY;
    l[u] = 0.0f;
#pragma unroll
    for (int n = 0; n < NT; ++n) acc[u][n] = f32x4{0, 0, 0, 0};
  }

  // The registers of a chunk's keys are loaded again as soon as its scores are done, those of its values after the second
  // product: each load has half a step to arrive.
  for (; c < ce; c += W) {
    const int j0 = c * kChunk;
    const bool more = c + W < ce;
    f32x4 s[RT][4];
#pragma unroll
    for (int st = 0; st < 4; ++st) {
      __builtin_amdgcn_sched_barrier(0);  // no more codes widened at a time than these products take
#pragma unroll
      for (int u = 0; u < RT; ++u) s[u][st] = f32x4{0, 0, 0, 0};
#pragma unroll
      for (int p = 0; p < NP; ++p)
#pragma unroll
        for (int k = 0; k < 2; ++k) {
          const f16x8 kf = widen8<FMT>(kw[st][p], k, nib);
#pragma unroll
          for (int u = 0; u < RT; ++u)
#pragma unroll
            for (int z = 0; z < NS; ++z) s[u][st] = mfma16(kf, qf[u][p][k][z], s[u][st]);
        }
    }
    if (more) load_keys(c + W);

    const float k1 = there ? ks : 1.0f, v1 = there ? vs : 1.0f;
    const float lv = __builtin_amdgcn_logf(v1), inv = 1.0f / v1;  // 4-bit codes: of position m of run g, as k1
    f16x8 w[RT][2][NS];
#pragma unroll
    for (int u = 0; u < RT; ++u) {
      if (!__all(there && j0 >= lo[u] && j0 + kChunk <= hi[u])) {
        int jg = j0 + 16 * g;
        asm volatile("" : "+v"(jg));  // a branch: few chunks need it, so nothing of it is kept in registers
#pragma unroll
        for (int st = 0; st < 4; ++st)
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const int j = jg + 4 * st + i;
            if (!there || j < lo[u] || j >= hi[u]) s[u][st][i] = -INFINITY;
          }
      }
      // a factor of 0 (a row of tiny queries) would make NaN of -inf
      const float ck = fmaxf(FMT == KM_KV_I4 ? cs[u] : cs[u] * k1, 0x1p-126f);
      if constexpr (FMT == KM_KV_I4)
        each<16>([&](auto e) {
          constexpr int i = e;
          s[u][i / 4][i % 4] = token_score<i>(s[u][i / 4][i % 4], ck, k1, lv);
        });
      float top = -INFINITY;
#pragma unroll
      for (int st = 0; st < 4; ++st)
#pragma unroll
        for (int i = 0; i < 4; ++i) top = fmaxf(top, s[u][st][i]);
      const float tl = FMT == KM_KV_I4 ? top : fmaf(top, ck, lv), Mn = fmaxf(M[u], max_groups(tl));
      // scales of 4-bit codes are too close to each other for that
      auto below = [&](float M) { return FMT != KM_KV_I4 && far_below(tl, tl - lv, M); };
      float iu = inv;
      if (__any(Mn > M[u] || below(M[u]))) {  // one branch for both: neither is common
        const float al = Mn == -INFINITY ? 1.0f : half_step(M[u], Mn);
        l[u] = l[u] * al * al;
#pragma unroll
        for (int n = 0; n < NT; ++n) acc[u][n] *= al * al;
        M[u] = Mn;
        if (below(Mn)) {
          iu = 0.0f;
#pragma unroll
          for (int st = 0; st < 4; ++st)
#pragma unroll
            for (int i = 0; i < 4; ++i) l[u] = far_add(l[u], fmaf(s[u][st][i], ck, kUp - 18.0f - Mn));
        }
      }
      const float up = kUp - (Mn == -INFINITY ? 0.0f : Mn);
      const float base = lv - (Mn == -INFINITY ? 0.0f : Mn) + kUp;
      float sum = 0.0f;
      if constexpr (FMT == KM_KV_I4) {
        each<16>([&](auto e) {
          constexpr int st = e / 4, i = e % 4, at = kv_place4(4 * (st % 2) + i);
          const float y = __builtin_amdgcn_exp2f(s[u][st][i] + up);
          sum = fmaf(kv_row_bcast<e>(inv), y, sum);
          const _Float16 y16 = (_Float16)y;
          w[u][st / 2][0][at] = y16;
          if constexpr (NS == 2) w[u][st / 2][1][at] = (_Float16)(y - (float)y16);
        });
        l[u] = fmaf(sum, kUnit, l[u]);
      } else {
#pragma unroll
        for (int st = 0; st < 4; ++st)
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const float y = __builtin_amdgcn_exp2f(fmaf(s[u][st][i], ck, base));
            sum += y;
            const _Float16 y16 = (_Float16)y;
            w[u][st / 2][0][4 * (st % 2) + i] = y16;
            if constexpr (NS == 2) w[u][st / 2][1][4 * (st % 2) + i] = (_Float16)(y - (float)y16);
          }
        l[u] = fmaf(sum * kUnit, iu, l[u]);  // not inv * kUnit: 1 / vs may be near the least normal number
      }
    }
    if constexpr (FMT == KM_KV_F8) {  // codes past the end may be NaN, which no weight of 0 takes out
      if (!__all(there && j0 + kChunk <= q.len)) {
        int left = there ? q.len - j0 - 16 * g : 0;
        asm volatile("" : "+v"(left));
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
          for (int y = 0; y < 4; ++y) {
            const int k = left - 4 * y;
            vw[n][y] &= k >= 4 ? 0xffffffffu : k <= 0 ? 0u : (1u << (8 * k)) - 1u;
          }
      }
    }
#pragma unroll
    for (int n = 0; n < NT; ++n) {
      if (n % 2 == 0) __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        const f16x8 vf = widen8<FMT>(vw[n], k, nib);
#pragma unroll
        for (int u = 0; u < RT; ++u)
#pragma unroll
          for (int z = 0; z < NS; ++z) acc[u][n] = mfma16(vf, w[u][k][z], acc[u][n]);
      }
    }
    if (more) {
      load_values(c + W);
      if (c + 2 * W < ce) pages(c + 2 * W);
    }
  }

  // the waves' results: scaled to a common maximum, then each wave adds up its share of the accumulators, in the waves' order
#pragma unroll
  for (int u = 0; u < RT; ++u) {
    l[u] = sum_groups(l[u]);
    if (l[u] != l[u]) M[u] = INFINITY;  // the maximum does not see NaN: the row's results are NaN from here
    if (g == 0) {
      sh[wave].m[u][m] = M[u];
      sh[wave].l[u][m] = l[u];
    }
  }
  __syncthreads();
#pragma unroll
  for (int u = 0; u < RT; ++u) {
    float Mx = -INFINITY, sum = 0.0f;
#pragma unroll
    for (int y = 0; y < W; ++y) Mx = fmaxf(Mx, sh[y].m[u][m]);
#pragma unroll
    for (int y = 0; y < W; ++y) {
      const float My = sh[y].m[u][m];  // -inf: the wave has nothing
      const float al = My == -INFINITY ? 0.0f : half_step(My, Mx);
      sum += sh[y].l[u][m] * al * al;
    }
    const float al = M[u] == -INFINITY ? 0.0f : half_step(M[u], Mx);
#pragma unroll
    for (int n = 0; n < NT; ++n) sh[wave].o[u * NT + n][lane] = acc[u][n] * (al * al);
    M[u] = Mx;
    l[u] = sum;
  }
  __syncthreads();
#pragma unroll
  for (int u = 0; u < RT; ++u) {
    const int r = r0 + 16 * u + m;
    if (r >= rows) continue;
    const RowAt at = row_at(A, C, q, h, r);
    const RowSum end = row_sum(M[u], l[u], kUp);
    float *o = part + u * part_floats(NT);
    for (int n = wave; n < NT; n += W) {
      f32x4 v = sh[0].o[u * NT + n][lane];
#pragma unroll
      for (int y = 1; y < W; ++y) v += sh[y].o[u * NT + n][lane];
      if (part) {
        *reinterpret_cast<f32x4 *>(o + (n * 64 + lane) * 4) = v;
      } else {
        const int i0 = 16 * n + 4 * g;
        v = v * end.a * end.b;
        const float y[4] = {v.x, v.y, v.z, v.w};
        if (i0 < d) store_o4(A, at.o + i0, y);
      }
    }
    if (wave == 0 && g == 0) {
      if (part) {
        o[NT * 256 + m] = M[u];
        o[NT * 256 + 16 + m] = l[u];
      } else if (A.lse) {
        A.lse[at.lse] = end.lse;
      }
    }
  }
}

// Waves to a SIMD that the registers have to leave room for.
template <int FMT, int NT, int RT, int NS, int W>
constexpr int attend_waves() {
  return NT > 8 ? 1 : FMT == KM_KV_I4 && RT == 1 && NS == 1 && W == kAttendWaves ? 3 : 2;
}

template <int FMT, int NT, int RT, int NS, bool ONE, int W>
__global__ __launch_bounds__(64 * W, (attend_waves<FMT, NT, RT, NS, W>())) void kv_attend_kernel(AttendArgs P) {
  __shared__ AttendWave<RT, NT> sh[W];
  constexpr int TR = 16 * RT;
  KvSeq q;
  if (!P.deal) {  // a workgroup per tile and split
    const uint32_t splits = max(P.splits, 1);
    uint32_t x = blockIdx.x / splits;
    const int split = (int)(blockIdx.x - x * splits);
    float *part = P.part + (int64_t)blockIdx.x * RT * part_floats(NT);
    const int rt = (int)(x % (uint32_t)P.rtiles);
    x /= (uint32_t)P.rtiles;
    const int h = (int)(x % (uint32_t)P.C.heads), b = (int)(x / (uint32_t)P.C.heads);
    if (!kv_seq(P.S, P.C.page, b, &q)) return;
    const int r0 = rt * TR, rows = q.n * P.A.group;
    int cb, ce, of;
    if (r0 < rows && tile_span(P, q, r0, min(r0 + TR, rows), split, &cb, &ce, &of))
      attend_tile<FMT, NT, RT, NS, ONE, W>(P, q, b, h, r0, cb, ce, of > 1 ? part : nullptr, sh);
    return;
  }
  const DealScan o = deal_all(P, TR);
  const int run = deal_run(P, o.all);
  if ((int64_t)run * blockIdx.x >= o.all) return;
  int at = run * (int)blockIdx.x, left = min(run, o.all - at), before;  // the place, and what is left to take
  int b = deal_find(P, TR, o, at, &before);
  at -= before;
  for (; left > 0; ++b) {
    const SeqChunks s = seq_chunks(P, b, TR, &q);
    const int cost = s.n + kTileCost, rtiles = s.tiles / P.C.heads;
    int tile = s.n ? (int)((uint32_t)at / (uint32_t)cost) : 0, skip = at - tile * cost;
    at = 0;
    for (; tile < s.tiles && left > 0; ++tile) {
      const int take = min(left, cost - skip);
      const int c0 = max(skip - kTileCost, 0), c1 = skip + take - kTileCost;
      if (c1 > c0) {
        // a tile that began in another workgroup, or one that is not finished here
        float *part = c1 - c0 == s.n ? nullptr
                                     : P.part + ((int64_t)blockIdx.x * 2 + (c0 == 0)) * RT * part_floats(NT);
        attend_tile<FMT, NT, RT, NS, ONE, W>(P, q, b, tile / rtiles, tile % rtiles * TR, s.c0 + c0, s.c0 + c1, part, sh);
      }
      left -= take;
      skip = 0;
    }
  }
}

// Joins the splits of R = 64 / G rows (G = 4: tiles of kv_attend_kernel, G = 2: of kv_prompt_kernel, whose accumulators lie
// the same way).  DEAL: the blocks are those of the workgroups that the tile was dealt to.  spread: a workgroup per
// accumulator of a lane, whose waves take the splits in turn and are added up in their order (few tiles, many splits);
// otherwise one for all of them, whose waves take the accumulators in turn.
constexpr int kJoinWaves = 8;

struct JoinSum {
  float M, l;
  f32x4 o;
};
// o += oy, l += ly of a partial result with maximum My
__device__ __forceinline__ void join_add(JoinSum &s, const float *My, const float *ly, const f32x4 *oy) {
  float M = s.M;
#pragma unroll
  for (int i = 0; i < 4; ++i) M = fmaxf(M, My[i]);
  const float Mu = M == -INFINITY ? 0.0f : M, a0 = half_step(s.M, Mu);
  s.l = s.l * a0 * a0;
  s.o *= a0 * a0;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const float al = My[i] == -INFINITY ? 0.0f : half_step(My[i], Mu);
    s.l = fmaf(ly[i] * al, al, s.l);
    s.o += oy[i] * (al * al);
  }
  s.M = M;
}

template <int NA, int G, bool DEAL>
__global__ __launch_bounds__(64 * kJoinWaves) void kv_join_kernel(AttendArgs P, int ru, int spread, float up) {
  constexpr int W = kJoinWaves, R = 64 / G, F = NA * 256 + 2 * R;  // rows, floats of a block
  __shared__ float sh[W][R], sl[W][R];
  __shared__ f32x4 so[W][64];
  const KvCache &C = P.C;
  const KvAttend &A = P.A;
  const uint32_t block = spread ? blockIdx.x / NA : blockIdx.x;
  uint32_t x = block / (uint32_t)ru;
  const int u = (int)(block - x * ru);
  const int64_t tile = x;
  const int rt = (int)(x % (uint32_t)P.rtiles);
  x /= (uint32_t)P.rtiles;
  const int h = (int)(x % (uint32_t)C.heads);
  const int b = (int)(x / (uint32_t)C.heads);
  KvSeq q;
  if (!kv_seq(P.S, C.page, b, &q)) return;
  const int rows = q.n * A.group, t0 = rt * ru * R, r0 = t0 + u * R;
  if (r0 >= rows) return;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), m = lane % R, g = lane / R;
  int splits;
  int64_t first, step;  // block of split 0, blocks from one split to the next
  int64_t lead = 0;     // split 0 lies this many blocks further
  if constexpr (DEAL) {
    const DealScan o = deal_all(P, ru * R);
    const uint32_t run = (uint32_t)deal_run(P, o.all);
    KvSeq z;
    const SeqChunks s = seq_chunks(P, b, ru * R, &z);
    const uint32_t t = deal_before(P, ru * R, o, b) + (s.n + kTileCost) * (h * (s.tiles / C.heads) + rt) + kTileCost;
    const uint32_t w0 = t / run, w1 = (t + s.n - 1) / run;
    splits = (int)(w1 - w0 + 1);
    first = (int64_t)w0 * 2 * ru + u;
    step = 2 * ru;
    lead = ru;
  } else {
    int cb, ce;
    tile_span(P, q, t0, min(t0 + ru * R, rows), 0, &cb, &ce, &splits);
    first = tile * P.splits * ru + u;
    step = ru;
  }
  if (splits == 1) return;  // already finished
  const int r = r0 + m;
  auto sums = [&](int n, int y0, int dy) {  // of splits y0, y0 + dy, ...
    JoinSum s{-INFINITY, 0.0f, {0, 0, 0, 0}};
    if (r >= rows) return s;
    for (; y0 < splits; y0 += 4 * dy) {
      float My[4], ly[4];
      f32x4 oy[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) {  // past the last split: the last one again, which does not count
        const int y = min(y0 + i * dy, splits - 1);
        const float *p = P.part + (first + y * step + (y == 0 ? lead : 0)) * F;
        My[i] = y0 + i * dy < splits ? p[NA * 256 + m] : -INFINITY;
        ly[i] = p[NA * 256 + R + m];
        oy[i] = *reinterpret_cast<const f32x4 *>(p + (n * 64 + lane) * 4);
      }
      join_add(s, My, ly, oy);
    }
    return s;
  };
  auto finish = [&](int n, const JoinSum &s) {
    if (r >= rows) return;
    const RowAt at = row_at(A, C, q, h, r);
    const RowSum end = row_sum(s.M, s.l, up);
    const f32x4 o = s.o * end.a * end.b;
    const float y[4] = {o.x, o.y, o.z, o.w};
    const int c = G == 4 ? 16 * n + 4 * g : 32 * (n / 4) + 8 * (n % 4) + 4 * g;
    if (c < C.d) store_o4(A, at.o + c, y);
    if (A.lse && n == 0 && g == 0) A.lse[at.lse] = end.lse;
  };
  if (!spread) {
    for (int n = wave; n < NA; n += W) finish(n, sums(n, 0, 1));
    return;
  }
  const int n = (int)(blockIdx.x - block * NA);
  JoinSum s = sums(n, wave, W);
  so[wave][lane] = s.o;
  if (g == 0) {
    sh[wave][m] = s.M;
    sl[wave][m] = s.l;
  }
  __syncthreads();
  if (wave) return;
#pragma unroll
  for (int y0 = 1; y0 < W; y0 += 4) {
    float My[4], ly[4];
    f32x4 oy[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int y = min(y0 + i, W - 1);
      My[i] = y0 + i < W ? sh[y][m] : -INFINITY;
      ly[i] = sl[y][m];
      oy[i] = so[y][lane];
    }
    join_add(s, My, ly, oy);
  }
  finish(n, s);
}

// ---- many rows: tiles of 64 positions shared by a workgroup through LDS ------------------------------------------------
//
// A wave takes 32 rows and the 32 x 32 x 16 products; the four waves of a workgroup share each tile of 64 positions, whose
// codes are widened to fp16 once and laid out in LDS.  As above the scores are computed transposed, with the keys'
// order chosen such that a lane ends with 8 consecutive positions of its row in consecutive registers: row m of a 32-key
// operand holds position m with bits 2 and 3 exchanged.  The running maximum moves only when a tile's exceeds it by
// more than kSlack: until then weights just grow, within fp16's range.
//
// The matrix cores and the vector unit (exponentials, widening) have about as much to do, so they overlap inside a wave too: the
// products of the next tile's scores are issued between this tile's exponentials, and the widening of later tiles between
// the second products.  Keys therefore run one tile ahead of values in LDS (two buffers each, one barrier per tile), and codes
// are loaded one tile before they are widened.
//
// Measured (prompt of 16384, 32 query heads of 128 on 8): 2.3 ms, 950 TFLOP/s, where a large fp16 library product reaches
// 1310 on this card (both run into its power limit, about 1.9 GHz).  The matrix cores are busy for 43 % of the time, the
// vector unit for 60 %, LDS for 40 %.  Two waves to a SIMD.  Tried: 64 rows to a wave, one wave to a SIMD (halves the LDS
// reads, 3.3 ms); eight waves to a workgroup (halves the widening, no change).  Heads of more than 128 dims leave a SIMD
// one wave only, and its phases in turn: 390 TFLOP/s at 256 (pages below 64 also spill up to 10 registers there).

// Weights begin at 2^kUp32 and may grow by kSlack.  Those below fp16's normal range are rounded to whole multiples of 2^-24, so to within 2^-33 of
// their row's largest, each times its value's scale (with kUp: 2^-40): all that a dim has where the row's heavy tokens have code 0 in it.
constexpr float kUp32 = 8.0f, kSlack = 7.0f;

typedef float f32x16v __attribute__((ext_vector_type(16)));

__device__ __forceinline__ f32x16v mfma32(f16x8 a, f16x8 b, f32x16v c) {
  return __builtin_amdgcn_mfma_f32_32x32x16_f16(a, b, c, 0, 0, 0);
}

// the larger of this lane's x and that of the lane 32 away
__device__ __forceinline__ float max_halves(float x) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}

// The order in which the sequences' row tiles are taken (up to 64 sequences, others side by side).
struct Order {
  bool ragged;  // lengths differ by more than an eighth: one sequence after the other, the longest first
  int b;        // then the k-th longest, else k
};
__device__ __forceinline__ Order order_of(const KvSeqs &S, int k) {
  if (S.n == 1 || S.n > 64) return {false, 0};
  const int lane = threadIdx.x & 63, len = lane < S.n ? S.lens[lane] : -1;
  int rank = 0, lo = INT32_MAX, hi = 0;
  for (int i = 0; i < S.n; ++i) {
    const int y = __builtin_amdgcn_readlane(len, i);
    rank += y > len || (y == len && i < lane);
    lo = min(lo, y);
    hi = max(hi, y);
  }
  if (lo >= hi - hi / 8) return {false, 0};
  return {true, __ffsll((long long)__ballot(lane < S.n && rank == k)) - 1};
}

// Floats of one (32 rows, split) block of partial results.
__host__ __device__ constexpr int part32_floats(int nd) { return nd * 1024 + 64; }

constexpr int kWaves = 4;  // of this kernel

template <int FMT, int ND, bool ONE>
__global__ __launch_bounds__(64 * kWaves, ND <= 4 ? 2 : 1) void kv_prompt_kernel(AttendArgs P) {
  constexpr int DP = 32 * ND, T = 64 * kWaves;
  constexpr int KLD = DP + 8, VLD = kChunk + 8;  // halves; 16 bytes more than the row: rows start in different banks
  constexpr bool I4 = FMT == KM_KV_I4;
  constexpr int PC = DP / (I4 ? 32 : 16);        // 16-byte pieces of a key
  constexpr int KN = kChunk * PC, VN = DP * 4;   // pieces of a tile
  constexpr int KP = (KN + T - 1) / T, VP = (VN + T - 1) / T;
  __shared__ __align__(16) _Float16 kt[2][kChunk * KLD], vt[2][DP * VLD];
  constexpr int NR = ONE ? 1 : 4;  // pages that a tile may lie in: its one, or one for each run of 16 positions
  // of these: key scale, log2 of the value scale and its inverse, 1 if the page is there
  __shared__ float4 sc[2][4];
  __shared__ float tsc[2][3][I4 ? kChunk : 1];  // 4-bit codes: the first three of every position
  const KvCache &C = P.C;
  const KvAttend &A = P.A;
  // Heads fastest: a head's workgroups share an XCD's L2 where their number is a multiple of 8.  Row tiles from the last on,
  // which see the most positions, the sequences' side by side where these are about as long, else one sequence after the
  // other (four pieces of prompts of 256 dims: of equal lengths 480 us, one after the other 525; ending at 2.1 to 4.8
  // thousand positions 660 side by side, 482 one after the other).
  uint32_t x = P.block0 + blockIdx.x;
  const int h = (int)(x % (uint32_t)C.heads);
  x /= (uint32_t)C.heads;
  const int split = (int)(x % (uint32_t)P.splits);
  x /= (uint32_t)P.splits;
  const Order by = order_of(P.S, (int)(x / (uint32_t)P.rtiles));
  const int b = by.ragged ? by.b : (int)(x % (uint32_t)P.S.n);
  const int rt = P.rtiles - 1 - (int)(by.ragged ? x % (uint32_t)P.rtiles : x / (uint32_t)P.S.n);
  const int64_t bh = (int64_t)b * C.heads + h;
  KvSeq q;
  if (!kv_seq(P.S, C.page, b, &q)) return;
  const int rows = q.n * A.group, r0 = rt * 32 * kWaves;
  if (r0 >= rows) return;
  int cb, ce, splits;
  if (!tile_span(P, q, r0, min(r0 + 32 * kWaves, rows), split, &cb, &ce, &splits)) return;
  const int t = threadIdx.x, lane = t & 63, m = lane & 31, g = lane >> 5;
  // Uniform: branches of a wave are branches, not masks (prompt of 16384: 2.30 ms, else 2.43).  With wider heads the
  // accumulators then no longer fit beside the rest (256 dims: 760 us instead of 638).
  const int wave = ND <= 4 ? __builtin_amdgcn_readfirstlane(t >> 6) : t >> 6;
  const int d = C.d;
  const KvNibbles nib = kv_nibbles();
  const int rw = r0 + 32 * wave;  // this wave's first row

  // the tiles of this wave's rows
  int jlo, jhi, any;
  row_span(A, q, min(rw, rows - 1), &jlo, &any);
  row_span(A, q, min(rw + 32, rows) - 1, &any, &jhi);
  const int wb = max(cb, jlo / kChunk), we = rw < rows ? min(ce, (int)cdiv(jhi, kChunk)) : cb;

  f32x16v acc[ND];
  float M = -INFINITY, l = 0.0f;
#pragma unroll
  for (int n = 0; n < ND; ++n)
#pragma unroll
    for (int i = 0; i < 16; ++i) acc[n][i] = 0.0f;

  const int64_t hb = kv_bytes<FMT>((int64_t)C.page * d);
  const int db = (int)kv_bytes<FMT>(d);
  const int pmask = C.page - 1;
  const int *table = P.S.table + (int64_t)b * P.S.table_ld;
  const int run = t & 3;  // this thread's value pieces are of this run of a tile
  // Loads have no conditions, so that they and the arithmetic around them stay in one block of code: positions behind the
  // end and pages that are not there read something of the cache that counts for nothing.
  const int last = max(q.len - 1, 0);
  auto page_of = [&](int j) {
    const int pg = table[min(j, last) >> C.shift];
    return ONE ? __builtin_amdgcn_readfirstlane(pg) : pg;
  };
  auto there_at = [&](int pg, int j) { return j < q.len && pg >= 0 && pg < C.pages; };
  auto page_at = [&](int pg) { return (int64_t)(pg >= 0 && pg < C.pages ? pg : 0) * C.heads + h; };
  constexpr int NK = ONE ? 1 : KP;
  int kpg[NK], vpg;  // pages of the codes that are loaded next
  u32x4 kc[KP];
  std::conditional_t<I4, u32x2, u32x4> vc[VP];
  float2 rsc;  // 4-bit codes: of position t / 4 (of 16) of this thread's run
  bool rthere;
  auto key_pages = [&](int c, int (&pg)[NK]) {
#pragma unroll
    for (int i = 0; i < NK; ++i) pg[i] = page_of(c * kChunk + (ONE ? 0 : (t + i * T) / PC));
  };
  auto value_page = [&](int c) { vpg = page_of(c * kChunk + (ONE ? 0 : 16 * run)); };
  auto load_keys = [&](int c, const int (&pg)[NK], u32x4 (&to)[KP]) {
    if constexpr (ONE) {
      const uint8_t *kp = C.k + page_at(pg[0]) * hb + ((c * kChunk) & pmask) * db;
#pragma unroll
      for (int i = 0; i < KP; ++i) {
        const int p = min(t + i * T, KN - 1);
        to[i] = *reinterpret_cast<const u32x4 *>(kp + (uint32_t)(p / PC * db + min(16 * (p % PC), db - 16)));
      }
    } else {
#pragma unroll
      for (int i = 0; i < KP; ++i) {
        const int p = min(t + i * T, KN - 1), tok = p / PC, cc = min(16 * (p % PC), db - 16);
        to[i] = *reinterpret_cast<const u32x4 *>(C.k + page_at(pg[i]) * hb + ((c * kChunk + tok) & pmask) * db + cc);
      }
    }
  };
  auto load_values = [&](int c) {
    const int j0 = c * kChunk + (ONE ? 0 : 16 * run);
    rthere = there_at(vpg, j0);
    const int64_t at = page_at(vpg);
    const uint8_t *vp = C.v + at * hb + kv_bytes<FMT>(j0 & pmask);
#pragma unroll
    for (int i = 0; i < VP; ++i)
      vc[i] = *reinterpret_cast<const std::remove_reference_t<decltype(vc[0])> *>(
          vp + (uint32_t)kv_bytes<FMT>(min((t >> 2) + i * (T / 4), d - 1) * C.page + (ONE ? 16 * run : 0)));
    if constexpr (I4) {
      const int64_t tok = at * C.page + (j0 & pmask) + (ONE ? 16 * run : 0) + ((t >> 2) & 15);
      rsc = float2{C.ks[tok], C.vs[tok]};
    } else {
      rsc = float2{C.ks[at], C.vs[at]};
    }
  };
  auto store_key = [&](int c, int i, const u32x4 (&from)[KP]) {
    const int p = t + i * T;
    if (KN % T != 0 && p >= KN) return;
    if constexpr (I4) {
      f16x8 *o = reinterpret_cast<f16x8 *>(&kt[c & 1][p / PC * KLD + 32 * (p % PC)]);
#pragma unroll
      for (int y = 0; y < 4; ++y) o[y] = kv_widen4x8(from[i][y], nib);
    } else {
      f16x8 *o = reinterpret_cast<f16x8 *>(&kt[c & 1][p / PC * KLD + 16 * (p % PC)]);
      o[0] = kv_widen8<FMT>(from[i].x, from[i].y);
      o[1] = kv_widen8<FMT>(from[i].z, from[i].w);
    }
  };
  auto store_keys = [&](int c, const u32x4 (&from)[KP]) {
#pragma unroll
    for (int i = 0; i < KP; ++i) store_key(c, i, from);
  };
  auto store_value = [&](int c, int i) {
    if (VN % T != 0 && t + i * T >= VN) return;
    f16x8 *o = reinterpret_cast<f16x8 *>(&vt[c & 1][((t >> 2) + i * (T / 4)) * VLD + 16 * run]);
    if constexpr (I4) {
      o[0] = kv_widen4x8(vc[i].x, nib);
      o[1] = kv_widen4x8(vc[i].y, nib);
    } else {
      o[0] = kv_widen8<FMT>(vc[i].x, vc[i].y);
      o[1] = kv_widen8<FMT>(vc[i].z, vc[i].w);
    }
  };
  auto store_values = [&](int c) {
#pragma unroll
    for (int i = 0; i < VP; ++i) store_value(c, i);
  };
  // codes past the end may be NaN, which no weight of 0 takes out
  auto clear_values = [&](int c) {
    if constexpr (FMT == KM_KV_F8) {
      int left = rthere ? q.len - c * kChunk - 16 * run : 0;
      if (left < 16) {
        asm volatile("" : "+v"(left));  // a branch: rarely taken
#pragma unroll
        for (int i = 0; i < VP; ++i)
#pragma unroll
          for (int y = 0; y < 4; ++y) {
            const int k = left - 4 * y;
            vc[i][y] &= k >= 4 ? 0xffffffffu : k <= 0 ? 0u : (1u << (8 * k)) - 1u;
          }
      }
    }
  };
  auto store_scales = [&](int c) {
    if constexpr (I4) {
      if (t < kChunk) {
        const int tok = 16 * run + (t >> 2);
        const bool in = rthere && c * kChunk + tok < q.len;
        tsc[c & 1][0][tok] = in ? rsc.x : 1.0f;
        tsc[c & 1][1][tok] = in ? __builtin_amdgcn_logf(rsc.y) : 0.0f;
        tsc[c & 1][2][tok] = in ? 1.0f / rsc.y : 1.0f;
      }
      if (t < 4) sc[c & 1][t] = float4{1.0f, 0.0f, 1.0f, rthere ? 1.0f : 0.0f};
    } else if (t < 4)
      sc[c & 1][t] = rthere ? float4{rsc.x, __builtin_amdgcn_logf(rsc.y), 1.0f / rsc.y, 1.0f}
                            : float4{1.0f, 0.0f, 1.0f, 0.0f};
  };
  const int krow = ((m & 4) << 1) | ((m & 8) >> 1) | (m & 19);  // bits 2 and 3 exchanged
  // operands of step k: keys of 32 positions at 16 dims, values of 32 dims at 16 positions
  constexpr int KS = 4 * ND, RD = 4;  // operands are read RD steps ahead
  auto key_at = [&](int c, int k) {
    return *reinterpret_cast<const f16x8 *>(&kt[c & 1][(32 * (k / (2 * ND)) + krow) * KLD + 16 * (k % (2 * ND)) + 8 * g]);
  };
  auto value_at = [&](int c, int k) {
    return *reinterpret_cast<const f16x8 *>(&vt[c & 1][(32 * (k % ND) + m) * VLD + 16 * (k / ND) + 8 * g]);
  };
  // The first tile's keys and values and the second's keys are asked for before the queries are looked at.
  u32x4 kc0[KP];
  if (cb < ce) {
    int kp0[NK], kp1[NK], vp1;
    key_pages(cb, kp0);
    key_pages(cb + 1, kp1);
    key_pages(cb + 2, kpg);
    value_page(cb + 1);
    vp1 = vpg;
    value_page(cb);
    load_keys(cb, kp0, kc0);
    load_values(cb);
    load_keys(cb + 1, kp1, kc);
    vpg = vp1;
  }

  f16x8 qf[2 * ND];
  float cs;
  int lo, hi;
  const int rq = min(rw + m, rows - 1);  // rows past the last repeat it and are not stored
  row_span(A, q, rq, &lo, &hi);
  const uint16_t *qp = static_cast<const uint16_t *>(A.q.p) + row_at(A, C, q, h, rq).q;
  u32x4 raw[ND][2];  // pairs of 8 values: dims 32 n + 8 g and 16 further
#pragma unroll
  for (int n = 0; n < ND; ++n)
#pragma unroll
    for (int i = 0; i < 2; ++i)
      raw[n][i] = *reinterpret_cast<const u32x4 *>(qp + min(32 * n + 16 * i, d - 16) + 8 * g);
  float top = 0.0f, f;
#pragma unroll
  for (int n = 0; n < ND; ++n) top = fmaxf(top, top16<1>(raw[n], A.type));
  q_scale(max_halves(top), A.scale, &f, &cs);
#pragma unroll
  for (int n = 0; n < ND; ++n) {
    float v[16];
    values16<1>(raw[n], A.type, v);
#pragma unroll
    for (int i = 0; i < 16; ++i)
      qf[2 * n + i / 8][place8<FMT>(i % 8)] = 32 * n + 16 * (i / 8) < d ? (_Float16)(v[i] * f) : (_Float16)0.0f;
  }

  if (cb < ce) {
    store_keys(cb, kc0);
    store_keys(cb + 1, kc);
    clear_values(cb);
    store_values(cb);
    store_scales(cb);
    load_keys(cb + 2, kpg, kc);
    load_values(cb + 1);
    key_pages(cb + 3, kpg);
    value_page(cb + 2);
  }
  f32x16v s[2];
  auto scores = [&](int c, int tt) {  // of 32 positions
    f32x16v o;
#pragma unroll
    for (int i = 0; i < 16; ++i) o[i] = 0.0f;
#pragma unroll
    for (int k = 0; k < 2 * ND; ++k) {
      const f16x8 a = *reinterpret_cast<const f16x8 *>(&kt[c & 1][(32 * tt + krow) * KLD + 16 * k + 8 * g]);
      o = mfma32(a, qf[k], o);
    }
    s[tt] = o;
  };
  __syncthreads();
  if (wb == cb && cb < we) {
    scores(cb, 0);
    scores(cb, 1);
  }
  __syncthreads();  // the first tile's keys have been read: the loop may write over them

  for (int c = cb; c < ce; ++c) {
    clear_values(c + 1);
    const bool mine = c >= wb && c < we;
    if (mine) {
      const int j0 = c * kChunk;
      float ks[NR], lv[NR], inv[NR];
      bool there = true;
      f16x8 ring[RD];
#pragma unroll
      for (int k = 0; k < RD; ++k) ring[k] = key_at(c + 1, k);
#pragma unroll
      for (int y = 0; y < NR; ++y) {
        const float4 z = sc[c & 1][y];
        ks[y] = z.x;
        lv[y] = z.y;
        inv[y] = z.z;
        there = there && z.w != 0.0f;
      }
      float ck[NR], base[NR], sum[4], tl[NR];
      if (!__all(there && j0 >= lo && j0 + kChunk <= hi)) {
        int jg = j0 + 8 * g;
        asm volatile("" : "+v"(jg));  // a branch: few tiles need it, so nothing of it is kept in registers
#pragma unroll
        for (int tt = 0; tt < 2; ++tt)
#pragma unroll
          for (int i = 0; i < 16; ++i) {
            const int j = jg + 32 * tt + 16 * (i >> 3) + (i & 7);
            if (j < lo || j >= hi || sc[c & 1][ONE ? 0 : 2 * tt + (i >> 3)].w == 0.0f) s[tt][i] = -INFINITY;
          }
      }
      float Mt = -INFINITY;
      float tk[2], tv[2], ti[2];  // 4-bit codes: of the positions of s[0] and s[1], one to a lane of sixteen
      const float c4 = fmaxf(cs, 0x1p-126f);
      if constexpr (I4) {
#pragma unroll
        for (int tt = 0; tt < 2; ++tt) {
          const int at = 32 * tt + 16 * ((lane >> 3) & 1) + 8 * g + (lane & 7);
          tk[tt] = tsc[c & 1][0][at];
          tv[tt] = tsc[c & 1][1][at];
          ti[tt] = tsc[c & 1][2][at];
          each<16>([&](auto e) {
            constexpr int i = e;
            s[tt][i] = token_score<i>(s[tt][i], c4, tk[tt], tv[tt]);
          });
        }
      }
#pragma unroll
      for (int y = 0; y < NR; ++y) {
        constexpr int E = 32 / NR;
        float top = -INFINITY;
#pragma unroll
        for (int i = E * y; i < E * (y + 1); ++i) top = fmaxf(top, s[i >> 4][i & 15]);
        // a factor of 0 (a row of tiny queries) would make NaN of -inf
        ck[y] = fmaxf(cs * ks[y], 0x1p-126f);
        tl[y] = I4 ? top : fmaf(top, ck[y], lv[y]);
        Mt = fmaxf(Mt, tl[y]);
      }
      Mt = max_halves(Mt);
      bool rare = Mt > M + kSlack;
#pragma unroll
      for (int y = 0; y < NR; ++y) rare = rare || (!I4 && far_below(tl[y], tl[y] - lv[y], M));
      if (__any(rare)) {
        const float Mn = fmaxf(M, Mt);
        const float al = Mn == -INFINITY ? 1.0f : half_step(M, Mn);
        l = l * al * al;
#pragma unroll
        for (int n = 0; n < ND; ++n) acc[n] *= al * al;
        M = Mn;
#pragma unroll
        for (int y = 0; y < NR; ++y) {
          constexpr int E = 32 / NR;
          if (I4 || !far_below(tl[y], tl[y] - lv[y], M)) continue;
          inv[y] = 0.0f;
#pragma unroll
          for (int i = E * y; i < E * (y + 1); ++i)
            l = far_add(l, fmaf(s[i >> 4][i & 15], ck[y], kUp32 - 18.0f - M));
        }
      }
      const float up = kUp32 - (M == -INFINITY ? 0.0f : M);
#pragma unroll
      for (int y = 0; y < NR; ++y) base[y] = lv[y] + up;
      // Steps of one product each, in this order: the operand of some steps ahead is read, the product is
      // issued, and what the vector unit does meanwhile follows.  First the scores of the next tile and this tile's
      // exponentials, 16 registers of scores at a time (the next tile's replace them), then the second products
      // and the widening of later tiles.
      f16x8 w[4];
      f32x16v o;
#pragma unroll
      for (int k = 0; k < KS; ++k) {
        const int tt = k / (2 * ND), kk = k % (2 * ND);
        __builtin_amdgcn_sched_barrier(0);
        const f16x8 a = ring[k % RD];
        ring[k % RD] = k + RD < KS ? key_at(c + 1, k + RD) : value_at(c, k + RD - KS);
        if (kk == 0) {
#pragma unroll
          for (int i = 0; i < 16; ++i) o[i] = 0.0f;
        }
        o = mfma32(a, qf[kk], o);
        // elements [e0, e1) of 16
        const int e0 = kk * 16 / (2 * ND), e1 = (kk + 1) * 16 / (2 * ND);
        if constexpr (I4) {
          each<16>([&](auto n) {
            constexpr int i = n;
            if (i < e0 || i >= e1) return;
            const int y = 2 * tt + (i >> 3);
            const float e = __builtin_amdgcn_exp2f(s[tt][i] + up), z = kv_row_bcast<i>(ti[tt]);
            sum[y] = (i & 7) ? fmaf(z, e, sum[y]) : z * e;
            w[y][kv_place4(i & 7)] = (_Float16)e;
          });
        } else {
#pragma unroll
          for (int i = e0; i < e1; ++i) {
            const int y = 2 * tt + (i >> 3);
            const float e = __builtin_amdgcn_exp2f(fmaf(s[tt][i], ck[y % NR], base[y % NR]));
            sum[y] = (i & 7) ? sum[y] + e : e;
            w[y][i & 7] = (_Float16)e;
          }
        }
        if (kk == 2 * ND - 1) s[tt] = o;
      }
#pragma unroll
      for (int k = 0; k < KS; ++k) {
        const int y = k / ND, n = k % ND;
        __builtin_amdgcn_sched_barrier(0);
        const f16x8 a = ring[(k + KS) % RD];
        if (k + RD < KS) ring[(k + KS) % RD] = value_at(c, k + RD);
        acc[n] = mfma32(a, w[y], acc[n]);
        if (n == 0) l = fmaf(sum[y] * kUnit, inv[y % NR], l);
        // the widening, a piece at a time
        const int p0 = k * (KP + VP) / KS, p1 = (k + 1) * (KP + VP) / KS;
#pragma unroll
        for (int i = p0; i < p1; ++i) {
          if (i < KP) store_key(c + 2, i, kc);
          else store_value(c + 1, i - KP);
        }
      }
      __builtin_amdgcn_sched_barrier(0);
    } else {
      if (c + 1 == wb && wb < we) {
        scores(c + 1, 0);
        scores(c + 1, 1);
      }
      store_keys(c + 2, kc);
      store_values(c + 1);
    }
    // keys of tile c + 2 and values of tile c + 1 are in LDS, the loads of the tiles after them begin
    store_scales(c + 1);
    load_keys(c + 3, kpg, kc);
    load_values(c + 2);
    key_pages(c + 4, kpg);
    value_page(c + 3);
    __syncthreads();
  }

  l += __shfl_xor(l, 32);
  if (M == INFINITY) l = NAN;  // scores past fp32's range: no weight is left to tell them from a row that sees nothing
  const int r = rw + m;
  if (r >= rows) return;
  if (splits > 1) {
    if (l != l) M = INFINITY;  // the maximum does not see NaN
    float *o = P.part + (((bh * P.rtiles + rt) * P.splits + split) * kWaves + wave) * part32_floats(ND);
#pragma unroll
    for (int n = 0; n < ND; ++n)
#pragma unroll
      for (int i = 0; i < 4; ++i)
        *reinterpret_cast<f32x4 *>(o + ((n * 4 + i) * 64 + lane) * 4) =
            f32x4{acc[n][4 * i], acc[n][4 * i + 1], acc[n][4 * i + 2], acc[n][4 * i + 3]};
    if (g == 0) {
      o[ND * 1024 + m] = M;
      o[ND * 1024 + 32 + m] = l;
    }
    return;
  }
  const RowAt at = row_at(A, C, q, h, r);
  const RowSum end = row_sum(M, l, kUp32);
#pragma unroll
  for (int n = 0; n < ND; ++n)
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int c = 32 * n + 8 * i + 4 * g;
      float z[4];
#pragma unroll
      for (int y = 0; y < 4; ++y) z[y] = acc[n][4 * i + y] * end.a * end.b;
      if (c < d) store_o4(A, at.o + c, z);
    }
  if (A.lse && g == 0) A.lse[at.lse] = end.lse;
}

struct Plan {
  bool prompt;
  int nt, rt, rtiles, deal, splits, per;
  bool wide;  // kWideWaves waves to a workgroup of kv_attend_kernel
  int spread;  // the join has a workgroup per accumulator of a lane
  int64_t tiles;
};

int dim_tiles(int d) {  // the instantiated widths
  const int t = (int)cdiv(d, 16);
  return t <= 4 ? 4 : t <= 5 ? 5 : t <= 6 ? 6 : t <= 8 ? 8 : t <= 12 ? 12 : 16;
}

int dim_tiles32(int d) {
  const int t = (int)cdiv(d, 32);
  return t <= 2 ? 2 : t <= 3 ? 3 : t <= 4 ? 4 : t <= 6 ? 6 : 8;
}

Plan plan(const KvCache &C, const KvSeqs &S, const KvAttend &A) {
  Plan p{};
  const int64_t rows = (int64_t)S.max_rows * A.group;
  // the most chunks that a tile's rows see
  const int64_t len = A.window ? std::min<int64_t>(S.max_len, (int64_t)A.window + S.max_rows + kChunk) : S.max_len;
  const int64_t chunks = std::max<int64_t>(1, cdiv(len, kChunk));
  p.prompt = rows > 32 && A.type != KM_T_F32;
  p.nt = p.prompt ? dim_tiles32(C.d) : dim_tiles(C.d);
  p.rt = p.prompt ? kWaves : rows > 16 && A.type != KM_T_F32 && p.nt <= 8 ? 2 : 1;
  p.rtiles = (int)cdiv(rows, (p.prompt ? 32 : 16) * p.rt);
  p.tiles = (int64_t)S.n * C.heads * p.rtiles;
  if (p.prompt) {
    p.per = (int)std::min(chunks, std::max<int64_t>(8, cdiv(p.tiles * chunks, 512)));
    p.spread = p.tiles * p.rt < 256;
  } else {
    // Short contexts, or tiles enough to fill the card several times: a workgroup for each tile and no join.  A
    // workgroup takes 6.5 us and 1.7 more per 256 positions (8 heads of 128); splitting it up and joining takes 14 us up to
    // some 4096 positions, more where tiles nearly fill the card by themselves: pieces of them are then short, and there are
    // many to join.  Where a workgroup per tile leaves every workgroup little to do, even splits; where it streams for long,
    // what differing lengths leave idle counts for more, and tiles are dealt out.  8 heads of 128 in bf16, the size that the
    // bounds below are from, lengths from 1 on:
    //   64 sequences up to 16384 (512 tiles): 194 us dealt out, 225 even splits; up to 4000: 56, a workgroup each 61
    //   256 up to 4000 (2048 tiles): 242 us dealt out, 213 a workgroup each; 128 up to 4000: 130 either way
    //   31 up to 3000 (248 tiles): 37 us dealt out, 27 a workgroup each; 31 of 6000 91 and 71; 24 up to 8000: 47 and 52
    //   16 up to 1500 (128 tiles): 19 us even splits, 15 a workgroup each; up to 3000: 23 and 25
    //   8 up to 1500 (64 tiles): 14 us even splits, 15 a workgroup each
    //   16 behind a window of 4096, 4 heads (64 tiles): 39 us dealt out, 28 even splits
    // Workgroups of four waves (wider heads, fp32) gain less from a workgroup each, up to 3000 positions: 31 of fp32 up to 3000 33 us
    // so, 40 dealt out, 24 up to 6000 55 and 47; 31 of 256 dims up to 3000 52 and 70, 24 up to 6000 97 and 94.
    // Workgroups of eight waves (accumulators of up to 128 dims, 16-bit types) have the loads of a CU in flight with half the
    // tiles' beginnings, ends and pieces to join, but wait for each other at both:
    //   a tile each, 32 up to 2000: 23.2 us with four waves, 20.8 with eight; one of 300 7.0 and 7.2 (64 dims)
    //   even splits, one head, 100000 positions: 22.7 and 17.9; one sequence of 1500, 8 heads: 11.3 and 12.9
    //   dealt out, 64 up to 16384: 194 and 187; 32 up to 8000: 48 and 51; 2 up to 29000 of 16 heads (32 tiles): 26 and 27;
    //   32 rows to a tile, 64 up to 4000: 68 and 104
    // Narrower heads keep four waves: dealt out, 64 up to 16384 of 64 dims 111 us with four and 118 with eight, of 80 139 and 144,
    // of 96 162 and 160; even splits are alike, but for one head, 100000 positions: 20 and 15.
    // Workgroups that run at a time with 128 dims, two waves to a SIMD (64 dims have room for three or four).  4-bit codes and 16 rows: three,
    // which pays where tiles are dealt out (64 up to 16384: 128 us, 159 with two in workgroups of eight), elsewhere a third more
    // pieces cost more than they gain (one sequence of 131071 40.6 us with 768, 38.9 with 512; 128 up to 4000 81 and 72), and short
    // tiles take eight waves as the other formats do (31 up to 3000: 30.5 us with four, 25.5 with eight).
    const int64_t cap = (int64_t)S.max_pages * C.page / kChunk + 1 + kTileCost;  // whatever max_len says
    const bool three = C.fmt == KM_KV_I4 && p.nt <= 8 && p.rt == 1 && A.type != KM_T_F32;
    const int64_t most = p.nt <= 8 ? 512 : 256;
    const bool eight = p.nt <= 8 && A.type != KM_T_F32;
    p.spread = p.tiles * p.rt < 256;
    const int64_t alone = p.tiles > 256    ? 32  // the most chunks of a tile that is not split up
                          : p.tiles >= 192 ? (eight ? 96 : 48)
                          : p.tiles >= 128 ? (eight && p.rt == 1 ? 32 : 24)
                                           : 16;
    if (p.rtiles > 4 || p.tiles >= 2 * most || chunks <= alone) {
      p.wide = eight && p.tiles <= 256 && chunks > 2 * kAttendWaves;
      p.per = (int)chunks;
    } else if (p.tiles * chunks <= 16 * most || S.n == 1 || p.tiles * cap >= INT32_MAX) {
      p.wide = eight && p.nt == 8 && (p.tiles * chunks > kAttendWaves * most || chunks > 1024);
      p.per = (int)(p.wide ? std::max<int64_t>(kWideWaves, cdiv(2 * p.tiles * chunks, most))
                           : std::max<int64_t>(kAttendWaves, cdiv(p.tiles * chunks, most)));
    } else {
      p.deal = 1;
      p.wide = eight && !three && p.nt == 8 && p.rt == 1 && chunks >= 160 && p.tiles >= 128;
      p.per = 2 * (p.wide ? kWideWaves : kAttendWaves);
      p.splits = (int)std::min<int64_t>(p.wide ? most / 2 : three ? 768 : most, cdiv(p.tiles * chunks, p.per));
      return p;
    }
  }
  p.splits = (int)cdiv(chunks, p.per);
  return p;
}

int accumulators(const Plan &p) { return p.nt * (p.prompt ? 4 : 1); }
int64_t join_blocks(const Plan &p) { return p.tiles * p.rt * (p.spread ? accumulators(p) : 1); }

template <int FMT>
km_status go_attend(const KvCache &C, const KvSeqs &S, const KvAttend &A, void *ws, hipStream_t s) {
  const Plan p = plan(C, S, A);
  AttendArgs P{C, S, A, p.rtiles, p.deal, p.splits, p.per, static_cast<float *>(ws), 0};
  auto go_prompt = [&](auto *kernel) {
    const int64_t blocks = p.tiles * p.splits, most = kv_piece(64 * kWaves);
    for (int64_t b = 0; b < blocks; b += most) {
      P.block0 = (uint32_t)b;
      kernel<<<dim3((unsigned)std::min(most, blocks - b)), 64 * kWaves, 0, s>>>(P);
    }
  };
  // In pieces of whole sequences where it takes some: an offset in the kernel costs single tokens 2 %.
  auto go = [&](auto *kernel, int waves) {
    const int64_t each = p.deal ? p.splits : p.tiles / S.n * p.splits, most = p.deal ? S.n : kv_piece(64 * waves) / each;
    for (int64_t b = 0; b < S.n; b += most) {
      AttendArgs Q = P;
      Q.S.n = (int)std::min(most, S.n - b);
      Q.S.table += b * S.table_ld;
      Q.S.lens += b;
      if (S.starts) {
        Q.S.starts += b;
      } else if (b) {
        const int64_t row = b * S.max_rows, elem = A.type == KM_T_F32 ? 4 : 2;
        Q.S.rows -= row;
        Q.A.q.p = static_cast<char *>(A.q.p) + row * A.q.row * elem;
        Q.A.out.p = static_cast<char *>(A.out.p) + row * A.out.row * elem;
        if (A.lse) Q.A.lse += row * C.heads * A.group;
      }
      kernel<<<dim3((unsigned)(p.deal ? each : Q.S.n * each)), 64 * waves, 0, s>>>(Q);
    }
  };
  // Calls of 1024 tiles and more are not split up: their pieces have no joins, and a join is one launch.
#define KV_J(NA, G, D, UP) \
  kv_join_kernel<NA, G, D><<<dim3((unsigned)join_blocks(p)), 64 * kJoinWaves, 0, s>>>(P, p.rt, p.spread, UP)
  if (p.prompt) {
#define KV_N(N)                                                                                                               \
  case N:                                                                                                                     \
    C.page >= kChunk ? go_prompt(kv_prompt_kernel<FMT, N, true>) : go_prompt(kv_prompt_kernel<FMT, N, false>);                \
    KMQ_LAUNCH_CHECK("kv_attend");                                                                                            \
    if (p.splits > 1) KV_J(4 * N, 2, false, kUp32);                                                                           \
    break;
    switch (p.nt) {
      KV_N(2)
      KV_N(3)
      KV_N(4)
      KV_N(6)
      KV_N(8)
    }
#undef KV_N
    KMQ_LAUNCH_CHECK("kv_attend");
    return KM_OK;
  }
#define KV_K(F, N, R, Z, W) \
  C.page >= kChunk ? go(kv_attend_kernel<F, N, R, Z, true, W>, W) : go(kv_attend_kernel<F, N, R, Z, false, W>, W)
#define KV_W(F, N, R)                                                       \
  if (N <= 8 && p.wide) KV_K(F, N, R, 1, (N <= 8 ? kWideWaves : kAttendWaves)); \
  else KV_K(F, N, R, 1, kAttendWaves);
#define KV_R(F, N)                                                \
  if (A.type == KM_T_F32) {                                       \
    KV_K(F, N, 1, 2, kAttendWaves);                               \
  } else if (N <= 8 && p.rt == 2) {                               \
    KV_W(F, N, (N <= 8 ? 2 : 1))                                  \
  } else {                                                        \
    KV_W(F, N, 1)                                                 \
  }
#define KV_N(N)                                                                                         \
  case N:                                                                                               \
    KV_R(FMT, N)                                                                                        \
    KMQ_LAUNCH_CHECK("kv_attend");                                                                      \
    if (p.deal)                                                                                         \
      KV_J(N, 4, true, kUp);                                                                            \
    else if (p.splits > 1)                                                                              \
      KV_J(N, 4, false, kUp);                                                                           \
    break;
  switch (p.nt) {
    KV_N(4)
    KV_N(5)
    KV_N(6)
    KV_N(8)
    KV_N(12)
    KV_N(16)
  }
#undef KV_N
#undef KV_R
#undef KV_W
#undef KV_K
#undef KV_J
  KMQ_LAUNCH_CHECK("kv_attend");
  return KM_OK;
}

}  // namespace
}  // namespace kmq
