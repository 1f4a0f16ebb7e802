// The attention weight that cached tokens get from a call's rows.
//
//   weight_j = decay weight_j + sum_i exp(scale <q_i, k_j> - lse_i)    over the rows i of the heads that share k_j
//
// The scores are computed again from the keys alone and the softmax statistics that the attention left, so nothing of size rows x
// positions is kept.  A position's sum belongs to one workgroup: no atomics, and an order that does not depend on scheduling.
//
// A wave takes 64 positions, whose codes it widens once and keeps in registers as the first operand (as in kv_attend.hpp, lane group
// g = lane / 16 ends with the scores of positions 16 g .. 16 g + 15 of its row), and goes through the rows 16 at a time.  Codes of all
// formats are exact in fp16 and in bf16, so 16-bit queries are the second operand as they are; fp32 ones take two halves of fp16
// after a power of two for each row.  bf16 queries reach 2^128, and their products with codes would leave fp32's range: such codes are
// taken times 2^-40 (weigh_down).  The sums of a row's lane are added up over the sixteen lanes at the end.
//
// Four ways (plan_weigh).  Single tokens: kv_weigh_tokens_kernel, bound by the bytes of the keys, 19 us for 78 MB of 16 sequences of
// 500 to 8192 tokens in int8 (13 at the rate of a read; the longest sequence's workgroups are the last).  A few hundred rows:
// kv_weigh_kernel, each wave with its own positions.  Prompts: kv_weigh_rows_kernel, the waves of a workgroup share tiles of rows in LDS;
// bound by tiles (a barrier each), the products (matrix cores 25 % busy) and the exponentials (a quarter of the vector unit's rate),
// which wait for each other: two prompts of 3133 and 5340 tokens, 4-bit codes, 244 us and 5 to join, 160 GFLOP.  Prompts of fp32 rows:
// kv_weigh_kernel with a workgroup's waves sharing 64 positions and taking the rows in turn.
#include "kv_attend.hpp"

namespace kmq {
namespace {

constexpr int kFewWaves = 4, kManyWaves = 8;  // of a workgroup

struct WeighArgs {
  KvCache C;
  KvSeqs S;
  KvAttend A;  // q, type, group, scale, causal, window, lse
  float *weight;
  float decay;
  int groups;  // workgroups of a sequence's head
  int step, step_tok, step_head;  // rows from a wave's tile to its next: tokens and heads of a token
  uint32_t group_inverse;         // 2^32 / group, rounded up
  uint32_t block0;
};

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));

// bf16 rows: a position's codes are taken times 2^-40, which is exact, or times 1.  f: the softmax's scale in base 2, ks: the position's.
// |<q, code>| is at most 2^128 448 256 < 2^145.  Where f ks < 1 the sums then stay below 2^105, what products lose below the least normal
// number changes a score by at most 2^-126 256 2^40 = 2^-78, and a factor that is raised to that number by less than 2^-21.  Elsewhere a sum past
// 2^128 is a score past 2^128, with which the row has no finite log-sum-exp, or past -2^128, which has no weight.  4-bit codes: ks lies within
// [2^-30, 2^30], so f alone decides (f ks < 2^60: at most 2^-18).
template <int FMT, int TYPE>
__device__ __forceinline__ float weigh_down(float f, float ks) {
  if constexpr (TYPE != KM_T_BF16) return 1.0f;
  return (FMT == KM_KV_I4 ? f < 0x1p30f : f * ks < 1.0f) ? 0x1p-40f : 1.0f;
}
// A factor of scores, not 0 and not infinite: -infinity (not seen) and 0 stay what they are.
__device__ __forceinline__ float weigh_bound(float x) { return fminf(fmaxf(x, 0x1p-126f), 0x1.fffffep127f); }
// What the products of 16-bit rows are multiplied by.
template <int FMT, int TYPE>
__device__ __forceinline__ float weigh_factor(float f, float ks) {
  const float up = 1.0f / weigh_down<FMT, TYPE>(f, ks);
  return weigh_bound(FMT == KM_KV_I4 || ks < 1.0f ? f * (ks * up) : (f * up) * ks);
}
// Codes as operands beside bf16 rows.
__device__ __forceinline__ f16x8 weigh_bf16(f16x8 x, float down) {
  typedef float f32x8 __attribute__((ext_vector_type(8)));
  f32x8 y;
#pragma unroll
  for (int i = 0; i < 8; ++i) y[i] = fmaf((float)x[i], down, 0.0f);  // widened and multiplied in one instruction
  return __builtin_bit_cast(f16x8, __builtin_convertvector(y, bf16x8));
}

// The sum over a lane's row of sixteen, in every lane.
__device__ __forceinline__ float sum_row(float x) {
#define KV_ROR(n) x += __uint_as_float(__builtin_amdgcn_update_dpp(0, __float_as_uint(x), 0x120 + n, 0xf, 0xf, false))
  KV_ROR(8);
  KV_ROR(4);
  KV_ROR(2);
  KV_ROR(1);
#undef KV_ROR
  return x;
}

// Waves to a SIMD that the registers have to leave room for.  fp32 rows of up to 128 dims: with room for three, 26 to 37 registers were spilled,
// 16 sequences of 500 to 8192 with 64 rows each 243 us in int8 and 300 in 4 bits, with two 168 and 165.
template <int TYPE, int NP, bool MANY>
constexpr int weigh_waves() {
  return MANY || TYPE == KM_T_F32 ? (NP <= 3 ? 2 : 1) : NP == 1 ? 4 : NP == 2 ? 3 : NP == 3 ? 2 : 1;
}

// A sequence without rows in the call: its weights times decay, by the workgroups of its heads.
__device__ __forceinline__ void weigh_idle(const WeighArgs &P, const KvSeq &q, int b, int h, int group) {
  if (P.decay == 1.0f) return;
  const KvCache &C = P.C;
  for (int64_t j = (int64_t)group * blockDim.x + threadIdx.x; j < q.len; j += (int64_t)P.groups * blockDim.x) {
    const int64_t pg = P.S.table[(int64_t)b * P.S.table_ld + (j >> C.shift)];
    if (pg < 0 || pg >= C.pages) continue;
    float *w = P.weight + (pg * C.heads + h) * C.page + (j & (C.page - 1));
    *w = P.decay != 0.0f ? *w * P.decay : 0.0f;
  }
}

// TYPE: bf16 and fp16 rows as they are, fp32 rows in two halves (NS = 2)
template <int FMT, int TYPE, int NP, bool MANY, bool ONE>
__global__ __launch_bounds__(64 * (MANY ? kManyWaves : kFewWaves), (weigh_waves<TYPE, NP, MANY>())) void kv_weigh_kernel(WeighArgs P) {
  constexpr int NS = TYPE == KM_T_F32 ? 2 : 1, W = MANY ? kManyWaves : kFewWaves;
  __shared__ float sh[MANY ? W : 1][kChunk];
  const KvCache &C = P.C;
  const KvAttend &A = P.A;
  uint32_t x = P.block0 + blockIdx.x;
  const int h = (int)(x % (uint32_t)C.heads);  // heads fastest: a head's workgroups share an XCD's L2 where they are a multiple of 8
  x /= (uint32_t)C.heads;
  // the sequences side by side: with many rows the first positions, which most rows see, begin first
  const int b = (int)(x % (uint32_t)P.S.n), group = (int)(x / (uint32_t)P.S.n);
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), m = lane & 15, g = lane >> 4;
  KvSeq q;
  if (!kv_seq(P.S, C.page, b, &q)) return;
  if (q.n == 0) return weigh_idle(P, q, b, h, group);
  const int d = C.d, rows = q.n * A.group;
  const KvNibbles nib = kv_nibbles();
  const int64_t hb = kv_bytes<FMT>((int64_t)C.page * d);
  const int db = (int)kv_bytes<FMT>(d);
  const int pmask = C.page - 1, last = q.len - 1, kr = m >> 2, ktok = m & 3;
  const int *table = P.S.table + (int64_t)b * P.S.table_ld;
  auto page_of = [&](int j) {
    const int pg = table[min(j, last) >> C.shift];
    return ONE ? __builtin_amdgcn_readfirstlane(pg) : pg;
  };
  auto there_at = [&](int pg) { return pg >= 0 && pg < C.pages; };
  auto head_at = [&](int pg) { return (int64_t)(there_at(pg) ? pg : 0) * C.heads + h; };
  // every wave's positions are behind the end at once (MANY), or no barrier follows
  for (int64_t c = MANY ? group : (int64_t)group * W + wave; c * kChunk < q.len;
       c += (int64_t)P.groups * (MANY ? 1 : W)) {
  const int j0 = (int)c * kChunk;
  // positions of this lane's scores: run g; the keys that it loads: run kr
  const int pv = page_of(j0 + (ONE ? 0 : 16 * g)), pk = ONE ? pv : page_of(j0 + 16 * kr);
  const int jm = j0 + 16 * g + m;  // the position whose weight this lane writes
  const bool there = there_at(pv), mine = there && jm < q.len;
  const int64_t at = head_at(pv) * C.page + (jm & pmask);
  const float old = mine && P.decay != 0.0f && jm < q.len - q.n ? P.weight[at] : 0.0f;

  const float f = A.scale * kLog2e;
  // keys; dims past d are 0
  f16x8 kf[4][NP][2];
  {
    float down = FMT == KM_KV_I4 || TYPE != KM_T_BF16 ? 1.0f : C.ks[head_at(pk)];
    down = weigh_down<FMT, TYPE>(f, down);
    asm("" : "+v"(down));  // no second copy of all that follows
    const uint8_t *kp = C.k + head_at(pk) * hb + ((j0 + (ONE ? 0 : 16 * kr)) & pmask) * db;
    Codes16<FMT> kw[4][NP];
#pragma unroll
    for (int st = 0; st < 4; ++st)
#pragma unroll
      for (int p = 0; p < NP; ++p) {
        const uint8_t *from = kp + 4 * st * db + ((ONE ? 16 * kr : 0) + ktok) * db + (int)kv_bytes<FMT>(min(64 * p + 16 * g, d - 16));
        kw[st][p] = *reinterpret_cast<const Codes16<FMT> *>(from);
      }
#pragma unroll
    for (int st = 0; st < 4; ++st)
#pragma unroll
      for (int p = 0; p < NP; ++p)
#pragma unroll
        for (int k = 0; k < 2; ++k) {
          kf[st][p][k] = widen8<FMT>(kw[st][p], k, nib);
          if (64 * p + 16 * g >= d) kf[st][p][k] = f16x8{0, 0, 0, 0, 0, 0, 0, 0};
          if constexpr (FMT == KM_KV_I4) {  // in the dims' order, as the queries lie
            const f16x8 y = kf[st][p][k];
            kf[st][p][k] = f16x8{y[0], y[2], y[4], y[6], y[1], y[3], y[5], y[7]};
          }
          if constexpr (TYPE == KM_T_BF16) kf[st][p][k] = weigh_bf16(kf[st][p][k], down);
        }
  }
  // what a score is multiplied by, for each of the lane's 16 positions; fp32 rows: the position's scale alone
  float ck[16];
  {
    if constexpr (FMT == KM_KV_I4) {
      const float ks = mine ? C.ks[at] : 1.0f;
      each<16>([&](auto e) { ck[e] = NS == 2 ? kv_row_bcast<e>(ks) : weigh_factor<FMT, TYPE>(f, kv_row_bcast<e>(ks)); });
    } else {
      const float ks = j0 + 16 * g < q.len && there ? C.ks[head_at(pv)] : 1.0f;
      ck[0] = NS == 2 ? ks : weigh_factor<FMT, TYPE>(f, ks);
#pragma unroll
      for (int e = 1; e < 16; ++e) ck[e] = ck[0];
    }
  }

  // the rows that may see one of the positions
  const int first = q.len - q.n;  // position of row 0
  int t0 = 0, t1 = q.n;
  if (A.causal) t0 = max(j0 - first, 0);
  if (A.window) t1 = (int)max((int64_t)0, min((int64_t)q.n, (int64_t)j0 + kChunk - 1 + A.window - first));
  // From the last rows, which most positions are seen by, to the first: workgroups that begin together go through the same rows at
  // the same time, and find them in L2.
  const int r1 = t1 * A.group, r_lo = (int)min((int64_t)t0 * A.group, (int64_t)rows) & ~15;
  int rt = ((r1 - 1) & ~15) - (MANY ? 16 * wave : 0);  // the first row of the tile that is loaded next
  int tok = max(rt, 0) / A.group, hq = max(rt, 0) - tok * A.group;  // its token and its place among the token's heads
  // Row rt + x (x < 16): tokens further on and place; a division by the group, as a product where that is exact.
  auto row_of = [&](int x, int *dt, int *dh) {
    const int y = hq + x;
    *dt = A.group == 1 ? y : A.group >= 16 ? (y >= A.group) : (int)__umulhi((uint32_t)y, P.group_inverse);
    *dh = y - *dt * A.group;
  };
  auto offset_of = [&](int dt, int dh) { return (int64_t)dt * A.q.row + (int64_t)dh * A.q.head; };
  u32x4 raw[NP][2 * NS];
  float lse;
  int pos;  // of this lane's row
  auto load = [&] {
    const char *base = static_cast<const char *>(A.q.p) +
                       ((q.row0 + tok) * A.q.row + (int64_t)h * A.group * A.q.head) * (2 * NS);  // of the tile's token
    int dt, dh;
    row_of(m, &dt, &dh);
    const bool in = rt + m < r1;  // rows behind the last: the tile's token's first one, which does not count there
    pos = first + min(tok + dt, q.n - 1);
    lse = in ? A.lse[(q.row0 + tok + dt) * C.heads * A.group + h * A.group + dh] : INFINITY;
    const char *qp = base + (in ? offset_of(dt, dh) * (2 * NS) : 0);
#pragma unroll
    for (int p = 0; p < NP; ++p)
#pragma unroll
      for (int i = 0; i < 2 * NS; ++i)
        raw[p][i] = reinterpret_cast<const u32x4 *>(qp + 2 * NS * min(64 * p + 16 * g, d - 16))[i];
  };
  auto next = [&] {
    rt -= P.step;
    tok -= P.step_tok;
    hq -= P.step_head;
    if (hq < 0) {
      hq += A.group;
      --tok;
    }
  };

  float sum[16];
#pragma unroll
  for (int e = 0; e < 16; ++e) sum[e] = 0.0f;
  if (rt >= r_lo) load();
  while (rt >= r_lo) {
    const bool counts = fabsf(lse) < INFINITY;
    const float nl = counts ? -lse * kLog2e : -INFINITY;
    f16x8 qf[NP][2][NS];
    float c32 = 1.0f;  // fp32 rows: what a score is multiplied by, 4-bit codes without the position's scale
    if (!__all(counts)) {  // rows that do not count may hold NaN
#pragma unroll
      for (int p = 0; p < NP; ++p)
#pragma unroll
        for (int k = 0; k < 2 * NS; ++k) raw[p][k] = counts ? raw[p][k] : u32x4{0, 0, 0, 0};
    }
    if constexpr (NS == 1) {
#pragma unroll
      for (int p = 0; p < NP; ++p)
#pragma unroll
        for (int k = 0; k < 2; ++k) qf[p][k][0] = __builtin_bit_cast(f16x8, raw[p][k]);
    } else {
      float v[NP][16], top = 0.0f;
#pragma unroll
      for (int p = 0; p < NP; ++p) {
        values16<2>(raw[p], KM_T_F32, v[p]);
#pragma unroll
        for (int i = 0; i < 16; ++i) top = fmaxf(top, fabsf(v[p][i]));
      }
      float f;
      q_scale(max_groups(top), A.scale, &f, &c32);
      c32 = weigh_bound(FMT == KM_KV_I4 ? c32 : c32 * ck[0]);
#pragma unroll
      for (int p = 0; p < NP; ++p)
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          const float y = v[p][i] * f;
          const _Float16 y16 = (_Float16)y;
          qf[p][i / 8][0][i % 8] = y16;
          qf[p][i / 8][1][i % 8] = (_Float16)(y - (float)y16);
        }
    }
    // positions that the row sees; the next rows are on their way meanwhile
    const int see0 = A.window ? max(pos + 1 - A.window, 0) : 0, see1 = A.causal ? max(pos + 1, 0) : q.len;
    next();
    if (rt >= r_lo) load();
    f32x4 s[4];
#pragma unroll
    for (int st = 0; st < 4; ++st) s[st] = f32x4{0, 0, 0, 0};
#pragma unroll
    for (int p = 0; p < NP; ++p)
#pragma unroll
      for (int k = 0; k < 2; ++k)
#pragma unroll
        for (int z = 0; z < NS; ++z)
#pragma unroll
          for (int st = 0; st < 4; ++st) {  // four sums in turn: none waits for its last product
            if constexpr (TYPE == KM_T_BF16)
              s[st] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, kf[st][p][k]),
                                                              __builtin_bit_cast(bf16x8, qf[p][k][z]), s[st], 0, 0, 0);
            else
              s[st] = mfma16(kf[st][p][k], qf[p][k][z], s[st]);
          }
    if constexpr (NS == 2 && FMT == KM_KV_I4) {
#pragma unroll
      for (int e = 0; e < 16; ++e) s[e / 4][e % 4] *= ck[e];
    }
    if (!__all(j0 >= see0 && j0 + kChunk <= see1)) {
      int jg = j0 + 16 * g;
      asm volatile("" : "+v"(jg));  // a branch: few tiles need it, so nothing of it is kept in registers
#pragma unroll
      for (int e = 0; e < 16; ++e) {
        const int j = jg + e;
        if (j < see0 || j >= see1) s[e / 4][e % 4] = -INFINITY;
      }
    }
#pragma unroll
    for (int e = 0; e < 16; ++e) sum[e] += __builtin_amdgcn_exp2f(fmaf(s[e / 4][e % 4], NS == 2 ? c32 : ck[e], nl));
  }

  float total = 0.0f;
#pragma unroll
  for (int e = 0; e < 16; ++e) {
    const float z = sum_row(sum[e]);
    total = m == e ? z : total;
  }
  if (MANY) {
    sh[wave][16 * g + m] = total;
    __syncthreads();
    total = 0.0f;
#pragma unroll
    for (int y = 0; y < W; ++y) total += sh[y][16 * g + m];
    __syncthreads();  // before the next positions' sums
  }
  if (mine && (!MANY || wave == 0)) P.weight[at] = fmaf(old, P.decay, total);
  }
}


// ---- up to 16 rows to a cache head: single tokens ---------------------------------------------------------------------------------
//
// The rows stay in registers, scaled to fp16 as in kv_attend.hpp, and a wave goes through chunks of 64 positions, the next one's codes
// and weights on their way meanwhile (16 sequences of 500 to 8192 tokens: 31 us without, 19 with both).
template <int FMT, int NS, int NP, bool ONE>
__global__ __launch_bounds__(64 * kFewWaves, NP <= 2 && NS == 1 ? 4 : 2) void kv_weigh_tokens_kernel(WeighArgs P) {
  const KvCache &C = P.C;
  const KvAttend &A = P.A;
  uint32_t x = P.block0 + blockIdx.x;
  const int h = (int)(x % (uint32_t)C.heads);  // heads fastest: a head's workgroups share an XCD's L2 where they are a multiple of 8
  x /= (uint32_t)C.heads;
  const int group = (int)(x % (uint32_t)P.groups), b = (int)(x / (uint32_t)P.groups);
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), m = lane & 15, g = lane >> 4;
  KvSeq q;
  if (!kv_seq(P.S, C.page, b, &q)) return;
  if (q.n == 0) return weigh_idle(P, q, b, h, group);
  const int d = C.d, rows = q.n * A.group, chunks = (int)cdiv(q.len, kChunk), step = P.groups * kFewWaves;
  const KvNibbles nib = kv_nibbles();
  const int64_t hb = kv_bytes<FMT>((int64_t)C.page * d);
  const int db = (int)kv_bytes<FMT>(d);
  const int pmask = C.page - 1, last = max(q.len - 1, 0), kr = m >> 2, ktok = m & 3;
  const int *table = P.S.table + (int64_t)b * P.S.table_ld;
  auto page_of = [&](int j) {
    const int pg = table[min(j, last) >> C.shift];
    return ONE ? __builtin_amdgcn_readfirstlane(pg) : pg;
  };
  auto there_at = [&](int pg) { return pg >= 0 && pg < C.pages; };
  auto head_at = [&](int pg) { return (int64_t)(there_at(pg) ? pg : 0) * C.heads + h; };
  int pk, pv;
  auto pages = [&](int c) {
    pv = page_of(c * kChunk + (ONE ? 0 : 16 * g));
    pk = ONE ? pv : page_of(c * kChunk + 16 * kr);
  };
  Codes16<FMT> kw[4][NP];
  float ks, old;  // 4-bit codes: scale of position m of run g; weight of that position
  bool mine;
  int64_t at;
  auto load_keys = [&](int c) {
    const uint8_t *kp = C.k + head_at(pk) * hb + ((c * kChunk + (ONE ? 0 : 16 * kr)) & pmask) * db;
#pragma unroll
    for (int st = 0; st < 4; ++st)
#pragma unroll
      for (int p = 0; p < NP; ++p)
        kw[st][p] = *reinterpret_cast<const Codes16<FMT> *>(
            kp + 4 * st * db + (uint32_t)(((ONE ? 16 * kr : 0) + ktok) * db + (int)kv_bytes<FMT>(min(64 * p + 16 * g, d - 16))));
  };
  auto load_rest = [&](int c) {
    const int j = c * kChunk + 16 * g + m;
    const bool there = there_at(pv);
    mine = there && j < q.len;
    at = head_at(pv) * C.page + (j & pmask);
    old = mine && P.decay != 0.0f && j < q.len - q.n ? P.weight[at] : 0.0f;
    if constexpr (FMT == KM_KV_I4) ks = mine ? C.ks[at] : 1.0f;
    else ks = there && c * kChunk + 16 * g < q.len ? C.ks[head_at(pv)] : 1.0f;
  };
  int c = group * kFewWaves + wave;
  if (c >= chunks) return;  // no barrier follows
  pages(c);
  load_keys(c);
  load_rest(c);
  if (c + step < chunks) pages(c + step);

  // this lane's row, its statistics and its span; rows behind the last and rows that do not count add nothing
  const int r = min(m, rows - 1);
  const RowAt row = row_at(A, C, q, h, r);
  int lo, hi;
  row_span(A, q, r, &lo, &hi);
  u32x4 raw[NP][2 * NS];
  const char *qp = static_cast<const char *>(A.q.p) + row.q * (2 * NS);
#pragma unroll
  for (int p = 0; p < NP; ++p)
#pragma unroll
    for (int i = 0; i < 2 * NS; ++i) raw[p][i] = reinterpret_cast<const u32x4 *>(qp + 2 * NS * min(64 * p + 16 * g, d - 16))[i];
  const float lse = A.lse[row.lse];
  const bool counts = m < rows && fabsf(lse) < INFINITY;
  const float nl = counts ? -lse * kLog2e : -INFINITY;
  f16x8 qf[NP][2][NS];
  float cs;
  {
    float top = 0.0f, f;
#pragma unroll
    for (int p = 0; p < NP; ++p) top = fmaxf(top, top16<NS>(raw[p], A.type));
    q_scale(max_groups(top), A.scale, &f, &cs);
#pragma unroll
    for (int p = 0; p < NP; ++p) {
      float v[16];
      values16<NS>(raw[p], A.type, v);
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        const float y = counts && 64 * p + 16 * g < d ? v[i] * f : 0.0f;  // rows that do not count may hold NaN
        const _Float16 y16 = (_Float16)y;
        qf[p][i / 8][0][place8<FMT>(i % 8)] = y16;
        if constexpr (NS == 2) qf[p][i / 8][1][place8<FMT>(i % 8)] = (_Float16)(y - (float)y16);
      }
    }
  }
  if (!counts) cs = 1.0f;

  for (; c < chunks; c += step) {
    const int j0 = c * kChunk;
    const bool more = c + step < chunks;
    f32x4 s[4];
#pragma unroll
    for (int st = 0; st < 4; ++st) {
      __builtin_amdgcn_sched_barrier(0);  // no more codes widened at a time than these products take
      s[st] = f32x4{0, 0, 0, 0};
#pragma unroll
      for (int p = 0; p < NP; ++p)
#pragma unroll
        for (int k = 0; k < 2; ++k) {
          const f16x8 kf = widen8<FMT>(kw[st][p], k, nib);
#pragma unroll
          for (int z = 0; z < NS; ++z) s[st] = mfma16(kf, qf[p][k][z], s[st]);
        }
    }
    if (more) load_keys(c + step);
    if (!__all(j0 >= lo && j0 + kChunk <= hi)) {
      int jg = j0 + 16 * g;
      asm volatile("" : "+v"(jg));  // a branch: few chunks need it, so nothing of it is kept in registers
#pragma unroll
      for (int e = 0; e < 16; ++e) {
        const int j = jg + e;
        if (j < lo || j >= hi) s[e / 4][e % 4] = -INFINITY;
      }
    }
    // a factor of 0 (a row of tiny queries) would make NaN of -inf
    const float ck = fmaxf(FMT == KM_KV_I4 ? cs : cs * ks, 0x1p-126f);
    float total = 0.0f;
    each<16>([&](auto n) {
      constexpr int e = n;
      float y = s[e / 4][e % 4];
      if constexpr (FMT == KM_KV_I4) y *= kv_row_bcast<e>(ks);
      y = sum_row(__builtin_amdgcn_exp2f(fmaf(y, ck, nl)));
      total = m == e ? y : total;
    });
    if (mine) P.weight[at] = fmaf(old, P.decay, total);
    if (more) {
      load_rest(c + step);
      if (c + 2 * step < chunks) pages(c + 2 * step);
    }
  }
}

// ---- many 16-bit rows ---------------------------------------------------------------------------------------------------
//
// A workgroup takes 256 positions, 64 to a wave, which stay in registers as the first operand of the 32 x 32 x 16 products, and
// the waves share tiles of 32 tokens of one query head, which pass through LDS (two buffers, a tile's loads a tile ahead).  The
// tiles of the rows that see the positions are split evenly over `splits` workgroups, whose sums kv_weigh_join_kernel adds up in order.
constexpr int kRowWaves = 4, kRowKeys = kRowWaves * kChunk, kRowTile = 32;

struct WeighRows {
  WeighArgs W;
  int splits;
  float *part;  // [n][heads][splits][groups * kRowKeys]
};

__device__ __forceinline__ bool weigh_split(const WeighRows &R, const KvSeq &q) {  // a longer one than was said is not split
  return R.splits > 1 && q.len <= R.W.groups * kRowKeys;
}

template <int FMT, int TYPE, int ND, bool ONE>
__global__ __launch_bounds__(64 * kRowWaves, ND <= 4 ? 2 : 1) void kv_weigh_rows_kernel(WeighRows R) {
  constexpr int T = 64 * kRowWaves, KS = 2 * ND, LD = 64 * ND + 16;  // bytes of a row in LDS, so that rows lie in different banks
  constexpr int NI = (ND + 1) / 2;                                   // 16-byte pieces of a tile to a thread
  __shared__ __align__(16) uint8_t qt[2][kRowTile * LD];
  __shared__ float stat[2][kRowTile];
  const WeighArgs &P = R.W;
  const KvCache &C = P.C;
  const KvAttend &A = P.A;
  uint32_t x = P.block0 + blockIdx.x;
  const int h = (int)(x % (uint32_t)C.heads);  // heads fastest: a head's workgroups share an XCD's L2 where they are a multiple of 8
  x /= (uint32_t)C.heads;
  // Neighbouring workgroups of an XCD go to its shader engines in turn, whatever these still have to do: splits, which are alike,
  // follow each other, then the sequences (sequences first, of 5340 and 3133 tokens: two of four engines had all of the longer one's,
  // 347 us).  The first positions, which most rows see, begin first.
  const int split = (int)(x % (uint32_t)R.splits);
  x /= (uint32_t)R.splits;
  const int b = (int)(x % (uint32_t)P.S.n), group0 = (int)(x / (uint32_t)P.S.n);
  KvSeq q;
  if (!kv_seq(P.S, C.page, b, &q)) return;
  if (q.n == 0 && split == 0) weigh_idle(P, q, b, h, group0);
  if (q.n == 0) return;
  const bool parts = weigh_split(R, q);
  if (!parts && split > 0) return;
  const int t = threadIdx.x, lane = t & 63, wave = __builtin_amdgcn_readfirstlane(t >> 6), m = lane & 31, g = lane >> 5;
  const int d = C.d, first = q.len - q.n;  // position of token 0
  const int64_t hb = kv_bytes<FMT>((int64_t)C.page * d);
  const int db = (int)kv_bytes<FMT>(d), pmask = C.page - 1, last = q.len - 1;
  const int *table = P.S.table + (int64_t)b * P.S.table_ld;
  auto page_of = [&](int j) {
    const int pg = table[min(j, last) >> C.shift];
    return ONE ? __builtin_amdgcn_readfirstlane(pg) : pg;
  };
  auto there_at = [&](int pg) { return pg >= 0 && pg < C.pages; };
  auto head_at = [&](int pg) { return (int64_t)(there_at(pg) ? pg : 0) * C.heads + h; };
  const KvNibbles nib = kv_nibbles();
  const int per = d / 8;  // pieces of a row
  int prow[NI];
  int64_t q_at[NI];  // from a tile's first token
#pragma unroll
  for (int i = 0; i < NI; ++i) {
    prow[i] = (t + i * T) / per;
    q_at[i] = prow[i] * A.q.row + 8 * (t + i * T - prow[i] * per);
  }

  for (int64_t gi = group0; gi * kRowKeys < q.len; gi += P.groups) {
    const int w0 = (int)gi * kRowKeys, j0 = w0 + wave * kChunk;
    const bool mine = j0 < q.len;
    // keys: row m of operand tt is position 32 tt + m
    f16x8 kf[2][KS];
    float ck[FMT == KM_KV_I4 ? 32 : 4];  // what a score is multiplied by
    if (mine) {
      const float f = A.scale * kLog2e;
#pragma unroll
      for (int tt = 0; tt < 2; ++tt) {
        const int j = j0 + 32 * tt + m, pg = page_of(ONE ? j0 : j);
        const uint8_t *kp = C.k + head_at(pg) * hb + (j & pmask) * db;
        float down = FMT == KM_KV_I4 || TYPE != KM_T_BF16 ? 1.0f : C.ks[head_at(pg)];
        down = weigh_down<FMT, TYPE>(f, down);
#pragma unroll
        for (int k = 0; k < KS; ++k) {
          const uint8_t *from = kp + (int)kv_bytes<FMT>(min(16 * k + 8 * g, d - 8));
          f16x8 y;
          if constexpr (FMT == KM_KV_I4) {
            y = kv_widen4x8(*reinterpret_cast<const uint32_t *>(from), nib);
            y = f16x8{y[0], y[2], y[4], y[6], y[1], y[3], y[5], y[7]};  // in the dims' order, as the queries lie
          } else {
            const u32x2 w = *reinterpret_cast<const u32x2 *>(from);
            y = kv_widen8<FMT>(w.x, w.y);
          }
          if (16 * k + 8 * g >= d) y = f16x8{0, 0, 0, 0, 0, 0, 0, 0};
          if constexpr (TYPE == KM_T_BF16) y = weigh_bf16(y, down);
          kf[tt][k] = y;
        }
      }
      if constexpr (FMT == KM_KV_I4) {
#pragma unroll
        for (int y = 0; y < 8; ++y) {  // positions 8 y + 4 g of the 64 and the next three: elements 4 y on
          const int j = j0 + 8 * y + 4 * g, pg = page_of(ONE ? j0 : j);
          const f32x4 ks = *reinterpret_cast<const f32x4 *>(C.ks + head_at(pg) * C.page + (j & pmask));
#pragma unroll
          for (int z = 0; z < 4; ++z) ck[4 * y + z] = there_at(pg) && j + z < q.len ? weigh_factor<FMT, TYPE>(f, ks[z]) : 1.0f;
        }
      } else {
#pragma unroll
        for (int y = 0; y < 4; ++y) {  // runs of 16
          const int j = j0 + 16 * y, pg = page_of(ONE ? j0 : j);
          ck[y] = there_at(pg) && j < q.len ? weigh_factor<FMT, TYPE>(f, C.ks[head_at(pg)]) : 1.0f;
        }
      }
    }
    // tiles of the tokens that see one of the positions: blocks [b0, b1) of 32 tokens, of one query head after the other
    int t0 = 0, t1 = q.n;
    if (A.causal) t0 = max(w0 - first, 0);
    if (A.window) t1 = (int)max((int64_t)0, min((int64_t)q.n, (int64_t)w0 + kRowKeys - 1 + A.window - first));
    const int b0 = t0 / kRowTile, b1 = max((t1 + kRowTile - 1) / kRowTile, b0), nb = b1 - b0;
    const int64_t tiles = (int64_t)nb * A.group, ns = parts ? R.splits : 1;
    const int z0 = (int)(tiles * split / ns), z1 = (int)(tiles * (split + 1) / ns);
    int lh = nb ? z0 / nb : 0, lb = b0 + z0 - lh * nb;  // head and block of the tile that is loaded next
    u32x4 raw[NI];
    float lse;  // of token t, in the first half of a wave
    auto load = [&] {
      const int64_t row = q.row0 + (int64_t)lb * kRowTile;
      const uint16_t *base = static_cast<const uint16_t *>(A.q.p) + row * A.q.row + (int64_t)(h * A.group + lh) * A.q.head;
      const int left = min(q.n - lb * kRowTile, kRowTile);
#pragma unroll
      for (int i = 0; i < NI; ++i) {
        const bool in = prow[i] < left;
        raw[i] = *reinterpret_cast<const u32x4 *>(base + (in ? q_at[i] : 0));
      }
      if (t < kRowTile) lse = t < left ? A.lse[(row + t) * C.heads * A.group + h * A.group + lh] : INFINITY;
      if (++lb == b1) {
        lb = b0;
        ++lh;
      }
    };
    auto store = [&](int z) {
#pragma unroll
      for (int i = 0; i < NI; ++i) {
        if (prow[i] >= kRowTile) continue;
        *reinterpret_cast<u32x4 *>(&qt[z & 1][prow[i] * LD + 16 * (t + i * T - prow[i] * per)]) = raw[i];
      }
      if (t < kRowTile) stat[z & 1][t] = fabsf(lse) < INFINITY ? -lse * kLog2e : -INFINITY;
    };
    float sum[32];
#pragma unroll
    for (int e = 0; e < 32; ++e) sum[e] = 0.0f;
    int cb = lb;  // block of the tile at hand
    if (z0 < z1) {
      load();
      store(z0);
      if (z0 + 1 < z1) load();
      __syncthreads();
    }
    for (int z = z0; z < z1; ++z) {
      if (z + 1 < z1) store(z + 1);
      if (z + 2 < z1) load();
      const int pos0 = first + cb * kRowTile;  // position of the tile's first token
      if (mine && (!A.causal || pos0 + kRowTile > j0) && (!A.window || (int64_t)pos0 < (int64_t)j0 + kChunk - 1 + A.window)) {
        f32x16v s[2];
#pragma unroll
        for (int tt = 0; tt < 2; ++tt)
#pragma unroll
          for (int i = 0; i < 16; ++i) s[tt][i] = 0.0f;
        const uint8_t *from = &qt[z & 1][m * LD];
#pragma unroll
        for (int k = 0; k < KS; ++k) {
          const f16x8 y = *reinterpret_cast<const f16x8 *>(from + 2 * min(16 * k + 8 * g, d - 8));
#pragma unroll
          for (int tt = 0; tt < 2; ++tt) {
            if constexpr (TYPE == KM_T_BF16)
              s[tt] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf16x8, kf[tt][k]), __builtin_bit_cast(bf16x8, y),
                                                              s[tt], 0, 0, 0);
            else
              s[tt] = mfma32(kf[tt][k], y, s[tt]);
          }
        }
        const float nl = stat[z & 1][m];
        if (__any(nl == -INFINITY)) {  // rows that do not count may hold NaN
#pragma unroll
          for (int e = 0; e < 32; ++e) s[e >> 4][e & 15] = nl == -INFINITY ? 0.0f : s[e >> 4][e & 15];
        }
        const int pos = pos0 + m;
        const int see0 = A.window ? max(pos + 1 - A.window, 0) : 0, see1 = A.causal ? max(pos + 1, 0) : q.len;
        if (!__all(j0 >= see0 && j0 + kChunk <= see1)) {
          int jg = j0 + 4 * g;
          asm volatile("" : "+v"(jg));  // a branch: few tiles need it, so nothing of it is kept in registers
#pragma unroll
          for (int e = 0; e < 32; ++e) {
            const int j = jg + 8 * (e >> 2) + (e & 3);
            if (j < see0 || j >= see1 || j >= q.len) s[e >> 4][e & 15] = -INFINITY;
          }
        }
#pragma unroll
        for (int e = 0; e < 32; ++e)
          sum[e] += __builtin_amdgcn_exp2f(fmaf(s[e >> 4][e & 15], ck[FMT == KM_KV_I4 ? e : e >> 3], nl));
      }
      if (++cb == b1) cb = b0;
      __syncthreads();
    }
    if (!mine) continue;
    // over the 32 tokens; lane m of a half then holds element m of its 32
    float total = 0.0f;
#pragma unroll
    for (int e = 0; e < 32; ++e) {
      float y = sum_row(sum[e]);
      y += __shfl_xor(y, 16);
      total = m == e ? y : total;
    }
    const int j = j0 + 8 * (m >> 2) + 4 * g + (m & 3), pg = page_of(ONE ? j0 : j);
    if (j >= q.len || !there_at(pg)) continue;
    if (parts) {
      R.part[(((int64_t)b * C.heads + h) * R.splits + split) * P.groups * kRowKeys + j] = total;
    } else {
      float *w = P.weight + head_at(pg) * C.page + (j & pmask);
      *w = fmaf(P.decay != 0.0f && j < first ? *w : 0.0f, P.decay, total);
    }
  }
}

__global__ __launch_bounds__(256) void kv_weigh_join_kernel(WeighRows R) {
  const WeighArgs &P = R.W;
  const KvCache &C = P.C;
  uint32_t x = P.block0 + blockIdx.x;
  const int gi = (int)(x % (uint32_t)P.groups);
  x /= (uint32_t)P.groups;
  const int h = (int)(x % (uint32_t)C.heads), b = (int)(x / (uint32_t)C.heads);
  KvSeq q;
  if (!kv_seq(P.S, C.page, b, &q) || q.n == 0 || !weigh_split(R, q)) return;
  const int j = gi * kRowKeys + threadIdx.x;
  if (j >= q.len) return;
  const int64_t pg = P.S.table[(int64_t)b * P.S.table_ld + (j >> C.shift)];
  if (pg < 0 || pg >= C.pages) return;
  const float *p = R.part + ((int64_t)b * C.heads + h) * R.splits * P.groups * kRowKeys + j;
  float total = 0.0f;
  for (int y = 0; y < R.splits; ++y) total += p[(int64_t)y * P.groups * kRowKeys];
  float *w = P.weight + (pg * C.heads + h) * C.page + (j & (C.page - 1));
  *w = fmaf(P.decay != 0.0f && j < q.len - q.n ? *w : 0.0f, P.decay, total);
}

// How a call is cut up.
enum WeighWay {
  kTokens,  // up to 16 rows to a cache head: kv_weigh_tokens_kernel
  kFew,     // each wave its own positions, all rows in turn
  kShare,   // fp32 rows: a workgroup's waves share 64 positions and take the rows in turn
  kRows     // 16-bit rows: kv_weigh_rows_kernel
};
struct WeighPlan {
  WeighWay way;
  int groups, splits;
};
// 32 heads of 128 on 8 unless said otherwise, codes in int8, bf16 rows:
//   kTokens or kFew: 16 sequences of 500 to 8192 tokens, one row each 19 us and 29, four rows 19 and 29
//   kFew or kRows: the same, 32 rows each (128 to a cache head) 60 us and 76, 64 rows 102 and 100; 64 of 500 to 4000, 64 rows 173 and 186, 128
//     rows 309 and 283; two of 3000 to 6000, 64 rows 21 and 23, 1000 rows 236 and 118; 4-bit codes 16 of 500 to 8192, 64 rows
//     101 and 110.  From 160 dims on kRows has one wave to a SIMD, and up to 192 kFew two, so that enough positions for all of the
//     card go through kFew: 16 of 500 to 8192, 500 rows of 160 dims 512 and 803, of 224 879 and 1149, of 256 1178 and 1180, 128 rows of 224 277 and
//     364, of 256 352 and 385 (4 bits 352 and 401); two of 3000 to 6000, 3000 rows of 192 dims 819 and 384, of 256 967 and 553, but 128 rows of
//     224 55 and 69.
//   kFew or kShare, fp32: 16 of 500 to 8192, 64 rows 170 us and 381, 200 rows 471 and 667; two of 3000 to 6000, 64 rows 36 and 56, 250 rows
//     119 and 118, 1000 rows 454 and 364; one of 2000, 32 rows 15 and 9, 64 rows 25 and 12
//   workgroups of kTokens, 512, 1024, 2048: 16 of 500 to 8192 22, 19, 19 us; one of 131071 27, 24, 26; 64 of 1 to 16384 (where
//     1024 are two to a head and 4096 eight) 163, 135, 125, with 4096 122
//   workgroups of kRows, 512, 1024, 1536, 2048: two prompts of 3133 and 5340 tokens 264, 230, 220, 224 us, without splits 422; pieces of 8
//     tiles at least, 16, 32: a prompt of 500 25, 32, 52
WeighPlan plan_weigh(const KvCache &C, const KvSeqs &S, const KvAttend &A) {
  WeighPlan p{kFew, 1, 1};
  const int64_t heads = (int64_t)S.n * C.heads, rows = (int64_t)S.max_rows * A.group;
  const int64_t alone = heads * cdiv(S.max_len, kChunk * kFewWaves);  // workgroups of kFew
  if (rows <= 16) p.way = kTokens;
  else if (A.type == KM_T_F32) p.way = rows >= 1024 || (rows > 64 && alone < 256) ? kShare : kFew;
  else p.way = rows >= 512 && S.max_rows >= kRowTile && (dim_tiles32(C.d) < 6 || alone < 1024) ? kRows : kFew;
  // Workgroups of a sequence's head: one for each of its pieces by the longest length that the caller knows, fewer where that is
  // more than 2^20 in all (a workgroup then takes several, as where a length is longer than was said).
  const int64_t pieces = cdiv(S.max_len, p.way == kShare ? kChunk : p.way == kRows ? kRowKeys : kChunk * kFewWaves);
  p.groups = (int)std::max<int64_t>(1, std::min(pieces, (1 << 20) / heads));
  // as many workgroups as run at a time, but not so few that lengths differ by whole workgroups
  if (p.way == kTokens) p.groups = (int)std::min<int64_t>(p.groups, std::max<int64_t>(8, cdiv(1024, heads)));
  // three times as many workgroups as run at a time, of eight tiles at least
  if (p.way == kRows)
    p.splits = (int)std::max<int64_t>(1, std::min(cdiv(1536, heads * p.groups), cdiv(S.max_rows, kRowTile) * A.group / 8));
  return p;
}

}  // namespace

int64_t kv_weigh_blocks(const KvCache &C, const KvSeqs &S, const KvAttend &A) {
  const WeighPlan p = plan_weigh(C, S, A);
  return (int64_t)S.n * C.heads * p.groups * p.splits;
}

size_t kv_weigh_scratch(const KvCache &C, const KvSeqs &S, const KvAttend &A) {
  const WeighPlan p = plan_weigh(C, S, A);
  return p.splits > 1 ? sizeof(float) * (size_t)S.n * C.heads * p.splits * p.groups * kRowKeys : 0;
}

km_status launch_kv_weigh(const KvCache &C, const KvSeqs &S, const KvAttend &A, float *weight, float decay, void *ws,
                          hipStream_t s) {
  const WeighPlan p = plan_weigh(C, S, A);
  const int waves = p.way == kShare ? kManyWaves : p.way == kRows ? kRowWaves : kFewWaves, threads = 64 * waves;
  const int step = p.way == kShare ? 16 * waves : 16;
  WeighRows R{{C, S, A, weight, decay, p.groups, step, step / A.group, step % A.group,
               (uint32_t)((((uint64_t)1 << 32) + A.group - 1) / A.group), 0},
              p.splits, static_cast<float *>(ws)};
  auto go = [&](auto *kernel, const auto &args, int64_t blocks) {
    const int64_t most = kv_piece(threads);
    auto a = args;
    for (int64_t b = 0; b < blocks; b += most) {
      if constexpr (std::is_same_v<decltype(a), WeighRows>) a.W.block0 = (uint32_t)b;
      else a.block0 = (uint32_t)b;
      kernel<<<dim3((unsigned)std::min(most, blocks - b)), threads, 0, s>>>(a);
    }
  };
  const int64_t blocks = kv_weigh_blocks(C, S, A);
#define KV_ONE(K, ...) C.page >= kChunk ? go(K<__VA_ARGS__, true>, KV_ARGS, blocks) : go(K<__VA_ARGS__, false>, KV_ARGS, blocks)
#define KV_ARGS R.W
#define KV_P(F, T, M)                                            \
  switch ((int)cdiv(C.d, 64)) {                                  \
    case 1: KV_ONE(kv_weigh_kernel, F, T, 1, M); break;          \
    case 2: KV_ONE(kv_weigh_kernel, F, T, 2, M); break;          \
    case 3: KV_ONE(kv_weigh_kernel, F, T, 3, M); break;          \
    default: KV_ONE(kv_weigh_kernel, F, T, 4, M);                \
  }
#define KV_S(F, NS)                                              \
  switch ((int)cdiv(C.d, 64)) {                                  \
    case 1: KV_ONE(kv_weigh_tokens_kernel, F, NS, 1); break;     \
    case 2: KV_ONE(kv_weigh_tokens_kernel, F, NS, 2); break;     \
    case 3: KV_ONE(kv_weigh_tokens_kernel, F, NS, 3); break;     \
    default: KV_ONE(kv_weigh_tokens_kernel, F, NS, 4);           \
  }
#define KV_R(F, T)                                               \
  switch (dim_tiles32(C.d)) {                                    \
    case 2: KV_ONE(kv_weigh_rows_kernel, F, T, 2); break;        \
    case 3: KV_ONE(kv_weigh_rows_kernel, F, T, 3); break;        \
    case 4: KV_ONE(kv_weigh_rows_kernel, F, T, 4); break;        \
    case 6: KV_ONE(kv_weigh_rows_kernel, F, T, 6); break;        \
    default: KV_ONE(kv_weigh_rows_kernel, F, T, 8);              \
  }
  auto of_format = [&](auto fmt) {
    constexpr int F = decltype(fmt)::value;
    if (p.way == kTokens) {
      if (A.type == KM_T_F32) KV_S(F, 2)
      else KV_S(F, 1)
    } else if (p.way == kShare) {
      KV_P(F, KM_T_F32, true)
    } else if (p.way == kFew) {
      if (A.type == KM_T_F32) KV_P(F, KM_T_F32, false)
      else if (A.type == KM_T_BF16) KV_P(F, KM_T_BF16, false)
      else KV_P(F, KM_T_F16, false)
    } else {
#undef KV_ARGS
#define KV_ARGS R
      if (A.type == KM_T_BF16) KV_R(F, KM_T_BF16)
      else KV_R(F, KM_T_F16)
    }
  };
  if (C.fmt == KM_KV_I8) of_format(std::integral_constant<int, KM_KV_I8>{});
  else if (C.fmt == KM_KV_F8) of_format(std::integral_constant<int, KM_KV_F8>{});
  else of_format(std::integral_constant<int, KM_KV_I4>{});
#undef KV_R
#undef KV_S
#undef KV_P
#undef KV_ARGS
#undef KV_ONE
  KMQ_LAUNCH_CHECK("kv_weigh");
  if (p.splits > 1) {
    go(kv_weigh_join_kernel, R, (int64_t)S.n * C.heads * p.groups);
    KMQ_LAUNCH_CHECK("kv_weigh");
  }
  return KM_OK;
}

}  // namespace kmq
