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
// after a power of two for each row.  The sums of a row's lane are added up over the sixteen lanes at the end.
//
// Few rows (one token of each sequence): each wave has its own positions; bound by the bytes of the keys.  Many rows: the
// workgroup's waves share their 64 positions and take the row tiles in turn, since there are few positions for the number of rows; bound by
// the exponentials (a quarter of the vector unit's rate) and the products.
#include "kv_attend.hpp"

namespace kmq {
namespace {

constexpr int kWeighWaves = 4;

struct WeighArgs {
  KvCache C;
  KvSeqs S;
  KvAttend A;  // q, type, group, scale, causal, window, lse
  float *weight;
  float decay;
  int groups;  // workgroups of a sequence's head
  int many;    // waves share their positions
  uint32_t block0;
};

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));

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

// TYPE: bf16 and fp16 rows as they are, fp32 rows in two halves (NS = 2)
template <int FMT, int TYPE, int NP, bool ONE>
__global__ __launch_bounds__(64 * kWeighWaves) void kv_weigh_kernel(WeighArgs P) {
  constexpr int NS = TYPE == KM_T_F32 ? 2 : 1;
  __shared__ float sh[kWeighWaves][kChunk];
  const KvCache &C = P.C;
  const KvAttend &A = P.A;
  uint32_t x = P.block0 + blockIdx.x;
  const int h = (int)(x % (uint32_t)C.heads);  // heads fastest: a head's workgroups share an XCD's L2 where they are a multiple of 8
  x /= (uint32_t)C.heads;
  const int b = (int)(x / (uint32_t)P.groups);
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), m = lane & 15, g = lane >> 4;
  const int group = (int)(x - (uint32_t)b * P.groups);
  KvSeq q;
  if (!kv_seq(P.S, C.page, b, &q) || q.n == 0) return;
  const int d = C.d, rows = q.n * A.group;
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
  // every wave's positions are behind the end at once (P.many), or no barrier follows
  for (int64_t c = P.many ? group : (int64_t)group * kWeighWaves + wave; c * kChunk < q.len;
       c += (int64_t)P.groups * (P.many ? 1 : kWeighWaves)) {
  const int j0 = (int)c * kChunk;
  // positions of this lane's scores: run g; the keys that it loads: run kr
  const int pv = page_of(j0 + (ONE ? 0 : 16 * g)), pk = ONE ? pv : page_of(j0 + 16 * kr);
  const int jm = j0 + 16 * g + m;  // the position whose weight this lane writes
  const bool there = there_at(pv), mine = there && jm < q.len;
  const int64_t at = head_at(pv) * C.page + (jm & pmask);
  const float old = mine && P.decay != 0.0f && jm < q.len - q.n ? P.weight[at] : 0.0f;

  // keys, dims past d are 0 in the queries
  f16x8 kf[4][NP][2];
  {
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
          kf[st][p][k] = widen8<FMT>(kw[st][p], k);
          if constexpr (FMT == KM_KV_I4) {  // in the dims' order, as the queries lie
            const f16x8 y = kf[st][p][k];
            kf[st][p][k] = f16x8{y[0], y[2], y[4], y[6], y[1], y[3], y[5], y[7]};
          }
          if constexpr (TYPE == KM_T_BF16) {
            typedef float f32x8 __attribute__((ext_vector_type(8)));
            kf[st][p][k] = __builtin_bit_cast(f16x8, __builtin_convertvector(__builtin_convertvector(kf[st][p][k], f32x8), bf16x8));
          }
        }
  }
  // what a score is multiplied by, for each of the lane's 16 positions; not 0, so that -infinity stays
  float ck[16];
  {
    const float f = A.scale * kLog2e;
    if constexpr (FMT == KM_KV_I4) {
      const float ks = mine ? C.ks[at] : 1.0f;
      each<16>([&](auto e) { ck[e] = fmaxf(f * kv_row_bcast<e>(ks), 0x1p-126f); });
    } else {
      const float ks = j0 + 16 * g < q.len && there ? C.ks[head_at(pv)] : 1.0f;
      ck[0] = fmaxf(f * ks, 0x1p-126f);
#pragma unroll
      for (int e = 1; e < 16; ++e) ck[e] = ck[0];
    }
  }

  // the rows that may see one of the positions
  const int first = q.len - q.n;  // position of row 0
  int t0 = 0, t1 = q.n;
  if (A.causal) t0 = max(j0 - first, 0);
  if (A.window) t1 = (int)max((int64_t)0, min((int64_t)q.n, (int64_t)j0 + kChunk - 1 + A.window - first));
  const int r1 = t1 * A.group;
  int r0 = (int)min((int64_t)t0 * A.group, (int64_t)rows) + (P.many ? 16 * wave : 0);
  const int step = P.many ? 16 * kWeighWaves : 16;

  float sum[16];
#pragma unroll
  for (int e = 0; e < 16; ++e) sum[e] = 0.0f;
  for (; r0 < r1; r0 += step) {
    const int r = min(r0 + m, rows - 1);
    const RowAt row = row_at(A, C, q, h, r);
    const float lse = r0 + m < r1 ? A.lse[row.lse] : INFINITY;
    const bool counts = fabsf(lse) < INFINITY;
    const float nl = counts ? -lse * kLog2e : -INFINITY;
    const char *qp = static_cast<const char *>(A.q.p) + row.q * (2 * NS);
    f16x8 qf[NP][2][NS];
    float c32 = 1.0f;
    if constexpr (NS == 1) {
#pragma unroll
      for (int p = 0; p < NP; ++p)
#pragma unroll
        for (int k = 0; k < 2; ++k) {
          u32x4 w = *reinterpret_cast<const u32x4 *>(qp + 2 * (min(64 * p + 16 * g, d - 16) + 8 * k));
          if (!counts || 64 * p + 16 * g >= d) w = u32x4{0, 0, 0, 0};  // rows that do not count may hold NaN
          qf[p][k][0] = __builtin_bit_cast(f16x8, w);
        }
    } else {
      float v[NP][16], top = 0.0f;
#pragma unroll
      for (int p = 0; p < NP; ++p) {
        u32x4 raw[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) raw[i] = reinterpret_cast<const u32x4 *>(qp + 4 * min(64 * p + 16 * g, d - 16))[i];
        values16<2>(raw, KM_T_F32, v[p]);
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          if (!counts || 64 * p + 16 * g >= d) v[p][i] = 0.0f;
          top = fmaxf(top, fabsf(v[p][i]));
        }
      }
      float f;
      q_scale(max_groups(top), 1.0f / kLog2e, &f, &c32);
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
    f32x4 s[4];
#pragma unroll
    for (int st = 0; st < 4; ++st) {
      s[st] = f32x4{0, 0, 0, 0};
#pragma unroll
      for (int p = 0; p < NP; ++p)
#pragma unroll
        for (int k = 0; k < 2; ++k)
#pragma unroll
          for (int z = 0; z < NS; ++z) {
            if constexpr (TYPE == KM_T_BF16)
              s[st] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, kf[st][p][k]),
                                                              __builtin_bit_cast(bf16x8, qf[p][k][z]), s[st], 0, 0, 0);
            else
              s[st] = mfma16(kf[st][p][k], qf[p][k][z], s[st]);
          }
    }
    if constexpr (NS == 2) {
#pragma unroll
      for (int e = 0; e < 16; ++e) s[e / 4][e % 4] *= c32;
    }
    int lo, hi;
    row_span(A, q, r, &lo, &hi);
    if (!__all(j0 >= lo && j0 + kChunk <= hi)) {
#pragma unroll
      for (int e = 0; e < 16; ++e) {
        const int j = j0 + 16 * g + e;
        if (j < lo || j >= hi) s[e / 4][e % 4] = -INFINITY;
      }
    }
#pragma unroll
    for (int e = 0; e < 16; ++e) sum[e] += __builtin_amdgcn_exp2f(fmaf(s[e / 4][e % 4], ck[e], nl));
  }

  float total = 0.0f;
#pragma unroll
  for (int e = 0; e < 16; ++e) {
    const float z = sum_row(sum[e]);
    total = m == e ? z : total;
  }
  if (P.many) {
    sh[wave][16 * g + m] = total;
    __syncthreads();
    total = 0.0f;
#pragma unroll
    for (int y = 0; y < kWeighWaves; ++y) total += sh[y][16 * g + m];
    __syncthreads();  // before the next positions' sums
  }
  if (mine && (!P.many || wave == 0)) P.weight[at] = fmaf(old, P.decay, total);
  }
}


// One wave per 64 positions and rows in turn, or all rows to each wave.
bool many_rows(const KvSeqs &S, const KvAttend &A) { return (int64_t)S.max_rows * A.group > 64; }

// Workgroups of a sequence's head: one for each of its pieces by the longest length that the caller knows, fewer where that is
// more than 2^20 in all (a workgroup then takes several, as where a length is longer than was said).
int groups_of(const KvCache &C, const KvSeqs &S, const KvAttend &A) {
  const int64_t pieces = cdiv(S.max_len, many_rows(S, A) ? kChunk : kChunk * kWeighWaves);
  return (int)std::max<int64_t>(1, std::min(pieces, (1 << 20) / ((int64_t)S.n * C.heads)));
}

}  // namespace

int64_t kv_weigh_blocks(const KvCache &C, const KvSeqs &S, const KvAttend &A) {
  return (int64_t)S.n * C.heads * groups_of(C, S, A);
}

km_status launch_kv_weigh(const KvCache &C, const KvSeqs &S, const KvAttend &A, float *weight, float decay, hipStream_t s) {
  WeighArgs P{C, S, A, weight, decay, groups_of(C, S, A), many_rows(S, A), 0};
  const int64_t blocks = kv_weigh_blocks(C, S, A), most = kv_piece(64 * kWeighWaves);
  auto go = [&](auto *kernel) {
    for (int64_t b = 0; b < blocks; b += most) {
      P.block0 = (uint32_t)b;
      kernel<<<dim3((unsigned)std::min(most, blocks - b)), 64 * kWeighWaves, 0, s>>>(P);
    }
  };
#define KV_P(F, T, N) \
  case N: \
    C.page >= kChunk ? go(kv_weigh_kernel<F, T, N, true>) : go(kv_weigh_kernel<F, T, N, false>); \
    break;
#define KV_T(F, T)                 \
  switch ((int)cdiv(C.d, 64)) {    \
    KV_P(F, T, 1)                  \
    KV_P(F, T, 2)                  \
    KV_P(F, T, 3)                  \
    KV_P(F, T, 4)                  \
  }
#define KV_F(F)                              \
  if (A.type == KM_T_F32) KV_T(F, KM_T_F32)  \
  else if (A.type == KM_T_BF16) KV_T(F, KM_T_BF16) \
  else KV_T(F, KM_T_F16)
  if (C.fmt == KM_KV_I8) {
    KV_F(KM_KV_I8)
  } else if (C.fmt == KM_KV_F8) {
    KV_F(KM_KV_F8)
  } else {
    KV_F(KM_KV_I4)
  }
#undef KV_F
#undef KV_T
#undef KV_P
  KMQ_LAUNCH_CHECK("kv_weigh");
  return KM_OK;
}

}  // namespace kmq
