// Attention over the 8-bit cache.
//
// o_i = sum_j p_ij v_j with p = softmax over the positions j that row i sees, in one pass over the cache with a running
// maximum: nothing of size rows x positions is written.  A code of either format is exact in fp16, so both products run
// on the fp16 matrix cores on the codes themselves and the page scales are applied outside:
//
//   t_ij = c_i ks_j <q'_i, kcode_j> + log2 vs_j   c_i = scale log2(e) 2^e_i, q'_i = q_i 2^-e_i in fp16
//   w_ij = 2^(t_ij - M_i + 15)                    M_i = the running maximum of t_ij
//   o_i  = (sum_j w_ij vcode_j) / l_i             l_i = sum_j w_ij / vs_j
//
// q'_i is the row times the power of two that brings its largest value to [2^13, 2^14): a 16-bit value stays exact down
// to 2^-27 of the row's largest.  Taking the maximum of the weight with its value scale keeps w in fp16's range for
// whatever scales the pages have; w is rounded to fp16 (2^-12 relative, down to 2^-29 of the largest weight) for
// the second product, l and every sum are fp32.  fp32 queries take two halves of q' and of w and twice the products.
//
// Layout.  One wave takes 64 positions and 16 rows at a time, without LDS.  The scores are computed transposed (keys are
// the matrix instruction's rows, queries its columns), and the keys of the four 16-key products are chosen so that lane
// group g = lane / 16 ends with the scores of positions 16 g .. 16 g + 15 of its query: exactly the operand of the second
// product, whose other operand is 16 contiguous bytes of one dim of the value page.  A page is 16 tokens or more, so
// a lane's 16 positions share one page and its scales.
#include "kv.hpp"

namespace kmq {
namespace {

constexpr int kChunk = 64;    // positions per step of a wave
constexpr float kLog2e = 1.44269504088896340736f;
constexpr float kUp = 15.0f;  // weights are at most 2^15

struct AttendArgs {
  KvCache C;
  KvSeqs S;
  KvAttend A;
  int rtiles;  // row tiles per sequence and head
  int splits;
  float *part;  // splits > 1: [tile][split] blocks of accumulators, then M and l
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

// Floats of one (tile, split) block of partial results: NT x 4 accumulators of 64 lanes per 16 rows, then M and l of
// the 16 rows.
__host__ __device__ constexpr int part_floats(int nt) { return nt * 256 + 32; }

// 16 values of a row as fp32, whatever their type (dims from c on; c + 16 <= d)
__device__ __forceinline__ void load_q16(const KvAttend &A, int64_t o, float *x) {
  if (A.type == KM_T_F32) kv_load<KM_T_F32, 16>(A.q.p, o, x);
  else if (A.type == KM_T_BF16) kv_load<KM_T_BF16, 16>(A.q.p, o, x);
  else kv_load<KM_T_F16, 16>(A.q.p, o, x);
}

__device__ __forceinline__ void store_o4(const KvAttend &A, int64_t o, const float *x) {
  if (A.type == KM_T_F32) kv_store<KM_T_F32, 4>(A.out.p, o, x);
  else if (A.type == KM_T_BF16) kv_store<KM_T_BF16, 4>(A.out.p, o, x);
  else kv_store<KM_T_F16, 4>(A.out.p, o, x);
}

// The power of two that takes a row whose largest magnitude is top to [2^13, 2^14), and what the products of the scaled
// row are multiplied by.  Exponents stay where the inverse is a normal number too.
__device__ __forceinline__ void q_scale(float top, float scale, float *f, float *c) {
  const int up = min(max(140 - (int)(__float_as_uint(top) >> 23), -126), 126);
  *f = __uint_as_float((uint32_t)(127 + up) << 23);
  *c = scale * kLog2e * __uint_as_float((uint32_t)(127 - up) << 23);
}

// The log of a row's sum of exp, its weights up to 2^up.  l = 0: the row saw no position.
__device__ __forceinline__ float log_sum(float M, float l, float up = kUp) {
  return l > 0.0f ? (M - up + __builtin_amdgcn_logf(l)) * 0.69314718055994530942f : (l == 0.0f ? -INFINITY : NAN);
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

template <int FMT, int NT, int RT, int NS>
__global__ __launch_bounds__(256) void kv_attend_kernel(AttendArgs P) {
  constexpr int NP = (NT + 3) / 4;  // groups of 64 dims
  __shared__ float sh_m[4][RT][16], sh_l[4][RT][16];
  __shared__ f32x4 sh_o[2][RT * NT][64];
  const KvCache &C = P.C;
  const KvAttend &A = P.A;
  int64_t x = blockIdx.x;
  const int split = (int)(x % P.splits);
  x /= P.splits;
  const int64_t tile = x;
  const int rt = (int)(x % P.rtiles);
  x /= P.rtiles;
  const int h = (int)(x % C.heads);
  const int b = (int)(x / C.heads);
  KvSeq q;
  if (!kv_seq(P.S, C.page, b, &q)) return;
  const int rows = q.n * A.group, r0 = rt * 16 * RT;
  if (r0 >= rows) return;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, m = lane & 15, g = lane >> 4;
  const int d = C.d;

  // the rows of this lane (rows past the last repeat it and are not stored), their scale and their spans
  f16x8 qf[RT][NP][2][NS];
  float cs[RT];
  int lo[RT], hi[RT];
#pragma unroll
  for (int u = 0; u < RT; ++u) {
    const int r = min(r0 + 16 * u + m, rows - 1);
    row_span(A, q, r, &lo[u], &hi[u]);
    const int64_t at = row_at(A, C, q, h, r).q;
    float v[NP][16];
    float top = 0.0f;
#pragma unroll
    for (int p = 0; p < NP; ++p) {
      const int c = 64 * p + 16 * g;
      if (c < d) {
        load_q16(A, at + c, v[p]);
      } else {
#pragma unroll
        for (int i = 0; i < 16; ++i) v[p][i] = 0.0f;
      }
#pragma unroll
      for (int i = 0; i < 16; ++i) top = fmaxf(top, fabsf(v[p][i]));
    }
    top = max_groups(top);
    float f;
    q_scale(top, A.scale, &f, &cs[u]);
#pragma unroll
    for (int p = 0; p < NP; ++p)
#pragma unroll
      for (int k = 0; k < 2; ++k)
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const float y = v[p][8 * k + i] * f;
          const _Float16 hi16 = (_Float16)y;
          qf[u][p][k][0][i] = hi16;
          if constexpr (NS == 2) qf[u][p][k][1][i] = (_Float16)(y - (float)hi16);
        }
  }
  // the tile's positions: from the first row's first to the last row's last
  int jlo, jhi, any;
  row_span(A, q, r0, &jlo, &any);
  row_span(A, q, min(r0 + 16 * RT, rows) - 1, &any, &jhi);
  const int c0 = jlo / kChunk, c1 = jhi > jlo ? (int)cdiv(jhi, kChunk) : c0;
  const int per = (c1 - c0 + P.splits - 1) / P.splits;
  const int cb = c0 + split * per, ce = min(cb + per, c1);

  f32x4 acc[RT][NT];
  float M[RT], l[RT];
#pragma unroll
  for (int u = 0; u < RT; ++u) {
    M[u] = -INFINITY;
    l[u] = 0.0f;
#pragma unroll
    for (int n = 0; n < NT; ++n) acc[u][n] = f32x4{0, 0, 0, 0};
  }

  const int64_t hb = (int64_t)C.page * d;  // bytes of a page's head
  const int pmask = C.page - 1;
  const int *table = P.S.table + (int64_t)b * P.S.table_ld;
  const int kr = m >> 2;                 // this lane's key rows lie in 16-token run kr, its values in run g
  const int ktok = m & 3;
  for (int c = cb + wave; c < ce; c += 4) {
    const int j0 = c * kChunk;
    // pages of the runs: past the sequence's end or outside the cache, page 0 is read and nothing of it counts
    const int tk = j0 + 16 * kr, tv = j0 + 16 * g;
    int64_t pk = tk < q.len ? table[tk >> C.shift] : 0;
    int64_t pv = tv < q.len ? table[tv >> C.shift] : -1;
    pk = pk >= 0 && pk < C.pages ? pk : 0;
    const bool there = pv >= 0 && pv < C.pages;
    pv = there ? pv : 0;
    const uint8_t *kp = C.k + (pk * C.heads + h) * hb + (int64_t)((tk & pmask) + ktok) * d;
    const uint8_t *vp = C.v + (pv * C.heads + h) * hb + (tv & pmask);
    const float ks = there ? C.ks[pv * C.heads + h] : 1.0f;
    const float vs = there ? C.vs[pv * C.heads + h] : 1.0f;

    u32x4 kw[4][NP];
#pragma unroll
    for (int st = 0; st < 4; ++st)
#pragma unroll
      for (int p = 0; p < NP; ++p)
        kw[st][p] = *reinterpret_cast<const u32x4 *>(kp + 4 * st * d + min(64 * p + 16 * g, d - 16));
    u32x4 vw[NT];
#pragma unroll
    for (int n = 0; n < NT; ++n)
      vw[n] = *reinterpret_cast<const u32x4 *>(vp + (int64_t)min(16 * n + m, d - 1) * C.page);

    f32x4 s[RT][4];
#pragma unroll
    for (int st = 0; st < 4; ++st) {
#pragma unroll
      for (int u = 0; u < RT; ++u) s[u][st] = f32x4{0, 0, 0, 0};
#pragma unroll
      for (int p = 0; p < NP; ++p)
#pragma unroll
        for (int k = 0; k < 2; ++k) {
          const f16x8 kf = kv_widen8<FMT>(kw[st][p][2 * k], kw[st][p][2 * k + 1]);
#pragma unroll
          for (int u = 0; u < RT; ++u)
#pragma unroll
            for (int z = 0; z < NS; ++z) s[u][st] = mfma16(kf, qf[u][p][k][z], s[u][st]);
        }
    }

    const float lv = __builtin_amdgcn_logf(vs), inv = 1.0f / vs;
    f16x8 w[RT][2][NS];
#pragma unroll
    for (int u = 0; u < RT; ++u) {
      const bool whole = __all(there && j0 >= lo[u] && j0 + kChunk <= hi[u]);
      if (!whole) {
#pragma unroll
        for (int st = 0; st < 4; ++st)
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const int j = tv + 4 * st + i;
            if (!there || j < lo[u] || j >= hi[u]) s[u][st][i] = -INFINITY;
          }
      }
      float top = -INFINITY;
#pragma unroll
      for (int st = 0; st < 4; ++st)
#pragma unroll
        for (int i = 0; i < 4; ++i) top = fmaxf(top, s[u][st][i]);
      const float ck = cs[u] * ks;
      const float t = top == -INFINITY ? -INFINITY : fmaf(top, ck, lv);
      const float Mn = fmaxf(M[u], max_groups(t));
      if (__any(Mn > M[u])) {
        const float al = Mn == -INFINITY ? 1.0f : __builtin_amdgcn_exp2f(M[u] - Mn);
        l[u] *= al;
#pragma unroll
        for (int n = 0; n < NT; ++n) acc[u][n] *= al;
        M[u] = Mn;
      }
      const float base = lv - (Mn == -INFINITY ? 0.0f : Mn) + kUp;
      float sum = 0.0f;
#pragma unroll
      for (int st = 0; st < 4; ++st)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          float y = __builtin_amdgcn_exp2f(fmaf(s[u][st][i], ck, base));
          if (!whole && s[u][st][i] == -INFINITY) y = 0.0f;
          sum += y;
          const _Float16 y16 = (_Float16)y;
          w[u][st / 2][0][4 * (st % 2) + i] = y16;
          if constexpr (NS == 2) w[u][st / 2][1][4 * (st % 2) + i] = (_Float16)(y - (float)y16);
        }
      l[u] = fmaf(sum, inv, l[u]);
    }
    if constexpr (FMT == KM_KV_F8) {  // codes past the end may be NaN, which no weight of 0 takes out
      if (j0 + kChunk > q.len || !__all(there)) {
        const int left = there ? q.len - tv : 0;
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
    for (int n = 0; n < NT; ++n)
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        const f16x8 vf = kv_widen8<FMT>(vw[n][2 * k], vw[n][2 * k + 1]);
#pragma unroll
        for (int u = 0; u < RT; ++u)
#pragma unroll
          for (int z = 0; z < NS; ++z) acc[u][n] = mfma16(vf, w[u][k][z], acc[u][n]);
      }
  }

  // the four waves' results: weights of a common maximum, then sums over the waves
#pragma unroll
  for (int u = 0; u < RT; ++u) {
    l[u] = sum_groups(l[u]);
    if (l[u] != l[u]) M[u] = INFINITY;  // the maximum does not see NaN: the row's results are NaN from here
    if (g == 0) {
      sh_m[wave][u][m] = M[u];
      sh_l[wave][u][m] = l[u];
    }
  }
  __syncthreads();
#pragma unroll
  for (int u = 0; u < RT; ++u) {
    const float Mx = fmaxf(fmaxf(sh_m[0][u][m], sh_m[1][u][m]), fmaxf(sh_m[2][u][m], sh_m[3][u][m]));
    float sum = 0.0f;
#pragma unroll
    for (int y = 0; y < 4; ++y) {
      const float My = sh_m[y][u][m];
      // a wave whose maximum is -inf has nothing; NaN stays NaN
      sum += My == -INFINITY ? 0.0f : sh_l[y][u][m] * __builtin_amdgcn_exp2f(My - Mx);
    }
    const float al = M[u] == -INFINITY ? 0.0f : __builtin_amdgcn_exp2f(M[u] - Mx);
#pragma unroll
    for (int n = 0; n < NT; ++n) acc[u][n] *= al;
    M[u] = Mx;
    l[u] = sum;
  }
  if (wave & 1) {
#pragma unroll
    for (int u = 0; u < RT; ++u)
#pragma unroll
      for (int n = 0; n < NT; ++n) sh_o[wave >> 1][u * NT + n][lane] = acc[u][n];
  }
  __syncthreads();
  if (!(wave & 1)) {
#pragma unroll
    for (int u = 0; u < RT; ++u)
#pragma unroll
      for (int n = 0; n < NT; ++n) acc[u][n] += sh_o[wave >> 1][u * NT + n][lane];
  }
  __syncthreads();
  if (wave == 2) {
#pragma unroll
    for (int u = 0; u < RT; ++u)
#pragma unroll
      for (int n = 0; n < NT; ++n) sh_o[0][u * NT + n][lane] = acc[u][n];
  }
  __syncthreads();
  if (wave) return;
#pragma unroll
  for (int u = 0; u < RT; ++u) {
    const int r = r0 + 16 * u + m;
    if (P.splits > 1) {
      float *o = P.part + ((tile * P.splits + split) * RT + u) * part_floats(NT);
#pragma unroll
      for (int n = 0; n < NT; ++n)
        *reinterpret_cast<f32x4 *>(o + (n * 64 + lane) * 4) = acc[u][n] + sh_o[0][u * NT + n][lane];
      if (g == 0) {
        o[NT * 256 + m] = M[u];
        o[NT * 256 + 16 + m] = l[u];
      }
      continue;
    }
    if (r >= rows) continue;
    const RowAt at = row_at(A, C, q, h, r);
    const float inv = l[u] == 0.0f ? 0.0f : 1.0f / l[u];
#pragma unroll
    for (int n = 0; n < NT; ++n) {
      const int c = 16 * n + 4 * g;
      const f32x4 v = (acc[u][n] + sh_o[0][u * NT + n][lane]) * inv;
      const float y[4] = {v.x, v.y, v.z, v.w};
      if (c < d) store_o4(A, at.o + c, y);
    }
    if (A.lse && g == 0) A.lse[at.lse] = log_sum(M[u], l[u]);
  }
}

// Joins the splits of a tile of 16 rows: one wave per four accumulators of a lane.
template <int NT>
__global__ __launch_bounds__(64) void kv_join_kernel(AttendArgs P, int rt16) {
  const KvCache &C = P.C;
  const KvAttend &A = P.A;
  const int n = blockIdx.x % NT;
  int64_t x = blockIdx.x / NT;
  const int u = (int)(x % rt16);
  x /= rt16;
  const int64_t tile = x;
  const int rt = (int)(x % P.rtiles);
  x /= P.rtiles;
  const int h = (int)(x % C.heads);
  const int b = (int)(x / C.heads);
  KvSeq q;
  if (!kv_seq(P.S, C.page, b, &q)) return;
  const int rows = q.n * A.group, r0 = (rt * rt16 + u) * 16;
  if (r0 >= rows) return;
  const int lane = threadIdx.x, m = lane & 15, g = lane >> 4;
  const float *base = P.part + (tile * P.splits * rt16 + u) * part_floats(NT);
  const int64_t step = (int64_t)rt16 * part_floats(NT);
  float Mx = -INFINITY;
  for (int y = 0; y < P.splits; ++y) Mx = fmaxf(Mx, base[y * step + NT * 256 + m]);
  float l = 0.0f;
  f32x4 o = {0, 0, 0, 0};
  for (int y = 0; y < P.splits; ++y) {
    const float *p = base + y * step;
    const float My = p[NT * 256 + m];
    if (My == -INFINITY) continue;
    const float al = __builtin_amdgcn_exp2f(My - Mx);
    l += p[NT * 256 + 16 + m] * al;
    o += *reinterpret_cast<const f32x4 *>(p + (n * 64 + lane) * 4) * al;
  }
  const int r = r0 + m;
  if (r >= rows) return;
  const RowAt at = row_at(A, C, q, h, r);
  const float inv = l == 0.0f ? 0.0f : 1.0f / l;
  o *= inv;
  const float y[4] = {o.x, o.y, o.z, o.w};
  const int c = 16 * n + 4 * g;
  if (c < C.d) store_o4(A, at.o + c, y);
  if (A.lse && n == 0 && g == 0) A.lse[at.lse] = log_sum(Mx, l);
}

// ---- many rows: tiles of 64 positions shared by a workgroup through LDS ------------------------------------------------
//
// A wave takes 32 RC rows and the 32 x 32 x 16 products; the four waves of a workgroup share each tile of 64 positions, whose
// codes are widened to fp16 once and laid out in LDS.  As above the scores are computed transposed, with the keys'
// order chosen such that a lane ends with 8 consecutive positions of its row in consecutive registers: row m of a 32-key
// operand holds position m with bits 2 and 3 exchanged.  The running maximum moves only when a tile's exceeds it by
// more than kSlack: until then weights just grow, within fp16's range.
//
// A wave has a SIMD's registers to itself, so the matrix cores and the vector unit overlap inside it: the products of the
// next tile's scores are issued with this tile's exponentials, and the widening of later tiles with the second products.
// Keys therefore run one tile ahead of values in LDS (two buffers each, one barrier per tile), and codes are loaded one tile
// before they are widened.

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

// Floats of one (32 rows, split) block of partial results.
__host__ __device__ constexpr int part32_floats(int nd) { return nd * 1024 + 64; }

constexpr int kWaves = 4;  // of this kernel

template <int FMT, int ND, int RC, bool ONE>
__global__ __launch_bounds__(64 * kWaves, ND <= 4 ? 2 : 1) void kv_prompt_kernel(AttendArgs P) {
  constexpr int DP = 32 * ND, T = 64 * kWaves;
  constexpr int KLD = DP + 8, VLD = kChunk + 8;  // halves; 16 bytes more than the row: rows start in different banks
  constexpr int PC = DP / 16;                    // 16-byte pieces of a key
  constexpr int KN = kChunk * PC, VN = DP * 4;   // pieces of a tile
  constexpr int KP = (KN + T - 1) / T, VP = (VN + T - 1) / T;
  __shared__ __align__(16) _Float16 kt[2][kChunk * KLD], vt[2][DP * VLD];
  constexpr int NR = ONE ? 1 : 4;  // pages that a tile may lie in: its one, or one for each run of 16 positions
  // of these: key scale, log2 of the value scale and its inverse, 1 if the page is there
  __shared__ float4 sc[2][4];
  const KvCache &C = P.C;
  const KvAttend &A = P.A;
  // heads fastest: a head's workgroups share an XCD's L2 where their number is a multiple of 8; last rows (the
  // most positions) first
  int64_t x = blockIdx.x;
  const int64_t bh = x % ((int64_t)P.S.n * C.heads);
  x /= (int64_t)P.S.n * C.heads;
  const int split = (int)(x % P.splits);
  const int rt = P.rtiles - 1 - (int)(x / P.splits);
  const int h = (int)(bh % C.heads);
  const int b = (int)(bh / C.heads);
  KvSeq q;
  if (!kv_seq(P.S, C.page, b, &q)) return;
  const int rows = q.n * A.group, r0 = rt * 32 * RC * kWaves;
  if (r0 >= rows) return;
  const int t = threadIdx.x, lane = t & 63, wave = t >> 6, m = lane & 31, g = lane >> 5;
  const int d = C.d;
  const int rw = r0 + 32 * RC * wave;  // this wave's first row

  f16x8 qf[RC][2 * ND];
  float cs[RC];
  int lo[RC], hi[RC];
#pragma unroll
  for (int u = 0; u < RC; ++u) {
    const int r = min(rw + 32 * u + m, rows - 1);
    row_span(A, q, r, &lo[u], &hi[u]);
    const int64_t at = row_at(A, C, q, h, r).q;
    float top = 0.0f;
    float v[2 * ND][8];
#pragma unroll
    for (int k = 0; k < 2 * ND; ++k) {
      const int c = 16 * k + 8 * g;
      if (c < d) {
        if (A.type == KM_T_BF16) kv_load<KM_T_BF16, 8>(A.q.p, at + c, v[k]);
        else kv_load<KM_T_F16, 8>(A.q.p, at + c, v[k]);
      } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[k][i] = 0.0f;
      }
#pragma unroll
      for (int i = 0; i < 8; ++i) top = fmaxf(top, fabsf(v[k][i]));
    }
    float f;
    q_scale(max_halves(top), A.scale, &f, &cs[u]);
#pragma unroll
    for (int k = 0; k < 2 * ND; ++k)
#pragma unroll
      for (int i = 0; i < 8; ++i) qf[u][k][i] = (_Float16)(v[k][i] * f);
  }
  // tiles of the workgroup's rows, and of this wave's
  int jlo, jhi, any;
  row_span(A, q, r0, &jlo, &any);
  row_span(A, q, min(r0 + 32 * RC * kWaves, rows) - 1, &any, &jhi);
  const int c0 = jlo / kChunk, c1 = jhi > jlo ? (int)cdiv(jhi, kChunk) : c0;
  const int per = (c1 - c0 + P.splits - 1) / P.splits;
  const int cb = c0 + split * per, ce = min(cb + per, c1);
  row_span(A, q, min(rw, rows - 1), &jlo, &any);
  row_span(A, q, min(rw + 32 * RC, rows) - 1, &any, &jhi);
  const int wb = max(cb, jlo / kChunk), we = rw < rows ? min(ce, (int)cdiv(jhi, kChunk)) : cb;

  f32x16v acc[RC][ND];
  float M[RC], l[RC];
#pragma unroll
  for (int u = 0; u < RC; ++u) {
    M[u] = -INFINITY;
    l[u] = 0.0f;
#pragma unroll
    for (int n = 0; n < ND; ++n)
#pragma unroll
      for (int i = 0; i < 16; ++i) acc[u][n][i] = 0.0f;
  }

  const int64_t hb = (int64_t)C.page * d;
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
  int kpg[ONE ? 1 : KP], vpg;  // pages of the codes that are loaded next
  u32x4 kc[KP], vc[VP];
  float2 rsc;
  bool rthere;
  auto key_pages = [&](int c) {
#pragma unroll
    for (int i = 0; i < (ONE ? 1 : KP); ++i) kpg[i] = page_of(c * kChunk + (ONE ? 0 : (t + i * T) / PC));
  };
  auto value_page = [&](int c) { vpg = page_of(c * kChunk + (ONE ? 0 : 16 * run)); };
  auto load_keys = [&](int c) {
    if constexpr (ONE) {
      const uint8_t *kp = C.k + page_at(kpg[0]) * hb + ((c * kChunk) & pmask) * d;
#pragma unroll
      for (int i = 0; i < KP; ++i) {
        const int p = min(t + i * T, KN - 1);
        kc[i] = *reinterpret_cast<const u32x4 *>(kp + (uint32_t)(p / PC * d + min(16 * (p % PC), d - 16)));
      }
    } else {
#pragma unroll
      for (int i = 0; i < KP; ++i) {
        const int p = min(t + i * T, KN - 1), tok = p / PC, cc = min(16 * (p % PC), d - 16);
        kc[i] = *reinterpret_cast<const u32x4 *>(C.k + page_at(kpg[i]) * hb + ((c * kChunk + tok) & pmask) * d + cc);
      }
    }
  };
  auto load_values = [&](int c) {
    const int j0 = c * kChunk + (ONE ? 0 : 16 * run);
    rthere = there_at(vpg, j0);
    const int64_t at = page_at(vpg);
    const uint8_t *vp = C.v + at * hb + (j0 & pmask);
#pragma unroll
    for (int i = 0; i < VP; ++i)
      vc[i] = *reinterpret_cast<const u32x4 *>(
          vp + (uint32_t)(min((t >> 2) + i * (T / 4), d - 1) * C.page + (ONE ? 16 * run : 0)));
    rsc = float2{C.ks[at], C.vs[at]};
  };
  auto store_key = [&](int c, int i) {
    const int p = t + i * T;
    if (KN % T != 0 && p >= KN) return;
    f16x8 *o = reinterpret_cast<f16x8 *>(&kt[c & 1][p / PC * KLD + 16 * (p % PC)]);
    o[0] = kv_widen8<FMT>(kc[i].x, kc[i].y);
    o[1] = kv_widen8<FMT>(kc[i].z, kc[i].w);
  };
  auto store_keys = [&](int c) {
#pragma unroll
    for (int i = 0; i < KP; ++i) store_key(c, i);
  };
  auto store_value = [&](int c, int i) {
    if (VN % T != 0 && t + i * T >= VN) return;
    f16x8 *o = reinterpret_cast<f16x8 *>(&vt[c & 1][((t >> 2) + i * (T / 4)) * VLD + 16 * run]);
    o[0] = kv_widen8<FMT>(vc[i].x, vc[i].y);
    o[1] = kv_widen8<FMT>(vc[i].z, vc[i].w);
  };
  auto store_values = [&](int c) {
#pragma unroll
    for (int i = 0; i < VP; ++i) store_value(c, i);
  };
  // codes past the end may be NaN, which no weight of 0 takes out
  auto clear_values = [&](int c) {
    if constexpr (FMT == KM_KV_F8) {
      const int left = rthere ? q.len - c * kChunk - 16 * run : 0;
      if (left < 16) {
        asm volatile("");  // a branch: rarely taken
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
    if (t < 4)
      sc[c & 1][t] = rthere ? float4{rsc.x, __builtin_amdgcn_logf(rsc.y), 1.0f / rsc.y, 1.0f}
                            : float4{1.0f, 0.0f, 1.0f, 0.0f};
  };
  const int krow = ((m & 4) << 1) | ((m & 8) >> 1) | (m & 19);  // bits 2 and 3 exchanged
  // operands of step k: keys of 32 positions at 16 dims, values of 32 dims at 16 positions
  constexpr int KS = 4 * ND;
  auto key_at = [&](int c, int k) {
    return *reinterpret_cast<const f16x8 *>(&kt[c & 1][(32 * (k / (2 * ND)) + krow) * KLD + 16 * (k % (2 * ND)) + 8 * g]);
  };
  auto value_at = [&](int c, int k) {
    return *reinterpret_cast<const f16x8 *>(&vt[c & 1][(32 * (k % ND) + m) * VLD + 16 * (k / ND) + 8 * g]);
  };
  f32x16v s[2][RC];
  auto scores = [&](int c, int tt) {  // of 32 positions
    f32x16v o[RC];
#pragma unroll
    for (int u = 0; u < RC; ++u)
#pragma unroll
      for (int i = 0; i < 16; ++i) o[u][i] = 0.0f;
#pragma unroll
    for (int k = 0; k < 2 * ND; ++k) {
      const f16x8 a = *reinterpret_cast<const f16x8 *>(&kt[c & 1][(32 * tt + krow) * KLD + 16 * k + 8 * g]);
#pragma unroll
      for (int u = 0; u < RC; ++u) o[u] = mfma32(a, qf[u][k], o[u]);
    }
#pragma unroll
    for (int u = 0; u < RC; ++u) s[tt][u] = o[u];
  };

  if (cb < ce) {
    key_pages(cb);
    value_page(cb);
    load_keys(cb);
    load_values(cb);
    store_keys(cb);
    clear_values(cb);
    store_values(cb);
    store_scales(cb);
    key_pages(cb + 1);
    load_keys(cb + 1);
    store_keys(cb + 1);
    key_pages(cb + 2);
    value_page(cb + 1);
    load_keys(cb + 2);
    load_values(cb + 1);
    key_pages(cb + 3);
    value_page(cb + 2);
  }
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
      f16x8 ring[4];
#pragma unroll
      for (int k = 0; k < 4; ++k) ring[k] = key_at(c + 1, k);
#pragma unroll
      for (int y = 0; y < NR; ++y) {
        const float4 z = sc[c & 1][y];
        ks[y] = z.x;
        lv[y] = z.y;
        inv[y] = z.z;
        there = there && z.w != 0.0f;
      }
      float ck[RC][NR], base[RC][NR], sum[RC][4];
#pragma unroll
      for (int u = 0; u < RC; ++u) {
        if (!__all(there && j0 >= lo[u] && j0 + kChunk <= hi[u])) {
          asm volatile("");  // a branch: few tiles need it
#pragma unroll
          for (int tt = 0; tt < 2; ++tt)
#pragma unroll
            for (int i = 0; i < 16; ++i) {
              const int j = j0 + 32 * tt + 16 * (i >> 3) + 8 * g + (i & 7);
              if (j < lo[u] || j >= hi[u] || sc[c & 1][ONE ? 0 : 2 * tt + (i >> 3)].w == 0.0f) s[tt][u][i] = -INFINITY;
            }
        }
        float Mt = -INFINITY;
#pragma unroll
        for (int y = 0; y < NR; ++y) {
          constexpr int E = 32 / NR;
          float top = -INFINITY;
#pragma unroll
          for (int i = E * y; i < E * (y + 1); ++i) top = fmaxf(top, s[i >> 4][u][i & 15]);
          // a factor of 0 (a row of tiny queries) would make NaN of -inf
          ck[u][y] = fmaxf(cs[u] * ks[y], 0x1p-126f);
          Mt = fmaxf(Mt, fmaf(top, ck[u][y], lv[y]));
        }
        Mt = max_halves(Mt);
        if (__any(Mt > M[u] + kSlack)) {
          const float Mn = fmaxf(M[u], Mt);
          const float al = Mn == -INFINITY ? 1.0f : __builtin_amdgcn_exp2f(M[u] - Mn);
          l[u] *= al;
#pragma unroll
          for (int n = 0; n < ND; ++n) acc[u][n] *= al;
          M[u] = Mn;
        }
        const float up = kUp32 - (M[u] == -INFINITY ? 0.0f : M[u]);
#pragma unroll
        for (int y = 0; y < NR; ++y) base[u][y] = lv[y] + up;
      }
      // Steps of one product (per 32 rows) each, in this order: the operand of four steps ahead is read, the product is
      // issued, and what the vector unit does meanwhile follows.  First the scores of the next tile and this tile's
      // exponentials, 16 registers of scores at a time (the next tile's replace them), then the second products
      // and the widening of later tiles.
      f16x8 w[RC][4];
      f32x16v o[RC];
#pragma unroll
      for (int k = 0; k < KS; ++k) {
        const int tt = k / (2 * ND), kk = k % (2 * ND);
        __builtin_amdgcn_sched_barrier(0);
        const f16x8 a = ring[k % 4];
        ring[k % 4] = k + 4 < KS ? key_at(c + 1, k + 4) : value_at(c, k + 4 - KS);
        if (kk == 0) {
#pragma unroll
          for (int u = 0; u < RC; ++u)
#pragma unroll
            for (int i = 0; i < 16; ++i) o[u][i] = 0.0f;
        }
#pragma unroll
        for (int u = 0; u < RC; ++u) o[u] = mfma32(a, qf[u][kk], o[u]);
        // elements [e0, e1) of 16
        const int e0 = kk * 16 / (2 * ND), e1 = (kk + 1) * 16 / (2 * ND);
#pragma unroll
        for (int u = 0; u < RC; ++u) {
#pragma unroll
          for (int i = e0; i < e1; ++i) {
            const int y = 2 * tt + (i >> 3);
            const float e = __builtin_amdgcn_exp2f(fmaf(s[tt][u][i], ck[u][y % NR], base[u][y % NR]));
            sum[u][y] = (i & 7) ? sum[u][y] + e : e;
            w[u][y][i & 7] = (_Float16)e;
          }
        }
        if (kk == 2 * ND - 1) {
#pragma unroll
          for (int u = 0; u < RC; ++u) s[tt][u] = o[u];
        }
      }
#pragma unroll
      for (int k = 0; k < KS; ++k) {
        const int y = k / ND, n = k % ND;
        __builtin_amdgcn_sched_barrier(0);
        const f16x8 a = ring[k % 4];
        if (k + 4 < KS) ring[k % 4] = value_at(c, k + 4);
#pragma unroll
        for (int u = 0; u < RC; ++u) acc[u][n] = mfma32(a, w[u][y], acc[u][n]);
        if (n == 0) {
#pragma unroll
          for (int u = 0; u < RC; ++u) l[u] = fmaf(sum[u][y], inv[y % NR], l[u]);
        }
        // the widening, a piece at a time
        const int p0 = k * (KP + VP) / KS, p1 = (k + 1) * (KP + VP) / KS;
#pragma unroll
        for (int i = p0; i < p1; ++i) {
          if (i < KP) store_key(c + 2, i);
          else store_value(c + 1, i - KP);
        }
      }
      __builtin_amdgcn_sched_barrier(0);
    } else {
      if (c + 1 == wb && wb < we) {
        scores(c + 1, 0);
        scores(c + 1, 1);
      }
      store_keys(c + 2);
      store_values(c + 1);
    }
    // keys of tile c + 2 and values of tile c + 1 are in LDS, the loads of the tiles after them begin
    store_scales(c + 1);
    load_keys(c + 3);
    load_values(c + 2);
    key_pages(c + 4);
    value_page(c + 3);
    __syncthreads();
  }

#pragma unroll
  for (int u = 0; u < RC; ++u) {
    l[u] += __shfl_xor(l[u], 32);
    const int r = rw + 32 * u + m;
    if (P.splits > 1) {
      if (rw + 32 * u >= rows) return;
      if (l[u] != l[u]) M[u] = INFINITY;  // the maximum does not see NaN
      const int64_t tile = ((bh * P.rtiles + rt) * kWaves + wave) * RC + u;
      float *o = P.part + (tile * P.splits + split) * part32_floats(ND);
#pragma unroll
      for (int n = 0; n < ND; ++n)
#pragma unroll
        for (int i = 0; i < 4; ++i)
          *reinterpret_cast<f32x4 *>(o + ((n * 4 + i) * 64 + lane) * 4) =
              f32x4{acc[u][n][4 * i], acc[u][n][4 * i + 1], acc[u][n][4 * i + 2], acc[u][n][4 * i + 3]};
      if (g == 0) {
        o[ND * 1024 + m] = M[u];
        o[ND * 1024 + 32 + m] = l[u];
      }
      continue;
    }
    if (r >= rows) continue;
    const RowAt at = row_at(A, C, q, h, r);
    const float inv = l[u] == 0.0f ? 0.0f : 1.0f / l[u];
#pragma unroll
    for (int n = 0; n < ND; ++n)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int c = 32 * n + 8 * i + 4 * g;
        const float z[4] = {acc[u][n][4 * i] * inv, acc[u][n][4 * i + 1] * inv, acc[u][n][4 * i + 2] * inv,
                            acc[u][n][4 * i + 3] * inv};
        if (c < d) store_o4(A, at.o + c, z);
      }
    if (A.lse && g == 0) A.lse[at.lse] = log_sum(M[u], l[u], kUp32);
  }
}

// Joins the splits of 32 rows: a wave per four accumulators of a lane.
template <int ND>
__global__ __launch_bounds__(64) void kv_prompt_join_kernel(AttendArgs P, int W) {
  const KvCache &C = P.C;
  const KvAttend &A = P.A;
  const int n = blockIdx.x % (4 * ND);
  const int64_t tile = blockIdx.x / (4 * ND);
  int64_t x = tile / W;
  const int rt = (int)(x % P.rtiles);
  x /= P.rtiles;
  const int h = (int)(x % C.heads);
  const int b = (int)(x / C.heads);
  KvSeq q;
  if (!kv_seq(P.S, C.page, b, &q)) return;
  const int rows = q.n * A.group, r0 = (rt * W + (int)(tile % W)) * 32;
  if (r0 >= rows) return;
  const int lane = threadIdx.x, m = lane & 31, g = lane >> 5;
  const float *base = P.part + tile * P.splits * part32_floats(ND);
  float Mx = -INFINITY;
  for (int y = 0; y < P.splits; ++y) Mx = fmaxf(Mx, base[(int64_t)y * part32_floats(ND) + ND * 1024 + m]);
  float l = 0.0f;
  f32x4 o = {0, 0, 0, 0};
  for (int y = 0; y < P.splits; ++y) {
    const float *p = base + (int64_t)y * part32_floats(ND);
    const float My = p[ND * 1024 + m];
    if (My == -INFINITY) continue;
    const float al = __builtin_amdgcn_exp2f(My - Mx);
    l += p[ND * 1024 + 32 + m] * al;
    o += *reinterpret_cast<const f32x4 *>(p + (n * 64 + lane) * 4) * al;
  }
  const int r = r0 + m;
  if (r >= rows) return;
  const RowAt at = row_at(A, C, q, h, r);
  o *= l == 0.0f ? 0.0f : 1.0f / l;
  const float y[4] = {o.x, o.y, o.z, o.w};
  const int c = 32 * (n / 4) + 8 * (n % 4) + 4 * g;
  if (c < C.d) store_o4(A, at.o + c, y);
  if (A.lse && n == 0 && g == 0) A.lse[at.lse] = log_sum(Mx, l, kUp32);
}

struct Plan {
  bool prompt;
  int nt, rt, rtiles, splits;
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

// 64 rows of a wave share the operands read from LDS, as far as a wave's 512 registers hold their accumulators
constexpr int row_tiles(int nd) { return 1; }

Plan plan(const KvCache &C, const KvSeqs &S, const KvAttend &A) {
  Plan p;
  const int64_t rows = (int64_t)S.max_rows * A.group;
  const int64_t len = A.window ? std::min<int64_t>(S.max_len, (int64_t)A.window + S.max_rows) : S.max_len;
  p.prompt = rows > 32 && A.type != KM_T_F32;
  if (p.prompt) {
    p.nt = dim_tiles32(C.d);
    p.rt = kWaves * row_tiles(p.nt);
    p.rtiles = (int)cdiv(rows, 32 * p.rt);
    p.tiles = (int64_t)S.n * C.heads * p.rtiles;
    const int64_t most = std::max<int64_t>(1, len / (8 * kChunk));
    p.splits = (int)std::min(most, std::max<int64_t>(1, 512 / p.tiles));
    return p;
  }
  p.nt = dim_tiles(C.d);
  p.rt = rows > 16 && A.type != KM_T_F32 ? 2 : 1;
  p.rtiles = (int)cdiv(rows, 16 * p.rt);
  p.tiles = (int64_t)S.n * C.heads * p.rtiles;
  // enough workgroups for every CU to hold two; a split of fewer than four chunks leaves waves without work
  const int64_t most = std::max<int64_t>(1, cdiv(len, 4 * kChunk));
  p.splits = (int)std::min(most, std::max<int64_t>(1, 512 / p.tiles));
  return p;
}

}  // namespace

int64_t kv_attend_blocks(const KvCache &C, const KvSeqs &S, const KvAttend &A) {
  const Plan p = plan(C, S, A);
  return p.tiles * std::max(p.splits, p.rt * p.nt * (p.prompt ? 4 : 1));  // the join's grid is the larger one
}

size_t kv_attend_scratch(const KvCache &C, const KvSeqs &S, const KvAttend &A) {
  const Plan p = plan(C, S, A);
  return p.splits > 1 ? sizeof(float) * (size_t)p.tiles * p.splits * p.rt *
                            (p.prompt ? part32_floats(p.nt) : part_floats(p.nt))
                      : 0;
}

km_status launch_kv_attend(const KvCache &C, const KvSeqs &S, const KvAttend &A, void *ws, hipStream_t s) {
  const Plan p = plan(C, S, A);
  AttendArgs P{C, S, A, p.rtiles, p.splits, static_cast<float *>(ws)};
  const dim3 grid((unsigned)(p.tiles * p.splits));
  if (p.prompt) {
#define KV_K(F, N)                                                                         \
  C.page >= kChunk ? kv_prompt_kernel<F, N, row_tiles(N), true><<<grid, 64 * kWaves, 0, s>>>(P) \
                   : kv_prompt_kernel<F, N, row_tiles(N), false><<<grid, 64 * kWaves, 0, s>>>(P)
#define KV_N(N)                                                                                                 \
  case N:                                                                                                       \
    if (C.fmt == KM_KV_I8) KV_K(KM_KV_I8, N);                                                                   \
    else KV_K(KM_KV_F8, N);                                                                                     \
    KMQ_LAUNCH_CHECK("kv_attend");                                                                              \
    if (p.splits > 1)                                                                                           \
      kv_prompt_join_kernel<N><<<dim3((unsigned)(p.tiles * p.rt * 4 * N)), 64, 0, s>>>(P, p.rt);                \
    break;
    switch (p.nt) {
      KV_N(2)
      KV_N(3)
      KV_N(4)
      KV_N(6)
      KV_N(8)
    }
#undef KV_N
#undef KV_K
    KMQ_LAUNCH_CHECK("kv_attend");
    return KM_OK;
  }
#define KV_K(F, N, R, Z) kv_attend_kernel<F, N, R, Z><<<grid, 256, 0, s>>>(P)
#define KV_R(F, N)                          \
  if (A.type == KM_T_F32) KV_K(F, N, 1, 2); \
  else if (p.rt == 2) KV_K(F, N, 2, 1);     \
  else KV_K(F, N, 1, 1);
#define KV_N(N)                                                                                         \
  case N:                                                                                               \
    if (C.fmt == KM_KV_I8) {                                                                            \
      KV_R(KM_KV_I8, N)                                                                                 \
    } else {                                                                                            \
      KV_R(KM_KV_F8, N)                                                                                 \
    }                                                                                                   \
    KMQ_LAUNCH_CHECK("kv_attend");                                                                      \
    if (p.splits > 1) kv_join_kernel<N><<<dim3((unsigned)(p.tiles * p.rt * N)), 64, 0, s>>>(P, p.rt);   \
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
#undef KV_K
  KMQ_LAUNCH_CHECK("kv_attend");
  return KM_OK;
}

}  // namespace kmq
