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

// The log of a row's sum of exp.  l = 0: the row saw no position.
__device__ __forceinline__ float log_sum(float M, float l) {
  return l > 0.0f ? (M - kUp + __builtin_amdgcn_logf(l)) * 0.69314718055994530942f : (l == 0.0f ? -INFINITY : NAN);
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
    const int e = (int)(__float_as_uint(top) >> 23);  // 0 .. 255
    // 2^(13 - (e - 127)), within the exponents whose inverse is a normal number too
    const int up = min(max(140 - e, -126), 126);
    const float f = __uint_as_float((uint32_t)(127 + up) << 23);
    cs[u] = A.scale * kLog2e * __uint_as_float((uint32_t)(127 - up) << 23);
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

struct Plan {
  int nt, rt, rtiles, splits;
  int64_t tiles;
};

int dim_tiles(int d) {  // the instantiated widths
  const int t = (int)cdiv(d, 16);
  return t <= 4 ? 4 : t <= 5 ? 5 : t <= 6 ? 6 : t <= 8 ? 8 : t <= 12 ? 12 : 16;
}

Plan plan(const KvCache &C, const KvSeqs &S, const KvAttend &A) {
  Plan p;
  p.nt = dim_tiles(C.d);
  const int64_t rows = (int64_t)S.max_rows * A.group;
  p.rt = rows > 16 && A.type != KM_T_F32 ? 2 : 1;
  p.rtiles = (int)cdiv(rows, 16 * p.rt);
  p.tiles = (int64_t)S.n * C.heads * p.rtiles;
  // enough workgroups for every CU to hold two; a split of fewer than four chunks leaves waves without work
  int64_t len = A.window ? std::min<int64_t>(S.max_len, (int64_t)A.window + S.max_rows) : S.max_len;
  const int64_t most = std::max<int64_t>(1, cdiv(len, 4 * kChunk));
  p.splits = (int)std::min(most, std::max<int64_t>(1, 512 / p.tiles));
  return p;
}

}  // namespace

int64_t kv_attend_blocks(const KvCache &C, const KvSeqs &S, const KvAttend &A) {
  const Plan p = plan(C, S, A);
  return p.tiles * std::max(p.splits, p.rt * p.nt);  // the join has a workgroup per 16 rows and 16 dims
}

size_t kv_attend_scratch(const KvCache &C, const KvSeqs &S, const KvAttend &A) {
  const Plan p = plan(C, S, A);
  return p.splits > 1 ? sizeof(float) * (size_t)p.tiles * p.splits * p.rt * part_floats(p.nt) : 0;
}

km_status launch_kv_attend(const KvCache &C, const KvSeqs &S, const KvAttend &A, void *ws, hipStream_t s) {
  const Plan p = plan(C, S, A);
  AttendArgs P{C, S, A, p.rtiles, p.splits, static_cast<float *>(ws)};
  const dim3 grid((unsigned)(p.tiles * p.splits));
#define KV_K(F, N, R, Z) kv_attend_kernel<F, N, R, Z><<<grid, 256, 0, s>>>(P)
#define KV_R(F, N)                     \
  if (A.type == KM_T_F32) KV_K(F, N, 1, 2); \
  else if (p.rt == 2) KV_K(F, N, 2, 1);     \
  else KV_K(F, N, 1, 1);
#define KV_N(N)                              \
  case N:                                    \
    if (C.fmt == KM_KV_I8) {                 \
      KV_R(KM_KV_I8, N)                      \
    } else {                                 \
      KV_R(KM_KV_F8, N)                      \
    }                                        \
    KMQ_LAUNCH_CHECK("kv_attend");           \
    if (p.splits > 1) kv_join_kernel<N><<<dim3((unsigned)(p.tiles * p.rt * N)), 64, 0, s>>>(P, p.rt); \
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
