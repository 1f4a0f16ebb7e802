// Writing keys and values into the 8-bit cache and reading them back.
//
// A page (a block of tokens of one head) has one scale, so one workgroup owns the page for the call: it finds the largest
// magnitude of the rows that the call writes there, takes the smaller multiplier of that and of the tokens already in the
// page, and codes the rows; if the multiplier shrank, the earlier tokens' codes are coded again.  Keys and values
// are different workgroups.  Values lie with their dims first (the attention's second product contracts tokens), so
// their codes turn through LDS on the way in and in registers on the way out.
//
// Both are bound by HBM: 3 bytes per 16-bit element.
#include "kv.hpp"

namespace kmq {
namespace {

constexpr int kThreads = 256;

template <int FMT>
constexpr float kQmax = FMT == KM_KV_I8 ? 127.0f : 448.0f;

// x * mul for a code: rounded to odd where the product is not exact (fp32 rows), so that the rounding to a code is
// that of the exact product.
template <int TYPE>
__device__ __forceinline__ float scaled(float x, float mul) {
  float p = x * mul;
  if constexpr (TYPE == KM_T_F32) {
    const float e = fmaf(x, mul, -p);
    if (e != 0.0f) {
      uint32_t u = __float_as_uint(p);
      if ((e < 0.0f) != (p < 0.0f)) u -= 1;  // the nearest was farther from zero
      p = __uint_as_float(u | 1u);
    }
  }
  return p;
}

// Four values already times the multiplier (in range) to codes, the first in the low byte.
template <int FMT>
__device__ __forceinline__ uint32_t code4(float a, float b, float c, float d) {
  if constexpr (FMT == KM_KV_I8) {
    // 1.5 * 2^23 leaves the nearest integer, ties to the even one, in the low bits
    constexpr float kR = 12582912.0f;
    const uint32_t lo = __builtin_amdgcn_perm(__float_as_uint(b + kR), __float_as_uint(a + kR), 0x0c0c0400u);
    const uint32_t hi = __builtin_amdgcn_perm(__float_as_uint(d + kR), __float_as_uint(c + kR), 0x0c0c0400u);
    return lo | (hi << 16);
  } else {
    const int lo = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
    return __builtin_amdgcn_cvt_pk_fp8_f32(c, d, lo, true);
  }
}

// NaN counts as 0 and an infinity as the largest finite magnitude of its page's rows.
__device__ __forceinline__ float tame(float x, float top) {
  return x == x ? fminf(fmaxf(x, -top), top) : 0.0f;
}

// The codes of a dword for a smaller multiplier: code * mul is exact, the quotient correctly rounded, and a quotient of
// such short numbers is never that close to the middle of two codes unless it is the middle.
template <int FMT>
__device__ __forceinline__ uint32_t recode4(uint32_t c, float mul, float was) {
  f16x2 lo, hi;
  kv_widen4<FMT>(c, &lo, &hi);
  return code4<FMT>((float)lo.x * mul / was, (float)lo.y * mul / was, (float)hi.x * mul / was, (float)hi.y * mul / was);
}

struct PageJob {
  int64_t pg;   // page, or -1
  int64_t row;  // row of the call at token i0
  int i0, i1;   // tokens of the page that the call's rows cover; none: i0 = i1
  int64_t row0;
  int lead;     // rows from row0 on that fall before position 0: zeros when read (the first page's workgroups write them)
};

// Job of workgroup x: touched page t of head h of sequence b.
__device__ __forceinline__ bool page_job(const KvCache &C, const KvSeqs &S, int64_t x, int touched, int *h,
                                         PageJob *j) {
  *h = (int)(x % C.heads);
  x /= C.heads;
  const int t = (int)(x % touched);
  const int b = (int)(x / touched);
  KvSeq q;
  if (!kv_seq(S, C.page, b, &q)) return false;
  const int first = max(q.len - q.n, 0);  // rows before position 0 have no place
  const int lead = q.n - (q.len - first);
  const int slot = (first >> C.shift) + t;
  const int p0 = slot << C.shift;
  j->row0 = q.row0;
  j->lead = t == 0 ? lead : 0;
  if (p0 >= q.len) {
    j->i0 = j->i1 = 0;
    return j->lead > 0;
  }
  j->i0 = max(first - p0, 0);
  j->i1 = min(q.len - p0, C.page);
  j->row = q.row0 + lead + (p0 + j->i0 - first);
  const int64_t pg = S.table[(int64_t)b * S.table_ld + slot];
  j->pg = pg >= 0 && pg < C.pages ? pg : -1;
  return true;
}

// bit patterns of magnitudes are ordered like the magnitudes
__device__ __forceinline__ uint32_t block_max(uint32_t m, uint32_t *sh) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) m = max(m, (uint32_t)__shfl_xor((int)m, o));
  if ((threadIdx.x & 63) == 0) sh[threadIdx.x >> 6] = m;
  __syncthreads();
  return max(max(sh[0], sh[1]), max(sh[2], sh[3]));
}

// LDS row of one token's codes: a dword more than its dims, so that the tokens of a dim lie in different banks
__device__ __forceinline__ int turn_ld(int d) { return d + 4; }

template <int FMT, int TYPE>
__global__ __launch_bounds__(kThreads) void kv_write_kernel(KvCache C, KvSeqs S, KvRows kr, KvRows vr, int touched) {
  extern __shared__ uint32_t turn[];  // values: codes of the new rows, [token][turn_ld]
  __shared__ uint32_t sh[4];
  const bool values = blockIdx.x & 1;
  int h;
  PageJob j;
  if (!page_job(C, S, blockIdx.x >> 1, touched, &h, &j) || j.i1 == 0 || j.pg < 0) return;
  const KvRows &src = values ? vr : kr;
  const int d = C.d, t = threadIdx.x;
  const int per = d / 8;  // groups of 8 dims in a row
  const int items = (j.i1 - j.i0) * per;
  const int64_t at = j.row * src.row + h * src.head;
  float *scale = (values ? C.vs : C.ks) + j.pg * C.heads + h;
  const float s_old = j.i0 ? *scale : 0.0f;

  uint32_t top = 0;
  for (int i = t; i < items; i += kThreads) {
    float x[8];
    kv_load<TYPE, 8>(src.p, at + (int64_t)(i / per) * src.row + (i % per) * 8, x);
#pragma unroll
    for (int u = 0; u < 8; ++u) {
      const uint32_t a = __float_as_uint(x[u]) & 0x7fffffffu;
      top = a < 0x7f800000u ? max(top, a) : top;
    }
  }
  const float a = __uint_as_float(block_max(top, sh));
  float mul = kv_mul_of_top(a, kQmax<FMT>);
  bool again = false;
  float was = 0.0f;
  if (j.i0) {
    was = kv_mul_of_scale(s_old);
    again = mul < was;
    mul = fminf(mul, was);
  }
  if (t == 0) *scale = 1.0f / mul;

  uint8_t *dst = (values ? C.v : C.k) + (j.pg * C.heads + h) * (int64_t)C.page * d;
  const int ld = turn_ld(d);
  for (int i = t; i < items; i += kThreads) {
    float x[8];
    const int r = i / per, c = (i % per) * 8;
    kv_load<TYPE, 8>(src.p, at + (int64_t)r * src.row + c, x);
#pragma unroll
    for (int u = 0; u < 8; ++u) x[u] = scaled<TYPE>(tame(x[u], a), mul);
    const u32x2 q = {code4<FMT>(x[0], x[1], x[2], x[3]), code4<FMT>(x[4], x[5], x[6], x[7])};
    if (values) {
      uint32_t *w = turn + (r * ld + c) / 4;
      w[0] = q.x;
      w[1] = q.y;
    } else {
      *reinterpret_cast<u32x2 *>(dst + (j.i0 + r) * d + c) = q;
    }
  }
  if (!values) {
    if (again) {
      u32x4 *o = reinterpret_cast<u32x4 *>(dst);
      for (int i = t; i < j.i0 * d / 16; i += kThreads) {
        u32x4 w = o[i];
#pragma unroll
        for (int u = 0; u < 4; ++u) w[u] = recode4<FMT>(w[u], mul, was);
        o[i] = w;
      }
    }
    return;
  }
  __syncthreads();
  const uint8_t *tb = reinterpret_cast<const uint8_t *>(turn);
  if (!again && j.i1 - j.i0 < 16) {  // a few tokens: their bytes alone
    for (int i = t; i < (j.i1 - j.i0) * d; i += kThreads) {
      const int r = i / d, c = i % d;
      dst[(int64_t)c * C.page + j.i0 + r] = tb[r * ld + c];
    }
    return;
  }
  // 16 tokens of one dim at a time; what lies in them before i0 is coded again or stays, what lies behind i1 stays
  const int g0 = again ? 0 : j.i0 / 16, g1 = (j.i1 + 15) / 16;
  for (int i = t; i < (g1 - g0) * d; i += kThreads) {
    const int c = i % d, g = g0 + i / d;
    u32x4 *o = reinterpret_cast<u32x4 *>(dst + (int64_t)c * C.page + g * 16);
    const bool whole = g * 16 >= j.i0 && g * 16 + 16 <= j.i1;
    u32x4 w = {0, 0, 0, 0};
    if (!whole) w = *o;
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      const uint32_t old = again ? recode4<FMT>(w[u], mul, was) : w[u];
      uint32_t n = 0;
#pragma unroll
      for (int y = 0; y < 4; ++y) {
        const int tok = g * 16 + u * 4 + y;
        const uint32_t keep = ((tok < j.i0 ? old : w[u]) >> (8 * y)) & 255u;
        n |= (tok >= j.i0 && tok < j.i1 ? (uint32_t)tb[(tok - j.i0) * ld + c] : keep) << (8 * y);
      }
      w[u] = n;
    }
    *o = w;
  }
}

// code * scale in fp32, rounded to the type; past its largest finite value that value
template <int TYPE>
__device__ __forceinline__ float value(float code, float s) {
  constexpr float top = TYPE == KM_T_F16 ? 65504.0f : TYPE == KM_T_BF16 ? 0x1.fep127f : 0x1.fffffep127f;
  return fminf(fmaxf(code * s, -top), top);
}

template <int FMT, int TYPE>
__global__ __launch_bounds__(kThreads) void kv_read_kernel(KvCache C, KvSeqs S, KvRows kr, KvRows vr, int touched) {
  const bool values = blockIdx.x & 1;
  int h;
  PageJob j;
  if (!page_job(C, S, blockIdx.x >> 1, touched, &h, &j)) return;
  const KvRows &out = values ? vr : kr;
  const int d = C.d, t = threadIdx.x;
  for (int i = t; i < j.lead * (d / 4); i += kThreads) {
    const float z[4] = {0, 0, 0, 0};
    kv_store<TYPE, 4>(out.p, (j.row0 + i / (d / 4)) * out.row + h * out.head + i % (d / 4) * 4, z);
  }
  if (j.i1 == 0) return;
  const int64_t at = j.row * out.row + h * out.head;
  const int64_t pg = j.pg < 0 ? 0 : j.pg;
  const float s = j.pg < 0 ? 0.0f : (values ? C.vs : C.ks)[pg * C.heads + h];
  const uint8_t *src = (values ? C.v : C.k) + (pg * C.heads + h) * (int64_t)C.page * d;
  if (!values) {
    const int per = d / 16;
    for (int i = t; i < (j.i1 - j.i0) * per; i += kThreads) {
      const int r = i / per, c = (i % per) * 16;
      u32x4 w = {0, 0, 0, 0};
      if (j.pg >= 0) w = *reinterpret_cast<const u32x4 *>(src + (j.i0 + r) * d + c);
      float x[16];
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        f16x2 lo, hi;
        kv_widen4<FMT>(w[u], &lo, &hi);
        x[4 * u] = value<TYPE>((float)lo.x, s);
        x[4 * u + 1] = value<TYPE>((float)lo.y, s);
        x[4 * u + 2] = value<TYPE>((float)hi.x, s);
        x[4 * u + 3] = value<TYPE>((float)hi.y, s);
      }
      kv_store<TYPE, 16>(out.p, at + (int64_t)r * out.row + c, x);
    }
    return;
  }
  // 16 tokens of four dims: four loads, sixteen rows of four values
  const int g0 = j.i0 / 16, g1 = (j.i1 + 15) / 16, per = d / 4;
  for (int i = t; i < (g1 - g0) * per; i += kThreads) {
    const int g = g0 + i / per, c = (i % per) * 4;
    u32x4 w[4];
#pragma unroll
    for (int y = 0; y < 4; ++y) {
      w[y] = u32x4{0, 0, 0, 0};
      if (j.pg >= 0) w[y] = *reinterpret_cast<const u32x4 *>(src + (int64_t)(c + y) * C.page + g * 16);
    }
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      f16x2 q[4][2];
#pragma unroll
      for (int y = 0; y < 4; ++y) kv_widen4<FMT>(w[y][u], &q[y][0], &q[y][1]);
#pragma unroll
      for (int z = 0; z < 4; ++z) {
        const int tok = g * 16 + u * 4 + z;
        if (tok < j.i0 || tok >= j.i1) continue;
        float x[4];
#pragma unroll
        for (int y = 0; y < 4; ++y) x[y] = value<TYPE>((float)q[y][z / 2][z % 2], s);
        kv_store<TYPE, 4>(out.p, at + (int64_t)(tok - j.i0) * out.row + c, x);
      }
    }
  }
}

int touched_pages(const KvCache &C, const KvSeqs &S) {
  return (int)std::min<int64_t>(S.max_pages, cdiv(S.max_rows - 1, C.page) + 1);
}

}  // namespace

int64_t kv_move_blocks(const KvCache &C, const KvSeqs &S) { return 2 * (int64_t)S.n * touched_pages(C, S) * C.heads; }

km_status launch_kv_write(const KvCache &C, const KvSeqs &S, KvRows k, KvRows v, int type, hipStream_t s) {
  const int touched = touched_pages(C, S);
  const size_t lds = (size_t)std::min(C.page, S.max_rows) * (C.d + 4);
  const dim3 grid((unsigned)kv_move_blocks(C, S));
#define KV_GO(F, T) kv_write_kernel<F, T><<<grid, kThreads, lds, s>>>(C, S, k, v, touched)
  if (C.fmt == KM_KV_I8) {
    if (type == KM_T_F32) KV_GO(KM_KV_I8, KM_T_F32);
    else if (type == KM_T_BF16) KV_GO(KM_KV_I8, KM_T_BF16);
    else KV_GO(KM_KV_I8, KM_T_F16);
  } else {
    if (type == KM_T_F32) KV_GO(KM_KV_F8, KM_T_F32);
    else if (type == KM_T_BF16) KV_GO(KM_KV_F8, KM_T_BF16);
    else KV_GO(KM_KV_F8, KM_T_F16);
  }
#undef KV_GO
  KMQ_LAUNCH_CHECK("kv_write");
  return KM_OK;
}

km_status launch_kv_read(const KvCache &C, const KvSeqs &S, KvRows k, KvRows v, int type, hipStream_t s) {
  const int touched = touched_pages(C, S);
  const dim3 grid((unsigned)kv_move_blocks(C, S));
#define KV_GO(F, T) kv_read_kernel<F, T><<<grid, kThreads, 0, s>>>(C, S, k, v, touched)
  if (C.fmt == KM_KV_I8) {
    if (type == KM_T_F32) KV_GO(KM_KV_I8, KM_T_F32);
    else if (type == KM_T_BF16) KV_GO(KM_KV_I8, KM_T_BF16);
    else KV_GO(KM_KV_I8, KM_T_F16);
  } else {
    if (type == KM_T_F32) KV_GO(KM_KV_F8, KM_T_F32);
    else if (type == KM_T_BF16) KV_GO(KM_KV_F8, KM_T_BF16);
    else KV_GO(KM_KV_F8, KM_T_F16);
  }
#undef KV_GO
  KMQ_LAUNCH_CHECK("kv_read");
  return KM_OK;
}

}  // namespace kmq
