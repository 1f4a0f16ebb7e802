// What the kernels share that move keys and values into pages, out of them and between them.
#pragma once

#include "kv.hpp"

namespace kmq {
namespace {

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

// Four values' codes, the first in the low byte.
template <int FMT, int TYPE>
__device__ __forceinline__ uint32_t code4(const float *x, float mul) {
  if constexpr (FMT == KM_KV_I8) {
    // 1.5 * 2^23 leaves the nearest integer of the exact product, ties to the even one, in the low bits
    uint32_t q[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) q[i] = __float_as_uint(fmaf(x[i], mul, 12582912.0f));
    return __builtin_amdgcn_perm(__builtin_amdgcn_perm(q[3], q[2], 0x0c0c0400u), __builtin_amdgcn_perm(q[1], q[0], 0x0c0c0400u),
                                 0x05040100u);
  } else {
    const int lo = __builtin_amdgcn_cvt_pk_fp8_f32(scaled<TYPE>(x[0], mul), scaled<TYPE>(x[1], mul), 0, false);
    return __builtin_amdgcn_cvt_pk_fp8_f32(scaled<TYPE>(x[2], mul), scaled<TYPE>(x[3], mul), lo, true);
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
  const float x[4] = {(float)lo.x * mul / was, (float)lo.y * mul / was, (float)hi.x * mul / was, (float)hi.y * mul / was};
  return code4<FMT, KM_T_BF16>(x, 1.0f);
}

struct PageJob {
  int64_t pg;   // page, or -1
  int64_t row;  // row of the call at token i0
  int i0, i1;   // tokens of the page that the call's rows cover; none: i0 = i1
  int64_t row0;
  int lead;     // rows from row0 on that fall before position 0: zeros when read (the first page's workgroups write them)
};

// Job of workgroup x: keys or values of touched page t of head h of sequence b.  A page's heads lie eight workgroups apart, on
// one XCD: their rows lie side by side (74631 tokens of 8 heads of 128, written and read back: 197 us, spread 205, both
// before rows were read whole).
__device__ __forceinline__ bool page_job(const KvCache &C, const KvSeqs &S, uint32_t x, int touched, bool *values, int *h,
                                         PageJob *j) {
  uint32_t y = x >> 3;
  const uint32_t part = y % (2u * C.heads);
  y = (y / (2u * C.heads)) * 8 + (x & 7);
  *values = part & 1;
  *h = (int)(part >> 1);
  const int t = (int)(y % (uint32_t)touched);
  const int b = (int)(y / (uint32_t)touched);
  if (b >= S.n) return false;
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

__device__ __forceinline__ uint32_t block_max(uint32_t m, uint32_t *sh) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) m = max(m, (uint32_t)__shfl_xor((int)m, o));
  const int waves = blockDim.x / 64;
  if (waves == 1) return m;
  __syncthreads();  // an earlier maximum has been read
  if ((threadIdx.x & 63) == 0) sh[threadIdx.x >> 6] = m;
  __syncthreads();
  m = sh[0];
  for (int y = 1; y < waves; ++y) m = max(m, sh[y]);
  return m;
}

// Eight values of a row as they lie in memory.
template <int TYPE>
struct Raw {
  u32x4 w[TYPE == KM_T_F32 ? 2 : 1];
};
template <int TYPE>
__device__ __forceinline__ Raw<TYPE> raw_load(const void *p, int64_t o) {
  Raw<TYPE> r;
  const u32x4 *q = reinterpret_cast<const u32x4 *>(static_cast<const char *>(p) + o * KvElem<TYPE>::bytes);
#pragma unroll
  for (int i = 0; i < (TYPE == KM_T_F32 ? 2 : 1); ++i) r.w[i] = q[i];
  return r;
}
template <int TYPE>
__device__ __forceinline__ void raw_values(const Raw<TYPE> &r, float *x) {
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    if constexpr (TYPE == KM_T_F32) {
      x[i] = __uint_as_float(r.w[i / 4][i % 4]);
    } else {
      const uint32_t w = r.w[0][i / 2];
      if constexpr (TYPE == KM_T_BF16) x[i] = __uint_as_float(i % 2 ? w & 0xffff0000u : w << 16);
      else x[i] = (float)__builtin_bit_cast(f16x2, w)[i % 2];
    }
  }
}
// Bit patterns of magnitudes are ordered like the magnitudes: the largest one, of 16-bit types in both halves of a
// dword.  kInf: the first pattern that is not finite.
template <int TYPE>
constexpr uint32_t kInf = TYPE == KM_T_F32 ? 0x7f800000u : TYPE == KM_T_BF16 ? 0x7f80u : 0x7c00u;
typedef uint16_t u16x2 __attribute__((ext_vector_type(2)));
template <int TYPE>
__device__ __forceinline__ uint32_t raw_max(uint32_t m, uint32_t w) {
  if constexpr (TYPE == KM_T_F32) {
    return max(m, w & 0x7fffffffu);
  } else {
    const uint32_t a = w & 0x7fff7fffu;
    return __builtin_bit_cast(uint32_t, __builtin_elementwise_max(__builtin_bit_cast(u16x2, m), __builtin_bit_cast(u16x2, a)));
  }
}

// A thread's place in a grid of rows of `per` items, and the one of a number of threads further on.
struct Place {
  int r, c;
};
__device__ __forceinline__ void advance(Place &p, int per, int dr, int dc) {
  p.r += dr;
  p.c += dc;
  if (p.c >= per) {
    p.c -= per;
    ++p.r;
  }
}

// Item i of a page's values: 16 tokens g of the four dims from c on.  Up to four groups of tokens (64 bytes of a dim's row)
// lie side by side, then the dims (rows of up to 128 bytes and more), then the other four groups of a page of 128.
__device__ __forceinline__ void group_of(int i, int ng, int quads, int *g, int *c) {
  const int bits = ng >= 4 ? 2 : ng - 1;  // of 1, 2 or 4 groups
  int q = i >> bits;
  *g = i & ((1 << bits) - 1);
  if (q >= quads) {
    q -= quads;
    *g += 4;
  }
  *c = 4 * q;
}

// The bytes y of four dwords as one dword each: a 4 x 4 transpose.
__device__ __forceinline__ void turn4(const uint32_t *a, uint32_t *o) {
  const uint32_t x = __builtin_amdgcn_perm(a[1], a[0], 0x05010400u), y = __builtin_amdgcn_perm(a[3], a[2], 0x05010400u);
  const uint32_t z = __builtin_amdgcn_perm(a[1], a[0], 0x07030602u), w = __builtin_amdgcn_perm(a[3], a[2], 0x07030602u);
  o[0] = __builtin_amdgcn_perm(y, x, 0x05040100u);
  o[1] = __builtin_amdgcn_perm(y, x, 0x07060302u);
  o[2] = __builtin_amdgcn_perm(w, z, 0x05040100u);
  o[3] = __builtin_amdgcn_perm(w, z, 0x07060302u);
}

// LDS row of one token's codes: a dword more than its dims, so that the tokens of a dim lie in different banks
__device__ __forceinline__ int turn_ld(int d) { return d + 4; }

// code * scale in fp32, rounded to the type; past its largest finite value that value
template <int TYPE>
__device__ __forceinline__ float value(float code, float s) {
  constexpr float top = TYPE == KM_T_F16 ? 65504.0f : TYPE == KM_T_BF16 ? 0x1.fep127f : 0x1.fffffep127f;
  return fminf(fmaxf(code * s, -top), top);
}

int touched_pages(const KvCache &C, const KvSeqs &S) {
  return (int)std::min<int64_t>(S.max_pages, cdiv(S.max_rows - 1, C.page) + 1);
}

}  // namespace
}  // namespace kmq
