// Writing keys and values into the 4-bit cache and reading them back.
//
// A row (the d values of a token and head) has its own scale, so rows do not depend on each other and nothing is ever coded
// again: with a the row's largest magnitude, mul = 7 / a without what lies below its eight leading bits, within [2^-30, 2^30], and
// the code is the whole number nearest to x * mul.  x * mul + 12582920 (1.5 * 2^23 + 8) in one fused step rounds the exact product
// to the nearest whole number, halves to the even one, and leaves code + 8 in the low bits.
//
// One workgroup takes a page's rows of one head, keys or values: lanes of a row (the next power of two of d / 8) take the row's
// maximum by shuffles.  Keys go out as they lie; values lie with their dims first, so their codes turn through LDS.  A byte of
// values holds two tokens, and a page's bytes have one owner, so what the call does not write of a byte is read and kept.
//
// Both move 2.5 bytes per 16-bit element and 4 per token and head, and keep the vector unit busy for 60 % of their time: 56691 tokens of 8
// heads of 128 in bf16 are written in 72 us (295 MB, 4.1 TB/s) and read back in 56 to 63 (4.7 to 5.3 TB/s; cards differ).  Maxima by row operations instead of LDS
// and codes gathered by byte permutes: 152 -> 143 us for both.
#include "kv_pages.hpp"

namespace kmq {
namespace {

constexpr int kMoveThreads = 256;
constexpr int kAhead = 4;  // rows (in a read, dwords) of a lane that are on their way at a time

// Eight values' codes + 8, a byte each, the first in the low byte.
template <bool CLAMP>
__device__ __forceinline__ u32x2 codes8(const float *x, float mul) {
  uint32_t q[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    float y = fmaf(x[i], mul, 12582920.0f);
    if constexpr (CLAMP) y = fminf(fmaxf(y, 12582913.0f), 12582927.0f);
    q[i] = __float_as_uint(y);
  }
  u32x2 o;
#pragma unroll
  for (int i = 0; i < 2; ++i)
    o[i] = __builtin_amdgcn_perm(__builtin_amdgcn_perm(q[4 * i + 3], q[4 * i + 2], 0x0c0c0400u),
                                 __builtin_amdgcn_perm(q[4 * i + 1], q[4 * i], 0x0c0c0400u), 0x05040100u);
  return o;
}
// The same, two to a byte.
__device__ __forceinline__ uint32_t halve8(u32x2 w) {
  return __builtin_amdgcn_perm(w.y | (w.y >> 4), w.x | (w.x >> 4), 0x06040200u);
}

// Values of the eight codes of a dword.
template <int TYPE>
__device__ __forceinline__ void values8(uint32_t w, float s, float *x) {
#pragma unroll
  for (int i = 0; i < 8; ++i) x[i] = value<TYPE>((float)((int)((w >> (4 * i)) & 15u) - 8), s);
}

// The largest of 4, 8, 16 or 32 neighbouring lanes, in each of them.
__device__ __forceinline__ uint32_t row_max(uint32_t m, int lanes) {
#define KV_DPP(ctrl) m = max(m, (uint32_t)__builtin_amdgcn_mov_dpp((int)m, ctrl, 0xf, 0xf, true))
  KV_DPP(0xb1);  // the other of two, the other two of four
  KV_DPP(0x4e);
  if (lanes > 4) KV_DPP(0x141);  // the mirrored lane of eight, of sixteen
  if (lanes > 8) KV_DPP(0x140);
#undef KV_DPP
  if (lanes > 16) m = max(m, (uint32_t)__shfl_xor((int)m, 16));
  return m;
}

template <int TYPE>
__global__ __launch_bounds__(kMoveThreads) void kv_write4_kernel(KvCache C, KvSeqs S, KvRows kr, KvRows vr, int touched,
                                                                 int lanes, uint32_t block0) {
  extern __shared__ uint32_t turn[];  // values: codes of the new rows, a byte each, [token][turn_ld]
  bool values;
  int h;
  PageJob j;
  if (!page_job(C, S, block0 + blockIdx.x, touched, &values, &h, &j) || j.i1 == 0 || j.pg < 0) return;
  const KvRows &src = values ? vr : kr;
  const int d = C.d, t = threadIdx.x, per = d / 8, rows = j.i1 - j.i0;
  const int64_t at = j.row * src.row + h * src.head;
  const int64_t head = j.pg * C.heads + h;
  float *scale = (values ? C.vs : C.ks) + head * C.page + j.i0;
  uint8_t *dst = (values ? C.v : C.k) + head * C.page * (d / 2);
  const int c = t % lanes, step = kMoveThreads / lanes, ld = turn_ld(d);
  const bool in = c < per;
  for (int r0 = 0; r0 < rows; r0 += step * kAhead) {
    Raw<TYPE> raw[kAhead];
#pragma unroll
    for (int i = 0; i < kAhead; ++i) {
      const int r = r0 + i * step + t / lanes;
#pragma unroll
      for (int y = 0; y < (TYPE == KM_T_F32 ? 2 : 1); ++y) raw[i].w[y] = u32x4{0, 0, 0, 0};
      if (in && r < rows) raw[i] = raw_load<TYPE>(src.p, at + (int64_t)r * src.row + c * 8);
    }
#pragma unroll
    for (int i = 0; i < kAhead; ++i) {
      if (r0 + i * step >= rows) break;
      const int r = r0 + i * step + t / lanes;
      uint32_t m = 0;
#pragma unroll
      for (int y = 0; y < (TYPE == KM_T_F32 ? 8 : 4); ++y) m = raw_max<TYPE>(m, raw[i].w[y / 4][y % 4]);
      if constexpr (TYPE != KM_T_F32) m = max(m & 0xffffu, m >> 16);
      m = row_max(m, lanes);
      float x[8];
      raw_values<TYPE>(raw[i], x);
      const bool wild = m >= kInf<TYPE>;  // infinities or NaN in the row
      if (__any(wild)) {
        uint32_t top = 0;
#pragma unroll
        for (int y = 0; y < 8; ++y) {
          const uint32_t a = __float_as_uint(x[y]) & 0x7fffffffu;
          top = a < 0x7f800000u ? max(top, a) : top;
        }
        top = row_max(top, lanes);
#pragma unroll
        for (int y = 0; y < 8; ++y) x[y] = tame(x[y], __uint_as_float(top));
        m = top;
      } else if constexpr (TYPE == KM_T_BF16) {
        m <<= 16;
      } else if constexpr (TYPE == KM_T_F16) {
        m = __float_as_uint((float)__builtin_bit_cast(f16x2, m).x);
      }
      const float mul = kv_mul4_of_top(__uint_as_float(m));
      // products are past 7 only where the multiplier is the least that there is
      const u32x2 w = __any(mul == 0x1p-30f) ? codes8<true>(x, mul) : codes8<false>(x, mul);
      if (!in || r >= rows) continue;
      if (c == 0) scale[r] = 1.0f / mul;
      if (values) {  // rows of turn are an odd number of dwords apart: two stores, not one of eight bytes
        turn[(r * ld + c * 8) / 4] = w.x;
        turn[(r * ld + c * 8) / 4 + 1] = w.y;
      } else {
        *reinterpret_cast<uint32_t *>(dst + (j.i0 + r) * (d / 2) + c * 4) = halve8(w);
      }
    }
  }
  if (!values) return;
  __syncthreads();
  // 16 tokens of four dims at a time, neighbouring threads the tokens of a dim's row
  const int ng = C.page / 16;
  for (int i = t; i < ng * (d / 4); i += kMoveThreads) {
    int g, c4;
    group_of(i, ng, d / 4, &g, &c4);
    const int k0 = g * 16 - j.i0;  // row of its first token
    if (k0 + 16 <= 0 || k0 >= rows) continue;
    uint8_t *o = dst + (c4 * C.page + g * 16) / 2;
    uint32_t a[8], b[4][2];  // pairs of tokens: four dims each; then [dim][eight tokens]
    if (k0 >= 0 && k0 + 16 <= rows) {
#pragma unroll
      for (int u = 0; u < 8; ++u) a[u] = turn[((k0 + 2 * u) * ld + c4) / 4] | (turn[((k0 + 2 * u + 1) * ld + c4) / 4] << 4);
    } else {
      u32x2 old[4];
#pragma unroll
      for (int y = 0; y < 4; ++y) old[y] = *reinterpret_cast<const u32x2 *>(o + y * C.page / 2);
#pragma unroll
      for (int u = 0; u < 8; ++u) {
        const int k = k0 + 2 * u;
        const bool lo = k >= 0 && k < rows, hi = k + 1 >= 0 && k + 1 < rows;
        const uint32_t keep = (lo ? 0u : 0x0f0f0f0fu) | (hi ? 0u : 0xf0f0f0f0u);
        uint32_t was = 0;
#pragma unroll
        for (int y = 0; y < 4; ++y) was |= ((old[y][u / 4] >> (8 * (u % 4))) & 255u) << (8 * y);
        a[u] = (was & keep) | (lo ? turn[(k * ld + c4) / 4] : 0u) | ((hi ? turn[((k + 1) * ld + c4) / 4] : 0u) << 4);
      }
    }
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      uint32_t z[4];
      turn4(a + 4 * u, z);
#pragma unroll
      for (int y = 0; y < 4; ++y) b[y][u] = z[y];
    }
#pragma unroll
    for (int y = 0; y < 4; ++y) *reinterpret_cast<u32x2 *>(o + y * C.page / 2) = u32x2{b[y][0], b[y][1]};
  }
}

template <int TYPE>
__global__ __launch_bounds__(kMoveThreads) void kv_read4_kernel(KvCache C, KvSeqs S, KvRows kr, KvRows vr, int touched,
                                                                uint32_t block0) {
  bool values;
  int h;
  PageJob j;
  if (!page_job(C, S, block0 + blockIdx.x, touched, &values, &h, &j)) return;
  const KvRows &out = values ? vr : kr;
  const int d = C.d, t = threadIdx.x, T = kMoveThreads;
  // by rows: there may be more values than 32 bits count
  for (Place p = {t / (d / 4), t % (d / 4)}; p.r < j.lead; advance(p, d / 4, T / (d / 4), T % (d / 4))) {
    const float z[4] = {0, 0, 0, 0};
    kv_store<TYPE, 4>(out.p, (j.row0 + p.r) * out.row + h * out.head + p.c * 4, z);
  }
  if (j.i1 == 0) return;
  const int64_t at = j.row * out.row + h * out.head;
  const bool there = j.pg >= 0;
  const int64_t head = (there ? j.pg : 0) * C.heads + h;  // read where there is none, and times 0
  const float *scale = (values ? C.vs : C.ks) + head * C.page;
  const uint8_t *src = (values ? C.v : C.k) + head * C.page * (d / 2);
  if (!values) {
    const int per = d / 8, rows = j.i1 - j.i0;
    for (int i0 = t; i0 < rows * per; i0 += T * kAhead) {
      uint32_t w[kAhead];
      float s[kAhead];
#pragma unroll
      for (int y = 0; y < kAhead; ++y) {
        const int i = min(i0 + y * T, rows * per - 1);  // without conditions, so that all are on their way
        w[y] = *reinterpret_cast<const uint32_t *>(src + j.i0 * (d / 2) + i * 4);
        s[y] = scale[j.i0 + i / per];
      }
#pragma unroll
      for (int y = 0; y < kAhead; ++y) {
        const int i = i0 + y * T, r = i / per, c = i - r * per;
        if (i >= rows * per) break;
        float x[8];
        values8<TYPE>(there ? w[y] : 0x88888888u, there ? s[y] : 0.0f, x);
        kv_store<TYPE, 8>(out.p, at + (int64_t)r * out.row + c * 8, x);
      }
    }
    return;
  }
  // 8 tokens of four dims; neighbouring threads take a row's dims, so that rows are written whole
  const int ng = C.page / 8;
  for (int i = t; i < ng * (d / 4); i += T) {
    const int g = i / (d / 4), c = 4 * (i - g * (d / 4));
    if (g * 8 >= j.i1 || g * 8 + 8 <= j.i0) continue;
    uint32_t w[4];
    f32x4 sc[2];
#pragma unroll
    for (int y = 0; y < 4; ++y) w[y] = *reinterpret_cast<const uint32_t *>(src + ((c + y) * C.page + g * 8) / 2);
#pragma unroll
    for (int y = 0; y < 2; ++y) sc[y] = *reinterpret_cast<const f32x4 *>(scale + g * 8 + 4 * y);
#pragma unroll
    for (int y = 0; y < 4; ++y) w[y] = there ? w[y] : 0x88888888u;
#pragma unroll
    for (int z = 0; z < 8; ++z) {
      const int tok = g * 8 + z;
      if (tok < j.i0 || tok >= j.i1) continue;
      const float s = there ? sc[z / 4][z % 4] : 0.0f;
      float x[4];
#pragma unroll
      for (int y = 0; y < 4; ++y) x[y] = value<TYPE>((float)((int)((w[y] >> (4 * z)) & 15u) - 8), s);
      kv_store<TYPE, 4>(out.p, at + (int64_t)(tok - j.i0) * out.row + c, x);
    }
  }
}

}  // namespace

km_status launch_kv_write4(const KvCache &C, const KvSeqs &S, KvRows k, KvRows v, int type, hipStream_t s) {
  const int touched = touched_pages(C, S);
  const size_t lds = (size_t)std::min(C.page, S.max_rows) * (C.d + 4);
  int lanes = 4;
  while (lanes < C.d / 8) lanes *= 2;
  const int64_t blocks = kv_move_blocks(C, S), most = kv_piece(kMoveThreads);
#define KV_GO(T)                                    \
  for (int64_t b = 0; b < blocks; b += most)        \
  kv_write4_kernel<T><<<dim3((unsigned)std::min(most, blocks - b)), kMoveThreads, lds, s>>>(C, S, k, v, touched, lanes, (uint32_t)b)
  if (type == KM_T_F32) KV_GO(KM_T_F32);
  else if (type == KM_T_BF16) KV_GO(KM_T_BF16);
  else KV_GO(KM_T_F16);
#undef KV_GO
  KMQ_LAUNCH_CHECK("kv_write");
  return KM_OK;
}

km_status launch_kv_read4(const KvCache &C, const KvSeqs &S, KvRows k, KvRows v, int type, hipStream_t s) {
  const int touched = touched_pages(C, S);
  const int64_t blocks = kv_move_blocks(C, S), most = kv_piece(kMoveThreads);
#define KV_GO(T)                                    \
  for (int64_t b = 0; b < blocks; b += most)        \
  kv_read4_kernel<T><<<dim3((unsigned)std::min(most, blocks - b)), kMoveThreads, 0, s>>>(C, S, k, v, touched, (uint32_t)b)
  if (type == KM_T_F32) KV_GO(KM_T_F32);
  else if (type == KM_T_BF16) KV_GO(KM_T_BF16);
  else KV_GO(KM_T_F16);
#undef KV_GO
  KMQ_LAUNCH_CHECK("kv_read");
  return KM_OK;
}

}  // namespace kmq
