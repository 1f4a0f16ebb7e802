// Writing keys and values into the 8-bit cache and reading them back.
//
// A page (a block of tokens of one head) has one scale, so one workgroup owns the page for the call: it finds the largest
// magnitude of the rows that the call writes there, takes the smaller multiplier of that and of the tokens already in the
// page, and codes the rows; if the multiplier shrank, the earlier tokens' codes are coded again.  Keys and values
// are different workgroups.  Values lie with their dims first (the attention's second product contracts tokens), so
// their codes turn through LDS on the way in and in registers on the way out.
//
// Both are bound by HBM: 3 bytes per 16-bit element, 4.6 and 5.7 TB/s for 74631 tokens of 8 heads of 128 (100 and 80 us;
// a large copy 4.7); fp32 rows, 82674 tokens, 5.6 and 4.1 TB/s (152 and 207 us).  One token: 3.1 and 3.7 us.  The rows of a page are read once and kept in registers (a
// workgroup has as many threads as that takes), its largest magnitude is taken on the bit patterns, and only a page that
// holds infinities or NaN looks at them one by one.
#include "kv_pages.hpp"

namespace kmq {
namespace {

constexpr int kItems = 4;  // groups of 8 values that a thread holds

template <int FMT, int TYPE>
__global__ __launch_bounds__(1024) void kv_write_kernel(KvCache C, KvSeqs S, KvRows kr, KvRows vr, int touched,
                                                        uint32_t block0) {
  extern __shared__ uint32_t turn[];  // values: codes of the new rows, [token][turn_ld]
  __shared__ uint32_t sh[16];
  bool values;
  int h;
  PageJob j;
  if (!page_job(C, S, block0 + blockIdx.x, touched, &values, &h, &j) || j.i1 == 0 || j.pg < 0) return;
  const KvRows &src = values ? vr : kr;
  const int d = C.d, t = threadIdx.x, T = blockDim.x;
  const int per = d / 8, rows = j.i1 - j.i0;  // items of 8 dims in a row
  const int64_t at = j.row * src.row + h * src.head;
  float *scale = (values ? C.vs : C.ks) + j.pg * C.heads + h;
  const float s_old = j.i0 ? *scale : 0.0f;

  const int dr = T / per, dc = T % per;
  const Place first = {t / per, t % per};
  Place p = first;
  Raw<TYPE> raw[kItems];
  uint32_t m = 0;
#pragma unroll
  for (int i = 0; i < kItems; ++i) {
    if (p.r < rows) {
      raw[i] = raw_load<TYPE>(src.p, at + (int64_t)p.r * src.row + p.c * 8);
    } else {
#pragma unroll
      for (int y = 0; y < (TYPE == KM_T_F32 ? 2 : 1); ++y) raw[i].w[y] = u32x4{0, 0, 0, 0};
    }
    advance(p, per, dr, dc);
  }
#pragma unroll
  for (int i = 0; i < kItems; ++i)
#pragma unroll
    for (int y = 0; y < (TYPE == KM_T_F32 ? 8 : 4); ++y) m = raw_max<TYPE>(m, raw[i].w[y / 4][y % 4]);
  if constexpr (TYPE != KM_T_F32) m = max(m & 0xffffu, m >> 16);
  m = block_max(m, sh);
  const bool wild = m >= kInf<TYPE>;  // infinities or NaN among the rows
  if (wild) {
    uint32_t top = 0;
#pragma unroll
    for (int i = 0; i < kItems; ++i) {
      float x[8];
      raw_values<TYPE>(raw[i], x);
#pragma unroll
      for (int y = 0; y < 8; ++y) {
        const uint32_t a = __float_as_uint(x[y]) & 0x7fffffffu;
        top = a < 0x7f800000u ? max(top, a) : top;
      }
    }
    m = block_max(top, sh);
  } else if constexpr (TYPE == KM_T_BF16) {
    m <<= 16;
  } else if constexpr (TYPE == KM_T_F16) {
    m = __float_as_uint((float)__builtin_bit_cast(f16x2, m).x);
  }
  const float top = __uint_as_float(m);
  float mul = kv_mul_of_top(top, kQmax<FMT>);
  bool again = false;
  float was = 0.0f;
  if (j.i0) {
    was = kv_mul_of_scale(s_old);
    again = mul < was;
    mul = fminf(mul, was);
  }
  if (T > 64) __syncthreads();  // every wave has read the scale
  if (t == 0) *scale = 1.0f / mul;

  uint8_t *dst = (values ? C.v : C.k) + (j.pg * C.heads + h) * (int64_t)C.page * d;
  const int ld = turn_ld(d);
  p = first;
#pragma unroll
  for (int i = 0; i < kItems; ++i) {
    if (p.r < rows) {
      float x[8];
      raw_values<TYPE>(raw[i], x);
      if (wild) {
#pragma unroll
        for (int u = 0; u < 8; ++u) x[u] = tame(x[u], top);
      }
      const u32x2 q = {code4<FMT, TYPE>(x, mul), code4<FMT, TYPE>(x + 4, mul)};
      if (values) {
        uint32_t *w = turn + (p.r * ld + p.c * 8) / 4;
        w[0] = q.x;
        w[1] = q.y;
      } else {
        *reinterpret_cast<u32x2 *>(dst + (j.i0 + p.r) * d + p.c * 8) = q;
      }
    }
    advance(p, per, dr, dc);
  }
  if (!values) {
    if (again) {
      u32x4 *o = reinterpret_cast<u32x4 *>(dst);
      for (int i = t; i < j.i0 * d / 16; i += T) {
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
  if (!again && rows < 16) {  // a few tokens: their bytes alone
    for (int r = 0; r < rows; ++r)
      for (int c = t; c < d; c += T) dst[c * C.page + j.i0 + r] = tb[r * ld + c];
    return;
  }
  // 16 tokens of four dims at a time, neighbouring threads the tokens of a dim's row.  What lies in a group before i0 is
  // coded again or stays, what lies behind i1 stays.
  const int ng = C.page / 16;
  for (int i = t; i < ng * (d / 4); i += T) {
    int g, c;
    group_of(i, ng, d / 4, &g, &c);
    const int k0 = g * 16 - j.i0;  // row of its first token
    if (g * 16 >= j.i1 || (!again && g * 16 + 16 <= j.i0)) continue;
    uint8_t *o = dst + c * C.page + g * 16;
    uint32_t w[4][4];  // [dim][four tokens]
    if (k0 >= 0 && k0 + 16 <= rows) {
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        uint32_t a[4], b[4];
#pragma unroll
        for (int y = 0; y < 4; ++y) a[y] = turn[((k0 + 4 * u + y) * ld + c) / 4];
        turn4(a, b);
#pragma unroll
        for (int y = 0; y < 4; ++y) w[y][u] = b[y];
      }
    } else {
#pragma unroll
      for (int y = 0; y < 4; ++y) {
        const u32x4 x = *reinterpret_cast<const u32x4 *>(o + y * C.page);
#pragma unroll
        for (int u = 0; u < 4; ++u) {
          const uint32_t old = again ? recode4<FMT>(x[u], mul, was) : x[u];
          uint32_t n = 0;
#pragma unroll
          for (int z = 0; z < 4; ++z) {
            const int k = k0 + 4 * u + z;
            const uint32_t keep = ((k < 0 ? old : x[u]) >> (8 * z)) & 255u;
            n |= (k >= 0 && k < rows ? (uint32_t)tb[k * ld + c + y] : keep) << (8 * z);
          }
          w[y][u] = n;
        }
      }
    }
#pragma unroll
    for (int y = 0; y < 4; ++y) *reinterpret_cast<u32x4 *>(o + y * C.page) = u32x4{w[y][0], w[y][1], w[y][2], w[y][3]};
  }
}

template <int FMT, int TYPE>
__global__ __launch_bounds__(1024) void kv_read_kernel(KvCache C, KvSeqs S, KvRows kr, KvRows vr, int touched,
                                                       uint32_t block0) {
  bool values;
  int h;
  PageJob j;
  if (!page_job(C, S, block0 + blockIdx.x, touched, &values, &h, &j)) return;
  const KvRows &out = values ? vr : kr;
  const int d = C.d, t = threadIdx.x, T = blockDim.x;
  // by rows: there may be more values than 32 bits count
  for (Place p = {t / (d / 4), t % (d / 4)}; p.r < j.lead; advance(p, d / 4, T / (d / 4), T % (d / 4))) {
    const float z[4] = {0, 0, 0, 0};
    kv_store<TYPE, 4>(out.p, (j.row0 + p.r) * out.row + h * out.head + p.c * 4, z);
  }
  if (j.i1 == 0) return;
  const int64_t at = j.row * out.row + h * out.head;
  const bool there = j.pg >= 0;
  const int64_t pg = there ? j.pg : 0;  // read where there is none, and times 0
  const float s = there ? (values ? C.vs : C.ks)[pg * C.heads + h] : 0.0f;
  const uint8_t *src = (values ? C.v : C.k) + (pg * C.heads + h) * (int64_t)C.page * d;
  if (!values) {
    const int per = d / 8, rows = j.i1 - j.i0, dr = T / per, dc = T % per;
    Place p = {t / per, t % per};
    u32x2 w[kItems];
    Place f = p;
#pragma unroll
    for (int i = 0; i < kItems; ++i) {
      w[i] = u32x2{0, 0};
      if (f.r < rows && there) w[i] = *reinterpret_cast<const u32x2 *>(src + (j.i0 + f.r) * d + f.c * 8);
      advance(f, per, dr, dc);
    }
#pragma unroll
    for (int i = 0; i < kItems; ++i) {
      if (p.r < rows) {
        float x[8];
#pragma unroll
        for (int u = 0; u < 2; ++u) {
          f16x2 lo, hi;
          kv_widen4<FMT>(w[i][u], &lo, &hi);
          x[4 * u] = value<TYPE>((float)lo.x, s);
          x[4 * u + 1] = value<TYPE>((float)lo.y, s);
          x[4 * u + 2] = value<TYPE>((float)hi.x, s);
          x[4 * u + 3] = value<TYPE>((float)hi.y, s);
        }
        kv_store<TYPE, 8>(out.p, at + (int64_t)p.r * out.row + p.c * 8, x);
      }
      advance(p, per, dr, dc);
    }
    return;
  }
  // 16 tokens of four dims: four loads, sixteen rows of four values.  Neighbouring threads take a row's dims, so that rows are
  // written whole; the codes of a dim's row are read from L1 again (69 thousand tokens of 8 heads of 96: 69 us,
  // with the tokens of a dim's row on neighbouring threads 90).
  const int ng = C.page / 16;
  for (int i = t; i < ng * (d / 4); i += T) {
    const int g = i / (d / 4), c = 4 * (i - g * (d / 4));
    if (g * 16 >= j.i1 || g * 16 + 16 <= j.i0) continue;
    u32x4 w[4];
#pragma unroll
    for (int y = 0; y < 4; ++y) {
      w[y] = u32x4{0, 0, 0, 0};
      if (there) w[y] = *reinterpret_cast<const u32x4 *>(src + (c + y) * C.page + g * 16);
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

// Threads that hold a page's rows, as many as the call can bring there.
int move_threads(const KvCache &C, const KvSeqs &S) {
  const int items = std::min(C.page, S.max_rows) * (C.d / 8);
  return std::min(1024, std::max(64, (int)cdiv(cdiv(items, kItems), 64) * 64));
}

}  // namespace

int64_t kv_move_blocks(const KvCache &C, const KvSeqs &S) {
  return cdiv((int64_t)S.n * touched_pages(C, S), 8) * 8 * 2 * C.heads;
}

km_status launch_kv_write(const KvCache &C, const KvSeqs &S, KvRows k, KvRows v, int type, hipStream_t s) {
  const int touched = touched_pages(C, S);
  const size_t lds = (size_t)std::min(C.page, S.max_rows) * (C.d + 4);
  const int threads = move_threads(C, S);
  const int64_t blocks = kv_move_blocks(C, S), most = kv_piece(threads);
#define KV_GO(F, T)                                       \
  for (int64_t b = 0; b < blocks; b += most)              \
  kv_write_kernel<F, T><<<dim3((unsigned)std::min(most, blocks - b)), threads, lds, s>>>(C, S, k, v, touched, (uint32_t)b)
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
  const int threads = move_threads(C, S);
  const int64_t blocks = kv_move_blocks(C, S), most = kv_piece(threads);
#define KV_GO(F, T)                                       \
  for (int64_t b = 0; b < blocks; b += most)              \
  kv_read_kernel<F, T><<<dim3((unsigned)std::min(most, blocks - b)), threads, 0, s>>>(C, S, k, v, touched, (uint32_t)b)
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
