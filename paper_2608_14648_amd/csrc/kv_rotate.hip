// Rotary positions: queries and keys turned by the positions of their rows, before the cache takes them.
//
// Pair (x, y) of a head at position p, frequency f: (x cos pf - y sin pf, x sin pf + y cos pf), times an amplitude.  pf reaches 2^31
// radians, so the turns pf / 2 pi and what is left of them past whole quarters are taken in 64 bits; the rest, at most pi / 4, goes
// to fp32 and into the Taylor polynomials of sine and cosine (degree 9 and 10: below 2^-28 of 1 at pi / 4).  Products and their sums
// are fp32, rounded once.
//
// Bound by HBM: each row is read and written once.  A workgroup takes some rows of a sequence, finds the sine and cosine of each
// row's pairs once (all heads of a row share them, and 64-bit arithmetic for every head would cost more than the row's bytes) and
// keeps them in LDS; a thread then turns VW pairs of a head at a time, in registers, so that rows may be turned in place.
// Measured: 12431 rows of 40 heads of 128 in fp16, 64 dims turned: 43 us for 255 MB, 5.9 TB/s, where the inputs repeat, 64 where they are
// new to the caches.  32 rows: 4.3 us, one row to a workgroup.
#include "kv.hpp"

namespace kmq {
namespace {

constexpr int kThreads = 256;
constexpr int kMostPairs = 512;  // sines and cosines of a workgroup's rows

struct RotateArgs {
  KvRotate R;
  int tr;     // rows of a workgroup
  int tiles;  // workgroups of a sequence
  uint32_t block0;
};

// sine and cosine of `turns` turns
__device__ __forceinline__ float2 turned(double turns) {
  const double quarters = rint(4.0 * turns);
  const float a = (float)((turns - 0.25 * quarters) * 6.283185307179586476925);
  const int quad = (int)((long long)quarters & 3);
  const float z = a * a;
  float s = fmaf(z, 2.75573192e-6f, -1.98412698e-4f);  // 1 / 9!, 1 / 7!
  s = fmaf(z, s, 8.33333333e-3f);
  s = fmaf(z, s, -1.66666667e-1f);
  s = fmaf(a * z, s, a);
  float c = fmaf(z, -2.75573192e-7f, 2.48015873e-5f);  // 1 / 10!, 1 / 8!
  c = fmaf(z, c, -1.38888889e-3f);
  c = fmaf(z, c, 4.16666667e-2f);
  c = fmaf(z, c, -0.5f);
  c = fmaf(z, c, 1.0f);
  const float sn = quad & 1 ? c : s, cn = quad & 1 ? s : c;
  return float2{quad & 2 ? -sn : sn, (quad + 1) & 2 ? -cn : cn};
}

// N values of a row, from and to memory in pieces of at most 16 bytes
template <int TYPE, int N>
struct Vec {
  static constexpr int bytes = N * KvElem<TYPE>::bytes;
  static constexpr int words = bytes >= 4 ? bytes / 4 : 1;
  uint32_t w[words];
  __device__ __forceinline__ void load(const void *p, int64_t o) {
    const char *a = static_cast<const char *>(p) + o * KvElem<TYPE>::bytes;
    if constexpr (bytes >= 16) {
#pragma unroll
      for (int i = 0; i < words; i += 4) *reinterpret_cast<u32x4 *>(w + i) = *reinterpret_cast<const u32x4 *>(a + 4 * i);
    } else if constexpr (bytes == 8) {
      *reinterpret_cast<u32x2 *>(w) = *reinterpret_cast<const u32x2 *>(a);
    } else if constexpr (bytes == 4) {
      w[0] = *reinterpret_cast<const uint32_t *>(a);
    } else {
      w[0] = *reinterpret_cast<const uint16_t *>(a);
    }
  }
  __device__ __forceinline__ void store(void *p, int64_t o) const {
    char *a = static_cast<char *>(p) + o * KvElem<TYPE>::bytes;
    if constexpr (bytes >= 16) {
#pragma unroll
      for (int i = 0; i < words; i += 4) *reinterpret_cast<u32x4 *>(a + 4 * i) = u32x4{w[i], w[i + 1], w[i + 2], w[i + 3]};
    } else if constexpr (bytes == 8) {
      *reinterpret_cast<u32x2 *>(a) = u32x2{w[0], w[1]};
    } else if constexpr (bytes == 4) {
      *reinterpret_cast<uint32_t *>(a) = w[0];
    } else {
      *reinterpret_cast<uint16_t *>(a) = (uint16_t)w[0];
    }
  }
  __device__ __forceinline__ float get(int i) const {
    if constexpr (TYPE == KM_T_F32) return __uint_as_float(w[i]);
    const uint32_t h = w[i / 2] >> (16 * (i % 2));
    if constexpr (TYPE == KM_T_BF16) return __uint_as_float(h << 16);
    return (float)__builtin_bit_cast(_Float16, (uint16_t)h);
  }
  __device__ __forceinline__ void set(const float *x) {
    if constexpr (TYPE == KM_T_F32) {
#pragma unroll
      for (int i = 0; i < N; ++i) w[i] = __float_as_uint(x[i]);
    } else {
#pragma unroll
      for (int i = 0; i < N; i += 2) w[i / 2] = kv_pack2<TYPE>(x[i], i + 1 < N ? x[i + 1] : 0.0f);
    }
  }
};

template <int TYPE, int VW>
__global__ __launch_bounds__(kThreads) void kv_rotate_kernel(RotateArgs P) {
  __shared__ float2 cs[kMostPairs];
  const KvRotate &R = P.R;
  const uint32_t x = P.block0 + blockIdx.x;
  const int t = threadIdx.x, pairs = R.dims / 2;
  int64_t row0, at;  // first row and its position
  int nr;
  if (R.positions) {
    row0 = (int64_t)x * P.tr;
    nr = (int)min((int64_t)P.tr, R.rows - row0);
    at = 0;
  } else {
    const int b = (int)(x / (uint32_t)P.tiles), first = (int)(x - (uint32_t)b * P.tiles) * P.tr;
    KvSeq q;
    if (!kv_seq(R.S, 1 << 30, b, &q)) return;
    nr = min(P.tr, q.n - first);
    row0 = q.row0 + first;
    at = (int64_t)q.len - q.n + first;
  }
  if (nr <= 0) return;
  const int units = R.d / (2 * VW), heads = R.q_heads + R.k_heads;  // a unit: VW pairs, or what is copied of as many
  const int total = nr * heads * units;
  struct Unit {
    Vec<TYPE, VW> a, b;
    int64_t to;
    int i0, i1, z;  // places of a and b in the row; of their sines, -1: copied
    bool key;
  };
  auto load = [&](int i) {
    Unit u;
    const int rh = i / units, c = i - rh * units;
    const int r = rh / heads;
    int h = rh - r * heads;
    u.key = h >= R.q_heads;
    h -= u.key ? R.q_heads : 0;
    const KvRows &in = u.key ? R.k : R.q, &out = u.key ? R.k_out : R.q_out;
    const int64_t from = (row0 + r) * in.row + h * in.head;
    u.to = (row0 + r) * out.row + h * out.head;
    const bool turn = c * VW < pairs;
    u.z = turn ? r * pairs + c * VW : -1;
    u.i0 = turn && !R.neighbours ? c * VW : 2 * c * VW;
    u.i1 = turn && !R.neighbours ? u.i0 + pairs : u.i0 + VW;
    u.a.load(in.p, from + u.i0);
    u.b.load(in.p, from + u.i1);
    return u;
  };
  // the first rows are on their way while the angles are worked out, later ones while others are turned
  Unit next;
  if (t < total) next = load(t);
  for (int i = t; i < nr * pairs; i += kThreads) {
    const int r = i / pairs, p = i - r * pairs;
    const int64_t pos = R.positions ? R.positions[row0 + r] : at + r;
    float2 z = turned((double)pos * (R.freq[p] * 0.159154943091895335769));
    cs[i] = float2{(R.inverse ? -z.x : z.x) * R.amplitude, z.y * R.amplitude};
  }
  __syncthreads();
  for (int i = t; i < total; i += kThreads) {
    Unit w = next;
    if (i + kThreads < total) next = load(i + kThreads);
    if (w.z < 0 && (w.key ? R.k_in_place : R.q_in_place)) continue;
    if (w.z >= 0) {
      const float2 *z = cs + w.z;
      float u[VW], v[VW];
      if (!R.neighbours) {
#pragma unroll
        for (int y = 0; y < VW; ++y) {
          const float p = w.a.get(y), q = w.b.get(y);
          u[y] = fmaf(p, z[y].y, -(q * z[y].x));
          v[y] = fmaf(p, z[y].x, q * z[y].y);
        }
      } else {
        float o[2 * VW];
#pragma unroll
        for (int y = 0; y < VW; ++y) {
          o[y] = w.a.get(y);
          o[VW + y] = w.b.get(y);
        }
#pragma unroll
        for (int y = 0; y < VW; ++y) {
          const float p = o[2 * y], q = o[2 * y + 1];
          o[2 * y] = fmaf(p, z[y].y, -(q * z[y].x));
          o[2 * y + 1] = fmaf(p, z[y].x, q * z[y].y);
        }
#pragma unroll
        for (int y = 0; y < VW; ++y) {
          u[y] = o[y];
          v[y] = o[VW + y];
        }
      }
      w.a.set(u);
      w.b.set(v);
    }
    void *out = w.key ? R.k_out.p : R.q_out.p;
    w.a.store(out, w.to + w.i0);
    w.b.store(out, w.to + w.i1);
  }
}

// Rows of a workgroup: as many as fill its threads with pairs, one where the call then has fewer workgroups than there are CUs.
int tile_rows(const KvRotate &R) {
  const int64_t rows = R.positions ? R.rows : std::min<int64_t>(R.S.rows, (int64_t)R.S.n * R.S.max_rows);
  const int most = std::max(1, std::min(8, kMostPairs / (R.dims / 2)));
  return (int)std::max<int64_t>(1, std::min<int64_t>(most, rows / 512));
}

}  // namespace

int64_t kv_rotate_blocks(const KvRotate &R) {
  const int tr = tile_rows(R);
  return R.positions ? cdiv(R.rows, tr) : (int64_t)R.S.n * cdiv(R.S.max_rows, tr);
}

km_status launch_kv_rotate(const KvRotate &R, int type, hipStream_t s) {
  RotateArgs P{R, tile_rows(R), 0, 0};
  P.tiles = R.positions ? 1 : (int)cdiv(R.S.max_rows, P.tr);
  const int64_t blocks = kv_rotate_blocks(R), most = kv_piece(kThreads);
  const int pairs = R.dims / 2;
  auto go = [&](auto *kernel) {
    for (int64_t b = 0; b < blocks; b += most) {
      P.block0 = (uint32_t)b;
      kernel<<<dim3((unsigned)std::min(most, blocks - b)), kThreads, 0, s>>>(P);
    }
  };
#define KV_V(T)                                    \
  if (pairs % 8 == 0) go(kv_rotate_kernel<T, 8>);  \
  else if (pairs % 4 == 0) go(kv_rotate_kernel<T, 4>); \
  else if (pairs % 2 == 0) go(kv_rotate_kernel<T, 2>); \
  else go(kv_rotate_kernel<T, 1>);
  if (type == KM_T_F32) {
    KV_V(KM_T_F32)
  } else if (type == KM_T_BF16) {
    KV_V(KM_T_BF16)
  } else {
    KV_V(KM_T_F16)
  }
#undef KV_V
  KMQ_LAUNCH_CHECK("kv_rotate");
  return KM_OK;
}

}  // namespace kmq
