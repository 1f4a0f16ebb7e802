// The key/value cache in 8 bits: launch-facing descriptions and the conversions that its kernels share.
#pragma once

#include "common.hpp"

namespace kmq {

typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

// Validated copies of km_kv_cache and km_kv_seqs.
struct KvCache {
  int fmt;
  int page;
  int shift;  // page = 1 << shift
  int heads;
  int d;
  int64_t pages;
  uint8_t *k;  // [pages][heads][page][d]
  uint8_t *v;  // [pages][heads][d][page]
  float *ks;   // [pages][heads]
  float *vs;
};

struct KvSeqs {
  int n;
  int max_pages;
  const int *table;
  int64_t table_ld;
  const int *lens;
  const int *starts;  // nullable: max_rows rows each
  int max_rows;
  int max_len;  // only chooses launch shapes
  int64_t rows;
};

// Rows of a call: [row][head][d], the last axis contiguous.
struct KvRows {
  void *p;
  int64_t row, head;  // strides in elements
};

// The rows of one sequence: its last n positions, ending at len.
struct KvSeq {
  int len;
  int n;
  int64_t row0;
};

// False: the sequence's numbers do not fit the call's (nothing is read or written for it).
__device__ __forceinline__ bool kv_seq(const KvSeqs &S, int page, int b, KvSeq *o) {
  o->len = S.lens[b];
  int64_t r0, r1;
  if (S.starts) {
    r0 = S.starts[b];
    r1 = S.starts[b + 1];
  } else {
    r0 = (int64_t)b * S.max_rows;
    r1 = r0 + S.max_rows;
  }
  o->row0 = r0;
  o->n = (int)(r1 - r0);
  return o->len >= 0 && (int64_t)o->len <= (int64_t)S.max_pages * page && r0 >= 0 && r1 >= r0 && r1 <= S.rows &&
         r1 - r0 <= S.max_rows;
}

// The multiplier x -> code keeps eight significant bits: a 16-bit x times it is exact in fp32, so the rounding to a
// code does not depend on how the product is formed.  The cache holds its inverse, from which it is found again.
__device__ __forceinline__ float kv_short(float x) { return __uint_as_float(__float_as_uint(x) & 0xffff0000u); }
__device__ __forceinline__ float kv_mul_of_top(float top, float qmax) {
  return kv_short(fminf(qmax / top, 0x1p100f));  // top = 0: 2^100
}
__device__ __forceinline__ float kv_mul_of_scale(float s) {
  const float m = kv_short((1.0f / s) * (1.0f + 0x1p-10f));  // a step of 8 bits is 2^-8 of it or more
  return m > 0.0f && m <= 0x1p100f ? m : 0x1p100f;           // a scale that was never written
}

// Four codes of a dword, 8 bits each, as halves: both formats' values are exact in fp16.
template <int FMT>
__device__ __forceinline__ void kv_widen4(uint32_t c, f16x2 *lo, f16x2 *hi) {
  if constexpr (FMT == KM_KV_I8) {
    c ^= 0x80808080u;  // code + 128 in the low byte of 1024's pattern is 1024 + code + 128
    const f16x2 off = {(_Float16)1152.0f, (_Float16)1152.0f};
    *lo = __builtin_bit_cast(f16x2, __builtin_amdgcn_perm(0x64646464u, c, 0x04010400u)) - off;
    *hi = __builtin_bit_cast(f16x2, __builtin_amdgcn_perm(0x64646464u, c, 0x04030402u)) - off;
  } else {
    *lo = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(c, 1.0f, false);
    *hi = __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(c, 1.0f, true);
  }
}

template <int FMT>
__device__ __forceinline__ f16x8 kv_widen8(uint32_t a, uint32_t b) {
  f16x2 x[4];
  kv_widen4<FMT>(a, x, x + 1);
  kv_widen4<FMT>(b, x + 2, x + 3);
  return f16x8{x[0].x, x[0].y, x[1].x, x[1].y, x[2].x, x[2].y, x[3].x, x[3].y};
}

// 16-bit and 32-bit rows
template <int TYPE>
struct KvElem {
  static constexpr int bytes = TYPE == KM_T_F32 ? 4 : 2;
};

template <int TYPE>
__device__ __forceinline__ uint32_t kv_pack2(float a, float b) {
  const f32x2 v = {a, b};
  if constexpr (TYPE == KM_T_BF16)
    return __builtin_bit_cast(uint32_t, __builtin_convertvector(v, bf16x2));
  else
    return __builtin_bit_cast(uint32_t, __builtin_convertvector(v, f16x2));
}

// N values to element offset o (an address aligned to their bytes, 16 at most)
template <int TYPE, int N>
__device__ __forceinline__ void kv_store(void *p, int64_t o, const float *x) {
  if constexpr (TYPE == KM_T_F32) {
    float *q = static_cast<float *>(p) + o;
#pragma unroll
    for (int i = 0; i < N; i += 4) *reinterpret_cast<f32x4 *>(q + i) = f32x4{x[i], x[i + 1], x[i + 2], x[i + 3]};
  } else {
    uint16_t *q = static_cast<uint16_t *>(p) + o;
    if constexpr (N % 8 == 0) {
#pragma unroll
      for (int i = 0; i < N; i += 8)
        *reinterpret_cast<u32x4 *>(q + i) = u32x4{kv_pack2<TYPE>(x[i], x[i + 1]), kv_pack2<TYPE>(x[i + 2], x[i + 3]),
                                                  kv_pack2<TYPE>(x[i + 4], x[i + 5]), kv_pack2<TYPE>(x[i + 6], x[i + 7])};
    } else {
      static_assert(N == 4, "4 values or whole groups of 8");
      *reinterpret_cast<u32x2 *>(q) = u32x2{kv_pack2<TYPE>(x[0], x[1]), kv_pack2<TYPE>(x[2], x[3])};
    }
  }
}

// The most workgroups of one launch: a grid has fewer than 2^32 threads.  What takes more is launched in pieces, of multiples of
// eight so that each keeps the others' order over the XCDs.
static inline int64_t kv_piece(int threads) { return (int64_t)(0xffffffffu / (unsigned)threads) & ~(int64_t)7; }

// kv_cache.hip
int64_t kv_move_blocks(const KvCache &C, const KvSeqs &S);
km_status launch_kv_write(const KvCache &C, const KvSeqs &S, KvRows k, KvRows v, int type, hipStream_t s);
km_status launch_kv_read(const KvCache &C, const KvSeqs &S, KvRows k, KvRows v, int type, hipStream_t s);

// kv_attend.hip
struct KvAttend {
  KvRows q, out;
  int type;
  int group;     // query heads per cache head
  float scale;   // of the products
  int causal;
  int window;    // 0: none
  float *lse;    // nullable, [rows][heads * group]
};
size_t kv_attend_scratch(const KvCache &C, const KvSeqs &S, const KvAttend &A);
// Whether one sequence of the call fits a launch (16-bit rows always do).
bool kv_attend_fits(const KvCache &C, const KvSeqs &S, const KvAttend &A);
int64_t kv_attend_blocks(const KvCache &C, const KvSeqs &S, const KvAttend &A);
km_status launch_kv_attend(const KvCache &C, const KvSeqs &S, const KvAttend &A, void *ws, hipStream_t s);

}  // namespace kmq
