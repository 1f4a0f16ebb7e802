// Eviction: each sequence and head keeps its tokens of the largest weight and closes the gaps in its pages.
//
// kv_select_kernel, a workgroup for each sequence and head: the K-th largest weight is found digit by digit (11, 11 and
// 10 bits of the weights' ordered bit patterns, a histogram in LDS for each), then one pass in the order of positions writes down
// who stays: all above it, and of those equal to it the first.  Few long sequences take several workgroups to a head and a kernel
// for each of these passes (kv_select_slice_kernel).  kv_gather_kernel, a workgroup for each page that tokens come to:
// builds the page's new contents in the workspace.  kv_scatter_kernel writes them over the page.  In place at once
// a page could be written before another has taken its tokens from it: page t takes from pages t and later.  A page whose tokens
// all stay where they are is left out of both.
//
// Measured: 8 sequences of 4100 tokens, 8 heads of 128 in int8, half of them kept: 12 us to choose (latency: three passes of dependent
// loads and counts), 33 to gather (a chain of loads to each token's page, values a byte at a time, quotients for codes whose page had another
// scale; the vector unit is busy two thirds of the time), 12 to scatter (34 MB each way, 5.5 TB/s).  One sequence of 100001 tokens, 4-bit
// codes, 8192 kept: six kernels of 4 to 8 us to choose, each of them mostly its launch and a chain of three dependent loads, 13 to gather, 5 to
// scatter.  The cache is made whole again between calls, here and below.
#include "kv_pages.hpp"

namespace kmq {
namespace {

constexpr int kSelect = 1024;  // threads
constexpr int kOwn = 8;        // consecutive positions of a thread at a time
constexpr int kBins = 2048;
constexpr int kGather = 256;
constexpr int kStage = 24576;  // bytes of values' pages that a workgroup takes into LDS

struct EvictArgs {
  KvCache C;
  KvSeqs S;
  KvEvict E;
  int tiles;        // pages that tokens may come to, of a sequence
  int *moved;       // [n][heads][tiles]: the page's contents change
  uint8_t *codes;   // [n][heads][tiles][2] pages of codes
  float *scales;    // [n][heads][tiles][2]: of a page (8 bits) or of its tokens
  float *weights;   // [n][heads][tiles][page]
  uint32_t block0;
};

// False: the sequence is left as it is (its length does not fit, or one of its pages is not there).
__device__ __forceinline__ bool evict_len(const KvCache &C, const KvSeqs &S, int b, int *len) {
  *len = S.lens[b];
  return *len >= 0 && (int64_t)*len <= (int64_t)S.max_pages * C.page;
}

// Ordered like the weights: NaN least, then -infinity to infinity.  Whole: counts as more than infinity.
__device__ __forceinline__ uint32_t weight_key(float w, bool whole) {
  const uint32_t u = __float_as_uint(w + 0.0f);  // -0 is 0
  const uint32_t k = w == w ? u ^ ((u >> 31) ? 0xffffffffu : 0x80000000u) : 0u;
  return whole ? 0xffffffffu : k;
}

// The K that a sequence keeps, 0 where it is left as it is, and what does not wait for the choice: the new length, the empty places of
// kept, no page moved.  All kept: their places.  Returns whether there is something to choose.
__device__ __forceinline__ bool select_begin(const EvictArgs &P, int b, int h, int *len, int *K) {
  const KvCache &C = P.C;
  const KvEvict &E = P.E;
  const int t = threadIdx.x;
  const int *table = P.S.table + (int64_t)b * P.S.table_ld;
  int *kept = E.kept + ((int64_t)b * C.heads + h) * E.max_keep;
  int *moved = P.moved + ((int64_t)b * C.heads + h) * P.tiles;
  bool fits = evict_len(C, P.S, b, len);
  if (fits) {
    bool gone = false;
    for (int p = t; p < (*len + C.page - 1) >> C.shift; p += kSelect) gone = gone || table[p] < 0 || table[p] >= C.pages;
    fits = !__syncthreads_or(gone);
  }
  *K = fits ? min(*len, max(0, min(E.keep[b], E.max_keep))) : 0;
  if (h == 0 && t == 0) E.lens[b] = fits ? *K : *len;
  for (int i = t; i < P.tiles; i += kSelect) moved[i] = 0;
  for (int i = *K + t; i < E.max_keep; i += kSelect) kept[i] = -1;
  if (*K < *len) return *K > 0;
  for (int i = t; i < *K; i += kSelect) kept[i] = i;
  return false;
}

// Of bins counters: the digit in which the left-th largest lies, and how many are left to take of it.
__device__ __forceinline__ void find_digit(const uint32_t *hist, int bins, int *digit, int *left, int *wave_sum, uint32_t *found) {
  const int t = threadIdx.x, lane = t & 63, wave = t >> 6;
  const int each = bins / kSelect;  // 2 or 1: thread t has digits bins - 1 - each * t and the ones below it
  int mine = 0;
  for (int i = 0; i < each; ++i) mine += (int)hist[bins - 1 - each * t - i];
  int sum = mine;
#pragma unroll
  for (int o = 1; o < 64; o *= 2) {
    const int y = __shfl_up(sum, o);
    if (lane >= o) sum += y;
  }
  if (lane == 63) wave_sum[wave] = sum;
  __syncthreads();
  int above = sum - mine;
  for (int y = 0; y < wave; ++y) above += wave_sum[y];
  if (above < *left && above + mine >= *left) {
    int i = 0;
    for (; i < each - 1; ++i) {
      const int n = (int)hist[bins - 1 - each * t - i];
      if (above + n >= *left) break;
      above += n;
    }
    found[0] = (uint32_t)(bins - 1 - each * t - i);
    found[1] = (uint32_t)(*left - above);
  }
  __syncthreads();
  *digit = (int)found[0];
  *left = (int)found[1];
  __syncthreads();  // before wave_sum and found are written again
}

__device__ constexpr int kShift[3] = {21, 10, 0}, kBits[3] = {11, 11, 10};

__global__ __launch_bounds__(kSelect) void kv_select_kernel(EvictArgs P) {
  __shared__ uint32_t hist[kBins];
  __shared__ int wave_a[kSelect / 64], wave_b[kSelect / 64];
  __shared__ uint32_t found[2];
  const KvCache &C = P.C;
  const KvEvict &E = P.E;
  const int h = (int)(blockIdx.x % (uint32_t)C.heads), b = (int)(blockIdx.x / (uint32_t)C.heads);
  const int t = threadIdx.x, lane = t & 63, wave = t >> 6;
  int *kept = E.kept + ((int64_t)b * C.heads + h) * E.max_keep;
  int *moved = P.moved + ((int64_t)b * C.heads + h) * P.tiles;
  const int *table = P.S.table + (int64_t)b * P.S.table_ld;
  int len, K;
  if (!select_begin(P, b, h, &len, &K)) return;
  // a thread's next positions j .. j + 7 lie in one page
  auto keys = [&](int j, uint32_t *k) {
    const int pg = table[j >> C.shift];
    const float *w = E.weight + ((int64_t)pg * C.heads + h) * C.page + (j & (C.page - 1));
    const f32x4 a = *reinterpret_cast<const f32x4 *>(w), z = *reinterpret_cast<const f32x4 *>(w + 4);
#pragma unroll
    for (int i = 0; i < kOwn; ++i)
      k[i] = weight_key(i < 4 ? a[i] : z[i - 4], j + i < E.first || j + i >= len - E.recent);
  };
  uint32_t prefix = 0;
  int left = K;  // how many to take of the keys that begin with prefix
#pragma unroll
  for (int pass = 0; pass < 3; ++pass) {
    const int shift = kShift[pass], bins = 1 << kBits[pass];
    for (int i = t; i < bins; i += kSelect) hist[i] = 0;
    __syncthreads();
    for (int j = kOwn * t; j < len; j += kOwn * kSelect) {
      uint32_t k[kOwn];
      keys(j, k);
#pragma unroll
      for (int i = 0; i < kOwn; ++i)
        if (j + i < len && (pass == 0 || k[i] >> (shift + kBits[pass]) == prefix)) atomicAdd(&hist[(k[i] >> shift) & (bins - 1)], 1u);
    }
    __syncthreads();
    int digit;
    find_digit(hist, bins, &digit, &left, wave_a, found);
    prefix = (prefix << kBits[pass]) | (uint32_t)digit;
  }
  // those above the key `prefix`, and the first `left` of those equal to it, in the order of positions
  int more0 = 0, same0 = 0;
  for (int j0 = 0; j0 < len; j0 += kOwn * kSelect) {
    const int j = j0 + kOwn * t;
    uint32_t k[kOwn];
    int more = 0, same = 0;
    if (j < len) {
      keys(j, k);
#pragma unroll
      for (int i = 0; i < kOwn; ++i) {
        more += j + i < len && k[i] > prefix;
        same += j + i < len && k[i] == prefix;
      }
    }
    int ms = more, ss = same;
#pragma unroll
    for (int o = 1; o < 64; o *= 2) {
      const int y = __shfl_up(ms, o), z = __shfl_up(ss, o);
      if (lane >= o) {
        ms += y;
        ss += z;
      }
    }
    if (lane == 63) {
      wave_a[wave] = ms;
      wave_b[wave] = ss;
    }
    __syncthreads();
    int mb = more0 + ms - more, sb = same0 + ss - same;
    for (int y = 0; y < kSelect / 64; ++y) {
      if (y < wave) {
        mb += wave_a[y];
        sb += wave_b[y];
      }
      more0 += wave_a[y];
      same0 += wave_b[y];
    }
    if (j < len) {
#pragma unroll
      for (int i = 0; i < kOwn; ++i) {
        if (j + i >= len) break;
        const bool up = k[i] > prefix, eq = k[i] == prefix;
        if (up || (eq && sb < left)) {
          const int at = mb + min(sb, left);
          kept[at] = j + i;
          if (at != j + i) moved[at >> C.shift] = 1;
        }
        mb += up;
        sb += eq;
      }
    }
    __syncthreads();
  }
}

// ---- few long sequences: the same with `slices` workgroups to a sequence's head, a kernel for each pass -------------------

struct SelectArgs {
  EvictArgs E;
  int slices;
  uint32_t *hist;  // [n * heads][3][kBins], counters of all slices
  int *ends;       // [n * heads][slices][2]: keys above the threshold and equal to it, of each slice
  int *state;      // [n * heads][8]: length, K (0, 0: nothing to choose), then prefix and left after each digit
};
constexpr int kState = 8;

__global__ __launch_bounds__(kSelect) void kv_select_begin_kernel(SelectArgs P) {
  const int bh = (int)blockIdx.x, h = bh % P.E.C.heads, b = bh / P.E.C.heads, t = threadIdx.x;
  int len, K;
  const bool some = select_begin(P.E, b, h, &len, &K);
  if (t < 2) P.state[kState * bh + t] = !some ? 0 : t ? K : len;
  for (int i = t; i < 3 * kBins; i += kSelect) P.hist[(int64_t)bh * 3 * kBins + i] = 0;
}

// PASS 0, 1, 2: counts a digit of the slice's keys.  3: counts its keys above the threshold and equal to it.  4: writes who stays.
template <int PASS>
__global__ __launch_bounds__(kSelect) void kv_select_slice_kernel(SelectArgs P) {
  constexpr int kCopies = 4;  // of each counter, for every fourth lane: lanes that count the same digit wait for each other
  __shared__ uint32_t hist[PASS < 3 ? kBins * kCopies : kSelect / 64 * 2];
  __shared__ int wave_sum[kSelect / 64];
  __shared__ uint32_t found[2];
  const KvCache &C = P.E.C;
  const KvEvict &E = P.E.E;
  const int bh = (int)(blockIdx.x / (uint32_t)P.slices), slice = (int)(blockIdx.x - (uint32_t)bh * P.slices);
  const int t = threadIdx.x, lane = t & 63, wave = t >> 6;
  int *state = P.state + kState * bh;
  const int len = state[0], K = state[1];
  if (K == 0) return;
  const int h = bh % C.heads, b = bh / C.heads;
  const int *table = P.E.S.table + (int64_t)b * P.E.S.table_ld;
  // this slice's positions [s0, s1); each wave has a run of them, 256 at a time
  constexpr int kStep = 4 * 64;
  const int64_t each = cdiv(cdiv(len, P.slices), kStep * (kSelect / 64)) * kStep * (kSelect / 64);
  const int64_t s0 = min(each * slice, (int64_t)len), s1 = min(s0 + each, (int64_t)len);
  const int64_t r0 = min(s0 + each / (kSelect / 64) * wave, s1), r1 = min(r0 + each / (kSelect / 64), s1);
  uint32_t prefix = 0;
  int left = K;
  uint32_t *all = P.hist + (int64_t)bh * 3 * kBins;
  if constexpr (PASS == 4) {
    prefix = (uint32_t)state[6];
    left = state[7];
  } else if constexpr (PASS > 0) {  // the digit that the last kernel counted; earlier ones are known
    constexpr int y = PASS - 1;
    if constexpr (y > 0) {
      prefix = (uint32_t)state[2 * y];
      left = state[2 * y + 1];
    }
    int digit;
    find_digit(all + y * kBins, 1 << kBits[y], &digit, &left, wave_sum, found);
    prefix = (prefix << kBits[y]) | (uint32_t)digit;
    if (slice == 0 && t == 0) {
      state[2 * y + 2] = (int)prefix;
      state[2 * y + 3] = left;
    }
  }
  // the weights of positions j .. j + 3, which lie in one page; behind the end those of the last four
  auto load = [&](int64_t j) {
    const int at = (int)min(j, (int64_t)((len - 1) & ~3));
    const int pg = table[at >> C.shift];
    return *reinterpret_cast<const f32x4 *>(E.weight + ((int64_t)pg * C.heads + h) * C.page + (at & (C.page - 1)));
  };
  auto key = [&](const f32x4 &w, int64_t j, int i) { return weight_key(w[i], j + i < E.first || j + i >= len - E.recent); };
  // f(weights, first position) for this wave's run, with the loads of four steps on their way
  auto each_step = [&](auto f) {
    for (int64_t j0 = r0 + 4 * lane; j0 - 4 * lane < r1; j0 += 4 * kStep) {
      f32x4 w[4];
#pragma unroll
      for (int y = 0; y < 4; ++y) w[y] = load(j0 + y * kStep);
#pragma unroll
      for (int y = 0; y < 4; ++y)
        if (j0 - 4 * lane + y * kStep < r1) f(w[y], j0 + y * kStep);
    }
  };
  if constexpr (PASS < 3) {
    constexpr int shift = kShift[PASS], bins = 1 << kBits[PASS];
    for (int i = t; i < bins * kCopies; i += kSelect) hist[i] = 0;
    __syncthreads();
    each_step([&](const f32x4 &w, int64_t j) {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const uint32_t k = key(w, j, i);
        if (j + i < r1 && (PASS == 0 || k >> (shift + kBits[PASS]) == prefix))
          atomicAdd(&hist[((k >> shift) & (bins - 1)) * kCopies + (lane & (kCopies - 1))], 1u);
      }
    });
    __syncthreads();
    for (int i = t; i < bins; i += kSelect) {
      const uint32_t n = hist[4 * i] + hist[4 * i + 1] + hist[4 * i + 2] + hist[4 * i + 3];
      if (n) atomicAdd(&all[PASS * kBins + i], n);  // whole numbers: in any order the same
    }
    return;
  }
  int more = 0, same = 0;
  each_step([&](const f32x4 &w, int64_t j) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const uint32_t k = key(w, j, i);
      more += j + i < r1 && k > prefix;
      same += j + i < r1 && k == prefix;
    }
  });
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) {
    more += __shfl_xor(more, o);
    same += __shfl_xor(same, o);
  }
  if (lane == 0) {
    hist[2 * wave] = (uint32_t)more;
    hist[2 * wave + 1] = (uint32_t)same;
  }
  __syncthreads();
  int *ends = P.ends + (int64_t)bh * P.slices * 2;
  if constexpr (PASS == 3) {
    if (t < 2) {
      int n = 0;
      for (int y = 0; y < kSelect / 64; ++y) n += (int)hist[2 * y + t];
      ends[2 * slice + t] = n;
    }
    return;
  }
  // what comes before this wave's run
  more = same = 0;
  for (int y = lane; y < slice; y += 64) {
    more += ends[2 * y];
    same += ends[2 * y + 1];
  }
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) {
    more += __shfl_xor(more, o);
    same += __shfl_xor(same, o);
  }
  for (int y = 0; y < wave; ++y) {
    more += (int)hist[2 * y];
    same += (int)hist[2 * y + 1];
  }
  int *kept = E.kept + (int64_t)bh * E.max_keep;
  int *moved = P.E.moved + (int64_t)bh * P.E.tiles;
  each_step([&](const f32x4 &w, int64_t j) {
    uint32_t k[4];
    int here = 0;  // both counts, 16 bits each
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      k[i] = key(w, j, i);
      here += j + i < r1 ? (k[i] > prefix) + (k[i] == prefix ? 1 << 16 : 0) : 0;
    }
    int sum = here;
#pragma unroll
    for (int o = 1; o < 64; o *= 2) {
      const int y = __shfl_up(sum, o);
      if (lane >= o) sum += y;
    }
    int m = more + ((sum - here) & 0xffff), e = same + ((sum - here) >> 16);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const bool up = j + i < r1 && k[i] > prefix, eq = j + i < r1 && k[i] == prefix;
      if (up || (eq && e < left)) {
        const int at = m + min(e, left);
        kept[at] = (int)(j + i);
        if (at != j + i) moved[at >> C.shift] = 1;
      }
      m += up;
      e += eq;
    }
    const int both = __shfl(sum, 63);
    more += both & 0xffff;
    same += both >> 16;
  });
}

struct EvictTile {
  int b, h, tile;
  bool values;
  int64_t bh, to;  // sequence and head; the page's head
  int n;           // tokens that come to the page
};
__device__ __forceinline__ bool evict_tile(const EvictArgs &P, EvictTile *o) {
  uint32_t x = P.block0 + blockIdx.x;
  o->values = x & 1;
  x >>= 1;
  o->h = (int)(x % (uint32_t)P.C.heads);
  x /= (uint32_t)P.C.heads;
  o->tile = (int)(x % (uint32_t)P.tiles);
  o->b = (int)(x / (uint32_t)P.tiles);
  o->bh = (int64_t)o->b * P.C.heads + o->h;
  if (!P.moved[o->bh * P.tiles + o->tile]) return false;  // then the sequence fits, and its pages are there
  o->n = min(P.C.page, P.E.lens[o->b] - (o->tile << P.C.shift));
  o->to = (int64_t)P.S.table[(int64_t)o->b * P.S.table_ld + o->tile] * P.C.heads + o->h;
  return true;
}

// Keys and values by one workgroup: what takes its time is the chain of loads to a token's page.  With one for each, and asked for one after
// the other, a call and its read back take 90 us instead of 82 in the example below, 78 instead of 74 for one sequence of 100001 tokens in 4
// bits.
template <int FMT>
__global__ __launch_bounds__(kGather) void kv_gather_kernel(EvictArgs P) {
  __shared__ int64_t from[128];  // page's head of each slot's token
  __shared__ int tok[128];
  __shared__ float was[2][128];  // keys, values
  __shared__ float top[2][2];
  __shared__ int lpage[128];  // page of the sequence of each slot's token
  __shared__ int64_t pages[128];
  __shared__ __align__(16) uint8_t stage[kStage];
  const KvCache &C = P.C;
  uint32_t x = P.block0 + blockIdx.x;
  const int h = (int)(x % (uint32_t)C.heads);
  x /= (uint32_t)C.heads;
  const int tile = (int)(x % (uint32_t)P.tiles), b = (int)(x / (uint32_t)P.tiles);
  const int t = threadIdx.x, page = C.page, d = C.d;
  const int *table = P.S.table + (int64_t)b * P.S.table_ld;
  const int64_t bh = (int64_t)b * C.heads + h, slot = bh * P.tiles + tile;
  // what does not depend on each other is asked for at once, before it is known whether the page changes
  const int64_t at_kept = ((int64_t)tile << C.shift) + t;
  const int pos_or = t < page && at_kept < P.E.max_keep ? P.E.kept[bh * P.E.max_keep + at_kept] : -1;
  const int own_page = table[tile], left = P.E.lens[b];
  if (!P.moved[slot]) return;  // else the sequence fits, and its pages are there
  const int n = min(page, left - (tile << C.shift));  // tokens that come to the page
  float sk = 0.0f, sv = 0.0f;
  if (t < page) {
    // slots behind the last keep their own
    const bool in = t < n;
    const int pos = in ? pos_or : 0;
    const int64_t f = (int64_t)(in ? table[pos >> C.shift] : own_page) * C.heads + h;
    const int k = in ? pos & (page - 1) : t;
    from[t] = f;
    tok[t] = k;
    lpage[t] = in ? pos >> C.shift : tile;
    if constexpr (FMT == KM_KV_I4) {
      P.scales[2 * slot * page + t] = C.ks[f * page + k];
      P.scales[(2 * slot + 1) * page + t] = C.vs[f * page + k];
    } else {
      sk = C.ks[f];
      sv = C.vs[f];
      was[0][t] = kv_mul_of_scale(sk);
      was[1][t] = kv_mul_of_scale(sv);
      if (!in) sk = sv = 0.0f;
    }
    P.weights[slot * page + t] = P.E.weight[f * page + k];
  }
  float mul[2] = {0.0f, 0.0f};
  bool again[2] = {false, false};
  if constexpr (FMT != KM_KV_I4) {  // the largest scales, in the first two waves
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) {
      sk = fmaxf(sk, __shfl_xor(sk, o));
      sv = fmaxf(sv, __shfl_xor(sv, o));
    }
    if (t < 128 && (t & 63) == 0) {
      top[0][t >> 6] = sk;
      top[1][t >> 6] = sv;
    }
  }
  __syncthreads();
  if constexpr (FMT != KM_KV_I4) {
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const float s = fmaxf(top[i][0], top[i][1]);
      mul[i] = kv_mul_of_scale(s);
      if (t == i) P.scales[2 * slot + i] = s;
      again[i] = __syncthreads_or(t < n && was[i][min(t, page - 1)] > mul[i]);
    }
  }
  const int64_t hb = kv_bytes<FMT>((int64_t)page * d);
  const int db = (int)kv_bytes<FMT>(d);
  uint8_t *out = P.codes + 2 * slot * hb;
  // codes whose multiplier was larger, for the page's
  auto coded = [&](int kind, uint32_t w, int i0, int di) {  // codes of slots i0, i0 + di, ...
    if constexpr (FMT != KM_KV_I4) {
      f16x2 lo, hi;
      kv_widen4<FMT>(w, &lo, &hi);
      float x[4] = {(float)lo.x, (float)lo.y, (float)hi.x, (float)hi.y};
#pragma unroll
      for (int y = 0; y < 4; ++y) x[y] = x[y] * mul[kind] / fmaxf(was[kind][i0 + y * di], mul[kind]);
      const uint32_t z = code4<FMT, KM_T_BF16>(x, 1.0f);
      uint32_t keep = 0;  // what lies behind the last slot
#pragma unroll
      for (int y = 0; y < 4; ++y) keep |= i0 + y * di < n && was[kind][i0 + y * di] > mul[kind] ? 0u : 255u << (8 * y);
      return (w & keep) | (z & ~keep);
    }
    return w;
  };
  const int per = db / 16;
  for (int i = t; i < page * per; i += kGather) {
    const int r = i / per, c = i - r * per;
    u32x4 w = *reinterpret_cast<const u32x4 *>(C.k + from[r] * hb + tok[r] * db + 16 * c);
    if (again[0]) {
#pragma unroll
      for (int y = 0; y < 4; ++y) w[y] = coded(0, w[y], r, 0);
    }
    *reinterpret_cast<u32x4 *>(out + r * db + 16 * c) = w;
  }
  out += hb;
  // Values are taken byte by byte out of rows of `page` bytes.  Where the pages that they come from fit (three of 64 tokens of 128 dims
  // in 8 bits, six in 4; of 128 tokens or 256 dims one and three), those go to LDS in whole lines first.  8 sequences of 4100 tokens, half kept,
  // their pages read back, with and without that: in 4 bits 61 and 64 us; in int8 82 and 77 (the LDS leaves room for six workgroups instead of
  // eight), in pages of 16 115 and 96, but where the sequences have been evicted before, so that most pages change little, 61 and 67.
  // Tokens come in the order of positions, so a page's are neighbours: which of the distinct pages is a slot's
  const int lane = t & 63;
  const bool f0 = lane < page && (lane == 0 || lpage[lane] != lpage[lane - 1]);
  const bool f1 = lane + 64 < page && lpage[lane + 64] != lpage[lane + 63];
  const uint64_t b0 = __ballot(f0), b1 = __ballot(f1);
  const int distinct = __popcll(b0) + __popcll(b1);
  auto nth = [&](int r) {
    return r < 64 ? __popcll(b0 & (~0ull >> (63 - r))) - 1 : __popcll(b0) + __popcll(b1 & (~0ull >> (127 - r))) - 1;
  };
  // 8 slots of a dim, neighbouring threads the slots of a dim's row; a thread's slots stay the same
  const int ng = page / 8, r0 = 8 * (t % ng);
  uint32_t half = 0;  // 4-bit codes: slots whose token is in the high half of its byte
#pragma unroll
  for (int y = 0; y < 8; ++y) half |= (uint32_t)(tok[r0 + y] & 1) << y;
  auto turn = [&](auto byte) {
    for (int c = t / ng; c < d; c += kGather / ng) {
      const int row = (int)kv_bytes<FMT>(c * page);
      uint32_t z[8], w[2] = {0, 0};
#pragma unroll
      for (int y = 0; y < 8; ++y) z[y] = byte(y, row);
      if constexpr (FMT == KM_KV_I4) {
#pragma unroll
        for (int y = 0; y < 8; ++y) w[0] |= ((z[y] >> (half >> y & 1 ? 4 : 0)) & 15u) << (4 * y);
        *reinterpret_cast<uint32_t *>(out + row + r0 / 2) = w[0];
      } else {
#pragma unroll
        for (int y = 0; y < 8; ++y) w[y / 4] |= z[y] << (8 * (y % 4));
        if (again[1]) {
          w[0] = coded(1, w[0], r0, 1);
          w[1] = coded(1, w[1], r0 + 4, 1);
        }
        *reinterpret_cast<u32x2 *>(out + row + r0) = u32x2{w[0], w[1]};
      }
    }
  };
  if (distinct * hb <= kStage) {
    if (t < 64) {
      if (f0) pages[nth(lane)] = from[lane];
      if (f1) pages[nth(lane + 64)] = from[lane + 64];
    }
    __syncthreads();
    const int n16 = (int)hb / 16, total = distinct * n16;
    for (int i0 = t; i0 < total; i0 += 4 * kGather) {
      u32x4 w[4];
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        const int i = min(i0 + u * kGather, total - 1), p = i / n16;
        w[u] = reinterpret_cast<const u32x4 *>(C.v + pages[p] * hb)[i - p * n16];
      }
#pragma unroll
      for (int u = 0; u < 4; ++u)
        if (i0 + u * kGather < total) reinterpret_cast<u32x4 *>(stage)[i0 + u * kGather] = w[u];
    }
    __syncthreads();
    int at[8];
#pragma unroll
    for (int y = 0; y < 8; ++y) at[y] = nth(r0 + y) * (int)hb + (int)kv_bytes<FMT>(tok[r0 + y]);
    turn([&](int y, int row) { return stage[at[y] + row]; });
  } else {
    const uint8_t *at[8];
#pragma unroll
    for (int y = 0; y < 8; ++y) at[y] = C.v + from[r0 + y] * hb + kv_bytes<FMT>(tok[r0 + y]);
    turn([&](int y, int row) { return at[y][row]; });
  }
}

template <int FMT>
__global__ __launch_bounds__(kGather) void kv_scatter_kernel(EvictArgs P) {
  const KvCache &C = P.C;
  EvictTile T;
  if (!evict_tile(P, &T)) return;
  const int t = threadIdx.x, page = C.page;
  const int64_t slot = T.bh * P.tiles + T.tile;
  const int64_t hb = kv_bytes<FMT>((int64_t)page * C.d);
  const u32x4 *in = reinterpret_cast<const u32x4 *>(P.codes + (2 * slot + T.values) * hb);
  u32x4 *out = reinterpret_cast<u32x4 *>((T.values ? C.v : C.k) + T.to * hb);
  for (int i = t; i < hb / 16; i += kGather) out[i] = in[i];
  float *scale = T.values ? C.vs : C.ks;
  if constexpr (FMT == KM_KV_I4) {
    if (t < page) scale[T.to * page + t] = P.scales[(2 * slot + T.values) * page + t];
  } else {
    if (t == 0) scale[T.to] = P.scales[2 * slot + T.values];
  }
  if (!T.values && t < page) P.E.weight[T.to * page + t] = P.weights[slot * page + t];
}

int tiles_of(const KvCache &C, const KvSeqs &S, int max_keep) {
  return (int)std::min<int64_t>(S.max_pages, cdiv(max_keep, C.page));
}

// Workgroups that choose for a sequence's head: one, but for few long sequences.  One workgroup and slices, 8 heads of 128 in 4 bits, 512 tokens
// kept, us of a whole call: one sequence of 24000 tokens 42 and 47, of 32000 48 and 46, of 40000 56 and 49, of 100001 106 and 52; four of
// 40000 67 and 70, of 64000 89 and 75; eight of 32000 72 and 84, of 64000 102 and 94; 16 of 64000 125 and 129, of 100001 165 and 165.
// Slices of 8192 positions instead of 4096: one of 100001 54 instead of 52, four of 64000 66 instead of 75.
int slices_of(const KvCache &C, const KvSeqs &S) {
  const int64_t heads = (int64_t)S.n * C.heads;
  return S.max_len > 32768 + 512 * heads && heads <= 128 ? (int)std::min(cdiv(S.max_len, 4096), 512 / heads) : 1;
}

// Bytes of each part of the workspace, 16-byte aligned.
struct Parts {
  size_t moved, codes, scales, weights, hist, ends, state;
};
Parts parts_of(const KvCache &C, const KvSeqs &S, int max_keep) {
  auto up = [](size_t x) { return (x + 15) & ~(size_t)15; };
  const size_t slots = (size_t)S.n * C.heads * tiles_of(C, S, max_keep);
  const bool i4 = C.fmt == KM_KV_I4;
  const int slices = slices_of(C, S);
  const size_t heads = slices > 1 ? (size_t)S.n * C.heads : 0;
  return {up(4 * slots),        up(2 * slots * C.page * C.d / (i4 ? 2 : 1)), up(8 * slots * (i4 ? C.page : 1)),
          up(4 * slots * C.page), 4 * heads * 3 * kBins,                       up(8 * heads * slices),
          up(4 * heads * kState)};
}

}  // namespace

size_t kv_evict_scratch(const KvCache &C, const KvSeqs &S, int max_keep) {
  const Parts p = parts_of(C, S, max_keep);
  return p.moved + p.codes + p.scales + p.weights + p.hist + p.ends + p.state;
}

int64_t kv_evict_blocks(const KvCache &C, const KvSeqs &S, int max_keep) {
  return (int64_t)2 * S.n * C.heads * tiles_of(C, S, max_keep);
}

km_status launch_kv_evict(const KvCache &C, const KvSeqs &S, const KvEvict &E, void *ws, hipStream_t s) {
  const Parts p = parts_of(C, S, E.max_keep);
  uint8_t *w = static_cast<uint8_t *>(ws);
  EvictArgs P{C, S, E, tiles_of(C, S, E.max_keep), reinterpret_cast<int *>(w), w + p.moved,
              reinterpret_cast<float *>(w + p.moved + p.codes), reinterpret_cast<float *>(w + p.moved + p.codes + p.scales), 0};
  const unsigned heads = (unsigned)(S.n * C.heads);
  if (const int slices = slices_of(C, S); slices > 1) {
    w += p.moved + p.codes + p.scales + p.weights;
    const SelectArgs A{P, slices, reinterpret_cast<uint32_t *>(w), reinterpret_cast<int *>(w + p.hist),
                       reinterpret_cast<int *>(w + p.hist + p.ends)};
    kv_select_begin_kernel<<<dim3(heads), kSelect, 0, s>>>(A);
    kv_select_slice_kernel<0><<<dim3(heads * slices), kSelect, 0, s>>>(A);
    kv_select_slice_kernel<1><<<dim3(heads * slices), kSelect, 0, s>>>(A);
    kv_select_slice_kernel<2><<<dim3(heads * slices), kSelect, 0, s>>>(A);
    kv_select_slice_kernel<3><<<dim3(heads * slices), kSelect, 0, s>>>(A);
    kv_select_slice_kernel<4><<<dim3(heads * slices), kSelect, 0, s>>>(A);
  } else {
    kv_select_kernel<<<dim3(heads), kSelect, 0, s>>>(P);
  }
  KMQ_LAUNCH_CHECK("kv_evict");
  const int64_t blocks = kv_evict_blocks(C, S, E.max_keep), most = kv_piece(kGather);
  auto go = [&](auto *kernel, int64_t blocks) {
    for (int64_t b = 0; b < blocks; b += most) {
      P.block0 = (uint32_t)b;
      kernel<<<dim3((unsigned)std::min(most, blocks - b)), kGather, 0, s>>>(P);
    }
  };
  if (C.fmt == KM_KV_I8) {
    go(kv_gather_kernel<KM_KV_I8>, blocks / 2);
    go(kv_scatter_kernel<KM_KV_I8>, blocks);
  } else if (C.fmt == KM_KV_F8) {
    go(kv_gather_kernel<KM_KV_F8>, blocks / 2);
    go(kv_scatter_kernel<KM_KV_F8>, blocks);
  } else {
    go(kv_gather_kernel<KM_KV_I4>, blocks / 2);
    go(kv_scatter_kernel<KM_KV_I4>, blocks);
  }
  KMQ_LAUNCH_CHECK("kv_evict");
  return KM_OK;
}

}  // namespace kmq
