// What the kernels of the paged cache and of the attention over it share: reading the table, which positions a row sees, the
// operands of the matrix instructions in bf16 and fp32, ragged batches.
#pragma once
#include "common.hpp"
#include "prefill_common.hpp"

namespace parse {

constexpr int KV_MAXSEQ = 4096;              // sequences of a table, prompts or sequences of a call
constexpr int KV_MAXTOKENS = 1 << 25;        // tokens that a table's row can name.  Tiles of them over 4096 rows are more than an int counts: whoever adds those up has a limit of its own

// rows times the heads that share a kv head: tiles of 128 of them stay countable also where offsets go back and forth (2^17 * 4096).  Blocks of 16 that go back and
// forth are not from 2^24 rows and 4095 prompts on: their sum is negative, and such a batch is passed over
constexpr int KV_MAXROWS = 1 << 24;

static inline bool aligned4(const void *p) { return (((uintptr_t)p) & 3u) == 0; }

// host-side checks: counts = the call changes refs and free_bits
int check_kv(const parse_kv *kv, bool counts);
int check_attend(const parse_kv *kv, int layer, const void *q, int64_t q_stride, int n_q, int rows, const int32_t *tok_offsets, const int32_t *seqs, float scale,
                 int window, int sinks, const void *out, int64_t out_stride, const float *lse);

// A word that every lane of the wavefront reads alike, through the scalar cache: it comes without a place in the queue of vector loads, whose
// order the staged tiles count on.
__device__ __forceinline__ int scalar_word(const int32_t *p) { return *(const __attribute__((address_space(4))) int32_t *)(uintptr_t)p; }

// a row's sequence: the table's row and its length; nothing where the number is out of range
struct KvSeq {
  int row, len;
};
__device__ __forceinline__ KvSeq kv_seq(const parse_kv &kv, const int32_t *__restrict__ seqs, int p) {
  const int s = seqs ? seqs[p] : p;
  if (s < 0 || s >= kv.n_seqs) return KvSeq{0, 0};
  return KvSeq{s, min(max(kv.len[s], 0), kv.max_pages * kv.page)};
}

// rows of a prompt, clamped to the batch
struct KvRows {
  int first, n;
};
__device__ __forceinline__ KvRows kv_rows(const int32_t *__restrict__ tok_offsets, int p, int rows) {
  if (!tok_offsets) return KvRows{p, p < rows ? 1 : 0};
  const int a = min(max(tok_offsets[p], 0), rows), b = min(max(tok_offsets[p + 1], 0), rows);
  return KvRows{a, max(b - a, 0)};
}

// Whether a row sees position j: j <= i and j >= lo or j < sinks, with lo the first position of its window.  Without branches: one
// select per score.  i < 0 (a prompt with more rows than its sequence has tokens): a window as long as an int goes would begin below what an int holds
__device__ __forceinline__ int kv_window_begin(int i, int window) { return window > 0 ? max(max(i, 0) - window + 1, 0) : 0; }
__device__ __forceinline__ bool kv_sees(int i, int lo, int sinks, int j) { return (j <= i) & ((j >= lo) | (j < sinks)); }

// ... of positions j0 .. j0 + 7, a bit each
__device__ __forceinline__ uint32_t kv_first_bits(int n) { return (1u << min(max(n, 0), 8)) - 1u; }
__device__ __forceinline__ uint32_t kv_sees8(int i, int lo, int sinks, int j0) {
  return kv_first_bits(i + 1 - j0) & (~kv_first_bits(lo - j0) | kv_first_bits(sinks - j0));
}

// The positions that rows at [i0, i1] see, in tiles of `tile` tokens: the tiles of the sinks, then those from the first
// row's window (all, without one) to i1.  Tile number t of them begins at token at(t) * tile.
struct KvSpan {
  int sink_tiles, skip, count;
  __device__ __forceinline__ int at(int t) const { return t < sink_tiles ? t : t + skip; }
};
__device__ __forceinline__ KvSpan kv_span(int i0, int i1, int window, int sinks, int tile) {
  KvSpan s{0, 0, 0};
  if (i1 < 0) return s;
  const int lo = kv_window_begin(i0, window);
  const int from = lo / tile, to = i1 / tile + 1;
  s.sink_tiles = (int)min(((int64_t)sinks + tile - 1) / tile, (int64_t)from);
  s.skip = from - s.sink_tiles;
  s.count = s.sink_tiles + to - from;
  return s;
}
// sum over the lanes up to this one: within rows of sixteen, then the rows' ends carried on (data moves from lane to lane in the vector unit, without LDS)
__device__ __forceinline__ int wave_scan(int v) {
  v += __builtin_amdgcn_update_dpp(0, v, 0x111, 0xf, 0xf, false);  // row_shr:1
  v += __builtin_amdgcn_update_dpp(0, v, 0x112, 0xf, 0xf, false);  // row_shr:2
  v += __builtin_amdgcn_update_dpp(0, v, 0x114, 0xf, 0xf, false);  // row_shr:4
  v += __builtin_amdgcn_update_dpp(0, v, 0x118, 0xf, 0xf, false);  // row_shr:8
  v += __builtin_amdgcn_update_dpp(0, v, 0x142, 0xa, 0xf, false);  // row_bcast:15, into rows 1 and 3
  v += __builtin_amdgcn_update_dpp(0, v, 0x143, 0xc, 0xf, false);  // row_bcast:31, into rows 2 and 3
  return v;
}

// pre[p] = sum of count(0) .. count(p - 1) for p = 0 .. P, by a whole workgroup; `wave_sums`: one int per wavefront, LDS
template <int THREADS, class F>
__device__ __forceinline__ void kv_prefix(int P, int *pre, int *wave_sums, F count) {
  const int per = (P + THREADS - 1) / THREADS, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  int mine = 0;
  for (int i = 0; i < per; ++i) {
    const int p = tid * per + i;
    if (p < P) { const int c = count(p); pre[p] = mine; mine += c; }
  }
  const int inc = wave_scan(mine);
  if (lane == 63) wave_sums[wave] = inc;
  __syncthreads();
  int base = inc - mine;
  for (int w = 0; w < wave; ++w) base += wave_sums[w];
  for (int i = 0; i < per; ++i) {
    const int p = tid * per + i;
    if (p < P) pre[p] += base;
  }
  if (tid == THREADS - 1) pre[P] = base + mine;
  __syncthreads();
}
// largest p in [0, P) with pre[p] <= v: the element that v belongs to (v < pre[P]; empty ones are passed over)
__device__ __forceinline__ int kv_find(const int *pre, int P, int v) {
  int lo = 0, hi = P - 1;
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (pre[mid] <= v) lo = mid; else hi = mid - 1;
  }
  return lo;
}

// The running maximum of a softmax may lag behind by this much, in powers of two: the sums are multiplied over only where a maximum grows
// by more (the first tile of a row, then hardly ever).  Weights are taken so much below the maximum that they are 1 at most however far it lags: sums reach as
// far as those of a softmax whose maximum is exact, and what falls below the smallest number is 2^-118 of the largest weight.
constexpr float AT_LAG = 8.f;
// Maxima are taken of the products q.k themselves; a weight is then one fused multiply-add and a 2^x.  That needs a positive scale: its
// sign goes to q, and a scale of zero makes q zero (so that a masked score of -inf is never multiplied by 0).
constexpr uint32_t AT_AS_IT_IS = 0, AT_TURNED = 1, AT_ZERO = 2;
static inline void at_scale(float given, float &scale, float &lag, uint32_t &q_sign) {
  scale = fabsf(given) * 1.4426950408889634f;
  q_sign = scale == 0.f ? AT_ZERO : given < 0.f ? AT_TURNED : AT_AS_IT_IS;
  if (scale == 0.f) scale = 1.f;
  lag = fminf(AT_LAG / scale, 3e38f);
}

// x / by for x < 2^24 and by <= 2^16: x * ceil(2^40 / by) >> 40 (x times what the quotient was rounded up by stays below 2^40)
struct KvDivisor {
  uint64_t times;
};
static inline KvDivisor kv_divisor(int by) { return KvDivisor{(((uint64_t)1 << 40) + by - 1) / by}; }
__device__ __forceinline__ int kv_divide(int x, KvDivisor by) { return (int)(((uint64_t)(uint32_t)x * by.times) >> 40); }

// Which prompt an item belongs to, where prompt p has count(rows, sequence) of them, numbered through.
struct KvItem {
  int first, n, row, len, item;                // rows, sequence, number of the item in its prompt; item < 0: there is no such one
};
// A wavefront alone, for up to 64 prompts: a lane reads a prompt's words, all at once.
template <class F>
__device__ __forceinline__ KvItem kv_item_wave(const parse_kv &kv, const int32_t *__restrict__ tok_offsets, const int32_t *__restrict__ seqs, int P, int rows, int item,
                                               F count) {
  const int lane = threadIdx.x & 63, p = min(lane, P - 1);
  const KvRows r = kv_rows(tok_offsets, p, rows);
  const KvSeq s = kv_seq(kv, seqs, p);
  const int mine = lane < P ? count(r, s) : 0, inc = wave_scan(mine);
  const int at = __builtin_amdgcn_readfirstlane(__popcll(__ballot(inc <= item)));    // prompts whose items all lie before
  KvItem f{0, 0, 0, 0, -1};
  if (at >= P) return f;
  f.first = __builtin_amdgcn_readlane(r.first, at);
  f.n = __builtin_amdgcn_readlane(r.n, at);
  f.row = __builtin_amdgcn_readlane(s.row, at);
  f.len = __builtin_amdgcn_readlane(s.len, at);
  f.item = item - (__builtin_amdgcn_readlane(inc, at) - __builtin_amdgcn_readlane(mine, at));
  return f;
}
// A workgroup, for any number; `pre`, `wave_sums`: as for kv_prefix
template <int THREADS, class F>
__device__ __forceinline__ KvItem kv_item(const parse_kv &kv, const int32_t *__restrict__ tok_offsets, const int32_t *__restrict__ seqs, int P, int rows, int item,
                                          int *pre, int *wave_sums, F count) {
  if (P <= 64) return kv_item_wave(kv, tok_offsets, seqs, P, rows, item, count);
  kv_prefix<THREADS>(P, pre, wave_sums, [&](int p) { return count(kv_rows(tok_offsets, p, rows), kv_seq(kv, seqs, p)); });
  KvItem f{0, 0, 0, 0, -1};
  if (item >= pre[P]) return f;
  const int p = __builtin_amdgcn_readfirstlane(kv_find(pre, P, item));
  const KvRows r = kv_rows(tok_offsets, p, rows);
  const KvSeq s = kv_seq(kv, seqs, p);
  f.first = __builtin_amdgcn_readfirstlane(r.first);
  f.n = __builtin_amdgcn_readfirstlane(r.n);
  f.row = __builtin_amdgcn_readfirstlane(s.row);
  f.len = __builtin_amdgcn_readfirstlane(s.len);
  f.item = item - __builtin_amdgcn_readfirstlane(pre[p]);
  return f;
}

// Eight consecutive values of a lane's operand row (columns of K, tokens of V).  bf16: one operand of a 16x16x32 or 32x32x16
// instruction; fp32: eight steps of 16x16x4 or 32x32x2, step e with every lane's value e.  Lane layouts are the same: operand
// row lane % M, the eight reduction indices 8 * (lane / M) + e.
template <class T> struct Op;
template <> struct Op<uint16_t> {
  typedef u32x4 frag;
  static __device__ __forceinline__ frag zero() { return u32x4{0, 0, 0, 0}; }
  static __device__ __forceinline__ frag load(const uint16_t *p) { return *reinterpret_cast<const u32x4 *>(p); }
  static __device__ __forceinline__ frag load_nt(const uint16_t *p) { return __builtin_nontemporal_load(reinterpret_cast<const u32x4 *>(p)); }
  static __device__ __forceinline__ f32x4 mma16(frag a, frag b, f32x4 c) {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(as_bf16x8(a), as_bf16x8(b), c, 0, 0, 0);
  }
  static __device__ __forceinline__ f32x16 mma32(frag a, frag b, f32x16 c) {
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(as_bf16x8(a), as_bf16x8(b), c, 0, 0, 0);
  }
  // q for a scale of either sign (at_scale): the scores' sign turned, or zeros
  static __device__ __forceinline__ frag sign(frag a, uint32_t s) {
#pragma unroll
    for (int w = 0; w < 4; ++w) a[w] = s == AT_ZERO ? 0u : a[w] ^ (s == AT_TURNED ? 0x80008000u : 0u);
    return a;
  }
  // weights in [0, 1]: rounded to bf16, 2^-8 relative at most, independent from token to token
  static __device__ __forceinline__ frag pack(const float *p) {
    return u32x4{cvt_pk_bf16(p[0], p[1]), cvt_pk_bf16(p[2], p[3]), cvt_pk_bf16(p[4], p[5]), cvt_pk_bf16(p[6], p[7])};
  }
  // ... and what that leaves of them, rounded again
  static __device__ __forceinline__ frag pack_rest(const float *p, frag r) {
    float d[8];
#pragma unroll
    for (int w = 0; w < 4; ++w) { d[2 * w] = p[2 * w] - __uint_as_float(r[w] << 16); d[2 * w + 1] = p[2 * w + 1] - __uint_as_float(r[w] & 0xffff0000u); }
    return pack(d);
  }
  // values whose bit of `keep` is clear become 0
  static __device__ __forceinline__ frag only(frag a, uint32_t keep) {
#pragma unroll
    for (int w = 0; w < 4; ++w) a[w] &= (keep >> (2 * w) & 1 ? 0xffffu : 0u) | (keep >> (2 * w + 1) & 1 ? 0xffff0000u : 0u);
    return a;
  }
  // infinities and NaN become the largest finite value of their sign; `most`: largest magnitude so far, in either half
  static __device__ __forceinline__ frag finite_only(frag a, uint32_t &most) {
    typedef __attribute__((ext_vector_type(2))) uint16_t u16x2;
#pragma unroll
    for (int w = 0; w < 4; ++w) {
      const u16x2 size = __builtin_bit_cast(u16x2, a[w] & 0x7fff7fffu);
      most = __builtin_bit_cast(uint32_t, __builtin_elementwise_max(size, __builtin_bit_cast(u16x2, most)));
      a[w] = (a[w] & 0x80008000u) | __builtin_bit_cast(uint32_t, __builtin_elementwise_min(size, u16x2{0x7f7f, 0x7f7f}));
    }
    return a;
  }
  static __device__ __forceinline__ float value(uint16_t b) { return bf16_to_f32(b); }
  static __device__ __forceinline__ bool finite(uint16_t b) { return (b & 0x7f80u) != 0x7f80u; }
  static __device__ __forceinline__ void store4(uint16_t *p, float a, float b, float c, float d) {
    *reinterpret_cast<u32x2 *>(p) = u32x2{cvt_pk_bf16(a, b), cvt_pk_bf16(c, d)};
  }
};
struct f32x8_2 {
  f32x4 lo, hi;
};
template <> struct Op<float> {
  typedef f32x8_2 frag;
  static __device__ __forceinline__ frag zero() { return frag{f32x4{0, 0, 0, 0}, f32x4{0, 0, 0, 0}}; }
  static __device__ __forceinline__ frag load(const float *p) {
    return frag{*reinterpret_cast<const f32x4 *>(p), *reinterpret_cast<const f32x4 *>(p + 4)};
  }
  static __device__ __forceinline__ frag load_nt(const float *p) {
    return frag{__builtin_nontemporal_load(reinterpret_cast<const f32x4 *>(p)), __builtin_nontemporal_load(reinterpret_cast<const f32x4 *>(p + 4))};
  }
  static __device__ __forceinline__ f32x4 mma16(frag a, frag b, f32x4 c) {
#pragma unroll
    for (int e = 0; e < 4; ++e) c = __builtin_amdgcn_mfma_f32_16x16x4f32(a.lo[e], b.lo[e], c, 0, 0, 0);
#pragma unroll
    for (int e = 0; e < 4; ++e) c = __builtin_amdgcn_mfma_f32_16x16x4f32(a.hi[e], b.hi[e], c, 0, 0, 0);
    return c;
  }
  static __device__ __forceinline__ f32x16 mma32(frag a, frag b, f32x16 c) {
#pragma unroll
    for (int e = 0; e < 4; ++e) c = __builtin_amdgcn_mfma_f32_32x32x2f32(a.lo[e], b.lo[e], c, 0, 0, 0);
#pragma unroll
    for (int e = 0; e < 4; ++e) c = __builtin_amdgcn_mfma_f32_32x32x2f32(a.hi[e], b.hi[e], c, 0, 0, 0);
    return c;
  }
  static __device__ __forceinline__ frag sign(frag a, uint32_t s) {
    const float by = s == AT_TURNED ? -1.f : 1.f;
#pragma unroll
    for (int e = 0; e < 4; ++e) { a.lo[e] = s == AT_ZERO ? 0.f : a.lo[e] * by; a.hi[e] = s == AT_ZERO ? 0.f : a.hi[e] * by; }
    return a;
  }
  static __device__ __forceinline__ frag pack(const float *p) { return frag{f32x4{p[0], p[1], p[2], p[3]}, f32x4{p[4], p[5], p[6], p[7]}}; }
  static __device__ __forceinline__ frag only(frag a, uint32_t keep) {
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      a.lo[e] = keep >> e & 1 ? a.lo[e] : 0.f;
      a.hi[e] = keep >> (e + 4) & 1 ? a.hi[e] : 0.f;
    }
    return a;
  }
  // infinities and NaN become 0; true if there was one
  static __device__ __forceinline__ bool finite_only(frag &a) {
    bool bad = false;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      if (!finite(a.lo[e])) { a.lo[e] = 0.f; bad = true; }
      if (!finite(a.hi[e])) { a.hi[e] = 0.f; bad = true; }
    }
    return bad;
  }
  static __device__ __forceinline__ float value(float v) { return v; }
  static __device__ __forceinline__ bool finite(float v) { return (__float_as_uint(v) & 0x7f800000u) != 0x7f800000u; }
  static __device__ __forceinline__ void store4(float *p, float a, float b, float c, float d) { *reinterpret_cast<f32x4 *>(p) = f32x4{a, b, c, d}; }
};

// max / sum with the lane 16 or 32 further on (and back): one lane swap instead of a trip through LDS
template <int N> __device__ __forceinline__ u32x2 lane_swap(float v) {
  const uint32_t u = __float_as_uint(v);
  if constexpr (N == 16) return __builtin_amdgcn_permlane16_swap(u, u, false, false);
  else return __builtin_amdgcn_permlane32_swap(u, u, false, false);
}
template <int N> __device__ __forceinline__ float lane_max(float v) {
  const u32x2 s = lane_swap<N>(v);
  return fmaxf(__uint_as_float(s[0]), __uint_as_float(s[1]));
}
template <int N> __device__ __forceinline__ float lane_sum(float v) {
  const u32x2 s = lane_swap<N>(v);
  return __uint_as_float(s[0]) + __uint_as_float(s[1]);
}

// 2^x of the vector unit: one rounding; below 2^-126 it is 0
__device__ __forceinline__ float at_exp2(float x) { return __builtin_amdgcn_exp2f(x); }
__device__ __forceinline__ float finite_or_0(float m) { return m == -INFINITY ? 0.f : m; }
// what is taken off scale * score (a weight is 2 to what is left), and the log-sum of weights that add up to l
__device__ __forceinline__ float at_base(float m, float scale) { return fmaf(finite_or_0(m), scale, AT_LAG); }
__device__ __forceinline__ float at_lse(float m, float scale, float l) { return (at_base(m, scale) + log2f(l)) * 0.6931471805599453f; }

}  // namespace parse
