// Which pages of a cache a new token reads: bounds of the pages' keys (parse_kv_bounds), scores from them and the best pages (parse_select_pages).
#include <algorithm>

#include "attend.hpp"

namespace parse {

constexpr int SP_THREADS = 256, SP_WAVES = SP_THREADS / 64;

// ---- bounds ----------------------------------------------------------------------------------------------------------
struct KbArgs {
  parse_kv kv;
  const void *K;
  void *bounds;                                      // of the first layer: [page][head][2][d]
  const int32_t *tok_offsets, *seqs;
  int P, layers;
  int64_t k_layer, b_layer;                          // elements
};

// smaller / larger of two, NaN if one of them is
__device__ __forceinline__ float kb_min(float a, float b) { return __builtin_elementwise_minimum(a, b); }
__device__ __forceinline__ float kb_max(float a, float b) { return __builtin_elementwise_maximum(a, b); }

// A wavefront has a page of one head: a load brings 64 pieces of eight columns, lane % 16 the token, so that the block's 16 tokens are the lanes of a row.
template <class T, int DT>
__global__ __launch_bounds__(SP_THREADS) void kv_bounds(KbArgs a) {
  constexpr int D = DT * 32;
  extern __shared__ int pre[];
  int *wave_sums = pre + a.P + 1;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, page = a.kv.page;
  const int heads = a.kv.n_kv * a.layers, per = (heads + SP_WAVES - 1) / SP_WAVES;
  for (int64_t w = blockIdx.x;; w += gridDim.x) {
    const int64_t number = w / per;
    if (number > 0x7fffffff) return;
    const KvItem f = kv_item<SP_THREADS>(a.kv, a.tok_offsets, a.seqs, a.P, 0x7fffffff, (int)number, pre, wave_sums,
                                         [&](const KvRows &r, const KvSeq &s) { return s.len / page - max(s.len - r.n, 0) / page; });
    if (f.item < 0) return;
    const int c = max(f.len - f.n, 0) / page + f.item, lh = (int)(w % per) * SP_WAVES + wave;
    const int id = a.kv.table[(int64_t)f.row * a.kv.max_pages + c];
    if (lh < heads && id >= 0 && id < a.kv.n_pages) {
      const int layer = lh / a.kv.n_kv, head = lh % a.kv.n_kv;
      const T *k = reinterpret_cast<const T *>(a.K) + layer * a.k_layer + ((int64_t)id * a.kv.n_kv + head) * page * D + lane * 8;
      float lo[DT][8], hi[DT][8];
#pragma unroll
      for (int p = 0; p < DT; ++p)
#pragma unroll
        for (int e = 0; e < 8; ++e) { lo[p][e] = INFINITY; hi[p][e] = -INFINITY; }
      for (int b = 0; b < page / 16; ++b) {
        float v[DT][8];
#pragma unroll
        for (int p = 0; p < DT; ++p) {
          const typename Op<T>::frag x = Op<T>::load(k + b * 16 * D + p * 512);
          if constexpr (sizeof(T) == 2) {
#pragma unroll
            for (int e = 0; e < 4; ++e) { v[p][2 * e] = __uint_as_float(x[e] << 16); v[p][2 * e + 1] = __uint_as_float(x[e] & 0xffff0000u); }
          } else {
#pragma unroll
            for (int e = 0; e < 4; ++e) { v[p][e] = x.lo[e]; v[p][4 + e] = x.hi[e]; }
          }
        }
#pragma unroll
        for (int p = 0; p < DT; ++p)
#pragma unroll
          for (int e = 0; e < 8; ++e) { lo[p][e] = kb_min(lo[p][e], v[p][e]); hi[p][e] = kb_max(hi[p][e], v[p][e]); }
      }
#pragma unroll
      for (int o = 8; o > 0; o >>= 1)
#pragma unroll
        for (int p = 0; p < DT; ++p)
#pragma unroll
          for (int e = 0; e < 8; ++e) { lo[p][e] = kb_min(lo[p][e], __shfl_xor(lo[p][e], o, 64)); hi[p][e] = kb_max(hi[p][e], __shfl_xor(hi[p][e], o, 64)); }
      T *to = reinterpret_cast<T *>(a.bounds) + layer * a.b_layer + ((int64_t)id * a.kv.n_kv + head) * 2 * D;
      if ((lane & 15) == 0) {
#pragma unroll
        for (int p = 0; p < DT; ++p) {
          T *t = to + (p * 4 + (lane >> 4)) * 8;
          Op<T>::store4(t, lo[p][0], lo[p][1], lo[p][2], lo[p][3]);
          Op<T>::store4(t + 4, lo[p][4], lo[p][5], lo[p][6], lo[p][7]);
          Op<T>::store4(t + D, hi[p][0], hi[p][1], hi[p][2], hi[p][3]);
          Op<T>::store4(t + D + 4, hi[p][4], hi[p][5], hi[p][6], hi[p][7]);
        }
      }
    }
    if (a.P > 64) __syncthreads();                                 // the prompts' sums are made anew
  }
}

// ---- scores ----------------------------------------------------------------------------------------------------------
struct SpArgs {
  parse_kv kv;
  const void *bounds, *q;                            // of the layer
  const int32_t *seqs;
  int64_t q_stride;
  int n_q, group, rows, top, first, last;
  uint64_t *keys;                                    // [row][head][max_pages]
  int32_t *sel;
};

// Doubles in their order as unsigned numbers; NaN is the largest, whatever its sign
__device__ __forceinline__ uint64_t sp_key(double v) {
  const int64_t b = __double_as_longlong(v);
  if (v != v) return ~0ull;
  return v == 0.0 ? 1ull << 63 : (uint64_t)(b ^ ((b >> 63) | (int64_t)(1ull << 63)));
}

// Columns of the table that are scored: [first, n - last) of n
struct SpCols {
  int n, begin, end;
};
__device__ __forceinline__ SpCols sp_cols(const SpArgs &a, int len) {
  const int n = (len + a.kv.page - 1) / a.kv.page;
  SpCols c{n, min(a.first, n), max(n - a.last, 0)};
  c.end = max(c.end, c.begin);
  return c;
}

// LP lanes have a page's bounds of one head, eight columns of one of the two each, and what of q they are multiplied with in 64 bits: the sum over the group's heads
// of what is positive goes with the largest, of what is negative with the least.  Sums in 64 bits because a choice hangs on neighbours in the order.
template <class T, int DT>
__global__ __launch_bounds__(SP_THREADS) void page_scores(SpArgs a) {
  constexpr int D = DT * 32, LP = DT <= 2 ? 8 * DT : DT <= 4 ? 32 : 64, PAGES = 64 / LP, AT_ONCE = 4;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, piece = lane % LP, slot = lane / LP;
  const int head = blockIdx.y, row = blockIdx.z;
  const KvSeq sq = kv_seq(a.kv, a.seqs, row);
  const SpCols cols = sp_cols(a, sq.len);
  if (cols.n <= a.top) return;                                     // all of them are taken
  const bool has = piece < D / 4;
  const int half = piece >= D / 8 ? 1 : 0, col = has ? (piece - half * (D / 8)) * 8 : 0;
  double q[8] = {0, 0, 0, 0, 0, 0, 0, 0};
  if (has) {
    const T *p = reinterpret_cast<const T *>(a.q) + (int64_t)row * a.q_stride + (int64_t)head * a.group * D + col;
    for (int h = 0; h < a.group; ++h)
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const float v = Op<T>::value(p[(int64_t)h * D + e]);
        q[e] += half ? (v > 0.f || v != v ? v : 0.f) : (v < 0.f || v != v ? v : 0.f);
      }
  }
  const int32_t *table = a.kv.table + (int64_t)sq.row * a.kv.max_pages;
  const T *bounds = reinterpret_cast<const T *>(a.bounds) + (int64_t)head * 2 * D + half * D + col;
  uint64_t *keys = a.keys + ((int64_t)row * a.kv.n_kv + head) * a.kv.max_pages;
  constexpr int STEP = SP_WAVES * PAGES * AT_ONCE;
  for (int64_t c0 = cols.begin + (int64_t)blockIdx.x * STEP; c0 < cols.end; c0 += (int64_t)gridDim.x * STEP) {
    typename Op<T>::frag x[AT_ONCE];
#pragma unroll
    for (int k = 0; k < AT_ONCE; ++k) {
      const int c = (int)min(c0 + (k * SP_WAVES + wave) * PAGES + slot, (int64_t)cols.end - 1), id = table[c];
      x[k] = Op<T>::load(bounds + (int64_t)(id >= 0 && id < a.kv.n_pages ? id : 0) * a.kv.n_kv * 2 * D);
    }
#pragma unroll
    for (int k = 0; k < AT_ONCE; ++k) {
      double s = 0.0;
      if (has) {
        float v[8];
        if constexpr (sizeof(T) == 2) {
#pragma unroll
          for (int e = 0; e < 4; ++e) { v[2 * e] = __uint_as_float(x[k][e] << 16); v[2 * e + 1] = __uint_as_float(x[k][e] & 0xffff0000u); }
        } else {
#pragma unroll
          for (int e = 0; e < 4; ++e) { v[e] = x[k].lo[e]; v[4 + e] = x[k].hi[e]; }
        }
#pragma unroll
        for (int e = 0; e < 8; ++e) s = fma(q[e], (double)(q[e] == 0.0 ? 0.f : v[e]), s);      // nothing of q times an infinity is nothing
      }
#pragma unroll
      for (int o = LP / 2; o > 0; o >>= 1) s += __shfl_xor(s, o, 64);
      const int64_t c = c0 + (k * SP_WAVES + wave) * PAGES + slot;
      if (piece == 0 && c < cols.end) keys[c] = sp_key(s);
    }
  }
}

// ---- choice ----------------------------------------------------------------------------------------------------------
// Sum over the threads before this one, and over all
__device__ __forceinline__ int sp_before(int v, int *sums, int &total) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, inc = wave_scan(v);
  __syncthreads();
  if (lane == 63) sums[wave] = inc;
  __syncthreads();
  int base = 0;
  total = 0;
#pragma unroll
  for (int w = 0; w < SP_WAVES; ++w) { base += w < wave ? sums[w] : 0; total += sums[w]; }
  return base + inc - v;
}

// A workgroup has a row's head: the key of the last page that is taken, eight bits after another from the first in which the keys differ, then the columns in order.
__global__ __launch_bounds__(SP_THREADS) void page_choice(SpArgs a) {
  __shared__ int hist[256], sums[SP_WAVES];
  __shared__ uint64_t wide[SP_WAVES];
  __shared__ int found[2];
  const int tid = threadIdx.x, head = blockIdx.x, row = blockIdx.y;
  const KvSeq sq = kv_seq(a.kv, a.seqs, row);
  const SpCols cols = sp_cols(a, sq.len);
  const int32_t *table = a.kv.table + (int64_t)sq.row * a.kv.max_pages;
  int32_t *sel = a.sel + ((int64_t)row * a.kv.n_kv + head) * a.top;
  const uint64_t *keys = a.keys + ((int64_t)row * a.kv.n_kv + head) * a.kv.max_pages;
  auto there = [&](int c) { const int id = table[c]; return id >= 0 && id < a.kv.n_pages; };
  uint64_t prefix = 0, mask = 0;                                   // the keys that are taken are those above prefix, and `ties` of those that agree with it
  int ties = 0;
  if (cols.n > a.top) {
    int mine = 0, always;
    for (int c = tid; c < cols.begin; c += SP_THREADS) mine += there(c);
    for (int c = cols.end + tid; c < cols.n; c += SP_THREADS) mine += there(c);
    sp_before(mine, sums, always);
    int want = a.top - always;                                     // of the scored ones
    uint64_t all_or = 0, all_and = ~0ull;
    int held = 0;
    for (int c = cols.begin + tid; c < cols.end; c += SP_THREADS)
      if (there(c)) { all_or |= keys[c]; all_and &= keys[c]; ++held; }
    int total;
    sp_before(held, sums, total);
    if (total <= want) ties = total;                               // all of them
    else if (want <= 0) prefix = mask = ~0ull;                     // none
    else {
      uint64_t differ[2] = {all_or, all_and};
#pragma unroll
      for (int o = 32; o > 0; o >>= 1) { differ[0] |= __shfl_xor(differ[0], o, 64); differ[1] &= __shfl_xor(differ[1], o, 64); }
      __syncthreads();
      if ((tid & 63) == 0) wide[tid >> 6] = differ[0];
      __syncthreads();
      all_or = wide[0] | wide[1] | wide[2] | wide[3];
      __syncthreads();
      if ((tid & 63) == 0) wide[tid >> 6] = differ[1];
      __syncthreads();
      all_and = wide[0] & wide[1] & wide[2] & wide[3];
      const uint64_t other = all_or ^ all_and;
      int shift = other ? 64 - __builtin_clzll(other) : 0;         // bits below this one differ
      mask = shift == 64 ? 0 : ~0ull << shift;
      prefix = all_and & mask;
      ties = want;
      int left = total;
      while (shift > 0 && left > ties) {
        const int bits = min(shift, 8), s = shift - bits;
        hist[tid] = 0;
        __syncthreads();
        for (int c = cols.begin + tid; c < cols.end; c += SP_THREADS)
          if (there(c) && (keys[c] & mask) == prefix) atomicAdd(&hist[(keys[c] >> s) & ((1u << bits) - 1)], 1);
        __syncthreads();
        // bins from the largest on: thread t has bin 255 - t
        const int n = hist[255 - tid];
        int sum;
        const int before = sp_before(n, sums, sum);
        if (before < ties && before + n >= ties) { found[0] = 255 - tid; found[1] = before; }
        __syncthreads();
        const int bin = found[0];
        left = hist[bin];
        ties -= found[1];
        prefix |= (uint64_t)bin << s;
        shift = s;
        mask = s == 64 ? 0 : ~0ull << s;
        __syncthreads();
      }
    }
  }
  int at = 0;
  for (int c0 = 0; c0 < cols.n; c0 += SP_THREADS) {
    const int c = c0 + tid;
    bool take = false, tie = false;
    if (c < cols.n && there(c)) {
      if (cols.n <= a.top || c < cols.begin || c >= cols.end) take = true;
      else {
        const uint64_t k = keys[c] & mask;
        take = k > prefix;
        tie = k == prefix;
      }
    }
    int total;
    const int earlier = sp_before(tie ? 1 : 0, sums, total);
    take |= tie && earlier < ties;
    ties -= min(ties, total);
    const int place = at + sp_before(take ? 1 : 0, sums, total);
    if (take && place < a.top) sel[place] = c;
    at += total;
  }
  for (int v = at + tid; v < a.top; v += SP_THREADS) sel[v] = -1;
}

template <class T>
static void kb_launch(const KbArgs &a, dim3 grid, size_t lds, hipStream_t s) {
  switch (a.kv.d / 32) {
    case 1: kv_bounds<T, 1><<<grid, SP_THREADS, lds, s>>>(a); break;
    case 2: kv_bounds<T, 2><<<grid, SP_THREADS, lds, s>>>(a); break;
    case 3: kv_bounds<T, 3><<<grid, SP_THREADS, lds, s>>>(a); break;
    case 4: kv_bounds<T, 4><<<grid, SP_THREADS, lds, s>>>(a); break;
    case 5: kv_bounds<T, 5><<<grid, SP_THREADS, lds, s>>>(a); break;
    case 6: kv_bounds<T, 6><<<grid, SP_THREADS, lds, s>>>(a); break;
    case 7: kv_bounds<T, 7><<<grid, SP_THREADS, lds, s>>>(a); break;
    default: kv_bounds<T, 8><<<grid, SP_THREADS, lds, s>>>(a); break;
  }
}
template <class T>
static void sp_launch(const SpArgs &a, dim3 grid, hipStream_t s) {
  switch (a.kv.d / 32) {
    case 1: page_scores<T, 1><<<grid, SP_THREADS, 0, s>>>(a); break;
    case 2: page_scores<T, 2><<<grid, SP_THREADS, 0, s>>>(a); break;
    case 3: page_scores<T, 3><<<grid, SP_THREADS, 0, s>>>(a); break;
    case 4: page_scores<T, 4><<<grid, SP_THREADS, 0, s>>>(a); break;
    case 5: page_scores<T, 5><<<grid, SP_THREADS, 0, s>>>(a); break;
    case 6: page_scores<T, 6><<<grid, SP_THREADS, 0, s>>>(a); break;
    case 7: page_scores<T, 7><<<grid, SP_THREADS, 0, s>>>(a); break;
    default: page_scores<T, 8><<<grid, SP_THREADS, 0, s>>>(a); break;
  }
}

static size_t sp_bytes(const parse_kv *kv, int rows) { return round_up((size_t)rows * kv->n_kv * kv->max_pages * 8, 256); }

}  // namespace parse

extern "C" {

using namespace parse;

size_t parse_kv_bounds_bytes(const parse_kv *kv) {
  return check_kv(kv, false) == PARSE_OK ? (size_t)kv->n_layers * kv->n_pages * kv->n_kv * 2 * kv->d * elem_size(kv->dtype) : 0;
}

int parse_kv_bounds(const parse_kv *kv, void *bounds, int32_t layer, const int32_t *tok_offsets, const int32_t *seqs, int32_t P, parse_stream stream) {
  const int st = check_kv(kv, false);
  if (st != PARSE_OK) return st;
  if (!bounds || P <= 0 || layer < -1) return PARSE_EINVAL;
  if (layer >= kv->n_layers || P > KV_MAXSEQ || (!seqs && P > kv->n_seqs)) return PARSE_ESHAPE;
  if (!aligned16(bounds) || !aligned4(tok_offsets) || !aligned4(seqs)) return PARSE_EALIGN;
  KbArgs a{};
  a.kv = *kv;
  a.k_layer = (int64_t)kv->n_pages * kv->n_kv * kv->page * kv->d;
  a.b_layer = (int64_t)kv->n_pages * kv->n_kv * 2 * kv->d;
  a.layers = layer < 0 ? kv->n_layers : 1;
  a.K = (const char *)kv->K + std::max(layer, 0) * a.k_layer * elem_size(kv->dtype);
  a.bounds = (char *)bounds + std::max(layer, 0) * a.b_layer * elem_size(kv->dtype);
  a.tok_offsets = tok_offsets; a.seqs = seqs; a.P = P;
  if ((int64_t)kv->n_kv * a.layers > INT32_MAX) return PARSE_ESHAPE;
  if (tok_offsets && (int64_t)P * kv->max_pages > INT32_MAX) return PARSE_ESHAPE;              // their pages are counted in an int
  const int64_t per = ((int64_t)kv->n_kv * a.layers + SP_WAVES - 1) / SP_WAVES;
  const int64_t most = per * P * (tok_offsets ? (int64_t)kv->max_pages : 1);
  const dim3 grid((uint32_t)std::min<int64_t>(most, 2048));
  const size_t lds = (P + 1 + SP_WAVES) * 4;
  if (kv->dtype == PARSE_BF16) kb_launch<uint16_t>(a, grid, lds, (hipStream_t)stream);
  else kb_launch<float>(a, grid, lds, (hipStream_t)stream);
  PARSE_LAUNCH_CHECK();
  return PARSE_OK;
}

size_t parse_select_pages_workspace_bytes(const parse_kv *kv, int32_t n_q, int32_t rows) {
  if (check_kv(kv, false) != PARSE_OK || n_q <= 0 || n_q % kv->n_kv != 0 || rows <= 0 || rows > KV_MAXSEQ) return 0;
  return sp_bytes(kv, rows);
}

int parse_select_pages(const parse_kv *kv, const void *bounds, int32_t layer, const void *q, int64_t q_stride, int32_t n_q, int32_t rows, const int32_t *seqs,
                       int32_t top, int32_t first, int32_t last, int32_t *pages, void *workspace, size_t workspace_bytes, parse_stream stream) {
  const int st = check_kv(kv, false);
  if (st != PARSE_OK) return st;
  if (!bounds || !q || !pages || n_q <= 0 || rows <= 0 || layer < 0 || top <= 0 || first < 0 || last < 1) return PARSE_EINVAL;
  if (layer >= kv->n_layers || n_q % kv->n_kv != 0 || n_q > 65536 || rows > KV_MAXSEQ || (!seqs && rows > kv->n_seqs) || q_stride < (int64_t)n_q * kv->d)
    return PARSE_ESHAPE;
  if ((int64_t)first + last > top || (int64_t)rows * kv->n_kv * top > INT32_MAX) return PARSE_ESHAPE;
  if (!aligned16(bounds) || !aligned16(q) || !aligned4(pages) || !aligned4(seqs) || q_stride % (16 / elem_size(kv->dtype)) != 0) return PARSE_EALIGN;
  if (!workspace || workspace_bytes < sp_bytes(kv, rows)) return PARSE_EWORKSPACE;
  if (!aligned16(workspace)) return PARSE_EALIGN;
  SpArgs a{};
  a.kv = *kv;
  a.bounds = (const char *)bounds + (size_t)layer * kv->n_pages * kv->n_kv * 2 * kv->d * elem_size(kv->dtype);
  a.q = q; a.seqs = seqs; a.q_stride = q_stride; a.n_q = n_q; a.group = n_q / kv->n_kv; a.rows = rows; a.top = top; a.first = first; a.last = last;
  a.keys = (uint64_t *)workspace; a.sel = pages;
  if (kv->max_pages > top) {
    const int64_t pairs = (int64_t)rows * kv->n_kv;
    const dim3 grid((uint32_t)std::min<int64_t>((kv->max_pages + 15) / 16, std::max<int64_t>(1, 4096 / pairs)), kv->n_kv, rows);
    if (kv->dtype == PARSE_BF16) sp_launch<uint16_t>(a, grid, (hipStream_t)stream);
    else sp_launch<float>(a, grid, (hipStream_t)stream);
    PARSE_LAUNCH_CHECK();
  }
  page_choice<<<dim3(kv->n_kv, rows), SP_THREADS, 0, (hipStream_t)stream>>>(a);
  PARSE_LAUNCH_CHECK();
  return PARSE_OK;
}

}  // extern "C"
