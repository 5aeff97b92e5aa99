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

// smaller of two, NaN if one of them is
__device__ __forceinline__ float kb_min(float a, float b) { return __builtin_elementwise_minimum(a, b); }

// Least over lanes that differ in one bit: N values a lane become N / 2, the lower ones where the bit is clear, the upper ones where it is set.  Bits 5 and 4 by exchanges of
// halves and rows of two registers, bits 3 and 2 value by value.
template <int BIT, int N> __device__ __forceinline__ void kb_fold(float *v) {
  const bool upper = threadIdx.x & BIT;
#pragma unroll
  for (int k = 0; k < N / 2; ++k) {
    const uint32_t x = __float_as_uint(v[k]), y = __float_as_uint(v[k + N / 2]), keep = upper ? y : x, give = upper ? x : y;
    u32x2 r;
    if constexpr (BIT == 32) r = __builtin_amdgcn_permlane32_swap(x, y, false, false);
    else if constexpr (BIT == 16) r = __builtin_amdgcn_permlane16_swap(x, y, false, false);
    else if constexpr (BIT == 8) r = u32x2{keep, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)give, 0x128, 0xf, 0xf, false)};       // a row turned by eight lanes
    else r = u32x2{keep, (uint32_t)__shfl_xor((int)give, BIT, 64)};
    v[k] = kb_min(__uint_as_float(r[0]), __uint_as_float(r[1]));
  }
}

// A wavefront has pages of single heads.  A load brings eight pieces of eight columns of eight tokens (heads of 32 columns: four of sixteen), so that lines are whole; a lane keeps the
// least of the tokens that it sees of its pieces, and lanes with other tokens of them fold, half by half (values and negated values side by side: the largest is the least of
// the negated).  Bound: reads; small calls by three dependent trips to memory.  A cache of 100003 tokens, 8 heads of 128 columns of bf16, pages of 64, 205 MB: 37.6 us, 5.4 TB/s; 8 prompts of
// 512, 32 heads, pages of 16 12.0.  Lanes with a token each (all pieces their own, 60 exchanges of single values): 39 and 15; whole rows of pieces a load (64 bytes a line) 42 and 13.
template <class T, int DT, bool NT>
__global__ __launch_bounds__(SP_THREADS) void kv_bounds(KbArgs a) {
  constexpr int D = DT * 32, LP = DT == 1 ? 4 : 8, OWN = LP / 4, G = (D / 8 + LP - 1) / LP, LEFT = LP / 4;      // lanes of a token, loads of a block, groups of pieces, columns left
  typedef typename Op<T>::frag frag;
  extern __shared__ int pre[];
  int *wave_sums = pre + a.P + 1;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, page = a.kv.page, blocks = page / 16;
  const int heads = a.kv.n_kv * a.layers, per = (heads + SP_WAVES - 1) / SP_WAVES;
  for (int64_t w = blockIdx.x;; w += gridDim.x) {
    const int64_t number = w / per;
    if (number > 0x7fffffff) return;
    const KvItem f = kv_item<SP_THREADS>(a.kv, a.tok_offsets, a.seqs, a.P, 0x7fffffff, (int)number, pre, wave_sums,
                                         [&](const KvRows &r, const KvSeq &s) { return s.len / page - max(s.len - r.n, 0) / page; });
    if (f.item < 0) return;
    const int c = max(f.len - f.n, 0) / page + f.item;
    const int id = a.kv.table[(int64_t)f.row * a.kv.max_pages + c];
    const int lh = (int)(w % per) * SP_WAVES + wave;
    if (id >= 0 && id < a.kv.n_pages && lh < heads) {
      const int layer = lh / a.kv.n_kv, head = lh - layer * a.kv.n_kv;
      const T *k = reinterpret_cast<const T *>(a.K) + layer * a.k_layer + ((int64_t)id * a.kv.n_kv + head) * page * D + lane / LP * 8;
      auto piece = [&](int g) { return g * LP + lane % LP; };
      auto has = [&](int g) { return D / 8 % LP == 0 || g < G - 1 || piece(g) < D / 8; };
      auto get = [&](frag *x, int b) {
#pragma unroll
        for (int g = 0; g < G; ++g)
#pragma unroll
          for (int t = 0; t < OWN; ++t) {
            const T *p = k + b * 16 * D + (has(g) ? piece(g) : 0) * 128 + t * (64 / LP) * 8;
            x[g * OWN + t] = NT ? Op<T>::load_nt(p) : Op<T>::load(p);
          }
      };
      float v[G][16];                                              // least of the columns, largest negated
#pragma unroll
      for (int i = 0; i < 16 * G; ++i) v[i / 16][i % 16] = INFINITY;
      auto take = [&](const frag *x) {
#pragma unroll
        for (int i = 0; i < G * OWN; ++i) {
          float z[8], *w = v[i / OWN];
          if constexpr (sizeof(T) == 2) {
#pragma unroll
            for (int e = 0; e < 4; ++e) { z[2 * e] = __uint_as_float(x[i][e] << 16); z[2 * e + 1] = __uint_as_float(x[i][e] & 0xffff0000u); }
          } else {
#pragma unroll
            for (int e = 0; e < 4; ++e) { z[e] = x[i].lo[e]; z[4 + e] = x[i].hi[e]; }
          }
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            w[e] = kb_min(w[e], z[e]);
            w[8 + e] = kb_min(w[8 + e], -z[e]);
          }
        }
      };
      frag x[G * OWN];
      get(x, 0);
      for (int b = 1; b < blocks; ++b) {
        frag y[G * OWN];
        get(y, b);
        take(x);
#pragma unroll
        for (int i = 0; i < G * OWN; ++i) x[i] = y[i];
      }
      take(x);
      // bit 5 chose least or largest, bit 4 the upper four columns, bit 3 of those the upper two, bit 2 the upper one
      const int at = (lane & 16 ? 4 : 0) + (lane & 8 ? 2 : 0) + (LP == 4 && (lane & 4) ? 1 : 0);
      T *to = reinterpret_cast<T *>(a.bounds) + layer * a.b_layer + ((int64_t)id * a.kv.n_kv + head) * 2 * D + (lane & 32 ? D : 0) + at;
#pragma unroll
      for (int g = 0; g < G; ++g) {
        kb_fold<32, 16>(v[g]);
        kb_fold<16, 8>(v[g]);
        kb_fold<8, 4>(v[g]);
        if constexpr (LP == 4) kb_fold<4, 2>(v[g]);
        typedef __attribute__((ext_vector_type(LEFT))) T out_t;
        out_t out;
#pragma unroll
        for (int e = 0; e < LEFT; ++e) {
          const float r = lane & 32 ? -v[g][e] : v[g][e];
          if constexpr (sizeof(T) == 2) out[e] = (T)(__float_as_uint(r) >> 16);            // it is one of the keys
          else out[e] = r;
        }
        if (has(g)) *reinterpret_cast<out_t *>(to + piece(g) * 8) = out;
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

// Lanes for a page's bounds of one head, eight columns of one of the two each
constexpr int sp_lanes(int d) { return d <= 32 ? 8 : d <= 64 ? 16 : d <= 128 ? 32 : 64; }

// Doubles in their order as unsigned numbers, NaN the largest, whatever its sign; below them a column without a page, above them one that is always taken
constexpr uint64_t SP_NONE = 0, SP_ALWAYS = ~0ull, SP_NAN = ~0ull - 1;
__device__ __forceinline__ uint64_t sp_key(double v) {
  const int64_t b = __double_as_longlong(v);
  const uint64_t k = v == 0.0 ? 1ull << 63 : (uint64_t)(b ^ ((b >> 63) | (int64_t)(1ull << 63)));
  return v != v ? SP_NAN : k;
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

// Sum over LP lanes of eight values a lane, LP >= 8: lane l of a group ends with that of value l % 8 (moves in the vector unit).
template <int CTRL> __device__ __forceinline__ double sp_move(double v) {
  const uint64_t u = (uint64_t)__double_as_longlong(v);
  const uint32_t lo = __builtin_amdgcn_update_dpp(0, (int)(uint32_t)u, CTRL, 0xf, 0xf, false), hi = __builtin_amdgcn_update_dpp(0, (int)(u >> 32), CTRL, 0xf, 0xf, false);
  return __longlong_as_double((int64_t)((uint64_t)hi << 32 | lo));
}
template <int CTRL, int N> __device__ __forceinline__ void sp_fold(double *v, bool upper) {
#pragma unroll
  for (int k = 0; k < N / 2; ++k) {
    const double keep = upper ? v[2 * k + 1] : v[2 * k], give = upper ? v[2 * k] : v[2 * k + 1];
    v[k] = keep + sp_move<CTRL>(give);
  }
}
template <int LP> __device__ __forceinline__ double sp_sum8(double *v) {
  const int lane = threadIdx.x & 63;
  sp_fold<0xb1, 8>(v, lane & 1);                                   // lane ^ 1
  sp_fold<0x4e, 4>(v, lane & 2);                                   // lane ^ 2
  // lane ^ 7 would turn the lowest two bits as well: a quarter round each, then lane ^ 4
  const double give = lane & 4 ? v[0] : v[1], keep = lane & 4 ? v[1] : v[0];
  double s = keep + __shfl_xor(give, 4, 64);
  if constexpr (LP > 8) s += __shfl_xor(s, 8, 64);
  if constexpr (LP > 16) s += __shfl_xor(s, 16, 64);
  if constexpr (LP > 32) s += __shfl_xor(s, 32, 64);
  return s;
}

// Scores of the pages from column c0 on, `step` further each time, by a wavefront: store(column, key).  LP lanes have a page's bounds of one head, eight columns of one of the
// two each, and what of q they are multiplied with in 64 bits: the sum over the group's heads of what is positive goes with the largest, of what is negative with the
// least.  Sums in 64 bits because a choice hangs on neighbours in the order.  Eight pages a lane on their way, the first of them before q.
// Bound: latency and 64-bit products; 1563 pages of 8 heads (6.4 MB of bounds) 6.7 us.
template <class T, int DT, class F>
__device__ __forceinline__ void score_pages(const SpArgs &a, int row, int head, const KvSeq &sq, const SpCols &cols, int64_t c0, int64_t step, F store) {
  constexpr int D = DT * 32, LP = sp_lanes(D), AT_ONCE = 8;
  typedef typename Op<T>::frag frag;
  const int lane = threadIdx.x & 63, piece = lane % LP, slot = lane / LP;
  const bool has = piece < D / 4;
  const int half = piece >= D / 8 ? 1 : 0, col = has ? (piece - half * (D / 8)) * 8 : 0;
  auto values = [](const frag &x, float *v) {
    if constexpr (sizeof(T) == 2) {
#pragma unroll
      for (int e = 0; e < 4; ++e) { v[2 * e] = __uint_as_float(x[e] << 16); v[2 * e + 1] = __uint_as_float(x[e] & 0xffff0000u); }
    } else {
#pragma unroll
      for (int e = 0; e < 4; ++e) { v[e] = x.lo[e]; v[4 + e] = x.hi[e]; }
    }
  };
  const int32_t *table = a.kv.table + (int64_t)sq.row * a.kv.max_pages;
  const T *bounds = reinterpret_cast<const T *>(a.bounds) + (int64_t)head * 2 * D + half * D + col;
  const int64_t page_elems = (int64_t)a.kv.n_kv * 2 * D;
  if (c0 >= cols.end) return;
  frag x[AT_ONCE];
  uint32_t there = 0;                                              // bit k: page k is there
  auto ask = [&](int64_t c) {
    int id[AT_ONCE];
#pragma unroll
    for (int k = 0; k < AT_ONCE; ++k) id[k] = table[(int)min(c + slot * AT_ONCE + k, (int64_t)cols.end - 1)];
#pragma unroll
    for (int k = 0; k < AT_ONCE; ++k) x[k] = Op<T>::load(bounds + ((unsigned)id[k] < (unsigned)a.kv.n_pages ? id[k] : 0) * page_elems);
    there = 0;
#pragma unroll
    for (int k = 0; k < AT_ONCE; ++k) there |= (unsigned)id[k] < (unsigned)a.kv.n_pages ? 1u << k : 0u;
  };
  ask(c0);
  double q[8] = {0, 0, 0, 0, 0, 0, 0, 0};
  {
    const T *p = reinterpret_cast<const T *>(a.q) + (int64_t)row * a.q_stride + (int64_t)head * a.group * D + col;
#pragma unroll 1
    for (int h0 = 0; h0 < a.group; h0 += 4) {
      frag y[4];
#pragma unroll
      for (int h = 0; h < 4; ++h) y[h] = Op<T>::load(p + (int64_t)min(h0 + h, a.group - 1) * D);
#pragma unroll
      for (int h = 0; h < 4; ++h) {
        float v[8];
        values(y[h], v);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const float part = half ? (v[e] < 0.f ? 0.f : v[e]) : (v[e] > 0.f ? 0.f : v[e]);      // a NaN stays in both
          q[e] += h0 + h < a.group && has ? part : 0.f;
        }
      }
    }
  }
#pragma unroll 1
  for (;;) {
    double s[AT_ONCE];
    bool odd = false;
#pragma unroll
    for (int k = 0; k < AT_ONCE; ++k) {
      float v[8];
      values(x[k], v);
      s[k] = 0.0;
#pragma unroll
      for (int e = 0; e < 8; ++e) s[k] = fma(q[e], (double)v[e], s[k]);
      odd |= s[k] != s[k];
    }
    if (__any(odd)) {                                              // nothing of q times an infinity is nothing: once more (read again, so that no register waits for it)
      ask(c0);
#pragma unroll
      for (int k = 0; k < AT_ONCE; ++k) {
        float v[8];
        values(x[k], v);
        s[k] = 0.0;
#pragma unroll
        for (int e = 0; e < 8; ++e) s[k] = fma(q[e], (double)(q[e] == 0.0 ? 0.f : v[e]), s[k]);
      }
    }
    const int64_t c = c0 + slot * AT_ONCE + (lane & 7);
    const bool of_page = there >> (lane & 7) & 1;
    c0 += step;
    const bool more = c0 < cols.end;
    if (more) ask(c0);
    const double sum = sp_sum8<LP>(s);
    if (piece < 8 && c < cols.end) store((int)c, of_page ? sp_key(sum) : SP_NONE);
    if (!more) return;
  }
}
template <int DT> constexpr int sp_pages() { return 8 * (64 / sp_lanes(DT * 32)); }      // of a wavefront at once

template <class T, int DT>
__global__ __launch_bounds__(SP_THREADS, 2) void page_scores(SpArgs a) {
  const int head = blockIdx.y, row = blockIdx.z;
  const KvSeq sq = kv_seq(a.kv, a.seqs, row);
  const SpCols cols = sp_cols(a, sq.len);
  if (cols.n <= a.top) return;                                     // all of them are taken
  uint64_t *keys = a.keys + ((int64_t)row * a.kv.n_kv + head) * a.kv.max_pages;
  constexpr int STEP = SP_WAVES * sp_pages<DT>();
  score_pages<T, DT>(a, row, head, sq, cols, cols.begin + (int64_t)blockIdx.x * STEP + (threadIdx.x >> 6) * sp_pages<DT>(), (int64_t)gridDim.x * STEP,
                     [&](int c, uint64_t key) { keys[c] = key; });
}

// ---- choice ----------------------------------------------------------------------------------------------------------
constexpr int SC_THREADS = 1024, SC_FUSED = 512, SC_BITS = 11;
constexpr int SC_MOST = 4096;                        // columns whose keys stay in LDS

template <int THREADS> struct ScShared {
  uint64_t keys[SC_MOST];
  int hist[1 << SC_BITS], count[2][THREADS / 64], found[2], columns[SC_MOST / 64];
};

// Sums over the lanes before this one of the workgroup's, and over all; `sums`: LDS that nobody reads any more
template <int WAVES> __device__ __forceinline__ int sc_before(int v, int *sums, int &total) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, inc = wave_scan(v);
  if (lane == 63) sums[wave] = inc;
  __syncthreads();
  const int of_wave = wave_scan(lane < WAVES ? sums[lane] : 0);
  total = __builtin_amdgcn_readlane(of_wave, WAVES - 1);
  return inc - v + (wave ? __builtin_amdgcn_readlane(of_wave, wave - 1) : 0);
}

// A workgroup has a row's head and n columns with their keys: the key of the last one that is taken, SC_BITS after another, then the columns in order, 64 after another.
// Loops are short and not unrolled: a launch's first pass through its code costs more than what it does (unrolled 11.9 us, so 8.4).  Bound: latency, two to three steps with three
// barriers each: 8.4 us for 64 of 1563 columns, 8 heads; with the scores in one launch 8.4 for 4 rows of 16
// heads and up to 44 columns, 18 for 32 rows of 8 heads and up to 500.
template <int THREADS, class F>
__device__ __forceinline__ void choose_pages(int n, int top, int32_t *__restrict__ sel, ScShared<THREADS> &sh, F key_of) {
  constexpr int WAVES = THREADS / 64, BINS = (1 << SC_BITS) / THREADS;      // bins of a thread
  typedef __attribute__((ext_vector_type(BINS))) int bins_t;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  uint64_t prefix = SP_NONE, mask = ~0ull;                         // keys above prefix are taken, and `ties` of those that agree with it
  int ties = 0;
  if (n > top) {
    int firm = 0, held = 0;
#pragma unroll 1
    for (int c0 = 0; c0 < n; c0 += THREADS) {
      const uint64_t k = c0 + tid < n ? key_of(c0 + tid) : SP_NONE;
      firm += __popcll(__ballot(k == SP_ALWAYS));
      held += __popcll(__ballot(k != SP_ALWAYS && k != SP_NONE));
    }
    if (lane == 0) { sh.count[0][wave] = firm; sh.count[1][wave] = held; }
    __syncthreads();
    firm = __builtin_amdgcn_readlane(wave_scan(lane < WAVES ? sh.count[0][lane] : 0), WAVES - 1);
    held = __builtin_amdgcn_readlane(wave_scan(lane < WAVES ? sh.count[1][lane] : 0), WAVES - 1);
    const int want = top - firm;                                   // of the others
    if (want <= 0) prefix = SP_ALWAYS - 1;
    else if (held > want) {
      mask = 0;
      ties = want;
      int left = held;
#pragma unroll 1
      for (int shift = 64; shift > 0 && left > ties;) {
        const int bits = min(shift, SC_BITS), s = shift - bits;
        *reinterpret_cast<bins_t *>(sh.hist + BINS * tid) = bins_t(0);
        __syncthreads();
#pragma unroll 1
        for (int c = tid; c < n; c += THREADS) {
          const uint64_t k = key_of(c);
          if (k != SP_NONE && k != SP_ALWAYS && (k & mask) == prefix) atomicAdd(&sh.hist[(k >> s) & ((1u << bits) - 1)], 1);
        }
        __syncthreads();
        // bins from the largest on, BINS a thread
        const int bin0 = (1 << SC_BITS) - BINS * (tid + 1);
        const bins_t in_bin = *reinterpret_cast<const bins_t *>(sh.hist + bin0);
        int mine = 0, sum;
#pragma unroll
        for (int b = 0; b < BINS; ++b) mine += in_bin[b];
        int before = sc_before<WAVES>(mine, sh.count[0], sum);
        if (before < ties && before + mine >= ties) {              // one thread's
          int b = BINS - 1, in = in_bin[BINS - 1];
#pragma unroll
          for (int x = BINS - 2; x >= 0; --x) {
            const bool on = b == x + 1 && before + in < ties;
            before += on ? in : 0;
            b = on ? x : b;
            in = on ? in_bin[x] : in;
          }
          sh.found[0] = bin0 + b;
          sh.found[1] = before;
        }
        __syncthreads();
        const int bin = sh.found[0];
        left = sh.hist[bin];
        ties -= sh.found[1];
        prefix |= (uint64_t)bin << s;
        shift = s;
        mask = ~0ull << s;
        __syncthreads();                                           // hist, found and count are read
      }
    }
  }
  auto judge = [&](int c, bool &take, bool &tie) {
    const uint64_t k = c < n ? key_of(c) : SP_NONE;
    const bool other = k != SP_NONE && k != SP_ALWAYS;
    take = k == SP_ALWAYS || (other && (k & mask) > prefix);
    tie = other && (k & mask) == prefix;
  };
  int at = 0;
#pragma unroll 1
  for (int begin = 0; begin < n; begin += SC_MOST) {
    const int end = min(begin + SC_MOST, n);
    // taken for sure, and ties, of 64 columns side by side, counted together; then of those before
#pragma unroll 1
    for (int c0 = begin; c0 < end; c0 += THREADS) {
      bool take, tie;
      judge(c0 + tid, take, tie);
      const int both = __popcll(__ballot(take)) | __popcll(__ballot(tie)) << 16;
      if (lane == 0) sh.columns[(c0 - begin) / 64 + wave] = both;
    }
    __syncthreads();
    const int groups = (end - begin + THREADS - 1) / THREADS * WAVES;
    static_assert(SC_MOST / 64 == 64, "a lane a group");
    const int mine = lane < groups ? sh.columns[lane] : 0, inc = wave_scan(mine), total = __builtin_amdgcn_readlane(inc, 63);
#pragma unroll 1
    for (int c0 = begin; c0 < end; c0 += THREADS) {
      bool take, tie;
      judge(c0 + tid, take, tie);
      const int before = __builtin_amdgcn_readlane(inc - mine, (c0 - begin) / 64 + wave);
      const uint64_t below = (1ull << lane) - 1, takes = __ballot(take), tied = __ballot(tie);
      const int ties_before = (before >> 16) + __popcll(tied & below);
      const int place = at + (before & 0xffff) + __popcll(takes & below) + min(ties, ties_before);
      if ((take || (tie && ties_before < ties)) && place < top) sel[place] = c0 + tid;      // equal keys: the lowest columns
    }
    const int of_ties = min(ties, total >> 16);
    at += (total & 0xffff) + of_ties;
    ties -= of_ties;
    __syncthreads();
  }
  for (int v = at + tid; v < top; v += THREADS) sel[v] = -1;
}

// The keys of the columns that are not scored
__device__ __forceinline__ uint64_t sp_unscored(const SpArgs &a, const int32_t *table, int c) {
  return (unsigned)table[c] < (unsigned)a.kv.n_pages ? SP_ALWAYS : SP_NONE;
}
__device__ __forceinline__ bool sp_scored(const SpArgs &a, const SpCols &cols, int c) { return cols.n > a.top && c >= cols.begin && c < cols.end; }

__global__ __launch_bounds__(SC_THREADS) void page_choice(SpArgs a) {
  __shared__ ScShared<SC_THREADS> sh;
  const int head = blockIdx.x, row = blockIdx.y;
  const KvSeq sq = kv_seq(a.kv, a.seqs, row);
  const SpCols cols = sp_cols(a, sq.len);
  const int32_t *table = a.kv.table + (int64_t)sq.row * a.kv.max_pages;
  const uint64_t *keys = a.keys + ((int64_t)row * a.kv.n_kv + head) * a.kv.max_pages;
  int32_t *sel = a.sel + ((int64_t)row * a.kv.n_kv + head) * a.top;
  auto key = [&](int c) { return sp_scored(a, cols, c) ? keys[c] : sp_unscored(a, table, c); };
  if (cols.n <= SC_MOST) {
#pragma unroll
    for (int i = 0; i < SC_MOST / SC_THREADS; ++i) {
      const int c = i * SC_THREADS + threadIdx.x;
      if (c < cols.n) sh.keys[c] = key(c);
    }
    __syncthreads();
    choose_pages<SC_THREADS>(cols.n, a.top, sel, sh, [&](int c) { return sh.keys[c]; });
  } else {
    choose_pages<SC_THREADS>(cols.n, a.top, sel, sh, key);
  }
}

// Both, for tables of SC_MOST columns at most: the keys stay in LDS.
template <class T, int DT>
__global__ __launch_bounds__(SC_FUSED, 2) void page_select(SpArgs a) {
  __shared__ ScShared<SC_FUSED> sh;
  const int head = blockIdx.x, row = blockIdx.y;
  const KvSeq sq = kv_seq(a.kv, a.seqs, row);
  const SpCols cols = sp_cols(a, sq.len);
  const int32_t *table = a.kv.table + (int64_t)sq.row * a.kv.max_pages;
  if (cols.n > a.top) {
    constexpr int STEP = SC_FUSED / 64 * sp_pages<DT>();
    score_pages<T, DT>(a, row, head, sq, cols, cols.begin + (threadIdx.x >> 6) * sp_pages<DT>(), STEP, [&](int c, uint64_t key) { sh.keys[c] = key; });
  }
#pragma unroll 1
  for (int c = threadIdx.x; c < cols.n; c += SC_FUSED)
    if (!sp_scored(a, cols, c)) sh.keys[c] = sp_unscored(a, table, c);
  __syncthreads();
  choose_pages<SC_FUSED>(cols.n, a.top, a.sel + ((int64_t)row * a.kv.n_kv + head) * a.top, sh, [&](int c) { return sh.keys[c]; });
}

template <class T, int DT>
static void kb_go(const KbArgs &a, dim3 grid, size_t lds, hipStream_t s) {
  // Loads past the caches for pools that do not stay there.  Without / with, us: pools of 67 MB (three in turn) 12.0 / 13.3, one of 410 MB 44.1 / 37.6
  if ((size_t)a.kv.n_layers * a.kv.n_pages * a.kv.n_kv * a.kv.page * a.kv.d * sizeof(T) * 2 > ((size_t)192 << 20)) kv_bounds<T, DT, true><<<grid, SP_THREADS, lds, s>>>(a);
  else kv_bounds<T, DT, false><<<grid, SP_THREADS, lds, s>>>(a);
}
template <class T>
static void kb_launch(const KbArgs &a, dim3 grid, size_t lds, hipStream_t s) {
  switch (a.kv.d / 32) {
    case 1: kb_go<T, 1>(a, grid, lds, s); break;
    case 2: kb_go<T, 2>(a, grid, lds, s); break;
    case 3: kb_go<T, 3>(a, grid, lds, s); break;
    case 4: kb_go<T, 4>(a, grid, lds, s); break;
    case 5: kb_go<T, 5>(a, grid, lds, s); break;
    case 6: kb_go<T, 6>(a, grid, lds, s); break;
    case 7: kb_go<T, 7>(a, grid, lds, s); break;
    default: kb_go<T, 8>(a, grid, lds, s); break;
  }
}
// One launch where a workgroup a head fills the card about once, or there is little to score.  Two launches / one, us, 128 columns of bf16, heads of all rows x columns of the
// table: 8 x 44 9.6 / 7.4, 8 x 512 10.2 / 13.8, 8 x 4000 16.8 / 65, 64 x 1000 17.8 / 23.8, 128 x 500 17.5 / 15.6, 256 x 300 19.9 / 14.3, 256 x 1500 54 / 39, 128 x 4000 61 / 75,
// 2048 x 200 69 / 81.
static bool sp_fused(const SpArgs &a) {
  const int64_t pairs = (int64_t)a.rows * a.kv.n_kv;
  return pairs <= 1024 && (a.kv.max_pages <= 256 || (a.kv.max_pages <= 2048 && pairs >= 128));
}
static_assert(SC_MOST >= 2048, "their keys stay in LDS");
template <class T, int DT>
static void sp_go(const SpArgs &a, hipStream_t s) {
  const int64_t pairs = (int64_t)a.rows * a.kv.n_kv;
  if (sp_fused(a)) {
    page_select<T, DT><<<dim3(a.kv.n_kv, a.rows), SC_FUSED, 0, s>>>(a);
    return;
  }
  if (a.kv.max_pages > a.top) {
    const int64_t step = (int64_t)SP_WAVES * sp_pages<DT>();
    const dim3 grid((uint32_t)std::min<int64_t>((a.kv.max_pages + step - 1) / step, std::max<int64_t>(1, 4096 / pairs)), a.kv.n_kv, a.rows);
    page_scores<T, DT><<<grid, SP_THREADS, 0, s>>>(a);
  }
  page_choice<<<dim3(a.kv.n_kv, a.rows), SC_THREADS, 0, s>>>(a);
}
template <class T>
static void sp_launch(const SpArgs &a, hipStream_t s) {
  switch (a.kv.d / 32) {
    case 1: sp_go<T, 1>(a, s); break;
    case 2: sp_go<T, 2>(a, s); break;
    case 3: sp_go<T, 3>(a, s); break;
    case 4: sp_go<T, 4>(a, s); break;
    case 5: sp_go<T, 5>(a, s); break;
    case 6: sp_go<T, 6>(a, s); break;
    case 7: sp_go<T, 7>(a, s); break;
    default: sp_go<T, 8>(a, s); break;
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
  // a prompt's whole pages are no more than the pool has
  const int64_t heads = (int64_t)kv->n_kv * a.layers, items = (int64_t)P * (tok_offsets ? std::min(kv->max_pages, kv->n_pages) : 1);
  const int64_t per = (heads + SP_WAVES - 1) / SP_WAVES;
  const dim3 grid((uint32_t)std::min<int64_t>(per * items, 2048));
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
  if (kv->dtype == PARSE_BF16) sp_launch<uint16_t>(a, (hipStream_t)stream);
  else sp_launch<float>(a, (hipStream_t)stream);
  PARSE_LAUNCH_CHECK();
  return PARSE_OK;
}

}  // extern "C"
