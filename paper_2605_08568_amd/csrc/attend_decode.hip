// Attention of one new token per sequence over the paged cache (parse_attend_decode).
#include <algorithm>
#include <type_traits>

#include "attend.hpp"

namespace parse {

constexpr int AD_WAVES = 4, AD_THREADS = AD_WAVES * 64;
constexpr int AD_STEP = 32;                          // tokens of a wavefront's step
constexpr int AD_HEADS = 16;                         // query heads of a workgroup, the N side of the 16-wide instruction
constexpr int AD_GROUPS = 512;                       // workgroups of a call: two for each compute unit
constexpr size_t AD_TICKET_BYTES = PARSE_ATTEND_DECODE_ZERO_BYTES;
static_assert(AD_GROUPS * 4 <= AD_TICKET_BYTES, "a ticket for every share of every column that has several");

struct AdArgs {
  parse_kv kv;
  const void *K, *V;                                 // of the layer
  const void *q;
  void *out;
  float *lse;
  const int32_t *seqs;
  int64_t q_stride, out_stride;
  int n_q, group, rows, shares, window, sinks;
  float scale, lag;                                  // |scale| times log2(e); AT_LAG in products of q and k
  uint32_t q_sign;
  float *part;                                       // [kv head][group of 16 heads][share][2] of AD_HEADS * (d + 2)
  int32_t *tickets;                                  // [kv head][group of 16 heads][share]: parts that have come of the row that begins in the share
};

template <class T>
__device__ __forceinline__ void ad_store(const AdArgs &a, int row, int head, int i, int D, float top, float ls, float os) {
  const float y = ls == 0.f ? 0.f : os / ls;
  T *out = reinterpret_cast<T *>(a.out) + (int64_t)row * a.out_stride + (int64_t)head * D + i;
  if constexpr (sizeof(T) == 2) *out = (uint16_t)cvt_pk_bf16(y, 0.f);
  else *out = y;
  if (a.lse && i == 0) a.lse[(int64_t)row * a.n_q + head] = at_lse(top, a.scale, ls);
}

// How the batch's steps are dealt out: sequence b has the steps [before, before + its count) of `total`, a workgroup `per` of them.
struct AdDeal {
  int total, per;
};
// A wavefront alone, for up to 64 sequences: lane b has sequence b's words
struct AdLane {
  KvSeq seq;
  KvSpan span;
  int before;
};
__device__ __forceinline__ KvSpan ad_span(const AdArgs &a, int len) { return kv_span(len - 1, len - 1, a.window, a.sinks, AD_STEP); }
__device__ __forceinline__ AdDeal ad_deal(const AdArgs &a, int total) {
  const int per = (total + a.shares - 1) / a.shares;
  return AdDeal{total, max((per + AD_WAVES - 1) / AD_WAVES, 1) * AD_WAVES};    // the wavefronts take turns
}
__device__ __forceinline__ AdDeal ad_lanes(const AdArgs &a, AdLane &w) {
  const int lane = threadIdx.x & 63;
  w.seq = kv_seq(a.kv, a.seqs, min(lane, a.rows - 1));
  w.span = ad_span(a, w.seq.len);
  const int mine = lane < a.rows ? w.span.count : 0;
  const int inc = wave_scan(mine);
  w.before = inc - mine;
  return ad_deal(a, __builtin_amdgcn_readlane(inc, 63));
}

// Row x is share x, whole, and nothing has to be joined, where no row has many more steps than an equal share would: three more a wavefront take about as long as
// a join, two where rows are few and none of them begins inside a share.  32 heads over 8, equal shares / rows: 16 caches of 100 to 200 tokens 16.8 / 9.2 us, of 30 to 500 18.1 /
// 11.8, 64 of 300 to 330 25.0 / 18.3, 64 of 2000 to 2300 99 / 90, 40 windows of 1000 40.9 / 34.8; 4 caches of 510 tokens 10.8 / 11.9, 1 of 250 10.3 / 8.5.
__device__ __host__ __forceinline__ int ad_slack(int rows) { return rows <= 4 ? 8 : 12; }
__device__ __forceinline__ bool ad_by_rows(const AdArgs &a, const AdDeal &deal, const AdLane &w) {
  return a.rows <= a.shares && !__any((int)(threadIdx.x & 63) < a.rows && w.span.count > deal.per + ad_slack(a.rows));
}
__device__ __forceinline__ bool ad_by_rows(const AdArgs &a, const AdDeal &deal, const int *pre) {
  if (a.rows > a.shares) return false;
  bool longer = false;
  for (int p = threadIdx.x; p < a.rows; p += AD_THREADS) longer |= pre[p + 1] - pre[p] > deal.per + ad_slack(a.rows);
  return !__syncthreads_or(longer);
}

template <bool SHARED>
__device__ __forceinline__ void ad_part(float *p, float v) {
  if (SHARED) __hip_atomic_store(p, v, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  else *p = v;
}
// The parts of row b: shares x0 .. x0 + parts - 1, of all heads of the workgroup, added in the order of the shares (same inputs, same bits).  A wavefront
// has a head's weights, then a thread has two columns of every so many parts.  `lds`: 2 * heads * parts floats; `per_head`: two numbers a head.
template <class T>
__device__ __forceinline__ void ad_join(const AdArgs &a, int b, int kvh, int hg, int heads, int x0, int parts, int before, int per, float *lds, float *per_head) {
  const int D = a.kv.d, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const float *base = a.part + ((int64_t)kvh * gridDim.z + hg) * a.shares * 2 * AD_HEADS * (D + 2);
  auto part_of = [&](int x) { return base + ((int64_t)(x0 + x) * 2 + ((int64_t)(x0 + x) * per <= before ? 1 : 0)) * AD_HEADS * (D + 2); };
  auto get = [&](const float *p) { return __hip_atomic_load(p, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); };
  for (int h = wave; h < heads; h += AD_WAVES) {
    float top = -INFINITY, ls = 0.f;
    for (int x = lane; x < parts; x += 64) {
      const float m = get(part_of(x) + AD_HEADS * D + h), l = get(part_of(x) + AD_HEADS * (D + 1) + h);
      lds[h * parts + x] = m;
      lds[(heads + h) * parts + x] = l;
      top = fmaxf(top, m);
    }
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor(top, o, 64));
    for (int x = lane; x < parts; x += 64) {
      const float by = at_exp2((lds[h * parts + x] - finite_or_0(top)) * a.scale);
      lds[h * parts + x] = by;
      ls += by * lds[(heads + h) * parts + x];
    }
    ls = wave_sum(ls);
    if (lane == 0) { per_head[h] = top; per_head[AD_HEADS + h] = ls; }
  }
  __syncthreads();
  auto columns = [&](auto at_once) {                               // two a thread, so many parts on their way
    constexpr int N = decltype(at_once)::value;
    for (int v = tid; v < heads * D / 2; v += AD_THREADS) {
      const int h = 2 * v / D, i = 2 * v % D;
      float y0 = 0.f, y1 = 0.f;
      for (int first = 0; first < parts; first += N) {
        uint64_t two[N];
#pragma unroll
        for (int k = 0; k < N; ++k)
          two[k] = __hip_atomic_load(reinterpret_cast<const uint64_t *>(part_of(min(first + k, parts - 1)) + h * D + i), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
#pragma unroll
        for (int k = 0; k < N; ++k) {
          const float by = lds[h * parts + min(first + k, parts - 1)];
          const bool is = first + k < parts;
          y0 = is ? fmaf(by, __uint_as_float((uint32_t)two[k]), y0) : y0;
          y1 = is ? fmaf(by, __uint_as_float((uint32_t)(two[k] >> 32)), y1) : y1;
        }
      }
      const int head = kvh * a.group + hg * AD_HEADS + h;
      ad_store<T>(a, b, head, i, D, per_head[h], per_head[AD_HEADS + h], y0);
      ad_store<T>(a, b, head, i + 1, D, per_head[h], per_head[AD_HEADS + h], y1);
    }
  };
  if (parts <= 2) columns(std::integral_constant<int, 2>{});
  else if (parts <= 16) columns(std::integral_constant<int, 8>{});
  else columns(std::integral_constant<int, 32>{});
}

// A workgroup has sixteen query heads of one kv head, and one share of all steps that the batch sees.
// A step of 32 tokens: s = K q (operand A = K, token rows; operand B = q, a query head a column), weights 2^(scale s - base), o += V^T p (operand A = V^T,
// column rows).  K's rows are taken in the order in which the scores come back as operand B: rows 4 q + 0..3 of the two instructions of a step are tokens
// 8 q + 0..3 and 8 q + 4..7, so that a lane's eight weights are the eight tokens whose V it has loaded, and nothing moves between lanes but, where a
// maximum grows by more than 2^8, that maximum.  The matrix units are used for their operand form: fifteen of sixteen columns may be empty, and still
// they take 1 / 20 of the time of the loads.
// Bound: reads.  Operands go straight from the pages into registers in pieces of 1 KiB (a page's layout is theirs), one step ahead of the one that is worked
// on where two steps fit the registers (bf16 up to 128 columns, fp32 up to 64; wider heads load a step, wait and work on it, while another wavefront's loads are on their way); a unit has 32 KiB on their way whatever is asked for, so that two workgroups a unit are enough, and more of them only cut the caches finer: 512 / 768 / 1024
// workgroups, 32 ragged caches of 32 heads 108 / 121 / 114 us, 192 windows 162 / 182 / 175.  Shares are equal in steps, not in rows: a batch of unlike lengths needs no plan.
// Measured, reads of the cache against 6.1 to 6.4 TB/s of a read-only stream of 2 GiB: 32 caches of 32 to 2048 tokens, 32 heads 5.9 TB/s (96 us), 100003 tokens of 8 heads
// 5.4 (76 us), 192 windows of 1024 5.6 (143 us), 256 caches of 300 tokens, 8 heads 5.4 (59 us); single short caches by latency (77 tokens 7.3 us).
// By width, 32 caches of 32 to 2048 tokens, 16 heads: bf16 128 / 160 / 256 columns 5.1 / 5.3 / 5.4 TB/s, fp32 64 / 96 / 128 columns 4.5 / 4.4 / 4.1, and 2.7 at 256, where one
// wavefront a SIMD has a step's 64 KiB on their way or none.
template <class T, int DT, bool NT, bool TICKETS>
__global__ __launch_bounds__(AD_THREADS, DT * sizeof(T) <= 16 ? 2 : 1) void attend_decode(AdArgs a) {
  constexpr int D = DT * 32, KB = D / 32, VB = D / 16;
  typedef typename Op<T>::frag frag;
  extern __shared__ char smem[];
  float *red = reinterpret_cast<float *>(smem);                    // [wave][head][D], [wave][head] twice
  float *red_m = red + AD_WAVES * AD_HEADS * D, *red_l = red_m + AD_WAVES * AD_HEADS;
  int *wave_sums = reinterpret_cast<int *>(red_l + AD_WAVES * AD_HEADS), *pre = wave_sums + AD_WAVES;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int n = lane & 15, quad = lane >> 4;
  const int share = blockIdx.x, kvh = blockIdx.y, hg = blockIdx.z;
  const bool few = a.rows <= 64;
  AdLane w{};
  AdDeal deal;
  if (few) {
    deal = ad_lanes(a, w);
  } else {
    kv_prefix<AD_THREADS>(a.rows, pre, wave_sums, [&](int p) { return ad_span(a, kv_seq(a.kv, a.seqs, p).len).count; });
    deal = ad_deal(a, pre[a.rows]);
  }
  const int heads = min(a.group - hg * AD_HEADS, AD_HEADS);
  for (int e = share; e < a.rows; e += a.shares) {                 // rows that see nothing
    const int count = few ? __builtin_amdgcn_readlane(w.span.count, e) : pre[e + 1] - pre[e];
    if (count > 0) continue;
    for (int v = tid; v < heads * D; v += AD_THREADS) {
      const int h = kvh * a.group + hg * AD_HEADS + v / D;
      reinterpret_cast<T *>(a.out)[(int64_t)e * a.out_stride + h * D + v % D] = 0;
      if (a.lse && v % D == 0) a.lse[(int64_t)e * a.n_q + h] = -INFINITY;
    }
  }
  const bool by_rows = few ? ad_by_rows(a, deal, w) : ad_by_rows(a, deal, pre);
  if (by_rows && share >= a.rows) return;
  const int64_t begin = by_rows ? (few ? __builtin_amdgcn_readlane(w.before, share) : __builtin_amdgcn_readfirstlane(pre[share])) : (int64_t)share * deal.per;
  const int64_t behind = by_rows ? begin + (few ? __builtin_amdgcn_readlane(w.span.count, share) : __builtin_amdgcn_readfirstlane(pre[share + 1] - pre[share])) : begin + deal.per;
  const int end = (int)min(behind, (int64_t)deal.total);
  if (begin >= end) return;
  const int64_t page_elems = (int64_t)a.kv.n_kv * a.kv.page * D, head0 = (int64_t)kvh * a.kv.page * D;
  const int tok = 8 * (n >> 2) + (n & 3);                          // the first instruction's row n: tokens 8 quad + 0..3 of a step come back to a lane
  const int page_bits = 31 - __builtin_clz(a.kv.page);
  // where this lane's pieces of K and of V stand in their block of sixteen tokens, elements
  const int k_in = quad * 128 + (tok & 15) * 8, v_in = ((quad & 1) * D + n) * 8;
  auto row_of = [&](int v) { return few ? 63 - __builtin_clzll(__ballot(lane < a.rows && w.before <= v && w.span.count > 0)) : kv_find(pre, a.rows, v); };
  auto before_of = [&](int e) { return few ? __builtin_amdgcn_readlane(w.before, e) : __builtin_amdgcn_readfirstlane(pre[e]); };
  auto count_of = [&](int e) { return few ? __builtin_amdgcn_readlane(w.span.count, e) : __builtin_amdgcn_readfirstlane(pre[e + 1] - pre[e]); };
  // Rows of the share.  Where they are four or more, of twelve steps or fewer on average, a wavefront has every fourth of those that lie in it whole, alone: nothing
  // meets, nobody waits (130 rows of one step, 8 kv heads of 256: 35 -> 21.5 us; 256 of ten steps 70 -> 68).  Other rows are worked on together, step by step in turn.
  const int b0 = row_of((int)begin), b1 = row_of(end - 1);
  const bool many = b1 - b0 >= AD_WAVES - 1 && deal.per <= 12 * (b1 - b0);
  const int whole0 = many ? b0 + (before_of(b0) < (int)begin ? 1 : 0) : b1 + 1, whole1 = many ? b1 - (before_of(b1) + count_of(b1) > end ? 1 : 0) : b1;
  int mine = __builtin_amdgcn_readfirstlane(whole0 + wave), shared = b0 < whole0 ? b0 : whole1 + 1;
  for (;;) {
    const bool alone = mine <= whole1;
    int b;
    if (alone) {
      b = mine;
      mine += AD_WAVES;
    } else {
      if (shared > b1) break;
      b = shared++;
      if (shared == whole0) shared = whole1 + 1;
    }
    const int before = before_of(b), count = count_of(b);
    if (count == 0) continue;
    KvSeq sq;
    if (few) sq = KvSeq{__builtin_amdgcn_readlane(w.seq.row, b), __builtin_amdgcn_readlane(w.seq.len, b)};
    else sq = kv_seq(a.kv, a.seqs, b);
    sq.row = __builtin_amdgcn_readfirstlane(sq.row);
    sq.len = __builtin_amdgcn_readfirstlane(sq.len);
    const KvSpan span = ad_span(a, sq.len);
    const int pos = sq.len - 1, lo = kv_window_begin(pos, a.window);
    const int first = max((int)begin - before, 0), last = min(end - before, count);
    const int start = alone ? 0 : first + wave, turn = alone ? 1 : AD_WAVES;   // the wavefront's steps
    const int32_t *table = a.kv.table + (int64_t)sq.row * a.kv.max_pages;
    frag qf[KB];
    {
      const T *q = reinterpret_cast<const T *>(a.q) + (int64_t)b * a.q_stride + (int64_t)(kvh * a.group + hg * AD_HEADS + min(n, heads - 1)) * D;
#pragma unroll
      for (int k = 0; k < KB; ++k) qf[k] = Op<T>::sign(Op<T>::load(q + 32 * k + 8 * quad), a.q_sign);
    }
    float m = -INFINITY, l = 0.f;
    f32x4 o[VB];
#pragma unroll
    for (int v = 0; v < VB; ++v) o[v] = f32x4{0.f, 0.f, 0.f, 0.f};
    // the pages of the wavefront's next 64 steps, a lane each: blocks of tokens 0..15 and 16..31, -1 for none
    int id_a = -1, id_b = -1;
    struct Step {
      frag k0[KB], k1[KB], v[VB];
      int t0;
      bool there_a, there_b;
    };
    // Operands of step number j of the wavefront, straight from the pages; all of them asked for before the step ahead of it is worked on
    auto load = [&](Step &x, int j) {
      const int u = start + j * turn;
      if ((j & 63) == 0) {
        const int t = span.at(min(u + lane * turn, count - 1)) * AD_STEP;
        id_a = table[min(t >> page_bits, a.kv.max_pages - 1)];
        id_b = table[min((t + 16) >> page_bits, a.kv.max_pages - 1)];
      }
      x.t0 = span.at(u) * AD_STEP;
      const int ida = __builtin_amdgcn_readlane(id_a, j & 63), idb = __builtin_amdgcn_readlane(id_b, j & 63);
      x.there_a = (unsigned)ida < (unsigned)a.kv.n_pages;
      x.there_b = (unsigned)idb < (unsigned)a.kv.n_pages;
      const int64_t at_a = (int64_t)(x.there_a ? ida : 0) * page_elems + head0 + (int64_t)(x.t0 & (a.kv.page - 1)) * D;
      const int64_t at_b = (int64_t)(x.there_b ? idb : 0) * page_elems + head0 + (int64_t)((x.t0 + 16) & (a.kv.page - 1)) * D;
      const T *kp = reinterpret_cast<const T *>(a.K) + (n < 8 ? at_a : at_b) + k_in;
      const T *vp = reinterpret_cast<const T *>(a.V) + (quad < 2 ? at_a : at_b) + v_in;
#pragma unroll
      for (int k = 0; k < KB; ++k) { x.k0[k] = NT ? Op<T>::load_nt(kp + k * 512) : Op<T>::load(kp + k * 512); x.k1[k] = NT ? Op<T>::load_nt(kp + k * 512 + 32) : Op<T>::load(kp + k * 512 + 32); }
#pragma unroll
      for (int v = 0; v < VB; ++v) x.v[v] = NT ? Op<T>::load_nt(vp + v * 128) : Op<T>::load(vp + v * 128);
    };
    auto work = [&](Step &x, auto careful) {
      f32x4 s0 = {0.f, 0.f, 0.f, 0.f}, s1 = s0;
#pragma unroll
      for (int k = 0; k < KB; ++k) { s0 = Op<T>::mma16(x.k0[k], qf[k], s0); s1 = Op<T>::mma16(x.k1[k], qf[k], s1); }
      float s[8];
#pragma unroll
      for (int e = 0; e < 4; ++e) { s[e] = s0[e]; s[4 + e] = s1[e]; }
      const bool whole = x.there_a && x.there_b && x.t0 + AD_STEP - 1 <= pos && (x.t0 >= lo || x.t0 + AD_STEP <= a.sinks);
      if (!whole) {                                                // what is not seen: no weight, and nothing of V to multiply it with
        uint32_t keep = 0;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const bool sees = (quad < 2 ? x.there_a : x.there_b) & kv_sees(pos, lo, a.sinks, x.t0 + 8 * quad + e);
          s[e] = sees ? s[e] : -INFINITY;
          keep |= (sees ? 1u : 0u) << e;
        }
#pragma unroll
        for (int v = 0; v < VB; ++v) x.v[v] = Op<T>::only(x.v[v], keep);
      }
      float top = s[0];
#pragma unroll
      for (int e = 1; e < 8; ++e) top = fmaxf(top, s[e]);
      if (__any(top > m + a.lag)) {
        const float grown = fmaxf(m, lane_max<32>(lane_max<16>(top)));
        const float by = at_exp2((m - finite_or_0(grown)) * a.scale);
        l *= by;
#pragma unroll
        for (int v = 0; v < VB; ++v) o[v] *= by;
        m = grown;
      }
      const float base = at_base(m, a.scale);
      float p[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) { p[e] = at_exp2(fmaf(s[e], a.scale, -base)); l += p[e]; }
      const frag pf = Op<T>::pack(p);
#pragma unroll
      for (int v = 0; v < VB; ++v) o[v] = Op<T>::mma16(x.v[v], pf, o[v]);
      if constexpr (sizeof(T) == 2) {                              // what the rounding of the weights left: the pipes are idle, and the result is as exact as from fp32 weights
        const frag rest = Op<T>::pack_rest(p, pf);
#pragma unroll
        for (int v = 0; v < VB; ++v) {
          if constexpr (decltype(careful)::value) {
            const f32x4 add = Op<T>::mma16(x.v[v], rest, f32x4{0.f, 0.f, 0.f, 0.f});
#pragma unroll
            for (int e = 0; e < 4; ++e) o[v][e] = fabsf(add[e]) < INFINITY ? o[v][e] + add[e] : o[v][e];
          } else {
            o[v] = Op<T>::mma16(x.v[v], rest, o[v]);
          }
        }
      }
    };
    const int steps = last > start ? (last - start + turn - 1) / turn : 0;
    Step even;
    if constexpr (DT * sizeof(T) <= 8) {                           // two steps fit the registers
      Step odd;
      if (steps > 0) load(even, 0);
      for (int j = 0; j < steps; j += 2) {
        if (j + 1 < steps) load(odd, j + 1);
        work(even, std::false_type{});
        if (j + 1 < steps) {
          if (j + 2 < steps) load(even, j + 2);
          work(odd, std::false_type{});
        }
      }
    } else {
      for (int j = 0; j < steps; ++j) {
        load(even, j);
        work(even, std::false_type{});
      }
    }
    if constexpr (sizeof(T) == 2) {
      // What the rounding left has either sign or is 0: times an infinity of V it makes NaN of the sum.  Where something that is not finite came out, once more
      // with the columns that meet an infinity or NaN left to the first product.  (Looked at once a row: 0 to 0.5 % of the time, 2 % at 256 columns; at every step 12 %.)
      f32x4 sum = {0.f, 0.f, 0.f, 0.f};                            // NaN where one of them is not finite
#pragma unroll
      for (int v = 0; v < VB; ++v)
#pragma unroll
        for (int e = 0; e < 4; ++e) sum[e] = fmaf(o[v][e], 0.f, sum[e]);
      if (__any((sum[0] + sum[1]) + (sum[2] + sum[3]) != 0.f)) {
        m = -INFINITY; l = 0.f;
#pragma unroll
        for (int v = 0; v < VB; ++v) o[v] = f32x4{0.f, 0.f, 0.f, 0.f};
        for (int j = 0; j < steps; ++j) {
          load(even, j);
          work(even, std::true_type{});
        }
      }
    }
    l = lane_sum<32>(lane_sum<16>(l));
    if (alone) {
      if (n < heads) {
        const int head = kvh * a.group + hg * AD_HEADS + n;
        const float by = l == 0.f ? 0.f : 1.f / l;
        T *out = reinterpret_cast<T *>(a.out) + (int64_t)b * a.out_stride + (int64_t)head * D + 4 * quad;
#pragma unroll
        for (int v = 0; v < VB; ++v) Op<T>::store4(out + 16 * v, o[v][0] * by, o[v][1] * by, o[v][2] * by, o[v][3] * by);
        if (a.lse && quad == 0) a.lse[(int64_t)b * a.n_q + head] = at_lse(m, a.scale, l);
      }
      continue;
    }
    // the wavefronts' sums meet
    __syncthreads();
    if (lane < 16) { red_m[wave * AD_HEADS + lane] = m; red_l[wave * AD_HEADS + lane] = l; }
#pragma unroll
    for (int v = 0; v < VB; ++v) *reinterpret_cast<f32x4 *>(red + (wave * AD_HEADS + n) * D + 16 * v + 4 * quad) = o[v];
    __syncthreads();
    const bool all = first == 0 && last == count;
    float *part = a.part + ((((int64_t)kvh * gridDim.z + hg) * a.shares + share) * 2 + (first == 0 ? 1 : 0)) * AD_HEADS * (D + 2);
    for (int v = tid; v < heads * D; v += AD_THREADS) {
      const int h = v / D, i = v % D;
      float top = -INFINITY, ls = 0.f, os = 0.f;
#pragma unroll
      for (int x = 0; x < AD_WAVES; ++x) top = fmaxf(top, red_m[x * AD_HEADS + h]);
#pragma unroll
      for (int x = 0; x < AD_WAVES; ++x) {
        const float by = at_exp2((red_m[x * AD_HEADS + h] - finite_or_0(top)) * a.scale);
        ls += by * red_l[x * AD_HEADS + h];
        os += by * red[(x * AD_HEADS + h) * D + i];
      }
      if (all) ad_store<T>(a, b, kvh * a.group + hg * AD_HEADS + h, i, D, top, ls, os);
      else {
        ad_part<TICKETS>(part + h * D + i, os);
        if (i == 0) { ad_part<TICKETS>(part + AD_HEADS * D + h, top); ad_part<TICKETS>(part + AD_HEADS * (D + 1) + h, ls); }
      }
    }
    if (TICKETS && !all) {
      // Parts and tickets are device-scope accesses, past the die's L2: every thread waits until its own stores are acknowledged, the barrier
      // collects all of them, then thread 0 draws.  The workgroup that draws a row's last ticket joins the row; nobody waits for anybody.
      const int x0 = before / deal.per, parts = (before + count - 1) / deal.per - x0 + 1;
      int32_t *ticket = a.tickets + ((int64_t)kvh * gridDim.z + hg) * a.shares + x0;
      asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
      __syncthreads();
      if (tid == 0) {
        const int t = __hip_atomic_fetch_add(ticket, 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        if (t == parts - 1) __hip_atomic_store(ticket, 0, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);    // ready for the next call
        *wave_sums = t == parts - 1;
      }
      __syncthreads();
      if (*wave_sums) ad_join<T>(a, b, kvh, hg, heads, x0, parts, before, deal.per, red, red_m);
    }
  }
}

// The parts of a row that more than one share had; workgroup (x, head) has row x or, where there are fewer shares, the row that begins in share x and goes on behind it.  The weights of all
// parts first, then four columns a thread of every so many parts, none of which waits for another.
template <class T>
__global__ __launch_bounds__(AD_THREADS) void attend_join(AdArgs a) {
  extern __shared__ char smem[];
  float *weight = reinterpret_cast<float *>(smem), *sums = weight + AD_GROUPS;       // [parts]; [part group][D] and two numbers a wavefront
  const int D = a.kv.d, tid = threadIdx.x, head = blockIdx.y, kvh = head / a.group, hg = head % a.group / AD_HEADS, h = head % a.group % AD_HEADS;
  const int zs = (a.group + AD_HEADS - 1) / AD_HEADS;
  int *wave_sums = reinterpret_cast<int *>(sums + AD_THREADS * 4 + 2 * AD_WAVES), *pre = wave_sums + AD_WAVES;
  const bool of_row = a.rows < a.shares;
  int b = blockIdx.x, before, count;
  AdDeal deal;
  if (a.rows <= 64) {
    AdLane w;
    deal = ad_lanes(a, w);
    if (ad_by_rows(a, deal, w)) return;
    if (!of_row) {
      const int64_t end = (int64_t)(blockIdx.x + 1) * deal.per;    // of the share
      if (end >= deal.total) return;
      b = 63 - __builtin_clzll(__ballot((int)(threadIdx.x & 63) < a.rows && w.before < (int)end && w.span.count > 0));
    }
    before = __builtin_amdgcn_readlane(w.before, b);
    count = __builtin_amdgcn_readlane(w.span.count, b);
  } else {
    kv_prefix<AD_THREADS>(a.rows, pre, wave_sums, [&](int p) { return ad_span(a, kv_seq(a.kv, a.seqs, p).len).count; });
    deal = ad_deal(a, pre[a.rows]);
    if (ad_by_rows(a, deal, pre)) return;
    if (!of_row) {
      const int64_t end = (int64_t)(blockIdx.x + 1) * deal.per;
      if (end >= deal.total) return;
      b = kv_find(pre, a.rows, (int)end - 1);
    }
    before = pre[b];
    count = pre[b + 1] - before;
  }
  if (count == 0) return;
  const int x0 = before / deal.per, x1 = (before + count - 1) / deal.per, parts = x1 - x0 + 1;
  if (parts == 1 || (!of_row && x0 != (int)blockIdx.x)) return;
  const float *base = a.part + ((int64_t)kvh * zs + hg) * a.shares * 2 * AD_HEADS * (D + 2);
  auto part_of = [&](int x) { return base + ((int64_t)(x0 + x) * 2 + ((int64_t)(x0 + x) * deal.per <= before ? 1 : 0)) * AD_HEADS * (D + 2); };
  float top = -INFINITY;
  for (int x = tid; x < parts; x += AD_THREADS) {
    const float m = part_of(x)[AD_HEADS * D + h];
    weight[x] = m;
    top = fmaxf(top, m);
  }
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor(top, o, 64));
  float *tops = sums + AD_THREADS * 4, *totals = tops + AD_WAVES;
  if ((tid & 63) == 0) tops[tid >> 6] = top;
  __syncthreads();
  top = fmaxf(fmaxf(tops[0], tops[1]), fmaxf(tops[2], tops[3]));
  float ls = 0.f;
  for (int x = tid; x < parts; x += AD_THREADS) {
    const float by = at_exp2((weight[x] - finite_or_0(top)) * a.scale);
    weight[x] = by;
    ls += by * part_of(x)[AD_HEADS * (D + 1) + h];
  }
  ls = wave_sum(ls);
  if ((tid & 63) == 0) totals[tid >> 6] = ls;
  __syncthreads();
  ls = (totals[0] + totals[1]) + (totals[2] + totals[3]);
  const int wide = D / 4, groups = AD_THREADS / wide, g = tid / wide, i = tid % wide;
  f32x4 os = {0.f, 0.f, 0.f, 0.f};
  if (g < groups) {
#pragma unroll 4
    for (int x = g; x < parts; x += groups) os += weight[x] * *reinterpret_cast<const f32x4 *>(part_of(x) + h * D + 4 * i);
    *reinterpret_cast<f32x4 *>(sums + (g * wide + i) * 4) = os;
  }
  __syncthreads();
  for (int v = tid; v < D; v += AD_THREADS) {
    float y = 0.f;
    for (int k = 0; k < groups; ++k) y += sums[k * D + v];
    ad_store<T>(a, b, head, v, D, top, ls, y);
  }
}

// shares of a kv head's tokens: one of them has no parts to join
static int ad_shares(const parse_kv *kv, int n_q) {
  const int columns = kv->n_kv * ((n_q / kv->n_kv + AD_HEADS - 1) / AD_HEADS);
  return columns >= AD_GROUPS ? 1 : AD_GROUPS / columns;
}
static size_t ad_bytes(const parse_kv *kv, int n_q) {
  const int columns = kv->n_kv * ((n_q / kv->n_kv + AD_HEADS - 1) / AD_HEADS);
  return AD_TICKET_BYTES + round_up((size_t)columns * ad_shares(kv, n_q) * 2 * AD_HEADS * (kv->d + 2) * 4, 256);
}

// One launch where the workgroup that comes last has little to join (at most 256 KiB of parts); where it has more, a second launch spreads it over the heads
static bool ad_tickets(const parse_kv *kv, int n_q) {
  const int64_t weights = (int64_t)ad_shares(kv, n_q) * std::min(n_q / kv->n_kv, AD_HEADS);
  return weights * kv->d <= 65536 && 2 * weights <= AD_WAVES * AD_HEADS * kv->d;    // ... in the LDS that the sums left
}

// Steps that a row has at most, by table and window alone
static int64_t ad_most_steps(const parse_kv *kv, int window, int sinks) {
  const int64_t steps = ((int64_t)kv->max_pages * kv->page + AD_STEP - 1) / AD_STEP;
  if (window == 0) return steps;
  return std::min(steps, ((int64_t)window + AD_STEP - 1) / AD_STEP + 1 + ((int64_t)sinks + AD_STEP - 1) / AD_STEP);
}
// The steps of all rows are added up and dealt out in an int; room for what rounding a share's number up adds (4 * AD_WAVES) and for the shares
constexpr int64_t AD_MAXSTEPS = INT32_MAX - 2 * AD_GROUPS;

// Whether table and window alone say that every row is a share's (ad_by_rows), whatever the lengths
static bool ad_sure(const AdArgs &a) { return a.rows <= a.shares && ad_most_steps(&a.kv, a.window, a.sinks) <= AD_WAVES + ad_slack(a.rows); }

template <class T, int DT, bool NT, bool TICKETS>
static int ad_launch(const AdArgs &a, hipStream_t s) {
  const int zs = (a.group + AD_HEADS - 1) / AD_HEADS, scan = a.rows > 64 ? a.rows + 1 : 0;
  const size_t lds = (size_t)AD_WAVES * AD_HEADS * (DT * 32 + 2) * 4 + (AD_WAVES + scan) * 4;
  PARSE_ALLOW_LDS((attend_decode<T, DT, NT, TICKETS>), 0, lds);
  attend_decode<T, DT, NT, TICKETS><<<dim3(a.shares, a.kv.n_kv, zs), AD_THREADS, lds, s>>>(a);
  PARSE_LAUNCH_CHECK();
  if (!TICKETS && a.shares > 1 && !ad_sure(a)) {
    attend_join<T><<<dim3(std::min(a.shares - 1, a.rows), a.n_q), AD_THREADS, (AD_GROUPS + AD_THREADS * 4 + 3 * AD_WAVES + scan) * 4, s>>>(a);
    PARSE_LAUNCH_CHECK();
  }
  return PARSE_OK;
}
// A pool larger than the last-level cache is taken to be new to it in every step: loads that do not stay there (100003 tokens of 8 heads 81.5 -> 77.8 us, 192 windows 162 -> 153); a
// smaller one may be found there again (four caches of 3000 to 4000 tokens, 16 heads of 64 columns: 18.1 us, 20.2 with such loads).  How much of a pool a call reads only the
// device knows, and between two calls for a layer stand those for the others.
template <class T, int DT>
static int ad_form(const AdArgs &a, hipStream_t s) {
  const bool nt = (size_t)a.kv.n_layers * a.kv.n_pages * a.kv.n_kv * a.kv.page * a.kv.d * sizeof(T) * 2 > ((size_t)192 << 20), tickets = ad_tickets(&a.kv, a.n_q);
  if (nt) return tickets ? ad_launch<T, DT, true, true>(a, s) : ad_launch<T, DT, true, false>(a, s);
  return tickets ? ad_launch<T, DT, false, true>(a, s) : ad_launch<T, DT, false, false>(a, s);
}
template <class T>
static int ad_width(const AdArgs &a, hipStream_t s) {
  switch (a.kv.d / 32) {
    case 1: return ad_form<T, 1>(a, s);
    case 2: return ad_form<T, 2>(a, s);
    case 3: return ad_form<T, 3>(a, s);
    case 4: return ad_form<T, 4>(a, s);
    case 5: return ad_form<T, 5>(a, s);
    case 6: return ad_form<T, 6>(a, s);
    case 7: return ad_form<T, 7>(a, s);
    default: return ad_form<T, 8>(a, s);
  }
}

int check_attend(const parse_kv *kv, int layer, const void *q, int64_t q_stride, int n_q, int rows, const int32_t *tok_offsets, const int32_t *seqs, float scale,
                 int window, int sinks, const void *out, int64_t out_stride, const float *lse) {
  const int st = check_kv(kv, false);
  if (st != PARSE_OK) return st;
  if (!q || !out || n_q <= 0 || rows <= 0 || layer < 0 || window < 0 || sinks < 0 || !(fabsf(scale) < 1e38f)) return PARSE_EINVAL;
  if (layer >= kv->n_layers || n_q % kv->n_kv != 0 || n_q > 65536 || (int64_t)rows * n_q > INT32_MAX) return PARSE_ESHAPE;
  if (q_stride < (int64_t)n_q * kv->d || out_stride < (int64_t)n_q * kv->d) return PARSE_ESHAPE;
  const int per16 = 16 / elem_size(kv->dtype);
  if (!aligned16(q) || !aligned16(out) || !aligned4(lse) || !aligned4(tok_offsets) || !aligned4(seqs) || q_stride % per16 != 0 || out_stride % per16 != 0) return PARSE_EALIGN;
  return PARSE_OK;
}

}  // namespace parse

extern "C" {

size_t parse_attend_decode_workspace_bytes(const parse_kv *kv, int32_t n_q, int32_t rows) {
  if (parse::check_kv(kv, false) != PARSE_OK || n_q <= 0 || n_q % kv->n_kv != 0 || n_q > 65536 || rows <= 0) return 0;
  return parse::ad_bytes(kv, n_q);
}

int parse_attend_decode(const parse_kv *kv, int32_t layer, const void *q, int64_t q_stride, int32_t n_q, int32_t rows, const int32_t *seqs, float scale,
                        int32_t window, int32_t sinks, void *out, int64_t out_stride, float *lse, void *workspace, size_t workspace_bytes,
                        parse_stream stream) {
  using namespace parse;
  const int st = check_attend(kv, layer, q, q_stride, n_q, rows, nullptr, seqs, scale, window, sinks, out, out_stride, lse);
  if (st != PARSE_OK) return st;
  if (rows > KV_MAXSEQ || (!seqs && rows > kv->n_seqs) || rows * ad_most_steps(kv, window, sinks) > AD_MAXSTEPS) return PARSE_ESHAPE;
  if (!workspace || workspace_bytes < ad_bytes(kv, n_q)) return PARSE_EWORKSPACE;
  if (!aligned16(workspace)) return PARSE_EALIGN;
  const size_t at = (size_t)layer * kv->n_pages * kv->n_kv * kv->page * kv->d * elem_size(kv->dtype);
  AdArgs a{};
  a.kv = *kv;
  a.K = (const char *)kv->K + at; a.V = (const char *)kv->V + at;
  a.q = q; a.out = out; a.lse = lse; a.seqs = seqs;
  a.q_stride = q_stride; a.out_stride = out_stride;
  a.n_q = n_q; a.group = n_q / kv->n_kv; a.rows = rows; a.window = window; a.sinks = sinks;
  a.shares = ad_shares(kv, n_q);
  at_scale(scale, a.scale, a.lag, a.q_sign);
  a.tickets = (int32_t *)workspace;
  a.part = (float *)((char *)workspace + AD_TICKET_BYTES);
  return kv->dtype == PARSE_BF16 ? ad_width<uint16_t>(a, (hipStream_t)stream) : ad_width<float>(a, (hipStream_t)stream);
}

}  // extern "C"
