// Attention of one new token per sequence where the work is cut by what is read, not by rows (parse_attend_shared, parse_attend_pages): the kernel that
// makes the parts and the one that joins them.
//
// The work of a kv head is a list of entries.  An entry is a set of query columns (row and query head) that read the same tokens:
//   a tile  up to TC columns of the rows that share a run of pages (the plan has made the list)
//   a row   the columns of one row, up to TC of its heads: what it has for itself (SHARED), or the pages that were chosen for it (LISTED)
// The steps (32 tokens) of all entries stand one after another and are dealt out to the workgroups in equal shares.  Where share x meets entry e there is a part: the
// columns' running maximum, sum of weights and weighted sum of V over the tokens that the share has of it.  Parts stand at column x * TC + base[e] of the
// workspace (base: columns of the entries before), which no two of them have in common.
#pragma once
#include "attend.hpp"

namespace parse {

constexpr int PT_WAVES = 4, PT_THREADS = PT_WAVES * 64;
constexpr int PT_STEP = 32;
constexpr int PT_LEVELS = 3;                         // runs of shared pages that a row may have one behind another
constexpr int PT_MAXENTRIES = 16384;

// Columns of a tile, in blocks of sixteen: what the registers hold of q and of the sums beside a step of K and V
template <class T, int DT> constexpr int pt_blocks() { return DT * (int)sizeof(T) <= 8 ? 4 : DT * (int)sizeof(T) <= 16 ? 2 : 1; }
static inline int pt_columns(int d, int dtype) { const int w = d / 32 * elem_size(dtype); return 16 * (w <= 8 ? 4 : w <= 16 ? 2 : 1); }

// ---- the plan's words
struct PtTile {
  int list, members, first, columns;                 // members of the run from `list` on; the tile's first column among theirs (member * group + head), how many
  int from, to, base, pos;                           // tokens [from, to), multiples of PT_STEP; columns of the tiles before; the shortest row's position
};
struct PtRow {
  int from, levels;                                  // first token of its own, runs
  int tile[PT_LEVELS], column[PT_LEVELS];            // first tile of the run, the row's first column among the run's
};
static_assert(sizeof(PtTile) == 32 && sizeof(PtRow) == 32, "read as words");
struct PtHead {
  int rows, group, columns, window, sinks, n_pages, max_pages, page;    // what the plan was made for
  int tiles, tile_columns, pad[6];
};
static_assert(sizeof(PtHead) == 64, "");
struct PtPlan {
  PtHead *head;
  PtRow *row;
  PtTile *tile;
  int32_t *list;                                     // [PT_LEVELS * rows]
  // only while it is made
  int4 *walk;                                        // [rows][PT_LEVELS]: from, to, leader, whether there is one
  unsigned long long *owner;                         // [n_pages]
  int32_t *users;                                    // [n_pages]
  size_t bytes;
};
static inline int64_t pt_most_tiles(int rows, int group, int columns) {
  return PT_LEVELS * ((int64_t)rows * group / columns + rows / 2 + 1);
}
static inline PtPlan pt_plan(const parse_kv *kv, int rows, int group, const void *plan) {
  PtPlan p;
  char *at = (char *)plan;
  auto take = [&](size_t n) { char *r = at; at += round_up(n, 64); return r; };
  p.head = (PtHead *)take(sizeof(PtHead));
  p.row = (PtRow *)take((size_t)rows * sizeof(PtRow));
  p.tile = (PtTile *)take((size_t)pt_most_tiles(rows, group, pt_columns(kv->d, kv->dtype)) * sizeof(PtTile));
  p.list = (int32_t *)take((size_t)PT_LEVELS * rows * 4);
  p.walk = (int4 *)take((size_t)rows * PT_LEVELS * 16);
  p.owner = (unsigned long long *)take((size_t)kv->n_pages * 8);
  p.users = (int32_t *)take((size_t)kv->n_pages * 4);
  p.bytes = at - (char *)plan;
  return p;
}

// ---- arguments
struct PtArgs {
  parse_kv kv;
  const void *K, *V;                                 // of the layer
  const void *q;
  void *out;
  float *lse;
  const int32_t *seqs;
  int64_t q_stride, out_stride;
  int n_q, group, rows, shares, per_row, window, sinks;      // per_row: entries of a row, ceil(group / TC)
  float scale, lag;
  uint32_t q_sign;
  PtPlan plan;                                       // SHARED
  int most_tiles;
  const int32_t *pages;                              // LISTED: [row][kv head][top]
  int top;
  int32_t *deal;                                     // {share, by rows, entries, 0, steps before entry 0 .. entries}
  float *part;
};
constexpr int PT_DEAL = 4;

// The tokens that rows at [i0, ...] see of [from, to), in tiles of PT_STEP; from is a multiple of it.  Tile number t begins at token at(t) * PT_STEP.
struct PtSpan {
  int f, sink_tiles, a, count;
  __device__ __forceinline__ int at(int t) const { return t < sink_tiles ? f + t : a + (t - sink_tiles); }
};
__device__ __forceinline__ PtSpan pt_span(int i0, int from, int to, int window, int sinks) {
  PtSpan s{from / PT_STEP, 0, from / PT_STEP, 0};
  if (to <= from) return s;
  const int end = (to + PT_STEP - 1) / PT_STEP;
  if (window > 0) {
    s.a = min(max(s.f, kv_window_begin(i0, window) / PT_STEP), end);
    const int st = (int)min(((int64_t)sinks + PT_STEP - 1) / PT_STEP, (int64_t)s.a);
    s.sink_tiles = max(st - s.f, 0);
  }
  s.count = s.sink_tiles + end - s.a;
  return s;
}

// The shortest sequence of a tile's rows: its table's row (its window reaches back the furthest, and no other of them has given up pages that it still holds) and
// position.  By a whole wavefront, a lane a row: a tile has no more rows than columns.
struct PtShortest {
  int row, pos;
};
__device__ __forceinline__ PtShortest pt_shortest(const PtArgs &a, const PtTile &t) {
  const int m0 = t.first / a.group, m1 = (t.first + t.columns - 1) / a.group, m = m0 + (int)(threadIdx.x & 63);
  const KvSeq q = kv_seq(a.kv, a.seqs, a.plan.list[t.list + min(m, m1)]);
  const int len = q.len > 0 ? q.len : 0x7fffffff;
  int least = len;
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) least = min(least, __shfl_xor(least, o, 64));
  const int at = __builtin_ctzll(__ballot(len == least));
  return PtShortest{__builtin_amdgcn_readlane(q.row, at), least == 0x7fffffff ? -1 : __builtin_amdgcn_readfirstlane(least) - 1};
}

// Whether the plan was made for such a call; one that was not shares nothing
__device__ __forceinline__ bool pt_fits(const PtArgs &a, int columns) {
  const PtHead &h = *a.plan.head;
  return h.rows == a.rows && h.group == a.group && h.columns == columns && h.window == a.window && h.sinks == a.sinks && h.n_pages == a.kv.n_pages &&
         h.max_pages == a.kv.max_pages && h.page == a.kv.page && h.tiles >= 0 && h.tiles <= a.most_tiles;
}

// Entry x is share x, whole, where no entry has many more steps than an equal share would
constexpr int PT_SLACK = 12;

// A step of 32 tokens: s = K q (operand A = K, token rows; operand B = q, a column of the entry), weights 2^(scale s - base), o += V^T p.  K's rows are taken in the order in
// which the scores come back as operand B: rows 4 q + 0..3 of the two instructions of a step are tokens 8 q + 0..3 and 8 q + 4..7, so that a lane's eight weights are
// the eight tokens whose V it has loaded.  Operands go straight from the pages into registers, a step ahead of the one that is worked on where two steps fit; they are
// multiplied with up to NB blocks of sixteen columns.  bf16: a weight is multiplied as two bf16 numbers, as in the decode attention.
template <class T, int DT, int NB, bool LISTED>
__global__ __launch_bounds__(PT_THREADS, NB == 1 && DT * sizeof(T) <= 8 ? 2 : 1) void attend_parts(PtArgs a) {
  constexpr int D = DT * 32, KB = D / 32, VB = D / 16, TC = 16 * NB, RD = D + 4;
  typedef typename Op<T>::frag frag;
  extern __shared__ char smem[];
  float *red = reinterpret_cast<float *>(smem);                    // [wave][16][RD]
  float *red_m = red + PT_WAVES * 16 * RD, *red_l = red_m + PT_WAVES * TC;       // [wave][TC]
  int *wave_sums = reinterpret_cast<int *>(red_l + PT_WAVES * TC), *pre = wave_sums + PT_WAVES;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int n = lane & 15, quad = lane >> 4;
  const int share = blockIdx.x, kvh = blockIdx.y;
  int tiles = 0, tile_columns = 0;
  bool fits = false;
  if constexpr (!LISTED) {
    fits = pt_fits(a, TC);
    if (fits) { tiles = a.plan.head->tiles; tile_columns = a.plan.head->tile_columns; }
  }
  const int entries = tiles + a.rows * a.per_row;
  const int list_steps = LISTED ? (int)(((int64_t)a.top * a.kv.page + PT_STEP - 1) / PT_STEP) : 0;
  auto own_span = [&](int row, const KvSeq &s) { return pt_span(s.len - 1, fits ? min(a.plan.row[row].from, s.len) : 0, s.len, a.window, a.sinks); };
  auto count_of = [&](int e) {
    if constexpr (LISTED) return list_steps;
    if (e < tiles) {
      const PtTile t = a.plan.tile[e];
      return pt_span(t.pos, t.from, t.to, a.window, a.sinks).count;
    }
    const int row = (e - tiles) / a.per_row;
    return own_span(row, kv_seq(a.kv, a.seqs, row)).count;
  };
  int total;
  bool longer = false;
  if constexpr (LISTED) {
    total = list_steps * entries;
  } else {
    kv_prefix<PT_THREADS>(entries, pre, wave_sums, count_of);
    total = pre[entries];
  }
  auto before_of = [&](int e) { return LISTED ? e * list_steps : pre[e]; };
  const int per = max(((total + a.shares - 1) / a.shares + PT_WAVES - 1) / PT_WAVES, 1) * PT_WAVES;
  bool by_rows = entries <= a.shares;
  if (by_rows) {
    for (int e = tid; e < entries; e += PT_THREADS) longer |= before_of(e + 1) - before_of(e) > per + PT_SLACK;
    by_rows = !__syncthreads_or(longer);
  }
  if (share == 0 && kvh == 0) {                                    // for the kernel that joins
    if (tid == 0) { a.deal[0] = per; a.deal[1] = by_rows; a.deal[2] = entries; }
    for (int e = tid; e <= entries; e += PT_THREADS) a.deal[PT_DEAL + e] = before_of(e);
  }
  if (by_rows && share >= entries) return;
  const int64_t begin = by_rows ? before_of(share) : (int64_t)share * per;
  const int end = (int)min(by_rows ? (int64_t)before_of(share + 1) : begin + per, (int64_t)total);
  if (begin >= end) return;
  const int64_t page_elems = (int64_t)a.kv.n_kv * a.kv.page * D, head0 = (int64_t)kvh * a.kv.page * D;
  const int tok = 8 * (n >> 2) + (n & 3);
  const int page_bits = 31 - __builtin_clz(a.kv.page);
  const int k_in = quad * 128 + (tok & 15) * 8, v_in = ((quad & 1) * D + n) * 8;
  const int e0 = LISTED ? (int)begin / list_steps : kv_find(pre, entries, (int)begin), e1 = LISTED ? (end - 1) / list_steps : kv_find(pre, entries, end - 1);
  float *parts = a.part + (int64_t)kvh * ((int64_t)a.shares * TC + (LISTED ? 0 : (int64_t)PT_LEVELS * a.rows * a.group) + (int64_t)a.rows * a.group) * RD;
  for (int e = __builtin_amdgcn_readfirstlane(e0); e <= e1; ++e) {
    const int before = __builtin_amdgcn_readfirstlane(before_of(e)), count = __builtin_amdgcn_readfirstlane(before_of(e + 1)) - before;
    if (count == 0) continue;
    // ---- the entry
    PtTile t{};
    int row = 0, z = 0, seq, columns, base, pos_of = -1;
    bool direct = false;
    int passed = 0;                                                // steps that were in sight when the plan was made and are no more
    PtSpan span{};
    const bool tile = !LISTED && e < tiles;
    if (tile) {
      t = a.plan.tile[e];
      const PtShortest s = pt_shortest(a, t);
      seq = s.row; columns = t.columns; base = t.base;
      span = pt_span(t.pos, t.from, t.to, a.window, a.sinks);
      passed = s.pos < 0 ? count : span.sink_tiles + max(pt_span(max(s.pos, t.pos), t.from, t.to, a.window, a.sinks).a - span.a, 0);
    } else {
      row = (e - tiles) / a.per_row; z = (e - tiles) % a.per_row;
      const KvSeq s = kv_seq(a.kv, a.seqs, row);
      seq = s.row; pos_of = s.len - 1;
      columns = min(a.group - z * TC, TC);
      base = tile_columns + row * a.group + z * TC;
      if constexpr (!LISTED) {
        span = own_span(row, s);
        direct = !fits || a.plan.row[row].levels == 0;
      } else {
        direct = true;
      }
    }
    seq = __builtin_amdgcn_readfirstlane(seq);
    columns = __builtin_amdgcn_readfirstlane(columns);
    base = __builtin_amdgcn_readfirstlane(base);
    const int first = max((int)begin - before, 0), last = min(end - before, count);
    const int start = (tile && first >= span.sink_tiles ? max(first, passed) : first) + wave;
    const int blocks = (columns + 15) / 16;
    const int32_t *table = a.kv.table + (int64_t)seq * a.kv.max_pages;
    const int32_t *list = LISTED ? a.pages + ((int64_t)row * a.kv.n_kv + kvh) * a.top : nullptr;
    frag qf[NB][KB];
    int pos[NB], lo[NB], least = 0x7fffffff, most = 0;
#pragma unroll
    for (int b = 0; b < NB; ++b) {
      const int c = min(16 * b + n, columns - 1);
      int r = row, h = z * TC + c;
      pos[b] = pos_of;
      if (tile) {
        const int f = t.first + c, m = f / a.group;
        r = a.plan.list[t.list + m];
        h = f - m * a.group;
        pos[b] = kv_seq(a.kv, a.seqs, r).len - 1;
      }
      lo[b] = LISTED ? 0 : kv_window_begin(pos[b], a.window);
      least = min(least, pos[b]);
      most = max(most, lo[b]);
      const T *q = reinterpret_cast<const T *>(a.q) + (int64_t)r * a.q_stride + (int64_t)(kvh * a.group + h) * D;
#pragma unroll
      for (int k = 0; k < KB; ++k) qf[b][k] = Op<T>::sign(Op<T>::load(q + 32 * k + 8 * quad), a.q_sign);
    }
#pragma unroll
    for (int o = 8; o > 0; o >>= 1) { least = min(least, __shfl_xor(least, o, 64)); most = max(most, __shfl_xor(most, o, 64)); }
    least = __builtin_amdgcn_readfirstlane(least);
    most = __builtin_amdgcn_readfirstlane(most);
    float m[NB], l[NB];
    f32x4 o[NB][VB];
    auto clear = [&]() {
#pragma unroll
      for (int b = 0; b < NB; ++b) {
        m[b] = -INFINITY; l[b] = 0.f;
#pragma unroll
        for (int v = 0; v < VB; ++v) o[b][v] = f32x4{0.f, 0.f, 0.f, 0.f};
      }
    };
    clear();
    // the wavefront's next 64 steps, a lane each: page and first token of their two halves, -1 for none
    int id_a = -1, id_b = -1, at_a = 0, at_b = 0;
    struct Step {
      frag k0[KB], k1[KB], v[VB];
      int ta, tb;
      bool there_a, there_b;
    };
    auto load = [&](Step &x, int j) {
      const int u = start + j * PT_WAVES;
      if ((j & 63) == 0) {
        const int mine = min(u + lane * PT_WAVES, count - 1);
        if constexpr (LISTED) {
          auto half = [&](int block, int &id, int &at) {           // block of sixteen tokens of the listed pages
            const int i = block >> (page_bits - 4);
            const int c = i < a.top ? list[i] : -1;
            const bool ok = (unsigned)c < (unsigned)a.kv.max_pages;
            id = ok ? table[c] : -1;
            at = (ok ? c : 0) * a.kv.page + (block & ((a.kv.page >> 4) - 1)) * 16;
          };
          half(2 * mine, id_a, at_a);
          half(2 * mine + 1, id_b, at_b);
        } else {
          at_a = span.at(mine) * PT_STEP;
          at_b = at_a + 16;
          id_a = table[min(at_a >> page_bits, a.kv.max_pages - 1)];
          id_b = table[min(at_b >> page_bits, a.kv.max_pages - 1)];
        }
      }
      const int ida = __builtin_amdgcn_readlane(id_a, j & 63), idb = __builtin_amdgcn_readlane(id_b, j & 63);
      x.ta = __builtin_amdgcn_readlane(at_a, j & 63);
      x.tb = LISTED ? __builtin_amdgcn_readlane(at_b, j & 63) : x.ta + 16;
      x.there_a = (unsigned)ida < (unsigned)a.kv.n_pages;
      x.there_b = (unsigned)idb < (unsigned)a.kv.n_pages;
      const int64_t pa = (int64_t)(x.there_a ? ida : 0) * page_elems + head0 + (int64_t)(x.ta & (a.kv.page - 1)) * D;
      const int64_t pb = (int64_t)(x.there_b ? idb : 0) * page_elems + head0 + (int64_t)(x.tb & (a.kv.page - 1)) * D;
      const T *kp = reinterpret_cast<const T *>(a.K) + (n < 8 ? pa : pb) + k_in;
      const T *vp = reinterpret_cast<const T *>(a.V) + (quad < 2 ? pa : pb) + v_in;
#pragma unroll
      for (int k = 0; k < KB; ++k) { x.k0[k] = Op<T>::load(kp + k * 512); x.k1[k] = Op<T>::load(kp + k * 512 + 32); }
#pragma unroll
      for (int v = 0; v < VB; ++v) x.v[v] = Op<T>::load(vp + v * 128);
    };
    // which of the lane's eight tokens a row at position i sees
    auto seen = [&](const Step &x, int i, int from) -> uint32_t {
      const bool there = quad < 2 ? x.there_a : x.there_b;
      const int j0 = (quad < 2 ? x.ta : x.tb) + 8 * (quad & 1);
      return there ? kv_sees8(i, from, LISTED ? 0 : a.sinks, j0) : 0u;
    };
    auto work = [&](Step &x, auto careful) {
      constexpr bool CAREFUL = decltype(careful)::value;
      const bool whole = x.there_a && x.there_b && x.ta + 15 <= least && x.tb + 15 <= least && (x.ta >= most || x.ta + PT_STEP <= a.sinks);
      uint32_t keep[NB];
      if (!whole) {                                                // what no column sees: nothing of V to multiply with
        uint32_t any = 0;
#pragma unroll
        for (int b = 0; b < NB; ++b) { keep[b] = seen(x, pos[b], lo[b]); any |= keep[b]; }
#pragma unroll
        for (int s = 8; s > 0; s >>= 1) any |= __shfl_xor(any, s, 64);
        if (!CAREFUL) {
#pragma unroll
          for (int v = 0; v < VB; ++v) x.v[v] = Op<T>::only(x.v[v], any);
        }
      } else {
#pragma unroll
        for (int b = 0; b < NB; ++b) keep[b] = 0xffu;
      }
#pragma unroll
      for (int b = 0; b < NB; ++b) {
        if (b >= blocks) break;
        f32x4 s0 = {0.f, 0.f, 0.f, 0.f}, s1 = s0;
#pragma unroll
        for (int k = 0; k < KB; ++k) { s0 = Op<T>::mma16(x.k0[k], qf[b][k], s0); s1 = Op<T>::mma16(x.k1[k], qf[b][k], s1); }
        float s[8];
#pragma unroll
        for (int e = 0; e < 4; ++e) { s[e] = s0[e]; s[4 + e] = s1[e]; }
        if (!whole) {
#pragma unroll
          for (int e = 0; e < 8; ++e) s[e] = keep[b] >> e & 1 ? s[e] : -INFINITY;
        }
        float top = s[0];
#pragma unroll
        for (int e = 1; e < 8; ++e) top = fmaxf(top, s[e]);
        if (__any(top > m[b] + a.lag)) {
          const float grown = fmaxf(m[b], lane_max<32>(lane_max<16>(top)));
          const float by = at_exp2((m[b] - finite_or_0(grown)) * a.scale);
          l[b] *= by;
#pragma unroll
          for (int v = 0; v < VB; ++v) o[b][v] *= by;
          m[b] = grown;
        }
        const float off = at_base(m[b], a.scale);
        float p[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) { p[e] = at_exp2(fmaf(s[e], a.scale, -off)); l[b] += p[e]; }
        const frag pf = Op<T>::pack(p);
        if constexpr (!CAREFUL) {
#pragma unroll
          for (int v = 0; v < VB; ++v) o[b][v] = Op<T>::mma16(x.v[v], pf, o[b][v]);
          if constexpr (sizeof(T) == 2) {
            const frag rest = Op<T>::pack_rest(p, pf);
#pragma unroll
            for (int v = 0; v < VB; ++v) o[b][v] = Op<T>::mma16(x.v[v], rest, o[b][v]);
          }
        } else {                                                   // column after column, each with what it sees of V
          for (int c = 0; c < 16; ++c) {
            const uint32_t sees = whole ? 0xffu : seen(x, __builtin_amdgcn_readlane(pos[b], c), __builtin_amdgcn_readlane(lo[b], c));
#pragma unroll
            for (int v = 0; v < VB; ++v) {
              const frag vc = Op<T>::only(x.v[v], sees);
              const f32x4 add = Op<T>::mma16(vc, pf, f32x4{0.f, 0.f, 0.f, 0.f});
              f32x4 more = {0.f, 0.f, 0.f, 0.f};
              if constexpr (sizeof(T) == 2) more = Op<T>::mma16(vc, Op<T>::pack_rest(p, pf), more);
#pragma unroll
              for (int e = 0; e < 4; ++e) o[b][v][e] += n == c ? add[e] + (fabsf(more[e]) < INFINITY ? more[e] : 0.f) : 0.f;
            }
          }
        }
      }
    };
    const int steps = last > start ? (last - start + PT_WAVES - 1) / PT_WAVES : 0;
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
    {
      // An infinity or NaN of V that some columns see and others do not makes NaN of a weight of zero, and so does what the rounding of a weight left.  Where
      // something that is not finite came out, once more column by column.
      f32x4 sum = {0.f, 0.f, 0.f, 0.f};                            // NaN where one of them is not finite
#pragma unroll
      for (int b = 0; b < NB; ++b)
#pragma unroll
        for (int v = 0; v < VB; ++v)
#pragma unroll
          for (int i = 0; i < 4; ++i) sum[i] = fmaf(o[b][v][i], 0.f, sum[i]);
      if (__any((sum[0] + sum[1]) + (sum[2] + sum[3]) != 0.f)) {
        clear();
        for (int j = 0; j < steps; ++j) {
          load(even, j);
          work(even, std::true_type{});
        }
      }
    }
    // ---- the wavefronts' sums meet, sixteen columns after another
#pragma unroll
    for (int b = 0; b < NB; ++b) l[b] = lane_sum<32>(lane_sum<16>(l[b]));
    __syncthreads();
    if (quad == 0) {
#pragma unroll
      for (int b = 0; b < NB; ++b) { red_m[wave * TC + 16 * b + n] = m[b]; red_l[wave * TC + 16 * b + n] = l[b]; }
    }
    const bool all = direct && first == 0 && last == count;
    float *part = parts + ((int64_t)share * TC + base) * RD;
#pragma unroll
    for (int b = 0; b < NB; ++b) {
      if (b >= blocks) break;
      if (b) __syncthreads();
#pragma unroll
      for (int v = 0; v < VB; ++v) *reinterpret_cast<f32x4 *>(red + (wave * 16 + n) * RD + 16 * v + 4 * quad) = o[b][v];
      __syncthreads();
      const int here = min(columns - 16 * b, 16);
      for (int w = tid; w < here * D; w += PT_THREADS) {
        const int h = w / D, i = w % D, c = 16 * b + h;
        float top = -INFINITY, ls = 0.f, os = 0.f;
#pragma unroll
        for (int x = 0; x < PT_WAVES; ++x) top = fmaxf(top, red_m[x * TC + c]);
#pragma unroll
        for (int x = 0; x < PT_WAVES; ++x) {
          const float by = at_exp2((red_m[x * TC + c] - finite_or_0(top)) * a.scale);
          ls += by * red_l[x * TC + c];
          os += by * red[(x * 16 + h) * RD + i];
        }
        if (all) {
          const int head = kvh * a.group + z * TC + c;
          const float y = ls == 0.f ? 0.f : os / ls;
          T *out = reinterpret_cast<T *>(a.out) + (int64_t)row * a.out_stride + (int64_t)head * D + i;
          if constexpr (sizeof(T) == 2) *out = (uint16_t)cvt_pk_bf16(y, 0.f);
          else *out = y;
          if (a.lse && i == 0) a.lse[(int64_t)row * a.n_q + head] = at_lse(top, a.scale, ls);
        } else {
          part[(int64_t)c * RD + i] = os;
          if (i == 0) { part[(int64_t)c * RD + D] = top; part[(int64_t)c * RD + D + 1] = ls; }
        }
      }
    }
    __syncthreads();
  }
}

// The parts of one row's head, in the order of entries and shares.  Workgroup (head, row); a wavefront has every fourth part, a lane D / 64 columns of it and more.
template <class T, bool LISTED>
__global__ __launch_bounds__(PT_THREADS) void attend_parts_join(PtArgs a, int TC) {
  extern __shared__ char smem[];
  const int D = a.kv.d, RD = D + 4, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int row = blockIdx.y, head = blockIdx.x, kvh = head / a.group, g = head % a.group;
  const int per = a.deal[0], by_rows = a.deal[1], entries = a.deal[2], tiles = entries - a.rows * a.per_row;
  const int32_t *pre = a.deal + PT_DEAL;
  PtRow rec{};
  int tile_columns = 0;
  if (!LISTED && tiles > 0) { rec = a.plan.row[row]; tile_columns = a.plan.head->tile_columns; }
  // up to PT_LEVELS tiles and the row's own entry: first share, parts, column of the first part
  int x0[PT_LEVELS + 1], count[PT_LEVELS + 1], col[PT_LEVELS + 1], parts = 0;
  const int levels = min(max(rec.levels, 0), PT_LEVELS);
#pragma unroll
  for (int s = 0; s <= PT_LEVELS; ++s) {
    x0[s] = count[s] = col[s] = 0;
    int e = -1, c = 0;
    if (s == PT_LEVELS) {
      e = tiles + row * a.per_row + g / TC;
      c = tile_columns + row * a.group + g;
    } else if (s < levels) {
      const int f = rec.column[s] + g;
      e = rec.tile[s] + f / TC;
      if (e >= 0 && e < tiles) c = a.plan.tile[e].base + f % TC;
      else e = -1;
    }
    if (e >= 0) {
      const int from = pre[e], to = pre[e + 1];
      if (to > from) {
        x0[s] = by_rows ? e : from / per;
        count[s] = by_rows ? 1 : (to - 1) / per - x0[s] + 1;
        col[s] = c;
        parts += count[s];
      }
    }
  }
  if (levels == 0 && parts == 1) return;                           // stored by the share that had it
  const float *base = a.part + (int64_t)kvh * ((int64_t)a.shares * TC + (LISTED ? 0 : (int64_t)PT_LEVELS * a.rows * a.group) + (int64_t)a.rows * a.group) * RD;
  auto part_of = [&](int x) {
    int s = 0;
#pragma unroll
    for (int k = 0; k < PT_LEVELS; ++k)
      if (s == k && x >= count[k]) { x -= count[k]; s = k + 1; }
    int at = x0[0], c = col[0];
#pragma unroll
    for (int k = 1; k <= PT_LEVELS; ++k)
      if (s == k) { at = x0[k]; c = col[k]; }
    return base + ((int64_t)(at + x) * TC + c) * RD;
  };
  float *tops = reinterpret_cast<float *>(smem), *sums = tops + PT_WAVES, *os = sums + PT_WAVES;       // [wave][D]
  float top = -INFINITY;
  for (int x = tid; x < parts; x += PT_THREADS) top = fmaxf(top, part_of(x)[D]);
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor(top, o, 64));
  if (lane == 0) tops[wave] = top;
  __syncthreads();
  top = fmaxf(fmaxf(tops[0], tops[1]), fmaxf(tops[2], tops[3]));
  float ls = 0.f, y[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 4
  for (int x = wave; x < parts; x += PT_WAVES) {
    const float *p = part_of(x);
    const float by = at_exp2((p[D] - finite_or_0(top)) * a.scale);
    ls += by * p[D + 1];
#pragma unroll
    for (int k = 0; k < 4; ++k)
      if (lane + 64 * k < D) y[k] = fmaf(by, p[lane + 64 * k], y[k]);
  }
#pragma unroll
  for (int k = 0; k < 4; ++k)
    if (lane + 64 * k < D) os[wave * D + lane + 64 * k] = y[k];
  if (lane == 0) sums[wave] = ls;
  __syncthreads();
  ls = (sums[0] + sums[1]) + (sums[2] + sums[3]);
  for (int i = tid; i < D; i += PT_THREADS) {
    const float v = (os[i] + os[D + i]) + (os[2 * D + i] + os[3 * D + i]);
    const float r = ls == 0.f ? 0.f : v / ls;
    T *out = reinterpret_cast<T *>(a.out) + (int64_t)row * a.out_stride + (int64_t)head * D + i;
    if constexpr (sizeof(T) == 2) *out = (uint16_t)cvt_pk_bf16(r, 0.f);
    else *out = r;
    if (a.lse && i == 0) a.lse[(int64_t)row * a.n_q + head] = at_lse(top, a.scale, ls);
  }
}

// ---- host
static inline int pt_shares(int n_kv, int workgroups) { return n_kv >= workgroups ? 1 : workgroups / n_kv; }
static inline size_t pt_deal_bytes(int64_t entries) { return round_up((PT_DEAL + (size_t)entries + 1) * 4, 256); }
static inline size_t pt_lds(int d, int TC, int64_t entries) { return (size_t)(PT_WAVES * 16 * (d + 4) + 2 * PT_WAVES * TC) * 4 + (PT_WAVES + (size_t)entries + 1) * 4; }

template <class T, bool LISTED>
static int pt_join_launch(const PtArgs &a, int TC, hipStream_t s) {
  attend_parts_join<T, LISTED><<<dim3(a.n_q, a.rows), PT_THREADS, (2 * PT_WAVES + PT_WAVES * a.kv.d) * 4, s>>>(a, TC);
  PARSE_LAUNCH_CHECK();
  return PARSE_OK;
}
template <class T, int DT, int NB, bool LISTED>
static int pt_launch(const PtArgs &a, int64_t entries, hipStream_t s) {
  const size_t lds = pt_lds(DT * 32, 16 * NB, LISTED ? 0 : entries);
  PARSE_ALLOW_LDS((attend_parts<T, DT, NB, LISTED>), 0, lds);
  attend_parts<T, DT, NB, LISTED><<<dim3(a.shares, a.kv.n_kv), PT_THREADS, lds, s>>>(a);
  PARSE_LAUNCH_CHECK();
  return pt_join_launch<T, LISTED>(a, 16 * NB, s);
}

}  // namespace parse
