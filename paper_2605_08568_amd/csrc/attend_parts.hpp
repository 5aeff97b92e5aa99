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
constexpr int PT_MAXENTRIES = 16384, PT_MAXENTRIES_WIDE = 8176;     // their sums stand in LDS beside the ring, which is 128 KiB for fp32 heads wider than 160 columns

// Blocks of sixteen columns that a wavefront has of a wide entry: what the registers hold of q and of the sums beside a step of K and V.  The four wavefronts make TC columns.
template <class T, int DT> constexpr int pt_blocks() { return DT * (int)sizeof(T) <= 8 ? 2 : 1; }
static inline int pt_columns(int d, int dtype) { return 64 * (d / 32 * elem_size(dtype) <= 8 ? 2 : 1); }
// Steps in LDS, the one that is worked on and those on their way: 64 KiB of them where two fit
template <class T, int DT> constexpr int pt_step_bytes() { return 2 * PT_STEP * DT * 32 * (int)sizeof(T); }
template <class T, int DT> constexpr int pt_stages() { return pt_step_bytes<T, DT>() >= 32768 ? 2 : pt_step_bytes<T, DT>() > 16384 ? 3 : 4; }
// Workgroups that a compute unit has at once
template <class T, int DT> constexpr int pt_at_once() { return DT * (int)sizeof(T) <= 8 ? 2 : 1; }

// ---- the plan's words
struct PtTile {
  int list, seq, first, columns;                     // members of the run from `list` on; the shortest row's row of the table; the tile's first column among the members' (member * group + head), how many
  int from, to, base, pos;                           // tokens [from, to), multiples of PT_STEP; columns of the tiles before; the shortest row's position
};
struct PtRow {
  int from, levels;                                  // first token of its own, runs
  int tile[PT_LEVELS], column[PT_LEVELS];            // first tile of the run, the row's first column among the run's
};
static_assert(sizeof(PtTile) == 32 && sizeof(PtRow) == 32, "read as words");
struct PtHead {
  int rows, group, columns, window, sinks, n_pages, max_pages, page;    // what the plan was made for
  int tiles, tile_columns, n_seqs, pad[5];
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
  int32_t *deal;                                     // {steps of a share, entry x is share x, entries, columns of the tiles, steps before entry 0 .. entries}
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

// The first token that a row sees may stand in a page that the row has given up: pages are given up by what the NEXT token sees, so the page that ends with this one's first
// token goes as well.  Its column, or -1 where the window does not begin with a page's last token.  (Of a page that holds a sink nothing is given up.)
__device__ __forceinline__ int pt_edge(const parse_kv &kv, int lo) { return ((lo + 1) & (kv.page - 1)) == 0 ? lo / kv.page : -1; }
__device__ __forceinline__ bool pt_holds(const parse_kv &kv, int row, int column) {
  return (unsigned)kv.table[(int64_t)row * kv.max_pages + column] < (unsigned)kv.n_pages;
}

// The shortest sequence of a tile's rows: its table's row (its window reaches back the furthest, and no longer one has given up less; of equally short ones one that still
// holds the page of the first token that they see) and position.  By a whole wavefront, a lane one or two rows: a tile has no more rows than its (at most 128) columns.
struct PtShortest {
  int row, pos;
};
__device__ __forceinline__ PtShortest pt_shortest(const PtArgs &a, const PtTile &t) {
  const int m0 = t.first / a.group, m1 = (t.first + t.columns - 1) / a.group, m = m0 + (int)(threadIdx.x & 63);
  KvSeq q = kv_seq(a.kv, a.seqs, a.plan.list[t.list + min(m, m1)]), r = q;
  if (m1 - m0 >= 64) r = kv_seq(a.kv, a.seqs, a.plan.list[t.list + min(m + 64, m1)]);
  auto len = [](const KvSeq &s) { return s.len > 0 ? s.len : 0x7fffffff; };
  int least = min(len(q), len(r));
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) least = min(least, __shfl_xor(least, o, 64));
  least = __builtin_amdgcn_readfirstlane(least);
  if (least == 0x7fffffff) return PtShortest{0, -1};
  const int edge = pt_edge(a.kv, kv_window_begin(least - 1, a.window));
  bool of_q = len(q) == least, of_r = len(r) == least;
  uint64_t q_lanes = __ballot(of_q), r_lanes = __ballot(of_r);
  if (edge >= 0 && __popcll(q_lanes | r_lanes) > 1) {
    of_q = of_q && pt_holds(a.kv, q.row, edge);
    of_r = of_r && pt_holds(a.kv, r.row, edge);
    if (__any(of_q || of_r)) { q_lanes = __ballot(of_q); r_lanes = __ballot(of_r); }
  }
  const int row = q_lanes ? __builtin_amdgcn_readlane(q.row, __builtin_ctzll(q_lanes)) : __builtin_amdgcn_readlane(r.row, __builtin_ctzll(r_lanes));
  return PtShortest{row, least - 1};
}

// Whether the plan was made for such a call; one that was not shares nothing
__device__ __forceinline__ bool pt_fits(const PtArgs &a, int columns) {
  const PtHead &h = *a.plan.head;
  return h.rows == a.rows && h.group == a.group && h.columns == columns && h.window == a.window && h.sinks == a.sinks && h.n_pages == a.kv.n_pages && h.n_seqs == a.kv.n_seqs &&
         h.max_pages == a.kv.max_pages && h.page == a.kv.page && h.tiles >= 0 && h.tiles <= a.most_tiles;
}

// ---- host
static inline int pt_shares(const parse_kv *kv) {
  const int workgroups = kv->d / 32 * elem_size(kv->dtype) <= 8 ? 512 : 256;         // what the card has at once (pt_at_once)
  return kv->n_kv >= workgroups ? 1 : workgroups / kv->n_kv;
}
static inline size_t pt_deal_bytes(int64_t entries) { return round_up((PT_DEAL + (size_t)entries + 1) * 4, 256); }

// The two kernels, for heads of any width (attend_parts_kernels.hpp); entries: how many there are at most
template <class T, bool LISTED> int pt_width(const PtArgs &a, int64_t entries, hipStream_t s);

}  // namespace parse
