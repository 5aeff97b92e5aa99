// Attention of one new token per sequence for batches that begin alike (parse_shared_plan, parse_attend_shared): pages that several sequences of a
// call hold at their front are read once for all of them.
#include <algorithm>
#include <type_traits>

#include "attend_parts.hpp"

namespace parse {

constexpr int SH_THREADS = 256, SH_ONE = 1024;
constexpr int SH_NEAR_ROWS = 64;                    // a lane each
// Tokens of a run that is worth a tile: a step a wavefront.  128 / 64, us with the join: 32 prompts of 100 tokens with 4 samples each of up to 200 more 33.5 / 53, 4 with 16 samples
// 16.1 / 35, one of 77 with 4 samples 13.1 / 12.4
constexpr int SH_LEAST = 128;

// ---- the plan: which rows hold the same pages ------------------------------------------------------------------------
// Only whole pages in front of a row's last token count (those stay as they are while the sequence grows), and of them what the row sees or a later token of it
// will see.  owner[page]: the shortest of the rows that hold it (of equal ones the first); users[page]: how many do.
// Four launches, or two (below), made once for all layers and steps; bound by their latency.  One workgroup for a small batch was slower than four launches of 18 to 23 us (24 with
// its atomics in memory, 29 in LDS).
struct ShRow {
  KvSeq seq;
  int columns, lo, page, sinks;
  bool windowed;
  __device__ __forceinline__ bool cares(int c) const { return !windowed || (int64_t)c * page < sinks || (c + 1) * page > lo; }
  // ... where the table's word is known: the page that ends with the window's first token may have been given up already (pt_edge), and then the row does not see that token either
  __device__ __forceinline__ bool cares(int c, bool there) const { return cares(c) && (there || !windowed || (int64_t)c * page < sinks || (c + 1) * page != lo + 1); }
};
__device__ __forceinline__ ShRow sh_row(const parse_kv &kv, const int32_t *seqs, int row, int window, int sinks) {
  ShRow r;
  r.seq = kv_seq(kv, seqs, row);
  r.columns = r.seq.len > 0 ? min((r.seq.len - 1) / kv.page, kv.max_pages) : 0;
  r.lo = kv_window_begin(r.seq.len - 1, window);
  r.page = kv.page; r.sinks = sinks; r.windowed = window > 0;
  return r;
}

template <bool COUNT>
__global__ __launch_bounds__(SH_THREADS) void shared_count(parse_kv kv, const int32_t *__restrict__ seqs, int window, int sinks, PtPlan plan) {
  const int row = blockIdx.y;
  const ShRow r = sh_row(kv, seqs, row, window, sinks);
  const int32_t *table = kv.table + (int64_t)r.seq.row * kv.max_pages;
  for (int c = blockIdx.x * SH_THREADS + threadIdx.x; c < r.columns; c += gridDim.x * SH_THREADS) {
    const int id = table[c];
    if (!r.cares(c) || (unsigned)id >= (unsigned)kv.n_pages) continue;
    if (COUNT) {
      atomicMin(&plan.owner[id], (unsigned long long)(uint32_t)r.seq.len << 32 | (uint32_t)row);
      atomicAdd(&plan.users[id], 1);
    } else {
      plan.owner[id] = ~0ull;
      plan.users[id] = 0;
    }
  }
}

// Where rows are few, a workgroup a row instead: owner and users of 256 columns at once from the rows' tables themselves, a thread a column, sixteen rows asked for together
// (a page counts in the column that it stands in: another would not be shared anyway).  One launch instead of three; three / one, us without what lies between them: 4 rows of
// 5 columns 8.5 / 5.4, 36 of 75 13.7 / 8.4, 32 of 132 13.1 / 7.8, 64 of 132 14.0 / 11.0, 48 of 470 21.5 / 16.4; 96 of 200 (two rows a lane, from LDS) 13.6 / 18.6.
struct ShNear {
  int owner[SH_THREADS], users[SH_THREADS];
};
struct ShOther {                                       // a lane a row
  int at, columns, lo, len;                            // first word of the table's row; columns that it cares for are below `columns`, and from `lo` on or below the sinks' end
};
__device__ __forceinline__ void shared_near(const parse_kv &kv, const ShRow &r, const int32_t *table, int rows, int c, const ShOther &all, ShNear &sh) {
  const bool care = c < r.columns && r.cares(c), sink = r.windowed && (int64_t)c * r.page < r.sinks;
  const int cc = min(c, kv.max_pages - 1), id = care ? table[cc] : -1;
  int least = 0x7fffffff, owner = -1, users = 0;
#pragma unroll 1
  for (int r0 = 0; r0 < rows; r0 += 16) {
    int x[16];
#pragma unroll
    for (int j = 0; j < 16; ++j) x[j] = (kv.table + __builtin_amdgcn_readlane(all.at, r0 + j))[cc];
#pragma unroll
    for (int j = 0; j < 16; ++j) {
      const int len = __builtin_amdgcn_readlane(all.len, r0 + j);
      const bool has = (x[j] == id) & (c < __builtin_amdgcn_readlane(all.columns, r0 + j)) & (sink | (c >= __builtin_amdgcn_readlane(all.lo, r0 + j)));
      users += has ? 1 : 0;
      owner = has & (len < least) ? r0 + j : owner;
      least = has ? min(least, len) : least;
    }
  }
  const bool there = care && (unsigned)id < (unsigned)kv.n_pages;
  sh.owner[threadIdx.x] = there ? owner : -1;
  sh.users[threadIdx.x] = there ? users : 0;
}

// A wavefront walks a row's columns.  A run ends where the pages have another owner or fewer users; one of two users and more that is long enough (with what
// shorter ones left before it: their rows hold that too) is the row's next level.  Then the columns are compared with the owner's: the row takes part as far as they agree.
template <bool NEAR>
__global__ __launch_bounds__(SH_THREADS) void shared_walk(parse_kv kv, const int32_t *__restrict__ seqs, int rows, int window, int sinks, PtPlan plan) {
  __shared__ ShNear near;
  const int tid = threadIdx.x, lane = tid & 63, page = kv.page, row = NEAR ? blockIdx.x : blockIdx.x * (SH_THREADS / 64) + (tid >> 6);
  if (row >= rows) return;
  const ShRow r = sh_row(kv, seqs, row, window, sinks);
  ShOther all{};
  if (NEAR) {
    const ShRow x = sh_row(kv, seqs, min(lane, rows - 1), window, sinks);
    all = ShOther{x.seq.row * kv.max_pages, lane < rows ? x.columns : 0, x.lo / page, x.seq.len};
  }
  const int32_t *table = kv.table + (int64_t)r.seq.row * kv.max_pages;
  auto there = [&](int id) { return (unsigned)id < (unsigned)kv.n_pages; };
  int4 found[PT_LEVELS];
#pragma unroll
  for (int l = 0; l < PT_LEVELS; ++l) found[l] = int4{0, 0, -1, 0};
  int level = 0, from = 0, have = 0, owner = -2, users = 0;        // from: tokens; have: columns since then that the row cares for
  auto ends = [&](int c, int now) {                                // the run before column c, with `now` columns
    const int to = c * page & ~(PT_STEP - 1);
    if (users < 2 || owner < 0 || (int64_t)now * page < SH_LEAST || to <= from || level >= PT_LEVELS) return false;
#pragma unroll
    for (int l = 0; l < PT_LEVELS; ++l)
      if (l == level) found[l] = int4{from, to, owner, 1};
    ++level;
    from = to;
    return true;
  };
  for (int c0 = 0; c0 < r.columns; c0 += 64) {
    if (NEAR && (c0 & (SH_THREADS - 1)) == 0) {
      if (c0 > 0) __syncthreads();                                 // the columns before are read
      shared_near(kv, r, table, rows, c0 + tid, all, near);
      __syncthreads();
    }
    if (NEAR && tid >= 64) continue;
    const int c = c0 + lane;
    bool care = c < r.columns && r.cares(c);
    int o = -1, k = 0;
    if (NEAR) {
      o = near.owner[(c0 & (SH_THREADS - 1)) + lane];
      k = near.users[(c0 & (SH_THREADS - 1)) + lane];
      care = care && r.cares(c, k > 0);
    } else if (care) {
      const int id = table[c];
      if (there(id)) { o = (int)(uint32_t)plan.owner[id]; k = plan.users[id]; }
      care = r.cares(c, there(id));
    }
    const uint64_t cared = __ballot(care), below = cared & ((1ull << lane) - 1);
    const int prev = below ? 63 - __builtin_clzll(below) : 0;
    int po = __shfl(o, prev, 64), pk = __shfl(k, prev, 64);
    if (!below) { po = owner; pk = users; }
    uint64_t breaks = __ballot(care && (o != po || k < pk));
    int counted = 0;                                               // lanes before this one are in `have`
    while (breaks) {
      const int b = __builtin_ctzll(breaks);
      breaks &= breaks - 1;
      have += __popcll(cared & ((1ull << b) - 1) & ~((1ull << counted) - 1));
      counted = b;
      owner = __builtin_amdgcn_readlane(po, b);
      users = __builtin_amdgcn_readlane(pk, b);
      if (ends(c0 + b, have)) have = (c0 + b) * page > from ? 1 : 0;
    }
    have += __popcll(cared & ~((1ull << counted) - 1));
    if (cared) {
      const int at = 63 - __builtin_clzll(cared);
      owner = __builtin_amdgcn_readlane(o, at);
      users = __builtin_amdgcn_readlane(k, at);
    }
  }
  if (NEAR && tid >= 64) return;
  ends(r.columns, have);
#pragma unroll
  for (int l = 0; l < PT_LEVELS; ++l) {
    if (l >= level) break;
    const int lead = found[l].z;
    if (lead == row) continue;
    const int32_t *other = kv.table + (int64_t)kv_seq(kv, seqs, min((unsigned)lead, (unsigned)rows - 1)).row * kv.max_pages;
    bool same = true;
    for (int c = found[l].x / page + lane; c < found[l].y / page; c += 64) {
      const int x = table[c], y = other[c];
      if (!r.cares(c, there(x))) continue;
      same &= x == y || (!there(x) && !there(y));
    }
    if (!__all(same)) level = l;
  }
  if (lane < PT_LEVELS) {
    int4 w = found[0];
#pragma unroll
    for (int l = 1; l < PT_LEVELS; ++l)
      if (lane == l) w = found[l];
    if (lane >= level) w.w = 0;
    plan.walk[(int64_t)row * PT_LEVELS + lane] = w;
  }
}

// One workgroup, of 256 threads where they have a row each (36 rows 7.7 us, 8.7 with 1024): the rows that agree with their owner become its group, groups of two and more get tiles, level after level.  A thread has consecutive rows.
template <int THREADS>
__global__ __launch_bounds__(THREADS) void shared_tiles(parse_kv kv, const int32_t *__restrict__ seqs, int rows, int group, int TC, int window, int sinks, PtPlan plan) {
  extern __shared__ int4 words[];
  const int4 *walk = plan.walk;
  const int wide = (rows + 3) & ~3;
  int *lead = reinterpret_cast<int *>(words), *users = lead + wide, *tile0 = users + wide, *list0 = tile0 + wide, *base0 = list0 + wide, *chain = base0 + wide;
  __shared__ int sums[3][THREADS / 64];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, per = (rows + THREADS - 1) / THREADS;
  const int r0 = tid * per, r1 = min(r0 + per, rows);
  for (int r = r0; r < r1; ++r) {
    chain[r] = 1;
    plan.row[r] = PtRow{0, 0, {0, 0, 0}, {0, 0, 0}};
  }
  if (tid < wide - rows) lead[rows + tid] = -1;
  int tiles = 0, listed = 0, columns = 0;
#pragma unroll 1
  for (int l = 0; l < PT_LEVELS; ++l) {
    __syncthreads();
    bool some = false;
    for (int r = r0; r < r1; ++r) {
      const int4 w = walk[r * PT_LEVELS + l];
      int of = -1;
      if (chain[r] && w.w && (unsigned)w.z < (unsigned)rows) {
        const int4 o = walk[w.z * PT_LEVELS + l];
        if (chain[w.z] && o.w && o.z == w.z && o.x == w.x && o.y == w.y) of = w.z;
      }
      lead[r] = of;
      users[r] = 0;
      some |= of >= 0;
    }
    if (!__syncthreads_or(some)) break;
    for (int r = r0; r < r1; ++r)
      if (lead[r] >= 0) atomicAdd(&users[lead[r]], 1);
    __syncthreads();
    for (int r = r0; r < r1; ++r) {
      const int of = lead[r];
      if (of >= 0 && users[of] < 2) lead[r] = -1;                  // its owner alone: nobody else looks at this word before the barrier but as a rank's
    }
    __syncthreads();
    int mine[3] = {0, 0, 0};
    for (int r = r0; r < r1; ++r) {
      chain[r] = lead[r] >= 0;
      if (lead[r] == r) {
        tile0[r] = mine[0]; list0[r] = mine[1]; base0[r] = mine[2];
        mine[0] += (users[r] * group + TC - 1) / TC;
        mine[1] += users[r];
        mine[2] += users[r] * group;
      }
    }
    int before[3], total[3];
#pragma unroll
    for (int k = 0; k < 3; ++k) {
      before[k] = wave_scan(mine[k]);
      if (lane == 63) sums[k][wave] = before[k];
      before[k] -= mine[k];
    }
    __syncthreads();
#pragma unroll
    for (int k = 0; k < 3; ++k) {
      total[k] = 0;
      for (int w = 0; w < THREADS / 64; ++w) { before[k] += w < wave ? sums[k][w] : 0; total[k] += sums[k][w]; }
    }
    for (int r = r0; r < r1; ++r)
      if (lead[r] == r) { tile0[r] += tiles + before[0]; list0[r] += listed + before[1]; base0[r] += columns + before[2]; }
    __syncthreads();
    for (int r = r0; r < r1; ++r) {
      const int of = lead[r];
      if (of < 0) continue;
      int rank = 0;
#pragma unroll 2
      for (int i = 0; i < r; i += 4) {
        const int4 x = *reinterpret_cast<const int4 *>(lead + i);
        rank += (x.x == of ? 1 : 0) + (x.y == of && i + 1 < r ? 1 : 0) + (x.z == of && i + 2 < r ? 1 : 0) + (x.w == of && i + 3 < r ? 1 : 0);
      }
      const int4 w = walk[r * PT_LEVELS + l];
      plan.list[list0[of] + rank] = r;
      plan.row[r].from = w.y;
      plan.row[r].levels = l + 1;
      plan.row[r].tile[l] = tile0[of];
      plan.row[r].column[l] = rank * group;
      if (of == r) {
        const int all = users[r] * group;
        const KvSeq of_r = kv_seq(kv, seqs, r);
        for (int f = 0, t = tile0[r]; f < all; f += TC, ++t)
          plan.tile[t] = PtTile{list0[r], of_r.row, f, min(TC, all - f), w.x, w.y, base0[r] + f, of_r.len - 1};
      }
    }
    tiles += total[0]; listed += total[1]; columns += total[2];
  }
  if (tid == 0) {
    PtHead h{};
    h.rows = rows; h.group = group; h.columns = TC; h.window = window; h.sinks = sinks; h.n_pages = kv.n_pages; h.max_pages = kv.max_pages; h.page = kv.page;
    h.tiles = tiles; h.tile_columns = columns; h.n_seqs = kv.n_seqs;
    *plan.head = h;
  }
}

static_assert((int64_t)KV_MAXSEQ * 256 * SH_THREADS <= INT32_MAX, "words of the tables where this is chosen");
static bool sh_near(const parse_kv *kv, int rows) {
  return rows <= SH_NEAR_ROWS && (int64_t)rows * ((kv->max_pages + SH_THREADS - 1) / SH_THREADS) <= 256;
}

// ---- the call
// Entries of a call at most; a kv head's columns of parts; 0 where the call is refused
struct AsSize {
  int64_t tiles, entries, columns;
  size_t bytes;
};
static bool as_size(const parse_kv *kv, int n_q, int rows, AsSize &z) {
  if (n_q <= 0 || n_q % kv->n_kv != 0 || n_q > 65536 || rows <= 0 || rows > KV_MAXSEQ || (int64_t)rows * n_q > INT32_MAX) return false;
  const int group = n_q / kv->n_kv, TC = pt_columns(kv->d, kv->dtype);
  z.tiles = pt_most_tiles(rows, group, TC);
  z.entries = z.tiles + (int64_t)rows * ((group + TC - 1) / TC);
  z.columns = (int64_t)pt_shares(kv) * TC + (int64_t)(PT_LEVELS + 1) * rows * group;
  z.bytes = pt_deal_bytes(z.entries) + round_up((size_t)z.columns * kv->n_kv * (kv->d + 4) * 4, 256);
  // the steps of all entries are added up in an int
  if (z.entries * (((int64_t)kv->max_pages * kv->page + PT_STEP - 1) / PT_STEP) > INT32_MAX - 65536) return false;
  return z.entries <= (kv->dtype == PARSE_F32 && kv->d > 160 ? PT_MAXENTRIES_WIDE : PT_MAXENTRIES);
}

}  // namespace parse

extern "C" {

using namespace parse;

size_t parse_shared_plan_bytes(const parse_kv *kv, int32_t n_q, int32_t rows) {
  AsSize z;
  if (check_kv(kv, false) != PARSE_OK || !as_size(kv, n_q, rows, z)) return 0;
  return pt_plan(kv, rows, n_q / kv->n_kv, nullptr).bytes;
}

int parse_shared_plan(const parse_kv *kv, int32_t n_q, int32_t rows, const int32_t *seqs, int32_t window, int32_t sinks, void *plan, size_t plan_bytes,
                      parse_stream stream) {
  const int st = check_kv(kv, false);
  if (st != PARSE_OK) return st;
  if (n_q <= 0 || rows <= 0 || window < 0 || sinks < 0) return PARSE_EINVAL;
  AsSize z;
  if (!as_size(kv, n_q, rows, z) || (!seqs && rows > kv->n_seqs)) return PARSE_ESHAPE;
  if (!aligned4(seqs)) return PARSE_EALIGN;
  const int group = n_q / kv->n_kv;
  if (!plan || plan_bytes < pt_plan(kv, rows, group, nullptr).bytes) return PARSE_EWORKSPACE;
  if (!aligned16(plan)) return PARSE_EALIGN;
  const PtPlan p = pt_plan(kv, rows, group, plan);
  hipStream_t s = (hipStream_t)stream;
  const size_t lds = (size_t)((rows + 3) & ~3) * 6 * 4;
  const int TC = pt_columns(kv->d, kv->dtype);
  const dim3 grid((uint32_t)std::min<int64_t>((kv->max_pages + SH_THREADS - 1) / SH_THREADS, std::max(1, 4096 / rows)), rows);
  if (sh_near(kv, rows)) {
    shared_walk<true><<<dim3(rows), SH_THREADS, 0, s>>>(*kv, seqs, rows, window, sinks, p);
  } else {
    shared_count<false><<<grid, SH_THREADS, 0, s>>>(*kv, seqs, window, sinks, p);
    PARSE_LAUNCH_CHECK();
    shared_count<true><<<grid, SH_THREADS, 0, s>>>(*kv, seqs, window, sinks, p);
    PARSE_LAUNCH_CHECK();
    shared_walk<false><<<dim3((rows + SH_THREADS / 64 - 1) / (SH_THREADS / 64)), SH_THREADS, 0, s>>>(*kv, seqs, rows, window, sinks, p);
  }
  PARSE_LAUNCH_CHECK();
  if (rows <= SH_THREADS) {
    shared_tiles<SH_THREADS><<<dim3(1), SH_THREADS, lds, s>>>(*kv, seqs, rows, group, TC, window, sinks, p);
  } else {
    PARSE_ALLOW_LDS(shared_tiles<SH_ONE>, 3 * SH_ONE / 64 * 4 + LDS_OF_VOTES, lds);
    shared_tiles<SH_ONE><<<dim3(1), SH_ONE, lds, s>>>(*kv, seqs, rows, group, TC, window, sinks, p);
  }
  PARSE_LAUNCH_CHECK();
  return PARSE_OK;
}

size_t parse_attend_shared_workspace_bytes(const parse_kv *kv, int32_t n_q, int32_t rows) {
  AsSize z;
  return check_kv(kv, false) == PARSE_OK && as_size(kv, n_q, rows, z) ? z.bytes : 0;
}

int parse_attend_shared(const parse_kv *kv, int32_t layer, const void *q, int64_t q_stride, int32_t n_q, int32_t rows, const int32_t *seqs, const void *plan,
                        size_t plan_bytes, float scale, int32_t window, int32_t sinks, void *out, int64_t out_stride, float *lse, void *workspace, size_t workspace_bytes,
                        parse_stream stream) {
  const int st = check_attend(kv, layer, q, q_stride, n_q, rows, nullptr, seqs, scale, window, sinks, out, out_stride, lse);
  if (st != PARSE_OK) return st;
  if (!plan) return PARSE_EINVAL;
  AsSize z;
  if (!as_size(kv, n_q, rows, z) || (!seqs && rows > kv->n_seqs)) return PARSE_ESHAPE;
  if (!workspace || workspace_bytes < z.bytes || plan_bytes < pt_plan(kv, rows, n_q / kv->n_kv, nullptr).bytes) return PARSE_EWORKSPACE;
  if (!aligned16(workspace) || !aligned16(plan)) return PARSE_EALIGN;
  const size_t at = (size_t)layer * kv->n_pages * kv->n_kv * kv->page * kv->d * elem_size(kv->dtype);
  const int TC = pt_columns(kv->d, kv->dtype);
  PtArgs a{};
  a.kv = *kv;
  a.K = (const char *)kv->K + at; a.V = (const char *)kv->V + at;
  a.q = q; a.out = out; a.lse = lse; a.seqs = seqs;
  a.q_stride = q_stride; a.out_stride = out_stride;
  a.n_q = n_q; a.group = n_q / kv->n_kv; a.rows = rows; a.window = window; a.sinks = sinks;
  a.shares = pt_shares(kv);
  a.per_row = (a.group + TC - 1) / TC;
  at_scale(scale, a.scale, a.lag, a.q_sign);
  a.plan = pt_plan(kv, rows, a.group, plan);
  a.most_tiles = (int)z.tiles;
  a.deal = (int32_t *)workspace;
  a.part = (float *)((char *)workspace + pt_deal_bytes(z.entries));
  return kv->dtype == PARSE_BF16 ? pt_width<uint16_t, false>(a, z.entries, (hipStream_t)stream) : pt_width<float, false>(a, z.entries, (hipStream_t)stream);
}

}  // extern "C"
