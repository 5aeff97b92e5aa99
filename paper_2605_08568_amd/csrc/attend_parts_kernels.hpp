// The kernels of attend_parts.hpp; a source file for each type of cache and kind of entry.
#pragma once
#include <algorithm>
#include <type_traits>

#include "attend_parts.hpp"

namespace parse {

// LDS of a workgroup but the entries' sums: the ring, or the wavefronts' sums
template <class T, int DT> constexpr int pt_lds_own() {
  const int ring = pt_stages<T, DT>() * pt_step_bytes<T, DT>(), sums = (PT_WAVES * 16 * (DT * 32 + 4) + 2 * PT_WAVES * 16) * 4;
  return ring > sums ? ring : sums;
}

// Steps of a share where there are tiles, at least.  8 / 12 / 16, us: 32 samples of 8192 tokens 39.5 / 42.4 / 46.9 with the join
constexpr int PT_WIDE_STEPS = 8;

// Steps of an equal share, in twos.  By fours / twos / ones, us: 36 rows behind a common text 30.5 / 28.4 / 29.6, 64 samples of 8192 tokens 39.2 / 36.9 / 35.6 (join 9.2 / 9.8 / 10.0), 128 samples
// 55.4 / 53.4 / 53.5, 96 rows of a window 36.0 / 38.1 / 38.1 (16 steps or 14); lists the same
__host__ __device__ constexpr int pt_share(int64_t total, int shares, int least) {
  const int even = (int)((total + shares - 1) / shares + 1) / 2 * 2;
  return even > least ? even : least;
}

// Entry x is share x, whole, where no entry has more steps than an equal share would and these: it costs what the longest entry is longer, and saves parts and, where rows
// share nothing, the join.  4 / 12 / 24, us with the join: 32 caches of 100 to 356 tokens 19.3 / 17.7 / 17.7, 32 lists of 32 pages of 32 30.9 / 31.1 / 36.0
constexpr int PT_SLACK = 12;

// A step of 32 tokens: s = K q (operand A = K, token rows; operand B = q, a column of the entry), weights 2^(scale s - base), o += V^T p.  K's rows are taken in the order in
// which the scores come back as operand B: rows 4 q + 0..3 of the two instructions of a step are tokens 8 q + 0..3 and 8 q + 4..7, so that a lane's eight weights are
// the eight tokens whose V it has loaded.  bf16: a weight is multiplied as two bf16 numbers, as in the decode attention.
//   narrow entries, up to sixteen columns: operands go straight from the pages into registers, a step ahead of the one that is worked on where two fit; the four wavefronts
//   take turns and their sums meet in LDS, or, where rows are many and short, a wavefront has a row alone
//   wide ones: a wavefront has up to NW blocks of sixteen columns; the steps go through a ring in LDS, filled by loads that write LDS, and are read by all four (the same columns
//     out of registers, every wavefront its own loads: 123 us where this takes 28)
// Bound, bf16 of 128 columns: small calls by latency (lengths and the plan, the entry's columns and pages, first loads, the meeting: four trips, 8 to 10 us); wide entries by the
// vector unit and by how few steps a share has: 32 samples of one text of 8192 tokens, 8 heads, 32/8, 27.5 us, 1.2 us a step of 128 columns; narrow entries by reads: 32 caches of 2049
// tokens 50 us, 5.4 TB/s.
template <class T, int DT, bool NT, bool LISTED>
__global__ __launch_bounds__(PT_THREADS, (pt_at_once<T, DT>())) void attend_parts(PtArgs a) {
  constexpr int D = DT * 32, KB = D / 32, VB = D / 16, NW = pt_blocks<T, DT>(), TC = 64 * NW, RD = D + 4, ST = pt_stages<T, DT>();
  constexpr int CHUNK = 16 * D * (int)sizeof(T), STAGE = 4 * CHUNK, LOADS = CHUNK / 1024;         // K and V of sixteen tokens each stand in one piece
  typedef typename Op<T>::frag frag;
  extern __shared__ char smem[];
  float *red = reinterpret_cast<float *>(smem);                    // [wave][16][RD], [wave][16] twice; or the ring
  float *red_m = red + PT_WAVES * 16 * RD, *red_l = red_m + PT_WAVES * 16;
  int *wave_sums = reinterpret_cast<int *>(smem + pt_lds_own<T, DT>()), *pre = wave_sums + 2 * PT_WAVES;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int n = lane & 15, quad = lane >> 4;
  const int share = blockIdx.x, kvh = blockIdx.y;
  int tiles = 0, tile_columns = 0, total;
  bool fits = false;
  // Steps of a list are what it has room for: which of its words are columns is not known here.  32 rows of 100 tokens, pages of 64: 7.7 us for lists of 2, 40.7 for lists of 64
  const int list_steps = LISTED ? (int)(((int64_t)a.top * a.kv.page + PT_STEP - 1) / PT_STEP) : 0;
  auto tile_span = [&](const PtTile &t) { return pt_span(t.pos, t.from, t.to, a.window, a.sinks); };
  auto own_span = [&](int from, const KvSeq &s) { return pt_span(s.len - 1, min(from, s.len), s.len, a.window, a.sinks); };
  auto from_of = [&](int row) { return fits ? a.plan.row[row].from : 0; };
  if constexpr (LISTED) {
    total = list_steps * a.rows * a.per_row;
  } else {
    // a thread's first tile and row are asked for before it is known how many there are, and whether the plan is this call's
    const PtTile t = a.plan.tile[min(tid, a.most_tiles - 1)];
    const int r = min(tid, a.rows - 1), from = a.plan.row[r].from;
    const KvSeq seq = kv_seq(a.kv, a.seqs, r);
    fits = pt_fits(a, TC);
    if (fits) { tiles = a.plan.head->tiles; tile_columns = a.plan.head->tile_columns; }
    if (tiles <= PT_THREADS && a.rows <= PT_THREADS) {
      const int of_tile = tid < tiles ? tile_span(t).count : 0, of_row = tid < a.rows ? own_span(fits ? from : 0, seq).count : 0;
      const int up_tile = wave_scan(of_tile), up_row = wave_scan(of_row * a.per_row);
      if (lane == 63) { wave_sums[wave] = up_tile; wave_sums[PT_WAVES + wave] = up_row; }
      __syncthreads();
      int before = up_tile - of_tile, behind = up_row - of_row * a.per_row;
      total = 0;
#pragma unroll
      for (int w = 0; w < PT_WAVES; ++w) {
        before += w < wave ? wave_sums[w] : 0;
        behind += wave_sums[w] + (w < wave ? wave_sums[PT_WAVES + w] : 0);
        total += wave_sums[w] + wave_sums[PT_WAVES + w];
      }
      if (tid < tiles) pre[tid] = before;
      if (tid < a.rows)
        for (int z = 0; z < a.per_row; ++z) pre[tiles + tid * a.per_row + z] = behind + z * of_row;
      if (tid == 0) pre[tiles + a.rows * a.per_row] = total;
      __syncthreads();
    } else {
      kv_prefix<PT_THREADS>(tiles + a.rows * a.per_row, pre, wave_sums, [&](int e) {
        if (e < tiles) return tile_span(a.plan.tile[e]).count;
        const int row = (e - tiles) / a.per_row;
        return own_span(from_of(row), kv_seq(a.kv, a.seqs, row)).count;
      });
      total = pre[tiles + a.rows * a.per_row];
    }
  }
  const int entries = tiles + a.rows * a.per_row;
  auto before_of = [&](int e) { return LISTED ? e * list_steps : pre[e]; };
  // Tiles are cut in shares of PT_WIDE_STEPS at least: a part of them is as many bytes as four steps, written and read again
  const int per = pt_share(total, a.shares, tiles > 0 ? PT_WIDE_STEPS : PT_WAVES);
  bool by_rows = entries <= a.shares;
  if (by_rows) {
    bool longer = false;
    for (int e = tid; e < entries; e += PT_THREADS) longer |= before_of(e + 1) - before_of(e) > per + PT_SLACK;
    const bool some = __any(longer);                               // with words of its own: __syncthreads_or has 256 bytes of LDS beside those that were asked for
    if (lane == 0) wave_sums[wave] = some;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < PT_WAVES; ++w) by_rows &= wave_sums[w] == 0;
  }
  if (share == 0 && kvh == 0) {                                    // for the kernel that joins
    if (tid == 0) *reinterpret_cast<int4 *>(a.deal) = int4{per, by_rows, entries, tile_columns};
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
  int e0, e1;                                                      // first and last entry of the share
  if constexpr (LISTED) {
    e0 = (int)begin / list_steps;
    e1 = (end - 1) / list_steps;
  } else if (entries <= 512) {
    e0 = e1 = -1;
    for (int e = 0; e < entries; e += 64) {
      const int v = pre[min(e + lane, entries)];
      e0 += __popcll(__ballot(e + lane < entries && v <= (int)begin));
      e1 += __popcll(__ballot(e + lane < entries && v < end));
    }
  } else {
    e0 = kv_find(pre, entries, (int)begin);
    e1 = kv_find(pre, entries, end - 1);
  }
  e0 = __builtin_amdgcn_readfirstlane(e0);
  e1 = __builtin_amdgcn_readfirstlane(e1);
  float *parts = a.part + (int64_t)kvh * ((int64_t)a.shares * TC + (LISTED ? 0 : (int64_t)PT_LEVELS * a.rows * a.group) + (int64_t)a.rows * a.group) * RD;
  // Rows of sixteen columns at most that a wavefront has alone: from `alone` on
  const int rows0 = max(e0, tiles);
  const bool many = a.group <= 16 && e1 - rows0 >= PT_WAVES - 1 && end - max((int)begin, before_of(rows0)) <= 12 * (e1 - rows0);
  const int alone = many ? rows0 : e1 + 1;
  int mine = alone + wave, common = e0;
  for (;;) {
    const bool by_all = common < alone;
    if (!by_all && mine > e1) break;
    const int e = __builtin_amdgcn_readfirstlane(by_all ? common : mine);
    if (by_all) ++common; else mine += PT_WAVES;
    const int before = __builtin_amdgcn_readfirstlane(before_of(e)), count = __builtin_amdgcn_readfirstlane(before_of(e + 1)) - before;
    if (count == 0) continue;
    // ---- the entry
    PtTile t{};
    int row = 0, z = 0, seq, columns, base, pos_of = -1;
    bool direct = LISTED;
    int passed = 0;                                                // steps that were in sight when the plan was made and are no more
    PtSpan span{};
    const bool tile = !LISTED && e < tiles;
    if (tile) {
      t = a.plan.tile[e];
      seq = t.seq; columns = t.columns; base = t.base;
      span = tile_span(t);
      if (a.window > 0) {                                          // pages behind the window may have been given up since, by some of the rows
        const PtShortest s = pt_shortest(a, t);
        if (s.pos >= 0) seq = s.row;
        passed = s.pos < 0 ? count : span.sink_tiles + max(pt_span(max(s.pos, t.pos), t.from, t.to, a.window, a.sinks).a - span.a, 0);
      }
    } else {
      row = (e - tiles) / a.per_row; z = (e - tiles) - row * a.per_row;
      const KvSeq s = kv_seq(a.kv, a.seqs, row);
      seq = s.row; pos_of = s.len - 1;
      columns = min(a.group - z * TC, TC);
      base = tile_columns + row * a.group + z * TC;
      if constexpr (!LISTED) {
        span = own_span(from_of(row), s);
        direct = !fits || a.plan.row[row].levels == 0;
      }
    }
    seq = __builtin_amdgcn_readfirstlane(seq);
    columns = __builtin_amdgcn_readfirstlane(columns);
    base = __builtin_amdgcn_readfirstlane(base);
    span.f = __builtin_amdgcn_readfirstlane(span.f);
    span.sink_tiles = __builtin_amdgcn_readfirstlane(span.sink_tiles);
    span.a = __builtin_amdgcn_readfirstlane(span.a);
    int first = max((int)begin - before, 0);
    const int last = min(end - before, count);
    const bool all = direct && first == 0 && last == count;
    if (tile && first >= span.sink_tiles) first = __builtin_amdgcn_readfirstlane(min(max(first, passed), last));
    const bool wide = columns > 16;
    const int32_t *table = a.kv.table + (int64_t)seq * a.kv.max_pages;
    const int32_t *list = LISTED ? a.pages + ((int64_t)row * a.kv.n_kv + kvh) * a.top : nullptr;
    float *part = parts + ((int64_t)share * TC + base) * RD;
    // NB: blocks of sixteen columns that this wavefront has, number wave + 4 b of a wide entry, the only one of a narrow one
    auto entry = [&](auto is_wide, auto of) {
      constexpr bool WIDE = decltype(is_wide)::value;
      constexpr int NB = decltype(of)::value, NA = NB > 0 ? NB : 1;
      auto column = [&](int b) { return WIDE ? 16 * (wave + PT_WAVES * b) + n : n; };
      frag qf[NA][KB];
      int pos[NA], lo[NA], in_table[NA], least = 0x7fffffff, most = 0;
      // q and what the columns see.  Three trips to memory one behind another: the rows go with the pages' numbers, q and the lengths with the first steps.
      int r[NA], h[NA];
      auto ask_rows = [&]() {
#pragma unroll
        for (int b = 0; b < NA; ++b) {
          const int c = min(column(b), columns - 1);
          r[b] = row; h[b] = z * TC + c;
          if (tile) {
            const int f = t.first + c, m = f / a.group;
            r[b] = a.plan.list[t.list + m];
            h[b] = f - m * a.group;
          }
        }
      };
      auto ask = [&]() {
#pragma unroll
        for (int b = 0; b < NA; ++b) {
          const T *q = reinterpret_cast<const T *>(a.q) + (int64_t)r[b] * a.q_stride + (int64_t)(kvh * a.group + h[b]) * D;
          pos[b] = pos_of;
          in_table[b] = seq;
          if (tile) {
            const KvSeq s = kv_seq(a.kv, a.seqs, r[b]);
            pos[b] = s.len - 1;
            in_table[b] = s.row;
          }
#pragma unroll
          for (int k = 0; k < KB; ++k) qf[b][k] = Op<T>::load(q + 32 * k + 8 * quad);
        }
      };
      auto asked = [&]() {
#pragma unroll
        for (int b = 0; b < NA; ++b) {
          lo[b] = LISTED ? 0 : kv_window_begin(pos[b], a.window);
          if (!LISTED && tile && a.window > 0) {                   // the table that is read is another row's: what this one has given up of it
            const int edge = pt_edge(a.kv, lo[b]);
            if (edge >= 0 && !pt_holds(a.kv, in_table[b], edge)) ++lo[b];
          }
          least = min(least, pos[b]);
          most = max(most, lo[b]);
        }
#pragma unroll
        for (int o = 8; o > 0; o >>= 1) { least = min(least, __shfl_xor(least, o, 64)); most = max(most, __shfl_xor(most, o, 64)); }
        least = __builtin_amdgcn_readfirstlane(least);
        most = __builtin_amdgcn_readfirstlane(most);
#pragma unroll
        for (int b = 0; b < NA; ++b)
#pragma unroll
          for (int k = 0; k < KB; ++k) qf[b][k] = Op<T>::sign(qf[b][k], a.q_sign);
      };
      float m[NA], l[NA];
      f32x4 o[NA][VB];
      auto clear = [&]() {
#pragma unroll
        for (int b = 0; b < NA; ++b) {
          m[b] = -INFINITY; l[b] = 0.f;
#pragma unroll
          for (int v = 0; v < VB; ++v) o[b][v] = f32x4{0.f, 0.f, 0.f, 0.f};
        }
      };
      clear();
      // Half (sixteen tokens) of a step: its page and first token; a page outside [0, n_pages): none
      auto place = [&](int u, int half, int &id, int &at) {
        if constexpr (LISTED) {
          const int block = 2 * u + half, i = block >> (page_bits - 4);
          const int c = i < a.top ? list[i] : -1;
          const bool ok = (unsigned)c < (unsigned)a.kv.max_pages;
          id = ok ? table[c] : -1;
          at = (ok ? c : 0) * a.kv.page + (block & ((a.kv.page >> 4) - 1)) * 16;
        } else {
          at = span.at(u) * PT_STEP + 16 * half;
          id = table[min(at >> page_bits, a.kv.max_pages - 1)];
        }
      };
      auto page_there = [&](int id) { return (unsigned)id < (unsigned)a.kv.n_pages; };
      struct Where {                                                 // of a step
        int ta, tb;
        bool there_a, there_b;
      };
      // which of the lane's eight tokens a row at position i sees
      auto seen = [&](const Where &x, int i, int from) -> uint32_t {
        const bool there = quad < 2 ? x.there_a : x.there_b;
        const int j0 = (quad < 2 ? x.ta : x.tb) + 8 * (quad & 1);
        return there ? kv_sees8(i, from, LISTED ? 0 : a.sinks, j0) : 0u;
      };
      auto whole_of = [&](const Where &x) {
        return x.there_a && x.there_b && x.ta + 15 <= least && x.tb + 15 <= least && (x.ta >= most || x.ta + PT_STEP <= a.sinks);
      };
      // weights of block b from the scores, the running maximum moved where it has to grow
      auto weigh = [&](int b, f32x4 s0, f32x4 s1, bool whole, uint32_t keep, float *p) {
        float s[8];
#pragma unroll
        for (int e = 0; e < 4; ++e) { s[e] = s0[e]; s[4 + e] = s1[e]; }
        if (!whole) {
#pragma unroll
          for (int e = 0; e < 8; ++e) s[e] = keep >> e & 1 ? s[e] : -INFINITY;
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
#pragma unroll
        for (int e = 0; e < 8; ++e) { p[e] = at_exp2(fmaf(s[e], a.scale, -off)); l[b] += p[e]; }
      };
      auto any_seen = [&](const Where &x, uint32_t *keep) {          // what no column of the wavefront sees: nothing of V to multiply with
        uint32_t any = 0;
#pragma unroll
        for (int b = 0; b < NA; ++b) { keep[b] = seen(x, pos[b], lo[b]); any |= keep[b]; }
#pragma unroll
        for (int s = 8; s > 0; s >>= 1) any |= __shfl_xor(any, s, 64);
        return any;
      };
      // ---- from pages into registers: steps start, start + turn, ...
      struct Step {
        frag k0[KB], k1[KB], v[VB];
        Where at;
      };
      int start = first, turn = 1, steps = max(last - first, 0);
      if (!WIDE && by_all) { start = first + wave; turn = PT_WAVES; steps = last > start ? (last - start + PT_WAVES - 1) / PT_WAVES : 0; }
      int id_a = -1, id_b = -1, at_a = 0, at_b = 0;                  // of the next 64 steps, a lane each
      auto load = [&](Step &x, int j) {
        if ((j & 63) == 0) {
          const int u = min(start + (j + lane) * turn, last - 1);
          place(u, 0, id_a, at_a);
          place(u, 1, id_b, at_b);
        }
        const int ida = __builtin_amdgcn_readlane(id_a, j & 63), idb = __builtin_amdgcn_readlane(id_b, j & 63);
        x.at.ta = __builtin_amdgcn_readlane(at_a, j & 63);
        x.at.tb = __builtin_amdgcn_readlane(at_b, j & 63);
        x.at.there_a = page_there(ida);
        x.at.there_b = page_there(idb);
        const int64_t pa = (int64_t)(x.at.there_a ? ida : 0) * page_elems + head0 + (int64_t)(x.at.ta & (a.kv.page - 1)) * D;
        const int64_t pb = (int64_t)(x.at.there_b ? idb : 0) * page_elems + head0 + (int64_t)(x.at.tb & (a.kv.page - 1)) * D;
        auto get = [](const T *p) { return NT ? Op<T>::load_nt(p) : Op<T>::load(p); };
        const T *kp = reinterpret_cast<const T *>(a.K) + (n < 8 ? pa : pb) + k_in;
        const T *vp = reinterpret_cast<const T *>(a.V) + (quad < 2 ? pa : pb) + v_in;
#pragma unroll
        for (int k = 0; k < KB; ++k) { x.k0[k] = get(kp + k * 512); x.k1[k] = get(kp + k * 512 + 32); }
#pragma unroll
        for (int v = 0; v < VB; ++v) x.v[v] = get(vp + v * 128);
      };
      if constexpr (!WIDE) {
        auto work = [&](Step &x) {
          f32x4 s0 = {0.f, 0.f, 0.f, 0.f}, s1 = s0;
#pragma unroll
          for (int k = 0; k < KB; ++k) { s0 = Op<T>::mma16(x.k0[k], qf[0][k], s0); s1 = Op<T>::mma16(x.k1[k], qf[0][k], s1); }
          const bool whole = whole_of(x.at);
          uint32_t keep[NA] = {};
          if (!whole) {
            const uint32_t any = any_seen(x.at, keep);
#pragma unroll
            for (int v = 0; v < VB; ++v) x.v[v] = Op<T>::only(x.v[v], any);
          }
          float p[8];
          weigh(0, s0, s1, whole, keep[0], p);
          const frag pf = Op<T>::pack(p);
#pragma unroll
          for (int v = 0; v < VB; ++v) o[0][v] = Op<T>::mma16(x.v[v], pf, o[0][v]);
          if constexpr (sizeof(T) == 2) {
            const frag rest = Op<T>::pack_rest(p, pf);
#pragma unroll
            for (int v = 0; v < VB; ++v) o[0][v] = Op<T>::mma16(x.v[v], rest, o[0][v]);
          }
        };
        Step even;
        if constexpr (DT * sizeof(T) <= 8) {                         // two steps fit the registers
          Step odd;
          ask_rows();
          if (steps > 0) load(even, 0);
          ask();
          asked();
          for (int j = 0; j < steps; j += 2) {
            if (j + 1 < steps) load(odd, j + 1);
            work(even);
            if (j + 1 < steps) {
              if (j + 2 < steps) load(even, j + 2);
              work(odd);
            }
          }
        } else {
          ask_rows();
          ask();
          asked();
          for (int j = 0; j < steps; ++j) {
            load(even, j);
            work(even);
          }
        }
      } else if (steps > 0) {
        // ---- through LDS.  Wavefront w stages K (0, 1) or V (2, 3) of a step's first or second sixteen tokens.  In the second half's K tokens t and t ^ 4 change places, so that
        // the sixteen rows of an operand (of a pair of quads four tokens of each half) stand in different banks.
        const char *const pool = (const char *)(wave < 2 ? a.K : a.V) + head0 * (int64_t)sizeof(T);
        const int from_lane = wave == 1 ? (sizeof(T) == 2 ? lane ^ 4 : lane ^ 8) : lane;
        uint32_t place_lo = 0, place_hi = 0;                         // of the next 64 steps to stage, a lane each: where this wavefront's sixteen tokens stand
        int there_ab = 0;                                            // of the next 64 steps to work on: there_a, there_b
        int staged = 0;
        auto stage = [&]() {
          if ((staged & 63) == 0) {
            int id, at;
            place(min(first + staged + lane, last - 1), wave & 1, id, at);
            const int64_t p = ((int64_t)(page_there(id) ? id : 0) * page_elems + (int64_t)(at & (a.kv.page - 1)) * D) * (int64_t)sizeof(T);
            place_lo = (uint32_t)p;
            place_hi = (uint32_t)(p >> 32);
          }
          const char *src = pool + ((uint64_t)(uint32_t)__builtin_amdgcn_readlane(place_hi, staged & 63) << 32 | (uint32_t)__builtin_amdgcn_readlane(place_lo, staged & 63)) + from_lane * 16;
          char *dst = smem + (staged % ST) * STAGE + wave * CHUNK;
#pragma unroll
          for (int q = 0; q < LOADS; ++q) __builtin_amdgcn_global_load_lds(PARSE_GLB_PTR(src + q * 1024), PARSE_LDS_PTR(dst + q * 1024), 16, 0, 0);
          ++staged;
        };
        auto look = [&](int j) {
          const int u = min(first + j + lane, last - 1);
          place(u, 0, id_a, at_a);
          place(u, 1, id_b, at_b);
          there_ab = (page_there(id_a) ? 1 : 0) | (page_there(id_b) ? 2 : 0);
        };
        ask_rows();
        look(0);
        if (e > e0) __syncthreads();                                 // the sums of the entry before are read
#pragma unroll
        for (int j = 0; j < ST - 1; ++j)
          if (j < steps) stage();
        ask();
        asked();
        // where this lane's pieces stand: rows 0..7 of an operand in the first half, 8..15 in the second
        const int k_at = (n < 8 ? 0 : CHUNK) + (quad * 16 + (tok & 15)) * 8 * (int)sizeof(T), k_turn = n < 8 ? 0 : 4 * 8 * (int)sizeof(T);
        const int v_at = 2 * CHUNK + (quad >> 1) * CHUNK + v_in * (int)sizeof(T);
#pragma unroll 1
        for (int j = 0; j < steps; ++j) {
          wait_slices<ST - 2, LOADS>(steps - 1 - j);
          wg_barrier();                                              // this step has landed for everybody, the one before it is read by everybody
          if (staged < steps) stage();
          if constexpr (NB > 0) {
            const int flags = __builtin_amdgcn_readlane(there_ab, j & 63);
            const Where x{__builtin_amdgcn_readlane(at_a, j & 63), __builtin_amdgcn_readlane(at_b, j & 63), (flags & 1) != 0, (flags & 2) != 0};
            const char *buf = smem + (j % ST) * STAGE;
            f32x4 s0[NB], s1[NB];
#pragma unroll
            for (int b = 0; b < NB; ++b) s0[b] = s1[b] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int k = 0; k < KB; ++k) {
              const frag k0 = Op<T>::load(reinterpret_cast<const T *>(buf + (k_at ^ k_turn)) + k * 512);
              const frag k1 = Op<T>::load(reinterpret_cast<const T *>(buf + (k_at ^ k_turn ^ (4 * 8 * (int)sizeof(T)))) + k * 512);
#pragma unroll
              for (int b = 0; b < NB; ++b) { s0[b] = Op<T>::mma16(k0, qf[b][k], s0[b]); s1[b] = Op<T>::mma16(k1, qf[b][k], s1[b]); }
            }
            const bool whole = whole_of(x);
            uint32_t keep[NA] = {}, any = 0xffu;
            if (!whole) any = any_seen(x, keep);
            frag vf[VB];                                             // before the weights: a branch stands among those
#pragma unroll
            for (int v = 0; v < VB; ++v) vf[v] = Op<T>::load(reinterpret_cast<const T *>(buf + v_at) + v * 128);
            frag pf[NB], rest[NB];
#pragma unroll
            for (int b = 0; b < NB; ++b) {
              float p[8];
              weigh(b, s0[b], s1[b], whole, keep[b], p);
              pf[b] = Op<T>::pack(p);
              if constexpr (sizeof(T) == 2) rest[b] = Op<T>::pack_rest(p, pf[b]);
            }
#pragma unroll
            for (int v = 0; v < VB; ++v) {
              if (!whole) vf[v] = Op<T>::only(vf[v], any);
#pragma unroll
              for (int b = 0; b < NB; ++b) {
                o[b][v] = Op<T>::mma16(vf[v], pf[b], o[b][v]);
                if constexpr (sizeof(T) == 2) o[b][v] = Op<T>::mma16(vf[v], rest[b], o[b][v]);
              }
            }
          }
          if (((j + 1) & 63) == 0) look(j + 1);
        }
      }
      if constexpr (NB > 0) {
        // An infinity or NaN of V that some columns see and others do not makes NaN of a weight of zero, and so does what the rounding of a weight left.  Where
        // something that is not finite came out, once more, from the pages, column by column, each with what it sees of V.
        f32x4 sum = {0.f, 0.f, 0.f, 0.f};                            // NaN where one of them is not finite
#pragma unroll
        for (int b = 0; b < NA; ++b)
#pragma unroll
          for (int v = 0; v < VB; ++v)
#pragma unroll
            for (int i = 0; i < 4; ++i) sum[i] = fmaf(o[b][v][i], 0.f, sum[i]);
        if (__any((sum[0] + sum[1]) + (sum[2] + sum[3]) != 0.f)) {
          clear();
#pragma unroll 1
          for (int j = 0; j < steps; ++j) {
            Step x;
            load(x, j);
            const bool whole = whole_of(x.at);
#pragma unroll
            for (int b = 0; b < NA; ++b) {
              f32x4 s0 = {0.f, 0.f, 0.f, 0.f}, s1 = s0;
#pragma unroll
              for (int k = 0; k < KB; ++k) { s0 = Op<T>::mma16(x.k0[k], qf[b][k], s0); s1 = Op<T>::mma16(x.k1[k], qf[b][k], s1); }
              float p[8];
              weigh(b, s0, s1, whole, whole ? 0xffu : seen(x.at, pos[b], lo[b]), p);
              const frag pf = Op<T>::pack(p);
              frag rest = pf;
              if constexpr (sizeof(T) == 2) rest = Op<T>::pack_rest(p, pf);
#pragma unroll 1
              for (int c = 0; c < 16; ++c) {
                const uint32_t sees = whole ? 0xffu : seen(x.at, __builtin_amdgcn_readlane(pos[b], c), __builtin_amdgcn_readlane(lo[b], c));
#pragma unroll
                for (int v = 0; v < VB; ++v) {
                  const frag vc = Op<T>::only(x.v[v], sees);
                  const f32x4 add = Op<T>::mma16(vc, pf, f32x4{0.f, 0.f, 0.f, 0.f});
                  f32x4 more = {0.f, 0.f, 0.f, 0.f};
                  if constexpr (sizeof(T) == 2) more = Op<T>::mma16(vc, rest, more);
#pragma unroll
                  for (int i = 0; i < 4; ++i) o[b][v][i] += n == c ? add[i] + (fabsf(more[i]) < INFINITY ? more[i] : 0.f) : 0.f;
                }
              }
            }
          }
        }
      }
#pragma unroll
      for (int b = 0; b < NA; ++b) l[b] = lane_sum<32>(lane_sum<16>(l[b]));
      if (WIDE || !by_all) {                                         // a column's sums are one wavefront's
#pragma unroll
        for (int b = 0; b < NB; ++b) {
          const int c = column(b);
          if (c >= columns) continue;
          if (all) {
            const int head = kvh * a.group + z * TC + c;
            const float by = l[b] == 0.f ? 0.f : 1.f / l[b];
            T *out = reinterpret_cast<T *>(a.out) + (int64_t)row * a.out_stride + (int64_t)head * D + 4 * quad;
#pragma unroll
            for (int v = 0; v < VB; ++v) Op<T>::store4(out + 16 * v, o[b][v][0] * by, o[b][v][1] * by, o[b][v][2] * by, o[b][v][3] * by);
            if (a.lse && quad == 0) a.lse[(int64_t)row * a.n_q + head] = at_lse(m[b], a.scale, l[b]);
          } else {
            float *to = part + (int64_t)c * RD;
#pragma unroll
            for (int v = 0; v < VB; ++v) *reinterpret_cast<f32x4 *>(to + 16 * v + 4 * quad) = o[b][v];
            if (quad == 0) { to[D] = m[b]; to[D + 1] = l[b]; }
          }
        }
        return;
      }
      // ---- the wavefronts' sums meet
      if constexpr (!WIDE) {
        __syncthreads();
        if (quad == 0) { red_m[wave * 16 + n] = m[0]; red_l[wave * 16 + n] = l[0]; }
#pragma unroll
        for (int v = 0; v < VB; ++v) *reinterpret_cast<f32x4 *>(red + (wave * 16 + n) * RD + 16 * v + 4 * quad) = o[0][v];
        __syncthreads();
        for (int w = tid; w < columns * D; w += PT_THREADS) {
          const int c = w / D, i = w % D;
          float top = -INFINITY, ls = 0.f, os = 0.f;
#pragma unroll
          for (int x = 0; x < PT_WAVES; ++x) top = fmaxf(top, red_m[x * 16 + c]);
#pragma unroll
          for (int x = 0; x < PT_WAVES; ++x) {
            const float by = at_exp2((red_m[x * 16 + c] - finite_or_0(top)) * a.scale);
            ls += by * red_l[x * 16 + c];
            os += by * red[(x * 16 + c) * RD + i];
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
        __syncthreads();
      }
    };
    // blocks of a wide entry that are this wavefront's
    const int blocks = ((columns + 15) / 16 - wave + PT_WAVES - 1) / PT_WAVES;
    if (!wide) entry(std::false_type{}, std::integral_constant<int, 1>{});
    else if (blocks <= 0) entry(std::true_type{}, std::integral_constant<int, 0>{});
    else if (blocks == 1) entry(std::true_type{}, std::integral_constant<int, 1>{});
    else entry(std::true_type{}, std::integral_constant<int, NW>{});
  }
}

// The parts of one row's head; workgroup (head, row).  Four columns a lane, so many parts at once as the workgroup has lanes for, four of them on their way each; a group of lanes
// joins its parts one after another, then the groups are joined, both in a fixed order.  Bound: three dependent trips to memory, then the parts' reads: 3.8 us (a part or two a
// row) to 10 (96 rows of a window); 8 for 32 rows of a text that is cut in 32 parts.
template <class T, int DT, bool LISTED>
__global__ __launch_bounds__(PT_THREADS) void attend_parts_join(PtArgs a) {
  constexpr int D = DT * 32, RD = D + 4, TC = 64 * pt_blocks<T, DT>(), LANES = D / 4, GROUPS = PT_THREADS / LANES, N = 4;
  __shared__ float tops[GROUPS], totals[GROUPS], sums[GROUPS * D];
  const int tid = threadIdx.x, g = tid / LANES, i = tid % LANES * 4;
  const int row = blockIdx.y, head = blockIdx.x, kvh = head / a.group, h = head - kvh * a.group;
  const int4 deal = *reinterpret_cast<const int4 *>(a.deal);
  const int per = deal.x, tiles = deal.z - a.rows * a.per_row, tile_columns = deal.w;
  const bool by_rows = deal.y != 0;
  const int32_t *pre = a.deal + PT_DEAL;
  PtRow rec{};
  if constexpr (!LISTED) {
    const PtRow r = a.plan.row[row];
    if (tiles > 0) rec = r;
  }
  // up to PT_LEVELS tiles and the row's own entry: first share, parts, column of the first part
  int x0[PT_LEVELS + 1], count[PT_LEVELS + 1], col[PT_LEVELS + 1], parts = 0;
  const int levels = min(max(rec.levels, 0), PT_LEVELS);
#pragma unroll
  for (int s = 0; s <= PT_LEVELS; ++s) {
    x0[s] = count[s] = col[s] = 0;
    int e = -1, c = 0;
    if (s == PT_LEVELS) {
      e = tiles + row * a.per_row + h / TC;
      c = tile_columns + row * a.group + h;
    } else if (s < levels) {
      const int f = rec.column[s] + h;
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
    int at = x0[0], c = col[0];
    bool found = x < count[0];
#pragma unroll
    for (int k = 1; k <= PT_LEVELS; ++k) {
      x -= found ? 0 : count[k - 1];
      at = found ? at : x0[k];
      c = found ? c : col[k];
      found |= x < count[k];
    }
    return base + ((int64_t)(at + x) * TC + c) * RD;
  };
  float top = -INFINITY, total = 0.f;
  f32x4 y = {0.f, 0.f, 0.f, 0.f};
  if (g < GROUPS) {
    for (int first = g; first < parts; first += N * GROUPS) {
      f32x4 o[N];
      float m[N], l[N];
#pragma unroll
      for (int k = 0; k < N; ++k) {
        const int x = first + k * GROUPS;
        const float *p = part_of(min(x, parts - 1));
        o[k] = *reinterpret_cast<const f32x4 *>(p + i);
        m[k] = x < parts ? p[D] : -INFINITY;
        l[k] = x < parts ? p[D + 1] : 0.f;
      }
      float grown = top;
#pragma unroll
      for (int k = 0; k < N; ++k) grown = fmaxf(grown, m[k]);
      const float by = at_exp2((top - finite_or_0(grown)) * a.scale);
      total *= by;
      y *= by;
#pragma unroll
      for (int k = 0; k < N; ++k) {
        const float w = at_exp2((m[k] - finite_or_0(grown)) * a.scale);
        total = fmaf(w, l[k], total);
        if (first + k * GROUPS < parts) y += w * o[k];
      }
      top = grown;
    }
    if (i == 0) { tops[g] = top; totals[g] = total; }
    *reinterpret_cast<f32x4 *>(sums + g * D + i) = y;
  }
  __syncthreads();
  const int groups = min(GROUPS, parts);
  if (tid < LANES) {
    float most = -INFINITY, ls = 0.f;
    for (int x = 0; x < groups; ++x) most = fmaxf(most, tops[x]);
    f32x4 v = {0.f, 0.f, 0.f, 0.f};
    for (int x = 0; x < groups; ++x) {
      const float w = at_exp2((tops[x] - finite_or_0(most)) * a.scale);
      ls = fmaf(w, totals[x], ls);
      v += w * *reinterpret_cast<const f32x4 *>(sums + x * D + i);
    }
#pragma unroll
    for (int e = 0; e < 4; ++e) v[e] = ls == 0.f ? 0.f : v[e] / ls;
    Op<T>::store4(reinterpret_cast<T *>(a.out) + (int64_t)row * a.out_stride + (int64_t)head * D + i, v[0], v[1], v[2], v[3]);
    if (a.lse && i == 0) a.lse[(int64_t)row * a.n_q + head] = at_lse(most, a.scale, ls);
  }
}

// ---- host
// Loads of narrow entries past the caches where what they bring in does not stay there anyway, as in the decode attention: pools larger than the last-level cache, lists of
// more than a third of it.  Without / with such loads, us: 32 caches of 2049 tokens of 8 heads (268 MB) 57.7 / 50.0, lists of 134 MB 29.3 / 27.0; pools of 95 MB (three in turn) 30.8 /
// 32.3, lists of 17 MB 9.2 / 11.4.  Wide entries read a page once a tile, several tiles of a run the same one: through the caches.
template <class T, int DT, bool LISTED>
static int pt_launch(const PtArgs &a, int64_t entries, hipStream_t s) {
  constexpr int most = sizeof(T) == 4 && DT > 5 ? PT_MAXENTRIES_WIDE : PT_MAXENTRIES;
  static_assert(pt_lds_own<T, DT>() + (2 * PT_WAVES + most + 1) * 4 <= 160 * 1024, "a unit's LDS");
  const size_t lds = pt_lds_own<T, DT>() + (2 * PT_WAVES + (LISTED ? 0 : (size_t)entries + 1)) * 4, page = (size_t)a.kv.page * DT * 32 * sizeof(T) * 2;
  const bool nt = LISTED ? (size_t)a.rows * a.kv.n_kv * a.top * page > ((size_t)96 << 20) : (size_t)a.kv.n_layers * a.kv.n_pages * a.kv.n_kv * page > ((size_t)192 << 20);
  if (nt) {
    PARSE_ALLOW_LDS((attend_parts<T, DT, true, LISTED>), 0, lds);
    attend_parts<T, DT, true, LISTED><<<dim3(a.shares, a.kv.n_kv), PT_THREADS, lds, s>>>(a);
  } else {
    PARSE_ALLOW_LDS((attend_parts<T, DT, false, LISTED>), 0, lds);
    attend_parts<T, DT, false, LISTED><<<dim3(a.shares, a.kv.n_kv), PT_THREADS, lds, s>>>(a);
  }
  PARSE_LAUNCH_CHECK();
  if (LISTED && entries <= a.shares) {                             // the lists' steps are the host's to count: whether every entry is a share's, whole
    const int64_t steps = ((int64_t)a.top * a.kv.page + PT_STEP - 1) / PT_STEP, total = steps * entries;
    if (steps <= pt_share(total, a.shares, PT_WAVES) + PT_SLACK) return PARSE_OK;
  }
  attend_parts_join<T, DT, LISTED><<<dim3(a.n_q, a.rows), PT_THREADS, 0, s>>>(a);
  PARSE_LAUNCH_CHECK();
  return PARSE_OK;
}
template <class T, bool LISTED>
int pt_width(const PtArgs &a, int64_t entries, hipStream_t s) {
  switch (a.kv.d / 32) {
    case 1: return pt_launch<T, 1, LISTED>(a, entries, s);
    case 2: return pt_launch<T, 2, LISTED>(a, entries, s);
    case 3: return pt_launch<T, 3, LISTED>(a, entries, s);
    case 4: return pt_launch<T, 4, LISTED>(a, entries, s);
    case 5: return pt_launch<T, 5, LISTED>(a, entries, s);
    case 6: return pt_launch<T, 6, LISTED>(a, entries, s);
    case 7: return pt_launch<T, 7, LISTED>(a, entries, s);
    default: return pt_launch<T, 8, LISTED>(a, entries, s);
  }
}

}  // namespace parse
