// Causal attention of the new tokens of a batch of prompts over the paged cache (parse_attend_prefill).
#include <algorithm>

#include "attend.hpp"

namespace parse {

struct ApArgs {
  parse_kv kv;
  const void *K, *V;                                 // of the layer
  const void *q;
  void *out;
  float *lse;
  const int32_t *tok_offsets, *seqs;
  int64_t q_stride, out_stride;
  int n_q, group, rows, P, window, sinks;
  KvDivisor by_group;
  int splits;                                        // workgroups that share the tokens of a tile of rows
  float *part;                                       // [tile of rows and kv head][split] of AP_ROWS * (d + 2): sums, maxima, totals
  float scale, lag;                                  // |scale| times log2(e); AT_LAG in products of q and k
  uint32_t q_sign;
};

constexpr int AP_WAVES = 4, AP_ROWS = AP_WAVES * 32, AP_TILE = 32;
// Tiles of tokens that a split has at least: about 8 us of them.  13 rows over 8192 tokens of 8 heads, bf16, 8 / 16 tiles: 33 / 24 us; fp32 tiles take four times as
// long: over 4000 tokens of 16 heads, 8 / 16 tiles: 58 / 88 us
__device__ __host__ __forceinline__ int ap_least(int dtype) { return dtype == PARSE_BF16 ? 16 : 4; }
constexpr int AP_GROUPS = 512;                       // workgroups that fill the card, two a compute unit

// The tiles of tokens [first, last) that a workgroup has of the `count` that its rows see, and how many share them
struct ApShare {
  int first, last, parts;
};
__device__ __forceinline__ ApShare ap_share(int count, int splits, int split, int least) {
  const int each = max((count + splits - 1) / splits, least), parts = max((count + each - 1) / each, 1);
  return ApShare{min(split * each, count), min((split + 1) * each, count), parts};
}
// tiles of rows of a prompt
__device__ __forceinline__ int ap_tiles(int n, int group, int tile) { return (int)(((int64_t)n * group + tile - 1) / tile); }

// fp32.  A workgroup has 128 rows of one kv head: row r of a prompt is head r % group of token r / group, so that shared heads read a tile of K and V once.
// Tiles of 32 tokens are staged in LDS as they stand in the pages, one while the one before it is worked on.  Both products have the cache's side as
// operand A and the rows as columns: a lane holds weights of one row only, the softmax needs one exchange between lane halves, and what comes out of
// the first product is what the second takes (K's rows are read in the order that makes it so).
// Bound: not by a unit.  The matrix units are busy for 31 to 47 % of the time at 64 to 128 columns (4 x 897 tokens of 16 heads of 128, window 284, 126 us, 55 TFLOP/s of 154; 2 x 1805 of
// 16 heads of 64 272 us, 49; 1 x 2000 of 16 heads of 96 181 us, 68): units run dry while the longest row tile of a causal prompt is worked on (of two wavefronts that a SIMD has room for
// at 64 and at 128 columns 0.9 and 1.3 are there on average, of the one at 96 0.9), and a wavefront has wait, barrier, first product, softmax and second product of a tile one after another (it waits 23
// to 39 % of its time).  Wider heads have one wavefront a SIMD; from 192 columns on registers go to memory (256: 596 bytes a lane, the matrix units busy 10 %, 1 x 1500 of 8 heads 492 us, 19 TFLOP/s).
// Small batches: latency, 4 x 64 tokens of 16 heads of 64 11.3 us, of which two tiles are 4 and what comes before the first 4.  Two wavefronts a SIMD at 128 columns: with the one that the compiler
// takes if left alone 176 us instead of 133, 19 x 124 tokens of 32 heads 103 -> 72; 96 columns 183 -> 230, so only at 128.  Not kept: twice and four times as many cuts, for the longest row tiles (2 x 1805
// tokens of 16 heads of 64 272 -> 238 and 213 us, 1 x 1024 of 128 101 -> 86 and 84, but 4 x 897 133 -> 165, 2000 of 96 183 -> 197 and 218: parts are written and read again).
template <int DT>
__global__ __launch_bounds__(AP_WAVES * 64, DT == 4 ? 2 : 1) void attend_prefill_f32(ApArgs a) {
  typedef float T;
  constexpr int NW = AP_WAVES, TK = AP_TILE, ST = 2;               // two stages: a tile is worked on, the next one is on its way
  constexpr int D = DT * 32, KB = D / 16, TB = TK / 16, TS = TK / 32, TM = NW * 32, THREADS = NW * 64;
  constexpr int BLOCK = 16 * D * (int)sizeof(T);                   // bytes of sixteen tokens of K, and of V
  constexpr int STAGE = 2 * TB * BLOCK, PIECES = STAGE / 1024, LOADS = PIECES / NW;
  static_assert(PIECES % NW == 0, "every wavefront stages as much");
  typedef typename Op<T>::frag frag;
  extern __shared__ char smem[];
  int *wave_sums = reinterpret_cast<int *>(smem + ST * STAGE), *pre = wave_sums + NW;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), n = lane & 31, half = lane >> 5;
  const int kvh = blockIdx.x % a.kv.n_kv, item = blockIdx.x / a.kv.n_kv, group = a.group;
  const KvItem f = kv_item<THREADS>(a.kv, a.tok_offsets, a.seqs, a.P, a.rows, item, pre, wave_sums, [&](const KvRows &r, const KvSeq &) { return ap_tiles(r.n, group, TM); });
  if (f.item < 0) return;
  const int n_rows = f.n, row0 = f.first, len = f.len;
  const int32_t *table = a.kv.table + (int64_t)f.row * a.kv.max_pages;
  const int r0 = (ap_tiles(n_rows, group, TM) - 1 - f.item) * TM;     // the rows that see most come first
  const int r_end = n_rows * group, base = len - n_rows;
  const int i0 = base + kv_divide(r0, a.by_group), i1 = base + kv_divide(min(r0 + TM, r_end) - 1, a.by_group);
  const KvSpan span = i1 < 0 ? KvSpan{0, 0, 0} : kv_span(max(i0, 0), i1, a.window, a.sinks, TK);
  const ApShare share = ap_share(span.count, a.splits, blockIdx.y, ap_least(a.kv.dtype));
  if ((int)blockIdx.y >= share.parts) return;

  // the pages of a tile's blocks of sixteen tokens, -1 for none; asked for a tile before they are used
  const int page_bits = 31 - __builtin_clz(a.kv.page);
  struct Ids { int id[TB]; };
  auto ids_of = [&](int u) {
    Ids r;
    const int t0 = span.at(u) * TK;
#pragma unroll
    for (int b = 0; b < TB; ++b) r.id[b] = scalar_word(table + min((t0 + 16 * b) >> page_bits, a.kv.max_pages - 1));
    return r;
  };
  const int64_t page_elems = (int64_t)a.kv.n_kv * a.kv.page * D, head0 = (int64_t)kvh * a.kv.page * D;
  auto ok = [&](int id) { return (unsigned)id < (unsigned)a.kv.n_pages; };
  auto stage = [&](int u, const Ids &ids, int buf) {
    const int t0 = span.at(u) * TK;
#pragma unroll
    for (int q = 0; q < LOADS; ++q) {
      const int piece = wave * LOADS + q, of_v = piece / (PIECES / 2), rest = piece % (PIECES / 2), block = rest / (BLOCK / 1024);
      int id = ids.id[0];
#pragma unroll
      for (int b = 1; b < TB; ++b) id = block == b ? ids.id[b] : id;
      id = ok(id) ? id : 0;
      const char *src = (const char *)(of_v ? a.V : a.K) + ((int64_t)id * page_elems + head0 + (int64_t)((t0 + 16 * block) & (a.kv.page - 1)) * D) * (int64_t)sizeof(T) +
                        (rest % (BLOCK / 1024)) * 1024;
      __builtin_amdgcn_global_load_lds(PARSE_GLB_PTR(src + lane * 16), PARSE_LDS_PTR(smem + buf * STAGE + piece * 1024), 16, 0, 0);
    }
  };
  Ids now{}, next{}, later{};                                      // of tiles u, u + 1, u + 2
  if (share.first < share.last) now = ids_of(share.first);
  if (share.first + 1 < share.last) next = ids_of(share.first + 1);

  // this lane's row, and the positions of the wavefront's rows
  const int r = r0 + wave * 32 + n, token = kv_divide(min(r, r_end - 1), a.by_group), head = kvh * group + (min(r, r_end - 1) - token * group);
  const int i = base + token;
  const int wi0 = base + kv_divide(min(r0 + wave * 32, r_end - 1), a.by_group), wi1 = base + kv_divide(min(r0 + wave * 32 + 31, r_end - 1), a.by_group);
  const int lo = kv_window_begin(i, a.window), wlo = kv_window_begin(wi0, a.window), whi = kv_window_begin(wi1, a.window);
  const bool idle = r0 + wave * 32 >= r_end;
  frag qf[KB];
  {
    const T *q = reinterpret_cast<const T *>(a.q) + (int64_t)(row0 + token) * a.q_stride + (int64_t)head * D + 8 * half;
#pragma unroll
    for (int k = 0; k < KB; ++k) qf[k] = Op<T>::sign(Op<T>::load(q + 16 * k), a.q_sign);
  }
  // q comes first: whoever waits for a tile has it
  asm volatile("" ::: "memory");
  if (share.first < share.last) stage(share.first, now, 0);
  float m = -INFINITY, l = 0.f;
  f32x16 o[DT];
#pragma unroll
  for (int d = 0; d < DT; ++d)
#pragma unroll
    for (int e = 0; e < 16; ++e) o[d][e] = 0.f;
  // the first product's operand row n of 32 tokens: token ktok, so that a lane half gets eight consecutive tokens of each sixteen
  const int ktok = 16 * (n >> 4) + 8 * ((n >> 2) & 1) + 4 * ((n >> 3) & 1) + (n & 3);

  int buf = 0;
  for (int u = share.first; u < share.last; ++u, buf ^= 1) {
    const int t0 = span.at(u) * TK;
    if (u + 2 < share.last) later = ids_of(u + 2);
    wait_vm<0>();
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    wg_barrier();                                                  // this tile has landed for everybody, the one before it is read by everybody
    if (u + 1 < share.last) stage(u + 1, next, buf ^ 1);
    const Ids ids = now;
    now = next; next = later;
    if (idle || t0 > wi1 || (t0 + TK <= wlo && t0 >= a.sinks)) continue;
    const T *ks = reinterpret_cast<const T *>(smem + buf * STAGE), *vs = reinterpret_cast<const T *>(smem + buf * STAGE + STAGE / 2);
    f32x16 sc[TS];
#pragma unroll
    for (int s = 0; s < TS; ++s) {
#pragma unroll
      for (int e = 0; e < 16; ++e) sc[s][e] = 0.f;
      const T *kr = ks + (2 * s + (ktok >> 4)) * 16 * D + (ktok & 15) * 8 + half * 128;
#pragma unroll
      for (int k = 0; k < KB; ++k) sc[s] = Op<T>::mma32(Op<T>::load(kr + k * 256), qf[k], sc[s]);
    }
    uint32_t blocks = 0;                                           // of sixteen tokens whose page is there
#pragma unroll
    for (int b = 0; b < TB; ++b) blocks |= (ok(ids.id[b]) ? 1u : 0u) << b;
    const bool whole = blocks == (1u << TB) - 1u && t0 + TK - 1 <= wi0 && (t0 >= whi || t0 + TK <= a.sinks);
    if (!whole) {
#pragma unroll
      for (int s = 0; s < TS; ++s)
#pragma unroll
        for (int x = 0; x < 16; ++x) {                             // register 8 b + e of block pair s holds token 32 s + 16 b + 8 half + e
          const bool sees = (bool)(blocks >> (2 * s + x / 8) & 1) & kv_sees(i, lo, a.sinks, t0 + 32 * s + 16 * (x / 8) + 8 * half + x % 8);
          sc[s][x] = sees ? sc[s][x] : -INFINITY;
        }
    }
    float top = -INFINITY;
#pragma unroll
    for (int s = 0; s < TS; ++s)
#pragma unroll
      for (int x = 0; x < 16; ++x) top = fmaxf(top, sc[s][x]);
    if (__any(top > m + a.lag)) {
      const float grown = fmaxf(m, lane_max<32>(top));
      const float by = at_exp2((m - finite_or_0(grown)) * a.scale);
      l *= by;
#pragma unroll
      for (int d = 0; d < DT; ++d) o[d] *= by;
      m = grown;
    }
    const float low = at_base(m, a.scale);
    frag pf[TB];
#pragma unroll
    for (int b = 0; b < TB; ++b) {
      float w[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) { w[e] = at_exp2(fmaf(sc[b / 2][8 * (b % 2) + e], a.scale, -low)); l += w[e]; sc[b / 2][8 * (b % 2) + e] = w[e]; }
      pf[b] = Op<T>::pack(w);
    }
    if (whole) {
#pragma unroll
      for (int b = 0; b < TB; ++b) {
        const T *vr = vs + b * 16 * D + (half * D + n) * 8;
#pragma unroll
        for (int d = 0; d < DT; ++d) o[d] = Op<T>::mma32(Op<T>::load(vr + d * 256), pf[b], o[d]);
      }
      continue;
    }
    bool bad = false;
#pragma unroll
    for (int b = 0; b < TB; ++b) {
      const T *vr = vs + b * 16 * D + (half * D + n) * 8;
      uint32_t keep = 0;                                           // tokens that some row of the wavefront sees
#pragma unroll
      for (int e = 0; e < 8; ++e) keep |= (blocks >> b & 1u & (kv_sees(wi1, wlo, a.sinks, t0 + 16 * b + 8 * half + e) ? 1u : 0u)) << e;
#pragma unroll
      for (int d = 0; d < DT; ++d) {
        frag vf = Op<T>::only(Op<T>::load(vr + d * 256), keep);
        bad |= Op<T>::finite_only(vf);
        o[d] = Op<T>::mma32(vf, pf[b], o[d]);
      }
    }
    // Infinities and NaN of V that some rows of the wavefront see and others do not: the product above had 0 in their place,
    // the rows that see them get them here, one token after another (0 times infinity would reach the others).
    if (__any(bad)) {
      for (int j = 0; j < TK; ++j) {
        const int b = j >> 4, h = j >> 3 & 1;
        float w = 0.f;
#pragma unroll
        for (int c = 0; c < TB; ++c)
#pragma unroll
          for (int e = 0; e < 8; ++e) w = ((c == b) & (e == (j & 7))) ? sc[c / 2][8 * (c % 2) + e] : w;
        w = __shfl(w, n + 32 * h, 64);
        const bool mine = (bool)(blocks >> b & 1) & kv_sees(i, lo, a.sinks, t0 + j);
        const T *vr = vs + b * 16 * D + h * D * 8 + (j & 7);
#pragma unroll
        for (int d = 0; d < DT; ++d)
#pragma unroll
          for (int x = 0; x < 16; ++x) {
            const T v = vr[(32 * d + 8 * (x / 4) + 4 * half + x % 4) * 8];
            const float add = w * Op<T>::value(v);
            o[d][x] = (mine & !Op<T>::finite(v)) ? o[d][x] + add : o[d][x];
          }
      }
    }
  }
  if (idle || r >= r_end) return;
  l = lane_sum<32>(l);
  const int row = wave * 32 + n;                                   // of the tile
  if (share.parts > 1) {
    float *part = a.part + ((int64_t)blockIdx.x * a.splits + blockIdx.y) * AP_ROWS * (D + 2);
#pragma unroll
    for (int d = 0; d < DT; ++d)
#pragma unroll
      for (int c = 0; c < 4; ++c)
        *reinterpret_cast<f32x4 *>(part + row * D + 32 * d + 8 * c + 4 * half) = f32x4{o[d][4 * c], o[d][4 * c + 1], o[d][4 * c + 2], o[d][4 * c + 3]};
    if (half == 0) { part[AP_ROWS * D + row] = m; part[AP_ROWS * (D + 1) + row] = l; }
    return;
  }
  const float by = l == 0.f ? 0.f : 1.f / l;
  T *out = reinterpret_cast<T *>(a.out) + (int64_t)(row0 + token) * a.out_stride + (int64_t)head * D;
#pragma unroll
  for (int d = 0; d < DT; ++d)
#pragma unroll
    for (int c = 0; c < 4; ++c)
      Op<T>::store4(out + 32 * d + 8 * c + 4 * half, o[d][4 * c] * by, o[d][4 * c + 1] * by, o[d][4 * c + 2] * by, o[d][4 * c + 3] * by);
  if (a.lse && half == 0) a.lse[(int64_t)(row0 + token) * a.n_q + head] = at_lse(m, a.scale, l);
}

// bf16: the same, with the products of one tile under the softmax of the tile before it: in an iteration a wavefront has the
// scores of tile u and the operands of K of tile u + 1 in registers, multiplies the latter between the exponentials of the former, and reads the
// operands of K of tile u + 2 between the products with V of tile u.  K is staged two tiles ahead of V; group j of loads is K of
// tile j and V of tile j - 2 (at the ends a tile that is there stands for the one that is not, so that all groups are alike).
// Of a tile (16 matrix instructions of 32 cycles a wavefront) the softmax takes 45 vector instructions and 16 exponentials, about as long; scalar work was a hundred
// instructions more before the places of 64 tiles were worked out at once (648 -> 574 us below).  Two wavefronts a SIMD, 128 rows a workgroup and two of them
// a unit: with 256 rows the eight wavefronts of a unit wait for each other at every tile (650 us and, 8 x 512 tokens, 81 against 607 and 63).
// Bound: large calls by power (one prompt of 8192 tokens, 32 heads over 8: 512 to 560 us = 0.98 to 1.07 PFLOP/s at 1.67 GHz; with zeros for data 394 us at the full clock; a large
// library product reaches 1.28).  Small ones by what is not a tile: of the time that workgroups have on their units, 8 x 512 tokens of 32 heads (44 us for 135 MB, 16 tiles at most), 35 % go before the
// first tile (6 us: lengths, then table and q, then K), 51 % on tiles (0.9 us each), 14 % on the stores, and for the last quarter of the call units run dry.  20 ragged prompts
// with a window: 14, 80 and 5 %, 0.97 us a tile.  One prompt of 2048 tokens, 32 heads over 8 (50 us): every workgroup has its place at once, and the longest row tile, 64 tiles of
// 0.84 us, is the call.  Wider heads: one workgroup a unit, and from 192 columns on registers go to memory (256: 1032 bytes a lane; 4 x 1000 of 16 heads over 4, 90 us, 363 TFLOP/s).
// CAREFUL: infinities and NaN of V in places that some rows of the workgroup see and others do not reach only the former (0 times infinity would
// reach the others).  Without, something that is not finite comes out where they are met: then nothing is stored and the answer is false.
constexpr int AP_STAGES = 4;                 // tiles of K, and of V, in LDS
constexpr int ap_lds_bytes(int DT) { return 2 * AP_STAGES * AP_TILE * DT * 32 * 2; }

template <int DT, bool CAREFUL>
__device__ __forceinline__ bool ap_rows(const ApArgs &a, const KvItem &f, char *smem) {
  typedef uint16_t T;
  typedef Op<T> O;
  typedef O::frag frag;
  constexpr int D = DT * 32, KB = D / 16, TK = AP_TILE, TB = 2, TM = AP_ROWS, THREADS = AP_WAVES * 64, ST = AP_STAGES;
  constexpr int BLOCK = 32 * D, TILE = TB * BLOCK, LOADS = BLOCK / 1024, AHEAD = ST - 1;   // groups on their way
  int *flag = reinterpret_cast<int *>(smem + 2 * ST * TILE);
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), n = lane & 31, half = lane >> 5;
  const int kvh = blockIdx.x % a.kv.n_kv, group = a.group;
  const int n_rows = f.n, row0 = f.first, len = f.len;
  const int32_t *table = a.kv.table + (int64_t)f.row * a.kv.max_pages;
  const int r0 = (ap_tiles(n_rows, group, TM) - 1 - f.item) * TM;     // the rows that see most come first
  const int r_end = n_rows * group, base = len - n_rows;
  const int i0 = base + kv_divide(r0, a.by_group), i1 = base + kv_divide(min(r0 + TM, r_end) - 1, a.by_group);
  const KvSpan span = i1 < 0 ? KvSpan{0, 0, 0} : kv_span(max(i0, 0), i1, a.window, a.sinks, TK);
  const ApShare share = ap_share(span.count, a.splits, blockIdx.y, ap_least(a.kv.dtype));
  if ((int)blockIdx.y >= share.parts) return true;
  const int count = share.last - share.first, groups = count > 0 ? count + 2 : 0;   // tiles are numbered from the share's first

  const int page_bits = 31 - __builtin_clz(a.kv.page);
  const int64_t page_elems = (int64_t)a.kv.n_kv * a.kv.page * D, head0 = (int64_t)kvh * a.kv.page * D;
  auto ok = [&](int id) { return (unsigned)id < (unsigned)a.kv.n_pages; };
  auto page_at = [&](int t) { return table[min(t >> page_bits, a.kv.max_pages - 1)]; };
  // Of every group wavefront w stages one block of sixteen tokens: w / 2 says K or V, w % 2 which block.  Where the tiles stand is worked out
  // for 64 of them at once, a lane each, and read lane by lane: scalar instructions for every tile would take as long as the products.
  const int of_v = wave >> 1, blk = wave & 1;
  const char *const pool = (const char *)(of_v ? a.V : a.K) + head0 * 2;
  int next_group = 0, next_slot = of_v ? ST - 2 : 0;
  uint32_t place_lo = 0, place_hi = 0;                             // lane j: bytes from pool to this wavefront's block of group 64 * (next_group / 64) + j
  auto places = [&]() {
    const int g = next_group + lane, t = span.at(share.first + (of_v ? max(min(g, groups - 1) - 2, 0) : min(g, count - 1))) * TK + 16 * blk, id = page_at(t);
    const int64_t at = (int64_t)(ok(id) ? id : 0) * (page_elems * 2) + (t & (a.kv.page - 1)) * (D * 2);
    place_lo = (uint32_t)at;
    place_hi = (uint32_t)(at >> 32);
  };
  uint32_t infos = 0;                                              // lane j: first token of tile 64 * (u / 64) + j, and
  constexpr uint32_t THERE_A = 1, THERE_B = 2, WHOLE = 4;          // pages of its two blocks there; every row of the workgroup sees all of it
  const int hi = kv_window_begin(i1, a.window), wglo = kv_window_begin(i0, a.window);
  auto look = [&](int u) {
    const int t0 = span.at(share.first + min(u + lane, count - 1)) * TK;
    const bool there_a = ok(page_at(t0)), there_b = ok(page_at(t0 + 16));
    const bool all = there_a & there_b & (t0 + TK - 1 <= i0) & ((t0 >= hi) | (t0 + TK <= a.sinks));
    infos = (uint32_t)t0 | (there_a ? THERE_A : 0u) | (there_b ? THERE_B : 0u) | (all ? WHOLE : 0u);
  };
  auto stage = [&]() {
    const char *src = pool + ((uint64_t)(uint32_t)__builtin_amdgcn_readlane(place_hi, next_group & 63) << 32 | (uint32_t)__builtin_amdgcn_readlane(place_lo, next_group & 63));
    char *dst = smem + of_v * ST * TILE + blk * BLOCK + next_slot * TILE;
#pragma unroll
    for (int q = 0; q < LOADS; q += 4) {
      // the offset moves both sides
      __builtin_amdgcn_global_load_lds(PARSE_GLB_PTR(src + q * 1024 + lane * 16), PARSE_LDS_PTR(dst + q * 1024), 16, 0, 0);
      if (q + 1 < LOADS) __builtin_amdgcn_global_load_lds(PARSE_GLB_PTR(src + q * 1024 + lane * 16), PARSE_LDS_PTR(dst + q * 1024), 16, 1024, 0);
      if (q + 2 < LOADS) __builtin_amdgcn_global_load_lds(PARSE_GLB_PTR(src + q * 1024 + lane * 16), PARSE_LDS_PTR(dst + q * 1024), 16, 2048, 0);
      if (q + 3 < LOADS) __builtin_amdgcn_global_load_lds(PARSE_GLB_PTR(src + q * 1024 + lane * 16), PARSE_LDS_PTR(dst + q * 1024), 16, 3072, 0);
    }
    next_slot = next_slot + 1 == ST ? 0 : next_slot + 1;
    if ((++next_group & 63) == 0) places();
  };

  // this lane's row, and the positions of the wavefront's rows
  const int r = r0 + wave * 32 + n, token = kv_divide(min(r, r_end - 1), a.by_group), head = kvh * group + (min(r, r_end - 1) - token * group);
  const int i = base + token;
  const int wi0 = base + kv_divide(min(r0 + wave * 32, r_end - 1), a.by_group), wi1 = base + kv_divide(min(r0 + wave * 32 + 31, r_end - 1), a.by_group);
  const int lo = kv_window_begin(i, a.window), wlo = kv_window_begin(wi0, a.window);
  const bool idle = r0 + wave * 32 >= r_end;
  frag qf[KB];
  {
    const T *q = reinterpret_cast<const T *>(a.q) + (int64_t)(row0 + token) * a.q_stride + (int64_t)head * D + 8 * half;
#pragma unroll
    for (int k = 0; k < KB; ++k) qf[k] = O::sign(O::load(q + 16 * k), a.q_sign);
  }
  asm volatile("" ::: "memory");                                   // q comes first: whoever waits for a tile has it
  if (groups) {
    places();
    look(0);
#pragma unroll
    for (int j = 0; j < ST; ++j)
      if (j < groups) stage();
  }
  float m = -INFINITY, l = 0.f;
  f32x16 o[DT], sc;
#pragma unroll
  for (int d = 0; d < DT; ++d)
#pragma unroll
    for (int e = 0; e < 16; ++e) o[d][e] = 0.f;
  const int ktok = 16 * (n >> 4) + 8 * ((n >> 2) & 1) + 4 * ((n >> 3) & 1) + (n & 3);
  const int k_at = ((ktok >> 4) * 16 * D + (ktok & 15) * 8 + half * 128) * 2, v_at = ST * TILE + (half * D + n) * 16;
  frag kf[KB];
  auto read_k = [&](int slot) {
#pragma unroll
    for (int k = 0; k < KB; ++k) kf[k] = O::load(reinterpret_cast<const T *>(smem + slot * TILE + k_at + k * 512));
  };
  auto first = [&]() {                                             // scores of the tile in kf
    f32x16 s;
#pragma unroll
    for (int e = 0; e < 16; ++e) s[e] = 0.f;
#pragma unroll
    for (int k = 0; k < KB; ++k) s = O::mma32(kf[k], qf[k], s);
    return s;
  };
  auto meet = [&]() {                                              // everybody's reads of LDS are done, everybody's loads so far have landed
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    wg_barrier();
  };
  if (groups) {
    wait_slices<AHEAD, LOADS>(min(ST - 1, groups - 1));            // group 0
    wg_barrier();
    read_k(0);
    sc = first();
    wait_slices<AHEAD - 1, LOADS>(min(ST - 1, groups - 1) - 1);
    meet();
    if (ST < groups) stage();
    read_k(1);
  }
  int slot = 0;                                                    // u % ST
  auto begin = [&](int u) {                                        // tile u of V and u + 2 of K are there; the loads that the freed places take
    if (u + 1 + AHEAD < groups) wait_vm<(AHEAD - 1) * LOADS>(); else wait_slices<AHEAD - 1, LOADS>(groups - 1 - (u + 2));
    meet();
    if (next_group < groups) stage();
  };
  auto lag = [&](const f32x16 &sc) {                               // the running maximum, where it has to grow
    float top = -INFINITY;
#pragma unroll
    for (int x = 0; x < 16; ++x) top = fmaxf(top, sc[x]);
    if (__any(top > m + a.lag)) {
      const float grown = fmaxf(m, lane_max<32>(top));
      const float by = at_exp2((m - finite_or_0(grown)) * a.scale);
      l *= by;
#pragma unroll
      for (int d = 0; d < DT; ++d) o[d] *= by;
      m = grown;
    }
  };
  const int last = idle ? -1 : wi1;                                // position of the wavefront's last row
  frag vf[DT * TB], pf[TB];
  auto read_v = [&]() {
    const T *vs = reinterpret_cast<const T *>(smem + v_at + slot * TILE);
#pragma unroll
    for (int b = 0; b < TB; ++b)
#pragma unroll
      for (int d = 0; d < DT; ++d) vf[b * DT + d] = O::load(vs + b * 16 * D + d * 256);
  };
  auto weigh = [&](const f32x16 &sc) {
    const float low = at_base(m, a.scale);
    float w[16];
#pragma unroll
    for (int x = 0; x < 16; ++x) { w[x] = at_exp2(fmaf(sc[x], a.scale, -low)); l += w[x]; }
    pf[0] = O::pack(w); pf[1] = O::pack(w + 8);
  };
  auto second = [&]() {
#pragma unroll
    for (int b = 0; b < TB; ++b)
#pragma unroll
      for (int d = 0; d < DT; ++d) o[d] = O::mma32(vf[b * DT + d], pf[b], o[d]);
  };
  // Tiles that some row does not see whole: what no row of the workgroup sees becomes 0 in V; infinities and NaN that some rows see and
  // others do not (0 times infinity would reach those) become the largest finite value of their sign, and the rows that see them get them from
  // patch().  One 16-byte piece (eight tokens of a column) a thread and step.
  int turn = 0;
  auto clean = [&](uint32_t info) {
    const int t0 = info & ~31u;
    uint32_t most = 0;
    for (int e = tid; e < TILE / 16; e += THREADS) {
      const int side = e / D;                                      // eight tokens
      const uint32_t keep = info & (side < 2 ? THERE_A : THERE_B) ? kv_sees8(i1, wglo, a.sinks, t0 + 8 * side) : 0u;
      T *at = reinterpret_cast<T *>(smem + ST * TILE + slot * TILE) + e * 8;
      const frag v = O::finite_only(O::only(O::load(at), keep), most);
      *reinterpret_cast<frag *>(at) = v;
    }
    const bool bad = (most & 0xffffu) >= 0x7f80u || most >= 0x7f800000u;
    if (__any(bad) && lane == 0) flag[turn] = 1;
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    wg_barrier();
    const int f = __builtin_amdgcn_readfirstlane(flag[turn]);
    turn ^= 1;
    if (tid == 0) flag[turn] = 0;                                  // everybody has read it: it was the one before
    return f != 0;
  };
  auto patch = [&](uint32_t info) {
    const int t0 = info & ~31u;
#pragma unroll 1
    for (int j = 0; j < TK; ++j) {
      const int b = j >> 4, h = j >> 3 & 1;
      if (!(info & (b ? THERE_B : THERE_A))) continue;
      const int id = page_at(t0 + 16 * b);
      uint32_t bits = 0;                                           // the weight as it was multiplied
#pragma unroll
      for (int x = 0; x < 16; ++x) bits = x == 8 * b + (j & 7) ? (x & 1 ? pf[x / 8][x % 8 / 2] & 0xffff0000u : pf[x / 8][x % 8 / 2] << 16) : bits;
      const float w = __shfl(__uint_as_float(bits), n + 32 * h, 64);
      const bool mine = kv_sees(i, lo, a.sinks, t0 + j);
      const T *vr = reinterpret_cast<const T *>(a.V) + (int64_t)id * page_elems + head0 + (int64_t)((t0 + 16 * b) & (a.kv.page - 1)) * D + h * D * 8 + (j & 7);
#pragma unroll
      for (int d = 0; d < DT; ++d)
#pragma unroll
        for (int x = 0; x < 16; ++x) {
          const T v = vr[(32 * d + 8 * (x / 4) + 4 * half + x % 4) * 8];
          const float add = w * O::value(v);
          o[d][x] = (mine & !O::finite(v)) ? o[d][x] + add : o[d][x];
          if (x % 4 == 3) asm volatile("" ::: "memory");           // few of these reads at a time: the path is rare, its registers are everybody's
        }
    }
  };
  bool odd = false;                                                // something of V was not finite in a tile that was cleaned
  auto tile = [&](int u, f32x16 &sc, f32x16 &sn) {                 // scores of tile u in sc; those of tile u + 1 come into sn
    const uint32_t info = __builtin_amdgcn_readlane(infos, u & 63);
    const int t0 = info & ~31u;
    begin(u);
    bool bad = false;
    if (!(info & WHOLE) && (CAREFUL || t0 + TK > len || (info & (THERE_A | THERE_B)) != (THERE_A | THERE_B))) bad = clean(info);
    if (t0 <= last) {
      if (!(info & WHOLE)) {
        // register 8 b + e holds token 16 b + 8 half + e
        const uint32_t bits = (info & THERE_A ? kv_sees8(i, lo, a.sinks, t0 + 8 * half) : 0u) | (info & THERE_B ? kv_sees8(i, lo, a.sinks, t0 + 16 + 8 * half) << 8 : 0u);
#pragma unroll
        for (int x = 0; x < 16; ++x) sc[x] = bits & (1u << x) ? sc[x] : -INFINITY;
      }
      lag(sc);
      read_v();
      sn = first();
      weigh(sc);
      read_k((slot + 2) % ST);
      second();
      if (CAREFUL) {
        if (bad) patch(info);
      } else {
        odd |= bad;
      }
    }
    if (((u + 1) & 63) == 0) look(u + 1);
    slot = slot + 1 == ST ? 0 : slot + 1;
  };
  f32x16 sn = sc;
  int u = 0;
  for (; u + 1 < count; u += 2) {
    tile(u, sc, sn);
    tile(u + 1, sn, sc);
  }
  if (u < count) tile(u, sc, sn);
  if (!CAREFUL) {
    float sum = odd ? INFINITY : l;
#pragma unroll
    for (int d = 0; d < DT; ++d)
#pragma unroll
      for (int x = 0; x < 16; ++x) sum = fmaf(o[d][x], 0.f, sum);  // NaN if one of them is not finite
    if (__any(!(fabsf(sum) < INFINITY)) && !idle && lane == 0) flag[2] = 1;
    __syncthreads();
    if (__builtin_amdgcn_readfirstlane(flag[2])) return false;
  }
  if (idle) return true;
  l = lane_sum<32>(l);
  if (share.parts > 1) {
    const int row = wave * 32 + n;                                 // of the tile
    float *part = a.part + ((int64_t)blockIdx.x * a.splits + blockIdx.y) * TM * (D + 2);
#pragma unroll
    for (int d = 0; d < DT; ++d)
#pragma unroll
      for (int c = 0; c < 4; ++c)
        *reinterpret_cast<f32x4 *>(part + row * D + 32 * d + 8 * c + 4 * half) = f32x4{o[d][4 * c], o[d][4 * c + 1], o[d][4 * c + 2], o[d][4 * c + 3]};
    if (half == 0) { part[TM * D + row] = m; part[TM * (D + 1) + row] = l; }
    return true;
  }
  const float by = l == 0.f ? 0.f : 1.f / l;
  // the lane halves hold columns 8 c + 0..3 and 8 c + 4..7 of a row: they swap, so that each has eight of them, of every other c
  T *out = reinterpret_cast<T *>(a.out) + (int64_t)(row0 + token) * a.out_stride + (int64_t)head * D + 8 * half;
#pragma unroll
  for (int d = 0; d < DT; ++d)
#pragma unroll
    for (int c = 0; c < 4; c += 2) {
      const float *u = reinterpret_cast<const float *>(&o[d]) + 4 * c;
      const u32x2 x = __builtin_amdgcn_permlane32_swap(cvt_pk_bf16(u[0] * by, u[1] * by), cvt_pk_bf16(u[4] * by, u[5] * by), false, false);
      const u32x2 y = __builtin_amdgcn_permlane32_swap(cvt_pk_bf16(u[2] * by, u[3] * by), cvt_pk_bf16(u[6] * by, u[7] * by), false, false);
      if (r < r_end) *reinterpret_cast<u32x4 *>(out + 32 * d + 8 * c) = u32x4{x[0], y[0], x[1], y[1]};
    }
  if (r >= r_end) return true;
  if (a.lse && half == 0) a.lse[(int64_t)(row0 + token) * a.n_q + head] = at_lse(m, a.scale, l);
  return true;
}

template <int DT>
__global__ __launch_bounds__(AP_WAVES * 64, DT <= 4 ? 2 : 1) void attend_prefill_bf16(ApArgs a) {
  extern __shared__ char smem[];                                   // AP_STAGES tiles of K, as many of V, three flags, the prompts' tiles
  int *flag = reinterpret_cast<int *>(smem + ap_lds_bytes(DT)), *wave_sums = flag + 3, *pre = wave_sums + AP_WAVES;
  const KvItem f = kv_item<AP_WAVES * 64>(a.kv, a.tok_offsets, a.seqs, a.P, a.rows, blockIdx.x / a.kv.n_kv, pre, wave_sums,
                                          [&](const KvRows &r, const KvSeq &) { return ap_tiles(r.n, a.group, AP_ROWS); });
  if (f.item < 0) return;
  if (threadIdx.x < 3) flag[threadIdx.x] = 0;                      // [2]: something is not finite
  if (!ap_rows<DT, false>(a, f, smem)) ap_rows<DT, true>(a, f, smem);
}

// Joins the parts of a tile of rows; workgroup (x, y) has four of the rows of tile and kv head x, a wavefront one of them, four columns a lane.
constexpr int AP_JOIN = AP_WAVES;
template <class T>
__global__ __launch_bounds__(AP_WAVES * 64) void ap_join(ApArgs a) {
  extern __shared__ int pre[];
  const int D = a.kv.d, group = a.group, kvh = blockIdx.x % a.kv.n_kv, lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const KvItem f = kv_item<AP_WAVES * 64>(a.kv, a.tok_offsets, a.seqs, a.P, a.rows, blockIdx.x / a.kv.n_kv, pre + AP_WAVES, pre,
                                          [&](const KvRows &r, const KvSeq &) { return ap_tiles(r.n, a.group, AP_ROWS); });
  if (f.item < 0) return;
  const int r0 = (ap_tiles(f.n, group, AP_ROWS) - 1 - f.item) * AP_ROWS, r_end = f.n * group, base = f.len - f.n;
  const int i0 = base + kv_divide(r0, a.by_group), i1 = base + kv_divide(min(r0 + AP_ROWS, r_end) - 1, a.by_group);
  const KvSpan span = i1 < 0 ? KvSpan{0, 0, 0} : kv_span(max(i0, 0), i1, a.window, a.sinks, AP_TILE);
  const int parts = ap_share(span.count, a.splits, 0, ap_least(a.kv.dtype)).parts;
  if (parts == 1) return;
  const float *first = a.part + (int64_t)blockIdx.x * a.splits * AP_ROWS * (D + 2);
  const int64_t next = (int64_t)AP_ROWS * (D + 2);
  {
    const int row = blockIdx.y * AP_JOIN + wave, r = r0 + row;
    if (r >= r_end) return;
    // lane x: part x; there are 64 at most
    const float m = lane < parts ? first[lane * next + AP_ROWS * D + row] : -INFINITY, l = lane < parts ? first[lane * next + AP_ROWS * (D + 1) + row] : 0.f;
    float top = m;
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor(top, o, 64));
    const float by = at_exp2((m - finite_or_0(top)) * a.scale), total = wave_sum(lane < parts ? l * by : 0.f);
    const float over = total == 0.f ? 0.f : 1.f / total;
    const int token = kv_divide(r, a.by_group), head = kvh * group + r - token * group;
    f32x4 o = {0.f, 0.f, 0.f, 0.f};
    if (4 * lane < D) {
#pragma unroll 16
      for (int x = 0; x < parts; ++x)
        o += __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(by), x)) * *reinterpret_cast<const f32x4 *>(first + x * next + row * D + 4 * lane);
      Op<T>::store4(reinterpret_cast<T *>(a.out) + (int64_t)(f.first + token) * a.out_stride + (int64_t)head * D + 4 * lane, o[0] * over, o[1] * over, o[2] * over,
                    o[3] * over);
    }
    if (a.lse && lane == 0) a.lse[(int64_t)(f.first + token) * a.n_q + head] = at_lse(top, a.scale, total);
  }
}

// tiles of rows, times kv heads: a prompt's last tile may be begun only, rows / tile + prompts in all
static int64_t ap_items(const parse_kv *kv, int n_q, int rows, int P) {
  return ((int64_t)rows * (n_q / kv->n_kv) / AP_ROWS + std::min(P, rows)) * kv->n_kv;
}
// Few rows over caches that may be long: the tokens are cut, so that the workgroups fill the card.  Known are the tiles and how much the table can hold.
static int ap_splits(const parse_kv *kv, int n_q, int rows, int P) {
  const int64_t items = ap_items(kv, n_q, rows, P), tiles = (int64_t)kv->max_pages * kv->page / AP_TILE;
  const int least = ap_least(kv->dtype);
  if (items * 2 > AP_GROUPS || tiles < 2 * least) return 1;
  return (int)std::min<int64_t>({AP_GROUPS / items, tiles / least, 64});
}
static size_t ap_bytes(const parse_kv *kv, int n_q, int rows, int P) {
  const int splits = ap_splits(kv, n_q, rows, P);
  return splits == 1 ? 0 : (size_t)ap_items(kv, n_q, rows, P) * splits * AP_ROWS * (kv->d + 2) * 4;
}

template <class T, class K>
static int ap_launch(const ApArgs &a, K kernel, size_t lds, hipStream_t s) {
  const int64_t items = ap_items(&a.kv, a.n_q, a.rows, a.P);
  if (items > INT32_MAX) return PARSE_ESHAPE;
  const size_t scan = (AP_WAVES + (a.P > 64 ? a.P + 1 : 0)) * 4;
  lds += scan;
  PARSE_ALLOW_LDS(kernel, 0, lds);
  kernel<<<dim3((uint32_t)items, a.splits), AP_WAVES * 64, lds, s>>>(a);
  PARSE_LAUNCH_CHECK();
  if (a.splits > 1) {
    ap_join<T><<<dim3((uint32_t)items, AP_ROWS / AP_JOIN), AP_WAVES * 64, scan, s>>>(a);
    PARSE_LAUNCH_CHECK();
  }
  return PARSE_OK;
}
template <int DT>
static int ap_launch_bf16(const ApArgs &a, hipStream_t s) {
  return ap_launch<uint16_t>(a, attend_prefill_bf16<DT>, ap_lds_bytes(DT) + 3 * 4, s);
}
template <int DT>
static int ap_launch_f32(const ApArgs &a, hipStream_t s) {
  return ap_launch<float>(a, attend_prefill_f32<DT>, (size_t)2 * 2 * AP_TILE * DT * 32 * 4, s);
}

static int ap_bf16(const ApArgs &a, hipStream_t s) {
  switch (a.kv.d / 32) {
    case 1: return ap_launch_bf16<1>(a, s);
    case 2: return ap_launch_bf16<2>(a, s);
    case 3: return ap_launch_bf16<3>(a, s);
    case 4: return ap_launch_bf16<4>(a, s);
    case 5: return ap_launch_bf16<5>(a, s);
    case 6: return ap_launch_bf16<6>(a, s);
    case 7: return ap_launch_bf16<7>(a, s);
    default: return ap_launch_bf16<8>(a, s);
  }
}
static int ap_f32(const ApArgs &a, hipStream_t s) {
  switch (a.kv.d / 32) {
    case 1: return ap_launch_f32<1>(a, s);
    case 2: return ap_launch_f32<2>(a, s);
    case 3: return ap_launch_f32<3>(a, s);
    case 4: return ap_launch_f32<4>(a, s);
    case 5: return ap_launch_f32<5>(a, s);
    case 6: return ap_launch_f32<6>(a, s);
    case 7: return ap_launch_f32<7>(a, s);
    default: return ap_launch_f32<8>(a, s);
  }
}

}  // namespace parse

extern "C" {

size_t parse_attend_prefill_workspace_bytes(const parse_kv *kv, int32_t n_q, int32_t rows, int32_t P) {
  if (parse::check_kv(kv, false) != PARSE_OK || n_q <= 0 || n_q % kv->n_kv != 0 || rows <= 0 || P <= 0) return 0;
  return parse::ap_bytes(kv, n_q, rows, P);
}

int parse_attend_prefill(const parse_kv *kv, int32_t layer, const void *q, int64_t q_stride, int32_t n_q, int32_t rows, const int32_t *tok_offsets,
                         const int32_t *seqs, int32_t P, float scale, int32_t window, int32_t sinks, void *out, int64_t out_stride, float *lse,
                         void *workspace, size_t workspace_bytes, parse_stream stream) {
  using namespace parse;
  const int st = check_attend(kv, layer, q, q_stride, n_q, rows, tok_offsets, seqs, scale, window, sinks, out, out_stride, lse);
  if (st != PARSE_OK) return st;
  if (P <= 0) return PARSE_EINVAL;
  if ((int64_t)rows * (n_q / kv->n_kv) > KV_MAXROWS || P > KV_MAXSEQ || (!seqs && P > kv->n_seqs) || (!tok_offsets && rows != P)) return PARSE_ESHAPE;
  const size_t need = ap_bytes(kv, n_q, rows, P);
  if (need && (!workspace || workspace_bytes < need)) return PARSE_EWORKSPACE;
  if (need && !aligned16(workspace)) return PARSE_EALIGN;
  const size_t at = (size_t)layer * kv->n_pages * kv->n_kv * kv->page * kv->d * elem_size(kv->dtype);
  ApArgs a{};
  a.kv = *kv;
  a.K = (const char *)kv->K + at; a.V = (const char *)kv->V + at;
  a.q = q; a.out = out; a.lse = lse; a.tok_offsets = tok_offsets; a.seqs = seqs;
  a.q_stride = q_stride; a.out_stride = out_stride;
  a.n_q = n_q; a.group = n_q / kv->n_kv; a.rows = rows; a.P = P; a.window = window; a.sinks = sinks;
  a.by_group = kv_divisor(a.group);
  a.splits = ap_splits(kv, n_q, rows, P);
  a.part = (float *)workspace;
  at_scale(scale, a.scale, a.lag, a.q_sign);
  return kv->dtype == PARSE_BF16 ? ap_bf16(a, (hipStream_t)stream) : ap_f32(a, (hipStream_t)stream);
}

}  // extern "C"
