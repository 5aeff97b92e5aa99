// Causal attention of the new tokens of a batch of prompts over the paged cache (parse_attend_prefill).
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
  int n_q, group, rows, P, tiles, window, sinks;
  float scale;                                       // times log2(e)
};

// A workgroup has NW * 32 rows of one kv head: row r of a prompt is head r % group of token r / group, so that shared
// heads read a tile of K and V once.  Tiles of TK tokens are staged in LDS as they stand in the pages.  Both products
// have the cache's side as operand A and the rows as columns: a lane holds weights of one row only, the softmax needs one
// exchange between lane halves, and what comes out of the first product is what the second takes.
template <class T, int DT, int NW, int TK>
__global__ __launch_bounds__(NW * 64) void attend_prefill(ApArgs a) {
  constexpr int D = DT * 32, KB = D / 16, TB = TK / 16, TS = TK / 32, TM = NW * 32, THREADS = NW * 64;
  constexpr int BLOCK = 16 * D * (int)sizeof(T);                   // bytes of sixteen tokens of K, and of V
  constexpr int STAGE = 2 * TB * BLOCK, PIECES = STAGE / 1024, LOADS = PIECES / NW;
  static_assert(PIECES % NW == 0, "every wavefront stages as much");
  typedef typename Op<T>::frag frag;
  extern __shared__ char smem[];
  int *wave_sums = reinterpret_cast<int *>(smem + 2 * STAGE), *pre = wave_sums + NW;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), n = lane & 31, half = lane >> 5;
  const int kvh = blockIdx.x % a.kv.n_kv, item = blockIdx.x / a.kv.n_kv, group = a.group;
  kv_prefix<THREADS>(a.P, pre, wave_sums, [&](int p) { return (int)(((int64_t)kv_rows(a.tok_offsets, p, a.rows).n * group + TM - 1) / TM); });
  if (item >= pre[a.P]) return;
  const int p = kv_find(pre, a.P, item);
  const KvRows pr = kv_rows(a.tok_offsets, p, a.rows);
  const KvSeq sq = kv_seq(a.kv, a.seqs, p);
  const int32_t *table = a.kv.table + (int64_t)sq.row * a.kv.max_pages;
  const int r0 = (pre[p + 1] - 1 - item) * TM;                     // the rows that see most come first
  const int r_end = pr.n * group, base = sq.len - pr.n;
  const int i0 = base + r0 / group, i1 = base + (min(r0 + TM, r_end) - 1) / group;
  const KvSpan span = i1 < 0 ? KvSpan{0, 0, 0} : kv_span(max(i0, 0), i1, a.window, a.sinks, TK);

  // this lane's row, and the positions of the wavefront's rows
  const int r = r0 + wave * 32 + n, token = min(r, r_end - 1) / group, head = kvh * group + (min(r, r_end - 1) - token * group);
  const int i = base + token;
  const int wi0 = base + min(r0 + wave * 32, r_end - 1) / group, wi1 = base + min(r0 + wave * 32 + 31, r_end - 1) / group;
  const int lo = kv_window_begin(i, a.window), wlo = kv_window_begin(wi0, a.window), whi = kv_window_begin(wi1, a.window);
  const bool idle = r0 + wave * 32 >= r_end;
  frag qf[KB];
  {
    const T *q = reinterpret_cast<const T *>(a.q) + (int64_t)(pr.first + token) * a.q_stride + (int64_t)head * D + 8 * half;
#pragma unroll
    for (int k = 0; k < KB; ++k) qf[k] = Op<T>::load(q + 16 * k);
  }
  float m = -INFINITY, l = 0.f;
  f32x16 o[DT];
#pragma unroll
  for (int d = 0; d < DT; ++d)
#pragma unroll
    for (int e = 0; e < 16; ++e) o[d][e] = 0.f;

  const int64_t head0 = (int64_t)kvh * a.kv.page * D, page_elems = (int64_t)a.kv.n_kv * a.kv.page * D;
  const int page_bits = 31 - __builtin_clz(a.kv.page);
  auto page_of = [&](int t) {                                      // of token t; -1 if there is none
    const int c = t >> page_bits, id = c < a.kv.max_pages ? table[c] : -1;
    return id >= 0 && id < a.kv.n_pages ? id : -1;
  };
  auto stage = [&](int t0, int buf) {
#pragma unroll
    for (int u = 0; u < LOADS; ++u) {
      const int piece = wave * LOADS + u, of_v = piece / (PIECES / 2), rest = piece % (PIECES / 2), block = rest / (BLOCK / 1024);
      const int id = max(page_of(t0 + 16 * block), 0);
      const char *src = (const char *)(of_v ? a.V : a.K) +
                        (id * page_elems + head0 + (int64_t)((t0 + 16 * block) & (a.kv.page - 1)) * D) * (int64_t)sizeof(T) + (rest % (BLOCK / 1024)) * 1024 + lane * 16;
      __builtin_amdgcn_global_load_lds(PARSE_GLB_PTR(src), PARSE_LDS_PTR(smem + buf * STAGE + piece * 1024), 16, 0, 0);
    }
  };
  // the first product's operand row n of 32 tokens: token ktok, so that a lane half gets eight consecutive tokens of each sixteen
  const int ktok = 16 * (n >> 4) + 8 * ((n >> 2) & 1) + 4 * ((n >> 3) & 1) + (n & 3);

  if (span.count > 0) stage(span.at(0) * TK, 0);
  for (int u = 0; u < span.count; ++u) {
    const int t0 = span.at(u) * TK, buf = u & 1;
    wait_vm<0>();
    __syncthreads();                                               // this tile has landed, the other buffer is read
    if (u + 1 < span.count) stage(span.at(u + 1) * TK, buf ^ 1);
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
    bool there = true;
    uint32_t blocks = 0;                                           // of sixteen tokens whose page is there
#pragma unroll
    for (int b = 0; b < TB; ++b) {
      const bool is = page_of(t0 + 16 * b) >= 0;
      blocks |= (is ? 1u : 0u) << b;
      there = there && is;
    }
    const bool whole = there && t0 + TK - 1 <= wi0 && (t0 >= whi || t0 + TK <= a.sinks);
#pragma unroll
    for (int s = 0; s < TS; ++s) sc[s] *= a.scale;
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
    if (__any(top > m + AT_LAG)) {
      const float grown = fmaxf(m, lane_max<32>(top));
      const float by = at_exp2(m - finite_or_0(grown));
      l *= by;
#pragma unroll
      for (int d = 0; d < DT; ++d) o[d] *= by;
      m = grown;
    }
    const float low = finite_or_0(m);
    frag pf[TB];
#pragma unroll
    for (int b = 0; b < TB; ++b) {
      float w[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) { w[e] = at_exp2(sc[b / 2][8 * (b % 2) + e] - low); l += w[e]; sc[b / 2][8 * (b % 2) + e] = w[e]; }
      pf[b] = Op<T>::pack(w);
    }
    bool bad = false;
#pragma unroll
    for (int b = 0; b < TB; ++b) {
      const T *vr = vs + b * 16 * D + (half * D + n) * 8;
      // tokens that some row of the wavefront sees
      uint32_t keep = 255;
      if (!whole) {
        keep = 0;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const int j = t0 + 16 * b + 8 * half + e;
          keep |= (blocks >> b & 1u & (kv_sees(wi1, wlo, a.sinks, j) ? 1u : 0u)) << e;
        }
      }
#pragma unroll
      for (int d = 0; d < DT; ++d) {
        frag vf = Op<T>::load(vr + d * 256);
        if (!whole) { vf = Op<T>::only(vf, keep); bad |= Op<T>::finite_only(vf); }
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
          for (int e = 0; e < 8; ++e)
            if (c == b && e == (j & 7)) w = sc[c / 2][8 * (c % 2) + e];
        w = __shfl(w, n + 32 * h, 64);
        if constexpr (sizeof(T) == 2) w = __uint_as_float(cvt_pk_bf16(w, 0.f) << 16);
        const bool mine = (bool)(blocks >> b & 1) & kv_sees(i, lo, a.sinks, t0 + j);
        const T *vr = vs + b * 16 * D + h * D * 8 + (j & 7);
#pragma unroll
        for (int d = 0; d < DT; ++d)
#pragma unroll
          for (int x = 0; x < 16; ++x) {
            const T v = vr[(32 * d + 8 * (x / 4) + 4 * half + x % 4) * 8];
            if (mine && !Op<T>::finite(v)) o[d][x] += w * Op<T>::value(v);
          }
      }
    }
  }
  if (idle || r >= r_end) return;
  l = lane_sum<32>(l);
  const float by = l == 0.f ? 0.f : 1.f / l;
  T *out = reinterpret_cast<T *>(a.out) + (int64_t)(pr.first + token) * a.out_stride + (int64_t)head * D;
#pragma unroll
  for (int d = 0; d < DT; ++d)
#pragma unroll
    for (int c = 0; c < 4; ++c)
      Op<T>::store4(out + 32 * d + 8 * c + 4 * half, o[d][4 * c] * by, o[d][4 * c + 1] * by, o[d][4 * c + 2] * by, o[d][4 * c + 3] * by);
  if (a.lse && half == 0) a.lse[(int64_t)(pr.first + token) * a.n_q + head] = (m + log2f(l)) * 0.6931471805599453f;
}

template <class T, int DT, int NW, int TK>
static int ap_launch(ApArgs &a, hipStream_t s) {
  // a prompt's last tile may be begun only: rows / tile + prompts in all
  const int64_t tiles = ((int64_t)a.rows * a.group) / (NW * 32) + min(a.P, a.rows);
  if (tiles * a.kv.n_kv > INT32_MAX) return PARSE_ESHAPE;
  const size_t lds = 2 * 2 * TK * DT * 32 * sizeof(T) + (NW + a.P + 1) * 4;
  PARSE_ALLOW_LDS((attend_prefill<T, DT, NW, TK>), 0, lds);
  attend_prefill<T, DT, NW, TK><<<dim3((uint32_t)(tiles * a.kv.n_kv)), NW * 64, lds, s>>>(a);
  PARSE_LAUNCH_CHECK();
  return PARSE_OK;
}
template <class T>
static int ap_width(ApArgs &a, hipStream_t s) {
  switch (a.kv.d / 32) {
    case 1: return ap_launch<T, 1, 4, 32>(a, s);
    case 2: return ap_launch<T, 2, 4, 32>(a, s);
    case 3: return ap_launch<T, 3, 4, 32>(a, s);
    case 4: return ap_launch<T, 4, 4, 32>(a, s);
    case 5: return ap_launch<T, 5, 4, 32>(a, s);
    case 6: return ap_launch<T, 6, 4, 32>(a, s);
    case 7: return ap_launch<T, 7, 4, 32>(a, s);
    default: return ap_launch<T, 8, 4, 32>(a, s);
  }
}

}  // namespace parse

extern "C" {

size_t parse_attend_prefill_workspace_bytes(const parse_kv *kv, int32_t n_q, int32_t rows, int32_t P) {
  if (parse::check_kv(kv, false) != PARSE_OK || n_q <= 0 || n_q % kv->n_kv != 0 || rows <= 0 || P <= 0) return 0;
  return 0;
}

int parse_attend_prefill(const parse_kv *kv, int32_t layer, const void *q, int64_t q_stride, int32_t n_q, int32_t rows, const int32_t *tok_offsets,
                         const int32_t *seqs, int32_t P, float scale, int32_t window, int32_t sinks, void *out, int64_t out_stride, float *lse,
                         void *workspace, size_t workspace_bytes, parse_stream stream) {
  using namespace parse;
  (void)workspace; (void)workspace_bytes;
  const int st = check_attend(kv, layer, q, q_stride, n_q, rows, tok_offsets, seqs, scale, window, sinks, out, out_stride, lse);
  if (st != PARSE_OK) return st;
  if (P <= 0) return PARSE_EINVAL;
  if ((int64_t)rows * (n_q / kv->n_kv) > KV_MAXROWS || P > KV_MAXSEQ || (!seqs && P > kv->n_seqs) || (!tok_offsets && rows != P)) return PARSE_ESHAPE;
  const size_t at = (size_t)layer * kv->n_pages * kv->n_kv * kv->page * kv->d * elem_size(kv->dtype);
  ApArgs a{};
  a.kv = *kv;
  a.K = (const char *)kv->K + at; a.V = (const char *)kv->V + at;
  a.q = q; a.out = out; a.lse = lse; a.tok_offsets = tok_offsets; a.seqs = seqs;
  a.q_stride = q_stride; a.out_stride = out_stride;
  a.n_q = n_q; a.group = n_q / kv->n_kv; a.rows = rows; a.P = P; a.window = window; a.sinks = sinks;
  a.scale = scale * 1.4426950408889634f;
  return kv->dtype == PARSE_BF16 ? ap_width<uint16_t>(a, (hipStream_t)stream) : ap_width<float>(a, (hipStream_t)stream);
}

}  // extern "C"
