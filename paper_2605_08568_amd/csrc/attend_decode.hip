// Attention of one new token per sequence over the paged cache (parse_attend_decode).
#include "attend.hpp"

namespace parse {

constexpr int AD_WAVES = 4, AD_THREADS = AD_WAVES * 64;
constexpr int AD_STEP = 32;                          // tokens of a wavefront's step
constexpr int AD_TILE = AD_WAVES * AD_STEP;
constexpr int AD_HEADS = 16;                         // query heads of a workgroup, the N side of the 16-wide instruction

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
};

// A workgroup has sixteen query heads of one kv head, and one share of all tokens that the batch sees.
template <class T, int DT>
__global__ __launch_bounds__(AD_THREADS) void attend_decode(AdArgs a) {
  constexpr int D = DT * 32, KB = D / 32, VB = D / 16;
  typedef typename Op<T>::frag frag;
  extern __shared__ char smem[];
  float *red = reinterpret_cast<float *>(smem);                    // [wave][head][D], [wave][head] twice
  float *red_m = red + AD_WAVES * AD_HEADS * D, *red_l = red_m + AD_WAVES * AD_HEADS;
  int *wave_sums = reinterpret_cast<int *>(red_l + AD_WAVES * AD_HEADS), *pre = wave_sums + AD_WAVES;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int n = lane & 15, quad = lane >> 4;
  const int share = blockIdx.x, kvh = blockIdx.y, hg = blockIdx.z;
  kv_prefix<AD_THREADS>(a.rows, pre, wave_sums, [&](int p) {
    const int i = kv_seq(a.kv, a.seqs, p).len - 1;
    return kv_span(i, i, a.window, a.sinks, AD_TILE).count;
  });
  const int total = pre[a.rows], per = max((total + a.shares - 1) / a.shares, 1);
  const int64_t begin = (int64_t)share * per;
  const int heads = min(a.group - hg * AD_HEADS, AD_HEADS);
  for (int e = share; e < a.rows; e += a.shares) {                 // rows that see nothing
    if (pre[e] != pre[e + 1]) continue;
    for (int v = tid; v < heads * D; v += AD_THREADS) {
      const int h = kvh * a.group + hg * AD_HEADS + v / D;
      reinterpret_cast<T *>(a.out)[(int64_t)e * a.out_stride + h * D + v % D] = 0;
      if (a.lse && v % D == 0) a.lse[(int64_t)e * a.n_q + h] = -INFINITY;
    }
  }
  if (begin >= total) return;
  const int end = (int)min(begin + per, (int64_t)total);
  const int64_t page_elems = (int64_t)a.kv.n_kv * a.kv.page * D;
  const int tok = 8 * (n >> 2) + (n & 3);                          // the first instruction's row n: tokens 8 quad + 0..3 of a step come back to a lane
  const int page_bits = 31 - __builtin_clz(a.kv.page);
  int b = kv_find(pre, a.rows, (int)begin);
  for (int at = (int)begin; at < end;) {
    const KvSeq sq = kv_seq(a.kv, a.seqs, b);
    const int pos = sq.len - 1, lo = kv_window_begin(pos, a.window);
    const KvSpan span = kv_span(pos, pos, a.window, a.sinks, AD_TILE);
    const int first = at - pre[b], last = min(end - pre[b], span.count);
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
    for (int u = first; u < last; ++u) {
      const int t0 = span.at(u) * AD_TILE + wave * AD_STEP;
      if (t0 > pos || (t0 + AD_STEP <= lo && t0 >= a.sinks)) continue;
      // the pages of the step's two blocks of sixteen tokens
      int id[2];
      bool there[2];
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        const int c = min((t0 + 16 * k) >> page_bits, a.kv.max_pages - 1);
        id[k] = table[c];
        there[k] = id[k] >= 0 && id[k] < a.kv.n_pages;
        if (!there[k]) id[k] = 0;
      }
      const int64_t head0 = (int64_t)kvh * a.kv.page * D;
      const int w0 = t0 & (a.kv.page - 1), w1 = (t0 + 16) & (a.kv.page - 1);
      const T *kp = reinterpret_cast<const T *>(a.K) + (n < 8 ? (int64_t)id[0] * page_elems + (int64_t)w0 * D : (int64_t)id[1] * page_elems + (int64_t)w1 * D) + head0 +
                    quad * 128 + (tok & 15) * 8;
      const T *vp = reinterpret_cast<const T *>(a.V) + (quad < 2 ? (int64_t)id[0] * page_elems + (int64_t)w0 * D : (int64_t)id[1] * page_elems + (int64_t)w1 * D) + head0 +
                    (quad & 1) * 8 * D + n * 8;
      frag k0[KB], k1[KB], vf[VB];
#pragma unroll
      for (int k = 0; k < KB; ++k) { k0[k] = Op<T>::load(kp + k * 512); k1[k] = Op<T>::load(kp + k * 512 + 32); }
#pragma unroll
      for (int v = 0; v < VB; ++v) vf[v] = Op<T>::load(vp + v * 128);
      f32x4 s0 = {0.f, 0.f, 0.f, 0.f}, s1 = s0;
#pragma unroll
      for (int k = 0; k < KB; ++k) { s0 = Op<T>::mma16(k0[k], qf[k], s0); s1 = Op<T>::mma16(k1[k], qf[k], s1); }
      float s[8];
#pragma unroll
      for (int e = 0; e < 4; ++e) { s[e] = s0[e]; s[4 + e] = s1[e]; }
      const bool whole = there[0] && there[1] && t0 + AD_STEP - 1 <= pos && (t0 >= lo || t0 + AD_STEP <= a.sinks);
      if (!whole) {                                                // what is not seen: no weight, and nothing of V to multiply it with
        uint32_t keep = 0;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const int j = t0 + 8 * quad + e;
          const bool sees = (quad < 2 ? there[0] : there[1]) & kv_sees(pos, lo, a.sinks, j);
          s[e] = sees ? s[e] : -INFINITY;
          keep |= (sees ? 1u : 0u) << e;
        }
#pragma unroll
        for (int v = 0; v < VB; ++v) vf[v] = Op<T>::only(vf[v], keep);
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
      const float base = finite_or_0(m) * a.scale;
      float p[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) { p[e] = at_exp2(fmaf(s[e], a.scale, -base)); l += p[e]; }
      const frag pf = Op<T>::pack(p);
#pragma unroll
      for (int v = 0; v < VB; ++v) o[v] = Op<T>::mma16(vf[v], pf, o[v]);
    }
    // the wavefronts' sums meet
    l = lane_sum<32>(lane_sum<16>(l));
    __syncthreads();
    if (lane < 16) { red_m[wave * AD_HEADS + lane] = m; red_l[wave * AD_HEADS + lane] = l; }
#pragma unroll
    for (int v = 0; v < VB; ++v) *reinterpret_cast<f32x4 *>(red + (wave * AD_HEADS + n) * D + 16 * v + 4 * quad) = o[v];
    __syncthreads();
    const bool all = first == 0 && last == span.count;
    float *part = a.part + ((((int64_t)kvh * gridDim.z + hg) * a.shares + share) * 2 + (first == 0 ? 1 : 0)) * AD_HEADS * (D + 2);
    for (int v = tid; v < heads * D; v += AD_THREADS) {
      const int h = v / D, i = v % D;
      float top = -INFINITY, ls = 0.f, os = 0.f;
#pragma unroll
      for (int w = 0; w < AD_WAVES; ++w) top = fmaxf(top, red_m[w * AD_HEADS + h]);
#pragma unroll
      for (int w = 0; w < AD_WAVES; ++w) {
        const float by = at_exp2((red_m[w * AD_HEADS + h] - finite_or_0(top)) * a.scale);
        ls += by * red_l[w * AD_HEADS + h];
        os += by * red[(w * AD_HEADS + h) * D + i];
      }
      if (all) {
        const int head = kvh * a.group + hg * AD_HEADS + h;
        const float y = ls == 0.f ? 0.f : os / ls;
        if constexpr (sizeof(T) == 2) reinterpret_cast<uint16_t *>(a.out)[(int64_t)b * a.out_stride + head * D + i] = (uint16_t)cvt_pk_bf16(y, 0.f);
        else reinterpret_cast<float *>(a.out)[(int64_t)b * a.out_stride + head * D + i] = y;
        if (a.lse && i == 0) a.lse[(int64_t)b * a.n_q + head] = (finite_or_0(top) * a.scale + log2f(ls)) * 0.6931471805599453f;
      } else {
        part[h * D + i] = os;
        if (i == 0) { part[AD_HEADS * D + h] = top; part[AD_HEADS * (D + 1) + h] = ls; }
      }
    }
    at = pre[b] + last;
    while (++b < a.rows && pre[b + 1] == at) {}
  }
}

// the parts of the rows that more than one share had
template <class T>
__global__ __launch_bounds__(AD_THREADS) void attend_join(AdArgs a) {
  extern __shared__ char smem[];
  int *wave_sums = reinterpret_cast<int *>(smem), *pre = wave_sums + AD_WAVES;
  const int D = a.kv.d, tid = threadIdx.x, b = blockIdx.x, kvh = blockIdx.y, hg = blockIdx.z;
  kv_prefix<AD_THREADS>(a.rows, pre, wave_sums, [&](int p) {
    const int i = kv_seq(a.kv, a.seqs, p).len - 1;
    return kv_span(i, i, a.window, a.sinks, AD_TILE).count;
  });
  const int total = pre[a.rows], per = max((total + a.shares - 1) / a.shares, 1);
  if (pre[b] == pre[b + 1]) return;
  const int x0 = pre[b] / per, x1 = (pre[b + 1] - 1) / per;
  if (x0 == x1) return;
  const int heads = min(a.group - hg * AD_HEADS, AD_HEADS);
  const float *parts = a.part + ((int64_t)kvh * gridDim.z + hg) * a.shares * 2 * AD_HEADS * (D + 2);
  for (int v = tid; v < heads * D; v += AD_THREADS) {
    const int h = v / D, i = v % D;
    float top = -INFINITY, ls = 0.f, os = 0.f;
    for (int x = x0; x <= x1; ++x) {
      const float *part = parts + ((int64_t)x * 2 + ((int64_t)x * per <= pre[b] ? 1 : 0)) * AD_HEADS * (D + 2);
      const float m = part[AD_HEADS * D + h], grown = fmaxf(top, m);
      const float was = at_exp2((top - finite_or_0(grown)) * a.scale), by = at_exp2((m - finite_or_0(grown)) * a.scale);
      ls = ls * was + by * part[AD_HEADS * (D + 1) + h];
      os = os * was + by * part[h * D + i];
      top = grown;
    }
    const int head = kvh * a.group + hg * AD_HEADS + h;
    const float y = ls == 0.f ? 0.f : os / ls;
    if constexpr (sizeof(T) == 2) reinterpret_cast<uint16_t *>(a.out)[(int64_t)b * a.out_stride + head * D + i] = (uint16_t)cvt_pk_bf16(y, 0.f);
    else reinterpret_cast<float *>(a.out)[(int64_t)b * a.out_stride + head * D + i] = y;
    if (a.lse && i == 0) a.lse[(int64_t)b * a.n_q + head] = (finite_or_0(top) * a.scale + log2f(ls)) * 0.6931471805599453f;
  }
}

// shares of a kv head's tokens: about four workgroups a compute unit in all
static int ad_shares(const parse_kv *kv, int n_q) {
  const int columns = kv->n_kv * ((n_q / kv->n_kv + AD_HEADS - 1) / AD_HEADS);
  return columns >= 1024 ? 1 : 1024 / columns;
}
static size_t ad_bytes(const parse_kv *kv, int n_q) {
  const int columns = kv->n_kv * ((n_q / kv->n_kv + AD_HEADS - 1) / AD_HEADS);
  return round_up((size_t)columns * ad_shares(kv, n_q) * 2 * AD_HEADS * (kv->d + 2) * 4, 256);
}

template <class T, int DT>
static int ad_launch(const AdArgs &a, hipStream_t s) {
  const int zs = (a.group + AD_HEADS - 1) / AD_HEADS;
  const size_t lds = (size_t)AD_WAVES * AD_HEADS * (DT * 32 + 2) * 4 + (AD_WAVES + a.rows + 1) * 4;
  PARSE_ALLOW_LDS((attend_decode<T, DT>), 0, lds);
  attend_decode<T, DT><<<dim3(a.shares, a.kv.n_kv, zs), AD_THREADS, lds, s>>>(a);
  PARSE_LAUNCH_CHECK();
  if (a.shares > 1) {
    attend_join<T><<<dim3(a.rows, a.kv.n_kv, zs), AD_THREADS, (AD_WAVES + a.rows + 1) * 4, s>>>(a);
    PARSE_LAUNCH_CHECK();
  }
  return PARSE_OK;
}
template <class T>
static int ad_width(const AdArgs &a, hipStream_t s) {
  switch (a.kv.d / 32) {
    case 1: return ad_launch<T, 1>(a, s);
    case 2: return ad_launch<T, 2>(a, s);
    case 3: return ad_launch<T, 3>(a, s);
    case 4: return ad_launch<T, 4>(a, s);
    case 5: return ad_launch<T, 5>(a, s);
    case 6: return ad_launch<T, 6>(a, s);
    case 7: return ad_launch<T, 7>(a, s);
    default: return ad_launch<T, 8>(a, s);
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
  if (rows > KV_MAXSEQ || (!seqs && rows > kv->n_seqs)) return PARSE_ESHAPE;
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
  a.part = (float *)workspace;
  return kv->dtype == PARSE_BF16 ? ad_width<uint16_t>(a, (hipStream_t)stream) : ad_width<float>(a, (hipStream_t)stream);
}

}  // extern "C"
