// Attention of one new token per sequence over listed pages of its cache (parse_attend_pages).
#include <algorithm>
#include <type_traits>

#include "attend_parts.hpp"

namespace parse {

// Columns of an entry: sixteen, unless a kv head has more query heads
static int al_columns(const parse_kv *kv, int n_q) { return n_q / kv->n_kv <= 16 ? 16 : pt_columns(kv->d, kv->dtype); }
static int al_shares(const parse_kv *kv, int n_q) { return pt_shares(kv->n_kv, al_columns(kv, n_q) == 16 ? 512 : 256); }

template <class T, int DT>
static int al_go(const PtArgs &a, int TC, int64_t entries, hipStream_t s) {
  if constexpr (pt_blocks<T, DT>() > 1)
    if (TC > 16) return pt_launch<T, DT, pt_blocks<T, DT>(), true>(a, entries, s);
  return pt_launch<T, DT, 1, true>(a, entries, s);
}
template <class T>
static int al_width(const PtArgs &a, int TC, int64_t entries, hipStream_t s) {
  switch (a.kv.d / 32) {
    case 1: return al_go<T, 1>(a, TC, entries, s);
    case 2: return al_go<T, 2>(a, TC, entries, s);
    case 3: return al_go<T, 3>(a, TC, entries, s);
    case 4: return al_go<T, 4>(a, TC, entries, s);
    case 5: return al_go<T, 5>(a, TC, entries, s);
    case 6: return al_go<T, 6>(a, TC, entries, s);
    case 7: return al_go<T, 7>(a, TC, entries, s);
    default: return al_go<T, 8>(a, TC, entries, s);
  }
}

struct AlSize {
  int TC, per_row;
  int64_t entries;
  size_t bytes;
};
static bool al_size(const parse_kv *kv, int n_q, int rows, int top, AlSize &z) {
  if (n_q <= 0 || n_q % kv->n_kv != 0 || n_q > 65536 || rows <= 0 || rows > KV_MAXSEQ || top <= 0 || (int64_t)rows * n_q > INT32_MAX) return false;
  const int group = n_q / kv->n_kv;
  z.TC = al_columns(kv, n_q);
  z.per_row = (group + z.TC - 1) / z.TC;
  z.entries = (int64_t)rows * z.per_row;
  const int64_t columns = (int64_t)al_shares(kv, n_q) * z.TC + (int64_t)rows * group;
  z.bytes = pt_deal_bytes(z.entries) + round_up((size_t)columns * kv->n_kv * (kv->d + 4) * 4, 256);
  return z.entries <= INT32_MAX && z.entries * (((int64_t)top * kv->page + PT_STEP - 1) / PT_STEP) <= INT32_MAX - 65536 &&
         (int64_t)rows * kv->n_kv * top <= INT32_MAX;
}

}  // namespace parse

extern "C" {

using namespace parse;

size_t parse_attend_pages_workspace_bytes(const parse_kv *kv, int32_t n_q, int32_t rows, int32_t top) {
  AlSize z;
  return check_kv(kv, false) == PARSE_OK && al_size(kv, n_q, rows, top, z) ? z.bytes : 0;
}

int parse_attend_pages(const parse_kv *kv, int32_t layer, const void *q, int64_t q_stride, int32_t n_q, int32_t rows, const int32_t *seqs, const int32_t *pages,
                       int32_t top, float scale, void *out, int64_t out_stride, float *lse, void *workspace, size_t workspace_bytes, parse_stream stream) {
  const int st = check_attend(kv, layer, q, q_stride, n_q, rows, nullptr, seqs, scale, 0, 0, out, out_stride, lse);
  if (st != PARSE_OK) return st;
  if (!pages || top <= 0) return PARSE_EINVAL;
  AlSize z;
  if (!al_size(kv, n_q, rows, top, z) || (!seqs && rows > kv->n_seqs)) return PARSE_ESHAPE;
  if (!aligned4(pages)) return PARSE_EALIGN;
  if (!workspace || workspace_bytes < z.bytes) return PARSE_EWORKSPACE;
  if (!aligned16(workspace)) return PARSE_EALIGN;
  const size_t at = (size_t)layer * kv->n_pages * kv->n_kv * kv->page * kv->d * elem_size(kv->dtype);
  PtArgs a{};
  a.kv = *kv;
  a.K = (const char *)kv->K + at; a.V = (const char *)kv->V + at;
  a.q = q; a.out = out; a.lse = lse; a.seqs = seqs;
  a.q_stride = q_stride; a.out_stride = out_stride;
  a.n_q = n_q; a.group = n_q / kv->n_kv; a.rows = rows;
  a.shares = al_shares(kv, n_q);
  a.per_row = z.per_row;
  at_scale(scale, a.scale, a.lag, a.q_sign);
  a.pages = pages; a.top = top;
  a.deal = (int32_t *)workspace;
  a.part = (float *)((char *)workspace + pt_deal_bytes(z.entries));
  return kv->dtype == PARSE_BF16 ? al_width<uint16_t>(a, z.TC, z.entries, (hipStream_t)stream) : al_width<float>(a, z.TC, z.entries, (hipStream_t)stream);
}

}  // extern "C"
