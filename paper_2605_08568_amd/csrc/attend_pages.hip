// Attention of one new token per sequence over listed pages of its cache (parse_attend_pages).
#include <algorithm>
#include <type_traits>

#include "attend_parts.hpp"

namespace parse {

struct AlSize {
  int TC, per_row;
  int64_t entries;
  size_t bytes;
};
static bool al_size(const parse_kv *kv, int n_q, int rows, int top, AlSize &z) {
  if (n_q <= 0 || n_q % kv->n_kv != 0 || n_q > 65536 || rows <= 0 || rows > KV_MAXSEQ || top <= 0 || (int64_t)rows * n_q > INT32_MAX) return false;
  const int group = n_q / kv->n_kv;
  z.TC = pt_columns(kv->d, kv->dtype);
  z.per_row = (group + z.TC - 1) / z.TC;
  z.entries = (int64_t)rows * z.per_row;
  const int64_t columns = (int64_t)pt_shares(kv) * z.TC + (int64_t)rows * group;
  z.bytes = pt_deal_bytes(z.entries) + round_up((size_t)columns * kv->n_kv * (kv->d + 4) * 4, 256);
  return z.entries <= INT32_MAX && z.entries * (((int64_t)top * kv->page + PT_STEP - 1) / PT_STEP) <= INT32_MAX - 65536 &&
         (int64_t)top * kv->page <= INT32_MAX && (int64_t)rows * kv->n_kv * top <= INT32_MAX;
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
  a.shares = pt_shares(kv);
  a.per_row = z.per_row;
  at_scale(scale, a.scale, a.lag, a.q_sign);
  a.pages = pages; a.top = top;
  a.deal = (int32_t *)workspace;
  a.part = (float *)((char *)workspace + pt_deal_bytes(z.entries));
  return kv->dtype == PARSE_BF16 ? pt_width<uint16_t, true>(a, z.entries, (hipStream_t)stream) : pt_width<float, true>(a, z.entries, (hipStream_t)stream);
}

}  // extern "C"
