// The paged key-value cache: its bookkeeping (clear, fork, reserve, trim, compact), the copies of pages, and the rows' way in.
#include <algorithm>

#include "attend.hpp"

namespace parse {

constexpr int KV_THREADS = 256, KV_ONE = 1024;       // of a workgroup among others, of one alone
constexpr int KV_MAXFORK = 1024, KV_FORK_COLUMNS = 8;

int check_kv(const parse_kv *kv, bool counts) {
  if (!kv || !kv->K || !kv->V || !kv->table || !kv->len) return PARSE_EINVAL;
  if (kv->dtype != PARSE_F32 && kv->dtype != PARSE_BF16) return PARSE_EINVAL;
  if (kv->n_layers <= 0 || kv->n_pages <= 0 || kv->n_kv <= 0 || kv->n_seqs <= 0 || kv->max_pages <= 0) return PARSE_EINVAL;
  if (counts && (!kv->refs || !kv->free_bits)) return PARSE_EINVAL;
  if (kv->page != 16 && kv->page != 32 && kv->page != 64 && kv->page != 128 && kv->page != 256) return PARSE_ESHAPE;
  if (kv->d < 32 || kv->d > 256 || kv->d % 32 != 0 || kv->n_kv > 1024 || kv->n_seqs > KV_MAXSEQ) return PARSE_ESHAPE;
  if ((int64_t)kv->max_pages * kv->page > KV_MAXTOKENS) return PARSE_ESHAPE;
  if (!aligned16(kv->K) || !aligned16(kv->V) || !aligned4(kv->table) || !aligned4(kv->len) || !aligned4(kv->refs) || !aligned4(kv->free_bits))
    return PARSE_EALIGN;
  return PARSE_OK;
}

// One user more or less.  The thread that takes the last user away (gives the first one) turns the page's bit.
__device__ __forceinline__ void page_take(const parse_kv &kv, int id) {
  if (atomicAdd(&kv.refs[id], 1) == 0) atomicAnd(&kv.free_bits[id >> 5], ~(1u << (id & 31)));
}
__device__ __forceinline__ void page_give(const parse_kv &kv, int id) {
  if (atomicSub(&kv.refs[id], 1) == 1) atomicOr(&kv.free_bits[id >> 5], 1u << (id & 31));
}
__device__ __forceinline__ bool page_ok(const parse_kv &kv, int id) { return id >= 0 && id < kv.n_pages; }

__device__ __forceinline__ uint32_t page_bits(const parse_kv &kv, int w) { return kv.n_pages - w * 32 >= 32 ? 0xffffffffu : (1u << (kv.n_pages - w * 32)) - 1u; }
__device__ __forceinline__ uint32_t free_word(const parse_kv &kv, int w) { return kv.free_bits[w] & page_bits(kv, w); }

__global__ __launch_bounds__(KV_THREADS) void kv_clear(parse_kv kv) {
  const int64_t first = (int64_t)blockIdx.x * KV_THREADS + threadIdx.x, step = (int64_t)gridDim.x * KV_THREADS;
  for (int64_t e = first; e < (int64_t)kv.n_seqs * kv.max_pages; e += step) kv.table[e] = -1;
  for (int64_t e = first; e < kv.n_seqs; e += step) kv.len[e] = 0;
  for (int64_t e = first; e < kv.n_pages; e += step) kv.refs[e] = 0;
  for (int64_t e = first; e < (kv.n_pages + 31) / 32; e += step) kv.free_bits[e] = page_bits(kv, (int)e);
}

// Workgroup = eight columns of the table: all sources into LDS, then the destinations.  A page stands in one column only, so
// that no other workgroup counts its users; users come before users go, so that no page is free in between.
__global__ __launch_bounds__(KV_THREADS) void kv_fork(parse_kv kv, const int32_t *__restrict__ src, const int32_t *__restrict__ dst, int n) {
  extern __shared__ int moved[];                                   // [n][columns], then [n] lengths
  const int c0 = blockIdx.x * KV_FORK_COLUMNS, cols = min(KV_FORK_COLUMNS, kv.max_pages - c0);
  auto pair = [&](int i, int &s, int &d) {
    s = src[i]; d = dst[i];
    return s >= 0 && s < kv.n_seqs && d >= 0 && d < kv.n_seqs;
  };
  int s, d;
  for (int e = threadIdx.x; e < n * KV_FORK_COLUMNS; e += KV_THREADS) {
    const int i = e / KV_FORK_COLUMNS, c = e % KV_FORK_COLUMNS;
    if (c >= cols || !pair(i, s, d)) continue;
    const int id = kv.table[(int64_t)s * kv.max_pages + c0 + c];
    moved[e] = id;
    if (s != d && page_ok(kv, id)) page_take(kv, id);
    if (c == 0 && blockIdx.x == 0) moved[n * KV_FORK_COLUMNS + i] = kv.len[s];
  }
  __syncthreads();
  for (int e = threadIdx.x; e < n * KV_FORK_COLUMNS; e += KV_THREADS) {
    const int i = e / KV_FORK_COLUMNS, c = e % KV_FORK_COLUMNS;
    if (c >= cols || !pair(i, s, d)) continue;
    if (s == d) continue;
    int32_t *to = kv.table + (int64_t)d * kv.max_pages + c0 + c;
    const int old = *to;
    *to = moved[e];
    if (page_ok(kv, old)) page_give(kv, old);
    if (c == 0 && blockIdx.x == 0) kv.len[d] = moved[n * KV_FORK_COLUMNS + i];
  }
}

// Workgroup = one sequence.
__global__ __launch_bounds__(KV_THREADS) void kv_trim(parse_kv kv, const int32_t *__restrict__ keep, int window, int sinks) {
  const int s = blockIdx.x, held = kv.len[s], most = kv.max_pages * kv.page;
  const int len = min(min(max(held, 0), most), keep ? max(keep[s], 0) : most);
  __syncthreads();                                                 // everybody has read the length
  int32_t *row = kv.table + (int64_t)s * kv.max_pages;
  for (int c = threadIdx.x; c < kv.max_pages; c += KV_THREADS) {
    const int id = row[c], a = c * kv.page, b = a + kv.page;
    if (id == -1) continue;
    if (a >= len || (window > 0 && a >= sinks && b <= len - window + 1)) {
      row[c] = -1;
      if (page_ok(kv, id)) page_give(kv, id);
    }
  }
  if (threadIdx.x == 0 && len != held) kv.len[s] = len;
}

// ---- workspace of reserve and compact: number of copies, then the copies {from, to}, then a list of page ids
struct KvWork {
  int32_t *count;
  int2 *copies;                                                    // [n_pages] at most
  int32_t *ids;                                                    // [n_pages]
};
static size_t kv_work_bytes(const parse_kv *kv) { return 16 + round_up((size_t)kv->n_pages * 8, 16) + round_up((size_t)kv->n_pages * 4, 16); }
static KvWork kv_work(const parse_kv *kv, void *ws) {
  char *p = (char *)ws;
  return KvWork{(int32_t *)p, (int2 *)(p + 16), (int32_t *)(p + 16 + round_up((size_t)kv->n_pages * 8, 16))};
}

// Sums that stop at the largest int: what 4096 sequences may ask for is more (2^33 pages), and more than any pool has in either case.  A wavefront's own sums
// stay below 2^30 (four sequences a lane).
__device__ __forceinline__ int add_capped(int a, int b) { return (int)min((uint32_t)a + (uint32_t)b, 0x7fffffffu); }
// ... over the lanes up to this one of the first sixteen
__device__ __forceinline__ int scan16_capped(int v) {
  v = add_capped(v, __builtin_amdgcn_update_dpp(0, v, 0x111, 0xf, 0xf, false));  // row_shr:1
  v = add_capped(v, __builtin_amdgcn_update_dpp(0, v, 0x112, 0xf, 0xf, false));  // row_shr:2
  v = add_capped(v, __builtin_amdgcn_update_dpp(0, v, 0x114, 0xf, 0xf, false));  // row_shr:4
  return add_capped(v, __builtin_amdgcn_update_dpp(0, v, 0x118, 0xf, 0xf, false));  // row_shr:8
}

// Exclusive sums over the threads of a workgroup alone, N of them at once; `sums`: [N][wavefronts], LDS that nobody reads any more.  `mine` becomes this thread's.
template <int N>
__device__ __forceinline__ void sums_before(int (&mine)[N], int (&total)[N], int (*sums)[KV_ONE / 64]) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  int inc[N];
#pragma unroll
  for (int k = 0; k < N; ++k) {
    inc[k] = wave_scan(mine[k]);
    if (lane == 63) sums[k][wave] = inc[k];
  }
  __syncthreads();
#pragma unroll
  for (int k = 0; k < N; ++k) {
    static_assert(KV_ONE / 64 == 16, "a wavefront a lane of one row of sixteen");
    const int of_wave = scan16_capped(sums[k][lane & 15]);
    total[k] = __builtin_amdgcn_readlane(of_wave, KV_ONE / 64 - 1);
    mine[k] = add_capped(inc[k] - mine[k], wave ? __builtin_amdgcn_readlane(of_wave, wave - 1) : 0);
  }
}

// One workgroup: what a sequence gets depends on all before it, and a batch's tables are small.  A thread has PER consecutive sequences and `words` consecutive words of
// the free pages.  Bound: latency, five dependent trips to memory (7.8 us for 48 sequences and 300 pages).
template <int PER>
__global__ __launch_bounds__(KV_ONE) void kv_reserve(parse_kv kv, const int32_t *__restrict__ n_new, int32_t *__restrict__ served, const int32_t *seqs, int P,
                                                     int32_t *seqs_served, KvWork ws) {
  __shared__ int begun[PER * KV_ONE], last[PER * KV_ONE], sums[3][KV_ONE / 64], copied;
  const int tid = threadIdx.x, page = kv.page, most = kv.max_pages * page;
  const int n_words = (kv.n_pages + 31) / 32, words = (n_words + KV_ONE - 1) / KV_ONE, w0 = tid * words, w1 = min(w0 + words, n_words);
  int found = 0;
  for (int w = w0; w < w1; ++w) found += __popc(free_word(kv, w));
  if (tid == 0) copied = 0;
  // begun[s]: the page that the next token of s goes to, if it has other users; -2: there is none where one should be
  int len[PER], more[PER], need[PER], users[PER];
#pragma unroll
  for (int i = 0; i < PER; ++i) {
    const int s = tid * PER + i;
    len[i] = more[i] = need[i] = users[i] = 0;
    begun[s] = -1;
    if (s >= kv.n_seqs) continue;
    len[i] = min(max(kv.len[s], 0), most);
    more[i] = max(n_new[s], 0);
    if (more[i] > most - len[i]) more[i] = 0;
    if (more[i] > 0) {
      need[i] = (len[i] + more[i] + page - 1) / page - (len[i] + page - 1) / page;
      if (len[i] % page != 0) {
        const int id = kv.table[(int64_t)s * kv.max_pages + len[i] / page];
        if (!page_ok(kv, id)) { begun[s] = -2; need[i] += 1; }
        else if ((users[i] = kv.refs[id]) > 1) begun[s] = id;
      }
    }
  }
  __syncthreads();
  bool copy[PER];
  int part[3] = {0, found, 0}, total[3];                           // pages that are needed, free pages, copies
#pragma unroll
  for (int i = 0; i < PER; ++i) {
    const int s = tid * PER + i, id = begun[s];
    copy[i] = false;
    if (id >= 0) {                                                 // the users before it have taken their copies
      int before = 0;
      for (int e = 0; e < s; ++e) before += begun[e] == id ? 1 : 0;
      copy[i] = users[i] - before > 1;
      need[i] += copy[i] ? 1 : 0;
    }
    part[0] += need[i];
    part[2] += copy[i] ? 1 : 0;
  }
  sums_before(part, total, sums);
  const int free_pages = total[1];
  int at = part[0], rank = part[1], slot = part[2];
#pragma unroll
  for (int i = 0; i < PER; ++i) {
    at = add_capped(at, need[i]);
    last[tid * PER + i] = at;                                      // pages that the sequences up to this one take
  }
  __syncthreads();                                                 // users and begun pages are looked at no more: they may change
  auto first_over = [&](int v) {                                   // first s with last[s] > v
    int lo = 0, hi = kv.n_seqs;
    while (lo < hi) {
      const int mid = (lo + hi) >> 1;
      if (last[mid] > v) hi = mid; else lo = mid + 1;
    }
    return lo;
  };
  // taken are the pages of the sequences before the first one that does not fit: the free ones of the lowest ids
  const int fit = first_over(free_pages), taken = fit > 0 ? last[fit - 1] : 0;
  for (int w = w0; w < w1 && rank < taken; ++w) {
    const uint32_t bits = free_word(kv, w);
    uint32_t left = bits;
    while (left && rank < taken) {
      const int id = w * 32 + __builtin_ctz(left);
      left &= left - 1;
      ws.ids[rank++] = id;
      kv.refs[id] = 1;
    }
    if (left != bits) kv.free_bits[w] = left;
  }
  __syncthreads();
#pragma unroll
  for (int i = 0; i < PER; ++i) {
    const int s = tid * PER + i;
    if (s >= kv.n_seqs) continue;
    const bool ok = more[i] > 0 && s < fit;
    if (served) served[s] = ok ? 1 : 0;
    if (!ok) { begun[s] = -1; continue; }
    kv.len[s] = len[i] + more[i];
    const int id = begun[s];
    if (copy[i]) {
      ws.copies[slot++] = int2{id, ws.ids[last[s] - need[i]]};     // copies of those that fit come first
      atomicSub(&kv.refs[id], 1);                                  // one user is left at least
      atomicAdd(&copied, 1);
    }
    begun[s] = copy[i] || id == -2 ? len[i] / page : (len[i] + page - 1) / page;   // from now on: column of its first new page, -1: not served
  }
  __syncthreads();
  if (tid == 0) *ws.count = copied;
  for (int p = tid; p < P; p += KV_ONE) {
    const int s = seqs ? seqs[p] : p;
    seqs_served[p] = s >= 0 && s < kv.n_seqs && begun[s] >= 0 ? s : -1;
  }
  for (int r = tid; r < taken; r += KV_ONE) {
    const int s = first_over(r);
    kv.table[(int64_t)s * kv.max_pages + begun[s] + r - (s > 0 ? last[s - 1] : 0)] = ws.ids[r];
  }
}

// One workgroup: which pages in use move where.
__global__ __launch_bounds__(KV_ONE) void kv_compact(parse_kv kv, int32_t *__restrict__ n_live, KvWork ws) {
  __shared__ int sums[3][KV_ONE / 64];
  const int tid = threadIdx.x, n_words = (kv.n_pages + 31) / 32, words = (n_words + KV_ONE - 1) / KV_ONE;
  const int w0 = tid * words, w1 = min((tid + 1) * words, n_words);
  auto used_word = [&](int w) { return ~kv.free_bits[w] & page_bits(kv, w); };
  auto below = [&](int w, int n) { return n >= (w + 1) * 32 ? 0xffffffffu : n <= w * 32 ? 0u : (1u << (n - w * 32)) - 1u; };   // bits of the ids under n
  int used[1] = {0}, all[1], moving[2] = {0, 0}, n_moving[2];       // holes, movers: as many
  for (int w = w0; w < w1; ++w) used[0] += __popc(used_word(w));
  sums_before(used, all, sums + 2);
  const int live = all[0];
  for (int w = w0; w < w1; ++w) {
    const uint32_t under = below(w, live);
    moving[0] += __popc(free_word(kv, w) & under);
    moving[1] += __popc(used_word(w) & ~under);
  }
  sums_before(moving, n_moving, sums);
  int hole = moving[0], mover = moving[1];
  for (int w = w0; w < w1; ++w)
    for (uint32_t f = free_word(kv, w) & below(w, live); f; f &= f - 1) ws.copies[hole++].y = w * 32 + __builtin_ctz(f);
  __syncthreads();
  for (int w = w0; w < w1; ++w) {
    for (uint32_t f = used_word(w) & ~below(w, live); f; f &= f - 1) {
      const int from = w * 32 + __builtin_ctz(f), to = ws.copies[mover].y;
      ws.copies[mover++].x = from;
      ws.ids[from] = to;
      kv.refs[to] = kv.refs[from];
      kv.refs[from] = 0;
    }
  }
  for (int w = w0; w < w1; ++w) kv.free_bits[w] = page_bits(kv, w) & ~below(w, live);
  if (tid == 0) {
    *ws.count = n_moving[1];
    ws.count[1] = live;
    if (n_live) *n_live = live;
  }
}

// Copies pages of all layers, K and V, in pieces of 16 KiB; after a compaction the table's entries follow.  Bound: reads and writes (793 MB of a compaction
// in 157 us, 5.0 TB/s; a copy of 2 GiB 4.9).
template <bool REMAP>
__global__ __launch_bounds__(KV_THREADS) void kv_copy(parse_kv kv, KvWork ws, int64_t page_bytes) {
  const int n = *ws.count;
  constexpr int PIECE = KV_THREADS * 64;
  const int pieces = (int)((page_bytes + PIECE - 1) / PIECE);
  const int64_t total = (int64_t)n * kv.n_layers * 2 * pieces;
  for (int64_t t = blockIdx.x; t < total; t += gridDim.x) {
    const int piece = (int)(t % pieces);
    const int64_t side = t / pieces;
    const int of_v = (int)(side & 1), layer = (int)((side >> 1) % kv.n_layers);
    const int2 c = ws.copies[(side >> 1) / kv.n_layers];
    char *base = (char *)(of_v ? kv.V : kv.K) + (int64_t)layer * kv.n_pages * page_bytes;
    const char *from = base + c.x * page_bytes;
    char *to = base + c.y * page_bytes;
    u32x4 v[4];
    const int64_t at = (int64_t)piece * PIECE + threadIdx.x * 16;
#pragma unroll
    for (int u = 0; u < 4; ++u)
      if (at + u * KV_THREADS * 16 < page_bytes) v[u] = *reinterpret_cast<const u32x4 *>(from + at + u * KV_THREADS * 16);
#pragma unroll
    for (int u = 0; u < 4; ++u)
      if (at + u * KV_THREADS * 16 < page_bytes) *reinterpret_cast<u32x4 *>(to + at + u * KV_THREADS * 16) = v[u];
  }
  if (REMAP) {
    const int live = ws.count[1];
    const int64_t entries = (int64_t)kv.n_seqs * kv.max_pages;
    for (int64_t e = (int64_t)blockIdx.x * KV_THREADS + threadIdx.x; e < entries; e += (int64_t)gridDim.x * KV_THREADS) {
      const int id = kv.table[e];
      if (id >= live && id < kv.n_pages) kv.table[e] = ws.ids[id];
    }
  }
}

// ---------------------------------------------------------------------------------------------------------
struct KaArgs {
  parse_kv kv;
  void *K, *V;                                       // of the layer
  const void *k, *v, *q;
  void *q_out;
  int64_t k_stride, v_stride, q_stride, q_out_stride;
  const int32_t *tok_offsets, *seqs;
  const float *rope;
  int n_q, rows, P, n_pos;
};

// eight values as floats, and back with one rounding
__device__ __forceinline__ void load8(const uint16_t *p, float *f) {
  const u32x4 v = *reinterpret_cast<const u32x4 *>(p);
#pragma unroll
  for (int w = 0; w < 4; ++w) { f[2 * w] = __uint_as_float(v[w] << 16); f[2 * w + 1] = __uint_as_float(v[w] & 0xffff0000u); }
}
__device__ __forceinline__ void load8(const float *p, float *f) {
  const f32x4 a = *reinterpret_cast<const f32x4 *>(p), b = *reinterpret_cast<const f32x4 *>(p + 4);
#pragma unroll
  for (int e = 0; e < 4; ++e) { f[e] = a[e]; f[4 + e] = b[e]; }
}
__device__ __forceinline__ void store8(uint16_t *p, const float *f) { *reinterpret_cast<u32x4 *>(p) = Op<uint16_t>::pack(f); }
__device__ __forceinline__ void store8(float *p, const float *f) {
  *reinterpret_cast<f32x4 *>(p) = f32x4{f[0], f[1], f[2], f[3]};
  *reinterpret_cast<f32x4 *>(p + 4) = f32x4{f[4], f[5], f[6], f[7]};
}

// Two neighbouring columns of eight tokens, and the same as two pieces of V
__device__ __forceinline__ void turn8(const uint16_t *from, int64_t stride, uint16_t *to) {
  uint32_t x[8];
#pragma unroll
  for (int t = 0; t < 8; ++t) x[t] = *reinterpret_cast<const uint32_t *>(from + t * stride);
  u32x4 lo, hi;
#pragma unroll
  for (int w = 0; w < 4; ++w) {
    lo[w] = (x[2 * w] & 0xffffu) | (x[2 * w + 1] << 16);
    hi[w] = (x[2 * w] >> 16) | (x[2 * w + 1] & 0xffff0000u);
  }
  reinterpret_cast<u32x4 *>(to)[0] = lo;
  reinterpret_cast<u32x4 *>(to)[1] = hi;
}
__device__ __forceinline__ void turn8(const float *from, int64_t stride, float *to) {
  float lo[8], hi[8];
#pragma unroll
  for (int t = 0; t < 8; ++t) {
    const float2 x = *reinterpret_cast<const float2 *>(from + t * stride);
    lo[t] = x.x; hi[t] = x.y;
  }
  store8(to, lo);
  store8(to + 8, hi);
}

// Workgroup (x, y) = one block of sixteen positions of a prompt, some of its heads.  A thread has one token's 8 columns and their 8 partners, whose angles it reads
// once, head after head (of K token fastest: the pieces of a column block are contiguous in the page); of V two columns of eight tokens, transposed
// in registers, or 8 columns of one token where not all eight are new.
// Bound: reads and writes of large batches (8 x 512 rows of 96 heads of 128, 201 MB in 50 us, 4.0 TB/s: rows are read in lines that stand 24 KB apart), latency of single
// rows (6.4 us for 32 of them).  Stores past the caches were 3 us faster at 8 x 512 and not taken: the attention reads these rows next.
template <class T>
__global__ __launch_bounds__(KV_THREADS) void kv_append(KaArgs a) {
  extern __shared__ int smem[];
  int *wave_sums = smem, *pre = smem + KV_THREADS / 64;
  const int D = a.kv.d, half = D / 2, pairs = D / 16, tid = threadIdx.x;     // pairs of pieces in a row
  for (int item = blockIdx.x;; item += gridDim.x) {
    const KvItem f = kv_item<KV_THREADS>(a.kv, a.tok_offsets, a.seqs, a.P, a.rows, item, pre, wave_sums,
                                         [&](const KvRows &r, const KvSeq &s) { return r.n == 0 ? 0 : ((s.len + 15) >> 4) - ((s.len - r.n) >> 4); });
    if (f.item < 0) return;
    const int base = f.len - f.n, block = (base >> 4) + f.item;     // positions 16 block + 0..15; before 0: rows without a place in the cache
    const int from = max(block * 16, base), tokens = min(block * 16 + 16, f.len) - from, row0 = f.first + from - base;
    const int c = block >> (27 - __builtin_clz(a.kv.page));        // 16 block / page
    const int id = block >= 0 && c < a.kv.max_pages ? a.kv.table[(int64_t)f.row * a.kv.max_pages + c] : -1;
    const bool there = page_ok(a.kv, id);
    // where the block stands for head 0; heads are page * D apart
    const int64_t spot = there ? (int64_t)id * a.kv.n_kv * a.kv.page * D + (int64_t)((block * 16) & (a.kv.page - 1)) * D : 0, step = (int64_t)a.kv.page * D;
    const int w0 = from & 15;                                      // first token's place in the block
    const int per = tokens * pairs, at_once = KV_THREADS / per, sub = tid / per, in = tid - sub * per;   // per <= 256
    auto angles = [&](int tok, int piece, float *cs, float *sn) {
      const float *t = a.rope + (int64_t)min(max(from + tok, 0), a.n_pos - 1) * D + 8 * piece;
      load8(t, cs);
      load8(t + half, sn);
    };
    auto turn = [&](const float *cs, const float *sn, float *lo, float *hi) {
      if (!a.rope) return;
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const float x = lo[e], y = hi[e];
        lo[e] = x * cs[e] - y * sn[e];
        hi[e] = y * cs[e] + x * sn[e];
      }
    };
    // two heads of a thread on their way; where they go, a head's columns and their partners are to_gap apart
    auto heads = [&](const T *src, T *to, int n, int64_t to_head, int to_gap, int y, const float *cs, const float *sn) {
      const int next = gridDim.y * at_once;
      for (int h = y * at_once + sub; h < n; h += 2 * next) {
        float lo[2][8], hi[2][8];
        const bool two = h + next < n;
        load8(src + (int64_t)h * D, lo[0]);
        load8(src + (int64_t)h * D + half, hi[0]);
        if (two) {
          load8(src + (int64_t)(h + next) * D, lo[1]);
          load8(src + (int64_t)(h + next) * D + half, hi[1]);
        }
        turn(cs, sn, lo[0], hi[0]);
        store8(to + h * to_head, lo[0]);
        store8(to + h * to_head + to_gap, hi[0]);
        if (two) {
          turn(cs, sn, lo[1], hi[1]);
          store8(to + (h + next) * to_head, lo[1]);
          store8(to + (h + next) * to_head + to_gap, hi[1]);
        }
      }
    };
    float cs[8], sn[8];
    if (there && sub < at_once) {
      const int piece = in / tokens, tok = in - piece * tokens;
      if (a.rope) angles(tok, piece, cs, sn);
      heads((const T *)a.k + (row0 + tok) * a.k_stride + 8 * piece, (T *)a.K + spot + piece * 128 + (w0 + tok) * 8, a.kv.n_kv, step, half * 16, blockIdx.y, cs, sn);
    }
    if (a.q && sub < at_once) {
      const int tok = in / pairs, piece = in - tok * pairs;
      if (a.rope) angles(tok, piece, cs, sn);
      heads((const T *)a.q + (row0 + tok) * a.q_stride + 8 * piece, (T *)a.q_out + (row0 + tok) * a.q_out_stride + 8 * piece, a.n_q, D, half, gridDim.y - 1 - blockIdx.y, cs, sn);
    }
    if (there) {
      const bool left = w0 == 0 && tokens >= 8, right = w0 <= 8 && w0 + tokens == 16;   // all eight of a half are new
      const int halves = (left ? 1 : 0) + (right ? 1 : 0), loose = tokens - 8 * halves;
      const int turns = halves * half, all = turns + loose * (D / 8);                   // work of a head
      for (int w = blockIdx.y * KV_THREADS + tid; w < all * a.kv.n_kv; w += gridDim.y * KV_THREADS) {
        const int h = w / all, u = w - h * all;
        if (u < turns) {
          const int side = halves == 2 ? (u >= half ? 1 : 0) : left ? 0 : 1, i = 2 * (u >= half ? u - half : u);
          turn8((const T *)a.v + (row0 + side * 8 - w0) * a.v_stride + (int64_t)h * D + i, a.v_stride, (T *)a.V + spot + h * step + (side * D + i) * 8);
        } else {
          const int v = u - turns, t = v / (D / 8), piece = v - t * (D / 8), tok = t + (left ? 8 : 0);
          const T *src = (const T *)a.v + (row0 + tok) * a.v_stride + (int64_t)h * D + piece * 8;
          T *to = (T *)a.V + spot + h * step + ((w0 + tok) / 8 * D + piece * 8) * 8 + (w0 + tok) % 8;
          T x[8];
          *reinterpret_cast<u32x4 *>(x) = *reinterpret_cast<const u32x4 *>(src);
          if constexpr (sizeof(T) == 4) reinterpret_cast<u32x4 *>(x)[1] = reinterpret_cast<const u32x4 *>(src)[1];
#pragma unroll
          for (int e = 0; e < 8; ++e) to[e * 8] = x[e];
        }
      }
    }
    if (a.P > 64) __syncthreads();                                 // the prompts' sums are made anew
  }
}

}  // namespace parse

extern "C" {

using namespace parse;

int parse_kv_clear(const parse_kv *kv, parse_stream stream) {
  const int st = check_kv(kv, true);
  if (st != PARSE_OK) return st;
  const int64_t most = std::max((int64_t)kv->n_seqs * kv->max_pages, (int64_t)kv->n_pages);
  kv_clear<<<dim3((uint32_t)std::min<int64_t>((most + KV_THREADS - 1) / KV_THREADS, 2048)), KV_THREADS, 0, (hipStream_t)stream>>>(*kv);
  PARSE_LAUNCH_CHECK();
  return PARSE_OK;
}

int parse_kv_fork(const parse_kv *kv, const int32_t *src, const int32_t *dst, int32_t n, parse_stream stream) {
  const int st = check_kv(kv, true);
  if (st != PARSE_OK) return st;
  if (!src || !dst || n <= 0) return PARSE_EINVAL;
  if (n > KV_MAXFORK) return PARSE_ESHAPE;
  if (!aligned4(src) || !aligned4(dst)) return PARSE_EALIGN;
  kv_fork<<<dim3((kv->max_pages + KV_FORK_COLUMNS - 1) / KV_FORK_COLUMNS), KV_THREADS, (size_t)n * (KV_FORK_COLUMNS + 1) * 4, (hipStream_t)stream>>>(*kv, src, dst, n);
  PARSE_LAUNCH_CHECK();
  return PARSE_OK;
}

int parse_kv_trim(const parse_kv *kv, const int32_t *keep, int32_t window, int32_t sinks, parse_stream stream) {
  const int st = check_kv(kv, true);
  if (st != PARSE_OK) return st;
  if (window < 0 || sinks < 0 || (!keep && window == 0)) return PARSE_EINVAL;
  if (!aligned4(keep)) return PARSE_EALIGN;
  kv_trim<<<dim3(kv->n_seqs), KV_THREADS, 0, (hipStream_t)stream>>>(*kv, keep, window, sinks);
  PARSE_LAUNCH_CHECK();
  return PARSE_OK;
}

size_t parse_kv_workspace_bytes(const parse_kv *kv) { return check_kv(kv, false) == PARSE_OK ? kv_work_bytes(kv) : 0; }

static int64_t kv_page_bytes(const parse_kv *kv) { return (int64_t)kv->n_kv * kv->page * kv->d * elem_size(kv->dtype); }

static int kv_reserve_call(const parse_kv *kv, const int32_t *n_new, int32_t *served, const int32_t *seqs, int32_t P, int32_t *seqs_served, void *workspace,
                           size_t workspace_bytes, parse_stream stream) {
  if (!workspace || workspace_bytes < kv_work_bytes(kv)) return PARSE_EWORKSPACE;
  if (!aligned4(n_new) || !aligned4(served) || !aligned16(workspace)) return PARSE_EALIGN;
  const KvWork ws = kv_work(kv, workspace);
  if (kv->n_seqs <= KV_ONE) kv_reserve<1><<<dim3(1), KV_ONE, 0, (hipStream_t)stream>>>(*kv, n_new, served, seqs, P, seqs_served, ws);
  else kv_reserve<KV_MAXSEQ / KV_ONE><<<dim3(1), KV_ONE, 0, (hipStream_t)stream>>>(*kv, n_new, served, seqs, P, seqs_served, ws);
  PARSE_LAUNCH_CHECK();
  kv_copy<false><<<dim3(2048), KV_THREADS, 0, (hipStream_t)stream>>>(*kv, ws, kv_page_bytes(kv));
  PARSE_LAUNCH_CHECK();
  return PARSE_OK;
}

int parse_kv_reserve(const parse_kv *kv, const int32_t *n_new, int32_t *served, void *workspace, size_t workspace_bytes, parse_stream stream) {
  const int st = check_kv(kv, true);
  if (st != PARSE_OK) return st;
  if (!n_new) return PARSE_EINVAL;
  return kv_reserve_call(kv, n_new, served, nullptr, 0, nullptr, workspace, workspace_bytes, stream);
}

int parse_kv_reserve_seqs(const parse_kv *kv, const int32_t *n_new, int32_t *served, const int32_t *seqs, int32_t P, int32_t *seqs_served, void *workspace,
                          size_t workspace_bytes, parse_stream stream) {
  const int st = check_kv(kv, true);
  if (st != PARSE_OK) return st;
  if (!n_new || !seqs_served || P <= 0) return PARSE_EINVAL;
  if (P > KV_MAXSEQ || (!seqs && P > kv->n_seqs)) return PARSE_ESHAPE;
  if (!aligned4(seqs) || !aligned4(seqs_served)) return PARSE_EALIGN;
  return kv_reserve_call(kv, n_new, served, seqs, P, seqs_served, workspace, workspace_bytes, stream);
}

int parse_kv_compact(const parse_kv *kv, int32_t *n_live, void *workspace, size_t workspace_bytes, parse_stream stream) {
  const int st = check_kv(kv, true);
  if (st != PARSE_OK) return st;
  if (!workspace || workspace_bytes < kv_work_bytes(kv)) return PARSE_EWORKSPACE;
  if (!aligned16(workspace) || !aligned4(n_live)) return PARSE_EALIGN;
  const KvWork ws = kv_work(kv, workspace);
  kv_compact<<<dim3(1), KV_ONE, 0, (hipStream_t)stream>>>(*kv, n_live, ws);
  PARSE_LAUNCH_CHECK();
  kv_copy<true><<<dim3(2048), KV_THREADS, 0, (hipStream_t)stream>>>(*kv, ws, kv_page_bytes(kv));
  PARSE_LAUNCH_CHECK();
  return PARSE_OK;
}

int parse_kv_append(const parse_kv *kv, int32_t layer, const void *k, int64_t k_stride, const void *v, int64_t v_stride, const void *q, int64_t q_stride,
                    void *q_out, int64_t q_out_stride, int32_t n_q, int32_t rows, const int32_t *tok_offsets, const int32_t *seqs, int32_t P,
                    const float *rope, int32_t n_pos, parse_stream stream) {
  const int st = check_kv(kv, false);
  if (st != PARSE_OK) return st;
  if (!k || !v || rows <= 0 || P <= 0 || layer < 0 || (!q != !q_out) || (q && n_q <= 0) || (rope && n_pos <= 0)) return PARSE_EINVAL;
  if (layer >= kv->n_layers || P > KV_MAXSEQ || rows > KV_MAXROWS || (!seqs && P > kv->n_seqs) || (!tok_offsets && rows != P)) return PARSE_ESHAPE;
  const int64_t width = (int64_t)kv->n_kv * kv->d;
  if (k_stride < width || v_stride < width) return PARSE_ESHAPE;
  if (q && (n_q > 65536 || q_stride < (int64_t)n_q * kv->d || q_out_stride < (int64_t)n_q * kv->d)) return PARSE_ESHAPE;
  const int per16 = 16 / elem_size(kv->dtype);
  if (!aligned16(k) || !aligned16(v) || !aligned16(q) || !aligned16(q_out) || !aligned16(rope) || k_stride % per16 != 0 || v_stride % per16 != 0)
    return PARSE_EALIGN;
  if (!aligned4(tok_offsets) || !aligned4(seqs)) return PARSE_EALIGN;
  if (q && (q_stride % per16 != 0 || q_out_stride % per16 != 0)) return PARSE_EALIGN;
  const size_t at = (size_t)layer * kv->n_pages * kv_page_bytes(kv);
  KaArgs a{*kv, (char *)kv->K + at, (char *)kv->V + at, k, v, q, q_out, k_stride, v_stride, q_stride, q_out_stride, tok_offsets, seqs, rope, n_q, rows, P, n_pos};
  // a prompt's first and last block may be begun only, and every block has a row.  About 4096 workgroups, all with as many heads (of blocks with as many rows as
  // they have on average)
  const int64_t blocks = std::min<int64_t>(rows / 16 + 2 * (int64_t)std::min(P, rows), rows);
  const int per = (int)std::min<int64_t>((rows + blocks - 1) / blocks, 16) * (kv->d / 16), at_once = KV_THREADS / per;
  const int most = (int)std::max<int64_t>(1, 4096 / blocks), turns = (kv->n_kv + at_once * most - 1) / (at_once * most);
  // ... four of a block at least where there is room: one has the heads of k, another those of q, all of them v
  const dim3 grid((uint32_t)std::min<int64_t>(blocks, 65536), (uint32_t)std::max((kv->n_kv + at_once * turns - 1) / (at_once * turns), std::min(most, 4)));
  const size_t lds = P > 64 ? (KV_THREADS / 64 + P + 1) * 4 : 0;
  if (kv->dtype == PARSE_BF16) kv_append<uint16_t><<<grid, KV_THREADS, lds, (hipStream_t)stream>>>(a);
  else kv_append<float><<<grid, KV_THREADS, lds, (hipStream_t)stream>>>(a);
  PARSE_LAUNCH_CHECK();
  return PARSE_OK;
}

}  // extern "C"
