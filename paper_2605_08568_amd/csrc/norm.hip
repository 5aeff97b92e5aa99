// Root-mean-square norm of rows with the residual added before (parse_rmsnorm), in the rows' type or in 8 bits with scales.
//     s = x + r,  r' = s rounded,  y = s / sqrt(mean s^2 + eps) * w;   8 bits: scale = largest |y| of a block / 448, q = y / scale rounded to e4m3
#include <algorithm>

#include "common.hpp"
#include "prefill_common.hpp"

namespace parse {

constexpr int RN_MAXD = 65536;
constexpr float RN_E4M3 = 448.f;                     // largest e4m3
constexpr float RN_LEAST = 0x1p-120f;                // smallest scale: its reciprocal and what it multiplies stay finite

struct RnArgs {
  const void *x, *residual, *weight;
  void *residual_out, *out;
  float *scales;
  int64_t x_stride, residual_stride, residual_out_stride, out_stride;   // elements
  int rows, d, block;                                // block: columns of a scale
  float eps;
};

template <class T> __device__ __forceinline__ void rn_load(const T *p, float *v);
template <> __device__ __forceinline__ void rn_load<uint16_t>(const uint16_t *p, float *v) {
  const u32x4 u = *reinterpret_cast<const u32x4 *>(p);
#pragma unroll
  for (int e = 0; e < 4; ++e) { v[2 * e] = __uint_as_float(u[e] << 16); v[2 * e + 1] = __uint_as_float(u[e] & 0xffff0000u); }
}
template <> __device__ __forceinline__ void rn_load<float>(const float *p, float *v) {
  const f32x4 a = *reinterpret_cast<const f32x4 *>(p), b = *reinterpret_cast<const f32x4 *>(p + 4);
#pragma unroll
  for (int e = 0; e < 4; ++e) { v[e] = a[e]; v[4 + e] = b[e]; }
}
__device__ __forceinline__ void rn_store(uint16_t *p, const float *v) {
  *reinterpret_cast<u32x4 *>(p) = u32x4{cvt_pk_bf16(v[0], v[1]), cvt_pk_bf16(v[2], v[3]), cvt_pk_bf16(v[4], v[5]), cvt_pk_bf16(v[6], v[7])};
}
__device__ __forceinline__ void rn_store(float *p, const float *v) {
  *reinterpret_cast<f32x4 *>(p) = f32x4{v[0], v[1], v[2], v[3]};
  *reinterpret_cast<f32x4 *>(p + 4) = f32x4{v[4], v[5], v[6], v[7]};
}
// largest magnitude that lets NaN through (fmaxf would drop it)
__device__ __forceinline__ float rn_most(float a, float b) { return a > b || a != a ? a : b; }

// LANES threads have a row, 8 * PIECES columns each in registers: x and r are read once, s is kept.  s is not rounded before the norm (r' is rounded for its store alone), squares are
// summed in 32 bits, y is rounded once: bf16 by half a step, 2^-8, e4m3 by 2^-4 of the value (the scale takes the block's largest to 448, the largest e4m3; the product with its
// rounded reciprocal is within 2^-23 of the quotient, so that a value as near to a tie may come out on its other side: one in 200000 against a quotient in 32 bits).
// Bound: reads and writes; 4096 rows of 4096 columns of bf16 with the residual 134 MB in 25 us, 5.3 TB/s (a large copy 5.1), in 8 bits with a scale every 128 columns 118 MB in 27 us, 4.3
// TB/s; one row 2.2 us, latency.
template <class T, class W, int LANES, int PIECES, bool E4M3>
__global__ __launch_bounds__(LANES < 256 ? 256 : LANES) void rmsnorm(RnArgs a) {
  constexpr int THREADS = LANES < 256 ? 256 : LANES, WAVES = LANES / 64;
  __shared__ float sums[2][THREADS / 64];
  const int tid = threadIdx.x, in = tid % LANES;
  const int row = blockIdx.x * (THREADS / LANES) + tid / LANES;
  const bool is = row < a.rows;
  const T *x = reinterpret_cast<const T *>(a.x) + (int64_t)(is ? row : 0) * a.x_stride;
  float s[PIECES][8], sq = 0.f;
#pragma unroll
  for (int k = 0; k < PIECES; ++k) {
    const int c = (k * LANES + in) * 8;
    if (is && c < a.d) {
      rn_load(x + c, s[k]);
      if (a.residual) {
        float r[8];
        rn_load(reinterpret_cast<const T *>(a.residual) + (int64_t)row * a.residual_stride + c, r);
#pragma unroll
        for (int e = 0; e < 8; ++e) s[k][e] += r[e];
      }
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e) s[k][e] = 0.f;
    }
#pragma unroll
    for (int e = 0; e < 8; ++e) sq = fmaf(s[k][e], s[k][e], sq);
  }
  sq = wave_sum(sq);
  if constexpr (WAVES > 1) {
    if ((tid & 63) == 0) sums[0][tid >> 6] = sq;
    __syncthreads();
    sq = 0.f;
#pragma unroll
    for (int w = 0; w < WAVES; ++w) sq += sums[0][w];
  }
  const float by = 1.f / sqrtf(sq / (float)a.d + a.eps);
  float most = 0.f;
#pragma unroll
  for (int k = 0; k < PIECES; ++k) {
    const int c = (k * LANES + in) * 8;
    if (is && c < a.d) {
      if (a.residual_out) rn_store(reinterpret_cast<T *>(a.residual_out) + (int64_t)row * a.residual_out_stride + c, s[k]);
      float w[8];
      rn_load(reinterpret_cast<const W *>(a.weight) + c, w);
#pragma unroll
      for (int e = 0; e < 8; ++e) s[k][e] = s[k][e] * by * w[e];
      if constexpr (!E4M3) {
        rn_store(reinterpret_cast<T *>(a.out) + (int64_t)row * a.out_stride + c, s[k]);
      } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) most = rn_most(most, fabsf(s[k][e]));
      }
    }
  }
  if constexpr (E4M3) {
    auto store = [&](int c, const float *y, float scale) {
      const float inv = 1.f / scale;
      u32x2 q;
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        int w = __builtin_amdgcn_cvt_pk_fp8_f32(y[4 * h] * inv, y[4 * h + 1] * inv, 0, false);
        q[h] = (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(y[4 * h + 2] * inv, y[4 * h + 3] * inv, w, true);
      }
      *reinterpret_cast<u32x2 *>(reinterpret_cast<uint8_t *>(a.out) + (int64_t)row * a.out_stride + c) = q;
    };
    auto scale_of = [](float m) { const float v = m / RN_E4M3; return v < RN_LEAST ? RN_LEAST : v; };
    if (a.block == a.d) {                                          // a scale a row
#pragma unroll
      for (int o = 32; o > 0; o >>= 1) most = rn_most(most, __shfl_xor(most, o, 64));
      if constexpr (WAVES > 1) {
        if ((tid & 63) == 0) sums[1][tid >> 6] = most;
        __syncthreads();
        most = 0.f;
#pragma unroll
        for (int w = 0; w < WAVES; ++w) most = rn_most(most, sums[1][w]);
      }
      const float scale = scale_of(most);
      if (is && in == 0) a.scales[row] = scale;
#pragma unroll
      for (int k = 0; k < PIECES; ++k) {
        const int c = (k * LANES + in) * 8;
        if (is && c < a.d) store(c, s[k], scale);
      }
    } else {                                                       // block / 8 consecutive lanes have a scale's columns
      const int lanes = a.block / 8;
#pragma unroll
      for (int k = 0; k < PIECES; ++k) {
        const int c = (k * LANES + in) * 8;
        float m = 0.f;
#pragma unroll
        for (int e = 0; e < 8; ++e) m = rn_most(m, fabsf(s[k][e]));
        for (int o = lanes / 2; o > 0; o >>= 1) m = rn_most(m, __shfl_xor(m, o, 64));
        const float scale = scale_of(m);
        if (is && c < a.d) {
          store(c, s[k], scale);
          if (in % lanes == 0) a.scales[(int64_t)row * (a.d / a.block) + c / a.block] = scale;
        }
      }
    }
  }
}

template <class T, class W, bool E4M3>
static int rn_piece(const RnArgs &a, hipStream_t s) {
  const int pieces = a.d / 8;
#define RN_GO(LANES, PIECES) rmsnorm<T, W, LANES, PIECES, E4M3><<<dim3((a.rows + (LANES < 256 ? 256 / LANES : 1) - 1) / (LANES < 256 ? 256 / LANES : 1)), LANES < 256 ? 256 : LANES, 0, s>>>(a)
  // Threads of a row x pieces of a thread; us for 2^24 values of bf16 with the residual, taken / the others: 1024 columns 64 x 2 26.9 / 256 x 1 27.1; 2048 256 x 1 25.0 / 64 x 4
  // 26.0; 4096 512 x 1 25.0 / 256 x 2 27.4, 64 x 8 24.1 (8 rows up to 0.6 longer); 8192 256 x 4 23.6 / 512 x 2 28.5, 1024 x 1 25.8; 16384 512 x 4 23.6 / 256 x 8 23.7 (8 rows 0.4
  // longer), 1024 x 2 27.8; 32768 1024 x 4 24.3 / 512 x 8 23.9 (8 rows 1 longer)
  if (pieces <= 64) RN_GO(64, 1);
  else if (pieces <= 128) RN_GO(64, 2);
  else if (pieces <= 256) RN_GO(256, 1);
  else if (pieces <= 512) RN_GO(512, 1);
  else if (pieces <= 1024) RN_GO(256, 4);
  else if (pieces <= 2048) RN_GO(512, 4);
  else if (pieces <= 4096) RN_GO(1024, 4);
  else RN_GO(1024, 8);
#undef RN_GO
  PARSE_LAUNCH_CHECK();
  return PARSE_OK;
}
// A launch has fewer than 2^32 threads: rows by 2^21, of which only the largest calls have more
template <class T, class W, bool E4M3>
static int rn_launch(const RnArgs &a, hipStream_t s) {
  constexpr int MOST = 1 << 21;
  for (int r0 = 0; r0 < a.rows; r0 += MOST) {
    RnArgs b = a;
    b.rows = std::min(a.rows - r0, MOST);
    b.x = (const T *)a.x + r0 * a.x_stride;
    if (a.residual) b.residual = (const T *)a.residual + r0 * a.residual_stride;
    if (a.residual_out) b.residual_out = (T *)a.residual_out + r0 * a.residual_out_stride;
    b.out = (char *)a.out + r0 * a.out_stride * (E4M3 ? 1 : (int)sizeof(T));
    if (a.scales) b.scales = a.scales + (int64_t)r0 * (a.d / a.block);
    const int st = rn_piece<T, W, E4M3>(b, s);
    if (st != PARSE_OK) return st;
  }
  return PARSE_OK;
}

}  // namespace parse

extern "C" int parse_rmsnorm(const void *x, int64_t x_stride, const void *residual, int64_t residual_stride, void *residual_out, int64_t residual_out_stride,
                             int32_t dtype, const void *weight, int32_t weight_dtype, int32_t rows, int32_t d, float eps, void *out, int64_t out_stride, float *scales,
                             int32_t block, parse_stream stream) {
  using namespace parse;
  if (!x || !weight || !out || rows <= 0 || d <= 0 || !(eps >= 0.f && eps < 1e38f)) return PARSE_EINVAL;
  if ((dtype != PARSE_F32 && dtype != PARSE_BF16) || (weight_dtype != PARSE_F32 && weight_dtype != PARSE_BF16)) return PARSE_EINVAL;
  if (scales ? block <= 0 : block != 0) return PARSE_EINVAL;
  if (d % 8 != 0 || d > RN_MAXD || rows > 1 << 30) return PARSE_ESHAPE;
  if (scales && block != d && ((block != 32 && block != 64 && block != 128 && block != 256) || d % block != 0)) return PARSE_ESHAPE;
  if (x_stride < d || out_stride < d || (residual && residual_stride < d) || (residual_out && residual_out_stride < d)) return PARSE_ESHAPE;
  const int per16 = 16 / elem_size(dtype);
  if (!aligned16(x) || !aligned16(weight) || !aligned16(residual) || !aligned16(residual_out) || x_stride % per16 != 0) return PARSE_EALIGN;
  if ((residual && residual_stride % per16 != 0) || (residual_out && residual_out_stride % per16 != 0)) return PARSE_EALIGN;
  if (scales ? (((uintptr_t)out & 7u) || out_stride % 8 != 0 || ((uintptr_t)scales & 3u)) : (!aligned16(out) || out_stride % per16 != 0)) return PARSE_EALIGN;
  const RnArgs a{x, residual, weight, residual_out, out, scales, x_stride, residual_stride, residual_out_stride, out_stride, rows, d, block, eps};
  hipStream_t s = (hipStream_t)stream;
  if (dtype == PARSE_BF16) {
    if (weight_dtype == PARSE_BF16) return scales ? rn_launch<uint16_t, uint16_t, true>(a, s) : rn_launch<uint16_t, uint16_t, false>(a, s);
    return scales ? rn_launch<uint16_t, float, true>(a, s) : rn_launch<uint16_t, float, false>(a, s);
  }
  if (weight_dtype == PARSE_BF16) return scales ? rn_launch<float, uint16_t, true>(a, s) : rn_launch<float, uint16_t, false>(a, s);
  return scales ? rn_launch<float, float, true>(a, s) : rn_launch<float, float, false>(a, s);
}
