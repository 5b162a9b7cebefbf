// symi_norm_fwd / symi_norm_bwd: layer norm and RMS norm of rows behind a residual sum, and their gradients.
//
// mean = sum R / d, rstd = 1 / sqrt(sum (R - mean)^2 / d + eps), Y = (R - mean) rstd w + b;
// with xh = (R - mean) rstd and g = dY w: dX = rstd (g - sum g / d - xh sum(g xh) / d) + dR, dw = sum dY xh, db = sum dY.
#include <math.h>

#include <algorithm>
#include <type_traits>

#include "common.h"

namespace symi {

constexpr int NORM_THREADS = 256;
constexpr int NORM_CHUNKS = 512;   // partial sums of dw and db at most

// 8 consecutive values of a row, in registers as fp32.
template <bool BF16>
__device__ __forceinline__ void load8(const void* p, long long at, float (&x)[8]) {
  if constexpr (BF16) {
    const u32x4_bf16 r = *reinterpret_cast<const u32x4_bf16*>(static_cast<const uint16_t*>(p) + at);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      x[2 * i] = __uint_as_float(r[i] << 16);
      x[2 * i + 1] = __uint_as_float(r[i] & 0xffff0000u);
    }
  } else {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const f32x4_f32 r = *reinterpret_cast<const f32x4_f32*>(static_cast<const float*>(p) + at + 4 * h);
#pragma unroll
      for (int i = 0; i < 4; ++i) x[4 * h + i] = r[i];
    }
  }
}
template <bool BF16>
__device__ __forceinline__ void store8(void* p, long long at, const float (&x)[8]) {
  if constexpr (BF16) {
    u32x4_bf16 r;
#pragma unroll
    for (int i = 0; i < 4; ++i) r[i] = pack_bf16x2(x[2 * i], x[2 * i + 1]);
    *reinterpret_cast<u32x4_bf16*>(static_cast<uint16_t*>(p) + at) = r;
  } else {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const f32x4_f32 r = {x[4 * h], x[4 * h + 1], x[4 * h + 2], x[4 * h + 3]};
      *reinterpret_cast<f32x4_f32*>(static_cast<float*>(p) + at + 4 * h) = r;
    }
  }
}
template <bool BF16>
__device__ __forceinline__ float as_stored(float x) {
  if constexpr (BF16) return bf16_to_f32(f32_to_bf16(x)); else return x;
}

// Sum over a workgroup, in the same order always; every thread gets it.
__device__ __forceinline__ float block_sum(float x, float* part) {
#pragma unroll
  for (int m = 32; m >= 1; m >>= 1) x += __shfl_xor(x, m, 64);
  __syncthreads();
  if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = x;
  __syncthreads();
  float s = 0.f;
  for (int w = 0; w < (int)blockDim.x / 64; ++w) s += part[w];
  return s;
}

// One workgroup a row; a thread reads back what it wrote itself.
template <bool BF16>
__global__ __launch_bounds__(NORM_THREADS) void norm_kernel(const void* X, const void* res, const float* __restrict__ w,
                                                            const float* __restrict__ b, void* R, void* Y, float* __restrict__ mean_out,
                                                            float* __restrict__ rstd_out, int d, int center, float eps) {
  __shared__ float part[NORM_THREADS / 64];
  const long long row = (long long)blockIdx.x * d;
  float s = 0.f;
  for (int c = threadIdx.x * 8; c < d; c += NORM_THREADS * 8) {
    float x[8];
    load8<BF16>(X, row + c, x);
    if (res) {
      float y[8];
      load8<BF16>(res, row + c, y);
#pragma unroll
      for (int i = 0; i < 8; ++i) x[i] = as_stored<BF16>(x[i] + y[i]);
      store8<BF16>(R, row + c, x);
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) s += x[i];
  }
  const void* const from = res ? R : X;
  const float mean = center ? block_sum(s, part) / (float)d : 0.f;
  float q = 0.f;
  for (int c = threadIdx.x * 8; c < d; c += NORM_THREADS * 8) {
    float x[8];
    load8<BF16>(from, row + c, x);
#pragma unroll
    for (int i = 0; i < 8; ++i) q += (x[i] - mean) * (x[i] - mean);
  }
  const float rstd = 1.f / sqrtf(block_sum(q, part) / (float)d + eps);
  for (int c = threadIdx.x * 8; c < d; c += NORM_THREADS * 8) {
    float x[8];
    load8<BF16>(from, row + c, x);
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = (x[i] - mean) * rstd * (w ? w[c + i] : 1.f) + (b ? b[c + i] : 0.f);
    store8<BF16>(Y, row + c, x);
  }
  if (threadIdx.x == 0) {
    if (mean_out) mean_out[blockIdx.x] = mean;
    if (rstd_out) rstd_out[blockIdx.x] = rstd;
  }
}

template <bool BF16>
__global__ __launch_bounds__(NORM_THREADS) void norm_bwd_kernel(const void* dY, const void* R, const float* __restrict__ mean_in,
                                                                const float* __restrict__ rstd_in, const float* __restrict__ w, const void* dR,
                                                                void* dX, int d, int center) {
  __shared__ float part[NORM_THREADS / 64];
  const long long row = (long long)blockIdx.x * d;
  const float mean = center ? mean_in[blockIdx.x] : 0.f, rstd = rstd_in[blockIdx.x];
  float level = 0.f, along = 0.f;
  for (int c = threadIdx.x * 8; c < d; c += NORM_THREADS * 8) {
    float g[8], x[8];
    load8<BF16>(dY, row + c, g);
    load8<BF16>(R, row + c, x);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const float gi = g[i] * (w ? w[c + i] : 1.f);
      level += gi;
      along += gi * ((x[i] - mean) * rstd);
    }
  }
  level = center ? block_sum(level, part) / (float)d : 0.f;
  along = block_sum(along, part) / (float)d;
  for (int c = threadIdx.x * 8; c < d; c += NORM_THREADS * 8) {
    float g[8], x[8], r[8] = {};
    load8<BF16>(dY, row + c, g);
    load8<BF16>(R, row + c, x);
    if (dR) load8<BF16>(dR, row + c, r);
#pragma unroll
    for (int i = 0; i < 8; ++i)
      x[i] = (g[i] * (w ? w[c + i] : 1.f) - level - (x[i] - mean) * rstd * along) * rstd + r[i];
    store8<BF16>(dX, row + c, x);
  }
}

// Sums over a chunk of rows; a thread has 8 columns.
template <bool BF16>
__global__ __launch_bounds__(NORM_THREADS) void norm_columns_kernel(const void* dY, const void* R, const float* __restrict__ mean_in,
                                                                    const float* __restrict__ rstd_in, float* __restrict__ part, int T, int d,
                                                                    int center, int chunk, int want_w, int want_b) {
  const int c = (blockIdx.x * NORM_THREADS + threadIdx.x) * 8;
  if (c >= d) return;
  const int t0 = blockIdx.y * chunk, t1 = min(T, t0 + chunk);
  float sw[8] = {}, sb[8] = {};
  for (int t = t0; t < t1; ++t) {
    const float mean = center ? mean_in[t] : 0.f, rstd = rstd_in[t];
    float g[8], x[8];
    load8<BF16>(dY, (long long)t * d + c, g);
    load8<BF16>(R, (long long)t * d + c, x);
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      sw[i] += g[i] * ((x[i] - mean) * rstd);
      sb[i] += g[i];
    }
  }
  float* const to = part + (long long)blockIdx.y * 2 * d + c;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    if (want_w) to[i] = sw[i];
    if (want_b) to[d + i] = sb[i];
  }
}

__global__ __launch_bounds__(NORM_THREADS) void norm_sum_kernel(const float* __restrict__ part, float* __restrict__ dw, float* __restrict__ db,
                                                                int chunks, int d) {
  const int c = blockIdx.x * NORM_THREADS + threadIdx.x;
  if (c >= d) return;
  float sw = 0.f, sb = 0.f;
  for (int k = 0; k < chunks; ++k) {
    if (dw) sw += part[(long long)k * 2 * d + c];
    if (db) sb += part[(long long)k * 2 * d + d + c];
  }
  if (dw) dw[c] = sw;
  if (db) db[c] = sb;
}

// Rows per partial sum: what T and d decide.
static int norm_chunk(const symi_cfg* c) { return std::max(1, cdiv(c->T, NORM_CHUNKS)); }

}  // namespace symi

using namespace symi;

extern "C" size_t symi_norm_workspace_bytes(const symi_cfg* cfg) {
  if (check_cfg(cfg, "symi_norm_workspace_bytes") != SYMI_OK) return 0;
  return align_up((size_t)cdiv(cfg->T, norm_chunk(cfg)) * 2 * cfg->d * sizeof(float), 256) + 256;
}

extern "C" int symi_norm_fwd(const symi_ctx* ctx, int center, float eps, const void* X, const void* residual, const float* w,
                             const float* b, void* R, void* Y, float* mean, float* rstd, void* stream) {
  SYMI_ENTER(ctx, "symi_norm_fwd");
  SYMI_REQUIRE(center == 0 || center == 1, "symi_norm_fwd", "center must be 0 or 1");
  SYMI_REQUIRE(eps >= 0.f && eps < INFINITY, "symi_norm_fwd", "eps must be finite and not negative");
  SYMI_REQUIRE((residual != nullptr) == (R != nullptr), "symi_norm_fwd", "R goes with residual: both or neither");
  if (cfg->T == 0) return SYMI_OK;
  SYMI_REQUIRE(X && Y, "symi_norm_fwd", "NULL pointer");
  hipStream_t st = as_stream(stream);
  if (cfg->dtype == SYMI_BF16)
    SYMI_TIMED(ctx, K_NORM, st, (norm_kernel<true><<<cfg->T, NORM_THREADS, 0, st>>>(X, residual, w, b, R, Y, mean, rstd, cfg->d, center, eps)));
  else
    SYMI_TIMED(ctx, K_NORM, st, (norm_kernel<false><<<cfg->T, NORM_THREADS, 0, st>>>(X, residual, w, b, R, Y, mean, rstd, cfg->d, center, eps)));
  SYMI_LAUNCH_CHECK("symi_norm_fwd");
  return SYMI_OK;
}

extern "C" int symi_norm_bwd(const symi_ctx* ctx, int center, const void* dY, const void* R, const float* mean, const float* rstd,
                             const float* w, const void* dR, void* dX, float* dw, float* db, void* ws, void* stream) {
  SYMI_ENTER(ctx, "symi_norm_bwd");
  SYMI_REQUIRE(center == 0 || center == 1, "symi_norm_bwd", "center must be 0 or 1");
  const int T = cfg->T, d = cfg->d;
  SYMI_REQUIRE(T == 0 || (dY && R && rstd && dX && (mean || !center)), "symi_norm_bwd", "NULL pointer");
  SYMI_REQUIRE(ws || !(dw || db), "symi_norm_bwd", "NULL workspace");
  hipStream_t st = as_stream(stream);
  float* const part = reinterpret_cast<float*>(align_up((size_t)ws, 256));
  const int chunk = norm_chunk(cfg), chunks = cdiv(T, chunk);
  const bool bf16 = cfg->dtype == SYMI_BF16;
  if (T > 0 && (dw || db)) {
    const dim3 grid(cdiv(d, NORM_THREADS * 8), chunks);
    if (bf16)
      SYMI_TIMED(ctx, K_NORM_BWD, st, (norm_columns_kernel<true><<<grid, NORM_THREADS, 0, st>>>(dY, R, mean, rstd, part, T, d, center, chunk, dw != nullptr, db != nullptr)));
    else
      SYMI_TIMED(ctx, K_NORM_BWD, st, (norm_columns_kernel<false><<<grid, NORM_THREADS, 0, st>>>(dY, R, mean, rstd, part, T, d, center, chunk, dw != nullptr, db != nullptr)));
  }
  if (T > 0) {
    if (bf16)
      SYMI_TIMED(ctx, K_NORM_BWD, st, (norm_bwd_kernel<true><<<T, NORM_THREADS, 0, st>>>(dY, R, mean, rstd, w, dR, dX, d, center)));
    else
      SYMI_TIMED(ctx, K_NORM_BWD, st, (norm_bwd_kernel<false><<<T, NORM_THREADS, 0, st>>>(dY, R, mean, rstd, w, dR, dX, d, center)));
  }
  if (dw || db) SYMI_TIMED(ctx, K_NORM_SUM, st, (norm_sum_kernel<<<cdiv(d, NORM_THREADS), NORM_THREADS, 0, st>>>(part, dw, db, chunks, d)));
  SYMI_LAUNCH_CHECK("symi_norm_bwd");
  return SYMI_OK;
}
