// symi_norm_fwd / symi_norm_bwd: layer norm and RMS norm of rows behind a residual sum, and their gradients.
//
// mean = sum R / d, rstd = 1 / sqrt(sum (R - mean)^2 / d + eps), Y = (R - mean) rstd w + b;
// with xh = (R - mean) rstd and g = dY w: dX = rstd (g - sum g / d - xh sum(g xh) / d) + dR, dw = sum dY xh, db = sum dY.
//
// Bound by bytes: a row is read once, stays in registers from its sums to its results and is written once; w and b are read once a workgroup.
// 65536 rows of 4096 in bf16 with a residual sum: forward 385 us (5.6 TB/s), gradients 392 us (5.5 TB/s, 5 of them the sums over the workgroups).  What
// it takes for that is few rows at a time, next to each other in memory: the forward pass with 16 to 24 KB of loads on their way to a compute unit 385, with
// twice as many 407; the gradients with 512 workgroups of every 512th row 392, with 1024 of them 407, with 512 of consecutive rows 424.
#include <math.h>

#include <algorithm>
#include <type_traits>

#include "common.h"

namespace symi {

constexpr int WIDE_THREADS = 1024;
constexpr int NORM_PARTS = 512;        // workgroups of the gradients, and so partial sums of dw and db, at most
constexpr int NORM_FLYING = 24576;     // bytes on their way to a compute unit
constexpr int NORM_IN_REGS = 16384, NORM_BWD_IN_REGS = 8192;   // widest rows that stay in registers

// 8 consecutive values of a row as they lie in memory: 16 or 32 bytes.
template <bool BF16> struct Eight {
  typedef uint32_t Raw __attribute__((ext_vector_type(4)));
  Raw r[BF16 ? 1 : 2];
  __device__ __forceinline__ void load(const void* p, long long at) {
    if constexpr (BF16) {
      r[0] = __builtin_bit_cast(Raw, *reinterpret_cast<const u32x4_bf16*>(static_cast<const uint16_t*>(p) + at));
    } else {
      const float* const q = static_cast<const float*>(p) + at;
      r[0] = __builtin_bit_cast(Raw, *reinterpret_cast<const f32x4_f32*>(q));
      r[1] = __builtin_bit_cast(Raw, *reinterpret_cast<const f32x4_f32*>(q + 4));
    }
  }
  __device__ __forceinline__ void clear() {
#pragma unroll
    for (int h = 0; h < (BF16 ? 1 : 2); ++h) r[h] = Raw{0, 0, 0, 0};
  }
  __device__ __forceinline__ void unpack(float (&x)[8]) const {
    if constexpr (BF16) {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        x[2 * i] = __uint_as_float(r[0][i] << 16);
        x[2 * i + 1] = __uint_as_float(r[0][i] & 0xffff0000u);
      }
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i) x[i] = __uint_as_float(r[i >> 2][i & 3]);
    }
  }
  __device__ __forceinline__ void pack(const float (&x)[8]) {
    if constexpr (BF16) {
#pragma unroll
      for (int i = 0; i < 4; ++i) r[0][i] = pack_bf16x2(x[2 * i], x[2 * i + 1]);
    } else {
#pragma unroll
      for (int i = 0; i < 8; ++i) r[i >> 2][i & 3] = __float_as_uint(x[i]);
    }
  }
  __device__ __forceinline__ void store(void* p, long long at) const {
    if constexpr (BF16) {
      *reinterpret_cast<u32x4_bf16*>(static_cast<uint16_t*>(p) + at) = __builtin_bit_cast(u32x4_bf16, r[0]);
    } else {
      float* const q = static_cast<float*>(p) + at;
      *reinterpret_cast<f32x4_f32*>(q) = __builtin_bit_cast(f32x4_f32, r[0]);
      *reinterpret_cast<f32x4_f32*>(q + 4) = __builtin_bit_cast(f32x4_f32, r[1]);
    }
  }
};
// 8 of w or b, or what stands for them
__device__ __forceinline__ void load_weights(const float* p, int c, int d, float none, float (&x)[8]) {
  if (p && c < d) {
    Eight<false> e;
    e.load(p, c);
    e.unpack(x);
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = none;
  }
}
template <bool BF16>
__device__ __forceinline__ void load8(const void* p, long long at, float (&x)[8]) {
  Eight<BF16> e;
  e.load(p, at);
  e.unpack(x);
}
template <bool BF16>
__device__ __forceinline__ void store8(void* p, long long at, const float (&x)[8]) {
  Eight<BF16> e;
  e.pack(x);
  e.store(p, at);
}
// Sum over groups of LANES (16 or 64) lanes, which all get it: rotations within 16 lanes, then two broadcasts of a row's last lane, as operands of the
// additions themselves (through ds_bpermute a sum over 64 lanes took 0.3 us).
template <int CTRL, int ROWS>
__device__ __forceinline__ float plus_dpp(float x) {
  return x + __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(x), CTRL, ROWS, 0xf, false));
}
template <int LANES>
__device__ __forceinline__ float lanes_sum(float x) {
  static_assert(LANES == 16 || LANES == 64, "a row of lanes or all of them");
  x = plus_dpp<0x128, 0xf>(x);   // row_ror:8
  x = plus_dpp<0x124, 0xf>(x);
  x = plus_dpp<0x122, 0xf>(x);
  x = plus_dpp<0x121, 0xf>(x);
  if constexpr (LANES == 64) {
    x = plus_dpp<0x142, 0xa>(x);   // row_bcast:15 into rows 1 and 3
    x = plus_dpp<0x143, 0xc>(x);   // row_bcast:31 into rows 2 and 3
    x = __int_as_float(__builtin_amdgcn_readlane(__float_as_int(x), 63));
  }
  return x;
}

// Sum over a workgroup, in the same order always; every thread gets it.
__device__ __forceinline__ float block_sum(float x, float* part) {
  x = lanes_sum<64>(x);
  __syncthreads();
  if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = x;
  __syncthreads();
  float s = 0.f;
  for (int w = 0; w < (int)blockDim.x / 64; ++w) s += part[w];
  return s;
}

// Rows of more than NORM_IN_REGS values: one workgroup a row, read three times; a thread reads back what it wrote itself.
template <bool BF16>
__global__ __launch_bounds__(WIDE_THREADS) void norm_wide_kernel(const void* X, const void* res, const float* __restrict__ w,
                                                                 const float* __restrict__ b, void* R, void* Y, float* __restrict__ mean_out,
                                                                 float* __restrict__ rstd_out, int T, int d, int center, float eps) {
  __shared__ float part[WIDE_THREADS / 64];
  const int t = flat_block();
  if (t >= T) return;
  const long long row = (long long)t * d;
  float s = 0.f;
  for (int c = threadIdx.x * 8; c < d; c += WIDE_THREADS * 8) {
    float x[8];
    load8<BF16>(X, row + c, x);
    if (res) {
      float y[8];
      load8<BF16>(res, row + c, y);
      Eight<BF16> e;
#pragma unroll
      for (int i = 0; i < 8; ++i) x[i] += y[i];
      e.pack(x);
      e.store(R, row + c);
      e.unpack(x);
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) s += x[i];
  }
  const void* const from = res ? R : X;
  const float mean = center ? block_sum(s, part) / (float)d : 0.f;
  float q = 0.f;
  for (int c = threadIdx.x * 8; c < d; c += WIDE_THREADS * 8) {
    float x[8];
    load8<BF16>(from, row + c, x);
#pragma unroll
    for (int i = 0; i < 8; ++i) q += (x[i] - mean) * (x[i] - mean);
  }
  const float rstd = 1.f / sqrtf(block_sum(q, part) / (float)d + eps);
  for (int c = threadIdx.x * 8; c < d; c += WIDE_THREADS * 8) {
    float x[8];
    load8<BF16>(from, row + c, x);
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = (x[i] - mean) * rstd * (w ? w[c + i] : 1.f) + (b ? b[c + i] : 0.f);
    store8<BF16>(Y, row + c, x);
  }
  if (threadIdx.x == 0) {
    if (mean_out) mean_out[t] = mean;
    if (rstd_out) rstd_out[t] = rstd;
  }
}

// A row in the registers of LANES threads, NV pieces of 8 values each; what they are goes by d alone, and with it every sum's order.
template <int LANES>
struct Rows {
  static constexpr int THREADS = LANES > 256 ? LANES : 256;
  static constexpr int AT_ONCE = THREADS / LANES;   // rows of a workgroup
  // groups of threads whose sums for dw and db are added up in the end
  static constexpr int GROUPS = LANES <= 64 ? THREADS / 64 : AT_ONCE;
};

// Sum over the threads of a row; the two partial arrays take turns, so that one barrier a sum is enough.
template <int LANES>
__device__ __forceinline__ float row_sum(float x, float (*part)[16], int& turn) {
  x = lanes_sum<(LANES < 64 ? LANES : 64)>(x);
  if constexpr (LANES > 64) {
    if ((threadIdx.x & 63) == 0) part[turn][threadIdx.x >> 6] = x;
    __syncthreads();
    x = 0.f;
#pragma unroll
    for (int w = 0; w < LANES / 64; ++w) x += part[turn][threadIdx.x / LANES * (LANES / 64) + w];
    turn ^= 1;
  }
  return x;
}

// Workgroups go through the rows with w and b in registers, the next row's loads in flight.
template <bool BF16, int LANES, int NV, bool RES>
__global__ __launch_bounds__(Rows<LANES>::THREADS) void norm_kernel(const void* X, const void* res, const float* __restrict__ w,
                                                                        const float* __restrict__ b, void* R, void* Y, float* __restrict__ mean_out,
                                                                        float* __restrict__ rstd_out, int T, int d, int center, float eps) {
  using G = Rows<LANES>;
  __shared__ float part[2][16];
  int turn = 0;
  const int l = threadIdx.x % LANES, sub = threadIdx.x / LANES;
  float ww[NV][8], bb[NV][8];
#pragma unroll
  for (int v = 0; v < NV; ++v) {
    const int c = (v * LANES + l) * 8;
    load_weights(w, c, d, 1.f, ww[v]);
    load_weights(b, c, d, 0.f, bb[v]);
  }
  const int step = gridDim.x * G::AT_ONCE;
  Eight<BF16> x[NV], y[NV];
  auto fetch = [&](long long t) {
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      const int c = (v * LANES + l) * 8;
      x[v].clear();
      if (RES) y[v].clear();
      if (c < d && t < T) {
        x[v].load(X, t * d + c);
        if (RES) y[v].load(res, t * d + c);
      }
    }
  };
  long long t = (long long)blockIdx.x * G::AT_ONCE + sub;
  fetch(t);
  for (long long t0 = (long long)blockIdx.x * G::AT_ONCE; t0 < T; t0 += step, t += step) {
    const bool in = t < T;
    float r[NV][8], s = 0.f;
    Eight<BF16> kept;
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      const int c = (v * LANES + l) * 8;
      x[v].unpack(r[v]);
      if (RES) {
        float z[8];
        y[v].unpack(z);
#pragma unroll
        for (int i = 0; i < 8; ++i) r[v][i] += z[i];
        kept.pack(r[v]);
        kept.unpack(r[v]);
        if (c < d && in) kept.store(R, t * d + c);
      }
#pragma unroll
      for (int i = 0; i < 8; ++i) s += r[v][i];
    }
    fetch(t + step);
    const float mean = center ? row_sum<LANES>(s, part, turn) / (float)d : 0.f;
    float q = 0.f;
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      if ((v * LANES + l) * 8 < d)
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          r[v][i] -= mean;
          q += r[v][i] * r[v][i];
        }
    }
    const float rstd = 1.f / sqrtf(row_sum<LANES>(q, part, turn) / (float)d + eps);
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      const int c = (v * LANES + l) * 8;
#pragma unroll
      for (int i = 0; i < 8; ++i) r[v][i] = r[v][i] * rstd * ww[v][i] + bb[v][i];
      kept.pack(r[v]);
      if (c < d && in) kept.store(Y, t * d + c);
    }
    if (l == 0 && in) {
      if (mean_out) mean_out[t] = mean;
      if (rstd_out) rstd_out[t] = rstd;
    }
  }
}

template <bool BF16>
__global__ __launch_bounds__(WIDE_THREADS) void norm_bwd_wide_kernel(const void* dY, const void* R, const float* __restrict__ mean_in,
                                                                const float* __restrict__ rstd_in, const float* __restrict__ w, const void* dR,
                                                                void* dX, int T, int d, int center) {
  __shared__ float part[WIDE_THREADS / 64];
  const int t = flat_block();
  if (t >= T) return;
  const long long row = (long long)t * d;
  const float mean = center ? mean_in[t] : 0.f, rstd = rstd_in[t];
  float level = 0.f, along = 0.f;
  for (int c = threadIdx.x * 8; c < d; c += WIDE_THREADS * 8) {
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
  for (int c = threadIdx.x * 8; c < d; c += WIDE_THREADS * 8) {
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

// Wide rows' sums over a chunk of rows; a thread has 8 columns.
template <bool BF16>
__global__ __launch_bounds__(256) void norm_columns_kernel(const void* dY, const void* R, const float* __restrict__ mean_in,
                                                                    const float* __restrict__ rstd_in, float* __restrict__ part, int T, int d,
                                                                    int center, int chunk, int want_w, int want_b) {
  const int c = (blockIdx.x * 256 + threadIdx.x) * 8;
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

// dw and db of few rows beside their gradient, in the same launch: a workgroup has 64 columns, 8 threads of 8 each, and every 32nd or 64th row.  The rows
// are read twice, by two workgroups, which costs less than the launch that would add partial sums up.
template <bool BF16, int THREADS>
__device__ __forceinline__ void few_columns(const void* dY, const void* R, const float* __restrict__ mean_in, const float* __restrict__ rstd_in,
                                            float* __restrict__ dw, float* __restrict__ db, int block, int T, int d, int center, float4 (*turned)[8][4]) {
  const int c = block * 64 + (threadIdx.x & 7) * 8, first = threadIdx.x >> 3;
  float sw[8] = {}, sb[8] = {};
  if (c < d) {
#pragma unroll 4
    for (int t = first; t < T; t += THREADS / 8) {
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
  }
  // of the 8 rows of a wavefront by exchange, of the wavefronts in order
#pragma unroll
  for (int m = 8; m < 64; m <<= 1)
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      sw[i] += __shfl_xor(sw[i], m, 64);
      sb[i] += __shfl_xor(sb[i], m, 64);
    }
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  if (lane < 8) {
    turned[wave][lane][0] = make_float4(sw[0], sw[1], sw[2], sw[3]);
    turned[wave][lane][1] = make_float4(sw[4], sw[5], sw[6], sw[7]);
    turned[wave][lane][2] = make_float4(sb[0], sb[1], sb[2], sb[3]);
    turned[wave][lane][3] = make_float4(sb[4], sb[5], sb[6], sb[7]);
  }
  __syncthreads();
  const int k = threadIdx.x & 63, which = threadIdx.x >> 6;   // a column of dw, of db
  float* const to = which == 0 ? dw : which == 1 ? db : nullptr;
  if (!to || block * 64 + k >= d) return;
  float s = 0.f;
#pragma unroll
  for (int w = 0; w < THREADS / 64; ++w) s += reinterpret_cast<const float*>(&turned[w][k >> 3][2 * which])[k & 7];
  to[block * 64 + k] = s;
}

// Gradient of the rows and the workgroup's sums for dw and db in one pass, a thread having the same columns of every row.  At any time the workgroups
// are at neighbouring rows.  FEW: the first `columns` workgroups have the columns' sums, and the others leave theirs.
template <bool BF16, int LANES, int NV, bool RES, bool FEW>
__global__ __launch_bounds__(Rows<LANES>::THREADS) void norm_bwd_kernel(const void* dY, const void* R, const float* __restrict__ mean_in,
                                                                        const float* __restrict__ rstd_in, const float* __restrict__ w, const void* dR,
                                                                        void* dX, float* __restrict__ part_out, int T, int d, int center, int want_w,
                                                                        int want_b, float* __restrict__ dw, float* __restrict__ db, int columns) {
  if constexpr (FEW) {
    if ((int)blockIdx.x < columns) {
      __shared__ float4 turned[Rows<LANES>::THREADS / 64][8][4];
      few_columns<BF16, Rows<LANES>::THREADS>(dY, R, mean_in, rstd_in, dw, db, blockIdx.x, T, d, center, turned);
      return;
    }
  }
  const int group = FEW ? blockIdx.x - columns : blockIdx.x, groups = FEW ? gridDim.x - columns : gridDim.x;
  using G = Rows<LANES>;
  __shared__ float part[4][16];
  const int l = threadIdx.x % LANES, sub = threadIdx.x / LANES, lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  float ww[NV][8], sw[NV][8] = {}, sb[NV][8] = {};
#pragma unroll
  for (int v = 0; v < NV; ++v) {
    load_weights(w, (v * LANES + l) * 8, d, 1.f, ww[v]);
  }
  const int step = groups * G::AT_ONCE;
  Eight<BF16> g[NV], x[NV], y[NV];
  float mean = 0.f, rstd = 0.f;
  auto fetch = [&](long long t) {
    const bool in = t < T;
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      const int c = (v * LANES + l) * 8;
      g[v].clear();
      x[v].clear();
      if (RES) y[v].clear();
      if (c < d && in) {
        g[v].load(dY, t * d + c);
        x[v].load(R, t * d + c);
        if (RES) y[v].load(dR, t * d + c);
      }
    }
    mean = in && center ? mean_in[t] : 0.f;
    rstd = in ? rstd_in[t] : 0.f;
  };
  long long t = (long long)group * G::AT_ONCE + sub;
  fetch(t);
  int turn = 0;
  for (long long t0 = (long long)group * G::AT_ONCE; t0 < T; t0 += step, t += step) {
    const bool in = t < T;
    float gg[NV][8], xh[NV][8], rr[NV][8];
    const float scale = rstd;
    float level = 0.f, along = 0.f;
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      g[v].unpack(gg[v]);
      x[v].unpack(xh[v]);
      if (RES) y[v].unpack(rr[v]);
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        xh[v][i] = in && (v * LANES + l) * 8 < d ? (xh[v][i] - mean) * scale : 0.f;   // no row: nothing that could be NaN
        sw[v][i] += gg[v][i] * xh[v][i];
        sb[v][i] += gg[v][i];
        gg[v][i] *= ww[v][i];
        level += gg[v][i];
        along += gg[v][i] * xh[v][i];
      }
    }
    fetch(t + step);
    // both sums over the row in one exchange
    level = lanes_sum<(LANES < 64 ? LANES : 64)>(level);
    along = lanes_sum<(LANES < 64 ? LANES : 64)>(along);
    if constexpr (LANES > 64) {
      if (lane == 0) {
        part[turn][wave] = level;
        part[turn + 1][wave] = along;
      }
      __syncthreads();
      level = along = 0.f;
#pragma unroll
      for (int k = 0; k < LANES / 64; ++k) {
        level += part[turn][sub * (LANES / 64) + k];
        along += part[turn + 1][sub * (LANES / 64) + k];
      }
      turn ^= 2;
    }
    level = center ? level / (float)d : 0.f;
    along /= (float)d;
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      const int c = (v * LANES + l) * 8;
#pragma unroll
      for (int i = 0; i < 8; ++i) gg[v][i] = (gg[v][i] - level - xh[v][i] * along) * scale + (RES ? rr[v][i] : 0.f);
      Eight<BF16> out;
      out.pack(gg[v]);
      if (c < d && in) out.store(dX, t * d + c);
    }
  }
  if (FEW || (!want_w && !want_b)) return;
  // the sums of the rows that the workgroup had at once: of a wavefront by exchange, of its wavefronts one after the other by the first
  float* const to = part_out + (long long)group * 2 * d;
  if constexpr (LANES < 64) {
#pragma unroll
    for (int v = 0; v < NV; ++v)
#pragma unroll
      for (int m = LANES; m < 64; m <<= 1)
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          sw[v][i] += __shfl_xor(sw[v][i], m, 64);
          sb[v][i] += __shfl_xor(sb[v][i], m, 64);
        }
  }
  if constexpr (G::GROUPS > 1) {
    __shared__ float4 turned[G::GROUPS - 1][NV * 4][LANES];
    const int group = LANES <= 64 ? wave : sub;
    const bool first = LANES >= 64 || lane < LANES;   // one lane of those that have the same sums
    if (group && first)
#pragma unroll
      for (int v = 0; v < NV; ++v)
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          turned[group - 1][4 * v + h][l] = make_float4(sw[v][4 * h], sw[v][4 * h + 1], sw[v][4 * h + 2], sw[v][4 * h + 3]);
          turned[group - 1][4 * v + 2 + h][l] = make_float4(sb[v][4 * h], sb[v][4 * h + 1], sb[v][4 * h + 2], sb[v][4 * h + 3]);
        }
    __syncthreads();
    if (group || !first) return;
#pragma unroll
    for (int q = 0; q < G::GROUPS - 1; ++q)
#pragma unroll
      for (int v = 0; v < NV; ++v)
#pragma unroll
        for (int h = 0; h < 2; ++h) {
          const float4 x = turned[q][4 * v + h][l], y = turned[q][4 * v + 2 + h][l];
          sw[v][4 * h] += x.x; sw[v][4 * h + 1] += x.y; sw[v][4 * h + 2] += x.z; sw[v][4 * h + 3] += x.w;
          sb[v][4 * h] += y.x; sb[v][4 * h + 1] += y.y; sb[v][4 * h + 2] += y.z; sb[v][4 * h + 3] += y.w;
        }
  }
#pragma unroll
  for (int v = 0; v < NV; ++v) {
    const int c = (v * LANES + l) * 8;
    if (c < d)
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        if (want_w) to[c + i] = sw[v][i];
        if (want_b) to[d + c + i] = sb[v][i];
      }
  }
}

// Column sums of the partial sums: wavefront w of 16 takes every 16th chunk of 64 columns, and the wavefronts are added in order.
constexpr int SUM_WAVES = 16;
__global__ __launch_bounds__(SUM_WAVES * 64) void norm_sum_kernel(const float* __restrict__ part, float* __restrict__ dw, float* __restrict__ db,
                                                                  int chunks, int d) {
  __shared__ float s[SUM_WAVES][64];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int c = blockIdx.x * 64 + lane;
  float* const to = blockIdx.y ? db : dw;
  if (!to) return;
  const float* const from = part + (long long)blockIdx.y * d + c;
  float x = 0.f;
  if (c < d)
#pragma unroll 8
    for (int k = wave; k < chunks; k += SUM_WAVES) x += from[(long long)k * 2 * d];
  s[wave][lane] = x;
  __syncthreads();
  if (wave == 0 && c < d) {
    x = 0.f;
#pragma unroll
    for (int w = 0; w < SUM_WAVES; ++w) x += s[w][lane];
    to[c] = x;
  }
}

// Threads of a row and pieces of 8 values each: one piece where that is a whole number of wavefronts.
static void norm_shape(int d, int& lanes, int& nv) {
  const int pieces = d / 8;
  lanes = pieces <= 32 ? 16 : pieces <= 128 ? 64 : pieces <= 256 ? 128 : pieces <= 1024 ? 512 : 1024;
  nv = pieces <= lanes ? 1 : 2;
}
static int rows_at_once(int lanes) { return lanes >= 256 ? 1 : 256 / lanes; }

// Partial sums for dw and db, which is workgroups: what T and d decide.
static int norm_parts(const symi_cfg* c) {
  if (c->d > NORM_BWD_IN_REGS) return std::min(c->T, NORM_PARTS);
  int lanes, nv;
  norm_shape(c->d, lanes, nv);
  return std::min(cdiv(c->T, rows_at_once(lanes)), c->T <= 2560 ? NORM_PARTS / 2 : NORM_PARTS);   // 777 x 1160 fp32: 10.7 -> 9.7 us
}

}  // namespace symi

using namespace symi;

extern "C" size_t symi_norm_workspace_bytes(const symi_cfg* cfg) {
  if (check_cfg(cfg, "symi_norm_workspace_bytes") != SYMI_OK) return 0;
  return align_up((size_t)norm_parts(cfg) * 2 * cfg->d * sizeof(float), 256) + 256;
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
  const int T = cfg->T, d = cfg->d;
  const bool bf16 = cfg->dtype == SYMI_BF16;
  if (d > NORM_IN_REGS) {
    if (bf16) SYMI_TIMED(ctx, K_NORM, st, (norm_wide_kernel<true><<<flat_grid(T), WIDE_THREADS, 0, st>>>(X, residual, w, b, R, Y, mean, rstd, T, d, center, eps)));
    else SYMI_TIMED(ctx, K_NORM, st, (norm_wide_kernel<false><<<flat_grid(T), WIDE_THREADS, 0, st>>>(X, residual, w, b, R, Y, mean, rstd, T, d, center, eps)));
  } else {
    int lanes, nv;
    norm_shape(d, lanes, nv);
    const int flying = std::max(lanes, 256) * nv * (bf16 ? 16 : 32) * (residual ? 2 : 1);   // bytes that a workgroup has on their way
    const int grid = std::min(cdiv(T, rows_at_once(lanes)), ctx->cus * std::max(1, NORM_FLYING / flying));
#define NORM_CASE(LL, NN)                                                                                                              \
  case LL * 8 + NN:                                                                                                                    \
    if (bf16 && residual)                                                                                                              \
      SYMI_TIMED(ctx, K_NORM, st, (norm_kernel<true, LL, NN, true><<<grid, Rows<LL>::THREADS, 0, st>>>(X, residual, w, b, R, Y, mean, rstd, T, d, center, eps)));   \
    else if (bf16)                                                                                                                     \
      SYMI_TIMED(ctx, K_NORM, st, (norm_kernel<true, LL, NN, false><<<grid, Rows<LL>::THREADS, 0, st>>>(X, residual, w, b, R, Y, mean, rstd, T, d, center, eps)));  \
    else if (residual)                                                                                                                 \
      SYMI_TIMED(ctx, K_NORM, st, (norm_kernel<false, LL, NN, true><<<grid, Rows<LL>::THREADS, 0, st>>>(X, residual, w, b, R, Y, mean, rstd, T, d, center, eps)));  \
    else                                                                                                                               \
      SYMI_TIMED(ctx, K_NORM, st, (norm_kernel<false, LL, NN, false><<<grid, Rows<LL>::THREADS, 0, st>>>(X, residual, w, b, R, Y, mean, rstd, T, d, center, eps))); \
    break;
#define NORM_CASES NORM_CASE(16, 1) NORM_CASE(16, 2) NORM_CASE(64, 1) NORM_CASE(64, 2) NORM_CASE(128, 2) NORM_CASE(512, 1) NORM_CASE(512, 2)
    switch (lanes * 8 + nv) {
      NORM_CASES NORM_CASE(1024, 2)
      default:
        set_error("symi_norm_fwd: no kernel for %d threads x %d pieces a row", lanes, nv);
        return SYMI_EUNSUPPORTED;
    }
#undef NORM_CASE
  }
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
  const int parts = norm_parts(cfg);
  const bool bf16 = cfg->dtype == SYMI_BF16;
  const int want_w = dw != nullptr, want_b = db != nullptr;
  if (T > 0 && d > NORM_BWD_IN_REGS) {
    const dim3 grid(cdiv(d, 256 * 8), parts);
    if (bf16) {
      if (want_w || want_b)
        SYMI_TIMED(ctx, K_NORM_BWD, st, (norm_columns_kernel<true><<<grid, 256, 0, st>>>(dY, R, mean, rstd, part, T, d, center, cdiv(T, parts), want_w, want_b)));
      SYMI_TIMED(ctx, K_NORM_BWD, st, (norm_bwd_wide_kernel<true><<<flat_grid(T), WIDE_THREADS, 0, st>>>(dY, R, mean, rstd, w, dR, dX, T, d, center)));
    } else {
      if (want_w || want_b)
        SYMI_TIMED(ctx, K_NORM_BWD, st, (norm_columns_kernel<false><<<grid, 256, 0, st>>>(dY, R, mean, rstd, part, T, d, center, cdiv(T, parts), want_w, want_b)));
      SYMI_TIMED(ctx, K_NORM_BWD, st, (norm_bwd_wide_kernel<false><<<flat_grid(T), WIDE_THREADS, 0, st>>>(dY, R, mean, rstd, w, dR, dX, T, d, center)));
    }
  } else if (T > 0) {
    int lanes, nv;
    norm_shape(d, lanes, nv);
    // Few rows: the sums beside the gradients, or where those take dY's place, in a launch before.  In one launch / with partial sums, us, bf16: 16 rows of 1160 3.9 / 7.6, 400 rows
    // 5.1 / 9.2, 1024 rows 13.2 / 11.7; 1024 rows of 4096, with twice the threads, 10.5 / 22.3, 2500 rows 22.3 / 29.9.
    const bool few = (want_w || want_b) && T <= (lanes > 256 ? 2560 : 768);
    const int columns = cdiv(d, 64), rows = cdiv(T, rows_at_once(lanes));
#define NORM_BWD(BB, LL, NN, RR)                                                                                                       \
  if (few) {                                                                                                                           \
    const int beside = dX == dY ? 0 : rows;                                                                                            \
    SYMI_TIMED(ctx, K_NORM_BWD, st, (norm_bwd_kernel<BB, LL, NN, RR, true><<<columns + beside, Rows<LL>::THREADS, 0, st>>>(dY, R, mean, rstd, w, dR, dX, nullptr, T, d, center, 0, 0, dw, db, columns))); \
    if (beside) break;                                                                                                                 \
  }                                                                                                                                    \
  SYMI_TIMED(ctx, K_NORM_BWD, st, (norm_bwd_kernel<BB, LL, NN, RR, false><<<parts, Rows<LL>::THREADS, 0, st>>>(dY, R, mean, rstd, w, dR, dX, part, T, d, center, few ? 0 : want_w, few ? 0 : want_b, nullptr, nullptr, 0)));
#define NORM_CASE(LL, NN)                                                                                                              \
  case LL * 8 + NN:                                                                                                                    \
    if (bf16 && dR) { NORM_BWD(true, LL, NN, true) }                                                                                   \
    else if (bf16) { NORM_BWD(true, LL, NN, false) }                                                                                   \
    else if (dR) { NORM_BWD(false, LL, NN, true) }                                                                                     \
    else { NORM_BWD(false, LL, NN, false) }                                                                                            \
    break;
    switch (lanes * 8 + nv) {
      NORM_CASES
      default:
        set_error("symi_norm_bwd: no kernel for %d threads x %d pieces a row", lanes, nv);
        return SYMI_EUNSUPPORTED;
    }
#undef NORM_CASE
#undef NORM_BWD
    if (few) {
      SYMI_LAUNCH_CHECK("symi_norm_bwd");
      return SYMI_OK;
    }
  }
  if (dw || db) SYMI_TIMED(ctx, K_NORM_SUM, st, (norm_sum_kernel<<<dim3(cdiv(d, 64), 2), SUM_WAVES * 64, 0, st>>>(part, dw, db, parts, d)));
  SYMI_LAUNCH_CHECK("symi_norm_bwd");
  return SYMI_OK;
}
