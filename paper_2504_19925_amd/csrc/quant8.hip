// symi_quant8 / symi_dequant8 / symi_product8 / symi_expert_fwd8: values in 8 bits with a power of two for every 128 along the reduction,
// and the experts' products of them.
//
// The scales are the powers that v_mfma_scale_f32_16x16x128_f8f6f4 multiplies by itself: one instruction reduces exactly one block of 128, so a
// product needs no vector work per block.  The instruction is issued with the weight as its first operand: a lane then has 4 consecutive
// output columns of one row.  A lane holds 32 of the 128 reduction indices of one row of each operand; any 32, as long as they are the same in both.
//
// The 8-bit matrix instructions align the products of 8 neighbouring indices to the largest exponent among them and drop what is below 2^-13 of it; sums
// of those, over the block and in the accumulator, are fp32 (probed with single products of 2^8 and 2^-j, a group's first and others).  Over random
// values that is 1.5e-5 of a result (2-norm), a hundredth of what rounding it to bf16 is.  Where a result is rounded to 8 bits it is more: 4 of 10000 hidden units of
// the experts come out one code further, and the experts' results are off by 2.0e-3 where sums in fp32 make it 1.66e-3, bf16's own (c5).  Tiles of few rows and fp32 contexts
// have no such loss: there codes become bf16 values, exactly, for the bf16 instruction, which keeps fp32's digits (8e-8) and has half the rate; the powers are put into the
// values (tiles of 128 rows, wherever their range allows) or the block's sum is scaled behind it.
#include <algorithm>
#include <type_traits>

#include "quant8.h"

namespace symi {

constexpr int Q_THREADS = 256;
constexpr int MAX_N8 = 1 << 22;

static int pitch8(int n) { return cdiv(n, QB) * QB; }
static int scale_pitch8(int n) { return cdiv(cdiv(n, QB), 4) * 4; }

// 8 values in fp32 from memory of the activation dtype
template <bool BF16>
__device__ __forceinline__ void load8q(const void* p, long long at, float (&x)[8]) {
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

// 16 lanes a block of a row.  limit: rows from *limit on are left out (nullptr: none are).  Bound by bytes: 196608 x 2048 in bf16 252 us, 4.8 TB/s.
template <bool BF16>
__global__ __launch_bounds__(Q_THREADS) void quant_rows_kernel(const void* __restrict__ X, uint8_t* __restrict__ q, uint8_t* __restrict__ s,
                                                               long long rows, int n, int p8, int sp, const int32_t* __restrict__ limit) {
  if (limit) rows = min(rows, (long long)*limit);
  const int l16 = threadIdx.x & 15;
  const long long total = rows * sp, step = (long long)gridDim.x * (Q_THREADS / 16);
  for (long long i = (long long)blockIdx.x * (Q_THREADS / 16) + (threadIdx.x >> 4); i < total; i += step) {
    const long long r = i / sp;
    const int blk = (int)(i - r * sp), c = blk * QB + l16 * 8;
    if (blk * QB >= p8) {
      if (l16 == 0) s[i] = 0;
      continue;
    }
    float x[8] = {};
    if (c < n) load8q<BF16>(X, r * n + c, x);
    int most = 0;
#pragma unroll
    for (int j = 0; j < 8; ++j) most = max(most, size_of(x[j]));
#pragma unroll
    for (int m = 8; m >= 1; m >>= 1) most = max(most, __shfl_xor(most, m, 16));
    const int e = scale_of(most);
    const float inv = inverse_of(e);
    *reinterpret_cast<uint2*>(q + r * p8 + c) = make_uint2(codes4(x[0], x[1], x[2], x[3], inv), codes4(x[4], x[5], x[6], x[7], inv));
    if (l16 == 0) s[i] = (uint8_t)e;
  }
}

// A workgroup a block of 128 x 128: 16 lanes a row, 16 rows at a time, all in registers until the largest is known.  128 weights of 2816 x 2048 in bf16 556 us, 4.0 TB/s.
template <bool BF16>
__global__ __launch_bounds__(Q_THREADS) void quant_blocks_kernel(const void* __restrict__ X, uint8_t* __restrict__ q, uint8_t* __restrict__ s,
                                                                 int rows, int n, int p8, int sp, int rb, unsigned blocks) {
  __shared__ int part[Q_THREADS / 64];
  const unsigned at = flat_block();
  if (at >= blocks) return;
  const int bc = at % sp;
  const long long br_all = at / sp;
  const int group = (int)(br_all / rb), br = (int)(br_all - (long long)group * rb);
  const int l16 = threadIdx.x & 15, c = bc * QB + l16 * 8;
  const long long si = br_all * sp + bc;
  if (bc * QB >= p8) {
    if (threadIdx.x == 0) s[si] = 0;
    return;
  }
  float x[8][8];
  int most = 0;
#pragma unroll
  for (int k = 0; k < 8; ++k) {
    const int r = br * QB + k * 16 + (threadIdx.x >> 4);
#pragma unroll
    for (int j = 0; j < 8; ++j) x[k][j] = 0.f;
    if (r < rows && c < n) load8q<BF16>(X, ((long long)group * rows + r) * n + c, x[k]);
#pragma unroll
    for (int j = 0; j < 8; ++j) most = max(most, size_of(x[k][j]));
  }
#pragma unroll
  for (int m = 32; m >= 1; m >>= 1) most = max(most, __shfl_xor(most, m, 64));
  if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = most;
  __syncthreads();
  most = max(max(part[0], part[1]), max(part[2], part[3]));
  const int e = scale_of(most);
  const float inv = inverse_of(e);
#pragma unroll
  for (int k = 0; k < 8; ++k) {
    const int r = br * QB + k * 16 + (threadIdx.x >> 4);
    if (r < rows)
      *reinterpret_cast<uint2*>(q + ((long long)group * rows + r) * p8 + c) =
          make_uint2(codes4(x[k][0], x[k][1], x[k][2], x[k][3], inv), codes4(x[k][4], x[k][5], x[k][6], x[k][7], inv));
  }
  if (threadIdx.x == 0) s[si] = (uint8_t)e;
}

// 8 values a thread.  196608 x 2048 in bf16 218 us, 5.5 TB/s.
template <bool BF16>
__global__ __launch_bounds__(Q_THREADS) void dequant_kernel(const uint8_t* __restrict__ q, const uint8_t* __restrict__ s, void* __restrict__ X,
                                                            long long groups, int rows, int n, int p8, int sp, int rb, int block) {
  const int per = n / 8;
  const long long total = groups * rows * per, step = (long long)gridDim.x * Q_THREADS;
  for (long long i = (long long)blockIdx.x * Q_THREADS + threadIdx.x; i < total; i += step) {
    const long long row = i / per;
    const int c = (int)(i - row * per) * 8;
    const long long group = row / rows;
    const int r = (int)(row - group * rows);
    const float scale = power_of(s[(group * rb + r / block) * sp + c / QB]);
    const uint2 w = *reinterpret_cast<const uint2*>(q + row * p8 + c);
    float x[8];
    const uint32_t ww[2] = {w.x, w.y};
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const auto lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)ww[h], false), hi = __builtin_amdgcn_cvt_pk_f32_fp8((int)ww[h], true);
      x[4 * h] = lo[0] * scale;
      x[4 * h + 1] = lo[1] * scale;
      x[4 * h + 2] = hi[0] * scale;
      x[4 * h + 3] = hi[1] * scale;
    }
    if constexpr (BF16) {
      u32x4_bf16 o;
#pragma unroll
      for (int j = 0; j < 4; ++j) o[j] = pack_bf16x2(x[2 * j], x[2 * j + 1]);
      *reinterpret_cast<u32x4_bf16*>(static_cast<uint16_t*>(X) + row * n + c) = o;
    } else {
      float* const to = static_cast<float*>(X) + row * n + c;
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const f32x4_f32 o = {x[4 * h], x[4 * h + 1], x[4 * h + 2], x[4 * h + 3]};
        *reinterpret_cast<f32x4_f32*>(to + 4 * h) = o;
      }
    }
  }
}

// ---------------------------------------------------------------- products
constexpr int THIN = 16;          // rows of a thin tile

// map of tiles of TM rows, slots one after the other
template <int TM>
__global__ __launch_bounds__(1024) void tiles8_kernel(const int32_t* __restrict__ offs, int S, int32_t* __restrict__ map) {
  __shared__ int32_t part[1024];
  const int tid = threadIdx.x, per = (S + 1023) / 1024, q0 = min(tid * per, S), q1 = min(q0 + per, S);
  int mine = 0;
  for (int q = q0; q < q1; ++q) mine += (offs[q + 1] - offs[q] + TM - 1) / TM;
  part[tid] = mine;
  __syncthreads();
  for (int o = 1; o < 1024; o <<= 1) {
    const int add = tid >= o ? part[tid - o] : 0;
    __syncthreads();
    part[tid] += add;
    __syncthreads();
  }
  int t = part[tid] - mine;
  if (tid == 1023) map[0] = part[1023];
  for (int q = q0; q < q1; ++q)
    for (int r = offs[q]; r < offs[q + 1]; r += TM, ++t) {
      map[4 + 2 * t] = r;
      map[5 + 2 * t] = q + ((min(offs[q + 1] - r, TM) - 1) << 16);
    }
}

// 8 codes (half h of 16, in two words) as bf16 values, exactly
__device__ __forceinline__ bf16x8_ widen(int lo, int hi) {
  typedef __bf16 bf16x2_ __attribute__((ext_vector_type(2)));
  const unsigned w[2] = {(unsigned)lo, (unsigned)hi};
  bf16x8_ r;
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const bf16x2_ x = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w[i], 1.f, false), y = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w[i], 1.f, true);
    r[4 * i] = x[0];
    r[4 * i + 1] = x[1];
    r[4 * i + 2] = y[0];
    r[4 * i + 3] = y[1];
  }
  return r;
}

// acc += the products of a block, scaled.  EXACT: through the bf16 instruction, the sum scaled behind it by the power of the lane's four outputs (sw); else sw is that of the
// weight row which the lane holds.
template <bool EXACT>
__device__ __forceinline__ void block_product(floatx4_& acc, const intx8& fw, const intx8& fa, int sw, int sa) {
  if constexpr (!EXACT) {
    acc = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(fw, fa, acc, 0, 0, 0, sw, 0, sa);
  } else {
    floatx4_ part = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int h = 0; h < 4; ++h) part = __builtin_amdgcn_mfma_f32_16x16x32_bf16(widen(fw[2 * h], fw[2 * h + 1]), widen(fa[2 * h], fa[2 * h + 1]), part, 0, 0, 0);
#pragma unroll
    for (int i = 0; i < 4; ++i) acc[i] += ldexpf(part[i], sw + sa - 254);
  }
}

// The same for one tile by a wavefront from the slots' offsets: lane l counts the tiles of consecutive slots, which saves the launch that writes the map (about 4 us,
// for half a microsecond in every workgroup).  False: there is no such tile.
constexpr int FIND_SLOTS = 256;
__device__ __forceinline__ bool find_thin(const int32_t* __restrict__ offs, int S, int tile, int& row0, int& rows, int& slot) {
  const int lane = threadIdx.x & 63, per = (S + 63) / 64, q0 = min(lane * per, S), q1 = min(q0 + per, S);
  int at[FIND_SLOTS / 64 + 1];
#pragma unroll
  for (int i = 0; i <= FIND_SLOTS / 64; ++i) at[i] = offs[min(q0 + i, q1)];
  int mine = 0;
#pragma unroll
  for (int i = 0; i < FIND_SLOTS / 64; ++i) mine += (at[i + 1] - at[i] + THIN - 1) / THIN;
  int upto = mine;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const int up = __shfl_up(upto, o, 64);
    if (lane >= o) upto += up;
  }
  const unsigned long long behind = __ballot(upto > tile);
  if (!behind) return false;
  int left = tile - (upto - mine), found = 0, first = 0, count = 0;
  bool open = true;
#pragma unroll
  for (int i = 0; i < FIND_SLOTS / 64; ++i) {
    const int n = (at[i + 1] - at[i] + THIN - 1) / THIN;
    if (open && left < n) {
      found = q0 + i;
      first = at[i] + left * THIN;
      count = min(at[i + 1] - first, THIN);
      open = false;
    }
    left -= n;
  }
  const int who = __ffsll(behind) - 1;
  slot = __builtin_amdgcn_readlane(found, who);
  row0 = __builtin_amdgcn_readlane(first, who);
  rows = __builtin_amdgcn_readlane(count, who);
  return true;
}

// A tile of 16 rows: a wavefront has 64 weight rows (in the experts' first product the gate and up rows of 32 hidden units) and every SPLIT-th block of the
// reduction, so that few rows still are many wavefronts with a short way each; their sums are added through LDS, in order.  Operands come straight from memory,
// 32 bytes a lane.  What bounds it is the weights' stream: 32 rows in 8 slots of 28672 x 4096 161 us, 5.8 TB/s (with the whole reduction in one wavefront 172); of 1024 x 1024
// 5.6 us (11.2).
//
// The experts' first product goes through the bf16 instruction: what the 8-bit one drops moves hidden units across code borders, a whole step of 8 bits each, which nothing averages
// out where rows are few (2 to 3 rows of 3296 and 2928 hidden units: off by 4.8e-3 and 5.8e-3 of the result with it, by 1.9e-3 and 1.65e-3, as with sums in fp32, without).  The
// weights' stream hides nearly all of the widening: both products of 32 rows in 8 slots, 4096 -> 14336 -> 4096, 276 -> 279 us, 96 rows 284 -> 287; 512 rows in 128 slots,
// 2048 -> 1408 -> 2048, 212 -> 215.
template <bool EXPERT> struct Thin {
  static constexpr int COLUMNS = EXPERT ? 4 : 1, SPLIT = 4, THREADS = 64 * COLUMNS * SPLIT;   // wavefronts side by side and along the reduction
};
template <bool BF16, bool EXPERT>
__global__ __launch_bounds__(Thin<EXPERT>::THREADS) void thin_product_kernel(Product8 p) {
  using G = Thin<EXPERT>;
  constexpr bool EXACT = EXPERT || !BF16;
  const int tile = blockIdx.x;
  int row0, rows, slot;
  if (p.slots <= FIND_SLOTS) {
    if (!find_thin(p.slot_offsets, p.slots, tile, row0, rows, slot)) return;
  } else {
    if (tile >= p.map[0]) return;
    row0 = p.map[4 + 2 * tile];
    const int entry = p.map[5 + 2 * tile];
    slot = entry & 0xffff;
    rows = (entry >> 16) + 1;
  }
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, r16 = lane & 15, quarter = lane >> 4;
  const int wc = wave % G::COLUMNS, part = wave / G::COLUMNS;
  const int slot_rows = EXPERT ? 2 * p.R : p.R, slot_blocks = (slot_rows + QB - 1) / QB;
  // first weight row of the wavefront
  const int n0 = EXPERT ? blockIdx.y * 128 + wc * 32 : blockIdx.y * 64;
  const int arow = row0 + min(r16, rows - 1);
  const uint8_t* const a = p.Aq + (long long)arow * p.p8 + quarter * 32;
  const uint8_t* const as = p.As + (long long)arow * p.sp;
  const uint8_t* w[4];
  const uint8_t* ws[4];
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const int first = n0 + 16 * (EXPERT ? j & 1 : j);
    int wr = min(first + r16, p.R - 1);
    if (EXPERT && j >= 2) wr += p.R;
    w[j] = p.Wq + ((long long)slot * slot_rows + wr) * p.p8 + quarter * 32;
    // of the weight row that this lane holds, or of its four outputs: 4 rows from a multiple of 4 on are in one block (16 up rows need not be)
    const int pr = EXACT ? min(first + 4 * quarter, p.R - 1) + (EXPERT && j >= 2 ? p.R : 0) : wr;
    ws[j] = p.Ws + ((long long)slot * slot_blocks + pr / QB) * p.sp;
  }
  floatx4_ acc[4] = {};
  const int nk = p.p8 / QB;
#pragma unroll 2
  for (int blk = part; blk < nk; blk += G::SPLIT) {
    const long long k = (long long)blk * QB;
    auto read = [&](const uint8_t* from) {
      const intx4_ lo = *reinterpret_cast<const intx4_*>(from + k), hi = *reinterpret_cast<const intx4_*>(from + k + 16);
      return __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
    };
    const intx8 fa = read(a);
    const int sa = as[blk];
    if constexpr (EXPERT) {
      // all loads ahead of the widening; mixed with it by the compiler they took 311 us for 279
      intx8 fw[4];
      int sw[4];
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        fw[j] = read(w[j]);
        sw[j] = ws[j][blk];
      }
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        block_product<EXACT>(acc[j], fw[j], fa, sw[j], sa);
        __builtin_amdgcn_sched_barrier(0);
      }
    } else {
#pragma unroll
      for (int j = 0; j < 4; ++j) block_product<EXACT>(acc[j], read(w[j]), fa, ws[j][blk], sa);
    }
  }
  __shared__ floatx4_ sums[G::SPLIT - 1][G::COLUMNS][4][64];
  if (part)
#pragma unroll
    for (int j = 0; j < 4; ++j) sums[part - 1][wc][j][lane] = acc[j];
  __syncthreads();
  if (!EXPERT && part) return;
  if (!part)
#pragma unroll
    for (int q = 0; q < G::SPLIT - 1; ++q)
#pragma unroll
      for (int j = 0; j < 4; ++j) acc[j] += sums[q][wc][j][lane];
  const int row = row0 + r16;
  const bool in = r16 < rows;
  if constexpr (!EXPERT) {
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int col = n0 + 16 * j + 4 * quarter;
      if (!in || col >= p.R) continue;
      if constexpr (BF16) {
        typedef uint32_t u32x2_bf16 __attribute__((ext_vector_type(2), aligned(2)));
        const u32x2_bf16 y = {pack_bf16x2(acc[j][0], acc[j][1]), pack_bf16x2(acc[j][2], acc[j][3])};
        *reinterpret_cast<u32x2_bf16*>(static_cast<uint16_t*>(p.Y) + (long long)row * p.R + col) = y;
      } else {
        *reinterpret_cast<f32x4_f32*>(static_cast<float*>(p.Y) + (long long)row * p.R + col) = __builtin_bit_cast(f32x4_f32, acc[j]);
      }
    }
  } else {
    __shared__ int part_most[4][16];
    float h[2][4];
    int most = 0;
    if (!part) {
#pragma unroll
      for (int j = 0; j < 2; ++j)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const int col = n0 + 16 * j + 4 * quarter + i;
          const float u = acc[j][i], v = acc[j + 2][i];
          h[j][i] = col < p.R ? u * sigmoid8(u) * v : 0.f;
          most = max(most, size_of(h[j][i]));
          if (in && col < p.R && p.UV) {
            p.UV[(long long)row * 2 * p.R + col] = f32_to_bf16(u);
            p.UV[(long long)row * 2 * p.R + p.R + col] = f32_to_bf16(v);
            p.H[(long long)row * p.R + col] = f32_to_bf16(h[j][i]);
          }
        }
      most = max(most, __shfl_xor(most, 16, 64));
      most = max(most, __shfl_xor(most, 32, 64));
      if (quarter == 0) part_most[wc][r16] = most;
    }
    __syncthreads();
    if (part || !in) return;
    most = max(max(part_most[0][r16], part_most[1][r16]), max(part_most[2][r16], part_most[3][r16]));
    const int e = scale_of(most);
    const float inv = inverse_of(e);
#pragma unroll
    for (int j = 0; j < 2; ++j)
      *reinterpret_cast<uint32_t*>(p.Hq + (long long)row * p.hp8 + n0 + 16 * j + 4 * quarter) = codes4(h[j][0], h[j][1], h[j][2], h[j][3], inv);
    uint8_t* const hs = p.Hs + (long long)row * p.hsp;
    if (wc == 0 && quarter == 0) {
      hs[blockIdx.y] = (uint8_t)e;
      if (blockIdx.y == gridDim.y - 1)      // zeros behind the last block
        for (int b = gridDim.y; b < p.hsp; ++b) hs[b] = 0;
    }
  }
}

struct Ws8 {
  size_t xq, xs, hq, hs, map, total;
};
static Ws8 ws8_layout(const symi_cfg* c) {
  Ws8 L;
  const size_t A = (size_t)c->T * c->k;
  size_t off = 0;
  L.xq = off;
  off += align_up(A * pitch8(c->d), 256);
  L.xs = off;
  off += align_up(A * scale_pitch8(c->d), 256);
  L.hq = off;
  off += align_up(A * pitch8(c->f), 256);
  L.hs = off;
  off += align_up(A * scale_pitch8(c->f), 256);
  L.map = off;
  off += align_up((4 + 2 * (A / THIN + c->S_tot + 1)) * sizeof(int32_t), 256);
  L.total = off + 256;
  return L;
}

// Rows of the products' tiles.  Up to 12 rows a slot on average (fp32: 32) the weights' stream is what counts: 8 slots of 4096 x 4096, us by thin / large tiles, 64 rows
// 31.8 / 40.2, 128 rows 43.9 / 40.4; fp32, 2048 x 2048, 256 rows 18.5 / 27.  Tiles of 128 rows where there are so few that each has a unit of its own (1000 rows, 1024 x
// 1024: 16.5 -> 11.9 against 256; 2048 rows in 8 slots of 4096 x 4096, where they would be a round and a quarter, 71 against 55).
static int tile_rows(const symi_ctx* ctx, int R, bool expert) {
  const symi_cfg* const c = &ctx->cfg;
  const long long A = (long long)c->T * c->k;
  if (A <= (c->dtype == SYMI_F32 ? 32LL : 12LL) * c->S_tot) return THIN;
  if (c->dtype == SYMI_F32) return 128;
  return (A / 128 + c->S_tot / 2) * cdiv(R, expert ? 128 : 256) <= ctx->cus ? 128 : 256;
}

// Whether a launch holds a product's tiles: columns of the thin ones are a grid's second coordinate; the large ones are workgroups of 256 threads in one dimension,
// which ends at 2^32 threads.  (No such product fits the memory: 2^24 tiles are 0.5 TB of weights or a result of 1 TB.)
static int tiles_fit(const symi_ctx* ctx, int rows, int R, bool expert, const char* who) {
  const symi_cfg* const c = &ctx->cfg;
  const long long tiles = ((long long)c->T * c->k / rows + c->S_tot) * cdiv(R, expert || c->dtype == SYMI_F32 ? 128 : 256);
  const bool fit = rows == THIN ? cdiv(R, expert ? 128 : 64) <= 65535 : tiles < (1 << 24) - 8;
  if (fit) return SYMI_OK;
  set_error("%s: more tiles than a launch can have", who);
  return SYMI_EUNSUPPORTED;
}

static void launch_tiles(const symi_ctx* ctx, int rows, const int32_t* offs, int32_t* map, hipStream_t st) {
  const int S = ctx->cfg.S_tot;
  if (rows == 256) SYMI_TIMED(ctx, K_TILES8, st, (tiles8_kernel<256><<<1, 1024, 0, st>>>(offs, S, map)));
  else if (rows == 128) SYMI_TIMED(ctx, K_TILES8, st, (tiles8_kernel<128><<<1, 1024, 0, st>>>(offs, S, map)));
  else if (S > FIND_SLOTS) SYMI_TIMED(ctx, K_TILES8, st, (tiles8_kernel<THIN><<<1, 1024, 0, st>>>(offs, S, map)));
}

static void launch_product(const symi_ctx* ctx, const Product8& p, int rows, bool expert, hipStream_t st) {
  if (rows > THIN) return launch_gemm8(ctx, p, rows, expert, st);
  const int tiles = ctx->cfg.T * ctx->cfg.k / THIN + ctx->cfg.S_tot;
  if (expert)
    SYMI_TIMED(ctx, K_EXPERT8, st, (thin_product_kernel<true, true><<<dim3(tiles, cdiv(p.R, 128)), Thin<true>::THREADS, 0, st>>>(p)));
  else if (ctx->cfg.dtype == SYMI_BF16)
    SYMI_TIMED(ctx, K_PRODUCT8, st, (thin_product_kernel<true, false><<<dim3(tiles, cdiv(p.R, 64)), Thin<false>::THREADS, 0, st>>>(p)));
  else
    SYMI_TIMED(ctx, K_PRODUCT8, st, (thin_product_kernel<false, false><<<dim3(tiles, cdiv(p.R, 64)), Thin<false>::THREADS, 0, st>>>(p)));
}

static void launch_quant_rows(const symi_ctx* ctx, bool bf16, const void* X, void* q, void* s, long long rows, int n, const int32_t* limit,
                              hipStream_t st) {
  const int sp = scale_pitch8(n);
  const int grid = (int)std::min<long long>((rows * sp + 15) / 16, 1 << 20);
  if (bf16)
    SYMI_TIMED(ctx, K_QUANT8, st, (quant_rows_kernel<true><<<grid, Q_THREADS, 0, st>>>(X, (uint8_t*)q, (uint8_t*)s, rows, n, pitch8(n), sp, limit)));
  else
    SYMI_TIMED(ctx, K_QUANT8, st, (quant_rows_kernel<false><<<grid, Q_THREADS, 0, st>>>(X, (uint8_t*)q, (uint8_t*)s, rows, n, pitch8(n), sp, limit)));
}

static int check_codes(const void* q, const void* s, const char* who) {
  SYMI_REQUIRE(((size_t)q & 15) == 0, who, "codes must be 16-byte aligned");
  SYMI_REQUIRE(((size_t)s & 3) == 0, who, "scales must be 4-byte aligned");
  return SYMI_OK;
}

static int check_values(int groups, int rows, int n, int block, const char* who) {
  SYMI_REQUIRE(groups >= 0 && rows >= 0, who, "negative number of groups or rows");
  SYMI_REQUIRE(n >= 8 && n % 8 == 0 && n <= MAX_N8, who, "n must be a multiple of 8, from 8 to 2^22");
  SYMI_REQUIRE(block == 1 || block == QB, who, "block must be 1 or 128");
  if ((long long)groups * rows > 0x7fffffffLL) {
    set_error("%s: more than 2^31 - 1 rows", who);
    return SYMI_EUNSUPPORTED;
  }
  return SYMI_OK;
}

}  // namespace symi

using namespace symi;

extern "C" int symi_pitch8(int n) {
  if (check_values(1, 1, n, 1, "symi_pitch8")) return SYMI_EINVAL;
  return pitch8(n);
}
extern "C" int symi_scale_pitch8(int n) {
  if (check_values(1, 1, n, 1, "symi_scale_pitch8")) return SYMI_EINVAL;
  return scale_pitch8(n);
}

extern "C" size_t symi_workspace8_bytes(const symi_cfg* cfg) {
  if (check_cfg(cfg, "symi_workspace8_bytes") != SYMI_OK) return 0;
  return ws8_layout(cfg).total;
}

extern "C" int symi_quant8(const symi_ctx* ctx, const void* X, int groups, int rows, int n, int block, void* q, void* s, void* stream) {
  SYMI_ENTER(ctx, "symi_quant8");
  if (int rc = check_values(groups, rows, n, block, "symi_quant8")) return rc;
  if (groups == 0 || rows == 0) return SYMI_OK;
  SYMI_REQUIRE(X && q && s, "symi_quant8", "NULL pointer");
  if (int rc = check_codes(q, s, "symi_quant8")) return rc;
  hipStream_t st = as_stream(stream);
  const bool bf16 = cfg->dtype == SYMI_BF16;
  if (block == 1) {
    launch_quant_rows(ctx, bf16, X, q, s, (long long)groups * rows, n, nullptr, st);
  } else {
    const int sp = scale_pitch8(n), rb = cdiv(rows, QB);
    const long long blocks = (long long)groups * rb * sp;
    if (blocks > 0x7fffffffLL) {
      set_error("symi_quant8: more than 2^31 - 1 blocks");
      return SYMI_EUNSUPPORTED;
    }
    if (bf16)
      SYMI_TIMED(ctx, K_QUANT8, st, (quant_blocks_kernel<true><<<flat_grid(blocks), Q_THREADS, 0, st>>>(X, (uint8_t*)q, (uint8_t*)s, rows, n, pitch8(n), sp, rb, (unsigned)blocks)));
    else
      SYMI_TIMED(ctx, K_QUANT8, st, (quant_blocks_kernel<false><<<flat_grid(blocks), Q_THREADS, 0, st>>>(X, (uint8_t*)q, (uint8_t*)s, rows, n, pitch8(n), sp, rb, (unsigned)blocks)));
  }
  SYMI_LAUNCH_CHECK("symi_quant8");
  return SYMI_OK;
}

extern "C" int symi_dequant8(const symi_ctx* ctx, const void* q, const void* s, int groups, int rows, int n, int block, void* X, void* stream) {
  SYMI_ENTER(ctx, "symi_dequant8");
  if (int rc = check_values(groups, rows, n, block, "symi_dequant8")) return rc;
  if (groups == 0 || rows == 0) return SYMI_OK;
  SYMI_REQUIRE(X && q && s, "symi_dequant8", "NULL pointer");
  if (int rc = check_codes(q, s, "symi_dequant8")) return rc;
  hipStream_t st = as_stream(stream);
  const int sp = scale_pitch8(n), rb = cdiv(rows, block);
  const long long pieces = (long long)groups * rows * (n / 8);
  const int grid = (int)std::min<long long>((pieces + Q_THREADS - 1) / Q_THREADS, 1 << 20);
  if (cfg->dtype == SYMI_BF16)
    SYMI_TIMED(ctx, K_DEQUANT8, st, (dequant_kernel<true><<<grid, Q_THREADS, 0, st>>>((const uint8_t*)q, (const uint8_t*)s, X, groups, rows, n, pitch8(n), sp, rb, block)));
  else
    SYMI_TIMED(ctx, K_DEQUANT8, st, (dequant_kernel<false><<<grid, Q_THREADS, 0, st>>>((const uint8_t*)q, (const uint8_t*)s, X, groups, rows, n, pitch8(n), sp, rb, block)));
  SYMI_LAUNCH_CHECK("symi_dequant8");
  return SYMI_OK;
}

extern "C" int symi_product8(const symi_ctx* ctx, const void* Aq, const void* As, const int32_t* slot_offsets, const void* Wq, const void* Ws,
                             int R, int n, void* Y, void* ws, void* stream) {
  SYMI_ENTER(ctx, "symi_product8");
  if (int rc = check_values(1, R, n, 1, "symi_product8")) return rc;
  SYMI_REQUIRE(R >= 8 && R % 8 == 0 && R <= MAX_N8, "symi_product8", "R must be a multiple of 8, from 8 to 2^22");
  if (cfg->T == 0) return SYMI_OK;
  SYMI_REQUIRE(Aq && As && slot_offsets && Wq && Ws && Y && ws, "symi_product8", "NULL pointer");
  if (int rc = check_codes(Aq, As, "symi_product8")) return rc;
  if (int rc = check_codes(Wq, Ws, "symi_product8")) return rc;
  hipStream_t st = as_stream(stream);
  int32_t* const map = reinterpret_cast<int32_t*>(align_up((size_t)ws, 256) + ws8_layout(cfg).map);
  const int tile = tile_rows(ctx, R, false);
  if (int rc = tiles_fit(ctx, tile, R, false, "symi_product8")) return rc;
  launch_tiles(ctx, tile, slot_offsets, map, st);
  const Product8 p = {(const uint8_t*)Aq, (const uint8_t*)As, (const uint8_t*)Wq, (const uint8_t*)Ws, slot_offsets, map, Y,
                      nullptr, nullptr, nullptr, nullptr, R, pitch8(n), scale_pitch8(n), 0, 0, cfg->S_tot};
  launch_product(ctx, p, tile, false, st);
  SYMI_LAUNCH_CHECK("symi_product8");
  return SYMI_OK;
}

extern "C" int symi_expert_fwd8(const symi_ctx* ctx, const void* Xp, const int32_t* slot_offsets, const void* W1q, const void* W1s, const void* W2q,
                                const void* W2s, void* UV, void* H, void* Yp, void* ws, void* stream) {
  SYMI_ENTER(ctx, "symi_expert_fwd8");
  if (cfg->dtype != SYMI_BF16) {
    set_error("symi_expert_fwd8: 8-bit experts need a bf16 context");
    return SYMI_EUNSUPPORTED;
  }
  SYMI_REQUIRE((UV != nullptr) == (H != nullptr), "symi_expert_fwd8", "UV and H: both or neither");
  if (cfg->T == 0) return SYMI_OK;
  SYMI_REQUIRE(Xp && slot_offsets && W1q && W1s && W2q && W2s && Yp && ws, "symi_expert_fwd8", "NULL pointer");
  if (int rc = check_codes(W1q, W1s, "symi_expert_fwd8")) return rc;
  if (int rc = check_codes(W2q, W2s, "symi_expert_fwd8")) return rc;
  hipStream_t st = as_stream(stream);
  const Ws8 L = ws8_layout(cfg);
  uint8_t* const base = reinterpret_cast<uint8_t*>(align_up((size_t)ws, 256));
  const int d = cfg->d, f = cfg->f, A = cfg->T * cfg->k;
  int32_t* const map = reinterpret_cast<int32_t*>(base + L.map);
  const int tile = std::max(tile_rows(ctx, f, true), tile_rows(ctx, d, false));
  if (int rc = tiles_fit(ctx, tile, f, true, "symi_expert_fwd8")) return rc;
  if (int rc = tiles_fit(ctx, tile, d, false, "symi_expert_fwd8")) return rc;
  launch_tiles(ctx, tile, slot_offsets, map, st);
  launch_quant_rows(ctx, true, Xp, base + L.xq, base + L.xs, A, d, slot_offsets + cfg->S_tot, st);
  Product8 p = {base + L.xq, base + L.xs, (const uint8_t*)W1q, (const uint8_t*)W1s, slot_offsets, map, nullptr, (uint16_t*)UV, (uint16_t*)H,
                base + L.hq, base + L.hs, f, pitch8(d), scale_pitch8(d), pitch8(f), scale_pitch8(f), cfg->S_tot};
  launch_product(ctx, p, tile, true, st);
  p.Aq = base + L.hq;
  p.As = base + L.hs;
  p.Wq = (const uint8_t*)W2q;
  p.Ws = (const uint8_t*)W2s;
  p.Y = Yp;
  p.R = d;
  p.p8 = pitch8(f);
  p.sp = scale_pitch8(f);
  launch_product(ctx, p, tile, false, st);
  SYMI_LAUNCH_CHECK("symi_expert_fwd8");
  return SYMI_OK;
}
