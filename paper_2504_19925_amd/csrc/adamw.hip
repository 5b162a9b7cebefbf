// symi_adamw_*: AdamW over many tensors in one launch, states in 32 bits or in 8 bits with a scale for every 256 values.
//
// symi_adamw_create cuts the tensors into chunks and writes the list into the caller's table; a workgroup takes one chunk,
// so the number of tensors costs nothing.  A block of 256 values is one wavefront, four values a lane.
//
// 8-bit states: m = a sign(c) (c / 127)^2 and v = a (c / 255)^4 with a the largest |value| of the block.  Codes lie closer
// where values are small: m reaches down to 6e-5 of a block's largest, v to 2e-10 (its root, which the update divides by,
// to 1.5e-5), at steps of 1.6 % near the top.  v moves by 1 - beta2 = 0.1 % a step, so rounding to the nearest code
// would hold it where it is; instead a value x between the neighbours lo and hi becomes hi with probability
// (x - lo) / (hi - lo), which keeps the mean.  v > 0 never becomes 0: the next step's m would be divided by eps alone.
// Values, codes and the comparison with the random number are single operations in a fixed order (no contraction), so that
// which code is taken does not depend on how the compiler fuses them.
#include <math.h>

#include <algorithm>
#include <new>
#include <type_traits>
#include <vector>

#include "common.h"

namespace symi {

constexpr uint32_t ADAMW_MAGIC = 0x41444d57u;
constexpr int ADAMW_BLOCK = 256;     // values that share a scale
constexpr int ADAMW_THREADS = 256;
constexpr int ADAMW_CHUNK = 4096;    // values of one workgroup
constexpr float SMALLEST = 1.17549435e-38f;
constexpr int POSITIVE_DENORMAL = 1 << 7;   // class of a number
constexpr float M_UNIT = (float)(1.0 / (127 * 127)), V_UNIT = (float)(1.0 / (255 * 255));

struct AdamwTensor {   // on the device
  void* param;
  float* master;
  const void* grad;
  void *m, *v;
  float *m_scale, *v_scale;
  long long n;
  unsigned first_block;   // of the tensor among all blocks: its place in the random numbers and the decoded states
  float decay;
  int kind;               // bit 0: bf16 param, 1: bf16 gradient, 2: 8-bit states
};
// Work of a workgroup: ADAMW_CHUNK values (four blocks a wavefront), or, of what a tensor has behind its last whole chunk, one block
// a wavefront: a small tensor or a ragged end is then as many workgroups and no chain of rounds.
struct AdamwChunk {
  int tensor;
  unsigned block;   // the first one; WHOLE: a whole chunk
};
constexpr unsigned WHOLE = 0x80000000u;
// So few values in all that none of it is cut into whole chunks, as their rounds would leave units idle.  us, whole chunks : one
// block a wavefront, 8-bit states: 0.2 million values 7.2 : 4.8, 1.6 million 12.7 : 9.6, 6.3 million 26.1 : 25.2, 12.5 million 40.8 :
// 43.9, 20.9 million 72.9 : 91.9; 32-bit ones 4.4 : 3.9, 9.9 : 9.4, 27.3 : 28.0, 70.5 : 67.0.
constexpr long long FINE_BELOW = 1LL << 23;

struct AdamwScalars {
  float lr, beta1, keep1, beta2, keep2, eps, wd, gscale, fix1, fix2, root2;
  uint32_t key;
};

__host__ __device__ inline uint32_t mix(uint32_t x) {
  x ^= x >> 16;
  x *= 0xBB67AE85u;
  x ^= x >> 15;
  x *= 0x6A09E667u;
  return x ^ (x >> 16);
}

__device__ __forceinline__ float m_value(float c, float a) {   // of a code with its sign
#pragma clang fp contract(off)
  return c * fabsf(c) * M_UNIT * a;
}
__device__ __forceinline__ float v_value(float c, float a) {
#pragma clang fp contract(off)
  const float q = c * c * V_UNIT;
  return q * q * a;
}

// The code of x >= 0 in a block of scale a (normal and finite): lo is the largest code but the last whose value is at
// most x.  guess is within one of it.
template <class Value>
__device__ __forceinline__ float code_between(float x, float a, float guess, float top, float u, Value value) {
#pragma clang fp contract(off)
  float lo = fminf(floorf(guess), top - 1.f);
  float below = value(lo, a), above = value(lo + 1.f, a);
  const bool under = below > x, over = above <= x && lo < top - 1.f;
  if (__builtin_expect(__ballot(under || over) != 0, 0)) {   // about one block in forty
    lo += under ? -1.f : over ? 1.f : 0.f;
    below = value(lo, a);
    above = value(lo + 1.f, a);
  }
  return x - below > u * (above - below) ? lo + 1.f : lo;
}

// Bits of the largest |value| of a wavefront: of floats without their sign the order is that of their bits, NaN on top.
template <int CTRL>
__device__ __forceinline__ uint32_t max_with(uint32_t x) {
  const uint32_t y = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, CTRL, 0xf, 0xf, true);
  return x > y ? x : y;
}
__device__ __forceinline__ uint32_t wave_max(uint32_t x) {
  x = max_with<0xb1>(x);    // lanes 1, 0, 3, 2 of four
  x = max_with<0x4e>(x);    // 2, 3, 0, 1
  x = max_with<0x141>(x);   // eight mirrored
  x = max_with<0x140>(x);   // sixteen mirrored
  x = max_with<0x142>(x);   // the last lane of each sixteen to the next sixteen
  x = max_with<0x143>(x);   // lane 31 to the upper half
  return (uint32_t)__builtin_amdgcn_readlane((int)x, 63);
}
// 0 for a block of nothing but denormal numbers, NaN for one that is not finite
__device__ __forceinline__ float scale_of(uint32_t bits) {
  return bits < 0x00800000u ? 0.f : bits < 0x7f800000u ? __uint_as_float(bits) : __uint_as_float(0x7fc00000u);
}

// Four values of a lane, as they lie in memory at any alignment.
typedef uint32_t u32x2_bf16 __attribute__((ext_vector_type(2), aligned(2)));
typedef uint32_t u32_codes __attribute__((aligned(1)));
template <bool BF16> struct Four {
  using Vec = std::conditional_t<BF16, u32x2_bf16, f32x4_f32>;
  using Elem = std::conditional_t<BF16, uint16_t, float>;
  static __device__ __forceinline__ Vec load(const void* p, long long at) { return *reinterpret_cast<const Vec*>(static_cast<const Elem*>(p) + at); }
  static __device__ __forceinline__ void store(void* p, long long at, const float (&x)[4]) {
    Vec v;
    if constexpr (BF16) {
      v[0] = pack_bf16x2(x[0], x[1]);
      v[1] = pack_bf16x2(x[2], x[3]);
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i) v[i] = x[i];
    }
    *reinterpret_cast<Vec*>(static_cast<Elem*>(p) + at) = v;
  }
  static __device__ __forceinline__ void unpack(Vec v, float (&x)[4]) {
    if constexpr (BF16) {
      x[0] = __uint_as_float(v[0] << 16);
      x[1] = __uint_as_float(v[0] & 0xffff0000u);
      x[2] = __uint_as_float(v[1] << 16);
      x[3] = __uint_as_float(v[1] & 0xffff0000u);
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i) x[i] = v[i];
    }
  }
  // the first `n` of them (the others 0), and back
  static __device__ __forceinline__ Vec load_some(const void* p, long long at, long long n) {
    const Elem* const q = static_cast<const Elem*>(p) + at;
    Vec v;
    if constexpr (BF16) {
      v[0] = (n > 0 ? q[0] : 0u) | (n > 1 ? q[1] : 0u) << 16;
      v[1] = (n > 2 ? q[2] : 0u) | (n > 3 ? q[3] : 0u) << 16;
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i) v[i] = i < n ? q[i] : 0.f;
    }
    return v;
  }
  static __device__ __forceinline__ void store_some(void* p, long long at, long long n, const float (&x)[4]) {
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (i < n) {
        if constexpr (BF16) static_cast<uint16_t*>(p)[at + i] = f32_to_bf16(x[i]); else static_cast<float*>(p)[at + i] = x[i];
      }
  }
};
__device__ __forceinline__ uint32_t load_codes(const void* p, long long at) { return *reinterpret_cast<const u32_codes*>(static_cast<const uint8_t*>(p) + at); }
__device__ __forceinline__ uint32_t load_codes_some(const void* p, long long at, long long n) {
  uint32_t x = 0;
#pragma unroll
  for (int i = 0; i < 4; ++i) x |= (i < n ? (uint32_t)static_cast<const uint8_t*>(p)[at + i] : 0u) << (8 * i);
  return x;
}
__device__ __forceinline__ void store_codes(void* p, long long at, uint32_t x) { *reinterpret_cast<u32_codes*>(static_cast<uint8_t*>(p) + at) = x; }
__device__ __forceinline__ void store_codes_some(void* p, long long at, long long n, uint32_t x) {
#pragma unroll
  for (int i = 0; i < 4; ++i)
    if (i < n) static_cast<uint8_t*>(p)[at + i] = (uint8_t)(x >> (8 * i));
}
__device__ __forceinline__ void decode(uint32_t mc, uint32_t vc, float am, float av, float (&m)[4], float (&v)[4]) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const float cm = (float)((int)(mc << (24 - 8 * i)) >> 24);
    m[i] = m_value(cm, am);
    v[i] = v_value((float)(vc >> (8 * i) & 255u), av);
  }
}

// What a lane holds of a block.
template <bool PARAM16, bool GRAD16, bool CODES>
struct AdamwBlock {
  typename Four<GRAD16>::Vec g;
  f32x4_f32 w, m, v;
  uint32_t mc, vc;
  float am, av;

  // left: how many of the lane's four values the tensor has (4 or more: all); FULL: all lanes' are there
  template <bool FULL>
  __device__ __forceinline__ void load(const AdamwTensor& t, long long block, long long at, long long left) {
    const void* const weights = PARAM16 ? (const void*)t.master : t.param;
    if (FULL) {
      g = Four<GRAD16>::load(t.grad, at);
      w = Four<false>::load(weights, at);
    } else {
      g = Four<GRAD16>::load_some(t.grad, at, left);
      w = Four<false>::load_some(weights, at, left);
    }
    if (CODES) {
      mc = FULL ? load_codes(t.m, at) : load_codes_some(t.m, at, left);
      vc = FULL ? load_codes(t.v, at) : load_codes_some(t.v, at, left);
      am = t.m_scale[block];
      av = t.v_scale[block];
    } else {
      m = FULL ? Four<false>::load(t.m, at) : Four<false>::load_some(t.m, at, left);
      v = FULL ? Four<false>::load(t.v, at) : Four<false>::load_some(t.v, at, left);
    }
  }

  template <bool FULL>
  __device__ __forceinline__ void step(const AdamwTensor& t, const AdamwScalars& h, float gscale, float wd, long long block, long long at,
                                       long long left, int lane) {
    float g_[4], w_[4], m_[4], v_[4], root[4];
    Four<GRAD16>::unpack(g, g_);
    Four<false>::unpack(w, w_);
    if (CODES) {
      decode(mc, vc, am, av, m_, v_);
    } else {
      Four<false>::unpack(m, m_);
      Four<false>::unpack(v, v_);
    }
    uint32_t big_m = 0, big_v = 0;
    {
#pragma clang fp contract(off)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float gr = g_[i] * gscale;
        m_[i] = m_[i] * h.beta1 + gr * h.keep1;
        v_[i] = v_[i] * h.beta2 + gr * h.keep2 * gr;
        if (CODES) {
          big_m = max(big_m, __float_as_uint(m_[i]) & 0x7fffffffu);
          big_v = max(big_v, __float_as_uint(v_[i]));   // never below 0; a NaN of any sign is on top
        }
      }
    }
    // Codes are bound by arithmetic: the instructions for root and reciprocal, each within one unit in the last place.  They take denormal
    // numbers for 0 (v of gradients below 1e-17 is one, and a denormal eps): there, as with 32-bit states, the functions.
    bool denormal = CODES && h.eps < SMALLEST;
    if (CODES) {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        root[i] = __builtin_amdgcn_sqrtf(v_[i]);
        denormal |= __builtin_amdgcn_classf(v_[i], POSITIVE_DENORMAL);
      }
    }
    if (CODES && __builtin_expect(__ballot(denormal) == 0, 1)) {
#pragma unroll
      for (int i = 0; i < 4; ++i) w_[i] -= h.lr * (m_[i] * h.fix1 * __builtin_amdgcn_rcpf(fmaf(root[i], h.root2, h.eps)) + wd * w_[i]);
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        w_[i] -= h.lr * (m_[i] * h.fix1 / (sqrtf(v_[i] * h.fix2) + h.eps) + wd * w_[i]);
        if (CODES) root[i] = sqrtf(v_[i]);
      }
    }
    if (FULL) {
      Four<false>::store(PARAM16 ? (void*)t.master : t.param, at, w_);
      if (PARAM16) Four<true>::store(t.param, at, w_);
      if (!CODES) {
        Four<false>::store(t.m, at, m_);
        Four<false>::store(t.v, at, v_);
      }
    } else {
      Four<false>::store_some(PARAM16 ? (void*)t.master : t.param, at, left, w_);
      if (PARAM16) Four<true>::store_some(t.param, at, left, w_);
      if (!CODES) {
        Four<false>::store_some(t.m, at, left, m_);
        Four<false>::store_some(t.v, at, left, v_);
      }
    }
    if (!CODES) return;
    const float am_ = scale_of(wave_max(big_m)), av_ = scale_of(wave_max(big_v));
    // the guesses: 127 sqrt(|m| / am), and 255 sqrt(root / sqrt(av)), as root is sqrt(v)
    const float to_m = 1.f / am_, to_v = 255.f * 255.f * __builtin_amdgcn_rsqf(av_);
    const uint32_t r0 = mix(((t.first_block + (unsigned)block) * 64u + lane) * 0x9E3779B1u + h.key);
    const uint32_t times[4] = {0x3C6EF373u, 0xA54FF53Bu, 0x510E527Fu, 0x9B05688Du};
    uint32_t mc_ = 0, vc_ = 0;
    if (am_ > 0.f) {   // the same in all lanes
      uint32_t c[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        uint32_t r = r0 * times[i];
        r ^= r >> 15;
        const float u = fmaf((float)(r & 0xffffu), 0x1p-16f, 0x1p-17f), x = fabsf(m_[i]);
        c[i] = (uint32_t)(int)copysignf(code_between(x, am_, 127.f * __builtin_amdgcn_sqrtf(x * to_m), 127.f, u, m_value), m_[i]);
      }
      // the lowest byte of each
      mc_ = __builtin_amdgcn_perm(__builtin_amdgcn_perm(c[3], c[2], 0x0c0c0400u), __builtin_amdgcn_perm(c[1], c[0], 0x0c0c0400u), 0x05040100u);
    }
    if (av_ > 0.f) {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        uint32_t r = r0 * times[i];
        r ^= r >> 15;
        const float u = fmaf((float)(r >> 16), 0x1p-16f, 0x1p-17f);
        const float c = code_between(v_[i], av_, __builtin_amdgcn_sqrtf(root[i] * to_v), 255.f, u, v_value);
        vc_ = __builtin_amdgcn_cvt_pk_u8_f32(v_[i] > 0.f ? fmaxf(c, 1.f) : 0.f, i, vc_);
      }
    }
    if (FULL) {
      store_codes(t.m, at, mc_);
      store_codes(t.v, at, vc_);
    } else {
      store_codes_some(t.m, at, left, mc_);
      store_codes_some(t.v, at, left, vc_);
    }
    if (lane == 0) {
      t.m_scale[block] = am_;
      t.v_scale[block] = av_;
    }
  }
};

constexpr int ADAMW_WAVES = ADAMW_THREADS / 64, ADAMW_ROUNDS = ADAMW_CHUNK / ADAMW_BLOCK / ADAMW_WAVES;

// A wavefront's blocks of a chunk, all loads first.
template <bool PARAM16, bool GRAD16, bool CODES>
__device__ __forceinline__ void adamw_chunk(const AdamwTensor& t, const AdamwScalars& h, float gscale, bool whole, long long first, int lane) {
  const float wd = t.decay * h.wd;
  if (whole) {
    AdamwBlock<PARAM16, GRAD16, CODES> b[ADAMW_ROUNDS];
#pragma unroll
    for (int k = 0; k < ADAMW_ROUNDS; ++k) b[k].template load<true>(t, first + k * ADAMW_WAVES, (first + k * ADAMW_WAVES) * ADAMW_BLOCK + lane * 4, 4);
#pragma unroll
    for (int k = 0; k < ADAMW_ROUNDS; ++k)
      b[k].template step<true>(t, h, gscale, wd, first + k * ADAMW_WAVES, (first + k * ADAMW_WAVES) * ADAMW_BLOCK + lane * 4, 4, lane);
    return;
  }
  const long long at = first * ADAMW_BLOCK + lane * 4;
  if (first * ADAMW_BLOCK >= t.n) return;
  AdamwBlock<PARAM16, GRAD16, CODES> b;
  if ((first + 1) * ADAMW_BLOCK <= t.n) {
    b.template load<true>(t, first, at, 4);
    b.template step<true>(t, h, gscale, wd, first, at, 4, lane);
  } else {
    b.template load<false>(t, first, at, t.n - at);
    b.template step<false>(t, h, gscale, wd, first, at, t.n - at, lane);
  }
}

// Bound by memory with 32-bit states: 202 million values, bf16 weights with masters, 1131 us, 3.24 GB fetched and 2.83 written (5.4 TB/s).  With
// 8-bit ones by memory and vector instructions alike: 539 million 1540 to 1590 us, 5.46 and 3.26 GB (5.6 TB/s), units busy all the time;
// 26 million with bf16 gradients 77 us.  Five wavefronts a SIMD instead of four: 2 % less with bf16 gradients, 4 % more with fp32 ones.
__global__ __launch_bounds__(ADAMW_THREADS) void adamw_kernel(const AdamwTensor* __restrict__ tensors,
                                                              const AdamwChunk* __restrict__ chunks, AdamwScalars h,
                                                              const float* __restrict__ grad_scale) {
  const AdamwChunk c = chunks[blockIdx.x];
  const AdamwTensor t = tensors[c.tensor];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const float gscale = grad_scale ? h.gscale * grad_scale[0] : h.gscale;
  const long long first = (c.block & ~WHOLE) + wave;
  const bool whole = c.block & WHOLE;
  switch (t.kind) {
    case 0: adamw_chunk<false, false, false>(t, h, gscale, whole, first, lane); break;
    case 1: adamw_chunk<true, false, false>(t, h, gscale, whole, first, lane); break;
    case 2: adamw_chunk<false, true, false>(t, h, gscale, whole, first, lane); break;
    case 3: adamw_chunk<true, true, false>(t, h, gscale, whole, first, lane); break;
    case 4: adamw_chunk<false, false, true>(t, h, gscale, whole, first, lane); break;
    case 5: adamw_chunk<true, false, true>(t, h, gscale, whole, first, lane); break;
    case 6: adamw_chunk<false, true, true>(t, h, gscale, whole, first, lane); break;
    default: adamw_chunk<true, true, true>(t, h, gscale, whole, first, lane);
  }
}

// A chunk is `parts` workgroups: two of two rounds each where there are whole chunks (539 million values 968 -> 908 us, 6.0 TB/s,
// 26 million 54.8 -> 51.0; four of one round 918 and 52.2), else one of one (6.3 million 11.6 us, 16.8 beside idle ones).
constexpr int DECODE_ROUNDS = 2;
__global__ __launch_bounds__(ADAMW_THREADS) void adamw_decode_kernel(const AdamwTensor* __restrict__ tensors,
                                                                     const AdamwChunk* __restrict__ chunks, int parts, unsigned groups,
                                                                     float* __restrict__ m_out, float* __restrict__ v_out) {
  const unsigned group = blockIdx.y * gridDim.x + blockIdx.x;
  if (group >= groups) return;
  const AdamwChunk c = chunks[group / (unsigned)parts];
  const unsigned part = group % (unsigned)parts;
  if (part && !(c.block & WHOLE)) return;
  const AdamwTensor t = tensors[c.tensor];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
#pragma unroll
  for (int k = 0; k < DECODE_ROUNDS; ++k) {
    if (k && !(c.block & WHOLE)) return;
    const long long block = (c.block & ~WHOLE) + (long long)(part * DECODE_ROUNDS + k) * ADAMW_WAVES + wave;
    const long long at = block * ADAMW_BLOCK + lane * 4, to = (long long)t.first_block * ADAMW_BLOCK + at, left = t.n - at;
    if (left <= 0) return;
    float m[4], v[4];
    if (t.kind & 4) {
      const bool all = left >= 4;
      decode(all ? load_codes(t.m, at) : load_codes_some(t.m, at, left), all ? load_codes(t.v, at) : load_codes_some(t.v, at, left),
             t.m_scale[block], t.v_scale[block], m, v);
    } else {
      Four<false>::unpack(Four<false>::load_some(t.m, at, left), m);
      Four<false>::unpack(Four<false>::load_some(t.v, at, left), v);
    }
    if (left >= 4) {
      Four<false>::store(m_out, to, m);
      Four<false>::store(v_out, to, v);
    } else {
      Four<false>::store_some(m_out, to, left, m);
      Four<false>::store_some(v_out, to, left, v);
    }
  }
}

}  // namespace symi

struct symi_adamw {
  uint32_t magic;
  int device;
  long long chunks, values;
  const symi::AdamwTensor* tensors;   // in the caller's table, the chunks behind them
  const symi::AdamwChunk* list;
  bool fine;   // no whole chunks
};

using namespace symi;

static int enter_adamw(const symi_ctx* ctx, const symi_adamw* opt, const char* who) {
  SYMI_ENTER(ctx, who);
  (void)cfg;
  SYMI_REQUIRE(opt && opt->magic == ADAMW_MAGIC, who, "opt is NULL or not a live one of symi_adamw_create");
  SYMI_REQUIRE(opt->device == ctx->device, who, "opt was created on another device than the context");
  return SYMI_OK;
}

// Checks the tensors; sizes of the description, in elements of each kind.
struct AdamwSizes {
  long long tensors, chunks, blocks;
  bool fine;
  size_t list_at() const { return align_up((size_t)tensors * sizeof(AdamwTensor), 256); }
  size_t bytes() const { return list_at() + (size_t)chunks * sizeof(AdamwChunk) + 256; }
};
static int check_tensors(const char* who, const symi_adamw_tensor* tensors, int count, AdamwSizes* out) {
  SYMI_REQUIRE(count >= 0 && (tensors || count == 0), who, "count < 0 or no tensors");
  AdamwSizes n = {0, 0, 0, false};
  long long values = 0;
  for (int i = 0; i < count; ++i) {
    const symi_adamw_tensor& s = tensors[i];
    const auto bad = [&](bool cond, const char* msg) {
      if (cond) set_error("%s: tensor %d: %s", who, i, msg);
      return cond;
    };
    if (bad(s.n < 0, "n < 0") || bad(s.state_bits != 32 && s.state_bits != 8, "state_bits must be 32 or 8") ||
        bad(s.param_dtype != SYMI_F32 && s.param_dtype != SYMI_BF16, "param_dtype must be SYMI_F32 or SYMI_BF16") ||
        bad(s.grad_dtype != SYMI_F32 && s.grad_dtype != SYMI_BF16, "grad_dtype must be SYMI_F32 or SYMI_BF16") ||
        bad(!(s.decay >= 0.f), "decay must be >= 0") ||
        bad(s.n && !(s.param && s.grad && s.m && s.v), "NULL pointer") ||
        bad(s.n && (s.param_dtype == SYMI_BF16) != (s.master != nullptr), "a bf16 param needs its master, an fp32 one has none") ||
        bad(s.n && ((s.state_bits == 8) != (s.m_scale != nullptr) || (s.state_bits == 8) != (s.v_scale != nullptr)),
            "8-bit states need their scales, 32-bit ones have none"))
      return SYMI_EINVAL;
    if (s.n >> 36 || (n.blocks += (s.n + ADAMW_BLOCK - 1) / ADAMW_BLOCK) > 1LL << 28) {
      set_error("%s: more than 2^28 blocks of 256 values", who);
      return SYMI_EUNSUPPORTED;
    }
    values += s.n;
  }
  n.fine = values < FINE_BELOW;
  for (int i = 0; i < count; ++i) {
    const long long whole = n.fine ? 0 : tensors[i].n / ADAMW_CHUNK, rest = tensors[i].n - whole * ADAMW_CHUNK;
    n.tensors += tensors[i].n > 0;
    n.chunks += whole + (rest + ADAMW_WAVES * ADAMW_BLOCK - 1) / (ADAMW_WAVES * ADAMW_BLOCK);
  }
  if (n.chunks >= 1LL << 24) {   // a workgroup each; the threads of a launch end at 2^32
    set_error("%s: more than 2^24 - 1 chunks of up to %d values", who, ADAMW_CHUNK);
    return SYMI_EUNSUPPORTED;
  }
  *out = n;
  return SYMI_OK;
}

extern "C" size_t symi_adamw_table_bytes(const symi_adamw_tensor* tensors, int count) {
  AdamwSizes n;
  return check_tensors("symi_adamw_table_bytes", tensors, count, &n) == SYMI_OK ? n.bytes() : 0;
}

extern "C" int symi_adamw_create(const symi_adamw_tensor* tensors, int count, void* table, symi_adamw** out, void* stream) {
  const char* const who = "symi_adamw_create";
  SYMI_REQUIRE(out, who, "out is NULL");
  *out = nullptr;
  AdamwSizes n;
  if (int rc = check_tensors(who, tensors, count, &n)) return rc;
  SYMI_REQUIRE(table || n.chunks == 0, who, "table is NULL");
  int dev = -1;
  if (hipGetDevice(&dev) != hipSuccess) {
    (void)hipGetLastError();
    set_error("%s: no usable HIP device is current", who);
    return SYMI_EHIP;
  }
  char* const to = reinterpret_cast<char*>(align_up(reinterpret_cast<size_t>(table), 256));
  std::vector<char> copy;
  symi_adamw* opt = nullptr;
  try {
    copy.resize(n.list_at() + (size_t)n.chunks * sizeof(AdamwChunk));
    opt = new symi_adamw();
  } catch (const std::exception&) {
    set_error("%s: out of host memory", who);
    return SYMI_EHIP;
  }
  AdamwTensor* t = reinterpret_cast<AdamwTensor*>(copy.data());
  AdamwChunk* c = reinterpret_cast<AdamwChunk*>(copy.data() + n.list_at());
  unsigned block = 0;
  int index = 0;
  for (int i = 0; i < count; ++i) {
    const symi_adamw_tensor& s = tensors[i];
    if (s.n == 0) continue;
    *t++ = {s.param, s.master, s.grad, s.m, s.v, s.m_scale, s.v_scale, s.n, block, s.decay,
            (s.param_dtype == SYMI_BF16) | (s.grad_dtype == SYMI_BF16) << 1 | (s.state_bits == 8) << 2};
    long long at = 0;
    for (; !n.fine && at + ADAMW_CHUNK <= s.n; at += ADAMW_CHUNK) *c++ = {index, (unsigned)(at / ADAMW_BLOCK) | WHOLE};
    for (; at < s.n; at += ADAMW_WAVES * ADAMW_BLOCK) *c++ = {index, (unsigned)(at / ADAMW_BLOCK)};
    block += (unsigned)((s.n + ADAMW_BLOCK - 1) / ADAMW_BLOCK);
    ++index;
  }
  opt->device = dev;
  opt->chunks = n.chunks;
  opt->values = n.blocks * ADAMW_BLOCK;
  opt->fine = n.fine;
  opt->tensors = reinterpret_cast<const AdamwTensor*>(to);
  opt->list = reinterpret_cast<const AdamwChunk*>(to + n.list_at());
  if (n.chunks) {
    hipStream_t st = as_stream(stream);
    hipError_t e = hipMemcpyAsync(to, copy.data(), copy.size(), hipMemcpyHostToDevice, st);
    if (e == hipSuccess) e = hipStreamSynchronize(st);
    if (e != hipSuccess) {
      set_error("%s: %s", who, hipGetErrorString(e));
      (void)hipGetLastError();
      delete opt;
      return SYMI_EHIP;
    }
  }
  opt->magic = ADAMW_MAGIC;
  *out = opt;
  return SYMI_OK;
}

extern "C" int symi_adamw_destroy(symi_adamw* opt) {
  if (!opt) return SYMI_OK;
  SYMI_REQUIRE(opt->magic == ADAMW_MAGIC, "symi_adamw_destroy", "not a live one of symi_adamw_create");
  opt->magic = 0;
  delete opt;
  return SYMI_OK;
}

extern "C" long long symi_adamw_values(const symi_adamw* opt) {
  return opt && opt->magic == ADAMW_MAGIC ? opt->values : 0;
}

extern "C" int symi_adamw_step(const symi_ctx* ctx, const symi_adamw* opt, const symi_adam* hp, const float* grad_scale,
                               uint32_t seed, void* stream) {
  const char* const who = "symi_adamw_step";
  if (int rc = enter_adamw(ctx, opt, who)) return rc;
  SYMI_REQUIRE(hp, who, "NULL pointer");
  SYMI_REQUIRE(hp->step >= 1, who, "step must be >= 1");
  SYMI_REQUIRE(hp->beta1 >= 0.f && hp->beta1 < 1.f && hp->beta2 >= 0.f && hp->beta2 < 1.f, who, "betas must lie in [0, 1)");
  SYMI_REQUIRE(hp->eps > 0.f, who, "eps must be positive");
  if (!opt->chunks) return SYMI_OK;
  AdamwScalars h;
  h.lr = hp->lr; h.beta1 = hp->beta1; h.keep1 = 1.f - hp->beta1; h.beta2 = hp->beta2; h.keep2 = 1.f - hp->beta2;
  h.eps = hp->eps; h.wd = hp->weight_decay; h.gscale = hp->grad_scale;
  h.fix1 = (float)(1.0 / (1.0 - pow((double)hp->beta1, hp->step)));
  h.fix2 = (float)(1.0 / (1.0 - pow((double)hp->beta2, hp->step)));
  h.root2 = (float)sqrt(1.0 / (1.0 - pow((double)hp->beta2, hp->step)));
  h.key = mix(mix(seed) + (uint32_t)hp->step);
  hipStream_t st = as_stream(stream);
  SYMI_TIMED(ctx, K_ADAMW, st, (adamw_kernel<<<(unsigned)opt->chunks, ADAMW_THREADS, 0, st>>>(opt->tensors, opt->list, h, grad_scale)));
  SYMI_LAUNCH_CHECK(who);
  return SYMI_OK;
}

extern "C" int symi_adamw_decode(const symi_ctx* ctx, const symi_adamw* opt, float* m, float* v, void* stream) {
  const char* const who = "symi_adamw_decode";
  if (int rc = enter_adamw(ctx, opt, who)) return rc;
  if (!opt->chunks) return SYMI_OK;
  SYMI_REQUIRE(m && v, who, "NULL pointer");
  hipStream_t st = as_stream(stream);
  const int parts = opt->fine ? 1 : ADAMW_ROUNDS / DECODE_ROUNDS;
  // two dimensions beyond 2^20 workgroups: the threads of one end at 2^32, which two workgroups a chunk can reach
  const unsigned groups = (unsigned)opt->chunks * parts, across = std::min(groups, 1u << 20);
  SYMI_TIMED(ctx, K_ADAMW_DECODE, st, (adamw_decode_kernel<<<dim3(across, (groups + across - 1) / across), ADAMW_THREADS, 0, st>>>(
      opt->tensors, opt->list, parts, groups, m, v)));
  SYMI_LAUNCH_CHECK(who);
  return SYMI_OK;
}
