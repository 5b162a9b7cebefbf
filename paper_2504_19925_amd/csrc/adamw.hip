// symi_adamw_*: AdamW over many tensors in one launch, states in 32 bits or in 8 bits with a scale for every 256 values.
//
// symi_adamw_create cuts the tensors into chunks and keeps the list on the device; a workgroup takes one chunk, so the
// number of tensors costs nothing.  A block of 256 values is one wavefront, four values a lane.
//
// 8-bit states: m = a sign(c) (c / 127)^2 and v = a (c / 255)^4 with a the largest |value| of the block.  Codes lie closer
// where values are small: m reaches down to 6e-5 of a block's largest, v to 2e-10 (its root, which the update divides by,
// to 1.5e-5), at steps of 1.6 % near the top.  v moves by 1 - beta2 = 0.1 % a step, so rounding to the nearest code
// would hold it where it is; instead a value x between the neighbours lo and hi becomes hi with probability
// (x - lo) / (hi - lo), which keeps the mean.  v > 0 never becomes 0: the next step's m would be divided by eps alone.
// Values, codes and the comparison with the random number are single operations in a fixed order (no contraction), so that
// which code is taken does not depend on how the compiler fuses them.
#include <math.h>

#include <new>
#include <vector>

#include "common.h"

namespace symi {

constexpr uint32_t ADAMW_MAGIC = 0x41444d57u;
constexpr int ADAMW_BLOCK = 256;     // values that share a scale
constexpr int ADAMW_THREADS = 256;
constexpr int ADAMW_CHUNK = 4096;    // values of one workgroup
constexpr float SMALLEST = 1.17549435e-38f;
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
struct AdamwChunk {
  int tensor;
  unsigned at;   // of the tensor's chunks
};

struct AdamwScalars {
  float lr, beta1, keep1, beta2, keep2, eps, wd, gscale, fix1, fix2;
  uint32_t key;
};

__host__ __device__ inline uint32_t mix(uint32_t x) {
  x ^= x >> 16;
  x *= 0xBB67AE85u;
  x ^= x >> 15;
  x *= 0x6A09E667u;
  return x ^ (x >> 16);
}

__device__ __forceinline__ float m_value(float c, float a) {
#pragma clang fp contract(off)
  return c * c * M_UNIT * a;
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
  float lo = fminf(fmaxf(floorf(guess), 0.f), top - 1.f);
  float below = value(lo, a), above = value(lo + 1.f, a);
  if (below > x) {
    lo -= 1.f;
    above = below;
    below = value(lo, a);
  } else if (above <= x && lo < top - 1.f) {
    lo += 1.f;
    below = above;
    above = value(lo + 1.f, a);
  }
  return x - below > u * (above - below) ? lo + 1.f : lo;
}

// Bits of the largest |value| of a wavefront: of floats without their sign the order is that of their bits, NaN on top.
__device__ __forceinline__ uint32_t wave_max(uint32_t x) {
#pragma unroll
  for (int m = 32; m >= 1; m >>= 1) {
    const uint32_t y = (uint32_t)__shfl_xor((int)x, m, 64);
    x = x > y ? x : y;
  }
  return x;
}
// 0 for a block of nothing but denormal numbers, NaN for one that is not finite
__device__ __forceinline__ float scale_of(uint32_t bits) {
  return bits < 0x00800000u ? 0.f : bits < 0x7f800000u ? __uint_as_float(bits) : __uint_as_float(0x7fc00000u);
}

// What a lane holds of an array: the values from `at` on that lie below n (`full`: all four, as one access).
template <bool BF16>
__device__ __forceinline__ void load4(const void* p, long long at, long long n, float (&x)[4]) {
#pragma unroll
  for (int i = 0; i < 4; ++i)
    x[i] = at + i >= n ? 0.f : BF16 ? bf16_to_f32(static_cast<const uint16_t*>(p)[at + i]) : static_cast<const float*>(p)[at + i];
}
template <bool BF16>
__device__ __forceinline__ void store4(void* p, long long at, long long n, const float (&x)[4]) {
#pragma unroll
  for (int i = 0; i < 4; ++i)
    if (at + i < n) {
      if (BF16) static_cast<uint16_t*>(p)[at + i] = f32_to_bf16(x[i]);
      else static_cast<float*>(p)[at + i] = x[i];
    }
}

template <bool PARAM16, bool GRAD16, bool CODES>
__device__ __forceinline__ void adamw_block(const AdamwTensor& t, const AdamwScalars& h, float gscale, long long block, int lane) {
  const long long at = block * ADAMW_BLOCK + lane * 4;
  float g[4], w[4], m[4], v[4];
  float* const weights = PARAM16 ? t.master : static_cast<float*>(t.param);
  load4<GRAD16>(t.grad, at, t.n, g);
  load4<false>(weights, at, t.n, w);
  if (CODES) {
    const float am = t.m_scale[block], av = t.v_scale[block];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float cm = at + i < t.n ? (float)static_cast<const int8_t*>(t.m)[at + i] : 0.f;
      const float cv = at + i < t.n ? (float)static_cast<const uint8_t*>(t.v)[at + i] : 0.f;
      m[i] = copysignf(m_value(cm, am), cm);
      v[i] = v_value(cv, av);
    }
  } else {
    load4<false>(t.m, at, t.n, m);
    load4<false>(t.v, at, t.n, v);
  }
  uint32_t big_m = 0, big_v = 0;
  {
#pragma clang fp contract(off)
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float gr = g[i] * gscale;
      m[i] = m[i] * h.beta1 + gr * h.keep1;
      v[i] = v[i] * h.beta2 + gr * h.keep2 * gr;
      big_m = max(big_m, __float_as_uint(m[i]) & 0x7fffffffu);
      big_v = max(big_v, __float_as_uint(v[i]) & 0x7fffffffu);
    }
  }
  const float wd = t.decay * h.wd;
#pragma unroll
  for (int i = 0; i < 4; ++i) w[i] -= h.lr * (m[i] * h.fix1 / (sqrtf(v[i] * h.fix2) + h.eps) + wd * w[i]);
  store4<false>(weights, at, t.n, w);
  if (PARAM16) store4<true>(t.param, at, t.n, w);
  if (!CODES) {
    store4<false>(t.m, at, t.n, m);
    store4<false>(t.v, at, t.n, v);
    return;
  }
  const float am = scale_of(wave_max(big_m)), av = scale_of(wave_max(big_v));
  const uint32_t r0 = mix(((t.first_block + (unsigned)block) * 64u + lane) * 0x9E3779B1u + h.key);
  const uint32_t times[4] = {0x3C6EF373u, 0xA54FF53Bu, 0x510E527Fu, 0x9B05688Du};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    uint32_t r = r0 * times[i];
    r ^= r >> 15;
    const float um = ((r & 0xffffu) + 0.5f) * 0x1p-16f, uv = ((r >> 16) + 0.5f) * 0x1p-16f;
    const float x = fabsf(m[i]);
    float cm = 0.f, cv = 0.f;
    if (am > 0.f) cm = copysignf(code_between(x, am, 127.f * sqrtf(x / am), 127.f, um, m_value), m[i]);
    if (av > 0.f) {
      cv = code_between(v[i], av, 255.f * sqrtf(sqrtf(v[i] / av)), 255.f, uv, v_value);
      if (v[i] > 0.f) cv = fmaxf(cv, 1.f);
    }
    if (at + i < t.n) {
      static_cast<int8_t*>(t.m)[at + i] = (int8_t)cm;
      static_cast<uint8_t*>(t.v)[at + i] = (uint8_t)cv;
    }
  }
  if (lane == 0) {
    t.m_scale[block] = am;
    t.v_scale[block] = av;
  }
}

__global__ __launch_bounds__(ADAMW_THREADS) void adamw_kernel(const AdamwTensor* __restrict__ tensors,
                                                              const AdamwChunk* __restrict__ chunks, AdamwScalars h,
                                                              const float* __restrict__ grad_scale) {
  const AdamwChunk c = chunks[blockIdx.x];
  const AdamwTensor t = tensors[c.tensor];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const float gscale = grad_scale ? h.gscale * grad_scale[0] : h.gscale;
  for (int k = wave; k < ADAMW_CHUNK / ADAMW_BLOCK; k += ADAMW_THREADS / 64) {
    const long long block = (long long)c.at * (ADAMW_CHUNK / ADAMW_BLOCK) + k;
    if (block * ADAMW_BLOCK >= t.n) return;
    switch (t.kind) {
      case 0: adamw_block<false, false, false>(t, h, gscale, block, lane); break;
      case 1: adamw_block<true, false, false>(t, h, gscale, block, lane); break;
      case 2: adamw_block<false, true, false>(t, h, gscale, block, lane); break;
      case 3: adamw_block<true, true, false>(t, h, gscale, block, lane); break;
      case 4: adamw_block<false, false, true>(t, h, gscale, block, lane); break;
      case 5: adamw_block<true, false, true>(t, h, gscale, block, lane); break;
      case 6: adamw_block<false, true, true>(t, h, gscale, block, lane); break;
      default: adamw_block<true, true, true>(t, h, gscale, block, lane);
    }
  }
}

__global__ __launch_bounds__(ADAMW_THREADS) void adamw_decode_kernel(const AdamwTensor* __restrict__ tensors,
                                                                     const AdamwChunk* __restrict__ chunks,
                                                                     float* __restrict__ m_out, float* __restrict__ v_out) {
  const AdamwChunk c = chunks[blockIdx.x];
  const AdamwTensor t = tensors[c.tensor];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  for (int k = wave; k < ADAMW_CHUNK / ADAMW_BLOCK; k += ADAMW_THREADS / 64) {
    const long long block = (long long)c.at * (ADAMW_CHUNK / ADAMW_BLOCK) + k;
    const long long at = block * ADAMW_BLOCK + lane * 4;
    if (block * ADAMW_BLOCK >= t.n) return;
    float m[4], v[4];
    if (t.kind & 4) {
      const float am = t.m_scale[block], av = t.v_scale[block];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float cm = at + i < t.n ? (float)static_cast<const int8_t*>(t.m)[at + i] : 0.f;
        const float cv = at + i < t.n ? (float)static_cast<const uint8_t*>(t.v)[at + i] : 0.f;
        m[i] = copysignf(m_value(cm, am), cm);
        v[i] = v_value(cv, av);
      }
    } else {
      load4<false>(t.m, at, t.n, m);
      load4<false>(t.v, at, t.n, v);
    }
    const long long to = (long long)t.first_block * ADAMW_BLOCK;
    store4<false>(m_out + to, at, t.n, m);
    store4<false>(v_out + to, at, t.n, v);
  }
}

}  // namespace symi

struct symi_adamw {
  uint32_t magic;
  int device, count;
  long long chunks, values;
  void* table;   // on the device: the tensors, then the chunks
  const symi::AdamwTensor* tensors;
  const symi::AdamwChunk* list;
};

using namespace symi;

static int enter_adamw(const symi_ctx* ctx, const symi_adamw* opt, const char* who) {
  SYMI_ENTER(ctx, who);
  (void)cfg;
  SYMI_REQUIRE(opt && opt->magic == ADAMW_MAGIC, who, "opt is NULL or not a live one of symi_adamw_create");
  SYMI_REQUIRE(opt->device == ctx->device, who, "opt was created on another device than the context");
  return SYMI_OK;
}

extern "C" int symi_adamw_create(const symi_adamw_tensor* tensors, int count, symi_adamw** out) {
  const char* const who = "symi_adamw_create";
  SYMI_REQUIRE(out, who, "out is NULL");
  *out = nullptr;
  SYMI_REQUIRE(count >= 0 && (tensors || count == 0), who, "count < 0 or no tensors");
  try {
    std::vector<AdamwTensor> list;
    std::vector<AdamwChunk> chunks;
    long long blocks = 0;
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
          bad(s.n && (s.state_bits == 8) != (s.m_scale != nullptr) , "8-bit states need their scales, 32-bit ones have none") ||
          bad(s.n && (s.state_bits == 8) != (s.v_scale != nullptr), "8-bit states need their scales, 32-bit ones have none"))
        return SYMI_EINVAL;
      if (s.n == 0) continue;
      const long long mine = s.n / ADAMW_BLOCK + (s.n % ADAMW_BLOCK != 0);
      if (s.n >> 36 || blocks + mine > 1LL << 28) {
        set_error("%s: more than 2^28 blocks of 256 values", who);
        return SYMI_EUNSUPPORTED;
      }
      list.push_back({s.param, s.master, s.grad, s.m, s.v, s.m_scale, s.v_scale, s.n, (unsigned)blocks, s.decay,
                      (s.param_dtype == SYMI_BF16) | (s.grad_dtype == SYMI_BF16) << 1 | (s.state_bits == 8) << 2});
      for (long long c = 0; c * ADAMW_CHUNK < s.n; ++c) chunks.push_back({(int)list.size() - 1, (unsigned)c});
      blocks += mine;
      if (chunks.size() >= 1u << 24) {   // a workgroup each; the threads of a launch end at 2^32
        set_error("%s: more than 2^24 - 1 chunks of %d values", who, ADAMW_CHUNK);
        return SYMI_EUNSUPPORTED;
      }
    }
    int dev = -1;
    if (hipGetDevice(&dev) != hipSuccess) {
      (void)hipGetLastError();
      set_error("%s: no usable HIP device is current", who);
      return SYMI_EHIP;
    }
    symi_adamw* const opt = new symi_adamw();
    opt->device = dev;
    opt->count = count;
    opt->chunks = (long long)chunks.size();
    opt->values = blocks * ADAMW_BLOCK;
    opt->table = nullptr;
    const size_t bytes1 = align_up(list.size() * sizeof(AdamwTensor), 256), bytes2 = chunks.size() * sizeof(AdamwChunk);
    if (bytes2) {
      hipError_t e = hipMalloc(&opt->table, bytes1 + bytes2);
      if (e == hipSuccess) e = hipMemcpy(opt->table, list.data(), list.size() * sizeof(AdamwTensor), hipMemcpyHostToDevice);
      if (e == hipSuccess) e = hipMemcpy(static_cast<char*>(opt->table) + bytes1, chunks.data(), bytes2, hipMemcpyHostToDevice);
      if (e != hipSuccess) {
        set_error("%s: %s", who, hipGetErrorString(e));
        (void)hipGetLastError();
        if (opt->table) (void)hipFree(opt->table);
        delete opt;
        return SYMI_EHIP;
      }
    }
    opt->tensors = static_cast<const AdamwTensor*>(opt->table);
    opt->list = reinterpret_cast<const AdamwChunk*>(static_cast<char*>(opt->table) + bytes1);
    opt->magic = ADAMW_MAGIC;
    *out = opt;
    return SYMI_OK;
  } catch (const std::bad_alloc&) {
    set_error("%s: out of host memory", who);
    return SYMI_EHIP;
  }
}

extern "C" int symi_adamw_destroy(symi_adamw* opt) {
  if (!opt) return SYMI_OK;
  SYMI_REQUIRE(opt->magic == ADAMW_MAGIC, "symi_adamw_destroy", "not a live one of symi_adamw_create");
  opt->magic = 0;
  if (opt->table) (void)hipFree(opt->table);
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
  SYMI_TIMED(ctx, K_ADAMW_DECODE, st, (adamw_decode_kernel<<<(unsigned)opt->chunks, ADAMW_THREADS, 0, st>>>(opt->tensors, opt->list, m, v)));
  SYMI_LAUNCH_CHECK(who);
  return SYMI_OK;
}
