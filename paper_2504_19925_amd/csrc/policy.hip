// symi_token_logp / symi_policy_loss: log probabilities of the chosen tokens, the clipped policy loss with a KL term, and
// the gradient of the logits.
//
// Per row of logits, in base 2 with c = log2(e) / temperature: t_j = c z_j, m = max t_j, s = sum 2^(t_j - m),
//   logp = ln 2 (t_a - m) - ln s,   dlogits_j = u ([j = a] - 2^(t_j - m) / s),   u = grad_scale w / temperature dL/dlogp.
// The weights are the caller's, so u needs nothing from other rows: one workgroup takes a row from its logits to
// their gradient.  Statistics and sums are fp32; the four sums over the rows are taken in 64 bits by one workgroup, in order.
#include <math.h>

#include <algorithm>
#include <type_traits>

#include "common.h"

namespace symi {

constexpr int SUM_THREADS = 1024;

struct PolicyScalars {
  float clip_low, clip_high, kl_coef, inv_temp, scale, c;   // c: log2(e) / temperature
};

// A 16-byte piece of a row as it lies in memory: 8 bf16 or 4 fp32 logits.
template <bool BF16> struct Piece {
  static constexpr int N = BF16 ? 8 : 4;
  using Elem = std::conditional_t<BF16, uint16_t, float>;
  using Vec = std::conditional_t<BF16, u32x4_bf16, f32x4_f32>;
  typedef uint32_t Raw __attribute__((ext_vector_type(4)));
  static __device__ __forceinline__ Raw load(const Elem* p) { return __builtin_bit_cast(Raw, *reinterpret_cast<const Vec*>(p)); }
  static __device__ __forceinline__ void store(Elem* p, Raw r) { *reinterpret_cast<Vec*>(p) = __builtin_bit_cast(Vec, r); }
  // the first n of its values, the others -inf
  static __device__ __forceinline__ Raw load_some(const Elem* p, int n) {
    uint32_t x[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if constexpr (BF16) {
        const uint32_t lo = 2 * i < n ? p[2 * i] : 0xff80u, hi = 2 * i + 1 < n ? p[2 * i + 1] : 0xff80u;
        x[i] = lo | hi << 16;
      } else {
        x[i] = __float_as_uint(i < n ? p[i] : -INFINITY);
      }
    }
    return Raw{x[0], x[1], x[2], x[3]};
  }
  static __device__ __forceinline__ void store_some(Elem* p, Raw r, int n) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if constexpr (BF16) {
        if (2 * i < n) p[2 * i] = (uint16_t)r[i];
        if (2 * i + 1 < n) p[2 * i + 1] = (uint16_t)(r[i] >> 16);
      } else if (i < n) {
        p[i] = __uint_as_float(r[i]);
      }
    }
  }
  static __device__ __forceinline__ void unpack(Raw r, float (&x)[N]) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if constexpr (BF16) {
        x[2 * i] = __uint_as_float(r[i] << 16);
        x[2 * i + 1] = __uint_as_float(r[i] & 0xffff0000u);
      } else {
        x[i] = __uint_as_float(r[i]);
      }
    }
  }
  static __device__ __forceinline__ Raw pack(const float (&x)[N]) {
    uint32_t y[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if constexpr (BF16) y[i] = pack_bf16x2(x[2 * i], x[2 * i + 1]); else y[i] = __float_as_uint(x[i]);
    }
    return Raw{y[0], y[1], y[2], y[3]};
  }
  static __device__ __forceinline__ Raw none() {
    const uint32_t x = BF16 ? 0xff80ff80u : 0xff800000u;
    return Raw{x, x, x, x};
  }
};

// Makes the compiler unpack a piece again where it is used again, in place of keeping both forms in registers.
template <class Raw>
__device__ __forceinline__ void forget(Raw& r) { asm volatile("" : "+v"(r)); }

__device__ __forceinline__ float exp2_(float x) { return __builtin_amdgcn_exp2f(x); }   // below 2^-126: 0

// (m, s) of a set of t: m its largest value, s the sum of 2^(t - m).
__device__ __forceinline__ void join(float& m, float& s, float m2, float s2) {
  const float top = fmaxf(m, m2);
  const float ref = top == -INFINITY ? 0.f : top;   // nothing but -inf so far: 2^(-inf - 0) = 0
  s = s * exp2_(m - ref) + s2 * exp2_(m2 - ref);
  m = top;
}

// What a token adds to the loss, and dL/dlogp.  clipped tokens have no gradient from their advantage.
struct Token {
  float gain, kl, slope;
  bool clipped;
};
__device__ __forceinline__ Token token_loss(const PolicyScalars& p, float logp, float old, bool has_ref, float ref, float A) {
  Token k;
  const float r = expf(logp - old);
  k.clipped = (A > 0.f && r > 1.f + p.clip_high) || (A < 0.f && r < 1.f - p.clip_low);
  k.gain = -A * (k.clipped ? (A > 0.f ? 1.f + p.clip_high : 1.f - p.clip_low) : r);
  k.slope = k.clipped ? 0.f : -A * r;
  k.kl = 0.f;
  if (has_ref) {
    const float far = ref - logp, e = expm1f(far);
    // e^x - x - 1 loses all digits near 0, where it is x^2 / 2 + x^3 / 6 + ...
    k.kl = fabsf(far) < 0.125f ? far * far * (0.5f + far * (1.f / 6 + far * (1.f / 24 + far * (1.f / 120 + far * (1.f / 720))))) : e - far;
    k.slope -= p.kl_coef * e;
  }
  return k;
}

// A workgroup of THREADS takes a row, every thread NV pieces of it at a time: whatever fits is read once and stays in
// registers from the logits to their gradient.  Of a longer row the last part stays, the ones before it are read again.
template <bool BF16, bool GRAD, int THREADS, int NV>
__global__ __launch_bounds__(THREADS) void policy_kernel(
    const void* logits, int V, int ld, const int32_t* __restrict__ action, const float* __restrict__ logp_old,
    const float* __restrict__ logp_ref, const float* __restrict__ advantage, const float* __restrict__ weight,
    float* __restrict__ logp, float4* __restrict__ terms, void* dlogits, PolicyScalars p) {
  using P = Piece<BF16>;
  constexpr int N = P::N, WAVES = THREADS / 64;
  __shared__ float ms[WAVES], ss[WAVES], za_s;
  const int tid = threadIdx.x;
  const long long t = blockIdx.x;
  const auto* const z = static_cast<const typename P::Elem*>(logits) + t * ld;
  auto* const dz = static_cast<typename P::Elem*>(dlogits) + (GRAD ? t * ld : 0);
  const int a = action[t];
  const float w = weight ? weight[t] : 1.f;
  const int whole = V / N;               // pieces that lie in the vocabulary
  if (w == 0.f || (unsigned)a >= (unsigned)V) {
    if (tid == 0) {
      logp[t] = 0.f;
      if (terms) terms[t] = float4{0.f, 0.f, 0.f, 0.f};
    }
    if (GRAD) {
      const typename P::Raw zero = {0, 0, 0, 0};
      for (int q = tid; q < ld / N; q += THREADS) P::store(dz + (long long)q * N, zero);
      if (tid < ld % N) dz[ld / N * N + tid] = 0;
    }
    return;
  }
  float old = 0.f, ref = 0.f, A = 0.f;   // requested with the row
  if (terms) {
    old = logp_old[t];
    A = advantage[t];
    if (logp_ref) ref = logp_ref[t];
  }
  typename P::Raw r[NV];
  const auto fetch = [&](int q0) {
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int q = q0 + i * THREADS + tid;
      r[i] = P::none();
      if (q < whole) r[i] = P::load(z + (long long)q * N);
      else if (q == whole) r[i] = P::load_some(z + (long long)q * N, V - whole * N);
    }
  };
  float m = -INFINITY, s = 0.f;
  constexpr int STEP = NV * THREADS;
  const int last = whole / STEP * STEP;   // where the part that stays begins
  for (int q0 = 0; q0 <= last; q0 += STEP) {
    fetch(q0);
    float top = -INFINITY;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      if (q0 + i * THREADS > whole) continue;
      float x[N];
      P::unpack(r[i], x);
#pragma unroll
      for (int j = 0; j < N; ++j) top = fmaxf(top, x[j]);
      if (q0 + i * THREADS + tid == a / N) {
#pragma unroll
        for (int j = 0; j < N; ++j)
          if (j == a % N) za_s = x[j];
      }
    }
    top *= p.c;
    const float base = fmaxf(m, top), from = base == -INFINITY ? 0.f : base;   // nothing but -inf so far
    s *= exp2_(m - from);
    m = base;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      if (q0 + i * THREADS > whole) continue;
      float x[N];
      forget(r[i]);
      P::unpack(r[i], x);
#pragma unroll
      for (int j = 0; j < N; ++j) s += exp2_(fmaf(x[j], p.c, -from));
    }
  }
#pragma unroll
  for (int k = 32; k >= 1; k >>= 1) join(m, s, __shfl_xor(m, k, 64), __shfl_xor(s, k, 64));
  if ((tid & 63) == 0) {
    ms[tid >> 6] = m;
    ss[tid >> 6] = s;
  }
  __syncthreads();
  m = ms[0];
  s = ss[0];
#pragma unroll
  for (int k = 1; k < WAVES; ++k) join(m, s, ms[k], ss[k]);
  const float lp = fmaf(za_s, p.c, -m) * 0.693147180559945309f - logf(s);
  if (tid == 0) logp[t] = lp;
  if (!terms) return;
  const Token k = token_loss(p, lp, old, logp_ref != nullptr, ref, A);
  if (tid == 0) terms[t] = float4{w * (k.gain + p.kl_coef * k.kl), w * k.gain, w * k.kl, k.clipped ? w : 0.f};
  if (!GRAD) return;
  // 2^24 moves from the factor into the exponent, so that the power is no denormal number, which would become 0, where the
  // gradient in single precision is one that is kept
  const float u = p.scale * p.inv_temp * w * k.slope, minus = -u / s * 0x1p-24f, from = m - 24.f;
  for (int q0 = last; q0 >= 0; q0 -= STEP) {
    if (q0 < last) fetch(q0);
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int q = q0 + i * THREADS + tid;
      if (q0 + i * THREADS > whole) continue;
      float x[N];
      forget(r[i]);
      P::unpack(r[i], x);
#pragma unroll
      for (int j = 0; j < N; ++j) x[j] = minus * exp2_(fmaf(x[j], p.c, -from));
      if (q == a / N) {
#pragma unroll
        for (int j = 0; j < N; ++j)
          if (j == a % N) x[j] += u;
      }
      if (q < whole) P::store(dz + (long long)q * N, P::pack(x));
      else if (q == whole) P::store_some(dz + (long long)q * N, P::pack(x), V - whole * N);
    }
  }
  for (int j = V + tid; j < ld; j += THREADS) dz[j] = 0;
}

__global__ __launch_bounds__(SUM_THREADS) void policy_sum_kernel(const float4* __restrict__ terms, int T, float* __restrict__ stats) {
  __shared__ double part[SUM_THREADS / 64][4];
  double sum[4] = {};
  for (long long t = threadIdx.x; t < T; t += SUM_THREADS) {
    const float4 x = terms[t];
    sum[0] += x.x; sum[1] += x.y; sum[2] += x.z; sum[3] += x.w;
  }
#pragma unroll
  for (int k = 0; k < 4; ++k) {
#pragma unroll
    for (int m = 32; m >= 1; m >>= 1) sum[k] += __shfl_xor(sum[k], m, 64);
    if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6][k] = sum[k];
  }
  __syncthreads();
  if (threadIdx.x < 4) {
    double all = 0.;
    for (int w = 0; w < SUM_THREADS / 64; ++w) all += part[w][threadIdx.x];
    stats[threadIdx.x] = (float)all;
  }
}

static int check_policy(const char* who, const symi_policy* hp, int V, int ld) {
  SYMI_REQUIRE(hp, who, "NULL pointer");
  SYMI_REQUIRE(V >= 1, who, "V < 1");
  SYMI_REQUIRE(ld >= V, who, "ld < V");
  SYMI_REQUIRE(hp->logits_dtype == SYMI_F32 || hp->logits_dtype == SYMI_BF16, who, "logits_dtype must be SYMI_F32 or SYMI_BF16");
  SYMI_REQUIRE(hp->inv_temperature > 0.f && hp->inv_temperature < INFINITY, who, "inv_temperature must be positive and finite");
  SYMI_REQUIRE(hp->clip_low >= 0.f && hp->clip_low <= 1.f && hp->clip_high >= 0.f, who, "clip_low must lie in [0, 1], clip_high must be >= 0");
  SYMI_REQUIRE(hp->kl_coef >= 0.f, who, "kl_coef must be >= 0");
  SYMI_REQUIRE(hp->grad_scale == hp->grad_scale, who, "grad_scale is NaN");
  return SYMI_OK;
}

static int policy_impl(const char* who, const symi_ctx* ctx, const symi_policy* hp, const void* logits, int V, int ld,
                       const int32_t* action, const float* logp_old, const float* logp_ref, const float* advantage,
                       const float* weight, float* logp, float4* terms, void* dlogits, hipStream_t st) {
  const PolicyScalars p = {hp->clip_low, hp->clip_high, hp->kl_coef, hp->inv_temperature, hp->grad_scale,
                           (float)(1.4426950408889634 * hp->inv_temperature)};
  const int T = ctx->cfg.T, kid = terms ? K_POLICY : K_TOKEN_LOGP;
  const bool bf16 = hp->logits_dtype == SYMI_BF16;
  const int pieces = V / (bf16 ? 8 : 4) + 1;
#define ROWS(BF16, GRAD, THREADS, NV)                                                                                  \
  SYMI_TIMED(ctx, kid, st, (policy_kernel<BF16, GRAD, THREADS, NV><<<T, THREADS, 0, st>>>(                             \
      logits, V, ld, action, logp_old, logp_ref, advantage, weight, logp, terms, dlogits, p)))
#define SIZES(BF16, GRAD)                                      \
  if (pieces <= 64 * 4) ROWS(BF16, GRAD, 64, 4);               \
  else if (pieces <= 256 * 4) ROWS(BF16, GRAD, 256, 4);        \
  else if (pieces <= 512 * 8) ROWS(BF16, GRAD, 512, 8);        \
  else if (pieces <= 1024 * 8) ROWS(BF16, GRAD, 1024, 8);      \
  else ROWS(BF16, GRAD, 1024, 16)
  if (bf16 && dlogits) { SIZES(true, true); }
  else if (bf16) { SIZES(true, false); }
  else if (dlogits) { SIZES(false, true); }
  else { SIZES(false, false); }
#undef SIZES
#undef ROWS
  SYMI_LAUNCH_CHECK(who);
  return SYMI_OK;
}

}  // namespace symi

using namespace symi;

extern "C" size_t symi_policy_workspace_bytes(const symi_cfg* cfg) {
  if (check_cfg(cfg, "symi_policy_workspace_bytes") != SYMI_OK) return 0;
  return align_up((size_t)cfg->T * sizeof(float4), 256) + 256;
}

extern "C" int symi_token_logp(const symi_ctx* ctx, const symi_policy* hp, const void* logits, int V, int ld,
                               const int32_t* action, const float* weight, float* logp, void* stream) {
  const char* const who = "symi_token_logp";
  SYMI_ENTER(ctx, who);
  if (int rc = check_policy(who, hp, V, ld)) return rc;
  if (cfg->T == 0) return SYMI_OK;
  SYMI_REQUIRE(logits && action && logp, who, "NULL pointer");
  return policy_impl(who, ctx, hp, logits, V, ld, action, nullptr, nullptr, nullptr, weight, logp, nullptr, nullptr, as_stream(stream));
}

extern "C" int symi_policy_loss(const symi_ctx* ctx, const symi_policy* hp, const void* logits, int V, int ld,
                                const int32_t* action, const float* logp_old, const float* logp_ref,
                                const float* advantage, const float* weight, float* logp, float* stats, void* dlogits,
                                void* ws, void* stream) {
  const char* const who = "symi_policy_loss";
  SYMI_ENTER(ctx, who);
  if (int rc = check_policy(who, hp, V, ld)) return rc;
  SYMI_REQUIRE(cfg->T == 0 || logp_ref || hp->kl_coef == 0.f, who, "kl_coef needs logp_ref");
  SYMI_REQUIRE(stats && ws && (cfg->T == 0 || (logits && action && logp_old && advantage && weight && logp)), who, "NULL pointer");
  hipStream_t st = as_stream(stream);
  float4* const terms = reinterpret_cast<float4*>(align_up(reinterpret_cast<size_t>(ws), 256));
  if (cfg->T)
    if (int rc = policy_impl(who, ctx, hp, logits, V, ld, action, logp_old, logp_ref, advantage, weight, logp, terms, dlogits, st)) return rc;
  SYMI_TIMED(ctx, K_POLICY_SUM, st, (policy_sum_kernel<<<1, SUM_THREADS, 0, st>>>(terms, cfg->T, stats)));
  SYMI_LAUNCH_CHECK(who);
  return SYMI_OK;
}
