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

constexpr int POLICY_THREADS = 256;
constexpr int SUM_THREADS = 1024;

struct PolicyScalars {
  float clip_low, clip_high, kl_coef, inv_temp, scale, c;   // c: log2(e) / temperature
};

template <bool BF16> struct Logit {
  using Elem = std::conditional_t<BF16, uint16_t, float>;
  static __device__ __forceinline__ float get(Elem x) {
    if constexpr (BF16) return bf16_to_f32(x); else return x;
  }
  static __device__ __forceinline__ Elem put(float x) {
    if constexpr (BF16) return f32_to_bf16(x); else return x;
  }
};

// (m, s) of a set of t: m its largest value, s the sum of 2^(t - m).
__device__ __forceinline__ void join(float& m, float& s, float m2, float s2) {
  const float top = fmaxf(m, m2);
  const float ref = top == -INFINITY ? 0.f : top;   // nothing but -inf so far: 2^(-inf - 0) = 0
  s = s * exp2f(m - ref) + s2 * exp2f(m2 - ref);
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

template <bool BF16>
__global__ __launch_bounds__(POLICY_THREADS) void policy_kernel(
    const void* logits, int V, int ld, const int32_t* __restrict__ action, const float* __restrict__ logp_old,
    const float* __restrict__ logp_ref, const float* __restrict__ advantage, const float* __restrict__ weight,
    float* __restrict__ logp, float4* __restrict__ terms, void* dlogits, PolicyScalars p) {
  using L = Logit<BF16>;
  __shared__ float ms[POLICY_THREADS / 64], ss[POLICY_THREADS / 64];
  const long long t = blockIdx.x;
  const auto* const z = static_cast<const typename L::Elem*>(logits) + t * ld;
  auto* const dz = static_cast<typename L::Elem*>(dlogits) + (dlogits ? t * ld : 0);
  const int a = action[t];
  const float w = weight ? weight[t] : 1.f;
  if (w == 0.f || (unsigned)a >= (unsigned)V) {
    if (threadIdx.x == 0) {
      logp[t] = 0.f;
      if (terms) terms[t] = float4{0.f, 0.f, 0.f, 0.f};
    }
    if (dlogits)
      for (int j = threadIdx.x; j < ld; j += POLICY_THREADS) dz[j] = L::put(0.f);
    return;
  }
  const float za = L::get(z[a]);
  float m = -INFINITY, s = 0.f;
  for (int j = threadIdx.x; j < V; j += POLICY_THREADS) join(m, s, L::get(z[j]) * p.c, 1.f);
#pragma unroll
  for (int k = 32; k >= 1; k >>= 1) join(m, s, __shfl_xor(m, k, 64), __shfl_xor(s, k, 64));
  if ((threadIdx.x & 63) == 0) {
    ms[threadIdx.x >> 6] = m;
    ss[threadIdx.x >> 6] = s;
  }
  __syncthreads();
  m = ms[0];
  s = ss[0];
#pragma unroll
  for (int k = 1; k < POLICY_THREADS / 64; ++k) join(m, s, ms[k], ss[k]);
  const float lp = (za * p.c - m) * 0.693147180559945309f - logf(s);
  if (threadIdx.x == 0) logp[t] = lp;
  if (!terms) return;
  const Token k = token_loss(p, lp, logp_old[t], logp_ref != nullptr, logp_ref ? logp_ref[t] : 0.f, advantage[t]);
  if (threadIdx.x == 0) terms[t] = float4{w * (k.gain + p.kl_coef * k.kl), w * k.gain, w * k.kl, k.clipped ? w : 0.f};
  if (!dlogits) return;
  const float u = p.scale * p.inv_temp * w * k.slope, inv_s = 1.f / s;
  for (int j = threadIdx.x; j < ld; j += POLICY_THREADS)
    dz[j] = L::put(j < V ? u * ((j == a ? 1.f : 0.f) - exp2f(L::get(z[j]) * p.c - m) * inv_s) : 0.f);
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
  if (hp->logits_dtype == SYMI_BF16)
    SYMI_TIMED(ctx, kid, st, (policy_kernel<true><<<T, POLICY_THREADS, 0, st>>>(logits, V, ld, action, logp_old, logp_ref, advantage, weight, logp, terms, dlogits, p)));
  else
    SYMI_TIMED(ctx, kid, st, (policy_kernel<false><<<T, POLICY_THREADS, 0, st>>>(logits, V, ld, action, logp_old, logp_ref, advantage, weight, logp, terms, dlogits, p)));
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
