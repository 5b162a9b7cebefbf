// symi_route_scored / symi_route_scored_bwd / symi_route_bias: routing by softmax or sigmoid scores, with a bias and groups.
//
// A wavefront has a token; lane l holds the classes l, l + 64, ...  What classes are compared by is binary64, so that the choice is that of
// the formula also where scores are a rounding apart.
#include <limits.h>
#include <math.h>

#include <algorithm>

#include "common.h"

namespace symi {

constexpr int SCORE_WAVES = 4;
constexpr int SCORE_MAX_K = 16;

// 1 / (1 + exp(-z)), with its digits also where exp(-z) is infinite
__device__ __forceinline__ float sigmoid_of(float z) {
  const float e = expf(-fabsf(z));
  return (z < 0.f ? e : 1.f) / (1.f + e);
}

struct ScoreArgs {
  const float *logits, *bias;
  int32_t* idx;
  float* gate;
  int32_t* hist;
  int T, E, k, renorm, sigmoid, groups, per, top_groups, group_top;   // per: classes of a group
  float scale;
};

__device__ __forceinline__ double wave_max(double x) {
#pragma unroll
  for (int m = 32; m >= 1; m >>= 1) x = fmax(x, __shfl_xor(x, m, 64));
  return x;
}
__device__ __forceinline__ double wave_sum(double x) {
#pragma unroll
  for (int m = 32; m >= 1; m >>= 1) x += __shfl_xor(x, m, 64);
  return x;
}

template <int NV>
__global__ __launch_bounds__(SCORE_WAVES * 64) void score_kernel(ScoreArgs a) {
  extern __shared__ char smem[];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  int32_t* const hist = reinterpret_cast<int32_t*>(smem);
  double* const by_s = reinterpret_cast<double*>(smem + (a.E * sizeof(int32_t) + 15) / 16 * 16) + wave * a.E;   // groups only
  for (int e = threadIdx.x; e < a.E; e += SCORE_WAVES * 64) hist[e] = 0;
  __syncthreads();
  for (long long t = (long long)blockIdx.x * SCORE_WAVES + wave; t < a.T; t += (long long)gridDim.x * SCORE_WAVES) {
    float z[NV];
    double by[NV], of[NV];   // what classes and groups are compared by; -inf: not to be chosen
    bool nan = false;
    double top = -INFINITY;
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      const int e = v * 64 + lane;
      z[v] = e < a.E ? a.logits[t * a.E + e] : -INFINITY;
      nan |= z[v] != z[v] || (!a.sigmoid && z[v] == INFINITY);
      top = fmax(top, (double)z[v]);
    }
    nan = __ballot(nan) != 0;
    double sum = 0.;
    if (!a.sigmoid) {
      top = wave_max(top);
#pragma unroll
      for (int v = 0; v < NV; ++v) sum += z[v] > -INFINITY ? exp((double)z[v] - top) : 0.;
      sum = wave_sum(sum);
    }
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      const int e = v * 64 + lane;
      const double s = a.sigmoid ? 1. / (1. + exp(-(double)z[v])) : exp((double)z[v] - top) / sum;
      by[v] = a.bias ? s + (double)(e < a.E ? a.bias[e] : 0.f) : (double)z[v];
      of[v] = !a.bias && a.group_top > 1 ? s : by[v];
      if (!(z[v] > -INFINITY) || !(by[v] > -INFINITY)) by[v] = of[v] = -INFINITY;
    }
    if (a.groups > 1) {
#pragma unroll
      for (int v = 0; v < NV; ++v)
        if (v * 64 + lane < a.E) by_s[v * 64 + lane] = of[v];
      __builtin_amdgcn_wave_barrier();
      double best = -INFINITY, second = -INFINITY;
      if (lane < a.groups)
        for (int i = 0; i < a.per; ++i) {
          const double x = by_s[lane * a.per + i];
          if (x > best) { second = best; best = x; } else if (x > second) second = x;
        }
      const double mine = a.group_top > 1 && second > -INFINITY ? best + second : best;
      int rank = 0;
      for (int g = 0; g < a.groups; ++g) {
        const double x = __shfl(mine, g, 64);
        rank += x > mine || (x == mine && g < lane);
      }
      const unsigned long long kept = __ballot(lane < a.groups && rank < a.top_groups);
#pragma unroll
      for (int v = 0; v < NV; ++v) {
        const int e = v * 64 + lane;
        if (e < a.E && !(kept >> (e / a.per) & 1)) by[v] = -INFINITY;
      }
      __builtin_amdgcn_wave_barrier();
    }
    unsigned taken = 0;
#pragma unroll
    for (int v = 0; v < NV; ++v)
      if (v * 64 + lane >= a.E) taken |= 1u << v;
    // lane j keeps the j-th choice
    int my_idx = 0;
    float my_z = -INFINITY;
    bool real = false;
    for (int j = 0; j < a.k; ++j) {
      double b = -INFINITY;
      int at = INT_MAX;
      float zb = 0.f;
#pragma unroll
      for (int v = 0; v < NV; ++v)
        if (!(taken >> v & 1) && (by[v] > b || at == INT_MAX)) { b = by[v]; at = v * 64 + lane; zb = z[v]; }
#pragma unroll
      for (int m = 32; m >= 1; m >>= 1) {
        const double ob = __shfl_xor(b, m, 64);
        const int oat = __shfl_xor(at, m, 64);
        const float oz = __shfl_xor(zb, m, 64);
        if (ob > b || (ob == b && oat < at)) { b = ob; at = oat; zb = oz; }
      }
      if ((at & 63) == lane) taken |= 1u << (at >> 6);
      if (j == lane) { my_idx = at; my_z = zb; real = b > -INFINITY; }
    }
    // gates, relative to the largest of the k
    float g;
    if (a.renorm) {
      const float part = a.sigmoid ? fminf(my_z, 0.f) : my_z;
      float m = real ? part : -INFINITY;
#pragma unroll
      for (int o = 8; o >= 1; o >>= 1) m = fmaxf(m, __shfl_xor(m, o, 64));
      g = real ? expf(part - m) : 0.f;
      if (a.sigmoid && real) g /= 1.f + expf(-fabsf(my_z));
      float s = g;
#pragma unroll
      for (int o = 8; o >= 1; o >>= 1) s += __shfl_xor(s, o, 64);
      g = real ? g / s : 0.f;
    } else if (a.sigmoid) {
      g = real ? sigmoid_of(my_z) : 0.f;
    } else {
      g = real ? expf(my_z - (float)top) / (float)sum : 0.f;
    }
    if (lane < a.k) {
      a.idx[t * a.k + lane] = my_idx;
      a.gate[t * a.k + lane] = nan ? NAN : a.scale * g;
      atomicAdd(&hist[my_idx], 1);
    }
  }
  __syncthreads();
  for (int e = threadIdx.x; e < a.E; e += SCORE_WAVES * 64)
    if (hist[e]) atomicAdd(&a.hist[e], hist[e]);
}

struct ScoreBwdArgs {
  const float* logits;
  const int32_t* idx;
  const float *gate, *dgate;
  float* dlogits;
  int T, E, k, renorm, sigmoid;
  float scale;
};

// dz of the chosen: renormalised g (dg - sum g dg), sigmoid: times (1 - s); a plain softmax: p_e ([e chosen] dg - sum p dg) for every class.
__global__ __launch_bounds__(SCORE_WAVES * 64) void score_bwd_kernel(ScoreBwdArgs a) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  for (long long t = (long long)blockIdx.x * SCORE_WAVES + wave; t < a.T; t += (long long)gridDim.x * SCORE_WAVES) {
    const float* const row = a.logits + t * a.E;
    int at = -1;
    float g = 0.f, dg = 0.f, z = 0.f;
    if (lane < a.k) {
      at = a.idx[t * a.k + lane];
      g = a.gate[t * a.k + lane] / a.scale;
      dg = a.dgate[t * a.k + lane] * a.scale;
      if (g == 0.f || (unsigned)at >= (unsigned)a.E) at = -1;   // only filled up
      else z = row[at];
    }
    if (at < 0) g = dg = 0.f;
    float dot = g * dg;
#pragma unroll
    for (int o = 8; o >= 1; o >>= 1) dot += __shfl_xor(dot, o, 64);
    dot = __shfl(dot, 0, 64);
    float dz = a.renorm ? g * (dg - dot) : g * dg;
    if (a.sigmoid) dz *= sigmoid_of(-z);
    const bool dense = !a.sigmoid && !a.renorm;
    float top = -INFINITY, sum = 0.f;
    if (dense) {
      for (int e = lane; e < a.E; e += 64) top = fmaxf(top, row[e]);
#pragma unroll
      for (int o = 32; o >= 1; o >>= 1) top = fmaxf(top, __shfl_xor(top, o, 64));
      for (int e = lane; e < a.E; e += 64) sum += row[e] > -INFINITY ? expf(row[e] - top) : row[e] == -INFINITY ? 0.f : NAN;
#pragma unroll
      for (int o = 32; o >= 1; o >>= 1) sum += __shfl_xor(sum, o, 64);
    }
    for (int e0 = 0; e0 < a.E; e0 += 64) {
      const int e = e0 + lane;
      float out = 0.f;
      if (dense && e < a.E) out = row[e] > -INFINITY ? -expf(row[e] - top) / sum * dot : row[e] == -INFINITY ? 0.f : NAN;
      for (int j = 0; j < a.k; ++j) {
        const int c = __shfl(at, j, 64);
        const float x = __shfl(dz, j, 64);
        if (c == e) out += x;
      }
      if (e < a.E) a.dlogits[t * a.E + e] = out;
    }
  }
}

__global__ __launch_bounds__(1024) void score_bias_kernel(const int32_t* __restrict__ hist, float rate, float* __restrict__ bias, int E) {
  __shared__ long long part[16];
  const int e = threadIdx.x;
  const long long h = e < E ? hist[e] : 0;
  long long s = h;
#pragma unroll
  for (int m = 32; m >= 1; m >>= 1) s += __shfl_xor(s, m, 64);
  if ((e & 63) == 0) part[e >> 6] = s;
  __syncthreads();
  s = 0;
  for (int w = 0; w < (int)blockDim.x / 64; ++w) s += part[w];
  if (e < E) {
    const long long off = s - h * E;
    if (off) bias[e] += off > 0 ? rate : -rate;
  }
}

static int check_score(const symi_cfg* c, const symi_score* hp, const char* who) {
  SYMI_REQUIRE(hp, who, "hp is NULL");
  SYMI_REQUIRE(hp->score == SYMI_SOFTMAX || hp->score == SYMI_SIGMOID, who, "score must be SYMI_SOFTMAX or SYMI_SIGMOID");
  SYMI_REQUIRE(hp->groups >= 1 && hp->groups <= 64 && c->E % hp->groups == 0, who, "groups must be a divisor of E, at most 64");
  SYMI_REQUIRE(hp->top_groups >= 1 && hp->top_groups <= hp->groups, who, "top_groups outside [1, groups]");
  SYMI_REQUIRE((long long)hp->top_groups * (c->E / hp->groups) >= c->k, who, "top_groups groups hold fewer than k classes");
  SYMI_REQUIRE(hp->group_top == 1 || (hp->group_top == 2 && c->E / hp->groups >= 2), who, "group_top must be 1 or 2, at most E / groups");
  SYMI_REQUIRE(hp->scale > 0.f && hp->scale < INFINITY, who, "scale must be positive and finite");
  return SYMI_OK;
}

static int score_grid(int T) { return std::min(cdiv(T, SCORE_WAVES), 4096); }

}  // namespace symi

using namespace symi;

extern "C" int symi_route_scored(const symi_ctx* ctx, const symi_score* hp, const float* logits, const float* bias, int32_t* idx,
                                 float* gate, int32_t* hist, void* stream) {
  SYMI_ENTER(ctx, "symi_route_scored");
  if (int rc = check_score(cfg, hp, "symi_route_scored")) return rc;
  SYMI_REQUIRE(hist && (cfg->T == 0 || (logits && idx && gate)), "symi_route_scored", "NULL pointer");
  hipStream_t st = as_stream(stream);
  const int E = cfg->E;
  launch_fill_i32(ctx, hist, E, 0, st);
  if (cfg->T > 0) {
    const ScoreArgs a = {logits, bias, idx, gate, hist, cfg->T, E, cfg->k, cfg->renorm, hp->score == SYMI_SIGMOID, hp->groups, E / hp->groups,
                         hp->top_groups, hp->group_top, hp->scale};
    const size_t sh = align_up(E * sizeof(int32_t), 16) + (hp->groups > 1 ? SCORE_WAVES * E * sizeof(double) : 0);
    const int grid = score_grid(cfg->T), threads = SCORE_WAVES * 64;
    if (E <= 64) SYMI_TIMED(ctx, K_SCORE, st, (score_kernel<1><<<grid, threads, sh, st>>>(a)));
    else if (E <= 128) SYMI_TIMED(ctx, K_SCORE, st, (score_kernel<2><<<grid, threads, sh, st>>>(a)));
    else if (E <= 256) SYMI_TIMED(ctx, K_SCORE, st, (score_kernel<4><<<grid, threads, sh, st>>>(a)));
    else SYMI_TIMED(ctx, K_SCORE, st, (score_kernel<16><<<grid, threads, sh, st>>>(a)));
  }
  SYMI_LAUNCH_CHECK("symi_route_scored");
  return SYMI_OK;
}

extern "C" int symi_route_scored_bwd(const symi_ctx* ctx, const symi_score* hp, const float* logits, const int32_t* idx,
                                     const float* gate, const float* dgate, float* dlogits, void* stream) {
  SYMI_ENTER(ctx, "symi_route_scored_bwd");
  if (int rc = check_score(cfg, hp, "symi_route_scored_bwd")) return rc;
  if (cfg->T == 0) return SYMI_OK;
  SYMI_REQUIRE(logits && idx && gate && dgate && dlogits, "symi_route_scored_bwd", "NULL pointer");
  hipStream_t st = as_stream(stream);
  const ScoreBwdArgs a = {logits, idx, gate, dgate, dlogits, cfg->T, cfg->E, cfg->k, cfg->renorm, hp->score == SYMI_SIGMOID, hp->scale};
  SYMI_TIMED(ctx, K_SCORE_BWD, st, (score_bwd_kernel<<<score_grid(cfg->T), SCORE_WAVES * 64, 0, st>>>(a)));
  SYMI_LAUNCH_CHECK("symi_route_scored_bwd");
  return SYMI_OK;
}

extern "C" int symi_route_bias(const symi_ctx* ctx, const int32_t* hist, float rate, float* bias, void* stream) {
  SYMI_ENTER(ctx, "symi_route_bias");
  SYMI_REQUIRE(hist && bias, "symi_route_bias", "NULL pointer");
  SYMI_REQUIRE(rate >= 0.f && rate < INFINITY, "symi_route_bias", "rate must be finite and not negative");
  hipStream_t st = as_stream(stream);
  SYMI_TIMED(ctx, K_SCORE_BIAS, st, (score_bias_kernel<<<1, (cfg->E + 63) / 64 * 64, 0, st>>>(hist, rate, bias, cfg->E)));
  SYMI_LAUNCH_CHECK("symi_route_bias");
  return SYMI_OK;
}
