// symi_route_scored / symi_route_scored_bwd / symi_route_bias: routing by softmax or sigmoid scores, with a bias and groups.
//
// The choice is that of binary64, but hardly any token needs it: classes are chosen in fp32, with the two behind the last choice, and where neighbours in
// that order are nearer than twice what fp32 can be off (nearest), those few are put in the order of their values in binary64.  Where that does not settle it (the
// second behind them is near too, the last group that stays and the first that does not are, a softmax, whose sum is needed, classes that are missing), the wavefront
// goes through the whole row in binary64 (choose_exactly).  Of tokens with 128 classes (normal logits, sigmoid) the one is the case for 0.04 %, the other for 0.004 %.  Without a bias
// classes are compared by their logits, exactly.
//
// G lanes hold a token's classes, up to 16 each in pieces of 4: piece p = v G + g lies in lane g, so that loads are whole lines, and the k rounds of
// largest, runner-up, ... scan few lanes' registers, with a butterfly of log2 G steps in DPP operands.  Sums of exponentials are taken along a tree over the
// pieces, the same for every G, so that a token's gates do not depend on its batch.
//
// Bound by instructions and their latency: 65536 tokens of 128 classes in 8 groups, sigmoid and bias, 49 us with the launches that clear the counts and move the bias, against 7
// of the bytes.  By calls with fewer choices, without groups, without a bias: a round takes 1.7, so the eight 14, the groups 8, the bias with its two rounds more 5, and 20 are launches,
// loads, scores, gates and counts.  16 tokens 12.2 us, of which the kernel is 10.3, one workgroup's chain: 0.4 a round, the groups 1.4.
#include <limits.h>
#include <math.h>

#include <algorithm>

#include "common.h"

namespace symi {

constexpr int SCORE_MOST = 16;          // wavefronts of a workgroup at most
constexpr int SCORE_MAX_K = 16;
constexpr int SCORE_LDS = 156 * 1024;   // of a workgroup at most
constexpr int BWD_WAVES = 4;
constexpr float LOG2E = 1.44269504f;
constexpr float U32 = 5.9604645e-8f;    // 2^-24

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
  int lanes;   // neighbouring lanes whose pieces of 4 make a group, where that is so, else 0
  int shift;   // their logarithm
  int alone;   // one workgroup holds the whole batch and stores its counts
};

// What a wavefront has in LDS besides the workgroup's counts and groups of classes.
struct ScoreLds {
  float* of;            // [tokens][E]: what groups are compared by; in choose_exactly [E] doubles
  float* group;         // [tokens][groups]
  int* chosen;          // [tokens][k + 2]: the classes (~class: it only fills up), the one behind them, whether their order is to be looked at
  float2* softmax;      // [tokens]: largest logit, sum
};
__host__ __device__ inline int score_lds_of(int E, int tokens) { return ((tokens > 2 ? tokens * 4 : 8) * E + 15) / 16 * 16; }
__host__ __device__ inline int score_lds_bytes(int E, int k, int groups, int tokens) {   // a multiple of 16
  return score_lds_of(E, tokens) + (tokens * (8 + 4 * groups + 4 * (k + 2)) + 15) / 16 * 16;
}
__device__ __forceinline__ ScoreLds score_lds(char* p, int E, int k, int groups, int tokens) {
  ScoreLds L;
  L.of = reinterpret_cast<float*>(p);
  p += score_lds_of(E, tokens);
  L.softmax = reinterpret_cast<float2*>(p);
  p += tokens * 8;
  L.group = reinterpret_cast<float*>(p);
  p += tokens * groups * 4;
  L.chosen = reinterpret_cast<int*>(p);
  return L;
}

// Orders a wavefront's own LDS operations, which the hardware carries out as they come.
__device__ __forceinline__ void wave_sync() {
  asm volatile("" ::: "memory");
  __builtin_amdgcn_wave_barrier();
  asm volatile("" ::: "memory");
}

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

// The word that the lane has to compare with in step STEP of a butterfly over 64 lanes: 0, 1: the other half, the other row of 16 lanes (the swap
// gives a pair that is the same in both); 2 .. 5: mirrored in a row, in half of it, and in four.
template <int STEP>
__device__ __forceinline__ void partner(int x, int& one, int& other) {
  if constexpr (STEP == 0) {
    const auto r = __builtin_amdgcn_permlane32_swap((unsigned)x, (unsigned)x, false, false);
    one = (int)r[0];
    other = (int)r[1];
  } else if constexpr (STEP == 1) {
    const auto r = __builtin_amdgcn_permlane16_swap((unsigned)x, (unsigned)x, false, false);
    one = (int)r[0];
    other = (int)r[1];
  } else {
    constexpr int ctrl = STEP == 2 ? 0x140 : STEP == 3 ? 0x141 : STEP == 4 ? 0x4e : 0xb1;
    one = x;
    other = __builtin_amdgcn_update_dpp(0, x, ctrl, 0xf, 0xf, false);
  }
}
template <int STEP>
__device__ __forceinline__ void better_of(float& b, int& at) {
  int x, y, i, j;
  partner<STEP>(__float_as_int(b), x, y);
  partner<STEP>(at, i, j);
  const float p = __int_as_float(x), q = __int_as_float(y);
  const bool second = q > p || (q == p && j < i);
  b = second ? q : p;
  at = second ? j : i;
}
template <int STEP>
__device__ __forceinline__ void better_of(double& b, int& at) {
  int xl, yl, xh, yh, i, j;
  partner<STEP>(__double2loint(b), xl, yl);
  partner<STEP>(__double2hiint(b), xh, yh);
  partner<STEP>(at, i, j);
  const double p = __hiloint2double(xh, xl), q = __hiloint2double(yh, yl);
  const bool second = q > p || (q == p && j < i);
  b = second ? q : p;
  at = second ? j : i;
}
// (value, class) of G lanes: the largest value, of equal ones the lowest class.
template <int G, class V>
__device__ __forceinline__ void best_of(V& b, int& at) {
  if constexpr (G >= 64) better_of<0>(b, at);
  if constexpr (G >= 32) better_of<1>(b, at);
  if constexpr (G >= 16) better_of<2>(b, at);
  if constexpr (G >= 8) better_of<3>(b, at);
  if constexpr (G >= 4) better_of<4>(b, at);
  if constexpr (G >= 2) better_of<5>(b, at);
}

// The choice for one token by a whole wavefront, in binary64: lane l looks at the classes l, l + 64, ...
__device__ __forceinline__ void choose_exactly(const ScoreArgs& a, const float* __restrict__ row, double* by, int* chosen) {
  const int lane = threadIdx.x & 63;
  double top = -INFINITY, sum = 0.;
  if (!a.sigmoid && (a.bias || a.group_top > 1)) {
    for (int e = lane; e < a.E; e += 64) top = fmax(top, (double)row[e]);
    top = wave_max(top);
    for (int e = lane; e < a.E; e += 64) sum += row[e] > -INFINITY ? exp((double)row[e] - top) : 0.;
    sum = wave_sum(sum);
  }
  auto score = [&](float z) { return a.sigmoid ? 1. / (1. + exp(-(double)z)) : exp((double)z - top) / sum; };
  // what classes are compared by; -inf: not to be chosen
  auto value = [&](int e, float z, bool of_group) {
    const double c = a.bias ? score(z) + (double)a.bias[e] : (double)z;
    if (!(z > -INFINITY) || !(c > -INFINITY)) return -(double)INFINITY;
    return of_group && !a.bias && a.group_top > 1 ? score(z) : c;
  };
  unsigned long long kept = ~0ull;
  if (a.groups > 1) {
    for (int e = lane; e < a.E; e += 64) by[e] = value(e, row[e], true);
    wave_sync();
    double best = -INFINITY, second = -INFINITY;
    if (lane < a.groups)
      for (int i = 0; i < a.per; ++i) {
        const double x = by[lane * a.per + i];
        if (x > best) {
          second = best;
          best = x;
        } else if (x > second) {
          second = x;
        }
      }
    const double mine = a.group_top > 1 && second > -INFINITY ? best + second : best;
    int rank = 0;
    for (int g = 0; g < a.groups; ++g) {
      const double x = __shfl(mine, g, 64);
      rank += x > mine || (x == mine && g < lane);
    }
    kept = __ballot(lane < a.groups && rank < a.top_groups);
    wave_sync();
  }
  for (int e = lane; e < a.E; e += 64) {
    const double x = value(e, row[e], false);
    by[e] = kept >> (a.groups > 1 ? e / a.per : 0) & 1 ? x : -INFINITY;
  }
  wave_sync();
  unsigned taken = 0;
  for (int j = 0; j < a.k; ++j) {
    double b = -INFINITY;
    int at = INT_MAX;
    for (int v = 0, e = lane; e < a.E; ++v, e += 64)
      if (!(taken >> v & 1) && (by[e] > b || at == INT_MAX)) {
        b = by[e];
        at = e;
      }
    best_of<64>(b, at);
    if ((at & 63) == lane) taken |= 1u << (at >> 6);
    if (lane == 0) chosen[j] = b > -INFINITY ? at : ~at;
  }
}

// The two largest values of a lane's and its partner's.
template <int CTRL>
__device__ __forceinline__ void two_of(float& best, float& second) {
  const float b = __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(best), CTRL, 0xf, 0xf, false));
  const float s = __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(second), CTRL, 0xf, 0xf, false));
  second = fmaxf(fminf(best, b), fmaxf(second, s));
  best = fmaxf(best, b);
}

// How near two values compared in fp32 may be to each other for their order to be that of binary64.  In units of U32 a sigmoid is off by at most
// 4 (an exponent of 2 |z| and 2, s (1 - s) |z| < 0.23, the sum and the reciprocal), a softmax by 45 (3 |x| + 2 of the exponential, |x| exp(-|x|) <
// 0.37, and of the sum the mean of that, at most 3 ln E + 2, with 12 additions); adding the bias, of at most `bias`, rounds once more.  Twice that, and some.
__device__ __forceinline__ float nearest(bool sigmoid, float bias) { return ((sigmoid ? 16.f : 128.f) + 4.f * (bias + 1.f)) * U32; }

template <int G, int NV>
__global__ __launch_bounds__(SCORE_MOST * 64) void score_kernel(ScoreArgs a) {
  extern __shared__ __attribute__((aligned(16))) char smem[];
  constexpr int TOKENS = 64 / G;        // of a wavefront
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, waves = blockDim.x >> 6;
  const int g = lane & (G - 1), sub = lane / G;
  const int E = a.E, E4 = (E + 3) / 4 * 4;
  int32_t* const hist = reinterpret_cast<int32_t*>(smem);
  float* const bias_s = reinterpret_cast<float*>(smem + E4 * 4);             // [E4]
  uint8_t* const group_of = reinterpret_cast<uint8_t*>(smem + E4 * 8);       // [E4]
  char* const mine = smem + E4 * 8 + (E4 + 15) / 16 * 16 + (size_t)wave * score_lds_bytes(E, a.k, a.groups, TOKENS);
  const ScoreLds L = score_lds(mine, E, a.k, a.groups, TOKENS);
  const bool grouped = a.groups > 1 && a.top_groups < a.groups;
  const bool by_score = a.bias != nullptr, scored_groups = grouped && (by_score || a.group_top > 1);
  const bool need_softmax = !a.sigmoid && (by_score || scored_groups || !a.renorm);
  float z[NV * 4];
  auto fetch = [&](long long t) {
    const bool valid = t < a.T;
    const float* const row = a.logits + (valid ? t : 0) * E;
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      const int c = (v * G + g) * 4;
      if (valid && c + 3 < E) {
        const f32x4_f32 q = *reinterpret_cast<const f32x4_f32*>(row + c);
#pragma unroll
        for (int i = 0; i < 4; ++i) z[4 * v + i] = q[i];
      } else {
#pragma unroll
        for (int i = 0; i < 4; ++i) z[4 * v + i] = valid && c + i < E ? row[c + i] : -INFINITY;
      }
    }
  };
  const long long first = (long long)blockIdx.x * waves * TOKENS + wave * TOKENS, step = (long long)gridDim.x * waves * TOKENS;
  fetch(first + sub);
  float largest = 0.f;      // |bias|
  for (int e = threadIdx.x; e < E4; e += blockDim.x) {
    hist[e] = 0;
    if (grouped) group_of[e] = (uint8_t)min(e / a.per, a.groups - 1);
    const float b = a.bias && e < E ? a.bias[e] : 0.f;
    bias_s[e] = b;
    if (fabsf(b) < INFINITY) largest = fmaxf(largest, fabsf(b));
  }
  __shared__ float largest_of[16];
#pragma unroll
  for (int m = 32; m >= 1; m >>= 1) largest = fmaxf(largest, __shfl_xor(largest, m, 64));
  if (lane == 0) largest_of[wave] = largest;
  __syncthreads();
  for (int w = 0; w < waves; ++w) largest = fmaxf(largest, largest_of[w]);
  const float closest = nearest(a.sigmoid, largest);

  for (long long t0 = first; t0 < a.T; t0 += step, fetch(t0 + sub)) {
    const bool valid = t0 + sub < a.T;
    bool nan = false;
    float top = -INFINITY, inv_sum = 0.f, sum = 0.f;
#pragma unroll
    for (int i = 0; i < NV * 4; ++i) {
      nan |= z[i] != z[i];
      top = fmaxf(top, z[i]);
    }
    if (!a.sigmoid) {
#pragma unroll
      for (int m = G >> 1; m >= 1; m >>= 1) top = fmaxf(top, __shfl_xor(top, m, 64));
      nan |= top == INFINITY;
    }
    if (need_softmax) {
      float part[NV];
#pragma unroll
      for (int v = 0; v < NV; ++v) {
        part[v] = 0.f;
#pragma unroll
        for (int i = 0; i < 4; ++i) part[v] += z[4 * v + i] > -INFINITY ? __builtin_amdgcn_exp2f((z[4 * v + i] - top) * LOG2E) : 0.f;
      }
#pragma unroll
      for (int h = NV / 2; h >= 1; h >>= 1)
#pragma unroll
        for (int v = 0; v < h; ++v) part[v] += part[v + h];
      sum = part[0];
#pragma unroll
      for (int m = G >> 1; m >= 1; m >>= 1) sum += __shfl_xor(sum, m, 64);
      inv_sum = 1.f / sum;
    }
    auto score = [&](float x) {
      return a.sigmoid ? __builtin_amdgcn_rcpf(1.f + __builtin_amdgcn_exp2f(-x * LOG2E)) : __builtin_amdgcn_exp2f((x - top) * LOG2E) * inv_sum;
    };
    bool look = false;      // exactly, at the whole row

    // what classes are compared by, in z's place; -inf: not to be chosen.  What groups are compared by goes to LDS.
#pragma unroll
    for (int v = 0; v < NV; ++v) {
      const int c = (v * G + g) * 4;
      float of[4], bias[4] = {};
      if (by_score) {
        const float4 q = c < E ? *reinterpret_cast<const float4*>(bias_s + c) : make_float4(0.f, 0.f, 0.f, 0.f);
        bias[0] = q.x;
        bias[1] = q.y;
        bias[2] = q.z;
        bias[3] = q.w;
      }
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float x = z[4 * v + i];
        const bool live = x > -INFINITY;
        float s = 0.f;
        if (by_score || scored_groups) s = score(x);
        float y = by_score ? s + bias[i] : x;
        if (!live || !(y > -INFINITY)) y = -INFINITY;
        of[i] = !by_score && scored_groups && live ? s : y;
        z[4 * v + i] = y;
      }
      if (grouped && a.lanes) {
        // the two largest of the piece, then of the lanes that have the group's other pieces
        float best = fmaxf(of[0], of[1]), second = fminf(of[0], of[1]);
        const float b2 = fmaxf(of[2], of[3]), s2 = fminf(of[2], of[3]);
        second = fmaxf(fminf(best, b2), fmaxf(second, s2));
        best = fmaxf(best, b2);
        if (a.lanes >= 2) two_of<0xb1>(best, second);
        if (a.lanes >= 4) two_of<0x4e>(best, second);
        if (a.lanes >= 8) two_of<0x141>(best, second);
        if (a.lanes >= 16) two_of<0x140>(best, second);
        const int gr = (v * G + g) >> a.shift;
        if (gr < a.groups && (g & (a.lanes - 1)) == 0) L.group[sub * a.groups + gr] = a.group_top > 1 && second > -INFINITY ? best + second : best;
        __builtin_amdgcn_sched_barrier(0);   // one piece after the other: side by side they take more registers than there are
      } else if (grouped && c < E) {
        float* const to = L.of + sub * E + c;
#pragma unroll
        for (int i = 0; i < 4; ++i)
          if (c + i < E) to[i] = of[i];
      }
    }
    if (grouped) {
      wave_sync();
      if (!a.lanes) {
        const int pairs = TOKENS * a.groups;
        for (int p = lane; p < pairs; p += 64) {
          const int tok = p / a.groups, gr = p - tok * a.groups;
          const float* const from = L.of + tok * E + gr * a.per;
          float best = -INFINITY, second = -INFINITY;
          int at = lane % a.per;              // every lane begins elsewhere: they would meet in the same banks
          for (int i = 0; i < a.per; ++i) {
            const float x = from[at];
            second = fmaxf(second, fminf(best, x));
            best = fmaxf(best, x);
            at = at + 1 == a.per ? 0 : at + 1;
          }
          L.group[p] = a.group_top > 1 && second > -INFINITY ? best + second : best;
        }
        wave_sync();
      }
      // a token's lanes rank its groups, each every G-th
      unsigned long long kept = 0;
      const float* const of_token = L.group + sub * a.groups;
      for (int g0 = 0; g0 < a.groups; g0 += G) {
        const int gr = g0 + g;
        const float mine_ = gr < a.groups ? of_token[gr] : -INFINITY;
        int rank = 0;
        bool close = false;         // one behind it is near
        for (int i = 0; i < a.groups; ++i) {
          const float x = of_token[i];
          const bool ahead = x > mine_ || (x == mine_ && i < gr);
          rank += ahead;
          close |= !ahead && i != gr && mine_ > -INFINITY && !(mine_ - x > 2.f * closest);
        }
        look |= scored_groups && close && rank == a.top_groups - 1;
        const unsigned long long in = __ballot(gr < a.groups && rank < a.top_groups) >> (sub * G);
        kept |= (G == 64 ? in : in & ((1ull << (G & 63)) - 1)) << g0;
      }
#pragma unroll
      for (int v = 0; v < NV; ++v) {
        const int c = (v * G + g) * 4;
        if (a.lanes) {
          const int gr = min((v * G + g) >> a.shift, 63);
          if (!(kept >> gr & 1))
#pragma unroll
            for (int i = 0; i < 4; ++i) z[4 * v + i] = -INFINITY;
        } else {
          const unsigned ids = c < E ? *reinterpret_cast<const unsigned*>(group_of + c) : 0u;
#pragma unroll
          for (int i = 0; i < 4; ++i)
            if (!(kept >> (ids >> (8 * i) & 0xff) & 1)) z[4 * v + i] = -INFINITY;
        }
      }
    }

    // the rounds; by score two more: the first that is not chosen may change places with the last that is, the one behind it may not be near
    unsigned taken = 0;
    float before = INFINITY;
    bool order = false;     // two of the chosen and the first behind them are near
    const int pitch = a.k + 2, rounds = by_score ? min(a.k + 2, E) : a.k;
    for (int j = 0; j < rounds; ++j) {
      float b = -INFINITY;
      int bc = 0;
#pragma unroll
      for (int i = 0; i < NV * 4; ++i) {
        const bool better = z[i] > b && !(taken >> i & 1u);
        b = better ? z[i] : b;
        bc = better ? i : bc;
      }
      const int own = b > -INFINITY ? ((bc >> 2) * G + g) * 4 + (bc & 3) : INT_MAX;
      int at = own;
      best_of<G>(b, at);
      if (at == own) taken |= 1u << bc;
      if (j < a.k) look |= at == INT_MAX;           // somebody has to fill up
      if (by_score && j > 0 && at != INT_MAX && !(before - b > closest)) {
        if (j <= a.k) order = true;
        else look |= order;
      }
      if (j <= a.k && g == 0) L.chosen[sub * pitch + j] = at;
      before = b;
    }
    if (rounds <= a.k && g == 0) L.chosen[sub * pitch + a.k] = INT_MAX;
    look |= order && !(a.sigmoid && a.k < SCORE_MAX_K);
    const unsigned long long lanes_of = (G == 64 ? ~0ull : (1ull << (G & 63)) - 1) << (sub * G);
    const bool bad = (__ballot(nan) & lanes_of) != 0;
    look = (__ballot(look) & lanes_of) != 0;
    if (g == 0) {
      L.softmax[sub] = make_float2(bad ? NAN : top, sum);   // NaN: the row is not a number
      L.chosen[sub * pitch + a.k + 1] = order && !look;
    }
    wave_sync();
    unsigned long long again = __ballot(g == 0 && valid && look);
    while (again) {
      const int tok = (__ffsll((unsigned long long)again) - 1) / G;
      again &= again - 1;
      choose_exactly(a, a.logits + (t0 + tok) * E, reinterpret_cast<double*>(L.of), L.chosen + tok * pitch);
      wave_sync();
    }

    // 16 lanes a token: where values are near, the k and the first behind them in the order of binary64; then gates relative to the largest of the k
    const int j = lane & 15;
    for (int u = 0; u < TOKENS; u += 4) {
      const int tok = u + (lane >> 4);
      const long long tt = t0 + tok;
      const bool there = tok < TOKENS && tt < a.T;
      const int c = there && j <= a.k ? L.chosen[tok * pitch + j] : INT_MAX;
      const bool real_c = c >= 0 && c != INT_MAX;
      const float x = real_c ? a.logits[tt * E + c] : 0.f;
      int at = j;
      if (__any(there && L.chosen[(there ? tok : 0) * pitch + a.k + 1])) {
        const double y = real_c ? 1. / (1. + exp(-(double)x)) + (double)bias_s[c] : -(double)INFINITY;
        int rank = 0;
        for (int i = 0; i <= a.k; ++i) {
          const double other = __shfl(y, i, 16);
          const int oc = __shfl(c, i, 16);
          rank += other > y || (other == y && oc < c);
        }
        if (there && L.chosen[tok * pitch + a.k + 1]) at = rank;
      }
      const bool here = there && at < a.k && j <= a.k;
      const bool real = here && real_c;
      const float2 q = L.softmax[there ? tok : 0];
      float gate;
      if (a.renorm) {
        const float low = a.sigmoid ? fminf(x, 0.f) : x;
        float m = real ? low : -INFINITY;
#pragma unroll
        for (int o = 8; o >= 1; o >>= 1) m = fmaxf(m, __shfl_xor(m, o, 64));
        gate = real ? expf(low - m) : 0.f;
        if (a.sigmoid && real) gate /= 1.f + expf(-fabsf(x));
        float s = gate;
#pragma unroll
        for (int o = 8; o >= 1; o >>= 1) s += __shfl_xor(s, o, 64);
        gate = real ? gate / s : 0.f;
      } else if (a.sigmoid) {
        gate = real ? sigmoid_of(x) : 0.f;
      } else {
        gate = real ? expf(x - q.x) / q.y : 0.f;
      }
      if (here) {
        const int e = real ? c : ~c;
        a.idx[tt * a.k + at] = e;
        a.gate[tt * a.k + at] = q.x != q.x ? NAN : a.scale * gate;
        atomicAdd(&hist[e], 1);
      }
    }
    wave_sync();
  }
  __syncthreads();
  for (int e = threadIdx.x; e < E; e += blockDim.x) {
    if (a.alone) a.hist[e] = hist[e];
    else if (hist[e]) atomicAdd(&a.hist[e], hist[e]);
  }
}

struct ScoreBwdArgs {
  const float* logits;
  const int32_t* idx;
  const float *gate, *dgate;
  float* dlogits;
  int T, E, k, renorm, sigmoid;
  float scale;
};

// dz of the chosen: renormalised g (dg - sum g dg), sigmoid: times (1 - s); a plain softmax: p_e ([e chosen] dg - sum p dg) for every class.  16 lanes a token:
// they put what the k classes get into a row of zeros in LDS and write the row.
__global__ __launch_bounds__(BWD_WAVES * 64) void score_bwd_kernel(ScoreBwdArgs a) {
  extern __shared__ __attribute__((aligned(16))) float rows[];
  const int j = threadIdx.x & 15, sub = threadIdx.x >> 4;
  constexpr int AT_ONCE = BWD_WAVES * 4;
  const int E = a.E, E4 = (E + 3) / 4 * 4;
  float* const out = rows + sub * E4;
  const bool dense = !a.sigmoid && !a.renorm;
  for (long long t = (long long)blockIdx.x * AT_ONCE + sub; t < a.T; t += (long long)gridDim.x * AT_ONCE) {
    const float* const row = a.logits + t * E;
    int at = -1;
    float g = 0.f, dg = 0.f, z = 0.f;
    if (j < a.k) {
      at = a.idx[t * a.k + j];
      g = a.gate[t * a.k + j] / a.scale;
      dg = a.dgate[t * a.k + j] * a.scale;
      if (g == 0.f || (unsigned)at >= (unsigned)E) at = -1;   // only filled up
      else if (a.sigmoid) z = row[at];
    }
    for (int c = j * 4; c < E4; c += 64) *reinterpret_cast<float4*>(out + c) = make_float4(0.f, 0.f, 0.f, 0.f);
    if (at < 0) g = dg = 0.f;
    float dot = g * dg;
#pragma unroll
    for (int o = 8; o >= 1; o >>= 1) dot += __shfl_xor(dot, o, 64);
    float dz = a.renorm ? g * (dg - dot) : g * dg;
    if (a.sigmoid) dz *= sigmoid_of(-z);
    float top = -INFINITY, sum = 0.f;
    if (dense) {
      for (int e = j; e < E; e += 16) top = fmaxf(top, row[e]);
#pragma unroll
      for (int o = 8; o >= 1; o >>= 1) top = fmaxf(top, __shfl_xor(top, o, 64));
      for (int e = j; e < E; e += 16) sum += row[e] == -INFINITY ? 0.f : expf(row[e] - top);
#pragma unroll
      for (int o = 8; o >= 1; o >>= 1) sum += __shfl_xor(sum, o, 64);
    }
    wave_sync();
    if (at >= 0) out[at] = dz;
    wave_sync();
    for (int c = j * 4; c < E; c += 64) {
      const float4 q = *reinterpret_cast<const float4*>(out + c);
      float x[4] = {q.x, q.y, q.z, q.w};
      if (dense)
#pragma unroll
        for (int i = 0; i < 4; ++i)
          if (c + i < E) x[i] -= row[c + i] == -INFINITY ? 0.f : expf(row[c + i] - top) / sum * dot;
      float* const to = a.dlogits + t * E + c;
      if (c + 3 < E) {
        const f32x4_f32 y = {x[0], x[1], x[2], x[3]};
        *reinterpret_cast<f32x4_f32*>(to) = y;
      } else {
#pragma unroll
        for (int i = 0; i < 4; ++i)
          if (c + i < E) to[i] = x[i];
      }
    }
    wave_sync();
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


// Lanes of a token: few, with up to 16 classes each (32 need more registers than a workgroup of 16 wavefronts has: 65536 tokens of 128 classes 55 us, 16 each
// 48); a small batch is spread over more of them, so that the chip is filled.
static void score_shape(int E, int T, int& G, int& NV) {
  const int vecs = cdiv(E, 4);
  G = 1;
  while (G * 4 < vecs) G <<= 1;
  while (G < vecs && G < 64 && (long long)T * G < 512LL * 256) G <<= 1;
  const int need = cdiv(vecs, G);
  NV = need <= 1 ? 1 : need <= 2 ? 2 : 4;
}

}  // namespace symi

using namespace symi;

extern "C" int symi_route_scored(const symi_ctx* ctx, const symi_score* hp, const float* logits, const float* bias, int32_t* idx,
                                 float* gate, int32_t* hist, void* stream) {
  SYMI_ENTER(ctx, "symi_route_scored");
  if (int rc = check_score(cfg, hp, "symi_route_scored")) return rc;
  SYMI_REQUIRE(hist && (cfg->T == 0 || (logits && idx && gate)), "symi_route_scored", "NULL pointer");
  hipStream_t st = as_stream(stream);
  const int E = cfg->E, T = cfg->T, k = cfg->k;
  int G, NV;
  score_shape(E, T, G, NV);
  const int per_wave = 64 / G;
  const int E4 = cdiv(E, 4) * 4, of_all = E4 * 8 + cdiv(E4, 16) * 16, of_wave = score_lds_bytes(E, k, hp->groups, per_wave);
  const int per = E / hp->groups, pieces = per % 4 ? 0 : per / 4;
  const int lanes = pieces && !(pieces & (pieces - 1)) && pieces <= std::min(G, 16) ? pieces : 0;
  // a small batch: one workgroup, which needs no cleared counts
  const bool alone = T > 0 && (long long)T * E * (k + 2) <= 32768 && T <= SCORE_MOST * per_wave && of_all + cdiv(T, per_wave) * of_wave <= SCORE_LDS;
  if (!alone) launch_fill_i32(ctx, hist, E, 0, st);
  if (T > 0) {
    const ScoreArgs a = {logits, bias, idx, gate, hist, T, E, k, cfg->renorm, hp->score == SYMI_SIGMOID, hp->groups, E / hp->groups,
                         hp->top_groups, hp->group_top, hp->scale, lanes, lanes ? __builtin_ctz(lanes) : 0, alone};
    // every workgroup adds its counts to the same E words, one after the other: as few of them as fill the chip
    int waves = alone ? cdiv(T, per_wave) : 1;
    while (!alone && waves < SCORE_MOST && cdiv(T, per_wave * waves) > ctx->cus && of_all + 2 * waves * of_wave <= SCORE_LDS) waves *= 2;
    const size_t sh = of_all + waves * of_wave;
    const int grid = alone ? 1 : std::min(cdiv(T, per_wave * waves), std::max(1, 16 / waves) * ctx->cus);
#define SYMI_SCORE_CASE(GG, NN)                                                                            \
  case GG * 16 + NN:                                                                                       \
    SYMI_TIMED(ctx, K_SCORE, st, (score_kernel<GG, NN><<<grid, waves * 64, sh, st>>>(a)));                 \
    break;
#define SYMI_SCORE_G(GG) SYMI_SCORE_CASE(GG, 1) SYMI_SCORE_CASE(GG, 2) SYMI_SCORE_CASE(GG, 4)
    switch (G * 16 + NV) {
      SYMI_SCORE_G(1) SYMI_SCORE_G(2) SYMI_SCORE_G(4) SYMI_SCORE_G(8) SYMI_SCORE_G(16) SYMI_SCORE_G(32) SYMI_SCORE_G(64)
      default:
        set_error("symi_route_scored: no kernel for %d lanes x %d pieces per token", G, NV);
        return SYMI_EUNSUPPORTED;
    }
#undef SYMI_SCORE_G
#undef SYMI_SCORE_CASE
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
  const int grid = std::min(cdiv(cfg->T, BWD_WAVES * 4), 8 * ctx->cus);
  const size_t sh = (size_t)BWD_WAVES * 4 * cdiv(cfg->E, 4) * 4 * sizeof(float);
  SYMI_TIMED(ctx, K_SCORE_BWD, st, (score_bwd_kernel<<<grid, BWD_WAVES * 64, sh, st>>>(a)));
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
