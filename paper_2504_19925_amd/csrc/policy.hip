// symi_token_logp / symi_policy_loss: log probabilities of the chosen tokens, the clipped policy loss with a KL term, and
// the gradient of the logits.
//
// Per row of logits, in base 2 with c = log2(e) / temperature: m = max z_j, s = sum 2^(c (z_j - m)),
//   logp = ln 2 c (z_a - m) - ln s,   dlogits_j = u ([j = a] - 2^(c (z_j - m)) / s),   u = grad_scale w / temperature dL/dlogp.
// The weights are the caller's, so u needs nothing from other rows: one workgroup takes a row from its logits to
// their gradient.  A row's statistics are fp32.  logp, and the differences that the ratio and the KL are exponentials of, are taken in 64
// bits from there; ratio, KL and a token's terms are fp32 again, and the four sums over the rows 64 bits, by one workgroup, in order.
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
  template <bool ONCE>   // nobody reads it again
  static __device__ __forceinline__ Raw load(const Elem* p) {
    const Vec* const q = reinterpret_cast<const Vec*>(p);
    return __builtin_bit_cast(Raw, ONCE ? __builtin_nontemporal_load(q) : *q);
  }
  static __device__ __forceinline__ void store(Elem* p, Raw r) { *reinterpret_cast<Vec*>(p) = __builtin_bit_cast(Vec, r); }
  static __device__ __forceinline__ float value(Elem x) {
    if constexpr (BF16) return bf16_to_f32(x); else return x;
  }
  static __device__ __forceinline__ Elem element(float x) {
    if constexpr (BF16) return f32_to_bf16(x); else return x;
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

// c (x - ref) in one operation, as c x - by with by = c ref rounded, where what the rounding makes of the power can be put right afterwards: by
// `rest`, 2^(by - c ref) to second order (the third is below 2^-25).  Elsewhere, among masks of -1e10 or -1e30, c x - by may be anything.
struct Exponent {
  float by, rest;
  bool near;
};
__device__ __forceinline__ Exponent exponent_of(float ref, float c) {
  const float by = ref * c, y = fmaf(ref, c, -by) * -0.693147181f;
  return {by, fmaf(y, fmaf(y, 0.5f, 1.f), 1.f), fabsf(by) < 0x1p18f};
}

// (m, s) of a set of logits: m the largest, s the sum of 2^(c (z - m)).
__device__ __forceinline__ void join(float& m, float& s, float m2, float s2, float c) {
  const float top = fmaxf(m, m2);
  const float ref = top == -INFINITY ? 0.f : top;   // nothing but -inf so far: 2^(c (-inf - 0)) = 0
  s = s * exp2_((m - ref) * c) + s2 * exp2_((m2 - ref) * c);
  m = top;
}

// What a token adds to the loss, and dL/dlogp.  clipped tokens have no gradient from their advantage.
struct Token {
  float gain, kl, slope;
  bool clipped;
};
__device__ __forceinline__ Token token_loss(const PolicyScalars& p, double logp, float old, bool has_ref, float ref, float A) {
  Token k;
  const float r = expf((float)(logp - old));
  k.clipped = (A > 0.f && r > 1.f + p.clip_high) || (A < 0.f && r < 1.f - p.clip_low);
  k.gain = A == 0.f ? 0.f : -A * (k.clipped ? (A > 0.f ? 1.f + p.clip_high : 1.f - p.clip_low) : r);   // also where r is infinite
  k.slope = k.clipped || A == 0.f ? 0.f : -A * r;
  k.kl = 0.f;
  if (has_ref) {
    const float far = (float)(ref - logp), e = expm1f(far);
    // e^x - x - 1 loses all digits near 0, where it is x^2 / 2 + x^3 / 6 + ...
    k.kl = fabsf(far) < 0.125f ? far * far * (0.5f + far * (1.f / 6 + far * (1.f / 24 + far * (1.f / 120 + far * (1.f / 720))))) : e - far;
    if (p.kl_coef > 0.f) k.slope -= p.kl_coef * e;   // a KL that is only looked at may be infinite
  }
  return k;
}

struct PolicyArgs {
  const void* logits;
  int V, ld;
  const int32_t* action;
  const float *logp_old, *logp_ref, *advantage, *weight;
  float* logp;
  float4* terms;
  void* dlogits;
  PolicyScalars p;
};

// The gradient of a logit is minus 2^(c (z - m)), with u more for the chosen token.  The power is taken as the square of its root:
// 2^(c (z - m)) itself would become 0 below 2^-126, where the gradient in single precision need not be 0, and an exponent that is
// moved up instead (m less a constant) loses the last bits of those near 0, which are most of the sum.  Halves are exact.
struct Slope {
  float u, minus, half_c, half_by, m;   // near: fma(z, half_c, -half_by) is the root's exponent
  bool near;
  __device__ __forceinline__ float of(float root) const { return minus * root * root; }
  __device__ __forceinline__ float of_near(float x) const { return of(exp2_(fmaf(x, half_c, -half_by))); }
  __device__ __forceinline__ float of_far(float x) const { return of(exp2_((x - m) * half_c)); }
};
__device__ __forceinline__ Slope slope_of(const PolicyScalars& p, float w, float slope, float m, float s) {
  const float u = p.scale * p.inv_temp * w * slope;
  const Exponent e = exponent_of(m, p.c);
  return {u, -u / s * (e.near ? e.rest : 1.f), 0.5f * p.c, 0.5f * e.by, m, e.near};
}

// What a workgroup does with a row of logits, every thread NV pieces of it at a time.
template <bool BF16, bool ONCE, int THREADS, int NV>
struct Row {
  using P = Piece<BF16>;
  using Elem = typename P::Elem;
  static constexpr int N = P::N, STEP = NV * THREADS;
  // Pieces begin at multiples of 16 bytes, wherever the row does (8192 rows of 4493 bf16, seven in eight of them unaligned: 46 us
  // with pieces that begin with the row, against 38 for rows of 4496).  The up to seven logits before the first piece
  // and behind the last one are the edge, one of them each of the threads below 16.
  const Elem* z;       // of the first piece
  int end, q, j;       // pieces; the chosen token's piece and place in it (or no piece)
  int V, head, tid, token;
  float c, edge;
  typename P::Raw r[NV];

  __device__ __forceinline__ Row(const PolicyArgs& g, long long t, int token, int tid) : V(g.V), tid(tid), token(token), c(g.p.c) {
    const Elem* const row = static_cast<const Elem*>(g.logits) + t * g.ld;
    head = min(g.V, (int)((16 - (reinterpret_cast<uintptr_t>(row) & 15)) % 16 / sizeof(Elem)));
    end = (g.V - head) / N;
    z = row + head;
    const int tail = head + end * N;
    q = token >= head && token < tail ? (token - head) / N : -1;
    j = (token - head) % N;
    edge = -INFINITY;
  }
  // the column of the thread's edge logit, or -1
  __device__ __forceinline__ int edge_column() const {
    if (tid < 8) return tid < head ? tid : -1;
    const int at = head + end * N + tid - 8;
    return tid < 16 && at < V ? at : -1;
  }
  // requested last, after the first pieces
  __device__ __forceinline__ void fetch_edge() {
    const int e = edge_column();
    if (e >= 0) edge = P::value(z[e - head]);
  }
  __device__ __forceinline__ void take_edge(float& m, float& s, float* chosen) {
    const int e = edge_column();
    if (e < 0) return;
    join(m, s, edge, 1.f, c);
    if (e == token) *chosen = edge;
  }
  __device__ __forceinline__ void give_edge(Elem* dz, const Slope& d) {
    const int e = edge_column();
    if (e >= 0) dz[e] = P::element((d.near ? d.of_near(edge) : d.of_far(edge)) + (e == token ? d.u : 0.f));
  }
  // the pieces q0 + tid, q0 + THREADS + tid, ... below `stop`
  __device__ __forceinline__ void fetch(int q0, int stop) {
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int at = q0 + i * THREADS + tid;
      r[i] = P::none();
      if (at < stop) r[i] = P::template load<ONCE>(z + (long long)at * N);
    }
  }
  // adds what is held to the thread's (m, s); the chosen token's logit goes to *chosen
  __device__ __forceinline__ void take(int q0, int stop, float& m, float& s, float* chosen) {
    float top = -INFINITY;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      if (q0 + i * THREADS >= stop) continue;
      float x[N];
      P::unpack(r[i], x);
#pragma unroll
      for (int k = 0; k < N; ++k) top = fmaxf(top, x[k]);
      if (q0 + i * THREADS + tid == q && q < stop) {
#pragma unroll
        for (int k = 0; k < N; ++k)
          if (k == j) *chosen = x[k];
      }
    }
    const float base = fmaxf(m, top), ref = base == -INFINITY ? 0.f : base;   // nothing but -inf so far
    s *= exp2_((m - ref) * c);
    m = base;
    const Exponent e = exponent_of(ref, c);
    float sum = 0.f;
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      if (q0 + i * THREADS >= stop) continue;
      float x[N];
      forget(r[i]);
      P::unpack(r[i], x);
#pragma unroll
      for (int k = 0; k < N; ++k) sum += exp2_(fmaf(x[k], c, -e.by));
    }
    sum *= e.rest;
    if (__builtin_expect(__ballot(!e.near) != 0, 0)) {   // anew; what is held stays as it is
      float far = 0.f;
#pragma unroll 1
      for (int at = q0 + tid; at < min(stop, q0 + STEP); at += THREADS) {
        float x[N];
        P::unpack(P::template load<ONCE>(z + (long long)at * N), x);
#pragma unroll
        for (int k = 0; k < N; ++k) far += exp2_((x[k] - ref) * c);
      }
      if (!e.near) sum = far;
    }
    s += sum;
  }
  __device__ __forceinline__ void give_piece(int at, float (&x)[N], Elem* dz, const Slope& d) {
    if (at == q) {
#pragma unroll
      for (int k = 0; k < N; ++k)
        if (k == j) x[k] += d.u;
    }
    P::store(dz + head + (long long)at * N, P::pack(x));
  }
  // writes the gradient of what is held; dz: of the row's first logit
  __device__ __forceinline__ void give(int q0, int stop, Elem* dz, const Slope& d) {
    if (__builtin_expect(!d.near, 0)) {
#pragma unroll 1
      for (int at = q0 + tid; at < min(stop, q0 + STEP); at += THREADS) {
        float x[N];
        P::unpack(P::template load<ONCE>(z + (long long)at * N), x);
#pragma unroll
        for (int k = 0; k < N; ++k) x[k] = d.of_far(x[k]);
        give_piece(at, x, dz, d);
      }
      return;
    }
#pragma unroll
    for (int i = 0; i < NV; ++i) {
      const int at = q0 + i * THREADS + tid;
      if (q0 + i * THREADS >= stop) continue;
      float x[N];
      forget(r[i]);
      P::unpack(r[i], x);
#pragma unroll
      for (int k = 0; k < N; ++k) x[k] = d.of_near(x[k]);
      if (at < stop) give_piece(at, x, dz, d);
    }
  }
};

__device__ __forceinline__ void join_wave(float& m, float& s, float c) {
#pragma unroll
  for (int k = 32; k >= 1; k >>= 1) join(m, s, __shfl_xor(m, k, 64), __shfl_xor(s, k, 64), c);
}
// (m, s) of a workgroup, in every thread.
template <int THREADS>
__device__ __forceinline__ void join_threads(float& m, float& s, float c) {
  __shared__ float ms[THREADS / 64], ss[THREADS / 64];
  join_wave(m, s, c);
  if (THREADS > 64 && (threadIdx.x & 63) == 0) {
    ms[threadIdx.x >> 6] = m;
    ss[threadIdx.x >> 6] = s;
  }
  __syncthreads();
  if (THREADS == 64) return;
  m = ms[0];
  s = ss[0];
#pragma unroll
  for (int k = 1; k < THREADS / 64; ++k) join(m, s, ms[k], ss[k], c);
}

// Zeros to p[0 .. n).
template <bool BF16>
__device__ __forceinline__ void clear(typename Piece<BF16>::Elem* p, int n, int tid, int threads) {
  using P = Piece<BF16>;
  const int head = min(n, (int)((16 - (reinterpret_cast<uintptr_t>(p) & 15)) % 16 / sizeof(typename P::Elem)));
  const int pieces = (n - head) / P::N, tail = head + pieces * P::N;
  for (int j = tid; j < head; j += threads) p[j] = 0;
  for (int q = tid; q < pieces; q += threads) P::store(p + head + (long long)q * P::N, typename P::Raw{0, 0, 0, 0});
  for (int j = tail + tid; j < n; j += threads) p[j] = 0;
}

__device__ __forceinline__ float4 terms_of(const PolicyScalars& p, float w, const Token& k) {
  return float4{w * (p.kl_coef > 0.f ? k.gain + p.kl_coef * k.kl : k.gain), w * k.gain, w * k.kl, k.clipped ? w : 0.f};
}
// In 64 bits, as a ratio exp(logp - logp_old) has the absolute error of logp, and 32 bits leave 5e-7 to a logp of -10; the
// logarithm is that of a number near 1 in 32 bits (off by 3e-8) and a multiple of ln 2.
__device__ __forceinline__ double logp_of(const PolicyScalars& p, float za, float m, float s) {
  int k;
  float f = frexpf(s, &k);
  if (f < 0.70710678f) {   // nearer to 1: the logarithm of 1 is 0
    f *= 2.f;
    k -= 1;
  }
  return (((double)za - (double)m) * (double)p.c - k) * 0.693147180559945309 - (double)logf(f);
}

// A workgroup of THREADS takes a row.  What fits is read once and stays in registers from the logits to their gradient; of a
// longer row the last STEP pieces stay and the ones before them are read again.
// Up to eight pieces a thread leave 64 registers: eight wavefronts a SIMD, two workgroups of 1024 a unit.
// Bound by memory on many rows: with the gradient 16384 of 131072 in bf16, a quarter masked, 1444 us, 3.2 GB fetched and 4.3 written
// (5.2 TB/s, vector units busy 61 %); without it 8192 of 50001, 40 % masked, 84 us, 0.51 GB (6.0 TB/s, busy 91 %).  777 rows of 32003 in
// fp32, a fifth masked, 42 us at 4.3 TB/s: 622 rows on places for 512 workgroups.  16 rows of 128000: 11 us, the exponentials of 16 units.
template <bool BF16, bool GRAD, int THREADS, int NV>
__global__ __launch_bounds__(THREADS, NV <= 8 ? 8 : 4) void policy_kernel(PolicyArgs g) {
  using R = Row<BF16, !GRAD, THREADS, NV>;
  __shared__ float chosen;
  const int tid = threadIdx.x;
  const long long t = blockIdx.x;
  const int token = g.action[t];
  R row(g, t, token, tid);
  auto* const dz = static_cast<typename R::Elem*>(g.dlogits) + (GRAD ? t * g.ld : 0);
  const float w = g.weight ? g.weight[t] : 1.f;
  if (w == 0.f || (unsigned)token >= (unsigned)g.V) {
    if (tid == 0) {
      g.logp[t] = 0.f;
      if (g.terms) g.terms[t] = float4{0.f, 0.f, 0.f, 0.f};
    }
    if (GRAD) clear<BF16>(dz, g.ld, tid, THREADS);
    return;
  }
  float old = 0.f, ref = 0.f, A = 0.f;   // requested with the row
  if (g.terms) {
    old = g.logp_old[t];
    A = g.advantage[t];
    if (g.logp_ref) ref = g.logp_ref[t];
  }
  const int end = row.end, last = end > R::STEP ? end - R::STEP : 0;   // from `last` on pieces stay
  float m = -INFINITY, s = 0.f;
  for (int q0 = 0; q0 < last; q0 += R::STEP) {
    row.fetch(q0, min(q0 + R::STEP, last));
    row.take(q0, min(q0 + R::STEP, last), m, s, &chosen);
  }
  row.fetch(last, end);
  row.fetch_edge();
  row.take(last, end, m, s, &chosen);
  row.take_edge(m, s, &chosen);
  join_threads<THREADS>(m, s, g.p.c);
  const double lp = logp_of(g.p, chosen, m, s);
  if (tid == 0) g.logp[t] = (float)lp;
  if (!g.terms) return;
  const Token k = token_loss(g.p, lp, old, g.logp_ref != nullptr, ref, A);
  if (tid == 0) g.terms[t] = terms_of(g.p, w, k);
  if (!GRAD) return;
  const Slope d = slope_of(g.p, w, k.slope, m, s);
  row.give(last, end, dz, d);
  row.give_edge(dz, d);
  for (int q0 = (last - 1) / R::STEP * R::STEP; last && q0 >= 0; q0 -= R::STEP) {   // what was read last is the nearest
    row.fetch(q0, min(q0 + R::STEP, last));
    row.give(q0, min(q0 + R::STEP, last), dz, d);
  }
  clear<BF16>(dz + g.V, g.ld - g.V, tid, THREADS);
}

// Few rows: every wavefront that policy_kernel would give a row is a workgroup of its own, in two launches.  The first
// leaves each wavefront's (m, s) and the chosen logit; the second joins them, reads the logits again and writes their
// gradient.  Which pieces a thread takes and how sums are joined is that of policy_kernel with a gradient, so a row's bits do not
// depend on the number of rows (only on where it begins within 16 bytes); without a gradient they do, see launch_rows.  The first workgroup of the second launch takes the sums over the tokens.
// Bound by latency, as the second reading comes from the caches; measured at wants_parts.
constexpr int SUM_SPLIT_THREADS = 256;
constexpr int PART_MAX = 16;         // wavefronts of a row
constexpr int PART_ROWS_MAX = 256;   // rows of a batch that is split

struct Parts {
  float2* ms;      // [T, wavefronts]
  float* chosen;   // [T]
};

template <bool BF16, int THREADS, int NV>
__global__ __launch_bounds__(64) void policy_part_kernel(PolicyArgs g, Parts parts) {
  using R = Row<BF16, false, THREADS, NV>;
  constexpr int WAVES = THREADS / 64;
  const int wave = blockIdx.x % WAVES;
  const long long t = blockIdx.x / WAVES;
  const int token = g.action[t];
  R row(g, t, token, wave * 64 + threadIdx.x);
  if (g.weight[t] == 0.f || (unsigned)token >= (unsigned)g.V) return;
  const int end = row.end, last = end > R::STEP ? end - R::STEP : 0;
  float m = -INFINITY, s = 0.f;
  for (int q0 = 0; q0 < last; q0 += R::STEP) {
    row.fetch(q0, min(q0 + R::STEP, last));
    row.take(q0, min(q0 + R::STEP, last), m, s, parts.chosen + t);
  }
  row.fetch(last, end);
  row.fetch_edge();
  row.take(last, end, m, s, parts.chosen + t);
  row.take_edge(m, s, parts.chosen + t);
  join_wave(m, s, g.p.c);
  if (threadIdx.x == 0) parts.ms[t * WAVES + wave] = float2{m, s};
}

template <int THREADS>
__device__ __forceinline__ void add_terms(double (&sum)[4], float* __restrict__ stats) {
  __shared__ double part[THREADS / 64][4];
#pragma unroll
  for (int k = 0; k < 4; ++k) {
#pragma unroll
    for (int m = 32; m >= 1; m >>= 1) sum[k] += __shfl_xor(sum[k], m, 64);
    if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6][k] = sum[k];
  }
  __syncthreads();
  if (threadIdx.x < 4) {
    double all = 0.;
    for (int w = 0; w < THREADS / 64; ++w) all += part[w][threadIdx.x];
    stats[threadIdx.x] = (float)all;
  }
}

// m and s of a row: those of its wavefronts, joined in order.
template <int WAVES, class Load>
__device__ __forceinline__ void join_waves(float& m, float& s, float c, Load load) {
  float2 x = load(0);
  m = x.x;
  s = x.y;
#pragma unroll
  for (int k = 1; k < WAVES; ++k) {
    x = load(k);
    join(m, s, x.x, x.y, c);
  }
}

template <bool BF16, int THREADS, int NV>
__global__ __launch_bounds__(SUM_SPLIT_THREADS) void policy_apply_kernel(PolicyArgs g, Parts parts, int T, float* __restrict__ stats) {
  using R = Row<BF16, true, THREADS, NV>;
  constexpr int WAVES = THREADS / 64;
  float m, s;
  if (blockIdx.x == 0) {
    double sum[4] = {};
    for (int t = threadIdx.x; t < T; t += SUM_SPLIT_THREADS) {
      const float w = g.weight[t];
      double lp = 0.;
      if (w != 0.f && (unsigned)g.action[t] < (unsigned)g.V) {
        join_waves<WAVES>(m, s, g.p.c, [&](int k) { return parts.ms[(long long)t * WAVES + k]; });
        lp = logp_of(g.p, parts.chosen[t], m, s);
        const Token k = token_loss(g.p, lp, g.logp_old[t], g.logp_ref != nullptr, g.logp_ref ? g.logp_ref[t] : 0.f, g.advantage[t]);
        const float4 x = terms_of(g.p, w, k);
        sum[0] += x.x; sum[1] += x.y; sum[2] += x.z; sum[3] += x.w;
      }
      g.logp[t] = (float)lp;
    }
    add_terms<SUM_SPLIT_THREADS>(sum, stats);
    return;
  }
  if (threadIdx.x >= 64) return;   // the other workgroups are a wavefront
  const int wave = (blockIdx.x - 1) % WAVES;
  const long long t = (blockIdx.x - 1) / WAVES;
  const int token = g.action[t];
  R row(g, t, token, wave * 64 + threadIdx.x);
  auto* const dz = static_cast<typename R::Elem*>(g.dlogits) + t * g.ld;
  const float w = g.weight[t];
  const int end = row.end;
  if (w == 0.f || (unsigned)token >= (unsigned)g.V) {
    clear<BF16>(dz, g.ld, row.tid, THREADS);
    return;
  }
  if (wave == 0) clear<BF16>(dz + g.V, g.ld - g.V, row.tid, 64);
  row.fetch(0, end);
  row.fetch_edge();
  join_waves<WAVES>(m, s, g.p.c, [&](int k) { return parts.ms[t * WAVES + k]; });
  const double lp = logp_of(g.p, parts.chosen[t], m, s);
  const Token k = token_loss(g.p, lp, g.logp_old[t], g.logp_ref != nullptr, g.logp_ref ? g.logp_ref[t] : 0.f, g.advantage[t]);
  const Slope d = slope_of(g.p, w, k.slope, m, s);
  row.give_edge(dz, d);
  for (int q0 = 0;;) {
    row.give(q0, end, dz, d);
    if ((q0 += R::STEP) >= end) break;
    row.fetch(q0, end);
  }
}

// One workgroup, so that the order is that of the tokens: 16384 tokens 12 us, 8192 7 us; with eight requests a thread in flight 0.2 us less.
__global__ __launch_bounds__(SUM_THREADS) void policy_sum_kernel(const float4* __restrict__ terms, int T, float* __restrict__ stats) {
  double sum[4] = {};
  for (long long t = threadIdx.x; t < T; t += SUM_THREADS) {
    const float4 x = terms[t];
    sum[0] += x.x; sum[1] += x.y; sum[2] += x.z; sum[3] += x.w;
  }
  add_terms<SUM_THREADS>(sum, stats);
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

struct PolicyWs {
  size_t terms, ms, chosen, total;
};
static PolicyWs policy_ws(const symi_cfg* c) {
  PolicyWs L;
  const size_t rows = std::min(c->T, PART_ROWS_MAX);
  L.terms = 0;
  L.ms = align_up((size_t)c->T * sizeof(float4), 256);
  L.chosen = L.ms + align_up(rows * PART_MAX * sizeof(float2), 256);
  L.total = L.chosen + align_up(rows * sizeof(float), 256) + 256;
  return L;
}

static PolicyScalars scalars(const symi_policy* hp) {
  return {hp->clip_low, hp->clip_high, hp->kl_coef, hp->inv_temperature, hp->grad_scale, (float)std::min(1.4426950408889634 * hp->inv_temperature, 3.4028234663852886e38)};
}

// The workgroup for a row with its gradient: f(THREADS, NV).  The smallest that holds the row comes first, with four to 16 pieces a
// thread: us for 8192 rows in bf16, threads x pieces, sums included.  V = 3000: 64 x 8 29, 128 x 8 30, 256 x 4 36; 10001: 256 x 4 74, 256 x 8
// 70, 512 x 4 81; 17010: 256 x 16 110, 512 x 8 112; 28000: 512 x 8 185, 512 x 12 172, 256 x 16 188; 45000: 512 x 12 286, 512 x 16
// 271; 50001: 512 x 16 300, 512 x 12 317.  Longer rows are read again in part, most of it from the memory-side cache: 4096
// of 100000 with eight pieces of 1024 threads 338, with 16 363; 16384 of 131072, a quarter masked, 1495 and 1451; 2048 of
// 200000 in fp32 880 and 776.
template <int X> using Int = std::integral_constant<int, X>;
template <class F>
static void by_length(int pieces, F f) {
  if (pieces <= 64 * 4) f(Int<64>(), Int<4>());
  else if (pieces <= 512) f(Int<128>(), Int<8>());
  else if (pieces <= 256 * 4) f(Int<256>(), Int<4>());
  else if (pieces <= 256 * 8) f(Int<256>(), Int<8>());
  else if (pieces <= 3000) f(Int<512>(), Int<8>());
  else if (pieces <= 512 * 9) f(Int<512>(), Int<12>());
  else if (pieces <= 512 * 16) f(Int<512>(), Int<16>());
  else if (pieces <= 12800) f(Int<1024>(), Int<8>());
  else f(Int<1024>(), Int<16>());
}

template <bool BF16>
static void launch_rows(const symi_ctx* ctx, int kid, const PolicyArgs& g, hipStream_t st) {
  const int T = ctx->cfg.T, pieces = cdiv(g.V, Piece<BF16>::N);
#define ROWS(GRAD, THREADS, NV) SYMI_TIMED(ctx, kid, st, (policy_kernel<BF16, GRAD, THREADS, NV><<<T, THREADS, 0, st>>>(g)))
  if (g.dlogits) {
    by_length(pieces, [&](auto threads, auto nv) { ROWS(true, decltype(threads)::value, decltype(nv)::value); });
  } else {
    // Nothing has to stay: eight pieces of 256 threads at a time (8192 of 32000 in bf16 82 us, 512 x 4 84), on few rows 512 threads (300 of
    // 131072: 20.7 against 22.9) or 1024 (16 of 128000: 11.9 against 13.8).  So a row's last bits depend on the batch here.
    if (pieces <= 64 * 4) ROWS(false, 64, 4);
    else if (pieces <= 256 * 4) ROWS(false, 256, 4);
    else if (T <= ctx->cus / 4 && pieces > 8192) ROWS(false, 1024, 8);
    else if (T < 4 * ctx->cus) ROWS(false, 512, 4);
    else ROWS(false, 256, 8);
  }
#undef ROWS
}

// Whether a row's wavefronts are workgroups of their own: while all of them together are at most four for each compute unit and, of rows of
// up to eight wavefronts, a wavefront's pieces of all rows at most 80000 (58000 of fp32 rows of eight), as every logit is read twice.  us with the gradient, one workgroup a
// row : split.  bf16 V = 131072: 16 rows 22.4 : 12.9, 64 25.2 : 20.6, 128 27.5 : 28.9; 65000: 64 rows 17.3 : 15.8, 96 18.0 : 18.4; 50001: 1 row
// 13.3 : 11.1, 64 14.9 : 13.4, 96 15.9 : 15.8, 128 17.1 : 17.5; 32000: 128 rows 13.3 : 12.8, 192 14.5 : 15.6; 16000: 16 rows 10.1 : 8.6, 160
// 10.9 : 10.4, 192 11.0 : 11.3, 256 11.8 : 12.6; 12000: 192 rows 10.3 : 9.8, 256 10.5 : 10.6; 4000: 16 rows 9.0 : 7.3, 256 9.2 : 7.9; fp32 V = 32003:
// 16 rows 11.9 : 11.1, 64 13.7 : 14.0, 96 14.4 : 15.9; 25000: 64 rows 12.3 : 11.8, 96 13.1 : 13.8; 16000: 96 rows 11.0 : 10.4, 128 11.5 : 11.7;
// 8000: 160 rows 10.1 : 9.8, 256 11.1 : 11.8.
static bool wants_parts(const symi_ctx* ctx, int pieces, bool bf16) {
  int waves = 0;
  by_length(pieces, [&](auto threads, auto) { waves = decltype(threads)::value / 64; });
  const int T = ctx->cfg.T;
  const long long each = waves == 8 && !bf16 ? 58000 : 80000;
  return T >= 1 && T <= PART_ROWS_MAX && waves > 1 && T * waves <= 4 * ctx->cus && (waves == PART_MAX || (long long)T * pieces <= waves * each);
}
template <bool BF16>
static void launch_parts(const symi_ctx* ctx, const PolicyArgs& g, const Parts& parts, float* stats, hipStream_t st) {
  const int T = ctx->cfg.T;
  by_length(cdiv(g.V, Piece<BF16>::N), [&](auto threads, auto nv) {
    constexpr int THREADS = decltype(threads)::value, NV = decltype(nv)::value, WAVES = THREADS / 64;
    if constexpr (WAVES > 1) {
      SYMI_TIMED(ctx, K_POLICY, st, (policy_part_kernel<BF16, THREADS, NV><<<T * WAVES, 64, 0, st>>>(g, parts)));
      SYMI_TIMED(ctx, K_POLICY_SUM, st, (policy_apply_kernel<BF16, THREADS, NV><<<T * WAVES + 1, SUM_SPLIT_THREADS, 0, st>>>(g, parts, T, stats)));
    }
  });
}

}  // namespace symi

using namespace symi;

extern "C" size_t symi_policy_workspace_bytes(const symi_cfg* cfg) {
  if (check_cfg(cfg, "symi_policy_workspace_bytes") != SYMI_OK) return 0;
  return policy_ws(cfg).total;
}

extern "C" int symi_token_logp(const symi_ctx* ctx, const symi_policy* hp, const void* logits, int V, int ld,
                               const int32_t* action, const float* weight, float* logp, void* stream) {
  const char* const who = "symi_token_logp";
  SYMI_ENTER(ctx, who);
  if (int rc = check_policy(who, hp, V, ld)) return rc;
  if (cfg->T == 0) return SYMI_OK;
  SYMI_REQUIRE(logits && action && logp, who, "NULL pointer");
  const PolicyArgs g = {logits, V, ld, action, nullptr, nullptr, nullptr, weight, logp, nullptr, nullptr, scalars(hp)};
  if (hp->logits_dtype == SYMI_BF16) launch_rows<true>(ctx, K_TOKEN_LOGP, g, as_stream(stream));
  else launch_rows<false>(ctx, K_TOKEN_LOGP, g, as_stream(stream));
  SYMI_LAUNCH_CHECK(who);
  return SYMI_OK;
}

extern "C" int symi_policy_loss(const symi_ctx* ctx, const symi_policy* hp, const void* logits, int V, int ld,
                                const int32_t* action, const float* logp_old, const float* logp_ref,
                                const float* advantage, const float* weight, float* logp, float* stats, void* dlogits,
                                void* ws, void* stream) {
  const char* const who = "symi_policy_loss";
  SYMI_ENTER(ctx, who);
  if (int rc = check_policy(who, hp, V, ld)) return rc;
  const int T = cfg->T;
  SYMI_REQUIRE(T == 0 || logp_ref || hp->kl_coef == 0.f, who, "kl_coef needs logp_ref");
  SYMI_REQUIRE(stats && ws && (T == 0 || (logits && action && logp_old && advantage && weight && logp)), who, "NULL pointer");
  hipStream_t st = as_stream(stream);
  const PolicyWs L = policy_ws(cfg);
  char* const w = reinterpret_cast<char*>(align_up(reinterpret_cast<size_t>(ws), 256));
  const PolicyArgs g = {logits, V, ld, action, logp_old, logp_ref, advantage, weight, logp, reinterpret_cast<float4*>(w + L.terms), dlogits, scalars(hp)};
  const bool bf16 = hp->logits_dtype == SYMI_BF16;
  if (dlogits && wants_parts(ctx, cdiv(V, bf16 ? 8 : 4), bf16)) {
    const Parts parts = {reinterpret_cast<float2*>(w + L.ms), reinterpret_cast<float*>(w + L.chosen)};
    if (bf16) launch_parts<true>(ctx, g, parts, stats, st);
    else launch_parts<false>(ctx, g, parts, stats, st);
  } else {
    if (T && bf16) launch_rows<true>(ctx, K_POLICY, g, st);
    else if (T) launch_rows<false>(ctx, K_POLICY, g, st);
    SYMI_TIMED(ctx, K_POLICY_SUM, st, (policy_sum_kernel<<<1, SUM_THREADS, 0, st>>>(g.terms, T, stats)));
  }
  SYMI_LAUNCH_CHECK(who);
  return SYMI_OK;
}
