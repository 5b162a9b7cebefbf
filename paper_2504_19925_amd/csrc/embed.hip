// symi_embed_fwd / symi_embed_bwd: the token embedding X[t] = scale * table[tokens[t]] and its gradient
// dTable[v] = scale * sum of dX[t] over the tokens t that are v, in fp32.
//
// The gradient needs the tokens of a row together and in an order that is the same on every run.  One launch sorts: a
// workgroup owns R consecutive rows of the table, reads all tokens, counts the ones below its rows (where its part of
// the sorted order begins) and packs the ones of its own rows in token order; its wavefronts then give each row's tokens
// their places.  Counts are integer sums and places come from ballots, so nothing depends on the order of atomics.
#include <algorithm>
#include <type_traits>

#include "common.h"

namespace symi {

constexpr int EMBED_THREADS = 256;
constexpr int SORT_THREADS = 1024;
constexpr int SORT_WAVES = SORT_THREADS / 64;
constexpr int SORT_ROWS_MAX = 8192;   // rows that one workgroup of the sort counts in LDS
constexpr int SORT_GROUPS = 256;

// A 16-byte piece of a row: 8 bf16 or 4 fp32 values.
template <bool BF16> struct Piece {
  static constexpr int N = BF16 ? 8 : 4;
  using Elem = std::conditional_t<BF16, uint16_t, float>;
  static __device__ __forceinline__ void load(const void* base, long long at, float (&x)[N]) {
    if constexpr (BF16) {
      const u32x4_bf16 q = *reinterpret_cast<const u32x4_bf16*>(static_cast<const uint16_t*>(base) + at);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        x[2 * i] = __uint_as_float(q[i] << 16);
        x[2 * i + 1] = __uint_as_float(q[i] & 0xffff0000u);
      }
    } else {
      const f32x4_f32 q = *reinterpret_cast<const f32x4_f32*>(static_cast<const float*>(base) + at);
#pragma unroll
      for (int i = 0; i < 4; ++i) x[i] = q[i];
    }
  }
  static __device__ __forceinline__ void store(void* base, long long at, const float (&x)[N]) {
    if constexpr (BF16) {
      u32x4_bf16 q;
#pragma unroll
      for (int i = 0; i < 4; ++i) q[i] = pack_bf16x2(x[2 * i], x[2 * i + 1]);
      *reinterpret_cast<u32x4_bf16*>(static_cast<uint16_t*>(base) + at) = q;
    } else {
      f32x4_f32 q;
#pragma unroll
      for (int i = 0; i < 4; ++i) q[i] = x[i];
      *reinterpret_cast<f32x4_f32*>(static_cast<float*>(base) + at) = q;
    }
  }
};

// lanes = 2^lg lanes share a token's row and walk it in pieces.
template <bool BF16>
__global__ __launch_bounds__(EMBED_THREADS) void embed_fwd_kernel(const int32_t* __restrict__ tokens,
                                                                  const void* __restrict__ table, void* __restrict__ X,
                                                                  int T, int V, int d, float scale, int lg) {
  using P = Piece<BF16>;
  const long long t = ((long long)blockIdx.x * EMBED_THREADS + threadIdx.x) >> lg;
  if (t >= T) return;
  const int lane = threadIdx.x & ((1 << lg) - 1), pieces = d / P::N;
  const int v = tokens[t];
  const bool inside = (unsigned)v < (unsigned)V;
  for (int c = lane; c < pieces; c += 1 << lg) {
    float x[P::N];
    if (inside) P::load(table, (long long)v * d + c * P::N, x);
#pragma unroll
    for (int i = 0; i < P::N; ++i) x[i] = inside ? x[i] * scale : 0.f;
    P::store(X, t * d + c * P::N, x);
  }
}

// Workgroup b: rows [b R, b R + R) of the table.  offs [V+1]: where each row's tokens begin in `order` [T], which lists
// the tokens (their places in the batch, ascending) row by row; packed and packed_key are its scratch.
__global__ __launch_bounds__(SORT_THREADS) void embed_sort_kernel(const int32_t* __restrict__ tokens, int T, int V, int R,
                                                                  int32_t* __restrict__ offs, int32_t* __restrict__ order,
                                                                  int32_t* packed, int32_t* packed_key) {
  __shared__ int32_t cursor[SORT_ROWS_MAX];
  __shared__ int32_t wave_less[SORT_WAVES], wave_own[SORT_WAVES], wave_sum[SORT_WAVES];
  constexpr int U = 8;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const long long v0 = (long long)blockIdx.x * R;
  const int rows = (int)(v0 + R < V ? R : V - v0);
  for (int r = threadIdx.x; r < rows; r += SORT_THREADS) cursor[r] = 0;
  // every wavefront reads a stretch of consecutive tokens
  const long long stretch = (((long long)T + SORT_WAVES - 1) / SORT_WAVES + 63) / 64 * 64;
  const long long lo = wave * stretch, hi = lo + stretch < T ? lo + stretch : T;
  const auto row_of = [&](long long i) -> int { return i < hi ? tokens[i] : -1; };
  const auto is_own = [&](int v) { return v >= 0 && (unsigned)v - (unsigned)v0 < (unsigned)rows; };
  int less = 0, own = 0;
  for (long long i = lo + lane; i < hi; i += 64 * U) {
    int v[U];
#pragma unroll
    for (int u = 0; u < U; ++u) v[u] = row_of(i + u * 64);
#pragma unroll
    for (int u = 0; u < U; ++u) {
      less += (unsigned)v[u] < (unsigned)v0;
      own += is_own(v[u]);
    }
  }
#pragma unroll
  for (int m = 32; m >= 1; m >>= 1) {
    less += __shfl_xor(less, m, 64);
    own += __shfl_xor(own, m, 64);
  }
  if (lane == 0) {
    wave_less[wave] = less;
    wave_own[wave] = own;
  }
  __syncthreads();
  int base = 0, count = 0, at = 0;
#pragma unroll
  for (int w = 0; w < SORT_WAVES; ++w) {
    base += wave_less[w];
    at += w < wave ? wave_own[w] : 0;
    count += wave_own[w];
  }
  at += base;
  for (long long i0 = lo; own && i0 < hi; i0 += 64 * U) {   // a wavefront without any skips it
    int v[U];
#pragma unroll
    for (int u = 0; u < U; ++u) v[u] = row_of(i0 + lane + u * 64);
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const bool mine = is_own(v[u]);
      const unsigned long long mask = __ballot(mine);
      if (mine) {
        const int to = at + __popcll(mask & ((1ull << lane) - 1));
        packed[to] = (int)(i0 + lane + u * 64);
        packed_key[to] = v[u] - (int)v0;
        atomicAdd(&cursor[v[u] - (int)v0], 1);
      }
      at += __popcll(mask);
    }
  }
  __syncthreads();
  // counts of the rows -> where their tokens begin
  const int each = (rows + SORT_THREADS - 1) / SORT_THREADS, r0 = threadIdx.x * each;
  int sum = 0;
  for (int r = r0; r < r0 + each && r < rows; ++r) sum += cursor[r];
  int before = sum;
#pragma unroll
  for (int m = 1; m < 64; m <<= 1) {
    const int x = __shfl_up(before, m, 64);
    if (lane >= m) before += x;
  }
  if (lane == 63) wave_sum[wave] = before;
  __syncthreads();
  before += base - sum;
#pragma unroll
  for (int w = 0; w < SORT_WAVES; ++w) before += w < wave ? wave_sum[w] : 0;
  for (int r = r0; r < r0 + each && r < rows; ++r) {
    const int n = cursor[r];
    cursor[r] = before;
    offs[v0 + r] = before;
    before += n;
  }
  if (v0 + rows == V && threadIdx.x == 0) offs[V] = base + count;
  __syncthreads();
  volatile int32_t* const at_row = cursor;   // a row's place is one wavefront's alone
  // wavefront w places the tokens of the rows w, w + 16, ...
  for (int i0 = 0; i0 < count; i0 += 64) {
    const bool there = i0 + lane < count;
    const int r = there ? packed_key[base + i0 + lane] : 0;
    const int t = there ? packed[base + i0 + lane] : 0;
    const bool mine = there && (r & (SORT_WAVES - 1)) == wave;
    unsigned long long left = __ballot(mine);
    while (left) {
      const int row = __builtin_amdgcn_readlane(r, (int)__builtin_ctzll(left));
      const unsigned long long same = __ballot(mine && r == row);
      const int to = at_row[row];
      if (mine && r == row) order[to + __popcll(same & ((1ull << lane) - 1))] = t;
      if (lane == 0) at_row[row] = to + __popcll(same);
      left &= ~same;
    }
  }
}

// A wavefront sums 64 pieces of one row over the row's tokens.
template <bool BF16>
__global__ __launch_bounds__(EMBED_THREADS) void embed_sum_kernel(const void* __restrict__ dX,
                                                                  const int32_t* __restrict__ offs,
                                                                  const int32_t* __restrict__ order, int V, int d,
                                                                  int parts, float scale, int accumulate,
                                                                  float* __restrict__ dTable) {
  using P = Piece<BF16>;
  const long long id = (long long)blockIdx.y * gridDim.x + blockIdx.x;
  const long long unit = id * (EMBED_THREADS / 64) + (threadIdx.x >> 6);
  const long long v = unit / parts;
  const int c = ((int)(unit % parts) * 64 + (threadIdx.x & 63)) * P::N;
  if (v >= V || c >= d) return;
  const int lo = offs[v], hi = offs[v + 1];
  if (lo == hi && accumulate) return;
  float sum[P::N] = {};
  for (int i = lo; i < hi; ++i) {
    float x[P::N];
    P::load(dX, (long long)order[i] * d + c, x);
#pragma unroll
    for (int j = 0; j < P::N; ++j) sum[j] += x[j];
  }
  float* const to = dTable + v * d + c;
#pragma unroll
  for (int h = 0; h < P::N; h += 4) {
    float y[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) y[j] = sum[h + j] * scale;
    if (accumulate) {
      float old[4];
      Piece<false>::load(to, h, old);
#pragma unroll
      for (int j = 0; j < 4; ++j) y[j] += old[j];
    }
    Piece<false>::store(to, h, y);
  }
}

struct EmbedWs {
  size_t offs, order, packed, packed_key, total;
};
static EmbedWs embed_ws(const symi_cfg* c, int V) {
  EmbedWs L;
  size_t off = 0;
  const auto take = [&](size_t bytes) { const size_t at = off; off += align_up(bytes, 256); return at; };
  L.offs = take(((size_t)V + 1) * sizeof(int32_t));
  L.order = take((size_t)c->T * sizeof(int32_t));
  L.packed = take((size_t)c->T * sizeof(int32_t));
  L.packed_key = take((size_t)c->T * sizeof(int32_t));
  L.total = off + 256;
  return L;
}

}  // namespace symi

using namespace symi;

extern "C" size_t symi_embed_workspace_bytes(const symi_cfg* cfg, int V) {
  if (check_cfg(cfg, "symi_embed_workspace_bytes") != SYMI_OK) return 0;
  if (V < 1) {
    set_error("symi_embed_workspace_bytes: V < 1");
    return 0;
  }
  return embed_ws(cfg, V).total;
}

extern "C" int symi_embed_fwd(const symi_ctx* ctx, const int32_t* tokens, const void* table, int V, float scale, void* X,
                              void* stream) {
  const char* const who = "symi_embed_fwd";
  SYMI_ENTER(ctx, who);
  SYMI_REQUIRE(V >= 1, who, "V < 1");
  if (cfg->T == 0) return SYMI_OK;
  SYMI_REQUIRE(tokens && table && X, who, "NULL pointer");
  const bool bf16 = cfg->dtype == SYMI_BF16;
  const int pieces = cfg->d / (bf16 ? 8 : 4);
  int lg = 0;
  while (lg < 8 && (1 << lg) < pieces) ++lg;
  const int grid = cdiv((long long)cfg->T << lg, EMBED_THREADS);
  hipStream_t st = as_stream(stream);
  if (bf16)
    SYMI_TIMED(ctx, K_EMBED_FWD, st, (embed_fwd_kernel<true><<<grid, EMBED_THREADS, 0, st>>>(tokens, table, X, cfg->T, V, cfg->d, scale, lg)));
  else
    SYMI_TIMED(ctx, K_EMBED_FWD, st, (embed_fwd_kernel<false><<<grid, EMBED_THREADS, 0, st>>>(tokens, table, X, cfg->T, V, cfg->d, scale, lg)));
  SYMI_LAUNCH_CHECK(who);
  return SYMI_OK;
}

extern "C" int symi_embed_bwd(const symi_ctx* ctx, const int32_t* tokens, const void* dX, int V, float scale, int accumulate,
                              float* dTable, void* ws, void* stream) {
  const char* const who = "symi_embed_bwd";
  SYMI_ENTER(ctx, who);
  SYMI_REQUIRE(V >= 1, who, "V < 1");
  SYMI_REQUIRE(accumulate == 0 || accumulate == 1, who, "accumulate must be 0 or 1");
  SYMI_REQUIRE(dTable && ws && (cfg->T == 0 || (tokens && dX)), who, "NULL pointer");
  const bool bf16 = cfg->dtype == SYMI_BF16;
  const EmbedWs L = embed_ws(cfg, V);
  char* const w = reinterpret_cast<char*>(align_up(reinterpret_cast<size_t>(ws), 256));
  const auto ints = [&](size_t at) { return reinterpret_cast<int32_t*>(w + at); };
  const int R = std::min(std::max(cdiv(V, SORT_GROUPS), 1), SORT_ROWS_MAX);
  hipStream_t st = as_stream(stream);
  SYMI_TIMED(ctx, K_EMBED_SORT, st, (embed_sort_kernel<<<cdiv(V, R), SORT_THREADS, 0, st>>>(
      tokens, cfg->T, V, R, ints(L.offs), ints(L.order), ints(L.packed), ints(L.packed_key))));
  const int parts = cdiv(cfg->d, 64 * (bf16 ? 8 : 4));
  const long long groups = ((long long)V * parts + 3) / 4;
  // workgroups over two dimensions: the threads of one end at 2^32
  const dim3 grid((unsigned)std::min(groups, 1LL << 20), (unsigned)((groups + (1LL << 20) - 1) >> 20));
  if (bf16)
    SYMI_TIMED(ctx, K_EMBED_SUM, st, (embed_sum_kernel<true><<<grid, EMBED_THREADS, 0, st>>>(
        dX, ints(L.offs), ints(L.order), V, cfg->d, parts, scale, accumulate, dTable)));
  else
    SYMI_TIMED(ctx, K_EMBED_SUM, st, (embed_sum_kernel<false><<<grid, EMBED_THREADS, 0, st>>>(
        dX, ints(L.offs), ints(L.order), V, cfg->d, parts, scale, accumulate, dTable)));
  SYMI_LAUNCH_CHECK(who);
  return SYMI_OK;
}
