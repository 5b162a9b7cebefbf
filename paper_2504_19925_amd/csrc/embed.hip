// symi_embed_fwd / symi_embed_bwd: the token embedding X[t] = scale * table[tokens[t]] and its gradient
// dTable[v] = scale * sum of dX[t] over the tokens t that are v, in fp32.
//
// The gradient needs the tokens of a row together and in an order that is the same on every run.  One launch sorts: the
// rows of the table are dealt out to workgroups like cards (the most frequent tokens are neighbours in many vocabularies),
// and each workgroup reads all tokens: it counts the ones of the workgroups before it, where its part of the sorted order
// begins, keeps its own ones in LDS and counts them by row and wavefront, then gives every one its place.  Counts are integer sums and places come from
// ballots, so nothing depends on the order of the additions in LDS.
#include <algorithm>
#include <type_traits>

#include "common.h"

namespace symi {

constexpr int EMBED_THREADS = 256;
constexpr int SORT_ROWS_MAX = 1024;   // rows that one workgroup of the sort counts in LDS, for each wavefront
constexpr int SORT_GROUPS = 256;      // workgroups, unless the rows are more

// A 16-byte piece of a row: 8 bf16 or 4 fp32 values.
template <bool BF16> struct Piece {
  static constexpr int N = BF16 ? 8 : 4;
  using Elem = std::conditional_t<BF16, uint16_t, float>;
  using Raw = std::conditional_t<BF16, u32x4_bf16, f32x4_f32>;
  static __device__ __forceinline__ Raw load(const void* base, long long at) {
    return *reinterpret_cast<const Raw*>(static_cast<const Elem*>(base) + at);
  }
  static __device__ __forceinline__ void unpack(Raw q, float (&x)[N]) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if constexpr (BF16) {
        x[2 * i] = __uint_as_float(q[i] << 16);
        x[2 * i + 1] = __uint_as_float(q[i] & 0xffff0000u);
      } else {
        x[i] = q[i];
      }
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

// 2^lg lanes share a token's row and walk it in pieces, R rows at a time.  Bound by memory: 65536 rows of d = 4096 in bf16, 5 %
// padding, from a table of 131072 rows: 148 us, 0.34 GB fetched and 0.54 written (5.9 TB/s).
template <bool BF16, int R>
__global__ __launch_bounds__(EMBED_THREADS) void embed_fwd_kernel(const int32_t* __restrict__ tokens,
                                                                  const void* __restrict__ table, void* __restrict__ X,
                                                                  int T, int V, int d, float scale, int lg) {
  using P = Piece<BF16>;
  const long long t0 = (((long long)blockIdx.x * EMBED_THREADS + threadIdx.x) >> lg) * R;
  if (t0 >= T) return;
  const int lane = threadIdx.x & ((1 << lg) - 1), pieces = d / P::N;
  int v[R];
#pragma unroll
  for (int r = 0; r < R; ++r) v[r] = t0 + r < T ? tokens[t0 + r] : -1;
  for (int c = lane; c < pieces; c += 1 << lg) {
    typename P::Raw x[R];
#pragma unroll
    for (int r = 0; r < R; ++r)
      if ((unsigned)v[r] < (unsigned)V) x[r] = P::load(table, (long long)v[r] * d + c * P::N);
#pragma unroll
    for (int r = 0; r < R; ++r) {
      if (R > 1 && t0 + r >= T) continue;
      const bool inside = (unsigned)v[r] < (unsigned)V;
      float y[P::N];
      P::unpack(x[r], y);
#pragma unroll
      for (int i = 0; i < P::N; ++i) y[i] = inside ? y[i] * scale : 0.f;
      P::store(X, (t0 + r) * d + c * P::N, y);
    }
  }
}

// Workgroup b of 2^lg: the rows v with v mod 2^lg = b.  span [V]: where each row's tokens begin and end in `order`, which lists
// the tokens (their places in the batch) row by row, in the order of the wavefronts; rows_of: the rows of the same list; total: its length.
// Bound by the instructions that look at a token, in every workgroup: 65536 tokens 21 us (vector units busy 58 %), 8192 7 us,
// most of it the latency of the launch and of three dependent loads.
constexpr int SORT_KEEP = 1408;       // own tokens that a wavefront keeps from the first reading; with more it reads again
constexpr int SORT_KEEP_T = 1 << 22;  // in batches of at most this many: place in the batch and place among the own rows in 32 bits
template <int WAVES, int U>
__global__ __launch_bounds__(WAVES * 64) void embed_sort_kernel(const int32_t* __restrict__ tokens, int T, int V, int lg,
                                                                int2* __restrict__ span, int32_t* __restrict__ order,
                                                                int32_t* __restrict__ rows_of, int32_t* __restrict__ total) {
  extern __shared__ int32_t count[];   // [WAVES, rows]: of a wavefront's tokens, then the place of its next one
  __shared__ int32_t wave_less[WAVES], wave_sum[WAVES];
  __shared__ uint32_t kept[WAVES][SORT_KEEP];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const unsigned b = blockIdx.x, low = (1u << lg) - 1;
  const int rows = (int)(((unsigned)V + low - b) >> lg);
  for (int i = threadIdx.x; i < WAVES * rows; i += WAVES * 64) count[i] = 0;
  __syncthreads();
  int32_t* const mine = count + wave * rows;
  // a wavefront reads every WAVES-th 64 U tokens
  constexpr int AHEAD = WAVES * 64 * U;
  const int lo = wave * 64 * U, hi = T;
  // 64 U tokens from i0 on; padding becomes 2^32 - 1
  const auto fetch = [&](long long i0, unsigned (&v)[U]) {
    const int32_t* const from = tokens + i0;
    if (i0 + 64 * U <= hi) {
#pragma unroll
      for (int u = 0; u < U; ++u) v[u] = (unsigned)from[u * 64 + lane];
    } else {
#pragma unroll
      for (int u = 0; u < U; ++u) v[u] = u * 64 + lane < hi - i0 ? (unsigned)from[u * 64 + lane] : 0xffffffffu;
    }
  };
  const int keep = T <= SORT_KEEP_T ? SORT_KEEP : 0;
  int less = 0, own = 0;
  unsigned v[U], ahead[U];
  if (lo < hi) fetch(lo, ahead);
  for (long long i0 = lo; i0 < hi; i0 += AHEAD) {
#pragma unroll
    for (int u = 0; u < U; ++u) v[u] = ahead[u] < (unsigned)V ? ahead[u] : 0xffffffffu;
    if (i0 + AHEAD < hi) fetch(i0 + AHEAD, ahead);
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const unsigned w = v[u] & low;   // of padding: the last workgroup's, but no row of it
      less += w < b;
      const bool is_own = w == b && v[u] != 0xffffffffu;
      const unsigned long long mask = __ballot(is_own);
      if (!mask) continue;
      const int to = own + __popcll(mask & ((1ull << lane) - 1));
      if (is_own) {
        if (to < keep) kept[wave][to] = ((unsigned)i0 + u * 64 + lane) << 10 | v[u] >> lg;
        else atomicAdd(&mine[v[u] >> lg], 1);
      }
      own += __popcll(mask);
    }
  }
  for (int k = 0; k < min(own, keep); k += 64) {   // the first one's equals at once: a frequent row's would wait for each other
    const bool there = k + lane < min(own, keep);
    const uint32_t r = kept[wave][min(k + lane, SORT_KEEP - 1)] & 1023u, first = (uint32_t)__builtin_amdgcn_readfirstlane((int)r);
    const unsigned long long same = __ballot(there && r == first);
    if (there && (r != first || lane == 0)) atomicAdd(&mine[r], lane == 0 ? (int)__popcll(same) : 1);
  }
#pragma unroll
  for (int m = 32; m >= 1; m >>= 1) less += __shfl_xor(less, m, 64);
  if (lane == 0) wave_less[wave] = less;
  __syncthreads();
  // counts -> where the tokens of a row and wavefront begin
  const int each = (rows + WAVES * 64 - 1) / (WAVES * 64), r0 = threadIdx.x * each;
  int sum = 0;
  for (int r = r0; r < r0 + each && r < rows; ++r)
#pragma unroll
    for (int w = 0; w < WAVES; ++w) sum += count[w * rows + r];
  int at = sum;
#pragma unroll
  for (int m = 1; m < 64; m <<= 1) {
    const int x = __shfl_up(at, m, 64);
    if (lane >= m) at += x;
  }
  if (lane == 63) wave_sum[wave] = at;
  __syncthreads();
  at -= sum;
#pragma unroll
  for (int w = 0; w < WAVES; ++w) at += wave_less[w] + (w < wave ? wave_sum[w] : 0);
  for (int r = r0; r < r0 + each && r < rows; ++r) {
    const int begin = at;
#pragma unroll
    for (int w = 0; w < WAVES; ++w) {
      const int n = count[w * rows + r];
      count[w * rows + r] = at;
      at += n;
    }
    span[((long long)r << lg) + b] = int2{begin, at};
  }
  if (b == low && threadIdx.x == WAVES * 64 - 1) *total = at;
  __syncthreads();
  volatile int32_t* const next = mine;
  // 64 tokens, the workgroup's own among them: equal ones take consecutive places
  const auto place = [&](bool is_own, unsigned v, int i) {
    int rank = 0;          // among the equal ones
    bool final = false;    // the last of them
    for (unsigned long long left = __ballot(is_own); left;) {
      const unsigned row = (unsigned)__builtin_amdgcn_readlane((int)v, (int)__builtin_ctzll(left));
      const unsigned long long same = __ballot(is_own && v == row);
      if (is_own && v == row) {
        rank = __popcll(same & ((1ull << lane) - 1));
        final = same >> lane == 1;
      }
      left &= ~same;
    }
    if (!is_own) return;
    const int p = next[v >> lg] + rank;
    order[p] = i;
    rows_of[p] = (int)v;
    if (final) next[v >> lg] = p + 1;
  };
  if (own <= keep) {
    for (int k = 0; k < own; k += 64) {
      const uint32_t x = kept[wave][min(k + lane, SORT_KEEP - 1)];
      place(k + lane < own, (x & 1023u) << lg | b, (int)(x >> 10));
    }
    return;
  }
  for (long long i0 = lo; i0 < hi; i0 += AHEAD) {
    fetch(i0, v);
#pragma unroll
    for (int u = 0; u < U; ++u) place((v[u] & low) == b && v[u] < (unsigned)V, v[u], (int)i0 + u * 64 + lane);
  }
}

// Sums: the sorted tokens are cut into chunks of C, whatever their rows, so that a row that half the batch chose is as much
// parallel work as any other.  A wavefront takes 64 pieces of the rows of a chunk: all tokens of the runs (equal rows) that begin in
// it.  Only a run of more than 2 C tokens across a multiple of its share is split, at those multiples: its parts go to `partial`
// [blocks of SHARE, 2, d], by the block in which they begin: in slot 1 where the run begins, else in slot 0.  embed_join
// adds them up in order.
// Sums and joins, us, with 16 : 32 : 64 tokens a share: 42750 tokens of d = 48 17 : 21 : 32, 19626 of 408, a third of them one row, 18 : 24 :
// 36, 8192 of 1024 19 : 24 : 36, 65536 of 1024, a quarter one row, 74 : 83 : 131, 65536 of 4096 348 : 347 : 375.
constexpr int SHARE = 16;          // a multiple of every C
constexpr int SHARES_MAX = 1024;   // of a run, as one workgroup adds them up: longer runs have larger shares
__device__ __forceinline__ int share_of(int2 run) {
  int S = SHARE;
  while (run.y - run.x > SHARES_MAX * S) S *= 2;
  return S;
}
__device__ __forceinline__ bool is_split(int2 run, int C, int S) { return run.y - run.x > 2 * C && run.x / S != (run.y - 1) / S; }
constexpr int SUM_ROWS = 8;   // rows that a wavefront has in flight

__device__ __forceinline__ void put_row(float* to, const float* x, float scale) {
  f32x4_f32 y;
#pragma unroll
  for (int j = 0; j < 4; ++j) y[j] = x[j] * scale;
  *reinterpret_cast<f32x4_f32*>(to) = y;
}
__device__ __forceinline__ void put_row(float* to, const float* x, float scale, f32x4_f32 old) {
#pragma unroll
  for (int j = 0; j < 4; ++j) old[j] = x[j] * scale + old[j];
  *reinterpret_cast<f32x4_f32*>(to) = old;
}

// Zeros to rows without tokens: FILL_PIECES pieces of four values from `first` on, below `all`.
constexpr int FILL_PIECES = 2048;
template <int THREADS>
__device__ __forceinline__ void fill_rows(const int2* __restrict__ span, long long first, long long all, int d, float* __restrict__ dTable) {
  const int per = d / 4;
  const long long v = first / per;
  const int begin = (int)(first - v * per);
#pragma unroll
  for (int k = 0; k < FILL_PIECES / THREADS; ++k) {
    const int i = k * THREADS + threadIdx.x;
    if (first + i >= all) return;
    const int2 s = span[v + (begin + i) / per];
    if (s.x == s.y) *reinterpret_cast<f32x4_f32*>(dTable + (first + i) * 4) = f32x4_f32{0.f, 0.f, 0.f, 0.f};
  }
}

// Bound by memory: 65536 tokens of d = 4096 in bf16 and a table of 65536 rows in 300 us, 0.55 GB fetched and 0.98 written
// (5.1 TB/s); 8192 of d = 1024, added to the table, 12 us, three loads one after another and the store.
template <bool BF16, bool ADD>
__global__ __launch_bounds__(EMBED_THREADS) void embed_sum_kernel(
    const void* __restrict__ dX, const int2* __restrict__ span, const int32_t* __restrict__ order,
    const int32_t* __restrict__ rows_of, const int32_t* __restrict__ total_of, int size, int d, int parts, int C, int units, float scale,
    float* __restrict__ dTable, float* __restrict__ partial, long long sum_groups, long long fill_to) {
  using P = Piece<BF16>;
  constexpr int N = P::N;
  const int lane = threadIdx.x & 63;
  const long long group = (long long)blockIdx.y * gridDim.x + blockIdx.x;
  if (group >= sum_groups) {
    fill_rows<EMBED_THREADS>(span, (group - sum_groups) * FILL_PIECES, fill_to, d, dTable);
    return;
  }
  const int unit = __builtin_amdgcn_readfirstlane((int)(group * (EMBED_THREADS / 64)) + (threadIdx.x >> 6));
  const int total = *total_of, chunk = unit / parts, lo = chunk * C;
  // the places around the chunk's, requested before anything about them is known (there are `size` of them)
  int row = rows_of[min(lo + lane, size - 1)], token = order[min(lo + lane, size - 1)];
  int begin = lo, end = min(lo + C, total);
  if (unit >= units || begin >= end) return;
  const int c = ((unit % parts) * 64 + lane) * N;
  const bool live = c < d;
  // places below head_end are a share of a run that began before, those from tail_begin on one of a run that goes on behind
  int head_end = lo, tail_begin = 0x7fffffff;
  {
    const int2 a = span[__builtin_amdgcn_readlane(row, 0)], z = span[__builtin_amdgcn_readlane(row, end - 1 - lo)];
    if (z.x >= lo && z.y > end) {
      const int S = share_of(z);
      if (is_split(z, C, S)) {
        end = (z.x / S + 1) * S;
        tail_begin = z.x;
      } else {
        end = z.y;
      }
    }
    if (a.x < lo) {
      const int S = share_of(a);
      if (lo % S == 0 && is_split(a, C, S)) {
        head_end = min(a.y, lo + S);
        end = max(end, head_end);
      } else {
        begin = a.y;
      }
    }
    if (begin >= end) return;
  }
  float sum[N] = {};
  for (int w0 = lo; w0 < end; w0 += 64) {   // lane i holds place w0 + i
    const int n = min(64, end - w0);
    if (w0 > lo) {
      row = rows_of[min(w0 + lane, size - 1)];
      token = order[min(w0 + lane, size - 1)];
    }
    // a run ends where the next token's row is another
    const int next = __shfl_down(row, 1, 64);
    const bool last = lane < n && (w0 + lane + 1 == end || (lane == 63 ? rows_of[w0 + 64] : next) != row);
    const unsigned long long ends = __ballot(last);
    for (int i0 = max(begin - w0, 0); i0 < n; i0 += SUM_ROWS) {
      typename P::Raw x[SUM_ROWS];
      f32x4_f32 old[SUM_ROWS][N / 4];
#pragma unroll
      for (int u = 0; u < SUM_ROWS; ++u) {
        const int i = i0 + u;
        if (i >= n) continue;
        if (live) x[u] = P::load(dX, (long long)__builtin_amdgcn_readlane(token, i) * d + c);
        if (ADD && live && (ends >> i & 1) && w0 + i >= head_end && w0 + i < tail_begin)
#pragma unroll
          for (int h = 0; h < N / 4; ++h)
            old[u][h] = *reinterpret_cast<const f32x4_f32*>(dTable + (long long)__builtin_amdgcn_readlane(row, i) * d + c + 4 * h);
      }
#pragma unroll
      for (int u = 0; u < SUM_ROWS; ++u) {
        const int i = i0 + u;
        if (i >= n) continue;
        float y[N];
        P::unpack(x[u], y);
#pragma unroll
        for (int j = 0; j < N; ++j) sum[j] += y[j];
        if (!(ends >> i & 1)) continue;
        if (live && w0 + i >= head_end && w0 + i < tail_begin) {
          float* const to = dTable + (long long)__builtin_amdgcn_readlane(row, i) * d + c;
#pragma unroll
          for (int h = 0; h < N / 4; ++h) {
            if (ADD) put_row(to + 4 * h, sum + 4 * h, scale, old[u][h]);
            else put_row(to + 4 * h, sum + 4 * h, scale);
          }
        } else if (live) {
          const bool tail = w0 + i >= head_end;
          float* const to = partial + ((long long)((tail ? tail_begin : lo) / SHARE) * 2 + tail) * d + c;
#pragma unroll
          for (int h = 0; h < N / 4; ++h) put_row(to + 4 * h, sum + 4 * h, 1.f);
        }
#pragma unroll
        for (int j = 0; j < N; ++j) sum[j] = 0.f;
      }
    }
  }
}

// Runs of more than JOIN_LONG shares: a workgroup takes 256 columns of those that begin in one of LONG_BLOCKS blocks, its wavefronts
// a part of the shares each.  The others: a wavefront takes 256 columns of those that begin in one of JOIN_BLOCKS blocks.  The workgroups
// behind those fill rows (between them instead they took as long).  Bound by latency, four loads one after another.  Joins of 8192
// tokens of d = 1024, 65536 of 4096 and 30000 of 2048 in fp32, 300 rows, all in workgroups of eight blocks : so, us: 9.1 : 8.0,
// 31 : 20, 16 : 9.6; with JOIN_BLOCKS 8 8.9, 21, 9.7, with 1 8, 25, 11.8.  Of the 65536 into 65536 rows, with the zeros beside them: 41 us,
// 0.04 GB fetched and 0.13 written.
constexpr int JOIN_WAVES = 8, JOIN_ROWS = 8, JOIN_BLOCKS = 4, JOIN_LONG = 16, LONG_BLOCKS = 64;
template <bool ADD>
__global__ __launch_bounds__(JOIN_WAVES * 64) void embed_join_kernel(const int2* __restrict__ span, const int32_t* __restrict__ rows_of,
                                                                     const int32_t* __restrict__ total_of, const float* __restrict__ partial,
                                                                     int size, int d, int C, int long_groups, int join_groups, int columns,
                                                                     long long fill_from, long long fill_to, float scale,
                                                                     float* __restrict__ dTable) {
  __shared__ float4 share[JOIN_WAVES][64];
  const long long group = (long long)blockIdx.y * gridDim.x + blockIdx.x;
  if (group >= join_groups) {
    fill_rows<JOIN_WAVES * 64>(span, fill_from + (group - join_groups) * FILL_PIECES, fill_to, d, dTable);
    return;
  }
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const bool is_long = group < long_groups;
  const int unit = is_long ? (int)group : ((int)group - long_groups) * JOIN_WAVES + wave;
  const int blocks = is_long ? LONG_BLOCKS : JOIN_BLOCKS, column = unit % columns;
  const int total = *total_of;
  // the run across the end of a block
  const long long hi = ((long long)(unit / columns) * blocks + lane + 1) * SHARE;
  const int row_of = rows_of[min(hi, (long long)size) - 1];   // beyond the total: anything
  const bool there = lane < blocks && hi < total;
  const int2 s = there ? span[row_of] : int2{0, 0};
  const int S_of = share_of(s), count_of = (s.y - 1) / S_of - s.x / S_of + 1;
  unsigned long long todo = __ballot(there && s.y > hi && s.x >= hi - SHARE && is_split(s, C, S_of) && (count_of > JOIN_LONG) == is_long);
  const int c = (column * 64 + lane) * 4;
  const bool live = c < d;
  for (; todo; todo &= todo - 1) {
    const int i = (int)__builtin_ctzll(todo), row = __builtin_amdgcn_readlane(row_of, i);
    // shares: slot 1 of this block, slot 0 of the blocks at the multiples of S behind it
    const int start = __builtin_amdgcn_readlane(s.x, i), S = __builtin_amdgcn_readlane(S_of, i), count = __builtin_amdgcn_readlane(count_of, i);
    const auto block_of = [&](int k) { return (k == 0 ? start : (start / S + k) * S) / SHARE; };
    const int each = is_long ? (count + JOIN_WAVES - 1) / JOIN_WAVES : count, begin = is_long ? wave * each : 0, end = min(begin + each, count);
    float* const to = dTable + (long long)row * d + c;
    f32x4_f32 old = {0.f, 0.f, 0.f, 0.f};
    if (ADD && live && begin == 0) old = *reinterpret_cast<const f32x4_f32*>(to);
    float4 sum = {0.f, 0.f, 0.f, 0.f};
    for (int k0 = begin; k0 < end && live; k0 += JOIN_ROWS) {
      float4 x[JOIN_ROWS];
#pragma unroll
      for (int u = 0; u < JOIN_ROWS; ++u)
        if (k0 + u < end) x[u] = *reinterpret_cast<const float4*>(partial + ((long long)block_of(k0 + u) * 2 + (k0 + u == 0)) * d + c);
#pragma unroll
      for (int u = 0; u < JOIN_ROWS; ++u)
        if (k0 + u < end) { sum.x += x[u].x; sum.y += x[u].y; sum.z += x[u].z; sum.w += x[u].w; }
    }
    float y[4] = {sum.x, sum.y, sum.z, sum.w};
    if (is_long) {
      share[wave][lane] = sum;
      __syncthreads();
#pragma unroll
      for (int w = 1; w < JOIN_WAVES; ++w) {
        const float4 o = share[w][lane];
        y[0] += o.x; y[1] += o.y; y[2] += o.z; y[3] += o.w;
      }
      __syncthreads();
    }
    if (live && begin == 0) {
      if (ADD) put_row(to, y, scale, old);
      else put_row(to, y, scale);
    }
  }
}

// Small batches, in one launch without a sort: a workgroup takes 64 pieces of one token's row.  It reads all tokens and does
// the work of the row if its token is the first of it: every wavefront sums the row's tokens of its part of the batch.  The
// workgroups behind those look which of their rows of the table the batch has and write zeros to the others.  Bound by latency:
// 1024 tokens of d = 128 in fp32 and 8000 rows (4.6 MB) 5.2 us.
constexpr int FEW_MAX = 2048;   // tokens
template <bool BF16, bool ADD, int WAVES, int STEPS>
__global__ __launch_bounds__(WAVES * 64) void embed_few_kernel(const int32_t* __restrict__ tokens, const void* __restrict__ dX, int T,
                                                                  int V, int d, int parts, float scale, float* __restrict__ dTable) {
  using P = Piece<BF16>;
  constexpr int N = P::N, THREADS = WAVES * 64;
  __shared__ float share[WAVES][64 * N];
  __shared__ int32_t has[1024 / 2 + 2];   // rows that 1024 pieces of four values touch, at least two pieces each
  __shared__ int32_t earlier;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const long long group = (long long)blockIdx.y * gridDim.x + blockIdx.x;
  if (group >= (long long)T * parts) {
    const long long first = (group - (long long)T * parts) * 1024, all = (long long)V * (d / 4);
    if (first >= all) return;
    const int per = d / 4;
    const long long v0 = first / per;
    const int begin = (int)(first - v0 * per), rows = (begin + 1023) / per + 1;
    for (int r = tid; r < rows; r += THREADS) has[r] = 0;
    __syncthreads();
    for (int t = tid; t < T; t += THREADS) {
      const long long r = tokens[t] - v0;
      if (r >= 0 && r < rows) has[r] = 1;
    }
    __syncthreads();
#pragma unroll
    for (int k = 0; k < 1024 / THREADS; ++k) {
      const int i = k * THREADS + tid;
      if (first + i < all && !has[(begin + i) / per]) *reinterpret_cast<f32x4_f32*>(dTable + (first + i) * 4) = f32x4_f32{0.f, 0.f, 0.f, 0.f};
    }
    return;
  }
  const int t0 = (int)(group / parts), c = ((int)(group % parts) * 64 + lane) * N;
  const int row = tokens[t0];
  if ((unsigned)row >= (unsigned)V) return;
  const bool live = c < d;
  if (tid == 0) earlier = 0;
  // a wavefront's part of the batch: STEPS times 64 tokens
  unsigned long long same[STEPS];
  bool before = false;
#pragma unroll
  for (int k = 0; k < STEPS; ++k) {
    const int t = (wave * STEPS + k) * 64 + lane;
    const bool is = t < T && tokens[t] == row;
    same[k] = __ballot(is);
    before |= is && t < t0;
  }
  __syncthreads();
  if (before) earlier = 1;
  __syncthreads();
  if (earlier) return;
  f32x4_f32 old[N / 4];
  float* const to = dTable + (long long)row * d + c;
  if (ADD && wave == 0 && live)
#pragma unroll
    for (int h = 0; h < N / 4; ++h) old[h] = *reinterpret_cast<const f32x4_f32*>(to + 4 * h);
  float sum[N] = {};
#pragma unroll
  for (int k = 0; k < STEPS; ++k) {
    unsigned long long left = same[k];
    while (left) {
      typename P::Raw x[SUM_ROWS];
      unsigned long long now = left;
#pragma unroll
      for (int u = 0; u < SUM_ROWS; ++u) {
        if (!now) continue;
        if (live) x[u] = P::load(dX, (long long)((wave * STEPS + k) * 64 + (int)__builtin_ctzll(now)) * d + c);
        now &= now - 1;
      }
#pragma unroll
      for (int u = 0; u < SUM_ROWS; ++u) {
        if (!left) continue;
        float y[N];
        P::unpack(x[u], y);
#pragma unroll
        for (int j = 0; j < N; ++j) sum[j] += y[j];
        left &= left - 1;
      }
    }
  }
#pragma unroll
  for (int j = 0; j < N; ++j) share[wave][j * 64 + lane] = sum[j];
  __syncthreads();
  if (wave != 0 || !live) return;
#pragma unroll
  for (int w = 1; w < WAVES; ++w)
#pragma unroll
    for (int j = 0; j < N; ++j) sum[j] += share[w][j * 64 + lane];
#pragma unroll
  for (int h = 0; h < N / 4; ++h) {
    if (ADD) put_row(to + 4 * h, sum + 4 * h, scale, old[h]);
    else put_row(to + 4 * h, sum + 4 * h, scale);
  }
}

// Tokens of a chunk: few while the chip has room for their wavefronts, more where the look-ups in front of the sums would count.
static int embed_chunk(const symi_cfg* c, int parts) {
  int C = 4;
  while (C < SHARE && (long long)c->T * parts > 16384LL * C) C *= 2;
  return C;
}

struct EmbedWs {
  size_t span, order, rows_of, count, partial, total;
  int parts, chunk, chunks;   // wavefronts across a row of dX; tokens of a chunk; chunks
};
static EmbedWs embed_ws(const symi_cfg* c, int V) {
  EmbedWs L;
  size_t off = 0;
  const auto take = [&](size_t bytes) { const size_t at = off; off += align_up(bytes, 256); return at; };
  L.span = take((size_t)V * sizeof(int2));
  L.order = take((size_t)c->T * sizeof(int32_t));
  L.rows_of = take((size_t)c->T * sizeof(int32_t));
  L.count = take(sizeof(int32_t));
  L.parts = cdiv(c->d, 64 * (c->dtype == SYMI_BF16 ? 8 : 4));
  L.chunk = embed_chunk(c, L.parts);
  L.chunks = cdiv(c->T, L.chunk);
  L.partial = take(((size_t)c->T / SHARE + 1) * 2 * c->d * sizeof(float));
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
  hipStream_t st = as_stream(stream);
  // Two rows at a time where every unit still has four workgroups: 65536 rows of d = 4096, bf16 157 -> 149 us (1.07 GB, 0.7 of them
  // distinct), 30000 of d = 1000, fp32 47 -> 36; four rows 152 and 38, eight 154 and 39.
  const bool many = cfg->T >= 8 * ctx->cus * (EMBED_THREADS >> lg);
#define FWD(BF16, R)                                                                                                       \
  SYMI_TIMED(ctx, K_EMBED_FWD, st, (embed_fwd_kernel<BF16, R><<<cdiv((long long)cdiv(cfg->T, R) << lg, EMBED_THREADS), EMBED_THREADS, 0, st>>>( \
      tokens, table, X, cfg->T, V, cfg->d, scale, lg)))
  if (bf16 && many) FWD(true, 2);
  else if (bf16) FWD(true, 1);
  else if (many) FWD(false, 2);
  else FWD(false, 1);
#undef FWD
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
  int2* const span = reinterpret_cast<int2*>(w + L.span);
  hipStream_t st = as_stream(stream);
  // workgroups over two dimensions: the threads of one end at 2^32
  const auto grid_of = [](long long groups) { return dim3((unsigned)std::min(groups, 1LL << 20), (unsigned)((groups + (1LL << 20) - 1) >> 20)); };
  // us on rows of d = 128 (one part), 1024 (two) and 4096 (eight), sorted : not.  512 tokens of d = 1024: 13 : 4; 1024 tokens 14 : 5.5,
  // 15 : 7.3, 19 : 24; 2048: 15 : 7.3, 17 : 12.5, 24 : 44; 3000: 16 : 11, 19 : 23, 28 : 77; 4096: 15.5 : 14.5, 19 : 30, 33 : 105.  With one
  // part the line would lie at 4000 tokens; it is where embed_few_kernel's eight wavefronts of 4 x 64 tokens end.  All 2048 tokens the same:
  // 20 : 35; what the tokens are is not known here.
  if (cfg->T <= 64 || (cfg->T <= FEW_MAX && (long long)cfg->T * L.parts <= 4096)) {
    const long long groups = (long long)cfg->T * L.parts + (accumulate ? 0 : ((long long)V * (cfg->d / 4) + 1023) / 1024);
    if (groups == 0) return SYMI_OK;
#define FEW_(BF16, ADD, WAVES, STEPS)                                                                                   \
  SYMI_TIMED(ctx, K_EMBED_SUM, st, (embed_few_kernel<BF16, ADD, WAVES, STEPS><<<grid_of(groups), WAVES * 64, 0, st>>>(  \
      tokens, dX, cfg->T, V, cfg->d, L.parts, scale, dTable)))
#define FEW(BF16, ADD) do { if (cfg->T <= 512) FEW_(BF16, ADD, 4, 2); else FEW_(BF16, ADD, 8, 4); } while (0)
    if (bf16 && accumulate) FEW(true, true);
    else if (bf16) FEW(true, false);
    else if (accumulate) FEW(false, true);
    else FEW(false, false);
#undef FEW
#undef FEW_
    SYMI_LAUNCH_CHECK(who);
    return SYMI_OK;
  }
  int lg = 0;
  while ((1LL << lg) < V && ((1 << lg) < SORT_GROUPS || cdiv(V, 1 << lg) > SORT_ROWS_MAX)) ++lg;
  const int rows = cdiv(V, 1 << lg);
#define SORT(WAVES, U)                                                                                                     \
  SYMI_TIMED(ctx, K_EMBED_SORT, st, (embed_sort_kernel<WAVES, U><<<1 << lg, WAVES * 64, WAVES * rows * sizeof(int32_t), st>>>( \
      tokens, cfg->T, V, lg, span, ints(L.order), ints(L.rows_of), ints(L.count))))
  if (cfg->T <= 4 * 64 * 8) SORT(4, 8);
  else SORT(16, 8);
#undef SORT
  float* const partial = reinterpret_cast<float*>(w + L.partial);
  const int units = L.chunks * L.parts;
  const long long sum_groups = (units + 3) / 4;
  // Rows without tokens get their zeros behind the sums (together they run at the rate of a copy; one after the other the
  // sums alone took 225 us and the zeros 145, in one launch 330), the last eighth of the table beside the joins, which are few
  // and wait for memory: c5's took 20 us by themselves.
  const long long pieces = accumulate ? 0 : (long long)V * (cfg->d / 4), fill_sum = pieces - pieces / 8;
  const auto fills = [](long long n) { return (n + FILL_PIECES - 1) / FILL_PIECES; };
  const dim3 grid = grid_of(sum_groups + fills(fill_sum));
#define SUM(BF16, ADD)                                                                                                      \
  SYMI_TIMED(ctx, K_EMBED_SUM, st, (embed_sum_kernel<BF16, ADD><<<grid, EMBED_THREADS, 0, st>>>(                            \
      dX, span, ints(L.order), ints(L.rows_of), ints(L.count), cfg->T, cfg->d, L.parts, L.chunk, units, scale, dTable, partial, sum_groups, fill_sum)))
  if (bf16 && accumulate) SUM(true, true);
  else if (bf16) SUM(true, false);
  else if (accumulate) SUM(false, true);
  else SUM(false, false);
#undef SUM
  {
    const int columns = cdiv(cfg->d, 256), long_groups = cdiv(cfg->T, SHARE * LONG_BLOCKS) * columns;
    const int join_groups = long_groups + cdiv((long long)cdiv(cfg->T, SHARE * JOIN_BLOCKS) * columns, JOIN_WAVES);
    const dim3 grid = grid_of(join_groups + fills(pieces - fill_sum));
#define JOIN(ADD)                                                                                         \
  SYMI_TIMED(ctx, K_EMBED_JOIN, st, (embed_join_kernel<ADD><<<grid, JOIN_WAVES * 64, 0, st>>>(            \
      span, ints(L.rows_of), ints(L.count), partial, cfg->T, cfg->d, L.chunk, long_groups, join_groups, columns, fill_sum, pieces, scale, dTable)))
    if (accumulate) JOIN(true);
    else JOIN(false);
#undef JOIN
  }
  SYMI_LAUNCH_CHECK(who);
  return SYMI_OK;
}
