// symi_product8 and symi_expert_fwd8 of many rows in bf16 contexts: 8-bit products in tiles of 256 rows and 256 weight rows.
//
// Four wavefronts of 128 x 128 outputs each (128 x 64 in a tile of at most 128 rows), a reduction step of 128, which is one block of powers and one
// v_mfma_scale_f32_16x16x128_f8f6f4 a 16 x 16 block: 64 of 32 cycles in a step.  Operands travel from memory to LDS directly, 16 bytes a lane, in two stages each of
// 32 KB; LDS holds 16-byte chunk c of a row r at c ^ ((r >> 1) & 7), without bank conflicts in the fragment reads.
//  - A step is four phases of two 16-row blocks against all columns.  The right fragments of a step stay in registers for all of it and are replaced one by
//    one in its last phase, each behind its last use, so that a right stage is free again from the second phase on; the left ones are read a phase ahead.  Two stages
//    of both so give a load three to six phases (1500 - 3000 cycles) to land.
//  - The powers of four steps are a word a row: loaded once in four steps, to LDS too, and read into 16 registers; the instruction picks the byte.
//  - Loads behind the last step read the last one again: nobody reads what they bring.
// c5 (524288 rows in 256 slots, 4096 x 2048): first product with its epilogue 8.15 ms, 2.16 PFLOP/s, second 3.86 ms, 2.28 PFLOP/s; thin tiles of 16 rows for all of it took
// 122 ms.  The library's plain product of 8192^3 reaches 2.67 PFLOP/s on the same card.  What is left are epilogues with idle matrix pipes and the clock that power leaves.
#include <algorithm>
#include <type_traits>

#include "quant8.h"

namespace symi {

constexpr int G8_THREADS = 256, G8_M = 256, G8_N = 256;
constexpr int G8_STAGE = 256 * QB;                 // bytes of an operand's stage
constexpr int G8_SCALES = 4 * G8_STAGE;            // two buffers of 1 KB for either operand
constexpr int G8_LDS = G8_SCALES + 4096;
// epilogue: 16 KB for every wavefront to turn its outputs around in, the hidden units' codes and the rows' largest
constexpr int G8_CODES = 4 * 16384, G8_CODE_PITCH = 144, G8_MOST = G8_CODES + 256 * G8_CODE_PITCH;
static_assert(G8_MOST + 4096 <= G8_LDS, "epilogue's part of LDS");
constexpr unsigned G8_OUTSIDE = 0xfffff000u;       // a store there is dropped

typedef unsigned uintx4_ __attribute__((ext_vector_type(4)));

template <int V> struct Int { static constexpr int value = V; };
template <int N, int I = 0, class F>
__device__ __forceinline__ void repeat(F&& f) {   // f(Int<0>{}) .. f(Int<N - 1>{})
  if constexpr (I < N) {
    f(Int<I>{});
    repeat<N, I + 1>(f);
  }
}

// LDS reads whose completion is awaited by hand, as the compiler would wait for the loads in flight to LDS before every one
template <int OFF>
__device__ __forceinline__ intx4_ read16(unsigned addr) {
  intx4_ v;
  asm volatile("ds_read_b128 %0, %1 offset:%2" : "=v"(v) : "v"(addr), "n"(OFF));
  return v;
}
template <int OFF>
__device__ __forceinline__ int read4(unsigned addr) {
  int v;
  asm volatile("ds_read_b32 %0, %1 offset:%2" : "=v"(v) : "v"(addr), "n"(OFF));
  return v;
}
template <int N>
__device__ __forceinline__ void wait_lds() {   // all but the last N LDS operations are through
  asm volatile("s_waitcnt lgkmcnt(%0)" ::"n"(N) : "memory");
}
template <int N>
__device__ __forceinline__ void wait_loads() {
  asm volatile("s_waitcnt vmcnt(%0)" ::"n"(N) : "memory");
}
// acc += w a; byte B of the words of powers
template <int B>
__device__ __forceinline__ void mfma8(floatx4_& acc, const intx8& w, const intx8& a, int sw, int sa) {
  asm volatile("v_mfma_scale_f32_16x16x128_f8f6f4 %0, %1, %2, %0, %3, %4 op_sel:[%5,%5,0] op_sel_hi:[%6,%6,0]"
               : "+a"(acc) : "v"(w), "v"(a), "v"(sw), "v"(sa), "n"(B & 1), "n"(B >> 1));
}

// NJ: 16-column blocks of a wavefront; 8: 2 x 2 wavefronts, 4: 1 x 4 (at most 128 rows)
template <bool EXPERT, int NJ>
__device__ __forceinline__ void gemm8_tile(const Product8& p, uint8_t* const lds, const int row0, const int row1, const int slot, const int bn) {
  constexpr int CW = 16 * NJ, UW = CW / 2;          // columns of a wavefront; hidden units
  constexpr int LA = NJ;                            // 1 KB loads of the left operand a wavefront and step
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int wm = NJ == 8 ? wave >> 1 : 0, wn = NJ == 8 ? wave & 1 : wave;
  const int quarter = lane >> 4, r16 = lane & 15;
  const int pitch = p.p8, n0 = bn * (EXPERT ? G8_N / 2 : G8_N);   // first weight row (hidden unit)
  const int slot_rows = EXPERT ? 2 * p.R : p.R, slot_blocks = (slot_rows + QB - 1) / QB;
  const int nk = pitch / QB, groups = (nk + 3) / 4;

  // tile column -> weight row, counted from n0 (32 bits of offset reach it): as it is, or of every 64 the gate rows of 32 hidden units and their up rows
  auto weight_row = [&](int c) {
    if (!EXPERT) return min(c, p.R - 1 - n0);
    return ((c >> 5) & 1) * p.R + min((c >> 6) * 32 + (c & 31), p.R - 1 - n0);
  };
  const uint8_t* const a_base = p.Aq + (long long)row0 * pitch;
  const uint8_t* const w_base = p.Wq + ((long long)slot * slot_rows + n0) * pitch;
  const int last = row1 - row0 - 1;
  // Loads: wavefront w, instruction j fills rows 8 LA w + 8 j .. of the left stage (64 w + 8 j of the right one), lane l row l / 8, chunk l % 8.
  // A scalar base a step, an offset a lane, and an immediate that counts in memory and in LDS: M0, the LDS base, stands in the middle of what an operand's
  // instructions fill and is written once for them; the offset takes the immediate back out (and the base sits 4 KB low, so that it stays positive).
  unsigned vo_a[LA], vo_w[8];
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    const int chunk = ((lane & 7) ^ (((lane >> 3) + 8 * j) >> 1 & 7)) * 16;
    if (j < LA) vo_a[j] = (unsigned)min(8 * LA * wave + 8 * j + (lane >> 3), last) * (unsigned)pitch + chunk + 4096u - (unsigned)((j - 4) * 1024);
    vo_w[j] = (unsigned)weight_row(64 * wave + 8 * j + (lane >> 3)) * (unsigned)pitch + chunk + 4096u - (unsigned)((j - 4) * 1024);
  }
  const unsigned vs_a = (unsigned)min(64 * wave + lane, last) * (unsigned)p.sp;
  const unsigned vs_w = (unsigned)((n0 + weight_row(64 * wave + lane)) / QB) * (unsigned)p.sp;
  const uint8_t* const sa_base = p.As + (long long)row0 * p.sp;
  const uint8_t* const sw_base = p.Ws + (long long)slot * slot_blocks * p.sp;
  const unsigned base = (unsigned)(size_t)(void __attribute__((address_space(3)))*)lds;
  // a load to LDS needs a wait state behind a write of M0, which the compiler does not put into inline assembly
  auto set_m0 = [&](unsigned at) { asm volatile("s_mov_b32 m0, %0\n\ts_nop 0" ::"s"(at) : "memory"); };
  auto load16 = [&](auto jc, unsigned vo, const uint8_t* from) {
    asm volatile("global_load_lds_dwordx4 %0, %1 offset:%2" ::"v"(vo), "s"(from - 4096), "n"((decltype(jc)::value - 4) * 1024) : "memory");
  };
  auto load_left = [&](auto jc, auto stagec, int step) {
    constexpr int j = decltype(jc)::value;
    if (j == 0) set_m0(base + decltype(stagec)::value * G8_STAGE + wave * (LA * 1024) + 4096);
    load16(jc, vo_a[j], a_base + (long long)min(step, nk - 1) * QB);
  };
  auto load_right = [&](auto jc, auto stagec, int step) {
    constexpr int j = decltype(jc)::value;
    if (j == 0) set_m0(base + (2 + decltype(stagec)::value) * G8_STAGE + wave * 8192 + 4096);
    load16(jc, vo_w[j], w_base + (long long)min(step, nk - 1) * QB);
  };
  auto load_powers = [&](int group) {
    const int from = min(group, groups - 1) * 4;
    const unsigned to = base + G8_SCALES + (group & 1) * 1024 + wave * 256;
    set_m0(to);
    asm volatile("global_load_lds_dword %0, %1" ::"v"(vs_a), "s"(sa_base + from) : "memory");
    set_m0(to + 2048);
    asm volatile("global_load_lds_dword %0, %1" ::"v"(vs_w), "s"(sw_base + from) : "memory");
  };
  // fragment reads: this lane's address in stage 0 for either half of its 32 reduction indices; block and stage are immediates
  unsigned ad_a[2], ad_w[2];
#pragma unroll
  for (int x = 0; x < 2; ++x) {
    const unsigned in = r16 * QB + (((4 * x + quarter) ^ (r16 >> 1 & 7)) * 16);
    ad_a[x] = base + wm * 128 * QB + in;
    ad_w[x] = base + 2 * G8_STAGE + wn * CW * QB + in;
  }
  unsigned ad_sa = base + G8_SCALES + (wm * 128 + r16) * 4, ad_sw = base + G8_SCALES + 2048 + (wn * CW + r16) * 4;
  intx8 fa[2][2], fw[NJ];
  int sa[8], sw[NJ];
  floatx4_ acc[8][NJ];
#pragma unroll
  for (int i = 0; i < 8; ++i)
#pragma unroll
    for (int j = 0; j < NJ; ++j) acc[i][j] = floatx4_{0.f, 0.f, 0.f, 0.f};
  auto join8 = [](intx4_ lo, intx4_ hi) { return __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7); };
  auto read_left = [&](auto setc, auto stagec, auto blkc) {   // row block blk
    constexpr int off = decltype(stagec)::value * G8_STAGE + decltype(blkc)::value * 16 * QB;
    const intx4_ lo = read16<off>(ad_a[0]), hi = read16<off>(ad_a[1]);
    fa[decltype(setc)::value][decltype(blkc)::value & 1] = join8(lo, hi);
  };
  auto read_right = [&](auto stagec, auto jc) {
    constexpr int off = decltype(stagec)::value * G8_STAGE + decltype(jc)::value * 16 * QB;
    const intx4_ lo = read16<off>(ad_w[0]), hi = read16<off>(ad_w[1]);
    fw[decltype(jc)::value] = join8(lo, hi);
  };
  auto read_sa = [&](auto ic) { sa[decltype(ic)::value] = read4<decltype(ic)::value * 64>(ad_sa); };
  auto read_sw = [&](auto jc) { sw[decltype(jc)::value] = read4<decltype(jc)::value * 64>(ad_sw); };

  // One phase of a step: B = step & 3 (the byte of the powers), stage B & 1.  In flight at its start: phase 0 the last reads of the right
  // fragments, else nothing but what is named.
  auto phase = [&](auto pc, auto bc, int step) {
    constexpr int P = decltype(pc)::value, B = decltype(bc)::value, S = B & 1;
    constexpr int SET = P & 1;
    if constexpr (P == 0) wait_lds<(B == 0 ? 5 : 4)>(); else wait_lds<0>();
    if constexpr (P == 1) __builtin_amdgcn_s_barrier();   // everybody has read the right stage: it is free
    if constexpr (P == 3) {
      wait_loads<8>();                       // the next step has landed (the 8 loads of the right operand of the one behind it may fly)
      __builtin_amdgcn_s_barrier();          // ... for everybody, and the left stage is free
    }
    __builtin_amdgcn_sched_barrier(0);
    repeat<2 * NJ>([&](auto mc) {
      constexpr int m = decltype(mc)::value, j = m >> 1, i = 2 * P + (m & 1);
      if constexpr (P == 0 && m == 2 * NJ - 4) wait_lds<(B == 0 ? 6 : 4)>();   // the last two right fragments; behind them 4 or 6 reads of this phase
      mfma8<B>(acc[i][j], fw[j], fa[SET][m & 1], sw[j], sa[i]);
      // reads: the next phase's left fragments
      if constexpr (P < 3) {
        if constexpr (P == 0 && B == 0 && m == 0) {
          read_sa(Int<6>{});
          read_sa(Int<7>{});
        }
        if constexpr (m == 1) read_left(Int<SET ^ 1>{}, Int<S>{}, Int<2 * P + 2>{});
        if constexpr (m == 3) read_left(Int<SET ^ 1>{}, Int<S>{}, Int<2 * P + 3>{});
      } else {
        if constexpr (m == 0) read_left(Int<0>{}, Int<S ^ 1>{}, Int<0>{});
        if constexpr (m == 1) read_left(Int<0>{}, Int<S ^ 1>{}, Int<1>{});
        if constexpr (B == 3 && m == 1) repeat<6>([&](auto ic) { read_sa(ic); });
        if constexpr (m & 1) {               // the block's last use is behind us
          if constexpr (B == 3) read_sw(Int<j>{});
          read_right(Int<S ^ 1>{}, Int<j>{});
        }
      }
      // loads: left operand of step + 2 in phase 3 and the next phase 0, right operand of step + 2 in phases 1 and 2
      constexpr int every = NJ / 2;          // MFMAs from load to load
      if constexpr (m % every == every - 1) {
        constexpr int L = m / every;         // 0 .. 3
        if constexpr (P == 3) {
          if constexpr (B == 1 && L == 0) load_powers((step >> 2) + 1);
          if constexpr (NJ == 8) load_left(Int<L>{}, Int<S>{}, step + 2);
          else if constexpr (L < 2) load_left(Int<L>{}, Int<S>{}, step + 2);
        }
        if constexpr (P == 0) {
          if constexpr (NJ == 8) load_left(Int<4 + L>{}, Int<S ^ 1>{}, step + 1);
          else if constexpr (L < 2) load_left(Int<2 + L>{}, Int<S ^ 1>{}, step + 1);
        }
        if constexpr (P == 1) load_right(Int<L>{}, Int<S>{}, step + 2);
        if constexpr (P == 2) load_right(Int<4 + L>{}, Int<S>{}, step + 2);
      }
      // on to the next group's powers before they are read
      if constexpr (P == 2 && B == 3 && m == 2 * NJ - 1) {
        const unsigned by = (step >> 2) & 1 ? 0u - 1024u : 1024u;
        ad_sa += by;
        ad_sw += by;
      }
      __builtin_amdgcn_sched_barrier(0);
    });
  };
  auto one_step = [&](auto bc, int step) {
    phase(Int<0>{}, bc, step);
    phase(Int<1>{}, bc, step);
    phase(Int<2>{}, bc, step);
    phase(Int<3>{}, bc, step);
  };

  load_powers(0);
  repeat<LA>([&](auto j) { load_left(j, Int<0>{}, 0); });
  repeat<8>([&](auto j) { load_right(j, Int<0>{}, 0); });
  repeat<8>([&](auto j) { load_right(j, Int<1>{}, 1); });
  repeat<LA / 2>([&](auto j) { load_left(j, Int<1>{}, 1); });   // the other half follows in phase 0
  wait_loads<8 + LA / 2>();
  __builtin_amdgcn_s_barrier();
  read_left(Int<0>{}, Int<0>{}, Int<0>{});
  read_left(Int<0>{}, Int<0>{}, Int<1>{});
  repeat<8>([&](auto i) { read_sa(i); });
  repeat<NJ>([&](auto j) {
    if constexpr (decltype(j)::value < NJ - 1) read_sw(j);
  });
  repeat<NJ>([&](auto j) {
    if constexpr (decltype(j)::value == NJ - 1) read_sw(j);
    read_right(Int<0>{}, j);
  });
  int t = 0;
  for (; t + 4 <= nk; t += 4) {
    one_step(Int<0>{}, t);
    one_step(Int<1>{}, t + 1);
    one_step(Int<2>{}, t + 2);
    one_step(Int<3>{}, t + 3);
  }
  if (t < nk) one_step(Int<0>{}, t);
  if (t + 1 < nk) one_step(Int<1>{}, t + 1);
  if (t + 2 < nk) one_step(Int<2>{}, t + 2);
  // What is still in flight must not outlive its registers and its place in LDS.
  wait_lds<0>();
#pragma unroll
  for (int j = 0; j < NJ; ++j) asm volatile("" : "+v"(fw[j]), "+v"(sw[j]));
#pragma unroll
  for (int i = 0; i < 8; ++i) asm volatile("" : "+v"(sa[i]));
  asm volatile("" : "+v"(fa[0][0]), "+v"(fa[0][1]));
  asm volatile("s_nop 15\n\ts_nop 15" ::: "memory");   // the last MFMAs
#pragma unroll
  for (int i = 0; i < 8; ++i)
#pragma unroll
    for (int j = 0; j < NJ; ++j) asm volatile("" : "+a"(acc[i][j]));
  wait_loads<0>();
  __syncthreads();

  // ---- epilogue.  A lane has row r16 of a block and 4 columns from 4 quarter on; wavefronts turn 32 rows at a time around in LDS, so that
  // stores cover whole lines.
  uint16_t* const stg = reinterpret_cast<uint16_t*>(lds + wave * 16384);
  auto store16 = [&](void* to, bool in, unsigned ofs, uint4 x) {   // out of range: dropped, without a branch
    const __amdgpu_buffer_rsrc_t rsrc = __builtin_amdgcn_make_buffer_rsrc(to, 0, (int)G8_OUTSIDE, 0x00020000);
    __builtin_amdgcn_raw_buffer_store_b128(__builtin_bit_cast(uintx4_, x), rsrc, (int)(in ? ofs : G8_OUTSIDE), 0, 0);
  };
  if constexpr (!EXPERT) {
    constexpr int LD = CW + 8, LB = CW / 8, NIT = 32 * LB / 64;
#pragma unroll
    for (int i2 = 0; i2 < 4; ++i2) {
      const int rbase = row0 + wm * 128 + i2 * 32;
#pragma unroll
      for (int ih = 0; ih < 2; ++ih)
#pragma unroll
        for (int j = 0; j < NJ; ++j) {
          const floatx4_ x = acc[2 * i2 + ih][j];
          *reinterpret_cast<uint2*>(stg + (ih * 16 + r16) * LD + 16 * j + 4 * quarter) = make_uint2(pack_bf16x2(x[0], x[1]), pack_bf16x2(x[2], x[3]));
        }
      asm volatile("" ::: "memory");   // a wavefront's LDS operations are carried out in order
      uint16_t* const to = static_cast<uint16_t*>(p.Y) + (long long)rbase * p.R;
      const int col = n0 + wn * CW + (lane & (LB - 1)) * 8;
      uint4 x[NIT];
#pragma unroll
      for (int it = 0; it < NIT; ++it) x[it] = *reinterpret_cast<const uint4*>(stg + (it * (64 / LB) + lane / LB) * LD + (lane & (LB - 1)) * 8);
#pragma unroll
      for (int it = 0; it < NIT; ++it) {
        const int rr = it * (64 / LB) + lane / LB;
        store16(to, rbase + rr < row1 && col < p.R, (unsigned)(rr * p.R + col) * 2u, x[it]);
      }
      asm volatile("" ::: "memory");
    }
  } else {
    // u and v give h, which stays in the gate's accumulators until the row's largest is known
    constexpr int LD = UW + 8, LB = UW / 8, NIT = 32 * LB / 64;
    int* const most_s = reinterpret_cast<int*>(lds + G8_MOST);
    const bool keep = p.UV != nullptr;
    const int f = p.R, hu0 = n0 + wn * UW;
#pragma unroll
    for (int i2 = 0; i2 < 4; ++i2) {
      const int rbase = row0 + wm * 128 + i2 * 32;
#pragma unroll
      for (int ih = 0; ih < 2; ++ih) {
        int most = 0;
#pragma unroll
        for (int q = 0; q < NJ / 2; ++q) {   // 16 hidden units
          const int g = 4 * (q >> 1) + (q & 1);
          floatx4_ u = acc[2 * i2 + ih][g], v = acc[2 * i2 + ih][g + 2], h;
          asm("" : "+v"(u), "+v"(v));        // one read of each accumulator
          // hidden units behind the last one count as nothing
          const bool in = hu0 + 16 * q + 4 * quarter < f;
#pragma unroll
          for (int c = 0; c < 4; ++c) {
            h[c] = in ? u[c] * sigmoid8(u[c]) * v[c] : 0.f;
            most = max(most, size_of(h[c]));
          }
          acc[2 * i2 + ih][g] = h;
          if (keep) {
            const int at = (ih * 16 + r16) * LD + 16 * q + 4 * quarter;
            *reinterpret_cast<uint2*>(stg + at) = make_uint2(pack_bf16x2(u[0], u[1]), pack_bf16x2(u[2], u[3]));
            *reinterpret_cast<uint2*>(stg + 32 * LD + at) = make_uint2(pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]));
            *reinterpret_cast<uint2*>(stg + 64 * LD + at) = make_uint2(pack_bf16x2(h[0], h[1]), pack_bf16x2(h[2], h[3]));
          }
        }
        most = max(most, __shfl_xor(most, 16, 64));
        most = max(most, __shfl_xor(most, 32, 64));
        if (quarter == 0) most_s[wn * 256 + wm * 128 + i2 * 32 + ih * 16 + r16] = most;
      }
      if (keep) {
        asm volatile("" ::: "memory");
        uint16_t* const uv = p.UV + (long long)rbase * 2 * f;
        uint16_t* const hh = p.H + (long long)rbase * f;
        const int hu = hu0 + (lane & (LB - 1)) * 8;
        uint4 xu[NIT], xv[NIT], xh[NIT];
#pragma unroll
        for (int it = 0; it < NIT; ++it) {
          const uint16_t* const at = stg + (it * (64 / LB) + lane / LB) * LD + (lane & (LB - 1)) * 8;
          xu[it] = *reinterpret_cast<const uint4*>(at);
          xv[it] = *reinterpret_cast<const uint4*>(at + 32 * LD);
          xh[it] = *reinterpret_cast<const uint4*>(at + 64 * LD);
        }
#pragma unroll
        for (int it = 0; it < NIT; ++it) {
          const int rr = it * (64 / LB) + lane / LB;
          const bool in = rbase + rr < row1 && hu < f;
          const unsigned o = (unsigned)(rr * f + hu) * 2u;
          store16(uv, in, o + (unsigned)(rr * f) * 2u, xu[it]);
          store16(uv + f, in, o + (unsigned)(rr * f) * 2u, xv[it]);
          store16(hh, in, o, xh[it]);
        }
        asm volatile("" ::: "memory");
      }
    }
    __syncthreads();
    uint8_t* const codes = lds + G8_CODES;
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const int r = wm * 128 + i * 16 + r16;
      int most = max(most_s[r], most_s[256 + r]);
      if (NJ == 4) most = max(most, max(most_s[512 + r], most_s[768 + r]));
      const int e = scale_of(most);
      const float inv = inverse_of(e);
#pragma unroll
      for (int q = 0; q < NJ / 2; ++q) {
        const floatx4_ h = acc[i][4 * (q >> 1) + (q & 1)];
        *reinterpret_cast<uint32_t*>(codes + r * G8_CODE_PITCH + wn * UW + 16 * q + 4 * quarter) = codes4(h[0], h[1], h[2], h[3], inv);
      }
      if (wn == 0 && quarter == 0 && row0 + r < row1) {
        uint8_t* const hs = p.Hs + (long long)(row0 + r) * p.hsp;
        hs[bn] = (uint8_t)e;
        if (bn == p.hp8 / QB - 1)
          for (int b = bn + 1; b < p.hsp; ++b) hs[b] = 0;
      }
    }
    __syncthreads();
    for (int i = tid; i < (row1 - row0) * 8; i += G8_THREADS)
      *reinterpret_cast<uint4*>(p.Hq + (long long)(row0 + (i >> 3)) * p.hp8 + n0 + (i & 7) * 16) =
          *reinterpret_cast<const uint4*>(codes + (i >> 3) * G8_CODE_PITCH + (i & 7) * 16);
  }
}

// Workgroup b runs on XCD b mod 8, each with an L2 of its own.  An XCD takes an eighth of the tiles in a row: of every 8 row tiles (of one slot,
// where it has that many) all column tiles, the row index fastest.
__device__ __forceinline__ bool deal8(int mts, int ntx, int& mt, int& bn) {
  const int n_tiles = mts * ntx, chunk = (n_tiles + 7) / 8;
  const int s = blockIdx.x >> 3, tile = (blockIdx.x & 7) * chunk + s;
  if (s >= chunk || tile >= n_tiles) return false;
  const int round = tile / (8 * ntx), in = tile - round * 8 * ntx, rows = min(8, mts - 8 * round);
  bn = __builtin_amdgcn_readfirstlane(in / rows);
  mt = __builtin_amdgcn_readfirstlane(8 * round + in % rows);
  return true;
}

template <bool EXPERT>
__global__ __launch_bounds__(G8_THREADS) void gemm8_kernel(Product8 p, int ntx) {
  __shared__ __attribute__((aligned(1024))) uint8_t lds[G8_LDS];
  int mt, bn;
  if (!deal8(p.map[0], ntx, mt, bn)) return;
  const int row0 = __builtin_amdgcn_readfirstlane(p.map[4 + 2 * mt]), entry = __builtin_amdgcn_readfirstlane(p.map[5 + 2 * mt]);
  const int slot = entry & 0xffff, row1 = row0 + (entry >> 16) + 1;
  if (row1 - row0 <= G8_M / 2) gemm8_tile<EXPERT, 4>(p, lds, row0, row1, slot, bn);
  else gemm8_tile<EXPERT, 8>(p, lds, row0, row1, slot, bn);
}

// ---- fp32 contexts: codes become bf16 values on their way into the bf16 instruction, which keeps fp32's digits and has half the rate.
// A tile of 128 x 128, 64 x 64 a wavefront, two or three workgroups a unit: while one widens codes (an instruction for two) another has the matrix pipes.  A step's
// 32 KB go through registers into LDS, loaded a step ahead.  Powers are put into the values as they are widened, exactly, where all of the tile's are between
// 2^-100 and 2^100; else (FAR) a block's sum is scaled behind it, which knows no limits.  The power of a block of zeros is 0 and takes its tile there: 15009 rows,
// 1160 -> 5488, with every tenth row zero 361 us for 264, 16384 rows in 8 slots of 4096 x 4096 890 for 571.  15009 rows, 1160 -> 5488: 268 us, 790 TFLOP/s with the half-filled last
// blocks; with the choice between the two made step by step, which costs registers, 514.
constexpr int W8_M = 128, W8_N = 128;

template <bool SCALED>
__device__ __forceinline__ void widen16(const intx4_ q, float scale, bf16x8_ (&out)[2]) {   // 16 codes
  typedef __bf16 bf16x2_ __attribute__((ext_vector_type(2)));
#pragma unroll
  for (int h = 0; h < 2; ++h)
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const unsigned w = (unsigned)q[2 * h + i];
      const bf16x2_ lo = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, SCALED ? scale : 1.f, false);
      const bf16x2_ hi = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, SCALED ? scale : 1.f, true);
      out[h][4 * i] = lo[0];
      out[h][4 * i + 1] = lo[1];
      out[h][4 * i + 2] = hi[0];
      out[h][4 * i + 3] = hi[1];
    }
}

template <bool FAR>
__device__ __forceinline__ void wide8_tile(const Product8& p, uint8_t* const lds, const int row0, const int last, const int slot, const int bn) {
  const int n0 = bn * W8_N;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, wm = wave >> 1, wn = wave & 1, quarter = lane >> 4, r16 = lane & 15;
  const int pitch = p.p8, nk = pitch / QB, slot_blocks = (p.R + QB - 1) / QB;
  const uint8_t* const a_base = p.Aq + (long long)row0 * pitch;
  const uint8_t* const w_base = p.Wq + ((long long)slot * p.R + n0) * pitch;
  // thread -> rows tid / 8 + 32 i, chunk tid % 8
  unsigned from_a[4], from_w[4], to[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int r = tid / 8 + 32 * i;
    from_a[i] = (unsigned)min(r, last) * (unsigned)pitch + (tid & 7) * 16;
    from_w[i] = (unsigned)min(r, p.R - 1 - n0) * (unsigned)pitch + (tid & 7) * 16;
    to[i] = r * QB + ((tid & 7) ^ (r >> 1 & 7)) * 16;
  }
  const uint8_t* sa_from[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) sa_from[i] = p.As + (long long)(row0 + min(wm * 64 + 16 * i + r16, last)) * p.sp;
  const uint8_t* const sw_from = p.Ws + ((long long)slot * slot_blocks + bn) * p.sp;   // a tile's columns are one block of rows of the weight
  intx4_ ra[4], rw[4];
  int pa[4], pw;
  auto fetch = [&](int k) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      ra[i] = *reinterpret_cast<const intx4_*>(a_base + (long long)k * QB + from_a[i]);
      rw[i] = *reinterpret_cast<const intx4_*>(w_base + (long long)k * QB + from_w[i]);
      pa[i] = sa_from[i][k];
    }
    pw = sw_from[k];
  };
  auto read = [&](int operand, int block, int x) {
    const int r = block * 16 + r16;
    return *reinterpret_cast<const intx4_*>(lds + operand * W8_M * QB + r * QB + ((4 * x + quarter) ^ (r >> 1 & 7)) * 16);
  };
  floatx4_ acc[4][4] = {};
  fetch(0);
  for (int k = 0; k < nk; ++k) {
    __syncthreads();
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      *reinterpret_cast<intx4_*>(lds + to[i]) = ra[i];
      *reinterpret_cast<intx4_*>(lds + W8_M * QB + to[i]) = rw[i];
    }
    int sa[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) sa[i] = pa[i];
    const int sw = pw;
    __syncthreads();
    if (k + 1 < nk) fetch(k + 1);
    if constexpr (!FAR) {
      const float scale_w = power_of(sw);
#pragma unroll
      for (int x = 0; x < 2; ++x) {
        bf16x8_ w[4][2];
#pragma unroll
        for (int j = 0; j < 4; ++j) widen16<true>(read(1, wn * 4 + j, x), scale_w, w[j]);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          bf16x8_ a[2];
          widen16<true>(read(0, wm * 4 + i, x), power_of(sa[i]), a);
#pragma unroll
          for (int h = 0; h < 2; ++h)
#pragma unroll
            for (int j = 0; j < 4; ++j) acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(w[j][h], a[h], acc[i][j], 0, 0, 0);
        }
      }
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        bf16x8_ a[2][2];
#pragma unroll
        for (int x = 0; x < 2; ++x) widen16<false>(read(0, wm * 4 + i, x), 1.f, a[x]);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          floatx4_ part = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
          for (int x = 0; x < 2; ++x) {
            bf16x8_ w[2];
            widen16<false>(read(1, wn * 4 + j, x), 1.f, w);
#pragma unroll
            for (int h = 0; h < 2; ++h) part = __builtin_amdgcn_mfma_f32_16x16x32_bf16(w[h], a[x][h], part, 0, 0, 0);
          }
#pragma unroll
          for (int c = 0; c < 4; ++c) acc[i][j][c] += ldexpf(part[c], sw + sa[i] - 254);
          __builtin_amdgcn_sched_barrier(0);   // one block after the other: in flight together they take all registers
        }
      }
    }
  }
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int r = wm * 64 + 16 * i + r16;
    if (r > last) continue;
    float* const y = static_cast<float*>(p.Y) + (long long)(row0 + r) * p.R + n0 + wn * 64 + 4 * quarter;
#pragma unroll
    for (int j = 0; j < 4; ++j)
      if (n0 + wn * 64 + 16 * j + 4 * quarter < p.R) *reinterpret_cast<f32x4_f32*>(y + 16 * j) = __builtin_bit_cast(f32x4_f32, acc[i][j]);
  }
}

// Whether one of the four bytes is outside 27 .. 227
__device__ __forceinline__ bool far4(unsigned w) {
  bool far = false;
#pragma unroll
  for (int i = 0; i < 4; ++i) far |= (w >> (8 * i) & 0xff) - 27u > 200u;
  return far;
}

__global__ __launch_bounds__(G8_THREADS, 2) void wide8_kernel(Product8 p, int ntx) {
  __shared__ __attribute__((aligned(16))) uint8_t lds[(W8_M + W8_N) * QB];
  int mt, bn;
  if (!deal8(p.map[0], ntx, mt, bn)) return;
  const int row0 = __builtin_amdgcn_readfirstlane(p.map[4 + 2 * mt]), entry = __builtin_amdgcn_readfirstlane(p.map[5 + 2 * mt]);
  const int slot = entry & 0xffff, last = entry >> 16;
  // the tile's powers: two threads a row, and the weight's; of the last four of a row those that there are
  const int nk = p.p8 / QB, half = threadIdx.x & 1;
  const uint8_t* const rows = p.As + (long long)(row0 + min((int)threadIdx.x >> 1, last)) * p.sp;
  const uint8_t* const weight = p.Ws + ((long long)slot * ((p.R + QB - 1) / QB) + bn) * p.sp;
  bool far = false;
  for (int k = 4 * half; k < nk; k += 8) {
    const unsigned keep = nk - k >= 4 ? 0u : 0x7f7f7f7fu << (8 * (nk - k));   // 2^0 for what is behind the end
    const unsigned mask = nk - k >= 4 ? ~0u : (1u << (8 * (nk - k))) - 1;
    far |= far4((*reinterpret_cast<const unsigned*>(rows + k) & mask) | keep);
    far |= far4((*reinterpret_cast<const unsigned*>(weight + k) & mask) | keep);
  }
  if (__syncthreads_or(far)) wide8_tile<true>(p, lds, row0, last, slot, bn);
  else wide8_tile<false>(p, lds, row0, last, slot, bn);
}

static unsigned grid8(const symi_ctx* ctx, int rows, int ntx) {
  const long long tiles = ((long long)ctx->cfg.T * ctx->cfg.k / rows + ctx->cfg.S_tot) * ntx;
  return (unsigned)((tiles + 7) / 8 * 8);
}

void launch_gemm8(const symi_ctx* ctx, const Product8& p, int rows, bool expert, hipStream_t st) {
  if (ctx->cfg.dtype != SYMI_BF16) {
    const int ntx = cdiv(p.R, W8_N);
    SYMI_TIMED(ctx, K_PRODUCT8, st, (wide8_kernel<<<grid8(ctx, rows, ntx), G8_THREADS, 0, st>>>(p, ntx)));
    return;
  }
  const int ntx = expert ? cdiv(p.R, G8_N / 2) : cdiv(p.R, G8_N);
  if (expert) SYMI_TIMED(ctx, K_EXPERT8, st, (gemm8_kernel<true><<<grid8(ctx, rows, ntx), G8_THREADS, 0, st>>>(p, ntx)));
  else SYMI_TIMED(ctx, K_PRODUCT8, st, (gemm8_kernel<false><<<grid8(ctx, rows, ntx), G8_THREADS, 0, st>>>(p, ntx)));
}

}  // namespace symi
