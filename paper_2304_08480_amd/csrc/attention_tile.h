// The attention kernels' common parts: tiles in the LDS, products of a tile with rows in registers, a wave's share of the forward pass.
//
// One side's rows are in registers, one row a lane (of 32), the other side's are walked in tiles that are brought into the LDS.  The 32 x 32 products are taken with
// the walked side as rows, so that a lane holds 16 values of its own row's softmax, and those values, rounded to bf16, are at once the B operand of the
// product that follows, whose A operand is the walked tile transposed.
#pragma once
#include "common.h"

#include <float.h>
#include <math.h>

namespace disco {
namespace {

typedef __attribute__((ext_vector_type(8))) __bf16 bf16x8;
typedef __attribute__((ext_vector_type(4))) __bf16 bf16x4;
typedef __attribute__((ext_vector_type(2))) __bf16 bf16x2;
typedef __attribute__((ext_vector_type(16))) float f32x16;
typedef __attribute__((ext_vector_type(4))) float f32x4;
typedef __attribute__((ext_vector_type(2))) float f32x2;
typedef __attribute__((ext_vector_type(4))) uint32_t u32x4;
typedef __attribute__((address_space(3))) bf16x4* lds_bf16x4;

constexpr float LOG2E = 1.4426950408889634f, LN2 = 0.6931471805599453f;

// Scores in base 2 from which on fp32 numbers are 2 apart.  Keys that are hidden by their scores (the type's lowest value in a channel) are far beyond it,
// alone in a row's first tiles or in all of them.  Forward, the rounding of the reference that is taken off them would be more than exp2 holds:
// it is taken off before they are multiplied into base 2.  Backward, lse tells the softmax of such a row no more: the row's values are taken as 0.
constexpr float FAR = 0x1p24f;
__device__ __forceinline__ float base2(float lse) {
  const float x = lse * LOG2E;
  return fabsf(x) < FAR || !(fabsf(lse) <= FLT_MAX) ? x : INFINITY;              // exp2(-inf) = 0
}

// A walked tile in the LDS: rows of DP elements, padded to a power of two of bytes, 16-byte pieces XOR-ed with bits of the row so that
// neither the 16 rows that a quarter-wave reads one piece of (ds_read_b128) nor the 4 rows that a half-wave reads 64 bytes of
// (ds_read_b64_tr_b16) share a bank.
template <int DP>
struct Layout {
  static_assert(DP == 32 || DP == 64 || DP == 96 || DP == 128);
  static constexpr int PITCH = DP == 32 ? 64 : DP == 64 ? 128 : 256;
  static constexpr int PIECES = DP / 8;
  __device__ static __forceinline__ int swizzle(int row) {
    if (PITCH == 64) return row >> 2 & 3;
    if (PITCH == 128) return (row >> 1 & 1) << 2 | (row >> 2 & 3);
    return (row & 3) << 2 | (row >> 2 & 3);
  }
  __device__ static __forceinline__ int at(int row, int piece) { return row * PITCH + ((piece ^ swizzle(row)) << 4); }
};

// ROWS rows of a matrix on their way to the LDS, through registers so that they are under way while the previous tile is used.  Rows
// past `rows` and pieces past the head's width are zeros, by the bounds of the buffer resource: they meet zeros or masked values, never what lies
// behind them.  LAST: nothing reads them after this, so they are not kept in the caches (the instruction's nt bit).
constexpr uint32_t NOWHERE = 0xfffffff0u;       // past the end of any buffer
__device__ __forceinline__ __amdgpu_buffer_rsrc_t rows_at(const __bf16* base, int64_t pitch, int rows, int most, int head_dim) {
  const uint64_t v = reinterpret_cast<uint64_t>(base);
  const uint32_t lo = __builtin_amdgcn_readfirstlane((uint32_t)v), hi = __builtin_amdgcn_readfirstlane((uint32_t)(v >> 32));
  const uint32_t n = rows <= 0 ? 0 : rows < most ? rows : most;
  const uint32_t bytes = n ? (n - 1) * (uint32_t)(pitch * 2) + (uint32_t)head_dim * 2 : 0;
  return __builtin_amdgcn_make_buffer_rsrc(reinterpret_cast<void*>((uint64_t)hi << 32 | lo), 0, __builtin_amdgcn_readfirstlane(bytes), 0x00020000);
}
template <int DP, int ROWS, int THREADS, bool LAST = false>
struct Stage {
  using L = Layout<DP>;
  static constexpr int ALL = ROWS * L::PIECES, N = (ALL + THREADS - 1) / THREADS;
  u32x4 v[N];
  uint32_t from[N];
  __device__ __forceinline__ void init(int64_t pitch, int head_dim) {
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int id = threadIdx.x % THREADS + i * THREADS, row = id / L::PIECES, piece = id % L::PIECES;
      from[i] = piece * 8 < head_dim && row < ROWS ? (uint32_t)row * (uint32_t)(pitch * 2) + piece * 16 : NOWHERE;
    }
  }
  __device__ __forceinline__ void fetch(const __bf16* base, int64_t pitch, int rows, int head_dim) {
    const __amdgpu_buffer_rsrc_t r = rows_at(base, pitch, rows, ROWS, head_dim);
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] = __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(r, from[i], 0, LAST ? 2 : 0));
  }
  __device__ __forceinline__ void put(char* lds) const {
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int id = threadIdx.x % THREADS + i * THREADS;
      if (ALL % THREADS == 0 || id < ALL) *reinterpret_cast<u32x4*>(lds + L::at(id / L::PIECES, id % L::PIECES)) = v[i];
    }
  }
};

// One row a lane as the B operand of DP / 16 products: lanes 0-31 hold channels 16 s + 0..7 of their row, lanes 32-63 the other 8.
template <int DP>
struct Rows {
  bf16x8 f[DP / 16];
  __device__ __forceinline__ void fetch(const __bf16* row, bool there, int head_dim) {
    const int half = (threadIdx.x & 63) >> 5;
#pragma unroll
    for (int s = 0; s < DP / 16; ++s) {
      u32x4 w = {0, 0, 0, 0};
      if (there && s * 16 + half * 8 < head_dim) w = *reinterpret_cast<const u32x4*>(row + s * 16 + half * 8);
      f[s] = __builtin_bit_cast(bf16x8, w);
    }
  }
};

__device__ __forceinline__ f32x16 mfma(bf16x8 a, bf16x8 b, f32x16 c) { return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0); }
__device__ __forceinline__ f32x16 zeros16() {
  f32x16 z;
#pragma unroll
  for (int i = 0; i < 16; ++i) z[i] = 0.f;
  return z;
}

// The order in which a block's LDS reads and matrix instructions are to be issued: AHEAD reads first, then MFMAS instructions with READS reads after
// each as long as there are any.  Left alone the compiler reads an operand just before its use, and every product waits for the LDS.
constexpr int AHEAD_P = 6, AHEAD_A = 8;
template <int AHEAD, int READS, int TOTAL, int MFMAS>
__device__ __forceinline__ void interleave() {
  __builtin_amdgcn_sched_group_barrier(0x100, AHEAD < TOTAL ? AHEAD : TOTAL, 0);
  constexpr int STEPS = AHEAD < TOTAL ? (TOTAL - AHEAD) / READS : 0;
#pragma unroll
  for (int i = 0; i < STEPS; ++i) {
    __builtin_amdgcn_sched_group_barrier(0x008, 1, 0);
    __builtin_amdgcn_sched_group_barrier(0x100, READS, 0);
  }
  __builtin_amdgcn_sched_group_barrier(0x008, MFMAS - STEPS, 0);
}

// 32 walked rows times the lanes' rows: element r of a lane is walked row 8 (r / 4) + 4 half + r % 4.  N such products at once, c[n] of
// the rows at lds + n STEP with b(n, s): they share the addresses, and no product waits for the one before it.  (The lane's address is hidden from the
// compiler: it would keep one register for each of the DP / 16 pieces, 16 more in accumulate(), and have none left for two waves a SIMD.)
template <int DP, int N, int STEP, class B>
__device__ __forceinline__ void products(f32x16 (&c)[N], const char* lds, B b) {
  using L = Layout<DP>;
  const int lane = threadIdx.x & 63;
  int base = L::at(lane & 31, lane >> 5);
  asm volatile("" : "+v"(base));
#pragma unroll
  for (int s = 0; s < DP / 16; ++s) {
    const char* at = lds + (base ^ s << 5);
#pragma unroll
    for (int n = 0; n < N; ++n) c[n] = mfma(*reinterpret_cast<const bf16x8*>(at + n * STEP), b(n, s, base), s ? c[n] : zeros16());
  }
  interleave<AHEAD_P, 1, DP / 16 * N, DP / 16 * N>();
}
// A wave in its matrix instructions goes before the other one of its SIMD, which then does its softmax in their shadow (one sequence of 8192, above: 302, 411
// and 601 us; without 323, 426 and 643; 8 of 1024, not causal, 16 heads of 64, forward 56 and 62).  The short kernels, whose waves wait for memory, gain nothing.
__device__ __forceinline__ void matrix_work(bool on) {
  if (on) __builtin_amdgcn_s_setprio(1);
  else __builtin_amdgcn_s_setprio(0);
}
__device__ __forceinline__ int walked(int r, int half) { return 8 * (r >> 2) + 4 * half + (r & 3); }

// A lane's values for 32 walked rows as the B operand of two products over 16 of them each, in the order of products().
struct Weights { bf16x8 f[2]; };
__device__ __forceinline__ Weights rounded(const f32x16& p) {
  Weights w;
#pragma unroll
  for (int j = 0; j < 2; ++j)
#pragma unroll
    for (int e = 0; e < 8; ++e) w.f[j][e] = (__bf16)p[8 * j + e];
  return w;
}
// acc_n[m] += (channels 32 m .. of 32 walked rows at lds + n STEP, transposed) x weights_n, N of them with shared addresses
template <int DP, int N, int STEP>
__device__ __forceinline__ void accumulate(f32x16 (*const (&acc)[N])[DP / 32], const char* lds, const Weights (&w)[N]) {
  using L = Layout<DP>;
  const int lane = threadIdx.x & 63, half = lane >> 5, in16 = lane & 15, high = lane >> 4 & 1;
  int base = L::at(4 * half + (in16 >> 2), 2 * high + ((in16 & 3) >> 1)) + 8 * (in16 & 1);
  asm volatile("" : "+v"(base));
#pragma unroll
  for (int m = 0; m < DP / 32; ++m) {
    // 8 rows on, the swizzle has bit 1 of the piece the other way round
    const char *even = lds + (base ^ m << 6), *odd = lds + 8 * L::PITCH + (base ^ (m << 6 | 32));
#pragma unroll
    for (int j = 0; j < 2; ++j)
#pragma unroll
      for (int n = 0; n < N; ++n) {
        const bf16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((lds_bf16x4)(even + 16 * j * L::PITCH + n * STEP));
        const bf16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((lds_bf16x4)(odd + 16 * j * L::PITCH + n * STEP));
        (*acc[n])[m] = mfma(__builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7), w[n].f[j], (*acc[n])[m]);
      }
  }
  interleave<AHEAD_A, 2, DP / 32 * 4 * N, DP / 32 * 2 * N>();
}

// A lane's row of an accumulated product, times f, as bf16.  The two halves of a wave hold 4 channels each of every 8 of a row: they exchange
// them, so that each stores 8.
template <int DP>
__device__ __forceinline__ void store_row(__bf16* row, const f32x16 (&acc)[DP / 32], float f, int head_dim, bool there) {
  const int half = (threadIdx.x & 63) >> 5;
#pragma unroll
  for (int m = 0; m < DP / 32; ++m)
#pragma unroll
    for (int g = 0; g < 4; g += 2) {
      u32x4 w;
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        const auto pack = [&](int r) {
          const bf16x2 v = {(__bf16)(acc[m][r] * f), (__bf16)(acc[m][r + 1] * f)};
          return __builtin_bit_cast(uint32_t, v);
        };
        const auto x = __builtin_amdgcn_permlane32_swap(pack(4 * g + 2 * e), pack(4 * g + 4 + 2 * e), false, false);
        w[e] = x[0];
        w[2 + e] = x[1];
      }
      const int c = 32 * m + 8 * (g + half);
      if (there && c < head_dim) *reinterpret_cast<u32x4*>(row + c) = w;
    }
}

__device__ __forceinline__ float other_half(float v) { return __shfl_xor(v, 32); }

// A workgroup's shape: SETS sets of WAVES waves.  All sets have the same WAVES times 32 rows in registers and each walks a share of every tile, PER rows
// of the WALK; what they have come to is joined at the end.  One set, unless few workgroups have long walks.
template <int DP, int WAVES, int SETS>
struct Shape {
  static constexpr int THREADS = 64 * WAVES * SETS, OWN = 32 * WAVES, PER = WAVES == 1 ? 32 : 64, WALK = PER * SETS;
  static constexpr int SUB = 32 * Layout<DP>::PITCH, SHARE = PER * Layout<DP>::PITCH, TILE = WALK * Layout<DP>::PITCH;
  static constexpr int ACC = DP * 128, JOIN = SETS / 2 * WAVES * (ACC + 512);      // accumulators of a wave; what is handed over at once
  static constexpr int LDS = 4 * TILE;
  static_assert(JOIN <= LDS);
};
template <int WAVES>
__device__ __forceinline__ int wave_of() { return (int)__builtin_amdgcn_readfirstlane(threadIdx.x >> 6) % WAVES; }
template <int WAVES>
__device__ __forceinline__ int set_of() { return (int)__builtin_amdgcn_readfirstlane(threadIdx.x >> 6) / WAVES; }

// A wave's accumulators into the LDS, 16 bytes a lane and row, and out of it: f times the own plus g times those.
template <int DP>
__device__ __forceinline__ void hand_over(char* lds, const f32x16 (&acc)[DP / 32]) {
  f32x4* to = reinterpret_cast<f32x4*>(lds) + (threadIdx.x & 63);
#pragma unroll
  for (int m = 0; m < DP / 32; ++m)
#pragma unroll
    for (int g = 0; g < 4; ++g) to[(m * 4 + g) * 64] = f32x4{acc[m][4 * g], acc[m][4 * g + 1], acc[m][4 * g + 2], acc[m][4 * g + 3]};
}
template <int DP>
__device__ __forceinline__ void take_over(const char* lds, f32x16 (&acc)[DP / 32], float own = 1.f, float other = 1.f) {
  const f32x4* from = reinterpret_cast<const f32x4*>(lds) + (threadIdx.x & 63);
#pragma unroll
  for (int m = 0; m < DP / 32; ++m)
#pragma unroll
    for (int g = 0; g < 4; ++g) {
      const f32x4 v = from[(m * 4 + g) * 64];
#pragma unroll
      for (int e = 0; e < 4; ++e) acc[m][4 * g + e] = fmaf(acc[m][4 * g + e], own, v[e] * other);
    }
}
// The sums of all sets to set 0, in halves: the same order in every call.
template <int DP, int WAVES, int SETS>
__device__ __forceinline__ void join(char* lds, int wave, int set, f32x16 (&acc)[DP / 32]) {
#pragma unroll
  for (int n = SETS / 2; n >= 1; n /= 2) {
    if (set >= n && set < 2 * n) hand_over<DP>(lds + ((set - n) * WAVES + wave) * (DP * 128), acc);
    __syncthreads();
    if (set < n) take_over<DP>(lds + (set * WAVES + wave) * (DP * 128), acc);
    __syncthreads();
  }
}

// A wave's share of the forward pass: 32 queries, one a lane, the keys walked, 64 a step with several waves to a set: two products that
// share their addresses, and one exchange of maxima.
template <int DP>
struct Forward {
  Rows<DP> q;
  f32x16 acc[DP / 32];
  float top = -INFINITY, total = 0.f;            // the lane's reference (not always its maximum) and its half's sum
  // SUBS times 32 keys from key j on; keys past `last` are masked where `edge`
  template <int SUBS>
  __device__ __forceinline__ void step(const char* lds_k, const char* lds_v, int j, bool edge, int last, float c) {
    constexpr int SUB = 32 * Layout<DP>::PITCH;
    const int half = (threadIdx.x & 63) >> 5;
    f32x16 s[SUBS];
    if (SUBS > 1) matrix_work(true);
    products<DP, SUBS, SUB>(s, lds_k, [&](int, int k, int) { return q.f[k]; });
    if (SUBS > 1) matrix_work(false);
    if (edge) {
      int most = last - j - 4 * half;
      asm volatile("" : "+v"(most));             // keeps the branch: as selects every tile would pay for it
#pragma unroll
      for (int n = 0; n < SUBS; ++n)
#pragma unroll
        for (int r = 0; r < 16; ++r)
          if (32 * n + walked(r, 0) > most) s[n][r] = -INFINITY;
    }
    float m = s[0][0];
#pragma unroll
    for (int n = 0; n < SUBS; ++n)
#pragma unroll
      for (int r = 0; r < 16; ++r) m = fmaxf(m, s[n][r]);
    m = fmaxf(m, other_half(m));
    // The reference follows the maximum only when a row's has risen by 2^8 since: sums stay below 2^8 times their number of terms, bf16 values keep their
    // relative precision, and the accumulators are rescaled a few times a row instead of at every step.
    if (__any((m - top) * c > 8.f)) {
      const float next = fmaxf(top, m), fade = __builtin_amdgcn_exp2f((top - fmaxf(next, -FLT_MAX)) * c);
      top = next;
      total *= fade;
#pragma unroll
      for (int d = 0; d < DP / 32; ++d) acc[d] *= fade;
    }
    float ref = top * c;
    const bool far = !(fabsf(ref) < FAR);
    if (__any(far)) {
      float base = far ? fmaxf(top, -FLT_MAX) : 0.f;      // minus infinity so far: such keys add nothing
      asm volatile("" : "+v"(base));                      // keeps the branch
#pragma unroll
      for (int n = 0; n < SUBS; ++n)
#pragma unroll
        for (int r = 0; r < 16; ++r) s[n][r] -= base;
      ref = far ? 0.f : ref;
    }
    float sum[2] = {0.f, 0.f};
    Weights w[SUBS];
#pragma unroll
    for (int n = 0; n < SUBS; ++n) {
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        s[n][r] = __builtin_amdgcn_exp2f(fmaf(s[n][r], c, -ref));
        sum[r & 1] += s[n][r];
      }
      w[n] = rounded(s[n]);
    }
    total += sum[0] + sum[1];
    if (SUBS > 1) matrix_work(true);
#pragma unroll
    for (int n = 0; n < SUBS; ++n) accumulate<DP, 1, 0>({&acc}, lds_v + n * SUB, {w[n]});
    if (SUBS > 1) matrix_work(false);
  }
};

// delta of a row all of whose keys are in one tile: sum P dP, which is <do, o> without the roundings of o to bf16 and of P on the way to it.  They are
// shared by all of a row's dS, and weigh most where its keys are few: a row of one key has no dq and adds nothing to its dk.  (Relative errors of dq and dk
// against 64 bits, packed causal batches of mean lengths from 10 to 60: 0.0024 for 0.0028 to 0.0032; of 0.0017 that is the rounding of dq and dk themselves.
// Rows of more keys would take a second walk, and lose little without it.)
__device__ __forceinline__ float own_delta(const f32x16& p, const f32x16& dp) {
  float d = 0.f;
#pragma unroll
  for (int r = 0; r < 16; ++r) d = fmaf(p[r], dp[r], d);
  return d + other_half(d);
}

template <int DP>
__device__ __forceinline__ void put_rows(char* lds, const Rows<DP>& r) {
  const int lane = threadIdx.x & 63, base = Layout<DP>::at(lane & 31, lane >> 5);
#pragma unroll
  for (int s = 0; s < DP / 16; ++s) *reinterpret_cast<bf16x8*>(lds + (base ^ s << 5)) = r.f[s];
}

template <int DP>
__device__ __forceinline__ void take_rows(const char* lds, Rows<DP>& r) {
  const int lane = threadIdx.x & 63, base = Layout<DP>::at(lane & 31, lane >> 5);
#pragma unroll
  for (int s = 0; s < DP / 16; ++s) r.f[s] = *reinterpret_cast<const bf16x8*>(lds + (base ^ s << 5));
}

}  // namespace
}  // namespace disco
