// Attention over packed sequences, forward and backward, for the towers that make the features of the loss.
//
//   S = scale q k^T (j <= i if causal), lse = log sum exp S, P = exp(S - lse), o = P v
//   dv = P^T do, dP = do v^T, delta = <do, o>, dS = P (dP - delta), dq = scale dS k, dk = scale dS^T q
//
// Three kernels for any lengths, two for short sequences (further down).  All of them keep one side's rows in registers, one row a lane (of 32), and walk the other side's in tiles that a workgroup
// brings into the LDS: forward and for dq 32 queries a wave, the keys are walked; for dk and dv 32 keys a wave, the queries are.  The 32 x 32 products are taken with the walked side as rows, so that a lane holds 16 values of its own
// row's softmax: maxima and sums are in-lane plus one exchange between the wave's halves, and the values, rounded to bf16, are at once the B
// operand of the product that follows (its reduction index may be in any order that both operands share).  That product's A operand is the
// walked tile transposed, which ds_read_b64_tr_b16 reads from the row-major tile.
//
// Two kernels for the backward pass instead of one: each gradient is summed by one wave in a fixed order, in registers, with neither
// atomics nor fp32 copies of dq, for 7 products instead of 5.
//
// Long sequences are bound by the SIMDs' issue: forward, matrix instructions take 45 % of the time and vector instructions 46 %, and with two
// waves a SIMD, which is what the registers allow, they overlap in part; the LDS has no conflicts.  One causal sequence of 8192, 16
// heads of 128 on 8: forward 303 us (905 TFLOP/s of the products below the diagonal), dq 410 (1005), dk and dv 598 (920); a large product by the vendor's
// library reaches 1150 on the same card.  What bounds short ones stands at their kernels.
//
// Scores, statistics and sums are fp32.  P and dS are rounded to bf16 (by at most 2^-8 of each value) for the matrix instruction, whose fp32 form has a
// sixteenth of the rate; in two bf16 parts each they would take one product more forward, of 2, and three more backward, of 7.  The sum of P that
// divides o is taken before that rounding.  delta is taken from o as stored, but for rows of few keys (own_delta).  Against 64 bits o is off by 0.0016 to
// 0.0020 of its norm and the gradients by 0.0022 to 0.0025; computed in fp32 throughout 0.0014 to 0.0017, their own rounding to bf16.
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

struct Args {
  int64_t tokens;
  int32_t sequences, heads, kv_heads, head_dim, causal;
  float scale;
  int64_t q_row, q_head, k_row, k_head, v_row, v_head, o_row, o_head;
  const int32_t* starts;
  const __bf16 *q, *k, *v, *o, *dout;
  __bf16 *out, *dq, *dk, *dv;
  float *lse, *delta;
  int32_t above;                // sequences of up to this many rows are another kernel's
};

// Which tile of T rows of which sequence a workgroup has.  Causal: tile i of queries has i + 1 tiles of keys to walk, the i-th last tile of keys
// i + 1 of queries.
//
// Up to 64 sequences: the tiles with the most to do first, so that the workgroups that take longest are not the last to start.  A lane has a
// sequence; N(k), the number of tiles that are the k-th or a later one of their sequence (that have at least k to do), falls with k, and slot n's tile has the
// largest k with N(k) > n.  (24 documents of 1 to 2048 tokens, 16 heads of 128, forward: 118 us;
// sequence by sequence, a tile and its mirror image together so that all are equal, 138.)
//
// More: sequence s owns the slots from starts[s] / T + s on, at least as many as it has tiles, whatever its start, so the tiles are found with no table
// and no count of them, for at most `sequences` idle workgroups more.  The search is 64 ways wide: two rounds of loads for thousands of sequences.
//
// What is read from `starts` is kept within [0, tokens].
struct Tile { int64_t first; int32_t len, row; };        // the sequence's first row and length, the tile's first row in it
template <int T, bool KEYS>
__device__ __forceinline__ bool find_tile(const Args& a, int slot, Tile& t) {
  const int lane = threadIdx.x & 63, tokens = (int)a.tokens;
  auto start = [&](int s) { const int v = a.starts[s]; return v < 0 ? 0 : v > tokens ? tokens : v; };
  int from, len, index;
  if (a.sequences <= 64) {
    const bool there = lane < a.sequences;
    const int first = there ? start(lane) : 0, mine = there ? start(lane + 1) - first : 0, tiles = mine > 0 ? (mine - 1) / T + 1 : 0;
    auto later = [&](int k) { return __builtin_amdgcn_readfirstlane(wave_reduce(tiles >= k ? tiles - k + 1 : 0, [](int x, int y) { return x + y; })); };
    if (slot >= later(1)) return false;
    int k = 1, over = __builtin_amdgcn_readfirstlane(wave_reduce(tiles, [](int x, int y) { return x > y ? x : y; })) + 1, before = 0;      // N(k) > slot >= N(over) = before
    while (over - k > 1) {
      const int mid = (k + over) / 2, n = later(mid);
      if (n > slot) k = mid;
      else { over = mid; before = n; }
    }
    const uint64_t members = __ballot(tiles >= k);
    const int rank = __builtin_amdgcn_mbcnt_hi((uint32_t)(members >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)members, 0));
    const uint64_t owner = __ballot(tiles >= k && rank == slot - before);
    if (owner == 0) return false;
    const int s = __ffsll((unsigned long long)owner) - 1;
    from = __builtin_amdgcn_readlane(first, s);
    len = __builtin_amdgcn_readlane(mine, s);
    index = k - 1;
  } else {
    int lo = 0, n = a.sequences;
    for (;;) {
      const int step = (n + 63) / 64, s = lo + lane * step;
      const bool below = lane * step < n && start(s) / T + s <= slot;
      const int count = __popcll(__ballot(below));
      if (count == 0) return false;
      const int taken = (count - 1) * step;
      lo += taken;
      n = n - taken < step ? n - taken : step;
      if (step == 1) break;
    }
    lo = __builtin_amdgcn_readfirstlane(lo);
    from = __builtin_amdgcn_readfirstlane(start(lo));
    len = __builtin_amdgcn_readfirstlane(start(lo + 1)) - from;
    index = slot - (from / T + lo);
  }
  // the same in every lane, and known to be
  index = __builtin_amdgcn_readfirstlane(index);
  from = __builtin_amdgcn_readfirstlane(from);
  len = __builtin_amdgcn_readfirstlane(len);
  const int count = (len + T - 1) / T;
  t.first = from;
  t.len = len;
  t.row = (KEYS && a.causal ? count - 1 - index : index) * T;
  return index >= 0 && index < count;
}

// What is left to the kernels that follow those for short sequences, f(tile) for the tiles of T rows of all longer ones dealt to `stride` groups of
// workgroups in turn.  They are launched before it is known that there are any, as few workgroups, and mostly end after one look at the lengths (4.8 us).  300 sequences of 10 to 197, of which a dozen are left, forward and backward: 100 us; with the search of
// find_tile for every tile 113.
template <int T, bool KEYS, class F>
__device__ __forceinline__ void each_rest(const Args& a, int group, int stride, F f) {
  const int lane = threadIdx.x & 63, tokens = (int)a.tokens;
  auto start = [&](int s) { const int v = a.starts[s]; return v < 0 ? 0 : v > tokens ? tokens : v; };
  bool any = false;
  for (int s = threadIdx.x; s < a.sequences; s += blockDim.x) any |= start(s + 1) - start(s) > a.above;
  if (!__syncthreads_or(any)) return;
  int next = group;                                                  // the group's next tile, counted from the first of the sequence at hand
#pragma nounroll
  for (int base = 0; base < a.sequences; base += 64) {
    const bool there = base + lane < a.sequences;
    const int first = there ? start(base + lane) : 0, len = there ? start(base + lane + 1) - first : 0;
#pragma nounroll
    for (uint64_t longer = __ballot(len > a.above); longer; longer &= longer - 1) {
      const int s = __ffsll((unsigned long long)longer) - 1;
      Tile t;
      t.first = __builtin_amdgcn_readlane(first, s);
      t.len = __builtin_amdgcn_readlane(len, s);
      const int count = (t.len - 1) / T + 1;
#pragma nounroll
      for (; next < count; next += stride) {
        t.row = (KEYS && a.causal ? count - 1 - next : next) * T;
        f(t);
      }
      next -= count;
    }
  }
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
// behind them.
constexpr uint32_t NOWHERE = 0xfffffff0u;       // past the end of any buffer
__device__ __forceinline__ __amdgpu_buffer_rsrc_t rows_at(const __bf16* base, int64_t pitch, int rows, int most, int head_dim) {
  const uint64_t v = reinterpret_cast<uint64_t>(base);
  const uint32_t lo = __builtin_amdgcn_readfirstlane((uint32_t)v), hi = __builtin_amdgcn_readfirstlane((uint32_t)(v >> 32));
  const uint32_t n = rows <= 0 ? 0 : rows < most ? rows : most;
  const uint32_t bytes = n ? (n - 1) * (uint32_t)(pitch * 2) + (uint32_t)head_dim * 2 : 0;
  return __builtin_amdgcn_make_buffer_rsrc(reinterpret_cast<void*>((uint64_t)hi << 32 | lo), 0, __builtin_amdgcn_readfirstlane(bytes), 0x00020000);
}
template <int DP, int ROWS, int THREADS>
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
    for (int i = 0; i < N; ++i) v[i] = __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(r, from[i], 0, 0));
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

template <int DP, int WAVES, int SETS>
__device__ __forceinline__ void forward_tile(const Args& a, const Tile& t, int head, char* lds) {
  using S = Shape<DP, WAVES, SETS>;
  const int kv = head / (a.heads / a.kv_heads), lane = threadIdx.x & 63, half = lane >> 5;
  const __bf16* k = a.k + t.first * a.k_row + kv * a.k_head;
  const __bf16* v = a.v + t.first * a.v_row + kv * a.v_head;
  const float c = a.scale * LOG2E;
  Stage<DP, S::WALK, S::THREADS> sk, sv;
  sk.init(a.k_row, a.head_dim);
  sv.init(a.v_row, a.head_dim);
  const int wave = wave_of<WAVES>(), set = set_of<WAVES>(), row = t.row, first = row + 32 * wave, mine = first + (lane & 31);
  sk.fetch(k, a.k_row, t.len, a.head_dim);
  sv.fetch(v, a.v_row, t.len, a.head_dim);
  Forward<DP> f;
  f.q.fetch(a.q + (t.first + mine) * a.q_row + head * a.q_head, mine < t.len, a.head_dim);
#pragma unroll
  for (int m = 0; m < DP / 32; ++m) f.acc[m] = zeros16();
  const int end = a.causal && row + S::OWN < t.len ? row + S::OWN : t.len;          // keys that the workgroup sees
  const int seen = first >= t.len ? 0 : a.causal && first + 32 < t.len ? first + 32 : t.len;      // and this wave
  const int last = a.causal && mine < t.len ? mine : t.len - 1;                     // the lane's last key
  const int whole = a.causal && first < t.len - 1 ? first + 1 : t.len;              // keys before this one need no mask
  sk.put(lds);
  sv.put(lds + S::TILE);
  __syncthreads();
  for (int j = 0, turn = 0; j < end; j += S::WALK, turn ^= 2 * S::TILE) {
    const bool more = j + S::WALK < end;
    if (more) {
      sk.fetch(k + (int64_t)(j + S::WALK) * a.k_row, a.k_row, t.len - j - S::WALK, a.head_dim);
      sv.fetch(v + (int64_t)(j + S::WALK) * a.v_row, a.v_row, t.len - j - S::WALK, a.head_dim);
    }
    const char *lds_k = lds + turn + set * S::SHARE, *lds_v = lds_k + S::TILE;
    const int share = j + set * S::PER;
    if (share < seen) f.template step<S::PER / 32>(lds_k, lds_v, share, share + S::PER > whole, last, c);
    if (more) {
      sk.put(lds + (turn ^ 2 * S::TILE));
      sv.put(lds + (turn ^ 2 * S::TILE) + S::TILE);
    }
    __syncthreads();
  }
  // Sets with references of their own: to the larger of two.  A set that has seen no key has -inf, 0 and zeros.
#pragma unroll
  for (int n = SETS / 2; n >= 1; n /= 2) {
    f32x2* const scalars = reinterpret_cast<f32x2*>(lds + SETS / 2 * WAVES * S::ACC) + (threadIdx.x & 63);
    if (set >= n && set < 2 * n) {
      hand_over<DP>(lds + ((set - n) * WAVES + wave) * S::ACC, f.acc);
      scalars[((set - n) * WAVES + wave) * 64] = f32x2{f.top, f.total};
    }
    __syncthreads();
    if (set < n) {
      const f32x2 other = scalars[(set * WAVES + wave) * 64];
      const float top = fmaxf(f.top, other[0]);
      const float x = f.top == top ? 1.f : __builtin_amdgcn_exp2f((f.top - top) * c), y = other[0] == top ? 1.f : __builtin_amdgcn_exp2f((other[0] - top) * c);
      take_over<DP>(lds + (set * WAVES + wave) * S::ACC, f.acc, x, y);
      f.total = fmaf(f.total, x, other[1] * y);
      f.top = top;
    }
    __syncthreads();
  }
  if (set) return;
  f.total += other_half(f.total);
  const bool there = mine < t.len;
  store_row<DP>(a.out + (t.first + mine) * a.o_row + head * a.o_head, f.acc, 1.f / f.total, a.head_dim, there);
  if (there && half == 0) a.lse[head * a.tokens + t.first + mine] = f.top * a.scale + __builtin_amdgcn_logf(f.total) * LN2;
}

// A workgroup's head.  Workgroups go to the eight dies in turn, each with a cache of its own: heads that share keys to the same die
// (24 documents of 1 to 2048 rows, 16 heads of 128 on 2: 142 MB read from memory for 298, 110 us for 113).
__device__ __forceinline__ int head_of(const Args& a) {
  const int i = blockIdx.x % a.heads;
  return a.heads % 8 ? i : i % 8 * (a.heads / 8) + i / 8;
}
template <int DP, int WAVES, int SETS>
__global__ __launch_bounds__(64 * WAVES * SETS, 2) void k_attention_fwd(Args a) {
  __shared__ __attribute__((aligned(16))) char lds[Shape<DP, WAVES, SETS>::LDS];        // keys and values, two tiles in turn
  Tile t;
  if (find_tile<32 * WAVES, false>(a, blockIdx.x / a.heads, t)) forward_tile<DP, WAVES, SETS>(a, t, head_of(a), lds);
}
template <int DP>
__global__ __launch_bounds__(256, 2) void k_attention_fwd_rest(Args a) {
  __shared__ __attribute__((aligned(16))) char lds[Shape<DP, 4, 1>::LDS];
  each_rest<128, false>(a, blockIdx.x / a.heads, gridDim.x / a.heads, [&](const Tile& t) { forward_tile<DP, 4, 1>(a, t, blockIdx.x % a.heads, lds); });
}

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

// dq, and delta = <do, o> of every row for the kernel of dk and dv, which runs after this one.  Three products a pair of tiles, S and dP with shared addresses.
template <int DP, int WAVES, int SETS>
__device__ __forceinline__ void queries_tile(const Args& a, const Tile& t, int head, char* lds) {
  using S = Shape<DP, WAVES, SETS>;
  const int kv = head / (a.heads / a.kv_heads), lane = threadIdx.x & 63, half = lane >> 5;
  const __bf16* k = a.k + t.first * a.k_row + kv * a.k_head;
  const __bf16* v = a.v + t.first * a.v_row + kv * a.v_head;
  const float c = a.scale * LOG2E;
  Stage<DP, S::WALK, S::THREADS> sk, sv;
  sk.init(a.k_row, a.head_dim);
  sv.init(a.v_row, a.head_dim);
  const int wave = wave_of<WAVES>(), set = set_of<WAVES>(), row = t.row, first = row + 32 * wave, mine = first + (lane & 31);
  const bool there = mine < t.len;
  sk.fetch(k, a.k_row, t.len, a.head_dim);
  sv.fetch(v, a.v_row, t.len, a.head_dim);
  Rows<DP> q, dout;
  q.fetch(a.q + (t.first + mine) * a.q_row + head * a.q_head, there, a.head_dim);
  dout.fetch(a.dout + (t.first + mine) * a.o_row + head * a.o_head, there, a.head_dim);
  float delta = 0.f;
  {
    Rows<DP> o;
    o.fetch(a.o + (t.first + mine) * a.o_row + head * a.o_head, there, a.head_dim);
#pragma unroll
    for (int s = 0; s < DP / 16; ++s)
#pragma unroll
      for (int e = 0; e < 8; ++e) delta = fmaf((float)o.f[s][e], (float)dout.f[s][e], delta);
    delta += other_half(delta);
  }
  const int64_t at = head * a.tokens + t.first + mine;
  const float lse2 = there ? base2(a.lse[at]) : 0.f;
  const int end = a.causal && row + S::OWN < t.len ? row + S::OWN : t.len;
  const int seen = first >= t.len ? 0 : a.causal && first + 32 < t.len ? first + 32 : t.len;
  const int last = a.causal && there ? mine : t.len - 1;
  const int whole = a.causal && first < t.len - 1 ? first + 1 : t.len;
  f32x16 acc[DP / 32];
#pragma unroll
  for (int m = 0; m < DP / 32; ++m) acc[m] = zeros16();
  sk.put(lds);
  sv.put(lds + S::TILE);
  __syncthreads();
  for (int j0 = 0, turn = 0; j0 < end; j0 += S::WALK, turn ^= 2 * S::TILE) {
    const bool more = j0 + S::WALK < end;
    if (more) {
      sk.fetch(k + (int64_t)(j0 + S::WALK) * a.k_row, a.k_row, t.len - j0 - S::WALK, a.head_dim);
      sv.fetch(v + (int64_t)(j0 + S::WALK) * a.v_row, a.v_row, t.len - j0 - S::WALK, a.head_dim);
    }
#pragma unroll
    for (int sub = 0; sub < S::PER; sub += 32) {
      const int j = j0 + set * S::PER + sub;
      if (j >= seen) break;
      const char* lds_k = lds + turn + set * S::SHARE + sub * Layout<DP>::PITCH;
      f32x16 s[2];                                                  // scores, and dP
      matrix_work(true);
      products<DP, 2, S::TILE>(s, lds_k, [&](int n, int i, int) { return n ? dout.f[i] : q.f[i]; });
      matrix_work(false);
      if (j + 32 > whole) {
        int most = last - j - 4 * half;
        asm volatile("" : "+v"(most));
#pragma unroll
        for (int r = 0; r < 16; ++r)
          if (walked(r, 0) > most) s[0][r] = -INFINITY;
      }
#pragma unroll
      for (int r = 0; r < 16; ++r) s[0][r] = __builtin_amdgcn_exp2f(fmaf(s[0][r], c, -lse2));
      if (seen <= 32) delta = own_delta(s[0], s[1]);
#pragma unroll
      for (int r = 0; r < 16; ++r) s[0][r] *= s[1][r] - delta;
      matrix_work(true);
      accumulate<DP, 1, 0>({&acc}, lds_k, {rounded(s[0])});
      matrix_work(false);
    }
    if (more) {
      sk.put(lds + (turn ^ 2 * S::TILE));
      sv.put(lds + (turn ^ 2 * S::TILE) + S::TILE);
    }
    __syncthreads();
  }
  join<DP, WAVES, SETS>(lds, wave, set, acc);
  if (set) return;
  if (there && half == 0) a.delta[at] = delta;
  store_row<DP>(a.dq + (t.first + mine) * a.q_row + head * a.q_head, acc, a.scale, a.head_dim, there);
}

template <int DP, int WAVES, int SETS>
__global__ __launch_bounds__(64 * WAVES * SETS, 2) void k_attention_bwd_q(Args a) {
  __shared__ __attribute__((aligned(16))) char lds[Shape<DP, WAVES, SETS>::LDS];
  Tile t;
  if (find_tile<32 * WAVES, false>(a, blockIdx.x / a.heads, t)) queries_tile<DP, WAVES, SETS>(a, t, head_of(a), lds);
}
template <int DP>
__global__ __launch_bounds__(256, 2) void k_attention_bwd_q_rest(Args a) {
  __shared__ __attribute__((aligned(16))) char lds[Shape<DP, 4, 1>::LDS];
  each_rest<128, false>(a, blockIdx.x / a.heads, gridDim.x / a.heads, [&](const Tile& t) { queries_tile<DP, 4, 1>(a, t, blockIdx.x % a.heads, lds); });
}

// dk and dv: 32 keys a wave; the queries of all heads that share the keys are walked, head by head, 32 rows a step for each set.  Four products a pair of
// tiles; two fifths of a wave's time are waiting, and there is no register left to ask for operands earlier.
template <int DP, int WAVES, int SETS>
struct Keys {
  static constexpr int SUB = 32 * Layout<DP>::PITCH, WALK = 32 * SETS, TILE = SETS * SUB;
  static constexpr int BOTH = 2 * TILE + 2 * WALK * (int)sizeof(float);      // queries, do, lse, delta
  // Wide heads: the accumulators of dk and dv take 2 DP registers a lane, k and v another DP; with v in the LDS two waves fit a SIMD.
  static constexpr bool V_IN_LDS = DP > 64;
  static constexpr int ALL = 2 * BOTH + (V_IN_LDS ? WAVES * SUB : 0);
  static_assert(SETS / 2 * WAVES * DP * 128 <= 2 * BOTH);
};
template <int DP, int WAVES, int SETS>
__device__ __forceinline__ void keys_tile(const Args& a, const Tile& t, int kv, char* lds) {
  using S = Keys<DP, WAVES, SETS>;
  constexpr int SUB = S::SUB, WALK = S::WALK, TILE = S::TILE, BOTH = S::BOTH;
  constexpr bool V_IN_LDS = S::V_IN_LDS;
  char* const lds_v = lds + 2 * BOTH;
  const int group = a.heads / a.kv_heads;
  const int lane = threadIdx.x & 63, half = lane >> 5, wave = wave_of<WAVES>(), set = set_of<WAVES>();
  const float c = a.scale * LOG2E;
  Stage<DP, WALK, 64 * WAVES * SETS> sq, so;
  sq.init(a.q_row, a.head_dim);
  so.init(a.o_row, a.head_dim);
  float next_lse = 0.f, next_delta = 0.f;
  const int row = t.row, first = row + 32 * wave, mine = first + (lane & 31);
  const bool there = mine < t.len;
  const int begin = a.causal ? row : 0;                            // the first walked query
  int head = kv * group, i = begin, next = begin;                  // what is fetched next, and the rows under way
  auto fetch = [&] {
    const int64_t from = t.first + i;
    sq.fetch(a.q + from * a.q_row + head * a.q_head, a.q_row, t.len - i, a.head_dim);
    so.fetch(a.dout + from * a.o_row + head * a.o_head, a.o_row, t.len - i, a.head_dim);
    next = i;
    if (threadIdx.x < WALK) {
      const int64_t at = head * a.tokens + t.first + (i + (int)threadIdx.x < t.len ? i + (int)threadIdx.x : t.len - 1);
      next_lse = a.lse[at];
      next_delta = a.delta[at];
    }
    i += WALK;
    if (i >= t.len) { i = begin; ++head; }
  };
  auto put = [&](char* to) {
    sq.put(to);
    so.put(to + TILE);
    if (threadIdx.x < WALK) {
      // rows past the last: exp2(-inf) = 0
      reinterpret_cast<float*>(to + 2 * TILE)[threadIdx.x] = next + (int)threadIdx.x < t.len ? base2(next_lse) : INFINITY;
      reinterpret_cast<float*>(to + 2 * TILE)[WALK + threadIdx.x] = next_delta;
    }
  };
  fetch();
  char* const own_v = lds_v + SUB * wave;
  Rows<DP> k, v;
  k.fetch(a.k + (t.first + mine) * a.k_row + kv * a.k_head, there, a.head_dim);
  v.fetch(a.v + (t.first + mine) * a.v_row + kv * a.v_head, there, a.head_dim);
  if (V_IN_LDS && set == 0) {
#pragma unroll
    for (int s = 0; s < DP / 16; ++s) *reinterpret_cast<bf16x8*>(own_v + Layout<DP>::at(lane & 31, 2 * s + half)) = v.f[s];
  }
  f32x16 dk[DP / 32], dv[DP / 32];
#pragma unroll
  for (int m = 0; m < DP / 32; ++m) dk[m] = dv[m] = zeros16();
  put(lds);
  __syncthreads();
  int at = begin;                                                  // what is used now
  for (int n = (t.len - begin + WALK - 1) / WALK * group, turn = 0; n > 0; --n, turn ^= 1) {
    const char* const now = lds + turn * BOTH;
    if (n > 1) fetch();
    const int from = at + 32 * set;
    if (first < t.len && from < t.len && !(a.causal && from + 32 <= first)) {
      f32x16 s[2];                                                  // scores, and dP
      matrix_work(true);
      products<DP, 2, TILE>(s, now + set * SUB, [&](int which, int p, int base) {
        if (!which) return k.f[p];
        return V_IN_LDS ? *reinterpret_cast<const bf16x8*>(own_v + (base ^ p << 5)) : v.f[p];
      });
      matrix_work(false);
      if (a.causal && from < first + 31) {
        int least = mine - from - 4 * half;
        asm volatile("" : "+v"(least));
#pragma unroll
        for (int r = 0; r < 16; ++r)
          if (walked(r, 0) < least) s[0][r] = -INFINITY;
      }
      const float* scalars = reinterpret_cast<const float*>(now + 2 * TILE) + 32 * set + 4 * half;
#pragma unroll
      for (int g = 0; g < 4; ++g) {
        const f32x4 l = *reinterpret_cast<const f32x4*>(scalars + 8 * g), d = *reinterpret_cast<const f32x4*>(scalars + WALK + 8 * g);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const int r = 4 * g + e;
          s[0][r] = __builtin_amdgcn_exp2f(fmaf(s[0][r], c, -l[e]));
          s[1][r] = s[0][r] * (s[1][r] - d[e]);
        }
      }
      matrix_work(true);
      accumulate<DP, 2, TILE>({&dk, &dv}, now + set * SUB, {rounded(s[1]), rounded(s[0])});
      matrix_work(false);
    }
    at += WALK;
    if (at >= t.len) at = begin;
    if (n > 1) put(lds + (turn ^ 1) * BOTH);
    __syncthreads();
  }
  join<DP, WAVES, SETS>(lds, wave, set, dk);
  join<DP, WAVES, SETS>(lds, wave, set, dv);
  if (set) return;
  store_row<DP>(a.dk + (t.first + mine) * a.k_row + kv * a.k_head, dk, a.scale, a.head_dim, there);
  store_row<DP>(a.dv + (t.first + mine) * a.v_row + kv * a.v_head, dv, 1.f, a.head_dim, there);
}

template <int DP, int WAVES, int SETS>
__global__ __launch_bounds__(64 * WAVES * SETS, 2) void k_attention_bwd_kv(Args a) {
  __shared__ __attribute__((aligned(16))) char lds[Keys<DP, WAVES, SETS>::ALL];
  Tile t;
  if (find_tile<32 * WAVES, true>(a, blockIdx.x / a.kv_heads, t)) keys_tile<DP, WAVES, SETS>(a, t, blockIdx.x % a.kv_heads, lds);
}
template <int DP>
__global__ __launch_bounds__(256, 2) void k_attention_bwd_kv_rest(Args a) {
  __shared__ __attribute__((aligned(16))) char lds[Keys<DP, 4, 1>::ALL];
  each_rest<128, true>(a, blockIdx.x / a.kv_heads, gridDim.x / a.kv_heads, [&](const Tile& t) { keys_tile<DP, 4, 1>(a, t, blockIdx.x % a.kv_heads, lds); });
}

// ---- Short sequences: a workgroup has all of one, WAVES tiles of 32 rows at most, for one head.  Every row is read from memory once and kept by its
// wave, 16 bytes a lane at a time, which is also how it goes into the LDS for the other waves; there is no walk to be kept supplied, no search for
// the tile, and the backward pass is one kernel: the queries' side first, then the waves put queries and do in the place of keys and values.
//
// A few tiles are bound by memory: 1024 captions of up to 77 tokens, causal, 8 heads of 64, 23 us forward and 47 backward, the rate of a copy.  Many are
// not: 128 x 197 patches, 12 heads of 64, take 41 to 45 (155 MB, 3.4 to 3.8 TB/s) and 113 to 120 (310 MB, 2.6 to 2.7 TB/s), where a workgroup
// reads, computes and stores one behind the other with one more on its compute unit to fill in: backward 1.5 waves a SIMD, a third of their time waiting, vector
// instructions 40 % of the time (S, dP and the exponentials are taken twice), matrix instructions 27 %.  Rows are read a whole tile at a time (by the
// lanes that own them, 32 bytes of each at once, they took 43 for 36 in the backward kernel of captions of up to 64).
template <int DP, int WAVES>
struct Short {
  static constexpr int ROWS = 32 * WAVES, SUB = 32 * Layout<DP>::PITCH, ALL = WAVES * SUB;
};
// The sequence of a workgroup, if it is one of these and the wave has rows of it.  (A wave without rows ends; the barriers do not wait for it.)
template <int WAVES>
__device__ __forceinline__ bool short_sequence(const Args& a, int s, int64_t& first, int& len) {
  const int tokens = (int)a.tokens, x = a.starts[s], y = a.starts[s + 1];
  const int from = x < 0 ? 0 : x > tokens ? tokens : x, to = y < 0 ? 0 : y > tokens ? tokens : y;
  first = __builtin_amdgcn_readfirstlane(from);
  len = __builtin_amdgcn_readfirstlane(to - from);
  return len > 32 * (int)__builtin_amdgcn_readfirstlane(threadIdx.x >> 6) && len <= 32 * WAVES;
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

// Between lanes of a wave that write rows into the LDS and lanes that read them there, either way round: what was issued before this is done before what
// comes after it.  One wave's LDS instructions keep their order by themselves, so this is no instruction; it is what keeps the compiler to it.
__device__ __forceinline__ void wave_exchange() {
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront", "local");
  __builtin_amdgcn_wave_barrier();
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront", "local");
}

template <int DP, int WAVES>
__global__ __launch_bounds__(64 * WAVES, DP <= 64 ? 3 : 2) void k_attention_fwd_short(Args a) {
  using S = Short<DP, WAVES>;
  __shared__ __attribute__((aligned(16))) char lds[2 * S::ALL];
  const int head = blockIdx.x % a.heads, kv = head / (a.heads / a.kv_heads);
  int64_t seq;
  int len;
  if (!short_sequence<WAVES>(a, blockIdx.x / a.heads, seq, len)) return;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63, half = lane >> 5, mine = 32 * wave + (lane & 31);
  const bool there = mine < len;
  Forward<DP> f;
  {
    Stage<DP, 32, 64> q, k, v;
    q.init(a.q_row, a.head_dim);
    k.init(a.k_row, a.head_dim);
    v.init(a.v_row, a.head_dim);
    const int64_t row = seq + 32 * wave;
    const int rows = len - 32 * wave;
    q.fetch(a.q + row * a.q_row + head * a.q_head, a.q_row, rows, a.head_dim);
    k.fetch(a.k + row * a.k_row + kv * a.k_head, a.k_row, rows, a.head_dim);
    v.fetch(a.v + row * a.v_row + kv * a.v_head, a.v_row, rows, a.head_dim);
    char *own = lds + wave * S::SUB;
    q.put(own);
    wave_exchange();
    take_rows<DP>(own, f.q);
    wave_exchange();
    k.put(own);
    v.put(own + S::ALL);
  }
#pragma unroll
  for (int m = 0; m < DP / 32; ++m) f.acc[m] = zeros16();
  const float c = a.scale * LOG2E;
  const int last = a.causal && there ? mine : len - 1, tiles = a.causal ? wave + 1 : (len + 31) / 32;
  __syncthreads();
  for (int t = 0; t < tiles; ++t)
    f.template step<1>(lds + t * S::SUB, lds + S::ALL + t * S::SUB, 32 * t, (a.causal && t == wave) || 32 * t + 32 > len, last, c);
  f.total += other_half(f.total);
  store_row<DP>(a.out + (seq + mine) * a.o_row + head * a.o_head, f.acc, 1.f / f.total, a.head_dim, there);
  if (there && half == 0) a.lse[head * a.tokens + seq + mine] = f.top * a.scale + __builtin_amdgcn_logf(f.total) * LN2;
}

// heads == kv_heads.  Six or eight tiles are two for each wave, the i-th and the i-th last (causal walks then add up to the same in every wave): with half
// the waves two workgroups fit a compute unit, and one computes while the other reads its rows or writes gradients (128 x 197, 12 heads of 64: 114 us
// for 137 with a wave for each tile; 300 causal sequences of 70 to 180, 8 heads: 82 for 80).
template <int DP, int TILES>
struct ShortBwd {
  static constexpr int OWN = DP <= 64 && TILES >= 6 ? 2 : 1, WAVES = TILES / OWN;
};
template <int DP, int TILES>
__global__ __launch_bounds__((64 * ShortBwd<DP, TILES>::WAVES), (DP <= 64 && TILES < 6 ? 3 : 2)) void k_attention_bwd_short(Args a) {
  using S = Short<DP, TILES>;
  constexpr int OWN = ShortBwd<DP, TILES>::OWN;
  __shared__ __attribute__((aligned(16))) char lds[2 * S::ALL];
  __shared__ __attribute__((aligned(16))) float row_lse[S::ROWS], row_delta[S::ROWS];
  const int head = blockIdx.x % a.heads;
  int64_t seq;
  int len;
  if (!short_sequence<TILES>(a, blockIdx.x / a.heads, seq, len)) return;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63, half = lane >> 5;
  const int tiles = (len + 31) / 32;
  const float c = a.scale * LOG2E;
  auto tile_of = [&](int i) { return i ? TILES - 1 - wave : wave; };
  Rows<DP> q[OWN], dout[OWN];
  float lse2[OWN], delta[OWN];
#pragma unroll
  for (int i = 0; i < OWN; ++i) {
    const int tile = tile_of(i), mine = 32 * tile + (lane & 31);
    lse2[i] = mine < len ? base2(a.lse[head * a.tokens + seq + mine]) : INFINITY;      // exp2(-inf) = 0
    delta[i] = 0.f;
    Stage<DP, 32, 64> sq, sk, sv, so, sd;
    sq.init(a.q_row, a.head_dim);
    sk.init(a.k_row, a.head_dim);
    sv.init(a.v_row, a.head_dim);
    so.init(a.o_row, a.head_dim);
    sd.init(a.o_row, a.head_dim);
    const int64_t row = seq + 32 * tile;
    const int rows = len - 32 * tile;
    sq.fetch(a.q + row * a.q_row + head * a.q_head, a.q_row, rows, a.head_dim);
    sd.fetch(a.dout + row * a.o_row + head * a.o_head, a.o_row, rows, a.head_dim);
    so.fetch(a.o + row * a.o_row + head * a.o_head, a.o_row, rows, a.head_dim);
    sk.fetch(a.k + row * a.k_row + head * a.k_head, a.k_row, rows, a.head_dim);
    sv.fetch(a.v + row * a.v_row + head * a.v_head, a.v_row, rows, a.head_dim);
    char* own = lds + tile * S::SUB;
    Rows<DP> o;
    sq.put(own);
    sd.put(own + S::ALL);
    wave_exchange();
    take_rows<DP>(own, q[i]);
    take_rows<DP>(own + S::ALL, dout[i]);
    wave_exchange();
    so.put(own);
    wave_exchange();
    take_rows<DP>(own, o);
    wave_exchange();
#pragma unroll
    for (int s = 0; s < DP / 16; ++s)
#pragma unroll
      for (int e = 0; e < 8; ++e) delta[i] = fmaf((float)o.f[s][e], (float)dout[i].f[s][e], delta[i]);
    delta[i] += other_half(delta[i]);
    sk.put(own);
    sv.put(own + S::ALL);
  }
  __syncthreads();
#pragma unroll
  for (int i = 0; i < OWN; ++i) {
    const int tile = tile_of(i), mine = 32 * tile + (lane & 31);
    if (tile >= tiles) break;
    f32x16 acc[DP / 32];
#pragma unroll
    for (int m = 0; m < DP / 32; ++m) acc[m] = zeros16();
    const int last = a.causal && mine < len ? mine : len - 1, end = a.causal ? tile + 1 : tiles;
    for (int t = 0; t < end; ++t) {
      const char* now = lds + t * S::SUB;
      f32x16 s[2];                                                  // scores, and dP
      products<DP, 2, S::ALL>(s, now, [&](int n, int p, int) { return n ? dout[i].f[p] : q[i].f[p]; });
      if ((a.causal && t == tile) || 32 * t + 32 > len) {
        int most = last - 32 * t - 4 * half;
        asm volatile("" : "+v"(most));
#pragma unroll
        for (int r = 0; r < 16; ++r)
          if (walked(r, 0) > most) s[0][r] = -INFINITY;
      }
#pragma unroll
      for (int r = 0; r < 16; ++r) s[0][r] = __builtin_amdgcn_exp2f(fmaf(s[0][r], c, -lse2[i]));
      if (end == 1) delta[i] = own_delta(s[0], s[1]);
#pragma unroll
      for (int r = 0; r < 16; ++r) s[0][r] *= s[1][r] - delta[i];
      accumulate<DP, 1, 0>({&acc}, now, {rounded(s[0])});
    }
    store_row<DP>(a.dq + (seq + mine) * a.q_row + head * a.q_head, acc, a.scale, a.head_dim, mine < len);
  }
  Rows<DP> k[OWN], v[OWN];
#pragma unroll
  for (int i = 0; i < OWN; ++i) {
    take_rows<DP>(lds + tile_of(i) * S::SUB, k[i]);
    take_rows<DP>(lds + S::ALL + tile_of(i) * S::SUB, v[i]);
  }
  __syncthreads();
#pragma unroll
  for (int i = 0; i < OWN; ++i) {
    const int tile = tile_of(i), mine = 32 * tile + (lane & 31);
    put_rows<DP>(lds + tile * S::SUB, q[i]);
    put_rows<DP>(lds + S::ALL + tile * S::SUB, dout[i]);
    if (half == 0) {
      row_lse[mine] = lse2[i];
      row_delta[mine] = delta[i];
    }
  }
  __syncthreads();
#pragma unroll
  for (int i = 0; i < OWN; ++i) {
    const int tile = tile_of(i), mine = 32 * tile + (lane & 31);
    if (tile >= tiles) break;
    f32x16 dk[DP / 32], dv[DP / 32];
#pragma unroll
    for (int m = 0; m < DP / 32; ++m) dk[m] = dv[m] = zeros16();
    for (int t = a.causal ? tile : 0; t < tiles; ++t) {
      const char* now = lds + t * S::SUB;
      f32x16 s[2];
      products<DP, 2, S::ALL>(s, now, [&](int n, int p, int) { return n ? v[i].f[p] : k[i].f[p]; });
      if (a.causal && t == tile) {
        int least = mine - 32 * t - 4 * half;
        asm volatile("" : "+v"(least));
#pragma unroll
        for (int r = 0; r < 16; ++r)
          if (walked(r, 0) < least) s[0][r] = -INFINITY;
      }
      const float *lse = row_lse + 32 * t + 4 * half, *del = row_delta + 32 * t + 4 * half;
#pragma unroll
      for (int g = 0; g < 4; ++g) {
        const f32x4 l = *reinterpret_cast<const f32x4*>(lse + 8 * g), d = *reinterpret_cast<const f32x4*>(del + 8 * g);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const int r = 4 * g + e;
          s[0][r] = __builtin_amdgcn_exp2f(fmaf(s[0][r], c, -l[e]));
          s[1][r] = s[0][r] * (s[1][r] - d[e]);
        }
      }
      accumulate<DP, 2, S::ALL>({&dk, &dv}, now, {rounded(s[1]), rounded(s[0])});
    }
    store_row<DP>(a.dk + (seq + mine) * a.k_row + head * a.k_head, dk, a.scale, a.head_dim, mine < len);
    store_row<DP>(a.dv + (seq + mine) * a.v_row + head * a.v_head, dv, 1.f, a.head_dim, mine < len);
  }
}

int check(const disco_attention_shape* s) {
  if (!s) return DISCO_ERR_NULL;
  if (s->tokens <= 0 || s->tokens > 0x7fffffff || s->sequences <= 0 || s->sequences > 1 << 24 || s->heads <= 0 || s->kv_heads <= 0 ||
      s->heads > 1 << 16 || s->heads % s->kv_heads != 0 || s->head_dim <= 0 || !(s->scale > 0.f) || !isfinite(s->scale * LOG2E))
    return DISCO_ERR_SHAPE;
  // a launch has less than 2^32 threads: 64 for a tile of 32 rows, up to 512 for a sequence
  if ((s->tokens / 32 + (int64_t)s->sequences * 8) * s->heads >= (int64_t)1 << 26) return DISCO_ERR_SHAPE;
  if (s->dtype != DISCO_BF16 || s->head_dim % 8 != 0 || s->head_dim > 128) return DISCO_ERR_UNSUPPORTED;
  // the rows of a walked tile, 256 at most, are addressed with 32 bits
  for (int64_t v : {s->q_row, s->k_row, s->v_row, s->o_row}) {
    if (v <= 0 || v > (int64_t)1 << 22) return DISCO_ERR_SHAPE;
    if (v % 8 != 0) return DISCO_ERR_UNSUPPORTED;
  }
  for (int64_t v : {s->q_head, s->k_head, s->v_head, s->o_head}) {
    if (v <= 0 || v > (int64_t)1 << 40) return DISCO_ERR_SHAPE;
    if (v % 8 != 0) return DISCO_ERR_UNSUPPORTED;
  }
  return DISCO_OK;
}

bool aligned(const void* p, uintptr_t n) { return (reinterpret_cast<uintptr_t>(p) & (n - 1)) == 0; }

Args args_of(const disco_attention_shape& s, const int32_t* starts) {
  Args a = {};
  a.tokens = s.tokens; a.sequences = s.sequences; a.heads = s.heads; a.kv_heads = s.kv_heads; a.head_dim = s.head_dim; a.causal = s.causal != 0;
  a.scale = s.scale;
  a.q_row = s.q_row; a.q_head = s.q_head; a.k_row = s.k_row; a.k_head = s.k_head;
  a.v_row = s.v_row; a.v_head = s.v_head; a.o_row = s.o_row; a.o_head = s.o_head;
  a.starts = starts;
  return a;
}

constexpr int COMPUTE_UNITS = 256;

// Tiles of 32 rows that the kernels for short sequences take, 0: none.  The lengths are on the device; the mean says what they may be.  2.8 times
// the mean where that is at most the widest: few sequences are longer (of lengths spread evenly over the decades from 4 to 77 the longest is 3.1 times the
// mean), and tiles that are not there cost the rest occupancy.  Forward and backward, 8 heads of 64: 500 sequences of 44, 63 us with 4 tiles, 79 with 6, 84
// without these kernels; 400 of 8 to 120, 59, 72 and 74; 150 of 4 to 77, 23 with 3 tiles, 51 with 2, which leave some.  The widest up to 4/5 of it:
// sequences of one length, as images have (128 x 197, 12 heads: 150 against 220 without).
//
// Short sequences of one length get more tiles than they fill by this, which goes by lengths that are spread.  Kernels forward and backward, heads of 64, tiles
// taken and tiles that they need: 512 x 50 on 12 heads 134 us with 6, 108 with 2; 1024 x 77, causal, on 8 heads 310 with 8, 270 with 3; 512 x 77 on 8 heads 151
// and 122; 512 x 96 on 12 heads 265 and 228; 256 x 128 on 12 heads 167 with 8, 143 with 4.  Only the longest length would tell, which the host does not have.
//
// None for few sequences of narrow heads that are short or, as causal ones mostly are, of different lengths: these kernels are five launches for three, and what
// they leave then takes longest.  Forward and backward, with them and without: 150 of 4 to 77 on 8 heads, 32 and 25 us where the host is the slower, 23 and
// 23 in a graph; 1000 of them 76 and 108; 40 of 1 to 1024 on 16 heads 181 and 111; 100 of 20 to 400 on 8 heads 95 and 82; but 12 images of 197 on 12 heads 37 and
// 50.  Batches of up to 96 rows leave nothing and are two launches (2 of 40: 10 and 14).
int short_tiles(const disco_attention_shape& s, bool backward) {
  if ((backward && s.heads != s.kv_heads) || s.sequences > 8192) return 0;
  const int widest = s.head_dim <= 64 ? 8 : 4;
  if (s.head_dim <= 64 && (s.causal || s.tokens <= (int64_t)s.sequences * 64) && s.tokens > 96 && (int64_t)s.sequences * s.heads <= 5 * COMPUTE_UNITS) return 0;
  for (int w : {2, 3, 4, 6})
    if (w <= widest && s.tokens * 28 <= (int64_t)s.sequences * (32 * w * 10)) return w;
  return s.tokens * 5 <= (int64_t)s.sequences * (32 * widest * 4) ? widest : 0;
}
template <int DP, class F>
void with_short(int tiles, F f) {
  if (tiles == 2) f(std::integral_constant<int, 2>());
  else if (tiles == 3) f(std::integral_constant<int, 3>());
  else if (tiles == 4) f(std::integral_constant<int, 4>());
  else if constexpr (DP <= 64) {
    if (tiles == 6) f(std::integral_constant<int, 6>());
    else f(std::integral_constant<int, 8>());
  }
}
// The workgroups of a kernel that takes what is left, whole slots: what the chip holds at once, as there is mostly nothing and they only end (1024 captions of
// up to 77 tokens, forward and backward: 96 us a pass; with four times as many workgroups 102).
unsigned rest_grid(const Args& a, int heads) {
  const int64_t groups = (2 * COMPUTE_UNITS + heads - 1) / heads, tiles = a.tokens / 128 + a.sequences;
  return (unsigned)((groups < tiles ? groups : tiles) * heads);
}
bool launched() { return hipGetLastError() == hipSuccess; }        // once a launch: asking clears the error

// Sets of waves that share rows where there are few: as many as their tiles leave room for in the LDS.
template <int DP>
constexpr int many_sets() { return DP <= 64 ? 8 : 4; }
// Whether tiles of 32 rows with many sets beat tiles of 128 with one: in steps of a walk (the two kinds' steps take about as long), for the mean length,
// as many times over as a compute unit has workgroups to run, one of the former or two of the latter at once; a workgroup's other work is worth 3 or 2
// steps.  Measured, forward, dq and dk / dv together, many sets / one: one causal sequence on 8 heads, width 64: 1024 rows 39 / 70 us, 2048 80 / 125, 4096
// 229 / 239, 8192 728 / 539; width 128: 1024 68 / 99, 2048 143 / 179, 4096 446 / 352; 4 sequences of 300 (not causal), width 128: 77 / 49.
template <int DP>
bool few(const Args& a, int heads) {
  const double walk = (double)a.tokens / a.sequences * (a.heads / heads);
  double narrow = (double)(a.tokens / 32 + a.sequences) * heads / COMPUTE_UNITS, wide = (double)(a.tokens / 128 + a.sequences) * heads / (2 * COMPUTE_UNITS);
  const double share = a.causal && narrow > 1 ? 0.5 : 1.0;             // causal walks are half as long on average, the longest as long
  narrow = narrow > 1 ? narrow : 1;
  wide = wide > 1 ? wide : 1;
  return narrow * (share * walk / (32 * many_sets<DP>()) + 3) < wide * (walk / 64 + 2);
}

// Two sets of waves for tiles of 128 rows, where there are at most 3 halves (causal, with half the work: 3) of them for a compute unit: dk and dv of one sequence of 8192, causal,
// head width 128, 16 heads on 8 of keys: 600 us against 928 with one set; on 16 of keys, two workgroups of one set a unit, 640 against 585.  Forward, 12 causal
// sequences of 1 to 2048, 16 heads of 128: 43 against 52, 24 of them 143 against 112; 16 of 1 to 4096, 8 heads of 64: 57 against 74.
template <int WAVES>
bool two_sets(const Args& a, int heads) { return WAVES > 1 && a.tokens / (32 * WAVES) * heads / (a.causal ? 2 : 1) <= COMPUTE_UNITS * 3 / 2; }

template <int DP, int WAVES>
bool forward(Args a, int tiles, hipStream_t st) {
  if (!tiles && WAVES > 1 && few<DP>(a, a.heads)) {
    constexpr int SETS = many_sets<DP>();
    const int64_t slots = a.tokens / 32 + a.sequences;
    k_attention_fwd<DP, 1, SETS><<<(unsigned)(slots * a.heads), 64 * SETS, 0, st>>>(a);
    return launched();
  }
  if (!tiles) {
    const int64_t slots = a.tokens / (32 * WAVES) + a.sequences;
    if (two_sets<WAVES>(a, a.heads)) k_attention_fwd<DP, WAVES, WAVES == 1 ? 1 : 2><<<(unsigned)(slots * a.heads), 128 * WAVES, 0, st>>>(a);
    else k_attention_fwd<DP, WAVES, 1><<<(unsigned)(slots * a.heads), 64 * WAVES, 0, st>>>(a);
    return launched();
  }
  a.above = 32 * tiles;
  with_short<DP>(tiles, [&](auto w) { k_attention_fwd_short<DP, w()><<<(unsigned)(a.sequences * a.heads), 64 * w(), 0, st>>>(a); });
  if (!launched()) return false;
  if (a.tokens <= a.above) return true;
  k_attention_fwd_rest<DP><<<rest_grid(a, a.heads), 256, 0, st>>>(a);
  return launched();
}
template <int DP, int WAVES>
bool backward(Args a, int tiles, hipStream_t st) {
  constexpr int SETS = many_sets<DP>();
  if (!tiles) {
    const int64_t wide = a.tokens / (32 * WAVES) + a.sequences, narrow = a.tokens / 32 + a.sequences;
    if (WAVES > 1 && few<DP>(a, a.heads)) {
      k_attention_bwd_q<DP, 1, SETS><<<(unsigned)(narrow * a.heads), 64 * SETS, 0, st>>>(a);
    } else if (two_sets<WAVES>(a, a.heads)) {
      k_attention_bwd_q<DP, WAVES, WAVES == 1 ? 1 : 2><<<(unsigned)(wide * a.heads), 128 * WAVES, 0, st>>>(a);
    } else {
      k_attention_bwd_q<DP, WAVES, 1><<<(unsigned)(wide * a.heads), 64 * WAVES, 0, st>>>(a);
    }
    if (!launched()) return false;
    if (WAVES > 1 && few<DP>(a, a.kv_heads)) {
      k_attention_bwd_kv<DP, 1, SETS><<<(unsigned)(narrow * a.kv_heads), 64 * SETS, 0, st>>>(a);
    } else {
      if (two_sets<WAVES>(a, a.kv_heads)) k_attention_bwd_kv<DP, WAVES, WAVES == 1 ? 1 : 2><<<(unsigned)(wide * a.kv_heads), 128 * WAVES, 0, st>>>(a);
      else k_attention_bwd_kv<DP, WAVES, 1><<<(unsigned)(wide * a.kv_heads), 64 * WAVES, 0, st>>>(a);
    }
    return launched();
  }
  a.above = 32 * tiles;
  with_short<DP>(tiles, [&](auto w) { k_attention_bwd_short<DP, w()><<<(unsigned)(a.sequences * a.heads), 64 * ShortBwd<DP, w()>::WAVES, 0, st>>>(a); });
  if (!launched()) return false;
  if (a.tokens <= a.above) return true;
  k_attention_bwd_q_rest<DP><<<rest_grid(a, a.heads), 256, 0, st>>>(a);
  if (!launched()) return false;
  k_attention_bwd_kv_rest<DP><<<rest_grid(a, a.kv_heads), 256, 0, st>>>(a);
  return launched();
}

// f with the head's width rounded up to a multiple of 32 and the waves of a workgroup as constants
template <class F>
int dispatch(const disco_attention_shape& s, int tiles, F f) {
  const int dp = (s.head_dim + 31) / 32;
  // Tiles of 32 or 128 rows.  Shared keys, 8 heads on 2, dq and dk / dv, one wave / four: 800 sequences of 30, width 64: 46 / 107 us; 200 of 150: 80 / 104;
  // 200 of 90, width 128: 119 / 97.
  const int waves = tiles || s.tokens > (int64_t)(dp <= 2 ? 160 : 64) * s.sequences ? 4 : 1;
#define DISCO_DP(N) \
  if (dp == N) return (waves == 1 ? f(std::integral_constant<int, 32 * N>(), std::integral_constant<int, 1>()) \
                                  : f(std::integral_constant<int, 32 * N>(), std::integral_constant<int, 4>())) ? DISCO_OK : DISCO_ERR_HIP
  DISCO_DP(1);
  DISCO_DP(2);
  DISCO_DP(3);
  DISCO_DP(4);
#undef DISCO_DP
  return DISCO_ERR_UNSUPPORTED;
}

}  // namespace
}  // namespace disco

using namespace disco;

extern "C" size_t disco_attention_workspace_bytes(const disco_attention_shape* shape) {
  if (check(shape) != DISCO_OK) return 0;
  return align_up((size_t)shape->heads * (size_t)shape->tokens * sizeof(float));
}

extern "C" int disco_attention_fwd(const disco_attention_shape* shape, const int32_t* starts, const void* q, const void* k, const void* v, void* o,
                                   float* lse, void* hip_stream) {
  if (!shape || !starts || !q || !k || !v || !o || !lse) return DISCO_ERR_NULL;
  if (const int st = check(shape)) return st;
  if (!aligned(starts, 4) || !aligned(q, 16) || !aligned(k, 16) || !aligned(v, 16) || !aligned(o, 16) || !aligned(lse, 4)) return DISCO_ERR_UNSUPPORTED;
  Args a = args_of(*shape, starts);
  a.q = static_cast<const __bf16*>(q); a.k = static_cast<const __bf16*>(k); a.v = static_cast<const __bf16*>(v);
  a.out = static_cast<__bf16*>(o); a.lse = lse;
  const int tiles = short_tiles(*shape, false);
  return dispatch(*shape, tiles, [&](auto dp, auto waves) { return forward<dp(), waves()>(a, tiles, static_cast<hipStream_t>(hip_stream)); });
}

extern "C" int disco_attention_bwd(const disco_attention_shape* shape, const int32_t* starts, const void* q, const void* k, const void* v,
                                   const void* o, const float* lse, const void* dout, void* dq, void* dk, void* dv, void* workspace,
                                   size_t workspace_bytes, void* hip_stream) {
  if (!shape || !starts || !q || !k || !v || !o || !lse || !dout || !dq || !dk || !dv) return DISCO_ERR_NULL;
  if (const int st = check(shape)) return st;
  if (!aligned(starts, 4) || !aligned(lse, 4)) return DISCO_ERR_UNSUPPORTED;
  for (const void* p : {q, k, v, o, dout, static_cast<const void*>(dq), static_cast<const void*>(dk), static_cast<const void*>(dv)})
    if (!aligned(p, 16)) return DISCO_ERR_UNSUPPORTED;
  if (!workspace || !aligned(workspace, 256) || workspace_bytes < disco_attention_workspace_bytes(shape)) return DISCO_ERR_WORKSPACE;
  Args a = args_of(*shape, starts);
  a.q = static_cast<const __bf16*>(q); a.k = static_cast<const __bf16*>(k); a.v = static_cast<const __bf16*>(v);
  a.o = static_cast<const __bf16*>(o); a.dout = static_cast<const __bf16*>(dout);
  a.dq = static_cast<__bf16*>(dq); a.dk = static_cast<__bf16*>(dk); a.dv = static_cast<__bf16*>(dv);
  a.lse = const_cast<float*>(lse); a.delta = static_cast<float*>(workspace);
  const int tiles = short_tiles(*shape, true);
  return dispatch(*shape, tiles, [&](auto dp, auto waves) { return backward<dp(), waves()>(a, tiles, static_cast<hipStream_t>(hip_stream)); });
}
