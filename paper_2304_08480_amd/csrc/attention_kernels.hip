// Attention over packed sequences, forward and backward, for the towers that make the features of the loss.
//
//   S = scale q k^T (j <= i if causal), lse = log sum exp S, P = exp(S - lse), o = P v
//   dv = P^T do, dP = do v^T, delta = <do, o>, dS = P (dP - delta), dq = scale dS k, dk = scale dS^T q
//
// All three kernels keep one side's rows in registers, one row a lane (of 32), and walk the other side's in tiles that a workgroup
// brings into the LDS: the forward kernel and the one of dq keep 32 queries a wave and walk the keys, the one of dk and dv keeps 32
// keys a wave and walks the queries.  The 32 x 32 products are taken with the walked side as rows, so that a lane holds 16 values of its own
// row's softmax: maxima and sums are in-lane plus one exchange between the wave's halves, and the values, rounded to bf16, are at once the B
// operand of the product that follows (its reduction index may be in any order that both operands share).  That product's A operand is the
// walked tile transposed, which ds_read_b64_tr_b16 reads from the row-major tile.
//
// Two kernels for the backward pass instead of one: each gradient is summed by one wave in a fixed order, in registers, with neither
// atomics nor fp32 copies of dq, for 7 products instead of 5.
//
// Scores, statistics and sums are fp32.  P and dS are rounded to bf16 (by at most 2^-8 of each value) for the matrix instruction; the sum of P that
// divides o is taken before that rounding.
#include "common.h"

#include <math.h>

namespace disco {
namespace {

typedef __attribute__((ext_vector_type(8))) __bf16 bf16x8;
typedef __attribute__((ext_vector_type(4))) __bf16 bf16x4;
typedef __attribute__((ext_vector_type(16))) float f32x16;
typedef __attribute__((ext_vector_type(4))) float f32x4;
typedef __attribute__((ext_vector_type(4))) uint32_t u32x4;
typedef __attribute__((address_space(3))) bf16x4* lds_bf16x4;

constexpr float LOG2E = 1.4426950408889634f, LN2 = 0.6931471805599453f;

struct Args {
  int64_t tokens;
  int32_t sequences, heads, kv_heads, head_dim, causal;
  float scale;
  int64_t q_row, q_head, k_row, k_head, v_row, v_head, o_row, o_head;
  const int32_t* starts;
  const __bf16 *q, *k, *v, *o, *dout;
  __bf16 *out, *dq, *dk, *dv;
  float *lse, *delta;
  int32_t slots;
};

// Which tile of T rows of which sequence a workgroup has.  Sequence s owns the slots from starts[s] / T + s on: at least as many as it has
// tiles, whatever its start, so the tiles are found with no table and no count of them, for at most `sequences` idle workgroups more.  The
// search is 64 ways wide: two rounds of loads for thousands of sequences.  What it reads is kept within [0, tokens].
struct Tile { int64_t first; int32_t len, row; };        // the sequence's first row and length, the tile's first row in it
template <int T>
__device__ __forceinline__ bool find_tile(const Args& a, int slot, Tile& t) {
  const int lane = threadIdx.x & 63, tokens = (int)a.tokens;
  auto start = [&](int s) { const int v = a.starts[s]; return v < 0 ? 0 : v > tokens ? tokens : v; };
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
  const int from = start(lo), to = start(lo + 1);
  t.first = __builtin_amdgcn_readfirstlane(from);
  t.len = __builtin_amdgcn_readfirstlane(to - from);
  t.row = (slot - (from / T + lo)) * T;
  t.row = __builtin_amdgcn_readfirstlane(t.row);
  return t.row < t.len;
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
// past `rows` and pieces past the head's width are zeros: they meet zeros or masked values, never what lies behind them.
template <int DP, int ROWS, int THREADS>
struct Stage {
  using L = Layout<DP>;
  static constexpr int ALL = ROWS * L::PIECES, N = (ALL + THREADS - 1) / THREADS;
  u32x4 v[N];
  __device__ __forceinline__ void fetch(const __bf16* base, int64_t pitch, int rows, int head_dim) {
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int id = threadIdx.x + i * THREADS, row = id / L::PIECES, piece = id % L::PIECES;
      v[i] = u32x4{0, 0, 0, 0};
      if (row < rows && row < ROWS && piece * 8 < head_dim) v[i] = *reinterpret_cast<const u32x4*>(base + row * pitch + piece * 8);
    }
  }
  __device__ __forceinline__ void put(char* lds) const {
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int id = threadIdx.x + i * THREADS;
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

// 32 walked rows from `row0` on times the lanes' rows: element r of a lane is walked row row0 + 8 (r / 4) + 4 half + r % 4.
template <int DP>
__device__ __forceinline__ f32x16 products(const char* lds, int row0, const Rows<DP>& b) {
  using L = Layout<DP>;
  const int lane = threadIdx.x & 63, row = row0 + (lane & 31), half = lane >> 5;
  f32x16 c = zeros16();
#pragma unroll
  for (int s = 0; s < DP / 16; ++s) c = mfma(*reinterpret_cast<const bf16x8*>(lds + L::at(row, 2 * s + half)), b.f[s], c);
  return c;
}
__device__ __forceinline__ int walked(int r, int half) { return 8 * (r >> 2) + 4 * half + (r & 3); }

// acc[m] += (channels 32 m .. of the 32 walked rows, transposed) x (p: the lanes' values for those rows, in the order of products())
template <int DP>
__device__ __forceinline__ void accumulate(f32x16 (&acc)[DP / 32], const char* lds, int row0, const f32x16& p) {
  using L = Layout<DP>;
  const int lane = threadIdx.x & 63, half = lane >> 5, in16 = lane & 15, high = lane >> 4 & 1;
#pragma unroll
  for (int j = 0; j < 2; ++j) {
    bf16x8 b;
#pragma unroll
    for (int e = 0; e < 8; ++e) b[e] = (__bf16)p[8 * j + e];
    const int row = row0 + 16 * j + 4 * half + (in16 >> 2);
#pragma unroll
    for (int m = 0; m < DP / 32; ++m) {
      const int piece = 4 * m + 2 * high + ((in16 & 3) >> 1), byte = 8 * (in16 & 1);
      const bf16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((lds_bf16x4)(lds + L::at(row, piece) + byte));
      const bf16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((lds_bf16x4)(lds + L::at(row + 8, piece) + byte));
      acc[m] = mfma(__builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7), b, acc[m]);
    }
  }
}

// A lane's row of an accumulated product, times f, as bf16: 4 consecutive channels a store.
template <int DP>
__device__ __forceinline__ void store_row(__bf16* row, const f32x16 (&acc)[DP / 32], float f, int head_dim) {
  const int half = (threadIdx.x & 63) >> 5;
#pragma unroll
  for (int m = 0; m < DP / 32; ++m)
#pragma unroll
    for (int g = 0; g < 4; ++g) {
      const int c = 32 * m + 8 * g + 4 * half;
      if (c < head_dim) {
        bf16x4 w;
#pragma unroll
        for (int e = 0; e < 4; ++e) w[e] = (__bf16)(acc[m][4 * g + e] * f);
        *reinterpret_cast<bf16x4*>(row + c) = w;
      }
    }
}

__device__ __forceinline__ float other_half(float v) { return __shfl_xor(v, 32); }

template <int DP, int WAVES>
struct Shape {
  static constexpr int THREADS = 64 * WAVES, OWN = 32 * WAVES;      // rows of the side in registers
  static constexpr int WALK = WAVES == 1 ? 32 : 64;                 // rows of a walked tile
  static constexpr int TILE = WALK * Layout<DP>::PITCH;
};

template <int DP, int WAVES>
__global__ __launch_bounds__(64 * WAVES) void k_attention_fwd(Args a) {
  using S = Shape<DP, WAVES>;
  __shared__ __attribute__((aligned(16))) char lds_k[S::TILE];
  __shared__ __attribute__((aligned(16))) char lds_v[S::TILE];
  const int head = blockIdx.x % a.heads;
  Tile t;
  if (!find_tile<S::OWN>(a, a.slots - 1 - (int)(blockIdx.x / a.heads), t)) return;
  const int kv = head / (a.heads / a.kv_heads), lane = threadIdx.x & 63, half = lane >> 5;
  const int first = t.row + 32 * (int)__builtin_amdgcn_readfirstlane(threadIdx.x >> 6), mine = first + (lane & 31);
  Rows<DP> q;
  q.fetch(a.q + (t.first + mine) * a.q_row + head * a.q_head, mine < t.len, a.head_dim);
  const __bf16* k = a.k + t.first * a.k_row + kv * a.k_head;
  const __bf16* v = a.v + t.first * a.v_row + kv * a.v_head;
  const int end = a.causal && t.row + S::OWN < t.len ? t.row + S::OWN : t.len;      // keys that the workgroup sees
  const int seen = a.causal && first + 32 < t.len ? first + 32 : t.len;             // and this wave
  const int last = a.causal && mine < t.len ? mine : t.len - 1;                     // the lane's last key
  const float c = a.scale * LOG2E;
  float top = -INFINITY, total = 0.f;
  f32x16 acc[DP / 32];
#pragma unroll
  for (int m = 0; m < DP / 32; ++m) acc[m] = zeros16();
  Stage<DP, S::WALK, S::THREADS> sk, sv;
  sk.fetch(k, a.k_row, t.len, a.head_dim);
  sv.fetch(v, a.v_row, t.len, a.head_dim);
  for (int j0 = 0; j0 < end; j0 += S::WALK) {
    __syncthreads();
    sk.put(lds_k);
    sv.put(lds_v);
    __syncthreads();
    if (j0 + S::WALK < end) {
      sk.fetch(k + (int64_t)(j0 + S::WALK) * a.k_row, a.k_row, t.len - j0 - S::WALK, a.head_dim);
      sv.fetch(v + (int64_t)(j0 + S::WALK) * a.v_row, a.v_row, t.len - j0 - S::WALK, a.head_dim);
    }
#pragma unroll
    for (int sub = 0; sub < S::WALK; sub += 32) {
      const int j = j0 + sub;
      if (j >= seen || first >= t.len) break;
      f32x16 s = products<DP>(lds_k, sub, q);
      if (j + 31 > first || j + 31 >= t.len) {
#pragma unroll
        for (int r = 0; r < 16; ++r)
          if (j + walked(r, half) > last) s[r] = -INFINITY;
      }
      float m = s[0];
#pragma unroll
      for (int r = 1; r < 16; ++r) m = fmaxf(m, s[r]);
      m = fmaxf(top, fmaxf(m, other_half(m)));
      const float fade = __builtin_amdgcn_exp2f((top - m) * c), ref = m * c;
      top = m;
      float sum = 0.f;
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        s[r] = __builtin_amdgcn_exp2f(fmaf(s[r], c, -ref));
        sum += s[r];
      }
      total = fmaf(total, fade, sum);
#pragma unroll
      for (int m2 = 0; m2 < DP / 32; ++m2) acc[m2] *= fade;
      accumulate<DP>(acc, lds_v, sub, s);
    }
  }
  total += other_half(total);
  if (mine < t.len) {
    store_row<DP>(a.out + (t.first + mine) * a.o_row + head * a.o_head, acc, 1.f / total, a.head_dim);
    if (half == 0) a.lse[head * a.tokens + t.first + mine] = top * a.scale + __builtin_amdgcn_logf(total) * LN2;
  }
}

// dq, and delta = <do, o> of every row for the kernel of dk and dv, which runs after this one.
template <int DP, int WAVES>
__global__ __launch_bounds__(64 * WAVES) void k_attention_bwd_q(Args a) {
  using S = Shape<DP, WAVES>;
  __shared__ __attribute__((aligned(16))) char lds_k[S::TILE];
  __shared__ __attribute__((aligned(16))) char lds_v[S::TILE];
  const int head = blockIdx.x % a.heads;
  Tile t;
  if (!find_tile<S::OWN>(a, a.slots - 1 - (int)(blockIdx.x / a.heads), t)) return;
  const int kv = head / (a.heads / a.kv_heads), lane = threadIdx.x & 63, half = lane >> 5;
  const int first = t.row + 32 * (int)__builtin_amdgcn_readfirstlane(threadIdx.x >> 6), mine = first + (lane & 31);
  const bool there = mine < t.len;
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
  if (there && half == 0) a.delta[at] = delta;
  const float lse2 = there ? a.lse[at] * LOG2E : 0.f;
  const __bf16* k = a.k + t.first * a.k_row + kv * a.k_head;
  const __bf16* v = a.v + t.first * a.v_row + kv * a.v_head;
  const int end = a.causal && t.row + S::OWN < t.len ? t.row + S::OWN : t.len;
  const int seen = a.causal && first + 32 < t.len ? first + 32 : t.len;
  const int last = a.causal && mine < t.len ? mine : t.len - 1;
  const float c = a.scale * LOG2E;
  f32x16 acc[DP / 32];
#pragma unroll
  for (int m = 0; m < DP / 32; ++m) acc[m] = zeros16();
  Stage<DP, S::WALK, S::THREADS> sk, sv;
  sk.fetch(k, a.k_row, t.len, a.head_dim);
  sv.fetch(v, a.v_row, t.len, a.head_dim);
  for (int j0 = 0; j0 < end; j0 += S::WALK) {
    __syncthreads();
    sk.put(lds_k);
    sv.put(lds_v);
    __syncthreads();
    if (j0 + S::WALK < end) {
      sk.fetch(k + (int64_t)(j0 + S::WALK) * a.k_row, a.k_row, t.len - j0 - S::WALK, a.head_dim);
      sv.fetch(v + (int64_t)(j0 + S::WALK) * a.v_row, a.v_row, t.len - j0 - S::WALK, a.head_dim);
    }
#pragma unroll
    for (int sub = 0; sub < S::WALK; sub += 32) {
      const int j = j0 + sub;
      if (j >= seen || first >= t.len) break;
      f32x16 s = products<DP>(lds_k, sub, q);
      const f32x16 dp = products<DP>(lds_v, sub, dout);
      const bool edge = j + 31 > first || j + 31 >= t.len;
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        const float p = __builtin_amdgcn_exp2f(fmaf(s[r], c, -lse2));
        s[r] = edge && j + walked(r, half) > last ? 0.f : p * (dp[r] - delta);
      }
      accumulate<DP>(acc, lds_k, sub, s);
    }
  }
  if (there) store_row<DP>(a.dq + (t.first + mine) * a.q_row + head * a.q_head, acc, a.scale, a.head_dim);
}

// dk and dv: 32 keys a wave; the queries of all heads that share the keys are walked, head by head.
template <int DP, int WAVES>
__global__ __launch_bounds__(64 * WAVES) void k_attention_bwd_kv(Args a) {
  using S = Shape<DP, WAVES>;
  constexpr int WALK = 32;
  __shared__ __attribute__((aligned(16))) char lds_q[WALK * Layout<DP>::PITCH];
  __shared__ __attribute__((aligned(16))) char lds_o[WALK * Layout<DP>::PITCH];
  __shared__ __attribute__((aligned(16))) float row_lse[WALK], row_delta[WALK];
  const int kv = blockIdx.x % a.kv_heads, group = a.heads / a.kv_heads;
  Tile t;
  if (!find_tile<S::OWN>(a, (int)(blockIdx.x / a.kv_heads), t)) return;
  const int lane = threadIdx.x & 63, half = lane >> 5;
  const int first = t.row + 32 * (int)__builtin_amdgcn_readfirstlane(threadIdx.x >> 6), mine = first + (lane & 31);
  const bool there = mine < t.len;
  Rows<DP> k, v;
  k.fetch(a.k + (t.first + mine) * a.k_row + kv * a.k_head, there, a.head_dim);
  v.fetch(a.v + (t.first + mine) * a.v_row + kv * a.v_head, there, a.head_dim);
  const float c = a.scale * LOG2E;
  const int begin = a.causal ? t.row / WALK * WALK : 0;            // the first walked query that sees a key of the tile
  const int tiles = (t.len - begin + WALK - 1) / WALK, all = tiles * group;
  f32x16 dk[DP / 32], dv[DP / 32];
#pragma unroll
  for (int m = 0; m < DP / 32; ++m) dk[m] = dv[m] = zeros16();
  Stage<DP, WALK, S::THREADS> sq, so;
  float next_lse = 0.f, next_delta = 0.f;
  auto fetch = [&](int n) {
    const int head = kv * group + n / tiles, i0 = begin + n % tiles * WALK;
    const int64_t row = t.first + i0;
    sq.fetch(a.q + row * a.q_row + head * a.q_head, a.q_row, t.len - i0, a.head_dim);
    so.fetch(a.dout + row * a.o_row + head * a.o_head, a.o_row, t.len - i0, a.head_dim);
    if (threadIdx.x < WALK) {
      // rows past the last: exp2(-inf) = 0
      const bool row_there = i0 + (int)threadIdx.x < t.len;
      const int64_t at = head * a.tokens + row + threadIdx.x;
      next_lse = row_there ? a.lse[at] * LOG2E : INFINITY;
      next_delta = row_there ? a.delta[at] : 0.f;
    }
  };
  fetch(0);
  for (int n = 0; n < all; ++n) {
    const int i = begin + n % tiles * WALK;
    __syncthreads();
    sq.put(lds_q);
    so.put(lds_o);
    if (threadIdx.x < WALK) {
      row_lse[threadIdx.x] = next_lse;
      row_delta[threadIdx.x] = next_delta;
    }
    __syncthreads();
    if (n + 1 < all) fetch(n + 1);
    if (first >= t.len || (a.causal && i + WALK <= first)) continue;
    f32x16 s = products<DP>(lds_q, 0, k);
    f32x16 dp = products<DP>(lds_o, 0, v);
    const bool edge = a.causal && i < first + 31;
#pragma unroll
    for (int g = 0; g < 4; ++g) {
      const f32x4 l = *reinterpret_cast<const f32x4*>(row_lse + 8 * g + 4 * half), d = *reinterpret_cast<const f32x4*>(row_delta + 8 * g + 4 * half);
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const int r = 4 * g + e;
        const float p = edge && i + walked(r, half) < mine ? 0.f : __builtin_amdgcn_exp2f(fmaf(s[r], c, -l[e]));
        dp[r] = edge && i + walked(r, half) < mine ? 0.f : p * (dp[r] - d[e]);
        s[r] = p;
      }
    }
    accumulate<DP>(dv, lds_o, 0, s);
    accumulate<DP>(dk, lds_q, 0, dp);
  }
  if (there) {
    store_row<DP>(a.dk + (t.first + mine) * a.k_row + kv * a.k_head, dk, a.scale, a.head_dim);
    store_row<DP>(a.dv + (t.first + mine) * a.v_row + kv * a.v_head, dv, 1.f, a.head_dim);
  }
}

int check(const disco_attention_shape* s) {
  if (!s) return DISCO_ERR_NULL;
  if (s->tokens <= 0 || s->tokens > 0x7fffffff || s->sequences <= 0 || s->sequences > 1 << 24 || s->heads <= 0 || s->kv_heads <= 0 ||
      s->heads > 1 << 16 || s->heads % s->kv_heads != 0 || s->head_dim <= 0 || !(s->scale > 0.f) || !isfinite(s->scale))
    return DISCO_ERR_SHAPE;
  // what one launch of 32-row tiles has workgroups for
  if ((s->tokens / 32 + s->sequences) * s->heads > 0x7fffffff) return DISCO_ERR_SHAPE;
  if (s->dtype != DISCO_BF16 || s->head_dim % 8 != 0 || s->head_dim > 128) return DISCO_ERR_UNSUPPORTED;
  const int64_t strides[] = {s->q_row, s->q_head, s->k_row, s->k_head, s->v_row, s->v_head, s->o_row, s->o_head};
  for (int64_t v : strides) {
    if (v <= 0 || v > (int64_t)1 << 31) return DISCO_ERR_SHAPE;
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

int waves_of(const disco_attention_shape& s) { return s.tokens <= (int64_t)96 * s.sequences ? 1 : 4; }

template <int DP, int WAVES>
bool forward(Args a, hipStream_t st) {
  a.slots = (int)(a.tokens / (32 * WAVES)) + a.sequences;
  k_attention_fwd<DP, WAVES><<<(unsigned)(a.slots * a.heads), 64 * WAVES, 0, st>>>(a);
  return hipGetLastError() == hipSuccess;
}
template <int DP, int WAVES>
bool backward(Args a, hipStream_t st) {
  a.slots = (int)(a.tokens / (32 * WAVES)) + a.sequences;
  k_attention_bwd_q<DP, WAVES><<<(unsigned)(a.slots * a.heads), 64 * WAVES, 0, st>>>(a);
  if (hipGetLastError() != hipSuccess) return false;
  k_attention_bwd_kv<DP, WAVES><<<(unsigned)(a.slots * a.kv_heads), 64 * WAVES, 0, st>>>(a);
  return hipGetLastError() == hipSuccess;
}

// f with the head's width rounded up to a multiple of 32 and the waves of a workgroup as constants
template <class F>
int dispatch(const disco_attention_shape& s, F f) {
  const int dp = (s.head_dim + 31) / 32, waves = waves_of(s);
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
  return dispatch(*shape, [&](auto dp, auto waves) { return forward<dp(), waves()>(a, static_cast<hipStream_t>(hip_stream)); });
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
  return dispatch(*shape, [&](auto dp, auto waves) { return backward<dp(), waves()>(a, static_cast<hipStream_t>(hip_stream)); });
}
