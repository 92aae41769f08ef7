// Attention of packed queries to packed keys and values of other lengths, forward and backward: what pools an image's patches, what lets one tower read another's
// states, and a single new query against all of them.
//
//   S = scale q k^T, lse = log sum exp S, P = exp(S - lse), o = P v
//   dv = P^T do, dP = do v^T, delta = <do, o>, dS = P (dP - delta), dq = scale dS k, dk = scale dS^T q
//
// Built from the tiles of attention_tile.h.  Forward and for dq a wave has 32 rows in registers and walks the keys; the rows are those of all query heads that share
// a key head, query by query: row r of a sequence and key head is query r / group of head r % group.  So a single query of eight heads is one
// tile that reads the keys once, and many queries read them once for all heads.  For dk and dv a wave has 32 keys and walks the queries, head by head.
//
// Few rows over long keys (a served query, a few latents) do not fill the chip: a sequence's keys are cut into shares of equal length, the same for all
// sequences, and workgroups walk one share each.  What they come to is joined by a second kernel, in the order of the shares; a sequence
// that is one share long stores its result itself.  The queries that are walked for dk and dv are cut the same way where keys are few.
//
// Bound by memory: the matrix instructions have a tenth of the time and vector instructions a quarter.  Heads are pieces of 128 or 256 bytes of a row; a plain
// reader of such pieces reaches 5.5 to 5.7 TB/s.  Here a workgroup waits for its starts, its rows, its first tiles, one after the other.  In microseconds:
//   512 images, one query each over 197 rows, 12 heads of 64: forward 58 (5.3 TB/s), backward 130 (4.8; keys and values read once, their gradients written);
//   256 captions of 4 to 77 over 197 rows, 12 heads of 64: forward 39, dq 43, dk and dv 60;
//   16 x 64 latents over 1 to 8192 rows, 16 heads of 128 on 8: forward 33 to 40 and 12 for the joint, dq 38 and 10, dk and dv 58;
//   one query of 4 sequences of up to 16384, 16 heads of 128 on 2, forward: 13 to 14 and 7 to 8.
// Many queries on many keys are bound by the products and what stands between them: 2 x 3000 on 3000, 8 heads of 64, forward and backward 241 to 253 (510 to 535 TFLOP/s), 4 x 2048
// on 4096, 16 heads of 128, 1160 (830).
// Keys and values are read for the last time by the kernels that write their gradients, which do not keep them in the caches; nor do they keep
// large dk and dv there (STREAM).  The images, forward and backward, took 182 us so, 199 if keys and values are kept, 220 if the gradients are too: the next forward pass
// waits for what was left in the caches to be written.
// The second reading, for dk and dv, is from the last-level cache: both sides in one launch, one behind the other, took 123 where the captions' two launches took 120 (before rows were
// staged and stored whole).
//
// Scores, softmax and sums are fp32, P and dS are rounded to bf16 for the matrix instruction, as in attention_kernels.hip: against 64 bits o and the gradients
// are off by 0.0023 to 0.0024 of their norm (in fp32 throughout by 0.0017, their own rounding to bf16).
#include "attention_tile.h"

namespace disco {
namespace {

constexpr int COMPUTE_UNITS = 256, STEP = 32;       // STEP: queries that the kernel of dk and dv walks at once

struct Args {
  int64_t q_tokens, k_tokens;
  int32_t sequences, heads, kv_heads, group, head_dim;
  int32_t q_longest, k_longest;
  float scale;
  int64_t q_row, q_head, k_row, k_head, v_row, v_head, o_row, o_head;
  const int32_t *q_starts, *k_starts;
  const __bf16 *q, *k, *v, *o, *dout;
  __bf16 *out, *dq, *dk, *dv;
  float *lse, *delta;
  int32_t tiles;                // of a sequence, all sequences alike; 0: they are searched for
  int32_t share, shares;        // keys to a share (walking queries: steps), and shares of the longest sequence
  int32_t compact;              // shares of the sequences one behind the other: only those that are there have workgroups
  int32_t stream;               // dk and dv go past the caches
  int64_t part_rows;            // rows of parts to a share
  float* parts;                 // share, row, channel
  f32x2* scalars;               // share, row: reference and sum of the softmax
};

struct Range { int first, len; };
__device__ __forceinline__ int bounded(int start, int64_t tokens) { return start < 0 ? 0 : start > (int)tokens ? (int)tokens : start; }
__device__ __forceinline__ Range range_of(const int32_t* starts, int64_t tokens, int longest, int s) {
  const int from = bounded(starts[s], tokens), len = bounded(starts[s + 1], tokens) - from;
  Range r;
  r.first = __builtin_amdgcn_readfirstlane(from);
  r.len = __builtin_amdgcn_readfirstlane(len < 0 ? 0 : len < longest ? len : longest);
  return r;
}

// Sequences own slots, sequence s those from starts[s] each / T + s on: at least as many as it has tiles of T rows, `each` of them to a token, whatever its start,
// so that they are found with no table.  The sequence that owns one, searched for 64 ways at once, and which of its slots it is; false: no sequence.
__device__ __forceinline__ bool find_slot(const int32_t* starts, int64_t tokens, int sequences, int each, int T, int slot, int& s, int& index) {
  const int lane = threadIdx.x & 63;
  auto first = [&](int i) { return bounded(starts[i], tokens) * each / T + i; };
  int lo = 0, n = sequences;
  for (;;) {
    const int step = (n + 63) / 64, i = lo + lane * step;
    const bool below = lane * step < n && first(i) <= slot;
    const int count = __popcll(__ballot(below));
    if (count == 0) return false;
    const int taken = (count - 1) * step;
    lo += taken;
    n = n - taken < step ? n - taken : step;
    if (step == 1) break;
  }
  s = __builtin_amdgcn_readfirstlane(lo);
  index = __builtin_amdgcn_readfirstlane(slot - first(lo));
  return true;
}
// Which tile of T rows of which sequence a slot is.  All sequences have a.tiles slots, or (0) are searched for.
template <int T>
__device__ __forceinline__ bool find_tile(const Args& a, const int32_t* starts, int64_t tokens, int longest, int each, int slot, int& s, Range& range, int& row) {
  int index;
  if (a.tiles) {
    s = slot / a.tiles;
    index = slot - s * a.tiles;
  } else if (!find_slot(starts, tokens, a.sequences, each, T, slot, s, index)) {
    return false;
  }
  s = __builtin_amdgcn_readfirstlane(s);
  range = range_of(starts, tokens, longest, s);
  row = __builtin_amdgcn_readfirstlane(index) * T;
  return row >= 0 && row < range.len * each;
}

// What a workgroup that walks keys has: rows from `row` on of a sequence and key head, and keys begin .. end of it.
struct Walk {
  int kv, row, share, begin, end;
  Range q, k;
  int64_t part;                 // the place of the key head's first row of the sequence in the share's parts
};
// First slot of a sequence's shares, and the row of a key head's first one in a share's parts.
__device__ __forceinline__ int64_t first_part(const Args& a, int s, int k_first, int q_first, int kv) {
  if (!a.compact) return ((int64_t)kv * a.q_tokens + q_first) * a.group;
  return ((int64_t)k_first / a.share + s) * a.part_rows + (int64_t)kv * a.q_longest * a.group;
}
template <int T>
__device__ __forceinline__ bool walk_of(const Args& a, Walk& w) {
  w.kv = blockIdx.x % a.kv_heads;
  const int rest = blockIdx.x / a.kv_heads;
  int s;
  if (a.tiles) {
    const int slot = rest / a.tiles;
    w.row = (rest - slot * a.tiles) * T;
    if (a.compact) {
      if (!find_slot(a.k_starts, a.k_tokens, a.sequences, 1, a.share, slot, s, w.share)) return false;
    } else {
      s = slot / a.shares;
      w.share = slot - s * a.shares;
    }
    w.q = range_of(a.q_starts, a.q_tokens, a.q_longest, s);
    if (w.row > 0 && w.row >= w.q.len * a.group) return false;       // the first tile is there for keys without queries
  } else {
    w.share = rest % a.shares;
    if (!find_tile<T>(a, a.q_starts, a.q_tokens, a.q_longest, a.group, rest / a.shares, s, w.q, w.row)) return false;
  }
  w.k = range_of(a.k_starts, a.k_tokens, a.k_longest, s);
  // (a sequence may own a slot more than it has shares, whose first key is past 32 bits behind 2^31 of them)
  if (w.share > 0 && (int64_t)w.share * a.share >= w.k.len) return false;      // the first share is there for rows without keys
  w.begin = w.share * a.share;
  w.end = w.k.len - w.begin < a.share ? w.k.len : w.begin + a.share;
  w.part = first_part(a, s, w.k.first, w.q.first, w.kv);
  return true;
}

// Where row r's query is.
struct Row {
  bool there;
  int64_t token;
  int head;
};
__device__ __forceinline__ Row row_of(const Args& a, const Range& q, int kv, int r) {
  Row x;
  x.there = r < q.len * a.group;
  const uint32_t i = a.group == 1 ? (uint32_t)r : (uint32_t)r / (uint32_t)a.group;
  x.token = (int64_t)q.first + i;
  x.head = kv * a.group + (r - (int)i * a.group);
  return x;
}

// An accumulated row in fp32, for the kernel that joins.
template <int DP>
__device__ __forceinline__ void store_part(float* row, const f32x16 (&acc)[DP / 32], bool there) {
  const int half = (threadIdx.x & 63) >> 5;
  if (!there) return;
#pragma unroll
  for (int m = 0; m < DP / 32; ++m)
#pragma unroll
    for (int g = 0; g < 4; ++g)
      *reinterpret_cast<f32x4*>(row + 32 * m + 8 * g + 4 * half) = f32x4{acc[m][4 * g], acc[m][4 * g + 1], acc[m][4 * g + 2], acc[m][4 * g + 3]};
}

// 32 accumulated rows, a row a lane, times f, as bf16 to the first `rows` of those at `to`: through 32 rows of the LDS that are the wave's own, so that a store
// instruction writes whole rows and not 32 bytes of each (the pooled images forward and backward 220 us instead of 230; o and dq, written so, gained nothing).
template <int DP>
__device__ __forceinline__ void store_rows(char* lds, __bf16* to, int64_t pitch, int rows, const f32x16 (&acc)[DP / 32], float f, int head_dim, bool stream) {
  using L = Layout<DP>;
  const int lane = threadIdx.x & 63, half = lane >> 5;
  wave_exchange();
#pragma unroll
  for (int m = 0; m < DP / 32; ++m)
#pragma unroll
    for (int g = 0; g < 4; ++g) {
      bf16x4 v;
#pragma unroll
      for (int e = 0; e < 4; ++e) v[e] = (__bf16)(acc[m][4 * g + e] * f);
      *reinterpret_cast<bf16x4*>(lds + L::at(lane & 31, 4 * m + g) + 8 * half) = v;
    }
  wave_exchange();
#pragma unroll
  for (int i = 0; i < 32 * L::PIECES / 64; ++i) {
    const int id = lane + i * 64, row = id / L::PIECES, piece = id % L::PIECES;
    const u32x4 v = *reinterpret_cast<const u32x4*>(lds + L::at(row, piece));
    if (row < rows && piece * 8 < head_dim) store_result(reinterpret_cast<u32x4*>(to + row * pitch + piece * 8), v, stream);
  }
}
// Backward, lse of a row that sees no key, or none that is not hidden by its score, says the same as one too large to be held: its values are 0.
__device__ __forceinline__ float row_base2(float lse) { return lse == -INFINITY ? INFINITY : base2(lse); }

// Backward, a score of minus infinity has P = dS = 0.  If it comes from an infinite channel of its key or query, that channel must not be multiplied by the 0: for the
// products with dS infinities count as zeros.  It changes nothing else, as every score that an infinity is in is infinite or no number, with a dS that is 0 or no
// number.  A wave that has a tile for itself looks at its scores, and takes the infinities out of the tile once they are taken.  Waves that share a tile look at their accumulators
// at the end, and walk again if there is no number among them.  Forward and backward, microseconds without / with that: 256 captions 143 / 139 (a register less, and a third
// wave), latents 146 / 149, 100 times 40 queries over 197 rows, 8 heads of 128, 93 / 96, 2 x 3000 on 3000, 8 heads of 64, 241 / 244, the pooled images 182 / 180.
// (Two forms of the product, one for either case, spill registers in every walk: the accumulators stand elsewhere in each.)
// ROWS rows of a tile in the LDS, by THREADS threads.
template <int DP, int ROWS, int THREADS>
__device__ __forceinline__ void without_infinities(char* lds) {
  using L = Layout<DP>;
  wave_exchange();
#pragma unroll 1
  for (int id = threadIdx.x % THREADS; id < ROWS * L::PIECES; id += THREADS) {
    u32x4* const at = reinterpret_cast<u32x4*>(lds + L::at(id / L::PIECES, id % L::PIECES));
    u32x4 w = *at;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      if ((w[e] & 0x7fffu) == 0x7f80u) w[e] &= 0xffff0000u;
      if ((w[e] & 0x7fff0000u) == 0x7f800000u) w[e] &= 0xffffu;
    }
    *at = w;
  }
  wave_exchange();
}
// Whether some lane's scores are minus infinity.
__device__ __forceinline__ bool hidden(const f32x16& s) {
  float m = s[0];
#pragma unroll
  for (int r = 1; r < 16; ++r) m = fminf(m, s[r]);
  return __any(m == -INFINITY);
}
// Whether a lane has accumulated something that is no number (or infinities that would come to one).
template <int N>
__device__ __forceinline__ bool no_number(const f32x16 (&acc)[N]) {
  float sum = 0.f;
#pragma unroll
  for (int m = 0; m < N; ++m)
#pragma unroll
    for (int r = 0; r < 16; ++r) sum += acc[m][r];
  return sum != sum;
}
// Whether any lane of the workgroup says so.
template <int WAVES>
__device__ __forceinline__ bool any_lane(bool v, int32_t (&said)[WAVES]) {
  int32_t all = __any(v);
  if (WAVES > 1) {
    if ((threadIdx.x & 63) == 0) said[threadIdx.x >> 6] = all;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < WAVES; ++w) all |= said[w];
  }
  return __builtin_amdgcn_readfirstlane(all) != 0;
}

// ---- forward

template <int DP, int WAVES>
__global__ __launch_bounds__(64 * WAVES, 2) void k_cross_fwd(Args a) {
  using S = Shape<DP, WAVES, 1>;
  __shared__ __attribute__((aligned(16))) char lds[S::LDS];
  Walk w;
  if (!walk_of<S::OWN>(a, w)) return;
  const int kv = w.kv, row = w.row, begin = w.begin, end = w.end;
  const Range &qs = w.q, &ks = w.k;
  if (row >= qs.len * a.group) return;
  const __bf16* k = a.k + (int64_t)ks.first * a.k_row + kv * a.k_head;
  const __bf16* v = a.v + (int64_t)ks.first * a.v_row + kv * a.v_head;
  const float c = a.scale * LOG2E;
  Stage<DP, S::WALK, S::THREADS> sk, sv;
  sk.init(a.k_row, a.head_dim);
  sv.init(a.v_row, a.head_dim);
  const int lane = threadIdx.x & 63, half = lane >> 5, wave = wave_of<WAVES>();
  const Row mine = row_of(a, qs, kv, row + 32 * wave + (lane & 31));
  const bool work = row + 32 * wave < qs.len * a.group;              // of the wave
  sk.fetch(k + (int64_t)begin * a.k_row, a.k_row, end - begin, a.head_dim);
  sv.fetch(v + (int64_t)begin * a.v_row, a.v_row, end - begin, a.head_dim);
  Forward<DP> f;
  f.q.fetch(a.q + mine.token * a.q_row + mine.head * a.q_head, mine.there, a.head_dim);
#pragma unroll
  for (int m = 0; m < DP / 32; ++m) f.acc[m] = zeros16();
  sk.put(lds);
  sv.put(lds + S::TILE);
  __syncthreads();
  for (int j = begin, turn = 0; j < end; j += S::WALK, turn ^= 2 * S::TILE) {
    const bool more = j + S::WALK < end;
    if (more) {
      sk.fetch(k + (int64_t)(j + S::WALK) * a.k_row, a.k_row, end - j - S::WALK, a.head_dim);
      sv.fetch(v + (int64_t)(j + S::WALK) * a.v_row, a.v_row, end - j - S::WALK, a.head_dim);
    }
    if (work) f.template step<S::PER / 32>(lds + turn, lds + turn + S::TILE, j, j + S::PER > end, end - 1, c);
    if (more) {
      sk.put(lds + (turn ^ 2 * S::TILE));
      sv.put(lds + (turn ^ 2 * S::TILE) + S::TILE);
    }
    __syncthreads();
  }
  f.total += other_half(f.total);
  if (ks.len > a.share) {
    const int64_t at = w.part + w.share * a.part_rows + row + 32 * wave + (lane & 31);
    store_part<DP>(a.parts + at * DP, f.acc, mine.there);
    if (mine.there && half == 0) a.scalars[at] = f32x2{f.top, f.total};
    return;
  }
  // no key, or none but such of minus infinity: zeros
  const bool none = f.total == 0.f;
  store_row<DP>(a.out + mine.token * a.o_row + mine.head * a.o_head, f.acc, none ? 0.f : 1.f / f.total, a.head_dim, mine.there);
  if (mine.there && half == 0) a.lse[mine.head * a.q_tokens + mine.token] = none ? -INFINITY : f.top * a.scale + __builtin_amdgcn_logf(f.total) * LN2;
}

// The sequence that token `t` is in: the last one that starts at or before it.
__device__ __forceinline__ int sequence_of(const int32_t* starts, int n, int t) {
  int lo = 0;
  while (n > 1) {
    const int mid = n / 2;
    if (starts[lo + mid] <= t) { lo += mid; n -= mid; }
    else n = mid;
  }
  return lo;
}

// Packed rows of all shares to rows of o and lse (FORWARD) or dq: eight channels a thread, GROUPS threads with a part of the shares each where rows are few.
template <int DP, bool FORWARD, int GROUPS>
__global__ __launch_bounds__(256) void k_cross_join_rows(Args a) {
  constexpr int PIECES = DP / 8, ROWS = 256 / (PIECES * GROUPS);
  __shared__ float shares[GROUPS > 1 ? 256 * 10 : 1];
  const int group = threadIdx.x / (PIECES * ROWS), own = threadIdx.x % (PIECES * ROWS), col = own % PIECES * 8;
  const int64_t rows = a.q_tokens * a.heads, at = (int64_t)blockIdx.x * ROWS + own / PIECES;
  // the row's shares, 0: there is no such row, or its sequence is one share long
  int n = 0, token = 0, head = 0;
  int64_t first = 0;
  if (at < rows && group < GROUPS) {
    const int kv = (int)(at / (a.q_tokens * a.group));
    const int64_t in = at - kv * (a.q_tokens * a.group);
    token = (int)(in / a.group);
    head = kv * a.group + (int)(in % a.group);
    const int s = sequence_of(a.q_starts, a.sequences, token);
    const int q0 = bounded(a.q_starts[s], a.q_tokens), q1 = bounded(a.q_starts[s + 1], a.q_tokens);
    const int k0 = bounded(a.k_starts[s], a.k_tokens), k1 = bounded(a.k_starts[s + 1], a.k_tokens);
    const int len = k1 - k0 < a.k_longest ? k1 - k0 : a.k_longest;
    if (token >= q0 && token < q1 && token - q0 < a.q_longest && len > a.share) n = (len - 1) / a.share + 1;
    first = first_part(a, s, k0, q0, kv) + (int64_t)(token - q0) * a.group + in % a.group;
  }
  const float c = a.scale * LOG2E;
  const int each = (n + GROUPS - 1) / GROUPS, begin = group * each, end = begin + each < n ? begin + each : n;
  const float* part = a.parts + first * DP + col;
  float sum[8], top = -INFINITY, total = 0.f;
#pragma unroll
  for (int e = 0; e < 8; ++e) sum[e] = 0.f;
  if (FORWARD) {
#pragma unroll 8
    for (int i = begin; i < end; ++i) top = fmaxf(top, a.scalars[i * a.part_rows + first][0]);
  }
#pragma unroll 4
  for (int i = begin; i < end; ++i) {
    const f32x4 x = *reinterpret_cast<const f32x4*>(part + i * a.part_rows * DP), y = *reinterpret_cast<const f32x4*>(part + i * a.part_rows * DP + 4);
    float w = 1.f;
    if (FORWARD) {
      const f32x2 one = a.scalars[i * a.part_rows + first];
      w = one[0] == top ? 1.f : __builtin_amdgcn_exp2f((one[0] - top) * c);
      total = fmaf(one[1], w, total);
    }
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      sum[e] = fmaf(x[e], w, sum[e]);
      sum[4 + e] = fmaf(y[e], w, sum[4 + e]);
    }
  }
  if (GROUPS > 1) {
#pragma unroll
    for (int e = 0; e < 8; ++e) shares[e * 256 + threadIdx.x] = sum[e];
    shares[8 * 256 + threadIdx.x] = top;
    shares[9 * 256 + threadIdx.x] = total;
    __syncthreads();
    if (group) return;
    for (int g = 1; g < GROUPS; ++g) {
      const int from = g * PIECES * ROWS + own;
      float x = 1.f, y = 1.f;
      if (FORWARD) {
        const float other = shares[8 * 256 + from], higher = fmaxf(top, other);
        x = top == higher ? 1.f : __builtin_amdgcn_exp2f((top - higher) * c);
        y = other == higher ? 1.f : __builtin_amdgcn_exp2f((other - higher) * c);
        top = higher;
        total = fmaf(total, x, shares[9 * 256 + from] * y);
      }
#pragma unroll
      for (int e = 0; e < 8; ++e) sum[e] = fmaf(sum[e], x, shares[e * 256 + from] * y);
    }
  }
  if (n == 0) return;
  const float f = !FORWARD ? a.scale : total == 0.f ? 0.f : 1.f / total;
  bf16x8 r;
#pragma unroll
  for (int e = 0; e < 8; ++e) r[e] = (__bf16)(sum[e] * f);
  __bf16* const to = FORWARD ? a.out + token * a.o_row + head * a.o_head : a.dq + token * a.q_row + head * a.q_head;
  if (col < a.head_dim) *reinterpret_cast<bf16x8*>(to + col) = r;
  if (FORWARD && col == 0) a.lse[head * a.q_tokens + token] = total == 0.f ? -INFINITY : top * a.scale + __builtin_amdgcn_logf(total) * LN2;
}

// ---- backward

// A wave alone with 128 channels may have more than half of a SIMD's registers: the LDS has room for five of them on a compute unit, not eight (captions of 22 on average over 197
// rows, 8 heads of 128, forward and backward: 145 us, 176 with some registers in memory).
template <int DP, int WAVES>
__global__ __launch_bounds__(64 * WAVES, WAVES == 1 && DP == 128 ? 1 : 2) void k_cross_bwd_q(Args a) {
  using S = Shape<DP, WAVES, 1>;
  __shared__ __attribute__((aligned(16))) char lds[S::LDS];
  Walk w;
  if (!walk_of<S::OWN>(a, w)) return;
  const int kv = w.kv, row = w.row, begin = w.begin, end = w.end;
  const Range &qs = w.q, &ks = w.k;
  if (row >= qs.len * a.group) return;
  const __bf16* k = a.k + (int64_t)ks.first * a.k_row + kv * a.k_head;
  const __bf16* v = a.v + (int64_t)ks.first * a.v_row + kv * a.v_head;
  const float c = a.scale * LOG2E;
  Stage<DP, S::WALK, S::THREADS> sk, sv;
  sk.init(a.k_row, a.head_dim);
  sv.init(a.v_row, a.head_dim);
  const int lane = threadIdx.x & 63, half = lane >> 5, wave = wave_of<WAVES>();
  const Row mine = row_of(a, qs, kv, row + 32 * wave + (lane & 31));
  const bool work = WAVES == 1 || row + 32 * wave < qs.len * a.group;
  sk.fetch(k + (int64_t)begin * a.k_row, a.k_row, end - begin, a.head_dim);
  sv.fetch(v + (int64_t)begin * a.v_row, a.v_row, end - begin, a.head_dim);
  Rows<DP> q, dout;
  q.fetch(a.q + mine.token * a.q_row + mine.head * a.q_head, mine.there, a.head_dim);
  dout.fetch(a.dout + mine.token * a.o_row + mine.head * a.o_head, mine.there, a.head_dim);
  float delta = 0.f;
  {
    Rows<DP> o;
    o.fetch(a.o + mine.token * a.o_row + mine.head * a.o_head, mine.there, a.head_dim);
#pragma unroll
    for (int s = 0; s < DP / 16; ++s)
#pragma unroll
      for (int e = 0; e < 8; ++e) delta = fmaf((float)o.f[s][e], (float)dout.f[s][e], delta);
    delta += other_half(delta);
  }
  const int64_t at = mine.head * a.q_tokens + mine.token;
  const float lse2 = mine.there ? row_base2(a.lse[at]) : 0.f;
  // dS of 32 keys from key j on
  auto weights = [&](char* lds_k, int j) {
    f32x16 s[2];                                                      // scores, and dP
    matrix_work(true);
    products<DP, 2, S::TILE>(s, lds_k, [&](int n, int i, int) { return n ? dout.f[i] : q.f[i]; });
    matrix_work(false);
    if (WAVES == 1 && hidden(s[0])) without_infinities<DP, 32, 64>(lds_k);       // for dq; nothing else reads them now
    if (j + 32 > end) {
      int most = end - 1 - j - 4 * half;
      asm volatile("" : "+v"(most));
#pragma unroll
      for (int r = 0; r < 16; ++r)
        if (walked(r, 0) > most) s[0][r] = -INFINITY;
    }
#pragma unroll
    for (int r = 0; r < 16; ++r) s[0][r] = __builtin_amdgcn_exp2f(fmaf(s[0][r], c, -lse2));
    if (ks.len <= 32) delta = own_delta(s[0], s[1]);
#pragma unroll
    for (int r = 0; r < 16; ++r) s[0][r] *= s[1][r] - delta;
    return rounded(s[0]);
  };
  f32x16 acc[DP / 32];
#pragma unroll
  for (int m = 0; m < DP / 32; ++m) acc[m] = zeros16();
  sk.put(lds);
  sv.put(lds + S::TILE);
  __syncthreads();
  for (int j0 = begin, turn = 0; j0 < end; j0 += S::WALK, turn ^= 2 * S::TILE) {
    const bool more = j0 + S::WALK < end;
    if (more) {
      sk.fetch(k + (int64_t)(j0 + S::WALK) * a.k_row, a.k_row, end - j0 - S::WALK, a.head_dim);
      sv.fetch(v + (int64_t)(j0 + S::WALK) * a.v_row, a.v_row, end - j0 - S::WALK, a.head_dim);
    }
#pragma unroll
    for (int sub = 0; sub < S::PER; sub += 32) {
      const int j = j0 + sub;
      if (!work || j >= end) break;
      char* const lds_k = lds + turn + sub * Layout<DP>::PITCH;
      const Weights ds = weights(lds_k, j);
      matrix_work(true);
      accumulate<DP, 1, 0>({&acc}, lds_k, {ds});
      matrix_work(false);
    }
    if (more) {
      sk.put(lds + (turn ^ 2 * S::TILE));
      sv.put(lds + (turn ^ 2 * S::TILE) + S::TILE);
    }
    __syncthreads();
  }
  if constexpr (WAVES > 1) {
    __shared__ int32_t said[WAVES];
    if (any_lane(mine.there && no_number(acc), said)) {
#pragma unroll
      for (int m = 0; m < DP / 32; ++m) acc[m] = zeros16();
      for (int j = begin; j < end; j += 32) {
        sk.fetch(k + (int64_t)j * a.k_row, a.k_row, end - j, a.head_dim);
        sv.fetch(v + (int64_t)j * a.v_row, a.v_row, end - j, a.head_dim);
        sk.put(lds);
        sv.put(lds + S::TILE);
        __syncthreads();
        Weights ds;
        if (work) ds = weights(lds, j);
        __syncthreads();
        without_infinities<DP, 32, S::THREADS>(lds);
        __syncthreads();
        if (work) accumulate<DP, 1, 0>({&acc}, lds, {ds});
        __syncthreads();
      }
    }
  }
  if (mine.there && half == 0 && w.share == 0) a.delta[at] = delta;
  if (ks.len > a.share) store_part<DP>(a.parts + (w.part + w.share * a.part_rows + row + 32 * wave + (lane & 31)) * DP, acc, mine.there);
  else store_row<DP>(a.dq + mine.token * a.q_row + mine.head * a.q_head, acc, a.scale, a.head_dim, mine.there);
}

// dk and dv: as the kernel of attention_kernels.hip, with the queries of another range.
template <int DP, int WAVES>
struct Keys {
  static constexpr int OWN = 32 * WAVES, TILE = 32 * Layout<DP>::PITCH;
  static constexpr int BOTH = 2 * TILE + 2 * STEP * (int)sizeof(float);      // queries, do, lse, delta
  static constexpr bool V_IN_LDS = DP > 64;
  static constexpr int ALL = 2 * BOTH + (V_IN_LDS ? WAVES * TILE : 0);
  static_assert(WAVES * TILE <= 2 * BOTH);                           // the waves' own rows, in the place of the walked tiles
};
template <int DP, int WAVES>
__global__ __launch_bounds__(64 * WAVES, 2) void k_cross_bwd_kv(Args a) {
  using S = Keys<DP, WAVES>;
  constexpr int TILE = S::TILE, BOTH = S::BOTH;
  constexpr bool V_IN_LDS = S::V_IN_LDS;
  __shared__ __attribute__((aligned(16))) char lds[S::ALL];
  char* const lds_v = lds + 2 * BOTH;
  const int kv = blockIdx.x % a.kv_heads, slot = blockIdx.x / a.kv_heads, share = slot % a.shares;
  int seq, row;
  Range ks;
  if (!find_tile<S::OWN>(a, a.k_starts, a.k_tokens, a.k_longest, 1, slot / a.shares, seq, ks, row)) return;
  const Range qs = range_of(a.q_starts, a.q_tokens, a.q_longest, seq);
  // steps of the walk: 32 queries of one head
  const int of_head = (qs.len + STEP - 1) / STEP, all = of_head * a.group, first_step = share * a.share;
  if (first_step > 0 && first_step >= all) return;                   // the first share is there for keys without queries
  const int steps = all - first_step < a.share ? all - first_step : a.share;
  const int lane = threadIdx.x & 63, half = lane >> 5, wave = wave_of<WAVES>();
  const float c = a.scale * LOG2E;
  Stage<DP, STEP, 64 * WAVES> sq, so;
  sq.init(a.q_row, a.head_dim);
  so.init(a.o_row, a.head_dim);
  float next_lse = 0.f, next_delta = 0.f;
  const bool there = row + 32 * wave + (lane & 31) < ks.len, work = row + 32 * wave < ks.len;
  char* const own = lds + TILE * wave;                               // 32 rows of the wave's, before and after the walk
  // what is fetched next, the rows under way, what is used now
  int head, i, next, at;
  auto start = [&] {
    head = kv * a.group + first_step / of_head;
    i = next = at = first_step % of_head * STEP;
  };
  auto fetch = [&] {
    const int64_t from = (int64_t)qs.first + i;
    sq.fetch(a.q + from * a.q_row + head * a.q_head, a.q_row, qs.len - i, a.head_dim);
    so.fetch(a.dout + from * a.o_row + head * a.o_head, a.o_row, qs.len - i, a.head_dim);
    next = i;
    if (threadIdx.x < STEP) {
      const int64_t one = head * a.q_tokens + qs.first + (i + (int)threadIdx.x < qs.len ? i + (int)threadIdx.x : qs.len - 1);
      next_lse = a.lse[one];
      next_delta = a.delta[one];
    }
    i += STEP;
    if (i >= qs.len) { i = 0; ++head; }
  };
  auto put = [&](char* to) {
    sq.put(to);
    so.put(to + TILE);
    if (threadIdx.x < STEP) {
      reinterpret_cast<float*>(to + 2 * TILE)[threadIdx.x] = next + (int)threadIdx.x < qs.len ? row_base2(next_lse) : INFINITY;
      reinterpret_cast<float*>(to + 2 * TILE)[STEP + threadIdx.x] = next_delta;
    }
  };
  f32x16 dk[DP / 32], dv[DP / 32];
#pragma unroll
  for (int m = 0; m < DP / 32; ++m) dk[m] = dv[m] = zeros16();
  if (steps > 0) {
    start();
    fetch();
    char* const own_v = lds_v + TILE * wave;
    Rows<DP> k, v;
    {
      // whole rows from memory, through the LDS to the lanes that own them (captions, dk and dv: 7 us less than with 32 bytes of each row to an instruction)
      Stage<DP, 32, 64, true> sk, sv;
      sk.init(a.k_row, a.head_dim);
      sv.init(a.v_row, a.head_dim);
      const int64_t from = (int64_t)ks.first + row + 32 * wave;
      sk.fetch(a.k + from * a.k_row + kv * a.k_head, a.k_row, ks.len - row - 32 * wave, a.head_dim);
      sv.fetch(a.v + from * a.v_row + kv * a.v_head, a.v_row, ks.len - row - 32 * wave, a.head_dim);
      sk.put(own);
      wave_exchange();
      take_rows<DP>(own, k);
      wave_exchange();
      sv.put(V_IN_LDS ? own_v : own);
      wave_exchange();
      if (!V_IN_LDS) take_rows<DP>(own, v);
    }
    __syncthreads();
    // dS and P of the 32 queries at `now`
    auto weights = [&](char* now, Weights (&w)[2]) {
      f32x16 s[2];                                                    // scores, and dP
      matrix_work(true);
      products<DP, 2, TILE>(s, now, [&](int which, int p, int base) {
        if (!which) return k.f[p];
        return V_IN_LDS ? *reinterpret_cast<const bf16x8*>(own_v + (base ^ p << 5)) : v.f[p];
      });
      matrix_work(false);
      if (WAVES == 1 && hidden(s[0])) without_infinities<DP, 32, 64>(now);       // for dk; nothing else reads them now
      // zeros past the last query times a key that is hidden by minus infinity are no numbers
      if (at + 32 > qs.len) {
        int most = qs.len - 1 - at - 4 * half;
        asm volatile("" : "+v"(most));
#pragma unroll
        for (int r = 0; r < 16; ++r)
          if (walked(r, 0) > most) s[0][r] = -INFINITY;
      }
      const float* scalars = reinterpret_cast<const float*>(now + 2 * TILE) + 4 * half;
#pragma unroll
      for (int g = 0; g < 4; ++g) {
        const f32x4 l = *reinterpret_cast<const f32x4*>(scalars + 8 * g), d = *reinterpret_cast<const f32x4*>(scalars + STEP + 8 * g);
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const int r = 4 * g + e;
          s[0][r] = __builtin_amdgcn_exp2f(fmaf(s[0][r], c, -l[e]));
          s[1][r] = s[0][r] * (s[1][r] - d[e]);
        }
      }
      w[0] = rounded(s[1]);
      w[1] = rounded(s[0]);
    };
    put(lds);
    __syncthreads();
    for (int n = steps, turn = 0; n > 0; --n, turn ^= 1) {
      char* const now = lds + turn * BOTH;
      if (n > 1) fetch();
      if (work) {
        Weights w[2];
        weights(now, w);
        matrix_work(true);
        accumulate<DP, 2, TILE>({&dk, &dv}, now, w);
        matrix_work(false);
      }
      at += STEP;
      if (at >= qs.len) at = 0;
      if (n > 1) put(lds + (turn ^ 1) * BOTH);
      __syncthreads();
    }
    if constexpr (WAVES > 1) {
      __shared__ int32_t said[WAVES];
      if (any_lane(there && no_number(dk), said)) {
#pragma unroll
        for (int m = 0; m < DP / 32; ++m) dk[m] = dv[m] = zeros16();
        start();
        for (int n = steps; n > 0; --n) {
          fetch();
          put(lds);
          __syncthreads();
          Weights w[2];
          if (work) weights(lds, w);
          __syncthreads();
          without_infinities<DP, 32, 64 * WAVES>(lds);
          __syncthreads();
          if (work) accumulate<DP, 2, TILE>({&dk, &dv}, lds, w);
          at += STEP;
          if (at >= qs.len) at = 0;
          __syncthreads();
        }
      }
    }
  }
  const int64_t first = (int64_t)ks.first + row + 32 * wave;
  if (all > a.share) {
    float* const part = a.parts + ((int64_t)(share * a.kv_heads + kv) * a.k_tokens + first + (lane & 31)) * (2 * DP);
    store_part<DP>(part, dk, there);
    store_part<DP>(part + DP, dv, there);
    return;
  }
  store_rows<DP>(own, a.dk + first * a.k_row + kv * a.k_head, a.k_row, ks.len - row - 32 * wave, dk, a.scale, a.head_dim, a.stream);
  store_rows<DP>(own, a.dv + first * a.v_row + kv * a.v_head, a.v_row, ks.len - row - 32 * wave, dv, 1.f, a.head_dim, a.stream);
}

template <int DP>
__global__ __launch_bounds__(256) void k_cross_join_keys(Args a) {
  constexpr int PIECES = 2 * DP / 8;
  const int64_t id = (int64_t)blockIdx.x * 256 + threadIdx.x, at = id / PIECES, rows = a.k_tokens * a.kv_heads;
  const int piece = (int)(id % PIECES), col = piece * 8 % DP;
  const bool values = piece * 8 >= DP;
  if (at >= rows) return;
  const int kv = (int)(at / a.k_tokens), token = (int)(at % a.k_tokens), s = sequence_of(a.k_starts, a.sequences, token);
  const int q0 = bounded(a.q_starts[s], a.q_tokens), q1 = bounded(a.q_starts[s + 1], a.q_tokens);
  const int k0 = bounded(a.k_starts[s], a.k_tokens), k1 = bounded(a.k_starts[s + 1], a.k_tokens);
  const int len = q1 - q0 < 0 ? 0 : q1 - q0 < a.q_longest ? q1 - q0 : a.q_longest, all = (len + STEP - 1) / STEP * a.group;
  if (token < k0 || token >= k1 || token - k0 >= a.k_longest || all <= a.share || col >= a.head_dim) return;
  const int n = (all - 1) / a.share + 1;
  const float* part = a.parts + at * (2 * DP) + piece * 8;
  float sum[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) sum[e] = 0.f;
#pragma unroll 4
  for (int i = 0; i < n; ++i) {
    const f32x4 x = *reinterpret_cast<const f32x4*>(part + i * rows * (2 * DP)), y = *reinterpret_cast<const f32x4*>(part + i * rows * (2 * DP) + 4);
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      sum[e] += x[e];
      sum[4 + e] += y[e];
    }
  }
  const float f = values ? 1.f : a.scale;
  bf16x8 r;
#pragma unroll
  for (int e = 0; e < 8; ++e) r[e] = (__bf16)(sum[e] * f);
  *reinterpret_cast<bf16x8*>((values ? a.dv + token * a.v_row + kv * a.v_head : a.dk + token * a.k_row + kv * a.k_head) + col) = r;
}

// ---- backward with few rows: all rows of a sequence and key head, up to 32, stand in the LDS of one workgroup, whose waves walk the keys, 32 at a time.
// A key's dk and dv are then whole at once, every key and value is read one time, and S and dP are taken one time for all three gradients: dS goes through the
// LDS to be the other operand of dq's product (5 products for 7).  One query over 197 rows, 512 times, 12 heads of 64, forward and backward: 180 us, 218 with
// the two kernels for any rows.  Two or three tiles of rows need the registers of two waves (256 captions of up to 77, tried before rows were stored whole: 148 us where the two
// kernels took 120).
template <int DP>
struct Few {
  static constexpr int WAVES = 4, SUB = 32 * Layout<DP>::PITCH, OWN = 3 * SUB, EACH = 2 * SUB, LDS = OWN + WAVES * EACH;
  static_assert(32 * Layout<32>::PITCH <= SUB);                      // dS in the place of the values
  static_assert(2 * DP * 128 <= LDS);                                // what join() hands over
};
// v over the 32 lanes of a half by addition
__device__ __forceinline__ float half_sum(float v) {
  v += dpp<0xB1>(v);
  v += dpp<0x4E>(v);
  v += dpp<0x141>(v);
  v += dpp<0x140>(v);
  const auto p = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  const uint32_t p0 = p[0], p1 = p[1];
  return __uint_as_float(p0) + __uint_as_float(p1);
}
// A wave's 32 x 32 weights, rows walked and a key a lane, through the LDS: a row a lane and the keys in the order of accumulate().
__device__ __forceinline__ Weights transposed(char* lds, const Weights& w) {
  using L = Layout<32>;
  const int lane = threadIdx.x & 63, half = lane >> 5, in16 = lane & 15, high = lane >> 4 & 1;
#pragma unroll
  for (int g = 0; g < 4; ++g) {
    const bf16x8 f = w.f[g / 2];
    const bf16x4 v = g % 2 ? __builtin_shufflevector(f, f, 4, 5, 6, 7) : __builtin_shufflevector(f, f, 0, 1, 2, 3);
    *reinterpret_cast<bf16x4*>(lds + L::at(lane & 31, g) + 8 * half) = v;
  }
  wave_exchange();
  const int base = L::at(4 * half + (in16 >> 2), 2 * high + ((in16 & 3) >> 1)) + 8 * (in16 & 1);
  Weights t;
#pragma unroll
  for (int j = 0; j < 2; ++j) {
    const bf16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((lds_bf16x4)(lds + base + 16 * j * L::PITCH));
    const bf16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4bf16((lds_bf16x4)(lds + 8 * L::PITCH + (base ^ 32) + 16 * j * L::PITCH));
    t.f[j] = __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7);
  }
  wave_exchange();
  return t;
}

template <int DP>
__global__ __launch_bounds__(256, DP > 64 ? 1 : 2) void k_cross_bwd_few(Args a) {
  using F = Few<DP>;
  constexpr int SUB = F::SUB, ROUND = 32 * F::WAVES;
  __shared__ __attribute__((aligned(16))) char lds[F::LDS];           // rows of q, of do, of q for dk; every wave's keys and values, then dS
  __shared__ __attribute__((aligned(16))) float row_lse[32], row_delta[32];
  Walk w;
  if (!walk_of<32>(a, w)) return;
  const int kv = w.kv, begin = w.begin, end = w.end;
  const Range &qs = w.q, &ks = w.k;
  const int lane = threadIdx.x & 63, half = lane >> 5, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int rows = qs.len * a.group;
  const __bf16* k = a.k + (int64_t)ks.first * a.k_row + kv * a.k_head;
  const __bf16* v = a.v + (int64_t)ks.first * a.v_row + kv * a.v_head;
  const float c = a.scale * LOG2E;
  Stage<DP, 32, 64, true> sk, sv;
  sk.init(a.k_row, a.head_dim);
  sv.init(a.v_row, a.head_dim);
  auto fetch = [&](int j) {
    sk.fetch(k + (int64_t)j * a.k_row, a.k_row, end - j, a.head_dim);
    sv.fetch(v + (int64_t)j * a.v_row, a.v_row, end - j, a.head_dim);
  };
  fetch(begin + 32 * wave);
  const Row mine = row_of(a, qs, kv, lane & 31);
  if (wave == 0) {
    Rows<DP> q, dout, o;
    q.fetch(a.q + mine.token * a.q_row + mine.head * a.q_head, mine.there, a.head_dim);
    dout.fetch(a.dout + mine.token * a.o_row + mine.head * a.o_head, mine.there, a.head_dim);
    o.fetch(a.o + mine.token * a.o_row + mine.head * a.o_head, mine.there, a.head_dim);
    float delta = 0.f;
#pragma unroll
    for (int s = 0; s < DP / 16; ++s)
#pragma unroll
      for (int e = 0; e < 8; ++e) delta = fmaf((float)o.f[s][e], (float)dout.f[s][e], delta);
    delta += other_half(delta);
    const float lse = mine.there ? a.lse[mine.head * a.q_tokens + mine.token] : 0.f;
    put_rows<DP>(lds, q);
    put_rows<DP>(lds + SUB, dout);
    put_rows<DP>(lds + 2 * SUB, q);
    // rows that see nothing, maybe for an infinity of their own
    if (__any(lse == -INFINITY)) without_infinities<DP, 32, 64>(lds + 2 * SUB);
    if (half == 0) {
      row_lse[lane] = mine.there ? row_base2(lse) : INFINITY;
      row_delta[lane] = delta;
    }
  }
  __syncthreads();
  char *const own = lds + F::OWN + wave * F::EACH, *const weights = own + SUB;
  f32x16 dq[DP / 32];
#pragma unroll
  for (int m = 0; m < DP / 32; ++m) dq[m] = zeros16();
  for (int j = begin + 32 * wave; j < end; j += ROUND) {
    sk.put(own);
    sv.put(own + SUB);
    wave_exchange();
    Rows<DP> rk, rv;
    take_rows<DP>(own, rk);
    take_rows<DP>(own + SUB, rv);
    wave_exchange();
    if (j + ROUND < end) fetch(j + ROUND);
    const int key = j + (lane & 31);
    f32x16 dk[DP / 32], dv[DP / 32];
#pragma unroll
    for (int m = 0; m < DP / 32; ++m) dk[m] = dv[m] = zeros16();
    if (rows > 0) {
      f32x16 s[2];                                                    // scores, and dP
      products<DP, 2, SUB>(s, lds, [&](int n, int p, int) { return n ? rv.f[p] : rk.f[p]; });
      if (hidden(s[0])) without_infinities<DP, 32, 64>(own);           // for dq; nothing else reads them now
      // rows past the last are zeros, which times a key that is hidden by minus infinity are no numbers; keys past the last are in no row's softmax
      if (j + 32 > end || rows < 32) {
        int most = key < end ? rows - 1 - 4 * half : -1;
        asm volatile("" : "+v"(most));
#pragma unroll
        for (int r = 0; r < 16; ++r)
          if (walked(r, 0) > most) s[0][r] = -INFINITY;
      }
      const float *lse = row_lse + 4 * half, *del = row_delta + 4 * half;
#pragma unroll
      for (int g = 0; g < 4; ++g) {
        const f32x4 l = *reinterpret_cast<const f32x4*>(lse + 8 * g);
#pragma unroll
        for (int e = 0; e < 4; ++e) s[0][4 * g + e] = __builtin_amdgcn_exp2f(fmaf(s[0][4 * g + e], c, -l[e]));
      }
      const Weights p = rounded(s[0]);
#pragma unroll
      for (int g = 0; g < 4; ++g) {
        f32x4 d = *reinterpret_cast<const f32x4*>(del + 8 * g);
        if (ks.len <= 32) {
#pragma unroll
          for (int e = 0; e < 4; ++e) d[e] = half_sum(s[0][4 * g + e] * s[1][4 * g + e]);      // of a row's few keys, as own_delta
        }
#pragma unroll
        for (int e = 0; e < 4; ++e) s[1][4 * g + e] = s[0][4 * g + e] * (s[1][4 * g + e] - d[e]);
      }
      const Weights ds = rounded(s[1]);
      accumulate<DP, 2, -SUB>({&dk, &dv}, lds + 2 * SUB, {ds, p});
      accumulate<DP, 1, 0>({&dq}, own, {transposed(weights, ds)});
    }
    store_rows<DP>(own, a.dk + (int64_t)(ks.first + j) * a.k_row + kv * a.k_head, a.k_row, end - j, dk, a.scale, a.head_dim, a.stream);
    store_rows<DP>(own + SUB, a.dv + (int64_t)(ks.first + j) * a.v_row + kv * a.v_head, a.v_row, end - j, dv, 1.f, a.head_dim, a.stream);
    wave_exchange();
  }
  __syncthreads();
  join<DP, 1, F::WAVES>(lds, 0, wave, dq);
  if (wave) return;
  if (ks.len > a.share) store_part<DP>(a.parts + (w.part + w.share * a.part_rows + (lane & 31)) * DP, dq, mine.there);
  else store_row<DP>(a.dq + mine.token * a.q_row + mine.head * a.q_head, dq, a.scale, a.head_dim, mine.there);
}

// ---- host

int check(const disco_cross_attention_shape* s) {
  if (!s) return DISCO_ERR_NULL;
  if (s->q_tokens <= 0 || s->q_tokens > 0x7fffffff || s->k_tokens <= 0 || s->k_tokens > 0x7fffffff || s->sequences <= 0 || s->sequences > 1 << 24 ||
      s->q_longest < 0 || s->k_longest < 0 || s->heads <= 0 || s->kv_heads <= 0 || s->heads > 1 << 16 || s->heads % s->kv_heads != 0 || s->head_dim <= 0 ||
      !(s->scale > 0.f) || !isfinite(s->scale * LOG2E))
    return DISCO_ERR_SHAPE;
  // rows and their tiles are counted in 32 bits, and a launch has less than 2^32 threads: 64 for a tile of 32 rows, up to 512 for a sequence
  if (s->q_tokens * (s->heads / s->kv_heads) > 0x7fffffff - 512) return DISCO_ERR_SHAPE;
  for (int64_t tokens : {s->q_tokens, s->k_tokens})
    if ((tokens / 32 + (int64_t)s->sequences * 8) * s->heads >= (int64_t)1 << 26) return DISCO_ERR_SHAPE;
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
bool launched() { return hipGetLastError() == hipSuccess; }        // once a launch: asking clears the error

// dk and dv of more bytes together are written past the caches.  One query each over 197 rows, 12 heads of 64, forward and backward with a copy of the gradients
// behind it: 24 MiB 37.0 us and 35.3 as they come, 48 MiB 61.0 and 62.0 (34.6 and 38.7 alone), 96 MiB 115 and 125 (63.5, 77.7), 192 MiB 211 and 228 (126, 146).
constexpr int64_t STREAM = (int64_t)32 << 20;
Args args_of(const disco_cross_attention_shape& s, const int32_t* q_starts, const int32_t* k_starts) {
  Args a = {};
  a.q_tokens = s.q_tokens; a.k_tokens = s.k_tokens; a.sequences = s.sequences; a.heads = s.heads; a.kv_heads = s.kv_heads; a.group = s.heads / s.kv_heads;
  a.head_dim = s.head_dim; a.scale = s.scale;
  a.q_longest = s.q_longest && s.q_longest < s.q_tokens ? s.q_longest : (int32_t)s.q_tokens;
  a.k_longest = s.k_longest && s.k_longest < s.k_tokens ? s.k_longest : (int32_t)s.k_tokens;
  a.q_row = s.q_row; a.q_head = s.q_head; a.k_row = s.k_row; a.k_head = s.k_head; a.v_row = s.v_row; a.v_head = s.v_head; a.o_row = s.o_row; a.o_head = s.o_head;
  a.q_starts = q_starts; a.k_starts = k_starts;
  a.stream = 2 * s.k_tokens * s.kv_heads * s.head_dim * (int64_t)sizeof(__bf16) > STREAM;
  return a;
}

// How a side's rows are cut: waves to a workgroup, tiles of a sequence (0: searched for) and slots of the launch; shares of the walk, whether they
// are compact, and the parts they leave.
struct Plan { int waves; int64_t slots; int tiles, share, shares, compact; int64_t part_rows; size_t parts, bytes; };

void cut_rows(int64_t rows, int64_t longest, int64_t sequences, int T, Plan& p) {
  const int64_t each = (longest + T - 1) / T, found = rows / T + sequences;
  p.tiles = each * sequences <= found ? (int)each : 0;
  p.slots = p.tiles ? each * sequences : found;
}

// Half of what the chip has room for: cut in two they would take as long again.  (2 x 3000 queries on 3000 keys, 8 heads of 64, 384 workgroups for dk and dv: 253 us
// forward and backward, 275 if they are cut.)
bool enough(int64_t workgroups, int64_t room) { return 2 * workgroups > room; }
// The share of a walk in units (keys, or steps of queries), `longest` and on average `mean` of them: as many workgroups as the chip has room for, `least`
// units to a share, which is a whole number of steps, and no more shares than `most`, nor, as every sequence has as many, than four times that room.
int share_of(int64_t workgroups, int64_t room, int64_t mean, int64_t longest, int least, int step, int64_t most) {
  int64_t share = (mean * workgroups + room - 1) / room;
  if (share < least) share = least;
  if (most > 4 * room / workgroups) most = 4 * room / workgroups;
  if (most < 1) most = 1;
  if (share * most < longest) share = (longest + most - 1) / most;
  share = (share + step - 1) / step * step;
  if (share >= longest || enough(workgroups, room)) share = longest > 0 ? longest : 1;
  return (int)share;
}
constexpr size_t MOST_PARTS = (size_t)1 << 28;       // bytes
// Keys to a share of rows' walk.  With a.q_longest known the shares of all sequences stand one behind the other (find_slot), with places for
// a longest sequence's rows each; else every sequence has as many as the longest.
void cut_keys(const Args& a, int64_t workgroups, int64_t room, int least, int step, size_t row_bytes, Plan& p) {
  const int64_t mean = a.k_tokens / a.sequences, rows = (int64_t)a.heads * (p.tiles ? a.q_longest : a.q_tokens);
  const int64_t fit = (int64_t)(MOST_PARTS / row_bytes) / rows;                                 // shares that fit
  p.compact = p.tiles != 0;
  if (p.compact) {
    const int64_t share = ((mean * workgroups + room - 1) / room + step - 1) / step * step;
    p.share = (int)(enough(workgroups, room) || share >= a.k_longest ? a.k_longest : share < least ? least : share);
  } else {
    p.share = share_of(workgroups, room, mean, a.k_longest, least, step, fit);
  }
  // enough workgroups, but some with far more to do than others
  const int64_t far = 4 * (mean > least ? mean : least) / step * step;
  if (p.compact && p.share > far) p.share = (int)far;
  if (p.compact && p.share < a.k_longest && a.k_tokens / p.share + a.sequences > fit) {
    // k_tokens / share + sequences is to fit
    const int64_t share = fit > a.sequences ? (a.k_tokens + fit - a.sequences - 1) / (fit - a.sequences) : a.k_longest;
    p.share = (int)(share >= a.k_longest ? a.k_longest : (share + step - 1) / step * step);
  }
  if (a.q_tokens * a.heads >= (int64_t)1 << 27) p.share = a.k_longest;                          // a thread for eight channels of a row has to fit the joining launch
  p.shares = (int)(((int64_t)a.k_longest + p.share - 1) / p.share);
  p.part_rows = rows;
  p.compact = p.compact && p.shares > 1;
  p.parts = p.shares == 1 ? 0 : (size_t)rows * (p.compact ? a.k_tokens / p.share + a.sequences : p.shares);
  p.bytes = p.parts * row_bytes;
}
int64_t slots_of(const Args& a, const Plan& p) {
  return p.compact ? (a.k_tokens / p.share + a.sequences) * p.tiles : p.slots * p.shares;
}
int padded(const Args& a) { return (a.head_dim + 31) / 32 * 32; }

Plan plan_rows(const Args& a) {
  Plan p = {};
  const int64_t rows = a.q_tokens * a.group, longest = (int64_t)a.q_longest * a.group, mean = rows / a.sequences;
  // Tiles of 128 rows read the keys once for four of 32; where most rows are fewer than that, a wave alone.  200 captions of 1 to 60, 22 on average, over 197 rows, 8
  // heads of 64, forward and backward: 75 us, with four waves 79; 100 of 40, heads of 128: 96, with one 104.
  p.waves = longest <= 32 || mean <= 24 ? 1 : 4;
  cut_rows(rows, longest, a.sequences, 32 * p.waves, p);
  // Shares of 256 keys for one wave and 512 for four, which leave 4 times as many rows of parts each: 64 latents over up to 8192, forward and backward, 149 us; of
  // 256 159, of 1024 160.  One token's, 256 20 us, 128 21, 64 23.
  const int step = p.waves == 1 ? 32 : 64, least = p.waves == 1 ? 256 : 512, room = p.waves == 1 ? 4 * COMPUTE_UNITS : 2 * COMPUTE_UNITS;
  cut_keys(a, p.slots * a.kv_heads, room, least, step, padded(a) * sizeof(float) + sizeof(f32x2), p);
  return p;
}
Plan plan_keys(const Args& a) {
  Plan p = {};
  const int64_t mean = a.k_tokens / a.sequences;
  p.waves = a.k_longest <= 32 || mean <= 24 ? 1 : 4;
  cut_rows(a.k_tokens, a.k_longest, a.sequences, 32 * p.waves, p);
  const int64_t workgroups = p.slots * a.kv_heads;
  const int64_t longest = (a.q_longest + STEP - 1) / STEP * (int64_t)a.group, middle = (a.q_tokens / a.sequences + STEP - 1) / STEP * a.group;
  const size_t bytes = (size_t)a.k_tokens * a.kv_heads * 2 * padded(a) * sizeof(float);
  // 8 steps at least: 5000 queries on 20 keys, 8 heads of 64, forward and backward 31 us, with 4 30, 16 38, all in one 178; 9000 on 77, 46, 47, 50 and 313
  p.share = share_of(workgroups, 2 * COMPUTE_UNITS, middle, longest, 8, 1, (int64_t)(MOST_PARTS / bytes));
  p.shares = (int)((longest + p.share - 1) / p.share);
  p.bytes = p.shares > 1 ? p.shares * bytes : 0;
  return p;
}
// All rows of a sequence and key head in one tile.
bool few_rows(const Args& a) { return (int64_t)a.q_longest * a.group <= 32; }
Plan plan_few(const Args& a) {
  Plan p = {};
  p.slots = a.sequences;
  p.tiles = 1;
  cut_keys(a, (int64_t)a.sequences * a.kv_heads, 2 * COMPUTE_UNITS, 256, 128, padded(a) * sizeof(float), p);
  return p;
}
// The plan into the arguments of a launch, and its workgroups.
unsigned use(const Plan& p, int64_t slots, Args& a) {
  a.tiles = p.tiles; a.share = p.share; a.shares = p.shares; a.compact = p.compact; a.part_rows = p.part_rows;
  return (unsigned)(slots * a.kv_heads);
}

template <int DP, bool FORWARD>
bool join_rows(const Args& a, hipStream_t st) {
  constexpr int PIECES = DP / 8, GROUPS = 8;
  const int64_t rows = a.q_tokens * a.heads;
  // few rows: not enough threads for the chip without more of them to a row
  if (rows * PIECES <= 64 * COMPUTE_UNITS * 4) {
    constexpr int ROWS = 256 / (PIECES * GROUPS);
    k_cross_join_rows<DP, FORWARD, GROUPS><<<(unsigned)((rows + ROWS - 1) / ROWS), 256, 0, st>>>(a);
  } else {
    constexpr int ROWS = 256 / PIECES;
    k_cross_join_rows<DP, FORWARD, 1><<<(unsigned)((rows + ROWS - 1) / ROWS), 256, 0, st>>>(a);
  }
  return launched();
}
template <int DP>
bool forward(Args a, const Plan& p, hipStream_t st) {
  const unsigned grid = use(p, slots_of(a, p), a);
  if (p.waves == 4) k_cross_fwd<DP, 4><<<grid, 256, 0, st>>>(a);
  else k_cross_fwd<DP, 1><<<grid, 64, 0, st>>>(a);
  if (!launched()) return false;
  return p.shares == 1 || join_rows<DP, true>(a, st);
}
template <int DP>
bool backward(Args a, const Plan& rows, const Plan& keys, hipStream_t st) {
  unsigned grid = use(rows, slots_of(a, rows), a);
  if (rows.waves == 4) k_cross_bwd_q<DP, 4><<<grid, 256, 0, st>>>(a);
  else k_cross_bwd_q<DP, 1><<<grid, 64, 0, st>>>(a);
  if (!launched()) return false;
  if (rows.shares > 1 && !join_rows<DP, false>(a, st)) return false;
  grid = use(keys, keys.slots * keys.shares, a);
  if (keys.waves == 4) k_cross_bwd_kv<DP, 4><<<grid, 256, 0, st>>>(a);
  else k_cross_bwd_kv<DP, 1><<<grid, 64, 0, st>>>(a);
  if (!launched()) return false;
  if (keys.shares == 1) return true;
  const unsigned joins = (unsigned)((a.k_tokens * a.kv_heads * (2 * DP / 8) + 255) / 256);
  k_cross_join_keys<DP><<<joins, 256, 0, st>>>(a);
  return launched();
}
template <int DP>
bool backward_few(Args a, const Plan& p, hipStream_t st) {
  const unsigned grid = use(p, slots_of(a, p), a);
  k_cross_bwd_few<DP><<<grid, 256, 0, st>>>(a);
  if (!launched()) return false;
  return p.shares == 1 || join_rows<DP, false>(a, st);
}
template <class F>
int dispatch(int head_dim, F f) {
  bool ok;
  switch ((head_dim + 31) / 32) {
    case 1: ok = f(std::integral_constant<int, 32>()); break;
    case 2: ok = f(std::integral_constant<int, 64>()); break;
    case 3: ok = f(std::integral_constant<int, 96>()); break;
    default: ok = f(std::integral_constant<int, 128>());
  }
  return ok ? DISCO_OK : DISCO_ERR_HIP;
}

size_t delta_bytes(const Args& a) { return align_up((size_t)a.heads * (size_t)a.q_tokens * sizeof(float)); }
// <do, o> of the rows, then what the shares come to
void workspace_of(void* workspace, Args& a, const Plan& p) {
  char* const at = static_cast<char*>(workspace);
  a.delta = reinterpret_cast<float*>(at);
  a.parts = reinterpret_cast<float*>(at + delta_bytes(a));
  a.scalars = reinterpret_cast<f32x2*>(a.parts + p.parts * padded(a));
}

}  // namespace
}  // namespace disco

using namespace disco;

extern "C" size_t disco_cross_attention_workspace_bytes(const disco_cross_attention_shape* shape) {
  if (check(shape) != DISCO_OK) return 0;
  const Args a = args_of(*shape, nullptr, nullptr);
  const size_t rows = plan_rows(a).bytes, back = few_rows(a) ? plan_few(a).bytes : plan_keys(a).bytes;
  return delta_bytes(a) + align_up(rows > back ? rows : back);
}

extern "C" int disco_cross_attention_fwd(const disco_cross_attention_shape* shape, const int32_t* q_starts, const int32_t* k_starts, const void* q,
                                         const void* k, const void* v, void* o, float* lse, void* workspace, size_t workspace_bytes, void* hip_stream) {
  if (!shape || !q_starts || !k_starts || !q || !k || !v || !o || !lse) return DISCO_ERR_NULL;
  if (const int st = check(shape)) return st;
  for (const void* p : {static_cast<const void*>(q_starts), static_cast<const void*>(k_starts), static_cast<const void*>(lse)})
    if (!aligned(p, 4)) return DISCO_ERR_UNSUPPORTED;
  for (const void* p : {q, k, v, static_cast<const void*>(o)})
    if (!aligned(p, 16)) return DISCO_ERR_UNSUPPORTED;
  if (!workspace || !aligned(workspace, 256) || workspace_bytes < disco_cross_attention_workspace_bytes(shape)) return DISCO_ERR_WORKSPACE;
  Args a = args_of(*shape, q_starts, k_starts);
  a.q = static_cast<const __bf16*>(q); a.k = static_cast<const __bf16*>(k); a.v = static_cast<const __bf16*>(v);
  a.out = static_cast<__bf16*>(o); a.lse = lse;
  const Plan p = plan_rows(a);
  workspace_of(workspace, a, p);
  return dispatch(shape->head_dim, [&](auto dp) { return forward<dp()>(a, p, static_cast<hipStream_t>(hip_stream)); });
}

extern "C" int disco_cross_attention_bwd(const disco_cross_attention_shape* shape, const int32_t* q_starts, const int32_t* k_starts, const void* q,
                                         const void* k, const void* v, const void* o, const float* lse, const void* dout, void* dq, void* dk, void* dv,
                                         void* workspace, size_t workspace_bytes, void* hip_stream) {
  if (!shape || !q_starts || !k_starts || !q || !k || !v || !o || !lse || !dout || !dq || !dk || !dv) return DISCO_ERR_NULL;
  if (const int st = check(shape)) return st;
  for (const void* p : {static_cast<const void*>(q_starts), static_cast<const void*>(k_starts), static_cast<const void*>(lse)})
    if (!aligned(p, 4)) return DISCO_ERR_UNSUPPORTED;
  for (const void* p : {q, k, v, o, dout, static_cast<const void*>(dq), static_cast<const void*>(dk), static_cast<const void*>(dv)})
    if (!aligned(p, 16)) return DISCO_ERR_UNSUPPORTED;
  if (!workspace || !aligned(workspace, 256) || workspace_bytes < disco_cross_attention_workspace_bytes(shape)) return DISCO_ERR_WORKSPACE;
  Args a = args_of(*shape, q_starts, k_starts);
  a.q = static_cast<const __bf16*>(q); a.k = static_cast<const __bf16*>(k); a.v = static_cast<const __bf16*>(v);
  a.o = static_cast<const __bf16*>(o); a.dout = static_cast<const __bf16*>(dout);
  a.dq = static_cast<__bf16*>(dq); a.dk = static_cast<__bf16*>(dk); a.dv = static_cast<__bf16*>(dv);
  a.lse = const_cast<float*>(lse);
  if (few_rows(a)) {
    const Plan p = plan_few(a);
    workspace_of(workspace, a, p);
    return dispatch(shape->head_dim, [&](auto dp) { return backward_few<dp()>(a, p, static_cast<hipStream_t>(hip_stream)); });
  }
  const Plan rows = plan_rows(a), keys = plan_keys(a);
  workspace_of(workspace, a, rows);
  return dispatch(shape->head_dim, [&](auto dp) { return backward<dp()>(a, rows, keys, static_cast<hipStream_t>(hip_stream)); });
}
