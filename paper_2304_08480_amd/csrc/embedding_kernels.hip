// Token table and learned places, and the tables' gradients.
//
//   y_i = scale E[id_i] + P[place_i],   dE[v] = scale sum of dy_i over id_i = v,   dP[p] = sum of dy_i over place_i = p
//
// Forward: a gather, bound by the rows written and by what the pass before has left of the table in the caches (26533 rows of 512 bf16 from fp32 tables: 12 us one
// call behind the other, 14 to 16 after a backward pass, which writes 100 MB; 78848 rows of 768: 52 after one).
//
// Backward, both tables in the same launches (microseconds for those two batches, vocabulary 49408, gradients fp32):
//   deal   blocks of 2048 rows, sorted in the LDS by their ids' low bits into `slices`, rows rising inside each.  Low bits, because the frequent ids, which
//          tokenizers number first, are then spread over all slices.  7, 12: latency of the sort, while a third of the gradients is cleared.
//   order  a workgroup for each slice: it counts the rows of its ids, each wave those of a share of the blocks, which gives the place of every (id, wave) in the
//          list; where its own part of the list starts is the sum of where the blocks have the slice begin.  Then every wave puts its rows in place, 64
//          at a time, or 256 where they are all of one id.  No atomics between workgroups; rows of an id rise.  18, the rest of the clearing; 38 where two thirds
//          of all rows have one id, which one workgroup then goes through.
//   sums   the list in pieces of equal length: each sums the rows of one id after another in fp32 in registers and stores what lies inside it whole.  17, and
//          46: 5.3 TB/s of gradients, read once for either table.
//   join   what a border of pieces cuts, from the pieces' parts.  8, 19: latency, of list, parts, and where an id has hundreds of pieces their sum.
// (A launch less, every workgroup looking through all ids for its own, took 51 and 119 us for the 27 and 50 of the first two.)
// The order of every sum is that of the rows, in pieces whose borders the number of rows says: equal calls give equal bits.
#include "rows.h"

#include <math.h>

namespace disco {
namespace {

struct Lookup {
  int64_t rows;
  int32_t d, vocabulary, places, wide_ids;       // places 0: none
  int32_t stream;                                // y past the caches
  float scale;
  const void *ids, *place, *table, *place_table;
  void* y;
};

__device__ __forceinline__ int64_t id_at(const void* ids, int64_t i, int wide) {
  return wide ? static_cast<const int64_t*>(ids)[i] : static_cast<const int32_t*>(ids)[i];
}

constexpr int THREADS = 256;
// A row's lanes, LANES of 8 columns each.  One row at a time for a group of lanes: waves enough are on the chip to keep the memory busy with one each (26 thousand rows
// of 512, when forward and backward took 72.5 us: with two rows asked for at once 72.7, with four 74.0, with eight 78).
template <bool TABLE_BF16, bool Y_BF16, int LANES, bool WHOLE>
__global__ __launch_bounds__(THREADS) void k_embedding(Lookup a) {
  constexpr int GROUPS = THREADS / LANES;
  const int lane = threadIdx.x % LANES;
  for (int64_t row = (int64_t)blockIdx.x * GROUPS + threadIdx.x / LANES; row < a.rows; row += (int64_t)gridDim.x * GROUPS) {
    int64_t id = id_at(a.ids, row, a.wide_ids), place = a.places ? id_at(a.place, row, a.wide_ids) : -1;
    if (id >= a.vocabulary) id = -1;
    if (place >= a.places) place = -1;
    for (int col = lane * 8; col < a.d; col += LANES * 8) {
      Eight<TABLE_BF16> e, p;
      e.clear();
      p.clear();
      if (id >= 0) e.template load<WHOLE>(a.table, id * a.d, col, a.d);
      if (place >= 0) p.template load<WHOLE>(a.place_table, place * a.d, col, a.d);
      float v[8];
#pragma unroll
      for (int c = 0; c < 8; ++c) v[c] = fmaf(a.scale, id >= 0 ? e.value(c) : 0.f, p.value(c));
      Eight<Y_BF16> y;
      y.set(v);
      y.template store<WHOLE>(a.y, row * a.d, col, a.d, a.stream);
    }
  }
}

// ---- gradients

struct Entry { int32_t row, id; };
// One table's: ids of the rows, its gradient, and what the workspace holds for it.
struct Side {
  const void* ids;
  void* grad;
  int32_t ids_of, slices, local;        // rows of the table; power of two; most ids of a slice
  float scale;
  Entry *dealt, *list;                  // block by block, slice by slice; all rows id by id
  int32_t* firsts;                      // slice, block: the first one's place in its block; one slice more
  int32_t* count;                       // rows in the list
  float* parts;                         // piece, run that began before it / that goes on behind it, column
};
struct Gradients {
  int64_t rows;
  int32_t d, wide_ids, grad_bf16, accumulate;
  int32_t pitch;                        // of the parts: d in whole pieces of eight
  int32_t piece;                        // rows of the list to a piece
  int32_t blocks;                       // of dealt rows
  int64_t to_clear, cleared;            // pieces of the gradients, and those that the first kernel clears
  int32_t stream;                       // they are cleared past the caches
  const void* dy;
  Side side[2];
};

constexpr int MOST_SLICES = 512, MOST_LOCAL = 2048, LOOK = 4;
constexpr int DEAL = 2048, DEAL_THREADS = 1024, DEAL_WAVES = DEAL_THREADS / 64, DEAL_EACH = DEAL / DEAL_THREADS;

// Lanes of the wave with the same `bits` lowest bits of v as this one.
__device__ __forceinline__ uint64_t lanes_like(int v, int bits) {
  uint64_t same = ~0ull;
  for (int i = 0; i < bits; ++i) {
    const uint64_t on = __ballot(v >> i & 1);
    same &= v >> i & 1 ? on : ~on;
  }
  return same;
}
__device__ __forceinline__ int lanes_before(uint64_t mask) { return __builtin_amdgcn_mbcnt_hi((uint32_t)(mask >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)mask, 0)); }

// Gradients of ids that do not occur are zeros: workgroups beside those that sort, which wait for the LDS and leave the memory idle, clear everything (101 MB of
// gradients, 26 thousand rows of 512, when this was tried: forward and backward 80 us for 87 with the rows that do not occur cleared by those that sort).  Each launch has a share,
// counted in pieces of 16 KiB.
constexpr int CLEAR = 16384;
__device__ __forceinline__ void clear_pieces(const Gradients& a, int64_t from, int64_t to) {
  int64_t done = 0;
  for (int i = 0; i < 2; ++i) {
    const Side& s = a.side[i];
    if (!s.grad) break;
    const int64_t bytes = (int64_t)s.ids_of * a.d * (a.grad_bf16 ? 2 : 4), pieces = (bytes + CLEAR - 1) / CLEAR;
    const int64_t begin = from < done ? 0 : from - done, end = to - done < pieces ? to - done : pieces;
    char* const grad = static_cast<char*>(s.grad);
    // 16 bytes a lane; an end that is not whole by its elements
    for (int64_t at = begin * CLEAR + threadIdx.x * 16; at < end * CLEAR && at < bytes; at += (int64_t)blockDim.x * 16) {
      if (at + 16 <= bytes) store_result(reinterpret_cast<any_u32x4*>(grad + at), u32x4{0, 0, 0, 0}, a.stream);
      else
        for (int64_t b = at; b < bytes; b += 2) *reinterpret_cast<uint16_t*>(grad + b) = 0;
    }
    done += pieces;
  }
}

// of pieces from .. to, workgroup `index` of `of` in each of gridDim.y
__device__ __forceinline__ void clear_share(const Gradients& a, int64_t from, int64_t to, int index, int of) {
  const int64_t workgroups = (int64_t)of * gridDim.y, at = (int64_t)blockIdx.y * of + index, share = (to - from + workgroups - 1) / workgroups;
  const int64_t begin = from + at * share, end = begin + share < to ? begin + share : to;
  if (begin < end) clear_pieces(a, begin, end);
}

template <bool WIDE>
__global__ __launch_bounds__(DEAL_THREADS) void k_embedding_deal(Gradients a) {
  extern __shared__ int32_t counts[];                                // wave, slice (one more: ids that the table does not have): rows, then the next one's place
  __shared__ int32_t sums[DEAL_WAVES], valid;
  __shared__ Entry dealt[DEAL];
  if ((int)blockIdx.x >= a.blocks) {
    clear_share(a, 0, a.cleared, blockIdx.x - a.blocks, gridDim.x - a.blocks);
    return;
  }
  const Side& s = a.side[blockIdx.y];
  const int slices = s.slices, bins = slices + 1, bits = __ffs(slices);
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  int32_t* const mine = counts + wave * bins;
  for (int i = threadIdx.x; i < DEAL_WAVES * bins; i += DEAL_THREADS) counts[i] = 0;
  Entry e[DEAL_EACH];
  int to[DEAL_EACH], rank[DEAL_EACH];
#pragma unroll
  for (int u = 0; u < DEAL_EACH; ++u) {
    const int64_t i = (int64_t)blockIdx.x * DEAL + (wave * DEAL_EACH + u) * 64 + lane;
    int64_t v = -1;
    if (i < a.rows) v = WIDE ? static_cast<const int64_t*>(s.ids)[i] : (int64_t)static_cast<const int32_t*>(s.ids)[i];
    const bool there = v >= 0 && v < s.ids_of;
    e[u] = Entry{(int32_t)i, there ? (int32_t)v : -1};
    to[u] = there ? (int)v & (slices - 1) : slices;
  }
  __syncthreads();
#pragma unroll
  for (int u = 0; u < DEAL_EACH; ++u) {
    const uint64_t same = lanes_like(to[u], bits);
    const int before = lanes_before(same);
    rank[u] = mine[to[u]] + before;
    wave_exchange();
    if (before == 0) mine[to[u]] += __popcll(same);
    wave_exchange();
  }
  __syncthreads();
  // exclusive sums over (slice, wave)
  int total = 0;
  if ((int)threadIdx.x < bins)
    for (int w = 0; w < DEAL_WAVES; ++w) total += counts[w * bins + threadIdx.x];
  int upto = total;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const int v = __shfl_up(upto, o);
    if (lane >= o) upto += v;
  }
  if (lane == 63) sums[wave] = upto;
  __syncthreads();
  for (int w = 0; w < wave; ++w) upto += sums[w];
  if ((int)threadIdx.x < bins) {
    int next = upto - total;
    s.firsts[(int64_t)threadIdx.x * a.blocks + blockIdx.x] = next;
    if ((int)threadIdx.x == slices) valid = next;
    for (int w = 0; w < DEAL_WAVES; ++w) {
      const int n = counts[w * bins + threadIdx.x];
      counts[w * bins + threadIdx.x] = next;
      next += n;
    }
  }
  __syncthreads();
#pragma unroll
  for (int u = 0; u < DEAL_EACH; ++u) dealt[mine[to[u]] + rank[u]] = e[u];
  __syncthreads();
#pragma unroll
  for (int u = 0; u < DEAL_EACH; ++u) {
    const int i = u * DEAL_THREADS + threadIdx.x;
    if (i < valid) s.dealt[(int64_t)blockIdx.x * DEAL + i] = dealt[i];
  }
}

// A wave's share of a slice's rows: a run of blocks, 64 of them at a time, a block a lane.
struct Dealt {
  const Side& s;
  int32_t* ends;                        // the wave's, of 64 blocks: rows up to their ends
  int slice, blocks, begin, end;
  int all, upto, shift;                 // rows of the blocks at hand; of the lane's block
  __device__ __forceinline__ void blocks_from(int base) {
    const int lane = threadIdx.x & 63, b = base + lane;
    int from = 0, n = 0;
    if (b < end) {
      from = s.firsts[(int64_t)slice * blocks + b];
      n = s.firsts[(int64_t)(slice + 1) * blocks + b] - from;
    }
    upto = n;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
      const int v = __shfl_up(upto, o);
      if (lane >= o) upto += v;
    }
    all = __builtin_amdgcn_readlane(upto, 63);
    // where a block's rows would start in the list of all, had it the blocks before it in front of it
    shift = b * DEAL + from - (upto - n);
    wave_exchange();
    ends[lane] = upto;
    wave_exchange();
  }
  __device__ __forceinline__ void rows_from(int at, Entry (&e)[LOOK]) const {
    const int lane = threadIdx.x & 63;
    const int behind = at + 64 * LOOK - 1, of = __popcll(__ballot(upto <= at));
    if (behind < all && of == __popcll(__ballot(upto <= behind))) {   // all of one block
      const Entry* const from = s.dealt + (int64_t)__builtin_amdgcn_readlane(shift, of) + at + lane;
#pragma unroll
      for (int u = 0; u < LOOK; ++u) e[u] = from[u * 64];
      return;
    }
#pragma unroll
    for (int u = 0; u < LOOK; ++u) {
      const int first = at + u * 64, last = first + 63 < all ? first + 63 : all - 1, i = first + lane;
      e[u] = Entry{0, -1};
      if (first >= all) continue;
      // mostly all of one block, or of few rows
      const int block = __popcll(__ballot(upto <= first));
      int to;
      if (block == __popcll(__ballot(upto <= last))) to = __builtin_amdgcn_readlane(shift, block);
      else {
        int own = 0;
#pragma unroll
        for (int step = 32; step > 0; step >>= 1)
          if (ends[own + step - 1] <= i) own += step;
        to = __shfl(shift, own);
      }
      if (i < all) e[u] = s.dealt[(int64_t)to + i];
    }
  }
  // f(row of the lane) for 64 rows at a time, in order, or many(rows) where all 64 LOOK are of one id; the next ones are asked for before.  KEPT: e holds all
  // rows, from the call before
  template <class F, class M>
  __device__ __forceinline__ void each(Entry (&e)[LOOK], bool kept, F f, M many) {
    for (int base = begin; base < end; base += 64) {
      if (!kept) {
        blocks_from(base);
        rows_from(0, e);
      }
      for (int at = 0; at < all; at += 64 * LOOK) {
        Entry next[LOOK];
        const bool more = at + 64 * LOOK < all;
        if (more) rows_from(at + 64 * LOOK, next);
        const int id = __builtin_amdgcn_readfirstlane(e[0].id);
        bool one = true;
#pragma unroll
        for (int u = 0; u < LOOK; ++u) one = one && e[u].id == id;      // a frequent one; -1 past the last row
        if (__all(one)) many(e, id);
        else {
#pragma unroll
          for (int u = 0; u < LOOK; ++u)
            if (at + u * 64 < all) f(e[u]);
        }
        if (more) {
#pragma unroll
          for (int u = 0; u < LOOK; ++u) e[u] = next[u];
        }
      }
    }
  }
};

template <int WAVES>
__global__ __launch_bounds__(64 * WAVES) void k_embedding_order(Gradients a, int slices) {
  constexpr int N = 64 * WAVES;
  extern __shared__ int32_t counts[];                                // wave, local id: rows, then the next one's place in the list
  __shared__ int32_t sums[WAVES], ends[WAVES][64];
  if ((int)blockIdx.x >= slices) {
    clear_share(a, a.cleared, a.to_clear, blockIdx.x - slices, gridDim.x - slices);
    return;
  }
  const Side& s = a.side[blockIdx.y];
  const int slice = blockIdx.x, blocks = a.blocks, shift = __ffs(s.slices) - 1, local = s.local, bits = 32 - __clz(local);
  if (slice >= s.slices) return;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  int32_t* const mine = counts + wave * local;
  for (int i = threadIdx.x; i < WAVES * local; i += N) counts[i] = 0;
  __syncthreads();
  const int share = (blocks + WAVES - 1) / WAVES, begin = wave * share;
  Dealt rows = {s, ends[wave], slice, blocks, begin, begin + share < blocks ? begin + share : blocks, 0, 0, 0};
  Entry now[LOOK];
  rows.each(now, false, [&](const Entry& e) {
    const bool there = e.id >= 0;
    // a frequent id: many lanes on one address
    const int id = __builtin_amdgcn_readfirstlane(e.id);
    const uint64_t same = __ballot(there && e.id == id);
    if (there && e.id != id) atomicAdd(&mine[e.id >> shift], 1);
    if (lane == 0) atomicAdd(&mine[id >> shift], __popcll(same));
  }, [&](const Entry (&)[LOOK], int id) {
    if (lane == 0) atomicAdd(&mine[id >> shift], 64 * LOOK);
  });
  // the rows of the slices before: where the blocks have this one begin
  int before = 0;
  for (int b = threadIdx.x; b < blocks; b += N) before += s.firsts[(int64_t)slice * blocks + b];
  before = wave_reduce(before, [](int x, int y) { return x + y; });
  if (lane == 0) sums[wave] = before;
  __syncthreads();
  int base = 0;
  for (int w = 0; w < WAVES; ++w) base += sums[w];
  // exclusive sums over (id, wave)
  for (int from = 0; from < local; from += N) {
    const int l = from + threadIdx.x;
    int total = 0;
    if (l < local)
      for (int w = 0; w < WAVES; ++w) total += counts[w * local + l];
    int upto = total;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
      const int v = __shfl_up(upto, o);
      if (lane >= o) upto += v;
    }
    __syncthreads();
    if (lane == 63) sums[wave] = upto;
    __syncthreads();
    int next = base + upto - total;
    for (int w = 0; w < WAVES; ++w) {
      if (w < wave) next += sums[w];
      base += sums[w];
    }
    if (l < local)
      for (int w = 0; w < WAVES; ++w) {
        const int n = counts[w * local + l];
        counts[w * local + l] = next;
        next += n;
      }
  }
  if (slice == s.slices - 1 && threadIdx.x == 0) *s.count = base;
  __syncthreads();
  rows.each(now, rows.end - rows.begin <= 64 && rows.all <= 64 * LOOK, [&](const Entry& e) {
    const bool there = e.id >= 0;
    const int which = there ? e.id >> shift : local;
    const bool one = __all(which == __builtin_amdgcn_readfirstlane(which));
    const uint64_t same = one ? ~0ull : lanes_like(which, bits);
    const int rank = lanes_before(same);
    const int place = there ? mine[which] : 0;
    wave_exchange();
    if (there && rank == 0) mine[which] = place + __popcll(same);
    wave_exchange();
    if (there) s.list[place + rank] = e;
  }, [&](const Entry (&e)[LOOK], int id) {
    const int place = mine[id >> shift];
    wave_exchange();
    if (lane == 0) mine[id >> shift] = place + 64 * LOOK;
    wave_exchange();
#pragma unroll
    for (int u = 0; u < LOOK; ++u) s.list[(int64_t)place + u * 64 + lane] = e[u];
  });
}

// scale times a sum to a row of the gradient, on top of what it holds if asked to
template <bool GRAD_BF16, bool WHOLE>
__device__ __forceinline__ void to_gradient(const Gradients& a, const Side& s, int64_t id, int col, const float (&sum)[8]) {
  float v[8];
  Eight<GRAD_BF16> g;
  if (a.accumulate) g.template load<WHOLE>(s.grad, id * a.d, col, a.d);
  else g.clear();
#pragma unroll
  for (int c = 0; c < 8; ++c) v[c] = fmaf(s.scale, sum[c], g.value(c));
  g.set(v);
  g.template store<WHOLE>(s.grad, id * a.d, col, a.d);
}

// A group of lanes has a piece and a block of columns.  It reads the list 32 rows at a time, a row a lane, and asks for the next SUM_AHEAD rows of dy while it
// adds the last ones up.
constexpr int SUM_AHEAD = 8, CHUNK = 32;
template <bool DY_BF16, bool GRAD_BF16, int LANES, bool WHOLE>
__global__ __launch_bounds__(THREADS) void k_embedding_sums(Gradients a, int columns) {
  constexpr int GROUPS = THREADS / LANES, EACH = LANES < CHUNK ? CHUNK / LANES : 1;
  const Side& s = a.side[blockIdx.y];
  const int count = *s.count, lane = threadIdx.x % LANES;
  // blocks of columns of a piece one behind the other
  const int64_t unit = (int64_t)blockIdx.x * GROUPS + threadIdx.x / LANES, piece = unit / columns;
  const int64_t begin = piece * a.piece;
  const bool work = begin < count;
  if (LANES == 64 && !work) return;                                  // groups that share a wave exchange rows of the list and stay together
  const int first = work ? (int)begin : 0, end = !work ? 0 : begin + a.piece < count ? (int)begin + a.piece : count;
  const int col = ((int)(unit % columns) * LANES + lane) * 8;
  const bool in = col < a.d;
  int now = work ? s.list[first].id : -1;
  bool whole = work && (begin == 0 || s.list[first - 1].id != now);  // the run at hand begins in this piece
  const int behind = work && end < count ? s.list[end].id : -1;
  float sum[8];
#pragma unroll
  for (int c = 0; c < 8; ++c) sum[c] = 0.f;
  auto flush = [&](bool ends) {
    if (!in) return;
    if (whole && ends) to_gradient<GRAD_BF16, WHOLE>(a, s, now, col, sum);
    else {
      Eight<false> p;
      p.set(sum);
      p.template store<true>(s.parts, (piece * 2 + whole) * a.pitch, col, a.d);
    }
  };
  for (int base = 0; base < a.piece; base += CHUNK) {
    const int left = end - first - base;                             // of the list, may be none
    if (LANES == 64 && left <= 0) break;
    Entry mine[EACH];
#pragma unroll
    for (int k = 0; k < EACH; ++k) {
      const int i = k * LANES + lane;
      mine[k] = i < left && i < CHUNK ? s.list[first + base + i] : Entry{0, -1};
    }
    auto entry = [&](int i) {
      Entry e;
      if (LANES == 64) {
        e.row = __builtin_amdgcn_readlane(mine[0].row, i);
        e.id = __builtin_amdgcn_readlane(mine[0].id, i);
      } else {
        e.row = __shfl(mine[i / LANES].row, i % LANES, LANES);
        e.id = __shfl(mine[i / LANES].id, i % LANES, LANES);
      }
      return e;
    };
    Eight<DY_BF16> g[2][SUM_AHEAD];
    auto fetch = [&](int batch) {
#pragma unroll
      for (int u = 0; u < SUM_AHEAD; ++u) {
        const Entry e = entry(batch * SUM_AHEAD + u);
        g[batch % 2][u].clear();
        if (in && e.id >= 0) g[batch % 2][u].template load<WHOLE>(a.dy, (int64_t)e.row * a.d, col, a.d);
      }
    };
    fetch(0);
#pragma unroll
    for (int batch = 0; batch < CHUNK / SUM_AHEAD; ++batch) {
      if (batch + 1 < CHUNK / SUM_AHEAD) fetch(batch + 1);
#pragma unroll
      for (int u = 0; u < SUM_AHEAD; ++u) {
        const int id = entry(batch * SUM_AHEAD + u).id;
        if (id >= 0 && id != now) {
          flush(true);
          now = id;
          whole = true;
#pragma unroll
          for (int c = 0; c < 8; ++c) sum[c] = 0.f;
        }
#pragma unroll
        for (int c = 0; c < 8; ++c) sum[c] += g[batch % 2][u].value(c);
      }
    }
  }
  if (work) flush(behind != now);
}

// A run that starts in a piece and goes on behind it: the parts of its pieces.  A wave looks at one piece's end; few parts it adds up by itself, many
// the workgroup does, one share of them to each group of lanes, the shares in order.  Blocks of columns are workgroups of their own.
constexpr int JOIN_THREADS = 1024, JOIN_WAVES = JOIN_THREADS / 64, FEW_PARTS = 16, JOIN_LANES = 32, JOIN_COLUMNS = JOIN_LANES * 8;
template <bool GRAD_BF16, bool WHOLE>
__global__ __launch_bounds__(JOIN_THREADS) void k_embedding_join(Gradients a) {
  constexpr int GROUPS = JOIN_THREADS / JOIN_LANES;
  __shared__ float shares[JOIN_THREADS * 8];
  __shared__ int32_t parts_of[JOIN_WAVES];
  const Side& s = a.side[blockIdx.y];
  const int count = *s.count, lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  // parts of the run that starts in piece p and goes on, 0: there is none
  auto run_of = [&](int64_t p) {
    const int64_t begin = p * a.piece, end = begin + a.piece;
    if (end >= count) return 0;
    const int id = s.list[end - 1].id;
    if (s.list[end].id != id) return 0;
    if (s.list[begin].id == id && begin > 0 && s.list[begin - 1].id == id) return 0;      // began before
    // the last piece that begins in the run, searched for 64 ways at once: list[begin + n piece] is of the run for n up to it
    int64_t n = 1, over = (count - begin + a.piece - 1) / a.piece;
    while (over - n > 1) {
      const int64_t step = (over - n + 63) / 64, at = begin + (n + (lane + 1) * step) * a.piece;
      const int more = __popcll(__ballot(at < count && s.list[at < count ? at : 0].id == id));
      over = n + (more + 1) * step < over ? n + (more + 1) * step : over;
      n += more * step;
    }
    return (int)n + 1;
  };
  auto add = [&](int64_t piece, int from, int to, int col, float (&sum)[8]) {
#pragma unroll
    for (int c = 0; c < 8; ++c) sum[c] = 0.f;
    if (col >= a.d) return;
#pragma unroll 8
    for (int n = from; n < to; ++n) {
      Eight<false> p;
      p.template load<true>(s.parts, ((piece + n) * 2 + (n == 0)) * a.pitch, col, a.d);
#pragma unroll
      for (int c = 0; c < 8; ++c) sum[c] += p.value(c);
    }
  };
  const int64_t own = (int64_t)blockIdx.x * JOIN_WAVES + wave;
  const int mine = __builtin_amdgcn_readfirstlane(run_of(own));
  if (lane == 0) parts_of[wave] = mine;
  const int col = (int)blockIdx.z * JOIN_COLUMNS + (int)(threadIdx.x % JOIN_LANES) * 8;
  if (mine > 0 && mine <= FEW_PARTS && lane < JOIN_LANES && col < a.d) {
    float sum[8];
    add(own, 0, mine, col, sum);
    to_gradient<GRAD_BF16, WHOLE>(a, s, s.list[(own + 1) * a.piece].id, col, sum);
  }
  __syncthreads();
  for (int w = 0; w < JOIN_WAVES; ++w) {
    const int n = parts_of[w];
    if (n <= FEW_PARTS) continue;
    const int64_t piece = (int64_t)blockIdx.x * JOIN_WAVES + w;
    const int group = threadIdx.x / JOIN_LANES, part = (n + GROUPS - 1) / GROUPS, from = group * part, to = from + part < n ? from + part : n;
    float sum[8];
    add(piece, from, to, col, sum);
    __syncthreads();
#pragma unroll
    for (int c = 0; c < 8; ++c) shares[c * JOIN_THREADS + threadIdx.x] = sum[c];
    __syncthreads();
    if (group == 0 && col < a.d) {
      const int groups = (n + part - 1) / part;
      for (int g = 1; g < groups; ++g)
#pragma unroll
        for (int c = 0; c < 8; ++c) sum[c] += shares[c * JOIN_THREADS + g * JOIN_LANES + threadIdx.x];
      to_gradient<GRAD_BF16, WHOLE>(a, s, s.list[(piece + 1) * a.piece].id, col, sum);
    }
  }
}

constexpr int64_t MOST_ROWS = (int64_t)1 << 27, MOST_IDS = (int64_t)MOST_SLICES * MOST_LOCAL;

int check(const disco_embedding_shape* s) {
  if (!s) return DISCO_ERR_NULL;
  if (s->rows <= 0 || s->rows > MOST_ROWS || s->vocabulary <= 0 || s->vocabulary > MOST_IDS || s->places < 0 || s->places > MOST_IDS || s->d <= 0 ||
      s->d > 1 << 14 || !isfinite(s->scale))
    return DISCO_ERR_SHAPE;
  for (int t : {s->table_dtype, s->y_dtype, s->grad_dtype})
    if (t != DISCO_F32 && t != DISCO_BF16) return DISCO_ERR_UNSUPPORTED;
  if (s->id_bits != 32 && s->id_bits != 64) return DISCO_ERR_UNSUPPORTED;
  return DISCO_OK;
}

bool aligned(const void* p, int n) { return (reinterpret_cast<uintptr_t>(p) & (n - 1)) == 0; }
// Workgroups of a lookup.  A launch has less than 2^32 threads, which from 2^26 rows on a group of lanes for each would pass: they take more rows each then.
constexpr int64_t MOST_LOOKUP = ((int64_t)1 << 31) / THREADS;
// Rows of more bytes are written past the caches: smaller ones are found there by what reads them next, larger ones only drive out the table.  Rows of 2048,
// with a copy of them behind it: 64 MiB 53.9 us and 49.2 as they come (17.5 and 26.2 alone), 80 MiB 66.1 and 67.3 (21.1, 35.1), 128 MiB 102 and 113 (31, 54).
constexpr int64_t STREAM_ROWS = (int64_t)72 << 20;
// Zeros of gradients likewise, up to the size of the last-level cache, beyond which they go there and out again anyway, and streaming stores are the slower
// ones.  8192 rows, with a copy of the gradient behind it: 72 MiB 129 us and 128 as they come, 96 MiB 159 and 163, 192 MiB 290 and 294, 256 MiB 365 and 357.
bool stream_zeros(int64_t bytes) { return bytes > (int64_t)88 << 20 && bytes <= (int64_t)224 << 20; }
int size_of(int dtype) { return dtype == DISCO_BF16 ? 2 : 4; }

// Lanes to a row of d columns: as few idle ones as can be, the most of those that have as few.
int lanes_of(int64_t d) {
  const int64_t pieces = (d + 7) / 8;
  int best = 64;
  for (int l : {32, 16})
    if ((pieces + l - 1) / l * l < (pieces + best - 1) / best * best) best = l;
  return best;
}
template <class F>
bool with_lanes(int lanes, F f) {
  return lanes == 64 ? f(std::integral_constant<int, 64>()) : lanes == 32 ? f(std::integral_constant<int, 32>()) : f(std::integral_constant<int, 16>());
}
template <class F>
bool with_bool(bool v, F f) { return v ? f(std::true_type()) : f(std::false_type()); }

// Rows of the list to a piece: enough pieces for the chip, few enough to be joined quickly where one id has most rows.
int piece_of(int64_t rows) {
  int n = 32;
  while (rows > (int64_t)n * 2048) n *= 2;
  return n;
}
int64_t pieces_of(int64_t rows) { return (rows + piece_of(rows) - 1) / piece_of(rows); }
int slices_of(int64_t ids) { return ids <= 256 * 512 ? 256 : MOST_SLICES; }
int64_t blocks_of(int64_t rows) { return (rows + DEAL - 1) / DEAL; }
// In turn: list, dealt, firsts (of as many slices as there may be), parts, count.
struct Offsets { size_t dealt, firsts, parts, count, all; };
Offsets offsets_of(const disco_embedding_shape& s) {
  Offsets o;
  o.dealt = align_up(s.rows * sizeof(Entry));
  o.firsts = o.dealt + align_up(blocks_of(s.rows) * DEAL * sizeof(Entry));
  o.parts = o.firsts + align_up((MOST_SLICES + 1) * blocks_of(s.rows) * sizeof(int32_t));
  o.count = o.parts + align_up(pieces_of(s.rows) * 2 * ((s.d + 7) / 8 * 8) * sizeof(float));
  o.all = o.count + 256;
  return o;
}
bool launched() { return hipGetLastError() == hipSuccess; }        // once a launch: asking clears the error

}  // namespace
}  // namespace disco

using namespace disco;

extern "C" size_t disco_embedding_workspace_bytes(const disco_embedding_shape* shape) {
  if (check(shape) != DISCO_OK) return 0;
  return offsets_of(*shape).all * (shape->places ? 2 : 1);
}

extern "C" int disco_embedding_fwd(const disco_embedding_shape* shape, const void* ids, const void* place, const void* table, const void* places,
                                   void* y, void* hip_stream) {
  if (!shape || !ids || !table || !y) return DISCO_ERR_NULL;
  if (const int st = check(shape)) return st;
  const disco_embedding_shape& s = *shape;
  if (s.places && (!place || !places)) return DISCO_ERR_NULL;
  if (!aligned(ids, s.id_bits / 8) || !aligned(table, size_of(s.table_dtype)) || !aligned(y, size_of(s.y_dtype))) return DISCO_ERR_UNSUPPORTED;
  if (s.places && (!aligned(place, s.id_bits / 8) || !aligned(places, size_of(s.table_dtype)))) return DISCO_ERR_UNSUPPORTED;
  Lookup a = {};
  a.rows = s.rows; a.d = (int32_t)s.d; a.vocabulary = (int32_t)s.vocabulary; a.places = (int32_t)s.places; a.wide_ids = s.id_bits == 64; a.scale = s.scale;
  a.ids = ids; a.place = place; a.table = table; a.place_table = places; a.y = y;
  a.stream = s.rows * s.d * size_of(s.y_dtype) > STREAM_ROWS;
  const hipStream_t st = static_cast<hipStream_t>(hip_stream);
  const bool ok = with_lanes(lanes_of(s.d), [&](auto lanes) {
    return with_bool(s.table_dtype == DISCO_BF16, [&](auto tb) {
      return with_bool(s.y_dtype == DISCO_BF16, [&](auto yb) {
        return with_bool(s.d % 8 == 0, [&](auto whole) {
          constexpr int ROWS = THREADS / lanes();
          const int64_t all = (s.rows + ROWS - 1) / ROWS;
          k_embedding<tb(), yb(), lanes(), whole()><<<(unsigned)(all < MOST_LOOKUP ? all : MOST_LOOKUP), THREADS, 0, st>>>(a);
          return launched();
        });
      });
    });
  });
  return ok ? DISCO_OK : DISCO_ERR_HIP;
}

extern "C" int disco_embedding_bwd(const disco_embedding_shape* shape, const void* ids, const void* place, const void* dy, int accumulate, void* dtable,
                                   void* dplaces, void* workspace, size_t workspace_bytes, void* hip_stream) {
  if (!shape || !dy || (!dtable && !dplaces)) return DISCO_ERR_NULL;
  if (const int st = check(shape)) return st;
  const disco_embedding_shape& s = *shape;
  if ((dtable && !ids) || (dplaces && !place)) return DISCO_ERR_NULL;
  if (dplaces && !s.places) return DISCO_ERR_SHAPE;
  if (!aligned(dy, size_of(s.y_dtype))) return DISCO_ERR_UNSUPPORTED;
  for (const void* p : {ids, place})
    if (!aligned(p, s.id_bits / 8)) return DISCO_ERR_UNSUPPORTED;
  for (const void* p : {static_cast<const void*>(dtable), static_cast<const void*>(dplaces)})
    if (!aligned(p, size_of(s.grad_dtype))) return DISCO_ERR_UNSUPPORTED;
  if (!workspace || !aligned(workspace, 256) || workspace_bytes < disco_embedding_workspace_bytes(shape)) return DISCO_ERR_WORKSPACE;
  Gradients a = {};
  a.rows = s.rows; a.d = (int32_t)s.d; a.wide_ids = s.id_bits == 64; a.grad_bf16 = s.grad_dtype == DISCO_BF16; a.accumulate = accumulate != 0;
  a.piece = piece_of(s.rows); a.pitch = (a.d + 7) / 8 * 8; a.dy = dy;
  const Offsets o = offsets_of(s);
  int sides = 0, local = 0, slices = 0;
  char* at = static_cast<char*>(workspace);
  auto side = [&](const void* of, void* grad, int64_t n, float scale) {
    if (!grad) return;
    Side& x = a.side[sides++];
    x.ids = of; x.grad = grad; x.ids_of = (int32_t)n; x.scale = scale;
    x.slices = slices_of(n);
    x.local = (int32_t)((n + x.slices - 1) / x.slices);
    x.list = reinterpret_cast<Entry*>(at);
    x.dealt = reinterpret_cast<Entry*>(at + o.dealt);
    x.firsts = reinterpret_cast<int32_t*>(at + o.firsts);
    x.parts = reinterpret_cast<float*>(at + o.parts);
    x.count = reinterpret_cast<int32_t*>(at + o.count);
    at += o.all;
    local = local > x.local ? local : x.local;
    slices = slices > x.slices ? slices : x.slices;
  };
  side(ids, dtable, s.vocabulary, s.scale);
  side(place, dplaces, s.places, 1.f);
  const hipStream_t st = static_cast<hipStream_t>(hip_stream);
  a.blocks = (int)blocks_of(s.rows);
  const size_t bins = (size_t)DEAL_WAVES * (slices + 1) * sizeof(int32_t);
  if (!a.accumulate)
    for (int i = 0; i < sides; ++i) a.to_clear += ((int64_t)a.side[i].ids_of * a.d * size_of(s.grad_dtype) + CLEAR - 1) / CLEAR;
  a.cleared = a.to_clear / 3;
  a.stream = stream_zeros(a.to_clear * CLEAR);
  auto clearing = [&](int64_t n) { return (int)((n < 256 ? n : 256) + sides - 1) / sides; };
  const dim3 deal(a.blocks + clearing(a.cleared), sides);
  if (a.wide_ids) k_embedding_deal<true><<<deal, DEAL_THREADS, bins, st>>>(a);
  else k_embedding_deal<false><<<deal, DEAL_THREADS, bins, st>>>(a);
  if (!launched()) return DISCO_ERR_HIP;
  // each wave counts for itself: four of them where the ids of a slice leave the LDS no room for more
  const dim3 order(slices + clearing(a.to_clear - a.cleared), sides);
  if (local <= 512) k_embedding_order<16><<<order, 1024, 16 * local * sizeof(int32_t), st>>>(a, slices);
  else k_embedding_order<4><<<order, 256, 4 * local * sizeof(int32_t), st>>>(a, slices);
  if (!launched()) return DISCO_ERR_HIP;
  const int64_t pieces = pieces_of(s.rows);
  const bool ok = with_bool(s.d % 8 == 0, [&](auto whole) {
    return with_bool(a.grad_bf16, [&](auto gb) {
      const bool summed = with_lanes(lanes_of(s.d), [&](auto lanes) {
        return with_bool(s.y_dtype == DISCO_BF16, [&](auto yb) {
          constexpr int GROUPS = THREADS / lanes();
          const int columns = ((int)s.d + lanes() * 8 - 1) / (lanes() * 8);
          k_embedding_sums<yb(), gb(), lanes(), whole()><<<dim3((unsigned)((pieces * columns + GROUPS - 1) / GROUPS), sides), THREADS, 0, st>>>(a, columns);
          return launched();
        });
      });
      if (!summed || pieces == 1) return summed;
      const dim3 join((unsigned)((pieces - 1 + JOIN_WAVES - 1) / JOIN_WAVES), sides, (unsigned)((s.d + JOIN_COLUMNS - 1) / JOIN_COLUMNS));
      k_embedding_join<gb(), whole()><<<join, JOIN_THREADS, 0, st>>>(a);
      return launched();
    });
  });
  return ok ? DISCO_OK : DISCO_ERR_HIP;
}
