// Norm of every query and key head and its rotation by the row's place, in one pass between the projection and the attention.
//
//   n = N(x) over a head's channels,  y = R n:  a' = a cos - b sin,  b' = a sin + b cos for every pair (a, b) of rotated channels
//   g = R^T dy,  dx = rstd (p - [mean p] - xhat mean(p xhat)),  p = g w,  xhat = (x - mean) rstd;  dw = sum g xhat,  db = sum g
//
// Bound by memory, at the rate of a copy (128 x 197 rows, 12 and 12 heads of 64, layer norms, bf16: forward 35 to 37 us, 4.2 to 4.5 TB/s, backward 46, 5.1, and 5 for the sums; 4 x 8192
// rows, 16 and 8 heads of 128, RMS: 82 and 102 us, 4.9 and 5.9, and 6; 13 x 769 rows, 5 heads and 1 of 80, fp32 to bf16: 12 us, 2.4, where 6 of 16 lanes have no
// channels and no two heads of a unit need be of one row).  A head is read once, kept by LANES lanes, 8 channels each, and written once.  A lane has both channels of its pairs, whichever way they
// are paired: pairs of halves are two loads of four channels, half the rotated width apart.  The norm is two exchanges between those lanes.
// A group of lanes takes HEADS heads at once, so that its loads are under way together; those of one row share cosines and sines.  The
// backward pass takes the statistics from x again, which it has to read anyway, instead of from memory.  Sums over rows and heads are added up in
// registers, one workgroup's groups in the LDS, and the workgroups' in a second kernel, in a fixed order.  fp32 throughout but what is stored.
// 4 heads at once: 84 us for the images forward and backward; 2 take 95, 8, for which the registers of four waves do not do, 117.
#include "rows.h"

#include <math.h>

namespace disco {
namespace {

constexpr int THREADS = 256, HEADS = 4, COMPUTE_UNITS = 256;

// The queries or the keys.
struct Part {
  const void *x, *dy;
  void* y;                              // backward: dx
  const float *w, *b;
  int64_t x_row, x_head, y_row, y_head; // y: backward dy as well; dx as x
  int32_t heads;
  int64_t all, units;                   // heads of all rows; HEADS to a unit
  unsigned workgroups;
};
struct Args {
  int32_t head_dim, rotated, x_bf16, y_bf16;
  int32_t stream;                       // what is stored goes past the caches
  int64_t places;
  float eps, inv_d;
  const int32_t* place;
  const float* rotation;
  Part part[2];
  float* sums;                          // workgroup, dw and db, channel
};

// v over LANES lanes by addition, the same in all of them
template <int LANES>
__device__ __forceinline__ float group_sum(float v) {
  if (LANES >= 2) v += dpp<0xB1>(v);
  if (LANES >= 4) v += dpp<0x4E>(v);
  if (LANES >= 8) v += dpp<0x141>(v);
  if (LANES >= 16) v += dpp<0x140>(v);
  if (LANES >= 32) {
    const auto p = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    const uint32_t p0 = p[0], p1 = p[1];
    v = __uint_as_float(p0) + __uint_as_float(p1);
  }
  return v;
}

// A lane's channels: four from `a` on and four from `b` on.
struct Lane {
  int a, b, pair;                       // pair: of its first one, -1: not rotated
  bool there;
};
template <bool HALVES>
__device__ __forceinline__ Lane lane_of(const Args& a, int lane) {
  Lane l;
  l.a = lane * 8;
  l.b = l.a + 4;
  l.there = l.a < a.head_dim;
  l.pair = l.a < a.rotated ? lane * 4 : -1;
  if (HALVES && l.pair >= 0) {
    l.a = lane * 4;
    l.b = a.rotated / 2 + l.a;
  }
  return l;
}
// A head's eight channels of a lane; offsets are multiples of four elements, bases of 16 bytes.
// LAST: nothing reads it after this, and it is not kept in the caches
template <bool LAST, class V>
__device__ __forceinline__ V load_as(const V* p) { return LAST ? __builtin_nontemporal_load(p) : *p; }
template <bool HALVES, bool BF16, bool LAST = false>
__device__ __forceinline__ Eight<BF16> load_head(const void* p, int64_t at, const Lane& l) {
  Eight<BF16> r;
  if (BF16) {
    const uint16_t* q = static_cast<const uint16_t*>(p) + at;
    if (HALVES) {
      const u32x2 x = load_as<LAST>(reinterpret_cast<const u32x2*>(q + l.a)), y = load_as<LAST>(reinterpret_cast<const u32x2*>(q + l.b));
      r.a = u32x4{x[0], x[1], y[0], y[1]};
    } else {
      r.a = load_as<LAST>(reinterpret_cast<const u32x4*>(q + l.a));
    }
    r.b = u32x4{0, 0, 0, 0};
  } else {
    const uint32_t* q = static_cast<const uint32_t*>(p) + at;
    r.a = load_as<LAST>(reinterpret_cast<const u32x4*>(q + l.a));
    r.b = load_as<LAST>(reinterpret_cast<const u32x4*>(q + l.b));
  }
  return r;
}
template <bool HALVES, bool BF16>
__device__ __forceinline__ void store_head(void* p, int64_t at, const Lane& l, const float (&v)[8], bool stream) {
  Eight<BF16> r;
  r.set(v);
  if (BF16) {
    uint16_t* q = static_cast<uint16_t*>(p) + at;
    if (HALVES) {
      store_result(reinterpret_cast<u32x2*>(q + l.a), u32x2{r.a[0], r.a[1]}, stream);
      store_result(reinterpret_cast<u32x2*>(q + l.b), u32x2{r.a[2], r.a[3]}, stream);
    } else {
      store_result(reinterpret_cast<u32x4*>(q + l.a), r.a, stream);
    }
  } else {
    uint32_t* q = static_cast<uint32_t*>(p) + at;
    store_result(reinterpret_cast<u32x4*>(q + l.a), r.a, stream);
    store_result(reinterpret_cast<u32x4*>(q + l.b), r.b, stream);
  }
}
__device__ __forceinline__ void load_channels(const float* p, const Lane& l, float otherwise, float (&v)[8]) {
#pragma unroll
  for (int e = 0; e < 8; ++e) v[e] = p && l.there ? p[(e < 4 ? l.a : l.b - 4) + e] : otherwise;
}
// Cosines and sines of a lane's four pairs at a row's place; `on`: it is rotated, and the table has the place.
struct Turn { float cos[4], sin[4]; bool on; };
__device__ __forceinline__ Turn turn_of(const Args& a, const Lane& l, int64_t row) {
  Turn t;
  t.on = false;
  if (l.pair >= 0) {
    const int64_t place = a.place ? a.place[row] : row;
    t.on = place >= 0 && place < a.places;
    if (t.on) {
      const float* p = a.rotation + place * a.rotated + l.pair;
      const u32x4 c = *reinterpret_cast<const u32x4*>(p), s = *reinterpret_cast<const u32x4*>(p + a.rotated / 2);
#pragma unroll
      for (int e = 0; e < 4; ++e) { t.cos[e] = __uint_as_float(c[e]); t.sin[e] = __uint_as_float(s[e]); }
    }
  }
  return t;
}
// Pair e of a lane is channels e and 4 + e (halves), or 2 e and 2 e + 1 (neighbours).
template <bool HALVES>
__device__ __forceinline__ void turn(float (&v)[8], const Turn& t, float way) {
  if (!t.on) return;
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    float &a = v[HALVES ? e : 2 * e], &b = v[HALVES ? 4 + e : 2 * e + 1];
    const float s = way * t.sin[e], x = a * t.cos[e] - b * s;
    b = a * s + b * t.cos[e];
    a = x;
  }
}
// Normalised channels in place of v, and 1 / sqrt(var + eps).  Channels past the head's are zeros before and do not matter after.
template <int NORM, int LANES>
__device__ __forceinline__ float normalise(const Args& a, const Lane& l, float (&v)[8]) {
  if (NORM == DISCO_NORM_LAYER) {
    float s = 0.f;
#pragma unroll
    for (int e = 0; e < 8; ++e) s += v[e];
    const float mean = group_sum<LANES>(s) * a.inv_d;
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = l.there ? v[e] - mean : 0.f;
  }
  float s = 0.f;
#pragma unroll
  for (int e = 0; e < 8; ++e) s = fmaf(v[e], v[e], s);
  const float rstd = 1.f / sqrtf(fmaf(group_sum<LANES>(s), a.inv_d, a.eps));
#pragma unroll
  for (int e = 0; e < 8; ++e) v[e] *= rstd;
  return rstd;
}

// Which part a workgroup has, and which of its workgroups it is.
__device__ __forceinline__ int part_of(const Args& a, unsigned& index) {
  const int which = blockIdx.x >= a.part[0].workgroups;
  index = blockIdx.x - (which ? a.part[0].workgroups : 0);
  return which;
}
// The heads of a unit.  Of one row if a row's are a whole number of units; FLAT: they are not, and a unit has the next ones in the order of rows.
template <bool FLAT>
struct Unit {
  int64_t row[HEADS];
  int head[HEADS];
  bool there[HEADS];
  __device__ __forceinline__ Unit(const Part& p, int64_t u) {
    const int64_t i = u * HEADS;
    row[0] = p.all >> 32 ? i / p.heads : (int64_t)((uint32_t)i / (uint32_t)p.heads);
    head[0] = (int)(i - row[0] * p.heads);
#pragma unroll
    for (int h = 0; h < HEADS; ++h) {
      if (h) {
        const bool next = FLAT && head[h - 1] + 1 == p.heads;
        row[h] = row[h - 1] + next;
        head[h] = next ? 0 : head[h - 1] + 1;
      }
      there[h] = !FLAT || i + h < p.all;
    }
  }
};

template <int NORM, int LANES, bool HALVES, bool X_BF16, bool Y_BF16, bool FLAT>
__global__ __launch_bounds__(THREADS) void k_head_norm(Args a) {
  unsigned index;
  const Part& p = a.part[part_of(a, index)];
  const Lane l = lane_of<HALVES>(a, threadIdx.x % LANES);
  float w[8], b[8];
  load_channels(p.w, l, 1.f, w);
  load_channels(p.b, l, 0.f, b);
  constexpr int GROUPS = THREADS / LANES;
  for (int64_t u = (int64_t)index * GROUPS + threadIdx.x / LANES; u < p.units; u += (int64_t)p.workgroups * GROUPS) {
    const Unit<FLAT> unit(p, u);
    Eight<X_BF16> x[HEADS];
#pragma unroll
    for (int h = 0; h < HEADS; ++h) {
      x[h].clear();
      if (l.there && unit.there[h]) x[h] = load_head<HALVES, X_BF16>(p.x, unit.row[h] * p.x_row + unit.head[h] * p.x_head, l);
    }
    Turn t = turn_of(a, l, unit.row[0]);
#pragma unroll
    for (int h = 0; h < HEADS; ++h) {
      if (FLAT && h && unit.there[h]) t = turn_of(a, l, unit.row[h]);
      float v[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e] = x[h].value(e);
      if (NORM != DISCO_NORM_NONE) {
        normalise<NORM, LANES>(a, l, v);
#pragma unroll
        for (int e = 0; e < 8; ++e) v[e] = fmaf(v[e], w[e], b[e]);
      }
      turn<HALVES>(v, t, 1.f);
      if (l.there && unit.there[h]) store_head<HALVES, Y_BF16>(p.y, unit.row[h] * p.y_row + unit.head[h] * p.y_head, l, v, a.stream);
    }
  }
}

template <int NORM, int LANES, bool HALVES, bool X_BF16, bool Y_BF16, bool FLAT>
__global__ __launch_bounds__(THREADS) void k_head_norm_bwd(Args a) {
  unsigned index;
  const Part& p = a.part[part_of(a, index)];
  const Lane l = lane_of<HALVES>(a, threadIdx.x % LANES);
  float w[8], dw[8], db[8];
  load_channels(p.w, l, 1.f, w);
#pragma unroll
  for (int e = 0; e < 8; ++e) dw[e] = db[e] = 0.f;
  constexpr int GROUPS = THREADS / LANES;
  for (int64_t u = (int64_t)index * GROUPS + threadIdx.x / LANES; u < p.units; u += (int64_t)p.workgroups * GROUPS) {
    const Unit<FLAT> unit(p, u);
    Eight<X_BF16> x[HEADS];
    Eight<Y_BF16> dy[HEADS];
    auto load = [&](auto last) {
#pragma unroll
      for (int h = 0; h < HEADS; ++h) {
        x[h].clear();
        dy[h].clear();
        if (l.there && unit.there[h]) {
          if (NORM != DISCO_NORM_NONE) x[h] = load_head<HALVES, X_BF16, last()>(p.x, unit.row[h] * p.x_row + unit.head[h] * p.x_head, l);
          dy[h] = load_head<HALVES, Y_BF16, last()>(p.dy, unit.row[h] * p.y_row + unit.head[h] * p.y_head, l);
        }
      }
    };
    // (the empty asm, as in store_result)
    if (a.stream) {
      asm volatile("");
      load(std::true_type());
      asm volatile("");
    } else {
      load(std::false_type());
    }
    Turn t = turn_of(a, l, unit.row[0]);
#pragma unroll
    for (int h = 0; h < HEADS; ++h) {
      if (FLAT && h && unit.there[h]) t = turn_of(a, l, unit.row[h]);
      float v[8], g[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        v[e] = x[h].value(e);
        g[e] = dy[h].value(e);
      }
      turn<HALVES>(g, t, -1.f);
      if (NORM != DISCO_NORM_NONE) {
        const float rstd = normalise<NORM, LANES>(a, l, v);
        // a head that is not there has gradients of 0, and with eps = 0 a norm of its zeros that is not finite
        const bool mine = l.there && unit.there[h];
        float middle = 0.f, along = 0.f;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          if (mine) {
            dw[e] = fmaf(g[e], v[e], dw[e]);
            db[e] += g[e];
          }
          g[e] *= w[e];
          middle += g[e];
          along = fmaf(g[e], v[e], along);
        }
        middle = NORM == DISCO_NORM_LAYER ? group_sum<LANES>(middle) * a.inv_d : 0.f;
        along = group_sum<LANES>(along) * a.inv_d;
#pragma unroll
        for (int e = 0; e < 8; ++e) g[e] = rstd * (g[e] - middle - v[e] * along);
      }
      if (l.there && unit.there[h]) store_head<HALVES, X_BF16>(p.y, unit.row[h] * p.x_row + unit.head[h] * p.x_head, l, g, a.stream);
    }
  }
  if (NORM == DISCO_NORM_NONE || !a.sums) return;
  __shared__ float all[16][THREADS];
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    all[e][threadIdx.x] = dw[e];
    all[8 + e][threadIdx.x] = db[e];
  }
  __syncthreads();
  // lane's element e of every group: channel (e < 4 ? a : b - 4) + e
  for (int i = threadIdx.x; i < 16 * LANES; i += THREADS) {
    const int lane = i % LANES, e = i / LANES;
    const Lane m = lane_of<HALVES>(a, lane);
    if (!m.there) continue;
    float s = 0.f;
    for (int g = 0; g < GROUPS; ++g) s += all[e][g * LANES + lane];
    a.sums[((int64_t)blockIdx.x * 2 + e / 8) * a.head_dim + (e % 8 < 4 ? m.a : m.b - 4) + e % 8] = s;
  }
}

// The workgroups' sums: 32 channels of one output a workgroup, 32 shares of the list, joined in order.
struct Totals { const float* sums; float* out[4]; unsigned workgroups[2]; int32_t head_dim; };
__global__ __launch_bounds__(1024) void k_head_norm_sums(Totals a) {
  __shared__ float shares[32][33];
  float* const out = a.out[blockIdx.y];
  if (!out) return;
  const int part = blockIdx.y / 2, which = blockIdx.y % 2, channel = blockIdx.x * 32 + threadIdx.x % 32, share = threadIdx.x / 32;
  const unsigned first = part ? a.workgroups[0] : 0, n = a.workgroups[part], each = (n + 31) / 32;
  float s = 0.f;
  if (channel < a.head_dim) {
#pragma unroll 8
    for (unsigned i = share * each; i < (share + 1) * each && i < n; ++i) s += a.sums[((int64_t)(first + i) * 2 + which) * a.head_dim + channel];
  }
  shares[share][threadIdx.x % 32] = s;
  __syncthreads();
  if (share == 0 && channel < a.head_dim) {
    for (int i = 1; i < 32; ++i) s += shares[i][threadIdx.x];
    out[channel] = s;
  }
}

constexpr int64_t MOST_STRIDE = (int64_t)1 << 40;

int check(const disco_head_norm_shape* s) {
  if (!s) return DISCO_ERR_NULL;
  if (s->tokens <= 0 || s->tokens > 0x7fffffff || s->heads <= 0 || s->heads > 1 << 16 || s->kv_heads < 0 || s->kv_heads > 1 << 16 || s->head_dim <= 0 ||
      s->rotated < 0 || s->rotated > s->head_dim || s->places < 0 || s->places > 0x7fffffff)
    return DISCO_ERR_SHAPE;
  if (s->norm != DISCO_NORM_NONE && (!(s->eps >= 0.f) || !isfinite(s->eps))) return DISCO_ERR_SHAPE;
  if (s->head_dim % 8 != 0 || s->head_dim > 256 || s->rotated % 8 != 0) return DISCO_ERR_UNSUPPORTED;
  if (s->norm != DISCO_NORM_NONE && s->norm != DISCO_NORM_LAYER && s->norm != DISCO_NORM_RMS) return DISCO_ERR_UNSUPPORTED;
  if (s->pairs != DISCO_PAIRS_HALVES && s->pairs != DISCO_PAIRS_NEIGHBOURS) return DISCO_ERR_UNSUPPORTED;
  for (int t : {s->x_dtype, s->y_dtype})
    if (t != DISCO_F32 && t != DISCO_BF16) return DISCO_ERR_UNSUPPORTED;
  auto strides = [](int64_t row, int64_t head) {
    if (row <= 0 || row > MOST_STRIDE || head <= 0 || head > MOST_STRIDE) return (int)DISCO_ERR_SHAPE;
    return (int)(row % 8 || head % 8 ? DISCO_ERR_UNSUPPORTED : DISCO_OK);
  };
  for (int st : {strides(s->q_row, s->q_head), strides(s->qn_row, s->qn_head)})
    if (st) return st;
  if (s->kv_heads)
    for (int st : {strides(s->k_row, s->k_head), strides(s->kn_row, s->kn_head)})
      if (st) return st;
  return DISCO_OK;
}
bool aligned(const void* p, int n) { return (reinterpret_cast<uintptr_t>(p) & (n - 1)) == 0; }
bool launched() { return hipGetLastError() == hipSuccess; }        // once a launch: asking clears the error

int lanes_of(int head_dim) { return head_dim <= 32 ? 4 : head_dim <= 64 ? 8 : head_dim <= 128 ? 16 : 32; }

// Workgroups of a call, those of the queries first.  Enough for the chip at most, in proportion to the parts' work; every part has one.
constexpr int MOST_WORKGROUPS = COMPUTE_UNITS * 8;
unsigned workgroups(const disco_head_norm_shape& s, int64_t (&units)[2], unsigned (&of)[2]) {
  const int groups = THREADS / lanes_of(s.head_dim);
  const int heads[2] = {s.heads, s.kv_heads};
  int64_t all = 0;
  for (int i = 0; i < 2; ++i) {
    units[i] = (s.tokens * heads[i] + HEADS - 1) / HEADS;
    all += (units[i] + groups - 1) / groups;
  }
  for (int i = 0; i < 2; ++i) {
    const int64_t want = (units[i] + groups - 1) / groups;
    const int64_t share = all <= MOST_WORKGROUPS ? want : want * MOST_WORKGROUPS / all;
    of[i] = (unsigned)(want && !share ? 1 : share);
  }
  return of[0] + of[1];
}
// Results of more bytes are written past the caches.  12 and 12 heads of 64, forward with a copy of the result behind it: 72 MiB 61.7 us and 59.1 as they come (33.6 and
// 36.1 alone), 96 MiB 79.7 and 79.6, 128 MiB 102 and 105 (54.0, 57.6), 192 MiB 151 and 152 (78.5, 84.0).  The
// backward pass then reads past them as well, forward and backward of 192 MiB 191 us, 198 if not; of 74 MiB it would take 100 for 88.
constexpr int64_t STREAM = (int64_t)96 << 20;
Args args_of(const disco_head_norm_shape& s, int dtype, const int32_t* place, const float* rotation) {
  Args a = {};
  a.head_dim = s.head_dim; a.rotated = s.rotated; a.places = s.places; a.eps = s.eps; a.inv_d = 1.f / s.head_dim; a.place = place; a.rotation = rotation;
  a.stream = s.tokens * (s.heads + s.kv_heads) * s.head_dim * (dtype == DISCO_BF16 ? 2 : 4) > STREAM;
  int64_t units[2];
  unsigned of[2];
  workgroups(s, units, of);
  for (int i = 0; i < 2; ++i) {
    Part& p = a.part[i];
    p.heads = i ? s.kv_heads : s.heads;
    p.all = s.tokens * p.heads;
    p.units = units[i];
    p.workgroups = of[i];
    p.x_row = i ? s.k_row : s.q_row; p.x_head = i ? s.k_head : s.q_head;
    p.y_row = i ? s.kn_row : s.qn_row; p.y_head = i ? s.kn_head : s.qn_head;
  }
  return a;
}

// f with norm, lanes, pairing, the types and how heads are dealt as constants
template <class F>
bool dispatch(const disco_head_norm_shape& s, F f) {
  auto rows = [&](auto... as) {
    return s.heads % HEADS || s.kv_heads % HEADS ? f(as..., std::true_type()) : f(as..., std::false_type());
  };
  auto types = [&](auto... as) {
    if (s.x_dtype == DISCO_BF16) return s.y_dtype == DISCO_BF16 ? rows(as..., std::true_type(), std::true_type()) : rows(as..., std::true_type(), std::false_type());
    return s.y_dtype == DISCO_BF16 ? rows(as..., std::false_type(), std::true_type()) : rows(as..., std::false_type(), std::false_type());
  };
  auto pairs = [&](auto norm, auto lanes) { return s.pairs == DISCO_PAIRS_HALVES ? types(norm, lanes, std::true_type()) : types(norm, lanes, std::false_type()); };
  auto width = [&](auto norm) {
    const int n = lanes_of(s.head_dim);
    if (n == 4) return pairs(norm, std::integral_constant<int, 4>());
    if (n == 8) return pairs(norm, std::integral_constant<int, 8>());
    if (n == 16) return pairs(norm, std::integral_constant<int, 16>());
    return pairs(norm, std::integral_constant<int, 32>());
  };
  if (s.norm == DISCO_NORM_NONE) return width(std::integral_constant<int, DISCO_NORM_NONE>());
  if (s.norm == DISCO_NORM_LAYER) return width(std::integral_constant<int, DISCO_NORM_LAYER>());
  return width(std::integral_constant<int, DISCO_NORM_RMS>());
}

}  // namespace
}  // namespace disco

using namespace disco;

extern "C" size_t disco_head_norm_workspace_bytes(const disco_head_norm_shape* shape) {
  if (check(shape) != DISCO_OK) return 0;
  int64_t units[2];
  unsigned of[2];
  return align_up((size_t)workgroups(*shape, units, of) * 2 * shape->head_dim * sizeof(float));
}

extern "C" int disco_head_norm_fwd(const disco_head_norm_shape* shape, const int32_t* place, const float* rotation, const void* q, const void* k,
                                   const float* w_q, const float* b_q, const float* w_k, const float* b_k, void* qn, void* kn, void* hip_stream) {
  if (!shape) return DISCO_ERR_NULL;
  if (const int st = check(shape)) return st;
  const disco_head_norm_shape& s = *shape;
  if (!q || !qn || (s.kv_heads && (!k || !kn)) || (s.rotated && s.places && !rotation)) return DISCO_ERR_NULL;
  for (const void* p : {q, k, static_cast<const void*>(qn), static_cast<const void*>(kn), static_cast<const void*>(rotation)})
    if (!aligned(p, 16)) return DISCO_ERR_UNSUPPORTED;
  for (const void* p : {static_cast<const void*>(place), static_cast<const void*>(w_q), static_cast<const void*>(b_q), static_cast<const void*>(w_k),
                        static_cast<const void*>(b_k)})
    if (!aligned(p, 4)) return DISCO_ERR_UNSUPPORTED;
  Args a = args_of(s, s.y_dtype, place, rotation);
  a.part[0].x = q; a.part[0].y = qn; a.part[0].w = w_q; a.part[0].b = b_q;
  a.part[1].x = k; a.part[1].y = kn; a.part[1].w = w_k; a.part[1].b = b_k;
  const hipStream_t st = static_cast<hipStream_t>(hip_stream);
  const bool ok = dispatch(s, [&](auto norm, auto lanes, auto halves, auto xb, auto yb, auto flat) {
    k_head_norm<norm(), lanes(), halves(), xb(), yb(), flat()><<<a.part[0].workgroups + a.part[1].workgroups, THREADS, 0, st>>>(a);
    return launched();
  });
  return ok ? DISCO_OK : DISCO_ERR_HIP;
}

extern "C" int disco_head_norm_bwd(const disco_head_norm_shape* shape, const int32_t* place, const float* rotation, const void* q, const void* k,
                                   const float* w_q, const float* w_k, const void* dqn, const void* dkn, void* dq, void* dk, float* dw_q, float* db_q,
                                   float* dw_k, float* db_k, void* workspace, size_t workspace_bytes, void* hip_stream) {
  if (!shape) return DISCO_ERR_NULL;
  if (const int st = check(shape)) return st;
  const disco_head_norm_shape& s = *shape;
  const bool normed = s.norm != DISCO_NORM_NONE;
  if (!dqn || !dq || (normed && !q) || (s.rotated && s.places && !rotation)) return DISCO_ERR_NULL;
  if (s.kv_heads && (!dkn || !dk || (normed && !k))) return DISCO_ERR_NULL;
  for (const void* p : {q, k, dqn, dkn, static_cast<const void*>(dq), static_cast<const void*>(dk), static_cast<const void*>(rotation)})
    if (!aligned(p, 16)) return DISCO_ERR_UNSUPPORTED;
  for (const void* p : {static_cast<const void*>(place), static_cast<const void*>(w_q), static_cast<const void*>(w_k), static_cast<const void*>(dw_q),
                        static_cast<const void*>(db_q), static_cast<const void*>(dw_k), static_cast<const void*>(db_k)})
    if (!aligned(p, 4)) return DISCO_ERR_UNSUPPORTED;
  float* const wanted[4] = {dw_q, db_q, s.kv_heads ? dw_k : nullptr, s.kv_heads ? db_k : nullptr};
  const bool sums = normed && (wanted[0] || wanted[1] || wanted[2] || wanted[3]);
  if (sums && (!workspace || !aligned(workspace, 256) || workspace_bytes < disco_head_norm_workspace_bytes(shape))) return DISCO_ERR_WORKSPACE;
  Args a = args_of(s, s.x_dtype, place, rotation);
  a.part[0].x = q; a.part[0].dy = dqn; a.part[0].y = dq; a.part[0].w = w_q;
  a.part[1].x = k; a.part[1].dy = dkn; a.part[1].y = dk; a.part[1].w = w_k;
  a.sums = sums ? static_cast<float*>(workspace) : nullptr;
  const hipStream_t st = static_cast<hipStream_t>(hip_stream);
  const bool ok = dispatch(s, [&](auto norm, auto lanes, auto halves, auto xb, auto yb, auto flat) {
    k_head_norm_bwd<norm(), lanes(), halves(), xb(), yb(), flat()><<<a.part[0].workgroups + a.part[1].workgroups, THREADS, 0, st>>>(a);
    return launched();
  });
  if (!ok) return DISCO_ERR_HIP;
  if (!sums) return DISCO_OK;
  Totals t = {a.sums, {wanted[0], wanted[1], wanted[2], wanted[3]}, {a.part[0].workgroups, a.part[1].workgroups}, s.head_dim};
  k_head_norm_sums<<<dim3((s.head_dim + 31) / 32, 4), 1024, 0, st>>>(t);
  return launched() ? DISCO_OK : DISCO_ERR_HIP;
}
