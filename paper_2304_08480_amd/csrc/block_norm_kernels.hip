// What stands between two blocks of a tower, in one pass over the rows: norm after a block, gate, residual sum, norm before the next block.
//
//   u = N_post(h) or h,  y = x_scale x + h_scale gate u,  n = N_pre(y)            N(z) = (z - mean) rstd w + b, or z rstd w + b (RMS)
//   t = dy + N_pre'(dn),  dx = x_scale t,  du = h_scale gate t,  dh = N_post'(du),  dgate = h_scale t u
//   N'(g) = rstd (a - [mean a] - zhat mean(a zhat)),  a = g w,  zhat = (z - mean) rstd;  dw = sum over rows g zhat,  db = sum over rows g
//
// Bound by memory up to 4096 columns (forward 39424 x 512 bf16, a norm before: 32 us, 5.0 TB/s; 10007 x 1001
// fp32, both norms, an element gate: 42 us, 4.8 TB/s; backward 16384 x 4096, fp32 stream, bf16 branch, both norms: 249 to 256 us, 4.8 TB/s; 50432 x 768
// bf16, where a quarter of the lanes have no columns: 133 us with the sums' kernel, 3.5 TB/s; a large copy reaches 4.7, calls that read more than they write
// more).  Wider rows with both norms are not, backward (see waves_bwd).  A row is read once, kept in registers (8 columns a lane, LANES lanes a row, so that rows of a few hundred columns
// share a wave and the widest take 16) and written once.  The variance is summed over the deviations from the mean, which are at
// hand, not taken as a difference of sums.  The backward pass adds the sums over rows up in registers, one workgroup's rows in the LDS, and
// the workgroups' in a second kernel, in a fixed order.  Everything is fp32 but what is stored.
#include "common.h"

#include <math.h>

namespace disco {
namespace {

typedef __attribute__((ext_vector_type(4))) uint32_t u32x4;

constexpr int COLS = 8;                 // a lane's columns
constexpr int MAX_D = 1024 * COLS;
constexpr int SUMS = 5;                 // dgate, dw_post, db_post, dw_pre, db_pre

struct Args {
  int64_t rows;
  int32_t d;
  int32_t post, pre, gate, x_bf16, h_bf16;
  float eps_post, eps_pre, x_scale, h_scale, inv_d;
  const void *x, *h, *gate_values, *dy, *dn, *y;
  const float *w_post, *b_post, *w_pre, *b_pre;
  void *out_y, *out_n, *dx, *dh, *dgate_rows;
  float* stats;
  float* sums[SUMS];                    // of the channels, where wanted
  float* parts;                         // workgroups x wanted sums x d
  int32_t wanted;
};

// 8 columns of a row from `col` on, as stored; zeros past the row's end.  Any alignment of the element: gfx950 takes unaligned vector
// accesses, and a row of an odd width starts anywhere.
struct Raw { u32x4 a, b; };
struct __attribute__((packed, aligned(2))) Any16 { u32x4 v; };
__device__ __forceinline__ Raw load_raw(const void* p, int64_t row, int d, int col, bool bf16) {
  Raw r = {u32x4{0, 0, 0, 0}, u32x4{0, 0, 0, 0}};
  if (bf16) {
    const uint16_t* q = static_cast<const uint16_t*>(p) + row * d + col;
    if (col + COLS <= d) r.a = reinterpret_cast<const Any16*>(q)->v;
    else {
#pragma unroll
      for (int e = 0; e < COLS; ++e)
        if (col + e < d) r.a[e / 2] |= (uint32_t)q[e] << (e % 2 * 16);
    }
  } else {
    const uint32_t* q = static_cast<const uint32_t*>(p) + row * d + col;
    if (col + COLS <= d) {
      r.a = reinterpret_cast<const Any16*>(q)->v;
      r.b = reinterpret_cast<const Any16*>(q + 4)->v;
    } else {
#pragma unroll
      for (int e = 0; e < COLS; ++e)
        if (col + e < d) (e < 4 ? r.a : r.b)[e % 4] = q[e];
    }
  }
  return r;
}
// In a kernel all of whose rows are bf16 the second half is never there and takes no registers.
template <bool NARROW>
__device__ __forceinline__ void values(const Raw& r, bool bf16, float (&v)[COLS]) {
  if (NARROW) bf16 = true;
  if (bf16) {
#pragma unroll
    for (int e = 0; e < COLS; ++e) v[e] = __uint_as_float(e % 2 ? r.a[e / 2] & 0xffff0000u : r.a[e / 2] << 16);
  } else {
#pragma unroll
    for (int e = 0; e < COLS; ++e) v[e] = __uint_as_float((e < 4 ? r.a : r.b)[e % 4]);
  }
}
__device__ __forceinline__ uint32_t bf16_bits(float f) { return __builtin_bit_cast(uint16_t, (__bf16)f); }   // to nearest even
// Stores 8 columns and leaves in v what they are as stored.
__device__ __forceinline__ void store(void* p, int64_t row, int d, int col, bool bf16, float (&v)[COLS]) {
  if (bf16) {
    uint16_t* q = static_cast<uint16_t*>(p) + row * d + col;
    u32x4 w;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      w[e] = bf16_bits(v[2 * e]) | bf16_bits(v[2 * e + 1]) << 16;
      v[2 * e] = __uint_as_float(w[e] << 16);
      v[2 * e + 1] = __uint_as_float(w[e] & 0xffff0000u);
    }
    if (col + COLS <= d) reinterpret_cast<Any16*>(q)->v = w;
    else {
#pragma unroll
      for (int e = 0; e < COLS; ++e)
        if (col + e < d) q[e] = (uint16_t)(w[e / 2] >> (e % 2 * 16));
    }
  } else {
    float* q = static_cast<float*>(p) + row * d + col;
    if (col + COLS <= d) {
      u32x4 lo, hi;
#pragma unroll
      for (int e = 0; e < 4; ++e) { lo[e] = __float_as_uint(v[e]); hi[e] = __float_as_uint(v[4 + e]); }
      reinterpret_cast<Any16*>(q)->v = lo;
      reinterpret_cast<Any16*>(q + 4)->v = hi;
    } else {
#pragma unroll
      for (int e = 0; e < COLS; ++e)
        if (col + e < d) q[e] = v[e];
    }
  }
}
// A channel's parameters: `none` without them and past the end
__device__ __forceinline__ void channels(const float* p, int d, int col, float none, float (&v)[COLS]) {
#pragma unroll
  for (int e = 0; e < COLS; ++e) v[e] = p && col + e < d ? p[col + e] : none;
}

// Sums over a row's lanes: inside 16, 32 or 64 lanes by lane exchanges, across waves through the LDS, one barrier each, two buffers in turn.
template <int LANES>
struct RowSum {
  static constexpr int WAVES = LANES > 64 ? LANES / 64 : 1, BLOCK = LANES > 256 ? LANES : 256;
  float (*lds)[BLOCK / 64][2];
  int turn;
  __device__ __forceinline__ float inside(float v) const {
    v += dpp<0xB1>(v);
    v += dpp<0x4E>(v);
    v += dpp<0x141>(v);
    v += dpp<0x140>(v);
    if (LANES > 16) v += __shfl_xor(v, 16);
    if (LANES > 32) v += __shfl_xor(v, 32);
    return v;
  }
  __device__ __forceinline__ void operator()(float& a, float& b) {
    a = inside(a);
    b = inside(b);
    if (WAVES > 1) {
      const int wave = threadIdx.x >> 6;
      if ((threadIdx.x & 63) == 0) { lds[turn][wave][0] = a; lds[turn][wave][1] = b; }
      __syncthreads();
      a = b = 0.f;
      const int from = wave / WAVES * WAVES;
#pragma unroll
      for (int w = 0; w < WAVES; ++w) { a += lds[turn][from + w][0]; b += lds[turn][from + w][1]; }
      turn ^= 1;
    }
  }
};

__device__ __forceinline__ float sum8(const float (&v)[COLS]) {
  return ((v[0] + v[1]) + (v[2] + v[3])) + ((v[4] + v[5]) + (v[6] + v[7]));
}

// Mean and 1 / sqrt(variance + eps) of a row (mean 0 for RMS).
template <int LANES>
__device__ __forceinline__ void statistics(RowSum<LANES>& total, const float (&z)[COLS], bool layer, int d, int col, float inv_d, float eps,
                                           float& mean, float& rstd) {
  float none = 0.f;
  mean = 0.f;
  if (layer) {
    float in[COLS];
#pragma unroll
    for (int e = 0; e < COLS; ++e) in[e] = col + e < d ? z[e] : 0.f;
    mean = sum8(in);
    total(mean, none);
    mean *= inv_d;
  }
  float sq[COLS];
#pragma unroll
  for (int e = 0; e < COLS; ++e) {
    const float c = col + e < d ? z[e] - mean : 0.f;
    sq[e] = c * c;
  }
  float var = sum8(sq);
  total(var, none);
  rstd = 1.f / sqrtf(var * inv_d + eps);
}

// Waves a SIMD that the kernels' registers are kept to, which the grids go by.
template <bool POST, bool PRE>
constexpr int waves_fwd() { return POST && PRE ? 4 : POST || PRE ? 5 : 7; }

template <int LANES, bool POST, bool PRE, bool NARROW>
__global__ __launch_bounds__(LANES > 256 ? LANES : 256, (waves_fwd<POST, PRE>())) void k_block_norm_fwd(Args a) {
  if (NARROW) a.x_bf16 = a.h_bf16 = 1;
  using R = RowSum<LANES>;
  constexpr int ROWS = R::BLOCK / LANES;
  __shared__ float lds[2][R::BLOCK / 64][2];
  R total = {lds, 0};
  const int lane = threadIdx.x % LANES, own = threadIdx.x / LANES, col = lane * COLS, d = a.d;
  float g[COLS], w2[COLS], b2[COLS], w1[COLS], b1[COLS];
  channels(a.gate == DISCO_GATE_CHANNEL ? static_cast<const float*>(a.gate_values) : nullptr, d, col, 1.f, g);
  if (POST) { channels(a.w_post, d, col, 1.f, w2); channels(a.b_post, d, col, 0.f, b2); }
  if (PRE) { channels(a.w_pre, d, col, 1.f, w1); channels(a.b_pre, d, col, 0.f, b1); }
  // a workgroup's rows run in step (barriers): a row that is not there is the last one again, and not stored
  for (int64_t r0 = (int64_t)blockIdx.x * ROWS; r0 < a.rows; r0 += (int64_t)gridDim.x * ROWS) {
    const bool there = r0 + own < a.rows;
    const int64_t row = there ? r0 + own : a.rows - 1;
    Raw rx = {}, rg = {};
    const Raw rh = load_raw(a.h, row, d, col, a.h_bf16);
    if (a.x) rx = load_raw(a.x, row, d, col, a.x_bf16);
    if (a.gate == DISCO_GATE_ELEMENT) rg = load_raw(a.gate_values, row, d, col, a.h_bf16);
    float h[COLS], y[COLS];
    values<NARROW>(rh, a.h_bf16, h);
    float m2 = 0.f, r2 = 0.f, m1 = 0.f, r1 = 0.f;
    if (POST) {
      statistics(total, h, a.post == DISCO_NORM_LAYER, d, col, a.inv_d, a.eps_post, m2, r2);
#pragma unroll
      for (int e = 0; e < COLS; ++e) h[e] = fmaf((h[e] - m2) * r2, w2[e], b2[e]);
    }
    if (a.gate == DISCO_GATE_ELEMENT) values<NARROW>(rg, a.h_bf16, g);
    values<NARROW>(rx, a.x_bf16, y);
#pragma unroll
    for (int e = 0; e < COLS; ++e) y[e] = fmaf(a.x_scale, y[e], a.h_scale * g[e] * h[e]);
    if (there) store(a.out_y, row, d, col, a.x_bf16, y);
    if (PRE) {
      statistics(total, y, a.pre == DISCO_NORM_LAYER, d, col, a.inv_d, a.eps_pre, m1, r1);
#pragma unroll
      for (int e = 0; e < COLS; ++e) y[e] = fmaf((y[e] - m1) * r1, w1[e], b1[e]);
      if (there) store(a.out_n, row, d, col, a.h_bf16, y);
    }
    if (there && lane == 0) *reinterpret_cast<Any16*>(a.stats + row * 4) = Any16{u32x4{__float_as_uint(m2), __float_as_uint(r2), __float_as_uint(m1), __float_as_uint(r1)}};
  }
}

// Waves a SIMD that the backward kernel's registers are kept to: what hides its loads is other rows' waves (50432 x 768 bf16, a norm before the next
// block, a gate for each channel: 204 us with 3 waves, 140 with 4; asking for the next row's data a row ahead costs the registers of a wave and 180).
// Rows of more than 4096 columns are workgroups of 1024 lanes, 4 waves a SIMD whatever this says: 128 registers, of which both norms' parameters and sums
// need more.  64 (all bf16) and 83 are kept in memory, and 8192 x 8192 take 385 us with an fp32 stream (3.1 TB/s) and 460 in bf16 (1.8 TB/s).
template <bool POST, bool PRE, bool NARROW>
constexpr int waves_bwd() { return POST && PRE ? (NARROW ? 3 : 2) : NARROW ? 4 : 3; }

template <int LANES, bool POST, bool PRE, bool NARROW>
__global__ __launch_bounds__(LANES > 256 ? LANES : 256, (waves_bwd<POST, PRE, NARROW>())) void k_block_norm_bwd(Args a) {
  if (NARROW) a.x_bf16 = a.h_bf16 = 1;
  using R = RowSum<LANES>;
  constexpr int ROWS = R::BLOCK / LANES;
  __shared__ float lds[2][R::BLOCK / 64][2];
  __shared__ float joined[R::BLOCK * COLS];
  R total = {lds, 0};
  const int lane = threadIdx.x % LANES, own = threadIdx.x / LANES, col = lane * COLS, d = a.d;
  float g[COLS], w2[COLS], b2[COLS], w1[COLS];
  channels(a.gate == DISCO_GATE_CHANNEL ? static_cast<const float*>(a.gate_values) : nullptr, d, col, 1.f, g);
  if (POST) { channels(a.w_post, d, col, 1.f, w2); channels(a.b_post, d, col, 0.f, b2); }
  if (PRE) channels(a.w_pre, d, col, 1.f, w1);
  float sum[SUMS][COLS];
#pragma unroll
  for (int k = 0; k < SUMS; ++k)
#pragma unroll
    for (int e = 0; e < COLS; ++e) sum[k][e] = 0.f;
  const bool need_h = POST || a.gate != DISCO_GATE_NONE;
  for (int64_t r0 = (int64_t)blockIdx.x * ROWS; r0 < a.rows; r0 += (int64_t)gridDim.x * ROWS) {
    const bool there = r0 + own < a.rows;
    const int64_t row = r0 + own;
    // a row that is not there is all zeros, and so is what it adds to the sums
    Raw ry = {}, rn = {}, rh = {}, rg = {}, rt = {};
    float m2 = 0.f, r2 = 0.f, m1 = 0.f, r1 = 0.f;
    if (there) {
      if (a.dy) rt = load_raw(a.dy, row, d, col, a.x_bf16);
      if (PRE) { ry = load_raw(a.y, row, d, col, a.x_bf16); rn = load_raw(a.dn, row, d, col, a.h_bf16); }
      if (need_h) rh = load_raw(a.h, row, d, col, a.h_bf16);
      if (a.gate == DISCO_GATE_ELEMENT) rg = load_raw(a.gate_values, row, d, col, a.h_bf16);
      const float* st = a.stats + row * 4;
      if (PRE) { m1 = st[2]; r1 = st[3]; }
      if (POST) { m2 = st[0]; r2 = st[1]; }
    }
    float t[COLS];
    values<NARROW>(rt, a.x_bf16, t);
    if (PRE) {
      float y[COLS], dn[COLS], p[COLS], q[COLS];
      values<NARROW>(ry, a.x_bf16, y);
      values<NARROW>(rn, a.h_bf16, dn);
#pragma unroll
      for (int e = 0; e < COLS; ++e) {
        y[e] = (y[e] - m1) * r1;
        p[e] = dn[e] * w1[e];
        q[e] = p[e] * y[e];
        sum[3][e] = fmaf(dn[e], y[e], sum[3][e]);
        sum[4][e] += dn[e];
      }
      float s1 = sum8(p), s2 = sum8(q);
      total(s1, s2);
      s1 = a.pre == DISCO_NORM_LAYER ? s1 * a.inv_d : 0.f;
      s2 *= a.inv_d;
#pragma unroll
      for (int e = 0; e < COLS; ++e) t[e] = col + e < d ? fmaf(r1, p[e] - s1 - y[e] * s2, t[e]) : 0.f;
    }
    {
      float dx[COLS];
#pragma unroll
      for (int e = 0; e < COLS; ++e) dx[e] = a.x_scale * t[e];
      if (there && a.dx) store(a.dx, row, d, col, a.x_bf16, dx);
    }
    float h[COLS];
    values<NARROW>(rh, a.h_bf16, h);
    if (a.gate == DISCO_GATE_ELEMENT) values<NARROW>(rg, a.h_bf16, g);
    float du[COLS], dg[COLS];
#pragma unroll
    for (int e = 0; e < COLS; ++e) {
      if (POST) h[e] = (h[e] - m2) * r2;
      const float u = POST ? fmaf(h[e], w2[e], b2[e]) : h[e];
      dg[e] = a.h_scale * t[e] * u;
      du[e] = a.h_scale * g[e] * t[e];
      sum[0][e] += dg[e];
    }
    if (there && a.dgate_rows) store(a.dgate_rows, row, d, col, a.h_bf16, dg);
    if (POST) {
      float p[COLS], q[COLS];
#pragma unroll
      for (int e = 0; e < COLS; ++e) {
        sum[1][e] = fmaf(du[e], h[e], sum[1][e]);
        sum[2][e] += du[e];
        p[e] = du[e] * w2[e];
        q[e] = p[e] * h[e];
      }
      float s1 = sum8(p), s2 = sum8(q);
      total(s1, s2);
      s1 = a.post == DISCO_NORM_LAYER ? s1 * a.inv_d : 0.f;
      s2 *= a.inv_d;
#pragma unroll
      for (int e = 0; e < COLS; ++e) du[e] = r2 * (p[e] - s1 - h[e] * s2);
    }
    if (there && a.dh) store(a.dh, row, d, col, a.h_bf16, du);
  }
  // one workgroup's sums; with a single workgroup they are the result
  int slot = 0;
#pragma unroll
  for (int k = 0; k < SUMS; ++k) {
    if (!a.sums[k]) continue;
    __syncthreads();
#pragma unroll
    for (int e = 0; e < COLS; ++e) joined[own * (LANES * COLS) + col + e] = sum[k][e];
    __syncthreads();
    float* to = gridDim.x == 1 ? a.sums[k] : a.parts + ((int64_t)blockIdx.x * a.wanted + slot) * d;
    for (int c = threadIdx.x; c < d; c += R::BLOCK) {
      float s = 0.f;
#pragma unroll
      for (int i = 0; i < ROWS; ++i) s += joined[i * (LANES * COLS) + c];
      to[c] = s;
    }
    ++slot;
  }
}

// The workgroups' sums: 64 columns by 16 shares of the workgroups, joined in order.
__global__ __launch_bounds__(1024) void k_block_norm_sums(Args a, int blocks) {
  __shared__ float part[16][64];
  const int c = blockIdx.x * 64 + (threadIdx.x & 63), share = threadIdx.x >> 6;
  float s = 0.f;
  if (c < a.d) {
    const float* p = a.parts + (int64_t)blockIdx.y * a.d + c;
#pragma unroll 16
    for (int b = share; b < blocks; b += 16) s += p[(int64_t)b * a.wanted * a.d];
  }
  part[share][threadIdx.x & 63] = s;
  __syncthreads();
  if (share == 0 && c < a.d) {
#pragma unroll
    for (int i = 1; i < 16; ++i) s += part[i][threadIdx.x];
    int slot = blockIdx.y;
    for (int k = 0; k < SUMS; ++k)
      if (a.sums[k] && slot-- == 0) a.sums[k][c] = s;
  }
}

bool dtype_ok(int t) { return t == DISCO_F32 || t == DISCO_BF16; }
bool norm_ok(int n) { return n == DISCO_NORM_NONE || n == DISCO_NORM_LAYER || n == DISCO_NORM_RMS; }
bool eps_ok(int n, float e) { return n == DISCO_NORM_NONE || (e >= 0.f && isfinite(e)); }
bool aligned(const void* p, int bf16) { return (reinterpret_cast<uintptr_t>(p) & (bf16 ? 1u : 3u)) == 0; }

int check(const disco_block_norm_shape* s) {
  if (!s) return DISCO_ERR_NULL;
  if (s->rows <= 0 || s->d <= 0 || s->d > MAX_D || s->rows > ((int64_t)1 << 40) / s->d) return DISCO_ERR_SHAPE;
  if (!norm_ok(s->post) || !norm_ok(s->pre) || s->gate < DISCO_GATE_NONE || s->gate > DISCO_GATE_ELEMENT || !dtype_ok(s->x_dtype) ||
      !dtype_ok(s->h_dtype))
    return DISCO_ERR_UNSUPPORTED;
  if (!eps_ok(s->post, s->eps_post) || !eps_ok(s->pre, s->eps_pre) || !isfinite(s->x_scale) || !isfinite(s->h_scale)) return DISCO_ERR_SHAPE;
  return DISCO_OK;
}

Args args_of(const disco_block_norm_shape& s) {
  Args a = {};
  a.rows = s.rows; a.d = (int32_t)s.d; a.post = s.post; a.pre = s.pre; a.gate = s.gate;
  a.x_bf16 = s.x_dtype == DISCO_BF16; a.h_bf16 = s.h_dtype == DISCO_BF16;
  a.eps_post = s.eps_post; a.eps_pre = s.eps_pre; a.x_scale = s.x_scale; a.h_scale = s.h_scale; a.inv_d = 1.f / (float)s.d;
  return a;
}

int lanes_of(int64_t d) {
  int lanes = 16;
  while (lanes * COLS < d) lanes *= 2;
  return lanes;
}
bool narrow_of(const disco_block_norm_shape& s) { return s.x_dtype == DISCO_BF16 && s.h_dtype == DISCO_BF16; }
// Workgroups: what the chip holds at once.  Each walks its rows with its parameters at hand, and none waits for another to end (39424 x 512 bf16 forward,
// 5 waves a SIMD: 32 us; 3.2 times as many workgroups 41, one for each four rows 79).
int64_t blocks_of(const disco_block_norm_shape& s, int waves) {
  const int lanes = lanes_of(s.d), each = lanes > 256 ? lanes / 256 : 1;
  const int64_t rows = lanes > 256 ? 1 : 256 / lanes, all = (s.rows + rows - 1) / rows, most = 256 * (waves < each ? 1 : waves / each);
  return all < most ? all : most;
}
template <class F>
void with_bool(bool v, F f) {
  if (v) f(std::true_type());
  else f(std::false_type());
}
template <class F>
void with_lanes(int64_t d, F f) {
  switch (lanes_of(d)) {
    case 16: return f(std::integral_constant<int, 16>());
    case 32: return f(std::integral_constant<int, 32>());
    case 64: return f(std::integral_constant<int, 64>());
    case 128: return f(std::integral_constant<int, 128>());
    case 256: return f(std::integral_constant<int, 256>());
    case 512: return f(std::integral_constant<int, 512>());
    default: return f(std::integral_constant<int, 1024>());
  }
}

// f(a norm after the block, one before the next, all rows bf16), as constants
template <class F>
void with_form(const disco_block_norm_shape& s, F f) {
  with_bool(s.post != DISCO_NORM_NONE, [&](auto post) {
    with_bool(s.pre != DISCO_NORM_NONE, [&](auto pre) { with_bool(narrow_of(s), [&](auto narrow) { f(post, pre, narrow); }); });
  });
}
int64_t bwd_blocks(const disco_block_norm_shape& s) {
  int64_t n = 0;
  with_form(s, [&](auto post, auto pre, auto narrow) { n = blocks_of(s, waves_bwd<post(), pre(), narrow()>()); });
  return n;
}

}  // namespace
}  // namespace disco

using namespace disco;

extern "C" size_t disco_block_norm_workspace_bytes(const disco_block_norm_shape* shape) {
  if (check(shape) != DISCO_OK) return 0;
  return align_up((size_t)bwd_blocks(*shape) * SUMS * (size_t)shape->d * sizeof(float));
}

extern "C" int disco_block_norm_fwd(const disco_block_norm_shape* shape, const void* x, const void* h, const void* gate, const float* w_post,
                                    const float* b_post, const float* w_pre, const float* b_pre, void* y, void* n, float* stats,
                                    void* hip_stream) {
  if (!shape || !h || !y || !stats) return DISCO_ERR_NULL;
  if (const int st = check(shape)) return st;
  if ((shape->gate != DISCO_GATE_NONE && !gate) || (shape->pre != DISCO_NORM_NONE && !n)) return DISCO_ERR_NULL;
  Args a = args_of(*shape);
  for (const void* p : {x, static_cast<const void*>(y)})
    if (!aligned(p, a.x_bf16)) return DISCO_ERR_UNSUPPORTED;
  for (const void* p : {h, static_cast<const void*>(n)})
    if (!aligned(p, a.h_bf16)) return DISCO_ERR_UNSUPPORTED;
  if (!aligned(gate, a.h_bf16 && a.gate == DISCO_GATE_ELEMENT)) return DISCO_ERR_UNSUPPORTED;
  for (const void* p : {w_post, b_post, w_pre, b_pre, static_cast<const float*>(stats)})
    if (!aligned(p, 0)) return DISCO_ERR_UNSUPPORTED;
  a.x = x; a.h = h; a.gate_values = gate; a.w_post = w_post; a.b_post = b_post; a.w_pre = w_pre; a.b_pre = b_pre;
  a.out_y = y; a.out_n = n; a.stats = stats;
  hipStream_t st = static_cast<hipStream_t>(hip_stream);
  with_lanes(a.d, [&](auto lanes) {
    constexpr int L = lanes(), B = L > 256 ? L : 256;
    with_form(*shape, [&](auto post, auto pre, auto narrow) {
      const unsigned grid = (unsigned)blocks_of(*shape, waves_fwd<post(), pre()>());
      k_block_norm_fwd<L, post(), pre(), narrow()><<<grid, B, 0, st>>>(a);
    });
  });
  return hipGetLastError() == hipSuccess ? DISCO_OK : DISCO_ERR_HIP;
}

extern "C" int disco_block_norm_bwd(const disco_block_norm_shape* shape, const void* dy, const void* dn, const void* h, const void* y, const void* gate,
                                    const float* w_post, const float* b_post, const float* w_pre, const float* stats, void* dx, void* dh, void* dgate,
                                    float* dw_post, float* db_post, float* dw_pre, float* db_pre, void* workspace, size_t workspace_bytes,
                                    void* hip_stream) {
  if (!shape || !dh) return DISCO_ERR_NULL;
  if (const int st = check(shape)) return st;
  const bool post = shape->post != DISCO_NORM_NONE, pre = shape->pre != DISCO_NORM_NONE, gated = shape->gate != DISCO_GATE_NONE;
  if ((gated && !gate) || ((gated || post) && !h) || (pre && (!dn || !y)) || (!pre && !dy) || ((post || pre) && !stats)) return DISCO_ERR_NULL;
  Args a = args_of(*shape);
  for (const void* p : {dy, y, static_cast<const void*>(dx)})
    if (!aligned(p, a.x_bf16)) return DISCO_ERR_UNSUPPORTED;
  for (const void* p : {dn, h, static_cast<const void*>(dh)})
    if (!aligned(p, a.h_bf16)) return DISCO_ERR_UNSUPPORTED;
  for (const void* p : {gate, static_cast<const void*>(dgate)})
    if (!aligned(p, a.h_bf16 && a.gate == DISCO_GATE_ELEMENT)) return DISCO_ERR_UNSUPPORTED;
  for (const void* p : {w_post, b_post, w_pre, stats, static_cast<const float*>(dw_post), static_cast<const float*>(db_post),
                        static_cast<const float*>(dw_pre), static_cast<const float*>(db_pre)})
    if (!aligned(p, 0)) return DISCO_ERR_UNSUPPORTED;
  if (!workspace || (reinterpret_cast<uintptr_t>(workspace) & 255) != 0 || workspace_bytes < disco_block_norm_workspace_bytes(shape))
    return DISCO_ERR_WORKSPACE;
  a.dy = dy; a.dn = dn; a.h = h; a.y = y; a.gate_values = gate; a.w_post = w_post; a.b_post = b_post; a.w_pre = w_pre;
  a.stats = const_cast<float*>(stats); a.dx = dx; a.dh = dh;
  a.dgate_rows = a.gate == DISCO_GATE_ELEMENT ? dgate : nullptr;
  a.sums[0] = a.gate == DISCO_GATE_CHANNEL ? static_cast<float*>(dgate) : nullptr;
  if (a.post) { a.sums[1] = dw_post; a.sums[2] = db_post; }
  if (a.pre) { a.sums[3] = dw_pre; a.sums[4] = db_pre; }
  for (float* s : a.sums) a.wanted += s != nullptr;
  a.parts = static_cast<float*>(workspace);
  const unsigned grid = (unsigned)bwd_blocks(*shape);
  hipStream_t st = static_cast<hipStream_t>(hip_stream);
  with_lanes(a.d, [&](auto lanes) {
    constexpr int L = lanes(), B = L > 256 ? L : 256;
    with_form(*shape, [&](auto post, auto pre, auto narrow) { k_block_norm_bwd<L, post(), pre(), narrow()><<<grid, B, 0, st>>>(a); });
  });
  if (hipGetLastError() != hipSuccess) return DISCO_ERR_HIP;
  if (a.wanted && grid > 1) k_block_norm_sums<<<dim3((unsigned)((a.d + 63) / 64), (unsigned)a.wanted), 1024, 0, st>>>(a, (int)grid);
  return hipGetLastError() == hipSuccess ? DISCO_OK : DISCO_ERR_HIP;
}
