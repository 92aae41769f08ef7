// Global norm of many gradients and clipping by it:  norm = sqrt(sum g^2),  dst = g min(1, max_norm / (norm + 1e-6)).
//
// Bound by memory: every gradient is read for the norm and again for the product, which needs all of them, and written once.  The tensors' pointers
// and sizes travel as kernel arguments, TABLE tensors a launch, so that a call copies nothing to the device, can be captured, and depends on no
// memory of the host's after it returns.  Inside a launch the tensors are cut into pieces of PIECE elements, dealt to the workgroups in turn,
// so that a launch is as even with one large tensor as with a hundred small ones.  150 million fp32 gradients in 292 tensors, three launches of either
// kernel: squares 132 us (4.5 TB/s), products 230 (5.2 TB/s), 5 for the sum of the squares between them; a few gradients in 4 tensors: 15 us, the launches.
//
// Squares are summed in fp64: a tower's 10^8 of them lose nothing, and the rate of fp64 is far above that of the memory.
#include "common.h"

#include <math.h>

namespace disco {
namespace {

typedef __attribute__((ext_vector_type(4))) uint32_t u32x4;

constexpr int TABLE = 112;                        // tensors a launch: 112 x 32 bytes of arguments
constexpr int THREADS = 256, UNROLL = 4;
constexpr int PIECE = THREADS * UNROLL * 8;       // elements: 16-byte loads of bf16, two of fp32
constexpr int BLOCKS = 2048;                      // workgroups a launch at most

struct Tensor { const void* src; void* dst; int64_t n; int32_t first; int32_t bf16; };      // first: its first piece
struct Table { Tensor t[TABLE]; int32_t count, pieces; };
static_assert(sizeof(Table) <= 3640, "kernel arguments");

struct __attribute__((packed, aligned(2))) Any16 { u32x4 v; };

// The tensor that piece p lies in: the last one that starts at or before it (tensors without elements have no pieces and are not listed).
__device__ __forceinline__ int tensor_of(const Table& table, int p) {
  int lo = 0, hi = table.count;
  while (hi - lo > 1) {
    const int mid = (lo + hi) / 2;
    if (table.t[mid].first <= p) lo = mid;
    else hi = mid;
  }
  return lo;
}

struct Eight { u32x4 a, b; };
__device__ __forceinline__ Eight load8(const void* p, int64_t at, int64_t n, bool bf16) {
  Eight r = {u32x4{0, 0, 0, 0}, u32x4{0, 0, 0, 0}};
  if (bf16) {
    const uint16_t* q = static_cast<const uint16_t*>(p) + at;
    if (at + 8 <= n) r.a = reinterpret_cast<const Any16*>(q)->v;
    else {
#pragma unroll
      for (int e = 0; e < 8; ++e)
        if (at + e < n) r.a[e / 2] |= (uint32_t)q[e] << (e % 2 * 16);
    }
  } else {
    const uint32_t* q = static_cast<const uint32_t*>(p) + at;
    if (at + 8 <= n) {
      r.a = reinterpret_cast<const Any16*>(q)->v;
      r.b = reinterpret_cast<const Any16*>(q + 4)->v;
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e)
        if (at + e < n) (e < 4 ? r.a : r.b)[e % 4] = q[e];
    }
  }
  return r;
}
__device__ __forceinline__ void values(const Eight& r, bool bf16, float (&v)[8]) {
#pragma unroll
  for (int e = 0; e < 8; ++e)
    v[e] = __uint_as_float(!bf16 ? (e < 4 ? r.a : r.b)[e % 4] : e % 2 ? r.a[e / 2] & 0xffff0000u : r.a[e / 2] << 16);
}
__device__ __forceinline__ uint32_t bf16_bits(float f) { return __builtin_bit_cast(uint16_t, (__bf16)f); }      // to nearest even
__device__ __forceinline__ void store8(void* p, int64_t at, int64_t n, bool bf16, const float (&v)[8]) {
  if (bf16) {
    uint16_t* q = static_cast<uint16_t*>(p) + at;
    if (at + 8 <= n) {
      u32x4 w;
#pragma unroll
      for (int e = 0; e < 4; ++e) w[e] = bf16_bits(v[2 * e]) | bf16_bits(v[2 * e + 1]) << 16;
      reinterpret_cast<Any16*>(q)->v = w;
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e)
        if (at + e < n) q[e] = (uint16_t)bf16_bits(v[e]);
    }
  } else {
    float* q = static_cast<float*>(p) + at;
    if (at + 8 <= n) {
      u32x4 lo, hi;
#pragma unroll
      for (int e = 0; e < 4; ++e) { lo[e] = __float_as_uint(v[e]); hi[e] = __float_as_uint(v[4 + e]); }
      reinterpret_cast<Any16*>(q)->v = lo;
      reinterpret_cast<Any16*>(q + 4)->v = hi;
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e)
        if (at + e < n) q[e] = v[e];
    }
  }
}

__device__ __forceinline__ double block_sum(double s) {
  __shared__ double part[16];
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) s += __shfl_xor(s, o);
  if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = s;
  __syncthreads();
  s = 0.0;
  for (int w = 0; w < (int)blockDim.x / 64; ++w) s += part[w];
  return s;
}

__global__ __launch_bounds__(THREADS) void k_grad_squares(Table table, double* parts) {
  double s = 0.0;
  for (int p = blockIdx.x; p < table.pieces; p += gridDim.x) {
    const Tensor& t = table.t[tensor_of(table, p)];
    const int64_t from = (int64_t)(p - t.first) * PIECE + threadIdx.x * 8;
    Eight r[UNROLL];
#pragma unroll
    for (int u = 0; u < UNROLL; ++u) r[u] = load8(t.src, from + u * THREADS * 8, t.n, t.bf16);
#pragma unroll
    for (int u = 0; u < UNROLL; ++u) {
      float v[8];
      values(r[u], t.bf16, v);
#pragma unroll
      for (int e = 0; e < 8; ++e) s = fma((double)v[e], (double)v[e], s);
    }
  }
  s = block_sum(s);
  if (threadIdx.x == 0) parts[blockIdx.x] = s;
}

__device__ __forceinline__ double sum_of(const double* parts, int n) {
  double s = 0.0;
#pragma unroll 4
  for (int i = threadIdx.x; i < n; i += blockDim.x) s += parts[i];
  return block_sum(s);
}

// The sum of the squares takes the place of the first partial sum, for the product.
__global__ __launch_bounds__(1024) void k_grad_norm(double* parts, int n, int accumulate, float* norm) {
  double s = sum_of(parts, n);
  if (threadIdx.x == 0) {
    parts[0] = s;
    if (accumulate) s = fma((double)*norm, (double)*norm, s);
    *norm = (float)sqrt(s);
  }
}

// The pieces run from the end of a tensor (and the host's tables from the end of the list): what the norm read last is still in the last-level
// cache.  Few partial sums are joined by every workgroup for itself, the norm's own launch is saved: all of them take the same order, so
// they come to the same norm, and the first one stores it.  Of many k_grad_norm has left one (n = 1); a given norm has none (n = 0).
// Norm and factor are fp64 up to the product: a norm beyond fp32, of gradients that are all finite, has a factor like any other.
__global__ __launch_bounds__(THREADS) void k_grad_scale(Table table, float max_norm, float* norm, const double* parts, int n) {
  double taken;
  if (n) {
    taken = sqrt(n == 1 ? parts[0] : sum_of(parts, n));
    if (blockIdx.x == 0 && threadIdx.x == 0) *norm = (float)taken;
  } else {
    taken = *norm;
  }
  const double quotient = max_norm / (taken + 1e-6), factor = quotient < 1.0 ? quotient : taken == taken ? 1.0 : taken;
  for (int p = blockIdx.x; p < table.pieces; p += gridDim.x) {
    const Tensor& t = table.t[tensor_of(table, p)];
    if (factor == 1.0 && t.src == t.dst) continue;
    const int64_t from = ((t.n + PIECE - 1) / PIECE - 1 - (p - t.first)) * PIECE + threadIdx.x * 8;
    Eight r[UNROLL];
#pragma unroll
    for (int u = 0; u < UNROLL; ++u) r[u] = load8(t.src, from + u * THREADS * 8, t.n, t.bf16);
#pragma unroll
    for (int u = 0; u < UNROLL; ++u) {
      float v[8];
      values(r[u], t.bf16, v);
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e] = (float)(v[e] * factor);
      store8(t.dst, from + u * THREADS * 8, t.n, t.bf16, v);
    }
  }
}

__global__ void k_grad_keep(const float* given, float* norm) {
  if (threadIdx.x == 0) *norm = *given;
}

constexpr int64_t MOST_TENSORS = (int64_t)1 << 20;
// fp64 partial sums of every launch
int64_t parts_of(int64_t count) { return (count / TABLE + 1) * BLOCKS; }

int check(const void* const* src, void* const* dst, const int64_t* elements, const int32_t* dtypes, int64_t count, bool writes) {
  if (count < 0 || count > MOST_TENSORS) return DISCO_ERR_SHAPE;
  if (count && (!src || !elements || !dtypes || (writes && !dst))) return DISCO_ERR_NULL;
  int64_t all = 0;
  for (int64_t i = 0; i < count; ++i) {
    if (elements[i] < 0 || elements[i] > (int64_t)1 << 40) return DISCO_ERR_SHAPE;
    if (elements[i] && (!src[i] || (writes && !dst[i]))) return DISCO_ERR_NULL;
    if (dtypes[i] != DISCO_F32 && dtypes[i] != DISCO_BF16) return DISCO_ERR_UNSUPPORTED;
    const uintptr_t mask = dtypes[i] == DISCO_BF16 ? 1 : 3;
    if ((reinterpret_cast<uintptr_t>(src[i]) | (writes ? reinterpret_cast<uintptr_t>(dst[i]) : 0)) & mask) return DISCO_ERR_UNSUPPORTED;
    all += elements[i] / PIECE + 1;
  }
  return all <= 0x7fffffff - BLOCKS ? DISCO_OK : DISCO_ERR_SHAPE;       // a workgroup counts pieces in 32 bits, up to its first that is not there
}

// f(table) for every TABLE tensors that have elements, from the list's first or from its last
template <class F>
bool tables(const void* const* src, void* const* dst, const int64_t* elements, const int32_t* dtypes, int64_t count, bool backwards, F f) {
  Table table;
  table.count = table.pieces = 0;
  for (int64_t k = 0; k < count; ++k) {
    const int64_t i = backwards ? count - 1 - k : k;
    if (elements[i]) {
      table.t[table.count++] = Tensor{src[i], dst ? dst[i] : nullptr, elements[i], table.pieces, dtypes[i] == DISCO_BF16};
      table.pieces += (int32_t)((elements[i] + PIECE - 1) / PIECE);
    }
    if (table.count == TABLE || (k + 1 == count && table.count)) {
      if (!f(table)) return false;
      table.count = table.pieces = 0;
    }
  }
  return true;
}
unsigned grid_of(const Table& t) { return (unsigned)(t.pieces < BLOCKS ? t.pieces : BLOCKS); }

// The squares' partial sums: how many (-1: a launch failed)
int squares(const void* const* src, const int64_t* elements, const int32_t* dtypes, int64_t count, double* parts, hipStream_t st) {
  int n = 0;
  const bool ok = tables(src, nullptr, elements, dtypes, count, false, [&](const Table& table) {
    k_grad_squares<<<grid_of(table), THREADS, 0, st>>>(table, parts + n);
    n += (int)grid_of(table);
    return hipGetLastError() == hipSuccess;
  });
  return ok ? n : -1;
}
bool norm_of(double* parts, int n, int accumulate, float* norm, hipStream_t st) {
  k_grad_norm<<<1, 1024, 0, st>>>(parts, n, accumulate, norm);
  return hipGetLastError() == hipSuccess;
}
// Partial sums that every workgroup joins for itself: up to four a thread.
constexpr int FEW = 4 * THREADS;

bool workspace_ok(const void* ws, size_t bytes, int64_t count) {
  return ws && (reinterpret_cast<uintptr_t>(ws) & 255) == 0 && bytes >= disco_grad_workspace_bytes(count);
}

}  // namespace
}  // namespace disco

using namespace disco;

extern "C" size_t disco_grad_workspace_bytes(int64_t count) {
  return count < 0 || count > MOST_TENSORS ? 0 : align_up((size_t)parts_of(count) * sizeof(double));
}

extern "C" int disco_grad_norm(const void* const* src, const int64_t* elements, const int32_t* dtypes, int64_t count, int accumulate, float* norm,
                               void* workspace, size_t workspace_bytes, void* hip_stream) {
  if (!norm) return DISCO_ERR_NULL;
  if (const int st = check(src, nullptr, elements, dtypes, count, false)) return st;
  if (reinterpret_cast<uintptr_t>(norm) & 3) return DISCO_ERR_UNSUPPORTED;
  if (!workspace_ok(workspace, workspace_bytes, count)) return DISCO_ERR_WORKSPACE;
  hipStream_t st = static_cast<hipStream_t>(hip_stream);
  double* parts = static_cast<double*>(workspace);
  const int n = squares(src, elements, dtypes, count, parts, st);
  return n >= 0 && norm_of(parts, n, accumulate, norm, st) ? DISCO_OK : DISCO_ERR_HIP;
}

extern "C" int disco_grad_clip(const void* const* src, void* const* dst, const int64_t* elements, const int32_t* dtypes, int64_t count, float max_norm,
                               const float* given, float* norm, void* workspace, size_t workspace_bytes, void* hip_stream) {
  if (!norm) return DISCO_ERR_NULL;
  if (const int st = check(src, dst, elements, dtypes, count, true)) return st;
  if (!(max_norm > 0.f)) return DISCO_ERR_SHAPE;
  if ((reinterpret_cast<uintptr_t>(norm) | reinterpret_cast<uintptr_t>(given)) & 3) return DISCO_ERR_UNSUPPORTED;
  if (!workspace_ok(workspace, workspace_bytes, count)) return DISCO_ERR_WORKSPACE;
  hipStream_t st = static_cast<hipStream_t>(hip_stream);
  double* parts = static_cast<double*>(workspace);
  int n = 0;
  if (!given) {
    n = squares(src, elements, dtypes, count, parts, st);
    if (n < 0) return DISCO_ERR_HIP;
    if (n == 0 || n > FEW) {
      if (!norm_of(parts, n, 0, norm, st)) return DISCO_ERR_HIP;
      n = 1;
    }
  } else if (given != norm) {
    k_grad_keep<<<1, 64, 0, st>>>(given, norm);
    if (hipGetLastError() != hipSuccess) return DISCO_ERR_HIP;
  }
  return tables(src, dst, elements, dtypes, count, true, [&](const Table& table) {
           k_grad_scale<<<grid_of(table), THREADS, 0, st>>>(table, max_norm, norm, parts, n);
           return hipGetLastError() == hipSuccess;
         }) ? DISCO_OK : DISCO_ERR_HIP;
}
