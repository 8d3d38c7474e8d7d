// Global gradient norm over many tensors, clipping by it, and the clipped SGD step of the digital parameters (normalisations, low-rank
// adapters): few launches for a whole network's tensors instead of a handful per tensor.  The squares are summed in double precision in
// a fixed order (a float's square is exact there and 2^200 of them do not overflow), so the result does not depend on the run.  HBM-bound: 45
// million elements 34 us for the norm (5.3 TB/s), 83 for the step (6.6 TB/s, part of the gradients from the caches), 58 for clipping them.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstdint>

#include "xbar.h"

namespace {

inline size_t align256(size_t x) { return (x + 255) & ~(size_t)255; }
inline int launched() { return hipGetLastError() == hipSuccess ? XBAR_OK : XBAR_EHIP; }

constexpr int kTensors = 128;          // of one launch: their table travels with the kernel's arguments (at most 4 KB)
typedef float f4 __attribute__((ext_vector_type(4)));

constexpr int kLoads = 4;              // quads of a thread in a whole chunk
constexpr size_t kChunk = 1024 * kLoads;   // elements that a block takes at a time, of one tensor
constexpr int kBlocks = 2048;          // of one launch

struct Table {
  const float* g[kTensors];
  float* p[kTensors];
  unsigned long long n[kTensors];
  uint32_t first[kTensors + 1];        // chunks before tensor i
  int tensors;
};
static_assert(sizeof(Table) + 64 <= 4096, "kernel arguments");

// The chunk's tensor, and its elements from and to.
struct Piece {
  int tensor;
  size_t from, to;
  __device__ __forceinline__ Piece(const Table& t, uint32_t chunk, size_t each = kChunk) {
    int lo = 0, hi = t.tensors - 1;    // the last tensor with first <= chunk (tensors without elements have no chunk)
    while (lo < hi) {
      const int mid = (lo + hi + 1) >> 1;
      if (t.first[mid] <= chunk) lo = mid;
      else hi = mid - 1;
    }
    tensor = lo;
    from = (size_t)(chunk - t.first[lo]) * each;
    to = from + each < t.n[lo] ? from + each : (size_t)t.n[lo];
  }
};

// Sum over a block's 256 threads in a fixed order, to all of them.
__device__ __forceinline__ double block_sum(double s, double (&red)[4]) {
#pragma unroll
  for (int d = 32; d; d >>= 1) s += __shfl_xor(s, d, 64);
  __syncthreads();
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = s;
  __syncthreads();
  return (red[0] + red[1]) + (red[2] + red[3]);
}

__device__ __forceinline__ void add_squares(double& s, const f4& v) {
#pragma unroll
  for (int e = 0; e < 4; ++e) s = __builtin_fma((double)v[e], (double)v[e], s);
}

// The norm of a few short tensors in one launch: one block, a wave takes every sixteenth piece of 1024 elements.
constexpr size_t kShort = 65536;       // elements in all
constexpr size_t kPiece = 1024;
__global__ __launch_bounds__(1024) void norm_short_kernel(const Table t, float* norm) {
  __shared__ double red[16];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  double s = 0.0;
  for (uint32_t piece = wave; piece < t.first[t.tensors]; piece += 16) {
    const Piece at(t, piece, kPiece);
    const float* g = t.g[at.tensor] + at.from;
    const int n = (int)(at.to - at.from);
    f4 v[4];
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      const int i = 256 * u + 4 * lane;
      v[u] = f4{0.0f, 0.0f, 0.0f, 0.0f};
      if (i + 3 < n) {
        v[u] = *reinterpret_cast<const f4*>(g + i);
      } else {
#pragma unroll
        for (int e = 0; e < 3; ++e)
          if (i + e < n) v[u][e] = g[i + e];
      }
    }
#pragma unroll
    for (int u = 0; u < 4; ++u) add_squares(s, v[u]);
  }
#pragma unroll
  for (int d = 32; d; d >>= 1) s += __shfl_xor(s, d, 64);
  if (lane == 0) red[wave] = s;
  __syncthreads();
  if (threadIdx.x == 0) {
    s = 0.0;
    for (int w = 0; w < 16; ++w) s += red[w];
    norm[0] = (float)::sqrt(s);
  }
}

__global__ __launch_bounds__(256) void norm_partial_kernel(const Table t, double* part) {
  __shared__ double red[4];
  double s = 0.0;
  for (uint32_t chunk = blockIdx.x; chunk < t.first[t.tensors]; chunk += gridDim.x) {
    const Piece at(t, chunk);
    const float* g = t.g[at.tensor];
    const f4* quads = reinterpret_cast<const f4*>(g + at.from) + threadIdx.x;
    if (at.to - at.from == kChunk) {                         // a whole chunk: all its loads in flight
      f4 v[kLoads];
#pragma unroll
      for (int u = 0; u < kLoads; ++u) v[u] = quads[256 * u];
#pragma unroll
      for (int u = 0; u < kLoads; ++u) add_squares(s, v[u]);
      continue;
    }
    const size_t last = (at.to - at.from) >> 2;
    for (size_t q = threadIdx.x; q < last; q += 256) add_squares(s, quads[q - threadIdx.x]);
    const size_t odd = at.from + (last << 2) + threadIdx.x;  // up to three, behind the tensor's last quad
    if (odd < at.to) s = __builtin_fma((double)g[odd], (double)g[odd], s);
  }
  s = block_sum(s, red);
  if (threadIdx.x == 0) part[blockIdx.x] = s;
}

__device__ __forceinline__ double total_of(const double* part, int parts, double (&red)[4]) {
  double s = 0.0;
  for (int k = threadIdx.x; k < parts; k += 256) s += part[k];
  return block_sum(s, red);
}

__global__ __launch_bounds__(256) void norm_final_kernel(const double* part, int parts, float* norm) {
  __shared__ double red[4];
  const double total = total_of(part, parts, red);
  if (threadIdx.x == 0) norm[0] = (float)::sqrt(total);
}

// g clipped: in double precision, where a factor that no float holds is one too, and rounded once.
__device__ __forceinline__ float clipped(float g, double c) { return (float)((double)g * c); }
// As the sgd kernel's step.
__device__ __forceinline__ float stepped(float p, float g, float lr) { return p - lr * g; }

// Parameters pass through once and leave the caches to the gradients, which are read twice (45 million elements: the two passes 50 + 89 us
// with ordinary loads and stores of the parameters -- the norm's pass then also waits for what the last step left to be written
// back --, 34 + 83 with these; reading the gradients from the back makes no difference).
// STEP: p <- p - lr (c g), else g <- c g; c = max_norm / norm where the norm is larger.  Every block adds up the partial sums itself.
template <bool STEP>
__global__ __launch_bounds__(256) void clip_kernel(const Table t, const double* part, int parts, float lr, float max_norm, float* norm) {
  __shared__ double red[4];
  const double total = total_of(part, parts, red), size = ::sqrt(total);
  if (norm && blockIdx.x == 0 && threadIdx.x == 0) norm[0] = (float)size;
  if (!(total < INFINITY)) return;                           // infinities or NaN among the gradients: nothing is moved
  const double c = size > (double)max_norm ? (double)max_norm / size : 1.0;
  if (!STEP && c == 1.0) return;
  for (uint32_t chunk = blockIdx.x; chunk < t.first[t.tensors]; chunk += gridDim.x) {
    const Piece at(t, chunk);
    const float* g = t.g[at.tensor];
    float* p = t.p[at.tensor];
    const f4* from = reinterpret_cast<const f4*>(g + at.from) + threadIdx.x;
    f4* to = reinterpret_cast<f4*>(p + at.from) + threadIdx.x;
    if (at.to - at.from == kChunk) {
      f4 v[kLoads], u[kLoads];
#pragma unroll
      for (int k = 0; k < kLoads; ++k) {
        v[k] = from[256 * k];
        if (STEP) u[k] = __builtin_nontemporal_load(to + 256 * k);
      }
#pragma unroll
      for (int k = 0; k < kLoads; ++k) {
#pragma unroll
        for (int e = 0; e < 4; ++e) v[k][e] = STEP ? stepped(u[k][e], clipped(v[k][e], c), lr) : clipped(v[k][e], c);
        if (STEP) __builtin_nontemporal_store(v[k], to + 256 * k);
        else to[256 * k] = v[k];
      }
      continue;
    }
    const size_t last = (at.to - at.from) >> 2;
    for (size_t q = threadIdx.x; q < last; q += 256) {
      f4 v = from[q - threadIdx.x];
      if (STEP) {
        const f4 u = to[q - threadIdx.x];
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] = stepped(u[e], clipped(v[e], c), lr);
      } else {
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] = clipped(v[e], c);
      }
      to[q - threadIdx.x] = v;
    }
    const size_t odd = at.from + (last << 2) + threadIdx.x;
    if (odd < at.to) p[odd] = STEP ? stepped(p[odd], clipped(g[odd], c), lr) : clipped(g[odd], c);
  }
}

struct Range {
  uintptr_t from, to;
  int written;
};

// Whether something that is written lies in one of the other ranges.
bool written_twice(Range* r, int n) {
  std::sort(r, r + n, [](const Range& a, const Range& b) { return a.from < b.from; });
  uintptr_t read_end = 0, written_end = 0;
  for (int i = 0; i < n; ++i) {
    if (r[i].from < written_end || (r[i].written && r[i].from < read_end)) return true;
    uintptr_t& end = r[i].written ? written_end : read_end;
    end = std::max(end, r[i].to);
  }
  return false;
}

int checked(const float* const* params, const float* const* grads, const size_t* sizes, int tensors, bool writes, const float* norm,
            const void* ws, size_t ws_bytes) {
  if (!grads || !sizes) return XBAR_EINVAL;
  if (tensors <= 0 || tensors > XBAR_GRADS_MAX_TENSORS) return XBAR_ESHAPE;
  size_t total = 0;
  for (int i = 0; i < tensors; ++i) {
    if (sizes[i] >= ((size_t)1 << 38) || (total += sizes[i]) >= ((size_t)1 << 40)) return XBAR_ESHAPE;
    if (sizes[i] && (!grads[i] || (reinterpret_cast<uintptr_t>(grads[i]) & 15u))) return XBAR_EALIGN;
    if (sizes[i] && params && (!params[i] || (reinterpret_cast<uintptr_t>(params[i]) & 15u))) return XBAR_EALIGN;
  }
  if (!norm || (reinterpret_cast<uintptr_t>(norm) & 15u) || !ws || (reinterpret_cast<uintptr_t>(ws) & 15u)) return XBAR_EALIGN;
  if (ws_bytes < xbar_grads_workspace_bytes(tensors)) return XBAR_EWORKSPACE;
  Range ranges[2 * XBAR_GRADS_MAX_TENSORS + 2];
  int n = 0;
  const uintptr_t to_norm = reinterpret_cast<uintptr_t>(norm), to_ws = reinterpret_cast<uintptr_t>(ws);
  ranges[n++] = Range{to_norm, to_norm + sizeof(float), 1};
  ranges[n++] = Range{to_ws, to_ws + xbar_grads_workspace_bytes(tensors), 1};
  for (int i = 0; i < tensors; ++i) {
    if (!sizes[i]) continue;
    const uintptr_t g = reinterpret_cast<uintptr_t>(grads[i]);
    ranges[n++] = Range{g, g + 4 * sizes[i], writes && !params};
    if (params) {
      const uintptr_t p = reinterpret_cast<uintptr_t>(params[i]);
      ranges[n++] = Range{p, p + 4 * sizes[i], 1};
    }
  }
  if (written_twice(ranges, n)) return XBAR_EINVAL;
  return XBAR_OK;
}

// The tables of the launches, one after another.
struct Launches {
  const float* const* params;
  const float* const* grads;
  const size_t* sizes;
  int tensors, next = 0;
  size_t each = kChunk;
  Table t;
  unsigned blocks = 0;
  bool more() {
    t.tensors = 0;
    t.first[0] = 0;
    while (next < tensors && t.tensors < kTensors) {
      const size_t chunks = (sizes[next] + each - 1) / each;
      if (chunks) {
        t.g[t.tensors] = grads[next];
        t.p[t.tensors] = const_cast<float*>(params ? params[next] : grads[next]);
        t.n[t.tensors] = sizes[next];
        t.first[t.tensors + 1] = t.first[t.tensors] + (uint32_t)chunks;
        ++t.tensors;
      }
      ++next;
    }
    blocks = std::min<unsigned>(t.first[t.tensors], kBlocks);
    return t.tensors > 0;
  }
};

int partial_sums(Launches l, double* part, int* parts, hipStream_t st) {
  *parts = 0;
  while (l.more()) {
    hipLaunchKernelGGL(norm_partial_kernel, dim3(l.blocks), dim3(256), 0, st, l.t, part + *parts);
    if (launched()) return XBAR_EHIP;
    *parts += (int)l.blocks;
  }
  return XBAR_OK;
}

template <bool STEP>
int clip(const float* const* params, const float* const* grads, const size_t* sizes, int tensors, float lr, float max_norm, float* norm,
         double* part, hipStream_t st) {
  Launches l{params, grads, sizes, tensors};
  int parts;
  if (partial_sums(l, part, &parts, st)) return XBAR_EHIP;
  bool first = true;
  while (l.more()) {
    hipLaunchKernelGGL(clip_kernel<STEP>, dim3(l.blocks), dim3(256), 0, st, l.t, part, parts, lr, max_norm, first ? norm : nullptr);
    if (launched()) return XBAR_EHIP;
    first = false;
  }
  if (first) {                                               // no elements at all: the norm is 0
    hipLaunchKernelGGL(norm_final_kernel, dim3(1), dim3(256), 0, st, part, 0, norm);
    return launched();
  }
  return XBAR_OK;
}

}  // namespace

extern "C" {

size_t xbar_grads_workspace_bytes(int tensors) {
  if (tensors <= 0 || tensors > XBAR_GRADS_MAX_TENSORS) return 0;
  return align256((size_t)((tensors + kTensors - 1) / kTensors) * kBlocks * sizeof(double));
}

int xbar_grad_norm(const float* const* grads, const size_t* sizes, int tensors, float* norm, void* ws, size_t ws_bytes, void* hip_stream) {
  const int rc = checked(nullptr, grads, sizes, tensors, false, norm, ws, ws_bytes);
  if (rc) return rc;
  hipStream_t st = reinterpret_cast<hipStream_t>(hip_stream);
  double* part = reinterpret_cast<double*>(ws);
  size_t total = 0;
  for (int i = 0; i < tensors; ++i) total += sizes[i];
  Launches l{nullptr, grads, sizes, tensors, 0, kPiece};
  if (total <= kShort && tensors <= kTensors && l.more()) {
    hipLaunchKernelGGL(norm_short_kernel, dim3(1), dim3(1024), 0, st, l.t, norm);
    return launched();
  }
  int parts;
  if (partial_sums(Launches{nullptr, grads, sizes, tensors}, part, &parts, st)) return XBAR_EHIP;
  hipLaunchKernelGGL(norm_final_kernel, dim3(1), dim3(256), 0, st, part, parts, norm);
  return launched();
}

int xbar_grad_clip(float* const* grads, const size_t* sizes, int tensors, float max_norm, float* norm, void* ws, size_t ws_bytes,
                   void* hip_stream) {
  const int rc = checked(nullptr, grads, sizes, tensors, true, norm, ws, ws_bytes);
  if (rc) return rc;
  if (!(max_norm > 0.0f)) return XBAR_EINVAL;
  return clip<false>(nullptr, grads, sizes, tensors, 0.0f, max_norm, norm, reinterpret_cast<double*>(ws),
                     reinterpret_cast<hipStream_t>(hip_stream));
}

int xbar_clip_sgd(float* const* params, const float* const* grads, const size_t* sizes, int tensors, float lr, float max_norm, float* norm,
                  void* ws, size_t ws_bytes, void* hip_stream) {
  if (!params) return XBAR_EINVAL;
  const int rc = checked(params, grads, sizes, tensors, true, norm, ws, ws_bytes);
  if (rc) return rc;
  if (!(max_norm > 0.0f) || !std::isfinite(lr)) return XBAR_EINVAL;
  return clip<true>(params, grads, sizes, tensors, lr, max_norm, norm, reinterpret_cast<double*>(ws),
                    reinterpret_cast<hipStream_t>(hip_stream));
}

}  // extern "C"
