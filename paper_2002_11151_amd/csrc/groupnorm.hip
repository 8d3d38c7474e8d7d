// Group normalisation with an activation, channels last: the normalisation of a digital peripheral that needs no batch -- statistics
// per sample and group of neighbouring channels -- so that a network runs one request, or trains on small batches.
//   z = gamma (x - mean) invstd + beta (+ skip),  y = act(z)
// Evaluated in double precision up to z, rounded once.  HBM-bound elementwise and reduction work.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <cstdint>

#include "xbar.h"

namespace {

inline bool aligned16(const void* p) { return p != nullptr && (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }
inline size_t align256(size_t x) { return (x + 255) & ~(size_t)255; }
inline int launched() { return hipGetLastError() == hipSuccess ? XBAR_OK : XBAR_EHIP; }
inline bool overlap(const void* a, size_t na, const void* b, size_t nb) {
  const uintptr_t p = reinterpret_cast<uintptr_t>(a), q = reinterpret_cast<uintptr_t>(b);
  return a && b && p < q + nb && q < p + na;
}

// VEC consecutive floats of memory (one, or four from a 16-byte boundary).
template <int VEC>
__device__ __forceinline__ void load_vec(const float* p, float (&v)[VEC]) {
  if constexpr (VEC == 4) {
    const float4 q = *reinterpret_cast<const float4*>(p);
    v[0] = q.x; v[1] = q.y; v[2] = q.z; v[3] = q.w;
  } else {
    v[0] = *p;
  }
}
template <int VEC>
__device__ __forceinline__ void store_vec(float* p, const float (&v)[VEC]) {
  if constexpr (VEC == 4) *reinterpret_cast<float4*>(p) = make_float4(v[0], v[1], v[2], v[3]);
  else *p = v[0];
}

// Activation of z, and its derivative there.  A ReLU decides by the sign of the double value: the backward pass evaluates z again, in
// the same operations, and finds the same side.
template <int ACT>
__device__ __forceinline__ float act_of(double z) {
  const float f = (float)z;
  if constexpr (ACT == XBAR_ACT_RELU) return z > 0.0 ? f : 0.0f;
  if constexpr (ACT == XBAR_ACT_SILU) return f / (1.0f + expf(-f));
  return f;
}
template <int ACT>
__device__ __forceinline__ float act_bwd(double z, float dy) {
  if constexpr (ACT == XBAR_ACT_RELU) return z > 0.0 ? dy : 0.0f;
  if constexpr (ACT == XBAR_ACT_SILU) {
    const float f = (float)z, s = 1.0f / (1.0f + expf(-f));
    return dy * (s * (1.0f + f * (1.0f - s)));
  }
  return dy;
}

struct Shape {
  int batch, positions, channels, groups, per_group;      // per_group: channels of a group
  int rows;                                               // positions of a block
  int chunks;                                             // blocks along a sample's positions
};

// A channel's normalisation in one sample.
struct Norm {
  double gamma, beta, mean, invstd;
  __device__ __forceinline__ double xhat(float x) const { return ((double)x - mean) * invstd; }
  __device__ __forceinline__ double z(double xh) const { return __builtin_fma(gamma, xh, beta); }
};

template <int VEC>
__device__ __forceinline__ void load_norm(Norm (&nm)[VEC], const Shape& s, int b, int c, const float* gamma, const float* beta,
                                          const float* mean, const float* invstd) {
#pragma unroll
  for (int e = 0; e < VEC; ++e) {
    const int g = b * s.groups + (c + e) / s.per_group;
    nm[e] = Norm{(double)gamma[c + e], (double)beta[c + e], (double)mean[g], (double)invstd[g]};
  }
}

// Sums of a block's positions per channel: part[sample][chunk][channel][2].  Forward: of x - x0 and its square, x0 = the first value of
// the sample's group, which keeps the digits of a group whose mean is large beside its spread.  BWD: of the error behind the
// activation and of its product with xhat.  A thread takes VEC neighbouring channels, LANES threads a strip of channels.
template <bool BWD, int ACT, int VEC, int LANES>
__global__ __launch_bounds__(256) void gn_partial_kernel(const float* x, const float* dy, const float* gamma, const float* beta,
                                                         const float* skip, const float* mean, const float* invstd, double* part, Shape s) {
  constexpr int G = 256 / LANES, CT = VEC * LANES, VALUES = 2 * CT, SHARES = 256 / VALUES;
  __shared__ double red[2][G][CT];
  __shared__ double shares[SHARES][VALUES];
  const int lane = threadIdx.x % LANES, grp = threadIdx.x / LANES;
  const int c = blockIdx.y * CT + VEC * lane, C = s.channels;
  const int b = blockIdx.x / s.chunks, chunk = blockIdx.x - b * s.chunks;
  const size_t base = (size_t)b * s.positions;
  const int r0 = chunk * s.rows, r1 = min(r0 + s.rows, s.positions);
  double s0[VEC], s1[VEC];
#pragma unroll
  for (int e = 0; e < VEC; ++e) s0[e] = s1[e] = 0.0;
  if (c < C) {
    Norm nm[VEC];
    float x0[VEC];
    if (BWD) load_norm<VEC>(nm, s, b, c, gamma, beta, mean, invstd);
    else
#pragma unroll
      for (int e = 0; e < VEC; ++e) x0[e] = x[base * C + (c + e) / s.per_group * s.per_group];
#pragma unroll 4
    for (int r = r0 + grp; r < r1; r += G) {
      const size_t at = (base + r) * C + c;
      float v[VEC], d[VEC], k[VEC];
      load_vec<VEC>(x + at, v);
      if (BWD) load_vec<VEC>(dy + at, d);
      if (BWD && ACT != XBAR_ACT_NONE && skip) load_vec<VEC>(skip + at, k);
#pragma unroll
      for (int e = 0; e < VEC; ++e) {
        if (BWD) {
          const double xh = nm[e].xhat(v[e]);
          double z = nm[e].z(xh);
          if (ACT != XBAR_ACT_NONE && skip) z += (double)k[e];
          const double g = (double)act_bwd<ACT>(z, d[e]);
          s0[e] += g;
          s1[e] = __builtin_fma(g, xh, s1[e]);
        } else {
          const double u = (double)v[e] - (double)x0[e];
          s0[e] += u;
          s1[e] = __builtin_fma(u, u, s1[e]);
        }
      }
    }
  }
#pragma unroll
  for (int e = 0; e < VEC; ++e) {
    red[0][grp][VEC * lane + e] = s0[e];
    red[1][grp][VEC * lane + e] = s1[e];
  }
  __syncthreads();
  const int value = threadIdx.x % VALUES, share = threadIdx.x / VALUES;     // every sum in a fixed order
  double t = 0.0;
#pragma unroll
  for (int g = share; g < G; g += SHARES) t += red[value / CT][g][value % CT];
  shares[share][value] = t;
  __syncthreads();
  const int cv = blockIdx.y * CT + value % CT;
  if (threadIdx.x < VALUES && cv < C) {
    t = 0.0;
#pragma unroll
    for (int k = 0; k < SHARES; ++k) t += shares[k][value];
    part[((size_t)blockIdx.x * C + cv) * 2 + value / CT] = t;
  }
}

// One wave per sample and group: forward mean and 1 / std, backward the two means over the group that dx needs.
template <bool BWD>
__device__ __forceinline__ void group_of_wave(const double* part, const Shape& s, int item, const float* x, const float* gamma, float eps,
                                              float* mean, float* invstd, double* coef) {
  const int lane = threadIdx.x & 63, b = item / s.groups, g = item - b * s.groups;
  const int values = s.chunks * s.per_group;
  double s0 = 0.0, s1 = 0.0;
  for (int i = lane; i < values; i += 64) {
    const int chunk = i / s.per_group, c = g * s.per_group + (i - chunk * s.per_group);
    const double* p = part + (((size_t)b * s.chunks + chunk) * s.channels + c) * 2;
    const double f = BWD ? (double)gamma[c] : 1.0;
    s0 = __builtin_fma(f, p[0], s0);
    s1 = __builtin_fma(f, p[1], s1);
  }
#pragma unroll
  for (int d = 32; d; d >>= 1) {
    s0 += __shfl_xor(s0, d, 64);
    s1 += __shfl_xor(s1, d, 64);
  }
  if (lane) return;
  const double n = (double)s.positions * s.per_group;
  if (BWD) {
    coef[(size_t)item * 2] = s0 / n;
    coef[(size_t)item * 2 + 1] = s1 / n;
  } else {
    const double m = s0 / n, var = s1 / n - m * m;
    mean[item] = (float)((double)x[(size_t)b * s.positions * s.channels + g * s.per_group] + m);
    invstd[item] = (float)(1.0 / ::sqrt((var < 0.0 ? 0.0 : var) + (double)eps));
  }
}

__global__ __launch_bounds__(256) void gn_final_fwd_kernel(const double* part, Shape s, const float* x, float eps, float* mean, float* invstd) {
  const int item = blockIdx.x * 4 + (threadIdx.x >> 6);
  if (item < s.batch * s.groups) group_of_wave<false>(part, s, item, x, nullptr, eps, mean, invstd, nullptr);
}

// The first waves take a sample's group each, the others a channel: its parameters' gradients over the batch.
__global__ __launch_bounds__(256) void gn_final_bwd_kernel(const double* part, Shape s, const float* gamma, double* coef, float* dgamma,
                                                           float* dbeta) {
  int item = blockIdx.x * 4 + (threadIdx.x >> 6);
  if (item < s.batch * s.groups) {
    group_of_wave<true>(part, s, item, nullptr, gamma, 0.0f, nullptr, nullptr, coef);
    return;
  }
  item -= s.batch * s.groups;
  if (item >= s.channels) return;
  const int lane = threadIdx.x & 63, all = s.batch * s.chunks;
  double s0 = 0.0, s1 = 0.0;
  for (int i = lane; i < all; i += 64) {
    s0 += part[((size_t)i * s.channels + item) * 2];
    s1 += part[((size_t)i * s.channels + item) * 2 + 1];
  }
#pragma unroll
  for (int d = 32; d; d >>= 1) {
    s0 += __shfl_xor(s0, d, 64);
    s1 += __shfl_xor(s1, d, 64);
  }
  if (lane == 0) {
    dbeta[item] = (float)s0;
    dgamma[item] = (float)s1;
  }
}

// y, or dx and dskip; blocks and threads as in gn_partial_kernel.
template <bool BWD, int ACT, int VEC, int LANES>
__global__ __launch_bounds__(256) void gn_apply_kernel(const float* x, const float* dy, const float* gamma, const float* beta,
                                                       const float* skip, const float* mean, const float* invstd, const double* coef,
                                                       float* out, float* dskip, Shape s) {
  constexpr int G = 256 / LANES, CT = VEC * LANES;
  const int lane = threadIdx.x % LANES, grp = threadIdx.x / LANES;
  const int c = blockIdx.y * CT + VEC * lane, C = s.channels;
  if (c >= C) return;
  const int b = blockIdx.x / s.chunks, chunk = blockIdx.x - b * s.chunks;
  const size_t base = (size_t)b * s.positions;
  const int r0 = chunk * s.rows, r1 = min(r0 + s.rows, s.positions);
  Norm nm[VEC];
  load_norm<VEC>(nm, s, b, c, gamma, beta, mean, invstd);
  double m0[VEC], m1[VEC];
  if (BWD)
#pragma unroll
    for (int e = 0; e < VEC; ++e) {
      const size_t g = (size_t)b * s.groups + (c + e) / s.per_group;
      m0[e] = coef[g * 2];
      m1[e] = coef[g * 2 + 1];
    }
#pragma unroll 4
  for (int r = r0 + grp; r < r1; r += G) {
    const size_t at = (base + r) * C + c;
    float v[VEC], d[VEC], k[VEC], o[VEC], q[VEC];
    load_vec<VEC>(x + at, v);
    if (BWD) load_vec<VEC>(dy + at, d);
    if ((!BWD || ACT != XBAR_ACT_NONE) && skip) load_vec<VEC>(skip + at, k);
#pragma unroll
    for (int e = 0; e < VEC; ++e) {
      const double xh = nm[e].xhat(v[e]);
      double z = nm[e].z(xh);
      if ((!BWD || ACT != XBAR_ACT_NONE) && skip) z += (double)k[e];
      if (BWD) {
        q[e] = act_bwd<ACT>(z, d[e]);
        o[e] = (float)(nm[e].invstd * (nm[e].gamma * (double)q[e] - m0[e] - xh * m1[e]));
      } else {
        o[e] = act_of<ACT>(z);
      }
    }
    store_vec<VEC>(out + at, o);
    if (BWD && dskip) store_vec<VEC>(dskip + at, q);
  }
}

// Strips of 64 channels, or of 16 where the rows have no more than 32; a block takes 32 to 512 positions, about 2048 blocks in all.
struct Plan {
  Shape s;
  int vec, lanes;
  dim3 grid;
  Plan(int batch, int positions, int channels, int groups) {
    vec = channels % 4 == 0 ? 4 : 1;
    const int strip = channels <= 32 ? 16 : 64, strips = (channels + strip - 1) / strip;
    lanes = strip / vec;
    const long long wanted = ((long long)batch * positions * strips + 2047) / 2048;
    const int rows = (int)std::min<long long>(512, std::max<long long>(32, wanted));
    const int chunks = (positions + rows - 1) / rows;
    s = Shape{batch, positions, channels, groups, channels / groups, rows, chunks};
    grid = dim3((unsigned)(batch * chunks), (unsigned)strips);
  }
  size_t sums() const { return (size_t)s.batch * s.chunks * s.channels * 2; }
  size_t bytes() const { return align256(sums() * sizeof(double)) + align256((size_t)s.batch * s.groups * 2 * sizeof(double)); }
};

// The limits on a shape: elements below 2^38, blocks of a launch below 2^24.
int shape_ok(int batch, int positions, int channels, int groups) {
  if (batch <= 0 || positions <= 0 || channels <= 0 || groups <= 0 || channels % groups) return XBAR_ESHAPE;
  if ((double)batch * positions * channels >= 274877906944.0 || channels > (1 << 20) || (double)batch * groups >= 33554432.0) return XBAR_ESHAPE;
  return (double)batch * Plan(batch, positions, channels, groups).s.chunks >= 16777216.0 ? XBAR_ESHAPE : XBAR_OK;
}

template <template <int, int, int> class LAUNCH, class... ARGS>
void dispatch(int act, int vec, int lanes, ARGS... args) {
  auto with_act = [&](auto a) {
    constexpr int ACT = decltype(a)::value;
    if (vec == 4) {
      if (lanes == 4) LAUNCH<ACT, 4, 4>::go(args...);
      else LAUNCH<ACT, 4, 16>::go(args...);
    } else {
      if (lanes == 16) LAUNCH<ACT, 1, 16>::go(args...);
      else LAUNCH<ACT, 1, 64>::go(args...);
    }
  };
  if (act == XBAR_ACT_RELU) with_act(std::integral_constant<int, XBAR_ACT_RELU>());
  else if (act == XBAR_ACT_SILU) with_act(std::integral_constant<int, XBAR_ACT_SILU>());
  else with_act(std::integral_constant<int, XBAR_ACT_NONE>());
}

struct Fwd {
  const float *x, *gamma, *beta, *skip;
  float *y, *mean, *invstd;
};
struct Bwd {
  const float *x, *dy, *gamma, *beta, *skip, *mean, *invstd;
  float *dx, *dskip;
};

template <int ACT, int VEC, int LANES>
struct PartialFwd {
  static void go(const Plan* p, const Fwd* a, double* part, hipStream_t st) {
    hipLaunchKernelGGL((gn_partial_kernel<false, XBAR_ACT_NONE, VEC, LANES>), p->grid, dim3(256), 0, st, a->x, (const float*)nullptr, a->gamma,
                       a->beta, (const float*)nullptr, (const float*)nullptr, (const float*)nullptr, part, p->s);
  }
};
template <int ACT, int VEC, int LANES>
struct ApplyFwd {
  static void go(const Plan* p, const Fwd* a, hipStream_t st) {
    hipLaunchKernelGGL((gn_apply_kernel<false, ACT, VEC, LANES>), p->grid, dim3(256), 0, st, a->x, (const float*)nullptr, a->gamma, a->beta,
                       a->skip, a->mean, a->invstd, (const double*)nullptr, a->y, (float*)nullptr, p->s);
  }
};
template <int ACT, int VEC, int LANES>
struct PartialBwd {
  static void go(const Plan* p, const Bwd* a, double* part, hipStream_t st) {
    hipLaunchKernelGGL((gn_partial_kernel<true, ACT, VEC, LANES>), p->grid, dim3(256), 0, st, a->x, a->dy, a->gamma, a->beta, a->skip, a->mean,
                       a->invstd, part, p->s);
  }
};
template <int ACT, int VEC, int LANES>
struct ApplyBwd {
  static void go(const Plan* p, const Bwd* a, const double* coef, hipStream_t st) {
    hipLaunchKernelGGL((gn_apply_kernel<true, ACT, VEC, LANES>), p->grid, dim3(256), 0, st, a->x, a->dy, a->gamma, a->beta, a->skip, a->mean,
                       a->invstd, coef, a->dx, a->dskip, p->s);
  }
};

}  // namespace

extern "C" {

size_t xbar_gn_workspace_bytes(int batch, int positions, int channels, int groups) {
  return shape_ok(batch, positions, channels, groups) ? 0 : Plan(batch, positions, channels, groups).bytes();
}

int xbar_gn_fwd(const float* x, const float* gamma, const float* beta, const float* skip, float* y, float* mean, float* invstd, int batch,
                int positions, int channels, int groups, float eps, int act, void* ws, size_t ws_bytes, void* hip_stream) {
  if (shape_ok(batch, positions, channels, groups)) return XBAR_ESHAPE;
  if (!aligned16(x) || !aligned16(gamma) || !aligned16(beta) || !aligned16(y) || !aligned16(mean) || !aligned16(invstd) || !aligned16(ws) ||
      (skip && !aligned16(skip)))
    return XBAR_EALIGN;
  if (!(eps >= 0.0f) || !std::isfinite(eps) || act < XBAR_ACT_NONE || act > XBAR_ACT_SILU) return XBAR_EINVAL;
  const size_t n = (size_t)batch * positions * channels * sizeof(float);
  if (overlap(y, n, x, n) || overlap(y, n, skip, n)) return XBAR_EINVAL;
  const Plan p(batch, positions, channels, groups);
  if (ws_bytes < p.bytes()) return XBAR_EWORKSPACE;
  hipStream_t st = reinterpret_cast<hipStream_t>(hip_stream);
  double* part = reinterpret_cast<double*>(ws);
  const Fwd a{x, gamma, beta, skip, y, mean, invstd};
  dispatch<PartialFwd>(XBAR_ACT_NONE, p.vec, p.lanes, &p, &a, part, st);
  if (launched()) return XBAR_EHIP;
  hipLaunchKernelGGL(gn_final_fwd_kernel, dim3((unsigned)((batch * groups + 3) / 4)), dim3(256), 0, st, part, p.s, x, eps, mean, invstd);
  if (launched()) return XBAR_EHIP;
  dispatch<ApplyFwd>(act, p.vec, p.lanes, &p, &a, st);
  return launched();
}

int xbar_gn_bwd(const float* x, const float* dy, const float* gamma, const float* beta, const float* skip, const float* mean,
                const float* invstd, float* dx, float* dgamma, float* dbeta, float* dskip, int batch, int positions, int channels, int groups,
                int act, void* ws, size_t ws_bytes, void* hip_stream) {
  if (shape_ok(batch, positions, channels, groups)) return XBAR_ESHAPE;
  if (!aligned16(x) || !aligned16(dy) || !aligned16(gamma) || !aligned16(beta) || !aligned16(mean) || !aligned16(invstd) || !aligned16(dx) ||
      !aligned16(dgamma) || !aligned16(dbeta) || !aligned16(ws) || (skip && !aligned16(skip)) || (dskip && !aligned16(dskip)))
    return XBAR_EALIGN;
  if (act < XBAR_ACT_NONE || act > XBAR_ACT_SILU || (dskip && !skip)) return XBAR_EINVAL;
  const size_t n = (size_t)batch * positions * channels * sizeof(float);
  if (overlap(dx, n, x, n) || overlap(dx, n, dy, n) || overlap(dx, n, skip, n) || overlap(dskip, n, x, n) || overlap(dskip, n, dy, n) ||
      overlap(dskip, n, skip, n) || overlap(dskip, n, dx, n))
    return XBAR_EINVAL;
  const Plan p(batch, positions, channels, groups);
  if (ws_bytes < p.bytes()) return XBAR_EWORKSPACE;
  hipStream_t st = reinterpret_cast<hipStream_t>(hip_stream);
  double* part = reinterpret_cast<double*>(ws);
  double* coef = reinterpret_cast<double*>(reinterpret_cast<char*>(ws) + align256(p.sums() * sizeof(double)));
  const Bwd a{x, dy, gamma, beta, skip, mean, invstd, dx, dskip};
  dispatch<PartialBwd>(act, p.vec, p.lanes, &p, &a, part, st);
  if (launched()) return XBAR_EHIP;
  hipLaunchKernelGGL(gn_final_bwd_kernel, dim3((unsigned)((batch * groups + channels + 3) / 4)), dim3(256), 0, st, part, p.s, gamma, coef, dgamma,
                     dbeta);
  if (launched()) return XBAR_EHIP;
  dispatch<ApplyBwd>(act, p.vec, p.lanes, &p, &a, coef, st);
  return launched();
}

}  // extern "C"
