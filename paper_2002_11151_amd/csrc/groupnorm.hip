// Group normalisation with an activation, channels last: the normalisation of a digital peripheral that needs no batch -- statistics
// per sample and group of neighbouring channels -- so that a network runs one request, or trains on small batches.
//   z = gamma (x - mean) invstd + beta (+ skip),  y = act(z)
// Evaluated in double precision up to z, rounded once.  HBM-bound elementwise and reduction work: 64 x 56 x 56 x 256 with a skip takes 39 us for the
// sums (5.3 TB/s), 5 for the statistics and 110 for the values (5.6 TB/s); 64 x 28 x 28 x 512 backward 82 us in one pass (3.8 TB/s).
#include <hip/hip_runtime.h>

#include <algorithm>
#include <climits>
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

// VEC consecutive floats of memory, from a boundary of as many.
template <int VEC>
__device__ __forceinline__ void load_vec(const float* p, float (&v)[VEC]) {
  if constexpr (VEC == 4) {
    const float4 q = *reinterpret_cast<const float4*>(p);
    v[0] = q.x; v[1] = q.y; v[2] = q.z; v[3] = q.w;
  } else if constexpr (VEC == 2) {
    const float2 q = *reinterpret_cast<const float2*>(p);
    v[0] = q.x; v[1] = q.y;
  } else {
    v[0] = *p;
  }
}
// PAST: past the caches.
template <int VEC, bool PAST = false>
__device__ __forceinline__ void store_vec(float* p, const float (&v)[VEC]) {
  typedef float f4 __attribute__((ext_vector_type(4)));
  if constexpr (VEC == 4 && PAST) __builtin_nontemporal_store(f4{v[0], v[1], v[2], v[3]}, reinterpret_cast<f4*>(p));
  else if constexpr (VEC == 4) *reinterpret_cast<float4*>(p) = make_float4(v[0], v[1], v[2], v[3]);
  else if constexpr (VEC == 2) *reinterpret_cast<float2*>(p) = make_float2(v[0], v[1]);
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

// A channel's normalisation in one sample: gamma (x - mean) invstd + beta = a x + b.  a is exact (a product of two floats), b rounded once, z
// once more: the digits of a double, whatever the mean, for one conversion and one operation.
struct Norm {
  double a, b;
  __device__ __forceinline__ Norm() {}
  __device__ __forceinline__ Norm(float gamma, float beta, float mean, float invstd) {
    a = (double)gamma * (double)invstd;
    b = __builtin_fma(-(double)mean, a, (double)beta);
  }
  __device__ __forceinline__ double z(float x) const { return __builtin_fma((double)x, a, b); }
};
// dx = invstd (gamma g - m0 - xhat m1), m0 and m1 the means over the group of gamma g and gamma g xhat: p g + q x + r.
struct Slope {
  double p, q, r;
  __device__ __forceinline__ Slope() {}
  __device__ __forceinline__ Slope(float gamma, float mean, float invstd, double m0, double m1) {
    const double is = (double)invstd;
    p = is * (double)gamma;
    q = -is * is * m1;
    r = __builtin_fma(-q, (double)mean, -is * m0);
  }
  __device__ __forceinline__ float dx(float g, float x) const { return (float)__builtin_fma((double)g, p, __builtin_fma((double)x, q, r)); }
};
// Sum of g xhat from those of g and of g x.
__device__ __forceinline__ double xhat_sum(double g, double gx, float mean, float invstd) {
  return (double)invstd * __builtin_fma(-(double)mean, g, gx);
}

template <int VEC>
__device__ __forceinline__ void load_norm(Norm (&nm)[VEC], const Shape& s, int b, int c, const float* gamma, const float* beta,
                                          const float* mean, const float* invstd) {
#pragma unroll
  for (int e = 0; e < VEC; ++e) {
    const int g = b * s.groups + (c + e) / s.per_group;
    nm[e] = Norm(gamma[c + e], beta[c + e], mean[g], invstd[g]);
  }
}

// ---- a group held in registers ---------------------------------------------------------------------
// TEAM threads keep all values of one sample's group, N vectors of VEC neighbouring channels each: memory is touched once in each
// direction and one launch does it all.  Element i of the group is vector i % q of position i / q (q vectors per position).
constexpr int team_block(int team) { return team < 256 ? 256 : team; }
constexpr int kXcds = 8;

// The team's group.  Blocks go round the eight chiplets, which have caches of their own: every chiplet gets neighbouring groups, which share
// cache lines where a group's channels do not fill them.
template <int TEAM>
__device__ __forceinline__ int team_item() {
  const int each = gridDim.x / kXcds, block = (blockIdx.x % kXcds) * each + blockIdx.x / kXcds;
  return block * (team_block(TEAM) / TEAM) + threadIdx.x / TEAM;
}

// Places of a thread's elements: its next one is TEAM elements on.
struct Walk {
  int row, c, dr, dc, q;
  __device__ __forceinline__ Walk(int t, int team, int vectors) : q(vectors) {
    row = t / q;
    c = t - row * q;
    dr = team / q;
    dc = team - dr * q;
  }
  __device__ __forceinline__ void next() {
    row += dr;
    c += dc;
    if (c >= q) {
      c -= q;
      ++row;
    }
  }
};

// Sums over the team, the same bits in all of its threads; red: shared, for teams of several waves.
template <int TEAM>
__device__ __forceinline__ void team_sum(double& a, double& b, double (&red)[2][team_block(TEAM) / 64]) {
#pragma unroll
  for (int d = (TEAM < 64 ? TEAM : 64) / 2; d; d >>= 1) {
    a += __shfl_xor(a, d, 64);
    b += __shfl_xor(b, d, 64);
  }
  if constexpr (TEAM > 64) {
    constexpr int W = TEAM / 64;
    const int wave = threadIdx.x / 64, first = wave / W * W;
    if ((threadIdx.x & 63) == 0) {
      red[0][wave] = a;
      red[1][wave] = b;
    }
    __syncthreads();
    a = b = 0.0;
#pragma unroll
    for (int w = 0; w < W; ++w) {
      a += red[0][first + w];
      b += red[1][first + w];
    }
  }
}

template <int ACT, int VEC, int TEAM, int N>
__global__ __launch_bounds__(team_block(TEAM)) void gn_held_fwd_kernel(const float* x, const float* gamma, const float* beta, const float* skip,
                                                                       float* y, float* mean, float* invstd, Shape s, float eps) {
  __shared__ double red[2][team_block(TEAM) / 64];
  const int item = team_item<TEAM>();
  const bool mine = item < s.batch * s.groups;
  const int b = mine ? item / s.groups : 0, g = mine ? item - b * s.groups : 0, q = s.per_group / VEC;
  const int count = mine ? s.positions * q : 0, t = threadIdx.x % TEAM, c0 = g * s.per_group;
  const size_t from = (size_t)b * s.positions * s.channels + c0;
  float v[N][VEC];
  {
    Walk at(t, TEAM, q);
#pragma unroll
    for (int j = 0; j < N; ++j, at.next())
      if (t + TEAM * j < count) load_vec<VEC>(x + from + (size_t)at.row * s.channels + at.c * VEC, v[j]);
  }
  const double x0 = mine ? (double)x[from] : 0.0;             // sums about the group's first value keep the digits of a small spread
  double s0 = 0.0, s1 = 0.0;
#pragma unroll
  for (int j = 0; j < N; ++j)
    if (t + TEAM * j < count)
#pragma unroll
      for (int e = 0; e < VEC; ++e) {
        const double u = (double)v[j][e] - x0;
        s0 += u;
        s1 = __builtin_fma(u, u, s1);
      }
  team_sum<TEAM>(s0, s1, red);
  const double n = (double)s.positions * s.per_group, m = s0 / n, var = s1 / n - m * m;
  const float mu = (float)(x0 + m), is = (float)(1.0 / ::sqrt((var < 0.0 ? 0.0 : var) + (double)eps));
  if (mine && t == 0) {
    mean[item] = mu;
    invstd[item] = is;
  }
  Walk at(t, TEAM, q);
#pragma unroll
  for (int j = 0; j < N; ++j, at.next())
    if (t + TEAM * j < count) {
      const size_t to = from + (size_t)at.row * s.channels + at.c * VEC;
      float ga[VEC], be[VEC], k[VEC], o[VEC];
      load_vec<VEC>(gamma + c0 + at.c * VEC, ga);
      load_vec<VEC>(beta + c0 + at.c * VEC, be);
      if (skip) load_vec<VEC>(skip + to, k);
#pragma unroll
      for (int e = 0; e < VEC; ++e) {
        double z = Norm(ga[e], be[e], mu, is).z(v[j][e]);
        if (skip) z += (double)k[e];
        o[e] = act_of<ACT>(z);
      }
      store_vec<VEC>(y + to, o);
    }
}

// Backward: only the errors stay in registers; x is read again for dx, from the caches, and four vectors of each tensor are on their way at a
// time, so that a compute unit holds two blocks of 512 threads (64 x 28 x 28 x 512: 92 us with both tensors held in 166 registers, 84.5 with 110).
// q divides TEAM, so that a thread's elements all lie in the same channels.  sums[sample][channel][2]: sums of g and of g xhat over the
// positions; with one sample they are dbeta and dgamma themselves and go there.
template <int ACT, int VEC, int TEAM, int N>
__global__ __launch_bounds__(team_block(TEAM)) void gn_held_bwd_kernel(const float* x, const float* dy, const float* gamma, const float* beta,
                                                                       const float* skip, const float* mean, const float* invstd, float* dx,
                                                                       float* dskip, double* sums, float* dgamma, float* dbeta, Shape s) {
  constexpr int BLOCK = team_block(TEAM), WAVE = TEAM < 64 ? TEAM : 64, VALUES = 2 * VEC;
  __shared__ double red[2][BLOCK / 64];
  __shared__ double channel[VALUES * BLOCK];
  const int item = team_item<TEAM>();
  const bool mine = item < s.batch * s.groups;
  const int b = mine ? item / s.groups : 0, g = mine ? item - b * s.groups : 0, q = s.per_group / VEC;
  const int count = mine ? s.positions * q : 0, t = threadIdx.x % TEAM, row = t / q, c = t - row * q, dr = TEAM / q;
  const int c0 = g * s.per_group;
  const size_t from = (size_t)b * s.positions * s.channels + (size_t)row * s.channels + c0 + c * VEC, step = (size_t)dr * s.channels;
  float d[N][VEC];
  float ga[VEC], be[VEC];
  load_vec<VEC>(gamma + c0 + c * VEC, ga);
  load_vec<VEC>(beta + c0 + c * VEC, be);
  const float mu = mine ? mean[item] : 0.0f, is = mine ? invstd[item] : 0.0f;
  Norm nm[VEC];
#pragma unroll
  for (int e = 0; e < VEC; ++e) nm[e] = Norm(ga[e], be[e], mu, is);
  double p[VALUES];                                            // p[2 e]: sum of g, p[2 e + 1]: of g x
#pragma unroll
  for (int i = 0; i < VALUES; ++i) p[i] = 0.0;
#pragma unroll
  for (int j0 = 0; j0 < N; j0 += 4) {
    float v[4][VEC];
#pragma unroll
    for (int j = j0; j < j0 + 4 && j < N; ++j)
      if (t + TEAM * j < count) {
        load_vec<VEC>(x + from + j * step, v[j - j0]);
        load_vec<VEC>(dy + from + j * step, d[j]);
      }
#pragma unroll
    for (int j = j0; j < j0 + 4 && j < N; ++j)
      if (t + TEAM * j < count) {
        float k[VEC];
        if (ACT != XBAR_ACT_NONE && skip) load_vec<VEC>(skip + from + j * step, k);
#pragma unroll
        for (int e = 0; e < VEC; ++e) {
          double z = nm[e].z(v[j - j0][e]);
          if (ACT != XBAR_ACT_NONE && skip) z += (double)k[e];
          d[j][e] = act_bwd<ACT>(z, d[j][e]);
          p[2 * e] += (double)d[j][e];
          p[2 * e + 1] = __builtin_fma((double)d[j][e], (double)v[j - j0][e], p[2 * e + 1]);
        }
      }
    __builtin_amdgcn_sched_barrier(0);
  }
  // Over the lanes with the same channels: every level exchanges half of what is left and keeps the other half, so that a lane ends up with
  // VALUES >> levels of the sums (or one, which several hold).
  int left = VALUES, which = 0;
#pragma unroll
  for (int level = 0, dist = WAVE / 2; dist; ++level, dist >>= 1) {
    if (dist >= q) {
      const int half = (VALUES >> level) / 2;
      if (half) {
        const bool upper = t & dist;
#pragma unroll
        for (int i = 0; i < half; ++i) {
          const double send = upper ? p[i] : p[i + half], keep = upper ? p[i + half] : p[i];
          p[i] = keep + __shfl_xor(send, dist, 64);
        }
        which += upper ? half : 0;
        left = half;
      } else {
        p[0] += __shfl_xor(p[0], dist, 64);
      }
    }
  }
  const int slots = q < WAVE ? TEAM / WAVE : dr, slot = q < WAVE ? t / WAVE : row;      // partial sums of a channel
  double* shared = channel + (threadIdx.x / TEAM) * (VALUES * TEAM);
#pragma unroll
  for (int i = 0; i < VALUES; ++i)
    if (i < left) shared[(slot * q + c) * VALUES + which + i] = p[i];
  __syncthreads();
  double s0 = 0.0, s1 = 0.0;
  for (int i = t; i < s.per_group; i += TEAM) {
    double sg = 0.0, sgx = 0.0;
    for (int k = 0; k < slots; ++k) {
      sg += shared[(k * s.per_group + i) * 2];
      sgx += shared[(k * s.per_group + i) * 2 + 1];
    }
    sgx = xhat_sum(sg, sgx, mu, is);
    const double f = (double)gamma[c0 + i];
    s0 = __builtin_fma(f, sg, s0);
    s1 = __builtin_fma(f, sgx, s1);
    if (mine && s.batch > 1) {
      double* to = sums + ((size_t)b * s.channels + c0 + i) * 2;
      to[0] = sg;
      to[1] = sgx;
    } else if (mine) {
      dbeta[c0 + i] = (float)sg;
      dgamma[c0 + i] = (float)sgx;
    }
  }
  team_sum<TEAM>(s0, s1, red);
  const double n = (double)s.positions * s.per_group;
  Slope sl[VEC];
#pragma unroll
  for (int e = 0; e < VEC; ++e) sl[e] = Slope(ga[e], mu, is, s0 / n, s1 / n);
#pragma unroll
  for (int j = 0; j < N; ++j)
    if (t + TEAM * j < count) {
      float o[VEC], again[VEC];
      load_vec<VEC>(x + from + j * step, again);
#pragma unroll
      for (int e = 0; e < VEC; ++e) {
        o[e] = sl[e].dx(d[j][e], again[e]);
      }
      store_vec<VEC>(dx + from + j * step, o);
      if (dskip) store_vec<VEC>(dskip + from + j * step, d[j]);
      if (j % 4 == 3) __builtin_amdgcn_sched_barrier(0);
    }
}

// Parameters' gradients: sums over `rows` rows of 2 C values; 16 values and 64 threads for each per block.
__global__ __launch_bounds__(1024) void gn_parameters_kernel(const double* sums, int rows, int C, float* dgamma, float* dbeta) {
  __shared__ double red[16][16];
  const int lane = threadIdx.x & 15, at = threadIdx.x >> 4, i = blockIdx.x * 16 + lane;
  double s = 0.0;
  if (i < 2 * C) {
    for (int r0 = at; r0 < rows; r0 += 64 * 8) {               // eight loads in flight
      double v[8];
#pragma unroll
      for (int k = 0; k < 8; ++k) v[k] = r0 + 64 * k < rows ? sums[(size_t)(r0 + 64 * k) * 2 * C + i] : 0.0;
#pragma unroll
      for (int k = 0; k < 8; ++k) s += v[k];
    }
  }
  s += __shfl_xor(s, 16, 64);
  s += __shfl_xor(s, 32, 64);
  if ((threadIdx.x & 63) < 16) red[threadIdx.x >> 6][lane] = s;
  __syncthreads();
  if (threadIdx.x < 16 && i < 2 * C) {
    s = 0.0;
#pragma unroll
    for (int w = 0; w < 16; ++w) s += red[w][lane];
    if (i & 1) dgamma[i >> 1] = (float)s;
    else dbeta[i >> 1] = (float)s;
  }
}

// ---- larger groups: sums, statistics and values in launches of their own -----------------------------
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
          double z = nm[e].z(v[e]);
          if (ACT != XBAR_ACT_NONE && skip) z += (double)k[e];
          const double g = (double)act_bwd<ACT>(z, d[e]);
          s0[e] += g;
          s1[e] = __builtin_fma(g, (double)v[e], s1[e]);
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
    if (BWD && value >= CT) {
      double g = 0.0;
#pragma unroll
      for (int k = 0; k < SHARES; ++k) g += shares[k][value - CT];
      const int item = b * s.groups + cv / s.per_group;
      t = xhat_sum(g, t, mean[item], invstd[item]);
    }
    part[((size_t)blockIdx.x * C + cv) * 2 + value / CT] = t;
  }
}

// TEAM threads per sample and group: forward mean and 1 / std, backward the two means over the group that dx needs.  Eight loads of a thread
// in flight.
template <bool BWD, int TEAM>
__global__ __launch_bounds__(team_block(TEAM)) void gn_final_kernel(const double* part, Shape s, const float* x, const float* gamma, float eps,
                                                                    float* mean, float* invstd, double* coef) {
  __shared__ double red[2][team_block(TEAM) / 64];
  const int item = blockIdx.x * (team_block(TEAM) / TEAM) + threadIdx.x / TEAM, t = threadIdx.x % TEAM;
  if (item >= s.batch * s.groups) return;                      // (all threads of a team, and a block is one team where it has to wait)
  const int b = item / s.groups, g = item - b * s.groups, c0 = g * s.per_group, values = s.chunks * s.per_group;
  const double* from = part + ((size_t)b * s.chunks * s.channels + c0) * 2;
  double s0 = 0.0, s1 = 0.0;
  Walk at(t, TEAM, s.per_group);
  for (int i0 = t; i0 < values; i0 += 8 * TEAM) {
    double2 p[8];
    float f[8];
#pragma unroll
    for (int u = 0; u < 8; ++u, at.next())
      if (i0 + u * TEAM < values) {
        p[u] = *reinterpret_cast<const double2*>(from + ((size_t)at.row * s.channels + at.c) * 2);
        if (BWD) f[u] = gamma[c0 + at.c];
      }
#pragma unroll
    for (int u = 0; u < 8; ++u)
      if (i0 + u * TEAM < values) {
        s0 = __builtin_fma(BWD ? (double)f[u] : 1.0, p[u].x, s0);
        s1 = __builtin_fma(BWD ? (double)f[u] : 1.0, p[u].y, s1);
      }
  }
  team_sum<TEAM>(s0, s1, red);
  if (t) return;
  const double n = (double)s.positions * s.per_group;
  if (BWD) {
    coef[(size_t)item * 2] = s0 / n;
    coef[(size_t)item * 2 + 1] = s1 / n;
  } else {
    const double m = s0 / n, var = s1 / n - m * m;
    mean[item] = (float)((double)x[(size_t)b * s.positions * s.channels + c0] + m);
    invstd[item] = (float)(1.0 / ::sqrt((var < 0.0 ? 0.0 : var) + (double)eps));
  }
}

// y, or dx and dskip; blocks and threads as in gn_partial_kernel.  PAST: outputs of more than half of the last-level cache, which the next
// reader would not find there, leave it to x (64 x 56 x 56 x 256 with a ReLU behind it 201 -> 187 us, alone 130 -> 112; 32 x 112 x 112 x 64, half as
// much, 95 -> 100: there the ordinary way).
template <bool BWD, int ACT, int VEC, int LANES, bool PAST>
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
  Slope sl[VEC];
  if (BWD)
#pragma unroll
    for (int e = 0; e < VEC; ++e) {
      const size_t g = (size_t)b * s.groups + (c + e) / s.per_group;
      sl[e] = Slope(gamma[c + e], mean[g], invstd[g], coef[g * 2], coef[g * 2 + 1]);
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
      double z = nm[e].z(v[e]);
      if ((!BWD || ACT != XBAR_ACT_NONE) && skip) z += (double)k[e];
      if (BWD) {
        q[e] = act_bwd<ACT>(z, d[e]);
        o[e] = sl[e].dx(q[e], v[e]);
      } else {
        o[e] = act_of<ACT>(z);
      }
    }
    store_vec<VEC, PAST>(out + at, o);
    if (BWD && dskip) store_vec<VEC, PAST>(dskip + at, q);
  }
}

// Strips of 64 channels, or of 16 where the rows have no more than 32; a block takes 32 to 512 positions, about 2048 blocks in all.
struct Plan {
  Shape s;
  int vec, lanes;
  dim3 grid;
  int held_vec, elements;      // of a group held in registers: floats and number of its vectors
  Plan(int batch, int positions, int channels, int groups) {
    vec = channels % 4 == 0 ? 4 : 1;
    const int strip = channels <= 32 ? 16 : 64, strips = (channels + strip - 1) / strip;
    lanes = strip / vec;
    const long long wanted = ((long long)batch * positions * strips + 2047) / 2048;
    const int rows = (int)std::min<long long>(512, std::max<long long>(32, wanted));
    const int chunks = (positions + rows - 1) / rows;
    s = Shape{batch, positions, channels, groups, channels / groups, rows, chunks};
    grid = dim3((unsigned)((long long)batch * chunks), (unsigned)strips);
    held_vec = s.per_group % 4 == 0 ? 4 : s.per_group % 2 == 0 ? 2 : 1;
    elements = (int)std::min<long long>(1 << 30, (long long)positions * (s.per_group / held_vec));
  }
  bool past() const { return (double)s.batch * s.positions * s.channels * sizeof(float) > 134217728.0; }
  // Threads that hold a group (0: too large, three launches instead).  Few threads where a few vectors each are enough, so that small groups
  // share a block; 512 with eight vectors each at most: with 16 a block fills a compute unit and nothing hides its loads (64 x 56 x 56 x 256 in
  // 32 groups, forward: 219 us, 200 with 1024 threads, against 167 in three launches).  us, held / three launches: forward 13 x 255 x 90 in 9
  // groups 15.1 / 19.9, 1 x 64 x 64 14.9 / 19.0; backward 128 x 1024 x 16 in 4 groups 17.4 / 24, 64 x 784 x 512 in 32 84.5 / 107.
  int team(bool backward) const {
    const int q = s.per_group / held_vec, most = 512 * 8;
    if (elements > most) return 0;
    const int t = elements <= 32 ? 16 : elements <= 256 ? 64 : elements <= 1024 ? 256 : 512;
    if (!backward) return t;
    if (q & (q - 1)) return 0;                               // a thread's elements have to lie in the same channels
    return t >= q ? t : q <= 64 ? 64 : q <= 256 ? 256 : q <= 512 ? 512 : 0;
  }
  dim3 held_grid(int team) const {
    const int teams = team_block(team) / team;
    const long long blocks = ((long long)s.batch * s.groups + teams - 1) / teams;
    return dim3((unsigned)((blocks + kXcds - 1) / kXcds * kXcds));
  }
  // A block of 1024 threads per group where there are few groups of many pairs of sums, else a wave (us, block / wave: one group of 25088 pairs 6.8 / 37,
  // of 564 3.0 / 2.5; 256 groups of 1600 4.8 / 6.4, of 512 4.9 / 4.9; 512 of 1600 6.2 / 6.7; 2048 of 800 15.7 / 7.3).
  template <bool BWD>
  void finish(const double* part, const float* x, const float* gamma, float eps, float* mean, float* invstd, double* coef, hipStream_t st) const {
    const int items = s.batch * s.groups;
    const bool block = items <= 512 && (long long)s.chunks * s.per_group > 1024;
    auto k = block ? gn_final_kernel<BWD, 1024> : gn_final_kernel<BWD, 64>;
    hipLaunchKernelGGL(k, dim3((unsigned)(block ? items : (items + 3) / 4)), dim3(block ? 1024 : 256), 0, st, part, s, x, gamma, eps, mean, invstd,
                       coef);
  }
  size_t sums() const { return (size_t)s.batch * s.chunks * s.channels * 2; }
  size_t bytes() const { return align256(sums() * sizeof(double)) + align256((size_t)s.batch * s.groups * 2 * sizeof(double)); }
};

// The limits on a shape: elements below 2^38, threads of a launch below 2^32, a block's positions and the 512 behind them within an int.
int shape_ok(int batch, int positions, int channels, int groups) {
  if (batch <= 0 || positions <= 0 || channels <= 0 || groups <= 0 || channels % groups) return XBAR_ESHAPE;
  if (positions > INT_MAX - 511) return XBAR_ESHAPE;
  if ((double)batch * positions * channels >= 274877906944.0 || channels > (1 << 20) || (double)batch * groups >= 33554432.0) return XBAR_ESHAPE;
  const Plan p(batch, positions, channels, groups);
  double threads = 256.0 * batch * p.s.chunks;
  for (const bool backward : {false, true})
    if (const int team = p.team(backward)) threads = std::max(threads, (double)p.held_grid(team).x * team_block(team));
  return threads >= 4294967296.0 ? XBAR_ESHAPE : XBAR_OK;
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

template <int ACT, int VEC>
struct Held {
  static int fwd(const Plan& p, const Fwd& a, float eps, hipStream_t st) {
    const int team = p.team(false);
    auto k = team == 16 ? gn_held_fwd_kernel<ACT, VEC, 16, 2> : team == 64 ? gn_held_fwd_kernel<ACT, VEC, 64, 4>
             : team == 256 ? gn_held_fwd_kernel<ACT, VEC, 256, 4> : gn_held_fwd_kernel<ACT, VEC, 512, 8>;
    hipLaunchKernelGGL(k, p.held_grid(team), dim3(team_block(team)), 0, st, a.x, a.gamma, a.beta, a.skip, a.y, a.mean, a.invstd, p.s, eps);
    return launched();
  }
  static int bwd(const Plan& p, const Bwd& a, double* sums, float* dgamma, float* dbeta, hipStream_t st) {
    const int team = p.team(true);
    auto k = team == 16 ? gn_held_bwd_kernel<ACT, VEC, 16, 2> : team == 64 ? gn_held_bwd_kernel<ACT, VEC, 64, 4>
             : team == 256 ? gn_held_bwd_kernel<ACT, VEC, 256, 4> : gn_held_bwd_kernel<ACT, VEC, 512, 8>;
    hipLaunchKernelGGL(k, p.held_grid(team), dim3(team_block(team)), 0, st, a.x, a.dy, a.gamma, a.beta, a.skip, a.mean, a.invstd, a.dx, a.dskip,
                       sums, dgamma, dbeta, p.s);
    return launched();
  }
};
template <class F>
int with_held(int act, int vec, F f) {
  auto with_act = [&](auto a) {
    constexpr int ACT = decltype(a)::value;
    return vec == 4 ? f(Held<ACT, 4>()) : vec == 2 ? f(Held<ACT, 2>()) : f(Held<ACT, 1>());
  };
  if (act == XBAR_ACT_RELU) return with_act(std::integral_constant<int, XBAR_ACT_RELU>());
  if (act == XBAR_ACT_SILU) return with_act(std::integral_constant<int, XBAR_ACT_SILU>());
  return with_act(std::integral_constant<int, XBAR_ACT_NONE>());
}

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
    auto k = VEC == 4 && p->past() ? gn_apply_kernel<false, ACT, VEC, LANES, VEC == 4> : gn_apply_kernel<false, ACT, VEC, LANES, false>;
    hipLaunchKernelGGL(k, p->grid, dim3(256), 0, st, a->x, (const float*)nullptr, a->gamma, a->beta, a->skip, a->mean, a->invstd, (const double*)nullptr, a->y, (float*)nullptr, p->s);
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
    auto k = VEC == 4 && p->past() ? gn_apply_kernel<true, ACT, VEC, LANES, VEC == 4> : gn_apply_kernel<true, ACT, VEC, LANES, false>;
    hipLaunchKernelGGL(k, p->grid, dim3(256), 0, st, a->x, a->dy, a->gamma, a->beta, a->skip, a->mean, a->invstd, coef, a->dx, a->dskip, p->s);
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
  const size_t each = (size_t)channels * sizeof(float), stats = (size_t)batch * groups * sizeof(float);
  const Plan p(batch, positions, channels, groups);
  if (overlap(y, n, x, n) || overlap(y, n, skip, n) || overlap(y, n, gamma, each) || overlap(y, n, beta, each) || overlap(y, n, mean, stats) ||
      overlap(y, n, invstd, stats) || overlap(y, n, ws, p.bytes()))
    return XBAR_EINVAL;
  if (ws_bytes < p.bytes()) return XBAR_EWORKSPACE;
  hipStream_t st = reinterpret_cast<hipStream_t>(hip_stream);
  double* part = reinterpret_cast<double*>(ws);
  const Fwd a{x, gamma, beta, skip, y, mean, invstd};
  if (p.team(false)) return with_held(act, p.held_vec, [&](auto k) { return k.fwd(p, a, eps, st); });
  dispatch<PartialFwd>(XBAR_ACT_NONE, p.vec, p.lanes, &p, &a, part, st);
  if (launched()) return XBAR_EHIP;
  p.finish<false>(part, x, nullptr, eps, mean, invstd, nullptr, st);
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
  const size_t each = (size_t)channels * sizeof(float), stats = (size_t)batch * groups * sizeof(float);
  const Plan p(batch, positions, channels, groups);
  for (const float* out : {dx, dskip})
    if (overlap(out, n, x, n) || overlap(out, n, dy, n) || overlap(out, n, skip, n) || overlap(out, n, gamma, each) || overlap(out, n, beta, each) ||
        overlap(out, n, mean, stats) || overlap(out, n, invstd, stats) || overlap(out, n, dgamma, each) || overlap(out, n, dbeta, each) ||
        overlap(out, n, ws, p.bytes()))
      return XBAR_EINVAL;
  if (overlap(dskip, n, dx, n)) return XBAR_EINVAL;
  if (ws_bytes < p.bytes()) return XBAR_EWORKSPACE;
  hipStream_t st = reinterpret_cast<hipStream_t>(hip_stream);
  double* part = reinterpret_cast<double*>(ws);
  double* coef = reinterpret_cast<double*>(reinterpret_cast<char*>(ws) + align256(p.sums() * sizeof(double)));
  const Bwd a{x, dy, gamma, beta, skip, mean, invstd, dx, dskip};
  const dim3 parameters((unsigned)((2 * channels + 15) / 16));
  if (p.team(true)) {
    const int rc = with_held(act, p.held_vec, [&](auto k) { return k.bwd(p, a, part, dgamma, dbeta, st); });
    if (rc || batch == 1) return rc;
    hipLaunchKernelGGL(gn_parameters_kernel, parameters, dim3(1024), 0, st, part, batch, channels, dgamma, dbeta);
    return launched();
  }
  dispatch<PartialBwd>(act, p.vec, p.lanes, &p, &a, part, st);
  if (launched()) return XBAR_EHIP;
  p.finish<true>(part, nullptr, gamma, 0.0f, nullptr, nullptr, coef, st);
  if (launched()) return XBAR_EHIP;
  hipLaunchKernelGGL(gn_parameters_kernel, parameters, dim3(1024), 0, st, part, batch * p.s.chunks, channels, dgamma, dbeta);
  if (launched()) return XBAR_EHIP;
  dispatch<ApplyBwd>(act, p.vec, p.lanes, &p, &a, coef, st);
  return launched();
}

}  // extern "C"
