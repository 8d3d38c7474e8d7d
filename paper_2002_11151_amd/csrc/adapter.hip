// Low-rank adapters of many requests beside a shared projection: the projection runs on programmed crossbars, whose devices are not
// written for every task; each task adds a digital correction of rank r,
//   T[m][r] = sum_k X[m][k] A[a][r][k],   Y[m][n] = base[m][n] + sum_r scale[a] T[m][r] B[a][r][n],   a = adapter of row m.
// A and B are kept the same way round (rows of the rank), so both directions are three products:
//   shrink  T = X A^T (forward),            dT = scale dY B^T (backward)          one pass over the wide operand
//   expand  Y = base + scale T B,           dX = base + dT A                      one pass over base and output
//   outer   dA = dT^T X, dB = scale T^T dY                                        one pass over the wide operand
// All on v_mfma_f32_16x16x4_f32: single precision throughout; at ranks of up to some 64 the products are bound by memory, not by the
// instruction's rate.  Rows are taken in the order of their adapters (the plan), in tiles and chunks that hold one adapter each.
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

typedef float f4 __attribute__((ext_vector_type(4)));

constexpr int kTileRows = 32;          // rows of a tile: two matrix tiles
constexpr int kMaxRank = 128;

// ---- the plan --------------------------------------------------------------------------------------
// Rows sorted by adapter (stable; rows without one last), cut into tiles of up to kTileRows and chunks of up to chunk_rows() rows.  A
// chunk of an adapter that has several gets a slot for its partial gradients.
struct Entry {
  int adapter, begin, count, slot;
};

struct PlanAt {
  int* head;            // magic, M, adapters, tiles, chunks
  int* perm;            // [M]
  int* start;           // [adapters + 2]: first sorted position of an adapter
  int* tile0;           // [adapters + 2]: first tile
  int* chunk0;          // [adapters + 2]: first chunk
  int* slot0;           // [adapters + 2]: first slot
  Entry* tiles;
  Entry* chunks;
};
constexpr int kMagic = 0x70ada37e;

__host__ __device__ inline int chunk_rows(int M) {
  const int many = (M / 32 + 31) / 32 * 32;
  return many > 256 ? many : 256;
}
inline long long max_tiles(int M, int adapters) { return (long long)M / kTileRows + std::min<long long>(M, (long long)adapters + 1) + 1; }
inline long long max_chunks(int M, int adapters) { return (long long)M / chunk_rows(M) + std::min<long long>(M, (long long)adapters + 1) + 1; }
inline long long max_slots(int M) { return 2ll * M / chunk_rows(M) + 2; }     // chunks of adapters with more than one

inline size_t plan_layout(void* base, int M, int adapters, PlanAt* at) {
  char* p = reinterpret_cast<char*>(base);
  size_t off = 0;
  auto take = [&](size_t bytes) {
    char* q = p + off;
    off += align256(bytes);
    return q;
  };
  PlanAt l;
  l.head = reinterpret_cast<int*>(take(8 * sizeof(int)));
  l.perm = reinterpret_cast<int*>(take((size_t)M * sizeof(int)));
  l.start = reinterpret_cast<int*>(take(((size_t)adapters + 2) * sizeof(int)));
  l.tile0 = reinterpret_cast<int*>(take(((size_t)adapters + 2) * sizeof(int)));
  l.chunk0 = reinterpret_cast<int*>(take(((size_t)adapters + 2) * sizeof(int)));
  l.slot0 = reinterpret_cast<int*>(take(((size_t)adapters + 2) * sizeof(int)));
  l.tiles = reinterpret_cast<Entry*>(take((size_t)max_tiles(M, adapters) * sizeof(Entry)));
  l.chunks = reinterpret_cast<Entry*>(take((size_t)max_chunks(M, adapters) * sizeof(Entry)));
  if (at) *at = l;
  return off;
}

__device__ __forceinline__ int bin_of(int id, int adapters) { return (unsigned)id < (unsigned)adapters ? id : adapters; }

// Rows of every adapter (bin `adapters`: rows without one), one wave per bin over all rows.
__global__ __launch_bounds__(256) void plan_count_kernel(const int32_t* rows, int M, int adapters, PlanAt p) {
  const int bin = blockIdx.x * 4 + (threadIdx.x >> 6), lane = threadIdx.x & 63;
  if (bin > adapters) return;
  int n = 0;
  for (int m = lane; m < M; m += 64) n += bin_of(rows[m], adapters) == bin;
#pragma unroll
  for (int d = 32; d; d >>= 1) n += __shfl_xor(n, d, 64);
  if (lane == 0) p.start[bin] = n;
}

// Exclusive prefix sums over the bins of rows, tiles, chunks and slots; one block.
__global__ __launch_bounds__(1024) void plan_prefix_kernel(int M, int adapters, PlanAt p) {
  __shared__ int part[4][16];
  __shared__ int carry[4];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, per_chunk = chunk_rows(M);
  if (threadIdx.x < 4) carry[threadIdx.x] = 0;
  __syncthreads();
  for (int b0 = 0; b0 <= adapters; b0 += 1024) {
    const int bin = b0 + threadIdx.x;
    int v[4] = {0, 0, 0, 0};
    if (bin <= adapters) {
      v[0] = p.start[bin];
      v[1] = (v[0] + kTileRows - 1) / kTileRows;
      v[2] = bin < adapters ? (v[0] + per_chunk - 1) / per_chunk : 0;
      v[3] = v[2] > 1 ? v[2] : 0;
    }
    int sum[4];
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      int s = v[q];
#pragma unroll
      for (int d = 1; d < 64; d <<= 1) {
        const int o = __shfl_up(s, d, 64);
        if (lane >= d) s += o;
      }
      sum[q] = s;
      if (lane == 63) part[q][wave] = s;
    }
    __syncthreads();
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      int before = carry[q];
      for (int w = 0; w < wave; ++w) before += part[q][w];
      sum[q] += before - v[q];
    }
    if (bin <= adapters) {
      p.start[bin] = sum[0];
      p.tile0[bin] = sum[1];
      p.chunk0[bin] = sum[2];
      p.slot0[bin] = sum[3];
    }
    __syncthreads();
    if (threadIdx.x == 1023)                                    // bins beyond the last count nothing
#pragma unroll
      for (int q = 0; q < 4; ++q) carry[q] = sum[q] + v[q];
    __syncthreads();
  }
  if (threadIdx.x == 0) {
    p.start[adapters + 1] = carry[0];
    p.tile0[adapters + 1] = carry[1];
    p.chunk0[adapters + 1] = carry[2];
    p.slot0[adapters + 1] = carry[3];
    p.head[0] = kMagic;
    p.head[1] = M;
    p.head[2] = adapters;
    p.head[3] = carry[1];
    p.head[4] = carry[2];
  }
}

// Places of a bin's rows, in their order, and its tiles and chunks; one wave per bin.
__global__ __launch_bounds__(256) void plan_place_kernel(const int32_t* rows, int M, int adapters, PlanAt p) {
  const int bin = blockIdx.x * 4 + (threadIdx.x >> 6), lane = threadIdx.x & 63;
  if (bin > adapters) return;
  const int begin = p.start[bin], end = p.start[bin + 1], id = bin < adapters ? bin : -1, per_chunk = chunk_rows(M);
  if (begin == end) return;
  int at = begin;
  for (int m0 = 0; m0 < M; m0 += 64) {
    const int m = m0 + lane;
    const bool mine = m < M && bin_of(rows[m], adapters) == bin;
    const unsigned long long all = __ballot(mine);
    if (mine) p.perm[at + __popcll(all & ((1ull << lane) - 1))] = m;
    at += __popcll(all);
  }
  const int tiles = (end - begin + kTileRows - 1) / kTileRows;
  for (int i = lane; i < tiles; i += 64) {
    const int from = begin + i * kTileRows;
    p.tiles[p.tile0[bin] + i] = Entry{id, from, min(kTileRows, end - from), 0};
  }
  if (id < 0) return;
  const int chunks = (end - begin + per_chunk - 1) / per_chunk;
  for (int i = lane; i < chunks; i += 64) {
    const int from = begin + i * per_chunk;
    p.chunks[p.chunk0[bin] + i] = Entry{id, from, min(per_chunk, end - from), chunks > 1 ? p.slot0[bin] + i : -1};
  }
}

__device__ __forceinline__ bool planned(const PlanAt& p, int M, int adapters) {
  return p.head[0] == kMagic && p.head[1] == M && p.head[2] == adapters;
}

// ---- the products ----------------------------------------------------------------------------------
__device__ __forceinline__ float wide(float x) { return x; }
__device__ __forceinline__ float wide(uint16_t x) { return __uint_as_float((uint32_t)x << 16); }   // bfloat16

// Four values from p on, those at place k and beyond `end` zero; QUADS: all or none of the four are inside, and p is aligned.
template <bool QUADS>
__device__ __forceinline__ f4 load4(const float* p, int k, int end) {
  f4 v = {0.0f, 0.0f, 0.0f, 0.0f};
  if constexpr (QUADS) {
    if (k < end) v = *reinterpret_cast<const f4*>(p);
  } else {
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (k + e < end) v[e] = p[e];
  }
  return v;
}
template <bool QUADS>
__device__ __forceinline__ f4 load4(const uint16_t* p, int k, int end) {
  f4 v = {0.0f, 0.0f, 0.0f, 0.0f};
  if constexpr (QUADS) {
    if (k < end) {
      const uint2 q = *reinterpret_cast<const uint2*>(p);
      v = f4{__uint_as_float(q.x << 16), __uint_as_float(q.x & 0xFFFF0000u), __uint_as_float(q.y << 16), __uint_as_float(q.y & 0xFFFF0000u)};
    }
  } else {
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (k + e < end) v[e] = wide(p[e]);
  }
  return v;
}
template <bool QUADS>
__device__ __forceinline__ void store4(float* p, f4 v, int k, int end) {
  if constexpr (QUADS) {
    if (k < end) *reinterpret_cast<f4*>(p) = v;
  } else {
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (k + e < end) p[e] = v[e];
  }
}

// part[split][sorted row][16 RT] = X A^T over the split's share of K.  Block: one tile, its four waves side by side along K, joined in
// LDS.  The instruction adds up over four k, one per quarter of the wave; a lane's 16-byte loads hold four neighbouring k of one row, so
// the four instructions of a step take k = 4 (lane / 16) + j from both operands.  Rows beyond the tile and ranks beyond the last repeat a
// valid one: their products are not stored.
template <class T, bool QUADS, int RT>
__global__ __launch_bounds__(256) void shrink_kernel(PlanAt plan, const float* X, const T* A, float* part, int M, int K, int rank, int adapters,
                                                     int per_split) {
  __shared__ float red[4][kTileRows][16 * RT];
  if (!planned(plan, M, adapters) || (int)blockIdx.x >= plan.head[3]) return;
  const Entry tile = plan.tiles[blockIdx.x];
  if (tile.adapter < 0) return;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, col = lane & 15, quarter = lane >> 4;
  const bool two = tile.count > 16;
  const float* x0 = X + (size_t)plan.perm[tile.begin + min(col, tile.count - 1)] * K;
  const float* x1 = X + (size_t)plan.perm[tile.begin + min(col + 16, tile.count - 1)] * K;
  const T* a[RT];
#pragma unroll
  for (int t = 0; t < RT; ++t) a[t] = A + ((size_t)tile.adapter * rank + min(16 * t + col, rank - 1)) * K;
  f4 acc[2][RT];
#pragma unroll
  for (int t = 0; t < RT; ++t) acc[0][t] = acc[1][t] = f4{0.0f, 0.0f, 0.0f, 0.0f};
  const int k0 = blockIdx.y * per_split, k1 = min(k0 + per_split, K);
  for (int k = k0 + 16 * wave + 4 * quarter; k < k1 + 4 * quarter; k += 64) {      // the same number of steps for the whole wave
    const f4 u = load4<QUADS>(x0 + k, k, k1);
    f4 w = u;
    if (two) w = load4<QUADS>(x1 + k, k, k1);
    f4 b[RT];
#pragma unroll
    for (int t = 0; t < RT; ++t) b[t] = load4<QUADS>(a[t] + k, k, k1);
#pragma unroll
    for (int j = 0; j < 4; ++j)
#pragma unroll
      for (int t = 0; t < RT; ++t) {
        acc[0][t] = __builtin_amdgcn_mfma_f32_16x16x4f32(u[j], b[t][j], acc[0][t], 0, 0, 0);
        if (two) acc[1][t] = __builtin_amdgcn_mfma_f32_16x16x4f32(w[j], b[t][j], acc[1][t], 0, 0, 0);
      }
  }
#pragma unroll
  for (int h = 0; h < 2; ++h)
#pragma unroll
    for (int t = 0; t < RT; ++t)
#pragma unroll
      for (int i = 0; i < 4; ++i) red[wave][16 * h + 4 * quarter + i][16 * t + col] = acc[h][t][i];
  __syncthreads();
  for (int i = threadIdx.x; i < tile.count * 16 * RT; i += 256) {
    const int row = i / (16 * RT), r = i - row * (16 * RT);
    part[((size_t)blockIdx.y * M + tile.begin + row) * (16 * RT) + r] = (red[0][row][r] + red[1][row][r]) + (red[2][row][r] + red[3][row][r]);
  }
}

// out = base + sum over ranks of scale (sum of the splits) B.  Block: one tile and 256 columns, a wave 64 of them; a lane's 16-byte
// loads of B hold four neighbouring columns, one for each of four matrix tiles, so that base and out are touched 16 bytes wide too.
// The blocks of the first columns also keep the sums (`kept`, times scale with KEEP_SCALED).
template <class T, bool QUADS, int RT, bool KEEP_SCALED>
__global__ __launch_bounds__(256) void expand_kernel(PlanAt plan, const float* base, const float* part, int splits, const float* scale, const T* B,
                                                     float* out, float* kept, int M, int N, int rank, int adapters) {
  __shared__ float ts[kTileRows][16 * RT + 1];
  if (!planned(plan, M, adapters) || (int)blockIdx.x >= plan.head[3]) return;
  const Entry tile = plan.tiles[blockIdx.x];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, col = lane & 15, quarter = lane >> 4;
  const int n = blockIdx.y * 256 + 64 * wave + 4 * col;
  if (tile.adapter < 0) {                                      // rows without an adapter: as they were
    if (out && out != base)
      for (int i = quarter; i < tile.count; i += 4) {
        const size_t at = (size_t)plan.perm[tile.begin + i] * N + n;
        store4<QUADS>(out + at, load4<QUADS>(base + at, n, N), n, N);
      }
    if (blockIdx.y == 0 && kept)
      for (int i = threadIdx.x; i < tile.count * rank; i += 256) kept[(size_t)plan.perm[tile.begin + i / rank] * rank + i % rank] = 0.0f;
    return;
  }
  const float f = scale[tile.adapter];
  for (int i = threadIdx.x; i < kTileRows * 16 * RT; i += 256) {
    const int row = i / (16 * RT), r = i - row * (16 * RT);
    float s = 0.0f;
    if (row < tile.count && r < rank) {
      for (int k = 0; k < splits; ++k) s += part[((size_t)k * M + tile.begin + row) * (16 * RT) + r];
      if (blockIdx.y == 0 && kept) kept[(size_t)plan.perm[tile.begin + row] * rank + r] = KEEP_SCALED ? f * s : s;
      s *= f;
    }
    ts[row][r] = s;
  }
  __syncthreads();
  if (!out) return;
  f4 acc[2][4];
#pragma unroll
  for (int e = 0; e < 4; ++e) acc[0][e] = acc[1][e] = f4{0.0f, 0.0f, 0.0f, 0.0f};
  const T* b = B + (size_t)tile.adapter * rank * N + n;
  const int steps = (rank + 3) / 4;
  for (int s = 0; s < steps; ++s) {
    const int r = 4 * s + quarter;
    const f4 w = load4<QUADS>(b + (size_t)r * N, n, r < rank ? N : 0);
    const float u = ts[col][r], v = ts[col + 16][r];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      acc[0][e] = __builtin_amdgcn_mfma_f32_16x16x4f32(u, w[e], acc[0][e], 0, 0, 0);
      acc[1][e] = __builtin_amdgcn_mfma_f32_16x16x4f32(v, w[e], acc[1][e], 0, 0, 0);
    }
  }
#pragma unroll
  for (int h = 0; h < 2; ++h)
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int row = 16 * h + 4 * quarter + i;
      if (row < tile.count) {
        const size_t at = (size_t)plan.perm[tile.begin + row] * N + n;
        f4 v = load4<QUADS>(base + at, n, N);
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] += acc[h][e][i];
        store4<QUADS>(out + at, v, n, N);
      }
    }
}

// grad[adapter][r][k] = scale sum_m S[m][r] X[m][k] over a chunk's rows: into the gradient where the adapter has no other chunk, else into
// the chunk's slot.  The instruction adds up over four rows, one per quarter of the wave.
template <bool QUADS, int RT>
__device__ __forceinline__ void outer_of(const PlanAt& plan, const Entry& chunk, int strip, const float* S, const float* X, float f, float* grad,
                                         float* slots, int K, int rank) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, col = lane & 15, quarter = lane >> 4;
  const int k = strip * 256 + 64 * wave + 4 * col;
  if (strip * 256 + 64 * wave >= K) return;
  f4 acc[RT][4];
#pragma unroll
  for (int t = 0; t < RT; ++t)
#pragma unroll
    for (int e = 0; e < 4; ++e) acc[t][e] = f4{0.0f, 0.0f, 0.0f, 0.0f};
  for (int i = 0; i < chunk.count; i += 4) {
    const bool in = i + quarter < chunk.count;
    const size_t m = (size_t)plan.perm[chunk.begin + min(i + quarter, chunk.count - 1)];
    const f4 x = load4<QUADS>(X + m * K + k, k, in ? K : 0);
    float s[RT];
#pragma unroll
    for (int t = 0; t < RT; ++t) s[t] = in ? S[m * rank + min(16 * t + col, rank - 1)] : 0.0f;
#pragma unroll
    for (int t = 0; t < RT; ++t)
#pragma unroll
      for (int e = 0; e < 4; ++e) acc[t][e] = __builtin_amdgcn_mfma_f32_16x16x4f32(s[t], x[e], acc[t][e], 0, 0, 0);
  }
  float* to = chunk.slot < 0 ? grad + (size_t)chunk.adapter * rank * K : slots + (size_t)chunk.slot * rank * K;
#pragma unroll
  for (int t = 0; t < RT; ++t)
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int r = 16 * t + 4 * quarter + i;
      if (r < rank) store4<QUADS>(to + (size_t)r * K + k, f4{f * acc[t][0][i], f * acc[t][1][i], f * acc[t][2][i], f * acc[t][3][i]}, k, K);
    }
}

struct Outer {
  const float *S, *X;       // S: [row][rank]
  float *grad, *slots;
  int K, strips;
};

// Both gradients in one launch: the first strips are dA's (S = dT), the others dB's (S = T, times scale).
template <bool QUADS, int RT>
__global__ __launch_bounds__(256) void outer_kernel(PlanAt plan, Outer a, Outer b, const float* scale, int M, int rank, int adapters) {
  if (!planned(plan, M, adapters) || (int)blockIdx.x >= plan.head[4]) return;
  const Entry chunk = plan.chunks[blockIdx.x];
  if ((int)blockIdx.y < a.strips) outer_of<QUADS, RT>(plan, chunk, blockIdx.y, a.S, a.X, 1.0f, a.grad, a.slots, a.K, rank);
  else outer_of<QUADS, RT>(plan, chunk, blockIdx.y - a.strips, b.S, b.X, scale[chunk.adapter], b.grad, b.slots, b.K, rank);
}

// Gradients of adapters with several chunks, or with none.
__global__ __launch_bounds__(256) void outer_join_kernel(PlanAt plan, Outer a, Outer b, int M, int rank, int adapters) {
  if (!planned(plan, M, adapters)) return;
  const int id = blockIdx.x, chunks = plan.chunk0[id + 1] - plan.chunk0[id];
  if (chunks == 1) return;
  const int slot = plan.slot0[id];
  for (int h = 0; h < 2; ++h) {
    const Outer& o = h ? b : a;
    const size_t each = (size_t)rank * o.K;
    for (size_t i = (size_t)blockIdx.y * 256 + threadIdx.x; i < each; i += (size_t)gridDim.y * 256) {
      float s = 0.0f;
      for (int k = 0; k < chunks; ++k) s += o.slots[(size_t)(slot + k) * each + i];
      o.grad[(size_t)id * each + i] = s;
    }
  }
}

// ---- launches --------------------------------------------------------------------------------------
inline int rank_tiles(int rank) { return rank <= 16 ? 1 : rank <= 32 ? 2 : rank <= 64 ? 4 : 8; }

// Shares of K: about 1024 blocks, at least one step of all four waves each, 32 at most (their sums are read by every block of columns).
struct Split {
  int splits, per_split;
  Split(int M, int K, int adapters) {
    const long long tiles = max_tiles(M, adapters);
    const int wanted = (int)std::max<long long>(1, std::min<long long>(32, 1024 / tiles));
    per_split = std::max(64, ((K + wanted - 1) / wanted + 63) / 64 * 64);
    splits = (K + per_split - 1) / per_split;
  }
};

int shape_ok(int M, int K, int N, int rank, int adapters) {
  if (M <= 0 || K <= 0 || N <= 0 || rank <= 0 || adapters <= 0 || rank > kMaxRank) return XBAR_ESHAPE;
  if (M > (1 << 24) || K >= (1 << 24) || N >= (1 << 24) || adapters > 65536) return XBAR_ESHAPE;
  if ((double)M * std::max(K, N) >= 274877906944.0 || (double)adapters * rank * std::max(K, N) >= 274877906944.0) return XBAR_ESHAPE;
  return XBAR_OK;
}

struct WorkAt {
  float *part, *dT, *slotsA, *slotsB;
};
size_t work_layout(void* ws, int op, int M, int K, int N, int rank, int adapters, WorkAt* at) {
  char* p = reinterpret_cast<char*>(ws);
  size_t off = 0;
  auto take = [&](size_t floats) {
    char* q = p + off;
    off += align256(floats * sizeof(float));
    return reinterpret_cast<float*>(q);
  };
  WorkAt w{};
  w.part = take((size_t)Split(M, op == XBAR_OP_FWD ? K : N, adapters).splits * M * 16 * rank_tiles(rank));
  if (op == XBAR_OP_BWD) {
    w.dT = take((size_t)M * rank);
    w.slotsA = take((size_t)max_slots(M) * rank * K);
    w.slotsB = take((size_t)max_slots(M) * rank * N);
  }
  if (at) *at = w;
  return off;
}

// Kernels of a type, of rows that are quads or not, and of a rank.
template <class T, bool QUADS, int RT>
struct Kernels {
  static int shrink(const PlanAt& plan, const float* X, const void* A, float* part, int M, int K, int rank, int adapters, const Split& s, hipStream_t st) {
    hipLaunchKernelGGL((shrink_kernel<T, QUADS, RT>), dim3((unsigned)max_tiles(M, adapters), (unsigned)s.splits), dim3(256), 0, st, plan, X,
                       reinterpret_cast<const T*>(A), part, M, K, rank, adapters, s.per_split);
    return launched();
  }
  template <bool KEEP_SCALED>
  static int expand(const PlanAt& plan, const float* base, const float* part, int splits, const float* scale, const void* B, float* out, float* kept,
                    int M, int N, int rank, int adapters, hipStream_t st) {
    hipLaunchKernelGGL((expand_kernel<T, QUADS, RT, KEEP_SCALED>), dim3((unsigned)max_tiles(M, adapters), out ? (unsigned)((N + 255) / 256) : 1u),
                       dim3(256), 0, st, plan, base, part, splits, scale, reinterpret_cast<const T*>(B), out, kept, M, N, rank, adapters);
    return launched();
  }
  static int outer(const PlanAt& plan, const Outer& a, const Outer& b, const float* scale, int M, int rank, int adapters, hipStream_t st) {
    hipLaunchKernelGGL((outer_kernel<QUADS, RT>), dim3((unsigned)max_chunks(M, adapters), (unsigned)(a.strips + b.strips)), dim3(256), 0, st, plan, a,
                       b, scale, M, rank, adapters);
    return launched();
  }
};

template <class F>
int with_kernels(int type, bool quads, int rank, F f) {
  auto with_rank = [&](auto t, auto q) {
    typedef decltype(t) T;
    constexpr bool Q = decltype(q)::value;
    switch (rank_tiles(rank)) {
      case 1: return f(Kernels<T, Q, 1>());
      case 2: return f(Kernels<T, Q, 2>());
      case 4: return f(Kernels<T, Q, 4>());
      default: return f(Kernels<T, Q, 8>());
    }
  };
  if (type == XBAR_BF16) return quads ? with_rank(uint16_t(), std::true_type()) : with_rank(uint16_t(), std::false_type());
  return quads ? with_rank(float(), std::true_type()) : with_rank(float(), std::false_type());
}

}  // namespace

extern "C" {

size_t xbar_adapter_plan_bytes(int M, int adapters) {
  return shape_ok(M, 1, 1, 1, adapters) ? 0 : plan_layout(nullptr, M, adapters, nullptr);
}

int xbar_adapter_plan(const int32_t* rows, int M, int adapters, void* plan, size_t plan_bytes, void* hip_stream) {
  if (shape_ok(M, 1, 1, 1, adapters)) return XBAR_ESHAPE;
  if (!aligned16(rows) || !aligned16(plan)) return XBAR_EALIGN;
  PlanAt p;
  if (plan_bytes < plan_layout(plan, M, adapters, &p)) return XBAR_EWORKSPACE;
  hipStream_t st = reinterpret_cast<hipStream_t>(hip_stream);
  const dim3 waves((unsigned)((adapters + 4) / 4));
  hipLaunchKernelGGL(plan_count_kernel, waves, dim3(256), 0, st, rows, M, adapters, p);
  if (launched()) return XBAR_EHIP;
  hipLaunchKernelGGL(plan_prefix_kernel, dim3(1), dim3(1024), 0, st, M, adapters, p);
  if (launched()) return XBAR_EHIP;
  hipLaunchKernelGGL(plan_place_kernel, waves, dim3(256), 0, st, rows, M, adapters, p);
  return launched();
}

size_t xbar_adapter_workspace_bytes(int op, int M, int K, int N, int rank, int adapters) {
  if (shape_ok(M, K, N, rank, adapters) || (op != XBAR_OP_FWD && op != XBAR_OP_BWD)) return 0;
  return work_layout(nullptr, op, M, K, N, rank, adapters, nullptr);
}

int xbar_adapter_fwd(const void* plan, size_t plan_bytes, const float* base, const float* X, const void* A, const void* B, int type,
                     const float* scale, float* Y, float* T, int M, int K, int N, int rank, int adapters, void* ws, size_t ws_bytes,
                     void* hip_stream) {
  if (shape_ok(M, K, N, rank, adapters)) return XBAR_ESHAPE;
  if (type != XBAR_F32 && type != XBAR_BF16) return XBAR_EINVAL;
  if (!aligned16(plan) || !aligned16(base) || !aligned16(X) || !aligned16(A) || !aligned16(B) || !aligned16(scale) || !aligned16(Y) ||
      (T && !aligned16(T)) || !aligned16(ws))
    return XBAR_EALIGN;
  PlanAt p;
  if (plan_bytes < plan_layout(const_cast<void*>(plan), M, adapters, &p)) return XBAR_EWORKSPACE;
  WorkAt w;
  if (ws_bytes < work_layout(ws, XBAR_OP_FWD, M, K, N, rank, adapters, &w)) return XBAR_EWORKSPACE;
  const size_t x = (size_t)M * K * 4, y = (size_t)M * N * 4, t = (size_t)M * rank * 4, each = type == XBAR_BF16 ? 2 : 4;
  const size_t a = (size_t)adapters * rank * K * each, b = (size_t)adapters * rank * N * each;
  if ((Y != base && overlap(Y, y, base, y)) || overlap(Y, y, X, x) || overlap(Y, y, A, a) || overlap(Y, y, B, b) || overlap(Y, y, T, t) ||
      overlap(T, t, X, x) || overlap(T, t, base, y) || overlap(T, t, A, a) || overlap(T, t, B, b))
    return XBAR_EINVAL;
  hipStream_t st = reinterpret_cast<hipStream_t>(hip_stream);
  const Split s(M, K, adapters);
  const int rc = with_kernels(type, K % 4 == 0, rank, [&](auto k) { return k.shrink(p, X, A, w.part, M, K, rank, adapters, s, st); });
  if (rc) return rc;
  return with_kernels(type, N % 4 == 0, rank, [&](auto k) {
    return k.template expand<false>(p, base, w.part, s.splits, scale, B, Y, T, M, N, rank, adapters, st);
  });
}

int xbar_adapter_bwd(const void* plan, size_t plan_bytes, const float* base, const float* dY, const float* X, const float* T, const void* A,
                     const void* B, int type, const float* scale, float* dX, float* dA, float* dB, int M, int K, int N, int rank, int adapters,
                     void* ws, size_t ws_bytes, void* hip_stream) {
  if (shape_ok(M, K, N, rank, adapters)) return XBAR_ESHAPE;
  if (type != XBAR_F32 && type != XBAR_BF16) return XBAR_EINVAL;
  if (!aligned16(plan) || (dX && !aligned16(base)) || !aligned16(dY) || !aligned16(X) || !aligned16(T) || !aligned16(A) || !aligned16(B) ||
      !aligned16(scale) || (dX && !aligned16(dX)) || !aligned16(dA) || !aligned16(dB) || !aligned16(ws))
    return XBAR_EALIGN;
  PlanAt p;
  if (plan_bytes < plan_layout(const_cast<void*>(plan), M, adapters, &p)) return XBAR_EWORKSPACE;
  WorkAt w;
  if (ws_bytes < work_layout(ws, XBAR_OP_BWD, M, K, N, rank, adapters, &w)) return XBAR_EWORKSPACE;
  const size_t each = type == XBAR_BF16 ? 2 : 4, na = (size_t)adapters * rank * K, nb = (size_t)adapters * rank * N;
  struct Tensor { const void* p; size_t bytes; };
  const Tensor in[] = {{dY, (size_t)M * N * 4}, {X, (size_t)M * K * 4}, {T, (size_t)M * rank * 4}, {A, na * each}, {B, nb * each},
                       {dX && dX != base ? base : nullptr, (size_t)M * K * 4}};
  const Tensor out[] = {{dX, (size_t)M * K * 4}, {dA, na * 4}, {dB, nb * 4}};
  for (int i = 0; i < 3; ++i) {
    for (const Tensor& q : in)
      if (overlap(out[i].p, out[i].bytes, q.p, q.bytes)) return XBAR_EINVAL;
    for (int j = 0; j < i; ++j)
      if (overlap(out[i].p, out[i].bytes, out[j].p, out[j].bytes)) return XBAR_EINVAL;
  }
  hipStream_t st = reinterpret_cast<hipStream_t>(hip_stream);
  const Split s(M, N, adapters);
  int rc = with_kernels(type, N % 4 == 0, rank, [&](auto k) { return k.shrink(p, dY, B, w.part, M, N, rank, adapters, s, st); });
  if (rc) return rc;
  rc = with_kernels(type, K % 4 == 0, rank, [&](auto k) {
    return k.template expand<true>(p, base, w.part, s.splits, scale, A, dX, w.dT, M, K, rank, adapters, st);
  });
  if (rc) return rc;
  const Outer oa{w.dT, X, dA, w.slotsA, K, (K + 255) / 256}, ob{T, dY, dB, w.slotsB, N, (N + 255) / 256};
  rc = with_kernels(XBAR_F32, K % 4 == 0 && N % 4 == 0, rank, [&](auto k) { return k.outer(p, oa, ob, scale, M, rank, adapters, st); });
  if (rc) return rc;
  const size_t most = (size_t)rank * std::max(K, N);
  hipLaunchKernelGGL(outer_join_kernel, dim3((unsigned)adapters, (unsigned)std::min<size_t>(64, (most + 1023) / 1024)), dim3(256), 0, st, p, oa, ob, M,
                     rank, adapters);
  return launched();
}

}  // extern "C"
