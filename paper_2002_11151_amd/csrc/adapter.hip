// Low-rank adapters of many requests beside a shared projection: the projection runs on programmed crossbars, whose devices are not
// written for every task; each task adds a digital correction of rank r,
//   T[m][r] = sum_k X[m][k] A[a][r][k],   Y[m][n] = base[m][n] + sum_r scale[a] T[m][r] B[a][r][n],   a = adapter of row m.
// A and B are kept the same way round (rows of the rank), so both directions are three products:
//   shrink  T = X A^T (forward),            dT = scale dY B^T (backward)          one pass over the wide operand
//   expand  Y = base + scale T B,           dX = base + dT A                      one pass over base and output
//   outer   dA = dT^T X, dB = scale T^T dY                                        one pass over the wide operand
// All on v_mfma_f32_16x16x4_f32: single precision throughout; 2 M r (K + N) operations at 154 TFLOP/s take as long as 4 M (K + 2 N) bytes at
// 5.2 TB/s at a rank of 90 or so (K = N): below that memory is the bound.  Rows are taken in the order of their adapters (the plan), in tiles and chunks that hold one adapter each.
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
  int* rows;            // [tiles][kTileRows]: rows of a tile, the last one repeated: known without the tile's entry
};
constexpr int kMagic = 0x70ada37e;

__host__ __device__ inline int chunk_rows(int M) {
  const int many = (M / 32 + 31) / 32 * 32;
  return many > 256 ? many : 256;
}
inline long long max_tiles(int M, int adapters) { return (long long)M / kTileRows + std::min<long long>(M, (long long)adapters + 1) + 1; }
inline long long max_chunks(int M, int adapters) { return (long long)M / chunk_rows(M) + std::min<long long>(M, (long long)adapters + 1) + 1; }
// Chunks of adapters with more than one.
inline long long max_slots(int M) { return 2ll * M / chunk_rows(M) + 2; }

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
  l.rows = reinterpret_cast<int*>(take((size_t)max_tiles(M, adapters) * kTileRows * sizeof(int)));
  if (at) *at = l;
  return off;
}

__device__ __forceinline__ int bin_of(int id, int adapters) { return (unsigned)id < (unsigned)adapters ? id : adapters; }

// Bins of rows m .. m + 3, -1 beyond M.
__device__ __forceinline__ int4 bins_of(const int32_t* rows, int m, int M, int adapters) {
  int4 v = make_int4(-1, -1, -1, -1);
  if (m + 3 < M) {
    const int4 id = *reinterpret_cast<const int4*>(rows + m);
    v = make_int4(bin_of(id.x, adapters), bin_of(id.y, adapters), bin_of(id.z, adapters), bin_of(id.w, adapters));
  } else {
    if (m < M) v.x = bin_of(rows[m], adapters);
    if (m + 1 < M) v.y = bin_of(rows[m + 1], adapters);
    if (m + 2 < M) v.z = bin_of(rows[m + 2], adapters);
  }
  return v;
}

// Rows of every adapter (bin `adapters`: rows without one), one wave per bin over all rows: this and the placing read rows x adapters numbers
// (65536 rows, 2048 adapters: 52 + 106 us, from the caches).
__global__ __launch_bounds__(256) void plan_count_kernel(const int32_t* rows, int M, int adapters, PlanAt p) {
  const int bin = blockIdx.x * 4 + (threadIdx.x >> 6), lane = threadIdx.x & 63;
  if (bin > adapters) return;
  int n = 0;
  for (int m0 = 0; m0 < M; m0 += 2048) {                        // eight loads in flight
    int4 id[8];
#pragma unroll
    for (int u = 0; u < 8; ++u) id[u] = bins_of(rows, m0 + 256 * u + 4 * lane, M, adapters);
#pragma unroll
    for (int u = 0; u < 8; ++u) n += (id[u].x == bin) + (id[u].y == bin) + (id[u].z == bin) + (id[u].w == bin);
  }
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
  int at = begin, last = 0;
  int* padded = p.rows + (size_t)p.tile0[bin] * kTileRows;
  const unsigned long long below = (1ull << lane) - 1;
  for (int m0 = 0; m0 < M; m0 += 2048) {
    int4 id[8];
#pragma unroll
    for (int u = 0; u < 8; ++u) id[u] = bins_of(rows, m0 + 256 * u + 4 * lane, M, adapters);
#pragma unroll
    for (int u = 0; u < 8; ++u) {
      const int four[4] = {id[u].x, id[u].y, id[u].z, id[u].w}, m = m0 + 256 * u + 4 * lane;
      unsigned long long all[4];
      int place = at;                                           // behind all of the lanes before
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        all[e] = __ballot(four[e] == bin);
        place += __popcll(all[e] & below);
        at += __popcll(all[e]);
      }
#pragma unroll
      for (int e = 0; e < 4; ++e)
        if (four[e] == bin) {
          p.perm[place] = m + e;
          padded[place - begin] = m + e;
          ++place;
        }
#pragma unroll
      for (int e = 0; e < 4; ++e)
        if (all[e]) last = max(last, m0 + 256 * u + 4 * (63 - __clzll(all[e])) + e);
    }
  }
  const int odd = (end - begin) % kTileRows;
  if (odd && lane < kTileRows - odd) padded[end - begin + lane] = last;
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

// The whole plan of a batch of up to 256 rows in one block and launch: a row's place is the number of rows before it in the order (adapter,
// row), counted from all pairs in LDS.  An adapter has one chunk at most.  (128 rows, 64 adapters: 6.8 us, one row 2.9; 300 rows, 64 adapters
// in three launches: 3.4 + 4.3 + 5.9.)
constexpr int kSmallPlan = 256;
static_assert(kSmallPlan <= 256, "chunk_rows() of the smallest batches");
__global__ __launch_bounds__(kSmallPlan) void plan_small_kernel(const int32_t* rows, int M, int adapters, PlanAt p) {
  __shared__ __align__(16) int ids[kSmallPlan];
  __shared__ int sorted[kSmallPlan], order[kSmallPlan], chunks_before[kSmallPlan];
  __shared__ int part[2][kSmallPlan / 64], edge[2][kSmallPlan / 64];
  const int i = threadIdx.x, lane = i & 63, wave = i >> 6;
  const int mine = i < M ? bin_of(rows[i], adapters) : adapters + 1;                // beyond M: behind all others
  ids[i] = mine;
  __syncthreads();
  int place = 0;
#pragma unroll 4
  for (int k = 0; k < M; k += 4) {
    const int4 v = *reinterpret_cast<const int4*>(ids + k);
    place += (v.x < mine || (v.x == mine && k < i)) + (v.y < mine || (v.y == mine && k + 1 < i)) + (v.z < mine || (v.z == mine && k + 2 < i)) +
             (v.w < mine || (v.w == mine && k + 3 < i));
  }
  if (i < M) {
    sorted[place] = mine;
    order[place] = i;
    p.perm[place] = i;
  }
  __syncthreads();
  const int bin = i < M ? sorted[i] : adapters + 1;
  const unsigned long long heads = __ballot(i <= M && (i == 0 || (i < M ? bin : adapters + 1) != sorted[i - 1])), below = (1ull << lane) - 1;
  if (lane == 0) {
    edge[0][wave] = heads ? 64 * wave + __ffsll(heads) - 1 : kSmallPlan;          // the wave's first run and last one
    edge[1][wave] = heads ? 64 * wave + 63 - __clzll(heads) : -1;
  }
  __syncthreads();
  const unsigned long long until = heads & (below | 1ull << lane), after = heads & ~(below | 1ull << lane);
  int begin = until ? 64 * wave + 63 - __clzll(until) : -1, end = after ? 64 * wave + __ffsll(after) - 1 : kSmallPlan;
#pragma unroll
  for (int w = 0; w < kSmallPlan / 64; ++w) {
    if (w < wave && !until) begin = max(begin, edge[1][w]);
    if (w > wave && !after) end = min(end, edge[0][w]);
  }
  end = min(end, M);
  const bool tile = i < M && (i - begin) % kTileRows == 0, chunk = i < M && i == begin && bin < adapters;
  const unsigned long long tiles = __ballot(tile), chunks = __ballot(chunk);
  if (lane == 0) {
    part[0][wave] = __popcll(tiles);
    part[1][wave] = __popcll(chunks);
  }
  __syncthreads();
  int t0 = __popcll(tiles & below), c0 = __popcll(chunks & below), all_tiles = 0, all_chunks = 0;
#pragma unroll
  for (int w = 0; w < kSmallPlan / 64; ++w) {
    t0 += w < wave ? part[0][w] : 0;
    c0 += w < wave ? part[1][w] : 0;
    all_tiles += part[0][w];
    all_chunks += part[1][w];
  }
  chunks_before[i] = c0;
  if (tile) {
    const int count = min(kTileRows, end - i);
    p.tiles[t0] = Entry{bin < adapters ? bin : -1, i, count, 0};
    int4* to = reinterpret_cast<int4*>(p.rows + t0 * kTileRows);
#pragma unroll
    for (int k = 0; k < kTileRows; k += 4)
      to[k / 4] = make_int4(order[i + min(k, count - 1)], order[i + min(k + 1, count - 1)], order[i + min(k + 2, count - 1)],
                            order[i + min(k + 3, count - 1)]);
  }
  if (chunk) p.chunks[c0] = Entry{bin, i, end - i, -1};
  if (i == 0) {
    p.head[0] = kMagic;
    p.head[1] = M;
    p.head[2] = adapters;
    p.head[3] = all_tiles;
    p.head[4] = all_chunks;
  }
  __syncthreads();
  for (int a = i; a <= adapters; a += kSmallPlan) {
    int from = 0, to = M;                                       // first place of this adapter or a later one
    while (from < to) {
      const int mid = (from + to) >> 1;
      if (sorted[mid] < a) from = mid + 1;
      else to = mid;
    }
    p.chunk0[a] = from < M ? chunks_before[from] : all_chunks;
  }
}

__device__ __forceinline__ bool planned(const PlanAt& p, int M, int adapters) {
  return p.head[0] == kMagic && p.head[1] == M && p.head[2] == adapters;
}

// ---- the products ----------------------------------------------------------------------------------
__device__ __forceinline__ float wide(uint16_t x) { return __uint_as_float((uint32_t)x << 16); }   // bfloat16

// The base passes through once and should not take the caches' room.  (The output is stored the ordinary way: 4096 x 4096 values and a ReLU
// that reads them take 57 us together, 62 if the output passes the caches by.)
__device__ __forceinline__ f4 once4(const float* p) { return __builtin_nontemporal_load(reinterpret_cast<const f4*>(p)); }

// Four values from p on, those at place k and beyond `end` zero; QUADS: all or none of the four are inside, and p is aligned.
template <bool QUADS, bool ONCE = false>
__device__ __forceinline__ f4 load4(const float* p, int k, int end) {
  f4 v = {0.0f, 0.0f, 0.0f, 0.0f};
  if constexpr (QUADS) {
    if (k < end) v = ONCE ? once4(p) : *reinterpret_cast<const f4*>(p);
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

// 4 x 4 transposition inside every four neighbouring lanes: register i of lane j goes to register j of lane i.  PERM: whose value a lane
// takes; upper lanes take the other's b for their a, lower lanes the other's a for their b.
template <int PERM>
__device__ __forceinline__ void exchange(float& a, float& b, bool upper) {
  const float from_a = __int_as_float(__builtin_amdgcn_mov_dpp(__float_as_int(a), PERM, 0xF, 0xF, true));
  const float from_b = __int_as_float(__builtin_amdgcn_mov_dpp(__float_as_int(b), PERM, 0xF, 0xF, true));
  a = upper ? from_b : a;
  b = upper ? b : from_a;
}
__device__ __forceinline__ void quad_transpose(f4& v0, f4& v1, f4& v2, f4& v3, bool odd, bool high) {
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    float a = v0[e], b = v1[e], c = v2[e], d = v3[e];
    exchange<0xB1>(a, b, odd);           // lanes 1 0 3 2
    exchange<0xB1>(c, d, odd);
    exchange<0x4E>(a, c, high);          // lanes 2 3 0 1
    exchange<0x4E>(b, d, high);
    v0[e] = a; v1[e] = b; v2[e] = c; v3[e] = d;
  }
}

// part[split][sorted row][16 RT] = X A^T over the split's share of K.  Block: one tile, its four waves side by side along K, joined in
// LDS.  A wave takes 64 k at a time.  The instruction wants lane = row + 16 slot, but loads in which neighbouring lanes lie in different
// rows cost an access of the vector cache per lane (measured: 61 per load instead of 16); so lane 4 g + j of quarter q loads k =
// 16 q + 4 j of row 4 g + i for i = 0 .. 3 (64 neighbouring bytes per four lanes), and a transposition inside the four lanes leaves every
// lane with its own row: register s holds k = 16 q + 4 s, from both operands, so instruction (s, e) adds up k = 16 q + 4 s + e over the
// quarters q.  Rows beyond the tile and ranks beyond the last repeat a valid one: their products are not stored.
// Bound by memory and the issue of loads and products together: 4096 x 4096 floats by rank 32 of 8 adapters 24 us (2.8 TB/s of X; 31 with a lane
// per row), 128 rows of 57 bfloat16 adapters of rank 16 8.1 us, one row 3.8.
template <class T, bool QUADS, int RT>
__global__ __launch_bounds__(256, RT == 1 ? 4 : RT == 2 ? 3 : RT == 4 ? 2 : 1) void shrink_kernel(PlanAt plan, const float* X, const T* A, float* part, int M, int K, int rank, int adapters,
                                                     int splits, int per_split) {
  __shared__ float red[4][kTileRows][16 * RT];
  const int item = blockIdx.x / splits, split = blockIdx.x - item * splits;       // neighbouring blocks: the same rows
  const Entry tile = plan.tiles[item];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, col = lane & 15, quarter = lane >> 4;
  const int four = col & ~3, ahead = 16 * quarter + 4 * (col & 3);
  int row_of_tile[2][4];                                        // on its way with the entry
#pragma unroll
  for (int h = 0; h < 2; ++h)
#pragma unroll
    for (int i = 0; i < 4; ++i) row_of_tile[h][i] = plan.rows[item * kTileRows + 16 * h + four + i];
  if (!planned(plan, M, adapters) || item >= plan.head[3] || tile.adapter < 0) return;
  const bool two = tile.count > 16, odd = lane & 1, high = lane & 2;
  const float* x[2][4];
#pragma unroll
  for (int h = 0; h < 2; ++h)
#pragma unroll
    for (int i = 0; i < 4; ++i) x[h][i] = X + (size_t)row_of_tile[h][i] * K + ahead;
  const T* a = A + (size_t)tile.adapter * rank * K;
  unsigned row[RT][4];
#pragma unroll
  for (int t = 0; t < RT; ++t)
#pragma unroll
    for (int i = 0; i < 4; ++i) row[t][i] = (unsigned)min(16 * t + four + i, rank - 1) * (unsigned)K + ahead;
  f4 acc[2][RT];
#pragma unroll
  for (int t = 0; t < RT; ++t) acc[0][t] = acc[1][t] = f4{0.0f, 0.0f, 0.0f, 0.0f};
  const int k1 = min((split + 1) * per_split, K);
  for (int k = split * per_split + 64 * wave; k < k1; k += 256) {
    f4 u[4], w[4] = {}, b[RT][4];
#pragma unroll
    for (int i = 0; i < 4; ++i) u[i] = load4<QUADS>(x[0][i] + k, k + ahead, k1);
    if (two)
#pragma unroll
      for (int i = 0; i < 4; ++i) w[i] = load4<QUADS>(x[1][i] + k, k + ahead, k1);
#pragma unroll
    for (int t = 0; t < RT; ++t)
#pragma unroll
      for (int i = 0; i < 4; ++i) b[t][i] = load4<QUADS>(a + (row[t][i] + (unsigned)k), k + ahead, k1);
    quad_transpose(u[0], u[1], u[2], u[3], odd, high);
    if (two) quad_transpose(w[0], w[1], w[2], w[3], odd, high);
#pragma unroll
    for (int t = 0; t < RT; ++t) {
      quad_transpose(b[t][0], b[t][1], b[t][2], b[t][3], odd, high);
#pragma unroll
      for (int s = 0; s < 4; ++s)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          acc[0][t] = __builtin_amdgcn_mfma_f32_16x16x4f32(u[s][e], b[t][s][e], acc[0][t], 0, 0, 0);
          if (two) acc[1][t] = __builtin_amdgcn_mfma_f32_16x16x4f32(w[s][e], b[t][s][e], acc[1][t], 0, 0, 0);
        }
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
    const int row_of = i / (16 * RT), r = i - row_of * (16 * RT);
    part[((size_t)split * M + tile.begin + row_of) * (16 * RT) + r] =
        (red[0][row_of][r] + red[1][row_of][r]) + (red[2][row_of][r] + red[3][row_of][r]);
  }
}

// Sum of `splits` values `each` apart, in their order, eight loads in flight.
__device__ __forceinline__ float sum_of_splits(const float* part, size_t each, int splits) {
  float s = 0.0f;
  for (int k0 = 0; k0 < splits; k0 += 8) {
    float v[8];
#pragma unroll
    for (int k = 0; k < 8; ++k) v[k] = part[(size_t)min(k0 + k, splits - 1) * each];
#pragma unroll
    for (int k = 0; k < 8; ++k) s += k0 + k < splits ? v[k] : 0.0f;
  }
  return s;
}

// out = base + sum over ranks of scale (sum of the splits) B.  Block: one tile and `cols` columns.  A wave takes 16 rows and 64 columns at a
// time: two waves the tile's halves and two column by column beside them, or all four side by side where the tile has up to 16 rows.
// A lane's 16-byte loads of B hold four neighbouring columns, one for each of four matrix tiles, so that base and out are touched 16
// bytes wide too; the first loads are on their way while the block adds up the splits.  The blocks of the first columns also keep the sums
// (`kept`: in the rows' own order).  4096 x 4096 outputs, rank 32: 42 us (3.2 TB/s; 32 without the loads of B, which are as many as those of the base
// and the output); 128 rows of 57 adapters 6.7; one row 3.6.
template <class T, bool QUADS, int RT>
__global__ __launch_bounds__(256, RT <= 2 ? 4 : 2) void expand_kernel(PlanAt plan, const float* base, const float* part, int splits, const float* scale, const T* B,
                                                        float* out, float* kept, int M, int N, int rank, int adapters, int cols, int strips) {
  __shared__ float ts[kTileRows][16 * RT + 1];
  const int item = blockIdx.x / strips, strip = blockIdx.x - item * strips;       // neighbouring blocks: the same rows
  const Entry tile = plan.tiles[item];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, col = lane & 15, quarter = lane >> 4;
  int row_of_tile[2][4];                                        // on its way with the entry
#pragma unroll
  for (int h = 0; h < 2; ++h)
#pragma unroll
    for (int i = 0; i < 4; ++i) row_of_tile[h][i] = plan.rows[item * kTileRows + 16 * h + 4 * quarter + i];
  if (!planned(plan, M, adapters) || item >= plan.head[3]) return;
  const int n1 = min((strip + 1) * cols, N);
  if (tile.adapter < 0) {                                      // rows without an adapter: as they were
    if (out != base)
      for (int i = quarter; i < tile.count; i += 4) {
        const size_t at = (size_t)plan.perm[tile.begin + i] * N;
        for (int n = strip * cols + 64 * wave + 4 * col; n < n1; n += 256)
          store4<QUADS>(out + at + n, load4<QUADS, true>(base + at + n, n, n1), n, n1);
      }
    if (strip == 0 && kept)
      for (int i = threadIdx.x; i < tile.count * rank; i += 256) kept[(size_t)plan.perm[tile.begin + i / rank] * rank + i % rank] = 0.0f;
    return;
  }
  const bool two = tile.count > 16;
  const int half = two ? 16 * (wave & 1) : 0, beside = two ? 128 : 256;           // first row of the wave, columns of all waves
  int n = strip * cols + 64 * (two ? wave >> 1 : wave);                           // of the wave; the lane's: + 4 col
  size_t row_at[4];
  bool in[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int row = half + 4 * quarter + i;
    in[i] = row < tile.count;
    row_at[i] = (size_t)(half ? row_of_tile[1][i] : row_of_tile[0][i]) * N + 4 * col;
  }
  const T* b = B + ((size_t)tile.adapter * rank + quarter) * N + 4 * col;
  constexpr int STEPS = 4 * RT, U = STEPS < 8 ? STEPS : 8;       // steps of four ranks; U of them loaded at a time
  f4 w[U], v[4];
  auto load_w = [&](int s0) {
#pragma unroll
    for (int s = 0; s < U; ++s) w[s] = load4<QUADS>(b + (size_t)(4 * (s0 + s)) * N + n, n + 4 * col, 4 * (s0 + s) + quarter < rank ? n1 : 0);
  };
  auto load_v = [&]() {
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = load4<QUADS, true>(base + row_at[i] + n, n + 4 * col, in[i] ? n1 : 0);
  };
  load_v();
  load_w(0);
  const float f = scale ? scale[tile.adapter] : 1.0f;
  for (int i = threadIdx.x; i < kTileRows * 16 * RT; i += 256) {
    const int row = i / (16 * RT), r = i - row * (16 * RT);
    float s = 0.0f;
    if (row < tile.count && r < rank) {
      s = sum_of_splits(part + (size_t)(tile.begin + row) * (16 * RT) + r, (size_t)M * 16 * RT, splits);
      if (strip == 0 && kept) kept[(size_t)plan.perm[tile.begin + row] * rank + r] = s;
      s *= f;
    }
    ts[row][r] = s;
  }
  __syncthreads();
  for (bool first = true; n < n1; n += beside, first = false) {
    if (!first) {
      load_v();
      load_w(0);
    }
    f4 acc[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) acc[e] = f4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll 1
    for (int s0 = 0; s0 < STEPS; s0 += U) {
      if (s0) load_w(s0);
#pragma unroll
      for (int s = 0; s < U; ++s) {
        const float t = ts[half + col][4 * (s0 + s) + quarter];
#pragma unroll
        for (int e = 0; e < 4; ++e) acc[e] = __builtin_amdgcn_mfma_f32_16x16x4f32(t, w[s][e], acc[e], 0, 0, 0);
      }
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
#pragma unroll
      for (int e = 0; e < 4; ++e) v[i][e] += acc[e][i];
      store4<QUADS>(out + row_at[i] + n, v[i], n + 4 * col, in[i] ? n1 : 0);
    }
  }
}

// sum[sorted row][16 RT] = scale times the sum of the splits, zero beyond the last rank.
template <int RT>
__global__ __launch_bounds__(256) void split_sum_kernel(PlanAt plan, const float* part, int splits, const float* scale, float* sum, int M, int rank,
                                                        int adapters) {
  const Entry tile = plan.tiles[blockIdx.x];
  if (!planned(plan, M, adapters) || (int)blockIdx.x >= plan.head[3] || tile.adapter < 0) return;
  const int i = blockIdx.y * 256 + threadIdx.x;
  if (i >= tile.count * 16 * RT) return;
  const size_t at = (size_t)tile.begin * 16 * RT + i;
  sum[at] = i % (16 * RT) < rank ? scale[tile.adapter] * sum_of_splits(part + at, (size_t)M * 16 * RT, splits) : 0.0f;
}

struct Outer {
  const float *S, *X;       // S: [row][rank], or [sorted row][stride] with `sorted`
  float *grad, *slots;
  int K, strips, stride, sorted;
};

// grad[adapter][r][k] = f sum_m S[m][r] X[m][k] over a chunk's rows: into the gradient where the adapter has no other chunk, else into
// the chunk's slot.  Block: 64 columns; its four waves take every fourth step of four rows each and are joined in LDS, two and two.  The
// instruction adds up over four rows, one per quarter of the wave.  A wave's loads of eight steps are in flight together (2048 rows, 4096 + 4096
// columns, rank 16: 66 us with one step's, 18 with these, 3.8 TB/s).
template <bool QUADS, int RT>
__device__ __forceinline__ void outer_of(const PlanAt& plan, const Entry& chunk, int strip, const Outer& o, float f, int rank, f4 (&red)[2][RT][4][64]) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, col = lane & 15, quarter = lane >> 4, K = o.K;
  const int k = strip * 64 + 4 * col;
  f4 acc[RT][4];
#pragma unroll
  for (int t = 0; t < RT; ++t)
#pragma unroll
    for (int e = 0; e < 4; ++e) acc[t][e] = f4{0.0f, 0.0f, 0.0f, 0.0f};
  constexpr int U = RT <= 2 ? 8 : RT == 4 ? 4 : 2;
  for (int i0 = 4 * wave; i0 < chunk.count; i0 += 16 * U) {
    int m[U];
    f4 x[U];
    float s[U][RT];
#pragma unroll
    for (int u = 0; u < U; ++u) m[u] = plan.perm[chunk.begin + min(i0 + 16 * u + quarter, chunk.count - 1)];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int i = i0 + 16 * u + quarter;
      const bool in = i < chunk.count;
      x[u] = load4<QUADS>(o.X + (size_t)m[u] * K + k, k, in ? K : 0);
      const float* from = o.S + (o.sorted ? (size_t)(chunk.begin + min(i, chunk.count - 1)) : (size_t)m[u]) * o.stride;
#pragma unroll
      for (int t = 0; t < RT; ++t) s[u][t] = in ? from[min(16 * t + col, rank - 1)] : 0.0f;
    }
#pragma unroll
    for (int u = 0; u < U; ++u)
      if (i0 + 16 * u < chunk.count)                           // the wave's first row of the step
#pragma unroll
        for (int t = 0; t < RT; ++t)
#pragma unroll
          for (int e = 0; e < 4; ++e) acc[t][e] = __builtin_amdgcn_mfma_f32_16x16x4f32(s[u][t], x[u][e], acc[t][e], 0, 0, 0);
  }
  for (int half = 2; half; half >>= 1) {                      // waves 2 and 3 to 0 and 1, then 1 to 0
    if (half == 1) __syncthreads();
    if (wave >= half && wave < 2 * half)
#pragma unroll
      for (int t = 0; t < RT; ++t)
#pragma unroll
        for (int e = 0; e < 4; ++e) red[wave - half][t][e][lane] = acc[t][e];
    __syncthreads();
    if (wave < half)
#pragma unroll
      for (int t = 0; t < RT; ++t)
#pragma unroll
        for (int e = 0; e < 4; ++e) acc[t][e] += red[wave][t][e][lane];
  }
  if (wave) return;
  float* to = chunk.slot < 0 ? o.grad + (size_t)chunk.adapter * rank * K : o.slots + (size_t)chunk.slot * rank * K;
#pragma unroll
  for (int t = 0; t < RT; ++t)
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int r = 16 * t + 4 * quarter + i;
      if (r < rank) store4<QUADS>(to + (size_t)r * K + k, f4{f * acc[t][0][i], f * acc[t][1][i], f * acc[t][2][i], f * acc[t][3][i]}, k, K);
    }
}

// Both gradients in one launch: the first strips are dA's (S = dT), the others dB's (S = T, times scale); behind the chunks a strip's
// blocks, `zeros` of them, clear the gradients of adapters without rows.
template <bool QUADS, int RT>
__global__ __launch_bounds__(256) void outer_kernel(PlanAt plan, Outer a, Outer b, const float* scale, int M, int rank, int adapters, int chunks,
                                                    int zeros) {
  __shared__ f4 red[2][RT][4][64];
  const int item = blockIdx.x / (a.strips + b.strips), strip = blockIdx.x - item * (a.strips + b.strips);
  if (item >= chunks) {
    if (!planned(plan, M, adapters)) return;
    const Outer& o = strip < a.strips ? a : b;
    const int k = (strip < a.strips ? strip : strip - a.strips) * 64 + (threadIdx.x & 63);
    if (k >= o.K) return;
    for (int id = item - chunks; id < adapters; id += zeros)
      if (plan.chunk0[id] == plan.chunk0[id + 1])
        for (int r = threadIdx.x >> 6; r < rank; r += 4) o.grad[((size_t)id * rank + r) * o.K + k] = 0.0f;
    return;
  }
  const Entry chunk = plan.chunks[item];
  if (!planned(plan, M, adapters) || item >= plan.head[4]) return;
  if (strip < a.strips) outer_of<QUADS, RT>(plan, chunk, strip, a, 1.0f, rank, red);
  else outer_of<QUADS, RT>(plan, chunk, strip - a.strips, b, scale[chunk.adapter], rank, red);
}

// Gradients of adapters with several chunks; VEC values per thread.
template <int VEC>
__global__ __launch_bounds__(256) void outer_join_kernel(PlanAt plan, Outer a, Outer b, int M, int rank, int adapters) {
  if (!planned(plan, M, adapters)) return;
  const int id = blockIdx.x, chunks = plan.chunk0[id + 1] - plan.chunk0[id];
  if (chunks < 2) return;
  const int slot = plan.slot0[id];
  for (int h = 0; h < 2; ++h) {
    const Outer& o = h ? b : a;
    const size_t each = (size_t)rank * o.K;
    for (size_t i = ((size_t)blockIdx.y * 256 + threadIdx.x) * VEC; i < each; i += (size_t)gridDim.y * 256 * VEC) {
      f4 s = {0.0f, 0.0f, 0.0f, 0.0f};
      for (int k0 = 0; k0 < chunks; k0 += 8) {                // eight loads in flight, added in their order
        f4 v[8];
#pragma unroll
        for (int k = 0; k < 8; ++k) v[k] = load4<VEC == 4>(o.slots + (size_t)(slot + min(k0 + k, chunks - 1)) * each + i, 0, k0 + k < chunks ? VEC : 0);
#pragma unroll
        for (int k = 0; k < 8; ++k) s += v[k];
      }
      store4<VEC == 4>(o.grad + (size_t)id * each + i, s, 0, VEC);
    }
  }
}

// ---- launches --------------------------------------------------------------------------------------
inline int rank_tiles(int rank) { return rank <= 16 ? 1 : rank <= 32 ? 2 : rank <= 64 ? 4 : 8; }

// Shares of K: about 1024 blocks, at least 64 k for each of the four waves, 16 at most (every block of columns adds them up again).
struct Split {
  int splits, per_split;
  Split(int M, int K, int adapters) {
    const long long tiles = max_tiles(M, adapters);
    const int wanted = (int)std::max<long long>(1, std::min<long long>(16, 1024 / tiles));
    per_split = ((K + wanted - 1) / wanted + 255) / 256 * 256;
    splits = (K + per_split - 1) / per_split;
  }
};

// Columns of a block of expand_kernel: 1024 where that leaves about 1024 blocks, else fewer, 256 at least.
inline int columns(int M, int N, int adapters) {
  int cols = 1024;
  while (cols > 256 && max_tiles(M, adapters) * ((N + cols - 1) / cols) < 1024) cols >>= 1;
  return cols;
}

int shape_ok(int M, int K, int N, int rank, int adapters) {
  if (M <= 0 || K <= 0 || N <= 0 || rank <= 0 || adapters <= 0 || rank > kMaxRank) return XBAR_ESHAPE;
  if (M > (1 << 24) || K >= (1 << 24) || N >= (1 << 24) || adapters > 65536) return XBAR_ESHAPE;
  const double wide = std::max(K, N);
  if (M * wide >= 274877906944.0 || adapters * rank * wide >= 274877906944.0 || rank * wide >= 1073741824.0) return XBAR_ESHAPE;
  // blocks of a launch: below 2^24 (a launch has fewer than 2^32 threads)
  const double most = std::max(max_tiles(M, adapters) * std::max(16.0, (wide + 255) / 256), (max_chunks(M, adapters) + 4) * ((double)K + N + 126) / 64);
  return most >= 16777216.0 ? XBAR_ESHAPE : XBAR_OK;
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
    w.dT = take((size_t)M * 16 * rank_tiles(rank));
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
    hipLaunchKernelGGL((shrink_kernel<T, QUADS, RT>), dim3((unsigned)(max_tiles(M, adapters) * s.splits)), dim3(256), 0, st, plan, X,
                       reinterpret_cast<const T*>(A), part, M, K, rank, adapters, s.splits, s.per_split);
    return launched();
  }
  static int expand(const PlanAt& plan, const float* base, const float* part, int splits, const float* scale, const void* B, float* out, float* kept,
                    int M, int N, int rank, int adapters, hipStream_t st) {
    const int cols = columns(M, N, adapters), strips = (N + cols - 1) / cols;
    hipLaunchKernelGGL((expand_kernel<T, QUADS, RT>), dim3((unsigned)(max_tiles(M, adapters) * strips)), dim3(256), 0, st, plan, base, part, splits,
                       scale, reinterpret_cast<const T*>(B), out, kept, M, N, rank, adapters, cols, strips);
    return launched();
  }
  static int split_sum(const PlanAt& plan, const float* part, int splits, const float* scale, float* sum, int M, int rank, int adapters, hipStream_t st) {
    hipLaunchKernelGGL(split_sum_kernel<RT>, dim3((unsigned)max_tiles(M, adapters), 2 * RT), dim3(256), 0, st, plan, part, splits, scale, sum, M, rank, adapters);
    return launched();
  }
  static int outer(const PlanAt& plan, const Outer& a, const Outer& b, const float* scale, int M, int rank, int adapters, hipStream_t st) {
    const int chunks = (int)max_chunks(M, adapters), zeros = std::min(adapters, 4);
    hipLaunchKernelGGL((outer_kernel<QUADS, RT>), dim3((unsigned)((chunks + zeros) * (a.strips + b.strips))), dim3(256), 0, st, plan, a, b, scale, M,
                       rank, adapters, chunks, zeros);
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

struct Tensor {
  const void* p;
  size_t bytes;
};
// Whether something that is written lies over something that is read, or over the rest of it.
template <size_t IN, size_t OUT>
bool overlapping(const Tensor (&in)[IN], const Tensor (&out)[OUT]) {
  for (size_t i = 0; i < OUT; ++i) {
    for (const Tensor& q : in)
      if (overlap(out[i].p, out[i].bytes, q.p, q.bytes)) return true;
    for (size_t j = 0; j < i; ++j)
      if (overlap(out[i].p, out[i].bytes, out[j].p, out[j].bytes)) return true;
  }
  return false;
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
  const size_t needed = plan_layout(plan, M, adapters, &p);
  if (plan_bytes < needed) return XBAR_EWORKSPACE;
  if (overlap(plan, needed, rows, (size_t)M * sizeof(int32_t))) return XBAR_EINVAL;
  hipStream_t st = reinterpret_cast<hipStream_t>(hip_stream);
  if (M <= kSmallPlan) {
    hipLaunchKernelGGL(plan_small_kernel, dim3(1), dim3(kSmallPlan), 0, st, rows, M, adapters, p);
    return launched();
  }
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
  const size_t each = type == XBAR_BF16 ? 2 : 4, y = (size_t)M * N * 4;
  const Tensor in[] = {{plan, plan_layout(nullptr, M, adapters, nullptr)}, {X, (size_t)M * K * 4}, {A, (size_t)adapters * rank * K * each},
                       {B, (size_t)adapters * rank * N * each}, {scale, (size_t)adapters * 4}, {Y != base ? base : nullptr, y}};
  const Tensor out[] = {{Y, y}, {T, (size_t)M * rank * 4}, {ws, work_layout(nullptr, XBAR_OP_FWD, M, K, N, rank, adapters, nullptr)}};
  if (overlapping(in, out)) return XBAR_EINVAL;
  hipStream_t st = reinterpret_cast<hipStream_t>(hip_stream);
  const Split s(M, K, adapters);
  const int rc = with_kernels(type, K % 4 == 0, rank, [&](auto k) { return k.shrink(p, X, A, w.part, M, K, rank, adapters, s, st); });
  if (rc) return rc;
  return with_kernels(type, N % 4 == 0, rank, [&](auto k) {
    return k.expand(p, base, w.part, s.splits, scale, B, Y, T, M, N, rank, adapters, st);
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
  const Tensor in[] = {{plan, plan_layout(nullptr, M, adapters, nullptr)}, {dY, (size_t)M * N * 4}, {X, (size_t)M * K * 4}, {T, (size_t)M * rank * 4},
                       {A, na * each}, {B, nb * each}, {scale, (size_t)adapters * 4}, {dX && dX != base ? base : nullptr, (size_t)M * K * 4}};
  const Tensor out[] = {{dX, (size_t)M * K * 4}, {dA, na * 4}, {dB, nb * 4},
                        {ws, work_layout(nullptr, XBAR_OP_BWD, M, K, N, rank, adapters, nullptr)}};
  if (overlapping(in, out)) return XBAR_EINVAL;
  hipStream_t st = reinterpret_cast<hipStream_t>(hip_stream);
  const Split s(M, N, adapters);
  int rc = with_kernels(type, N % 4 == 0, rank, [&](auto k) { return k.shrink(p, dY, B, w.part, M, N, rank, adapters, s, st); });
  if (rc) return rc;
  rc = with_kernels(XBAR_F32, true, rank, [&](auto k) { return k.split_sum(p, w.part, s.splits, scale, w.dT, M, rank, adapters, st); });
  if (rc) return rc;
  if (dX) {
    rc = with_kernels(type, K % 4 == 0, rank,
                      [&](auto k) { return k.expand(p, base, w.dT, 1, (const float*)nullptr, A, dX, (float*)nullptr, M, K, rank, adapters, st); });
    if (rc) return rc;
  }
  const Outer oa{w.dT, X, dA, w.slotsA, K, (K + 63) / 64, 16 * rank_tiles(rank), 1}, ob{T, dY, dB, w.slotsB, N, (N + 63) / 64, rank, 0};
  rc = with_kernels(XBAR_F32, K % 4 == 0 && N % 4 == 0, rank, [&](auto k) { return k.outer(p, oa, ob, scale, M, rank, adapters, st); });
  if (rc) return rc;
  if (M <= chunk_rows(M)) return XBAR_OK;                       // no adapter has two chunks
  const bool quads = (size_t)rank * K % 4 == 0 && (size_t)rank * N % 4 == 0;
  const size_t most = (size_t)rank * std::max(K, N) / (quads ? 4 : 1);
  hipLaunchKernelGGL(quads ? outer_join_kernel<4> : outer_join_kernel<1>, dim3((unsigned)adapters, (unsigned)std::min<size_t>(256, (most + 255) / 256)),
                     dim3(256), 0, st, p, oa, ob, M, rank, adapters);
  return launched();
}

}  // extern "C"
