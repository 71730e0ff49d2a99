// Low-rank adapters of many requests beside a shared projection: y[r] = sum_s base[s][r] + scale_a B_a (A_a x[r]), a = row_adapter[r].
//
// Two launches: h[r] = scale_a A_a x[r] in fp32 (a reduction over k by the waves of a workgroup), then h B^T beside the base.  Rows go
// sixteen at a time.  One product serves all of them that have the same adapter, the first of these rows being its leader; every row takes
// its results from the product of its own adapter, so no row's numbers meet another's weights.  The second product keeps h whole:
// it is split into three bf16 parts of 8 bits each, which the matrix cores take side by side.
//
// The bank:
//   head  [n_slots] scale fp32, [n_slots] rank i32 (0: empty)
//   slot  A: [rank tiles of 16][k / 32][64 lanes][8]   operand of a 16 x 16 x 32 product: lane l rank l % 16, inputs 8 (l / 16) .. + 7
//         B: [n / 16][rank tiles][32 lanes][8]         lane l output l % 16, ranks 8 (l / 16) .. + 7 of 16; the other half of a 32-deep
//                                                      product takes the same numbers again, for another part of h
// Ranks, inputs and outputs past the matrices are zeros.
// h between the launches: [row][rank tiles][high, middle, low part, zeros][16]
//
// What bounds it: waiting for one load after another (a row's adapter, its rank, h, weights), twice.  One row of 4096, 7.8 us replayed, two
// launches of 4; 64 rows of 64 adapters of rank 16, 4096 to 12288 beside fp32, 17.3 us (8.3 and 9.8 for 31 MB in all, at the rate of a large read 4.5);
// 1100 rows in runs of one adapter of rank 64, 12288 to 4096 beside two partial sums, 36 us (20.1 and 16.5 for 83 MB, at that rate 12.2).
#include "sl_common.h"

namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x4_unaligned __attribute__((ext_vector_type(4), aligned(4)));
typedef __bf16 bf16x4_unaligned __attribute__((ext_vector_type(4), aligned(2)));

constexpr int kRows = 16;

struct Bank {
  unsigned char* p;
  int n_slots, rank_tiles, n, k;                          // rank_tiles: of the largest rank
  __host__ __device__ size_t head() const { return ((size_t)n_slots * 8 + 255) / 256 * 256; }
  __host__ __device__ size_t a_bytes() const { return (size_t)rank_tiles * ((k + 31) / 32) * 1024; }
  __host__ __device__ size_t slot_bytes() const { return a_bytes() + (size_t)((n + 15) / 16) * rank_tiles * 512; }
  __device__ float* scales() const { return (float*)p; }
  __device__ int32_t* ranks() const { return (int32_t*)p + n_slots; }
  __device__ bf16_t* a_of(int slot) const { return (bf16_t*)(p + head() + (size_t)slot * slot_bytes()); }
  __device__ bf16_t* b_of(int slot) const { return (bf16_t*)(p + head() + (size_t)slot * slot_bytes() + a_bytes()); }
};

__global__ __launch_bounds__(256) void adapters_init_kernel(int32_t* head, int words) {
  const int i = blockIdx.x * 256 + threadIdx.x;
  if (i < words) head[i] = 0;
}

__global__ __launch_bounds__(256) void adapters_pack_kernel(Bank bank, int slot, int rank, float scale, const bf16_t* a, const bf16_t* b) {
  const int64_t start = (int64_t)blockIdx.x * 256 + threadIdx.x, step = (int64_t)gridDim.x * 256;
  if (start == 0) {
    bank.scales()[slot] = scale;
    bank.ranks()[slot] = rank;
  }
  const int tiles = (rank + 15) / 16, blocks_k = (bank.k + 31) / 32, tiles_n = (bank.n + 15) / 16;
  bf16x8* to_a = (bf16x8*)bank.a_of(slot);
  for (int64_t i = start; i < (int64_t)tiles * blocks_k * 64; i += step) {
    const int lane = (int)(i & 63), r = (int)(i / 64 / blocks_k) * 16 + (lane & 15), c = (int)(i / 64 % blocks_k) * 32 + (lane >> 4) * 8;
    bf16x8 v = {};
    if (r < rank && c < bank.k) v = *(const bf16x8*)(a + (size_t)r * bank.k + c);       // k is a multiple of 8
    to_a[i] = v;
  }
  bf16x8* to_b = (bf16x8*)bank.b_of(slot);
  for (int64_t i = start; i < (int64_t)tiles_n * tiles * 32; i += step) {
    const int lane = (int)(i & 31), tile = (int)(i / 32 % tiles), row = (int)(i / 32 / tiles) * 16 + (lane & 15), c = tile * 16 + (lane >> 4) * 8;
    bf16x8 v = {};
    if (row < bank.n)
      for (int e = 0; e < 8; ++e)
        if (c + e < rank) v[e] = b[(size_t)row * rank + c + e];
    to_b[i] = v;
  }
}

// The lane's row's adapter, -1 where there is none, its rank tiles and scale.  (The id is asked for without waiting for the row count.)
struct Adapter {
  int id, tiles;
  float scale;
};
__device__ inline Adapter adapter_of_row(const Bank& bank, const int32_t* row_adapter, int r, int m_upper, const int32_t* m_dev, int& m) {
  int a = row_adapter[min(r, m_upper - 1)];
  m = min(*m_dev, m_upper);
  const bool there = r < m && a >= 0 && a < bank.n_slots;
  a = there ? a : 0;
  const int tiles = (bank.ranks()[a] + 15) / 16;
  const float scale = bank.scales()[a];
  return there && tiles > 0 ? Adapter{a, tiles, scale} : Adapter{-1, 0, 0.f};
}

// The three parts of v, of 8 bits each
__device__ inline void split3(float v, bf16_t& a, bf16_t& b, bf16_t& c) {
  a = (bf16_t)v;
  b = (bf16_t)(v - (float)a);
  c = (bf16_t)(v - (float)a - (float)b);
}

// h for 16 rows and RT rank tiles: workgroup (rows, place, tiles) takes the adapters of these rows, every gridDim.y-th of them, one after another.
//
// The rows pass through LDS, 512 inputs at a time: a wave loads 1 KiB of one row, and takes 32 inputs of all sixteen as an operand.  (An
// operand loaded from row-major memory is 64 bytes of each of sixteen rows that lie a power of two apart.)  Pieces of 16 bytes that would
// meet in one bank are kept apart by an exclusive or of their row with their place.  P chunks share a barrier, and the next P are on their way.
template <int RT, int P>
__global__ __launch_bounds__(1024) void adapters_down_kernel(Bank bank, const bf16_t* x, const int32_t* row_adapter, const int32_t* m_dev, int m_upper,
                                                             bf16_t* h) {
  constexpr int kWaves = 16, kChunk = 512, kChunkBytes = kRows * kChunk * 2;
  extern __shared__ __attribute__((aligned(16))) unsigned char lds[];      // rows [2][P][16][512], and after them part [kWaves][RT][row][rank]
  auto part = reinterpret_cast<float(*)[RT][16][16]>(lds);
  const int r0 = blockIdx.x * kRows, lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), q = lane >> 4;
  int m;
  const Adapter mine = adapter_of_row(bank, row_adapter, r0 + (lane & 15), m_upper, m_dev, m);
  if (r0 >= m) return;
  const int own = mine.id;
  const int tile = blockIdx.z * RT, blocks = (bank.k + 31) / 32, chunks = (bank.k + kChunk - 1) / kChunk;
  const bf16_t* xr = x + (size_t)min(r0 + wave, m - 1) * bank.k + lane * 8;
  unsigned char* put = lds + wave * 1024 + (lane ^ wave) * 16;
  const unsigned char* get = lds + (lane & 15) * 1024 + ((wave * 4 + q) ^ (lane & 15)) * 16;
  uint64_t todo = __ballot(own >= 0) & 0xffff;
  for (int place = 0; todo; ++place) {
    const int leader = __builtin_ctzll(todo), a = __builtin_amdgcn_readlane(own, leader), tiles = __builtin_amdgcn_readlane(mine.tiles, leader);
    const uint64_t its = __ballot(own == a);
    todo &= ~its;
    if (place % gridDim.y != blockIdx.y || tile >= tiles) continue;
    const bf16x8* w[RT];                                  // (a tile past the last is read as the last and not stored)
#pragma unroll
    for (int t = 0; t < RT; ++t) w[t] = (const bf16x8*)bank.a_of(a) + ((size_t)min(tile + t, tiles - 1) * blocks + wave) * 64 + lane;
    bf16x8 xs[P], ws[P][RT];
    auto ask = [&](int p, int c) __attribute__((always_inline)) {
      xs[p] = bf16x8{};                                   // (inputs past the last are zeros, and the last block is read for those behind it)
      if (c * kChunk + lane * 8 < bank.k) xs[p] = *(const bf16x8*)(xr + c * kChunk);
#pragma unroll
      for (int t = 0; t < RT; ++t) ws[p][t] = w[t][(ptrdiff_t)min(c * 16, blocks - 1 - wave) * 64];
    };
    f32x4 acc[RT] = {};
#pragma unroll
    for (int p = 0; p < P; ++p) ask(p, p);
    for (int c0 = 0, side = 0; c0 < chunks; c0 += P, side ^= P * kChunkBytes) {
      bf16x8 now[P][RT];
#pragma unroll
      for (int p = 0; p < P; ++p) {
        *(bf16x8*)(put + side + p * kChunkBytes) = xs[p];
#pragma unroll
        for (int t = 0; t < RT; ++t) now[p][t] = ws[p][t];
      }
      if (c0 + P < chunks)
#pragma unroll
        for (int p = 0; p < P; ++p) ask(p, c0 + P + p);
      __syncthreads();
#pragma unroll
      for (int p = 0; p < P; ++p) {
        const bf16x8 v = *(const bf16x8*)(get + side + p * kChunkBytes);
#pragma unroll
        for (int t = 0; t < RT; ++t) acc[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(now[p][t], v, acc[t], 0, 0, 0);
      }
    }
    __syncthreads();
#pragma unroll
    for (int t = 0; t < RT; ++t) *(f32x4*)&part[wave][t][lane & 15][q * 4] = acc[t];
    __syncthreads();
    const float scale = __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(mine.scale), leader));
    for (int i = threadIdx.x; i < RT * 256; i += 1024) {
      const int t = i / 256, at = i / 16 % 16, rank = i % 16;
      if (tile + t >= tiles || !(its >> at & 1)) continue;
      float sum = 0.f;
#pragma unroll
      for (int v = 0; v < kWaves; ++v) sum += part[v][t][at][rank];
      bf16_t* out = h + (((size_t)(r0 + at) * bank.rank_tiles + tile + t) * 4) * 16 + rank;
      split3(scale * sum, out[0], out[16], out[32]);
      out[48] = (bf16_t)0.f;
    }
    __syncthreads();
  }
}

// 16 rows, 16 CT columns a wave and four times as many a workgroup.  The products of one adapter and rank tile are a step; D steps are asked for at
// once, while the D before them are worked on.  Results pass through LDS, so that base and y are read and written along their rows (64 CT columns of one at a time; in the
// products' own layout they are 64 bytes of each of sixteen rows, a power of two apart).
template <typename T, int CT, int D>
__global__ __launch_bounds__(256) void adapters_up_kernel(Bank bank, const bf16_t* h, const int32_t* row_adapter, const int32_t* m_dev, int m_upper,
                                                          const float* base, int splits, T* y) {
  constexpr int kCols = 64 * CT, kUnits = kCols / 4;      // units: four columns of a row
  extern __shared__ __attribute__((aligned(16))) unsigned char lds[];      // h of the 16 rows, and after the products their results
  auto sh = reinterpret_cast<float(*)[kCols + 4]>(lds);
  const int r0 = blockIdx.y * kRows, lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), r = r0 + (lane & 15);
  int m;
  const Adapter mine = adapter_of_row(bank, row_adapter, r, m_upper, m_dev, m);
  if (r0 >= m) return;
  const int tiles_n = (bank.n + 15) / 16, first = (blockIdx.x * 4 + wave) * CT, col0 = blockIdx.x * kCols, own = mine.id, rr = min(r, m - 1);
  const bool wide = bank.n % 4 == 0;                      // four columns of a row at once
  // base: the first two planes are asked for here and added up behind the products
  auto plane = [&](int j, int s) __attribute__((always_inline)) {
    const int unit = j * 256 + threadIdx.x, row = r0 + unit / kUnits, col = col0 + unit % kUnits * 4;
    f32x4 v = {};
    if (!base || s >= splits || row >= m || col >= bank.n) return v;
    const float* from = base + ((size_t)s * m_upper + row) * bank.n + col;
    if (wide) return (f32x4)*(const f32x4_unaligned*)from;
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (col + e < bank.n) v[e] = from[e];
    return v;
  };
  f32x4 sum[CT], then[CT];
#pragma unroll
  for (int j = 0; j < CT; ++j) sum[j] = plane(j, 0);
#pragma unroll
  for (int j = 0; j < CT; ++j) then[j] = plane(j, 1);
  // (rows of h lie behind one another, in LDS 16 bytes further apart; those of rows without an adapter hold whatever they hold: nothing is taken of them)
  const int row_pieces = bank.rank_tiles * 8;
  for (int i = threadIdx.x; i < min(kRows, m - r0) * row_pieces; i += 256)
    *(uint4*)(lds + (i / row_pieces * (row_pieces + 1) + i % row_pieces) * 16) = *(const uint4*)(h + (size_t)r0 * row_pieces * 8 + i * 8);
  __syncthreads();
  const bf16x8* hr = (const bf16x8*)lds + (rr - r0) * (row_pieces + 1) + (lane >> 4);
  uint64_t todo = first < tiles_n ? __ballot(own >= 0) & 0xffff : 0;
  int a = -1, t = 0, tiles = 0;                           // the step that comes next
  f32x4 acc[CT] = {}, out[CT] = {};
  auto next = [&]() {
    if (++t < tiles) return;
    t = 0;
    if (todo) {
      const int row = __builtin_ctzll(todo);
      a = __builtin_amdgcn_readlane(own, row);
      tiles = __builtin_amdgcn_readlane(mine.tiles, row);
      todo &= ~__ballot(own == a);
    } else {
      a = -1;
      tiles = 0;
    }
  };
  next();
  struct Steps {
    bf16x8 w[D][CT];
    int a[D], t[D];
  };
  auto ask = [&](Steps& s) __attribute__((always_inline)) {
#pragma unroll
    for (int d = 0; d < D; ++d) {
      s.a[d] = a;
      s.t[d] = t;
      if (a < 0) continue;
#pragma unroll
      for (int c = 0; c < CT; ++c)
        s.w[d][c] = *((const bf16x8*)bank.b_of(a) + ((size_t)min(first + c, tiles_n - 1) * tiles + t) * 32 + (lane & 31));
      next();
    }
  };
  auto work = [&](const Steps& s) __attribute__((always_inline)) {
#pragma unroll
    for (int d = 0; d < D; ++d) {
      if (s.a[d] < 0) break;
      const bf16x8 hi = hr[s.t[d] * 8], lo = hr[s.t[d] * 8 + 4];
#pragma unroll
      for (int c = 0; c < CT; ++c) {
        const f32x4 zero = {};
        acc[c] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(s.w[d][c], lo, s.t[d] == 0 ? zero : acc[c], 0, 0, 0);
        acc[c] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(s.w[d][c], hi, acc[c], 0, 0, 0);
        if (own == s.a[d]) out[c] = acc[c];
      }
    }
  };
  Steps even, odd;
  ask(even);
  while (even.a[0] >= 0) {
    ask(odd);
    work(even);
    ask(even);
    work(odd);
  }
  __syncthreads();
#pragma unroll
  for (int c = 0; c < CT; ++c) *(f32x4*)&sh[lane & 15][(wave * CT + c) * 16 + (lane >> 4) * 4] = out[c];
  // An infinity among the weights meets parts of h that are zero, its own or those in the padding: what came out as NaN is summed again with h in one
  // part.  (Seldom, so all is asked for again; the sum of the results tells whether, without a test of each.)
  float all = 0.f;
#pragma unroll
  for (int c = 0; c < CT; ++c) all += (out[c][0] + out[c][1]) + (out[c][2] + out[c][3]);
  if (__any(all != all)) {
#pragma unroll 1
    for (int i = 0; i < 4 * CT; ++i) {
      float* result = &sh[lane & 15][wave * CT * 16 + i / 4 * 16 + (lane >> 4) * 4 + i % 4];
      if (*result == *result) continue;
      const bf16_t* parts = h + (size_t)rr * bank.rank_tiles * 64;
      const bf16_t* w = bank.b_of(own) + ((size_t)min(first + i / 4, tiles_n - 1) * mine.tiles * 32 + (lane >> 4) * 4 + i % 4) * 8;
      float v = 0.f;
      for (int k = 0; k < mine.tiles * 16; ++k) {
        const bf16_t* p = parts + k / 16 * 64 + k % 16;
        v += ((float)p[0] + (float)p[16] + (float)p[32]) * (float)w[k / 8 * 128 + k % 8];
      }
      *result = v;
    }
  }
  __syncthreads();
  for (int s = 2;; ++s) {
#pragma unroll
    for (int j = 0; j < CT; ++j) sum[j] += then[j];
    if (s >= splits) break;
#pragma unroll
    for (int j = 0; j < CT; ++j) then[j] = plane(j, s);
  }
#pragma unroll
  for (int j = 0; j < CT; ++j) {
    const int unit = j * 256 + threadIdx.x, row = r0 + unit / kUnits, col = col0 + unit % kUnits * 4;
    if (row >= m || col >= bank.n) continue;
    const f32x4 v = sum[j] + *(const f32x4*)&sh[unit / kUnits][unit % kUnits * 4];
    T* to = y + (size_t)row * bank.n + col;
    if (wide) {
      if constexpr (sizeof(T) == 2) {
        bf16x4_unaligned b;
#pragma unroll
        for (int e = 0; e < 4; ++e) b[e] = (bf16_t)v[e];
        *(bf16x4_unaligned*)to = b;
      } else {
        *(f32x4_unaligned*)to = v;
      }
    } else {
#pragma unroll
      for (int e = 0; e < 4; ++e)
        if (col + e < bank.n) st<T>::stv(to + e, v[e]);
    }
  }
}

Bank bank_of(const sl_adapters* ad) { return Bank{(unsigned char*)ad->bank, ad->n_slots, sl_cdiv(ad->max_rank, 16), ad->n, ad->k}; }

}  // namespace

size_t slk_adapters_bytes(const sl_adapters* ad) {
  const Bank b = bank_of(ad);
  return b.head() + (size_t)b.n_slots * b.slot_bytes();
}

int slk_adapters_init(hipStream_t s, const sl_adapters* ad) {
  hipLaunchKernelGGL(adapters_init_kernel, dim3(sl_cdiv(2 * ad->n_slots, 256)), dim3(256), 0, s, (int32_t*)ad->bank, 2 * ad->n_slots);
  SL_LAUNCH_CHECK();
  return SL_OK;
}

int slk_adapters_pack(hipStream_t s, const sl_adapters* ad, int slot, int rank, float scale, const void* a, const void* b) {
  const int64_t pieces = ((int64_t)ad->k / 32 + ad->n / 32 + 2) * sl_cdiv(max(rank, 1), 16) * 64;
  hipLaunchKernelGGL(adapters_pack_kernel, dim3((unsigned)min((int64_t)1024, pieces / 256 + 1)), dim3(256), 0, s, bank_of(ad), slot, rank, scale,
                     (const bf16_t*)a, (const bf16_t*)b);
  SL_LAUNCH_CHECK();
  return SL_OK;
}

size_t slk_adapters_workspace_bytes(const sl_adapters* ad, int m_upper) { return (size_t)m_upper * sl_cdiv(ad->max_rank, 16) * 128; }

int slk_adapters_forward(hipStream_t s, const sl_adapters* ad, const void* x, const int32_t* row_adapter, const int32_t* m_dev, int m_upper,
                         const float* base, int splits, float* y_f32, void* y_bf16, void* workspace) {
  const Bank bank = bank_of(ad);
  bf16_t* h = (bf16_t*)workspace;
  // Rank tiles a workgroup: as many as leave a workgroup for every second CU (each reads the rows again).  The whole call with 1 / 2 / 4 tiles, us: 1100
  // rows of rank 64 and 12288 inputs 45.4 / 37.2 / 40.8, 2048 rows of rank 64 and 4096 33.6 / 34.3 / 32.4, 512 rows of rank 64 17.5 / 17.6 / 18.4, 64 rows of
  // rank 64 23.3 / 24.8 / 27.6.  Adapters of sixteen rows side by side: all of them while that is no more than four workgroups a
  // CU, and two at least.  One / by this rule / sixteen: 16 rows of 16 adapters 52 / 13.1 / 13.2 us, 512 rows of 64 63 / 23.4 / 23.7, 2048 rows
  // of 64 93 / 65 / 71, 2048 rows in runs of 200 25.3 / 22.2 / 26.3.
  const int tiles = bank.rank_tiles, groups = sl_cdiv(m_upper, kRows);
#define DOWN_RUN(RT, P)                                                                                                            \
  do {                                                                                                                             \
    static unsigned long long done = 0;                                                                                            \
    constexpr int lds = (2 * P > RT ? 2 * P : RT) * 16384;                                                                              \
    SL_ALLOW_DYNAMIC_LDS(done, (adapters_down_kernel<RT, P>), lds);                                                                  \
    const int z = sl_cdiv(tiles, RT), side = max(2, min(16, 1024 / (groups * z)));                                                   \
    hipLaunchKernelGGL((adapters_down_kernel<RT, P>), dim3(groups, min(side, m_upper), z), dim3(1024), lds, s, bank, (const bf16_t*)x,  \
                       row_adapter, m_dev, m_upper, h);                                                                              \
  } while (0)
  if (tiles >= 4 && groups * sl_cdiv(tiles, 4) >= 128) DOWN_RUN(4, 2);
  else if (tiles >= 2 && groups * sl_cdiv(tiles, 2) >= 128) DOWN_RUN(2, 2);
  else DOWN_RUN(1, 2);
#undef DOWN_RUN
  SL_LAUNCH_CHECK();
  // Column tiles a wave: more of them share the reading of h and of the rows' adapters, once there are waves enough.  The whole call with 1 / 2 /
  // 4, us, adapters of rank 16 at random: 64 rows by 4096 (1024 waves of one tile) 13.9 / 14.6 / 17.6, 64 by 8192 (2048) 15.1 / 15.3 / 18.0, 64 by 12288 (3,000)
  // 17.1 / 17.2 / 19.2, 128 by 8192 (4096) 18.3 / 17.6 / 19.1, 128 by 12288 (6,000) 21.4 / 20.3 / 20.8, 256 by 8192 (8192) 24.8 / 23.9 / 21.8, 256 by 12288
  // (12,000) 29.6 / 27.9 / 24.4, 2048 by 4096 (33,000) 76.7 / 73.1 / 65.4; of rank 64, 64 by 12288 28.9 / 30.5 / 39.0, 128 by 12288 in runs 15.3 / 14.4 / 14.8.
#define UP_RUN(T, CT, D, Y)                                                                                                         \
  hipLaunchKernelGGL((adapters_up_kernel<T, CT, D>), dim3(sl_cdiv(sl_cdiv(ad->n, 16), 4 * CT), groups), dim3(256),    \
                     max(kRows * (tiles * 8 + 1) * 16, kRows * (64 * CT + 4) * 4), s, bank, h, row_adapter, m_dev, m_upper, base, splits, Y)
#define UP_BY_SIZE(T, Y)                                                     \
  do {                                                                       \
    const int64_t waves = (int64_t)sl_cdiv(ad->n, 16) * groups;              \
    if (waves < 2048) UP_RUN(T, 1, 4, Y);                                    \
    else if (waves < 8192) UP_RUN(T, 2, 4, Y);                               \
    else UP_RUN(T, 4, 1, Y);                                                 \
  } while (0)
  if (y_f32) UP_BY_SIZE(float, y_f32);
  else UP_BY_SIZE(bf16_t, (bf16_t*)y_bf16);
#undef UP_BY_SIZE
#undef UP_RUN
  SL_LAUNCH_CHECK();
  return SL_OK;
}
