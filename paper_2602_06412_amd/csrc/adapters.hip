// Low-rank adapters of many requests beside a shared projection: y[r] = sum_s base[s][r] + scale_a B_a (A_a x[r]), a = row_adapter[r].
//
// Two launches: h[r] = A_a x[r] in fp32 (a reduction over k: workgroups along it, partial sums in the workspace), then scale h B^T beside
// the base.  A workgroup takes 16 rows.  One of its products serves all of them that have the same adapter, its leader being the
// first of these; every row's results come from the product of its own adapter, so no row's numbers meet another's weights.
// The second product keeps h whole: scale h is split into three bf16 parts of 8 bits each, which the matrix cores take side by side.
//
// The bank:
//   head  [n_slots] scale fp32, [n_slots] rank i32 (0: empty)
//   slot  A: [rank tiles of 16][k / 32][64 lanes][8]   operand of a 16 x 16 x 32 product: lane l rank l % 16, inputs 8 (l / 16) .. + 7
//         B: [n / 16][rank tiles][32 lanes][8]         lane l output l % 16, ranks 8 (l / 16) .. + 7 of 16; the other half of a 32-deep
//                                                      product takes the same numbers again, for another part of h
// Ranks, inputs and outputs past the matrices are zeros.
#include "sl_common.h"

namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));

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

// Of the 16 rows from r0 on (lane l: row r0 + l % 16): the lane's adapter, -1 where there is none
__device__ inline int adapter_of_row(const Bank& bank, const int32_t* row_adapter, int r, int m) {
  const int a = r < m ? row_adapter[r] : -1;
  return a >= 0 && a < bank.n_slots && bank.ranks()[a] > 0 ? a : -1;
}

// h[split][row][ranks] for the rows of one adapter among 16: workgroup (row, split, rank tile), if the row is the first of its adapter
__global__ __launch_bounds__(256) void adapters_down_kernel(Bank bank, const bf16_t* x, const int32_t* row_adapter, const int32_t* m_dev, int m_upper,
                                                            int splits, float* h) {
  const int m = min(*m_dev, m_upper), row = blockIdx.x;
  if (row >= m) return;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, r0 = row & ~(kRows - 1), r = r0 + (lane & 15);
  const int own = adapter_of_row(bank, row_adapter, r, m), a = __builtin_amdgcn_readlane(own, row - r0);
  if (a < 0 || __builtin_ctzll(__ballot(own == a)) != row - r0) return;
  const int tile = blockIdx.z;
  if (tile * 16 >= bank.ranks()[a]) return;
  const int blocks = (bank.k + 31) / 32, b0 = (int)((int64_t)blocks * blockIdx.y / splits), b1 = (int)((int64_t)blocks * (blockIdx.y + 1) / splits);
  const bf16x8* w = (const bf16x8*)bank.a_of(a) + (size_t)tile * blocks * 64;
  const bf16_t* xr = x + (size_t)min(r, m - 1) * bank.k;
  f32x4 acc = {};
  for (int b = b0 + wave; b < b1; b += 4) {
    const int c = b * 32 + (lane >> 4) * 8;
    bf16x8 v = {};
    if (c < bank.k) v = *(const bf16x8*)(xr + c);
    acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(w[(size_t)b * 64 + lane], v, acc, 0, 0, 0);
  }
  __shared__ f32x4 part[4][64];
  part[wave][lane] = acc;
  __syncthreads();
  if (wave == 0 && own == a) {
    const f32x4 sum = (part[0][lane] + part[1][lane]) + (part[2][lane] + part[3][lane]);
    *(f32x4*)(h + ((size_t)blockIdx.y * m_upper + r) * bank.rank_tiles * 16 + tile * 16 + (lane >> 4) * 4) = sum;
  }
}

__device__ inline void split3(float v, bf16_t& a, bf16_t& b, bf16_t& c) {
  a = (bf16_t)v;
  b = (bf16_t)(v - (float)a);
  c = (bf16_t)(v - (float)a - (float)b);
}

// 16 rows, 64 columns a workgroup
template <typename T>
__global__ __launch_bounds__(256) void adapters_up_kernel(Bank bank, const float* h, int h_splits, const int32_t* row_adapter, const int32_t* m_dev,
                                                          int m_upper, const float* base, int splits, T* y) {
  const int m = min(*m_dev, m_upper), r0 = blockIdx.y * kRows;
  if (r0 >= m) return;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, r = r0 + (lane & 15), tile_n = blockIdx.x * 4 + wave;
  if (tile_n * 16 >= bank.n) return;
  const int own = adapter_of_row(bank, row_adapter, r, m);
  f32x4 y4 = {};
  uint64_t todo = __ballot(own >= 0) & 0xffff;
  while (todo) {
    const int a = __builtin_amdgcn_readlane(own, __builtin_ctzll(todo));
    const uint64_t rows = __ballot(own == a);
    todo &= ~rows;
    const int rank = bank.ranks()[a], tiles = (rank + 15) / 16;
    const float scale = bank.scales()[a];
    const bf16x8* w = (const bf16x8*)bank.b_of(a) + (size_t)tile_n * tiles * 32 + (lane & 31);
    f32x4 acc = {};
    for (int t = 0; t < tiles; ++t) {
      bf16x8 first = {}, second = {};
      if (own == a) {
        float v[8] = {};
        for (int s = 0; s < h_splits; ++s) {
          const float* from = h + ((size_t)s * m_upper + r) * bank.rank_tiles * 16 + t * 16 + (lane >> 4 & 1) * 8;
          for (int e = 0; e < 8; ++e) v[e] += from[e];
        }
        for (int e = 0; e < 8; ++e) {
          bf16_t p0, p1, p2;
          split3(scale * v[e], p0, p1, p2);
          first[e] = lane < 32 ? p0 : p1;
          second[e] = lane < 32 ? p2 : (bf16_t)0.f;
        }
      }
      acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(w[(size_t)t * 32], second, acc, 0, 0, 0);
      acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(w[(size_t)t * 32], first, acc, 0, 0, 0);
    }
    if (own == a) y4 = acc;
  }
  if (r >= m) return;
  for (int e = 0; e < 4; ++e) {
    const int c = tile_n * 16 + (lane >> 4) * 4 + e;
    if (c >= bank.n) break;
    float sum = 0.f;
    for (int s = 0; base && s < splits; ++s) sum += base[((size_t)s * m_upper + r) * bank.n + c];
    st<T>::stv(y + (size_t)r * bank.n + c, sum + y4[e]);
  }
}

Bank bank_of(const sl_adapters* ad) { return Bank{(unsigned char*)ad->bank, ad->n_slots, sl_cdiv(ad->max_rank, 16), ad->n, ad->k}; }

// Workgroups along k
int down_splits(int k) { return min(8, sl_cdiv(k, 512)); }

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

size_t slk_adapters_workspace_bytes(const sl_adapters* ad, int m_upper) {
  return (size_t)down_splits(ad->k) * m_upper * sl_cdiv(ad->max_rank, 16) * 16 * 4;
}

int slk_adapters_forward(hipStream_t s, const sl_adapters* ad, const void* x, const int32_t* row_adapter, const int32_t* m_dev, int m_upper,
                         const float* base, int splits, float* y_f32, void* y_bf16, void* workspace) {
  const Bank bank = bank_of(ad);
  const int h_splits = down_splits(ad->k);
  hipLaunchKernelGGL(adapters_down_kernel, dim3(m_upper, h_splits, bank.rank_tiles), dim3(256), 0, s, bank, (const bf16_t*)x, row_adapter, m_dev,
                     m_upper, h_splits, (float*)workspace);
  SL_LAUNCH_CHECK();
  const dim3 grid(sl_cdiv(ad->n, 64), sl_cdiv(m_upper, kRows));
  if (y_f32)
    hipLaunchKernelGGL((adapters_up_kernel<float>), grid, dim3(256), 0, s, bank, (const float*)workspace, h_splits, row_adapter, m_dev, m_upper, base,
                       splits, y_f32);
  else
    hipLaunchKernelGGL((adapters_up_kernel<bf16_t>), grid, dim3(256), 0, s, bank, (const float*)workspace, h_splits, row_adapter, m_dev, m_upper, base,
                       splits, (bf16_t*)y_bf16);
  SL_LAUNCH_CHECK();
  return SL_OK;
}
