// Writing rows of K and V into the paged 8-bit cache, and reading them back.
#include "kv8.h"

namespace {

// max |x| of a wave's vector, NaN if one of its numbers is NaN (fmaxf would drop it)
__device__ inline float amax_or_nan(float most, bool nan) {
  most = wave_max(most);
  return __any(nan) ? __builtin_nanf("") : most;
}

// One vector of D numbers: NP consecutive ones in each of its lanes.
template <int D>
struct Vec {
  static constexpr int NP = D > 64 ? D / 64 : 1;
  static __device__ bool mine(int lane) { return lane * NP < D; }
};

template <typename T, int D>
__device__ inline void quantise(const T* x, int lane, float (&code)[Vec<D>::NP], float& scale) {
  constexpr int NP = Vec<D>::NP;
  float v[NP], most = 0.f;
  bool nan = false;
#pragma unroll
  for (int e = 0; e < NP; ++e) {
    v[e] = Vec<D>::mine(lane) ? st<T>::ld(x + lane * NP + e) : 0.f;
    nan |= v[e] != v[e];
    most = fmaxf(most, fabsf(v[e]));
  }
  most = amax_or_nan(most, nan);
  scale = most < __builtin_inff() ? most / 127.f : __builtin_nanf("");
#pragma unroll
  for (int e = 0; e < NP; ++e) code[e] = scale > 0.f ? fminf(fmaxf(rintf(v[e] / scale), -127.f), 127.f) : 0.f;
}

// One wave per row and head.
template <typename T, int D>
__global__ __launch_bounds__(256) void kv8_write_kernel(Kv8View kv, const T* k, const T* v, int64_t k_stride, int64_t v_stride,
                                                        const int32_t* row_pos, const int32_t* cu_rows, int m_upper) {
  using Tile = Kv8Tile<D>;
  constexpr int NP = Vec<D>::NP;
  const int lane = threadIdx.x & 63, head = blockIdx.y * 4 + (threadIdx.x >> 6), r = blockIdx.x;
  if (head >= kv.heads) return;
  const int b = kv8_sequence_of(cu_rows, kv.batch, r);
  const int pos = row_pos[r];
  if (b >= kv.batch || pos < 0 || pos >= kv.slots()) return;
  if (r + 1 < m_upper && r + 1 < cu_rows[b + 1] && row_pos[r + 1] == pos) return;      // the last of rows that name one slot is kept
  const int page = kv.table[(size_t)b * kv.max_pages + (pos >> kv.page_shift)];
  if (page < 0 || page >= kv.n_pages) return;
  unsigned char* tile = kv.tile<D>(page, head, pos);
  const int slot = pos & 15;
  float kc[NP], vc[NP], ks, vs;
  quantise<T, D>(k + (size_t)r * k_stride + head * D, lane, kc, ks);
  quantise<T, D>(v + (size_t)r * v_stride + head * D, lane, vc, vs);
  if (Vec<D>::mine(lane)) {
#pragma unroll
    for (int e = 0; e < NP; ++e) {
      tile[Tile::k_at(slot, lane * NP + e)] = (unsigned char)(signed char)(int)kc[e];
      tile[Tile::v_at(slot, lane * NP + e)] = (unsigned char)((int)vc[e] + 128);
    }
  }
  if (lane == 0) {
    reinterpret_cast<float*>(tile + Tile::kKs)[slot] = ks;
    reinterpret_cast<float*>(tile + Tile::kVs)[slot] = vs;
  }
}

template <typename T, int D>
__global__ __launch_bounds__(256) void kv8_read_kernel(Kv8View kv, T* k, T* v, int64_t k_stride, int64_t v_stride,
                                                       const int32_t* row_pos, const int32_t* cu_rows, int m_upper) {
  using Tile = Kv8Tile<D>;
  constexpr int NP = Vec<D>::NP;
  const int lane = threadIdx.x & 63, head = blockIdx.y * 4 + (threadIdx.x >> 6), r = blockIdx.x;
  if (head >= kv.heads) return;
  const int b = kv8_sequence_of(cu_rows, kv.batch, r);
  if (b >= kv.batch) return;
  const int pos = row_pos[r];
  const bool in = pos >= 0 && pos < kv.slots();
  const int page = in ? kv.table[(size_t)b * kv.max_pages + (pos >> kv.page_shift)] : -1;
  const bool ok = page >= 0 && page < kv.n_pages;
  const unsigned char* tile = ok ? kv.tile<D>(page, head, pos) : kv.pool;
  const int slot = pos & 15;
  const float ks = ok ? reinterpret_cast<const float*>(tile + Tile::kKs)[slot] : 0.f;
  const float vs = ok ? reinterpret_cast<const float*>(tile + Tile::kVs)[slot] : 0.f;
  if (!Vec<D>::mine(lane)) return;
#pragma unroll
  for (int e = 0; e < NP; ++e) {
    const int dim = lane * NP + e;
    const float kq = ok ? (float)(signed char)tile[Tile::k_at(slot, dim)] : 0.f;
    const float vq = ok ? (float)((int)tile[Tile::v_at(slot, dim)] - 128) : 0.f;
    st<T>::stv(k + (size_t)r * k_stride + head * D + dim, kq * ks);
    st<T>::stv(v + (size_t)r * v_stride + head * D + dim, vq * vs);
  }
}

}  // namespace

#define KV8_BY_HEAD(T, CALL)                 \
  switch (d) {                               \
    case 32: CALL(T, 32); break;             \
    case 64: CALL(T, 64); break;             \
    case 128: CALL(T, 128); break;           \
    case 256: CALL(T, 256); break;           \
    default: return SL_EINVAL;               \
  }

int slk_kv8_write(hipStream_t s, const Kv8View& kv, int d, int dtype, const void* k, const void* v, int64_t k_stride, int64_t v_stride,
                  const int32_t* row_pos, const int32_t* cu_rows, int m_upper) {
  const dim3 grid(m_upper, sl_cdiv(kv.heads, 4));
#define KV8_CALL(T, D) \
  hipLaunchKernelGGL((kv8_write_kernel<T, D>), grid, dim3(256), 0, s, kv, (const T*)k, (const T*)v, k_stride, v_stride, row_pos, cu_rows, m_upper)
  if (dtype == SL_BF16) { KV8_BY_HEAD(bf16_t, KV8_CALL) } else { KV8_BY_HEAD(float, KV8_CALL) }
#undef KV8_CALL
  SL_LAUNCH_CHECK();
  return SL_OK;
}

int slk_kv8_read(hipStream_t s, const Kv8View& kv, int d, int dtype, void* k, void* v, int64_t k_stride, int64_t v_stride,
                 const int32_t* row_pos, const int32_t* cu_rows, int m_upper) {
  const dim3 grid(m_upper, sl_cdiv(kv.heads, 4));
#define KV8_CALL(T, D) \
  hipLaunchKernelGGL((kv8_read_kernel<T, D>), grid, dim3(256), 0, s, kv, (T*)k, (T*)v, k_stride, v_stride, row_pos, cu_rows, m_upper)
  if (dtype == SL_BF16) { KV8_BY_HEAD(bf16_t, KV8_CALL) } else { KV8_BY_HEAD(float, KV8_CALL) }
#undef KV8_CALL
  SL_LAUNCH_CHECK();
  return SL_OK;
}
