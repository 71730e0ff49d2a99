// A token for each row from its filtered posterior, with a given uniform number.
//
// Every filter keeps a beginning of the row's order (z descending, id ascending), so what is kept is a threshold: the key of the last
// kept z and, among the tokens of that very z, the last kept id.  Weights are whole numbers, W = rint(2^44 exp((z - max) / T)): at most
// 2^18 of them add up to less than 2^63, in any order and from any thread, to the same sum.
#include "sl_common.h"

namespace {

constexpr int kThreads = 1024, kWaves = kThreads / 64;
constexpr double kUnit = 17592186044416.0;                // 2^44

struct SampleArgs {
  const void* logits;
  int64_t row_stride;
  int n_rows, vocab, m_upper;
  const int32_t *row_map, *m_dev, *top_k;
  const float *temperature, *top_p, *min_p, *uniform;
  int32_t* token;
  float* prob;
  int32_t* kept;
};

// fp32 as a number whose order is that of z (both zeros alike)
__device__ inline uint32_t key_of(float z) {
  const uint32_t u = __float_as_uint(z + 0.f);
  return u ^ (u >> 31 ? 0xffffffffu : 0x80000000u);
}
__device__ inline float of_key(uint32_t k) { return __uint_as_float(k ^ (k >> 31 ? 0x80000000u : 0xffffffffu)); }
// a token that may be drawn: neither NaN nor -infinity
__device__ inline bool allowed(float z) { return z > -__builtin_inff(); }

__device__ inline uint64_t weight_of(float z, float most, double heat) {
  if (z == most) return (uint64_t)kUnit;                  // (an infinity, too)
  return most < __builtin_inff() ? (uint64_t)rint(exp(((double)z - (double)most) / heat) * kUnit) : 0;
}

struct Shared {
  uint64_t bins[256];
  uint64_t sums[kWaves];
  uint64_t found;
  uint32_t word;
  int index;
};

// sum over the block of the threads before this one; `whole` gets the sum of all
__device__ inline uint64_t before_me(uint64_t v, Shared& sh, uint64_t& whole) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  uint64_t sum = v;
  for (int o = 1; o < 64; o <<= 1) {
    const uint64_t below = __shfl_up((unsigned long long)sum, o, 64);
    if (lane >= o) sum += below;
  }
  __syncthreads();
  if (lane == 63) sh.sums[wave] = sum;
  __syncthreads();
  uint64_t at = 0;
  whole = 0;
  for (int w = 0; w < kWaves; ++w) {
    if (w < wave) at += sh.sums[w];
    whole += sh.sums[w];
  }
  return at + sum - v;
}

template <typename T>
__global__ __launch_bounds__(kThreads) void sample_filtered_kernel(SampleArgs a) {
  __shared__ Shared sh;
  const int r = blockIdx.x, tid = threadIdx.x, v_all = a.vocab;
  if (r >= min(*a.m_dev, a.m_upper)) return;
  const int row = a.row_map ? a.row_map[r] : r;
  const bool there = row >= 0 && row < a.n_rows;
  const T* z = (const T*)a.logits + (size_t)(there ? row : 0) * a.row_stride;
  const int share = (v_all + kThreads - 1) / kThreads, lo = min(tid * share, v_all), hi = there ? min(lo + share, v_all) : lo;

  // the first of the order, and how many may be drawn
  uint64_t best = 0;                                      // key, then lowest id
  int count = 0;
  for (int i = lo; i < hi; ++i) {
    const float x = st<T>::ld(z + i);
    if (!allowed(x)) continue;
    ++count;
    best = max(best, (uint64_t)key_of(x) << 32 | (uint32_t)~i);
  }
  for (int o = 32; o; o >>= 1) best = max(best, (uint64_t)__shfl_xor((unsigned long long)best, o, 64));
  if ((tid & 63) == 0) sh.sums[tid >> 6] = best;
  __syncthreads();
  for (int w = 0; w < kWaves; ++w) best = max(best, sh.sums[w]);
  uint64_t whole;
  if (tid == 0) sh.index = v_all;
  before_me((uint64_t)count, sh, whole);
  const int n = (int)whole;
  const float heat = a.temperature ? a.temperature[r] : 1.f, p = a.top_p ? a.top_p[r] : 1.f, least = a.min_p ? a.min_p[r] : 0.f;
  const int k = a.top_k ? a.top_k[r] : 0;
  if (n == 0 || !(heat > 0.f) || k == 1 || p <= 0.f || least > 1.f) {      // one token at most
    if (tid == 0) {
      a.token[r] = n ? (int32_t)~(uint32_t)best : 0;
      if (a.prob) a.prob[r] = n ? 1.f : 0.f;
      if (a.kept) a.kept[r] = n ? 1 : 0;
    }
    return;
  }
  const float most = of_key((uint32_t)(best >> 32));
  uint32_t last_key = 0;                                  // kept: allowed, and key above last_key, or the same and id <= last_id
  int last_id = v_all;
  auto is_kept = [&](float x, int i) {
    const uint32_t key = key_of(x);
    return allowed(x) && (key > last_key || (key == last_key && i <= last_id));
  };
  // Narrow what is kept to the fewest whose count (or weight) reaches the goal: the key byte by byte, then the id.
  auto narrow = [&](bool by_weight, double goal) {
    uint32_t prefix = 0;
    uint64_t above = 0;
    for (int shift = 24; shift >= 0; shift -= 8) {
      for (int i = tid; i < 256; i += kThreads) sh.bins[i] = 0;
      __syncthreads();
      for (int i = lo; i < hi; ++i) {
        const float x = st<T>::ld(z + i);
        const uint32_t key = key_of(x);
        if (!is_kept(x, i) || (shift < 24 && key >> (shift + 8) != prefix)) continue;
        atomicAdd((unsigned long long*)&sh.bins[key >> shift & 255], (unsigned long long)(by_weight ? weight_of(x, most, heat) : 1));
      }
      __syncthreads();
      if (tid == 0) {
        int b = 255;
        uint64_t sum = above;
        while (b > 0 && (double)(sum + sh.bins[b]) < goal) sum += sh.bins[b--];
        sh.found = sum;
        sh.word = prefix << 8 | (uint32_t)b;
      }
      __syncthreads();
      above = sh.found;
      prefix = sh.word;
    }
    // of the tokens with that key, as many as it takes
    const uint64_t each = by_weight ? weight_of(of_key(prefix), most, heat) : 1;
    int ties = 0;
    for (int i = lo; i < hi; ++i) {
      const float x = st<T>::ld(z + i);
      ties += is_kept(x, i) && key_of(x) == prefix;
    }
    uint64_t all_ties;
    const uint64_t ties_before = before_me((uint64_t)ties, sh, all_ties);
    uint64_t need = 1;
    if (each > 0 && goal > (double)above) need = (uint64_t)max(1.0, floor((goal - (double)above) / (double)each));
    while (need > 1 && (double)(above + (need - 1) * each) >= goal) --need;
    while (need < all_ties && (double)(above + need * each) < goal) ++need;
    if (need > all_ties) need = all_ties;
    if (ties_before < need && need <= ties_before + ties) {
      uint64_t seen = ties_before;
      for (int i = lo; i < hi; ++i) {
        const float x = st<T>::ld(z + i);
        if (is_kept(x, i) && key_of(x) == prefix && ++seen == need) {
          sh.index = i;
          break;
        }
      }
    }
    __syncthreads();
    last_id = sh.index;
    last_key = prefix;
    __syncthreads();
  };
  if (k > 0 && k < n) narrow(false, (double)k);
  if (p < 1.f) {
    uint64_t mine = 0;
    for (int i = lo; i < hi; ++i) {
      const float x = st<T>::ld(z + i);
      if (is_kept(x, i)) mine += weight_of(x, most, heat);
    }
    before_me(mine, sh, whole);
    narrow(true, (double)p * (double)whole);
  }
  const double enough = least > 0.f ? (double)least * kUnit : 0.0;
  uint64_t mine = 0, number = 0;
  for (int i = lo; i < hi; ++i) {
    const float x = st<T>::ld(z + i);
    if (!is_kept(x, i)) continue;
    const uint64_t w = weight_of(x, most, heat);
    if (least > 0.f && (double)w < enough) continue;
    mine += w;
    ++number;
  }
  uint64_t numbers;
  before_me(number, sh, numbers);
  const uint64_t at = before_me(mine, sh, whole);
  const float u = a.uniform[r];
  const double goal = (double)(u > 0.f ? fminf(u, 0x1.fffffep-1f) : 0.f) * (double)whole;
  if ((double)at <= goal && (double)(at + mine) > goal) {
    uint64_t sum = at;
    for (int i = lo; i < hi; ++i) {
      const float x = st<T>::ld(z + i);
      if (!is_kept(x, i)) continue;
      const uint64_t w = weight_of(x, most, heat);
      if (least > 0.f && (double)w < enough) continue;
      sum += w;
      if ((double)sum > goal) {
        a.token[r] = i;
        if (a.prob) a.prob[r] = (float)((double)w / (double)whole);
        if (a.kept) a.kept[r] = (int32_t)numbers;
        break;
      }
    }
  }
}

}  // namespace

size_t slk_sample_filtered_bytes(int m_upper, int vocab) { return 256; }

int slk_sample_filtered(hipStream_t s, const void* logits, int dtype, int64_t row_stride, int n_rows, int vocab, const int32_t* row_map,
                        const int32_t* m_dev, int m_upper, const float* temperature, const int32_t* top_k, const float* top_p, const float* min_p,
                        const float* uniform, int32_t* token, float* prob, int32_t* kept, void* workspace) {
  const SampleArgs a{logits, row_stride, n_rows, vocab, m_upper, row_map, m_dev, top_k, temperature, top_p, min_p, uniform, token, prob, kept};
  if (dtype == SL_BF16) hipLaunchKernelGGL((sample_filtered_kernel<bf16_t>), dim3(m_upper), dim3(kThreads), 0, s, a);
  else hipLaunchKernelGGL((sample_filtered_kernel<float>), dim3(m_upper), dim3(kThreads), 0, s, a);
  SL_LAUNCH_CHECK();
  return SL_OK;
}
