// Rotary positions of rows of queries and keys, as a call of its own.
//
// A pair (a, b) turns by t = 2 pi pos f: (a cos t - b sin t, a sin t + b cos t).  Frequencies are kept in turns per slot, so the whole
// turns of pos f fall away in one fused step: the product with all of its bits, of which fp64 alone would lose as much as 2^-25 of a turn at
// the largest positions, less a whole number, rounded once.  What is left is taken to within an eighth of a turn by exact steps of a quarter, and
// there the Taylor sums of sine and cosine, through the 11th and 12th power (the next terms are below 1e-11), are rounded to fp32 once.
//
// What bounds it is reading and writing the rows: 5533 rows of 32 + 32 heads of 128 bf16 take 36 us, which is the rate of a large copy (4.9 TB/s);
// 137 rows of fp32, half of each head turned, 8 us where the caller marshals each call, and 4 us replayed from a graph, of which 3 are a launch's own.
#include "sl_common.h"

namespace {

constexpr int kThreads = 256, kMaxRot = 1024;

struct RopeSide {
  const void* in;
  void* out;
  int64_t in_stride, out_stride;
  int heads;
};

struct RopeArgs {
  RopeSide side[2];                                       // queries, keys
  const double* freqs;
  const int32_t *row_pos, *m_dev;
  int m_upper, d, rot;
  float amplitude;
};

// amplitude (cos, sin) of 2 pi pos f
__device__ inline float2 turn_of(double pos, double f, float amplitude) {
  const double turns = fma(pos, f, -rint(pos * f));
  const double quarter = rint(4.0 * turns);
  const double x = (turns - 0.25 * quarter) * 6.283185307179586476925, y = x * x;      // |x| <= pi / 4
  const double s = x * fma(y, fma(y, fma(y, fma(y, fma(y, -1.0 / 39916800, 1.0 / 362880), -1.0 / 5040), 1.0 / 120), -1.0 / 6), 1.0);
  const double c = fma(y, fma(y, fma(y, fma(y, fma(y, fma(y, 1.0 / 479001600, -1.0 / 3628800), 1.0 / 40320), -1.0 / 720), 1.0 / 24), -0.5), 1.0);
  const int q = (int)quarter & 3;
  const double cq = q & 1 ? s : c, sq = q & 1 ? c : s;
  return make_float2((float)((q == 1 || q == 2 ? -cq : cq) * amplitude), (float)((q >= 2 ? -sq : sq) * amplitude));
}

// V numbers that lie together, as fp32
template <int V, typename T>
__device__ inline void load_v(const T* p, float (&v)[V]) {
  if constexpr (V == 1) {
    v[0] = st<T>::ld(p);
  } else if constexpr (V == 8) {
    ld8(p, v);
  } else if constexpr (sizeof(T) == 2) {
    const bf16x4_t u = *reinterpret_cast<const bf16x4_t*>(p);
#pragma unroll
    for (int e = 0; e < 4; ++e) v[e] = (float)u[e];
  } else {
    ld4f(p, v);
  }
}
template <int V, typename T>
__device__ inline void store_v(T* p, const float (&v)[V]) {
  if constexpr (V == 1) st<T>::stv(p, v[0]);
  else if constexpr (V == 8) st8(p, v);
  else if constexpr (sizeof(T) == 2) st4(p, v);
  else *reinterpret_cast<float4*>(p) = make_float4(v[0], v[1], v[2], v[3]);
}

// A workgroup turns one row; a thread takes V pairs at a time, and V single numbers behind them.  The turns of a row are formed once, for all of its
// heads.
template <typename TI, typename TO, bool PAIRS, int V>
__global__ __launch_bounds__(kThreads) void rope_rows_kernel(RopeArgs a) {
  __shared__ __attribute__((aligned(16))) float cosine[kMaxRot / 2], sine[kMaxRot / 2];
  const int r = blockIdx.x;
  if (r >= min(*a.m_dev, a.m_upper)) return;
  const double pos = a.row_pos[r];
  const int half = a.rot / 2, rest = a.d - a.rot;
  for (int j = threadIdx.x; j < half; j += kThreads) {
    const float2 t = turn_of(pos, a.freqs[j], a.amplitude);
    cosine[j] = t.x;
    sine[j] = t.y;
  }
  __syncthreads();
  const int n = half / V, n_rest = rest / V;
  for (int w = 0; w < 2; ++w) {
    const RopeSide& x = a.side[w];
    const TI* in = (const TI*)x.in + (size_t)r * x.in_stride;
    TO* out = (TO*)x.out + (size_t)r * x.out_stride;
    for (int i = threadIdx.x; i < x.heads * n; i += kThreads) {
      const int h = i / n, j = (i - h * n) * V, at = h * a.d + (PAIRS ? 2 * j : j), with = at + (PAIRS ? V : half);
      float u[V], v[V], p[V], q[V];
      load_v<V>(in + at, u);
      load_v<V>(in + with, v);
#pragma unroll
      for (int e = 0; e < V; ++e) {
        // of neighbours in pairs the first V numbers are half of the pairs, the second V the other half
        constexpr int kHalf = V / 2;
        const float c = cosine[j + e], s = sine[j + e];
        const float f = !PAIRS || V == 1 ? u[e] : e < kHalf ? u[2 * e % V] : v[2 * e % V], g = !PAIRS || V == 1 ? v[e] : e < kHalf ? u[(2 * e + 1) % V] : v[(2 * e + 1) % V];
        p[e] = f * c - g * s;
        q[e] = f * s + g * c;
      }
      if constexpr (PAIRS && V > 1) {
#pragma unroll
        for (int e = 0; e < V / 2; ++e) {
          u[2 * e] = p[e];
          u[2 * e + 1] = q[e];
          v[2 * e] = p[V / 2 + e];
          v[2 * e + 1] = q[V / 2 + e];
        }
        store_v<V>(out + at, u);
        store_v<V>(out + with, v);
      } else {
        store_v<V>(out + at, p);
        store_v<V>(out + with, q);
      }
    }
    if ((const void*)in == (const void*)out) continue;
    for (int i = threadIdx.x; i < x.heads * n_rest; i += kThreads) {
      const int h = i / n_rest, at = h * a.d + a.rot + (i - h * n_rest) * V;
      float u[V];
      load_v<V>(in + at, u);
      store_v<V>(out + at, u);
    }
  }
}

__global__ __launch_bounds__(kThreads) void rope_freqs_kernel(double* freqs, int rot, double theta, int scaling, double factor, double original_len,
                                                              double low_turns, double high_turns) {
  const int j = blockIdx.x * kThreads + threadIdx.x;
  if (j >= rot / 2) return;
  if (scaling == SL_ROPE_BASE) theta *= pow(factor, (double)rot / (rot - 2));
  double f = pow(theta, -2.0 * j / rot) / 6.283185307179586476925;
  if (scaling == SL_ROPE_LINEAR) f /= factor;
  if (scaling == SL_ROPE_TURNS) {
    const double g = fmin(fmax((original_len * f - low_turns) / (high_turns - low_turns), 0.0), 1.0);
    f = g * f + (1.0 - g) * (f / factor);
  }
  freqs[j] = f;
}

}  // namespace

int slk_rope_freqs(hipStream_t s, double* freqs, int rot, double theta, int scaling, double factor, double original_len, double low_turns,
                   double high_turns) {
  hipLaunchKernelGGL(rope_freqs_kernel, dim3(sl_cdiv(rot / 2, kThreads)), dim3(kThreads), 0, s, freqs, rot, theta, scaling, factor, original_len,
                     low_turns, high_turns);
  SL_LAUNCH_CHECK();
  return SL_OK;
}

int slk_rope_rows(hipStream_t s, const void* q, int64_t q_stride, void* q_out, int64_t q_out_stride, int n_heads, const void* k, int64_t k_stride,
                  void* k_out, int64_t k_out_stride, int n_kv_heads, int dtype_in, int dtype_out, int d, int rot, int pairs, const double* freqs,
                  float amplitude, const int32_t* row_pos, const int32_t* m_dev, int m_upper) {
  const RopeArgs a{{{q, q_out, q_stride, q_out_stride, n_heads}, {k, k_out, k_stride, k_out_stride, k ? n_kv_heads : 0}},
                   freqs, row_pos, m_dev, m_upper, d, rot, amplitude};
  // numbers at a time: eight of bf16 where pairs lie apart, else four, if every piece of them is aligned.  40 heads of 128 bf16, replayed, 8 / 4 / 1 at a
  // time, us: apart 64 rows 3.2 / 3.4 / 4.4, 512 rows 4.0 / 4.2 / 5.4, 2048 rows 7.9 / 8.3 / 11.1, 8192 rows 26.0 / 26.0 / 30.7; interleaved
  // 512 rows 4.3 / 4.1 / 5.3, 2048 rows 9.1 / 7.7 / 10.3, 8192 rows 26.8 / 25.9 / 29.8.
  const int most = dtype_in == SL_BF16 && dtype_out == SL_BF16 && !pairs ? 8 : 4;
  auto fits = [&](int v) {
    auto side = [&](const RopeSide& x) {
      return ((uintptr_t)x.in % (v * sl_tsize(dtype_in)) | (uintptr_t)x.out % (v * sl_tsize(dtype_out))) == 0 && x.in_stride % v == 0 && x.out_stride % v == 0;
    };
    return rot / 2 % v == 0 && (d - rot) % v == 0 && d % v == 0 && side(a.side[0]) && (!k || side(a.side[1]));
  };
  const int v = fits(most) ? most : fits(4) ? 4 : 1;
#define ROPE_LAUNCH(TI, TO, PAIRS, V) hipLaunchKernelGGL((rope_rows_kernel<TI, TO, PAIRS, V>), dim3(m_upper), dim3(kThreads), 0, s, a)
#define ROPE_BY_LAYOUT(TI, TO, V)                                                             \
  do {                                                                                        \
    if (pairs) ROPE_LAUNCH(TI, TO, true, V); else ROPE_LAUNCH(TI, TO, false, V);                \
  } while (0)
#define ROPE_RUN(TI, TO)                                                                      \
  do {                                                                                        \
    if (v == 1) ROPE_BY_LAYOUT(TI, TO, 1); else ROPE_BY_LAYOUT(TI, TO, 4);                      \
  } while (0)
  if (dtype_in == SL_BF16) {
    if (dtype_out == SL_BF16) {
      if (v == 8) ROPE_LAUNCH(bf16_t, bf16_t, false, 8); else ROPE_RUN(bf16_t, bf16_t);
    } else {
      ROPE_RUN(bf16_t, float);
    }
  } else {
    if (dtype_out == SL_BF16) ROPE_RUN(float, bf16_t); else ROPE_RUN(float, float);
  }
#undef ROPE_BY_LAYOUT
#undef ROPE_LAUNCH
#undef ROPE_RUN
  SL_LAUNCH_CHECK();
  return SL_OK;
}
