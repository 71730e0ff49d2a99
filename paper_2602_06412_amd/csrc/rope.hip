// Rotary positions of rows of queries and keys, as a call of its own.
//
// A pair (a, b) turns by t = 2 pi pos f: (a cos t - b sin t, a sin t + b cos t).  Frequencies are kept in turns per slot, so the whole
// turns of pos f fall away exactly in fp64 (and what the product's rounding left, as much as 2^-26 of a turn at the largest positions, is
// added again), what is left is taken to within an eighth of a turn by exact steps of a quarter, and there the Taylor sums of sine and
// cosine, through the 11th and 12th power (the next terms are below 1e-11), are rounded to fp32 once.
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
  const double product = pos * f, turns = (product - rint(product)) + fma(pos, f, -product);
  const double quarter = rint(4.0 * turns);
  const double x = (turns - 0.25 * quarter) * 6.283185307179586476925, y = x * x;      // |x| <= pi / 4
  const double s = x * fma(y, fma(y, fma(y, fma(y, fma(y, -1.0 / 39916800, 1.0 / 362880), -1.0 / 5040), 1.0 / 120), -1.0 / 6), 1.0);
  const double c = fma(y, fma(y, fma(y, fma(y, fma(y, fma(y, 1.0 / 479001600, -1.0 / 3628800), 1.0 / 40320), -1.0 / 720), 1.0 / 24), -0.5), 1.0);
  const int q = (int)quarter & 3;
  const double cq = q & 1 ? s : c, sq = q & 1 ? c : s;
  return make_float2((float)((q == 1 || q == 2 ? -cq : cq) * amplitude), (float)((q >= 2 ? -sq : sq) * amplitude));
}

// A workgroup turns one row; a thread takes pairs, and single numbers behind them.
template <typename TI, typename TO, bool PAIRS>
__global__ __launch_bounds__(kThreads) void rope_rows_kernel(RopeArgs a) {
  __shared__ float2 turn[kMaxRot / 2];
  const int r = blockIdx.x;
  if (r >= min(*a.m_dev, a.m_upper)) return;
  const double pos = a.row_pos[r];
  const int half = a.rot / 2, rest = a.d - a.rot;
  for (int j = threadIdx.x; j < half; j += kThreads) turn[j] = turn_of(pos, a.freqs[j], a.amplitude);
  __syncthreads();
  for (int w = 0; w < 2; ++w) {
    const RopeSide& x = a.side[w];
    const TI* in = (const TI*)x.in + (size_t)r * x.in_stride;
    TO* out = (TO*)x.out + (size_t)r * x.out_stride;
    for (int i = threadIdx.x; i < x.heads * half; i += kThreads) {
      const int h = i / half, j = i - h * half, at = h * a.d + (PAIRS ? 2 * j : j), with = at + (PAIRS ? 1 : half);
      const float u = st<TI>::ld(in + at), v = st<TI>::ld(in + with);
      const float2 t = turn[j];
      st<TO>::stv(out + at, u * t.x - v * t.y);
      st<TO>::stv(out + with, u * t.y + v * t.x);
    }
    if ((const void*)in == (const void*)out) continue;
    for (int i = threadIdx.x; i < x.heads * rest; i += kThreads) {
      const int h = i / rest, at = h * a.d + a.rot + i - h * rest;
      st<TO>::stv(out + at, st<TI>::ld(in + at));
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
#define ROPE_RUN(TI, TO)                                                                                                      \
  do {                                                                                                                        \
    if (pairs) hipLaunchKernelGGL((rope_rows_kernel<TI, TO, true>), dim3(m_upper), dim3(kThreads), 0, s, a);                  \
    else hipLaunchKernelGGL((rope_rows_kernel<TI, TO, false>), dim3(m_upper), dim3(kThreads), 0, s, a);                       \
  } while (0)
  if (dtype_in == SL_BF16) {
    if (dtype_out == SL_BF16) ROPE_RUN(bf16_t, bf16_t); else ROPE_RUN(bf16_t, float);
  } else {
    if (dtype_out == SL_BF16) ROPE_RUN(float, bf16_t); else ROPE_RUN(float, float);
  }
#undef ROPE_RUN
  SL_LAUNCH_CHECK();
  return SL_OK;
}
