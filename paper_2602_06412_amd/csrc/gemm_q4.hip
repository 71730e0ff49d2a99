// Products of a few bf16 rows with 4-bit weights: y = x W^T, W[j, i] = s[j, i / g] (q[j, i] - z[j, i / g]).
//
// A code q in 0..15 as a byte is the e4m3 number q 2^-9 (a subnormal, or a normal with the smallest exponent), so the conversion
// from e4m3 to bf16 with a scale of 2^9 yields two exact bf16 integers an instruction; the zero point and the scale of a
// group are applied to sums:
//   sum_i x_i s (q_i - z) = s ( sum_i x_i q_i  -  z sum_i x_i ),
// both sums from the matrix cores in fp32 (the second against a block of ones).
//
// Weights as the kernel reads them, one block per 16 columns and 128 indexes of the reduction:
//   codes  [64 lanes][4 products][8 codes]: lane l holds column l % 16, indexes 32 j + 8 (l / 16) .. + 7 of product j; in its
//          32-bit word code i < 4 is the low half of byte i, code 4 + i the high half
//   params [128 / g groups][16 columns]: scale (bf16) in the upper, zero point (bf16) in the lower half of a word
// Columns and indexes past the matrix have code, scale and zero point 0.
#include "sl_common.h"

namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
typedef float f32x4 __attribute__((ext_vector_type(4)));

constexpr int kCols = 16, kDepth = 128, kCodeBytes = 1024;
__host__ __device__ constexpr int q4_block_bytes(int group) { return kCodeBytes + kDepth / group * kCols * 4; }

__global__ __launch_bounds__(256) void q4_pack_kernel(const unsigned char* codes, const bf16_t* scales, const unsigned char* zeros, int n,
                                                      int k, int group, unsigned char* packed, int blocks_k, size_t blocks) {
  const size_t blk = (size_t)blockIdx.x * 4 + (threadIdx.x >> 6);
  if (blk >= blocks) return;
  const int lane = threadIdx.x & 63, kb = (int)(blk % blocks_k), col = (int)(blk / blocks_k) * kCols + (lane & 15);
  unsigned char* dst = packed + blk * q4_block_bytes(group);
  uint32_t w[4];
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const int i0 = kb * kDepth + j * 32 + (lane >> 4) * 8;
    w[j] = 0;
    if (col < n && i0 < k) {                               // k is a multiple of 8
      const unsigned char* src = codes + (size_t)col * (k / 2) + i0 / 2;
#pragma unroll
      for (int e = 0; e < 8; ++e) w[j] |= (uint32_t)((src[e / 2] >> (e % 2 * 4)) & 15) << (e % 4 * 8 + e / 4 * 4);
    }
  }
  reinterpret_cast<uint4*>(dst)[lane] = make_uint4(w[0], w[1], w[2], w[3]);
  const int groups = (k + group - 1) / group, here = kDepth / group;
  for (int i = lane; i < here * kCols; i += 64) {
    const int c = (int)(blk / blocks_k) * kCols + i % kCols, gi = kb * here + i / kCols;
    uint32_t p = 0;
    if (c < n && gi < groups) {
      const size_t at = (size_t)c * groups + gi;
      const float z = zeros ? (float)(zeros[at] & 15) : 8.f;
      p = (uint32_t)__builtin_bit_cast(unsigned short, scales[at]) << 16 | __builtin_bit_cast(unsigned short, (bf16_t)z);
    }
    reinterpret_cast<uint32_t*>(dst + kCodeBytes)[i] = p;
  }
}

// one thread per group of one row: range, scale, zero point, codes
template <typename T>
__global__ __launch_bounds__(256) void q4_quantize_kernel(const T* w, int n, int k, int group, int groups, unsigned char* codes, bf16_t* scales,
                                                          unsigned char* zeros) {
  const size_t at = (size_t)blockIdx.x * 256 + threadIdx.x;
  if (at >= (size_t)n * groups) return;
  const int row = (int)(at / groups), i0 = (int)(at % groups) * group, i1 = min(i0 + group, k);
  const T* src = w + (size_t)row * k;
  float lo = 0.f, hi = 0.f;
  bool finite = true;
  for (int i = i0; i < i1; ++i) {
    const float v = st<T>::ld(src + i);
    finite &= fabsf(v) < __builtin_inff();
    lo = fminf(lo, v);
    hi = fmaxf(hi, v);
  }
  const float raw = zeros ? (hi - lo) / 15.f : fmaxf(hi, -lo) / 7.f;
  const bf16_t sb = (bf16_t)(finite ? raw : __builtin_nanf(""));
  const float s = (float)sb;
  const bool some = s > 0.f && s < __builtin_inff();
  const float z = zeros ? (some ? fminf(fmaxf(rintf(-lo / s), 0.f), 15.f) : 0.f) : 8.f;
  scales[at] = sb;
  if (zeros) zeros[at] = (unsigned char)z;
  for (int i = i0; i < i1; i += 2) {
    unsigned c[2];
#pragma unroll
    for (int e = 0; e < 2; ++e)
      c[e] = (unsigned)(some ? fminf(fmaxf(rintf(st<T>::ld(src + i + e) / s) + z, 0.f), 15.f) : z);
    codes[(size_t)row * (k / 2) + i / 2] = (unsigned char)(c[0] | c[1] << 4);
  }
}

__device__ inline bf16x8 q4_to_bf16(uint32_t w) {
  const uint32_t lo = w & 0x0f0f0f0fu, hi = (w >> 4) & 0x0f0f0f0fu;
  const bf16x2 a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, 512.f, false), b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, 512.f, true);
  const bf16x2 c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, 512.f, false), d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, 512.f, true);
  return bf16x8{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
}

constexpr int kWaves = 4;

// One workgroup: 16 columns, 16 MT rows; its waves take the 128-deep blocks of the reduction in turn and add up in LDS.
template <int GS, int MT>
__global__ __launch_bounds__(64 * kWaves) void q4_linear_kernel(const bf16_t* x, const unsigned char* packed, const int32_t* m_dev, int m_upper,
                                                                int n, int k, float* y_f32, bf16_t* y_bf16, const int32_t* row_map) {
  constexpr int kBlock = q4_block_bytes(32 * GS);
  __shared__ float sh[kWaves][16 * MT][kCols + 1];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, col = lane & 15, grp = lane >> 4;
  const int m = min(*m_dev, m_upper), m0 = blockIdx.y * 16 * MT;
  if (m0 >= m) return;
  const int blocks_k = (k + kDepth - 1) / kDepth;
  const unsigned char* wp = packed + (size_t)blockIdx.x * blocks_k * kBlock;
  const bf16_t* xr[MT];
#pragma unroll
  for (int t = 0; t < MT; ++t) xr[t] = x + (size_t)min(m0 + 16 * t + col, m - 1) * k;
  bf16x8 ones;
#pragma unroll
  for (int e = 0; e < 8; ++e) ones[e] = (bf16_t)1.f;
  f32x4 y[MT] = {};
  for (int kb = wave; kb < blocks_k; kb += kWaves) {
    const uint4 c4 = reinterpret_cast<const uint4*>(wp + (size_t)kb * kBlock)[lane];
    const uint32_t c[4] = {c4.x, c4.y, c4.z, c4.w};
#pragma unroll
    for (int j = 0; j < 4; j += GS) {
      f32x4 acc[MT] = {}, sum[MT] = {};
#pragma unroll
      for (int i = 0; i < GS; ++i) {
        const bf16x8 wf = q4_to_bf16(c[j + i]);
        const int at = kb * kDepth + (j + i) * 32 + grp * 8;
#pragma unroll
        for (int t = 0; t < MT; ++t) {
          bf16x8 xf = {};
          if (at < k) xf = *reinterpret_cast<const bf16x8*>(xr[t] + at);
          acc[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(wf, xf, acc[t], 0, 0, 0);
          sum[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(ones, xf, sum[t], 0, 0, 0);
        }
      }
      const uint4 p = reinterpret_cast<const uint4*>(wp + (size_t)kb * kBlock + kCodeBytes + j / GS * kCols * 4)[grp];
      const uint32_t ps[4] = {p.x, p.y, p.z, p.w};
#pragma unroll
      for (int t = 0; t < MT; ++t)
#pragma unroll
        for (int e = 0; e < 4; ++e)
          y[t][e] = fmaf(__uint_as_float(ps[e] & 0xffff0000u), fmaf(-__uint_as_float(ps[e] << 16), sum[t][e], acc[t][e]), y[t][e]);
    }
  }
#pragma unroll
  for (int t = 0; t < MT; ++t)
#pragma unroll
    for (int e = 0; e < 4; ++e) sh[wave][16 * t + col][4 * grp + e] = y[t][e];
  __syncthreads();
  for (int i = threadIdx.x; i < 16 * MT * kCols; i += 64 * kWaves) {
    const int r = m0 + i / kCols, c = blockIdx.x * kCols + i % kCols;
    if (r >= m || c >= n) continue;
    float v = 0.f;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) v += sh[w][i / kCols][i % kCols];
    if (y_f32) y_f32[(size_t)r * n + c] = v;
    else y_bf16[(size_t)(row_map ? row_map[r] : r) * n + c] = (bf16_t)v;
  }
}

}  // namespace

size_t slk_q4_bytes(int n, int k, int group) { return (size_t)sl_cdiv(n, kCols) * sl_cdiv(k, kDepth) * q4_block_bytes(group); }

int slk_q4_pack(hipStream_t s, const void* codes, const void* scales, const void* zeros, int n, int k, int group, void* packed) {
  const int blocks_k = sl_cdiv(k, kDepth);
  const size_t blocks = (size_t)sl_cdiv(n, kCols) * blocks_k;
  hipLaunchKernelGGL(q4_pack_kernel, dim3((unsigned)((blocks + 3) / 4)), dim3(256), 0, s, (const unsigned char*)codes, (const bf16_t*)scales,
                     (const unsigned char*)zeros, n, k, group, (unsigned char*)packed, blocks_k, blocks);
  SL_LAUNCH_CHECK();
  return SL_OK;
}

int slk_q4_quantize(hipStream_t s, const void* w, int dtype, int n, int k, int group, void* codes, void* scales, void* zeros) {
  const int groups = sl_cdiv(k, group);
  const dim3 grid((unsigned)(((size_t)n * groups + 255) / 256));
  if (dtype == SL_BF16)
    hipLaunchKernelGGL((q4_quantize_kernel<bf16_t>), grid, dim3(256), 0, s, (const bf16_t*)w, n, k, group, groups, (unsigned char*)codes,
                       (bf16_t*)scales, (unsigned char*)zeros);
  else
    hipLaunchKernelGGL((q4_quantize_kernel<float>), grid, dim3(256), 0, s, (const float*)w, n, k, group, groups, (unsigned char*)codes,
                       (bf16_t*)scales, (unsigned char*)zeros);
  SL_LAUNCH_CHECK();
  return SL_OK;
}

int slk_q4_linear(hipStream_t s, const void* x, const void* packed, const int32_t* m_dev, int m_upper, int n, int k, int group, float* y_f32,
                  void* y_bf16, const int32_t* row_map) {
  const int mt = m_upper <= 16 ? 1 : m_upper <= 32 ? 2 : 4;
  const dim3 grid(sl_cdiv(n, kCols), sl_cdiv(m_upper, 16 * mt));
#define Q4_CALL(GS, MT)                                                                                                                      \
  hipLaunchKernelGGL((q4_linear_kernel<GS, MT>), grid, dim3(64 * kWaves), 0, s, (const bf16_t*)x, (const unsigned char*)packed, m_dev, m_upper, \
                     n, k, y_f32, (bf16_t*)y_bf16, row_map)
#define Q4_BY_ROWS(GS)                                                                      \
  do {                                                                                      \
    if (mt == 1) Q4_CALL(GS, 1); else if (mt == 2) Q4_CALL(GS, 2); else Q4_CALL(GS, 4);     \
  } while (0)
  if (group == 32) Q4_BY_ROWS(1); else if (group == 64) Q4_BY_ROWS(2); else Q4_BY_ROWS(4);
#undef Q4_BY_ROWS
#undef Q4_CALL
  SL_LAUNCH_CHECK();
  return SL_OK;
}
