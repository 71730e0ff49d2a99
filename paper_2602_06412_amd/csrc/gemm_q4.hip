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

constexpr int kWaves = 8;

// One workgroup: 16 CT columns, 16 MT rows; its waves take the 128-deep blocks of the reduction in turn and add up in LDS.
//
// Rows pass through LDS, each wave's through a part of its own: an operand has 16 rows side by side in a wave's lanes, and loaded
// so from row-major memory every lane is an access of its own (16 bytes a cycle of the address unit, which was busy 70 to 88 % of
// the time).  Here eight lanes take a row's 128 consecutive bytes and the operand is read back from LDS; 16-byte
// pieces of a row that would meet in one bank are kept apart by an exclusive or of their row with their place.
// A wave asks for a block's weights and rows one block ahead.
template <int GS, int MT, int CT>
__global__ __launch_bounds__(64 * kWaves) void q4_linear_kernel(const bf16_t* x, const unsigned char* packed, const int32_t* m_dev, int m_upper,
                                                                int n, int k, float* y_f32, bf16_t* y_bf16, const int32_t* row_map) {
  constexpr int kBlock = q4_block_bytes(32 * GS), kGroups = 4 / GS;
  constexpr int kSumBytes = kWaves * 16 * (16 * CT + 4) * 4, kRowBytes = kWaves * MT * 4096;
  __shared__ __attribute__((aligned(16))) unsigned char lds[kSumBytes > kRowBytes ? kSumBytes : kRowBytes];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), col = lane & 15, grp = lane >> 4;
  const int m = min(*m_dev, m_upper), m0 = blockIdx.y * 16 * MT;
  if (m0 >= m) return;
  const int blocks_k = (k + kDepth - 1) / kDepth, tiles_n = (n + kCols - 1) / kCols;
  const unsigned char* wp[CT];                            // (a tile of columns past the last one is read as the last and not stored)
#pragma unroll
  for (int c = 0; c < CT; ++c) wp[c] = packed + (size_t)min((int)blockIdx.x * CT + c, tiles_n - 1) * blocks_k * kBlock;
  // loads of rows: lane l takes piece l % 8 (8 numbers) of row l / 8, four loads to 16 rows of a block
  const bf16_t* xr[MT][2];
#pragma unroll
  for (int t = 0; t < MT; ++t)
#pragma unroll
    for (int i = 0; i < 2; ++i) xr[t][i] = x + (size_t)min(m0 + 16 * t + 8 * i + (lane >> 3), m - 1) * k + (lane & 7) * 8;
  unsigned char* mine = lds + wave * (MT * 4096);
  const int put = ((lane & 3) * 16 + ((lane >> 3) ^ (lane & 7))) * 16 + (lane >> 2 & 1) * 1024;     // of rows 0 .. 7; rows 8 .. 15 at put ^ 128
  const int get0 = (grp * 16 + (col ^ grp)) * 16, get1 = (grp * 16 + (col ^ (grp + 4))) * 16;       // of even and odd products

  uint4 w[CT], wn[CT], p[CT][kGroups], pn[CT][kGroups], xn[MT][4];
  auto ask = [&](int kb) {
#pragma unroll
    for (int c = 0; c < CT; ++c) {
      const unsigned char* b = wp[c] + (size_t)kb * kBlock;
      wn[c] = reinterpret_cast<const uint4*>(b)[lane];
#pragma unroll
      for (int g = 0; g < kGroups; ++g) pn[c][g] = reinterpret_cast<const uint4*>(b + kCodeBytes + g * kCols * 4)[grp];
    }
    const int at = kb * kDepth;
#pragma unroll
    for (int t = 0; t < MT; ++t)
#pragma unroll
      for (int i = 0; i < 4; ++i) {                       // k is a multiple of 8: a lane's 8 numbers are all there or none
        const int d = at + i / 2 * 64;
        uint4 v = make_uint4(0, 0, 0, 0);
        if (at + kDepth <= k || d + (lane & 7) * 8 < k) v = *reinterpret_cast<const uint4*>(xr[t][i % 2] + d);
        xn[t][i] = v;
      }
  };
  bf16x8 ones;
#pragma unroll
  for (int e = 0; e < 8; ++e) ones[e] = (bf16_t)1.f;
  f32x4 y[MT][CT] = {};
  int kb = wave;
  if (kb < blocks_k) ask(kb);
  for (; kb < blocks_k; kb += kWaves) {
#pragma unroll
    for (int c = 0; c < CT; ++c) {
      w[c] = wn[c];
#pragma unroll
      for (int g = 0; g < kGroups; ++g) p[c][g] = pn[c][g];
    }
#pragma unroll
    for (int t = 0; t < MT; ++t)
#pragma unroll
      for (int i = 0; i < 4; ++i) *reinterpret_cast<uint4*>(mine + t * 4096 + i / 2 * 2048 + (i % 2 ? put ^ 128 : put)) = xn[t][i];
    if (kb + kWaves < blocks_k) ask(kb + kWaves);
#pragma unroll
    for (int g = 0; g < kGroups; ++g) {
      f32x4 acc[MT][CT], sum[MT];
#pragma unroll
      for (int i = 0; i < GS; ++i) {
        const int j = g * GS + i;
        bf16x8 wf[CT];
#pragma unroll
        for (int c = 0; c < CT; ++c) wf[c] = q4_to_bf16(j == 0 ? w[c].x : j == 1 ? w[c].y : j == 2 ? w[c].z : w[c].w);
        const f32x4 zero = {};
#pragma unroll
        for (int t = 0; t < MT; ++t) {
          const bf16x8 xf = *reinterpret_cast<const bf16x8*>(mine + t * 4096 + j * 1024 + (j % 2 ? get1 : get0));
          sum[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(ones, xf, i ? sum[t] : zero, 0, 0, 0);
#pragma unroll
          for (int c = 0; c < CT; ++c) acc[t][c] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(wf[c], xf, i ? acc[t][c] : zero, 0, 0, 0);
        }
      }
#pragma unroll
      for (int c = 0; c < CT; ++c) {
        const uint32_t ps[4] = {p[c][g].x, p[c][g].y, p[c][g].z, p[c][g].w};
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const float scale = __uint_as_float(ps[e] & 0xffff0000u), z = __uint_as_float(ps[e] << 16);
#pragma unroll
          for (int t = 0; t < MT; ++t) y[t][c][e] = fmaf(scale, fmaf(-z, sum[t][e], acc[t][c][e]), y[t][c][e]);
        }
      }
    }
  }
  auto sh = reinterpret_cast<float(*)[16][16 * CT + 4]>(lds);      // [wave][row][column]
  __syncthreads();
  const int first = blockIdx.x * 16 * CT;
#pragma unroll
  for (int t = 0; t < MT; ++t) {
    if (m0 + 16 * t >= m) break;
    if (t) __syncthreads();
#pragma unroll
    for (int c = 0; c < CT; ++c) *reinterpret_cast<f32x4*>(&sh[wave][col][16 * c + 4 * grp]) = y[t][c];
    __syncthreads();
    for (int i = threadIdx.x; i < 64 * CT; i += 64 * kWaves) {
      const int r = m0 + 16 * t + i / (4 * CT), c = i % (4 * CT) * 4;
      if (r >= m || first + c >= n) continue;
      f32x4 v = {};
#pragma unroll
      for (int s = 0; s < kWaves; ++s) v += *reinterpret_cast<const f32x4*>(&sh[s][i / (4 * CT)][c]);
      const size_t at = (size_t)(row_map ? row_map[r] : r) * n + first + c;
#pragma unroll
      for (int e = 0; e < 4; ++e)
        if (first + c + e < n) {
          if (y_f32) y_f32[at + e] = v[e];
          else y_bf16[at + e] = (bf16_t)v[e];
        }
    }
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
  const int tiles = sl_cdiv(m_upper, 16);
#ifndef FM
  int mt = tiles >= 2 ? 2 : 1, ct = 2;
#else
  int mt = FM, ct = FC;
#endif
  const dim3 grid(sl_cdiv(n, kCols * ct), sl_cdiv(m_upper, 16 * mt));
#define Q4_CALL(GS, MT, CT)                                                                                                                      \
  hipLaunchKernelGGL((q4_linear_kernel<GS, MT, CT>), grid, dim3(64 * kWaves), 0, s, (const bf16_t*)x, (const unsigned char*)packed, m_dev, m_upper, \
                     n, k, y_f32, (bf16_t*)y_bf16, row_map)
#define Q4_BY_TILE(GS)                             \
  do {                                             \
    if (mt == 1 && ct == 1) Q4_CALL(GS, 1, 1);     \
    else if (mt == 1 && ct == 2) Q4_CALL(GS, 1, 2); \
    else if (mt == 1) Q4_CALL(GS, 1, 4);           \
    else if (mt == 2 && ct == 1) Q4_CALL(GS, 2, 1); \
    else if (mt == 2 && ct == 2) Q4_CALL(GS, 2, 2); \
    else if (mt == 2) Q4_CALL(GS, 2, 4);           \
    else Q4_CALL(GS, 4, 2);                        \
  } while (0)
  if (group == 32) Q4_BY_TILE(1); else if (group == 64) Q4_BY_TILE(2); else Q4_BY_TILE(4);
#undef Q4_BY_TILE
#undef Q4_CALL
  SL_LAUNCH_CHECK();
  return SL_OK;
}
