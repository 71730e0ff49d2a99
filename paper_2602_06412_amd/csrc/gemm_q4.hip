// Products of a few bf16 rows with 4-bit weights: y = x W^T, W[j, i] = s[j, i / g] (q[j, i] - z[j, i / g]).
//
// A code q in 0..15 as a byte is the e4m3 number q 2^-9 (a subnormal, or a normal with the smallest exponent), so the conversion
// from e4m3 to bf16 with a scale of 2^9 yields two exact bf16 integers an instruction; the zero point and the scale of a
// group are applied to sums:
//   sum_i x_i s (q_i - z) = s ( sum_i x_i q_i  -  z sum_i x_i ),
// the first from the matrix cores in fp32, the second added up in fp32 as rows pass through LDS.  (A code in the upper bits of a
// bf16 mantissa, 16 + q, costs as many instructions and an offset three times as large to be taken off again.)
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

// over the L = 4, 8 or 16 neighbouring lanes that hold a group, in all of them
template <int L, typename F>
__device__ inline float over_lanes(float v, F f) {
  auto moved = [](uint32_t x) { return __uint_as_float(x); };
  v = f(v, moved(__builtin_amdgcn_mov_dpp(__float_as_uint(v), 0xB1, 15, 15, true)));             // lane ^ 1
  v = f(v, moved(__builtin_amdgcn_mov_dpp(__float_as_uint(v), 0x4E, 15, 15, true)));             // lane ^ 2
  if (L >= 8) v = f(v, moved(__builtin_amdgcn_mov_dpp(__float_as_uint(v), 0x141, 15, 15, true)));        // 7 - lane, of 8
  if (L >= 16) v = f(v, moved(__builtin_amdgcn_mov_dpp(__float_as_uint(v), 0x140, 15, 15, true)));       // 15 - lane, of 16
  return v;
}

// Range, scale, zero point and codes; eight numbers a lane, group / 8 lanes a group.  24576 x 4096 bf16 take 92 us (253 MB, 2.8 TB/s:
// bound by vector instructions, 310 a wave, the pipes busy throughout; it runs once, when weights are loaded); a thread for each group
// took 3.7 ms.
template <typename T, int GROUP>
__global__ __launch_bounds__(256) void q4_quantize_kernel(const T* w, int n, int k, int groups, unsigned char* codes, bf16_t* scales, unsigned char* zeros) {
  constexpr int L = GROUP / 8;
  const uint32_t lanes = (uint32_t)groups * L;             // of a row
  const uint64_t first = (uint64_t)blockIdx.x * 256, row0 = first / lanes;
  const uint32_t in = (uint32_t)(first - row0 * lanes) + threadIdx.x, up = in / lanes, at = in - up * lanes;
  const uint64_t row = row0 + up;
  const bool there = row < (uint64_t)n && at * 8 < (uint32_t)k;       // k is a multiple of 8: a lane's numbers are all there or none
  float v[8] = {}, lo = 0.f, hi = 0.f, most = 0.f;
  if (there) {
    const T* src = w + row * k + at * 8;
    if constexpr (sizeof(T) == 2) ld8(src, v); else ld8f(src, v);
  }
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    most = v[e] != v[e] ? __builtin_inff() : fmaxf(most, fabsf(v[e]));
    lo = fminf(lo, v[e]);
    hi = fmaxf(hi, v[e]);
  }
  auto larger = [](float x, float y) { return fmaxf(x, y); };
  most = over_lanes<L>(most, larger);
  hi = over_lanes<L>(hi, larger);
  lo = over_lanes<L>(lo, [](float x, float y) { return fminf(x, y); });
  const float span = hi - lo;                              // infinity where all weights are finite: one at each end of fp32's range
  const float raw = !zeros ? most / 7.f : span < __builtin_inff() ? span / 15.f : hi / 15.f - lo / 15.f;
  const bf16_t sb = (bf16_t)(most < __builtin_inff() ? raw : __builtin_nanf(""));
  const float s = (float)sb;
  const bool some = s > 0.f && s < __builtin_inff();
  const float z = !zeros ? 8.f : some ? fminf(fmaxf(rintf(-lo / s), 0.f), 15.f) : 0.f;
  uint32_t c = 0;
#pragma unroll
  for (int e = 0; e < 8; ++e) c |= (uint32_t)(some ? fminf(fmaxf(rintf(v[e] / s) + z, 0.f), 15.f) : z) << (4 * e);
  if (!there) return;
  *reinterpret_cast<uint32_t*>(codes + row * (k / 2) + at * 4) = c;
  if (at % L == 0) {
    scales[row * groups + at / L] = sb;
    if (zeros) zeros[row * groups + at / L] = (unsigned char)z;
  }
}

__device__ inline bf16x8 q4_to_bf16(uint32_t w) {
  const uint32_t lo = w & 0x0f0f0f0fu, hi = (w >> 4) & 0x0f0f0f0fu;
  const bf16x2 a = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, 512.f, false), b = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(lo, 512.f, true);
  const bf16x2 c = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, 512.f, false), d = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(hi, 512.f, true);
  return bf16x8{a[0], a[1], b[0], b[1], c[0], c[1], d[0], d[1]};
}

// sum over the 4 or 8 neighbouring lanes that hold one row's pieces, in all of them
template <int N>
__device__ inline float sum_neighbours(float v) {
  v += __uint_as_float(__builtin_amdgcn_mov_dpp(__float_as_uint(v), 0xB1, 15, 15, true));          // lane ^ 1
  v += __uint_as_float(__builtin_amdgcn_mov_dpp(__float_as_uint(v), 0x4E, 15, 15, true));          // lane ^ 2
  if (N == 8) v += __uint_as_float(__builtin_amdgcn_mov_dpp(__float_as_uint(v), 0x141, 15, 15, true));      // 7 - lane, of 8
  return v;
}
__device__ inline float sum_of_piece(const uint4& v) {
  const bf16x2 one = {(bf16_t)1.f, (bf16_t)1.f};
  float s = __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2, v.x), one, 0.f, false);
  s = __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2, v.y), one, s, false);
  s = __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2, v.z), one, s, false);
  return __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2, v.w), one, s, false);
}

// One workgroup: 16 MT rows, WN waves side by side of 16 CT columns each, WK such groups along the reduction, which add up in LDS
// at the end.  A wave asks U blocks (128 deep) of its group ahead for weights and rows.
//
// Rows pass through LDS, once for the WN waves of a group, and with them goes the sum of each group of weights' inputs.  An
// operand has 16 rows side by side in a wave's lanes, and loaded so from row-major memory every lane is an access of its own (16
// bytes a cycle of the address unit, which was busy 70 % of the time: 61 rows, n = 4096, k = 12288 took 53 us; 33 through LDS with the
// rest as it was, 18 to 21 now).  Here eight
// lanes take a row's 128 consecutive bytes; 16-byte pieces that would meet in one bank are kept apart by an exclusive or of their row
// with their place.
template <int GS, int MT, int CT, int WN, int WK, int U>
__global__ __launch_bounds__(64 * WN * WK) void q4_linear_kernel(const bf16_t* x, const unsigned char* packed, const int32_t* m_dev, int m_upper, int n,
                                                               int k, float* y_f32, bf16_t* y_bf16, const int32_t* row_map) {
  constexpr int kBlock = q4_block_bytes(32 * GS), kGroups = 4 / GS, kUnits = (MT * 2 + WN - 1) / WN, kWidth = 16 * CT * WN;
  constexpr int kBufs = WN > 1 ? 2 : 1;                   // a group of several waves writes one while the other is read
  constexpr int kRowBytes = WK * kBufs * MT * 4096, kSumBytes = WK * 16 * (kWidth + 4) * 4;
  __shared__ __attribute__((aligned(16))) unsigned char lds[kRowBytes > kSumBytes ? kRowBytes : kSumBytes];
  __shared__ float sums[WK][kBufs][kGroups][16 * MT];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), col = lane & 15, grp = lane >> 4;
  const int wn = wave % WN, wk = wave / WN;
  const int m = min(*m_dev, m_upper), m0 = blockIdx.y * 16 * MT;
  if (m0 >= m) return;
  const int blocks_k = (k + kDepth - 1) / kDepth, tiles_n = (n + kCols - 1) / kCols;
  const unsigned char* wp[CT];                            // (a tile of columns past the last one is read as the last and not stored)
#pragma unroll
  for (int c = 0; c < CT; ++c) wp[c] = packed + (size_t)min((int)(blockIdx.x * WN + wn) * CT + c, tiles_n - 1) * blocks_k * kBlock;
  const int put = ((lane & 3) * 16 + ((lane >> 3) ^ (lane & 7))) * 16 + (lane >> 2 & 1) * 1024;     // as below, rows 0 .. 7
  const int get0 = (grp * 16 + (col ^ grp)) * 16, get1 = (grp * 16 + (col ^ (grp + 4))) * 16;
  // a wave's share of the rows: 8 rows q % 2 of tile q / 2, eight lanes to 128 bytes of a row.  Rows past the count are read as the
  // last one (they end in results that are not stored), pieces past k as the last one and then cleared
  const bf16_t* xr[kUnits];
#pragma unroll
  for (int u = 0; u < kUnits; ++u) xr[u] = x + (size_t)min(m0 + 8 * (wn + u * WN) + (lane >> 3), m - 1) * k + (lane & 7) * 8;
  uint4 w[U][CT], p[U][CT][kGroups], xn[U][kUnits][2];
  auto ask = [&](int s, int kb) {
#pragma unroll
    for (int c = 0; c < CT; ++c) {
      const unsigned char* b = wp[c] + (size_t)kb * kBlock;
      w[s][c] = reinterpret_cast<const uint4*>(b)[lane];
#pragma unroll
      for (int g = 0; g < kGroups; ++g) p[s][c][g] = reinterpret_cast<const uint4*>(b + kCodeBytes + g * kCols * 4)[grp];
    }
#pragma unroll
    for (int u = 0; u < kUnits; ++u) {
      xn[s][u][0] = *reinterpret_cast<const uint4*>(xr[u] + min(kb * kDepth, k - 8 - (lane & 7) * 8));
      xn[s][u][1] = *reinterpret_cast<const uint4*>(xr[u] + min(kb * kDepth + 64, k - 8 - (lane & 7) * 8));
    }
  };
  f32x4 y[MT][CT] = {};
  const int steps = (blocks_k + WK - 1) / WK;
#pragma unroll
  for (int s = 0; s < U; ++s)
    ask(s, min(s * WK + wk, blocks_k - 1));
  for (int it0 = 0; it0 < steps; it0 += U)
#pragma unroll
  for (int s = 0; s < U; ++s) {
    const int it = it0 + s, kb = it * WK + wk;
    if (it >= steps) break;
    unsigned char* buf = lds + (wk * kBufs + it % kBufs) * (MT * 4096);
    if (kb * kDepth + kDepth > k) {                       // the last block, or one past it
#pragma unroll
      for (int u = 0; u < kUnits; ++u)
#pragma unroll
        for (int i = 0; i < 2; ++i)
          if (kb * kDepth + 64 * i + (lane & 7) * 8 >= k) xn[s][u][i] = make_uint4(0, 0, 0, 0);
    }
#pragma unroll
      for (int u = 0; u < kUnits; ++u) {
        const int q = wn + u * WN;
        if (2 * MT % WN == 0 || q < 2 * MT) {
          unsigned char* dst = buf + q / 2 * 4096 + (q % 2 ? put ^ 128 : put);
          *reinterpret_cast<uint4*>(dst) = xn[s][u][0];
          *reinterpret_cast<uint4*>(dst + 2048) = xn[s][u][1];
          const float a = sum_of_piece(xn[s][u][0]), b = sum_of_piece(xn[s][u][1]);
          float* to = &sums[wk][it % kBufs][0][8 * q + (lane >> 3)];
          if (GS == 4) {
            const float v = sum_neighbours<8>(a + b);
            if ((lane & 7) == 0) to[0] = v;
          } else if (GS == 2) {
            const float v = sum_neighbours<8>(a), v2 = sum_neighbours<8>(b);
            if ((lane & 7) == 0) { to[0] = v; to[16 * MT] = v2; }
          } else {
            const float v = sum_neighbours<4>(a), v2 = sum_neighbours<4>(b);
            if ((lane & 3) == 0) { to[(lane >> 2 & 1) * 16 * MT] = v; to[(2 + (lane >> 2 & 1)) * 16 * MT] = v2; }
          }
        }
      }
    if (WN > 1) {
      __syncthreads();
    } else {                                              // rows of the wave's own: LDS serves a wave in order
      __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
      __builtin_amdgcn_wave_barrier();
    }
#pragma unroll
    for (int g = 0; g < kGroups; ++g) {
      f32x4 acc[MT][CT];
#pragma unroll
      for (int i = 0; i < GS; ++i) {
        const int j = g * GS + i;
        bf16x8 wf[CT];
#pragma unroll
        for (int c = 0; c < CT; ++c) wf[c] = q4_to_bf16(j == 0 ? w[s][c].x : j == 1 ? w[s][c].y : j == 2 ? w[s][c].z : w[s][c].w);
        const f32x4 zero = {};
#pragma unroll
        for (int t = 0; t < MT; ++t) {
          const bf16x8 xf = *reinterpret_cast<const bf16x8*>(buf + t * 4096 + j * 1024 + (j % 2 ? get1 : get0));
#pragma unroll
          for (int c = 0; c < CT; ++c) acc[t][c] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(wf[c], xf, i ? acc[t][c] : zero, 0, 0, 0);
        }
      }
      float sx[MT];
#pragma unroll
      for (int t = 0; t < MT; ++t) sx[t] = sums[wk][it % kBufs][g][16 * t + col];
#pragma unroll
      for (int c = 0; c < CT; ++c) {
        const uint32_t ps[4] = {p[s][c][g].x, p[s][c][g].y, p[s][c][g].z, p[s][c][g].w};
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const float scale = __uint_as_float(ps[e] & 0xffff0000u), z = __uint_as_float(ps[e] << 16);
#pragma unroll
          for (int t = 0; t < MT; ++t) y[t][c][e] = fmaf(scale, fmaf(-z, sx[t], acc[t][c][e]), y[t][c][e]);
        }
      }
    }
    ask(s, min(kb + U * WK, blocks_k - 1));
  }
  auto sh = reinterpret_cast<float(*)[16][kWidth + 4]>(lds);
  const int first = blockIdx.x * kWidth;
#pragma unroll
  for (int t = 0; t < MT; ++t) {
    if (m0 + 16 * t >= m) break;
    __syncthreads();
#pragma unroll
    for (int c = 0; c < CT; ++c) *reinterpret_cast<f32x4*>(&sh[wk][col][(wn * CT + c) * 16 + 4 * grp]) = y[t][c];
    __syncthreads();
    for (int i = threadIdx.x; i < 4 * kWidth; i += 64 * WN * WK) {
      const int r = m0 + 16 * t + i / (kWidth / 4), c = i % (kWidth / 4) * 4;
      if (r >= m || first + c >= n) continue;
      f32x4 v = {};
#pragma unroll
      for (int s = 0; s < WK; ++s) v += *reinterpret_cast<const f32x4*>(&sh[s][i / (kWidth / 4)][c]);
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
  const dim3 grid((unsigned)(((uint64_t)n * groups * (group / 8) + 255) / 256));
#define Q4_CALL(T, G) \
  hipLaunchKernelGGL((q4_quantize_kernel<T, G>), grid, dim3(256), 0, s, (const T*)w, n, k, groups, (unsigned char*)codes, (bf16_t*)scales, (unsigned char*)zeros)
#define Q4_BY_GROUP(T) \
  do { if (group == 32) Q4_CALL(T, 32); else if (group == 64) Q4_CALL(T, 64); else Q4_CALL(T, 128); } while (0)
  if (dtype == SL_BF16) Q4_BY_GROUP(bf16_t); else Q4_BY_GROUP(float);
#undef Q4_BY_GROUP
#undef Q4_CALL
  SL_LAUNCH_CHECK();
  return SL_OK;
}

int slk_q4_linear(hipStream_t s, const void* x, const void* packed, const int32_t* m_dev, int m_upper, int n, int k, int group, float* y_f32,
                  void* y_bf16, const int32_t* row_map) {
  // Tiles, us by tile (rows x columns, waves side by side x along the reduction), a node of a graph over four sets of weights, groups of
  // 128; * is what the rule takes:
  //   n, k, rows            16x16,1x16  16x32,1x8  16x48,1x8  32x32,1x8  32x128,4x2
  //   4096, 4096, 1             4.8 *      6.0        6.8        7.7        16.4
  //   4096, 12288, 16           9.4 *     13.0       15.2       17.4        43.6
  //   4096, 2048, 1             3.5 *      3.8        4.4        4.8         8.7
  //   4096, 1920, 1             3.5        3.9 *      4.5        5.1         9.3
  //   4096, 1024, 1             3.5        3.1 *      3.4        3.7         5.6
  //   4352, 4096, 1             7.3        6.1 *      6.9        7.8        16.4
  //   8192, 4096, 16            8.0        6.4 *      7.3        8.1        16.6
  //   8704, 4096, 16           10.7        8.4        7.3 *     11.1        16.7
  //   12288, 4096, 16          11.2        8.8        7.8 *     11.7        16.8
  //   24576, 4096, 8           19.5       11.8       11.7 *     16.3        17.6
  //   4096, 4096, 32            7.8        6.2 *      7.3        8.3        17.1
  //   4096, 12288, 61          30.2       20.2       26.1       18.3 *      44.0
  //   12288, 4096, 48          28.7       16.7       15.0       17.1        17.3 *
  //   4096, 4096, 128          24.6       13.8       15.6       12.2 *      17.0
  //   6144, 4096, 100          32.7       18.2       17.5       16.7        17.0 *
  //   12288, 4096, 64          37.5       19.7       18.7       18.0        17.4 *
  //   12288, 4096, 100         62.9       32.4       29.5       30.6        24.6 *
  //   24576, 4096, 224        254        131        122        110          75.3 *
  // Few rows are a matter of the weights' latency: workgroups enough for all CUs, many waves along the reduction, and as many columns as
  // still leave one workgroup to a CU.  16 waves want 16 blocks to share out: with 15 the rule is 10 % off, with 8 eight waves are the
  // better ones.  Many rows are a matter of unpacking weights and of moving rows: a large tile whose waves share them, once there are
  // enough of it; at 192 workgroups of it the two are within 4 %, at 128 it takes 1.4 times as long, at 384 0.8.  (33 to 48 rows of wide
  // matrices are 15 % off: three row tiles in the room of four.)
  const int64_t rows16 = sl_cdiv(m_upper, 16), tiles_n = sl_cdiv(n, kCols), blocks_k = sl_cdiv(k, kDepth);
#define Q4_RUN(GS, MT, CT, WN, WK, U)                                                                                                  \
  hipLaunchKernelGGL((q4_linear_kernel<GS, MT, CT, WN, WK, U>), dim3(sl_cdiv(n, kCols * CT * WN), sl_cdiv(m_upper, 16 * MT)),          \
                     dim3(64 * WN * WK), 0, s, (const bf16_t*)x, (const unsigned char*)packed, m_dev, m_upper, n, k, y_f32,             \
                     (bf16_t*)y_bf16, row_map)
#define Q4_BY_TILE(GS)                                                                                                                 \
  do {                                                                                                                                 \
    if (rows16 >= 3 && (int64_t)sl_cdiv(n, 128) * sl_cdiv(m_upper, 32) >= 192) Q4_RUN(GS, 2, 2, 4, 2, 2);                                       \
    else if (rows16 >= 3) Q4_RUN(GS, 2, 2, 1, 8, 1);                                                                                   \
    else if (rows16 == 1 && tiles_n <= 256 && blocks_k >= 16) Q4_RUN(GS, 1, 1, 1, 16, 1);                                              \
    else if (tiles_n * rows16 <= 512) Q4_RUN(GS, 1, 2, 1, 8, 1);                                                                       \
    else Q4_RUN(GS, 1, 3, 1, 8, 1);                                                                                                    \
  } while (0)
  if (group == 32) Q4_BY_TILE(1); else if (group == 64) Q4_BY_TILE(2); else Q4_BY_TILE(4);
#undef Q4_BY_TILE
#undef Q4_RUN
  SL_LAUNCH_CHECK();
  return SL_OK;
}
