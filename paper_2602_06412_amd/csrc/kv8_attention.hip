// Attention of a few rows per sequence over the paged 8-bit cache.
//
//   o[r, h] = sum_{p < L_r} P_p V[p],  P = softmax(scale q[r, h] . K[p]),  L_r = min(seq_len, row_len[r], the table's slots)
//
// The rows of a sequence times the query heads that share a K/V head are one list of queries; 16 of them are a tile, the columns
// of the matrix products: S^T = K Q^T (16 slots x 16 queries) and O^T = V^T P^T.  S^T leaves in lane l the scores of query l % 16
// and slots 4 (l / 16) .. + 3 of a tile, which is the operand the second product wants, so probabilities never leave registers.
//
// Unpacking codes is what such a kernel would spend its time on: an integer-to-float conversion costs a wave four times an
// addition, and as bf16 by conversion K and V took 14 us per step of 64 slots and wave where three waves shared a SIMD.  So
//   K is not unpacked: the product is one of 8-bit integers, the query being a fixed-point number of three signed bytes,
//     q = 2^(e - 22) (65536 a + 256 b + c), 2^(e-1) <= max|q| < 2^e: 23 bits of the row's largest number, as good as fp32's own sums.
//     Each byte's product starts from the integer 0x4B400000, whose bits are the float 1.5 * 2^23, so that the result, below 2^22
//     for 256 dimensions, is that float plus itself: one subtraction instead of a conversion.
//   V becomes half precision in two operations a pair: 0x6400 + (code + 128) are the bits of the half 1024 + code + 128.
//   A probability times V's scale goes in as two halves (22 bits), scaled by a power of two per query so that the largest seen lies
//     below 2^14: what is 2^38 times smaller than it is dropped.  One half would leave 11 bits, against a result rounded to 8 in
//     bf16, but to 24 in fp32.
// Scores, maximum, sum and output accumulate in fp32.
#include "kv8.h"

namespace {

typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
constexpr float kNegInf = -__builtin_inff();
constexpr int kMagicBits = 0x4B400000;
constexpr float kMagic = 12582912.f;                      // its float
constexpr int kTop = 14;                                  // probabilities lie below 2^kTop

// a lane's share of an 8-bit operand: 16 bytes (8 with d = 32)
template <int E> struct Piece;
template <> struct Piece<8> {
  typedef uint2 type;
  static __device__ i32x4 mfma(const uint2& a, const uint2& b, i32x4 c) {
    return __builtin_amdgcn_mfma_i32_16x16x32_i8(__builtin_bit_cast(long, a), __builtin_bit_cast(long, b), c, 0, 0, 0);
  }
};
template <> struct Piece<16> {
  typedef uint4 type;
  static __device__ i32x4 mfma(const uint4& a, const uint4& b, i32x4 c) {
    return __builtin_amdgcn_mfma_i32_16x16x64_i8(__builtin_bit_cast(i32x4, a), __builtin_bit_cast(i32x4, b), c, 0, 0, 0);
  }
};
template <typename P>
__device__ inline uint32_t word(const P& p, int i) { return reinterpret_cast<const uint32_t*>(&p)[i]; }

// V's codes (each + 128) of 4 slots of one tile and 4 of the next, as halves
__device__ inline f16x8 v_halves(uint32_t a, uint32_t b) {
  const f16x2 off = {(_Float16)1152.f, (_Float16)1152.f};
  const f16x2 r0 = __builtin_bit_cast(f16x2, __builtin_amdgcn_perm(0x64646464u, a, 0x04010400u)) - off;
  const f16x2 r1 = __builtin_bit_cast(f16x2, __builtin_amdgcn_perm(0x64646464u, a, 0x04030402u)) - off;
  const f16x2 r2 = __builtin_bit_cast(f16x2, __builtin_amdgcn_perm(0x64646464u, b, 0x04010400u)) - off;
  const f16x2 r3 = __builtin_bit_cast(f16x2, __builtin_amdgcn_perm(0x64646464u, b, 0x04030402u)) - off;
  return f16x8{r0[0], r0[1], r1[0], r1[1], r2[0], r2[1], r3[0], r3[1]};
}

// x = 2^-22 times three signed bytes in base 256, for x of at most 2^22 in magnitude
__device__ inline void three_bytes(float x, int& a, int& b, int& c) {
  const int i = (int)rintf(x);
  c = (int)(signed char)i;
  const int j = (i - c) >> 8;
  b = (int)(signed char)j;
  a = (j - b) >> 8;
}

struct Kv8Attn {
  const void* q;
  void* out;
  float* part;                                            // partial results of the chunks, or null: one chunk
  const int32_t *cu_rows, *seq_len, *row_len;
  int64_t q_stride, out_stride;
  int n_heads, share, m_upper, len_upper;                 // share = query heads per K/V head
  int chunk, chunks;                                      // slots a workgroup takes, and how many such there are
  float scale_log2;                                       // scale * log2(e): probabilities are powers of two
  __device__ int rows_of(int b, int& row0) const {
    row0 = min(max(cu_rows[b], 0), m_upper);
    return min(max(cu_rows[b + 1] - row0, 0), m_upper - row0);
  }
  __device__ int limit_of(int b, int r, int slots) const {
    int n = min(min(max(seq_len[b], 0), slots), len_upper);
    if (row_len) n = min(n, row_len[r]);
    return n;
  }
  // partial sums [row and head][chunk][d], behind them maximum and sum [row and head][chunk]
  __device__ float* sums(size_t rh, int c, int d) const { return part + (rh * chunks + c) * d; }
  __device__ float2* stats(size_t rh, int c, int d) const {
    return reinterpret_cast<float2*>(part + (size_t)m_upper * n_heads * chunks * d) + rh * chunks + c;
  }
};

// Tile `t` of `width` queries -> its sequence, its first query there, the sequence's rows; false past the last tile.  A wave
// asks together: 64 sequences' tiles at once, added up along the lanes.
__device__ inline bool kv8_tile_of(const Kv8Attn& a, int batch, int width, int t, int& b, int& first, int& row0, int& rows) {
  const int lane = threadIdx.x & 63;
  for (int b0 = 0; b0 < batch; b0 += 64) {
    int start = 0, n = 0;
    if (b0 + lane < batch) n = a.rows_of(b0 + lane, start);
    const int tiles = (n * a.share + width - 1) / width;
    int upto = tiles;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
      const int before = __shfl_up(upto, o, 64);
      if (lane >= o) upto += before;
    }
    const uint64_t past = __ballot(upto > t);
    if (past) {
      const int at = __builtin_ffsll((long long)past) - 1;
      b = __builtin_amdgcn_readfirstlane(b0 + at);
      first = __builtin_amdgcn_readfirstlane((t - __shfl(upto - tiles, at, 64)) * width);
      row0 = __builtin_amdgcn_readfirstlane(__shfl(start, at, 64));
      rows = __builtin_amdgcn_readfirstlane(__shfl(n, at, 64));
      return true;
    }
    t -= __shfl(upto, 63, 64);
  }
  return false;
}

constexpr int kWaves = 4, kStepTiles = 4;                 // a wave takes 64 slots a step
constexpr int kStep = 16 * kStepTiles;

// One workgroup: one K/V head, QT tiles of 16 queries, one chunk of the slots; its waves take the steps in turn.
template <typename T, int D, int QT>
__global__ __launch_bounds__(64 * kWaves) void kv8_attention_kernel(Kv8View kv, Kv8Attn a) {
  using Tile = Kv8Tile<D>;
  constexpr int E = Tile::E, CH = Tile::CH, DT = D / 16;
  typedef typename Piece<E>::type piece;
  __shared__ float o_sh[kWaves][16][D + 4];
  __shared__ float m_sh[kWaves][16 * QT], l_sh[kWaves][16 * QT];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), col = lane & 15, grp = lane >> 4;
  const int kvh = blockIdx.y, chunk0 = blockIdx.z * a.chunk;
  int b, first, row0, rows;
  if (!kv8_tile_of(a, kv.batch, 16 * QT, blockIdx.x, b, first, row0, rows)) return;
  const int queries = rows * a.share;
  int limit[QT], most = 0, least = 1 << 30;               // of the tile's queries
  piece qd[QT][CH][3];                                    // the query's bytes
  int qe[QT];                                             // its exponent - 22
  float qnan[QT];                                         // NaN for a query that is not finite, else 0
#pragma unroll
  for (int t = 0; t < QT; ++t) {
    const int f = first + 16 * t + col;
    const bool live = f < queries;
    const int r = row0 + (live ? f / a.share : 0), h = kvh * a.share + (live ? f % a.share : 0);
    limit[t] = live ? a.limit_of(b, r, kv.slots()) : 0;
    most = max(most, limit[t]);
    if (live) least = min(least, limit[t]);
    const T* qr = (const T*)a.q + (size_t)r * a.q_stride + (size_t)h * D;
    float x[CH][E];
    uint32_t big = 0;
#pragma unroll
    for (int c = 0; c < CH; ++c)
#pragma unroll
      for (int u = 0; u < E; u += 8) {
        float y[8];
        if constexpr (sizeof(T) == 2) ld8(qr + c * 4 * E + grp * E + u, y); else ld8f(qr + c * 4 * E + grp * E + u, y);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          x[c][u + e] = y[e];
          big = max(big, __float_as_uint(y[e]) & 0x7fffffffu);
        }
      }
    big = max(big, (uint32_t)__shfl_xor((int)big, 16, 64));
    big = max(big, (uint32_t)__shfl_xor((int)big, 32, 64));
    const bool finite = big < 0x7f800000u;
    const int e = finite ? __builtin_amdgcn_frexp_expf(__uint_as_float(big)) : 0;
    qe[t] = e - 22;
    qnan[t] = finite ? 0.f : __builtin_nanf("");
#pragma unroll
    for (int c = 0; c < CH; ++c) {
      uint32_t w[3][E / 4] = {};
#pragma unroll
      for (int u = 0; u < E; ++u) {
        int d[3];
        three_bytes(finite ? __builtin_amdgcn_ldexpf(x[c][u], 22 - e) : 0.f, d[0], d[1], d[2]);
#pragma unroll
        for (int p = 0; p < 3; ++p) w[p][u / 4] |= (uint32_t)(d[p] & 255) << (u % 4 * 8);
      }
#pragma unroll
      for (int p = 0; p < 3; ++p) __builtin_memcpy(&qd[t][c][p], w[p], E);
    }
  }
#pragma unroll
  for (int o = 8; o > 0; o >>= 1) {
    most = max(most, __shfl_xor(most, o, 64));
    least = min(least, __shfl_xor(least, o, 64));
  }
  most = __builtin_amdgcn_readfirstlane(most);
  least = __builtin_amdgcn_readfirstlane(least);
  if (a.part && chunk0 >= most) return;                   // the join does not ask for it
  const int end = min(most, chunk0 + a.chunk);

  f32x4 o[QT][DT] = {};
  float m[QT], l[QT];                                     // of this wave's slots; l of this lane's
  int top[QT];                                            // o is scaled by 2^(kTop - top)
#pragma unroll
  for (int t = 0; t < QT; ++t) { m[t] = kNegInf; l[t] = 0.f; top[t] = -300; }
  int pages = 0;                                          // lane i: the page of tile i % 4 of the (i / 4)-th of 16 steps
  for (int s0 = chunk0 + wave * kStep, step = 0; s0 < end; s0 += kWaves * kStep, ++step) {
    if (step % 16 == 0) {
      const int slot = s0 + (lane / kStepTiles) * (kWaves * kStep) + lane % kStepTiles * 16;
      pages = slot < end ? kv.table[(size_t)b * kv.max_pages + (slot >> kv.page_shift)] : -1;
    }
    const unsigned char* tile[kStepTiles];
    bool ok[kStepTiles], whole = s0 + kStep <= least;     // whole: every query sees every slot of the step
#pragma unroll
    for (int j = 0; j < kStepTiles; ++j) {
      const int page = __builtin_amdgcn_readlane(pages, step % 16 * kStepTiles + j);
      ok[j] = page >= 0 && page < kv.n_pages;
      whole &= ok[j];
      tile[j] = kv.tile<D>(ok[j] ? page : 0, kvh, s0 + 16 * j);
    }
    piece kc[kStepTiles][CH], vc[kStepTiles][CH];
    f32x4 ks[kStepTiles], vs[kStepTiles];
#pragma unroll
    for (int j = 0; j < kStepTiles; ++j) {
#pragma unroll
      for (int c = 0; c < CH; ++c) kc[j][c] = reinterpret_cast<const piece*>(tile[j])[c * 64 + lane];
      ks[j] = *reinterpret_cast<const f32x4*>(tile[j] + Tile::kKs + 16 * grp);
    }
#pragma unroll
    for (int j = 0; j < kStepTiles; ++j) {
      vs[j] = *reinterpret_cast<const f32x4*>(tile[j] + Tile::kVs + 16 * grp);
#pragma unroll
      for (int c = 0; c < CH; ++c) vc[j][c] = reinterpret_cast<const piece*>(tile[j] + Tile::kV)[c * 64 + lane];
    }
    float s[QT][kStepTiles][4];
#pragma unroll
    for (int j = 0; j < kStepTiles; ++j)
#pragma unroll
      for (int t = 0; t < QT; ++t) {
        const i32x4 zero = {kMagicBits, kMagicBits, kMagicBits, kMagicBits};
        i32x4 acc[3] = {zero, zero, zero};
#pragma unroll
        for (int c = 0; c < CH; ++c)
#pragma unroll
          for (int p = 0; p < 3; ++p) acc[p] = Piece<E>::mfma(kc[j][c], qd[t][c][p], acc[p]);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const float x = fmaf(__int_as_float(acc[0][i]) - kMagic, 65536.f,
                               fmaf(__int_as_float(acc[1][i]) - kMagic, 256.f, __int_as_float(acc[2][i]) - kMagic));
          s[t][j][i] = __builtin_amdgcn_ldexpf(fmaf(x, ks[j][i] * a.scale_log2, qnan[t]), qe[t]);
        }
      }
    if (!whole) {
#pragma unroll
      for (int j = 0; j < kStepTiles; ++j)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const int slot = s0 + 16 * j + 4 * grp + i;
#pragma unroll
          for (int t = 0; t < QT; ++t)
            if (!ok[j] || slot >= limit[t]) s[t][j][i] = kNegInf;
        }
    }
    f16x8 hi[QT][kStepTiles / 2], lo[QT][kStepTiles / 2];
#pragma unroll
    for (int t = 0; t < QT; ++t) {
      float best = kNegInf, w[kStepTiles][4], most_w = 0.f;
#pragma unroll
      for (int j = 0; j < kStepTiles; ++j)
#pragma unroll
        for (int i = 0; i < 4; ++i) best = fmaxf(best, s[t][j][i]);
      best = fmaxf(best, __shfl_xor(best, 16, 64));
      best = fmaxf(best, __shfl_xor(best, 32, 64));
      const float m_new = fmaxf(m[t], best), base = m_new == kNegInf ? 0.f : m_new;
      float sum = 0.f;
#pragma unroll
      for (int j = 0; j < kStepTiles; ++j)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const float x = s[t][j][i], p = __builtin_amdgcn_exp2f(x - base);
          sum += p;
          w[j][i] = x == kNegInf ? 0.f : p * vs[j][i];    // (the scale of a slot that this query does not see may be NaN)
          most_w = fmaxf(most_w, w[j][i]);
        }
      most_w = fmaxf(most_w, __shfl_xor(most_w, 16, 64));
      most_w = fmaxf(most_w, __shfl_xor(most_w, 32, 64));
      const int top_new = max(top[t], most_w > 0.f ? __builtin_amdgcn_frexp_expf(most_w) : -300);
      const float alpha = __builtin_amdgcn_exp2f(m[t] - base);
      l[t] = fmaf(l[t], alpha, sum);
      if (__any(top_new != top[t] || m_new != m[t])) {
        const float beta = __builtin_amdgcn_ldexpf(alpha, top[t] - top_new);
#pragma unroll
        for (int i = 0; i < DT; ++i) o[t][i] *= beta;
      }
      m[t] = m_new;
      top[t] = top_new;
#pragma unroll
      for (int j = 0; j < kStepTiles; ++j)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const float x = __builtin_amdgcn_ldexpf(w[j][i], kTop - top_new);
          const _Float16 h = (_Float16)x;
          hi[t][j / 2][j % 2 * 4 + i] = h;
          lo[t][j / 2][j % 2 * 4 + i] = (_Float16)(x - (float)h);
        }
    }
#pragma unroll
    for (int j = 0; j < kStepTiles; j += 2)
#pragma unroll
      for (int c = 0; c < CH; ++c)
#pragma unroll
        for (int u = 0; u < E / 4; ++u) {
          const f16x8 vf = v_halves(word(vc[j][c], u), word(vc[j + 1][c], u));
#pragma unroll
          for (int t = 0; t < QT; ++t) {
            f32x4& acc = o[t][c * (E / 4) + u];
            acc = __builtin_amdgcn_mfma_f32_16x16x32_f16(vf, hi[t][j / 2], acc, 0, 0, 0);
            acc = __builtin_amdgcn_mfma_f32_16x16x32_f16(vf, lo[t][j / 2], acc, 0, 0, 0);
          }
        }
  }
#pragma unroll
  for (int t = 0; t < QT; ++t) {
    l[t] += __shfl_xor(l[t], 16, 64);
    l[t] += __shfl_xor(l[t], 32, 64);
    if (grp == 0) { m_sh[wave][16 * t + col] = m[t]; l_sh[wave][16 * t + col] = l[t]; }
  }
  // the waves' partial results, 16 threads to a query
  constexpr int PER = D / 16;
  const int c = threadIdx.x / 16, dim0 = threadIdx.x % 16 * PER;
#pragma unroll
  for (int t = 0; t < QT; ++t) {
    if (t) __syncthreads();
#pragma unroll
    for (int i = 0; i < DT; ++i)
#pragma unroll
      for (int e = 0; e < 4; ++e) o_sh[wave][col][16 * i + 4 * grp + e] = __builtin_amdgcn_ldexpf(o[t][i][e], top[t] - kTop);
    __syncthreads();
    const int f = first + 16 * t + c;
    if (f >= queries) continue;
    float best = kNegInf, sum = 0.f, acc[PER] = {};
#pragma unroll
    for (int w = 0; w < kWaves; ++w) best = fmaxf(best, m_sh[w][16 * t + c]);
#pragma unroll
    for (int w = 0; w < kWaves; ++w) {
      const float mw = m_sh[w][16 * t + c], lw = l_sh[w][16 * t + c];
      const float part = mw == kNegInf && lw == 0.f ? 0.f : __builtin_amdgcn_exp2f(mw - best);
      sum = fmaf(part, lw, sum);
#pragma unroll
      for (int e = 0; e < PER; ++e) acc[e] = fmaf(part, o_sh[w][c][dim0 + e], acc[e]);
    }
    const int r = row0 + f / a.share, h = kvh * a.share + f % a.share;
    if (a.part) {
      const size_t rh = (size_t)r * a.n_heads + h;
#pragma unroll
      for (int e = 0; e < PER; ++e) a.sums(rh, blockIdx.z, D)[dim0 + e] = acc[e];
      if (dim0 == 0) *a.stats(rh, blockIdx.z, D) = make_float2(best, sum);
    } else {
#pragma unroll
      for (int e = 0; e < PER; ++e)
        st<T>::stv((T*)a.out + (size_t)r * a.out_stride + (size_t)h * D + dim0 + e, sum == 0.f ? 0.f : acc[e] / sum);
    }
  }
}

// The chunks' partial results of one row and head, joined by one wave in the chunks' order.
template <typename T, int D>
__global__ __launch_bounds__(256) void kv8_join_kernel(Kv8View kv, Kv8Attn a) {
  constexpr int NP = D > 64 ? D / 64 : 1;
  const int lane = threadIdx.x & 63, r = blockIdx.x, h = blockIdx.y * 4 + (threadIdx.x >> 6);
  if (h >= a.n_heads) return;
  const int b = kv8_sequence_of(a.cu_rows, kv.batch, r);
  if (b >= kv.batch) return;
  const int n = (a.limit_of(b, r, kv.slots()) + a.chunk - 1) / a.chunk;
  const size_t rh = (size_t)r * a.n_heads + h;
  float top = kNegInf;
  for (int c = lane; c < n; c += 64) top = fmaxf(top, a.stats(rh, c, D)->x);
  top = wave_max(top);
  float sum = 0.f, acc[NP] = {};
  for (int c0 = 0; c0 < n; c0 += 64) {
    float2 ml = make_float2(kNegInf, 0.f);
    if (c0 + lane < n) ml = *a.stats(rh, c0 + lane, D);
    const float w = ml.x == kNegInf && ml.y == 0.f ? 0.f : __builtin_amdgcn_exp2f(ml.x - top);
    sum += w * ml.y;
    for (int c = 0; c < min(64, n - c0); ++c) {
      const float wc = __shfl(w, c, 64);
      if (lane * NP < D) {
#pragma unroll
        for (int e = 0; e < NP; ++e) acc[e] += wc * a.sums(rh, c0 + c, D)[lane * NP + e];
      }
    }
  }
  sum = wave_sum(sum);
  if (lane * NP < D) {
#pragma unroll
    for (int e = 0; e < NP; ++e)
      st<T>::stv((T*)a.out + (size_t)r * a.out_stride + (size_t)h * D + lane * NP + e, sum == 0.f ? 0.f : acc[e] / sum);
  }
}

struct Kv8Plan { int qt, tiles, chunk, chunks; };

// How a call is cut: queries per workgroup by how many a sequence has on average, slots per workgroup so that a few thousand
// workgroups share the work.  Bounds only: the same for every call with the same bounds.
Kv8Plan kv8_plan(const Kv8View& kv, int d, int dtype, int n_heads, int m_upper, int len_upper) {
  Kv8Plan p;
  const int64_t queries = (int64_t)m_upper * (n_heads / kv.heads);
  p.qt = queries > 16 * (int64_t)kv.batch && !(d == 256 && dtype == SL_F32) ? 2 : 1;
  // every sequence rounds its queries up to a tile, and a tile holds one at least
  const int64_t most = queries / (16 * p.qt) + kv.batch;
  p.tiles = (int)(queries < most ? queries : most);
  const int pieces = sl_cdiv(len_upper < 1 ? 1 : len_upper, kWaves * kStep);
  int want = (int)(4096 / ((int64_t)p.tiles * kv.heads));
  want = want < 1 ? 1 : want > pieces ? pieces : want;
  p.chunk = sl_cdiv(pieces, want) * kWaves * kStep;
  p.chunks = sl_cdiv(len_upper < 1 ? 1 : len_upper, p.chunk);
  return p;
}

}  // namespace

size_t slk_kv8_attention_bytes(const Kv8View& kv, int d, int n_heads, int m_upper, int len_upper) {
  if (m_upper == 0) return 256;
  int chunks = 1;                                         // of either type of queries
  for (int dtype : {SL_F32, SL_BF16}) chunks = max(chunks, kv8_plan(kv, d, dtype, n_heads, m_upper, len_upper).chunks);
  return chunks == 1 ? 256 : sl_align_up((size_t)m_upper * n_heads * chunks * (d + 2) * sizeof(float), 256);
}

int slk_kv8_attention(hipStream_t s, const Kv8View& kv, int d, int dtype, const void* q, int64_t q_stride, int n_heads,
                      const int32_t* cu_rows, const int32_t* seq_len, const int32_t* row_len, int m_upper, int len_upper, float scale,
                      void* out, int64_t out_stride, void* workspace) {
  const Kv8Plan p = kv8_plan(kv, d, dtype, n_heads, m_upper, len_upper);
  const Kv8Attn a{q, out, p.chunks == 1 ? nullptr : (float*)workspace, cu_rows, seq_len, row_len, q_stride, out_stride, n_heads,
                  n_heads / kv.heads, m_upper, len_upper, p.chunk, p.chunks, (float)((double)scale * 1.4426950408889634)};
  const dim3 grid(p.tiles, kv.heads, p.chunks), join(m_upper, sl_cdiv(n_heads, 4));
#define KV8_CALL(T, D)                                                                                           \
  do {                                                                                                           \
    constexpr int kMost = sizeof(T) == 4 && D == 256 ? 1 : 2;                                                    \
    if (p.qt == 1) hipLaunchKernelGGL((kv8_attention_kernel<T, D, 1>), grid, dim3(64 * kWaves), 0, s, kv, a);    \
    else hipLaunchKernelGGL((kv8_attention_kernel<T, D, kMost>), grid, dim3(64 * kWaves), 0, s, kv, a);          \
    if (a.part) hipLaunchKernelGGL((kv8_join_kernel<T, D>), join, dim3(256), 0, s, kv, a);                       \
  } while (0)
#define KV8_BY_HEAD(T)                 \
  switch (d) {                         \
    case 32: KV8_CALL(T, 32); break;   \
    case 64: KV8_CALL(T, 64); break;   \
    case 128: KV8_CALL(T, 128); break; \
    case 256: KV8_CALL(T, 256); break; \
    default: return SL_EINVAL;         \
  }
  if (dtype == SL_BF16) { KV8_BY_HEAD(bf16_t) } else { KV8_BY_HEAD(float) }
#undef KV8_BY_HEAD
#undef KV8_CALL
  SL_LAUNCH_CHECK();
  return SL_OK;
}
