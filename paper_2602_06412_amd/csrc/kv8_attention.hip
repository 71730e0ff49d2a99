// Attention of a few rows per sequence over the paged 8-bit cache.
//
//   o[r, h] = sum_{p < L_r} P_p V[p],  P = softmax(scale q[r, h] . K[p]),  L_r = min(seq_len, row_len[r], the table's slots)
//
// The rows of a sequence times the query heads that share a K/V head are one list of queries; 16 of them are a tile, the columns
// of the matrix products: S^T = K Q^T (16 slots x 16 queries) and O^T = V^T P^T.  S^T leaves in lane l the scores of query l % 16
// and slots 4 (l / 16) .. + 3 of a tile, which is the operand the second product wants, so probabilities never leave registers.
//
// Precision: codes are integers below 128, exact in bf16.  A bf16 query is exact, an fp32 query goes in as three bf16 parts
// (24 bits).  K's scale multiplies the fp32 score, V's scale the probability, and that product goes into the second multiplication
// as two bf16 parts (16 bits, for bf16 results) or three (fp32 results); one part would leave 8 bits, an error of half a step of
// the result even where one slot takes all the weight.  Scores, maximum, sum and output accumulate in fp32.
#include "kv8.h"

namespace {

typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
constexpr float kNegInf = -__builtin_inff();

// 8 codes (8 bytes) as bf16
__device__ inline bf16x8 codes_to_bf16(uint32_t lo, uint32_t hi) {
  bf16x8 r;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    r[i] = (bf16_t)(float)(signed char)(lo >> (8 * i));
    r[4 + i] = (bf16_t)(float)(signed char)(hi >> (8 * i));
  }
  return r;
}

// x as NP bf16 numbers that add up to it, to 8 NP bits
template <int NP>
__device__ inline void split_bf16(const float (&x)[8], bf16x8 (&part)[NP]) {
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    float rest = x[e];
#pragma unroll
    for (int p = 0; p < NP; ++p) {
      part[p][e] = (bf16_t)rest;
      rest -= (float)part[p][e];
    }
  }
}

template <typename T> struct Parts { static constexpr int q = 1, p = 2; };
template <> struct Parts<float> { static constexpr int q = 3, p = 3; };

template <int E> struct Piece;
template <> struct Piece<8> { typedef uint2 type; };
template <> struct Piece<16> { typedef uint4 type; };
template <int E>
__device__ inline void words(const typename Piece<E>::type& v, uint32_t (&w)[E / 4]) {
  w[0] = v.x; w[1] = v.y;
  if constexpr (E == 16) { w[2] = v.z; w[3] = v.w; }
}

struct Kv8Attn {
  const void* q;
  void* out;
  const int32_t *cu_rows, *seq_len, *row_len;
  int64_t q_stride, out_stride;
  int n_heads, share, m_upper, len_upper;                           // share = query heads per K/V head
  float scale_log2;                                       // scale * log2(e): probabilities are powers of two
};

// Tile `t` of queries -> its sequence and its first query there; false past the last tile.
__device__ inline bool kv8_tile_of(const Kv8Attn& a, int batch, int t, int& b, int& first, int& row0, int& rows) {
  for (b = 0; b < batch; ++b) {
    row0 = min(max(a.cu_rows[b], 0), a.m_upper);
    rows = min(max(a.cu_rows[b + 1] - row0, 0), a.m_upper - row0);
    const int tiles = (rows * a.share + 15) / 16;
    if (t < tiles) { first = t * 16; return true; }
    t -= tiles;
  }
  return false;
}

constexpr int kWaves = 4, kStepTiles = 4;                 // a wave takes 64 slots a step

template <typename T, int D>
__global__ __launch_bounds__(64 * kWaves) void kv8_attention_kernel(Kv8View kv, Kv8Attn a) {
  using Tile = Kv8Tile<D>;
  constexpr int E = Tile::E, CH = Tile::CH, NQ = Parts<T>::q, NP = Parts<T>::p, DT = D / 16;
  __shared__ float o_sh[kWaves][16][D + 4];
  __shared__ float m_sh[kWaves][16], l_sh[kWaves][16];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, col = lane & 15, grp = lane >> 4;
  const int kvh = blockIdx.y;
  int b, first, row0, rows;
  if (!kv8_tile_of(a, kv.batch, blockIdx.x, b, first, row0, rows)) return;
  const int f = first + col;
  const bool live = f < rows * a.share;
  const int r = row0 + (live ? f / a.share : 0), h = kvh * a.share + (live ? f % a.share : 0);
  int limit = min(min(max(a.seq_len[b], 0), kv.slots()), a.len_upper);
  if (a.row_len) limit = min(limit, a.row_len[r]);
  if (!live) limit = 0;
  int most = limit;
#pragma unroll
  for (int o = 8; o > 0; o >>= 1) most = max(most, __shfl_xor(most, o, 64));

  bf16x8 qf[CH * E / 8][NQ];
  const T* qr = (const T*)a.q + (size_t)r * a.q_stride + (size_t)h * D;
#pragma unroll
  for (int c = 0; c < CH; ++c)
#pragma unroll
    for (int t = 0; t < E / 8; ++t) {
      float x[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) x[e] = st<T>::ld(qr + c * 4 * E + grp * E + t * 8 + e);
      split_bf16<NQ>(x, qf[c * (E / 8) + t]);
    }

  f32x4 o[DT] = {};
  float m = kNegInf, l = 0.f;                             // of this wave's slots; l of this lane's
  for (int s0 = wave * 16 * kStepTiles; s0 < most; s0 += kWaves * 16 * kStepTiles) {
    const unsigned char* tile[kStepTiles];
    bool ok[kStepTiles];
#pragma unroll
    for (int t = 0; t < kStepTiles; ++t) {
      const int slot = s0 + 16 * t;
      const int page = slot < most ? kv.table[(size_t)b * kv.max_pages + (slot >> kv.page_shift)] : -1;
      ok[t] = page >= 0 && page < kv.n_pages;
      tile[t] = kv.tile<D>(ok[t] ? page : 0, kvh, slot);
    }
    float s[kStepTiles][4], vs[kStepTiles][4], top = kNegInf;
#pragma unroll
    for (int t = 0; t < kStepTiles; ++t) {
      f32x4 acc = {};
#pragma unroll
      for (int c = 0; c < CH; ++c) {
        uint32_t w[E / 4];
        words<E>(reinterpret_cast<const typename Piece<E>::type*>(tile[t])[c * 64 + lane], w);
#pragma unroll
        for (int u = 0; u < E / 8; ++u) {
          const bf16x8 kf = codes_to_bf16(w[2 * u], w[2 * u + 1]);
#pragma unroll
          for (int p = 0; p < NQ; ++p) acc = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf, qf[c * (E / 8) + u][p], acc, 0, 0, 0);
        }
      }
      const f32x4 ks = *reinterpret_cast<const f32x4*>(tile[t] + Tile::kKs + 16 * grp);
      const f32x4 sc = *reinterpret_cast<const f32x4*>(tile[t] + Tile::kVs + 16 * grp);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const bool seen = ok[t] && s0 + 16 * t + 4 * grp + i < limit;
        s[t][i] = seen ? acc[i] * (ks[i] * a.scale_log2) : kNegInf;
        vs[t][i] = seen ? sc[i] : 0.f;
        top = fmaxf(top, s[t][i]);
      }
    }
    top = fmaxf(top, __shfl_xor(top, 16, 64));
    top = fmaxf(top, __shfl_xor(top, 32, 64));
    const float m_new = fmaxf(m, top), m_use = m_new == kNegInf ? 0.f : m_new;
    const float alpha = exp2f(m - m_use);
    m = m_new;
    l *= alpha;
#pragma unroll
    for (int i = 0; i < DT; ++i) o[i] *= alpha;
#pragma unroll
    for (int t = 0; t < kStepTiles; t += 2) {
      float w[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const float p = exp2f(s[t + i / 4][i % 4] - m_use);
        l += p;
        w[i] = p * vs[t + i / 4][i % 4];
      }
      bf16x8 pf[NP];
      split_bf16<NP>(w, pf);
#pragma unroll
      for (int c = 0; c < CH; ++c) {
        uint32_t w0[E / 4], w1[E / 4];
        words<E>(reinterpret_cast<const typename Piece<E>::type*>(tile[t] + Tile::kV)[c * 64 + lane], w0);
        words<E>(reinterpret_cast<const typename Piece<E>::type*>(tile[t + 1] + Tile::kV)[c * 64 + lane], w1);
#pragma unroll
        for (int u = 0; u < E / 4; ++u) {
          const bf16x8 vf = codes_to_bf16(w0[u], w1[u]);
#pragma unroll
          for (int p = 0; p < NP; ++p)
            o[c * (E / 4) + u] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vf, pf[p], o[c * (E / 4) + u], 0, 0, 0);
        }
      }
    }
  }
  l += __shfl_xor(l, 16, 64);
  l += __shfl_xor(l, 32, 64);
  if (grp == 0) { m_sh[wave][col] = m; l_sh[wave][col] = l; }
#pragma unroll
  for (int i = 0; i < DT; ++i) *reinterpret_cast<f32x4*>(&o_sh[wave][col][16 * i + 4 * grp]) = o[i];
  __syncthreads();
  for (int i = threadIdx.x; i < 16 * D; i += 64 * kWaves) {
    const int c = i / D, dim = i % D, fq = first + c;
    if (fq >= rows * a.share) continue;
    float top = kNegInf, sum = 0.f, acc = 0.f;
#pragma unroll
    for (int w = 0; w < kWaves; ++w) top = fmaxf(top, m_sh[w][c]);
#pragma unroll
    for (int w = 0; w < kWaves; ++w) {
      const float f2 = m_sh[w][c] == kNegInf && l_sh[w][c] == 0.f ? 0.f : exp2f(m_sh[w][c] - top);
      sum += f2 * l_sh[w][c];
      acc += f2 * o_sh[w][c][dim];
    }
    T* dst = (T*)a.out + (size_t)(row0 + fq / a.share) * a.out_stride + (size_t)(kvh * a.share + fq % a.share) * D + dim;
    st<T>::stv(dst, sum == 0.f ? 0.f : acc / sum);
  }
}

}  // namespace

size_t slk_kv8_attention_bytes(const Kv8View&, int, int, int, int) { return 256; }

int slk_kv8_attention(hipStream_t s, const Kv8View& kv, int d, int dtype, const void* q, int64_t q_stride, int n_heads,
                      const int32_t* cu_rows, const int32_t* seq_len, const int32_t* row_len, int m_upper, int len_upper, float scale,
                      void* out, int64_t out_stride, void* workspace) {
  Kv8Attn a{q, out, cu_rows, seq_len, row_len, q_stride, out_stride, n_heads, n_heads / kv.heads, m_upper, len_upper,
            (float)((double)scale * 1.4426950408889634)};
  // every sequence rounds its queries up to a tile of 16, and a tile holds one at least
  const int64_t queries = (int64_t)m_upper * a.share;
  const int64_t tiles = queries < queries / 16 + kv.batch ? queries : queries / 16 + kv.batch;
  const dim3 grid((unsigned)tiles, kv.heads);
#define KV8_CALL(T, D) hipLaunchKernelGGL((kv8_attention_kernel<T, D>), grid, dim3(64 * kWaves), 0, s, kv, a)
#define KV8_BY_HEAD(T)               \
  switch (d) {                       \
    case 32: KV8_CALL(T, 32); break; \
    case 64: KV8_CALL(T, 64); break; \
    case 128: KV8_CALL(T, 128); break; \
    case 256: KV8_CALL(T, 256); break; \
    default: return SL_EINVAL;       \
  }
  if (dtype == SL_BF16) { KV8_BY_HEAD(bf16_t) } else { KV8_BY_HEAD(float) }
#undef KV8_BY_HEAD
#undef KV8_CALL
  SL_LAUNCH_CHECK();
  return SL_OK;
}
