// Attention of a few rows per sequence over the paged 8-bit cache.
//
//   o[r, h] = sum_{p < L_r} P_p V[p],  P = softmax(scale q[r, h] . K[p]),  L_r = min(seq_len, row_len[r], the table's slots)
//
// The rows of a sequence times the query heads that share a K/V head are one list of queries; 16 of them are a tile, the columns
// of the matrix products: S^T = K Q^T (16 slots x 16 queries) and O^T = V^T P^T.  S^T leaves in lane l the scores of query l % 16
// and slots 4 (l / 16) .. + 3 of a tile, which is the operand the second product wants, so probabilities never leave registers.
//
// Unpacking codes is what such a kernel would spend its instructions on: with K and V converted to bf16, 1.5 a number, the largest
// case took 291 us, 180 as follows (its loads alone 170 at that stage).  For bf16 queries and results:
//   K is not unpacked: the product is one of 8-bit integers, the query being a fixed-point number of three signed bytes,
//     q = 2^(e - 22) (65536 a + 256 b + c), 2^(e-1) <= max|q| < 2^e.  Of 8 significant bits none is lost down to 2^-15 of the head's
//     largest number; what lies below loses the bits under 2^-23 of it.
//     Each byte's product starts from the integer 0x4B400000, whose bits are the float 1.5 * 2^23, so that the result, below 2^22
//     for 256 dimensions, is that float plus itself: one subtraction instead of a conversion.
//   V becomes half precision in two operations a pair: 0x6400 + (code + 128) are the bits of the half 1024 + code + 128.
//   A probability times V's scale goes in as two halves (22 bits), scaled by a power of two per query so that the largest seen lies
//     below 2^14: what is 2^38 times smaller than it is dropped.  One half would leave 11 bits, against a result rounded to 8.
//     "The largest" is what is left of it: as the maximum rises, weights seen before shrink, and the power of two follows
//     (kept from them as they were, it dropped a slot that held all the weight where earlier values were 10^12 larger).
// For fp32 neither will do: a query's small numbers beside a large one, and a slot's small share of a dimension where the largest
// slot holds nothing, have 24 bits of their own.  There K and V are converted to bf16, exactly, and a query's number and a weight go in
// as three bf16 each, which hold all 24 bits at any size; products are exact, sums fp32.
// Scores, maximum, sum and output accumulate in fp32.
#include "kv8.h"
#include <type_traits>

namespace {

typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef _Float16 f16x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x8 __attribute__((ext_vector_type(8)));
typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef float f32x4 __attribute__((ext_vector_type(4)));
constexpr float kNegInf = -__builtin_inff();
constexpr int kMagicBits = 0x4B400000;
constexpr float kMagic = 12582912.f;                      // its float
constexpr int kTop = 14;                                  // probabilities lie below 2^kTop

// a lane's share of an 8-bit operand: 16 bytes (8 with d = 32)
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
template <int E> struct Piece;
template <> struct Piece<8> {
  typedef u32x2 type;
  static __device__ i32x4 mfma(u32x2 a, u32x2 b, i32x4 c) {
    return __builtin_amdgcn_mfma_i32_16x16x32_i8(__builtin_bit_cast(long, a), __builtin_bit_cast(long, b), c, 0, 0, 0);
  }
};
template <> struct Piece<16> {
  typedef u32x4 type;
  static __device__ i32x4 mfma(u32x4 a, u32x4 b, i32x4 c) {
    return __builtin_amdgcn_mfma_i32_16x16x64_i8(__builtin_bit_cast(i32x4, a), __builtin_bit_cast(i32x4, b), c, 0, 0, 0);
  }
};
// (loads of codes that no other workgroup asks for go past the caches' replacement: the loads alone, 830 MB of twelve sequences of like
// length, 133 us instead of 153)
template <bool ONCE, typename P>
__device__ inline P ask(const P* p) {
  return ONCE ? __builtin_nontemporal_load(p) : *p;
}

// the other lanes' value, 16 / 32 lanes away, taken into a maximum or a sum without going through LDS
template <typename F>
__device__ inline float across_groups(float x, F f) {
  auto a = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  x = f(__uint_as_float(a[0]), __uint_as_float(a[1]));
  auto b = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return f(__uint_as_float(b[0]), __uint_as_float(b[1]));
}
__device__ inline float max_across(float x) { return across_groups(x, [](float a, float b) { return fmaxf(a, b); }); }
__device__ inline float sum_across(float x) { return across_groups(x, [](float a, float b) { return a + b; }); }

// V's codes (each + 128) of 4 slots of one tile and 4 of the next, as halves
__device__ inline f16x8 v_halves(uint32_t a, uint32_t b) {
  const f16x2 off = {(_Float16)1152.f, (_Float16)1152.f};
  const f16x2 r0 = __builtin_bit_cast(f16x2, __builtin_amdgcn_perm(0x64646464u, a, 0x04010400u)) - off;
  const f16x2 r1 = __builtin_bit_cast(f16x2, __builtin_amdgcn_perm(0x64646464u, a, 0x04030402u)) - off;
  const f16x2 r2 = __builtin_bit_cast(f16x2, __builtin_amdgcn_perm(0x64646464u, b, 0x04010400u)) - off;
  const f16x2 r3 = __builtin_bit_cast(f16x2, __builtin_amdgcn_perm(0x64646464u, b, 0x04030402u)) - off;
  return f16x8{r0[0], r0[1], r1[0], r1[1], r2[0], r2[1], r3[0], r3[1]};
}

// eight codes, signed bytes, as bf16
__device__ inline bf16x8 codes_bf16(uint32_t a, uint32_t b) {
  bf16x8 r;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    r[i] = (__bf16)(float)(signed char)(a >> (8 * i));
    r[4 + i] = (__bf16)(float)(signed char)(b >> (8 * i));
  }
  return r;
}

// a number as three bf16, all of its 24 bits
__device__ inline void three_bf16(float x, __bf16& h, __bf16& m, __bf16& l) {
  h = (__bf16)x;
  const float r = x - (float)h;
  m = (__bf16)r;
  l = (__bf16)(r - (float)m);
}

// Four numbers of at most 2^22 in magnitude as three signed bytes each, base 256: byte p of all four in w[p].  A number plus
// 0x808080 has unsigned bytes, each 128 more than the signed ones; flipping their top bits takes the 128 off again.
__device__ inline void signed_bytes(const float (&x)[4], uint32_t (&w)[3]) {
  uint32_t j[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) j[i] = ((uint32_t)(int)rintf(x[i]) + 0x808080u) ^ 0x808080u;
  const uint32_t low01 = __builtin_amdgcn_perm(j[1], j[0], 0x05040100u), low23 = __builtin_amdgcn_perm(j[3], j[2], 0x05040100u);
  const uint32_t high = __builtin_amdgcn_perm(j[1], j[0], 0x0c0c0602u);
  w[0] = __builtin_amdgcn_perm(__builtin_amdgcn_perm(j[3], j[2], 0x0c0c0602u), high, 0x05040100u);
  w[1] = __builtin_amdgcn_perm(low23, low01, 0x07050301u);
  w[2] = __builtin_amdgcn_perm(low23, low01, 0x06040200u);
}

constexpr int kResident = 3;                              // workgroups of a CU that registers let run at once (2 with d = 256)
// Pieces wanted, in rounds of what runs at once.  us at 1, 2, 3, 4 rounds (heads of 128 but where stated): one row in each of 8 ragged
// sequences 60, 53, 57, 57; 16 long ragged ones 163, 157, 151, 155; 12 long ones of like length 135, 136, 141, 141; 16 rows of 64
// heads over 8 97, 78, 79, 101; 64 rows of 2048 slots 22.7, 22.7, 23.5, 23.9; ragged ones of 256 a head 37, 43, 43, 43.  One longer
// round ends when its last workgroup does, many short ones start often; two are never far from the best.
constexpr int kRounds = 2;
// Units of a piece, at least; up to 512 slots a segment is one piece and the second launch falls away.  us at 1, 2, 4, 8: 64 rows of
// 2048 slots 25.9, 26.0, 22.7, 25.1; one row of 4096 slots 18.5, 16.8, 17.7, 23.3; one row in each of 8 ragged sequences 53, 53, 53, 58.
constexpr int kLeast = 4;

// A segment is a tile of queries with one K/V head: sequence by sequence, head by head, tile by tile.  Segments are cut into pieces of
// nearly equal length, one for each workgroup, so long that there are about a.pieces of them however ragged the lengths are
// (every workgroup works that out from the row counts and lengths).  Of a segment in several pieces each leaves a partial result,
// and a second launch joins those.
struct Kv8Attn {
  const void* q;
  void* out;
  float* part;                                            // partial results
  const int32_t *cu_rows, *seq_len, *row_len;
  int64_t q_stride, out_stride;
  int n_heads, share, m_upper, len_upper;                 // share = query heads per K/V head
  int unit, pieces;                                       // slots a length is counted in; pieces wanted
  float scale_log2;                                       // scale * log2(e): probabilities are powers of two
  // partial p: results [16 queries][d], each a mean over the slots of its piece; behind all of them maximum and sum.  Fewer than
  // 2 pieces: a segment of n units in k > 1 pieces has k < n / c + 1 < 2 n / c, where all n together are at most c pieces
  __device__ float* sums(int p, int col, int d) const { return part + ((size_t)p * 16 + col) * d; }
  __device__ float2* stats(int p, int col, int d) const { return reinterpret_cast<float2*>(part + (size_t)pieces * 32 * d) + (size_t)p * 16 + col; }
};

struct Kv8Sequence { int row0, rows, len, tiles, units; };      // tiles of its queries, units of its length (one at least)

__device__ inline Kv8Sequence kv8_sequence(const Kv8View& kv, const Kv8Attn& a, int b) {
  Kv8Sequence s;
  s.row0 = min(max(a.cu_rows[b], 0), a.m_upper);
  s.rows = min(max(a.cu_rows[b + 1] - s.row0, 0), a.m_upper - s.row0);
  s.len = min(min(max(a.seq_len[b], 0), kv.slots()), a.len_upper);
  s.tiles = (s.rows * a.share + 15) / 16;
  s.units = max((s.len + a.unit - 1) / a.unit, 1);
  return s;
}

__device__ inline int wave_sum_int(int x) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) x += __shfl_xor(x, o, 64);
  return __builtin_amdgcn_readfirstlane(x);
}

// Units of a piece, at most, from all segments' units; a wave asks for 64 sequences at a time and keeps the first 64.
__device__ inline int kv8_piece(const Kv8View& kv, const Kv8Attn& a, Kv8Sequence& mine) {
  const int lane = threadIdx.x & 63;
  int all = 0;
  for (int b = lane; b < kv.batch; b += 64) {
    const Kv8Sequence s = kv8_sequence(kv, a, b);
    if (b == lane) mine = s;
    all += s.tiles * kv.heads * s.units;
  }
  all = wave_sum_int(all);
  return max((all + a.pieces - 1) / a.pieces, kLeast);
}

constexpr int kWaves = 4, ST = 2, kStep = 16 * ST;        // a wave takes 32 slots a step
constexpr int kUnit = kWaves * kStep, kPages = 64 / ST;

// slots [from, end) of one segment: K/V head `kvh`, the 16 queries from `first` on of sequence b
template <typename T, int D, bool ONCE>
struct Kv8Segment {
  using Tile = Kv8Tile<D>;
  static constexpr int E = Tile::E, CH = Tile::CH, DT = D / 16;
  static constexpr bool kFull = sizeof(T) == 4;           // all 24 bits of queries and weights
  typedef typename Piece<E>::type piece;
  typedef float Sums[kWaves][16][D + 4];
  typedef uint32_t Bytes[CH][3][64][E / 4];               // the queries' bytes
  typedef uint32_t Parts[CH][E / 8][3][64][4];            // the queries' bf16, eight a lane
  struct Apart { Sums o; __attribute__((aligned(16))) Bytes q; };
  struct OneAfterTheOther { union { Sums o; __attribute__((aligned(16))) Parts q; }; };
  struct Shared : std::conditional<kFull, OneAfterTheOther, Apart>::type {
    float m[kWaves][16], l[kWaves][16];
  };
  static __device__ __forceinline__ void run(const Kv8View& kv, const Kv8Attn& a, Shared& sh, int b, const Kv8Sequence& seq, int kvh, int first,
                                             int from, int end, int part);
};

template <typename T, int D, bool ONCE>
__device__ __forceinline__ void Kv8Segment<T, D, ONCE>::run(const Kv8View& kv, const Kv8Attn& a, Shared& sh, int b, const Kv8Sequence& seq, int kvh,
                                                            int first, int from, int end, int part) {
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), col = lane & 15, grp = lane >> 4;
  const int queries = seq.rows * a.share, row0 = seq.row0, len = seq.len;
  // the codes of a step: K's are asked for one step ahead once the scores are done, V's once the sums are
  int pages = 0;                                          // lane i: the page of tile i % ST of the (i / ST)-th of kPages steps
  auto ask_pages = [&](int s0) {
    const int slot = s0 + (lane / ST) * (kWaves * kStep) + lane % ST * 16;
    pages = slot < end ? kv.table[(size_t)b * kv.max_pages + (slot >> kv.page_shift)] : -1;
  };
  const unsigned char* tile[ST];
  int ok = 0;                                             // bit j: tile j is on a page
  piece kc[ST][CH], vc[ST][CH];
  f32x4 ks[ST], vs[ST];
  auto ask_k = [&](int s0, int step) {
    ok = 0;
#pragma unroll
    for (int j = 0; j < ST; ++j) {
      const int page = __builtin_amdgcn_readlane(pages, step % kPages * ST + j);
      const bool there = page >= 0 && page < kv.n_pages;
      ok |= there << j;
      tile[j] = kv.tile<D>(there ? page : 0, kvh, s0 + 16 * j);
#pragma unroll
      for (int c = 0; c < CH; ++c) kc[j][c] = ask<ONCE>(reinterpret_cast<const piece*>(tile[j]) + c * 64 + lane);
      ks[j] = *reinterpret_cast<const f32x4*>(tile[j] + Tile::kKs + 16 * grp);
    }
  };
  auto ask_v = [&]() {
#pragma unroll
    for (int j = 0; j < ST; ++j) {
      vs[j] = *reinterpret_cast<const f32x4*>(tile[j] + Tile::kVs + 16 * grp);
#pragma unroll
      for (int c = 0; c < CH; ++c) vc[j][c] = ask<ONCE>(reinterpret_cast<const piece*>(tile[j] + Tile::kV) + c * 64 + lane);
    }
  };
  int s0 = from + wave * kStep;
  ask_pages(s0);

  const int f = first + col;
  const bool live = f < queries;
  constexpr int QW = E * sizeof(T) / 16;                  // 16-byte words of this lane's share of a chunk
  u32x4 x[CH][QW];
  int limit = 0;
  {
    const int r = row0 + (live ? f / a.share : 0), h = kvh * a.share + (live ? f % a.share : 0);
    if (live) limit = a.row_len ? min(len, a.row_len[r]) : len;
    const T* qr = (const T*)a.q + (size_t)r * a.q_stride + (size_t)h * D;
#pragma unroll
    for (int c = 0; c < CH; ++c)
#pragma unroll
      for (int u = 0; u < QW; ++u) x[c][u] = reinterpret_cast<const u32x4*>(qr + c * 4 * E + grp * E)[u];
  }
  auto x_at = [&](int c, int u) {                         // number u of chunk c
    if constexpr (sizeof(T) == 2) return __uint_as_float(u % 2 ? x[c][u / 8][u / 2 % 4] & 0xffff0000u : x[c][u / 8][u / 2 % 4] << 16);
    else return __uint_as_float(x[c][u / 4][u % 4]);
  };
  ask_k(s0, 0);                                           // (a wave without a step of its own asks for page 0: no branch)
  ask_v();
  // every wave knows its queries' exponents; the bytes are shared out among the waves
  uint32_t big = 0;
#pragma unroll
  for (int c = 0; c < CH; ++c)
#pragma unroll
    for (int u = 0; u < E; ++u) big = max(big, __float_as_uint(x_at(c, u)) & 0x7fffffffu);
  big = __float_as_uint(across_groups(__uint_as_float(big), [](float p, float q) {
    return __uint_as_float(max(__float_as_uint(p), __float_as_uint(q)));
  }));
  const bool finite = big < 0x7f800000u;
  const int qe = finite ? __builtin_amdgcn_frexp_expf(__uint_as_float(big)) : 0;
  if constexpr (kFull) {
#pragma unroll
    for (int c = 0; c < CH; ++c)
#pragma unroll
      for (int u = 0; u < E; u += 8)
        if ((c * E + u) / 8 % kWaves == wave) {
          bf16x8 w[3];
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            __bf16 h, mid, low;
            three_bf16(__builtin_amdgcn_ldexpf(x_at(c, u + i), 22 - qe), h, mid, low);
            w[0][i] = h;
            w[1][i] = mid;
            w[2][i] = low;
          }
#pragma unroll
          for (int p = 0; p < 3; ++p) *reinterpret_cast<bf16x8*>(sh.q[c][u / 8][p][lane]) = w[p];
        }
  } else {
#pragma unroll
    for (int c = 0; c < CH; ++c)
#pragma unroll
      for (int u = 0; u < E; u += 4)
        if ((c * E + u) / 4 % kWaves == wave) {
          float y[4];
          uint32_t w[3];
#pragma unroll
          for (int i = 0; i < 4; ++i) y[i] = __builtin_amdgcn_ldexpf(x_at(c, u + i), 22 - qe);
          signed_bytes(y, w);
#pragma unroll
          for (int p = 0; p < 3; ++p) sh.q[c][p][lane][u / 4] = w[p];
        }
  }
  // scores come out in powers of two: 2^(qe - 22), scale and log2(e) in one factor; NaN for a query that is not finite
  const float unit = finite ? __builtin_amdgcn_ldexpf(a.scale_log2, qe - 22) : __builtin_nanf("");
  const float unit_a = unit * 65536.f, unit_b = unit * 256.f, unit_c = -kMagic * unit;
  int most = limit, least = live ? limit : 1 << 30;
#pragma unroll
  for (int o = 8; o > 0; o >>= 1) {
    most = max(most, __shfl_xor(most, o, 64));
    least = min(least, __shfl_xor(least, o, 64));
  }
  most = __builtin_amdgcn_readfirstlane(most);
  least = __builtin_amdgcn_readfirstlane(least);
  end = min(most, end);
  __syncthreads();

  f32x4 o[DT] = {};
  float m = kNegInf, l = 0.f;                             // of this wave's slots; l of this lane's
  int top = -300;                                         // o is scaled by 2^(kTop - top)
  float peak = kNegInf;                                   // binary exponent of the largest weight so far, before a maximum is taken off
  for (int step = 0; s0 < end; ++step) {
    const int here = s0, ok_here = ok;
    const bool whole = here + kStep <= least && ok == (1 << ST) - 1;      // every query sees every slot of the step
    s0 += kWaves * kStep;
    float s[ST][4];
    if constexpr (kFull) {
      f32x4 acc[ST][3] = {};
#pragma unroll
      for (int c = 0; c < CH; ++c)
#pragma unroll
        for (int u = 0; u < E / 8; ++u) {
          __builtin_amdgcn_sched_barrier(0);
          bf16x8 k[ST];
#pragma unroll
          for (int j = 0; j < ST; ++j) k[j] = codes_bf16(kc[j][c][2 * u], kc[j][c][2 * u + 1]);
#pragma unroll
          for (int p = 0; p < 3; ++p) {
            const bf16x8 x = *reinterpret_cast<const bf16x8*>(sh.q[c][u][p][lane]);
#pragma unroll
            for (int j = 0; j < ST; ++j) acc[j][p] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(k[j], x, acc[j][p], 0, 0, 0);
          }
        }
#pragma unroll
      for (int j = 0; j < ST; ++j)
#pragma unroll
        for (int i = 0; i < 4; ++i) s[j][i] = ks[j][i] * unit * (acc[j][0][i] + (acc[j][1][i] + acc[j][2][i]));
    } else
#pragma unroll
    for (int j = 0; j < ST; ++j) {
      const i32x4 zero = {kMagicBits, kMagicBits, kMagicBits, kMagicBits};
      i32x4 acc[3] = {zero, zero, zero};
#pragma unroll
      for (int c = 0; c < CH; ++c)
#pragma unroll
        for (int p = 0; p < 3; ++p) acc[p] = Piece<E>::mfma(kc[j][c], *reinterpret_cast<const piece*>(sh.q[c][p][lane]), acc[p]);
#pragma unroll
      for (int i = 0; i < 4; ++i)
        s[j][i] = ks[j][i] * fmaf(__int_as_float(acc[0][i]) - kMagic, unit_a,
                                  fmaf(__int_as_float(acc[1][i]) - kMagic, unit_b, fmaf(__int_as_float(acc[2][i]), unit, unit_c)));
    }
    if (s0 < end) {
      if ((step + 1) % kPages == 0) ask_pages(s0);
      ask_k(s0, step + 1);
    }
    if (!whole) {                                         // (the scale of a slot that this query does not see may be NaN)
#pragma unroll
      for (int j = 0; j < ST; ++j)
#pragma unroll
        for (int i = 0; i < 4; ++i)
          if (!(ok_here >> j & 1) || here + 16 * j + 4 * grp + i >= limit) {
            s[j][i] = kNegInf;
            vs[j][i] = 0.f;
          }
    }
    float best = kNegInf;
#pragma unroll
    for (int j = 0; j < ST; ++j)
#pragma unroll
      for (int i = 0; i < 4; ++i) best = fmaxf(best, s[j][i]);
    const float m_new = fmaxf(m, max_across(best)), base = m_new == kNegInf ? 0.f : m_new;
    float sum = 0.f, most_w = 0.f;
#pragma unroll
    for (int j = 0; j < ST; ++j)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const float p = __builtin_amdgcn_exp2f(s[j][i] - base);
        sum += p;
        s[j][i] = p * vs[j][i];
        most_w = fmaxf(most_w, s[j][i]);
      }
    most_w = max_across(most_w);
    // weights below 2^now are added in this step, what is left of earlier ones lies below 2^(peak - base); scores far beyond fp32's
    // integers may miss the latter, which costs bits and no more: o's own scale is whatever top is
    const int now = most_w > 0.f ? __builtin_amdgcn_frexp_expf(most_w) : -300;
    peak = fmaxf(peak, most_w > 0.f ? base + (float)now : kNegInf);
    const int top_new = max(now, (int)fmaxf(ceilf(peak - base), -300.f));
    const float alpha = __builtin_amdgcn_exp2f(m - base);
    l = fmaf(l, alpha, sum);
    if (__any(top_new != top || m_new != m)) {
      const float beta = __builtin_amdgcn_ldexpf(alpha, top - top_new);
#pragma unroll
      for (int i = 0; i < DT; ++i) o[i] *= beta;
    }
    m = m_new;
    top = top_new;
    if constexpr (kFull) {
      bf16x8 w[3];
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        __bf16 h, mid, low;
        three_bf16(__builtin_amdgcn_ldexpf(s[i / 4][i % 4], kTop - top), h, mid, low);
        w[0][i] = h;
        w[1][i] = mid;
        w[2][i] = low;
      }
#pragma unroll
      for (int c = 0; c < CH; ++c)
#pragma unroll
        for (int u = 0; u < E / 4; ++u) {
          const bf16x8 v = codes_bf16(vc[0][c][u] ^ 0x80808080u, vc[1][c][u] ^ 0x80808080u);
          f32x4& ou = o[c * (E / 4) + u];
#pragma unroll
          for (int p = 0; p < 3; ++p) ou = __builtin_amdgcn_mfma_f32_16x16x32_bf16(v, w[p], ou, 0, 0, 0);
        }
    } else
#pragma unroll
    for (int j = 0; j < ST; j += 2) {
      f16x8 hi, lo;
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const float w = __builtin_amdgcn_ldexpf(s[j + i / 4][i % 4], kTop - top);
        hi[i] = (_Float16)w;
        lo[i] = (_Float16)(w - (float)hi[i]);
      }
#pragma unroll
      for (int c = 0; c < CH; ++c) {
#pragma unroll
        for (int u = 0; u < E / 4; u += 2) {
          const f16x8 v0 = v_halves(vc[j][c][u], vc[j + 1][c][u]), v1 = v_halves(vc[j][c][u + 1], vc[j + 1][c][u + 1]);
          f32x4 &o0 = o[c * (E / 4) + u], &o1 = o[c * (E / 4) + u + 1];
          o0 = __builtin_amdgcn_mfma_f32_16x16x32_f16(v0, hi, o0, 0, 0, 0);
          o1 = __builtin_amdgcn_mfma_f32_16x16x32_f16(v1, hi, o1, 0, 0, 0);
          o0 = __builtin_amdgcn_mfma_f32_16x16x32_f16(v0, lo, o0, 0, 0, 0);
          o1 = __builtin_amdgcn_mfma_f32_16x16x32_f16(v1, lo, o1, 0, 0, 0);
        }
      }
    }
    if (s0 < end) ask_v();
  }
  // The waves' partial results, 16 threads to a query.  A wave's sums are divided by its own sum of probabilities while they are still
  // in their power of two, and a piece's leave it divided by the piece's: a mean of finite values is finite, their sum need not be.
  // (Addresses from here on are worked out here: computed ahead of the loop, as the compiler would, they cost it 26 registers that
  // it does not have.)
  int tid = threadIdx.x, share = a.share;
  asm volatile("" : "+v"(tid), "+s"(share));
  l = sum_across(l);
  if constexpr (kFull) __syncthreads();                   // the sums lie where the queries were
  const int lane_e = tid & 63, col_e = lane_e & 15, grp_e = lane_e >> 4;
  if (grp_e == 0) { sh.m[wave][col_e] = m; sh.l[wave][col_e] = l; }
  const float per = l == 0.f ? 0.f : 1.f / l;
#pragma unroll
  for (int c = 0; c < CH; ++c)
#pragma unroll
    for (int e = 0; e < 4; ++e)
#pragma unroll
      for (int u = 0; u < E / 4; ++u)                     // dims (E / 4) row + u of the chunk
        sh.o[wave][col_e][c * 4 * E + E / 4 * (4 * grp_e + e) + u] = __builtin_amdgcn_ldexpf(o[c * (E / 4) + u][e] * per, top - kTop);
  __syncthreads();
  constexpr int PER = D / 16;
  const int c = tid / 16, dim0 = tid % 16 * PER, fq = first + c;
  if (fq >= queries) return;
  float best = kNegInf, sum = 0.f, part_w[kWaves], acc[PER] = {};
#pragma unroll
  for (int w = 0; w < kWaves; ++w) best = fmaxf(best, sh.m[w][c]);
#pragma unroll
  for (int w = 0; w < kWaves; ++w) {
    const float mw = sh.m[w][c], lw = sh.l[w][c];
    part_w[w] = mw == kNegInf && lw == 0.f ? 0.f : __builtin_amdgcn_exp2f(mw - best) * lw;
    sum += part_w[w];
  }
  const float inv = sum == 0.f ? 0.f : 1.f / sum;
#pragma unroll
  for (int w = 0; w < kWaves; ++w) {
    part_w[w] *= inv;
#pragma unroll
    for (int e = 0; e < PER; ++e) acc[e] = fmaf(part_w[w], sh.o[w][c][dim0 + e], acc[e]);
  }
  if (part >= 0) {
#pragma unroll
    for (int e = 0; e < PER; ++e) a.sums(part, c, D)[dim0 + e] = acc[e];
    if (dim0 == 0) *a.stats(part, c, D) = make_float2(best, sum);
  } else {
    const int r = row0 + fq / share, h = kvh * share + fq % share;
#pragma unroll
    for (int e = 0; e < PER; ++e) st<T>::stv((T*)a.out + (size_t)r * a.out_stride + (size_t)h * D + dim0 + e, acc[e]);
  }
}

template <typename T, int D, bool ONCE>
__global__ __launch_bounds__(64 * kWaves, D == 256 ? 2 : kResident) void kv8_attention_kernel(Kv8View kv, Kv8Attn a) {
  __shared__ typename Kv8Segment<T, D, ONCE>::Shared sh;
  const int lane = threadIdx.x & 63;
  Kv8Sequence s{0, 0, 0, 0, 1};
  const int each = kv8_piece(kv, a, s);
  int u = blockIdx.x, partials = 0;                       // this workgroup's piece, counted from sequence b0's first; partials before it
  int b = -1, in = 0, pieces = 1;                         // its sequence, its place there, and in how many pieces a segment is cut
  Kv8Sequence seq{0, 0, 0, 1, 1};
  for (int b0 = 0; b0 < kv.batch && b < 0; b0 += 64) {
    if (b0) {
      if (b0 + lane < kv.batch) s = kv8_sequence(kv, a, b0 + lane);
      else s.tiles = 0;
    }
    const int cut = (s.units + each - 1) / each, n = s.tiles * kv.heads * cut;      // pieces of a segment, of the sequence
    int upto = n, part = cut > 1 ? n : 0;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
      const int x = __shfl_up(upto, o, 64), y = __shfl_up(part, o, 64);
      if (lane >= o) { upto += x; part += y; }
    }
    const uint64_t past = __ballot(upto > u);
    const int at = past ? __builtin_ffsll((long long)past) - 1 : 63;
    if (past) {
      b = b0 + at;
      seq.row0 = __builtin_amdgcn_readlane(s.row0, at);
      seq.rows = __builtin_amdgcn_readlane(s.rows, at);
      seq.len = __builtin_amdgcn_readlane(s.len, at);
      seq.tiles = __builtin_amdgcn_readlane(s.tiles, at);
      seq.units = __builtin_amdgcn_readlane(s.units, at);
      pieces = __builtin_amdgcn_readlane(cut, at);
      in = u - __builtin_amdgcn_readlane(upto - n, at);
      partials += __builtin_amdgcn_readlane(part - n, at) + in;
    } else {
      u -= __builtin_amdgcn_readlane(upto, 63);
      partials += __builtin_amdgcn_readlane(part, 63);
    }
  }
  if (b < 0) return;
  const int segment = in / pieces, i = in % pieces, kvh = segment / seq.tiles, p = pieces > 1 ? partials : -1;
  if (in < 0 || kvh >= kv.heads || p < -1 || p >= 2 * a.pieces) return;        // (rows that are no prefix sums may overflow the counts)
  const int u0 = (int)((int64_t)seq.units * i / pieces), u1 = (int)((int64_t)seq.units * (i + 1) / pieces);
  Kv8Segment<T, D, ONCE>::run(kv, a, sh, b, seq, kvh, segment % seq.tiles * 16, u0 * a.unit, min(seq.len, u1 * a.unit), p);
}

// The partial results of one row and head, joined by one workgroup: D / 4 threads take a partial, the groups of such threads
// the partials in turn, and the groups' sums are added in their order.
template <typename T, int D>
__global__ __launch_bounds__(256) void kv8_join_kernel(Kv8View kv, Kv8Attn a) {
  constexpr int kGroups = 256 / (D / 4);
  __shared__ float w_sh[256];
  __shared__ float4 sum_sh[kGroups][D / 4];
  const int lane = threadIdx.x & 63, r = blockIdx.x, h = blockIdx.y, group = threadIdx.x / (D / 4), at = threadIdx.x % (D / 4);
  const int b = __builtin_amdgcn_readfirstlane(kv8_sequence_of(a.cu_rows, kv.batch, r));
  if (b >= kv.batch) return;
  Kv8Sequence seq{0, 0, 0, 0, 1};
  const int each = kv8_piece(kv, a, seq);
  int before = 0;                                         // partials of the sequences before this one
  for (int b0 = 0; b0 < kv.batch; b0 += 64) {
    if (b0 && b0 + lane < kv.batch) seq = kv8_sequence(kv, a, b0 + lane);
    const int cut = (seq.units + each - 1) / each;
    before += b0 + lane < b && cut > 1 ? seq.tiles * kv.heads * cut : 0;
    if (b < b0 + 64) break;
  }
  before = wave_sum_int(before);
  const int row0 = __builtin_amdgcn_readlane(seq.row0, b % 64), tiles = __builtin_amdgcn_readlane(seq.tiles, b % 64);
  const int n = (__builtin_amdgcn_readlane(seq.units, b % 64) + each - 1) / each;
  if (n <= 1) return;                                     // written where it was computed
  const int f = (r - row0) * a.share + h % a.share, col = f % 16;
  const int p0 = before + (h / a.share * tiles + f / 16) * n;
  if (r < row0 || before < 0 || p0 < 0 || p0 + n > 2 * a.pieces) return;
  // (every wave works out the same maximum and sum; of the first 64 partials a lane's own stays in registers)
  const float2 own = lane < n ? *a.stats(p0 + lane, col, D) : make_float2(kNegInf, 0.f);
  float best = own.x;
  for (int c = lane + 64; c < n; c += 64) best = fmaxf(best, a.stats(p0 + c, col, D)->x);
  best = wave_max(best);
  auto weight = [&](float2 ml) { return ml.x == kNegInf && ml.y == 0.f ? 0.f : __builtin_amdgcn_exp2f(ml.x - best) * ml.y; };
  float sum = weight(own);
  for (int c = lane + 64; c < n; c += 64) sum += weight(*a.stats(p0 + c, col, D));
  sum = wave_sum(sum);
  const float inv = sum == 0.f ? 0.f : 1.f / sum;
  float4 acc = make_float4(0.f, 0.f, 0.f, 0.f);
  for (int c0 = 0; c0 < n; c0 += 256) {
    if (c0) __syncthreads();
    float2 ml = own;
    if ((c0 || threadIdx.x >= 64) && c0 + (int)threadIdx.x < n) ml = *a.stats(p0 + c0 + threadIdx.x, col, D);
    w_sh[threadIdx.x] = weight(ml) * inv;                 // (past n: never read)
    __syncthreads();
    const int here = min(256, n - c0);
#pragma unroll 4
    for (int c = group; c < here; c += kGroups) {
      const float4 p = reinterpret_cast<const float4*>(a.sums(p0 + c0 + c, col, D))[at];
      const float wc = w_sh[c];
      acc.x = fmaf(wc, p.x, acc.x); acc.y = fmaf(wc, p.y, acc.y); acc.z = fmaf(wc, p.z, acc.z); acc.w = fmaf(wc, p.w, acc.w);
    }
  }
  sum_sh[group][at] = acc;
  __syncthreads();
  if (threadIdx.x >= D / 4) return;
#pragma unroll
  for (int g = 1; g < kGroups; ++g) {
    const float4 p = sum_sh[g][at];
    acc.x += p.x; acc.y += p.y; acc.z += p.z; acc.w += p.w;
  }
  T* dst = (T*)a.out + (size_t)r * a.out_stride + (size_t)h * D + at * 4;
  const float v[4] = {acc.x, acc.y, acc.z, acc.w};
  if constexpr (sizeof(T) == 2) st4(dst, v); else *reinterpret_cast<float4*>(dst) = acc;
}

struct Kv8Plan { int unit, wgs, pieces; bool once, split; };

// By the bounds alone: the same for every call with the same bounds.
Kv8Plan kv8_plan(const Kv8View& kv, int d, int n_heads, int m_upper, int len_upper) {
  Kv8Plan p;
  // every sequence rounds its queries up to a tile, and a tile holds one at least
  const int64_t queries = (int64_t)m_upper * (n_heads / kv.heads), most = queries / 16 + kv.batch;
  const int64_t segments = (queries < most ? queries : most) * kv.heads;
  p.unit = kUnit;
  while (segments * (len_upper / p.unit + 1) > 1 << 30) p.unit *= 2;          // units are counted in 32 bits
  const int64_t units = segments * (len_upper / p.unit + 1);
  p.pieces = kRounds * 256 * (d == 256 ? 2 : kResident);                            // a few rounds of what registers let run at once
  p.wgs = (int)(units < segments + p.pieces ? units : segments + p.pieces);
  p.split = len_upper > p.unit * kLeast;
  p.once = queries <= 16 * (int64_t)kv.batch;
  return p;
}

}  // namespace

size_t slk_kv8_attention_bytes(const Kv8View& kv, int d, int n_heads, int m_upper, int len_upper) {
  if (m_upper == 0) return 256;
  const Kv8Plan p = kv8_plan(kv, d, n_heads, m_upper, len_upper);
  return p.split ? sl_align_up((size_t)p.pieces * 32 * (d + 2) * sizeof(float), 256) : 256;
}

int slk_kv8_attention(hipStream_t s, const Kv8View& kv, int d, int dtype, const void* q, int64_t q_stride, int n_heads,
                      const int32_t* cu_rows, const int32_t* seq_len, const int32_t* row_len, int m_upper, int len_upper, float scale,
                      void* out, int64_t out_stride, void* workspace) {
  const Kv8Plan p = kv8_plan(kv, d, n_heads, m_upper, len_upper);
  const Kv8Attn a{q, out, (float*)workspace, cu_rows, seq_len, row_len, q_stride, out_stride, n_heads, n_heads / kv.heads, m_upper,
                  len_upper, p.unit, p.pieces, (float)((double)scale * 1.4426950408889634)};
  const dim3 join(m_upper, n_heads);
#define KV8_CALL(T, D)                                                                                                  \
  do {                                                                                                                  \
    if (p.once) hipLaunchKernelGGL((kv8_attention_kernel<T, D, true>), dim3(p.wgs), dim3(64 * kWaves), 0, s, kv, a);    \
    else hipLaunchKernelGGL((kv8_attention_kernel<T, D, false>), dim3(p.wgs), dim3(64 * kWaves), 0, s, kv, a);          \
    if (p.split) hipLaunchKernelGGL((kv8_join_kernel<T, D>), join, dim3(256), 0, s, kv, a);                             \
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
