// A token for each row from its filtered posterior, with a given uniform number.
//
// Every filter keeps a beginning of the row's order (z descending, id ascending), so what is kept is a border: all tokens above one number
// and, in order of ids, some of those that equal it.  Weights are whole numbers, W = rint(2^44 exp((z - max) / T)): at most 2^18 of them
// add up to less than 2^63, in any order and from any thread, to the same sum.
//
// A workgroup takes a row and passes over it as often as it has to, 32 to 64 bytes a thread in flight.  Of bf16 that is twice (counts, with the
// largest number; then weights in order of ids), and what bounds it is those reads and an LDS access a token: 1024 rows of 126464, top-p and min-p, 113 us,
// 4.6 TB/s over both passes (one read of all rows at the rate of a large one: 38 us); 64 rows, top-k and top-p, 36 us, each
// on a CU of its own: 506 KB in two passes, at 14 GB/s with the searches for two borders among them (1 row: top-p 36 us, top-k 26).  Several workgroups a row, in three
// launches, gained where there is no filter (64 rows 28 -> 21 us, 1 row 26 -> 18) and a tenth with top-p, but were slower for top-k (27 -> 30), for many rows and
// for short ones: one workgroup it is.
//
// Weights.  2^t = 2^n T[i] 2^(r / 256) with 256 t = 256 n + i + r, |r| <= 1 / 2: a table of 256 powers and a sum of four terms, off by
// less than 2^-51 of itself.
// bf16.  A weight depends on 16 bits, and logits take a few thousand of the 65536 numbers.  These are counted one by one (LDS, an atomic
// add of one a token): order, sums of weights and borders follow from counts times weights, and the exponential is
// taken once for each number that occurs; the last pass reads the weights of what is kept from a table.  Numbers below 2^-10 in size, nearly
// half of the 65536 and hardly any logit, share one bin and are weighed token by token.  The pass also finds the largest number if that is positive and not tiny; rows of
// log-probabilities are passed over once more for it (64 rows, top-p 36 -> 38 us, top-k 28 -> 37; 1024 rows 114 -> 136 and 90 -> 135).  Numbers that are all tiny, or all
// alike, meet in one place of LDS, token by token: a row of 126464 zeros takes 530 us with top-p, 1024 of them 1950 (no filter 62 and 228).
// fp32, and bf16 where that does not do (a border among the tiny numbers, a temperature in the hundreds): the border's key in three
// steps of 11, 11 and 10 bits that add up weights (or counts) for each value of the digit.  The first is a pass over the row; the second lists the
// keys that begin with the first's digit, in LDS, and it and the third work on the list (if that has no room for all, on the row).  What bounds
// it is the fp64 of a weight for each token and pass: 64 rows of 126464 fp32, top-p, 116 to 121 us (130 with three passes over the row),
// top-k 63 to 65 (76; 68 with a pass of its own for the first digit), both 92, no filter 50; 1 row 115, 61, 87 and 47.
#include "sl_common.h"

namespace {

constexpr int kBins = 6144, kDigits = 2048;
constexpr int kTiny = 0x3a7f;                             // the largest bf16 below 2^-10: its 15 lower bits
constexpr int kMiddle = 2560;                             // the tiny numbers' bin: above it numbers to 2^10, below it to -2^18
constexpr int kTinyList = 4096;                           // (16-bit numbers, where the parts' sums come later)
constexpr int kList = 8192;
constexpr int kMaxParts = 1024;                           // 64 times 16 bytes of 1024 threads: 2^18 fp32 numbers
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

struct Shared {
  union {
    uint32_t counts[kBins + 64];                          // (the last: what is beyond the bins, a place for each lane)
    uint64_t weights[kBins + 2];
    struct {
      uint64_t digits[kDigits];
      uint32_t list[kList];                               // keys that begin with the border's first digit
    };
  };
  struct {                                                // of a wave's part of a piece, in order of ids
    uint64_t sum[kMaxParts];
    uint32_t ties[kMaxParts];
  } part;
  double powers[256];
  uint64_t sums[16], sums2[16];
  uint32_t numbers[16];
  uint64_t found, found2, tiny;
  uint32_t tinies, listed;
  uint32_t word;
  int index;
  float most[16];
};
static_assert(sizeof(Shared) <= 64 * 1024, "two workgroups a CU");
static_assert(kTinyList * 2 <= sizeof(Shared::part.sum), "the list of tiny numbers");

// fp32 as a number whose order is that of z (both zeros alike)
__device__ inline uint32_t key_of(float z) {
  const uint32_t u = __float_as_uint(z + 0.f);
  return u ^ (u >> 31 ? 0xffffffffu : 0x80000000u);
}
__device__ inline float of_key(uint32_t k) { return __uint_as_float(k ^ (k >> 31 ? 0x80000000u : 0xffffffffu)); }
// a token that may be drawn: neither NaN nor -infinity.  (A comparison with -infinity itself in a ballot comes out of the compiler as "not
// equal", which is true of NaN.)
__device__ inline bool allowed(float z) { return z >= -3.402823466e38f; }

typedef short s16x2 __attribute__((ext_vector_type(2)));
typedef unsigned short u16x2 __attribute__((ext_vector_type(2)));

struct Weigher {
  double most, rate;                                      // rate: 256 log2(e) / temperature
  const double* powers;
  __device__ __forceinline__ uint64_t operator()(float z) const {
    constexpr double kRound = 6755399441055744.0, L = 0.0027076061740622863;      // 1.5 2^52; ln 2 / 256
    const double t = fmax(((double)z - most) * rate, -16384.0), y = t + kRound, r = (t - (y - kRound)) * L;
    const int n = (int)(uint32_t)__double_as_longlong(y);
    const double p = fma(r, fma(r, fma(r, fma(r, 1.0 / 24, 1.0 / 6), 0.5), 1.0), 1.0) * powers[n & 255];
    const uint64_t w = (uint64_t)__double_as_longlong(ldexp(p, 44 + (n >> 8)) + 4503599627370496.0) & 0xfffffffffffffull;
    return (double)z == most ? (uint64_t)kUnit : w;       // (an infinity, too)
  }
};

// sum over the block of the threads before this one; `whole` gets the sum of all
template <int NT>
__device__ inline uint64_t before_me(uint64_t v, Shared& sh, uint64_t& whole) {
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const uint64_t sum = wave_scan(v);
  __syncthreads();
  if (lane == 63) sh.sums[wave] = sum;
  __syncthreads();
  const uint64_t waves = wave_scan(lane < NT / 64 ? sh.sums[lane] : 0);
  whole = lane_of(waves, NT / 64 - 1);
  return (wave ? lane_of(waves, wave - 1) : 0) + sum - v;
}

// two sums at once, in place
template <int NT>
__device__ inline void before_me2(uint64_t& v, uint32_t& n, Shared& sh, uint64_t& v_all, uint32_t& n_all) {
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const uint64_t sum = wave_scan(v);
  const uint32_t number = wave_scan32(n);
  __syncthreads();
  if (lane == 63) {
    sh.sums[wave] = sum;
    sh.sums2[wave] = number;
  }
  __syncthreads();
  const uint64_t waves = wave_scan(lane < NT / 64 ? sh.sums[lane] : 0), numbers = wave_scan(lane < NT / 64 ? sh.sums2[lane] : 0);
  v_all = lane_of(waves, NT / 64 - 1);
  n_all = (uint32_t)lane_of(numbers, NT / 64 - 1);
  v = (wave ? lane_of(waves, wave - 1) : 0) + sum - v;
  n = (uint32_t)(wave ? lane_of(numbers, wave - 1) : 0) + number - n;
}

typedef uint32_t piece_t __attribute__((ext_vector_type(4), aligned(2)));

// A row in pieces of 16 bytes a thread: piece c of thread t holds ids (c NT + t) kVec ..; what is past the row is -infinity.  Rows begin where
// they like (the loads take any address).
template <typename T, int NT>
struct Row {
  static constexpr int kVec = st<T>::kVec, kSpan = NT * kVec, kThreads = NT, kBits = 128 / kVec;
  const T* z;
  int vocab;
  uint4 only;                                             // of a row of one piece or less: it

  __device__ __forceinline__ int n() const { return (vocab + kSpan - 1) / kSpan; }
  __device__ __forceinline__ uint4 fetch(int c) const {
    const int id = c * kSpan + threadIdx.x * kVec, over = id + kVec - vocab;
    if (over <= 0) {
      const piece_t p = *reinterpret_cast<const piece_t*>(z + id);
      return make_uint4(p.x, p.y, p.z, p.w);
    }
    // the row's end: its last 16 bytes, moved down, and -infinities
    constexpr uint64_t kNone = kVec == 8 ? 0xff80ff80ff80ff80ull : 0xff800000ff800000ull;
    uint64_t lo = kNone, hi = kNone;
    if (over < kVec) {
      if (vocab >= kVec) {
        const piece_t p = *reinterpret_cast<const piece_t*>(z + vocab - kVec);
        lo = (uint64_t)p.y << 32 | p.x;
        hi = (uint64_t)p.w << 32 | p.z;
#pragma unroll 1
        for (int i = 0; i < over; ++i) {
          lo = lo >> kBits | hi << (64 - kBits);
          hi = hi >> kBits | kNone << (64 - kBits);
        }
      } else {                                            // (a row of less than 16 bytes)
#pragma unroll 1
        for (int i = vocab - 1; i >= 0; --i) {
          hi = hi << kBits | lo >> (64 - kBits);
          if constexpr (kVec == 8) lo = lo << kBits | __builtin_bit_cast(unsigned short, z[i]);
          else lo = lo << kBits | __float_as_uint((float)z[i]);
        }
      }
    }
    return make_uint4((uint32_t)lo, (uint32_t)(lo >> 32), (uint32_t)hi, (uint32_t)(hi >> 32));
  }
  __device__ __forceinline__ static float number(const uint4& p, int e) {
    const uint32_t x = p.x, y = p.y, z = p.z, w = p.w;    // (values: of references the compiler makes a place in memory)
    if constexpr (kVec == 8) {
      const uint32_t u = e < 4 ? e < 2 ? x : y : e < 6 ? z : w;
      return __uint_as_float(e & 1 ? u & 0xffff0000u : u << 16);
    } else {
      return __uint_as_float(e < 2 ? e == 0 ? x : y : e == 2 ? z : w);
    }
  }
  // f(piece's number, its 16 bytes): two pieces are worked on while the next two are on their way
  template <typename F>
  __device__ __forceinline__ void pieces(F f) const {
    const int full = vocab / kSpan;
    auto whole = [&](int c) __attribute__((always_inline)) {
      const piece_t p = *reinterpret_cast<const piece_t*>(z + (size_t)c * kSpan + threadIdx.x * kVec);
      return make_uint4(p.x, p.y, p.z, p.w);
    };
    auto work = [&](int c, const uint4& p) __attribute__((always_inline)) {
      f(c, p);
      __builtin_amdgcn_sched_barrier(0);                  // (one after another: registers)
    };
    uint4 a[2] = {}, b[2] = {}, last = {};
    if (full * kSpan < vocab) last = full ? fetch(full) : only;
#pragma unroll
    for (int i = 0; i < 2; ++i)
      if (i < full) a[i] = whole(i);
#pragma unroll 1
    for (int c = 0; c < full; c += 4) {
#pragma unroll
      for (int i = 0; i < 2; ++i)
        if (c + 2 + i < full) b[i] = whole(c + 2 + i);
      work(c, a[0]);
      if (c + 1 < full) work(c + 1, a[1]);
#pragma unroll
      for (int i = 0; i < 2; ++i)
        if (c + 4 + i < full) a[i] = whole(c + 4 + i);
      if (c + 2 < full) work(c + 2, b[0]);
      if (c + 3 < full) work(c + 3, b[1]);
    }
    if (full * kSpan < vocab) work(full, last);
  }
  // f(z)
  template <int UNROLL, typename F>
  __device__ __forceinline__ void each(F f) const {
    pieces([&](int, const uint4& p) __attribute__((always_inline)) {
#pragma unroll UNROLL
      for (int e = 0; e < kVec; ++e) f(number(p, e));
    });
  }
};

// The fewest of `there` equal weights that bring `above` to the goal
__device__ inline uint64_t fewest(uint64_t above, uint64_t each, uint64_t there, double goal) {
  uint64_t need = 1;
  if (each > 0 && goal > (double)above) need = (uint64_t)fmax(1.0, fmin(floor((goal - (double)above) * __builtin_amdgcn_rcp((double)each)), (double)there));      // (or one beside)
  while (need > 1 && (double)(above + (need - 1) * each) >= goal) --need;
  while (need < there && (double)(above + need * each) < goal) ++need;
  return need < there ? need : there;
}

// The draw: weigh(piece, f, g) calls f(e, tie, weight) for each token of a piece: whether it is on the border, and the weight of one above, and
// g(e, weight) for what weighs more than f was told.  Of the tokens on the border the first `need` weigh `each`.  kept: the number of
// tokens kept, or -1; then above(piece) counts a lane's tokens above the border.  any(piece): whether the wave has a token to keep.
template <typename R, typename A, typename W, typename N>
__device__ __forceinline__ void draw(const R& row, Shared& sh, const SampleArgs& a, int r, uint32_t need, uint64_t each, int kept, A any, W weigh, N above) {
  constexpr int NT = R::kThreads, kParts = NT / 64, kMine = kMaxParts / NT;
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), parts = row.n() * kParts;
  const bool count = a.kept && kept < 0;
  uint32_t number = 0;
  row.pieces([&](int c, const uint4& p) __attribute__((always_inline)) {
    uint64_t sum = 0;
    uint32_t ties = 0;
    if (any(p)) {
      weigh(p, [&](int, bool tie, uint64_t w) __attribute__((always_inline)) {
        sum += w;
        ties += __popcll(__ballot(tie));
      }, [&](int, uint64_t w) __attribute__((always_inline)) { sum += w; });
      if (count) number += above(p);
      sum = wave_scan(sum);
    }
    if (lane == 63) {
      sh.part.sum[c * kParts + wave] = sum;
      sh.part.ties[c * kParts + wave] = ties;
    }
  });
  if (count) number = wave_scan32(number);
  if (lane == 63) sh.numbers[wave] = number;
  __syncthreads();
  // sums up to each part, neighbouring parts a thread
  uint64_t sums = 0;
  uint32_t ties = 0;
#pragma unroll
  for (int i = 0; i < kMine; ++i) {
    const int at = tid * kMine + i;
    if (at < parts) {
      sums += sh.part.sum[at];
      ties += sh.part.ties[at];
    }
  }
  uint64_t all_sums;
  uint32_t all_ties;
  const uint64_t own_sums = sums;
  const uint32_t own_ties = ties;
  before_me2<NT>(sums, ties, sh, all_sums, all_ties);
  const uint64_t whole = all_sums + min(all_ties, need) * each;
  const float u = a.uniform[r];
  const double goal = (double)(u > 0.f ? fminf(u, 0x1.fffffep-1f) : 0.f) * (double)whole;
  if ((double)(sums + min(ties, need) * each) <= goal && (double)(sums + own_sums + min(ties + own_ties, need) * each) > goal) {
    int at = tid * kMine;
    for (; at < tid * kMine + kMine - 1; ++at) {
      const uint64_t s = sums + sh.part.sum[at];
      const uint32_t t = ties + sh.part.ties[at];
      if ((double)(s + min(t, need) * each) > goal) break;
      sums = s;
      ties = t;
    }
    sh.index = at;
    sh.found = sums;
    sh.word = ties;
  }
  if (a.kept && tid == 0) {
    if (count) {
      kept = (int)min(all_ties, need);
      for (int w = 0; w < kParts; ++w) kept += (int)sh.numbers[w];
    }
    a.kept[r] = kept;
  }
  __syncthreads();
  if (sh.index % kParts != wave) return;
  // the part that holds it, once more
  const int c = sh.index / kParts, id = c * R::kSpan + tid * R::kVec;
  const uint4 p = row.vocab < R::kSpan ? row.only : row.fetch(c);
  uint64_t w[R::kVec] = {}, mine = 0;
  uint32_t tie[R::kVec] = {}, my_ties = 0;
  weigh(p, [&](int e, bool is_tie, uint64_t v) __attribute__((always_inline)) {
    w[e] = v;
    my_ties += tie[e] = is_tie;
  }, [&](int e, uint64_t v) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < R::kVec; ++i) w[i] += i == e ? v : 0;
  });
  uint32_t at = sh.word + wave_scan32(my_ties) - my_ties;
  const uint32_t taken = min(sh.word, need);
#pragma unroll
  for (int e = 0; e < R::kVec; ++e) {
    if (tie[e] && at < need) w[e] = each;
    at += tie[e];
    mine += w[e];
  }
  uint64_t run = sh.found + taken * each + wave_scan(mine) - mine;
#pragma unroll
  for (int e = 0; e < R::kVec; ++e) {
    if ((double)run <= goal && (double)(run + w[e]) > goal) {
      a.token[r] = id + e;
      if (a.prob) a.prob[r] = (float)((double)w[e] / (double)whole);
    }
    run += w[e];
  }
}

// Bins of bf16 numbers, in descending order.  With u = max(0, size - kTiny), sizes being the lower 15 bits, the bin is kMiddle - u for positive numbers
// and kMiddle + u for negative ones: the tiny numbers of both signs are the middle bin.
constexpr int kAllowed = kMiddle + 0x7f80 - kTiny;        // -infinity's
__device__ inline int bin_of(float z) {
  const int bits = (int)(__float_as_uint(z) >> 16), u = max(0, (bits & 0x7fff) - kTiny);
  return bits >> 15 ? kMiddle + u : kMiddle - u;
}
__device__ inline float number_of(int b) {
  return __uint_as_float((uint32_t)(b < kMiddle ? kTiny + kMiddle - b : (kTiny + b - kMiddle) | 0x8000) << 16);
}

// f(e, SIZE times the bin) for the eight numbers of a piece; bins from `most` on, numbers beyond bin 0, NaNs and -infinity are `most`.  Returns whether one of them is
// tiny.  (Step by step for all four words: each step waits for the one before.)
template <int SIZE, typename F>
__device__ __forceinline__ bool each_bin(int most, const uint4& piece, F f) {
  constexpr unsigned short kScale = SIZE >= 4 ? 4 : 1, kFar = SIZE >= 4 ? kBins - kMiddle + 64 : 0x7fff;      // (farther ones as far: 4 (middle + u) stays below 2^16)
  const uint32_t w[4] = {piece.x, piece.y, piece.z, piece.w};
  const u16x2 limit = u16x2{1, 1} * (unsigned short)(most * kScale), middle = u16x2{1, 1} * (unsigned short)(kMiddle * kScale);
  u16x2 u[4], sign[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) u[i] = __builtin_bit_cast(u16x2, w[i] & 0x7fff7fffu);
#pragma unroll
  for (int i = 0; i < 4; ++i) sign[i] = __builtin_bit_cast(u16x2, __builtin_bit_cast(s16x2, w[i]) >> 15);
#pragma unroll
  for (int i = 0; i < 4; ++i) u[i] = __builtin_elementwise_sub_sat(u[i], u16x2{kTiny, kTiny});
  const u16x2 least = __builtin_elementwise_min(__builtin_elementwise_min(u[0], u[1]), __builtin_elementwise_min(u[2], u[3]));
#pragma unroll
  for (int i = 0; i < 4; ++i) sign[i] = (~sign[i] & (unsigned short)(-2 * kScale)) | kScale;      // -SCALE, or SCALE
#pragma unroll
  for (int i = 0; i < 4; ++i) u[i] = __builtin_elementwise_min(u[i], u16x2{kFar, kFar});
#pragma unroll
  for (int i = 0; i < 4; ++i) u[i] = u[i] * sign[i] + middle;
#pragma unroll
  for (int i = 0; i < 4; ++i) u[i] = __builtin_elementwise_min(u[i], limit);
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const uint32_t b = __builtin_bit_cast(uint32_t, u[i]);
    f(2 * i, (b & 0xffff) * (SIZE / kScale));
    f(2 * i + 1, (b >> 16) * (SIZE / kScale));
  }
  return least[0] == 0 || least[1] == 0;
}

// The largest bits of a piece's numbers, in two parts: of positive bf16 numbers their bits are in their order, and any negative one's are below.
__device__ __forceinline__ s16x2 largest_of(const uint4& p) {
  const auto two = [](uint32_t w) { return __builtin_bit_cast(s16x2, w); };
  return __builtin_elementwise_max(__builtin_elementwise_max(two(p.x), two(p.y)), __builtin_elementwise_max(two(p.z), two(p.w)));
}

// f(e) for the tiny numbers of a piece
template <typename F>
__device__ __forceinline__ void each_tiny(const uint4& piece, F f) {
  const uint32_t w[4] = {piece.x, piece.y, piece.z, piece.w};
  uint32_t mask = 0;
#pragma unroll
  for (int e = 0; e < 8; ++e) mask |= ((w[e / 2] >> (e & 1 ? 16 : 0)) & 0x7fff) <= (uint32_t)kTiny ? 1u << e : 0;
  while (mask) {
    f(__builtin_ctz(mask));
    mask &= mask - 1;
  }
}

template <typename T, int NT>
__global__ __launch_bounds__(NT, 4) void sample_filtered_kernel(SampleArgs a) {
  __shared__ __attribute__((aligned(16))) Shared sh;
  constexpr int kWaves = NT / 64;
  const int r = blockIdx.x, tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  // (asked for together with the row count)
  const int at = a.row_map ? a.row_map[r] : r, k = a.top_k ? a.top_k[r] : 0;
  const float heat = a.temperature ? a.temperature[r] : 1.f, p = a.top_p ? a.top_p[r] : 1.f, least = a.min_p ? a.min_p[r] : 0.f;
  if (r >= min(*a.m_dev, a.m_upper)) return;
  const bool there = at >= 0 && at < a.n_rows;
  Row<T, NT> row;
  row.z = (const T*)a.logits + (size_t)(there ? at : 0) * a.row_stride;
  row.vocab = there ? a.vocab : 0;
  row.only = row.vocab < Row<T, NT>::kSpan ? row.fetch(0) : uint4{};
  if (tid < 256) sh.powers[tid] = exp2(tid / 256.0);

  // the first of the order alone
  const bool one = !(heat > 0.f) || k == 1 || p <= 0.f || least > 1.f;
  const bool by_count = k > 0 && k < a.vocab && !one, by_mass = p < 1.f && !one, count = sizeof(T) == 2 && (by_count || by_mass);
  float most = -__builtin_inff();
  auto tiny_list = reinterpret_cast<unsigned short*>(sh.part.sum);
  if (count) {
    for (int i = tid; i < kBins / 4; i += NT) reinterpret_cast<uint4*>(sh.counts)[i] = make_uint4(0, 0, 0, 0);
    if (tid == 0) sh.tiny = sh.tinies = 0;
    __syncthreads();
    s16x2 top = {-0x8000, -0x8000};                       // the largest positive number's bits
    row.pieces([&](int, const uint4& piece) __attribute__((always_inline)) {
      const bool small = each_bin<4>(kBins + lane, piece, [&](int, uint32_t at) __attribute__((always_inline)) {
        atomicAdd(reinterpret_cast<uint32_t*>(reinterpret_cast<unsigned char*>(sh.counts) + at), 1u);
      });
      top = __builtin_elementwise_max(top, largest_of(piece));
      if (small) each_tiny(piece, [&](int e) __attribute__((always_inline)) {
        const uint32_t i = atomicAdd(&sh.tinies, 1u);
        if (i < kTinyList) tiny_list[i] = (unsigned short)(__float_as_uint(Row<T, NT>::number(piece, e)) >> 16);
      });
    });
    most = wave_max((float)max(top[0], top[1]));
    if (lane == 0) sh.most[wave] = most;
    __syncthreads();
    const int bits = (int)wave_max(lane < kWaves ? sh.most[lane] : -__builtin_inff());
    most = bits > kTiny && bits <= kTiny + kMiddle ? __uint_as_float((uint32_t)bits << 16) : -__builtin_inff();
    __syncthreads();
  }
  const bool unfiltered = a.kept && !(k > 0 && k < a.vocab) && !(p < 1.f) && !(least > 0.f);      // then all tokens are kept: how many?
  int kept = -1;
  // (fp32: the first digit of top-k's border is counted where the maximum is found)
  const bool early = sizeof(T) == 4 && by_count;
  if (!allowed(most)) {
    uint32_t number = 0;
    if (early) {
      for (int i = tid; i < kDigits; i += NT) sh.digits[i] = 0;
      __syncthreads();
    }
    row.pieces([&](int, const uint4& piece) __attribute__((always_inline)) {
#pragma unroll
      for (int e = 0; e < Row<T, NT>::kVec; ++e) most = fmaxf(most, Row<T, NT>::number(piece, e));
      if (early) {
#pragma unroll
        for (int e = 0; e < Row<T, NT>::kVec; ++e) {
          const float z = Row<T, NT>::number(piece, e);
          if (allowed(z)) atomicAdd((unsigned long long*)&sh.digits[key_of(z) >> 21], 1ull);
        }
      }
      if (unfiltered) {
#pragma unroll
        for (int e = 0; e < Row<T, NT>::kVec; ++e) number += __popcll(__ballot(allowed(Row<T, NT>::number(piece, e))));
      }
    });
    most = wave_max(most);
    if (lane == 0) {
      sh.most[wave] = most;
      sh.numbers[wave] = number;
    }
    __syncthreads();
    most = wave_max(lane < kWaves ? sh.most[lane] : -__builtin_inff());
    if (unfiltered) kept = __builtin_amdgcn_readlane(wave_scan32(lane < kWaves ? sh.numbers[lane] : 0), 63);
  }
  if (!allowed(most)) {
    if (tid == 0) {
      a.token[r] = 0;
      if (a.prob) a.prob[r] = 0.f;
      if (a.kept) a.kept[r] = 0;
    }
    return;
  }
  if (one) kept = 1;
  const double enough = least > 0.f && !one ? (double)least * kUnit : 0.0;
  const Weigher weight{(double)most, 369.32993046757463 / (double)heat, sh.powers};

  if constexpr (sizeof(T) == 2) {
    const int first_bin = bin_of(most);
    int border = kAllowed;                                // kept: bins below the border, and of the border's tokens the first `need`
    uint32_t need = 0;
    uint64_t each = 0;
    // whether the bins do: they hold the largest number, and there is no weight beyond them
    bool counted = !one && most < __builtin_inff() && first_bin >= 0 && first_bin < kBins && weight(number_of(kBins - 1)) == 0 && (!count || sh.tinies <= kTinyList);
    if (one && first_bin >= 0 && first_bin < kBins && first_bin != kMiddle) {
      counted = true;
      border = first_bin;
      need = 1;
      each = (uint64_t)kUnit;
    }
    if (counted && count) {
      for (uint32_t i = tid; i < sh.tinies; i += NT)
        atomicAdd((unsigned long long*)&sh.tiny, (unsigned long long)weight(__uint_as_float((uint32_t)tiny_list[i] << 16)));
      __syncthreads();
      // neighbouring bins a thread
      constexpr int kMine = kBins / NT;
      const uint64_t tiny = sh.tiny;
      uint64_t mass = 0, total;
      uint32_t n[kMine], number = 0, all;
#pragma unroll
      for (int i = 0; i < kMine; ++i) {
        const int b = tid * kMine + i;
        n[i] = sh.counts[b];
        number += n[i];
      }
      if (__any(number > 0)) {
#pragma unroll
        for (int i = 0; i < kMine; ++i) {
          const int b = tid * kMine + i;
          const uint64_t w = n[i] * weight(number_of(b));
          mass += b == kMiddle ? tiny : w;
        }
      }
      const uint64_t my_mass = mass;
      const uint32_t my_number = number;
      before_me2<NT>(mass, number, sh, total, all);
#pragma unroll 1
      for (int round = 0; round < 2; ++round) {
        if (!(round ? by_mass : by_count)) continue;
        if (!round && (uint32_t)k > all) {                // (whether more tokens lie beyond the bins is not known)
          counted = false;
          break;
        }
        const double goal = round ? (double)p * (double)total : (double)k;
        const double before = round ? (double)mass : (double)number, up_to = round ? (double)(mass + my_mass) : (double)(number + my_number);
        if (before < goal && goal <= up_to) {
          sh.index = tid;
          sh.found = mass;
          sh.word = number;
        }
        __syncthreads();
        // every wave finds the number on its own
        const int b = sh.index * kMine + lane;
        const uint32_t n = lane >= kMine ? 0 : b == border ? need : b < min(border, kBins) ? sh.counts[b] : 0;
        const uint64_t w = n && b != kMiddle ? weight(number_of(b)) : 0, here = n == 0 ? 0 : b == kMiddle ? tiny : n * w;
        const uint64_t masses = sh.found + wave_scan(here);
        const uint32_t counts = sh.word + wave_scan32(n);
        const int first = __builtin_ctzll(__ballot((round ? (double)masses : (double)counts) >= goal || lane == kMine - 1));
        const uint32_t n_there = __builtin_amdgcn_readlane(n, first), n_before = __builtin_amdgcn_readlane(counts - n, first);
        const uint64_t m_before = lane_of(masses - here, first);
        border = sh.index * kMine + first;
        if (border == kMiddle) {
          counted = false;
          break;
        }
        each = lane_of(w, first);
        need = round ? fewest(m_before, each, n_there, goal) : k - n_before;
        kept = n_before + need;
        total = m_before + need * each;
        __syncthreads();
      }
    }
    if (counted && enough > 0) {
      // the first bin whose weight is not enough: near where the logarithm says
      const int b = bin_of((float)((double)most + (double)heat * log((double)least))) - 31 + lane;
      const float tiny_most = 0x1.fep-11f;                 // the largest bf16 below 2^-10
      const bool tiny_first = (double)weight(fminf(most, tiny_most)) >= enough, tiny_last = (double)weight(-tiny_most) >= enough;
      const bool passes = b <= first_bin || (b < kBins && (b == kMiddle ? tiny_last : (double)weight(number_of(b)) >= enough));
      const uint64_t passing = __ballot(passes);
      if (!(passing & 1) || passing >> 63 || (most > -tiny_most && tiny_first != tiny_last)) {
        counted = false;
      } else {
        const int limit = lane_of((uint64_t)(uint32_t)b, 0) + __builtin_ctzll(~passing);
        if (limit <= border) {
          border = limit;
          need = 0;
          kept = -1;
        }
      }
    }
    if (counted) {
      // weights of the bins that are kept, as far as they are not 0 (exp(-31.2) 2^44 is below 1/2); a 0 for the border and one for all others
      const int table = one ? border : min(min(border, kBins), bin_of((float)((double)most - 31.2 * (double)heat)) + 2);
      __syncthreads();
      for (int b = first_bin + tid; b <= table + 1; b += NT) sh.weights[b] = b < table && b != kMiddle ? weight(number_of(b)) : 0;
      __syncthreads();
      const uint32_t on_border = need > 0 && border == table ? border * 8 : 0xffff;      // (tokens of a border further down weigh nothing)
      // where what is kept is positive, a wave looks at its largest number first (positive bf16 numbers are in the order of their bits)
      const int lowest = table < kMiddle ? (int)(__float_as_uint(number_of(table)) >> 16) : -0x8000;
      draw(row, sh, a, r, need, each, kept, [&](const uint4& p) __attribute__((always_inline)) {
        const s16x2 m = largest_of(p);
        return (bool)__any(max(m[0], m[1]) >= lowest);
      }, [&](const uint4& piece, auto f, auto g) __attribute__((always_inline)) {
        const bool small = each_bin<8>(table + 1, piece, [&](int e, uint32_t at) __attribute__((always_inline)) {
          f(e, at == on_border, *reinterpret_cast<const uint64_t*>(reinterpret_cast<const unsigned char*>(sh.weights) + at));
        });
        if (small && kMiddle < table) each_tiny(piece, [&](int e) __attribute__((always_inline)) { g(e, weight(Row<T, NT>::number(piece, e))); });
      }, [&](const uint4& piece) __attribute__((always_inline)) {
        uint32_t n = 0;
        each_bin<1>(kAllowed, piece, [&](int, uint32_t b) __attribute__((always_inline)) { n += (int)b < border; });
        return n;
      });
      return;
    }
  }

  // the border's key digit by digit: by count, then by mass
  __syncthreads();
  if (!one && !unfiltered) kept = -1;
  constexpr int kSlow = sizeof(T) == 2 ? 1 : 4;           // (of bf16 rows few come here)
  uint32_t border = one ? key_of(most) : 0x007fffffu;     // (-infinity's)
  uint32_t need = one;
  uint64_t each = one ? (uint64_t)kUnit : 0, over = 0;
  auto inside = [&](uint32_t key, float z) __attribute__((always_inline)) { return allowed(z) && key >= border; };
#pragma unroll 1
  for (int round = 0; round < 2; ++round) {
    if (!(round ? by_mass : by_count)) continue;
    double goal = 0;
    bool none = false;                                    // no border: all tokens are kept
    uint32_t prefix = 0;
    uint64_t above = 0;
    int shift = 32;
    bool listed = false;
#pragma unroll 1
    for (int step = 0; step < 3; ++step) {
      const int bits = step < 2 ? 11 : 10, upper = shift;
      shift -= bits;
      const bool counted = early && !round && step == 0;
      for (int i = tid; i < kDigits && !counted; i += NT) sh.digits[i] = 0;
      if (tid == 0 && step == 0) sh.listed = 0;
      __syncthreads();
      auto add = [&](uint32_t key, float z) __attribute__((always_inline)) {
        atomicAdd((unsigned long long*)&sh.digits[key >> shift & ((1 << bits) - 1)], (unsigned long long)(round ? weight(z) : 1));
      };
      if (step == 1) {
        row.template each<kSlow>([&](float z) __attribute__((always_inline)) {
          const uint32_t key = key_of(z);
          const bool in = inside(key, z) && key >> upper == prefix;
          const uint64_t all = __ballot(in);
          if (!all) return;
          int at = 0;
          if (lane == 0) at = (int)atomicAdd(&sh.listed, (uint32_t)__popcll(all));
          at = __builtin_amdgcn_readfirstlane(at) + __builtin_amdgcn_mbcnt_hi((uint32_t)(all >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)all, 0));
          if (in && at < kList) sh.list[at] = key;
        });
        __syncthreads();
        listed = sh.listed <= kList;
      }
      if (listed) {
        for (uint32_t i = tid; i < sh.listed; i += NT) {
          const uint32_t key = sh.list[i];
          if (step == 1 || key >> upper == prefix) add(key, of_key(key));
        }
      } else if (!counted) {
        row.template each<kSlow>([&](float z) __attribute__((always_inline)) {
          const uint32_t key = key_of(z);
          if (inside(key, z) && (step == 0 || key >> upper == prefix)) add(key, z);
        });
      }
      __syncthreads();
      // neighbouring digits a thread, descending
      constexpr int kMine = kDigits / NT;
      const int top = (1 << bits) - 1 - kMine * tid;
      uint64_t sum = 0, whole;
      for (int i = 0; i < kMine; ++i) sum += top - i >= 0 ? sh.digits[top - i] : 0;
      uint64_t run = above + before_me<NT>(sum, sh, whole);
      if (step == 0) {
        // (of tokens with the border's key of the first round the digits hold all: `over` too many)
        none = !round && (uint64_t)k >= whole;
        if (none) break;
        goal = round ? (double)p * (double)(whole - over) : (double)k;
      }
      if ((double)run < goal && (double)(run + sum) >= goal) {
        int digit = top;
        while ((double)(run + sh.digits[digit]) < goal) run += sh.digits[digit--];
        sh.found = run;
        sh.word = prefix << bits | (uint32_t)digit;
        sh.found2 = sh.digits[digit];
      }
      __syncthreads();
      above = sh.found;
      prefix = sh.word;
    }
    if (none) continue;
    // (tokens with the border's key of the first round: `need` of them, whatever the digits have added up)
    const uint64_t w = weight(of_key(prefix)), unit = round ? w : 1;
    const uint64_t there = unit ? sh.found2 / unit : 1;
    need = (uint32_t)fewest(above, unit, prefix == border ? need : there, goal);
    over = (there - need) * w;
    each = w;
    border = prefix;
    __syncthreads();
  }
  if (enough > 0) {
    uint32_t under = 0;                                   // the last key whose weight is not enough
#pragma unroll 1
    for (uint32_t bit = 1u << 31; bit; bit >>= 1)
      if (under + bit < key_of(most) && (double)weight(of_key(under + bit)) < enough) under += bit;
    if (under >= border) {
      border = under;
      need = 0;
    }
  }
  draw(row, sh, a, r, need, each, kept, [](const uint4&) { return true; }, [&](const uint4& piece, auto f, auto g) __attribute__((always_inline)) {
#pragma unroll
    for (int e = 0; e < Row<T, NT>::kVec; ++e) {
      const float z = Row<T, NT>::number(piece, e);
      const uint32_t key = key_of(z);
      const bool above = allowed(z) && key > border;
      f(e, allowed(z) && key == border, sizeof(T) == 4 && above ? weight(z) : 0);
    }
    if constexpr (sizeof(T) == 2) {
#pragma unroll 1
      for (int e = 0; e < 8; ++e) {
        const float z = Row<T, NT>::number(piece, e);
        if (allowed(z) && key_of(z) > border) g(e, weight(z));
      }
    }
  }, [&](const uint4& piece) __attribute__((always_inline)) {
    uint32_t n = 0;
#pragma unroll
    for (int e = 0; e < Row<T, NT>::kVec; ++e) {
      const float z = Row<T, NT>::number(piece, e);
      n += allowed(z) && key_of(z) > border;
    }
    return n;
  });
}

}  // namespace

int slk_sample_filtered(hipStream_t s, const void* logits, int dtype, int64_t row_stride, int n_rows, int vocab, const int32_t* row_map,
                        const int32_t* m_dev, int m_upper, const float* temperature, const int32_t* top_k, const float* top_p, const float* min_p,
                        const float* uniform, int32_t* token, float* prob, int32_t* kept) {
  const SampleArgs a{logits, row_stride, n_rows, vocab, m_upper, row_map, m_dev, top_k, temperature, top_p, min_p, uniform, token, prob, kept};
#define SAMPLE_RUN(T, NT) hipLaunchKernelGGL((sample_filtered_kernel<T, NT>), dim3(m_upper), dim3(NT), 0, s, a)
  // Rows beyond the CUs: two workgroups of 512 threads a CU pass over more rows at a time, one of 1024 over a row faster.  512 / 1024 threads,
  // us, top-p: 126464 bf16 64 rows 40.6 / 36.3, 256 rows 46.5 / 41.9, 300 rows 59 / 65, 512 rows 63 / 78, 1024 rows 117 / 145; 8192 bf16 256 rows
  // 12.4 / 13.4, 512 rows 16 / 24; 126464 fp32 256 rows 175 / 135, 300 rows 230 / 179, 384 rows 236 / 239, 512 rows 247 / 254; 8192 fp32
  // 300 rows 25.1 / 25.7, 384 rows 25 / 34.  And few rows that are short, of which most is waiting for one another: 3 rows of 1024 bf16 9.6 / 11.0,
  // 8192 bf16 12.0 / 13.0, 16384 bf16 14.3 / 14.8, 1024 fp32 11.2 / 12.8, 4096 fp32 15.0 / 15.7, 8192 fp32 19.7 / 18.8 (256 threads are slower than 512).
  const bool many = m_upper > (dtype == SL_BF16 ? 256 : 320) || vocab * sl_tsize(dtype) <= 16384;
  if (dtype == SL_BF16) {
    if (many) SAMPLE_RUN(bf16_t, 512); else SAMPLE_RUN(bf16_t, 1024);
  } else {
    if (many) SAMPLE_RUN(float, 512); else SAMPLE_RUN(float, 1024);
  }
#undef SAMPLE_RUN
  SL_LAUNCH_CHECK();
  return SL_OK;
}
