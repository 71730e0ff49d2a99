// Writing rows of K and V into the paged 8-bit cache, and reading them back.
#include "kv8.h"

namespace {

typedef float f32x4 __attribute__((ext_vector_type(4)));

// A wave works on a quad, 4 slots of one tile, of as many heads as it has lanes for: D / 4 lanes a head, 4 neighbouring dims each.
// So a lane's 4 dims of 4 slots of V are one 16-byte store, and after a 4 x 4 exchange among four lanes so are 16 dims of one
// slot of K.  A quad's wave belongs to the first of the adjacent rows that share it; rows of a prompt so come four at a time,
// scattered rows one by one, and of rows that name the same slot one wave sees all and keeps the last.
//
// Where rows are many, 5533 rows of 32 heads x 128 in bf16, 91 MB read and 47 written, take 42 us (a copy of as many bytes 29): vector
// instructions beside memory, 890 a wave, the pipes busy 68 % of the time.  Read back 26 us, which is memory.  A wave for each row and head with byte stores took 103 and 76; all loads of a quad before its first
// conversion, and the positions of its rows in one load by the lanes, were 73 to 42.
template <int D>
struct Quad {
  static constexpr int kLanes = D / 4, kHeads = 64 / kLanes;
};

struct Kv8Rows {
  const int32_t *row_pos, *cu_rows;
  int64_t k_stride, v_stride;
  int m_upper;
};

// The row's quad (of its sequence), or -1 if it has no slot in the table.
__device__ inline int quad_of(const Kv8View& kv, int pos) { return pos >= 0 && pos < kv.slots() ? pos >> 2 : -1; }

// This wave's quads among rows [r0, r0 + rows): bit i: row r0 + i is the first of its quad's and this wave's to do.
template <int ROWS>
__device__ inline uint32_t kv8_leaders(const Kv8View& kv, const Kv8Rows& a, int r0, int wave) {
  const int lane = threadIdx.x & 63, r = r0 + lane, last = min(a.cu_rows[kv.batch], a.m_upper);
  bool leads = lane < ROWS && r < last && r >= max(a.cu_rows[0], 0);
  if (leads) {
    const int q = quad_of(kv, a.row_pos[r]);
    leads = q < 0 || r == 0 || quad_of(kv, a.row_pos[r - 1]) != q;
  }
  // a sequence's first row leads as well
  for (int b = 0; b < kv.batch; b += 64) {
    const int start = b + lane < kv.batch ? a.cu_rows[b + lane] : -1;
    uint64_t mine = __ballot(start >= r0 && start < min(r0 + ROWS, last));
    while (mine) {
      const int at = __builtin_ffsll((long long)mine) - 1;
      mine &= mine - 1;
      if (r == __builtin_amdgcn_readlane(start, at)) leads = true;
    }
  }
  uint32_t all = (uint32_t)__ballot(leads), own = 0;
  for (int i = 0; all; ++i) {
    if (i % 4 == wave) own |= all & -all;
    all &= all - 1;
  }
  return own;
}

// The rows from r on that share quad `quad`: how many of the next 64, and their slots' places, lane by lane.
__device__ inline int kv8_run(const Kv8View& kv, const Kv8Rows& a, int r, int end, int quad, int& pos) {
  const int at = r + (threadIdx.x & 63);
  pos = at < end ? a.row_pos[at] : -1;
  const uint64_t other = __ballot(at >= end || quad_of(kv, pos) != quad);
  return other ? __builtin_ffsll((long long)other) - 1 : 64;
}

// quad transposition: lane i of four gets word i of each of the four
__device__ inline void exchange4(uint32_t (&w)[4]) {
  const int lane = threadIdx.x;
  const bool odd = lane & 1, high = lane & 2;
#pragma unroll
  for (int i = 0; i < 4; i += 2) {                        // with the neighbour: words 0, 1 and 2, 3
    const uint32_t give = odd ? w[i] : w[i + 1], got = __builtin_amdgcn_mov_dpp(give, 0xB1, 15, 15, true);
    if (odd) w[i] = got; else w[i + 1] = got;
  }
#pragma unroll
  for (int i = 0; i < 2; ++i) {                           // with the neighbouring pair: words 0, 2 and 1, 3
    const uint32_t give = high ? w[i] : w[i + 2], got = __builtin_amdgcn_mov_dpp(give, 0x4E, 15, 15, true);
    if (high) w[i] = got; else w[i + 2] = got;
  }
}

// maximum over the LANES neighbours of a head, in all of them: within 16 lanes by moving lanes, beyond by swapping rows of lanes
template <int LANES>
__device__ inline float max_of_lanes(float x) {
  auto with = [](float v, uint32_t moved) { return fmaxf(v, __uint_as_float(moved)); };
  x = with(x, __builtin_amdgcn_mov_dpp(__float_as_uint(x), 0xB1, 15, 15, true));        // lane ^ 1
  x = with(x, __builtin_amdgcn_mov_dpp(__float_as_uint(x), 0x4E, 15, 15, true));        // lane ^ 2
  x = with(x, __builtin_amdgcn_mov_dpp(__float_as_uint(x), 0x141, 15, 15, true));       // 7 - lane, of 8
  if constexpr (LANES >= 16) x = with(x, __builtin_amdgcn_mov_dpp(__float_as_uint(x), 0x140, 15, 15, true));      // 15 - lane, of 16
  if constexpr (LANES >= 32) {
    const auto p = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    x = fmaxf(__uint_as_float(p[0]), __uint_as_float(p[1]));
  }
  if constexpr (LANES >= 64) {
    const auto p = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
    x = fmaxf(__uint_as_float(p[0]), __uint_as_float(p[1]));
  }
  return x;
}

template <typename T>
__device__ inline void load4(const T* p, float (&v)[4]) {
  if constexpr (sizeof(T) == 2) {
    const uint2 u = *reinterpret_cast<const uint2*>(p);
    v[0] = __uint_as_float(u.x << 16); v[1] = __uint_as_float(u.x & 0xffff0000u);
    v[2] = __uint_as_float(u.y << 16); v[3] = __uint_as_float(u.y & 0xffff0000u);
  } else {
    ld4f(p, v);
  }
}
template <typename T>
__device__ inline void store4(T* p, const float (&v)[4]) {
  if constexpr (sizeof(T) == 2) st4(p, v); else *reinterpret_cast<float4*>(p) = make_float4(v[0], v[1], v[2], v[3]);
}

// Codes of a lane's 4 numbers, in a word, and the scale of the vector that its LANES lanes hold.  rint(x / scale) wants the rounded
// quotient: from the correctly rounded reciprocal of a scale in the middle of the range, a product and two steps of correction
// with exact remainders give it (Markstein); other scales divide.
template <int LANES>
__device__ inline uint32_t quantise(const float (&v)[4], float& scale) {
  float most = 0.f;
  bool nan = false;
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    nan |= v[e] != v[e];
    most = fmaxf(most, fabsf(v[e]));
  }
  most = max_of_lanes<LANES>(nan ? __builtin_inff() : most);
  scale = most < __builtin_inff() ? most / 127.f : __builtin_nanf("");
  const float y = 1.f / scale;
  float q[4];
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    q[e] = v[e] * y;
    q[e] = fmaf(fmaf(-q[e], scale, v[e]), y, q[e]);
    q[e] = fmaf(fmaf(-q[e], scale, v[e]), y, q[e]);
  }
  const bool plain = scale > 1e-30f && scale < 1e30f;
  if (__any(!plain)) {
#pragma unroll
    for (int e = 0; e < 4; ++e)
      if (!plain) q[e] = scale > 0.f ? v[e] / scale : 0.f;
  }
  uint32_t w = 0;
#pragma unroll
  for (int e = 0; e < 4; ++e) w |= (uint32_t)((int)fminf(fmaxf(rintf(q[e]), -127.f), 127.f) & 255) << (8 * e);
  return w;
}

// 4 x 4 bytes, rows slots and columns dims, to columns slots
__device__ inline void transpose_bytes(const uint32_t (&s)[4], uint32_t (&d)[4]) {
  const uint32_t a = __builtin_amdgcn_perm(s[1], s[0], 0x05010400u), b = __builtin_amdgcn_perm(s[3], s[2], 0x05010400u);      // dims 0, 1
  const uint32_t c = __builtin_amdgcn_perm(s[1], s[0], 0x07030602u), e = __builtin_amdgcn_perm(s[3], s[2], 0x07030602u);      // dims 2, 3
  d[0] = __builtin_amdgcn_perm(b, a, 0x05040100u);
  d[1] = __builtin_amdgcn_perm(b, a, 0x07060302u);
  d[2] = __builtin_amdgcn_perm(e, c, 0x05040100u);
  d[3] = __builtin_amdgcn_perm(e, c, 0x07060302u);
}

// ROWS rows of one group of heads a workgroup, its four waves the quads in turn.
template <typename T, int D, int ROWS>
__global__ __launch_bounds__(256) void kv8_write_kernel(Kv8View kv, const T* k, const T* v, Kv8Rows a) {
  using Tile = Kv8Tile<D>;
  constexpr int LANES = Quad<D>::kLanes, E = Tile::E;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), r0 = blockIdx.x * ROWS;
  // (lanes past the last head stay, on that head's numbers, and store nothing: the wave asks together)
  const int mine = blockIdx.y * Quad<D>::kHeads + lane / LANES, head = min(mine, kv.heads - 1), dim = lane % LANES * 4;
  uint32_t todo = kv8_leaders<ROWS>(kv, a, r0, wave);
  while (todo) {
    int r = r0 + __builtin_ctz(todo);
    todo &= todo - 1;
    const int b = kv8_sequence_of(a.cu_rows, kv.batch, r);
    const int quad = __builtin_amdgcn_readfirstlane(quad_of(kv, a.row_pos[r]));
    if (b >= kv.batch || quad < 0) continue;
    const int page = __builtin_amdgcn_readfirstlane(kv.table[(size_t)b * kv.max_pages + (quad >> (kv.page_shift - 2))]);
    if (page < 0 || page >= kv.n_pages) continue;
    const int end = min(a.cu_rows[b + 1], a.m_upper);
    int from[4] = {-1, -1, -1, -1};                       // the last row of each slot
    for (int n = 64; n == 64; r += n) {
      int pos;
      n = kv8_run(kv, a, r, end, quad, pos);
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const uint64_t rows = __ballot(lane < n && (pos & 3) == j);
        if (rows) from[j] = r + 63 - __builtin_clzll(rows);
      }
    }
    // (a slot that no row names takes another's numbers, which are not stored: all loads at once, without branches)
    const int some = max(max(from[0], from[1]), max(from[2], from[3]));
    float kx[4][4], vx[4][4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const size_t row = from[j] >= 0 ? from[j] : some;
      load4(k + row * a.k_stride + head * D + dim, kx[j]);
      load4(v + row * a.v_stride + head * D + dim, vx[j]);
    }
    uint32_t kc[4], vc[4], vt[4];
    float ks[4] = {}, vs[4] = {};
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      kc[j] = vc[j] = 0;
      if (ROWS == 4 && from[j] < 0) continue;             // (scattered rows: 9.4 us for 6.9; of prompts all four are there, 42 for 45)
      kc[j] = quantise<LANES>(kx[j], ks[j]);
      vc[j] = quantise<LANES>(vx[j], vs[j]) ^ 0x80808080u;          // code + 128
    }
    const int slot = quad * 4 & 15;
    unsigned char* tile = kv.tile<D>(page, head, quad * 4);
    exchange4(kc);                                        // now 16 dims of slot i, the lane's place among four
    const int i = lane & 3, first = dim & ~15;
    const int own = i == 0 ? from[0] : i == 1 ? from[1] : i == 2 ? from[2] : from[3];
    if (own >= 0 && mine == head) {
      if constexpr (E == 16) {
        *reinterpret_cast<uint4*>(tile + Tile::k_at(slot + i, first)) = make_uint4(kc[0], kc[1], kc[2], kc[3]);
      } else {
        *reinterpret_cast<uint2*>(tile + Tile::k_at(slot + i, first)) = make_uint2(kc[0], kc[1]);
        *reinterpret_cast<uint2*>(tile + Tile::k_at(slot + i, first + 8)) = make_uint2(kc[2], kc[3]);
      }
      if (dim < 16) {
        reinterpret_cast<float*>(tile + Tile::kKs)[slot + i] = i == 0 ? ks[0] : i == 1 ? ks[1] : i == 2 ? ks[2] : ks[3];
        reinterpret_cast<float*>(tile + Tile::kVs)[slot + i] = i == 0 ? vs[0] : i == 1 ? vs[1] : i == 2 ? vs[2] : vs[3];
      }
    }
    transpose_bytes(vc, vt);
    if (mine != head) continue;
    if (from[0] >= 0 && from[1] >= 0 && from[2] >= 0 && from[3] >= 0) {
      if constexpr (E == 16) {
        *reinterpret_cast<uint4*>(tile + Tile::v_at(slot, dim)) = make_uint4(vt[0], vt[1], vt[2], vt[3]);
      } else {
        *reinterpret_cast<uint2*>(tile + Tile::v_at(slot, dim)) = make_uint2(vt[0], vt[1]);
        *reinterpret_cast<uint2*>(tile + Tile::v_at(slot, dim + 2)) = make_uint2(vt[2], vt[3]);
      }
    } else {
#pragma unroll
      for (int j = 0; j < 4; ++j)
        if (from[j] >= 0) {
#pragma unroll
          for (int e = 0; e < 4; ++e) tile[Tile::v_at(slot + j, dim + e)] = (unsigned char)(vc[j] >> (8 * e));
        }
    }
  }
}

template <typename T, int D, int ROWS>
__global__ __launch_bounds__(256) void kv8_read_kernel(Kv8View kv, T* k, T* v, Kv8Rows a) {
  using Tile = Kv8Tile<D>;
  constexpr int LANES = Quad<D>::kLanes, E = Tile::E;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), r0 = blockIdx.x * ROWS;
  // (lanes past the last head stay, on that head's numbers, and store nothing: the wave asks together)
  const int mine = blockIdx.y * Quad<D>::kHeads + lane / LANES, head = min(mine, kv.heads - 1), dim = lane % LANES * 4;
  uint32_t todo = kv8_leaders<ROWS>(kv, a, r0, wave);
  while (todo) {
    int r = r0 + __builtin_ctz(todo);
    todo &= todo - 1;
    const int b = kv8_sequence_of(a.cu_rows, kv.batch, r);
    if (b >= kv.batch) continue;
    const int quad = __builtin_amdgcn_readfirstlane(quad_of(kv, a.row_pos[r]));
    int page = -1;
    if (quad >= 0) page = __builtin_amdgcn_readfirstlane(kv.table[(size_t)b * kv.max_pages + (quad >> (kv.page_shift - 2))]);
    const int end = quad < 0 ? r + 1 : min(a.cu_rows[b + 1], a.m_upper);      // (a row without a slot leads itself)
    int pos, n = kv8_run(kv, a, r, end, quad, pos);
    uint32_t kc[4] = {}, vw[4] = {0x80808080u, 0x80808080u, 0x80808080u, 0x80808080u};      // zeros
    f32x4 ks = {}, vs = {};
    if (page >= 0 && page < kv.n_pages) {
      const unsigned char* tile = kv.tile<D>(page, head, quad * 4);
      const int slot = quad * 4 & 15, i = lane & 3, first = dim & ~15;
      if constexpr (E == 16) {
        const uint4 x = *reinterpret_cast<const uint4*>(tile + Tile::k_at(slot + i, first)), y = *reinterpret_cast<const uint4*>(tile + Tile::v_at(slot, dim));
        kc[0] = x.x; kc[1] = x.y; kc[2] = x.z; kc[3] = x.w;
        vw[0] = y.x; vw[1] = y.y; vw[2] = y.z; vw[3] = y.w;
      } else {
        const uint2 x0 = *reinterpret_cast<const uint2*>(tile + Tile::k_at(slot + i, first)), x1 = *reinterpret_cast<const uint2*>(tile + Tile::k_at(slot + i, first + 8));
        const uint2 y0 = *reinterpret_cast<const uint2*>(tile + Tile::v_at(slot, dim)), y1 = *reinterpret_cast<const uint2*>(tile + Tile::v_at(slot, dim + 2));
        kc[0] = x0.x; kc[1] = x0.y; kc[2] = x1.x; kc[3] = x1.y;
        vw[0] = y0.x; vw[1] = y0.y; vw[2] = y1.x; vw[3] = y1.y;
      }
      ks = *reinterpret_cast<const f32x4*>(tile + Tile::kKs + 4 * slot);
      vs = *reinterpret_cast<const f32x4*>(tile + Tile::kVs + 4 * slot);
    }
    exchange4(kc);                                        // now the lane's 4 dims of the four slots, as vw after its exchange
    uint32_t vc[4];
    transpose_bytes(vw, vc);
    for (int i = 0; i < n; ++i, ++r) {
      const int j = __builtin_amdgcn_readlane(pos, i) & 3;
      const uint32_t kj = j == 0 ? kc[0] : j == 1 ? kc[1] : j == 2 ? kc[2] : kc[3], vj = j == 0 ? vc[0] : j == 1 ? vc[1] : j == 2 ? vc[2] : vc[3];
      const float s = j == 0 ? ks[0] : j == 1 ? ks[1] : j == 2 ? ks[2] : ks[3], t = j == 0 ? vs[0] : j == 1 ? vs[1] : j == 2 ? vs[2] : vs[3];
      float kx[4], vx[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        kx[e] = (float)(signed char)(kj >> (8 * e)) * s;
        vx[e] = (float)(signed char)((vj >> (8 * e)) ^ 0x80u) * t;
      }
      if (mine == head) {
        store4(k + (size_t)r * a.k_stride + head * D + dim, kx);
        store4(v + (size_t)r * a.v_stride + head * D + dim, vx);
      }
      if (i == 63) {                                      // (more than 64 rows of one quad: the next 64)
        n = kv8_run(kv, a, r + 1, end, quad, pos);
        i = -1;
      }
    }
  }
}

}  // namespace

#define KV8_BY_HEAD(T, CALL)                 \
  switch (d) {                               \
    case 32: CALL(T, 32); break;             \
    case 64: CALL(T, 64); break;             \
    case 128: CALL(T, 128); break;           \
    case 256: CALL(T, 256); break;           \
    default: return SL_EINVAL;               \
  }

// Rows a workgroup takes: four, a quad a wave, while rows are few and each may be a quad of its own; sixteen when there are so many
// that most of them join another row's quad and a workgroup of four would find nothing to do for three of its waves.
constexpr int kFewRows = 2048;

int slk_kv8_write(hipStream_t s, const Kv8View& kv, int d, int dtype, const void* k, const void* v, int64_t k_stride, int64_t v_stride,
                  const int32_t* row_pos, const int32_t* cu_rows, int m_upper) {
  const Kv8Rows a{row_pos, cu_rows, k_stride, v_stride, m_upper};
  const int rows = m_upper <= kFewRows ? 4 : 16;
  const dim3 grid(sl_cdiv(m_upper, rows), sl_cdiv(kv.heads * (d / 4), 64));
#define KV8_CALL(T, D)                                                                                                              \
  do {                                                                                                                              \
    if (rows == 4) hipLaunchKernelGGL((kv8_write_kernel<T, D, 4>), grid, dim3(256), 0, s, kv, (const T*)k, (const T*)v, a);         \
    else hipLaunchKernelGGL((kv8_write_kernel<T, D, 16>), grid, dim3(256), 0, s, kv, (const T*)k, (const T*)v, a);                  \
  } while (0)
  if (dtype == SL_BF16) { KV8_BY_HEAD(bf16_t, KV8_CALL) } else { KV8_BY_HEAD(float, KV8_CALL) }
#undef KV8_CALL
  SL_LAUNCH_CHECK();
  return SL_OK;
}

int slk_kv8_read(hipStream_t s, const Kv8View& kv, int d, int dtype, void* k, void* v, int64_t k_stride, int64_t v_stride,
                 const int32_t* row_pos, const int32_t* cu_rows, int m_upper) {
  const Kv8Rows a{row_pos, cu_rows, k_stride, v_stride, m_upper};
  const int rows = m_upper <= kFewRows ? 4 : 16;
  const dim3 grid(sl_cdiv(m_upper, rows), sl_cdiv(kv.heads * (d / 4), 64));
#define KV8_CALL(T, D)                                                                                             \
  do {                                                                                                             \
    if (rows == 4) hipLaunchKernelGGL((kv8_read_kernel<T, D, 4>), grid, dim3(256), 0, s, kv, (T*)k, (T*)v, a);     \
    else hipLaunchKernelGGL((kv8_read_kernel<T, D, 16>), grid, dim3(256), 0, s, kv, (T*)k, (T*)v, a);              \
  } while (0)
  if (dtype == SL_BF16) { KV8_BY_HEAD(bf16_t, KV8_CALL) } else { KV8_BY_HEAD(float, KV8_CALL) }
#undef KV8_CALL
  SL_LAUNCH_CHECK();
  return SL_OK;
}
