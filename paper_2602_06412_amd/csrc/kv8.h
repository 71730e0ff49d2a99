// The paged 8-bit K/V cache: addressing and what its kernels share.
//
// A vector of d_head numbers of one row and one head is kept as 8-bit codes and one fp32 scale: scale = max|x| / 127, code =
// rint(x / scale), value = code * scale.  16 slots of one head are a tile,
//   [K codes 16 d][V codes 16 d][16 K scales][16 V scales]
// and a page holds page_slots / 16 tiles of every head, a head's tiles behind one another.  Inside a tile the codes lie in the
// order in which the matrix cores take them (16-row products, lane l: row l % 16, the (l / 16)-th quarter of the reduction), so a
// lane's share of an operand is one load of 16 bytes (8 with d = 32) and a wave's load is one contiguous KiB:
//   K  [d / 4E][4][16 slots][E dims]            signed bytes, E = 16 (8 with d = 32): the operand of a product of 8-bit integers
//   V  [d / 4E][4][16][E / 4 dims][4 slots]     code + 128; reduction over slots: the scores' product K Q^T leaves slots
//                                               4 (l / 16) .. + 3 of a tile in lane l, so probabilities become the second
//                                               product's operand in place; a lane's E / 4 dims are neighbours, one in each of
//                                               as many products, so that a block of neighbouring dims and slots is one store
#pragma once
#include "sl_common.h"

template <int D>
struct Kv8Tile {
  static constexpr int E = D >= 64 ? 16 : 8;              // bytes a lane loads at once
  static constexpr int CH = D / (4 * E);                  // such loads for the K (or V) codes of a tile
  static constexpr int kV = 16 * D, kKs = 32 * D, kVs = 32 * D + 64, kBytes = 32 * D + 128;
  __host__ __device__ static constexpr int k_at(int slot, int dim) {
    return ((dim / (4 * E)) * 64 + (dim % (4 * E)) / E * 16 + slot) * E + dim % E;
  }
  __host__ __device__ static constexpr int v_at(int slot, int dim) {
    return kV + ((dim / (4 * E)) * 64 + slot / 4 * 16 + dim % (4 * E) / (E / 4)) * E + dim % (E / 4) * 4 + slot % 4;
  }
};

// The cache as its kernels see it.
struct Kv8View {
  unsigned char* pool;
  const int32_t* table;                                   // [batch][max_pages]
  int n_pages, page_shift, heads, batch, max_pages;       // page_slots = 1 << page_shift
  __device__ int slots() const { return max_pages << page_shift; }
  // first byte of the tile that holds slot `slot` (of a sequence) of `head` in page `page`
  template <int D>
  __device__ unsigned char* tile(int page, int head, int slot) const {
    const int tiles = 1 << (page_shift - 4);
    return pool + (((size_t)page * heads + head) * tiles + ((slot >> 4) & (tiles - 1))) * Kv8Tile<D>::kBytes;
  }
};

// The sequence that row r belongs to: the number of entries of cu_rows[1 .. batch] that are <= r (batch if r is behind the last
// sequence).  A whole wave asks at once, at most SL_MAX_BATCH entries in independent loads.
__device__ inline int kv8_sequence_of(const int32_t* cu_rows, int batch, int r) {
  const int lane = threadIdx.x & 63;
  int n = 0;
#pragma unroll
  for (int i = 0; i < (SL_MAX_BATCH + 63) / 64; ++i) {
    const int b = i * 64 + lane;
    if (i * 64 < batch) n += __popcll(__ballot(b < batch && cu_rows[min(b, batch - 1) + 1] <= r));
  }
  return n;
}

int slk_kv8_write(hipStream_t s, const Kv8View& kv, int d, int dtype, const void* k, const void* v, int64_t k_stride, int64_t v_stride,
                  const int32_t* row_pos, const int32_t* cu_rows, int m_upper);
int slk_kv8_read(hipStream_t s, const Kv8View& kv, int d, int dtype, void* k, void* v, int64_t k_stride, int64_t v_stride,
                 const int32_t* row_pos, const int32_t* cu_rows, int m_upper);
size_t slk_kv8_attention_bytes(const Kv8View& kv, int d, int n_heads, int m_upper, int len_upper);
int slk_kv8_attention(hipStream_t s, const Kv8View& kv, int d, int dtype, const void* q, int64_t q_stride, int n_heads,
                      const int32_t* cu_rows, const int32_t* seq_len, const int32_t* row_len, int m_upper, int len_upper, float scale,
                      void* out, int64_t out_stride, void* workspace);
