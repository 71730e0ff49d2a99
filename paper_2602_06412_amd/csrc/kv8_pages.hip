// Pages of the 8-bit cache from the lengths that sequences want: page table, rows of the new slots and their places in the pool.
//
// With p(l) = ceil(l / page_slots), a sequence that shrinks gives up entries p(new) .. p(old) - 1 of its table and one that grows takes
// entries p(old) .. p(new) - 1.  Numbered in order of sequence and entry, page number i taken is page number i given up; if more are
// taken, the further ones come from the top of the stack, and if more are given up, the further ones go on top of it.  So every place
// that is written depends on prefix sums over the sequences alone, and one pass does everything:
//   pieces     an entry of a growing sequence's table that holds new slots: its page, and the rows of its slots.  Who takes a page that is
//              given up also clears the entry that it came from, so that no two lanes touch one entry
//   returns    a page given up and not taken: onto the stack, and its entry cleared
//   copies     (states apart) all other entries of the table and of the stack
// Every workgroup forms the prefix sums again from the lengths, a wave for all 255 sequences, lanes moved instead of LDS: no second launch, no
// atomics.  What bounds it is the chain of loads and sums of that wave and one search in them, not bytes.  Replayed from a graph, into another state: 3
// sequences 4.3 us (3 us are a launch's own), 255 sequences that decode 5.4 us, 64 sequences of which half want 176000 slots more, not all of which fit, 6.6 us.
// In place: 8 sequences that decode 3.1 us, 255 sequences 5.3 us, of which 1.5 are the copy of the lengths that goes before.
#include "sl_common.h"

namespace {

constexpr int kSeqs = 256, kThreads = 256;

struct Pages {
  int32_t *table, *seq_len, *stack, *n_free;
};

struct PagesArgs {
  Pages from, to;
  const int32_t *seq_len, *n_free;                        // as they were before the call, whatever is written meanwhile
  const int32_t* want;
  int32_t *cu_rows, *row_pos, *row_len, *row_seq;
  int64_t* row_slot;
  int n_pages, page_shift, batch, max_pages, m_upper, apart;
};

struct Plan {
  int old_len[kSeqs], new_len[kSeqs];
  int gone[kSeqs + 1], taken[kSeqs + 1], rows[kSeqs + 1], pieces[kSeqs + 1];      // prefix sums
  int free_pages;
};

__device__ inline int pages_of(int len, int shift) { return (int)(((int64_t)len + (1 << shift) - 1) >> shift); }

// first index b of start[0 .. kSeqs] with start[b] <= i < start[b + 1]
__device__ inline int owner(const int* start, int i) {
  int b = 0;
#pragma unroll
  for (int step = kSeqs / 2; step; step >>= 1)
    if (start[b + step] <= i) b += step;
  return b;
}

// By one wave, four sequences a lane.
__device__ void make_plan(const PagesArgs& a, Plan& p) {
  const int lane = threadIdx.x & 63, shift = a.page_shift;
  const int64_t most = (int64_t)a.max_pages << shift;      // <= 2^30
  const int free_pages = min(max(*a.n_free, 0), a.n_pages);
  int old_len[4], want[4], gone[4], need[4], more[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int b = lane * 4 + i;
    const bool there = b < a.batch;
    old_len[i] = there ? (int)min((int64_t)max(a.seq_len[b], 0), most) : 0;
    want[i] = there ? a.want[b] : 0;
    if (want[i] < 0 || want[i] > most) want[i] = old_len[i];
    const int change = pages_of(want[i], shift) - pages_of(old_len[i], shift);
    gone[i] = max(-change, 0);
    need[i] = max(change, 0);
    more[i] = max(want[i] - old_len[i], 0);
  }
  // sequences that there is no room for stay.  Those before the first of them are served; what they leave is too little for it, and for
  // others behind it: these stay too, and the rest is looked at again.
  const uint32_t gone_to_me = wave_scan32(gone[0] + gone[1] + gone[2] + gone[3]);
  const int64_t left = (int64_t)free_pages + (uint32_t)__builtin_amdgcn_readlane(gone_to_me, 63);
  while (true) {
    const int64_t needs = (int64_t)need[0] + need[1] + need[2] + need[3], mores = (int64_t)more[0] + more[1] + more[2] + more[3];
    int64_t n = (int64_t)wave_scan(needs) - needs, m = (int64_t)wave_scan(mores) - mores, n_left = 0, m_left = 0;      // left for the first without room
    int first = 4;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if (first == 4 && (n + need[i] > left || m + more[i] > a.m_upper)) {
        first = i;
        n_left = left - n;
        m_left = a.m_upper - m;
      }
      n += need[i];
      m += more[i];
    }
    const uint64_t without = __ballot(first < 4);
    if (!without) break;
    const int where = __builtin_ctzll(without), first_seq = where * 4 + __builtin_amdgcn_readlane(first, where);
    n_left = (int64_t)lane_of(n_left, where);
    m_left = (int64_t)lane_of(m_left, where);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      if (lane * 4 + i < first_seq || (need[i] <= n_left && more[i] <= m_left)) continue;
      want[i] -= more[i];
      need[i] = more[i] = 0;
    }
  }
  uint32_t v[4][4];                                       // [what][sequence]: given up, taken, rows, pieces
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    v[0][i] = gone[i];
    v[1][i] = need[i];
    v[2][i] = more[i];
    v[3][i] = more[i] ? pages_of(want[i], shift) - (old_len[i] >> shift) : 0;
  }
  int* const to[4] = {p.gone, p.taken, p.rows, p.pieces};
#pragma unroll
  for (int w = 0; w < 4; ++w) {
    const uint32_t own = v[w][0] + v[w][1] + v[w][2] + v[w][3], sum = w ? wave_scan32(own) : gone_to_me;
    uint32_t at = sum - own;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      to[w][lane * 4 + i] = (int)at;
      at += v[w][i];
    }
    if (lane == 63) to[w][kSeqs] = (int)sum;
  }
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    p.old_len[lane * 4 + i] = old_len[i];
    p.new_len[lane * 4 + i] = want[i];
  }
  if (lane == 0) p.free_pages = free_pages;
}

__global__ __launch_bounds__(kThreads) void kv8_pages_kernel(PagesArgs a) {
  __shared__ Plan p;
  if (threadIdx.x < 64) make_plan(a, p);
  __syncthreads();
  const int tid = threadIdx.x, shift = a.page_shift, page_slots = 1 << shift;
  const int gone = p.gone[kSeqs], taken = p.taken[kSeqs], rows = p.rows[kSeqs], pieces = p.pieces[kSeqs];
  if (blockIdx.x == 0) {
    if (tid < a.batch) {
      a.cu_rows[tid] = p.rows[tid];
      a.to.seq_len[tid] = p.new_len[tid];
    }
    if (tid == 0) {
      a.cu_rows[a.batch] = rows;
      *a.to.n_free = min(p.free_pages + gone - taken, a.n_pages);
    }
  }
  // entry of the table that the page number i given up stands in
  auto gone_entry = [&](int i) {
    const int b = owner(p.gone, i);
    return (size_t)b * a.max_pages + pages_of(p.new_len[b], shift) + (i - p.gone[b]);
  };
  // pieces: as many lanes as a page has slots, at most a wave
  const int lanes = min(page_slots, 64), teams = kThreads / lanes, me = tid & (lanes - 1);
  for (int piece = blockIdx.x * teams + tid / lanes; piece < pieces; piece += gridDim.x * teams) {
    const int b = owner(p.pieces, piece), old_len = p.old_len[b], new_len = p.new_len[b];
    const int j = (old_len >> shift) + piece - p.pieces[b], first_new = pages_of(old_len, shift);
    const size_t entry = (size_t)b * a.max_pages + j;
    int page = 0;
    if (me == 0) {
      if (j >= first_new) {
        const int i = p.taken[b] + j - first_new;
        if (i < gone) {
          const size_t source = gone_entry(i);
          page = a.from.table[source];
          a.to.table[source] = -1;
        } else {
          page = a.from.stack[p.free_pages - 1 - (i - gone)];
        }
        a.to.table[entry] = page;
      } else {
        page = a.from.table[entry];
      }
    }
    page = __shfl(page, 0, lanes);
    const int64_t slots = page >= 0 && page < a.n_pages ? (int64_t)page << shift : -1;
    for (int s = max(old_len, j << shift) + me; s < min((int64_t)new_len, ((int64_t)j + 1) << shift); s += lanes) {
      const int r = p.rows[b] + s - old_len;              // < m_upper
      a.row_pos[r] = s;
      if (a.row_len) a.row_len[r] = s + 1;
      if (a.row_seq) a.row_seq[r] = b;
      if (a.row_slot) a.row_slot[r] = slots < 0 ? -1 : slots + (s & (page_slots - 1));
    }
  }
  const int start = blockIdx.x * kThreads + tid, step = gridDim.x * kThreads;
  for (int64_t i = (int64_t)taken + start; i < gone; i += step) {
    const size_t source = gone_entry((int)i);
    const int64_t top = p.free_pages + i - taken;
    if (top < a.n_pages) a.to.stack[top] = a.from.table[source];
    a.to.table[source] = -1;
  }
  if (!a.apart) return;
  for (int i = start; i < a.batch * a.max_pages; i += step) {      // (<= 2^30)
    const int b = i / a.max_pages, j = i - b * a.max_pages;
    const int had = pages_of(p.old_len[b], shift), has = pages_of(p.new_len[b], shift);
    if (j < min(had, has) || j >= max(had, has)) a.to.table[i] = a.from.table[i];
  }
  const int pushed = max(gone - taken, 0);
  for (int i = start; i < a.n_pages; i += step)
    if (i < p.free_pages || i - p.free_pages >= pushed) a.to.stack[i] = a.from.stack[i];
}

__global__ __launch_bounds__(kThreads) void kv8_pages_lengths_kernel(const int32_t* seq_len, const int32_t* n_free, int batch, int32_t* out) {
  const int i = threadIdx.x;
  if (i <= batch) out[i] = i == batch ? *n_free : seq_len[i];
}

__global__ __launch_bounds__(kThreads) void kv8_pages_init_kernel(Pages to, int n_pages, int batch, int64_t entries) {
  const int64_t start = (int64_t)blockIdx.x * kThreads + threadIdx.x, step = (int64_t)gridDim.x * kThreads;
  for (int64_t i = start; i < entries; i += step) to.table[i] = -1;
  for (int64_t i = start; i < n_pages; i += step) to.stack[i] = n_pages - 1 - (int)i;
  if (start < batch) to.seq_len[start] = 0;
  if (start == 0) *to.n_free = n_pages;
}

// One number a thread, and at most 1024 workgroups, each of which forms the sums.  Replayed, us: numbers a workgroup 2048 / 512 / 256 / 128,
// 255 sequences that decode 9.4 / 6.2 / 5.4 / 5.4; workgroups at most 512 / 1024 / 2048, 64 sequences with prompts 7.7 / 6.6 / 6.6, 255 sequences of as many
// as 4096 pages that decode 9.5 / 8.6 / 8.5, 255 with prompts in pages of 64 11.3 / 9.2 / 8.5, in pages of 16 6.2 / 6.3 / 6.6, 255 of 4112 pages that all end, in
// place, 9.2 / 7.7 / 8.0.
unsigned grid_for(int64_t numbers) { return (unsigned)max((int64_t)1, min((int64_t)1024, (numbers + 255) / 256)); }

}  // namespace

size_t slk_kv8_pages_bytes(int batch) { return (size_t)(batch + 1) * 4; }

int slk_kv8_pages_init(hipStream_t s, const sl_kv8_pages* p) {
  const Pages to{p->page_table, p->seq_len, p->free_pages, p->n_free};
  const int64_t entries = (int64_t)p->batch * p->max_pages;
  hipLaunchKernelGGL(kv8_pages_init_kernel, dim3(grid_for(entries + p->n_pages)), dim3(kThreads), 0, s, to, p->n_pages, p->batch, entries);
  SL_LAUNCH_CHECK();
  return SL_OK;
}

int slk_kv8_pages_resize(hipStream_t s, const sl_kv8_pages* from, const sl_kv8_pages* to, const int32_t* want_len, int32_t* cu_rows, int32_t* row_pos,
                         int32_t* row_len, int32_t* row_seq, int64_t* row_slot, int m_upper, void* workspace) {
  PagesArgs a;
  a.from = Pages{from->page_table, from->seq_len, from->free_pages, from->n_free};
  a.to = Pages{to->page_table, to->seq_len, to->free_pages, to->n_free};
  a.apart = from->page_table != to->page_table;
  a.want = want_len;
  a.cu_rows = cu_rows; a.row_pos = row_pos; a.row_len = row_len; a.row_seq = row_seq; a.row_slot = row_slot;
  a.n_pages = from->n_pages;
  a.page_shift = __builtin_ctz((unsigned)from->page_slots);
  a.batch = from->batch;
  a.max_pages = from->max_pages;
  a.m_upper = m_upper;
  a.seq_len = from->seq_len;
  a.n_free = from->n_free;
  // In place a step may give up all pages that there are, however few its rows.  One workgroup does it without the copy below, if its lanes go few times
  // over the pieces of new rows and over those pages.  One / many workgroups, replayed, us, where every sequence takes a slot, and where all end: 8
  // sequences of 32 pages 3.1 / 4.6 and 3.0 / 4.5, 32 of 32 4.1 / 5.1 and 4.8 / 4.9, 64 of 64 5.7 / 5.1 and 11.5 / 4.9, 255 of 64 15.7 / 5.4 and 38.7 / 5.0,
  // 64 of 1024 5.8 / 5.2 and 148 / 5.0, 255 of 4112 15 / 5.2 and 2392 / 7.6.
  const int64_t entries = (int64_t)a.batch * a.max_pages, gives = min(entries, (int64_t)a.n_pages);
  const int64_t pieces = min((int64_t)m_upper, 2 * (int64_t)a.batch + m_upper / from->page_slots);
  const bool one = !a.apart && pieces * min(from->page_slots, 64) <= 2048 && gives <= 8192;
  const unsigned grid = one ? 1 : grid_for(m_upper + (a.apart ? entries + a.n_pages : gives));
  if (!a.apart && grid > 1) {
    // in place: the first workgroup writes lengths that others may not have read yet, so all read a copy
    hipLaunchKernelGGL(kv8_pages_lengths_kernel, dim3(1), dim3(kThreads), 0, s, from->seq_len, from->n_free, a.batch, (int32_t*)workspace);
    SL_LAUNCH_CHECK();
    a.seq_len = (const int32_t*)workspace;
    a.n_free = a.seq_len + a.batch;
  }
  hipLaunchKernelGGL(kv8_pages_kernel, dim3(grid), dim3(kThreads), 0, s, a);
  SL_LAUNCH_CHECK();
  return SL_OK;
}
