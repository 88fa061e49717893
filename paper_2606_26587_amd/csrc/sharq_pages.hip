// Page tables of the paged cache on the GPU: row offsets, lengths, pages and
// slot maps of a step from the requests' lengths; the reordering of tables and
// token ids behind beam search's choice; copies of partly filled pages.
//
// All of it is whole numbers, and every result is a fixed function of the
// inputs: pages are given out and taken back in the order of sequences and
// columns, by prefix sums, not in the order in which atomics happen to land.

#include "sharq_attn.hpp"
#include "sharq_serve.hpp"

namespace sharq {

// a + b, at most `top` (both are at most that, and top < 2^31)
__device__ __forceinline__ uint32_t add_most(uint32_t a, uint32_t b, uint32_t top) {
  const uint32_t s = a + b;
  return s < top ? s : top;
}

// Sum of v over the workgroup's threads before this one, saturating at top, and the total; `mem`: a word a wavefront,
// another one than that of the scan before.
__device__ __forceinline__ uint32_t block_scan(uint32_t v, uint32_t top, uint32_t* mem, uint32_t& total) {
  const int lane = (int)threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
  uint32_t x = v;
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    const uint32_t o = (uint32_t)__shfl_up((int)x, d);
    if (lane >= d) x = add_most(x, o, top);
  }
  if (lane == 63) mem[wave] = x;
  __syncthreads();
  uint32_t w = lane < kAssignThreads / 64 ? mem[lane] : 0;   // of all wavefronts, by each of them
#pragma unroll
  for (int d = 1; d < kAssignThreads / 64; d <<= 1) {
    const uint32_t o = (uint32_t)__shfl_up((int)w, d);
    if (lane >= d) w = add_most(w, o, top);
  }
  total = (uint32_t)__builtin_amdgcn_readlane((int)w, kAssignThreads / 64 - 1);
  const uint32_t before = wave ? (uint32_t)__builtin_amdgcn_readlane((int)w, wave ? wave - 1 : 0) : 0;
  const uint32_t left = (uint32_t)__shfl_up((int)x, 1);
  return lane ? add_most(left, before, top) : before;
}

// The page of the k-th column that the call fills: from the top of the stack down, -1 when it is empty.
__device__ __forceinline__ int assigned_page(const AssignArgs& a, int there, int k) {
  return k < there ? a.free[there - 1 - k] : -1;
}

// Sequence s's columns held..need-1, the first of which is the k-th that the call fills, by the wavefront.  One
// column, the usual case, was its lane's.
__device__ __forceinline__ void assign_columns(const AssignArgs& a, int there, int s, int held, int k, int n, int from) {
  for (int i = from + ((int)threadIdx.x & 63); i < n; i += 64) {
    const int page = assigned_page(a, there, k + i);
    a.table[s * a.ldt + held + i] = page;
    if (a.own) a.own[s * a.ldt + held + i] = page;
  }
}

// The columns of 64 sequences, a lane each.
__device__ __forceinline__ void assign_wave(const AssignArgs& a, int there, int s, int held, int k, int n) {
  if (n > 0) {
    const int page = assigned_page(a, there, k);
    a.table[s * a.ldt + held] = page;
    if (a.own) a.own[s * a.ldt + held] = page;
  }
  unsigned long long more = __ballot(n > 1);
  while (more) {
    const int l = __builtin_ctzll(more);
    more &= more - 1;
    assign_columns(a, there, __builtin_amdgcn_readlane(s, l), __builtin_amdgcn_readlane(held, l),
                   __builtin_amdgcn_readlane(k, l), __builtin_amdgcn_readlane(n, l), 1);
  }
}

// A row of the call: `first` is its sequence's first row, `given` the number of columns filled before the sequence's.
__device__ __forceinline__ void assign_row(const AssignArgs& a, int there, int row, int s, int pos, int held, int given) {
  if (a.row_seq) a.row_seq[row] = s;
  if (a.positions) a.positions[row] = pos;
  if (a.slots) {
    const int col = pos >> a.page_shift;
    const int page = col < held ? a.table[s * a.ldt + col] : assigned_page(a, there, given + col - held);
    a.slots[row] = page >= 0 && page < a.pages ? (page << a.page_shift) + (pos & ((1 << a.page_shift) - 1)) : -1;
  }
}

// The pages in columns lo..hi-1 of a row of a table, 64 at a time and four of these on their way together (without
// conditions: what is past the end is the last one again): f(whether there is one, it).
template <typename Fn>
__device__ __forceinline__ void each_page(const int32_t* row, int lo, int hi, int pages, Fn f) {
  const int lane = (int)threadIdx.x & 63;
  for (int c0 = lo; c0 < hi; c0 += 256) {
    int page[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int c = c0 + 64 * i + lane;
      page[i] = row[c < hi ? c : hi - 1];
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) f(c0 + 64 * i + lane < hi && page[i] >= 0 && page[i] < pages, page[i]);
  }
}

// One workgroup: offsets, lengths and columns of all sequences by prefix sums,
// pages that go back onto the stack, and (WHOLE) the pages that leave it and the
// rows.  A chain of latencies: the count, the lengths, three scans, the pages
// that go back read for their number and again for their places (columns may hold
// none), which all wavefronts share.  256 sequences, 950 rows: 7.3 us, one launch;
// 4096 with 65000 rows and 100 that end: 22.8 and 5.0 us for the rows, two launches
// (45 with each wavefront on the pages of its own 64 sequences).
template <bool WHOLE>
__global__ __launch_bounds__(kAssignThreads) void k_kv_assign(AssignArgs a) {
  constexpr int kItems = WHOLE ? 2 : 4, kPass = kItems * kAssignThreads;
  __shared__ uint32_t mem[3][kAssignThreads / 64];
  __shared__ int l_end[WHOLE ? kAssignSeqs : 1], l_given[WHOLE ? kAssignSeqs : 1], l_held[WHOLE ? kAssignSeqs : 1],
      l_len[WHOLE ? kAssignSeqs : 1];
  __shared__ int g_seq[kPass], g_lo[kPass], g_hi[kPass], g_n[kPass], g_count;   // sequences that give pages back
  const int tid = (int)threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int size = 1 << a.page_shift;
  const int on_stack = kv_clamp(*a.count, 0, a.pages);
  const int32_t* const from = a.own ? a.own : a.table;
  const uint32_t top = (uint32_t)a.rows;
  uint32_t rows = 0, given = 0, back = 0;   // of the sequences before these
  for (int s0 = 0; s0 < a.seqs; s0 += kPass) {
    int keep[kItems] = {}, add[kItems] = {}, held[kItems] = {};
#pragma unroll
    for (int i = 0; i < kItems; ++i) {
      const int s = s0 + tid * kItems + i;
      if (s < a.seqs) keep[i] = a.keep[s], add[i] = a.add[s], held[i] = a.held[s];
    }
    if (tid == 0) g_count = 0;
    uint32_t in[kItems], mine = 0, total;
#pragma unroll
    for (int i = 0; i < kItems; ++i) {
      keep[i] = kv_clamp(keep[i], 0, a.max_len);
      add[i] = kv_clamp(add[i], 0, a.max_len - keep[i]);
      held[i] = kv_clamp(held[i], 0, a.cols);
      in[i] = (uint32_t)(add[i] < a.rows ? add[i] : a.rows);
      mine = add_most(mine, in[i], top);
    }
    uint32_t at = add_most(rows, block_scan(mine, top, mem[0], total), top);
    rows = add_most(rows, total, top);
    int first[kItems], len[kItems], need[kItems], fresh[kItems], place[kItems];
    mine = 0;
#pragma unroll
    for (int i = 0; i < kItems; ++i) {
      first[i] = (int)at;
      at = add_most(at, in[i], top);
      len[i] = keep[i] + ((int)at - first[i]), need[i] = (len[i] + size - 1) >> a.page_shift;
      fresh[i] = need[i] > held[i] ? need[i] - held[i] : 0;
      mine += (uint32_t)fresh[i];
      place[i] = -1;
      if (held[i] > need[i]) {   // in any order: each has its own number
        place[i] = atomicAdd(&g_count, 1);
        g_seq[place[i]] = s0 + tid * kItems + i, g_lo[place[i]] = need[i], g_hi[place[i]] = held[i];
      }
    }
    uint32_t g = given + block_scan(mine, 0x7FFFFFFFu, mem[1], total);   // behind its barrier the list is whole
    given += total;
    for (int e = wave; e < g_count; e += kAssignThreads / 64) {
      int n = 0;
      each_page(from + g_seq[e] * a.ldt, __builtin_amdgcn_readfirstlane(g_lo[e]),
                __builtin_amdgcn_readfirstlane(g_hi[e]), a.pages, [&](bool there, int) { n += __popcll(__ballot(there)); });
      if (lane == 0) g_n[e] = n;
    }
    __syncthreads();
    uint32_t n_back[kItems];
    mine = 0;
#pragma unroll
    for (int i = 0; i < kItems; ++i) {
      n_back[i] = place[i] >= 0 ? (uint32_t)g_n[place[i]] : 0;
      mine += n_back[i];
    }
    uint32_t b = back + block_scan(mine, 0x7FFFFFFFu, mem[2], total);
    back += total;
#pragma unroll
    for (int i = 0; i < kItems; ++i) {
      const int s = s0 + tid * kItems + i;
      if (place[i] >= 0) g_n[place[i]] = (int)b;   // now where they go
      b += n_back[i];
      if (s < a.seqs) {
        a.offs[s] = first[i];
        a.lens[s] = len[i];
        a.held_out[s] = need[i];
        const int end = first[i] + (len[i] - keep[i]);
        if (WHOLE) l_end[s] = end, l_given[s] = (int)g, l_held[s] = held[i], l_len[s] = len[i];
        else a.ws[s] = (int)g, a.ws[a.seqs + s] = held[i];
      }
      g += (uint32_t)fresh[i];
    }
    __syncthreads();
    for (int e = wave; e < g_count; e += kAssignThreads / 64) {
      int64_t to = (int64_t)on_stack + g_n[e];
      each_page(from + g_seq[e] * a.ldt, __builtin_amdgcn_readfirstlane(g_lo[e]),
                __builtin_amdgcn_readfirstlane(g_hi[e]), a.pages, [&](bool there, int page) {
        const unsigned long long is = __ballot(there);
        const int64_t mine_to = to + __popcll(is & ((1ull << lane) - 1));
        if (there && mine_to < a.pages) a.free[mine_to] = page;
        to += __popcll(is);
      });
    }
    __syncthreads();   // the list is read
  }
  const int64_t all = (int64_t)on_stack + back;
  const int there = all < a.pages ? (int)all : a.pages;
  if (tid == 0) {
    a.offs[a.seqs] = (int)rows;
    *a.count_out = there > (int)given ? there - (int)given : 0;
    if (a.missing) *a.missing = (int)given > there ? (int)given - there : 0;
    if (!WHOLE) a.ws[2 * a.seqs] = there;
  }
  if (!WHOLE) return;
  __syncthreads();
  for (int s0 = tid & ~63; s0 < a.seqs; s0 += (int)blockDim.x) {
    const int s = s0 + lane;
    int held = 0, n = 0, k = 0;
    if (s < a.seqs) held = l_held[s], k = l_given[s], n = ((l_len[s] + size - 1) >> a.page_shift) - held;
    assign_wave(a, there, s, held, k, n);
  }
  if (!a.row_seq && !a.positions && !a.slots) return;
  for (int row = tid; row < (int)rows; row += (int)blockDim.x) {
    int s = 0, hi = a.seqs;   // the first sequence that ends behind the row
    while (s < hi) {
      const int mid = (s + hi) / 2;
      if (l_end[mid] <= row) s = mid + 1;
      else hi = mid;
    }
    assign_row(a, there, row, s, l_len[s] - (l_end[s] - row), l_held[s], l_given[s]);
  }
}

// Where there is more to write: rows, 256 a workgroup, and behind them the sequences' new columns, 256 sequences a
// workgroup.
__global__ __launch_bounds__(256) void k_kv_assign_rows(AssignArgs a, unsigned row_blocks) {
  const int tid = (int)threadIdx.x, lane = tid & 63;
  const int there = a.ws[2 * a.seqs];
  if (blockIdx.x >= row_blocks) {
    const int s = (int)(blockIdx.x - row_blocks) * 256 + tid;
    int held = 0, n = 0, k = 0;
    if (s < a.seqs) k = a.ws[s], held = a.ws[a.seqs + s], n = a.held_out[s] - held;
    assign_wave(a, there, s, held, k, n);
    return;
  }
  const int total = a.offs[a.seqs], row0 = (int)(blockIdx.x * 256 + (tid & ~63)), row = row0 + lane;
  if (row0 >= total) return;
  const KvBatchArgs b{a.offs, a.lens, nullptr, 0, a.seqs, a.rows, a.max_len};
  int s = a.seqs;
  bool found = false;
  // lanes hold the ends of 64 sequences; each looks for the first that ends behind its row
  for (int base = find_seq(b, row0); base < a.seqs && !__all(found); base += 64) {
    const int e = base + lane < a.seqs ? a.offs[base + lane + 1] : 0x7FFFFFFF;
    int lo = 0;
#pragma unroll
    for (int d = 32; d >= 1; d >>= 1) lo += __shfl(e, lo + d - 1) <= row ? d : 0;
    lo += __shfl(e, lo) <= row ? 1 : 0;
    if (!found && lo < 64) s = base + lo, found = true;
  }
  if (row >= total || s >= a.seqs) return;
  const int end = a.offs[s + 1];
  assign_row(a, there, row, s, a.lens[s] - (end - row), a.ws[a.seqs + s], a.ws[s]);
}

// ---------------------------------------------------------------------------
// Reordering behind beam search's choice
// ---------------------------------------------------------------------------

// What becomes of a group's beams, in the lanes of a wavefront: lane i < beams holds beam i's parent, and the beam
// whose partly filled page it goes on in: its parent's for a parent's first child, one without children for the others
// (there are as many).
struct Heirs {
  int parent, page_of;
  bool first;
};

__device__ __forceinline__ Heirs heirs_of(const int32_t* parents, int beams, int lane) {
  Heirs h{0, 0, true};
  if (lane < beams) h.parent = kv_clamp(parents[lane], 0, beams - 1);
  unsigned long long has = 0;   // parents with children
  for (int i = 0; i < beams; ++i) {
    const int p = __builtin_amdgcn_readlane(h.parent, i);
    if (i == lane) h.first = !((has >> p) & 1);
    has |= 1ull << p;
  }
  const unsigned long long below = (1ull << lane) - 1;
  const unsigned long long more = __ballot(lane < beams && !h.first);
  const unsigned long long none = __ballot(lane < beams && !((has >> lane) & 1));
  h.page_of = h.parent;
  if (lane < beams && !h.first) {   // the k-th further child takes the k-th parent without children
    unsigned long long m = none;
    for (int k = __popcll(more & below); k > 0; --k) m &= m - 1;
    h.page_of = __builtin_ctzll(m);
  }
  return h;
}

// A wavefront: 64 columns of a group's page tables, or of its token ids.  All
// beams' entries are read before any is written, so both work in place.  Bound by
// latency: parents, length, entries, stores; 48 groups of 8 over up to 1300 tokens 5.2 us.
__global__ __launch_bounds__(256) void k_beam_reorder(ReorderArgs a, int table_units, int units) {
  extern __shared__ int32_t lds_all[];
  const int lane = (int)threadIdx.x & 63, wave = (int)threadIdx.x >> 6, beams = a.beams;
  const int per = (units + 3) / 4, g = (int)(blockIdx.x / (unsigned)per);
  const int unit = (int)(blockIdx.x % (unsigned)per) * 4 + wave;
  if (unit >= units) return;   // no barrier follows
  int32_t* const lds = lds_all + wave * beams * 64;
  const int size = 1 << a.page_shift;
  const Heirs h = heirs_of(a.parents + (int64_t)g * beams, beams, lane);
  const int len = kv_clamp(a.lens[(int64_t)g * beams], 0, 0x7FFFFFFE);
  const bool is_ids = unit >= table_units;
  const int64_t row0 = (int64_t)g * beams;
  if (is_ids) {
    const int t = (unit - table_units) * 64 + lane;
    if (__builtin_amdgcn_readfirstlane(t) > len) return;
    const bool old = t < len && t < a.id_cols;
    if (old)
#pragma unroll 8
      for (int i = 0; i < beams; ++i) lds[i * 64 + lane] = a.ids[(row0 + i) * a.ldi + t];
    for (int i = 0; i < beams; ++i) {
      const int p = __builtin_amdgcn_readlane(h.parent, i);
      if (old) a.ids_out[(row0 + i) * a.ldio + t] = lds[p * 64 + lane];
      else if (t == len && t < a.id_cols) a.ids_out[(row0 + i) * a.ldio + t] = a.tokens[row0 + i];
    }
    return;
  }
  const int c = unit * 64 + lane, whole = len >> a.page_shift, part = len & (size - 1);
  const bool open = part != 0 && whole < a.cols;   // a page that is partly filled
  if (c < a.cols)
#pragma unroll 8
    for (int i = 0; i < beams; ++i) lds[i * 64 + lane] = a.table[(row0 + i) * a.ldt + c];
  wave_sync();
  if (c < a.cols)
    for (int i = 0; i < beams; ++i) {
      const int p = __builtin_amdgcn_readlane(h.parent, i), q = __builtin_amdgcn_readlane(h.page_of, i);
      const int from = c < whole ? p : c == whole && open ? q : i;
      a.table_out[(row0 + i) * a.ldto + c] = lds[from * 64 + lane];
    }
  // the copies, by the wavefront that has the partly filled pages' column
  if (unit != (open ? whole / 64 : 0) || lane >= beams || !a.copies) return;
  const bool copy = open && !h.first;
  int32_t* const to = a.copies + (row0 + lane) * 3;
  to[0] = copy ? lds[h.parent * 64 + whole % 64] : -1;
  to[1] = copy ? lds[h.page_of * 64 + whole % 64] : -1;
  to[2] = copy ? part : -1;
}

typedef uint32_t v4u __attribute__((ext_vector_type(4)));

// The first tokens of pages into other pages, keys and values of a head: a copy, a
// head and (large pages) a part of it to a workgroup.  384 entries of which 40% copy,
// 8 heads of 128 in E4M3, pages of 64: 5 us for 18 MB in and out (18.5 us with the values in
// an array that the compiler kept in LDS).
template <int F>
__global__ __launch_bounds__(256) void k_kv_copy(KvCacheArgs c, const int32_t* copies, int D, int parts) {
  const int tid = (int)threadIdx.x, part = (int)(blockIdx.x % (unsigned)parts);
  const int head = (int)(blockIdx.x / (unsigned)parts % (unsigned)c.heads);
  const int64_t j = blockIdx.x / (unsigned)parts / (unsigned)c.heads;
  const int src = copies[3 * j], dst = copies[3 * j + 1], n = kv_clamp(copies[3 * j + 2], 0, 1 << c.page_shift);
  if (src < 0 || src >= c.pages || dst < 0 || dst >= c.pages || src == dst || n == 0) return;
  const int64_t from = kv_row(src, 0, c.pages, c.heads, head, c.page_shift);
  const int64_t to = kv_row(dst, 0, c.pages, c.heads, head, c.page_shift);
  const int bytes = copy_row_bytes(D, F), chunks = n * (bytes / 16);   // of K, and of V
  const int begin = part * kCopyChunks, end = 2 * chunks < begin + kCopyChunks ? 2 * chunks : begin + kCopyChunks;
  if (begin >= end) return;
  v4u x[kCopyChunks / 256];
#pragma unroll
  for (int i = 0; i < kCopyChunks / 256; ++i) {   // without conditions: a place past the end reads the last one again
    const int at = begin + i * 256 + tid < end ? begin + i * 256 + tid : end - 1;
    const uint8_t* const row = (at < chunks ? c.k : c.v) + from * bytes;
    x[i] = *reinterpret_cast<const v4u*>(row + 16 * (int64_t)(at < chunks ? at : at - chunks));
  }
#pragma unroll
  for (int i = 0; i < kCopyChunks / 256; ++i) {
    const int at = begin + i * 256 + tid;
    uint8_t* const row = (at < chunks ? c.k : c.v) + to * bytes;
    if (at < end) *reinterpret_cast<v4u*>(row + 16 * (int64_t)(at < chunks ? at : at - chunks)) = x[i];
  }
  if (F == kKvBf16 || part != 0) return;
  // scales: bytes of K and of V
  const int per = F == kKvMx ? D / 32 : 1, scales = F == kKvMx ? n * per : (n + kF8Block - 1) / kF8Block;
  const int64_t sf = F == kKvMx ? from * per : from / kF8Block, st = F == kKvMx ? to * per : to / kF8Block;
  for (int i = tid; i < 2 * scales; i += 256) {
    uint8_t* const s = i < scales ? c.ks : c.vs;
    const int at = i < scales ? i : i - scales;
    s[st + at] = s[sf + at];
  }
}

// ---------------------------------------------------------------------------
// Launches
// ---------------------------------------------------------------------------

hipError_t launch_kv_assign(const AssignArgs& a, hipStream_t st) {
  if (assign_whole(a.seqs, a.rows)) {
    k_kv_assign<true><<<1, kAssignThreads, 0, st>>>(a);
    return hipGetLastError();
  }
  k_kv_assign<false><<<1, kAssignThreads, 0, st>>>(a);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  const bool maps = a.row_seq || a.positions || a.slots;
  const unsigned rows = maps ? (unsigned)(((int64_t)a.rows + 255) / 256) : 0;
  k_kv_assign_rows<<<rows + (unsigned)((a.seqs + 255) / 256), 256, 0, st>>>(a, rows);
  return hipGetLastError();
}

hipError_t launch_beam_reorder(const ReorderArgs& a, int64_t groups, hipStream_t st) {
  const int table_units = a.table ? (int)reorder_units(a.cols > 0 ? a.cols : 1) : 0;   // the first writes the copies too
  const int units = table_units + (a.ids ? (int)reorder_units(a.id_cols) : 0);
  const dim3 g((unsigned)(groups * ((units + 3) / 4)));
  k_beam_reorder<<<g, 256, 4 * a.beams * 64 * sizeof(int32_t), st>>>(a, table_units, units);
  return hipGetLastError();
}

hipError_t launch_kv_copy(const KvCacheArgs& c, const int32_t* copies, int64_t n, int D, int fmt, hipStream_t st) {
  const int parts = (int)copy_parts(1 << c.page_shift, D, fmt);
  const dim3 g((unsigned)(n * c.heads * parts));
  if (fmt == kKvBf16) k_kv_copy<kKvBf16><<<g, 256, 0, st>>>(c, copies, D, parts);
  else if (fmt == kKvMx) k_kv_copy<kKvMx><<<g, 256, 0, st>>>(c, copies, D, parts);
  else k_kv_copy<kKvF8><<<g, 256, 0, st>>>(c, copies, D, parts);
  return hipGetLastError();
}

}  // namespace sharq
