// Pages of a cache: which block holds which rows of whom.  The whole state is the view's block table and lengths (and the blocks
// that the caller holds for itself): who uses a block is counted from them in every call, so nothing can drift from it.
//
// An update makes the next table from the last one: request b continues request parent[b] (itself, another: a fork, none: it
// ends) with new_lens[b] rows.  Blocks are only taken from those that nobody used before the call, in rising order, so
// what a copy reads is never what another copy writes.  A half-filled block that a request will write into and others keep is
// copied for it; of several that all write into it the one with the most rows there (of those, the first) keeps it: whatever it appends
// lies behind the others' rows, also of those for whose copy no block is left and who stay in this one.
// A compaction moves the live blocks behind the front into the holes of the front, both in rising order.
//
// All of it is whole numbers, and none depends on the order of atomics.  A few dependent launches over 4 bytes an entry of the
// table and 13 a block of the pool: bound by the launches.  The copies are bound by the bytes.  64 requests over a pool of 65536 blocks:
// an update 2 + 4 + 5 + 3.5 + 5.5 us and a copy of their tails 4; a compaction's plan 29 us in six launches, its copy of 1.9 GB (read and written) 370, 5.1 TB/s.
#include "lfps_internal.h"

namespace lfps {

namespace {

constexpr int kPageThreads = 256;
constexpr int kChunk = 4096;               // blocks of the pool that a workgroup counts: 16 a thread

struct PagesArgs {
  Shape s;
  KvPage pg;
  const int32_t* seq_lens;
  const int32_t* held;                     // [n_blocks] or NULL
  const int32_t* parent;                   // [B] or NULL: every request continues itself
  const int32_t* new_lens;                 // [B]
  int32_t n_chunks;
  // workspace
  uint8_t* live;                           // [n_blocks] used by the table, or held
  int32_t* writers;                        // [n_blocks] requests that will write into this half-filled block
  int32_t* holders;                        // [n_blocks] entries of the new table with it, where there are writers
  uint32_t* keeper;                        // [n_blocks] the largest writer_rank of them
  int32_t* list;                           // [n_blocks] free blocks; compaction: holes, from n_blocks / 2 on movers
  int32_t* chunk;                          // [n_chunks] free (compaction: live) blocks of every chunk
};

__device__ __forceinline__ int length_of(const PagesArgs& a, int b) {
  const int n = a.seq_lens[b];
  return n < 0 ? 0 : (n > a.s.Lcap ? a.s.Lcap : n);
}
__device__ __forceinline__ int blocks_of(const PagesArgs& a, int rows) { return (int)(((int64_t)rows + (1 << a.pg.shift) - 1) >> a.pg.shift); }
__device__ __forceinline__ int entry_of(const PagesArgs& a, int b, int j) {
  return RowMap<true>::kept_in_pool(a.pg, a.pg.table[(int64_t)b * a.pg.table_stride + j]);
}
__device__ __forceinline__ bool is_held(const PagesArgs& a, int x) { return a.held && a.held[x] != 0; }

// What becomes of request b.
struct Next {
  int parent, rows, length;                // rows kept of the parent's; rows wanted
  int kept, wanted;                        // the same in blocks
  int tail;                                // the half-filled block that it will write into, or -1
};
// Rows of its last kept block, 0 where that is full.
__device__ __forceinline__ int rows_in_tail(const PagesArgs& a, const Next& x) { return x.rows & ((1 << a.pg.shift) - 1); }
__device__ __forceinline__ Next next_of(const PagesArgs& a, int b) {
  Next x;
  x.parent = a.parent ? a.parent[b] : b;
  const bool ends = x.parent < 0 || x.parent >= a.s.B;
  x.parent = ends ? 0 : x.parent;
  const int n = length_of(a, x.parent), want = a.new_lens[b];
  x.length = ends || want < 0 ? 0 : (want > a.s.Lcap ? a.s.Lcap : want);
  x.rows = n < x.length ? n : x.length;
  x.kept = blocks_of(a, x.rows);
  x.wanted = blocks_of(a, x.length);
  x.tail = x.length > x.rows && rows_in_tail(a, x) ? entry_of(a, x.parent, x.kept - 1) : -1;
  return x;
}
// Who of a block's writers comes first: who has more rows in it, then the lower number (either below 2^16).
__device__ __forceinline__ uint32_t writer_rank(const PagesArgs& a, int b, const Next& x) { return (uint32_t)rows_in_tail(a, x) << 16 | (uint32_t)(a.s.B - b); }
// Does it get a copy of that block?  (After the counting.)
__device__ __forceinline__ bool copies(const PagesArgs& a, int b, const Next& x) {
  return x.tail >= 0 && (is_held(a, x.tail) || a.holders[x.tail] > a.writers[x.tail] || a.keeper[x.tail] != writer_rank(a, b, x));
}

// Sum over the workgroup, in every thread.
__device__ __forceinline__ int block_sum(int x) {
  __shared__ int part[kPageThreads / 64];
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) x += __shfl_xor(x, d);
  __syncthreads();
  if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = x;
  __syncthreads();
  int sum = 0;
#pragma unroll
  for (int w = 0; w < kPageThreads / 64; ++w) sum += part[w];
  return sum;
}
// Sum over the threads before mine.
__device__ __forceinline__ int block_before(int x) {
  __shared__ int part[kPageThreads / 64];
  const int incl = wave_inclusive_sum(x), wave = threadIdx.x >> 6;
  __syncthreads();
  if ((threadIdx.x & 63) == 63) part[wave] = incl;
  __syncthreads();
  int before = incl - x;
#pragma unroll
  for (int w = 0; w < kPageThreads / 64; ++w) before += w < wave ? part[w] : 0;
  return before;
}

// The marks of my 16 blocks of a chunk, bit i: block 16 tid + i is live; and which of them exist.
__device__ __forceinline__ uint32_t live_bits(const PagesArgs& a, int chunk, uint32_t* there) {
  const int x0 = chunk * kChunk + 16 * (int)threadIdx.x, n = a.pg.n_blocks - x0;
  uint32_t bits = 0;
  *there = n >= 16 ? 0xFFFFu : (n <= 0 ? 0u : (1u << n) - 1u);
  if (n <= 0) return 0;
  const u32x4 w = *reinterpret_cast<const u32x4*>(a.live + x0);            // (the marks are padded to whole chunks)
#pragma unroll
  for (int i = 0; i < 16; ++i) bits |= ((w[i / 4] >> (8 * (i % 4))) & 1u) << i;
  if (a.held) {
    for (int i = 0; i < 16 && i < n; ++i) bits |= (a.held[x0 + i] != 0 ? 1u : 0u) << i;
  }
  return bits & *there;
}

}  // namespace

__global__ __launch_bounds__(kPageThreads) void k_pages_clear(u32x4* p, int64_t n) {
  const int64_t i = (int64_t)blockIdx.x * kPageThreads + threadIdx.x;
  if (i < n) p[i] = u32x4{0, 0, 0, 0};
}

// grid (parts of a row of the table, B): who is used now, and who will be written into
__global__ __launch_bounds__(kPageThreads) void k_pages_mark(PagesArgs a) {
  const int b = blockIdx.y, used = blocks_of(a, length_of(a, b));
  for (int j = blockIdx.x * kPageThreads + threadIdx.x; j < used; j += gridDim.x * kPageThreads) a.live[entry_of(a, b, j)] = 1;
  if (a.new_lens && blockIdx.x == 0 && threadIdx.x == 0) {
    const Next x = next_of(a, b);
    if (x.tail >= 0) {
      atomicAdd(a.writers + x.tail, 1);
      atomicMax(a.keeper + x.tail, writer_rank(a, b, x));
    }
  }
}

// grid: the chunks of the pool, then (update) B * parts of the rows of the table
__global__ __launch_bounds__(kPageThreads) void k_pages_count(PagesArgs a, int parts) {
  if ((int)blockIdx.x < a.n_chunks) {
    uint32_t there;
    const uint32_t live = live_bits(a, blockIdx.x, &there);
    const int n = block_sum(__popc(a.new_lens ? there & ~live : live));
    if (threadIdx.x == 0) a.chunk[blockIdx.x] = n;
    return;
  }
  const int x = blockIdx.x - a.n_chunks, b = x / parts;
  const Next next = next_of(a, b);
  for (int j = (x % parts) * kPageThreads + threadIdx.x; j < next.kept; j += parts * kPageThreads) {
    const int e = entry_of(a, next.parent, j);
    if (a.writers[e] > 0) atomicAdd(a.holders + e, 1);
  }
}

// grid n_chunks: the free blocks in order
__global__ __launch_bounds__(kPageThreads) void k_pages_free_list(PagesArgs a) {
  int before = 0;
  for (int c = threadIdx.x; c < (int)blockIdx.x; c += kPageThreads) before += a.chunk[c];
  before = block_sum(before);
  uint32_t there;
  const uint32_t live = live_bits(a, blockIdx.x, &there);
  uint32_t free = there & ~live;
  int at = before + block_before(__popc(free));
  for (; free; free &= free - 1) a.list[at++] = blockIdx.x * kChunk + 16 * threadIdx.x + __ffs(free) - 1;
}

// grid (parts of a row, B): the new table, lengths and copies
__global__ __launch_bounds__(kPageThreads) void k_pages_write(PagesArgs a, int32_t* __restrict__ table_out, int32_t* __restrict__ lens_out,
                                                              int32_t* __restrict__ copies_out, int32_t* flags) {
  const int b = blockIdx.y;
  int before = 0, free = 0;
  for (int i = threadIdx.x; i < b; i += kPageThreads) {
    const Next x = next_of(a, i);
    before += (copies(a, i, x) ? 1 : 0) + x.wanted - x.kept;
  }
  before = block_sum(before);
  for (int c = threadIdx.x; c < a.n_chunks; c += kPageThreads) free += a.chunk[c];
  free = block_sum(free);
  const Next x = next_of(a, b);
  const int copy = copies(a, b, x) ? 1 : 0, need = copy + x.wanted - x.kept;
  int got = free - before;
  got = got < 0 ? 0 : (got > need ? need : got);
  const bool copied = copy && got > 0;
  const int grown = copy && !copied ? 0 : got - copy;                  // new blocks behind the kept ones
  const int32_t* mine = a.list + before;
  for (int j = blockIdx.x * kPageThreads + threadIdx.x; j < a.pg.table_stride; j += gridDim.x * kPageThreads) {
    int e = -1;
    if (j < x.kept) e = copied && j == x.kept - 1 ? mine[0] : entry_of(a, x.parent, j);
    else if (j < x.kept + grown) e = mine[copy + j - x.kept];
    table_out[(int64_t)b * a.pg.table_stride + j] = e;
  }
  if (blockIdx.x == 0 && threadIdx.x == 0) {
    int length = x.length;
    if (got < need) {
      const int64_t room = (int64_t)(x.kept + grown) << a.pg.shift;
      length = copy && !copied ? x.rows : (room < length ? (int)room : length);
      atomicOr(flags, LFPS_FLAG_PAGES_FULL);
    }
    lens_out[b] = length;
    copies_out[3 * b] = copied ? x.tail : -1;
    copies_out[3 * b + 1] = copied ? mine[0] : -1;
    copies_out[3 * b + 2] = copied ? rows_in_tail(a, x) : 0;
  }
}

namespace {
// Live blocks in all, and those of them in front: below that number.
__device__ __forceinline__ void live_totals(const PagesArgs& a, int* total, int* front) {
  int n = 0, f = 0;
  for (int c = threadIdx.x; c < a.n_chunks; c += kPageThreads) n += a.chunk[c];
  n = block_sum(n);
  const int edge = n / kChunk;                                          // the chunk in which the front ends
  for (int c = threadIdx.x; c < edge; c += kPageThreads) f += a.chunk[c];
  if (edge < a.n_chunks) {
    uint32_t there;
    const uint32_t live = live_bits(a, edge, &there);
    const int below = n - (edge * kChunk + 16 * (int)threadIdx.x);       // of my 16 blocks
    f += __popc(live & (below >= 16 ? 0xFFFFu : (below <= 0 ? 0u : (1u << below) - 1u)));
  }
  *total = n;
  *front = block_sum(f);
}
}  // namespace

// grid n_chunks: holes of the front and live blocks behind it, both in order
__global__ __launch_bounds__(kPageThreads) void k_pages_move_lists(PagesArgs a) {
  int total, front, before = 0;
  live_totals(a, &total, &front);
  for (int c = threadIdx.x; c < (int)blockIdx.x; c += kPageThreads) before += a.chunk[c];
  before = block_sum(before);
  uint32_t there;
  const uint32_t live = live_bits(a, blockIdx.x, &there);
  int rank = before + block_before(__popc(live));                       // live blocks below mine
  const int x0 = blockIdx.x * kChunk + 16 * (int)threadIdx.x;
  int32_t* movers = a.list + a.pg.n_blocks / 2;
  for (int i = 0; i < 16; ++i) {
    if (!(there >> i & 1u)) break;
    const int x = x0 + i;
    if (live >> i & 1u) {
      if (x >= total) movers[rank - front] = x;
      ++rank;
    } else if (x < total) {
      a.list[x - rank] = x;
    }
  }
}

// grid: blocks of the pool, 256 a workgroup: the moves and where every block is afterwards
__global__ __launch_bounds__(kPageThreads) void k_pages_moves(PagesArgs a, int32_t* __restrict__ moves, int32_t* __restrict__ map,
                                                              int32_t* __restrict__ n_live) {
  int total, front;
  live_totals(a, &total, &front);
  const int x = blockIdx.x * kPageThreads + threadIdx.x;
  if (x == 0) *n_live = total;
  if (x >= a.pg.n_blocks) return;
  const bool live = a.live[x] != 0 || is_held(a, x);
  if (x < total || !live) map[x] = live ? x : -1;                        // (a mover's is written by its move)
  if (x < a.pg.n_blocks / 2) {
    const bool there = x < total - front;
    const int from = there ? a.list[a.pg.n_blocks / 2 + x] : -1, to = there ? a.list[x] : -1;
    if (there) map[from] = to;
    moves[3 * (int64_t)x] = from;
    moves[3 * (int64_t)x + 1] = to;
    moves[3 * (int64_t)x + 2] = there ? 1 << a.pg.shift : 0;
  }
}

// grid (parts of a row, B)
__global__ __launch_bounds__(kPageThreads) void k_pages_rename(PagesArgs a, const int32_t* __restrict__ map, int32_t* __restrict__ table_out) {
  const int b = blockIdx.y, used = blocks_of(a, length_of(a, b));
  for (int j = blockIdx.x * kPageThreads + threadIdx.x; j < a.pg.table_stride; j += gridDim.x * kPageThreads)
    table_out[(int64_t)b * a.pg.table_stride + j] = j < used ? map[entry_of(a, b, j)] : -1;
}

// grid (list entries in turn, shares of an entry's (K or V, KV head)): the first rows of a block into another
__global__ __launch_bounds__(kPageThreads) void k_pages_copy(KvView kv, int Hkv, int elem_k, int elem_v, const int32_t* __restrict__ list, int n) {
  for (int i = blockIdx.x; i < n; i += gridDim.x) {
    const int from = list[3 * (int64_t)i], to = list[3 * (int64_t)i + 1];
    int rows = list[3 * (int64_t)i + 2];
    if (from < 0 || to < 0 || from >= kv.page.n_blocks || to >= kv.page.n_blocks || from == to || rows <= 0) continue;
    rows = rows > 1 << kv.page.shift ? 1 << kv.page.shift : rows;
    for (int w = blockIdx.y; w < 2 * Hkv; w += gridDim.y) {
      const bool is_v = w >= Hkv;
      const int g = is_v ? w - Hkv : w, elem = is_v ? elem_v : elem_k;
      const char* src = (const char*)(is_v ? kv.v : kv.k);
      const int64_t at = ((int64_t)from * kv.stride_b + (int64_t)g * kv.stride_h) * elem, pitch = kv.stride_n * elem;
      const int64_t move = ((int64_t)to - from) * kv.stride_b * elem;
      const int per = kD * elem / 16, shift = elem == 4 ? 5 : (elem == 2 ? 4 : 3);     // 16-byte pieces of a row
      for (int p = threadIdx.x; p < rows * per; p += kPageThreads) {
        const char* x = src + at + (int64_t)(p >> shift) * pitch + 16 * (p & (per - 1));
        *reinterpret_cast<u32x4*>(const_cast<char*>(x) + move) = *reinterpret_cast<const u32x4*>(x);
      }
    }
  }
}

namespace {

int64_t align16(int64_t x) { return (x + 15) & ~(int64_t)15; }
int64_t chunks_of(int n_blocks) { return ((int64_t)n_blocks + kChunk - 1) / kChunk; }

PagesArgs pages_args(const Shape& s, const KvView& kv, const int32_t* held, void* work) {
  PagesArgs a = {};
  a.s = s;
  a.pg = kv.page;
  a.seq_lens = kv.seq_lens;
  a.held = held;
  const int64_t n = kv.page.n_blocks;
  a.n_chunks = (int)chunks_of(kv.page.n_blocks);
  char* p = (char*)work;
  a.live = (uint8_t*)p;
  p += (int64_t)a.n_chunks * kChunk;
  a.writers = (int32_t*)p;
  p += align16(4 * n);
  a.holders = (int32_t*)p;
  p += align16(4 * n);
  a.keeper = (uint32_t*)p;
  p += align16(4 * n);
  a.list = (int32_t*)p;
  p += align16(4 * n);
  a.chunk = (int32_t*)p;
  return a;
}
// Workgroups for a row of the table: 1024 entries each.
int row_parts(const KvPage& pg) { return (pg.table_stride + 1023) / 1024; }

void clear_counts(const PagesArgs& a, hipStream_t st) {
  // the marks; of an update the three counts behind them too
  const int64_t n = ((int64_t)a.n_chunks * kChunk + (a.new_lens ? 3 * align16(4 * (int64_t)a.pg.n_blocks) : 0)) / 16;
  hipLaunchKernelGGL(k_pages_clear, dim3((unsigned)((n + kPageThreads - 1) / kPageThreads)), dim3(kPageThreads), 0, st, (u32x4*)a.live, n);
}

}  // namespace

int64_t pages_workspace_bytes(int32_t n_blocks) {
  return chunks_of(n_blocks) * kChunk + 4 * align16(4 * (int64_t)n_blocks) + align16(4 * chunks_of(n_blocks));
}

hipError_t launch_pages_update(const Shape& s, const KvView& kv, const int32_t* parent, const int32_t* new_lens, const int32_t* held,
                               int32_t* table_out, int32_t* lens_out, int32_t* copies_out, void* work, int32_t* flags, hipStream_t st) {
  PagesArgs a = pages_args(s, kv, held, work);
  a.parent = parent;
  a.new_lens = new_lens;
  const int parts = row_parts(kv.page);
  const dim3 rows((unsigned)parts, (unsigned)s.B);
  clear_counts(a, st);
  hipLaunchKernelGGL(k_pages_mark, rows, dim3(kPageThreads), 0, st, a);
  hipLaunchKernelGGL(k_pages_count, dim3((unsigned)(a.n_chunks + s.B * parts)), dim3(kPageThreads), 0, st, a, parts);
  hipLaunchKernelGGL(k_pages_free_list, dim3((unsigned)a.n_chunks), dim3(kPageThreads), 0, st, a);
  hipLaunchKernelGGL(k_pages_write, rows, dim3(kPageThreads), 0, st, a, table_out, lens_out, copies_out, flags);
  return hipGetLastError();
}

hipError_t launch_pages_compact(const Shape& s, const KvView& kv, const int32_t* held, int32_t* table_out, int32_t* moves, int32_t* map,
                                int32_t* n_live, void* work, hipStream_t st) {
  const PagesArgs a = pages_args(s, kv, held, work);
  const dim3 rows((unsigned)row_parts(kv.page), (unsigned)s.B);
  clear_counts(a, st);
  hipLaunchKernelGGL(k_pages_mark, rows, dim3(kPageThreads), 0, st, a);
  hipLaunchKernelGGL(k_pages_count, dim3((unsigned)a.n_chunks), dim3(kPageThreads), 0, st, a, 1);
  hipLaunchKernelGGL(k_pages_move_lists, dim3((unsigned)a.n_chunks), dim3(kPageThreads), 0, st, a);
  hipLaunchKernelGGL(k_pages_moves, dim3((unsigned)((a.pg.n_blocks + kPageThreads - 1) / kPageThreads)), dim3(kPageThreads), 0, st, a, moves, map, n_live);
  hipLaunchKernelGGL(k_pages_rename, rows, dim3(kPageThreads), 0, st, a, map, table_out);
  return hipGetLastError();
}

hipError_t launch_pages_copy(const Shape& s, int dtype, const KvView& kv, const int32_t* list, int n, hipStream_t st) {
  const int elem = dtype == LFPS_F32 ? 4 : 2;
  int shares = 2 * s.Hkv;                                    // of a short list, so that the chip is filled
  while (shares > 1 && (int64_t)n * shares > 4096) shares = (shares + 1) / 2;
  hipLaunchKernelGGL(k_pages_copy, dim3((unsigned)(n < 4096 ? n : 4096), (unsigned)shares), dim3(kPageThreads), 0, st, kv, s.Hkv,
                     kv.k_fp8 ? 1 : elem, kv.v_fp8 ? 1 : elem, list, n);
  return hipGetLastError();
}

}  // namespace lfps
