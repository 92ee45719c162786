// Eviction: of the n_b rows of a request every KV head keeps m = min(n_b, budget): the first n_sink, the n_recent newest, and between them those of
// the largest accumulated weight (equal ones: the lower rows; NaN: as the least).  They move to the front, in order, and with them their weights.
//
// k_evict_plan, a workgroup a (request, KV head), or where that leaves CUs without work several that all find the cut and share the rest: the weight at
// the cut by three passes of a histogram over the bits of its order-preserving key, then the rows that are kept, in order: every wave has a stretch of
// the rows, counts what it keeps, and writes it behind what the waves before it keep.  Up to 32768 rows stay in registers from the first pass to the last; of more, every pass reads them again.
// k_evict_move carries the rows.  In place (kept rows only ever move down) a workgroup takes a slice of every row in order, a stretch at a
// time: all of it is read before any of it is written, and what later stretches read lies behind what this one writes, so that they are asked
// for before it is.
//
// Few requests are bound by latency: one of 32768 rows cut to a quarter, 8 heads in bf16, 40 us: the plan 17.8 (keys read, three histograms of which each
// waits for the one before, list written), the move 22 (two stretches in a row; the bytes 14).  (Their first forms took 107 together; with
// the keys in LDS the plan took 38.)  Many are bound by the bytes: 32 requests of 300 to 9000 rows cut to about half into other FP8 pages,
// 0.44 GB 112 us: the plan 17, the move 80 to 91, 4.4 to 5 TB/s.
#include "tile_attn.h"

namespace lfps {

namespace {

constexpr int kPlanThreads = 1024, kPlanWaves = kPlanThreads / 64, kBins = 2048;
// Copies of a histogram, sixteen lanes each: weights of one octave are few bins, and additions to one of them are one after the other (32768 rows of 8
// heads, with what the waves left added up by a scan instead of sixteen reads: 21.1 -> 17.8 us).
constexpr int kCopies = 4;
constexpr int kPlanEach = 32, kPlanChunk = kPlanThreads * kPlanEach;       // weights of a thread; rows of the workgroup at a time
constexpr int kPlanBatch = 8;
constexpr int kMoveU = 8;                              // pieces of 16 bytes that a thread has on its way

__device__ __forceinline__ uint32_t weight_key(float x) { return x != x ? 1u : f2key(x + 0.f); }      // (-0 is 0; a NaN below all numbers)

// Of what the waves left: the sum of those before mine, and of all.
__device__ __forceinline__ int before_mine(const int (&sums)[kPlanWaves], int wave, int* all) {
  const int lane = threadIdx.x & 63, x = wave_inclusive_sum(lane < kPlanWaves ? sums[lane < kPlanWaves ? lane : 0] : 0);
  *all = __builtin_amdgcn_readlane(x, kPlanWaves - 1);
  return wave > 0 ? __builtin_amdgcn_readlane(x, wave - 1) : 0;
}

struct Cut {
  int n, m, sinks, last;               // rows; kept ones; kept first ones; where the kept newest begin
  __device__ __forceinline__ Cut(int n_, int budget, int n_sink, int n_recent) : n(n_) {
    m = budget < 0 ? 0 : (budget < n ? budget : n);
    sinks = n_sink < m ? n_sink : m;
    const int recent = n_recent < m - sinks ? n_recent : m - sinks;
    last = n - recent;
  }
};

}  // namespace

__global__ __launch_bounds__(kPlanThreads) void k_evict_plan(Shape s, const int32_t* __restrict__ seq_lens, const float* __restrict__ mass,
                                                             const int32_t* __restrict__ budget, int n_sink, int n_recent, float* __restrict__ mass_out,
                                                             int32_t* __restrict__ kept, int32_t* __restrict__ lens_out, int log2_shares) {
  __shared__ __attribute__((aligned(16))) int bins[kBins][kCopies];
  __shared__ int sums[2][kPlanWaves], found[2];
  const int bg = blockIdx.x, b = bg / s.Hkv, tid = threadIdx.x, lane = tid & 63, wave = wave_of();
  const Cut cut(length_of(s, seq_lens, b), budget[b], n_sink, n_recent);
  if (bg % s.Hkv == 0 && blockIdx.y == 0 && tid == 0) lens_out[b] = cut.m;
  if (cut.m == 0) return;
  // (behind the last row the loads give 0)
  const __amdgpu_buffer_rsrc_t w = __builtin_amdgcn_make_buffer_rsrc((void*)(mass + (int64_t)bg * s.Lcap), 0, 4 * cut.n, 0x00020000);
  // Chunk c's rows of a thread, `each` of them: row(c, i), in the order chunk, wave, i, lane.  Their keys: the first and the newest ones' above all,
  // those of rows that are not there below all.  So the m largest keys are kept, of equal ones the lower rows.
  const int chunks = (cut.n + kPlanChunk - 1) / kPlanChunk, each = chunks > 1 ? kPlanEach : (cut.n + kPlanThreads - 1) / kPlanThreads;
  uint32_t key[kPlanEach];
  auto row = [&](int c, int i) { return c * kPlanChunk + (wave * each + i) * 64 + lane; };
  auto weight = [&](int c, int i0, int i) { return (uint32_t)__builtin_amdgcn_raw_buffer_load_b32(w, 4 * row(c, i0) + 256 * i, 0, 0); };
  // f(i) for all i below `each` and some behind, whose keys are 0, in batches: a taken branch for every further i took longer than most f.
  // (The count is one that the compiler cannot know again: comparisons with it, kept for every loop, would fill the scalar registers.)
  auto batches = [&](auto f) __attribute__((always_inline)) {
    int e = each;
    asm volatile("" : "+s"(e));
#pragma unroll
    for (int i0 = 0; i0 < kPlanEach; i0 += kPlanBatch)
      if (i0 < e) f(i0);
  };
  auto fetch = [&](int c) __attribute__((always_inline)) {
    batches([&](int i0) __attribute__((always_inline)) {
#pragma unroll
      for (int i = 0; i < kPlanBatch; ++i) key[i0 + i] = weight(c, i0, i);
    });
    batches([&](int i0) __attribute__((always_inline)) {
#pragma unroll
      for (int i = i0; i < i0 + kPlanBatch; ++i) key[i] = weight_key(__uint_as_float(key[i]));
      const int r0 = row(c, i0) - lane;
      if (r0 < cut.sinks || r0 + 64 * kPlanBatch > cut.last || i0 + kPlanBatch > each) {
#pragma unroll
        for (int i = i0; i < i0 + kPlanBatch; ++i) {
          const int r = row(c, i);
          key[i] = r >= cut.n || i >= each ? 0u : (r < cut.sinks || r >= cut.last ? 0xFFFFFFFFu : key[i]);
        }
      }
    });
  };
  // The key at the cut, from its highest bits down: `least` is its bits so far, `left` how many of those that have these bits are kept; then the list.
  uint32_t least = 0, known = 0;                             // known: which bits
  int left = cut.m, shift = 32;
  int base = 0, equals_before = 0;                           // kept rows, and rows at the cut, of the chunks before
#pragma unroll 1
  for (int pass = 0; pass < 4; ++pass) {
    const int bits = pass < 2 ? 11 : 10;
    if (pass < 3) {
      shift -= bits;
      for (int i = tid; i < kBins; i += kPlanThreads) *reinterpret_cast<u32x4*>(bins[i]) = u32x4{0, 0, 0, 0};
      __syncthreads();
    }
#pragma unroll 1
    for (int c = 0; c < chunks; ++c) {
      if (chunks > 1 || pass == 0) fetch(c);
      if (pass < 3) {
        const uint32_t mask = (1u << bits) - 1;
        batches([&](int i0) __attribute__((always_inline)) {
#pragma unroll
          for (int i = i0; i < i0 + kPlanBatch; ++i)
            if (key[i] && ((key[i] ^ least) & known) == 0) atomicAdd(&bins[(key[i] >> shift) & mask][lane % kCopies], 1);
        });
        continue;
      }
      // of my wave's rows: kept whatever else is, and in the upper half those at the cut (at most 2048 of either); and of those before my part
      const int all_batches = (each + kPlanBatch - 1) / kPlanBatch;
      const int part0 = (all_batches * (int)blockIdx.y >> log2_shares) * kPlanBatch, part1 = (all_batches * ((int)blockIdx.y + 1) >> log2_shares) * kPlanBatch;
      int mine = 0, early = 0;
      batches([&](int i0) __attribute__((always_inline)) {
        early = i0 == part0 ? mine : early;
#pragma unroll
        for (int i = i0; i < i0 + kPlanBatch; ++i) mine += key[i] > least ? 1 : (key[i] == least ? 1 << 16 : 0);
      });
      mine = wave_inclusive_sum(mine);
      early = __builtin_amdgcn_readlane(wave_inclusive_sum(early), 63);
      if (lane == 63) {
        sums[0][wave] = mine & 0xFFFF;
        sums[1][wave] = mine >> 16;
      }
      __syncthreads();
      int all_sure, all_equal;
      int place = base + before_mine(sums[0], wave, &all_sure), equals = equals_before + before_mine(sums[1], wave, &all_equal);
      place += early & 0xFFFF;
      equals += early >> 16;
      // (base counts the rows at the cut that were kept)
      place += (equals < left ? equals : left) - (equals_before < left ? equals_before : left);
      int32_t* const to = kept + (int64_t)bg * s.Lcap;
      float* const to_mass = mass_out + (int64_t)bg * s.Lcap;
      auto rank = [](uint64_t mask) { return (int)__builtin_amdgcn_mbcnt_hi((uint32_t)(mask >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)mask, 0)); };
      batches([&](int i0) __attribute__((always_inline)) {
        if (i0 < part0 || i0 >= part1) return;
        uint32_t x[kPlanBatch];
#pragma unroll
        for (int i = 0; i < kPlanBatch; ++i) x[i] = weight(c, i0, i);
#pragma unroll
        for (int i = 0; i < kPlanBatch; ++i) {
          const uint32_t k = key[i0 + i];
          const uint64_t same = __ballot(k == least);
          bool keep = k > least;
          if (same) keep = keep || (k == least && equals + rank(same) < left);
          const uint64_t all = __ballot(keep);
          if (keep) {
            const int at = place + rank(all);
            to[at] = row(c, i0 + i);
            to_mass[at] = __uint_as_float(x[i]);
          }
          equals += __popcll(same);
          place += __popcll(all);
        }
      });
      const int equals_after = equals_before + all_equal;
      base += all_sure + (equals_after < left ? equals_after : left) - (equals_before < left ? equals_before : left);
      equals_before = equals_after;
      __syncthreads();
    }
    if (pass == 3) break;
    __syncthreads();
    // thread t has the t-th highest bin or two: those above them come from the threads before
    auto bin = [&](int i) {
      const u32x4 x = *reinterpret_cast<const u32x4*>(bins[i]);
      return (int)((x[0] + x[1]) + (x[2] + x[3]));
    };
    const int mine = (1 << bits) / kPlanThreads, top = (1 << bits) - 1 - tid * mine, high = bin(top), low = mine > 1 ? bin(top - 1) : 0;
    int above = wave_inclusive_sum(high + low), all;
    if (lane == 63) sums[0][wave] = above;
    above -= high + low;
    __syncthreads();
    above += before_mine(sums[0], wave, &all);
    if (above < left && left <= above + high + low) {
      const bool second = left > above + high;
      found[0] = top - second;
      found[1] = left - above - (second ? high : 0);
    }
    __syncthreads();
    least |= (uint32_t)found[0] << shift;
    known |= ((1u << bits) - 1) << shift;
    left = found[1];
    __syncthreads();
  }
}

// A workgroup moves `slice` pieces of 16 bytes of every kept row: grid (B * Hkv; slices of K's row, then of V's; in place: 1, else parts of the kept
// rows).  A group's slices come from one XCD, where they share the lines that they do not fill.
template <bool kInPlace, int kThreads>
__global__ __launch_bounds__(kThreads) void k_evict_move(Shape s, KvView kv, KvView to, int k_bytes, int v_bytes, int slice, const int32_t* __restrict__ budget,
                                                         const int32_t* __restrict__ kept) {
  const int bg = blockIdx.x, b = bg / s.Hkv, g = bg % s.Hkv, n = length_of(s, kv.seq_lens, b);
  const int m = budget[b] < 0 ? 0 : (budget[b] < n ? budget[b] : n);
  if (kInPlace && m == n) return;
  const int k_slices = kD * k_bytes / 16 / slice;
  const bool is_v = (int)blockIdx.y >= k_slices;
  const int esz = is_v ? v_bytes : k_bytes, piece = slice * ((int)blockIdx.y - (is_v ? k_slices : 0)) + (int)threadIdx.x % slice;
  const int rows = kThreads / slice, step = rows * kMoveU, mine = (int)threadIdx.x / slice;
  const int64_t group = (int64_t)g * kv.stride_h, group_to = (int64_t)g * to.stride_h;
  const char* const from_base = (const char*)(is_v ? kv.v : kv.k) + 16 * piece;
  char* const to_base = (char*)const_cast<void*>(is_v ? to.v : to.k) + 16 * piece;
  const int32_t* const list = kept + (int64_t)bg * s.Lcap;
  const int first = kInPlace ? 0 : (int)blockIdx.z * step, end = kInPlace ? m : (first + step < m ? first + step : m);
  if (first >= end) return;
  struct Stretch {
    int from[kMoveU];
    u32x4 x[kMoveU];
  };
  auto look = [&](int i0, int (&from)[kMoveU]) {              // rows that do not move, or are not there: -1
#pragma unroll
    for (int u = 0; u < kMoveU; ++u) {
      const int i = i0 + u * rows + mine;
      from[u] = list[i < end ? i : end - 1];
      if (i >= end || (kInPlace && from[u] == i)) from[u] = -1;
    }
  };
  auto read = [&](Stretch& t) {
    int64_t off[kMoveU];
#pragma unroll
    for (int u = 0; u < kMoveU; ++u) {
      const int r = t.from[u] < 0 ? 0 : t.from[u];
      off[u] = kv.page.table ? RowMap<true>::offset_in(kv.page, RowMap<true>::block(kv.page, b, r), r, kv.stride_b, kv.stride_n)
                             : (int64_t)b * kv.stride_b + (int64_t)r * kv.stride_n;
    }
#pragma unroll
    for (int u = 0; u < kMoveU; ++u)
      if (t.from[u] >= 0) t.x[u] = *reinterpret_cast<const u32x4*>(from_base + (group + off[u]) * esz);
  };
  auto write = [&](int i0, const Stretch& t) {
#pragma unroll
    for (int u = 0; u < kMoveU; ++u) {
      const int i = i0 + u * rows + mine;
      if (t.from[u] < 0) continue;
      int64_t off = (int64_t)b * to.stride_b + (int64_t)i * to.stride_n;
      if (to.page.table) {
        const int e = RowMap<true>::block(to.page, b, i);
        if ((uint32_t)e >= (uint32_t)to.page.n_blocks) continue;
        off = RowMap<true>::offset_in(to.page, e, i, to.stride_b, to.stride_n);
      }
      *reinterpret_cast<u32x4*>(to_base + (group_to + off) * esz) = t.x[u];
    }
  };
  Stretch t;
  look(first, t.from);
  read(t);
  if constexpr (!kInPlace) {
    write(first, t);
  } else {
    for (int i0 = 0;; i0 += step) {
      const bool more = i0 + step < end;
      Stretch next;
      if (more) look(i0 + step, next.from);
      __builtin_amdgcn_s_waitcnt(0x0f70);                    // vmcnt(0): what I read is here
      __syncthreads();                                       // ... and what the others read
      if (more) read(next);                                  // (rows behind those that are written now)
      write(i0, t);
      if (!more) break;
      t = next;
    }
  }
}

hipError_t launch_evict(const Shape& s, int dtype, const KvView& kv, const float* mass, const int32_t* budget, int n_sink, int n_recent, const KvView* to,
                        float* mass_out, int32_t* kept, int32_t* lens_out, hipStream_t st) {
  const int e = dtype == LFPS_F32 ? 4 : 2, k_bytes = kv.k_fp8 ? 1 : e, v_bytes = kv.v_fp8 ? 1 : e;
  const int groups = s.B * s.Hkv, pieces = kD * (k_bytes < v_bytes ? k_bytes : v_bytes) / 16;
  const int log2_shares = groups <= 64 ? 2 : (groups <= 128 ? 1 : 0);
  hipLaunchKernelGGL(k_evict_plan, dim3((unsigned)groups, 1u << log2_shares), dim3(kPlanThreads), 0, st, s, kv.seq_lens, mass, budget, n_sink, n_recent, mass_out, kept, lens_out,
                     log2_shares);
  if (!to) {
    // the widest slices that give every CU a workgroup, of at least half a 64-byte piece of memory (one request of 32768 rows cut to a quarter, 8 heads
    // in bf16: of 64 bytes 46.5 us in all, of 32 43.0, of 16 45.5; the group's XCD has both halves)
    int slice = 2;
    while (slice < pieces && (int64_t)groups * kD * (k_bytes + v_bytes) / 16 / (2 * slice) >= 256) slice *= 2;
    const dim3 grid((unsigned)groups, (unsigned)(kD * (k_bytes + v_bytes) / 16 / slice));
    hipLaunchKernelGGL((k_evict_move<true, 1024>), grid, dim3(1024), 0, st, s, kv, kv, k_bytes, v_bytes, slice, budget, kept);
  } else {
    const int step = 256 / pieces * kMoveU;
    const dim3 grid((unsigned)groups, (unsigned)(kD * (k_bytes + v_bytes) / 16 / pieces), (unsigned)((s.Lcap + step - 1) / step));
    hipLaunchKernelGGL((k_evict_move<false, 256>), grid, dim3(256), 0, st, s, kv, *to, k_bytes, v_bytes, pieces, budget, kept);
  }
  return hipGetLastError();
}

}  // namespace lfps
