// Eviction: of the n_b rows of a request every KV head keeps m = min(n_b, budget): the first n_sink, the n_recent newest, and between them those of
// the largest accumulated weight (equal ones: the lower rows; NaN: as the least).  They move to the front, in order, and with them their weights.
//
// k_evict_plan, a workgroup a (request, KV head): the weight at the cut by three passes of a histogram over the bits of its order-preserving key,
// then the rows that are kept, in order: every wave has a stretch of the rows, counts what it keeps, and writes it behind what the waves
// before it keep.
// k_evict_move carries the rows.  In place (kept rows only ever move down) a workgroup takes a slice of 64 bytes of every row in order, a stretch at a
// time: all of it is read before any of it is written, and what later stretches read lies behind what this one writes.
#include "tile_attn.h"

namespace lfps {

namespace {

constexpr int kPlanThreads = 1024, kPlanWaves = kPlanThreads / 64, kBins = 2048;
constexpr int kMoveThreads = 512, kMoveU = 4;          // rows pieces of 16 bytes that a thread has on its way

__device__ __forceinline__ uint32_t weight_key(float x) { return x != x ? 0u : f2key(x + 0.f); }      // (-0 is 0)

struct Cut {
  int n, m, sinks, last, pick;         // rows; kept ones; kept first ones; where the kept newest begin; kept ones between
  __device__ __forceinline__ Cut(int n_, int budget, int n_sink, int n_recent) : n(n_) {
    m = budget < 0 ? 0 : (budget < n ? budget : n);
    sinks = n_sink < m ? n_sink : m;
    const int recent = n_recent < m - sinks ? n_recent : m - sinks;
    last = n - recent;
    pick = m - sinks - recent;
  }
};

}  // namespace

__global__ __launch_bounds__(kPlanThreads) void k_evict_plan(Shape s, const int32_t* __restrict__ seq_lens, const float* __restrict__ mass,
                                                             const int32_t* __restrict__ budget, int n_sink, int n_recent, float* __restrict__ mass_out,
                                                             int32_t* __restrict__ kept, int32_t* __restrict__ lens_out) {
  __shared__ int bins[kBins], sums[kPlanWaves][2], found[2];
  const int bg = blockIdx.x, b = bg / s.Hkv, tid = threadIdx.x, lane = tid & 63, wave = wave_of();
  const Cut cut(length_of(s, seq_lens, b), budget[b], n_sink, n_recent);
  if (bg % s.Hkv == 0 && tid == 0) lens_out[b] = cut.m;
  const float* const w = mass + (int64_t)bg * s.Lcap;
  // the key at the cut, from its highest bits down: `least` is its bits so far, `left` how many of those that have these bits are kept
  uint32_t least = 0;
  int left = cut.pick;
  if (left > 0) {
    int shift = 32;
    for (int pass = 0; pass < 3; ++pass) {
      const int bits = pass < 2 ? 11 : 10, before = shift;
      shift -= bits;
      for (int i = tid; i < kBins; i += kPlanThreads) bins[i] = 0;
      __syncthreads();
      for (int i = cut.sinks + tid; i < cut.last; i += kPlanThreads) {
        const uint32_t key = weight_key(w[i]);
        if (pass == 0 || key >> before == least >> before) atomicAdd(&bins[(key >> shift) & ((1 << bits) - 1)], 1);
      }
      __syncthreads();
      if (wave == 0) {                                       // lane l has the bins of the l-th highest part of them
        constexpr int kEach = kBins / 64;
        const int each = (1 << bits) / 64, top = (1 << bits) - 1 - lane * each;
        int sum = 0;
        for (int i = 0; i < each; ++i) sum += bins[top - i];
        int above = wave_inclusive_sum(sum) - sum;
        if (above < left && left <= above + sum) {
          int i = 0;
          while (above + bins[top - i] < left) above += bins[top - i++];
          found[0] = top - i;
          found[1] = left - above;
        }
        static_assert(kEach * 64 == kBins, "");
      }
      __syncthreads();
      least |= (uint32_t)found[0] << shift;
      left = found[1];
      __syncthreads();
    }
  }
  // of my wave's rows: kept whatever else is, and at the cut
  const int each = ((cut.n + kPlanWaves - 1) / kPlanWaves + 63) & ~63, from = wave * each, to = from + each < cut.n ? from + each : cut.n;
  auto look = [&](int i, float x, bool* at_cut) {
    const bool between = i >= cut.sinks && i < cut.last;
    const uint32_t key = weight_key(x);
    *at_cut = i < to && between && cut.pick > 0 && key == least;
    return i < to && (!between || (cut.pick > 0 && key > least));
  };
  int sure = 0, equal = 0;
  for (int i0 = from; i0 < to; i0 += 64) {
    const int i = i0 + lane;
    bool at_cut;
    const bool keep = look(i, w[i < to ? i : to - 1], &at_cut);
    sure += __popcll(__ballot(keep));
    equal += __popcll(__ballot(at_cut));
  }
  if (lane == 0) {
    sums[wave][0] = sure;
    sums[wave][1] = equal;
  }
  __syncthreads();
  int place = 0, equals = 0;
  for (int i = 0; i < wave; ++i) {
    place += sums[i][0];
    equals += sums[i][1];
  }
  place += equals < left ? equals : left;
  const uint64_t below = ((uint64_t)1 << lane) - 1;
  for (int i0 = from; i0 < to; i0 += 64) {
    const int i = i0 + lane;
    const float x = w[i < to ? i : to - 1];
    bool at_cut;
    const bool keep = look(i, x, &at_cut);
    const uint64_t same = __ballot(at_cut);
    const bool mine = keep || (at_cut && equals + __popcll(same & below) < left);
    const uint64_t all = __ballot(mine);
    if (mine) {
      const int64_t at = (int64_t)bg * s.Lcap + place + __popcll(all & below);
      kept[at] = i;
      mass_out[at] = x;
    }
    equals += __popcll(same);
    place += __popcll(all);
  }
}

// kInPlace: grid (slices of four pieces of K's row, then of V's; B * Hkv); else (parts of the kept rows; B * Hkv; K, V).
template <bool kInPlace>
__global__ __launch_bounds__(kMoveThreads) void k_evict_move(Shape s, KvView kv, KvView to, int k_bytes, int v_bytes, const int32_t* __restrict__ budget,
                                                             const int32_t* __restrict__ kept) {
  const int bg = blockIdx.y, b = bg / s.Hkv, g = bg % s.Hkv, n = length_of(s, kv.seq_lens, b);
  const int m = budget[b] < 0 ? 0 : (budget[b] < n ? budget[b] : n);
  if (kInPlace && m == n) return;
  constexpr int kSlice = 4;                                  // pieces of 16 bytes
  const int k_slices = kD * k_bytes / 16 / kSlice;
  const bool is_v = kInPlace ? (int)blockIdx.x >= k_slices : blockIdx.z == 1;
  const int esz = is_v ? v_bytes : k_bytes, pieces = kInPlace ? kSlice : kD * esz / 16;
  const int piece = (kInPlace ? kSlice * ((int)blockIdx.x - (is_v ? k_slices : 0)) : 0) + (int)threadIdx.x % pieces;
  const int rows = kMoveThreads / pieces;
  auto address = [&](const KvView& c, int i, bool* there) {
    const CacheRows<char> rows_of(is_v ? c.v : c.k, c, 0, 0);
    int64_t off = (int64_t)g * c.stride_h;
    *there = true;
    if (c.page.table) {
      const int e = RowMap<true>::block(c.page, b, i);
      *there = (uint32_t)e < (uint32_t)c.page.n_blocks;
      off += RowMap<true>::offset_in(c.page, e, i, c.stride_b, c.stride_n);
    } else {
      off += (int64_t)b * c.stride_b + (int64_t)i * c.stride_n;
    }
    return reinterpret_cast<u32x4*>(const_cast<char*>(rows_of.base) + off * esz) + piece;
  };
  const int32_t* const mine = kept + (int64_t)bg * s.Lcap;
  const int step = rows * kMoveU, first = kInPlace ? 0 : blockIdx.x * step, hop = kInPlace ? step : step * (int)gridDim.x;
  for (int i0 = first; i0 < m; i0 += hop) {
    u32x4 x[kMoveU];
    int from[kMoveU];
#pragma unroll
    for (int u = 0; u < kMoveU; ++u) {
      const int i = i0 + u * rows + (int)threadIdx.x / pieces;
      bool there;
      from[u] = i < m ? mine[i] : -1;
      if (from[u] >= 0) x[u] = *address(kv, from[u], &there);
    }
    if (kInPlace) {
      __builtin_amdgcn_s_waitcnt(0x0f70);                    // vmcnt(0): what I read is here
      __syncthreads();
    }
#pragma unroll
    for (int u = 0; u < kMoveU; ++u) {
      const int i = i0 + u * rows + (int)threadIdx.x / pieces;
      bool there = false;
      if (from[u] < 0 || (kInPlace && from[u] == i)) continue;
      u32x4* const at = address(to, i, &there);
      if (there) *at = x[u];
    }
    if (kInPlace) __syncthreads();
  }
}

hipError_t launch_evict(const Shape& s, int dtype, const KvView& kv, const float* mass, const int32_t* budget, int n_sink, int n_recent, const KvView* to,
                        float* mass_out, int32_t* kept, int32_t* lens_out, hipStream_t st) {
  const int e = dtype == LFPS_F32 ? 4 : 2, k_bytes = kv.k_fp8 ? 1 : e, v_bytes = kv.v_fp8 ? 1 : e;
  hipLaunchKernelGGL(k_evict_plan, dim3((unsigned)(s.B * s.Hkv)), dim3(kPlanThreads), 0, st, s, kv.seq_lens, mass, budget, n_sink, n_recent, mass_out, kept,
                     lens_out);
  if (!to) {
    const dim3 grid((unsigned)(kD * (k_bytes + v_bytes) / 64), (unsigned)(s.B * s.Hkv));
    hipLaunchKernelGGL((k_evict_move<true>), grid, dim3(kMoveThreads), 0, st, s, kv, kv, k_bytes, v_bytes, budget, kept);
  } else {
    const dim3 grid((unsigned)((s.Lcap + 255) / 256 < 64 ? (s.Lcap + 255) / 256 : 64), (unsigned)(s.B * s.Hkv), 2);
    hipLaunchKernelGGL((k_evict_move<false>), grid, dim3(kMoveThreads), 0, st, s, kv, *to, k_bytes, v_bytes, budget, kept);
  }
  return hipGetLastError();
}

}  // namespace lfps
