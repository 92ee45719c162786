// One decode step's full attention over all n_b rows (as the full-attention baseline) for a batch in which groups of requests share
// their first rows: those are read once for a group, not once for every request, and its members' query heads are rows of one product.
//
//   part 1  per group, KV head and part of the shared rows: up to 256 query rows (members x heads) against them (k_prefix_shared)
//   part 2  per item of a request's own rows and KV head: its G heads against those (attention.hip)
//   part 3  the parts of a (request, head) joined:  o = sum_i e^(m_i - m) acc_i / sum_i e^(m_i - m) l_i
//
// Bound by the bytes of K and V, read once, while a group has few members; by the matrix units where it has many.  The query stays
// fp32, as a sum of 16-bit terms, and so do the weights (tile_attn.h): the results are fp32 ones as everywhere in the library, 0.4 to 1.5e-6
// from 64 bits where fp32 sums of the same rows are 0.5 to 2.6e-6.
//
// 32 heads over 8 KV heads: 64 requests over 32768 shared rows and 28267 own ones in bf16 127 us (part 1 86: 1000 TFLOP/s, of five products
// where two would do in 16 bits; part 2 29, 4.0 TB/s; part 3 9), 32 requests in four groups over 40000 and 34000 rows of FP8 69 us (37,
// 27, 5), four over 2049 rows 20 us (10.5, 5.5, 5).
#include "tile_pipe.h"

namespace lfps {

namespace {

struct PrefixArgs {
  Shape s;
  KvView kv;
  const float* q;
  PrefixGroups groups;
  float* part;                   // [B, Hq, splits] partial results over the shared rows
  OwnRows own;
  float* own_part;               // [items, Hkv, G, D + 2] over the requests' own (launch_full_attn_own)
  int32_t splits;
};

// FP8 keys and values are fp16 operands here: two fp16 terms hold a query or a weight to 22 bits, of bf16 ones it takes three.
// (Two of bf16 were 2.7e-6 from 64 bits, these are 0.5e-6.)
template <typename TK, typename TV>
using PrefixOp = typename std::conditional<sizeof(TK) == 1 && sizeof(TV) == 1, f16x8, typename InLds<TK>::Op>::type;

// Query rows (member, head) from row0 on of the requests from b0 to b1, over rows [lo, hi) of request `from`; slot: of the partials.
template <typename TK, typename TV, int kKeyWaves>
__device__ __forceinline__ void prefix_tile(char* lds, const PrefixArgs& a, int b0, int b1, int row0, int g, int from, int lo, int hi, int slot) {
  typedef PrefixOp<TK, TV> Op;
  constexpr int kTerms = std::is_same<Op, float>::value ? 1 : 2;
  const Shape& s = a.s;
  const int G = s.G, shift = G == 4 ? 2 : G - 1;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), h = lane >> 5;
  const int rows = (b1 - b0) << shift;
  int m = row0 + (wave / kKeyWaves) * 32 + (lane & 31);
  const bool valid = m < rows;
  m = valid ? m : rows - 1;
  const int b = b0 + (m >> shift), head = g * G + (m & (G - 1));
  RowState<Op, kTerms> st;
  st.clear();
  if (lo < hi) {
    const int n = length_of(s, a.kv.seq_lens, b);
    const int limit = valid ? (n < hi ? n : hi) : 0;
    const CacheRows<TK> K(a.kv.k, a.kv, from, g);
    const CacheRows<TV> V(a.kv.v, a.kv, from, g);
    tile_loop<TK, TV, kKeyWaves>(lds, K, V, lo, hi, [&](auto& q) { q.load(a.q + ((int64_t)b * s.Hq + head) * kD, h); }, limit, st);
  }
  RowOut<float> to = {nullptr, nullptr};
  if (valid) to.part = a.part + (((int64_t)b * s.Hq + head) * a.splits + slot) * kPartFloats;
  tile_finish<Op, kTerms, kKeyWaves>(lds, st, to);
}

// The same for 256 rows of 16-bit operands, with the loop of tile_pipe.h.
template <int kKind, typename TK, typename TV>
__device__ __forceinline__ void prefix_pipe(char* lds, const PrefixArgs& a, int b0, int b1, int row0, int g, int lo, int hi, int slot) {
  typedef PrefixOp<TK, TV> Op;
  const Shape& s = a.s;
  const int G = s.G, shift = G == 4 ? 2 : G - 1, lane = threadIdx.x & 63, h = lane >> 5, rows = (b1 - b0) << shift;
  int m = row0 + 32 * wave_of() + (lane & 31);
  const bool valid = m < rows;
  m = valid ? m : rows - 1;
  const int b = b0 + (m >> shift), head = g * G + (m & (G - 1)), n = length_of(s, a.kv.seq_lens, b);
  PipeState<Op, 2> st;
  st.clear();
  st.limit = n < hi ? n : hi;
  if (lo < hi) {
    int least = hi;                                              // of the members' lengths: keys that all rows see
    for (int i = b0 + row0 / G + lane; i < b1 && i < b0 + (row0 + kPipeRows) / G; i += 64) least = min(least, length_of(s, a.kv.seq_lens, i));
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) least = min(least, __shfl_xor(least, d));
    st.q.load(a.q + ((int64_t)b * s.Hq + head) * kD, h, PipeState<Op, 2>::kRest ? (lds_char*)lds + kRestAt + wave_of() * kRestWave : nullptr);
    const CacheRows<TK> K(a.kv.k, a.kv, b0, g);
    const CacheRows<TV> V(a.kv.v, a.kv, b0, g);
    pipe_loop<kKind, TK, TV>(lds, K, V, lo, hi, __builtin_amdgcn_readfirstlane(least), row0 + 32 * wave_of() < rows, st);
  }
  if (valid) st.finish((float*)nullptr, a.part + (((int64_t)b * s.Hq + head) * a.splits + slot) * kPartFloats, h);
}

// The items of the rows that requests have for themselves, by one workgroup beside those of part 1: as many rows an item as make kOwnWorkgroups workgroups of
// all, kOwnLeast at least, and no more items of a request than k_prefix_merge takes.
__device__ __forceinline__ int own_item_rows(int64_t total, int most, int wanted) {
  int64_t per = (total + wanted - 1) / wanted;
  const int64_t of_longest = (most + kMaxSplits - 1) / kMaxSplits;
  per = per > of_longest ? (per < most ? per : most) : of_longest;
  return per <= kOwnLeast ? kOwnLeast : (int)((per + 15) & ~(int64_t)15);
}
__device__ __forceinline__ void plan_own(char* lds, const PrefixArgs& a) {
  const Shape& s = a.s;
  const int lane = threadIdx.x & 63, wave = wave_of(), waves = blockDim.x >> 6;
  int64_t* const sums = reinterpret_cast<int64_t*>(lds);           // [waves], and behind them the waves' largest
  int* const largest = reinterpret_cast<int*>(sums + 8);
  int64_t total = 0;
  int most = 0;
  for (int b = threadIdx.x; b < s.B; b += blockDim.x) {
    int lo = 0, hi = a.groups.n - 1;                              // the last group that begins at b or before
    while (lo < hi) {
      const int mid = (lo + hi + 1) >> 1;
      if (a.groups.start[mid] <= b) lo = mid;
      else hi = mid - 1;
    }
    int b0, b1, shared;
    group_at(s, a.kv.seq_lens, a.groups, lo, &b0, &b1, &shared);
    const int n = length_of(s, a.kv.seq_lens, b), first = b < b0 || b >= b1 ? -1 : min(shared, n), mine = first < 0 ? 0 : n - first;
    a.own.first[b] = first;
    total += mine;
    most = max(most, mine);
  }
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    total += __shfl_xor(total, d);
    most = max(most, __shfl_xor(most, d));
  }
  if (lane == 0) {
    sums[wave] = total;
    largest[wave] = most;
  }
  __syncthreads();
  total = 0;
  for (int w = 0; w < waves; ++w) {
    total += sums[w];
    most = max(most, largest[w]);
  }
  const int per = own_item_rows(total, most, own_items_most(s) - s.B);
  int* const counts = largest + 8;                                 // [2][waves]
  int base = 0, turn = 0;
  for (int b_first = 0; b_first < s.B; b_first += blockDim.x, turn ^= 8) {
    const int b = b_first + threadIdx.x;
    int first = 0, n = 0;
    if (b < s.B) {
      first = a.own.first[b];                                      // (my own store)
      n = first < 0 ? first : length_of(s, a.kv.seq_lens, b);
    }
    const int items = (n - first + per - 1) / per;
    int upto = items;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) {
      const int x = __shfl_up(upto, d);
      if (lane >= d) upto += x;
    }
    if (lane == 63) counts[turn + wave] = upto;
    __syncthreads();
    int at = base + upto - items;
    for (int w = 0; w < waves; ++w) {
      if (w < wave) at += counts[turn + w];
      base += counts[turn + w];
    }
    if (b < s.B) {
      a.own.item[b] = at;
      for (int r = first; r < n; r += per) a.own.items[at++] = OwnItem{b, r, min(r + per, n), 0};
    }
  }
  if (threadIdx.x == 0) a.own.item[s.B] = base;
}

// Query rows of a workgroup of k_prefix_shared.
template <typename TK, int kKeyWaves>
constexpr int shared_rows() { return kKeyWaves == 1 && sizeof(TK) != 4 ? kPipeRows : 32 * (4 / kKeyWaves); }

}  // namespace

// grid 1 + Hkv * splits * tiles
template <typename TK, typename TV, int kKeyWaves, int kKind>
__global__ __launch_bounds__((shared_rows<TK, kKeyWaves>() == kPipeRows ? kPipeThreads : kTileThreads)) void k_prefix_shared(PrefixArgs a) {
  request_arguments<decltype(&k_prefix_shared<TK, TV, kKeyWaves, kKind>)>();
  constexpr int kRows = shared_rows<TK, kKeyWaves>();
  __shared__ __attribute__((aligned(16))) char lds[kRows == kPipeRows ? pipe_lds<PrefixOp<TK, TV>, 2>() : tile_lds<TK, TV, kKeyWaves>()];
  if (blockIdx.x == 0) return plan_own(lds, a);
  const int block = blockIdx.x - 1, g = block % a.s.Hkv, x0 = block / a.s.Hkv, split = x0 % a.splits, x = x0 / a.splits;
  const int per = kRows / a.s.G;
  auto first_tile = [&](int i) {
    const int b = a.groups.start[i];
    return (b < 0 ? 0 : (b > a.s.B ? a.s.B : b)) / per + i;
  };
  const int i = last_not_above(a.groups.n - 1, x, first_tile);
  int b0, b1, shared;
  group_at(a.s, a.kv.seq_lens, a.groups, i, &b0, &b1, &shared);
  const int row0 = (x - first_tile(i)) * kRows;
  if (row0 < 0 || row0 >= (b1 - b0) * a.s.G) return;
  int lo, hi;
  split_rows(0, shared, a.splits, split, tile_rows(kKeyWaves), &lo, &hi);
  if constexpr (kRows == kPipeRows) prefix_pipe<kKind, TK, TV>(lds, a, b0, b1, row0, g, lo, hi, split);
  else prefix_tile<TK, TV, kKeyWaves>(lds, a, b0, b1, row0, g, b0, lo, hi, split);
}

// a wave a (request, head)
__global__ __launch_bounds__(kTileThreads) void k_prefix_merge(PrefixArgs a, float* __restrict__ out) {
  request_arguments<decltype(&k_prefix_merge)>();
  const Shape& s = a.s;
  const int row = blockIdx.x * (kTileThreads / 64) + wave_of();
  if (row >= s.B * s.Hq) return;
  const int b = row / s.Hq, h = row % s.Hq, item = a.own.item[b], own = a.own.item[b + 1] - item;
  if (a.own.first[b] < 0) return;
  const float* const part = a.part + (int64_t)row * a.splits * kPartFloats;
  const int64_t step = (int64_t)s.Hkv * s.G * (kD + 2);
  const float* const mine = a.own_part + item * step + (int64_t)h * (kD + 2);
  const float unit = s.G == 1 ? 1.f : kLog2e;                 // (with grouping those parts' scores are natural ones)
  auto at = [&](int i) { return i < a.splits ? part + (int64_t)i * kPartFloats : mine + (i - a.splits) * step; };
  put2(out + (int64_t)row * kD + 2 * (threadIdx.x & 63),
       join_parts(a.splits + own, at, [&](int i) { return at(i)[kD] * (i < a.splits ? 1.f : unit); }, [&](int i) { return at(i)[kD + 1]; }));
}

namespace {

template <typename TK, typename TV>
hipError_t prefix_t(PrefixArgs a, int dtype, float* out, int64_t part_rows, hipStream_t st) {
  const Shape& s = a.s;
  const int64_t heads = (int64_t)s.B * s.Hq;
  // The rows of a group of ordinary size decide how many a workgroup takes.  16-bit operands: up to 64 rows, tiles of 32 with a wave a
  // quarter of the keys; more, 256 rows with the pipelined loop.  Over 8192 rows of 8 KV heads, us of the whole call with either: bf16
  // groups of 32 rows 27.3 / 30.5, 48 32.8 / 31.8, 64 30.4 / 32.4, 80 51.0 / 33.9, 128 39.5 / 37.9; FP8 26.1 / 29.5, 31.4 / 30.6, 29.1 / 32.5,
  // 48.6 / 34.1, 38.0 / 38.7.  (Tiles of 64 rows with half the keys a wave: 30.3, 35.1, 32.8, 45.1, 40.3 in bf16, never the best.)
  // fp32: tiles of 64 rows, of 128 where a group fills them.
  // Form and parts follow from the number of groups, not from their sizes and prefixes, which are on the device.  Groups that are unlike
  // pay for it: 32 requests over 30000 rows take 80 us with 500 rows each of their own, and 576 beside 32 groups of one request (170 where
  // those are one group with a prefix of 0); a pair over 30000 beside 31 pairs over 100 rows takes 778, walked by a workgroup a KV head.
  const int size = (s.B + a.groups.n - 1) / a.groups.n, rows = size * s.G;
  const int key_waves = rows > 64 ? 1 : (sizeof(TK) == 4 ? 2 : 4);
  const int per = key_waves == 1 ? shared_rows<TK, 1>() : 32 * (4 / key_waves);
  const int tiles = s.B / (per / s.G) + a.groups.n;          // room for any groups; of groups of one size there are `usual`
  const int64_t usual = (int64_t)a.groups.n * ((size * s.G + per - 1) / per);
  // The workspace: parts of the shared rows; the plan of the own ones, and their parts.
  const int64_t own_rows = (int64_t)own_items_most(s) * s.Hq, plan_rows = own_plan_rows_for(s.B, s.Hkv);
  const int64_t room = (part_rows - own_rows - plan_rows) / heads, by_len = (s.Lcap + 127) / 128;          // room: at least 1 (part_rooms.h)
  int64_t splits = (256 + usual * s.Hkv - 1) / (usual * s.Hkv);
  for (const int64_t most : {room, by_len, (int64_t)kMaxSplits}) splits = splits < most ? splits : most;
  a.splits = (int)splits;
  a.own_part = a.part + heads * a.splits * kPartFloats;
  a.own.items = reinterpret_cast<OwnItem*>(a.own_part + own_rows * kPartFloats);
  a.own.first = reinterpret_cast<int32_t*>(a.own.items + own_items_most(s));
  a.own.item = a.own.first + s.B;
  const unsigned grid = 1 + (unsigned)(s.Hkv * a.splits * tiles);
#define LFPS_SHARED(KW, KIND) \
  hipLaunchKernelGGL((k_prefix_shared<TK, TV, KW, KIND>), dim3(grid), dim3(per == kPipeRows ? kPipeThreads : kTileThreads), 0, st, a)
  const int kind = sizeof(TK) == 4 ? kAnyRows : rows_kind(a.kv);
  if (key_waves == 1 && kind == kAnyRows) LFPS_SHARED(1, kAnyRows);
  else if constexpr (sizeof(TK) == 4) LFPS_SHARED(2, kAnyRows);
  else {
    if (key_waves == 4) LFPS_SHARED(4, kAnyRows);
    else if (kind == kSlab) LFPS_SHARED(1, kSlab);
    else LFPS_SHARED(1, kPages);
  }
#undef LFPS_SHARED
  const hipError_t e = launch_full_attn_own(s, dtype, a.q, a.kv, a.own, a.own_part, st);
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL(k_prefix_merge, dim3((unsigned)((heads + 3) / 4)), dim3(kTileThreads), 0, st, a, out);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_prefix_attn(const Shape& s, int dtype, const KvView& kv, const float* q, const int32_t* group_start,
                              const int32_t* prefix_len, int n_groups, float* out, float* part, int64_t part_rows, hipStream_t st) {
  const PrefixArgs a = {s, kv, q, {group_start, prefix_len, n_groups}, part, {}, nullptr, 1};
  if (dtype == LFPS_F32) return prefix_t<float, float>(a, dtype, out, part_rows, st);
  if (dtype == LFPS_F16) return prefix_t<_Float16, _Float16>(a, dtype, out, part_rows, st);
  if (kv.k_fp8 && kv.v_fp8) return prefix_t<uint8_t, uint8_t>(a, dtype, out, part_rows, st);
  if (kv.k_fp8) return prefix_t<uint8_t, uint16_t>(a, dtype, out, part_rows, st);
  if (kv.v_fp8) return prefix_t<uint16_t, uint8_t>(a, dtype, out, part_rows, st);
  return prefix_t<uint16_t, uint16_t>(a, dtype, out, part_rows, st);
}

}  // namespace lfps
