// One decode step's full attention over all n_b rows (as the full-attention baseline) for a batch in which groups of requests share
// their first rows: those are read once for a group, not once for every request, and its members' query heads are rows of one product.
//
//   part 1  per group, KV head and part of the shared rows: up to 128 query rows (members x heads) against them
//   part 2  per request, KV head and part of its own rows: its G heads against those
//   part 3  the parts of a (request, head) joined:  o = sum_i e^(m_i - m) acc_i / sum_i e^(m_i - m) l_i
//
// Bound by the bytes of K and V, read once, while a group has few members; by the matrix units where it has many.  The query stays
// fp32, as a sum of 16-bit terms, and so do the weights (tile_attn.h): the results are fp32 ones as everywhere in the library.
#include "tile_attn.h"

namespace lfps {

namespace {

struct PrefixArgs {
  Shape s;
  KvView kv;
  const float* q;
  const int32_t* group_start;    // [n_groups + 1]
  const int32_t* prefix_len;     // [n_groups]
  int32_t n_groups;
  float* part;                   // [B, Hq, splits + own_splits] partial results
  int32_t splits, own_splits;    // parts of the shared rows and of a request's own
  int32_t tiles;                 // row tiles of all groups, at most
};

__device__ __forceinline__ int length_of(const Shape& s, const int32_t* seq_lens, int b) {
  const int n = seq_lens[b];
  return n < 0 ? 0 : (n > s.Lcap ? s.Lcap : n);
}
// The members [b0, b1) of group i and the rows that they share, whatever the arrays hold.
__device__ __forceinline__ void group_of(const PrefixArgs& a, int i, int* b0, int* b1, int* shared) {
  const int x = a.group_start[i], y = a.group_start[i + 1], p = a.prefix_len[i];
  *b0 = x < 0 ? 0 : (x > a.s.B ? a.s.B : x);
  *b1 = y < *b0 ? *b0 : (y > a.s.B ? a.s.B : y);
  const int n = *b0 < a.s.B ? length_of(a.s, a.kv.seq_lens, *b0) : 0;
  *shared = p < 0 ? 0 : (p > n ? n : p);
}
// The group that request b is in, or -1.
__device__ __forceinline__ int find_group(const PrefixArgs& a, int b, int* shared) {
  const int i = last_not_above(a.n_groups - 1, b, [&](int j) { return a.group_start[j]; });
  int b0, b1;
  group_of(a, i, &b0, &b1, shared);
  return b >= b0 && b < b1 ? i : -1;
}

// Query rows (member, head) from row0 on of the requests from b0 to b1, over rows [lo, hi) of request `from`; slot: of the partials.
template <typename TK, typename TV, int kKeyWaves>
__device__ __forceinline__ void prefix_tile(char* lds, const PrefixArgs& a, int b0, int b1, int row0, int g, int from, int lo, int hi, int slot) {
  typedef typename InLds<TK>::Op Op;
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
    typename RowState<Op, kTerms>::Query q;
    q.load(a.q + ((int64_t)b * s.Hq + head) * kD, h);
    const CacheRows<TK> K(a.kv.k, a.kv, from, g);
    const CacheRows<TV> V(a.kv.v, a.kv, from, g);
    tile_loop<TK, TV, Op, kTerms, kKeyWaves>(lds, K, V, lo, hi, q, limit, st);
  }
  RowOut<float> to = {nullptr, nullptr};
  if (valid) to.part = a.part + (((int64_t)b * s.Hq + head) * (a.splits + a.own_splits) + slot) * kPartFloats;
  tile_finish<Op, kTerms, kKeyWaves>(lds, st, to);
}

}  // namespace

// grid Hkv * splits * tiles
template <typename TK, typename TV, int kKeyWaves>
__global__ __launch_bounds__(kTileThreads) void k_prefix_shared(PrefixArgs a) {
  constexpr int kRows = 32 * (4 / kKeyWaves);
  __shared__ __attribute__((aligned(16))) char lds[tile_lds<TK, TV, kKeyWaves>()];
  const int g = blockIdx.x % a.s.Hkv, x0 = blockIdx.x / a.s.Hkv, split = x0 % a.splits, x = x0 / a.splits;
  const int per = kRows / a.s.G;
  auto first_tile = [&](int i) {
    const int b = a.group_start[i];
    return (b < 0 ? 0 : (b > a.s.B ? a.s.B : b)) / per + i;
  };
  const int i = last_not_above(a.n_groups - 1, x, first_tile);
  int b0, b1, shared;
  group_of(a, i, &b0, &b1, &shared);
  const int row0 = (x - first_tile(i)) * kRows;
  if (row0 < 0 || row0 >= (b1 - b0) * a.s.G) return;
  int lo, hi;
  split_rows(0, shared, a.splits, split, tile_rows(kKeyWaves), &lo, &hi);
  prefix_tile<TK, TV, kKeyWaves>(lds, a, b0, b1, row0, g, b0, lo, hi, split);
}

// grid Hkv * own_splits * B
template <typename TK, typename TV>
__global__ __launch_bounds__(kTileThreads) void k_prefix_own(PrefixArgs a) {
  constexpr int kKeyWaves = few_key_waves<TK>();
  __shared__ __attribute__((aligned(16))) char lds[tile_lds<TK, TV, kKeyWaves>()];
  const int g = blockIdx.x % a.s.Hkv, x0 = blockIdx.x / a.s.Hkv, split = x0 % a.own_splits, b = x0 / a.own_splits;
  int shared, lo, hi;
  if (find_group(a, b, &shared) < 0) return;
  const int n = length_of(a.s, a.kv.seq_lens, b);
  split_rows(shared < n ? shared : n, n, a.own_splits, split, tile_rows(kKeyWaves), &lo, &hi);
  prefix_tile<TK, TV, kKeyWaves>(lds, a, b, b + 1, 0, g, b, lo, hi, a.splits + split);
}

// 32 lanes a (request, head)
__global__ __launch_bounds__(kTileThreads) void k_prefix_merge(PrefixArgs a, float* __restrict__ out) {
  const int row = blockIdx.x * (kTileThreads / 32) + threadIdx.x / 32, b = row / a.s.Hq, lane32 = threadIdx.x & 31;
  const int rows = a.s.B * a.s.Hq;
  // (both halves of a wave take part in the search)
  const int first = __builtin_amdgcn_readfirstlane(row), second = first + 1;
  int shared;
  const int ba = (first < rows ? first : rows - 1) / a.s.Hq, bb = (second < rows ? second : rows - 1) / a.s.Hq;
  const int ga = find_group(a, ba, &shared), gb = ba == bb ? ga : find_group(a, bb, &shared);
  if (row >= rows || (b == ba ? ga : gb) < 0) return;
  const int n = a.splits + a.own_splits;
  put4(out + (int64_t)row * kD + 4 * lane32, merge_parts(a.part + (int64_t)row * n * kPartFloats, n, lane32));
}

namespace {

template <typename TK, typename TV>
hipError_t prefix_t(PrefixArgs a, float* out, int64_t part_rows, hipStream_t st) {
  const Shape& s = a.s;
  const int64_t heads = (int64_t)s.B * s.Hq;
  // The rows of a group of ordinary size decide how many a workgroup takes: more share a row of the cache, fewer leave no wave idle.
  const int rows = (s.B + a.n_groups - 1) / a.n_groups * s.G;
  const int key_waves = rows > 64 ? 1 : (rows > 32 || sizeof(TK) == 4 ? 2 : 4);
  a.tiles = s.B / (32 * (4 / key_waves) / s.G) + a.n_groups;
  auto parts = [&](int64_t groups, int64_t most) {
    int64_t n = (512 + groups - 1) / groups;
    const int64_t by_len = (s.Lcap + 255) / 256;
    if (n > by_len) n = by_len;
    if (n > most) n = most;
    return (int)(n < 1 ? 1 : n);
  };
  const int64_t room = part_rows / heads;                   // at least 2
  a.own_splits = parts((int64_t)s.B * s.Hkv, room / 2 < kMaxSplits ? room / 2 : kMaxSplits);
  a.splits = parts((int64_t)a.tiles * s.Hkv, room - a.own_splits < kMaxSplits ? room - a.own_splits : kMaxSplits);
  const unsigned grid = (unsigned)(s.Hkv * a.splits * a.tiles);
  if (key_waves == 1) hipLaunchKernelGGL((k_prefix_shared<TK, TV, 1>), dim3(grid), dim3(kTileThreads), 0, st, a);
  else if (key_waves == 2) hipLaunchKernelGGL((k_prefix_shared<TK, TV, 2>), dim3(grid), dim3(kTileThreads), 0, st, a);
  else if constexpr (sizeof(TK) != 4) hipLaunchKernelGGL((k_prefix_shared<TK, TV, 4>), dim3(grid), dim3(kTileThreads), 0, st, a);
  hipLaunchKernelGGL((k_prefix_own<TK, TV>), dim3((unsigned)(s.Hkv * a.own_splits * s.B)), dim3(kTileThreads), 0, st, a);
  hipLaunchKernelGGL(k_prefix_merge, dim3((unsigned)((heads + 7) / 8)), dim3(kTileThreads), 0, st, a, out);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_prefix_attn(const Shape& s, int dtype, const KvView& kv, const float* q, const int32_t* group_start,
                              const int32_t* prefix_len, int n_groups, float* out, float* part, int64_t part_rows, hipStream_t st) {
  const PrefixArgs a = {s, kv, q, group_start, prefix_len, n_groups, part, 1, 1, 1};
  if (dtype == LFPS_F32) return prefix_t<float, float>(a, out, part_rows, st);
  if (dtype == LFPS_F16) return prefix_t<_Float16, _Float16>(a, out, part_rows, st);
  if (kv.k_fp8 && kv.v_fp8) return prefix_t<uint8_t, uint8_t>(a, out, part_rows, st);
  if (kv.k_fp8) return prefix_t<uint8_t, uint16_t>(a, out, part_rows, st);
  if (kv.v_fp8) return prefix_t<uint16_t, uint8_t>(a, out, part_rows, st);
  return prefix_t<uint16_t, uint16_t>(a, out, part_rows, st);
}

}  // namespace lfps
