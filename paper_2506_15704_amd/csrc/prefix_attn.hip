// One decode step's full attention over all n_b rows (as the full-attention baseline) for a batch in which groups of requests share
// their first rows: those are read once for a group, not once for every request, and its members' query heads are rows of one product.
//
//   part 1  per group, KV head and part of the shared rows: up to 128 query rows (members x heads) against them
//   part 2  per request, KV head and part of its own rows: its G heads against those (attention.hip)
//   part 3  the parts of a (request, head) joined:  o = sum_i e^(m_i - m) acc_i / sum_i e^(m_i - m) l_i
//
// Bound by the bytes of K and V, read once, while a group has few members; by the matrix units where it has many.  The query stays
// fp32, as a sum of 16-bit terms, and so do the weights (tile_attn.h): the results are fp32 ones as everywhere in the library.
#include "tile_pipe.h"

namespace lfps {

namespace {

struct PrefixArgs {
  Shape s;
  KvView kv;
  const float* q;
  PrefixGroups groups;
  float* part;                   // [B, Hq, splits] partial results over the shared rows
  float* own_part;               // [B, Hkv, own_splits, G, D + 2] over each request's own (launch_full_attn_own)
  int32_t splits, own_splits;
};

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
  if (valid) to.part = a.part + (((int64_t)b * s.Hq + head) * a.splits + slot) * kPartFloats;
  tile_finish<Op, kTerms, kKeyWaves>(lds, st, to);
}

// The same for 256 rows of 16-bit operands, with the loop of tile_pipe.h.
template <int kKind, typename TK, typename TV>
__device__ __forceinline__ void prefix_pipe(char* lds, const PrefixArgs& a, int b0, int b1, int row0, int g, int lo, int hi, int slot) {
  typedef typename InLds<TK>::Op Op;
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
    st.q.load(a.q + ((int64_t)b * s.Hq + head) * kD, h);
    const CacheRows<TK> K(a.kv.k, a.kv, b0, g);
    const CacheRows<TV> V(a.kv.v, a.kv, b0, g);
    pipe_loop<kKind, TK, TV>(lds, K, V, lo, hi, __builtin_amdgcn_readfirstlane(least), row0 + 32 * wave_of() < rows, st);
  }
  if (valid) st.finish((float*)nullptr, a.part + (((int64_t)b * s.Hq + head) * a.splits + slot) * kPartFloats, h);
}

// Query rows of a workgroup of k_prefix_shared.
template <typename TK, int kKeyWaves>
constexpr int shared_rows() { return kKeyWaves == 1 && sizeof(TK) != 4 ? kPipeRows : 32 * (4 / kKeyWaves); }

}  // namespace

// grid Hkv * splits * tiles
template <typename TK, typename TV, int kKeyWaves, int kKind>
__global__ __launch_bounds__((shared_rows<TK, kKeyWaves>() == kPipeRows ? kPipeThreads : kTileThreads)) void k_prefix_shared(PrefixArgs a) {
  constexpr int kRows = shared_rows<TK, kKeyWaves>();
  __shared__ __attribute__((aligned(16))) char lds[kRows == kPipeRows ? kPipeLds : tile_lds<TK, TV, kKeyWaves>()];
  const int g = blockIdx.x % a.s.Hkv, x0 = blockIdx.x / a.s.Hkv, split = x0 % a.splits, x = x0 / a.splits;
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
  const Shape& s = a.s;
  const int row = blockIdx.x * (kTileThreads / 64) + wave_of();
  if (row >= s.B * s.Hq) return;
  const int b = row / s.Hq, h = row % s.Hq, first = first_own_row(s, a.kv.seq_lens, a.groups, b);
  if (first < 0) return;
  const int n = length_of(s, a.kv.seq_lens, b), own = first < n ? own_parts(n - first, a.own_splits) : 0;
  const float* const part = a.part + (int64_t)row * a.splits * kPartFloats;
  const int64_t step = (int64_t)s.G * (kD + 2);
  const float* const mine = a.own_part + ((int64_t)(b * s.Hkv + h / s.G) * a.own_splits) * step + (int64_t)(h % s.G) * (kD + 2);
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
  // The rows of a group of ordinary size decide how many a workgroup takes: more share a row of the cache, fewer leave no wave idle.
  const int rows = (s.B + a.groups.n - 1) / a.groups.n * s.G;
  const int key_waves = rows > 64 ? 1 : (rows > 32 || sizeof(TK) == 4 ? 2 : 4);
  const int per = key_waves == 1 ? shared_rows<TK, 1>() : 32 * (4 / key_waves);
  const int tiles = s.B / (per / s.G) + a.groups.n;
  auto parts = [&](int64_t wanted, int64_t groups, int64_t most) {
    int64_t n = (wanted + groups - 1) / groups;
    const int64_t by_len = (s.Lcap + 255) / 256;
    if (n > by_len) n = by_len;
    if (n > most) n = most;
    return (int)(n < 1 ? 1 : n);
  };
  const int64_t room = part_rows / heads;                   // at least 2
  a.own_splits = parts(2048, (int64_t)s.B * s.Hkv, room / 2 < kMaxSplits ? room / 2 : kMaxSplits);
  a.splits = parts(per == kPipeRows ? 256 : 512, (int64_t)tiles * s.Hkv, room - a.own_splits < kMaxSplits ? room - a.own_splits : kMaxSplits);
  a.own_part = a.part + heads * a.splits * kPartFloats;
  const unsigned grid = (unsigned)(s.Hkv * a.splits * tiles);
#define LFPS_SHARED(KW, KIND) \
  hipLaunchKernelGGL((k_prefix_shared<TK, TV, KW, KIND>), dim3(grid), dim3(per == kPipeRows ? kPipeThreads : kTileThreads), 0, st, a)
  const int kind = sizeof(TK) == 4 ? kAnyRows : rows_kind(a.kv);
  if (key_waves == 2) LFPS_SHARED(2, kAnyRows);
  else if (key_waves == 1 && kind == kAnyRows) LFPS_SHARED(1, kAnyRows);
  else if constexpr (sizeof(TK) != 4) {
    if (key_waves == 4) LFPS_SHARED(4, kAnyRows);
    else if (kind == kSlab) LFPS_SHARED(1, kSlab);
    else LFPS_SHARED(1, kPages);
  }
#undef LFPS_SHARED
  const hipError_t e = launch_full_attn_own(s, dtype, a.q, a.kv, a.groups, a.own_part, a.own_splits, st);
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL(k_prefix_merge, dim3((unsigned)((heads + 3) / 4)), dim3(kTileThreads), 0, st, a, out);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_prefix_attn(const Shape& s, int dtype, const KvView& kv, const float* q, const int32_t* group_start,
                              const int32_t* prefix_len, int n_groups, float* out, float* part, int64_t part_rows, hipStream_t st) {
  const PrefixArgs a = {s, kv, q, {group_start, prefix_len, n_groups}, part, nullptr, 1, 1};
  if (dtype == LFPS_F32) return prefix_t<float, float>(a, dtype, out, part_rows, st);
  if (dtype == LFPS_F16) return prefix_t<_Float16, _Float16>(a, dtype, out, part_rows, st);
  if (kv.k_fp8 && kv.v_fp8) return prefix_t<uint8_t, uint8_t>(a, dtype, out, part_rows, st);
  if (kv.k_fp8) return prefix_t<uint8_t, uint16_t>(a, dtype, out, part_rows, st);
  if (kv.v_fp8) return prefix_t<uint16_t, uint8_t>(a, dtype, out, part_rows, st);
  return prefix_t<uint16_t, uint16_t>(a, dtype, out, part_rows, st);
}

}  // namespace lfps
