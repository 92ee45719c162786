// Groups of requests that share their first rows (lfps_prefix_attn_decode), as the kernels read them.
#pragma once
#include "lfps_internal.h"

namespace lfps {

struct PrefixGroups {
  const int32_t* start;      // [n + 1]
  const int32_t* shared;     // [n]
  int32_t n;
};

__device__ __forceinline__ int length_of(const Shape& s, const int32_t* seq_lens, int b) {
  const int n = seq_lens[b];
  return n < 0 ? 0 : (n > s.Lcap ? s.Lcap : n);
}

// The last i in [0, n] with start(i) <= x, for a rising start with start(0) <= x: 64 places a round, by the whole wave.  Of a start that
// does not rise, some i in [0, n].
template <typename Start>
__device__ __forceinline__ int last_not_above(int n, int x, Start start) {
  const int lane = threadIdx.x & 63;
  int lo = 0, span = n + 1;
  while (span > 1) {
    const int step = (span + 63) >> 6;
    const int i = lo + lane * step;
    const int last = i < lo + span ? i : lo + span - 1;
    const int got = __popcll(__ballot(i < lo + span && start(last) <= x));
    const int to = lo + (got > 0 ? got - 1 : 0) * step;
    span = lo + span - to < step ? lo + span - to : step;
    lo = to;
  }
  return __builtin_amdgcn_readfirstlane(lo);
}

// The members [b0, b1) of group i and the rows that they share, whatever the arrays hold.
__device__ __forceinline__ void group_at(const Shape& s, const int32_t* seq_lens, const PrefixGroups& p, int i, int* b0, int* b1, int* shared) {
  const int x = p.start[i], y = p.start[i + 1], m = p.shared[i];
  *b0 = x < 0 ? 0 : (x > s.B ? s.B : x);
  *b1 = y < *b0 ? *b0 : (y > s.B ? s.B : y);
  const int n = *b0 < s.B ? length_of(s, seq_lens, *b0) : 0;
  *shared = m < 0 ? 0 : (m > n ? n : m);
}
// The first row that request b has for itself; below 0: it is in no group.  The whole wave calls.
__device__ __forceinline__ int first_own_row(const Shape& s, const int32_t* seq_lens, const PrefixGroups& p, int b) {
  const int i = last_not_above(p.n - 1, b, [&](int j) { return p.start[j]; });
  int b0, b1, shared;
  group_at(s, seq_lens, p, i, &b0, &b1, &shared);
  return b >= b0 && b < b1 ? shared : -1;
}

// Full attention of every request over the rows that it has for itself: part [B, Hkv, n_split, G, D + 2], of which a request over n
// such rows has own_parts(n, n_split), each as in the full-attention baseline.
__host__ __device__ __forceinline__ int rows_per_split(int n, int n_split) { return (((n + n_split - 1) / n_split) + 15) & ~15; }
__host__ __device__ __forceinline__ int own_parts(int n, int n_split) {
  const int per = rows_per_split(n, n_split);
  return (n + per - 1) / per;
}
hipError_t launch_full_attn_own(const Shape& s, int dtype, const float* q, const KvView& kv, const PrefixGroups& groups, float* part,
                                int n_split, hipStream_t st);

}  // namespace lfps
