// Packed tokens of requests (lfps_append, lfps_prompt_attn) and groups of requests that share their first rows (lfps_prefix_attn_decode),
// as the kernels read them.
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

// Tokens [c0, c1) of request b of n_tokens packed ones, whatever cu holds.
__device__ __forceinline__ void request_tokens(const int32_t* cu, int n_tokens, int b, int* c0, int* c1) {
  const int x = cu[b], y = cu[b + 1];
  *c0 = x < 0 ? 0 : (x > n_tokens ? n_tokens : x);
  *c1 = y < *c0 ? *c0 : (y > n_tokens ? n_tokens : y);
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

// The rows that the requests have for themselves, cut into items of no more than some number of rows, the same for all: what their lengths
// ask for, so that a long request is cut into many and a short one into one.  Made by plan_own, once a call, on the device.
// (With the same number of parts for each request, most workgroups of a batch of unlike lengths found nothing to do, and the chip holds
// 768 of them at a time: 64 requests of 1 to 900 rows 35 -> 29 us, 32 of 100 to 2000 in FP8 33 -> 27.  64, 128 and 256 rows at least: 77.5, 78.3
// and 83.2 us of the whole FP8 call.)
struct OwnItem { int32_t b, begin, end, unused; };
struct OwnRows {
  int32_t* first;            // [B] a request's first row of its own; below 0: it is in no group
  int32_t* item;             // [B + 1] its first item; of B: the number of all
  OwnItem* items;            // [own_items_most]
};
__host__ __device__ inline int own_items_most(const Shape& s) { return own_items_for(s.B, s.Hkv); }

// Full attention over the items' rows: part [items, Hkv, G, D + 2], each as of a part in the full-attention baseline.
hipError_t launch_full_attn_own(const Shape& s, int dtype, const float* q, const KvView& kv, const OwnRows& own, float* part, hipStream_t st);

}  // namespace lfps
