// The kernels of packed tokens' attention, over all rows up to a token's own (prompt_attn.hip) or over a window and the first rows
// (window_attn.hip).
#pragma once
#include "tile_pipe.h"


namespace lfps {

namespace {

// Which rows a token at row p sees: all up to its own; or of these the newest `window` and the first n_sink.
struct SeesAll {
  __device__ __forceinline__ AllRows walk(int, int, int) const { return {}; }
  __host__ int most(int cap, int) const { return cap; }
  __host__ bool few_apart(int) const { return true; }
};
struct SeesWindow {
  int32_t window, n_sink;
  // the first row of the token's window; 0: it misses none
  __device__ __forceinline__ int from(int p) const {
    const int f = p + 1 > window ? p + 1 - window : 0;
    return f <= n_sink ? 0 : f;
  }
  // for a tile of tokens at rows first .. last, of which mine is at p: the first rows, then those from the first window's on, in eights
  __device__ __forceinline__ GapRows walk(int first, int last, int p) const {
    const int lo = from(first) & ~7, sinks = n_sink < lo ? n_sink : lo, at = (sinks + 7) & ~7, by = lo - at;
    const int all = from(last) - by;
    return {at, by, from(last) == 0 ? 0 : (all > at ? all : at), n_sink, from(p) - by};
  }
  // rows that a tile of `tokens` walks at most
  __host__ int most(int cap, int tokens) const {
    const int64_t n = (int64_t)window + n_sink + tokens + 128;
    return n < cap ? (int)n : cap;
  }
  // May requests of few tokens, whose tile walks `rows` at most, have a kernel of their own?
  __host__ bool few_apart(int rows) const { return rows > 6000; }
};

template <typename TQ, typename See>
struct PromptArgs {
  Shape s;
  KvView kv;
  const TQ* q;
  int64_t q_stride;        // elements between tokens of q
  const int32_t* cu;
  int32_t n_tokens;
  TQ* out;
  float* part;
  int32_t splits, few_splits;    // parts of a tile's rows in the two kernels; few_splits 0: k_prompt_few is not launched
  int64_t few_part;              // where the latter's partial results begin, in rows
  int32_t few_by_token;          // and whether they lie by token, or else in room for few_tokens of every request
  See see;
};

template <typename A>
__device__ __forceinline__ void tokens_of(const A& a, int b, int* c0, int* c1) {
  request_tokens(a.cu, a.n_tokens, b, c0, c1);
}
template <typename TK>
constexpr int few_most() { return 32 * (4 / few_key_waves<TK>()); }      // query rows of a request that k_prompt_few takes
// The partial results of token i (of those from c0 on of request b), a row of `splits` of them.
template <typename A>
__device__ __forceinline__ int64_t part_row(const A& a, bool few, int most, int b, int c0, int i, int head) {
  if (!few) return ((int64_t)(c0 + i) * a.s.Hq + head) * a.splits;
  const int64_t token = a.few_by_token ? c0 + i : (int64_t)b * (most / a.s.G) + i;
  return a.few_part + (token * a.s.Hq + head) * a.few_splits;
}

// Rows [row0, row0 + 32 * row waves) of request b's tokens (token row0 / G, heads fastest), KV head g, part `split` of `splits`.
template <typename TK, typename TV, int kKeyWaves, typename TQ, typename See>
__device__ __forceinline__ void prompt_tile(char* lds, const PromptArgs<TQ, See>& a, int b, int g, int c0, int c1, int row0, int split) {
  constexpr bool kFew = kKeyWaves > 1;
  const int splits = kFew ? a.few_splits : a.splits;
  typedef typename InLds<TK>::Op Op;
  constexpr int kRowWaves = 4 / kKeyWaves;
  const Shape& s = a.s;
  const int G = s.G, shift = G == 4 ? 2 : G - 1;                // G = 1, 2, 4
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), nrow = lane & 31, h = lane >> 5;
  const int n = length_of(s, a.kv.seq_lens, b), t = c1 - c0, rows = t << shift;
  auto seen = [&](int token) {                                  // cache rows that a token of the request sees
    const int pos = n - t + token + 1;
    return pos < 0 ? 0 : pos;
  };
  int m = row0 + (wave / kKeyWaves) * 32 + nrow;
  const bool valid = m < rows;
  m = valid ? m : rows - 1;
  const int token = m >> shift, head = g * G + (m & (G - 1));
  const int last = (row0 + 32 * kRowWaves < rows ? row0 + 32 * kRowWaves : rows) - 1;
  const auto walk = a.see.walk(seen(row0 >> shift) - 1, seen(last >> shift) - 1, seen(token) - 1);
  const int limit = valid ? walk.steps(seen(token)) : 0;
  int lo, hi;
  split_rows(0, walk.steps(seen(last >> shift)), splits, split, tile_rows(kKeyWaves), &lo, &hi);
  RowState<Op, 1> st;
  st.clear();
  if (lo < hi) {
    const CacheRows<TK> K(a.kv.k, a.kv, b, g);
    const CacheRows<TV> V(a.kv.v, a.kv, b, g);
    tile_loop<TK, TV, kKeyWaves>(lds, K, V, lo, hi, [&](auto& q) { q.load(a.q + (int64_t)(c0 + token) * a.q_stride + head * kD, h); }, limit, st, walk);
  }
  RowOut<TQ> to = {nullptr, nullptr};
  if (valid) {
    if (splits > 1) to.part = a.part + (part_row(a, kFew, few_most<TK>(), b, c0, token, head) + split) * kPartFloats;
    else to.out = a.out + ((int64_t)(c0 + token) * s.Hq + head) * kD;
  }
  tile_finish<Op, 1, kKeyWaves>(lds, st, to);
}

// The same with the loop of tile_pipe.h.
template <int kKind, typename TK, typename TV, typename TQ, typename See>
__device__ __forceinline__ void prompt_pipe(char* lds, const PromptArgs<TQ, See>& a, int b, int g, int c0, int c1, int row0, int split) {
  typedef typename InLds<TK>::Op Op;
  const Shape& s = a.s;
  const int G = s.G, shift = G == 4 ? 2 : G - 1;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), h = lane >> 5;
  const int n = length_of(s, a.kv.seq_lens, b), t = c1 - c0, rows = t << shift;
  auto seen = [&](int token) {
    const int pos = n - t + token + 1;
    return pos < 0 ? 0 : pos;
  };
  const int last = (row0 + kPipeRows < rows ? row0 + kPipeRows : rows) - 1;
  int m = row0 + 32 * wave + (lane & 31);
  const bool valid = m < rows;
  m = valid ? m : rows - 1;                                     // (rows that are not there repeat the last one)
  const int token = m >> shift, head = g * G + (m & (G - 1));
  const auto walk = a.see.walk(seen(row0 >> shift) - 1, seen(last >> shift) - 1, seen(token) - 1);
  int lo, hi;
  split_rows(0, walk.steps(seen(last >> shift)), a.splits, split, kPipeKeys, &lo, &hi);
  PipeState<Op> st;
  st.clear();
  st.limit = walk.steps(seen(token));
  lds_char* room = (lds_char*)lds + wave * (kPipeLds / kPipeWaves & ~15);
  if (lo < hi) {
    const CacheRows<TK> K(a.kv.k, a.kv, b, g);
    const CacheRows<TV> V(a.kv.v, a.kv, b, g);
    auto query = [&](int i) __attribute__((always_inline)) {
      const int x = min(row0 + 32 * wave + i, rows - 1);
      return reinterpret_cast<const char*>(a.q + (int64_t)(c0 + (x >> shift)) * a.q_stride + (g * G + (x & (G - 1))) * kD);
    };
    room = pipe_loop<kKind, TK, TV>(lds, K, V, lo, hi, walk.steps(seen(row0 >> shift)), row0 + 32 * wave < rows, st, walk, query);
  }
  if (a.splits > 1) {
    if (valid) st.finish((TQ*)nullptr, a.part + (part_row(a, false, 0, b, c0, token, head) + split) * kPartFloats, h);
    return;
  }
  const int first = row0 + 32 * wave;
  st.template finish_rows<TQ>(room, [&](int i) {
    const int x = first + i;
    return x < rows ? a.out + ((int64_t)(c0 + (x >> shift)) * s.Hq + g * G + (x & (G - 1))) * kD : nullptr;
  });
}

}  // namespace

template <typename TK>
constexpr int tile_query_rows() { return sizeof(TK) == 4 ? 128 : kPipeRows; }      // of a workgroup of k_prompt_tiles
template <typename TK>
constexpr int tile_threads() { return sizeof(TK) == 4 ? kTileThreads : kPipeThreads; }

// grid Hkv * splits * (tiles of all requests, at most T G / tile_query_rows + B), the latest rows of a request first: they see most
template <int kKind, typename TK, typename TV, typename TQ, typename See>
__global__ __launch_bounds__(tile_threads<TK>(), sizeof(TK) == 4 ? 1 : 2) void k_prompt_tiles(PromptArgs<TQ, See> a, int tiles) {
  constexpr int kRows = tile_query_rows<TK>();
  const int G = a.s.G, per = kRows / G;
  const int g = blockIdx.x % a.s.Hkv, x0 = blockIdx.x / a.s.Hkv, split = x0 % a.splits, x = tiles - 1 - x0 / a.splits;
  // tile x is among those of the last request b with cu[b] / per + b <= x: a request has no more tiles than lie between
  auto first_tile = [&](int i) {
    const int c = a.cu[i];
    return (c < 0 ? 0 : (c > a.n_tokens ? a.n_tokens : c)) / per + i;
  };
  const int b = last_not_above(a.s.B - 1, x, first_tile);
  int c0, c1;
  tokens_of(a, b, &c0, &c1);
  const int row0 = (x - first_tile(b)) * kRows;
  if (row0 < 0 || row0 >= (c1 - c0) * G) return;
  if (a.few_splits && (c1 - c0) * G <= few_most<TK>()) return;
  if constexpr (sizeof(TK) == 4) {
    __shared__ __attribute__((aligned(16))) char lds[tile_lds<TK, TV, 1>()];
    prompt_tile<TK, TV, 1>(lds, a, b, g, c0, c1, row0, split);
  } else {
    __shared__ __attribute__((aligned(16))) char lds[kPipeLds];
    prompt_pipe<kKind, TK, TV>(lds, a, b, g, c0, c1, row0, split);
  }
}

// grid Hkv * few_splits * B
template <typename TK, typename TV, typename TQ, typename See>
__global__ __launch_bounds__(kTileThreads) void k_prompt_few(PromptArgs<TQ, See> a) {
  request_arguments<decltype(&k_prompt_few<TK, TV, TQ, See>)>();
  constexpr int kKeyWaves = few_key_waves<TK>();
  __shared__ __attribute__((aligned(16))) char lds[tile_lds<TK, TV, kKeyWaves>()];
  const int g = blockIdx.x % a.s.Hkv, x0 = blockIdx.x / a.s.Hkv, split = x0 % a.few_splits, b = x0 / a.few_splits;
  int c0, c1;
  tokens_of(a, b, &c0, &c1);
  if (c0 >= c1 || (int64_t)(c1 - c0) * a.s.G > few_most<TK>()) return;
  prompt_tile<TK, TV, kKeyWaves>(lds, a, b, g, c0, c1, 0, split);
}

// The parts of a row -> its output row, a wave a (token, head).  few: of every request's first most / G tokens, if it has no more; else
// of every token of the other requests.
template <typename TQ, typename See>
__global__ __launch_bounds__(kTileThreads) void k_prompt_merge(PromptArgs<TQ, See> a, int few, int most) {
  request_arguments<decltype(&k_prompt_merge<TQ, See>)>();
  const int Hq = a.s.Hq, x = blockIdx.x * (kTileThreads / 64) + wave_of(), head = x % Hq, y = x / Hq;
  int b, i, c0, c1;
  if (few) {
    b = y / (most / a.s.G);
    i = y % (most / a.s.G);
    if (b >= a.s.B) return;
    tokens_of(a, b, &c0, &c1);
  } else {
    if (y >= a.n_tokens) return;
    b = last_not_above(a.s.B - 1, y, [&](int j) { return a.cu[j]; });
    tokens_of(a, b, &c0, &c1);
    i = y - c0;
  }
  const int t = c1 - c0;
  if (i < 0 || i >= t || (few != 0) != (a.few_splits && (int64_t)t * a.s.G <= most)) return;
  const float* const part = a.part + part_row(a, few != 0, most, b, c0, i, head) * kPartFloats;
  auto at = [&](int j) { return part + (int64_t)j * kPartFloats; };
  put2(a.out + ((int64_t)(c0 + i) * Hq + head) * kD + 2 * (threadIdx.x & 63),
       join_parts(few ? a.few_splits : a.splits, at, [&](int j) { return at(j)[kD]; }, [&](int j) { return at(j)[kD + 1]; }));
}

namespace {

template <typename TK, typename TV, typename TQ, typename See>
hipError_t prompt_t(const Shape& s, const KvView& kv, const See& see, const void* q, int64_t q_stride, const int32_t* cu, int n_tokens, void* out,
                    float* part, int64_t part_rows, hipStream_t st) {
  constexpr int kMost = few_most<TK>();
  PromptArgs<TQ, See> a = {s, kv, (const TQ*)q, q_stride, cu, n_tokens, (TQ*)out, part, 1, 0, 0, 0, see};
  const int per = tile_query_rows<TK>() / s.G;
  // As many parts as give every CU a workgroup (either kernel's LDS has room for one), where the rows' partial results have room.
  auto parts = [&](int64_t groups, int64_t rows, int64_t room) {
    int64_t n = (256 + groups - 1) / groups;
    if (n * rows > room) n = room / rows;
    const int64_t by_len = (see.most(s.Lcap, per) + 127) / 128;
    if (n > by_len) n = by_len;
    if (n > kMaxSplits) n = kMaxSplits;
    return (int)(n < 1 ? 1 : n);
  };
  // k_prompt_few makes 32 rows of work for a request of one token where k_prompt_tiles makes 256, but of 16-bit operands the latter's
  // loop asks for rows earlier and hides a stage's parts behind each other: it is the quicker one until the requests fill the chip by
  // themselves.  us, few / tiles: one token over 4100 rows of 8 KV heads 15.5 / 13.3, over 32768 38.1 / 33.1; 16 requests of 4 tokens
  // over 4100 rows 64.8 / 54.4 (FP8 65.0 / 49.9), of one over 8192 109 / 120 (111 / 87); 64 of one over 2048 112 / 123 (112 / 91), of
  // seven 113 / 171 (112 / 136).  fp32: 32 / 50, 135 / 239, 270 / 464, 514 / 900.  The rule looks at neither the format nor the lengths,
  // and so takes the slower one in two of these: bf16 16 of one over 8192 (120), FP8 64 of one over 2048 (112).
  // Only where the tiles are not many more than the requests: their number decides how many parts either has, and a single token over many
  // rows needs many, beside a prompt too (2048 tokens and seven single ones over 30000 rows 247 / 689, 512 and three over 16000 83 / 118;
  // eight ragged prompts of many tokens, where k_prompt_few finds nothing to do, 214 / 211).  What is left:
  // the tiles are those that the batch and n_tokens leave room for, not those that are there.  9 to 63 tokens over many rows beside a
  // long prompt are a workgroup a KV head (20 behind 30000 rows beside 2048: 607 us), and so are the few requests with tokens in a
  // context of many (20 tokens of one request behind 32768 rows: 41 us in a context of one, 335 of 16, 665 of 64; 512 tokens 319, 440, 771).
  const bool small = sizeof(TK) != 4 && s.B * s.Hkv <= 128 && n_tokens <= (int64_t)per * s.B;
  const bool all_few = !small && (int64_t)n_tokens * s.G <= kMost;
  // Over a short window a tile of few tokens is no longer than the others, and where the requests have a tile's tokens on average the two launches
  // cost more than they bring (six ragged fp16 chunks, window 517: 121 / 116 us; seven tokens and 512, window 5500: 131 / 97; one of 1000 and seven of 3,
  // window 4096: 128 / 132; 32 of 5, which have less: 105 / 213).
  const bool none_few = small || (!all_few && (s.B == 1 || (sizeof(TK) != 4 && n_tokens >= (int64_t)per * s.B && !see.few_apart(see.most(s.Lcap, per)))));
  const int tiles = n_tokens / per + s.B;
  if (!all_few) a.splits = parts((int64_t)tiles * s.Hkv, (int64_t)n_tokens * s.Hq, part_rows);
  if (a.splits > 1) a.few_part = (int64_t)n_tokens * s.Hq * a.splits;
  if (!none_few) {
    const int64_t room = (int64_t)s.B * (kMost / s.G);
    a.few_by_token = n_tokens <= room;
    a.few_splits = parts((int64_t)(s.B < n_tokens ? s.B : n_tokens) * s.Hkv, (a.few_by_token ? n_tokens : room) * s.Hq, part_rows - a.few_part);
  }
  const dim3 grid((unsigned)(s.Hkv * a.splits * tiles));
  if (!all_few) {
    const int kind = sizeof(TK) == 4 ? kAnyRows : rows_kind(kv);
    if (kind == kAnyRows) hipLaunchKernelGGL((k_prompt_tiles<kAnyRows, TK, TV, TQ, See>), grid, dim3(tile_threads<TK>()), 0, st, a, tiles);
    if constexpr (sizeof(TK) != 4) {
      if (kind == kSlab) hipLaunchKernelGGL((k_prompt_tiles<kSlab, TK, TV, TQ, See>), grid, dim3(tile_threads<TK>()), 0, st, a, tiles);
      if (kind == kPages) hipLaunchKernelGGL((k_prompt_tiles<kPages, TK, TV, TQ, See>), grid, dim3(tile_threads<TK>()), 0, st, a, tiles);
    }
  }
  if (!none_few)
    hipLaunchKernelGGL((k_prompt_few<TK, TV, TQ, See>), dim3((unsigned)(s.Hkv * a.few_splits * s.B)), dim3(kTileThreads), 0, st, a);
  auto merge = [&](int few, int64_t rows) {
    hipLaunchKernelGGL((k_prompt_merge<TQ, See>), dim3((unsigned)((rows + 3) / 4)), dim3(kTileThreads), 0, st, a, few, kMost);
  };
  if (a.splits > 1) merge(0, (int64_t)n_tokens * s.Hq);
  if (a.few_splits > 1) merge(1, (int64_t)s.B * (kMost / s.G) * s.Hq);
  return hipGetLastError();
}

}  // namespace

}  // namespace lfps
