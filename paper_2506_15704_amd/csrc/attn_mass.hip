// Accumulated attention weight: what the newest tokens of a request, packed, give every row of its cache, summed over them and the heads of a KV group,
//
//   mass[b, g, j] = (j < held_b ? decay * mass[b, g, j] : 0) + sum_{t, h in g} softmax_j(q[t, h] . K[b, g, j] / sqrt(D)).
//
// A weight needs the sum over its whole row, so the products are made twice, on the matrix units: k_mass_stats finds every query row's largest score
// and sum, k_mass_add the weights.  Scores are made as S^T = K Q^T in both: a lane has one query row and 16 of 32 keys.  In the first kernel a wave keeps
// its query rows in registers while the keys stream through LDS, and a lane the maximum and sum of its own keys; in the second a wave keeps its keys
// while the queries stream, and a lane the sum of its own queries' weights for each key.  So either reduces over lanes once, at the end, and the sums
// come in the same order every time.
//
// Long prompts are bound by the vector unit: a score costs three instructions, one of them an exponential of four times an ordinary one's cycles, in either
// kernel (81 % of the busy SIMDs' time in the first).  32 heads over 8 KV heads: 8192 tokens in bf16 620 us, two products of 550 GFLOP in all at 890 TFLOP/s;
// prompts of 5449 and 7958 tokens over FP8 pages 842 to 880 (by the profiler k_mass_stats 475, k_mass_add 460, k_mass_sum 5).  Requests of few tokens
// (k_mass_few) are bound by the bytes of K, read twice: 32 tokens over 32768 rows 37 to 40 us by the card, 17.6 + 4.7 + 18.5 by the profiler, where K's 67 MB are 14.
#include "tile_attn.h"

namespace lfps {

namespace {

constexpr int kMassThreads = 256, kMassWaves = kMassThreads / 64;
constexpr int kMassChunk = 1024;                       // query rows that a workgroup of k_mass_add takes at least, if there are as many
constexpr int kMassRing = 4;                           // stages of streamed rows in LDS
constexpr float kMassLazy = 6.f;                       // growth of a maximum, in powers of two, that is let pass
constexpr float kMassUnit = kLog2e * 0.08838834764831845f;      // from products to scores in powers of two

// Blocks of 32 rows that a wave keeps in registers: of 16-bit operands two, so that a row read from LDS serves two products.  A stage of streamed
// rows is 16 KB.
template <typename Op>
struct MassShape {
  static constexpr bool kF32 = std::is_same<Op, float>::value;
  static constexpr int kBlocks = kF32 ? 1 : 2, kMine = 32 * kBlocks, kRows = kMassWaves * kMine;       // of a wave; of a workgroup
  static constexpr int kRowBytes = kF32 ? 512 : 256, kStage = kF32 ? 32 : 64, kSubs = kStage / 32, kBytes = kStage * kRowBytes;
};

template <typename TQ>
struct MassArgs {
  Shape s;
  KvView kv;
  const TQ* q;
  int64_t q_stride;
  const int32_t *cu, *held;
  int32_t n_tokens, t0, t1;        // the tokens of this launch
  float decay;
  float* stats;                    // [Hkv, t1 - t0, G, 2] of a query row: its largest score in powers of two, the inverse of the sum of the weights from there
  float* split_stats;              // [splits, Hkv, t1 - t0, G, 2] of its parts, if there are several: the sums themselves
  int32_t splits;
  int32_t chunks;                  // of the query rows of a request
  int32_t few_rows;                // requests of up to so many query rows are k_mass_few's (-1: none, not even those of no tokens)
  float* sums;                     // [chunks, B * Hkv, Lcap] what the chunks of query rows leave for the rows that they see, if there are several
  float* mass;
};

// A row's 128 channels as the operands of lane (n, h): of step s the chunk 16 s + 8 h .. + 7, of fp32 the channels 8 s + 4 h .. + 3.
template <typename Op>
struct MassRow {
  Op x[8];
  __device__ __forceinline__ static Op chunk(const lds_char* rows, int c, int n, int h) {
    return *(const __attribute__((address_space(3))) Op*)(rows + n * 256 + 16 * chunk_place(n, 2 * c + h));
  }
  template <typename T>
  __device__ __forceinline__ void load(const T* p, int h) {
#pragma unroll
    for (int c = 0; c < 8; ++c) x[c] = *reinterpret_cast<const Op*>(p + 16 * c + 8 * h);
  }
  __device__ __forceinline__ void load(const lds_char* rows, int n, int h) {
#pragma unroll
    for (int c = 0; c < 8; ++c) x[c] = chunk(rows, c, n, h);
  }
};
template <>
struct MassRow<float> {
  f32x4 x[16];
  __device__ __forceinline__ static f32x4 chunk(const lds_char* rows, int c, int n, int h) {
    return *(const __attribute__((address_space(3))) f32x4*)(rows + n * 512 + 16 * chunk_place_f32(n, 2 * c + h));
  }
  __device__ __forceinline__ void load(const float* p, int h) {
#pragma unroll
    for (int c = 0; c < 16; ++c) x[c] = *reinterpret_cast<const f32x4*>(p + 8 * c + 4 * h);
  }
  __device__ __forceinline__ void load(const lds_char* rows, int n, int h) {
#pragma unroll
    for (int c = 0; c < 16; ++c) x[c] = chunk(rows, c, n, h);
  }
};

// out[i] = 32 rows in LDS times my block i, or with kLdsIsKeys = false my blocks times the rows in LDS (keys are the first operand), and beside the
// products, in eight pieces, beside(0) .. beside(7): vector instructions that do not wait for them.  (Left to itself the compiler puts all products
// first, and reads their operands one product ahead.)
template <bool kLdsIsKeys, typename Op, int kBlocks, typename Beside>
__device__ __forceinline__ void mass_scores(f32x16 (&out)[kBlocks], const lds_char* rows, const MassRow<Op> (&mine)[kBlocks], int n, int h, Beside beside) {
  if constexpr (std::is_same<Op, float>::value) {
    f32x4 a[3] = {MassRow<float>::chunk(rows, 0, n, h), MassRow<float>::chunk(rows, 1, n, h)};
#pragma unroll
    for (int c = 0; c < 16; ++c) {
      __builtin_amdgcn_sched_barrier(0);
      if (c + 2 < 16) a[(c + 2) % 3] = MassRow<float>::chunk(rows, c + 2, n, h);
#pragma unroll
      for (int e = 0; e < 4; ++e)
#pragma unroll
        for (int i = 0; i < kBlocks; ++i) {
          const f32x16 before = c + e == 0 ? zeros16() : out[i];
          out[i] = kLdsIsKeys ? mfma32(a[c % 3][e], mine[i].x[c][e], before) : mfma32(mine[i].x[c][e], a[c % 3][e], before);
        }
      if (c % 2) beside(c / 2);
    }
  } else {
    Op a[3] = {MassRow<Op>::chunk(rows, 0, n, h), MassRow<Op>::chunk(rows, 1, n, h)};
#pragma unroll
    for (int c = 0; c < 8; ++c) {
      __builtin_amdgcn_sched_barrier(0);
      if (c + 2 < 8) a[(c + 2) % 3] = MassRow<Op>::chunk(rows, c + 2, n, h);
#pragma unroll
      for (int i = 0; i < kBlocks; ++i) {
        const f32x16 before = c == 0 ? zeros16() : out[i];
        out[i] = kLdsIsKeys ? mfma32(a[c % 3], mine[i].x[c], before) : mfma32(mine[i].x[c], a[c % 3], before);
      }
      beside(c);
    }
  }
  __builtin_amdgcn_sched_barrier(0);
}

// All but the newest kNewer requests to memory of this wave have been answered.
template <int kNewer>
__device__ __forceinline__ void answered_but() { __builtin_amdgcn_s_waitcnt(0x0f70 | (kNewer & 15) | (kNewer >> 4 << 14)); }

// The key of a lane's product r among 32.
__device__ __forceinline__ int key_of(int r, int h) { return 8 * (r / 4) + 4 * h + r % 4; }

// Tokens [c0, c1) of request b that this launch takes, and the cache row of token 0, were it the request's.
template <typename A>
__device__ __forceinline__ int launch_tokens(const A& a, int b, int* c0, int* c1) {
  request_tokens(a.cu, a.n_tokens, b, c0, c1);
  const int first = length_of(a.s, a.kv.seq_lens, b) - *c1;
  *c0 = *c0 < a.t0 ? a.t0 : *c0;
  *c1 = *c1 > a.t1 ? a.t1 : *c1;
  return first;
}

}  // namespace

// grid Hkv * splits * tiles (of kRows query rows; at most T G / rows + B), the latest rows first: they see most.
// Stage j of keys is in LDS slot j % 4.  While a wave's weights of 32 keys are made, the products of the next 32 run; when the last 32 of stage j - 1
// are, a barrier says that nobody reads its slot any more and that stage j is there, and stage j + 3 is asked for (FP8: it comes from registers when
// its turn is next but one).
template <typename TK, typename TQ>
__global__ __launch_bounds__(kMassThreads, sizeof(TK) == 4 ? 1 : 2) void k_mass_stats(MassArgs<TQ> a, int tiles) {
  typedef typename InLds<TQ>::Op Op;
  typedef MassShape<Op> M;
  constexpr int kBlocks = M::kBlocks;
  __shared__ __attribute__((aligned(16))) char lds_[kMassRing * M::kBytes];
  const Shape& s = a.s;
  const int G = s.G, shift = G == 4 ? 2 : G - 1, per = M::kRows / G;
  const int g = blockIdx.x % s.Hkv, x0 = blockIdx.x / s.Hkv, split = x0 % a.splits, x = tiles - 1 - x0 / a.splits;
  auto first_tile = [&](int i) {
    const int c = a.cu[i];
    return ((c < a.t0 ? a.t0 : (c > a.t1 ? a.t1 : c)) - a.t0) / per + i;
  };
  const int b = last_not_above(s.B - 1, x, first_tile);
  int c0, c1;
  const int first = launch_tokens(a, b, &c0, &c1);
  const int row0 = (x - first_tile(b)) * M::kRows, rows = c1 > c0 ? (c1 - c0) << shift : 0;
  if (row0 < 0 || row0 >= rows || (a.few_rows == 128 && rows <= 128)) return;      // (of 256 rows k_mass_few's statistics spill registers: 64 / 60 us in all)
  const int lane = threadIdx.x & 63, wave = wave_of(), n = lane & 31, h = lane >> 5;
  auto seen = [&](int m) {                                     // keys that query row m sees
    const int y = first + c0 + (m >> shift) + 1;
    return y < 0 ? 0 : y;
  };
  const int last = (row0 + M::kRows < rows ? row0 + M::kRows : rows) - 1;
  int lo, hi;
  split_rows(0, seen(last), a.splits, split, M::kStage, &lo, &hi);
  const int mine0 = row0 + M::kMine * wave;
  int m[kBlocks], limit[kBlocks];
#pragma unroll
  for (int i = 0; i < kBlocks; ++i) {
    m[i] = mine0 + 32 * i + n;
    limit[i] = m[i] < rows ? seen(m[i]) : 0;
    limit[i] = limit[i] < hi ? limit[i] : hi;
  }
  int least = mine0 + M::kMine <= rows ? seen(mine0) : 0;      // keys that all of my rows see
  least = least < hi ? least : hi;
  float top[kBlocks], l[kBlocks][4];
#pragma unroll
  for (int i = 0; i < kBlocks; ++i) {
    top[i] = -INFINITY;
#pragma unroll
    for (int e = 0; e < 4; ++e) l[i][e] = 0.f;
  }
  if (lo < hi) {
    lds_char* const lds = (lds_char*)lds_;
    const CacheRows<TK> K(a.kv.k, a.kv, b, g);
    typedef StageFeed<TK, M::kStage / kMassWaves, Op> Feed;
    Feed feed;
    typename Feed::Places at;
    const int stages = (hi - lo + M::kStage - 1) / M::kStage;
    auto slot = [&](int j) { return lds + (j & (kMassRing - 1)) * M::kBytes; };
    auto row_of = [&](int j) { return lo + j * M::kStage; };
    // stage j, whose places have been looked up; then the look-up of the next one comes first: waiting for it need be no wait for the rows (the compiler,
    // which does not know here whether there are pages, makes it one for all requests)
    auto ask = [&](int j) {
      at.aim(K, row_of(j), hi, lane);
      __builtin_amdgcn_sched_barrier(0);
      if (j + 1 < stages) at.look_up(K, row_of(j + 1), hi, lane);
      __builtin_amdgcn_sched_barrier(0);
      feed.ask(K, at.off, slot(j), lane);
      __builtin_amdgcn_sched_barrier(0);
    };
    constexpr int kAhead = kMassRing - 1;                      // stages that are on their way
    at.look_up(K, lo, hi, lane);
    for (int j = 0; j <= kAhead && j < stages; ++j) {
      ask(j);
      if (j < kAhead) feed.put(slot(j), lane);                 // (FP8: the last one stays in registers)
    }
    MassRow<Op> q[kBlocks];
#pragma unroll
    for (int i = 0; i < kBlocks; ++i) {
      const int token = c0 + ((m[i] < rows ? m[i] : rows - 1) >> shift);
      q[i].load(a.q + (int64_t)token * a.q_stride + (g * G + (m[i] & (G - 1))) * kD, h);
    }
    answered_but<0>();
    __syncthreads();
    const int subs = (hi - lo + 31) / 32;
    // between the products of the keys 32 i .. and those of the next: where these begin a stage j, stage j - 1 has been read
    auto turn = [&](int i) __attribute__((always_inline)) {
      if ((i + 1) % M::kSubs != 0 || i + 1 >= subs) return;
      const int j = (i + 1) / M::kSubs;
      if (Feed::kDirect && j + 2 < stages) answered_but<2 * Feed::kLoads>();
      else if (Feed::kDirect) answered_but<0>();
      __syncthreads();
      if (!Feed::kDirect && j + kAhead - 1 < stages) feed.put(slot(j + kAhead - 1), lane);
      if (j + kAhead < stages) ask(j + kAhead);
    };
    // the weights of the keys 32 i .. of the walk, from y, beside the products of the next 32, to next
    auto step = [&](int i, f32x16 (&y)[kBlocks], f32x16 (&next)[kBlocks]) __attribute__((always_inline)) {
      const int key0 = lo + 32 * i;
      if (key0 + 32 > least) {                                 // (some of my rows do not see all of them)
#pragma unroll
        for (int c = 0; c < kBlocks; ++c)
#pragma unroll
          for (int r = 0; r < 16; ++r) y[c][r] = key0 + key_of(r, h) < limit[c] ? y[c][r] : -INFINITY;
      }
      turn(i);
      float from[kBlocks];
      auto weigh = [&](int c) __attribute__((always_inline)) {
        if (c < kBlocks) {                                     // (block c's new maximum)
          float mx = fmaxf(y[c][0], y[c][1]);
#pragma unroll
          for (int r = 2; r < 16; r += 2) mx = fmaxf(fmaxf(mx, y[c][r]), y[c][r + 1]);
          mx *= kMassUnit;
          const bool grows = mx > top[c] + kMassLazy;
          const float shrink = grows ? __builtin_amdgcn_exp2f(top[c] - mx) : 1.f;      // (0 on the first keys)
          top[c] = grows ? mx : top[c];
          from[c] = top[c] == -INFINITY ? 0.f : top[c];
#pragma unroll
          for (int e = 0; e < 4; ++e) l[c][e] *= shrink;
        } else {
          constexpr int kAll = 16 * kBlocks, kPieces = 8 - kBlocks;
#pragma unroll
          for (int e = kAll * (c - kBlocks) / kPieces; e < kAll * (c - kBlocks + 1) / kPieces; ++e)
            l[e / 16][e % 4] += __builtin_amdgcn_exp2f(fmaf(y[e / 16][e % 16], kMassUnit, -from[e / 16]));
        }
      };
      const lds_char* const keys = slot((i + 1) / M::kSubs) + (i + 1) % M::kSubs * (32 * M::kRowBytes);
      mass_scores<true, Op, kBlocks>(next, keys, q, n, h, weigh);       // (behind the last keys: what lies there, unused)
    };
    if (mine0 < rows) {
      f32x16 even[kBlocks], odd[kBlocks];
      mass_scores<true, Op, kBlocks>(even, slot(0), q, n, h, [](int) {});
      for (int i = 0; i < subs; i += 2) {
        step(i, even, odd);
        if (i + 1 >= subs) break;
        step(i + 1, odd, even);
      }
    } else {                                                   // (a wave without rows only brings its share of the keys)
      for (int i = 0; i < subs; ++i) turn(i);
    }
  }
#pragma unroll
  for (int i = 0; i < kBlocks; ++i) {
    const float sum = (l[i][0] + l[i][1]) + (l[i][2] + l[i][3]), other_top = __shfl_xor(top[i], 32), other = __shfl_xor(sum, 32);
    const float mx = fmaxf(top[i], other_top);
    // (a half that has seen nothing has a sum of 0, or of NaN scores a NaN)
    auto part = [&](float t, float y) { return y != y ? y : (t == -INFINITY ? 0.f : y * __builtin_amdgcn_exp2f(t - mx)); };
    const float both = part(top[i], sum) + part(other_top, other);
    if (h == 0 && m[i] < rows) {
      const int64_t count = a.t1 - a.t0, row = (g * count + (c0 - a.t0)) * G + m[i];
      if (a.splits > 1) *reinterpret_cast<f32x2t*>(a.split_stats + 2 * (split * count * s.Hq + row)) = f32x2t{mx, both};
      else *reinterpret_cast<f32x2t*>(a.stats + 2 * row) = f32x2t{mx == -INFINITY ? 0.f : mx, both == 0.f ? 0.f : 1.f / both};
    }
  }
}

// The parts of every query row, joined: 16 rows a workgroup, 16 threads a row.
__global__ __launch_bounds__(256) void k_mass_join(const float* __restrict__ split_stats, float* __restrict__ stats, int64_t rows, int splits) {
  __shared__ f32x2t half[4][16];
  const int64_t row = (int64_t)blockIdx.x * 16 + (threadIdx.x & 15), at = row < rows ? row : rows - 1;
  constexpr int kEach = kMaxSplits / 16;
  const f32x2t* const part = reinterpret_cast<const f32x2t*>(split_stats) + at;
  f32x2t x[kEach];
#pragma unroll
  for (int i = 0; i < kEach; ++i) {
    const int p = (int)(threadIdx.x >> 4) + 16 * i;
    x[i] = part[(p < splits ? p : 0) * rows];
    if (p >= splits) x[i] = f32x2t{-INFINITY, 0.f};
  }
  float mx = -INFINITY, sum = 0.f;
  auto scaled = [&](f32x2t y) { return y[1] != y[1] ? y[1] : (y[0] == -INFINITY ? 0.f : y[1] * __builtin_amdgcn_exp2f(y[0] - mx)); };
#pragma unroll
  for (int i = 0; i < kEach; ++i) mx = fmaxf(mx, x[i][0]);
  mx = fmaxf(mx, __shfl_xor(mx, 16));
  mx = fmaxf(mx, __shfl_xor(mx, 32));
#pragma unroll
  for (int i = 0; i < kEach; ++i) sum += scaled(x[i]);
  sum += __shfl_xor(sum, 16);
  sum += __shfl_xor(sum, 32);
  if ((threadIdx.x & 63) < 16) half[threadIdx.x >> 6][threadIdx.x & 15] = f32x2t{mx, sum};
  __syncthreads();
  if (threadIdx.x >= 16 || row >= rows) return;
#pragma unroll
  for (int w = 0; w < 4; ++w) mx = fmaxf(mx, half[w][threadIdx.x][0]);
  sum = 0.f;
#pragma unroll
  for (int w = 0; w < 4; ++w) sum += scaled(half[w][threadIdx.x]);
  reinterpret_cast<f32x2t*>(stats)[row] = f32x2t{mx == -INFINITY ? 0.f : mx, sum == 0.f ? 0.f : 1.f / sum};
}

// Query rows of a chunk, of `all`; and the first row that sees keys from `tile` on, a multiple of kStage, `first` being the place of row 0's token.
template <int kStage>
__device__ __forceinline__ int chunk_rows(int all, int chunks) {
  const int even = ((all + chunks - 1) / chunks + kStage - 1) & ~(kStage - 1);
  return even > kMassChunk ? even : kMassChunk;
}
template <int kStage>
__device__ __forceinline__ int first_to_see(int tile, int first, int shift) { return tile > first ? ((tile - first) << shift) & ~(kStage - 1) : 0; }

// grid (B * Hkv, tiles of kRows keys, chunks of query rows: of every request the same number).  Workgroups go round the XCDs, and within one round its
// shader engines, in the order of their numbers, and one that waits for a place keeps the others waiting: with the tiles first, of which the later
// ones are seen by fewer, the first engines of every XCD had twice the work of the average (8192 tokens of 32 heads 528 us); where a round of groups
// is two to the XCD, its engines would have one request each, so their order changes from tile to tile (prompts of 5449 and 7958 tokens 551 -> 462 us).
// (As many workgroups as the chip holds, which took the parts from a line with a counter, spilled registers: 489.)
// A wave's keys come through the ring's slot of its number into registers; then the query rows stream through it as the keys do in k_mass_stats.
template <typename TK, typename TQ>
__global__ __launch_bounds__(kMassThreads, sizeof(TK) == 4 ? 1 : 2) void k_mass_add(MassArgs<TQ> a) {
  typedef typename InLds<TQ>::Op Op;
  typedef MassShape<Op> M;
  constexpr int kBlocks = M::kBlocks, kBytes = M::kBytes + M::kStage * 8;      // (with the rows' statistics)
  static_assert(kMassWaves == kMassRing && M::kMine * M::kRowBytes == M::kBytes, "a slot is a wave's keys");
  __shared__ __attribute__((aligned(16))) char lds_[kMassRing * kBytes];       // (one array: of several the compiler waits for all requests before any read)
  request_arguments<decltype(&k_mass_add<TK, TQ>)>();
  const Shape& s = a.s;
  const int G = s.G, shift = G == 4 ? 2 : G - 1, chunks = a.chunks;
  const int bg = (blockIdx.x + 8 * (blockIdx.y / 2)) % (s.B * s.Hkv), b = bg / s.Hkv, g = bg % s.Hkv, tile = blockIdx.y * M::kRows;
  const int len = length_of(s, a.kv.seq_lens, b);
  if (tile >= len) return;
  const int lane = threadIdx.x & 63, wave = wave_of(), n = lane & 31, h = lane >> 5;
  int c0, c1;
  const int first = launch_tokens(a, b, &c0, &c1);
  const int all = c1 > c0 ? (c1 - c0) << shift : 0, chunk = chunk_rows<M::kStage>(all, chunks), at_chunk = blockIdx.z, chunk0 = at_chunk * chunk;
  const int rows = all - chunk0 < chunk ? all : chunk0 + chunk;
  int m0 = first_to_see<M::kStage>(tile, first + c0, shift);
  m0 = m0 < chunk0 ? chunk0 : m0;
  if (all <= a.few_rows) return;
  if (m0 >= rows && chunks > 1) return;                     // (k_mass_sum leaves such chunks out)
  const int key0 = tile + M::kMine * wave;
  float sum[kBlocks][16];
#pragma unroll
  for (int i = 0; i < kBlocks; ++i)
#pragma unroll
    for (int r = 0; r < 16; ++r) sum[i][r] = 0.f;
  lds_char* const lds = (lds_char*)lds_;
  if (m0 < rows) {
    auto slot = [&](int j) { return lds + (j & (kMassRing - 1)) * kBytes; };
    MassRow<Op> k[kBlocks];
    {
      const CacheRows<TK> K(a.kv.k, a.kv, b, g);
      typedef StageFeed<TK, M::kMine, Op> Feed;                // (as many rows as a wave's: "stage" rows kMine * wave .. are my own keys)
      Feed feed;
      typename Feed::Places at;
      at.look_up(K, tile, len, lane);
      at.aim(K, tile, len, lane);
      lds_char* const mine = slot(wave) - wave * M::kBytes;    // (the feed adds its own rows' places)
      feed.ask(K, at.off, mine, lane);
      feed.put(mine, lane);
      wave_lds_order();
      __builtin_amdgcn_s_waitcnt(0x0070);                      // vmcnt(0) lgkmcnt(0)
      wave_lds_order();
#pragma unroll
      for (int i = 0; i < kBlocks; ++i) k[i].load(slot(wave) + 32 * i * M::kRowBytes, n, h);
      __builtin_amdgcn_s_waitcnt(0xc07f);                      // lgkmcnt(0)
      __syncthreads();
    }
    // a stage of query rows: 1 KB an instruction, lane l fills the l-th 16 bytes of it with the chunk that belongs there; and their statistics, 4
    // bytes a lane
    constexpr int kPieces = M::kRowBytes / 16, kEach = 64 / kPieces, kWaveRows = M::kStage / kMassWaves, kLoads = kWaveRows / kEach;
    const int stages = (rows - m0 + M::kStage - 1) / M::kStage;
    const float* const stats = a.stats + 2 * (((int64_t)g * (a.t1 - a.t0) + (c0 - a.t0)) * G);
    // My pieces of a stage, counted from its first query row: a stage begins with a token.
    int64_t off[kLoads];
    auto place_of = [&](int i, int row) {                      // of query row `row` of those that the pieces are counted from
      const int r = kWaveRows * wave + kEach * i + lane / kPieces, place = lane % kPieces;
      return ((int64_t)(row >> shift) * a.q_stride + (row & (G - 1)) * kD) * (int64_t)sizeof(TQ) + 16 * (M::kF32 ? chunk_place_f32(r, place) : chunk_place(r, place));
    };
    auto my_row = [&](int i) { return kWaveRows * wave + kEach * i + lane / kPieces; };
#pragma unroll
    for (int i = 0; i < kLoads; ++i) off[i] = place_of(i, my_row(i));
    auto ask = [&](int j) __attribute__((always_inline)) {
      lds_char* const to = slot(j);
      const int m = m0 + j * M::kStage;
      const char* const q = reinterpret_cast<const char*>(a.q + (int64_t)(c0 + (m >> shift)) * a.q_stride + g * G * kD);
      const char* p[kLoads];
#pragma unroll
      for (int i = 0; i < kLoads; ++i) p[i] = q + off[i];
      int row = kWaveRows * wave + lane / 2;
      if (m + M::kStage > rows) {                              // (rows that are not there repeat the last one)
        const int last = rows - 1 - m;
#pragma unroll
        for (int i = 0; i < kLoads; ++i) p[i] = q + place_of(i, my_row(i) < last ? my_row(i) : last);
        row = row < last ? row : last;
      }
#pragma unroll
      for (int i = 0; i < kLoads; ++i)
        __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) char*)p[i],
                                         (__attribute__((address_space(3))) void*)(to + (kWaveRows * wave + kEach * i) * M::kRowBytes), 16, 0, 0);
      if (lane < 2 * kWaveRows)
        __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) char*)(stats + 2 * (int64_t)m + (2 * row + (lane & 1))),
                                         (__attribute__((address_space(3))) void*)(to + M::kBytes + kWaveRows * wave * 8), 4, 0, 0);
    };
    constexpr int kRequests = kLoads + 1;
    for (int j = 0; j < kMassRing && j < stages; ++j) ask(j);
    answered_but<0>();
    __syncthreads();
    const int subs = (rows - m0 + 31) / 32;
    // as in k_mass_stats; of stage j - 1 the statistics have been read too.  (The compiler puts a wait for all requests in front of most of these barriers.)
    auto turn = [&](int i) __attribute__((always_inline)) {
      if ((i + 1) % M::kSubs != 0 || i + 1 >= subs) return;
      const int j = (i + 1) / M::kSubs;
      if (j + 2 < stages) answered_but<2 * kRequests>();
      else answered_but<0>();
      __builtin_amdgcn_s_waitcnt(0xc07f);                      // lgkmcnt(0)
      __syncthreads();
      if (j + kMassRing - 1 < stages) ask(j + kMassRing - 1);
    };
    auto step = [&](int i, f32x16 (&y)[kBlocks], f32x16 (&next)[kBlocks]) __attribute__((always_inline)) {
      f32x2t st = *(const __attribute__((address_space(3))) f32x2t*)(slot(i / M::kSubs) + M::kBytes + 8 * (i % M::kSubs * 32 + n));
      const int mi = m0 + 32 * i;
      if (mi + 32 > rows || first + c0 + (mi >> shift) < key0 + M::kMine - 1) {      // not all of these queries see all of my keys
        const int pos = mi + n < rows ? first + c0 + ((mi + n) >> shift) - key0 : -1;
        const bool none = st[1] != st[1];                       // (a row of NaN: its scores say so, for its factor would to all keys)
        if (none) st = f32x2t{0.f, 0.f};
#pragma unroll
        for (int e = 0; e < 16 * kBlocks; ++e) {
          const float x = none ? __builtin_nanf("") : y[e / 16][e % 16];
          y[e / 16][e % 16] = 32 * (e / 16) + key_of(e % 16, h) <= pos ? x : -INFINITY;
        }
      }
      turn(i);
      auto weigh = [&](int c) __attribute__((always_inline)) {
        constexpr int kAll = 16 * kBlocks;
#pragma unroll
        for (int e = kAll * c / 8; e < kAll * (c + 1) / 8; ++e)
          sum[e / 16][e % 16] = fmaf(__builtin_amdgcn_exp2f(fmaf(y[e / 16][e % 16], kMassUnit, -st[0])), st[1], sum[e / 16][e % 16]);
      };
      const lds_char* const queries = slot((i + 1) / M::kSubs) + (i + 1) % M::kSubs * (32 * M::kRowBytes);
      mass_scores<false, Op, kBlocks>(next, queries, k, n, h, weigh);
    };
    if (key0 < len) {
      f32x16 even[kBlocks], odd[kBlocks];
      // (the first queries, which see none of my keys, are the other waves')
      int skip = ((key0 - first - c0) << shift) - m0;
      skip = skip < 0 ? 0 : skip / 32;
      skip = skip < subs ? skip : subs;
      for (int i = 0; i < skip; ++i) turn(i);
      if (skip < subs) mass_scores<false, Op, kBlocks>(even, slot(skip / M::kSubs) + skip % M::kSubs * (32 * M::kRowBytes), k, n, h, [](int) {});
      for (int i = skip; i < subs; i += 2) {
        step(i, even, odd);
        if (i + 1 >= subs) break;
        step(i + 1, odd, even);
      }
    } else {
      for (int i = 0; i < subs; ++i) turn(i);
    }
    __syncthreads();
  }
  float* const mine = reinterpret_cast<float*>(lds_) + wave * M::kMine;
#pragma unroll
  for (int kb = 0; kb < kBlocks; ++kb)
#pragma unroll
    for (int r = 0; r < 16; ++r) {
      float x = row16_sum(sum[kb][r]);
      x += __shfl_xor(x, 16);
      if (n == 0) mine[32 * kb + key_of(r, h)] = x;
    }
  wave_lds_order();
  const int key = key0 + lane;
  if (lane < M::kMine && key < len) {
    if (chunks > 1) {
      a.sums[((int64_t)at_chunk * (s.B * s.Hkv) + bg) * s.Lcap + key] = mine[lane];
    } else {
      float* const to = a.mass + (int64_t)bg * s.Lcap + key;
      const int held = a.held ? a.held[b] : 0;
      *to = mine[lane] + (a.t0 > 0 ? *to : (key < held ? a.decay * *to : 0.f));
    }
  }
}

// A lane's operands of a row of the cache as they are stored.
template <typename TK, typename Op>
struct MassRaw {
  static constexpr int kChunks = sizeof(TK) == 4 ? 16 : 8;
  typedef typename std::conditional<sizeof(TK) == 1, u32x2, typename std::conditional<sizeof(TK) == 4, f32x4, Op>::type>::type Chunk;
  Chunk x[kChunks];
  __device__ __forceinline__ void load(const TK* p, int h) {
#pragma unroll
    for (int c = 0; c < kChunks; ++c) x[c] = *reinterpret_cast<const Chunk*>(p + kD / kChunks * c + kD / kChunks / 2 * h);
  }
  __device__ __forceinline__ auto chunk(int c) const {
    if constexpr (sizeof(TK) == 1) return fp8x8_to<Op>(x[c][0], x[c][1]);
    else return x[c];
  }
};

// Requests of few query rows, up to kFew: all of these stay in LDS, and a wave streams keys of its own through its registers, 32 at a time, the next ones on
// their way, with nobody to wait for.  kStats: the rows' largest scores and sums over my keys (grid y: a part of them each); else the weights (in turn).
// grid (B * Hkv, parts: steps of 128 keys in turn).  32 tokens of 32 heads over 32768 rows: statistics 19.6 -> 17.6 us, where only the waves with query
// rows of their own had work in k_mass_stats; weights 29.9 -> 18.4, where k_mass_add waits for its keys, then for the queries, and has two stages of work (for
// 512 / 768 / 1024 / 1536 workgroups 19.7 / 18.4 / 21.3 / 21.4; statistics joined here: 24.1, where k_mass_join takes 4.7, and 44 us in all for 40.6).
// 64 tokens, 256 rows: 70 -> 60 us in all.  fp32, six requests of 4 to 40 tokens of 4 heads over 9000 to 20600 rows: 159 -> 123 us, of which
// ten are launches that find no request of more.
template <typename TK, typename TQ, int kFew, bool kStats>
__global__ __launch_bounds__(kMassThreads, !kStats && kFew == 128 && sizeof(TQ) == 2 ? 3 : 2) void k_mass_few(MassArgs<TQ> a, int parts) {
  request_arguments<decltype(&k_mass_few<TK, TQ, kFew, kStats>)>();
  typedef typename InLds<TQ>::Op Op;
  typedef MassShape<Op> M;
  constexpr int kSubs = kFew / 32, kStep = 32 * kMassWaves, kPieces = M::kRowBytes / 16, kMinePieces = kFew * kPieces / kMassThreads;
  __shared__ __attribute__((aligned(16))) char lds_[kFew * M::kRowBytes + (kStats ? kMassWaves * kFew * 8 : 0)];
  const Shape& s = a.s;
  const int G = s.G, shift = G == 4 ? 2 : G - 1, bg = blockIdx.x, b = bg / s.Hkv, g = bg % s.Hkv, len = length_of(s, a.kv.seq_lens, b);
  const int lane = threadIdx.x & 63, wave = wave_of(), n = lane & 31, h = lane >> 5;
  int at = kStep * (int)blockIdx.y;
  if (at >= len && !kStats) return;
  int c0, c1;
  const int first = launch_tokens(a, b, &c0, &c1), rows = c1 > c0 ? (c1 - c0) << shift : 0, subs = (rows + 31) / 32;
  if (rows > a.few_rows || (kStats && rows == 0)) return;
  lds_char* const lds = (lds_char*)lds_;
  const CacheRows<TK> K(a.kv.k, a.kv, b, g);
  auto my_row = [&](int step) {
    const int r = step + 32 * wave + n;
    return r < len ? r : len - 1;
  };
  const int64_t count = a.t1 - a.t0, row0 = ((int64_t)g * count + (c0 - a.t0)) * G;      // of the statistics
  float top[kSubs], l[kSubs];
  f32x2t st[kSubs];
#pragma unroll
  for (int u = 0; u < kSubs; ++u) {
    top[u] = -INFINITY;
    l[u] = 0.f;
    st[u] = f32x2t{0.f, 0.f};                                  // (of rows that are not there: their weights too)
  }
  if (at < len) {
    int entry = K.entry(my_row(at));
    u32x4 x[kMinePieces];                                      // my pieces of the queries; rows that are not there are 0
#pragma unroll
    for (int i = 0; i < kMinePieces; ++i) {
      const int piece = (int)threadIdx.x + kMassThreads * i, r = piece / kPieces, place = piece % kPieces;
      const int chunk = M::kF32 ? chunk_place_f32(r, place) : chunk_place(r, place);
      x[i] = u32x4{0, 0, 0, 0};
      if (r < rows)
        x[i] = *reinterpret_cast<const u32x4*>(a.q + (int64_t)(c0 + (r >> shift)) * a.q_stride + (g * G + (r & (G - 1))) * kD + 16 / (int)sizeof(TQ) * chunk);
    }
    if constexpr (!kStats) {
#pragma unroll
      for (int u = 0; u < kSubs; ++u)
        if (32 * u + n < rows) st[u] = *reinterpret_cast<const f32x2t*>(a.stats + 2 * (row0 + 32 * u + n));
    }
    MassRaw<TK, Op> raw;
    raw.load(K.at(my_row(at), entry), h);
    const int stride = kStep * parts;
    entry = K.entry(my_row(at + stride));
#pragma unroll
    for (int i = 0; i < kMinePieces; ++i) *(__attribute__((address_space(3))) u32x4*)(lds + 16 * ((int)threadIdx.x + kMassThreads * i)) = x[i];
    __syncthreads();
    const int held = a.held ? a.held[b] : 0;
    for (; at < len; at += stride) {
      MassRow<Op> k[1];
#pragma unroll
      for (int c = 0; c < MassRaw<TK, Op>::kChunks; ++c) k[0].x[c] = raw.chunk(c);
      if (at + stride < len) {
        raw.load(K.at(my_row(at + stride), entry), h);
        entry = K.entry(my_row(at + 2 * stride));
      }
      const int key0 = at + 32 * wave;
      if (key0 >= len) continue;
      const int mine = key0 + key_of(lane & 15, h);            // the key whose sum I have in the end
      float* const to = a.mass + (int64_t)bg * s.Lcap + mine;
      float old = 0.f;
      if constexpr (!kStats) old = mine < len && (a.t0 > 0 || mine < held) ? *to * (a.t0 > 0 ? 1.f : a.decay) : 0.f;
      float sum[16];
#pragma unroll
      for (int r = 0; r < 16; ++r) sum[r] = 0.f;
      const bool all_seen = key0 + 31 <= first + c0;
#pragma unroll
      for (int u = 0; u < kSubs; ++u) {
        if (u >= subs) break;
        f32x16 y[1];
        mass_scores<false, Op, 1>(y, lds + 32 * u * M::kRowBytes, k, n, h, [](int) {});
        float from = st[u][0], factor = st[u][1];
        // (as in k_mass_add; and a row that is not there is 0, whose product with an infinity is not, so that no statistics hide it)
        if (!all_seen || (!kStats && 32 * u + 32 > rows)) {
          const int m = 32 * u + n, pos = m < rows ? first + c0 + (m >> shift) - key0 : -1;
          const bool none = !kStats && factor != factor;
          if (none) from = factor = 0.f;
#pragma unroll
          for (int r = 0; r < 16; ++r) {
            const float v = none ? __builtin_nanf("") : y[0][r];
            y[0][r] = key_of(r, h) <= pos ? v : -INFINITY;
          }
        }
        if constexpr (kStats) {
          float mx = fmaxf(y[0][0], y[0][1]);
#pragma unroll
          for (int r = 2; r < 16; r += 2) mx = fmaxf(fmaxf(mx, y[0][r]), y[0][r + 1]);
          mx *= kMassUnit;
          const bool grows = mx > top[u] + kMassLazy;
          const float shrink = grows ? __builtin_amdgcn_exp2f(top[u] - mx) : 1.f;      // (0 on the first keys)
          top[u] = grows ? mx : top[u];
          from = top[u] == -INFINITY ? 0.f : top[u];
          float e[4] = {l[u] * shrink, 0.f, 0.f, 0.f};
#pragma unroll
          for (int r = 0; r < 16; ++r) e[r % 4] += __builtin_amdgcn_exp2f(fmaf(y[0][r], kMassUnit, -from));
          l[u] = (e[0] + e[1]) + (e[2] + e[3]);
          __builtin_amdgcn_sched_barrier(0);                   // (registers: one block's products at a time)
        } else {
#pragma unroll
          for (int r = 0; r < 16; ++r) sum[r] = fmaf(__builtin_amdgcn_exp2f(fmaf(y[0][r], kMassUnit, -from)), factor, sum[r]);
        }
      }
      if constexpr (!kStats) {
        // over the 32 lanes of a half: lane j of 16 is left with the sum of product j
#define LFPS_HALVE(W, GIVEN)                                                      \
  _Pragma("unroll") for (int i = 0; i < W; ++i) {                                 \
        const bool up = lane & W;                                                     \
        const float keep = up ? sum[i + W] : sum[i], give = up ? sum[i] : sum[i + W]; \
        sum[i] = keep + GIVEN;                                                        \
  }
        LFPS_HALVE(8, row16_rotate<8>(give))
        LFPS_HALVE(4, __shfl_xor(give, 4))
        LFPS_HALVE(2, __shfl_xor(give, 2))
        LFPS_HALVE(1, __shfl_xor(give, 1))
#undef LFPS_HALVE
        const float total = sum[0] + __shfl_xor(sum[0], 16);
        if (!(lane & 16) && mine < len) *to = total + old;
      }
    }
  }
  if constexpr (kStats) {
    // a row's parts: of the two halves of a wave, then of the four waves
    typedef __attribute__((address_space(3))) f32x2t* Parts;
    const Parts left = (Parts)(lds + kFew * M::kRowBytes);
    auto from_there = [](float t, float y, float mx) { return y != y ? y : (t == -INFINITY ? 0.f : y * __builtin_amdgcn_exp2f(t - mx)); };
#pragma unroll
    for (int u = 0; u < kSubs; ++u) {
      const float other_top = __shfl_xor(top[u], 32), other = __shfl_xor(l[u], 32), mx = fmaxf(top[u], other_top);
      if (h == 0) left[wave * kFew + 32 * u + n] = f32x2t{mx, from_there(top[u], l[u], mx) + from_there(other_top, other, mx)};
    }
    __syncthreads();
    const int m = threadIdx.x;
    if (m < rows) {
      float mx = -INFINITY, sum = 0.f;
#pragma unroll
      for (int w = 0; w < kMassWaves; ++w) mx = fmaxf(mx, left[w * kFew + m][0]);
#pragma unroll
      for (int w = 0; w < kMassWaves; ++w) sum += from_there(left[w * kFew + m][0], left[w * kFew + m][1], mx);
      if (a.splits > 1) *reinterpret_cast<f32x2t*>(a.split_stats + 2 * (blockIdx.y * count * s.Hq + row0 + m)) = f32x2t{mx, sum};
      else *reinterpret_cast<f32x2t*>(a.stats + 2 * (row0 + m)) = f32x2t{mx == -INFINITY ? 0.f : mx, sum == 0.f ? 0.f : 1.f / sum};
    }
  }
}

// The chunks' sums, in order.  grid (rows / 256, B * Hkv).  kRows, kStage: of k_mass_add
template <int kRows, int kStage, typename A>
__global__ __launch_bounds__(256) void k_mass_sum(A a) {
  const int chunks = a.chunks, bg = blockIdx.y, b = bg / a.s.Hkv, key = blockIdx.x * 256 + threadIdx.x, G = a.s.G, shift = G == 4 ? 2 : G - 1;
  if (key >= length_of(a.s, a.kv.seq_lens, b)) return;
  int c0, c1;
  const int first = launch_tokens(a, b, &c0, &c1), all = c1 > c0 ? (c1 - c0) << shift : 0, chunk = chunk_rows<kStage>(all, chunks);
  if (all <= a.few_rows) return;
  const int m0 = first_to_see<kStage>(key / kRows * kRows, first + c0, shift);
  const float* const from = a.sums + (int64_t)bg * a.s.Lcap + key;
  float sum = 0.f;
  if (m0 < all) {
#pragma unroll 4
    for (int c = m0 / chunk; c < (all + chunk - 1) / chunk; ++c) sum += from[(int64_t)c * gridDim.y * a.s.Lcap];
  }
  float* const to = a.mass + (int64_t)bg * a.s.Lcap + key;
  const int held = a.held ? a.held[b] : 0;
  *to = sum + (a.t0 > 0 ? *to : (key < held ? a.decay * *to : 0.f));
}

template <typename TK, typename TQ>
static hipError_t mass_t(MassArgs<TQ> a, float* work, int64_t room, hipStream_t st) {
  typedef MassShape<typename InLds<TQ>::Op> M;
  const int64_t most = room / 2 / a.s.Hq;                            // tokens that the workspace has room for
  // (by the average: what a request has is known on the device)
  const int64_t all = (int64_t)a.n_tokens * a.s.G, wide = M::kF32 ? 128 : 256;
  a.few_rows = all <= (int64_t)128 * a.s.B ? 128 : (all <= wide * a.s.B ? (int)wide : -1);
  const int per = M::kRows / a.s.G;
  const int64_t groups = (int64_t)a.s.B * a.s.Hkv, masses = groups * a.s.Lcap, steps = (a.s.Lcap + 32 * kMassWaves - 1) / (32 * kMassWaves);
  auto few = [&](auto stats, int64_t workgroups, int64_t most_parts) {
    constexpr bool kStats = decltype(stats)::value;
    int64_t parts = (workgroups + groups - 1) / groups;
    parts = parts < steps ? parts : steps;
    parts = parts < most_parts ? parts : most_parts;
    parts = parts < 1 ? 1 : parts;
    if (kStats) a.splits = (int)parts;
    const dim3 grid((unsigned)groups, (unsigned)parts);
    if (kStats || a.few_rows == 128) hipLaunchKernelGGL((k_mass_few<TK, TQ, 128, kStats>), grid, dim3(kMassThreads), 0, st, a, (int)parts);
    else hipLaunchKernelGGL((k_mass_few<TK, TQ, M::kF32 ? 128 : 256, false>), grid, dim3(kMassThreads), 0, st, a, (int)parts);
  };
  for (int t0 = 0; t0 == 0 || t0 < a.n_tokens; t0 = a.t1) {           // (also of no tokens: what is held decays)
    a.t0 = t0;
    a.t1 = a.n_tokens - t0 > most ? t0 + (int)most : a.n_tokens;
    const int n = a.t1 - t0, tiles = n / per + a.s.B;
    const int64_t rows = (int64_t)n * a.s.Hq, left = room - 2 * rows;
    a.stats = work;
    a.split_stats = a.sums = work + 2 * rows;                         // (the parts are joined before there are sums)
    const int64_t queries = (int64_t)n * a.s.G;
    const bool others = queries > a.few_rows;                         // (else no request has more)
    if (n > 0) {
      const int64_t by_room = left / 2 / rows < kMaxSplits ? left / 2 / rows : kMaxSplits;
      if (a.few_rows == 128) {
        few(std::true_type{}, 512, by_room);
      } else {
        const int64_t tile_groups = (int64_t)tiles * a.s.Hkv, by_len = (a.s.Lcap + 255) / 256;
        int64_t splits = (512 + tile_groups - 1) / tile_groups;
        if (splits > by_room) splits = by_room;
        if (splits > by_len) splits = by_len;
        a.splits = (int)(splits < 1 ? 1 : splits);
      }
      if (others || a.few_rows != 128) hipLaunchKernelGGL((k_mass_stats<TK, TQ>), dim3((unsigned)(tiles * a.s.Hkv * a.splits)), dim3(kMassThreads), 0, st, a, tiles);
      if (a.splits > 1)
        hipLaunchKernelGGL(k_mass_join, dim3((unsigned)((rows + 15) / 16)), dim3(256), 0, st, a.split_stats, a.stats, rows, a.splits);
    }
    // Of the query rows as many chunks as make work for the whole chip many times over: not all tiles are seen by all of them.  (The prompts above, for
    // 4096 / 6000 / 8192 / 12000 parts: 461 / 462 / 470 / 484 us.)
    const int64_t key_tiles = (a.s.Lcap + M::kRows - 1) / M::kRows, wanted = 6000;
    int64_t chunks = (wanted + key_tiles * a.s.B * a.s.Hkv - 1) / (key_tiles * a.s.B * a.s.Hkv);
    if (chunks > (queries + kMassChunk - 1) / kMassChunk) chunks = (queries + kMassChunk - 1) / kMassChunk;
    if (chunks * masses > left) chunks = left / masses;
    a.chunks = (int)(chunks < 1 ? 1 : chunks);
    if (a.few_rows > 0) few(std::false_type{}, a.few_rows == 128 && !M::kF32 ? 768 : 512, steps);
    if (others) hipLaunchKernelGGL((k_mass_add<TK, TQ>), dim3((unsigned)(a.s.B * a.s.Hkv), (unsigned)key_tiles, (unsigned)a.chunks), dim3(kMassThreads), 0, st, a);
    if (others && a.chunks > 1)
      hipLaunchKernelGGL((k_mass_sum<M::kRows, M::kStage, MassArgs<TQ>>), dim3((unsigned)((a.s.Lcap + 255) / 256), (unsigned)(a.s.B * a.s.Hkv)), dim3(256), 0, st, a);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess || a.n_tokens == 0) return e;
  }
  return hipSuccess;
}

hipError_t launch_attn_mass(const Shape& s, int dtype, const KvView& kv, const void* q, int64_t q_stride, const int32_t* cu, int n_tokens,
                            const int32_t* held, float decay, float* mass, float* part, int64_t part_rows, hipStream_t st) {
#define LFPS_MASS(TK, TQ)                                                                                                              \
  return mass_t<TK, TQ>(MassArgs<TQ>{s, kv, (const TQ*)q, q_stride, cu, held, n_tokens, 0, 0, decay, nullptr, nullptr, 1, 1, 0, nullptr, mass}, \
                        part, part_rows * kPartFloats, st)
  if (dtype == LFPS_F32) LFPS_MASS(float, float);
  if (dtype == LFPS_F16) LFPS_MASS(_Float16, _Float16);
  if (kv.k_fp8) LFPS_MASS(uint8_t, uint16_t);
  LFPS_MASS(uint16_t, uint16_t);
#undef LFPS_MASS
}

}  // namespace lfps
