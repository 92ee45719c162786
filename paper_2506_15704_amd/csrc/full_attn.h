// Full attention of single queries over the rows of a request, of a window of it, or of items of them: the kernels, and how what they leave is joined.
#pragma once
#include "prefix_groups.h"

#include <tuple>
#include <type_traits>

namespace lfps {

constexpr int kAttnThreads = 256;       // full attention

// Rows [begin, end) of request b and KV head g, and which part of all they make: a split of the request, or an item of its own rows.
__host__ __device__ __forceinline__ int rows_per_split(int n, int n_split) { return (((n + n_split - 1) / n_split) + 15) & ~15; }
struct RowsOf { int b, g, begin, end; int64_t part; int at, by; };      // (from row `at` on: the cache's row `by` further up)
// Further arguments of the kernels: what else than all rows of a request they take or leave.
struct WindowRows { int32_t window, n_sink; };        // the newest `window` rows of a request and its first n_sink
struct ScoresTo { float* score; int64_t stride; };    // all rows, whose scores go to score [B, Hq, stride] (no grouping: in powers of two)
// Waves a SIMD that the compiler has to leave room for.  Only windows of four heads over 16-bit rows need more registers than three leave, and spill 1 to 6
// of them outside the loop: shorter walks gain, longer ones lose.  us, three / as many registers as it takes: 32 requests, window 512 20.8 / 22.2, 4096
// 94.4 / 92.4, 64 requests 178 / 172, one, 4096 13.4 / 13.4.  With scores 6 to 43 would be spilled, up to ten of them in every turn of the loop: 16 requests of
// 2000 to 32768 rows, slabs 320 / 256, pages 279 / 265; 16 of 4096 rows, slabs 69.5 / 51.0, pages 57.7 / 56.2 (of 300 to 4096, pages 42.8 / 46.2).
template <typename... Own>
constexpr int attn_waves() { return (std::is_same<Own, WindowRows>::value || ...) ? 3 : 1; }
// The rows of a window in order: the first `at` of the cache, then those from `at + by` on, `count` in all.
__device__ __forceinline__ void window_rows(const WindowRows& w, int n, int* at, int* by, int* count) {
  const int lo = n > w.window ? n - w.window : 0;
  *at = w.n_sink < lo ? w.n_sink : lo;
  *by = lo - *at;
  *count = n - *by;
}
// The shape with the rows that a kernel takes of a request at most.
template <typename... Own>
__host__ __device__ __forceinline__ Shape walked(const Shape& s, const Own&...) { return s; }
__host__ __device__ __forceinline__ Shape walked(const Shape& s, const WindowRows& w) {
  const int64_t most = (int64_t)w.window + w.n_sink;
  Shape fewer = s;
  fewer.Lcap = most < s.Lcap ? (int)most : s.Lcap;
  return fewer;
}
__device__ __forceinline__ RowsOf rows_of_block(const Shape& s, const int32_t* seq_lens, int n_split) {
  const int bg = blockIdx.y, b = bg / s.Hkv, split = blockIdx.x;
  int n = seq_lens[b];
  n = n < 0 ? 0 : (n > s.Lcap ? s.Lcap : n);
  const int rps = rows_per_split(n, n_split), begin = split * rps;
  return {b, bg % s.Hkv, begin, (begin + rps < n) ? begin + rps : n, (int64_t)bg * n_split + split, 0, 0};
}
__device__ __forceinline__ RowsOf rows_of_block(const Shape& s, const int32_t* seq_lens, int n_split, const ScoresTo&) {
  return rows_of_block(s, seq_lens, n_split);
}
__device__ __forceinline__ RowsOf rows_of_block(const Shape& s, const int32_t* seq_lens, int n_split, const WindowRows& w) {
  const int bg = blockIdx.y, b = bg / s.Hkv, split = blockIdx.x;
  int at, by, n;
  window_rows(w, length_of(s, seq_lens, b), &at, &by, &n);
  const int rps = rows_per_split(n, n_split), begin = split * rps;
  return {b, bg % s.Hkv, begin, (begin + rps < n) ? begin + rps : n, (int64_t)bg * n_split + split, at, by};
}
__device__ __forceinline__ RowsOf rows_of_block(const Shape& s, const int32_t*, int, const OwnRows& own) {
  const int i = blockIdx.x, g = blockIdx.y;
  if (i >= own.item[s.B]) return {0, g, 0, 0, 0, 0, 0};
  const OwnItem at = own.items[i];
  return {at.b, g, at.begin, at.end, (int64_t)i * s.Hkv + g, 0, 0};
}

// x[u] = the elements at at(u), past the caches or not.  (A choice at run time between the two forms of one load is merged by the
// compiler, into the ordinary one: the kernels hold their loops twice.)
template <bool kOnce, typename Raw, int U, typename At>
__device__ __forceinline__ void load_rows(Raw (&x)[U], At at) {
#pragma unroll
  for (int u = 0; u < U; ++u) {
    if constexpr (kOnce) x[u].load_once(at(u));
    else x[u].load(at(u));
  }
}

// The weight of a partial result whose largest score lies x <= 0 from the largest of all.  Without grouping the scores are held as
// powers of two (k_full_attn_single).
template <int G>
__device__ __forceinline__ float part_weight(float x) { return G == 1 ? __builtin_amdgcn_exp2f(x) : exp_below<false>(x); }

// The four waves of a workgroup (a wave without rows: m = -inf, weight 0) -> po [G, D+2]: acc[D], m, l.  All threads call, after a
// barrier.
template <int G>
__device__ __forceinline__ void merge_waves(const float (&red_acc)[4][G][kD], const float (&red_m)[4][G],
                                            const float (&red_l)[4][G], float* __restrict__ po) {
  for (int e = threadIdx.x; e < G * kD; e += kAttnThreads) {
    const int h = e / kD, c = e % kD;
    const float mx = fmaxf(fmaxf(red_m[0][h], red_m[1][h]), fmaxf(red_m[2][h], red_m[3][h]));
    float a = 0.f, ls = 0.f;
#pragma unroll
    for (int w = 0; w < 4; ++w) {
      const float f = (red_m[w][h] == -INFINITY) ? 0.f : part_weight<G>(red_m[w][h] - mx);
      a = fmaf(red_acc[w][h][c], f, a);
      ls = fmaf(red_l[w][h], f, ls);
    }
    po[h * (kD + 2) + c] = a;
    if (c == 0) {
      po[h * (kD + 2) + kD] = mx;
      po[h * (kD + 2) + kD + 1] = ls;
    }
  }
}

// The sums over the 16 lanes of a row of lanes of a[0 .. G-1], G = 2 or 4: lane j receives that of a[j % G].  (A butterfly
// over lane distances 1, 2, 4, 8 in which the first log2 G steps also share the G sums out: 11 instructions instead of 16.)
template <int G>
__device__ __forceinline__ float row16_shared_sums(float (&a)[G], int j) {
#define LFPS_DPP(v, ctrl) __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), ctrl, 0xf, 0xf, false))
  const bool odd = j & 1;
  float x, y[G / 2];
#pragma unroll
  for (int h = 0; h < G / 2; ++h) {
    const float keep = odd ? a[2 * h + 1] : a[2 * h], give = odd ? a[2 * h] : a[2 * h + 1];
    y[h] = keep + LFPS_DPP(give, 0xB1);                      // quad_perm 1 0 3 2
  }
  if constexpr (G == 2) {
    x = y[0];
    x += LFPS_DPP(x, 0x4E);                                  // quad_perm 2 3 0 1
  } else {
    const bool upper = j & 2;
    const float keep = upper ? y[1] : y[0], give = upper ? y[0] : y[1];
    x = keep + LFPS_DPP(give, 0x4E);
  }
  // (lanes j and j ^ 4, then j ^ 8, by rotation: every lane of a quad holds another sum)
  x += row16_rotate<4>(x);                                   // with the next one, the pairs' sums agree
  x += row16_rotate<8>(x);
  return x;
#undef LFPS_DPP
}

// G = 2 or 4.  grid (n_split, B*Hkv); part [B*Hkv, n_split, G, D+2]: acc[D], m, l
//
// A wave takes U groups of four rows at a time, 16 lanes a row, 8 channels a lane, for K and for V.  The G sums of a row are
// shared out over its lanes, so that a lane makes the softmax step for one head and its own rows only, once per tile; the
// weights reach the lanes that hold the values through LDS.  The rows of K and of V are in flight in turn, those of one while
// the other is used.  Bound by the bytes of K and V in 16 bits (64 groups x 32K rows, 1.07 GB: 168.5 us with the merge, 199 with an
// earlier form), by the multiply-adds in FP8 (the same rows: 112 us, 233): when every lane made the step for all heads and each of
// its rows, a row cost the same whatever it took to fetch.  U = 16 for FP8 leaves two waves per SIMD: 13 us slower.
// Rows of a contiguous cache are counted, not looked up across lanes, which made every load wait for LDS: bf16 172.5 -> 168.5 us, FP8
// 114 -> 112, 8 x 16384 in FP8 57.2 -> 56.9, 16 x 8480 60.0 -> 59.3.
// (The dot products on the matrix units were as fast, 169 to 180 us, but 1.3 times as far from 64 bits where a few rows carry
// the weight: large scores are sums of like-signed products there.)
// kMayOnce: rows past the caches where the rows that the requests hold outgrow the memory-side cache (kKeptStreamBytes; 8 x 32K rows 195 against
// 207 us with the kernel as it was); fewer are found there by the next call, whatever the context has room for (8 x 8192 of
// 131072 rows in bf16 52.9 -> 48.8 us, 8 x 16384 in FP8 62.3 -> 57.3, against that capacity deciding).
template <typename TK, typename T, int G, bool kPaged, bool kMayOnce, typename... Own>
__global__ __launch_bounds__(kAttnThreads, attn_waves<Own...>()) void k_full_attn(Shape s, const float* __restrict__ q,
                                                            const TK* __restrict__ K, const T* __restrict__ V,
                                                            int64_t stride_b, int64_t stride_h, int64_t stride_n,
                                                            KvPage pg, const int32_t* __restrict__ seq_lens,
                                                            float* __restrict__ part, int n_split, float scale, Own... own) {
  // (items are short, and more of their workgroups fit with the half of rows in flight: 32 requests in FP8 75.9 -> 72.5 us, bf16 the same)
  constexpr bool kItems = (std::is_same<Own, OwnRows>::value || ...), kGap = (std::is_same<Own, WindowRows>::value || ...);
  constexpr bool kScores = (std::is_same<Own, ScoresTo>::value || ...);
  constexpr int U = kItems || sizeof(TK) == 4 ? 4 : 8, kRows = 4 * U;
  constexpr int kShare = 16 / G;                            // lanes of a row that hold the same head's sum
  constexpr int NV = U > kShare ? U / kShare : 1;           // (row, head) pairs of a lane
  __shared__ float red_acc[4][G][kD];
  __shared__ float weight[4][kRows][G];
  __shared__ float red_m[4][G], red_l[4][G];
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int j = lane & 15, rs = lane >> 4;
  const RowsOf here = rows_of_block(s, seq_lens, n_split, own...);
  const int b = here.b, g = here.g, r_begin = here.begin, r_end = here.end;
  if (r_begin >= r_end) return;
  const bool once_here = kMayOnce && outgrow_cache(s, held_rows(walked(s, own...), seq_lens), kD * (int)(sizeof(TK) + sizeof(T)), kKeptStreamBytes);

  float qr[G][8];
#pragma unroll
  for (int h = 0; h < G; ++h) {
    const float* qh = q + ((int64_t)b * s.Hq + (int64_t)g * G + h) * kD + 8 * j;
#pragma unroll
    for (int c = 0; c < 8; ++c) qr[h][c] = qh[c] * scale;
  }
  using Rows = RowMap<kPaged>;
  const TK* Kbg = K + Rows::base(b, g, stride_b, stride_h) + 8 * j;
  const T* Vbg = V + Rows::base(b, g, stride_b, stride_h) + 8 * j;
  // Rows past the end are read from the last row and weigh nothing, so no load sits behind a branch.
  auto clamped = [&](int r) {
    const int x = r < r_end ? r : r_end - 1;
    return kGap && x >= here.at ? x + here.by : x;
  };
  // the tile at r0: paged, its row r0 + lane as a physical row; else its first row
  auto rows_of = [&](int r0) { return kPaged ? Rows::phys(pg, b, clamped(r0 + lane)) : r0; };
  auto row_value = [&](int x, int u) {                      // of row 4 u + rs
    return kPaged ? __builtin_amdgcn_ds_bpermute(4 * rs + 16 * u, x) : clamped(x + 4 * u + rs);
  };
  Raw8<TK> kt[U];                                           // kt[u], vt[u]: my channels of row 4 u + rs
  Raw8<T> vt[U];
  auto fetch_k = [&](auto once, int phys) {
    load_rows<decltype(once)::value>(kt, [&](int u) { return Kbg + Rows::offset(pg, row_value(phys, u), stride_b, stride_n); });
  };
  auto fetch_v = [&](auto once, int phys) {
    load_rows<decltype(once)::value>(vt, [&](int u) { return Vbg + Rows::offset(pg, row_value(phys, u), stride_b, stride_n); });
  };
  // my pairs: head j % G and the rows 4 u + rs with u = t * kShare + j / G
  const int my_u = j / G;
  const bool mine = my_u < U;
  float m = -INFINITY, l = 0.f;                             // of head j % G: largest score so far; the sum over my rows
  float acc[G][8];
#pragma unroll
  for (int h = 0; h < G; ++h)
#pragma unroll
    for (int c = 0; c < 8; ++c) acc[h][c] = 0.f;

  float* to_scores = nullptr;                               // of the group; with head j % G's offset
  uint32_t my_scores = 0;
  if constexpr (kScores) {
    const ScoresTo& to = std::get<0>(std::tie(own...));
    to_scores = to.score + ((int64_t)b * s.Hq + g * G) * to.stride;
    my_scores = (uint32_t)(j % G) * (uint32_t)to.stride;
  }
  constexpr int kStep = 4 * kRows;                          // wave w takes tiles w, w + 4, ...
  auto walk = [&](auto once) {
  int r0 = r_begin + kRows * wave;
  int phys = rows_of(r0), phys_next = rows_of(r0 + kStep);
  fetch_k(once, phys);
  fetch_v(once, phys);
  for (; r0 < r_end; r0 += kStep) {
    float v[NV];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      float x[8], a[G];
      kt[u].get(x);
#pragma unroll
      for (int h = 0; h < G; ++h) {
        a[h] = qr[h][0] * x[0];
#pragma unroll
        for (int c = 1; c < 8; ++c) a[h] = fmaf(qr[h][c], x[c], a[h]);
      }
      const float sum = row16_shared_sums<G>(a, j);
      v[u / kShare] = u % kShare == 0 || my_u == u % kShare ? sum : v[u / kShare];
      if (u % 2) __builtin_amdgcn_sched_barrier(0);         // (registers: two rows' elements at a time as fp32)
    }
    phys = phys_next;
    phys_next = rows_of(r0 + 2 * kStep);
    if constexpr (kPaged) __builtin_amdgcn_sched_barrier(0);      // the look-up before the rows: its wait must not include them
    fetch_k(once, phys);
    if constexpr (kScores) {
#pragma unroll
      for (int t = 0; t < NV; ++t) {
        const int r = r0 + 4 * (t * kShare + my_u) + rs;
        if (mine && r < r_end) to_scores[my_scores + (uint32_t)r] = v[t];
      }
    }
    if constexpr (kGap || kScores) {
      if (r0 + kRows > r_end) {                               // (a row that is not there weighs 0, which an infinity in its place would not let be)
#pragma unroll
        for (int u = 0; u < U; ++u)
          if (r0 + 4 * u + rs >= r_end) vt[u] = Raw8<T>{};
      }
    }
    // one online-softmax step
    bool ok[NV];
    float mx = m;
#pragma unroll
    for (int t = 0; t < NV; ++t) {
      ok[t] = mine && r0 + 4 * (t * kShare + my_u) + rs < r_end;
      mx = ok[t] ? fmaxf(mx, v[t]) : mx;
    }
    mx = fmaxf(mx, row16_rotate<8>(mx));
    mx = fmaxf(mx, row16_rotate<4>(mx));
    if constexpr (G == 2) mx = fmaxf(mx, row16_rotate<2>(mx));
    mx = fmaxf(mx, __shfl_xor(mx, 16));
    mx = fmaxf(mx, __shfl_xor(mx, 32));
    const float alpha = mx == -INFINITY ? 1.f : exp_below<false>(m - mx);      // (0 on the first tile)
    l *= alpha;
    m = mx;
    wave_lds_order();                                                // (the weights of the tile before have been read)
#pragma unroll
    for (int t = 0; t < NV; ++t) {
      const float e = exp_below<false>(v[t] - mx);
      const float p = ok[t] && v[t] != -INFINITY ? e : 0.f;
      l += p;
      if (mine) weight[wave][4 * (t * kShare + my_u) + rs][j % G] = p;
    }
    wave_lds_order();
    if (__ballot(alpha != 1.f)) {
#pragma unroll
      for (int h = 0; h < G; ++h) {
        const float a = __int_as_float(__builtin_amdgcn_readlane(__float_as_int(alpha), h));
#pragma unroll
        for (int c = 0; c < 8; ++c) acc[h][c] *= a;
      }
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      float x[8], p[G];
      vt[u].get(x);
#pragma unroll
      for (int h = 0; h < G; ++h) p[h] = weight[wave][4 * u + rs][h];
#pragma unroll
      for (int h = 0; h < G; ++h)
#pragma unroll
        for (int c = 0; c < 8; ++c) acc[h][c] = fmaf(p[h], x[c], acc[h][c]);
      if (u % 2) __builtin_amdgcn_sched_barrier(0);
    }
    fetch_v(once, phys);
  }
  };
  if (once_here) walk(std::true_type{});
  else walk(std::false_type{});

  // the lanes of the wave, then the four waves (a wave without rows: m = -inf, weight 0)
#pragma unroll
  for (int d = G; d < 64; d <<= 1) l += __shfl_xor(l, d);
#pragma unroll
  for (int h = 0; h < G; ++h)
#pragma unroll
    for (int c = 0; c < 8; ++c) {
      acc[h][c] += __shfl_xor(acc[h][c], 16);
      acc[h][c] += __shfl_xor(acc[h][c], 32);
    }
  if (rs == 0) {
#pragma unroll
    for (int h = 0; h < G; ++h)
#pragma unroll
      for (int c = 0; c < 8; ++c) red_acc[wave][h][8 * j + c] = acc[h][c];
    if (j < G) {
      red_m[wave][j] = m;
      red_l[wave][j] = l;
    }
  }
  __syncthreads();
  merge_waves<G>(red_acc, red_m, red_l, part + here.part * G * (kD + 2));
}

// The same without grouping (G = 1), where nothing is to be shared out: the four rows that a wave instruction covers keep a state
// of their own (largest score, sum, values) until the end, so a tile needs no step across its rows.  A wave takes 16 rows at a
// time, two tiles in flight.  Every lane of a row makes its exponentials: scores are kept in units of ln 2 (the query is multiplied
// by log2(e) / sqrt(D), rounded once), so that an exponential needs no product whose rounding would have to be corrected.  In
// k_full_attn's form the few tiles of a short row waited longer for each other: 1 x 8192 rows of 8 heads in bf16 10.9 -> 9.85 us,
// in FP8 10.6 -> 9.7, 1 x 16384 in fp32 29.4 -> 28.6, 1 x 32768 in FP8 21.2 -> 19.7; 32 x 30000 in bf16 571 -> 567.
// Paged, one look-up serves both tiles: with one each, its wait came twice as often and the compiler kept fewer loads in flight (FP8
// 16 x 32768 169.2 -> 166.5 us, bf16 325.9 -> 323.2, 1 x 8192 11.7 -> 11.3).
template <typename TK, typename T, bool kPaged, bool kMayOnce, typename... Own>
__global__ __launch_bounds__(kAttnThreads) void k_full_attn_single(Shape s, const float* __restrict__ q,
                                                                   const TK* __restrict__ K, const T* __restrict__ V,
                                                                   int64_t stride_b, int64_t stride_h, int64_t stride_n,
                                                                   KvPage pg, const int32_t* __restrict__ seq_lens,
                                                                   float* __restrict__ part, int n_split, float, Own... own) {
  constexpr double kLog2Scale = 0.08838834764831845 * 1.4426950408889634;
  constexpr float kHi = (float)kLog2Scale, kLo = (float)(kLog2Scale - (double)kHi);
  constexpr bool kGap = (std::is_same<Own, WindowRows>::value || ...), kScores = (std::is_same<Own, ScoresTo>::value || ...);
  constexpr int U = 4, kRows = 4 * U;
  __shared__ float red_acc[4][1][kD];
  __shared__ float red_m[4][1], red_l[4][1];
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int j = lane & 15, rs = lane >> 4;
  const RowsOf here = rows_of_block(s, seq_lens, n_split, own...);
  const int b = here.b, g = here.g, r_begin = here.begin, r_end = here.end;
  if (r_begin >= r_end) return;
  const bool once_here = kMayOnce && outgrow_cache(s, held_rows(walked(s, own...), seq_lens), kD * (int)(sizeof(TK) + sizeof(T)), kKeptStreamBytes);

  float qr[8];
#pragma unroll
  for (int c = 0; c < 8; ++c) {
    const float x = q[((int64_t)b * s.Hkv + g) * kD + 8 * j + c];
    qr[c] = fmaf(x, kHi, x * kLo);
  }
  using Rows = RowMap<kPaged>;
  const TK* Kbg = K + Rows::base(b, g, stride_b, stride_h) + 8 * j;
  const T* Vbg = V + Rows::base(b, g, stride_b, stride_h) + 8 * j;

  // Rows past the end are read from the last row and weigh nothing, so no load sits behind a branch.
  struct Tile {
    Raw8<TK> k[U];                                          // my channels of row 4 u + rs
    Raw8<T> v[U];
  };
  auto clamped = [&](int r) {
    const int x = r < r_end ? r : r_end - 1;
    return kGap && x >= here.at ? x + here.by : x;
  };
  float* to_scores = nullptr;
  if constexpr (kScores) {
    const ScoresTo& to = std::get<0>(std::tie(own...));
    to_scores = to.score + ((int64_t)b * s.Hkv + g) * to.stride;
  }
  constexpr int kStep = 4 * kRows;                          // wave w takes tiles w, w + 4, ...
  // paged: the rows of the tiles at r0 and r0 + kStep as physical rows, in lanes 0-15 and 16-31
  auto rows_of = [&](int r0) { return kPaged ? Rows::phys(pg, b, clamped(r0 + j + (rs & 1) * kStep)) : 0; };
  auto issue = [&](auto once, Tile& t, int r0, int phys, int first_lane) {
    int64_t off[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int p = kPaged ? __builtin_amdgcn_ds_bpermute(4 * rs + 16 * u + 4 * first_lane, phys) : clamped(r0 + 4 * u + rs);
      off[u] = Rows::offset(pg, p, stride_b, stride_n);
    }
    load_rows<decltype(once)::value>(t.k, [&](int u) { return Kbg + off[u]; });
    load_rows<decltype(once)::value>(t.v, [&](int u) { return Vbg + off[u]; });
    __builtin_amdgcn_sched_barrier(0);                      // (moved down to their uses, the loads of one tile would wait for the other's)
  };
  float m = -INFINITY, l = 0.f, acc[8];                     // of the rows rs mod 4
#pragma unroll
  for (int c = 0; c < 8; ++c) acc[c] = 0.f;
  auto consume = [&](const Tile& t, int r0) {
    float sc[U], p[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      float x[8];
      t.k[u].get(x);
      float a = qr[0] * x[0];
#pragma unroll
      for (int c = 1; c < 8; ++c) a = fmaf(qr[c], x[c], a);
      sc[u] = row16_butterfly_sum(a);
    }
    if constexpr (kScores) {                                // (all lanes of a row hold its score: lane u of them stores that of the u-th row)
      const float mine = j == 0 ? sc[0] : (j == 1 ? sc[1] : (j == 2 ? sc[2] : sc[3]));
      if (j < U && r0 + 4 * j + rs < r_end) to_scores[r0 + 4 * j + rs] = mine;
    }
    float mx = m;
#pragma unroll
    for (int u = 0; u < U; ++u) mx = r0 + 4 * u + rs < r_end ? fmaxf(mx, sc[u]) : mx;
    const float from = mx == -INFINITY ? 0.f : mx;          // (no row yet, or only scores of -inf: they weigh 0)
    const float alpha = __builtin_amdgcn_exp2f(m - from);   // (0 on the first tile)
    l *= alpha;
    m = mx;
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const float e = __builtin_amdgcn_exp2f(sc[u] - from);
      p[u] = r0 + 4 * u + rs < r_end ? e : 0.f;
      l += p[u];
    }
#pragma unroll
    for (int c = 0; c < 8; ++c) acc[c] *= alpha;
#pragma unroll
    for (int u = 0; u < U; ++u) {
      float x[8];
      t.v[u].get(x);
      if constexpr (kGap || kScores) {
        if (r0 + kRows > r_end) {                           // (as above)
#pragma unroll
          for (int c = 0; c < 8; ++c) x[c] = r0 + 4 * u + rs < r_end ? x[c] : 0.f;
        }
      }
#pragma unroll
      for (int c = 0; c < 8; ++c) acc[c] = fmaf(p[u], x[c], acc[c]);
    }
  };

  auto walk = [&](auto once) {
  Tile ta, tb;
  int r0 = r_begin + kRows * wave;
  int phys = rows_of(r0);
  issue(once, ta, r0, phys, 0);
  for (; r0 < r_end; r0 += 2 * kStep) {
    const int phys_next = rows_of(r0 + 2 * kStep);
    if constexpr (kPaged) __builtin_amdgcn_sched_barrier(0);      // the look-up before the rows: its wait must not include them
    issue(once, tb, r0 + kStep, phys, 16);
    consume(ta, r0);
    issue(once, ta, r0 + 2 * kStep, phys_next, 0);
    consume(tb, r0 + kStep);
    phys = phys_next;
  }
  };
  if (once_here) walk(std::true_type{});
  else walk(std::false_type{});

  // the four lane groups of the wave (one without rows: m = -inf, weight 0), then the four waves
  float mx = fmaxf(m, __shfl_xor(m, 16));
  mx = fmaxf(mx, __shfl_xor(mx, 32));
  const float f = m == -INFINITY ? 0.f : part_weight<1>(m - mx);
  l *= f;
  l += __shfl_xor(l, 16);
  l += __shfl_xor(l, 32);
#pragma unroll
  for (int c = 0; c < 8; ++c) {
    acc[c] *= f;
    acc[c] += __shfl_xor(acc[c], 16);
    acc[c] += __shfl_xor(acc[c], 32);
  }
  if (rs == 0) {
#pragma unroll
    for (int c = 0; c < 8; ++c) red_acc[wave][0][8 * j + c] = acc[c];
    if (j == 0) {
      red_m[wave][0] = mx;
      red_l[wave][0] = l;
    }
  }
  __syncthreads();
  merge_waves<1>(red_acc, red_m, red_l, part + here.part * (kD + 2));
}

// The parts of a row: of part i (of n <= 64) the largest score and the sum of the weights from there, in lane i of a wave (others: -inf, 0).
// Leaves the largest score of all (0: nothing was seen), the inverse of the sum (0 then), and the part's own weight.  Scores as the kernels leave
// them: without grouping in powers of two.
template <int G>
__device__ __forceinline__ void weigh_parts(float m, float l, float* from, float* inverse, float* weight) {
  float mx = m;
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) mx = fmaxf(mx, __shfl_xor(mx, d));
  const float w = m == -INFINITY ? 0.f : part_weight<G>(m - mx);
  float sum = l != l ? l : w * l;              // (all scores of a part NaN: its largest is -inf)
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) sum += __shfl_xor(sum, d);
  *from = mx == -INFINITY ? 0.f : mx;
  *inverse = sum == 0.f ? 0.f : 1.f / sum;
  *weight = l != l ? l : w;
}

// The output row of head hg of a group from its n parts at part (a wave; two channels a lane).
template <int G>
__device__ __forceinline__ f32x2t join_head(const float* part, int n, int hg, float* from, float* inverse) {
  const int lane = threadIdx.x & 63;
  const int64_t step = (int64_t)G * (kD + 2);
  const float* const p = part + hg * (kD + 2);
  const float m = lane < n ? p[lane * step + kD] : -INFINITY, l = lane < n ? p[lane * step + kD + 1] : 0.f;
  float w;
  weigh_parts<G>(m, l, from, inverse, &w);
  f32x2t a = {0.f, 0.f};
  constexpr int kU = 8;
  for (int i0 = 0; i0 < n; i0 += kU) {
    f32x2t x[kU];
#pragma unroll
    for (int u = 0; u < kU; ++u) x[u] = *reinterpret_cast<const f32x2t*>(p + (i0 + u < n ? i0 + u : n - 1) * step + 2 * lane);
#pragma unroll
    for (int u = 0; u < kU; ++u) {
      const float wu = i0 + u < n ? __int_as_float(__builtin_amdgcn_readlane(__float_as_int(w), (i0 + u) & 63)) : 0.f;
      if (i0 + u < n) {
        a[0] = fmaf(x[u][0], wu, a[0]);
        a[1] = fmaf(x[u][1], wu, a[1]);
      }
    }
  }
  return f32x2t{a[0] * *inverse, a[1] * *inverse};
}

}  // namespace lfps
