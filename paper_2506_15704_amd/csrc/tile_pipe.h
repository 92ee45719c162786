// The body of the prompt kernel, and of large groups of a shared prefix, for 16-bit operands (bf16, fp16; FP8 rows as bf16 in prompts, as
// fp16 in prefixes): tile_attn.h's products, made for the matrix units' rate.
//
// Steps, over 16384 tokens of 32 heads in bf16: rows through registers, 128 query rows a workgroup, 5.09 ms; straight into LDS, a maximum that
// is followed lazily 2.17; 256 query rows, places without bank conflicts, scores of the next stage beside the weights of this one
// 1.94; the two waves of a SIMD half a stage apart, requests between the products 1.89.  A stage of 64 keys takes 3100 to 3250 cycles of
// which 2048 are the matrix unit's; the clock falls to 1.75 to 2.0 GHz meanwhile, and cards differ by 3% in it.
#pragma once
#include "tile_attn.h"

namespace lfps {

constexpr int kPipeWaves = 8, kPipeKeys = 64, kPipeRows = 32 * kPipeWaves;       // of a workgroup; keys of a stage; query rows
constexpr int kPipeThreads = 64 * kPipeWaves, kFeedRows = kPipeKeys / kPipeWaves;   // rows of a stage that a wave brings
constexpr float kLazy = 6.f;                         // growth of a maximum, in powers of two, that is let pass

typedef const __attribute__((address_space(1))) char global_char;

// How the rows of a cache lie: a slab; pages of eight rows and more; anything (smaller pages, rows very far apart).  In the first two
// the rows that a wave brings of a stage lie at offsets of 32 bits from the first, whose place is then the wave's.
enum { kSlab = 0, kPages = 1, kAnyRows = 2 };
__host__ inline int rows_kind(const KvView& kv) {
  if (kv.stride_n >= (1 << 20) || (kv.page.table && (1 << kv.page.shift) < kFeedRows)) return kAnyRows;
  return kv.page.table ? kPages : kSlab;
}

// The rows of a stage that a wave brings, eight, of K or V.  16-bit elements go from memory to LDS without
// registers, four rows an instruction: lane l fills place l % 16 of row l / 16, so it asks for the chunk that belongs there.
// Rows from `end` on are the last one again, also whole stages of them: they are read by nobody's weights but 0.
// aim works out where a stage's rows lie, ask asks for them: the one is scalar work for when there is time, the other a few instructions.
template <typename T, int kKind, typename Op>
struct Feed {
  static constexpr bool kDirect = sizeof(T) == 2;
  static constexpr int kLoads = kFeedRows / (kDirect ? 4 : 8);     // FP8: eight rows a load, through registers
  u32x4 x[kDirect ? 1 : kLoads];
  const char* base;                                  // the wave's first row
  uint32_t off[kLoads];                              // my pieces from there
  const char* from[kKind == kAnyRows ? kLoads : 1];  // kAnyRows: my pieces

  __device__ __forceinline__ static int row(int i, int lane) { return kFeedRows / kLoads * i + (kDirect ? lane >> 4 : lane >> 3); }
  __device__ __forceinline__ static int piece(int i, int lane) {                  // of a row of the cache, in bytes
    return kDirect ? 16 * ((lane & 15) ^ mix(kFeedRows * wave_of() + row(i, lane))) : 16 * (lane & 7);
  }
  // entry: of the block table, for the wave's first row (first_row; kAnyRows looks its own up)
  __device__ __forceinline__ void aim(const CacheRows<T>& c, int w0, int end, int entry, int lane) {
    const int last = end - 1 - w0;
    if constexpr (kKind == kAnyRows) {
#pragma unroll
      for (int i = 0; i < kLoads; ++i) {
        const int r = w0 + min(row(i, lane), last);
        from[i] = reinterpret_cast<const char*>(c.at(r, c.entry(r))) + piece(i, lane);
      }
    } else {
      const int64_t first = kKind == kPages ? RowMap<true>::offset_in(c.pg, entry, w0, c.stride_b, c.stride_n) : w0 * c.stride_n;
      base = reinterpret_cast<const char*>(c.base + first);
#pragma unroll
      for (int i = 0; i < kLoads; ++i)
        off[i] = __umul24((uint32_t)min(row(i, lane), last), (uint32_t)c.stride_n * (uint32_t)sizeof(T)) + (uint32_t)piece(i, lane);
    }
  }
  __device__ __forceinline__ void ask(lds_char* stage, int wave) {
#pragma unroll
    for (int i = 0; i < kLoads; ++i) {
      const char* p = kKind == kAnyRows ? from[i] : base + off[i];
      if constexpr (kDirect)
        __builtin_amdgcn_global_load_lds((global_char*)p, (__attribute__((address_space(3))) void*)(stage + (kFeedRows * wave + 4 * i) * 256), 16, 0, 0);
      else
        x[i] = *reinterpret_cast<const u32x4*>(p);
    }
  }
  // FP8: what has arrived becomes Op's type in the stage
  __device__ __forceinline__ void put(lds_char* stage, int lane, int wave) const {
    if constexpr (!kDirect) {
#pragma unroll
      for (int i = 0; i < kLoads; ++i) {
        const int r = kFeedRows * wave + row(i, lane), c = lane & 7;
        typedef __attribute__((address_space(3))) Op* Lds;
        *(Lds)(stage + r * 256 + 16 * chunk_place(r, 2 * c)) = fp8x8_to<Op>(x[i][0], x[i][1]);
        *(Lds)(stage + r * 256 + 16 * chunk_place(r, 2 * c + 1)) = fp8x8_to<Op>(x[i][2], x[i][3]);
      }
    }
  }
};
// The first row that a wave brings of a stage, given where it would be: one that exists.
__device__ __forceinline__ int first_row(int w0, int end) {
  return __builtin_amdgcn_readfirstlane(w0 < end ? w0 : (end - 1) & ~(kFeedRows - 1));
}

// 32 query rows of a wave.  kTerms: 16-bit terms of the query and of the weights (see RowState).  The third one of a query in bf16 terms
// is in LDS (kRest), for want of registers: its products come last of a chunk's.  Two terms of the weights leave 2^-18 of each, which
// is 1e-6 of the output, as much as fp32 sums of a few thousand products have; a third costs an eighth of the time (64 requests over
// 32768 shared rows).
template <typename Op, int kTerms = 1>
struct PipeState {
  static constexpr bool kRest = query_terms<Op, kTerms>() > kTerms;
  static constexpr float kLift = std::is_same<Op, f16x8>::value ? 8.f : 0.f;       // (as there; times 2^kLazy it still is an fp16 number)
  f32x16 o[4];
  float m, l[4];                             // four sums, so that none waits for the one before
  QueryTile<Op, kTerms> q;
  int limit;

  __device__ __forceinline__ void clear() {
    m = -INFINITY;
#pragma unroll
    for (int i = 0; i < 4; ++i) l[i] = 0.f;
#pragma unroll
    for (int d = 0; d < 4; ++d)
#pragma unroll
      for (int r = 0; r < 16; ++r) o[d][r] = 0.f;
  }

  // Operands of the scores' products 4 g .. + 3 of a stage: channel chunks 2 g and 2 g + 1 for either 32 keys.
  __device__ __forceinline__ static void load_keys(Op (&a)[4], const lds_char* k, int g, int n, int h) {
#pragma unroll
    for (int i = 0; i < 4; ++i)
      a[i] = *(const __attribute__((address_space(3))) Op*)(k + (32 * (i & 1) + n) * 256 + 16 * chunk_place(n, 2 * (2 * g + (i >> 1)) + h));
  }
  __device__ __forceinline__ void add_scores(f32x16 (&s)[2], const Op (&a)[4], int g, const lds_char* rest) const {
    Op x[2];
    if constexpr (kRest) {
#pragma unroll
      for (int i = 0; i < 2; ++i) x[i] = *(const __attribute__((address_space(3))) Op*)(rest + 1024 * (2 * g + i) + 16 * (threadIdx.x & 63));
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int c = 2 * g + (i >> 1);
#pragma unroll
      for (int t = kTerms - 1; t >= 0; --t)
        s[i & 1] = mfma32(a[i], q.x[t][c], c == 0 && t == kTerms - 1 ? zeros16() : s[i & 1]);
    }
    if constexpr (kRest) {
#pragma unroll
      for (int i = 0; i < 4; ++i) s[i & 1] = mfma32(a[i], x[i >> 1], s[i & 1]);
    }
  }
  // Operands of the values' products of 16 keys, step t.
  __device__ __forceinline__ static void load_values(Op (&a)[4], const lds_char* v, int t, int lane) {
    const int h = lane >> 5, i = lane & 15, key = 4 * h + (i >> 2);
    typedef __attribute__((address_space(3))) s16x4* Lds;
#pragma unroll
    for (int d = 0; d < 4; ++d) {
      const int chunk = 4 * d + 2 * ((lane >> 4) & 1) + ((i & 3) >> 1);
      union {
        s16x4 half[2];
        Op op;
      } x;
      x.half[0] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((Lds)(v + key * 256 + 16 * chunk_place(key, chunk) + 8 * (i & 1) + t * (16 * 256)));
      x.half[1] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((Lds)(v + (key + 8) * 256 + 16 * chunk_place(key + 8, chunk) + 8 * (i & 1) + t * (16 * 256)));
      a[d] = x.op;
    }
  }
  // w: weights of step t as weights() left them, rounded (one term) or, of two, whole in s.
  __device__ __forceinline__ void add_values(const Op (&a)[4], const Op& w, const f32x16 (&s)[2], int t) {
    if constexpr (kTerms == 1) {
#pragma unroll
      for (int d = 0; d < 4; ++d) o[d] = mfma32(a[d], w, o[d]);
    } else {
      Op x[kTerms];
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        typedef typename std::conditional<std::is_same<Op, bf16x8>::value, __bf16, _Float16>::type Elem;
        float p = s[t / 2][8 * (t % 2) + i];
#pragma unroll
        for (int u = 0; u < kTerms; ++u) {
          x[u][i] = (Elem)p;
          p -= (float)x[u][i];
        }
      }
#pragma unroll
      for (int u = kTerms - 1; u >= 0; --u)
#pragma unroll
        for (int d = 0; d < 4; ++d) o[d] = mfma32(a[d], x[u], o[d]);
    }
  }

  // The values of a stage key by key, of those that the row sees (see any_not_finite).
  template <typename Sees>
  __device__ __forceinline__ void add_values_apart(const Op (&w)[4], const f32x16 (&s)[2], const lds_char* v, int lane, Sees sees) {
    auto weight = [&](int i) {                                   // of the 32 that I hold
      float x = 0.f;
#pragma unroll
      for (int e = 0; e < 32; ++e) x = e == i ? (kTerms == 1 ? (float)w[e / 8][e % 8] : s[e / 16][e % 16]) : x;
      return x;
    };
    add_apart<Op>(o, weight, v, kPipeKeys, sees, lane);
  }

  // Scores of keys that the row does not see: behind its limit, and in its gap.  (One after the other: both conditions in one choice go by way of the
  // scalar unit.)
  template <typename Rows>
  __device__ __forceinline__ void hide(f32x16 (&s)[2], int first, int h, const Rows& rows) const {
    auto keep = [&](auto sees) __attribute__((always_inline)) {
#pragma unroll
      for (int b = 0; b < 2; ++b)
#pragma unroll
        for (int r = 0; r < 16; ++r) s[b][r] = sees(32 * b + 8 * (r / 4) + r % 4) ? s[b][r] : -INFINITY;
    };
    keep(AllRows().seen_from(first + 4 * h, limit));
    if constexpr (Rows::kGap) keep(rows.past_gap_from(first + 4 * h));
  }
  __device__ __forceinline__ static float largest(const f32x16 (&s)[2]) {
    float mx[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) mx[i] = fmaxf(s[i / 2][8 * (i % 2)], s[i / 2][8 * (i % 2) + 1]);
#pragma unroll
    for (int r = 2; r < 8; r += 2)
#pragma unroll
      for (int i = 0; i < 4; ++i) mx[i] = fmaxf(fmaxf(mx[i], s[i / 2][8 * (i % 2) + r]), s[i / 2][8 * (i % 2) + r + 1]);
    return fmaxf(fmaxf(mx[0], mx[1]), fmaxf(mx[2], mx[3]));
  }
  // mx: the largest of my scores of a stage.  Follows the row's maximum, and brings the sums so far in line with it.
  __device__ __forceinline__ void follow(float mx) {
    const auto both = __builtin_amdgcn_permlane32_swap(__float_as_int(mx), __float_as_int(mx), false, false);
    mx = fmaxf(__int_as_float(both[0]), __int_as_float(both[1])) * q.unit;
    const float before = m;
    const float now = mx > before + kLazy ? mx : before;              // (from -inf on the first keys)
    if (__ballot(now != before)) {
      const float shrink = now == before ? 1.f : __builtin_amdgcn_exp2f(before - now);
      m = now;
#pragma unroll
      for (int i = 0; i < 4; ++i) l[i] *= shrink;
#pragma unroll
      for (int d = 0; d < 4; ++d)
#pragma unroll
        for (int r = 0; r < 16; ++r) o[d][r] *= shrink;
    }
  }
  // The weights of my scores 4 u .. + 3 of a stage, and the sum of them: as they are rounded, two an instruction; of two terms in place.
  __device__ __forceinline__ void weights(f32x16 (&s)[2], Op (&w)[4], int u, float at) {
#pragma unroll
    for (int i = 0; i < 4; i += 2) {
      const int e = 4 * u + i;
      f32x2t p;
      p[0] = __builtin_amdgcn_exp2f(fmaf(s[e / 16][e % 16], q.unit, -at));
      p[1] = __builtin_amdgcn_exp2f(fmaf(s[e / 16][e % 16 + 1], q.unit, -at));
      if constexpr (kTerms == 2) {
        s[e / 16][e % 16] = p[0];
        s[e / 16][e % 16 + 1] = p[1];
        l[e / 2 % 4] += p[0];
        l[(e / 2 + 2) % 4] += p[1];
      } else if constexpr (std::is_same<Op, bf16x8>::value) {
        const bf16x2t z = __builtin_convertvector(p, bf16x2t);
        w[e / 8][e % 8] = z[0];
        w[e / 8][e % 8 + 1] = z[1];
        l[e / 2 % 4] = __builtin_amdgcn_fdot2_f32_bf16(z, bf16x2t{(__bf16)1.f, (__bf16)1.f}, l[e / 2 % 4], false);
      } else {
        const f16x2t z = {(_Float16)p[0], (_Float16)p[1]};
        w[e / 8][e % 8] = z[0];
        w[e / 8][e % 8 + 1] = z[1];
        l[e / 2 % 4] = __builtin_amdgcn_fdot2(z, f16x2t{(_Float16)1.f, (_Float16)1.f}, l[e / 2 % 4], false);
      }
    }
  }
  // The results of the wave's 32 rows by way of 8 KB of LDS, so that a store is four whole rows: to(i) is where the wave's row i goes, nullptr:
  // nowhere.  (Straight from the registers a store is 16 bytes of 32 rows each, and took the last 3 us of a workgroup.)
  template <typename TO, typename To>
  __device__ __forceinline__ void finish_rows(lds_char* room, To to) const {
    static_assert(sizeof(TO) == 2, "");
    const int lane = threadIdx.x & 63, n = lane & 31, h = lane >> 5;
    const float half = (l[0] + l[1]) + (l[2] + l[3]), sum = half + __shfl_xor(half, 32), inv = sum == 0.f ? 0.f : 1.f / sum;
    typedef typename std::conditional<std::is_same<TO, uint16_t>::value, __bf16, _Float16>::type Elem;
    typedef Elem Elem4 __attribute__((ext_vector_type(4)));
#pragma unroll
    for (int d = 0; d < 4; ++d)
#pragma unroll
      for (int r = 0; r < 16; r += 4) {
        const f32x4 y = {o[d][r] * inv, o[d][r + 1] * inv, o[d][r + 2] * inv, o[d][r + 3] * inv};
        *(__attribute__((address_space(3))) Elem4*)(room + n * 256 + 16 * chunk_place(n, 4 * d + r / 4) + 8 * h) = __builtin_convertvector(y, Elem4);
      }
    wave_lds_order();
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const int i = 4 * j + (lane >> 4);
      TO* const p = to(i);
      if (p) *reinterpret_cast<u32x4*>(p + 8 * (lane & 15)) = *(const __attribute__((address_space(3))) u32x4*)(room + i * 256 + 16 * chunk_place(i, lane & 15));
    }
  }
  // The row's result, or with part != nullptr a part of it.  The lanes of a row's two halves call together.
  template <typename TO>
  __device__ __forceinline__ void finish(TO* out, float* part, int h) const {
    const float half = (l[0] + l[1]) + (l[2] + l[3]), sum = half + __shfl_xor(half, 32), inv = sum == 0.f ? 0.f : 1.f / sum;
#pragma unroll
    for (int d = 0; d < 4; ++d)
#pragma unroll
      for (int r = 0; r < 16; r += 4) {
        const f32x4 y = {o[d][r], o[d][r + 1], o[d][r + 2], o[d][r + 3]};
        const int c = 32 * d + 2 * r + 4 * h;
        if (part) put4(part + c, y);
        else put4(out + c, f32x4{y[0] * inv, y[1] * inv, y[2] * inv, y[3] * inv});
      }
    if (part && h == 0) {
      part[kD] = m - kLift;              // (what the weights are powers of two from)
      part[kD + 1] = sum;
    }
  }
};

// The loop.  A stage has a half for the vector units (its scores become weights) and a half for the matrix units (its values, then the
// scores of the next stage).  Waves 0-3 are half a stage ahead of waves 4-7, with which they share the SIMDs: while one of a SIMD's
// two waves keeps the matrix unit, the other has the vector unit.  A barrier ends every half.
//
// While a wave keeps the matrix unit full, the other one of the SIMD hardly gets a request to memory out (280 cycles each, against 22
// beside a wave that does anything else): all requests are made in matrix halves, between the products.  They are for K two stages ahead and V one
// (of j: K of j + 3 and V of j + 2, counted from the weights that are in use), so in LDS are three stages of either; the places were last
// read at least a half before, and what was asked for has arrived at the end of the wave's next vector half, a half before anyone
// reads it.  (Transposed reads from LDS wait for everything that is on its way there: requests come behind a matrix half's last.)
//
// A matrix half is eight groups of four products; the operands of the group after the next are read before a group's products,
// those of the first two before the barrier.
constexpr int kPipeStage = kPipeKeys * 256, kPipeStages = 3, kPipeLds = 2 * kPipeStages * kPipeStage + 16;
constexpr int kRestAt = 2 * kPipeStages * kPipeStage, kRestWave = 8 * 1024;       // third terms of the query rows, instead of those 16 bytes
template <typename Op, int kTerms>
constexpr int pipe_lds() { return PipeState<Op, kTerms>::kRest ? kRestAt + kPipeWaves * kRestWave : kPipeLds; }
// least: keys that all rows of the workgroup see.
// active: the wave has rows of its own; one that has none only brings its share of the cache's.
// Returns 8 KB of LDS that are the wave's from then on: of the four stages that nothing is on its way to any more.
// rows: the cache's rows that [first, end) stand for.
// query(i): the wave's query row i.  They come through LDS, whole rows an instruction, into places of the later stages: 10500 cycles until they and the
// first keys are there, where all workgroups begin at once (asked for by lanes each for its own row, 32 bytes of 32 rows an instruction, 12200; 16384
// tokens, window 1024, 351 -> 348 us).  HeldRows: st.q is filled already.
struct HeldRows {};
__device__ __forceinline__ lds_char* query_room(lds_char* lds, int wave) {
  const int stage = (wave >> 1 & 1) + 1, of_v = wave >> 2;
  return lds + (of_v * kPipeStages + stage) * kPipeStage + (wave & 1) * (kPipeStage / 2);
}
template <int kKind, typename TK, typename TV, typename Op, int kTerms, typename Rows = AllRows, typename Query = HeldRows>
__device__ __forceinline__ lds_char* pipe_loop(char* lds_, const CacheRows<TK>& K, const CacheRows<TV>& V, int first, int end, int least, bool active,
                                          PipeState<Op, kTerms>& st, const Rows& rows = Rows(), const Query& query = Query()) {
  lds_char* const lds = (lds_char*)lds_;
  const int lane = threadIdx.x & 63, wave = wave_of(), n = lane & 31, h = lane >> 5;
  const bool late = wave >= kPipeWaves / 2;
  Feed<TK, kKind, Op> fk;
  Feed<TV, kKind, Op> fv;
  constexpr int kV = kPipeStages * kPipeStage;
  const int row_end = rows.end(end);
  auto row_of = [&](int k) { return first_row(rows.row(k + kFeedRows * wave), row_end); };
  auto look_up = [&](int k) { return kKind == kPages ? RowMap<true>::block(K.pg, K.b, row_of(k)) : 0; };
  auto uniform = [](int e) { return __builtin_amdgcn_readfirstlane(e); };
  constexpr bool kRest = PipeState<Op, kTerms>::kRest;
  const lds_char* const rest = lds + kRestAt + wave * kRestWave;
  int* const found = (int*)(lds_ + 2 * kPipeStages * kPipeStage) + (late ? 1 : 0);      // stage (its end) with a value that is not finite
  if (!kRest && (threadIdx.x & (64 * kPipeWaves / 2 - 1)) == 0) *found = 0;
  auto landed = [] { __builtin_amdgcn_s_waitcnt(0x0f70); };     // vmcnt(0): what I asked for is in LDS
  int e_v = look_up(first + 2 * kPipeKeys), e_k = look_up(first + 3 * kPipeKeys), e_new = 0;      // of the next to be asked for
  const int e_first[3] = {look_up(first), look_up(first + kPipeKeys), e_v};
  constexpr bool kQuery = !std::is_same<Query, HeldRows>::value;
  Feed<TK, kKind, Op> fk_first[3];                               // K of the first three stages, V of two
  Feed<TV, kKind, Op> fv_first[2];
  auto ask_first = [&](int i) __attribute__((always_inline)) {
    const int k = first + i * kPipeKeys, e = uniform(e_first[i]);
    fk_first[i].aim(K, row_of(k), row_end, e, lane);
    fk_first[i].ask(lds + i * kPipeStage, wave);
    if constexpr (kQuery) {
      if (i == 0) {                                              // (they lie where the other stages will, but V's first)
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          const int r = 4 * j + (lane >> 4);
          __builtin_amdgcn_global_load_lds((global_char*)(query(r) + 16 * chunk_place(r, lane & 15)),
                                           (__attribute__((address_space(3))) void*)(query_room(lds, wave) + 1024 * j), 16, 0, 0);
        }
      }
    }
    __builtin_amdgcn_sched_barrier(0);
    if (i < 2) {
      fv_first[i].aim(V, row_of(k), row_end, e, lane);
      fv_first[i].ask(lds + kV + i * kPipeStage, wave);
    }
    __builtin_amdgcn_sched_barrier(0);
  };
  auto put_first = [&](int i) __attribute__((always_inline)) {
    fk_first[i].put(lds + i * kPipeStage, lane, wave);
    if (i < 2) fv_first[i].put(lds + kV + i * kPipeStage, lane, wave);
  };
  constexpr bool kDirect = Feed<TK, kKind, Op>::kDirect && Feed<TV, kKind, Op>::kDirect;
  constexpr int kBehind = kDirect ? Feed<TV, kKind, Op>::kLoads : 0;      // requests behind those for the queries
  ask_first(0);
  if constexpr (kQuery) {
    __builtin_amdgcn_s_waitcnt(0x0f70 | kBehind);      // vmcnt(kBehind)
    wave_lds_order();
    st.q.load(query_room(lds, wave), n, h);
    __builtin_amdgcn_s_waitcnt(0xc07f);                // lgkmcnt(0): its place is free
  } else {
    ask_first(1);
    ask_first(2);
  }
  put_first(0);
  if constexpr (!kQuery) {
    put_first(1);
    put_first(2);
  }
  landed();      // (V of the first stage too: the early waves read all of it before the next barrier that has a wait in front of it)
  __syncthreads();
  if constexpr (kQuery) {
    ask_first(1);
    ask_first(2);
  }
  f32x16 s[2];                                // scores of a stage
  constexpr int kAhead = kTerms == 1 ? 2 : 1, kOperands = kAhead + 1;      // groups read ahead (of two terms a group is twice as long)
  Op w[4], a[kOperands][4];                   // its weights; operands
#pragma unroll
  for (int g = 0; g < 4; ++g) {
    st.load_keys(a[0], lds, g, n, h);
    st.add_scores(s, a[0], g, rest);
  }
  if constexpr (kQuery) {
    put_first(1);
    put_first(2);
  }
  __syncthreads();                            // (K of the first stage has been read)
  if (late) {
    landed();
    __syncthreads();
  }
  int k0 = first, now = 0, next = kPipeStage, last = 2 * kPipeStage;      // places of this stage, the next, the one after
  auto stage = [&](auto masked, auto works) {
    constexpr bool kMasked = decltype(masked)::value != 0, kWorks = decltype(works)::value;
    // vector half
    if constexpr (kWorks) {
      if constexpr (kMasked) {
        if constexpr (decltype(masked)::value == 2) st.hide(s, k0, h, rows);
        else st.hide(s, k0, h, AllRows());
      }
      st.follow(st.largest(s));
      const float at = st.m == -INFINITY ? 0.f : st.m - (PipeState<Op, kTerms>::kLift);
#pragma unroll
      for (int u = 0; u < 8; ++u) st.weights(s, w, u, at);
    }
    if (k0 > first) {                                            // (the first stages' rows are there)
      fk.put(lds + last, lane, wave);
      fv.put(lds + kV + next, lane, wave);
      e_v = e_k;
      e_k = e_new;
    }
    fk.aim(K, row_of(k0 + 3 * kPipeKeys), row_end, uniform(e_k), lane);
    fv.aim(V, row_of(k0 + 2 * kPipeKeys), row_end, uniform(e_v), lane);
    landed();
    const lds_char* const v = lds + kV + now;
    const lds_char* const k = lds + next;                        // (of the last stage: what lies there, unused)
    bool apart = false;
    if (kMasked && kRest) {                                      // values that a row must not meet?
      apart = any_not_finite<Op>(v, kPipeStage);
    } else if (kMasked) {                                        // four waves share the rows out
      constexpr int kShare = kPipeStage / (kPipeWaves / 2);
      if (any_not_finite<Op>(v + (wave % (kPipeWaves / 2)) * kShare, kShare)) *found = k0 + kPipeKeys;
    }
    if constexpr (kWorks) {
#pragma unroll
      for (int i = 0; i < kAhead; ++i) st.load_values(a[i], v, i, lane);
    }
    __syncthreads();
    // matrix half
    if constexpr (kWorks) {
      if (kMasked && !kRest) apart = *(volatile int*)found == k0 + kPipeKeys;
      if (apart) st.add_values_apart(w, s, v, lane, rows.seen_from(k0, st.limit));
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        __builtin_amdgcn_sched_barrier(0);
        const int to = i + kAhead;
        if (to < 4) st.load_values(a[to % kOperands], v, to, lane);
        else if (to < 8) st.load_keys(a[to % kOperands], k, to - 4, n, h);
        if (i < 4) {
          if (!apart) st.add_values(a[i % kOperands], w[i], s, i);
        } else st.add_scores(s, a[i % kOperands], i - 4, rest);
        if (i == 2) e_new = look_up(k0 + 4 * kPipeKeys);
        if (i == 3) fk.ask(lds + now, wave);
        if (i == 4) fv.ask(lds + kV + last, wave);
      }
      __builtin_amdgcn_sched_barrier(0);
    } else {
      e_new = look_up(k0 + 4 * kPipeKeys);
      fk.ask(lds + now, wave);
      fv.ask(lds + kV + last, wave);
    }
    __syncthreads();
    k0 += kPipeKeys;
    const int free = now;
    now = next;
    next = last;
    last = free;
  };
  const std::integral_constant<int, 2> gap;
  const std::integral_constant<int, 1> limit;
  const std::integral_constant<int, 0> no;
  const std::true_type works;
  const std::false_type idle;
  if (active) {
    if constexpr (Rows::kGap)
      while (k0 < rows.clear && k0 < end) stage(gap, works);
    while (k0 + kPipeKeys <= least && k0 < end) stage(no, works);
    while (k0 < end) stage(limit, works);
  } else {
    if constexpr (Rows::kGap)
      while (k0 < rows.clear && k0 < end) stage(limit, idle);
    while (k0 + kPipeKeys <= least && k0 < end) stage(no, idle);
    while (k0 < end) stage(limit, idle);
  }
  if (!late) __syncthreads();
  // (the last stage has asked for rows of K into what is now the last stage, and of V into the next)
  const int of_wave[4] = {now, next, kV + now, kV + last};
  return lds + (wave < 2 ? of_wave[0] : (wave < 4 ? of_wave[1] : (wave < 6 ? of_wave[2] : of_wave[3]))) + (wave & 1) * (kPipeStage / 2);
}

}  // namespace lfps
