// The prompt kernel's body for 16-bit operands (bf16, fp16, FP8 converted to bf16): tile_attn.h's products, made for the matrix
// units' rate.
#pragma once
#include "tile_attn.h"

namespace lfps {

constexpr int kPipeWaves = 8, kPipeKeys = 64, kPipeRows = 32 * kPipeWaves;       // of a workgroup; keys of a stage; query rows
constexpr int kPipeThreads = 64 * kPipeWaves, kFeedRows = kPipeKeys / kPipeWaves;   // rows of a stage that a wave brings
constexpr float kLazy = 6.f;                         // growth of a maximum, in powers of two, that is let pass

typedef __attribute__((address_space(3))) char lds_char;
typedef const __attribute__((address_space(1))) char global_char;

// How the rows of a cache lie: a slab; pages of eight rows and more; anything (smaller pages, rows very far apart).  In the first two
// the rows that a wave brings of a stage lie at offsets of 32 bits from the first, whose place is then the wave's.
enum { kSlab = 0, kPages = 1, kAnyRows = 2 };
__host__ inline int rows_kind(const KvView& kv) {
  if (kv.stride_n >= (1 << 20) || (kv.page.table && (1 << kv.page.shift) < kFeedRows)) return kAnyRows;
  return kv.page.table ? kPages : kSlab;
}

__device__ __forceinline__ int wave_of() { return __builtin_amdgcn_readfirstlane(threadIdx.x >> 6); }

// The rows of a stage that a wave brings, eight, of K or V.  16-bit elements go from memory to LDS without
// registers, four rows an instruction: lane l fills place l % 16 of row l / 16, so it asks for the chunk that belongs there.
// Rows from `end` on are the last one again: they are read by nobody's weights but 0.  The block table's entries are asked for a
// stage ahead.
template <typename T, int kKind>
struct Feed {
  static constexpr bool kDirect = sizeof(T) == 2;
  static constexpr int kLoads = kFeedRows / (kDirect ? 4 : 8);     // FP8: eight rows a load, through registers
  static constexpr int kEntries = kKind == kAnyRows ? kLoads : 1;
  u32x4 x[kDirect ? 1 : kLoads];
  int entry[kEntries];
  uint32_t whole[kLoads];                            // my pieces' places where all of the rows are there

  __device__ __forceinline__ void begin(const CacheRows<T>& c, int lane) {
#pragma unroll
    for (int i = 0; i < kLoads; ++i) whole[i] = place(c, row(i, lane), i, lane);
  }
  __device__ __forceinline__ static uint32_t place(const CacheRows<T>& c, int r, int i, int lane) {
    return __umul24((uint32_t)r, (uint32_t)c.stride_n * (uint32_t)sizeof(T)) + (uint32_t)piece(i, lane);    // (a pitch below 2^24)
  }

  __device__ __forceinline__ static int row(int i, int lane) { return kFeedRows / kLoads * i + (kDirect ? lane >> 4 : lane >> 3); }
  __device__ __forceinline__ static int piece(int i, int lane) {                  // of a row of the cache, in bytes
    return kDirect ? 16 * ((lane & 15) ^ mix((kFeedRows * wave_of()) + row(i, lane))) : 16 * (lane & 7);
  }
  // The wave's first row of the stage, one that exists.
  __device__ __forceinline__ static int first_row(int k0, int end, int wave) {
    const int w0 = k0 + kFeedRows * wave;
    return __builtin_amdgcn_readfirstlane(w0 < end ? w0 : (end - 1) & ~(kFeedRows - 1));
  }
  __device__ __forceinline__ void look_up(const CacheRows<T>& c, int k0, int end, int lane, int wave) {
    if (kKind == kSlab || !c.pg.table) return;
    const int w0 = first_row(k0, end, wave), last = end - 1 - w0;
#pragma unroll
    for (int i = 0; i < kEntries; ++i) {
      const int r = kKind == kPages ? 0 : row(i, lane);
      entry[i] = RowMap<true>::block(c.pg, c.b, w0 + (r < last ? r : last));
    }
  }
  __device__ __forceinline__ void one(const char* from, lds_char* stage, int i, int wave) {
    if constexpr (kDirect)
      __builtin_amdgcn_global_load_lds((global_char*)from, (__attribute__((address_space(3))) void*)(stage + (kFeedRows * wave + 4 * i) * 256), 16, 0, 0);
    else
      x[i] = *reinterpret_cast<const u32x4*>(from);
  }
  __device__ __forceinline__ void ask(const CacheRows<T>& c, lds_char* stage, int k0, int end, int lane, int wave) {
    const int w0 = first_row(k0, end, wave), last = end - 1 - w0;
    if constexpr (kKind == kAnyRows) {
#pragma unroll
      for (int i = 0; i < kLoads; ++i) {
        const int r = row(i, lane);
        one(reinterpret_cast<const char*>(c.at(w0 + (r < last ? r : last), entry[i])) + piece(i, lane), stage, i, wave);
      }
    } else {
      const int64_t first = kKind == kPages ? RowMap<true>::offset_in(c.pg, __builtin_amdgcn_readfirstlane(entry[0]), w0, c.stride_b, c.stride_n)
                                            : w0 * c.stride_n;
      const char* base = reinterpret_cast<const char*>(c.base + first);
      if (last >= kFeedRows - 1) {
#pragma unroll
        for (int i = 0; i < kLoads; ++i) one(base + whole[i], stage, i, wave);
      } else {
#pragma unroll
        for (int i = 0; i < kLoads; ++i) {
          const int r = row(i, lane);
          one(base + place(c, r < last ? r : last, i, lane), stage, i, wave);
        }
      }
    }
  }
  // FP8: what has arrived becomes bf16 in the stage
  __device__ __forceinline__ void put(lds_char* stage, int lane, int wave) const {
    if constexpr (!kDirect) {
#pragma unroll
      for (int i = 0; i < kLoads; ++i) {
        const int r = kFeedRows * wave + row(i, lane), c = lane & 7;
        typedef __attribute__((address_space(3))) bf16x8* Lds;
        *(Lds)(stage + r * 256 + 16 * chunk_place(r, 2 * c)) = fp8x8_to_bf16x8(x[i][0], x[i][1]);
        *(Lds)(stage + r * 256 + 16 * chunk_place(r, 2 * c + 1)) = fp8x8_to_bf16x8(x[i][2], x[i][3]);
      }
    }
  }
};

// 32 query rows of a wave.
template <typename Op>
struct PipeState {
  typedef RowState<Op, 1> Tile;
  f32x16 o[4];
  float m, l;
  typename Tile::Query q;
  int limit;

  __device__ __forceinline__ void clear() {
    m = -INFINITY;
    l = 0.f;
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
  __device__ __forceinline__ void add_scores(f32x16 (&s)[2], const Op (&a)[4], int g) const {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int c = 2 * g + (i >> 1);
      if (c == 0) {
        f32x16 zero;
#pragma unroll
        for (int r = 0; r < 16; ++r) zero[r] = 0.f;
        s[i & 1] = mfma32(a[i], q.x[0][c], zero);
      } else {
        s[i & 1] = mfma32(a[i], q.x[0][c], s[i & 1]);
      }
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
  __device__ __forceinline__ void add_values(const Op (&a)[4], const Op& w) {
#pragma unroll
    for (int d = 0; d < 4; ++d) o[d] = mfma32(a[d], w, o[d]);
  }

  // Scores of keys that the row does not see.
  __device__ __forceinline__ void hide(f32x16 (&s)[2], int first, int h) const {
#pragma unroll
    for (int b = 0; b < 2; ++b)
#pragma unroll
      for (int r = 0; r < 16; ++r)
        if (first + 32 * b + 8 * (r / 4) + 4 * h + r % 4 >= limit) s[b][r] = -INFINITY;
  }
  __device__ __forceinline__ static float largest(const f32x16& s, float mx) {
#pragma unroll
    for (int r = 0; r < 16; ++r) mx = fmaxf(mx, s[r]);
    return mx;
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
      l *= shrink;
#pragma unroll
      for (int d = 0; d < 4; ++d)
#pragma unroll
        for (int r = 0; r < 16; ++r) o[d][r] *= shrink;
    }
  }
  // The weights of my scores 4 u .. + 3 of a stage, and the sum of them as they are rounded (two an instruction).
  __device__ __forceinline__ void weights(const f32x16 (&s)[2], Op (&w)[4], int u, float at) {
#pragma unroll
    for (int i = 0; i < 4; i += 2) {
      const int e = 4 * u + i;
      f32x2t p;
      p[0] = __builtin_amdgcn_exp2f(fmaf(s[e / 16][e % 16], q.unit, -at));
      p[1] = __builtin_amdgcn_exp2f(fmaf(s[e / 16][e % 16 + 1], q.unit, -at));
      if constexpr (std::is_same<Op, bf16x8>::value) {
        const bf16x2t z = __builtin_convertvector(p, bf16x2t);
        w[e / 8][e % 8] = z[0];
        w[e / 8][e % 8 + 1] = z[1];
        l = __builtin_amdgcn_fdot2_f32_bf16(z, bf16x2t{(__bf16)1.f, (__bf16)1.f}, l, false);
      } else {
        const f16x2t z = {(_Float16)p[0], (_Float16)p[1]};
        w[e / 8][e % 8] = z[0];
        w[e / 8][e % 8 + 1] = z[1];
        l = __builtin_amdgcn_fdot2(z, f16x2t{(_Float16)1.f, (_Float16)1.f}, l, false);
      }
    }
  }
};

// The loop.  Stage j: scores of j + 1 beside the weights of j, then the values of j.  In LDS are K of two stages and V of two; what
// a stage has read is asked for again at its end, K three stages ahead and V one, and has arrived behind the first half of the next:
// one barrier a stage, between its weights and its values.  (Transposed reads from LDS wait for everything that is on its way there, so
// nothing may be asked for between a barrier and the values' reads.)
// The order inside a stage is written down in groups of four products: the operands of the next group are read first, and every
// product has its share of the vector work beside it; left to itself the compiler reads an operand just before its product.
constexpr int kPipeStage = kPipeKeys * 256;
struct PipeLds {
  lds_char* k[2];
  lds_char* v[2];
};
// Four products, each followed by kVector vector instructions, and kReads reads from LDS ahead of them.
template <int kReads, int kVector>
__device__ __forceinline__ void group_order() {
  __builtin_amdgcn_sched_group_barrier(0x100, kReads, 0);
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    __builtin_amdgcn_sched_group_barrier(0x8, 1, 0);
    __builtin_amdgcn_sched_group_barrier(0x2, kVector, 0);
  }
  __builtin_amdgcn_sched_barrier(0);
}
template <int kKind, typename TK, typename TV, typename Op>
__device__ __forceinline__ void pipe_loop(const PipeLds lds, const CacheRows<TK>& K, const CacheRows<TV>& V, int first, int end,
                                          PipeState<Op>& st) {
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), n = lane & 31, h = lane >> 5;
  int least = st.limit;
#pragma unroll
  for (int d = 1; d < 32; d <<= 1) least = min(least, __shfl_xor(least, d));
  least = __builtin_amdgcn_readfirstlane(least);
  Feed<TK, kKind> fk;
  Feed<TV, kKind> fv;
  auto arrived = [&] {
    __builtin_amdgcn_s_waitcnt(0x0f70);       // vmcnt(0): what I asked for is in LDS
    __syncthreads();                          // and what all did
  };
  auto ask_k = [&](lds_char* to, int k) {     // and the table's entries for the stage after it
    if (k < end) fk.ask(K, to, k, end, lane, wave);
    fk.look_up(K, k + kPipeKeys, end, lane, wave);
  };
  auto ask_v = [&](lds_char* to, int k) {
    if (k < end) fv.ask(V, to, k, end, lane, wave);
    fv.look_up(V, k + kPipeKeys, end, lane, wave);
  };
  fk.begin(K, lane);
  fv.begin(V, lane);
  fk.look_up(K, first, end, lane, wave);
  fv.look_up(V, first, end, lane, wave);
  ask_k(lds.k[0], first);
  fk.put(lds.k[0], lane, wave);
  ask_k(lds.k[1], first + kPipeKeys);
  if (first + kPipeKeys < end) fk.put(lds.k[1], lane, wave);
  ask_v(lds.v[0], first);
  arrived();
  f32x16 s[2][2];                             // scores of this stage and the next, by parity
  {
    Op a[4];
#pragma unroll
    for (int g = 0; g < 4; ++g) {
      st.load_keys(a, lds.k[0], g, n, h);
      st.add_scores(s[0], a, g);
    }
  }
  __syncthreads();
  ask_k(lds.k[0], first + 2 * kPipeKeys);
  float mx = st.largest(s[0][1], st.largest(s[0][0], -INFINITY));     // of my scores of the stage (where nothing is hidden)
  int k0 = first;
  auto stage = [&](auto parity, auto masked) {
    constexpr int P = decltype(parity)::value;
    constexpr bool kMasked = decltype(masked)::value;
    Op w[4], a[2][4];
    st.load_keys(a[0], lds.k[1 - P], 0, n, h);                   // (of the last stage: what lies there, unused)
    if (kMasked) {
      st.hide(s[P], k0, h);
      mx = st.largest(s[P][1], st.largest(s[P][0], -INFINITY));
    }
    st.follow(mx);
    const float at = st.m == -INFINITY ? 0.f : st.m - PipeState<Op>::Tile::kLift;
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int g = 0; g < 4; ++g) {
      if (g < 3) st.load_keys(a[(g + 1) & 1], lds.k[1 - P], g + 1, n, h);
      st.add_scores(s[1 - P], a[g & 1], g);
      st.weights(s[P], w, g, at);
      if (g < 3) group_order<4, 3>();
      else group_order<0, 3>();
    }
    if (k0 + 2 * kPipeKeys < end) fk.put(lds.k[P], lane, wave);
    fv.put(lds.v[P], lane, wave);
    arrived();
    st.load_values(a[0], lds.v[P], 0, lane);
#pragma unroll
    for (int t = 0; t < 4; ++t) {
      if (t < 3) st.load_values(a[(t + 1) & 1], lds.v[P], t + 1, lane);
      st.add_values(a[t & 1], w[t]);
      if (t < 2) {
        st.weights(s[P], w, 4 + 2 * t, at);
        st.weights(s[P], w, 5 + 2 * t, at);
      } else if (!kMasked) {
        mx = st.largest(s[1 - P][t - 2], t == 2 ? -INFINITY : mx);
      }
      if (t < 2) group_order<8, 6>();
      else if (t == 2) group_order<8, 2>();
      else group_order<0, 2>();
    }
    ask_k(lds.k[1 - P], k0 + 3 * kPipeKeys);
    ask_v(lds.v[1 - P], k0 + kPipeKeys);
    k0 += kPipeKeys;
  };
  const std::integral_constant<int, 0> even;
  const std::integral_constant<int, 1> odd;
  while (k0 + 2 * kPipeKeys <= least && k0 + kPipeKeys < end) {
    stage(even, std::false_type{});
    stage(odd, std::false_type{});
  }
  while (k0 < end) {
    stage(even, std::true_type{});
    if (k0 < end) stage(odd, std::true_type{});
  }
}

}  // namespace lfps
