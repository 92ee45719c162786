// Attention of many query rows over a range of a request's cache rows on the matrix units: the body shared by the prompt kernel
// (prompt_attn.hip) and the shared-prefix kernel (prefix_attn.hip).
//
//   o[m] = sum_j p_mj V_j / sum_j p_mj,   p_mj = exp((q_m . K_j - max_j q_m . K_j) / sqrt(D)),   j < limit(m)
//
// in one pass over K and V: a running maximum per row, sums rescaled when it grows (online softmax).  The G heads of a KV group see
// the same rows, so a query row m is a (token, head) pair, heads fastest, and a workgroup's rows share every K and V row.
//
// A wave owns 32 query rows.  Scores are computed transposed, S^T = K Q^T, by 32x32 matrix instructions: a lane then holds one
// query row's scores (its column) for 16 of 32 keys, so maximum and sum are taken in registers with one exchange between
// the wave's halves, and the weights are the second product's operand (O^T = V^T P^T) as they lie, if the keys of that
// product are taken in the order in which the first one leaves them: V is read from LDS transposed, four keys a lane
// (ds_read_b64_tr), with each half of the wave reading the keys it holds weights for.
#pragma once
#include "prefix_groups.h"

#include <type_traits>

namespace lfps {

constexpr int kTileThreads = 256;            // four waves
constexpr float kLog2e = 1.4426950408889634f;

typedef float f32x16 __attribute__((ext_vector_type(16)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x2t __attribute__((ext_vector_type(2)));
typedef _Float16 f16x2t __attribute__((ext_vector_type(2)));
typedef __attribute__((address_space(3))) char lds_char;

// The rows [.., end) of one request and KV head as a kernel reads them.
template <typename T>
struct CacheRows {
  const T* base;                             // row 0 of the request (contiguous) or of the pool, at the KV head
  int64_t stride_b, stride_n;
  KvPage pg;
  int b;
  __device__ __forceinline__ CacheRows(const void* p, const KvView& kv, int b_, int g) : stride_b(kv.stride_b), stride_n(kv.stride_n), pg(kv.page), b(b_) {
    base = (const T*)p + (kv.page.table ? (int64_t)0 : (int64_t)b_ * kv.stride_b) + (int64_t)g * kv.stride_h;
  }
  __device__ __forceinline__ int entry(int r) const { return pg.table ? RowMap<true>::block(pg, b, r) : 0; }
  __device__ __forceinline__ const T* at(int r, int e) const {
    return base + (pg.table ? RowMap<true>::offset_in(pg, e, r, stride_b, stride_n) : (int64_t)r * stride_n);
  }
};

// ---- the rows that a loop walks --------------------------------------------------------------------------------
// All of a range, in which a query row sees those below its limit; or a range with a gap: from row `at` of the walk on (a multiple of eight), it has
// the cache's rows `by` further up.  All else is counted along the walk: a query row does not see its rows [sinks, from) either, and from `clear` on
// none of the workgroup's misses one for its window.
struct AllRows {
  static constexpr bool kGap = false;
  __device__ __forceinline__ int row(int k) const { return k; }
  __device__ __forceinline__ int end(int e) const { return e; }
  __device__ __forceinline__ int steps(int e) const { return e; }
  // is key `key` of those from row `base` on seen by a query row of this limit?
  __device__ __forceinline__ auto seen_from(int base, int limit) const {
    return [seen = limit - base](int key) { return key < seen; };
  }
};
struct GapRows {
  static constexpr bool kGap = true;
  int at, by, clear, sinks, from;
  __device__ __forceinline__ int row(int k) const { return k < at ? k : k + by; }
  __device__ __forceinline__ int end(int e) const { return e > at ? e + by : e; }      // of the cache's rows, for a walk that ends at e
  __device__ __forceinline__ int steps(int e) const { return e - by; }                 // and the other way round, e > at + by
  __device__ __forceinline__ auto past_gap_from(int base) const {               // (a key's place in the gap is one unsigned comparison)
    return [first = sinks - base, gap = (uint32_t)(from > sinks ? from - sinks : 0)](int key) { return (uint32_t)(key - first) >= gap; };
  }
  __device__ __forceinline__ auto seen_from(int base, int limit) const {        // (no branches: a key's place in the gap is one unsigned comparison)
    return [seen = limit - base, first = sinks - base, gap = (uint32_t)(from > sinks ? from - sinks : 0)](int key) {
      return (bool)((int)(key < seen) & (int)((uint32_t)(key - first) >= gap));
    };
  }
};

// ---- the elements in LDS and in the matrix instructions ------------------------------------------------------
// A row in LDS is kRowBytes long, in chunks of 16 bytes; chunk c of row r lies at place c ^ mix(r) of the row.  The LDS has 64 banks of
// four bytes, which is 16 chunks: sixteen consecutive rows read at one chunk (scores), and four rows at four neighbouring chunks (16-bit
// values), come from different ones.  (With c ^ 2 (r & 7), whose eight places serve half of that, the LDS took twice as long.)
__device__ __forceinline__ int mix(int r) { return ((r & 3) << 2) | ((r >> 2) & 3); }
// fp32 values are read along a row, in two rows four apart at once.
__device__ __forceinline__ int mix_f32(int r) { return (r & 3) | ((r & 4) << 1) | ((r & 8) >> 1); }
__device__ __forceinline__ int chunk_place(int r, int c) { return c ^ mix(r); }
__device__ __forceinline__ int chunk_place_f32(int r, int c) { return c ^ mix_f32(r); }

template <typename T>
struct InLds { typedef bf16x8 Op; static constexpr int kRowBytes = 256; };       // bf16, and FP8 (every value is a bf16 and an fp16 value)
template <>
struct InLds<_Float16> { typedef f16x8 Op; static constexpr int kRowBytes = 256; };
template <>
struct InLds<float> { typedef float Op; static constexpr int kRowBytes = 512; };

__device__ __forceinline__ f32x16 mfma32(bf16x8 a, bf16x8 b, f32x16 c) { return __builtin_amdgcn_mfma_f32_32x32x16_bf16(a, b, c, 0, 0, 0); }
__device__ __forceinline__ f32x16 mfma32(f16x8 a, f16x8 b, f32x16 c) { return __builtin_amdgcn_mfma_f32_32x32x16_f16(a, b, c, 0, 0, 0); }
__device__ __forceinline__ f32x16 mfma32(float a, float b, f32x16 c) { return __builtin_amdgcn_mfma_f32_32x32x2f32(a, b, c, 0, 0, 0); }

__device__ __forceinline__ int wave_of() { return __builtin_amdgcn_readfirstlane(threadIdx.x >> 6); }

// Eight FP8 values as eight of Op (exact).
template <typename Op>
__device__ __forceinline__ Op fp8x8_to(uint32_t w0, uint32_t w1) {
  Op x;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const uint32_t w = i < 2 ? w0 : w1;
    if constexpr (std::is_same<Op, bf16x8>::value) {
      const bf16x2t y = i % 2 ? __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, 1.f, true) : __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, 1.f, false);
      x[2 * i] = y[0];
      x[2 * i + 1] = y[1];
    } else {
      const f16x2t y = i % 2 ? __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w, 1.f, true) : __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w, 1.f, false);
      x[2 * i] = y[0];
      x[2 * i + 1] = y[1];
    }
  }
  return x;
}

// The kRows rows of a stage, of K or V, that a wave brings.  16- and 32-bit elements go from memory to LDS without registers, 1 KB an
// instruction: lane l fills the l-th 16 bytes of it, so it asks for the chunk that belongs there.  FP8 goes through registers and
// becomes Op's type.  Rows from `end` on are the last one again: they are read by nobody's weights but 0.
template <typename T, int kRows, typename Op>
struct StageFeed {
  static constexpr bool kDirect = sizeof(T) > 1;
  static constexpr int kPieces = kD * (int)sizeof(T) / 16, kRowsOfLoad = 64 / kPieces, kLoads = kRows / kRowsOfLoad;
  u32x4 x[kDirect ? 1 : kLoads];

  __device__ __forceinline__ static int row(int i, int lane) { return kRows * wave_of() + kRowsOfLoad * i + lane / kPieces; }
  __device__ __forceinline__ static int piece(int i, int lane) {          // of a row of the cache, in bytes
    const int place = lane % kPieces, r = row(i, lane);
    return 16 * (!kDirect ? place : (sizeof(T) == 4 ? chunk_place_f32(r, place) : chunk_place(r, place)));
  }
  // Where the rows of a stage lie.  The block table's entries are read a stage before they are used, and all places are made before
  // any row is asked for: waits for an entry are waits for every row that is on its way to LDS (16 of them, one after the other, were
  // 4.8 us of the 15 of a workgroup over 128 rows).  K and V of one element size lie at the same offsets.
  struct Places {
    int e[kLoads];
    int64_t off[kLoads];
    template <typename Rows = AllRows>
    __device__ __forceinline__ void look_up(const CacheRows<T>& c, int k0, int end, int lane, const Rows& rows = Rows()) {
      if (!c.pg.table) return;
#pragma unroll
      for (int i = 0; i < kLoads; ++i) e[i] = c.entry(rows.row(min(k0 + row(i, lane), end - 1)));
    }
    template <typename Rows = AllRows>
    __device__ __forceinline__ void aim(const CacheRows<T>& c, int k0, int end, int lane, const Rows& rows = Rows()) {
      if (c.pg.table) {
#pragma unroll
        for (int i = 0; i < kLoads; ++i) off[i] = RowMap<true>::offset_in(c.pg, e[i], rows.row(min(k0 + row(i, lane), end - 1)), c.stride_b, c.stride_n);
      } else {
#pragma unroll
        for (int i = 0; i < kLoads; ++i) off[i] = (int64_t)rows.row(min(k0 + row(i, lane), end - 1)) * c.stride_n;
      }
    }
  };
  __device__ __forceinline__ void ask(const CacheRows<T>& c, const int64_t (&off)[kLoads], lds_char* stage, int lane) {
#pragma unroll
    for (int i = 0; i < kLoads; ++i) {
      const char* p = reinterpret_cast<const char*>(c.base + off[i]) + piece(i, lane);
      if constexpr (kDirect)
        __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) char*)p,
                                         (__attribute__((address_space(3))) void*)(stage + (kRows * wave_of() + kRowsOfLoad * i) * InLds<T>::kRowBytes), 16, 0, 0);
      else
        x[i] = *reinterpret_cast<const u32x4*>(p);
    }
  }
  __device__ __forceinline__ void put(lds_char* stage, int lane) const {
    if constexpr (!kDirect) {
#pragma unroll
      for (int i = 0; i < kLoads; ++i) {
        const int r = row(i, lane), c = lane % kPieces;
        typedef __attribute__((address_space(3))) Op* Lds;
        *(Lds)(stage + r * 256 + 16 * chunk_place(r, 2 * c)) = fp8x8_to<Op>(x[i][0], x[i][1]);
        *(Lds)(stage + r * 256 + 16 * chunk_place(r, 2 * c + 1)) = fp8x8_to<Op>(x[i][2], x[i][3]);
      }
    }
  }
};

// ---- the query rows of a wave ---------------------------------------------------------------------------------
// Lane (n, h) (n = lane % 32, h = lane / 32) holds of query row n the channels that the first product wants from it: of step s
// the chunk 16 s + 8 h .. + 7 (16-bit operands; kTerms > 1: an fp32 query as a sum of that many 16-bit terms), of fp32 operands
// the channels 8 s + 4 h .. + 3.  `unit`: the factor from the products to scores in powers of two.
template <typename Op, int kTerms>
struct QueryTile {
  Op x[kTerms][8];
  float unit;
  __device__ __forceinline__ void load(const typename std::conditional<std::is_same<Op, bf16x8>::value, uint16_t, _Float16>::type* q, int h) {
    static_assert(kTerms == 1, "");
#pragma unroll
    for (int s = 0; s < 8; ++s) x[0][s] = *reinterpret_cast<const Op*>(q + 16 * s + 8 * h);
    unit = kLog2e * 0.08838834764831845f;
  }
  // The same from 32 rows in LDS, mine the n-th.
  __device__ __forceinline__ void load(const lds_char* rows, int n, int h) {
    static_assert(kTerms == 1, "");
#pragma unroll
    for (int s = 0; s < 8; ++s) x[0][s] = *(const __attribute__((address_space(3))) Op*)(rows + n * 256 + 16 * chunk_place(n, 2 * s + h));
    unit = kLog2e * 0.08838834764831845f;
  }
  // An fp32 row.  fp16 terms are taken of the row scaled by a power of two that
  // puts its largest element just below 2^14, so that any fp32 query fits and the second term keeps its bits.
  // rest: what the terms leave, as one term more, chunk after chunk (each 64 lanes' 16 bytes).
  __device__ __forceinline__ void load(const float* q, int h, lds_char* rest = nullptr) {
    float f[8][8];
    float big = 0.f;
#pragma unroll
    for (int s = 0; s < 8; ++s) {
      const f32x4 a = *reinterpret_cast<const f32x4*>(q + 16 * s + 8 * h), b = *reinterpret_cast<const f32x4*>(q + 16 * s + 8 * h + 4);
#pragma unroll
      for (int c = 0; c < 4; ++c) {
        f[s][c] = a[c];
        f[s][4 + c] = b[c];
      }
#pragma unroll
      for (int c = 0; c < 8; ++c) big = fmaxf(big, fabsf(f[s][c]));
    }
    unit = kLog2e * 0.08838834764831845f;
    float up = 1.f;
    if constexpr (std::is_same<Op, f16x8>::value) {
      big = fmaxf(big, __shfl_xor(big, 32));
      int e = 0;
      if (big > 0.f && big < INFINITY) e = 14 - (((__float_as_int(big) >> 23) & 255) - 126);
      e = e > 100 ? 100 : e;                                   // (2^e and its inverse stay normal; below 2^-86 a row scores 0 in any case)
      up = __int_as_float((127 + e) << 23);
      unit *= __int_as_float((127 - e) << 23);
    }
#pragma unroll
    for (int s = 0; s < 8; ++s) {
      Op left;
#pragma unroll
      for (int c = 0; c < 8; c += 2) {
        f32x2t y = {f[s][c] * up, f[s][c + 1] * up};
        typedef typename std::conditional<std::is_same<Op, bf16x8>::value, __bf16, _Float16>::type Elem;
#pragma unroll
        for (int t = 0; t < kTerms; ++t)
#pragma unroll
          for (int i = 0; i < 2; ++i) {
            x[t][s][c + i] = (Elem)y[i];
            y[i] -= (float)x[t][s][c + i];
          }
        left[c] = (Elem)y[0];
        left[c + 1] = (Elem)y[1];
      }
      if (rest) *(__attribute__((address_space(3))) Op*)(rest + 1024 * s + 16 * (threadIdx.x & 63)) = left;
    }
  }
};
template <int kTerms>
struct QueryTile<float, kTerms> {
  f32x4 x[16];
  float unit;
  __device__ __forceinline__ void load(const float* q, int h) {
#pragma unroll
    for (int s = 0; s < 16; ++s) x[s] = *reinterpret_cast<const f32x4*>(q + 8 * s + 4 * h);
    unit = kLog2e * 0.08838834764831845f;
  }
};

// ---- values that are not finite ------------------------------------------------------------------------------
// A row that does not see a key gives it the weight 0, and 0 times an infinity or NaN among that key's values is not 0.  Where some
// row of a wave does not see all keys of a step, the step's values are looked through; if any is not finite, they are taken in key
// by key, by the rows that see the key.
template <typename Op>
__device__ __forceinline__ bool any_not_finite(const lds_char* rows, int bytes) {
  // One more than an exponent of ones is a carry into the sign's place.
  constexpr bool kF32 = std::is_same<Op, float>::value, kF16 = std::is_same<Op, f16x8>::value;
  constexpr uint32_t kExp = kF32 ? 0x7F800000u : (kF16 ? 0x7C007C00u : 0x7F807F80u), kOne = kF32 ? 0x00800000u : (kF16 ? 0x04000400u : 0x00800080u);
  uint32_t carries = 0;
#pragma unroll 4
  for (int at = 16 * (threadIdx.x & 63); at < bytes; at += 1024) {
    const u32x4 x = *(const __attribute__((address_space(3))) u32x4*)(rows + at);
#pragma unroll
    for (int i = 0; i < 4; ++i) carries |= (x[i] & kExp) + kOne;
  }
  return __ballot((carries & (kF32 ? 0x80000000u : 0x80008000u)) != 0) != 0;
}
// o += weights of `keys` keys (a multiple of 32) times their values at v, key by key on the vector units, of keys that the row sees(key).
// weight(i, half): my weight of the i-th of the keys that that half of the wave holds.  Slow, and small: almost no call comes here.
template <typename Op, typename Weight, typename Sees>
__device__ __forceinline__ void add_apart(f32x16 (&o)[4], Weight weight, const lds_char* v, int keys, Sees sees, int lane) {
  const int h = lane >> 5;
#pragma unroll 1
  for (int key = 0; key < keys; ++key) {
    const float mine = weight((key >> 3) * 4 + (key & 3)), other = __shfl_xor(mine, 32);
    const float w = h == ((key >> 2) & 1) ? mine : other;
    if (!sees(key)) continue;
#pragma unroll
    for (int d = 0; d < 4; ++d)
#pragma unroll
      for (int r = 0; r < 16; r += 4) {
        float x[4];
        if constexpr (std::is_same<Op, float>::value) {
#pragma unroll
          for (int i = 0; i < 4; ++i)
            x[i] = *(const __attribute__((address_space(3))) float*)(v + key * 512 + 16 * chunk_place_f32(key, 2 * r + 4 * h + i) + 4 * d);
        } else {
          typedef typename std::conditional<std::is_same<Op, bf16x8>::value, __bf16, _Float16>::type Elem;
          typedef Elem Elem4 __attribute__((ext_vector_type(4)));
          const Elem4 y = *(const __attribute__((address_space(3))) Elem4*)(v + key * 256 + 16 * chunk_place(key, 4 * d + r / 4) + 8 * h);
#pragma unroll
          for (int i = 0; i < 4; ++i) x[i] = (float)y[i];
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) o[d][r + i] = fmaf(w, x[i], o[d][r + i]);
      }
  }
}
__device__ __forceinline__ f32x16 zeros16() {
  f32x16 z;
#pragma unroll
  for (int r = 0; r < 16; ++r) z[r] = 0.f;
  return z;
}

// ---- the state of a wave's 32 rows ----------------------------------------------------------------------------
// kTerms: 1: the query is 16-bit and the weights are rounded to 16 bits, as the output will be; 2: fp32 query and results.  An fp32
// query, and an fp32 weight, is then the sum of query_terms 16-bit ones: three of bf16, which hold it whole, two of fp16 (2^-22 is left).
// Two of bf16 leave 2^-18 of each: 1.2 to 1.5e-6 from 64 bits with a few hundred rows, where these are 0.5e-6.
template <typename Op, int kTerms>
constexpr int query_terms() { return kTerms == 1 ? 1 : (std::is_same<Op, bf16x8>::value ? 3 : 2); }
template <typename Op, int kTerms>
struct RowState {
  static constexpr int kWeightTerms = query_terms<Op, kTerms>();
  typedef QueryTile<Op, query_terms<Op, kTerms>()> Query;
  static constexpr bool kF32 = std::is_same<Op, float>::value;
  static constexpr int kRowBytes = kF32 ? 512 : 256;
  // Weights of fp16 values are held 2^14 (2^8 with one term) times as large, or those below 2^-24 of the row's largest would be lost.
  static constexpr float kLift = std::is_same<Op, f16x8>::value ? (kTerms == 1 ? 8.f : 14.f) : 0.f;
  f32x16 o[4];                               // of row n: with i = 8 (r / 4) + 4 h + r % 4, channel 32 d + i, of fp32 operands 4 i + d
  float m, l;                                // largest score so far, in powers of two; the sum of the weights of my half's keys

  __device__ __forceinline__ void clear() {
#pragma unroll
    for (int d = 0; d < 4; ++d)
#pragma unroll
      for (int r = 0; r < 16; ++r) o[d][r] = 0.f;
    m = -INFINITY;
    l = 0.f;
  }

  // Scores of the 32 keys whose rows begin at `k`.
  __device__ __forceinline__ static f32x16 scores(const char* k, const Query& q, int n, int h) {
    f32x16 s;
#pragma unroll
    for (int r = 0; r < 16; ++r) s[r] = 0.f;
    if constexpr (kF32) {
#pragma unroll
      for (int c = 0; c < 16; ++c) {
        const f32x4 a = *reinterpret_cast<const f32x4*>(k + n * 512 + 16 * chunk_place_f32(n, 2 * c + h));
#pragma unroll
        for (int i = 0; i < 4; ++i) s = mfma32(a[i], q.x[c][i], s);
      }
    } else {
#pragma unroll
      for (int c = 0; c < 8; ++c) {
        const Op a = *reinterpret_cast<const Op*>(k + n * 256 + 16 * chunk_place(n, 2 * c + h));
#pragma unroll
        for (int t = query_terms<Op, kTerms>() - 1; t >= 0; --t) s = mfma32(a, q.x[t][c], s);
      }
    }
    return s;
  }

  // The eight values that lane (n, h) puts into the second product's step t (keys 16 t .. + 15 of those at `v`), channel block d.
  __device__ __forceinline__ static Op values(const char* v, int t, int d, int lane) {
    const int h = lane >> 5, i = lane & 15, key = 16 * t + 4 * h + (i >> 2), chunk = 4 * d + 2 * ((lane >> 4) & 1) + ((i & 3) >> 1);
    typedef __attribute__((address_space(3))) s16x4* Lds;
    union {
      s16x4 half[2];
      Op op;
    } x;
    x.half[0] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((Lds)(v + key * 256 + 16 * chunk_place(key, chunk) + 8 * (i & 1)));
    x.half[1] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((Lds)(v + (key + 8) * 256 + 16 * chunk_place(key + 8, chunk) + 8 * (i & 1)));
    return x.op;
  }

  // One step of kBlocks * 32 keys: scores s (products) -> weights, sums and values.  first: position of the first key; limit: the
  // keys that row n sees; masked: some row of the wave sees fewer than all of these.
  template <int kBlocks, typename Rows>
  __device__ __forceinline__ void step(f32x16 (&s)[kBlocks], const char* v, float unit, int first, int limit, bool masked, int lane, const Rows& rows) {
    const int h = lane >> 5;
    float mx = m;
    const auto sees = rows.seen_from(first + 4 * h, limit);
#pragma unroll
    for (int b = 0; b < kBlocks; ++b)
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        s[b][r] *= unit;
        if (masked) s[b][r] = sees(32 * b + 8 * (r / 4) + r % 4) ? s[b][r] : -INFINITY;
        mx = fmaxf(mx, s[b][r]);
      }
    mx = fmaxf(mx, __shfl_xor(mx, 32));
    const float at = mx == -INFINITY ? 0.f : mx - kLift;       // (a row that has seen nothing yet: weights 0, not NaN)
    const float shrink = mx == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(m - mx);
    m = mx;
    l *= shrink;
#pragma unroll
    for (int d = 0; d < 4; ++d)
#pragma unroll
      for (int r = 0; r < 16; ++r) o[d][r] *= shrink;
#pragma unroll
    for (int b = 0; b < kBlocks; ++b)
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        s[b][r] = __builtin_amdgcn_exp2f(s[b][r] - at);
        l += s[b][r];
      }
#pragma unroll
    for (int b = 0; b < kBlocks; ++b) {
      const char* const vb = v + 32 * b * kRowBytes;
      if (masked && any_not_finite<Op>((const lds_char*)vb, 32 * kRowBytes)) {
        auto weight = [&](int i) {
          float x = 0.f;
#pragma unroll
          for (int r = 0; r < 16; ++r) x = r == i ? s[b][r] : x;
          return x;
        };
        add_apart<Op>(o, weight, (const lds_char*)vb, 32, rows.seen_from(first + 32 * b, limit), lane);
      } else {
        add_values(s[b], vb, lane);
      }
    }
  }

  // o += weights of 32 keys times their values
  __device__ __forceinline__ void add_values(const f32x16& p, const char* v, int lane) {
    if constexpr (kF32) {
      const int h = lane >> 5, n = lane & 31;
#pragma unroll
      for (int r = 0; r < 16; ++r) {                             // (a lane's four channels are one read)
        const int key = 8 * (r / 4) + 4 * h + r % 4;
        const f32x4 x = *reinterpret_cast<const f32x4*>(v + key * 512 + 16 * chunk_place_f32(key, n));
#pragma unroll
        for (int d = 0; d < 4; ++d) o[d] = mfma32(x[d], p[r], o[d]);
      }
    } else {
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        Op w[kWeightTerms];
#pragma unroll
        for (int i = 0; i < 8; i += 2) {
          f32x2t y = {p[8 * t + i], p[8 * t + i + 1]};
#pragma unroll
          for (int u = 0; u < kWeightTerms; ++u) {
            if constexpr (std::is_same<Op, bf16x8>::value) {
              const bf16x2t z = __builtin_convertvector(y, bf16x2t);
              w[u][i] = z[0];
              w[u][i + 1] = z[1];
              y[0] -= (float)z[0];
              y[1] -= (float)z[1];
            } else {
              const _Float16 z0 = (_Float16)y[0], z1 = (_Float16)y[1];
              w[u][i] = z0;
              w[u][i + 1] = z1;
              y[0] -= (float)z0;
              y[1] -= (float)z1;
            }
          }
        }
#pragma unroll
        for (int d = 0; d < 4; ++d) {
          const Op a = values(v, t, d, lane);
#pragma unroll
          for (int u = kWeightTerms - 1; u >= 0; --u) o[d] = mfma32(a, w[u], o[d]);
        }
      }
    }
  }
};

// LDS of one workgroup: two stages of kRows rows of K and of V.
template <typename T>
constexpr int stage_bytes(int rows) { return rows * InLds<T>::kRowBytes; }
constexpr int tile_rows(int key_waves) { return key_waves == 4 ? 128 : 64; }
constexpr int kJoinRow = kD + 4;             // floats of a row whose key waves' results are added up in LDS
template <typename TK, typename TV, int kKeyWaves>
constexpr int tile_lds() {
  const int stages = 2 * (stage_bytes<TK>(tile_rows(kKeyWaves)) + stage_bytes<TV>(tile_rows(kKeyWaves))), join = kKeyWaves > 1 ? 4 * 32 * kJoinRow * 4 : 0;
  return stages > join ? stages : join;
}
// Few rows: all four waves share the keys of one tile of 32 rows; two tiles of fp32, whose stages are twice as large.
template <typename T>
constexpr int few_key_waves() { return sizeof(T) == 4 ? 2 : 4; }

// The loop of a workgroup whose four waves are 4 / kKeyWaves rows of waves (32 query rows each) by kKeyWaves (which share a stage's
// keys), over the rows [first, end).  load_q: brings my query row's operand, which nothing waits for until the first rows have been
// asked for.  limit: the keys that my query row sees.
template <typename TK, typename TV, int kKeyWaves, typename Op, int kTerms, typename LoadQ, typename Rows = AllRows>
__device__ __forceinline__ void tile_loop(char* lds, const CacheRows<TK>& K, const CacheRows<TV>& V, int first, int end, LoadQ load_q,
                                          int limit, RowState<Op, kTerms>& st, const Rows& rows = Rows()) {
  constexpr int kRows = tile_rows(kKeyWaves), kBlocks = kRows / 32 / kKeyWaves;
  constexpr int kStageK = stage_bytes<TK>(kRows), kStage = kStageK + stage_bytes<TV>(kRows);
  const int lane = threadIdx.x & 63, n = lane & 31, h = lane >> 5, mine = (wave_of() % kKeyWaves) * kBlocks * 32;
  int most = limit, least = limit;
#pragma unroll
  for (int d = 1; d < 32; d <<= 1) {
    most = max(most, __shfl_xor(most, d));
    least = min(least, __shfl_xor(least, d));
  }
  most = __builtin_amdgcn_readfirstlane(most);
  least = __builtin_amdgcn_readfirstlane(least);
  int begun = 0;                              // from there on none of my wave's rows misses one for its window
  if constexpr (Rows::kGap) {
    begun = rows.from;
#pragma unroll
    for (int d = 1; d < 32; d <<= 1) begun = max(begun, __shfl_xor(begun, d));
    begun = __builtin_amdgcn_readfirstlane(begun);
  }
  lds_char* const stages = (lds_char*)lds;
  StageFeed<TK, kRows / 4, Op> fk;
  StageFeed<TV, kRows / 4, Op> fv;
  typename decltype(fk)::Places pk;
  typename decltype(fv)::Places pv;
  constexpr bool kAlike = sizeof(TK) == sizeof(TV);
  auto look_up = [&](int k) {
    pk.look_up(K, k, end, lane, rows);
    if constexpr (!kAlike) pv.look_up(V, k, end, lane, rows);
  };
  auto ask = [&](int k, int to) {
    pk.aim(K, k, end, lane, rows);
    if constexpr (!kAlike) pv.aim(V, k, end, lane, rows);
    __builtin_amdgcn_sched_barrier(0);
    fk.ask(K, pk.off, stages + to, lane);
    if constexpr (kAlike) fv.ask(V, pk.off, stages + to + kStageK, lane);
    else fv.ask(V, pv.off, stages + to + kStageK, lane);
  };
  auto put = [&](int to) {
    fk.put(stages + to, lane);
    fv.put(stages + to + kStageK, lane);
  };
  look_up(first);
  ask(first, 0);
  if (first + kRows < end) look_up(first + kRows);
  typename RowState<Op, kTerms>::Query q;
  load_q(q);
  put(0);
  int at = 0;
  for (int k0 = first; k0 < end; k0 += kRows, at = kStage - at) {
    const bool more = k0 + kRows < end;
    if constexpr (kKeyWaves == 4) {           // a wave reads the rows that it brings, and no others
      wave_lds_order();
      __builtin_amdgcn_s_waitcnt(0x0070);     // vmcnt(0) lgkmcnt(0): they are in LDS, and the other stage has been read
      wave_lds_order();
    } else {
      __builtin_amdgcn_s_waitcnt(0x0f70);     // vmcnt(0)
      __syncthreads();                        // what all asked for is there; nobody reads the other stage any more
    }
    if (more) {
      ask(k0 + kRows, kStage - at);
      if (k0 + 2 * kRows < end) look_up(k0 + 2 * kRows);
    }
    const char* k = lds + at + mine * InLds<TK>::kRowBytes;
    const char* v = lds + at + kStageK + mine * InLds<TV>::kRowBytes;
#pragma unroll
    for (int b = 0; b < kBlocks; ++b) {
      const int k_mine = k0 + mine + 32 * b;
      if (k_mine < most) {
        f32x16 s[1] = {RowState<Op, kTerms>::scores(k + 32 * b * InLds<TK>::kRowBytes, q, n, h)};
        st.template step<1>(s, v + 32 * b * InLds<TV>::kRowBytes, q.unit, k_mine, limit, k_mine + 32 > least || (Rows::kGap && k_mine < begun), lane, rows);
      }
    }
    if (more) put(kStage - at);
  }
}

// My four channels from the returned one on, of o[d][r .. r + 3] (fp32 operands: of o[0 .. 3][r + d]).
template <typename Op>
__device__ __forceinline__ int four_channels(const f32x16 (&o)[4], int d, int r, int h, f32x4* x) {
  constexpr bool kF32 = std::is_same<Op, float>::value;
#pragma unroll
  for (int i = 0; i < 4; ++i) (*x)[i] = kF32 ? o[i][r + d] : o[d][r + i];
  return kF32 ? 4 * (2 * r + 4 * h + d) : 32 * d + 2 * r + 4 * h;
}

// Where a row's result goes: the output row, or a partial.  Both null: nowhere.
template <typename TO>
struct RowOut {
  TO* out;
  float* part;
};
__device__ __forceinline__ void put2(float* p, f32x2t x) { *reinterpret_cast<f32x2t*>(p) = x; }
__device__ __forceinline__ void put2(uint16_t* p, f32x2t x) { *reinterpret_cast<bf16x2t*>(p) = __builtin_convertvector(x, bf16x2t); }
__device__ __forceinline__ void put2(_Float16* p, f32x2t x) { *reinterpret_cast<f16x2t*>(p) = __builtin_convertvector(x, f16x2t); }
__device__ __forceinline__ void put4(float* p, f32x4 x) { *reinterpret_cast<f32x4*>(p) = x; }
__device__ __forceinline__ void put4(uint16_t* p, f32x4 x) {
  typedef __bf16 bf16x4 __attribute__((ext_vector_type(4)));
  *reinterpret_cast<bf16x4*>(p) = __builtin_convertvector(x, bf16x4);
}
__device__ __forceinline__ void put4(_Float16* p, f32x4 x) {
  typedef _Float16 f16x4 __attribute__((ext_vector_type(4)));
  *reinterpret_cast<f16x4*>(p) = __builtin_convertvector(x, f16x4);
}

// The results of a workgroup's rows, after its loop.  All threads call; `to`: of my query row.  Key waves are added up in LDS first.
template <typename Op, int kTerms, int kKeyWaves, typename TO>
__device__ __forceinline__ void tile_finish(char* lds, RowState<Op, kTerms>& st, RowOut<TO> to) {
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), n = lane & 31, h = lane >> 5;
  st.l += __shfl_xor(st.l, 32);
  if constexpr (kKeyWaves > 1) {
    constexpr int kRow = kJoinRow;
    float* mine = reinterpret_cast<float*>(lds) + (wave * 32 + n) * kRow;
    __syncthreads();                          // (the stages have been read)
#pragma unroll
    for (int d = 0; d < 4; ++d)
#pragma unroll
      for (int r = 0; r < 16; r += 4) {
        f32x4 x;
        const int c = four_channels<Op>(st.o, d, r, h, &x);
        *reinterpret_cast<f32x4*>(mine + c) = x;
      }
    if (h == 0) {
      mine[kD] = st.m;
      mine[kD + 1] = st.l;
    }
    __syncthreads();
    // wave w of its row of waves makes the channel block(s) w * 4 / kKeyWaves ..
    const float* rows = reinterpret_cast<const float*>(lds) + ((wave / kKeyWaves) * kKeyWaves * 32 + n) * kRow;
    float mx = -INFINITY, f[kKeyWaves], ls = 0.f;
#pragma unroll
    for (int w = 0; w < kKeyWaves; ++w) mx = fmaxf(mx, rows[w * 32 * kRow + kD]);
#pragma unroll
    for (int w = 0; w < kKeyWaves; ++w) {
      const float mw = rows[w * 32 * kRow + kD];
      f[w] = mw == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(mw - mx);
      ls = fmaf(rows[w * 32 * kRow + kD + 1], f[w], ls);
    }
    st.m = mx;
    st.l = ls;
    constexpr int kMine = 4 / kKeyWaves;
#pragma unroll
    for (int j = 0; j < kMine; ++j) {
      const int d = (wave % kKeyWaves) * kMine + j;
#pragma unroll
      for (int r = 0; r < 16; r += 4) {
        f32x4 a = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int w = 0; w < kKeyWaves; ++w) {
          const f32x4 x = *reinterpret_cast<const f32x4*>(rows + w * 32 * kRow + 32 * d + 2 * r + 4 * h);
#pragma unroll
          for (int i = 0; i < 4; ++i) a[i] = fmaf(x[i], f[w], a[i]);
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) st.o[j][r + i] = a[i];
      }
    }
  }
  constexpr int kMine = 4 / kKeyWaves;
  const int d0 = (wave % kKeyWaves) * kMine;
  const float inv = st.l == 0.f ? 0.f : 1.f / st.l;
#pragma unroll
  for (int j = 0; j < kMine; ++j)
#pragma unroll
    for (int r = 0; r < 16; r += 4) {
      f32x4 x = {st.o[j][r], st.o[j][r + 1], st.o[j][r + 2], st.o[j][r + 3]};
      int c = 32 * (d0 + j) + 2 * r + 4 * h;
      if constexpr (kKeyWaves == 1) c = four_channels<Op>(st.o, j, r, h, &x);
      if (to.part) put4(to.part + c, x);
      else if (to.out) put4(to.out + c, f32x4{x[0] * inv, x[1] * inv, x[2] * inv, x[3] * inv});
    }
  if (to.part && h == 0 && d0 == 0) {
    to.part[kD] = st.m - RowState<Op, kTerms>::kLift;         // (what the weights are powers of two from)
    to.part[kD + 1] = st.l;
  }
}

// n <= 128 parts of a row joined, by a whole wave, two channels a lane: part i is at(i), with score(i) its largest score in powers of two
// (-inf: it holds nothing) and sum(i) the sum of its weights.  All scores come in one load, a lane a part, and the parts' rows eight at a
// time.  What is not finite in a part shows in the row, also where the part weighs 0, as it does in rows of one part.  (32 lanes a row that walked the parts one by one: 17.8 us for 17 parts of 160 rows.)
template <typename At, typename Score, typename Sum>
__device__ __forceinline__ f32x2t join_parts(int n, At at, Score score, Sum sum) {
  const int lane = threadIdx.x & 63;
  float m[2], f[2], l = 0.f;
  constexpr int kU = 8;
  f32x2t x[kU], a = {0.f, 0.f};
  auto fetch = [&](int i0) {
#pragma unroll
    for (int u = 0; u < kU; ++u) x[u] = *reinterpret_cast<const f32x2t*>(at(i0 + u < n ? i0 + u : n - 1) + 2 * lane);
  };
  fetch(0);
#pragma unroll
  for (int j = 0; j < 2; ++j) {
    const int i = lane + 64 * j < n ? lane + 64 * j : n - 1;
    m[j] = lane + 64 * j < n ? score(i) : -INFINITY;
    f[j] = lane + 64 * j < n ? sum(i) : 0.f;
  }
  float mx = fmaxf(m[0], m[1]);
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) mx = fmaxf(mx, __shfl_xor(mx, d));
#pragma unroll
  for (int j = 0; j < 2; ++j) {
    // (no score: nothing was seen, or all that was is NaN, and then so is the sum)
    const float w = f[j] != f[j] ? NAN : (m[j] == -INFINITY ? 0.f : __builtin_amdgcn_exp2f(m[j] - mx));
    l += w > 0.f || w != w ? w * f[j] : 0.f;
    f[j] = w;
  }
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) l += __shfl_xor(l, d);
  for (int i0 = 0;;) {
#pragma unroll
    for (int u = 0; u < kU; ++u) {
      const int i = i0 + u;
      if (i < n) {
        const float w = __int_as_float(__builtin_amdgcn_readlane(__float_as_int(i < 64 ? f[0] : f[1]), i & 63));
        a[0] = fmaf(x[u][0], w, a[0]);
        a[1] = fmaf(x[u][1], w, a[1]);
      }
    }
    i0 += kU;
    if (i0 >= n) break;
    fetch(i0);
  }
  const float inv = l == 0.f ? 0.f : 1.f / l;
  return f32x2t{a[0] * inv, a[1] * inv};
}

// Part `split` of n of the rows [first, end): whole stages.
__device__ __forceinline__ void split_rows(int first, int end, int n, int split, int stage, int* lo, int* hi) {
  int per = (end - first + n - 1) / n;
  per = (per + stage - 1) / stage * stage;
  per = per < stage ? stage : per;
  const int64_t at = first + (int64_t)split * per;
  *lo = at < end ? (int)at : end;
  *hi = at + per < end ? (int)(at + per) : end;
}

}  // namespace lfps
