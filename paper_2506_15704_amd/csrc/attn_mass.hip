// Accumulated attention weight: what the newest tokens of a request, packed, give every row of its cache, summed over them and the heads of a KV group,
//
//   mass[b, g, j] = (j < held_b ? decay * mass[b, g, j] : 0) + sum_{t, h in g} softmax_j(q[t, h] . K[b, g, j] / sqrt(D)).
//
// A weight needs the sum over its whole row, so the products are made twice, on the matrix units: k_mass_stats finds every query row's largest score
// and sum, k_mass_add the weights.  Scores are made as S^T = K Q^T in both: a lane has one query row and 16 of 32 keys.  In the first kernel a wave keeps
// its query rows in registers while the keys stream through LDS, and a lane the maximum and sum of its own keys; in the second a wave keeps its keys
// while the queries stream, and a lane the sum of its own queries' weights for each key.  So either reduces over lanes once, at the end, and the sums
// come in the same order every time.
#include "tile_attn.h"

namespace lfps {

namespace {

constexpr int kMassThreads = 256, kMassStage = 64;     // keys or query rows of a stage
constexpr float kMassLazy = 6.f;                       // growth of a maximum, in powers of two, that is let pass

// Blocks of 32 rows that a wave keeps in registers: of 16-bit operands two, so that a row read from LDS serves two products.
template <typename Op>
constexpr int mass_blocks() { return std::is_same<Op, float>::value ? 1 : 2; }
template <typename Op>
constexpr int mass_rows() { return 4 * 32 * mass_blocks<Op>(); }        // of a workgroup

template <typename TQ>
struct MassArgs {
  Shape s;
  KvView kv;
  const TQ* q;
  int64_t q_stride;
  const int32_t *cu, *held;
  int32_t n_tokens, t0, t1;        // the tokens of this launch
  float decay;
  float* stats;                    // [t1 - t0, Hq, splits, 2] of a query row: its largest score in powers of two, the sum of the weights from there; whole
                                   // rows (one split): the sum's inverse
  int32_t splits;
  float* mass;
};

// A row's 128 channels as the operands of lane (n, h): of step s the chunk 16 s + 8 h .. + 7, of fp32 the channels 8 s + 4 h .. + 3.
template <typename Op>
struct MassRow {
  Op x[8];
  template <typename T>
  __device__ __forceinline__ void load(const T* p, int h) {
#pragma unroll
    for (int s = 0; s < 8; ++s) {
      if constexpr (sizeof(T) == 1) {
        const u32x2 w = *reinterpret_cast<const u32x2*>(p + 16 * s + 8 * h);
        x[s] = fp8x8_to<Op>(w[0], w[1]);
      } else {
        x[s] = *reinterpret_cast<const Op*>(p + 16 * s + 8 * h);
      }
    }
  }
};
template <>
struct MassRow<float> {
  f32x4 x[16];
  __device__ __forceinline__ void load(const float* p, int h) {
#pragma unroll
    for (int s = 0; s < 16; ++s) x[s] = *reinterpret_cast<const f32x4*>(p + 8 * s + 4 * h);
  }
};

// out[i] = 32 rows in LDS times my block i, or with kLdsIsKeys = false my blocks times the rows in LDS (keys are the first operand).
template <bool kLdsIsKeys, typename Op, int kBlocks>
__device__ __forceinline__ void mass_scores(f32x16 (&out)[kBlocks], const lds_char* rows, const MassRow<Op> (&mine)[kBlocks], int n, int h) {
#pragma unroll
  for (int i = 0; i < kBlocks; ++i) out[i] = zeros16();
  if constexpr (std::is_same<Op, float>::value) {
#pragma unroll
    for (int c = 0; c < 16; ++c) {
      const f32x4 a = *(const __attribute__((address_space(3))) f32x4*)(rows + n * 512 + 16 * chunk_place_f32(n, 2 * c + h));
#pragma unroll
      for (int e = 0; e < 4; ++e)
#pragma unroll
        for (int i = 0; i < kBlocks; ++i)
          out[i] = kLdsIsKeys ? mfma32(a[e], mine[i].x[c][e], out[i]) : mfma32(mine[i].x[c][e], a[e], out[i]);
    }
  } else {
#pragma unroll
    for (int c = 0; c < 8; ++c) {
      const Op a = *(const __attribute__((address_space(3))) Op*)(rows + n * 256 + 16 * chunk_place(n, 2 * c + h));
#pragma unroll
      for (int i = 0; i < kBlocks; ++i) out[i] = kLdsIsKeys ? mfma32(a, mine[i].x[c], out[i]) : mfma32(mine[i].x[c], a, out[i]);
    }
  }
}

constexpr float kMassUnit = kLog2e * 0.08838834764831845f;      // from products to scores in powers of two
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

// grid Hkv * splits * tiles (of mass_rows query rows; at most T G / rows + B), the latest rows first: they see most
template <typename TK, typename TQ>
__global__ __launch_bounds__(kMassThreads, sizeof(TK) == 4 ? 1 : 2) void k_mass_stats(MassArgs<TQ> a, int tiles) {
  typedef typename InLds<TQ>::Op Op;
  constexpr int kBlocks = mass_blocks<Op>(), kRows = mass_rows<Op>(), kBytes = kMassStage * InLds<TQ>::kRowBytes;
  __shared__ __attribute__((aligned(16))) char lds_[2 * kBytes];
  const Shape& s = a.s;
  const int G = s.G, shift = G == 4 ? 2 : G - 1, per = kRows / G;
  const int g = blockIdx.x % s.Hkv, x0 = blockIdx.x / s.Hkv, split = x0 % a.splits, x = tiles - 1 - x0 / a.splits;
  auto first_tile = [&](int i) {
    const int c = a.cu[i];
    return ((c < a.t0 ? a.t0 : (c > a.t1 ? a.t1 : c)) - a.t0) / per + i;
  };
  const int b = last_not_above(s.B - 1, x, first_tile);
  int c0, c1;
  const int first = launch_tokens(a, b, &c0, &c1);
  const int row0 = (x - first_tile(b)) * kRows, rows = c1 > c0 ? (c1 - c0) << shift : 0;
  if (row0 < 0 || row0 >= rows) return;
  const int lane = threadIdx.x & 63, wave = wave_of(), n = lane & 31, h = lane >> 5;
  auto seen = [&](int m) {                                     // keys that query row m sees
    const int y = first + c0 + (m >> shift) + 1;
    return y < 0 ? 0 : y;
  };
  const int last = (row0 + kRows < rows ? row0 + kRows : rows) - 1;
  int lo, hi;
  split_rows(0, seen(last), a.splits, split, kMassStage, &lo, &hi);
  const int mine0 = row0 + 32 * kBlocks * wave;
  int m[kBlocks], limit[kBlocks];
  MassRow<Op> q[kBlocks];
#pragma unroll
  for (int i = 0; i < kBlocks; ++i) {
    m[i] = mine0 + 32 * i + n;
    limit[i] = m[i] < rows ? seen(m[i]) : 0;
  }
  const int least = mine0 + 32 * kBlocks <= rows ? seen(mine0) : 0;      // keys that all of my rows see, and that any does
  const int most = mine0 < rows ? seen(mine0 + 32 * kBlocks - 1 < last ? mine0 + 32 * kBlocks - 1 : last) : 0;
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
    StageFeed<TK, kMassStage / 4, Op> feed;
    typename decltype(feed)::Places at;
    at.look_up(K, lo, hi, lane);
    at.aim(K, lo, hi, lane);
    feed.ask(K, at.off, lds, lane);
    if (lo + kMassStage < hi) at.look_up(K, lo + kMassStage, hi, lane);
#pragma unroll
    for (int i = 0; i < kBlocks; ++i) {
      const int token = c0 + ((m[i] < rows ? m[i] : rows - 1) >> shift);
      q[i].load(a.q + (int64_t)token * a.q_stride + (g * G + (m[i] & (G - 1))) * kD, h);
    }
    feed.put(lds, lane);
    int now = 0;
    for (int k0 = lo; k0 < hi; k0 += kMassStage, now = kBytes - now) {
      const bool more = k0 + kMassStage < hi;
      __builtin_amdgcn_s_waitcnt(0x0f70);                      // vmcnt(0)
      __syncthreads();                                         // what all asked for is there; nobody reads the other stage any more
      if (more) {
        at.aim(K, k0 + kMassStage, hi, lane);
        feed.ask(K, at.off, lds + kBytes - now, lane);
        if (k0 + 2 * kMassStage < hi) at.look_up(K, k0 + 2 * kMassStage, hi, lane);
      }
#pragma unroll
      for (int kb = 0; kb < kMassStage / 32; ++kb) {
        const int key0 = k0 + 32 * kb;
        if (key0 < most) {
          f32x16 y[kBlocks];
          mass_scores<true, Op, kBlocks>(y, lds + now + 32 * kb * InLds<TQ>::kRowBytes, q, n, h);
#pragma unroll
          for (int i = 0; i < kBlocks; ++i) {
            if (key0 + 32 > least || key0 + 32 > hi) {
              const int end = limit[i] < hi ? limit[i] : hi;
#pragma unroll
              for (int r = 0; r < 16; ++r) y[i][r] = key0 + key_of(r, h) < end ? y[i][r] : -INFINITY;
            }
            float mx = fmaxf(y[i][0], y[i][1]);
#pragma unroll
            for (int r = 2; r < 16; r += 2) mx = fmaxf(fmaxf(mx, y[i][r]), y[i][r + 1]);
            mx *= kMassUnit;
            const float now_top = mx > top[i] + kMassLazy ? mx : top[i];
            if (__ballot(now_top != top[i])) {
              const float shrink = now_top == top[i] ? 1.f : __builtin_amdgcn_exp2f(top[i] - now_top);
#pragma unroll
              for (int e = 0; e < 4; ++e) l[i][e] *= shrink;
              top[i] = now_top;
            }
            const float from = top[i] == -INFINITY ? 0.f : top[i];
#pragma unroll
            for (int r = 0; r < 16; ++r) l[i][r % 4] += __builtin_amdgcn_exp2f(fmaf(y[i][r], kMassUnit, -from));
          }
        }
      }
      if (more) feed.put(lds + kBytes - now, lane);
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
      float* const to = a.stats + (((int64_t)(c0 - a.t0 + (m[i] >> shift)) * s.Hq + g * G + (m[i] & (G - 1))) * a.splits + split) * 2;
      const bool whole = a.splits == 1;
      *reinterpret_cast<f32x2t*>(to) = f32x2t{whole && mx == -INFINITY ? 0.f : mx, whole ? (both == 0.f ? 0.f : 1.f / both) : both};
    }
  }
}

// The parts of a query row -> its first part's place, as of one part.
__global__ __launch_bounds__(256) void k_mass_join(float* __restrict__ stats, int64_t rows, int splits) {
  const int64_t x = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (x >= rows) return;
  const f32x2t* const part = reinterpret_cast<const f32x2t*>(stats) + x * splits;
  float mx = -INFINITY, sum = 0.f;
  for (int i = 0; i < splits; ++i) mx = fmaxf(mx, part[i][0]);
  for (int i = 0; i < splits; ++i) {
    const float y = part[i][1];
    sum += y != y ? y : (part[i][0] == -INFINITY ? 0.f : y * __builtin_amdgcn_exp2f(part[i][0] - mx));
  }
  *reinterpret_cast<f32x2t*>(stats + x * splits * 2) = f32x2t{mx == -INFINITY ? 0.f : mx, sum == 0.f ? 0.f : 1.f / sum};
}

// grid (tiles of mass_rows keys, B * Hkv): the first ones are seen by most
template <typename TK, typename TQ>
__global__ __launch_bounds__(kMassThreads, sizeof(TK) == 4 ? 1 : 2) void k_mass_add(MassArgs<TQ> a) {
  typedef typename InLds<TQ>::Op Op;
  constexpr int kBlocks = mass_blocks<Op>(), kKeys = mass_rows<Op>(), kRowBytes = InLds<TQ>::kRowBytes, kBytes = kMassStage * kRowBytes;
  __shared__ __attribute__((aligned(16))) char lds_[2 * kBytes];
  __shared__ float sums[4][32 * kBlocks];
  const Shape& s = a.s;
  const int G = s.G, shift = G == 4 ? 2 : G - 1;
  const int bg = blockIdx.y, b = bg / s.Hkv, g = bg % s.Hkv, tile = blockIdx.x * kKeys, len = length_of(s, a.kv.seq_lens, b);
  if (tile >= len) return;
  const int lane = threadIdx.x & 63, wave = wave_of(), n = lane & 31, h = lane >> 5;
  int c0, c1;
  const int first = launch_tokens(a, b, &c0, &c1);
  const int rows = c1 > c0 ? (c1 - c0) << shift : 0;
  int from = tile - (first + c0);                              // the first token that sees a key of the tile
  from = from < 0 ? 0 : from;
  const int key0 = tile + 32 * kBlocks * wave;
  float sum[kBlocks][16];
#pragma unroll
  for (int i = 0; i < kBlocks; ++i)
#pragma unroll
    for (int r = 0; r < 16; ++r) sum[i][r] = 0.f;
  const int m0 = (from << shift) & ~(kMassStage - 1);
  if (m0 < rows) {
    lds_char* const lds = (lds_char*)lds_;
    // a stage of query rows: 1 KB an instruction, lane l fills the l-th 16 bytes of it with the chunk that belongs there
    constexpr int kPieces = kRowBytes / 16, kEach = 64 / kPieces, kLoads = kMassStage / 4 / kEach;
    auto ask = [&](int m, lds_char* stage) {
#pragma unroll
      for (int i = 0; i < kLoads; ++i) {
        const int r = kMassStage / 4 * wave + kEach * i + lane / kPieces, place = lane % kPieces;
        const int row = m + r < rows ? m + r : rows - 1;
        const char* const p = reinterpret_cast<const char*>(a.q + (int64_t)(c0 + (row >> shift)) * a.q_stride + (g * G + (row & (G - 1))) * kD) +
                              16 * (sizeof(TQ) == 4 ? chunk_place_f32(r, place) : chunk_place(r, place));
        __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) char*)p,
                                         (__attribute__((address_space(3))) void*)(stage + (kMassStage / 4 * wave + kEach * i) * kRowBytes), 16, 0, 0);
      }
    };
    constexpr int kSubs = kMassStage / 32;
    f32x2t st[kSubs], next[kSubs];                             // of my query rows of a stage
    auto stats = [&](int m, f32x2t (&to)[kSubs]) {
#pragma unroll
      for (int i = 0; i < kSubs; ++i) {
        const int row = m + 32 * i + n < rows ? m + 32 * i + n : rows - 1;
        to[i] = *reinterpret_cast<const f32x2t*>(a.stats + ((int64_t)(c0 - a.t0 + (row >> shift)) * s.Hq + g * G + (row & (G - 1))) * a.splits * 2);
      }
    };
    ask(m0, lds);
    stats(m0, next);
    const CacheRows<TK> K(a.kv.k, a.kv, b, g);
    MassRow<Op> k[kBlocks];
#pragma unroll
    for (int i = 0; i < kBlocks; ++i) {
      const int row = key0 + 32 * i + n < len ? key0 + 32 * i + n : len - 1;
      k[i].load(K.at(row, K.entry(row)), h);
    }
    int now = 0;
    for (int m = m0; m < rows; m += kMassStage, now = kBytes - now) {
      __builtin_amdgcn_s_waitcnt(0x0f70);                      // vmcnt(0)
      __syncthreads();
#pragma unroll
      for (int i = 0; i < kSubs; ++i) st[i] = next[i];
      if (m + kMassStage < rows) {
        ask(m + kMassStage, lds + kBytes - now);
        stats(m + kMassStage, next);
      }
      if (key0 >= len) continue;
#pragma unroll
      for (int i = 0; i < kSubs; ++i) {
        const int mi = m + 32 * i;
        const int pos = mi + n < rows ? first + c0 + ((mi + n) >> shift) : -1;      // my query's row
        const int most = first + c0 + ((mi + 31 < rows ? mi + 31 : rows - 1) >> shift);
        if (mi >= rows || most < key0) continue;
        f32x16 y[kBlocks];
        mass_scores<false, Op, kBlocks>(y, lds + now + 32 * i * kRowBytes, k, n, h);
        if (mi + 32 <= rows && first + c0 + (mi >> shift) >= key0 + 32 * kBlocks - 1) {
#pragma unroll
          for (int kb = 0; kb < kBlocks; ++kb)
#pragma unroll
            for (int r = 0; r < 16; ++r) sum[kb][r] = fmaf(__builtin_amdgcn_exp2f(fmaf(y[kb][r], kMassUnit, -st[i][0])), st[i][1], sum[kb][r]);
        } else {
#pragma unroll
          for (int kb = 0; kb < kBlocks; ++kb)
#pragma unroll
            for (int r = 0; r < 16; ++r) {
              const float e = __builtin_amdgcn_exp2f(fmaf(y[kb][r], kMassUnit, -st[i][0])) * st[i][1];
              sum[kb][r] += key0 + 32 * kb + key_of(r, h) <= pos ? e : 0.f;
            }
        }
      }
    }
  }
#pragma unroll
  for (int kb = 0; kb < kBlocks; ++kb)
#pragma unroll
    for (int r = 0; r < 16; ++r) {
      float x = row16_sum(sum[kb][r]);
      x += __shfl_xor(x, 16);
      if (n == 0) sums[wave][32 * kb + key_of(r, h)] = x;
    }
  wave_lds_order();
  const int key = key0 + lane;
  if (lane < 32 * kBlocks && key < len) {
    float* const to = a.mass + (int64_t)bg * s.Lcap + key;
    const int held = a.held ? a.held[b] : 0;
    *to = sums[wave][lane] + (a.t0 > 0 ? *to : (key < held ? a.decay * *to : 0.f));
  }
}

template <typename TK, typename TQ>
static hipError_t mass_t(MassArgs<TQ> a, int64_t room, hipStream_t st) {
  typedef typename InLds<TQ>::Op Op;
  constexpr int kRows = mass_rows<Op>();
  const int64_t most = room / 2 / a.s.Hq;                            // tokens that the workspace has room for
  const int per = kRows / a.s.G;
  const dim3 keys((unsigned)((a.s.Lcap + kRows - 1) / kRows), (unsigned)(a.s.B * a.s.Hkv));
  for (int t0 = 0; t0 == 0 || t0 < a.n_tokens; t0 = a.t1) {           // (also of no tokens: what is held decays)
    a.t0 = t0;
    a.t1 = a.n_tokens - t0 > most ? t0 + (int)most : a.n_tokens;
    const int n = a.t1 - t0, tiles = n / per + a.s.B;
    if (n > 0) {
      const int64_t groups = (int64_t)tiles * a.s.Hkv, rows = (int64_t)n * a.s.Hq, by_len = (a.s.Lcap + 255) / 256;
      int64_t splits = (512 + groups - 1) / groups;
      if (splits * rows * 2 > room) splits = room / 2 / rows;
      if (splits > by_len) splits = by_len;
      a.splits = (int)(splits > kMaxSplits ? kMaxSplits : (splits < 1 ? 1 : splits));
      hipLaunchKernelGGL((k_mass_stats<TK, TQ>), dim3((unsigned)(groups * a.splits)), dim3(kMassThreads), 0, st, a, tiles);
      if (a.splits > 1) hipLaunchKernelGGL(k_mass_join, dim3((unsigned)((rows + 255) / 256)), dim3(256), 0, st, a.stats, rows, a.splits);
    }
    hipLaunchKernelGGL((k_mass_add<TK, TQ>), keys, dim3(kMassThreads), 0, st, a);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess || a.n_tokens == 0) return e;
  }
  return hipSuccess;
}

hipError_t launch_attn_mass(const Shape& s, int dtype, const KvView& kv, const void* q, int64_t q_stride, const int32_t* cu, int n_tokens,
                            const int32_t* held, float decay, float* mass, float* part, int64_t part_rows, hipStream_t st) {
#define LFPS_MASS(TK, TQ)                                                                                                  \
  return mass_t<TK, TQ>(MassArgs<TQ>{s, kv, (const TQ*)q, q_stride, cu, held, n_tokens, 0, 0, decay, part, 1, mass}, part_rows * kPartFloats, st)
  if (dtype == LFPS_F32) LFPS_MASS(float, float);
  if (dtype == LFPS_F16) LFPS_MASS(_Float16, _Float16);
  if (kv.k_fp8) LFPS_MASS(uint8_t, uint16_t);
  LFPS_MASS(uint16_t, uint16_t);
#undef LFPS_MASS
}

}  // namespace lfps
