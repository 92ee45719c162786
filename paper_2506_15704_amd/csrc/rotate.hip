// The newest tokens' heads between the projection and the attention: every query and key head is brought to unit mean square
// (y = x / sqrt(mean x^2 + eps) * w), its first channels are turned in pairs by the angles that the token's position gives
// ((a, b) -> (a cos - b sin, b cos + a sin), angle = position[axis of the pair] * frequency of the pair), and keys and values go into the
// cache as lfps_append puts them there, each value rounded once.
//
// An angle is reduced in 64 bits: position * frequency (up to 55 bits) as a product and its rounding error, and of it / 2 pi whole turns taken off before
// the product is rounded, then the nearest quarter turn before it becomes fp32, so that a position of 2^31 is turned as exactly as one of 16; the sine
// and cosine of what is left, at most pi / 4, are their Taylor sums.  A wave has a token's angles, made by a lane a pair, and serves eight or sixteen of its head rows; other
// waves make them again.
//
// Bound by the bytes: eight prompts of 1000 to 6000 tokens, 32 + 16 heads in bf16, 0.63 GB in and out, 116 us, 5.4 TB/s (a large copy reaches 5.0; part
// of the bytes stay in the memory-side cache); 0.30 GB in fp16 57 us, 5.3.  32 single tokens 4.1 us in the kernel, 10.5 with the call.
#include "stored_rows.h"
#include "tile_attn.h"

namespace lfps {

namespace {

// 2 pi * turns -> cosine and sine
__device__ __forceinline__ f32x2t turn(int position, float frequency) {
  constexpr double kHi = 0.15915494309189535, kLo = -9.8393381857794e-18;      // 1 / (2 pi)
  const double p = (double)position * (double)frequency, rest = fma((double)position, (double)frequency, -p);
  double f = fma(p, kHi, -__builtin_rint(p * kHi)) + fma(p, kLo, rest * kHi);
  const double quarter = __builtin_rint(4.0 * f);
  f -= 0.25 * quarter;
  const float y = (float)(f * 6.283185307179586), z = y * y;
  const float s = y * fmaf(z, fmaf(z, fmaf(z, fmaf(z, 1.f / 362880.f, -1.f / 5040.f), 1.f / 120.f), -1.f / 6.f), 1.f);
  const float c = fmaf(z, fmaf(z, fmaf(z, fmaf(z, fmaf(z, -1.f / 3628800.f, 1.f / 40320.f), -1.f / 720.f), 1.f / 24.f), -0.5f), 1.f);
  const int k = (int)quarter;
  const float a = k & 1 ? -s : c, b = k & 1 ? c : s;
  return k & 2 ? f32x2t{-a, -b} : f32x2t{a, b};
}

// The sum over the eight lanes of a row, in each of them.
__device__ __forceinline__ float row8_sum(float x) {
#define LFPS_DPP(v, ctrl) __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), ctrl, 0xf, 0xf, false))
  x += LFPS_DPP(x, 0xB1);     // quad_perm 1 0 3 2
  x += LFPS_DPP(x, 0x4E);     // quad_perm 2 3 0 1
  x += LFPS_DPP(x, 0x141);    // row_half_mirror
#undef LFPS_DPP
  return x;
}

template <typename TS>
struct RotateArgs {
  Shape s;
  KvView kv;
  Rotary rot;
  const TS *q, *k_new, *v_new;
  int64_t stride_t;
  const int32_t *positions, *cu;
  int32_t n_tokens, waves;       // waves of a token
  void* q_out;
};

}  // namespace

// A wave has a token, eight of its Hq + 2 Hkv head rows at a time: eight lanes a row, eight pairs a lane.  kNext: pair i is the channels
// 2 i and 2 i + 1; else i and i + rotary_dim / 2, and the channels behind the turned ones are taken in such pairs too.
template <typename TS, typename TK, typename TV, typename TQ, bool kNext>
__global__ __launch_bounds__(256) void k_rotate_append(RotateArgs<TS> a) {
  request_arguments<decltype(&k_rotate_append<TS, TK, TV, TQ, kNext>)>();
  __shared__ f32x2t turns[4][64];
  const Shape& s = a.s;
  const int lane = threadIdx.x & 63, wave = wave_of(), l = lane & 7;
  const int64_t x = (int64_t)blockIdx.x * 4 + wave;
  if (x >= (int64_t)a.n_tokens * a.waves) return;
  const int token = __builtin_amdgcn_readfirstlane((int)(x / a.waves)), part = (int)(x % a.waves);
  const int b = last_not_above(s.B - 1, token, [&](int i) { return a.cu[i]; });
  int c0, c1;
  request_tokens(a.cu, a.n_tokens, b, &c0, &c1);
  if (token < c0 || token >= c1) return;
  const int row = length_of(s, a.kv.seq_lens, b) - c1 + token;
  const int half = a.rot.rotary_dim / 2;
  if (lane < half) {
    int axis = a.rot.pair_axis ? a.rot.pair_axis[lane] : 0;
    axis = axis < 0 ? 0 : (axis >= a.rot.n_axes ? a.rot.n_axes - 1 : axis);
    turns[wave][lane] = turn(a.positions ? a.positions[(int64_t)axis * a.n_tokens + token] : row, a.rot.inv_freq[lane]);
  }
  wave_lds_order();
  const bool turned = 8 * l < half;
  f32x2t t[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) t[e] = turns[wave][8 * l + e];
  const int at0 = kNext ? 16 * l : (turned ? 8 * l : 8 * l + half), at1 = kNext ? 16 * l + 8 : (turned ? 8 * l + half : 8 * l + 64);
  const int rows = s.Hq + 2 * s.Hkv;
  for (int h = 8 * part + (lane >> 3); h < rows; h += 8 * a.waves) {
    const int kind = h < s.Hq ? 0 : (h < s.Hq + s.Hkv ? 1 : 2), head = kind == 0 ? h : (h - s.Hq) % s.Hkv;
    const TS* const from = (kind == 0 ? a.q : (kind == 1 ? a.k_new : a.v_new)) + (int64_t)token * a.stride_t + head * kD;
    float y[2][8];
    load8(from + at0, y[0]);
    load8(from + at1, y[1]);
    const float* const weight = kind == 0 ? a.rot.q_weight : (kind == 1 ? a.rot.k_weight : nullptr);
    if (weight) {
      float sum = 0.f;
#pragma unroll
      for (int e = 0; e < 8; ++e) sum = fmaf(y[0][e], y[0][e], fmaf(y[1][e], y[1][e], sum));
      sum = row8_sum(sum);
      const float unit = 1.f / sqrtf(fmaf(sum, 1.f / kD, a.rot.eps));
      float w[2][8];
      load8(weight + at0, w[0]);
      load8(weight + at1, w[1]);
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        y[0][e] = y[0][e] * unit * w[0][e];
        y[1][e] = y[1][e] * unit * w[1][e];
      }
    }
    if (turned && kind < 2) {
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        float& p = kNext ? y[e / 4][e % 4 * 2] : y[0][e];
        float& r = kNext ? y[e / 4][e % 4 * 2 + 1] : y[1][e];
        const float u = p, v = r;
        p = u * t[e][0] - v * t[e][1];
        r = fmaf(v, t[e][0], u * t[e][1]);
      }
    }
    if (kind == 0) {
      if (row < 0) {
#pragma unroll
        for (int e = 0; e < 8; ++e) y[0][e] = y[1][e] = 0.f;
      }
      TQ* const to = (TQ*)a.q_out + ((int64_t)token * s.Hq + head) * kD;
      store8(to + at0, y[0]);
      store8(to + at1, y[1]);
    } else if (row >= 0) {
      const CacheRows<TK> K(a.kv.k, a.kv, b, head);
      const CacheRows<TV> V(a.kv.v, a.kv, b, head);
      const int e = K.entry(row);
      if (a.kv.page.table && (uint32_t)e >= (uint32_t)a.kv.page.n_blocks) continue;       // (as in lfps_append)
      if (kind == 1) {
        TK* const to = const_cast<TK*>(K.at(row, e));
        store8(to + at0, y[0]);
        store8(to + at1, y[1]);
      } else {
        TV* const to = const_cast<TV*>(V.at(row, e));
        Convert8<TS, TV>::move(from + at0, to + at0);
        Convert8<TS, TV>::move(from + at1, to + at1);
      }
    }
  }
}

template <typename TS, typename TK, typename TV, typename TQ>
static hipError_t rotate_t(const RotateArgs<TS>& a, hipStream_t st) {
  const dim3 grid((unsigned)(((int64_t)a.n_tokens * a.waves + 3) / 4));
  if (a.rot.interleaved) hipLaunchKernelGGL((k_rotate_append<TS, TK, TV, TQ, true>), grid, dim3(256), 0, st, a);
  else hipLaunchKernelGGL((k_rotate_append<TS, TK, TV, TQ, false>), grid, dim3(256), 0, st, a);
  return hipGetLastError();
}

hipError_t launch_rotate_append(const Shape& s, int dtype, const KvView& kv, const Rotary& rot, const void* q, const void* k_new, const void* v_new,
                                int64_t stride_t, const int32_t* positions, const int32_t* cu, int n_tokens, void* q_out, bool q_f32, hipStream_t st) {
  // A wave takes eight rows, or sixteen where that leaves as many waves as the chip holds (8192) and an element is not four bytes wide.  us by graphs,
  // eight / sixteen, 32 + 16 heads: bf16 64 tokens 3.4 / 4.0, 1024 6.6 / 6.5, 2048 11.3 / 10.0, 4096 19.6 / 17.5, 16384 79.2 / 76.4; FP8 cache
  // 2048 11.5 / 10.2, 16384 78 / 71.3; fp32 2048 18.0 / 18.0, 16384 147 / 153; all 48 rows: bf16 64 tokens 6.3, 4096 18.1, 16384 81.
  const int blocks = (s.Hq + 2 * s.Hkv + 7) / 8;
  const int waves = dtype != LFPS_F32 && (int64_t)n_tokens * blocks >= 8192 ? (blocks + 1) / 2 : blocks;
#define LFPS_ROTATE(TS, TK, TV)                                                                                                   \
  do {                                                                                                                            \
    const RotateArgs<TS> a = {s, kv, rot, (const TS*)q, (const TS*)k_new, (const TS*)v_new, stride_t, positions, cu, n_tokens, waves, q_out}; \
    return q_f32 ? rotate_t<TS, TK, TV, float>(a, st) : rotate_t<TS, TK, TV, TS>(a, st);                                          \
  } while (0)
  if (dtype == LFPS_F32) LFPS_ROTATE(float, float, float);
  if (dtype == LFPS_F16) LFPS_ROTATE(_Float16, _Float16, _Float16);
  if (kv.k_fp8 && kv.v_fp8) LFPS_ROTATE(uint16_t, uint8_t, uint8_t);
  if (kv.k_fp8) LFPS_ROTATE(uint16_t, uint8_t, uint16_t);
  if (kv.v_fp8) LFPS_ROTATE(uint16_t, uint16_t, uint8_t);
  LFPS_ROTATE(uint16_t, uint16_t, uint16_t);
#undef LFPS_ROTATE
}

}  // namespace lfps
