// Accumulated attention weight: what the newest tokens of a request, packed, give every row of its cache, summed over them and the heads of a KV group,
//
//   mass[b, g, j] = (j < held_b ? decay * mass[b, g, j] : 0) + sum_{t, h in g} softmax_j(q[t, h] . K[b, g, j] / sqrt(D)).
//
// A weight needs the sum over its whole row, so the products are made twice: for the rows' sums, and for the weights.
#include "tile_attn.h"

namespace lfps {

namespace {

template <typename TQ>
struct MassArgs {
  Shape s;
  KvView kv;
  const TQ* q;
  int64_t q_stride;
  const int32_t *cu, *held;        // cu == nullptr: token t is request t's newest row
  int32_t n_tokens, t0, t1;        // the tokens of this launch
  float decay;
  float* stats;                    // [t1 - t0, Hq, 2] of a query row: its largest score, the inverse of the sum of the weights from there
  float* mass;
};

template <typename A>
__device__ __forceinline__ int token_row(const A& a, int b, int token, int* c0, int* c1) {
  if (a.cu) {
    request_tokens(a.cu, a.n_tokens, b, c0, c1);
  } else {
    *c0 = b;
    *c1 = b + 1;
  }
  return length_of(a.s, a.kv.seq_lens, b) - *c1 + token;
}

template <typename TK, typename TQ, int G>
__device__ __forceinline__ void dots(const TK* k, const float (&x)[G][8], float (&y)[G]) {
  float z[8];
  load8(k, z);
#pragma unroll
  for (int h = 0; h < G; ++h) {
    float sum = 0.f;
#pragma unroll
    for (int c = 0; c < 8; ++c) sum = fmaf(x[h][c], z[c], sum);
    y[h] = row16_butterfly_sum(sum);
  }
}
template <typename TQ, int G>
__device__ __forceinline__ void queries(const TQ* q, int j, float (&x)[G][8]) {
#pragma unroll
  for (int h = 0; h < G; ++h) {
    load8(q + h * kD + 8 * j, x[h]);
#pragma unroll
    for (int c = 0; c < 8; ++c) x[h][c] *= 0.08838834764831845f;
  }
}

}  // namespace

// A workgroup has a token and a KV head, 16 lanes of it a row.
template <typename TK, typename TQ, int G>
__global__ __launch_bounds__(256) void k_mass_stats(MassArgs<TQ> a) {
  __shared__ float m_s[16][G], l_s[16][G];
  const Shape& s = a.s;
  const int token = a.t0 + blockIdx.x / s.Hkv, g = blockIdx.x % s.Hkv, j = threadIdx.x & 15, r = threadIdx.x >> 4;
  const int b = a.cu ? last_not_above(s.B - 1, token, [&](int i) { return a.cu[i]; }) : token;
  int c0, c1;
  const int row = token_row(a, b, token, &c0, &c1);
  if (token < c0 || token >= c1) return;
  float x[G][8], m[G], l[G];
  queries<TQ, G>(a.q + token * a.q_stride + g * G * kD, j, x);
#pragma unroll
  for (int h = 0; h < G; ++h) {
    m[h] = -INFINITY;
    l[h] = 0.f;
  }
  const CacheRows<TK> K(a.kv.k, a.kv, b, g);
  for (int i = r; i <= row; i += 16) {
    float y[G];
    dots<TK, TQ, G>(K.at(i, K.entry(i)) + 8 * j, x, y);
#pragma unroll
    for (int h = 0; h < G; ++h) {
      const float mx = fmaxf(m[h], y[h]), from = mx == -INFINITY ? 0.f : mx;
      l[h] = fmaf(l[h], exp_below<false>(m[h] - from), exp_below<false>(y[h] - from));
      m[h] = mx;
    }
  }
  if (j == 0) {
#pragma unroll
    for (int h = 0; h < G; ++h) {
      m_s[r][h] = m[h];
      l_s[r][h] = l[h];
    }
  }
  __syncthreads();
  if (threadIdx.x < G) {
    const int h = threadIdx.x;
    float mx = -INFINITY, sum = 0.f;
    for (int i = 0; i < 16; ++i) mx = fmaxf(mx, m_s[i][h]);
    for (int i = 0; i < 16; ++i) {
      const float w = m_s[i][h] == -INFINITY ? 0.f : exp_below<false>(m_s[i][h] - mx);
      sum += l_s[i][h] != l_s[i][h] || w > 0.f ? w * l_s[i][h] : 0.f;
    }
    float* const to = a.stats + ((int64_t)(token - a.t0) * s.Hq + g * G + h) * 2;
    to[0] = mx == -INFINITY ? 0.f : mx;
    to[1] = sum == 0.f ? 0.f : 1.f / sum;
  }
}

// A workgroup has 16 rows of a request and KV head.
template <typename TK, typename TQ, int G>
__global__ __launch_bounds__(256) void k_mass_add(MassArgs<TQ> a) {
  const Shape& s = a.s;
  const int bg = blockIdx.y, b = bg / s.Hkv, g = bg % s.Hkv, j = threadIdx.x & 15;
  const int at = blockIdx.x * 16 + (threadIdx.x >> 4), n = length_of(s, a.kv.seq_lens, b);
  if (at >= n) return;
  const CacheRows<TK> K(a.kv.k, a.kv, b, g);
  const TK* const k = K.at(at, K.entry(at)) + 8 * j;
  int c0, c1;
  const int first = token_row(a, b, 0, &c0, &c1);              // row of token 0, were it the request's
  int t = at - first;                                          // the first token that sees the row
  t = t < c0 ? c0 : t;
  t = t < a.t0 ? a.t0 : t;
  float sum = 0.f;
  for (const int end = c1 < a.t1 ? c1 : a.t1; t < end; ++t) {
    float x[G][8], y[G];
    queries<TQ, G>(a.q + t * a.q_stride + g * G * kD, j, x);
    dots<TK, TQ, G>(k, x, y);
    const float* const st = a.stats + ((int64_t)(t - a.t0) * s.Hq + g * G) * 2;
#pragma unroll
    for (int h = 0; h < G; ++h) sum = fmaf(exp_below<false>(y[h] - st[2 * h]), st[2 * h + 1], sum);
  }
  if (j == 0) {
    float* const to = a.mass + (int64_t)bg * s.Lcap + at;
    const int held = a.held ? a.held[b] : 0;
    *to = sum + (a.t0 > 0 ? *to : (at < held ? a.decay * *to : 0.f));
  }
}

template <typename TK, typename TQ>
static hipError_t mass_t(MassArgs<TQ> a, int64_t room, hipStream_t st) {
  const int64_t most = room / 2 / a.s.Hq;
  const dim3 rows((unsigned)((a.s.Lcap + 15) / 16), (unsigned)(a.s.B * a.s.Hkv));
  for (int t0 = 0; t0 == 0 || t0 < a.n_tokens; t0 = a.t1) {           // (also of no tokens: what is held decays)
    a.t0 = t0;
    a.t1 = a.n_tokens - t0 > most ? t0 + (int)most : a.n_tokens;
#define LFPS_MASS_G(G)                                                                                             \
  do {                                                                                                             \
    if (a.t1 > t0) hipLaunchKernelGGL((k_mass_stats<TK, TQ, G>), dim3((unsigned)((a.t1 - t0) * a.s.Hkv)), dim3(256), 0, st, a); \
    hipLaunchKernelGGL((k_mass_add<TK, TQ, G>), rows, dim3(256), 0, st, a);                                        \
  } while (0)
    if (a.s.G == 1) LFPS_MASS_G(1);
    else if (a.s.G == 2) LFPS_MASS_G(2);
    else LFPS_MASS_G(4);
#undef LFPS_MASS_G
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess || a.n_tokens == 0) return e;
  }
  return hipSuccess;
}

hipError_t launch_attn_mass(const Shape& s, int dtype, const KvView& kv, const void* q, int64_t q_stride, const int32_t* cu, int n_tokens,
                            const int32_t* held, float decay, float* mass, float* part, int64_t part_rows, hipStream_t st) {
#define LFPS_MASS(TK, TQ)                                                                                                  \
  return mass_t<TK, TQ>(MassArgs<TQ>{s, kv, (const TQ*)q, q_stride, cu, held, n_tokens, 0, 0, decay, part, mass}, part_rows * kPartFloats, st)
  if (dtype == LFPS_F32) LFPS_MASS(float, float);
  if (dtype == LFPS_F16) LFPS_MASS(_Float16, _Float16);
  if (kv.k_fp8) LFPS_MASS(uint8_t, uint16_t);
  LFPS_MASS(uint16_t, uint16_t);
#undef LFPS_MASS
}

hipError_t launch_attn_mass_decode(const Shape& s, int dtype, const KvView& kv, const float* q, const int32_t* held, float decay, float* mass,
                                   float* part, int64_t part_rows, hipStream_t st) {
#define LFPS_MASS(TK)                                                                                                      \
  return mass_t<TK, float>(MassArgs<float>{s, kv, q, (int64_t)s.Hq * kD, nullptr, held, s.B, 0, 0, decay, part, mass}, part_rows * kPartFloats, st)
  if (dtype == LFPS_F32) LFPS_MASS(float);
  if (dtype == LFPS_F16) LFPS_MASS(_Float16);
  if (kv.k_fp8) LFPS_MASS(uint8_t);
  LFPS_MASS(uint16_t);
#undef LFPS_MASS
}

}  // namespace lfps
