// Attention over a sliding window and the first rows: the token at row p sees the rows j <= p with j > p - window or j < n_sink.  The newest
// tokens of every request, packed, and a decode step's single ones.
#include "prompt_tiles.h"

namespace lfps {

namespace {

// Of the rows that a token at row p sees, in order: how many there are, and the i-th.
struct Seen {
  int sinks, lo, count;
  __device__ __forceinline__ Seen(int p, int window, int n_sink) {
    lo = p + 1 > window ? p + 1 - window : 0;
    sinks = n_sink < lo ? n_sink : lo;
    count = p < 0 ? 0 : sinks + p + 1 - lo;
  }
  __device__ __forceinline__ int row(int i) const { return i < sinks ? i : i - sinks + lo; }
};

// Eight fp32, bf16 or fp16 values of a query row.
template <typename TQ>
__device__ __forceinline__ void query8(const TQ* p, float (&x)[8]) { load8(p, x); }

}  // namespace

// A workgroup has a token and a KV head, 16 lanes of it a row, eight channels a lane.  cu == nullptr: token t is request t's newest row.
template <typename TK, typename TV, typename TQ, int G>
__global__ __launch_bounds__(256) void k_window_rows(Shape s, KvView kv, const TQ* __restrict__ q, int64_t q_stride, const int32_t* __restrict__ cu,
                                                     int n_tokens, int window, int n_sink, TQ* __restrict__ out) {
  __shared__ float acc_s[16][G][kD], m_s[16][G], l_s[16][G];
  const int token = blockIdx.x / s.Hkv, g = blockIdx.x % s.Hkv, j = threadIdx.x & 15, r = threadIdx.x >> 4;
  int b = token, row;
  if (cu) {
    b = last_not_above(s.B - 1, token, [&](int i) { return cu[i]; });
    int c0, c1;
    request_tokens(cu, n_tokens, b, &c0, &c1);
    if (token < c0 || token >= c1) return;
    row = length_of(s, kv.seq_lens, b) - c1 + token;
  } else {
    row = length_of(s, kv.seq_lens, b) - 1;
  }
  const Seen seen(row, window, n_sink);
  float x[G][8], acc[G][8], m[G], l[G];
#pragma unroll
  for (int h = 0; h < G; ++h) {
    query8(q + token * q_stride + (g * G + h) * kD + 8 * j, x[h]);
    m[h] = -INFINITY;
    l[h] = 0.f;
#pragma unroll
    for (int c = 0; c < 8; ++c) {
      x[h][c] *= 0.08838834764831845f;
      acc[h][c] = 0.f;
    }
  }
  const CacheRows<TK> K(kv.k, kv, b, g);
  const CacheRows<TV> V(kv.v, kv, b, g);
  for (int i = r; i < seen.count; i += 16) {
    const int at = seen.row(i), e = K.entry(at);
    float k[8], v[8];
    load8(K.at(at, e) + 8 * j, k);
    load8(V.at(at, e) + 8 * j, v);
#pragma unroll
    for (int h = 0; h < G; ++h) {
      float y = 0.f;
#pragma unroll
      for (int c = 0; c < 8; ++c) y = fmaf(x[h][c], k[c], y);
      y = row16_butterfly_sum(y);
      const float mx = fmaxf(m[h], y), from = mx == -INFINITY ? 0.f : mx;
      const float shrink = exp_below<false>(m[h] - from), p = exp_below<false>(y - from);
      m[h] = mx;
      l[h] = fmaf(l[h], shrink, p);
#pragma unroll
      for (int c = 0; c < 8; ++c) acc[h][c] = fmaf(acc[h][c], shrink, p * v[c]);
    }
  }
#pragma unroll
  for (int h = 0; h < G; ++h) {
#pragma unroll
    for (int c = 0; c < 8; ++c) acc_s[r][h][8 * j + c] = acc[h][c];
    if (j == 0) {
      m_s[r][h] = m[h];
      l_s[r][h] = l[h];
    }
  }
  __syncthreads();
  for (int e = threadIdx.x; e < G * kD; e += 256) {
    const int h = e / kD, c = e % kD;
    float mx = -INFINITY, sum = 0.f, y = 0.f;
    for (int i = 0; i < 16; ++i) mx = fmaxf(mx, m_s[i][h]);
    for (int i = 0; i < 16; ++i) {
      const float w = l_s[i][h] != l_s[i][h] ? NAN : (m_s[i][h] == -INFINITY ? 0.f : exp_below<false>(m_s[i][h] - mx));
      sum += w > 0.f || w != w ? w * l_s[i][h] : 0.f;
      y = fmaf(w, acc_s[i][h][c], y);
    }
    y = sum == 0.f ? 0.f : y / sum;
    TQ* const to = out + ((int64_t)token * s.Hq + g * G + h) * kD + c;
    if constexpr (std::is_same<TQ, uint16_t>::value) *reinterpret_cast<__bf16*>(to) = (__bf16)y;
    else *to = (TQ)y;
  }
}

template <typename TK, typename TV, typename TQ>
static hipError_t window_t(const Shape& s, const KvView& kv, const void* q, int64_t q_stride, const int32_t* cu, int n_tokens, int window, int n_sink,
                           void* out, hipStream_t st) {
  const dim3 grid((unsigned)(n_tokens * s.Hkv));
#define LFPS_WINDOW_G(G) \
  hipLaunchKernelGGL((k_window_rows<TK, TV, TQ, G>), grid, dim3(256), 0, st, s, kv, (const TQ*)q, q_stride, cu, n_tokens, window, n_sink, (TQ*)out)
  if (s.G == 1) LFPS_WINDOW_G(1);
  else if (s.G == 2) LFPS_WINDOW_G(2);
  else LFPS_WINDOW_G(4);
#undef LFPS_WINDOW_G
  return hipGetLastError();
}

hipError_t launch_window_attn(const Shape& s, int dtype, const KvView& kv, const void* q, int64_t q_stride, const int32_t* cu, int n_tokens, int window,
                              int n_sink, void* out, float* part, int64_t part_rows, hipStream_t st) {
#define LFPS_WINDOW(TK, TV, TQ) return prompt_t<TK, TV, TQ>(s, kv, SeesWindow{window, n_sink}, q, q_stride, cu, n_tokens, out, part, part_rows, st)
  if (dtype == LFPS_F32) LFPS_WINDOW(float, float, float);
  if (dtype == LFPS_F16) LFPS_WINDOW(_Float16, _Float16, _Float16);
  if (kv.k_fp8 && kv.v_fp8) LFPS_WINDOW(uint8_t, uint8_t, uint16_t);
  if (kv.k_fp8) LFPS_WINDOW(uint8_t, uint16_t, uint16_t);
  if (kv.v_fp8) LFPS_WINDOW(uint16_t, uint8_t, uint16_t);
  LFPS_WINDOW(uint16_t, uint16_t, uint16_t);
#undef LFPS_WINDOW
}

hipError_t launch_window_attn_decode(const Shape& s, int dtype, const KvView& kv, const float* q, int window, int n_sink, float* out, float* part,
                                     int64_t part_rows, hipStream_t st) {
#define LFPS_WINDOW(TK, TV) return window_t<TK, TV, float>(s, kv, q, (int64_t)s.Hq * kD, nullptr, s.B, window, n_sink, out, st)
  if (dtype == LFPS_F32) LFPS_WINDOW(float, float);
  if (dtype == LFPS_F16) LFPS_WINDOW(_Float16, _Float16);
  if (kv.k_fp8 && kv.v_fp8) LFPS_WINDOW(uint8_t, uint8_t);
  if (kv.k_fp8) LFPS_WINDOW(uint8_t, uint16_t);
  if (kv.v_fp8) LFPS_WINDOW(uint16_t, uint8_t);
  LFPS_WINDOW(uint16_t, uint16_t);
#undef LFPS_WINDOW
}

}  // namespace lfps
