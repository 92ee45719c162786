// The newest rows of every request into its cache: token i of the t_b packed tokens of request b becomes row n_b - t_b + i.  A
// copy of t_b * Hkv rows of K and of V, from rows with a stride of their own (slices of a fused projection) to wherever the
// cache has them; FP8 caches convert, to nearest even, values beyond +-448 (infinities too) to +-448, NaN to NaN.  Bound by the
// bytes; a decode step's call by its latency: 32 tokens of 8 heads into FP8 pages 3.7 us, 25776 tokens of 8 heads in bf16 (211 MB read and
// written) 37 us, 5.7 TB/s.
#include "stored_rows.h"
#include "tile_attn.h"

namespace lfps {

// 16 lanes a (token, KV head), 8 channels a lane
template <typename TS, typename TK, typename TV>
__global__ __launch_bounds__(256) void k_append(Shape s, KvView kv, const TS* __restrict__ k_new, const TS* __restrict__ v_new, int64_t stride_t,
                                                const int32_t* __restrict__ cu, int n_tokens) {
  request_arguments<decltype(&k_append<TS, TK, TV>)>();
  const int64_t x = (int64_t)blockIdx.x * 16 + (threadIdx.x >> 4);
  const int g = (int)(x % s.Hkv), c = 8 * (threadIdx.x & 15);
  const int64_t token = x / s.Hkv;
  // the request of the wave's first row; the others' are it or follow
  const int64_t wave_token = ((int64_t)blockIdx.x * 16 + (threadIdx.x >> 6) * 4) / s.Hkv;
  int b = last_not_above(s.B - 1, __builtin_amdgcn_readfirstlane((int)(wave_token < n_tokens ? wave_token : n_tokens - 1)), [&](int i) { return cu[i]; });
  if (token >= n_tokens) return;
  const int t = (int)token;
  while (b + 1 < s.B && cu[b + 1] <= t) ++b;
  int c0, c1;
  request_tokens(cu, n_tokens, b, &c0, &c1);
  if (t < c0 || t >= c1) return;
  int n = kv.seq_lens[b];
  n = n < 0 ? 0 : (n > s.Lcap ? s.Lcap : n);
  const int64_t row = (int64_t)n - c1 + t;                   // (c1 > t: below n)
  if (row < 0) return;
  const int64_t from = token * stride_t + g * kD + c;
  const CacheRows<TK> K(kv.k, kv, b, g);
  const CacheRows<TV> V(kv.v, kv, b, g);
  const int e = K.entry((int)row);
  if (kv.page.table && (uint32_t)e >= (uint32_t)kv.page.n_blocks) return;       // (readers clamp; a write would be into someone's block)
  Convert8<TS, TK>::move(k_new + from, const_cast<TK*>(K.at((int)row, e)) + c);
  Convert8<TS, TV>::move(v_new + from, const_cast<TV*>(V.at((int)row, e)) + c);
}

hipError_t launch_append(const Shape& s, int dtype, const KvView& kv, const void* k_new, const void* v_new, int64_t stride_t,
                         const int32_t* cu, int n_tokens, hipStream_t st) {
  const dim3 grid((unsigned)(((int64_t)n_tokens * s.Hkv + 15) / 16));
#define LFPS_APPEND(TS, TK, TV) \
  hipLaunchKernelGGL((k_append<TS, TK, TV>), grid, dim3(256), 0, st, s, kv, (const TS*)k_new, (const TS*)v_new, stride_t, cu, n_tokens)
  if (dtype == LFPS_F32) LFPS_APPEND(float, float, float);
  else if (dtype == LFPS_F16) LFPS_APPEND(_Float16, _Float16, _Float16);
  else if (kv.k_fp8 && kv.v_fp8) LFPS_APPEND(uint16_t, uint8_t, uint8_t);
  else if (kv.k_fp8) LFPS_APPEND(uint16_t, uint8_t, uint16_t);
  else if (kv.v_fp8) LFPS_APPEND(uint16_t, uint16_t, uint8_t);
  else LFPS_APPEND(uint16_t, uint16_t, uint16_t);
#undef LFPS_APPEND
  return hipGetLastError();
}

}  // namespace lfps
