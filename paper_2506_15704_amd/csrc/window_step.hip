// A decode step's attention over a window and the first rows: the kernels of the full attention over fewer rows, which count the rows past the gap on,
// and the join of their parts.  Cut by the most rows that a window and the first ones can be, not by the context's.  Bound by the bytes of K and V:
// 32 requests, window 4096, FP8 pages, 0.27 GB 69 us, 3.9 TB/s (with a wave a head and no parts 295).
#include "full_attn.h"

namespace lfps {

// grid B * Hq / 4, a wave a head
template <int G>
__global__ __launch_bounds__(256) void k_window_join(Shape s, const int32_t* __restrict__ seq_lens, const float* __restrict__ part, int n_split,
                                                     WindowRows w, float* __restrict__ out) {
  const int bh = blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  if (bh >= s.B * s.Hq) return;
  const int b = bh / s.Hq, h = bh % s.Hq, g = h / G;
  int at, by, n;
  window_rows(w, length_of(s, seq_lens, b), &at, &by, &n);
  f32x2t y = {0.f, 0.f};
  if (n > 0) {
    const int rps = rows_per_split(n, n_split);
    float from, inverse;
    y = join_head<G>(part + ((int64_t)(b * s.Hkv + g) * n_split) * G * (kD + 2), (n + rps - 1) / rps, h % G, &from, &inverse);
  }
  *reinterpret_cast<f32x2t*>(out + (int64_t)bh * kD + 2 * (threadIdx.x & 63)) = y;
}

template <typename TK, typename T>
static hipError_t window_step_t(const Shape& s, const float* q, const KvView& kv, const WindowRows& w, float* part, float* out, hipStream_t st) {
  const Shape fewer = walked(s, w);
  const int n_split = full_attn_splits(fewer);
  const dim3 grid(n_split, s.B * s.Hkv), block(kAttnThreads), heads((s.B * s.Hq + 3) / 4);
  const float scale = 0.08838834764831845f;
  // (as in the full attention: 16 requests of 16384 rows, bf16 pages, window of all of them 210 -> 184 us)
  const bool once = sizeof(TK) < 4 && (int64_t)s.B * s.Hkv * fewer.Lcap * kD * (int64_t)(sizeof(TK) + sizeof(T)) > kKeptStreamBytes;
#define LFPS_WINDOW_P(KERNEL, PAGED, ONCE, ...)                                                                           \
  hipLaunchKernelGGL((KERNEL<TK, T, ##__VA_ARGS__, PAGED, ONCE, WindowRows>), grid, block, 0, st, s, q, (const TK*)kv.k,  \
                     (const T*)kv.v, kv.stride_b, kv.stride_h, kv.stride_n, kv.page, kv.seq_lens, part, n_split, scale, w)
#define LFPS_WINDOW(G, KERNEL, ...)                                           \
  if (kv.page.table) {                                                        \
    if (once) LFPS_WINDOW_P(KERNEL, true, sizeof(TK) < 4, ##__VA_ARGS__);     \
    else LFPS_WINDOW_P(KERNEL, true, false, ##__VA_ARGS__);                   \
  } else {                                                                    \
    if (once) LFPS_WINDOW_P(KERNEL, false, sizeof(TK) < 4, ##__VA_ARGS__);    \
    else LFPS_WINDOW_P(KERNEL, false, false, ##__VA_ARGS__);                  \
  }                                                                           \
  hipLaunchKernelGGL((k_window_join<G>), heads, dim3(256), 0, st, s, kv.seq_lens, part, n_split, w, out)
  switch (s.G) {
    case 1: LFPS_WINDOW(1, k_full_attn_single); break;
    case 2: LFPS_WINDOW(2, k_full_attn, 2); break;
    case 4: LFPS_WINDOW(4, k_full_attn, 4); break;
    default: return hipErrorInvalidValue;
  }
#undef LFPS_WINDOW
#undef LFPS_WINDOW_P
  return hipGetLastError();
}

hipError_t launch_window_attn_decode(const Shape& s, int dtype, const KvView& kv, const float* q, int window, int n_sink, float* out, float* part,
                                     hipStream_t st) {
  const WindowRows w = {window, n_sink};
  if (dtype == LFPS_F32) return window_step_t<float, float>(s, q, kv, w, part, out, st);
  if (dtype == LFPS_F16) return window_step_t<_Float16, _Float16>(s, q, kv, w, part, out, st);
  if (kv.k_fp8 && kv.v_fp8) return window_step_t<uint8_t, uint8_t>(s, q, kv, w, part, out, st);
  if (kv.k_fp8) return window_step_t<uint8_t, uint16_t>(s, q, kv, w, part, out, st);
  if (kv.v_fp8) return window_step_t<uint16_t, uint8_t>(s, q, kv, w, part, out, st);
  return window_step_t<uint16_t, uint16_t>(s, q, kv, w, part, out, st);
}

}  // namespace lfps
