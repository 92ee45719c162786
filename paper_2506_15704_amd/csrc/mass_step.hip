// A decode step's full attention that adds its weights up: the kernels of the full attention, which leave the scores too, and one that joins their
// parts into the output and, now that the sums over whole rows are known, makes the scores weights:
//
//   mass[b, g, j] = (j < held_b ? decay * mass[b, g, j] : 0) + sum_{h in g} softmax_j(q[b, h] . K[b, g, j] / sqrt(D))
//
// so that K and V are read once.  The scores are 4 G bytes a row on the way out and back beside 4 D of K and V in 16 bits.  Bound by the bytes: 16
// requests of 2000 to 32768 rows, bf16 pages, 1.21 GB 258 us, 4.7 TB/s, where the attention alone takes 200 (with a wave a head and two passes over K
// 2411, with registers for three waves a SIMD 266: attn_waves).  The scores' stores are 23 of the difference, V's rows behind the last one 12, this kernel 13; stores of four
// tiles at a time through LDS, scores with the heads side by side, stores past the caches and rows of zeros for those behind the last one
// were no faster.
#include "full_attn.h"

namespace lfps {

constexpr int kMassChunk = 1024;             // rows of a workgroup

// grid (1 + chunks, B * Hkv): the first workgroup of a group makes its heads' output rows, a wave a head, the others take rows.
template <int G>
__global__ __launch_bounds__(256) void k_mass_step(Shape s, const int32_t* __restrict__ seq_lens, const float* __restrict__ part, int n_split,
                                                   ScoresTo from, const int32_t* __restrict__ held, float decay, float* __restrict__ mass,
                                                   float* __restrict__ out) {
  __shared__ float top[G], inverse[G];
  const int bg = blockIdx.y, b = bg / s.Hkv, g = bg % s.Hkv, lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int n = length_of(s, seq_lens, b), row0 = ((int)blockIdx.x - 1) * kMassChunk;
  if (row0 >= n && blockIdx.x) return;
  const int rps = rows_per_split(n, n_split), parts = n > 0 ? (n + rps - 1) / rps : 0;
  const float* const mine = part + (int64_t)bg * n_split * G * (kD + 2);
  if (blockIdx.x == 0) {
    if (wave >= G) return;
    float m, l;
    const f32x2t y = parts ? join_head<G>(mine, parts, wave, &m, &l) : f32x2t{0.f, 0.f};
    *reinterpret_cast<f32x2t*>(out + ((int64_t)b * s.Hq + g * G + wave) * kD + 2 * lane) = y;
    return;
  }
  constexpr int kEach = kMassChunk / 256;
  float x[G][kEach], old[kEach];
  const float* const scores = from.score + ((int64_t)b * s.Hq + g * G) * from.stride;
  float* const to = mass + (int64_t)bg * s.Lcap;
  const int keep = held ? held[b] : 0;
#pragma unroll
  for (int i = 0; i < kEach; ++i) {
    const int r = row0 + 256 * i + (int)threadIdx.x, at = r < n ? r : n - 1;
#pragma unroll
    for (int h = 0; h < G; ++h) x[h][i] = scores[h * from.stride + at];
    old[i] = at < keep ? to[at] : 0.f;
  }
  if (wave < G) {
    const float* const p = mine + wave * (kD + 2) + (int64_t)lane * G * (kD + 2);
    float m, l, w;
    weigh_parts<G>(lane < parts ? p[kD] : -INFINITY, lane < parts ? p[kD + 1] : 0.f, &m, &l, &w);
    top[wave] = m;
    inverse[wave] = l;
  }
  __syncthreads();
#pragma unroll
  for (int i = 0; i < kEach; ++i) {
    const int r = row0 + 256 * i + (int)threadIdx.x;
    float sum = 0.f;
#pragma unroll
    for (int h = 0; h < G; ++h) sum = fmaf(part_weight<G>(x[h][i] - top[h]), inverse[h], sum);
    if (r < n) to[r] = sum + (r < keep ? decay * old[i] : 0.f);
  }
}

template <typename TK, typename T>
static hipError_t mass_step_t(const Shape& s, const float* q, const KvView& kv, const ScoresTo& to, const int32_t* held, float decay, float* mass, float* out,
                              float* part, int n_split, hipStream_t st) {
  const dim3 grid(n_split, s.B * s.Hkv), block(kAttnThreads), rows(1 + (s.Lcap + kMassChunk - 1) / kMassChunk, s.B * s.Hkv);
  const float scale = 0.08838834764831845f;
  const bool once = sizeof(TK) < 4 && (int64_t)s.B * s.Hkv * s.Lcap * kD * (int64_t)(sizeof(TK) + sizeof(T)) > kKeptStreamBytes;      // (as in the full attention)
#define LFPS_STEP_P(KERNEL, PAGED, ONCE, ...)                                                                              \
  hipLaunchKernelGGL((KERNEL<TK, T, ##__VA_ARGS__, PAGED, ONCE, ScoresTo>), grid, block, 0, st, s, q, (const TK*)kv.k,     \
                     (const T*)kv.v, kv.stride_b, kv.stride_h, kv.stride_n, kv.page, kv.seq_lens, part, n_split, scale, to)
#define LFPS_STEP(G, KERNEL, ...)                                                   \
  if (kv.page.table) {                                                              \
    if (once) LFPS_STEP_P(KERNEL, true, sizeof(TK) < 4, ##__VA_ARGS__);             \
    else LFPS_STEP_P(KERNEL, true, false, ##__VA_ARGS__);                           \
  } else {                                                                          \
    if (once) LFPS_STEP_P(KERNEL, false, sizeof(TK) < 4, ##__VA_ARGS__);            \
    else LFPS_STEP_P(KERNEL, false, false, ##__VA_ARGS__);                          \
  }                                                                                 \
  hipLaunchKernelGGL((k_mass_step<G>), rows, dim3(256), 0, st, s, kv.seq_lens, part, n_split, to, held, decay, mass, out)
  switch (s.G) {
    case 1: LFPS_STEP(1, k_full_attn_single); break;
    case 2: LFPS_STEP(2, k_full_attn, 2); break;
    case 4: LFPS_STEP(4, k_full_attn, 4); break;
    default: return hipErrorInvalidValue;
  }
#undef LFPS_STEP
#undef LFPS_STEP_P
  return hipGetLastError();
}

hipError_t launch_mass_step(const Shape& s, int dtype, const KvView& kv, const float* q, const int32_t* held, float decay, float* mass, float* out,
                            float* score, int64_t score_stride, float* part, int n_split, hipStream_t st) {
  const ScoresTo to = {score, score_stride};
#define LFPS_STEP(TK, T) return mass_step_t<TK, T>(s, q, kv, to, held, decay, mass, out, part, n_split, st)
  if (dtype == LFPS_F32) LFPS_STEP(float, float);
  if (dtype == LFPS_F16) LFPS_STEP(_Float16, _Float16);
  if (kv.k_fp8 && kv.v_fp8) LFPS_STEP(uint8_t, uint8_t);
  if (kv.k_fp8) LFPS_STEP(uint8_t, uint16_t);
  if (kv.v_fp8) LFPS_STEP(uint16_t, uint8_t);
  LFPS_STEP(uint16_t, uint16_t);
#undef LFPS_STEP
}

}  // namespace lfps
