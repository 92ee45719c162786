// S4 — sparse attention over the selected rows (Eq. 1), and the full-attention baseline
// (Sec. 1 with idx = every row; the "full attention" upper bound of Sec. 5).
//
// Sparse: the scores of the selected rows are already known (from S3, or recomputed by the
// per-head score kernel), so the softmax maximum is known before any V row is read and the
// partial sums of the waves merge by plain addition.  One workgroup of 4, 8 or 16 waves per
// (b, h): wave w gathers its share of the head's rows, 16 lanes per V row, 16-byte loads, sixteen
// independent row loads in flight per wave; the partial sums meet in LDS and the output row is
// written once (no partials in global memory, no second kernel).
//
// Full: split-K over contiguous row ranges with the G heads of a group sharing every K and V row; a wave keeps the running
// (max, sum, acc) of its heads, without grouping a lane group of 16 that of its rows, merged with the online-softmax rule.
#include "attend.h"
#include "full_attn.h"

namespace lfps {

// grid B*Hq * kParts, kSparseWaves waves per workgroup
template <typename T, int kSparseWaves, bool kPaged, int kParts>
__global__ __launch_bounds__(kSparseWaves * 64) void k_sparse_attn(Shape s, const T* __restrict__ V, int64_t stride_b,
                                                                int64_t stride_h, int64_t stride_n, KvPage pg,
                                                                const int32_t* __restrict__ seq_lens,
                                                                const int32_t* __restrict__ idx,
                                                                const float* __restrict__ idx_score,
                                                                const int32_t* __restrict__ kk,
                                                                float* __restrict__ out,
                                                                const int32_t* __restrict__ skip_if) {
  __shared__ AttendShared sm;
  request_arguments<decltype(&k_sparse_attn<T, kSparseWaves, kPaged, kParts>)>();
  const HeadPlace at = place_of_block_for<kParts>(s.B, s.Hkv, s.G, blockIdx.x);
  const int bh = at.bh, b = at.b, g = at.g;
  if (at.none) return;
  if (skip_if && skip_if[bh] != 0) return;            // bypassed head: the gate wrote its output row
  int n = seq_lens[b];
  n = n < 0 ? 0 : (n > s.Lcap ? s.Lcap : n);
  int kb = kk[b];
  kb = kb < 0 ? 0 : (kb > s.kmax ? s.kmax : kb);
  attend_rows<T, kSparseWaves, kPaged, kParts>(sm, V, stride_b, stride_h, stride_n, pg, b, g, n, kb,
                                               idx + (int64_t)bh * s.kmax, idx_score + (int64_t)bh * s.kmax, false, 0.f,
                                               out + (int64_t)bh * kD, at.part);
}

template <typename T>
static hipError_t launch_sparse_t(const Shape& s, const KvView& kv, const int32_t* idx, const float* idx_score,
                                  const int32_t* k, float* out, const int32_t* skip_if, hipStream_t st) {
  // as many waves per head as keep every head's workgroup resident at once (256 CUs x 32 waves)
  const int heads = s.B * s.Hq;
  const T* V = (const T*)kv.v;
#define LFPS_LAUNCH_SPARSE_P(NW, PAGED, PARTS)                                                                           \
  hipLaunchKernelGGL((k_sparse_attn<T, NW, PAGED, PARTS>), dim3(attend_blocks(s, PARTS)), dim3(NW * 64), 0, st, s, V, kv.stride_b, \
                     kv.stride_h, kv.stride_n, kv.page, kv.seq_lens, idx, idx_score, k, out, skip_if)
#define LFPS_LAUNCH_SPARSE(NW, PARTS)          \
  if (kv.page.table) {                         \
    LFPS_LAUNCH_SPARSE_P(NW, true, PARTS);     \
  } else {                                     \
    LFPS_LAUNCH_SPARSE_P(NW, false, PARTS);    \
  }
  if (attend_parts(s, kv) == 4) {
    LFPS_LAUNCH_SPARSE(16, 4)
  } else if (heads * 16 <= 4096) {
    LFPS_LAUNCH_SPARSE(16, 1)
  } else if (heads * 8 <= 4096) {
    LFPS_LAUNCH_SPARSE(8, 1)
  } else {
    LFPS_LAUNCH_SPARSE(4, 1)
  }
#undef LFPS_LAUNCH_SPARSE
#undef LFPS_LAUNCH_SPARSE_P
  return hipGetLastError();
}

hipError_t launch_sparse_attn(const Shape& s, int dtype, const KvView& kv, const int32_t* idx, const float* idx_score,
                              const int32_t* k, float* out, const int32_t* skip_if, hipStream_t st) {
  if (dtype == LFPS_BF16 && kv.v_fp8) return launch_sparse_t<uint8_t>(s, kv, idx, idx_score, k, out, skip_if, st);
  if (dtype == LFPS_F16) return launch_sparse_t<_Float16>(s, kv, idx, idx_score, k, out, skip_if, st);
  return dtype == LFPS_BF16 ? launch_sparse_t<uint16_t>(s, kv, idx, idx_score, k, out, skip_if, st)
                            : launch_sparse_t<float>(s, kv, idx, idx_score, k, out, skip_if, st);
}

// ============================================================================ full attention
int full_attn_splits(const Shape& s) {
  int ns = (2048 + s.B * s.Hkv - 1) / (s.B * s.Hkv);
  int by_len = (s.Lcap + 255) / 256;       // at least 256 rows per split
  if (ns > by_len) ns = by_len;
  if (ns > kMaxSplits) ns = kMaxSplits;
  return ns < 1 ? 1 : ns;
}

// grid B*Hq, 128 threads.  Bound by latency (1 MB of partials per 256 heads and 8 splits): the maxima and sums of all
// splits are fetched by one load each (a lane per split), the partial rows eight at a time.  Walking the splits one
// after the other took 29 us at 256 heads x 32 splits, this form 7.6 (full attention over 8 x 32K: 224 -> 207 us).
__global__ __launch_bounds__(kD) void k_full_merge(Shape s, const int32_t* __restrict__ seq_lens,
                                                   const float* __restrict__ part, int n_split,
                                                   float* __restrict__ out) {
  static_assert(kMaxSplits <= 64, "a lane per split");
  __shared__ float wgt[64], sum[64];
  const int bh = blockIdx.x, b = bh / s.Hq, h = bh % s.Hq, g = h / s.G, hg = h % s.G, c = threadIdx.x;
  int n = seq_lens[b];
  n = n < 0 ? 0 : (n > s.Lcap ? s.Lcap : n);
  if (n == 0) {
    out[(int64_t)bh * kD + c] = 0.f;
    return;
  }
  const int rps = rows_per_split(n, n_split);
  const int nv = (n + rps - 1) / rps;
  const int64_t step = (int64_t)s.G * (kD + 2);      // from one split's partials to the next one's
  const float* pb = part + ((int64_t)(b * s.Hkv + g) * n_split) * step + (int64_t)hg * (kD + 2);
  constexpr int kU = 8;
  float x[kU];
  auto fetch = [&](int sp0) {
#pragma unroll
    for (int u = 0; u < kU; ++u) x[u] = pb[(sp0 + u < nv ? sp0 + u : nv - 1) * step + c];
  };
  fetch(0);
  if (c < 64) {
    const int sp = c < nv ? c : nv - 1;
    const float m = pb[sp * step + kD];
    sum[c] = pb[sp * step + kD + 1];
    float mx = m;
#pragma unroll
    for (int d = 1; d < 64; d <<= 1) mx = fmaxf(mx, __shfl_xor(mx, d));
    wgt[c] = s.G == 1 ? part_weight<1>(m - mx) : part_weight<2>(m - mx);
  }
  __syncthreads();
  float a = 0.f, l = 0.f;
  for (int sp0 = 0;;) {
#pragma unroll
    for (int u = 0; u < kU; ++u) {
      if (sp0 + u < nv) {
        a = fmaf(x[u], wgt[sp0 + u], a);
        l = fmaf(sum[sp0 + u], wgt[sp0 + u], l);
      }
    }
    sp0 += kU;
    if (sp0 >= nv) break;
    fetch(sp0);
  }
  out[(int64_t)bh * kD + c] = a / l;
}

template <typename TK, typename T>
static hipError_t launch_full_t(const Shape& s, const float* q, const KvView& kv, float* part, int n_split,
                                hipStream_t st) {
  const dim3 grid(n_split, s.B * s.Hkv), block(kAttnThreads);
  const float scale = 0.08838834764831845f;
  // (the kernels ask how many rows are held; fp32 rows: a lane's eight channels are two loads, which would fetch the line twice)
  const bool once = sizeof(TK) < 4 && (int64_t)s.B * s.Hkv * s.Lcap * kD * (int64_t)(sizeof(TK) + sizeof(T)) > kKeptStreamBytes;
#define LFPS_LAUNCH_FULL_P(KERNEL, PAGED, ONCE, ...)                                                                    \
  hipLaunchKernelGGL((KERNEL<TK, T, ##__VA_ARGS__, PAGED, ONCE>), grid, block, 0, st, s, q, (const TK*)kv.k,             \
                     (const T*)kv.v, kv.stride_b, kv.stride_h, kv.stride_n, kv.page, kv.seq_lens, part, n_split, scale)
#define LFPS_LAUNCH_FULL(KERNEL, ...)                                                   \
  if (kv.page.table) {                                                                  \
    if (once) LFPS_LAUNCH_FULL_P(KERNEL, true, sizeof(TK) < 4, ##__VA_ARGS__);          \
    else LFPS_LAUNCH_FULL_P(KERNEL, true, false, ##__VA_ARGS__);                        \
  } else {                                                                              \
    if (once) LFPS_LAUNCH_FULL_P(KERNEL, false, sizeof(TK) < 4, ##__VA_ARGS__);         \
    else LFPS_LAUNCH_FULL_P(KERNEL, false, false, ##__VA_ARGS__);                       \
  }
  switch (s.G) {
    case 1: LFPS_LAUNCH_FULL(k_full_attn_single); break;
    case 2: LFPS_LAUNCH_FULL(k_full_attn, 2); break;
    case 4: LFPS_LAUNCH_FULL(k_full_attn, 4); break;
    default: return hipErrorInvalidValue;
  }
#undef LFPS_LAUNCH_FULL
#undef LFPS_LAUNCH_FULL_P
  return hipGetLastError();
}

hipError_t launch_full_attn(const Shape& s, int dtype, const float* q, const KvView& kv, float* part, int n_split,
                            hipStream_t st) {
  if (dtype == LFPS_BF16 && kv.k_fp8 && kv.v_fp8) return launch_full_t<uint8_t, uint8_t>(s, q, kv, part, n_split, st);
  if (dtype == LFPS_BF16 && kv.k_fp8) return launch_full_t<uint8_t, uint16_t>(s, q, kv, part, n_split, st);
  if (dtype == LFPS_BF16 && kv.v_fp8) return launch_full_t<uint16_t, uint8_t>(s, q, kv, part, n_split, st);
  if (dtype == LFPS_F16) return launch_full_t<_Float16, _Float16>(s, q, kv, part, n_split, st);
  return dtype == LFPS_BF16 ? launch_full_t<uint16_t, uint16_t>(s, q, kv, part, n_split, st)
                            : launch_full_t<float, float>(s, q, kv, part, n_split, st);
}

template <typename TK, typename T>
static hipError_t launch_full_own_t(const Shape& s, const float* q, const KvView& kv, const OwnRows& own, float* part, hipStream_t st) {
  const dim3 grid(own_items_most(s), s.Hkv), block(kAttnThreads);
  const float scale = 0.08838834764831845f;
#define LFPS_LAUNCH_OWN_P(KERNEL, PAGED, ...)                                                                             \
  hipLaunchKernelGGL((KERNEL<TK, T, ##__VA_ARGS__, PAGED, false, OwnRows>), grid, block, 0, st, s, q, (const TK*)kv.k, \
                     (const T*)kv.v, kv.stride_b, kv.stride_h, kv.stride_n, kv.page, kv.seq_lens, part, 0, scale, own)
#define LFPS_LAUNCH_OWN(KERNEL, ...)                              \
  if (kv.page.table) LFPS_LAUNCH_OWN_P(KERNEL, true, ##__VA_ARGS__); \
  else LFPS_LAUNCH_OWN_P(KERNEL, false, ##__VA_ARGS__);
  switch (s.G) {
    case 1: LFPS_LAUNCH_OWN(k_full_attn_single) break;
    case 2: LFPS_LAUNCH_OWN(k_full_attn, 2) break;
    case 4: LFPS_LAUNCH_OWN(k_full_attn, 4) break;
    default: return hipErrorInvalidValue;
  }
#undef LFPS_LAUNCH_OWN
#undef LFPS_LAUNCH_OWN_P
  return hipGetLastError();
}

hipError_t launch_full_attn_own(const Shape& s, int dtype, const float* q, const KvView& kv, const OwnRows& own, float* part, hipStream_t st) {
  if (dtype == LFPS_F32) return launch_full_own_t<float, float>(s, q, kv, own, part, st);
  if (dtype == LFPS_F16) return launch_full_own_t<_Float16, _Float16>(s, q, kv, own, part, st);
  if (kv.k_fp8 && kv.v_fp8) return launch_full_own_t<uint8_t, uint8_t>(s, q, kv, own, part, st);
  if (kv.k_fp8) return launch_full_own_t<uint8_t, uint16_t>(s, q, kv, own, part, st);
  if (kv.v_fp8) return launch_full_own_t<uint16_t, uint8_t>(s, q, kv, own, part, st);
  return launch_full_own_t<uint16_t, uint16_t>(s, q, kv, own, part, st);
}

hipError_t launch_full_merge(const Shape& s, const int32_t* seq_lens, const float* part, int n_split, float* out,
                             hipStream_t st) {
  hipLaunchKernelGGL(k_full_merge, dim3(s.B * s.Hq), dim3(kD), 0, st, s, seq_lens, part, n_split, out);
  return hipGetLastError();
}

}  // namespace lfps
