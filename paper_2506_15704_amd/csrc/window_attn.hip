// Attention over a sliding window and the first rows: the token at row p sees the rows j <= p with j > p - window or j < n_sink.  The newest
// tokens of every request, packed, and a decode step's single ones.
#include "prompt_tiles.h"

namespace lfps {

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

}  // namespace lfps
