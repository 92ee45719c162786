// Attention over a sliding window and the first rows: the newest tokens of every request, packed; the token at row p sees the rows j <= p with
// j > p - window or j < n_sink.  (A decode step's single tokens: window_step.hip.)
//
// The kernels of the prompts over fewer rows: a tile of tokens walks the first rows, rounded up to eights, and behind them those from its first token's
// window on, as if they lay together; only the steps at the window's two edges and behind the first rows look which rows a token sees.  Weights are
// rounded as the prompts' are: of 16-bit queries to 16 bits for the product with V, so that the matrix units take them in one term, and their sum is of
// the rounded ones.  The result, rounded to the same type, is 1.8e-3 (bf16) and 2.3e-4 (fp16) from 64 bits, of which its own rounding alone makes 1.7e-3
// and 2.1e-4.
// Bound by the matrix units, less closely than whole prompts: a tile of 64 tokens walks 1100 rows where each of them sees 1028, and what a workgroup
// does once (first rows asked for, waited for and scored, edges, results stored) comes every 17 stages.  32 heads over 8 KV heads, bf16: 16384 tokens,
// window 1024, 337 us, 793 TFLOP/s of the 1392 that a large library product reaches (a window of one row, which is all fixed cost, 110); six chunks
// of 100 to 4000 tokens of 16 heads in fp16, window 517, 100 to 109 us by the card; five tokens, window 1024, 11.7 us in two launches.
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
