// Causal attention of the newest tokens of every request over its cache: whole prompts, chunks behind rows that are there already, a
// few drafted tokens, single ones.  Tokens of all requests are packed; token i of the t_b of request b sits at row n_b - t_b + i
// and sees the rows up to its own.
//
// Two kernels.  k_prompt_tiles: a workgroup has 256 query rows of one (request, KV head) with the loop of tile_pipe.h, 128 over fp32
// caches with that of tile_attn.h, and streams the rows they see; bound by the matrix units.  k_prompt_few: requests whose tokens fill no
// more than one wave's rows (fp32: two), where there are many of them; the waves share the keys; bound by the bytes of K and V.
// Where the rows alone do not fill the chip, those that they see are cut into parts that k_prompt_merge joins.
// Which kernel takes a request is decided on the device by its number of tokens, so one call takes any mixture.
//
// 32 heads over 8 KV heads: 16384 tokens in bf16 1.90 ms, 1160 TFLOP/s of the 1370 that the largest products of the BLAS library reach
// here; 8192 behind 24576 rows of FP8 pages 3.34 ms, 1150; eight prompts of 61 to 4096 tokens over 16 heads in fp16 232 us, 710; two of
// 944 and 1307 in fp32 269 us, 79 of 155 TFLOP/s; five tokens over 4104 rows 15.5 us in two launches (cards differ: 214 to 233, 13.4 to 15.8).  What each step gave is beside
// the loops.
#include "prompt_tiles.h"

namespace lfps {

hipError_t launch_prompt_attn(const Shape& s, int dtype, const KvView& kv, const void* q, int64_t q_stride, const int32_t* cu,
                              int n_tokens, void* out, float* part, int64_t part_rows, hipStream_t st) {
#define LFPS_PROMPT(TK, TV, TQ) return prompt_t<TK, TV, TQ>(s, kv, SeesAll{}, q, q_stride, cu, n_tokens, out, part, part_rows, st)
  if (dtype == LFPS_F32) LFPS_PROMPT(float, float, float);
  if (dtype == LFPS_F16) LFPS_PROMPT(_Float16, _Float16, _Float16);
  if (kv.k_fp8 && kv.v_fp8) LFPS_PROMPT(uint8_t, uint8_t, uint16_t);
  if (kv.k_fp8) LFPS_PROMPT(uint8_t, uint16_t, uint16_t);
  if (kv.v_fp8) LFPS_PROMPT(uint16_t, uint8_t, uint16_t);
  LFPS_PROMPT(uint16_t, uint16_t, uint16_t);
#undef LFPS_PROMPT
}

}  // namespace lfps
