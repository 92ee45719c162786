// The prompt kernel's body for 16-bit operands (bf16, fp16, FP8 converted to bf16): tile_attn.h's products, made for the matrix
// units' rate.
#pragma once
#include "tile_attn.h"

namespace lfps {

constexpr int kPipeKeys = 64, kPipeRows = 128;       // keys of a stage, query rows of a workgroup
constexpr float kLazy = 6.f;                         // growth of a maximum, in powers of two, that is let pass

typedef __attribute__((address_space(3))) char lds_char;
typedef const __attribute__((address_space(1))) char global_char;

// The 16 rows [k0 + 16 wave, + 16) of a stage that a wave brings, of K or V.  16-bit elements go from memory to LDS without
// registers, four rows an instruction: lane l fills place l % 16 of row l / 16, so it asks for the chunk that belongs there.
template <typename T>
struct Feed {
  static constexpr bool kDirect = sizeof(T) == 2;
  static constexpr int kLoads = kDirect ? 4 : 2;     // FP8: eight rows a load, through registers
  static constexpr int kRowsOfLoad = 16 / kLoads;
  u32x4 x[kDirect ? 1 : kLoads];

  __device__ __forceinline__ static int row(int i, int lane) { return kRowsOfLoad * i + (kDirect ? lane >> 4 : lane >> 3); }
  __device__ __forceinline__ static int bytes(int i, int lane) {                  // of the lane's piece in its row of the cache
    return kDirect ? 16 * ((lane & 15) ^ (2 * (row(i, lane) & 7))) : 16 * (lane & 7);
  }
  __device__ __forceinline__ void one(const char* from, lds_char* stage, int i, int wave) {
    if constexpr (kDirect)
      __builtin_amdgcn_global_load_lds((global_char*)from, (__attribute__((address_space(3))) void*)(stage + (16 * wave + 4 * i) * 256), 16, 0, 0);
    else
      x[i] = *reinterpret_cast<const u32x4*>(from);
  }
  // c: rows of the request; offsets: of my pieces from the first of the wave's rows (where `alike`: a page or slab of equal strides)
  __device__ __forceinline__ void ask(const CacheRows<T>& c, lds_char* stage, int k0, int end, bool alike, int lane, int wave) {
    int w0 = k0 + 16 * wave;                                                    // the wave's first row, one that exists
    w0 = w0 < end ? w0 : (end - 1) & ~15;
    w0 = __builtin_amdgcn_readfirstlane(w0);
    const int last = end - 1 - w0;
    if (alike) {
      const char* base = reinterpret_cast<const char*>(c.at(w0, c.entry(w0)));
      const int pitch = (int)c.stride_n * (int)sizeof(T);
#pragma unroll
      for (int i = 0; i < kLoads; ++i) {
        int r = row(i, lane);
        r = r < last ? r : last;
        one(base + (uint32_t)(r * pitch + bytes(i, lane)), stage, i, wave);
      }
    } else {
#pragma unroll
      for (int i = 0; i < kLoads; ++i) {
        int r = row(i, lane);
        r = w0 + (r < last ? r : last);
        one(reinterpret_cast<const char*>(c.at(r, c.entry(r))) + bytes(i, lane), stage, i, wave);
      }
    }
  }
  // FP8: what has arrived becomes bf16 in the stage
  __device__ __forceinline__ void put(lds_char* stage, int lane, int wave) const {
    if constexpr (!kDirect) {
#pragma unroll
      for (int i = 0; i < kLoads; ++i) {
        const int r = 16 * wave + row(i, lane), c = lane & 7;
        typedef __attribute__((address_space(3))) bf16x8* Lds;
        *(Lds)(stage + r * 256 + 16 * chunk_place(r, 2 * c)) = fp8x8_to_bf16x8(x[i][0], x[i][1]);
        *(Lds)(stage + r * 256 + 16 * chunk_place(r, 2 * c + 1)) = fp8x8_to_bf16x8(x[i][2], x[i][3]);
      }
    }
  }
};

// 32 query rows of a wave.
template <typename Op>
struct PipeState {
  typedef RowState<Op, 1> Tile;
  f32x16 o[4];
  float m, l;
  typename Tile::Query q;
  int limit;

  __device__ __forceinline__ void clear() {
    m = -INFINITY;
    l = 0.f;
#pragma unroll
    for (int d = 0; d < 4; ++d)
#pragma unroll
      for (int r = 0; r < 16; ++r) o[d][r] = 0.f;
  }

  // Scores of the 32 keys at `k`.
  __device__ __forceinline__ void scores(f32x16& s, const lds_char* k, int n, int h) const {
#pragma unroll
    for (int r = 0; r < 16; ++r) s[r] = 0.f;
#pragma unroll
    for (int c = 0; c < 8; ++c)
      s = mfma32(*(const __attribute__((address_space(3))) Op*)(k + n * 256 + 16 * chunk_place(n, 2 * c + h)), q.x[0][c], s);
  }

  // Scores of kBlocks * 32 keys -> weights w; returns what the sums so far have to be multiplied with, before these weights' values
  // are added.
  template <bool kMasked, int kBlocks>
  __device__ __forceinline__ float weights(f32x16 (&s)[kBlocks], Op (&w)[2 * kBlocks], int first, int h) {
    float mx = -INFINITY;
#pragma unroll
    for (int b = 0; b < kBlocks; ++b)
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        if (kMasked && first + 32 * b + 8 * (r / 4) + 4 * h + r % 4 >= limit) s[b][r] = -INFINITY;
        mx = fmaxf(mx, s[b][r]);
      }
    {
      const auto both = __builtin_amdgcn_permlane32_swap(__float_as_int(mx), __float_as_int(mx), false, false);
      mx = fmaxf(__int_as_float(both[0]), __int_as_float(both[1]));
    }
    mx *= q.unit;
    const float before = m;
    const float now = mx > before + kLazy ? mx : before;              // (from -inf on the first keys)
    const float at = now == -INFINITY ? 0.f : now - Tile::kLift;
    const float shrink = now == before ? 1.f : __builtin_amdgcn_exp2f(before - now);
    float sum = 0.f;
#pragma unroll
    for (int b = 0; b < kBlocks; ++b)
#pragma unroll
      for (int r = 0; r < 16; r += 2) {
        f32x2t p;
        p[0] = __builtin_amdgcn_exp2f(fmaf(s[b][r], q.unit, -at));
        p[1] = __builtin_amdgcn_exp2f(fmaf(s[b][r + 1], q.unit, -at));
        sum += p[0];
        sum += p[1];
        if constexpr (std::is_same<Op, bf16x8>::value) {
          const bf16x2t z = __builtin_convertvector(p, bf16x2t);
          w[2 * b + r / 8][r % 8] = z[0];
          w[2 * b + r / 8][r % 8 + 1] = z[1];
        } else {
          w[2 * b + r / 8][r % 8] = (_Float16)p[0];
          w[2 * b + r / 8][r % 8 + 1] = (_Float16)p[1];
        }
      }
    m = now;
    l = fmaf(l, shrink, sum);
    return shrink;
  }

  __device__ __forceinline__ static Op values(const lds_char* v, int t, int d, int lane) {
    const int h = lane >> 5, i = lane & 15, key = 4 * h + (i >> 2), chunk = 4 * d + 2 * ((lane >> 4) & 1) + ((i & 3) >> 1);
    typedef __attribute__((address_space(3))) s16x4* Lds;
    union {
      s16x4 half[2];
      Op op;
    } a;
    const lds_char* at = v + key * 256 + 16 * chunk_place(key, chunk) + 8 * (i & 1) + t * (16 * 256);
    a.half[0] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((Lds)at);
    a.half[1] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((Lds)(at + 8 * 256));
    return a.op;
  }
  template <int kSteps>
  __device__ __forceinline__ void add_values(const Op (&w)[kSteps], const lds_char* v, int lane) {
#pragma unroll
    for (int t = 0; t < kSteps; ++t)
#pragma unroll
      for (int d = 0; d < 4; ++d) o[d] = mfma32(values(v, t, d, lane), w[t], o[d]);
  }
  __device__ __forceinline__ void rescale(float shrink) {
    if (__ballot(shrink != 1.f)) {
#pragma unroll
      for (int d = 0; d < 4; ++d)
#pragma unroll
        for (int r = 0; r < 16; ++r) o[d][r] *= shrink;
    }
  }
};

// LDS: two stages of K, then two of V
constexpr int kPipeStage = kPipeKeys * 256, kPipeLds = 4 * kPipeStage;
template <typename TK, typename TV, typename Op>
__device__ __forceinline__ void pipe_loop(char* lds_, const CacheRows<TK>& K, const CacheRows<TV>& V, int first, int end, PipeState<Op>& st) {
  lds_char* const lds = (lds_char*)lds_;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), n = lane & 31, h = lane >> 5;
  int least = st.limit;
#pragma unroll
  for (int d = 1; d < 32; d <<= 1) least = min(least, __shfl_xor(least, d));
  least = __builtin_amdgcn_readfirstlane(least);
  const bool alike = (K.pg.table == nullptr || K.pg.shift >= 4) && K.stride_n < (1 << 24);
  Feed<TK> fk;
  Feed<TV> fv;
  int now = 0;
  constexpr int kV = 2 * kPipeStage;
  fk.ask(K, lds, first, end, alike, lane, wave);
  fv.ask(V, lds + kV, first, end, alike, lane, wave);
  fk.put(lds, lane, wave);
  fv.put(lds + kV, lane, wave);
  int k0 = first;
  auto stage = [&](auto masked) {
    const bool more = k0 + kPipeKeys < end;
    const int next = now ^ kPipeStage;
    __builtin_amdgcn_s_waitcnt(0x0f70);       // vmcnt(0): what I asked for is in LDS
    __syncthreads();                          // and what all did; nobody reads the other stage any more
    if (more) {
      fk.ask(K, lds + next, k0 + kPipeKeys, end, alike, lane, wave);
      fv.ask(V, lds + kV + next, k0 + kPipeKeys, end, alike, lane, wave);
    }
    f32x16 s[2];
    Op w[4];
    st.scores(s[0], lds + now, n, h);
    st.scores(s[1], lds + now + 32 * 256, n, h);
    st.rescale(st.template weights<decltype(masked)::value>(s, w, k0, h));
    st.add_values(w, lds + kV + now, lane);
    if (more) {
      fk.put(lds + next, lane, wave);
      fv.put(lds + kV + next, lane, wave);
    }
    now = next;
    k0 += kPipeKeys;
  };
  while (k0 < end && k0 + kPipeKeys <= least) stage(std::false_type{});
  while (k0 < end) stage(std::true_type{});
}

}  // namespace lfps
