// What the two attention kernels share.
#pragma once

#include "serve.cuh"

namespace qcfg {

struct AttnArgs {
  PoolView pool;
  CacheView cache;
  BatchView batch;
  const void* q;
  void* out;
  int64_t q_row, q_head, o_row, o_head;
  int q_heads, causal, window;
  int uncut;                // every tile to one block (see kUncutTokens)
  float scale;              // sm_scale * log2(e)
  void* work;
  unsigned* err;
};

// Attention of many rows (prompt.cu); false: not a case for it
bool prompt_pays(Ctx* ctx, const AttnArgs& a, int dtype, int64_t rows);
int launch_prompt(Ctx* ctx, const AttnArgs& a, int dtype, cudaStream_t st);

namespace {

// Weights are 2^(bias + x - ref).  The bias leaves 16-bit calls seven more binary orders below the largest weight; fp32 calls hold a
// weight in two fp16 numbers and take none: an exponent's rounding is relative to its size, which is small then for the weights that
// count.
template <bool WIDE> __host__ __device__ constexpr float weight_bias() { return WIDE ? 0.0f : 7.0f; }

// The tokens the row at position pos sees: [lo, hi), empty as hi <= lo.
__device__ __forceinline__ void seen_range(const AttnArgs& a, int64_t pos, int len, int& lo, int& hi) {
  hi = pos < 0 ? 0 : a.causal ? (int)(pos + 1) : len;
  lo = a.window > 0 && pos + 1 > a.window ? (int)(pos + 1) - a.window : 0;
}

__device__ __forceinline__ uint32_t h2_bits(__half2 h) { return *reinterpret_cast<uint32_t*>(&h); }
__device__ __forceinline__ uint32_t pack_h2(float a, float b) { return h2_bits(__floats2half2_rn(a, b)); }
__device__ __forceinline__ float ex2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
__device__ __forceinline__ float lg2(float x) {
  float y;
  asm("lg2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
// Two bytes of a word of codes plus 128 as fp16 codes: 0x6400 + b is 1024 + b.  `magic` is 0x64646464, read from shared memory once: as a
// compile-time constant it cost 118 of the 870 instructions that a run of the streaming kernel took then.
template <uint32_t SEL>
__device__ __forceinline__ uint32_t two_codes(uint32_t biased, uint32_t magic) {
  const uint32_t w = __byte_perm(biased, magic, SEL);
  const __half2 off = __floats2half2_rn(1152.0f, 1152.0f);
  return h2_bits(__hsub2(*reinterpret_cast<const __half2*>(&w), off));
}
// The power of two that brings a row's largest element (its bit pattern without sign) to 2^12 .. 2^13; its inverse goes into the row's factor
__device__ __forceinline__ int row_shift(unsigned top) {
  int shift = 12 - ((int)(top >> 23) - 127);
  if (top == 0 || top >= 0x7f800000u) shift = 0;
  return shift > 120 ? 120 : shift;
}
__device__ __forceinline__ float exp2_of(int e) { return __uint_as_float((unsigned)(127 + e) << 23); }

}  // namespace

}  // namespace qcfg
