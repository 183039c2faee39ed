// Linear layers with a scale for each token: codes of Eq. 1 row by row, and the int8 product whose rescale takes the row's scale.
#include <algorithm>

#include "serve.cuh"

namespace qcfg {

namespace {

// A block for each row: the row's maximum, then its codes (the second read comes from L1 or L2).
constexpr int kTokenThreads = 256;
template <typename T>
__global__ void __launch_bounds__(kTokenThreads) quantize_tokens_kernel(const T* x, int64_t cols, int64_t ld, float qmax, int8_t* q, int64_t ldq,
                                                                        float* scale, unsigned* err) {
  pdl_entry();
  __shared__ unsigned tops[kTokenThreads / 32];
  const int64_t row = blockIdx.x;
  x += row * ld;
  q += row * ldq;
  unsigned top = 0, odd = 0;
  for (int64_t c = threadIdx.x; c < cols; c += kTokenThreads) {
    const unsigned a = abs_bits(to_float<T>(x[c]));
    if (a < 0x7f800000u) top = a > top ? a : top; else odd = 1;
  }
  top = warp_max_u(top);
  if ((threadIdx.x & 31) == 0) tops[threadIdx.x >> 5] = top;
  if (__syncthreads_or(odd) && threadIdx.x == 0) atomicOr(err, ERR_NONFINITE);
#pragma unroll
  for (int w = 0; w < kTokenThreads / 32; ++w) top = tops[w] > top ? tops[w] : top;
  const float absmax = __uint_as_float(top), inv = inv_scale_of(absmax, qmax);
  for (int64_t c = threadIdx.x; c < ldq; c += kTokenThreads) {
    const float f = c < cols ? to_float<T>(x[c]) : 0.0f;
    q[c] = (int8_t)(finite_bits(f) ? code_of(f, inv, qmax) : 0);
  }
  if (threadIdx.x == 0) scale[row] = scale_of(absmax, qmax);
}

// y = act(float(acc) * (scale_x[m] * scale_w[n]) + bias[n])
template <typename T>
__global__ void __launch_bounds__(256) rescale_kernel(const int32_t* acc, int64_t m, int64_t n, const float* sx, const float* sw, const float* bias,
                                                      int act, T* y, int64_t ldy) {
  pdl_entry();
  const int64_t total = m * n;
  for (int64_t e = (int64_t)blockIdx.x * 256 + threadIdx.x; e < total; e += (int64_t)gridDim.x * 256) {
    const int64_t r = e / n, c = e - r * n;
    float v = (float)acc[e] * (sx[r] * sw[c]);
    if (bias) v += bias[c];
    if (act == QCFG_ACT_RELU) v = fmaxf(v, 0.0f);
    else if (act == QCFG_ACT_GELU_TANH) v = gelu_tanh(v);
    y[r * ldy + c] = from_float<T>(v);
  }
}

inline int64_t up(int64_t v, int64_t a) { return (v + a - 1) / a * a; }

}  // namespace

int launch_quantize_tokens(Ctx* ctx, const void* x, int dtype, int64_t rows, int64_t cols, int64_t ld, int bits, int8_t* q, int64_t ldq, float* scale,
                           cudaStream_t st) {
  if (rows == 0) return QCFG_OK;
  const dim3 grid((unsigned)rows), block(kTokenThreads);
  const float qmax = qmax_of(bits);
  if (dtype == QCFG_FP32) launch_pdl(quantize_tokens_kernel<float>, grid, block, 0, st, (const float*)x, cols, ld, qmax, q, ldq, scale, err_word(ctx));
  else if (dtype == QCFG_BF16) launch_pdl(quantize_tokens_kernel<__nv_bfloat16>, grid, block, 0, st, (const __nv_bfloat16*)x, cols, ld, qmax, q, ldq, scale, err_word(ctx));
  else launch_pdl(quantize_tokens_kernel<__half>, grid, block, 0, st, (const __half*)x, cols, ld, qmax, q, ldq, scale, err_word(ctx));
  count_launch(ctx);
  return check_cuda(ctx, cudaGetLastError(), "quantize_tokens");
}

int launch_gemm_token(Ctx* ctx, const TokenGemm& t, cudaStream_t st) {
  int32_t* acc = (int32_t*)scratch(ctx, (size_t)(t.m * t.n * 4));
  if (!acc) return set_error(ctx, QCFG_ENOMEM, "gemm_i8_token: no memory for the accumulators");
  GemmArgs g{};
  g.a = t.qx; g.lda = t.ldx; g.b = t.qw; g.ldb = t.ldw; g.m = t.m; g.n = t.n; g.k = t.k;
  g.acc = acc;
  const int rc = launch_gemm(ctx, g, st);
  if (rc) return rc;
  const dim3 grid((unsigned)std::min<int64_t>((t.m * t.n + 255) / 256, 148 * 16)), block(256);
  if (t.dtype == QCFG_FP32) launch_pdl(rescale_kernel<float>, grid, block, 0, st, acc, t.m, t.n, t.sx, t.sw, t.bias, t.act, (float*)t.y, t.ldy);
  else if (t.dtype == QCFG_BF16) launch_pdl(rescale_kernel<__nv_bfloat16>, grid, block, 0, st, acc, t.m, t.n, t.sx, t.sw, t.bias, t.act, (__nv_bfloat16*)t.y, t.ldy);
  else launch_pdl(rescale_kernel<__half>, grid, block, 0, st, acc, t.m, t.n, t.sx, t.sw, t.bias, t.act, (__half*)t.y, t.ldy);
  count_launch(ctx);
  return check_cuda(ctx, cudaGetLastError(), "gemm_i8_token");
}

// codes [m x ldq], then the scales
int64_t linear_work(int64_t m, int64_t k) { return up(m * up(k, 16), 256) + up(m * 4, 256); }
int launch_linear(Ctx* ctx, const void* x, int x_dtype, int64_t ldx, int bits, const TokenGemm& t_in, void* work, cudaStream_t st) {
  TokenGemm t = t_in;
  t.ldx = up(t.k, 16);
  int8_t* codes = (int8_t*)work;
  float* scale = (float*)(codes + up(t.m * t.ldx, 256));
  t.qx = codes;
  t.sx = scale;
  const int rc = launch_quantize_tokens(ctx, x, x_dtype, t.m, t.k, ldx, bits, codes, t.ldx, scale, st);
  return rc ? rc : launch_gemm_token(ctx, t, st);
}

}  // namespace qcfg
