// Linear layers with a scale for each token: codes of Eq. 1 row by row, and the int8 product whose rescale takes the row's scale.
#include "serve.cuh"

namespace qcfg {

namespace {

// WPR warps (1 or 8) for each row, which they read once and keep in registers while it fits: HELD pieces of 16 bytes a thread, or
// with VEC false (rows not on 16-byte boundaries) single elements.  What does not fit is read twice, the second time from L2.
constexpr int kTokenThreads = 256;
template <typename T, bool VEC> __host__ __device__ constexpr int held_pieces() { return VEC ? 8 : 16; }
template <typename T, int WPR, bool VEC>
__global__ void __launch_bounds__(kTokenThreads) quantize_tokens_kernel(const T* __restrict__ x, int64_t rows, int64_t cols, int64_t ld, float qmax,
                                                                        int8_t* __restrict__ q, int64_t ldq, float* __restrict__ scale, unsigned* err) {
  pdl_entry();
  constexpr int V = VEC ? Vec<T>::N : 1, HELD = held_pieces<T, VEC>(), N = 32 * WPR;
  __shared__ unsigned tops[8];
  const int64_t row = WPR == 8 ? (int64_t)blockIdx.x : (int64_t)blockIdx.x * 8 + (threadIdx.x >> 5);
  const int t = WPR == 8 ? threadIdx.x : threadIdx.x & 31;
  if (WPR == 1 && row >= rows) return;
  x += row * ld;
  q += row * ldq;
  const int pieces = (int)(cols / V);
  float held[HELD][V];
  unsigned top = 0, odd = 0;
  auto get = [&](int p, float (&f)[V]) {
    if (VEC) load_vec<T>(x + (int64_t)p * V, reinterpret_cast<float(&)[Vec<T>::N]>(f));
    else f[0] = to_float<T>(x[p]);
  };
  auto see = [&](float f) {
    const unsigned a = abs_bits(f);
    if (a < 0x7f800000u) top = a > top ? a : top; else odd = 1;
  };
#pragma unroll
  for (int i = 0; i < HELD; ++i) {
    if (t + i * N < pieces) get(t + i * N, held[i]);
    else {
#pragma unroll
      for (int j = 0; j < V; ++j) held[i][j] = 0.0f;
    }
  }
#pragma unroll
  for (int i = 0; i < HELD; ++i)
#pragma unroll
    for (int j = 0; j < V; ++j) see(held[i][j]);
  for (int p = t + HELD * N; p < pieces; p += N) {
    float f[V];
    get(p, f);
#pragma unroll
    for (int j = 0; j < V; ++j) see(f[j]);
  }
  const int64_t tail = (int64_t)pieces * V + t;          // fewer than V elements
  const float last = tail < cols ? to_float<T>(x[tail]) : 0.0f;
  see(last);
  top = warp_max_u(top);
  if (WPR == 8) {
    if ((t & 31) == 0) tops[t >> 5] = top;
    if (__syncthreads_or(odd) && t == 0) atomicOr(err, ERR_NONFINITE);
#pragma unroll
    for (int w = 0; w < 8; ++w) top = tops[w] > top ? tops[w] : top;
  } else if (__any_sync(0xffffffffu, odd) && t == 0) {
    atomicOr(err, ERR_NONFINITE);
  }
  const float absmax = __uint_as_float(top), inv = inv_scale_of(absmax, qmax);
  auto put = [&](int p, const float (&f)[V]) {
    union { uint2 w2; uint32_t w; int8_t b[8]; } c;
#pragma unroll
    for (int j = 0; j < V; ++j) c.b[j] = (int8_t)(finite_bits(f[j]) ? code_of(f[j], inv, qmax) : 0);
    int8_t* to = q + (int64_t)p * V;
    if (V == 8) *reinterpret_cast<uint2*>(to) = c.w2;
    else if (V == 4) *reinterpret_cast<uint32_t*>(to) = c.w;
    else *to = c.b[0];
  };
#pragma unroll
  for (int i = 0; i < HELD; ++i)
    if (t + i * N < pieces) put(t + i * N, held[i]);
  for (int p = t + HELD * N; p < pieces; p += N) {
    float f[V];
    get(p, f);
    put(p, f);
  }
  for (int64_t c = tail; c < ldq; c += N) q[c] = (int8_t)(c == tail && c < cols && finite_bits(last) ? code_of(last, inv, qmax) : 0);
  if (t == 0) scale[row] = scale_of(absmax, qmax);
}

inline int64_t up(int64_t v, int64_t a) { return (v + a - 1) / a * a; }

}  // namespace

template <typename T>
static void quantize_as(Ctx* ctx, const T* x, int64_t rows, int64_t cols, int64_t ld, float qmax, int8_t* q, int64_t ldq, float* scale, cudaStream_t st) {
  const bool vec = (uintptr_t)x % 16 == 0 && (rows == 1 || ld * (int64_t)sizeof(T) % 16 == 0);
  // a warp a row where a row fits its registers and there are rows enough to fill the GPU
  const bool narrow = rows >= 8 * sm_count(ctx) && cols <= 32 * (vec ? Vec<T>::N * held_pieces<T, true>() : held_pieces<T, false>());
  const dim3 grid((unsigned)(narrow ? (rows + 7) / 8 : rows)), block(kTokenThreads);
  const auto go = [&](auto kernel) { launch_pdl(kernel, grid, block, 0, st, x, rows, cols, ld, qmax, q, ldq, scale, err_word(ctx)); };
  if (narrow) vec ? go(quantize_tokens_kernel<T, 1, true>) : go(quantize_tokens_kernel<T, 1, false>);
  else vec ? go(quantize_tokens_kernel<T, 8, true>) : go(quantize_tokens_kernel<T, 8, false>);
}
int launch_quantize_tokens(Ctx* ctx, const void* x, int dtype, int64_t rows, int64_t cols, int64_t ld, int bits, int8_t* q, int64_t ldq, float* scale,
                           cudaStream_t st) {
  if (rows == 0) return QCFG_OK;
  const float qmax = qmax_of(bits);
  if (dtype == QCFG_FP32) quantize_as(ctx, (const float*)x, rows, cols, ld, qmax, q, ldq, scale, st);
  else if (dtype == QCFG_BF16) quantize_as(ctx, (const __nv_bfloat16*)x, rows, cols, ld, qmax, q, ldq, scale, st);
  else quantize_as(ctx, (const __half*)x, rows, cols, ld, qmax, q, ldq, scale, st);
  count_launch(ctx);
  return check_cuda(ctx, cudaGetLastError(), "quantize_tokens");
}

int launch_gemm_token(Ctx* ctx, const TokenGemm& t, cudaStream_t st) {
  GemmArgs g{};
  g.a = t.qx; g.lda = t.ldx; g.b = t.qw; g.ldb = t.ldw; g.m = t.m; g.n = t.n; g.k = t.k;
  g.scale_x = 1.0f; g.scale_w = t.sw; g.scale_rows = t.sx; g.bias = t.bias; g.act = t.act;
  g.y = (float*)t.y; g.ldy = t.ldy;
  g.y_kind = t.dtype == QCFG_FP32 ? 3 : t.dtype == QCFG_BF16 ? 2 : 5;
  return launch_gemm(ctx, g, st);
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
