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
                                                                        int8_t* __restrict__ q, int64_t ldq, float* __restrict__ scale, int late, unsigned* err) {
  // late: the next kernel may begin only once everything in front of this one has completed (see few_tokens_kernel)
  if (late) asm volatile("griddepcontrol.wait;\n\tgriddepcontrol.launch_dependents;" ::: "memory");
  else pdl_entry();
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

// ---- a few tokens: the weights are the traffic ---------------------------------------------------
//
// acc^T = W X^T with the 16 weight rows of a unit as the rows of an MMA (int8, sums exact in any order) and the tokens as its columns,
// NT tiles of 8.  One block per SM; its 16 warps share a unit's reduction, 128 bytes of a row at a time, and add up through shared
// memory.  A warp keeps the next kAhead steps (64 bytes of 16 rows) of weights on their way to its registers: 16 warps x 4 x 1 KB in
// flight per SM, asked for once and never cached in L1, where the tokens' codes stay.  A step's 16 bytes of a lane are
// operand words of two products as they lie in memory, of the weights and of the codes alike, since the sum may run in any order.
// Behind quantize_tokens (early) the first weights are fetched before its end: it lets this kernel begin only after everything in front
// of it has completed, so the weights are there.
// With X_RAW the tokens come as they are, and every block turns them into codes in shared memory while its first weights arrive.
constexpr int kFewWarps = 16, kAhead = 4;
constexpr int kRawElements = 16384, kRawTokens = 8;      // X_RAW up to this many

__device__ __forceinline__ uint4 load_once(const void* p) {
  uint4 v;
  asm volatile("ld.global.nc.L1::no_allocate.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "l"(p));
  return v;
}
__device__ __forceinline__ void mma_s8(int (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
  asm("mma.sync.aligned.m16n8k32.row.col.s32.s8.s8.s32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
      : "+r"(c[0]), "+r"(c[1]), "+r"(c[2]), "+r"(c[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

struct FewArgs {
  TokenGemm t;
  const void* x;       // X_RAW
  int64_t ldx;
  float qmax;
  int early;
  unsigned* err;
};

__host__ __device__ constexpr int raw_pitch(int64_t k) { return (int)((k + 15) / 16 * 16 + 16); }

template <typename TX, typename TY, int NT, bool X_RAW>
__global__ void __launch_bounds__(32 * kFewWarps, 1) few_tokens_kernel(const FewArgs a) {
  extern __shared__ __align__(16) uint8_t few_smem[];
  __shared__ float raw_scale[kRawTokens];
  __shared__ unsigned raw_top[kFewWarps];
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, g = lane >> 2, t4 = lane & 3;
  const int m = (int)a.t.m;
  const int64_t n = a.t.n;
  const int chunks = (int)((a.t.k + 15) / 16);                       // of 16 bytes
  const int rounds = (chunks + 8 * kFewWarps - 1) / (8 * kFewWarps);  // of 128 bytes per warp
  const int steps = (2 * rounds + kAhead - 1) / kAhead * kAhead;
  const int units = (int)((n + 15) / 16);
  int* sums = reinterpret_cast<int*>(few_smem);                      // [2][warp][NT * 4][32]
  int8_t* codes = reinterpret_cast<int8_t*>(few_smem + 2 * kFewWarps * NT * 512);

  if (!X_RAW && a.early) asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  else pdl_entry();

  // step i of a warp: chunks of the 128 bytes (i / 2) * 16 + warp, first or second half
  auto chunk_of = [&](int i) { return ((i >> 1) * kFewWarps + warp) * 8 + (i & 1) * 4 + t4; };
  int load_unit = blockIdx.x, load_step = 0;
  uint4 w[kAhead][2];
  auto fetch = [&](uint4 (&to)[2]) {
    const int c = chunk_of(load_step);
    to[0] = to[1] = make_uint4(0, 0, 0, 0);
    if (load_unit < units && c < chunks) {
      const int64_t r0 = (int64_t)load_unit * 16 + g, r1 = r0 + 8;
      if (r0 < n) to[0] = load_once(a.t.qw + r0 * a.t.ldw + c * 16);
      if (r1 < n) to[1] = load_once(a.t.qw + r1 * a.t.ldw + c * 16);
    }
    if (++load_step == steps) { load_step = 0; load_unit += gridDim.x; }
  };
#pragma unroll
  for (int i = 0; i < kAhead; ++i) fetch(w[i]);
  if (!X_RAW && a.early) asm volatile("griddepcontrol.wait;" ::: "memory");

  const int pitch = raw_pitch(a.t.k);
  if (X_RAW) {         // warp: part `part` of `parts` of token `tok`
    const int parts = kFewWarps / m, tok = warp / parts, part = warp - tok * parts;
    const TX* x = reinterpret_cast<const TX*>(a.x) + (int64_t)tok * a.ldx;
    const int k = (int)a.t.k;
    unsigned top = 0, odd = 0;
    if (tok < m)
      for (int c = part * 32 + lane; c < k; c += 32 * parts) {
        const unsigned b = abs_bits(to_float<TX>(x[c]));
        if (b < 0x7f800000u) top = b > top ? b : top; else odd = 1;
      }
    top = warp_max_u(top);
    if (lane == 0) raw_top[warp] = top;
    if (__syncthreads_or(odd) && tid == 0) atomicOr(a.err, ERR_NONFINITE);
    if (tok < m) {
      for (int p = 0; p < parts; ++p) top = raw_top[tok * parts + p] > top ? raw_top[tok * parts + p] : top;
      const float absmax = __uint_as_float(top), inv = inv_scale_of(absmax, a.qmax);
      for (int c = part * 32 + lane; c < pitch; c += 32 * parts) {
        const float f = c < k ? to_float<TX>(x[c]) : 0.0f;
        codes[tok * pitch + c] = (int8_t)(finite_bits(f) ? code_of(f, inv, a.qmax) : 0);
      }
      if (part == 0 && lane == 0) raw_scale[tok] = scale_of(absmax, a.qmax);
    }
    __syncthreads();
  }

  int buffer = 0;
  for (int unit = blockIdx.x; unit < units; unit += gridDim.x) {
    int acc[NT][4];
#pragma unroll
    for (int j = 0; j < NT; ++j)
#pragma unroll
      for (int c = 0; c < 4; ++c) acc[j][c] = 0;
    for (int i = 0; i < steps; i += kAhead) {
#pragma unroll
      for (int p = 0; p < kAhead; ++p) {
        const uint4 w0 = w[p][0], w1 = w[p][1];
        const int c = chunk_of(i + p);
        uint4 x[NT];
#pragma unroll
        for (int j = 0; j < NT; ++j) {
          const int tok = 8 * j + g;
          x[j] = make_uint4(0, 0, 0, 0);
          if (c < chunks && tok < m)
            x[j] = X_RAW ? *reinterpret_cast<const uint4*>(codes + tok * pitch + c * 16)
                         : __ldg(reinterpret_cast<const uint4*>(a.t.qx + (int64_t)tok * a.t.ldx + c * 16));
        }
        fetch(w[p]);
#pragma unroll
        for (int j = 0; j < NT; ++j) {
          mma_s8(acc[j], w0.x, w1.x, w0.y, w1.y, x[j].x, x[j].y);
          mma_s8(acc[j], w0.z, w1.z, w0.w, w1.w, x[j].z, x[j].w);
        }
      }
    }
    int* mine = sums + buffer * kFewWarps * NT * 128;
    buffer ^= 1;
#pragma unroll
    for (int j = 0; j < NT; ++j)
#pragma unroll
      for (int c = 0; c < 4; ++c) mine[(warp * NT * 4 + j * 4 + c) * 32 + lane] = acc[j][c];
    __syncthreads();                   // the other buffer is free behind it: everybody is done with the unit before
    for (int e = tid; e < 16 * m; e += 32 * kFewWarps) {
      const int tok = e >> 4, r = e & 15;
      const int64_t col = (int64_t)unit * 16 + r;
      if (col >= n) continue;
      const int* from = mine + ((tok >> 3) * 4 + (r >> 3) * 2 + (tok & 1)) * 32 + (r & 7) * 4 + ((tok & 7) >> 1);
      int sum = 0;
#pragma unroll
      for (int v = 0; v < kFewWarps; ++v) sum += from[v * NT * 128];
      float y = __fmul_rn((float)sum, __fmul_rn(X_RAW ? raw_scale[tok] : __ldg(a.t.sx + tok), __ldg(a.t.sw + col)));
      if (a.t.bias) y += __ldg(a.t.bias + col);
      if (a.t.act == QCFG_ACT_RELU) y = fmaxf(y, 0.0f);
      else if (a.t.act == QCFG_ACT_GELU_TANH) y = gelu_tanh(y);
      reinterpret_cast<TY*>(a.t.y)[(int64_t)tok * a.t.ldy + col] = from_float<TY>(y);
    }
  }
}

inline int64_t up(int64_t v, int64_t a) { return (v + a - 1) / a * a; }

}  // namespace

template <typename T>
static void quantize_as(Ctx* ctx, const T* x, int64_t rows, int64_t cols, int64_t ld, float qmax, int8_t* q, int64_t ldq, float* scale, int late, cudaStream_t st) {
  const bool vec = (uintptr_t)x % 16 == 0 && (rows == 1 || ld * (int64_t)sizeof(T) % 16 == 0);
  // a warp a row where a row fits its registers and there are rows enough to fill the GPU
  const bool narrow = rows >= 8 * sm_count(ctx) && cols <= 32 * (vec ? Vec<T>::N * held_pieces<T, true>() : held_pieces<T, false>());
  const dim3 grid((unsigned)(narrow ? (rows + 7) / 8 : rows)), block(kTokenThreads);
  const auto go = [&](auto kernel) { launch_pdl(kernel, grid, block, 0, st, x, rows, cols, ld, qmax, q, ldq, scale, late, err_word(ctx)); };
  if (narrow) vec ? go(quantize_tokens_kernel<T, 1, true>) : go(quantize_tokens_kernel<T, 1, false>);
  else vec ? go(quantize_tokens_kernel<T, 8, true>) : go(quantize_tokens_kernel<T, 8, false>);
}
static int quantize_rows(Ctx* ctx, const void* x, int dtype, int64_t rows, int64_t cols, int64_t ld, int bits, int8_t* q, int64_t ldq, float* scale,
                         int late, cudaStream_t st) {
  if (rows == 0) return QCFG_OK;
  const float qmax = qmax_of(bits);
  if (dtype == QCFG_FP32) quantize_as(ctx, (const float*)x, rows, cols, ld, qmax, q, ldq, scale, late, st);
  else if (dtype == QCFG_BF16) quantize_as(ctx, (const __nv_bfloat16*)x, rows, cols, ld, qmax, q, ldq, scale, late, st);
  else quantize_as(ctx, (const __half*)x, rows, cols, ld, qmax, q, ldq, scale, late, st);
  count_launch(ctx);
  return check_cuda(ctx, cudaGetLastError(), "quantize_tokens");
}
int launch_quantize_tokens(Ctx* ctx, const void* x, int dtype, int64_t rows, int64_t cols, int64_t ld, int bits, int8_t* q, int64_t ldq, float* scale,
                           cudaStream_t st) {
  return quantize_rows(ctx, x, dtype, rows, cols, ld, bits, q, ldq, scale, 0, st);
}

template <typename TX, typename TY, int NT, bool X_RAW>
static int few_as(Ctx* ctx, const FewArgs& a, cudaStream_t st) {
  const int smem = 2 * kFewWarps * NT * 512 + (X_RAW ? (int)a.t.m * raw_pitch(a.t.k) : 0);
  constexpr int most = 2 * kFewWarps * NT * 512 + (X_RAW ? 2 * kRawElements : 0);
  static DeviceOnce once;
  const cudaError_t e = once.smem(device_of(ctx), (const void*)few_tokens_kernel<TX, TY, NT, X_RAW>, most);
  if (e != cudaSuccess) return check_cuda(ctx, e, "linear_i8");
  const int64_t units = (a.t.n + 15) / 16;
  launch_pdl(few_tokens_kernel<TX, TY, NT, X_RAW>, dim3((unsigned)(units < sm_count(ctx) ? units : sm_count(ctx))), dim3(32 * kFewWarps), smem, st, a);
  count_launch(ctx);
  return check_cuda(ctx, cudaGetLastError(), "linear_i8");
}
template <typename TY>
static int few_codes(Ctx* ctx, const FewArgs& a, cudaStream_t st) {
  const int64_t m = a.t.m;
  if (m <= 8) return few_as<float, TY, 1, false>(ctx, a, st);
  if (m <= 16) return few_as<float, TY, 2, false>(ctx, a, st);
  if (m <= 24) return few_as<float, TY, 3, false>(ctx, a, st);
  if (m <= 32) return few_as<float, TY, 4, false>(ctx, a, st);
  return few_as<float, TY, 6, false>(ctx, a, st);
}
template <typename TX>
static int few_raw(Ctx* ctx, const FewArgs& a, cudaStream_t st) {
  return a.t.dtype == QCFG_FP32 ? few_as<TX, float, 1, true>(ctx, a, st) : a.t.dtype == QCFG_BF16 ? few_as<TX, __nv_bfloat16, 1, true>(ctx, a, st)
                                                                                                 : few_as<TX, __half, 1, true>(ctx, a, st);
}
constexpr int kFewTokens = 48;
static int launch_few(Ctx* ctx, const TokenGemm& t, int early, cudaStream_t st) {
  const FewArgs a{t, nullptr, 0, 0.0f, early, err_word(ctx)};
  return t.dtype == QCFG_FP32 ? few_codes<float>(ctx, a, st) : t.dtype == QCFG_BF16 ? few_codes<__nv_bfloat16>(ctx, a, st) : few_codes<__half>(ctx, a, st);
}

int launch_gemm_token(Ctx* ctx, const TokenGemm& t, cudaStream_t st) {
  if (t.m <= kFewTokens) return launch_few(ctx, t, 0, st);
  GemmArgs g{};
  g.a = t.qx; g.lda = t.ldx; g.b = t.qw; g.ldb = t.ldw; g.m = t.m; g.n = t.n; g.k = t.k;
  g.scale_x = 1.0f; g.scale_w = t.sw; g.scale_rows = t.sx; g.bias = t.bias; g.act = t.act;
  g.y = (float*)t.y; g.ldy = t.ldy;
  g.y_kind = t.dtype == QCFG_FP32 ? 3 : t.dtype == QCFG_BF16 ? 2 : 5;
  return launch_gemm(ctx, g, st);
}

// codes [m x ldq], then the scales
int64_t linear_work(int64_t m, int64_t k) { return m <= kRawTokens && m * k <= kRawElements ? 0 : up(m * up(k, 16), 256) + up(m * 4, 256); }
int launch_linear(Ctx* ctx, const void* x, int x_dtype, int64_t ldx, int bits, const TokenGemm& t_in, void* work, cudaStream_t st) {
  if (t_in.m <= kRawTokens && t_in.m * t_in.k <= kRawElements) {
    const FewArgs a{t_in, x, ldx, qmax_of(bits), 0, err_word(ctx)};
    return x_dtype == QCFG_FP32 ? few_raw<float>(ctx, a, st) : x_dtype == QCFG_BF16 ? few_raw<__nv_bfloat16>(ctx, a, st) : few_raw<__half>(ctx, a, st);
  }
  TokenGemm t = t_in;
  t.ldx = up(t.k, 16);
  int8_t* codes = (int8_t*)work;
  float* scale = (float*)(codes + up(t.m * t.ldx, 256));
  t.qx = codes;
  t.sx = scale;
  const int few = t.m <= kFewTokens;
  const int rc = quantize_rows(ctx, x, x_dtype, t.m, t.k, ldx, bits, codes, t.ldx, scale, few, st);
  return rc ? rc : few ? launch_few(ctx, t, 1, st) : launch_gemm_token(ctx, t, st);
}

}  // namespace qcfg
