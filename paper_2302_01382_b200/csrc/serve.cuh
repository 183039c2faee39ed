// Shared by the kernels that serve a model at 8 bits: element types, the paged cache as kernels see it, ragged batches.
#pragma once

#include <cuda_fp16.h>

#include <atomic>

#include "common.cuh"

namespace qcfg {

// Raises a kernel's shared-memory limit when a device first launches it (a driver call of a microsecond).
struct DeviceOnce {
  std::atomic<uint64_t> done{0};
  cudaError_t smem(int device, const void* kernel, int bytes) {
    const uint64_t bit = 1ull << (device & 63);
    if (device < 64 && (done.load(std::memory_order_acquire) & bit)) return cudaSuccess;
    const cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes);
    if (e == cudaSuccess && device < 64) done.fetch_or(bit, std::memory_order_release);
    return e;
  }
};

struct PoolView {
  int32_t* table;      // [max_seqs][max_pages]
  int32_t* len;
  int32_t* refs;
  int32_t n_pages, page, max_seqs, max_pages;
  int32_t* refused = nullptr;      // null: nothing is ever refused
};
struct CacheView {
  int8_t *k, *v;       // [n_pages][heads][page][dim]
  float *k_absmax, *v_absmax;
  int32_t heads, dim;
};
constexpr int kPlanMost = 8192;      // entries of a call that hands pages out
struct BatchView {
  const int32_t* seqs;
  const int32_t* starts;
  int32_t n;
  int64_t rows;
};

// ----- pages.cu -------------------------------------------------------------------------
int launch_kv_extend(Ctx* ctx, const PoolView& p, const BatchView& b, cudaStream_t st);
// Lays the pool out for n_seqs sequences of seq_len tokens (the last may be shorter), rows in all: fills table, len and
// refs of the pool and the batch over it.
int launch_kv_layout(Ctx* ctx, const PoolView& p, int32_t* seqs, int32_t* starts, int seq_len, int64_t rows, cudaStream_t st);
int launch_kv_free(Ctx* ctx, const PoolView& p, const int32_t* seqs, int n, cudaStream_t st);
int launch_kv_fork(Ctx* ctx, const PoolView& p, const int32_t* parents, const int32_t* children, int n, int32_t* src, int32_t* dst, cudaStream_t st);
int launch_kv_compact(Ctx* ctx, const PoolView& p, int32_t* map, cudaStream_t st);
int launch_kv_copy(Ctx* ctx, const PoolView& p, const CacheView& c, const int32_t* src, const int32_t* dst, int n, cudaStream_t st);
int launch_kv_append(Ctx* ctx, const PoolView& p, const CacheView& c, const BatchView& b, const void* k, const void* v, int dtype,
                     int64_t row_stride, int64_t head_stride, cudaStream_t st);
int launch_kv_read(Ctx* ctx, const PoolView& p, const CacheView& c, const BatchView& b, const int32_t* first, void* k, void* v, int dtype,
                   cudaStream_t st);

// ----- attention.cu ---------------------------------------------------------------------
int64_t kv_attention_work(Ctx* ctx, const CacheView& c, int max_len);
int launch_kv_attention(Ctx* ctx, const PoolView& p, const CacheView& c, const BatchView& b, const void* q, int64_t q_row, int64_t q_head,
                        int q_heads, void* out, int64_t o_row, int64_t o_head, int dtype, int max_rows, int max_len, float scale, int causal,
                        int window, void* work, cudaStream_t st);

// ----- token.cu ---------------------------------------------------------------------------
struct TokenGemm {       // y = act(float(qx qw^T) * (sx[m] * sw[n]) + bias[n])
  const int8_t* qx; int64_t ldx;
  const int8_t* qw; int64_t ldw;
  int64_t m, n, k;
  const float* sx;
  const float* sw;
  const float* bias;     // optional
  int act;
  void* y; int dtype; int64_t ldy;
  int64_t rows = 0;      // rows of qx that can be read, where there are more than m
  int early = 0;         // the kernel in front waits before it lets this one begin: qw may be read at once
};
int launch_quantize_tokens(Ctx* ctx, const void* x, int dtype, int64_t rows, int64_t cols, int64_t ld, int bits, int8_t* q, int64_t ldq, float* scale,
                           cudaStream_t st);
int launch_gemm_token(Ctx* ctx, const TokenGemm& t, cudaStream_t st);
int64_t linear_work(int64_t m, int64_t k);
// t.qx and t.sx are not read: the codes of x go through `work`
int launch_linear(Ctx* ctx, const void* x, int x_dtype, int64_t ldx, int bits, const TokenGemm& t, void* work, cudaStream_t st);

namespace {

constexpr float kQmax8 = 127.0f;

// Both scales of Eq. 1 at 8 bits from a maximum: one IEEE division each.
__device__ __forceinline__ float scale_of(float absmax, float qmax = kQmax8) { return absmax == 0.0f ? 1.0f : __fdiv_rn(absmax, qmax); }
__device__ __forceinline__ float inv_scale_of(float absmax, float qmax = kQmax8) { return absmax == 0.0f ? 1.0f : __fdiv_rn(qmax, absmax); }

// clamp(round_half_even(x * inv)) of a finite x.  The product is NaN only for x = 0 with an infinite inverse (a maximum
// below 2^-121): that is code 0.
__device__ __forceinline__ int code_of(float x, float inv, float qmax = kQmax8) {
  const float p = __fmul_rn(x, inv);
  return p == p ? __float2int_rn(fminf(fmaxf(p, -qmax), qmax)) : 0;
}
__device__ __forceinline__ bool finite_bits(float x) { return abs_bits(x) < 0x7f800000u; }

template <typename T> __device__ __forceinline__ float to_float(T v);
template <> __device__ __forceinline__ float to_float<float>(float v) { return v; }
template <> __device__ __forceinline__ float to_float<__nv_bfloat16>(__nv_bfloat16 v) { return __bfloat162float(v); }
template <> __device__ __forceinline__ float to_float<__half>(__half v) { return __half2float(v); }
template <typename T> __device__ __forceinline__ T from_float(float v);
template <> __device__ __forceinline__ float from_float<float>(float v) { return v; }
template <> __device__ __forceinline__ __nv_bfloat16 from_float<__nv_bfloat16>(float v) { return __float2bfloat16_rn(v); }
template <> __device__ __forceinline__ __half from_float<__half>(float v) { return __float2half_rn(v); }

// 16 bytes of T as floats
template <typename T> struct Vec { static constexpr int N = 16 / sizeof(T); };
template <typename T>
__device__ __forceinline__ void load_vec(const T* p, float (&f)[Vec<T>::N]) {
  union { uint4 u; T t[Vec<T>::N]; } w;
  w.u = __ldg(reinterpret_cast<const uint4*>(p));
#pragma unroll
  for (int i = 0; i < Vec<T>::N; ++i) f[i] = to_float<T>(w.t[i]);
}

// Rows [lo, hi) of entry i.  False: they are not rows of the tensors, or end before they begin; then there are none.
__device__ __forceinline__ bool entry_rows(const BatchView& b, int i, int64_t& lo, int64_t& hi) {
  if (b.starts) {
    lo = b.starts[i];
    hi = b.starts[i + 1];
  } else {
    lo = i;
    hi = i + 1;
  }
  const bool ok = lo >= 0 && lo <= hi && hi <= b.rows;
  if (!ok) lo = hi = 0;
  return ok;
}
// The table row of entry i, or -1 (none; out of range: reported)
__device__ __forceinline__ int entry_seq(const BatchView& b, const PoolView& p, int i, unsigned* err) {
  const int s = b.seqs[i];
  if (s < p.max_seqs) return s < 0 ? -1 : s;
  atomicOr(err, ERR_PAGE);
  return -1;
}
__device__ __forceinline__ int seq_len(const PoolView& p, int s) {
  const int64_t most = (int64_t)p.max_pages * p.page;
  const int len = p.len[s];
  return len < 0 ? 0 : (len > most ? (int)most : len);
}
// Exclusive prefix sum over a block of up to 1024 threads; `total` gets the sum.  `buf`: 33 integers of shared memory.
__device__ __forceinline__ int block_scan(int v, int* buf, int& total) {
  const int lane = threadIdx.x & 31, w = threadIdx.x >> 5, nw = (blockDim.x + 31) >> 5;
  int s = v;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int t = __shfl_up_sync(0xffffffffu, s, o);
    if (lane >= o) s += t;
  }
  __syncthreads();
  if (lane == 31) buf[w] = s;
  __syncthreads();
  if (w == 0) {
    int t = lane < nw ? buf[lane] : 0;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int u = __shfl_up_sync(0xffffffffu, t, o);
      if (lane >= o) t += u;
    }
    buf[lane] = t;
  }
  __syncthreads();
  total = buf[nw - 1];
  return s - v + (w ? buf[w - 1] : 0);
}

}  // namespace

}  // namespace qcfg
