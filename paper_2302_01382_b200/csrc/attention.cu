// Attention over the paged 8-bit cache: out = softmax(sm_scale * q k^T) v with k = code * A_k / 127, v = code * A_v / 127, A the
// maximum of the token's page and head.
#include "serve.cuh"

namespace qcfg {

namespace {

struct AttnArgs {
  PoolView pool;
  CacheView cache;
  BatchView batch;
  const void* q;
  void* out;
  int64_t q_row, q_head, o_row, o_head;
  int q_heads, causal, window;
  float scale;
  unsigned* err;
};

// The tokens a row sees: [lo, hi), empty as hi <= lo.
__device__ __forceinline__ void seen_range(const AttnArgs& a, int64_t pos, int len, int& lo, int& hi) {
  hi = a.causal ? (int)(pos + 1) : len;
  lo = a.window > 0 && pos + 1 > a.window ? (int)(pos + 1) - a.window : 0;
  if (pos < 0) hi = 0;
}

// A warp for each row and head: a token at a time, one running maximum.
constexpr int kWarps = 4;
template <typename T>
__global__ void __launch_bounds__(32 * kWarps) kv_attention_rows(AttnArgs a) {
  pdl_entry();
  const int lane = threadIdx.x & 31;
  const int64_t row = blockIdx.x;
  const int h = blockIdx.y * kWarps + (threadIdx.x >> 5);
  if (h >= a.q_heads) return;
  int i = (int)row;
  if (a.batch.starts) {
    int count = 0;
    for (int e = lane; e < a.batch.n; e += 32) count += a.batch.starts[e] <= row;
    i = __reduce_add_sync(0xffffffffu, count) - 1;
  }
  if (i < 0 || i >= a.batch.n) return;
  int64_t r0, r1;
  entry_rows(a.batch, i, r0, r1);
  if (row >= r1) return;
  const int s = entry_seq(a.batch, a.pool, i, a.err);
  const int len = s < 0 ? 0 : seq_len(a.pool, s);
  int lo, hi;
  seen_range(a, len - (r1 - row), len, lo, hi);
  const int dim = a.cache.dim, hk = h / (a.q_heads / a.cache.heads), page = a.pool.page;
  const T* q = (const T*)a.q + row * a.q_row + h * a.q_head;
  float qv[8], acc[8], top = -INFINITY, sum = 0.0f;
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    qv[j] = lane + 32 * j < dim ? to_float<T>(q[lane + 32 * j]) : 0.0f;
    acc[j] = 0.0f;
  }
  for (int t = lo; t < hi; ++t) {
    const int number = a.pool.table[(int64_t)s * a.pool.max_pages + t / page];
    if (number < 0 || number >= a.pool.n_pages) {
      if (lane == 0) atomicOr(a.err, ERR_PAGE);
      continue;
    }
    const int64_t block = (int64_t)number * a.cache.heads + hk, at = (block * page + t % page) * dim;
    float dot = 0.0f;
#pragma unroll
    for (int j = 0; j < 8; ++j)
      if (lane + 32 * j < dim) dot = fmaf(qv[j], (float)a.cache.k[at + lane + 32 * j], dot);
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) dot += __shfl_xor_sync(0xffffffffu, dot, o);
    const float x = dot * scale_of(a.cache.k_absmax[block]) * a.scale;
    const float now = fmaxf(top, x), keep = expf(top - now), e = expf(x - now), w = e * scale_of(a.cache.v_absmax[block]);
    sum = sum * keep + e;
    top = now;
#pragma unroll
    for (int j = 0; j < 8; ++j)
      if (lane + 32 * j < dim) acc[j] = acc[j] * keep + w * (float)a.cache.v[at + lane + 32 * j];
  }
  T* out = (T*)a.out + row * a.o_row + h * a.o_head;
#pragma unroll
  for (int j = 0; j < 8; ++j)
    if (lane + 32 * j < dim) out[lane + 32 * j] = from_float<T>(sum == 0.0f ? 0.0f : acc[j] / sum);
}

template <typename T>
void rows_as(const AttnArgs& a, cudaStream_t st) {
  launch_pdl(kv_attention_rows<T>, dim3((unsigned)a.batch.rows, (a.q_heads + kWarps - 1) / kWarps), dim3(32 * kWarps), 0, st, a);
}

}  // namespace

int64_t kv_attention_work(Ctx*, const CacheView&, int, int64_t, int) { return 0; }

int launch_kv_attention(Ctx* ctx, const PoolView& p, const CacheView& c, const BatchView& b, const void* q, int64_t q_row, int64_t q_head,
                        int q_heads, void* out, int64_t o_row, int64_t o_head, int dtype, int, int, float scale, int causal, int window, void*,
                        cudaStream_t st) {
  if (b.n == 0 || b.rows == 0) return QCFG_OK;
  const AttnArgs a{p, c, b, q, out, q_row, q_head, o_row, o_head, q_heads, causal, window, scale, err_word(ctx)};
  if (dtype == QCFG_FP32) rows_as<float>(a, st);
  else if (dtype == QCFG_BF16) rows_as<__nv_bfloat16>(a, st);
  else rows_as<__half>(a, st);
  count_launch(ctx);
  return check_cuda(ctx, cudaGetLastError(), "kv_attention");
}

}  // namespace qcfg
