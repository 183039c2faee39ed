// Linear layers with a scale for each token: codes of Eq. 1 row by row, and the int8 product whose rescale takes the row's scale.
#include <type_traits>

#include "serve.cuh"

namespace qcfg {

namespace {

// WPR warps (1 or 8) for each row, which they read once and keep in registers, as it came, while it fits: HELD pieces of 16 bytes a
// thread (2, 4 or 8: the fewer, the more rows are on their way).  What does not fit is read twice, the second time from L2.  With VEC
// false (rows not on 16-byte boundaries) a piece is cut out of the two aligned ones it lies in, at the row's ends element by element.
// HBM bounds it once an element costs no more than its share: clamp and round in two operations (magic number, low byte), the
// test for NaN, Inf and an infinite inverse once a row.  12288 x 768 bf16 21.3 -> 8.6 us against the first form, which held floats; fp32
// 10.5 us (4.5 TB/s).  1037 x 4001 fp16, rows off 16-byte boundaries: 11.7 us element by element, 8.0 this way.
constexpr int kTokenThreads = 256, kHeldMost = 8;
// Bytes of the codes of elements that are all finite, with a finite inverse
__device__ __forceinline__ uint32_t code_bits(float x, float inv, float qmax) {
  float c;
  asm("min.xorsign.abs.f32 %0, %1, %2;" : "=f"(c) : "f"(__fmul_rn(x, inv)), "f"(qmax));
  return __float_as_uint(__fadd_rn(c, 12582912.0f));
}
__device__ __forceinline__ uint32_t low_bytes(uint32_t a, uint32_t b, uint32_t c, uint32_t d) {
  return __byte_perm(__byte_perm(a, b, 0x0040), __byte_perm(c, d, 0x0040), 0x5410);
}
template <typename T, int WPR, int HELD, bool VEC>
__global__ void __launch_bounds__(kTokenThreads, HELD == 2 ? 6 : HELD == 4 ? 5 : 4) quantize_tokens_kernel(const T* __restrict__ x, int64_t rows, int64_t cols, int64_t ld, float qmax,
                                                                        int8_t* __restrict__ q, int64_t ldq, float* __restrict__ scale, int late, unsigned* err) {
  // late: the next kernel may begin only once everything in front of this one has completed (see few_tokens_kernel)
  if (late) asm volatile("griddepcontrol.wait;\n\tgriddepcontrol.launch_dependents;" ::: "memory");
  else pdl_entry();
  constexpr int V = Vec<T>::N, N = 32 * WPR;
  union Piece { uint4 u; T t[Vec<T>::N]; };
  __shared__ unsigned tops[8];
  const int64_t row = WPR == 8 ? (int64_t)blockIdx.x : (int64_t)blockIdx.x * 8 + (threadIdx.x >> 5);
  const int t = WPR == 8 ? threadIdx.x : threadIdx.x & 31;
  if (WPR == 1 && row >= rows) return;
  x += row * ld;
  q += row * ldq;
  const int pieces = (int)(cols / V);
  Piece held[HELD];
  unsigned top = 0;
  const int off = VEC ? 0 : (int)(reinterpret_cast<uintptr_t>(x) & 15);                  // bytes behind a boundary
  const int whole = VEC ? 0 : (int)((cols * (int64_t)sizeof(T) + off) / 16) - 1;       // pieces 1 .. whole - 1 lie in two aligned ones of the row
  auto get = [&](int p, Piece& f) {
    if (VEC || off == 0) {
      f.u = __ldg(reinterpret_cast<const uint4*>(x) + p);
    } else if (p >= 1 && p < whole) {
      const uint4* from = reinterpret_cast<const uint4*>(reinterpret_cast<const char*>(x) - off) + p;
      const uint4 a = __ldg(from), b = __ldg(from + 1);
      const uint32_t c[8] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
      uint32_t d[6], e[5];
#pragma unroll
      for (int i = 0; i < 6; ++i) d[i] = off & 8 ? c[i + 2] : c[i];
#pragma unroll
      for (int i = 0; i < 5; ++i) e[i] = off & 4 ? d[i + 1] : d[i];
      const uint32_t bits = 8 * (off & 3);
      f.u = make_uint4(__funnelshift_r(e[0], e[1], bits), __funnelshift_r(e[1], e[2], bits), __funnelshift_r(e[2], e[3], bits), __funnelshift_r(e[3], e[4], bits));
    } else {
#pragma unroll
      for (int j = 0; j < V; ++j) f.t[j] = x[(int64_t)p * V + j];
    }
  };
  auto largest = [&](const Piece& f) {        // a NaN or Inf orders above all others
#pragma unroll
    for (int j = 0; j < V; ++j) {
      const unsigned a = abs_bits(to_float<T>(f.t[j]));
      top = a > top ? a : top;
    }
  };
#pragma unroll
  for (int i = 0; i < HELD; ++i) {
    held[i].u = make_uint4(0, 0, 0, 0);
    if (t + i * N < pieces) get(t + i * N, held[i]);
  }
#pragma unroll
  for (int i = 0; i < HELD; ++i)
    if (t + i * N < pieces) largest(held[i]);
  Piece f;
  for (int p = t + HELD * N; p < pieces; p += N) {
    get(p, f);
    largest(f);
  }
  const int64_t tail = (int64_t)pieces * V + t;          // fewer than V elements
  Piece last;
  last.u = make_uint4(0, 0, 0, 0);
  if (tail < cols) last.t[0] = x[tail];
  {
    const unsigned a = abs_bits(to_float<T>(last.t[0]));
    top = a > top ? a : top;
  }
  auto over_row = [&](unsigned v) {
    v = __reduce_max_sync(0xffffffffu, v);
    if (WPR == 8) {
      __syncthreads();
      if ((t & 31) == 0) tops[t >> 5] = v;
      __syncthreads();
#pragma unroll
      for (int w = 0; w < 8; ++w) v = tops[w] > v ? tops[w] : v;
    }
    return v;
  };
  top = over_row(top);
  const bool odd = top >= 0x7f800000u;
  if (odd) {             // the largest of the others
    if (t == 0) atomicOr(err, ERR_NONFINITE);
    unsigned other = 0;
    for (int64_t c = t; c < cols; c += N) {
      const unsigned a = abs_bits(to_float<T>(x[c]));
      if (a < 0x7f800000u && a > other) other = a;
    }
    top = over_row(other);
  }
  const float absmax = __uint_as_float(top), inv = inv_scale_of(absmax, qmax);
  if (odd || !finite_bits(inv)) {
    for (int64_t c = t; c < ldq; c += N) {
      const float v = c < cols ? to_float<T>(x[c]) : 0.0f;
      q[c] = (int8_t)(finite_bits(v) ? code_of(v, inv, qmax) : 0);
    }
  } else {
    auto put = [&](int p, const Piece& f) {
      uint32_t b[Vec<T>::N];
#pragma unroll
      for (int j = 0; j < V; ++j) b[j] = code_bits(to_float<T>(f.t[j]), inv, qmax);
      int8_t* to = q + (int64_t)p * V;
      if constexpr (V == 8) *reinterpret_cast<uint2*>(to) = make_uint2(low_bytes(b[0], b[1], b[2], b[3]), low_bytes(b[4], b[5], b[6], b[7]));
      else *reinterpret_cast<uint32_t*>(to) = low_bytes(b[0], b[1], b[2], b[3]);
    };
#pragma unroll
    for (int i = 0; i < HELD; ++i)
      if (t + i * N < pieces) put(t + i * N, held[i]);
    for (int p = t + HELD * N; p < pieces; p += N) {
      get(p, f);
      put(p, f);
    }
    for (int64_t c = tail; c < ldq; c += N) q[c] = c == tail && c < cols ? (int8_t)code_bits(to_float<T>(last.t[0]), inv, qmax) : (int8_t)0;
  }
  if (t == 0) scale[row] = scale_of(absmax, qmax);
}

// ---- a few tokens: the weights are the traffic ---------------------------------------------------
//
// acc^T = W X^T with 16 weight rows as the rows of an MMA (int8, sums exact in any order) and the tokens as its columns, NT tiles of 8.
// One block per SM; it takes up to few_tiles<NT>() tiles of 16 rows at once, its 16 warps share their reduction, every 16th run of 128
// bytes to a warp, and add up through shared memory once at the end (a sum behind each tile of 16 rows cost as much as its weights).
// A step is one run of one tile, 2 KB: a warp copies it (cp.async) in whole lines into its own ring of kAhead steps, chunk c of row r at
// c ^ (r & 7), and takes the MMAs' operands from there with ldmatrix.  96 KB of weights are in flight per SM; the tokens' codes come from L1.
// Behind quantize_tokens (early) the first weights are fetched before its end: it lets this kernel begin only after everything in front
// of it has completed, so the weights are there.
// With X_RAW the tokens come as they are, and every block turns them into codes in shared memory while its first weights arrive.
constexpr int kFewWarps = 16, kAhead = 4, kStep = 2048;
constexpr int kRingBytes = kFewWarps * kAhead * kStep;
constexpr int kRawElements = 16384, kRawTokens = 8;      // X_RAW up to this many
template <int NT> __host__ __device__ constexpr int few_tiles() { return NT == 1 ? 8 : 4; }      // accumulators: NT x 4 registers each
template <int NT> __host__ __device__ constexpr int sum_tiles() { return NT <= 2 ? 4 : 2; }      // tiles added up at a time
template <int NT> __host__ __device__ constexpr int few_bytes() {      // the ring, and the sums in its place once it is empty
  return kRingBytes > kFewWarps * sum_tiles<NT>() * NT * 512 ? kRingBytes : kFewWarps * sum_tiles<NT>() * NT * 512;
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
  constexpr int RT = few_tiles<NT>(), ST = sum_tiles<NT>();
  extern __shared__ __align__(16) uint8_t few_smem[];
  __shared__ float raw_scale[kRawTokens];
  __shared__ unsigned raw_top[kFewWarps];
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, g = lane >> 2, t4 = lane & 3;
  const int m = (int)a.t.m;
  const int64_t n = a.t.n;
  const int chunks = (int)((a.t.k + 15) / 16);                       // of 16 bytes
  const int runs_all = (chunks + 7) / 8, runs = runs_all > warp ? (runs_all - warp + kFewWarps - 1) / kFewWarps : 0;
  // this block's tiles
  const int64_t tiles = (n + 15) / 16;
  const int tile_lo = (int)(tiles * blockIdx.x / gridDim.x), tile_hi = (int)(tiles * (blockIdx.x + 1) / gridDim.x);
  int* sums = reinterpret_cast<int*>(few_smem);                      // [warp][tile][NT * 4][32]
  int8_t* codes = reinterpret_cast<int8_t*>(few_smem + few_bytes<NT>());
  const uint32_t ring = (uint32_t)__cvta_generic_to_shared(few_smem) + warp * kAhead * kStep;

  if (!X_RAW && a.early) asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  else pdl_entry();

  // the weights of a pass (up to RT tiles), run by run, tile by tile
  int pass_lo = tile_lo, count = min(RT, tile_hi - tile_lo), load_run = 0, load_tile = 0;
  uint32_t fill = 0;
  const uint32_t put_even = (lane >> 3) * 128 + (((lane & 7) ^ (lane >> 3)) << 4), put_odd = put_even ^ 64u;      // rows 0-3 and 8-11, 4-7 and 12-15
  auto fetch = [&]() {
    if (load_run < runs) {
      const int c = min((load_run * kFewWarps + warp) * 8 + (lane & 7), chunks - 1);      // chunks behind the last meet codes of zero
      const int64_t r0 = (int64_t)(pass_lo + load_tile) * 16 + (lane >> 3);
#pragma unroll
      for (int i = 0; i < 4; ++i) {      // rows behind the last are read as the last; their sums go nowhere
        const int64_t r = min(r0 + 4 * i, n - 1);
        asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(ring + (i & 1 ? put_odd : put_even) + fill + i * 512), "l"(a.t.qw + r * a.t.ldw + c * 16) : "memory");
      }
      if (++load_tile == count) { load_tile = 0; ++load_run; }
    }
    fill = fill == (kAhead - 1) * kStep ? 0 : fill + kStep;
    asm volatile("cp.async.commit_group;" ::: "memory");
  };
#pragma unroll
  for (int i = 0; i < kAhead - 1; ++i) fetch();
  if (!X_RAW && a.early) asm volatile("griddepcontrol.wait;" ::: "memory");

  const int pitch = raw_pitch(a.t.k);
  if (X_RAW) {         // warp: part `part` of `parts` of token `tok`
    const int parts = kFewWarps / m, tok = warp / parts, part = warp - tok * parts;
    const TX* x = reinterpret_cast<const TX*>(a.x) + (int64_t)tok * a.ldx;
    const int k = (int)a.t.k;
    // pieces of 16 bytes, kept in registers, where all rows allow it: kRawElements over the block's threads at most
    constexpr int V = Vec<TX>::N, HELD = kRawElements / (32 * kFewWarps) / V;
    const bool vec = ((uintptr_t)a.x | (uintptr_t)(a.ldx * sizeof(TX))) % 16 == 0 && k % V == 0 && HELD * parts * 32 * V >= k;
    float held[HELD][V];
    unsigned top = 0, odd = 0;
    auto see = [&](float f) {
      const unsigned b = abs_bits(f);
      if (b < 0x7f800000u) top = b > top ? b : top; else odd = 1;
    };
    if (tok < m) {
      if (vec) {
#pragma unroll
        for (int i = 0; i < HELD; ++i) {
          const int c = ((i * parts + part) * 32 + lane) * V;
          if (c < k) load_vec<TX>(x + c, held[i]);
          else {
#pragma unroll
            for (int j = 0; j < V; ++j) held[i][j] = 0.0f;
          }
        }
#pragma unroll
        for (int i = 0; i < HELD; ++i)
#pragma unroll
          for (int j = 0; j < V; ++j) see(held[i][j]);
      } else {
        for (int c = part * 32 + lane; c < k; c += 32 * parts) see(to_float<TX>(x[c]));
      }
    }
    top = warp_max_u(top);
    if (lane == 0) raw_top[warp] = top;
    if (__syncthreads_or(odd) && tid == 0) atomicOr(a.err, ERR_NONFINITE);
    if (tok < m) {
      for (int p = 0; p < parts; ++p) top = raw_top[tok * parts + p] > top ? raw_top[tok * parts + p] : top;
      const float absmax = __uint_as_float(top), inv = inv_scale_of(absmax, a.qmax);
      auto code = [&](float f) { return (int8_t)(finite_bits(f) ? code_of(f, inv, a.qmax) : 0); };
      if (vec) {
#pragma unroll
        for (int i = 0; i < HELD; ++i) {
          const int c = ((i * parts + part) * 32 + lane) * V;
          if (c >= k) continue;
          union { uint2 w2; uint32_t w; int8_t b[8]; } o;
#pragma unroll
          for (int j = 0; j < V; ++j) o.b[j] = code(held[i][j]);
          if (V == 8) *reinterpret_cast<uint2*>(codes + tok * pitch + c) = o.w2;
          else *reinterpret_cast<uint32_t*>(codes + tok * pitch + c) = o.w;
        }
        for (int c = k + part * 32 + lane; c < pitch; c += 32 * parts) codes[tok * pitch + c] = 0;
      } else {
        for (int c = part * 32 + lane; c < pitch; c += 32 * parts) codes[tok * pitch + c] = c < k ? code(to_float<TX>(x[c])) : (int8_t)0;
      }
      if (part == 0 && lane == 0) raw_scale[tok] = scale_of(absmax, a.qmax);
    }
    __syncthreads();
  }

  // this lane's tokens; those behind the last are read as the last, their sums go nowhere
  const int8_t* token[NT];
#pragma unroll
  for (int j = 0; j < NT; ++j) {
    const int tok = min(8 * j + g, m - 1);
    token[j] = X_RAW ? codes + tok * pitch : a.t.qx + (int64_t)tok * a.t.ldx;
  }
  uint32_t drain = 0;
  // lanes 8 i .. 8 i + 7 give the rows of matrix i: rows 0-7 and 8-15 of the first 16 bytes, then of the next
  const uint32_t get_row = lane & 15, get_at = ring + get_row * 128, get_flip = (lane >> 4) ^ (get_row & 7);
  for (;;) {
    int acc[RT][NT][4];
#pragma unroll
    for (int r = 0; r < RT; ++r)
#pragma unroll
      for (int j = 0; j < NT; ++j)
#pragma unroll
        for (int c = 0; c < 4; ++c) acc[r][j][c] = 0;
    for (int i = 0; i < runs; ++i) {
      const int c = (i * kFewWarps + warp) * 8;
      uint32_t x[4][NT][2];              // [32 bytes][tokens][half]
#pragma unroll
      for (int k = 0; k < 4; ++k)
#pragma unroll
        for (int j = 0; j < NT; ++j)
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            const uint32_t* from = reinterpret_cast<const uint32_t*>(token[j] + (c + 2 * k + h) * 16) + t4;
            x[k][j][h] = 0;
            if (c + 2 * k + h < chunks) x[k][j][h] = X_RAW ? *from : __ldg(from);
          }
#pragma unroll
      for (int r = 0; r < RT; ++r) {
        if (r >= count) break;
        asm volatile("cp.async.wait_group %0;" ::"n"(kAhead - 2) : "memory");
        __syncwarp();                    // the step has arrived for all lanes, and all are done with the one before
        fetch();
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          uint32_t w[4];
          asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0,%1,%2,%3}, [%4];"
                       : "=r"(w[0]), "=r"(w[1]), "=r"(w[2]), "=r"(w[3]) : "r"(get_at + drain + ((get_flip ^ (2 * k)) << 4)));
#pragma unroll
          for (int j = 0; j < NT; ++j) mma_s8(acc[r][j], w[0], w[1], w[2], w[3], x[k][j][0], x[k][j][1]);
        }
        drain = drain == (kAhead - 1) * kStep ? 0 : drain + kStep;
      }
    }
    asm volatile("cp.async.wait_group 0;" ::: "memory");
#pragma unroll
    for (int r0 = 0; r0 < RT; r0 += ST) {
      if (r0 >= count) break;
      __syncthreads();                 // the ring is empty, or the tiles before have been added up
#pragma unroll
      for (int r = r0; r < r0 + ST && r < RT; ++r)
#pragma unroll
        for (int j = 0; j < NT; ++j)
#pragma unroll
          for (int c = 0; c < 4; ++c)
            if (r < count) sums[((warp * ST + r - r0) * NT * 4 + j * 4 + c) * 32 + lane] = acc[r][j][c];
      __syncthreads();
      const int here = min(ST, count - r0) * 16;             // rows
      for (int e = tid; e < here * m; e += 32 * kFewWarps) {
        const int tok = e / here, row = e - tok * here, r = row & 15;
        const int64_t col = (int64_t)(pass_lo + r0) * 16 + row;
        if (col >= n) continue;
        const int* from = sums + (row >> 4) * NT * 128 + ((tok >> 3) * 4 + (r >> 3) * 2 + (tok & 1)) * 32 + (r & 7) * 4 + ((tok & 7) >> 1);
        int sum = 0;
#pragma unroll
        for (int v = 0; v < kFewWarps; ++v) sum += from[v * ST * NT * 128];
        float y = __fmul_rn((float)sum, __fmul_rn(X_RAW ? raw_scale[tok] : __ldg(a.t.sx + tok), __ldg(a.t.sw + col)));
        if (a.t.bias) y += __ldg(a.t.bias + col);
        if (a.t.act == QCFG_ACT_RELU) y = fmaxf(y, 0.0f);
        else if (a.t.act == QCFG_ACT_GELU_TANH) y = gelu_tanh(y);
        reinterpret_cast<TY*>(a.t.y)[(int64_t)tok * a.t.ldy + col] = from_float<TY>(y);
      }
    }
    pass_lo += count;
    if (pass_lo >= tile_hi) return;
    count = min(RT, tile_hi - pass_lo);
    load_run = load_tile = 0;
    fill = drain = 0;                  // (the empty fetches behind a pass's last step have moved one and not the other)
    __syncthreads();                   // the sums have been read
#pragma unroll
    for (int i = 0; i < kAhead - 1; ++i) fetch();
  }
}

inline int64_t up(int64_t v, int64_t a) { return (v + a - 1) / a * a; }

}  // namespace

template <typename T>
static void quantize_as(Ctx* ctx, const T* x, int64_t rows, int64_t cols, int64_t ld, float qmax, int8_t* q, int64_t ldq, float* scale, int late, cudaStream_t st) {
  const bool vec = (uintptr_t)x % 16 == 0 && (rows == 1 || ld * (int64_t)sizeof(T) % 16 == 0);
  // a warp a row where a row fits its registers and there are rows enough to fill the GPU
  const int64_t pieces = (cols + Vec<T>::N - 1) / Vec<T>::N;
  const bool narrow = rows >= 8 * sm_count(ctx) && pieces <= 32 * kHeldMost;
  const int64_t each = (pieces + (narrow ? 31 : 255)) / (narrow ? 32 : 256);      // of a thread
  const dim3 grid((unsigned)(narrow ? (rows + 7) / 8 : rows)), block(kTokenThreads);
  const auto go = [&](auto kernel) { launch_pdl(kernel, grid, block, 0, st, x, rows, cols, ld, qmax, q, ldq, scale, late, err_word(ctx)); };
  const auto held = [&](auto warps, auto aligned) {
    constexpr int W = decltype(warps)::value;
    constexpr bool A = decltype(aligned)::value;
    if (each <= 2) go(quantize_tokens_kernel<T, W, 2, A>);
    else if (each <= 4) go(quantize_tokens_kernel<T, W, 4, A>);
    else go(quantize_tokens_kernel<T, W, 8, A>);
  };
  using Yes = std::true_type;
  using No = std::false_type;
  using One = std::integral_constant<int, 1>;
  using Eight = std::integral_constant<int, 8>;
  if (narrow) vec ? held(One(), Yes()) : held(One(), No());
  else vec ? held(Eight(), Yes()) : held(Eight(), No());
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
  const int smem = few_bytes<NT>() + (X_RAW ? (int)a.t.m * raw_pitch(a.t.k) : 0);
  constexpr int most = few_bytes<NT>() + (X_RAW ? kRawElements + 32 * kRawTokens : 0);
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
  if (a.t.m <= 8) return few_as<float, TY, 1, false>(ctx, a, st);
  if (a.t.m <= 16) return few_as<float, TY, 2, false>(ctx, a, st);
  return a.t.m <= 24 ? few_as<float, TY, 3, false>(ctx, a, st) : few_as<float, TY, 4, false>(ctx, a, st);
}
template <typename TX>
static int few_raw(Ctx* ctx, const FewArgs& a, cudaStream_t st) {
  return a.t.dtype == QCFG_FP32 ? few_as<TX, float, 1, true>(ctx, a, st) : a.t.dtype == QCFG_BF16 ? few_as<TX, __nv_bfloat16, 1, true>(ctx, a, st)
                                                                                                 : few_as<TX, __half, 1, true>(ctx, a, st);
}
// Whether a product goes this way or in the GEMM's tiles of 128 rows.  us, this way / tiles, codes ready, other weights with each call, so that
// they come from HBM, tokens x k x n:
//   1 x 4096 x 16384 13.0 / 15.2    8 x 4096 x 16384 14.2 / 15.3    8 x 4096 x 50257 39.7 / 47.0    8 x 768 x 3072 2.8 / 4.7
//   16 x 4096 x 16384 16.0 / 15.2   16 x 2048 x 32000 19.5 / 15.7   24 x 4096 x 16384 21.2 / 15.3   32 x 4096 x 16384 29.1 / 15.2
//   16 x 1024 x 4096 3.9 / 5.5      24 x 768 x 768 3.0 / 4.4        24 x 1024 x 4096 4.6 / 5.5      24 x 4096 x 4096 9.3 / 11.1
//   24 x 16384 x 4096 22.0 / 33.6   24 x 8192 x 8192 18.2 / 19.9    32 x 16384 x 4096 30.4 / 33.7   17 x 4096 x 9472 12.5 / 12.3
// The GEMM narrows its tiles to 64 columns and fewer for up to 64 columns a SM, and its ring of eight stages then holds too few weights.
static bool few_pays(Ctx* ctx, int64_t m, int64_t n) { return m <= 8 || (m <= 32 && n <= 64 * (int64_t)sm_count(ctx)); }
static int launch_few(Ctx* ctx, const TokenGemm& t, cudaStream_t st) {
  const FewArgs a{t, nullptr, 0, 0.0f, t.early, err_word(ctx)};
  return t.dtype == QCFG_FP32 ? few_codes<float>(ctx, a, st) : t.dtype == QCFG_BF16 ? few_codes<__nv_bfloat16>(ctx, a, st) : few_codes<__half>(ctx, a, st);
}

int launch_gemm_token(Ctx* ctx, const TokenGemm& t, cudaStream_t st) {
  if (few_pays(ctx, t.m, t.n)) return launch_few(ctx, t, st);
  GemmArgs g{};
  g.a = t.qx; g.lda = t.ldx; g.b = t.qw; g.ldb = t.ldw; g.m = t.m; g.n = t.n; g.k = t.k; g.a_rows = t.rows; g.b_early = t.early;
  g.scale_x = 1.0f; g.scale_w = t.sw; g.scale_rows = t.sx; g.bias = t.bias; g.act = t.act;
  g.y = (float*)t.y; g.ldy = t.ldy;
  g.y_kind = t.dtype == QCFG_FP32 ? 3 : t.dtype == QCFG_BF16 ? 2 : 5;
  return launch_gemm(ctx, g, st);
}

constexpr int kCodePitch = 128;      // rows of whole lines, for the TMA loads: 1037 x 4001 by 2311 26.8 -> 24.6 us against the next multiple of 16
// codes [m x ldq] and room up to a multiple of 32 rows (see GemmArgs::a_rows), then the scales
int64_t linear_work(int64_t m, int64_t k) { return m <= kRawTokens && m * k <= kRawElements ? 0 : up(up(m, 32) * up(k, kCodePitch), 256) + up(m * 4, 256); }
int launch_linear(Ctx* ctx, const void* x, int x_dtype, int64_t ldx, int bits, const TokenGemm& t_in, void* work, cudaStream_t st) {
  if (t_in.m <= kRawTokens && t_in.m * t_in.k <= kRawElements) {
    const FewArgs a{t_in, x, ldx, qmax_of(bits), 0, err_word(ctx)};
    return x_dtype == QCFG_FP32 ? few_raw<float>(ctx, a, st) : x_dtype == QCFG_BF16 ? few_raw<__nv_bfloat16>(ctx, a, st) : few_raw<__half>(ctx, a, st);
  }
  TokenGemm t = t_in;
  t.ldx = up(t.k, kCodePitch);
  int8_t* codes = (int8_t*)work;
  t.rows = up(t.m, 32);
  float* scale = (float*)(codes + up(t.rows * t.ldx, 256));
  t.qx = codes;
  t.sx = scale;
  t.early = 1;
  const int rc = quantize_rows(ctx, x, x_dtype, t.m, t.k, ldx, bits, codes, t.ldx, scale, 1, st);
  return rc ? rc : launch_gemm_token(ctx, t, st);
}

}  // namespace qcfg
