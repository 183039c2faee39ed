// Attention over the paged 8-bit cache: out = softmax(sm_scale * q k^T) v with k = code * A_k / 127, v = code * A_v / 127, A the
// maximum of the token's page and head.
//
// The codes go to the tensor cores as fp16, which holds them exactly, and never exist as numbers of 16 bits in memory: a page's
// scale multiplies the finished scores (keys) or the weights (values).  Queries are fp16 after a power of two has brought
// their row's largest element to 2^12 .. 2^13, so bf16 and fp16 ones lose nothing above 2^-38 of the row; fp32 ones are the sum
// of two fp16 numbers.  Weights are e = 2^(14 + x - max) times the page's share of the largest value scale seen, in fp16
// (fp32 calls: the sum of two), which leaves 28 binary orders below the largest weight before the fp16 grid coarsens.
#include <algorithm>

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
  float scale;              // sm_scale * log2(e)
  void* work;
  unsigned* err;
};

// The tokens the row at position pos sees: [lo, hi), empty as hi <= lo.
__device__ __forceinline__ void seen_range(const AttnArgs& a, int64_t pos, int len, int& lo, int& hi) {
  hi = pos < 0 ? 0 : a.causal ? (int)(pos + 1) : len;
  lo = a.window > 0 && pos + 1 > a.window ? (int)(pos + 1) - a.window : 0;
}

// ---- few rows: warps stream the cache -----------------------------------------------------------
//
// Work is counted in units of 64 tokens of one (entry, cache head, tile of 16 rows); a row is a (query token, head of the
// group).  All units of a call form one sequence that the resident blocks share evenly, so a ragged batch, a single long context and many
// short ones load the GPU alike.  A block works through its units segment by segment (a segment: units of one tile); a tile cut
// between blocks leaves its parts in `work`, and a second kernel joins them in a fixed order.
// Within a segment each of the four warps takes every fourth run of 32 tokens, with its own ring of stages (cp.async) and its own
// running maximum: nothing is synchronised until the segment ends.
constexpr int kUnit = 64;           // tokens
constexpr int kRun = 32;            // tokens a warp takes at a time
constexpr int kRows = 16;           // rows of a tile (M of the MMA)
constexpr int kStreamWarps = 4;
constexpr int kMinUnits = 2;        // a block takes at least this many
constexpr float kWeightBias = 14.0f;

template <int DP> __host__ __device__ constexpr int stream_stages() { return DP == 64 ? 4 : 3; }
template <int DP> __host__ __device__ constexpr int stage_bytes() { return 2 * kRun * DP + 32; }             // keys, values, four maxima
template <int DP> __host__ __device__ constexpr int stream_blocks() { return DP == 256 ? 1 : 2; }            // per SM
template <int DP, bool WIDE> __host__ __device__ constexpr int query_bytes() { return (WIDE ? 2 : 1) * kRows * DP * 2; }
template <int DP, bool WIDE>
__host__ __device__ constexpr int stream_smem() {
  return query_bytes<DP, WIDE>() + kStreamWarps * stream_stages<DP>() * stage_bytes<DP>();
}
constexpr int kMaxStreamGrid = 148 * 2;

struct PartMeta {         // of a block: the cut tile that its first segment finishes
  int64_t row0;           // first row of the entry
  int first;              // block that holds the tile's first part, -1: none
  int rows, tile, head;
  int pad[2];
};
template <int DP> __host__ __device__ constexpr int64_t part_floats() { return kRows * DP + 2 * kRows; }     // accumulators, maxima, sums

__device__ __forceinline__ uint32_t h2_bits(__half2 h) { return *reinterpret_cast<uint32_t*>(&h); }
__device__ __forceinline__ uint32_t pack_h2(float a, float b) { return h2_bits(__floats2half2_rn(a, b)); }
__device__ __forceinline__ float ex2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
__device__ __forceinline__ void mma16816(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
  asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
               : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
// Bytes `lo`, `hi` (selector 0x4H4L) of a word of codes plus 128 as two fp16 codes: 0x6400 + b is 1024 + b
template <uint32_t SEL>
__device__ __forceinline__ uint32_t two_codes(uint32_t biased) {
  const uint32_t w = __byte_perm(biased, 0x64646464u, SEL);
  const __half2 off = __floats2half2_rn(1152.0f, 1152.0f);
  return h2_bits(__hsub2(*reinterpret_cast<const __half2*>(&w), off));
}
__device__ __forceinline__ void cp_async16(uint32_t dst, const void* src) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(src) : "memory");
}
__device__ __forceinline__ void cp_async4(uint32_t dst, const void* src) {
  asm volatile("cp.async.ca.shared.global [%0], [%1], 4;" ::"r"(dst), "l"(src) : "memory");
}
__device__ __forceinline__ void cp_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N> __device__ __forceinline__ void cp_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }
__device__ __forceinline__ uint32_t smem_at(const void* p) { return (uint32_t)__cvta_generic_to_shared(p); }
__device__ __forceinline__ uint4 lds128(uint32_t a) {
  uint4 v;
  asm volatile("ld.shared.v4.b32 {%0,%1,%2,%3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(a));
  return v;
}
__device__ __forceinline__ uint2 lds64(uint32_t a) {
  uint2 v;
  asm volatile("ld.shared.v2.b32 {%0,%1}, [%2];" : "=r"(v.x), "=r"(v.y) : "r"(a));
  return v;
}

// Where 16-byte chunk `chunk` of token `row` (0..31) of a run lies.  A warp reads keys as rows {0,4},{1,5},.. x four chunks and values as rows
// 0..3 or 4..7 x neighbouring chunks (16 or 8 bytes): the exclusive-or keeps both free of bank conflicts.
template <int DP>
__device__ __forceinline__ uint32_t chunk_at(int row, int chunk) {
  if (DP == 64) return (uint32_t)((row >> 1) * 128 + ((((row & 1) << 2) | chunk) ^ (2 * ((row >> 1) & 3))) * 16);
  const int f = (2 * (row & 3)) ^ (row & 4);
  return (uint32_t)(row * DP + (chunk & ~7) * 16 + ((chunk & 7) ^ f) * 16);
}

// What an entry of the batch asks for.
struct Entry {
  int64_t row0, rows;
  int s, len, tiles, units;      // tiles of 16 rows, units per tile and head
};
__device__ __forceinline__ Entry entry_of(const AttnArgs& a, int i) {
  Entry e;
  int64_t hi;
  entry_rows(a.batch, i, e.row0, hi);
  e.rows = hi - e.row0;
  e.s = a.batch.seqs[i];
  e.len = e.s < 0 || e.s >= a.pool.max_seqs ? 0 : seq_len(a.pool, e.s);
  e.tiles = (int)((e.rows * (a.q_heads / a.cache.heads) + kRows - 1) / kRows);
  e.units = e.len ? (e.len + kUnit - 1) / kUnit : 1;
  return e;
}
__device__ __forceinline__ int64_t entry_units(const AttnArgs& a, const Entry& e) { return (int64_t)e.tiles * e.units * a.cache.heads; }

// First unit of block b of `blocks` sharing `total`
__device__ __forceinline__ int64_t share_at(int64_t total, int blocks, int b) { return total / blocks * b + min((int64_t)b, total % blocks); }
__device__ __forceinline__ int share_of(int64_t total, int blocks, int64_t unit) {      // the block that has it
  const int64_t each = total / blocks, more = total % blocks;
  return unit < more * (each + 1) ? (int)(unit / (each + 1)) : (int)(more + (unit - more * (each + 1)) / each);
}

template <typename T, int DP>
__global__ void __launch_bounds__(32 * kStreamWarps, stream_blocks<DP>()) kv_attention_stream(const AttnArgs a) {
  pdl_entry();
  constexpr bool WIDE = sizeof(T) == 4;
  constexpr int ST = stream_stages<DP>(), SB = stage_bytes<DP>(), NT = DP / 8;
  extern __shared__ __align__(128) uint8_t smem[];
  __shared__ int64_t scan[kStreamWarps], found[2];
  __shared__ float row_scale[kRows], merge_top[kStreamWarps][kRows], merge_sum[kStreamWarps][kRows];
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, g = lane >> 2, t4 = lane & 3;
  const int group = a.q_heads / a.cache.heads, dim = a.cache.dim, page = a.pool.page;
  PartMeta* meta = reinterpret_cast<PartMeta*>(a.work);
  float* parts = reinterpret_cast<float*>(meta + kMaxStreamGrid);

  // ---- this block's share: the sum over all entries, then the entry its first unit lies in
  int64_t total = 0;
  for (int i0 = 0; i0 < a.batch.n; i0 += 32 * kStreamWarps) {
    const int i = i0 + tid;
    int64_t u = i < a.batch.n ? entry_units(a, entry_of(a, i)) : 0;
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) u += __shfl_xor_sync(0xffffffffu, u, o);
    __syncthreads();
    if (lane == 0) scan[warp] = u;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < kStreamWarps; ++w) total += scan[w];
  }
  const int blocks = (int)max((int64_t)1, min((int64_t)gridDim.x, total / kMinUnits));
  const int me = blockIdx.x;
  if (tid == 0) meta[me].first = -1;
  if (me >= blocks || total == 0) return;
  int64_t at = share_at(total, blocks, me);
  const int64_t end = share_at(total, blocks, me + 1);
  int entry = 0;
  int64_t entry_at = 0;            // first unit of the entry
  {
    int64_t before = 0;
    bool done = false;
    for (int i0 = 0; i0 < a.batch.n && !done; i0 += 32 * kStreamWarps) {
      const int i = i0 + tid;
      const int64_t u = i < a.batch.n ? entry_units(a, entry_of(a, i)) : 0;
      int64_t s = u;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const int64_t v = __shfl_up_sync(0xffffffffu, s, o);
        if (lane >= o) s += v;
      }
      __syncthreads();
      if (lane == 31) scan[warp] = s;
      __syncthreads();
      int64_t mine = before;
#pragma unroll
      for (int w = 0; w < kStreamWarps; ++w) {
        if (w < warp) mine += scan[w];
        before += scan[w];
      }
      if (u > 0 && mine + s - u <= at && at < mine + s) { found[0] = i; found[1] = mine + s - u; }
      done = at < before;
    }
    __syncthreads();
    entry = (int)found[0];
    entry_at = found[1];
  }
  Entry E = entry_of(a, entry);

  const uint32_t q_sm = smem_at(smem);
  const uint32_t ring = q_sm + query_bytes<DP, WIDE>() + warp * ST * SB;
  float* merged = reinterpret_cast<float*>(smem + query_bytes<DP, WIDE>());     // the ring again, once it is empty

  while (at < end) {
    while (at >= entry_at + entry_units(a, E)) {
      entry_at += entry_units(a, E);
      E = entry_of(a, ++entry);
    }
    if (tid == 0 && E.s >= a.pool.max_seqs) atomicOr(a.err, ERR_PAGE);
    const int64_t item = (at - entry_at) / E.units;
    const int u0 = (int)((at - entry_at) % E.units), u1 = (int)min((int64_t)E.units, u0 + (end - at));
    const int hk = (int)(item / E.tiles), tile = (int)(item % E.tiles);
    const int64_t r_first = (int64_t)tile * kRows;         // first row of the tile in the entry
    const int r_count = (int)min((int64_t)kRows, E.rows * group - r_first);

    // ---- queries: eight threads a row, in the order the MMA's A operand wants
    {
      const int r = tid >> 3, part = tid & 7;
      const int64_t row = (r_first + r) / group;
      const int head = hk * group + (int)((r_first + r) % group);
      const T* q = reinterpret_cast<const T*>(a.q) + (E.row0 + row) * a.q_row + head * a.q_head;
      constexpr int V = Vec<T>::N;
      float v[DP / 8];
      unsigned top = 0;
#pragma unroll
      for (int c = 0; c < DP / 8 / V; ++c) {
        float f[V];
        const int d = (c * 8 + part) * V;
        if (r < r_count && d < dim) load_vec<T>(q + d, f);
        else {
#pragma unroll
          for (int j = 0; j < V; ++j) f[j] = 0.0f;
        }
#pragma unroll
        for (int j = 0; j < V; ++j) {
          v[c * V + j] = f[j];
          const unsigned b = abs_bits(f[j]);
          top = b > top ? b : top;
        }
      }
#pragma unroll
      for (int o = 1; o < 8; o <<= 1) {
        const unsigned b = __shfl_xor_sync(0xffffffffu, top, o);
        top = b > top ? b : top;
      }
      // 2^(12 - exponent of the largest): its inverse goes into the row's factor
      int shift = 12 - ((int)(top >> 23) - 127);
      if (top == 0 || top >= 0x7f800000u) shift = 0;
      shift = shift > 120 ? 120 : shift;
      const float up = __uint_as_float((unsigned)(127 + shift) << 23);
#pragma unroll
      for (int c = 0; c < DP / 8 / V; ++c)
#pragma unroll
        for (int j = 0; j < V; j += 2) {
          const int d = (c * 8 + part) * V + j;
          const int step = (d >> 6) * 4 + ((d & 15) >> 2), ln = (r & 7) * 4 + ((d & 63) >> 4), reg = (r >> 3) + (d & 2);
          const uint32_t to = q_sm + ((step * 32 + ln) * 4 + reg) * 4;
          const float x = v[c * V + j] * up, y = v[c * V + j + 1] * up;
          const __half2 hi = __floats2half2_rn(x, y);
          asm volatile("st.shared.b32 [%0], %1;" ::"r"(to), "r"(h2_bits(hi)) : "memory");
          if (WIDE)
            asm volatile("st.shared.b32 [%0], %1;" ::"r"(to + kRows * DP * 2),
                         "r"(pack_h2(x - __low2float(hi), y - __high2float(hi))) : "memory");
        }
      if (part == 0) row_scale[r] = a.scale * __uint_as_float((unsigned)(127 - shift) << 23);
    }
    __syncthreads();

    // ---- what this thread's two rows see, and what all rows do
    int lo[2], hi[2], all_lo = 0, all_hi = 0x7fffffff, any_lo = 0x7fffffff, any_hi = 0;
    float f_row[2];
#pragma unroll
    for (int z = 0; z < 2; ++z) {
      const int r = g + 8 * z;
      lo[z] = 0;
      hi[z] = 0;
      if (r < r_count) seen_range(a, E.len - E.rows + (r_first + r) / group, E.len, lo[z], hi[z]);
      f_row[z] = row_scale[r];
      all_lo = max(all_lo, lo[z]);
      all_hi = min(all_hi, hi[z]);
      any_lo = min(any_lo, r < r_count && hi[z] > lo[z] ? lo[z] : 0x7fffffff);
      any_hi = max(any_hi, hi[z]);
    }
    all_lo = __reduce_max_sync(0xffffffffu, all_lo);
    all_hi = __reduce_min_sync(0xffffffffu, all_hi);
    any_lo = __reduce_min_sync(0xffffffffu, any_lo);
    any_hi = __reduce_max_sync(0xffffffffu, any_hi);
    // runs of 32 tokens that some row sees, within the segment
    const int run_lo = max(u0 * (kUnit / kRun), any_lo / kRun);
    const int run_hi = min(u1 * (kUnit / kRun), (any_hi + kRun - 1) / kRun);
    const int n_runs = run_hi - run_lo > warp ? (run_hi - run_lo - warp + kStreamWarps - 1) / kStreamWarps : 0;

    float acc[NT][4], top[2] = {-INFINITY, -INFINITY}, sum[2] = {0.0f, 0.0f}, unit = 0.0f;
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
      for (int j = 0; j < 4; ++j) acc[n][j] = 0.0f;

    // pages of the next 32 runs: lane l holds those of run l of the window, for its first and second 16 tokens
    int pages[2] = {-1, -1}, window_at = -32;
    auto look_up = [&](int i) {        // i: first run of the window
      window_at = i;
#pragma unroll
      for (int z = 0; z < 2; ++z) {
        const int tok = (run_lo + warp + (i + lane) * kStreamWarps) * kRun + 16 * z;
        int p = -1;
        if (i + lane < n_runs && tok < E.len) {
          p = a.pool.table[(int64_t)E.s * a.pool.max_pages + tok / page];
          if (p < 0 || p >= a.pool.n_pages) { atomicOr(a.err, ERR_PAGE); p = -1; }
        }
        pages[z] = p;
      }
    };
    auto issue = [&](int i) {
      if (i < n_runs) {
        if (i >= window_at + 32) look_up(i);
        const uint32_t to = ring + (i % ST) * SB;
        const int tok = (run_lo + warp + i * kStreamWarps) * kRun;
#pragma unroll
        for (int z = 0; z < 2; ++z) {
          const int p = __shfl_sync(0xffffffffu, pages[z], i - window_at);
          if (p < 0) continue;
          const int64_t block = (int64_t)p * a.cache.heads + hk;
          const int64_t from = block * page * dim + (int64_t)((tok + 16 * z) % page) * dim;
          auto copy = [&](int c, int chunks) {
            const int row = c / chunks, ch = c - row * chunks;
            const uint32_t o = chunk_at<DP>(16 * z + row, ch);
            cp_async16(to + o, a.cache.k + from + c * 16);
            cp_async16(to + kRun * DP + o, a.cache.v + from + c * 16);
          };
          if (dim == DP) {
#pragma unroll
            for (int c = 0; c < DP / 32; ++c) copy(lane + 32 * c, DP / 16);
          } else {
            for (int c = lane; c < dim; c += 32) copy(c, dim / 16);
          }
          if (lane < 2) cp_async4(to + 2 * kRun * DP + (2 * lane + z) * 4, (lane ? a.cache.v_absmax : a.cache.k_absmax) + block);
        }
      }
      cp_commit();
    };
#pragma unroll
    for (int i = 0; i < ST - 1; ++i) issue(i);

    int valid_at = -32;                // the same window's validity, kept apart: issue() runs ahead of the use
    unsigned valid[2] = {0, 0};
    for (int i = 0; i < n_runs; ++i) {
      if (i >= valid_at + 32) {
        valid_at = i;
#pragma unroll
        for (int z = 0; z < 2; ++z) {
          const int tok = (run_lo + warp + (i + lane) * kStreamWarps) * kRun + 16 * z;
          bool ok = i + lane < n_runs && tok < E.len;
          if (ok) {
            const int p = a.pool.table[(int64_t)E.s * a.pool.max_pages + tok / page];
            ok = p >= 0 && p < a.pool.n_pages;
          }
          valid[z] = __ballot_sync(0xffffffffu, ok);
        }
      }
      cp_wait<ST - 2>();
      __syncwarp();
      const uint32_t ks = ring + (i % ST) * SB, vs = ks + kRun * DP;
      const int tok = (run_lo + warp + i * kStreamWarps) * kRun;
      const bool ok0 = valid[0] >> (i - valid_at) & 1u, ok1 = valid[1] >> (i - valid_at) & 1u;

      // scores
      float s[4][4];
#pragma unroll
      for (int n = 0; n < 4; ++n)
#pragma unroll
        for (int j = 0; j < 4; ++j) s[n][j] = 0.0f;
#pragma unroll
      for (int h = 0; h < DP / 64; ++h) {
        uint32_t qa[4][4], ql[WIDE ? 4 : 1][4];
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          const uint4 w = lds128(q_sm + ((h * 4 + k) * 32 + lane) * 16);
          qa[k][0] = w.x; qa[k][1] = w.y; qa[k][2] = w.z; qa[k][3] = w.w;
          if (WIDE) {
            const uint4 l = lds128(q_sm + kRows * DP * 2 + ((h * 4 + k) * 32 + lane) * 16);
            ql[k][0] = l.x; ql[k][1] = l.y; ql[k][2] = l.z; ql[k][3] = l.w;
          }
        }
#pragma unroll
        for (int n = 0; n < 4; ++n) {
          const int row = n * 8 + (g >> 1) + 4 * (g & 1);
          const uint4 w = lds128(ks + chunk_at<DP>(row, h * 4 + t4));
          const uint32_t words[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
          for (int k = 0; k < 4; ++k) {
            const uint32_t b = words[k] ^ 0x80808080u;
            const uint32_t b0 = two_codes<0x4140>(b), b1 = two_codes<0x4342>(b);
            mma16816(s[n], qa[k], b0, b1);
            if (WIDE) mma16816(s[n], ql[k], b0, b1);
          }
        }
      }
      // scales of the two halves
      float amax[4];
      {
        const uint4 w = lds128(ks + 2 * kRun * DP);
        amax[0] = __uint_as_float(w.x); amax[1] = __uint_as_float(w.y); amax[2] = __uint_as_float(w.z); amax[3] = __uint_as_float(w.w);
      }
      float kf[2] = {scale_of(amax[0]), scale_of(amax[1])};
      // a page of zeros must not set the unit
      float vf[2] = {ok0 ? __fdiv_rn(amax[2], kQmax8) : 0.0f, ok1 ? __fdiv_rn(amax[3], kQmax8) : 0.0f};
      if (!ok0) kf[0] = 1.0f;
      if (!ok1) kf[1] = 1.0f;

      if (tok < all_lo || tok + kRun > all_hi || !ok0 || !ok1) {
#pragma unroll
        for (int n = 0; n < 4; ++n)
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            const int t = tok + n * 8 + t4 + 4 * (j & 1);
            if (t < lo[j >> 1] || t >= hi[j >> 1] || !(n < 2 ? ok0 : ok1)) s[n][j] = -INFINITY;
          }
      }
      // softmax: factors are positive, so the largest product comes from the largest score
      float f[2][2], shift[2], keep[2];
#pragma unroll
      for (int z = 0; z < 2; ++z) {
#pragma unroll
        for (int p = 0; p < 2; ++p) f[z][p] = fmaxf(f_row[z] * kf[p], 1.2e-38f);
        float m = fmaxf(fmaxf(fmaxf(s[0][2 * z], s[0][2 * z + 1]), fmaxf(s[1][2 * z], s[1][2 * z + 1])) * f[z][0],
                        fmaxf(fmaxf(s[2][2 * z], s[2][2 * z + 1]), fmaxf(s[3][2 * z], s[3][2 * z + 1])) * f[z][1]);
        m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, 1));
        m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, 2));
        m = fmaxf(m, top[z]);
        const float ref = m == -INFINITY ? 0.0f : m;
        keep[z] = ex2(top[z] - ref);
        top[z] = m;
        shift[z] = kWeightBias - ref;
        sum[z] *= keep[z];
      }
      float now = fmaxf(unit, fmaxf(vf[0], vf[1]));
      if (now > 0.0f) now = fmaxf(now, 1.2e-38f);
      const float inv = now > 0.0f ? __fdiv_rn(1.0f, now) : 0.0f, change = unit * inv;
      unit = now;
      if (__any_sync(0xffffffffu, keep[0] * change != 1.0f || keep[1] * change != 1.0f)) {
        const float c0 = keep[0] * change, c1 = keep[1] * change;
#pragma unroll
        for (int n = 0; n < NT; ++n) {
          acc[n][0] *= c0;
          acc[n][1] *= c0;
          acc[n][2] *= c1;
          acc[n][3] *= c1;
        }
      }
      uint32_t pa[2][4], pl[WIDE ? 2 : 1][4];
#pragma unroll
      for (int p = 0; p < 2; ++p) {
        const float share = vf[p] * inv;
#pragma unroll
        for (int n = 0; n < 2; ++n)
#pragma unroll
          for (int z = 0; z < 2; ++z) {
            const float e0 = ex2(fmaf(s[2 * p + n][2 * z], f[z][p], shift[z]));
            const float e1 = ex2(fmaf(s[2 * p + n][2 * z + 1], f[z][p], shift[z]));
            sum[z] += e0 + e1;
            const float w0 = e0 * share, w1 = e1 * share;
            const __half2 h = __floats2half2_rn(w0, w1);
            pa[p][2 * n + z] = h2_bits(h);
            if (WIDE) pl[p][2 * n + z] = pack_h2(w0 - __low2float(h), w1 - __high2float(h));
          }
      }
      // values
#pragma unroll
      for (int p = 0; p < 2; ++p) {
        const int row = 16 * p + t4;
        constexpr int LINES = DP >= 128 ? DP / 128 : 1, WORDS = DP >= 128 ? 4 : 2;
#pragma unroll
        for (int h = 0; h < LINES; ++h) {
          uint32_t w[4][WORDS];
#pragma unroll
          for (int k = 0; k < 4; ++k) {
            const int r = row + 4 * k;
            if (DP >= 128) {
              const uint4 x = lds128(vs + chunk_at<DP>(r, h * 8 + g));
              w[k][0] = x.x; w[k][1] = x.y; w[k][WORDS - 2] = x.z; w[k][WORDS - 1] = x.w;
            } else {
              const uint2 x = lds64(vs + chunk_at<DP>(r, g >> 1) + (g & 1) * 8);
              w[k][0] = x.x; w[k][1] = x.y;
            }
          }
#pragma unroll
          for (int q = 0; q < WORDS; ++q) {
            const uint32_t x0 = w[0][q] ^ 0x80808080u, x1 = w[1][q] ^ 0x80808080u, x2 = w[2][q] ^ 0x80808080u, x3 = w[3][q] ^ 0x80808080u;
            const uint32_t y[2][2] = {{__byte_perm(x0, x1, 0x5140), __byte_perm(x0, x1, 0x7362)}, {__byte_perm(x2, x3, 0x5140), __byte_perm(x2, x3, 0x7362)}};
#pragma unroll
            for (int b = 0; b < 4; ++b) {
              const uint32_t b0 = b & 1 ? two_codes<0x4342>(y[0][b >> 1]) : two_codes<0x4140>(y[0][b >> 1]);
              const uint32_t b1 = b & 1 ? two_codes<0x4342>(y[1][b >> 1]) : two_codes<0x4140>(y[1][b >> 1]);
              mma16816(acc[(h * WORDS + q) * 4 + b], pa[p], b0, b1);
              if (WIDE) mma16816(acc[(h * WORDS + q) * 4 + b], pl[p], b0, b1);
            }
          }
        }
      }
      __syncwarp();
      issue(i + ST - 1);
    }
    cp_wait<0>();

    // ---- the four warps' parts of the segment, then out
#pragma unroll
    for (int z = 0; z < 2; ++z) {
      sum[z] += __shfl_xor_sync(0xffffffffu, sum[z], 1);
      sum[z] += __shfl_xor_sync(0xffffffffu, sum[z], 2);
      if (t4 == 0) merge_top[warp][g + 8 * z] = top[z];
    }
    __syncthreads();                   // also: every warp's ring is empty
    float m_all[2], factor[2];
#pragma unroll
    for (int z = 0; z < 2; ++z) {
      m_all[z] = -INFINITY;
#pragma unroll
      for (int w = 0; w < kStreamWarps; ++w) m_all[z] = fmaxf(m_all[z], merge_top[w][g + 8 * z]);
      factor[z] = top[z] == -INFINITY ? 0.0f : ex2(top[z] - m_all[z]);
      if (t4 == 0) merge_sum[warp][g + 8 * z] = sum[z] * factor[z];
      factor[z] *= unit;
    }
    // column n * 8 + c of the accumulators is the element c * 16 + n of its 128-element line (64: c * 8 + n)
    constexpr int PITCH = DP + 4;
#pragma unroll
    for (int n = 0; n < NT; ++n) {
      const int d = DP >= 128 ? (n / 16) * 128 + (2 * t4) * 16 + n % 16 : (2 * t4) * 8 + n;
      constexpr int STEP = DP >= 128 ? 16 : 8;
#pragma unroll
      for (int z = 0; z < 2; ++z) {
        float* to = merged + (warp * kRows + g + 8 * z) * PITCH + d;
        to[0] = acc[n][2 * z] * factor[z];
        to[STEP] = acc[n][2 * z + 1] * factor[z];
      }
    }
    __syncthreads();
    const bool whole = u0 == 0 && u1 == E.units;
    float* part = parts + ((int64_t)me * 2 + (u0 > 0 ? 0 : 1)) * part_floats<DP>();
    for (int e = tid; e < kRows * DP / 4; e += 32 * kStreamWarps) {
      const int r = e / (DP / 4), d = (e - r * (DP / 4)) * 4;
      float4 v = make_float4(0, 0, 0, 0);
#pragma unroll
      for (int w = 0; w < kStreamWarps; ++w) {
        const float4 x = *reinterpret_cast<const float4*>(merged + (w * kRows + r) * PITCH + d);
        v.x += x.x; v.y += x.y; v.z += x.z; v.w += x.w;
      }
      if (!whole) {
        *reinterpret_cast<float4*>(part + r * DP + d) = v;
        continue;
      }
      if (r >= r_count || d >= dim) continue;
      float l = 0.0f;
#pragma unroll
      for (int w = 0; w < kStreamWarps; ++w) l += merge_sum[w][r];
      const float inv = l > 0.0f ? __fdiv_rn(1.0f, l) : (l == 0.0f ? 0.0f : l);
      T* out = reinterpret_cast<T*>(a.out) + (E.row0 + (r_first + r) / group) * a.o_row + (hk * group + (r_first + r) % group) * a.o_head + d;
      union { T t[4]; uint4 w4; uint2 w2; } o;
      o.t[0] = from_float<T>(v.x * inv);
      o.t[1] = from_float<T>(v.y * inv);
      o.t[2] = from_float<T>(v.z * inv);
      o.t[3] = from_float<T>(v.w * inv);
      if (WIDE) *reinterpret_cast<uint4*>(out) = o.w4;
      else *reinterpret_cast<uint2*>(out) = o.w2;
    }
    if (!whole) {
      if (tid < kRows) {
        float m = -INFINITY, l = 0.0f;
#pragma unroll
        for (int w = 0; w < kStreamWarps; ++w) {
          m = fmaxf(m, merge_top[w][tid]);
          l += merge_sum[w][tid];
        }
        part[kRows * DP + tid] = m;
        part[kRows * DP + kRows + tid] = l;
      }
      if (tid == 0 && u0 > 0 && u1 == E.units) {
        PartMeta o;
        o.row0 = E.row0;
        o.first = share_of(total, blocks, at - u0);
        o.rows = (int)E.rows;
        o.tile = tile;
        o.head = hk;
        meta[me] = o;
      }
    }
    __syncthreads();
    at += u1 - u0;
  }
}

// Joins the parts of the tile that block blockIdx.x of the kernel above finished: a slice of 16 elements of each row.
constexpr int kJoinThreads = 64;
template <typename T, int DP>
__global__ void __launch_bounds__(kJoinThreads) kv_attention_join(const AttnArgs a) {
  pdl_entry();
  const PartMeta* meta = reinterpret_cast<const PartMeta*>(a.work);
  const float* parts = reinterpret_cast<const float*>(meta + kMaxStreamGrid);
  const int last = blockIdx.x, first = meta[last].first;
  if (first < 0) return;
  const PartMeta o = meta[last];
  const int r = threadIdx.x >> 2, d = blockIdx.y * 16 + (threadIdx.x & 3) * 4;
  const int group = a.q_heads / a.cache.heads;
  const int64_t r_at = (int64_t)o.tile * kRows + r;
  if (r_at >= (int64_t)o.rows * group || d >= a.cache.dim) return;
  // the first block's last segment is its second part, every later block's first segment its first
  float top = -INFINITY;
  for (int b = first; b <= last; ++b) top = fmaxf(top, parts[((int64_t)b * 2 + (b == first)) * part_floats<DP>() + kRows * DP + r]);
  float l = 0.0f;
  float4 v = make_float4(0, 0, 0, 0);
  for (int b = first; b <= last; ++b) {
    const float* p = parts + ((int64_t)b * 2 + (b == first)) * part_floats<DP>();
    const float m = p[kRows * DP + r];
    const float f = m == -INFINITY ? 0.0f : ex2(m - top);
    const float4 x = *reinterpret_cast<const float4*>(p + r * DP + d);
    l += f * p[kRows * DP + kRows + r];
    v.x += f * x.x; v.y += f * x.y; v.z += f * x.z; v.w += f * x.w;
  }
  const float inv = l > 0.0f ? __fdiv_rn(1.0f, l) : (l == 0.0f ? 0.0f : l);
  T* out = reinterpret_cast<T*>(a.out) + (o.row0 + r_at / group) * a.o_row + (o.head * group + r_at % group) * a.o_head + d;
  out[0] = from_float<T>(v.x * inv);
  out[1] = from_float<T>(v.y * inv);
  out[2] = from_float<T>(v.z * inv);
  out[3] = from_float<T>(v.w * inv);
}

template <int DP>
constexpr int64_t stream_work() { return kMaxStreamGrid * (int64_t)sizeof(PartMeta) + 2 * kMaxStreamGrid * part_floats<DP>() * 4; }

template <typename T, int DP>
int stream_as(Ctx* ctx, const AttnArgs& a, cudaStream_t st) {
  constexpr int smem = stream_smem<DP, sizeof(T) == 4>();
  static_assert(smem >= query_bytes<DP, sizeof(T) == 4>() + kStreamWarps * kRows * (DP + 4) * 4, "the parts of a segment are joined where the ring was");
  static_assert(stream_blocks<DP>() * (smem + 2048) <= 227 * 1024, "resident blocks");
  const cudaError_t e = cudaFuncSetAttribute(kv_attention_stream<T, DP>, cudaFuncAttributeMaxDynamicSharedMemorySize, smem);
  if (e != cudaSuccess) return check_cuda(ctx, e, "kv_attention");
  const int grid = std::min(sm_count(ctx) * stream_blocks<DP>(), kMaxStreamGrid);
  launch_pdl(kv_attention_stream<T, DP>, dim3(grid), dim3(32 * kStreamWarps), smem, st, a);
  launch_pdl(kv_attention_join<T, DP>, dim3(grid, DP / 16), dim3(kJoinThreads), 0, st, a);
  count_launch(ctx, 2);
  return check_cuda(ctx, cudaGetLastError(), "kv_attention");
}
template <typename T>
int stream_of(Ctx* ctx, const AttnArgs& a, cudaStream_t st) {
  return a.cache.dim <= 64 ? stream_as<T, 64>(ctx, a, st) : a.cache.dim <= 128 ? stream_as<T, 128>(ctx, a, st) : stream_as<T, 256>(ctx, a, st);
}

}  // namespace

int64_t kv_attention_work(Ctx*, const CacheView& c, int, int64_t, int) {
  return c.dim <= 64 ? stream_work<64>() : c.dim <= 128 ? stream_work<128>() : stream_work<256>();
}

int launch_kv_attention(Ctx* ctx, const PoolView& p, const CacheView& c, const BatchView& b, const void* q, int64_t q_row, int64_t q_head,
                        int q_heads, void* out, int64_t o_row, int64_t o_head, int dtype, int, int, float scale, int causal, int window, void* work,
                        cudaStream_t st) {
  if (b.n == 0 || b.rows == 0) return QCFG_OK;
  const AttnArgs a{p, c, b, q, out, q_row, q_head, o_row, o_head, q_heads, causal, window, scale * 1.44269504088896f, work, err_word(ctx)};
  return dtype == QCFG_FP32 ? stream_of<float>(ctx, a, st) : dtype == QCFG_BF16 ? stream_of<__nv_bfloat16>(ctx, a, st) : stream_of<__half>(ctx, a, st);
}

}  // namespace qcfg
