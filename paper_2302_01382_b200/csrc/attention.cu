// Attention over the paged 8-bit cache: out = softmax(sm_scale * q k^T) v with k = code * A_k / 127, v = code * A_v / 127, A the
// maximum of the token's page and head.
//
// The codes go to the tensor cores as fp16, which holds them exactly, and never exist as numbers of 16 bits in memory: a page's
// scale multiplies the finished scores (keys) or the weights (values).  Queries are fp16 after a power of two has brought
// their row's largest element to 2^12 .. 2^13, so bf16 and fp16 ones lose nothing above 2^-38 of the row; fp32 ones are the sum
// of two fp16 numbers.  Weights are e = 2^(7 + x - ref) times their page's value scale, against
// the largest such product the row has seen, in fp16 (fp32 calls: 2^(x - ref), the sum of two), with either reference at most 8 (6) below
// the running maximum: 21 binary orders and more below the largest product before the fp16 grid coarsens.
#include <algorithm>

#include "attention.cuh"

namespace qcfg {

namespace {

// ---- warps stream the cache ------------------------------------------------------------------------
//
// Work is counted in units of 64 tokens of one (entry, cache head, tile of rows); a row is a (query token, head of the group).
// All units of a call form one sequence that the resident blocks share evenly, so a ragged batch, a single long context and many
// short ones load the GPU alike; a tile counts kSetup units more for what it costs to begin.  A block works through its units
// segment by segment (a segment: units of one tile); a tile cut between blocks leaves its parts in `work`, and a second
// kernel joins them in a fixed order.
// Within a segment each of the four warps takes every fourth run of 32 tokens, with its own ring of stages (cp.async) and its own
// running maximum: nothing is synchronised until the segment ends.
//
// The products are taken the other way round, scores^T = K q^T and out^T += V^T weights^T: then the tokens and the elements fill the 16 rows
// of an MMA and the query rows its 8 columns, so that a group of up to 8 heads leaves no half of a product unused, and the
// conversions of codes (1.25 and 1.5 instructions each, what bounds this kernel next to HBM) are shared by all NR column tiles.
// In the A operand an element of K is (token, dimension), of V^T (dimension, token); the sums run over dimensions and
// tokens in any order, so both are read 16 bytes at a time as they lie in memory.
//
// HBM bounds it, and close behind it the issue slots: 64 entries of one bf16 token over contexts of 8000, 32 heads on 8 of 128, 119 us;
// one over 131000 tokens 57 us (both 4.7 TB/s, 71% of the measured copy rate, the second kernel's 5 us and the first's start included).
constexpr int kUnit = 64;           // tokens
constexpr int kSetup = 2;           // units
constexpr int kRun = 32;            // tokens a warp takes at a time
constexpr int kStreamWarps = 4;
constexpr int kMinUnits = 2;        // a block takes at least this many
// ref follows the running maximum only when a score passes it by more than `slack` binary orders, so that sums and accumulators are
// rescaled a few times in a context and not at every new maximum; a weight stays below 2^15.  fp32 calls take most of fp16's room above 1
// for the digits of small weights instead: a second half ends at 2^-25, and a weight is held times 2^9, so its 22 bits reach down to 2^-12
// of the largest and what is lost of smaller ones is 2^-34 of it.  (Held as they are, 40000 tokens of weight 2^-21.5 gave a sum off by 1%.
// 2^13 with 2 orders of slack: 32 entries of 16 tokens over 1000, 16 heads on 8 of 64, 48 -> 54 us, 50 this way: rows move too often.)
template <bool WIDE> __host__ __device__ constexpr float weight_slack() { return WIDE ? 6.0f : 8.0f; }
template <bool WIDE> __host__ __device__ constexpr int weight_order() { return WIDE ? 9 : 0; }
// A row's weights are multiplied with their page's value scale times `low` = 2^(weight_order - d), which follows the row's largest such
// product as ref follows its largest score: so what a row keeps depends on nothing but the tokens it sees, whatever the values of others
// in its tile.  (One factor for the tile, the largest scale seen by any of its rows, cost causal rows in front of values 2^20 times as
// large all their digits.)  In 16-bit calls the product that sets d becomes a power of two, which fp16 holds as it is.
template <int DP> __host__ __device__ constexpr int stage_bytes() { return 2 * kRun * DP + 32; }             // keys, values, four maxima
template <int DP, int NR> __host__ __device__ constexpr int stream_blocks() { return DP == 256 ? 1 : DP == 128 ? (NR == 4 ? 2 : 3) : NR == 1 ? 4 : NR == 2 ? 3 : 2; }    // per SM
template <int DP, int NR> __host__ __device__ constexpr int stream_stages() { return DP == 256 ? 3 : DP == 128 ? (NR == 4 ? 3 : 2) : (NR == 1 ? 3 : 4); }
template <int DP, int NR, bool WIDE> __host__ __device__ constexpr int query_bytes() { return (WIDE ? 2 : 1) * 8 * NR * DP * 2; }
template <int DP, int NR, bool WIDE>
__host__ __device__ constexpr int stream_smem() {
  return query_bytes<DP, NR, WIDE>() + kStreamWarps * stream_stages<DP, NR>() * stage_bytes<DP>();
}
constexpr int kMaxStreamGrid = 148 * 4;

struct PartMeta {         // of a block: the cut tile that its first segment finishes
  int64_t row0;           // first row of the entry
  int first;              // block that holds the tile's first part, -1: none
  int rows, tile, head;
  int pad[2];
};
template <int DP, int NR> __host__ __device__ constexpr int64_t part_floats() { return 8 * NR * DP + 16 * NR; }     // accumulators, maxima, sums

__device__ __forceinline__ void mma16816(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
  asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
               : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
// Transposes an 8 x 8 matrix of 16-bit elements: lane 4 g + t holds elements 2 t and 2 t + 1 of row g before and after
__device__ __forceinline__ uint32_t transpose8(uint32_t v) {
  uint32_t o;
  asm volatile("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(o) : "r"(v));
  return o;
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
// 0..3 or 4..7 x neighbouring chunks (16 or 8 bytes): the exclusive-or keeps both free of bank conflicts.  Everything in it that is
// not a compile-time constant depends on the lane alone: the offsets below are computed once, and what else differs between a lane's
// accesses is an immediate or the flip of bit 6.  (With the whole expression at each access a run took 1030 instructions, 740 this way.)
template <int DP>
__device__ __forceinline__ uint32_t chunk_at(int row, int chunk) {
  if (DP == 64) return (uint32_t)((row >> 1) * 128 + ((((row & 1) << 2) | chunk) ^ (2 * ((row >> 1) & 3))) * 16);
  const int f = (2 * (row & 3)) ^ (row & 4);
  return (uint32_t)(row * DP + (chunk & ~7) * 16 + ((chunk & 7) ^ f) * 16);
}

// What an entry of the batch asks for.
struct Entry {
  int64_t row0, rows;
  int s, len, tiles, units;      // tiles of 8 * NR rows, units per tile and head
};
template <int NR>
__device__ __forceinline__ Entry entry_of(const AttnArgs& a, int i) {
  Entry e;
  int64_t hi;
  entry_rows(a.batch, i, e.row0, hi);
  e.rows = hi - e.row0;
  e.s = a.batch.seqs[i];
  e.len = e.s < 0 || e.s >= a.pool.max_seqs ? 0 : seq_len(a.pool, e.s);
  e.tiles = (int)((e.rows * (a.q_heads / a.cache.heads) + 8 * NR - 1) / (8 * NR));
  e.units = kSetup + (e.len ? (e.len + kUnit - 1) / kUnit : 1);
  return e;
}
__device__ __forceinline__ int64_t entry_units(const AttnArgs& a, const Entry& e) { return (int64_t)e.tiles * (a.uncut ? 1 : e.units) * a.cache.heads; }

// a / b of numbers that are not negative: 64-bit divisions take a hundred instructions, and both fit 32 bits but in huge batches
__device__ __forceinline__ int64_t quotient(int64_t a, int64_t b) {
  return ((uint64_t)a | (uint64_t)b) >> 32 ? a / b : (int64_t)((uint32_t)a / (uint32_t)b);
}
// How `total` units fall to `blocks` blocks: the first `more` get one more than `each`
struct Shares {
  int64_t each;
  int more, blocks;
  __device__ __forceinline__ Shares(int64_t total, int grid, int least) {
    blocks = (int)max((int64_t)1, min((int64_t)grid, quotient(total, least)));
    each = quotient(total, blocks);
    more = (int)(total - each * blocks);
  }
  __device__ __forceinline__ int64_t first(int b) const { return each * b + min(b, more); }
  __device__ __forceinline__ int owner(int64_t unit) const {
    const int64_t head = more * (each + 1);
    return unit < head ? (int)quotient(unit, each + 1) : more + (int)quotient(unit - head, each);
  }
};

template <typename T, int DP, int NR>
__global__ void __launch_bounds__(32 * kStreamWarps, stream_blocks<DP, NR>()) kv_attention_stream(const AttnArgs a) {
  pdl_entry();
  constexpr bool WIDE = sizeof(T) == 4;
  constexpr int ST = stream_stages<DP, NR>(), SB = stage_bytes<DP>(), MT = DP / 16, ROWS = 8 * NR;
  extern __shared__ __align__(128) uint8_t smem[];
  __shared__ int64_t scan[kStreamWarps], found[2];
  __shared__ uint32_t magic_word;
  __shared__ float row_scale[ROWS], merge_top[kStreamWarps][ROWS], merge_sum[kStreamWarps][ROWS];
  __shared__ __align__(16) float low_of[kStreamWarps][ROWS], d_of[kStreamWarps][ROWS];
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, g = lane >> 2, t4 = lane & 3;
  const int group = a.q_heads / a.cache.heads, dim = a.cache.dim, page = a.pool.page;
  PartMeta* meta = reinterpret_cast<PartMeta*>(a.work);
  float* parts = reinterpret_cast<float*>(meta + kMaxStreamGrid);

  if (tid == 0) magic_word = 0x64646464u;

  // ---- this block's share: the sum over all entries, then the entry its first unit lies in
  auto units_of = [&](int i) { return i < a.batch.n ? entry_units(a, entry_of<NR>(a, i)) : (int64_t)0; };
  if (blockIdx.x == gridDim.x - 1)         // (the others would report the same)
    for (int i = tid; i < a.batch.n; i += 32 * kStreamWarps) {
      int64_t lo, hi;
      if (!entry_rows(a.batch, i, lo, hi)) atomicOr(a.err, ERR_PAGE);
    }
  // inclusive sums over the block's threads; `sum` gets the total
  auto scan_units = [&](int64_t u, int64_t& sum) {
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int64_t v = __shfl_up_sync(0xffffffffu, u, o);
      if (lane >= o) u += v;
    }
    __syncthreads();
    if (lane == 31) scan[warp] = u;
    __syncthreads();
    sum = 0;
#pragma unroll
    for (int w = 0; w < kStreamWarps; ++w) {
      if (w < warp) u += scan[w];
      sum += scan[w];
    }
    return u;
  };
  int64_t total, mine = units_of(tid), upto = scan_units(mine, total);
  for (int i0 = 32 * kStreamWarps; i0 < a.batch.n; i0 += 32 * kStreamWarps) {
    int64_t sum;
    scan_units(units_of(i0 + tid), sum);
    total += sum;
  }
  const Shares shares(total, gridDim.x, a.uncut ? 1 : kSetup + kMinUnits);
  const int me = blockIdx.x;
  if (tid == 0 && !a.uncut) meta[me].first = -1;
  if (me >= shares.blocks || total == 0) return;
  int64_t at = shares.first(me);
  const int64_t end = shares.first(me + 1);
  for (int i0 = 0;;) {
    if (mine > 0 && upto - mine <= at && at < upto) { found[0] = i0 + tid; found[1] = upto - mine; }
    i0 += 32 * kStreamWarps;
    if (i0 >= a.batch.n) break;
    __syncthreads();
    if (tid == 32 * kStreamWarps - 1) scan[0] = upto;
    __syncthreads();
    const int64_t before = scan[0];
    int64_t sum;
    mine = units_of(i0 + tid);
    upto = before + scan_units(mine, sum);
  }
  __syncthreads();
  const uint32_t magic = *(volatile uint32_t*)&magic_word;
  int entry = (int)found[0];
  int64_t entry_at = found[1];     // first unit of the entry
  Entry E = entry_of<NR>(a, entry);

  const uint32_t q_sm = smem_at(smem);
  const uint32_t ring = q_sm + query_bytes<DP, NR, WIDE>() + warp * ST * SB;
  float* merged = reinterpret_cast<float*>(smem + query_bytes<DP, NR, WIDE>());     // the ring again, once it is empty
  const int key = (g >> 1) + 4 * (g & 1);                  // token of row g of a tile of scores^T
  const uint32_t copy_at = chunk_at<DP>(lane / (DP / 16), lane % (DP / 16)), key_at = chunk_at<DP>(key, t4),
                 val_at = kRun * DP + (DP == 64 ? chunk_at<DP>(t4, g >> 1) + (g & 1) * 8 : chunk_at<DP>(t4, g));

  while (at < end) {
    while (at >= entry_at + entry_units(a, E)) {
      entry_at += entry_units(a, E);
      E = entry_of<NR>(a, ++entry);
    }
    const int per_tile = a.uncut ? 1 : E.units, n_units = E.units - kSetup;
    const int64_t item = quotient(at - entry_at, per_tile);
    const int v0 = (int)(at - entry_at - item * per_tile), v1 = (int)min((int64_t)per_tile, v0 + (end - at));
    const int u0 = a.uncut ? 0 : max(v0 - kSetup, 0), u1 = a.uncut ? n_units : max(v1 - kSetup, 0);
    at += v1 - v0;
    if (u1 == 0) continue;                                 // ends before the tile's first token
    if (tid == 0 && E.s >= a.pool.max_seqs) atomicOr(a.err, ERR_PAGE);
    const int hk = (int)quotient(item, E.tiles), tile = (int)(item - (int64_t)hk * E.tiles);
    // the tile's first row: token t_first of the entry, head h_first of the group
    const int64_t t_first = quotient((int64_t)tile * ROWS, group);
    const unsigned h_first = (unsigned)((int64_t)tile * ROWS - t_first * group);
    const int r_count = (int)min((int64_t)ROWS, E.rows * group - (int64_t)tile * ROWS);

    // ---- queries, in the order the MMA's B operand wants: eight threads a row
#pragma unroll
    for (int r0 = 0; r0 < ROWS; r0 += 16) {
      const int r = r0 + (tid >> 3), part = tid & 7;
      if (ROWS >= 16 || r < ROWS) {
        const unsigned row = (h_first + r) / (unsigned)group, head = hk * group + (h_first + r - row * group);
        const T* q = reinterpret_cast<const T*>(a.q) + (E.row0 + t_first + row) * a.q_row + head * a.q_head;
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
          const unsigned b = __shfl_xor_sync(__activemask(), top, o);
          top = b > top ? b : top;
        }
        const int shift = row_shift(top);
        const float up = top < 0x7f800000u ? exp2_of(shift) : __int_as_float(0x7fffffff);      // an Inf makes the row NaN, like a NaN
#pragma unroll
        for (int c = 0; c < DP / 8 / V; ++c)
#pragma unroll
          for (int j = 0; j < V; j += 2) {
            const int d = (c * 8 + part) * V + j;
            const int ln = (r & 7) * 4 + ((d & 63) >> 4), step = (d & 15) >> 2, reg = (step & 1) * 2 + ((d & 3) >> 1);
            const uint32_t to = q_sm + (((((r >> 3) * (DP / 64) + (d >> 6)) * 2 + (step >> 1)) * 32 + ln) * 4 + reg) * 4;
            const float x = v[c * V + j] * up, y = v[c * V + j + 1] * up;
            const __half2 hi = __floats2half2_rn(x, y);
            asm volatile("st.shared.b32 [%0], %1;" ::"r"(to), "r"(h2_bits(hi)) : "memory");
            if (WIDE)
              asm volatile("st.shared.b32 [%0], %1;" ::"r"(to + ROWS * DP * 2),
                           "r"(pack_h2(x - __low2float(hi), y - __high2float(hi))) : "memory");
          }
        if (part == 0) row_scale[r] = a.scale * exp2_of(-shift);
      }
    }
    __syncthreads();

    // ---- what this thread's rows (8 n + 2 t4 + z) see, and what all rows do; rows that do not exist see everything
    int lo[NR][2], hi[NR][2], all_lo = 0, all_hi = 0x7fffffff, any_lo = 0x7fffffff, any_hi = 0;
    float f_row[NR][2];
#pragma unroll
    for (int n = 0; n < NR; ++n)
#pragma unroll
      for (int z = 0; z < 2; ++z) {
        const int r = 8 * n + 2 * t4 + z;
        lo[n][z] = 0;
        hi[n][z] = 0x7fffffff;
        f_row[n][z] = row_scale[r];
        if (r >= r_count) continue;
        seen_range(a, E.len - E.rows + t_first + (h_first + r) / (unsigned)group, E.len, lo[n][z], hi[n][z]);
        all_lo = max(all_lo, lo[n][z]);
        all_hi = min(all_hi, hi[n][z]);
        any_lo = min(any_lo, hi[n][z] > lo[n][z] ? lo[n][z] : 0x7fffffff);
        any_hi = max(any_hi, hi[n][z]);
      }
    all_lo = __reduce_max_sync(0xffffffffu, all_lo);
    all_hi = __reduce_min_sync(0xffffffffu, all_hi);
    any_lo = __reduce_min_sync(0xffffffffu, any_lo);
    any_hi = __reduce_max_sync(0xffffffffu, any_hi);
    // runs of 32 tokens that some row sees, within the segment
    const int run_lo = max(u0 * (kUnit / kRun), any_lo / kRun);
    const int run_hi = min(u1 * (kUnit / kRun), (any_hi + kRun - 1) / kRun);
    const int n_runs = run_hi - run_lo > warp ? (run_hi - run_lo - warp + kStreamWarps - 1) / kStreamWarps : 0;

    float acc[MT][NR][4], ref[NR][2], sum[NR][2];
    float least = 0.0f;                // of the warp's rows: a bound of d
#pragma unroll
    for (int n = 0; n < NR; ++n) {
      ref[n][0] = ref[n][1] = -INFINITY;
      sum[n][0] = sum[n][1] = 0.0f;
#pragma unroll
      for (int m = 0; m < MT; ++m)
#pragma unroll
        for (int j = 0; j < 4; ++j) acc[m][n][j] = 0.0f;
    }
    // `low` of the rows: in shared memory, read once a run (in registers, where one for 8 rows is, they cost the forms of more rows 4 to 10% in spills)
    float *low_row = low_of[warp] + 2 * t4, *d_row = d_of[warp] + 2 * t4;
    if (lane < ROWS) {
      low_of[warp][lane] = (float)(1 << weight_order<WIDE>());
      d_of[warp][lane] = 0.0f;
    }
    float2 low_here = make_float2(0.0f, 0.0f);      // (NR = 1)
    __syncwarp();

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
    uint32_t fill = 0;
    auto issue = [&](int i) {
      if (i < n_runs) {
        if (i >= window_at + 32) look_up(i);
        const uint32_t to = ring + fill;
        const int tok = (run_lo + warp + i * kStreamWarps) * kRun;
#pragma unroll
        for (int z = 0; z < 2; ++z) {
          const int p = __shfl_sync(0xffffffffu, pages[z], i - window_at);
          if (p < 0) {                 // no such tokens: a maximum of -1 says so
            if (lane < 2) asm volatile("st.shared.b32 [%0], %1;" ::"r"(to + 2 * kRun * DP + (2 * lane + z) * 4), "r"(0xbf800000u) : "memory");
            continue;
          }
          const int64_t block = (int64_t)p * a.cache.heads + hk;
          const int64_t from = (block * page + ((tok + 16 * z) & (page - 1))) * dim + lane * 16;
          const int8_t *k_from = a.cache.k + from, *v_from = a.cache.v + from;
          if (dim == DP) {
            const uint32_t even = to + z * 16 * DP + copy_at, odd = to + z * 16 * DP + (copy_at ^ 64u);
#pragma unroll
            for (int c = 0; c < DP / 32; ++c) {                 // the copy's row is lane / (DP / 16) + c * (512 / DP)
              const bool flip = DP == 64 ? false : DP == 128 ? (c & 1) : ((c ^ (c >> 1)) & 1);
              cp_async16((flip ? odd : even) + c * 512, k_from + c * 512);
              cp_async16((flip ? odd : even) + c * 512 + kRun * DP, v_from + c * 512);
            }
          } else {
            for (int c = lane; c < dim; c += 32) {
              const int row = c / (dim / 16), ch = c - row * (dim / 16);
              const uint32_t o = to + chunk_at<DP>(16 * z + row, ch);
              cp_async16(o, k_from + (c - lane) * 16);
              cp_async16(o + kRun * DP, v_from + (c - lane) * 16);
            }
          }
          if (lane < 2) cp_async4(to + 2 * kRun * DP + (2 * lane + z) * 4, (lane ? a.cache.v_absmax : a.cache.k_absmax) + block);
        }
      }
      fill = fill == (ST - 1) * SB ? 0 : fill + SB;
      cp_commit();
    };
#pragma unroll
    for (int i = 0; i < ST - 1; ++i) issue(i);

    uint32_t drain = 0;
    bool fresh = true;                 // some row has no reference yet
    for (int i = 0; i < n_runs; ++i) {
      cp_wait<ST - 2>();
      __syncwarp();                    // the run has arrived for all lanes, and all are done with the one before, whose stage is filled again
      issue(i + ST - 1);
      const uint32_t stage = ring + drain;
      const uint32_t k_even = stage + key_at, k_odd = stage + (key_at ^ 64u), v_even = stage + val_at, v_odd = stage + (val_at ^ 64u);
      drain = drain == (ST - 1) * SB ? 0 : drain + SB;
      const int tok = (run_lo + warp + i * kStreamWarps) * kRun;

      // scores^T: tile p are the tokens 16 p .. 16 p + 15, row r of it the token with r's bits 0 and 1, 2 exchanged
      float s[2][NR][4];
#pragma unroll
      for (int p = 0; p < 2; ++p)
#pragma unroll
        for (int n = 0; n < NR; ++n)
#pragma unroll
          for (int j = 0; j < 4; ++j) s[p][n][j] = 0.0f;
#pragma unroll
      for (int h = 0; h < DP / 64; ++h) {
        uint32_t q[NR][8], ql[WIDE ? NR : 1][8];
#pragma unroll
        for (int n = 0; n < NR; ++n)
#pragma unroll
          for (int k = 0; k < 2; ++k) {
            const uint4 w = lds128(q_sm + (((n * (DP / 64) + h) * 2 + k) * 32 + lane) * 16);
            q[n][4 * k] = w.x; q[n][4 * k + 1] = w.y; q[n][4 * k + 2] = w.z; q[n][4 * k + 3] = w.w;
            if (WIDE) {
              const uint4 l = lds128(q_sm + ROWS * DP * 2 + (((n * (DP / 64) + h) * 2 + k) * 32 + lane) * 16);
              ql[n][4 * k] = l.x; ql[n][4 * k + 1] = l.y; ql[n][4 * k + 2] = l.z; ql[n][4 * k + 3] = l.w;
            }
          }
#pragma unroll
        for (int p = 0; p < 2; ++p) {
          const uint32_t from = (DP > 64 && (h & 1) ? k_odd : k_even) + (h >> 1) * 128 + 16 * p * DP;
          const uint4 x = lds128(from), y = lds128(from + 8 * DP);
          const uint32_t xw[4] = {x.x, x.y, x.z, x.w}, yw[4] = {y.x, y.y, y.z, y.w};
#pragma unroll
          for (int k = 0; k < 4; ++k) {
            const uint32_t xb = xw[k] ^ 0x80808080u, yb = yw[k] ^ 0x80808080u;
            const uint32_t op[4] = {two_codes<0x4140>(xb, magic), two_codes<0x4140>(yb, magic), two_codes<0x4342>(xb, magic), two_codes<0x4342>(yb, magic)};
#pragma unroll
            for (int n = 0; n < NR; ++n) {
              mma16816(s[p][n], op, q[n][2 * k], q[n][2 * k + 1]);
              if (WIDE) mma16816(s[p][n], op, ql[n][2 * k], ql[n][2 * k + 1]);
            }
          }
        }
      }
      // scales of the two tiles, the values' with their binary logarithm; a maximum of -1 marks tokens that are not there
      float kf[2], vf[2], lv[2];
      bool ok[2];
      {
        const uint4 w = lds128(stage + 2 * kRun * DP);
        const float k_max[2] = {__uint_as_float(w.x), __uint_as_float(w.y)}, v_max[2] = {__uint_as_float(w.z), __uint_as_float(w.w)};
#pragma unroll
        for (int p = 0; p < 2; ++p) {
          ok[p] = !(k_max[p] < 0.0f);
          kf[p] = ok[p] && k_max[p] > 0.0f ? k_max[p] * (1.0f / kQmax8) : 1.0f;      // the scale but for its last bit
          vf[p] = ok[p] ? v_max[p] * (1.0f / kQmax8) : 0.0f;
          lv[p] = lg2(fmaxf(vf[p], 1.2e-38f));
        }
      }
      if (tok < all_lo || tok + kRun > all_hi || !ok[0] || !ok[1]) {
#pragma unroll
        for (int p = 0; p < 2; ++p)
#pragma unroll
          for (int n = 0; n < NR; ++n)
#pragma unroll
            for (int j = 0; j < 4; ++j) {
              const int t = tok + 16 * p + key + 8 * (j >> 1);
              if (t < lo[n][j & 1] || t >= hi[n][j & 1] || !ok[p]) s[p][n][j] = -INFINITY;
            }
      }
      // exponents of the weights against the reference in use
      float over = -INFINITY;
#pragma unroll
      for (int n = 0; n < NR; ++n)
#pragma unroll
        for (int z = 0; z < 2; ++z) {
          const float shift = weight_bias<WIDE>() - (ref[n][z] == -INFINITY ? 0.0f : ref[n][z]);
#pragma unroll
          for (int p = 0; p < 2; ++p) {
            const float f = fmaxf(f_row[n][z] * kf[p], 1.2e-38f);
#pragma unroll
            for (int j = 0; j < 2; ++j) {
              float& x = s[p][n][2 * j + z];
              x = fmaf(x, f, shift);
              over = fmaxf(over, x);
            }
          }
        }
      const float most = weight_bias<WIDE>() + weight_slack<WIDE>() - fmaxf(fmaxf(lv[0], lv[1]) - least, 0.0f);
      if (__any_sync(0xffffffffu, over > most) || fresh) {
        fresh = false;
        least = 127.0f;
#pragma unroll
        for (int n = 0; n < NR; ++n) {
          if (NR > 1) {                // eight rows at a time: mostly it is one row that has to move
            over = ref[n][0] == -INFINITY || ref[n][1] == -INFINITY ? INFINITY : -INFINITY;
#pragma unroll
            for (int p = 0; p < 2; ++p)
#pragma unroll
              for (int j = 0; j < 4; ++j) over = fmaxf(over, s[p][n][j]);
            if (!__any_sync(0xffffffffu, over > most)) {
              least = fminf(least, fminf(d_row[8 * n], d_row[8 * n + 1]));
              continue;
            }
          }
#pragma unroll
          for (int z = 0; z < 2; ++z) {
            const float was = ref[n][z] == -INFINITY ? 0.0f : ref[n][z];
            const float m0 = fmaxf(s[0][n][z], s[0][n][2 + z]), m1 = fmaxf(s[1][n][z], s[1][n][2 + z]);
            float m = fmaxf(m0, m1), v = fmaxf(m0 + lv[0], m1 + lv[1]);
#pragma unroll
            for (int o = 4; o < 32; o <<= 1) {
              m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
              v = fmaxf(v, __shfl_xor_sync(0xffffffffu, v, o));
            }
            m = fmaxf(m - weight_bias<WIDE>() + was, ref[n][z]);
            v = v - weight_bias<WIDE>() + was;
            const float base = m == -INFINITY ? 0.0f : m, d_was = d_row[8 * n + z], v_was = ref[n][z] + d_was;
            float d = m == -INFINITY ? 0.0f : m == ref[n][z] && v <= v_was ? d_was : fminf(fmaxf(fmaxf(v, v_was) - m, -110.0f), 122.0f);
            if (WIDE) d = ceilf(d);        // a whole number, so that sums and accumulators are rescaled alike to the last bit
            const float keep = ex2(ref[n][z] - base), keep_values = keep * ex2(fminf(d_was - d, 126.0f)), low = ex2(weight_order<WIDE>() - d);
            ref[n][z] = m;
            __syncwarp();
            if (g == 0) {
              low_row[8 * n + z] = low;
              d_row[8 * n + z] = d;
            }
            if (NR == 1) (z ? low_here.y : low_here.x) = low;
            least = fminf(least, d);
            fresh |= m == -INFINITY;
            sum[n][z] *= keep;
#pragma unroll
            for (int p = 0; p < 2; ++p)
#pragma unroll
              for (int j = 0; j < 2; ++j) s[p][n][2 * j + z] += was - base;
#pragma unroll
            for (int t = 0; t < MT; ++t) {
              acc[t][n][z] *= keep_values;
              acc[t][n][2 + z] *= keep_values;
            }
          }
        }
        fresh = __any_sync(0xffffffffu, fresh);
        least = (float)__reduce_min_sync(0xffffffffu, (int)floorf(least));
        __syncwarp();
      }
      float2 low2[NR];
#pragma unroll
      for (int n = 0; n < NR; ++n) low2[n] = NR > 1 ? *reinterpret_cast<const float2*>(low_row + 8 * n) : low_here;
      uint32_t w_hi[2][NR][2], w_lo[WIDE ? 2 : 1][NR][2];
#pragma unroll
      for (int p = 0; p < 2; ++p) {
#pragma unroll
        for (int n = 0; n < NR; ++n) {
          // (kept finite: tokens a row does not see have weights of 0; one of 2^-110 and less may lose by it)
          const float share0 = fminf(vf[p] * low2[n].x, 8.5e37f), share1 = fminf(vf[p] * low2[n].y, 8.5e37f);
#pragma unroll
          for (int j = 0; j < 2; ++j) {
            const float e0 = ex2(s[p][n][2 * j]), e1 = ex2(s[p][n][2 * j + 1]);
            sum[n][0] += e0;
            sum[n][1] += e1;
            const float w0 = e0 * share0, w1 = e1 * share1;
            const __half2 h = __floats2half2_rn(w0, w1);
            w_hi[p][n][j] = transpose8(h2_bits(h));
            if (WIDE) w_lo[p][n][j] = transpose8(pack_h2(w0 - __low2float(h), w1 - __high2float(h)));
          }
        }
      }
      // out^T: byte 2 m of a thread's elements is row g of tile m, byte 2 m + 1 row g + 8
#pragma unroll
      for (int p = 0; p < 2; ++p) {
        constexpr int LINES = DP >= 128 ? DP / 128 : 1, WORDS = DP >= 128 ? 4 : 2;
#pragma unroll
        for (int h = 0; h < LINES; ++h) {
          uint32_t w[4][WORDS];
#pragma unroll
          for (int k = 0; k < 4; ++k) {
            const uint32_t from = (k & 1 ? v_odd : v_even) + (16 * p + 4 * k) * DP + h * 128;
            if (DP >= 128) {
              const uint4 x = lds128(from);
              w[k][0] = x.x; w[k][1] = x.y; w[k][WORDS - 2] = x.z; w[k][WORDS - 1] = x.w;
            } else {
              const uint2 x = lds64(from);
              w[k][0] = x.x; w[k][1] = x.y;
            }
          }
#pragma unroll
          for (int q = 0; q < WORDS; ++q) {
            const uint32_t x0 = w[0][q] ^ 0x80808080u, x1 = w[1][q] ^ 0x80808080u, x2 = w[2][q] ^ 0x80808080u, x3 = w[3][q] ^ 0x80808080u;
#pragma unroll
            for (int b = 0; b < 2; ++b) {
              const uint32_t y0 = __byte_perm(x0, x1, b ? 0x7362 : 0x5140), y1 = __byte_perm(x2, x3, b ? 0x7362 : 0x5140);
              const uint32_t op[4] = {two_codes<0x4140>(y0, magic), two_codes<0x4342>(y0, magic), two_codes<0x4140>(y1, magic), two_codes<0x4342>(y1, magic)};
#pragma unroll
              for (int n = 0; n < NR; ++n) {
                mma16816(acc[(h * WORDS + q) * 2 + b][n], op, w_hi[p][n][0], w_hi[p][n][1]);
                if (WIDE) mma16816(acc[(h * WORDS + q) * 2 + b][n], op, w_lo[p][n][0], w_lo[p][n][1]);
              }
            }
          }
        }
      }
    }
    cp_wait<0>();

    // ---- the four warps' parts of the segment, then out
#pragma unroll
    for (int n = 0; n < NR; ++n)
#pragma unroll
      for (int z = 0; z < 2; ++z) {
#pragma unroll
        for (int o = 4; o < 32; o <<= 1) sum[n][z] += __shfl_xor_sync(0xffffffffu, sum[n][z], o);
        if (g == 0) merge_top[warp][8 * n + 2 * t4 + z] = ref[n][z];
      }
    __syncthreads();                   // also: every warp's ring is empty
    constexpr int PITCH = DP + 4;
#pragma unroll
    for (int n = 0; n < NR; ++n)
#pragma unroll
      for (int z = 0; z < 2; ++z) {
        const int r = 8 * n + 2 * t4 + z;
        float m = -INFINITY;
#pragma unroll
        for (int w = 0; w < kStreamWarps; ++w) m = fmaxf(m, merge_top[w][r]);
        float factor = ref[n][z] == -INFINITY ? 0.0f : ex2(ref[n][z] - m);
        if (g == 0) merge_sum[warp][r] = sum[n][z] * factor;
        factor = __fdiv_rn(factor, low_row[8 * n + z]);
        float* to = merged + (warp * ROWS + r) * PITCH;
#pragma unroll
        for (int t = 0; t < MT; ++t) {
          const int d = DP >= 128 ? (t / 8) * 128 + g * 16 + (t % 8) * 2 : g * 8 + t * 2;
          *reinterpret_cast<float2*>(to + d) = make_float2(acc[t][n][z] * factor, acc[t][n][2 + z] * factor);
        }
      }
    __syncthreads();
    const bool whole = u0 == 0 && u1 == n_units;
    float* part = parts + ((int64_t)me * 2 + (u0 > 0 ? 0 : 1)) * part_floats<DP, NR>();
    for (int e = tid; e < ROWS * DP / 4; e += 32 * kStreamWarps) {
      const int r = e / (DP / 4), d = (e - r * (DP / 4)) * 4;
      float4 v = make_float4(0, 0, 0, 0);
#pragma unroll
      for (int w = 0; w < kStreamWarps; ++w) {
        const float4 x = *reinterpret_cast<const float4*>(merged + (w * ROWS + r) * PITCH + d);
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
      const unsigned row = (h_first + r) / (unsigned)group, head = hk * group + (h_first + r - row * group);
      T* out = reinterpret_cast<T*>(a.out) + (E.row0 + t_first + row) * a.o_row + head * a.o_head + d;
      union { T t[4]; uint4 w4; uint2 w2; } o;
      o.t[0] = from_float<T>(v.x * inv);
      o.t[1] = from_float<T>(v.y * inv);
      o.t[2] = from_float<T>(v.z * inv);
      o.t[3] = from_float<T>(v.w * inv);
      if (WIDE) *reinterpret_cast<uint4*>(out) = o.w4;
      else *reinterpret_cast<uint2*>(out) = o.w2;
    }
    if (!whole) {
      if (tid < ROWS) {
        float m = -INFINITY, l = 0.0f;
#pragma unroll
        for (int w = 0; w < kStreamWarps; ++w) {
          m = fmaxf(m, merge_top[w][tid]);
          l += merge_sum[w][tid];
        }
        part[ROWS * DP + tid] = m;
        part[ROWS * DP + ROWS + tid] = l;
      }
      if (tid == 0 && u0 > 0 && u1 == n_units) {
        PartMeta o;
        o.row0 = E.row0;
        o.first = shares.owner(entry_at + item * E.units + kSetup);      // the block of the tile's first tokens
        o.rows = (int)E.rows;
        o.tile = tile;
        o.head = hk;
        meta[me] = o;
      }
    }
    __syncthreads();
  }
}

// Joins the parts of the tile that block blockIdx.x of the kernel above finished: 16 elements of each row, every kJoinWays-th part to a
// group of threads.
constexpr int kJoinWays = 8;
template <typename T, int DP, int NR>
__global__ void __launch_bounds__(32 * NR * kJoinWays) kv_attention_join(const AttnArgs a) {
  pdl_entry();
  constexpr int ROWS = 8 * NR;
  __shared__ float4 values[kJoinWays][32 * NR];
  __shared__ float tops[kJoinWays][ROWS], sums[kJoinWays][ROWS];
  const PartMeta* meta = reinterpret_cast<const PartMeta*>(a.work);
  const float* parts = reinterpret_cast<const float*>(meta + kMaxStreamGrid);
  const int last = blockIdx.x, first = meta[last].first;
  if (first < 0) return;
  const PartMeta o = meta[last];
  const int way = threadIdx.x / (32 * NR), e = threadIdx.x % (32 * NR);
  const int r = e >> 2, d = blockIdx.y * 16 + (e & 3) * 4;
  // the first block's last segment is its second part, every later block's first segment its first
  float top = -INFINITY, l = 0.0f;
  float4 v = make_float4(0, 0, 0, 0);
  for (int b = first + way; b <= last; b += kJoinWays) {
    const float* p = parts + ((int64_t)b * 2 + (b == first)) * part_floats<DP, NR>();
    const float m = p[ROWS * DP + r], s = p[ROWS * DP + ROWS + r];
    const float4 x = *reinterpret_cast<const float4*>(p + r * DP + d);
    const float now = fmaxf(top, m), base = now == -INFINITY ? 0.0f : now, keep = ex2(top - base), f = ex2(m - base);
    top = now;
    l = l * keep + s * f;
    v.x = v.x * keep + x.x * f;
    v.y = v.y * keep + x.y * f;
    v.z = v.z * keep + x.z * f;
    v.w = v.w * keep + x.w * f;
  }
  values[way][e] = v;
  if ((e & 3) == 0) { tops[way][r] = top; sums[way][r] = l; }
  __syncthreads();
  if (way) return;
#pragma unroll
  for (int w = 1; w < kJoinWays; ++w) top = fmaxf(top, tops[w][r]);
  const float base = top == -INFINITY ? 0.0f : top;
  l = 0.0f;
  v = make_float4(0, 0, 0, 0);
#pragma unroll
  for (int w = 0; w < kJoinWays; ++w) {
    const float f = ex2(tops[w][r] - base);
    const float4 x = values[w][e];
    l += sums[w][r] * f;
    v.x += x.x * f; v.y += x.y * f; v.z += x.z * f; v.w += x.w * f;
  }
  const int group = a.q_heads / a.cache.heads;
  const int64_t r_at = (int64_t)o.tile * ROWS + r;
  if (r_at >= (int64_t)o.rows * group || d >= a.cache.dim) return;
  const int64_t row = quotient(r_at, group);
  const float inv = l > 0.0f ? __fdiv_rn(1.0f, l) : (l == 0.0f ? 0.0f : l);
  T* out = reinterpret_cast<T*>(a.out) + (o.row0 + row) * a.o_row + (o.head * group + (r_at - row * group)) * a.o_head + d;
  out[0] = from_float<T>(v.x * inv);
  out[1] = from_float<T>(v.y * inv);
  out[2] = from_float<T>(v.z * inv);
  out[3] = from_float<T>(v.w * inv);
}

template <int DP, int NR>
constexpr int64_t stream_work() { return kMaxStreamGrid * ((int64_t)sizeof(PartMeta) + 2 * part_floats<DP, NR>() * 4); }

template <typename T, int DP, int NR>
int stream_as(Ctx* ctx, const AttnArgs& a, cudaStream_t st) {
  constexpr bool WIDE = sizeof(T) == 4;
  constexpr int smem = stream_smem<DP, NR, WIDE>();
  static_assert(smem >= query_bytes<DP, NR, WIDE>() + kStreamWarps * 8 * NR * (DP + 4) * 4, "the parts of a segment are joined where the ring was");
  static_assert(stream_blocks<DP, NR>() * (smem + 2048) <= 227 * 1024, "resident blocks");
  static DeviceOnce once;
  const cudaError_t e = once.smem(device_of(ctx), (const void*)kv_attention_stream<T, DP, NR>, smem);
  if (e != cudaSuccess) return check_cuda(ctx, e, "kv_attention");
  const int grid = std::min(sm_count(ctx) * stream_blocks<DP, NR>(), kMaxStreamGrid);
  launch_pdl(kv_attention_stream<T, DP, NR>, dim3(grid), dim3(32 * kStreamWarps), smem, st, a);
  count_launch(ctx);
  if (!a.uncut) {
    launch_pdl(kv_attention_join<T, DP, NR>, dim3(grid, DP / 16), dim3(32 * NR * kJoinWays), 0, st, a);
    count_launch(ctx);
  }
  return check_cuda(ctx, cudaGetLastError(), "kv_attention");
}
// rows: of the longest entry, as far as known
template <typename T>
int stream_of(Ctx* ctx, const AttnArgs& a, int64_t rows, cudaStream_t st) {
  if (a.cache.dim > 128) return rows <= 8 ? stream_as<T, 256, 1>(ctx, a, st) : stream_as<T, 256, 2>(ctx, a, st);
  if (a.cache.dim > 64) {
    if (rows <= 8) return stream_as<T, 128, 1>(ctx, a, st);
    if constexpr (sizeof(T) == 2)
      if (rows > 16) return stream_as<T, 128, 4>(ctx, a, st);
    return stream_as<T, 128, 2>(ctx, a, st);
  }
  return rows <= 8 ? stream_as<T, 64, 1>(ctx, a, st) : rows <= 16 ? stream_as<T, 64, 2>(ctx, a, st) : stream_as<T, 64, 4>(ctx, a, st);
}

}  // namespace

// Contexts known to be no longer than this are not cut: the second kernel and its working memory cost more than an uneven load.
// us, single bf16 tokens, uncut / cut, entries x cache heads x group, dim:
//   1 x 8 x 4, 128    256 tokens 8.5 / 11.7    512 11.0 / 11.9    1024 16.3 / 12.0
//   8 x 12 x 1, 64    256 tokens 8.8 / 10.3    512 12.1 / 11.3    1024 17.9 / 12.7
//   64 x 8 x 4, 128   256 tokens 15.4 / 20.0   512 20.7 / 25.3    1024 38.6 / 36.9    2048 66.8 / 58.2
constexpr int kUncutTokens = 512;

int64_t kv_attention_work(Ctx*, const CacheView& c, int max_len) {
  if (max_len > 0 && max_len <= kUncutTokens) return 0;
  return c.dim <= 64 ? stream_work<64, 4>() : c.dim <= 128 ? stream_work<128, 4>() : stream_work<256, 2>();
}

int launch_kv_attention(Ctx* ctx, const PoolView& p, const CacheView& c, const BatchView& b, const void* q, int64_t q_row, int64_t q_head,
                        int q_heads, void* out, int64_t o_row, int64_t o_head, int dtype, int max_rows, int max_len, float scale, int causal, int window,
                        void* work, cudaStream_t st) {
  if (b.n == 0 || b.rows == 0) return QCFG_OK;
  const int uncut = max_len > 0 && max_len <= kUncutTokens;
  const AttnArgs a{p, c, b, q, out, q_row, q_head, o_row, o_head, q_heads, causal, window, uncut, scale * 1.44269504088896f, work, err_word(ctx)};
  int64_t rows = !b.starts ? 1 : max_rows > 0 ? max_rows : (b.rows + b.n - 1) / b.n;
  if (prompt_pays(ctx, a, dtype, rows)) return launch_prompt(ctx, a, dtype, st);
  rows *= q_heads / c.heads;
  return dtype == QCFG_FP32 ? stream_of<float>(ctx, a, rows, st) : dtype == QCFG_BF16 ? stream_of<__nv_bfloat16>(ctx, a, rows, st)
                                                                                       : stream_of<__half>(ctx, a, rows, st);
}

}  // namespace qcfg
