// Attention over the paged 8-bit cache for prompts: many query rows, so the products are the work and go to tcgen05.
//
// A block owns 256 query rows of one cache head, as two tiles of 128 rows (the M of an MMA); a row is a (query token, head of the
// group).  It walks the tokens its rows see in steps of 128:
//   warps 0-3, 4-7   one thread a row of tile 0 / tile 1: scores from TMEM, running reference, weights back to TMEM as fp16
//                    (over the scores they come from), which is where the second product takes its A operand from.
//   warps 8-10       bring the codes of the next step from global memory to registers, and turn the present ones into fp16 in shared
//                    memory: 128-byte rows, 128B swizzle, for keys (K-major B operand) and values (MN-major) alike.
//   warp 11          issues the MMAs: S0, S1, then for each step O0 += P0 V, S0 of the next step, O1 += P1 V, S1 of the next step.
//                    While one tile's weights are computed, the tensor core works for the other.
// Each step and tile costs 2 x 128 x 128 x dim products (1024 cycles for both tiles at dim 128, twice) and 128 x 128 exponentials
// (16 per cycle: 2048 cycles for both tiles): the exponentials and the tensor core are equally long.  43% of the issue slots are used.
//
// What bounds it is neither but the chain of one tile: a step takes 4300 cycles, 2450 for a warp's 32 rows of weights (also where it
// has its scheduler to itself), 350 until the tensor core knows of them, 1500 for the two products and the way back.  A block
// costs 14000 cycles besides its steps (who it is, the queries, the first codes, the output).  4 entries of up to 2048 bf16 tokens behind up
// to 4000, 32 heads on 8 of 128: 367 us, 836 TFLOP/s, 51% of the measured bf16 rate; 32 entries of up to 384 fp32 tokens, 12 heads of 64: 73 us.
// Tried against 370 us then: scores, weights and products in halves of 64 tokens, so that a tile never waits (403: 48 MMAs a step in
// place of 32, at 54 cycles each whatever their width), weights in halves only (398), a warp that issues for each tile (448: registers),
// queries fetched before the TMEM is there (383: registers).
// Numbers as in the streaming kernel: codes are exact in fp16, a page's key scale multiplies the scores' factor, its value scale the
// weights.
#include <algorithm>

#include "attention.cuh"
#include "ptx.cuh"

namespace qcfg {

namespace {

constexpr int kTileRows = 128;
constexpr int kStepTokens = 128;
constexpr int kGroups = kStepTokens / 16;        // scales are looked up for each 16 tokens
constexpr int kSoftWarps = 8, kConvWarps = 3;      // and one that issues: three warps a scheduler, 168 registers a thread
constexpr int kPromptThreads = 32 * (kSoftWarps + kConvWarps + 1);
constexpr int kTables = 4;
// fp32: the second half of a weight, at most 2^-12 of it (2^4), is held times this, so that the many small weights of a long context
// keep their digits: as it is it would end at 2^-25, next to a largest weight of 1 (100 tokens, values up to 9.5: off by 1.3e-6).
constexpr float kRest = 1024.0f;

template <int D, bool WIDE> __host__ __device__ constexpr int q_tile_bytes() { return kTileRows * D * 2 * (WIDE ? 2 : 1); }
template <int D> __host__ __device__ constexpr int kv_tile_bytes() { return kStepTokens * D * 2; }
template <int D, bool WIDE> __host__ __device__ constexpr int prompt_smem() {
  const int used = 1024 + 2 * q_tile_bytes<D, WIDE>() + 4 * kv_tile_bytes<D>();
  return used < 118 * 1024 ? 118 * 1024 : used;  // one block per SM: it takes all of the TMEM
}

struct __align__(16) Scales {          // of a step
  float key[kGroups];    // -1: no such tokens
  float value[kGroups], log_value[kGroups], inv_value[kGroups];
};

__device__ __forceinline__ void mma_f16(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t accumulate) {
  asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\ttcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n\t}"
               ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"(accumulate) : "memory");
}
__device__ __forceinline__ void mma_f16_ta(uint32_t d, uint32_t a_tmem, uint64_t b, uint32_t idesc, uint32_t accumulate) {
  asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\ttcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}"
               ::"r"(d), "r"(a_tmem), "l"(b), "r"(idesc), "r"(accumulate) : "memory");
}
__device__ __forceinline__ void tmem_ld16(uint32_t taddr, uint32_t (&v)[16]) {
  asm volatile("tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];"
               : "=r"(v[0]), "=r"(v[1]), "=r"(v[2]), "=r"(v[3]), "=r"(v[4]), "=r"(v[5]), "=r"(v[6]), "=r"(v[7]), "=r"(v[8]), "=r"(v[9]), "=r"(v[10]),
                 "=r"(v[11]), "=r"(v[12]), "=r"(v[13]), "=r"(v[14]), "=r"(v[15]) : "r"(taddr));
}
__device__ __forceinline__ void tmem_st8(uint32_t taddr, const uint32_t (&v)[8]) {
  asm volatile("tcgen05.st.sync.aligned.32x32b.x8.b32 [%8], {%0, %1, %2, %3, %4, %5, %6, %7};"
               ::"r"(v[0]), "r"(v[1]), "r"(v[2]), "r"(v[3]), "r"(v[4]), "r"(v[5]), "r"(v[6]), "r"(v[7]), "r"(taddr) : "memory");
}
__device__ __forceinline__ void tmem_st16(uint32_t taddr, const uint32_t (&v)[16]) {
  asm volatile("tcgen05.st.sync.aligned.32x32b.x16.b32 [%16], {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15};"
               ::"r"(v[0]), "r"(v[1]), "r"(v[2]), "r"(v[3]), "r"(v[4]), "r"(v[5]), "r"(v[6]), "r"(v[7]), "r"(v[8]), "r"(v[9]), "r"(v[10]), "r"(v[11]),
                 "r"(v[12]), "r"(v[13]), "r"(v[14]), "r"(v[15]), "r"(taddr) : "memory");
}
__device__ __forceinline__ void tmem_st_wait() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }

// Descriptor of a tile of 128-byte rows, 128B swizzle: 8-row groups 1024 bytes apart, and (MN-major) 64-element blocks `lead` bytes apart
__device__ __forceinline__ uint64_t tile_desc(uint32_t addr, uint32_t lead) {
  return (uint64_t)((addr >> 4) & 0x3FFFu) | (uint64_t)(lead >> 4) << 16 | (uint64_t)(1024 >> 4) << 32 | 1ull << 46 | 2ull << 61;
}

template <typename T, int D>
__global__ void __launch_bounds__(kPromptThreads, 1) kv_attention_prompt(const AttnArgs a) {
  asm volatile("griddepcontrol.wait;" ::: "memory");
  constexpr bool WIDE = sizeof(T) == 4;
  constexpr int HALVES = D / 64, HALF = kTileRows * 128;              // bytes of 64 columns of a tile
  constexpr int kUnitOrder = WIDE ? 4 : 0;                            // fp32 calls hold weights times 2^4
  constexpr uint32_t kCols = 512, kPart = WIDE ? 16 : 8;             // columns of the weights of 16 tokens (fp32: two fp16 numbers each)
  extern __shared__ uint8_t raw_smem[];
  __shared__ uint64_t bars[15];
  __shared__ uint32_t tmem_at, magic_word;
  __shared__ int abort_word;
  __shared__ struct { int64_t row0; int rows, nth, seq, len, claim; } mine;
  __shared__ Scales scales[kTables];
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  const int group = a.q_heads / a.cache.heads, page = a.pool.page, item = blockIdx.x / a.cache.heads, hk = blockIdx.x - item * a.cache.heads;
  const int per_tile = kTileRows / group, per_block = 2 * per_tile;    // query tokens

  // ---- which rows: entry i owns the blocks starts[i] / per_block + i .. of each head, the last tokens (the longest rows) first.  A thread
  // looks at an entry, so that all that has to be known is fetched at once.
  if (tid == 0) mine.claim = -1;
  __syncthreads();
  for (int i0 = 0; i0 < a.batch.n; i0 += kPromptThreads) {
    const int i = i0 + tid;
    if (i < a.batch.n) {
      int64_t r0, r1;
      if (!entry_rows(a.batch, i, r0, r1)) atomicOr(a.err, ERR_PAGE);
      const int q = entry_seq(a.batch, a.pool, i, a.err), held = q < 0 ? 0 : seq_len(a.pool, q);
      const int64_t nth = item - (a.batch.starts ? (int64_t)a.batch.starts[i] / per_block + i : 2 * (int64_t)i);
      if (nth >= 0 && nth < (r1 - r0 + per_block - 1) / per_block && atomicCAS(&mine.claim, -1, i) == -1) {      // one at most, where starts ascend
        mine.row0 = r0;
        mine.rows = (int)(r1 - r0);
        mine.nth = (int)nth;
        mine.seq = q;
        mine.len = held;
      }
    }
  }
  __syncthreads();
  if (mine.claim < 0) return;
  const int64_t row0 = mine.row0;
  const int rows = mine.rows, s = mine.seq, len = mine.len;
  const int t_first = ((rows + per_block - 1) / per_block - 1 - mine.nth) * per_block;              // first query token
  const int t_last = min(t_first + per_block, rows) - 1;
  const bool two = t_first + per_tile < rows;                          // the second tile has rows
  // the tokens seen: both ends ascend with the position
  int seen_lo, seen_hi, unused;
  seen_range(a, (int64_t)len - rows + t_last, len, unused, seen_hi);
  seen_range(a, max((int64_t)len - rows + t_first, (int64_t)0), len, seen_lo, unused);
  const int tok_lo = seen_hi > 0 ? seen_lo / kStepTokens * kStepTokens : 0;
  const int steps = seen_hi > tok_lo ? (seen_hi - tok_lo + kStepTokens - 1) / kStepTokens : 0;

  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(raw_smem) + 1023) & ~(uintptr_t)1023);
  const uint32_t q_sm = smem_u32(smem), k_sm = q_sm + 2 * q_tile_bytes<D, WIDE>(), v_sm = k_sm + 2 * kv_tile_bytes<D>();
  const uint32_t bar = smem_u32(bars);
  const uint32_t k_full = bar, k_empty = bar + 16, v_full = bar + 32, v_empty = bar + 48, s_full = bar + 64, p_ready = bar + 80, o_done = bar + 96, q_full = bar + 112;
  volatile int* abort_flag = &abort_word;
  if (tid == 0) {
    for (int i = 0; i < 2; ++i) {
      mbar_init(k_full + 8 * i, kConvWarps);
      mbar_init(v_full + 8 * i, kConvWarps);
      mbar_init(k_empty + 8 * i, 1);
      mbar_init(v_empty + 8 * i, 1);
      mbar_init(s_full + 8 * i, 1);
      mbar_init(p_ready + 8 * i, 4);
      mbar_init(o_done + 8 * i, 1);
    }
    mbar_init(q_full, kSoftWarps);
    abort_word = 0;
    magic_word = 0x64646464u;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (warp == kSoftWarps + kConvWarps) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_u32(&tmem_at)), "r"(kCols) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = tmem_at;
  // TMEM columns: scores (then weights) of the tiles, accumulators, and for fp32 those of the second
  // halves: an MMA's sum is not rounded but cut, so small products are not added to large sums one by one
  const uint32_t s_at = tmem, o_at = tmem + 256, l_at = tmem + 384;
  // The next kernel may begin only now: it could take the TMEM of an SM in front of this block, and then wait for it.
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");

  if (steps > 0 && warp >= kSoftWarps && warp < kSoftWarps + kConvWarps) {
    // ------------------------------------------------------------------ codes to fp16
    const int cw = warp - kSoftWarps;              // runs of 8 tokens cw, cw + 3, ... of a step's 16
    constexpr int RUNS = (kStepTokens / 8 + kConvWarps - 1) / kConvWarps;
    const uint32_t magic = *(volatile uint32_t*)&magic_word;
    const int32_t* table = a.pool.table + (int64_t)(s < 0 ? 0 : s) * a.pool.max_pages;
    // lanes 0-7: the page of a group of 16 tokens, -1 where there is none
    auto look_up = [&](int step) {
      const int tok = tok_lo + step * kStepTokens + 16 * (lane & 7);
      if (step >= steps || tok >= len) return -1;
      const int p = __ldg(table + tok / page);
      if (p >= 0 && p < a.pool.n_pages) return p;
      if (lane < 8 && cw == 0) atomicOr(a.err, ERR_PAGE);
      return -1;
    };
    // a warp-wide access: 8 tokens x 4 chunks of 16 codes
    const int r8 = lane >> 2, c4 = lane & 3;
    const uint32_t put = (uint32_t)(r8 * 128), flip = (uint32_t)r8;
    // Where a lane's codes of its runs lie in both tensors.  Tokens that are not there are read from page 0: whatever the codes are, they
    // are numbers, their scores are masked and their weights 0.
    int in_page[RUNS];
    int64_t place[RUNS];
#pragma unroll
    for (int o = 0; o < RUNS; ++o) in_page[o] = ((hk * page + ((8 * (cw + o * kConvWarps)) & (page - 1)) + r8) * D + c4 * 16);
    const int page_bytes = a.cache.heads * page * D;
    auto find = [&](int pages) {
#pragma unroll
      for (int o = 0; o < RUNS; ++o) place[o] = (int64_t)max(__shfl_sync(0xffffffffu, pages, min((cw + o * kConvWarps) >> 1, kGroups - 1)), 0) * page_bytes + in_page[o];
    };
    auto load = [&](const int8_t* base, uint4 (&to)[RUNS * HALVES]) {
#pragma unroll
      for (int o = 0; o < RUNS; ++o) {
        if (cw + o * kConvWarps >= kStepTokens / 8) break;
#pragma unroll
        for (int h = 0; h < HALVES; ++h) to[o * HALVES + h] = __ldg(reinterpret_cast<const uint4*>(base + place[o] + h * 64));
      }
    };
    auto store = [&](uint32_t tile, const uint4 (&from)[RUNS * HALVES]) {
#pragma unroll
      for (int o = 0; o < RUNS; ++o) {
        const int run = cw + o * kConvWarps;
        if (run >= kStepTokens / 8) break;
#pragma unroll
        for (int h = 0; h < HALVES; ++h) {
          uint4 v = from[o * HALVES + h];
          asm volatile("" : "+r"(v.x), "+r"(v.y), "+r"(v.z), "+r"(v.w) :: "memory");      // not in front of the wait for the stage
          const uint32_t x = v.x ^ 0x80808080u, y = v.y ^ 0x80808080u, z = v.z ^ 0x80808080u, w = v.w ^ 0x80808080u;
          const uint32_t at = tile + put + run * 1024 + h * HALF;
          st_shared_v4(at + (((2 * c4) ^ flip) << 4), two_codes<0x4140>(x, magic), two_codes<0x4342>(x, magic), two_codes<0x4140>(y, magic), two_codes<0x4342>(y, magic));
          st_shared_v4(at + (((2 * c4 + 1) ^ flip) << 4), two_codes<0x4140>(z, magic), two_codes<0x4342>(z, magic), two_codes<0x4140>(w, magic), two_codes<0x4342>(w, magic));
        }
      }
    };
    uint4 kc[RUNS * HALVES], vc[RUNS * HALVES];
    float k_max = -1.0f, v_max = -1.0f;
    auto load_scales = [&](int pages) {            // the first warp's lanes 0-7
      k_max = v_max = -1.0f;
      if (cw == 0 && lane < kGroups && pages >= 0) {
        k_max = __ldg(a.cache.k_absmax + (int64_t)pages * a.cache.heads + hk);
        v_max = __ldg(a.cache.v_absmax + (int64_t)pages * a.cache.heads + hk);
      }
    };
    int next = look_up(0);
    find(next);
    load(a.cache.k, kc);
    load_scales(next);
    load(a.cache.v, vc);
    next = look_up(1);

    for (int j = 0; j < steps; ++j) {
      const uint32_t st = j & 1, ph = (j >> 1) & 1;
      if (j >= 2 && !mbar_wait_warp(k_empty + 8 * st, ph ^ 1, abort_flag, a.err)) break;
      store(k_sm + st * kv_tile_bytes<D>(), kc);
      if (cw == 0 && lane < kGroups) {
        Scales& sc = scales[j % kTables];
        const int g = lane;
        const bool ok = k_max >= 0.0f;
        sc.key[g] = !ok ? -1.0f : k_max > 0.0f ? k_max * (1.0f / kQmax8) : 1.0f;
        const float value = ok ? fmaxf(v_max * (1.0f / kQmax8), 1.2e-38f) : 1.2e-38f;       // (a page of zeros may have any)
        sc.value[g] = value;
        sc.log_value[g] = log2f(value);
        sc.inv_value[g] = __fdiv_rn(1.0f, value);
      }
      asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
      __syncwarp();
      if (lane == 0) mbar_arrive(k_full + 8 * st);
      if (j + 1 < steps) {
        find(next);
        load(a.cache.k, kc);
        load_scales(next);
      }
      if (j >= 2 && !mbar_wait_warp(v_empty + 8 * st, ph ^ 1, abort_flag, a.err)) break;
      store(v_sm + st * kv_tile_bytes<D>(), vc);
      asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
      __syncwarp();
      if (lane == 0) mbar_arrive(v_full + 8 * st);
      if (j + 1 < steps) load(a.cache.v, vc);
      next = look_up(j + 2);
    }
  } else if (steps > 0 && warp == kSoftWarps + kConvWarps) {
    // ------------------------------------------------------------------ products
    // fp32 accumulators, fp16 operands; the second product's B operand (values) is MN-major
    constexpr uint32_t kIdescS = (1u << 4) | ((uint32_t)(kStepTokens >> 3) << 17) | ((uint32_t)(kTileRows >> 4) << 24);
    constexpr uint32_t kIdescO = (1u << 4) | (1u << 16) | ((uint32_t)(D >> 3) << 17) | ((uint32_t)(kTileRows >> 4) << 24);
    const bool elected = elect_one();
    const int n_tiles = two ? 2 : 1;
    bool ok = true;
    auto product_s = [&](int i, int j) {
      const uint64_t k0 = tile_desc(k_sm + (j & 1) * kv_tile_bytes<D>(), 16);
#pragma unroll
      for (int part = 0; part < (WIDE ? 2 : 1); ++part) {       // the queries' second halves first: they are added up while the sum is small
        const uint64_t q0 = tile_desc(q_sm + i * q_tile_bytes<D, WIDE>() + (WIDE && part == 0 ? kTileRows * D * 2 : 0), 16);
#pragma unroll
        for (int k = 0; k < D / 16; ++k) {
          const uint32_t off = ((k >> 2) * HALF + (k & 3) * 32) >> 4;
          mma_f16(s_at + 128 * i, q0 + off, k0 + off, kIdescS, part + k > 0);
        }
      }
      tc_commit(s_full + 8 * i);
    };
    auto product_o = [&](int i, int j) {
      const uint64_t v0 = tile_desc(v_sm + (j & 1) * kv_tile_bytes<D>(), HALF);
#pragma unroll
      for (int part = 0; part < (WIDE ? 2 : 1); ++part)
#pragma unroll
        for (int k = 0; k < kStepTokens / 16; ++k)
          mma_f16_ta((part ? l_at : o_at) + D * i, s_at + 128 * i + kPart * k + 8 * part, v0 + ((k * 2048) >> 4), kIdescO, j + k > 0);
    };
    ok = mbar_wait_warp(q_full, 0, abort_flag, a.err) && mbar_wait_warp(k_full, 0, abort_flag, a.err);
    tc_fence_after();
    if (ok) {
      if (elected) {
        for (int i = 0; i < n_tiles; ++i) product_s(i, 0);
        tc_commit(k_empty);
      }
      __syncwarp();
    }
    for (int j = 0; j < steps && ok; ++j) {
      const uint32_t st = j & 1, ph = (j >> 1) & 1, st1 = st ^ 1, ph1 = ((j + 1) >> 1) & 1;
      const bool more = j + 1 < steps;
      ok = mbar_wait_warp(v_full + 8 * st, ph, abort_flag, a.err) && (!more || mbar_wait_warp(k_full + 8 * st1, ph1, abort_flag, a.err));
      for (int i = 0; i < n_tiles && ok; ++i) {
        ok = mbar_wait_warp(p_ready + 8 * i, j & 1, abort_flag, a.err);
        if (!ok) break;
        tc_fence_after();
        if (elected) {
          product_o(i, j);
          if (more) product_s(i, j + 1);
          else tc_commit(o_done + 8 * i);
          if (i == n_tiles - 1) {
            tc_commit(v_empty + 8 * st);
            if (more) tc_commit(k_empty + 8 * st1);
          }
        }
        __syncwarp();
      }
    }
    __syncwarp();
  } else if (warp < kSoftWarps) {
    // ------------------------------------------------------------------ queries: a thread a row
    int lo = 0, hi = 0x7fffffff, out_row = -1, out_head = 0;
    float row_f = 0.0f;
    // Rows are read and written whole, LPR lanes each: a lane for each row would touch 32 rows with every access.
    constexpr int V = Vec<T>::N, LPR = D / V, RPA = 32 / LPR;          // elements a lane, lanes a row, rows an access
    const int my_chunk = lane % LPR;
    {
      const int tile = warp >> 2, r = tid & 127;
      const int tok = t_first + tile * per_tile + r / group;
      const T* q = nullptr;
      if (r < per_tile * group && tok < rows) {
        out_row = tok;
        out_head = hk * group + r % group;
        q = reinterpret_cast<const T*>(a.q) + (row0 + tok) * a.q_row + out_head * a.q_head;
        seen_range(a, (int64_t)len - rows + tok, len, lo, hi);
      }
      union Piece { uint4 u; T t[V]; } held[LPR];
#pragma unroll
      for (int c = 0; c < LPR; ++c) {
        const T* from = reinterpret_cast<const T*>(__shfl_sync(0xffffffffu, reinterpret_cast<unsigned long long>(q), c * RPA + lane / LPR));
        held[c].u = from ? __ldg(reinterpret_cast<const uint4*>(from) + my_chunk) : make_uint4(0, 0, 0, 0);
      }
      int shift = 0;
#pragma unroll
      for (int c = 0; c < LPR; ++c) {
        unsigned top = 0;
#pragma unroll
        for (int j = 0; j < V; ++j) top = max(top, abs_bits(to_float<T>(held[c].t[j])));
#pragma unroll
        for (int o = 1; o < LPR; o <<= 1) top = max(top, __shfl_xor_sync(0xffffffffu, top, o));
        const int row = c * RPA + lane / LPR, up_by = row_shift(top);
        // the row's own thread needs it too
#pragma unroll
        for (int k = 0; k < RPA; ++k) {
          const int other = __shfl_sync(0xffffffffu, up_by, k * LPR);
          if (lane == c * RPA + k) shift = other;
        }
        const float up = top < 0x7f800000u ? exp2_of(up_by) : __int_as_float(0x7fffffff);      // an Inf makes the row NaN, like a NaN
        uint32_t w[V / 2], l[V / 2];
#pragma unroll
        for (int j = 0; j < V / 2; ++j) {
          const float x = to_float<T>(held[c].t[2 * j]) * up, y = to_float<T>(held[c].t[2 * j + 1]) * up;
          const __half2 h = __floats2half2_rn(x, y);
          w[j] = h2_bits(h);
          l[j] = pack_h2(x - __low2float(h), y - __high2float(h));
        }
        const int at8 = my_chunk * V / 8, r128 = 32 * (warp & 3) + row;       // 16 bytes of fp16
        const uint32_t to = q_sm + tile * q_tile_bytes<D, WIDE>() + r128 * 128 + (at8 >> 3) * HALF + (((at8 & 7) ^ (r128 & 7)) << 4);
        if constexpr (WIDE) {
          const uint32_t half = (my_chunk & 1) * 8;
          asm volatile("st.shared.v2.b32 [%0], {%1, %2};" ::"r"(to + half), "r"(w[0]), "r"(w[1]) : "memory");
          asm volatile("st.shared.v2.b32 [%0], {%1, %2};" ::"r"(to + half + kTileRows * D * 2), "r"(l[0]), "r"(l[1]) : "memory");
        } else {
          st_shared_v4(to, w[0], w[1], w[2], w[3]);
        }
      }
      row_f = a.scale * exp2_of(-shift);
      asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
      __syncwarp();
      if (lane == 0) mbar_arrive(q_full);
    }
    // ------------------------------------------------------------------ weights
    const int i = warp >> 2;
    const uint32_t lanes = (uint32_t)(32 * (warp & 3)) << 16;
    const uint32_t s_row = s_at + 128 * i + lanes, o_row = o_at + D * i + lanes, l_row = l_at + D * i + lanes;
    float ref = -INFINITY, sum = 0.0f;
    // Weights are multiplied with their page's value scale times `low`, a power of two that follows the row's largest such product as
    // ref follows its largest score (2^value_ref; low = the weights' unit times 2^(ref - value_ref)): so what a row keeps depends on
    // nothing but the tokens it sees, whatever the values of others in the block.
    float value_ref = -INFINITY, low = exp2_of(kUnitOrder);
    bool ok = true, fresh = true;      // fresh: no reference yet
    const int n = i == 0 || two ? steps : 0;
    for (int j = 0; j < n; ++j) {
      const int tok = tok_lo + j * kStepTokens;
      const int from = lo - tok, to = hi - tok;               // of this step's tokens the row sees [from, to)
      if (!mbar_wait_warp(s_full + 8 * i, j & 1, abort_flag, a.err)) { ok = false; break; }
      tc_fence_after();
      const Scales& sc = scales[j % kTables];
      // fp32 calls multiply weights with their scale; others add its logarithm to the exponent and take it out of the sums of 16: 64
      // products a step less (4 entries of 2048 tokens behind 4000, 32 heads on 8 of 128: 711 -> 684 us), for digits that 16 bits do not hold
      float f[kGroups], value[kGroups], inv_value[WIDE ? 1 : kGroups];
#pragma unroll
      for (int g = 0; g < kGroups; g += 4) {
        *reinterpret_cast<float4*>(f + g) = *reinterpret_cast<const float4*>(sc.key + g);
        *reinterpret_cast<float4*>(value + g) = *reinterpret_cast<const float4*>((WIDE ? sc.value : sc.log_value) + g);
        if constexpr (!WIDE) *reinterpret_cast<float4*>(inv_value + g) = *reinterpret_cast<const float4*>(sc.inv_value + g);
      }
      bool some = false;
#pragma unroll
      for (int g = 0; g < kGroups; ++g) {
        some |= f[g] < 0.0f;
        f[g] = fmaxf(row_f * f[g], 1.2e-38f);
      }
      const bool masked = __any_sync(0xffffffffu, some || from > 0 || to < kStepTokens);
      // which of 32 tokens are seen, a bit each (a comparison and a look at the scale for each token made such steps 5 times as long)
      auto seen_bits = [&](int c) {
        const int first = from - 32 * c, end = to - 32 * c;
        const uint32_t below = end <= 0 ? 0u : end >= 32 ? 0xffffffffu : (1u << end) - 1u;
        const uint32_t above = first <= 0 ? 0xffffffffu : first >= 32 ? 0u : 0xffffffffu << first;
        return below & above & (sc.key[2 * c] < 0.0f ? 0xffff0000u : 0xffffffffu) & (sc.key[2 * c + 1] < 0.0f ? 0xffffu : 0xffffffffu);
      };
      // Weights of BLOCK x 32 tokens at a time (all of them; fp32, with twice as many to hold, 32), over scores that have been read: group
      // g of 16 in columns kPart * g on.  The next 32 scores are on their way meanwhile.  The reference is a whole number, and moves only
      // when a row has none yet or a sum of 16 weights no longer fits fp16: what has been written and summed up is then scaled by a
      // power of two.  So no maximum is taken of most scores.
      constexpr int BLOCK = WIDE ? 1 : 4;
      float part = 0.0f;             // of the step's exponentials
#pragma unroll
      for (int b = 0; b < 4; b += BLOCK) {
        uint32_t p[2 * BLOCK][8], l[WIDE ? 2 : 1][WIDE ? 8 : 1];
        float block_part;
        bool large;
        auto take = [&]() {
          const float shift = weight_bias<WIDE>() - (ref == -INFINITY ? 0.0f : ref);
          const float inv_low = __uint_as_float((254u << 23) - __float_as_uint(low)), log_low = shift + (float)((int)(__float_as_uint(low) >> 23) - 127);
          block_part = 0.0f;
          large = false;
          uint32_t v[2][32];
          tmem_ld32_issue(s_row + 32 * b, v[0]);
#pragma unroll
          for (int c = b; c < b + BLOCK; ++c) {
            uint32_t (&x32)[32] = v[(c - b) & 1];
            tmem_ld_wait();
            if (c + 1 < b + BLOCK) tmem_ld32_issue(s_row + 32 * (c + 1), v[(c + 1 - b) & 1]);
            if (masked) {
              const uint32_t seen = seen_bits(c);
#pragma unroll
              for (int k = 0; k < 32; ++k) x32[k] = seen & 1u << k ? x32[k] : 0xff800000u;
            }
            float2 both_at, both_share;
            if constexpr (!WIDE) {
              both_at = __fadd2_rn(make_float2(value[2 * c], value[2 * c + 1]), make_float2(log_low, log_low));
              both_share = __fmul2_rn(make_float2(inv_value[2 * c], inv_value[2 * c + 1]), make_float2(inv_low, inv_low));
            }
#pragma unroll
            for (int z = 0; z < 2; ++z) {
              const float f1 = f[2 * c + z];
              float at1, share1;
              if constexpr (WIDE) {
                at1 = shift;
                share1 = fminf(value[2 * c + z] * low, 8.5e37f);          // (kept finite for tokens not seen; a weight of 2^-110 and less may lose)
              } else {                       // never below 2^-100, so that the sums keep what the values lose
                at1 = fmaxf(z ? both_at.y : both_at.x, shift - 100.0f);
                share1 = fminf(z ? both_share.y : both_share.x, 0x1p100f);
              }
              const float2 fg = make_float2(f1, f1), at = make_float2(at1, at1), share = make_float2(share1, share1);
              float2 acc[2] = {make_float2(0.0f, 0.0f), make_float2(0.0f, 0.0f)};
#pragma unroll
              for (int k = 0; k < 8; ++k) {
                const float2 x = __ffma2_rn(make_float2(__uint_as_float(x32[16 * z + 2 * k]), __uint_as_float(x32[16 * z + 2 * k + 1])), fg, at);
                const float2 e = make_float2(ex2(x.x), ex2(x.y));
                acc[k & 1] = __fadd2_rn(acc[k & 1], e);
                const float2 w = WIDE ? __fmul2_rn(e, share) : e;
                const __half2 h = __floats2half2_rn(w.x, w.y);
                p[2 * (c - b) + z][k] = h2_bits(h);
                if constexpr (WIDE) {
                  const float2 rest = __fmul2_rn(__fadd2_rn(w, make_float2(-__low2float(h), -__high2float(h))), make_float2(kRest, kRest));
                  l[z][k] = pack_h2(rest.x, rest.y);
                }
              }
              acc[0] = __fadd2_rn(acc[0], acc[1]);
              const float of16 = acc[0].x + acc[0].y;
              large |= !((WIDE ? of16 * share1 : of16) <= 65504.0f);       // (a NaN counts; it stays one)
              block_part = WIDE ? block_part + of16 : fmaf(of16, share1, block_part);
            }
          }
          large |= !(block_part <= 0x1p40f);
        };
        bool move = fresh;                 // of the row's reference; written once, so that a step's code stays in the instruction cache and in registers
#pragma unroll 1
        for (int go = 0; go < 2; ++go) {
          if (__any_sync(0xffffffffu, move)) {
            float most = -INFINITY, most_value = -INFINITY;
#pragma unroll 1
            for (int g = 2 * b; g < 2 * (b + BLOCK); ++g) {
              uint32_t x[16];
              tmem_ld16(s_row + 16 * g, x);
              tmem_ld_wait();
              const uint32_t seen = masked ? seen_bits(g >> 1) >> (16 * (g & 1)) : 0xffffu;
              float m = -INFINITY;
#pragma unroll
              for (int k = 0; k < 16; ++k) m = fmaxf(m, seen & 1u << k ? __uint_as_float(x[k]) : -INFINITY);
              m *= fmaxf(row_f * sc.key[g], 1.2e-38f);
              most = fmaxf(most, m);
              most_value = fmaxf(most_value, m + (float)((int)(__float_as_uint(sc.value[g]) >> 23) - 126));      // the order the scale does not reach
            }
            const float was = ref, value_was = value_ref;
            if (move) {
              ref = fmaxf(ref, ceilf(most));
              value_ref = fmaxf(value_ref, ceilf(most_value));
            }
            fresh = ref == -INFINITY;
            if (!fresh) {
              value_ref = fmaxf(value_ref, ref - 110.0f);
              low = exp2_of(kUnitOrder - (int)(value_ref - ref));
            }
            const float keep = ex2(was - (fresh ? 0.0f : ref)), keep_values = ex2(value_was - (fresh ? 0.0f : value_ref));
            if (__any_sync(0xffffffffu, keep != 1.0f || keep_values != 1.0f)) {
              sum *= keep;
              part *= keep;
              if constexpr (WIDE) {            // this step's weights so far: both halves as one number, halved anew behind the factor
                if (b > 0) tmem_st_wait();     // loads are not ordered behind stores that have not been waited for
#pragma unroll 1
                for (int h = 0; h < 2 * b; ++h) {
                  uint32_t w[16];
                  tmem_ld16(s_row + 16 * h, w);
                  tmem_ld_wait();
#pragma unroll
                  for (int k = 0; k < 8; ++k) {
                    const float2 e = __half22float2(*reinterpret_cast<const __half2*>(&w[k])), r = __half22float2(*reinterpret_cast<const __half2*>(&w[8 + k]));
                    const float x = fmaf(r.x, 1.0f / kRest, e.x) * keep_values, y = fmaf(r.y, 1.0f / kRest, e.y) * keep_values;
                    const __half2 hi = __floats2half2_rn(x, y);
                    w[k] = h2_bits(hi);
                    w[8 + k] = pack_h2((x - __low2float(hi)) * kRest, (y - __high2float(hi)) * kRest);
                  }
                  tmem_st16(s_row + 16 * h, w);
                }
              }
              // the products so far have been completed in front of these scores
#pragma unroll 1
              for (int h = 0; j > 0 && h < (WIDE ? 2 : 1) * D / 16; ++h) {
                const uint32_t at = h < D / 16 ? o_row + 16 * h : l_row + 16 * (h - D / 16);
                uint32_t w[16];
                tmem_ld16(at, w);
                tmem_ld_wait();
#pragma unroll
                for (int k = 0; k < 16; ++k) w[k] = __float_as_uint(__uint_as_float(w[k]) * keep_values);
                tmem_st16(at, w);
              }
              tmem_st_wait();
            }
          }
          take();
          move = large;
          if (!__any_sync(0xffffffffu, move)) break;
        }
        part += block_part;
#pragma unroll
        for (int g = 0; g < 2 * BLOCK; ++g) {
          tmem_st8(s_row + kPart * (2 * b + g), p[g]);
          if constexpr (WIDE) tmem_st8(s_row + kPart * (2 * b + g) + 8, l[g]);
        }
      }
      sum += part;
      tmem_st_wait();
      tc_fence_before();
      __syncwarp();
      if (lane == 0) mbar_arrive(p_ready + 8 * i);
    }
    // ---- out
    if (n > 0 && ok) ok = mbar_wait_warp(o_done + 8 * i, 0, abort_flag, a.err);
    if (ok && (i == 0 || two)) {
      tc_fence_after();
      float inv = sum > 0.0f ? __fdiv_rn(1.0f, sum) : (sum == 0.0f ? 0.0f : sum);
      inv *= __uint_as_float((254u << 23) - __float_as_uint(low));      // its inverse: a power of two
      // through the tile's queries, which nobody reads any more: a warp's 32 rows of D elements
      const uint32_t stage = q_sm + i * q_tile_bytes<D, WIDE>() + (warp & 3) * 32 * D * (int)sizeof(T);
#pragma unroll
      for (int c = 0; c < D / 32; ++c) {
        if (n == 0) break;               // nothing is seen (and the queries may still be on their way to shared memory)
        uint32_t v[32];
        tmem_ld32_issue(o_row + 32 * c, v);
        tmem_ld_wait();
        if constexpr (WIDE) {
          uint32_t u[32];
          tmem_ld32_issue(l_row + 32 * c, u);
          tmem_ld_wait();
#pragma unroll
          for (int k = 0; k < 32; ++k) v[k] = __float_as_uint(fmaf(__uint_as_float(u[k]), 1.0f / kRest, __uint_as_float(v[k])));
        }
#pragma unroll
        for (int k = 0; k < 32; k += V) {
          union { uint4 u; T t[V]; } w;
#pragma unroll
          for (int e = 0; e < V; ++e) w.t[e] = from_float<T>(sum == 0.0f ? 0.0f : __uint_as_float(v[k + e]) * inv);
          const int chunk = (32 * c + k) / V;
          st_shared_v4(stage + lane * D * (int)sizeof(T) + ((chunk ^ (lane & (LPR - 1))) << 4), w.u.x, w.u.y, w.u.z, w.u.w);
        }
      }
      __syncwarp();
      T* out = out_row < 0 ? nullptr : reinterpret_cast<T*>(a.out) + (row0 + out_row) * a.o_row + out_head * a.o_head;
#pragma unroll
      for (int c = 0; c < LPR; ++c) {
        const int row = c * RPA + lane / LPR;
        T* to = reinterpret_cast<T*>(__shfl_sync(0xffffffffu, reinterpret_cast<unsigned long long>(out), row));
        uint4 w;
        asm volatile("ld.shared.v4.b32 {%0,%1,%2,%3}, [%4];" : "=r"(w.x), "=r"(w.y), "=r"(w.z), "=r"(w.w)
                     : "r"(stage + row * D * (int)sizeof(T) + ((my_chunk ^ (row & (LPR - 1))) << 4)));
        if (to) reinterpret_cast<uint4*>(to)[my_chunk] = n > 0 ? w : make_uint4(0, 0, 0, 0);
      }
    }
  }
  tc_fence_before();
  __syncthreads();
  if (warp == kSoftWarps + kConvWarps) {
    tc_fence_after();
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(kCols) : "memory");
  }
}

// Blocks of a launch: entry i owns those from starts[i] / per_block + i on, for each head
int64_t prompt_blocks(const AttnArgs& a) {
  const int per_block = 2 * (kTileRows / (a.q_heads / a.cache.heads));
  return (a.batch.starts ? a.batch.rows / per_block + a.batch.n : 2 * (int64_t)a.batch.n) * a.cache.heads;
}

template <typename T, int D>
int prompt_as(Ctx* ctx, const AttnArgs& a, cudaStream_t st) {
  constexpr int smem = prompt_smem<D, sizeof(T) == 4>();
  static DeviceOnce once;
  const cudaError_t e = once.smem(device_of(ctx), (const void*)kv_attention_prompt<T, D>, smem);
  if (e != cudaSuccess) return check_cuda(ctx, e, "kv_attention");
  launch_pdl(kv_attention_prompt<T, D>, dim3((unsigned)prompt_blocks(a)), dim3(kPromptThreads), smem, st, a);
  count_launch(ctx);
  return check_cuda(ctx, cudaGetLastError(), "kv_attention");
}

}  // namespace

// Whether a call goes this way or streams the cache, by the rows of the longest entry as far as known.  A block takes 256 rows through the
// whole context, so there have to be blocks for a good part of the SMs; streaming cuts the context instead, and repeats the
// conversion of the codes for every 32 rows.  us, this way / streaming, entries x new tokens behind a context, heads x group, dim:
//   8 heads x 4, 128   8 x 8, 1000 27 / 36      8 x 64, 1000 32 / 71     32 x 4, 1000 42 / 32     32 x 8, 1000 47 / 60    32 x 16, 1000 46 / 87
//                      64 x 4, 4000 201 / 105   64 x 8, 4000 189 / 192   64 x 16, 4000 180 / 253
//                      1 x 64, 1000 31 / 37     1 x 64, 30000 488 / 171  1 x 512, 1000 38 / 113   1 x 512, 30000 502 / 1127
//   12 heads x 1, 64   8 x 32, 1000 24 / 26     8 x 64, 1000 25 / 28     8 x 128, 1000 24 / 39    32 x 32, 300 32 / 25    32 x 64, 300 34 / 35
//          (fp32)      32 x 32, 300 38 / 28     32 x 64, 300 41 / 39     4 x 128, 300 20 / 18     32 x 384, 0 71 / 177
bool prompt_pays(Ctx* ctx, const AttnArgs& a, int dtype, int64_t rows) {
  const int group = a.q_heads / a.cache.heads;
  if (group > kTileRows || (a.cache.dim != 64 && a.cache.dim != 128) || (dtype == QCFG_FP32 && a.cache.dim != 64)) return false;
  if (prompt_blocks(a) > 0x7fffffff) return false;       // (a grid's limit; the streaming kernel's grid does not grow with the batch)
  const int64_t blocks = std::max<int64_t>(a.batch.n, (a.batch.rows * group + 255) / 256) * a.cache.heads;
  return rows * group >= (a.cache.dim == 128 ? 32 : 64) && 3 * blocks >= sm_count(ctx);
}

int launch_prompt(Ctx* ctx, const AttnArgs& a, int dtype, cudaStream_t st) {
  if (dtype == QCFG_FP32) return prompt_as<float, 64>(ctx, a, st);
  if (dtype == QCFG_BF16) return a.cache.dim == 64 ? prompt_as<__nv_bfloat16, 64>(ctx, a, st) : prompt_as<__nv_bfloat16, 128>(ctx, a, st);
  return a.cache.dim == 64 ? prompt_as<__half, 64>(ctx, a, st) : prompt_as<__half, 128>(ctx, a, st);
}

}  // namespace qcfg
