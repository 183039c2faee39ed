// The paged 8-bit key/value cache: sequences take, share, give back and move pages (integers only, on the device, so that a
// captured step can run them), and keys and values are written to pages and read back.
//
// A page of a head is quantized with one maximum (Eq. 1 at b = 8 over page_tokens x head_dim values).
#include <cooperative_groups.h>

#include <algorithm>

#include "serve.cuh"

namespace cg = cooperative_groups;

namespace qcfg {

namespace {

constexpr int kPlanThreads = 1024;
constexpr int kPlanCluster = 8;          // CTAs of the calls that walk whole tables
constexpr unsigned kMark = 0x80000000u;  // a length whose sequence a running call has claimed

__device__ __forceinline__ int pages_for(int64_t tokens, int page) { return (int)((tokens + page - 1) / page); }

// Hands the lowest free pages out: page of rank r (0 .. total-1) goes to take(r, page).  One block.  False: fewer than `total`
// are free, nothing has been taken.  Two walks over the counts, each ending as soon as it has seen enough.
template <typename Take>
__device__ bool take_pages(const PoolView& p, int total, int* buf, Take take) {
  if (total == 0) return true;
  for (int pass = 0; pass < 2; ++pass) {
    int seen = 0;
    for (int p0 = 0; p0 < p.n_pages && seen < total; p0 += 4 * kPlanThreads) {
      const int at = p0 + 4 * threadIdx.x;
      unsigned free = 0;
#pragma unroll
      for (int j = 0; j < 4; ++j)
        if (at + j < p.n_pages && p.refs[at + j] == 0) free |= 1u << j;
      int sum;
      int rank = seen + block_scan(__popc(free), buf, sum);
      if (pass)
#pragma unroll
        for (int j = 0; j < 4; ++j)
          if ((free >> j & 1u) && rank < total) take(rank++, at + j);
      seen += sum;
    }
    if (seen < total) return false;
    __syncthreads();
  }
  return true;
}

// Exclusive prefix sums of need[0..n) in place, returns the total.  One block.
__device__ int scan_needs(int* need, int n, int* buf) {
  int base = 0;
  for (int i0 = 0; i0 < n; i0 += kPlanThreads) {
    const int i = i0 + threadIdx.x;
    int sum;
    const int before = block_scan(i < n ? need[i] : 0, buf, sum);
    if (i < n) need[i] = base + before;
    base += sum;
  }
  __syncthreads();
  return base;
}
// The last i with first[i] <= r (first ascends; entries without pages share a value with the next)
__device__ __forceinline__ int owner_of(const int* first, int n, int r) {
  int lo = 0, hi = n;
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (first[mid] <= r) lo = mid; else hi = mid;
  }
  return lo;
}

// Sequences get longer.  One block: a decoding step asks for a page now and then, and most calls end before the walk.
__global__ void __launch_bounds__(kPlanThreads) kv_extend_kernel(PoolView p, BatchView b, unsigned* err) {
  pdl_entry();
  extern __shared__ int sh[];
  int* need = sh;                  // [n] pages wanted, then their prefix sums
  int* grown = sh + b.n;           // [n] new length; -1: not claimed by this entry
  __shared__ int buf[33], bad;
  if (threadIdx.x == 0) bad = 0;
  __syncthreads();
  for (int i = threadIdx.x; i < b.n; i += kPlanThreads) {
    int64_t lo, hi;
    const int s = b.seqs[i];
    need[i] = 0;
    grown[i] = -1;
    if (!entry_rows(b, i, lo, hi) || s >= p.max_seqs) bad = 1;
    if (s < 0 || s >= p.max_seqs) continue;
    const int old = (int)atomicOr(reinterpret_cast<unsigned*>(p.len) + s, kMark);
    if (old < 0) { bad = 1; continue; }
    const int64_t len = old + (hi - lo);
    if (len > (int64_t)p.max_pages * p.page) bad = 1;
    else need[i] = pages_for(len, p.page) - pages_for(old, p.page);
    grown[i] = len > 0x7fffffff ? old : (int)len;
  }
  __syncthreads();
  const int total = scan_needs(need, b.n, buf);
  bool ok = bad == 0;
  if (ok)
    ok = take_pages(p, total, buf, [&](int rank, int page) {
      const int i = owner_of(need, b.n, rank), s = b.seqs[i];
      const int old = (int)((unsigned)p.len[s] & ~kMark);
      p.table[(int64_t)s * p.max_pages + pages_for(old, p.page) + rank - need[i]] = page;
      p.refs[page] = 1;
    });
  __syncthreads();
  // an append behind a refused call must not take the last tokens for the ones that got no room
  for (int i = threadIdx.x; i < b.n; i += kPlanThreads) {
    const int s = b.seqs[i];
    if (p.refused && s >= 0 && s < p.max_seqs) p.refused[s] = !ok;
    if (grown[i] < 0) continue;
    int* len = p.len + s;
    *len = ok ? grown[i] : (int)((unsigned)*len & ~kMark);
  }
  if (!ok && threadIdx.x == 0) atomicOr(err, ERR_PAGE);
}

// Gives pages back: a table entry counts for the block that takes it out, so a sequence listed twice loses its pages once.
__global__ void __launch_bounds__(128) kv_free_kernel(PoolView p, const int32_t* seqs, unsigned* err) {
  pdl_entry();
  const int s = seqs[blockIdx.x];
  if (s >= p.max_seqs && threadIdx.x == 0) atomicOr(err, ERR_PAGE);
  if (s < 0 || s >= p.max_seqs) return;
  int* row = p.table + (int64_t)s * p.max_pages;
  for (int j = threadIdx.x; j < p.max_pages; j += 128) {
    if (row[j] == -1) continue;
    const int page = atomicExch(row + j, -1);
    if (page >= 0 && page < p.n_pages) atomicSub(p.refs + page, 1);
    else if (page != -1) atomicOr(err, ERR_PAGE);
  }
  if (threadIdx.x == 0) {
    p.len[s] = 0;
    if (p.refused) p.refused[s] = 0;
  }
}

// One cluster: its first block checks the forks and takes their pages, then all blocks copy the table rows, a warp each.
__global__ void __cluster_dims__(kPlanCluster, 1, 1) __launch_bounds__(kPlanThreads)
kv_fork_kernel(PoolView p, const int32_t* parents, const int32_t* children, int n, int32_t* src, int32_t* dst, unsigned* err) {
  pdl_entry();
  extern __shared__ int sh[];
  int* need = sh;                  // [n]
  int* length = sh + n;            // [n] the parent's length; -1: nothing to do
  __shared__ int buf[33], bad;
  cg::cluster_group cluster = cg::this_cluster();
  if (cluster.block_rank() == 0) {
    if (threadIdx.x == 0) bad = 0;
    __syncthreads();
    for (int f = threadIdx.x; f < n; f += kPlanThreads) {
      const int from = parents[f], to = children[f];
      need[f] = 0;
      length[f] = -1;
      src[f] = -1;
      dst[f] = -1;
      if (to >= p.max_seqs || (to >= 0 && (from < 0 || from >= p.max_seqs))) { bad = 1; continue; }
      if (to < 0) continue;
      // a child holds nothing and no other entry has claimed it
      if (atomicCAS(reinterpret_cast<unsigned*>(p.len) + to, 0u, kMark) != 0u) { bad = 1; continue; }
      const int len = (int)((unsigned)p.len[from] & ~kMark);
      if (len > (int64_t)p.max_pages * p.page) { bad = 1; length[f] = 0; continue; }
      length[f] = len;
      need[f] = len % p.page != 0;
    }
    __syncthreads();
    const int total = scan_needs(need, n, buf);
    bool ok = bad == 0;
    if (ok)
      ok = take_pages(p, total, buf, [&](int rank, int page) {
        const int f = owner_of(need, n, rank), full = length[f] / p.page;
        src[f] = p.table[(int64_t)parents[f] * p.max_pages + full];
        dst[f] = page;
        p.table[(int64_t)children[f] * p.max_pages + full] = page;
        p.refs[page] = 1;
      });
    if (threadIdx.x == 0) {
      bad = !ok;
      if (!ok) atomicOr(err, ERR_PAGE);
    }
  }
  cluster.sync();
  const int failed = *cluster.map_shared_rank(&bad, 0);
  const int* lengths = cluster.map_shared_rank(length, 0);
  const int lane = threadIdx.x & 31;
  // claims were made on lengths of 0; a failed entry that claimed nothing has length -1 and is not touched
  for (int f = cluster.block_rank() * (kPlanThreads / 32) + (threadIdx.x >> 5); f < n; f += kPlanCluster * (kPlanThreads / 32)) {
    const int len = lengths[f];
    if (len < 0) continue;
    const int32_t* from = p.table + (int64_t)parents[f] * p.max_pages;
    int32_t* to = p.table + (int64_t)children[f] * p.max_pages;
    if (!failed)
      for (int j = lane; j < len / p.page; j += 32) {
        const int page = from[j];
        to[j] = page;
        if (page >= 0 && page < p.n_pages) atomicAdd(p.refs + page, 1);
        else atomicOr(err, ERR_PAGE);
      }
    if (lane == 0) {
      p.len[children[f]] = failed ? 0 : len;
      if (p.refused && !failed) p.refused[children[f]] = 0;
    }
  }
  cluster.sync();                  // the first block's shared memory has been read
}

// Live pages move down.  One cluster; block r walks the slice [r * slice, ...) of the counts.
__global__ void __cluster_dims__(kPlanCluster, 1, 1) __launch_bounds__(kPlanThreads)
kv_compact_kernel(PoolView p, int32_t* map, unsigned* err) {
  pdl_entry();
  int32_t* hole_list = map + p.n_pages;
  __shared__ int buf[33], live_here, counts[2];
  cg::cluster_group cluster = cg::this_cluster();
  const int rank = cluster.block_rank();
  const int slice = (p.n_pages + kPlanCluster - 1) / kPlanCluster;
  const int lo = min(rank * slice, p.n_pages), hi = min(lo + slice, p.n_pages);
  int sum = 0, total;
  for (int i = lo + threadIdx.x; i < hi; i += kPlanThreads) sum += p.refs[i] > 0;
  block_scan(sum, buf, total);
  if (threadIdx.x == 0) live_here = total;
  cluster.sync();
  int live = 0;
  for (int r = 0; r < kPlanCluster; ++r) live += *cluster.map_shared_rank(&live_here, r);
  // holes below `live` and movers at or above it, per slice and before this one
  int holes = 0, movers = 0, n_holes, n_movers;
  for (int i = lo + threadIdx.x; i < hi; i += kPlanThreads) {
    const bool used = p.refs[i] > 0;
    holes += !used && i < live;
    movers += used && i >= live;
  }
  block_scan(holes, buf, n_holes);
  block_scan(movers, buf, n_movers);
  if (threadIdx.x == 0) { counts[0] = n_holes; counts[1] = n_movers; }
  cluster.sync();
  int hole_at = 0, mover_at = 0;
  for (int r = 0; r < rank; ++r) {
    const int* c = cluster.map_shared_rank(counts, r);
    hole_at += c[0];
    mover_at += c[1];
  }
  // the holes in order
  for (int i0 = lo; i0 < hi; i0 += kPlanThreads) {
    const int i = i0 + threadIdx.x;
    const bool hole = i < hi && i < live && p.refs[i] <= 0;
    const int r = hole_at + block_scan(hole, buf, total);
    if (hole) hole_list[r] = i;
    if (i < hi && i < live) map[i] = hole ? -1 : i;
    hole_at += total;
  }
  cluster.sync();
  // movers take them in order, and counts follow (nobody reads a count below `live` any more)
  for (int i0 = lo; i0 < hi; i0 += kPlanThreads) {
    const int i = i0 + threadIdx.x;
    const int refs = i < hi && i >= live ? p.refs[i] : 0;
    const int r = mover_at + block_scan(refs > 0, buf, total);
    if (refs > 0) {
      const int to = hole_list[r];
      map[i] = to;
      p.refs[to] = refs;
      p.refs[i] = 0;
    } else if (i < hi && i >= live) {
      map[i] = -1;
    }
    mover_at += total;
  }
  cluster.sync();
  // table rows, a warp each
  const int lane = threadIdx.x & 31;
  for (int s = rank * (kPlanThreads / 32) + (threadIdx.x >> 5); s < p.max_seqs; s += kPlanCluster * (kPlanThreads / 32)) {
    int32_t* row = p.table + (int64_t)s * p.max_pages;
    const int pages = min(pages_for(max(p.len[s], 0), p.page), p.max_pages);
    for (int j = lane; j < pages; j += 32) {
      const int page = row[j];
      if (page < live) {
        if (page < 0) atomicOr(err, ERR_PAGE);
        continue;
      }
      if (page >= p.n_pages) { atomicOr(err, ERR_PAGE); continue; }
      row[j] = map[page];
    }
  }
}

// Page copies: a block moves up to 16 KB of one page's codes, the first block of a page its maxima too.  HBM bounds it: the 136 MB
// that a compaction moves (half of 96 sequences of up to 2600 tokens live, 8 heads of 128) take 22 us, 6.3 TB/s.
constexpr int kCopyThreads = 256;
constexpr int kCopyBytes = 16384;
__global__ void __launch_bounds__(kCopyThreads) kv_copy_kernel(CacheView c, int n_pages, int64_t page_bytes, const int32_t* src,
                                                               const int32_t* dst, unsigned* err) {
  pdl_entry();
  const int i = blockIdx.x;
  const int to = dst[i], from = src ? src[i] : i;
  if (to < 0 || from < 0 || to == from) return;
  if (to >= n_pages || from >= n_pages) {
    if (threadIdx.x == 0) atomicOr(err, ERR_PAGE);
    return;
  }
  const int64_t at = (int64_t)blockIdx.y * kCopyBytes;
  const int64_t end = min(at + kCopyBytes, page_bytes);
  int8_t* base = blockIdx.z ? c.v : c.k;
  const uint4* s = reinterpret_cast<const uint4*>(base + from * page_bytes);
  uint4* d = reinterpret_cast<uint4*>(base + to * page_bytes);
  uint4 v[4];
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const int64_t o = at / 16 + threadIdx.x + j * kCopyThreads;
    if (o * 16 < end) v[j] = s[o];
  }
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    const int64_t o = at / 16 + threadIdx.x + j * kCopyThreads;
    if (o * 16 < end) d[o] = v[j];
  }
  if (blockIdx.y == 0) {
    float* a = blockIdx.z ? c.v_absmax : c.k_absmax;
    for (int h = threadIdx.x; h < c.heads; h += kCopyThreads) a[(int64_t)to * c.heads + h] = a[(int64_t)from * c.heads + h];
  }
}

// What a block of a ragged batch works on.  Entry i owns the items starts[i] / unit + 2 i, ...; a thread looks at an entry, so that
// everything that has to be known of the block's own is fetched at once.
struct Claim {
  int64_t row0;
  int entry, rows, nth, seq, len, twice, refused;
};
// twice: whether the sequence is listed by another entry too, refused: whether it got no room (both only where asked for).
// Whole block; false: nothing to do.
__device__ __forceinline__ bool claim_item(const PoolView& p, const BatchView& b, int64_t item, int unit, bool want_twice, Claim* c, unsigned* err) {
  if (threadIdx.x == 0) { c->entry = -1; c->twice = 0; }
  __syncthreads();
  for (int i0 = 0; i0 < b.n; i0 += blockDim.x) {
    const int i = i0 + threadIdx.x;
    if (i >= b.n) break;
    int64_t lo, hi;
    if (!entry_rows(b, i, lo, hi)) atomicOr(err, ERR_PAGE);
    const int64_t first = b.starts ? (int64_t)b.starts[i] / unit + 2 * (int64_t)i : i;
    const int64_t nth = item - first;
    const int s = b.seqs[i];
    const bool known = s >= 0 && s < p.max_seqs;
    const int len = known ? seq_len(p, s) : 0, refused = want_twice && known && p.refused ? p.refused[s] : 0;
    // the bound of a run of items: those of the next entry begin behind rows / unit + 2 of this one's
    if (nth >= 0 && nth < (b.starts ? (hi - lo) / unit + 2 : 1) && hi > lo && atomicCAS(&c->entry, -1, i) == -1) {
      c->row0 = lo;
      c->rows = (int)(hi - lo);
      c->nth = (int)nth;
      c->seq = s;
      c->len = len;
      c->refused = refused;
    }
  }
  __syncthreads();
  if (c->entry < 0) return false;
  if (c->seq >= p.max_seqs && threadIdx.x == 0) atomicOr(err, ERR_PAGE);
  if (want_twice) {
    for (int i = threadIdx.x; i < b.n; i += blockDim.x)
      if (i != c->entry && b.seqs[i] == c->seq) c->twice = 1;
    __syncthreads();
  }
  return true;
}

// New keys and values of a run of pages: a block takes 8 / W heads, W warps a head (1, 2, 4 or 8: as many as it takes to keep a page of
// a head in registers, kAppendHeld pieces of 16 bytes a lane, so that it is read once; what does not fit is read twice).  To find a
// page takes five loads one behind the other, longer than to write it: a block writes both tensors and, of 16 tokens, two pages.
// Divisions for each piece bounded it before; now those loads and HBM do.  8 prompts of up to 2000 fp32 tokens into pages of 16, 8 heads
// of 128, written and read back: 94 -> 74 us (3.4 TB/s, 51% of the measured copy rate; 40 of them to write); 64 single tokens 7.9 us.
constexpr int kAppendThreads = 256, kAppendHeld = 8;
template <typename T, int W>
__global__ void __launch_bounds__(kAppendThreads, 3) kv_append_kernel(PoolView p, CacheView c, BatchView b, const T* k, const T* v, int64_t row_stride,
                                                                      int64_t head_stride, int run, unsigned* err) {
  pdl_entry();
  constexpr int V = Vec<T>::N, N = 32 * W;
  __shared__ Claim own;
  __shared__ unsigned tops[8];
  if (!claim_item(p, b, blockIdx.x, run * p.page, true, &own, err)) return;
  const int s = own.seq, len = own.len;
  if (s < 0 || s >= p.max_seqs) return;
  const int64_t old = (int64_t)len - own.rows;     // tokens before this call
  if (old < 0 || own.twice || own.refused) {
    if (threadIdx.x == 0) atomicOr(err, ERR_PAGE);
    return;
  }
  const int warp = threadIdx.x >> 5, h = blockIdx.y * (8 / W) + warp / W, t = threadIdx.x & (N - 1);
  const bool here = h < c.heads;                   // (W > 1: a block's warps meet)
  if (W == 1 && !here) return;
  const int per_row = c.dim / V;
  // the own.nth run of pages, counted from the one the first new token lies in
  const int64_t j_first = (old / (run * p.page) + own.nth) * run;
  for (int64_t j = max(j_first, old / p.page); j < j_first + run && j * p.page < len; ++j) {
    const int number = p.table[(int64_t)s * p.max_pages + j];
    if (number < 0 || number >= p.n_pages || p.refs[number] != 1) {
      if (threadIdx.x == 0) atomicOr(err, ERR_PAGE);
      continue;
    }
    const int64_t block = (int64_t)number * c.heads + (here ? h : 0);
    const int t0 = (int)(max(old, j * p.page) - j * p.page);           // new tokens of the page: [t0, t1)
    const int t1 = (int)(min((int64_t)len, (j + 1) * p.page) - j * p.page);
    const int n_vec = here ? (t1 - t0) * per_row : 0;
    const int z_last = gridDim.z == 2 ? blockIdx.z : 1;
#pragma unroll 1
    for (int z = gridDim.z == 2 ? blockIdx.z : 0; z <= z_last; ++z) {
      int8_t* codes = (z ? c.v : c.k) + block * p.page * c.dim;
      float* absmax = (z ? c.v_absmax : c.k_absmax) + block;
      const T* x = (z ? v : k) + (own.row0 + j * p.page + t0 - old) * row_stride + h * head_stride;
      const float before = t0 > 0 && here ? *absmax : 0.0f;
      union Piece { uint4 u; T t[V]; } held[kAppendHeld];
      // piece t + i N of the page's new tokens, i ascending: a division once, then steps
      const int row_step = N / per_row, col_step = N - row_step * per_row;
      int row = t / per_row, col = t - row * per_row;
      const int row_first = row, col_first = col;
      auto next = [&]() {
        const T* from = x + row * row_stride + col * V;
        row += row_step;
        col += col_step;
        if (col >= per_row) { col -= per_row; ++row; }
        return from;
      };
      unsigned top = 0;
      auto see = [&](const Piece& f) {                 // a NaN or Inf orders above all others
#pragma unroll
        for (int q = 0; q < V; ++q) {
          const unsigned a = abs_bits(to_float<T>(f.t[q]));
          top = a > top ? a : top;
        }
      };
#pragma unroll
      for (int i = 0; i < kAppendHeld; ++i)
        if (t + i * N < n_vec) held[i].u = __ldg(reinterpret_cast<const uint4*>(next()));
#pragma unroll
      for (int i = 0; i < kAppendHeld; ++i)
        if (t + i * N < n_vec) see(held[i]);
      Piece f;
      const int row_held = row, col_held = col;          // of the first piece not held
      for (int e = t + kAppendHeld * N; e < n_vec; e += N) {
        f.u = __ldg(reinterpret_cast<const uint4*>(next()));
        see(f);
      }
      auto over_head = [&](unsigned m) {
        m = __reduce_max_sync(0xffffffffu, m);
        if (W > 1) {
          __syncthreads();
          if ((threadIdx.x & 31) == 0) tops[warp] = m;
          __syncthreads();
#pragma unroll
          for (int w = 0; w < W; ++w) m = max(m, tops[warp / W * W + w]);
        }
        return m;
      };
      top = over_head(top);
      const bool odd = top >= 0x7f800000u;
      if (W > 1 ? __syncthreads_or(odd) : odd) {       // the largest of the others
        if (odd && t == 0) atomicOr(err, ERR_NONFINITE);
        unsigned other = 0;
        row = row_first;
        col = col_first;
        for (int e = t; e < n_vec; e += N) {
          f.u = __ldg(reinterpret_cast<const uint4*>(next()));
#pragma unroll
          for (int q = 0; q < V; ++q) {
            const unsigned a = abs_bits(to_float<T>(f.t[q]));
            if (a < 0x7f800000u && a > other) other = a;
          }
        }
        top = over_head(other);
      }
      if (!here) continue;
      const float fresh = __uint_as_float(top), now = before > fresh ? before : fresh;
      const float inv = inv_scale_of(now);
      const bool plain = !odd && finite_bits(inv);
      auto put = [&](int e, const Piece& f) {
        union { uint32_t w[V / 4]; int8_t b[V]; } q;
        if (plain) {
#pragma unroll
          for (int g = 0; g < V / 4; ++g) {
            uint32_t w[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {              // clamp, then round by a magic number: the low byte is the code
              float y;
              asm("min.xorsign.abs.f32 %0, %1, %2;" : "=f"(y) : "f"(__fmul_rn(to_float<T>(f.t[4 * g + i]), inv)), "f"(kQmax8));
              w[i] = __float_as_uint(__fadd_rn(y, 12582912.0f));
            }
            q.w[g] = __byte_perm(__byte_perm(w[0], w[1], 0x0040), __byte_perm(w[2], w[3], 0x0040), 0x5410);
          }
        } else {
#pragma unroll
          for (int g = 0; g < V; ++g) {
            const float y = to_float<T>(f.t[g]);
            q.b[g] = (int8_t)(finite_bits(y) ? code_of(y, inv) : 0);
          }
        }
        uint32_t* to = reinterpret_cast<uint32_t*>(codes + t0 * c.dim + e * V);
        if (V == 8) *reinterpret_cast<uint2*>(to) = make_uint2(q.w[0], q.w[V / 4 - 1]);
        else to[0] = q.w[0];
      };
#pragma unroll
      for (int i = 0; i < kAppendHeld; ++i)
        if (t + i * N < n_vec) put(t + i * N, held[i]);
      row = row_held;
      col = col_held;
      for (int e = t + kAppendHeld * N; e < n_vec; e += N) {
        f.u = __ldg(reinterpret_cast<const uint4*>(next()));
        put(e, f);
      }
      if (t0 > 0 && now > before && before > 0.0f) {   // the earlier codes on the new grid
        const float ratio = __fdiv_rn(before, now);
        for (int e = t; e < t0 * c.dim / 4; e += N) {
          char4* to = reinterpret_cast<char4*>(codes) + e;
          const char4 q = *to;
          *to = make_char4((signed char)__float2int_rn(q.x * ratio), (signed char)__float2int_rn(q.y * ratio),
                           (signed char)__float2int_rn(q.z * ratio), (signed char)__float2int_rn(q.w * ratio));
        }
      }
      if (t == 0) *absmax = now;
    }
  }
}

// Values of cached tokens: a block takes 4 tokens (of one page, as positions count), a warp a row of keys or of values, written whole.
// Small blocks: what bounds a block is the four loads one behind the other that lead to its codes, so many of them have to be under way
// (the prompts above: 32 us).
constexpr int kReadTokens = 4, kReadThreads = 64 * kReadTokens;
template <typename T>
__global__ void __launch_bounds__(kReadThreads, 5) kv_read_kernel(PoolView p, CacheView c, BatchView b, const int32_t* first_tok, T* k, T* v, unsigned* err) {
  pdl_entry();
  __shared__ Claim own;
  if (!claim_item(p, b, blockIdx.x, kReadTokens, false, &own, err)) return;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, z = warp & 1;
  const int64_t from = first_tok[own.entry];
  // positions of this block: the own.nth run of 4 from the one `from` lies in (floor, for negative ones too)
  const int64_t run = (from >= 0 ? from / kReadTokens : -((-from + kReadTokens - 1) / kReadTokens)) + own.nth;
  const int64_t pos = run * kReadTokens + (warp >> 1);
  T* out = z ? v : k;
  if (!out || pos < from || pos >= from + own.rows) return;
  out += (own.row0 + pos - from) * c.heads * c.dim;
  int number = -1;
  if (own.seq >= 0 && own.seq < p.max_seqs && pos >= 0 && pos < own.len) {
    number = p.table[(int64_t)own.seq * p.max_pages + pos / p.page];
    if (number < 0 || number >= p.n_pages) {
      if (lane == 0) atomicOr(err, ERR_PAGE);
      number = -1;
    }
  }
  const int quads = c.dim / 4, head_bytes = p.page * c.dim;
  const int step_h = 32 / quads, step_d = 4 * (32 - step_h * quads);
  const int64_t block = (int64_t)max(number, 0) * c.heads;
  const int8_t* codes = (z ? c.v : c.k) + (block * p.page + (number < 0 ? 0 : pos % p.page)) * c.dim;
  const float* absmax = (z ? c.v_absmax : c.k_absmax) + block;
  // 32 heads at a time: lane i holds the scale of the i-th, element lane + 32 e of [heads][quads] is the lane's e-th
  for (int h0 = 0; h0 < c.heads; h0 += 32) {
    const int nh = min(32, c.heads - h0), n = nh * quads;
    const float mine = number < 0 ? 0.0f : lane < nh ? scale_of(absmax[h0 + lane]) : 1.0f;
    int h = lane / quads, d = 4 * (lane - h * quads);
    T* to = out + h0 * c.dim + 4 * lane;
    constexpr int kBatch = 8;
    for (int e0 = 0; e0 < n; e0 += 32 * kBatch, to += 128 * kBatch) {
      char4 q[kBatch];
      float f[kBatch];
#pragma unroll
      for (int i = 0; i < kBatch; ++i) {
        q[i] = make_char4(0, 0, 0, 0);
        if (number >= 0 && e0 + 32 * i + lane < n) q[i] = *reinterpret_cast<const char4*>(codes + (int64_t)(h0 + h) * head_bytes + d);
        f[i] = __shfl_sync(0xffffffffu, mine, h & 31);
        h += step_h;
        d += step_d;
        if (d >= c.dim) { d -= c.dim; ++h; }
      }
#pragma unroll
      for (int i = 0; i < kBatch; ++i) {
        if (e0 + 32 * i + lane >= n) continue;
        union { T t[4]; uint4 w4; uint2 w2; } o;
        o.t[0] = from_float<T>(q[i].x * f[i]);
        o.t[1] = from_float<T>(q[i].y * f[i]);
        o.t[2] = from_float<T>(q[i].z * f[i]);
        o.t[3] = from_float<T>(q[i].w * f[i]);
        if (sizeof(T) == 4) *reinterpret_cast<uint4*>(to + 128 * i) = o.w4;
        else *reinterpret_cast<uint2*>(to + 128 * i) = o.w2;
      }
    }
  }
}

// A pool whose sequences all have the same length: sequence i holds the pages i * max_pages and on.
__global__ void __launch_bounds__(256) kv_layout_kernel(PoolView p, int32_t* seqs, int32_t* starts, int seq_len, int64_t rows) {
  pdl_entry();
  const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (i <= p.max_seqs) {
    const int64_t lo = min(i * seq_len, rows);
    starts[i] = (int32_t)lo;
    if (i < p.max_seqs) {
      seqs[i] = (int32_t)i;
      p.len[i] = (int32_t)min((int64_t)seq_len, rows - lo);
    }
  }
  if (i < p.n_pages) {
    const int64_t lo = i / p.max_pages * seq_len + i % p.max_pages * p.page;      // its first token's row
    const bool held = lo < rows;
    p.table[i] = held ? (int32_t)i : -1;
    p.refs[i] = held ? 1 : 0;
  }
}

}  // namespace

int launch_kv_layout(Ctx* ctx, const PoolView& p, int32_t* seqs, int32_t* starts, int seq_len, int64_t rows, cudaStream_t st) {
  launch_pdl(kv_layout_kernel, dim3((unsigned)((std::max(p.n_pages, p.max_seqs + 1) + 255) / 256)), dim3(256), 0, st, p, seqs, starts, seq_len, rows);
  count_launch(ctx);
  return check_cuda(ctx, cudaGetLastError(), "kv_layout");
}
int launch_kv_extend(Ctx* ctx, const PoolView& p, const BatchView& b, cudaStream_t st) {
  if (b.n == 0) return QCFG_OK;
  const size_t smem = (size_t)b.n * 8;
  if (smem > 40000) {
    const cudaError_t e = cudaFuncSetAttribute(kv_extend_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kPlanMost * 8);
    if (e != cudaSuccess) return check_cuda(ctx, e, "kv_extend");
  }
  launch_pdl(kv_extend_kernel, dim3(1), dim3(kPlanThreads), smem, st, p, b, err_word(ctx));
  count_launch(ctx);
  return check_cuda(ctx, cudaGetLastError(), "kv_extend");
}
int launch_kv_free(Ctx* ctx, const PoolView& p, const int32_t* seqs, int n, cudaStream_t st) {
  if (n == 0) return QCFG_OK;
  launch_pdl(kv_free_kernel, dim3(n), dim3(128), 0, st, p, seqs, err_word(ctx));
  count_launch(ctx);
  return check_cuda(ctx, cudaGetLastError(), "kv_free");
}
int launch_kv_fork(Ctx* ctx, const PoolView& p, const int32_t* parents, const int32_t* children, int n, int32_t* src, int32_t* dst, cudaStream_t st) {
  if (n == 0) return QCFG_OK;
  const size_t smem = (size_t)n * 8;
  if (smem > 40000) {
    const cudaError_t e = cudaFuncSetAttribute(kv_fork_kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kPlanMost * 8);
    if (e != cudaSuccess) return check_cuda(ctx, e, "kv_fork");
  }
  launch_pdl(kv_fork_kernel, dim3(kPlanCluster), dim3(kPlanThreads), smem, st, p, parents, children, n, src, dst, err_word(ctx));
  count_launch(ctx);
  return check_cuda(ctx, cudaGetLastError(), "kv_fork");
}
int launch_kv_compact(Ctx* ctx, const PoolView& p, int32_t* map, cudaStream_t st) {
  if (p.n_pages == 0) return QCFG_OK;
  launch_pdl(kv_compact_kernel, dim3(kPlanCluster), dim3(kPlanThreads), 0, st, p, map, err_word(ctx));
  count_launch(ctx);
  return check_cuda(ctx, cudaGetLastError(), "kv_compact");
}
int launch_kv_copy(Ctx* ctx, const PoolView& p, const CacheView& c, const int32_t* src, const int32_t* dst, int n, cudaStream_t st) {
  if (n == 0) return QCFG_OK;
  const int64_t bytes = (int64_t)c.heads * p.page * c.dim;
  const dim3 grid(n, (unsigned)((bytes + kCopyBytes - 1) / kCopyBytes), 2);
  launch_pdl(kv_copy_kernel, grid, dim3(kCopyThreads), 0, st, c, p.n_pages, bytes, src, dst, err_word(ctx));
  count_launch(ctx);
  return check_cuda(ctx, cudaGetLastError(), "kv_copy_pages");
}
template <typename T>
static void append_as(Ctx* ctx, const PoolView& p, const CacheView& c, const BatchView& b, const void* k, const void* v, int64_t row_stride,
                      int64_t head_stride, cudaStream_t st) {
  // a row each: one page of an entry, few bytes of it, and both tensors at once; else runs of 32 tokens or a page
  const bool single = b.rows <= b.n;
  const int run = single || p.page > 16 ? 1 : 2;
  const int64_t items = b.starts ? b.rows / (run * p.page) + 2 * (int64_t)b.n : b.n;
  const int64_t pieces = (single ? 1 : p.page) * c.dim / Vec<T>::N, warps = (pieces + 32 * kAppendHeld - 1) / (32 * kAppendHeld);
  const auto go = [&](auto kernel, int w) {
    launch_pdl(kernel, dim3((unsigned)items, (c.heads * w + 7) / 8, single ? 2 : 1), dim3(kAppendThreads), 0, st, p, c, b, (const T*)k, (const T*)v, row_stride,
               head_stride, run, err_word(ctx));
  };
  if (warps <= 1) go(kv_append_kernel<T, 1>, 1);
  else if (warps <= 2) go(kv_append_kernel<T, 2>, 2);
  else if (warps <= 4) go(kv_append_kernel<T, 4>, 4);
  else go(kv_append_kernel<T, 8>, 8);
}
int launch_kv_append(Ctx* ctx, const PoolView& p, const CacheView& c, const BatchView& b, const void* k, const void* v, int dtype,
                     int64_t row_stride, int64_t head_stride, cudaStream_t st) {
  if (b.n == 0 || b.rows == 0) return QCFG_OK;
  if (dtype == QCFG_FP32) append_as<float>(ctx, p, c, b, k, v, row_stride, head_stride, st);
  else if (dtype == QCFG_BF16) append_as<__nv_bfloat16>(ctx, p, c, b, k, v, row_stride, head_stride, st);
  else append_as<__half>(ctx, p, c, b, k, v, row_stride, head_stride, st);
  count_launch(ctx);
  return check_cuda(ctx, cudaGetLastError(), "kv_append");
}
template <typename T>
static void read_as(Ctx* ctx, const PoolView& p, const CacheView& c, const BatchView& b, const int32_t* first, void* k, void* v, cudaStream_t st) {
  launch_pdl(kv_read_kernel<T>, dim3((unsigned)(b.starts ? b.rows / kReadTokens + 2 * (int64_t)b.n : b.n)), dim3(kReadThreads), 0, st, p, c, b, first, (T*)k, (T*)v,
             err_word(ctx));
}
int launch_kv_read(Ctx* ctx, const PoolView& p, const CacheView& c, const BatchView& b, const int32_t* first, void* k, void* v, int dtype,
                   cudaStream_t st) {
  if (b.n == 0 || b.rows == 0) return QCFG_OK;
  if (dtype == QCFG_FP32) read_as<float>(ctx, p, c, b, first, k, v, st);
  else if (dtype == QCFG_BF16) read_as<__nv_bfloat16>(ctx, p, c, b, first, k, v, st);
  else read_as<__half>(ctx, p, c, b, first, k, v, st);
  count_launch(ctx);
  return check_cuda(ctx, cudaGetLastError(), "kv_read");
}

}  // namespace qcfg
