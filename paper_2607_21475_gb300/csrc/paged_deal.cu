// Pages dealt to the sequences of a step from their lengths, and the maps of the step's
// tokens: block tables, packed offsets, positions and slots.
//
// With P positions to a page, a sequence of `len` cached tokens holds the blocks
// [lo, hi) of its row; n new tokens need ceil((len + n) / P) - hi pages more, and with a
// window w the blocks below floor((len - w + 1) / P) are of no use to them.  All that is a
// prefix sum over the sequences (pages given back, pages wanted, tokens; then of those that
// are served) and copies whose places it tells.  Nothing of this is much work; what bounds
// it is the chain of dependent steps: lengths -> sums -> pages -> slots, in one launch of
// one cluster.
//
// Up to kDealSeqs sequences every CTA sums over all of them and keeps the sums in shared
// memory.  Each page, given back or taken, and each token is then a number whose sequence
// a thread finds by bisection, so that a long prompt's pages spread over all threads, and
// nothing waits for what another thread writes: a page taken is read where it lay, in
// the list or, if it is given back by this very call, in its old owner's row.  Only the
// outputs that may be inputs wait (one cluster barrier) until every CTA has read them.
// More sequences than that: a thread per few sequences, sums exchanged through distributed
// shared memory, a warp per sequence's pages.  The results are the same.
// Measured: 256 steps, of which 5 leave (2000 pages given back) 4.2 us; 64 requests, 103k
// tokens of prompts among them, 7.4 us; a launch and the chain of loads take 3.  A
// programmatic dependent of what precedes it on the stream.
#include <cuda_runtime.h>

#include "common.cuh"
#include "decode_tile.cuh"
#include "internal.h"
#include "paged.cuh"
#include "ptx.cuh"

namespace ebd {

constexpr int kDealThreads = 1024;
// Threads where they are one per sequence and, over 8 CTAs, one per token: their barriers and
// sums are the cheaper (one sequence 2.5 us against 2.9 with 1024, 256 3.0 / 3.4, 384 3.1 / 3.6, 512
// 3.45 / 3.55).
constexpr int kDealFewThreads = 512;
// CTAs of a cluster: 8, 16 where many tokens are to be mapped (256 steps, 2000 pages given
// back: 1 CTA 7.0 us, 2 6.0, 4 5.3, 8 4.4; 100k tokens of prompts: 4 12.0 us, 8 8.5, 16 7.5)
constexpr int kDealCluster = 8, kDealLargeCluster = 16;
constexpr int kDealSeqs = 4096;       // sequences whose sums every CTA keeps
constexpr int kDealOffsets = 8192;    // packed offsets kept in shared memory (many sequences)

struct DealArgs {
  int batch, page_shift, n_pages, max_blocks, n_tokens, window;
  const int32_t *n_new, *seq_len, *held, *n_free;
  int32_t *free_pages, *block_table;
  int32_t *seq_len_out, *held_out, *n_free_out, *cu_new, *served, *positions;
  int64_t* slots;
  int32_t* dev_status;
};

// What one sequence asks for.
struct Ask {
  int n, len, lo, hi;
  int keep;         // first block kept
  long long pages;  // wanted
  long long some;   // tokens
  bool fits;        // its row has room for it
};

__device__ __forceinline__ Ask deal_ask(const DealArgs& a, int b, bool& bad) {
  Ask k;
  k.n = a.n_new[b];
  const int len = a.seq_len[b], lo = a.held[2 * b], hi = a.held[2 * b + 1];
  k.len = max(len, 0);
  k.hi = min(max(hi, 0), a.max_blocks);
  k.lo = min(max(lo, 0), k.hi);
  bad |= k.len != len || k.hi != hi || k.lo != lo;
  k.keep = k.lo;
  k.pages = k.some = 0;
  k.fits = true;
  if (k.n < 0) {  // leaves
    k.keep = k.hi;
    return k;
  }
  if (a.window > 0) {
    const long long first = (long long)k.len - a.window + 1;
    if (first > 0) k.keep = min(max(k.lo, (int)(first >> a.page_shift)), k.hi);
  }
  if (k.n > 0) {
    const long long P = 1ll << a.page_shift;
    const long long after = ((long long)k.len + k.n + P - 1) >> a.page_shift;
    k.fits = after <= a.max_blocks;
    if (k.fits) {
      k.pages = after > k.hi ? after - k.hi : 0;
      k.some = k.n;
    }
  }
  return k;
}

// The place of a number in sums[0 .. n] (not falling, sums[0] = 0): the i with
// sums[i] <= x < sums[i + 1].
__device__ __forceinline__ int place_in(const int* sums, int n, int x) {
  int i = 0, end = n - 1;
  while (i < end) {
    const int mid = (i + end) >> 1;
    if (sums[mid + 1] > x) end = mid;
    else i = mid + 1;
  }
  return i;
}

// Three sums that stop at a bound each (below 2^31): what matters of a larger one is that
// it is larger, and sums that stop can be formed in any order.
struct Three {
  uint32_t v[3];
};
__device__ __forceinline__ Three add_up_to(Three a, const Three& b, const Three& most) {
#pragma unroll
  for (int i = 0; i < 3; ++i) a.v[i] = min(a.v[i] + b.v[i], most.v[i]);
  return a;
}
// (not unrolled: the code runs once a call, and fetching it would take longer than that)
__device__ __forceinline__ Three warp_sums_up_to(Three x, const Three& most) {
  const int lane = threadIdx.x & 31;
#pragma unroll 1
  for (int o = 1; o < 32; o <<= 1) {
    Three u;
#pragma unroll
    for (int i = 0; i < 3; ++i) u.v[i] = __shfl_up_sync(0xffffffffu, x.v[i], o);
    if (lane >= o) x = add_up_to(x, u, most);
  }
  return x;
}
// Sums of x over the block's threads before this one; total: over all.
__device__ __forceinline__ Three block_sums_up_to(const Three& x, const Three& most, Three& total,
                                                  Three* warp_s) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, warps = blockDim.x >> 5;
  const Three up = warp_sums_up_to(x, most);
  if (lane == 31) warp_s[warp] = up;
  __syncthreads();
  // every warp sums the warps' sums itself
  const Three all = warp_sums_up_to(lane < warps ? warp_s[lane] : Three{{0, 0, 0}}, most);
  Three before;
#pragma unroll
  for (int i = 0; i < 3; ++i) {
    total.v[i] = __shfl_sync(0xffffffffu, all.v[i], 31);
    const uint32_t w = __shfl_sync(0xffffffffu, all.v[i], warp > 0 ? warp - 1 : 0);
    const uint32_t l = __shfl_up_sync(0xffffffffu, up.v[i], 1);
    before.v[i] = min((warp > 0 ? w : 0u) + (lane > 0 ? l : 0u), most.v[i]);
  }
  return before;
}

// What the CTAs keep of every sequence: sums before it (of pages given back, pages taken,
// packed tokens, runs of them that share a page), its length, its first and end block.
struct DealSums {
  int *back, *take, *cu, *run, *len, *lo, *hi;
  __device__ __forceinline__ DealSums(int* p, int batch)
      : back(p), take(p + batch + 1), cu(p + 2 * (batch + 1)), run(p + 3 * (batch + 1)),
        len(p + 4 * (batch + 1)), lo(p + 5 * (batch + 1)), hi(p + 6 * (batch + 1)) {}
  static size_t bytes(int batch) { return 7 * ((size_t)batch + 1) * 4; }
};

// PER: sequences of a thread, at most.  RUNS: tokens are mapped by runs that share a page
// (many tokens), else one by one, without the runs' sums.
template <int PER, bool RUNS>
__global__ void __launch_bounds__(kDealThreads, 1) paged_deal_kernel(const DealArgs a) {
  extern __shared__ int sums_s[];
  __shared__ Three warp_s[2][32];
  const uint32_t ranks = gridDim.x, rank = cluster_rank();
  // (neighbouring warps of the work in different CTAs)
  const int threads = blockDim.x * ranks;
  const int tid = ((threadIdx.x >> 5) * ranks + rank) * 32 + (threadIdx.x & 31);
  const DealSums of(sums_s, a.batch);
  grid_launch_dependents();
  grid_dependency_wait();
  const int b0 = min((int)threadIdx.x * PER, a.batch), mine = min(PER, a.batch - b0);
  bool bad = false, short_of = false;

  // given back, wanted, tokens: up to each of the thread's sequences and of it
  Ask ask[PER];
  const Three most = {{(uint32_t)a.n_pages + 1u, (uint32_t)a.n_pages + 1u, (uint32_t)a.n_tokens + 1u}};
  auto asked = [&](const Ask& k) {
    return Three{{(uint32_t)min(k.keep - k.lo, a.n_pages),
                  (uint32_t)min(k.pages, (long long)a.n_pages + 1),
                  (uint32_t)min(k.some, (long long)a.n_tokens + 1)}};
  };
  Three x = {{0, 0, 0}}, all;
#pragma unroll
  for (int i = 0; i < PER; ++i) {
    if (i >= mine) break;
    ask[i] = deal_ask(a, b0 + i, bad);
    x = add_up_to(x, asked(ask[i]), most);
  }
  const int had = a.n_free[0], n_free = min(max(had, 0), a.n_pages);
  bad |= had != n_free;
  __syncwarp();
  cluster_arrive_release();  // the inputs that may be outputs were read
  const Three before = block_sums_up_to(x, most, all, warp_s[0]);
  // the list cannot hold more than all pages: what a wrong table would add is lost
  const int n_back = min((int)all.v[0], a.n_pages - n_free), n_all = n_free + n_back;
  bad |= (int)all.v[0] > n_back;

  // who is served: a request for pages that are not there holds back the later ones that
  // need pages too
  Three upto = before, y = {{0, 0, 0}};
  uint32_t ok = 0;
  // of a served sequence: the runs of its tokens that share a page, its pages, its tokens
  const Three most_served = {{(uint32_t)a.n_tokens + 1u, most.v[1], most.v[2]}};
  auto served_sums = [&](const Ask& k) {
    Three r = asked(k);
    r.v[0] = RUNS && k.some > 0 ? (uint32_t)((k.len + (int)k.some - 1) >> a.page_shift) -
                                      (k.len >> a.page_shift) + 1
                                : 0;
    return r;
  };
#pragma unroll
  for (int i = 0; i < PER; ++i) {
    if (i >= mine) break;
    const Ask& k = ask[i];
    of.back[b0 + i] = min((int)upto.v[0], n_back);
    of.len[b0 + i] = k.len;
    of.lo[b0 + i] = k.lo;
    of.hi[b0 + i] = k.hi;
    upto = add_up_to(upto, asked(k), most);
    if (k.fits && (k.pages == 0 || (int)upto.v[1] <= n_all) &&
        (k.n <= 0 || upto.v[2] <= (uint32_t)a.n_tokens)) {
      ok |= 1u << i;
      y = add_up_to(y, served_sums(k), most_served);
    } else {
      short_of = true;
    }
  }
  Three got = all, taken = before;
  if (RUNS || (int)all.v[1] > n_all || all.v[2] > (uint32_t)a.n_tokens)  // (not all are served)
    taken = block_sums_up_to(y, most_served, got, warp_s[1]);
#pragma unroll
  for (int i = 0; i < PER; ++i) {
    if (i >= mine) break;
    of.take[b0 + i] = (int)taken.v[1];
    of.cu[b0 + i] = (int)taken.v[2];
    if (RUNS) of.run[b0 + i] = (int)taken.v[0];
    if (ok >> i & 1) taken = add_up_to(taken, served_sums(ask[i]), most_served);
  }
  const int n_take = (int)got.v[1], total = (int)got.v[2];
  if (threadIdx.x == 0) of.back[a.batch] = n_back, of.take[a.batch] = n_take, of.cu[a.batch] = total;
  if (threadIdx.x == 0 && RUNS) of.run[a.batch] = (int)got.v[0];
  __syncthreads();

  // Where the j-th page given back lies, and the j-th taken.  (Read by ordinary loads: the call
  // before this one may still be writing when this kernel begins.)
  auto given = [&](int j) {
    const int o = place_in(of.back, a.batch, j);
    return a.block_table + (size_t)o * a.max_blocks + of.lo[o] + (j - of.back[o]);
  };
  auto taken_at = [&](int j) {
    const int p = n_all - 1 - j;
    return p < n_free ? a.free_pages + p : given(p - n_free);
  };
  // The page of a block of sequence b.
  auto page_at = [&](int b, int block) {
    const int fresh = block - of.hi[b];
    return *(fresh < 0 ? a.block_table + (size_t)b * a.max_blocks + block
                       : taken_at(of.take[b] + fresh));
  };
  auto write = [&](int t, int pos, int page) {
    const bool in_pool = (unsigned)page < (unsigned)a.n_pages;
    bad |= !in_pool;
    if (a.positions) a.positions[t] = pos;
    if (a.slots)
      a.slots[t] =
          in_pool ? ((int64_t)page << a.page_shift) + (pos & ((1 << a.page_shift) - 1)) : -1;
  };
  const int n_tokens = a.positions || a.slots ? a.n_tokens : 0;
  // Tokens, or the runs of them that share a page, and pages given back and taken, one after
  // another.
  const int n_maps = n_tokens == 0 ? 0 : RUNS ? ((int)got.v[0] + 31) / 32 * 32 : total;
  for (long long w = tid; w < (long long)n_maps + n_back + n_take; w += threads) {
    if (w < n_maps && !RUNS) {
      const int t = (int)w, b = place_in(of.cu, a.batch, t), pos = of.len[b] + (t - of.cu[b]);
      write(t, pos, page_at(b, pos >> a.page_shift));
    } else if (w < n_maps) {  // 32 runs to a warp: a lane looks one up, all write its tokens
      const int lane = threadIdx.x & 31;
      int t = 0, pos = 0, n = 0, page = 0;
      if (w < (int)got.v[0]) {
        const int b = place_in(of.run, a.batch, (int)w), len = of.len[b];
        const int block = (len >> a.page_shift) + ((int)w - of.run[b]);
        pos = max(len, block << a.page_shift);
        n = min(len + of.cu[b + 1] - of.cu[b], (block + 1) << a.page_shift) - pos;
        t = of.cu[b] + pos - len;
        page = page_at(b, block);
      }
      if (__reduce_max_sync(0xffffffffu, n) <= 2) {
        for (int q = 0; q < n; ++q) write(t + q, pos + q, page);
      } else {
        for (int src = 0; src < 32; ++src) {
          const int m = __shfl_sync(0xffffffffu, n, src), t1 = __shfl_sync(0xffffffffu, t, src);
          const int pos1 = __shfl_sync(0xffffffffu, pos, src);
          const int page1 = __shfl_sync(0xffffffffu, page, src);
          for (int q = lane; q < m; q += 32) write(t1 + q, pos1 + q, page1);
        }
      }
    } else if (const int j = (int)(w - n_maps); j < n_back) {
      a.free_pages[n_free + j] = *given(j);
    } else {
      const int k = j - n_back, b = place_in(of.take, a.batch, k), page = *taken_at(k);
      bad |= (unsigned)page >= (unsigned)a.n_pages;
      a.block_table[(size_t)b * a.max_blocks + of.hi[b] + (k - of.take[b])] = page;
    }
  }
  for (int t = total + tid; t < n_tokens; t += threads) {
    if (a.positions) a.positions[t] = 0;
    if (a.slots) a.slots[t] = -1;
  }
  __syncwarp();
  cluster_wait_acquire();
  if (rank == 0) {
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      if (i >= mine) break;
      const int b = b0 + i;
      const Ask& k = ask[i];
      const bool served = ok >> i & 1, leaves = k.n < 0;
      a.seq_len_out[b] = leaves ? 0 : served ? k.len + (int)k.some : k.len;
      a.held_out[2 * b] = leaves ? 0 : k.keep;
      a.held_out[2 * b + 1] = leaves ? 0 : served ? k.hi + (int)k.pages : k.hi;
      a.cu_new[b] = of.cu[b];
      if (a.served) a.served[b] = served;
    }
    if (threadIdx.x == 0) {
      a.cu_new[a.batch] = total;
      a.n_free_out[0] = n_all - n_take;
    }
    if (short_of) raise_status(a.dev_status, EBD_DEV_CAPACITY);
  }
  if (bad) raise_status(a.dev_status, EBD_DEV_RANGE);
}

// Exclusive sums over the threads of the cluster (in order of rank, then thread) of
// x[0 .. N), and their totals.  `part` [N] of every CTA holds its own sums meanwhile.
template <int N>
__device__ __forceinline__ void cluster_scan(long long (&x)[N], long long (&total)[N],
                                             long long (*warp_sums)[3], long long* part,
                                             uint32_t rank, uint32_t ranks) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  long long up[N];
#pragma unroll
  for (int i = 0; i < N; ++i) {
    up[i] = x[i];
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const long long u = __shfl_up_sync(0xffffffffu, up[i], o);
      if (lane >= o) up[i] += u;
    }
    if (lane == 31) warp_sums[warp][i] = up[i];
  }
  __syncthreads();
  if (warp == 0) {
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const long long own = warp_sums[lane][i];
      long long s = own;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const long long u = __shfl_up_sync(0xffffffffu, s, o);
        if (lane >= o) s += u;
      }
      warp_sums[lane][i] = s - own;
      if (lane == 31) part[i] = s;
    }
  }
  __syncwarp();
  cluster_barrier();
#pragma unroll
  for (int i = 0; i < N; ++i) {
    long long before = 0, all = 0;
    for (uint32_t r = 0; r < ranks; ++r) {
      const uint32_t at = cluster_map(smem_u32(&part[i]), r);
      const long long p = (long long)ld_cluster_u32(at) | (long long)ld_cluster_u32(at + 4) << 32;
      if (r < rank) before += p;
      all += p;
    }
    x[i] = before + warp_sums[warp][i] + up[i] - x[i];
    total[i] = all;
  }
}

__global__ void __launch_bounds__(kDealThreads, 1) paged_deal_many_kernel(const DealArgs a) {
  __shared__ long long warp_sums[2][32][3], part[2][3];
  __shared__ int cu_s[kDealOffsets + 1];
  grid_launch_dependents();
  grid_dependency_wait();
  const uint32_t ranks = gridDim.x, rank = cluster_rank();
  const int lane = threadIdx.x & 31;
  const int threads = kDealThreads * ranks, tid = rank * kDealThreads + threadIdx.x;
  const int per = (a.batch + threads - 1) / threads;  // sequences of a thread: tid * per ..
  const int b0 = min((long long)tid * per, (long long)a.batch), b1 = min(b0 + per, a.batch);
  bool bad = false, short_of = false;
  auto sync_all = [&]() {
    __syncwarp();
    cluster_barrier();
  };

  // what is given back and what is wanted, up to each thread
  long long x[3] = {0, 0, 0}, all[3];
  for (int b = b0; b < b1; ++b) {
    const Ask k = deal_ask(a, b, bad);
    x[0] += k.keep - k.lo;
    x[1] += k.pages;
    x[2] += k.some;
  }
  const int had = a.n_free[0], n_free = min(max(had, 0), a.n_pages);
  bad |= had != n_free;
  cluster_scan(x, all, warp_sums[0], part[0], rank, ranks);
  // the list cannot hold more than all pages: what a wrong table would add is lost
  const int n_all = (int)min((long long)n_free + all[0], (long long)a.n_pages);
  bad |= (long long)n_free + all[0] > a.n_pages;

  // pages given back, in order of sequence and block; a warp copies one sequence's
  // together.  And who is served: a request for pages that are not there holds back the
  // later ones that need pages too.
  long long y[2] = {0, 0}, got[2];
  long long back = x[0], want = x[1], some = x[2];
  uint32_t ok_bits = 0;  // of the thread's sequences (at most 8)
  for (int i = 0; i < per; ++i) {
    const int b = b0 + i;
    Ask k = {};
    if (b < b1) k = deal_ask(a, b, bad);
    const int gone = k.keep - k.lo;
    for (uint32_t left = __ballot_sync(0xffffffffu, gone > 0); left; left &= left - 1) {
      const int src = __ffs(left) - 1;
      const int sb = __shfl_sync(0xffffffffu, b, src), lo = __shfl_sync(0xffffffffu, k.lo, src);
      const int n = __shfl_sync(0xffffffffu, gone, src);
      const long long at = __shfl_sync(0xffffffffu, back, src) + n_free;
      for (int j = lane; j < n && at + j < a.n_pages; j += 32)
        a.free_pages[at + j] = a.block_table[(size_t)sb * a.max_blocks + lo + j];
    }
    back += gone;
    if (b < b1) {
      want += k.pages;
      some += k.some;
      const bool ok = k.fits && (k.pages == 0 || want <= n_all) &&
                      (k.n <= 0 || some <= a.n_tokens);
      short_of |= !ok;
      if (ok) {
        ok_bits |= 1u << i;
        y[0] += k.pages;
        y[1] += k.some;
      }
    }
  }
  // (its barriers also order the pages given back before they are taken)
  cluster_scan(y, got, warp_sums[1], part[1], rank, ranks);

  long long taken = y[0], tokens = y[1];
  for (int i = 0; i < per; ++i) {
    const int b = b0 + i;
    Ask k = {};
    bool ignore = false;
    if (b < b1) k = deal_ask(a, b, ignore);
    const bool ok = ok_bits >> i & 1;
    const int need = ok ? (int)k.pages : 0;
    for (uint32_t left = __ballot_sync(0xffffffffu, need > 0); left; left &= left - 1) {
      const int src = __ffs(left) - 1;
      const int sb = __shfl_sync(0xffffffffu, b, src), hi = __shfl_sync(0xffffffffu, k.hi, src);
      const int n = __shfl_sync(0xffffffffu, need, src);
      const int top = n_all - 1 - (int)__shfl_sync(0xffffffffu, taken, src);
      for (int j = lane; j < n; j += 32) {
        const int page = __ldcg(a.free_pages + top - j);
        bad |= (unsigned)page >= (unsigned)a.n_pages;
        a.block_table[(size_t)sb * a.max_blocks + hi + j] = page;
      }
    }
    if (b < b1) {
      taken += need;
      if (ok) tokens += k.some;
      const bool leaves = k.n < 0;
      // (each read by this thread only, before: the outputs may be the inputs)
      a.seq_len_out[b] = leaves ? 0 : ok ? k.len + (int)k.some : k.len;
      a.held_out[2 * b] = leaves ? 0 : k.keep;
      a.held_out[2 * b + 1] = leaves ? 0 : k.hi + need;
      a.cu_new[b + 1] = (int)tokens;
      if (a.served) a.served[b] = ok;
    }
  }
  const int total = (int)got[1];
  if (tid == 0) {
    a.cu_new[0] = 0;
    a.n_free_out[0] = n_all - (int)got[0];
  }
  if (a.positions || a.slots) {
    sync_all();
    const bool in_smem = a.batch <= kDealOffsets;
    if (in_smem) {
      for (int i = threadIdx.x; i <= a.batch; i += kDealThreads) cu_s[i] = __ldcg(a.cu_new + i);
      __syncthreads();
    }
    for (int t = tid; t < a.n_tokens; t += threads) {
      int pos = 0;
      int64_t slot = -1;
      if (t < total) {
        int b = 0, end = a.batch - 1;  // the first sequence whose tokens end after t
        while (b < end) {
          const int mid = (b + end) >> 1;
          if ((in_smem ? cu_s[mid + 1] : __ldcg(a.cu_new + mid + 1)) > t) end = mid;
          else b = mid + 1;
        }
        const int c1 = in_smem ? cu_s[b + 1] : __ldcg(a.cu_new + b + 1);
        pos = __ldcg(a.seq_len_out + b) - (c1 - t);
        const int page =
            __ldcg(a.block_table + (size_t)b * a.max_blocks + (pos >> a.page_shift));
        if ((unsigned)page < (unsigned)a.n_pages)
          slot = ((int64_t)page << a.page_shift) + (pos & ((1 << a.page_shift) - 1));
        else
          bad = true;
      }
      if (a.positions) a.positions[t] = pos;
      if (a.slots) a.slots[t] = slot;
    }
  }
  if (bad) raise_status(a.dev_status, EBD_DEV_RANGE);
  if (short_of) raise_status(a.dev_status, EBD_DEV_CAPACITY);
  // no CTA leaves while another may still read its shared memory
  __syncwarp();
  cluster_barrier();
}

static bool overlap(const void* p, size_t n, const void* q, size_t m) {
  const uintptr_t a = (uintptr_t)p, b = (uintptr_t)q;
  return a < b + m && b < a + n;
}

}  // namespace ebd

using namespace ebd;

extern "C" ebd_status ebd_paged_deal(int32_t batch, int32_t page_size, int32_t n_pages,
                                     int32_t max_blocks, int32_t n_tokens, int32_t window,
                                     const int32_t* n_new, const int32_t* seq_len,
                                     const int32_t* held, const int32_t* n_free,
                                     int32_t* free_pages, int32_t* block_table,
                                     int32_t* seq_len_out, int32_t* held_out, int32_t* n_free_out,
                                     int32_t* cu_new, int32_t* served, int32_t* positions,
                                     int64_t* slots, int32_t* dev_status, void* stream) {
  if (batch < 1 || n_pages < 1 || max_blocks < 1 || n_tokens < 0 || window < 0)
    return EBD_ERR_INVALID;
  if (page_size < 8 || page_size > 1024 || (page_size & (page_size - 1)) != 0)
    return EBD_ERR_UNSUPPORTED;
  if ((long long)max_blocks * page_size > 0x7ff00000LL || batch > 65535) return EBD_ERR_UNSUPPORTED;
  // (a number a step past the last, and twice a sum's bound, still fit 31 and 32 bits)
  if (n_tokens > 0x7fff0000 || n_pages > 0x7fff0000) return EBD_ERR_UNSUPPORTED;
  if (!n_new || !seq_len || !held || !n_free || !free_pages || !block_table || !seq_len_out ||
      !held_out || !n_free_out || !cu_new || !dev_status)
    return EBD_ERR_INVALID;
  const size_t B = (size_t)batch * 4;
  // an output is its input or apart from it: a shifted one would be read after it is written
  if ((seq_len_out != seq_len && overlap(seq_len_out, B, seq_len, B)) ||
      (held_out != held && overlap(held_out, 2 * B, held, 2 * B)))
    return EBD_ERR_INVALID;
  DealArgs a = {};
  a.batch = batch;
  a.page_shift = 31 - __builtin_clz((unsigned)page_size);
  a.n_pages = n_pages;
  a.max_blocks = max_blocks;
  a.n_tokens = n_tokens;
  a.window = window;
  a.n_new = n_new;
  a.seq_len = seq_len;
  a.held = held;
  a.n_free = n_free;
  a.free_pages = free_pages;
  a.block_table = block_table;
  a.seq_len_out = seq_len_out;
  a.held_out = held_out;
  a.n_free_out = n_free_out;
  a.cu_new = cu_new;
  a.served = served;
  a.positions = positions;
  a.slots = slots;
  a.dev_status = dev_status;
  const bool small = batch <= kDealThreads && n_tokens <= kDealCluster * kDealFewThreads;
  const int threads = small && batch <= kDealFewThreads ? kDealFewThreads : kDealThreads;
  const int per = (batch + threads - 1) / threads;
  auto kern = batch > kDealSeqs ? paged_deal_many_kernel
              : small           ? paged_deal_kernel<1, false>
              : per == 1        ? paged_deal_kernel<1, true>
                                : paged_deal_kernel<kDealSeqs / kDealThreads, true>;
  cudaLaunchConfig_t cfg = {};
  cfg.blockDim = dim3(threads);
  if (batch <= kDealSeqs) {
    cfg.dynamicSmemBytes = DealSums::bytes(batch);
    if (cfg.dynamicSmemBytes > 40 * 1024 &&
        cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize,
                             (int)DealSums::bytes(kDealSeqs)) != cudaSuccess)
      return EBD_ERR_CUDA;
  }
  static ClusterMemo memo[2];
  const int want = small || batch > kDealSeqs ? kDealCluster : kDealLargeCluster;
  cfg.gridDim = dim3(cluster_ctas(want, kDealLargeCluster, memo[per > 1], kern, threads,
                                  cfg.dynamicSmemBytes));
  cfg.stream = (cudaStream_t)stream;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = cfg.gridDim.x;
  attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
  attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[1].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 2;
  return cuda_status(cudaLaunchKernelEx(&cfg, kern, a));
}
