// Pages dealt to the sequences of a step from their lengths, and the maps of the step's
// tokens: block tables, packed offsets, positions and slots.
//
// With P positions to a page, a sequence of `len` cached tokens holds the blocks
// [lo, hi) of its row; n new tokens need ceil((len + n) / P) - hi pages more, and with a
// window w the blocks below floor((len - w + 1) / P) are of no use to them.  All that is a
// prefix sum over the sequences, three times two numbers (pages given back, pages wanted,
// tokens), and copies whose places it tells.  Nothing of this is much work; what bounds
// it is the chain of dependent steps: lengths -> sums -> pages -> slots.  One cluster
// of CTAs does it in one launch, a thread per few sequences, and the sums' parts are
// exchanged through distributed shared memory; the results are the same whatever
// the cluster's size.
#include <cuda_runtime.h>

#include "common.cuh"
#include "internal.h"
#include "paged.cuh"
#include "ptx.cuh"

namespace ebd {

constexpr int kDealThreads = 1024;
constexpr int kDealCluster = 8;       // CTAs of a large deal
constexpr int kDealOffsets = 8192;    // packed offsets kept in shared memory

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
  if (ranks > 1) cluster_barrier();
  else __syncthreads();
#pragma unroll
  for (int i = 0; i < N; ++i) {
    long long before = 0, all = 0;
    for (uint32_t r = 0; r < ranks; ++r) {
      long long p = part[i];
      if (ranks > 1) {
        const uint32_t at = cluster_map(smem_u32(&part[i]), r);
        p = (long long)ld_cluster_u32(at) | (long long)ld_cluster_u32(at + 4) << 32;
      }
      if (r < rank) before += p;
      all += p;
    }
    x[i] = before + warp_sums[warp][i] + up[i] - x[i];
    total[i] = all;
  }
}

__global__ void __launch_bounds__(kDealThreads, 1) paged_deal_kernel(const DealArgs a) {
  __shared__ long long warp_sums[2][32][3], part[2][3];
  __shared__ int cu_s[kDealOffsets + 1];
  const uint32_t ranks = gridDim.x, rank = ranks > 1 ? cluster_rank() : 0;
  const int lane = threadIdx.x & 31;
  const int threads = kDealThreads * ranks, tid = rank * kDealThreads + threadIdx.x;
  const int per = (a.batch + threads - 1) / threads;  // sequences of a thread: tid * per ..
  const int b0 = min((long long)tid * per, (long long)a.batch), b1 = min(b0 + per, a.batch);
  bool bad = false, short_of = false;
  auto sync_all = [&]() {
    __syncwarp();
    if (ranks > 1) cluster_barrier();
    else __syncthreads();
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
  if (ranks > 1) cluster_barrier();
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
  const bool small = batch <= kDealThreads && n_tokens <= 2 * kDealThreads;
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(small ? 1 : kDealCluster);
  cfg.blockDim = dim3(kDealThreads);
  cfg.stream = (cudaStream_t)stream;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = cfg.gridDim.x;
  attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  return cuda_status(cudaLaunchKernelEx(&cfg, paged_deal_kernel, a));
}
