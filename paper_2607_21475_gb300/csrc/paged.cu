// Gather of kept rows from a paged cache into a compact cache, and the checks
// that the paged entry points share.
//
// The gather reads and writes every kept row once (4 d * elem bytes per row of
// K and V together), so HBM bounds it, if enough rows are in flight: the chain
// index -> page number -> row is three dependent loads, which a warp goes
// through for 8 rows at once (4 rows: 26.0 us, 16 rows: 22.6 us).  Measured: a
// quarter of 8 caches of 12-16k tokens (4 heads x 128, bf16) 22.6 us, 5.0 TB/s (74%
// of the measured copy peak) as a kernel, 24.1 us, 4.7 TB/s in a row of calls; one
// small cache 3.1 us.
#include <cuda_runtime.h>

#include "common.cuh"
#include "internal.h"
#include "paged.cuh"

namespace ebd {

constexpr int kPagedGatherThreads = 256;
constexpr int kGatherFlight = 4;
constexpr int kGatherRows = 8;

ebd_status check_paged(const ebd_paged_cache* c) {
  if (!c || !c->K_pages || !c->V_pages || !c->block_table || !c->seq_len) return EBD_ERR_INVALID;
  if (c->dtype != EBD_F32 && c->dtype != EBD_BF16) return EBD_ERR_INVALID;
  if (c->batch < 1 || c->n_kv_heads < 1 || c->head_dim < 1 || c->n_pages < 1 ||
      c->max_blocks < 1)
    return EBD_ERR_INVALID;
  if (c->page_size < 8 || c->page_size > 1024 || (c->page_size & (c->page_size - 1)) != 0)
    return EBD_ERR_UNSUPPORTED;
  if ((c->n_pages > 1 && c->page_stride < 1) || (c->n_kv_heads > 1 && c->head_stride < 1) ||
      c->page_stride < 0 || c->head_stride < 0 || c->row_stride < c->head_dim)
    return EBD_ERR_INVALID;
  // positions are int32, and so is a tile's end past the last one
  if ((long long)c->max_blocks * c->page_size > 0x7ff00000LL) return EBD_ERR_UNSUPPORTED;
  return EBD_OK;
}

// 16-byte rows: every (page, head, row) starts on a 16-byte boundary.
bool paged_aligned16(const ebd_paged_cache* c) {
  const int wide = c->dtype == EBD_F32 ? 4 : 8;
  return aligned16(c->K_pages) && aligned16(c->V_pages) && c->page_stride % wide == 0 &&
         c->head_stride % wide == 0 && c->row_stride % wide == 0 && c->head_dim % wide == 0;
}

// One warp takes 8 kept rows of a unit: lane i < 8 finds row i's place (index,
// page), then the warp copies the rows' chunks, `cpr` of 16 bytes each, with
// kGatherFlight chunks of K and of V in flight per lane.  The view's strides are
// in chunks.
__global__ void __launch_bounds__(kPagedGatherThreads)
    paged_gather_kernel(const uint4* __restrict__ K, const uint4* __restrict__ V, PagedView v,
                        const int32_t* __restrict__ idx_c, const int32_t* __restrict__ n_kept,
                        int cap, int cpr, uint4* __restrict__ Kc, uint4* __restrict__ Vc,
                        int32_t* dev_status) {
  const int unit = blockIdx.y, b = unit / v.n_kv_heads, h = unit - b * v.n_kv_heads;
  const int lane = threadIdx.x & 31;
  const int p0 = (blockIdx.x * (kPagedGatherThreads / 32) + (threadIdx.x >> 5)) * kGatherRows;
  if (p0 >= cap) return;
  // the three loads do not wait for one another; a row past n_kept is dropped below
  const int kept = n_kept[unit], len = v.seq_len[b];
  const int r = lane < kGatherRows && p0 + lane < cap ? idx_c[(size_t)unit * cap + p0 + lane] : -1;
  const int n = min(min(max(kept, 0), cap) - p0, kGatherRows);
  if (n <= 0) return;
  long long src = -1;
  if (lane < n && (unsigned)r < (unsigned)max(len, 0)) {
    const int page = page_of(v, b, r);
    if (page >= 0) src = slot_offset(v, page, h, r);
    else raise_status(dev_status, EBD_DEV_RANGE);
  }
  __syncwarp();
  const size_t dst = ((size_t)unit * cap + p0) * cpr;
  const int total = n * cpr;
  for (int i0 = lane; i0 < total + lane; i0 += 32 * kGatherFlight) {
    uint4 kv[kGatherFlight], vv[kGatherFlight];
    bool ok[kGatherFlight];
#pragma unroll
    for (int f = 0; f < kGatherFlight; ++f) {
      const int i = i0 + 32 * f, row = i / cpr;
      const long long at = __shfl_sync(0xffffffffu, src, row & (kGatherRows - 1));
      ok[f] = i < total && at >= 0;
      if (ok[f]) {
        kv[f] = __ldg(K + at + (i - row * cpr));
        vv[f] = __ldg(V + at + (i - row * cpr));
      }
    }
#pragma unroll
    for (int f = 0; f < kGatherFlight; ++f) {
      if (ok[f]) {
        Kc[dst + i0 + 32 * f] = kv[f];
        Vc[dst + i0 + 32 * f] = vv[f];
      }
    }
  }
}

}  // namespace ebd

using namespace ebd;

extern "C" ebd_status ebd_paged_gather(const ebd_paged_cache* cache, const int32_t* idx_c,
                                       const int32_t* n_kept, int32_t capacity, void* K_c,
                                       void* V_c, int32_t* dev_status, void* stream) {
  const ebd_status st = check_paged(cache);
  if (st != EBD_OK) return st;
  if (!idx_c || !n_kept || !K_c || !V_c || !dev_status || capacity < 1) return EBD_ERR_INVALID;
  const int eb = cache->dtype == EBD_F32 ? 4 : 2;
  if (cache->head_dim * eb % 16 != 0) return EBD_ERR_UNSUPPORTED;
  if (!paged_aligned16(cache) || !aligned16(K_c) || !aligned16(V_c)) return EBD_ERR_INVALID;
  const long long units = (long long)cache->batch * cache->n_kv_heads;
  if (units > 65535) return EBD_ERR_UNSUPPORTED;
  const int cpr = cache->head_dim * eb / 16, wide = 16 / eb;
  PagedView v = paged_view(*cache);
  v.page_stride /= wide;
  v.head_stride /= wide;
  v.row_stride /= wide;
  const int per_block = kPagedGatherThreads / 32 * kGatherRows;
  const int bx = (capacity + per_block - 1) / per_block;
  paged_gather_kernel<<<dim3((unsigned)bx, (unsigned)units), kPagedGatherThreads, 0,
                        (cudaStream_t)stream>>>((const uint4*)cache->K_pages,
                                                (const uint4*)cache->V_pages, v, idx_c, n_kept,
                                                capacity, cpr, (uint4*)K_c, (uint4*)V_c,
                                                dev_status);
  return launch_status();
}
