// Gather of kept rows from a paged cache into a compact cache, and the checks
// that the paged entry points share.
//
// The gather reads and writes every kept row once (4 d * elem bytes per row of
// K and V together), so HBM bounds it.  A thread moves 16-byte chunks, four in
// flight: the chain index -> page number -> row is three dependent loads, and
// neighbouring lanes share the first two.
#include <cuda_runtime.h>

#include "common.cuh"
#include "internal.h"
#include "paged.cuh"

namespace ebd {

constexpr int kPagedGatherThreads = 256;
constexpr int kPagedGatherUnroll = 4;

ebd_status check_paged(const ebd_paged_cache* c) {
  if (!c || !c->K_pages || !c->V_pages || !c->block_table || !c->seq_len) return EBD_ERR_INVALID;
  if (c->dtype != EBD_F32 && c->dtype != EBD_BF16) return EBD_ERR_INVALID;
  if (c->batch < 1 || c->n_kv_heads < 1 || c->head_dim < 1 || c->n_pages < 1 ||
      c->max_blocks < 1)
    return EBD_ERR_INVALID;
  if (c->page_size < 8 || c->page_size > 1024 || (c->page_size & (c->page_size - 1)) != 0)
    return EBD_ERR_UNSUPPORTED;
  if (c->page_stride < 0 || c->head_stride < 0 || c->row_stride < c->head_dim)
    return EBD_ERR_INVALID;
  // positions are int32
  if ((long long)c->max_blocks * c->page_size > 0x7fffffffLL) return EBD_ERR_UNSUPPORTED;
  return EBD_OK;
}

// 16-byte rows: every (page, head, row) starts on a 16-byte boundary.
bool paged_aligned16(const ebd_paged_cache* c) {
  const int wide = c->dtype == EBD_F32 ? 4 : 8;
  return aligned16(c->K_pages) && aligned16(c->V_pages) && c->page_stride % wide == 0 &&
         c->head_stride % wide == 0 && c->row_stride % wide == 0 && c->head_dim % wide == 0;
}

// cpr: 16-byte chunks per row; the view's strides are in chunks too.
__global__ void __launch_bounds__(kPagedGatherThreads)
    paged_gather_kernel(const uint4* __restrict__ K, const uint4* __restrict__ V, PagedView v,
                        const int32_t* __restrict__ idx_c, const int32_t* __restrict__ n_kept,
                        int cap, int cpr, uint4* __restrict__ Kc, uint4* __restrict__ Vc,
                        int32_t* dev_status) {
  const int unit = blockIdx.y, b = unit / v.n_kv_heads, h = unit - b * v.n_kv_heads;
  const int len = v.seq_len[b];
  const long long items = (long long)min(max(n_kept[unit], 0), cap) * cpr;
  const long long stride = (long long)gridDim.x * kPagedGatherThreads;
  const int32_t* idx = idx_c + (size_t)unit * cap;
  const size_t dst_base = (size_t)unit * cap * cpr;
  bool bad = false;
  for (long long it0 = (long long)blockIdx.x * kPagedGatherThreads + threadIdx.x; it0 < items;
       it0 += stride * kPagedGatherUnroll) {
    uint4 kv[kPagedGatherUnroll], vv[kPagedGatherUnroll];
    long long src[kPagedGatherUnroll];
#pragma unroll
    for (int u = 0; u < kPagedGatherUnroll; ++u) {
      const long long it = it0 + u * stride;
      src[u] = -1;
      if (it < items) {
        const int p = (int)(it / cpr);
        const int r = idx[p];
        if ((unsigned)r < (unsigned)max(len, 0)) {
          const int page = page_of(v, b, r);
          if (page >= 0) src[u] = slot_offset(v, page, h, r) + (it - (long long)p * cpr);
          else bad = true;
        }
      }
    }
#pragma unroll
    for (int u = 0; u < kPagedGatherUnroll; ++u) {
      if (src[u] >= 0) {
        kv[u] = __ldg(K + src[u]);
        vv[u] = __ldg(V + src[u]);
      }
    }
#pragma unroll
    for (int u = 0; u < kPagedGatherUnroll; ++u) {
      if (src[u] >= 0) {
        Kc[dst_base + it0 + u * stride] = kv[u];
        Vc[dst_base + it0 + u * stride] = vv[u];
      }
    }
  }
  if (bad) raise_status(dev_status, EBD_DEV_RANGE);
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
  const long long per_block = (long long)kPagedGatherThreads * kPagedGatherUnroll;
  long long bx = ((long long)capacity * cpr + per_block - 1) / per_block;
  const long long most = ((long long)sm_count() * 8 + units - 1) / units;
  if (bx > most) bx = most;
  paged_gather_kernel<<<dim3((unsigned)bx, (unsigned)units), kPagedGatherThreads, 0,
                        (cudaStream_t)stream>>>((const uint4*)cache->K_pages,
                                                (const uint4*)cache->V_pages, v, idx_c, n_kept,
                                                capacity, cpr, (uint4*)K_c, (uint4*)V_c,
                                                dev_status);
  return launch_status();
}
