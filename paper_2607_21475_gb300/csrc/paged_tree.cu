// Around attention of a drafted tree over a paged cache: the masks and positions of its
// tokens, and the rows of an accepted path moved to where the next step expects them.
//
// A tree's tokens come packed like any new tokens, parents before children; token i of a
// sequence names its parent's number (-1: the last cached token).  Bit j of its mask row
// says that j is i or an ancestor of it, and it stands at position base + depth, base
// being the cached tokens before the tree.  A warp walks one token's line of ancestors
// over the parents in shared memory, a lane per 32-bit word of the row: as many steps as
// the token is deep, 30 to 40 cycles each.
//
// After verification tokens path[0] < path[1] < .. of the tree are kept: row base + path[i]
// of every layer and head moves to base + i.  A thread has one 16-byte column of a head and
// walks the path upwards: path[i] >= i, so no source is overwritten before it is read,
// neither within a step of kKeepFlight loads and then their stores nor by earlier ones.
// HBM and the chain lengths -> path -> pages -> rows bound it.
//
// Both are programmatic dependents of what precedes them on the stream, and let the next
// kernel of that kind begin.  Since they may begin before the kernel that writes their inputs
// ends, nothing that it may write is declared constant (const __restrict__, __ldg): such a load
// may be moved before the wait, or served from a cache that the wait does not clear.
// Measured: masks of 16 to 64 tokens 2.3-3 us; paths of up to 8 of 64 tokens of 32 sequences
// in 28 layers (8 heads x 128, bf16) 5.2 us, 16 MB of rows; one small layer 2.6 us.
#include <cuda_runtime.h>

#include "common.cuh"
#include "decode_tile.cuh"
#include "internal.h"
#include "paged.cuh"
#include "paged_attn.cuh"

namespace ebd {

constexpr int kTreeWarps = 8;
constexpr int kTreeMost = 1024;  // new tokens of a sequence with a tree mask
constexpr int kKeepThreads = 256;
constexpr int kKeepFlight = 4;
constexpr int kKeepMoves = 32;   // path entries placed at a time

// Block (x, b): tokens kTreeWarps x .. of sequence b.
__global__ void __launch_bounds__(kTreeWarps * 32)
    tree_masks_kernel(const int32_t* parents, const int32_t* cu, const int32_t* seq_len,
                      int n_tokens, int max_new, int words, int window, uint32_t* mask,
                      int32_t* positions, int32_t* dev_status) {
  __shared__ int parent_s[kTreeMost];
  const int b = blockIdx.y, lane = threadIdx.x & 31, first = blockIdx.x * kTreeWarps;
  grid_launch_dependents();
  grid_dependency_wait();
  const int c0 = cu[b], c1 = cu[b + 1], len = seq_len[b];
  const int t0 = min(max(c0, 0), n_tokens), t1 = min(max(c1, t0), n_tokens);
  const int n = min(t1 - t0, max_new);
  // (places past the last offset are empty, as a deal leaves them)
  const bool odd = t0 != c0 || t0 + n != c1 || len < n || (b == 0 && c0 != 0);
  if (odd && blockIdx.x == 0 && threadIdx.x == 0) raise_status(dev_status, EBD_DEV_RANGE);
  const int upto = min(n, first + kTreeWarps);  // a line of ancestors goes down
  if (first >= upto) return;
  bool bad = false;
  for (int i = threadIdx.x; i < upto; i += kTreeWarps * 32) {
    int p = parents[t0 + i];
    if (p < -1 || p >= i) {  // no earlier token: taken for -1
      bad |= i >= first;
      p = -1;
    }
    parent_s[i] = p;
  }
  if (bad) raise_status(dev_status, EBD_DEV_RANGE);
  __syncthreads();
  const int i = first + (threadIdx.x >> 5);
  if (i >= upto) return;
  uint32_t word = 0;
  int depth = 0;
  for (int p = i; p >= 0; p = parent_s[p], ++depth)
    if (p >> 5 == lane && (window == 0 || depth < window)) word |= 1u << (p & 31);
  const size_t t = t0 + i;
  if (lane < words) mask[t * words + lane] = word;
  if (lane == 0) positions[t] = len - n + depth - 1;
}

// Block (x, layer): sequence x.  The view's strides and layer_stride are in chunks of 16
// bytes, `cpr` of them to a row.
__global__ void __launch_bounds__(kKeepThreads)
    paged_keep_kernel(uint4* K, uint4* V, PagedView v,
                      long long layer_stride, int cpr, const int32_t* cu, const int32_t* path,
                      const int32_t* n_kept, int max_path, int32_t* seq_len_out,
                      int32_t* dev_status) {
  __shared__ long long from_s[kKeepMoves], to_s[kKeepMoves];
  __shared__ int kept_s, moves_s;
  const int b = blockIdx.x, lane = threadIdx.x & 31;
  grid_launch_dependents();
  grid_dependency_wait();
  // the path's first entries do not wait for the lengths
  const int32_t* row = path + (size_t)b * max_path;
  const int p_first = lane < max_path ? row[lane] : 0;
  const int c0 = cu[b], c1 = cu[b + 1], len_b = v.seq_len[b], kept_b = n_kept[b];
  const long long most = (long long)v.max_blocks << v.page_shift;
  const int len = (int)min((long long)max(len_b, 0), most);
  const int n = min(max(c1, c0) - c0, len);  // the tree's tokens: the sequence's last ones
  const int base = len - n;
  const int k = min(max(kept_b, 0), min(max_path, n));
  bool bad = len != len_b || c1 - c0 != n || kept_b != k;
  K += blockIdx.y * layer_stride;
  V += blockIdx.y * layer_stride;
  // (one pool for both: its rows move once)
  const int columns = (K == V ? 1 : 2) * v.n_kv_heads * cpr;
  // the path is good up to the first entry that does not rise or is no new token
  int kept = k;
  for (int i0 = 0; i0 < kept; i0 += kKeepMoves) {
    if (threadIdx.x < 32) {
      const int i = i0 + lane;
      int p = p_first, before = __shfl_up_sync(0xffffffffu, p_first, 1);
      if (i0 > 0) p = i < kept ? row[i] : 0, before = i < kept ? row[i - 1] : -1;
      if (i == 0) before = -1;
      const uint32_t wrong =
          __ballot_sync(0xffffffffu, i < kept && (p <= before || p >= n || p < 0));
      const int good = wrong ? i0 + __ffs(wrong) - 1 : kept;
      bad |= wrong != 0;
      long long from = -1, to = -1;
      if (i < good && p != i) {
        const int page0 = page_of(v, b, base + p), page1 = page_of(v, b, base + i);
        if (page0 >= 0 && page1 >= 0) {
          from = slot_offset(v, page0, 0, base + p);
          to = slot_offset(v, page1, 0, base + i);
        } else {
          raise_status(dev_status, EBD_DEV_RANGE);
        }
      }
      // only rows that move, in order
      const uint32_t move = __ballot_sync(0xffffffffu, to >= 0);
      if (to >= 0) {
        const int at = __popc(move & ((1u << lane) - 1));
        from_s[at] = from;
        to_s[at] = to;
      }
      if (lane == 0) {
        kept_s = good;
        moves_s = __popc(move);
      }
    }
    __syncthreads();
    kept = kept_s;
    const int moves = moves_s;
    for (int c = threadIdx.x; c < columns && moves > 0; c += kKeepThreads) {
      const int r = c / cpr, h = r < v.n_kv_heads ? r : r - v.n_kv_heads;
      uint4* pool = (r < v.n_kv_heads ? K : V) + h * v.head_stride + (c - r * cpr);
      for (int m = 0; m < moves; m += kKeepFlight) {
        uint4 x[kKeepFlight];
#pragma unroll
        for (int f = 0; f < kKeepFlight; ++f)
          if (m + f < moves) x[f] = pool[from_s[m + f]];
#pragma unroll
        for (int f = 0; f < kKeepFlight; ++f)
          if (m + f < moves) pool[to_s[m + f]] = x[f];
      }
    }
    __syncthreads();
  }
  if (threadIdx.x == 0) {
    if (bad) raise_status(dev_status, EBD_DEV_RANGE);
    if (blockIdx.y == 0 && seq_len_out) seq_len_out[b] = base + kept;
  }
}

}  // namespace ebd

using namespace ebd;

extern "C" ebd_status ebd_tree_masks(int32_t batch, int32_t n_tokens, int32_t max_new,
                                     const int32_t* parents, const int32_t* cu_new,
                                     const int32_t* seq_len, int32_t window, uint32_t* mask,
                                     int32_t mask_words, int32_t* positions, int32_t* dev_status,
                                     void* stream) {
  if (batch < 1 || n_tokens < 0 || max_new < (n_tokens > 0) || window < 0 ||
      mask_words < (n_tokens > 0))
    return EBD_ERR_INVALID;
  if (max_new > 32ll * mask_words) return EBD_ERR_INVALID;
  if (max_new > kTreeMost || mask_words > kTreeMost / 32 || batch > 65535)
    return EBD_ERR_UNSUPPORTED;
  if (n_tokens == 0) return EBD_OK;
  if (!parents || !cu_new || !seq_len || !mask || !positions) return EBD_ERR_INVALID;
  return launch_dependent(tree_masks_kernel, dim3((max_new + kTreeWarps - 1) / kTreeWarps, batch),
                          kTreeWarps * 32, 0, (cudaStream_t)stream, parents, cu_new, seq_len,
                          n_tokens, max_new, mask_words, window, mask, positions, dev_status);
}

extern "C" ebd_status ebd_paged_keep(const ebd_paged_cache* cache, int32_t n_layers,
                                     int64_t layer_stride, const int32_t* cu_new,
                                     const int32_t* path, int32_t max_path,
                                     const int32_t* n_accepted, int32_t* seq_len_out,
                                     int32_t* dev_status, void* stream) {
  const ebd_status st = check_paged(cache);
  if (st != EBD_OK) return st;
  if (n_layers < 1 || (n_layers > 1 && layer_stride < 1) || max_path < 1) return EBD_ERR_INVALID;
  if (!cu_new || !path || !n_accepted || !dev_status) return EBD_ERR_INVALID;
  // the lengths are read by every block: the new ones go elsewhere
  if (seq_len_out) {
    const uintptr_t p = (uintptr_t)seq_len_out, q = (uintptr_t)cache->seq_len;
    const size_t bytes = (size_t)cache->batch * 4;
    if (p < q + bytes && q < p + bytes) return EBD_ERR_INVALID;
  }
  const int eb = cache->dtype == EBD_F32 ? 4 : 2, wide = 16 / eb;
  if (cache->head_dim * eb % 16 != 0) return EBD_ERR_UNSUPPORTED;
  if (!paged_aligned16(cache) || (n_layers > 1 && layer_stride % wide != 0))
    return EBD_ERR_INVALID;
  if (n_layers > 65535) return EBD_ERR_UNSUPPORTED;
  PagedView v = paged_view(*cache);
  v.page_stride /= wide;
  v.head_stride /= wide;
  v.row_stride /= wide;
  return launch_dependent(
      paged_keep_kernel, dim3((unsigned)cache->batch, (unsigned)n_layers), kKeepThreads, 0,
      (cudaStream_t)stream, (uint4*)cache->K_pages, (uint4*)cache->V_pages, v,
      n_layers > 1 ? layer_stride / wide : 0ll, cache->head_dim / wide, cu_new, path, n_accepted,
      max_path, seq_len_out, dev_status);
}
