// Device view of a paged KV cache (ebd_paged_cache) and the helpers that the
// paged operators share.
#pragma once

#include <cuda_runtime.h>
#include <stddef.h>
#include <stdint.h>

#include "../../include/ebd.h"
#include "common.cuh"

namespace ebd {

struct PagedView {
  const int32_t* block_table;  // [batch, max_blocks]
  const int32_t* seq_len;      // [batch]
  int n_kv_heads, n_pages, batch, max_blocks;
  int page_shift;              // log2(page_size)
  long long page_stride, head_stride, row_stride;  // elements
};

__host__ inline PagedView paged_view(const ebd_paged_cache& c) {
  PagedView v;
  v.block_table = c.block_table;
  v.seq_len = c.seq_len;
  v.n_kv_heads = c.n_kv_heads;
  v.n_pages = c.n_pages;
  v.batch = c.batch;
  v.max_blocks = c.max_blocks;
  v.page_shift = 31 - __builtin_clz((unsigned)c.page_size);
  v.page_stride = c.page_stride;
  v.head_stride = c.head_stride;
  v.row_stride = c.row_stride;
  return v;
}

// Page that holds position pos of sequence b; -1 when the position lies past
// the block table or the table names a page outside the pool.
__device__ __forceinline__ int page_of(const PagedView& v, int b, int pos) {
  const int blk = pos >> v.page_shift;
  if (pos < 0 || blk >= v.max_blocks) return -1;
  const int p = v.block_table[(size_t)b * v.max_blocks + blk];
  return (unsigned)p < (unsigned)v.n_pages ? p : -1;
}

// Element offset of (page, kv head, position) in K_pages / V_pages; 64-bit, a
// pool may hold more than 2^31 elements.
__device__ __forceinline__ long long slot_offset(const PagedView& v, int page, int h, int pos) {
  return (long long)page * v.page_stride + (long long)h * v.head_stride +
         (long long)(pos & ((1 << v.page_shift) - 1)) * v.row_stride;
}

// Sequence of packed token t: the first whose tokens end after it (cu [batch + 1]).
// odd: an offset steps back past t.  Whole warp, one t.
__device__ __forceinline__ int sequence_of(const int32_t* cu, int batch, int t, int lane,
                                           bool& odd) {
  int b = 0;
  odd = false;
  for (int i = lane; i - lane < batch; i += 32) {
    const bool before = i < batch && cu[i + 1] <= t;
    const uint32_t ended = __ballot_sync(0xffffffffu, before);
    if (ended == 0xffffffffu) {
      b += 32;
      continue;
    }
    b += __ffs(~ended) - 1;
    odd = (ended & (ended + 1)) != 0;
    break;
  }
  return b;
}

// New tokens and length of sequence b, forced into the ranges that the call
// was given (n_tokens packed tokens, at most max_new per sequence, max_blocks
// pages): whatever the device arrays hold, nothing is read or written outside.
struct SeqSpan {
  int t0;    // first packed token
  int n;     // new tokens
  int len;   // keys in the cache, new tokens included
  bool bad;  // an entry was outside its range
};

// padded: places past the last offset are empty, no mistake.
__device__ __forceinline__ SeqSpan seq_span(const PagedView& v, const int32_t* cu, int b,
                                            int n_tokens, int max_new, bool padded) {
  const int c0 = cu[b], c1 = cu[b + 1], l = v.seq_len[b];
  SeqSpan s;
  s.t0 = min(max(c0, 0), n_tokens);
  const int t1 = min(max(c1, s.t0), n_tokens);
  s.n = min(t1 - s.t0, max_new);
  const long long most = (long long)v.max_blocks << v.page_shift;
  s.len = (int)min((long long)max(l, 0), most);
  // the offsets run from 0 to n_tokens: what lies before or after is no sequence's
  s.bad = s.t0 != c0 || s.t0 + s.n != c1 || s.len != l || (b == 0 && c0 != 0) ||
          (!padded && b == v.batch - 1 && c1 != n_tokens);
  return s;
}

}  // namespace ebd
