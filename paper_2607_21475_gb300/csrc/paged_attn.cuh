// Work split and partial results shared by the paged-attention kernels.
//
// An item is one (sequence, KV head, m-tile): `tokens` new tokens with the query
// heads of the group (row = token x head, token-major) over the key tiles of
// BN positions that at least one row sees.  Items in order of (sequence, head, m-tile) form
// one line of work, each as long as its key tiles and `item_cost` tiles more (the
// time that beginning and ending an item takes), and CTA c of n takes
// [c share, (c + 1) share) of it, whatever items that belongs to: every CTA gets
// the same work however ragged the batch is.  A CTA's range is cut at
// item boundaries into pieces; the pieces of an item that more than one CTA
// holds leave (o / l, log2-sum) in the workspace and a merge kernel joins them
// in CTA order, so results do not depend on timing.  The lengths are on the
// device only, so one warp of each CTA finds the CTA's place on that line.
#pragma once

#include <cuda_runtime.h>
#include <stddef.h>
#include <stdint.h>

#include "common.cuh"
#include "internal.h"
#include "paged.cuh"

namespace ebd {

// What a CTA leaves for the merge: whether its first piece continues an item
// that an earlier CTA began (1: and does not end it, 2: and ends it), and the
// item that its last piece begins without ending (b < 0: none).
struct PieceRecord {
  int cont;
  int b, h, m;
};

struct PagedAttnArgs {
  const void *q, *K_pages, *V_pages;
  PagedView pv;
  const int32_t* cu;
  long long q_ts, q_hs;
  void* y;
  float* lse;  // nullable
  int n_tokens, max_new, group, window;
  float scale2;  // scale * log2(e)
  int32_t* dev_status;
  // split results: slot 2 c of CTA c for a piece that continues an item, slot
  // 2 c + 1 for one that begins an item without ending it
  PieceRecord* rec;  // [n_cta]
  float* part_lse;   // [2 n_cta][slot rows], log2 units
  float* part_o;     // [2 n_cta][slot rows][D]
  // A kernel with few rows per item cuts a large group into slices of at most
  // `slice` query heads; each slice is a head of its own on the line of items.
  int heads;         // KV heads x slices
  int slices, slice;
  int tokens;        // new tokens per item
  int half_tokens;   // of those, how many the slot's first 128 rows hold
  int min_share;     // least work per CTA, in key tiles
  int item_cost;     // work of an item beside its key tiles, in key tiles
};

// KV head, first query head and number of query heads of (sliced) head h.
struct HeadSlice {
  int kvh, q0, n;
};
__device__ __forceinline__ HeadSlice head_slice(const PagedAttnArgs& a, int h) {
  HeadSlice s;
  s.kvh = a.slices == 1 ? h : h / a.slices;
  const int g0 = (h - s.kvh * a.slices) * a.slice;
  s.q0 = s.kvh * a.group + g0;
  s.n = min(a.slice, a.group - g0);
  return s;
}

// Key tiles [kb, ke) of m-tile m; an item with nothing to see keeps one (fully
// masked) tile, so that its rows get written.
template <int BN>
__device__ __forceinline__ void item_range(const PagedAttnArgs& a, int n, int len, int m, int& kb,
                                           int& ke) {
  const int first = m * a.tokens, last = min(n, first + a.tokens) - 1, p0 = len - n;
  const int k_end = p0 + last + 1;  // <= len
  kb = 0;
  ke = 1;
  if (k_end > 0) {
    if (a.window > 0) kb = max(0, p0 + first - a.window + 1) / BN;
    ke = (k_end + BN - 1) / BN;
  }
}

struct WorkStart {
  int b, h, m;
  int off;          // work of the item that earlier CTAs have
  long long count;  // work of this CTA
};

__device__ __forceinline__ long long warp_scan_add(long long v, int lane) {
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const long long u = __shfl_up_sync(0xffffffffu, v, o);
    if (lane >= o) v += u;
  }
  return v;
}

// Work of one head of the sequences base + lane (lane = 0..31).
template <int BN>
__device__ __forceinline__ long long sequence_tiles(const PagedAttnArgs& a, int base, int lane,
                                                    bool report) {
  const int b = base + lane;
  SeqSpan sp = {};
  if (b < a.pv.batch) {
    sp = seq_span(a.pv, a.cu, b, a.n_tokens, a.max_new);
    if (report && sp.bad) raise_status(a.dev_status, EBD_DEV_RANGE);
  }
  const int mt = (sp.n + a.tokens - 1) / a.tokens;
  long long c = 0;
  for (int m = 0; m < min(mt, 4); ++m) {
    int kb, ke;
    item_range<BN>(a, sp.n, sp.len, m, kb, ke);
    c += ke - kb + a.item_cost;
  }
  // long chunks: the warp walks the remaining m-tiles of one sequence together
  for (uint32_t left = __ballot_sync(0xffffffffu, mt > 4); left; left &= left - 1) {
    const int src = __ffs(left) - 1;
    const int n = __shfl_sync(0xffffffffu, sp.n, src), len = __shfl_sync(0xffffffffu, sp.len, src);
    const int k = __shfl_sync(0xffffffffu, mt, src);
    long long sum = 0;
    for (int m = 4 + lane; m < k; m += 32) {
      int kb, ke;
      item_range<BN>(a, n, len, m, kb, ke);
      sum += ke - kb + a.item_cost;
    }
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
    if (lane == src) c += sum;
  }
  return c;
}

__device__ __forceinline__ long long divide(long long x, long long y) {
  return ((x | y) >> 32) == 0 ? (long long)((uint32_t)x / (uint32_t)y) : x / y;
}

// Where CTA `cta` begins on the line, and how much of it is its own; one whole warp.
template <int BN>
__device__ __forceinline__ WorkStart find_work(const PagedAttnArgs& a, int cta, int n_cta,
                                               int lane) {
  const int H = a.heads;
  long long total = 0, c = 0;
  for (int base = 0; base < a.pv.batch; base += 32) {
    c = sequence_tiles<BN>(a, base, lane, cta == 0);
    total += H * c;
  }
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) total += __shfl_xor_sync(0xffffffffu, total, o);
  const long long share = max((long long)a.min_share, divide(total + n_cta - 1, n_cta));
  long long at = cta * share;
  WorkStart w = {0, 0, 0, 0, 0};
  if (at >= total) return w;
  w.count = min(share, total - at);
  for (int base = 0; base < a.pv.batch; base += 32) {
    if (a.pv.batch > 32) c = sequence_tiles<BN>(a, base, lane, false);
    const long long upto = warp_scan_add(c * H, lane);
    const uint32_t past = __ballot_sync(0xffffffffu, upto > at);
    if (past) {
      const int src = __ffs(past) - 1;
      at -= __shfl_sync(0xffffffffu, upto - c * H, src);
      c = __shfl_sync(0xffffffffu, c, src);
      w.b = base + src;
      break;
    }
    at -= __shfl_sync(0xffffffffu, upto, 31);
  }
  w.h = (int)divide(at, c);
  at -= w.h * c;
  const SeqSpan sp = seq_span(a.pv, a.cu, w.b, a.n_tokens, a.max_new);
  const int mt = (sp.n + a.tokens - 1) / a.tokens;
  if (mt == 1) {
    w.off = (int)at;
    return w;
  }
  for (int base = 0; base < mt; base += 32) {
    int kb = 0, ke = -a.item_cost;
    if (base + lane < mt) item_range<BN>(a, sp.n, sp.len, base + lane, kb, ke);
    const long long work = ke - kb + a.item_cost, upto = warp_scan_add(work, lane);
    const uint32_t past = __ballot_sync(0xffffffffu, upto > at);
    if (past) {
      const int src = __ffs(past) - 1;
      w.m = base + src;
      w.off = (int)(at - __shfl_sync(0xffffffffu, upto - work, src));
      break;
    }
    at -= __shfl_sync(0xffffffffu, upto, 31);
  }
  return w;
}

// Walks a CTA's pieces; every role of the CTA walks the same ones.
template <int BN>
struct PieceWalk {
  int b, h, m, mt;
  SeqSpan sp;
  int kb, ke;    // the item's tiles
  int cur, end;  // this piece's
  long long left;  // work after this piece; -1: no piece

  __device__ __forceinline__ PieceWalk(const PagedAttnArgs& a, const WorkStart& w)
      : b(w.b), h(w.h), m(w.m), left(w.count) {
    if (left <= 0) {
      left = -1;
      return;
    }
    load(a);
    take(a, w.off);
    if (cur == end) next(a);
  }
  __device__ __forceinline__ void load(const PagedAttnArgs& a) {
    sp = seq_span(a.pv, a.cu, b, a.n_tokens, a.max_new);
    mt = (sp.n + a.tokens - 1) / a.tokens;
    item_range<BN>(a, sp.n, sp.len, m, kb, ke);
  }
  // This CTA's tiles of the item, of which earlier CTAs have `off`: an item's own
  // cost comes first, so a share that ends within it has no tile.
  __device__ __forceinline__ void take(const PagedAttnArgs& a, int off) {
    const int most = ke - kb + a.item_cost - off, mine = (int)min((long long)most, left);
    cur = kb + max(0, off - a.item_cost);
    end = kb + max(0, off + mine - a.item_cost);
    left -= mine;
  }
  __device__ __forceinline__ bool live() const { return left >= 0; }
  // New tokens of the item, and the first one's number in the sequence.
  __device__ __forceinline__ int tokens(const PagedAttnArgs& a) const {
    return min(a.tokens, sp.n - m * a.tokens);
  }
  __device__ __forceinline__ int first(const PagedAttnArgs& a) const { return m * a.tokens; }
  // Slot of this piece's partial result; -1: the piece is a whole item.
  __device__ __forceinline__ int slot(int cta) const {
    return cur > kb ? 2 * cta : (end < ke ? 2 * cta + 1 : -1);
  }
  __device__ __forceinline__ void next(const PagedAttnArgs& a) {
    do {
      if (left <= 0) {
        left = -1;
        return;
      }
      if (++m < mt) {
        item_range<BN>(a, sp.n, sp.len, m, kb, ke);
      } else {
        m = 0;
        if (++h == a.heads) {
          h = 0;
          do {
            if (++b >= a.pv.batch) {  // the arrays changed under the call: stop
              left = -1;
              return;
            }
            load(a);
          } while (mt == 0);
        } else {
          item_range<BN>(a, sp.n, sp.len, m, kb, ke);
        }
      }
      take(a, 0);
    } while (cur == end);
  }
};

// Enters a piece into the CTA's record.
template <int BN>
__device__ __forceinline__ void record_piece(PieceRecord& r, const PieceWalk<BN>& p, bool first) {
  if (first && p.cur > p.kb) {
    r.cont = p.end < p.ke ? 1 : 2;
  } else if (p.end < p.ke) {
    r.b = p.b;
    r.h = p.h;
    r.m = p.m;
  }
}

// Launches a kernel as a programmatic dependent of whatever precedes it in the
// stream: its prologue overlaps that kernel's tail (it waits before it reads or
// writes memory).
template <typename... Params, typename... Args>
inline ebd_status launch_dependent(void (*kern)(Params...), dim3 grid, int threads, int smem,
                                   cudaStream_t s, Args... args) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = grid;
  cfg.blockDim = dim3(threads);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = s;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  return cuda_status(cudaLaunchKernelEx(&cfg, kern, args...));
}

// Joins the pieces of split items.  `a` as the attention kernel had it.
ebd_status launch_paged_merge(const PagedAttnArgs& a, bool bf16, int head_dim, int slot_rows,
                              int n_cta, cudaStream_t s);

// Bytes of the split results of n_cta CTAs.
size_t paged_split_bytes(int n_cta, int slot_rows, int head_dim);
// Points a's split arrays into the workspace.
void paged_split_layout(PagedAttnArgs& a, void* ws, int n_cta, int slot_rows);

ebd_status launch_paged_tc(PagedAttnArgs a, const ebd_paged_cache& c, int n_cta,
                           cudaStream_t s);
constexpr int kTcSlotRows = 256;  // rows of a partial result

}  // namespace ebd
