// Work split and partial results shared by the paged-attention kernels.
//
// An item is one (sequence, KV head, m-tile): `tokens` new tokens with the query
// heads of the group (row = token x head, token-major) over the key tiles of
// BN positions that at least one row sees.  Items in order of (sequence, head, m-tile) form
// one line of work, each as long as its key tiles' work and `item_cost` more (the
// time that beginning and ending an item takes), and CTA c of n takes
// [c share, (c + 1) share) of it, whatever items that belongs to: every CTA gets
// the same work however ragged the batch is.  A CTA's range is cut at
// item boundaries into pieces; the pieces of an item that more than one CTA
// holds leave (o / l, log2-sum) in the workspace and a merge kernel joins them
// in CTA order, so results do not depend on timing.  The lengths are on the
// device only, so one warp of each CTA finds the CTA's place on that line (32-bit
// arithmetic: the entry point refuses what could be longer).
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
// item that its last piece begins without ending: its head, first packed token and
// number of tokens (0: no such item).
struct PieceRecord {
  int cont;
  int h, token, tokens;
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
  float* part_o;     // [2 n_cta][slot rows / 32][D / 4][32 rows][4]: a warp that has a
                     // row per lane reads and writes whole lines
  // A kernel with few rows per item cuts a large group into slices of at most
  // `slice` query heads; each slice is a head of its own on the line of items.
  int heads;         // KV heads x slices
  int slices, slice;
  int tokens;        // new tokens per item
  int half_tokens;   // of those, how many the slot's first 128 rows hold
  int slot_rows;     // rows of a partial result: 8, 16 or a multiple of 32
  int part_step;     // floats between 4-channel groups of a row in part_o
  int tile_work;     // work of a key tile of an item of at most half_tokens tokens,
  int full_work;     // and of a larger item
  int min_share;     // least work per CTA
  int item_cost;     // work of an item beside its key tiles
  // Tree attention: which of its sequence's new tokens each one sees, in place of those
  // up to it, and where each stands (for the window over the earlier positions).
  const uint32_t* mask;      // [n_tokens][mask_words]; null: causal
  const int32_t* positions;  // [n_tokens]; needed with a window
  int mask_words;
  bool padded;               // (host) places past the last offset are empty, no mistake
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

// The first position that a token at position p sees.
__device__ __forceinline__ int first_seen(const PagedAttnArgs& a, int p) {
  return a.window > 0 && p >= a.window ? p - a.window + 1 : 0;
}

// The first position that a tree's token t sees before the tree, which begins at position
// base; it is the tree's token number i, and stands between base and base + i.
__device__ __forceinline__ int tree_first_seen(const PagedAttnArgs& a, int t, int base, int i,
                                               bool& bad) {
  if (a.window == 0) return 0;
  const int p = a.positions[t], at = min(max(p, base), base + i);
  bad |= p != at;
  return min(first_seen(a, at), max(base, 0));
}

// Mask words w, w + 1 of new token t, as one.  (Ordinary loads: the kernel that writes them may
// not have ended when this one begins.)
__device__ __forceinline__ uint64_t tree_words(const PagedAttnArgs& a, int t, int w) {
  const uint32_t* row = a.mask + (size_t)t * a.mask_words;
  const uint32_t lo = w < a.mask_words ? row[w] : 0u;
  const uint32_t hi = w + 1 < a.mask_words ? row[w + 1] : 0u;
  return (uint64_t)hi << 32 | lo;
}

// Which of the BN = 32 or 64 keys from position k0 on (bit j: key k0 + j) the tree's token t
// sees: lo and later before the tree, and those of its mask up to itself (number i).
template <int BN>
__device__ __forceinline__ uint64_t tree_visible(const PagedAttnArgs& a, int t, int i, int base,
                                                 int lo, int k0) {
  const int at = k0 - base;  // number of the first key as a new token
  uint64_t bits = 0;
  if (at > -BN) {
    if (at >= 0) {
      bits = tree_words(a, t, at >> 5) >> (at & 31);
      if (BN == 64 && (at & 31))
        bits |= tree_words(a, t, (at >> 5) + 2) << (64 - (at & 31));
    } else {
      bits = tree_words(a, t, 0) << -at;
    }
    const int own = i - at;  // (numbers after its own are hidden)
    if (own < 63) bits &= own < 0 ? 0 : (2ull << own) - 1;
  }
  const int skip = lo - k0, end = -at;  // earlier positions: keys skip .. end - 1
  if (end > 0) {
    uint64_t early = end >= 64 ? ~0ull : (1ull << end) - 1;
    if (skip > 0) early &= skip >= 64 ? 0 : ~0ull << skip;
    bits |= early;
  }
  return bits;
}

// Key tiles [kb, ke) of m-tile m; an item with nothing to see keeps one (fully
// masked) tile, so that its rows get written.
template <int BN, bool TREE>
__device__ __forceinline__ void item_range(const PagedAttnArgs& a, int n, int len, int m, int& kb,
                                           int& ke) {
  const int first = m * a.tokens, last = min(n, first + a.tokens) - 1, p0 = len - n;
  const int k_end = p0 + last + 1;  // <= len
  kb = 0;
  ke = 1;
  if (k_end > 0) {
    // (a tree's tokens may all stand where it begins)
    kb = first_seen(a, TREE ? p0 : p0 + first) / BN;
    ke = (k_end + BN - 1) / BN;
  }
}

// Work of a key tile of m-tile m of n new tokens.
__device__ __forceinline__ int tile_work(const PagedAttnArgs& a, int n, int m) {
  return n - m * a.tokens > a.half_tokens ? a.full_work : a.tile_work;
}

// Channel 0 of row `row` of a partial result; channels 4 c .. + 3 are c part_step
// floats further.
template <int D>
__device__ __forceinline__ float* part_row(const PagedAttnArgs& a, int slot, int row) {
  return a.part_o + ((size_t)slot * a.slot_rows + (row & ~31)) * D + (row & 31) * 4;
}

struct WorkStart {
  int b, h, m;
  int off;     // work of the item that earlier CTAs have
  int count;   // work of this CTA
  int mt;      // m-tiles of the sequence
  SeqSpan sp;  // and its span
};

__device__ __forceinline__ int warp_scan_add(int v, int lane) {
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int u = __shfl_up_sync(0xffffffffu, v, o);
    if (lane >= o) v += u;
  }
  return v;
}

// Work of one head of the sequences base + lane (lane = 0..31), their spans and m-tiles.
template <int BN, bool TREE, bool PADDED>
__device__ __forceinline__ int sequence_work(const PagedAttnArgs& a, int base, int lane,
                                             bool report, SeqSpan& sp, int& mt) {
  const int b = base + lane;
  sp = SeqSpan{};
  if (b < a.pv.batch) {
    sp = seq_span(a.pv, a.cu, b, a.n_tokens, a.max_new, PADDED);
    if (report && sp.bad) raise_status(a.dev_status, EBD_DEV_RANGE);
  }
  mt = (int)((uint32_t)(sp.n + a.tokens - 1) / (uint32_t)a.tokens);
  int c = 0;
  for (int m = 0; m < min(mt, 4); ++m) {
    int kb, ke;
    item_range<BN, TREE>(a, sp.n, sp.len, m, kb, ke);
    c += (ke - kb) * tile_work(a, sp.n, m) + a.item_cost;
  }
  // long chunks: the warp walks the remaining m-tiles of one sequence together
  for (uint32_t left = __ballot_sync(0xffffffffu, mt > 4); left; left &= left - 1) {
    const int src = __ffs(left) - 1;
    const int n = __shfl_sync(0xffffffffu, sp.n, src), len = __shfl_sync(0xffffffffu, sp.len, src);
    const int k = __shfl_sync(0xffffffffu, mt, src);
    int sum = 0;
    for (int m = 4 + lane; m < k; m += 32) {
      int kb, ke;
      item_range<BN, TREE>(a, n, len, m, kb, ke);
      sum += (ke - kb) * tile_work(a, n, m) + a.item_cost;
    }
    sum = __reduce_add_sync(0xffffffffu, sum);
    if (lane == src) c += sum;
  }
  return c;
}

// Where CTA `cta` begins on the line, and how much of it is its own; one whole warp.
template <int BN, bool TREE, bool PADDED>
__device__ __forceinline__ WorkStart find_work(const PagedAttnArgs& a, int cta, int n_cta,
                                               int lane) {
  const int H = a.heads;
  SeqSpan sp;
  int total = 0, c = 0, upto = 0, mt = 0;
  for (int base = 0; base < a.pv.batch; base += 32) {
    c = sequence_work<BN, TREE, PADDED>(a, base, lane, cta == 0, sp, mt);
    upto = warp_scan_add(c * H, lane);
    total += __shfl_sync(0xffffffffu, upto, 31);
  }
  const int share = max(a.min_share, (int)((uint32_t)(total + n_cta - 1) / (uint32_t)n_cta));
  int at = cta * share;
  WorkStart w = {};
  if (at >= total) return w;
  const int count = min(share, total - at);
  for (int base = 0; base < a.pv.batch; base += 32) {
    if (a.pv.batch > 32) {
      c = sequence_work<BN, TREE, PADDED>(a, base, lane, false, sp, mt);
      upto = warp_scan_add(c * H, lane);
    }
    const uint32_t past = __ballot_sync(0xffffffffu, upto > at);
    if (past) {
      const int src = __ffs(past) - 1;
      at -= __shfl_sync(0xffffffffu, upto - c * H, src);
      c = __shfl_sync(0xffffffffu, c, src);
      w.b = base + src;
      w.mt = __shfl_sync(0xffffffffu, mt, src);
      w.sp.t0 = __shfl_sync(0xffffffffu, sp.t0, src);
      w.sp.n = __shfl_sync(0xffffffffu, sp.n, src);
      w.sp.len = __shfl_sync(0xffffffffu, sp.len, src);
      w.count = count;
      break;
    }
    at -= __shfl_sync(0xffffffffu, upto, 31);
  }
  if (w.count == 0) return w;  // the arrays changed under the call: no work
  w.h = (int)((uint32_t)at / (uint32_t)c);
  at -= w.h * c;
  if (w.mt == 1) {
    w.off = at;
    return w;
  }
  for (int base = 0; base < w.mt; base += 32) {
    int work = 0;
    if (base + lane < w.mt) {
      int kb, ke;
      item_range<BN, TREE>(a, w.sp.n, w.sp.len, base + lane, kb, ke);
      work = (ke - kb) * tile_work(a, w.sp.n, base + lane) + a.item_cost;
    }
    const int end = warp_scan_add(work, lane);
    const uint32_t past = __ballot_sync(0xffffffffu, end > at);
    if (past) {
      const int src = __ffs(past) - 1;
      w.m = base + src;
      w.off = at - __shfl_sync(0xffffffffu, end - work, src);
      break;
    }
    at -= __shfl_sync(0xffffffffu, end, 31);
  }
  return w;
}

// Walks a CTA's pieces; every role of the CTA walks the same ones.
template <int BN, bool TREE>
struct PieceWalk {
  int b, h, m, mt;
  SeqSpan sp;
  int kb, ke;    // the item's tiles
  int cur, end;  // this piece's
  int left;      // work after this piece; -1: no piece

  __device__ __forceinline__ PieceWalk(const PagedAttnArgs& a, const WorkStart& w)
      : b(w.b), h(w.h), m(w.m), mt(w.mt), sp(w.sp), left(w.count) {
    if (left <= 0) {
      left = -1;
      return;
    }
    item_range<BN, TREE>(a, sp.n, sp.len, m, kb, ke);
    take(a, w.off);
    if (cur == end) next(a);
  }
  __device__ __forceinline__ void load(const PagedAttnArgs& a) {
    sp = seq_span(a.pv, a.cu, b, a.n_tokens, a.max_new, true);  // (nothing is reported here)
    mt = (int)((uint32_t)(sp.n + a.tokens - 1) / (uint32_t)a.tokens);
    item_range<BN, TREE>(a, sp.n, sp.len, m, kb, ke);
  }
  // This CTA's tiles of the item, of which earlier CTAs have the first `off` of its
  // work: an item's own cost comes first, so a share that ends within it has no
  // tile; a tile cut in two is the later CTA's.
  __device__ __forceinline__ void take(const PagedAttnArgs& a, int off) {
    const uint32_t each = tile_work(a, sp.n, m);
    const int most = (ke - kb) * (int)each + a.item_cost - off, mine = min(most, left);
    cur = off <= a.item_cost ? kb : kb + (int)((uint32_t)(off - a.item_cost) / each);
    end = mine == most ? ke : kb + (int)((uint32_t)max(0, off + mine - a.item_cost) / each);
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
        item_range<BN, TREE>(a, sp.n, sp.len, m, kb, ke);
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
          item_range<BN, TREE>(a, sp.n, sp.len, m, kb, ke);
        }
      }
      take(a, 0);
    } while (cur == end);
  }
};

// Enters a piece into the CTA's record.
template <int BN, bool TREE>
__device__ __forceinline__ void record_piece(const PagedAttnArgs& a, PieceRecord& r,
                                             const PieceWalk<BN, TREE>& p, bool first) {
  if (first && p.cur > p.kb) {
    r.cont = p.end < p.ke ? 1 : 2;
  } else if (p.end < p.ke) {
    r.h = p.h;
    r.token = p.sp.t0 + p.first(a);
    r.tokens = p.tokens(a);
  }
}

__device__ __forceinline__ void round_to(float x, float& y) { y = x; }
__device__ __forceinline__ void round_to(float x, __nv_bfloat16& y) { y = __float2bfloat16_rn(x); }

// C consecutive values of a row, in one access.
template <typename T, int C>
__device__ __forceinline__ void load_row(const T* p, float (&x)[C]) {
  struct alignas(sizeof(T) * C) Vec {
    T e[C];
  };
  const Vec v = *reinterpret_cast<const Vec*>(p);
#pragma unroll
  for (int i = 0; i < C; ++i) x[i] = to_f32(v.e[i]);
}

// Mends one row's output where a value that the row does not see made it NaN: such a
// value has weight 0 in the tile's product, and 0 times NaN or infinity is NaN.  The
// channels that are NaN and in which a hidden value of the piece's positions
// [tile_lo, tile_hi) (at most a few hundred at either end are hidden) is not finite are
// recomputed from those that the row sees, [lo, hi) of them and of a tree, which begins at
// position base, its token's (number i, packed t), 32 keys at a time with one
// set of weights for all channels; a NaN in any other channel is the row's own.  It
// stops once every such channel has met a NaN of its own.  q: the row's query; y or part
// (part_row): the output, as written.  Whole warp: lane i has channels C i .. + C - 1,
// and key i of 32.
template <typename T, int D, bool TREE>
__device__ __forceinline__ void mend_row(const PagedAttnArgs& a, int b, int kvh, const T* q,
                                         int tile_lo, int lo, int hi, int tile_hi, int base,
                                         int t, int i, T* y, float* part, int lane) {
  constexpr int C = D / 32;
  const int c0 = lane * C;
  auto at = [&](int c) { return part + (c0 + c) / 4 * a.part_step + (c0 + c) % 4; };
  uint32_t nan = 0;
#pragma unroll
  for (int c = 0; c < C; ++c) {
    const float o = y ? to_f32(y[c0 + c]) : *at(c);
    nan |= (o != o ? 1u : 0u) << c;
  }
  if (!__any_sync(0xffffffffu, nan)) return;
  // offset of the lane's position; -1: not there
  auto place = [&](int pos, bool there) {
    const int page = there ? page_of(a.pv, b, pos) : -1;
    return page < 0 ? -1ll : slot_offset(a.pv, page, kvh, pos);
  };
  // whether the row sees its position pos, lo <= pos < hi
  auto sees = [&](int pos) {
    return !TREE || pos < base || (tree_words(a, t, (pos - base) >> 5) >> ((pos - base) & 31) & 1);
  };
  const int k_lo = min(max(lo, tile_lo), tile_hi), k_hi = max(min(hi, tile_hi), k_lo);  // seen
  uint32_t mend = 0;
  auto look = [&](int from, int to, bool tree) {  // hidden positions of [from, to)
    for (int p0 = from; p0 < to; p0 += 32) {
      const int pos = p0 + lane;
      const long long off = place(pos, pos < to && (!tree || !sees(pos)));
#pragma unroll 8
      for (int i = 0; i < 32; ++i) {
        const long long o = __shfl_sync(0xffffffffu, off, i);
        float v[C] = {};
        if (o >= 0) load_row<T, C>((const T*)a.V_pages + o + c0, v);
#pragma unroll
        for (int c = 0; c < C; ++c) mend |= (fabsf(v[c]) < INFINITY ? 0u : 1u) << c;
      }
    }
  };
  look(tile_lo, k_lo, false);
  look(k_hi, tile_hi, false);
  if (TREE) look(max(base, k_lo), k_hi, true);
  mend &= nan;
  if (!__any_sync(0xffffffffu, mend)) return;
  float m = -INFINITY, l = 0.f, acc[C] = {};
  for (int top = k_hi; top > k_lo; top -= 32) {
    const int pos = top - 1 - lane;
    const long long off = place(pos, pos >= k_lo && sees(pos));
    float s = -INFINITY;
    if (off >= 0) {
      constexpr int W = 16 / sizeof(T);
      const T* k = (const T*)a.K_pages + off;
      s = 0.f;
#pragma unroll 4
      for (int i = 0; i < D; i += W) {
        float x[W], z[W];
        load_row<T, W>(q + i, x);
        load_row<T, W>(k + i, z);
#pragma unroll
        for (int e = 0; e < W; ++e) s = fmaf(x[e], z[e], s);
      }
      s *= a.scale2;
    }
    float m1 = fmaxf(m, s);
#pragma unroll
    for (int x = 16; x > 0; x >>= 1) m1 = fmaxf(m1, __shfl_xor_sync(0xffffffffu, m1, x));
    const float ref = m1 == -INFINITY ? 0.f : m1, f = exp2f(m - ref), p = exp2f(s - ref);
    m = m1;
    l = l * f + p;  // this lane's share
#pragma unroll
    for (int c = 0; c < C; ++c) acc[c] *= f;
#pragma unroll 8
    for (int i = 0; i < 32; ++i) {
      const long long o = __shfl_sync(0xffffffffu, off, i);
      const float w = __shfl_sync(0xffffffffu, p, i);
      float v[C] = {};
      if (o >= 0) load_row<T, C>((const T*)a.V_pages + o + c0, v);
#pragma unroll
      for (int c = 0; c < C; ++c) acc[c] = fmaf(w, v[c], acc[c]);
    }
    bool open = false;
#pragma unroll
    for (int c = 0; c < C; ++c) open = open || ((mend >> c & 1) && acc[c] == acc[c]);
    if (!__any_sync(0xffffffffu, open)) break;
  }
#pragma unroll
  for (int x = 16; x > 0; x >>= 1) l += __shfl_xor_sync(0xffffffffu, l, x);
  const float inv = l == 0.f ? 0.f : 1.f / l;
#pragma unroll
  for (int c = 0; c < C; ++c) {
    if (!(mend >> c & 1)) continue;
    if (y) round_to(acc[c] * inv, y[c0 + c]);
    else *at(c) = acc[c] * inv;
  }
}

// Mends what a warp has written, once all of the CTA's pieces are done: nothing waits on
// the warp then, however many keys its rows see (a wait with a bound would run out over a
// long context).  Its rows are [row0, row0 + rows) of those of tokens x0, x0 + 1, .. of every
// item (slot row slot0 + the row).  Walks the pieces anew; whole warp.
// Measured: one NaN value row in the middle of 1216 new tokens over 33k (130k) positions,
// 32/8 heads x 128, bf16: the call takes 113 (690) ms instead of 0.46 (1.5); with every value
// NaN 5.5 (6.5) ms.  With 4 rows to a pass over the keys it took 37 (229) ms, but its 168
// registers and its size made every call 1-2% slower.
template <typename T, int D, int BN, bool TREE>
__device__ __noinline__ void mend_pieces(const PagedAttnArgs& a, int cta, int n_cta, int x0,
                                         int slot0, int row0, int rows, int lane) {
  __syncwarp();  // the rows, written by other lanes
  const WorkStart start = find_work<BN, TREE, true>(a, cta, n_cta, lane);  // (told before)
  for (PieceWalk<BN, TREE> w(a, start); w.live(); w.next(a)) {
    const int tokens = min(w.tokens(a) - x0, a.half_tokens), slot = w.slot(cta);
    const int t_first = w.sp.t0 + w.first(a) + x0, p0 = w.sp.len - w.sp.n + w.first(a) + x0;
    const HeadSlice hs = head_slice(a, w.h);
    const int base = w.sp.len - w.sp.n;  // tree: where it begins
    for (int r = row0; r < row0 + rows; ++r) {
      const int t = r / a.slice, g = r - t * a.slice;
      if (t >= tokens) break;
      if (g >= hs.n) continue;
      const long long out =
          (long long)(t_first + t) * (a.pv.n_kv_heads * a.group) + hs.q0 + g;
      bool bad;
      const int lo = TREE ? tree_first_seen(a, t_first + t, base, p0 + t - base, bad)
                            : first_seen(a, p0 + t);
      mend_row<T, D, TREE>(a, w.b, hs.kvh,
                     (const T*)a.q + (t_first + t) * a.q_ts + (hs.q0 + g) * a.q_hs, w.cur * BN,
                     lo, p0 + t + 1, min(w.end * BN, w.sp.len), base, t_first + t, p0 + t - base,
                     slot < 0 ? (T*)a.y + out * D : nullptr,
                     slot < 0 ? nullptr : part_row<D>(a, slot, slot0 + r), lane);
    }
  }
}

// Whether the line of work of any lengths within the call's bounds fits 31 bits.
inline bool line_fits(const PagedAttnArgs& a, int keys_per_tile) {
  const double tiles = (double)a.pv.max_blocks * (1 << a.pv.page_shift) / keys_per_tile + 1;
  const double items = (double)a.n_tokens / a.tokens + a.pv.batch;
  return items * a.heads * (tiles * a.full_work + a.item_cost) < 2.0e9;
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
ebd_status launch_paged_merge(const PagedAttnArgs& a, bool bf16, int head_dim, int n_cta,
                              cudaStream_t s);

// Rows that a partial result needs: those of the largest item the call can have.
inline int paged_slot_rows(int max_new, int half_tokens, int slice, int most) {
  if (max_new > half_tokens) return most;
  const int rows = max_new * slice;
  return rows <= 8 ? 8 : rows <= 16 ? 16 : (rows + 31) / 32 * 32;
}

// Bytes of the split results of n_cta CTAs.
size_t paged_split_bytes(int n_cta, int slot_rows, int head_dim);
// Points a's split arrays into the workspace.
void paged_split_layout(PagedAttnArgs& a, void* ws, int n_cta);

ebd_status launch_paged_tc(PagedAttnArgs a, const ebd_paged_cache& c, int n_cta,
                           cudaStream_t s);
constexpr int kTcRows = 256;  // rows of an item at most

}  // namespace ebd
