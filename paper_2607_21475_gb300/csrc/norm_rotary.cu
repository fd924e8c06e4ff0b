// Norms of queries and keys per head with the rotation to their positions in the same
// pass, the gradient of that, and the append of new keys and values to a paged cache
// with both on the way.
//
// A row x (one head of one token, d channels) becomes
//   y = R_p(w * x r),   r = (mean x^2 + eps)^(-1/2),
// w the norm's weight (one for all heads or one per head), R_p the rotation of
// rotary.cu; float32 arithmetic, one rounding.  With u = R_p^T dy (the rotation being
// linear, its transpose is the inverse turn), g = u w and z = x r the gradient is
//   dx = r (g - z mean(g z)),   dw = sum of u z over the rows that share w.
//
// Both directions move rows (forward 2, backward 3 per row), so HBM bounds them at large
// sizes, a launch and a chain of loads at small ones; in between it is their instructions,
// which is why the arithmetic is in packed pairs, the weight is multiplied into the turn's
// factors once a token, and whole turning heads of 64, 128 and 256 channels have forms of
// their own that ask nothing about a lane's chunks (16k tokens x 28 heads x 128, bf16: 413
// instructions per warp and 4 rows and 54 us at first, 203 and 39 us now).  A row is shared
// by L lanes, L a power of two, each with U pairs of chunks that turn together, so that a
// row's sums are log2 L shuffles; a warp takes 32 / L heads of a token at a time and has
// three steps' rows on their way through shared memory.  The backward pass has an even share
// of all steps per warp, and its rows are asked for from token to token; the weight's
// gradient is summed per lane, per warp, per block and over the blocks, in that fixed order.
// Measured, bf16, 28 heads x 128: 16384 tokens 38.8 us, 6.3 TB/s (93% of the measured copy
// peak); gradient of 8192 tokens 34.6 us, 5.2 TB/s (77%: instructions, 57% of the issue
// slots, and 16 warps per SM, 128 registers each); 8 ragged chunks of 9.4k tokens in all
// appended (28/4 heads) 37.1 us, 4.8 TB/s; append step of 32 sequences (32/8 heads) 3.3 us.
// All are programmatic dependents of what precedes them on the stream.
#include <cuda_runtime.h>
#include <float.h>
#include <math.h>

#include <type_traits>

#include "common.cuh"
#include "decode_tile.cuh"
#include "internal.h"
#include "paged.cuh"
#include "paged_attn.cuh"
#include "ptx.cuh"
#include "rotary.cuh"

namespace ebd {

constexpr int kNormWarps = 8;
// resident blocks of 256 threads (prompt of 16k tokens: 4 blocks, with spills, 46 us against
// 39 with 3; ragged chunks appended: 3 blocks 38.6 us against 37.6 with 2)
constexpr int kNormBlocks = 3, kAppendNormBlocks = 2, kNormBackBlocks = 2;
constexpr int kNormMaxDim = 512;
// (fewer where a lane holds several pairs of a row: its arrays would spill)
constexpr int norm_blocks(int blocks, int u, int vec) {
  return u > 1 && u * vec >= 8 ? blocks - 1 : blocks;
}

// A norm's weight: element (head h, channel c) at h * hs + c.
struct NormWeight {
  const void* p;  // null: the rows are not normalised
  long long hs;   // 0: one for all heads
  bool f32;       // float32, otherwise bf16
  bool wide;      // rows on 16-byte boundaries
};

struct NormArgs {
  Rows x, y;             // rows and their destination (backward: x and dx)
  Rows dy;               // backward
  Rows k, v;             // append
  void *K_pages, *V_pages;
  PagedView pv;
  const int32_t* cu;         // append by offsets [batch + 1]
  const int64_t* slots;      // append by slots [n_tokens]
  const int32_t* positions;  // [n_tokens]; nullable where cu gives them
  const float2* table;       // [n_pos, rot / 2]; null: no rotation
  NormWeight wx, wk;
  int n_pos;
  int n_tokens, n_x, n_kv;   // heads of x; kv heads (append)
  int head_dim;
  int units, rot_units, half_off, rot;  // as in the rotation: pairs of chunks of a row
  int lanes;                 // L
  int parts;                 // warps per token
  float eps, inv_d;
  bool wide_table;
  int32_t* dev_status;
};

// Packed float32 pairs: two operations to an instruction (the passes would be bound by
// their instructions otherwise).
__device__ __forceinline__ float2 both(float x) { return make_float2(x, x); }

// A lane's part of a row, 2 VEC channels: lo[i] and hi[i] turn together.  Half layout: the
// unit's first and second chunk; pairs layout: the even and odd channels of both.
template <int VEC>
struct Part {
  float lo[VEC], hi[VEC];
};

template <typename T, int VEC, bool PAIRS>
__device__ __forceinline__ void widen(const Piece<T, VEC>& r, Part<VEC>& x) {
#pragma unroll
  for (int i = 0; i < VEC; ++i) {
    if (!PAIRS) {
      x.lo[i] = to_f32(r.a.e[i]);
      x.hi[i] = to_f32(r.b.e[i]);
    } else {
      const Chunk<T, VEC>& c = i < VEC / 2 ? r.a : r.b;
      x.lo[i] = to_f32(c.e[2 * i % VEC]);
      x.hi[i] = to_f32(c.e[2 * i % VEC + 1]);
    }
  }
}
// Two neighbouring elements from float32.
__device__ __forceinline__ void from_f32x2(float x, float y, float& a, float& b) { a = x, b = y; }
__device__ __forceinline__ void from_f32x2(float x, float y, __nv_bfloat16& a, __nv_bfloat16& b) {
  const __nv_bfloat162 v = __floats2bfloat162_rn(x, y);
  a = v.x;
  b = v.y;
}
template <typename T, int VEC, bool PAIRS>
__device__ __forceinline__ void narrow(const Part<VEC>& x, Piece<T, VEC>& r) {
  if constexpr (VEC == 1) {
    from_f32(x.lo[0], r.a.e[0]);
    from_f32(x.hi[0], r.b.e[0]);
  } else {
#pragma unroll
    for (int i = 0; i < VEC; i += 2) {
      if (!PAIRS) {
        from_f32x2(x.lo[i], x.lo[i + 1], r.a.e[i], r.a.e[i + 1]);
        from_f32x2(x.hi[i], x.hi[i + 1], r.b.e[i], r.b.e[i + 1]);
      } else {
        from_f32x2(x.lo[i / 2], x.hi[i / 2], r.a.e[i], r.a.e[i + 1]);
        from_f32x2(x.lo[(VEC + i) / 2], x.hi[(VEC + i) / 2], r.b.e[i], r.b.e[i + 1]);
      }
    }
  }
}

// f(i, lo pair i, hi pair i) for every two of a part's pairs of channels, packed; VEC = 1:
// one in a pair's first half.
template <int VEC, typename F>
__device__ __forceinline__ void each_two(Part<VEC>& x, F f) {
  if constexpr (VEC == 1) {
    float2 lo = make_float2(x.lo[0], 0.f), hi = make_float2(x.hi[0], 0.f);
    f(0, lo, hi);
    x.lo[0] = lo.x;
    x.hi[0] = hi.x;
  } else {
#pragma unroll
    for (int i = 0; i < VEC; i += 2) {
      float2 lo = make_float2(x.lo[i], x.lo[i + 1]), hi = make_float2(x.hi[i], x.hi[i + 1]);
      f(i, lo, hi);
      x.lo[i] = lo.x, x.lo[i + 1] = lo.y;
      x.hi[i] = hi.x, x.hi[i + 1] = hi.y;
    }
  }
}
template <int VEC>
__device__ __forceinline__ float2 two(const float (&v)[VEC], int i) {
  if constexpr (VEC == 1) return make_float2(v[0], 0.f);
  else return make_float2(v[i], v[i + 1]);
}

// Cosines and sines of a unit's pairs.
template <int VEC>
struct Angles {
  float c[VEC], s[VEC];
};

// A lane's place in a row: U units, the j-th of them with chunks at channels c1, c2 = c1 +
// gap.  FL > 0: rows of FL lanes, each with one unit of two chunks that turn.
template <int VEC, bool PAIRS, int U, int FL>
struct Place {
  static constexpr bool kFull = FL > 0;
  int lanes, sub;
  int c1[U], c2[U];  // -1: the row has none
  bool turns[U], all[U];  // the unit does; its second chunk too (pairs layout)
  __device__ __forceinline__ Place(const NormArgs& a, int lane)
      : lanes(kFull ? FL : a.lanes), sub(lane & (lanes - 1)) {
#pragma unroll
    for (int j = 0; j < U; ++j) {
      const int u = sub + lanes * j;
      if (kFull) {
        c1[j] = PAIRS ? 2 * VEC * sub : VEC * sub;
        c2[j] = c1[j] + (PAIRS ? VEC : VEC * FL);
        turns[j] = all[j] = true;
      } else {
        c1[j] = c2[j] = -1;
        if (u < a.units) unit_channels<VEC, PAIRS>(a, u, c1[j], c2[j]);
        turns[j] = u < a.rot_units;
        all[j] = !PAIRS || (c2[j] >= 0 && c2[j] < a.rot);
      }
    }
  }
  __device__ __forceinline__ int per_warp() const { return 32 / lanes; }
  __device__ __forceinline__ bool first(int j) const { return kFull || c1[j] >= 0; }
  __device__ __forceinline__ bool second(int j) const { return kFull || c2[j] >= 0; }
  __device__ __forceinline__ bool turn(int j) const { return kFull || turns[j]; }
  __device__ __forceinline__ bool turn_all(int j) const { return kFull || all[j]; }
  // Sum over the lanes that share a row.
  __device__ __forceinline__ float row_sum(float v) const {
#pragma unroll
    for (int o = 1; o < (kFull ? FL : 32); o <<= 1) {
      const float u = __shfl_xor_sync(0xffffffffu, v, o);
      if (kFull || o < lanes) v += u;
    }
    return v;
  }
};

// The unit's pairs that turn: none, the first chunk's (pairs layout), all.
template <int VEC, bool PAIRS>
__device__ __forceinline__ void turn(const Angles<VEC>& t, bool all, float sign, Part<VEC>& x) {
  each_two<VEC>(x, [&](int i, float2& lo, float2& hi) {
    float2 c = two(t.c, i), s = two(t.s, i);
    s.x *= sign, s.y *= sign;
    const float2 ns = make_float2(-s.x, -s.y);
    // VEC = 2 in the pairs layout: one pair of each chunk
    const float2 lo1 = __ffma2_rn(lo, c, __fmul2_rn(hi, ns));
    const float2 hi1 = __ffma2_rn(lo, s, __fmul2_rn(hi, c));
    if (PAIRS && VEC == 2) {
      lo.x = lo1.x, hi.x = hi1.x;
      if (all) lo.y = lo1.y, hi.y = hi1.y;
    } else if (all || i < VEC / 2) {
      lo = lo1, hi = hi1;
    }
  });
}

template <int VEC, bool PAIRS>
__device__ __forceinline__ void load_angles(const NormArgs& a, int tpos, int u, Angles<VEC>& t) {
  const float2* row = a.table + (size_t)tpos * (a.rot / 2) + u * VEC;
  const int n = PAIRS ? min(VEC, a.rot / 2 - u * VEC) : VEC;
  if (VEC % 2 == 0 && a.wide_table) {
#pragma unroll
    for (int i = 0; i + 1 < VEC; i += 2) {
      if (PAIRS && i >= n) break;
      const float4 f = __ldg(reinterpret_cast<const float4*>(row + i));
      t.c[i] = f.x, t.s[i] = f.y;
      t.c[i + 1] = f.z, t.s[i + 1] = f.w;
    }
  } else {
#pragma unroll
    for (int i = 0; i < VEC; ++i) {
      if (PAIRS && i >= n) break;
      const float2 f = __ldg(row + i);
      t.c[i] = f.x, t.s[i] = f.y;
    }
  }
}

// A unit's turn with the weight in it: lo' = ll lo + lh hi, hi' = hl lo + hh hi, in the order
// of the plain rotation's roundings (without a weight the two agree bit for bit).
template <int VEC>
struct Factors {
  float ll[VEC], lh[VEC], hl[VEC], hh[VEC];

  __device__ __forceinline__ void set(const Angles<VEC>& t, const Part<VEC>& w, bool turns) {
#pragma unroll
    for (int i = 0; i < VEC; ++i) {
      ll[i] = turns ? t.c[i] * w.lo[i] : w.lo[i];
      lh[i] = -t.s[i] * w.hi[i];
      hl[i] = t.s[i] * w.lo[i];
      hh[i] = turns ? t.c[i] * w.hi[i] : w.hi[i];
    }
  }
  // (a chunk that stays beside one that turns, pairs layout: its factors are the weight)
  __device__ __forceinline__ void second_stays(const Part<VEC>& w) {
#pragma unroll
    for (int i = VEC / 2; i < VEC; ++i) ll[i] = w.lo[i], hh[i] = w.hi[i];
  }
  // turns: the unit does; all: its second chunk too (pairs layout).
  template <bool PAIRS>
  __device__ __forceinline__ void turn(bool turns, bool all, float by, Part<VEC>& x) const {
    const float2 by2 = both(by);
    if (!turns) {
      each_two<VEC>(x, [&](int i, float2& lo, float2& hi) {
        lo = __fmul2_rn(__fmul2_rn(lo, two(ll, i)), by2);
        hi = __fmul2_rn(__fmul2_rn(hi, two(hh, i)), by2);
      });
      return;
    }
    each_two<VEC>(x, [&](int i, float2& lo, float2& hi) {
      const float2 h = __fmul2_rn(hi, two(hh, i));
      float2 l1 = __ffma2_rn(lo, two(ll, i), __fmul2_rn(hi, two(lh, i)));
      float2 h1 = __ffma2_rn(lo, two(hl, i), h);
      if (PAIRS && !all && i >= VEC / 2) l1 = __fmul2_rn(lo, two(ll, i)), h1 = h;
      if (PAIRS && !all && VEC == 2) {  // one pair of each chunk
        l1.y = lo.y * ll[1];
        h1.y = h.y;
      }
      lo = __fmul2_rn(l1, by2);
      hi = __fmul2_rn(h1, by2);
    });
  }
};

// The weight of a unit's channels in a head.
template <typename T, int VEC, bool PAIRS>
__device__ __forceinline__ void load_weight(const NormWeight& w, int h, int c1, int c2,
                                            Part<VEC>& out) {
  if (c1 < 0) return;
  auto load = [&](auto piece) {
    using P = decltype(piece);
    using Elem = std::remove_reference_t<decltype(piece.a.e[0])>;
    const Elem* p = (const Elem*)w.p + h * w.hs;
    auto chunk = [&](int c, auto& to) {
      constexpr int kBytes = VEC * sizeof(Elem);
      if (kBytes % 16 == 0 && w.wide) {
#pragma unroll
        for (int i = 0; i < kBytes / 16; ++i)
          reinterpret_cast<uint4*>(&to)[i] = __ldg(reinterpret_cast<const uint4*>(p + c) + i);
      } else {
#pragma unroll
        for (int i = 0; i < VEC; ++i) to.e[i] = p[c + i];
      }
    };
    P r = piece;
    chunk(c1, r.a);
    if (c2 >= 0) chunk(c2, r.b);
    widen<Elem, VEC, PAIRS>(r, out);
  };
  if (w.f32) load(Piece<float, VEC>{});
  else load(Piece<__nv_bfloat16, VEC>{});
}

// 2^-64: rows whose sum of squares leaves float32's range are scaled by it first.
constexpr float kRowScale = 5.421010862427522e-20f;

// Rows on their way to a warp, N of them to a step (the backward pass: x and dy): kAhead
// steps are asked for ahead.  Wide chunks wait in shared memory, where their number costs
// no registers; every lane reads back what it asked for, so nothing is synchronised.
// Elements and pairs wait in registers, one step ahead.
template <typename T, int VEC, int U, int N>
struct RowRing {
  static constexpr bool kShared = VEC * sizeof(T) == 16;
  static constexpr int kStages = U == 1 ? 4 : 2;
  static constexpr int kAhead = kShared ? kStages - 1 : 1;
  static constexpr int kBytes = kShared ? kNormWarps * kStages * N * U * 2 * 512 : 0;
  static constexpr int kStageBytes = N * U * 2 * 512;
  unsigned char* base;     // this lane's part of the warp's first stage
  int in = 0, out = 0;     // stages' offsets
  Piece<T, VEC> next[kShared ? 1 : 2][N][U];  // (by elements)

  // smem: kBytes for the block
  __device__ __forceinline__ explicit RowRing(void* smem)
      : base((unsigned char*)smem + (threadIdx.x >> 5) * kStages * kStageBytes +
             (threadIdx.x & 31) * 16) {}
  // src: the rows, if there are any
  template <typename P>
  __device__ __forceinline__ void fetch(const P& place, const T* const (&src)[N], bool any) {
#pragma unroll
    for (int n = 0; n < N; ++n) {
#pragma unroll
      for (int j = 0; j < U; ++j) {
        if constexpr (kShared) {
          unsigned char* to = base + in + (n * U + j) * 1024;
          if (any && place.first(j)) cp_async16(to, src[n] + place.c1[j]);
          if (any && place.second(j)) cp_async16(to + 512, src[n] + place.c2[j]);
        } else {
          next[0][n][j] = next[1][n][j];
          if (!any) continue;
          if (place.first(j)) load_chunk<T, VEC>(src[n] + place.c1[j], next[1][n][j].a);
          if (place.second(j)) load_chunk<T, VEC>(src[n] + place.c2[j], next[1][n][j].b);
        }
      }
    }
    if constexpr (kShared) {
      cp_async_commit();
      in = in + kStageBytes == kStages * kStageBytes ? 0 : in + kStageBytes;
    }
  }
  // The step fetched kAhead fetches ago; zeros where a row has no chunk.
  template <typename P>
  __device__ __forceinline__ void take(const P& place, Piece<T, VEC> (&r)[N][U]) {
    if constexpr (kShared) cp_async_wait<kAhead>();
#pragma unroll
    for (int n = 0; n < N; ++n)
#pragma unroll
      for (int j = 0; j < U; ++j) {
        if constexpr (kShared) {
          const unsigned char* from = base + out + (n * U + j) * 1024;
          uint4 v = *reinterpret_cast<const uint4*>(from);
          uint4 w = *reinterpret_cast<const uint4*>(from + 512);
          if (!place.first(j)) v = make_uint4(0, 0, 0, 0);
          if (!place.second(j)) w = make_uint4(0, 0, 0, 0);
          *reinterpret_cast<uint4*>(&r[n][j].a) = v;
          *reinterpret_cast<uint4*>(&r[n][j].b) = w;
        } else {
          r[n][j] = next[0][n][j];
#pragma unroll
          for (int i = 0; i < VEC; ++i) {
            if (!place.first(j)) from_f32(0.f, r[n][j].a.e[i]);
            if (!place.second(j)) from_f32(0.f, r[n][j].b.e[i]);
          }
        }
      }
    if constexpr (kShared) out = out + kStageBytes == kStages * kStageBytes ? 0 : out + kStageBytes;
  }
  __device__ __forceinline__ void drain() {
    if constexpr (kShared) cp_async_wait<0>();
  }
};

template <typename T, int VEC, bool PAIRS, bool APPEND, int U, int FL>
__global__ void __launch_bounds__(kNormWarps * 32, norm_blocks(APPEND ? kAppendNormBlocks : kNormBlocks, U, VEC))
    norm_rotary_kernel(const NormArgs a) {
  using Ring = RowRing<T, VEC, U, 1>;
  __shared__ uint4 ring_s[Ring::kBytes / 16 + 1];
  const int lane = threadIdx.x & 31;
  grid_launch_dependents();
  grid_dependency_wait();
  const long long w = (long long)blockIdx.x * kNormWarps + (threadIdx.x >> 5);
  const int t = a.parts == 1 ? (int)w : (int)(w / a.parts), part = (int)(w - (long long)t * a.parts);
  if (t >= a.n_tokens) return;
  const int heads = a.n_x + (APPEND ? 2 * a.n_kv : 0);
  const Place<VEC, PAIRS, U, FL> place(a, lane);
  const int sub = place.sub, g = lane / place.lanes, step = place.per_warp() * a.parts;
  int hb = part * place.per_warp();  // first head of the warp's step
  const T* xp = (const T*)a.x.p + t * a.x.ts;
  const T* kp = (const T*)a.k.p + t * a.k.ts;
  const T* vp = (const T*)a.v.p + t * a.v.ts;
  Ring ring(ring_s);
  int hf = hb + g;  // the next head to fetch, and (not append) its row
  const T* xf = xp + hf * a.x.hs;
  const long long x_step = step * a.x.hs;
  auto fetch = [&]() {
    const T* p = xf;
    if (APPEND)
      p = hf < a.n_x         ? xp + hf * a.x.hs
          : hf < a.n_x + a.n_kv ? kp + (hf - a.n_x) * a.k.hs
                                : vp + (hf - a.n_x - a.n_kv) * a.v.hs;
    const T* const src[1] = {p};
    ring.fetch(place, src, hf < heads);
    hf += step;
    xf += x_step;
  };
#pragma unroll
  for (int k = 0; k < Ring::kAhead; ++k) fetch();

  int pos = 0, page = -1;
  long long at = -1;  // the token's row of head 0 in the pools
  if (APPEND && a.slots) {
    const int64_t slot = a.slots[t];
    if (slot == -1) {  // no token here
      ring.drain();
      return;
    }
    pos = a.positions ? a.positions[t] : 0;
    const int64_t page64 = slot >> a.pv.page_shift;
    if (slot >= 0 && page64 < a.pv.n_pages) {
      page = (int)page64;
      at = slot_offset(a.pv, page, 0, (int)(slot & ((1 << a.pv.page_shift) - 1)));
    }
  } else if (APPEND) {
    // the offsets run from 0 to n_tokens; the first token's warp looks at both ends
    const int c_first = t == 0 ? a.cu[0] : 0, c_last = t == 0 ? a.cu[a.pv.batch] : a.n_tokens;
    bool odd;
    const int b = sequence_of(a.cu, a.pv.batch, t, lane, odd);
    bool none = b >= a.pv.batch;  // no sequence's token: no place for it
    int c0 = 0, c1 = 0, len = 0;
    if (!none) c0 = a.cu[b], c1 = a.cu[b + 1], len = a.pv.seq_len[b];
    none |= t < c0;
    odd |= none | (c_first != 0) | (c_last != a.n_tokens);
    if (lane == 0 && odd) raise_status(a.dev_status, EBD_DEV_RANGE);
    if (none) {
      ring.drain();
      return;
    }
    pos = len - (min(c1, a.n_tokens) - t);
    page = page_of(a.pv, b, pos);
    if (page >= 0) at = slot_offset(a.pv, page, 0, pos);
    if (a.positions) pos = a.positions[t];
  } else if (a.positions) {
    pos = a.positions[t];
  }
  const int tpos = a.table ? min(max(pos, 0), a.n_pos - 1) : 0;
  // 0: x, 1: keys, 2: values
  auto set_of = [&](int h) { return !APPEND || h < a.n_x ? 0 : h < a.n_x + a.n_kv ? 1 : 2; };
  Factors<VEC> f[U];
  int held = -1;  // the set whose factors are in f
  auto load_factors = [&](int h, int set) {
    const NormWeight& w = set == 0 ? a.wx : a.wk;
    if (set > 1 || (held == set && w.hs == 0)) return;
    held = set;
#pragma unroll
    for (int j = 0; j < U; ++j) {
      Angles<VEC> t;
      if (place.turn(j)) load_angles<VEC, PAIRS>(a, tpos, sub + place.lanes * j, t);
      Part<VEC> wt;
#pragma unroll
      for (int i = 0; i < VEC; ++i) wt.lo[i] = wt.hi[i] = 1.f;
      if (w.p)
        load_weight<T, VEC, PAIRS>(w, set == 0 ? h : h - a.n_x, place.c1[j], place.c2[j], wt);
      f[j].set(t, wt, place.turn(j));
      if (PAIRS && !place.turn_all(j)) f[j].second_stays(wt);
    }
  };
  if (hb + g < heads) load_factors(hb + g, set_of(hb + g));
  if (lane == 0 && ((APPEND && page < 0) || (a.table && tpos != pos)))
    raise_status(a.dev_status, EBD_DEV_RANGE);
  T* yp = (T*)a.y.p + t * a.y.ts;
  T* yh = yp + (hb + g) * a.y.hs;  // (not append) the step's row
  const long long y_step = step * a.y.hs;

  for (; hb < heads; hb += step, yh += y_step) {
    fetch();
    Piece<T, VEC> r[1][U];
    ring.take(place, r);
    const int h = hb + g, set = set_of(h);
    const bool live = h < heads;
    Part<VEC> x[U];
#pragma unroll
    for (int j = 0; j < U; ++j) widen<T, VEC, PAIRS>(r[0][j], x[j]);
    auto squares = [&]() {
      float2 s0 = make_float2(0.f, 0.f), s1 = s0;
#pragma unroll
      for (int j = 0; j < U; ++j)
        each_two<VEC>(x[j], [&](int, float2& lo, float2& hi) {
          s0 = __ffma2_rn(lo, lo, s0);
          s1 = __ffma2_rn(hi, hi, s1);
        });
      const float2 s = __fadd2_rn(s0, s1);
      return place.row_sum(live ? s.x + s.y : 0.f);
    };
    float ss = squares(), eps = a.eps;
    const bool normed = live && set < 2 && (set == 0 ? a.wx.p : a.wk.p) != nullptr;
    if (__any_sync(0xffffffffu, normed && !(ss < INFINITY))) {
      if (normed && !(ss < INFINITY)) {
        eps = 0.f;  // below the sum's rounding
#pragma unroll
        for (int j = 0; j < U; ++j)
#pragma unroll
          for (int i = 0; i < VEC; ++i) x[j].lo[i] *= kRowScale, x[j].hi[i] *= kRowScale;
      }
      ss = squares();
    }
    if (!live) continue;
    T* dst;
    if (!APPEND) {
      dst = yh;
    } else if (set == 0) {
      dst = yp + h * a.y.hs;
    } else {
      if (at < 0) continue;
      const int kh = h - a.n_x - (set == 2 ? a.n_kv : 0);
      dst = (T*)(set == 2 ? a.V_pages : a.K_pages) + at + kh * a.pv.head_stride;
    }
    if (set < 2) {
      load_factors(h, set);
      const float inv = normed ? __frsqrt_rn(fmaf(ss, a.inv_d, eps)) : 1.f;
#pragma unroll
      for (int j = 0; j < U; ++j) {
        f[j].template turn<PAIRS>(place.turn(j), place.turn_all(j), inv, x[j]);
        narrow<T, VEC, PAIRS>(x[j], r[0][j]);
      }
    }
#pragma unroll
    for (int j = 0; j < U; ++j) {
      if (place.first(j)) store_chunk<T, VEC>(dst + place.c1[j], r[0][j].a);
      if (place.second(j)) store_chunk<T, VEC>(dst + place.c2[j], r[0][j].b);
    }
  }
}

// PER_HEAD: a block has one head (blockIdx.y), a warp's groups of lanes have tokens; else
// they have heads of a token.  Leaves the block's sum of the weight's gradient in
// partial[blockIdx.x][blockIdx.y][d].
template <typename T, int VEC, bool PAIRS, int U, bool PER_HEAD, int FL>
__global__ void __launch_bounds__(kNormWarps * 32, norm_blocks(kNormBackBlocks, U, VEC))
    norm_backward_kernel(const NormArgs a, float* __restrict__ partial) {
  extern __shared__ __align__(16) unsigned char smem[];  // the rows' ring; then, in its place:
  float* red = reinterpret_cast<float*>(smem);           // [warps][units of all lanes][2 VEC]
  using Ring = RowRing<T, VEC, U, 2>;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const Place<VEC, PAIRS, U, FL> place(a, lane);
  const int L = place.lanes, sub = place.sub, per_warp = place.per_warp(), g = lane / L;
  grid_launch_dependents();  // the sum over blocks, which waits for this kernel's end
  grid_dependency_wait();
  Part<VEC> wt[U], acc[U];
#pragma unroll
  for (int j = 0; j < U; ++j) {
#pragma unroll
    for (int i = 0; i < VEC; ++i) wt[j].lo[i] = wt[j].hi[i] = acc[j].lo[i] = acc[j].hi[i] = 0.f;
    load_weight<T, VEC, PAIRS>(a.wx, PER_HEAD ? blockIdx.y : 0, place.c1[j], place.c2[j], wt[j]);
  }

  // Steps of the call: 32 / L heads of a token, or tokens of the block's head, one after
  // another; a warp has an even share of them, its rows asked for from token to token.
  const int per_token = PER_HEAD ? 1 : (a.n_x + per_warp - 1) / per_warp;
  const long long steps = PER_HEAD ? (a.n_tokens + per_warp - 1) / per_warp
                                   : (long long)a.n_tokens * per_token;
  const long long warps = (long long)gridDim.x * kNormWarps, w = (long long)warp * gridDim.x + blockIdx.x;
  const long long q0 = steps * w / warps, q1 = steps * (w + 1) / warps;
  struct At {
    int t, h;  // a step's token and head for these lanes
  };
  auto first_at = [&](long long q) {
    At p;
    p.t = PER_HEAD ? (int)q * per_warp + g : (int)(q / per_token);
    p.h = PER_HEAD ? blockIdx.y : (int)(q - (long long)p.t * per_token) * per_warp + g;
    return p;
  };
  auto next_at = [&](At& p) {
    if (PER_HEAD) {
      p.t += per_warp;
    } else if ((p.h += per_warp) - g >= a.n_x) {
      p.h = g;
      ++p.t;
    }
  };
  auto there = [&](const At& p) { return p.t < a.n_tokens && p.h < a.n_x; };
  Ring ring(smem);
  At ahead = first_at(q0);
  long long qf = q0;  // the next step to fetch
  auto fetch = [&]() {
    const T* const src[2] = {(const T*)a.x.p + ahead.t * a.x.ts + ahead.h * a.x.hs,
                             (const T*)a.dy.p + ahead.t * a.dy.ts + ahead.h * a.dy.hs};
    ring.fetch(place, src, qf < q1 && there(ahead));
    next_at(ahead);
    ++qf;
  };
#pragma unroll
  for (int k = 0; k < Ring::kAhead; ++k) fetch();
  At at = first_at(q0);
  Angles<VEC> angles[U];
  int token = -1;  // whose angles these are
  int pos = 0;     // position of the next token
  if (a.positions && q0 < q1 && at.t < a.n_tokens) pos = a.positions[at.t];
  for (long long q = q0; q < q1; ++q, next_at(at)) {
    if (at.t != token) {
      token = at.t;
      const int tpos = a.table ? min(max(pos, 0), a.n_pos - 1) : 0;
      if (there(at) && sub == 0 && a.table && tpos != pos)
        raise_status(a.dev_status, EBD_DEV_RANGE);
#pragma unroll
      for (int j = 0; j < U; ++j)
        if (place.turn(j)) load_angles<VEC, PAIRS>(a, tpos, sub + L * j, angles[j]);
      const int after = PER_HEAD ? token + per_warp : token + 1;
      if (a.positions && after < a.n_tokens) pos = a.positions[after];
    }
    fetch();
    Piece<T, VEC> r[2][U];
    ring.take(place, r);
    const bool live = there(at);
    Part<VEC> x[U], u[U];  // u: R^T dy
#pragma unroll
    for (int j = 0; j < U; ++j) {
      widen<T, VEC, PAIRS>(r[0][j], x[j]);
      widen<T, VEC, PAIRS>(r[1][j], u[j]);
      if (place.turn(j)) turn<VEC, PAIRS>(angles[j], place.turn_all(j), -1.f, u[j]);
    }
    float ss, gx;
    auto sums = [&]() {
      float2 s0 = make_float2(0.f, 0.f), s1 = s0;
#pragma unroll
      for (int j = 0; j < U; ++j)
        each_two<VEC>(x[j], [&](int i, float2& lo, float2& hi) {
          s0 = __ffma2_rn(lo, lo, s0);
          s0 = __ffma2_rn(hi, hi, s0);
          s1 = __ffma2_rn(__fmul2_rn(two(u[j].lo, i), two(wt[j].lo, i)), lo, s1);
          s1 = __ffma2_rn(__fmul2_rn(two(u[j].hi, i), two(wt[j].hi, i)), hi, s1);
        });
      ss = place.row_sum(live ? s0.x + s0.y : 0.f);
      gx = place.row_sum(live ? s1.x + s1.y : 0.f);
    };
    sums();
    float eps = a.eps, scale = 1.f;
    if (__any_sync(0xffffffffu, !(ss < INFINITY))) {
      if (!(ss < INFINITY)) {
        eps = 0.f;
        scale = kRowScale;
#pragma unroll
        for (int j = 0; j < U; ++j)
#pragma unroll
          for (int i = 0; i < VEC; ++i) x[j].lo[i] *= kRowScale, x[j].hi[i] *= kRowScale;
      }
      sums();
    }
    if (!live) continue;
    T* out = (T*)a.y.p + at.t * a.y.ts + at.h * a.y.hs;
    const float inv = __frsqrt_rn(fmaf(ss, a.inv_d, eps));
    const float2 inv2 = both(inv), back = both(inv * scale);
    const float2 mean = both(-gx * inv * a.inv_d * (inv * scale));  // -r mean of g z
#pragma unroll
    for (int j = 0; j < U; ++j) {
      each_two<VEC>(x[j], [&](int i, float2& lo, float2& hi) {
        const float2 z0 = __fmul2_rn(lo, inv2), z1 = __fmul2_rn(hi, inv2);
        const float2 u0 = two(u[j].lo, i), u1 = two(u[j].hi, i);
        const float2 a0 = __ffma2_rn(u0, z0, two(acc[j].lo, i));
        const float2 a1 = __ffma2_rn(u1, z1, two(acc[j].hi, i));
        acc[j].lo[i] = a0.x, acc[j].hi[i] = a1.x;
        if constexpr (VEC > 1) acc[j].lo[i + 1] = a0.y, acc[j].hi[i + 1] = a1.y;
        lo = __ffma2_rn(z0, mean, __fmul2_rn(__fmul2_rn(u0, two(wt[j].lo, i)), back));
        hi = __ffma2_rn(z1, mean, __fmul2_rn(__fmul2_rn(u1, two(wt[j].hi, i)), back));
      });
      narrow<T, VEC, PAIRS>(x[j], r[0][j]);
      if (place.first(j)) store_chunk<T, VEC>(out + place.c1[j], r[0][j].a);
      if (place.second(j)) store_chunk<T, VEC>(out + place.c2[j], r[0][j].b);
    }
  }

  // the block's sum, in a fixed order: lanes, then warps
  __syncthreads();
  const int wide = L * U * 2 * VEC;
#pragma unroll
  for (int j = 0; j < U; ++j)
#pragma unroll
    for (int i = 0; i < 2 * VEC; ++i) {
      float v = i < VEC ? acc[j].lo[i % VEC] : acc[j].hi[i % VEC];
      for (int o = L; o < 32; o <<= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
      if (g == 0) red[warp * wide + (sub + L * j) * 2 * VEC + i] = v;
    }
  __syncthreads();
  float* dst = partial + ((size_t)blockIdx.x * gridDim.y + blockIdx.y) * a.head_dim;
  for (int k = threadIdx.x; k < wide; k += kNormWarps * 32) {
    const int u = k / (2 * VEC), i = k - u * 2 * VEC, e = i % VEC;
    if (u >= a.units) continue;
    int c1, c2;
    unit_channels<VEC, PAIRS>(a, u, c1, c2);
    // lo[e] (i < VEC) and hi[e]: chunk and element
    const bool second = PAIRS ? e >= VEC / 2 : i >= VEC;
    if (second && c2 < 0) continue;
    const int c = (second ? c2 : c1) + (PAIRS ? 2 * e % VEC + (i >= VEC) : e);
    float v = 0.f;
#pragma unroll
    for (int x = 0; x < kNormWarps; ++x) v += red[x * wide + k];
    dst[c] = v;
  }
}

// dweight[i] = sum over the n blocks of partial[block][i], i < total; 32 columns per block,
// warp w sums the blocks w, w + 32, .., and the warps' sums are added in a fixed order.
constexpr int kReduceWarps = 32;
__global__ void __launch_bounds__(kReduceWarps * 32)
    norm_weight_reduce_kernel(const float* __restrict__ partial, int n, int total,
                              float* __restrict__ dweight) {
  __shared__ float s[kReduceWarps][33];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, i = blockIdx.x * 32 + lane;
  grid_launch_dependents();
  grid_dependency_wait();
  float v = 0.f;
  if (i < total) {
#pragma unroll 5
    for (int k = warp; k < n; k += kReduceWarps) v += partial[(size_t)k * total + i];
  }
  s[warp][lane] = v;
  __syncthreads();
  // warp w has columns w of the block: a lane per warp's sum
  const int col = blockIdx.x * 32 + warp;
  v = s[lane][warp];
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  if (lane == 0 && col < total) dweight[col] = v;
}

// Shape of a row's lanes for chunks of VEC elements; false: too many units.
template <int VEC>
static bool norm_shape(NormArgs& a, bool pairs, int max_u) {
  const int rot_chunks = a.rot / VEC, chunks = a.head_dim / VEC;
  a.half_off = a.rot / 2;
  a.rot_units = pairs ? (rot_chunks + 1) / 2 : rot_chunks / 2;
  a.units = pairs ? (chunks + 1) / 2 : a.rot_units + (chunks - rot_chunks + 1) / 2;
  a.wide_table = a.rot % 4 == 0 && (uintptr_t)a.table % 16 == 0;
  a.lanes = 1;
  while (a.lanes < 32 && a.lanes < a.units) a.lanes *= 2;
  return a.units <= a.lanes * max_u;
}

template <typename T, int VEC, bool PAIRS, bool APPEND, int U, int FL>
static ebd_status launch_norm_u(NormArgs a, cudaStream_t s) {
  const int heads = a.n_x + (APPEND ? 2 * a.n_kv : 0);
  // one row per lane while the call has fewer warps than the GPU holds (latency), up to
  // sixteen pairs of chunks per lane beyond that
  const int many = (heads * a.lanes + 31) / 32, few = (heads * a.lanes * U + 511) / 512;
  a.parts = (long long)a.n_tokens * many <= (long long)sm_count() * 32 ? many : few;
  const long long blocks = ((long long)a.n_tokens * a.parts + kNormWarps - 1) / kNormWarps;
  if (blocks > 0x7fffffffLL) return EBD_ERR_UNSUPPORTED;
  return launch_dependent(norm_rotary_kernel<T, VEC, PAIRS, APPEND, U, FL>, dim3((unsigned)blocks),
                          kNormWarps * 32, 0, s, a);
}

// Blocks of the backward pass along its rows (times the heads where each has a weight).
static int norm_back_blocks(long long steps, int heads) {
  const long long want = (steps + kNormWarps - 1) / kNormWarps;
  long long most = (long long)sm_count() * kNormBackBlocks / heads;
  if (most < 1) most = 1;
  return (int)(want < most ? want : most);
}

struct NormBackward {
  float *partial, *dweight;
};

template <typename T, int VEC, bool PAIRS, int U, int FL>
static ebd_status launch_norm_back_u(NormArgs a, const NormBackward& bw, cudaStream_t s) {
  const bool per_head = a.wx.hs != 0;
  const int per_warp = 32 / a.lanes;
  const long long steps = per_head ? (a.n_tokens + per_warp - 1) / per_warp
                                   : (long long)a.n_tokens * ((a.n_x + per_warp - 1) / per_warp);
  const int blocks = norm_back_blocks(steps, per_head ? a.n_x : 1);
  const int total = (per_head ? a.n_x : 1) * a.head_dim;
  const int sums = kNormWarps * a.lanes * U * 2 * VEC * 4, ring = RowRing<T, VEC, U, 2>::kBytes;
  const int smem = sums > ring ? sums : ring;
  const dim3 grid(blocks, per_head ? a.n_x : 1);
  auto kern = per_head ? norm_backward_kernel<T, VEC, PAIRS, U, true, FL>
                       : norm_backward_kernel<T, VEC, PAIRS, U, false, FL>;
  if (smem > 48 * 1024 &&
      cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, smem) != cudaSuccess)
    return EBD_ERR_CUDA;
  const ebd_status st = launch_dependent(kern, grid, kNormWarps * 32, smem, s, a, bw.partial);
  if (st != EBD_OK) return st;
  return launch_dependent(norm_weight_reduce_kernel, dim3((total + 31) / 32), kReduceWarps * 32, 0, s,
                          (const float*)bw.partial, blocks, total, bw.dweight);
}

// One launch for chunks of VEC elements: the pass and the units per lane, of which rows of
// 512 channels need at most 1 (bf16) or 2 (float32) in wide chunks, 8 by elements and 4 by
// pairs.
template <typename T, int VEC, bool PAIRS, bool APPEND>
static ebd_status launch_norm_v(NormArgs a, const NormBackward* bw, cudaStream_t s) {
  constexpr bool kWide = VEC * sizeof(T) == 16;
  constexpr int kMore = kNormMaxDim / (64 * VEC) > 1 ? kNormMaxDim / (64 * VEC) : 1;
  constexpr int kLess = kWide ? 1 : 2;
  if (!norm_shape<VEC>(a, PAIRS, kMore)) return EBD_ERR_UNSUPPORTED;
  const bool less = a.units <= a.lanes * kLess;
  auto launch = [&](auto u, auto fl) {
    constexpr int U = decltype(u)::value, FL = decltype(fl)::value;
    if constexpr (!APPEND) {
      if (bw) return launch_norm_back_u<T, VEC, PAIRS, U, FL>(a, *bw, s);
    }
    return launch_norm_u<T, VEC, PAIRS, APPEND, U, FL>(a, s);
  };
  using std::integral_constant;
  using One = integral_constant<int, 1>;
  if constexpr (kWide) {
    // whole heads of 64, 128 and 256 channels turn: nothing is asked of a lane's chunks
    constexpr int L64 = 64 / (2 * VEC);
    if (a.rot == a.head_dim) {
      if (a.head_dim == 64) return launch(One{}, integral_constant<int, L64>{});
      if (a.head_dim == 128) return launch(One{}, integral_constant<int, 2 * L64>{});
      if (a.head_dim == 256) return launch(One{}, integral_constant<int, 4 * L64>{});
    }
  }
  using None = integral_constant<int, 0>;
  return less ? launch(integral_constant<int, kLess>{}, None{})
              : launch(integral_constant<int, kMore>{}, None{});
}

// 16-byte accesses where every row and the rotated part allow them; otherwise
// single elements (half) or single pairs (pairs).
template <typename T, bool APPEND>
static ebd_status launch_norm_t(const NormArgs& a, bool pairs, const NormBackward* bw,
                                cudaStream_t s) {
  constexpr int kWide = 16 / (int)sizeof(T);
  auto rows_ok = [&](int vec) {
    const int e = sizeof(T);
    bool ok = a.n_x == 0 || (rows_aligned(a.x, vec, e) && rows_aligned(a.y, vec, e));
    if (bw) ok = ok && rows_aligned(a.dy, vec, e);
    if (APPEND)
      ok = ok && rows_aligned(a.k, vec, e) && rows_aligned(a.v, vec, e) &&
           (uintptr_t)a.K_pages % (vec * e) == 0 && (uintptr_t)a.V_pages % (vec * e) == 0 &&
           a.pv.page_stride % vec == 0 && a.pv.head_stride % vec == 0 && a.pv.row_stride % vec == 0;
    return ok && a.head_dim % vec == 0;
  };
  const bool wide = (pairs ? a.rot : a.rot / 2) % kWide == 0 && rows_ok(kWide);
  if (pairs) {
    if (wide) return launch_norm_v<T, kWide, true, APPEND>(a, bw, s);
    // an odd head_dim or stride would split a pair's 2-element access
    if (rows_ok(2)) return launch_norm_v<T, 2, true, APPEND>(a, bw, s);
    return EBD_ERR_UNSUPPORTED;
  }
  if (wide) return launch_norm_v<T, kWide, false, APPEND>(a, bw, s);
  return launch_norm_v<T, 1, false, APPEND>(a, bw, s);
}

static NormWeight norm_weight(const void* p, ebd_dtype dtype, int64_t hs) {
  const int wide = dtype == EBD_F32 ? 4 : 8;
  return NormWeight{p, hs, dtype == EBD_F32, aligned16(p) && hs % wide == 0};
}

// Checks that the three entry points share; `rot` comes back 0 without a table.
static ebd_status check_norm(ebd_dtype dtype, int n_tokens, int head_dim, ebd_rotary_layout layout,
                             float eps, ebd_dtype weight_dtype, const float* table, int n_pos,
                             int& rot) {
  if (dtype != EBD_F32 && dtype != EBD_BF16) return EBD_ERR_INVALID;
  if (weight_dtype != EBD_F32 && weight_dtype != dtype) return EBD_ERR_INVALID;
  if (layout != EBD_ROTARY_HALF && layout != EBD_ROTARY_PAIRS) return EBD_ERR_INVALID;
  if (n_tokens < 0 || head_dim < 1) return EBD_ERR_INVALID;
  // (a subnormal eps would be flushed, and a row of zeros divided by zero)
  if (!(eps >= FLT_MIN) || !(eps < INFINITY)) return EBD_ERR_INVALID;
  // (token numbers a step past the last one still fit 31 bits)
  if (head_dim > kNormMaxDim || n_tokens > 0x7fffff00) return EBD_ERR_UNSUPPORTED;
  if (!table) {
    rot = 0;
    return EBD_OK;
  }
  if (n_pos < 1 || rot < 2 || rot > head_dim || rot % 2 != 0 || (uintptr_t)table % 8 != 0)
    return EBD_ERR_INVALID;
  return EBD_OK;
}

}  // namespace ebd

using namespace ebd;

extern "C" ebd_status ebd_norm_rotary(
    ebd_dtype dtype, int32_t n_tokens, int32_t n_heads, int32_t head_dim, const void* x,
    int64_t x_token_stride, int64_t x_head_stride, const void* weight, ebd_dtype weight_dtype,
    int64_t weight_head_stride, float eps, const int32_t* positions, const float* table,
    int32_t n_pos, int32_t rotary_dim, ebd_rotary_layout layout, void* y, int64_t y_token_stride,
    int64_t y_head_stride, int32_t* dev_status, void* stream) {
  int rot = rotary_dim;
  const ebd_status st =
      check_norm(dtype, n_tokens, head_dim, layout, eps, weight_dtype, table, n_pos, rot);
  if (st != EBD_OK) return st;
  if (n_heads < 1 || weight_head_stride < 0) return EBD_ERR_INVALID;
  if (n_tokens == 0) return EBD_OK;
  if (!x || !y || !weight || (table && !positions)) return EBD_ERR_INVALID;
  NormArgs a = {};
  a.x = Rows{x, x_token_stride, x_head_stride};
  a.y = Rows{y, y_token_stride, y_head_stride};
  a.positions = table ? positions : nullptr;
  a.table = (const float2*)table;
  a.wx = norm_weight(weight, weight_dtype, weight_head_stride);
  a.n_pos = n_pos;
  a.n_tokens = n_tokens;
  a.n_x = n_heads;
  a.head_dim = head_dim;
  a.rot = rot;
  a.eps = eps;
  a.inv_d = 1.f / head_dim;
  a.dev_status = dev_status;
  const bool pairs = layout == EBD_ROTARY_PAIRS && table;
  cudaStream_t s = (cudaStream_t)stream;
  return dtype == EBD_F32 ? launch_norm_t<float, false>(a, pairs, nullptr, s)
                          : launch_norm_t<__nv_bfloat16, false>(a, pairs, nullptr, s);
}

extern "C" size_t ebd_norm_rotary_backward_workspace_bytes(int32_t n_heads, int32_t head_dim,
                                                           int32_t per_head) {
  if (n_heads < 1 || head_dim < 1) return 0;
  const size_t rows = per_head ? (size_t)n_heads : 1;
  size_t blocks = (size_t)sm_count() * kNormBackBlocks / rows;
  if (blocks < 1) blocks = 1;
  return align_up(blocks * rows * head_dim * 4, 256);
}

extern "C" ebd_status ebd_norm_rotary_backward(
    ebd_dtype dtype, int32_t n_tokens, int32_t n_heads, int32_t head_dim, const void* dy,
    int64_t dy_token_stride, int64_t dy_head_stride, const void* x, int64_t x_token_stride,
    int64_t x_head_stride, const void* weight, ebd_dtype weight_dtype, int64_t weight_head_stride,
    float eps, const int32_t* positions, const float* table, int32_t n_pos, int32_t rotary_dim,
    ebd_rotary_layout layout, void* dx, int64_t dx_token_stride, int64_t dx_head_stride,
    float* dweight, int32_t* dev_status, void* workspace, size_t ws_bytes, void* stream) {
  int rot = rotary_dim;
  const ebd_status st =
      check_norm(dtype, n_tokens, head_dim, layout, eps, weight_dtype, table, n_pos, rot);
  if (st != EBD_OK) return st;
  if (n_heads < 1 || n_heads > 65535 || weight_head_stride < 0 || !dweight) return EBD_ERR_INVALID;
  cudaStream_t s = (cudaStream_t)stream;
  const bool per_head = weight_head_stride != 0;
  if (n_tokens == 0)  // no row: the weight's gradient is zero
    return cuda_status(
        cudaMemsetAsync(dweight, 0, (size_t)(per_head ? n_heads : 1) * head_dim * 4, s));
  if (!dy || !x || !dx || !weight || (table && !positions)) return EBD_ERR_INVALID;
  const size_t need = ebd_norm_rotary_backward_workspace_bytes(n_heads, head_dim, per_head);
  if (ws_bytes < need) return EBD_ERR_CAPACITY;
  if (!workspace || !aligned16(workspace)) return EBD_ERR_INVALID;
  NormArgs a = {};
  a.x = Rows{x, x_token_stride, x_head_stride};
  a.y = Rows{dx, dx_token_stride, dx_head_stride};
  a.dy = Rows{dy, dy_token_stride, dy_head_stride};
  a.positions = table ? positions : nullptr;
  a.table = (const float2*)table;
  a.wx = norm_weight(weight, weight_dtype, weight_head_stride);
  a.n_pos = n_pos;
  a.n_tokens = n_tokens;
  a.n_x = n_heads;
  a.head_dim = head_dim;
  a.rot = rot;
  a.eps = eps;
  a.inv_d = 1.f / head_dim;
  a.dev_status = dev_status;
  const bool pairs = layout == EBD_ROTARY_PAIRS && table;
  const NormBackward bw = {(float*)workspace, dweight};
  return dtype == EBD_F32 ? launch_norm_t<float, false>(a, pairs, &bw, s)
                          : launch_norm_t<__nv_bfloat16, false>(a, pairs, &bw, s);
}

extern "C" ebd_status ebd_paged_append_norm(
    const ebd_paged_cache* cache, int32_t n_tokens, const int32_t* cu_new, const int64_t* slots,
    const int32_t* positions, const void* k_new, int64_t k_token_stride, int64_t k_head_stride,
    const void* v_new, int64_t v_token_stride, int64_t v_head_stride, const void* k_weight,
    int64_t k_weight_head_stride, const void* q_weight, int64_t q_weight_head_stride,
    ebd_dtype weight_dtype, float eps, const float* table, int32_t n_pos, int32_t rotary_dim,
    ebd_rotary_layout layout, int32_t n_q_heads, const void* q, int64_t q_token_stride,
    int64_t q_head_stride, void* q_out, int64_t q_out_token_stride, int64_t q_out_head_stride,
    int32_t* dev_status, void* stream) {
  ebd_status st = check_paged(cache);
  if (st != EBD_OK) return st;
  int rot = rotary_dim;
  st = check_norm((ebd_dtype)cache->dtype, n_tokens, cache->head_dim, layout, eps, weight_dtype,
                  table, n_pos, rot);
  if (st != EBD_OK) return st;
  if (n_q_heads < 0 || k_weight_head_stride < 0 || q_weight_head_stride < 0)
    return EBD_ERR_INVALID;
  if (n_q_heads > 0 && !table && !q_weight) return EBD_ERR_INVALID;  // nothing to do to q
  if (n_tokens == 0) return EBD_OK;
  // a token's place is told by the offsets or by its slot, one of the two; a slot tells
  // no position
  if (!cu_new == !slots || (slots && table && !positions)) return EBD_ERR_INVALID;
  if (!k_new || !v_new || !dev_status || (n_q_heads > 0 && (!q || !q_out))) return EBD_ERR_INVALID;
  NormArgs a = {};
  a.x = Rows{q, q_token_stride, q_head_stride};
  a.y = Rows{q_out, q_out_token_stride, q_out_head_stride};
  a.k = Rows{k_new, k_token_stride, k_head_stride};
  a.v = Rows{v_new, v_token_stride, v_head_stride};
  a.K_pages = cache->K_pages;
  a.V_pages = cache->V_pages;
  a.pv = paged_view(*cache);
  a.cu = cu_new;
  a.slots = slots;
  a.positions = table ? positions : nullptr;
  a.table = (const float2*)table;
  a.wx = norm_weight(q_weight, weight_dtype, q_weight_head_stride);
  a.wk = norm_weight(k_weight, weight_dtype, k_weight_head_stride);
  a.n_pos = n_pos;
  a.n_tokens = n_tokens;
  a.n_x = n_q_heads;
  a.n_kv = cache->n_kv_heads;
  a.head_dim = cache->head_dim;
  a.rot = rot;
  a.eps = eps;
  a.inv_d = 1.f / cache->head_dim;
  a.dev_status = dev_status;
  const bool pairs = layout == EBD_ROTARY_PAIRS && table;
  cudaStream_t s = (cudaStream_t)stream;
  return cache->dtype == EBD_F32 ? launch_norm_t<float, true>(a, pairs, nullptr, s)
                                 : launch_norm_t<__nv_bfloat16, true>(a, pairs, nullptr, s);
}
