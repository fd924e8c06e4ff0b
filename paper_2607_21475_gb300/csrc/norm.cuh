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
// factors once a token, and heads of 64, 128 and 256 channels have forms of their own in
// which every lane has two chunks and, where the whole head turns, asks nothing about them
// (16k tokens x 28 heads x 128, bf16: 413 instructions per warp and 4 rows and 54 us at
// first, 203 and 38 us now).  A row is shared by L lanes, L a power of two, each with U units
// of two chunks, so that a row's sums are log2 L shuffles; neighbouring lanes have
// neighbouring chunks in both layouts (chunks side by side in a lane, pairs layout: 62 us).
// A warp takes 32 / L heads of a token at a time and has three steps' rows on their way
// through shared memory.  The backward pass has an even share of all steps per warp, and its
// rows are asked for from token to token; the weight's gradient is summed per lane, per
// warp, per block and over the blocks (few rows: of one cluster), in that fixed order.
// Measured, bf16, 28 heads x 128: 16384 tokens 38.4 us in either layout, 6.3 TB/s (94% of the
// measured copy peak), half of each head turning 43.4, a weight per head 51.9; gradient of
// 8192 tokens 34.5 us, 5.2 TB/s (77%: instructions, 57% of the issue slots, and 16 warps per
// SM, 128 registers each), a weight per head 43.4; 8 ragged chunks of 9.4k tokens in all
// appended (28/4 heads) 33.7 us, 5.3 TB/s; append step of 32 sequences (32/8 heads) 3.3 us.
// All are programmatic dependents of what precedes them on the stream.
#pragma once

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
constexpr int kNormBackBlocks = 2;  // resident blocks of 256 threads
// Resident blocks of the forward pass: 3 spill where lanes ask whether their chunks turn or
// have a weight per head (ragged chunks appended: 3 blocks 34.1 us against 37.1 with 2; with
// spills 47-58).
constexpr int norm_forward_blocks(int elem, bool all, bool heads) {
  return elem == 4 || (all && !heads) ? 3 : 2;
}
constexpr int kNormMaxDim = 512;
// Heads of a token (append: with the keys' and values'): the next one that a lane asks for lies
// up to (kAhead + 1) U / 16 times as many past the last, once at most.
constexpr int kNormMaxHeads = 0x3fff0000;
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
  float least;               // sums of squares below it are formed anew (rescale_row)
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

// A lane's place in a row: U units of two chunks, at channels c1 and c2.  Half layout: the
// chunks that turn together, then those that stay; pairs layout: chunks L apart, so that in
// both neighbouring lanes have neighbouring chunks.  FL > 0: rows of FL lanes with one whole
// unit each; ALL: every one turns.
template <int VEC, bool PAIRS, int U, int FL, bool ALL>
struct Place {
  static constexpr bool kFull = FL > 0;
  int lanes, sub;
  int c1[U], c2[U];       // -1: the row has none
  bool turns[U], all[U];  // the unit does; its second chunk too (pairs layout)
  static __device__ __forceinline__ void channels(const NormArgs& a, int lanes, int sub, int j,
                                                  int& c1, int& c2) {
    if (PAIRS) {
      c1 = VEC * (sub + 2 * lanes * j);
      c2 = c1 + VEC * lanes;
    } else {
      const int u = sub + lanes * j, v = u - a.rot_units;
      if (ALL || v < 0) {
        c1 = VEC * u;
        c2 = c1 + (ALL ? VEC * FL : a.half_off);
        return;
      }
      c1 = a.rot + VEC * v;
      c2 = c1 + VEC * (a.units - a.rot_units);
    }
    if (!kFull && c1 >= a.head_dim) c1 = -1;
    if (!kFull && (c1 < 0 || c2 >= a.head_dim)) c2 = -1;
  }
  __device__ __forceinline__ Place(const NormArgs& a, int lane)
      : lanes(kFull ? FL : a.lanes), sub(lane & (lanes - 1)) {
#pragma unroll
    for (int j = 0; j < U; ++j) {
      channels(a, lanes, sub, j, c1[j], c2[j]);
      turns[j] = c1[j] >= 0 && c1[j] < (PAIRS ? a.rot : a.half_off);
      all[j] = PAIRS ? c2[j] >= 0 && c2[j] < a.rot : turns[j];
      if (!kFull && !PAIRS && sub + lanes * j >= a.units) c1[j] = c2[j] = -1;
    }
  }
  __device__ __forceinline__ int per_warp() const { return 32 / lanes; }
  __device__ __forceinline__ bool first(int j) const { return kFull || c1[j] >= 0; }
  __device__ __forceinline__ bool second(int j) const { return kFull || c2[j] >= 0; }
  __device__ __forceinline__ bool turn(int j) const { return ALL || turns[j]; }
  __device__ __forceinline__ bool turn_all(int j) const { return ALL || all[j]; }
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

// (second: the second chunk turns too, pairs layout)
template <int VEC, bool PAIRS>
__device__ __forceinline__ void load_angles(const NormArgs& a, int tpos, int c1, int c2,
                                            bool second, Angles<VEC>& t) {
  constexpr int kRun = PAIRS ? VEC / 2 : VEC;  // pairs of a chunk, side by side in the table
  auto load = [&](const float2* p, int i0) {
    if (kRun % 2 == 0 && a.wide_table) {
#pragma unroll
      for (int i = 0; i + 1 < kRun; i += 2) {
        const float4 f = __ldg(reinterpret_cast<const float4*>(p + i));
        t.c[i0 + i] = f.x, t.s[i0 + i] = f.y;
        t.c[i0 + i + 1] = f.z, t.s[i0 + i + 1] = f.w;
      }
    } else {
#pragma unroll
      for (int i = 0; i < kRun; ++i) {
        const float2 f = __ldg(p + i);
        t.c[i0 + i] = f.x, t.s[i0 + i] = f.y;
      }
    }
  };
  const float2* row = a.table + (size_t)tpos * (a.rot / 2);
  load(row + (PAIRS ? c1 / 2 : c1), 0);
  if constexpr (PAIRS)
    if (second) load(row + c2 / 2, kRun);
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

// Rows whose sum of squares leaves float32's range are scaled by a power of two first.
// Down, 2^-70, where it is not finite: values are below 2^128, so those of a scaled row are
// below 2^58 and 512 squares of them below 2^125; one of such a row's values is at least
// 2^59.5, and 2^-21 when scaled and squared.
// Up, 2^64, where squares that are flushed (below 2^-126) count beside eps: from 2^-102 on what
// they could add to the mean changes r by 2^-25 at most; below it rows with a sum under 2^-60
// are scaled (beside a larger sum the flushed squares do not count): values below 2^-30, eps
// between 2^2 and 2^26 then.  Calls with such an eps take the forms by elements and pairs, the
// only ones that ask: the second comparison cost the 16-byte forms 0.7 to 2.7% (16k tokens x
// 28 x 80 bf16 48.2 -> 49.5 us), for an eps that is hardly ever asked for.
constexpr float kRowDown = 8.470329472543003e-22f, kRowUp = 18446744073709551616.f;
constexpr float kSmallEps = 1.9721522630525295e-31f, kSmallSum = 8.673617379884035e-19f;
template <typename T, int VEC>
constexpr bool kWideRows = VEC * sizeof(T) == 16;

// Whether a row's sum of squares asks for that.
template <typename T, int VEC>
__device__ __forceinline__ bool out_of_range(const NormArgs& a, float ss) {
  if (!kWideRows<T, VEC> && ss < a.least) return true;
  return !(ss < INFINITY);
}
// Scales such a row, eps too; the scale.
template <typename T, int VEC, int U>
__device__ __forceinline__ float rescale_row(float ss, float& eps, Part<VEC> (&x)[U]) {
  const bool up = !kWideRows<T, VEC> && ss < 1.f;
  const float scale = up ? kRowUp : kRowDown;
  eps = up ? eps * kRowUp * kRowUp : 0.f;  // (0: below the sum's rounding)
  auto times = [&](float v) {              // (not flushed: a row may be of subnormal values)
    asm("mul.rn.f32 %0, %0, %1;" : "+f"(v) : "f"(scale));
    return v;
  };
#pragma unroll
  for (int j = 0; j < U; ++j)
#pragma unroll
    for (int i = 0; i < VEC; ++i) x[j].lo[i] = times(x[j].lo[i]), x[j].hi[i] = times(x[j].hi[i]);
  return scale;
}

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

// Shape of a row's lanes for chunks of VEC elements; false: too many units.
template <int VEC>
inline bool norm_shape(NormArgs& a, bool pairs, int max_u) {
  const int rot_chunks = a.rot / VEC, chunks = a.head_dim / VEC;
  a.half_off = a.rot / 2;
  a.rot_units = pairs ? 0 : rot_chunks / 2;
  a.units = pairs ? (chunks + 1) / 2 : a.rot_units + (chunks - rot_chunks + 1) / 2;
  a.wide_table = a.rot % 4 == 0 && (uintptr_t)a.table % 16 == 0;
  a.least = a.eps < kSmallEps ? kSmallSum : 0.f;
  a.lanes = 1;
  while (a.lanes < 32 && a.lanes < a.units) a.lanes *= 2;
  return a.units <= a.lanes * max_u;
}

struct NormBackward {
  float *partial, *dweight;
};

// One launch for chunks of VEC elements: the pass and the units per lane, of which rows of
// 512 channels need at most 1 (bf16) or 2 (float32) in wide chunks, 8 by elements and 4 by
// pairs.
enum NormPass { kNormForward, kNormAppend, kNormBackward };
// Each defined in the translation unit of its pass.
template <typename T, int VEC, bool PAIRS, bool APPEND, int U, int FL, bool ALL>
ebd_status launch_norm_u(NormArgs a, cudaStream_t s);
template <typename T, int VEC, bool PAIRS, int U, int FL, bool ALL>
ebd_status launch_norm_back_u(NormArgs a, const NormBackward& bw, cudaStream_t s);

template <typename T, int VEC, bool PAIRS, NormPass PASS>
ebd_status launch_norm_v(NormArgs a, const NormBackward* bw, cudaStream_t s) {
  constexpr bool kWide = VEC * sizeof(T) == 16;
  constexpr int kMore = kNormMaxDim / (64 * VEC) > 1 ? kNormMaxDim / (64 * VEC) : 1;
  constexpr int kLess = kWide ? 1 : 2;
  if (!norm_shape<VEC>(a, PAIRS, kMore)) return EBD_ERR_UNSUPPORTED;
  const bool less = a.units <= a.lanes * kLess;
  auto launch = [&](auto u, auto fl, auto all) {
    constexpr int U = decltype(u)::value, FL = decltype(fl)::value;
    constexpr bool ALL = decltype(all)::value;
    if constexpr (PASS == kNormBackward)
      return launch_norm_back_u<T, VEC, PAIRS, U, FL, ALL>(a, *bw, s);
    else
      return launch_norm_u<T, VEC, PAIRS, PASS == kNormAppend, U, FL, ALL>(a, s);
  };
  using std::integral_constant;
  using One = integral_constant<int, 1>;
  if constexpr (kWide) {
    // heads of 64, 128 and 256 channels: every lane has two chunks
    constexpr int L64 = 64 / (2 * VEC);
    auto full = [&](auto fl) {
      return a.rot == a.head_dim ? launch(One{}, fl, std::true_type{})
                                 : launch(One{}, fl, std::false_type{});
    };
    if (a.head_dim == 64) return full(integral_constant<int, L64>{});
    if (a.head_dim == 128) return full(integral_constant<int, 2 * L64>{});
    if (a.head_dim == 256) return full(integral_constant<int, 4 * L64>{});
  }
  using None = integral_constant<int, 0>;
  return less ? launch(integral_constant<int, kLess>{}, None{}, std::false_type{})
              : launch(integral_constant<int, kMore>{}, None{}, std::false_type{});
}

// 16-byte accesses where every row, the rotated part and eps (kSmallEps) allow them; otherwise
// single elements (half) or single pairs (pairs).
template <typename T, NormPass PASS>
ebd_status launch_norm_t(const NormArgs& a, bool pairs, const NormBackward* bw, cudaStream_t s) {
  constexpr int kWide = 16 / (int)sizeof(T);
  auto rows_ok = [&](int vec) {
    const int e = sizeof(T);
    bool ok = a.n_x == 0 || (rows_aligned(a.x, vec, e) && rows_aligned(a.y, vec, e));
    if (PASS == kNormBackward) ok = ok && rows_aligned(a.dy, vec, e);
    if (PASS == kNormAppend)
      ok = ok && rows_aligned(a.k, vec, e) && rows_aligned(a.v, vec, e) &&
           (uintptr_t)a.K_pages % (vec * e) == 0 && (uintptr_t)a.V_pages % (vec * e) == 0 &&
           a.pv.page_stride % vec == 0 && a.pv.head_stride % vec == 0 && a.pv.row_stride % vec == 0;
    return ok && a.head_dim % vec == 0;
  };
  const bool wide =
      !(a.eps < kSmallEps) && (pairs ? a.rot : a.rot / 2) % kWide == 0 && rows_ok(kWide);
  if (pairs) {
    if (wide) return launch_norm_v<T, kWide, true, PASS>(a, bw, s);
    // an odd head_dim or stride would split a pair's 2-element access
    if (rows_ok(2)) return launch_norm_v<T, 2, true, PASS>(a, bw, s);
    return EBD_ERR_UNSUPPORTED;
  }
  if (wide) return launch_norm_v<T, kWide, false, PASS>(a, bw, s);
  return launch_norm_v<T, 1, false, PASS>(a, bw, s);
}

inline NormWeight norm_weight(const void* p, ebd_dtype dtype, int64_t hs) {
  const int wide = dtype == EBD_F32 ? 4 : 8;
  return NormWeight{p, hs, dtype == EBD_F32, aligned16(p) && hs % wide == 0};
}

// Checks that the three entry points share; `rot` comes back 0 without a table.
inline ebd_status check_norm(ebd_dtype dtype, int n_tokens, int head_dim, ebd_rotary_layout layout,
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
