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
// Both directions move rows (forward 2, backward 3 per row; some 7 and 13 FMAs per
// channel), so HBM bounds them at large sizes, a launch and a chain of loads at small
// ones.  A row is shared by L lanes, L a power of two, each with U pairs of chunks that
// turn together, so that a row's sums are log2 L shuffles; a warp takes 32 / L heads
// of one token at a time, keeps the token's angles and the weight in registers and
// has two steps' rows in flight.
#include <cuda_runtime.h>
#include <math.h>

#include "common.cuh"
#include "decode_tile.cuh"
#include "internal.h"
#include "paged.cuh"
#include "paged_attn.cuh"
#include "rotary.cuh"

namespace ebd {

constexpr int kNormWarps = 8;
constexpr int kNormBlocks = 3, kNormBackBlocks = 2;  // resident blocks of 256 threads
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

// The weight of channels c .. c + VEC - 1 of a head.
template <int VEC>
__device__ __forceinline__ void load_weight(const NormWeight& w, int h, int c, float* out) {
  const long long at = h * w.hs + c;
  if (w.f32) {
    const float* p = (const float*)w.p + at;
    if (VEC % 4 == 0 && w.wide) {
#pragma unroll
      for (int i = 0; i + 3 < VEC; i += 4) {
        const float4 f = __ldg(reinterpret_cast<const float4*>(p + i));
        out[i] = f.x, out[i + 1] = f.y, out[i + 2] = f.z, out[i + 3] = f.w;
      }
    } else {
#pragma unroll
      for (int i = 0; i < VEC; ++i) out[i] = __ldg(p + i);
    }
  } else {
    const __nv_bfloat16* p = (const __nv_bfloat16*)w.p + at;
    if (VEC % 4 == 0 && w.wide) {
#pragma unroll
      for (int i = 0; i + 3 < VEC; i += 4) {
        const uint2 f = __ldg(reinterpret_cast<const uint2*>(p + i));
        out[i] = bf16_lo(f.x), out[i + 1] = bf16_hi(f.x);
        out[i + 2] = bf16_lo(f.y), out[i + 3] = bf16_hi(f.y);
      }
    } else {
#pragma unroll
      for (int i = 0; i < VEC; ++i) out[i] = __bfloat162float(p[i]);
    }
  }
}

// Cosines and sines of unit u's pairs at row tpos of the table.
template <int VEC, bool PAIRS>
__device__ __forceinline__ void load_unit_angles(const NormArgs& a, int tpos, int u,
                                                 float (&cs)[VEC], float (&sn)[VEC]) {
  if (u >= a.rot_units) return;
  const float2* row = a.table + (size_t)tpos * (a.rot / 2) + u * VEC;
  const int n = PAIRS ? min(VEC, a.rot / 2 - u * VEC) : VEC;
  if (VEC % 2 == 0 && a.wide_table) {
#pragma unroll
    for (int i = 0; i + 1 < VEC; i += 2) {
      if (PAIRS && i >= n) break;
      const float4 f = __ldg(reinterpret_cast<const float4*>(row + i));
      cs[i] = f.x;
      sn[i] = f.y;
      cs[i + 1] = f.z;
      sn[i + 1] = f.w;
    }
  } else {
#pragma unroll
    for (int i = 0; i < VEC; ++i) {
      if (PAIRS && i >= n) break;
      const float2 f = __ldg(row + i);
      cs[i] = f.x;
      sn[i] = f.y;
    }
  }
}

// Turns the pairs of a unit's two chunks (p: the first, q: the second), rot: the first
// channel that stays, c2 the second chunk's channel.
template <int VEC, bool PAIRS>
__device__ __forceinline__ void turn_unit(float (&p)[VEC], float (&q)[VEC], const float (&cs)[VEC],
                                          const float (&sn)[VEC], float sign, int c2, int rot) {
  auto turn = [&](float& e0, float& e1, int i) {
    const float a = e0, b = e1, s = sn[i] * sign;
    e0 = a * cs[i] - b * s;
    e1 = b * cs[i] + a * s;
  };
  if (PAIRS) {
#pragma unroll
    for (int i = 0; i < VEC / 2; ++i) turn(p[2 * i], p[2 * i + 1], i);
    if (c2 >= 0 && c2 < rot) {
#pragma unroll
      for (int i = 0; i < VEC / 2; ++i) turn(q[2 * i], q[2 * i + 1], VEC / 2 + i);
    }
  } else {
#pragma unroll
    for (int i = 0; i < VEC; ++i) turn(p[i], q[i], i);
  }
}

// Sum over the L lanes that share a row.
__device__ __forceinline__ float row_sum(float v, int lanes) {
  for (int o = 1; o < lanes; o <<= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
  return v;
}

// 2^-64: rows whose sum of squares leaves float32's range are scaled by it first.
constexpr float kRowScale = 5.421010862427522e-20f;

template <typename T, int VEC>
__device__ __forceinline__ void scale_chunk(Chunk<T, VEC>& c, float f) {
#pragma unroll
  for (int i = 0; i < VEC; ++i) from_f32(to_f32(c.e[i]) * f, c.e[i]);
}

template <typename T, int VEC>
__device__ __forceinline__ void widen(const Chunk<T, VEC>& c, float (&x)[VEC]) {
#pragma unroll
  for (int i = 0; i < VEC; ++i) x[i] = to_f32(c.e[i]);
}
template <typename T, int VEC>
__device__ __forceinline__ void narrow(const float (&x)[VEC], Chunk<T, VEC>& c) {
#pragma unroll
  for (int i = 0; i < VEC; ++i) from_f32(x[i], c.e[i]);
}

template <typename T, int VEC, bool PAIRS, bool APPEND, int U>
__global__ void __launch_bounds__(kNormWarps * 32, norm_blocks(kNormBlocks, U, VEC))
    norm_rotary_kernel(const NormArgs a) {
  const int lane = threadIdx.x & 31;
  const long long w = (long long)blockIdx.x * kNormWarps + (threadIdx.x >> 5);
  const int t = a.parts == 1 ? (int)w : (int)(w / a.parts), part = (int)(w - (long long)t * a.parts);
  if (t >= a.n_tokens) return;
  const int L = a.lanes, sub = lane & (L - 1), per_warp = 32 / L;
  const int heads = a.n_x + (APPEND ? 2 * a.n_kv : 0);
  const int step = per_warp * a.parts;
  int hb = part * per_warp;  // first head of the warp's step
  const int g = lane / L;
  const T* xp = (const T*)a.x.p + t * a.x.ts;
  const T* kp = (const T*)a.k.p + t * a.k.ts;
  const T* vp = (const T*)a.v.p + t * a.v.ts;
  auto load = [&](int h, Piece<T, VEC> (&r)[U]) {
    if (h >= heads) return;
    const T* src = !APPEND || h < a.n_x  ? xp + h * a.x.hs
                   : h < a.n_x + a.n_kv ? kp + (h - a.n_x) * a.k.hs
                                        : vp + (h - a.n_x - a.n_kv) * a.v.hs;
#pragma unroll
    for (int j = 0; j < U; ++j) {
      const int u = sub + L * j;
      if (u >= a.units) break;
      int c1, c2;
      unit_channels<VEC, PAIRS>(a, u, c1, c2);
      load_chunk<T, VEC>(src + c1, r[j].a);
      if (c2 >= 0) load_chunk<T, VEC>(src + c2, r[j].b);
    }
  };
  Piece<T, VEC> r0[U], r1[U];
  load(hb + g, r0);
  load(hb + g + step, r1);

  // 0: x, 1: keys, 2: values
  auto set_of = [&](int h) { return !APPEND || h < a.n_x ? 0 : h < a.n_x + a.n_kv ? 1 : 2; };
  float wt[U][2 * VEC];
  int held = -1;  // the set whose weight is in wt
  auto load_weights = [&](int h, int set) {
    const NormWeight& w = set == 0 ? a.wx : a.wk;
    if (!w.p || (held == set && w.hs == 0)) return;
    held = set;
    const int head = set == 0 ? h : h - a.n_x;
#pragma unroll
    for (int j = 0; j < U; ++j) {
      const int u = sub + L * j;
      if (u >= a.units) break;
      int c1, c2;
      unit_channels<VEC, PAIRS>(a, u, c1, c2);
      load_weight<VEC>(w, head, c1, &wt[j][0]);
      if (c2 >= 0) load_weight<VEC>(w, head, c2, &wt[j][VEC]);
    }
  };
  if (hb + g < heads && set_of(hb + g) < 2) load_weights(hb + g, set_of(hb + g));

  int pos = 0, page = -1;
  long long at = -1;  // the token's row of head 0 in the pools
  if (APPEND && a.slots) {
    const int64_t slot = a.slots[t];
    if (slot == -1) return;  // no token here
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
    if (none) return;
    pos = len - (min(c1, a.n_tokens) - t);
    page = page_of(a.pv, b, pos);
    if (page >= 0) at = slot_offset(a.pv, page, 0, pos);
    if (a.positions) pos = a.positions[t];
  } else if (a.positions) {
    pos = a.positions[t];
  }
  const int tpos = a.table ? min(max(pos, 0), a.n_pos - 1) : 0;
  float cs[U][VEC], sn[U][VEC];
#pragma unroll
  for (int j = 0; j < U; ++j) load_unit_angles<VEC, PAIRS>(a, tpos, sub + L * j, cs[j], sn[j]);
  if (lane == 0 && ((APPEND && page < 0) || (a.table && tpos != pos)))
    raise_status(a.dev_status, EBD_DEV_RANGE);
  T* yp = (T*)a.y.p + t * a.y.ts;

  // normalises, turns and stores one row's pieces; whole warp
  auto store = [&](int h, Piece<T, VEC> (&r)[U]) {
    const bool live = h < heads;
    const int set = set_of(h);
    const bool normed = live && set < 2 && (set == 0 ? a.wx.p : a.wk.p) != nullptr;
    auto squares = [&]() {
      float ss = 0.f;
      if (normed) {
#pragma unroll
        for (int j = 0; j < U; ++j) {
          const int u = sub + L * j;
          if (u >= a.units) break;
          int c1, c2;
          unit_channels<VEC, PAIRS>(a, u, c1, c2);
          float x[VEC];
          widen(r[j].a, x);
#pragma unroll
          for (int i = 0; i < VEC; ++i) ss = fmaf(x[i], x[i], ss);
          if (c2 >= 0) {
            widen(r[j].b, x);
#pragma unroll
            for (int i = 0; i < VEC; ++i) ss = fmaf(x[i], x[i], ss);
          }
        }
      }
      return row_sum(ss, L);
    };
    float ss = squares(), eps = a.eps;
    if (__any_sync(0xffffffffu, !(ss < INFINITY))) {
      if (!(ss < INFINITY)) {
        eps = 0.f;  // below the sum's rounding
#pragma unroll
        for (int j = 0; j < U; ++j) {
          scale_chunk(r[j].a, kRowScale);
          scale_chunk(r[j].b, kRowScale);
        }
      }
      ss = squares();
    }
    if (!live) return;
    const float inv = __frsqrt_rn(fmaf(ss, a.inv_d, eps));
    if (normed) load_weights(h, set);
    T* dst;
    if (!APPEND || set == 0) {
      dst = yp + h * a.y.hs;
    } else {
      if (at < 0) return;
      const int kh = h - a.n_x - (set == 2 ? a.n_kv : 0);
      dst = (T*)(set == 2 ? a.V_pages : a.K_pages) + at + kh * a.pv.head_stride;
    }
#pragma unroll
    for (int j = 0; j < U; ++j) {
      const int u = sub + L * j;
      if (u >= a.units) break;
      int c1, c2;
      unit_channels<VEC, PAIRS>(a, u, c1, c2);
      if (set < 2) {
        float p[VEC], q[VEC];
        widen(r[j].a, p);
        widen(r[j].b, q);
        if (normed) {
#pragma unroll
          for (int i = 0; i < VEC; ++i) {
            p[i] *= inv * wt[j][i];
            q[i] *= inv * wt[j][VEC + i];
          }
        }
        if (u < a.rot_units) turn_unit<VEC, PAIRS>(p, q, cs[j], sn[j], 1.f, c2, a.rot);
        narrow(p, r[j].a);
        narrow(q, r[j].b);
      }
      store_chunk<T, VEC>(dst + c1, r[j].a);
      if (c2 >= 0) store_chunk<T, VEC>(dst + c2, r[j].b);
    }
  };
  for (; hb < heads; hb += 2 * step) {
    store(hb + g, r0);
    load(hb + g + 2 * step, r0);
    if (hb + step >= heads) break;
    store(hb + g + step, r1);
    load(hb + g + 3 * step, r1);
  }
}

// PER_HEAD: a block has one head (blockIdx.y), a warp's groups of lanes have tokens; else
// they have heads of a token.  Leaves the block's sum of the weight's gradient in
// partial[blockIdx.x][blockIdx.y][d].
template <typename T, int VEC, bool PAIRS, int U, bool PER_HEAD>
__global__ void __launch_bounds__(kNormWarps * 32, norm_blocks(kNormBackBlocks, U, VEC))
    norm_backward_kernel(const NormArgs a, float* __restrict__ partial) {
  extern __shared__ float red[];  // [warps][units of all lanes][2 VEC]
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int L = a.lanes, sub = lane & (L - 1), per_warp = 32 / L, g = lane / L;
  const long long items =
      PER_HEAD ? (a.n_tokens + per_warp - 1) / per_warp : (long long)a.n_tokens * a.parts;
  const int step = per_warp * a.parts;

  float wt[U][2 * VEC], acc[U][2 * VEC];
  int ch1[U], ch2[U];
#pragma unroll
  for (int j = 0; j < U; ++j) {
    const int u = sub + L * j;
    ch1[j] = ch2[j] = -1;
    if (u < a.units) {
      unit_channels<VEC, PAIRS>(a, u, ch1[j], ch2[j]);
      const int head = PER_HEAD ? blockIdx.y : 0;
      load_weight<VEC>(a.wx, head, ch1[j], &wt[j][0]);
      if (ch2[j] >= 0) load_weight<VEC>(a.wx, head, ch2[j], &wt[j][VEC]);
    }
#pragma unroll
    for (int i = 0; i < 2 * VEC; ++i) acc[j][i] = 0.f;
  }

  for (long long item = (long long)blockIdx.x * kNormWarps + warp; item < items;
       item += (long long)gridDim.x * kNormWarps) {
    int t, h;
    if (PER_HEAD) {
      t = (int)(item * per_warp) + g;
      h = blockIdx.y;
    } else {
      t = (int)(item / a.parts);
      h = (int)(item - (long long)t * a.parts) * per_warp + g;
    }
    const int hend = PER_HEAD ? h + 1 : a.n_x;
    const bool there = t < a.n_tokens;
    auto load = [&](int h, Piece<T, VEC> (&x)[U], Piece<T, VEC> (&dy)[U]) {
      if (!there || h >= hend) return;
      const T* xp = (const T*)a.x.p + t * a.x.ts + h * a.x.hs;
      const T* dp = (const T*)a.dy.p + t * a.dy.ts + h * a.dy.hs;
#pragma unroll
      for (int j = 0; j < U; ++j) {
        if (ch1[j] < 0) break;
        load_chunk<T, VEC>(xp + ch1[j], x[j].a);
        load_chunk<T, VEC>(dp + ch1[j], dy[j].a);
        if (ch2[j] >= 0) {
          load_chunk<T, VEC>(xp + ch2[j], x[j].b);
          load_chunk<T, VEC>(dp + ch2[j], dy[j].b);
        }
      }
    };
    Piece<T, VEC> x0[U], d0[U], x1[U], d1[U];
    load(h, x0, d0);
    const int pos = there && a.positions ? a.positions[t] : 0;
    const int tpos = a.table ? min(max(pos, 0), a.n_pos - 1) : 0;
    if (there && sub == 0 && a.table && tpos != pos) raise_status(a.dev_status, EBD_DEV_RANGE);
    float cs[U][VEC], sn[U][VEC];
#pragma unroll
    for (int j = 0; j < U; ++j) load_unit_angles<VEC, PAIRS>(a, tpos, sub + L * j, cs[j], sn[j]);
    // one row; whole warp
    auto row = [&](int h, Piece<T, VEC> (&x)[U], Piece<T, VEC> (&dy)[U]) {
      const bool live = there && h < hend;
      float u[U][2 * VEC];  // R^T dy
#pragma unroll
      for (int j = 0; j < U; ++j) {
        if (!live || ch1[j] < 0) break;
        float p[VEC], q[VEC];
        widen(dy[j].a, p);
        widen(dy[j].b, q);
        if (sub + L * j < a.rot_units)
          turn_unit<VEC, PAIRS>(p, q, cs[j], sn[j], -1.f, ch2[j], a.rot);
#pragma unroll
        for (int i = 0; i < VEC; ++i) u[j][i] = p[i], u[j][VEC + i] = q[i];
      }
      float ss, gx;
      auto sums = [&]() {
        ss = gx = 0.f;
#pragma unroll
        for (int j = 0; j < U; ++j) {
          if (!live || ch1[j] < 0) break;
          float v[VEC];
          widen(x[j].a, v);
#pragma unroll
          for (int i = 0; i < VEC; ++i) {
            ss = fmaf(v[i], v[i], ss);
            gx = fmaf(u[j][i] * wt[j][i], v[i], gx);
          }
          if (ch2[j] >= 0) {
            widen(x[j].b, v);
#pragma unroll
            for (int i = 0; i < VEC; ++i) {
              ss = fmaf(v[i], v[i], ss);
              gx = fmaf(u[j][VEC + i] * wt[j][VEC + i], v[i], gx);
            }
          }
        }
        ss = row_sum(ss, L);
        gx = row_sum(gx, L);
      };
      sums();
      float eps = a.eps, scale = 1.f;
      if (__any_sync(0xffffffffu, !(ss < INFINITY))) {
        if (!(ss < INFINITY)) {
          eps = 0.f;
          scale = kRowScale;
#pragma unroll
          for (int j = 0; j < U; ++j) {
            scale_chunk(x[j].a, kRowScale);
            scale_chunk(x[j].b, kRowScale);
          }
        }
        sums();
      }
      if (!live) return;
      const float inv = __frsqrt_rn(fmaf(ss, a.inv_d, eps));
      const float mean = gx * inv * a.inv_d;  // of g z
      const float back = inv * scale;
      T* out = (T*)a.y.p + t * a.y.ts + h * a.y.hs;
#pragma unroll
      for (int j = 0; j < U; ++j) {
        if (ch1[j] < 0) break;
        float v[VEC];
        auto half = [&](Chunk<T, VEC>& c, int o) {
          widen(c, v);
#pragma unroll
          for (int i = 0; i < VEC; ++i) {
            const float z = v[i] * inv, uu = u[j][o + i];
            acc[j][o + i] = fmaf(uu, z, acc[j][o + i]);
            v[i] = (uu * wt[j][o + i] - z * mean) * back;
          }
          narrow(v, c);
        };
        half(x[j].a, 0);
        store_chunk<T, VEC>(out + ch1[j], x[j].a);
        if (ch2[j] >= 0) {
          half(x[j].b, VEC);
          store_chunk<T, VEC>(out + ch2[j], x[j].b);
        }
      }
    };
    if (PER_HEAD) {
      row(h, x0, d0);
    } else {
      // (h - g: the warp's step is the same in all lanes)
      load(h + step, x1, d1);
      for (; h - g < a.n_x; h += 2 * step) {
        row(h, x0, d0);
        load(h + 2 * step, x0, d0);
        if (h - g + step >= a.n_x) break;
        row(h + step, x1, d1);
        load(h + 3 * step, x1, d1);
      }
    }
  }

  // the block's sum, in a fixed order: lanes, then warps
  const int wide = L * U * 2 * VEC;
#pragma unroll
  for (int j = 0; j < U; ++j)
#pragma unroll
    for (int i = 0; i < 2 * VEC; ++i) {
      float v = acc[j][i];
      for (int o = L; o < 32; o <<= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
      if (g == 0) red[warp * wide + (sub + L * j) * 2 * VEC + i] = v;
    }
  __syncthreads();
  float* dst = partial + ((size_t)blockIdx.x * gridDim.y + blockIdx.y) * a.head_dim;
  for (int k = threadIdx.x; k < wide; k += kNormWarps * 32) {
    const int u = k / (2 * VEC), i = k - u * 2 * VEC;
    if (u >= a.units) continue;
    int c1, c2;
    unit_channels<VEC, PAIRS>(a, u, c1, c2);
    if (i >= VEC && c2 < 0) continue;
    float v = 0.f;
#pragma unroll
    for (int x = 0; x < kNormWarps; ++x) v += red[x * wide + k];
    dst[i < VEC ? c1 + i : c2 + i - VEC] = v;
  }
}

// dweight[i] = sum over the n blocks of partial[block][i], i < total; 32 columns per block,
// warp w sums the blocks w, w + 8, ..
__global__ void __launch_bounds__(256)
    norm_weight_reduce_kernel(const float* __restrict__ partial, int n, int total,
                              float* __restrict__ dweight) {
  __shared__ float s[8][32];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, i = blockIdx.x * 32 + lane;
  grid_dependency_wait();
  float v = 0.f;
  if (i < total) {
#pragma unroll 8
    for (int k = warp; k < n; k += 8) v += partial[(size_t)k * total + i];
  }
  s[warp][lane] = v;
  __syncthreads();
  if (warp == 0 && i < total) {
    v = 0.f;
#pragma unroll
    for (int k = 0; k < 8; ++k) v += s[k][lane];
    dweight[i] = v;
  }
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

template <typename T, int VEC, bool PAIRS, bool APPEND, int U>
static ebd_status launch_norm_u(NormArgs a, cudaStream_t s) {
  const int heads = a.n_x + (APPEND ? 2 * a.n_kv : 0);
  // one row per lane while the call has fewer warps than the GPU holds (latency), up to
  // sixteen pairs of chunks per lane beyond that
  const int many = (heads * a.lanes + 31) / 32, few = (heads * a.lanes * U + 511) / 512;
  a.parts = (long long)a.n_tokens * many <= (long long)sm_count() * 32 ? many : few;
  const long long blocks = ((long long)a.n_tokens * a.parts + kNormWarps - 1) / kNormWarps;
  if (blocks > 0x7fffffffLL) return EBD_ERR_UNSUPPORTED;
  norm_rotary_kernel<T, VEC, PAIRS, APPEND, U>
      <<<(unsigned)blocks, kNormWarps * 32, 0, s>>>(a);
  return launch_status();
}

// Blocks of the backward pass along its rows (times the heads where each has a weight).
static int norm_back_blocks(long long items, int heads) {
  const long long want = (items + kNormWarps - 1) / kNormWarps;
  long long most = (long long)sm_count() * kNormBackBlocks / heads;
  if (most < 1) most = 1;
  return (int)(want < most ? want : most);
}

struct NormBackward {
  float *partial, *dweight;
};

template <typename T, int VEC, bool PAIRS, int U>
static ebd_status launch_norm_back_u(NormArgs a, const NormBackward& bw, cudaStream_t s) {
  const bool per_head = a.wx.hs != 0;
  const int per_warp = 32 / a.lanes;
  // whole tokens per warp, unless there are too few for every warp of the GPU
  const int steps = (a.n_x + per_warp - 1) / per_warp;
  const long long warps = (long long)sm_count() * kNormBackBlocks * kNormWarps;
  long long parts = (warps + a.n_tokens - 1) / a.n_tokens;
  a.parts = (int)(parts < steps ? parts : steps);
  const long long items =
      per_head ? (a.n_tokens + per_warp - 1) / per_warp : (long long)a.n_tokens * a.parts;
  const int blocks = norm_back_blocks(items, per_head ? a.n_x : 1);
  const int total = (per_head ? a.n_x : 1) * a.head_dim;
  const int smem = kNormWarps * a.lanes * U * 2 * VEC * 4;
  const dim3 grid(blocks, per_head ? a.n_x : 1);
  if (per_head)
    norm_backward_kernel<T, VEC, PAIRS, U, true><<<grid, kNormWarps * 32, smem, s>>>(a, bw.partial);
  else
    norm_backward_kernel<T, VEC, PAIRS, U, false><<<grid, kNormWarps * 32, smem, s>>>(a, bw.partial);
  const ebd_status st = launch_status();
  if (st != EBD_OK) return st;
  return launch_dependent(norm_weight_reduce_kernel, dim3((total + 31) / 32), 256, 0, s,
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
  if constexpr (!APPEND) {
    if (bw)
      return less ? launch_norm_back_u<T, VEC, PAIRS, kLess>(a, *bw, s)
                  : launch_norm_back_u<T, VEC, PAIRS, kMore>(a, *bw, s);
  }
  return less ? launch_norm_u<T, VEC, PAIRS, APPEND, kLess>(a, s)
              : launch_norm_u<T, VEC, PAIRS, APPEND, kMore>(a, s);
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
  if (!(eps > 0.f) || !(eps < INFINITY)) return EBD_ERR_INVALID;
  if (head_dim > kNormMaxDim) return EBD_ERR_UNSUPPORTED;
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
