// The forward pass of the norms with the rotation: on its own (norm_rotary.cu) and on the way
// into a paged cache (norm_append.cu).
#pragma once

#include "norm.cuh"

namespace ebd {

// HEADS: a weight per head (append: of keys or queries), multiplied row by row; else it is in
// the turn's factors.
template <typename T, int VEC, bool PAIRS, bool APPEND, int U, int FL, bool ALL, bool HEADS>
__global__ void __launch_bounds__(kNormWarps * 32, norm_blocks(norm_forward_blocks(sizeof(T), ALL, HEADS), U, VEC))
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
  const Place<VEC, PAIRS, U, FL, ALL> place(a, lane);
  const int sub = place.sub, g = lane / place.lanes, step = place.per_warp() * a.parts;
  int hb = part * place.per_warp();  // first head of the warp's step
  Ring ring(ring_s);
  int hf = hb + g;  // the next head to fetch, and (not append) its row
  const T* xf = (const T*)a.x.p + t * a.x.ts + hf * a.x.hs;
  const long long x_step = step * a.x.hs;
  auto fetch = [&]() {
    const T* p = xf;
    if (APPEND) {
      const bool q = hf < a.n_x, k = hf < a.n_x + a.n_kv;
      const int h = q ? hf : k ? hf - a.n_x : hf - a.n_x - a.n_kv;
      const Rows& r = q ? a.x : k ? a.k : a.v;
      p = (const T*)r.p + t * r.ts + h * r.hs;
    }
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
  auto load_factors = [&](int set) {
    if (set > 1 || held == set) return;
    held = set;
    const NormWeight& w = set == 0 ? a.wx : a.wk;
#pragma unroll
    for (int j = 0; j < U; ++j) {
      Angles<VEC> t;
      if (place.turn(j))
        load_angles<VEC, PAIRS>(a, tpos, place.c1[j], place.c2[j], place.turn_all(j), t);
      Part<VEC> wt;
#pragma unroll
      for (int i = 0; i < VEC; ++i) wt.lo[i] = wt.hi[i] = 1.f;
      if (!HEADS && w.p) load_weight<T, VEC, PAIRS>(w, 0, place.c1[j], place.c2[j], wt);
      f[j].set(t, wt, place.turn(j));
      if (PAIRS && !place.turn_all(j)) f[j].second_stays(wt);
    }
  };
  if (hb + g < heads) load_factors(set_of(hb + g));
  if (lane == 0 && ((APPEND && page < 0) || (a.table && tpos != pos)))
    raise_status(a.dev_status, EBD_DEV_RANGE);
  T* yh = (T*)a.y.p + t * a.y.ts + (hb + g) * a.y.hs;  // (not append) the step's row
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
    const bool off = normed && out_of_range<T, VEC>(a, ss);
    if (__any_sync(0xffffffffu, off)) {
      if (off) rescale_row<T, VEC, U>(ss, eps, x);
      ss = squares();
    }
    if (!live) continue;
    T* dst;
    if (!APPEND) {
      dst = yh;
    } else if (set == 0) {
      dst = (T*)a.y.p + t * a.y.ts + h * a.y.hs;
    } else {
      if (at < 0) continue;
      const int kh = h - a.n_x - (set == 2 ? a.n_kv : 0);
      dst = (T*)(set == 2 ? a.V_pages : a.K_pages) + at + kh * a.pv.head_stride;
    }
    if (set < 2) {
      load_factors(set);
      const float inv = normed ? __frsqrt_rn(fmaf(ss, a.inv_d, eps)) : 1.f;
      const NormWeight& w = set == 0 ? a.wx : a.wk;
      if (HEADS && normed) {
#pragma unroll
        for (int j = 0; j < U; ++j) {
          Part<VEC> wt;
          load_weight<T, VEC, PAIRS>(w, set == 0 ? h : h - a.n_x, place.c1[j], place.c2[j], wt);
          each_two<VEC>(x[j], [&](int i, float2& lo, float2& hi) {
            lo = __fmul2_rn(lo, two(wt.lo, i));
            hi = __fmul2_rn(hi, two(wt.hi, i));
          });
        }
      }
#pragma unroll
      for (int j = 0; j < U; ++j) {
        f[j].template turn<PAIRS>(place.turn(j), place.turn_all(j), inv, x[j]);
        Piece<T, VEC> out;
        narrow<T, VEC, PAIRS>(x[j], out);
        // (what is neither normalised nor turned is copied: arithmetic would flush subnormals)
        if (!APPEND || normed || place.turn(j)) r[0][j].a = out.a;
        if (!APPEND || normed || place.turn_all(j)) r[0][j].b = out.b;
      }
    }
#pragma unroll
    for (int j = 0; j < U; ++j) {
      if (place.first(j)) store_chunk<T, VEC>(dst + place.c1[j], r[0][j].a);
      if (place.second(j)) store_chunk<T, VEC>(dst + place.c2[j], r[0][j].b);
    }
  }
}

template <typename T, int VEC, bool PAIRS, bool APPEND, int U, int FL, bool ALL>
ebd_status launch_norm_u(NormArgs a, cudaStream_t s) {
  const int heads = a.n_x + (APPEND ? 2 * a.n_kv : 0);
  // one row per lane while the call has fewer warps than the GPU holds (latency), up to
  // sixteen pairs of chunks per lane beyond that
  const long long units = (long long)heads * a.lanes;
  const long long many = (units + 31) / 32, few = (units * U + 511) / 512;
  a.parts = (int)(many * a.n_tokens <= (long long)sm_count() * 32 ? many : few);
  const long long blocks = ((long long)a.n_tokens * a.parts + kNormWarps - 1) / kNormWarps;
  if (blocks > 0x7fffffffLL) return EBD_ERR_UNSUPPORTED;
  const bool each = (a.wx.p && a.wx.hs) || (APPEND && a.wk.p && a.wk.hs);
  return launch_dependent(each ? norm_rotary_kernel<T, VEC, PAIRS, APPEND, U, FL, ALL, true>
                               : norm_rotary_kernel<T, VEC, PAIRS, APPEND, U, FL, ALL, false>,
                          dim3((unsigned)blocks), kNormWarps * 32, 0, s, a);
}

}  // namespace ebd
