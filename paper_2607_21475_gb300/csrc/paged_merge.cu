// Joins the pieces of attention items that several CTAs worked on:
//   y = sum_p 2^(s_p - M) o_p / sum_p 2^(s_p - M),  lse = (M + log2 sum_p 2^(s_p - M)) ln 2,
// over the pieces p, with o_p each piece's own weighted mean and s_p its log2-sum
// (M the largest).  A warp joins 16 channels of up to 32 rows, a row per lane; where
// an item has 8 or 16 rows at most, 4 or 2 lanes share a row's pieces and add
// up in a fixed order.  The partial results were written just before and come
// from L2.  What bounds it is its chain of loads (records, pieces):
// 4.5-7 us for 151 items of up to 35 rows or of 256 rows x 64 channels, 12 us for 151
// of 256 x 128.
// Launched as a programmatic dependent of the attention kernel.
#include <cuda_runtime.h>
#include <math.h>

#include "decode_tile.cuh"
#include "paged_attn.cuh"

namespace ebd {

constexpr int kMergeWarps = 8;
constexpr int kMergeChannels = 16;

__device__ __forceinline__ void store16(float* p, const float (&v)[16]) {
#pragma unroll
  for (int i = 0; i < 4; ++i)
    reinterpret_cast<float4*>(p)[i] =
        make_float4(v[4 * i], v[4 * i + 1], v[4 * i + 2], v[4 * i + 3]);
}
__device__ __forceinline__ void store16(__nv_bfloat16* p, const float (&v)[16]) {
#pragma unroll
  for (int i = 0; i < 2; ++i)
    reinterpret_cast<uint4*>(p)[i] =
        make_uint4(pack_bf16(v[8 * i], v[8 * i + 1]), pack_bf16(v[8 * i + 2], v[8 * i + 3]),
                   pack_bf16(v[8 * i + 4], v[8 * i + 5]), pack_bf16(v[8 * i + 6], v[8 * i + 7]));
}

// FLIGHT: pieces of a lane in flight.
template <typename T, int D, int FLIGHT>
__global__ void __launch_bounds__(kMergeWarps * 32)
    paged_merge_kernel(const PagedAttnArgs a, int n_cta) {
  grid_dependency_wait();
  const int c0 = blockIdx.x, lane = threadIdx.x & 31;
  const PieceRecord r = a.rec[c0];
  // the item goes on through the first pieces of the following CTAs: up to the
  // first that does not just continue it (32 records at a time)
  int c1 = c0 + 1;
  bool on = c1 + lane < n_cta - 1 && a.rec[c1 + lane].cont == 1;
  if (r.tokens < 1 || r.tokens > a.tokens || r.token < 0 || r.token > a.n_tokens - r.tokens ||
      (unsigned)r.h >= (unsigned)a.heads)
    return;  // none begun here
  const int rows = r.tokens * a.slice;
  // this warp's rows of the slot (its second half starts at row 128) and channels
  constexpr int kParts = D / kMergeChannels;
  const int task = blockIdx.y * kMergeWarps + (threadIdx.x >> 5);
  const int part = task % kParts, row0 = task / kParts * 32;
  const int half_rows = a.half_tokens * a.slice;
  if (row0 >= (rows > half_rows ? 128 + rows - half_rows : rows)) return;
  const HeadSlice hs = head_slice(a, r.h);
  for (;;) {
    const uint32_t off = ~__ballot_sync(0xffffffffu, on);
    if (off) {
      c1 += __ffs(off) - 1;
      break;
    }
    c1 += 32;
    on = c1 + lane < n_cta - 1 && a.rec[c1 + lane].cont == 1;
  }
  const int n = c1 - c0 + 1;
  // lanes: `wide` rows, 32 / wide lanes share a row's pieces
  const int wide = rows <= 8 ? 8 : rows <= 16 ? 16 : 32;
  const int row = row0 + (lane & (wide - 1)), k0 = lane / wide, by = 32 / wide;
  const int i = row < 128 ? row : half_rows + row - 128;  // row of the item
  const bool live = i < rows && (row >= 128 || i < half_rows);
  float M = -INFINITY, sum = 0.f, o[kMergeChannels] = {};
  for (int k = k0; k < n && live; k += by * FLIGHT) {
    float s[FLIGHT];
    float4 v[FLIGHT][kMergeChannels / 4];
#pragma unroll
    for (int e = 0; e < FLIGHT; ++e) {
      const int p = k + e * by, slot = 2 * (c0 + p) + (p == 0);
      s[e] = -INFINITY;
      if (p < n) {
        s[e] = a.part_lse[(size_t)slot * a.slot_rows + row];
        const float* src = part_row<D>(a, slot, row) + part * (kMergeChannels / 4) * a.part_step;
#pragma unroll
        for (int c = 0; c < kMergeChannels / 4; ++c)
          v[e][c] = *reinterpret_cast<const float4*>(src + c * a.part_step);
      } else {
#pragma unroll
        for (int c = 0; c < kMergeChannels / 4; ++c) v[e][c] = make_float4(0.f, 0.f, 0.f, 0.f);
      }
    }
    float top = M;
#pragma unroll
    for (int e = 0; e < FLIGHT; ++e) top = fmaxf(top, s[e]);
    const float base = top == -INFINITY ? 0.f : top;
    const float f = exp2f(M - base);
    M = top;
    sum *= f;
#pragma unroll
    for (int c = 0; c < kMergeChannels; ++c) o[c] *= f;
#pragma unroll
    for (int e = 0; e < FLIGHT; ++e) {
      const float w = exp2f(s[e] - base);
      sum += w;
#pragma unroll
      for (int c = 0; c < kMergeChannels / 4; ++c) {
        o[4 * c] = fmaf(w, v[e][c].x, o[4 * c]);
        o[4 * c + 1] = fmaf(w, v[e][c].y, o[4 * c + 1]);
        o[4 * c + 2] = fmaf(w, v[e][c].z, o[4 * c + 2]);
        o[4 * c + 3] = fmaf(w, v[e][c].w, o[4 * c + 3]);
      }
    }
  }
  for (int x = wide; x < 32; x <<= 1) {
    const float m1 = __shfl_xor_sync(0xffffffffu, M, x), s1 = __shfl_xor_sync(0xffffffffu, sum, x);
    const float top = fmaxf(M, m1), base = top == -INFINITY ? 0.f : top;
    const float f0 = exp2f(M - base), f1 = exp2f(m1 - base);
    M = top;
    sum = sum * f0 + s1 * f1;
#pragma unroll
    for (int c = 0; c < kMergeChannels; ++c)
      o[c] = o[c] * f0 + __shfl_xor_sync(0xffffffffu, o[c], x) * f1;
  }
  const int t = i / a.slice, g = i - t * a.slice;
  if (!live || k0 > 0 || g >= hs.n) return;
  const long long out =
      (long long)(r.token + t) * (a.pv.n_kv_heads * a.group) + hs.q0 + g;
  const float inv = sum == 0.f ? 0.f : 1.f / sum;
#pragma unroll
  for (int c = 0; c < kMergeChannels; ++c) o[c] *= inv;
  store16((T*)a.y + out * D + part * kMergeChannels, o);
  if (a.lse && part == 0) a.lse[out] = sum == 0.f ? -INFINITY : (M + log2f(sum)) * kLn2;
}

size_t paged_split_bytes(int n_cta, int slot_rows, int head_dim) {
  const size_t rows = (size_t)2 * n_cta * slot_rows;
  return align_up(n_cta * sizeof(PieceRecord), 256) + align_up(rows * 4, 256) +
         rows * head_dim * 4;
}

void paged_split_layout(PagedAttnArgs& a, void* ws, int n_cta) {
  char* p = (char*)ws;
  a.rec = (PieceRecord*)p;
  p += align_up(n_cta * sizeof(PieceRecord), 256);
  a.part_lse = (float*)p;
  p += align_up((size_t)2 * n_cta * a.slot_rows * 4, 256);
  a.part_o = (float*)p;
  a.part_step = 4 * (a.slot_rows < 32 ? a.slot_rows : 32);
}

template <typename T, int D>
static ebd_status launch_merge_t(const PagedAttnArgs& a, int n_cta, cudaStream_t s) {
  const int rows = a.slot_rows > 32 ? a.slot_rows : 32;
  const int tasks = (rows + 31) / 32 * (D / kMergeChannels);
  const dim3 grid(n_cta - 1, (tasks + kMergeWarps - 1) / kMergeWarps);
  // items of few rows often have many pieces, and there are few warps then
  if (a.slot_rows <= 32)
    return launch_dependent(paged_merge_kernel<T, D, 4>, grid, kMergeWarps * 32, 0, s, a, n_cta);
  return launch_dependent(paged_merge_kernel<T, D, 2>, grid, kMergeWarps * 32, 0, s, a, n_cta);
}

ebd_status launch_paged_merge(const PagedAttnArgs& a, bool bf16, int head_dim, int n_cta,
                              cudaStream_t s) {
  if (n_cta <= 1) return EBD_OK;
  if (bf16)
    return head_dim == 128 ? launch_merge_t<__nv_bfloat16, 128>(a, n_cta, s)
                           : launch_merge_t<__nv_bfloat16, 64>(a, n_cta, s);
  return head_dim == 128 ? launch_merge_t<float, 128>(a, n_cta, s)
                         : launch_merge_t<float, 64>(a, n_cta, s);
}

}  // namespace ebd
