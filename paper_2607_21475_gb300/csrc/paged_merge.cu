// Joins the pieces of attention items that several CTAs worked on:
//   y = sum_p 2^(s_p - M) o_p / sum_p 2^(s_p - M),  lse = (M + log2 sum_p 2^(s_p - M)) ln 2,
// over the pieces p in CTA order, with o_p each piece's own weighted mean and
// s_p its log2-sum (M the largest).  A warp joins one row, or four at a time where
// an item has many rows of few pieces; the partial results were written just
// before and come from L2.  What bounds it is its chain of loads (record, span,
// weights, rows): 5-9 us for 151 items of 4 to 256 rows.  Launched as a
// programmatic dependent of the attention kernel.
#include <cuda_runtime.h>
#include <math.h>

#include "decode_tile.cuh"
#include "paged_attn.cuh"

namespace ebd {

constexpr int kMergeWarps = 8;
constexpr int kMergeFlight = 4;  // pieces in flight per warp

__device__ __forceinline__ void store_row(float* p, int lane, float4 v) {
  reinterpret_cast<float4*>(p)[lane] = v;
}
__device__ __forceinline__ void store_row(float* p, int lane, float2 v) {
  reinterpret_cast<float2*>(p)[lane] = v;
}
__device__ __forceinline__ void store_row(__nv_bfloat16* p, int lane, float4 v) {
  reinterpret_cast<uint2*>(p)[lane] = make_uint2(pack_bf16(v.x, v.y), pack_bf16(v.z, v.w));
}
__device__ __forceinline__ void store_row(__nv_bfloat16* p, int lane, float2 v) {
  reinterpret_cast<uint32_t*>(p)[lane] = pack_bf16(v.x, v.y);
}
__device__ __forceinline__ void add_scaled(float4& o, float f, const float4& v) {
  o.x = fmaf(f, v.x, o.x);
  o.y = fmaf(f, v.y, o.y);
  o.z = fmaf(f, v.z, o.z);
  o.w = fmaf(f, v.w, o.w);
}
__device__ __forceinline__ void add_scaled(float2& o, float f, const float2& v) {
  o.x = fmaf(f, v.x, o.x);
  o.y = fmaf(f, v.y, o.y);
}
__device__ __forceinline__ float4 scaled(const float4& v, float f) {
  return make_float4(v.x * f, v.y * f, v.z * f, v.w * f);
}
__device__ __forceinline__ float2 scaled(const float2& v, float f) {
  return make_float2(v.x * f, v.y * f);
}

// VT: the float vector that a lane of a warp owns of a row (D / 32 floats).
template <typename T, typename VT>
__global__ void __launch_bounds__(kMergeWarps * 32)
    paged_merge_kernel(const PagedAttnArgs a, int n_cta) {
  grid_dependency_wait();
  const int c0 = blockIdx.x, lane = threadIdx.x & 31;
  const PieceRecord r = a.rec[c0];
  if ((unsigned)r.b >= (unsigned)a.pv.batch) return;
  const SeqSpan sp = seq_span(a.pv, a.cu, r.b, a.n_tokens, a.max_new);
  const int rows = min(a.tokens, sp.n - r.m * a.tokens) * a.slice;
  const HeadSlice hs = head_slice(a, r.h);
  // the item goes on through the first pieces of the following CTAs: up to the
  // first that does not just continue it (32 records at a time)
  int c1 = c0 + 1;
  for (;; c1 += 32) {
    const bool on = c1 + lane < n_cta - 1 && a.rec[c1 + lane].cont == 1;
    const uint32_t off = ~__ballot_sync(0xffffffffu, on);
    if (off) {
      c1 += __ffs(off) - 1;
      break;
    }
  }
  constexpr int D = 32 * (int)(sizeof(VT) / 4);
  const int hq = a.pv.n_kv_heads * a.group;
  const int n = c1 - c0 + 1;
  // piece k of row `row` in part_lse, and (times D) in part_o
  const auto place = [&](int k, int row) {
    return (size_t)(2 * (c0 + k) + (k == 0)) * a.slot_rows + row;
  };
  // row i of the item is token t, head g; the slot's second half starts at row 128
  const auto row_of = [&](int i) {
    return i < a.half_tokens * a.slice ? i : 128 + i - a.half_tokens * a.slice;
  };
  const auto write = [&](int i, const VT& o, float sum, float M) {
    const int t = i / a.slice, g = i - t * a.slice;
    if (g >= hs.n) return;
    const long long out = (long long)(sp.t0 + r.m * a.tokens + t) * hq + hs.q0 + g;
    store_row((T*)a.y + out * D, lane, scaled(o, sum == 0.f ? 0.f : 1.f / sum));
    if (a.lse && lane == 0) a.lse[out] = sum == 0.f ? -INFINITY : (M + log2f(sum)) * kLn2;
  };
  const int w0 = blockIdx.y * kMergeWarps + (threadIdx.x >> 5), ws = gridDim.y * kMergeWarps;
  if (n <= 8 && rows > 64) {
    // few pieces of many rows: four rows at a time, lane 8 e + k weighs piece k of row e
    for (int i0 = w0 * 4; i0 < rows; i0 += ws * 4) {
      VT v[4][2];  // the first two pieces' rows do not wait for the weights
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const int row = row_of(min(i0 + e, rows - 1));
#pragma unroll
        for (int k = 0; k < 2; ++k)
          v[e][k] = reinterpret_cast<const VT*>(a.part_o + place(k, row) * D)[lane];
      }
      const float s = (lane & 7) < n
                          ? a.part_lse[place(lane & 7, row_of(min(i0 + (lane >> 3), rows - 1)))]
                          : -INFINITY;
      float M = s;
#pragma unroll
      for (int o = 1; o < 8; o <<= 1) M = fmaxf(M, __shfl_xor_sync(0xffffffffu, M, o));
      const float f = exp2f(s - (M == -INFINITY ? 0.f : M));
      float sum = f;
#pragma unroll
      for (int o = 1; o < 8; o <<= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        VT o = {};
#pragma unroll
        for (int k = 0; k < 2; ++k)
          add_scaled(o, __shfl_sync(0xffffffffu, f, 8 * e + k), v[e][k]);
        const int row = row_of(min(i0 + e, rows - 1));
        for (int k = 2; k < n; ++k)
          add_scaled(o, __shfl_sync(0xffffffffu, f, 8 * e + k),
                     reinterpret_cast<const VT*>(a.part_o + place(k, row) * D)[lane]);
        const float se = __shfl_sync(0xffffffffu, sum, 8 * e);
        const float me = __shfl_sync(0xffffffffu, M, 8 * e);
        if (i0 + e < rows) write(i0 + e, o, se, me);
      }
    }
    return;
  }
  for (int i = w0; i < rows; i += ws) {
    const int row = row_of(i);
    // lane k keeps the weight of piece k of 32; the rows' loads do not wait for it
    float s0 = lane < n ? a.part_lse[place(lane, row)] : -INFINITY;
    float M = s0;
    for (int k = 32 + lane; k < n; k += 32) M = fmaxf(M, a.part_lse[place(k, row)]);
    M = warp_max(M);
    const float base = M == -INFINITY ? 0.f : M;
    float sum = 0.f;
    VT o = {};
    for (int k0 = 0; k0 < n; k0 += 32) {
      if (k0 > 0) s0 = k0 + lane < n ? a.part_lse[place(k0 + lane, row)] : -INFINITY;
      const float f = exp2f(s0 - base);
      sum += f;
      const int k = min(32, n - k0);
      for (int j = 0; j < k; j += kMergeFlight) {
        VT v[kMergeFlight];
#pragma unroll
        for (int e = 0; e < kMergeFlight; ++e)
          if (j + e < k)
            v[e] = reinterpret_cast<const VT*>(a.part_o + place(k0 + j + e, row) * D)[lane];
#pragma unroll
        for (int e = 0; e < kMergeFlight; ++e) {
          const float fe = __shfl_sync(0xffffffffu, f, (j + e) & 31);
          if (j + e < k) add_scaled(o, fe, v[e]);
        }
      }
    }
    write(i, o, warp_sum(sum), M);
  }
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
}

ebd_status launch_paged_merge(const PagedAttnArgs& a, bool bf16, int head_dim, int n_cta,
                              cudaStream_t s) {
  if (n_cta <= 1) return EBD_OK;
  // large items are joined four rows per warp (256 rows of 2 pieces: 13.4 us for 151
  // items, a row per warp 18.2), small ones, often of many pieces, a row per warp
  const int most = min(a.max_new, a.tokens) * a.slice;
  const int per_block = most > 64 ? 4 * kMergeWarps : kMergeWarps;
  const dim3 grid(n_cta - 1, (most + per_block - 1) / per_block);
  const int threads = kMergeWarps * 32;
  if (bf16 && head_dim == 128)
    return launch_dependent(paged_merge_kernel<__nv_bfloat16, float4>, grid, threads, 0, s, a,
                            n_cta);
  if (bf16)
    return launch_dependent(paged_merge_kernel<__nv_bfloat16, float2>, grid, threads, 0, s, a,
                            n_cta);
  if (head_dim == 128)
    return launch_dependent(paged_merge_kernel<float, float4>, grid, threads, 0, s, a, n_cta);
  return launch_dependent(paged_merge_kernel<float, float2>, grid, threads, 0, s, a, n_cta);
}

}  // namespace ebd
