// The gradient of the norms with the rotation (mathematics and figures: norm.cuh).
#include "norm.cuh"

namespace ebd {

// PER_HEAD: a block has one head (blockIdx.y), a warp's groups of lanes have tokens; else
// they have heads of a token.  Leaves the block's sum of the weight's gradient in
// partial[blockIdx.x][blockIdx.y][d]; without partial the grid's rows of blocks are clusters,
// which add their blocks' sums up through distributed shared memory.
template <typename T, int VEC, bool PAIRS, int U, bool PER_HEAD, int FL, bool ALL>
__global__ void __launch_bounds__(kNormWarps * 32, norm_blocks(kNormBackBlocks, U, VEC))
    norm_backward_kernel(const NormArgs a, float* __restrict__ partial,
                         float* __restrict__ dweight) {
  extern __shared__ __align__(16) unsigned char smem[];  // the rows' ring; then, in its place:
  float* red = reinterpret_cast<float*>(smem);           // [warps][units of all lanes][2 VEC]
  using Ring = RowRing<T, VEC, U, 2>;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const Place<VEC, PAIRS, U, FL, ALL> place(a, lane);
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
        if (place.turn(j))
          load_angles<VEC, PAIRS>(a, tpos, place.c1[j], place.c2[j], place.turn_all(j), angles[j]);
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
    const bool off = live && out_of_range<T, VEC>(a, ss);
    if (__any_sync(0xffffffffu, off)) {
      if (off) scale = rescale_row<T, VEC, U>(ss, eps, x);
      sums();
    }
    if (!live) continue;
    T* out = (T*)a.y.p + at.t * a.y.ts + at.h * a.y.hs;
    const float inv = __frsqrt_rn(fmaf(ss, a.inv_d, eps));
    const float2 inv2 = both(inv);
    const float2 mean = both(-gx * inv * a.inv_d * inv);  // -r mean of g z, up to the row's scale
#pragma unroll
    for (int j = 0; j < U; ++j) {
      each_two<VEC>(x[j], [&](int i, float2& lo, float2& hi) {
        const float2 z0 = __fmul2_rn(lo, inv2), z1 = __fmul2_rn(hi, inv2);
        const float2 u0 = two(u[j].lo, i), u1 = two(u[j].hi, i);
        const float2 a0 = __ffma2_rn(u0, z0, two(acc[j].lo, i));
        const float2 a1 = __ffma2_rn(u1, z1, two(acc[j].hi, i));
        acc[j].lo[i] = a0.x, acc[j].hi[i] = a1.x;
        if constexpr (VEC > 1) acc[j].lo[i + 1] = a0.y, acc[j].hi[i + 1] = a1.y;
        lo = __ffma2_rn(z0, mean, __fmul2_rn(__fmul2_rn(u0, two(wt[j].lo, i)), inv2));
        hi = __ffma2_rn(z1, mean, __fmul2_rn(__fmul2_rn(u1, two(wt[j].hi, i)), inv2));
      });
      if (off)  // (last: r itself may lie below float32's normal numbers)
        each_two<VEC>(x[j], [&](int, float2& lo, float2& hi) {
          lo = __fmul2_rn(lo, both(scale));
          hi = __fmul2_rn(hi, both(scale));
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
  float* sum = red + kNormWarps * wide;  // (clusters)
  float* dst =
      partial ? partial + ((size_t)blockIdx.x * gridDim.y + blockIdx.y) * a.head_dim : sum;
  for (int k = threadIdx.x; k < wide; k += kNormWarps * 32) {
    const int u = k / (2 * VEC), i = k - u * 2 * VEC, e = i % VEC;
    if (!PAIRS && u >= a.units) continue;
    int c1, c2;
    Place<VEC, PAIRS, U, FL, ALL>::channels(a, L, u & (L - 1), u / L, c1, c2);
    // lo[e] (i < VEC) and hi[e]: chunk and element
    const bool second = PAIRS ? e >= VEC / 2 : i >= VEC;
    if ((second ? c2 : c1) < 0) continue;
    const int c = (second ? c2 : c1) + (PAIRS ? 2 * e % VEC + (i >= VEC) : e);
    float v = 0.f;
#pragma unroll
    for (int x = 0; x < kNormWarps; ++x) v += red[x * wide + k];
    dst[c] = v;
  }
  if (partial) return;
  __syncwarp();
  cluster_barrier();
  const uint32_t ranks = gridDim.x, rank = cluster_rank();
  for (int c = rank * kNormWarps * 32 + threadIdx.x; c < a.head_dim; c += ranks * kNormWarps * 32) {
    float v = 0.f;
    for (uint32_t r = 0; r < ranks; ++r) v += ld_cluster_f32(cluster_map(smem_u32(sum + c), r));
    dweight[(size_t)blockIdx.y * a.head_dim + c] = v;
  }
  __syncwarp();
  cluster_barrier();  // no block leaves while another reads its sum
}

// dweight[i] = sum over the n blocks of partial[block][i], i < total; 32 columns per block,
// warp w sums the blocks w, w + 32, .., and the warps' sums are added in a fixed order.
// (It begins before the other kernel ends: its loads are not declared constant.)
constexpr int kReduceWarps = 32;
__global__ void __launch_bounds__(kReduceWarps * 32)
    norm_weight_reduce_kernel(const float* partial, int n, int total, float* dweight) {
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

// Blocks of the backward pass along its rows (times the heads where each has a weight).
static int norm_back_blocks(long long steps, int heads) {
  const long long want = (steps + kNormWarps - 1) / kNormWarps;
  long long most = (long long)sm_count() * kNormBackBlocks / heads;
  if (most < 1) most = 1;
  return (int)(want < most ? want : most);
}

constexpr int kNormCluster = 16;  // blocks of a cluster at most
// Steps (of a row of blocks) that one cluster takes: one to each of its warps.  It then saves
// the second launch; with a second step per warp that launch's many blocks are the quicker.  One
// cluster against two launches, us in a graph (in a row of calls): 28 heads x 128, bf16, 7 steps
// 3.7 / 4.1 (4.3 / 5.3), 126 4.2 / 4.5 (4.7 / 5.2), 252 5.2 / 4.6 (5.7 / 5.2), 1022 8.9 / 6.2
// (9.5 / 6.6); a weight per head, 4 x 64, f32, 128 steps 3.6 / 3.9 (4.1 / 5.4), 256 4.5 / 4.1 (5.2 /
// 5.3), 512 6.1 / 4.4 (7.1 / 5.3).
constexpr int kNormFewSteps = kNormCluster * kNormWarps;

template <typename T, int VEC, bool PAIRS, int U, int FL, bool ALL>
ebd_status launch_norm_back_u(NormArgs a, const NormBackward& bw, cudaStream_t s) {
  const bool per_head = a.wx.hs != 0;
  const int per_warp = 32 / a.lanes;
  const long long steps = per_head ? (a.n_tokens + per_warp - 1) / per_warp
                                   : (long long)a.n_tokens * ((a.n_x + per_warp - 1) / per_warp);
  const int rows = per_head ? a.n_x : 1;  // of blocks: those that share a weight's gradient
  // Few steps: a cluster per row, which adds its sums up itself, in place of a second launch.
  const bool few = steps <= kNormFewSteps;
  const int most = norm_back_blocks(steps, rows);
  int blocks = most;
  if (few) blocks = (int)((steps + kNormWarps - 1) / kNormWarps);
  if (few && blocks > kNormCluster) blocks = kNormCluster;
  const int total = rows * a.head_dim;
  const int sums = kNormWarps * a.lanes * U * 2 * VEC * 4 + (few ? a.head_dim * 4 : 0);
  const int ring = RowRing<T, VEC, U, 2>::kBytes, smem = sums > ring ? sums : ring;
  auto kern = per_head ? norm_backward_kernel<T, VEC, PAIRS, U, true, FL, ALL>
                       : norm_backward_kernel<T, VEC, PAIRS, U, false, FL, ALL>;
  if (smem > 48 * 1024 &&
      cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, smem) != cudaSuccess)
    return EBD_ERR_CUDA;
  static ClusterMemo memo[2];
  if (few) blocks = cluster_ctas(blocks, kNormCluster, memo[per_head], kern, kNormWarps * 32, smem);
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(blocks, rows);
  cfg.blockDim = dim3(kNormWarps * 32);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = s;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = blocks;
  attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = few ? 2 : 1;
  float* partial = few ? nullptr : bw.partial;
  const ebd_status st = cuda_status(cudaLaunchKernelEx(&cfg, kern, a, partial, bw.dweight));
  if (st != EBD_OK || few) return st;
  return launch_dependent(norm_weight_reduce_kernel, dim3((total + 31) / 32), kReduceWarps * 32, 0, s,
                          (const float*)bw.partial, blocks, total, bw.dweight);
}

}  // namespace ebd

using namespace ebd;

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
  return dtype == EBD_F32 ? launch_norm_t<float, kNormBackward>(a, pairs, &bw, s)
                          : launch_norm_t<__nv_bfloat16, kNormBackward>(a, pairs, &bw, s);
}
