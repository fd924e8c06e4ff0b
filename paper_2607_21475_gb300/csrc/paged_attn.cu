// Attention of each sequence's new tokens over its paged cache,
//   y_i = sum_j softmax_j(scale q_i . k_j) v_j,  max(0, p_i - window + 1) <= j <= p_i,
// and its log-sum-exp: the entry point, and the float32 kernel (the bf16 one is
// in paged_attn_tc.cu).
//
// Online softmax: running maximum m, sum l and output o in float32, rescaled by
// e^(m - m') when a tile raises the maximum.  An item is 32 rows, keys come in
// tiles of 32 (four CTAs per SM at 64 channels, two at 128), the next tile copied
// by cp.async while this one is worked on.  128 threads as 8 x 16: thread (ty, tx)
// owns rows 4 ty .. + 3, keys tx + 16 j of a tile's logits and channels 4 tx + 64 j
// of the output; the weights go through shared memory, four keys to a load.
// Measured: three ragged prompts of up to 512 tokens (4 heads x 64) 30.7 us:
// finding the work and the first tile 5 us, four tiles per CTA at 2140 cycles per
// tile and SM (FMAs 1024; reads of shared memory bound them), the merge 7 us.  Single
// tokens use one warp of the four: 8 sequences of 4k (32/8 heads x 128) 98 us, 2.7 TB/s.
#include <cuda_runtime.h>
#include <math.h>

#include "common.cuh"
#include "decode_tile.cuh"
#include "internal.h"
#include "paged_attn.cuh"
#include "ptx.cuh"

namespace ebd {

constexpr int kAttnRows = 32;
constexpr int kAttnThreads = 128;

template <int D>
struct SimtLayout {
  static constexpr int kKeys = 32;
  static constexpr int kCtasPerSm = D == 128 ? 2 : 4;
  static constexpr int kQ = 0;  // [rows][D + 4]
  static constexpr int kK = kQ + kAttnRows * (D + 4);      // [2][keys][D + 4]
  static constexpr int kV = kK + 2 * kKeys * (D + 4);      // [2][keys][D]
  static constexpr int kP = kV + 2 * kKeys * D;            // [rows][keys + 4]
  static constexpr int kOff = kP + kAttnRows * (kKeys + 4);  // [2][keys] row offsets, 64 bits
  static constexpr int kStart = kOff + 4 * kKeys;
  static constexpr int kAbsent = kStart + 12;  // [4] keys of a tile without a row, by tile number
  static constexpr int kFloats = kAbsent + 4;
};

__device__ __forceinline__ void load4(const float* p, float (&x)[4]) {
  const float4 v = *reinterpret_cast<const float4*>(p);
  x[0] = v.x; x[1] = v.y; x[2] = v.z; x[3] = v.w;
}
__device__ __forceinline__ void store4(float* p, const float (&x)[4]) {
  *reinterpret_cast<float4*>(p) = make_float4(x[0], x[1], x[2], x[3]);
}
// 16 bytes global -> shared; zeros when `ok` is false (nothing is read then).
__device__ __forceinline__ void cp_async16_or_zero(void* dst, const void* src, bool ok) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(smem_u32(dst)), "l"(src),
               "r"(ok ? 16 : 0)
               : "memory");
}

template <int D>
__global__ void __launch_bounds__(kAttnThreads, SimtLayout<D>::kCtasPerSm)
    paged_attn_f32_kernel(const PagedAttnArgs a) {
  using L = SimtLayout<D>;
  constexpr int BN = L::kKeys, NK = BN / 16;  // keys per thread
  extern __shared__ float4 smem4[];
  float* sm = reinterpret_cast<float*>(smem4);
  float *Qs = sm + L::kQ, *Ps = sm + L::kP;
  long long* offs = reinterpret_cast<long long*>(sm + L::kOff);
  uint32_t* absent_s = reinterpret_cast<uint32_t*>(sm + L::kAbsent);
  const int tx = threadIdx.x & 15, ty = threadIdx.x >> 4;
  WorkStart* start_s = reinterpret_cast<WorkStart*>(sm + L::kStart);
  static_assert(sizeof(WorkStart) <= 12 * 4, "start");
  grid_dependency_wait();
  if (threadIdx.x < 32) {
    const WorkStart w = find_work<BN>(a, blockIdx.x, gridDim.x, threadIdx.x);
    if (threadIdx.x == 0) *start_s = w;
  }
  __syncthreads();
  bool bad = false, first = true;
  bool nan = false;  // a NaN in this thread's outputs
  PieceRecord record = {0, 0, 0, 0};
  for (PieceWalk<BN> w(a, *start_s); w.live(); w.next(a)) {
    record_piece(a, record, w, first);
    first = false;
    const HeadSlice hs = head_slice(a, w.h);
    const int tokens = w.tokens(a), t_first = w.sp.t0 + w.first(a);
    const int p0 = w.sp.len - w.sp.n + w.first(a);  // position of the item's first token
    const int seen = first_seen(a, p0);  // pages before it may have been released
    // Row threadIdx.x of key tile j: its offset in the pools; -1 past the sequence's
    // end, where nothing is read
    auto find_row = [&](int j) {
      const int pos = j * BN + threadIdx.x;
      if (pos >= w.sp.len) return -1ll;
      const int page = page_of(a.pv, w.b, pos);
      bad |= page < 0 && pos >= seen;
      return page < 0 ? -1ll : slot_offset(a.pv, page, hs.kvh, pos);
    };
    auto copy = [&](int j) {  // key tile j into stage j & 1
      float *Ks = sm + L::kK + (j & 1) * BN * (D + 4), *Vs = sm + L::kV + (j & 1) * BN * D;
      const long long* off = offs + (j & 1) * BN;
#pragma unroll
      for (int i = threadIdx.x; i < BN * (D / 4); i += kAttnThreads) {
        const int r = i / (D / 4), c = i % (D / 4) * 4;
        const long long o = off[r];
        cp_async16_or_zero(Ks + r * (D + 4) + c, (const float*)a.K_pages + max(o, 0ll) + c, o >= 0);
        cp_async16_or_zero(Vs + r * D + c, (const float*)a.V_pages + max(o, 0ll) + c, o >= 0);
      }
      cp_async_commit();
    };
    // Enters the rows that the first warp found.  A tile's absent keys are read while
    // it is worked on, when the warp may be two tiles ahead: four places.
    auto put_row = [&](int j, long long row) {
      static_assert(BN == 32, "a lane per key");
      offs[(j & 1) * BN + threadIdx.x] = row;
      const uint32_t absent = __ballot_sync(0xffffffffu, row < 0);
      if (threadIdx.x == 0) absent_s[j & 3] = absent;
    };
    __syncthreads();  // the last piece's readers are done
    if (threadIdx.x < BN) {
      put_row(w.cur, find_row(w.cur));
      if (w.cur + 1 < w.end) put_row(w.cur + 1, find_row(w.cur + 1));
    }
    __syncthreads();
    copy(w.cur);
    for (int i = threadIdx.x; i < kAttnRows * (D / 4); i += kAttnThreads) {
      const int r = i / (D / 4), c = i % (D / 4) * 4, t = r / a.slice, g = r - t * a.slice;
      float x[4] = {0.f, 0.f, 0.f, 0.f};
      if (t < tokens && g < hs.n)
        load4((const float*)a.q + (t_first + t) * a.q_ts + (hs.q0 + g) * a.q_hs + c, x);
      store4(Qs + r * (D + 4) + c, x);
    }
    int hi[4], lo[4];  // keys that this thread's rows see
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int p = p0 + min((ty * 4 + i) / a.slice, tokens - 1);
      hi[i] = p + 1;
      lo[i] = first_seen(a, p);
    }
    float m[4], l[4], o[4][D / 16];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      m[i] = -INFINITY;
      l[i] = 0.f;
#pragma unroll
      for (int c = 0; c < D / 16; ++c) o[i][c] = 0.f;
    }
    // A warp whose 8 rows are all past the item's last leaves the arithmetic to the
    // others, which are bound by shared-memory reads
    const bool live = (threadIdx.x >> 5) * 8 < tokens * a.slice;
    for (int j = w.cur; j < w.end; ++j) {
      const int k0 = j * BN;
      const float *Ks = sm + L::kK + (j & 1) * BN * (D + 4), *Vs = sm + L::kV + (j & 1) * BN * D;
      cp_async_wait<0>();
      __syncthreads();  // tile j is there for all, and stage j + 1 is read no more
      if (j + 1 < w.end) copy(j + 1);
      // the rows of the tile after it: found while this one is worked on
      long long row = -1;
      if (j + 2 < w.end && threadIdx.x < BN) row = find_row(j + 2);
      if (live) {
        float s[4][NK] = {};
        // sums of 16 channels, then of those: one running sum of 128 has 2.3 times the
        // rounding error
#pragma unroll 1
        for (int c0 = 0; c0 < D; c0 += 16) {
          float part[4][NK] = {};
#pragma unroll
          for (int c = c0; c < c0 + 16; c += 4) {
            float q[4][4], k[NK][4];
#pragma unroll
            for (int i = 0; i < 4; ++i) load4(Qs + (ty * 4 + i) * (D + 4) + c, q[i]);
#pragma unroll
            for (int e = 0; e < NK; ++e) load4(Ks + (tx + 16 * e) * (D + 4) + c, k[e]);
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
              for (int e = 0; e < NK; ++e)
#pragma unroll
                for (int z = 0; z < 4; ++z) part[i][e] = fmaf(q[i][z], k[e][z], part[i][e]);
          }
#pragma unroll
          for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int e = 0; e < NK; ++e) s[i][e] += part[i][e];
        }
        const uint32_t absent = absent_s[j & 3];
        bool all = absent == 0;  // every row of the warp sees every key of the tile
#pragma unroll
        for (int i = 0; i < 4; ++i) all = all && lo[i] <= k0 && hi[i] >= k0 + BN;
        all = __all_sync(0xffffffffu, all);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          float top = m[i];
#pragma unroll
          for (int e = 0; e < NK; ++e) {
            const int pos = k0 + tx + 16 * e;
            s[i][e] = all || (pos >= lo[i] && pos < hi[i] && !(absent >> (tx + 16 * e) & 1))
                          ? s[i][e]
                          : -INFINITY;
            top = fmaxf(top, s[i][e]);
          }
#pragma unroll
          for (int x = 8; x > 0; x >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, x));
          // nothing seen yet: every weight is 0
          const float base = top == -INFINITY ? 0.f : __fmul_rn(top, a.scale2);
          const float f = exp2f(__fmul_rn(m[i], a.scale2) - base);
          m[i] = top;
          float sum = 0.f;
#pragma unroll
          for (int e = 0; e < NK; ++e) {
            // fused: a logit of 16 rounded first would leave 7e-7 in the largest weights
            const float p = exp2f(fmaf(s[i][e], a.scale2, -base));
            sum += p;
            Ps[(ty * 4 + i) * (BN + 4) + tx + 16 * e] = p;
          }
          l[i] = l[i] * f + sum;  // this thread's share
#pragma unroll
          for (int c = 0; c < D / 16; ++c) o[i][c] *= f;
        }
        __syncwarp();  // a warp reads the weights of its own rows only
        // hidden keys have weight 0; a hidden value that is not finite is mended at the end
#pragma unroll 2
        for (int k = 0; k < BN; k += 4) {
          float p[4][4];
#pragma unroll
          for (int i = 0; i < 4; ++i) load4(Ps + (ty * 4 + i) * (BN + 4) + k, p[i]);
#pragma unroll
          for (int z = 0; z < 4; ++z)
#pragma unroll
            for (int c = 0; c < D / 64; ++c) {
              float v[4];
              load4(Vs + (k + z) * D + c * 64 + tx * 4, v);
#pragma unroll
              for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int e = 0; e < 4; ++e)
                  o[i][c * 4 + e] = fmaf(p[i][z], v[e], o[i][c * 4 + e]);
            }
        }
      }
      // (stage j & 1's offsets were read before this tile's barrier)
      if (j + 2 < w.end && threadIdx.x < BN) put_row(j + 2, row);
      __syncwarp();  // before the next tile's weights
    }
    const int slot = w.slot(blockIdx.x);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
#pragma unroll
      for (int x = 8; x > 0; x >>= 1) l[i] += __shfl_xor_sync(0xffffffffu, l[i], x);
      const int r = ty * 4 + i, t = r / a.slice, g = r - t * a.slice;
      const bool mine = t < tokens && g < hs.n;
      const long long out = (long long)(t_first + t) * (a.pv.n_kv_heads * a.group) + hs.q0 + g;
      float* dst = slot < 0 ? (float*)a.y + out * D : part_row<D>(a, slot, r);
      const int step = slot < 0 ? 4 : a.part_step;  // between 4-channel groups
      const float inv = l[i] == 0.f ? 0.f : 1.f / l[i];
#pragma unroll
      for (int c = 0; c < D / 64; ++c) {
        float x[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          x[e] = o[i][c * 4 + e] * inv;
          nan = nan || (mine && x[e] != x[e]);
        }
        if (mine) store4(dst + (c * 16 + tx) * step, x);
      }
      const float lse2 =
          l[i] == 0.f ? -INFINITY : __fmul_rn(m[i], a.scale2) + log2f(l[i]);
      if (mine && tx == 0 && slot >= 0) a.part_lse[(size_t)slot * a.slot_rows + r] = lse2;
      if (mine && tx == 0 && slot < 0 && a.lse) a.lse[out] = lse2 * kLn2;
    }
  }
  if (__any_sync(0xffffffffu, nan))
    mend_pieces<float, D, BN>(a, blockIdx.x, gridDim.x, 0, 0, (threadIdx.x >> 5) * 8, 8,
                              threadIdx.x & 31);
  if (threadIdx.x == 0) a.rec[blockIdx.x] = record;
  if (bad) raise_status(a.dev_status, EBD_DEV_RANGE);
}

// Query heads per slice of a group: equal slices of at most kAttnRows heads.
static int f32_slice(int group) {
  const int slices = (group + kAttnRows - 1) / kAttnRows;
  return (group + slices - 1) / slices;
}

static int f32_ctas(int head_dim) {
  return sm_count() * (head_dim == 128 ? SimtLayout<128>::kCtasPerSm : SimtLayout<64>::kCtasPerSm);
}

template <int D>
static ebd_status launch_paged_f32(PagedAttnArgs a, int n_cta, cudaStream_t s) {
  const int smem = SimtLayout<D>::kFloats * 4;
  if (cudaFuncSetAttribute(paged_attn_f32_kernel<D>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                           smem) != cudaSuccess)
    return EBD_ERR_CUDA;
  const int slice = f32_slice(a.group);
  a.slices = (a.group + slice - 1) / slice;
  a.slice = slice;
  a.heads = a.pv.n_kv_heads * a.slices;
  a.tokens = a.half_tokens = kAttnRows / a.slice;
  a.tile_work = a.full_work = 1;
  a.min_share = 2;
  a.item_cost = 1;
  if (!line_fits(a, SimtLayout<D>::kKeys)) return EBD_ERR_UNSUPPORTED;
  const ebd_status st =
      launch_dependent(paged_attn_f32_kernel<D>, dim3(n_cta), kAttnThreads, smem, s, a);
  if (st != EBD_OK) return st;
  return launch_paged_merge(a, false, D, n_cta, s);
}

}  // namespace ebd

using namespace ebd;

namespace ebd {

static int attention_ctas(const ebd_paged_cache& c) {
  return c.dtype == EBD_F32 ? f32_ctas(c.head_dim) : sm_count();
}

static int attention_slot_rows(const ebd_paged_cache& c, int group, int max_new) {
  if (c.dtype == EBD_F32) {
    const int slice = f32_slice(group);
    return paged_slot_rows(max_new, kAttnRows / slice, slice, kAttnRows);
  }
  return paged_slot_rows(max_new, 128 / group, group, kTcRows);
}

}  // namespace ebd

extern "C" size_t ebd_paged_attention_workspace_bytes(const ebd_paged_cache* cache,
                                                      int32_t n_q_heads, int32_t max_new) {
  if (check_paged(cache) != EBD_OK || n_q_heads < 1 || max_new < 1) return 0;
  if (n_q_heads % cache->n_kv_heads != 0) return 0;
  const int group = n_q_heads / cache->n_kv_heads;
  if (group > 128) return 0;
  return paged_split_bytes(attention_ctas(*cache), attention_slot_rows(*cache, group, max_new),
                           cache->head_dim);
}

extern "C" ebd_status ebd_paged_attention(const ebd_paged_cache* cache, int32_t n_tokens,
                                          int32_t max_new, int32_t n_q_heads,
                                          const int32_t* cu_new, const void* q,
                                          int64_t q_token_stride, int64_t q_head_stride,
                                          float scale, int32_t window, void* y, float* lse,
                                          int32_t* dev_status, void* workspace, size_t ws_bytes,
                                          void* stream) {
  const ebd_status st = check_paged(cache);
  if (st != EBD_OK) return st;
  if (n_tokens < 0 || max_new < (n_tokens > 0) || n_q_heads < 1 ||
      n_q_heads % cache->n_kv_heads != 0)
    return EBD_ERR_INVALID;
  if (!(scale > 0.f) || !(scale < INFINITY) || window < 0) return EBD_ERR_INVALID;
  if (cache->head_dim != 64 && cache->head_dim != 128) return EBD_ERR_UNSUPPORTED;
  const int group = n_q_heads / cache->n_kv_heads;
  if (group > 128 || cache->batch > 65535 || cache->n_kv_heads > 65535) return EBD_ERR_UNSUPPORTED;
  if (n_tokens == 0) return EBD_OK;
  if (!cu_new || !q || !y || !dev_status) return EBD_ERR_INVALID;
  const int wide = cache->dtype == EBD_F32 ? 4 : 8;
  if (!paged_aligned16(cache) || !aligned16(q) || !aligned16(y) || q_token_stride % wide != 0 ||
      q_head_stride % wide != 0)
    return EBD_ERR_INVALID;
  if (q_token_stride < (n_tokens > 1) || q_head_stride < (n_q_heads > 1)) return EBD_ERR_INVALID;
  const size_t need = ebd_paged_attention_workspace_bytes(cache, n_q_heads, max_new);
  if (ws_bytes < need) return EBD_ERR_CAPACITY;
  if (need > 0 && (!workspace || !aligned16(workspace))) return EBD_ERR_INVALID;
  PagedAttnArgs a = {};
  a.q = q;
  a.K_pages = cache->K_pages;
  a.V_pages = cache->V_pages;
  a.pv = paged_view(*cache);
  a.cu = cu_new;
  a.q_ts = q_token_stride;
  a.q_hs = q_head_stride;
  a.y = y;
  a.lse = lse;
  a.n_tokens = n_tokens;
  a.max_new = max_new;
  a.group = group;
  a.window = window;
  a.scale2 = scale * kLog2e;
  a.dev_status = dev_status;
  cudaStream_t s = (cudaStream_t)stream;
  const int n_cta = attention_ctas(*cache);
  a.slot_rows = attention_slot_rows(*cache, group, max_new);
  paged_split_layout(a, workspace, n_cta);
  if (cache->dtype == EBD_F32)
    return cache->head_dim == 128 ? launch_paged_f32<128>(a, n_cta, s)
                                  : launch_paged_f32<64>(a, n_cta, s);
  return launch_paged_tc(a, *cache, n_cta, s);
}
