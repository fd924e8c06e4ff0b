// Attention of each sequence's new tokens over its paged cache,
//   y_i = sum_j softmax_j(scale q_i . k_j) v_j,  max(0, p_i - window + 1) <= j <= p_i,
// and its log-sum-exp, with an online softmax: running maximum m, sum l and
// output o in float32, rescaled by e^(m - m') when a tile raises the maximum.
//
// A CTA takes 32 rows of one (sequence, KV head): the G query heads of the
// group times the new tokens, token-major, so that all heads of the group read
// each key and value once.  Keys come in tiles of 64, converted to float32 in
// shared memory.  128 threads as 8 x 16: thread (ty, tx) owns rows 4 ty .. + 3,
// keys tx + 16 j of a tile's logits and channels 4 tx + 64 j of the output.
#include <cuda_runtime.h>
#include <math.h>

#include "common.cuh"
#include "internal.h"
#include "paged_attn.cuh"

namespace ebd {

constexpr int kAttnRows = 32;
constexpr int kAttnKeys = 64;
constexpr int kAttnThreads = 128;

template <int D>
struct SimtLayout {
  static constexpr int kQ = 0;  // [rows][D + 4]
  static constexpr int kK = kQ + kAttnRows * (D + 4);
  static constexpr int kV = kK + kAttnKeys * (D + 4);
  static constexpr int kP = kV + kAttnKeys * D;  // [rows][keys + 4]
  static constexpr int kFloats = kP + kAttnRows * (kAttnKeys + 4);
};

__device__ __forceinline__ void load4(const float* p, float (&x)[4]) {
  const float4 v = *reinterpret_cast<const float4*>(p);
  x[0] = v.x; x[1] = v.y; x[2] = v.z; x[3] = v.w;
}
__device__ __forceinline__ void store4(float* p, const float (&x)[4]) {
  *reinterpret_cast<float4*>(p) = make_float4(x[0], x[1], x[2], x[3]);
}
template <typename T, int D>
__global__ void __launch_bounds__(kAttnThreads) paged_attn_simt_kernel(const PagedAttnArgs a) {
  using L = SimtLayout<D>;
  extern __shared__ float4 smem4[];
  float* sm = reinterpret_cast<float*>(smem4);
  float *Qs = sm + L::kQ, *Ks = sm + L::kK, *Vs = sm + L::kV, *Ps = sm + L::kP;
  const int tx = threadIdx.x & 15, ty = threadIdx.x >> 4;
  const int b = blockIdx.z, h = blockIdx.y, row0 = blockIdx.x * kAttnRows;
  const SeqSpan sp = seq_span(a.pv, a.cu, b, a.n_tokens, a.max_new);
  if (sp.bad && threadIdx.x == 0 && h == 0 && row0 == 0) raise_status(a.dev_status, EBD_DEV_RANGE);
  const int rows = min(sp.n * a.group - row0, kAttnRows);
  if (rows <= 0) return;
  const int hq = a.pv.n_kv_heads * a.group;
  const int p0 = sp.len - sp.n;  // position of the first new token

  for (int i = threadIdx.x; i < kAttnRows * (D / 4); i += kAttnThreads) {
    const int r = i / (D / 4), c = i % (D / 4) * 4;
    float x[4] = {0.f, 0.f, 0.f, 0.f};
    if (r < rows) {
      const int t = (row0 + r) / a.group, g = (row0 + r) - t * a.group;
      load4((const T*)a.q + (sp.t0 + t) * a.q_ts + (h * a.group + g) * a.q_hs + c, x);
    }
    store4(Qs + r * (D + 4) + c, x);
  }
  int hi[4], lo[4];  // keys that this thread's rows see
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int r = ty * 4 + i, p = p0 + (row0 + min(r, rows - 1)) / a.group;
    hi[i] = min(p + 1, sp.len);
    lo[i] = a.window > 0 ? max(0, p - a.window + 1) : 0;
  }
  const int p_first = p0 + row0 / a.group, p_last = p0 + (row0 + rows - 1) / a.group;
  const int k_end = min(p_last + 1, sp.len);
  const int k_begin = (a.window > 0 ? max(0, p_first - a.window + 1) : 0) / kAttnKeys * kAttnKeys;

  float m[4], l[4], o[4][D / 16];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    m[i] = -INFINITY;
    l[i] = 0.f;
#pragma unroll
    for (int c = 0; c < D / 16; ++c) o[i][c] = 0.f;
  }
  for (int k0 = k_begin; k0 < k_end; k0 += kAttnKeys) {
    __syncthreads();
    for (int i = threadIdx.x; i < kAttnKeys * (D / 4); i += kAttnThreads) {
      const int r = i / (D / 4), c = i % (D / 4) * 4, pos = k0 + r;
      float kx[4] = {0.f, 0.f, 0.f, 0.f}, vx[4] = {0.f, 0.f, 0.f, 0.f};
      if (pos < k_end) {  // what lies past the last key seen is never read
        const int page = page_of(a.pv, b, pos);
        if (page >= 0) {
          const long long off = slot_offset(a.pv, page, h, pos) + c;
          load4((const T*)a.K_pages + off, kx);
          load4((const T*)a.V_pages + off, vx);
        } else {
          raise_status(a.dev_status, EBD_DEV_RANGE);
        }
      }
      store4(Ks + r * (D + 4) + c, kx);
      store4(Vs + r * D + c, vx);
    }
    __syncthreads();
    float s[4][4] = {};
#pragma unroll 4
    for (int c = 0; c < D; c += 4) {
      float q[4][4], k[4][4];
#pragma unroll
      for (int i = 0; i < 4; ++i) load4(Qs + (ty * 4 + i) * (D + 4) + c, q[i]);
#pragma unroll
      for (int j = 0; j < 4; ++j) load4(Ks + (tx + 16 * j) * (D + 4) + c, k[j]);
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j)
#pragma unroll
          for (int e = 0; e < 4; ++e) s[i][j] = fmaf(q[i][e], k[j][e], s[i][j]);
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      float top = m[i];
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const int pos = k0 + tx + 16 * j;
        s[i][j] = pos >= lo[i] && pos < hi[i] ? s[i][j] * a.scale2 : -INFINITY;
        top = fmaxf(top, s[i][j]);
      }
#pragma unroll
      for (int x = 8; x > 0; x >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, x));
      const float base = top == -INFINITY ? 0.f : top;  // nothing seen yet: every weight is 0
      const float f = exp2f(m[i] - base);
      m[i] = top;
      float sum = 0.f;
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const float p = exp2f(s[i][j] - base);
        sum += p;
        Ps[(ty * 4 + i) * (kAttnKeys + 4) + tx + 16 * j] = p;
      }
#pragma unroll
      for (int x = 8; x > 0; x >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, x);
      l[i] = l[i] * f + sum;
#pragma unroll
      for (int c = 0; c < D / 16; ++c) o[i][c] *= f;
    }
    __syncwarp();
    const int nk = min(kAttnKeys, k_end - k0);
    for (int k = 0; k < nk; ++k) {
      float p[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) p[i] = Ps[(ty * 4 + i) * (kAttnKeys + 4) + k];
#pragma unroll
      for (int c = 0; c < D / 64; ++c) {
        float v[4];
        load4(Vs + k * D + c * 64 + tx * 4, v);
#pragma unroll
        for (int i = 0; i < 4; ++i)
          // a key that the row does not see adds nothing, whatever its value holds
          if (k0 + k >= lo[i] && k0 + k < hi[i]) {
#pragma unroll
            for (int e = 0; e < 4; ++e) o[i][c * 4 + e] = fmaf(p[i], v[e], o[i][c * 4 + e]);
          }
      }
    }
  }
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int r = ty * 4 + i;
    if (r >= rows) continue;
    const int t = (row0 + r) / a.group, g = (row0 + r) - t * a.group;
    const long long out = (long long)(sp.t0 + t) * hq + h * a.group + g;
    const float inv = l[i] > 0.f ? 1.f / l[i] : (l[i] == 0.f ? 0.f : l[i]);  // NaN stays
#pragma unroll
    for (int c = 0; c < D / 64; ++c) {
      float x[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) x[e] = o[i][c * 4 + e] * inv;
      store4((T*)a.y + out * D + c * 64 + tx * 4, x);
    }
    if (a.lse && tx == 0) a.lse[out] = l[i] == 0.f ? -INFINITY : (m[i] + log2f(l[i])) * kLn2;
  }
}

template <typename T, int D>
static ebd_status launch_paged_simt(const PagedAttnArgs& a, cudaStream_t s) {
  const int smem = SimtLayout<D>::kFloats * 4;
  auto kern = paged_attn_simt_kernel<T, D>;
  if (cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, smem) !=
      cudaSuccess)
    return EBD_ERR_CUDA;
  const long long mt = ((long long)a.max_new * a.group + kAttnRows - 1) / kAttnRows;
  if (mt > 0x7fffffffLL) return EBD_ERR_UNSUPPORTED;
  kern<<<dim3((unsigned)mt, a.pv.n_kv_heads, a.pv.batch), kAttnThreads, smem, s>>>(a);
  return launch_status();
}

}  // namespace ebd

using namespace ebd;

extern "C" size_t ebd_paged_attention_workspace_bytes(const ebd_paged_cache* cache,
                                                      int32_t n_q_heads, int32_t max_new) {
  if (check_paged(cache) != EBD_OK || n_q_heads < 1 || max_new < 1) return 0;
  if (cache->dtype != EBD_BF16) return 0;
  return paged_split_bytes(sm_count(), kTcSlotRows, cache->head_dim);
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
  if (n_tokens < 0 || max_new < 0 || n_q_heads < 1 || n_q_heads % cache->n_kv_heads != 0)
    return EBD_ERR_INVALID;
  if (!(scale > 0.f) || !(scale < INFINITY) || window < 0) return EBD_ERR_INVALID;
  if (cache->head_dim != 64 && cache->head_dim != 128) return EBD_ERR_UNSUPPORTED;
  const int group = n_q_heads / cache->n_kv_heads;
  if (group > 128 || cache->batch > 65535 || cache->n_kv_heads > 65535) return EBD_ERR_UNSUPPORTED;
  if (n_tokens == 0 || max_new == 0) return EBD_OK;
  if (!cu_new || !q || !y || !dev_status) return EBD_ERR_INVALID;
  const int wide = cache->dtype == EBD_F32 ? 4 : 8;
  if (!paged_aligned16(cache) || !aligned16(q) || !aligned16(y) || q_token_stride < 0 ||
      q_head_stride < 0 || q_token_stride % wide != 0 || q_head_stride % wide != 0)
    return EBD_ERR_INVALID;
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
  if (cache->dtype == EBD_F32)
    return cache->head_dim == 128 ? launch_paged_simt<float, 128>(a, s)
                                  : launch_paged_simt<float, 64>(a, s);
  const int n_cta = sm_count();
  paged_split_layout(a, workspace, n_cta, kTcSlotRows);
  a.min_share = 4;
  return launch_paged_tc(a, *cache, n_cta, s);
}
