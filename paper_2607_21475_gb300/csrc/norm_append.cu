// Append of new keys and values to a paged cache with their norms and the rotation on the way:
// the entry point (kernel: norm_forward.cuh, mathematics and figures: norm.cuh).
#include "norm_forward.cuh"

using namespace ebd;

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
  if (n_q_heads + 2ll * cache->n_kv_heads > kNormMaxHeads) return EBD_ERR_UNSUPPORTED;
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
  return cache->dtype == EBD_F32 ? launch_norm_t<float, kNormAppend>(a, pairs, nullptr, s)
                                 : launch_norm_t<__nv_bfloat16, kNormAppend>(a, pairs, nullptr, s);
}
