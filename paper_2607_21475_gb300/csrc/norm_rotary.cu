// Norms of queries and keys per head with the rotation to their positions: the entry point
// (kernel: norm_forward.cuh, mathematics and figures: norm.cuh).
#include "norm_forward.cuh"

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
  if (n_heads > kNormMaxHeads) return EBD_ERR_UNSUPPORTED;
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
  return dtype == EBD_F32 ? launch_norm_t<float, kNormForward>(a, pairs, nullptr, s)
                          : launch_norm_t<__nv_bfloat16, kNormForward>(a, pairs, nullptr, s);
}
