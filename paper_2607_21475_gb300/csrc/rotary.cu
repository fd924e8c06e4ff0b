// Rotary positions: the (cos, sin) table, the rotation of queries or keys, and
// the append of new keys and values to a paged cache with the rotation on the
// way.
//
// Pair i of a head (channels (i, i + R/2) in the half layout, (2i, 2i + 1) in
// the pairs layout, R = rotary_dim) at position p turns by p * f_i:
//   a' = a cos - b sin,  b' = b cos + a sin,
// in float32, rounded once to the tensor's type.  The inverse (sin -> -sin) is
// also the gradient, the rotation being orthogonal.  Channels from R on are
// copied.
//
// Both kernels only move data (3 FMAs per element moved), so what bounds them
// is HBM at large sizes and the launch's load chain at small ones.  A warp
// takes one token (append: its sequence, position and page are then found once
// per warp, the sequence by a ballot over 32 offsets at a time) and its lanes
// take (head, pair of 16-byte chunks): neighbouring lanes read neighbouring chunks
// of a head's row, and a lane keeps one unit's cosines and sines in registers
// for all heads it walks, two rows in flight.  Small calls give every lane one
// unit (a token then spans several warps), so that a decode step costs one pass of
// the load chain.
// Measured: rotation of 16384 tokens x 28 heads x 128, bf16: 38.4 us, 6.3 TB/s
// (94% of the measured copy peak); append of 8 ragged chunks (28/4 heads, 10.7k
// tokens) 33.6 us, 5.9 TB/s; append step of 32 sequences (32/8 heads) 3.2 us.
#include <cuda_runtime.h>

#include "common.cuh"
#include "internal.h"
#include "paged.cuh"

namespace ebd {

constexpr int kRotWarps = 8;
// resident blocks of 256 threads: 64 registers per thread, 80 for the append (whose
// rows wait longer; 4 blocks with spills: 53 us against 42 us on ragged prompt chunks)
constexpr int kRotBlocks = 4, kAppendBlocks = 3;

__global__ void rotary_table_kernel(const double* __restrict__ inv_freq, int n_freq,
                                    long long total, double mscale, float2* __restrict__ table) {
  for (long long i = (long long)blockIdx.x * blockDim.x + threadIdx.x; i < total;
       i += (long long)gridDim.x * blockDim.x) {
    const long long pos = i / n_freq;
    double s, c;
    // double: a float32 angle of a position near 10^5 is off by 4e-3 radians
    sincos((double)pos * inv_freq[i - pos * n_freq], &s, &c);
    table[i] = make_float2((float)(c * mscale), (float)(s * mscale));
  }
}

// VEC elements of T as one access.
template <typename T, int VEC>
struct alignas(VEC * sizeof(T)) Chunk {
  T e[VEC];
};

// A chunk's load and store, marked for early eviction from L2 where it is 16 bytes:
// each is used once here, and a long prompt's otherwise push each other's
// unwritten lines out in the middle of the stream (16k-token prompt 47.7 us with
// plain accesses, 38.9 us with the stores marked, 38.1 us with both).
template <typename T, int VEC>
__device__ __forceinline__ void load_chunk(const T* p, Chunk<T, VEC>& c) {
  if constexpr (VEC * sizeof(T) == 16)
    *reinterpret_cast<uint4*>(&c) = __ldcs(reinterpret_cast<const uint4*>(p));
  else
    c = *reinterpret_cast<const Chunk<T, VEC>*>(p);
}
template <typename T, int VEC>
__device__ __forceinline__ void store_chunk(T* p, const Chunk<T, VEC>& c) {
  if constexpr (VEC * sizeof(T) == 16)
    __stcs(reinterpret_cast<uint4*>(p), *reinterpret_cast<const uint4*>(&c));
  else
    *reinterpret_cast<Chunk<T, VEC>*>(p) = c;
}

__device__ __forceinline__ void from_f32(float x, float& y) { y = x; }
__device__ __forceinline__ void from_f32(float x, __nv_bfloat16& y) { y = __float2bfloat16_rn(x); }

// One set of rows: element (token t, head h, channel c) at p[t * ts + h * hs + c].
struct Rows {
  const void* p;
  long long ts, hs;
};

struct RotaryArgs {
  Rows x;                // q (append) or x (rotary)
  Rows y;                // its destination
  Rows k, v;             // append only
  void *K_pages, *V_pages;
  PagedView pv;
  const int32_t* cu;         // append: [batch + 1]
  const int32_t* positions;  // rotary: [n_tokens]
  const float2* table;       // [n_pos, rot / 2]; null: no rotation
  int n_pos;
  int n_tokens, n_x, n_kv;   // heads of x; kv heads (0: rotary)
  int head_dim;
  int units;                 // pairs of chunks of a row
  int rot_units;             // how many of them are rotated (pairs: in part or whole)
  int half_off;              // half layout: rot / 2
  int rot;
  int parts;                 // warps per token
  float sin_sign;            // -1: inverse
  bool wide_table;           // two pairs of the table per 16-byte access
  int32_t* dev_status;
};

// A lane's share of one row: two chunks.
template <typename T, int VEC>
struct Piece {
  Chunk<T, VEC> a, b;
};

// Channels of unit u's chunks (c2 < 0: the row has no second one).  Half layout:
// units below rot_units are the chunk pairs (u VEC, rot / 2 + u VEC) that turn
// together, later ones neighbouring chunks of the copied channels.  Pairs layout:
// neighbouring chunks, turned where they lie below rot.
template <int VEC, bool PAIRS>
__device__ __forceinline__ void unit_channels(const RotaryArgs& a, int u, int& c1, int& c2) {
  if (!PAIRS && u < a.rot_units) {
    c1 = u * VEC;
    c2 = a.half_off + c1;
  } else {
    c1 = PAIRS ? 2 * u * VEC : a.rot + 2 * (u - a.rot_units) * VEC;
    c2 = c1 + VEC < a.head_dim ? c1 + VEC : -1;
  }
}

// STEADY: 32 * parts is a multiple of the units, so that a lane keeps its unit
// (and its angles) from head to head.  Rows are loaded one step ahead: the first
// ones before the token's place is known, the next ones before these are stored.
template <typename T, int VEC, bool PAIRS, bool APPEND, bool STEADY>
__global__ void __launch_bounds__(kRotWarps * 32, APPEND ? kAppendBlocks : kRotBlocks)
    rotary_kernel(const RotaryArgs a) {
  const int lane = threadIdx.x & 31;
  const long long w = (long long)blockIdx.x * kRotWarps + (threadIdx.x >> 5);
  const int t = a.parts == 1 ? (int)w : (int)(w / a.parts), part = (int)(w - (long long)t * a.parts);
  if (t >= a.n_tokens) return;

  const int heads = a.n_x + (APPEND ? 2 * a.n_kv : 0);
  const int stride = 32 * a.parts, step = stride / a.units, rest = stride - step * a.units;
  int h = (part * 32 + lane) / a.units, u = part * 32 + lane - h * a.units;
  const T* xp = (const T*)a.x.p + t * a.x.ts;
  const T* kp = (const T*)a.k.p + t * a.k.ts;
  const T* vp = (const T*)a.v.p + t * a.v.ts;
  auto load = [&](int h, int u, Piece<T, VEC>& r) {
    if (h >= heads) return;
    int c1, c2;
    unit_channels<VEC, PAIRS>(a, u, c1, c2);
    const T* src = !APPEND || h < a.n_x  ? xp + h * a.x.hs
                   : h < a.n_x + a.n_kv ? kp + (h - a.n_x) * a.k.hs
                                        : vp + (h - a.n_x - a.n_kv) * a.v.hs;
    load_chunk<T, VEC>(src + c1, r.a);
    if (c2 >= 0) load_chunk<T, VEC>(src + c2, r.b);
  };
  auto next = [&](int& h, int& u) {
    h += step;
    if (!STEADY) {
      u += rest;
      if (u >= a.units) {
        u -= a.units;
        ++h;
      }
    }
  };
  Piece<T, VEC> r0, r1;
  int h1 = h, u1 = u;
  next(h1, u1);
  load(h, u, r0);
  load(h1, u1, r1);

  int pos, b = 0, page = -1;
  if (APPEND) {
    // the offsets run from 0 to n_tokens; the first token's warp looks at both ends
    const int c_first = t == 0 ? a.cu[0] : 0, c_last = t == 0 ? a.cu[a.pv.batch] : a.n_tokens;
    bool odd;
    b = sequence_of(a.cu, a.pv.batch, t, lane, odd);
    bool none = b >= a.pv.batch;  // no sequence's token: no place for it
    int c0 = 0, c1 = 0, len = 0;
    if (!none) c0 = a.cu[b], c1 = a.cu[b + 1], len = a.pv.seq_len[b];
    none |= t < c0;
    odd |= none | (c_first != 0) | (c_last != a.n_tokens);
    if (lane == 0 && odd) raise_status(a.dev_status, EBD_DEV_RANGE);
    if (none) return;
    pos = len - (min(c1, a.n_tokens) - t);
    page = page_of(a.pv, b, pos);
  } else {
    pos = a.positions[t];
  }
  const int tpos = min(max(pos, 0), a.n_pos - 1);

  float cs[VEC], sn[VEC];  // the pairs of a unit
  auto load_angles = [&](int u) {
    if (u >= a.rot_units) return;
    const float2* row = a.table + (size_t)tpos * (a.rot / 2) + u * VEC;
    const int n = PAIRS ? min(VEC, a.rot / 2 - u * VEC) : VEC;
    if (VEC % 2 == 0 && a.wide_table) {
#pragma unroll
      for (int i = 0; i + 1 < VEC; i += 2) {
        if (PAIRS && i >= n) break;
        const float4 f = __ldg(reinterpret_cast<const float4*>(row + i));
        cs[i] = f.x;
        sn[i] = f.y * a.sin_sign;
        cs[i + 1] = f.z;
        sn[i + 1] = f.w * a.sin_sign;
      }
    } else {
#pragma unroll
      for (int i = 0; i < VEC; ++i) {
        if (PAIRS && i >= n) break;
        const float2 f = __ldg(row + i);
        cs[i] = f.x;
        sn[i] = f.y * a.sin_sign;
      }
    }
  };
  if (STEADY) load_angles(u);
  if (lane == 0 && ((APPEND && page < 0) || (a.table && tpos != pos)))
    raise_status(a.dev_status, EBD_DEV_RANGE);
  T* yp = (T*)a.y.p + t * a.y.ts;
  const long long slot = page >= 0 ? slot_offset(a.pv, page, 0, pos) : -1;
  // turns and stores one row's piece
  auto store = [&](int h, int u, Piece<T, VEC>& r) {
    if (h >= heads) return;
    int c1, c2;
    unit_channels<VEC, PAIRS>(a, u, c1, c2);
    const bool is_v = APPEND && h >= a.n_x + a.n_kv;
    if (u < a.rot_units && !is_v) {
      if (!STEADY) load_angles(u);
      auto turn = [&](T& e0, T& e1, int i) {
        const float p = to_f32(e0), q = to_f32(e1);
        from_f32(p * cs[i] - q * sn[i], e0);
        from_f32(q * cs[i] + p * sn[i], e1);
      };
      if (PAIRS) {
#pragma unroll
        for (int i = 0; i < VEC / 2; ++i) turn(r.a.e[2 * i], r.a.e[2 * i + 1], i);
        if (c2 >= 0 && c2 < a.rot) {
#pragma unroll
          for (int i = 0; i < VEC / 2; ++i)
            turn(r.b.e[2 * i], r.b.e[2 * i + 1], VEC / 2 + i);
        }
      } else {
#pragma unroll
        for (int i = 0; i < VEC; ++i) turn(r.a.e[i], r.b.e[i], i);
      }
    }
    T* dst;
    if (!APPEND || h < a.n_x) {
      dst = yp + h * a.y.hs;
    } else {
      if (slot < 0) return;
      const int kh = h - a.n_x - (is_v ? a.n_kv : 0);
      dst = (T*)(is_v ? a.V_pages : a.K_pages) + slot + kh * a.pv.head_stride;
    }
    store_chunk<T, VEC>(dst + c1, r.a);
    if (c2 >= 0) store_chunk<T, VEC>(dst + c2, r.b);
  };
  while (h < heads) {
    store(h, u, r0);
    h = h1;
    u = u1;
    next(h, u);
    load(h, u, r0);
    if (h1 >= heads) break;
    store(h1, u1, r1);
    h1 = h;
    u1 = u;
    next(h1, u1);
    load(h1, u1, r1);
  }
}

// A row access of `vec` elements is aligned at every (token, head).
static bool rows_aligned(const Rows& r, int vec, int elem) {
  return ((uintptr_t)r.p % (vec * elem)) == 0 && r.ts % vec == 0 && r.hs % vec == 0;
}

template <typename T, int VEC, bool PAIRS, bool APPEND>
static ebd_status launch_rotary_v(RotaryArgs a, int head_dim, cudaStream_t s) {
  const int rot = a.table ? a.rot : 0;
  a.rot = rot;
  a.half_off = rot / 2;
  a.head_dim = head_dim;
  const int chunks_of_rot = rot / VEC, chunks_of_row = head_dim / VEC;
  a.rot_units = PAIRS ? (chunks_of_rot + 1) / 2 : chunks_of_rot / 2;
  a.units = PAIRS ? (chunks_of_row + 1) / 2
                  : a.rot_units + (chunks_of_row - chunks_of_rot + 1) / 2;
  a.wide_table = rot % 4 == 0 && (uintptr_t)a.table % 16 == 0;
  const int chunks = (a.n_x + (APPEND ? 2 * a.n_kv : 0)) * a.units;
  // one chunk pair per lane while the call has fewer warps than the GPU holds
  // (latency), up to sixteen rows per lane beyond that
  const int few = (chunks + 511) / 512, many = (chunks + 31) / 32;
  a.parts = (long long)a.n_tokens * many <= (long long)sm_count() * 32 ? many : few;
  // a few warps more per token, where that lets every lane keep its unit
  for (int p = a.parts; p < a.parts + 4; ++p)
    if (32 * p % a.units == 0) {
      a.parts = p;
      break;
    }
  const long long blocks = ((long long)a.n_tokens * a.parts + kRotWarps - 1) / kRotWarps;
  if (blocks > 0x7fffffffLL) return EBD_ERR_UNSUPPORTED;
  if (32 * a.parts % a.units == 0)
    rotary_kernel<T, VEC, PAIRS, APPEND, true>
        <<<(unsigned)blocks, kRotWarps * 32, 0, s>>>(a);
  else
    rotary_kernel<T, VEC, PAIRS, APPEND, false>
        <<<(unsigned)blocks, kRotWarps * 32, 0, s>>>(a);
  return launch_status();
}

// 16-byte accesses where every row and the rotated part allow them; otherwise
// single elements (half) or single pairs (pairs).  16384 tokens x 28 heads x 80 channels in
// bf16, half layout: 32 rotated 27 us (5.4 TB/s), 20 rotated, by elements, 46 us (3.2 TB/s).
template <typename T, bool APPEND>
static ebd_status launch_rotary_t(const RotaryArgs& a, int head_dim, bool pairs, bool cache_ok,
                                  cudaStream_t s) {
  constexpr int kWide = 16 / (int)sizeof(T);
  const int rot = a.table ? a.rot : 0;
  const bool wide = (pairs ? rot : rot / 2) % kWide == 0 && head_dim % kWide == 0 && cache_ok &&
                    (a.n_x == 0 || (rows_aligned(a.x, kWide, sizeof(T)) &&
                                    rows_aligned(a.y, kWide, sizeof(T)))) &&
                    (!APPEND || (rows_aligned(a.k, kWide, sizeof(T)) &&
                                 rows_aligned(a.v, kWide, sizeof(T))));
  if (pairs) {
    // an odd head_dim or stride would split a pair's 2-element access
    const bool two = head_dim % 2 == 0 &&
                     (a.n_x == 0 || (rows_aligned(a.x, 2, sizeof(T)) &&
                                     rows_aligned(a.y, 2, sizeof(T)))) &&
                     (!APPEND || (rows_aligned(a.k, 2, sizeof(T)) &&
                                  rows_aligned(a.v, 2, sizeof(T)) &&
                                  a.pv.page_stride % 2 == 0 && a.pv.head_stride % 2 == 0 &&
                                  a.pv.row_stride % 2 == 0 &&
                                  (uintptr_t)a.K_pages % (2 * sizeof(T)) == 0 &&
                                  (uintptr_t)a.V_pages % (2 * sizeof(T)) == 0));
    if (wide) return launch_rotary_v<T, kWide, true, APPEND>(a, head_dim, s);
    if (two) return launch_rotary_v<T, 2, true, APPEND>(a, head_dim, s);
    return EBD_ERR_UNSUPPORTED;
  }
  if (wide) return launch_rotary_v<T, kWide, false, APPEND>(a, head_dim, s);
  return launch_rotary_v<T, 1, false, APPEND>(a, head_dim, s);
}

}  // namespace ebd

using namespace ebd;

extern "C" ebd_status ebd_rotary_table(const double* inv_freq, int32_t n_freq, int32_t n_pos,
                                       double mscale, float* table, void* stream) {
  if (!inv_freq || !table || n_freq < 1 || n_pos < 1) return EBD_ERR_INVALID;
  if ((uintptr_t)table % 8 != 0) return EBD_ERR_INVALID;
  const long long total = (long long)n_freq * n_pos;
  long long blocks = (total + 255) / 256;
  if (blocks > (long long)sm_count() * 16) blocks = (long long)sm_count() * 16;
  rotary_table_kernel<<<(unsigned)blocks, 256, 0, (cudaStream_t)stream>>>(
      inv_freq, n_freq, total, mscale, (float2*)table);
  return launch_status();
}

extern "C" ebd_status ebd_rotary(ebd_dtype dtype, int32_t n_tokens, int32_t n_heads,
                                 int32_t head_dim, int32_t rotary_dim, ebd_rotary_layout layout,
                                 int32_t inverse, const void* x, int64_t x_token_stride,
                                 int64_t x_head_stride, const int32_t* positions,
                                 const float* table, int32_t n_pos, void* y,
                                 int64_t y_token_stride, int64_t y_head_stride,
                                 int32_t* dev_status, void* stream) {
  if (dtype != EBD_F32 && dtype != EBD_BF16) return EBD_ERR_INVALID;
  if (layout != EBD_ROTARY_HALF && layout != EBD_ROTARY_PAIRS) return EBD_ERR_INVALID;
  if (n_tokens < 0 || n_heads < 1 || head_dim < 1 || n_pos < 1) return EBD_ERR_INVALID;
  if (rotary_dim < 2 || rotary_dim > head_dim || rotary_dim % 2 != 0) return EBD_ERR_INVALID;
  if (n_tokens == 0) return EBD_OK;
  if (!x || !y || !positions || !table || (uintptr_t)table % 8 != 0) return EBD_ERR_INVALID;
  RotaryArgs a = {};
  a.x = Rows{x, x_token_stride, x_head_stride};
  a.y = Rows{y, y_token_stride, y_head_stride};
  a.positions = positions;
  a.table = (const float2*)table;
  a.n_pos = n_pos;
  a.n_tokens = n_tokens;
  a.n_x = n_heads;
  a.rot = rotary_dim;
  a.sin_sign = inverse ? -1.f : 1.f;
  a.dev_status = dev_status;
  const bool pairs = layout == EBD_ROTARY_PAIRS;
  cudaStream_t s = (cudaStream_t)stream;
  return dtype == EBD_F32 ? launch_rotary_t<float, false>(a, head_dim, pairs, true, s)
                          : launch_rotary_t<__nv_bfloat16, false>(a, head_dim, pairs, true, s);
}

extern "C" ebd_status ebd_paged_append(
    const ebd_paged_cache* cache, int32_t n_tokens, const int32_t* cu_new, const void* k_new,
    int64_t k_token_stride, int64_t k_head_stride, const void* v_new, int64_t v_token_stride,
    int64_t v_head_stride, const float* table, int32_t n_pos, int32_t rotary_dim,
    ebd_rotary_layout layout, int32_t n_q_heads, const void* q, int64_t q_token_stride,
    int64_t q_head_stride, void* q_out, int64_t q_out_token_stride, int64_t q_out_head_stride,
    int32_t* dev_status, void* stream) {
  const ebd_status st = check_paged(cache);
  if (st != EBD_OK) return st;
  if (layout != EBD_ROTARY_HALF && layout != EBD_ROTARY_PAIRS) return EBD_ERR_INVALID;
  if (n_tokens < 0 || n_q_heads < 0) return EBD_ERR_INVALID;
  if (table && (n_pos < 1 || rotary_dim < 2 || rotary_dim > cache->head_dim ||
                rotary_dim % 2 != 0 || (uintptr_t)table % 8 != 0))
    return EBD_ERR_INVALID;
  if (n_q_heads > 0 && !table) return EBD_ERR_INVALID;  // nothing to do to q
  if (n_tokens == 0) return EBD_OK;
  if (!cu_new || !k_new || !v_new || !dev_status || (n_q_heads > 0 && (!q || !q_out)))
    return EBD_ERR_INVALID;
  RotaryArgs a = {};
  a.x = Rows{q, q_token_stride, q_head_stride};
  a.y = Rows{q_out, q_out_token_stride, q_out_head_stride};
  a.k = Rows{k_new, k_token_stride, k_head_stride};
  a.v = Rows{v_new, v_token_stride, v_head_stride};
  a.K_pages = cache->K_pages;
  a.V_pages = cache->V_pages;
  a.pv = paged_view(*cache);
  a.cu = cu_new;
  a.table = (const float2*)table;
  a.n_pos = table ? n_pos : 0x7fffffff;
  a.n_tokens = n_tokens;
  a.n_x = n_q_heads;
  a.n_kv = cache->n_kv_heads;
  a.rot = rotary_dim;
  a.sin_sign = 1.f;
  a.dev_status = dev_status;
  const int eb = cache->dtype == EBD_F32 ? 4 : 2;
  const int wide = 16 / eb;
  const bool cache_ok = aligned16(cache->K_pages) && aligned16(cache->V_pages) &&
                        cache->page_stride % wide == 0 && cache->head_stride % wide == 0 &&
                        cache->row_stride % wide == 0;
  const bool pairs = layout == EBD_ROTARY_PAIRS && table;
  cudaStream_t s = (cudaStream_t)stream;
  return cache->dtype == EBD_F32
             ? launch_rotary_t<float, true>(a, cache->head_dim, pairs, cache_ok, s)
             : launch_rotary_t<__nv_bfloat16, true>(a, cache->head_dim, pairs, cache_ok, s);
}
