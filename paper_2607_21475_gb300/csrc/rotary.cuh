// Row accesses shared by the rotation and the norms: chunks of a row, a lane's pair
// of them, strided sets of rows.
#pragma once

#include <cuda_runtime.h>
#include <stdint.h>

#include "common.cuh"

namespace ebd {

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

// A lane's share of one row: two chunks.
template <typename T, int VEC>
struct Piece {
  Chunk<T, VEC> a, b;
};

// Channels of unit u's chunks (c2 < 0: the row has no second one).  Half layout:
// units below rot_units are the chunk pairs (u VEC, rot / 2 + u VEC) that turn
// together, later ones neighbouring chunks of the copied channels.  Pairs layout:
// neighbouring chunks, turned where they lie below rot.
template <int VEC, bool PAIRS, typename Args>
__device__ __forceinline__ void unit_channels(const Args& a, int u, int& c1, int& c2) {
  if (!PAIRS && u < a.rot_units) {
    c1 = u * VEC;
    c2 = a.half_off + c1;
  } else {
    c1 = PAIRS ? 2 * u * VEC : a.rot + 2 * (u - a.rot_units) * VEC;
    c2 = c1 + VEC < a.head_dim ? c1 + VEC : -1;
  }
}

// A row access of `vec` elements is aligned at every (token, head).
inline bool rows_aligned(const Rows& r, int vec, int elem) {
  return ((uintptr_t)r.p % (vec * elem)) == 0 && r.ts % vec == 0 && r.hs % vec == 0;
}

}  // namespace ebd
