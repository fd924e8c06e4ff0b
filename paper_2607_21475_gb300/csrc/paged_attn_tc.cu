// Paged attention on the 5th-generation tensor cores: bf16, head_dim 64 / 128.
//
// An item is two MMA tiles X = A, B of 128 rows, whole tokens with all heads of
// the group each; keys come in tiles of 64.  Per key tile and X:  S_X = Q_X K^T
// (both operands in shared memory), the softmax warps turn S_X into weights P_X,
// and O_X += P_X V with P_X read from tensor memory.  Tensor memory (512
// columns): O_A, O_B (128 columns each, D used) and two buffers of 64 columns of
// S_A and of S_B; P_X (bf16) overwrites the first 32 columns of its S_X buffer.
// With two buffers the product S of the next tile is ready when the softmax of
// this one ends.  128-key tiles fit only one buffer each, and that chain (S
// product, softmax, O product, S product) took 3490 cycles per 128 keys of two X
// against 2050 of MMA work; this form takes 1410 per 64 keys.  The price is the S
// product's rate: at N = 64 it reads Q again for half the keys, and shared memory
// holds it to 2/3 of the MMA rate (1280 cycles of MMA work per 64 keys).
//
// What bounds it: a chunk of 4096 tokens over 16k positions (28/4 heads, d = 128)
// runs at 1.71 PFLOP/s (493 us, 89% of the measured bf16 peak) at the full clock and
// at 1.55-1.6 (525-541 us) under the power cap of a long run; a decode batch of 32
// sequences streams its cache at 6.9-7.0 TB/s (at the copy peak); head_dim 64 and short
// windows are bound by the softmax warps (mixed batch with a window of 1024: 42 us,
// 1370 cycles per tile of two X, 1070 of one; decode of 32 x 16k at 64 channels: 209 us,
// 5.1 TB/s); one sequence of 6k tokens by latencies (12.7 us, of which about 8000 cycles
// pass before the first product).
//
// The softmax keeps one row per thread.  Its reference m moves only when a
// tile's maximum exceeds it by more than 2^8 (in the weight), so that O_X is
// rarely rescaled; the result is the same, sums and weights being relative to
// the same m.  Weights are rounded to bf16 for the second product (their sum is
// of the unrounded ones), which costs at most 2^-8 of the largest value, as
// the result's own rounding does.
//
// Roles: warps 0-3 / 4-7 softmax and epilogue of A / B, warps 8 / 9 issue the
// MMAs of A / B, warp 10 the TMA copies of K and V (one box per page and 64
// channels; pages past the sequence's end are read past the pool's end, and
// keys of pages outside the pool, which the softmax hides, before its beginning:
// both fill zeros), warp 11 walks the CTA's pieces, copies the query rows and clears
// the value rows of a tile past the sequence's end (weight 0 times whatever a
// page holds there must stay 0).
//
// Every wait is bounded (~2 s): a timeout raises EBD_DEV_TIMEOUT, the roles
// leave their loops, copies and MMAs in flight are waited for and the tensor
// memory is released.
#include <cuda.h>
#include <cudaTypedefs.h>
#include <cuda_runtime.h>
#include <math.h>

#include <mutex>

#include "decode_tile.cuh"
#include "paged_attn.cuh"
#include "ptx.cuh"
#include "tcgen05_attn.cuh"

namespace ebd {

constexpr int kTcBN = 64;
constexpr int kTcAttnThreads = 384;

template <int D>
struct PagedTcLayout {
  static constexpr int kHalves = D / 64;
  static constexpr int kQBox = 128 * 128;      // 128 rows x 64 bf16
  static constexpr int kQTile = kHalves * kQBox;
  static constexpr int kBox = kTcBN * 128;     // 64 rows x 64 bf16
  static constexpr int kTile = kHalves * kBox;
  static constexpr int kStages = D == 128 ? 5 : 8;  // of K, and of V
  static constexpr int kQ = 0;                 // two tiles
  static constexpr int kK = 2 * kQTile;
  static constexpr int kV = kK + kStages * kTile;
  static constexpr int kBar = kV + kStages * kTile;
  static constexpr int kBytes = kBar + 1024;
};

// One piece of the CTA's work, as the roles see it.
struct Piece {
  int cur, end;     // key tiles; equal: no piece, the work is done
  int b, h, len;    // sequence, KV head, keys in the cache
  int token;        // packed number of the first token
  int pos;          // its position
  int tokens;
  int slot;         // partial result, -1: the output itself
  int first;        // number of the first token among the sequence's new ones
  int absent;       // a key that it sees has no page; told with q_full, so that the softmax
                    // asks once a piece (once a tile: mixed batch 41.5 -> 42.9 us,
                    // 4096-token chunk 490 -> 503 us at the full clock)
};
constexpr int kPieceSlots = 4;
constexpr int kPieceReaders = 11;  // warps that read a piece
// Keys of a tile (bit i: key i) whose page is outside the pool, by the CTA's tile
// number.  A tile's entry is written before its K copy is announced and read before
// its P is, and tile t + stages is copied after S of t, which follows P of t - 2: more
// than stages + 2 entries are never in use.
constexpr int kAbsentSlots = 16;

struct TcBars {
  uint64_t q_full, q_empty;
  uint64_t s_full[2][2], p_full[2][2], o_full[2][2];  // [X][S buffer]
  uint64_t fixed, done[2];
  uint64_t k_full[8], k_empty[8], v_full[8], v_empty[8];
  uint64_t piece_full[kPieceSlots], piece_empty[kPieceSlots];
  uint64_t absent[kAbsentSlots];
  Piece piece[kPieceSlots];
  uint32_t tmem;
};
static_assert(sizeof(TcBars) <= 1024, "barriers");
static_assert(PagedTcLayout<64>::kStages + 2 <= kAbsentSlots &&
                  PagedTcLayout<128>::kStages + 2 <= kAbsentSlots,
              "absent keys");

// max(a, b, c) in one instruction.
__device__ __forceinline__ float max3(float a, float b, float c) {
  float r;
  asm("max.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
  return r;
}

// TREE: new tokens see each other by a mask.  A row's 64 bits for a tile that touches the
// tree are found while the tile's product runs, and select its logits; the other tiles take
// the same path as causal ones, and so does the time (one 6k-token sequence, 16 drafted
// tokens, 28/4 heads x 128: 15.2 us, 14.9 causal; trees of 40-64 tokens of 32 dialogues
// of 2k-32k, 32/8 x 128: 422 us at the full clock, 440-514 under the power cap, tensor pipe
// 75% active, its 256-row tiles 81% filled).
// PADDED: places past the last offset are empty, no mistake (a form of its own: asked at run
// time, the causal kernels took longer, a 4096-token chunk over 16k 493 -> 499 us).
template <int D, bool TREE, bool PADDED>
__global__ void __launch_bounds__(kTcAttnThreads, 1)
    paged_attn_tc_kernel(const __grid_constant__ CUtensorMap tmQ,
                         const __grid_constant__ CUtensorMap tmK,
                         const __grid_constant__ CUtensorMap tmV, const PagedAttnArgs a) {
  using L = PagedTcLayout<D>;
  constexpr int KS = L::kStages;
  extern __shared__ __align__(1024) unsigned char smem[];
  TcBars* bar = reinterpret_cast<TcBars*>(smem + L::kBar);

  const int warp = __shfl_sync(0xffffffffu, threadIdx.x >> 5, 0), lane = threadIdx.x & 31;
  const int cta = blockIdx.x;
  if (warp == 8) {
    tmem_alloc(&bar->tmem, 512);
    tmem_relinquish();
  } else if (warp == 9) {
    if (lane < kAbsentSlots) bar->absent[lane] = 0;
    if (lane == 0) {
      mbar_init(&bar->q_full, 2);
      mbar_init(&bar->q_empty, 2);
      for (int x = 0; x < 2; ++x) {
        mbar_init(&bar->done[x], 1);
        for (int b = 0; b < 2; ++b) {
          mbar_init(&bar->s_full[x][b], 1);
          mbar_init(&bar->p_full[x][b], 4);
          mbar_init(&bar->o_full[x][b], 1);
        }
      }
      mbar_init(&bar->fixed, 32);
      for (int i = 0; i < kPieceSlots; ++i) {
        mbar_init(&bar->piece_full[i], 1);
        mbar_init(&bar->piece_empty[i], kPieceReaders);
      }
      for (int s = 0; s < KS; ++s) {
        mbar_init(&bar->k_full[s], 1);
        mbar_init(&bar->k_empty[s], 2);
        mbar_init(&bar->v_full[s], 1);
        mbar_init(&bar->v_empty[s], 2);
      }
      fence_barrier_init();
    }
  }
  // the rows past an X's last query row (none where the group divides 128) are
  // never loaded: numbers, once
  const int used = a.half_tokens * a.group;
  for (int i = threadIdx.x; i < (128 - used) * 8 * 2 * L::kHalves; i += kTcAttnThreads) {
    const int box = i / ((128 - used) * 8), at = i - box * ((128 - used) * 8);
    *reinterpret_cast<uint4*>(smem + L::kQ + box * L::kQBox + used * 128 + at * 16) =
        make_uint4(0, 0, 0, 0);
  }
  fence_proxy_async_smem();
  grid_dependency_wait();  // nothing of the caller's was read or written so far
  WorkStart start = {};
  if (warp == 11) start = find_work<kTcBN, TREE, PADDED>(a, cta, gridDim.x, lane);
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = bar->tmem;
  bool ok = true;
  // The i-th piece; a reading warp takes it with read_piece and hands its place
  // back with drop_piece.
  auto read_piece = [&](uint32_t i, Piece& w) {
    if (!mbar_wait_warp(&bar->piece_full[i % kPieceSlots], (i / kPieceSlots) & 1))
      return ok = false;
    w = bar->piece[i % kPieceSlots];
    return w.cur < w.end;
  };
  auto drop_piece = [&](uint32_t i) {
    __syncwarp();
    if (lane == 0) mbar_arrive(&bar->piece_empty[i % kPieceSlots]);
  };
  Piece w;

  if (warp < 8) {
    // ---------------- softmax and epilogue: one row per thread
    const int x = warp >> 2, row = (warp & 3) * 32 + lane;
    const uint32_t lane_base = (uint32_t)((warp & 3) * 32) << 16;
    const uint32_t sS = tmem + 256 + x * 128 + lane_base;
    const uint32_t sO = tmem + x * 128 + lane_base;
    uint32_t it = 0;     // tiles of X so far: S buffer it & 1
    uint32_t tile0 = 0;  // tiles of the CTA before this piece
    bool nonfinite = false;  // an output of the thread's rows was NaN or infinite
    const int rt = row / a.group, g = row - rt * a.group;
    for (uint32_t i = 0; read_piece(i, w); tile0 += w.end - w.cur, drop_piece(i++)) {
      // the X's tokens [x0, x0 + tokens); rows past the last repeat its last token
      const int x0 = x * a.half_tokens, tokens = min(w.tokens - x0, a.half_tokens);
      if (tokens <= 0) continue;
      const int tok = x0 + min(rt, tokens - 1);
      const int pos = w.pos + tok;
      const int base = w.pos - w.first;  // tree: where it begins
      bool astray = false;
      const int hi = TREE ? base : pos + 1;  // up to here every key from lo on is seen
      const int lo = TREE ? tree_first_seen(a, w.token + tok, base, w.first + tok, astray)
                          : first_seen(a, pos);
      if (TREE && astray) raise_status(a.dev_status, EBD_DEV_RANGE);
      // (whether keys are absent is known by the first product)
      if (!mbar_wait_warp(&bar->s_full[x][it & 1], (it >> 1) & 1)) {
        ok = false;
        break;
      }
      const bool absent_keys = bar->piece[i % kPieceSlots].absent;
      const int edge = absent_keys ? 0x7fffffff : lo;  // every tile is looked at then
      float m = -INFINITY, l = 0.f;
      for (int j = w.cur; j < w.end; ++j, ++it) {
        const int k0 = j * kTcBN;
        const uint32_t buf = sS + (it & 1) * 64;
        uint64_t visible = 0;
        if (TREE && __any_sync(0xffffffffu, hi - k0 < kTcBN || edge > k0))
          visible = tree_visible<kTcBN>(a, w.token + tok, w.first + tok, base, lo, k0);
        if (!mbar_wait_warp(&bar->s_full[x][it & 1], (it >> 1) & 1)) {
          ok = false;
          break;
        }
        tc_fence_after();
        uint32_t s[64];
        tmem_ld64(buf, s);
        tmem_ld_wait();
        if (__any_sync(0xffffffffu, hi - k0 < kTcBN || edge > k0)) {
          if (TREE) {
            const uint32_t v0 = (uint32_t)visible, v1 = (uint32_t)(visible >> 32);
#pragma unroll
            for (int i = 0; i < 64; ++i)
              if (!((i < 32 ? v0 : v1) >> (i & 31) & 1)) s[i] = __float_as_uint(-INFINITY);
          } else {
            const int chi = hi - k0, clo = lo - k0;
#pragma unroll
            for (int i = 0; i < 64; ++i)
              if (i >= chi || i < clo) s[i] = __float_as_uint(-INFINITY);
          }
          if (absent_keys) {
            const uint64_t absent = bar->absent[(tile0 + (j - w.cur)) % kAbsentSlots];
#pragma unroll
            for (int i = 0; i < 64; ++i)
              if (absent >> i & 1) s[i] = __float_as_uint(-INFINITY);
          }
        }
        float t4[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) t4[i] = __uint_as_float(s[i]);
#pragma unroll
        for (int i = 4; i < 60; i += 8)
#pragma unroll
          for (int e = 0; e < 4; ++e)
            t4[e] = max3(t4[e], __uint_as_float(s[i + 2 * e]), __uint_as_float(s[i + 2 * e + 1]));
        float top = fmaxf(max3(t4[0], t4[1], t4[2]),
                          max3(t4[3], __uint_as_float(s[60]), __uint_as_float(s[61])));
        top = max3(top, __uint_as_float(s[62]), __uint_as_float(s[63]));
        const bool grow = m > -INFINITY && (top - m) * a.scale2 > kRescaleLog2;
        if (__any_sync(0xffffffffu, grow)) {
          // O_X holds the tiles before this one: wait for their product
          if (!mbar_wait_warp(&bar->o_full[x][(it - 1) & 1], ((it - 1) >> 1) & 1)) {
            ok = false;
            break;
          }
          tc_fence_after();
          const float m1 = fmaxf(m, top);
          const float f = m > -INFINITY ? exp2f((m - m1) * a.scale2) : 1.f;
          l *= f;
          m = m1;
          // 16 columns at a time: the logits stay in registers meanwhile
#pragma unroll 1
          for (int c = 0; c < D; c += 16) {
            uint32_t o[16];
            tmem_ld16(sO + c, o);
            tmem_ld_wait();
#pragma unroll
            for (int i = 0; i < 16; ++i) o[i] = __float_as_uint(__uint_as_float(o[i]) * f);
            tmem_st16(sO + c, o);
          }
        } else if (m == -INFINITY) {
          m = top;  // nothing but zeros in O_X so far
        }
        const float base = m == -INFINITY ? 0.f : m * a.scale2;
        const float2 sc2 = make_float2(a.scale2, a.scale2), nb = make_float2(-base, -base);
        float2 sum0 = make_float2(0.f, 0.f), sum1 = sum0;
        uint32_t p[32];
#pragma unroll
        for (int i = 0; i < 32; i += 2) {
          float2 e = __ffma2_rn(
              make_float2(__uint_as_float(s[2 * i]), __uint_as_float(s[2 * i + 1])), sc2, nb);
          float2 f = __ffma2_rn(
              make_float2(__uint_as_float(s[2 * i + 2]), __uint_as_float(s[2 * i + 3])), sc2, nb);
          e.x = exp2f(e.x);
          e.y = exp2f(e.y);
          f.x = exp2f(f.x);
          f.y = exp2f(f.y);
          sum0 = __fadd2_rn(sum0, e);
          sum1 = __fadd2_rn(sum1, f);
          p[i] = pack_bf16(e.x, e.y);
          p[i + 1] = pack_bf16(f.x, f.y);
        }
        tmem_st32(buf, p);
        l += (sum0.x + sum0.y) + (sum1.x + sum1.y);
        tmem_st_wait();
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(&bar->p_full[x][it & 1]);
      }
      if (!ok) break;
      if (!mbar_wait_warp(&bar->o_full[x][(it - 1) & 1], ((it - 1) >> 1) & 1)) {
        ok = false;
        break;
      }
      tc_fence_after();
      const int slot = w.slot;
      const float inv = l == 0.f ? 0.f : 1.f / l;
      const bool mine = rt < tokens;
      const float lse2 = l == 0.f ? -INFINITY : m * a.scale2 + log2f(l);
      const long long out = (long long)(w.token + tok) * (a.pv.n_kv_heads * a.group) +
                            w.h * a.group + g;
      float* part = part_row<D>(a, slot, x * 128 + row);  // when slot >= 0
#pragma unroll
      for (int c = 0; c < D; c += 32) {
        uint32_t o[32];
        __syncwarp();
        tmem_ld32(sO + c, o);
        tmem_ld_wait();
        float z0 = 0.f, z1 = 0.f;  // NaN where an output is NaN or infinite
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          z0 = fmaf(__uint_as_float(o[i]), 0.f, z0);
          z1 = fmaf(__uint_as_float(o[16 + i]), 0.f, z1);
        }
        nonfinite = nonfinite || (mine && z0 + z1 != 0.f);
        if (!mine) {
        } else if (slot >= 0) {
          float* dst = part + c / 4 * a.part_step;
#pragma unroll
          for (int i = 0; i < 8; ++i)
            *reinterpret_cast<float4*>(dst + i * a.part_step) = make_float4(
                __uint_as_float(o[4 * i]) * inv, __uint_as_float(o[4 * i + 1]) * inv,
                __uint_as_float(o[4 * i + 2]) * inv, __uint_as_float(o[4 * i + 3]) * inv);
        } else {
          uint4* dst = reinterpret_cast<uint4*>((__nv_bfloat16*)a.y + out * D + c);
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            uint32_t q[4];
#pragma unroll
            for (int e = 0; e < 4; ++e)
              q[e] = pack_bf16(__uint_as_float(o[8 * i + 2 * e]) * inv,
                               __uint_as_float(o[8 * i + 2 * e + 1]) * inv);
            dst[i] = make_uint4(q[0], q[1], q[2], q[3]);
          }
        }
      }
      if (mine) {
        if (slot >= 0) a.part_lse[(size_t)slot * a.slot_rows + x * 128 + row] = lse2;
        else if (a.lse) a.lse[out] = l == 0.f ? -INFINITY : lse2 * kLn2;
      }
      __syncwarp();
      tc_fence_before();  // the reads of O_X, before the next item's first product
    }
    if (ok && __any_sync(0xffffffffu, nonfinite))
      mend_pieces<__nv_bfloat16, D, kTcBN, TREE>(a, cta, gridDim.x, x * a.half_tokens, x * 128,
                                           (warp & 3) * 32, 32, lane);
  } else if (warp < 10) {
    // ---------------- MMA issue: a warp per X (one thread's instructions between
    // the MMAs of both would take longer than the MMAs)
    const int x = warp - 8;
    if (elect_one()) {
      const uint32_t idesc_s = umma_idesc_bf16_f32(128, kTcBN);
      const uint32_t idesc_o = umma_idesc_bf16_f32_bt(128, D);
      // descriptors once; a step along them is an addition to the start address
      const uint64_t qd = umma_desc_k_sw128(smem_u32(smem + L::kQ + x * L::kQTile));
      const uint64_t kd = umma_desc_k_sw128(smem_u32(smem + L::kK));
      const uint64_t vd = umma_desc_mn_sw128(smem_u32(smem + L::kV), L::kBox);
      const uint32_t tS = tmem + 256 + x * 128, tO = tmem + x * 128;
      uint32_t ks = 0, kph = 0, vs = 0, vph = 0;  // ring positions and phases
      uint32_t n_s = 0, n_o = 0;                  // products issued so far
      uint32_t items = 0, fixes = 0;
      auto s_mma = [&](bool last) {
        if (!mbar_wait_bounded(&bar->k_full[ks], kph)) return false;
        // S overwrites the weights of two tiles ago: their product has to be done
        const uint32_t b = n_s & 1;
        if (n_s >= 2 && !mbar_wait_bounded(&bar->o_full[x][b], ((n_s >> 1) - 1) & 1)) return false;
        tc_fence_after();
        const uint64_t bd = kd + ks * (L::kTile >> 4);
        const uint32_t d = tS + b * 64;
#pragma unroll
        for (int kk = 0; kk < D / 16; ++kk)
          umma_bf16(d, qd + (uint32_t)(((kk >> 2) * L::kQBox + (kk & 3) * 32) >> 4),
                    bd + (uint32_t)(((kk >> 2) * L::kBox + (kk & 3) * 32) >> 4), idesc_s, kk > 0);
        umma_commit(&bar->s_full[x][b]);
        umma_commit(&bar->k_empty[ks]);
        if (last) umma_commit(&bar->q_empty);
        ++n_s;
        if (++ks == KS) ks = 0, kph ^= 1;
        return true;
      };
      auto o_mma = [&](bool first, bool fix) {
        const uint32_t b = n_o & 1;
        if (!mbar_wait_bounded(&bar->v_full[vs], vph)) return false;
        if (fix && !mbar_wait_bounded(&bar->fixed, fixes++ & 1)) return false;
        if (!mbar_wait_bounded(&bar->p_full[x][b], (n_o >> 1) & 1)) return false;
        tc_fence_after();
        const uint64_t bd = vd + vs * (L::kTile >> 4);
        const uint32_t p = tS + b * 64;
#pragma unroll
        for (int kk = 0; kk < kTcBN / 16; ++kk)
          umma_bf16_ta(tO, p + kk * 8, bd + (uint32_t)(kk * (2048 >> 4)), idesc_o, !first || kk > 0);
        umma_commit(&bar->o_full[x][b]);
        umma_commit(&bar->v_empty[vs]);
        ++n_o;
        if (++vs == KS) vs = 0, vph ^= 1;
        return true;
      };
      for (; ok; ++items) {
        const uint32_t at = items % kPieceSlots;
        ok = mbar_wait_bounded(&bar->piece_full[at], (items / kPieceSlots) & 1);
        if (!ok) break;
        const int n = bar->piece[at].end - bar->piece[at].cur;
        const bool two = bar->piece[at].tokens > a.half_tokens;
        // value rows to be cleared first
        const bool ragged_end = bar->piece[at].len < bar->piece[at].end * kTcBN;
        mbar_arrive(&bar->piece_empty[at]);
        if (n <= 0) break;
        ok = mbar_wait_bounded(&bar->q_full, items & 1);
        if (x == 1 && !two) {
          // A does the item alone.  B still follows every stage and gives its
          // consent to each reuse: no barrier's phase can pass it by.
          // (the last value tile is cleared only after q_empty: before its wait)
          if (ok && n == 1) mbar_arrive(&bar->q_empty);
          for (int t = 0; ok && t < n; ++t) {
            ok = mbar_wait_bounded(&bar->k_full[ks], kph) &&
                 mbar_wait_bounded(&bar->v_full[vs], vph) &&
                 (!ragged_end || t + 1 < n || mbar_wait_bounded(&bar->fixed, fixes++ & 1));
            mbar_arrive(&bar->k_empty[ks]);
            mbar_arrive(&bar->v_empty[vs]);
            if (++ks == KS) ks = 0, kph ^= 1;
            if (++vs == KS) vs = 0, vph ^= 1;
            if (t + 2 == n) mbar_arrive(&bar->q_empty);
          }
          continue;
        }
        ok = ok && s_mma(n == 1) && (n == 1 || s_mma(n == 2));
        for (int t = 0; ok && t < n; ++t) {
          ok = o_mma(t == 0, ragged_end && t + 1 == n);
          if (ok && t + 2 < n) ok = s_mma(t + 3 == n);
        }
      }
      umma_commit(&bar->done[x]);
      mbar_wait_bounded(&bar->done[x], 0);
    }
    ok = __all_sync(0xffffffffu, ok);
  } else if (warp == 10) {
    // ---------------- K and V copies, in the order K0 K1 V0 K2 V1 ... of the MMAs
    uint32_t nk = 0, nv = 0;  // tiles issued
    const int page = 1 << a.pv.page_shift;
    const int box = min(page, kTcBN), boxes = kTcBN / box;  // boxes of keys per tile
    bool any_absent = false;
    for (uint32_t i = 0; ok && read_piece(i, w); drop_piece(i++)) {
      // lane i: one box of a tile (keys bx * box .., channels half * 64 ..).  The
      // lanes look up 32 pages at a time (a lookup per tile would hold up the
      // copies by its latency); past the pool where there is none, before it (-1)
      // where the table names a page outside.
      const int bx = lane / L::kHalves, half = lane - bx * L::kHalves;
      int block0 = 0, entry = 0, held = 0;  // pages of blocks block0 .. + held - 1
      // pages before it may have been released
      const int seen = first_seen(a, TREE ? w.pos - w.first : w.pos);
      auto page_at = [&](int j) {
        const int first = (j * kTcBN) >> a.pv.page_shift;
        const int last = (j * kTcBN + kTcBN - 1) >> a.pv.page_shift;
        if (last >= block0 + held) {
          block0 = first;
          held = 32;
          const int blk = block0 + lane, pos = blk << a.pv.page_shift;
          entry = a.pv.n_pages;
          if (blk < a.pv.max_blocks && pos < w.len) {
            const int p = page_of(a.pv, w.b, pos);
            if (p >= 0 || pos + page > seen) entry = p;
          }
          any_absent = any_absent || __any_sync(0xffffffffu, entry < 0);  // (the entries begin as zeros)
        }
        return __shfl_sync(0xffffffffu, entry,
                           (((j * kTcBN + bx * box) >> a.pv.page_shift) - block0) & 31);
      };
      // Tells the softmax which keys of K tile nk are absent.
      auto tell_absent = [&](int pg) {
        uint64_t absent = 0;
        uint32_t out = __ballot_sync(0xffffffffu, pg < 0 && half == 0 && bx < boxes);
        for (; out; out &= out - 1)
          absent |= (box == 64 ? ~0ull : (1ull << box) - 1)
                    << ((__ffs(out) - 1) / L::kHalves * box);
        if (lane == 0) bar->absent[nk % kAbsentSlots] = absent;
      };
      auto copy = [&](const CUtensorMap* tm, int base, uint64_t* full, uint64_t* empty,
                      uint32_t n, int j, int pg) {
        const uint32_t slot = n % KS;
        if (n >= KS && !mbar_wait_warp(&empty[slot], (n / KS - 1) & 1)) return false;
        if (base == L::kK && any_absent) tell_absent(pg);
        if (lane == 0) mbar_arrive_expect_tx(&full[slot], L::kTile);
        __syncwarp();
        if (bx < boxes)
          tma_load_4d(smem + base + slot * L::kTile + half * L::kBox + bx * box * 128, tm,
                      half * 64, (j * kTcBN + bx * box) & (page - 1), w.h, pg, &full[slot]);
        __syncwarp();
        return true;
      };
      int pg = page_at(w.cur), next_pg = 0;
      ok = copy(&tmK, L::kK, bar->k_full, bar->k_empty, nk, w.cur, pg);
      if (ok) ++nk;
      for (int j = w.cur; ok && j < w.end; ++j) {
        if (j + 1 < w.end) {
          next_pg = page_at(j + 1);
          ok = copy(&tmK, L::kK, bar->k_full, bar->k_empty, nk, j + 1, next_pg);
          if (!ok) break;
          ++nk;
        }
        ok = copy(&tmV, L::kV, bar->v_full, bar->v_empty, nv, j, pg);
        if (!ok) break;
        ++nv;
        pg = next_pg;
      }
    }
    if (any_absent && lane == 0) raise_status(a.dev_status, EBD_DEV_RANGE);
    // every copy has landed before the block may end
    for (uint32_t i = nk > KS ? nk - KS : 0; i < nk; ++i)
      mbar_wait_bounded(&bar->k_full[i % KS], (i / KS) & 1);
    for (uint32_t i = nv > KS ? nv - KS : 0; i < nv; ++i)
      mbar_wait_bounded(&bar->v_full[i % KS], (i / KS) & 1);
  } else {
    // ---------------- the CTA's pieces; query rows; value rows past the end
    PieceWalk<kTcBN, TREE> walk(a, start);
    uint32_t items = 0, pushed = 0, tile0 = 0;  // tile0: tiles before this piece
    bool all = false;  // the end of the work was told
    PieceRecord record = {0, 0, 0, 0};
    // Tells the roles pieces up to the limit-th.
    auto push = [&](uint32_t limit) {
      for (; !all && pushed < limit; ++pushed) {
        const uint32_t at = pushed % kPieceSlots;
        if (pushed >= kPieceSlots &&
            !mbar_wait_warp(&bar->piece_empty[at], (pushed / kPieceSlots - 1) & 1))
          return false;
        Piece p = {};
        all = !walk.live();
        if (!all) {
          p.cur = walk.cur;
          p.end = walk.end;
          p.b = walk.b;
          p.h = walk.h;
          p.len = walk.sp.len;
          p.token = walk.sp.t0 + walk.first(a);
          p.pos = walk.sp.len - walk.sp.n + walk.first(a);
          p.tokens = walk.tokens(a);
          p.first = walk.first(a);
          p.slot = walk.slot(cta);
          record_piece(a, record, walk, pushed == 0);
        } else if (lane == 0) {
          a.rec[cta] = record;
        }
        if (lane == 0) {
          bar->piece[at] = p;
          mbar_arrive(&bar->piece_full[at]);
        }
        __syncwarp();
        if (!all) walk.next(a);
      }
      return true;
    };
    for (;; tile0 += w.end - w.cur, ++items) {
      if (!push(items + 1)) {
        ok = false;
        break;
      }
      if (all && items + 1 >= pushed) break;  // the last one pushed says that there are no more
      w = bar->piece[items % kPieceSlots];
      if (items > 0 && !mbar_wait_warp(&bar->q_empty, (items - 1) & 1)) {
        ok = false;
        break;
      }
      if (lane == 0) {
        const int nx = w.tokens > a.half_tokens ? 2 : 1;
        mbar_arrive_expect_tx(&bar->q_full, nx * L::kHalves * a.half_tokens * a.group * 128);
        for (int x = 0; x < nx; ++x)
#pragma unroll
          for (int h = 0; h < L::kHalves; ++h)
            tma_load_3d(smem + L::kQ + x * L::kQTile + h * L::kQBox, &tmQ, h * 64, w.h * a.group,
                        w.token + x * a.half_tokens, &bar->q_full);
      }
      __syncwarp();
      // The second arrival on q_full says that the piece's pages were looked up: the
      // first one's now, the others' a piece ahead.
      if (items > 0 && lane == 0) mbar_arrive(&bar->q_full);
      for (int turn = items > 0; ok && turn < 2; ++turn) {
        // two pieces ahead: the one two before this must have been dropped by then
        if (turn == 1 && !push(items + 3)) ok = false;
        const uint32_t at = items + turn;
        if (!ok || at + all >= pushed) break;
        const Piece& p = bar->piece[at % kPieceSlots];
        const int seen = first_seen(a, TREE ? p.pos - p.first : p.pos);
        const int first = max(p.cur * kTcBN, seen) >> a.pv.page_shift;
        const int past = min(p.end * kTcBN, p.len);
        bool out = false;
#pragma unroll 4
        for (int blk = first + lane; blk << a.pv.page_shift < past; blk += 32)
          out |= page_of(a.pv, p.b, blk << a.pv.page_shift) < 0;
        out = __any_sync(0xffffffffu, out);
        if (lane == 0) {
          bar->piece[at % kPieceSlots].absent = out;
          if (at == 0) mbar_arrive(&bar->q_full);
        }
        __syncwarp();
      }
      if (!ok) break;
      if (w.len < w.end * kTcBN) {
        // The piece's last value tile.  Its stage's phase is certain only once the
        // piece's last S product is done (q_empty): the stage's earlier tile
        // has landed by then, and no later one can take the stage before the
        // rows are cleared.
        const uint32_t at = tile0 + (w.end - w.cur) - 1;
        if (!mbar_wait_warp(&bar->q_empty, items & 1) ||
            !mbar_wait_warp(&bar->v_full[at % KS], (at / KS) & 1)) {
          ok = false;
          break;
        }
        const int first = w.len - (w.end - 1) * kTcBN;  // rows from here on are cleared
        unsigned char* v = smem + L::kV + (at % KS) * L::kTile;
        for (int i = max(first, 0) * 8 + lane; i < kTcBN * 8; i += 32)
#pragma unroll
          for (int h = 0; h < L::kHalves; ++h)
            *reinterpret_cast<uint4*>(v + h * L::kBox + i * 16) = make_uint4(0, 0, 0, 0);
        fence_proxy_async_smem();
        mbar_arrive(&bar->fixed);
      }
    }
  }
  if (!ok) {
    raise_status(a.dev_status, EBD_DEV_TIMEOUT);
    // the merge finds nothing to join
    if (warp == 11 && lane == 0) a.rec[cta] = PieceRecord{0, 0, 0, 0};
  }
  tc_fence_before();
  __syncthreads();
  if (warp == 8) {
    tc_fence_after();
    tmem_dealloc(tmem, 512);
  }
}

static PFN_cuTensorMapEncodeTiled_v12000 paged_encoder() {
  static PFN_cuTensorMapEncodeTiled_v12000 fn = nullptr;
  static std::once_flag once;
  std::call_once(once, [] {
    void* p = nullptr;
    cudaDriverEntryPointQueryResult q;
    if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &p, 12000, cudaEnableDefault,
                                         &q) == cudaSuccess &&
        q == cudaDriverEntryPointSuccess)
      fn = reinterpret_cast<PFN_cuTensorMapEncodeTiled_v12000>(p);
  });
  return fn;
}

// [page, head, row, channel] of one pool; box: 64 channels x rows of one page.
static bool encode_pool(CUtensorMap* map, const ebd_paged_cache& c, const void* base,
                        int box_rows) {
  auto enc = paged_encoder();
  if (!enc) return false;
  const cuuint64_t dims[4] = {(cuuint64_t)c.head_dim, (cuuint64_t)c.page_size,
                              (cuuint64_t)c.n_kv_heads, (cuuint64_t)c.n_pages};
  // a dimension of one entry never steps: any valid stride will do for it
  auto bytes = [&](int64_t s, int n) { return (cuuint64_t)(n > 1 ? s * 2 : c.head_dim * 2); };
  const cuuint64_t strides[3] = {bytes(c.row_stride, c.page_size),
                                 bytes(c.head_stride, c.n_kv_heads),
                                 bytes(c.page_stride, c.n_pages)};
  const cuuint32_t box[4] = {64, (cuuint32_t)box_rows, 1, 1}, one[4] = {1, 1, 1, 1};
  return enc(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 4, const_cast<void*>(base), dims, strides, box,
             one, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
             CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// Queries [token, head, channel]; box: 64 channels x the group's heads x the tokens
// of one X.
static bool encode_queries(CUtensorMap* map, const PagedAttnArgs& a, int head_dim) {
  auto enc = paged_encoder();
  if (!enc) return false;
  const int hq = a.pv.n_kv_heads * a.group;
  const cuuint64_t dims[3] = {(cuuint64_t)head_dim, (cuuint64_t)hq, (cuuint64_t)a.n_tokens};
  const cuuint64_t strides[2] = {(cuuint64_t)(hq > 1 ? a.q_hs * 2 : head_dim * 2),
                                 (cuuint64_t)(a.n_tokens > 1 ? a.q_ts * 2 : head_dim * 2)};
  const cuuint32_t box[3] = {64, (cuuint32_t)a.group, (cuuint32_t)a.half_tokens};
  const cuuint32_t one[3] = {1, 1, 1};
  return enc(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 3, const_cast<void*>(a.q), dims, strides, box,
             one, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
             CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <int D>
static ebd_status launch_tc_t(const PagedAttnArgs& a, const ebd_paged_cache& c, int n_cta,
                              cudaStream_t s) {
  CUtensorMap tmQ, tmK, tmV;
  const int box = c.page_size < kTcBN ? c.page_size : kTcBN;
  if (!encode_queries(&tmQ, a, D) || !encode_pool(&tmK, c, c.K_pages, box) || !encode_pool(&tmV, c, c.V_pages, box))
    return EBD_ERR_CUDA;
  constexpr int smem = PagedTcLayout<D>::kBytes;
  auto kern = a.mask     ? paged_attn_tc_kernel<D, true, true>
              : a.padded ? paged_attn_tc_kernel<D, false, true>
                         : paged_attn_tc_kernel<D, false, false>;
  if (cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, smem) != cudaSuccess)
    return EBD_ERR_CUDA;
  return launch_dependent(kern, dim3(n_cta), kTcAttnThreads, smem, s, tmQ, tmK, tmV, a);
}

ebd_status launch_paged_tc(PagedAttnArgs a, const ebd_paged_cache& c, int n_cta,
                           cudaStream_t s) {
  // whole tokens in each X of 128 rows (126 of them used at G = 7): one TMA box
  a.heads = a.pv.n_kv_heads;
  a.slices = 1;
  a.slice = a.group;
  a.half_tokens = 128 / a.group;
  a.tokens = 2 * a.half_tokens;
  // measured: 1070 cycles per tile of one X, 1370 of two (64 channels); equal weights
  // left CTAs between 52k and 82k cycles of work in the mixed batch, these 64k to 77k.
  // 16 mixed sequences of up to 5k tokens, half of them single steps, 2 : 3 against equal
  // weights (and 2 : 4), us: 64 channels with a window of 1024 41.4 / 43.5 (46.2), without
  // 67 / 70 (81); 128 channels with the window 54.2 / 55.0 (62.4), without 89 / 86 (108), and
  // over 3-16k positions 413-423 / 350-390 (510): there equal weights are better
  a.tile_work = 2;
  a.full_work = 3;
  a.min_share = 8;  // more than a tile: a CTA in the middle of an item has one at least
  a.item_cost = 8;
  if (!line_fits(a, kTcBN)) return EBD_ERR_UNSUPPORTED;
  const ebd_status st =
      c.head_dim == 128 ? launch_tc_t<128>(a, c, n_cta, s) : launch_tc_t<64>(a, c, n_cta, s);
  if (st != EBD_OK) return st;
  return launch_paged_merge(a, true, c.head_dim, n_cta, s);
}

}  // namespace ebd
