// What the tiled matrix products of the classification head (xent.hip) and of linear layers
// (linear.hip) share: rows of any width in chunks of 8, stores, tile order.
#pragma once
#include <algorithm>

#include "dma_pipe.h"

namespace fg {
namespace tiles {

using namespace dma;

using P128 = Pipe<64, 2, 2, 2, 128, 128>;  // 4 waves of 64 x 64
using P64 = Pipe<64, 3, 2, 2, 64, 64>;     // 4 waves of 32 x 32

// Rows are taken in chunks of 8 elements. A width that is no multiple of 8 has a last
// chunk that begins before its place, at width - 8, so that nothing outside the row is
// read or written; what it repeats is left out of sums over the width (logits), and
// written twice, alike, where the width is an output's (dh, dW).
__device__ __forceinline__ int chunk_at(int c, int width) { return min(c, width - 8); }

// 8 elements of a row from column c on, zeros past its end.
__device__ __forceinline__ u32x4 row8(const uint16_t *row, int c, int n) {
  if (c + 8 <= n) return reinterpret_cast<const Any16 *>(row + c)->v;
  u32x4 v = {0, 0, 0, 0};
#pragma unroll
  for (int e = 0; e < 8; ++e)
    if (c + e < n) v[e >> 1] |= (uint32_t)row[c + e] << (16 * (e & 1));
  return v;
}
__device__ __forceinline__ void put8(uint16_t *row, int c, int n, const u32x4 &v) {
  if (c + 8 <= n) {
    reinterpret_cast<Any16 *>(row + c)->v = v;
    return;
  }
#pragma unroll
  for (int e = 0; e < 8; ++e)
    if (c + e < n) row[c + e] = (uint16_t)(v[e >> 1] >> (16 * (e & 1)));
}

// A barrier for what waves exchange in LDS: global stores on their way are not waited
// for (__syncthreads does; at the end of a tile that is a trip to memory).
__device__ __forceinline__ void lds_barrier() {
  asm volatile("" ::: "memory");
  wait_lds();
  barrier_nofence();
}

// This wave's part of the ring, 64 WM bytes, once every wave is done reading it.
template <class P>
__device__ __forceinline__ uint8_t *wave_buf(const Ring &R, int wave) {
  constexpr int S = 64 * P::WM, PER = P::A_BYTES / S;
  static_assert(PER > 0 && (P::NW + PER - 1) / PER <= P::NS, "the ring stages a store");
  uint8_t *buf = R.a[0];
#pragma unroll
  for (int k = 1; k < (P::NW + PER - 1) / PER; ++k)
    if (wave / PER == k) buf = R.a[k];
  return buf + (wave % PER) * S;
}

// Writes 8 columns of a row of `width` elements that were computed as chunk c.
__device__ __forceinline__ void put_chunk(uint16_t *row, int c, int width, const u32x4 &v) {
  put8(row, width >= 8 ? chunk_at(c, width) : c, width, v);
}

// 16-bit store of a wave's block: pack(i, j, g) gives 4 consecutive columns of lane
// row 32 j + lane % 32, put(row, column, 8 values) writes them, both counted in the
// block. 32 rows at a time go through this wave's buffer, 16-byte chunks permuted
// by the row, so that neighbouring lanes write one row's consecutive bytes.
template <class P, class Pack, class Put>
__device__ __forceinline__ void store16(uint8_t *buf, int lane, Pack &&pack, Put &&put) {
  constexpr int CPW = P::WM / 8, RB = P::WM * 2, SH = CPW == 16 ? 0 : CPW == 8 ? 1 : 2;
#pragma unroll
  for (int j = 0; j < P::FN; ++j) {
    const int p = lane & 31;
#pragma unroll
    for (int i = 0; i < P::FM; ++i)
#pragma unroll
      for (int g = 0; g < 4; ++g)
        *reinterpret_cast<u32x2 *>(buf + p * RB +
                                   (((4 * i + g) ^ ((p >> SH) & (CPW - 1))) << 4) +
                                   8 * (lane >> 5)) = pack(i, j, g);
    wait_lds();
    __builtin_amdgcn_wave_barrier();
    constexpr int RPI = 64 / CPW;
    const int q = lane % CPW;
    u32x4 d[32 / RPI];
#pragma unroll
    for (int k = 0; k < 32 / RPI; ++k) {
      const int r = k * RPI + lane / CPW;
      d[k] = *reinterpret_cast<const u32x4 *>(buf + r * RB + ((q ^ ((r >> SH) & (CPW - 1))) << 4));
    }
#pragma unroll
    for (int k = 0; k < 32 / RPI; ++k) put(32 * j + k * RPI + lane / CPW, 8 * q, d[k]);
    wait_lds();
    __builtin_amdgcn_wave_barrier();
  }
}

__device__ __forceinline__ uint32_t pack2(float a, float b, bool bf) {
  if (bf) {
    typedef __bf16 b2 __attribute__((ext_vector_type(2)));
    return __builtin_bit_cast(uint32_t, b2{(__bf16)a, (__bf16)b});
  }
  typedef _Float16 h2 __attribute__((ext_vector_type(2)));
  return __builtin_bit_cast(uint32_t, h2{(_Float16)a, (_Float16)b});
}

__device__ __forceinline__ __amdgpu_buffer_rsrc_t rsrc(const void *p, uint32_t bytes) {
  return __builtin_amdgcn_make_buffer_rsrc(const_cast<void *>(p), 0, (int)bytes, kRsrcFlags);
}

// ---- tile order -----------------------------------------------------------------------
// Tiles of a band, see tile_map (8192 x 4096 x 131072: logits 3.50 -> 3.38 ms a piece and
// products 6.94 -> 6.81 against bands of one; of eight 3.41 and 6.90).
constexpr int kBand = 4;
// Tile (x, y, part) of n1 tiles along y at place v of the order that tile_map lays down.
__device__ __forceinline__ bool find_tile(const TileMap &tm, int block, int n1, int &x, int &y,
                                          int &part) {
  int i, z;
  if (!tm.decode(block, i, x, z)) return false;
  const int nb = (n1 + tm.n0 - 1) / tm.n0;
  part = z / nb;
  y = (z - part * nb) * tm.n0 + i;
  return y < n1;
}

inline int64_t up(int64_t n, int64_t unit) { return (n + unit - 1) / unit * unit; }

// Tiles in bands of up to kBand along the second axis (classes, or output rows), in which
// the first axis comes next and the parts of a sum last: an XCD, which runs some 32
// tiles at a time, then reads 4 + 8 panels of operands for them and not 16 + 2.
inline TileMap tile_map(int64_t n0, int64_t n1, int64_t n2) {
  const int64_t b = std::min<int64_t>(n1, kBand), nb = (n1 + b - 1) / b;
  return {(int32_t)b, (int32_t)n0, (int32_t)(nb * n2), (int32_t)((b * n0 * nb * n2 + 7) / 8),
          kOutputMajor};
}

struct Shape {
  int tile, ns, kper;  // tile: index; parts of the sum, length of one
};

}  // namespace tiles
}  // namespace fg
