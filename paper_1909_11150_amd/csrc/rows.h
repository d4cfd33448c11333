// Rows of any width, stride and element alignment in chunks of 8 elements, and the 8-bit
// checkpoint of an activation.
#pragma once
#include "common.h"
#include "dma_pipe.h"

namespace fg {
namespace rows {

// Element types by their code.
template <int DT>
struct TypeOf;
template <>
struct TypeOf<FG_F16> {
  using T = _Float16;
};
template <>
struct TypeOf<FG_BF16> {
  using T = __bf16;
};
template <>
struct TypeOf<FG_F32> {
  using T = float;
};

// 8 elements as they are in memory.
template <class T>
struct Raw {
  u32x4 w[sizeof(T) / 2];
};

// Loads chunk c (a multiple of 8) of a row of at least 8 elements. Where the row ends within
// or before the chunk, the last 8 elements come in its place; values() moves them. No branch:
// several chunks' loads are on their way together.
template <class T>
__device__ __forceinline__ Raw<T> load_raw(const T *row, int c, int cols) {
  Raw<T> r;
  const T *p = row + min(c, cols - 8);
#pragma unroll
  for (int k = 0; k < (int)(sizeof(T) / 2); ++k)
    r.w[k] = reinterpret_cast<const Any16 *>(p + 8 / (sizeof(T) / 2) * k)->v;
  return r;
}

// ... of a row of fewer.
template <class T>
__device__ __forceinline__ Raw<T> load_narrow(const T *row, int c, int cols) {
  T v[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) v[e] = c + e < cols ? row[c + e] : (T)0.f;
  return __builtin_bit_cast(Raw<T>, v);
}

// Elements that belong before chunk c where the row's last 8 came in its place; 8 and more: all.
__device__ __forceinline__ int before(int c, int cols) { return c - min(c, cols - 8); }

// The chunk's elements as fp32, zeros past the row's end.
template <class T>
__device__ __forceinline__ void values(const Raw<T> &r, int c, int cols, float (&v)[8]) {
  typedef T t8 __attribute__((ext_vector_type(8)));
  Raw<T> x = r;
  if (cols >= 8) {
    const int s = before(c, cols);
    if (cols % 8 == 0) {
#pragma unroll
      for (int k = 0; k < (int)(sizeof(T) / 2); ++k)
        if (s) x.w[k] = u32x4{0, 0, 0, 0};
    } else if constexpr (sizeof(T) == 2) {
      // whole words by selection, the odd element by a shift across words
      u32x4 w = x.w[0];
      w = s & 8 || s >= 16 ? u32x4{0, 0, 0, 0} : w;
      w = s & 4 ? u32x4{w[2], w[3], 0, 0} : w;
      w = s & 2 ? u32x4{w[1], w[2], w[3], 0} : w;
      const uint32_t sh = 16 * (s & 1);
#pragma unroll
      for (int d = 0; d < 4; ++d)
        x.w[0][d] = __builtin_amdgcn_alignbit(d < 3 ? w[d + 1] : 0u, w[d], sh);
    } else {
      uint32_t w[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) w[e] = s >= 8 ? 0u : r.w[e / 4][e % 4];
#pragma unroll
      for (int b = 4; b; b >>= 1)
#pragma unroll
        for (int e = 0; e < 8; ++e) w[e] = s & b ? (e + b < 8 ? w[e + b] : 0u) : w[e];
#pragma unroll
      for (int e = 0; e < 8; ++e) x.w[e / 4][e % 4] = w[e];
    }
  }
  const t8 q = __builtin_bit_cast(t8, x);
#pragma unroll
  for (int e = 0; e < 8; ++e) v[e] = (float)q[e];
}

template <class T>
__device__ __forceinline__ Raw<T> load_any(const T *row, int c, int cols) {
  return cols >= 8 ? load_raw(row, c, cols) : load_narrow(row, c, cols);
}

template <class T>
__device__ __forceinline__ void load8(const T *row, int c, int cols, float (&v)[8]) {
  values<T>(load_any(row, c, cols), c, cols, v);
}

// Rounds 8 values once to T and writes those within the row: its last ones, where they are
// fewer, in pieces of 4, 2 and 1.
template <class T>
__device__ __forceinline__ void store8(T *row, int c, int cols, const float (&v)[8]) {
  T q[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) q[e] = (T)v[e];
  const Raw<T> r = __builtin_bit_cast(Raw<T>, q);
  T *p = row + c;
  if (c + 8 <= cols) {
#pragma unroll
    for (int k = 0; k < (int)(sizeof(T) / 2); ++k)
      reinterpret_cast<Any16 *>(p + 8 / (sizeof(T) / 2) * k)->v = r.w[k];
    return;
  }
  const int n = cols - c;
  if (n <= 0) return;
  typedef uint16_t bits;
  if constexpr (sizeof(T) == 2) {
    u32x2 w = {r.w[0][0], r.w[0][1]};
    if (n & 4) {
      reinterpret_cast<Any8 *>(p)->v = w;
      w = u32x2{r.w[0][2], r.w[0][3]};
      p += 4;
    }
    uint32_t h = w[0];
    if (n & 2) {
      reinterpret_cast<Any4 *>(p)->v = h;
      h = w[1];
      p += 2;
    }
    if (n & 1) *reinterpret_cast<bits *>(p) = (bits)h;
  } else {
    u32x4 w = r.w[0];
    if (n & 4) {
      reinterpret_cast<Any16 *>(p)->v = w;
      w = r.w[1];
      p += 4;
    }
    uint32_t h = w[0];
    if (n & 2) {
      reinterpret_cast<Any8 *>(p)->v = u32x2{w[0], w[1]};
      h = w[2];
      p += 2;
    }
    if (n & 1) reinterpret_cast<Any4 *>(p)->v = h;
  }
}

// ---- across lanes ----------------------------------------------------------------------
// The value of the lane whose number differs in bit O, for values that agree within groups of
// O lanes (a mirrored row then is as good as an exchange): VALU moves, no trip through LDS.
template <int O>
__device__ __forceinline__ uint32_t across(uint32_t v) {
  static_assert(O == 1 || O == 2 || O == 4 || O == 8, "within a row of 16 lanes");
  constexpr int kCtrl = O == 1 ? 0xB1 : O == 2 ? 0x4E : O == 4 ? 0x141 : 0x140;
  return (uint32_t)__builtin_amdgcn_mov_dpp((int)v, kCtrl, 0xF, 0xF, true);
}
// Joins each lane's value with those of the TL - 1 lanes beside it, in all of them.
template <int TL, class Join>
__device__ __forceinline__ uint32_t join_lanes(uint32_t v, Join &&join) {
  if constexpr (TL >= 2) v = join(v, across<1>(v));
  if constexpr (TL >= 4) v = join(v, across<2>(v));
  if constexpr (TL >= 8) v = join(v, across<4>(v));
  if constexpr (TL >= 16) v = join(v, across<8>(v));
  if constexpr (TL >= 32) {
    const auto p = __builtin_amdgcn_permlane16_swap(v, v, false, false);
    v = join(p[0], p[1]);
  }
  if constexpr (TL >= 64) {
    const auto p = __builtin_amdgcn_permlane32_swap(v, v, false, false);
    v = join(p[0], p[1]);
  }
  return v;
}
template <int TL>
__device__ __forceinline__ float sum_lanes(float v) {
  return __builtin_bit_cast(
      float, join_lanes<TL>(__builtin_bit_cast(uint32_t, v), [](uint32_t a, uint32_t b) {
        return __builtin_bit_cast(
            uint32_t, __builtin_bit_cast(float, a) + __builtin_bit_cast(float, b));
      }));
}
template <int TL>
__device__ __forceinline__ uint32_t max_lanes(uint32_t v) {
  return join_lanes<TL>(v, [](uint32_t a, uint32_t b) { return max(a, b); });
}

// ---- 8-bit checkpoints ---------------------------------------------------------------
// rows x cols values in row-major codes (signed bytes, rows padded with zeros to a multiple
// of 32 columns), then one byte for each 32 columns of a row: the biased exponent b, at least
// 8, of the largest magnitude; a code stands for code * 2^(b - 133), so the largest is 64 ..
// 127 steps. A power of two makes packing exact but for the one rounding, and the value exact
// in fp16 and bf16 where it came from that type: 7 bits, and no bit below the type's last one
// (128 steps would leave fp16's range at its top: codes end at 127, one step's error there).
// Infinities and NaN are the code -128, which comes back as NaN: what a checkpoint loses must
// not hide an overflow from the gradients' check.
struct Packed {
  int8_t *codes;
  uint8_t *exps;
  int32_t wide;    // columns of a row of codes
};
__host__ __device__ inline int64_t packed_cols(int64_t cols) { return (cols + 31) / 32 * 32; }
__host__ __device__ inline Packed packed_at(const void *p, int64_t rows, int64_t cols) {
  const int64_t wide = packed_cols(cols);
  int8_t *codes = static_cast<int8_t *>(const_cast<void *>(p));
  return {codes, reinterpret_cast<uint8_t *>(codes + rows * wide), (int32_t)wide};
}

constexpr uint32_t kInf = 0x7F800000u;
__device__ __forceinline__ uint32_t magnitude(float v) {
  return __builtin_bit_cast(uint32_t, v) & 0x7FFFFFFFu;
}
__device__ __forceinline__ uint32_t finite_magnitude(float v) {  // 0 where v is no number
  const uint32_t u = magnitude(v);
  return u < kInf ? u : 0u;
}
// Of the largest magnitude of a group.
__device__ __forceinline__ uint32_t group_exp(uint32_t top) { return max(top >> 23, 8u); }
__device__ __forceinline__ float step_of(uint32_t b) {
  return __builtin_bit_cast(float, (b - 6u) << 23);
}
__device__ __forceinline__ float steps_of(uint32_t b) {  // its reciprocal
  return __builtin_bit_cast(float, (260u - b) << 23);
}
// A number's code in the low byte: adding 1.5 * 2^23 rounds to a whole number, halves to even,
// and leaves it in the sum's low bits.
__device__ __forceinline__ uint32_t code_of(float v, float inv) {
  constexpr float k = 12582912.f;
  return __builtin_bit_cast(uint32_t,
                            __builtin_amdgcn_fmed3f(fmaf(v, inv, k), k - 127.f, k + 127.f));
}
__device__ __forceinline__ uint32_t any_code_of(float v, float inv) {
  return magnitude(v) < kInf ? code_of(v, inv) : 0x80u;
}
__device__ __forceinline__ uint32_t bytes4(uint32_t a, uint32_t b, uint32_t c, uint32_t d) {
  const uint32_t lo = __builtin_amdgcn_perm(b, a, 0x0C0C0400u);
  const uint32_t hi = __builtin_amdgcn_perm(d, c, 0x0C0C0400u);
  return lo | hi << 16;
}

// Packs a group of 32 values that lies in several lanes, N a lane: `widest` takes a lane's
// largest magnitude to the group's. Returns the exponent; q: the codes, four a word. Groups
// with infinities or NaN (rare) go a slower way, all lanes of the wave together.
template <int N, class Widest>
__device__ __forceinline__ uint32_t pack_group(const float (&v)[N], uint32_t (&q)[N / 4],
                                               Widest &&widest) {
  uint32_t top = 0;
#pragma unroll
  for (int e = 0; e < N; ++e) top = max(top, magnitude(v[e]));
  top = widest(top);
  if (__builtin_expect(__any(top >= kInf), 0)) {
    top = 0;
#pragma unroll
    for (int e = 0; e < N; ++e) top = max(top, finite_magnitude(v[e]));
    top = widest(top);
    const float inv = steps_of(group_exp(top));
#pragma unroll
    for (int g = 0; g < N / 4; ++g)
      q[g] = bytes4(any_code_of(v[4 * g], inv), any_code_of(v[4 * g + 1], inv),
                    any_code_of(v[4 * g + 2], inv), any_code_of(v[4 * g + 3], inv));
    return group_exp(top);
  }
  const uint32_t b = group_exp(top);
  const float inv = steps_of(b);
#pragma unroll
  for (int g = 0; g < N / 4; ++g)
    q[g] = bytes4(code_of(v[4 * g], inv), code_of(v[4 * g + 1], inv), code_of(v[4 * g + 2], inv),
                  code_of(v[4 * g + 3], inv));
  return b;
}

// 8 codes as values.
__device__ __forceinline__ void decode8(const u32x2 &q, uint32_t b, float (&v)[8]) {
  const float step = step_of(b);
#pragma unroll
  for (int e = 0; e < 8; ++e) v[e] = (float)(int8_t)(q[e >> 2] >> (8 * (e & 3))) * step;
  // a byte 0x80 somewhere: the code of what is no number
  const u32x2 u = {q[0] ^ 0x80808080u, q[1] ^ 0x80808080u};
  const uint32_t z = ((u[0] - 0x01010101u) & ~u[0]) | ((u[1] - 0x01010101u) & ~u[1]);
  if (__builtin_expect((z & 0x80808080u) != 0, 0)) {
#pragma unroll
    for (int e = 0; e < 8; ++e)
      if ((uint8_t)(u[e >> 2] >> (8 * (e & 3))) == 0) v[e] = __builtin_nanf("");
  }
}

// Packs this lane's 8 values of a row, 4 lanes (a multiple of 4 and the next three) to a
// group of 32 columns; every lane of the four takes part, those past the end with zeros.
__device__ __forceinline__ void pack8(const Packed &p, int64_t row, int c, const float (&v)[8]) {
  uint32_t q[2];
  const uint32_t b = pack_group<8>(
      v, q, [](uint32_t top) __attribute__((always_inline)) { return max_lanes<4>(top); });
  if (c >= p.wide) return;
  *reinterpret_cast<u32x2 *>(p.codes + row * p.wide + c) = u32x2{q[0], q[1]};
  if (c % 32 == 0) p.exps[row * (p.wide / 32) + c / 32] = (uint8_t)b;
}

// Sums of n rows of fp32 parts, `stride` elements apart, over 16 columns from c0 on (fewer
// where `wide`, a multiple of 4, ends): 256 threads, 4 columns and every 64th row each, then
// the 64 sums of a column in order. The sum of column c0 + i is thread i's, i < 16. (Threads
// past the 256th wait only.)
constexpr int kSumLds = 64 * 5 * 16;
__device__ __forceinline__ void sum_columns(const float *part, int n, int64_t stride, int c0,
                                            int wide, void *lds, float &sum) {
  f32x4(*sh)[5] = static_cast<f32x4(*)[5]>(lds);
  const int t = threadIdx.x, c = min(c0 + 4 * (t & 3), wide - 4);
  f32x4 s = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 8
  for (int k = t >> 2; k < n && t < 256; k += 64)
    s += *reinterpret_cast<const f32x4 *>(part + k * stride + c);
  if (t < 256) sh[t >> 2][t & 3] = s;
  __syncthreads();
  sum = 0.f;
  if (t < 16) {
    const float *p = reinterpret_cast<const float *>(&sh[0][0]) + t;
#pragma unroll 8
    for (int k = 0; k < 64; ++k) sum += p[20 * k];
  }
}

}  // namespace rows
}  // namespace fg
