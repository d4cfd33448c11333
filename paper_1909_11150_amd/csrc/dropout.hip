// Dropout whose mask comes from a counter-based generator and is stored nowhere.
//
// y = z + keep * x / q (q: the probability of keeping), or with a gate dx =
// keep * (gate > 0) * dy / q. The mask is a function of the element's index, a
// seed, a step and a site, so the backward pass draws it again.
//
// Generator: Philox 4x32 (Salmon, Moraes, Dror, Shaw, "Parallel random numbers:
// as easy as 1, 2, 3", 2011) with 7 rounds, the fewest the paper finds to pass
// its whole battery of tests. One block of 128 bits decides 8 elements, 16 bits
// each: a 32-bit number per element would double the integer multiplies, which
// run at a quarter of the VALU rate, for a finer p than 1/65536.
//
// Bound by memory: one read, one read of the residual or gate, one write. Measured
// (MI355X): 65536 x 256 fp16 slices of 1024-wide buffers 11.2 us (6.0 TB/s, as much as a
// copy of that size, which the caches serve in part), their gated gradients 17.5 us (5.7),
// 16384 x 4096 bf16 with a residual 73 us (5.5; a 2 GiB copy runs at 5.0), 8191 rows of
// 1023 of 1030 fp32 to dense ones 14.2 us (4.7). Strided rows off the 16-byte grid take one
// element per lane and access: 16383 rows of 4095 of 4099 fp32 131 us (4.1 TB/s), fp16 114 us
// (2.4), bf16 with a residual 119 us (3.4).
#include <algorithm>

#include "dma_pipe.h"

namespace fg {
namespace dropout {

constexpr int kThreads = 256;

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

struct Args {
  const void *x, *z;
  void *y;
  const int32_t *step_count;
  int64_t xl, yl, zl;    // row strides, elements
  uint64_t n;            // elements
  uint32_t cols;         // 0: one dense row
  uint32_t k0, k1, step, site;
  uint32_t threshold;    // kept: 16 bits below it
  float scale;
  dma::FastDiv div;      // by a row's blocks (vector kernel) or elements
};

// The 8 decisions of block b: bit e is set where element 8 b + e is kept.
__device__ __forceinline__ uint32_t keep8(uint32_t b, const Args &a, uint32_t step) {
  uint32_t c0 = b, c1 = 0, c2 = step, c3 = a.site, k0 = a.k0, k1 = a.k1;
#pragma unroll
  for (int r = 0; r < 7; ++r) {
    const uint64_t p = (uint64_t)c0 * 0xD2511F53u, q = (uint64_t)c2 * 0xCD9E8D57u;
    c0 = (uint32_t)(q >> 32) ^ c1 ^ k0;
    c1 = (uint32_t)q;
    c2 = (uint32_t)(p >> 32) ^ c3 ^ k1;
    c3 = (uint32_t)p;
    k0 += 0x9E3779B9u;
    k1 += 0xBB67AE85u;
  }
  const uint32_t w[4] = {c0, c1, c2, c3};
  uint32_t keep = 0;
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    keep |= (uint32_t)((w[j] & 0xFFFFu) < a.threshold) << (2 * j);
    keep |= (uint32_t)((w[j] >> 16) < a.threshold) << (2 * j + 1);
  }
  return keep;
}

__device__ __forceinline__ uint32_t step_of(const Args &a) {
  return a.step + (a.step_count ? (uint32_t)*a.step_count : 0u);
}

// 8 consecutive elements as fp32. 16-bit ones take one 16-byte access.
template <class T>
__device__ __forceinline__ void load8(const T *p, float (&v)[8]) {
  if constexpr (sizeof(T) == 2) {
    typedef T t8 __attribute__((ext_vector_type(8)));
    const t8 q = __builtin_bit_cast(t8, *reinterpret_cast<const u32x4 *>(p));
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = (float)q[e];
  } else {
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const f32x4 q = *reinterpret_cast<const f32x4 *>(p + 4 * h);
#pragma unroll
      for (int e = 0; e < 4; ++e) v[4 * h + e] = q[e];
    }
  }
}

template <class T>
__device__ __forceinline__ void store8(T *p, const float (&v)[8]) {
  if constexpr (sizeof(T) == 2) {
    typedef T t8 __attribute__((ext_vector_type(8)));
    t8 q;
#pragma unroll
    for (int e = 0; e < 8; ++e) q[e] = (T)v[e];
    *reinterpret_cast<u32x4 *>(p) = __builtin_bit_cast(u32x4, q);
  } else {
#pragma unroll
    for (int h = 0; h < 2; ++h)
      *reinterpret_cast<f32x4 *>(p + 4 * h) =
          f32x4{v[4 * h], v[4 * h + 1], v[4 * h + 2], v[4 * h + 3]};
  }
}

enum { kPlain = 0, kResidual = 1, kGate = 2 };

// A dropped element is +0 whatever it was (infinities and NaN too): selected,
// not multiplied.
template <int Z>
__device__ __forceinline__ float apply(float x, float z, bool keep, float scale) {
#pragma clang fp contract(off)  // the product is rounded whatever is added to it
  if (Z == kGate) keep = keep && z > 0.f;
  // the empty asm keeps the product an fp32 instruction of its own: fused with the
  // rounding to fp16 it would be fma(x, scale, +0), which turns -0 into +0
  float v = x * scale;
  asm("" : "+v"(v));
  v = keep ? v : 0.f;
  return Z == kResidual ? z + v : v;
}

// One block (8 elements) per lane and turn: rows whose blocks are aligned.
template <int DT, int Z>
__global__ __launch_bounds__(kThreads) void dropout_kernel(Args a) {
  using T = typename TypeOf<DT>::T;
  const uint32_t step = step_of(a);
  const uint64_t nb = (a.n + 7) / 8, stride = (uint64_t)gridDim.x * kThreads;
  for (uint64_t b = (uint64_t)blockIdx.x * kThreads + threadIdx.x; b < nb; b += stride) {
    uint64_t ox = b * 8, oy = ox, oz = ox;
    if (a.cols) {
      const uint32_t row = a.div.div((uint32_t)b), c = ((uint32_t)b - row * (a.cols / 8)) * 8;
      ox = row * a.xl + c, oy = row * a.yl + c, oz = row * a.zl + c;
    }
    const T *x = static_cast<const T *>(a.x) + ox, *z = static_cast<const T *>(a.z) + oz;
    T *y = static_cast<T *>(a.y) + oy;
    if (b * 8 + 8 <= a.n) {
      float v[8], w[8];
      load8(x, v);
      if (Z != kPlain) load8(z, w);
      const uint32_t keep = keep8((uint32_t)b, a, step);
#pragma unroll
      for (int e = 0; e < 8; ++e)
        v[e] = apply<Z>(v[e], Z ? w[e] : 0.f, keep >> e & 1, a.scale);
      store8(y, v);
    } else {  // the end of a dense tensor
      const uint32_t keep = keep8((uint32_t)b, a, step);
      for (int e = 0; e < (int)(a.n - b * 8); ++e)
        y[e] = (T)apply<Z>((float)x[e], Z ? (float)z[e] : 0.f, keep >> e & 1, a.scale);
    }
  }
}

// Any width, stride and alignment: a wave decides 512 consecutive elements, a
// block per lane, and then takes them 64 at a time, so that its accesses are
// contiguous within a row; each lane fetches its decision from the lane that drew
// it.
template <int DT, int Z>
__global__ __launch_bounds__(kThreads) void dropout_any_kernel(Args a) {
  using T = typename TypeOf<DT>::T;
  const uint32_t step = step_of(a);
  const int lane = threadIdx.x & 63;
  const uint64_t waves = (uint64_t)gridDim.x * (kThreads / 64);
  for (uint64_t w = (uint64_t)blockIdx.x * (kThreads / 64) + threadIdx.x / 64; w * 512 < a.n;
       w += waves) {
    const uint32_t mine = keep8((uint32_t)(w * 64 + lane), a, step);
    const uint64_t row0 = w * 512 / a.cols;
    const uint32_t rem = (uint32_t)(w * 512 - row0 * a.cols);
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const uint32_t keep = __shfl(mine, 8 * j + (lane >> 3)) >> (lane & 7) & 1;
      const uint32_t e = rem + 64 * j + lane, r = a.div.div(e), c = e - r * a.cols;
      const uint64_t row = row0 + r;
      if (w * 512 + 64 * j + lane < a.n) {
        const float x = (float)static_cast<const T *>(a.x)[row * a.xl + c];
        const float z = Z ? (float)static_cast<const T *>(a.z)[row * a.zl + c] : 0.f;
        static_cast<T *>(a.y)[row * a.yl + c] = (T)apply<Z>(x, z, keep, a.scale);
      }
    }
  }
}

template <int DT, int Z>
hipError_t launch(const Args &a, bool vec, hipStream_t st) {
  const uint64_t per = vec ? (uint64_t)kThreads * 8 : (uint64_t)kThreads / 64 * 512;
  const uint32_t grid = (uint32_t)std::min<uint64_t>((a.n + per - 1) / per, 256 * 32);
  if (vec)
    hipLaunchKernelGGL((dropout_kernel<DT, Z>), dim3(grid), dim3(kThreads), 0, st, a);
  else
    hipLaunchKernelGGL((dropout_any_kernel<DT, Z>), dim3(grid), dim3(kThreads), 0, st, a);
  return hipGetLastError();
}

template <int DT>
hipError_t launch_z(const Args &a, int z, bool vec, hipStream_t st) {
  return z == kGate       ? launch<DT, kGate>(a, vec, st)
         : z == kResidual ? launch<DT, kResidual>(a, vec, st)
                          : launch<DT, kPlain>(a, vec, st);
}

}  // namespace dropout

hipError_t launch_dropout(const fg_dropout_desc &d, const void *x, const void *z, bool gate,
                          void *y, const int32_t *step_count, hipStream_t st) {
  using namespace dropout;
  Args a{};
  a.x = x, a.z = z, a.y = y, a.step_count = step_count;
  a.xl = d.x_ld ? d.x_ld : d.cols;
  a.yl = d.y_ld ? d.y_ld : d.cols;
  a.zl = d.z_ld ? d.z_ld : d.cols;
  a.n = (uint64_t)d.rows * (uint64_t)d.cols;
  a.k0 = (uint32_t)d.seed, a.k1 = (uint32_t)(d.seed >> 32);
  a.step = d.step, a.site = d.site;
  a.threshold = dropout_threshold(d.p);
  a.scale = a.threshold ? 65536.f / (float)a.threshold : 0.f;
  const int esz = d.dtype == FG_F32 ? 4 : 2, unit = 16 / esz;
  const bool dense = d.rows == 1 || (a.xl == d.cols && a.yl == d.cols && (!z || a.zl == d.cols));
  const bool aligned = (((uintptr_t)x | (uintptr_t)y | (uintptr_t)z) & 15) == 0;
  const bool rows8 = d.cols % 8 == 0 && a.xl % unit == 0 && a.yl % unit == 0 &&
                     (!z || a.zl % unit == 0);
  const bool vec = aligned && (dense || rows8);
  a.cols = vec && dense ? 0 : (uint32_t)d.cols;
  a.div = dma::make_fastdiv(!a.cols ? 1 : vec ? a.cols / 8 : a.cols);
  const int zk = !z ? kPlain : gate ? kGate : kResidual;
  return d.dtype == FG_F32    ? launch_z<FG_F32>(a, zk, vec, st)
         : d.dtype == FG_BF16 ? launch_z<FG_BF16>(a, zk, vec, st)
                              : launch_z<FG_F16>(a, zk, vec, st);
}

}  // namespace fg
