// Codes of an 8-bit checkpoint back into rows: a launch of its own (act8.hip), or workgroups of
// another's.
#pragma once
#include "rows.h"

namespace fg {
namespace act8 {

using namespace rows;

constexpr int kThreads = 256;

struct Args {
  const void *x;
  void *y;
  int64_t ld;
  Packed p;
  uint32_t n;         // chunks of 8 columns
  int32_t cols;
  dma::FastDiv div;   // by a row's chunks
};

inline Args args_of(const fg_act8_desc &d, const void *x, void *y, void *packed) {
  Args a{};
  a.x = x, a.y = y;
  a.ld = d.x_ld ? d.x_ld : d.cols;
  a.p = packed_at(packed, d.rows, d.cols);
  a.n = (uint32_t)(d.rows * (a.p.wide / 8));
  a.cols = (int32_t)d.cols;
  a.div = dma::make_fastdiv((uint32_t)(a.p.wide / 8));
  return a;
}
inline uint32_t blocks_of(const Args &a) {
  return (uint32_t)((a.n + (uint64_t)kThreads - 1) / kThreads);
}

template <int DT>
__device__ __forceinline__ void unpack_block(const Args &a, uint32_t block) {
  using T = typename TypeOf<DT>::T;
  const uint64_t i = (uint64_t)block * kThreads + threadIdx.x;
  if (i >= a.n) return;
  const uint32_t row = a.div.div((uint32_t)i);
  const int c = 8 * (int)((uint32_t)i - row * (uint32_t)(a.p.wide / 8));
  if (c >= a.cols) return;
  float v[8];
  decode8(*reinterpret_cast<const u32x2 *>(a.p.codes + (int64_t)row * a.p.wide + c),
          a.p.exps[(int64_t)row * (a.p.wide / 32) + c / 32], v);
  store8(static_cast<T *>(a.y) + row * a.ld, c, a.cols, v);
}

}  // namespace act8
}  // namespace fg
