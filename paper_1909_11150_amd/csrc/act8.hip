// Activations kept in 8 bits from the forward to the backward pass (format: rows.h).
//
// Bound by memory: an fp16 element is read in 2 bytes and written in 33/32, and back. A lane
// takes 8 columns, so that its access is 16 bytes of a 16-bit type, and 4 lanes beside each
// other a group: its largest magnitude goes around in two moves between lanes, no LDS. 65536 x
// 256 fp16 of rows of 1024: packed in 11.0 us, unpacked in 10.3 (50.9 MB each way, 4.6 and 4.9
// TB/s; called one after the other without a profiler 20.5 us for both, 5.0 TB/s); 8191 x 1023
// bf16, whose rows begin at odd words, 7.0 and 6.6 us (3.6 and 3.9 TB/s).
#include "act8.h"

namespace fg {
namespace act8 {

template <int DT>
__global__ __launch_bounds__(kThreads) void act8_pack_kernel(Args a) {
  using T = typename TypeOf<DT>::T;
  const uint64_t i = (uint64_t)blockIdx.x * kThreads + threadIdx.x;
  if (i >= a.n) return;  // (a.n is a multiple of 4: groups stay whole)
  const uint32_t row = a.div.div((uint32_t)i);
  const int c = 8 * (int)((uint32_t)i - row * (uint32_t)(a.p.wide / 8));
  float v[8];
  load8(static_cast<const T *>(a.x) + row * a.ld, c, a.cols, v);
  pack8(a.p, row, c, v);
}

template <int DT>
__global__ __launch_bounds__(kThreads) void act8_unpack_kernel(Args a) {
  unpack_block<DT>(a, blockIdx.x);
}

template <int DT>
hipError_t launch(const Args &a, bool pack, hipStream_t st) {
  const dim3 grid(blocks_of(a)), block(kThreads);
  if (pack)
    hipLaunchKernelGGL(act8_pack_kernel<DT>, grid, block, 0, st, a);
  else
    hipLaunchKernelGGL(act8_unpack_kernel<DT>, grid, block, 0, st, a);
  return hipGetLastError();
}

}  // namespace act8

size_t act8_size(int64_t rows, int64_t cols) {
  const int64_t wide = rows::packed_cols(cols);
  return (size_t)(rows * wide + rows * (wide / 32));
}

hipError_t launch_act8(const fg_act8_desc &d, const void *x, void *y, void *packed,
                       hipStream_t st) {
  const act8::Args a = act8::args_of(d, x, y, packed);
  const bool pack = x != nullptr;
  return d.dtype == FG_F16    ? act8::launch<FG_F16>(a, pack, st)
         : d.dtype == FG_BF16 ? act8::launch<FG_BF16>(a, pack, st)
                              : act8::launch<FG_F32>(a, pack, st);
}

}  // namespace fg
