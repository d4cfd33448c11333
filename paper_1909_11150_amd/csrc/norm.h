// Layer norm's teams (norm.hip: forward, norm_grad.hip: gradients).
#pragma once
#include "rows.h"

namespace fg {
namespace norm {

using namespace rows;

// TL lanes of a wave (W = 1), or W waves, take a row of up to 8 * TEAM * N columns.
template <int TL_, int W_, int N_, int NT_ = 64 * W_ < 256 ? 256 : 64 * W_>
struct Team {
  static constexpr int TL = TL_, W = W_, N = N_, NT = NT_;
  static constexpr int TEAM = TL * W, TEAMS = NT / TEAM, WIDE = 8 * TEAM * N;
  static constexpr int MORE_THAN = TL == 8 ? 0 : WIDE / 2;  // columns of its rows
  static __device__ __forceinline__ int col(int t, int n) { return 8 * (t + TEAM * n); }
};

// The team's sums of R values, in every lane. red: LDS of R * NT / 64 floats (W > 1) that no
// other exchange uses before the next barrier.
template <class M, int R>
__device__ __forceinline__ void team_sums(float (&v)[R], float *red) {
#pragma unroll
  for (int k = 0; k < R; ++k) v[k] = sum_lanes<M::TL>(v[k]);
  if constexpr (M::W > 1) {
    const int wave = threadIdx.x >> 6;
    if ((threadIdx.x & 63) == 0) {
#pragma unroll
      for (int k = 0; k < R; ++k) red[wave * R + k] = v[k];
    }
    __syncthreads();
#pragma unroll
    for (int k = 0; k < R; ++k) v[k] = 0.f;
#pragma unroll
    for (int i = 0; i < M::W; ++i)
#pragma unroll
      for (int k = 0; k < R; ++k) v[k] += red[(wave / M::W * M::W + i) * R + k];
  }
}
struct FwdArgs {
  const void *x, *weight, *bias;
  void *y;
  float2 *stats;
  Packed packed;
  int64_t rows, x_ld, y_ld;
  int32_t cols;
  float inv, eps;    // 1 / cols
};

// Workgroups of the forward pass: 4 waves a SIMD where they are of 4 waves, which the chip holds
// at once, each taking several rows with the next one's loads on their way. With 512, 1024, 1280,
// 2048 of them: 16384 x 1024 fp16 14.5, 13.8, 14.5, 13.9 us; 65536 x 512 fp16 with the checkpoint
// 45, 35.8, 34.0, 34.2; 2000 x 12001 fp32 39, 45, 47, 52.
constexpr int kFwdBlocks = 1024;

// f.go<type, TL, W, N>() for the team that takes a row. Backward, where 16 sums a chunk stay in
// registers, wide rows take more waves with a chunk to a lane each (16384 x 1024 fp16 27.5 us,
// 31.1 with two; both passes of 3000 x 5000 fp16 from the checkpoint 58, 65 with two); forward,
// two chunks and half the exchanges (8192 x 4096 bf16 25.0 us, 29.6 with one).
enum Pass { kForward, kGrad };
template <int DT, Pass P, class F>
hipError_t for_cols(int cols, const F &f) {
  constexpr int W = P == kForward ? 1 : 2, N = P == kForward ? 2 : 1;
  return cols <= 64     ? f.template go<DT, 8, 1, 1>()
         : cols <= 128  ? f.template go<DT, 16, 1, 1>()
         : cols <= 256  ? f.template go<DT, 32, 1, 1>()
         : cols <= 512  ? f.template go<DT, 64, 1, 1>()
         : cols <= 1024 ? f.template go<DT, 64, W, N>()
         : cols <= 2048 ? f.template go<DT, 64, 2 * W, N>()
         : cols <= 4096 ? f.template go<DT, 64, 4 * W, N>()
         : cols <= 8192 ? f.template go<DT, 64, 8 * W, N>()
                        : f.template go<DT, 64, 16, 2>();
}
template <Pass P, class F>
hipError_t for_team(int dtype, int cols, const F &f) {
  return dtype == FG_F16    ? for_cols<FG_F16, P>(cols, f)
         : dtype == FG_BF16 ? for_cols<FG_BF16, P>(cols, f)
                            : for_cols<FG_F32, P>(cols, f);
}

}  // namespace norm
}  // namespace fg
