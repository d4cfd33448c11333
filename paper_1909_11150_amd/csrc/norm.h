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
  static __device__ __forceinline__ int col(int t, int n) { return 8 * (t + TEAM * n); }
};

// The team's sum, in every lane. red: LDS of NT / 64 floats for each of the alternating
// places (W > 1), so that one barrier per sum is enough.
template <class M>
__device__ __forceinline__ float team_sum(float v, float *red, int place) {
#pragma unroll
  for (int o = M::TL / 2; o; o >>= 1) v += __shfl_xor(v, o);
  if constexpr (M::W > 1) {
    float *at = red + place * (M::NT / 64);
    const int wave = threadIdx.x >> 6;
    if ((threadIdx.x & 63) == 0) at[wave] = v;
    __syncthreads();
    v = 0.f;
#pragma unroll
    for (int k = 0; k < M::W; ++k) v += at[wave / M::W * M::W + k];
  }
  return v;
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

constexpr int kFwdBlocks = 2048;
constexpr int kMaxCols = 16384;

// f.go<type, TL, W, N>() for the smallest team that holds a row.
template <int DT, class F>
hipError_t for_cols(int cols, const F &f) {
  return cols <= 64     ? f.template go<DT, 8, 1, 1>()
         : cols <= 128  ? f.template go<DT, 16, 1, 1>()
         : cols <= 256  ? f.template go<DT, 32, 1, 1>()
         : cols <= 512  ? f.template go<DT, 64, 1, 1>()
         : cols <= 1024 ? f.template go<DT, 64, 1, 2>()
         : cols <= 2048 ? f.template go<DT, 64, 2, 2>()
         : cols <= 4096 ? f.template go<DT, 64, 4, 2>()
         : cols <= 8192 ? f.template go<DT, 64, 8, 2>()
                        : f.template go<DT, 64, 8, 4>();
}
template <class F>
hipError_t for_team(int dtype, int cols, const F &f) {
  return dtype == FG_F16    ? for_cols<FG_F16>(cols, f)
         : dtype == FG_BF16 ? for_cols<FG_BF16>(cols, f)
                            : for_cols<FG_F32>(cols, f);
}

}  // namespace norm
}  // namespace fg
