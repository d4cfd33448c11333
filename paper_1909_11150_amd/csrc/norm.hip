// Layer norm of rows, and its gradients.
//
//   y = (x - mean) rstd w + b,  rstd = (mean((x - mean)^2) + eps)^(-1/2)
//   g = dy w,  xh = (x - mean) rstd
//   dx = add + rstd (g - mean(g) - xh mean(g xh)),  dw = sum dy xh,  db = sum dy
//
// Bound by memory. A team of lanes takes a row whole into registers, 8 columns a lane and
// chunk: 8 to 64 lanes of a wave, then 2 to 16 waves. So a row is read once, its mean and the
// squares about it are summed from registers, and the next row's loads are on their way
// meanwhile. A row may lie far from zero, and a sum of C alike terms rounds each time: a mean so
// found is off by some parts in 2^24 of itself, which may be more than the row's spread. So
// the mean is x0 + mean(x - x0), x0 the row's first element, and the squares' pass sums d =
// x - mean too, whose mean is what the first one missed:
//   more = mean(d),  var = mean(d^2) - more^2,  y = (d - more) rstd w + b.
// With x0, more is small against the spread whatever the row, and var no difference of large
// numbers (a constant row is exact). One more sum in an exchange that is there. (16384 x 1024
// fp16 12.8 -> 13.8 us, 20000 x 777 bf16 14.6 -> 16.0, 4096 x 8192 fp32 45.1 -> 46.5; with
// kernels for rows that 8 divides 65536 x 256 fp16 16.3 -> 15.8.) The gradients of weight and bias are summed down
// the rows in registers, a team's columns being always the same, then over a workgroup's
// teams in LDS; the workgroups' sums go to the workspace and a second kernel adds them in
// order. Everything is summed in fp32 and in a fixed order.
//
// Measured, forward: 8192 x 4096 bf16 24.8 us (5.4 TB/s, part of it from the Infinity Cache; 27
// from memory), 65536 x 512 fp16 with the checkpoint of x 35.7 (4.7 TB/s); a single row 2.8.
#include <algorithm>

#include "norm.h"

namespace fg {
namespace norm {

// EVEN: 8 divides the columns, no masks within a chunk.
template <int DT, int TL, int W, int N, bool EVEN>
__global__ __launch_bounds__((Team<TL, W, N>::NT)) void norm_fwd_kernel(FwdArgs a) {
  using T = typename TypeOf<DT>::T;
  using M = Team<TL, W, N>;
  __shared__ float red[W > 1 ? 3 * M::NT / 64 : 1];
  const int t = threadIdx.x % M::TEAM, team = threadIdx.x / M::TEAM;
  const int cols = EVEN ? a.cols / 8 * 8 : a.cols;  // (the compiler knows its low bits)
  __builtin_assume(cols > (EVEN && M::MORE_THAN < 7 ? 7 : M::MORE_THAN));
  const T *x = static_cast<const T *>(a.x), *w = static_cast<const T *>(a.weight),
          *b = static_cast<const T *>(a.bias);
  T *y = static_cast<T *>(a.y);
  Raw<T> rw[N], rb[N], next[N];
  T first;   // of the next row
#pragma unroll
  for (int n = 0; n < N; ++n) {
    const int c = M::col(t, n);
    if (w) rw[n] = load_any(w, c, cols);
    if (b) rb[n] = load_any(b, c, cols);
  }
  const int64_t step = (int64_t)gridDim.x * M::TEAMS;
  int64_t r0 = (int64_t)blockIdx.x * M::TEAMS;
  auto load = [&](int64_t r) __attribute__((always_inline)) {
    const T *row = x + min(r, a.rows - 1) * a.x_ld;
#pragma unroll
    for (int n = 0; n < N; ++n) next[n] = load_any(row, M::col(t, n), cols);
    first = row[0];
  };
  // v, element e of chunk n, less `by`; past the row's end 0 as v is
  auto less = [&](float v, float by, int n, int e) __attribute__((always_inline)) {
    const int c = M::col(t, n);
    return v - ((EVEN ? c : c + e) < cols ? by : 0.f);
  };
  load(r0 + team);
  for (; r0 < a.rows; r0 += step) {
    const int64_t r = r0 + team;
    const bool on = r < a.rows;
    const float x0 = (float)first;
    float v[N][8], s = 0.f;
#pragma unroll
    for (int n = 0; n < N; ++n) {
      values<T>(next[n], M::col(t, n), cols, v[n]);
#pragma unroll
      for (int e = 0; e < 8; ++e) s += less(v[n][e], x0, n, e);
    }
    if (r0 + step < a.rows) load(r + step);
    if (a.packed.codes && on) {
#pragma unroll
      for (int n = 0; n < N; ++n) pack8(a.packed, r, M::col(t, n), v[n]);
    }
    float s1[1] = {s}, s2[2] = {0.f, 0.f};
    team_sums<M, 1>(s1, red);
    const float m0 = fmaf(s1[0], a.inv, x0);
#pragma unroll
    for (int n = 0; n < N; ++n)
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const float d = v[n][e] = less(v[n][e], m0, n, e);
        s2[0] += d;
        s2[1] = fmaf(d, d, s2[1]);
      }
    team_sums<M, 2>(s2, red + M::NT / 64);
    const float more = s2[0] * a.inv, var = fmaf(-more, more, s2[1] * a.inv);
    const float rstd = 1.f / sqrtf((var < 0.f ? 0.f : var) + a.eps);  // (NaN stays)
    if (!on) continue;
    if (a.stats && t == 0) a.stats[r] = float2{m0 + more, rstd};
#pragma unroll
    for (int n = 0; n < N; ++n) {
      const int c = M::col(t, n);
      float g[8], h[8];
      if (w) values<T>(rw[n], c, cols, g);
      if (b) values<T>(rb[n], c, cols, h);
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        float o = fmaf(v[n][e], rstd, -more * rstd);
        if (w) o *= g[e];
        v[n][e] = b ? o + h[e] : o;
      }
      store8(y + r * a.y_ld, c, cols, v[n]);
    }
  }
}

struct Fwd {
  const FwdArgs &a;
  hipStream_t st;
  template <int DT, int TL, int W, int N>
  hipError_t go() const {
    using M = Team<TL, W, N>;
    const int64_t blocks = std::min<int64_t>((a.rows + M::TEAMS - 1) / M::TEAMS, kFwdBlocks);
    const dim3 grid((uint32_t)blocks), block(M::NT);
    if (a.cols % 8 == 0)
      hipLaunchKernelGGL((norm_fwd_kernel<DT, TL, W, N, true>), grid, block, 0, st, a);
    else
      hipLaunchKernelGGL((norm_fwd_kernel<DT, TL, W, N, false>), grid, block, 0, st, a);
    return hipGetLastError();
  }
};

}  // namespace norm

hipError_t launch_layer_norm_fwd(const fg_norm_desc &d, const void *x, const void *weight,
                                 const void *bias, void *y, float *stats, void *packed,
                                 hipStream_t st) {
  norm::FwdArgs a{};
  a.x = x, a.weight = weight, a.bias = bias, a.y = y;
  a.stats = reinterpret_cast<float2 *>(stats);
  if (packed) a.packed = rows::packed_at(packed, d.rows, d.cols);
  a.rows = d.rows, a.cols = (int32_t)d.cols;
  a.x_ld = d.x_ld ? d.x_ld : d.cols, a.y_ld = d.y_ld ? d.y_ld : d.cols;
  a.inv = (float)(1.0 / (double)d.cols), a.eps = (float)d.eps;
  return norm::for_team<norm::kForward>(d.dtype, a.cols, norm::Fwd{a, st});
}

}  // namespace fg
