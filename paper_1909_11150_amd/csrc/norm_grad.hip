// Layer norm's gradients (formulas and layout: norm.hip).
#include <algorithm>

#include "norm.h"

namespace fg {
namespace norm {

struct BwdArgs {
  const void *dy, *x, *weight, *add;
  void *dx;
  const float2 *stats;
  Packed packed;       // PACKED: x's place
  float *part;         // [workgroup][2][wide] sums of dy xh and of dy; null: not wanted
  int64_t rows, dy_ld, x_ld, add_ld, dx_ld;
  int32_t cols;
  float inv;
};

// 8 waves a workgroup, or a row's 16.
template <int TL, int W, int N>
using Grad = Team<TL, W, N, W <= 8 ? 512 : 64 * W>;

// What a row's gradient needs, on its way.
template <class T, int N, bool PACKED>
struct Loads {
  Raw<T> dy[N], add[N];
  Raw<T> x[PACKED ? 1 : N];
  u32x2 code[PACKED ? N : 1];
  uint32_t exp[PACKED ? N : 1];
  float2 stat;
};

// Bound by memory: 65536 x 512 fp16 from the checkpoint 36.1 us (4.7 TB/s), 8192 x 4096 bf16
// with another gradient to add 44.5 (6.0 TB/s, part of it from the Infinity Cache), then 5 us
// for the join of the workgroups' sums. Eight waves a workgroup: half as many parts to join as
// with four. Bounds: with a chunk to a lane, the registers of two workgroups on a CU (4 waves a
// SIMD), which all types need so that one's loads cover the other's exchanges.
template <int DT, int TL, int W, int N, bool PACKED>
__global__ __launch_bounds__((Grad<TL, W, N>::NT),
                             N == 1 ? 4 : 2) void norm_bwd_kernel(BwdArgs a) {
  using T = typename TypeOf<DT>::T;
  using M = Grad<TL, W, N>;
  constexpr int FOLD = M::TEAMS / 2;  // teams whose sums wait in LDS at a time
  constexpr int LDS = FOLD * M::TEAM * N * 16;
  constexpr int EX = 4 * (M::NT / 64);  // the sums' exchange, two of them in turn
  // 16 waves with two chunks a lane each have no registers for the next row's loads, nor for the
  // weights in fp32: with both, 250 of them spilled (both passes of 2048 x 16384 bf16 398 us,
  // 112 without).
  constexpr bool kAhead = W < 16 || N == 1;
  __shared__ __attribute__((aligned(16))) float lds[LDS > EX ? LDS : EX];
  const int t = threadIdx.x % M::TEAM, team = threadIdx.x / M::TEAM, cols = a.cols;
  __builtin_assume(cols > M::MORE_THAN);
  const T *dy = static_cast<const T *>(a.dy), *x = static_cast<const T *>(a.x),
          *w = static_cast<const T *>(a.weight), *add = static_cast<const T *>(a.add);
  T *dx = static_cast<T *>(a.dx);
  Raw<T> rw[N];
  float aw[N][8] = {}, ab[N][8] = {};
#pragma unroll
  for (int n = 0; n < N; ++n)
    if (w) rw[n] = load_any(w, M::col(t, n), cols);
  Loads<T, N, PACKED> next;
  auto load = [&](int64_t r) __attribute__((always_inline)) {
    r = min(r, a.rows - 1);
    next.stat = a.stats[r];
#pragma unroll
    for (int n = 0; n < N; ++n) {
      const int c = M::col(t, n);
      next.dy[n] = load_any(dy + r * a.dy_ld, c, cols);
      if constexpr (PACKED) {
        const int q = min(c, a.packed.wide - 8);
        next.code[n] = *reinterpret_cast<const u32x2 *>(a.packed.codes + r * a.packed.wide + q);
        next.exp[n] = a.packed.exps[r * (a.packed.wide / 32) + q / 32];
      } else {
        next.x[n] = load_any(x + r * a.x_ld, c, cols);
      }
      if (add) next.add[n] = load_any(add + r * a.add_ld, c, cols);
    }
  };
  const int64_t step = (int64_t)gridDim.x * M::TEAMS;
  int64_t r0 = (int64_t)blockIdx.x * M::TEAMS;
  if (kAhead) load(r0 + team);
  int turn = 0;
  for (; r0 < a.rows; r0 += step, turn ^= 1) {
    const int64_t r = r0 + team;
    const bool on = r < a.rows, ragged = r0 + M::TEAMS > a.rows;  // (the latter for all alike)
    if (!kAhead) {
      load(r);
      // the weights stay as they are in memory, not taken out of the loop in fp32
#pragma unroll
      for (int n = 0; n < N; ++n)
#pragma unroll
        for (u32x4 &q : rw[n].w) asm volatile("" : "+v"(q));
    }
    const Loads<T, N, PACKED> now = next;
    if (kAhead && r0 + step < a.rows) load(r + step);
    float g[N][8], xh[N][8], s[2] = {0.f, 0.f};
#pragma unroll
    for (int n = 0; n < N; ++n) {
      const int c = M::col(t, n);
      values<T>(now.dy[n], c, cols, g[n]);  // zeros past the row's end: no masks below
      if constexpr (PACKED)
        decode8(now.code[n], now.exp[n], xh[n]);
      else
        values<T>(now.x[n], c, cols, xh[n]);
      float wv[8];
      if (w) values<T>(rw[n], c, cols, wv);
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        float &gv = g[n][e], &xv = xh[n][e];
        xv = (xv - now.stat.x) * now.stat.y;
        if (ragged && !on) gv = xv = 0.f;
        aw[n][e] = fmaf(gv, xv, aw[n][e]);
        ab[n][e] += gv;
        if (w) gv *= wv[e];
        s[0] += gv;
        s[1] = fmaf(gv, xv, s[1]);
      }
    }
    if (!dx) continue;  // (the same for all)
    team_sums<M, 2>(s, lds + 2 * (M::NT / 64) * turn);
    if (!on) continue;
    const float s1 = s[0] * a.inv, s2 = s[1] * a.inv;
#pragma unroll
    for (int n = 0; n < N; ++n) {
      const int c = M::col(t, n);
      float o[8];
      if (add) values<T>(now.add[n], c, cols, o);
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const float d = (g[n][e] - s1 - xh[n][e] * s2) * now.stat.y;
        o[e] = add ? o[e] + d : d;
      }
      store8(dx + r * a.dx_ld, c, cols, o);
    }
  }
  if (!a.part) return;
  // the workgroup's teams, halves onto halves
  for (int half = M::TEAMS / 2; half; half >>= 1) {
    __syncthreads();
    f32x4 *at = reinterpret_cast<f32x4 *>(lds);
    if (team >= half && team < 2 * half) {
#pragma unroll
      for (int n = 0; n < N; ++n)
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          const float *v = k < 2 ? aw[n] + 4 * k : ab[n] + 4 * (k - 2);
          at[((team - half) * N * 4 + 4 * n + k) * M::TEAM + t] = f32x4{v[0], v[1], v[2], v[3]};
        }
    }
    __syncthreads();
    if (team < half) {
#pragma unroll
      for (int n = 0; n < N; ++n)
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          float *v = k < 2 ? aw[n] + 4 * k : ab[n] + 4 * (k - 2);
          const f32x4 q = at[(team * N * 4 + 4 * n + k) * M::TEAM + t];
#pragma unroll
          for (int e = 0; e < 4; ++e) v[e] += q[e];
        }
    }
  }
  if (team) return;
  float *out = a.part + (size_t)blockIdx.x * 2 * M::WIDE;
#pragma unroll
  for (int n = 0; n < N; ++n)
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const float *v = k < 2 ? aw[n] + 4 * k : ab[n] + 4 * (k - 2);
      *reinterpret_cast<f32x4 *>(out + (k / 2) * M::WIDE + M::col(t, n) + 4 * (k & 1)) =
          f32x4{v[0], v[1], v[2], v[3]};
    }
}

// Sums the workgroups' parts, in order: 16 columns of one of the two gradients a workgroup.
struct JoinArgs {
  const float *part;
  void *dweight, *dbias;   // either may be null
  int32_t n, wide, cols;
  int32_t *flag;
};
template <int DT>
__global__ __launch_bounds__(256) void norm_join_kernel(JoinArgs a) {
  using T = typename TypeOf<DT>::T;
  T *out = static_cast<T *>(blockIdx.y ? a.dbias : a.dweight);
  if (!out) return;
  const int c = 16 * (int)blockIdx.x + (threadIdx.x & 15);
  __shared__ __attribute__((aligned(16))) uint8_t lds[kSumLds];
  float s;
  sum_columns(a.part + (int64_t)blockIdx.y * a.wide, a.n, 2 * (int64_t)a.wide,
              16 * (int)blockIdx.x, a.wide, lds, s);
  bool bad = false;
  if (threadIdx.x < 16 && c < a.cols) {
    const T v = (T)s;
    out[c] = v;
    bad = !(fabsf((float)v) < INFINITY);
  }
  if (a.flag) flag_nonfinite(a.flag, bad);
}

struct Plan {
  int64_t blocks, wide;
};
struct MakePlan {
  int64_t rows;
  Plan *p;
  template <int DT, int TL, int W, int N>
  hipError_t go() const {
    using M = Grad<TL, W, N>;
    p->wide = M::WIDE;
    // Two a CU, one of wide rows: the fewest parts to join that keep the memory busy (both passes
    // of 65536 x 512 fp16 with 256, 512, 1024 workgroups: 94, 89, 91 us; of 4099 x 1003 fp32 27.5,
    // 28.5, 33; of 8192 x 4096 bf16 with 128, 256: 99, 80).
    p->blocks = std::min<int64_t>((rows + M::TEAMS - 1) / M::TEAMS, M::WIDE <= 1024 ? 512 : 256);
    return hipSuccess;
  }
};
Plan make_plan(int64_t rows, int64_t cols) {
  Plan p{};
  (void)for_cols<FG_F16, kGrad>((int)cols, MakePlan{rows, &p});
  return p;
}

struct Bwd {
  const BwdArgs &a;
  int64_t blocks;
  hipStream_t st;
  template <int DT, int TL, int W, int N, bool PACKED>
  hipError_t launch() const {
    hipLaunchKernelGGL((norm_bwd_kernel<DT, TL, W, N, PACKED>), dim3((uint32_t)blocks),
                       dim3(Grad<TL, W, N>::NT), 0, st, a);
    return hipGetLastError();
  }
  template <int DT, int TL, int W, int N>
  hipError_t go() const {
    // (8192 x 4096 bf16: from x 50 us by 8 waves to a row, 45 by 4; packed 49.6 and 51.5)
    if constexpr (W == 8 && N == 1)
      if (!a.packed.codes) return launch<DT, TL, 4, 2, false>();
    return a.packed.codes ? launch<DT, TL, W, N, true>() : launch<DT, TL, W, N, false>();
  }
};

}  // namespace norm

size_t layer_norm_ws_bytes(const fg_norm_desc &d) {
  const norm::Plan p = norm::make_plan(d.rows, d.cols);
  return (size_t)p.blocks * 2 * p.wide * 4;
}

hipError_t launch_layer_norm_bwd(const fg_norm_desc &d, const void *dy, const void *x,
                                 const void *packed, const float *stats, const void *weight,
                                 const void *add, void *dx, void *dweight, void *dbias,
                                 int32_t *flag, void *ws, hipStream_t st) {
  const norm::Plan p = norm::make_plan(d.rows, d.cols);
  const bool sums = dweight || dbias;
  const auto ld = [&](int64_t v) { return v ? v : d.cols; };
  norm::BwdArgs a{};
  a.dy = dy, a.x = x, a.weight = weight, a.add = add, a.dx = dx;
  a.stats = reinterpret_cast<const float2 *>(stats);
  if (packed) a.packed = rows::packed_at(packed, d.rows, d.cols);
  a.part = sums ? static_cast<float *>(ws) : nullptr;
  a.rows = d.rows;
  a.dy_ld = ld(d.y_ld), a.x_ld = ld(d.x_ld), a.add_ld = ld(d.add_ld), a.dx_ld = ld(d.dx_ld);
  a.cols = (int32_t)d.cols;
  a.inv = (float)(1.0 / (double)d.cols);
  if (d.rows) {
    const hipError_t e = norm::for_team<norm::kGrad>(d.dtype, a.cols, norm::Bwd{a, p.blocks, st});
    if (e != hipSuccess) return e;
  }
  if (!sums) return hipSuccess;
  const norm::JoinArgs j = {a.part, dweight, dbias, (int32_t)(d.rows ? p.blocks : 0),
                            (int32_t)p.wide, a.cols, flag};
  const dim3 grid((uint32_t)((d.cols + 15) / 16), 2), block(256);
  if (d.dtype == FG_F16)
    hipLaunchKernelGGL(norm::norm_join_kernel<FG_F16>, grid, block, 0, st, j);
  else if (d.dtype == FG_BF16)
    hipLaunchKernelGGL(norm::norm_join_kernel<FG_BF16>, grid, block, 0, st, j);
  else
    hipLaunchKernelGGL(norm::norm_join_kernel<FG_F32>, grid, block, 0, st, j);
  return hipGetLastError();
}

}  // namespace fg
