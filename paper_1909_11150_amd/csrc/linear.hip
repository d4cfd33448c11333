// Linear layers with bias, activation and residual in the product's epilogue, and their
// gradients.
//
//   z = x w^T + b,  y = residual + act(z)
//   dz = dy act'(z),  dx = dz w,  dw = dz^T x,  db = sum of dz over the rows
//
// Bound by the matrix pipes where all three sizes are long (the forward pass by itself 464 us of
// 16384 x 2048 -> 8192 bf16, 1.18 PFLOP/s; with bias, gelu and checkpoint 540, and 577 to 593 in a
// step, whose products leave the clock lower), by memory where the sum is short (65536 x 256 ->
// 1024: 59 us, 98 with them) or the rows are few.
//
// Products run on the MFMA tiles that dma_pipe.h feeds by LDS DMA. The forward tile holds
// outputs x rows, so 32 consecutive outputs of a row lie in two lanes' registers: bias,
// activation and the 8-bit checkpoint of z (a step for each 32 columns) are made there, and
// one rounding writes y. Its operands' rows both lie along the sum. Backward, dz is formed
// once (16 bits, the matrix pipes' type) while its columns are summed for db; dx and dw are
// one launch, whose operands by rows of the sum are read with transposing LDS reads. Long
// sums with few tiles are split and joined in order; the join does the epilogue then.
#include <string.h>

#include <algorithm>

#include "act8.h"
#include "tiles.h"

namespace fg {
namespace linear {

using namespace tiles;
using rows::Packed;
using rows::TypeOf;

// 128 x 128 in a ring of four, for launches of a workgroup per CU or less: with two, each
// stage waits for its loads (dx of 4096 x 1024 -> 4096 43.1 -> 35.8 us).
using P128D = Pipe<64, 4, 2, 2, 128, 128>;
// For short sums, where the beginning and end are most of the work: three workgroups of 128 x
// 128 a CU, or two of 256 outputs x 128 rows with 16 waves between them, one in its epilogue
// while another loads.
using S128 = Pipe<32, 3, 2, 2, 128, 128>;
using S256 = Pipe<32, 3, 4, 2, 256, 128>;
struct FwdTiles {
  using T256 = Pipe<64, 2, 2, 4, 256, 256>;
};
struct BwdTiles {
  using T256 = Pipe<32, 5, 2, 4, 256, 256>;
};

// ---- activations ---------------------------------------------------------------------
// Phi(-|z|), Phi the normal distribution's function, as 2^P(|z|): the logarithm is smooth, so a
// polynomial of degree 7 fitted here keeps 5.7e-6 of the value (fp32 steps included; a result's
// rounding to fp16 is 4.9e-4) up to |z| = 6, and falls on beyond, where Phi(-|z|) < 1e-9. No
// reciprocal, and the digits of far negative z stay: 14 instructions for gelu, of which the
// exponential takes four turns.
__device__ __forceinline__ float phi_below(float z) {
  const float a = fabsf(z);
  float r = fmaf(a, -1.83478636e-6f, 6.15977578e-5f);
  r = fmaf(r, a, -9.30520317e-4f);
  r = fmaf(r, a, 8.50787166e-3f);
  r = fmaf(r, a, -5.39600260e-2f);
  r = fmaf(r, a, -0.458464442f);
  r = fmaf(r, a, -1.15125102f);
  r = fmaf(r, a, -0.999995298f);
  return __builtin_amdgcn_exp2f(r);
}
// z Phi(z) = max(z, 0) - |z| Phi(-|z|). Infinities give 0 and themselves, NaN NaN.
__device__ __forceinline__ float gelu(float z) {
  // (medians: fminf and fmaxf would first quiet their NaN, two instructions more)
  return fmaf(-__builtin_amdgcn_fmed3f(fabsf(z), 0.f, 64.f), phi_below(z),
              __builtin_amdgcn_fmed3f(z, 0.f, INFINITY));
}
// Phi(z) + z exp(-z^2 / 2) / sqrt(2 pi). For negative z Phi is phi_below itself: as 1 less its
// complement, what is left of it at z = -5 would be off by 3e-3 (0.5 + copysign(0.5 - p, z) is).
__device__ __forceinline__ float gelu_slope(float z) {
  const float bell = __builtin_amdgcn_exp2f(z * z * -0.72134752f);
  const float p = phi_below(z), phi = z < 0.f ? p : 1.f - p;
  return fmaf(__builtin_amdgcn_fmed3f(z, -64.f, 64.f) * 0.39894228f, bell, phi);
}
__device__ __forceinline__ float apply(float z, int act) {
  return act == FG_ACT_RELU ? (z < 0.f ? 0.f : z) : act == FG_ACT_GELU ? gelu(z) : z;
}

__device__ __forceinline__ float to_f32(uint32_t half, bool bf) {
  return bf ? __builtin_bit_cast(float, half << 16) : h_to_f32((uint16_t)half);
}

// ---- forward -------------------------------------------------------------------------
struct Epilogue {
  const uint16_t *bias, *residual;
  uint16_t *y, *z;
  int64_t y_ld, r_ld, z_ld;
  Packed packed;
  int32_t out, act;
};
struct FwdArgs {
  const uint16_t *w, *x;
  int64_t w_ld, x_ld;
  int32_t K, kper;        // the sum's length (at least 8); of a part (a multiple of 64)
  int64_t rows;
  int32_t ntile;          // tiles of outputs
  Epilogue e;
  float *part;            // [parts][rows][Mq] or null
  int64_t pstride;
  int32_t Mq;
};

// Keeps the compiler from working on more of the accumulators at once than it has registers
// for: without it the 256 x 128 tile spills 8 of them (at the same times: 65536 x 256 -> 1024 59
// us either way).
__device__ __forceinline__ void apart() { __builtin_amdgcn_sched_barrier(0); }

// A block's activation, into registers of its own: changed in place under a branch, the whole
// tile's accumulators would be copied, and some spilled.
__device__ __forceinline__ void activate(float (&v)[16], const f32x16 &z, int act) {
  if (act == FG_ACT_GELU) {
#pragma unroll
    for (int e = 0; e < 16; ++e) v[e] = gelu(z[e]);
  } else if (act == FG_ACT_RELU) {
#pragma unroll
    for (int e = 0; e < 16; ++e) v[e] = z[e] < 0.f ? 0.f : z[e];
  } else {
#pragma unroll
    for (int e = 0; e < 16; ++e) v[e] = z[e];
  }
}

// Rows n0 .. of a matrix of nrow rows as a buffer: what lies past the last row reads zeros and
// is not written.
__device__ __forceinline__ __amdgpu_buffer_rsrc_t rows_from(const void *p, int64_t n0, int64_t ld,
                                                            int64_t nrow, int width, int esz) {
  const int left = (int)min((int64_t)256, nrow - n0);
  return rsrc(static_cast<const uint8_t *>(p) + n0 * ld * esz,
              left > 0 ? (uint32_t)((left - 1) * (int)ld + width) * (uint32_t)esz : 0u);
}

// A wave's block of y: residual and result go through this wave's buffer, 32 rows at a time,
// 16-byte chunks permuted by the row, so that neighbouring lanes read and write one row's
// consecutive bytes. One rounding of residual + act(z). The buffers' range checks take the
// place of branches around every access, with which the epilogue takes as long as a sum of
// 1000; a row's last chunk, where 8 does not divide it, goes element by element.
template <class P>
__device__ __forceinline__ void store_rows(const f32x16 (&acc)[P::FM][P::FN], uint8_t *buf,
                                           int lane, int act, const uint16_t *residual,
                                           int64_t r_ld, uint16_t *y, int64_t y_ld, int64_t n0,
                                           int m0, int64_t nrow, int out) {
  constexpr int CPW = P::WM / 8, RB = P::WM * 2, SH = CPW == 16 ? 0 : CPW == 8 ? 1 : 2;
  constexpr int RPI = 64 / CPW;
  const int q = lane % CPW, m = m0 + 8 * q;
  auto place = [&](int r, int c) __attribute__((always_inline)) {
    return buf + r * RB + ((c ^ ((r >> SH) & (CPW - 1))) << 4);
  };
  const int64_t first = n0 + lane / CPW;
  const __amdgpu_buffer_rsrc_t rs_y = rows_from(y, n0, y_ld, nrow, out, 2);
  const __amdgpu_buffer_rsrc_t rs_r = rows_from(residual, n0, r_ld, nrow, out, 2);
  const unsigned yo = m + 8 <= out ? (unsigned)(lane / CPW * (int)y_ld + m) * 2u : kOOB;
  const unsigned ro = m + 8 <= out ? (unsigned)(lane / CPW * (int)r_ld + m) * 2u : kOOB;
  const bool edge = out % 8 && m0 + P::WM > out;       // (of the wave)
  const bool tail = edge && m < out && m + 8 > out;
#pragma unroll
  for (int j = 0; j < P::FN; ++j) {
    if (residual) {
      u32x4 d[32 / RPI];
#pragma unroll
      for (int k = 0; k < 32 / RPI; ++k) {
        d[k] = __builtin_amdgcn_raw_buffer_load_b128(
            rs_r, (int)(ro + (unsigned)((32 * j + k * RPI) * (int)r_ld) * 2u), 0, 0);
        const int64_t n = first + 32 * j + k * RPI;
        if (edge && tail && n < nrow) d[k] = row8(residual + n * r_ld, m, out);
      }
#pragma unroll
      for (int k = 0; k < 32 / RPI; ++k)
        *reinterpret_cast<u32x4 *>(place(k * RPI + lane / CPW, q)) = d[k];
      wait_lds();
      __builtin_amdgcn_wave_barrier();
    }
#pragma unroll
    for (int i = 0; i < P::FM; ++i) {
      float v[16];
      activate(v, acc[i][j], act);
#pragma unroll
      for (int g = 0; g < 4; ++g) {
        u32x2 *at = reinterpret_cast<u32x2 *>(place(lane & 31, 4 * i + g) + 8 * (lane >> 5));
        float *o = v + 4 * g;
        if (residual) {
          const u32x2 q = *at;
#pragma unroll
          for (int e = 0; e < 4; ++e) o[e] += to_f32(q[e >> 1] >> (16 * (e & 1)) & 0xFFFFu, P::BF);
        }
        *at = u32x2{pack2(o[0], o[1], P::BF), pack2(o[2], o[3], P::BF)};
      }
      apart();
    }
    wait_lds();
    __builtin_amdgcn_wave_barrier();
    u32x4 d[32 / RPI];
#pragma unroll
    for (int k = 0; k < 32 / RPI; ++k)
      d[k] = *reinterpret_cast<const u32x4 *>(place(k * RPI + lane / CPW, q));
#pragma unroll
    for (int k = 0; k < 32 / RPI; ++k) {
      __builtin_amdgcn_raw_buffer_store_b128(
          d[k], rs_y, (int)(yo + (unsigned)((32 * j + k * RPI) * (int)y_ld) * 2u), 0, 0);
      const int64_t n = first + 32 * j + k * RPI;
      if (edge && tail && n < nrow) put8(y + n * y_ld, m, out, d[k]);
    }
    wait_lds();
    __builtin_amdgcn_wave_barrier();
  }
}

// A wave's block of z as 8-bit codes: a group of 32 outputs of a row is 16 registers of this
// lane and of the one 32 further, which exchange halves, so that each writes 16 bytes.
template <class P>
__device__ __forceinline__ void pack_block(const f32x16 (&acc)[P::FM][P::FN], const Packed &p,
                                           int64_t n0, int m0, int64_t nrow, int out, int lane) {
  const bool up = lane >= 32;
  const __amdgpu_buffer_rsrc_t rs_q = rows_from(p.codes, n0, p.wide, nrow, p.wide, 1);
  const __amdgpu_buffer_rsrc_t rs_e = rows_from(p.exps, n0, p.wide / 32, nrow, p.wide / 32, 1);
#pragma unroll
  for (int j = 0; j < P::FN; ++j)
#pragma unroll
    for (int i = 0; i < P::FM; ++i) {
      float v[16];
#pragma unroll
      for (int e = 0; e < 16; ++e) v[e] = acc[i][j][e];
      if (m0 + 32 * i + 32 > out) {  // (weights past the end are zeros, but 0 x NaN is not)
#pragma unroll
        for (int e = 0; e < 16; ++e)
          if (m0 + 32 * i + 8 * (e >> 2) + 4 * (lane >> 5) + (e & 3) >= out) v[e] = 0.f;
      }
      uint32_t q[4];
      const uint32_t b =
          rows::pack_group<16>(v, q, [](uint32_t top) __attribute__((always_inline)) {
            const auto p = __builtin_amdgcn_permlane32_swap(top, top, false, false);
            return max(p[0], p[1]);
          });
      // the lower lane's words 2 and 3 for the upper one's 0 and 1
      const auto s0 = __builtin_amdgcn_permlane32_swap(q[0], q[2], false, false);
      const auto s1 = __builtin_amdgcn_permlane32_swap(q[1], q[3], false, false);
      const int r = 32 * j + (lane & 31), m = m0 + 32 * i;
      const bool in = m < p.wide;
      __builtin_amdgcn_raw_buffer_store_b128(
          u32x4{s0[0], s0[1], s1[0], s1[1]}, rs_q,
          in ? r * p.wide + m + (up ? 16 : 0) : (int)kOOB, 0, 0);
      __builtin_amdgcn_raw_buffer_store_b8((uint8_t)b, rs_e,
                                           in && !up ? r * (p.wide / 32) + m / 32 : (int)kOOB, 0,
                                           0);
      apart();
    }
}

// 4 elements of a vector of n from c on, zeros past its end.
__device__ __forceinline__ void load4(const uint16_t *p, int c, int n, bool bf, float (&v)[4]) {
  if (c + 4 <= n) {
    const u32x2 q = reinterpret_cast<const Any8 *>(p + c)->v;
#pragma unroll
    for (int e = 0; e < 4; ++e) v[e] = to_f32(q[e >> 1] >> (16 * (e & 1)) & 0xFFFFu, bf);
    return;
  }
#pragma unroll
  for (int e = 0; e < 4; ++e) v[e] = c + e < n ? to_f32(p[c + e], bf) : 0.f;
}

template <class P>
__device__ __forceinline__ void epilogue(f32x16 (&acc)[P::FM][P::FN], const Epilogue &a,
                                         uint8_t *buf, int lane, int64_t n0, int m0,
                                         int64_t nrow) {
#pragma unroll
  for (int i = 0; i < P::FM; ++i) {
    u32x2 q[4] = {};
    if (a.bias) {
#pragma unroll
      for (int g = 0; g < 4; ++g) {
        const int m = m0 + 32 * i + 8 * g + 4 * (lane >> 5);
        if (m + 4 <= a.out) q[g] = reinterpret_cast<const Any8 *>(a.bias + m)->v;
        if (m0 + P::WM > a.out && m < a.out && m + 4 > a.out)
#pragma unroll
          for (int e = 0; e < 3; ++e)
            if (m + e < a.out) q[g][e >> 1] |= (uint32_t)a.bias[m + e] << (16 * (e & 1));
      }
    }
#pragma unroll
    for (int v = 0; v < 16; ++v) {
      const float b = to_f32(q[v >> 2][v >> 1 & 1] >> (16 * (v & 1)) & 0xFFFFu, P::BF);
#pragma unroll
      for (int j = 0; j < P::FN; ++j) acc[i][j][v] += b;
    }
    apart();
  }
  if (a.z)
    store_rows<P>(acc, buf, lane, FG_ACT_NONE, nullptr, 0, a.z, a.z_ld, n0, m0, nrow, a.out);
  if (a.packed.codes) pack_block<P>(acc, a.packed, n0, m0, nrow, a.out, lane);
  store_rows<P>(acc, buf, lane, a.act, a.residual, a.r_ld, a.y, a.y_ld, n0, m0, nrow, a.out);
}

// fp32 sums of a wave's block to a part of a split sum.
template <class P>
__device__ __forceinline__ void store_part(const f32x16 (&acc)[P::FM][P::FN], float *part, int Mq,
                                           int lane, int64_t n0, int m0, int64_t nrow) {
#pragma unroll
  for (int j = 0; j < P::FN; ++j) {
    const int64_t n = n0 + 32 * j + (lane & 31);
    if (n >= nrow) continue;
#pragma unroll
    for (int i = 0; i < P::FM; ++i)
#pragma unroll
      for (int g = 0; g < 4; ++g) {
        const int m = m0 + 32 * i + 8 * g + 4 * (lane >> 5);
        if (m < Mq)
          *reinterpret_cast<f32x4 *>(part + n * Mq + m) =
              f32x4{acc[i][j][4 * g], acc[i][j][4 * g + 1], acc[i][j][4 * g + 2],
                    acc[i][j][4 * g + 3]};
      }
  }
}

template <class P>
__global__ __launch_bounds__(P::NT, P::WPE) void linear_fwd_kernel(FwdArgs a, TileMap tm) {
  FG_DMA_RING(P, R);
  constexpr int PA = P::PA, PB = P::PB, BK = P::BK;
  int tx, ty, split;  // rows, outputs, part
  if (!find_tile(tm, blockIdx.x, a.ntile, tx, ty, split)) return;
  const int64_t n0 = (int64_t)tx * P::TN;
  const int m0 = ty * P::TM;
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int wm0 = (wave / P::WGN) * P::WM, wn0 = (wave % P::WGN) * P::WN;
  const int kbeg = split * a.kper, kend = min(a.K, kbeg + a.kper);
  const int nst = kend > kbeg ? (kend - kbeg + BK - 1) / BK : 0;

  const int wrows = min(P::TM, a.e.out - m0);
  const int xrows = (int)min((int64_t)P::TN, a.rows - n0);
  const __amdgpu_buffer_rsrc_t rs_w =
      rsrc(a.w + m0 * a.w_ld, (uint32_t)((wrows - 1) * (int)a.w_ld + a.K) * 2u);
  const __amdgpu_buffer_rsrc_t rs_x =
      rsrc(a.x + n0 * a.x_ld, (uint32_t)((xrows - 1) * (int)a.x_ld + a.K) * 2u);
  const KmSlot<PA> as = km_slots<BK, PA>(wave, lane);
  const KmSlot<PB> bs = km_slots<BK, PB>(wave, lane);
  unsigned oa[PA], ob[PB], la[PA], lb[PB];
  // offsets in the last stage: its last chunk may begin before its place (both operands'
  // alike), and chunks past the end are zeros
  const int kl = kbeg + (nst - 1) * BK;
  auto tail = [&](unsigned o, int coff) __attribute__((always_inline)) {
    return kl + coff < a.K ? o + 2u * (chunk_at(kl + coff, a.K) - coff) : kOOB;
  };
#pragma unroll
  for (int jj = 0; jj < PA; ++jj) {
    oa[jj] = (unsigned)(as.row[jj] * (int)a.w_ld + as.coff[jj]) * 2u;
    la[jj] = tail(oa[jj], as.coff[jj]);
    oa[jj] += 2u * kbeg;
  }
#pragma unroll
  for (int jj = 0; jj < PB; ++jj) {
    ob[jj] = (unsigned)(bs.row[jj] * (int)a.x_ld + bs.coff[jj]) * 2u;
    lb[jj] = tail(ob[jj], bs.coff[jj]);
    ob[jj] += 2u * kbeg;
  }
  auto issue = [&](int st, int slot) __attribute__((always_inline)) {
    uint8_t *ta = R.a[slot], *tb = R.b[slot];
    const bool last = st + 1 == nst;
    const unsigned k0 = 2u * BK * st;
#pragma unroll
    for (int jj = 0; jj < PB; ++jj)
      dma16(rs_x, tb + dma_dst<PB>(wave, jj), last ? lb[jj] : ob[jj] + k0);
#pragma unroll
    for (int jj = 0; jj < PA; ++jj)
      dma16(rs_w, ta + dma_dst<PA>(wave, jj), last ? la[jj] : oa[jj] + k0);
  };
  // the last chunk's repeated elements: zeros in both operands, whatever they are
  auto fix = [&](Frags<P> &f, int it, int ks) __attribute__((always_inline)) {
    if (a.K % 8 == 0 || it + 1 != nst) return;
    const int over = kl + 16 * ks + 8 * (lane >> 5) + 8 - a.K;  // 1 .. 7: that chunk
    const int cut = over < 8 ? over : 0;
    u32x4 m;
#pragma unroll
    for (int d = 0; d < 4; ++d)
      m[d] = (2 * d < cut ? 0u : 0xFFFFu) | (2 * d + 1 < cut ? 0u : 0xFFFF0000u);
#pragma unroll
    for (int i = 0; i < P::FM; ++i) f.a[i] &= m;
#pragma unroll
    for (int j = 0; j < P::FN; ++j) f.b[j] &= m;
  };
  f32x16 acc[P::FM][P::FN];
  zero<P>(acc);
  pipeline<P, true, true>(acc, R, nst, wm0, wn0, lane, issue, NoFold{}, fix);
  if (a.part) {
    store_part<P>(acc, a.part + split * a.pstride, a.Mq, lane, n0 + wn0, m0 + wm0, a.rows);
    return;
  }
  lds_barrier();  // every wave is done reading the ring
  epilogue<P>(acc, a.e, wave_buf<P>(R, wave), lane, n0 + wn0, m0 + wm0, a.rows);
}

// ---- forward, few rows -----------------------------------------------------------------
// Up to 16 NB rows (tokens served one by one): bound by reading the weights once. A workgroup
// takes 8 A8 outputs and NB blocks of 16 rows, its NW waves a run of the sum each. A wave
// feeds itself: a ring of its own in LDS, whose stages of 64 columns come by DMA in whole
// 128-byte lines, so that it waits for nothing but its oldest loads and some 100 KiB a CU are
// always on their way. The waves' sums meet in LDS at the end, in order.
// (A 24 x 4096 -> 4096 in 11.6 us with its weights from memory, of 6.7 that a copy needs; tiles
// 13.9. One row, 2048 -> 8192: 9.5 and 13.0; 8192 -> 32768: 99 and 117, of 107.)
// More than 32 rows of more than 8192 outputs are the tiles' (64 x 4096 -> 16384 36.3 us, 40.2
// here; 64 x 512 -> 16384 8.5 and 10.7; 64 x 2048 -> 8192 15.3 and 11.9).
inline bool few_rows(int64_t rows, int64_t out) { return rows <= (out <= 8192 ? 64 : 32); }
template <bool BF>
__device__ __forceinline__ f32x4 mfma16(const u32x4 &a, const u32x4 &b, const f32x4 &c) {
  if (BF)
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf8, a),
                                                   __builtin_bit_cast(bf8, b), c, 0, 0, 0);
  return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(half8, a),
                                                __builtin_bit_cast(half8, b), c, 0, 0, 0);
}

template <int A8_, int NB_, int NW_>
struct Few {
  static constexpr int A8 = A8_, OUT = 8 * A8;        // outputs
  static constexpr int MB = (A8 + 1) / 2, NB = NB_, NW = NW_, NT = 64 * NW;
  static constexpr int A = 1024 * A8, STAGE = A + 2048 * NB;  // bytes of 64 columns
  static constexpr int LOADS = A8 + 2 * NB;                   // DMA instructions, 8 rows each
  static constexpr int FIT = 152 * 1024 / (NW * STAGE), NS = FIT < 8 ? FIT : 8;
  static_assert(NS >= 2 && (NS - 1) * LOADS < 64, "ring depth, vmcnt range");
};

// Waits until at most n of the wave's stages, and N of them, are on their way.
template <class F, int N>
__device__ __forceinline__ void wait_younger(int n) {
  if constexpr (N == 0) {
    wait_vm<0>();
  } else {
    if (n >= N)
      wait_vm<N * F::LOADS>();
    else
      wait_younger<F, N - 1>(n);
  }
}

template <bool BF, class F>
__global__ __launch_bounds__(F::NT) void linear_few_kernel(FwdArgs a) {
  constexpr int A8 = F::A8, MB = F::MB, NB = F::NB, NW = F::NW, NS = F::NS;
  __shared__ __attribute__((aligned(1024))) uint8_t lds[NW * NS * F::STAGE];
  const int lane = threadIdx.x & 63;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int m0 = blockIdx.x * F::OUT, K = a.K, rows = (int)a.rows;
  const int out = min(a.e.out, m0 + F::OUT);  // this workgroup's end
  uint8_t *ring = lds + wave * NS * F::STAGE;
  // what the end needs, on its way meanwhile: outputs m .. m + 3 of row n, a block of 16 x 16
  // for each wave in turn
  constexpr int NE = (MB * NB + NW - 1) / NW;
  const Epilogue &e = a.e;
  float bias[NE][4] = {}, res[NE][4] = {};
#pragma unroll
  for (int k = 0; k < NE; ++k) {
    const int id = wave + NW * k, m = m0 + 16 * (id / NB) + 4 * (lane >> 4),
              n = 16 * (id % NB) + (lane & 15);
    if (id >= MB * NB || n >= rows || m >= out) continue;
    if (e.bias) load4(e.bias, m, out, BF, bias[k]);
    if (e.residual) load4(e.residual + n * e.r_ld, m, out, BF, res[k]);
  }
  const __amdgpu_buffer_rsrc_t rs_w =
      rsrc(a.w + m0 * a.w_ld, (uint32_t)((out - m0 - 1) * (int)a.w_ld + K) * 2u);
  const __amdgpu_buffer_rsrc_t rs_x = rsrc(a.x, (uint32_t)((rows - 1) * (int)a.x_ld + K) * 2u);
  // a DMA instruction fills 8 rows; lane: row lane / 8, the chunk that belongs at its place
  const int r8 = lane >> 3;
  unsigned wo[A8], xo[2 * NB];
  int ch[2];
#pragma unroll
  for (int h = 0; h < 2; ++h) ch[h] = 8 * ((lane & 7) ^ kmaj_swz<64>(8 * h + r8));
#pragma unroll
  for (int b = 0; b < A8; ++b) wo[b] = (unsigned)((8 * b + r8) * (int)a.w_ld) * 2u;
#pragma unroll
  for (int b = 0; b < 2 * NB; ++b) xo[b] = (unsigned)((8 * b + r8) * (int)a.x_ld) * 2u;
  const int stages = (K + 63) / 64, per = (stages + NW - 1) / NW;
  const int first = wave * per, run = min(per, stages - first);
  // Each workgroup begins its runs elsewhere: where all read the same part of rows of a power
  // of two bytes, few memory channels serve them.
  const int turn = run > 0 ? (int)(blockIdx.x % (unsigned)run) : 0;
  auto column = [&](int st) __attribute__((always_inline)) {
    const int to = st + turn;
    return 64 * (first + (to < run ? to : to - run));
  };
  auto issue = [&](int st, int slot) __attribute__((always_inline)) {
    uint8_t *to = ring + slot * F::STAGE;
    const int k0 = column(st);
    // a last chunk of fewer than 8 begins earlier, in both operands alike
    auto at = [&](unsigned row, int c) __attribute__((always_inline)) {
      return c < K ? row + 2u * chunk_at(c, K) : kOOB;
    };
#pragma unroll
    for (int b = 0; b < A8; ++b) dma16(rs_w, to + 1024 * b, at(wo[b], k0 + ch[b & 1]));
#pragma unroll
    for (int b = 0; b < 2 * NB; ++b) dma16(rs_x, to + F::A + 1024 * b, at(xo[b], k0 + ch[b & 1]));
  };
  f32x4 acc[MB][NB];
#pragma unroll
  for (int i = 0; i < MB; ++i)
#pragma unroll
    for (int j = 0; j < NB; ++j) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};
  auto stage = [&](int st, int slot) __attribute__((always_inline)) {
    const uint8_t *at = ring + slot * F::STAGE;
    const int k0 = column(st);
#pragma unroll
    for (int ks = 0; ks < 2; ++ks) {
      const int c = 4 * ks + (lane >> 4);
      u32x4 fa[MB], fb[NB];
#pragma unroll
      for (int b = 0; b < MB; ++b)
        fa[b] = *reinterpret_cast<const u32x4 *>(
            at + 2048 * b + kmaj_off<64>(lane & (A8 == 1 ? 7 : 15), c));
#pragma unroll
      for (int b = 0; b < NB; ++b)
        fb[b] = *reinterpret_cast<const u32x4 *>(at + F::A + 2048 * b + kmaj_off<64>(lane & 15, c));
      if (K % 8 && k0 + 64 > K) {  // what the last chunk repeats: zeros, whatever it is
        const int over = k0 + 8 * c + 8 - K, cut = over < 8 ? over : 0;
        u32x4 m;
#pragma unroll
        for (int d = 0; d < 4; ++d)
          m[d] = (2 * d < cut ? 0u : 0xFFFFu) | (2 * d + 1 < cut ? 0u : 0xFFFF0000u);
#pragma unroll
        for (int b = 0; b < MB; ++b) fa[b] &= m;
#pragma unroll
        for (int b = 0; b < NB; ++b) fb[b] &= m;
      }
#pragma unroll
      for (int i = 0; i < MB; ++i)
#pragma unroll
        for (int j = 0; j < NB; ++j) acc[i][j] = mfma16<BF>(fa[i], fb[j], acc[i][j]);
    }
  };
#pragma unroll
  for (int s = 0; s < NS - 1; ++s)
    if (s < run) issue(s, s);
  int slot = 0;
  for (int st = 0; st < run; ++st) {
    // this wave has read the slot that it fills now
    wait_lds();
    asm volatile("" ::: "memory");
    if (st + NS - 1 < run) issue(st + NS - 1, slot ? slot - 1 : NS - 1);
    wait_younger<F, NS - 1>(run - 1 - st);
    asm volatile("" ::: "memory");
    stage(st, slot);
    slot = slot + 1 < NS ? slot + 1 : 0;
  }
  wait_lds();
  __syncthreads();
  f32x4 *sums = reinterpret_cast<f32x4 *>(lds);
  static_assert(NW * MB * NB * 1024 <= (int)sizeof(lds), "the sums take the rings' place");
#pragma unroll
  for (int i = 0; i < MB; ++i)
#pragma unroll
    for (int j = 0; j < NB; ++j) sums[((i * NB + j) * NW + wave) * 64 + lane] = acc[i][j];
  __syncthreads();
#pragma unroll
  for (int k = 0; k < NE; ++k) {
    const int id = wave + NW * k, m = m0 + 16 * (id / NB) + 4 * (lane >> 4),
              n = 16 * (id % NB) + (lane & 15);
    if (id >= MB * NB || n >= rows || m >= out) continue;
    float v[4] = {};
#pragma unroll
    for (int w = 0; w < NW; ++w) {
      const f32x4 q = sums[(id * NW + w) * 64 + lane];
#pragma unroll
      for (int i = 0; i < 4; ++i) v[i] += q[i];
    }
    auto put = [&](uint16_t *row) __attribute__((always_inline)) {
      const u32x2 q = {pack2(v[0], v[1], BF), pack2(v[2], v[3], BF)};
#pragma unroll
      for (int i = 0; i < 4; ++i)
        if (m + i < out) row[m + i] = (uint16_t)(q[i >> 1] >> (16 * (i & 1)));
    };
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] += bias[k][i];
    if (e.z) put(e.z + n * e.z_ld);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      v[i] = apply(v[i], e.act);
      if (e.residual) v[i] += res[k][i];
    }
    put(e.y + n * e.y_ld);
  }
}

// ---- the gradient of z -----------------------------------------------------------------
struct DzArgs {
  const uint16_t *dy, *z;
  Packed packed;
  uint16_t *dz;          // null: sums only
  float *part;           // [row blocks][Mp] or null
  int64_t rows, dy_ld, z_ld, per;   // rows of a workgroup
  int32_t out, Mp, act, tlog;       // 2^tlog lanes side by side
  uint32_t cblocks, blocks;         // workgroups side by side; all
};

// dz = dy act'(z), rounded to the type that the products take (the matrix pipes' operands have 16
// bits; it is all by which dx and dw differ from products of dz in fp32: off the exact values by
// 2.9e-4 in norm, 2.1e-4 without, of 65536 x 256 -> 1024 fp16, and 2.3e-3, 1.7e-3 without, of 16384
// x 2048 -> 8192 bf16), in rows of a multiple of 8 with zeros behind them; its columns' fp32 sums per workgroup, before the rounding. Bound by
// memory: the next kRows rows are on their way while these are worked on. KEPT: z in 16 bits
// or (1) its checkpoint; EVEN: 8 divides the columns, no masks.
// 16384 x 8192 bf16 from z's checkpoint, gelu: 161 us, 4.2 TB/s (175, 4.4, with the checkpoint of
// 2048 columns of x); 65536 x 1024 fp16 74 us, 4.5 (86, 4.5, with 256).
constexpr int kRows = 4;
template <class T, int ACT, int KEPT, bool EVEN>
struct DzLoads {
  rows::Raw<T> d[kRows], h[ACT && !KEPT ? kRows : 1];
  u32x2 q[ACT && KEPT ? kRows : 1];
  uint32_t e[ACT && KEPT ? kRows : 1];
  static __device__ __forceinline__ rows::Raw<T> raw(const T *row, int c, int cols) {
    if constexpr (EVEN)
      return __builtin_bit_cast(rows::Raw<T>, reinterpret_cast<const Any16 *>(row + c)->v);
    else
      return rows::load_any(row, c, cols);
  }
  __device__ __forceinline__ void load(const DzArgs &a, int64_t r, int teams, int c) {
    const T *dy = reinterpret_cast<const T *>(a.dy), *z = reinterpret_cast<const T *>(a.z);
#pragma unroll
    for (int k = 0; k < kRows; ++k) {
      const int64_t n = min(r + k * teams, a.rows - 1);
      d[k] = raw(dy + n * a.dy_ld, c, a.out);
      if constexpr (ACT && KEPT) {
        q[k] = *reinterpret_cast<const u32x2 *>(a.packed.codes + n * a.packed.wide + c);
        e[k] = a.packed.exps[n * (a.packed.wide / 32) + c / 32];
      } else if constexpr (ACT != 0) {
        h[k] = raw(z + n * a.z_ld, c, a.out);
      }
    }
  }
  static __device__ __forceinline__ void numbers(const rows::Raw<T> &r, int c, int cols,
                                                 float (&v)[8]) {
    if constexpr (EVEN) {
      typedef T t8 __attribute__((ext_vector_type(8)));
      const t8 x = __builtin_bit_cast(t8, r);
#pragma unroll
      for (int i = 0; i < 8; ++i) v[i] = (float)x[i];
    } else {
      rows::values<T>(r, c, cols, v);
    }
  }
};

// The workgroups behind these unpack x's checkpoint, if any: no launch of its own.
template <int DT, int ACT, int KEPT, bool EVEN>
__global__ __launch_bounds__(256) void linear_dz_kernel(DzArgs a, act8::Args x) {
  using T = typename TypeOf<DT>::T;
  using Loads = DzLoads<T, ACT, KEPT, EVEN>;
  __shared__ float sums[256][9];
  if (blockIdx.x >= a.blocks) {
    act8::unpack_block<DT>(x, blockIdx.x - a.blocks);
    return;
  }
  const int by = (int)(blockIdx.x / a.cblocks), bx = (int)(blockIdx.x - by * a.cblocks);
  const int tl = 1 << a.tlog, t = threadIdx.x & (tl - 1), team = threadIdx.x >> a.tlog;
  const int teams = 256 >> a.tlog;
  const int c = 8 * (bx * tl + t);
  const int64_t r0 = (int64_t)by * a.per + team, r1 = min(a.rows, r0 - team + a.per);
  T *dz = reinterpret_cast<T *>(a.dz);
  float s[8] = {};
  if (c < a.Mp) {
    Loads next;
    next.load(a, r0, teams, c);
    for (int64_t r = r0; r < r1; r += kRows * teams) {
      const Loads now = next;
      if (r + kRows * teams < r1) next.load(a, r + kRows * teams, teams, c);
#pragma unroll
      for (int k = 0; k < kRows; ++k) {
        const int64_t n = r + k * teams;
        if (n >= r1) break;
        float g[8], v[8];
        Loads::numbers(now.d[k], c, a.out, g);
        if constexpr (ACT != 0) {
          if constexpr (KEPT)
            rows::decode8(now.q[k], now.e[k], v);
          else
            Loads::numbers(now.h[k], c, a.out, v);
#pragma unroll
          for (int i = 0; i < 8; ++i) {
            if constexpr (ACT == FG_ACT_RELU)
              g[i] = v[i] > 0.f ? g[i] : v[i] != v[i] ? v[i] : 0.f;
            else
              g[i] *= gelu_slope(v[i]);
            if (!EVEN && c + i >= a.out) g[i] = 0.f;
          }
        }
#pragma unroll
        for (int i = 0; i < 8; ++i) s[i] += g[i];
        if (dz)
          *reinterpret_cast<u32x4 *>(dz + n * a.Mp + c) =
              u32x4{pack2(g[0], g[1], DT == FG_BF16), pack2(g[2], g[3], DT == FG_BF16),
                    pack2(g[4], g[5], DT == FG_BF16), pack2(g[6], g[7], DT == FG_BF16)};
      }
    }
  }
  if (!a.part) return;
#pragma unroll
  for (int i = 0; i < 8; ++i) sums[threadIdx.x][i] = s[i];
  __syncthreads();
  for (int k = threadIdx.x; k < 8 * tl; k += 256) {
    const int col = 8 * bx * tl + k;
    if (col >= a.Mp) break;
    float v = 0.f;
    for (int j = 0; j < teams; ++j) v += sums[(j << a.tlog) + k / 8][k % 8];
    a.part[(int64_t)by * a.Mp + col] = v;
  }
}

// The sums of the row blocks, in order: 16 columns a workgroup, 64 lanes' runs of them each. In
// the products' launch, where there is one.
struct SumArgs {
  const float *part;
  uint16_t *out;
  int32_t n, Mp, cols;
  int32_t *flag;
};
template <class T>
__device__ __forceinline__ void sum_block(const SumArgs &a, int block, void *lds) {
  const int c = 16 * block + (threadIdx.x & 15);
  float s;
  rows::sum_columns(a.part, a.n, a.Mp, 16 * block, a.Mp, lds, s);
  bool bad = false;
  if (threadIdx.x < 16 && c < a.cols) {
    const T v = (T)s;
    reinterpret_cast<T *>(a.out)[c] = v;
    bad = !(fabsf((float)v) < INFINITY);
  }
  if (a.flag) flag_nonfinite(a.flag, bad);
}
template <int DT>
__global__ __launch_bounds__(256) void linear_sum_kernel(SumArgs a) {
  __shared__ __attribute__((aligned(16))) uint8_t lds[rows::kSumLds];
  sum_block<typename TypeOf<DT>::T>(a, blockIdx.x, lds);
}

// ---- products of the gradients ---------------------------------------------------------
// out[n][m] = sum_k A[k][m] B(n, k): A's rows (of w: outputs; of x: rows) lie across the sum;
// dz is B, by rows n (dx, k: outputs) or columns n (dw, k: rows). Bound by the matrix pipes: both
// gradients of 16384 x 2048 -> 8192 bf16 take 845 us, 1.30 PFLOP/s at 74% of the pipes' cycles
// and 1.7 GHz, which the board's power allows. 65536 x 256 -> 1024, 103 us, is a third of them:
// dz is read twice, and a product's tiles have sums of 256 or a share of 65536.
struct ProdArgs {
  const uint16_t *a;
  int64_t a_ld;
  int32_t a_cols;            // at least 8
  const uint16_t *b;
  int64_t b_ld;
  int32_t b_cols;            // a multiple of 8
  int64_t N, K;              // rows of the output; the sum's length
  int64_t kper;              // of a part (a multiple of 64)
  int32_t M, ntile;
  uint16_t *out;             // null: fp32 sums to part
  int64_t out_ld;
  float *part;               // [parts][N][Mq]
  int64_t pstride;
  int32_t Mq;
  int32_t *flag;
};

template <class P, bool DX>
__device__ __forceinline__ void product_tile(const ProdArgs &a, const TileMap &tm, int block,
                                             const Ring &R) {
  constexpr int PA = P::PA, PB = P::PB, BK = P::BK;
  int tx, ty, split;  // columns m, rows n, part
  if (!find_tile(tm, block, a.ntile, tx, ty, split)) return;
  const int m0 = tx * P::TM;
  const int64_t n0 = (int64_t)ty * P::TN;
  const int64_t kbeg = split * a.kper, kend = min(a.K, kbeg + a.kper);
  const int nst = kend > kbeg ? (int)((kend - kbeg + BK - 1) / BK) : 0;
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int wm0 = (wave / P::WGN) * P::WM, wn0 = (wave % P::WGN) * P::WN;

  const MnSlot<PA> as = mn_slots<P::RBA, PA>(wave, lane);
  unsigned oa[PA], ob[PB], lb[PB];
#pragma unroll
  for (int jj = 0; jj < PA; ++jj)
    oa[jj] = m0 + as.ncol[jj] < a.a_cols
                 ? (unsigned)(as.krow[jj] * (int)a.a_ld + chunk_at(m0 + as.ncol[jj], a.a_cols)) * 2u
                 : kOOB;
  const uint16_t *pa = a.a + kbeg * a.a_ld, *pb = nullptr;
  // dx: all of the tile's rows of dz; kend is their end but for the last part's
  const int64_t kcol = min((int64_t)a.b_cols, kbeg + a.kper);
  const int brows = (int)min((int64_t)P::TN, a.N - n0);
  __amdgpu_buffer_rsrc_t rs_rows;
  if constexpr (DX) {
    const KmSlot<PB> bs = km_slots<BK, PB>(wave, lane);
    rs_rows = rsrc(a.b + n0 * a.b_ld, (uint32_t)((brows - 1) * (int)a.b_ld + a.b_cols) * 2u);
    const int kl = (int)kbeg + (nst - 1) * BK;
#pragma unroll
    for (int jj = 0; jj < PB; ++jj) {
      const unsigned o = (unsigned)(bs.row[jj] * (int)a.b_ld + bs.coff[jj]) * 2u;
      ob[jj] = o + 2u * (unsigned)kbeg;
      lb[jj] = kl + bs.coff[jj] < kcol ? o + 2u * (unsigned)kl : kOOB;
    }
  } else {
    const MnSlot<PB> bs = mn_slots<P::RBB, PB>(wave, lane);
    pb = a.b + kbeg * a.b_ld + n0;
#pragma unroll
    for (int jj = 0; jj < PB; ++jj)
      ob[jj] = n0 + bs.ncol[jj] < a.b_cols
                   ? (unsigned)(bs.krow[jj] * (int)a.b_ld + bs.ncol[jj]) * 2u
                   : kOOB;
  }
  int64_t left = kend - kbeg;
  auto issue = [&](int st, int slot) __attribute__((always_inline)) {
    uint8_t *ta = R.a[slot], *tb = R.b[slot];
    const int r = (int)min(left, (int64_t)BK);
    const __amdgpu_buffer_rsrc_t rs_a = rsrc(pa, (uint32_t)((r - 1) * (int)a.a_ld + a.a_cols) * 2u);
    if constexpr (DX) {
      const bool last = st + 1 == nst;
      const unsigned k0 = 2u * BK * st;
#pragma unroll
      for (int jj = 0; jj < PB; ++jj)
        dma16(rs_rows, tb + dma_dst<PB>(wave, jj), last ? lb[jj] : ob[jj] + k0);
    } else {
      const __amdgpu_buffer_rsrc_t rs_b =
          rsrc(pb, (uint32_t)((r - 1) * (int)a.b_ld + a.b_cols - (int)n0) * 2u);
#pragma unroll
      for (int jj = 0; jj < PB; ++jj) dma16(rs_b, tb + dma_dst<PB>(wave, jj), ob[jj]);
      pb += BK * a.b_ld;
    }
#pragma unroll
    for (int jj = 0; jj < PA; ++jj) dma16(rs_a, ta + dma_dst<PA>(wave, jj), oa[jj]);
    pa += BK * a.a_ld;
    left -= BK;
  };
  f32x16 acc[P::FM][P::FN];
  zero<P>(acc);
  pipeline<P, false, DX>(acc, R, nst, wm0, wn0, lane, issue);
  if (a.part) {
    store_part<P>(acc, a.part + split * a.pstride, a.Mq, lane, n0 + wn0, m0 + wm0, a.N);
    return;
  }
  lds_barrier();  // every wave is done reading the ring
  bool bad = false;
  const __amdgpu_buffer_rsrc_t rs_out = rows_from(a.out, n0 + wn0, a.out_ld, a.N, a.M, 2);
  store16<P>(
      wave_buf<P>(R, wave), lane,
      [&](int i, int j, int g) __attribute__((always_inline)) {
        const f32x16 &c = acc[i][j];
        return u32x2{pack2(c[4 * g], c[4 * g + 1], P::BF),
                     pack2(c[4 * g + 2], c[4 * g + 3], P::BF)};
      },
      [&](int r, int c, const u32x4 &d) __attribute__((always_inline)) {
        const int64_t n = n0 + wn0 + r;
        const int m = m0 + wm0 + c;
        const bool in = n < a.N && m < a.M;
        constexpr uint32_t EX = P::BF ? 0x7F80u : 0x7C00u;
        if (!DX) {
          bool inf = false;
#pragma unroll
          for (int e = 0; e < 8; ++e) inf |= (d[e >> 1] >> (16 * (e & 1)) & EX) == EX;
          bad |= inf && in;
        }
        if (a.M >= 8)
          __builtin_amdgcn_raw_buffer_store_b128(
              d, rs_out, in ? (r * (int)a.out_ld + chunk_at(m, a.M)) * 2 : (int)kOOB, 0, 0);
        else if (in)
          put8(a.out + n * a.out_ld, m, a.M, d);
      });
  if (!DX && a.flag) flag_nonfinite(a.flag, bad);
}

// Both in one launch: neither waits for the other's last tiles. The one whose sums (their
// parts) are longer takes the first workgroups, `first` of them; the last ones sum up dbias.
template <class P>
__global__ __launch_bounds__(P::NT, P::WPE) void linear_products_kernel(ProdArgs dx, TileMap tx,
                                                                        ProdArgs dw, TileMap tw,
                                                                        SumArgs sum, int first,
                                                                        int both, int dx_first) {
  FG_DMA_RING(P, R);
  const int block = blockIdx.x;
  if (block >= both) {
    static_assert(P::A_BYTES >= rows::kSumLds, "room for the sums");
    using T = typename TypeOf<P::BF ? FG_BF16 : FG_F16>::T;
    sum_block<T>(sum, block - both, R.a[0]);
    return;
  }
  const bool leads = block < first;
  const int at = leads ? block : block - first;
  if (leads == (dx_first != 0))
    product_tile<P, true>(dx, tx, at, R);
  else
    product_tile<P, false>(dw, tw, at, R);
}

// ---- joins -----------------------------------------------------------------------------
// The parts of split sums, in their order: 8 columns of a row per lane, or per 2^slog lanes
// with a run of the parts each, whose sums then meet in LDS.
struct JoinArgs {
  const float *part;
  int64_t pstride, rows;
  int32_t nsplit, M, Mq;
  uint16_t *out;
  int64_t out_ld;
  int32_t *flag;
  int32_t slog;
};
// Lanes to a sum: 256 parts of 64 x 24 sums took 25 us by single lanes.
inline int shared_log(int nsplit) { return nsplit < 16 ? 0 : nsplit < 64 ? 2 : 4; }
__device__ __forceinline__ void joined(const float *p, int nsplit, int64_t pstride, float (&v)[8]) {
#pragma unroll
  for (int e = 0; e < 8; ++e) v[e] = 0.f;
#pragma unroll 4
  for (int s = 0; s < nsplit; ++s, p += pstride)
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const f32x4 x = *reinterpret_cast<const f32x4 *>(p + 4 * h);
#pragma unroll
      for (int e = 0; e < 4; ++e) v[4 * h + e] += x[e];
    }
}
template <int DT>
__device__ __forceinline__ u32x4 rounded(const float (&v)[8]) {
  u32x4 d;
#pragma unroll
  for (int e = 0; e < 4; ++e) d[e] = pack2(v[2 * e], v[2 * e + 1], DT == FG_BF16);
  return d;
}
template <int DT>
__global__ __launch_bounds__(256) void linear_join_kernel(JoinArgs dx, JoinArgs dw, int nx) {
  __shared__ float sums[256][8];
  const bool first = (int)blockIdx.x < nx;
  const JoinArgs &a = first ? dx : dw;
  const int wide = 256 >> a.slog, t = threadIdx.x & (wide - 1), share = threadIdx.x / wide;
  const int64_t i = (int64_t)(first ? blockIdx.x : blockIdx.x - nx) * wide + t;
  const int c8 = a.Mq / 8;
  const int64_t n = i / c8;
  const int m = (int)(i - n * c8) * 8;
  const int per = (a.nsplit + (1 << a.slog) - 1) >> a.slog, s0 = share * per;
  bool bad = false;
  float v[8] = {};
  if (n < a.rows)
    joined(a.part + s0 * a.pstride + n * a.Mq + m, min(per, a.nsplit - s0), a.pstride, v);
  if (a.slog) {
#pragma unroll
    for (int e = 0; e < 8; ++e) sums[threadIdx.x][e] = v[e];
    __syncthreads();
    for (int k = 1; !share && k < 1 << a.slog; ++k)
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e] += sums[k * wide + t][e];
  }
  if (n < a.rows && !share) {
    const u32x4 d = rounded<DT>(v);
    constexpr uint32_t EX = DT == FG_BF16 ? 0x7F80u : 0x7C00u;
#pragma unroll
    for (int e = 0; e < 8; ++e) bad |= (d[e >> 1] >> (16 * (e & 1)) & EX) == EX;
    put_chunk(a.out + n * a.out_ld, m, a.M, d);
  }
  if (a.flag) flag_nonfinite(a.flag, bad);
}

// ... of the forward product, with its epilogue: lanes by columns, rounded up to a
// checkpoint's groups.
struct JoinFwd {
  const float *part;
  int64_t pstride, rows;
  int32_t nsplit, Mq, wide;
  Epilogue e;
};
template <int DT>
__global__ __launch_bounds__(256) void linear_join_fwd_kernel(JoinFwd a) {
  using T = typename TypeOf<DT>::T;
  const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
  const int c8 = a.wide / 8;
  const int64_t n = i / c8;
  const int m = (int)(i - n * c8) * 8;
  if (n >= a.rows) return;  // (whole groups of 4 lanes)
  const Epilogue &e = a.e;
  float v[8] = {};
  if (m < e.out) {
    joined(a.part + n * a.Mq + m, a.nsplit, a.pstride, v);
    if (e.bias) {
      float b[8];
      rows::load8(reinterpret_cast<const T *>(e.bias), m, e.out, b);
#pragma unroll
      for (int k = 0; k < 8; ++k) v[k] += b[k];
    }
#pragma unroll
    for (int k = 0; k < 8; ++k)
      if (m + k >= e.out) v[k] = 0.f;
    if (e.z) rows::store8(reinterpret_cast<T *>(e.z) + n * e.z_ld, m, e.out, v);
  }
  if (e.packed.codes) rows::pack8(e.packed, n, m, v);
  if (m >= e.out) return;
  float r[8] = {};
  if (e.residual)
    rows::load8(reinterpret_cast<const T *>(e.residual) + n * e.r_ld, m, e.out, r);
#pragma unroll
  for (int k = 0; k < 8; ++k) {
    v[k] = apply(v[k], e.act);
    if (e.residual) v[k] += r[k];
  }
  rows::store8(reinterpret_cast<T *>(e.y) + n * e.y_ld, m, e.out, v);
}

// Rows of fewer than 8 elements, padded with zeros to 8.
__global__ __launch_bounds__(256) void linear_pad_kernel(const uint16_t *x, int64_t ld, int32_t n,
                                                         uint16_t *to, int64_t rows) {
  const int64_t r = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (r < rows) *reinterpret_cast<u32x4 *>(to + r * 8) = row8(x + r * ld, 0, n);
}

// ---- host ------------------------------------------------------------------------------
// Tile and number of parts for up to two products of a launch: the least of the times
// estimated for rounds of the workgroups that the chip holds. A round of m workgroups whose
// sums are k long takes f + e x + k (g + h x), x = m / (256 occ): its beginning and end, and
// each stage, both longer where the chip is full. A join takes a start and its bytes' time.
// Forward: fitted to 420 timings (22 shapes of 100 .. 65536 rows and 64 .. 8000 columns, by
// every tile in 1 .. 64 parts), the choice within 1.5% of the best on average. Gradients, each
// alone and both: to 7800 (94 shapes of 200 .. 100000 rows and 16 .. 8000 columns), the choice
// within 4% (weighted by the time's root; with forward's constants and tiles 9%). On 86 other
// shapes the calls for both gain 4% by it, those for dx 8%, for dw 4%, a tile for one alone
// included.
enum { kT64, kT128, kT256, kT128D, kS256, kTiles, kS128 = kTiles };
constexpr int kSideM[] = {64, 128, 256, 128, 256}, kSideN[] = {64, 128, 256, 128, 128};
struct Cost {
  int occ;
  double f, e, g, h;
};
struct Costs {
  int tiles;
  Cost c[kTiles];
  double join, rate;   // us; bytes a us
};
constexpr Costs kFwd = {4,
                        {{3, 0.0, 2.2, .0029, .0043},
                         {2, 0.6, 3.5, .0068, .0053},
                         {1, 7.6, 0.0, .0151, .0020},
                         {1, 2.2, 1.6, .0060, .0012}},
                        3.75, 6.2e6};
constexpr Costs kBwd = {5,
                        {{3, 3.1, 0.0, .0030, .0068},
                         {2, 1.5, 3.7, .0078, .0038},
                         {1, 6.8, 1.9, .0117, .0052},
                         {1, 5.6, 0.0, .0059, .0022},
                         {2, 2.7, 3.3, .0119, .0070}},
                        2.5, 3.2e6};
struct Need {
  int64_t M, N, K;
};
double round_of(const Cost &c, double m, double k) {
  const double x = m / (256.0 * c.occ);
  return c.f + c.e * x + k * (c.g + c.h * x);
}
// n workgroups of k on average, the longest first.
double rounds(const Cost &c, double n, double k, double longest) {
  const double slots = 256.0 * c.occ, full = (double)(int64_t)(n / slots), rest = n - full * slots;
  return std::max(full * round_of(c, slots, k) + (rest > 0 ? round_of(c, rest, k) : 0.0),
                  round_of(c, std::min(n, slots), longest));
}
struct Parts {
  double n, k, join;   // workgroups; length of a part; time to join
  int ns, kper;
};
int64_t tiles_of(const Need &p, int t) {
  return up(p.M, kSideM[t]) / kSideM[t] * (up(p.N, kSideN[t]) / kSideN[t]);
}
// The numbers of parts worth a look.
int parts_of(const Need &p, const Costs &cost, int t, Parts (&out)[10]) {
  const int64_t tiles = tiles_of(p, t);
  int n = 0;
  for (int ns = 1; ns <= 512; ns *= 2) {
    const int64_t kper = std::max<int64_t>(64, ((p.K + ns - 1) / ns + 63) / 64 * 64);
    const int64_t parts = std::max<int64_t>(1, (p.K + kper - 1) / kper);
    if (ns > 1 && (kper < 128 || tiles * parts > 4096)) break;
    out[n++] = {(double)(tiles * parts), (double)kper,
                parts > 1 ? (double)parts * p.M * p.N * 8 / cost.rate : 0.0, (int)parts,
                (int)kper};
  }
  return n;
}
void pick(const Costs &cost, const Need *p, int np, Shape *s) {
  double best = 1e300;
  for (int t = 0; t < cost.tiles; ++t) {
    Parts a[10], b[10];
    const int na = parts_of(p[0], cost, t, a), nb = np > 1 ? parts_of(p[1], cost, t, b) : 1;
    if (np == 1) b[0] = {0, 0, 0, 0, 0};
    for (int i = 0; i < na; ++i)
      for (int j = 0; j < nb; ++j) {
        const double n = a[i].n + b[j].n;
        double us = rounds(cost.c[t], n, (a[i].n * a[i].k + b[j].n * b[j].k) / n,
                           std::max(a[i].k, b[j].k)) + a[i].join + b[j].join;
        if (a[i].join + b[j].join > 0) us += cost.join;
        if (us >= best) continue;
        best = us;
        s[0] = {t, a[i].ns, a[i].kper};
        if (np > 1) s[1] = {t, b[j].ns, b[j].kper};
      }
  }
}

// The tile for one product whose parts are settled.
int tile_for(const Costs &cost, const Need &p, const Shape &s) {
  int best = s.tile;
  double least = 1e300;
  for (int t = 0; t < cost.tiles; ++t) {
    const double us = rounds(cost.c[t], (double)(tiles_of(p, t) * s.ns), s.kper, s.kper);
    if (us < least) least = us, best = t;
  }
  return best;
}

// Forward sums of up to 512 by the tiles for them, where there is more than one round of those:
// S256 unless S128 has fewer outputs past the end. Before and with them, with gelu, bias and
// checkpoint; and with bias and residual, fp16: 65536 x 256 -> 1024 104 -> 91 us, 100 -> 87;
// 44017 x 200 -> 700 70 -> 56, 90 -> 49; 100000 x 104 -> 6448 1026 -> 987, 847 -> 847; 30000 x 333
// -> 1111 98 -> 89, 140 -> 116; 16384 x 512 -> 2048 69 -> 66, 58 -> 58. One round of 8192 x 256 ->
// 2048 29 -> 29, 24.5 -> 23; sums of 768 (16384 -> 4096) 156 -> 160, 144 -> 153.
Shape for_short_sums(const Shape &s, const Need &p) {
  if (p.K > 512 || s.ns > 1 || (s.tile != kT128 && s.tile != kT256)) return s;
  const bool wide = up(p.M, 256) == up(p.M, 128);
  const int64_t n = ((p.N + 127) / 128) * (wide ? up(p.M, 256) / 256 : up(p.M, 128) / 128);
  return n > 256 * (wide ? 2 : 3) ? Shape{wide ? kS256 : kS128, s.ns, s.kper} : s;
}

struct Plan {
  int64_t rows, in, out, in8, out8, K;   // K: columns of x and w as the products read them
  bool narrow;                           // fewer than 8: padded copies
  Shape s1, s2, s3;                      // forward, dx, dw
  int tile;                              // of the gradients
  int tlog;
  int64_t cblocks, rblocks, per;         // of the kernel that forms dz
  // workspace, bytes
  size_t xpad, wpad, p1, xu, dz, db, pdx, pdw, total;
};

// Its sizes, and the padded copies: all that the kernel of few rows needs.
struct Layout {
  size_t at = 0;
  size_t take(size_t bytes) {
    const size_t was = at;
    at += (bytes + 255) / 256 * 256;
    return was;
  }
};
Plan sizes_of(const fg_linear_desc &d, bool grad) {
  Plan p{};
  p.rows = d.rows, p.in = d.in, p.out = d.out;
  p.in8 = up(p.in, 8), p.out8 = up(p.out, 8);
  p.narrow = p.in < 8;
  p.K = std::max<int64_t>(p.in, 8);
  Layout l;
  p.wpad = l.take(p.narrow ? (size_t)p.out * 16 : 0);
  if (!grad) p.xpad = l.take(p.narrow ? (size_t)p.rows * 16 : 0);
  p.total = l.at;
  return p;
}

Plan forward_plan(const fg_linear_desc &d) {
  Plan p = sizes_of(d, false);
  const Need fwd = {p.out, p.rows, p.K};
  pick(kFwd, &fwd, 1, &p.s1);
  p.s1 = for_short_sums(p.s1, fwd);
  Layout l{p.total};
  p.p1 = l.take(p.s1.ns > 1 ? (size_t)p.s1.ns * p.rows * p.out8 * 4 : 0);
  p.total = l.at;
  return p;
}

// Of the gradients' products a call wants these.
enum { kDx = 1, kDw = 2, kBoth = 3 };
// Both are one launch, with one tile; each alone in the same parts, for the same bits.
void gradient_plans(const fg_linear_desc &d, Plan (&out)[3]) {
  Plan p = sizes_of(d, true);
  const Need need[2] = {{p.in, p.rows, p.out8}, {p.in, p.out, p.rows}};
  Shape s[2] = {};
  pick(kBwd, need, 2, s);
  p.s2 = s[0], p.s3 = s[1];
  p.tlog = 0;
  while (p.tlog < 6 && (8 << p.tlog) < p.out8) ++p.tlog;
  p.cblocks = (p.out8 + (8 << p.tlog) - 1) / (8 << p.tlog);
  const int64_t teams = 256 >> p.tlog;
  p.rblocks = std::max<int64_t>(
      1, std::min<int64_t>((p.rows + 4 * teams - 1) / (4 * teams), 2048 / p.cblocks));
  p.per = up((std::max<int64_t>(p.rows, 1) + p.rblocks - 1) / p.rblocks, 4 * teams);
  p.rblocks = std::max<int64_t>(1, (p.rows + p.per - 1) / p.per);
  Layout l{p.total};
  p.xu = l.take((size_t)p.rows * p.in8 * 2);
  p.dz = l.take(d.act != FG_ACT_NONE || p.out % 8 ? (size_t)p.rows * p.out8 * 2 : 0);
  p.db = l.take((size_t)p.rblocks * p.out8 * 4);
  for (int want = kDx; want <= kBoth; ++want) {
    Plan &q = out[want - 1] = p;
    Layout own = l;
    q.tile = want == kBoth ? s[0].tile : tile_for(kBwd, need[want - 1], s[want - 1]);
    q.pdx = own.take(want & kDx && p.s2.ns > 1 ? (size_t)p.s2.ns * p.rows * p.in8 * 4 : 0);
    q.pdw = own.take(want & kDw && p.s3.ns > 1 ? (size_t)p.s3.ns * p.out * p.in8 * 4 : 0);
    q.total = own.at;
  }
}

// Functions of the descriptor alone, remembered for a few of them by each host thread: a call
// asks for its plan twice, and a look at every tile takes longer than a launch. One place holds
// both passes of a layer, each found when it is first asked for.
struct Plans {
  fg_linear_desc d;
  bool used, fwd, grad;
  Plan f, g[3];       // forward; dx, dw, both
  size_t grad_bytes;  // workspace of any of the latter
};
Plans &plans_of(const fg_linear_desc &d) {
  constexpr int kPlans = 32;
  static thread_local Plans kept[kPlans] = {};
  static thread_local unsigned next = 0;
  for (Plans &e : kept)
    if (e.used && !memcmp(&e.d, &d, sizeof(d))) return e;
  Plans &e = kept[next++ % kPlans];
  e.d = d;
  e.used = true, e.fwd = e.grad = false;
  return e;
}
const Plan &fwd_plan(const fg_linear_desc &d) {
  Plans &e = plans_of(d);
  if (!e.fwd) e.f = forward_plan(d), e.fwd = true;
  return e.f;
}
const Plans &grad_plans(const fg_linear_desc &d) {
  Plans &e = plans_of(d);
  if (!e.grad) {
    gradient_plans(d, e.g);
    e.grad_bytes = std::max({e.g[0].total, e.g[1].total, e.g[2].total});
    e.grad = true;
  }
  return e;
}

#define FG_TRY(x)                      \
  do {                                 \
    const hipError_t e_ = (x);         \
    if (e_ != hipSuccess) return e_;   \
  } while (0)

#define FG_LINEAR_TILE(FN, TS, tile, bf, ...)                                              \
  ((tile) == kT128D  ? ((bf) ? FN<Bf16<P128D>>(__VA_ARGS__) : FN<P128D>(__VA_ARGS__))       \
   : (tile) == kT256 ? ((bf) ? FN<Bf16<TS::T256>>(__VA_ARGS__) : FN<TS::T256>(__VA_ARGS__)) \
   : (tile) == kT128 ? ((bf) ? FN<Bf16<P128>>(__VA_ARGS__) : FN<P128>(__VA_ARGS__))         \
                     : ((bf) ? FN<Bf16<P64>>(__VA_ARGS__) : FN<P64>(__VA_ARGS__)))

template <class P>
hipError_t launch_fwd(FwdArgs a, int ns, hipStream_t st) {
  a.ntile = (a.e.out + P::TM - 1) / P::TM;
  const TileMap tm = tile_map((a.rows + P::TN - 1) / P::TN, a.ntile, ns);
  hipLaunchKernelGGL(linear_fwd_kernel<P>, dim3(8 * tm.per), dim3(P::NT), 0, st, a, tm);
  return hipGetLastError();
}

hipError_t launch_fwd_of(const Shape &s, bool bf, const FwdArgs &a, hipStream_t st) {
  if (s.tile == kS256)
    return bf ? launch_fwd<Bf16<S256>>(a, s.ns, st) : launch_fwd<S256>(a, s.ns, st);
  if (s.tile == kS128)
    return bf ? launch_fwd<Bf16<S128>>(a, s.ns, st) : launch_fwd<S128>(a, s.ns, st);
  return FG_LINEAR_TILE(launch_fwd, FwdTiles, s.tile, bf, a, s.ns, st);
}

template <bool BF, class F>
hipError_t launch_few_of(const FwdArgs &a, hipStream_t st) {
  hipLaunchKernelGGL((linear_few_kernel<BF, F>), dim3((uint32_t)((a.e.out + F::OUT - 1) / F::OUT)),
                     dim3(F::NT), 0, st, a);
  return hipGetLastError();
}
template <bool BF>
hipError_t launch_few(const FwdArgs &a, hipStream_t st) {
  // Outputs of a workgroup: at most some 2 workgroups a CU, and no more of them than fill the
  // chip. 1 row of 2048 -> 2048 by 8, 16, 32, 64: 4.5, 4.4, 5.3, 6.1 us; of 4096 -> 4096 12.0,
  // 9.2, 10.4, 13.9; of 2048 -> 8192 14.6, 10.6, 9.2, 9.7; of 2048 -> 16384 32: 16.8, 64: 15.6.
  const int out = a.e.out;
  if (a.rows <= 16)
    return out <= 2048   ? launch_few_of<BF, Few<1, 1, 8>>(a, st)
           : out <= 4096 ? launch_few_of<BF, Few<2, 1, 8>>(a, st)
           : out <= 8192 ? launch_few_of<BF, Few<4, 1, 4>>(a, st)
                         : launch_few_of<BF, Few<8, 1, 4>>(a, st);
  if (a.rows <= 32)
    return out <= 2048   ? launch_few_of<BF, Few<1, 2, 8>>(a, st)
           : out <= 4096 ? launch_few_of<BF, Few<2, 2, 8>>(a, st)
           : out <= 8192 ? launch_few_of<BF, Few<4, 2, 4>>(a, st)
                         : launch_few_of<BF, Few<8, 2, 4>>(a, st);
  return out <= 2048   ? launch_few_of<BF, Few<1, 4, 4>>(a, st)
         : out <= 4096 ? launch_few_of<BF, Few<2, 4, 4>>(a, st)
                       : launch_few_of<BF, Few<4, 4, 4>>(a, st);  // (up to 8192)
}

template <class P>
hipError_t launch_products(ProdArgs dx, int nsx, ProdArgs dw, int nsw, const SumArgs &sum,
                           hipStream_t st) {
  dx.ntile = (int32_t)((dx.N + P::TN - 1) / P::TN);
  dw.ntile = (int32_t)((dw.N + P::TN - 1) / P::TN);
  const TileMap none{1, 1, 0, 0, kOutputMajor};
  const TileMap tx = nsx ? tile_map((dx.M + P::TM - 1) / P::TM, dx.ntile, nsx) : none;
  const TileMap tw = nsw ? tile_map((dw.M + P::TM - 1) / P::TM, dw.ntile, nsw) : none;
  const int dx_first = !nsw || (nsx && dx.kper >= dw.kper);
  const int both = 8 * (tx.per + tw.per), sums = sum.out ? (sum.cols + 15) / 16 : 0;
  hipLaunchKernelGGL(linear_products_kernel<P>, dim3(both + sums), dim3(P::NT), 0, st, dx, tx, dw,
                     tw, sum, 8 * (dx_first ? tx.per : tw.per), both, dx_first);
  return hipGetLastError();
}

hipError_t launch_products_of(int tile, bool bf, const ProdArgs &dx, int nsx, const ProdArgs &dw,
                              int nsw, const SumArgs &sum, hipStream_t st) {
  if (tile == kS256)
    return bf ? launch_products<Bf16<S256>>(dx, nsx, dw, nsw, sum, st)
              : launch_products<S256>(dx, nsx, dw, nsw, sum, st);
  return FG_LINEAR_TILE(launch_products, BwdTiles, tile, bf, dx, nsx, dw, nsw, sum, st);
}

template <int DT, int ACT, int KEPT>
hipError_t launch_dz_of(const DzArgs &a, const act8::Args &x, hipStream_t st) {
  const dim3 grid(a.blocks + act8::blocks_of(x)), block(256);
  if (a.out % 8 == 0)
    hipLaunchKernelGGL((linear_dz_kernel<DT, ACT, KEPT, true>), grid, block, 0, st, a, x);
  else
    hipLaunchKernelGGL((linear_dz_kernel<DT, ACT, KEPT, false>), grid, block, 0, st, a, x);
  return hipGetLastError();
}
template <int DT>
hipError_t launch_dz(const DzArgs &a, const act8::Args &x, hipStream_t st) {
  const bool kept = a.packed.codes != nullptr;
  if (a.act == FG_ACT_NONE) return launch_dz_of<DT, FG_ACT_NONE, 0>(a, x, st);
  if (a.act == FG_ACT_RELU)
    return kept ? launch_dz_of<DT, FG_ACT_RELU, 1>(a, x, st)
                : launch_dz_of<DT, FG_ACT_RELU, 0>(a, x, st);
  return kept ? launch_dz_of<DT, FG_ACT_GELU, 1>(a, x, st)
              : launch_dz_of<DT, FG_ACT_GELU, 0>(a, x, st);
}

hipError_t pad(const uint16_t *x, int64_t ld, int64_t n, uint16_t *to, int64_t rows,
               hipStream_t st) {
  hipLaunchKernelGGL(linear_pad_kernel, dim3((uint32_t)((rows + 255) / 256)), dim3(256), 0, st, x,
                     ld, (int32_t)n, to, rows);
  return hipGetLastError();
}

}  // namespace linear

// Without a checkpoint of z to write, few rows have a kernel that splits no sums over workgroups.
size_t linear_fwd_ws_bytes(const fg_linear_desc &d, bool packed_z) {
  return linear::few_rows(d.rows, d.out) && !packed_z ? linear::sizes_of(d, false).total
                                                      : linear::fwd_plan(d).total;
}
// (a training step's workspace serves its forward pass too)
size_t linear_ws_bytes(const fg_linear_desc &d, bool grad) {
  const size_t fwd = linear_fwd_ws_bytes(d, d.act != FG_ACT_NONE);
  return grad ? std::max(fwd, linear::grad_plans(d).grad_bytes) : fwd;
}

hipError_t launch_linear_fwd(const fg_linear_desc &d, const void *x, const void *w,
                             const void *bias, const void *residual, void *y, void *z,
                             void *packed_z, void *ws, hipStream_t st) {
  using namespace linear;
  const bool few = few_rows(d.rows, d.out) && !packed_z;
  const Plan p = few ? sizes_of(d, false) : fwd_plan(d);
  uint8_t *base = static_cast<uint8_t *>(ws);
  const bool bf = d.dtype == FG_BF16;
  FwdArgs a{};
  a.w = (const uint16_t *)w, a.x = (const uint16_t *)x;
  a.w_ld = d.w_ld ? d.w_ld : p.in, a.x_ld = d.x_ld ? d.x_ld : p.in;
  if (p.narrow) {
    uint16_t *wp = (uint16_t *)(base + p.wpad), *xp = (uint16_t *)(base + p.xpad);
    FG_TRY(pad(a.w, a.w_ld, p.in, wp, p.out, st));
    FG_TRY(pad(a.x, a.x_ld, p.in, xp, p.rows, st));
    a.w = wp, a.x = xp, a.w_ld = a.x_ld = 8;
  }
  a.K = (int32_t)p.K, a.kper = p.s1.kper, a.rows = p.rows;
  Epilogue &e = a.e;
  e.bias = (const uint16_t *)bias, e.residual = (const uint16_t *)residual;
  e.y = (uint16_t *)y, e.z = (uint16_t *)z;
  const auto ld = [&](int64_t v) { return v ? v : p.out; };
  e.y_ld = ld(d.y_ld), e.r_ld = ld(d.r_ld), e.z_ld = ld(d.z_ld);
  if (packed_z) e.packed = rows::packed_at(packed_z, p.rows, p.out);
  e.out = (int32_t)p.out, e.act = d.act;
  if (few)
    return bf ? launch_few<true>(a, st) : launch_few<false>(a, st);
  a.Mq = (int32_t)p.out8, a.pstride = p.rows * p.out8;
  const bool split = p.s1.ns > 1;
  if (split) a.part = (float *)(base + p.p1);
  FG_TRY(launch_fwd_of(p.s1, bf, a, st));
  if (!split) return hipSuccess;
  const JoinFwd j = {a.part, a.pstride, p.rows, p.s1.ns, a.Mq, (int32_t)up(p.out, 32), e};
  const dim3 grid((uint32_t)((p.rows * (j.wide / 8) + 255) / 256)), block(256);
  if (bf)
    hipLaunchKernelGGL(linear_join_fwd_kernel<FG_BF16>, grid, block, 0, st, j);
  else
    hipLaunchKernelGGL(linear_join_fwd_kernel<FG_F16>, grid, block, 0, st, j);
  return hipGetLastError();
}

hipError_t launch_linear_bwd(const fg_linear_desc &d, const void *dy, const void *x,
                             const void *packed_x, const void *w, const void *z,
                             const void *packed_z, void *dx, void *dw, void *dbias,
                             int32_t *flag, void *ws, hipStream_t st) {
  using namespace linear;
  const Plan p = grad_plans(d).g[((dx && !dw) ? kDx : (dw && !dx) ? kDw : kBoth) - 1];
  uint8_t *base = static_cast<uint8_t *>(ws);
  const bool bf = d.dtype == FG_BF16;
  const auto ld = [&](int64_t v, int64_t width) { return v ? v : width; };

  // dz, and the parts of its columns' sums
  DzArgs z1{};
  z1.dy = (const uint16_t *)dy, z1.dy_ld = ld(d.y_ld, p.out);
  z1.z = (const uint16_t *)z, z1.z_ld = ld(d.z_ld, p.out);
  if (packed_z) z1.packed = rows::packed_at(packed_z, p.rows, p.out);
  const bool formed = (dx || dw) && (d.act != FG_ACT_NONE || p.out % 8);
  z1.dz = formed ? (uint16_t *)(base + p.dz) : nullptr;
  z1.part = dbias ? (float *)(base + p.db) : nullptr;
  z1.rows = p.rows, z1.per = p.per;
  z1.out = (int32_t)p.out, z1.Mp = (int32_t)p.out8, z1.act = d.act, z1.tlog = p.tlog;
  z1.cblocks = (uint32_t)p.cblocks, z1.blocks = (uint32_t)(p.cblocks * p.rblocks);
  const bool unpacked = dw && packed_x && p.rows, first = (formed || dbias) && p.rows;
  const fg_act8_desc u = {p.rows, p.in, p.in8, d.dtype};
  if (first) {
    act8::Args au{};
    if (unpacked) au = act8::args_of(u, nullptr, base + p.xu, const_cast<void *>(packed_x));
    FG_TRY((bf ? launch_dz<FG_BF16> : launch_dz<FG_F16>)(z1, au, st));
  } else if (unpacked) {
    FG_TRY(launch_act8(u, nullptr, base + p.xu, const_cast<void *>(packed_x), st));
  }
  SumArgs sum{};
  if (dbias)
    sum = {z1.part, (uint16_t *)dbias, (int32_t)(p.rows ? p.rblocks : 0), (int32_t)p.out8,
           (int32_t)p.out, flag};
  if (dbias && !dw && !(dx && p.rows)) {  // no product's launch to join
    const dim3 grid((uint32_t)((p.out + 15) / 16)), block(256);
    if (bf)
      hipLaunchKernelGGL(linear_sum_kernel<FG_BF16>, grid, block, 0, st, sum);
    else
      hipLaunchKernelGGL(linear_sum_kernel<FG_F16>, grid, block, 0, st, sum);
    return hipGetLastError();
  }

  ProdArgs a{}, b{};
  a.b = b.b = formed ? z1.dz : z1.dy;
  a.b_ld = b.b_ld = formed ? p.out8 : z1.dy_ld;
  a.b_cols = b.b_cols = (int32_t)p.out8;
  a.a_cols = b.a_cols = (int32_t)p.K;
  a.M = b.M = (int32_t)p.in, a.Mq = b.Mq = (int32_t)p.in8;
  JoinArgs jx{}, jw{};
  int nsx = 0, nsw = 0;
  if (dx && p.rows) {
    a.a = (const uint16_t *)w, a.a_ld = ld(d.w_ld, p.in);
    if (p.narrow) {
      uint16_t *to = (uint16_t *)(base + p.wpad);
      FG_TRY(pad(a.a, a.a_ld, p.in, to, p.out, st));
      a.a = to, a.a_ld = 8;
    }
    nsx = p.s2.ns;
    a.N = p.rows, a.K = p.out, a.kper = p.s2.kper;
    a.out_ld = ld(d.dx_ld, p.in);
    a.pstride = p.rows * p.in8;
    (nsx > 1 ? (void *&)a.part : (void *&)a.out) = nsx > 1 ? (void *)(base + p.pdx) : dx;
    jx = {a.part, a.pstride, p.rows, nsx, a.M, a.Mq, (uint16_t *)dx, a.out_ld, nullptr,
          shared_log(nsx)};
  }
  if (dw) {
    b.a = (const uint16_t *)x, b.a_ld = ld(d.x_ld, p.in);
    if (unpacked) {
      b.a = (const uint16_t *)(base + p.xu), b.a_ld = p.in8;
    }
    if (p.narrow && p.rows) {
      uint16_t *to = (uint16_t *)(base + p.xu);  // (each row onto itself where it is there)
      FG_TRY(pad(b.a, b.a_ld, p.in, to, p.rows, st));
      b.a = to, b.a_ld = 8;
    }
    nsw = p.s3.ns;
    b.N = p.out, b.K = p.rows, b.kper = p.s3.kper;
    b.out_ld = ld(d.dw_ld, p.in);
    b.pstride = p.out * p.in8;
    (nsw > 1 ? (void *&)b.part : (void *&)b.out) = nsw > 1 ? (void *)(base + p.pdw) : dw;
    b.flag = flag;
    jw = {b.part, b.pstride, p.out, nsw, b.M, b.Mq, (uint16_t *)dw, b.out_ld, flag,
          shared_log(nsw)};
  }
  if (!nsx && !nsw) return hipSuccess;
  FG_TRY(launch_products_of(p.tile, bf, a, nsx, b, nsw, sum, st));
  const auto blocks = [&](int64_t n, const JoinArgs &j) {
    const int wide = 256 >> j.slog;
    return (n * (p.in8 / 8) + wide - 1) / wide;
  };
  const int64_t bx = nsx > 1 ? blocks(p.rows, jx) : 0, bw = nsw > 1 ? blocks(p.out, jw) : 0;
  if (!bx && !bw) return hipSuccess;
  const dim3 grid((uint32_t)(bx + bw)), block(256);
  if (bf)
    hipLaunchKernelGGL(linear_join_kernel<FG_BF16>, grid, block, 0, st, jx, jw, (int)bx);
  else
    hipLaunchKernelGGL(linear_join_kernel<FG_F16>, grid, block, 0, st, jx, jw, (int)bx);
  return hipGetLastError();
}

}  // namespace fg
