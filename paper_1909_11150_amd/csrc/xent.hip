// Softmax cross entropy of a linear head, with its gradients, over any number of
// classes; the logits are never stored.
//
//   l = h W^T,  lse = log sum_v exp(l_v),  loss = w (lse - l_target)
//   G = w (exp(l - lse) - onehot),  dh = c G W,  dW = c G^T h
//
// Rows whose target is no class (or whose weight is 0) are masked. The live rows
// are first copied one after another into the workspace, so masked rows cost no
// matrix work, and whatever they hold, infinities and NaN too, reaches nothing.
//
// Products run on MFMA tiles fed by LDS DMA (dma_pipe.h), in pieces of the live
// rows and tiles of the classes:
//   logits   one tile of l in the accumulators, classes x rows, so a row's classes
//            lie in one lane's registers (and its neighbour's half): the tile's
//            maximum m and sum of exp(l - m) per row are stored; for gradients also
//            2^15 exp(l - m) in fp16, the only trace of a logit in memory, for the
//            rows of one piece;
//   softmax  joins a row's tiles into lse, and turns the numerators into 2^15 G in
//            the features' type, in place;
//   product  dh = G W and dW = G^T h, whose strided operands are read with
//            transposing LDS reads; the sum over the classes (rows) is split where
//            there are few tiles, and joined in a fixed order.
// The gradients thus take three products of rows x hidden x classes; without the
// numerators they would take four.
//
// Up to 256 classes (pixels' classes) one tile holds them all: a single kernel goes
// from the features to losses and G, and rows stay where they are, masked ones being
// left out by the DMA (an offset out of range reads zeros). Up to 64 rows, and up to 256 of
// small calls, they stay in place too, and no kernel runs ahead to find the live ones. Sums
// of at most 64 terms (dW of up to 64 rows, dh of up to 64 classes) have a kernel of their
// own, bound by writing them.
//
// Measured (MI355X, fp16 unless noted; rates count the live rows' three products, or
// one for losses alone): 8192 x 4096 x 131072 (rows, hidden, classes) bf16 with
// gradients 20.6 ms (1.22 PFLOP/s; the kernels' clock is held to 1.6 - 1.85 GHz by the
// board's power); 2048 x 1024 x 32000 0.45 ms (0.85); losses of 4096 x 2048 x 32768
// 0.45 ms (1.09) and of 48 x 2048 x 65536 bf16 56 us (4.8 TB/s); gradients of
// 65536 x 512 x 12 54 us (2.4 TB/s).
#include <algorithm>

#include "tiles.h"

namespace fg {
namespace xent {

using namespace tiles;

constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;
// Numerators and G are held times 2^kUp: the largest is then 2^15 (between 2^14 and 2^15
// where rows have weights), within fp16, and values down to 2^-29 of that keep all their
// bits (2^-14 otherwise).
constexpr int kUp = 15;
constexpr int kTickets = 64;    // softmax workgroups up to which the last one sums up
constexpr int kFew = 1024;      // rows up to which the softmax kernel takes 4 per workgroup
constexpr int kCount = 1024;    // rows of a workgroup of the counting kernel
constexpr int kDirect = 8192;   // rows up to which there is none
constexpr int kWide = 1 << 27;  // rows beyond which a workgroup copies 32, not 16

// The largest, 8 waves of 128 x 64: 64-deep stages for the logits' operands, whose rows
// lie along the sum (whole 128-byte lines: 8192 x 4096 x 131072 in two pieces 3.48 ms a
// piece, 3.84 with 32-deep ones); 32-deep ones, five in the ring, for the products',
// whose rows lie across it (7.0 ms, 7.4 with 64-deep ones). Smaller tiles twice per CU
// (256 x 128) took 4.8 and 8.8 ms, 4 waves of 128 x 128 3.8 and 8.0.
struct LogitTiles {
  using T256 = Pipe<64, 2, 2, 4, 256, 256>;
};
struct ProdTiles {
  using T256 = Pipe<32, 5, 2, 4, 256, 256>;
};
// Up to 32 and 64 classes, by 128 rows: bound by the features' stream. With a workgroup
// per CU or less (kSparse rows) a deep ring keeps it going; with more, more workgroups
// per CU and a ring of two: 8192 x 2048 x 20 losses 14.8 us (21.6 with two stages), 262144 x
// 64 x 12 losses 23.5 (29.4 with four), gradients of 65536 x 512 x 12 46.8 (48.3).
using PSparse32 = Pipe<64, 4, 1, 4, 32, 128>;
using PSparse64 = Pipe<64, 3, 1, 4, 64, 128>;
using PClass32 = Pipe<64, 2, 1, 4, 32, 128>;
using PClass64 = Pipe<64, 2, 1, 4, 64, 128>;
constexpr int kSparse = 256 * 128;
// 65 .. 128 and .. 256 classes by 64 rows while those tiles fit the chip at once, two to a
// CU (72 and 80 KiB of LDS each): 8543 x 1024 x 86 losses 13.6 us (17.8 by 128 rows), 32768 x
// 1024 x 100 18.4 (21.0), 16000 x 1024 x 200 18.7 (28.9 by 256 rows), 17000, 24000 and 32768 x
// 1024 x 200 20.9, 22.3 and 24.2 (29); beyond that 40000 x 1024 x 100 25.3, not 21.7, and
// 40000 x 1024 x 200 34.8, not 29.7.
using PHalf128 = Pipe<64, 3, 2, 2, 128, 64>;
using PHalf256 = Pipe<64, 2, 4, 2, 256, 64>;
constexpr int kHalf = 512 * 64;

// What the first kernels find out, read by the others.
struct Found {
  int32_t live;     // rows
  int32_t wexp;     // weights are taken times 2^wexp: the largest in (2^14, 2^15]
  float mult;       // G W and G^T h times this are the gradients
  float wsum;
  uint32_t ticket;  // workgroups done (losses only)
};

// ---- live rows -----------------------------------------------------------------
struct RowArgs {
  const uint16_t *h;
  int64_t h_ld;
  const int32_t *target;
  const float *weight;
  int32_t T, H, Hp, V;
  int32_t nb;            // workgroups of the counting kernel; 0: the copies count
  double scale;
  int32_t mean;
  int32_t *count;        // live rows per counted block, then before it
  double *wsum;
  float *wmax;
  Found *found;
  int32_t *idx, *ctarget;
  float *cweight;
  uint64_t *mark;        // a bit per row: live (up to 256 classes)
  uint16_t *hc;
  float *loss, *lse;
  uint16_t *dh;          // null: no gradients of the features
  int64_t dh_ld;
};

__device__ __forceinline__ bool live_row(const RowArgs &a, int r, float &w) {
  w = 1.f;
  if (r >= a.T || (uint32_t)a.target[r] >= (uint32_t)a.V) return false;
  if (a.weight) w = a.weight[r];
  return w != 0.f;
}

template <class T>
__device__ __forceinline__ T wave_sum(T v) {
#pragma unroll
  for (int o = 32; o; o >>= 1) v += __shfl_xor(v, o);
  return v;
}
__device__ __forceinline__ float wave_max(float v) {
#pragma unroll
  for (int o = 32; o; o >>= 1) v = fmaxf(v, __shfl_xor(v, o));
  return v;
}

__device__ __forceinline__ Found make_found(int mean, double scale, int live, double sum,
                                            float mx) {
  // no live row, or weights that cancel: a mean of nothing has no gradient
  const double den = mean ? sum : 1.0;
  // Weights are brought up by a power of two, which rounds nothing and reaches the smallest
  // (the reciprocal of one below 2^-128 is infinite). An infinite one leaves no gradient a
  // number.
  int e = 0;
  if (mx > 0.f && frexpf(mx, &e) == 0.5f) --e;  // mx in (2^(e - 1), 2^e]
  const int wexp = kUp - e;
  const double mult = den != 0.0 ? ldexp(scale / den, -wexp) : 0.0;
  return {live, wexp, mx == INFINITY ? NAN : (float)mult, (float)sum, 0};
}
__device__ __forceinline__ void put_found(const RowArgs &a, int live, double sum, float mx) {
  *a.found = make_found(a.mean, a.scale, live, sum, mx);
}

// Up to 64 rows: they stay in place, and every kernel finds out by itself, a row per
// lane, what the kernels above find for more.
struct Tiny {
  const int32_t *target;
  const float *weight;
  int32_t T, V, mean;  // T = 0: more rows
  double scale;
};
__device__ __forceinline__ Found tiny_found(const Tiny &t, uint64_t &mark) {
  const int r = threadIdx.x & 63;
  float w = 1.f;
  bool on = r < t.T && (uint32_t)t.target[r] < (uint32_t)t.V;
  if (on && t.weight) w = t.weight[r];
  on = on && w != 0.f;
  mark = __ballot(on);
  const int live = __popcll(mark);
  if (!t.weight) return make_found(t.mean, t.scale, live, (double)live, live ? 1.f : 0.f);
  return make_found(t.mean, t.scale, live, wave_sum(on ? (double)w : 0.0),
                    wave_max(on ? fabsf(w) : 0.f));
}

// Some more rows in place: a wave of the logits' kernel finds it for the others.
constexpr int kWave = 256;  // rows
__device__ __forceinline__ void find_rows(const Tiny &t, int lane, uint64_t *mark, Found *found) {
  int live = 0;
  double sum = 0;
  float mx = 0.f;
#pragma unroll
  for (int k = 0; k < kWave / 64; ++k) {
    const int r = 64 * k + lane;
    float w = 1.f;
    bool on = r < t.T && (uint32_t)t.target[r] < (uint32_t)t.V;
    if (on && t.weight) w = t.weight[r];
    on = on && w != 0.f;
    const uint64_t m = __ballot(on);
    if (lane == 0 && 64 * k < t.T) mark[k] = m;
    live += __popcll(m);
    if (on) {
      sum += w;
      mx = fmaxf(mx, fabsf(w));
    }
  }
  sum = wave_sum(sum);
  mx = wave_max(mx);
  if (lane == 0) *found = make_found(t.mean, t.scale, live, sum, mx);
}

// Unweighted rows of few classes: the kernel that finds the losses also counts each
// tile's live rows, and those after it add the counts up, every workgroup by itself up to
// kTiles tiles, beyond by one workgroup in a launch between. With the line at 256, 512 and
// 1024 tiles, gradients of 12 classes: 32769 x 256 25.7, 23.5 and 24.2 us, 65536 x 512 47.0,
// 46.0 and 46.0, 65537 x 512 46.6, 47.0 and 45.1, 131073 x 256 48.2, 48.4 and 49.0 (51.6 at
// 2048).
constexpr int kTiles = 512;
struct Counts {
  const int32_t *live;
  int32_t n, mean;  // n = 0: not so
  double scale;
};
// The counts, a few per lane: loaded well before they are used.
struct Counted {
  int c[kTiles / 64];
  __device__ __forceinline__ void load(const Counts &a) {
#pragma unroll
    for (int k = 0; k < kTiles / 64; ++k) {
      const int i = 64 * k + (threadIdx.x & 63);
      c[k] = i < a.n ? a.live[i] : 0;
    }
  }
  __device__ __forceinline__ Found found(const Counts &a) const {
    int n = 0;
#pragma unroll
    for (int k = 0; k < kTiles / 64; ++k) n += c[k];
    n = wave_sum(n);
    return make_found(a.mean, a.scale, n, (double)n, 1.f);
  }
};

// Live rows, their weights' sum and largest magnitude, per block of 1024 rows; the
// totals too where there is one block.
__global__ __launch_bounds__(256) void xent_count_kernel(RowArgs a) {
  __shared__ double ws[4];
  __shared__ float wm[4];
  __shared__ int cn[4];
  int n = 0;
  double sum = 0;
  float mx = 0.f;
#pragma unroll
  for (int k = 0; k < kCount / 256; ++k) {
    float w;
    const int r = blockIdx.x * kCount + k * 256 + threadIdx.x;
    const bool on = live_row(a, r, w);
    const uint64_t mark = __ballot(on);
    if (a.mark && (threadIdx.x & 63) == 0 && r < a.T) a.mark[r >> 6] = mark;
    if (on) {
      ++n;
      sum += w;
      mx = fmaxf(mx, fabsf(w));
    }
  }
  n = wave_sum(n);
  sum = wave_sum(sum);
  mx = wave_max(mx);
  if ((threadIdx.x & 63) == 0) {
    const int k = threadIdx.x >> 6;
    cn[k] = n, ws[k] = sum, wm[k] = mx;
  }
  __syncthreads();
  if (threadIdx.x == 0) {
    n = cn[0] + cn[1] + cn[2] + cn[3];
    sum = (ws[0] + ws[1]) + (ws[2] + ws[3]);
    mx = fmaxf(fmaxf(wm[0], wm[1]), fmaxf(wm[2], wm[3]));
    a.count[blockIdx.x] = n;
    a.wsum[blockIdx.x] = sum;
    a.wmax[blockIdx.x] = mx;
    if (gridDim.x == 1) put_found(a, n, sum, mx);
  }
}

// One workgroup: counts become the live rows before each block; the totals.
__global__ __launch_bounds__(1024) void xent_scan_kernel(RowArgs a) {
  __shared__ double ws[16];
  __shared__ float wm[16];
  __shared__ int cn[16];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  int base = 0;
  double sum = 0;
  float mx = 0.f;
  for (int b0 = 0; b0 < a.nb; b0 += 1024) {
    const int b = b0 + threadIdx.x;
    const int c = b < a.nb ? a.count[b] : 0;
    if (b < a.nb) {
      sum += a.wsum[b];
      mx = fmaxf(mx, a.wmax[b]);
    }
    int incl = c;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
      const int v = __shfl_up(incl, o);
      if (lane >= o) incl += v;
    }
    __syncthreads();
    if (lane == 63) cn[wave] = incl;
    __syncthreads();
    int before = base;
    for (int k = 0; k < wave; ++k) before += cn[k];
    if (b < a.nb) a.count[b] = before + incl - c;
    for (int k = 0; k < 16; ++k) base += cn[k];
  }
  sum = wave_sum(sum);
  mx = wave_max(mx);
  if (lane == 0) ws[wave] = sum, wm[wave] = mx;
  __syncthreads();
  if (threadIdx.x == 0) {
    for (int k = 1; k < 16; ++k) {
      sum += ws[k];
      mx = fmaxf(mx, wm[k]);
    }
    put_found(a, base, sum, mx);
  }
}

// Copies live rows to their places, in order; results of masked rows are written
// here. (What stands after the last live row is never read into a result.) 4 R rows
// per workgroup. Up to kDirect rows every workgroup counts the live ones before its
// own by itself, and one more finds the totals: two launches fewer.
template <int R>
__global__ __launch_bounds__(256) void xent_rows_kernel(RowArgs a) {
  __shared__ int cn[4];
  __shared__ double ws[4];
  __shared__ float wm[4];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int r0 = blockIdx.x * 4 * R, blk = a.nb ? r0 / kCount : 0;
  const bool totals = r0 >= a.T;
  // live rows before r0, of this counted block where blocks are counted
  int n = 0;
  double sum = 0;
  float mx = 0.f;
  const int end = min(r0, a.T);
  constexpr int B = 8;  // loads in flight
  for (int r = blk * kCount + threadIdx.x; r < end; r += 256 * B) {
    int32_t t[B];
    float w[B];
#pragma unroll
    for (int k = 0; k < B; ++k) t[k] = a.target[min(r + 256 * k, a.T - 1)];
#pragma unroll
    for (int k = 0; k < B; ++k) w[k] = a.weight ? a.weight[min(r + 256 * k, a.T - 1)] : 1.f;
#pragma unroll
    for (int k = 0; k < B; ++k) {
      const bool on = r + 256 * k < end && (uint32_t)t[k] < (uint32_t)a.V && w[k] != 0.f;
      n += on;
      if (totals && on) {
        sum += w[k];
        mx = fmaxf(mx, fabsf(w[k]));
      }
    }
  }
  n = wave_sum(n);
  if (lane == 0) cn[wave] = n;
  if (totals) {
    sum = wave_sum(sum);
    mx = wave_max(mx);
    if (lane == 0) ws[wave] = sum, wm[wave] = mx;
    __syncthreads();
    if (threadIdx.x == 0)
      put_found(a, cn[0] + cn[1] + cn[2] + cn[3], (ws[0] + ws[1]) + (ws[2] + ws[3]),
                fmaxf(fmaxf(wm[0], wm[1]), fmaxf(wm[2], wm[3])));
    return;
  }
  __syncthreads();
  const int before = (a.nb ? a.count[blk] : 0) + cn[0] + cn[1] + cn[2] + cn[3];
  float w = 0.f;
  const bool mine = lane < 4 * R && live_row(a, r0 + lane, w);
  const uint64_t mask = __ballot(mine);
  const int place = before + __popcll(mask & ((1ull << lane) - 1));
  if (wave == 0 && lane < 4 * R) {
    const int r = r0 + lane;
    if (mine) {
      a.idx[place] = r;
      a.ctarget[place] = a.target[r];
      a.cweight[place] = w;
    } else if (r < a.T) {
      a.loss[r] = 0.f;
      if (a.lse) a.lse[r] = 0.f;
    }
  }
#pragma unroll
  for (int j = 0; j < R; ++j) {
    const int k = 4 * j + wave, r = r0 + k, to = __shfl(place, k);
    const bool on = mask >> k & 1;
    const uint16_t *src = a.h + (int64_t)r * a.h_ld;
    for (int c = 8 * lane; on && c < a.H; c += 512)
      *reinterpret_cast<u32x4 *>(a.hc + (size_t)to * a.Hp + c) = row8(src, c, a.H);
    if (!on && a.dh && r < a.T)
      for (int c = 8 * lane; c < a.H; c += 512)
        put8(a.dh + (int64_t)r * a.dh_ld, c, a.H, u32x4{0, 0, 0, 0});
  }
}

// Rows of fewer than 8 elements, padded with zeros to 8.
__global__ __launch_bounds__(256) void xent_pad_kernel(const uint16_t *w, int64_t ld, int32_t H,
                                                       uint16_t *wc, int32_t V) {
  const int r = blockIdx.x * 256 + threadIdx.x;
  if (r < V) *reinterpret_cast<u32x4 *>(wc + (size_t)r * 8) = row8(w + r * ld, 0, H);
}

// ---- logits ------------------------------------------------------------------------
struct LogitArgs {
  const uint16_t *w;
  int64_t w_ld;
  int32_t wh;             // elements of a row (of w and of hc), at least 8
  int32_t V;
  const uint16_t *hc;     // the piece's first row
  int32_t Hp;             // its stride
  Found *found;
  int32_t place;          // rows in place, all Tc of them
  Tiny all;               // T > 0: the first tile finds the live ones
  uint64_t *mark;
  int32_t stream;         // one tile of rows: each tile of classes begins its sum elsewhere
  int32_t row0, Tc;       // first live row of the piece, rows it may have
  const int32_t *ctarget;
  uint16_t *e;            // [Tc][Vp] numerators, fp16 (STORE)
  int32_t Vp;
  float2 *stats;          // [tile of classes][Tc]: numerators times 2^x are exp(l); sum
  float *tlogit;          // [Tc]
};

// exp(l) 2^scale_of(m) is the numerator of l in a tile whose largest logit is m (all
// -inf, where no class of a tile is possible: any finite scale gives zeros).
__device__ __forceinline__ float scale_of(float m) {
  return m == -INFINITY ? 15.f : 15.f - m * kLog2e;
}

__device__ __forceinline__ int piece_rows(const Found *f, int row0, int Tc) {
  return min(max(f->live - row0, 0), Tc);
}

// Classes past the last one, of a wave's classes from v0 on: logit -inf.
template <class P>
__device__ __forceinline__ void no_class(f32x16 (&acc)[P::FM][P::FN], int v0, int V, int lane) {
#pragma unroll
  for (int i = 0; i < P::FM; ++i)
#pragma unroll
    for (int v = 0; v < 16; ++v)
      if (v0 + 32 * i + 8 * (v >> 2) + 4 * (lane >> 5) + (v & 3) >= V)
#pragma unroll
        for (int j = 0; j < P::FN; ++j) acc[i][j][v] = -INFINITY;
}

template <class P>
__host__ __device__ __forceinline__ int stages(int wh) {
  return (wh + P::BK - 1) / P::BK;
}

// The logit of class t (counted from this wave's first) of this lane's row, if the lane
// holds it: selected, one store at the caller's (a branch per element spills its masks).
template <class P>
__device__ __forceinline__ bool pick(const f32x16 (&acc)[P::FM][P::FN], int j, int t, int lane,
                                     float &x) {
  x = 0.f;
#pragma unroll
  for (int i = 0; i < P::FM; ++i)
#pragma unroll
    for (int v = 0; v < 16; ++v)
      x = t - 4 * (lane >> 5) == 32 * i + 8 * (v >> 2) + (v & 3) ? acc[i][j][v] : x;
  return t >= 0 && t < P::WM && (t >> 2 & 1) == lane >> 5;
}

// Stages whose order may turn: all, or all but the last, which `fix` below has to find among
// the pipeline's last ones where the width is no multiple of 8.
template <class P>
__device__ __forceinline__ int turning(int wh) {
  return stages<P>(wh) - (wh % 8 != 0);
}

// A tile of logits: oa, ob: this lane's first chunks in the weights' and the
// features' buffers. TURN: the sum begins at stage `first` of the turning ones and comes
// round to it.
template <class P, bool TURN>
__device__ __forceinline__ void logit_sums(f32x16 (&acc)[P::FM][P::FN], const Ring &R,
                                           __amdgpu_buffer_rsrc_t rs_w,
                                           __amdgpu_buffer_rsrc_t rs_h,
                                           const unsigned (&oa)[P::PA],
                                           const unsigned (&ob)[P::PB], const KmSlot<P::PA> &as,
                                           const KmSlot<P::PB> &bs, int wh, int first, int wave,
                                           int wm0, int wn0, int lane) {
  constexpr int PA = P::PA, PB = P::PB, BK = P::BK;
  const int nst = stages<P>(wh), turn = turning<P>(wh);
  // offsets in the last stage: its last chunk may begin before its place, and chunks
  // past the end are zeros. Selected, not branched to: the main loop's scheduling
  // regions span whole steps (a branch cost 3.5% of the largest product).
  const int kl = (nst - 1) * BK;
  auto tail = [&](unsigned o, int coff) __attribute__((always_inline)) {
    return kl + coff < wh ? o + 2u * (chunk_at(kl + coff, wh) - coff) : kOOB;
  };
  unsigned la[PA], lb[PB];
#pragma unroll
  for (int jj = 0; jj < PA; ++jj) la[jj] = tail(oa[jj], as.coff[jj]);
#pragma unroll
  for (int jj = 0; jj < PB; ++jj) lb[jj] = tail(ob[jj], bs.coff[jj]);
  auto issue = [&](int st, int slot) __attribute__((always_inline)) {
    uint8_t *ta = R.a[slot], *tb = R.b[slot];
    const int to = st + first;
    const int at = !TURN || st >= turn ? st : to < turn ? to : to - turn;
    const bool last = at + 1 == nst;
    const unsigned k0 = 2u * BK * at;
#pragma unroll
    for (int jj = 0; jj < PB; ++jj)
      dma16(rs_h, tb + dma_dst<PB>(wave, jj), last ? lb[jj] : ob[jj] + k0);
#pragma unroll
    for (int jj = 0; jj < PA; ++jj)
      dma16(rs_w, ta + dma_dst<PA>(wave, jj), last ? la[jj] : oa[jj] + k0);
  };
  // the last chunk's repeated elements: zeros in both operands, whatever they are (called
  // in the pipeline's last stages alone: the chunk's stage is its last, turned or not)
  auto fix = [&](Frags<P> &f, int it, int ks) __attribute__((always_inline)) {
    if (wh % 8 == 0 || it + 1 != nst) return;
    const int over = (nst - 1) * BK + 16 * ks + 8 * (lane >> 5) + 8 - wh;  // 1 .. 7: that chunk
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
  zero<P>(acc);
  pipeline<P, true, true>(acc, R, nst, wm0, wn0, lane, issue, NoFold{}, fix);
}

template <class P, bool STORE>
__global__ __launch_bounds__(P::NT, P::WPE) void xent_logits_kernel(LogitArgs a, TileMap tm) {
  FG_DMA_RING(P, R);
  constexpr int PA = P::PA, PB = P::PB, BK = P::BK;
  int tx, ty, tz;  // rows, classes
  if (!find_tile(tm, blockIdx.x, (a.V + P::TM - 1) / P::TM, tx, ty, tz)) return;
  const int n0 = tx * P::TN, m0 = ty * P::TM;
  const int rows = a.place ? a.Tc : piece_rows(a.found, a.row0, a.Tc);
  if (n0 >= rows) return;
  if (a.place && blockIdx.x == 0 && threadIdx.x == 0) a.found->ticket = 0;
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int wm = wave / P::WGN, wm0 = wm * P::WM, wn0 = (wave % P::WGN) * P::WN;

  const int wrows = min(P::TM, a.V - m0);
  const __amdgpu_buffer_rsrc_t rs_w =
      rsrc(a.w + m0 * a.w_ld, (uint32_t)((wrows - 1) * a.w_ld + a.wh) * 2u);
  // (in place: to the last row's end; masked rows' logits are numbers no one reads)
  const int hrows = a.place ? min(P::TN, rows - n0) : P::TN;
  const __amdgpu_buffer_rsrc_t rs_h =
      rsrc(a.hc + (size_t)n0 * a.Hp, (uint32_t)((hrows - 1) * a.Hp + a.wh) * 2u);
  const KmSlot<PA> as = km_slots<BK, PA>(wave, lane);
  const KmSlot<PB> bs = km_slots<BK, PB>(wave, lane);
  unsigned oa[PA], ob[PB];
#pragma unroll
  for (int jj = 0; jj < PA; ++jj) oa[jj] = (unsigned)(as.row[jj] * (int)a.w_ld + as.coff[jj]) * 2u;
#pragma unroll
  for (int jj = 0; jj < PB; ++jj) ob[jj] = (unsigned)(bs.row[jj] * a.Hp + bs.coff[jj]) * 2u;
  int target[P::FN];  // the rows' targets, counted from this wave's first class
#pragma unroll
  for (int j = 0; j < P::FN; ++j) {
    const int n = n0 + wn0 + 32 * j + (lane & 31);
    target[j] = n < rows ? (int)((unsigned)a.ctarget[n] - (unsigned)(m0 + wm0)) : -1;
  }
  f32x16 acc[P::FM][P::FN];
  // With one tile of rows the weights stream from memory: where all workgroups read the
  // same part of rows of a power of two bytes, few memory channels serve them. So each
  // begins elsewhere: 48 x 2048 x 65536 73.7 -> 55.7 us (4.8 TB/s), 48 x 4096 x 65536 129
  // -> 107. (Not in the largest tiles, whose products it slows by 2%.)
  constexpr bool TURN = P::TN < 256;
  const int first =
      TURN && a.stream ? (int)(blockIdx.x % (unsigned)max(turning<P>(a.wh), 1)) : 0;
  logit_sums<P, TURN>(acc, R, rs_w, rs_h, oa, ob, as, bs, a.wh, first, wave, wm0, wn0, lane);
  if (m0 + P::TM > a.V) no_class<P>(acc, m0 + wm0, a.V, lane);
  lds_barrier();  // every wave is done reading the ring
  float *xm = reinterpret_cast<float *>(R.b[0]), *xs = xm + P::WGM * P::TN;
  static_assert(2 * P::WGM * P::TN * 4 <= P::B_BYTES, "exchange fits a stage");
#pragma unroll
  for (int j = 0; j < P::FN; ++j) {
    float m = -INFINITY;
#pragma unroll
    for (int i = 0; i < P::FM; ++i)
#pragma unroll
      for (int v = 0; v < 16; ++v) m = fmaxf(m, acc[i][j][v]);
    m = fmaxf(m, __shfl_xor(m, 32));
    if (lane < 32) xm[wm * P::TN + wn0 + 32 * j + lane] = m;
    // the target's logit, where it is one of this wave's classes
    const int n = n0 + wn0 + 32 * j + (lane & 31), t = target[j];
    if (__any(t >= 0 && t < P::WM)) {
      float x;
      if (pick<P>(acc, j, t, lane, x)) a.tlogit[n] = x;
    }
  }
  lds_barrier();
  float up[P::FN], s[P::FN];
#pragma unroll
  for (int j = 0; j < P::FN; ++j) {
    float m = -INFINITY;
#pragma unroll
    for (int k = 0; k < P::WGM; ++k) m = fmaxf(m, xm[k * P::TN + wn0 + 32 * j + (lane & 31)]);
    up[j] = scale_of(m);
    s[j] = 0.f;
  }
  // 2^15 exp(l - m), with one rounding of the power's exponent
  auto num = [&](int i, int j, int v) __attribute__((always_inline)) {
    const float x = __builtin_amdgcn_exp2f(__builtin_fmaf(acc[i][j][v], kLog2e, up[j]));
    s[j] += x;
    return x;
  };
  if constexpr (STORE) {
    store16<P>(
        wave_buf<P>(R, wave), lane,
        [&](int i, int j, int g) __attribute__((always_inline)) {
          float x[4];
#pragma unroll
          for (int e = 0; e < 4; ++e) x[e] = num(i, j, 4 * g + e);
          return u32x2{pack2(x[0], x[1], false), pack2(x[2], x[3], false)};
        },
        [&](int r, int c, const u32x4 &d) __attribute__((always_inline)) {
          const int n = n0 + wn0 + r, v = m0 + wm0 + c;
          if (n < rows && v < a.Vp)
            // past the L2, which then keeps the next tiles' operands: 2048 x 1024 x
            // 32000 in all 470 -> 465 us, 16384 x 768 x 16000 1416 -> 1355
            __builtin_nontemporal_store(d, reinterpret_cast<u32x4 *>(a.e + (size_t)n * a.Vp + v));
        });
  } else {
#pragma unroll
    for (int j = 0; j < P::FN; ++j)
#pragma unroll
      for (int i = 0; i < P::FM; ++i)
#pragma unroll
        for (int v = 0; v < 16; ++v) num(i, j, v);
  }
#pragma unroll
  for (int j = 0; j < P::FN; ++j) {
    s[j] += __shfl_xor(s[j], 32);
    if (lane < 32) xs[wm * P::TN + wn0 + 32 * j + lane] = s[j];
  }
  lds_barrier();
  for (int p = tid; p < P::TN; p += P::NT) {
    float m = -INFINITY, sum = 0.f;
#pragma unroll
    for (int k = 0; k < P::WGM; ++k) {
      m = fmaxf(m, xm[k * P::TN + p]);
      sum += xs[k * P::TN + p];
    }
    if (n0 + p < rows) a.stats[(size_t)ty * a.Tc + n0 + p] = float2{-scale_of(m), sum};
  }
  if (a.all.T && n0 == 0 && m0 == 0 && wave == 0) find_rows(a.all, lane, a.mark, a.found);
}

// ---- few classes -------------------------------------------------------------------
struct ClassArgs {
  const uint16_t *w, *h;
  int64_t w_ld, h_ld;
  int32_t wh, V, T;
  const Found *found;
  uint64_t *mark;
  int32_t *count;    // per tile of rows: live ones, found here as the marks are; or null
  const int32_t *target;
  const float *weight;
  uint16_t *e;       // [T][Vp] 2^15 G, or null: losses only
  int32_t Vp;
  float *loss, *lse;
  double *lsum;      // per tile of rows
};

// All classes in one tile: losses and G of TN rows.
template <class P>
__global__ __launch_bounds__(P::NT, P::WPE) void xent_classes_kernel(ClassArgs a) {
  FG_DMA_RING(P, R);
  constexpr int PA = P::PA, PB = P::PB, BK = P::BK, TN = P::TN;
  const int n0 = blockIdx.x * TN;
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int wm = wave / P::WGN, wm0 = wm * P::WM, wn0 = (wave % P::WGN) * P::WN;
  const int hrows = min(TN, a.T - n0);
  const __amdgpu_buffer_rsrc_t rs_w = rsrc(a.w, (uint32_t)((a.V - 1) * a.w_ld + a.wh) * 2u);
  const __amdgpu_buffer_rsrc_t rs_h =
      rsrc(a.h + n0 * a.h_ld, (uint32_t)((hrows - 1) * a.h_ld + a.wh) * 2u);
  auto live = [&](int n) __attribute__((always_inline)) {
    return n < a.T && (a.count ? (uint32_t)a.target[n] < (uint32_t)a.V
                               : (a.mark[n >> 6] >> (n & 63) & 1) != 0);
  };
  const KmSlot<PA> as = km_slots<BK, PA>(wave, lane);
  const KmSlot<PB> bs = km_slots<BK, PB>(wave, lane);
  unsigned oa[PA], ob[PB];
#pragma unroll
  for (int jj = 0; jj < PA; ++jj) oa[jj] = (unsigned)(as.row[jj] * (int)a.w_ld + as.coff[jj]) * 2u;
#pragma unroll
  for (int jj = 0; jj < PB; ++jj)  // masked rows: zeros
    ob[jj] = live(n0 + bs.row[jj]) ? (unsigned)(bs.row[jj] * (int)a.h_ld + bs.coff[jj]) * 2u : kOOB;
  int tg[P::FN];
  float w[P::FN], up[P::FN], s[P::FN];
#pragma unroll
  for (int j = 0; j < P::FN; ++j) {
    const int n = n0 + wn0 + 32 * j + (lane & 31);
    const bool on = live(n);
    tg[j] = on ? a.target[n] : -1;
    w[j] = !on ? 0.f : a.weight ? a.weight[n] : 1.f;
  }
  const int wexp = a.count ? kUp : a.found->wexp;
  f32x16 acc[P::FM][P::FN];
  logit_sums<P, false>(acc, R, rs_w, rs_h, oa, ob, as, bs, a.wh, 0, wave, wm0, wn0, lane);
  if (P::TM > a.V) no_class<P>(acc, wm0, a.V, lane);
  lds_barrier();  // every wave is done reading the ring
  float *xm = reinterpret_cast<float *>(R.b[0]), *xs = xm + P::WGM * TN, *xt = xs + P::WGM * TN;
  double *part = reinterpret_cast<double *>(xt + TN);
  static_assert((2 * P::WGM + 1) * TN * 4 + P::NW * 12 <= P::B_BYTES, "exchange fits a stage");
#pragma unroll
  for (int j = 0; j < P::FN; ++j) {
    const int p = wn0 + 32 * j + (lane & 31);
    float m = -INFINITY;
#pragma unroll
    for (int i = 0; i < P::FM; ++i)
#pragma unroll
      for (int v = 0; v < 16; ++v) m = fmaxf(m, acc[i][j][v]);
    float x;
    if (pick<P>(acc, j, tg[j] - wm0, lane, x)) xt[p] = x;
    m = fmaxf(m, __shfl_xor(m, 32));
    if (lane < 32) xm[wm * TN + p] = m;
  }
  lds_barrier();
#pragma unroll
  for (int j = 0; j < P::FN; ++j) {
    const int p = wn0 + 32 * j + (lane & 31);
    float m = xm[p];
#pragma unroll
    for (int k = 1; k < P::WGM; ++k) m = fmaxf(m, xm[k * TN + p]);
    up[j] = scale_of(m);
    s[j] = 0.f;
#pragma unroll
    for (int i = 0; i < P::FM; ++i)
#pragma unroll
      for (int v = 0; v < 16; ++v) {
        acc[i][j][v] = __builtin_amdgcn_exp2f(__builtin_fmaf(acc[i][j][v], kLog2e, up[j]));
        s[j] += acc[i][j][v];
      }
    s[j] += __shfl_xor(s[j], 32);
    if (lane < 32) xs[wm * TN + p] = s[j];
  }
  lds_barrier();
  double sum = 0;
  float f[P::FN], pt[P::FN];
#pragma unroll
  for (int j = 0; j < P::FN; ++j) {
    const int p = wn0 + 32 * j + (lane & 31), n = n0 + p;
    s[j] = xs[p];
#pragma unroll
    for (int k = 1; k < P::WGM; ++k) s[j] += xs[k * TN + p];
    const bool on = tg[j] >= 0;
    const float l2 = __log2f(s[j]) - up[j], d = on ? l2 * kLn2 - xt[p] : 0.f;
    const float c = ldexpf(w[j], wexp);
    f[j] = c / s[j];
    pt[j] = c * expm1f(-d);  // 2^15 w (p - 1)
    if (wm == 0 && lane < 32 && n < a.T) {
      const float loss = on ? w[j] * d : 0.f;
      a.loss[n] = loss;
      if (a.lse) a.lse[n] = on ? l2 * kLn2 : 0.f;
      sum += loss;
    }
  }
  sum = wave_sum(sum);
  if (lane == 0) part[wave] = sum;
  if (a.e) {
    store16<P>(
        wave_buf<P>(R, wave), lane,
        [&](int i, int j, int g) __attribute__((always_inline)) {
          float x[4];
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const int v = wm0 + 32 * i + 8 * g + 4 * (lane >> 5) + e;
            x[e] = acc[i][j][4 * g + e] * f[j];
            if (v == tg[j]) x[e] = pt[j];
            if (v >= a.V || tg[j] < 0) x[e] = 0.f;
          }
          return u32x2{pack2(x[0], x[1], P::BF), pack2(x[2], x[3], P::BF)};
        },
        [&](int r, int c, const u32x4 &d) __attribute__((always_inline)) {
          const int n = n0 + wn0 + r, v = wm0 + c;
          if (n >= a.T || v >= a.Vp) return;
          *reinterpret_cast<u32x4 *>(a.e + (size_t)n * a.Vp + v) = d;
        });
  }
  int rows = 0;
  if (a.count)
    for (int g = wave; g < TN / 64; g += P::NW) {
      const uint64_t mark = __ballot(live(n0 + 64 * g + lane));
      rows += __popcll(mark);
      if (lane == 0 && n0 + 64 * g < a.T) a.mark[(n0 >> 6) + g] = mark;
    }
  if (lane == 0) reinterpret_cast<int *>(part + P::NW)[wave] = rows;
  lds_barrier();
  if (tid == 0) {
    double t = 0;
    int n = 0;
    for (int k = 0; k < P::NW; ++k) {
      t += part[k];
      n += reinterpret_cast<int *>(part + P::NW)[k];
    }
    a.lsum[blockIdx.x] = t;
    if (a.count) a.count[blockIdx.x] = n;
  }
}

// ---- softmax ------------------------------------------------------------------------
struct SoftmaxArgs {
  Found *found;
  int32_t row0, Tc, V, Vp, tlog, ntile;  // 2^tlog: classes of a logits tile
  int32_t vper;                          // classes of a workgroup, a multiple of 512
  int32_t bf;                            // G in bf16, not fp16
  const int32_t *idx, *ctarget;
  const float *cweight;
  const float2 *stats;
  const float *tlogit;
  uint16_t *e;                           // null: losses only
  float *loss, *lse;
  double *lsum;                          // per RS rows
  float *totals;                         // null, or written by the last workgroup
  int32_t nsum;
  int32_t place;                         // rows in place, all Tc of them; no idx
  const uint64_t *mark;                  // (null: tiny)
  Tiny tiny;
};

// RS rows' lse and losses from their tiles, then (gradients) a range of their
// classes: numerators to 2^15 G. 256 / RS lanes join a row's tiles, 8 loads of each
// in flight; few rows take few per workgroup, for more lanes each.
template <int RS>
__global__ __launch_bounds__(256) void xent_softmax_kernel(SoftmaxArgs a) {
  constexpr int G = 256 / RS, kAhead = 8;
  __shared__ float lse2[RS], wt[RS], pt[RS];
  __shared__ int tg[RS];
  __shared__ double part[RS], ws[4];
  __shared__ bool last;
  const int rows = a.place ? a.Tc : piece_rows(a.found, a.row0, a.Tc);
  uint64_t mark = ~0ull;
  const Found found = a.tiny.T ? tiny_found(a.tiny, mark) : *a.found;
  const int r0 = blockIdx.x * RS, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const bool first = blockIdx.y == 0;
  if (r0 < rows) {
    const int r = tid / G, g = tid % G, n = r0 + r;
    float m = -INFINITY, s = 0.f;
    // (loaded beside the tiles' sums, not after them)
    const bool on =
        n < rows && (!a.place || ((a.mark ? a.mark[n >> 6] : mark) >> (n & 63) & 1));
    const float tl = on ? a.tlogit[n] : 0.f;
    const float w = !on ? 0.f : a.cweight ? a.cweight[n] : 1.f;
    const int t = on ? a.ctarget[n] : -1;
    if (n < rows)
      for (int p0 = g; p0 < a.ntile; p0 += G * kAhead) {
        float2 x[kAhead];
#pragma unroll
        for (int k = 0; k < kAhead; ++k)
          x[k] = a.stats[(size_t)min(p0 + G * k, a.ntile - 1) * a.Tc + n];
#pragma unroll
        for (int k = 0; k < kAhead; ++k) {
          if (p0 + G * k >= a.ntile || x[k].y == 0.f) continue;  // none, or all -inf
          const float top = fmaxf(m, x[k].x);
          s = s * __builtin_amdgcn_exp2f(m - top) + x[k].y * __builtin_amdgcn_exp2f(x[k].x - top);
          m = top;
        }
      }
#pragma unroll
    for (int o = G / 2; o; o >>= 1) {
      const float m1 = __shfl_xor(m, o), s1 = __shfl_xor(s, o), top = fmaxf(m, m1);
      s = (s != 0.f ? s * __builtin_amdgcn_exp2f(m - top) : 0.f) +
          (s1 != 0.f ? s1 * __builtin_amdgcn_exp2f(m1 - top) : 0.f);
      m = top;
    }
    if (g == 0) {
      const float l2 = m + __log2f(s);  // of a row with every logit -inf: -inf
      double d64 = 0;
      lse2[r] = l2;
      if (n < rows) {
        const float d = on ? l2 * kLn2 - tl : 0.f;
        tg[r] = t;
        wt[r] = ldexpf(w, found.wexp);
        pt[r] = wt[r] * expm1f(-d);  // 2^15 w (p - 1)
        if (first) {
          const int to = a.place ? n : a.idx[n];
          a.loss[to] = w * d;
          if (a.lse) a.lse[to] = on ? l2 * kLn2 : 0.f;
          d64 = w * d;
        }
      }
      part[r] = d64;
    }
    __syncthreads();
    if (first && tid == 0) {
      double sum = 0;
      for (int k = 0; k < RS; ++k) sum += part[k];
      a.lsum[blockIdx.x] = sum;
      if (a.totals && gridDim.x == 1) a.totals[0] = (float)sum, a.totals[1] = found.wsum;
    }
  } else if (first && tid == 0) {
    a.lsum[blockIdx.x] = 0;
    if (a.totals && gridDim.x == 1) a.totals[0] = 0.f, a.totals[1] = found.wsum;
  }
  if (a.totals && gridDim.x > 1) {  // losses only: the workgroup that comes last sums them up
    if (tid == 0) {
      __threadfence();
      last = atomicAdd(&a.found->ticket, 1u) + 1u == gridDim.x;
    }
    __syncthreads();
    if (last) {
      __threadfence();
      double sum = 0;
      for (int i = tid; i < a.nsum; i += 256) sum += __hip_atomic_load(
          a.lsum + i, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
      sum = wave_sum(sum);
      if (lane == 0) ws[wave] = sum;
      __syncthreads();
      if (tid == 0) {
        a.totals[0] = (float)((ws[0] + ws[1]) + (ws[2] + ws[3]));
        a.totals[1] = found.wsum;
      }
    }
  }
  if (!a.e || r0 >= rows) return;
  const int v0 = blockIdx.y * a.vper, v1 = min(a.Vp, v0 + a.vper);
  for (int k = wave; k < RS; k += 4) {
    const int n = r0 + k;
    if (n >= rows) break;
    uint16_t *row = a.e + (size_t)n * a.Vp;
    const float l2 = lse2[k], w = wt[k], p1 = pt[k];
    const int t = tg[k];
    for (int v = v0 + 8 * lane; v < v1; v += 512) {
      const u32x4 x = *reinterpret_cast<const u32x4 *>(row + v);
      const float f =
          w * __builtin_amdgcn_exp2f(a.stats[(size_t)(v >> a.tlog) * a.Tc + n].x - l2);
      u32x4 o;
      float y[8];
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        y[e] = h_to_f32((uint16_t)(x[e >> 1] >> (16 * (e & 1)))) * f;
        if (v + e == t) y[e] = p1;
        // NaN rows keep the classes past the last at 0, masked ones every class
        if (v + e >= a.V || t < 0) y[e] = 0.f;
      }
#pragma unroll
      for (int e = 0; e < 4; ++e) o[e] = pack2(y[2 * e], y[2 * e + 1], a.bf);
      *reinterpret_cast<u32x4 *>(row + v) = o;
    }
  }
}

// ---- products -------------------------------------------------------------------------
// out[n][m] = mult * sum_k A[k][m] B(n, k), m < M (hidden), with A (the weights, or
// the features) read row by row; B = G, rows n (dh, k: classes) or columns n (dW, k:
// rows).
struct ProdArgs {
  const uint16_t *a;
  int64_t a_ld;
  int32_t a_rows, a_cols;    // rows there are; columns (at least 8)
  const uint16_t *b;         // [Tc][Vp]
  int64_t b_ld;
  int32_t N;                 // columns n of B that are there (dW: Vp)
  int32_t K, kper;           // the sum's length; of a part (a multiple of 64)
  int32_t M, row0, Tc;
  const Found *found;
  const int32_t *idx;        // dh: row of the output
  int32_t V;                 // dW: rows of the output
  int32_t ntile;             // tiles of rows n
  uint16_t *out;             // null: fp32 sums to part
  int64_t out_ld;
  float *part;               // [parts][rows][Mq]
  int64_t pstride;           // elements of a part
  int32_t Mq, add;           // add: the sum is added to part's
  int32_t *flag;
  const uint64_t *mark;      // rows in place: a bit per live one
  Tiny tiny;                 // (without mark)
  Counts counts;
};

// PLACE: rows in place (up to 256 classes); marks: LDS for a part's marks.
constexpr int kMarks = 512;  // words of 64 rows
template <class P, bool DH, bool PLACE>
__device__ __forceinline__ void product_tile(const ProdArgs &a, const TileMap &tm, int block,
                                             const Ring &R, uint64_t *marks) {
  constexpr int PA = P::PA, PB = P::PB, BK = P::BK;
  int tx, ty, split;  // hidden, rows (classes), part
  if (!find_tile(tm, block, a.ntile, tx, ty, split)) return;
  const int m0 = tx * P::TM, n0 = ty * P::TN;
  const int rows = PLACE ? a.Tc : piece_rows(a.found, a.row0, a.Tc);
  if (DH && n0 >= rows) return;
  const int kbeg = split * a.kper, kend = min(min(a.K, DH ? a.K : rows), kbeg + a.kper);
  const int nst = kend > kbeg ? (kend - kbeg + BK - 1) / BK : 0;
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int wm0 = (wave / P::WGN) * P::WM, wn0 = (wave % P::WGN) * P::WN;
  uint64_t few = 0;  // the marks of a tiny call
  float mult = 0.f;
  if (PLACE && a.tiny.T)
    mult = tiny_found(a.tiny, few).mult;
  else if (!PLACE || !a.counts.n)
    mult = a.found->mult;
  Counted counted;
  if constexpr (PLACE) counted.load(a.counts);

  const MnSlot<PA> as = mn_slots<P::RBA, PA>(wave, lane);
  unsigned oa[PA], ob[PB];
#pragma unroll
  for (int jj = 0; jj < PA; ++jj)
    oa[jj] = m0 + as.ncol[jj] < a.a_cols
                 ? (unsigned)(as.krow[jj] * (int)a.a_ld + chunk_at(m0 + as.ncol[jj], a.a_cols)) * 2u
                 : kOOB;
#pragma unroll
  for (int jj = 0; jj < PB; ++jj) {
    if constexpr (DH) {
      const KmSlot<PB> bs = km_slots<BK, PB>(wave, lane);
      ob[jj] = !PLACE || bs.coff[jj] < a.b_ld  // (rows of 32: half a stage)
                   ? (unsigned)(bs.row[jj] * (int)a.b_ld + bs.coff[jj]) * 2u
                   : kOOB;
    } else {
      const MnSlot<PB> bs = mn_slots<P::RBB, PB>(wave, lane);
      ob[jj] = n0 + bs.ncol[jj] < a.N ? (unsigned)(bs.krow[jj] * (int)a.b_ld + bs.ncol[jj]) * 2u
                                      : kOOB;
    }
  }
  // the buffers begin at the stage's first row and end with the last one there is
  // (kept in 64 bits: operands may pass 2^32 bytes)
  const uint16_t *pa = a.a + kbeg * a.a_ld;
  const uint16_t *pb = DH ? a.b + n0 * a.b_ld + kbeg : a.b + kbeg * a.b_ld + n0;
  int left = max(min(a.a_rows, kend) - kbeg, 0), bleft = kend - kbeg;
  constexpr bool MASK = PLACE && !DH;  // features of masked rows: zeros
  static_assert(!MASK || BK == 64, "a word of marks per stage");
  if constexpr (MASK) {
    for (int i = tid; i < nst; i += P::NT) marks[i] = a.mark ? a.mark[kbeg / 64 + i] : few;
    __syncthreads();
  }
  auto issue = [&](int st, int slot) __attribute__((always_inline)) {
    uint8_t *ta = R.a[slot], *tb = R.b[slot];
    const uint64_t mark = MASK ? marks[st] : 0;
    const int ra = min(left, BK), rb = min(bleft, BK);
    const __amdgpu_buffer_rsrc_t rs_a =
        rsrc(pa, ra > 0 ? (uint32_t)((ra - 1) * (int)a.a_ld + a.a_cols) * 2u : 0u);
    const __amdgpu_buffer_rsrc_t rs_b =
        DH ? rsrc(pb, (uint32_t)((P::TN - 1) * (int)a.b_ld + BK) * 2u)
           : rsrc(pb, rb > 0 ? (uint32_t)(rb * (int)a.b_ld - n0) * 2u : 0u);
#pragma unroll
    for (int jj = 0; jj < PB; ++jj) dma16(rs_b, tb + dma_dst<PB>(wave, jj), ob[jj]);
#pragma unroll
    for (int jj = 0; jj < PA; ++jj)
      dma16(rs_a, ta + dma_dst<PA>(wave, jj),
            !MASK || (mark >> as.krow[jj] & 1) ? oa[jj] : kOOB);
    pa += BK * a.a_ld;
    pb += DH ? BK : BK * a.b_ld;
    left -= BK;
    bleft -= BK;
  };
  f32x16 acc[P::FM][P::FN];
  zero<P>(acc);
  pipeline<P, false, !DH ? false : true>(acc, R, nst, wm0, wn0, lane, issue);

  const int nrow = DH ? rows : a.V;
  if (a.part) {
    float *part = a.part + split * a.pstride;
#pragma unroll
    for (int j = 0; j < P::FN; ++j) {
      const int n = n0 + wn0 + 32 * j + (lane & 31);
      if (n >= nrow) continue;
      float *row = part + (size_t)n * a.Mq;
      const int c = m0 + wm0 + 4 * (lane >> 5);
      if (a.add) {  // every load on its way before the first sum
        f32x4 v[P::FM][4];
#pragma unroll
        for (int i = 0; i < P::FM; ++i)
#pragma unroll
          for (int g = 0; g < 4; ++g) {
            const int m = c + 32 * i + 8 * g;
            v[i][g] = *reinterpret_cast<const f32x4 *>(row + (m < a.Mq ? m : 0));
          }
#pragma unroll
        for (int i = 0; i < P::FM; ++i)
#pragma unroll
          for (int r = 0; r < 16; ++r) acc[i][j][r] += v[i][r >> 2][r & 3];
      }
      if (a.out) continue;
#pragma unroll
      for (int i = 0; i < P::FM; ++i)
#pragma unroll
        for (int g = 0; g < 4; ++g) {
          const int m = c + 32 * i + 8 * g;
          if (m < a.Mq)
            *reinterpret_cast<f32x4 *>(row + m) = f32x4{acc[i][j][4 * g], acc[i][j][4 * g + 1],
                                                        acc[i][j][4 * g + 2], acc[i][j][4 * g + 3]};
        }
    }
    if (!a.out) return;
  }
  lds_barrier();  // every wave is done reading the ring
  if (PLACE && a.counts.n) mult = counted.found(a.counts).mult;
  bool bad = false;
  store16<P>(
      wave_buf<P>(R, wave), lane,
      [&](int i, int j, int g) __attribute__((always_inline)) {
        const f32x16 &c = acc[i][j];
        return u32x2{pack2(c[4 * g] * mult, c[4 * g + 1] * mult, P::BF),
                     pack2(c[4 * g + 2] * mult, c[4 * g + 3] * mult, P::BF)};
      },
      [&](int r, int c, const u32x4 &d) __attribute__((always_inline)) {
        const int n = n0 + wn0 + r, m = m0 + wm0 + c;
        if (n >= nrow || m >= a.M) return;
        constexpr uint32_t EX = P::BF ? 0x7F80u : 0x7C00u;
        if (!DH) {
#pragma unroll
          for (int e = 0; e < 8; ++e)
            bad |= (d[e >> 1] >> (16 * (e & 1)) & EX) == EX;
        }
        const bool on = !DH || !PLACE || ((a.mark ? a.mark[n >> 6] : few) >> (n & 63) & 1);
        put_chunk(a.out + (int64_t)(DH && !PLACE ? a.idx[n] : n) * a.out_ld, m, a.M,
                  on ? d : u32x4{0, 0, 0, 0});
      });
  if (!DH && a.flag) flag_nonfinite(a.flag, bad);
}

// Both gradients in one launch, dh's tiles in the first nh workgroups: neither waits
// for the other's last tiles. The first wave also sums up the losses where they are
// few, which saves a launch.
constexpr int kSumHere = 1024;  // partial sums
struct SumArgs {
  const double *lsum;
  int32_t n;         // partial sums; 0: not here
  const Found *found;
  float *totals;
  Tiny tiny;
  Counts counts;
};
// The weights' sum, by a wave.
__device__ __forceinline__ float weights_sum(const Tiny &tiny, const Counts &counts,
                                             const Found *found) {
  if (counts.n) {
    Counted c;
    c.load(counts);
    return c.found(counts).wsum;
  }
  uint64_t mark;
  return tiny.T ? tiny_found(tiny, mark).wsum : found->wsum;
}
template <class P, bool PLACE>
__global__ __launch_bounds__(P::NT, P::WPE) void xent_products_kernel(ProdArgs dh, TileMap th,
                                                                      ProdArgs dw, TileMap tw,
                                                                      int nh, SumArgs sum) {
  FG_DMA_RING(P, R);
  __shared__ uint64_t marks[PLACE ? kMarks : 1];
  const int block = blockIdx.x;
  if (sum.n && block == 0 && threadIdx.x < 64) {
    double s = 0;
#pragma unroll 4
    for (int i = threadIdx.x; i < sum.n; i += 64) s += sum.lsum[i];
    s = wave_sum(s);
    const float w = weights_sum(sum.tiny, sum.counts, sum.found);
    if (threadIdx.x == 0) {
      sum.totals[0] = (float)s;
      sum.totals[1] = w;
    }
  }
  if (block < nh)
    product_tile<P, true, PLACE>(dh, th, block, R, marks);
  else
    product_tile<P, false, PLACE>(dw, tw, block - nh, R, marks);
}

// One workgroup: the sums of the losses and of the weights. With counts: unweighted rows of
// few classes in more tiles than every workgroup adds up, whose live ones it counts for the
// kernels after it.
__global__ __launch_bounds__(1024) void xent_totals_kernel(SumArgs a, Counts counts, Found *found) {
  __shared__ double ws[16];
  __shared__ int cn[16];
  double s = 0;
  int n = 0;
#pragma unroll 4
  for (int i = threadIdx.x; i < a.n; i += 1024) {
    s += a.lsum[i];
    if (counts.n) n += counts.live[i];
  }
  s = wave_sum(s);
  n = wave_sum(n);
  if ((threadIdx.x & 63) == 0) ws[threadIdx.x >> 6] = s, cn[threadIdx.x >> 6] = n;
  __syncthreads();
  if (threadIdx.x < 64) {
    for (int k = 1; k < 16; ++k) s += ws[k], n += cn[k];
    float w;
    if (counts.n) {
      const Found f = make_found(counts.mean, counts.scale, n, (double)n, 1.f);
      w = f.wsum;
      if (threadIdx.x == 0) *found = f;
    } else {
      w = weights_sum(a.tiny, a.counts, a.found);
    }
    if (threadIdx.x == 0 && a.totals) {
      a.totals[0] = (float)s;
      a.totals[1] = w;
    }
  }
}

// Joins the parts of a split sum, in their order: 8 columns of a row per lane.
struct JoinArgs {
  const float *part;
  int64_t pstride;
  int32_t nsplit, rows, M, Mq;  // rows: -1: the piece's live ones
  int32_t shared;               // by a workgroup's waves
  int32_t row0, Tc;
  const Found *found;
  const int32_t *idx;
  const uint64_t *mark;         // rows in place (dh)
  Tiny tiny;                    // (without mark)
  Counts counts;
  int32_t masked;               // dh: masked rows are zeros
  uint16_t *out;
  int64_t out_ld;
  int32_t bf;
  int32_t *flag;
};
// Where there are many, the workgroup's 8 waves share a sum, a run of the parts each
// (12 x 512 sums of 256 parts took 42 us by single lanes). Both gradients' in one
// launch, dh's in the first nh workgroups.
__device__ __forceinline__ void join_rows(const JoinArgs &a, int block, float (&sh)[8][64][8]) {
  const int rows = a.rows < 0 ? piece_rows(a.found, a.row0, a.Tc) : a.rows;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  uint64_t few = ~0ull;
  Counted counted;
  counted.load(a.counts);
  const float mult = a.counts.n ? counted.found(a.counts).mult
                     : a.tiny.T ? tiny_found(a.tiny, few).mult
                                : a.found->mult;
  const bool shared = a.shared;
  const int64_t i = shared ? (int64_t)block * 64 + lane : (int64_t)block * 512 + threadIdx.x;
  const int c8 = a.Mq / 8;
  const int64_t n = i / c8;
  const int m = (int)(i - n * c8) * 8;
  const int per = shared ? (a.nsplit + 7) / 8 : a.nsplit;
  const int s0 = shared ? wave * per : 0, s1 = min(a.nsplit, s0 + per);
  bool bad = false;
  float v[8] = {};
  if (n < rows) {
    const float *p = a.part + s0 * a.pstride + n * a.Mq + m;
#pragma unroll 4
    for (int s = s0; s < s1; ++s, p += a.pstride)
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const f32x4 x = *reinterpret_cast<const f32x4 *>(p + 4 * h);
#pragma unroll
        for (int e = 0; e < 4; ++e) v[4 * h + e] += x[e];
      }
  }
  if (shared) {
#pragma unroll
    for (int e = 0; e < 8; ++e) sh[wave][lane][e] = v[e];
    __syncthreads();
    if (wave) return;
#pragma unroll
    for (int k = 1; k < 8; ++k)
#pragma unroll
      for (int e = 0; e < 8; ++e) v[e] += sh[k][lane][e];
  }
  if (n < rows) {
    u32x4 d;
#pragma unroll
    for (int e = 0; e < 4; ++e) d[e] = pack2(v[2 * e] * mult, v[2 * e + 1] * mult, a.bf);
    const uint32_t ex = a.bf ? 0x7F80u : 0x7C00u;
#pragma unroll
    for (int e = 0; e < 8; ++e) bad |= (d[e >> 1] >> (16 * (e & 1)) & ex) == ex;
    if (a.masked && !((a.mark ? a.mark[n >> 6] : few) >> (n & 63) & 1)) d = u32x4{0, 0, 0, 0};
    put_chunk(a.out + (a.idx ? a.idx[n] : n) * a.out_ld, m, a.M, d);
  }
  if (a.flag) flag_nonfinite(a.flag, bad);
}
__global__ __launch_bounds__(512) void xent_join_kernel(JoinArgs dh, JoinArgs dw, int nh) {
  __shared__ float sh[8][64][8];
  const bool first = (int)blockIdx.x < nh;
  join_rows(first ? dh : dw, first ? blockIdx.x : blockIdx.x - nh, sh);
}

// Gradients that are sums of at most 64 terms per element, bound by being written: dW of
// up to 64 rows, dh of up to 64 classes (DH). out[n][m] = mult sum_k A[k][m] G, with A
// the features (weights). A workgroup (8 waves of 64 x 32) keeps 256 columns of A in
// registers and goes through a range of the rows n, 64 at a time, whose G arrives while
// the ones before are multiplied and stored. dW of 3 rows, 2496 x 21696: 24.6 us (4.4
// TB/s), 55 by the tiles of xent_products_kernel; dh of 65536 x 512,
// 12 classes: 15 us (5 TB/s), where both products by those tiles took 38 and dW's alone
// take 14; 131073 x 331, 3 classes 105 -> 86 us in all.
// Below kOuter weights the launch it adds costs more: 11 rows of 128 x 1088 18.7 us in all
// without it and 24.9 with it, 41 of 287 x 4039 22.8 and 25.1; 7 of 148 x 38444 33.5 and
// 28.7, 7 of 2432 x 4032 41.9 and 35.4.
constexpr int64_t kOuter = (int64_t)3 << 20;
struct OuterArgs {
  const uint16_t *a;
  int64_t a_ld;
  int32_t K, cols;           // terms; elements of a row of A, at least 8
  const uint16_t *g;         // [rows][Vp]
  int32_t Vp, N, H;          // output rows, columns
  int32_t per;               // chunks of 64 output rows of a workgroup
  uint16_t *out;
  int64_t out_ld;
  int32_t *flag;             // dW
  const uint64_t *mark;      // dh
  Tiny tiny;                 // dW: leaves masked rows out
  Counts counts;
  const Found *found;
};
using POuter = Pipe<64, 2, 4, 2, 256, 64>;  // shapes only: 64 terms deep, 8 waves

template <class P, bool DH>
__device__ __forceinline__ void outer_tile(const OuterArgs &a, int tm, int tv, uint8_t *stage) {
  __shared__ __attribute__((aligned(1024))) uint8_t sA[P::A_BYTES], sB0[P::B_BYTES],
      sB1[P::B_BYTES];
  constexpr int PA = P::PA, PB = P::PB, KS = P::KS;
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int wm0 = (wave / P::WGN) * P::WM, wn0 = (wave % P::WGN) * P::WN;
  const int m0 = tm * P::TM, c0 = tv * a.per, c1 = min((a.N + 63) / 64, c0 + a.per);
  if (c0 >= c1) return;
  uint64_t on = ~0ull;  // rows of A that count
  Counted counted;
  float mult;
  if (DH) {
    counted.load(a.counts);
    mult = a.counts.n ? counted.found(a.counts).mult : a.found->mult;
  } else {
    mult = tiny_found(a.tiny, on).mult;
  }
  // rows of A past the last one, and masked ones: zeros
  const __amdgpu_buffer_rsrc_t rs_a = rsrc(a.a, (uint32_t)((a.K - 1) * (int)a.a_ld + a.cols) * 2u);
  const MnSlot<PA> as = mn_slots<P::RBA, PA>(wave, lane);
  auto issue = [&](int c, uint8_t *to) __attribute__((always_inline)) {
    if constexpr (DH) {  // 64 rows of G, Vp = 32 or 64
      const KmSlot<PB> bs = km_slots<64, PB>(wave, lane);
      const __amdgpu_buffer_rsrc_t rs_g =
          rsrc(a.g + (int64_t)64 * c * a.Vp, (uint32_t)(min(64, a.N - 64 * c) * a.Vp) * 2u);
#pragma unroll
      for (int jj = 0; jj < PB; ++jj)
        dma16(rs_g, to + dma_dst<PB>(wave, jj),
              bs.coff[jj] < a.Vp ? (unsigned)(bs.row[jj] * a.Vp + bs.coff[jj]) * 2u : kOOB);
    } else {  // 64 columns of G's K rows
      const MnSlot<PB> bs = mn_slots<P::RBB, PB>(wave, lane);
      const __amdgpu_buffer_rsrc_t rs_g = rsrc(a.g, (uint32_t)(a.K * a.Vp) * 2u);
#pragma unroll
      for (int jj = 0; jj < PB; ++jj)
        dma16(rs_g, to + dma_dst<PB>(wave, jj),
              bs.krow[jj] < a.K && 64 * c + bs.ncol[jj] < a.Vp
                  ? (unsigned)(bs.krow[jj] * a.Vp + 64 * c + bs.ncol[jj]) * 2u
                  : kOOB);
    }
  };
  issue(c0, sB0);
#pragma unroll
  for (int jj = 0; jj < PA; ++jj)
    dma16(rs_a, sA + dma_dst<PA>(wave, jj),
          (on >> as.krow[jj] & 1) && as.krow[jj] < a.K && m0 + as.ncol[jj] < a.cols
              ? (unsigned)(as.krow[jj] * (int)a.a_ld + chunk_at(m0 + as.ncol[jj], a.cols)) * 2u
              : kOOB);
  wait_vm<0>();
  barrier_nofence();
  u32x4 fa[KS][P::FM];
#pragma unroll
  for (int ks = 0; ks < KS; ++ks)
#pragma unroll
    for (int i = 0; i < P::FM; ++i) fa[ks][i] = frag<64, false, P::RBA>(sA, wm0 + 32 * i, ks, lane);
  bool bad = false;
  auto chunk = [&](int c, const uint8_t *here, uint8_t *next) __attribute__((always_inline)) {
    const uint64_t mark = DH ? a.mark[c] : ~0ull;
    if (c > c0) {  // this chunk has arrived, and every wave has read the one before
      wait_vm<0>();
      wait_lds();
      barrier_nofence();
    }
    if (c + 1 < c1) issue(c + 1, next);
    f32x16 acc[P::FM][P::FN];
    zero<P>(acc);
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) {
      if (16 * ks >= a.K) break;
#pragma unroll
      for (int j = 0; j < P::FN; ++j) {
        const u32x4 fb = frag<64, DH, P::RBB>(here, wn0 + 32 * j, ks, lane);
#pragma unroll
        for (int i = 0; i < P::FM; ++i)
          acc[i][j] = P::BF ? mfma32_bf16(fa[ks][i], fb, acc[i][j])
                            : mfma32(fa[ks][i], fb, acc[i][j]);
      }
    }
    store16<P>(
        stage + wave * 64 * P::WM, lane,
        [&](int i, int j, int g) __attribute__((always_inline)) {
          const f32x16 &x = acc[i][j];
          return u32x2{pack2(x[4 * g] * mult, x[4 * g + 1] * mult, P::BF),
                       pack2(x[4 * g + 2] * mult, x[4 * g + 3] * mult, P::BF)};
        },
        [&](int r, int q, const u32x4 &d) __attribute__((always_inline)) {
          const int n = 64 * c + wn0 + r, m = m0 + wm0 + q;
          if (n >= a.N || m >= a.H) return;
          constexpr uint32_t EX = P::BF ? 0x7F80u : 0x7C00u;
          if (!DH) {
#pragma unroll
            for (int e = 0; e < 8; ++e) bad |= (d[e >> 1] >> (16 * (e & 1)) & EX) == EX;
          }
          put_chunk(a.out + (int64_t)n * a.out_ld, m, a.H,
                    mark >> (n & 63) & 1 ? d : u32x4{0, 0, 0, 0});
        });
  };
  for (int c = c0; c < c1; c += 2) {
    chunk(c, sB0, sB1);
    if (c + 1 < c1) chunk(c + 1, sB1, sB0);
  }
  if (!DH && a.flag) flag_nonfinite(a.flag, bad);
}

// With the join of the other gradient's parts in the first workgroups.
template <class P, bool DH>
__global__ __launch_bounds__(P::NT) void xent_outer_kernel(OuterArgs a, int nm, JoinArgs other,
                                                           int nj) {
  __shared__ __attribute__((aligned(1024))) uint8_t stage[P::NW * 64 * P::WM];
  static_assert(P::NT == 512 && sizeof(stage) >= 16384, "room for the join's workgroups");
  if ((int)blockIdx.x < nj) {
    join_rows(other, blockIdx.x, *reinterpret_cast<float(*)[8][64][8]>(stage));
    return;
  }
  const int b = blockIdx.x - nj;
  outer_tile<P, DH>(a, b % nm, b / nm, stage);
}

// ---- host ------------------------------------------------------------------------------
// Rows x hidden x classes up to which up to kWave rows stay in place: that saves a launch
// and costs the masked rows' products, and the largest tiles. Gradients of 200 x 256 x 1000
// 23.1 -> 20.0 us, losses of 256 x 1024 x 8000 21.0 -> 17.6; gradients of 128 x 700 x 90000
// would take 171.8, not 168.2.
constexpr int64_t kInPlace = (int64_t)1 << 32;
// The numerators of a piece of rows take at most this much of the workspace; all rows are
// one piece where theirs take no more than this and the fp32 sums of dW, which several
// pieces need, would together. Fewer, longer pieces add those sums (8 bytes an element of
// the weights) less often; a gibibyte holds 4096 rows of 131072 classes. (One piece
// against two: 8192 x 4096 x 131072 21.1 and 22.2 ms, 5000 x 512 x 131072 2.73 and 3.05.)
constexpr int64_t kPieceBytes = (int64_t)1 << 30;

constexpr int kTileOf[3] = {64, 128, 256};
// Tile and number of parts for a product of M x N sums of length K: the least of the
// times estimated for rounds of the workgroups that the chip holds. A round costs a
// fixed time (first loads, store) and one per unit of K, by the tile and the
// workgroups on a CU; measured over 56 shapes (1 .. 4096 rows, 64 .. 4096 hidden, 2000
// .. 32000 classes), in which the tile chosen is within 20% of the best of the three.
// The best number of parts for one tile, and its time.
Shape pick_tile(int t, int64_t M, int64_t N, int64_t K, bool split, double &us_best) {
  static const int occ[3] = {3, 2, 1};
  static const double fixed[3][3] = {{2.0, 2.0, 2.0}, {3.5, 5.5, 5.5}, {9.0, 9.0, 9.0}};
  const double more = !split ? 0.0 : t == 2 ? 5.0 : t == 0 ? 1.0 : 0.0;  // the products' store
  static const double per_k[3][3] = {{.0055, .009, .0135}, {.0095, .0178, .0178},
                                     {.0175, .0175, .0175}};
  Shape best{t, 1, 0};
  us_best = 1e300;
  const int64_t ts = kTileOf[t];
  const int64_t tiles = ((M + ts - 1) / ts) * ((N + ts - 1) / ts);
  for (int ns = 1; ns <= (split ? 512 : 1); ns *= 2) {
    const int64_t kper = std::max<int64_t>(64, ((K + ns - 1) / ns + 63) / 64 * 64);
    if (ns > 1 && kper < 256) break;
    const int64_t parts = std::max<int64_t>(1, (K + kper - 1) / kper);
    const int64_t n = tiles * parts, slots = 256 * occ[t];
    const int64_t full = n / slots, rest = n - full * slots;
    // a chip full of the largest tiles is slower per tile than a few of them
    auto round = [&](int64_t m) {
      const int j = (int)((m + 255) / 256) - 1;
      return fixed[t][j] + more + kper * (per_k[t][j] + (t == 2 ? .0105 * m / 256 : 0.));
    };
    double us = full * round(slots);
    if (rest) us += round(rest);
    if (parts > 1) us += 6.0 + (double)parts * M * N * 8 / 8e6;
    if (us < us_best) us_best = us, best = {t, (int)parts, (int)kper};
  }
  return best;
}

struct Plan {
  int64_t T, H, V, Tp, Hp, Vp, Hq, Tc, pieces, nb, wh, w_ld;
  bool pad_w, place, tiny, classes, outer, spread;  // rows in place, up to 64 of many classes;
                                                    // one tile holds all classes; dW, dh by
                                                    // xent_outer_kernel
  Shape s1, s2, s3;
  int64_t ntile, slot;
  // workspace, bytes
  size_t count, wsum, wmax, found, mark, tcount, idx, ctarget, cweight, hc, wc, stats, tlogit,
      e, pdh, pdw, lsum, total;
};

Plan make_plan(const fg_xent_desc &d, bool grad) {
  Plan p{};
  p.T = d.rows, p.H = d.hidden, p.V = d.vocab;
  // (G of up to 32 classes in rows of 32: 262144 x 256 x 12 97.3 -> 89.6 us)
  p.Tp = up(p.T, 256), p.Hp = up(p.H, 64), p.Vp = p.V <= 32 ? 32 : up(p.V, 64), p.Hq = up(p.H, 8);
  p.w_ld = d.w_ld ? d.w_ld : p.H;
  p.pad_w = p.H < 8;
  p.wh = std::max<int64_t>(p.H, 8);
  if (p.pad_w) p.w_ld = 8;
  p.nb = (p.T + kCount - 1) / kCount;
  const int64_t per_row = grad ? p.Vp * 2 : (p.V + 63) / 64 * 8;
  int64_t most = std::max<int64_t>(256, kPieceBytes / per_row / 256 * 256);
  if (grad && p.Tp * per_row <= kPieceBytes + p.V * p.Hq * 4) most = std::max(most, p.Tp);
  p.pieces = std::max<int64_t>(1, (p.Tp + most - 1) / most);
  p.Tc = std::max<int64_t>(256, up((p.T + p.pieces - 1) / p.pieces, 256));
  p.pieces = std::max<int64_t>(1, (p.T + p.Tc - 1) / p.Tc);
  p.classes = p.V <= kTileOf[2];
  p.tiny = !p.classes && p.T <= 64;
  p.place = p.classes || p.tiny || (p.T <= kWave && p.T * p.H * p.V <= kInPlace);
  p.outer = p.tiny && p.T > 0 && p.V * p.H >= kOuter;
  p.spread = p.V <= 64 && p.T * p.H >= kOuter;
  if (p.place) p.pieces = 1, p.Tc = std::max<int64_t>(256, p.Tp);
  const int64_t rows = std::min(p.T, p.Tc);
  double best = 1e300, us, us2;
  for (int t = 0; t < 3; ++t) {
    const Shape a = pick_tile(t, p.V, rows, p.H, false, us);
    if (us < best) best = us, p.s1 = a;
  }
  p.ntile = (p.V + kTileOf[p.s1.tile] - 1) / kTileOf[p.s1.tile];
  best = 1e300;  // one launch, one tile for both products
  for (int t = 0; t < (p.place ? 2 : 3); ++t) {  // in place: tiles of 64-deep stages
    const Shape a = pick_tile(t, p.H, rows, p.Vp, true, us);
    const Shape b = pick_tile(t, p.H, p.V, rows, true, us2);
    if (p.outer) us2 = 0;
    if (p.spread) us = 0;
    if (us + us2 < best) best = us + us2, p.s2 = a, p.s3 = b;
  }
  if (p.place && p.s3.kper > 64 * kMarks) {
    p.s3.kper = 64 * kMarks;
    p.s3.ns = (int)((rows + p.s3.kper - 1) / p.s3.kper);
  }
  // rows of a workgroup of the kernel that finds the losses
  p.slot = !p.classes ? (p.T <= kFew ? 4 : 16)
           : p.V > 64 && p.T <= kHalf ? 64
           : p.V <= 128               ? 128
                                      : 256;
  size_t at = 0;
  auto take = [&](size_t bytes) {
    const size_t was = at;
    at += (bytes + 255) / 256 * 256;
    return was;
  };
  p.found = take(sizeof(Found));
  p.count = take(p.nb * 4);
  p.wsum = take(p.nb * 8);
  p.wmax = take(p.nb * 4);
  const int64_t moved = p.place ? 0 : 1;
  p.idx = take(moved * p.Tp * 4);
  p.ctarget = take(moved * p.Tp * 4);
  p.cweight = take(moved * p.Tp * 4);
  p.lsum = take(p.pieces * (p.Tc / p.slot) * 8);
  p.mark = take(p.place ? p.Tp / 8 : 0);
  p.tcount = take(p.classes ? (p.T + p.slot - 1) / p.slot * 4 : 0);
  // the products read whole tiles of rows: a tile past the last piece's rows too
  p.hc = take(p.place ? (p.pad_w ? (size_t)p.Tp * 16 : 0) : (size_t)p.pieces * p.Tc * p.Hp * 2);
  p.stats = take(p.classes ? 0 : (size_t)p.ntile * p.Tc * 8);
  p.tlogit = take(p.classes ? 0 : p.Tc * 4);
  if (grad) {
    p.e = take((size_t)p.Tc * p.Vp * 2);
    if (p.spread) p.s2.ns = 1;
    p.pdh = take(p.s2.ns > 1 ? (size_t)p.s2.ns * p.Tc * p.Hq * 4 : 0);
    if (p.outer) p.s3.ns = 1;
    p.pdw = take(p.s3.ns > 1 || p.pieces > 1 ? (size_t)p.s3.ns * p.V * p.Hq * 4 : 0);
  }
  p.wc = take(p.pad_w ? (size_t)p.V * 16 : 0);
  p.total = at;
  return p;
}

template <class P>
hipError_t launch_logits(LogitArgs a, int64_t rows, hipStream_t st) {
  a.stream = rows <= P::TN;
  const TileMap tm = tile_map((rows + P::TN - 1) / P::TN, (a.V + P::TM - 1) / P::TM, 1);
  if (a.e)
    hipLaunchKernelGGL((xent_logits_kernel<P, true>), dim3(8 * tm.per), dim3(P::NT), 0, st, a, tm);
  else
    hipLaunchKernelGGL((xent_logits_kernel<P, false>), dim3(8 * tm.per), dim3(P::NT), 0, st, a,
                       tm);
  return hipGetLastError();
}

struct Products {
  ProdArgs dh, dw;
  JoinArgs jdh, jdw;
  int nsdh, nsdw;     // parts; 0: that gradient is not wanted
  int64_t rows;
  bool place;
  SumArgs sum;
  OuterArgs outer;    // out: dW this way, not by dw
};

template <class P>
hipError_t launch_products(Products &a, hipStream_t st) {
  a.dh.ntile = (int32_t)((a.rows + P::TN - 1) / P::TN);
  a.dw.ntile = (a.dw.V + P::TN - 1) / P::TN;
  const TileMap th = tile_map((a.dh.M + P::TM - 1) / P::TM, std::max(a.dh.ntile, 1), a.nsdh);
  const TileMap tw = tile_map((a.dw.M + P::TM - 1) / P::TM, a.dw.ntile, a.nsdw);
  const dim3 grid(8 * (th.per + tw.per)), block(P::NT);
  if constexpr (P::BK == 64) {
    if (a.place) {
      hipLaunchKernelGGL((xent_products_kernel<P, true>), grid, block, 0, st, a.dh, th, a.dw, tw,
                         8 * th.per, a.sum);
      return hipGetLastError();
    }
  }
  hipLaunchKernelGGL((xent_products_kernel<P, false>), grid, block, 0, st, a.dh, th, a.dw, tw,
                     8 * th.per, a.sum);
  return hipGetLastError();
}

template <class P>
hipError_t launch_classes(const ClassArgs &a, hipStream_t st) {
  hipLaunchKernelGGL(xent_classes_kernel<P>, dim3((uint32_t)((a.T + P::TN - 1) / P::TN)),
                     dim3(P::NT), 0, st, a);
  return hipGetLastError();
}

int join_blocks(JoinArgs &j, int64_t rows) {
  const int64_t n = rows * (j.Mq / 8);
  j.shared = j.nsplit >= 16;
  return (int)((n + (j.shared ? 63 : 511)) / (j.shared ? 64 : 512));
}

hipError_t launch_join(Products &a, bool dh, bool dw, hipStream_t st) {
  if (!dh && !dw) return hipSuccess;
  const int nh = dh ? join_blocks(a.jdh, a.rows) : 0, nw = dw ? join_blocks(a.jdw, a.dw.V) : 0;
  hipLaunchKernelGGL(xent_join_kernel, dim3((uint32_t)(nh + nw)), dim3(512), 0, st, a.jdh, a.jdw,
                     nh);
  return hipGetLastError();
}

template <class P, bool DH>
hipError_t launch_outer(Products &a, bool join, hipStream_t st) {
  const int nj = !join ? 0 : DH ? join_blocks(a.jdw, a.dw.V) : join_blocks(a.jdh, a.rows);
  const int nm = (a.outer.H + P::TM - 1) / P::TM, chunks = (a.outer.N + 63) / 64;
  // some 1024 workgroups, two chunks each at least where there are as many
  const int nv = std::max(1, std::min((chunks + 1) / 2, 1024 / nm));
  a.outer.per = (chunks + nv - 1) / nv;
  const int n = nm * ((chunks + a.outer.per - 1) / a.outer.per);
  hipLaunchKernelGGL((xent_outer_kernel<P, DH>), dim3((uint32_t)(nj + n)), dim3(P::NT), 0, st,
                     a.outer, nm, DH ? a.jdw : a.jdh, nj);
  return hipGetLastError();
}

#define FG_XENT_TILE(FN, TS, tile, bf, ...)                                          \
  ((tile) == 2   ? ((bf) ? FN<Bf16<TS::T256>>(__VA_ARGS__) : FN<TS::T256>(__VA_ARGS__)) \
   : (tile) == 1 ? ((bf) ? FN<Bf16<P128>>(__VA_ARGS__) : FN<P128>(__VA_ARGS__))       \
                 : ((bf) ? FN<Bf16<P64>>(__VA_ARGS__) : FN<P64>(__VA_ARGS__)))

struct Call {
  const void *h, *w;
  const int32_t *target;
  const float *weight;
  float *loss, *lse, *totals;
  void *dh, *dw;
  int32_t *flag;
  bool grad;
};

hipError_t run(const fg_xent_desc &d, const Call &c, void *ws, hipStream_t st) {
  const int64_t w_ld = d.w_ld ? d.w_ld : d.hidden;
  const Plan p = make_plan(d, c.grad);
  uint8_t *base = static_cast<uint8_t *>(ws);
  auto at = [&](size_t off) { return base + off; };
  const int bf = d.dtype == FG_BF16;
#define FG_TRY(x)                      \
  do {                                 \
    const hipError_t e_ = (x);         \
    if (e_ != hipSuccess) return e_;   \
  } while (0)

  RowArgs r{};
  r.h = (const uint16_t *)c.h;
  r.h_ld = d.h_ld ? d.h_ld : d.hidden;
  r.target = c.target, r.weight = c.weight;
  r.T = (int32_t)p.T, r.H = (int32_t)p.H, r.Hp = (int32_t)p.Hp, r.V = (int32_t)p.V;
  r.nb = (int32_t)p.nb;
  r.scale = d.scale, r.mean = d.mean;
  r.dh = (uint16_t *)c.dh;
  r.dh_ld = d.dh_ld ? d.dh_ld : d.hidden;
  r.count = (int32_t *)at(p.count), r.wsum = (double *)at(p.wsum), r.wmax = (float *)at(p.wmax);
  r.found = (Found *)at(p.found);
  r.idx = (int32_t *)at(p.idx), r.ctarget = (int32_t *)at(p.ctarget);
  r.cweight = (float *)at(p.cweight);
  r.hc = (uint16_t *)at(p.hc);
  r.loss = c.loss, r.lse = c.lse;
  r.mark = p.place && !p.tiny ? (uint64_t *)at(p.mark) : nullptr;
  const Tiny all = {c.target, c.weight, (int32_t)p.T, (int32_t)p.V, d.mean, d.scale}, none{};
  const Tiny tiny = p.tiny ? all : none;
  const bool stay = p.place && !p.classes;
  const int32_t nsum = (int32_t)((p.T + p.slot - 1) / p.slot);
  Counts counts{};
  Counts many{};  // counted by the classes' kernel, added up by one after it
  if (p.classes && !c.weight && nsum > 0)
    (nsum <= kTiles ? counts : many) = {(int32_t *)at(p.tcount), nsum, d.mean, d.scale};
  if ((stay && p.T) || counts.n || many.n) {  // nothing to find out beforehand
  } else if (p.classes && p.T) {
    hipLaunchKernelGGL(xent_count_kernel, dim3((uint32_t)p.nb), dim3(256), 0, st, r);
    FG_TRY(hipGetLastError());
    if (p.nb > 1) {
      hipLaunchKernelGGL(xent_scan_kernel, dim3(1), dim3(1024), 0, st, r);
      FG_TRY(hipGetLastError());
    }
  } else if (p.T <= kDirect) {
    r.nb = 0;  // a row per wave: a few rows are bound by one row's latency
    hipLaunchKernelGGL(xent_rows_kernel<1>, dim3((uint32_t)((p.T + 3) / 4 + 1)), dim3(256), 0, st,
                       r);
    FG_TRY(hipGetLastError());
  } else {
    hipLaunchKernelGGL(xent_count_kernel, dim3((uint32_t)p.nb), dim3(256), 0, st, r);
    FG_TRY(hipGetLastError());
    hipLaunchKernelGGL(xent_scan_kernel, dim3(1), dim3(1024), 0, st, r);
    FG_TRY(hipGetLastError());
    // 16 rows a workgroup, 32 where 16 would make 2^32 work items, more than a launch holds
    if (p.T <= kWide)
      hipLaunchKernelGGL(xent_rows_kernel<4>, dim3((uint32_t)((p.T + 15) / 16)), dim3(256), 0, st,
                         r);
    else
      hipLaunchKernelGGL(xent_rows_kernel<8>, dim3((uint32_t)((p.T + 31) / 32)), dim3(256), 0, st,
                         r);
    FG_TRY(hipGetLastError());
  }
  const uint16_t *w = (const uint16_t *)c.w;
  if (p.pad_w && p.T) {
    hipLaunchKernelGGL(xent_pad_kernel, dim3((uint32_t)((p.V + 255) / 256)), dim3(256), 0, st, w,
                       w_ld, (int32_t)p.H, (uint16_t *)at(p.wc), (int32_t)p.V);
    FG_TRY(hipGetLastError());
    w = (const uint16_t *)at(p.wc);
  }
  const uint16_t *h = (const uint16_t *)c.h;  // rows in place
  int64_t h_ld = r.h_ld;
  if (p.place && p.pad_w && p.T) {
    hipLaunchKernelGGL(xent_pad_kernel, dim3((uint32_t)((p.T + 255) / 256)), dim3(256), 0, st, h,
                       h_ld, (int32_t)p.H, (uint16_t *)at(p.hc), (int32_t)p.T);
    FG_TRY(hipGetLastError());
    h = (const uint16_t *)at(p.hc);
    h_ld = 8;
  }
  const SumArgs sum = {(const double *)at(p.lsum), nsum, r.found, c.totals, tiny, counts};
  bool summed = false;
  for (int64_t i = 0; i < p.pieces; ++i) {
    const int64_t row0 = i * p.Tc, rows = std::min(p.Tc, p.T - row0);
    const uint16_t *hc = r.hc + (size_t)row0 * p.Hp;
    double *lsum = (double *)at(p.lsum) + i * (p.Tc / p.slot);
    if (p.classes && rows > 0) {
      ClassArgs l{};
      l.w = w, l.h = h, l.w_ld = p.w_ld, l.h_ld = h_ld;
      l.wh = (int32_t)p.wh, l.V = (int32_t)p.V, l.T = (int32_t)p.T;
      l.found = r.found, l.mark = r.mark, l.target = c.target, l.weight = c.weight;
      l.e = c.grad ? (uint16_t *)at(p.e) : nullptr, l.Vp = (int32_t)p.Vp;
      l.loss = c.loss, l.lse = c.lse, l.lsum = lsum;
      l.count = counts.n || many.n ? (int32_t *)at(p.tcount) : nullptr;
      const bool sparse = p.T <= kSparse;
      FG_TRY(p.V <= 32    ? sparse ? (bf ? launch_classes<Bf16<PSparse32>>(l, st)
                                         : launch_classes<PSparse32>(l, st))
                                   : (bf ? launch_classes<Bf16<PClass32>>(l, st)
                                         : launch_classes<PClass32>(l, st))
             : p.V <= 64  ? sparse ? (bf ? launch_classes<Bf16<PSparse64>>(l, st)
                                         : launch_classes<PSparse64>(l, st))
                                   : (bf ? launch_classes<Bf16<PClass64>>(l, st)
                                         : launch_classes<PClass64>(l, st))
             : p.slot == 64 ? p.V <= 128 ? (bf ? launch_classes<Bf16<PHalf128>>(l, st)
                                               : launch_classes<PHalf128>(l, st))
                                         : (bf ? launch_classes<Bf16<PHalf256>>(l, st)
                                               : launch_classes<PHalf256>(l, st))
             : p.V <= 128 ? (bf ? launch_classes<Bf16<P128>>(l, st) : launch_classes<P128>(l, st))
                          : (bf ? launch_classes<Bf16<LogitTiles::T256>>(l, st)
                                : launch_classes<LogitTiles::T256>(l, st)));
      if (many.n) {
        hipLaunchKernelGGL(xent_totals_kernel, dim3(1), dim3(1024), 0, st, sum, many, r.found);
        FG_TRY(hipGetLastError());
        summed = true;
      }
    } else if (rows > 0) {
      LogitArgs l{};
      l.w = w, l.w_ld = p.w_ld, l.wh = (int32_t)p.wh, l.V = (int32_t)p.V;
      l.hc = stay ? h : hc, l.Hp = (int32_t)(stay ? h_ld : p.Hp);
      l.found = r.found, l.row0 = (int32_t)row0;
      l.Tc = (int32_t)(stay ? p.T : p.Tc), l.place = stay;
      if (stay && !p.tiny) l.all = all, l.mark = r.mark;
      l.ctarget = stay ? c.target : r.ctarget + row0;
      l.e = c.grad ? (uint16_t *)at(p.e) : nullptr, l.Vp = (int32_t)p.Vp;
      l.stats = (float2 *)at(p.stats), l.tlogit = (float *)at(p.tlogit);
      FG_TRY(FG_XENT_TILE(launch_logits, LogitTiles, p.s1.tile, bf, l, rows, st));
      SoftmaxArgs s{};
      s.found = r.found, s.row0 = (int32_t)row0, s.Tc = l.Tc, s.tiny = tiny;
      s.place = stay, s.mark = r.mark;
      s.V = (int32_t)p.V, s.Vp = (int32_t)p.Vp;
      s.tlog = 6 + p.s1.tile, s.ntile = (int32_t)p.ntile;
      s.bf = bf;
      s.idx = r.idx + row0, s.ctarget = l.ctarget;
      s.cweight = stay ? c.weight : r.cweight + row0;
      s.stats = l.stats, s.tlogit = l.tlogit, s.e = l.e;
      s.loss = c.loss, s.lse = c.lse, s.lsum = lsum;
      // workgroups: 2048, where the classes give as many ranges of 512
      const int64_t blocks = (rows + p.slot - 1) / p.slot;
      int64_t ny = c.grad ? std::min<int64_t>((p.Vp + 511) / 512,
                                              std::max<int64_t>(1, 2048 / blocks)) : 1;
      s.vper = (int32_t)up((p.Vp + ny - 1) / ny, 512);
      ny = c.grad ? (p.Vp + s.vper - 1) / s.vper : 1;
      if (!c.grad && p.pieces == 1 && blocks <= kTickets)
        s.totals = c.totals, s.nsum = nsum, summed = true;
      hipLaunchKernelGGL(p.slot == 4 ? xent_softmax_kernel<4> : xent_softmax_kernel<16>,
                         dim3((uint32_t)blocks, (uint32_t)ny), dim3(256), 0, st, s);
      FG_TRY(hipGetLastError());
    }
    if (!c.grad) continue;
    const bool last = i + 1 == p.pieces;
    Products g{};
    g.rows = rows;
    g.place = p.place;
    ProdArgs &a = g.dh;
    a.b = (const uint16_t *)at(p.e), a.b_ld = p.Vp;
    a.M = (int32_t)p.H, a.Mq = (int32_t)p.Hq;
    a.row0 = (int32_t)row0, a.Tc = (int32_t)(p.place ? p.T : p.Tc), a.found = r.found;
    a.V = (int32_t)p.V;
    a.mark = r.mark, a.tiny = tiny, a.counts = counts;
    JoinArgs &j = g.jdh;
    j.M = a.M, j.Mq = a.Mq, j.row0 = a.row0, j.Tc = a.Tc, j.found = r.found, j.bf = bf;
    j.tiny = tiny, j.counts = counts;
    g.dw = a, g.jdw = j;
    bool join_dh = false, join_dw = false;
    if (c.dh && rows > 0 && p.spread) {
      OuterArgs &o = g.outer;
      o.a = w, o.a_ld = p.w_ld, o.K = (int32_t)p.V, o.cols = (int32_t)p.wh;
      o.g = a.b, o.Vp = (int32_t)p.Vp, o.N = (int32_t)p.T, o.H = (int32_t)p.H;
      o.out = (uint16_t *)c.dh, o.out_ld = r.dh_ld;
      o.mark = r.mark, o.counts = counts, o.found = r.found;
    } else if (c.dh && rows > 0) {
      const bool split = p.s2.ns > 1;
      g.nsdh = p.s2.ns;
      a.a = w, a.a_ld = p.w_ld, a.a_rows = (int32_t)p.V, a.a_cols = (int32_t)p.wh;
      a.K = (int32_t)p.Vp, a.kper = p.s2.kper;
      a.idx = r.idx + row0;
      a.out = split ? nullptr : (uint16_t *)c.dh, a.out_ld = r.dh_ld;
      a.part = split ? (float *)at(p.pdh) : nullptr, a.pstride = p.Tc * p.Hq;
      j.part = a.part, j.pstride = a.pstride, j.nsplit = p.s2.ns;
      j.rows = p.place ? (int32_t)p.T : -1;
      j.idx = p.place ? nullptr : a.idx, j.mark = r.mark, j.masked = p.place;
      j.out = (uint16_t *)c.dh, j.out_ld = a.out_ld;
      join_dh = split;
    }
    if (c.dw && p.outer) {
      OuterArgs &o = g.outer;
      o.a = h, o.a_ld = h_ld, o.K = tiny.T, o.cols = (int32_t)p.wh;
      o.g = a.b, o.Vp = (int32_t)p.Vp, o.N = (int32_t)p.V, o.H = (int32_t)p.H;
      o.out = (uint16_t *)c.dw, o.out_ld = d.dw_ld ? d.dw_ld : d.hidden;
      o.flag = c.flag, o.tiny = tiny;
    } else if (c.dw) {
      ProdArgs &b = g.dw;
      JoinArgs &q = g.jdw;
      const bool split = p.s3.ns > 1;
      g.nsdw = p.s3.ns;
      b.a = p.place ? h : hc, b.a_ld = p.place ? h_ld : p.Hp;
      b.a_rows = (int32_t)(p.place ? p.T : p.Tc), b.a_cols = (int32_t)p.wh;
      b.N = (int32_t)p.Vp;
      b.K = (int32_t)p.Tc, b.kper = p.s3.kper;
      b.out = split || !last ? nullptr : (uint16_t *)c.dw;
      b.out_ld = d.dw_ld ? d.dw_ld : d.hidden;
      b.part = split || p.pieces > 1 ? (float *)at(p.pdw) : nullptr, b.pstride = p.V * p.Hq;
      b.add = i > 0;
      b.flag = c.flag;
      q.part = b.part, q.pstride = b.pstride, q.nsplit = p.s3.ns, q.rows = (int32_t)p.V;
      q.out = (uint16_t *)c.dw, q.out_ld = b.out_ld, q.flag = c.flag;
      join_dw = split && last;
    }
    if (g.nsdh || g.nsdw) {
      if (c.totals && last && !summed && nsum <= kSumHere) {
        g.sum = sum;
        summed = nsum > 0;
      }
      FG_TRY(FG_XENT_TILE(launch_products, ProdTiles, p.s2.tile, bf, g, st));
    }
    if (g.outer.out && p.spread)
      FG_TRY((bf ? launch_outer<Bf16<POuter>, true> : launch_outer<POuter, true>)(g, join_dw, st));
    else if (g.outer.out)
      FG_TRY((bf ? launch_outer<Bf16<POuter>, false> : launch_outer<POuter, false>)(g, join_dh, st));
    else
      FG_TRY(launch_join(g, join_dh, join_dw, st));
  }
  if (c.totals && !summed) {
    hipLaunchKernelGGL(xent_totals_kernel, dim3(1), dim3(1024), 0, st, sum, Counts{}, r.found);
    FG_TRY(hipGetLastError());
  }
  return hipSuccess;
}

}  // namespace xent

size_t linear_xent_ws_bytes(const fg_xent_desc &d, bool grad) {
  return xent::make_plan(d, grad).total;
}

hipError_t launch_linear_xent(const fg_xent_desc &d, const void *h, const void *w,
                              const int32_t *target, const float *weight, float *loss,
                              float *lse, float *totals, void *dh, void *dw, int32_t *flag,
                              bool grad, void *ws, hipStream_t st) {
  return xent::run(d, {h, w, target, weight, loss, lse, totals, dh, dw, flag, grad}, ws, st);
}

}  // namespace fg
