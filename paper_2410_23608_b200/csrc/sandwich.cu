// The norms around a block (Sec. 3.2 names the block's branch and its residual; the paper does not describe its norms): the
// branch's result z is normalised, gated, scaled and added to the residual stream x, and the sum is normalised for what follows:
//   a_t = scale * gate_t * (g_post zh_t + b_post),  zh_t = norm(z_row(t));  y_t = x_t + a_t;  n_t = g_pre norm(y_t) + b_pre.
// norm is LayerNorm or RMS.  Rows of z may be packed: a token without one passes x on.
//
// Backward, with d = dy + (gradient of n through its norm), which is dx:  da = d gate scale, dz = gradient of da g_post through
// its norm.  Everything that is summed over rows follows from two sums per channel, A = sum d gate zh and B = sum d gate:
// dg_post = scale A, db_post = scale B, dscale = g_post A + b_post B; with a gate per image, from A_b = sum d zh and
// B_b = sum d over its rows: dgate_b = scale (g_post A_b + b_post B_b), A = sum_b gate_b A_b.  So four running sums per channel
// (the other two: sum dn yh, sum dn) in registers serve six gradients.
//
// Both directions are bound by bytes, and nearly as much by the instructions on a row: in the backward's first form, every value
// converted and every parameter read again in each of its three steps, 18 432 rows of 768 took 102 us against 26 for their
// bytes.  So a row belongs to as many warps as leave a thread one 16-byte chunk (two beyond 512 chunks), arithmetic is on pairs of
// fp32, products of parameters are held in registers, and the next row's loads are on their way under the arithmetic of
// a row.  Statistics and sums are fp32; y and n are rounded once, n from the unrounded y.  Normalised values are (v - m) r: as v r - m r,
// with m r rounded, they lost as many bits as the mean has deviations.  Sums run in a fixed order: results
// are bitwise reproducible.
#include "simt_stage.cuh"
#include "sm100_ptx.cuh"
#include "spa_common.cuh"

namespace spa {
namespace {

using ptx::add2;
using ptx::fma2;
using ptx::mul2;
using ptx::pair;
using ptx::unpair;

constexpr int kMaxChunks = 1024;  // 16-byte chunks of a row: 8 192 bf16 or 4 096 fp32 channels
constexpr int kSums = 4;          // running sums per channel of the backward: A, B, sum dn yh, sum dn
// Rows that a CTA has under way with W warps to a row, and its threads.  Backward: one CTA per SM, whose sums are one line to join.
__host__ __device__ constexpr int groups_of(int W, bool bwd) {
  return bwd ? (W == 1 ? 12 : W == 2 ? 6 : W == 3 ? 4 : W == 4 ? 3 : W <= 8 ? 2 : 1) : (W == 1 ? 8 : W == 2 ? 4 : W == 3 ? 3 : W <= 6 ? 2 : 1);
}
__host__ __device__ constexpr int threads_of(int W, bool bwd) { return 32 * W * groups_of(W, bwd); }

struct Args {
  const uint4 *x, *z, *dn, *dy, *y;   // rows of Q chunks; dn, dy optional
  const int32_t* z_row;               // optional
  const void* gate;
  const uint4 *scale, *g_post, *b_post, *g_pre, *b_pre;  // optional
  float* stats;                       // [4][rows]: mean and 1 / deviation of z's row, of y's
  uint4 *out_y, *out_n;               // forward
  uint4 *dx, *dz;                     // backward
  void* dgate;
  float *part, *part_gate;            // per CTA [kSums][C]; per unit of an image's rows [2][C]
  int rows, N, Q, C, z_rows, kind, rows_per_cta;
  unsigned long long n_magic;         // t / N = t * n_magic >> 40 for t, N <= 2^20: n_magic = 2^40 / N + 1 is off by N / 2^40 at most
  bool gate_f32;                      // dgate of a gate per token: fp32
  float eps;
};

// The rows that a group has on their way, in shared memory: a thread copies its own chunks of the kA arrays of a row, asynchronously,
// kDepth rows ahead (registers hold one row ahead at most: 16 rows of 1.5 KB per SM in flight instead of 64, 18 432 rows of 768
// backward 47 us), and its warp's first lanes the row's scalars.  Nobody else reads them but the warp.
__device__ __forceinline__ uint4 lds16(uint32_t at) {
  uint4 v;
  asm volatile("ld.shared.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(at) : "memory");
  return v;
}
__device__ __forceinline__ void sts16(uint32_t at, const uint4& v) {
  asm volatile("st.shared.v4.u32 [%0], {%1, %2, %3, %4};" ::"r"(at), "r"(v.x), "r"(v.y), "r"(v.z), "r"(v.w) : "memory");
}
template <int kA, int kCh, int kDepth, int kThreads, int kRows = 1> struct Ring {
  static constexpr int kSlot = kA * kCh * kThreads * 16, kScalars = kThreads / 32 * 32 * kRows;  // kA: of all kRows rows of a slot
  static constexpr int kBytes = kDepth * (kSlot + kScalars);
  uint32_t base, at, scalar;  // addresses in shared memory: the ring's, this thread's first chunk and its warp's scalars of the slot
  __device__ __forceinline__ explicit Ring(uint32_t b) : base(b) { rewind(); }
  __device__ __forceinline__ void rewind() {
    at = base + threadIdx.x * 16;
    scalar = base + kDepth * kSlot + (threadIdx.x >> 5) * 32 * kRows;
  }
  __device__ __forceinline__ void next() {
    at += kSlot;
    scalar += kScalars;
    if (at >= base + kDepth * kSlot) rewind();
  }
  static constexpr int kArray = kCh * kThreads * 16, kChunk = kThreads * 16;
  __device__ __forceinline__ void copy(int array, int k, const uint4* from) const {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(at + array * kArray + k * kChunk), "l"(__cvta_generic_to_global(from)) : "memory");
  }
  __device__ __forceinline__ void copy_scalar(int i, const float* from) const {
    asm volatile("cp.async.ca.shared.global [%0], [%1], 4;" ::"r"(scalar + 4 * i), "l"(__cvta_generic_to_global(from)) : "memory");
  }
  __device__ __forceinline__ uint4 get(int array, int k) const { return lds16(at + array * kArray + k * kChunk); }
  __device__ __forceinline__ float4 scalars(int row = 0) const {  // eight floats a row
    const uint4 v = lds16(scalar + 32 * row);
    return make_float4(__uint_as_float(v.x), __uint_as_float(v.y), __uint_as_float(v.z), __uint_as_float(v.w));
  }
  __device__ __forceinline__ float fifth(int row) const { return ptx::lds_f32(scalar + 32 * row + 16); }
  // Chunks past the end of a row are never copied: they are read as zeros, like the others, when they have been cleared once.
  __device__ __forceinline__ void clear(int t0, int stride, int Q) {
    for (int slot = 0; slot < kDepth; ++slot, next())
#pragma unroll
      for (int k = 0; k < kCh; ++k)
        if (t0 + stride * k >= Q) {
#pragma unroll
          for (int i = 0; i < kA; ++i) sts16(at + i * kArray + k * kChunk, make_uint4(0u, 0u, 0u, 0u));
        }
  }
};

// Sums of kN values over the group's threads, in every one of them.  Two or four values go through a warp together: each step
// leaves every lane half of the values it had, so that 6 shuffles serve four values instead of 20.  Calls alternate between two
// lines of shared memory: a warp that writes a line again has met the others at the barrier in between, behind their reads of it.
template <int W> struct GroupSum {
  uint32_t line, other;  // [W][8] floats of this group each
  int id, warp, lane;
  template <int kN> __device__ __forceinline__ void operator()(float (&v)[kN]) {
    static_assert(kN <= 4 || kN == 6, "a line has room for eight, in fours, twos and ones");
    if constexpr (W == 1 && kN == 1) {
      v[0] = warp_sum(v[0]);
    } else {
      const uint32_t mine = line + 32 * warp;
      constexpr int k4 = kN / 4 * 4, k2 = (kN - k4) / 2 * 2;
      if constexpr (k4 == 4) {
        const bool up = (lane & 16) != 0, up8 = (lane & 8) != 0;
        float a = (up ? v[1] : v[0]) + __shfl_xor_sync(0xffffffffu, up ? v[0] : v[1], 16);
        float b = (up ? v[3] : v[2]) + __shfl_xor_sync(0xffffffffu, up ? v[2] : v[3], 16);
        a = (up8 ? b : a) + __shfl_xor_sync(0xffffffffu, up8 ? a : b, 8);
#pragma unroll
        for (int o = 4; o > 0; o >>= 1) a += __shfl_xor_sync(0xffffffffu, a, o);
        if ((lane & 7) == 0) ptx::sts_s32(mine + 4 * ((lane >> 4) + ((lane >> 2) & 2)), __float_as_int(a));
      }
      if constexpr (k2 == 2) {
        const bool up = (lane & 16) != 0;
        float a = (up ? v[k4 + 1] : v[k4]) + __shfl_xor_sync(0xffffffffu, up ? v[k4] : v[k4 + 1], 16);
#pragma unroll
        for (int o = 8; o > 0; o >>= 1) a += __shfl_xor_sync(0xffffffffu, a, o);
        if ((lane & 15) == 0) ptx::sts_s32(mine + 4 * (k4 + (lane >> 4)), __float_as_int(a));
      }
      if constexpr (kN - k4 - k2 == 1) {
        const float a = warp_sum(v[kN - 1]);
        if (lane == 0) ptx::sts_s32(mine + 4 * (kN - 1), __float_as_int(a));
      }
      if constexpr (W > 1) asm volatile("bar.sync %0, %1;" ::"r"(id + 1), "n"(32 * W) : "memory");
      else __syncwarp();
#pragma unroll
      for (int w = 0; w < W; ++w) {
        const uint4 l = lds16(line + 32 * w);
        float f[8] = {__uint_as_float(l.x), __uint_as_float(l.y), __uint_as_float(l.z), __uint_as_float(l.w)};
        if constexpr (kN > 4) {
          const uint4 m = lds16(line + 32 * w + 16);
          f[4] = __uint_as_float(m.x);
          f[5] = __uint_as_float(m.y);
        }
#pragma unroll
        for (int i = 0; i < kN; ++i) v[i] = w == 0 ? f[i] : v[i] + f[i];
      }
      const uint32_t t = line;
      line = other;
      other = t;
    }
  }
};

// A chunk as pairs of fp32 and back
template <typename T> constexpr int kPairs = Vec16<T>::kElems / 2;
__device__ __forceinline__ void to_pairs(const uint4& v, uint64_t (&p)[2]) {
  p[0] = pair(v.x, v.y);
  p[1] = pair(v.z, v.w);
}
__device__ __forceinline__ void to_pairs(const uint4& v, uint64_t (&p)[4]) {
  const uint32_t w[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) p[i] = pair(w[i] << 16, w[i] & 0xffff0000u);
}
__device__ __forceinline__ uint4 from_pairs(const uint64_t (&p)[2]) {
  uint4 v;
  unpair(p[0], v.x, v.y);
  unpair(p[1], v.z, v.w);
  return v;
}
__device__ __forceinline__ uint4 from_pairs(const uint64_t (&p)[4]) {
  uint32_t w[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    float a, b;
    unpair(p[i], a, b);
    w[i] = ptx::bf16_pair(a, b);
  }
  return make_uint4(w[0], w[1], w[2], w[3]);
}
__device__ __forceinline__ uint64_t both(float v) { return pair(v, v); }
__device__ __forceinline__ float sum_of(uint64_t p) {
  float a, b;
  unpair(p, a, b);
  return a + b;
}

// A chunk of a parameter, `fill` where it is absent
template <typename T> __device__ __forceinline__ void param(const uint4* p, int q, bool in, float fill, uint64_t (&v)[kPairs<T>]) {
  if (p != nullptr && in) {
    to_pairs(p[q], v);
  } else {
#pragma unroll
    for (int i = 0; i < kPairs<T>; ++i) v[i] = both(fill);
  }
}

__device__ __forceinline__ float sigmoid(float s) { return 1.f / (1.f + expf(-s)); }

template <int kGate> constexpr bool kGateRows = kGate == SPA_GATE_IMAGE || kGate == SPA_GATE_TOKEN;  // gates of C values

template <int kGate> constexpr int kFwdArrays = kGateRows<kGate> ? 3 : 2;
constexpr int kFwdDepth = 4;

template <typename T, int W, int kCh, int kGate>
__global__ void __launch_bounds__(threads_of(W, false), kCh == 1 ? 1024 / threads_of(W, false) : 1) sandwich_fwd_kernel(const Args a) {
  pdl_entry();
  constexpr int P = kPairs<T>, G = 32 * W;
  __shared__ __align__(16) float red[groups_of(W, false) * 16 * W];
  const int grp = threadIdx.x / G, t0 = threadIdx.x % G;
  const uint32_t lines = ptx::smem_u32(red + grp * 16 * W);
  GroupSum<W> sum{lines, lines + 32 * W, grp, t0 >> 5, (int)threadIdx.x & 31};
  const float inv_c = 1.f / a.C;
  const bool layer = a.kind == SPA_NORM_LAYER;
  // y = x + gate (cw zh + cb), n = cp norm(y) + bp
  uint64_t cw[kCh][P], cb[kCh][P], cp[kCh][P], bp[kCh][P];
#pragma unroll
  for (int k = 0; k < kCh; ++k) {
    const int q = t0 + G * k;
    const bool in = q < a.Q;
    uint64_t sc[P];
    param<T>(a.scale, q, in, 1.f, sc);
    param<T>(a.g_post, q, in, 1.f, cw[k]);
    param<T>(a.b_post, q, in, 0.f, cb[k]);
    param<T>(a.g_pre, q, in, 1.f, cp[k]);
    param<T>(a.b_pre, q, in, 0.f, bp[k]);
#pragma unroll
    for (int i = 0; i < P; ++i) { cw[k][i] = mul2(cw[k][i], sc[i]); cb[k][i] = mul2(cb[k][i], sc[i]); }
  }
  // mean (0 for RMS) and 1 / deviation of the row v, whose chunks past the end are zero; its chunks without the mean
  auto statistics = [&](uint64_t (&v)[kCh][P], float& mean, float& rstd) {
    mean = 0.f;
    if (layer) {
      uint64_t s = 0ull;
#pragma unroll
      for (int k = 0; k < kCh; ++k)
#pragma unroll
        for (int i = 0; i < P; ++i) s = add2(s, v[k][i]);
      float t[1] = {sum_of(s)};
      sum(t);
      mean = t[0] * inv_c;
    }
    const uint64_t m = both(-mean);
    uint64_t ss = 0ull;
#pragma unroll
    for (int k = 0; k < kCh; ++k)
      if (t0 + G * k < a.Q) {
#pragma unroll
        for (int i = 0; i < P; ++i) { v[k][i] = add2(v[k][i], m); ss = fma2(v[k][i], v[k][i], ss); }
      }
    float t[1] = {sum_of(ss)};
    sum(t);
    rstd = rsqrtf(t[0] * inv_c + a.eps);
  };
  extern __shared__ __align__(16) uint8_t ring_s[];
  Ring<kFwdArrays<kGate>, kCh, kFwdDepth, threads_of(W, false)> ring(ptx::smem_u32(ring_s));
  auto row_of = [&](int t) { return a.z_row != nullptr && t < a.rows ? ld_dep(a.z_row + t) : t; };
  auto has_row = [&](int zr) { return zr >= 0 && zr < a.z_rows; };
  auto fetch = [&](int t, int zr) {
    if (t < a.rows) {
      // places in chunks: below 2^30
      const unsigned at = t * a.Q + t0, zat = zr * a.Q + t0;
      const unsigned gat = kGate == SPA_GATE_IMAGE ? (unsigned)((unsigned long long)t * a.n_magic >> 40) * a.Q + t0 : at;
#pragma unroll
      for (int k = 0; k < kCh; ++k) {
        if (t0 + G * k < a.Q) {
          ring.copy(0, k, a.x + (at + G * k));
          if (has_row(zr)) {
            ring.copy(1, k, a.z + (zat + G * k));
            if (kGateRows<kGate>) ring.copy(kGateRows<kGate> ? 2 : 0, k, static_cast<const uint4*>(a.gate) + (gat + G * k));
          }
        }
      }
      if (kGate == SPA_GATE_SCORE && sum.lane == 0) ring.copy_scalar(0, static_cast<const float*>(a.gate) + t);
    }
    cp_async_commit();
  };
  const int step = gridDim.x * groups_of(W, false);
  int t = blockIdx.x * groups_of(W, false) + grp;
  ring.clear(t0, G, a.Q);
  int zr[kFwdDepth + 1];  // rows of z of the tokens on their way, and of one more
#pragma unroll
  for (int i = 0; i <= kFwdDepth; ++i) zr[i] = row_of(t + i * step);
#pragma unroll
  for (int i = 0; i < kFwdDepth; ++i) {
    fetch(t + i * step, zr[i]);
    ring.next();
  }
  for (; t < a.rows; t += step) {
    const bool has = has_row(zr[0]);
    cp_async_wait<kFwdDepth - 1>();
    __syncwarp();
    uint4 xr[kCh], zv[kCh], gr[kCh];
#pragma unroll
    for (int k = 0; k < kCh; ++k) {
      xr[k] = ring.get(0, k);
      zv[k] = ring.get(1, k);  // without a row: what was there, and is not used
      if (kGateRows<kGate>) gr[k] = ring.get(kGateRows<kGate> ? 2 : 0, k);
    }
    const float score = kGate == SPA_GATE_SCORE ? ring.scalars().x : 0.f;
    __syncwarp();
    fetch(t + kFwdDepth * step, zr[kFwdDepth]);
    ring.next();
#pragma unroll
    for (int i = 0; i < kFwdDepth; ++i) zr[i] = zr[i + 1];
    zr[kFwdDepth] = row_of(t + (kFwdDepth + 1) * step);
    uint64_t v[kCh][P];
    float m1 = 0.f, r1 = 0.f, m2 = 0.f, r2 = 0.f;
    const unsigned at = t * a.Q + t0;
    if (has) {
#pragma unroll
      for (int k = 0; k < kCh; ++k) to_pairs(zv[k], v[k]);
      statistics(v, m1, r1);
      const uint64_t r = both(r1), w = both(kGate == SPA_GATE_SCORE ? sigmoid(score) : 1.f);
#pragma unroll
      for (int k = 0; k < kCh; ++k) {
        uint64_t x[P], g[P];
        to_pairs(xr[k], x);
        if (kGateRows<kGate>) to_pairs(gr[k], g);
#pragma unroll
        for (int i = 0; i < P; ++i) {
          const uint64_t b = fma2(mul2(v[k][i], r), cw[k][i], cb[k][i]);
          v[k][i] = kGate == SPA_GATE_NONE ? add2(b, x[i]) : fma2(b, kGateRows<kGate> ? g[i] : w, x[i]);
        }
        if (t0 + G * k < a.Q) a.out_y[at + G * k] = from_pairs(v[k]);
        else {
#pragma unroll
          for (int i = 0; i < P; ++i) v[k][i] = 0ull;
        }
      }
    } else {
#pragma unroll
      for (int k = 0; k < kCh; ++k) {
        to_pairs(xr[k], v[k]);
        if (t0 + G * k < a.Q) a.out_y[at + G * k] = xr[k];
      }
    }
    if (a.out_n != nullptr) {
      statistics(v, m2, r2);
      const uint64_t r = both(r2);
#pragma unroll
      for (int k = 0; k < kCh; ++k) {
        if (t0 + G * k < a.Q) {
#pragma unroll
          for (int i = 0; i < P; ++i) v[k][i] = fma2(mul2(v[k][i], r), cp[k][i], bp[k][i]);
          a.out_n[at + G * k] = from_pairs(v[k]);
        }
      }
    }
    if (t0 == 0 && a.stats != nullptr) {
      a.stats[t] = m1;
      a.stats[a.rows + t] = r1;
      a.stats[2 * a.rows + t] = m2;
      a.stats[3 * a.rows + t] = r2;
    }
  }
}

template <int kGate> constexpr int kBwdArrays = kGate == SPA_GATE_TOKEN ? 5 : 4;
// Rows that a group takes together, whose sums share shuffles and barriers: a row's steps depend on one another, and with one at a time
// 18 432 rows of 768 took 43 us whatever their bytes.  And how many such steps ahead they are copied.
// Two need 168 registers, so CTAs of 384 threads: 18 432 rows of 768 46.5 -> 44 us, 9 216 of 1 536 51 -> 46; with CTAs of 512 (8 and 16
// warps to a row) they spill: 8 184 rows of 4 096 109 -> 120.
template <int W, int kCh> constexpr int kBwdRows = kCh == 1 && W != 8 && W != 16 ? 2 : 1;
template <int W, int kCh> constexpr int kBwdDepth = kCh == 1 && kBwdRows<W, kCh> == 1 ? 3 : 2;

// A CTA has a share of the rows, one behind the other.  With a gate per image the sums A_b and B_b leave it at the end of each image
// or share: the line of image b from CTA c is line b + c, since one of the two goes up from each to the next.
template <typename T, int W, int kCh, int kGate>
__global__ void __launch_bounds__(threads_of(W, true), 1) sandwich_bwd_kernel(const Args a) {
  pdl_entry();
  constexpr int P = kPairs<T>, G = 32 * W, kG = groups_of(W, true);
  constexpr bool kImage = kGate == SPA_GATE_IMAGE;
  constexpr int kDepth = kBwdDepth<W, kCh>, R = kBwdRows<W, kCh>, kStep = kG * R;
  using Rows = Ring<kBwdArrays<kGate> * R, kCh, kDepth, threads_of(W, true), R>;
  // the ring, and in its place, when it is empty, [kG][2][C] sums; behind them, with a gate per image, [2][C]: sum of gate_b A_b,
  // of gate_b B_b
  extern __shared__ __align__(16) uint8_t smem[];
  float* acc_s = reinterpret_cast<float*>(smem);
  __shared__ __align__(16) float red[kG * 16 * W];
  const int grp = threadIdx.x / G, t0 = threadIdx.x % G;
  const uint32_t lines = ptx::smem_u32(red + grp * 16 * W);
  GroupSum<W> sum{lines, lines + 32 * W, grp, t0 >> 5, (int)threadIdx.x & 31};
  const float inv_c = 1.f / a.C;
  const bool layer = a.kind == SPA_NORM_LAYER;
  uint64_t sA[kCh][P] = {}, sB[kCh][P] = {}, sG[kCh][P] = {}, sN[kCh][P] = {};
  const int acc_bytes = kG * 2 * a.C * 4;
  float* run = reinterpret_cast<float*>(smem + (acc_bytes > Rows::kBytes ? acc_bytes : Rows::kBytes));
  if (kImage)
    for (int c = threadIdx.x; c < 2 * a.C; c += threads_of(W, true)) run[c] = 0.f;
  // two running sums of every group, added up in the order of the groups, to out(c, first, second)
  auto join = [&](const uint64_t (&u)[kCh][P], const uint64_t (&w)[kCh][P], auto out) {
    __syncthreads();
    float* mine = acc_s + grp * 2 * a.C;
#pragma unroll
    for (int k = 0; k < kCh; ++k) {
      const int q = t0 + G * k;
      if (q < a.Q) {
#pragma unroll
        for (int i = 0; i < P; i += 2) {
          *reinterpret_cast<ulonglong2*>(mine + (q * P + i) * 2) = make_ulonglong2(u[k][i], u[k][i + 1]);
          *reinterpret_cast<ulonglong2*>(mine + a.C + (q * P + i) * 2) = make_ulonglong2(w[k][i], w[k][i + 1]);
        }
      }
    }
    __syncthreads();
    for (int c = threadIdx.x; c < a.C; c += threads_of(W, true)) {
      float s = 0.f, r = 0.f;
#pragma unroll
      for (int g = 0; g < kG; ++g) { s += acc_s[g * 2 * a.C + c]; r += acc_s[g * 2 * a.C + a.C + c]; }
      out(c, s, r);
    }
  };
  // gz = d gate cw; a / gate = cw zh + cb (for the gradient of a gate that is not per image)
  uint64_t cp[kCh][P], cw[kCh][P], cb[kCh][P];
  auto products = [&](const uint4* gate) {  // with a gate per image, cw holds the image's gate too
#pragma unroll
    for (int k = 0; k < kCh; ++k) {
      const int q = t0 + G * k;
      const bool in = q < a.Q;
      uint64_t sc[P], g[P];
      param<T>(a.scale, q, in, 1.f, sc);
      param<T>(a.g_post, q, in, 1.f, cw[k]);
      param<T>(a.b_post, q, in, 0.f, cb[k]);
      if (kImage) param<T>(gate, q, in, 0.f, g);
#pragma unroll
      for (int i = 0; i < P; ++i) {
        cw[k][i] = mul2(cw[k][i], kImage ? mul2(sc[i], g[i]) : sc[i]);
        cb[k][i] = mul2(cb[k][i], sc[i]);
      }
    }
  };
#pragma unroll
  for (int k = 0; k < kCh; ++k) param<T>(a.g_pre, t0 + G * k, t0 + G * k < a.Q, 1.f, cp[k]);
  if (!kImage) products(nullptr);
  Rows ring(ptx::smem_u32(smem));
  auto has_row = [&](int zr) { return zr >= 0 && zr < a.z_rows; };
  const int share = blockIdx.x * a.rows_per_cta, share_end = share + a.rows_per_cta < a.rows ? share + a.rows_per_cta : a.rows;
  for (int begin = share, end; begin < share_end; begin = end) {
    const int image = kImage ? begin / a.N : 0;
    end = kImage && (image + 1) * a.N < share_end ? (image + 1) * a.N : share_end;
    if (kImage) products(static_cast<const uint4*>(a.gate) + (long long)image * a.Q);
    auto row_of = [&](int t) { return a.z_row != nullptr && t < end ? ld_dep(a.z_row + t) : t; };
    auto fetch = [&](int t, const int (&zr)[R]) {
#pragma unroll
      for (int r = 0; r < R; ++r, t += kG) {
        if (t >= end) continue;
        const bool has = has_row(zr[r]);
        const unsigned at = t * a.Q + t0, zat = zr[r] * a.Q + t0;  // places in chunks: below 2^30
#pragma unroll
        for (int k = 0; k < kCh; ++k) {
          if (t0 + G * k < a.Q) {
            if (a.dn != nullptr) {
              ring.copy(r, k, a.dn + (at + G * k));
              ring.copy(R + r, k, a.y + (at + G * k));
            }
            if (a.dy != nullptr) ring.copy(2 * R + r, k, a.dy + (at + G * k));
            if (has) {
              ring.copy(3 * R + r, k, a.z + (zat + G * k));
              if (kGate == SPA_GATE_TOKEN) ring.copy(kGate == SPA_GATE_TOKEN ? 4 * R + r : 0, k, static_cast<const uint4*>(a.gate) + (at + G * k));
            }
          }
        }
        if (sum.lane < 4) ring.copy_scalar(8 * r + sum.lane, a.stats + (unsigned)(sum.lane * a.rows + t));
        if (kGate == SPA_GATE_SCORE && sum.lane == 4) ring.copy_scalar(8 * r + 4, static_cast<const float*>(a.gate) + t);
      }
      cp_async_commit();
    };
    ring.clear(t0, G, a.Q);
    int t = begin + grp, zr[kDepth + 1][R];  // rows of z of the tokens on their way, and of the next ones
#pragma unroll
    for (int i = 0; i <= kDepth; ++i)
#pragma unroll
      for (int r = 0; r < R; ++r) zr[i][r] = row_of(t + i * kStep + r * kG);
#pragma unroll
    for (int i = 0; i < kDepth; ++i) {
      fetch(t + i * kStep, zr[i]);
      ring.next();
    }
    for (; t < end; t += kStep) {
      cp_async_wait<kDepth - 1>();
      __syncwarp();
      const uint4 zero = make_uint4(0u, 0u, 0u, 0u);
      uint4 nr[R][kCh], yr[R][kCh], dr[R][kCh], zv[R][kCh], gr[R][kGate == SPA_GATE_TOKEN ? kCh : 1];
      float m1[R], r1[R], m2[R], r2[R], score[R];
      bool has[R], there[R];
      unsigned at[R], zat[R];
#pragma unroll
      for (int r = 0; r < R; ++r) {
        there[r] = r == 0 || t + r * kG < end;
        has[r] = there[r] && has_row(zr[0][r]);
        at[r] = (t + r * kG) * a.Q + t0;
        zat[r] = zr[0][r] * a.Q + t0;
#pragma unroll
        for (int k = 0; k < kCh; ++k) {
          nr[r][k] = ring.get(r, k);
          yr[r][k] = ring.get(R + r, k);
          dr[r][k] = ring.get(2 * R + r, k);
          zv[r][k] = ring.get(3 * R + r, k);
          if constexpr (kGate == SPA_GATE_TOKEN) gr[r][k] = ring.get(4 * R + r, k);
        }
        const float4 sc = ring.scalars(r);
        m1[r] = sc.x;
        r1[r] = sc.y;
        m2[r] = sc.z;
        r2[r] = sc.w;
        score[r] = kGate == SPA_GATE_SCORE ? ring.fifth(r) : 0.f;
        // what was not copied: whatever was there
        if (!there[r] || a.dn == nullptr) {
          m2[r] = r2[r] = 0.f;
#pragma unroll
          for (int k = 0; k < kCh; ++k) nr[r][k] = yr[r][k] = zero;
        }
        if (!there[r] || a.dy == nullptr) {
#pragma unroll
          for (int k = 0; k < kCh; ++k) dr[r][k] = zero;
        }
        if (!has[r]) {
          m1[r] = r1[r] = 0.f;
#pragma unroll
          for (int k = 0; k < kCh; ++k) {
            zv[r][k] = zero;
            if constexpr (kGate == SPA_GATE_TOKEN) gr[r][k] = zero;
          }
        }
      }
      __syncwarp();
      fetch(t + kDepth * kStep, zr[kDepth]);
      ring.next();
#pragma unroll
      for (int r = 0; r < R; ++r) {
#pragma unroll
        for (int i = 0; i < kDepth; ++i) zr[i][r] = zr[i + 1][r];
        zr[kDepth][r] = row_of(t + (kDepth + 1) * kStep + r * kG);
      }
      // ---- through the norm behind the sum: d, the gradient of y
      uint64_t d[R][kCh][P];
      if (a.dn != nullptr) {
        uint64_t yh[R][kCh][P];
        float s[2 * R];
#pragma unroll
        for (int r = 0; r < R; ++r) {
          const uint64_t rs = both(r2[r]), m = both(-m2[r]);
          uint64_t s1 = 0ull, s2 = 0ull;
#pragma unroll
          for (int k = 0; k < kCh; ++k) {
            uint64_t n[P];
            to_pairs(nr[r][k], n);
            to_pairs(yr[r][k], yh[r][k]);
#pragma unroll
            for (int i = 0; i < P; ++i) {  // chunks past the end: n is zero
              yh[r][k][i] = mul2(add2(yh[r][k][i], m), rs);
              sG[k][i] = fma2(n[i], yh[r][k][i], sG[k][i]);
              sN[k][i] = add2(sN[k][i], n[i]);
              d[r][k][i] = mul2(n[i], cp[k][i]);
              s1 = add2(s1, d[r][k][i]);
              s2 = fma2(d[r][k][i], yh[r][k][i], s2);
            }
          }
          s[2 * r] = sum_of(s1);
          s[2 * r + 1] = sum_of(s2);
        }
        sum(s);
        // d = dy + (g - mean g - yh mean(g yh)) / deviation
#pragma unroll
        for (int r = 0; r < R; ++r) {
          const uint64_t rs = both(r2[r]), a1 = both(layer ? -s[2 * r] * inv_c * r2[r] : 0.f), a2 = both(-s[2 * r + 1] * inv_c * r2[r]);
#pragma unroll
          for (int k = 0; k < kCh; ++k) {
            uint64_t y[P];
            to_pairs(dr[r][k], y);
#pragma unroll
            for (int i = 0; i < P; ++i) d[r][k][i] = add2(y[i], fma2(d[r][k][i], rs, fma2(yh[r][k][i], a2, a1)));
          }
        }
      } else {
#pragma unroll
        for (int r = 0; r < R; ++r)
#pragma unroll
          for (int k = 0; k < kCh; ++k) to_pairs(dr[r][k], d[r][k]);
      }
      // ---- through gate, scale and the norm in front of the sum
      constexpr int kU = kGate == SPA_GATE_SCORE ? 3 : 2;
      uint64_t zh[R][kCh][P];
      float u[kU * R];
#pragma unroll
      for (int r = 0; r < R; ++r) {
        if (kGate == SPA_GATE_SCORE) score[r] = has[r] ? sigmoid(score[r]) : 0.f;  // without a row it may be NaN, or was not copied
        const uint64_t rs = both(r1[r]), m = both(-m1[r]), w = both(score[r]);
        uint64_t u1 = 0ull, u2 = 0ull, u3 = 0ull;
#pragma unroll
        for (int k = 0; k < kCh; ++k) {
          const bool in = t0 + G * k < a.Q;
          if (in && there[r]) a.dx[at[r] + G * k] = from_pairs(d[r][k]);
          uint64_t g[P];
          to_pairs(zv[r][k], zh[r][k]);
          if constexpr (kGate == SPA_GATE_TOKEN) to_pairs(gr[r][k], g);
#pragma unroll
          for (int i = 0; i < P; ++i) {
            if (!in || !has[r]) d[r][k][i] = 0ull;  // past the end: the means' part; without a row: nothing
            zh[r][k][i] = mul2(add2(zh[r][k][i], m), rs);
            if (kGate == SPA_GATE_SCORE) u3 = fma2(d[r][k][i], fma2(zh[r][k][i], cw[k][i], cb[k][i]), u3);
            if constexpr (kGate == SPA_GATE_TOKEN) {
              const uint64_t dg = mul2(d[r][k][i], fma2(zh[r][k][i], cw[k][i], cb[k][i]));
              d[r][k][i] = mul2(d[r][k][i], g[i]);
              g[i] = dg;
            }
            if (kGate == SPA_GATE_SCORE) d[r][k][i] = mul2(d[r][k][i], w);
            sA[k][i] = fma2(d[r][k][i], zh[r][k][i], sA[k][i]);
            sB[k][i] = add2(sB[k][i], d[r][k][i]);
            d[r][k][i] = mul2(d[r][k][i], cw[k][i]);  // gz
            u1 = add2(u1, d[r][k][i]);
            u2 = fma2(d[r][k][i], zh[r][k][i], u2);
          }
          if constexpr (kGate == SPA_GATE_TOKEN) {
            if (in && there[r] && a.dgate != nullptr) {
              if (a.gate_f32) {
#pragma unroll
                for (int i = 0; i < P; i += 2)
                  static_cast<ulonglong2*>(a.dgate)[(size_t)(at[r] + G * k) * (P / 2) + i / 2] = make_ulonglong2(g[i], g[i + 1]);
              } else {
                static_cast<uint4*>(a.dgate)[at[r] + G * k] = from_pairs(g);
              }
            }
          }
        }
        u[2 * r] = sum_of(u1);
        u[2 * r + 1] = sum_of(u2);
        if constexpr (kGate == SPA_GATE_SCORE) u[2 * R + r] = sum_of(u3);
      }
      bool any = false;
#pragma unroll
      for (int r = 0; r < R; ++r) any = any || has[r];
      if (any) sum(u);  // the same for the whole group
#pragma unroll
      for (int r = 0; r < R; ++r) {
        if constexpr (kGate == SPA_GATE_SCORE) {
          if (t0 == 0 && there[r] && a.dgate != nullptr)
            static_cast<float*>(a.dgate)[t + r * kG] = has[r] ? u[2 * R + r] * score[r] * (1.f - score[r]) : 0.f;
        }
        if (has[r]) {
          const uint64_t rs = both(r1[r]), a1 = both(layer ? -u[2 * r] * inv_c * r1[r] : 0.f), a2 = both(-u[2 * r + 1] * inv_c * r1[r]);
#pragma unroll
          for (int k = 0; k < kCh; ++k) {
            if (t0 + G * k < a.Q) {
#pragma unroll
              for (int i = 0; i < P; ++i) d[r][k][i] = fma2(d[r][k][i], rs, fma2(zh[r][k][i], a2, a1));
              a.dz[zat[r] + G * k] = from_pairs(d[r][k]);
            }
          }
        }
      }
    }
    cp_async_wait<0>();
    if (kImage) {  // (join starts with a barrier: the ring is empty)
      float* to = a.part_gate + (size_t)(blockIdx.x + image) * 2 * a.C;
      const T* g = static_cast<const T*>(a.gate) + (size_t)image * a.C;
      join(sA, sB, [&](int c, float A, float B) {
        to[c] = A;
        to[a.C + c] = B;
        const float w = to_f32<T>(g[c]);
        run[c] = fmaf(w, A, run[c]);
        run[a.C + c] = fmaf(w, B, run[a.C + c]);
      });
#pragma unroll
      for (int k = 0; k < kCh; ++k)
#pragma unroll
        for (int i = 0; i < P; ++i) sA[k][i] = sB[k][i] = 0ull;
      __syncthreads();  // the sums' memory becomes the ring again
    }
  }
  float* to = a.part + (size_t)blockIdx.x * kSums * a.C;
  if (kImage) {
    __syncthreads();
    for (int c = threadIdx.x; c < 2 * a.C; c += threads_of(W, true)) to[c] = run[c];
  } else {
    join(sA, sB, [&](int c, float A, float B) { to[c] = A; to[a.C + c] = B; });
  }
  join(sG, sN, [&](int c, float A, float B) { to[2 * a.C + c] = A; to[3 * a.C + c] = B; });
}

// The parameters' gradients from the CTAs' sums, added up in their order: 32 channels a block, blockIdx.x = 0; and with a gate per
// image, per_block images for each further blockIdx.x, their gradients from their lines: a block to an image, or where they have at most
// kAloneLines each, a warp (a block to each of 32 images of 576 x 768: 3 us more; a warp to each of 16 of 196 x 384 fp32, ten lines: 1 us more).
constexpr int kJoinLanes = 16, kAloneLines = 8;
// A sum with what its additions round off (each is a fp32 number that the additions themselves give: Moller's and Knuth's two-sum): a chain of 148
// lines in fp32 was off by six times the result's own rounding.
struct ExactSum {
  float sum = 0.f, rest = 0.f;
  __device__ __forceinline__ void add(float x) {
    const float s = sum + x, t = s - sum;
    rest += (sum - (s - t)) + (x - t);
    sum = s;
  }
  __device__ __forceinline__ double value() const { return fabsf(sum) < __uint_as_float(0x7f800000u) ? (double)sum + rest : (double)sum; }
};
// In the order that they are written in: the loads of a round first, whatever the lines' number (else the kernel waits for memory line by line: 1 us)
__device__ __forceinline__ float ld_f32(const float* p) {
  float v;
  asm volatile("ld.global.f32 %0, [%1];" : "=f"(v) : "l"(p));
  return v;
}
// Lines l, l + lanes, ... of kS sums of C channels each, kAtOnce of them on their way together
template <int kAtOnce, int kS>
__device__ __forceinline__ void join_lines(ExactSum (&v)[kSums], const float* at, int l, int lanes, int lines, int C) {
  const size_t step = (size_t)lanes * kS * C;
  const float* last = at;
  at += (size_t)l * kS * C;
  for (; l < lines; l += kAtOnce * lanes) {
    float f[kAtOnce][kS];
#pragma unroll
    for (int i = 0; i < kAtOnce; ++i, at += step)
#pragma unroll
      for (int k = 0; k < kS; ++k) f[i][k] = ld_f32((l + i * lanes < lines ? at : last) + (unsigned)(k * C));
#pragma unroll
    for (int i = 0; i < kAtOnce; ++i)
#pragma unroll
      for (int k = 0; k < kS; ++k) v[k].add(l + i * lanes < lines ? f[i][k] : 0.f);
  }
}
template <typename T>
__global__ void __launch_bounds__(32 * kJoinLanes)
sandwich_join_kernel(const float* part, const float* part_gate, int ctas, int B, int N, int per_block, int rows_per_cta, int C, const T* scale, const T* g_post,
                     const T* b_post, float* __restrict__ dgate, float* __restrict__ dscale, float* __restrict__ dg_post,
                     float* __restrict__ db_post, float* __restrict__ dg_pre, float* __restrict__ db_pre) {
  pdl_entry();
  __shared__ float s[kSums][kJoinLanes][33], rest[kSums][kJoinLanes][33];
  __shared__ double total[kSums][32];
  const int x = threadIdx.x & 31, y = threadIdx.x >> 5, c = blockIdx.y * 32 + x;
  const bool images = blockIdx.x > 0, alone = images && per_block > 1;  // alone: a thread has an image's lines by itself
  const int b = ((int)blockIdx.x - 1) * per_block + (alone ? y : 0);
  if (alone && b >= B) return;  // (without a barrier behind it)
  // an image's lines: those of the CTAs whose rows it has a part of
  const int c0 = images ? (int)((long long)b * N / rows_per_cta) : 0;
  const int lines = images ? (int)(((long long)b * N + N - 1) / rows_per_cta) - c0 + 1 : ctas;
  const float* from = images ? part_gate + (size_t)(b + c0) * 2 * C : part;
  const float sc = scale != nullptr && c < C ? to_f32<T>(scale[c]) : 1.f, gp = g_post != nullptr && c < C ? to_f32<T>(g_post[c]) : 1.f;
  const float bp = b_post != nullptr && c < C ? to_f32<T>(b_post[c]) : 0.f;
  ExactSum v[kSums];
  if (c < C) {
    if (alone) join_lines<kAloneLines, 2>(v, from + c, 0, 1, lines, C);
    else if (images) join_lines<5, 2>(v, from + c, y, kJoinLanes, lines, C);
    else join_lines<5, kSums>(v, from + c, y, kJoinLanes, lines, C);  // 148 lines are two rounds
  }
  if (alone) {
    if (c < C) dgate[(size_t)b * C + c] = (float)((double)sc * (gp * v[0].value() + bp * v[1].value()));
    return;
  }
#pragma unroll
  for (int k = 0; k < kSums; ++k) { s[k][y][x] = v[k].sum; rest[k][y][x] = v[k].rest; }
  __syncthreads();
  if (y < kSums) {  // a warp to a sum
    ExactSum& u = v[0];
    u = ExactSum{s[y][0][x], rest[y][0][x]};
#pragma unroll
    for (int l = 1; l < kJoinLanes; ++l) { u.add(s[y][l][x]); u.rest += rest[y][l][x]; }
    total[y][x] = u.value();
  }
  __syncthreads();
  if (y != 0 || c >= C) return;
  const double t[kSums] = {total[0][x], total[1][x], total[2][x], total[3][x]};
  if (images) {
    dgate[(size_t)b * C + c] = (float)((double)sc * (gp * t[0] + bp * t[1]));
    return;
  }
  if (dscale != nullptr) dscale[c] = (float)(gp * t[0] + bp * t[1]);
  if (dg_post != nullptr) dg_post[c] = (float)(sc * t[0]);
  if (db_post != nullptr) db_post[c] = (float)(sc * t[1]);
  if (dg_pre != nullptr) dg_pre[c] = (float)t[2];
  if (db_pre != nullptr) db_pre[c] = (float)t[3];
}

int chunks_of(const spa_params& p) { return p.C / (p.dtype == SPA_F32 ? 4 : 8); }

// Warps to a row: as few as leave a thread one chunk, up to sixteen
int warps_of(int Q) {
  for (int w : {1, 2, 3, 4, 6, 8, 12})
    if (Q <= 32 * w) return w;
  return 16;
}

// The backward's shares of rows.  Images of one token: their gate is one per token, and no sum leaves a CTA for it.  A thread adds at most
// kMostChain rows one after the other, and a CTA the sums of as many images: each addition is off by 2^-24 of the sum, and 2^20 rows of 4 096 had
// chains of 7 085.  More CTAs then, in whole grids.
constexpr int kMostChain = 256;
struct Plan { int ctas, rows_per_cta, gate_kind; };
Plan bwd_plan(const spa_params& p, const spa_sandwich& s) {
  const int groups = groups_of(warps_of(chunks_of(p)), true), rows = p.B * p.N;
  Plan r;
  r.gate_kind = s.gate_kind == SPA_GATE_IMAGE && p.N == 1 ? (int)SPA_GATE_TOKEN : s.gate_kind;
  const int most = kMostChain * (r.gate_kind == SPA_GATE_IMAGE && p.N < groups ? p.N : groups);  // rows of a share
  int ctas = (rows + groups - 1) / groups;
  ctas = ctas < 1 ? 1 : (ctas > kNumSMs ? kNumSMs : ctas);
  if ((rows + ctas - 1) / ctas > most) ctas = (rows + most * kNumSMs - 1) / (most * kNumSMs) * kNumSMs;
  r.rows_per_cta = rows > 0 ? (rows + ctas - 1) / ctas : 1;
  r.ctas = rows > 0 ? (rows + r.rows_per_cta - 1) / r.rows_per_cta : 1;
  return r;
}

Args args_of(const spa_params& p, const spa_sandwich& s, const void* z, const int32_t* z_row) {
  Args a = {};
  a.z = (const uint4*)z;
  a.z_row = z_row;
  a.gate = s.gate;
  a.scale = (const uint4*)s.scale;
  a.g_post = (const uint4*)s.g_post;
  a.b_post = (const uint4*)s.b_post;
  a.g_pre = (const uint4*)s.g_pre;
  a.b_pre = (const uint4*)s.b_pre;
  a.rows = p.B * p.N;
  a.N = p.N;
  a.n_magic = (1ull << 40) / p.N + 1;
  a.Q = chunks_of(p);
  a.C = p.C;
  a.z_rows = z_row != nullptr ? p.capacity : p.B * p.N;
  a.kind = s.kind;
  a.eps = s.eps;
  return a;
}

template <typename T, int W, int kCh, int kGate> int fwd_launch(const Args& a, cudaStream_t st) {
  const int need = (a.rows + groups_of(W, false) - 1) / groups_of(W, false), most = kNumSMs * (1024 / threads_of(W, false));
  auto kern = sandwich_fwd_kernel<T, W, kCh, kGate>;
  constexpr int kSmem = Ring<kFwdArrays<kGate>, kCh, kFwdDepth, threads_of(W, false)>::kBytes;
  static DeviceOnce attr;
  cudaError_t e = attr.run([&] { return cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, kSmem); });
  if (e != cudaSuccess) { set_cuda_error(e, "sandwich_fwd_kernel"); return SPA_ERR_CUDA; }
  launch_pdl(kern, need < most ? need : most, threads_of(W, false), kSmem, st, a);
  SPA_CUDA_CHECK_LAUNCH("sandwich_fwd_kernel");
  return SPA_OK;
}

template <typename T, int W, int kCh, int kGate> int bwd_launch(const Args& a, const Plan& pl, cudaStream_t st) {
  auto kern = sandwich_bwd_kernel<T, W, kCh, kGate>;
  constexpr int kRing = Ring<kBwdArrays<kGate> * kBwdRows<W, kCh>, kCh, kBwdDepth<W, kCh>, threads_of(W, true), kBwdRows<W, kCh>>::kBytes;
  auto bytes = [](int channels) {
    const int acc = groups_of(W, true) * 2 * channels * (int)sizeof(float);
    return (acc > kRing ? acc : kRing) + (kGate == SPA_GATE_IMAGE ? 2 * channels * (int)sizeof(float) : 0);
  };
  const int smem = bytes(a.C), kMost = bytes(32 * W * kCh * Vec16<T>::kElems);
  static DeviceOnce attr;
  cudaError_t e = attr.run([&] { return cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, kMost); });
  if (e != cudaSuccess) { set_cuda_error(e, "sandwich_bwd_kernel"); return SPA_ERR_CUDA; }
  launch_pdl(kern, pl.ctas, threads_of(W, true), smem, st, a);
  SPA_CUDA_CHECK_LAUNCH("sandwich_bwd_kernel");
  return SPA_OK;
}

// WHICH<T, warps, chunks of a thread, gate>
#define SPA_BY_WARPS(WHICH, T, GATE, ...)                          \
  switch (warps_of(a.Q)) {                                         \
    case 1: return WHICH<T, 1, 1, GATE>(__VA_ARGS__);              \
    case 2: return WHICH<T, 2, 1, GATE>(__VA_ARGS__);              \
    case 3: return WHICH<T, 3, 1, GATE>(__VA_ARGS__);              \
    case 4: return WHICH<T, 4, 1, GATE>(__VA_ARGS__);              \
    case 6: return WHICH<T, 6, 1, GATE>(__VA_ARGS__);              \
    case 8: return WHICH<T, 8, 1, GATE>(__VA_ARGS__);              \
    case 12: return WHICH<T, 12, 1, GATE>(__VA_ARGS__);            \
    default:                                                       \
      if (a.Q <= 512) return WHICH<T, 16, 1, GATE>(__VA_ARGS__);   \
      return WHICH<T, 16, 2, GATE>(__VA_ARGS__);                   \
  }
template <typename T, int kGate> int fwd_by_warps(const Args& a, cudaStream_t st) { SPA_BY_WARPS(fwd_launch, T, kGate, a, st) }
template <typename T, int kGate> int bwd_by_warps(const Args& a, const Plan& pl, cudaStream_t st) { SPA_BY_WARPS(bwd_launch, T, kGate, a, pl, st) }
#undef SPA_BY_WARPS
#define SPA_BY_GATE(KIND, WHICH, ...)                                                                             \
  (p.dtype == SPA_F32 ? ((KIND) == SPA_GATE_NONE    ? WHICH<float, SPA_GATE_NONE>(__VA_ARGS__)         \
                         : (KIND) == SPA_GATE_SCORE ? WHICH<float, SPA_GATE_SCORE>(__VA_ARGS__)        \
                         : (KIND) == SPA_GATE_IMAGE ? WHICH<float, SPA_GATE_IMAGE>(__VA_ARGS__)        \
                                                         : WHICH<float, SPA_GATE_TOKEN>(__VA_ARGS__))       \
                      : ((KIND) == SPA_GATE_NONE    ? WHICH<__nv_bfloat16, SPA_GATE_NONE>(__VA_ARGS__)  \
                         : (KIND) == SPA_GATE_SCORE ? WHICH<__nv_bfloat16, SPA_GATE_SCORE>(__VA_ARGS__) \
                         : (KIND) == SPA_GATE_IMAGE ? WHICH<__nv_bfloat16, SPA_GATE_IMAGE>(__VA_ARGS__) \
                                                         : WHICH<__nv_bfloat16, SPA_GATE_TOKEN>(__VA_ARGS__)))

}  // namespace

bool sandwich_supported(const spa_params& p) { return chunks_of(p) <= kMaxChunks; }

size_t sandwich_workspace_bytes(const spa_params& p, const spa_sandwich& s) {
  const Plan pl = bwd_plan(p, s);
  const size_t lines = (size_t)pl.ctas * kSums + (pl.gate_kind == SPA_GATE_IMAGE ? ((size_t)pl.ctas + p.B) * 2 : 0);
  return lines * p.C * sizeof(float) + 256;
}

int launch_sandwich(const spa_params& p, const spa_sandwich& s, const void* x, const void* z, const int32_t* z_row, void* y,
                    void* n, float* stats, cudaStream_t st) {
  Args a = args_of(p, s, z, z_row);
  a.x = (const uint4*)x;
  a.out_y = (uint4*)y;
  a.out_n = (uint4*)n;
  a.stats = stats;
  return SPA_BY_GATE(s.gate_kind, fwd_by_warps, a, st);
}

int launch_sandwich_bwd(const spa_params& p, const spa_sandwich& s, const void* dn, const void* dy, const void* y, const void* z,
                        const int32_t* z_row, const float* stats, void* dx, void* dz, void* dgate, float* dscale, float* dg_post,
                        float* db_post, float* dg_pre, float* db_pre, void* workspace, cudaStream_t st) {
  const Plan pl = bwd_plan(p, s);
  Args a = args_of(p, s, z, z_row);
  a.dn = (const uint4*)dn;
  a.dy = (const uint4*)dy;
  a.y = (const uint4*)y;
  a.stats = const_cast<float*>(stats);
  a.dx = (uint4*)dx;
  a.dz = (uint4*)dz;
  a.dgate = dgate;
  a.part = static_cast<float*>(workspace);
  a.part_gate = a.part + (size_t)pl.ctas * kSums * p.C;
  a.rows_per_cta = pl.rows_per_cta;
  a.gate_f32 = pl.gate_kind != s.gate_kind;
  const int rc = SPA_BY_GATE(pl.gate_kind, bwd_by_warps, a, pl, st);
  if (rc != SPA_OK) return rc;
  const bool images = pl.gate_kind == SPA_GATE_IMAGE && dgate != nullptr;
  if (!images && dscale == nullptr && dg_post == nullptr && db_post == nullptr && dg_pre == nullptr && db_pre == nullptr) return SPA_OK;
  const int per_block = p.N / pl.rows_per_cta + 2 <= kAloneLines ? kJoinLanes : 1;  // an image has at most so many lines
  const dim3 grid(images ? 1 + (p.B + per_block - 1) / per_block : 1, (p.C + 31) / 32);
#define SPA_JOIN(T)                                                                                                       \
  launch_pdl(sandwich_join_kernel<T>, grid, 32 * kJoinLanes, 0, st, a.part, a.part_gate, pl.ctas, p.B, p.N, per_block, pl.rows_per_cta, p.C, \
             (const T*)s.scale, (const T*)s.g_post, (const T*)s.b_post, (float*)dgate, dscale, dg_post, db_post, dg_pre, db_pre)
  if (p.dtype == SPA_F32) SPA_JOIN(float); else SPA_JOIN(__nv_bfloat16);
#undef SPA_JOIN
  SPA_CUDA_CHECK_LAUNCH("sandwich_join_kernel");
  return SPA_OK;
}

}  // namespace spa
