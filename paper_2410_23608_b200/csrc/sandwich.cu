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
// Both directions are bound by bytes: every operand is read once, every result written once, all loads of a row are issued
// together.  A row belongs to a group of W warps, sized so that a thread holds one to four 16-byte chunks (two in the
// backward, whose running sums take 32 registers a chunk).  Statistics and sums are fp32; y and n are rounded once, n from the
// unrounded y.  Sums run in a fixed order: results are bitwise reproducible.
#include "spa_common.cuh"

namespace spa {
namespace {

constexpr int kMaxChunks = 1024;  // 16-byte chunks of a row: 8 192 bf16 or 4 096 fp32 channels
constexpr int kSums = 4;          // running sums per channel of the backward: A, B, sum dn yh, sum dn
template <int W> constexpr int kThreads = W == 16 ? 512 : 256;
template <int W> constexpr int kGroups = kThreads<W> / (32 * W);

struct Args {
  const uint4 *x, *z, *dn, *dy, *y;   // rows of Q chunks; dn, dy optional
  const int32_t* z_row;               // optional
  const void* gate;
  const uint4 *scale, *g_post, *b_post, *g_pre, *b_pre;  // optional
  float* stats;                       // [4][rows]: mean and 1 / deviation of z's row, of y's
  uint4 *out_y, *out_n;               // forward
  uint4 *dx, *dz;                     // backward; dz optional
  void* dgate;
  float *part, *part_gate;            // per CTA [kSums][C]; per unit of an image's rows [2][C]
  int rows, N, Q, C, z_rows, kind, gate_kind, units, splits;
  float eps;
};

// Sums of a and b over the group's threads, in every one of them.  Calls alternate between two lines of `red`: a warp that
// writes a line again has met the others at the barrier in between, behind their reads of it.
template <int W> struct GroupSum {
  float* red;  // [2][W][2] of this group
  int id, warp, lane, turn;
  __device__ __forceinline__ void operator()(float& a, float& b) {
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) {
      a += __shfl_xor_sync(0xffffffffu, a, o);
      b += __shfl_xor_sync(0xffffffffu, b, o);
    }
    if constexpr (W > 1) {
      float* line = red + turn * 2 * W;
      if (lane == 0) { line[2 * warp] = a; line[2 * warp + 1] = b; }
      asm volatile("bar.sync %0, %1;" ::"r"(id + 1), "n"(32 * W) : "memory");
      a = b = 0.f;
#pragma unroll
      for (int w = 0; w < W; ++w) { a += line[2 * w]; b += line[2 * w + 1]; }
      turn ^= 1;
    }
  }
};

template <typename T> __device__ __forceinline__ void chunk_or(const uint4* p, int q, float fill, float* f) {
  if (p != nullptr) {
    Vec16<T>::to_float(p[q], f);
  } else {
#pragma unroll
    for (int e = 0; e < Vec16<T>::kElems; ++e) f[e] = fill;
  }
}

__device__ __forceinline__ float sigmoid(float s) { return 1.f / (1.f + expf(-s)); }

template <typename T, int W, int kCh>
__global__ void __launch_bounds__(kThreads<W>) sandwich_fwd_kernel(const Args a) {
  pdl_entry();
  constexpr int E = Vec16<T>::kElems, G = 32 * W;
  __shared__ float red[kGroups<W> * 4 * W];
  const int grp = threadIdx.x / G, t0 = threadIdx.x % G;
  GroupSum<W> sum{red + grp * 4 * W, grp, t0 >> 5, (int)threadIdx.x & 31, 0};
  const float inv_c = 1.f / a.C;
  const bool layer = a.kind == SPA_NORM_LAYER;
  // mean (0 for RMS) and 1 / deviation of the row v
  auto statistics = [&](const float (&v)[kCh][E], float& mean, float& rstd) {
    float s = 0.f, none = 0.f;
    mean = 0.f;
    if (layer) {
#pragma unroll
      for (int k = 0; k < kCh; ++k)
        if (t0 + G * k < a.Q) {
#pragma unroll
          for (int e = 0; e < E; ++e) s += v[k][e];
        }
      sum(s, none);
      mean = s * inv_c;
    }
    float ss = 0.f;
    none = 0.f;
#pragma unroll
    for (int k = 0; k < kCh; ++k)
      if (t0 + G * k < a.Q) {
#pragma unroll
        for (int e = 0; e < E; ++e) { const float d = v[k][e] - mean; ss = fmaf(d, d, ss); }
      }
    sum(ss, none);
    rstd = rsqrtf(ss * inv_c + a.eps);
  };
  for (int t = blockIdx.x * kGroups<W> + grp; t < a.rows; t += gridDim.x * kGroups<W>) {
    int zr = t;
    if (a.z_row != nullptr) zr = ld_dep(a.z_row + t);
    const bool has = zr >= 0 && zr < a.z_rows;
    const long long at = (long long)t * a.Q, zat = (long long)zr * a.Q;
    uint4 xr[kCh], zv[kCh], gr[kCh];
    float score = 0.f;
    const uint4* gate16 = static_cast<const uint4*>(a.gate) + (a.gate_kind == SPA_GATE_IMAGE ? (long long)(t / a.N) * a.Q : at);
    const bool gates = a.gate_kind == SPA_GATE_IMAGE || a.gate_kind == SPA_GATE_TOKEN;
#pragma unroll
    for (int k = 0; k < kCh; ++k) {
      const int q = t0 + G * k;
      xr[k] = zv[k] = gr[k] = make_uint4(0u, 0u, 0u, 0u);
      if (q < a.Q) {
        xr[k] = ld_stream16(a.x + at + q);
        if (has) {
          zv[k] = ld_stream16(a.z + zat + q);
          if (gates) gr[k] = gate16[q];
        }
      }
    }
    if (has && a.gate_kind == SPA_GATE_SCORE) score = sigmoid(static_cast<const float*>(a.gate)[t]);
    float v[kCh][E], m1 = 0.f, r1 = 0.f;
    if (has) {
#pragma unroll
      for (int k = 0; k < kCh; ++k) Vec16<T>::to_float(zv[k], v[k]);
      statistics(v, m1, r1);
    }
#pragma unroll
    for (int k = 0; k < kCh; ++k) {
      const int q = t0 + G * k;
      float x[E];
      Vec16<T>::to_float(xr[k], x);
      if (has && q < a.Q) {
        float gp[E], bp[E], sc[E], g[E];
        chunk_or<T>(a.g_post, q, 1.f, gp);
        chunk_or<T>(a.b_post, q, 0.f, bp);
        chunk_or<T>(a.scale, q, 1.f, sc);
        Vec16<T>::to_float(gr[k], g);
#pragma unroll
        for (int e = 0; e < E; ++e) {
          const float w = gates ? g[e] : (a.gate_kind == SPA_GATE_SCORE ? score : 1.f);
          x[e] = fmaf(fmaf((v[k][e] - m1) * r1, gp[e], bp[e]), sc[e] * w, x[e]);
        }
      }
#pragma unroll
      for (int e = 0; e < E; ++e) v[k][e] = x[e];
      if (q < a.Q) a.out_y[at + q] = has ? Vec16<T>::from_float(x) : xr[k];
    }
    float m2 = 0.f, r2 = 0.f;
    if (a.out_n != nullptr) {
      statistics(v, m2, r2);
#pragma unroll
      for (int k = 0; k < kCh; ++k) {
        const int q = t0 + G * k;
        if (q < a.Q) {
          float gp[E], bp[E], o[E];
          chunk_or<T>(a.g_pre, q, 1.f, gp);
          chunk_or<T>(a.b_pre, q, 0.f, bp);
#pragma unroll
          for (int e = 0; e < E; ++e) o[e] = fmaf((v[k][e] - m2) * r2, gp[e], bp[e]);
          a.out_n[at + q] = Vec16<T>::from_float(o);
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

// Rows are taken in units: with a gate per image a unit is a split of one image's rows, so that its sums A_b and B_b leave the CTA
// at its end; otherwise a CTA has one unit, its share of all rows.
template <typename T, int W, int kCh>
__global__ void __launch_bounds__(kThreads<W>) sandwich_bwd_kernel(const Args a) {
  pdl_entry();
  constexpr int E = Vec16<T>::kElems, G = 32 * W, kG = kGroups<W>;
  extern __shared__ __align__(16) float acc_s[];  // [kG][2][C], and behind it, with a gate per image, [2][C]: sum of gate_b A_b, of gate_b B_b
  __shared__ float red[kG * 4 * W];
  const int grp = threadIdx.x / G, t0 = threadIdx.x % G;
  GroupSum<W> sum{red + grp * 4 * W, grp, t0 >> 5, (int)threadIdx.x & 31, 0};
  const float inv_c = 1.f / a.C;
  const bool layer = a.kind == SPA_NORM_LAYER, per_image = a.gate_kind == SPA_GATE_IMAGE;
  float sA[kCh][E] = {}, sB[kCh][E] = {}, sG[kCh][E] = {}, sN[kCh][E] = {};
  float* run = acc_s + (size_t)kG * 2 * a.C;
  if (per_image)
    for (int c = threadIdx.x; c < 2 * a.C; c += kThreads<W>) run[c] = 0.f;  // each thread its own, also below
  // two running sums of every group, added up in the order of the groups, to out(c, first, second)
  auto join = [&](const float (&u)[kCh][E], const float (&w)[kCh][E], auto out) {
    __syncthreads();
    float* mine = acc_s + grp * 2 * a.C;
#pragma unroll
    for (int k = 0; k < kCh; ++k) {
      const int q = t0 + G * k;
      if (q < a.Q) {
#pragma unroll
        for (int e = 0; e < E; e += 4) {
          *reinterpret_cast<float4*>(mine + q * E + e) = make_float4(u[k][e], u[k][e + 1], u[k][e + 2], u[k][e + 3]);
          *reinterpret_cast<float4*>(mine + a.C + q * E + e) = make_float4(w[k][e], w[k][e + 1], w[k][e + 2], w[k][e + 3]);
        }
      }
    }
    __syncthreads();
    for (int c = threadIdx.x; c < a.C; c += kThreads<W>) {
      float s = 0.f, r = 0.f;
#pragma unroll
      for (int g = 0; g < kG; ++g) { s += acc_s[g * 2 * a.C + c]; r += acc_s[g * 2 * a.C + a.C + c]; }
      out(c, s, r);
    }
  };
  for (int unit = blockIdx.x; unit < a.units; unit += gridDim.x) {
    int first = unit * kG + grp, step = a.units * kG, end = a.rows, image = 0;
    if (per_image) {
      image = unit / a.splits;
      const int split = unit - image * a.splits, per = (a.N + a.splits - 1) / a.splits;
      first = image * a.N + split * per + grp;
      step = kG;
      end = image * a.N + (split * per + per < a.N ? split * per + per : a.N);
    }
    for (int t = first; t < end; t += step) {
      int zr = t;
      if (a.z_row != nullptr) zr = ld_dep(a.z_row + t);
      const bool has = zr >= 0 && zr < a.z_rows;
      const long long at = (long long)t * a.Q, zat = (long long)zr * a.Q;
      const uint4* gate16 = static_cast<const uint4*>(a.gate) + (per_image ? (long long)image * a.Q : at);
      const bool gates = per_image || a.gate_kind == SPA_GATE_TOKEN;
      const uint4 zero = make_uint4(0u, 0u, 0u, 0u);
      uint4 nr[kCh], dr[kCh], yr[kCh], zv[kCh], gr[kCh];
#pragma unroll
      for (int k = 0; k < kCh; ++k) {
        const int q = t0 + G * k;
        const bool in = q < a.Q;
        nr[k] = in && a.dn != nullptr ? ld_stream16(a.dn + at + q) : zero;
        yr[k] = in && a.dn != nullptr ? ld_stream16(a.y + at + q) : zero;
        dr[k] = in && a.dy != nullptr ? ld_stream16(a.dy + at + q) : zero;
        zv[k] = in && has ? ld_stream16(a.z + zat + q) : zero;
        gr[k] = in && has && gates ? gate16[q] : zero;
      }
      const float m1 = a.stats[t], r1 = a.stats[a.rows + t];
      float m2 = 0.f, r2 = 0.f, score = 1.f;
      if (a.dn != nullptr) { m2 = a.stats[2 * a.rows + t]; r2 = a.stats[3 * a.rows + t]; }
      if (a.gate_kind == SPA_GATE_SCORE) score = sigmoid(static_cast<const float*>(a.gate)[t]);
      // ---- through the norm behind the sum: d, the gradient of y
      float d[kCh][E];
      float s1 = 0.f, s2 = 0.f;
      if (a.dn != nullptr) {
#pragma unroll
        for (int k = 0; k < kCh; ++k) {
          const int q = t0 + G * k;
          if (q < a.Q) {
            float n[E], y[E], gp[E];
            Vec16<T>::to_float(nr[k], n);
            Vec16<T>::to_float(yr[k], y);
            chunk_or<T>(a.g_pre, q, 1.f, gp);
#pragma unroll
            for (int e = 0; e < E; ++e) {
              const float yh = (y[e] - m2) * r2, g = n[e] * gp[e];
              s1 += g;
              s2 = fmaf(g, yh, s2);
              sG[k][e] = fmaf(n[e], yh, sG[k][e]);
              sN[k][e] += n[e];
            }
          }
        }
        sum(s1, s2);
        s1 = layer ? s1 * inv_c : 0.f;
        s2 *= inv_c;
      }
      float u1 = 0.f, u2 = 0.f;
#pragma unroll
      for (int k = 0; k < kCh; ++k) {
        const int q = t0 + G * k;
        Vec16<T>::to_float(dr[k], d[k]);
        if (q < a.Q) {
          if (a.dn != nullptr) {
            float n[E], y[E], gp[E];
            Vec16<T>::to_float(nr[k], n);
            Vec16<T>::to_float(yr[k], y);
            chunk_or<T>(a.g_pre, q, 1.f, gp);
#pragma unroll
            for (int e = 0; e < E; ++e) d[k][e] += (n[e] * gp[e] - s1 - (y[e] - m2) * r2 * s2) * r2;
          }
          a.dx[at + q] = Vec16<T>::from_float(d[k]);
          if (has) {
            float z[E], g[E], gp[E], sc[E], bp[E];
            Vec16<T>::to_float(zv[k], z);
            Vec16<T>::to_float(gr[k], g);
            chunk_or<T>(a.g_post, q, 1.f, gp);
            chunk_or<T>(a.scale, q, 1.f, sc);
            float o[E];
            if (a.gate_kind == SPA_GATE_TOKEN) chunk_or<T>(a.b_post, q, 0.f, bp);
#pragma unroll
            for (int e = 0; e < E; ++e) {
              const float zh = (z[e] - m1) * r1, w = gates ? g[e] : score;
              const float dw = per_image ? d[k][e] : d[k][e] * w;
              sA[k][e] = fmaf(dw, zh, sA[k][e]);
              sB[k][e] += dw;
              const float gz = d[k][e] * w * sc[e] * gp[e];
              u1 += gz;
              u2 = fmaf(gz, zh, u2);
              if (a.gate_kind == SPA_GATE_TOKEN) o[e] = d[k][e] * sc[e] * fmaf(zh, gp[e], bp[e]);
            }
            if (a.gate_kind == SPA_GATE_TOKEN) {
              if (a.dgate != nullptr) static_cast<uint4*>(a.dgate)[at + q] = Vec16<T>::from_float(o);
            }
          } else if (a.gate_kind == SPA_GATE_TOKEN && a.dgate != nullptr) {
            static_cast<uint4*>(a.dgate)[at + q] = zero;
          }
        }
      }
      if (has) {
        // score: dgate = score (1 - score) sum d scale (g_post zh + b_post)
        if (a.gate_kind == SPA_GATE_SCORE && a.dgate != nullptr) {
          float v = 0.f, none = 0.f;
#pragma unroll
          for (int k = 0; k < kCh; ++k) {
            const int q = t0 + G * k;
            if (q < a.Q) {
              float z[E], gp[E], sc[E], bp[E];
              Vec16<T>::to_float(zv[k], z);
              chunk_or<T>(a.g_post, q, 1.f, gp);
              chunk_or<T>(a.scale, q, 1.f, sc);
              chunk_or<T>(a.b_post, q, 0.f, bp);
#pragma unroll
              for (int e = 0; e < E; ++e) v = fmaf(d[k][e] * sc[e], fmaf((z[e] - m1) * r1, gp[e], bp[e]), v);
            }
          }
          sum(v, none);
          if (t0 == 0) static_cast<float*>(a.dgate)[t] = v * score * (1.f - score);
        }
        sum(u1, u2);
        u1 = layer ? u1 * inv_c : 0.f;
        u2 *= inv_c;
#pragma unroll
        for (int k = 0; k < kCh; ++k) {
          const int q = t0 + G * k;
          if (q < a.Q) {
            float z[E], g[E], gp[E], sc[E], o[E];
            Vec16<T>::to_float(zv[k], z);
            Vec16<T>::to_float(gr[k], g);
            chunk_or<T>(a.g_post, q, 1.f, gp);
            chunk_or<T>(a.scale, q, 1.f, sc);
#pragma unroll
            for (int e = 0; e < E; ++e) {
              const float w = gates ? g[e] : score;
              o[e] = (d[k][e] * w * sc[e] * gp[e] - u1 - (z[e] - m1) * r1 * u2) * r1;
            }
            a.dz[zat + q] = Vec16<T>::from_float(o);
          }
        }
      } else if (a.gate_kind == SPA_GATE_SCORE && a.dgate != nullptr && t0 == 0) {
        static_cast<float*>(a.dgate)[t] = 0.f;
      }
    }
    if (per_image) {
      float* to = a.part_gate + (size_t)unit * 2 * a.C;
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
        for (int e = 0; e < E; ++e) sA[k][e] = sB[k][e] = 0.f;
    }
  }
  float* to = a.part + (size_t)blockIdx.x * kSums * a.C;
  if (per_image) {
    __syncthreads();
    for (int c = threadIdx.x; c < 2 * a.C; c += kThreads<W>) to[c] = run[c];
  } else {
    join(sA, sB, [&](int c, float A, float B) { to[c] = A; to[a.C + c] = B; });
  }
  join(sG, sN, [&](int c, float A, float B) { to[2 * a.C + c] = A; to[3 * a.C + c] = B; });
}

// The parameters' gradients from the CTAs' sums, added up in their order: 32 channels a block, blockIdx.x = 0; and with a gate per
// image, blockIdx.x = 1 + image, its gradient from the units of its rows.
constexpr int kJoinLanes = 16;
template <typename T>
__global__ void __launch_bounds__(32 * kJoinLanes)
sandwich_join_kernel(const float* part, const float* part_gate, int ctas, int splits, int C, const T* scale, const T* g_post,
                     const T* b_post, float* __restrict__ dgate, float* __restrict__ dscale, float* __restrict__ dg_post,
                     float* __restrict__ db_post, float* __restrict__ dg_pre, float* __restrict__ db_pre) {
  pdl_entry();
  __shared__ float s[kSums][kJoinLanes][33];
  const int x = threadIdx.x & 31, y = threadIdx.x >> 5, c = blockIdx.y * 32 + x;
  const bool images = blockIdx.x > 0;
  const int lines = images ? splits : ctas, sums = images ? 2 : kSums;
  const float* from = images ? part_gate + (size_t)(blockIdx.x - 1) * splits * 2 * C : part;
  float v[kSums] = {};
  if (c < C) {
#pragma unroll 4
    for (int l = y; l < lines; l += kJoinLanes) {
#pragma unroll
      for (int k = 0; k < kSums; ++k)
        if (k < sums) v[k] += from[((size_t)l * sums + k) * C + c];
    }
  }
#pragma unroll
  for (int k = 0; k < kSums; ++k) s[k][y][x] = v[k];
  __syncthreads();
  if (y != 0 || c >= C) return;
#pragma unroll
  for (int k = 0; k < kSums; ++k) {
    v[k] = 0.f;
    for (int l = 0; l < kJoinLanes; ++l) v[k] += s[k][l][x];
  }
  const float sc = scale != nullptr ? to_f32<T>(scale[c]) : 1.f, gp = g_post != nullptr ? to_f32<T>(g_post[c]) : 1.f;
  const float bp = b_post != nullptr ? to_f32<T>(b_post[c]) : 0.f;
  if (images) {
    dgate[(size_t)(blockIdx.x - 1) * C + c] = sc * fmaf(gp, v[0], bp * v[1]);
    return;
  }
  if (dscale != nullptr) dscale[c] = fmaf(gp, v[0], bp * v[1]);
  if (dg_post != nullptr) dg_post[c] = sc * v[0];
  if (db_post != nullptr) db_post[c] = sc * v[1];
  if (dg_pre != nullptr) dg_pre[c] = v[2];
  if (db_pre != nullptr) db_pre[c] = v[3];
}

int chunks_of(const spa_params& p) { return p.C / (p.dtype == SPA_F32 ? 4 : 8); }

// Warps to a row: as few as leave a thread `most` chunks or fewer
int warps_of(int Q, int most) {
  int w = 1;
  while (w < 16 && Q > 32 * w * most) w *= 2;
  return w;
}

// Units of rows: per image so many splits that the CTAs of the grid have one each; otherwise one per CTA.
struct Plan { int ctas, units, splits, warps; };
Plan bwd_plan(const spa_params& p, const spa_sandwich& s) {
  Plan r;
  r.warps = warps_of(chunks_of(p), 2);
  const int groups = r.warps == 16 ? 1 : 8 / r.warps, most = kNumSMs * (r.warps == 16 ? 1 : 2), rows = p.B * p.N;
  if (s.gate_kind == SPA_GATE_IMAGE) {
    r.splits = p.B >= most || p.B == 0 ? 1 : most / p.B;
    const int useful = (p.N + groups - 1) / groups;
    if (r.splits > useful) r.splits = useful;
    r.units = p.B * r.splits;
  } else {
    r.splits = 1;
    r.units = (rows + groups - 1) / groups;
    if (r.units > most) r.units = most;
  }
  r.ctas = r.units < most ? r.units : most;
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
  a.Q = chunks_of(p);
  a.C = p.C;
  a.z_rows = z_row != nullptr ? p.capacity : p.B * p.N;
  a.kind = s.kind;
  a.gate_kind = s.gate_kind;
  a.eps = s.eps;
  return a;
}

template <typename T, int W, int kCh> int fwd_launch(const Args& a, cudaStream_t st) {
  const int need = (a.rows + kGroups<W> - 1) / kGroups<W>, most = kNumSMs * (W == 16 ? 3 : 6);
  launch_pdl(sandwich_fwd_kernel<T, W, kCh>, need < most ? need : most, kThreads<W>, 0, st, a);
  SPA_CUDA_CHECK_LAUNCH("sandwich_fwd_kernel");
  return SPA_OK;
}

template <typename T, int W, int kCh> int bwd_launch(const Args& a, const Plan& pl, cudaStream_t st) {
  auto kern = sandwich_bwd_kernel<T, W, kCh>;
  const size_t smem = (size_t)(kGroups<W> + 1) * 2 * a.C * sizeof(float);
  constexpr int kMost = (kGroups<W> + 1) * 2 * 32 * W * kCh * Vec16<T>::kElems * (int)sizeof(float);
  static DeviceOnce attr;
  cudaError_t e = attr.run([&] { return cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, kMost); });
  if (e != cudaSuccess) { set_cuda_error(e, "sandwich_bwd_kernel"); return SPA_ERR_CUDA; }
  launch_pdl(kern, pl.ctas, kThreads<W>, smem, st, a);
  SPA_CUDA_CHECK_LAUNCH("sandwich_bwd_kernel");
  return SPA_OK;
}

}  // namespace

bool sandwich_supported(const spa_params& p) { return chunks_of(p) <= kMaxChunks; }

size_t sandwich_workspace_bytes(const spa_params& p, const spa_sandwich& s) {
  const Plan pl = bwd_plan(p, s);
  const size_t lines = (size_t)pl.ctas * kSums + (s.gate_kind == SPA_GATE_IMAGE ? (size_t)pl.units * 2 : 0);
  return lines * p.C * sizeof(float) + 256;
}

int launch_sandwich(const spa_params& p, const spa_sandwich& s, const void* x, const void* z, const int32_t* z_row, void* y,
                    void* n, float* stats, cudaStream_t st) {
  Args a = args_of(p, s, z, z_row);
  a.x = (const uint4*)x;
  a.out_y = (uint4*)y;
  a.out_n = (uint4*)n;
  a.stats = stats;
#define SPA_FWD(T)                                                                                   \
  do {                                                                                               \
    const int w = warps_of(a.Q, 4), ch = (a.Q + 32 * w - 1) / (32 * w);                              \
    if (w == 1 && ch == 1) return fwd_launch<T, 1, 1>(a, st);                                        \
    if (w == 1 && ch == 2) return fwd_launch<T, 1, 2>(a, st);                                        \
    if (w == 1 && ch == 3) return fwd_launch<T, 1, 3>(a, st);                                        \
    if (w == 1) return fwd_launch<T, 1, 4>(a, st);                                                   \
    if (w == 2) return ch <= 3 ? fwd_launch<T, 2, 3>(a, st) : fwd_launch<T, 2, 4>(a, st);            \
    if (w == 4) return ch <= 3 ? fwd_launch<T, 4, 3>(a, st) : fwd_launch<T, 4, 4>(a, st);            \
    return ch <= 3 ? fwd_launch<T, 8, 3>(a, st) : fwd_launch<T, 8, 4>(a, st);                        \
  } while (0)
  if (p.dtype == SPA_F32) SPA_FWD(float);
  SPA_FWD(__nv_bfloat16);
#undef SPA_FWD
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
  a.units = pl.units;
  a.splits = pl.splits;
  int rc = SPA_OK;
#define SPA_BWD(T)                                                                                   \
  do {                                                                                               \
    const bool one = a.Q <= 32 * pl.warps;                                                           \
    if (pl.warps == 1) rc = one ? bwd_launch<T, 1, 1>(a, pl, st) : bwd_launch<T, 1, 2>(a, pl, st);   \
    else if (pl.warps == 2) rc = bwd_launch<T, 2, 2>(a, pl, st);                                     \
    else if (pl.warps == 4) rc = bwd_launch<T, 4, 2>(a, pl, st);                                     \
    else if (pl.warps == 8) rc = bwd_launch<T, 8, 2>(a, pl, st);                                     \
    else rc = bwd_launch<T, 16, 2>(a, pl, st);                                                       \
  } while (0)
  if (p.dtype == SPA_F32) SPA_BWD(float); else SPA_BWD(__nv_bfloat16);
#undef SPA_BWD
  if (rc != SPA_OK) return rc;
  const bool images = s.gate_kind == SPA_GATE_IMAGE && dgate != nullptr;
  if (!images && dscale == nullptr && dg_post == nullptr && db_post == nullptr && dg_pre == nullptr && db_pre == nullptr) return SPA_OK;
  const dim3 grid(images ? 1 + p.B : 1, (p.C + 31) / 32);
#define SPA_JOIN(T)                                                                                                       \
  launch_pdl(sandwich_join_kernel<T>, grid, 32 * kJoinLanes, 0, st, a.part, a.part_gate, pl.ctas, pl.splits, p.C,         \
             (const T*)s.scale, (const T*)s.g_post, (const T*)s.b_post, (float*)dgate, dscale, dg_post, db_post, dg_pre, db_pre)
  if (p.dtype == SPA_F32) SPA_JOIN(float); else SPA_JOIN(__nv_bfloat16);
#undef SPA_JOIN
  SPA_CUDA_CHECK_LAUNCH("sandwich_join_kernel");
  return SPA_OK;
}

}  // namespace spa
