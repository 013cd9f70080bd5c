// Attention backward with a bias by relative position, segments of at most 128 rows (Sec. 3.1: the backbone's windows; Sec. 3.2:
// containers and small selections), on tcgen05 tensor cores in one pass.
//
// The two passes of attn_tc.cu evaluate S, its bias, the exponentials, dP and dS of every pair twice, and a tile of 128 rows
// that are of many segments walks the keys of all of them: windows of 49 rows use a quarter of the values.  Here a tile is as many
// whole segments, one behind the other, as fit 128 rows, of one head:
//   S = Q K^T, dP = dO V^T (128 x 128, fp32 in TMEM);  P = 2^(S + bias - lse), dS = P (dP - D) where a row and a column are of one segment,
//   zero elsewhere, to shared memory as bf16;  dV = P^T dO, dK = dS^T Q, dQ = dS K;
// and dS to the bins of the table's gradient, as in the dQ pass.  Two threads share a row, 64 columns each in groups of 32, and a warp
// passes over the groups that none of its rows has columns in.  A tile's steps follow one another and two CTAs share an SM, so
// that one computes while the other waits.  A CTA takes a few segments of one head at a time and tiles them itself.
// What bounds it is the chain of a tile's steps: 512 windows of 7 x 7, 12 heads of 32, 91 us against 24 for their bytes, issue slots half
// full, the memory a fifth.
#include <math_constants.h>

#include "attn_rel.cuh"
#include "attn_tc.cuh"

namespace spa {
namespace {

constexpr int kThreads = 256;
constexpr int kMaxChunk = 32;  // segments that a CTA takes at a time
constexpr int kPairMax = 64;   // rows of a segment of which two make a tile

template <int D> struct Smem {
  static constexpr int kTile = HeadTile<D>::kTileBytes;
  static constexpr int kOp = 128 * 128 * 2;        // P or dS: two panels of 64 keys, 128 query rows of 128 bytes each
  static constexpr bool kTwo = D == 32;            // a buffer for each; at d = 64 dS follows P, when dV has been computed
  static constexpr int kQ = 0, kK = kTile, kDO = 2 * kTile, kP = 3 * kTile, kDS = kTwo ? kP + kOp : kP;
  static constexpr int kV = kP, kO = kTwo ? kDS : kP + kTile;  // needed only until the first products and D
  static constexpr int kBar = kDS + kOp;           // barriers, TMEM slot, the tile's bound
  static constexpr int kSeg = kBar + 64;           // offsets of the CTA's segments
  static constexpr int kPos = kSeg + 192;          // the tile's key positions
  static constexpr int kTable = kPos + 128 * 4;    // the head's table, and behind it the bins, two words each
  static constexpr int kBytes = kTable + 1024;     // and the alignment of the base
};

template <int D>
__global__ void __launch_bounds__(kThreads, 2)
rel_bwd_short_kernel(const __grid_constant__ CUtensorMap tm_qkv, const __grid_constant__ CUtensorMap tm_do,
                     const __grid_constant__ CUtensorMap tm_o, const float* lse, float* delta, const int32_t* seg, int n_seg, int chunk,
                     int least, int capacity, int C, int H, float scale, __nv_bfloat16* __restrict__ dqkv, const RelBwd rel, int32_t* d_status) {
  using HT = HeadTile<D>;
  using SM = Smem<D>;
  constexpr int kTile = SM::kTile, kOp = SM::kOp, kDh = D / 2;
  constexpr float kLog2e = 1.4426950408889634f;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  // warps w and w + 4 may touch the same quarter of the TMEM lanes: they share 32 rows and split the columns
  const int quarter = warp & 3, half = warp >> 2, rl = quarter * 32 + lane;
  const int n_chunks = (n_seg + chunk - 1) / chunk, n_items = n_chunks * H;

  extern __shared__ uint8_t smem_raw[];
  const uint32_t smem_base = (ptx::smem_u32(smem_raw) + 1023u) & ~1023u;
  uint8_t* smem_al = smem_raw + (smem_base - ptx::smem_u32(smem_raw));
  const uint32_t q_s = smem_base + SM::kQ, k_s = smem_base + SM::kK, do_s = smem_base + SM::kDO;
  const uint32_t p_s = smem_base + SM::kP, ds_s = smem_base + SM::kDS;
  const uint32_t bar_ld = smem_base + SM::kBar, bar_s = bar_ld + 8, bar_p = bar_ld + 16, bar_acc = bar_ld + 24, bar_drain = bar_ld + 32;
  const uint32_t tmem_slot = bar_ld + 40, abort_any = bar_ld + 44;
  uint32_t* tile_bound = reinterpret_cast<uint32_t*>(smem_al + SM::kBar + 48);
  int32_t* seg_s = reinterpret_cast<int32_t*>(smem_al + SM::kSeg);
  const uint32_t pos_s = smem_base + SM::kPos, table_s = smem_base + SM::kTable, bins_s = table_s + rel.view.pitch * 4;
  uint8_t *table = smem_al + SM::kTable, *bins = table + rel.view.pitch * 4;

  if (tid == 0) {
    ptx::prefetch_tensormap(&tm_qkv);
    ptx::prefetch_tensormap(&tm_do);
    ptx::prefetch_tensormap(&tm_o);
    for (int b = 0; b < 5; ++b) ptx::mbar_init(bar_ld + 8 * b, 1);
    ptx::sts_s32(abort_any, 0);
    ptx::fence_mbar_init();
  }
  pdl_entry();
  const int Np = packed_rows(seg, n_seg, capacity);
  if (warp == 0) ptx::tmem_alloc(tmem_slot, 256);
  ptx::tc_fence_before_sync();
  __syncthreads();  // barriers and the TMEM address are visible
  ptx::tc_fence_after_sync();
  const uint32_t tmem = (uint32_t)ptx::lds_s32(tmem_slot);
  const uint32_t lane_base = (uint32_t)(quarter * 32) << 16;
  const float scale_log2e = scale * kLog2e;
  bool ok = true;  // a wait that gave up: everyone learns of it at the next barrier, and the CTA leaves its loops together
  auto wait = [&](uint32_t b, uint32_t parity) {
    ok = ptx::mbar_wait_or_abort_warp(b, parity, abort_any, d_status, SPA_ERR_TIMEOUT) && ok;
  };
  bool failed = false;
  uint32_t parity = 0;

  // the grid is a multiple of H: all of a CTA's items are of one head, whose table and bound it fetches once
  const int h = blockIdx.x % H;
  const float4* from = reinterpret_cast<const float4*>(rel.view.bias + (long long)h * rel.view.pitch);
  for (int i = tid; i < rel.view.pitch / 4; i += kThreads) reinterpret_cast<float4*>(table)[i] = from[i];
  float head_v;
  const int head_exp = rel_exponent(rel_head_bound(rel.grad, h, head_v));
  for (int item = blockIdx.x; item < n_items && !failed; item += gridDim.x) {
    const int s0 = item / H * chunk, count = n_seg - s0 < chunk ? n_seg - s0 : chunk;
    if (tid <= count) {
      const int o = ld_dep(seg + s0 + tid);
      seg_s[tid] = o < 0 ? 0 : (o < Np ? o : Np);
    }
    __syncthreads();
    int first = 0;
    auto length = [&](int s) { return seg_s[s + 1] - seg_s[s]; };
    for (;;) {
      // ---- the next tile: whole segments of `least` to 128 rows; the others are other kernels'
      while (first < count && (length(first) < least || length(first) > kShortMax)) ++first;
      if (first == count) break;
      const int lo = seg_s[first];
      int end = first + 1;
      while (end < count && length(end) >= least && length(end) <= kShortMax && seg_s[end + 1] - lo <= 128) ++end;
      const int n = seg_s[end] - lo;
      if (tid == 0) {
        *tile_bound = 0u;  // the others add to it behind their wait for the copies
        ptx::mbar_expect_tx(bar_ld, 5 * kTile);
        ptx::tma_load_2d(q_s, &tm_qkv, bar_ld, h * D, lo);
        ptx::tma_load_2d(k_s, &tm_qkv, bar_ld, C + h * D, lo);
        ptx::tma_load_2d(smem_base + SM::kV, &tm_qkv, bar_ld, 2 * C + h * D, lo);
        ptx::tma_load_2d(do_s, &tm_do, bar_ld, h * D, lo);
        ptx::tma_load_2d(smem_base + SM::kO, &tm_o, bar_ld, h * D, lo);
      }
      for (int i = tid; i < rel.view.pitch / 2; i += kThreads) reinterpret_cast<uint4*>(bins)[i] = make_uint4(0u, 0u, 0u, 0u);
      const int row = lo + rl;
      const bool valid = rl < n;
      const int own_pos = rel.view.pos[row];
      if (half == 0) ptx::sts_s32(pos_s + 4 * rl, -4 * own_pos);
      float my_lse = 0.f, row_peak = 0.f;
      int c_lo = 0, c_hi = 0;  // the row's columns
      if (valid) {
        my_lse = lse[(long long)h * capacity + row];
        if (rel.grad.peak != nullptr) row_peak = rel.grad.peak[(long long)h * capacity + row];
        int a = first, b = end;  // seg_s[a] <= row < seg_s[b]
        while (b - a > 1) {
          const int mid = (a + b) >> 1;
          if (seg_s[mid] <= row) a = mid; else b = mid;
        }
        c_lo = seg_s[a] - lo;
        c_hi = seg_s[b] - lo;
      }
      wait(bar_ld, parity);
      // ---- D_i = dO_i . O_i (both tiles carry the same swizzle: equal positions hold equal columns) and |dO_i|^2
      float my_D = 0.f, row_norm = 0.f;
      if (valid) {
        constexpr int kChunks = HT::kRowBytes / 16;
        const uint8_t *po = smem_al + SM::kO + rl * HT::kRowBytes, *pg = smem_al + SM::kDO + rl * HT::kRowBytes;
        const int rot = chunk_rot<D>(rl);
#pragma unroll
        for (int c = 0; c < kChunks; ++c) {
          float a[8], b[8];
          Vec16<__nv_bfloat16>::to_float(*reinterpret_cast<const uint4*>(po + ((c ^ rot) << 4)), a);
          Vec16<__nv_bfloat16>::to_float(*reinterpret_cast<const uint4*>(pg + ((c ^ rot) << 4)), b);
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            my_D = fmaf(a[e], b[e], my_D);
            row_norm = fmaf(b[e], b[e], row_norm);
          }
        }
        if (half == 0) {
          delta[(long long)h * capacity + row] = my_D;
          rel_check_row(rel.grad, h, my_lse, my_D);
        }
      }
      // a row without a key (lse = -inf, by its biases) has no weights
      my_lse = my_lse == -CUDART_INF_F ? CUDART_INF_F : my_lse * kLog2e;
      const uint32_t most = __reduce_max_sync(0xffffffffu, valid ? rel_row_bound(head_v, row_norm, row_peak) : 0u);
      if (half == 0 && lane == 0) atomicMax(tile_bound, most);
      // lines behind the tile's rows are other segments' or unspecified memory: the products behind sum over the rows of Q, K and dO
      {
        constexpr int kChunks = HT::kRowBytes / 16;
        for (int c = tid; c < (128 - n) * kChunks; c += kThreads) {
          const int off = (n + c / kChunks) * HT::kRowBytes + (c % kChunks) * 16;
          *reinterpret_cast<uint4*>(smem_al + SM::kQ + off) = make_uint4(0, 0, 0, 0);
          *reinterpret_cast<uint4*>(smem_al + SM::kK + off) = make_uint4(0, 0, 0, 0);
          *reinterpret_cast<uint4*>(smem_al + SM::kDO + off) = make_uint4(0, 0, 0, 0);
        }
        ptx::fence_proxy_async_smem();
      }
      ptx::tc_fence_before_sync();
      if (__syncthreads_or(!ok)) { failed = true; break; }  // tiles, positions and bins are ready, D has been taken from O
      ptx::tc_fence_after_sync();
      if (warp == 0) {
        constexpr uint32_t kIdescS = ptx::idesc_bf16_f32(128, 128, false, false);
        if (ptx::elect_one()) {
#pragma unroll
          for (int k = 0; k < D / 16; ++k)  // S = Q K^T
            ptx::mma_bf16(tmem, HT::kmajor(q_s, k), HT::kmajor(k_s, k), kIdescS, k != 0 ? 1u : 0u);
#pragma unroll
          for (int k = 0; k < D / 16; ++k)  // dP = dO V^T
            ptx::mma_bf16(tmem + 128, HT::kmajor(do_s, k), HT::kmajor(smem_base + SM::kV, k), kIdescS, k != 0 ? 1u : 0u);
          ptx::mma_commit(bar_s);
        }
        __syncwarp();
      }
      const int bound_exp = rel_exponent(__uint_as_float(*reinterpret_cast<volatile uint32_t*>(tile_bound)));
      const float bin_scale = rel_item_scale(bound_exp);
      const int bin_shift = rel_item_shift(rel.grad, bound_exp, head_exp);
      const uint32_t bias_at = 4 * (rel.view.center + own_pos);
      wait(bar_s, parity);
      ptx::tc_fence_after_sync();
      // ---- P and dS of this thread's 64 columns, 32 at a time (V and O have been read: the products above have completed)
      uint8_t* prow = smem_al + SM::kP + half * (kOp / 2) + rl * 128;
      uint8_t* dsrow = smem_al + SM::kDS + half * (kOp / 2) + rl * 128;
      const int rsw = rl & 7;
      uint32_t pk_ds[2][16];
#pragma unroll
      for (int part = 0; part < 2; ++part) {
        const int col0 = half * 64 + part * 32;
        const bool need = col0 < c_hi && col0 + 32 > c_lo;
        uint32_t pk_p[16];
#pragma unroll
        for (int j = 0; j < 16; ++j) pk_p[j] = pk_ds[part][j] = 0u;
        if (__any_sync(0xffffffffu, need)) {
          uint32_t rs[32], rp[32];
          ptx::tmem_ld_32x32(tmem + lane_base + col0, rs);
          ptx::tmem_ld_32x32(tmem + lane_base + 128 + col0, rp);
          ptx::tmem_ld_wait();
          if (need) {
            const uint64_t scale2 = ptx::pair(scale_log2e, scale_log2e), lse2 = ptx::pair(-my_lse, -my_lse), D2 = ptx::pair(-my_D, -my_D);
            const uint32_t pos_at = pos_s + 4 * col0;
            RelKeys<> keys(pos_at);
#pragma unroll
            for (int j = 0; j < 32; j += 4) {
              int k[4];
              keys.next(j, 32, k);
#pragma unroll
              for (int u = 0; u < 4; u += 2) {
                const float b0 = ptx::lds_f32(table_s + bias_at + k[u]), b1 = ptx::lds_f32(table_s + bias_at + k[u + 1]);
                const uint64_t s2 = ptx::fma2(ptx::pair(rs[j + u], rs[j + u + 1]), scale2, ptx::pair(b0, b1));
                ptx::unpair(ptx::add2(s2, lse2), rs[j + u], rs[j + u + 1]);
                ptx::unpair(ptx::add2(ptx::pair(rp[j + u], rp[j + u + 1]), D2), rp[j + u], rp[j + u + 1]);
              }
            }
            if (!(col0 >= c_lo && col0 + 32 <= c_hi)) {
#pragma unroll
              for (int j = 0; j < 32; ++j)
                if ((unsigned)(col0 + j - c_lo) >= (unsigned)(c_hi - c_lo)) { rs[j] = 0xff800000u; rp[j] = 0u; }  // p = 2^-inf = 0
            }
#pragma unroll
            for (int j = 0; j < 32; ++j) rs[j] = __float_as_uint(ptx::ex2_approx(__uint_as_float(rs[j])));
            // the table's gradient: a pair's bin is where its bias came from
            RelKeys<> again(pos_at);
#pragma unroll
            for (int j = 0; j < 32; j += 4) {
              int k[4];
              again.next(j, 32, k);
              uint32_t hi[4], lo[4];
#pragma unroll
              for (int u = j; u < j + 4; u += 2) {
                pk_p[u >> 1] = ptx::bf16_pair(__uint_as_float(rs[u]), __uint_as_float(rs[u + 1]));
                const uint64_t d = ptx::mul2(ptx::pair(rs[u], rs[u + 1]), ptx::pair(rp[u], rp[u + 1]));
                float d0, d1;
                ptx::unpair(d, d0, d1);
                pk_ds[part][u >> 1] = ptx::bf16_pair(d0, d1);
                rel_fixed(d, bin_scale, hi + u - j, lo + u - j);
              }
#pragma unroll
              for (int u = 0; u < 4; ++u) rel_bin(bins_s + bias_at + k[u], rel.view.pitch * 4, hi[u], lo[u]);
            }
          }
          __syncwarp();
        }
#pragma unroll
        for (int c = 0; c < 4; ++c)
          *reinterpret_cast<uint4*>(prow + (((part * 4 + c) ^ rsw) << 4)) = make_uint4(pk_p[4 * c], pk_p[4 * c + 1], pk_p[4 * c + 2], pk_p[4 * c + 3]);
      }
      auto store_ds = [&]() {
#pragma unroll
        for (int part = 0; part < 2; ++part)
#pragma unroll
          for (int c = 0; c < 4; ++c)
            *reinterpret_cast<uint4*>(dsrow + (((part * 4 + c) ^ rsw) << 4)) =
                make_uint4(pk_ds[part][4 * c], pk_ds[part][4 * c + 1], pk_ds[part][4 * c + 2], pk_ds[part][4 * c + 3]);
      };
      constexpr uint32_t kIdescT = ptx::idesc_bf16_f32(128, D, true, true);   // A = P^T or dS^T (MN-major), B MN-major
      constexpr uint32_t kIdescQ = ptx::idesc_bf16_f32(128, D, false, true);  // A = dS (K-major), B = K (MN-major)
      if (SM::kTwo) store_ds();
      ptx::fence_proxy_async_smem();
      ptx::tc_fence_before_sync();
      if (__syncthreads_or(!ok)) { failed = true; break; }  // P is there; every thread holds its fp32 values: their columns take the results
      ptx::tc_fence_after_sync();
      if (warp == 0) {
        if (ptx::elect_one()) {
#pragma unroll
          for (int k = 0; k < 8; ++k)  // dV = P^T dO: 16 query rows per step
            ptx::mma_bf16(tmem, ptx::smem_desc_sw128(p_s + k * 2048, kOp / 2, 1024), HT::mnmajor(do_s, k), kIdescT, k != 0 ? 1u : 0u);
          if (!SM::kTwo) ptx::mma_commit(bar_p);
        }
        __syncwarp();
      }
      if (!SM::kTwo) {
        wait(bar_p, parity);
        store_ds();
        ptx::fence_proxy_async_smem();
        ptx::tc_fence_before_sync();
        if (__syncthreads_or(!ok)) { failed = true; break; }
        ptx::tc_fence_after_sync();
      }
      if (warp == 0) {
        if (ptx::elect_one()) {
#pragma unroll
          for (int k = 0; k < 8; ++k)  // dK = dS^T Q
            ptx::mma_bf16(tmem + D, ptx::smem_desc_sw128(ds_s + k * 2048, kOp / 2, 1024), HT::mnmajor(q_s, k), kIdescT, k != 0 ? 1u : 0u);
#pragma unroll
          for (int k = 0; k < 8; ++k)  // dQ = dS K: 16 keys per step, 64 keys per panel
            ptx::mma_bf16(tmem + 2 * D, ptx::smem_desc_sw128(ds_s + (k >> 2) * (kOp / 2) + (k & 3) * 32, 16, 1024), HT::mnmajor(k_s, k),
                          kIdescQ, k != 0 ? 1u : 0u);
          ptx::mma_commit(bar_acc);
        }
        __syncwarp();
      }
      // ---- the tile's bins to the head's sums, under the products
      rel_flush<kThreads>(rel, reinterpret_cast<const int*>(bins), h, bin_shift, tid);
      wait(bar_acc, parity);
      ptx::tc_fence_after_sync();
      // ---- dV, dK, dQ rows as bf16 into the Q, K, dO tiles' memory (idle now), from where whole lines go out
      bool again_k = false, again_q = false;
#pragma unroll
      for (int a = 0; a < 3; ++a) {
        const float mul = a == 0 ? 1.f : scale;
        uint32_t r[kDh];
        if (kDh == 32) ptx::tmem_ld_32x32(tmem + lane_base + a * D + half * kDh, r);
        else ptx::tmem_ld_32x16(tmem + lane_base + a * D + half * kDh, r);
        ptx::tmem_ld_wait();
        const int rot = chunk_rot<D>(rl);
        float sum = 0.f;
#pragma unroll
        for (int g = 0; g < kDh / 8; ++g) {
          float v[8];
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            v[e] = __uint_as_float(r[g * 8 + e]) * mul;
            sum += fabsf(v[e]);
          }
          *reinterpret_cast<uint4*>(smem_al + a * kTile + rl * HT::kRowBytes + (((half * (kDh / 8) + g) ^ rot) << 4)) =
              Vec16<__nv_bfloat16>::from_float(v);
        }
        const bool bad = !(sum < CUDART_INF_F);
        if (a < 2) again_k = again_k || bad; else again_q = bad;
      }
      // several segments share the tile: see rel_redo
      if (valid && end > first + 1) {
        if (again_q) rel_redo(rel.grad, false, half, h, row);
        if (again_k) rel_redo(rel.grad, true, half, h, row);
      }
      ptx::tc_fence_before_sync();
      if (__syncthreads_or(!ok)) { failed = true; break; }
      const long long ld = 3LL * C;
      copy_tile_out<D, kThreads>(smem_al, dqkv + 2 * C + h * D, ld, lo, lo + n, tid);           // dV
      copy_tile_out<D, kThreads>(smem_al + kTile, dqkv + C + h * D, ld, lo, lo + n, tid);       // dK
      copy_tile_out<D, kThreads>(smem_al + 2 * kTile, dqkv + h * D, ld, lo, lo + n, tid);       // dQ
      ptx::fence_proxy_async_smem();  // the next tile's copies take this memory
      parity ^= 1;
      first = end;
      __syncthreads();
    }
    __syncthreads();  // the offsets' memory is free for the next segments
  }
  if (failed) {  // what is in flight lands before the memory is released
    if (tid == 0) ptx::mbar_wait(bar_ld, parity);
    if (warp == 0) {
      if (ptx::elect_one()) ptx::mma_commit(bar_drain);
      __syncwarp();
      ptx::mbar_wait(bar_drain, 0);
    }
    __syncwarp();
  }
  ptx::tc_fence_before_sync();
  __syncthreads();
  if (warp == 0) {
    ptx::tc_fence_after_sync();
    ptx::tmem_dealloc(tmem, 256);
  }
}

// ------------------------------------------------------------------------------------------------
// Segments of at most 64 rows, two to a tile: rows 0 - 63 are segment a's, rows 64 - 127 segment b's, and a row's 64 columns of S and
// dP are its own segment's alone.  Every operand is laid out as blocks of 64 rows [a][zeros][b]:
//   S = [Q_a; 0] K_a^T + [0; Q_b] K_b^T in 64 columns of TMEM (and dP likewise): the two 128-row operands begin at a and at the zeros;
//   dV = P^T dO, K a step of queries: P^T's columns a | b begin 8 KB apart, so that the steps of a see a and zeros, those of b zeros and b;
//   dQ as S, dK as dV.
// Nothing is computed for a pair of different segments, each thread has one group of 32 columns, and three CTAs fit an SM (d = 32):
// S and dP take 128 columns of TMEM instead of 256, V and O lie where P will, dS follows P.  Zeros times an infinity or NaN of the other
// segment are NaN: lines behind a segment are cleared, rows of dQ, dK and dV are formed again (rel_redo), and where K is not
// finite, the head's column of dtable is NaN (as where V, dO or a row's statistics are).
template <int D> struct PairSmem {
  static constexpr int kB = 64 * D * 2;            // a block of Q, K, V, dO or O
  static constexpr int kOp = 64 * 128;             // a block of P or dS: 64 query rows of 64 keys
  static constexpr int kQ = 0, kDO = 3 * kB, kK = 6 * kB, kP = 8 * kB;
  static constexpr int kV = kP, kVb = D == 32 ? kP + kB : kP + 2 * kOp;
  static constexpr int kO = D == 32 ? kP + 2 * kOp : kP + 3 * kOp;
  static constexpr int kBar = kP + 3 * kOp + (D == 32 ? 0 : 2 * kB);
  static constexpr int kSeg = kBar + 64;
  static constexpr int kPos = kSeg + 192;
  static constexpr int kTable = kPos + 128 * 4;
  static constexpr int kBytes = kTable + 1024;
  static constexpr int kTmem = D == 32 ? 128 : 256;
  static constexpr int kPerSm = D == 32 ? 3 : 2;
  static constexpr int kMost = (228 * 1024 / kPerSm - 1024) / 16 * 16;
};

template <int D>
__global__ void __launch_bounds__(kThreads, PairSmem<D>::kPerSm)
rel_bwd_pair_kernel(const __grid_constant__ CUtensorMap tm_qkv, const __grid_constant__ CUtensorMap tm_do,
                    const __grid_constant__ CUtensorMap tm_o, const float* lse, float* delta, const int32_t* seg, int n_seg, int chunk,
                    int capacity, int C, int H, float scale, __nv_bfloat16* __restrict__ dqkv, const RelBwd rel, int32_t* d_status) {
  using HT = HeadTile<D>;
  using SM = PairSmem<D>;
  constexpr int kB = SM::kB, kOp = SM::kOp, kDh = D / 2, kChunks = HT::kRowBytes / 16;
  constexpr float kLog2e = 1.4426950408889634f;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int quarter = warp & 3, half = warp >> 2, rl = quarter * 32 + lane;
  const int which = quarter >> 1, rr = rl & 63;  // the row's segment, a or b, and its place there
  const int n_chunks = (n_seg + chunk - 1) / chunk, n_items = n_chunks * H;

  extern __shared__ uint8_t smem_raw[];
  const uint32_t smem_base = (ptx::smem_u32(smem_raw) + 1023u) & ~1023u;
  uint8_t* smem_al = smem_raw + (smem_base - ptx::smem_u32(smem_raw));
  auto q_off = [](int s) { return SM::kQ + 2 * kB * s; };
  auto do_off = [](int s) { return SM::kDO + 2 * kB * s; };
  auto k_off = [](int s) { return SM::kK + kB * s; };
  auto v_off = [](int s) { return s == 0 ? SM::kV : SM::kVb; };
  auto o_off = [](int s) { return SM::kO + kB * s; };
  const uint32_t p_s = smem_base + SM::kP;
  const uint32_t bar_ld = smem_base + SM::kBar, bar_s = bar_ld + 8, bar_p = bar_ld + 16, bar_acc = bar_ld + 24, bar_drain = bar_ld + 32;
  const uint32_t tmem_slot = bar_ld + 40, abort_any = bar_ld + 44;
  uint32_t* tile_bound = reinterpret_cast<uint32_t*>(smem_al + SM::kBar + 48);
  int32_t* seg_s = reinterpret_cast<int32_t*>(smem_al + SM::kSeg);
  const uint32_t pos_s = smem_base + SM::kPos, table_s = smem_base + SM::kTable, bins_s = table_s + rel.view.pitch * 4;
  uint8_t *table = smem_al + SM::kTable, *bins = table + rel.view.pitch * 4;

  if (tid == 0) {
    ptx::prefetch_tensormap(&tm_qkv);
    ptx::prefetch_tensormap(&tm_do);
    ptx::prefetch_tensormap(&tm_o);
    for (int b = 0; b < 5; ++b) ptx::mbar_init(bar_ld + 8 * b, 1);
    ptx::sts_s32(abort_any, 0);
    ptx::fence_mbar_init();
  }
  for (int i = tid; i < kB / 16; i += kThreads) {  // the blocks of zeros
    reinterpret_cast<uint4*>(smem_al + SM::kQ + kB)[i] = make_uint4(0u, 0u, 0u, 0u);
    reinterpret_cast<uint4*>(smem_al + SM::kDO + kB)[i] = make_uint4(0u, 0u, 0u, 0u);
  }
  for (int i = tid; i < kOp / 16; i += kThreads) reinterpret_cast<uint4*>(smem_al + SM::kP + kOp)[i] = make_uint4(0u, 0u, 0u, 0u);
  ptx::fence_proxy_async_smem();
  pdl_entry();
  const int Np = packed_rows(seg, n_seg, capacity);
  if (warp == 0) ptx::tmem_alloc(tmem_slot, SM::kTmem);
  ptx::tc_fence_before_sync();
  __syncthreads();  // barriers, zeros and the TMEM address are visible
  ptx::tc_fence_after_sync();
  const uint32_t tmem = (uint32_t)ptx::lds_s32(tmem_slot);
  const uint32_t lane_base = (uint32_t)(quarter * 32) << 16;
  const float scale_log2e = scale * kLog2e;
  bool ok = true;
  auto wait = [&](uint32_t b, uint32_t parity) {
    ok = ptx::mbar_wait_or_abort_warp(b, parity, abort_any, d_status, SPA_ERR_TIMEOUT) && ok;
  };
  bool failed = false;
  uint32_t parity = 0;

  // the grid is a multiple of H: all of a CTA's items are of one head, whose table and bound it fetches once
  const int h = blockIdx.x % H;
  const float4* from = reinterpret_cast<const float4*>(rel.view.bias + (long long)h * rel.view.pitch);
  for (int i = tid; i < rel.view.pitch / 4; i += kThreads) reinterpret_cast<float4*>(table)[i] = from[i];
  float head_v;
  const int head_exp = rel_exponent(rel_head_bound(rel.grad, h, head_v));
  for (int item = blockIdx.x; item < n_items && !failed; item += gridDim.x) {
    const int s0 = item / H * chunk, count = n_seg - s0 < chunk ? n_seg - s0 : chunk;
    if (tid <= count) {
      const int o = ld_dep(seg + s0 + tid);
      seg_s[tid] = o < 0 ? 0 : (o < Np ? o : Np);
    }
    __syncthreads();
    auto length = [&](int s) { return seg_s[s + 1] - seg_s[s]; };
    int next = 0;
    auto take = [&](int& lo, int& n) {  // the next segment of at most 64 rows; n = 0: there is none
      while (next < count && (length(next) <= 0 || length(next) > kPairMax)) ++next;
      n = next < count ? length(next) : 0;
      lo = next < count ? seg_s[next] : 0;
      ++next;
    };
    for (;;) {
      int lo_a, n_a, lo_b, n_b;
      take(lo_a, n_a);
      if (n_a == 0) break;
      take(lo_b, n_b);
      if (tid == 0) {
        *tile_bound = 0u;  // the others add to it behind their wait for the copies
        ptx::mbar_expect_tx(bar_ld, (n_b > 0 ? 10 : 5) * kB);
        for (int s = 0; s < (n_b > 0 ? 2 : 1); ++s) {
          const int lo = s == 0 ? lo_a : lo_b;
          ptx::tma_load_2d(smem_base + q_off(s), &tm_qkv, bar_ld, h * D, lo);
          ptx::tma_load_2d(smem_base + k_off(s), &tm_qkv, bar_ld, C + h * D, lo);
          ptx::tma_load_2d(smem_base + v_off(s), &tm_qkv, bar_ld, 2 * C + h * D, lo);
          ptx::tma_load_2d(smem_base + do_off(s), &tm_do, bar_ld, h * D, lo);
          ptx::tma_load_2d(smem_base + o_off(s), &tm_o, bar_ld, h * D, lo);
        }
      }
      for (int i = tid; i < rel.view.pitch / 2; i += kThreads) reinterpret_cast<uint4*>(bins)[i] = make_uint4(0u, 0u, 0u, 0u);
      const int lo = which == 0 ? lo_a : lo_b, n = which == 0 ? n_a : n_b, row = lo + rr;
      const bool valid = rr < n;
      const int own_pos = rel.view.pos[row];
      if (half == 0) ptx::sts_s32(pos_s + 4 * rl, -4 * own_pos);
      float my_lse = 0.f, row_peak = 0.f;
      if (valid) {
        my_lse = lse[(long long)h * capacity + row];
        if (rel.grad.peak != nullptr) row_peak = rel.grad.peak[(long long)h * capacity + row];
      }
      wait(bar_ld, parity);
      // ---- D_i = dO_i . O_i (both blocks carry the same swizzle: equal positions hold equal columns), |dO_i|^2, whether K is finite
      float my_D = 0.f, row_norm = 0.f;
      if (valid) {
        const uint8_t *po = smem_al + o_off(which) + rr * HT::kRowBytes, *pg = smem_al + do_off(which) + rr * HT::kRowBytes;
        const uint8_t* pk = smem_al + k_off(which) + rr * HT::kRowBytes;
        const int rot = chunk_rot<D>(rr);
#pragma unroll
        for (int c = 0; c < kChunks; ++c) {
          float a[8], b[8];
          Vec16<__nv_bfloat16>::to_float(*reinterpret_cast<const uint4*>(po + ((c ^ rot) << 4)), a);
          Vec16<__nv_bfloat16>::to_float(*reinterpret_cast<const uint4*>(pg + ((c ^ rot) << 4)), b);
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            my_D = fmaf(a[e], b[e], my_D);
            row_norm = fmaf(b[e], b[e], row_norm);
          }
        }
        float k_abs = 0.f;
#pragma unroll
        for (int c = 0; c < kChunks / 2; ++c) {  // the row's two threads look at half of it each
          float a[8];
          Vec16<__nv_bfloat16>::to_float(*reinterpret_cast<const uint4*>(pk + (((half * (kChunks / 2) + c) ^ rot) << 4)), a);
#pragma unroll
          for (int e = 0; e < 8; ++e) k_abs = fmaxf(k_abs, fabsf(a[e]) < CUDART_INF_F ? 0.f : 1.f);
        }
        if (k_abs != 0.f) rel.grad.bad[h] = 1;
        if (half == 0) {
          delta[(long long)h * capacity + row] = my_D;
          rel_check_row(rel.grad, h, my_lse, my_D);
        }
      }
      my_lse = my_lse == -CUDART_INF_F ? CUDART_INF_F : my_lse * kLog2e;  // a row without a key has no weights
      const uint32_t most = __reduce_max_sync(0xffffffffu, valid ? rel_row_bound(head_v, row_norm, row_peak) : 0u);
      if (half == 0 && lane == 0) atomicMax(tile_bound, most);
      // lines behind the segments' rows are other segments', unspecified memory, or an earlier tile's
      for (int i = tid; i < (128 - n_a - n_b) * kChunks; i += kThreads) {
        int line = i / kChunks, s = 0;
        if (line < 64 - n_a) line += n_a; else { line += n_b - (64 - n_a); s = 1; }
        const int off = line * HT::kRowBytes + i % kChunks * 16;
        *reinterpret_cast<uint4*>(smem_al + q_off(s) + off) = make_uint4(0, 0, 0, 0);
        *reinterpret_cast<uint4*>(smem_al + k_off(s) + off) = make_uint4(0, 0, 0, 0);
        *reinterpret_cast<uint4*>(smem_al + v_off(s) + off) = make_uint4(0, 0, 0, 0);
        *reinterpret_cast<uint4*>(smem_al + do_off(s) + off) = make_uint4(0, 0, 0, 0);
      }
      ptx::fence_proxy_async_smem();
      ptx::tc_fence_before_sync();
      if (__syncthreads_or(!ok)) { failed = true; break; }  // blocks, positions and bins are ready, D has been taken from O
      ptx::tc_fence_after_sync();
      if (warp == 0) {
        constexpr uint32_t kIdescS = ptx::idesc_bf16_f32(128, 64, false, false);
        if (ptx::elect_one()) {
#pragma unroll
          for (int s = 0; s < 2; ++s)
#pragma unroll
            for (int k = 0; k < D / 16; ++k)  // S = [Q_a; 0] K_a^T + [0; Q_b] K_b^T
              ptx::mma_bf16(tmem, HT::kmajor(smem_base + SM::kQ + s * kB, k), HT::kmajor(smem_base + k_off(s), k), kIdescS, s + k != 0 ? 1u : 0u);
#pragma unroll
          for (int s = 0; s < 2; ++s)
#pragma unroll
            for (int k = 0; k < D / 16; ++k)  // dP = [dO_a; 0] V_a^T + [0; dO_b] V_b^T
              ptx::mma_bf16(tmem + 64, HT::kmajor(smem_base + SM::kDO + s * kB, k), HT::kmajor(smem_base + v_off(s), k), kIdescS, s + k != 0 ? 1u : 0u);
          ptx::mma_commit(bar_s);
        }
        __syncwarp();
      }
      const int bound_exp = rel_exponent(__uint_as_float(*reinterpret_cast<volatile uint32_t*>(tile_bound)));
      const float bin_scale = rel_item_scale(bound_exp);
      const int bin_shift = rel_item_shift(rel.grad, bound_exp, head_exp);
      const uint32_t bias_at = 4 * (rel.view.center + own_pos);
      wait(bar_s, parity);
      ptx::tc_fence_after_sync();
      // ---- P and dS of this thread's 32 columns, 16 at a time (V and O have been read: the products above have completed)
      const int col0 = half * 32;
      uint8_t* prow = smem_al + SM::kP + 2 * kOp * which + rr * 128;
      const int rsw = rr & 7;
      uint32_t pk_ds[16];
#pragma unroll
      for (int part = 0; part < 2; ++part) {
        uint32_t pk_p[8], rs[16], rp[16];
        const int c0 = col0 + part * 16;
        ptx::tmem_ld_32x16(tmem + lane_base + c0, rs);
        ptx::tmem_ld_32x16(tmem + lane_base + 64 + c0, rp);
        ptx::tmem_ld_wait();
#pragma unroll
        for (int j = 0; j < 8; ++j) pk_p[j] = pk_ds[part * 8 + j] = 0u;
        if (valid && c0 < n) {
          const uint64_t scale2 = ptx::pair(scale_log2e, scale_log2e), lse2 = ptx::pair(-my_lse, -my_lse), D2 = ptx::pair(-my_D, -my_D);
          const uint32_t pos_at = pos_s + 4 * (64 * which + c0);
          RelKeys<> keys(pos_at);
#pragma unroll
          for (int j = 0; j < 16; j += 4) {
            int k[4];
            keys.next(j, 16, k);
#pragma unroll
            for (int u = 0; u < 4; u += 2) {
              const float b0 = ptx::lds_f32(table_s + bias_at + k[u]), b1 = ptx::lds_f32(table_s + bias_at + k[u + 1]);
              const uint64_t s2 = ptx::fma2(ptx::pair(rs[j + u], rs[j + u + 1]), scale2, ptx::pair(b0, b1));
              ptx::unpair(ptx::add2(s2, lse2), rs[j + u], rs[j + u + 1]);
              ptx::unpair(ptx::add2(ptx::pair(rp[j + u], rp[j + u + 1]), D2), rp[j + u], rp[j + u + 1]);
            }
          }
          if (c0 + 16 > n) {
#pragma unroll
            for (int j = 0; j < 16; ++j)
              if (c0 + j >= n) { rs[j] = 0xff800000u; rp[j] = 0u; }  // p = 2^-inf = 0
          }
#pragma unroll
          for (int j = 0; j < 16; ++j) rs[j] = __float_as_uint(ptx::ex2_approx(__uint_as_float(rs[j])));
          // the table's gradient: a pair's bin is where its bias came from
          RelKeys<> again(pos_at);
#pragma unroll
          for (int j = 0; j < 16; j += 4) {
            int k[4];
            again.next(j, 16, k);
            uint32_t hi[4], lo[4];
#pragma unroll
            for (int u = j; u < j + 4; u += 2) {
              pk_p[u >> 1] = ptx::bf16_pair(__uint_as_float(rs[u]), __uint_as_float(rs[u + 1]));
              const uint64_t d = ptx::mul2(ptx::pair(rs[u], rs[u + 1]), ptx::pair(rp[u], rp[u + 1]));
              float d0, d1;
              ptx::unpair(d, d0, d1);
              pk_ds[part * 8 + (u >> 1)] = ptx::bf16_pair(d0, d1);
              rel_fixed(d, bin_scale, hi + u - j, lo + u - j);
            }
#pragma unroll
            for (int u = 0; u < 4; ++u) rel_bin(bins_s + bias_at + k[u], rel.view.pitch * 4, hi[u], lo[u]);
          }
        }
        __syncwarp();
#pragma unroll
        for (int c = 0; c < 2; ++c)
          *reinterpret_cast<uint4*>(prow + (((half * 4 + part * 2 + c) ^ rsw) << 4)) =
              make_uint4(pk_p[4 * c], pk_p[4 * c + 1], pk_p[4 * c + 2], pk_p[4 * c + 3]);
      }
      constexpr uint32_t kIdescT = ptx::idesc_bf16_f32(128, D, true, true);   // A = P^T or dS^T (MN-major), B MN-major
      constexpr uint32_t kIdescQ = ptx::idesc_bf16_f32(128, D, false, true);  // A = dS (K-major), B = K (MN-major)
      ptx::fence_proxy_async_smem();
      ptx::tc_fence_before_sync();
      if (__syncthreads_or(!ok)) { failed = true; break; }  // P is there; every thread holds its fp32 values: their columns take the results
      ptx::tc_fence_after_sync();
      if (warp == 0) {
        if (ptx::elect_one()) {
#pragma unroll
          for (int s = 0; s < 2; ++s)
#pragma unroll
            for (int k = 0; k < 4; ++k)  // dV = P^T dO: 16 queries of a segment per step
              ptx::mma_bf16(tmem, ptx::smem_desc_sw128(p_s + s * kOp + k * 2048, kOp, 1024), HT::mnmajor(smem_base + do_off(s), k), kIdescT,
                            s + k != 0 ? 1u : 0u);
          ptx::mma_commit(bar_p);
        }
        __syncwarp();
      }
      // ---- the tile's bins to the head's sums, under the products
      rel_flush<kThreads>(rel, reinterpret_cast<const int*>(bins), h, bin_shift, tid);
      wait(bar_p, parity);  // dS takes the memory of P
#pragma unroll
      for (int c = 0; c < 4; ++c)
        *reinterpret_cast<uint4*>(prow + (((half * 4 + c) ^ rsw) << 4)) = make_uint4(pk_ds[4 * c], pk_ds[4 * c + 1], pk_ds[4 * c + 2], pk_ds[4 * c + 3]);
      ptx::fence_proxy_async_smem();
      ptx::tc_fence_before_sync();
      if (__syncthreads_or(!ok)) { failed = true; break; }
      ptx::tc_fence_after_sync();
      if (warp == 0) {
        if (ptx::elect_one()) {
#pragma unroll
          for (int s = 0; s < 2; ++s)
#pragma unroll
            for (int k = 0; k < 4; ++k)  // dK = dS^T Q
              ptx::mma_bf16(tmem + D, ptx::smem_desc_sw128(p_s + s * kOp + k * 2048, kOp, 1024), HT::mnmajor(smem_base + q_off(s), k), kIdescT,
                            s + k != 0 ? 1u : 0u);
#pragma unroll
          for (int s = 0; s < 2; ++s)
#pragma unroll
            for (int k = 0; k < 4; ++k)  // dQ = [dS_a; 0] K_a + [0; dS_b] K_b: 16 keys per step
              ptx::mma_bf16(tmem + 2 * D, ptx::smem_desc_sw128(p_s + s * kOp + k * 32, 16, 1024), HT::mnmajor(smem_base + k_off(s), k), kIdescQ,
                            s + k != 0 ? 1u : 0u);
          ptx::mma_commit(bar_acc);
        }
        __syncwarp();
      }
      wait(bar_acc, parity);
      ptx::tc_fence_after_sync();
      // ---- dV, dK, dQ rows as bf16 into the K, Q and dO blocks (idle now), from where whole lines go out
      bool again_k = false, again_q = false;
#pragma unroll
      for (int a = 0; a < 3; ++a) {
        const float mul = a == 0 ? 1.f : scale;
        uint32_t r[kDh];
        if (kDh == 32) ptx::tmem_ld_32x32(tmem + lane_base + a * D + half * kDh, r);
        else ptx::tmem_ld_32x16(tmem + lane_base + a * D + half * kDh, r);
        ptx::tmem_ld_wait();
        uint8_t* to = smem_al + (a == 0 ? k_off(which) : a == 1 ? q_off(which) : do_off(which)) + rr * HT::kRowBytes;
        const int rot = chunk_rot<D>(rr);
        float sum = 0.f;
#pragma unroll
        for (int g = 0; g < kDh / 8; ++g) {
          float v[8];
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            v[e] = __uint_as_float(r[g * 8 + e]) * mul;
            sum += fabsf(v[e]);
          }
          *reinterpret_cast<uint4*>(to + (((half * (kDh / 8) + g) ^ rot) << 4)) = Vec16<__nv_bfloat16>::from_float(v);
        }
        const bool bad = !(sum < CUDART_INF_F);
        if (a < 2) again_k = again_k || bad; else again_q = bad;
      }
      if (valid && n_b > 0) {
        if (again_q) rel_redo(rel.grad, false, half, h, row);
        if (again_k) rel_redo(rel.grad, true, half, h, row);
      }
      ptx::tc_fence_before_sync();
      if (__syncthreads_or(!ok)) { failed = true; break; }
      const long long ld = 3LL * C;
#pragma unroll
      for (int a = 0; a < 3; ++a) {
        __nv_bfloat16* dst = dqkv + (a == 0 ? 2 * C : a == 1 ? C : 0) + h * D;
#pragma unroll
        for (int i = tid; i < 128 * kChunks; i += kThreads) {
          const int r = i / kChunks, c = i % kChunks, s = r >> 6, q = r & 63;
          const uint8_t* src = smem_al + (a == 0 ? k_off(s) : a == 1 ? q_off(s) : do_off(s)) + q * HT::kRowBytes + ((c ^ chunk_rot<D>(q)) << 4);
          if (q < (s == 0 ? n_a : n_b))
            *reinterpret_cast<uint4*>(dst + (long long)((s == 0 ? lo_a : lo_b) + q) * ld + c * 8) = *reinterpret_cast<const uint4*>(src);
        }
      }
      ptx::fence_proxy_async_smem();  // the next tile's copies take this memory
      parity ^= 1;
      __syncthreads();
    }
    __syncthreads();  // the offsets' memory is free for the next segments
  }
  if (failed) {  // what is in flight lands before the memory is released
    if (tid == 0) ptx::mbar_wait(bar_ld, parity);
    if (warp == 0) {
      if (ptx::elect_one()) ptx::mma_commit(bar_drain);
      __syncwarp();
      ptx::mbar_wait(bar_drain, 0);
    }
    __syncwarp();
  }
  ptx::tc_fence_before_sync();
  __syncthreads();
  if (warp == 0) {
    ptx::tc_fence_after_sync();
    ptx::tmem_dealloc(tmem, SM::kTmem);
  }
}

// Segments that a CTA takes at a time: so many that it gets about two items (512 windows of 7 x 7, 12 heads of 32: four 105 us, two 93, one 109); by fours, of which the
// tiles take two, three or four together.
int chunk_of(int n_seg, int H, int ctas) {
  long long chunk = (long long)n_seg * H / (2 * ctas);
  chunk = chunk < 1 ? 1 : (chunk > kMaxChunk ? kMaxChunk : chunk);
  return (int)(chunk >= 4 ? chunk & ~3ll : chunk);
}

template <int D>
int launch_pair(const spa_params& p, const void* qkv, const void* ao, const float* lse, const void* dao, const int32_t* seg, int n_seg,
                const RelBwd& rel, void* dqkv, float* delta, int32_t* d_status, cudaStream_t st) {
  CUtensorMap tm_qkv, tm_do, tm_o;
  if (!make_tmap_bf16_2d(&tm_qkv, qkv, 3ull * p.C, p.capacity, 6ull * p.C, D, 64, D * 2) ||
      !make_tmap_bf16_2d(&tm_do, dao, (uint64_t)p.C, p.capacity, 2ull * p.C, D, 64, D * 2) ||
      !make_tmap_bf16_2d(&tm_o, ao, (uint64_t)p.C, p.capacity, 2ull * p.C, D, 64, D * 2))
    return SPA_ERR_UNSUPPORTED;
  auto kern = rel_bwd_pair_kernel<D>;
  static DeviceOnce attr;
  cudaError_t ea = attr.run([&] { return cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, PairSmem<D>::kMost); });
  if (ea != cudaSuccess) { set_cuda_error(ea, "rel_bwd_pair_kernel"); return SPA_ERR_CUDA; }
  const int ctas = PairSmem<D>::kPerSm * kNumSMs / p.H * p.H, chunk = chunk_of(n_seg, p.H, ctas);
  const long long items = (long long)((n_seg + chunk - 1) / chunk) * p.H;
  launch_pdl(kern, (int)(items < ctas ? items : ctas), kThreads, PairSmem<D>::kBytes + 3 * rel.view.pitch * 4, st, tm_qkv, tm_do, tm_o, lse, delta,
             seg, n_seg, chunk, p.capacity, p.C, p.H, softmax_scale_of(p), (__nv_bfloat16*)dqkv, rel, d_status);
  SPA_CUDA_CHECK_LAUNCH("rel_bwd_pair_kernel");
  return SPA_OK;
}

template <int D>
int launch(const spa_params& p, const void* qkv, const void* ao, const float* lse, const void* dao, const int32_t* seg, int n_seg,
           const RelBwd& rel, void* dqkv, float* delta, int least, int32_t* d_status, cudaStream_t st) {
  CUtensorMap tm_qkv, tm_do, tm_o;
  if (!make_tmap_bf16_2d(&tm_qkv, qkv, 3ull * p.C, p.capacity, 6ull * p.C, D, 128, D * 2) ||
      !make_tmap_bf16_2d(&tm_do, dao, (uint64_t)p.C, p.capacity, 2ull * p.C, D, 128, D * 2) ||
      !make_tmap_bf16_2d(&tm_o, ao, (uint64_t)p.C, p.capacity, 2ull * p.C, D, 128, D * 2))
    return SPA_ERR_UNSUPPORTED;
  auto kern = rel_bwd_short_kernel<D>;
  const int smem = Smem<D>::kBytes + 3 * rel.view.pitch * 4;
  static DeviceOnce attr;
  cudaError_t ea = attr.run([&] { return cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, kTwoPerSm); });
  if (ea != cudaSuccess) { set_cuda_error(ea, "rel_bwd_short_kernel"); return SPA_ERR_CUDA; }
  const int ctas = 2 * kNumSMs / p.H * p.H, chunk = chunk_of(n_seg, p.H, ctas);
  const long long items = (long long)((n_seg + chunk - 1) / chunk) * p.H;
  launch_pdl(kern, (int)(items < ctas ? items : ctas), kThreads, smem, st, tm_qkv, tm_do, tm_o, lse, delta, seg, n_seg, chunk,
             least, p.capacity, p.C, p.H, softmax_scale_of(p), (__nv_bfloat16*)dqkv, rel, d_status);
  SPA_CUDA_CHECK_LAUNCH("rel_bwd_short_kernel");
  return SPA_OK;
}

}  // namespace

// Backward, us, two passes -> one pass (and the two for longer segments): 512 windows of 7 x 7, 12 heads of 32, 228 -> 124, of two to a tile
// 91; of 64, 288 -> 163 -> 155; 128 images of 10 x 10, 12 heads of 64, 173 -> 92; of 14 x 14 with 5 to 60 % selected 105 -> 96.  The line counts rows of
// the capacity, since the host does not know the segments: where they are longer than 128 after all, images of 14 x 14 with 60 to 100 %
// selected, 280 -> 315, all 370 -> 382.
bool attention_rel_bwd_short_applies(const spa_params& p, int n_seg, const RelView& view) {
  const int base = p.C / p.H == 64 ? Smem<64>::kBytes : Smem<32>::kBytes;
  return n_seg >= 1 && (long long)p.capacity <= 256ll * n_seg && base + 3 * view.pitch * 4 <= kTwoPerSm;
}

int launch_attention_rel_bwd_short(const spa_params& p, const void* qkv, const void* ao, const float* lse, const void* dao,
                                   const int32_t* seg, int n_seg, const RelBwd& rel, void* dqkv, float* delta, int32_t* d_status,
                                   cudaStream_t st) {
  // Two to a tile where most segments are of at most 64 rows and the tables fit (124 -> 91 and 163 -> 155 above; one image per segment and
  // 64 rows or less on average would take in selections of which half are longer: 128 images of 14 x 14 110 -> 155).  A segment is of one
  // image, which may rule out longer ones.
  const bool d64 = p.C / p.H == 64;
  const bool pairs = (p.N <= kPairMax || (n_seg >= 2 * p.B && (long long)p.capacity <= (long long)kPairMax * n_seg)) &&
                     (d64 ? PairSmem<64>::kBytes <= PairSmem<64>::kMost - 3 * rel.view.pitch * 4
                          : PairSmem<32>::kBytes <= PairSmem<32>::kMost - 3 * rel.view.pitch * 4);
  if (pairs) {
    const int rc = d64 ? launch_pair<64>(p, qkv, ao, lse, dao, seg, n_seg, rel, dqkv, delta, d_status, st)
                       : launch_pair<32>(p, qkv, ao, lse, dao, seg, n_seg, rel, dqkv, delta, d_status, st);
    if (rc != SPA_OK || p.N <= kPairMax) return rc;
  }
  const int least = pairs ? kPairMax + 1 : 1;
  return d64 ? launch<64>(p, qkv, ao, lse, dao, seg, n_seg, rel, dqkv, delta, least, d_status, st)
             : launch<32>(p, qkv, ao, lse, dao, seg, n_seg, rel, dqkv, delta, least, d_status, st);
}

}  // namespace spa
