// Attention with a learned bias by relative position: what its kernels share.
//
// A token at row y and column x of a rows x cols grid has the position p = y W + x, W = 2 cols - 1, so that the offset between
// two tokens is one subtraction: off = p_i - p_j + (rows - 1) W + cols - 1, a number below (2 rows - 1) W.  The table of buckets
// is expanded to one value per head and offset before the attention kernel runs; any two positions give an offset inside it,
// also those of tokens of different images, so no look-up needs a check.
//
// The table's gradient adds dS_ij to the bin of off(i, j).  Bins are integers: dS times a power of two, so that the order in
// which the CTAs' atomics arrive changes nothing.  The power comes from a bound on |dS| that is known beforehand:
//   |dS_ij| = P_ij |dO_i . v_j - D_i| <= 2 P_ij |dO_i| max_j |v_j|     (O_i is a mean of the v_j)
#pragma once

#include "simt_stage.cuh"
#include "sm100_ptx.cuh"
#include "spa_common.cuh"

namespace spa {

struct RelView {          // what the forward and backward kernels read
  const int32_t* pos;     // [capacity + 128]
  const float* bias;      // [H][pitch]: the table's value of every offset
  unsigned* counters;     // [H] forward: row tiles of a head that have been drawn
  uint32_t* redo;         // forward: [1 + 4 H capacity], see rel_fwd_note
  int pitch, entries, center;
};

// What the preparation works from, for a forward kernel that does it itself
struct RelRaw {
  const int32_t *idx, *bucket;
  const void* table;
  int cols, N, tokens, n_buckets;
};
// Entries below this mask: beside any other they have no weight, and where a row has nothing else, its logarithm of the sum would have no bits
// left for S (a type's lowest value times log2 e is not even finite).  Such rows are rows without a key.
constexpr float kRelMasked = -1e6f;
__device__ __forceinline__ float rel_entry(float v, float mul) { return (v < kRelMasked ? __uint_as_float(0xff800000u) : v) * mul; }
// Position of packed row i (< the packed rows) whose token is t; before: the token of the row before it (or t), start: its segment's first
// row.  An error in d_status for a token out of range, or a segment with tokens of two images.
template <typename Start>
__device__ __forceinline__ int rel_position(int t, int before, int i, int N, int cols, int tokens, Start start, int32_t* d_status) {
  if ((unsigned)t >= (unsigned)tokens) {
    record_status(d_status, SPA_ERR_INVALID_ARG);
    return 0;
  }
  const int n = t % N;
  if (t / N != before / N && start() != i) record_status(d_status, SPA_ERR_INVALID_ARG);
  return n / cols * (2 * cols - 1) + n % cols;
}

// kN values from a 16-byte boundary on, all of them NaN.  A row that its own values have made NaN has nothing to be formed again: a call whose
// inputs are NaN everywhere (after a step that diverged) formed every row so, 18 images of 24 x 24 with 77 to 576 rows, 4 heads of 64, 0.09 -> 557 ms.
template <int kN> __device__ __forceinline__ bool rel_all_nan(const __nv_bfloat16* v) {
  const uint32_t* w = reinterpret_cast<const uint32_t*>(v);  // a bf16 is NaN where its bits without the sign are above those of infinity
#pragma unroll 1
  for (int i = 0; i < kN / 2; ++i)
    if ((w[i] & 0x7fffu) <= 0x7f80u || (w[i] >> 16 & 0x7fffu) <= 0x7f80u) return false;
  return true;
}
// sum of a_e b_e over D values each from a 16-byte boundary on (a loop: what is formed again leaves the registers to the kernel around it)
template <int D> __device__ __forceinline__ float rel_dot(const __nv_bfloat16* a, const __nv_bfloat16* b) {
  float sum = 0.f;
#pragma unroll 1
  for (int c = 0; c < D / 8; ++c) {
    float f[8], g[8];
    Vec16<__nv_bfloat16>::to_float(reinterpret_cast<const uint4*>(a)[c], f);
    Vec16<__nv_bfloat16>::to_float(reinterpret_cast<const uint4*>(b)[c], g);
#pragma unroll
    for (int e = 0; e < 8; ++e) sum = fmaf(f[e], g[e], sum);
  }
  return sum;
}
// acc_e += w v_e
template <int kN> __device__ __forceinline__ void rel_axpy(float (&acc)[kN], float w, const __nv_bfloat16* v) {
#pragma unroll
  for (int c = 0; c < kN / 8; ++c) {
    float f[8];
    Vec16<__nv_bfloat16>::to_float(reinterpret_cast<const uint4*>(v)[c], f);
#pragma unroll
    for (int e = 0; e < 8; ++e) acc[8 * c + e] = fmaf(w, f[e], acc[8 * c + e]);
  }
}
// The lanes' sums, times mul, as kN values from a 16-byte boundary on
template <int kN> __device__ __forceinline__ void rel_store_sums(float (&acc)[kN], float mul, __nv_bfloat16* to) {
#pragma unroll
  for (int e = 0; e < kN; ++e) acc[e] = warp_sum(acc[e]) * mul;
  if ((threadIdx.x & 31) == 0)
#pragma unroll
    for (int c = 0; c < kN / 8; ++c) reinterpret_cast<uint4*>(to)[c] = Vec16<__nv_bfloat16>::from_float(acc + 8 * c);
}

// A half of a row of the forward's output that is not finite: {row, head, half}, and the CTA's entry before it (numbers from 1 on; 0:
// none), of which `last` in shared memory is the last.  The CTA that notes it down forms it again.
// v: the row's own half of V.  A call, not in line: with the loads in the kernel around it 8 frames of 47 x 83 took 88 us instead of 83.
template <int D>
__device__ __noinline__ void rel_fwd_note(uint32_t* redo, uint32_t* last, int capacity, int row, int h, int half, const __nv_bfloat16* v) {
  if (rel_all_nan<D / 2>(v)) return;
  const uint32_t at = 2u * ((uint32_t)h * capacity + row) + half + 1u;
  redo[2 * at - 1] = (uint32_t)row | (uint32_t)h << 20 | (uint32_t)half << 28;
  redo[2 * at] = atomicExch(last, at);
}

constexpr int kRelBlocks = kNumSMs;  // CTAs of the kernel that prepares a call, each with its own maxima
struct RelGrad {
  // [H][places] sums of dS times 2^(bits - exponent of the head's bound): a place for each bucket, or, where they are few
  // (rel_few_buckets), one for each offset, and rel_fold_kernel behind the attention
  unsigned long long* acc;
  const int32_t* place;  // [entries]: the buckets, or the offsets themselves (a NULL for these, and a branch, made the dQ pass 3 % slower)
  const float* bound;       // [kRelBlocks][H][2] largest |v_j|^2 and |dO_i|^2
  const float* peak;        // [H][capacity] log of the row's largest probability, optional
  int32_t* bad;             // [H] a row's statistics are not finite
  uint32_t* redo;           // [1 + 4 H capacity] how many, and which parts of rows are to be formed again
  int places, H;
  int bits;                 // see rel_bits
  uint32_t most_redo;       // 4 H capacity
};

// A zero weight times an infinity or NaN of another segment in the same tile is NaN.  Halves of rows of dQ (keys = false), or of dK and dV, that
// are not finite are noted down, and formed again behind the attention from their own segment's rows alone.
__device__ __forceinline__ void rel_redo(const RelGrad& g, bool keys, int half, int h, int row) {
  const uint32_t at = atomicAdd(g.redo, 1u);
  if (at < g.most_redo) g.redo[1 + at] = (uint32_t)row | (uint32_t)h << 20 | (keys ? 1u : 0u) << 28 | (uint32_t)half << 29;
}
// The same where segments may be long, but for what its own values have made NaN: dQ by its row's logarithm of the sum (lse) or D (delta), of which one
// makes every dS of the row NaN; dK and dV by those of the token's own row among the queries: lse makes P and dS NaN, D dS, so dK, and where
// its half of a row of dO (own_do) is NaN, dV is.  bad: kBadQ, kBadK, kBadV.  A call, not in line, as rel_fwd_note is.  (Segments of up to 128
// rows are formed again in no time: 64 of 7 x 7, 6 heads of 64, NaN everywhere, the backward takes as long as with numbers.)
constexpr uint32_t kBadQ = 1, kBadK = 2, kBadV = 4;
template <int D>
__device__ __noinline__ void rel_note(uint32_t* redo, uint32_t most, uint32_t row, uint32_t h, uint32_t half, uint32_t bad, float lse, float delta,
                                      const __nv_bfloat16* own_do) {
  if (lse != lse) return;
  if (delta != delta) bad &= kBadV;
  auto note = [&](uint32_t keys) {
    const uint32_t at = atomicAdd(redo, 1u);
    if (at < most) redo[1 + at] = row | h << 20 | keys << 28 | half << 29;
  };
  if (bad & kBadQ) note(0u);
  if ((bad & kBadK) || ((bad & kBadV) && !rel_all_nan<D / 2>(own_do))) note(1u);
}
template <int D>
__device__ __forceinline__ void rel_redo_long(const RelGrad& g, uint32_t bad, int half, int h, int row, float lse, float delta,
                                              const __nv_bfloat16* dao, int C) {
  rel_note<D>(g.redo, g.most_redo, (uint32_t)row, (uint32_t)h, (uint32_t)half, bad, lse, delta, dao + (long long)row * C + h * D + half * (D / 2));
}

// Bits of the head's bound in the sums: as many as 64 hold.  The pairs of a query in a bin have dS of no more than the bound together (their P sum
// to one), the bound is taken up to a power of two, and D from a rounded O makes it 2^-8 more: capacity 2^bits < 2^62 1.01.  (A unit of 2^46 is what a
// float's exponent holds beside the least bound.)
constexpr int kRelMostBits = 46;
inline int rel_bits(int capacity) {
  int log2_rows = 0;
  while ((1 << log2_rows) < capacity) ++log2_rows;
  return 62 - log2_rows < kRelMostBits ? 62 - log2_rows : kRelMostBits;
}

// Exponent e of a bound b < 2^e; zero and values too small for the scale's exponent count as the smallest.
__device__ __forceinline__ int rel_exponent(float b) {
  const int e = (int)((__float_as_uint(b) >> 23) & 0xffu) - 126;
  return e < -80 ? -80 : e;
}
__device__ __forceinline__ float rel_power(int n) { return __uint_as_float((uint32_t)(127 + n) << 23); }

// 2 max |dO| max |v| of a head, and max |v|, by a converged warp.  Maxima of bit patterns: a NaN is larger than every number.  Squares that
// underflow count as the smallest normal number: a bound may be too large, not too small.
constexpr uint32_t kLeastSquare = 0x00800000u;
__device__ __forceinline__ float rel_head_bound(const RelGrad& g, int h, float& most_v) {
  const int lane = threadIdx.x & 31;
  uint32_t v = kLeastSquare, d = kLeastSquare;
#pragma unroll
  for (int i = 0; i < (kRelBlocks + 31) / 32; ++i) {
    if (lane + 32 * i < kRelBlocks) {
      const float2 b = *reinterpret_cast<const float2*>(g.bound + ((long long)(lane + 32 * i) * g.H + h) * 2);
      v = max(v, __float_as_uint(b.x));
      d = max(d, __float_as_uint(b.y));
    }
  }
  v = __reduce_max_sync(0xffffffffu, v);
  d = __reduce_max_sync(0xffffffffu, d);
  most_v = sqrtf(__uint_as_float(v));
  return 2.f * most_v * sqrtf(__uint_as_float(d));
}
__device__ __forceinline__ float rel_head_bound(const RelGrad& g, int h) {
  float most_v;
  return rel_head_bound(g, h, most_v);
}
// The same of a row, from |dO|^2 and the logarithm of its largest probability, as a bit pattern
__device__ __forceinline__ uint32_t rel_row_bound(float most_v, float square, float peak) {
  const float d = square < __uint_as_float(kLeastSquare) ? __uint_as_float(kLeastSquare) : square;  // a NaN stays one
  return __float_as_uint(2.f * most_v * sqrtf(d) * ptx::ex2_approx(peak * 1.4426950408889634f)) & 0x7fffffffu;
}

// A row whose logarithm of the sum (NaN, +inf) or D is not finite has dS that are not
__device__ __forceinline__ void rel_check_row(const RelGrad& g, int h, float lse, float D) {
  if (!(lse < __uint_as_float(0x7f800000u)) || !(fabsf(D) < __uint_as_float(0x7f800000u))) g.bad[h] = 1;
}

// v to the place of table entry `at`
__device__ __forceinline__ void rel_add(const RelGrad& g, int h, int at, long long v) {
  const int b = g.place[at];
  if ((unsigned)b < (unsigned)g.places && v != 0) atomicAdd(g.acc + (long long)h * g.places + b, (unsigned long long)v);
}
// Few buckets for many offsets: atomics of all CTAs would queue for the few sums.  us, places by bucket -> by offset, with 25 buckets: 128
// images of 14 x 14 with 30 to 60 % selected, 12 heads of 64, 146 -> 114, 512 windows of 7 x 7 (6.8 offsets to a bucket), 12 heads of 32, 102 -> 94, fp32 64
// images of 14 x 14, 6 heads of 64, 1178 -> 313.  Folding costs 1 to 2 us: with 225 buckets the first takes 111 either way.
inline bool rel_few_buckets(int entries, int n_buckets) { return entries >= 4 * (long long)n_buckets; }

// What the kernels with a bias by relative position are given beside the others' arguments.  shared_bins: the table's gradient is
// summed in shared memory, item by item; else pair by pair in global memory.
struct RelBwd {
  RelView view;
  RelGrad grad;
  bool shared_bins;
};
// An item's pairs are multiples of 2^-43 of the item's bound: 21 bits in front of a point, to which a pair is rounded by the addition of a number
// whose unit that is, and the rest, which the next fma has exactly (|rest| <= 1/2), to 2^-22 by the addition of 3.  As pairs of fp32, without a
// conversion.  The two parts go to two words of a bin, which has at most one pair of each of the item's 128 query rows, since a token is in its
// segment once: 2^21 (1.01 of it, see rel_bits) and 2^21 times 2^7 overflow neither.  (30 bits of a pair, by a conversion and ten bits of the
// integer to one word: one row of V 1 000 times as large as the others, in another image, took the gradient's error from below 2e-7 to up to
// 5e-4, since the bound that all rows of a head share was 1 000 times what they needed.  32 images of 24 x 24, 12 heads of 64, backward
// 192 -> 190 us, with the pairs' way to their bins moved behind the announcement of dS.  One word of 23 bits: an error of 3.6e-5 without any such row.)
constexpr int kRelHigh = 21, kRelLow = 22, kRelItemBits = kRelHigh + kRelLow;
constexpr uint32_t kRelUnits = 0x4b400000u;  // 1.5 * 2^23: adding it rounds |x| < 2^22 to an integer, in the low bits
constexpr uint32_t kRelRest = 0x40400000u;   // 3, to whose side |x| <= 1/2 is rounded to 2^-22
__device__ __forceinline__ float rel_item_scale(int bound_exp) { return rel_power(kRelHigh - bound_exp); }
// Units of an item's scale to those of the head's: a shift to the left
__device__ __forceinline__ int rel_item_shift(const RelGrad& g, int bound_exp, int head_exp) { return g.bits - head_exp - (kRelItemBits - bound_exp); }
__device__ __forceinline__ void rel_fixed(uint64_t d, float scale, uint32_t* hi, uint32_t* lo) {  // of two pairs
  const uint64_t s = ptx::pair(scale, scale), t = ptx::fma2(d, s, ptx::pair(kRelUnits, kRelUnits));
  const uint64_t u = ptx::fma2(d, s, ptx::fma2(t, ptx::pair(-1.f, -1.f), ptx::pair(kRelUnits + 3, kRelUnits + 3)));  // 3 - hi, exact
  ptx::unpair(t, hi[0], hi[1]);
  ptx::unpair(u, lo[0], lo[1]);
#pragma unroll
  for (int i = 0; i < 2; ++i) { hi[i] -= kRelUnits; lo[i] -= kRelRest; }
}
__device__ __forceinline__ void rel_bin(uint32_t at, uint32_t pitch_bytes, uint32_t hi, uint32_t lo) {
  ptx::red_add_s32(at, (int)lo);
  ptx::red_add_s32(at + pitch_bytes, (int)hi);
}
__device__ __forceinline__ long long rel_joined(int hi, int lo) { return ((long long)hi << kRelLow) + lo; }
// The fp32-FMA kernels: up to 46 bits of a pair in three words, 16 bits to each of the lower two; 32 query rows
constexpr int kRelThird = 16;
__device__ __forceinline__ void rel_bin3(int* bin, int pitch, long long v) {
  atomicAdd(bin, (int)v & ((1 << kRelThird) - 1));
  atomicAdd(bin + pitch, (int)(v >> kRelThird) & ((1 << kRelThird) - 1));
  atomicAdd(bin + 2 * pitch, (int)(v >> 2 * kRelThird));
}
template <int kThreads> __device__ __forceinline__ void rel_flush3(const RelGrad& g, const int* bins, int entries, int pitch, int h, int tid) {
  for (int i = tid; i < entries; i += kThreads)
    rel_add(g, h, i, ((long long)bins[2 * pitch + i] << 2 * kRelThird) + ((long long)bins[pitch + i] << kRelThird) + bins[i]);
}
// A sum in units of an item's scale as one in units of the head's, to nearest (|v| <= 2^52)
__device__ __forceinline__ long long rel_shifted(long long v, int shift) {
  if (shift >= 0) return v << shift;
  const int n = shift > -60 ? -shift : 60;
  return (v + (1ll << (n - 1))) >> n;
}

// Positions of a tile's columns from shared memory, four at a time, and where registers allow (kAhead) a step before they are used: the
// forward of 8 frames of 47 x 83 87 -> 82 us; the dQ pass spills with it.
template <bool kAhead = true> struct RelKeys {
  uint32_t at;
  int ahead[4];
  __device__ __forceinline__ explicit RelKeys(uint32_t addr) : at(addr) {
    if (kAhead) ptx::lds_4s32(at, ahead);
  }
  __device__ __forceinline__ void next(int j, int n, int (&k)[4]) {  // columns j .. j + 3 of n
    if (!kAhead) {
      ptx::lds_4s32(at + 4 * j, k);
      return;
    }
#pragma unroll
    for (int u = 0; u < 4; ++u) k[u] = ahead[u];
    if (j + 4 < n) ptx::lds_4s32(at + 4 * (j + 4), ahead);
  }
};

// The bins of an item to the head's sums, by kThreads threads: four at a time, so that the look-ups of their buckets do not wait for
// one another
template <int kThreads>
__device__ __forceinline__ void rel_flush(const RelBwd& rel, const int* bins, int h, int shift, int tid) {
  for (int i = tid; i < rel.view.entries; i += 4 * kThreads) {
    long long v[4];
    int b[4];
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      const int at = i + u * kThreads;
      v[u] = at < rel.view.entries ? rel_joined(bins[rel.view.pitch + at], bins[at]) : 0;
      b[u] = v[u] != 0 ? rel.grad.place[at] : -1;
    }
#pragma unroll
    for (int u = 0; u < 4; ++u)
      if ((unsigned)b[u] < (unsigned)rel.grad.places)
        atomicAdd(rel.grad.acc + (long long)h * rel.grad.places + b[u], (unsigned long long)rel_shifted(v[u], shift));
  }
}

constexpr int kTwoPerSm = (228 * 1024 - 2 * 1024) / 2 / 16 * 16;  // shared memory of a CTA of which an SM holds two

// The backward of segments of at most 128 rows in one pass (attn_rel_short.cu), where most are so short and the tables fit
bool attention_rel_bwd_short_applies(const spa_params& p, int n_seg, const RelView& view);
int launch_attention_rel_bwd_short(const spa_params& p, const void* qkv, const void* ao, const float* lse, const void* dao,
                                   const int32_t* seg, int n_seg, const RelBwd& rel, void* dqkv, float* delta, int32_t* d_status,
                                   cudaStream_t st);
int launch_attention_rel_fwd_tc(const spa_params& p, const void* qkv, const int32_t* seg, int n_seg, const RelView& rel, void* ao,
                                float* lse, float* peak, const RelRaw* raw, int32_t* d_status, cudaStream_t st);
bool attention_rel_fwd_prepares(const spa_params& p, int pitch);  // launch_attention_rel_fwd_tc with raw, and no preparation before it
int launch_attention_rel_bwd_tc(const spa_params& p, const void* qkv, const void* ao, const float* lse, const void* dao,
                                const int32_t* seg, int n_seg, const RelView& view, const RelGrad& grad, void* dqkv, float* delta,
                                int32_t* d_status, cudaStream_t st);
int launch_attention_rel_fwd_simt(const spa_params& p, const void* qkv, const int32_t* seg, int n_seg, const RelView& rel, void* ao,
                                  float* lse, float* peak, cudaStream_t st);
int launch_attention_rel_bwd_simt(const spa_params& p, const void* qkv, const void* ao, const float* lse, const void* dao,
                                  const int32_t* seg, int n_seg, const RelView& rel, const RelGrad& grad, void* dqkv, cudaStream_t st);

}  // namespace spa
