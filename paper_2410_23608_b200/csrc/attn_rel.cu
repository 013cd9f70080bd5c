// Attention with a learned bias by buckets of relative position, around the attention kernels: what comes before them (the table
// expanded to one value per offset, the tokens' positions, the bounds that the table's gradient is scaled by) and behind them
// (the gradient from its integer bins).  The backbone that the paper's blocks belong to (Sec. 3.1) has such a bias in every
// attention; with packed rows it goes by the tokens' places on the grid, which idx keeps.
#include <math_constants.h>

#include "attn_rel.cuh"
#include "spa_tc.cuh"

namespace spa {
namespace {

constexpr int kPrepThreads = 512;
constexpr float kLog2e = 1.4426950408889634f;  // the tensor-core kernels take exponentials in base 2

bool use_tc(const spa_params& p) { return !(p.flags & SPA_FLAG_SIMT_ONLY) && tc_attention_fwd_supported(p); }

struct Prep {
  const void* table;
  const int32_t *bucket, *idx, *seg;
  const void *qkv, *dao;  // backward only
  float* bias;
  int32_t *pos, *owner, *bad, *place;
  uint32_t* redo;
  unsigned* counters;
  unsigned long long *acc, *acc_off;
  float* bound;
  int n_seg, capacity, B, N, rows, cols, n_buckets, entries, pitch, C, H;
  float mul;
};

// kRelBlocks CTAs.  Forward and backward: bias[h][o] = table[bucket[o]][h] * mul, the rows' positions, the check of idx.  Backward:
// cleared bins, the last row of every token (two rows of one token show behind the attention), and per CTA and head the largest
// |v|^2 and |dO|^2 of its rows.
template <typename T, int D, bool kBwd>
__global__ void __launch_bounds__(kPrepThreads) rel_prep_kernel(const Prep a, int32_t* d_status) {
  pdl_entry();
  extern __shared__ uint32_t top[];  // [H][2]
  const int tid = blockIdx.x * kPrepThreads + threadIdx.x, all = gridDim.x * kPrepThreads;
  const T* table = static_cast<const T*>(a.table);
  if (kBwd)
    for (int i = threadIdx.x; i < 2 * a.H; i += kPrepThreads) top[i] = 0u;
  const int Np = packed_rows(a.seg, a.n_seg, a.capacity);
  if (kBwd && tid == 0) *a.redo = 0u;
  if (!kBwd)
    for (int h = tid; h < a.H; h += all) a.counters[h] = 0u;
  for (int o = tid; o < a.pitch; o += all) {
    const int b = o < a.entries ? a.bucket[o] : 0;
    const bool ok = (unsigned)b < (unsigned)a.n_buckets;
    if (!ok) record_status(d_status, SPA_ERR_INVALID_ARG);
    for (int h = 0; h < a.H; ++h)
      a.bias[(long long)h * a.pitch + o] = rel_entry(ok ? to_f32<T>(table[(long long)b * a.H + h]) : 0.f, a.mul);
  }
  for (int i = tid; i < a.capacity + 128; i += all) {
    int p = 0;
    if (i < Np) {
      const int t = ld_dep(a.idx + i), before = i > 0 ? ld_dep(a.idx + i - 1) : t;
      p = rel_position(t, before, i, a.N, a.cols, a.B * a.N, [&] { return ld_dep(a.seg + find_segment(a.seg, a.n_seg, i)); }, d_status);
      if (kBwd && (unsigned)t < (unsigned)(a.B * a.N)) a.owner[t] = i;
    }
    a.pos[i] = p;
  }
  if constexpr (kBwd) {
    for (int i = tid; i < a.n_buckets * a.H; i += all) a.acc[i] = 0ull;
    if (a.acc_off != nullptr)
      for (int i = tid; i < a.pitch * a.H; i += all) {
        a.acc_off[i] = 0ull;
        if (i < a.pitch) a.place[i] = i;
      }
    for (int i = tid; i < a.H; i += all) a.bad[i] = 0;
    __syncthreads();
    // A thread has one chunk of a row, the same one of every row it looks at, and neighbouring lanes the other chunks of its head:
    // whole lines per load, and a maximum per thread.  (A thread per row and head read its line in eight loads, which went to L2
    // eight times when the attention kernel's waiting CTAs had left the first-level cache 28 KB: 15 -> 113 us.)
    constexpr int E = Vec16<T>::kElems, kLanes = D / E, kRows = 4;
    const int Q = a.C / E, per = Q < kPrepThreads ? kPrepThreads / Q : 1;  // rows side by side
    for (int c0 = 0; c0 < Q; c0 += kPrepThreads) {
      const int c = c0 + (per > 1 ? threadIdx.x % Q : threadIdx.x), r = per > 1 ? threadIdx.x / Q : 0;
      const bool mine = c < Q && r < per;
      uint32_t most_v = 0u, most_d = 0u;
      for (int row0 = blockIdx.x * per + r; __any_sync(0xffffffffu, row0 < Np); row0 += kRows * gridDim.x * per) {
        uint4 v[kRows], d[kRows];
#pragma unroll
        for (int i = 0; i < kRows; ++i) {
          const long long row = row0 + i * (int)gridDim.x * per;
          v[i] = d[i] = make_uint4(0u, 0u, 0u, 0u);
          if (mine && row < Np) {
            v[i] = reinterpret_cast<const uint4*>(a.qkv)[(3 * row + 2) * Q + c];
            d[i] = reinterpret_cast<const uint4*>(a.dao)[row * Q + c];
          }
        }
#pragma unroll
        for (int i = 0; i < kRows; ++i) {
          float f[E], sv = 0.f, sd = 0.f;
          Vec16<T>::to_float(v[i], f);
#pragma unroll
          for (int e = 0; e < E; ++e) sv = fmaf(f[e], f[e], sv);
          Vec16<T>::to_float(d[i], f);
#pragma unroll
          for (int e = 0; e < E; ++e) sd = fmaf(f[e], f[e], sd);
#pragma unroll
          for (int o = kLanes / 2; o > 0; o >>= 1) {
            sv += __shfl_xor_sync(0xffffffffu, sv, o);
            sd += __shfl_xor_sync(0xffffffffu, sd, o);
          }
          most_v = max(most_v, __float_as_uint(sv) & 0x7fffffffu);
          most_d = max(most_d, __float_as_uint(sd) & 0x7fffffffu);
        }
      }
      if (mine && c % kLanes == 0) {
        atomicMax(top + 2 * (c / kLanes), most_v);
        atomicMax(top + 2 * (c / kLanes) + 1, most_d);
      }
    }
    __syncthreads();
    for (int i = threadIdx.x; i < 2 * a.H; i += kPrepThreads) a.bound[(long long)blockIdx.x * 2 * a.H + i] = __uint_as_float(top[i]);
  }
}

// A half of a row of dQ, or of dK and dV, from the rows of its own segment (see rel_redo), by a warp: the pairs to its lanes.
struct Redo {
  RelView view;
  const __nv_bfloat16 *qkv, *dao;
  const float *lse, *delta;
  __nv_bfloat16* dqkv;
  int C;
  float scale;
};
template <int D> __device__ void redo_row(const Redo& r, const int32_t* seg, int n_seg, int capacity, int Np, uint32_t what) {
  const int row = what & 0xfffff, h = (what >> 20) & 0xff, e0 = ((what >> 29) & 1) * (D / 2), lane = threadIdx.x & 31;
  const bool keys = (what >> 28) & 1;
  const long long ld = 3LL * r.C;
  const int col = h * D;
  const RowSeg s = row_segment(seg, n_seg, Np, row);
  const float *bias = r.view.bias + (long long)h * r.view.pitch + r.view.center, *lse = r.lse + (long long)h * capacity;
  const float* delta = r.delta + (long long)h * capacity;
  float acc1[D / 2] = {}, acc2[D / 2] = {};  // dQ | dK and dV
  for (int k = s.lo + lane; k < s.hi; k += 32) {
    const int q = keys ? k : row, j = keys ? row : k;
    const __nv_bfloat16 *Q = r.qkv + q * ld + col, *K = r.qkv + j * ld + r.C + col, *dO = r.dao + (long long)q * r.C + col;
    const float l = lse[q], dp = rel_dot<D>(dO, K + r.C);
    const float p = l == -CUDART_INF_F ? 0.f : exp2f(fmaf(rel_dot<D>(Q, K), r.scale * kLog2e, bias[r.view.pos[q] - r.view.pos[j]]) - l * kLog2e);
    rel_axpy<D / 2>(acc1, p * (dp - delta[q]), (keys ? Q : K) + e0);
    if (keys) rel_axpy<D / 2>(acc2, p, dO + e0);
  }
  __nv_bfloat16* to = r.dqkv + row * ld + col + e0;
  rel_store_sums<D / 2>(acc1, r.scale, to + (keys ? r.C : 0));
  if (keys) rel_store_sums<D / 2>(acc2, 1.f, to + 2 * r.C);
}

// Sums by offset to the buckets' (see rel_few_buckets).  Neighbouring offsets are mostly of one bucket: a warp adds such up first.
__global__ void __launch_bounds__(256) rel_fold_kernel(const unsigned long long* off, unsigned long long* acc, const int32_t* bucket, int entries,
                                                       int pitch, int n_buckets, int H) {
  pdl_entry();
  const int lane = threadIdx.x & 31, all = gridDim.x * 256;
  for (int i = blockIdx.x * 256 + threadIdx.x; i - lane < pitch * H; i += all) {  // whole warps
    const int h = i / pitch, at = i % pitch;
    const bool in = i < pitch * H && at < entries;
    const int b = in ? bucket[at] : -1, key = in && (unsigned)b < (unsigned)n_buckets ? h * n_buckets + b : -1;
    unsigned long long v = key >= 0 ? off[i] : 0ull;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {  // the first lane of 2 o takes what the first of their second half has
      const unsigned long long w = __shfl_xor_sync(0xffffffffu, v, o);
      if (__shfl_xor_sync(0xffffffffu, key, o) == key) {
        if ((lane & (2 * o - 1)) == 0) v += w;
        else if ((lane & (2 * o - 1)) == o) v = 0ull;
      }
    }
    if (v != 0ull) atomicAdd(acc + key, v);
  }
}

// dtable = acc / scale, NaN for a head with values that are not finite.  A token with two rows: an error in d_status.  D: behind
// the tensor-core kernels, heads of D, the rows that they noted down; 0: no such rows.
template <int D>
__global__ void __launch_bounds__(256) rel_finish_kernel(const RelGrad g, const unsigned long long* acc, int n_buckets, const Redo r, const int32_t* seg, int n_seg, int capacity,
                                                         const int32_t* idx, const int32_t* owner, int tokens,
                                                         float* __restrict__ dtable, int32_t* d_status) {
  pdl_entry();
  extern __shared__ float unit[];  // [H] value of a bin's least bit
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  for (int h = warp; h < g.H; h += 8) {
    const float b = rel_head_bound(g, h);
    const bool ok = b < __uint_as_float(0x7f800000u) && ld_dep(g.bad + h) == 0;
    if (lane == 0) unit[h] = ok ? rel_power(rel_exponent(b) - g.bits) : __uint_as_float(0x7fc00000u);
  }
  __syncthreads();
  const int tid = blockIdx.x * 256 + threadIdx.x, all = gridDim.x * 256;
  for (int i = tid; i < n_buckets * g.H; i += all) {
    const int h = i % g.H;
    dtable[i] = (float)((double)(long long)acc[(long long)h * n_buckets + i / g.H] * (double)unit[h]);
  }
  const int Np = packed_rows(seg, n_seg, capacity);
  for (int i = tid; i < Np; i += all) {
    const int t = ld_dep(idx + i);
    if ((unsigned)t < (unsigned)tokens && ld_dep(owner + t) != i) record_status(d_status, SPA_ERR_INVALID_ARG);
  }
  if constexpr (D != 0) {
    const uint32_t noted = (uint32_t)ld_dep(reinterpret_cast<const int32_t*>(g.redo)), n = noted < g.most_redo ? noted : g.most_redo;
    for (uint32_t i = blockIdx.x * 8 + warp; i < n; i += gridDim.x * 8) redo_row<D>(r, seg, n_seg, capacity, Np, g.redo[1 + i]);
  }
}

size_t aligned(size_t n) { return (n + 255) & ~(size_t)255; }

struct Layout {
  size_t pos, bias, acc, acc_off, place, bound, bad, owner, delta, redo, end;
  int entries, pitch, center;
  bool few;
};
Layout layout(const spa_params& p, const spa_rel_bias& r) {
  Layout l;
  const int W = 2 * r.cols - 1;
  l.entries = (2 * r.rows - 1) * W;
  l.pitch = (l.entries + 3) & ~3;
  l.center = (r.rows - 1) * W + r.cols - 1;
  size_t at = 0;
  auto take = [&](size_t bytes) { const size_t here = at; at += aligned(bytes); return here; };
  l.pos = take(((size_t)p.capacity + 128) * 4);
  l.bias = take((size_t)p.H * l.pitch * 4);
  l.acc = take((size_t)r.n_buckets * p.H * 8);
  l.few = rel_few_buckets(l.entries, r.n_buckets);
  l.acc_off = take(l.few ? (size_t)l.pitch * p.H * 8 : 0);
  l.place = take(l.few ? (size_t)l.pitch * 4 : 0);
  l.bound = take((size_t)kRelBlocks * p.H * 8);
  l.bad = take((size_t)p.H * 4);
  l.owner = take((size_t)p.B * p.N * 4);
  if (p.dtype == SPA_BF16) {  // whatever kernels take it
    l.delta = take((size_t)p.H * p.capacity * 4);
    l.redo = take(((size_t)4 * p.H * p.capacity + 1) * 4);
  } else {
    l.delta = l.redo = take(4);
  }
  l.end = at;
  return l;
}

int launch_prep(const spa_params& p, const spa_rel_bias& r, const Layout& l, char* ws, const int32_t* seg, int n_seg, const int32_t* idx,
                const void* qkv, const void* dao, float mul, int32_t* d_status, cudaStream_t st) {
  Prep a = {};
  a.table = r.table;
  a.bucket = r.bucket;
  a.idx = idx;
  a.seg = seg;
  a.qkv = qkv;
  a.dao = dao;
  a.bias = (float*)(ws + l.bias);
  a.pos = (int32_t*)(ws + l.pos);
  a.owner = (int32_t*)(ws + l.owner);
  a.bad = (int32_t*)(ws + l.bad);
  a.redo = (uint32_t*)(ws + l.redo);
  a.counters = (unsigned*)(ws + l.bad);  // forward and backward use one or the other
  a.acc = (unsigned long long*)(ws + l.acc);
  a.acc_off = l.few ? (unsigned long long*)(ws + l.acc_off) : nullptr;
  a.place = (int32_t*)(ws + l.place);
  a.bound = (float*)(ws + l.bound);
  a.n_seg = n_seg;
  a.capacity = p.capacity;
  a.B = p.B;
  a.N = p.N;
  a.rows = r.rows;
  a.cols = r.cols;
  a.n_buckets = r.n_buckets;
  a.entries = l.entries;
  a.pitch = l.pitch;
  a.C = p.C;
  a.H = p.H;
  a.mul = mul;
  const size_t smem = dao != nullptr ? (size_t)2 * p.H * sizeof(uint32_t) : 0;
#define SPA_PREP(T, D)                                                                                                       \
  do {                                                                                                                       \
    if (dao != nullptr) launch_pdl(rel_prep_kernel<T, D, true>, kRelBlocks, kPrepThreads, smem, st, a, d_status);            \
    else launch_pdl(rel_prep_kernel<T, D, false>, kRelBlocks, kPrepThreads, smem, st, a, d_status);                          \
  } while (0)
  const int d = p.C / p.H;
  if (p.dtype == SPA_F32) { if (d == 32) SPA_PREP(float, 32); else SPA_PREP(float, 64); }
  else if (d == 32) SPA_PREP(__nv_bfloat16, 32);
  else SPA_PREP(__nv_bfloat16, 64);
#undef SPA_PREP
  SPA_CUDA_CHECK_LAUNCH("rel_prep_kernel");
  return SPA_OK;
}

RelView view(const Layout& l, char* ws) {
  return RelView{(const int32_t*)(ws + l.pos), (const float*)(ws + l.bias), (unsigned*)(ws + l.bad), (uint32_t*)(ws + l.redo),
                 l.pitch, l.entries, l.center};
}

}  // namespace

size_t rel_workspace_bytes(const spa_params& p, const spa_rel_bias& r) { return layout(p, r).end; }

int launch_attention_rel_fwd(const spa_params& p, const spa_rel_bias& r, const void* qkv, const int32_t* seg, int n_seg,
                             const int32_t* idx, void* ao, float* lse, float* peak, void* workspace, int32_t* d_status, cudaStream_t st) {
  const Layout l = layout(p, r);
  char* ws = static_cast<char*>(workspace);
  const bool tc = use_tc(p);
  if (tc && attention_rel_fwd_prepares(p, l.pitch)) {
    const RelRaw raw{idx, r.bucket, r.table, r.cols, p.N, p.B * p.N, r.n_buckets};
    return launch_attention_rel_fwd_tc(p, qkv, seg, n_seg, view(l, ws), ao, lse, peak, &raw, d_status, st);
  }
  int rc = launch_prep(p, r, l, ws, seg, n_seg, idx, nullptr, nullptr, tc ? kLog2e : 1.f, d_status, st);
  if (rc != SPA_OK) return rc;
  if (tc) return launch_attention_rel_fwd_tc(p, qkv, seg, n_seg, view(l, ws), ao, lse, peak, nullptr, d_status, st);
  return launch_attention_rel_fwd_simt(p, qkv, seg, n_seg, view(l, ws), ao, lse, peak, st);
}

int launch_attention_rel_bwd(const spa_params& p, const spa_rel_bias& r, const void* qkv, const void* ao, const float* lse,
                             const float* peak, const void* dao, const int32_t* seg, int n_seg, const int32_t* idx, void* dqkv,
                             float* dtable, void* workspace, int32_t* d_status, cudaStream_t st) {
  const Layout l = layout(p, r);
  char* ws = static_cast<char*>(workspace);
  const bool tc = use_tc(p);
  int rc = launch_prep(p, r, l, ws, seg, n_seg, idx, qkv, dao, tc ? kLog2e : 1.f, d_status, st);
  if (rc != SPA_OK) return rc;
  RelGrad g = {};
  unsigned long long* acc = (unsigned long long*)(ws + l.acc);
  g.acc = l.few ? (unsigned long long*)(ws + l.acc_off) : acc;
  g.place = l.few ? (const int32_t*)(ws + l.place) : r.bucket;
  g.places = l.few ? l.pitch : r.n_buckets;
  g.bound = (const float*)(ws + l.bound);
  g.peak = peak;
  g.bad = (int32_t*)(ws + l.bad);
  g.redo = (uint32_t*)(ws + l.redo);
  g.H = p.H;
  g.bits = rel_bits(p.capacity);
  g.most_redo = 4u * p.H * p.capacity;
  rc = tc ? launch_attention_rel_bwd_tc(p, qkv, ao, lse, dao, seg, n_seg, view(l, ws), g, dqkv, (float*)(ws + l.delta), d_status, st)
          : launch_attention_rel_bwd_simt(p, qkv, ao, lse, dao, seg, n_seg, view(l, ws), g, dqkv, st);
  if (rc != SPA_OK) return rc;
  if (l.few) {
    const int ctas = (l.pitch * p.H + 255) / 256;
    launch_pdl(rel_fold_kernel, ctas < 4 * kNumSMs ? ctas : 4 * kNumSMs, 256, 0, st, g.acc, acc, r.bucket, l.entries, l.pitch, r.n_buckets, p.H);
    SPA_CUDA_CHECK_LAUNCH("rel_fold_kernel");
  }
  const long long work = (long long)r.n_buckets * p.H > p.capacity ? (long long)r.n_buckets * p.H : p.capacity;
  // behind the tensor-core kernels a CTA per SM, should there be rows to form again
  const int grid = (int)(!tc && (work + 1023) / 1024 < kNumSMs ? (work + 1023) / 1024 : kNumSMs);
  const Redo redo{view(l, ws), (const __nv_bfloat16*)qkv, (const __nv_bfloat16*)dao, lse, (const float*)(ws + l.delta), (__nv_bfloat16*)dqkv,
                  p.C, softmax_scale_of(p)};
  launch_pdl(!tc ? rel_finish_kernel<0> : p.C / p.H == 64 ? rel_finish_kernel<64> : rel_finish_kernel<32>, grid, 256, (size_t)p.H * sizeof(float), st, g, acc, r.n_buckets, redo, seg, n_seg, p.capacity,
             idx, (const int32_t*)(ws + l.owner), p.B * p.N, dtable, d_status);
  SPA_CUDA_CHECK_LAUNCH("rel_finish_kernel");
  return SPA_OK;
}

}  // namespace spa
