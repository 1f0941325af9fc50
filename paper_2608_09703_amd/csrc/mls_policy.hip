// Clipped policy loss with a KL term on token log-probabilities, and its gradient.
// Per counted token t with advantage A and ratio r = exp(logp - old):
//   L = -min(r A, clip(r, 1 - lo, 1 + hi) A) + beta k,
//   k = exp(ref - logp) - (ref - logp) - 1        (an estimate of KL(policy || reference), >= 0)
//   dL/dlogp = -r A  where r A <= clip(r) A, else 0,  plus beta (1 - exp(ref - logp)).
// loss = sum_t w_t L_t with w = 1 / N over the N counted tokens, or with
// w = 1 / (S n_s) over the S sequences that have a counted token, n_s of them in
// sequence s.
//
// 13 to 17 bytes read and 4 written per token, and launches for few of them.
// Everything is computed in 64 bits from the fp32 inputs, so that whether a ratio is
// clipped does not depend on a rounding. Forward kernel, us for 2^20 tokens: 6.9, with
// a reference (its bytes and exponential) 8.3, with a mask 7.4, with 1,024 sequences
// (search, advantage and count by sequence) 9.1, with all of these 14.4: what takes
// the time there is the loads that wait for one another (search, count, mask), not the
// exponentials. The gradient is written by the forward, without the 1 / N or 1 / S
// that is known only once every token has been counted, but with a power of two near
// it (of all tokens or sequences), so that what fp32 holds of the mean it holds in
// between; the backward multiplies the rest and the upstream gradient in. Sums leave
// the blocks as 64-bit parts that one block adds in block order: results are bitwise
// reproducible.
#include <math.h>

#include <algorithm>

#include "mls_device.h"
#include "mls_launch.h"
#include "mls_wave.h"

namespace mls {

namespace {

constexpr int kPolThreads = 256;
constexpr int kPolTok = 4;                        // tokens per thread
constexpr int kPolTile = kPolThreads * kPolTok;   // tokens per block
constexpr int kPolSums = 4;                       // loss, KL, clipped, counted (tokens or sequences)
constexpr int kPolFinThreads = 1024;
constexpr int kPolOneBlock = 1024 * kPolTok;
constexpr int64_t kPolCountBlocks = 1 << 20;

// Start of sequence s inside [0, N]: offsets out of range are clamped, so that a
// bad one reads no memory outside the arrays.
__device__ __forceinline__ int64_t seq_begin(const PolicyArgs& a, int64_t s) {
  const int64_t c = a.cu[s];
  return c < 0 ? 0 : c > a.N ? a.N : c;
}

// Sequence of token t: the last one that begins at or before t (t lies inside
// [begin of the first, end of the last)).
__device__ __forceinline__ int64_t seq_of(const PolicyArgs& a, int64_t t) {
  int64_t lo = 0, hi = a.S;  // begin(lo) <= t < begin(hi)
  while (hi - lo > 1) {
    const int64_t m = (lo + hi) >> 1;
    if (a.cu[m] <= t)
      lo = m;
    else
      hi = m;
  }
  return lo;
}

// Counted tokens of every sequence under a mask, one block a sequence (and, past
// kPolCountBlocks of them, one more after it: a launch has at most 2^32 threads): 16
// mask bytes a thread and step, four steps in flight. NT threads: 1,024 for sequences of 64k
// tokens and more on average (2 of 500,000: 435 us byte by byte with 256 threads, 17
// with these), else 256, of which a short one needs few.
typedef unsigned int u32x4_byte_t __attribute__((ext_vector_type(4), aligned(1)));
__device__ __forceinline__ int nonzero_bytes(uint32_t w) {
  // bit 7 of each byte: the byte is not 0 (no carry leaves a byte)
  return __popc((((w & 0x7f7f7f7fu) + 0x7f7f7f7fu) | w) & 0x80808080u);
}
template <int NT>
__global__ __launch_bounds__(NT) void policy_count_kernel(PolicyArgs a) {
  __shared__ int part[NT / 64];
  for (int64_t s = blockIdx.x;;) {
    const int64_t b = seq_begin(a, s), e = seq_begin(a, s + 1);
    int n = 0;
#pragma unroll 4
    for (int64_t t = b + (int64_t)threadIdx.x * 16; t < e; t += NT * 16) {
      if (t + 16 <= e) {
        const u32x4_byte_t m = *reinterpret_cast<const u32x4_byte_t*>(a.mask + t);
        n += nonzero_bytes(m.x) + nonzero_bytes(m.y) + nonzero_bytes(m.z) + nonzero_bytes(m.w);
      } else {
        for (int64_t k = t; k < e; ++k) n += a.mask[k] ? 1 : 0;
      }
    }
    n = wave_sum(n);
    if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = n;
    __syncthreads();
    if (threadIdx.x == 0) {
      n = 0;
      for (int k = 0; k < NT / 64; ++k) n += part[k];
      a.counts[s] = n;
    }
    s += gridDim.x;
    if (s >= a.S) break;
    __syncthreads();  // part is written again
  }
}

__device__ __forceinline__ int64_t seq_count(const PolicyArgs& a, int64_t s) {
  if (a.mask) return a.counts[s];
  const int64_t n = seq_begin(a, s + 1) - seq_begin(a, s);
  return n > 0 ? n : 0;
}

// The loss and its companions from the sums over all tokens; thread 0 of a block.
__device__ __forceinline__ void write_losses(const PolicyArgs& a, const double* s) {
  const double inv = s[3] > 0.0 ? 1.0 / s[3] : 0.0;
  *a.loss = (float)(s[0] * inv);
  if (a.kl) *a.kl = (float)(s[1] * inv);
  if (a.clipped) *a.clipped = (float)(s[2] * inv);
  if (a.grad) a.grad[a.N] = (float)(inv / a.grad_scale);
}

// Sum over the block of each of kPolSums values; valid in thread 0. red: one row per wave.
template <int NT>
__device__ __forceinline__ void block_totals(double* v, double (*red)[kPolSums]) {
#pragma unroll
  for (int q = 0; q < kPolSums; ++q) v[q] = wave_sum(v[q]);
  if ((threadIdx.x & 63) == 0)
#pragma unroll
    for (int q = 0; q < kPolSums; ++q) red[threadIdx.x >> 6][q] = v[q];
  __syncthreads();
  if (threadIdx.x != 0) return;
#pragma unroll
  for (int q = 0; q < kPolSums; ++q) {
    v[q] = 0.0;
    for (int w = 0; w < NT / 64; ++w) v[q] += red[w][q];
  }
}

// Number of sequences with a counted token, this thread's share.
template <int NT>
__device__ __forceinline__ double live_sequences(const PolicyArgs& a) {
  double n = 0.0;
  for (int64_t s = threadIdx.x; s < a.S; s += NT) n += seq_count(a, s) > 0 ? 1.0 : 0.0;
  return n;
}

// Four consecutive values from t on, those below N.
typedef float f32x4_any_t __attribute__((ext_vector_type(4), aligned(4)));
__device__ __forceinline__ void load_four(const float* p, int64_t t, int64_t N, float* v) {
  if (t + kPolTok <= N) {
    const f32x4_any_t x = *reinterpret_cast<const f32x4_any_t*>(p + t);
    v[0] = x.x;
    v[1] = x.y;
    v[2] = x.z;
    v[3] = x.w;
  } else {
#pragma unroll
    for (int i = 0; i < kPolTok; ++i) v[i] = t + i < N ? p[t + i] : 0.f;
  }
}
__device__ __forceinline__ void store_four(float* p, int64_t t, int64_t N, const float* v) {
  if (t + kPolTok <= N) {
    *reinterpret_cast<f32x4_any_t*>(p + t) = f32x4_any_t{v[0], v[1], v[2], v[3]};
  } else {
#pragma unroll
    for (int i = 0; i < kPolTok; ++i)
      if (t + i < N) p[t + i] = v[i];
  }
}

// NT threads a block. Up to kPolOneBlock tokens one block of 1,024 takes all of them
// and writes the losses itself: a launch less where launches are what counts (8
// sequences of 200 tokens: 6.4 + 6.8 us in two launches, 7.6 in one).
template <int NT>
__global__ __launch_bounds__(NT) void policy_fwd_kernel(PolicyArgs a) {
  __shared__ double red[NT / 64][kPolSums];
  double sum[kPolSums] = {0.0, 0.0, 0.0, 0.0};
  // tokens that belong to a sequence
  const int64_t begin = a.cu ? seq_begin(a, 0) : 0, end = a.cu ? seq_begin(a, a.S) : a.N;
  const int64_t t0 = (int64_t)blockIdx.x * NT * kPolTok + threadIdx.x * kPolTok;
  float lpv[kPolTok], oldv[kPolTok], refv[kPolTok], advv[kPolTok], g[kPolTok];
  bool on[kPolTok];
  load_four(a.logp, t0, a.N, lpv);
  load_four(a.old_logp, t0, a.N, oldv);
  if (a.ref) load_four(a.ref, t0, a.N, refv);
  if (!a.per_seq) load_four(a.adv, t0, a.N, advv);
#pragma unroll
  for (int i = 0; i < kPolTok; ++i) {
    const int64_t t = t0 + i;
    on[i] = t >= begin && t < end && (!a.mask || a.mask[t]);
  }
  int64_t s = -1, s_end = 0;
  double seq_w = 1.0, seq_a = 0.0;
#pragma unroll
  for (int i = 0; i < kPolTok; ++i) {
    const int64_t t = t0 + i;
    g[i] = 0.f;
    if (!on[i]) continue;
    if ((a.per_seq || a.by_seq) && (s < 0 || t >= s_end)) {
      s = seq_of(a, t);
      s_end = a.cu[s + 1];
      if (a.per_seq) seq_a = a.adv[s];
      if (a.by_seq) seq_w = 1.0 / (double)seq_count(a, s);
    }
    const double lp = lpv[i];
    const double adv = a.per_seq ? seq_a : (double)advv[i];
    const double r = exp(lp - (double)oldv[i]);
    const double free = r * adv, bound = fmin(fmax(r, a.lo), a.hi) * adv;
    const bool take = !(free > bound);
    double l = take ? -free : -bound, dl = take ? -free : 0.0, k = 0.0;
    if (a.ref) {
      // next to the reference k is x^2 / 2, of which the difference loses digits (all of
      // them for x of a few fp32 steps): the series there, off by 2^-48, where the
      // difference at its border is off by 2^-32 (expm1 throughout: 1 us of 15 more)
      const double x = (double)refv[i] - lp, ex = exp(x);
      k = ex - x - 1.0;
      if (fabs(x) < 0x1p-10) k = x * x * (0.5 + x * (1.0 / 6 + x * (1.0 / 24 + x * (1.0 / 120))));
      l += a.beta * k;
      dl += a.beta * (1.0 - ex);
    }
    sum[0] += seq_w * l;
    sum[1] += seq_w * k;
    sum[2] += take ? 0.0 : seq_w;
    sum[3] += 1.0;
    g[i] = (float)(seq_w * dl * a.grad_scale);
  }
  if (a.grad) store_four(a.grad, t0, a.N, g);
  if (a.by_seq) sum[3] = gridDim.x == 1 ? live_sequences<NT>(a) : 0.0;
  block_totals<NT>(sum, red);
  if (threadIdx.x != 0) return;
  if (gridDim.x == 1) {
    write_losses(a, sum);
  } else {
#pragma unroll
    for (int q = 0; q < kPolSums; ++q) a.part[(int64_t)blockIdx.x * kPolSums + q] = sum[q];
  }
}

__global__ __launch_bounds__(kPolFinThreads) void policy_finish_kernel(PolicyArgs a, int n_parts) {
  __shared__ double red[kPolFinThreads / 64][kPolSums];
  double sum[kPolSums] = {0.0, 0.0, 0.0, 0.0};
  for (int k = threadIdx.x; k < n_parts; k += kPolFinThreads)
#pragma unroll
    for (int q = 0; q < kPolSums; ++q) sum[q] += a.part[(int64_t)k * kPolSums + q];
  if (a.by_seq) sum[3] = live_sequences<kPolFinThreads>(a);
  block_totals<kPolFinThreads>(sum, red);
  if (threadIdx.x == 0) write_losses(a, sum);
}

// g_logp = grad * upstream * (what is left of 1 / (tokens or sequences counted))
// (a token without a gradient keeps its exact zero, whatever the upstream one is)
__global__ __launch_bounds__(kPolThreads) void policy_bwd_kernel(int64_t N, const float* grad, const float* g_loss,
                                                                 float* g_logp) {
  const float c = grad[N] * g_loss[0];
  const int64_t t0 = (int64_t)blockIdx.x * kPolTile + threadIdx.x * kPolTok;
  float g[kPolTok];
  load_four(grad, t0, N, g);
#pragma unroll
  for (int i = 0; i < kPolTok; ++i) g[i] = g[i] == 0.f ? 0.f : g[i] * c;
  store_four(g_logp, t0, N, g);
}

}  // namespace

namespace {
int64_t tiles_of(int64_t N) { return (N + kPolTile - 1) / kPolTile; }
}  // namespace

size_t policy_part_bytes(int64_t N) { return (size_t)tiles_of(N) * kPolSums * sizeof(double); }

hipError_t launch_policy_count(const PolicyArgs& a, hipStream_t stream) {
  const dim3 grid((unsigned)std::min<int64_t>(a.S, kPolCountBlocks));
  if (a.N / a.S >= 65536)
    hipLaunchKernelGGL(policy_count_kernel<1024>, grid, dim3(1024), 0, stream, a);
  else
    hipLaunchKernelGGL(policy_count_kernel<256>, grid, dim3(256), 0, stream, a);
  return hipGetLastError();
}

hipError_t launch_policy_fwd(const PolicyArgs& a, hipStream_t stream) {
  if (a.N <= kPolOneBlock)
    hipLaunchKernelGGL(policy_fwd_kernel<1024>, dim3(1), dim3(1024), 0, stream, a);
  else
    hipLaunchKernelGGL(policy_fwd_kernel<kPolThreads>, dim3((unsigned)tiles_of(a.N)), dim3(kPolThreads), 0, stream, a);
  return hipGetLastError();
}

bool policy_finishes(int64_t N) { return N <= kPolOneBlock; }

hipError_t launch_policy_finish(const PolicyArgs& a, hipStream_t stream) {
  hipLaunchKernelGGL(policy_finish_kernel, dim3(1), dim3(kPolFinThreads), 0, stream, a, (int)tiles_of(a.N));
  return hipGetLastError();
}

hipError_t launch_policy_bwd(int64_t N, const float* grad, const float* g_loss, float* g_logp, hipStream_t stream) {
  hipLaunchKernelGGL(policy_bwd_kernel, dim3((unsigned)tiles_of(N)), dim3(kPolThreads), 0, stream, N, grad,
                     g_loss, g_logp);
  return hipGetLastError();
}

}  // namespace mls
