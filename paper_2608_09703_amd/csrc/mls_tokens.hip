// Token log-probabilities: what stands around the tile kernels (mls_fused.hip) and
// the gradient products (mls_gemm.hip).
//
// Only the tokens that count are computed: prompt and padding tokens, a quarter to
// two thirds of a post-training batch, are left out of every product. Their
// positions are packed in order (pack), the hidden states of the others copied
// together (gather) and the products run on those rows, whose number they read from
// the device; log-probabilities (merge) and grad_h (scatter) go back to the tokens'
// places. What an ignored token's hidden state holds does not matter, NaN included.
// The copies are T d elements in and out, memory-bound, against 2 T V d operations
// a product: at T = 4,096, d = 4,352, V = 49,152 they take 70 of 3,520 us.
#include <math.h>

#include "mls_device.h"
#include "mls_launch.h"
#include "mls_merge.h"
#include "mls_vec.h"
#include "mls_wave.h"

namespace mls {

namespace {

constexpr int kPackThreads = 1024;
constexpr int kPackTok = 4;  // tokens per thread and round

// One block walks the tokens in order: rank[t] = number of counting tokens before t
// (or -1), index = its inverse. Ignored tokens get their zeros here.
__global__ __launch_bounds__(kPackThreads) void token_pack_kernel(TokenArgs a) {
  __shared__ int wave_n[kPackThreads / 64];
  __shared__ int bad_any[kPackThreads / 64];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  int base = 0;
  int bad = 0;
  for (int64_t t0 = 0; t0 < a.T; t0 += kPackThreads * kPackTok) {
    const int64_t t = t0 + (int64_t)threadIdx.x * kPackTok;
    bool ok[kPackTok];
    int n = 0;
#pragma unroll
    for (int i = 0; i < kPackTok; ++i) {
      const int64_t y = t + i < a.T ? a.tokens[t + i] : a.ignore_index;
      ok[i] = y != a.ignore_index && y >= 0 && y < a.V;
      bad |= y != a.ignore_index && !ok[i];
      n += ok[i] ? 1 : 0;
    }
    const int incl = wave_incl_scan(n);
    if (lane == 63) wave_n[wave] = incl;
    __syncthreads();
    int before = base;
    for (int w = 0; w < kPackThreads / 64; ++w) {
      before += w < wave ? wave_n[w] : 0;
      base += wave_n[w];
    }
    int r = before + incl - n;
#pragma unroll
    for (int i = 0; i < kPackTok; ++i) {
      if (t + i >= a.T) continue;
      a.rank[t + i] = ok[i] ? r : -1;
      if (ok[i]) {
        a.index[r++] = (int32_t)(t + i);
      } else {
        a.logp[t + i] = 0.f;
        if (a.entropy) a.entropy[t + i] = 0.f;
      }
    }
    __syncthreads();  // wave_n is written again
  }
  bad = wave_sum(bad);
  if (lane == 0) bad_any[wave] = bad;
  __syncthreads();
  if (threadIdx.x != 0) return;
  bad = 0;
  for (int w = 0; w < kPackThreads / 64; ++w) bad |= bad_any[w];
  a.header[0] = base;
  a.header[1] = bad ? MLS_DEVFLAG_LABEL_RANGE : 0;
}

// Scales of rows are not smaller than with this as 1 - p: far above what kept logits
// may add to each other entry (e^-32, see kKeptRange; below it they would count for
// more than those entries themselves).
constexpr float kMinRest = 0x1p-40f;

// One wave per token and, for the rows behind the last one, per row: copies the
// token's hidden state to its row and its id along.
// Backward: with q = 1 - p[y] the logit gradient is G = s E, s = g q / tau and
// E = (onehot(y) - p) / q, and the products run on E, rounded to bfloat16, whose own
// token's entry is 1. That entry carries most of G, and whole rows of grad_W when few
// tokens count: rounded as g q / tau it left them up to 2^-8 off in every element at
// once. s goes into the copied hidden states for grad_W (sum_t E s h: one rounding an
// element, which the others average) and, in fp32, into grad_h's rows after the product.
template <typename E>
__global__ __launch_bounds__(kThreads) void token_gather_kernel(TokenArgs a) {
  using S = typename E::storage;
  constexpr int kPer = 16 / E::kBytes;  // elements per 16-byte access
  const int lane = threadIdx.x & 63;
  const int64_t t = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
  if (t >= a.T_pad) return;
  S* hc = static_cast<S*>(a.hc);
  S* hs = static_cast<S*>(a.hs);
  if (t >= a.header[0]) {
    for (int64_t k = (int64_t)lane * kPer; k < a.d; k += 64 * kPer) {
      if (hc) *reinterpret_cast<uint4*>(hc + t * a.d + k) = make_uint4(0, 0, 0, 0);
      if (hs) *reinterpret_cast<uint4*>(hs + t * a.d + k) = make_uint4(0, 0, 0, 0);
    }
  }
  if (t >= a.T) return;
  const int64_t r = a.rank[t];
  if (r < 0) return;
  const int64_t y = a.tokens[t];
  const S* h = static_cast<const S*>(a.h) + t * a.d;
  float scale = 0.f, rest = 0.f;
  if (hs) {
    rest = fmaxf(a.q[r], kMinRest);
    scale = a.g[t] / a.tau * rest;
  }
  for (int64_t k = (int64_t)lane * kPer; k < a.d; k += 64 * kPer) {
    const uint4 hv = *reinterpret_cast<const uint4*>(h + k);
    if (hc) *reinterpret_cast<uint4*>(hc + r * a.d + k) = hv;
    if (hs) {
      float v[kPer];
      Chunk<E>::unpack(hv, v);
#pragma unroll
      for (int i = 0; i < kPer; ++i) v[i] *= scale;
      *reinterpret_cast<uint4*>(hs + r * a.d + k) = Chunk<E>::pack(v);
    }
  }
  if (lane != 0) return;
  a.tokens_c[r] = y;
  if (hs) {
    a.g_c[r] = a.tau / rest;
    a.scale[r] = scale;
  }
}

// Row merge (one sub-model, temperature tau). With m the maximum of all logits, S the
// records' sum of exp((l - m) / tau) over the other entries and e that of the token's own,
//   q = 1 - p = S / (S + e),  logp = log(1 - q) where q is small, else (l_y - m) / tau - log(S + e),
//   entropy = logsumexp(l / tau) - mean_p(l) / tau.
// TOK tokens a block, a thread a token and TOK / 256 of its records (added pairwise, in
// a fixed tree): one up to 256 tokens, else the losses' four, in us for TOK 4 / 1: T = 96,
// V = 97,683 24 / 12; T = 18, V = 105,482 17 / 10; T = 651, V = 121,655 21 / 25.
constexpr int64_t kMergeFew = 256;
template <int TOK>
__global__ __launch_bounds__(kThreads) void token_merge_kernel(TokenArgs a) {
  constexpr int GRP = kThreads / TOK;
  __shared__ float4 sh[GRP][TOK];
  const int tl = threadIdx.x % TOK;
  const int grp = threadIdx.x / TOK;
  const int64_t tc = (int64_t)blockIdx.x * TOK + tl;
  const int64_t live = (int64_t)a.header[0] - a.t0;
  const int64_t Tc = live < a.Tc ? live : a.Tc;
  if ((int64_t)blockIdx.x * TOK >= Tc) return;
  const float inv_tau = 1.0f / a.tau;
  const float ct = kLog2e * inv_tau;
  RowState<1> st = {{-INFINITY}, {0.f}, {0.f}, {0.f}};
  if (tc < Tc) {
    const float4* part = a.partials + (tc / kFusedBN) * a.n_rec * kFusedBN + tc % kFusedBN;
#pragma unroll 4
    for (int j = grp; j < a.n_rec; j += GRP) {
      const float4 rec = part[(int64_t)j * kFusedBN];
      if (rec.x != -INFINITY) absorb<1>(st, ct, &rec);  // else rows all beyond V
    }
  }
  sh[grp][tl] = make_float4(st.m[0], st.s1[0], st.st[0], st.xr[0]);
#pragma unroll
  for (int w = GRP / 2; w >= 1; w >>= 1) {
    __syncthreads();
    if (grp < w) {
      const float4 rec = sh[grp + w][tl];
      if (rec.x != -INFINITY) {
        absorb<1>(st, ct, &rec);
        if (w > 1) sh[grp][tl] = make_float4(st.m[0], st.s1[0], st.st[0], st.xr[0]);
      }
    }
  }
  if (grp != 0 || tc >= Tc) return;
  const int64_t r = a.t0 + tc;
  const int64_t t = a.index[r];
  const float own = a.own[r];
  const float e = fast_exp2((own - st.m[0]) * ct);
  const float sum = st.st[0] + e;
  const float q = st.st[0] / sum;
  const float lse = st.m[0] * inv_tau + logf(sum);
  const float lp = q < 0.5f ? log1pf(-q) : (own - st.m[0]) * inv_tau - logf(sum);
  a.lse[r] = lse;
  a.q[r] = q;
  a.logp[t] = lp;
  if (a.entropy) a.entropy[t] = lse - fmaf(e, own, st.xr[0]) / (a.tau * sum);
  if (!isfinite(lp)) atomicOr(a.header + 1, MLS_DEVFLAG_NONFINITE);
}

// Logit gradients of a vocabulary chunk from the kept logits:
//   E = g_c / tau (onehot(y) - softmax(l / tau)),  l / tau = m / tau - d
// (see the gather), with the kept distance d (kKeptRange's form) to the record's maximum m. One wave per row and 512
// columns, 16-byte accesses; bound by the 4 bytes an element that it moves, where the
// tile kernel computes 2 d operations an element again. T = 4,096 (3,071 counted),
// d = 4,352, V = 49,152: 106 us (5.7 TB/s) for 1,200, and the forward's stores cost
// it 43; T = 1,531, d = 1,000, V = 32,003: 37 for 139. Rows
// behind the last are 0 as far as a K-tile of the products reads.
constexpr int kGradSpan = 512;
__global__ __launch_bounds__(kThreads) void token_grad_kernel(TokenArgs a) {
  const int lane = threadIdx.x & 63;
  const int64_t r = (int64_t)blockIdx.y * 4 + (threadIdx.x >> 6);
  const int64_t vc = (int64_t)blockIdx.x * kGradSpan + (int64_t)lane * 8;  // column of the chunk
  const int64_t n = a.header[0];
  if (r >= (n + kRowsKTile - 1) / kRowsKTile * kRowsKTile || r >= a.T_pad || vc >= a.cols) return;
  uint16_t* out = a.slab + r * a.ld_slab + vc;
  if (r >= n) {
    *reinterpret_cast<uint4*>(out) = make_uint4(0, 0, 0, 0);
    return;
  }
  const int64_t v = a.v0 + vc;
  const float m = a.partials[((r / kFusedBN) * a.n_rec + v / a.rec_rows) * kFusedBN + r % kFusedBN].x;
  const uint4 w4 = load16_nt(a.kept + r * a.ld_kept + v);
  const uint32_t w[4] = {w4.x, w4.y, w4.z, w4.w};
  const float inv_tau = 1.0f / a.tau;
  const float mt = fmaf(m, kLog2e * inv_tau, -a.lse[r] * kLog2e);
  const float c = a.g_c[r] * inv_tau;
  const int yrel = (int)(a.tokens_c[r] - v);
  float g[8];
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const uint32_t d = (i & 1) ? w[i >> 1] >> 16 : w[i >> 1] & 0xffffu;
    const float p = fast_exp2(fmaf((float)d, -kLog2e * kKeptRange / 65535.f, mt));
    g[i] = v + i < a.V ? -c * p : 0.f;
  }
  if (yrel >= 0 && yrel < 8) {
    const float own = a.q[r] * c;  // 1, up to the floor of the rest
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (i == yrel) g[i] = own;
  }
  *reinterpret_cast<uint4*>(out) = Chunk<Bf16>::pack(g);
}

// grad_h by token: the sum of its row's K parts, in order, times the row's scale, or
// zeros (with accumulate, nothing) where it does not count. One wave per token and 256
// columns, 4 elements a lane (both widths' granularity).
constexpr int kScatterSpan = 256;
template <typename O>
__global__ __launch_bounds__(kThreads) void token_scatter_kernel(TokenArgs a) {
  const int lane = threadIdx.x & 63;
  const int64_t t = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
  const int64_t k = (int64_t)blockIdx.y * kScatterSpan + (int64_t)lane * 4;
  if (t >= a.T || k >= a.d) return;
  const int64_t r = a.rank[t];
  if (r < 0 && a.accumulate) return;
  typename Elt<O>::type* out = static_cast<typename Elt<O>::type*>(a.grad_h) + t * a.d + k;
  float v[4] = {0.f, 0.f, 0.f, 0.f};
  if (r >= 0) {
    const float* src = a.gh_c + r * a.d + k;
    load4<false>(src, v);
#pragma unroll 8
    for (int s = 1; s < a.gh_parts; ++s) {
      float p[4];
      load4<false>(src + s * a.T * a.d, p);
#pragma unroll
      for (int i = 0; i < 4; ++i) v[i] += p[i];
    }
    const float scale = a.scale[r];
    float o[4] = {0.f, 0.f, 0.f, 0.f};
    if (a.accumulate) load4<false>(out, o);
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = fmaf(v[i], scale, o[i]);
  }
  store4<false>(out, v);
}

}  // namespace

hipError_t launch_token_pack(const TokenArgs& a, hipStream_t stream) {
  hipLaunchKernelGGL(token_pack_kernel, dim3(1), dim3(kPackThreads), 0, stream, a);
  return hipGetLastError();
}

hipError_t launch_token_gather(const TokenArgs& a, bool f32, hipStream_t stream) {
  const dim3 grid((unsigned)((a.T_pad + 3) / 4));
  if (f32)
    hipLaunchKernelGGL(token_gather_kernel<F32>, grid, dim3(kThreads), 0, stream, a);
  else
    hipLaunchKernelGGL(token_gather_kernel<Bf16>, grid, dim3(kThreads), 0, stream, a);
  return hipGetLastError();
}

hipError_t launch_token_grad(const TokenArgs& a, hipStream_t stream) {
  const dim3 grid((unsigned)((a.cols + kGradSpan - 1) / kGradSpan), (unsigned)((a.T_pad + 3) / 4));
  if (a.T_pad > 4 * 65535ll) return hipErrorInvalidValue;
  hipLaunchKernelGGL(token_grad_kernel, grid, dim3(kThreads), 0, stream, a);
  return hipGetLastError();
}

hipError_t launch_token_merge(const TokenArgs& a, hipStream_t stream) {
  if (a.T <= kMergeFew)
    hipLaunchKernelGGL(token_merge_kernel<1>, dim3((unsigned)a.Tc), dim3(kThreads), 0, stream, a);
  else
    hipLaunchKernelGGL(token_merge_kernel<kRowTok>, dim3((unsigned)((a.Tc + kRowTok - 1) / kRowTok)), dim3(kThreads),
                       0, stream, a);
  return hipGetLastError();
}

hipError_t launch_token_scatter(const TokenArgs& a, hipStream_t stream) {
  const dim3 grid((unsigned)((a.T + 3) / 4), (unsigned)((a.d + kScatterSpan - 1) / kScatterSpan));
  if (a.out_f32)
    hipLaunchKernelGGL(token_scatter_kernel<F32>, grid, dim3(kThreads), 0, stream, a);
  else
    hipLaunchKernelGGL(token_scatter_kernel<Bf16>, grid, dim3(kThreads), 0, stream, a);
  return hipGetLastError();
}

}  // namespace mls
