// Layer norm of the hidden states in front of a head, forward and backward.
// Per row x of d entries, with weight w and an optional bias b:
//   mu = mean(x),  r = 1 / sqrt(mean((x - mu)^2) + eps),  xh = (x - mu) r,  y = xh w + b
//   gx = r (u - mean(u) - xh mean(u xh))  with u = gy w,
//   gw = sum_t gy xh,   gb = sum_t gy.
//
// Memory-bound: a pass reads and writes each row once. The W waves of a row hold
// it in registers, CPL chunks of 16 bytes a lane, so the deviations are taken
// from the mean itself (no sum of squares to cancel against). Each wave centres
// its own part first and the parts are joined by the pairwise formula
//   sum (x - mu)^2 = sum_w [ M_w + n_w (mu_w - mu)^2 ],
// which costs one barrier a row. A block takes G rows at a time and goes on by
// gridDim.x * G, with w and b (backward: w and the running sums of gw and gb) in
// registers; a block's parts of gw and gb leave once, in fp32, and a second
// kernel adds them in block order, so the results are bitwise reproducible.
#include <math.h>

#include <algorithm>

#include "mls_device.h"
#include "mls_launch.h"
#include "mls_vec.h"
#include "mls_wave.h"

namespace mls {

namespace {

constexpr int kNormMaxWaves = 16;
constexpr int kNormLaneElts = 16;  // entries of a row per lane: more spill in the backward's 128 registers
constexpr int64_t kNormMaxWidth = 16384;
constexpr int kNormRedCols = 64;
constexpr int kNormRedRows = 16;

// Which entries of a row a lane holds: element i of chunk c of lane j among the
// row's L lanes. VEC: 16 consecutive bytes a chunk. Otherwise (a width, stride or
// address that is no multiple of 16 bytes) single entries, neighbours in
// neighbouring lanes.
template <typename A, bool VEC>
struct RowMap {
  static constexpr int VE = 16 / A::kBytes;
  __device__ __forceinline__ static int at(int c, int i, int j, int L) {
    return VEC ? (c * L + j) * VE + i : (c * VE + i) * L + j;
  }
};

__device__ __forceinline__ float widen(uint16_t v) { return __uint_as_float((uint32_t)v << 16); }
__device__ __forceinline__ float widen(float v) { return v; }

template <bool NT>
__device__ __forceinline__ void load_chunk(const uint16_t* p, float* v) { load8<NT>(p, v); }
template <bool NT>
__device__ __forceinline__ void load_chunk(const float* p, float* v) { load4<NT>(p, v); }
template <bool NT>
__device__ __forceinline__ void store_chunk(uint16_t* p, const float* v) { store8<NT>(p, v); }
template <bool NT>
__device__ __forceinline__ void store_chunk(float* p, const float* v) { store4<NT>(p, v); }

// A row's entries of this lane; zeros past the row's end and on dead rows.
template <typename A, int CPL, bool VEC>
__device__ __forceinline__ void load_row(const typename Elt<A>::type* p, int d, int j, int L, bool live,
                                         float (&v)[CPL][RowMap<A, VEC>::VE]) {
  using M = RowMap<A, VEC>;
#pragma unroll
  for (int c = 0; c < CPL; ++c) {
    if (VEC) {
      const int k = M::at(c, 0, j, L);
      if (live && k < d) {
        load_chunk<false>(p + k, v[c]);
      } else {
#pragma unroll
        for (int i = 0; i < M::VE; ++i) v[c][i] = 0.f;
      }
    } else {
#pragma unroll
      for (int i = 0; i < M::VE; ++i) {
        const int k = M::at(c, i, j, L);
        v[c][i] = (live && k < d) ? widen(p[k]) : 0.f;
      }
    }
  }
}

template <typename A, int CPL, bool VEC>
__device__ __forceinline__ void store_row(typename Elt<A>::type* p, int d, int j, int L,
                                          const float (&v)[CPL][RowMap<A, VEC>::VE]) {
  using M = RowMap<A, VEC>;
#pragma unroll
  for (int c = 0; c < CPL; ++c) {
    if (VEC) {
      const int k = M::at(c, 0, j, L);
      if (k < d) store_chunk<false>(p + k, v[c]);
    } else {
#pragma unroll
      for (int i = 0; i < M::VE; ++i) {
        const int k = M::at(c, i, j, L);
        if (k < d) p[k] = to_storage<A>(v[c][i]);
      }
    }
  }
}

// Entries of a parameter (bf16 or fp32) in the lane's layout; `fill` past the end.
template <typename A, int CPL, bool VEC>
__device__ __forceinline__ void load_param(const void* p, bool f32, int d, int j, int L, float fill,
                                           float (&v)[CPL][RowMap<A, VEC>::VE]) {
  using M = RowMap<A, VEC>;
#pragma unroll
  for (int c = 0; c < CPL; ++c)
#pragma unroll
    for (int i = 0; i < M::VE; ++i) {
      const int k = M::at(c, i, j, L);
      v[c][i] = k >= d ? fill : f32 ? static_cast<const float*>(p)[k] : widen(static_cast<const uint16_t*>(p)[k]);
    }
}

template <typename A, int CPL, bool VEC, bool MULTI>
__global__ __launch_bounds__(MULTI ? 1024 : 512) void layer_norm_fwd_kernel(NormArgs a) {
  using M = RowMap<A, VEC>;
  typedef typename Elt<A>::type TA;
  __shared__ float4 red[2][kNormMaxWaves];
  const int d = a.d, W = a.waves, L = W * 64, G = blockDim.x / L;
  const int g = threadIdx.x / L, j = threadIdx.x % L;
  const int wave = threadIdx.x >> 6, first = g * W;
  float w[CPL][M::VE], b[CPL][M::VE], x[CPL][M::VE];
  load_param<A, CPL, VEC>(a.weight, a.param_f32, d, j, L, 0.f, w);
  if (a.bias)
    load_param<A, CPL, VEC>(a.bias, a.param_f32, d, j, L, 0.f, b);
  else
#pragma unroll
    for (int c = 0; c < CPL; ++c)
#pragma unroll
      for (int i = 0; i < M::VE; ++i) b[c][i] = 0.f;
  float n = 0.f;  // entries of this wave
#pragma unroll
  for (int c = 0; c < CPL; ++c)
#pragma unroll
    for (int i = 0; i < M::VE; ++i) n += M::at(c, i, j, L) < d ? 1.f : 0.f;
  n = wave_sum(n);
  // means by division: exact where the sum is (a constant row has no deviations)
  const float fn = n > 0.f ? n : 1.f, fd = (float)d;
  int par = 0;
  for (int64_t t0 = (int64_t)blockIdx.x * G; t0 < a.T; t0 += (int64_t)gridDim.x * G, par ^= 1) {
    const int64_t t = t0 + g;
    const bool live = t < a.T;  // dead rows still join the barriers
    load_row<A, CPL, VEC>(static_cast<const TA*>(a.x) + t * a.ld_x, d, j, L, live, x);
    float s = 0.f;
#pragma unroll
    for (int c = 0; c < CPL; ++c)
#pragma unroll
      for (int i = 0; i < M::VE; ++i) s += x[c][i];
    s = wave_sum(s);
    const float mw = s / fn;
    float q = 0.f;
#pragma unroll
    for (int c = 0; c < CPL; ++c)
#pragma unroll
      for (int i = 0; i < M::VE; ++i) {
        const float e = M::at(c, i, j, L) < d ? x[c][i] - mw : 0.f;
        q = fmaf(e, e, q);
      }
    q = wave_sum(q);
    float mu = mw, var = q;
    if (MULTI) {
      if ((threadIdx.x & 63) == 0) red[par][wave] = make_float4(s, q, n, mw);
      __syncthreads();
      float tot = 0.f;
      for (int k = 0; k < W; ++k) tot += red[par][first + k].x;
      mu = tot / fd;
      var = 0.f;
      for (int k = 0; k < W; ++k) {
        const float4 p = red[par][first + k];
        const float e = p.w - mu;
        var += fmaf(p.z * e, e, p.y);
      }
    }
    const float r = 1.f / sqrtf(var / fd + a.eps);
    if (!live) continue;
    if (a.stats && j == 0) {
      a.stats[t] = mu;
      a.stats[a.T + t] = r;
    }
#pragma unroll
    for (int c = 0; c < CPL; ++c)
#pragma unroll
      for (int i = 0; i < M::VE; ++i) x[c][i] = fmaf((x[c][i] - mu) * r, w[c][i], b[c][i]);
    store_row<A, CPL, VEC>(static_cast<TA*>(a.y) + t * d, d, j, L, x);
  }
}

template <typename A, int CPL, bool VEC, bool MULTI>
__global__ __launch_bounds__(MULTI ? 1024 : 512) void layer_norm_bwd_kernel(NormArgs a) {
  using M = RowMap<A, VEC>;
  typedef typename Elt<A>::type TA;
  __shared__ float2 red[2][kNormMaxWaves];
  extern __shared__ float sums[];  // [2][d], only with G > 1
  const int d = a.d, W = a.waves, L = W * 64, G = blockDim.x / L;
  const int g = threadIdx.x / L, j = threadIdx.x % L;
  const int wave = threadIdx.x >> 6, first = g * W;
  const float inv_d = 1.f / (float)d;
  float w[CPL][M::VE], gw[CPL][M::VE], gb[CPL][M::VE], x[CPL][M::VE], u[CPL][M::VE];
  load_param<A, CPL, VEC>(a.weight, a.param_f32, d, j, L, 0.f, w);
#pragma unroll
  for (int c = 0; c < CPL; ++c)
#pragma unroll
    for (int i = 0; i < M::VE; ++i) gw[c][i] = gb[c][i] = 0.f;
  int par = 0;
  for (int64_t t0 = (int64_t)blockIdx.x * G; t0 < a.T; t0 += (int64_t)gridDim.x * G, par ^= 1) {
    const int64_t t = t0 + g;
    const bool live = t < a.T;
    load_row<A, CPL, VEC>(static_cast<const TA*>(a.x) + t * a.ld_x, d, j, L, live, x);
    load_row<A, CPL, VEC>(static_cast<const TA*>(a.g_y) + t * d, d, j, L, live, u);
    const float mu = live ? a.stats[t] : 0.f, r = live ? a.stats[a.T + t] : 0.f;
    float s0 = 0.f, s1 = 0.f;
#pragma unroll
    for (int c = 0; c < CPL; ++c)
#pragma unroll
      for (int i = 0; i < M::VE; ++i) {
        // past the end of a row u and w are 0
        const float xh = (x[c][i] - mu) * r, gy = u[c][i];
        gw[c][i] = fmaf(gy, xh, gw[c][i]);
        gb[c][i] += gy;
        x[c][i] = xh;
        u[c][i] = gy * w[c][i];
        s0 += u[c][i];
        s1 = fmaf(u[c][i], xh, s1);
      }
    s0 = wave_sum(s0);
    s1 = wave_sum(s1);
    if (MULTI) {
      if ((threadIdx.x & 63) == 0) red[par][wave] = make_float2(s0, s1);
      __syncthreads();
      s0 = s1 = 0.f;
      for (int k = 0; k < W; ++k) {
        const float2 p = red[par][first + k];
        s0 += p.x;
        s1 += p.y;
      }
    }
    if (!live || !a.g_x) continue;
    const float c0 = s0 * inv_d, c1 = s1 * inv_d;
#pragma unroll
    for (int c = 0; c < CPL; ++c)
#pragma unroll
      for (int i = 0; i < M::VE; ++i) x[c][i] = r * (u[c][i] - fmaf(x[c][i], c1, c0));
    store_row<A, CPL, VEC>(static_cast<TA*>(a.g_x) + t * d, d, j, L, x);
  }
  // the block's parts: the groups' sums one after the other, in group order
  if (!a.part) return;
  for (int k = 0; k < G; ++k) {
    if (g == k) {
      float* out = a.part + (int64_t)blockIdx.x * 2 * d;
#pragma unroll
      for (int c = 0; c < CPL; ++c)
#pragma unroll
        for (int i = 0; i < M::VE; ++i) {
          const int e = M::at(c, i, j, L);
          if (e >= d) continue;
          float vw = gw[c][i], vb = gb[c][i];
          if (k > 0) {
            vw += sums[e];
            vb += sums[d + e];
          }
          if (k < G - 1) {
            sums[e] = vw;
            sums[d + e] = vb;
          } else {
            out[e] = vw;
            out[d + e] = vb;
          }
        }
    }
    __syncthreads();
  }
}

// gw and gb from the blocks' parts [n][2][d].
__global__ __launch_bounds__(kNormRedCols* kNormRedRows) void layer_norm_param_kernel(NormArgs a, int n) {
  __shared__ float sh[kNormRedRows][kNormRedCols];
  const int c = threadIdx.x % kNormRedCols, r = threadIdx.x / kNormRedCols;
  const int e = blockIdx.x * kNormRedCols + c;  // of 2 d columns: gw, then gb
  const int n_col = 2 * a.d;
  float s = 0.f;
  if (e < n_col) {
#pragma unroll 8
    for (int k = r; k < n; k += kNormRedRows) s += a.part[(int64_t)k * n_col + e];
  }
  sh[r][c] = s;
  __syncthreads();
  if (r != 0 || e >= n_col) return;
  s = 0.f;
#pragma unroll
  for (int k = 0; k < kNormRedRows; ++k) s += sh[k][c];
  void* out = e < a.d ? a.g_weight : a.g_bias;
  if (!out) return;
  const int k = e < a.d ? e : e - a.d;
  if (a.param_f32)
    static_cast<float*>(out)[k] = s;
  else
    static_cast<uint16_t*>(out)[k] = to_storage<Bf16>(s);
}

template <typename A, int CPL, bool VEC>
hipError_t launch_fwd_shape(const NormArgs& a, const NormShape& sh, hipStream_t s) {
  const dim3 grid(sh.blocks), block(sh.waves * sh.groups * 64);
  if (sh.waves > 1)
    hipLaunchKernelGGL((layer_norm_fwd_kernel<A, CPL, VEC, true>), grid, block, 0, s, a);
  else
    hipLaunchKernelGGL((layer_norm_fwd_kernel<A, CPL, VEC, false>), grid, block, 0, s, a);
  return hipGetLastError();
}

template <typename A, int CPL, bool VEC>
hipError_t launch_bwd_shape(const NormArgs& a, const NormShape& sh, hipStream_t s) {
  const dim3 grid(sh.blocks), block(sh.waves * sh.groups * 64);
  const size_t lds = sh.groups > 1 && a.part ? 2 * (size_t)a.d * sizeof(float) : 0;
  if (sh.waves > 1)
    hipLaunchKernelGGL((layer_norm_bwd_kernel<A, CPL, VEC, true>), grid, block, lds, s, a);
  else
    hipLaunchKernelGGL((layer_norm_bwd_kernel<A, CPL, VEC, false>), grid, block, lds, s, a);
  return hipGetLastError();
}

template <typename A, bool VEC>
hipError_t launch_norm_cpl(const NormArgs& a, const NormShape& sh, bool bwd, hipStream_t s) {
  if (sh.cpl == 1) return bwd ? launch_bwd_shape<A, 1, VEC>(a, sh, s) : launch_fwd_shape<A, 1, VEC>(a, sh, s);
  if (sh.cpl == 2) return bwd ? launch_bwd_shape<A, 2, VEC>(a, sh, s) : launch_fwd_shape<A, 2, VEC>(a, sh, s);
  if constexpr (A::kBytes == 4) {
    if (sh.cpl == 3) return bwd ? launch_bwd_shape<A, 3, VEC>(a, sh, s) : launch_fwd_shape<A, 3, VEC>(a, sh, s);
    if (sh.cpl == 4) return bwd ? launch_bwd_shape<A, 4, VEC>(a, sh, s) : launch_fwd_shape<A, 4, VEC>(a, sh, s);
  }
  return hipErrorInvalidValue;
}

hipError_t launch_norm(const NormArgs& a, const NormShape& sh, bool f32, bool bwd, hipStream_t s) {
  const int ve = f32 ? 4 : 8;
  if (sh.waves < 1 || sh.waves * sh.groups > kNormMaxWaves || sh.blocks < 1 ||
      (int64_t)sh.waves * 64 * sh.cpl * ve < a.d || a.waves != sh.waves)
    return hipErrorInvalidValue;
  if (sh.vec)
    return f32 ? launch_norm_cpl<F32, true>(a, sh, bwd, s) : launch_norm_cpl<Bf16, true>(a, sh, bwd, s);
  return f32 ? launch_norm_cpl<F32, false>(a, sh, bwd, s) : launch_norm_cpl<Bf16, false>(a, sh, bwd, s);
}

}  // namespace

int64_t norm_max_width() { return kNormMaxWidth; }

NormShape norm_shape(int64_t T, int64_t d, bool f32, bool vec, bool bwd) {
  NormShape sh;
  const int ve = f32 ? 4 : 8;
  const int chunks = (int)((d + ve - 1) / ve);
  sh.cpl = sh.waves = 0;
  for (int c = 1; c <= kNormLaneElts / ve; ++c) {
    const int w = (chunks + 64 * c - 1) / (64 * c);
    // fewest idle lanes, then the fewest waves
    if (w <= kNormMaxWaves && (sh.cpl == 0 || c * w <= sh.cpl * sh.waves)) {
      sh.cpl = c;
      sh.waves = w;
    }
  }
  sh.vec = vec;
  sh.groups = sh.waves >= 4 ? 1 : sh.waves == 1 ? 4 : 2;
  const int64_t most = bwd ? 512 : 2048;
  sh.blocks = (int)std::min<int64_t>(most, (T + sh.groups - 1) / sh.groups);
  return sh;
}

hipError_t launch_layer_norm_fwd(const NormArgs& a, const NormShape& sh, bool f32, hipStream_t stream) {
  return launch_norm(a, sh, f32, false, stream);
}

hipError_t launch_layer_norm_bwd(const NormArgs& a, const NormShape& sh, bool f32, hipStream_t stream) {
  return launch_norm(a, sh, f32, true, stream);
}

hipError_t launch_layer_norm_params(const NormArgs& a, int n_parts, hipStream_t stream) {
  const dim3 grid((unsigned)((2 * a.d + kNormRedCols - 1) / kNormRedCols));
  hipLaunchKernelGGL(layer_norm_param_kernel, grid, dim3(kNormRedCols * kNormRedRows), 0, stream, a, n_parts);
  return hipGetLastError();
}

}  // namespace mls
