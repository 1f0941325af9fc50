// Layer norm of the hidden states in front of a head, forward and backward.
// Per row x of d entries, with weight w and an optional bias b:
//   mu = mean(x),  r = 1 / sqrt(mean((x - mu)^2) + eps),  xh = (x - mu) r,  y = xh w + b
//   gx = r (u - mean(u) - xh mean(u xh))  with u = gy w,
//   gw = sum_t gy xh,   gb = sum_t gy.
//
// Memory-bound: a pass reads and writes each row once. The W waves of a row hold
// it in registers as it was loaded, CPL chunks of 16 bytes a lane, so the deviations
// are taken from the mean itself (no sum of squares to cancel against). Each wave
// centres its own part first and the parts are joined by the pairwise formula
//   sum (x - mu)^2 = sum_w [ M_w + n_w (mu_w - mu)^2 ],
// which costs one barrier. R rows go through it together, so that enough loads are
// in flight for each. A block takes G * R rows at a time and goes on by gridDim.x *
// G * R, with w and b (backward: w and the running sums of gw and gb) in registers;
// a block's parts of gw and gb leave once, in fp32, and a second kernel adds them in
// block order, so the results are bitwise reproducible.
//
// Rows may begin at any element: 16-byte accesses need no 16-byte address here. Only
// a width that is no multiple of the chunk has a last, partial chunk (TAIL).
#include <math.h>

#include <algorithm>

#include "mls_device.h"
#include "mls_launch.h"
#include "mls_vec.h"
#include "mls_wave.h"

namespace mls {

namespace {

constexpr int kNormMaxWaves = 16;  // of a row, and of a block
constexpr int kNormMaxRows = 4;    // a group takes together
constexpr int64_t kNormMaxWidth = 16384;
constexpr int kNormRedCols = 64;
constexpr int kNormRedRows = 16;

// Chunk c of lane j holds entries [at, at + kN) of a row of L lanes.
template <typename A>
__device__ __forceinline__ int chunk_at(int c, int j, int L) {
  return (c * L + j) * Chunk<A>::kN;
}

// A row's chunks of this lane, as stored; zeros past the row's end and on dead rows.
template <typename A, int CPL, bool NT>
__device__ __forceinline__ void load_row(const typename Elt<A>::type* p, int d, int j, int L, bool live,
                                         uint4 (&v)[CPL]) {
  constexpr int N = Chunk<A>::kN;
#pragma unroll
  for (int c = 0; c < CPL; ++c) {
    const int k = chunk_at<A>(c, j, L);
    v[c] = make_uint4(0, 0, 0, 0);
    if (live && k + N <= d) {
      v[c] = load16_any<NT>(p + k);
    } else if (live && k < d) {
      float e[N];
#pragma unroll
      for (int i = 0; i < N; ++i) e[i] = k + i < d ? widen(p[k + i]) : 0.f;
      v[c] = Chunk<A>::pack(e);  // exact: the values are of the type
    }
  }
}

template <typename A, bool NT>
__device__ __forceinline__ void store_chunk(typename Elt<A>::type* p, int d, int k, const float* v) {
  constexpr int N = Chunk<A>::kN;
  if (k + N <= d) {
    store16_any<NT>(p + k, Chunk<A>::pack(v));
  } else if (k < d) {
#pragma unroll
    for (int i = 0; i < N; ++i)
      if (k + i < d) p[k + i] = to_storage<A>(v[i]);
  }
}

// Where the waves of a row leave their parts: wave k of group g puts row q's at slot
// (q, its own), and lane 16 q + k of every wave of the group reads it back, so that
// one read and a sum over 16 lanes join up to four rows.
struct RowSlots {
  int W, wave, first, lane, k, q;
  __device__ __forceinline__ RowSlots(int waves, int g)
      : W(waves), wave(threadIdx.x >> 6), first(g * waves), lane(threadIdx.x & 63), k(lane & 15), q(lane >> 4) {}
  __device__ __forceinline__ int mine(int row) const { return row * kNormMaxWaves + wave; }
  __device__ __forceinline__ bool live(int rows) const { return k < W && q < rows; }
  __device__ __forceinline__ int theirs() const { return q * kNormMaxWaves + first + k; }
};

// Entries of a parameter (bf16 or fp32) in the lane's layout; zeros past the end.
// Wide loads: a block's first rows wait for these.
template <typename A, int CPL>
__device__ __forceinline__ void load_param(const void* p, bool f32, int d, int j, int L,
                                           float (&v)[CPL][Chunk<A>::kN]) {
  constexpr int N = Chunk<A>::kN;
#pragma unroll
  for (int c = 0; c < CPL; ++c) {
    const int k = chunk_at<A>(c, j, L);
    if (k + N <= d) {
      uint4 raw[2] = {make_uint4(0, 0, 0, 0), make_uint4(0, 0, 0, 0)};
      if (f32) {
#pragma unroll
        for (int h = 0; h < N / 4; ++h) raw[h] = load16_any<false>(static_cast<const float*>(p) + k + 4 * h);
      } else if (N == 8) {
        raw[0] = load16_any<false>(static_cast<const uint16_t*>(p) + k);
      } else {
        typedef unsigned int u32x2_any_t __attribute__((ext_vector_type(2), aligned(2)));
        const u32x2_any_t r = *reinterpret_cast<const u32x2_any_t*>(static_cast<const uint16_t*>(p) + k);
        raw[0].x = r.x;
        raw[0].y = r.y;
      }
      float x[8], y[8];
      Chunk<F32>::unpack(raw[0], x);
      Chunk<F32>::unpack(raw[1], x + 4);
      Chunk<Bf16>::unpack(raw[0], y);
#pragma unroll
      for (int i = 0; i < N; ++i) v[c][i] = f32 ? x[i] : y[i];
    } else {
#pragma unroll
      for (int i = 0; i < N; ++i)
        v[c][i] = k + i >= d ? 0.f
                  : f32      ? static_cast<const float*>(p)[k + i]
                             : widen(static_cast<const uint16_t*>(p)[k + i]);
    }
  }
}

template <typename A, int CPL, int R, bool TAIL, bool MULTI, bool NT>
__global__ __launch_bounds__(MULTI ? 1024 : 256) void layer_norm_fwd_kernel(NormArgs a) {
  typedef typename Elt<A>::type TA;
  constexpr int N = Chunk<A>::kN;
  __shared__ float4 red[2][kNormMaxWaves * kNormMaxRows];
  const int d = a.d, W = a.waves, L = W * 64, G = blockDim.x / L;
  const int g = threadIdx.x / L, j = threadIdx.x % L;
  const RowSlots sl(W, g);
  float w[CPL][N], b[CPL][N];
  load_param<A, CPL>(a.weight, a.param_f32, d, j, L, w);
  if (a.bias)
    load_param<A, CPL>(a.bias, a.param_f32, d, j, L, b);
  else
#pragma unroll
    for (int c = 0; c < CPL; ++c)
#pragma unroll
      for (int i = 0; i < N; ++i) b[c][i] = 0.f;
  float n = 0.f;  // entries of this wave
#pragma unroll
  for (int c = 0; c < CPL; ++c) n += (float)min(N, max(0, d - chunk_at<A>(c, j, L)));
  n = wave_sum(n);
  // means by division: exact where the sum is (a constant row has no deviations)
  const float fn = n > 0.f ? n : 1.f, fd = (float)d;
  int par = 0;
  for (int64_t t0 = (int64_t)blockIdx.x * G * R; t0 < a.T; t0 += (int64_t)gridDim.x * G * R, par ^= 1) {
    uint4 x[R][CPL];
    float mu[R], var[R];
#pragma unroll
    for (int q = 0; q < R; ++q) {
      const int64_t t = t0 + q * G + g;  // dead rows still join the barrier
      load_row<A, CPL, NT>(static_cast<const TA*>(a.x) + t * a.ld_x, d, j, L, t < a.T, x[q]);
    }
#pragma unroll
    for (int q = 0; q < R; ++q) {
      float v[CPL][N], s = 0.f, m2 = 0.f;
#pragma unroll
      for (int c = 0; c < CPL; ++c) {
        Chunk<A>::unpack(x[q][c], v[c]);
#pragma unroll
        for (int i = 0; i < N; ++i) s += v[c][i];
      }
      s = wave_sum(s);
      const float mw = s / fn;
#pragma unroll
      for (int c = 0; c < CPL; ++c) {
        const int k = chunk_at<A>(c, j, L);
#pragma unroll
        for (int i = 0; i < N; ++i) {
          const float e = k + (TAIL ? i : 0) < d ? v[c][i] - mw : 0.f;
          m2 = fmaf(e, e, m2);
        }
      }
      m2 = wave_sum(m2);
      mu[q] = mw;
      var[q] = m2;
      if (MULTI && sl.lane == 0) red[par][sl.mine(q)] = make_float4(s, m2, n, mw);
    }
    if (MULTI) {
      __syncthreads();
      const float4 p = sl.live(R) ? red[par][sl.theirs()] : make_float4(0.f, 0.f, 0.f, 0.f);
      const float m = row16_sum(p.x) / fd;
      const float e = p.w - m;
      const float v = row16_sum(fmaf(p.z * e, e, p.y));
#pragma unroll
      for (int q = 0; q < R; ++q) {
        mu[q] = lane_read(m, 16 * q);
        var[q] = lane_read(v, 16 * q);
      }
    }
#pragma unroll
    for (int q = 0; q < R; ++q) {
      const int64_t t = t0 + q * G + g;
      if (t >= a.T) continue;
      const float r = 1.f / sqrtf(var[q] / fd + a.eps);
      if (a.stats && j == 0) {
        a.stats[t] = mu[q];
        a.stats[a.T + t] = r;
      }
#pragma unroll
      for (int c = 0; c < CPL; ++c) {
        float v[N];
        Chunk<A>::unpack(x[q][c], v);
#pragma unroll
        for (int i = 0; i < N; ++i) v[i] = fmaf((v[i] - mu[q]) * r, w[c][i], b[c][i]);
        store_chunk<A, NT>(static_cast<TA*>(a.y) + t * d, d, chunk_at<A>(c, j, L), v);
      }
    }
  }
}

template <typename A, int CPL, int R, bool MULTI, bool NT>
__global__ __launch_bounds__(MULTI ? 1024 : 512) void layer_norm_bwd_kernel(NormArgs a) {
  typedef typename Elt<A>::type TA;
  constexpr int N = Chunk<A>::kN;
  __shared__ float2 red[2][kNormMaxWaves * kNormMaxRows];
  extern __shared__ float sums[];  // [2][d], only with G > 1
  const int d = a.d, W = a.waves, L = W * 64, G = blockDim.x / L;
  const int g = threadIdx.x / L, j = threadIdx.x % L;
  const RowSlots sl(W, g);
  const float inv_d = 1.f / (float)d;
  float w[CPL][N], gw[CPL][N], gb[CPL][N];
  load_param<A, CPL>(a.weight, a.param_f32, d, j, L, w);
#pragma unroll
  for (int c = 0; c < CPL; ++c)
#pragma unroll
    for (int i = 0; i < N; ++i) gw[c][i] = gb[c][i] = 0.f;
  int par = 0;
  for (int64_t t0 = (int64_t)blockIdx.x * G * R; t0 < a.T; t0 += (int64_t)gridDim.x * G * R, par ^= 1) {
    uint4 x[R][CPL], y[R][CPL];
    float mu[R], r[R], s0[R], s1[R];
#pragma unroll
    for (int q = 0; q < R; ++q) {
      const int64_t t = t0 + q * G + g;
      const bool live = t < a.T;
      load_row<A, CPL, NT>(static_cast<const TA*>(a.x) + t * a.ld_x, d, j, L, live, x[q]);
      load_row<A, CPL, NT>(static_cast<const TA*>(a.g_y) + t * d, d, j, L, live, y[q]);
      mu[q] = live ? a.stats[t] : 0.f;
      r[q] = live ? a.stats[a.T + t] : 0.f;
    }
#pragma unroll
    for (int q = 0; q < R; ++q) {
      s0[q] = s1[q] = 0.f;
#pragma unroll
      for (int c = 0; c < CPL; ++c) {
        float xv[N], gv[N];
        Chunk<A>::unpack(x[q][c], xv);
        Chunk<A>::unpack(y[q][c], gv);
#pragma unroll
        for (int i = 0; i < N; ++i) {
          // past the end of a row gy and w are 0
          const float xh = (xv[i] - mu[q]) * r[q], u = gv[i] * w[c][i];
          gw[c][i] = fmaf(gv[i], xh, gw[c][i]);
          gb[c][i] += gv[i];
          s0[q] += u;
          s1[q] = fmaf(u, xh, s1[q]);
        }
      }
      s0[q] = wave_sum(s0[q]);
      s1[q] = wave_sum(s1[q]);
      if (MULTI && sl.lane == 0) red[par][sl.mine(q)] = make_float2(s0[q], s1[q]);
    }
    if (MULTI) {
      __syncthreads();
      const float2 p = sl.live(R) ? red[par][sl.theirs()] : make_float2(0.f, 0.f);
      const float p0 = row16_sum(p.x), p1 = row16_sum(p.y);
#pragma unroll
      for (int q = 0; q < R; ++q) {
        s0[q] = lane_read(p0, 16 * q);
        s1[q] = lane_read(p1, 16 * q);
      }
    }
    if (!a.g_x) continue;
#pragma unroll
    for (int q = 0; q < R; ++q) {
      const int64_t t = t0 + q * G + g;
      if (t >= a.T) continue;
      const float c0 = s0[q] * inv_d, c1 = s1[q] * inv_d;
#pragma unroll
      for (int c = 0; c < CPL; ++c) {
        float xv[N], gv[N];
        Chunk<A>::unpack(x[q][c], xv);
        Chunk<A>::unpack(y[q][c], gv);
#pragma unroll
        for (int i = 0; i < N; ++i) {
          const float xh = (xv[i] - mu[q]) * r[q];
          gv[i] = r[q] * (fmaf(gv[i], w[c][i], -c0) - xh * c1);
        }
        store_chunk<A, NT>(static_cast<TA*>(a.g_x) + t * d, d, chunk_at<A>(c, j, L), gv);
      }
    }
  }
  // the block's parts: the groups' sums one after the other, in group order
  if (!a.part) return;
  for (int k = 0; k < G; ++k) {
    if (g == k) {
      float* out = a.part + (int64_t)blockIdx.x * 2 * d;
#pragma unroll
      for (int c = 0; c < CPL; ++c)
#pragma unroll
        for (int i = 0; i < N; ++i) {
          const int e = chunk_at<A>(c, j, L) + i;
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

template <typename A, int CPL, int R, bool MULTI, bool NT>
hipError_t launch_shape(const NormArgs& a, const NormShape& sh, bool bwd, hipStream_t s) {
  const dim3 grid(sh.blocks), block(sh.waves * sh.groups * 64);
  const size_t lds = bwd && sh.groups > 1 && a.part ? 2 * (size_t)a.d * sizeof(float) : 0;
  if (bwd)
    hipLaunchKernelGGL((layer_norm_bwd_kernel<A, CPL, R, MULTI, NT>), grid, block, lds, s, a);
  else if (a.d % Chunk<A>::kN)
    hipLaunchKernelGGL((layer_norm_fwd_kernel<A, CPL, R, true, MULTI, NT>), grid, block, 0, s, a);
  else
    hipLaunchKernelGGL((layer_norm_fwd_kernel<A, CPL, R, false, MULTI, NT>), grid, block, 0, s, a);
  return hipGetLastError();
}

template <typename A, bool MULTI, bool NT>
hipError_t launch_rows(const NormArgs& a, const NormShape& sh, bool bwd, hipStream_t s) {
  if (sh.cpl == 1 && sh.rows == 1) return launch_shape<A, 1, 1, MULTI, NT>(a, sh, bwd, s);
  if (sh.cpl == 1 && sh.rows == 2) return launch_shape<A, 1, 2, MULTI, NT>(a, sh, bwd, s);
  if (sh.cpl == 2 && sh.rows == 1) return launch_shape<A, 2, 1, MULTI, NT>(a, sh, bwd, s);
  if constexpr (A::kBytes == 4) {
    if (sh.cpl == 4 && sh.rows == 1) return launch_shape<A, 4, 1, MULTI, NT>(a, sh, bwd, s);
  }
  return hipErrorInvalidValue;
}

template <typename A>
hipError_t launch_norm(const NormArgs& a, const NormShape& sh, bool bwd, hipStream_t s) {
  if (sh.waves < 1 || sh.groups < 1 || sh.waves * sh.groups > (sh.waves > 1 ? kNormMaxWaves : bwd ? 8 : 4) ||
      sh.blocks < 1 || (int64_t)sh.waves * 64 * sh.cpl * Chunk<A>::kN < a.d || a.waves != sh.waves)
    return hipErrorInvalidValue;
  if (sh.waves > 1)
    return sh.nt ? launch_rows<A, true, true>(a, sh, bwd, s) : launch_rows<A, true, false>(a, sh, bwd, s);
  return sh.nt ? launch_rows<A, false, true>(a, sh, bwd, s) : launch_rows<A, false, false>(a, sh, bwd, s);
}

}  // namespace

int64_t norm_max_width() { return kNormMaxWidth; }

// Chosen by timing, forward / backward us (each pass in a process of its own order,
// the least of two to four):
// - waves: one chunk a lane while a row then has at most 4 (fp32: 8) waves, else two
//   (fp32: up to four). 32768 x 4352 bf16, 9 waves of one chunk against 5 of two:
//   144 / 187 and 127 / 162; 16384 x 2305 bf16, 5 against 3: 50 / 81 and 44 / 66;
//   16384 x 4096 fp32, 8 of two against 4 of four: 93 / 136 and 93 / 143.
// - rows: two at a time with one chunk a lane, where every block has them. 32768 x
//   1024 bf16, four, two, one: 32 / 43, 28 / 40, 32 / 39; four spill at 16 entries a
//   lane.
// - blocks: at 32768 x 4352 the forward takes 115 to 124 us with 1024 to 3072 blocks
//   and 197 with 16384, whose first rows wait for weight and bias; at 32768 x 1024 it
//   takes 31 with 1024 and 28 with 3072. The backward's parts are read again: 512 or
//   768 blocks 162 / 193.
// - non-temporal accesses where a row array is 64 MiB or more (32768 x 4352: 153 -> 137
//   us forward, 190 -> 162 backward with its shape; 16384 x 4096 fp32 backward 158 ->
//   136) and the default below, where the caches still hold what comes next (4096 x
//   2304 bf16: 20 -> 23 with them).
// At 32768 x 4352 the two passes move 570 and 856 MB: 4.6 and 5.3 TB/s of the 5.1 that
// a device copy of this size reaches.
NormShape norm_shape(int64_t T, int64_t d, bool f32, bool bwd) {
  constexpr int64_t kFwdBlocks = 3072, kBwdBlocks = 512, kNtBytes = 64ll << 20;
  NormShape sh;
  const int n = f32 ? 4 : 8, max_waves = f32 ? 8 : 4;
  const int chunks = (int)((d + n - 1) / n);
  for (sh.cpl = 1; chunks > 64 * sh.cpl * max_waves && sh.cpl < 16 / n; sh.cpl *= 2) {
  }
  sh.waves = (chunks + 64 * sh.cpl - 1) / (64 * sh.cpl);
  sh.groups = std::max(1, (bwd ? 8 : 4) / sh.waves);
  const int64_t most = bwd ? kBwdBlocks : kFwdBlocks;
  sh.rows = sh.cpl == 1 && T >= most * sh.groups * 2 ? 2 : 1;
  const int64_t step = (int64_t)sh.groups * sh.rows;
  sh.blocks = (int)std::min<int64_t>(most, (T + step - 1) / step);
  sh.nt = T * d * (f32 ? 4 : 2) >= kNtBytes;
  return sh;
}

hipError_t launch_layer_norm_fwd(const NormArgs& a, const NormShape& sh, bool f32, hipStream_t stream) {
  return f32 ? launch_norm<F32>(a, sh, false, stream) : launch_norm<Bf16>(a, sh, false, stream);
}

hipError_t launch_layer_norm_bwd(const NormArgs& a, const NormShape& sh, bool f32, hipStream_t stream) {
  return f32 ? launch_norm<F32>(a, sh, true, stream) : launch_norm<Bf16>(a, sh, true, stream);
}

hipError_t launch_layer_norm_params(const NormArgs& a, int n_parts, hipStream_t stream) {
  const dim3 grid((unsigned)((2 * a.d + kNormRedCols - 1) / kNormRedCols));
  hipLaunchKernelGGL(layer_norm_param_kernel, grid, dim3(kNormRedCols * kNormRedRows), 0, stream, a, n_parts);
  return hipGetLastError();
}

}  // namespace mls
