// Global L2 norm of many gradient tensors, and their scaling by
//   c = min(1, max_norm / norm)
// (the gradient clipping of the paper's recipe, section 3: 1.0).
//
// Memory-bound: one read of every tensor for the norm, one read and one write for
// the scaling. Many small tensors next to a few large ones, so tiles of a fixed
// number of elements are dealt to the blocks of one launch whichever tensor they
// lie in (a search over the tensors' first tiles, kept in the kernel's arguments).
// Squares are added in 64 bits: they neither overflow nor vanish for any bf16 or
// fp32 value, and a sum over billions of elements keeps its digits. Every block
// leaves one part; one block adds the parts in a fixed order, so the norm is
// bitwise reproducible. The scaling takes the tiles in the reverse order: what
// the norm read last is still in the memory-side cache.
#include <math.h>

#include <algorithm>

#include "mls_device.h"
#include "mls_launch.h"
#include "mls_vec.h"
#include "mls_wave.h"

namespace mls {

namespace {

constexpr int kClipThreads = 256;
constexpr int kClipUnroll = 4;                                 // 16-byte loads in flight per lane
constexpr int kClipTile = kClipThreads * kClipUnroll * 8;      // elements per tile
constexpr int kClipBlocks = 2048;                              // blocks (and parts) of a launch
constexpr int kClipFinThreads = 1024;

__device__ __forceinline__ double wave_total(double v) {
#pragma unroll
  for (int o = 32; o >= 1; o >>= 1) v += __shfl_xor(v, o, 64);
  return v;
}

// Tensor that tile `tile` lies in.
template <class Args>
__device__ __forceinline__ int tensor_of(const Args& a, int tile) {
  int lo = 0, hi = a.count;
  while (hi - lo > 1) {
    const int m = (lo + hi) >> 1;
    if (a.tile_begin[m] <= tile)
      lo = m;
    else
      hi = m;
  }
  return lo;
}

__device__ __forceinline__ float widen(uint16_t v) { return __uint_as_float((uint32_t)v << 16); }
__device__ __forceinline__ float widen(float v) { return v; }

// Calls f(values, first element, count) for the lane's groups of 8 consecutive
// elements of [k0, k0 + kClipTile) below n, or for single elements where the
// addresses are not multiples of 16 bytes.
template <typename S>
__device__ __forceinline__ double tile_squares(const S* p, int64_t k0, int64_t n, bool vec) {
  double s0 = 0.0, s1 = 0.0;
  if (vec && k0 + kClipTile <= n) {
    float v[kClipUnroll][8];
#pragma unroll
    for (int i = 0; i < kClipUnroll; ++i) load8<false>(p + k0 + ((int64_t)i * kClipThreads + threadIdx.x) * 8, v[i]);
#pragma unroll
    for (int i = 0; i < kClipUnroll; ++i)
#pragma unroll
      for (int q = 0; q < 8; q += 2) {
        s0 = fma((double)v[i][q], (double)v[i][q], s0);
        s1 = fma((double)v[i][q + 1], (double)v[i][q + 1], s1);
      }
  } else {
    const int64_t end = k0 + kClipTile < n ? k0 + kClipTile : n;
#pragma unroll 8
    for (int64_t k = k0 + threadIdx.x; k < end; k += kClipThreads) {
      const double x = widen(p[k]);
      s0 = fma(x, x, s0);
    }
  }
  return s0 + s1;
}

__global__ __launch_bounds__(kClipThreads) void grad_norm_kernel(GradNormArgs a) {
  __shared__ double red[kClipThreads / 64];
  double s = 0.0;
  for (int tile = blockIdx.x; tile < a.tiles; tile += gridDim.x) {
    const int i = tensor_of(a, tile);
    const int64_t k0 = (int64_t)(tile - a.tile_begin[i]) * kClipTile;
    const bool vec = ((uintptr_t)a.data[i] & 15) == 0;
    const int64_t n = a.n[i] & kClipCountMask;
    s += (a.n[i] & kClipF32) ? tile_squares(static_cast<const float*>(a.data[i]), k0, n, vec)
                             : tile_squares(static_cast<const uint16_t*>(a.data[i]), k0, n, vec);
  }
  s = wave_total(s);
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = s;
  __syncthreads();
  if (threadIdx.x == 0) a.part[blockIdx.x] = (red[0] + red[1]) + (red[2] + red[3]);
}

__global__ __launch_bounds__(kClipFinThreads) void grad_norm_finish_kernel(const double* part, int n, double max_norm,
                                                                          float* norm, float* coef) {
  __shared__ double red[kClipFinThreads / 64];
  double s = 0.0;
  for (int k = threadIdx.x; k < n; k += kClipFinThreads) s += part[k];
  s = wave_total(s);
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = s;
  __syncthreads();
  if (threadIdx.x != 0) return;
  s = 0.0;
  for (int w = 0; w < kClipFinThreads / 64; ++w) s += red[w];
  const double x = sqrt(s);
  *norm = (float)x;
  // a norm that is NaN or infinite scales nothing
  if (coef) *coef = x > max_norm && isfinite(x) ? (float)(max_norm / x) : 1.f;
}

template <typename S, typename E>
__device__ __forceinline__ void scale_tile(const S* p, S* out, int64_t k0, int64_t n, bool vec, float c) {
  if (vec && k0 + kClipTile <= n) {
    float v[kClipUnroll][8];
#pragma unroll
    for (int i = 0; i < kClipUnroll; ++i) load8<false>(p + k0 + ((int64_t)i * kClipThreads + threadIdx.x) * 8, v[i]);
#pragma unroll
    for (int i = 0; i < kClipUnroll; ++i) {
#pragma unroll
      for (int q = 0; q < 8; ++q) v[i][q] *= c;
      store8<false>(out + k0 + ((int64_t)i * kClipThreads + threadIdx.x) * 8, v[i]);
    }
  } else {
    const int64_t end = k0 + kClipTile < n ? k0 + kClipTile : n;
#pragma unroll 8
    for (int64_t k = k0 + threadIdx.x; k < end; k += kClipThreads) out[k] = to_storage<E>(widen(p[k]) * c);
  }
}

__global__ __launch_bounds__(kClipThreads) void grad_scale_kernel(GradScaleArgs a) {
  const float c = *a.coef;
  for (int k = blockIdx.x; k < a.tiles; k += gridDim.x) {
    const int tile = a.tiles - 1 - k;
    const int i = tensor_of(a, tile);
    if (c == 1.f && a.data[i] == a.out[i]) continue;  // in place: as it is
    const int64_t k0 = (int64_t)(tile - a.tile_begin[i]) * kClipTile;
    const bool vec = (((uintptr_t)a.data[i] | (uintptr_t)a.out[i]) & 15) == 0;
    const int64_t n = a.n[i] & kClipCountMask;
    if (a.n[i] & kClipF32)
      scale_tile<float, F32>(static_cast<const float*>(a.data[i]), static_cast<float*>(a.out[i]), k0, n, vec, c);
    else
      scale_tile<uint16_t, Bf16>(static_cast<const uint16_t*>(a.data[i]), static_cast<uint16_t*>(a.out[i]), k0, n,
                                 vec, c);
  }
}

}  // namespace

int64_t clip_tiles(int64_t n) { return (n + kClipTile - 1) / kClipTile; }
int clip_blocks(int64_t tiles) { return (int)std::min<int64_t>(kClipBlocks, tiles); }

hipError_t launch_grad_norm(const GradNormArgs& a, hipStream_t stream) {
  hipLaunchKernelGGL(grad_norm_kernel, dim3(clip_blocks(a.tiles)), dim3(kClipThreads), 0, stream, a);
  return hipGetLastError();
}

hipError_t launch_grad_norm_finish(const double* part, int n, double max_norm, float* norm, float* coef,
                                   hipStream_t stream) {
  hipLaunchKernelGGL(grad_norm_finish_kernel, dim3(1), dim3(kClipFinThreads), 0, stream, part, n, max_norm, norm,
                     coef);
  return hipGetLastError();
}

hipError_t launch_grad_scale(const GradScaleArgs& a, hipStream_t stream) {
  hipLaunchKernelGGL(grad_scale_kernel, dim3(clip_blocks(a.tiles)), dim3(kClipThreads), 0, stream, a);
  return hipGetLastError();
}

}  // namespace mls
