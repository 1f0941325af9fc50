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
// the norm read last is still in the memory-side cache. It reads and writes past the
// caches (each byte is touched once more), the norm through them. us for 219 tensors of
// 503 million bf16 elements, norm and scaling: 174 + 340; with tiles of 4 chunks and the
// default policy 211 + 365; all non-temporal 159 + 359; with 192 MB kept in the caches
// between the passes by choice, and the rest past them, 175 + 370. 214 million fp32
// elements: 201 + 419, 231 + 449, 178 + 443, 209 + 469. That is 5.8 and 5.9 TB/s, where
// a device copy reaches 5.1.
// Tensors may begin at any element: 16-byte accesses need no 16-byte address here.
#include <math.h>

#include <algorithm>

#include "mls_device.h"
#include "mls_launch.h"
#include "mls_vec.h"
#include "mls_wave.h"

namespace mls {

namespace {

constexpr int kClipThreads = 256;
constexpr int kClipUnroll = 8;                                 // chunks of 16 bytes per lane and tile
constexpr int kClipTileBytes = kClipThreads * kClipUnroll * 16;
constexpr int kClipBlocks = 2048;                              // blocks (and parts) of a launch
constexpr int kClipFinThreads = 1024;

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

// One tile of a tensor: lane chunk i holds elements at k0 + (i * kClipThreads + tid) * kN.
template <typename E>
__device__ __forceinline__ int64_t tile_at(int64_t k0, int i) {
  return k0 + ((int64_t)i * kClipThreads + threadIdx.x) * Chunk<E>::kN;
}

template <typename E>
__device__ __forceinline__ double tile_squares(const void* data, int64_t k0, int64_t n) {
  constexpr int N = Chunk<E>::kN;
  const typename E::storage* p = static_cast<const typename E::storage*>(data);
  double s0 = 0.0, s1 = 0.0;
  if (k0 + kClipUnroll * kClipThreads * N <= n) {
    uint4 r[kClipUnroll];
#pragma unroll
    for (int i = 0; i < kClipUnroll; ++i) r[i] = load16_any<false>(p + tile_at<E>(k0, i));
#pragma unroll
    for (int i = 0; i < kClipUnroll; ++i) {
      float v[N];
      Chunk<E>::unpack(r[i], v);
#pragma unroll
      for (int q = 0; q < N; q += 2) {
        s0 = fma((double)v[q], (double)v[q], s0);
        s1 = fma((double)v[q + 1], (double)v[q + 1], s1);
      }
    }
  } else {  // a tensor's last tile, element by element
    for (int64_t k = k0 + threadIdx.x; k < n; k += kClipThreads) {
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
    const int64_t t = tile - a.tile_begin[i], n = a.n[i] & kClipCountMask;
    s += (a.n[i] & kClipF32) ? tile_squares<F32>(a.data[i], t * (kClipTileBytes / 4), n)
                             : tile_squares<Bf16>(a.data[i], t * (kClipTileBytes / 2), n);
  }
  s = wave_sum(s);
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = s;
  __syncthreads();
  if (threadIdx.x == 0) a.part[blockIdx.x] = (red[0] + red[1]) + (red[2] + red[3]);
}

__global__ __launch_bounds__(kClipFinThreads) void grad_norm_finish_kernel(const double* part, int n, double max_norm,
                                                                          float* norm, float* coef) {
  __shared__ double red[kClipFinThreads / 64];
  double s = 0.0;
  for (int k = threadIdx.x; k < n; k += kClipFinThreads) s += part[k];
  s = wave_sum(s);
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = s;
  __syncthreads();
  if (threadIdx.x != 0) return;
  s = 0.0;
  for (int w = 0; w < kClipFinThreads / 64; ++w) s += red[w];
  const double x = sqrt(s);
  const float f = (float)x;
  *norm = f;
  // a norm that is NaN or infinite, as the caller sees it in fp32, scales nothing
  if (coef) *coef = x > max_norm && isfinite(f) ? (float)(max_norm / x) : 1.f;
}

template <typename E>
__device__ __forceinline__ void scale_tile(const void* data, void* dst, int64_t k0, int64_t n, float c) {
  constexpr int N = Chunk<E>::kN;
  const typename E::storage* p = static_cast<const typename E::storage*>(data);
  typename E::storage* out = static_cast<typename E::storage*>(dst);
  if (k0 + kClipUnroll * kClipThreads * N <= n) {
    uint4 r[kClipUnroll];
#pragma unroll
    for (int i = 0; i < kClipUnroll; ++i) r[i] = load16_any<true>(p + tile_at<E>(k0, i));
#pragma unroll
    for (int i = 0; i < kClipUnroll; ++i) {
      float v[N];
      Chunk<E>::unpack(r[i], v);
#pragma unroll
      for (int q = 0; q < N; ++q) v[q] *= c;
      store16_any<true>(out + tile_at<E>(k0, i), Chunk<E>::pack(v));
    }
  } else {
    for (int64_t k = k0 + threadIdx.x; k < n; k += kClipThreads) out[k] = to_storage<E>(widen(p[k]) * c);
  }
}

__global__ __launch_bounds__(kClipThreads) void grad_scale_kernel(GradScaleArgs a) {
  const float c = *a.coef;
  for (int k = blockIdx.x; k < a.tiles; k += gridDim.x) {
    const int tile = a.tiles - 1 - k;
    const int i = tensor_of(a, tile);
    if (c == 1.f && a.data[i] == a.out[i]) continue;  // in place: as it is
    const int64_t t = tile - a.tile_begin[i], n = a.n[i] & kClipCountMask;
    if (a.n[i] & kClipF32)
      scale_tile<F32>(a.data[i], a.out[i], t * (kClipTileBytes / 4), n, c);
    else
      scale_tile<Bf16>(a.data[i], a.out[i], t * (kClipTileBytes / 2), n, c);
  }
}

}  // namespace

int64_t clip_tiles(int64_t n, bool f32) {
  const int64_t per = kClipTileBytes / (f32 ? 4 : 2);
  return (n + per - 1) / per;
}
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
