// Rows as 8-bit integers, for the head product on them: per row x of d entries
//   s = the float32 number next to max |x| / 127,  q = the integer next to x / s
// (ties to even), in [-127, 127].
//
// q is next to the exact quotient: the rounded quotient's integer is put right where it
// is not the nearest one. With r = x - q s, which one fused multiply-add gives exactly
// (|r| < s, and x and q s are multiples of one bit of s or less), the test 2 |r| > s has
// no rounding.
//
// A row with an infinity or NaN in it has the scale NaN and zeros.
#include <math.h>

#include "mls_device.h"
#include "mls_launch.h"
#include "mls_vec.h"
#include "mls_wave.h"

namespace mls {

namespace {

constexpr int kQuantThreads = 256;

__device__ __forceinline__ int quantize(float x, float s) {
#pragma clang fp contract(off)
  float q = rintf(x / s);
  const float r = 2.f * fmaf(-q, s, x);
  const float up = r > 0.f ? 1.f : -1.f;
  if (fabsf(r) > s || (fabsf(r) == s && ((int)q & 1))) q += up;
  return (int)fminf(fmaxf(q, -127.f), 127.f);
}

template <typename E>
__global__ __launch_bounds__(kQuantThreads) void quantize_rows_kernel(QuantArgs a) {
  __shared__ float red[kQuantThreads / 64];
  const int64_t t = blockIdx.x;
  const typename E::storage* x = static_cast<const typename E::storage*>(a.x) + t * a.ld;
  float m = 0.f;
  bool odd = false;
  for (int i = threadIdx.x; i < a.d; i += kQuantThreads) {
    const float v = fabsf(widen(x[i]));
    odd = odd || !(v < INFINITY);
    m = fmaxf(m, v);
  }
  m = odd ? INFINITY : m;
  m = wave_max(m);
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = m;
  __syncthreads();
  m = red[0];
#pragma unroll
  for (int w = 1; w < kQuantThreads / 64; ++w) m = fmaxf(m, red[w]);
  const float s = m < INFINITY ? m / 127.f : __uint_as_float(0x7fc00000u);
  if (threadIdx.x == 0) a.scale[t] = s;
  int8_t* q = a.q + t * a.d;
  for (int i = threadIdx.x; i < a.d; i += kQuantThreads)
    q[i] = (int8_t)(s > 0.f ? quantize(widen(x[i]), s) : 0);
}

}  // namespace

hipError_t launch_quantize_rows(const QuantArgs& a, hipStream_t stream) {
  const dim3 grid((unsigned)a.T);
  if (a.f32)
    hipLaunchKernelGGL(quantize_rows_kernel<F32>, grid, dim3(kQuantThreads), 0, stream, a);
  else
    hipLaunchKernelGGL(quantize_rows_kernel<Bf16>, grid, dim3(kQuantThreads), 0, stream, a);
  return hipGetLastError();
}

}  // namespace mls
