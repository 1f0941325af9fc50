// Rows as 8-bit integers, for the head product on them: per row x of d entries
//   s = the float32 number next to max |x| / 127,  q = the integer next to x / s
// (ties to even), in [-127, 127].
//
// q is next to the exact quotient: the integer from a rounded quotient is put right where
// it is not the nearest one. With r = x - q s, which one fused multiply-add gives exactly
// (|r| < s, and x and q s are multiples of half a bit of s), the test 2 |r| > s has no
// rounding.
//
// A row with an infinity or NaN in it has the scale NaN and zeros.
//
// Bound by its bytes: a row is loaded once, into the registers of 16 or 64 lanes, whose
// maximum needs no barrier, or for few rows of a block's 256.
#include <math.h>

#include "mls_device.h"
#include "mls_launch.h"
#include "mls_vec.h"
#include "mls_wave.h"

namespace mls {

namespace {

constexpr int kQuantThreads = 256;
// Rows up to which a block takes one at a time. d = 4,352, bf16, a block / a wave to a row: 8,192
// rows 28.8 / 32.5 us, 16,384 53.5 / 49.7, 49,152 145 / 128 (5.0 TB/s).
constexpr int kFewRows = 8192;

// The integer next to x / s.
__device__ __forceinline__ int quantize(float x, float s) {
#pragma clang fp contract(off)
  float q = rintf(x / s);
  const float r = 2.f * fmaf(-q, s, x);
  if (fabsf(r) > s || (fabsf(r) == s && ((int)q & 1))) q += r > 0.f ? 1.f : -1.f;
  return (int)fminf(fmaxf(q, -127.f), 127.f);
}

// The largest magnitude so far, as the bits of a float32 (of a bfloat16: two halves of a
// word apart). Bits of infinities and NaN are above every number's.
template <typename E>
struct Peak;
template <>
struct Peak<F32> {
  uint32_t m = 0;
  __device__ __forceinline__ void add(uint32_t w) {
    w &= 0x7fffffffu;
    m = w > m ? w : m;
  }
  __device__ __forceinline__ void add(float x) { add(__float_as_uint(x)); }
  __device__ __forceinline__ int bits() const { return (int)m; }
};
template <>
struct Peak<Bf16> {
  typedef unsigned short u16x2 __attribute__((ext_vector_type(2)));
  u16x2 m = {0, 0};
  __device__ __forceinline__ void add(uint32_t w) {
    m = __builtin_elementwise_max(m, __builtin_bit_cast(u16x2, w & 0x7fff7fffu));
  }
  __device__ __forceinline__ void add(uint16_t x) { add((uint32_t)x); }
  __device__ __forceinline__ int bits() const { return (int)(m.x > m.y ? m.x : m.y) << 16; }
};

template <int LANES>
__device__ __forceinline__ int lanes_max(int v) {
  auto up = [&](int o) { v = o > v ? o : v; };
  up(dpp_move<dppc::kXor1>(v, 0));
  up(dpp_move<dppc::kXor2>(v, 0));
  up(dpp_move<dppc::kHalfMirror>(v, 0));
  up(dpp_move<dppc::kMirror>(v, 0));
  if (LANES == 16) return v;
  const int a = lane_read(v, 0), b = lane_read(v, 16), c = lane_read(v, 32), d = lane_read(v, 48);
  v = a > b ? a : b;
  up(c);
  up(d);
  return v;
}

// The integers of a chunk as bytes. x inv + kMagic has the integer next to x inv in its
// low bits (ties to even); x inv is within 127 x 2^-24 = 8e-6 of x / s, so only where it
// comes as near to the middle between two integers as kNear says can that be another one
// than x / s's (one chunk of a wave in fifty), and quantize() is asked.
constexpr float kMagic = 12582912.f;  // 1.5 x 2^23
constexpr float kNear = 0.49998f;

template <typename E>
__device__ __forceinline__ void put_chunk(int8_t* p, uint4 r, float s, float inv) {
  constexpr int N = Chunk<E>::kN;
  typedef uint32_t words __attribute__((ext_vector_type(N / 4), aligned(1)));
  float v[N];
  uint32_t u[N];
  Chunk<E>::unpack(r, v);
  float off = inv > 0.f ? 0.f : 1.f;  // (no inverse: a scale of 0, NaN, or too small for one)
#pragma unroll
  for (int i = 0; i < N; ++i) {
    const float y = fmaf(v[i], inv, kMagic);
    u[i] = __float_as_uint(y);
    off = fmaxf(off, fabsf(fmaf(v[i], inv, kMagic - y)));
  }
  if (__ballot(off > kNear) != 0) {
#pragma unroll
    for (int i = 0; i < N; ++i) u[i] = s > 0.f ? (uint32_t)quantize(v[i], s) : 0u;
  }
  words w;
#pragma unroll
  for (int i = 0; i < N / 4; ++i) {
    const uint32_t lo = __builtin_amdgcn_perm(u[4 * i + 1], u[4 * i], 0x0c0c0400u);
    const uint32_t hi = __builtin_amdgcn_perm(u[4 * i + 3], u[4 * i + 2], 0x04000c0cu);
    w[i] = lo | hi;
  }
  *reinterpret_cast<words*>(p) = w;
}

// LANES lanes take a row of up to C chunks each; chunk c of a row is lane c % LANES's.
// C = 0: rows of any width, read twice.
template <typename E, int LANES, int C>
__global__ __launch_bounds__(kQuantThreads) void quantize_rows_kernel(QuantArgs a) {
  constexpr int N = Chunk<E>::kN;
  __shared__ int red[kQuantThreads / 64];
  const int l = threadIdx.x % LANES;
  const int64_t t = (int64_t)blockIdx.x * (kQuantThreads / LANES) + threadIdx.x / LANES;
  const bool in = t < a.T;  // (all lanes of a wave stay for the maximum)
  const typename E::storage* x = static_cast<const typename E::storage*>(a.x) + (in ? t : a.T - 1) * a.ld;
  const int whole = a.d / N;
  const int rest = a.d % N;  // entries of a last, shorter chunk: lane whole % LANES's
  uint4 raw[C > 0 ? C : 1];
  Peak<E> peak;
  auto look = [&](uint4 r) {
    peak.add(r.x);
    peak.add(r.y);
    peak.add(r.z);
    peak.add(r.w);
  };
  if constexpr (C > 0) {
#pragma unroll
    for (int c = 0; c < C; ++c) {
      raw[c] = make_uint4(0u, 0u, 0u, 0u);
      if (c * LANES + l < whole) raw[c] = load16_any<false>(x + (int64_t)(c * LANES + l) * N);
    }
#pragma unroll
    for (int c = 0; c < C; ++c) look(raw[c]);
  } else {
    for (int c = l; c < whole; c += LANES) look(load16_any<false>(x + (int64_t)c * N));
  }
  if (rest && l == whole % LANES)
    for (int i = 0; i < rest; ++i) peak.add(x[(int64_t)whole * N + i]);
  int m = lanes_max<LANES == 16 ? 16 : 64>(peak.bits());
  if constexpr (LANES == kQuantThreads) {
    if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = m;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < kQuantThreads / 64; ++w) m = red[w] > m ? red[w] : m;
  }
  if (!in) return;
  const float s = m < 0x7f800000 ? __int_as_float(m) / 127.f : __uint_as_float(0x7fc00000u);
  if (l == 0) a.scale[t] = s;
  const float inv = s > 1e-36f ? 1.f / s : 0.f;
  int8_t* q = a.q + t * a.d;
  if constexpr (C > 0) {
#pragma unroll
    for (int c = 0; c < C; ++c)
      if (c * LANES + l < whole) put_chunk<E>(q + (int64_t)(c * LANES + l) * N, raw[c], s, inv);
  } else {
    for (int c = l; c < whole; c += LANES) put_chunk<E>(q + (int64_t)c * N, load16_any<false>(x + (int64_t)c * N), s, inv);
  }
  if (rest && l == whole % LANES)
    for (int i = 0; i < rest; ++i)
      q[(int64_t)whole * N + i] = (int8_t)(s > 0.f ? quantize(widen(x[(int64_t)whole * N + i]), s) : 0);
}

// (a launch takes less than 2^32 threads: more rows go in pieces)
template <typename E, int LANES, int C>
hipError_t launch_quant(const QuantArgs& all, hipStream_t stream) {
  constexpr int rows = kQuantThreads / LANES;
  constexpr int64_t piece = (int64_t)rows << 23;
  for (int64_t t = 0; t < all.T; t += piece) {
    QuantArgs a = all;
    a.x = static_cast<const typename E::storage*>(all.x) + t * all.ld;
    a.q += t * all.d;
    a.scale += t;
    a.T = all.T - t < piece ? all.T - t : piece;
    hipLaunchKernelGGL((quantize_rows_kernel<E, LANES, C>), dim3((unsigned)((a.T + rows - 1) / rows)),
                       dim3(kQuantThreads), 0, stream, a);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

template <typename E>
hipError_t launch_quant_e(const QuantArgs& a, hipStream_t stream) {
  const int chunks = a.d / Chunk<E>::kN;
  if (chunks <= 64) return launch_quant<E, 16, 4>(a, stream);
  const int per = (chunks + 63) / 64;
  if (a.T <= kFewRows) {
    const int of_block = (chunks + kQuantThreads - 1) / kQuantThreads;
    if (of_block == 1) return launch_quant<E, kQuantThreads, 1>(a, stream);
    if (of_block <= 3) return launch_quant<E, kQuantThreads, 3>(a, stream);
    if (of_block <= 6) return launch_quant<E, kQuantThreads, 6>(a, stream);
  }
  if (per <= 2) return launch_quant<E, 64, 2>(a, stream);
  if (per <= 4) return launch_quant<E, 64, 4>(a, stream);
  if (per <= 6) return launch_quant<E, 64, 6>(a, stream);
  if (per <= 9) return launch_quant<E, 64, 9>(a, stream);
  if (per <= 16) return launch_quant<E, 64, 16>(a, stream);
  return launch_quant<E, 64, 0>(a, stream);
}

}  // namespace

hipError_t launch_quantize_rows(const QuantArgs& a, hipStream_t stream) {
  return a.f32 ? launch_quant_e<F32>(a, stream) : launch_quant_e<Bf16>(a, stream);
}

}  // namespace mls
