// The head step of nested speculative decoding (paper section 2, paragraph
// "Speculative Decoding"; the measured setting of section 3, "Speculative
// Decoding Throughput": greedy or nucleus top-p 0.9 sampling at temperature
// 0.4, a smaller sub-model drafting gamma tokens and a larger one verifying).
//
// 1. head_logits_kernel: logits[t][v] = sum_k o[t][k] W[v][k] in fp32, on the
//    MFMA tile core (tiles from 64 vocabulary rows x 32 tokens to 192 x 128, by
//    the rule at head_tile); the fp32 tile is staged in LDS and leaves the block
//    as 16-byte stores of token-major rows.
//    Decode batches are small, so the [rows, V] logits are cheap next to the
//    head itself.
// 2. sample_kernel: one 1024-thread block per row. The row's sampling
//    distribution is softmax(l / temperature) restricted to the nucleus: the
//    most probable tokens (ties: lower index first) up to and including the
//    first one at which the kept mass reaches top_p. The nucleus threshold is
//    the largest exp-weight value theta whose "weight >= theta" mass still
//    reaches top_p of the total (found as described below); tokens tied at theta are kept in
//    index order as far as needed. A draw with uniform u returns the smallest
//    index whose cumulative kept weight in index order exceeds u times the
//    kept total.
// 3. verify_kernel: one block per sequence tests its gamma drafts: the draft
//    token x is kept when u * q(x) < p(x); at the first rejection the next
//    token is drawn from max(0, p - q); if all are kept, one more token is drawn
//    from the verifier's distribution after the drafts. Greedy mode compares
//    with the verifier's argmax (lowest index on ties).
//
// All reductions run in a fixed order, so results are bitwise reproducible.
#include <math.h>

#include "mls_core.h"
#include "mls_device.h"
#include "mls_launch.h"
#include "mls_rowdist.h"
#include "mls_wave.h"

namespace mls {

namespace {

// ---------------------------------------------------------------------------
// 1. head logits
// ---------------------------------------------------------------------------

template <class Mma, typename E>
__global__ __launch_bounds__(Mma::NT, Mma::kBM == 64 ? 1 : 2) void head_logits_kernel(HeadArgs a) {
  constexpr int BM = Mma::kBM;  // vocabulary rows
  constexpr int BN = Mma::kBN;  // tokens
  constexpr int FM = Mma::FM;
  constexpr int FN = Mma::FN;
  constexpr int NT = Mma::NT;
  constexpr int kChunks = BM / 4;          // 16-byte chunks (4 floats) per token row of the tile
  constexpr int kSw = kChunks & -kChunks;  // chunk swizzle span: XOR stays inside aligned groups
  // the fp32 tile leaves in one pass, or in one pass per wave column when it
  // is larger than the stage memory
  constexpr int kPasses = (BN * BM * 4 + Mma::kSmemBytes - 1) / Mma::kSmemBytes;
  constexpr int kTok = BN / kPasses;  // tokens per pass
  static_assert(kPasses == 1 || kPasses == Mma::kWGN, "one pass, or one per wave column");
  static_assert(kTok * BM * 4 <= Mma::kSmemBytes, "a pass fits in the stage memory");
  __shared__ __attribute__((aligned(16))) char smem[Mma::kSmemBytes];

  const int tid = threadIdx.x;
  const int lane = tid & 63;
  const int wave = tid >> 6;
  const int wm = wave % Mma::kWGM;
  const int wn = wave / Mma::kWGM;
  const int bl = xcd_remap(blockIdx.x, gridDim.x);
  int vt, tt;
  tile_coords(bl, a.n_vt, a.n_tt, a.group_v, vt, tt);
  const int64_t vbase = (int64_t)vt * BM;
  const int64_t tbase = (int64_t)tt * BN;
  const int64_t kb = a.d * E::kBytes;

  Mma mma;
  mma.run(static_cast<const char*>(a.W), kb, vbase, a.V, static_cast<const char*>(a.o), kb, tbase,
          a.T, kb, smem, tid);

  // stage: token row t of a pass holds kChunks chunks of 4 vocabulary entries,
  // chunk c at c ^ (t % kSw)
  float* st = reinterpret_cast<float*>(smem);
  const bool vec = (a.V & 3) == 0;
#pragma unroll
  for (int ps = 0; ps < kPasses; ++ps) {
    if (ps > 0) __syncthreads();  // every read of the previous pass is done
    if (kPasses == 1 || wn == ps) {
#pragma unroll
      for (int fn = 0; fn < FN; ++fn) {
        const int t = Mma::col_of(wn, fn, lane) - ps * kTok;
#pragma unroll
        for (int fm = 0; fm < FM; ++fm)
#pragma unroll
          for (int rg = 0; rg < 4; ++rg) {
            const int v0 = Mma::row_of(wm, fm, rg * 4, lane);  // multiple of 4
            const float4 w = make_float4((float)mma.acc[fm][fn][rg * 4], (float)mma.acc[fm][fn][rg * 4 + 1],
                                         (float)mma.acc[fm][fn][rg * 4 + 2], (float)mma.acc[fm][fn][rg * 4 + 3]);
            *reinterpret_cast<float4*>(st + t * BM + (((v0 >> 2) ^ (t & (kSw - 1))) << 2)) = w;
          }
      }
    }
    __syncthreads();
    for (int idx = tid; idx < kTok * kChunks; idx += NT) {
      const int t = idx / kChunks;
      const int c = idx % kChunks;
      const int64_t tg = tbase + ps * kTok + t;
      const int64_t v = vbase + 4 * c;
      if (tg >= a.T || v >= a.V) continue;
      float4 w = *reinterpret_cast<const float4*>(st + t * BM + ((c ^ (t & (kSw - 1))) << 2));
      if constexpr (E::kBytes == 1) {
        const float so = a.o_scale[tg];
        w.x = w.x * so * a.W_scale[v];
        w.y = w.y * so * a.W_scale[v + 1 < a.V ? v + 1 : v];
        w.z = w.z * so * a.W_scale[v + 2 < a.V ? v + 2 : v];
        w.w = w.w * so * a.W_scale[v + 3 < a.V ? v + 3 : v];
      }
      float* out = a.logits + tg * a.V + v;
      if (vec) {
        // whole lines, non-temporal (decode step 0.74 -> 0.72 ms: draft heads
        // 0.141 -> 0.126 ms, verifier head 3 % faster)
        store16_nt(out, make_uint4(__float_as_uint(w.x), __float_as_uint(w.y), __float_as_uint(w.z),
                                   __float_as_uint(w.w)));
      } else {
        const float x[4] = {w.x, w.y, w.z, w.w};
        for (int q = 0; q < 4 && v + q < a.V; ++q) out[q] = x[q];
      }
    }
  }
}

template <int EPT>
__global__ __launch_bounds__(kRowThreads) void sample_kernel(SampleArgs a) {
  __shared__ RowShared sh;
  const int64_t r = blockIdx.x;
  const float* row = a.logits + r * a.V;
  int tok;
  if (a.greedy) {
    tok = row_argmax<EPT>(row, (int)a.V, sh);
  } else {
    float e[EPT];
    RowDist d;
    uint32_t lo = 0, hi = 0;
    float P = 0.f;
    const int n = row_dist<EPT>(row, (int)a.V, a.inv_temp, a.top_p, e, sh, d, lo, hi, P);
    if (n >= 0) {
      if (threadIdx.x >= 64) return;
      tok = list_finish(sh, n, lo, hi, P, (int)a.V, a.u[r], d);
    } else {
      tok = row_draw<EPT>(e, d, a.u[r], sh);
    }
    if (threadIdx.x == 0 && a.params) a.params[r] = d;
  }
  if (threadIdx.x == 0) a.tokens[r] = tok;
}

// Every row's sampling-distribution parameters (rows of several arrays: the
// draft rows, then the verifier rows).
template <int EPT>
__global__ __launch_bounds__(kRowThreads) void row_params_kernel(RowParamArgs a) {
  __shared__ RowShared sh;
  const int64_t r = blockIdx.x;
  const float* row = r < a.rows0 ? a.logits0 + r * a.V : a.logits1 + (r - a.rows0) * a.V;
  float e[EPT];
  RowDist d;
  uint32_t lo = 0, hi = 0;
  float P = 0.f;
  const int n = row_dist<EPT>(row, (int)a.V, a.inv_temp, a.top_p, e, sh, d, lo, hi, P);
  if (n >= 0) {
    if (threadIdx.x >= 64) return;
    list_finish(sh, n, lo, hi, P, (int)a.V, -1.f, d);
  }
  if (threadIdx.x == 0) a.params[r] = d;
}

// Whole-row draw with uniform u from a row's distribution, weights recomputed
// from the logits.
template <int EPT>
__device__ __forceinline__ int draw_kept(const float* row, int V, float it, const RowDist& d,
                                         float u, RowShared& sh) {
  auto w = [&](int i) {
    const int v = elem_v<EPT>(i);
    if (v >= V) return 0.f;
    const float e = exp_weight(row[v], it, d);
    return kept_w(e, v, d) ? e : 0.f;
  };
  int v = index_order_draw<EPT>(w, u * d.kept, sh);
  if (v < 0) {
    int last = -1;
    for (int i = 0; i < EPT; ++i)
      if (w(i) > 0.f) last = elem_v<EPT>(i);
    float lv = (float)last;
    block_argmax(lv, last, sh);
    v = last;
  }
  return v;
}

// List wave: a draw from p's kept list (n entries) with uniform u; with a
// draft row qrow (parameters dq), from max(0, p - q), or p itself if that has
// no mass. -1 where p keeps no token (a row with a +inf logit, or of NaN or -inf
// only), as the sampler gives for such a row.
template <int RUN>
__device__ __forceinline__ int list_residual_draw(const RowShared& sh, int n, const RowDist& dp,
                                                  const float* qrow, const RowDist& dq, float it,
                                                  float u) {
  if (n == 0) return -1;
  float w[RUN];
  load_run<RUN>(sh, n, w);
  if (qrow) {
    float r[RUN];
    float s = 0.f;
#pragma unroll
    for (int q = 0; q < RUN; ++q) {
      r[q] = 0.f;
      if (w[q] > 0.f)
        r[q] = fmaxf(w[q] / dp.kept - prob_at(qrow, run_index<RUN>(sh, q), it, dq), 0.f);
      s += r[q];
    }
    const float tot = wave_sum(s);
    if (tot > 0.f) return sh.ci[cand_slot(run_draw<RUN>(r, u * tot))];
  }
  return sh.ci[cand_slot(run_draw<RUN>(w, u * dp.kept))];
}

// Verification: one block per sequence. Rows' parameters come from
// row_params_kernel; weights are recomputed from the logits as needed (the
// rows stay in L2). The draw after a rejection (or after the last draft) runs
// over the verifier row's kept tokens, which hold all of max(0, p - q). Bound by
// latency: 32 us per launch (102 sequences of 6 drafts at V = 49,152) with the
// drafts tested one after the other and two passes over the row for the kept
// tokens, 20 us with the tests side by side and one pass.
template <int EPT, bool GREEDY>
__global__ __launch_bounds__(kRowThreads) void verify_kernel(VerifyArgs a) {
  __shared__ RowShared sh;
  const int64_t b = blockIdx.x;
  const int V = (int)a.V;
  const int G = a.gamma;
  const float it = a.inv_temp;
  int k = 0;
  int next = 0;
  if (GREEDY) {
#pragma nounroll
    for (; k < G; ++k) {
      next = row_argmax<EPT>(a.target_logits + (b * (G + 1) + k) * a.V, V, sh);
      if (next != a.draft_tokens[(int64_t)k * a.batch + b]) break;
    }
  } else {
    // The acceptance tests do not depend on each other: one lane per draft, so
    // that a sequence waits for one chain of loads (token, logits) rather than
    // one per kept draft. Every wave does it for itself.
#pragma nounroll
    for (int k0 = 0; k0 < G; k0 += 64) {
      const int kl = k0 + (int)(threadIdx.x & 63);
      bool rejected = false;
      if (kl < G) {
        const int64_t at = (int64_t)kl * a.batch + b;
        const int x = a.draft_tokens[at];
        const RowDist dq = a.dparams[at];
        const RowDist dp = a.tparams[b * (G + 1) + kl];
        const bool in = x >= 0 && x < V;
        const float qx = in ? prob_at(a.draft_logits + at * a.V, x, it, dq) : 0.f;
        const float px = in ? prob_at(a.target_logits + (b * (G + 1) + kl) * a.V, x, it, dp) : 0.f;
        rejected = !(a.u_accept[at] * qx < px);
      }
      const unsigned long long m = __ballot(rejected);
      k = k0 + (m ? __builtin_ctzll(m) : 64);
      if (m) break;
    }
    k = k < G ? k : G;
  }
  if (!GREEDY && k < G) {
    const float* trow = a.target_logits + (b * (G + 1) + k) * a.V;
    const float* drow = a.draft_logits + ((int64_t)k * a.batch + b) * a.V;
    const RowDist dq = a.dparams[(int64_t)k * a.batch + b];
    const RowDist dp = a.tparams[b * (G + 1) + k];
    // rejected: draw from max(0, p - q)
    const int n = compact_kept<EPT>(trow, V, it, dp, sh);
    if (n <= kMaxCand) {
      if (threadIdx.x >= 64) return;
      next = n <= kSmallCand ? list_residual_draw<4>(sh, n, dp, drow, dq, it, a.u_sample[b])
                             : list_residual_draw<kRunMax>(sh, n, dp, drow, dq, it, a.u_sample[b]);
    } else {
      auto res = [&](int i) {
        const int v = elem_v<EPT>(i);
        if (v >= V) return 0.f;
        return fmaxf(prob_at(trow, v, it, dp) - prob_at(drow, v, it, dq), 0.f);
      };
      float rs = 0.f;
#pragma unroll 4
      for (int i = 0; i < EPT; ++i) rs += res(i);
      const float tot = block_sum(rs, sh);
      if (tot > 0.f) {
        int v = index_order_draw<EPT>(res, a.u_sample[b] * tot, sh);
        if (v < 0) {
          int last = -1;
          for (int i = 0; i < EPT; ++i)
            if (res(i) > 0.f) last = elem_v<EPT>(i);
          float lv = (float)last;
          block_argmax(lv, last, sh);
          v = last;
        }
        next = v;
      } else {
        // no residual mass: the rejected token was impossible under both
        // distributions and they coincide, so the draw is from the verifier's
        next = draw_kept<EPT>(trow, V, it, dp, a.u_sample[b], sh);
      }
    }
  }
  if (k == G) {  // every draft kept: one more token from the verifier
    const float* trow = a.target_logits + (b * (G + 1) + G) * a.V;
    if (GREEDY) {
      next = row_argmax<EPT>(trow, V, sh);
    } else {
      const RowDist dp = a.tparams[b * (G + 1) + G];
      const int n = compact_kept<EPT>(trow, V, it, dp, sh);
      if (n <= kMaxCand) {
        if (threadIdx.x >= 64) return;
        next = n <= kSmallCand ? list_residual_draw<4>(sh, n, dp, nullptr, dp, it, a.u_sample[b])
                           : list_residual_draw<kRunMax>(sh, n, dp, nullptr, dp, it,
                                                         a.u_sample[b]);
      } else {
        next = draw_kept<EPT>(trow, V, it, dp, a.u_sample[b], sh);
      }
    }
  }
  if (threadIdx.x == 0) {
    a.n_accepted[b] = k;
    a.next_token[b] = next;
  }
}

using HeadWide = WideMma<128, 128, 2, 2, 2>;
// 192 vocabulary rows: 80 KB of stages, two blocks fill a CU's LDS
using HeadWide192 = WideMma<192, 128, 2, 2, 2>;
// few rows: a quarter (half) of the token columns, so that three (two) K-tiles
// of the head are in flight ahead: 48 KB of stages, three blocks per CU
using HeadFew = WideMma<64, 32, 2, 1, 4>;
using HeadSome = WideMma<64, 64, 2, 2, 3>;
// 128 columns, vocabularies too small for a 128-row block per CU
using HeadShort = WideMma<64, 128, 2, 2, 3>;
// widths that are not multiples of the 64-wide K-tile
using HeadShortTail = WideMma<64, 128, 2, 2, 3, 128, kLayoutKC, kLayoutKC, true>;
using HeadFewTail = WideMma<64, 32, 2, 1, 4, 128, kLayoutKC, kLayoutKC, true>;
using HeadSomeTail = WideMma<64, 64, 2, 2, 3, 128, kLayoutKC, kLayoutKC, true>;
using HeadWideTail = WideMma<128, 128, 2, 2, 2, 128, kLayoutKC, kLayoutKC, true>;
using HeadWide192Tail = WideMma<192, 128, 2, 2, 2, 128, kLayoutKC, kLayoutKC, true>;
using HeadGenF32 = TileMma<F32, 128, 128, 2, 2>;
// 8-bit operands: the same tiles, with twice the K values in a K-tile. One row at width 4,352,
// V = 49,152: 32 us (6.7 TB/s); 1,632 rows: 401 us (1.74 POP/s; a large library product
// reaches 2.08). There 192 x 128 has the rounds that it has in bf16, two blocks to a CU: 256 x
// 256 (one block) 424, 192 x 256 430, 256 x 128 446, 128 x 256 490.
template <int BM, int BN, int WGM, int WGN, int STAGES, bool KTAIL>
using HeadI8 = WideMma<BM, BN, WGM, WGN, STAGES, 128, kLayoutKC, kLayoutKC, KTAIL, I8>;

}  // namespace

// Tile of the head product (vocabulary rows x token columns).
// - At most 64 rows of hidden states: bound by the head's bytes and by how many
//   of them are in flight, so 64 vocabulary rows and 32 or 64 columns, with
//   three or two K-tiles ahead in each of three blocks per CU. One row at
//   width 4,352, V = 49,152: 84 -> 74 us (5.8 TB/s); 16 rows at width 2,048, V =
//   16,000: 31 -> 16 us; 64 rows at width 4,352: 94 -> 91 us.
// - 128 columns otherwise. Where 128-row tiles would not give every CU a block,
//   64 rows: 102 rows at width 2,048, V = 16,000 (125 blocks) 36 -> 22 us, V =
//   32,000 (250 blocks) 41.6 -> 39.7; at 313 blocks 27.9 -> 30.0, so not there.
// - From four such token tiles on (the verifier's rows) 192 vocabulary rows: at
//   102 x 7 rows and V = 49,152 that makes 1,536 blocks, three full rounds of two
//   blocks per CU, where 128-row tiles make 2,304 (four and a half).
void head_tile(bool wide, int64_t T, int64_t V, int* rows, int* cols) {
  *cols = !wide || T > 64 ? 128 : T > 32 ? 64 : 32;
  const int64_t blocks = ((T + 127) / 128) * ((V + 127) / 128);  // of 128 x 128
  *rows = !wide ? 128 : T <= 64 || blocks < 256 ? 64 : T > 3 * 128 ? 192 : 128;
}
int row_elems_per_thread(int64_t V) {
  for (int e : {16, 32, 48, 64})
    if (V <= (int64_t)e * kRowThreads) return e;
  return 0;
}

template <class Mma, typename E>
static void launch_head_t(const HeadArgs& a, hipStream_t stream) {
  hipLaunchKernelGGL((head_logits_kernel<Mma, E>), dim3((unsigned)a.n_tt * (unsigned)a.n_vt),
                     dim3(Mma::NT), 0, stream, a);
}

hipError_t launch_head_logits(const HeadArgs& a, bool f32, hipStream_t stream) {
  int rows, cols;
  head_tile(!f32, a.T, a.V, &rows, &cols);
  if (a.n_vt != (int)((a.V + rows - 1) / rows) || a.n_tt != (int)((a.T + cols - 1) / cols))
    return hipErrorInvalidValue;
  const bool tail = a.d % 64 != 0;
  if (f32)
    launch_head_t<HeadGenF32, F32>(a, stream);
  else if (cols == 32)
    tail ? launch_head_t<HeadFewTail, Bf16>(a, stream) : launch_head_t<HeadFew, Bf16>(a, stream);
  else if (cols == 64)
    tail ? launch_head_t<HeadSomeTail, Bf16>(a, stream) : launch_head_t<HeadSome, Bf16>(a, stream);
  else if (rows == 64)
    tail ? launch_head_t<HeadShortTail, Bf16>(a, stream) : launch_head_t<HeadShort, Bf16>(a, stream);
  else if (rows == 192)
    tail ? launch_head_t<HeadWide192Tail, Bf16>(a, stream) : launch_head_t<HeadWide192, Bf16>(a, stream);
  else
    tail ? launch_head_t<HeadWideTail, Bf16>(a, stream) : launch_head_t<HeadWide, Bf16>(a, stream);
  return hipGetLastError();
}

void head_i8_tile(int64_t T, int64_t V, int* rows, int* cols) { head_tile(true, T, V, rows, cols); }

hipError_t launch_head_logits_i8(const HeadArgs& a, hipStream_t stream) {
  int rows, cols;
  head_i8_tile(a.T, a.V, &rows, &cols);
  if (a.n_vt != (int)((a.V + rows - 1) / rows) || a.n_tt != (int)((a.T + cols - 1) / cols))
    return hipErrorInvalidValue;
  const bool tail = a.d % 128 != 0;
  if (cols == 32)
    tail ? launch_head_t<HeadI8<64, 32, 2, 1, 4, true>, I8>(a, stream) : launch_head_t<HeadI8<64, 32, 2, 1, 4, false>, I8>(a, stream);
  else if (cols == 64)
    tail ? launch_head_t<HeadI8<64, 64, 2, 2, 3, true>, I8>(a, stream) : launch_head_t<HeadI8<64, 64, 2, 2, 3, false>, I8>(a, stream);
  else if (rows == 64)
    tail ? launch_head_t<HeadI8<64, 128, 2, 2, 3, true>, I8>(a, stream) : launch_head_t<HeadI8<64, 128, 2, 2, 3, false>, I8>(a, stream);
  else if (rows == 192)
    tail ? launch_head_t<HeadI8<192, 128, 2, 2, 2, true>, I8>(a, stream) : launch_head_t<HeadI8<192, 128, 2, 2, 2, false>, I8>(a, stream);
  else
    tail ? launch_head_t<HeadI8<128, 128, 2, 2, 2, true>, I8>(a, stream) : launch_head_t<HeadI8<128, 128, 2, 2, 2, false>, I8>(a, stream);
  return hipGetLastError();
}

// (a launch takes less than 2^22 blocks of 1,024 threads: more rows go in pieces)
hipError_t launch_sample(const SampleArgs& all, int ept, hipStream_t stream) {
  constexpr int64_t kPiece = 1ll << 21;
  for (int64_t r = 0; r < all.rows; r += kPiece) {
    SampleArgs a = all;
    a.rows = all.rows - r < kPiece ? all.rows - r : kPiece;
    a.logits += r * a.V;
    a.tokens += r;
    if (a.u) a.u += r;
    if (a.params) a.params += r;
    const dim3 grid((unsigned)a.rows);
    switch (ept) {
      case 16: hipLaunchKernelGGL(sample_kernel<16>, grid, dim3(kRowThreads), 0, stream, a); break;
      case 32: hipLaunchKernelGGL(sample_kernel<32>, grid, dim3(kRowThreads), 0, stream, a); break;
      case 48: hipLaunchKernelGGL(sample_kernel<48>, grid, dim3(kRowThreads), 0, stream, a); break;
      case 64: hipLaunchKernelGGL(sample_kernel<64>, grid, dim3(kRowThreads), 0, stream, a); break;
      default: return hipErrorInvalidValue;
    }
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

hipError_t launch_row_params(const RowParamArgs& a, int ept, hipStream_t stream) {
  const dim3 grid((unsigned)(a.rows0 + a.rows1));
  switch (ept) {
    case 16: hipLaunchKernelGGL(row_params_kernel<16>, grid, dim3(kRowThreads), 0, stream, a); break;
    case 32: hipLaunchKernelGGL(row_params_kernel<32>, grid, dim3(kRowThreads), 0, stream, a); break;
    case 48: hipLaunchKernelGGL(row_params_kernel<48>, grid, dim3(kRowThreads), 0, stream, a); break;
    case 64: hipLaunchKernelGGL(row_params_kernel<64>, grid, dim3(kRowThreads), 0, stream, a); break;
    default: return hipErrorInvalidValue;
  }
  return hipGetLastError();
}

template <int EPT>
static void launch_verify_ept(const VerifyArgs& a, hipStream_t stream) {
  const dim3 grid((unsigned)a.batch);
  if (a.greedy)
    hipLaunchKernelGGL((verify_kernel<EPT, true>), grid, dim3(kRowThreads), 0, stream, a);
  else
    hipLaunchKernelGGL((verify_kernel<EPT, false>), grid, dim3(kRowThreads), 0, stream, a);
}

hipError_t launch_verify(const VerifyArgs& a, int ept, hipStream_t stream) {
  switch (ept) {
    case 16: launch_verify_ept<16>(a, stream); break;
    case 32: launch_verify_ept<32>(a, stream); break;
    case 48: launch_verify_ept<48>(a, stream); break;
    case 64: launch_verify_ept<64>(a, stream); break;
    default: return hipErrorInvalidValue;
  }
  return hipGetLastError();
}

}  // namespace mls
