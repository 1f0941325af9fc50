// Verification of a tree of drafted tokens (paper section 2, paragraph "Speculative
// Decoding", which verifies a chain; a tree holds several continuations, and one pass of
// the verifier scores them all).
//
// From the root down, at node c with p_1 the verifier's sampling distribution there and
// q the draft's: child x of c, in node order, is taken when u q(x) < p_j(x); otherwise
// p_{j+1} is max(0, p_j - q) over its mass, and the next child is tried. When none is
// left, the next token is drawn from what p has become. With children drawn from q one by
// one this leaves the verifier's distribution as it is. Without a draft's distribution q
// is all on the child: u < p_j(x), and p_{j+1} is p_j without x. Greedy: a child that is
// the verifier's argmax.
//
// A child's index is above its parent's, so one pass over the nodes in order, each tested
// if its parent is where the walk stands, is the whole walk.
//
// Which tokens a distribution keeps (top_p) is in its row's record, in float32; the
// probabilities of kept tokens, their differences and the draws are in 64 bits, so that a
// token is decided by the numbers given and not by roundings along the way.
#include <math.h>

#include "mls_device.h"
#include "mls_launch.h"
#include "mls_wave.h"

namespace mls {

namespace {

constexpr int kTreeThreads = 1024;
constexpr int kTreeWaves = kTreeThreads / 64;
constexpr int kMaxNodes = 64;
constexpr int kMaxSlabs = 64;  // of kTreeThreads tokens: rows of up to 65,536

struct TreeShared {
  double red[kTreeWaves];
  double seg[kMaxSlabs * kTreeWaves];
  float fval[kTreeWaves];
  int ival[kTreeWaves];
  int pick;
  double before;
  int32_t token[kMaxNodes];
  int32_t parent[kMaxNodes];
  float u[kMaxNodes];
};

__device__ __forceinline__ double block_sum(double v, TreeShared& sh) {
  v = wave_sum(v);
  if ((threadIdx.x & 63) == 0) sh.red[threadIdx.x >> 6] = v;
  __syncthreads();
  double s = 0.0;
#pragma unroll
  for (int i = 0; i < kTreeWaves; ++i) s += sh.red[i];
  __syncthreads();
  return s;
}

// One row's sampling distribution.
struct Row {
  const float* logits;
  RowDist d;
  double norm;  // 1 / (sum of kept weights); 0: the row keeps no token
};

// Whether the record keeps token v: by the float32 weight, formed as the record's was.
__device__ __forceinline__ bool kept(const Row& r, float logit, int v, float inv_temp) {
#pragma clang fp contract(off)
  const float scaled = logit * inv_temp;
  const float e = fast_exp2((scaled - r.d.m) * kLog2e);
  return e > r.d.theta || (e == r.d.theta && e > 0.f && v <= r.d.tie_cut);
}
__device__ __forceinline__ double weight(const Row& r, float logit, double temperature) {
  return exp((double)logit / temperature - (double)r.d.m);
}
__device__ __forceinline__ double prob(const Row& r, int v, const TreeVerifyArgs& a) {
  if (r.norm == 0.0) return 0.0;
  const float l = r.logits[v];
  return kept(r, l, v, a.inv_temp) ? weight(r, l, (double)a.temperature) * r.norm : 0.0;
}

__device__ __forceinline__ Row open_row(const float* logits, const RowDist* d, const TreeVerifyArgs& a,
                                        TreeShared& sh) {
  Row r;
  r.logits = logits;
  r.d = *d;
  double s = 0.0;
  for (int v = threadIdx.x; v < a.V; v += kTreeThreads) {
    const float l = logits[v];
    if (kept(r, l, v, a.inv_temp)) s += weight(r, l, (double)a.temperature);
  }
  s = block_sum(s, sh);
  r.norm = s > 0.0 && s < INFINITY ? 1.0 / s : 0.0;
  return r;
}

// Argmax with the lowest index on ties; -1 without a logit above -inf.
__device__ __forceinline__ int row_argmax(const float* logits, int V, TreeShared& sh) {
  float best = -INFINITY;
  int at = 0x7fffffff;
  for (int v = threadIdx.x; v < V; v += kTreeThreads) {
    const float l = logits[v];
    if (l > best) {
      best = l;
      at = v;
    }
  }
  wave_argmax(best, at);
  const int w = threadIdx.x >> 6;
  if ((threadIdx.x & 63) == 0) {
    sh.fval[w] = best;
    sh.ival[w] = at;
  }
  __syncthreads();
  best = sh.fval[0];
  at = sh.ival[0];
  for (int i = 1; i < kTreeWaves; ++i)
    if (argmax_better(sh.fval[i], sh.ival[i], best, at)) {
      best = sh.fval[i];
      at = sh.ival[i];
    }
  __syncthreads();
  return at == 0x7fffffff ? -1 : at;
}

// Smallest index whose cumulative weight in index order exceeds `target`; the last index
// of positive weight where rounding leaves the target at the sum; -1 without any.
template <class Wt>
__device__ __forceinline__ int draw_index(Wt wt, int V, double u, TreeShared& sh) {
  const int wave = threadIdx.x >> 6;
  const int lane = threadIdx.x & 63;
  const int slabs = (V + kTreeThreads - 1) / kTreeThreads;
  for (int s = 0; s < slabs; ++s) {
    const int v = s * kTreeThreads + (int)threadIdx.x;
    const double w = v < V ? wt(v) : 0.0;
    double t = 0.0;
    if (__ballot(w > 0.0) != 0) t = wave_sum(w);
    if (lane == 0) sh.seg[s * kTreeWaves + wave] = t;
  }
  if (threadIdx.x == 0) sh.pick = -1;
  __syncthreads();
  if (wave == 0) {
    // each lane owns a run of segments, in index order
    const int n = slabs * kTreeWaves;
    const int per = (n + 63) / 64;
    double run = 0.0;
    for (int k = 0; k < per; ++k)
      if (lane * per + k < n) run += sh.seg[lane * per + k];
    const double incl = wave_incl_scan(run);
    const double target = u * lane_read(incl, 63);
    double before = incl - run;
    int found = -1;
    int last = -1;
    double found_before = 0.0, last_before = 0.0;
    for (int k = 0; k < per; ++k) {
      const int i = lane * per + k;
      const double s = i < n ? sh.seg[i] : 0.0;
      if (s > 0.0) {
        last = i;
        last_before = before;
        if (found < 0 && before + s > target) {
          found = i;
          found_before = before;
        }
      }
      before += s;
    }
    const unsigned long long hit = __ballot(found >= 0);
    const unsigned long long some = __ballot(last >= 0);
    if (hit) {
      if (lane == __builtin_ctzll(hit)) {
        sh.pick = found;
        sh.before = found_before - target;
      }
    } else if (some) {
      if (lane == 63 - __builtin_clzll(some)) {
        sh.pick = last;
        sh.before = last_before - target;
      }
    }
  }
  __syncthreads();
  const int seg = sh.pick;
  const double ahead = sh.before;  // what comes before the segment, less the target
  __syncthreads();
  if (seg < 0) return -1;
  if (wave == seg % kTreeWaves) {
    const int v = (seg / kTreeWaves) * kTreeThreads + (int)threadIdx.x;
    const double w = v < V ? wt(v) : 0.0;
    const double incl = wave_incl_scan(w);
    const unsigned long long m = __ballot(w > 0.0 && ahead + incl > 0.0);
    const unsigned long long pos = __ballot(w > 0.0);
    const int l = m ? __builtin_ctzll(m) : 63 - __builtin_clzll(pos);
    if (lane == 0) sh.pick = (seg / kTreeWaves) * kTreeThreads + wave * 64 + l;
  }
  __syncthreads();
  const int v = sh.pick;
  __syncthreads();
  return v;
}

template <bool GREEDY>
__global__ __launch_bounds__(kTreeThreads) void tree_verify_kernel(TreeVerifyArgs a) {
  __shared__ TreeShared sh;
  __shared__ double scale[kMaxNodes];
  __shared__ int32_t gone[kMaxNodes];
  const int64_t b = blockIdx.x;
  const int64_t row0 = b * a.n;
  if ((int)threadIdx.x < a.n) {
    const int64_t i = row0 + threadIdx.x;
    sh.token[threadIdx.x] = threadIdx.x > 0 ? a.tokens[i] : -1;
    sh.parent[threadIdx.x] = a.parents ? a.parents[i] : (int)threadIdx.x - 1;
    sh.u[threadIdx.x] = GREEDY || threadIdx.x == 0 ? 0.f : a.u_accept[i];
    a.path[i] = threadIdx.x == 0 ? 0 : -1;
  }
  __syncthreads();
  int cur = 0;
  int depth = 0;
  int rejected = 0;
  Row p, q;
  q.norm = 0.0;
  int best = -1;
  auto open = [&]() {
    const float* t = a.target + (row0 + cur) * a.V;
    rejected = 0;
    if (GREEDY) {
      best = row_argmax(t, a.V, sh);
    } else {
      p = open_row(t, a.tparams + row0 + cur, a, sh);
      q.norm = -1.0;  // opened when a child asks for it
    }
  };
  // p after the children turned down so far, at token v
  auto left = [&](int v) {
    double r = prob(p, v, a);
    if (r == 0.0) return 0.0;
    if (a.draft) {
      if (rejected == 0) return r;
      const double qv = prob(q, v, a);
      for (int j = 0; j < rejected; ++j)
        if (scale[j] != 0.0) r = fmax(r - qv, 0.0) * scale[j];
      return r;
    }
    for (int j = 0; j < rejected; ++j)
      if (gone[j] == v) return 0.0;
    return rejected == 0 ? r : r * scale[rejected - 1];
  };
  open();
#pragma nounroll
  for (int i = 1; i < a.n; ++i) {
    if (sh.parent[i] != cur) continue;
    const int x = sh.token[i];
    const bool in = x >= 0 && x < a.V;
    bool take;
    if (GREEDY) {
      take = in && x == best;
    } else {
      if (a.draft && q.norm < 0.0) q = open_row(a.draft + (row0 + cur) * a.V, a.dparams + row0 + cur, a, sh);
      const double px = in ? left(x) : 0.0;
      const double qx = !a.draft ? 1.0 : in ? prob(q, x, a) : 0.0;
      take = (double)sh.u[i] * qx < px;
      if (!take) {
        // the mass that is left, and 1 over it
        double s = 0.0;
        if (a.draft) {
          for (int v = threadIdx.x; v < a.V; v += kTreeThreads) {
            const double r = left(v);
            if (r > 0.0) s += fmax(r - prob(q, v, a), 0.0);
          }
        } else {
          for (int v = threadIdx.x; v < a.V; v += kTreeThreads)
            if (v != x) {
              bool was = false;
              for (int j = 0; j < rejected; ++j) was = was || gone[j] == v;
              if (!was) s += prob(p, v, a);
            }
        }
        s = block_sum(s, sh);
        // (no mass left: p stays as it was)
        if (a.draft || s > 0.0) {
          if (threadIdx.x == 0) {
            scale[rejected] = s > 0.0 ? 1.0 / s : 0.0;
            gone[rejected] = x;
          }
          ++rejected;
        }
        __syncthreads();
      }
    }
    if (take) {
      cur = i;
      ++depth;
      if (threadIdx.x == 0) a.path[row0 + depth] = i;
      open();
    }
  }
  int next;
  if (GREEDY)
    next = best;
  else
    next = draw_index(left, a.V, (double)a.u_sample[b], sh);
  if (threadIdx.x == 0) {
    a.n_accepted[b] = depth;
    a.next_token[b] = next;
  }
}

}  // namespace

hipError_t launch_tree_verify(const TreeVerifyArgs& a, hipStream_t stream) {
  const dim3 grid((unsigned)a.batch);
  if (a.greedy)
    hipLaunchKernelGGL(tree_verify_kernel<true>, grid, dim3(kTreeThreads), 0, stream, a);
  else
    hipLaunchKernelGGL(tree_verify_kernel<false>, grid, dim3(kTreeThreads), 0, stream, a);
  return hipGetLastError();
}

}  // namespace mls
