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
//
// A distribution that keeps up to kMaxCand tokens is opened once into a list, one token
// to a thread, in index order: what becomes of p at that node, children turned down and
// the draw, then takes place in registers and a few barriers, and reads q at the listed
// tokens only. Opening a row is nearly all the time (its load, its threshold, a few
// dependent steps on one CU), so the rows of each tree's first nodes are opened
// beforehand, side by side, and left in the workspace (tree_rows_kernel); rows that the
// walk reaches beyond them it opens itself. Larger distributions (top_p = 1, flat rows) have
// their list in the workspace, with what is left of p and q at each of its tokens.
#include <math.h>

#include "mls_device.h"
#include "mls_launch.h"
#include "mls_rowdist.h"
#include "mls_wave.h"

namespace mls {

namespace {

constexpr int kTreeThreads = kRowThreads;
constexpr int kTreeWaves = kTreeThreads / 64;
constexpr int kMaxNodes = 64;
constexpr int kAhead = 8;      // entries of a large list that a thread has in flight
constexpr int kMaxSlabs = 64;  // of kTreeThreads tokens: rows of up to 65,536
static_assert(kMaxCand <= kTreeThreads, "a thread owns at most one token of a list");

// An opened row in the workspace; its list is idx[kMaxCand], p[kMaxCand].
struct TreeRow {
  RowDist d;
  int32_t n;    // tokens of its list; -1: none, the row keeps more
  double norm;  // 1 / (sum of kept weights); 0: the row keeps no token
  double top;
};

struct Row {
  const float* logits;
  RowDist d;
  double norm;
  double top;
};

// How rows are sampled.
struct Settings {
  int V;
  float inv_temp;     // the record's
  double inv_temp64;  // the probabilities'
  float top_p;
};

// What opening a row takes.
struct OpenShared {
  RowShared row;
  double red[kTreeWaves];
  RowDist d;
};

struct TreeShared {
  Row row[2];  // the present node's: the verifier's, the draft's
  double red[2][kTreeWaves];
  double seg[kMaxSlabs * kTreeWaves];
  double scale[kMaxNodes];
  int32_t gone[kMaxNodes];
  int pick;
  double before;
  double at[kMaxNodes][2];  // what is left of p, and q, at each node's token
  int32_t token[kMaxNodes];
  int32_t parent[kMaxNodes];
  float u[kMaxNodes];
};

__device__ __forceinline__ double block_sum(double v, double* red) {
  v = wave_sum(v);
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
  __syncthreads();
  double s = 0.0;
#pragma unroll
  for (int i = 0; i < kTreeWaves; ++i) s += red[i];
  return s;
}
// (two buffers in turn: the next sum's writes do not meet this one's reads)
__device__ __forceinline__ double block_sum(double v, TreeShared& ts, int& turn) {
  turn ^= 1;
  return block_sum(v, ts.red[turn]);
}

// exp(logit / temperature - top) of a kept token, 2e-14 off at most: with t the integer next
// to y / ln 2, 2^t times the exponential's series at y - t ln 2, whose first term left out
// is 0.35^12 / 12!. A few of these per token are most of the arithmetic (the library's
// exp and the division are three times as many operations). (kMostLog: see top_of.)
constexpr double kMostLog = 600.0;
__device__ __forceinline__ double weight(double top, float logit, double inv_temp) {
  const double y = fmin(fma((double)logit, inv_temp, -top), kMostLog);
  const double t = rint(y * 1.4426950408889634074);
  const double f = fma(t, -0.69314718055994530942, y);
  double e = 1.0 / 39916800.0;
  e = fma(e, f, 1.0 / 3628800.0);
  e = fma(e, f, 1.0 / 362880.0);
  e = fma(e, f, 1.0 / 40320.0);
  e = fma(e, f, 1.0 / 5040.0);
  e = fma(e, f, 1.0 / 720.0);
  e = fma(e, f, 1.0 / 120.0);
  e = fma(e, f, 1.0 / 24.0);
  e = fma(e, f, 1.0 / 6.0);
  e = fma(e, f, 0.5);
  e = fma(e, f, 1.0);
  e = fma(e, f, 1.0);
  return ldexp(e, (int)t);
}
__device__ __forceinline__ double prob_of(const Row& r, float logit, int v, const Settings& a) {
  if (r.norm == 0.0 || !kept_w(exp_weight(logit, a.inv_temp, r.d), v, r.d)) return 0.0;
  return weight(r.top, logit, a.inv_temp64) * r.norm;
}
__device__ __forceinline__ double prob(const Row& r, int v, const Settings& a) {
  return prob_of(r, r.logits[v], v, a);
}

// max(0, p - q) of a token. Where both are the same number, formed on two ways (weights 2e-14 off, sums
// in another order, a fused multiply-add), it is none: rows that are alike have nothing left, and
// no distribution of roundings.
__device__ __forceinline__ double left_of(double p, double q) {
  const double d = p - q;
  return d > p * 0x1p-42 ? d : 0.0;
}

// Calls f(logit, v, in) for the wave's range of the row, 64 tokens after 64 in index order,
// kAhead loads in flight.
template <class F>
__device__ __forceinline__ void for_wave_range(const float* logits, int V, F f) {
  const int per = ((V + kTreeThreads - 1) / kTreeThreads) * 64;  // tokens of a wave
  const int first = (threadIdx.x >> 6) * per + (threadIdx.x & 63);
#pragma nounroll
  for (int i0 = 0; i0 < per; i0 += 64 * kAhead) {
    float l[kAhead];
#pragma unroll
    for (int u = 0; u < kAhead; ++u) {
      const int v = first + i0 + 64 * u;
      l[u] = logits[v < V && i0 + 64 * u < per ? v : 0];
    }
#pragma unroll
    for (int u = 0; u < kAhead; ++u) {
      const int v = first + i0 + 64 * u;
      f(l[u], v, v < V && i0 + 64 * u < per);
    }
  }
}

// A row as a thread knows it: its distribution, and where it keeps few enough tokens the
// list, whose entry i < n is thread i's (idx, p normalised; p is 0 for an entry that is not
// kept); n is -1 for larger ones.
struct Opened {
  RowDist d;
  double norm;
  double top;
  int n;
  int idx;
  double p;
};

// What a row's weights are relative to: its record's maximum, a float32 product. What that is off
// by is a factor that all weights share, and norm takes out. Far from 0 this factor, e to the
// 2^-23 of the maximum, would leave the numbers there are: there it is the largest logit's
// product in 64 bits, from below. Where even that is more than e^kMostLog off (the maximum past
// 2^60), the largest weights are kMostLog's, and neighbouring logits' are 0 beside them.
constexpr float kFarTop = 16777216.f;
__device__ __forceinline__ double top_of(const float* logits, const RowDist& d, const Settings& a, double* red) {
  if (!(fabsf(d.m) > kFarTop)) return (double)d.m;
  float x = -INFINITY;
  for_wave_range(logits, a.V, [&](float l, int, bool in) { x = in ? fmaxf(x, l) : x; });
  x = wave_max(x);
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = (double)x;
  __syncthreads();
  double m = red[0];
#pragma unroll
  for (int i = 1; i < kTreeWaves; ++i) m = fmax(m, red[i]);
  __syncthreads();  // (the caller sums there next)
  m *= a.inv_temp64;
  return m - fabs(m) * 0x1p-52;
}

// Opens a row, its record given or found. Larger ones' weights are summed where `sum` asks
// for it. All threads call it.
template <int EPT>
__device__ __forceinline__ Opened open_row(const float* logits, const RowDist* rec, const Settings& a, bool sum,
                                           OpenShared& os) {
  Opened r;
  RowShared& sh = os.row;
  __syncthreads();  // the list of the last row has been read
  int n;
  if (rec) {
    r.d = *rec;
    n = compact_kept<EPT>(logits, a.V, a.inv_temp, r.d, sh);
  } else {
    float e[EPT];
    uint32_t lo = 0, hi = 0;
    float P = 0.f;
    n = row_dist<EPT>(logits, a.V, a.inv_temp, a.top_p, e, sh, r.d, lo, hi, P);
    if (n >= 0) {
      if (threadIdx.x < 64) {
        list_finish(sh, n, lo, hi, P, a.V, -1.f, r.d);
        if (threadIdx.x == 0) os.d = r.d;
      }
      __syncthreads();
      r.d = os.d;
    } else {
      n = kMaxCand + 1;
    }
  }
  r.top = top_of(logits, r.d, a, os.red);
  r.n = n <= kMaxCand ? n : -1;
  r.idx = -1;
  r.p = 0.0;
  double s = 0.0;
  if (r.n >= 0) {
    if ((int)threadIdx.x < n) {
      r.idx = sh.ci[cand_slot(threadIdx.x)];
      if (kept_w(sh.cw[cand_slot(threadIdx.x)], r.idx, r.d)) r.p = weight(r.top, logits[r.idx], a.inv_temp64);
    }
    s = r.p;
  } else if (sum) {
    for_wave_range(logits, a.V, [&](float l, int v, bool in) {
      const bool k = in && kept_w(exp_weight(l, a.inv_temp, r.d), v, r.d);
      if (__ballot(k) != 0 && k) s += weight(r.top, l, a.inv_temp64);
    });
  }
  s = block_sum(s, os.red);
  r.norm = s > 0.0 && s < INFINITY ? 1.0 / s : 0.0;
  r.p *= r.norm;
  return r;
}

// The same from within the walk: a function of its own, so that a row's elements, which
// take all of a thread's registers, do not share them with the walk's state.
template <int EPT>
__device__ __noinline__ Opened open_far(const float* logits, const RowDist* rec, Settings a, bool sum) {
  __shared__ OpenShared os;
  return open_row<EPT>(logits, rec, a, sum, os);
}

// The list of a row that keeps more than a thread's one token each: tokens in index order
// and their weights, in the workspace; their number, and 1 / (sum of the weights) in r.norm.
// Each wave counts and then places the tokens of its own range of the row.
__device__ __forceinline__ int open_large(const Settings& a, TreeShared& ts, int& turn, Row& r, int32_t* li,
                                          double* lr) {
  const int wave = threadIdx.x >> 6;
  int count = 0;
  for_wave_range(r.logits, a.V, [&](float l, int v, bool in) {
    count += __builtin_popcountll(__ballot(in && kept_w(exp_weight(l, a.inv_temp, r.d), v, r.d)));
  });
  __syncthreads();  // (ts.gone has been read)
  if ((threadIdx.x & 63) == 0) ts.gone[wave] = count;
  __syncthreads();
  int at = 0, n = 0;
#pragma unroll
  for (int w = 0; w < kTreeWaves; ++w) {
    if (w == wave) at = n;
    n += ts.gone[w];
  }
  double s = 0.0;
  for_wave_range(r.logits, a.V, [&](float l, int v, bool in) {
    const bool k = in && kept_w(exp_weight(l, a.inv_temp, r.d), v, r.d);
    const unsigned long long m = __ballot(k);
    if (m == 0) return;
    if (k) {
      const int pos = at + lanes_below(m);
      const double w = weight(r.top, l, a.inv_temp64);
      li[pos] = v;
      lr[pos] = w;
      s += w;
    }
    at += __builtin_popcountll(m);
  });
  s = block_sum(s, ts, turn);  // (and its barrier shows the block the list)
  r.norm = s > 0.0 && s < INFINITY ? 1.0 / s : 0.0;
  return r.norm == 0.0 ? 0 : n;
}

// Opens a row of one of the `ready` first nodes of each tree: the verifier's of every node
// that the tree has (with its list), then the draft's of those that have a child (its record
// and norm; the walk reads q at p's tokens only).
template <int EPT>
__global__ __launch_bounds__(kTreeThreads) void tree_rows_kernel(TreeVerifyArgs a) {
  __shared__ OpenShared os;
  const int64_t row = blockIdx.x;  // [verifier, draft][batch][ready]
  const int64_t half = a.batch * a.ready;
  const bool draft = row >= half;
  const int64_t in = draft ? row - half : row;
  const int64_t b = in / a.ready;
  const int i = (int)(in - b * a.ready);
  const int lane = threadIdx.x & 63;
  // (every wave asks for itself)
  const int parent = lane < a.n ? (a.parents ? a.parents[b * a.n + lane] : lane - 1) : -1;
  if (draft && __ballot(lane < a.n && lane > i && parent == i) == 0) return;
  const int up = __builtin_amdgcn_readlane(parent, i);
  if (i > 0 && (up < 0 || up >= i)) return;
  const int64_t at = b * a.n + i;
  const RowDist* rec = draft && a.dparams ? a.dparams + at : nullptr;
  const Settings set{a.V, a.inv_temp, 1.0 / (double)a.temperature, a.top_p};
  const Opened r = open_row<EPT>((draft ? a.draft : a.target) + at * a.V, rec, set, draft, os);
  if (!draft && (int)threadIdx.x < r.n) {
    a.list_idx[row * kMaxCand + threadIdx.x] = r.idx;
    a.list_p[row * kMaxCand + threadIdx.x] = r.p;
  }
  if (threadIdx.x == 0) {
    TreeRow t;
    t.d = r.d;
    t.n = r.n;
    t.norm = r.norm;
    t.top = r.top;
    static_cast<TreeRow*>(a.ready_rows)[row] = t;
  }
}

// Smallest index whose cumulative weight in index order exceeds u times the sum; the last
// index of positive weight where rounding leaves the target at the sum; -1 without any.
template <class Wt>
__device__ __forceinline__ int draw_index(Wt wt, int V, double u, TreeShared& ts) {
  const int wave = threadIdx.x >> 6;
  const int lane = threadIdx.x & 63;
  const int slabs = (V + kTreeThreads - 1) / kTreeThreads;
  __syncthreads();
  for (int s = 0; s < slabs; ++s) {
    const int v = s * kTreeThreads + (int)threadIdx.x;
    const double w = v < V ? wt(v) : 0.0;
    double t = 0.0;
    if (__ballot(w > 0.0) != 0) t = wave_sum(w);
    if (lane == 0) ts.seg[s * kTreeWaves + wave] = t;
  }
  if (threadIdx.x == 0) ts.pick = -1;
  __syncthreads();
  if (wave == 0) {
    // each lane owns a run of segments, in index order
    const int n = slabs * kTreeWaves;
    const int per = (n + 63) / 64;
    double run = 0.0;
    for (int k = 0; k < per; ++k)
      if (lane * per + k < n) run += ts.seg[lane * per + k];
    const double incl = wave_incl_scan(run);
    const double target = u * lane_read(incl, 63);
    double before = incl - run;
    int found = -1;
    int last = -1;
    double found_before = 0.0, last_before = 0.0;
    for (int k = 0; k < per; ++k) {
      const int i = lane * per + k;
      const double s = i < n ? ts.seg[i] : 0.0;
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
        ts.pick = found;
        ts.before = found_before - target;
      }
    } else if (some) {
      if (lane == 63 - __builtin_clzll(some)) {
        ts.pick = last;
        ts.before = last_before - target;
      }
    }
  }
  __syncthreads();
  const int seg = ts.pick;
  const double ahead = ts.before;  // what comes before the segment, less the target
  __syncthreads();
  if (seg < 0) return -1;
  if (wave == seg % kTreeWaves) {
    const int v = (seg / kTreeWaves) * kTreeThreads + (int)threadIdx.x;
    const double w = v < V ? wt(v) : 0.0;
    const double incl = wave_incl_scan(w);
    const unsigned long long m = __ballot(w > 0.0 && ahead + incl > 0.0);
    const unsigned long long pos = __ballot(w > 0.0);
    const int l = m ? __builtin_ctzll(m) : 63 - __builtin_clzll(pos);
    if (lane == 0) ts.pick = (seg / kTreeWaves) * kTreeThreads + wave * 64 + l;
  }
  __syncthreads();
  return ts.pick;
}

// The same over a list, thread i its entry i.
__device__ __forceinline__ int draw_list(int idx, double w, double u, TreeShared& ts) {
  const int wave = threadIdx.x >> 6;
  const int lane = threadIdx.x & 63;
  const double incl = wave_incl_scan(w);
  __syncthreads();
  if (lane == 63) ts.seg[wave] = incl;
  if (threadIdx.x == 0) ts.pick = -1;
  __syncthreads();
  double before = 0.0, total = 0.0;
#pragma unroll
  for (int i = 0; i < kTreeWaves; ++i) {
    if (i == wave) before = total;
    total += ts.seg[i];
  }
  const double target = u * total;
  const unsigned long long hit = __ballot(w > 0.0 && before + incl > target);
  const unsigned long long some = __ballot(w > 0.0);
  // each wave's first entry past the target, or its last one of all
  if (lane == 0) {
    ts.gone[wave] = hit ? wave * 64 + __builtin_ctzll(hit) : -1;
    ts.gone[kTreeWaves + wave] = some ? wave * 64 + 63 - __builtin_clzll(some) : -1;
  }
  __syncthreads();
  int pick = -1;
  for (int i = kTreeWaves - 1; i >= 0; --i) pick = ts.gone[i] >= 0 ? ts.gone[i] : pick;
  if (pick < 0)
    for (int i = 0; i < kTreeWaves; ++i) pick = ts.gone[kTreeWaves + i] >= 0 ? ts.gone[kTreeWaves + i] : pick;
  if (pick >= 0 && (int)threadIdx.x == pick) ts.pick = idx;
  __syncthreads();
  return ts.pick;
}

template <int EPT, bool GREEDY>
__global__ __launch_bounds__(kTreeThreads) void tree_verify_kernel(TreeVerifyArgs a) {
  __shared__ TreeShared ts;
  const Settings set{a.V, a.inv_temp, 1.0 / (double)a.temperature, a.top_p};
  const int64_t b = blockIdx.x;
  const int64_t row0 = b * a.n;
  if ((int)threadIdx.x < a.n) {
    const int64_t i = row0 + threadIdx.x;
    ts.token[threadIdx.x] = threadIdx.x > 0 ? a.tokens[i] : -1;
    ts.parent[threadIdx.x] = a.parents ? a.parents[i] : (int)threadIdx.x - 1;
    ts.u[threadIdx.x] = GREEDY || threadIdx.x == 0 ? 0.f : a.u_accept[i];
    ts.at[threadIdx.x][0] = ts.at[threadIdx.x][1] = 0.0;
    a.path[i] = threadIdx.x == 0 ? 0 : -1;
  }
  __syncthreads();
  int turn = 0;
  int cur = 0;
  int depth = 0;
  int rejected = 0;
  int best = -1;
  // the present node: with a list (n >= 0) the thread's token of it, what
  // has become of its probability, and q there
  const Row& p = ts.row[0];
  const Row& q = ts.row[1];
  bool q_open = false;
  int n = 0;
  int idx = -1;
  double r = 0.0, qi = 0.0;
  // A larger list: N tokens, what is left of p at each over `over`, and q there.
  const int64_t large = b * a.V;
  int32_t* const li = a.large_idx + large;
  double* lr = a.large_p + large;
  double* lr2 = a.large_p2 + large;
  double* const lq = a.large_q + large;
  int N = 0;
  double over = 0.0;
  // What the children turned down so far have left of p at token v, from the rows.
  auto left = [&](int v) {
    double x = prob(p, v, set);
    if (x == 0.0 || rejected == 0) return x;
    if (a.draft) {
      const double qv = prob(q, v, set);
      for (int j = 0; j < rejected; ++j) x = left_of(x, qv) * ts.scale[j];
      return x;
    }
    // (each factor is 1 over the mass left of the step before, which the last one alone is not; in
    // the list's order, so that a token has the same bits here and there)
    for (int j = 0; j < rejected; ++j) {
      if (ts.gone[j] == v) return 0.0;
      x *= ts.scale[j];
    }
    return x;
  };
  bool want_q = false;  // the row to open next: the draft's at this node, or the verifier's at a new one
  int i = 1;
  for (;;) {
    const float* logits = (want_q ? a.draft : a.target) + (row0 + cur) * a.V;
    if constexpr (GREEDY) {
      __shared__ RowShared sh;
      best = row_argmax<EPT>(logits, a.V, sh);
    } else {
      Row x;
      int xn, xi;
      double xp;
      if (cur < a.ready) {
        const int64_t at = (want_q ? a.batch * a.ready : 0) + b * a.ready + cur;
        const TreeRow t = static_cast<const TreeRow*>(a.ready_rows)[at];
        x.logits = logits;
        x.d = t.d;
        x.norm = t.norm;
        x.top = t.top;
        xn = t.n;
        const bool in = !want_q && (int)threadIdx.x < xn;
        xi = in ? a.list_idx[at * kMaxCand + threadIdx.x] : -1;
        xp = in ? a.list_p[at * kMaxCand + threadIdx.x] : 0.0;
      } else {
        const Opened o = open_far<EPT>(logits, want_q && a.dparams ? a.dparams + row0 + cur : nullptr, set, want_q);
        x.logits = logits;
        x.d = o.d;
        x.norm = o.norm;
        x.top = o.top;
        xn = o.n;
        xi = o.idx;
        xp = o.p;
      }
      if (!want_q && xn < 0) {
        N = open_large(set, ts, turn, x, li, lr);
        over = x.norm;
      }
      __syncthreads();  // nothing reads the row that leaves
      if (threadIdx.x == 0) ts.row[want_q ? 1 : 0] = x;
      __syncthreads();
      if (want_q) {
        q_open = true;
        if (n >= 0) {
          qi = idx >= 0 ? prob(q, idx, set) : 0.0;
        } else {
#pragma nounroll
          for (int k0 = threadIdx.x; k0 < N; k0 += kTreeThreads * kAhead) {
            int v[kAhead];
            float l[kAhead];
#pragma unroll
            for (int u = 0; u < kAhead; ++u) {
              const int k = k0 + u * kTreeThreads;
              v[u] = li[k < N ? k : 0];
            }
#pragma unroll
            for (int u = 0; u < kAhead; ++u) l[u] = x.logits[v[u]];
#pragma unroll
            for (int u = 0; u < kAhead; ++u) {
              const int k = k0 + u * kTreeThreads;
              if (k < N) lq[k] = prob_of(x, l[u], v[u], set);
            }
          }
        }
      } else {
        n = xn;
        idx = xi;
        r = xp;
        q_open = false;
        rejected = 0;
      }
    }
    want_q = false;
    bool take = false;
#pragma nounroll
    for (; i < a.n; ++i) {
      if (ts.parent[i] != cur) continue;
      const int x = ts.token[i];
      const bool in = x >= 0 && x < a.V;
      if (GREEDY) {
        take = in && x == best;
        if (take) break;
        continue;
      }
      if (a.draft && !q_open) {
        want_q = true;
        break;
      }
      double px, qx;
      if (n >= 0) {
        // from the thread that holds x, if any (a token that p does not keep is not taken)
        if (idx == x && in) {
          ts.at[i][0] = r;
          ts.at[i][1] = qi;
        }
        __syncthreads();
        px = ts.at[i][0];
        qx = a.draft ? ts.at[i][1] : 1.0;
      } else {
        px = in ? left(x) : 0.0;
        qx = !a.draft ? 1.0 : in ? prob(q, x, set) : 0.0;
      }
      take = (double)ts.u[i] * qx < px;
      if (take) break;
      // what is left of p, over its mass (no mass left: p stays as it was)
      double s = 0.0;
      if (n >= 0) {
        const double w = a.draft ? left_of(r, qi) : idx == x ? 0.0 : r;
        s = block_sum(w, ts, turn);
        if (s > 0.0) r = w * (1.0 / s);
      } else {
        // (a thread reads and writes its own entries)
#pragma nounroll
        for (int k0 = threadIdx.x; k0 < N; k0 += kTreeThreads * kAhead) {
          double w[kAhead], qw[kAhead];
          int v[kAhead];
#pragma unroll
          for (int u = 0; u < kAhead; ++u) {
            const int k = k0 + u * kTreeThreads;
            w[u] = lr[k < N ? k : 0];
            qw[u] = a.draft ? lq[k < N ? k : 0] : 0.0;
            v[u] = a.draft ? 0 : li[k < N ? k : 0];
          }
#pragma unroll
          for (int u = 0; u < kAhead; ++u) {
            const int k = k0 + u * kTreeThreads;
            const double y = a.draft ? left_of(w[u] * over, qw[u]) : v[u] == x ? 0.0 : w[u] * over;
            if (k < N) {
              s += y;
              lr2[k] = y;
            }
          }
        }
        s = block_sum(s, ts, turn);
        if (s > 0.0) {
          double* const t = lr;
          lr = lr2;
          lr2 = t;
          over = 1.0 / s;
          if (threadIdx.x == 0) {
            ts.scale[rejected] = over;
            ts.gone[rejected] = x;
          }
          ++rejected;
        }
        __syncthreads();
      }
    }
    if (take) {
      cur = i;
      ++depth;
      ++i;
      if (threadIdx.x == 0) a.path[row0 + depth] = cur;
    } else if (!want_q) {
      break;
    }
  }
  int next;
  if (GREEDY) {
    next = best;
  } else if (n >= 0) {
    next = draw_list(idx, r, (double)a.u_sample[b], ts);
  } else {
    __syncthreads();  // the block sees what its threads have left
    next = N > 0 ? draw_index([&](int k) { return lr[k]; }, N, (double)a.u_sample[b], ts) : -1;
    if (next >= 0) next = li[next];
  }
  if (threadIdx.x == 0) {
    a.n_accepted[b] = depth;
    a.next_token[b] = next;
  }
}

template <int EPT>
hipError_t launch_tree_ept(const TreeVerifyArgs& a, hipStream_t stream) {
  const dim3 block(kTreeThreads);
  if (a.greedy) {
    hipLaunchKernelGGL((tree_verify_kernel<EPT, true>), dim3((unsigned)a.batch), block, 0, stream, a);
    return hipGetLastError();
  }
  if (a.ready > 0) {
    const int64_t rows = a.batch * a.ready * (a.draft ? 2 : 1);
    hipLaunchKernelGGL(tree_rows_kernel<EPT>, dim3((unsigned)rows), block, 0, stream, a);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  hipLaunchKernelGGL((tree_verify_kernel<EPT, false>), dim3((unsigned)a.batch), block, 0, stream, a);
  return hipGetLastError();
}

}  // namespace

// Rows opened beforehand: a block each, one on a CU. 102 trees of 16 nodes at V = 49,152
// (with the walk): 256 rows 228 us, 512 211, 1,024 184, 2,048 213, 4,096 229. Half of them are the
// draft's: without a draft 512 are opened (the same trees, nucleus 0.9: 91 us).
constexpr int64_t kReadyRows = 1024;
static int tree_ready_nodes(int64_t batch, int64_t n) {
  const int64_t k = kReadyRows / (2 * batch);
  return (int)(k < n ? k : n);
}
size_t tree_workspace(TreeVerifyArgs& a, void* workspace) {
  const int64_t lists = a.batch * tree_ready_nodes(a.batch, a.n);
  const int64_t entries = a.batch * ((a.V + 1) / 2 * 2);
  uintptr_t p = reinterpret_cast<uintptr_t>(workspace);
  auto take = [&](int64_t bytes) {
    const uintptr_t at = p;
    p += bytes;
    return reinterpret_cast<char*>(at);
  };
  a.ready_rows = take(2 * lists * sizeof(TreeRow));
  a.list_p = reinterpret_cast<double*>(take(lists * kMaxCand * 8));
  a.large_p = reinterpret_cast<double*>(take(entries * 8));
  a.large_p2 = reinterpret_cast<double*>(take(entries * 8));
  a.large_q = reinterpret_cast<double*>(take(entries * 8));
  a.list_idx = reinterpret_cast<int32_t*>(take(lists * kMaxCand * 4));
  a.large_idx = reinterpret_cast<int32_t*>(take(entries * 4));
  return (size_t)(p - reinterpret_cast<uintptr_t>(workspace));
}

hipError_t launch_tree_verify(TreeVerifyArgs a, int ept, hipStream_t stream) {
  a.ready = a.greedy ? 0 : tree_ready_nodes(a.batch, a.n);
  switch (ept) {
    case 16: return launch_tree_ept<16>(a, stream);
    case 32: return launch_tree_ept<32>(a, stream);
    case 48: return launch_tree_ept<48>(a, stream);
    case 64: return launch_tree_ept<64>(a, stream);
    default: return hipErrorInvalidValue;
  }
}

}  // namespace mls
