// A row's sampling distribution, by one block of 1024 threads: the parameters of
// softmax(l / temperature) restricted to the nucleus, and draws from it (see the head
// step's comment for the definition).
#pragma once

#include <math.h>

#include "mls_device.h"
#include "mls_launch.h"
#include "mls_wave.h"

namespace mls {

namespace {

// ---------------------------------------------------------------------------
// per-row sampling distribution
// ---------------------------------------------------------------------------
//
// One 1024-thread block per row. Element i of a thread sits at vocabulary
// index v = 64 EPT wave + 64 i + lane: each wave owns a contiguous range of
// 64 EPT tokens, a slab i of it is one coalesced 256-byte load, and index
// order is (wave, slab, lane).
//
// Nucleus threshold. With `total` the sum of the row's exp weights and
// P = top_p * total, theta is the largest weight value whose mass
// S(theta) = sum(weight >= theta) still reaches P. S(c) >= P for some c puts
// theta at c or above, and every kept token among the weights >= c.
// 1. A close c for the price of a few LDS atomics: the largest weight of each
//    of a thread's kGroups runs of elements (4,096 in a row) enters a histogram
//    of mass over the weights' upper bits. From the top down, the first bin
//    edge c at which these maxima alone hold P has S(c) >= P, and where the
//    nucleus is small against the number of runs, c lies little below theta.
// 2. The weights >= c, a few per wave, move in index order to an LDS list; one
//    wave finds theta among them, resolves ties and draws.
// 3. Rows whose nucleus is too large for step 1 or the list take a radix
//    selection over all weights >= c0 = (1 - top_p) total / V (the weights
//    below c0 hold less than (1 - top_p) of the mass): a histogram of 64-bit
//    fixed-point masses (2^-44; sums do not depend on the order of the atomics)
//    over eight bins per octave names the bin that holds theta; if the weights
//    from that bin's lower edge up still overflow the list, three more levels
//    over the remaining bits give theta itself.
//
// The kernel lasts as long as one row's serial chain on its CU: load and
// maximum 4.7 us at V = 49,152, exp weights and sum 2.7 us (both bound by the
// CU), then barriers, scans of the thread's elements and the list wave. At 102
// such rows (nucleus 0.9 at temperature 0.4) a launch took 24 us with a list of
// every weight >= c0 (some 2,000 of them), three bound raises on it and a
// four-way threshold search, and 22 us with the radix selection for every row;
// it takes 15.5 us (one row: 20 -> 12 us; the records of 714 verifier rows:
// 73 -> 51 us).

constexpr int kRowThreads = 1024;
constexpr int kRowWaves = kRowThreads / 64;
constexpr int kMaxEPT = 64;
constexpr int kRunMax = 16;              // candidate entries per lane of the list wave
constexpr int kMaxCand = 64 * kRunMax;   // candidates one wave holds
constexpr int kSmallCand = 4 * 64;       // lists searched with 4 entries per lane
constexpr int kGroups = 4;               // runs of a thread's elements with a maximum each
constexpr int kRegion = 256;             // list entries per wave before they are joined
constexpr int kMaxShift = 21;            // bins of the maxima: four per octave,
constexpr int kMaxBins = 64;             // 16 octaves (the last bin: everything below)
constexpr int kTopShift = 20;            // radix selection: the bits from here up,
constexpr int kBins = 512;               // weights down to 2^-64 (c0 >= 2^-40)
constexpr uint32_t kOne = 0x3f800000u;   // weight 1, the largest

// LDS slot of list entry j: one gap after every 16 entries, so that the lanes
// of the list wave, each reading a run of consecutive entries, hit different
// banks.
__device__ __forceinline__ int cand_slot(int j) { return j + (j >> 4); }
constexpr int kCandSlots = kMaxCand + kMaxCand / 16;

struct RowShared {
  unsigned long long hist[kBins]; // mass per bin, 2^-44
  unsigned maxhist[kMaxBins];     // mass of the runs' maxima per bin, 2^-15
  float bw[kRowWaves * kRegion];  // one list region per wave, in index order
  int bi[kRowWaves * kRegion];
  float cw[kCandSlots];           // candidate list, index order
  int ci[kCandSlots];             // their vocabulary indices
  float seg[kMaxEPT * kRowWaves]; // per (wave, slab) sums for whole-row index-order scans
  float scr[64];                  // list wave: the threshold bin's entries
  float rmax[kRowWaves];
  float rsum[kRowWaves];
  float red[kRowWaves];
  int ired[kRowWaves];
  int wcnt[kRowWaves];            // per-wave list counts
  float bcast[4];
  int ibcast[4];
};

// A row's exp weights are formed in several places (the distribution's
// parameters, then draws and probabilities recomputed from the logits); they
// must agree bitwise, so the product and the difference are rounded on their
// own and never contracted into an FMA.
__device__ __forceinline__ float scaled_logit(float l, float inv_temp) {
#pragma clang fp contract(off)
  return l * inv_temp;
}
__device__ __forceinline__ float weight_of(float scaled, float m) {
#pragma clang fp contract(off)
  return fast_exp2((scaled - m) * kLog2e);
}

// Block-wide reductions in a fixed order (every thread gets the result).
__device__ __forceinline__ float block_sum(float v, RowShared& sh) {
  v = wave_sum(v);
  const int w = threadIdx.x >> 6;
  if ((threadIdx.x & 63) == 0) sh.red[w] = v;
  __syncthreads();
  float s = 0.f;
#pragma unroll
  for (int i = 0; i < kRowWaves; ++i) s += sh.red[i];
  __syncthreads();
  return s;
}
__device__ __forceinline__ int block_count(int v, RowShared& sh) {
  v = wave_sum(v);
  const int w = threadIdx.x >> 6;
  if ((threadIdx.x & 63) == 0) sh.ired[w] = v;
  __syncthreads();
  int s = 0;
#pragma unroll
  for (int i = 0; i < kRowWaves; ++i) s += sh.ired[i];
  __syncthreads();
  return s;
}
// The waves' results, one per lane of each 16-lane row, combined in a fixed
// order. Used with an LDS array of its own each time, so one barrier suffices.
static_assert(kRowWaves == 16, "one DPP row holds the waves' results");
__device__ __forceinline__ float block_max_once(float v, float* red) {
  v = wave_max(v);
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
  __syncthreads();
  return wave_max(red[threadIdx.x & 15]);
}
__device__ __forceinline__ float block_sum_once(float v, float* red) {
  v = wave_sum(v);
  if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = v;
  __syncthreads();
  return row16_sum(red[threadIdx.x & 15]);
}

// Argmax with the lowest index on ties.
__device__ __forceinline__ void block_argmax(float& val, int& idx, RowShared& sh) {
  wave_argmax(val, idx);
  const int w = threadIdx.x >> 6;
  if ((threadIdx.x & 63) == 0) {
    sh.red[w] = val;
    sh.ired[w] = idx;
  }
  __syncthreads();
  val = sh.red[0];
  idx = sh.ired[0];
#pragma unroll
  for (int i = 1; i < kRowWaves; ++i)
    if (argmax_better(sh.red[i], sh.ired[i], val, idx)) {
      val = sh.red[i];
      idx = sh.ired[i];
    }
  __syncthreads();
}

// Vocabulary index of the thread's element i.
template <int EPT>
__device__ __forceinline__ int elem_v(int i) {
  return (int)(threadIdx.x >> 6) * (64 * EPT) + 64 * i + (int)(threadIdx.x & 63);
}

// Number of the thread's elements inside the row: element i exists iff
// i < elems_in_row (a compare with a constant, so no per-element index needs
// to stay live).
template <int EPT>
__device__ __forceinline__ int elems_in_row(int V) {
  const int v0 = elem_v<EPT>(0);
  return V > v0 ? (V - v0 + 63) >> 6 : 0;
}

// The thread's EPT logits of a row, x[i] = row[elem_v(i)], as buffer loads
// over the row's V * 4 bytes: one per-lane offset, the slab as a scalar
// offset, and indices past the row read 0 from the hardware range check, so
// every load is unconditional and all of them are in flight together.
// Callers mask v >= V themselves.
template <int EPT>
__device__ __forceinline__ void load_row(const float* row, int V, float* x) {
  const __amdgpu_buffer_rsrc_t rs =
      __builtin_amdgcn_make_buffer_rsrc((void*)row, (short)0, V * 4, 0x00020000);
  const int base = elem_v<EPT>(0) * 4;
#pragma unroll
  for (int i = 0; i < EPT; ++i)
    x[i] = __builtin_bit_cast(float, __builtin_amdgcn_raw_buffer_load_b32(rs, base, 256 * i, 0));
}

__device__ __forceinline__ int lanes_below(unsigned long long m) {
  return (int)__builtin_amdgcn_mbcnt_hi((unsigned)(m >> 32),
                                        __builtin_amdgcn_mbcnt_lo((unsigned)m, 0u));
}

// Smallest index whose cumulative weight in index order exceeds `target`,
// over the whole row; weight(i) gives the thread's i-th weight. Returns -1 if
// the total does not exceed it.
template <int EPT, class Wt>
__device__ __forceinline__ int index_order_draw(Wt weight, float target, RowShared& sh) {
  const int wave = threadIdx.x >> 6;
  const int lane = threadIdx.x & 63;
  // per (slab, wave) sums
#pragma unroll
  for (int i = 0; i < EPT; ++i) {
    const float s = wave_sum(weight(i));
    if (lane == 0) sh.seg[wave * EPT + i] = s;
  }
  __syncthreads();
  // wave 0 scans the 16 EPT segment sums in index order (each lane owns a run of them)
  if (wave == 0) {
    constexpr int NSEG = EPT * kRowWaves;
    constexpr int PER = NSEG / 64;
    float run = 0.f;
#pragma unroll
    for (int q = 0; q < PER; ++q) run += sh.seg[lane * PER + q];
    const float incl = wave_incl_scan(run);
    float before = incl - run;
    int found = -1;
    float found_before = 0.f;
#pragma unroll
    for (int q = 0; q < PER; ++q) {
      const int sidx = lane * PER + q;
      const float s = sh.seg[sidx];
      if (found < 0 && s > 0.f && before + s > target) {
        found = sidx;
        found_before = before;
      }
      before += s;
    }
    // the first lane (in index order) that found its segment wins
    const unsigned long long m = __ballot(found >= 0);
    if (lane == 0) sh.ibcast[0] = -1;
    if (m && lane == __builtin_ctzll(m)) {
      sh.ibcast[0] = found;
      sh.bcast[0] = found_before;
    }
  }
  __syncthreads();
  const int sidx = sh.ibcast[0];
  const float base = sh.bcast[0];
  __syncthreads();
  if (sidx < 0) return -1;
  const int swave = sidx / EPT;
  const int slab = sidx % EPT;
  // inside the segment: the owning wave scans its 64 lanes
  if (wave == swave) {
    float x = 0.f;
#pragma unroll
    for (int i = 0; i < EPT; ++i)
      if (i == slab) x = weight(i);
    const float incl = wave_incl_scan(x);
    const unsigned long long m = __ballot(x > 0.f && base + incl > target);
    int pick;
    if (m) {
      pick = __builtin_ctzll(m);
    } else {  // rounding: take the last positive weight of the segment
      const unsigned long long pos = __ballot(x > 0.f);
      pick = pos ? 63 - __builtin_clzll(pos) : 0;
    }
    if (lane == 0) sh.ibcast[1] = swave * (64 * EPT) + slab * 64 + pick;
  }
  __syncthreads();
  const int v = sh.ibcast[1];
  __syncthreads();
  return v;
}

__device__ __forceinline__ bool kept_w(float e, int v, const RowDist& d) {
  return e > d.theta || (e == d.theta && e > 0.f && v <= d.tie_cut);
}

// Keeps the compiler from carrying compares of the thread's elements (a mask of
// two scalar registers each) from one pass over them to the next: it would
// spill them.
template <int EPT>
__device__ __forceinline__ void pass_fence(float* w) {
#pragma unroll
  for (int i = 0; i < EPT; ++i) asm volatile("" : "+v"(w[i]));
}

// Writes the row elements of bit patterns >= lo (lo > 0, no negative elements)
// to the LDS list in index order, at cand_slot(position), and returns how many
// there are. Index order is (wave, slab, lane): each wave writes its elements to
// its own region, then moves them behind those of the waves before it. Where
// the total exceeds kMaxCand or a wave's number its region, nothing is moved
// and a number above kMaxCand is returned.
template <int EPT>
__device__ __forceinline__ int compact_row(float* w, uint32_t lo, RowShared& sh) {
  const int lane = threadIdx.x & 63;
  const int wave = threadIdx.x >> 6;
  pass_fence<EPT>(w);
  int pos0 = 0;  // wave-uniform
#pragma unroll
  for (int i = 0; i < EPT; ++i) {
    const bool f = __float_as_uint(w[i]) >= lo;
    const unsigned long long b = __ballot(f);
    if (b == 0) continue;  // most slabs hold no entry
    if (f) {
      const int pos = pos0 + lanes_below(b);
      if (pos < kRegion) {
        sh.bw[wave * kRegion + pos] = w[i];
        sh.bi[wave * kRegion + pos] = elem_v<EPT>(i);
      }
    }
    pos0 += __builtin_popcountll(b);
  }
  if (lane == 0) sh.wcnt[wave] = pos0;
  __syncthreads();
  const int cnt = sh.wcnt[lane & (kRowWaves - 1)];  // the 16 counts, in every lane row
  const int incl = row16_incl_scan(cnt);
  const int total = lane_read(incl, kRowWaves - 1);
  if (total > kMaxCand || __ballot(cnt > kRegion) != 0) return kMaxCand + 1;
  const int at = wave == 0 ? 0 : lane_read(incl, wave - 1);
  for (int j = lane; j < pos0; j += 64) {
    sh.cw[cand_slot(at + j)] = sh.bw[wave * kRegion + j];
    sh.ci[cand_slot(at + j)] = sh.bi[wave * kRegion + j];
  }
  __syncthreads();
  return total;
}

// ---- list wave (wave 0, all lanes active): lane l holds entries [l RUN, (l + 1) RUN)

template <int RUN>
__device__ __forceinline__ void load_run(const RowShared& sh, int n, float (&w)[RUN]) {
  const int lane = threadIdx.x & 63;
#pragma unroll
  for (int q = 0; q < RUN; ++q) {
    const int j = lane * RUN + q;
    w[q] = j < n ? sh.cw[cand_slot(j)] : 0.f;
  }
}

template <int RUN>
__device__ __forceinline__ int run_index(const RowShared& sh, int q) {
  return sh.ci[cand_slot((int)(threadIdx.x & 63) * RUN + q)];
}

// Position in the list of the first entry (index order) whose cumulative
// weight exceeds `target`; the last positive entry when rounding leaves the
// target at or above the sum; 0 when every weight is 0, which the callers rule
// out (a row that keeps no token has no list to draw from).
template <int RUN>
__device__ __forceinline__ int run_draw(const float (&kw)[RUN], float target) {
  const int lane = threadIdx.x & 63;
  float run = 0.f;
#pragma unroll
  for (int q = 0; q < RUN; ++q) run += kw[q];
  const float incl = wave_incl_scan(run);
  const unsigned long long hit = __ballot(run > 0.f && incl > target);
  const unsigned long long pos = __ballot(run > 0.f);
  if (!pos) return 0;
  const int L = hit ? __builtin_ctzll(hit) : 63 - __builtin_clzll(pos);
  int j = 0;
  if (lane == L) {
    float acc = incl - run;
    int first = -1, last = 0;
#pragma unroll
    for (int q = 0; q < RUN; ++q) {
      if (kw[q] > 0.f) {
        acc += kw[q];
        last = q;
        if (first < 0 && acc > target) first = q;
      }
    }
    j = lane * RUN + (first >= 0 ? first : last);
  }
  return __builtin_amdgcn_readlane(j, L);
}

// Theta from the list (list wave; n entries): the largest value whose mass
// reaches P, which lies in [lo, hi) (bit patterns). Four-way steps (three
// probes, three independent reductions; the probed sets are nested and summed
// in the same order, so the computed masses are ordered like the exact ones)
// until at most 64 entries lie in the bracket. The mass at or above hi is then
// fixed, those entries move to one per lane (through `scr`), and each lane
// takes the mass at or above its own entry: the largest entry whose mass
// reaches P is theta, with no further search.
template <int RUN>
__device__ __forceinline__ float list_theta(const float (&w)[RUN], uint32_t lo, uint32_t hi,
                                            float P, float* scr) {
  const int lane = threadIdx.x & 63;
  int n2;
  for (;;) {
    int inside = 0;
#pragma unroll
    for (int q = 0; q < RUN; ++q) {
      const uint32_t b = __float_as_uint(w[q]);
      inside += b >= lo && b < hi ? 1 : 0;
    }
    n2 = wave_sum(inside);
    if (RUN == 1 || n2 <= 64 || hi - lo <= 3) break;
    const uint32_t st = (hi - lo) >> 2;
    const uint32_t m1 = lo + st, m2 = m1 + st, m3 = m2 + st;
    float p1 = 0.f, p2 = 0.f, p3 = 0.f;
#pragma unroll
    for (int q = 0; q < RUN; ++q) {
      const uint32_t b = __float_as_uint(w[q]);
      p1 += b >= m1 ? w[q] : 0.f;
      p2 += b >= m2 ? w[q] : 0.f;
      p3 += b >= m3 ? w[q] : 0.f;
    }
    const int g1 = __builtin_amdgcn_readfirstlane(wave_sum(p1) >= P ? 1 : 0);
    const int g2 = __builtin_amdgcn_readfirstlane(wave_sum(p2) >= P ? 1 : 0);
    const int g3 = __builtin_amdgcn_readfirstlane(wave_sum(p3) >= P ? 1 : 0);
    if (g3) {
      lo = m3;
    } else if (g2) {
      lo = m2;
      hi = m3;
    } else if (g1) {
      lo = m1;
      hi = m2;
    } else {
      hi = m1;
    }
  }
  if (n2 == 0) return __uint_as_float(lo);  // rounding: the entries at or above hi are kept
  if (n2 > 64) {  // three or fewer bit patterns with more than 64 entries (ties): one probe each
    for (uint32_t b = hi - 1; b > lo; --b) {
      float p = 0.f;
#pragma unroll
      for (int q = 0; q < RUN; ++q) p += __float_as_uint(w[q]) >= b ? w[q] : 0.f;
      if (__builtin_amdgcn_readfirstlane(wave_sum(p) >= P ? 1 : 0)) return __uint_as_float(b);
    }
    return __uint_as_float(lo);
  }
  float base = 0.f;
  int cnt = 0;
#pragma unroll
  for (int q = 0; q < RUN; ++q) {
    const uint32_t b = __float_as_uint(w[q]);
    base += b >= hi ? w[q] : 0.f;
    cnt += (b >= lo && b < hi) ? 1 : 0;
  }
  const float B = wave_sum(base);
  int pos = wave_incl_scan(cnt) - cnt;
#pragma unroll
  for (int q = 0; q < RUN; ++q) {
    const uint32_t b = __float_as_uint(w[q]);
    if (b >= lo && b < hi) scr[pos++] = w[q];
  }
  const float x = lane < n2 ? scr[lane] : 0.f;
  float part[4] = {B, 0.f, 0.f, 0.f};  // (entries n2 .. 63 are 0 and add nothing)
  for (int k = 0; k < n2; k += 4) {
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      const float y = lane_read(x, k + q);
      part[q] += y >= x ? y : 0.f;
    }
  }
  const float mass = (part[0] + part[1]) + (part[2] + part[3]);
  // (the smallest entry's mass reaches P up to rounding; it is taken if none does)
  const float smallest = -wave_max(lane < n2 ? -x : -INFINITY);
  const float best = wave_max(lane < n2 && mass >= P ? x : 0.f);
  return best > 0.f ? best : smallest;
}

// Completes a row's distribution from its list (list wave; theta in [lo, hi)): theta, the
// tie cut and the kept mass. `kw` receives the kept weights of the lane's run.
template <int RUN>
__device__ __forceinline__ void run_dist(RowShared& sh, int n, uint32_t lo, uint32_t hi, float P,
                                         int V, RowDist& d, float (&kw)[RUN]) {
  const int lane = threadIdx.x & 63;
  float w[RUN];
  load_run<RUN>(sh, n, w);
  const float th = list_theta<RUN>(w, lo, hi, P, sh.scr);
  d.theta = th;
  float above = 0.f;
  int ties = 0;
#pragma unroll
  for (int q = 0; q < RUN; ++q) {
    above += w[q] > th ? w[q] : 0.f;
    ties += w[q] == th ? 1 : 0;  // th > 0, so padding zeros never tie
  }
  const float mass_above = wave_sum(above);
  const int n_tie = wave_sum(ties);
  int k = n_tie;
  if (n_tie > 1) {
    k = (int)ceilf((P - mass_above) / th);
    k = k < 1 ? 1 : (k > n_tie ? n_tie : k);
  }
  d.tie_cut = V;
  if (k < n_tie) {  // vocabulary index of the k-th tied entry (the list is in index order)
    const int incl = wave_incl_scan(ties);
    const int L = __builtin_ctzll(__ballot(incl >= k));
    int cut = 0;
    if (lane == L) {
      int seen = incl - ties;
#pragma unroll
      for (int q = 0; q < RUN; ++q)
        if (w[q] == th && ++seen == k) cut = run_index<RUN>(sh, q);
    }
    d.tie_cut = __builtin_amdgcn_readlane(cut, L);
  }
  float kp = 0.f;
#pragma unroll
  for (int q = 0; q < RUN; ++q) {
    kw[q] = w[q] > th || (w[q] == th && run_index<RUN>(sh, q) <= d.tie_cut) ? w[q] : 0.f;
    kp += kw[q];
  }
  d.kept = wave_sum(kp);
}

__device__ __forceinline__ unsigned long long fixed_mass(float e) {
  return (unsigned long long)(e * 17592186044416.f);  // 2^44; a row's sum stays below 2^60
}

// The first bin, from bin 0 on, at which `above` plus the masses up to it reach
// P (2^-44 units); `above` becomes the mass before that bin. -1 if none does.
// Every wave runs it on its own.
template <int NB>
__device__ __forceinline__ int pick_bin(const unsigned long long* hist, double P, double& above) {
  constexpr int PER = NB / 64;
  const int lane = threadIdx.x & 63;
  double h[PER];
  double run = 0.0;
#pragma unroll
  for (int q = 0; q < PER; ++q) {
    h[q] = (double)hist[lane * PER + q];
    run += h[q];
  }
  const double incl = wave_incl_scan(run);
  const unsigned long long hit = __ballot(above + incl >= P);
  if (!hit) return -1;
  const int L = __builtin_ctzll(hit);
  double before = above + incl - run;
  int bin = PER - 1;
  bool found = false;
#pragma unroll
  for (int q = 0; q < PER; ++q) {
    if (!found) {
      if (q == PER - 1 || before + h[q] >= P) {
        bin = q;
        found = true;
      } else {
        before += h[q];
      }
    }
  }
  above = lane_read(before, L);
  return L * PER + __builtin_amdgcn_readlane(bin, L);
}

// Loads a row and computes its sampling distribution. `e` receives the
// thread's exp weights exp(l / T - max) (0 beyond V). With a nucleus that fits
// the list, the weights of bit patterns >= `lo` are left there and their number
// is returned: then only m and total are set in d, and the list wave completes
// it (run_dist; theta lies in [lo, hi)). Otherwise the whole distribution is in
// d for every thread and -1 is returned.
template <int EPT>
__device__ __forceinline__ int row_dist(const float* row, int V, float inv_temp, float top_p,
                                        float* e, RowShared& sh, RowDist& d, uint32_t& lo,
                                        uint32_t& hi, float& P) {
  constexpr int kRun = EPT / kGroups;
  load_row<EPT>(row, V, e);
  if (threadIdx.x < kMaxBins) sh.maxhist[threadIdx.x] = 0;
  const int nv = elems_in_row<EPT>(V);
  float mx[kGroups];
#pragma unroll
  for (int g = 0; g < kGroups; ++g) {
    mx[g] = -INFINITY;
#pragma unroll
    for (int i = g * kRun; i < (g + 1) * kRun; ++i) {
      e[i] = i < nv ? scaled_logit(e[i], inv_temp) : -INFINITY;
      mx[g] = fmaxf(mx[g], e[i]);
    }
  }
  d.m = block_max_once(fmaxf(fmaxf(mx[0], mx[1]), fmaxf(mx[2], mx[3])), sh.rmax);
  const float m = d.m == -INFINITY ? 0.f : d.m;  // a row of -inf: every weight 0
  float s = 0.f;
#pragma unroll
  for (int i = 0; i < EPT; ++i) {
    e[i] = weight_of(e[i], m);
    s += e[i];
  }
  const bool nucleus = top_p < 1.f;
  if (nucleus) {
#pragma unroll
    for (int g = 0; g < kGroups; ++g) {
      const float w = weight_of(mx[g], m);  // the run's largest weight
      const int bin = (int)(kOne >> kMaxShift) - (int)(__float_as_uint(w) >> kMaxShift);
      if (bin >= 0 && bin < kMaxBins - 1) atomicAdd(&sh.maxhist[bin], (unsigned)(w * 32768.f));
    }
  }
  d.total = block_sum_once(s, sh.rsum);
  d.theta = 0.f;
  d.tie_cut = V;
  d.kept = d.total;
  if (!nucleus) return -1;
  P = top_p * d.total;
  lo = 0;
  hi = kOne + 1;  // nothing is above 1
  {
    // rounded down, the masses never overstate the maxima's
    const unsigned incl = wave_incl_scan((int)sh.maxhist[threadIdx.x & 63]);
    const unsigned long long hit = __ballot((float)incl >= P * 32768.f * 1.000001f);
    if (hit && d.total > 0.f) {
      const uint32_t c = ((kOne >> kMaxShift) - (uint32_t)__builtin_ctzll(hit)) << kMaxShift;
      const int n = compact_row<EPT>(e, c, sh);
      if (n <= kMaxCand) {
        lo = c;
        return n;
      }
    }
  }
  // radix selection over all weights >= c0 (at most 1)
  __syncthreads();
  for (int b = threadIdx.x; b < kBins; b += kRowThreads) sh.hist[b] = 0;
  __syncthreads();
  const float c0 = (1.f - top_p) * d.total / (float)V;
  pass_fence<EPT>(e);
#pragma unroll
  for (int i = 0; i < EPT; ++i) {
    const bool in = e[i] >= c0 && e[i] > 0.f;
    if (__ballot(in) == 0) continue;
    if (in) {
      const int bin = (int)(kOne >> kTopShift) - (int)(__float_as_uint(e[i]) >> kTopShift);
      atomicAdd(&sh.hist[bin < kBins ? bin : kBins - 1], fixed_mass(e[i]));
    }
  }
  __syncthreads();
  const double Pd = (double)P * 17592186044416.0;
  double above = 0.0;
  const int bin = pick_bin<kBins>(sh.hist, Pd, above);
  if (bin >= 0 && bin < kBins - 1 && d.total > 0.f) {
    lo = ((kOne >> kTopShift) - (uint32_t)bin) << kTopShift;
    if (bin > 0) hi = lo + (1u << kTopShift);
    const int n = compact_row<EPT>(e, lo, sh);
    if (n <= kMaxCand) return n;
    // the nucleus overflows the list: the bin's remaining bits, 8 + 8 + 4 at a time
#pragma unroll 1
    for (int shift = kTopShift; shift > 0;) {
      const int bits = shift >= 8 ? 8 : shift;
      const int sh2 = shift - bits;
      __syncthreads();  // the previous level's histogram has been read
      if (threadIdx.x < 256) sh.hist[threadIdx.x] = 0;
      __syncthreads();
      pass_fence<EPT>(e);
#pragma unroll
      for (int i = 0; i < EPT; ++i) {
        const uint32_t b = __float_as_uint(e[i]);
        const bool in = b >= lo && b < hi;
        if (__ballot(in) == 0) continue;
        if (in) atomicAdd(&sh.hist[((1 << bits) - 1) - (int)((b - lo) >> sh2)], fixed_mass(e[i]));
      }
      __syncthreads();
      const int k = pick_bin<256>(sh.hist, Pd, above);
      // (the masses of the level add up to the bin's, so some digit reaches P)
      lo += (uint32_t)(((1 << bits) - 1) - (k < 0 ? (1 << bits) - 1 : k)) << sh2;
      hi = lo + (1u << sh2);
      shift = sh2;
    }
  } else {
    // no weight (or NaN), or rounding left the histogram's mass below P (top_p
    // within an ulp of 1): the largest bit pattern b with sum(e >= b) >= P;
    // sum(e >= 0) = total does
    while (hi - lo > 1) {
      const uint32_t mid = lo + (hi - lo) / 2;
      float part = 0.f;
#pragma unroll
      for (int i = 0; i < EPT; ++i) part += __float_as_uint(e[i]) >= mid ? e[i] : 0.f;
      if (block_sum(part, sh) >= P)
        lo = mid;
      else
        hi = mid;
    }
  }
  d.theta = __uint_as_float(lo);
  float above_f = 0.f;
  int ties = 0;
#pragma unroll
  for (int i = 0; i < EPT; ++i) {
    above_f += e[i] > d.theta ? e[i] : 0.f;
    ties += (e[i] == d.theta && e[i] > 0.f) ? 1 : 0;
  }
  const float mass_above = block_sum(above_f, sh);
  const int n_tie = block_count(ties, sh);
  int k = n_tie;
  if (n_tie > 1 && d.theta > 0.f) {
    k = (int)ceilf((P - mass_above) / d.theta);
    k = k < 1 ? 1 : (k > n_tie ? n_tie : k);
  }
  // index of the k-th tied token (counts are exact in fp32 up to 2^24)
  const float th = d.theta;
  d.tie_cut = k >= n_tie ? V
                         : index_order_draw<EPT>(
                               [&](int i) { return (e[i] == th && e[i] > 0.f) ? 1.f : 0.f; },
                               (float)k - 0.5f, sh);
  float kp = 0.f;
#pragma unroll
  for (int i = 0; i < EPT; ++i) {
    const int v = elem_v<EPT>(i);
    kp += kept_w(e[i], v, d) ? e[i] : 0.f;
  }
  d.kept = block_sum(kp, sh);
  return -1;
}

// Whole-row draw from a row's distribution with uniform u (weights in `e`,
// parameters in d); `e` is overwritten with the kept weights.
template <int EPT>
__device__ __forceinline__ int row_draw(float* e, const RowDist& d, float u, RowShared& sh) {
  int last = -1;
#pragma unroll
  for (int i = 0; i < EPT; ++i) {
    const int v = elem_v<EPT>(i);
    e[i] = kept_w(e[i], v, d) ? e[i] : 0.f;
    if (e[i] > 0.f) last = v;
  }
  int v = index_order_draw<EPT>([&](int i) { return e[i]; }, u * d.kept, sh);
  if (v < 0) {  // rounding pushed the target past the total: the last kept index
    float lv = (float)last;
    int li = last;
    block_argmax(lv, li, sh);
    v = li;
  }
  return v;
}

template <int EPT>
__device__ __forceinline__ int row_argmax(const float* row, int V, RowShared& sh) {
  float x[EPT];
  load_row<EPT>(row, V, x);
  const int nv = elems_in_row<EPT>(V);
  float best = -INFINITY;
  int bi = 0x7fffffff;
#pragma unroll
  for (int i = 0; i < EPT; ++i) {
    if (i < nv && x[i] > best) {  // the index increases with i: strict > keeps the lowest
      best = x[i];
      bi = i;
    }
  }
  bi = bi == 0x7fffffff ? bi : elem_v<EPT>(0) + 64 * bi;
  block_argmax(best, bi, sh);
  return bi == 0x7fffffff ? -1 : bi;  // no logit above -inf: no token
}

// The distribution from the list (list wave), then (with u >= 0) a draw;
// returns the drawn token (or -1 without a draw).
template <int RUN>
__device__ __forceinline__ int list_finish_run(RowShared& sh, int n, uint32_t lo, uint32_t hi,
                                               float P, int V, float u, RowDist& d) {
  float kw[RUN];
  run_dist<RUN>(sh, n, lo, hi, P, V, d, kw);
  if (u < 0.f) return -1;
  const int j = run_draw<RUN>(kw, u * d.kept);
  return sh.ci[cand_slot(j)];
}
// One, 4 or 16 entries per lane.
__device__ __forceinline__ int list_finish(RowShared& sh, int n, uint32_t lo, uint32_t hi, float P,
                                           int V, float u, RowDist& d) {
  return n <= 64           ? list_finish_run<1>(sh, n, lo, hi, P, V, u, d)
         : n <= kSmallCand ? list_finish_run<4>(sh, n, lo, hi, P, V, u, d)
                           : list_finish_run<kRunMax>(sh, n, lo, hi, P, V, u, d);
}

// Exp weight of logit x under a row's parameters, with row_dist's arithmetic.
__device__ __forceinline__ float exp_weight(float logit, float inv_temp, const RowDist& d) {
  return weight_of(scaled_logit(logit, inv_temp), d.m);
}

// Kept, normalised probability of token v (v < V).
__device__ __forceinline__ float prob_at(const float* row, int v, float inv_temp,
                                         const RowDist& d) {
  const float e = exp_weight(row[v], inv_temp, d);
  return kept_w(e, v, d) ? e / d.kept : 0.f;
}

// Compacts the kept tokens of row p (weights recomputed from the logits) into
// the LDS list; returns their number.
template <int EPT>
__device__ __forceinline__ int compact_kept(const float* prow, int V, float it, const RowDist& dp,
                                            RowShared& sh) {
  float w[EPT];
  load_row<EPT>(prow, V, w);
  const int nv = elems_in_row<EPT>(V);
  const int v0 = elem_v<EPT>(0);
#pragma unroll
  for (int i = 0; i < EPT; ++i) {
    const float e = exp_weight(w[i], it, dp);
    w[i] = i < nv && kept_w(e, v0 + 64 * i, dp) ? e : 0.f;
  }
  return compact_row<EPT>(w, 1u, sh);  // every positive weight
}

}  // namespace

}  // namespace mls
