// Attention of a tree of drafted tokens over a paged cache (paper section 2, paragraph
// "Speculative Decoding": the verifier scores all drafted tokens in one pass over the
// cache it shares with the draft).
//
// For node i of sequence b with context length L, head h and key head h / group,
//   o = sum_t w_t v_t / sum_t w_t,  w_t = exp(scale q . k_t),
// over t < L and over the entries L + j of the nodes j on i's way to the root (i among
// them). A row keeps a running maximum m and sum; w is taken relative to m, in base 2.
//
// What bounds it is the entries' bytes, read once per block of rows: 4 sequences of 65,536
// entries, 34 heads of 128, one row: 698 us, 6.5 TB/s (a large copy: 4.9 TB/s, reads alone
// about 6.6); 102 of up to 1,536 entries, 16 nodes, 24 heads of 96: 227 us, 5.4 TB/s. float32: 102
// of 1,280, 24 heads of 96: 440 us with one node (5.5 TB/s), 471 with 16; 4 of 32,768, 34 heads of
// 128: 821 us with one node, 988 with 32 (4.6 TB/s, 74 TFLOP/s).
//
// A block takes up to 64 rows (nodes x heads of one key head) and one part of the
// entries; its waves take the part's tiles in turn, each for itself, and join their
// sums at the end. Nothing goes through LDS on the way there, and no wave waits for
// another: the two products are laid out so that each one's operands are what loads and
// the other product leave in a lane's registers. (More rows than that read the entries
// too often: a second kernel below, whose waves share them.)
//   S^T = K Q^T   v_mfma 16x16x32: lane (g = lane / 16, r = lane % 16) brings 16 bytes of
//                 entry r's head and 16 bytes of row r; it receives row r's scores with
//                 entries 4 g .. 4 g + 3 of each 16.
//   O^T = V^T P^T the contraction runs over entries in any order that both operands
//                 share: lane (g, r) brings as K values just those entries, for row r its
//                 own weights; of V it has loaded these entries' elements DE r .. DE r +
//                 DE - 1 (DE = D / 16), and product m takes element m of each, entry pairs
//                 joined by one byte permute. A lane's results are row r's elements
//                 4 DE g .. 4 DE g + 4 DE - 1.
// float32 is laid out the same way on v_mfma 16x16x4 (no permutes: one value a register).
//
// Entries 16 s .. 16 s + 15 of a sequence lie in one page, so page numbers and page
// addresses are scalar.
#include <math.h>

#include "mls_core.h"
#include "mls_device.h"
#include "mls_launch.h"
#include "mls_wave.h"

namespace mls {

namespace {

constexpr int kAttnWaves = 4;
// Few blocks with short sequences: more waves to a block, and no parts to join. One
// sequence of 700 entries, 16 heads of 64: two launches of 7.4 and 3.6 us before.
constexpr int kShortWaves = 8;
// A row's weights are relative to a maximum that is brought up to date only where a score
// passes it by this much (base 2): the weights stay below 2^8, which costs the sums nothing.
constexpr float kMaxSlack = 8.f;
// ... and a row's before its first entry: finite, so that a row that has none (every
// score -inf) adds weights of 0 and no NaN; the lowest number, so that no score is below it.
constexpr float kNoMax = -3.40282347e38f;
// Up to here a fused multiply-add may take a row's maximum off the exact product: the two
// roundings differ by 2^-5 at most, which all of the row's weights share. Beyond, the product
// is rounded first, as the maximum's was.
constexpr float kFusedMax = 1048576.f;

template <typename E>
struct AttnTile;
template <>
struct AttnTile<Bf16> {
  static constexpr int kSubs = 2;  // runs of 16 entries of a tile
};
template <>
struct AttnTile<F32> {
  static constexpr int kSubs = 1;
};

// A set of nodes, in two words. (Not in one of 64 bits: that is tested by a 64-bit shift, and
// such a shift by a count in the last vector register that a kernel is given has now and then
// shifted by register 0 instead, so that rows took part in nodes that they do not see.)
struct Nodes {
  uint32_t lo, hi;
};
__device__ __forceinline__ Nodes only_node(int j) {
  const uint32_t bit = 1u << (j & 31);
  return {j & 32 ? 0u : bit, j & 32 ? bit : 0u};
}
__device__ __forceinline__ bool meet(Nodes a, Nodes b) { return ((a.lo & b.lo) | (a.hi & b.hi)) != 0; }
__device__ __forceinline__ bool none_of(Nodes a) { return (a.lo | a.hi) == 0; }

// The nodes on the way from each node to the root, none for a node that the tree does not
// have. One thread per node.
__device__ __forceinline__ Nodes ancestors(const int32_t* parents, int i, int n) {
  Nodes m = {0u, 0u};
  for (;;) {  // i falls with every step
    const Nodes x = only_node(i);
    m.lo |= x.lo;
    m.hi |= x.hi;
    const int p = parents[i];
    if (p == -1) return m;
    if (p < 0 || p >= i) return {0u, 0u};
    i = p;
  }
}

// Cache policy of the entries' loads. Where one block alone reads an entry and the cache is
// larger than the memory side's 256 MB, non-temporal: 4 sequences of 65,536 entries, 34
// heads of 128, one row: 783 -> 698 us (6.5 TB/s), 32 rows 838 -> 797; 102 of 1,280
// entries, 16 rows 421 -> 387. Not where row tiles share them (16 sequences, 320 rows of
// one key head: 164 -> 171), nor where the memory side may still hold them (197 MB: 59 -> 71).
constexpr int kLoadKeep = 0;
constexpr int kLoadOnce = 2;

// Loads of NB bytes, a multiple of 4, at lane offset `voff` and scalar offset `soff` of a
// buffer.
template <int NB, int AUX>
__device__ __forceinline__ void load_bytes(__amdgpu_buffer_rsrc_t rs, int voff, int soff, uint32_t* r) {
  typedef uint32_t words4 __attribute__((ext_vector_type(4)));
  typedef uint32_t words3 __attribute__((ext_vector_type(3)));
  typedef uint32_t words2 __attribute__((ext_vector_type(2)));
  if constexpr (NB >= 16) {
    const words4 v = __builtin_bit_cast(words4, __builtin_amdgcn_raw_buffer_load_b128(rs, voff, soff, AUX));
#pragma unroll
    for (int i = 0; i < 4; ++i) r[i] = v[i];
    if constexpr (NB > 16) load_bytes<NB - 16, AUX>(rs, voff + 16, soff, r + 4);
  } else if constexpr (NB == 12) {
    const words3 v = __builtin_bit_cast(words3, __builtin_amdgcn_raw_buffer_load_b96(rs, voff, soff, AUX));
#pragma unroll
    for (int i = 0; i < 3; ++i) r[i] = v[i];
  } else if constexpr (NB == 8) {
    const words2 v = __builtin_bit_cast(words2, __builtin_amdgcn_raw_buffer_load_b64(rs, voff, soff, AUX));
    r[0] = v[0];
    r[1] = v[1];
  } else {
    static_assert(NB == 4, "whole words");
    r[0] = __builtin_amdgcn_raw_buffer_load_b32(rs, voff, soff, AUX);
  }
}

// A word of values with infinities and NaN taken out.
template <typename E>
__device__ __forceinline__ uint32_t finite_word(uint32_t x);
template <>
__device__ __forceinline__ uint32_t finite_word<F32>(uint32_t x) {
  return (x & 0x7f800000u) == 0x7f800000u ? 0u : x;
}
template <>
__device__ __forceinline__ uint32_t finite_word<Bf16>(uint32_t x) {
  x = (x & 0x7f800000u) == 0x7f800000u ? x & 0xffffu : x;
  return (x & 0x7f80u) == 0x7f80u ? x & 0xffff0000u : x;
}

template <typename E, int D, int RT, int AUX>
struct Attn {
  static constexpr int DE = D / 16;                     // elements of a lane's piece of an entry of V
  static constexpr int SUBS = AttnTile<E>::kSubs;
  static constexpr int KT = 16 * SUBS;                  // entries of a tile
  static constexpr int VB = DE * E::kBytes;             // bytes of such a piece
  static constexpr int VW = VB / 4;
  static constexpr int KC = D * E::kBytes / 64;         // 16-byte pieces of a lane's share of an entry of K
  static constexpr int ROWS = 16 * RT;
  static constexpr int LD = D + 4;                      // floats of a row in LDS
  // Registers of a lane that hold sums, queries, keys and values. Two waves a SIMD have
  // 256 each: below 192 everything else fits beside them (bf16, heads of 128, 32 rows: 160,
  // 215 in all). Asked for, the compiler also keeps the sums out of the accumulation
  // registers, which it otherwise copies them to and from.
  static constexpr int kHeld = RT * DE * 4 + (RT + SUBS) * KC * 4 + SUBS * 4 * VW;
  static constexpr int kWaves = kHeld < 192 ? 2 : 1;

  uint4 qf[RT][KC];
  uint32_t kf[SUBS][KC][4];
  uint32_t vf[SUBS * 4][VW];
  f32x4_t acc[RT][DE];
  float m[RT];
  float l[RT];
  bool far;  // some row's maximum is beyond kFusedMax

  // The 16 entries from t0 on (head hk) in one pool: a scalar base, so that a lane's part
  // of any address is one 32-bit offset. (The host has checked that 16 entries span less
  // than 2 GiB.)
  __device__ __forceinline__ static __amdgpu_buffer_rsrc_t run_rsrc(const char* pool, const AttnArgs& a, int32_t page,
                                                                    int hk, int t0) {
    const int64_t off = (int64_t)page * a.c.s_page + (int64_t)hk * a.c.s_head +
                        (int64_t)(t0 & ((1 << a.c.page_log2) - 1)) * a.c.s_entry;
    return uniform_rsrc(pool + off * 16, (int)(15 * a.c.s_entry * 16) + D * E::kBytes);
  }
  __device__ __forceinline__ void load_k(const AttnArgs& a, const int32_t* page, int hk, int t0, int lane) {
    const int voff = ((lane & 15) * (int)a.c.s_entry + (lane >> 4)) * 16;
#pragma unroll
    for (int s = 0; s < SUBS; ++s) {
      const __amdgpu_buffer_rsrc_t rs = run_rsrc(a.c.k, a, page[s], hk, t0 + 16 * s);
#pragma unroll
      for (int c = 0; c < KC; ++c) load_bytes<16, AUX>(rs, voff + 64 * c, 0, kf[s][c]);
    }
  }
  __device__ __forceinline__ void load_v(const AttnArgs& a, const int32_t* page, int hk, int t0, int lane) {
    const int voff = 4 * (lane >> 4) * (int)a.c.s_entry * 16 + (lane & 15) * VB;
#pragma unroll
    for (int s = 0; s < SUBS; ++s) {
      const __amdgpu_buffer_rsrc_t rs = run_rsrc(a.c.v, a, page[s], hk, t0 + 16 * s);
#pragma unroll
      for (int i = 0; i < 4; ++i) load_bytes<VB, AUX>(rs, voff, i * (int)a.c.s_entry * 16, vf[4 * s + i]);
    }
  }

  // scores of the tile, s[t][sub]
  __device__ __forceinline__ void scores(f32x4_t (&s)[RT][SUBS]) const {
#pragma unroll
    for (int t = 0; t < RT; ++t)
#pragma unroll
      for (int u = 0; u < SUBS; ++u) {
        s[t][u] = f32x4_t{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int c = 0; c < KC; ++c) {
          const uint4 k = make_uint4(kf[u][c][0], kf[u][c][1], kf[u][c][2], kf[u][c][3]);
          if constexpr (E::kBytes == 2) {
            s[t][u] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, k),
                                                              __builtin_bit_cast(bf16x8_t, qf[t][c]), s[t][u], 0, 0, 0);
          } else {
            const uint32_t kw[4] = {k.x, k.y, k.z, k.w};
            const uint32_t qw[4] = {qf[t][c].x, qf[t][c].y, qf[t][c].z, qf[t][c].w};
#pragma unroll
            for (int j = 0; j < 4; ++j)
              s[t][u] = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(kw[j]), __uint_as_float(qw[j]), s[t][u], 0,
                                                             0, 0);
          }
        }
      }
  }

  // Product m's operand from pieces of V (w[entry][word])
  __device__ __forceinline__ static uint4 v_pairs(const uint32_t (&w)[SUBS * 4][VW], int mm) {
    uint32_t x[4];
    const uint32_t sel = (mm & 1) ? 0x07060302u : 0x05040100u;
#pragma unroll
    for (int p = 0; p < 4; ++p) x[p] = __builtin_amdgcn_perm(w[2 * p + 1][mm >> 1], w[2 * p][mm >> 1], sel);
    return make_uint4(x[0], x[1], x[2], x[3]);
  }
  // acc + sum over the tile's entries of w's element m times the weights p
  __device__ __forceinline__ static f32x4_t v_product(const uint32_t (&w)[SUBS * 4][VW], int mm,
                                                      const f32x4_t (&p)[SUBS], uint4 pb, f32x4_t c) {
    if constexpr (E::kBytes == 2) {
      return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, v_pairs(w, mm)),
                                                     __builtin_bit_cast(bf16x8_t, pb), c, 0, 0, 0);
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i)
        c = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(w[i][mm]), p[0][i], c, 0, 0, 0);
      return c;
    }
  }
  __device__ __forceinline__ static uint4 pack_weights(const f32x4_t (&p)[SUBS]) {
    if constexpr (E::kBytes == 2) {
      bf16x8_t b;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        b[i] = static_cast<__bf16>(p[0][i]);
        b[4 + i] = static_cast<__bf16>(p[SUBS - 1][i]);
      }
      return __builtin_bit_cast(uint4, b);
    } else {
      return make_uint4(0u, 0u, 0u, 0u);
    }
  }

  // Tiles in which not every row sees every entry: `see[t]` has the nodes that the lane's
  // row sees, `first` the node of the tile's entry 0 (below 0: context, which every row
  // sees); runs without a page and entries past the last node are seen by none.
  __device__ __forceinline__ void mask(f32x4_t (&s)[RT][SUBS], const Nodes (&see)[RT], int first, int n,
                                       const bool (&page)[SUBS], int lane) {
    const int g4 = 4 * (lane >> 4);
#pragma unroll
    for (int u = 0; u < SUBS; ++u)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int node = first + 16 * u + g4 + i;
        const Nodes bit = only_node(node);
#pragma unroll
        for (int t = 0; t < RT; ++t) {
          const bool in = page[u] && node < n && (node < 0 || meet(see[t], bit));
          s[t][u][i] = in ? s[t][u][i] : -INFINITY;
        }
        // what no row sees is not used, whatever it holds
        if (!page[u] || node >= n) {
#pragma unroll
          for (int w = 0; w < VW; ++w) vf[4 * u + i][w] = 0;
        }
      }
  }

  // Infinities and NaN among the values of nodes: a row that does not see the node must
  // not take part in them, which 0 x inf would. They are taken out here (true where there
  // were any), and added to the rows that see them when the block's sums are joined.
  __device__ __forceinline__ bool take_out_odd(int first, int lane) {
    bool odd = false;
#pragma unroll
    for (int e = 0; e < SUBS * 4; ++e) {
      const bool node = first + 16 * (e >> 2) + 4 * (lane >> 4) + (e & 3) >= 0;  // (all rows see the context)
#pragma unroll
      for (int w = 0; w < VW; ++w) {
        const uint32_t x = node ? finite_word<E>(vf[e][w]) : vf[e][w];
        odd = odd || x != vf[e][w];
        vf[e][w] = x;
      }
    }
    return odd;
  }

  // Queries of the rows from row0 on, and the nodes they see.
  __device__ __forceinline__ void take_rows(const AttnArgs& a, int b, int hk, int row0, bool any,
                                            const Nodes* nodes, Nodes (&see)[RT], int lane) {
#pragma unroll
    for (int t = 0; t < RT; ++t) {
      const int r = row0 + 16 * t + (lane & 15);
      const bool in = r < a.rows && any;
      const int node = in ? r / a.group : 0;
      const int h = hk * a.group + (in ? r - node * a.group : 0);
      see[t] = {0u, 0u};
      if (in) see[t] = nodes[node];
      const char* q = a.q + ((int64_t)b * a.q_batch + (int64_t)node * a.q_node + (int64_t)h * a.q_head) * 16;
#pragma unroll
      for (int c = 0; c < KC; ++c) {
        qf[t][c] = make_uint4(0u, 0u, 0u, 0u);
        if (in) qf[t][c] = *reinterpret_cast<const uint4*>(q + 64 * c + 16 * (lane >> 4));
      }
      m[t] = kNoMax;
      l[t] = 0.f;
#pragma unroll
      for (int mm = 0; mm < DE; ++mm) acc[t][mm] = f32x4_t{0.f, 0.f, 0.f, 0.f};
    }
    far = false;
  }

  // The scores of the tile at entry t0 become weights (for bf16 products in pb), maxima and
  // sums of weights follow; true where nodes' values were infinite or NaN.
  __device__ __forceinline__ bool weigh(f32x4_t (&s)[RT][SUBS], uint4 (&pb)[RT], const AttnArgs& a,
                                        const Nodes (&see)[RT], int t0, int ctx, const bool (&ok)[SUBS],
                                        int lane) {
    bool odd = false;
    bool whole = t0 + KT <= ctx;
#pragma unroll
    for (int u = 0; u < SUBS; ++u) whole = whole && ok[u];
    if (!whole) {
      mask(s, see, t0 - ctx, a.n, ok, lane);
      odd = take_out_odd(t0 - ctx, lane);
    }
    // (a NaN score passes neither test and makes its row NaN)
    float top[RT];
    bool grow = false;
#pragma unroll
    for (int t = 0; t < RT; ++t) {
      top[t] = s[t][0][0];
#pragma unroll
      for (int u = 0; u < SUBS; ++u)
#pragma unroll
        for (int i = 0; i < 4; ++i) top[t] = fmaxf(top[t], s[t][u][i]);
      top[t] *= a.scale;  // (above 0)
      grow = grow || top[t] >= m[t] + kMaxSlack;
    }
    if (__ballot(grow) != 0) {
      // (each row by its own scores: its bits do not depend on what the other rows see)
      bool beyond = false;
#pragma unroll
      for (int t = 0; t < RT; ++t) {
        float mx = fmaxf(top[t], __shfl_xor(top[t], 16, 64));
        mx = fmaxf(mx, __shfl_xor(mx, 32, 64));
        const float mn = mx >= m[t] + kMaxSlack ? mx : m[t];
        const float f = m[t] == mn ? 1.f : fast_exp2(m[t] - mn);
        m[t] = mn;
        beyond = beyond || (fabsf(mn) > kFusedMax && (mn > kNoMax || mx == kNoMax));
        l[t] *= f;
#pragma unroll
        for (int mm = 0; mm < DE; ++mm) acc[t][mm] *= f;
      }
      far = __ballot(beyond) != 0;
    }
    if (far) {
#pragma clang fp contract(off)
#pragma unroll
      for (int t = 0; t < RT; ++t) {
        const bool beyond = fabsf(m[t]) > kFusedMax;
#pragma unroll
        for (int u = 0; u < SUBS; ++u)
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const float y = s[t][u][i] * a.scale;
            const float z = fmaf(s[t][u][i], a.scale, -m[t]);
            s[t][u][i] = beyond ? y - m[t] : z;
          }
      }
    } else {
#pragma unroll
      for (int t = 0; t < RT; ++t)
#pragma unroll
        for (int u = 0; u < SUBS; ++u)
#pragma unroll
          for (int i = 0; i < 4; ++i) s[t][u][i] = fmaf(s[t][u][i], a.scale, -m[t]);
    }
#pragma unroll
    for (int t = 0; t < RT; ++t) {
#pragma unroll
      for (int u = 0; u < SUBS; ++u)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          s[t][u][i] = fast_exp2(s[t][u][i]);
          l[t] += s[t][u][i];
        }
      // bf16 weights, as the values are: up to 2^-8 of each, in both directions. (A weight's two
      // halves would be two products. 102 trees of 16 nodes: results 2.3e-3 off those in 64 bits,
      // with float32 weights 1.7e-3, which is the results' own rounding.)
      pb[t] = pack_weights(s[t]);
    }
    return odd;
  }

  __device__ __forceinline__ void add_values(const f32x4_t (&s)[RT][SUBS], const uint4 (&pb)[RT]) {
#pragma unroll
    for (int mm = 0; mm < DE; ++mm)
#pragma unroll
      for (int t = 0; t < RT; ++t) acc[t][mm] = v_product(vf, mm, s[t], pb[t], acc[t][mm]);
  }

  // Row tile t's sums times f to LDS, row after row.
  __device__ __forceinline__ void put_sums(float (*o)[LD], int t, float f, int lane) const {
    float* p = &o[lane & 15][4 * DE * (lane >> 4)];
#pragma unroll
    for (int j = 0; j < 4 * DE; j += 4)
      *reinterpret_cast<float4*>(p + j) =
          make_float4(acc[t][j % DE][j / DE] * f, acc[t][(j + 1) % DE][(j + 1) / DE] * f,
                      acc[t][(j + 2) % DE][(j + 2) / DE] * f, acc[t][(j + 3) % DE][(j + 3) / DE] * f);
  }
};

template <typename E>
__device__ __forceinline__ void store_out(void* out, int64_t i, float4 v) {
  if constexpr (E::kBytes == 2) {
    uint2 r;
    r.x = (uint32_t)to_storage<Bf16>(v.x) | ((uint32_t)to_storage<Bf16>(v.y) << 16);
    r.y = (uint32_t)to_storage<Bf16>(v.z) | ((uint32_t)to_storage<Bf16>(v.w) << 16);
    *reinterpret_cast<uint2*>(static_cast<uint16_t*>(out) + i) = r;
  } else {
    *reinterpret_cast<float4*>(static_cast<float*>(out) + i) = v;
  }
}

// What sequence b attends to: `ctx` entries of context, and with its nodes' `total`, as far as
// the table's row reaches (the parts cover no more); 0 for one that takes no part.
struct Span {
  int ctx;
  int total;
};
__device__ __forceinline__ Span span_of(const AttnArgs& a, int64_t b) {
  const int32_t len = a.c.lengths[b];
  if (len < 0) return {0, 0};
  const int64_t room = a.c.table_pages << a.c.page_log2;
  const int64_t all = (int64_t)len + a.n;
  return {len, (int)(all < room ? all : room)};
}

// Adds the infinities and NaN among elements d .. d + 3 of the values of the nodes `see`
// whose entries lie in [t_begin, t_end).
template <typename E>
__device__ __forceinline__ void add_odd(const AttnArgs& a, int b, int hk, int d, Nodes see, int t_begin,
                                     int t_end, int ctx, float4& v) {
  for (int j = 0; j < a.n; ++j) {
    const int64_t t = (int64_t)ctx + j;
    const int64_t pg = t >> a.c.page_log2;
    if (!meet(see, only_node(j)) || t < t_begin || t >= t_end || pg >= a.c.table_pages) continue;
    const int32_t id = a.c.table[(int64_t)b * a.c.table_ld + pg];
    if (id < 0 || id >= a.c.pages) continue;
    const char* p = a.c.v + ((int64_t)id * a.c.s_page + (int64_t)hk * a.c.s_head +
                             (int64_t)(t & ((1 << a.c.page_log2) - 1)) * a.c.s_entry) * 16;
    float x[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const typename E::storage e = reinterpret_cast<const typename E::storage*>(p)[d + i];
      uint32_t bits;
      if constexpr (E::kBytes == 2)
        bits = (uint32_t)e << 16;
      else
        bits = __float_as_uint(e);
      x[i] = (bits & 0x7f800000u) == 0x7f800000u ? __uint_as_float(bits) : 0.f;
    }
    // (nothing else: a zero keeps its sign)
    v.x = x[0] != 0.f ? v.x + x[0] : v.x;
    v.y = x[1] != 0.f ? v.y + x[1] : v.y;
    v.z = x[2] != 0.f ? v.z + x[2] : v.z;
    v.w = x[3] != 0.f ? v.w + x[3] : v.w;
  }
}

// What a block works on.
struct Block {
  int b, hk, sp;
  int tile;            // row tile
  int t_begin, t_end;  // entries
  int ctx;
  bool alone;  // the sequence has one part
};

// Four elements of a row whose sums are complete in the block: the result, or a part's sums
// (v; l the sum of weights, relative to mm).
template <typename E, int D>
__device__ __forceinline__ void end_row(const AttnArgs& a, const Block& at, int tile_rows, int row,
                                        const Nodes* nodes, bool odd, int d, float mm, float l, float4 v) {
  const int node = row / a.group;
  const Nodes see = nodes[node];
  if (odd) add_odd<E>(a, at.b, at.hk, d, see, at.t_begin, at.t_end, at.ctx, v);
  if (at.alone) {
    const bool none = at.t_end == 0 || none_of(see) || l == 0.f;
    const float inv = none ? 0.f : 1.f / l;
    const int h = at.hk * a.group + row - node * a.group;
    store_out<E>(a.out, (((int64_t)at.b * a.n + node) * a.heads + h) * D + d,
                 none ? make_float4(0.f, 0.f, 0.f, 0.f) : make_float4(v.x * inv, v.y * inv, v.z * inv, v.w * inv));
    return;
  }
  const int64_t tile = ((int64_t)at.b * a.c.kv_heads + at.hk) * a.n_tiles + at.tile;
  const int64_t rec = (tile * a.splits + at.sp) * tile_rows + row % tile_rows;
  *reinterpret_cast<float4*>(a.acc + rec * D + d) = v;
  // (a node that is not there: no weight in any part)
  if (d == 0) *reinterpret_cast<float2*>(a.ml + rec * 2) = make_float2(mm, none_of(see) ? 0.f : l);
}

// The block's place, nodes and ancestors; false where it has nothing to do.
__device__ __forceinline__ bool find_block(const AttnArgs& a, Block& at, int& total) {
  // Blocks go to the 8 XCDs in turn. The row tiles of one part, which read the same
  // entries, follow each other on one XCD; parts of one sequence go to all of them (in one
  // range of blocks an XCD, the longest sequence's XCD was the last: 4 sequences of 44,000
  // to 65,536 entries 805 us).
  const int turn = blockIdx.x / 8;
  at.tile = turn % a.n_rt;
  int x = (turn / a.n_rt) * 8 + blockIdx.x % 8;
  if (x >= (int)a.c.batch * a.c.kv_heads * a.splits) return false;
  at.sp = x % a.splits;
  x /= a.splits;
  at.hk = x % a.c.kv_heads;
  at.b = x / a.c.kv_heads;
  const Span span = span_of(a, at.b);
  total = span.total;
  at.ctx = span.ctx;
  at.t_begin = (int)((int64_t)at.sp * a.part < total ? at.sp * a.part : total);
  at.t_end = total - at.t_begin > a.part ? at.t_begin + a.part : total;
  at.alone = total <= a.part;
  return at.sp == 0 || at.t_begin < total;
}

// Page of a run of 16 entries; without one, page 0's bytes are read and not used.
__device__ __forceinline__ int32_t page_of(const AttnArgs& a, const int32_t* table, int t, int total, bool& ok) {
  const int64_t pg = t >> a.c.page_log2;
  ok = t < total && pg < a.c.table_pages;
  const int32_t p = __builtin_amdgcn_readfirstlane(ok ? table[pg] : -1);
  ok = p >= 0 && p < a.c.pages;
  return ok ? p : 0;
}

template <typename E, int D, int RT, int WAVES, int AUX>
__global__ __launch_bounds__(64 * WAVES, (WAVES > kAttnWaves ? WAVES / 4 : Attn<E, D, RT, AUX>::kWaves))
void tree_attention_kernel(AttnArgs a) {
  using A = Attn<E, D, RT, AUX>;
  constexpr int kThreadsOf = 64 * WAVES;
  constexpr int SUBS = A::SUBS;
  constexpr int ROWS = A::ROWS;
  __shared__ __attribute__((aligned(16))) float o_sh[WAVES][16][A::LD];
  __shared__ float m_sh[WAVES][ROWS];
  __shared__ float l_sh[WAVES][ROWS];
  __shared__ Nodes see_sh[64];
  __shared__ int32_t parent_sh[64];
  __shared__ int odd_sh;  // some node's values were infinite or NaN

  const int tid = threadIdx.x;
  const int lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  Block at;
  int total;
  if (!find_block(a, at, total)) return;
  const int b = at.b, hk = at.hk, t_begin = at.t_begin, t_end = at.t_end, ctx = at.ctx;

  A w;
  const int32_t* table = a.c.table + (int64_t)b * a.c.table_ld;
  auto pages_of = [&](int t0, int32_t (&id)[SUBS], bool (&ok)[SUBS]) {
#pragma unroll
    for (int s = 0; s < SUBS; ++s) id[s] = page_of(a, table, t0 + 16 * s, total, ok[s]);
  };

  int t0 = t_begin + wave * A::KT;
  int32_t id[SUBS];
  bool ok[SUBS];
  if (t0 < t_end) {  // (under way while the tree is looked at)
    pages_of(t0, id, ok);
    w.load_k(a, id, hk, t0, lane);
    w.load_v(a, id, hk, t0, lane);
  }

  if (tid == 0) odd_sh = 0;
  if (tid < a.n) parent_sh[tid] = a.parents ? a.parents[(int64_t)b * a.n + tid] : tid - 1;
  __syncthreads();
  if (tid < a.n) see_sh[tid] = ancestors(parent_sh, tid, a.n);
  __syncthreads();

  Nodes see[RT];
  const int row0 = at.tile * ROWS;
  w.take_rows(a, b, hk, row0, total > 0, see_sh, see, lane);

  for (; t0 < t_end; t0 += WAVES * A::KT) {
    const int tn = t0 + WAVES * A::KT;
    int32_t id_n[SUBS];
    bool ok_n[SUBS];
    if (tn < t_end) pages_of(tn, id_n, ok_n);
    f32x4_t s[RT][SUBS];
    w.scores(s);
    if (tn < t_end) w.load_k(a, id_n, hk, tn, lane);
    uint4 pb[RT];
    if (w.weigh(s, pb, a, see, t0, ctx, ok, lane)) odd_sh = 1;
    w.add_values(s, pb);
    if (tn < t_end) w.load_v(a, id_n, hk, tn, lane);
#pragma unroll
    for (int u = 0; u < SUBS; ++u) {
      id[u] = id_n[u];
      ok[u] = ok_n[u];
    }
  }

  // the waves' sums, relative to the largest of their maxima
#pragma unroll
  for (int t = 0; t < RT; ++t) {
    float l = w.l[t];
    l += __shfl_xor(l, 16, 64);
    l += __shfl_xor(l, 32, 64);
    if (lane < 16) {
      m_sh[wave][16 * t + lane] = w.m[t];
      l_sh[wave][16 * t + lane] = l;
    }
  }
  __syncthreads();
#pragma unroll
  for (int t = 0; t < RT; ++t) {
    const int r = 16 * t + (lane & 15);
    float m = m_sh[0][r];
#pragma unroll
    for (int i = 1; i < WAVES; ++i) m = fmaxf(m, m_sh[i][r]);
    const float f = w.m[t] == m ? 1.f : fast_exp2(w.m[t] - m);
    if (t > 0) __syncthreads();  // the last tile's rows have been read
    w.put_sums(o_sh[wave], t, f, lane);
    __syncthreads();
    for (int i = tid; i < 16 * (D / 4); i += kThreadsOf) {
      const int rl = i / (D / 4);
      const int d = 4 * (i % (D / 4));
      const int r2 = 16 * t + rl;
      if (row0 + r2 >= a.rows) continue;
      float mm = m_sh[0][r2];
#pragma unroll
      for (int k = 1; k < WAVES; ++k) mm = fmaxf(mm, m_sh[k][r2]);
      float l = 0.f;
      float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
      for (int k = 0; k < WAVES; ++k) {
        l += l_sh[k][r2] * (m_sh[k][r2] == mm ? 1.f : fast_exp2(m_sh[k][r2] - mm));
        const float4 p = *reinterpret_cast<const float4*>(&o_sh[k][rl][d]);
        v.x += p.x;
        v.y += p.y;
        v.z += p.z;
        v.w += p.w;
      }
      end_row<E, D>(a, at, ROWS, row0 + r2, see_sh, odd_sh != 0, d, mm, l, v);
    }
  }
}

// ---------------------------------------------------------------------------
// many rows of one key head (bf16): shared heads under trees of more than a few nodes
// ---------------------------------------------------------------------------
//
// The four waves of a block take a row tile each and the same entries, which come to LDS
// once: 64 at a time, two buffers, by loads that go there directly (wave w brings the w-th
// 16, whose page it looks up). From LDS on, a wave's lanes take what they would have loaded,
// and all else is as above. Row tiles that load for themselves read everything once per
// tile from the second-level and memory-side caches, at their 10 TB/s: 16 sequences of 8,000
// entries, 320 rows of each of two heads of 128: 126 -> 95 us (440 TFLOP/s); 256 rows of 4
// heads of 96: 122 -> 108; 64 sequences of 2,000, 128 rows of 4 heads of 128: 98 -> 78. What
// bounds it: the exponentials, sums and packing between the two products, with two waves a SIMD
// to hide them behind (matrix units 20 % busy, waves waiting 43 % of the time); masks are in
// the tiles with nodes or missing pages alone.
//
// A run of 16 entries of K has its 16-byte chunks rotated per entry (K's reads take one
// chunk of 16 entries at a time); V lies as it is (its reads take whole entries).

constexpr int kStageEntries = 64;

template <int D>
__device__ __forceinline__ int k_place(int entry, int chunk) {
  if constexpr (D == 128) return chunk ^ (entry & 15);
  if constexpr (D == 64) return chunk ^ (entry & 7) ^ ((entry >> 3) & 1);
  return (chunk + (entry >> 2)) % (D / 8);
}

template <int LOADS>
__device__ __forceinline__ void load_run(__amdgpu_buffer_rsrc_t rs, const int (&off)[LOADS], char* lds) {
#pragma unroll
  for (int j = 0; j < LOADS; ++j)
    __builtin_amdgcn_raw_ptr_buffer_load_lds(rs, (lds_void_t*)(lds + j * 1024), 16, off[j], 0, 0, 0);
}

template <int D, int RT>
__global__ __launch_bounds__(64 * kAttnWaves, 2) void many_rows_attention_kernel(AttnArgs a) {
  using A = Attn<Bf16, D, RT, kLoadKeep>;
  constexpr int ROWS = A::ROWS;
  constexpr int CPR = D / 8;          // chunks of an entry's head
  constexpr int LOADS = CPR / 4;      // of a run of 16 entries: 64 chunks each
  constexpr int kRun = 16 * D * 2;    // bytes of a run
  constexpr int kBuf = kStageEntries * D * 2;
  constexpr int kStage = 2 * kBuf;    // K, then V
  static_assert(kAttnWaves * 16 == kStageEntries, "a run to each wave");
  static_assert(kAttnWaves * 16 * A::LD * 4 <= 2 * kStage, "the end's rows fit the buffers");
  __shared__ __attribute__((aligned(16))) char stage[2 * kStage];
  __shared__ Nodes see_sh[64];
  __shared__ int32_t parent_sh[64];
  __shared__ int run_ok[2][kAttnWaves];  // whether a run of the stage has a page
  __shared__ int odd_sh;

  const int tid = threadIdx.x;
  const int lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  Block at;
  int total;
  if (!find_block(a, at, total)) return;
  const int b = at.b, hk = at.hk, t_begin = at.t_begin, t_end = at.t_end, ctx = at.ctx;
  at.tile = at.tile * kAttnWaves + wave;
  const int32_t* table = a.c.table + (int64_t)b * a.c.table_ld;

  int koff[LOADS], voff[LOADS];  // a lane's chunks of a run
#pragma unroll
  for (int j = 0; j < LOADS; ++j) {
    const int slot = j * 64 + lane;
    const int e = slot / CPR;
    const int p = slot % CPR;
    int c;  // the chunk whose place is p
    if constexpr (D == 128)
      c = p ^ (e & 15);
    else if constexpr (D == 64)
      c = p ^ (e & 7) ^ ((e >> 3) & 1);
    else
      c = (p + CPR - (e >> 2)) % CPR;
    koff[j] = (e * (int)a.c.s_entry + c) * 16;
    voff[j] = (e * (int)a.c.s_entry + p) * 16;
  }
  auto issue = [&](int t, int buf) {  // the stage at entry t
    char* base = stage + buf * kStage;
    const int tw = t + 16 * wave;
    bool ok;
    const int32_t page = page_of(a, table, tw, total, ok);
    if (lane == 0) run_ok[buf][wave] = ok ? 1 : 0;
    const __amdgpu_buffer_rsrc_t rk = A::run_rsrc(a.c.k, a, page, hk, tw);
    const __amdgpu_buffer_rsrc_t rv = A::run_rsrc(a.c.v, a, page, hk, tw);
    load_run<LOADS>(rk, koff, base + wave * kRun);
    load_run<LOADS>(rv, voff, base + kBuf + wave * kRun);
  };
  if (t_begin < t_end) issue(t_begin, 0);

  if (tid == 0) odd_sh = 0;
  if (tid < a.n) parent_sh[tid] = a.parents ? a.parents[(int64_t)b * a.n + tid] : tid - 1;
  __syncthreads();
  if (tid < a.n) see_sh[tid] = ancestors(parent_sh, tid, a.n);
  __syncthreads();

  A w;
  Nodes see[RT];
  const int row0 = at.tile * ROWS;
  w.take_rows(a, b, hk, row0, total > 0, see_sh, see, lane);

  int buf = 0;
  for (int t0 = t_begin; t0 < t_end; t0 += kStageEntries) {
    // the stage has arrived, for every wave; and no wave reads the other buffer any more
    wait_vmcnt<0>();
    stage_barrier();
    if (t0 + kStageEntries < t_end) issue(t0 + kStageEntries, buf ^ 1);
    const char* base = stage + buf * kStage;
    auto take_k = [&](int half) {
#pragma unroll
      for (int u = 0; u < 2; ++u)
#pragma unroll
        for (int c = 0; c < A::KC; ++c) {
          const int e = lane & 15;
          const uint4 x = *reinterpret_cast<const uint4*>(base + (2 * half + u) * kRun + e * D * 2 +
                                                          k_place<D>(e, 4 * c + (lane >> 4)) * 16);
          w.kf[u][c][0] = x.x; w.kf[u][c][1] = x.y; w.kf[u][c][2] = x.z; w.kf[u][c][3] = x.w;
        }
    };
    auto take_v = [&](int half) {
#pragma unroll
      for (int u = 0; u < 2; ++u)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const uint32_t* p = reinterpret_cast<const uint32_t*>(base + kBuf + (2 * half + u) * kRun +
                                                                (4 * (lane >> 4) + i) * D * 2 + (lane & 15) * A::VB);
          if constexpr (A::VW == 4) {
            const uint4 x = *reinterpret_cast<const uint4*>(p);
            w.vf[4 * u + i][0] = x.x; w.vf[4 * u + i][1] = x.y; w.vf[4 * u + i][2] = x.z; w.vf[4 * u + i][3] = x.w;
          } else {
#pragma unroll
            for (int k = 0; k < A::VW; ++k) w.vf[4 * u + i][k] = p[k];
          }
        }
    };
    take_k(0);
#pragma unroll
    for (int half = 0; half < 2; ++half) {
      const int t = t0 + half * A::KT;
      if (t >= t_end) break;
      take_v(half);  // (on the way while the scores are formed)
      f32x4_t s[RT][2];
      w.scores(s);
      if (half == 0) take_k(1);  // (and while the weights are)
      bool ok[2];
#pragma unroll
      for (int u = 0; u < 2; ++u) ok[u] = __builtin_amdgcn_readfirstlane(run_ok[buf][2 * half + u]) != 0;
      uint4 pb[RT];
      if (w.weigh(s, pb, a, see, t, ctx, ok, lane)) odd_sh = 1;
      w.add_values(s, pb);
    }
    buf ^= 1;
  }

  // each wave's rows, through its part of the buffers
  __syncthreads();
  float(*o)[A::LD] = reinterpret_cast<float(*)[A::LD]>(stage + wave * 16 * A::LD * 4);
#pragma unroll
  for (int t = 0; t < RT; ++t) {
    float l = w.l[t];
    l += __shfl_xor(l, 16, 64);
    l += __shfl_xor(l, 32, 64);
    if (t > 0) __syncthreads();  // the last tile's rows have been read
    w.put_sums(o, t, 1.f, lane);
    __syncthreads();
    for (int i0 = 0; i0 < 16 * (D / 4); i0 += 64) {
      const int i = i0 + lane;
      const int rl = i / (D / 4);
      const int d = 4 * (i % (D / 4));
      const float lr = __shfl(l, rl, 64);
      const float mr = __shfl(w.m[t], rl, 64);
      const int row = row0 + 16 * t + rl;
      if (row < a.rows)
        end_row<Bf16, D>(a, at, ROWS, row, see_sh, odd_sh != 0, d, mr, lr, *reinterpret_cast<const float4*>(&o[rl][d]));
    }
  }
}

// Joins the parts of a sequence that has several: a thread per four elements of a row.
template <typename E>
__global__ __launch_bounds__(256) void attn_join_kernel(AttnArgs a, int D) {
  const int tile_rows = a.tile;
  const int64_t per = (int64_t)a.n * a.heads * (D / 4);
  const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
  const int64_t b = i / per;
  if (b >= a.c.batch) return;
  const int total = span_of(a, b).total;
  if (total <= a.part) return;
  const int in = (int)(i - b * per);
  const int d = 4 * (in % (D / 4));
  const int nh = in / (D / 4);
  const int node = nh / a.heads;
  const int h = nh - node * a.heads;
  const int hk = h / a.group;
  const int r = node * a.group + (h - hk * a.group);
  const int parts = (total + a.part - 1) / a.part;
  const int64_t rec = (((b * a.c.kv_heads + hk) * a.n_tiles + r / tile_rows) * a.splits) * tile_rows + r % tile_rows;
  float m = -INFINITY;
  for (int s = 0; s < parts; ++s) {
    const float2 ml = *reinterpret_cast<const float2*>(a.ml + (rec + (int64_t)s * tile_rows) * 2);
    m = fmaxf(m, ml.x);
  }
  float l = 0.f;
  float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
  for (int s = 0; s < parts; ++s) {
    const int64_t x = rec + (int64_t)s * tile_rows;
    const float2 ml = *reinterpret_cast<const float2*>(a.ml + x * 2);
    const float f = ml.x == m ? 1.f : fast_exp2(ml.x - m);
    const float4 p = *reinterpret_cast<const float4*>(a.acc + x * D + d);
    l += ml.y * f;
    v.x += p.x * f;
    v.y += p.y * f;
    v.z += p.z * f;
    v.w += p.w * f;
  }
  const float inv = l == 0.f ? 0.f : 1.f / l;
  store_out<E>(a.out, ((b * a.n + node) * a.heads + h) * (int64_t)D + d,
               l == 0.f ? make_float4(0.f, 0.f, 0.f, 0.f) : make_float4(v.x * inv, v.y * inv, v.z * inv, v.w * inv));
}

constexpr int kWideRow = 128;    // bytes of a head up to which a tile has 64 rows
constexpr int kMiddleRow = 768;  // and 32
constexpr int kShortRow = 384;   // and up to which kShortWaves waves of 16 rows have registers

template <typename E, int D, int RT, int WAVES, int AUX>
hipError_t launch_attn_k(const AttnArgs& a, int64_t blocks, hipStream_t stream) {
  hipLaunchKernelGGL((tree_attention_kernel<E, D, RT, WAVES, AUX>), dim3((unsigned)blocks), dim3(64 * WAVES), 0, stream,
                     a);
  return hipGetLastError();
}

constexpr int kManyTile = 32;

template <typename E, int D>
hipError_t launch_attn_d(const AttnArgs& a, int64_t blocks, hipStream_t stream) {
  constexpr int kHeadBytes = D * E::kBytes;
  if constexpr (E::kBytes == 2 && (D == 64 || D == 96 || D == 128))
    if (a.many) {
      hipLaunchKernelGGL((many_rows_attention_kernel<D, kManyTile / 16>), dim3((unsigned)blocks), dim3(64 * kAttnWaves), 0,
                         stream, a);
      return hipGetLastError();
    }
  constexpr int kMost = kHeadBytes <= kWideRow ? 4 : kHeadBytes <= kMiddleRow ? 2 : 1;  // 16 rows each
  switch (a.tile) {
    case 16:
      if constexpr (kHeadBytes <= kShortRow)
        if (a.shorts) return launch_attn_k<E, D, 1, kShortWaves, kLoadKeep>(a, blocks, stream);
      return a.once ? launch_attn_k<E, D, 1, kAttnWaves, kLoadOnce>(a, blocks, stream)
                    : launch_attn_k<E, D, 1, kAttnWaves, kLoadKeep>(a, blocks, stream);
    case 32:
      if constexpr (kMost >= 2)
        return a.once ? launch_attn_k<E, D, 2, kAttnWaves, kLoadOnce>(a, blocks, stream)
                      : launch_attn_k<E, D, 2, kAttnWaves, kLoadKeep>(a, blocks, stream);
      break;
    case 64:
      if constexpr (kMost >= 4)
        return a.once ? launch_attn_k<E, D, 4, kAttnWaves, kLoadOnce>(a, blocks, stream)
                      : launch_attn_k<E, D, 4, kAttnWaves, kLoadKeep>(a, blocks, stream);
      break;
  }
  return hipErrorInvalidValue;
}

template <typename E>
hipError_t launch_attn(const AttnArgs& a, int D, int64_t blocks, hipStream_t stream) {
  switch (D) {
    case 32: return launch_attn_d<E, 32>(a, blocks, stream);
    case 64: return launch_attn_d<E, 64>(a, blocks, stream);
    case 96: return launch_attn_d<E, 96>(a, blocks, stream);
    case 128: return launch_attn_d<E, 128>(a, blocks, stream);
    case 192: return launch_attn_d<E, 192>(a, blocks, stream);
    case 256: return launch_attn_d<E, 256>(a, blocks, stream);
    default: return hipErrorInvalidValue;
  }
}

}  // namespace

// Rows of a tile. Its queries and sums lie in registers beside the entries in flight; more
// rows share each entry's load, but one wave a SIMD (heads of 128 and 64 rows) waits for
// most of it: 16 sequences of 8,000 entries, 320 rows of each of two heads of 128 in tiles
// of 64 / 32 / 16: 162 / 130 / 195 us; 64 rows of each of 16 heads of 64: 126 / 144 / 204.
// `ways`: the tiles of one row tile that run side by side, in the shortest parts. Where they
// would leave the chip idle, smaller tiles are shorter: 7 sequences of 900 entries, 36 rows
// of 3 float32 heads of 64: 21 -> 16 us.
int attn_tile_rows(int32_t rows, int32_t head_bytes, int64_t ways) {
  int tile = head_bytes <= kWideRow ? 64 : head_bytes <= kMiddleRow ? 32 : 16;
  while (tile > 16 && (rows <= tile / 2 || ways * ((rows + tile - 1) / tile) < 512)) tile /= 2;
  return tile;
}
// Many rows: a block takes kAttnWaves tiles of kManyTile, where that leaves no part of the
// chip idle (4 sequences of 500 entries, 80 rows of 4 heads of 64: 18 us, tiles of 16 rows 14)
// and its tiles are not half of them empty (64 rows of 16 heads of 64: 161 us, one tile of 64
// rows 127).
bool attn_many(int32_t rows, int32_t D, bool f32, int64_t ways) {
  constexpr int kBlock = kAttnWaves * kManyTile;
  return !f32 && rows > kBlock / 2 && (D == 64 || D == 96 || D == 128) && ways * ((rows + kBlock - 1) / kBlock) >= 256;
}
int attn_many_tile() { return kManyTile; }
int attn_many_tiles() { return kAttnWaves; }
// blocks: of one part each; entries: that a table's row has room for. With it / without, us:
// 16 blocks, heads of 64: 511 entries 7.0 / 9.2, 1,023 9.6 / 10.3, 1,343 11.2 / 10.9, 2,047 14.9 / 12.1;
// 16 blocks, heads of 128: 511 10.3 / 11.5, 767 12.3 / 11.9, 1,535 19.0 / 13.5;
// 256 blocks: heads of 64, 511 7.9 / 11.9, 1,535 19.1 / 22.4, 2,047 24.4 / 27.3, of 96, 1,535 27.0 / 30.0;
// heads of 64, 1,343 entries: 384 blocks 24.0 / 27.7, 1,024 59.0 / 54.4.
// One border for all: the widest heads of few blocks lose above 700 entries, many blocks would
// still gain beyond it.
bool attn_short(int64_t blocks, int64_t entries, int32_t rows, int32_t head_bytes) {
  return blocks <= 256 && entries <= 1536 && rows <= 16 && head_bytes <= kShortRow;
}

hipError_t launch_tree_attention(const AttnArgs& a, int32_t D, bool f32, hipStream_t stream) {
  const int64_t blocks = (a.c.batch * a.c.kv_heads * a.splits + 7) / 8 * 8 * a.n_rt;
  hipError_t e = f32 ? launch_attn<F32>(a, D, blocks, stream) : launch_attn<Bf16>(a, D, blocks, stream);
  if (e != hipSuccess || a.splits == 1) return e;
  const int64_t threads = a.c.batch * a.n * a.heads * (D / 4);
  const dim3 grid((unsigned)((threads + 255) / 256));
  if (f32)
    hipLaunchKernelGGL(attn_join_kernel<F32>, grid, dim3(256), 0, stream, a, (int)D);
  else
    hipLaunchKernelGGL(attn_join_kernel<Bf16>, grid, dim3(256), 0, stream, a, (int)D);
  return hipGetLastError();
}

}  // namespace mls
