// Entries of a paged key-value cache: writing a step's drafted tokens or a prompt, and
// moving an accepted path's entries together (paper section 2, paragraph "Speculative
// Decoding": the verifier reuses the draft's cache, and drafted entries that are not
// accepted leave it).
//
// Both only move bytes, 16 at a time: an entry's head is 64 to 512 contiguous bytes on
// either side, so every access covers whole lines. Page numbers and positions from the
// device are checked against the pool before they become addresses.
#include "mls_device.h"
#include "mls_launch.h"

namespace mls {

namespace {

constexpr int kCacheThreads = 256;
constexpr int kWriteUnroll = 4;  // chunks of a thread in flight, of the keys and of the values each
constexpr int kTileHeads = 8;    // heads of a block's tile
constexpr int kMoveBatch = 4;    // entries loaded before the first of them is stored

// Chunk offset of entry `t` (head 0, layer 0) of sequence b in the pool; -1 where the
// table has no such page.
__device__ __forceinline__ int64_t entry_at(const CacheArgs& c, int64_t b, int64_t t) {
  const int64_t pg = t >> c.page_log2;
  if (t < 0 || pg >= c.table_pages) return -1;
  const int32_t id = c.table[b * c.table_ld + pg];
  if (id < 0 || id >= c.pages) return -1;
  return id * c.s_page + (t & ((1 << c.page_log2) - 1)) * c.s_entry;
}

// Bound by its bytes: one read and one write of each. A block takes 8 heads of the 16
// entries of one run of a page, so that both sides move pieces of 2 KB and more (the
// step's entries lie head behind head, a page's entry behind entry): entry after entry with
// all heads, every write of a wave began at one place of a head's 4 KB, and five layers of
// 102 trees took 27 us each.
__global__ __launch_bounds__(kCacheThreads) void cache_write_kernel(CacheWriteArgs a) {
  const int64_t b = blockIdx.y;
  const int32_t len = a.c.lengths[b];
  int32_t n = a.counts ? a.counts[b] : a.n;
  n = n < a.n ? n : a.n;
  const int head_tiles = (a.c.kv_heads + kTileHeads - 1) / kTileHeads;
  const int run = blockIdx.x / head_tiles;
  const int h0 = (blockIdx.x - run * head_tiles) * kTileHeads;
  if (len < 0 || n <= 0) return;
  const int64_t t0 = (((int64_t)len >> 4) + run) << 4;  // the run's first entry
  const int i0 = (int)(t0 - len);                       // ... and new entry: below 0 in front of them
  if (i0 >= n) return;
  const int64_t at = entry_at(a.c, b, t0);
  if (at < 0) return;
  const uint32_t chunks = (uint32_t)a.c.chunks;
  const uint32_t total = 16u * kTileHeads * chunks;
#pragma nounroll
  for (uint32_t x0 = threadIdx.x; x0 < total; x0 += kCacheThreads * kWriteUnroll) {
    u32x4_t rk[kWriteUnroll] = {}, rv[kWriteUnroll] = {};
    int64_t to[kWriteUnroll];
#pragma unroll
    for (int u = 0; u < kWriteUnroll; ++u) {
      const uint32_t x = x0 + u * kCacheThreads;
      const uint32_t eh = x / chunks;
      const uint32_t ch = x - eh * chunks;
      const int h = h0 + (int)(eh % kTileHeads);
      const int e = (int)(eh / kTileHeads);
      const int i = i0 + e;
      const bool in = x < total && i >= 0 && i < n && h < a.c.kv_heads;
      to[u] = in ? (at + e * a.c.s_entry + h * a.c.s_head + ch) * 16 : -1;
      // (a piece that is not there: the first one is read, and not used)
      const int64_t from = in ? (b * a.s_batch + i * a.s_node + h * a.s_head + ch) * 16 : 0;
      rk[u] = *reinterpret_cast<const u32x4_t*>(a.k + from);
      rv[u] = *reinterpret_cast<const u32x4_t*>(a.v + from);
    }
#pragma unroll
    for (int u = 0; u < kWriteUnroll; ++u) {
      if (to[u] >= 0) {
        *reinterpret_cast<u32x4_t*>(a.c.k + to[u]) = rk[u];
        *reinterpret_cast<u32x4_t*>(a.c.v + to[u]) = rv[u];
      }
    }
  }
}

// Entry len + j takes what entry len + path[j] held, for j = 0 .. n_accepted. One wave
// lists the moves that there are (many an accepted node is in place already). A thread
// then owns one chunk of one head for all of them and goes through them in order, a batch
// of loads before its stores: with path[j] > j (nodes come after their ancestors) no entry
// is overwritten before it has been read, and nothing needs a second buffer or a barrier.
// Bound by its chain of loads (length, path, table, entry): 102 sequences, five layers of 34
// heads, two nodes accepted on average: 7 us.
__global__ __launch_bounds__(kCacheThreads) void cache_compact_kernel(CacheCompactArgs a) {
  __shared__ int64_t from_sh[64];
  __shared__ int64_t to_sh[64];
  __shared__ int moves_sh;
  const int64_t b = blockIdx.y;
  const int32_t len = a.c.lengths[b];
  int32_t acc = a.n_accepted[b];
  acc = acc < a.n ? acc : a.n - 1;
  const bool idle = len < 0 || acc < 0;
  if (blockIdx.x == 0 && threadIdx.x == 0) a.new_lengths[b] = idle ? len : len + acc + 1;
  if (idle) return;
  if (threadIdx.x < 64) {
    const int j = threadIdx.x;
    const int32_t node = j <= acc ? a.path[b * a.n + j] : -1;
    const bool later = node > j && node < a.n;  // (else in place, or no node of the tree)
    const int64_t from = later ? entry_at(a.c, b, (int64_t)len + node) : -1;
    const int64_t to = later ? entry_at(a.c, b, (int64_t)len + j) : -1;
    const bool move = from >= 0 && to >= 0;
    const unsigned long long m = __ballot(move);
    if (move) {
      const int at = (int)__builtin_amdgcn_mbcnt_hi((uint32_t)(m >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)m, 0));
      from_sh[at] = from;
      to_sh[at] = to;
    }
    if (j == 0) moves_sh = __builtin_popcountll(m);
  }
  __syncthreads();
  const int moves = moves_sh;
  const uint32_t per = (uint32_t)a.c.kv_heads * (uint32_t)a.c.chunks;
  const uint32_t x = blockIdx.x * (uint32_t)kCacheThreads + threadIdx.x;
  const uint32_t layer = x / per;
  if (layer >= (uint32_t)a.c.layers) return;
  const uint32_t hc = x - layer * per;
  const uint32_t h = hc / (uint32_t)a.c.chunks;
  const int64_t off = layer * a.c.s_layer + h * a.c.s_head + (hc - h * a.c.chunks);
#pragma nounroll
  for (int m0 = 0; m0 < moves; m0 += kMoveBatch) {
    u32x4_t rk[kMoveBatch], rv[kMoveBatch];
#pragma unroll
    for (int u = 0; u < kMoveBatch; ++u) {
      const int64_t from = (from_sh[m0 + u < moves ? m0 + u : m0] + off) * 16;
      rk[u] = *reinterpret_cast<const u32x4_t*>(a.c.k + from);
      rv[u] = *reinterpret_cast<const u32x4_t*>(a.c.v + from);
    }
#pragma unroll
    for (int u = 0; u < kMoveBatch; ++u) {
      if (m0 + u >= moves) break;
      const int64_t to = (to_sh[m0 + u] + off) * 16;
      *reinterpret_cast<u32x4_t*>(a.c.k + to) = rk[u];
      *reinterpret_cast<u32x4_t*>(a.c.v + to) = rv[u];
    }
  }
}

}  // namespace

int64_t cache_write_blocks(int64_t n, int64_t kv_heads) {
  return ((n + 15) / 16 + 1) * ((kv_heads + kTileHeads - 1) / kTileHeads);
}

hipError_t launch_cache_write(const CacheWriteArgs& a, hipStream_t stream) {
  const int64_t blocks = cache_write_blocks(a.n, a.c.kv_heads);
  hipLaunchKernelGGL(cache_write_kernel, dim3((unsigned)blocks, (unsigned)a.c.batch), dim3(kCacheThreads), 0, stream, a);
  return hipGetLastError();
}

hipError_t launch_cache_compact(const CacheCompactArgs& a, hipStream_t stream) {
  const int64_t total = (int64_t)a.c.layers * a.c.kv_heads * a.c.chunks;
  hipLaunchKernelGGL(cache_compact_kernel,
                     dim3((unsigned)((total + kCacheThreads - 1) / kCacheThreads), (unsigned)a.c.batch),
                     dim3(kCacheThreads), 0, stream, a);
  return hipGetLastError();
}

}  // namespace mls
