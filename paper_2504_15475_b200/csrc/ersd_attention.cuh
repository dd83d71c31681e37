// What the two attention kernels share: the call's parameters, which keys a row sees, and the tiles of keys that
// a tile of rows has to go through.
#pragma once
#include "ersd_host.h"

namespace ersd {

// Rows of a (sequence, kv head) are the rows of the chunk times the query heads that share the kv head:
// packed row m = r * group + g is row r of head kv_head * group + g.
struct AttentionParams {
  const void *q, *k, *v;
  void* out;
  const int32_t *table, *context_lens, *row_counts;
  int64_t table_stride;
  int64_t q_b, q_r, q_h, o_b, o_r, o_h;                  // strides in elements
  int64_t k_page, k_token, k_head, v_page, v_token, v_head;
  int B, R, heads, group, dim;
  int page_size, num_pages, capacity;  // capacity: slots of a sequence
  uint32_t page_magic, page_shift;     // slot / page_size = slot * page_magic >> page_shift, for slots below 2^30
  int window, sinks;
  float scale_log2;                    // scale * log2(e): the softmax works in powers of two
  int row_tiles, split;
  int tree;
  uint8_t parent[ERSD_MAX_ROWS], depth[ERSD_MAX_ROWS];
};

// n / d = n * magic >> shift for n < 2^30: with 2^(l-1) < d <= 2^l and magic = (2^(30+l) + e) / d, e < d, the product is
// off by n e / d < 2^(30+l) / d, less than the step to the next multiple.
static inline void set_page_size(AttentionParams& p, int d) {
  int l = 0;
  while ((1ll << l) < d) ++l;
  p.page_size = d;
  p.page_magic = (uint32_t)(((1ull << (30 + l)) + (uint64_t)d - 1) / (uint64_t)d);
  p.page_shift = (uint32_t)(30 + l);
}
__device__ __forceinline__ int page_of(const AttentionParams& p, int slot) {
  return (int)((uint64_t)(uint32_t)slot * p.page_magic >> p.page_shift);
}

// The kernel of tensor-core products, where it applies to the call's types and strides (else ERSD_EUNSUPPORTED);
// p.split = 0: chosen there.
__attribute__((visibility("hidden"))) int launch_attention_tensor(AttentionParams& p, int max_context, cudaStream_t st);

// Positions before the rows of sequence b (with the rows' own, below 2^30, they stay below 2^31).
__device__ __forceinline__ int context_of(const AttentionParams& p, int b) { return min(max(0, p.context_lens[b]), (1 << 30) - 1); }

// What a tile of rows [r0, r1) of a sequence has to read: slots [0, sink_hi) and [lo, hi), in tiles of N slots
// that start at multiples of N.
struct KeyRange {
  int ctx, lo, hi, sink_hi;
  int sink_tiles, first, tiles;  // tile t is slots from tile_start(t) on
  // A slot outside both is seen by no row of the tile.
  __device__ __forceinline__ bool dead(int slot) const { return slot >= hi || (slot >= sink_hi && slot < lo); }
};

template <int N>
__device__ __forceinline__ int tile_start(const KeyRange& k, int t) {
  return (t < k.sink_tiles ? t : k.first + t - k.sink_tiles) * N;
}

// (min_depth: of the rows of the tile; a chain's row r has depth r)
template <int N>
__device__ __forceinline__ KeyRange key_range(const AttentionParams& p, int ctx, int r1, int min_depth) {
  KeyRange k;
  k.ctx = ctx;
  k.hi = min(p.capacity, ctx + r1);
  k.lo = 0;
  k.sink_hi = 0;
  if (p.window) {
    k.lo = max(0, min(ctx + min_depth - p.window + 1, k.hi));
    k.sink_hi = min(p.sinks, k.lo);
    // A chunk's own slots are not in the order of their positions: none of them is left out.
    if (p.tree && k.lo > ctx) k.lo = ctx;
    k.sink_hi = min(k.sink_hi, k.lo);
  }
  k.first = k.lo / N;
  k.sink_tiles = min((k.sink_hi + N - 1) / N, k.first);
  k.tiles = k.sink_tiles + (k.hi + N - 1) / N - k.first;
  return k;
}

}  // namespace ersd
