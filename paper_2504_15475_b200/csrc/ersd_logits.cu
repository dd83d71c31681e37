// Penalties, biases and masks on logits: ersd_process_logits.
//
// Bytes bound the operator: every row is read and written once.  Few tokens are changed by more than the mask,
// and which ones is the same for all rows of a sequence, up to the drafted tokens on a row's path.  So one block
// takes a slice of the vocabulary for ALL rows of a sequence, and each of its warps a chunk of kChunk tokens: bulk
// copies bring the chunk of one row after the other into a ring of shared memory while the block counts the
// history's tokens that fall into its slice (integers: no order of the atomics changes a result) and lists those
// that occur; the warp changes the listed tokens and the masked ones in shared memory, and a bulk copy takes the
// chunk away.  A chunk of which the mask allows nothing is not read.
//
// Measured on one B200, bfloat16: 64 chains of nine rows x 128256 tokens behind up to 4096 tokens, all penalties and 64 biases,
// 67 us (4.4 TB/s; without any change 48 us: the rest is latency, a lane's listed tokens one after the other in every row,
// with an instruction issued in half of the cycles); 32 trees of 17 rows x 151936 under masks 81 us (68 without
// penalties); one float32 row of 32000 in 4.1 us.
// Counts of 4096 tokens by each block that shares a sequence's rows are what a small batch costs: one such chain 10.8 us.
#include <cuda_bf16.h>
#include <math.h>

#include <mutex>
#include <type_traits>

#include "ersd_host.h"

namespace ersd {

namespace {

constexpr int kChunk = 1024;          // tokens of a warp's chunk: 32 to a lane
constexpr int kRing = 4;              // rows of a chunk in shared memory
constexpr int kLogitWarps = 4;        // that have a chunk; as many more help to count the history
constexpr int kLogitThreads = 2 * 32 * kLogitWarps;
constexpr int kMaskRing = 8;          // rows of its mask
constexpr int kSlice = kLogitWarps * kChunk;
constexpr int kLead = 8;              // most tokens a row's chunks start before the slice: see below
constexpr int kSpan = kSlice + kLead;
constexpr int kLists = kLogitWarps + 1;
constexpr int kMany = 64;             // tokens with an entry from which on a chunk is shared, see below
constexpr int kMaxVocab = 65535 * kSlice - (kLead - 1);  // a grid has 65535 slices
constexpr int kFewBlocks = 8;         // to an SM, of which up to four run at a time: up to here kFew, see below
constexpr int kSharers = 1 + kLogitWarps;  // its own warp and those that have none
// An entry of the table: how often the token occurs behind the prompt, and
constexpr uint32_t kSeen = 1u << 31;     // that it is in the history
constexpr uint32_t kDrafted = 1u << 30;  // that it is among the drafted tokens: its count depends on the row
constexpr uint32_t kBiased = 1u << 29;   // that it has a bias, whose index + 1 is here where the history is short ...
constexpr int kBiasShift = 13;
constexpr uint32_t kShortCount = (1u << kBiasShift) - 1, kLongCount = kBiased - 1;  // ... and else in a table of its own

struct LogitParams {
  const void* in;
  void* out;
  int64_t ld_in, ld_out;
  int B, R, V;
  int in_place;
  int long_history;  // counts may need more than kShortCount
  const int32_t *history, *history_lens, *prompt_lens, *draft_tokens;
  int history_width, tree;
  const float *repetition, *presence, *frequency;
  const int32_t* bias_tokens;
  const float* bias_values;
  int64_t bias_stride;
  int bias_count;
  const uint32_t* mask;
  int64_t mask_stride_b, mask_stride_r;
  uint8_t parent[ERSD_MAX_ROWS];
};

template <typename T>
__device__ __forceinline__ float to_float(T x);
template <>
__device__ __forceinline__ float to_float<float>(float x) { return x; }
template <>
__device__ __forceinline__ float to_float<__nv_bfloat16>(__nv_bfloat16 x) { return __bfloat162float(x); }
template <typename T>
__device__ __forceinline__ T from_float(float x);
template <>
__device__ __forceinline__ float from_float<float>(float x) { return x; }
template <>
__device__ __forceinline__ __nv_bfloat16 from_float<__nv_bfloat16>(float x) { return __float2bfloat16_rn(x); }

__device__ __forceinline__ uint32_t shared_address(const void* p) { return (uint32_t)__cvta_generic_to_shared(p); }
// Four bytes to shared memory without a register that waits for them; zeros where `there` is false.
__device__ __forceinline__ void copy_word(uint32_t* to, const uint32_t* from, bool there) {
  asm volatile("cp.async.ca.shared.global [%0], [%1], 4, %2;" ::"r"(shared_address(to)), "l"(from), "r"(there ? 4 : 0) : "memory");
}
// The top bit of `hi` in all bits of the upper half, that of `lo` in all of the lower.
__device__ __forceinline__ uint32_t spread_tops(uint32_t hi, uint32_t lo) {
  uint32_t d;
  asm("prmt.b32 %0, %1, %2, 0xBBFF;" : "=r"(d) : "r"(hi), "r"(lo));
  return d;
}
__device__ __forceinline__ void bulk_load(void* to, const void* from, uint32_t bytes, uint64_t* full) {
  asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(shared_address(to)),
               "l"(from), "r"(bytes), "r"(shared_address(full))
               : "memory");
}
__device__ __forceinline__ void bulk_store(void* to, const void* from, uint32_t bytes) {
  asm volatile("cp.async.bulk.global.shared::cta.bulk_group [%0], [%1], %2;" ::"l"(to), "r"(shared_address(from)), "r"(bytes) : "memory");
}

template <typename T>
struct LogitShared {
  T ring[kLogitWarps][kRing][kChunk];
  uint64_t full[kLogitWarps][kRing];
  uint32_t table[kSpan];             // counts and flags of the slice's tokens
  uint32_t touched[kLists][32];      // by chunk of the table: bit j of word w: token w + 32 j has an entry (neighbours,
                                     // the frequent tokens, fall to different lanes)
  int32_t draft[ERSD_MAX_ROWS];
  uint8_t parent[ERSD_MAX_ROWS];
  int listed[kLogitWarps];           // tokens of a warp's chunk that have an entry
  // behind it, where they are needed (room that is not taken lets more blocks onto an SM):
  //   uint32_t bias_at[kSpan];                              1 + index of the token's bias
  //   uint32_t mask[kLogitWarps][kMaskRing][2][32];         the one or two words in which a lane's bits are
};
constexpr size_t kBiasBytes = sizeof(uint32_t) * kSpan, kMaskBytes = sizeof(uint32_t) * kLogitWarps * kMaskRing * 32;

// kVary: rows of the input start at different distances from a 16-byte boundary (else what a warp's chunk is, is
// worked out once and not for every row).
// kFew: few blocks, so that a block's own time counts: several may share a sequence's rows, and a block's warps the
// chunk with the most to change.  With many blocks others fill what a waiting block leaves, and only what this takes
// by itself would show (64 chains of nine rows, 2048 blocks: 71.5 us instead of 67; 32 chains 39 instead of 43).
template <typename T, bool kVary, bool kFew>
__global__ void __launch_bounds__(kLogitThreads) process_logits_kernel(const __grid_constant__ LogitParams p) {
  extern __shared__ __align__(128) char raw[];
  LogitShared<T>& sh = *(LogitShared<T>*)raw;
  uint32_t* const bias_at = (uint32_t*)(raw + sizeof sh);
  const bool own_biases = p.bias_count && p.long_history;
  constexpr int kPer16 = 16 / (int)sizeof(T);
  const int b = blockIdx.x, tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int s0 = (int)blockIdx.y * kSlice;
  // with few sequences several blocks may share the rows: this one has `rows` of them from row0 on, which it counts from 0
  const int row0 = kFew ? (int)((int64_t)p.R * blockIdx.z / gridDim.z) : 0;
  const int rows = kFew ? (int)((int64_t)p.R * (blockIdx.z + 1) / gridDim.z) - row0 : p.R;
  // Chunks start on 16-byte boundaries of the input, `lead` tokens before the slice's own start.  Where all rows
  // have the same lead the table starts there, and a warp's chunk is a chunk of the table; else it starts kLead
  // before, and a warp's chunk of a row lies in two chunks of the table.
  auto lead_of = [&](int r) {
    return (int)(((uintptr_t)((const T*)p.in + ((int64_t)b * p.R + row0 + r) * p.ld_in) / sizeof(T)) & (kPer16 - 1));
  };
  const int base = s0 - (kVary ? kLead : lead_of(0));
  const bool changes = p.history || p.draft_tokens || p.bias_count;
  // (a lane's bits are one word where the rows' chunks start on words, as in rows on 16-byte boundaries)
  const int per_row = kVary || lead_of(0) ? 64 : 32;
  uint32_t* const masks = bias_at + (own_biases ? kSpan : 0) + warp * (kMaskRing * per_row) + lane;
  if (changes) {
    for (int i = tid; i < kSpan; i += kLogitThreads) sh.table[i] = 0;
    if (own_biases)
      for (int i = tid; i < kSpan; i += kLogitThreads) bias_at[i] = 0;
    if (p.tree)
      for (int n = tid; n < ERSD_MAX_ROWS; n += kLogitThreads) sh.parent[n] = p.parent[n];
    if (tid < kLists * 32) sh.touched[tid >> 5][tid & 31] = 0;
  }
  if (warp < kLogitWarps && lane < kRing) {
    asm volatile("mbarrier.init.shared::cta.b64 [%0], 1;" ::"r"(shared_address(&sh.full[warp][lane])) : "memory");
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  __syncwarp();
  asm volatile("griddepcontrol.wait;" ::: "memory");

  const int mask_words = (p.V + 31) >> 5;
  struct Piece {     // a warp's chunk of a row: tokens [lo, hi), of which [a, z) lie in whole 16 bytes
    int start, lo, hi, a, z;
  };
  auto piece_of = [&](int r) {
    Piece c;
    c.start = s0 - lead_of(r) + warp * kChunk;
    c.lo = max(c.start, 0);
    c.hi = min(c.start + kChunk, p.V);
    c.a = c.start + (c.lo - c.start + kPer16 - 1) / kPer16 * kPer16;
    c.z = c.start + (max(c.hi, c.start) - c.start) / kPer16 * kPer16;
    if (c.z < c.a) c.a = c.z = max(c.hi, c.lo);  // (none: the ends take all)
    return c;
  };
  const Piece first = piece_of(0);
  const T* const in0 = (const T*)p.in + ((int64_t)b * p.R + row0) * p.ld_in;
  T* const out0 = (T*)p.out + ((int64_t)b * p.R + row0) * p.ld_out;
  const uint32_t* const mask0 = p.mask ? p.mask + b * p.mask_stride_b + row0 * p.mask_stride_r : nullptr;
  // This lane's 32 bits of row r's mask lie in one word or two, which are asked for kMaskRing - 1 rows ahead.
  auto ask_mask = [&](int r) {
    if (p.mask && r < rows) {
      const int bit = (kVary ? piece_of(r).start : first.start) + lane * 32, w = bit >> 5;
      const uint32_t* m = mask0 + r * p.mask_stride_r;
      const bool lo = w >= 0 && w < mask_words, hi = (bit & 31) && w + 1 >= 0 && w + 1 < mask_words;
      copy_word(masks + r % kMaskRing * per_row, lo ? m + w : m, lo);
      if (per_row == 64) copy_word(masks + r % kMaskRing * per_row + 32, hi ? m + w + 1 : m, hi);
    }
    asm volatile("cp.async.commit_group;" ::: "memory");
  };
  auto bits_of = [&](int r) {
    if (!p.mask) return 0xFFFFFFFFu;
    if (per_row == 32) return masks[r % kMaskRing * per_row];
    const int bit = (kVary ? piece_of(r).start : first.start) + lane * 32;
    return __funnelshift_r(masks[r % kMaskRing * per_row], masks[r % kMaskRing * per_row + 32], bit & 31);
  };
  // Asks for the warp's chunk of row r, unless `allow` (this lane's bits) has nothing in any lane.
  auto load = [&](int r, uint32_t allow) {
    const Piece c = kVary ? piece_of(r) : first;
    T* to = sh.ring[warp][r % kRing];
    const T* in = in0 + r * p.ld_in;
    const bool wanted = __any_sync(0xFFFFFFFFu, allow != 0) && c.lo < c.hi;
    if (lane == 0) {
      const uint32_t bytes = wanted ? (uint32_t)(c.z - c.a) * (uint32_t)sizeof(T) : 0u, full = shared_address(&sh.full[warp][r % kRing]);
      if (bytes) {
        asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(full), "r"(bytes) : "memory");
        bulk_load(to + (c.a - c.start), in + c.a, bytes, &sh.full[warp][r % kRing]);
      } else {
        asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(full) : "memory");
      }
    }
    if (wanted && (c.a > c.lo || c.z < c.hi)) {  // the row's ends, which no bulk copy takes
      for (int t = c.lo + lane; t < min(c.a, c.hi); t += 32) to[t - c.start] = in[t];
      for (int t = max(c.z, c.lo) + lane; t < c.hi; t += 32) to[t - c.start] = in[t];
    }
  };

  const bool streams = (!p.in_place || p.mask) && warp < kLogitWarps;
  if (streams) {
#pragma unroll
    for (int r = 0; r < kMaskRing - 1; ++r) ask_mask(r);
    asm volatile("cp.async.wait_group %0;" ::"n"(kMaskRing - kRing) : "memory");
#pragma unroll
    for (int r = 0; r < kRing - 1; ++r)
      if (r < rows) load(r, bits_of(r));
  }

  float rep = 1.0f, pres = 0.0f, freq = 0.0f;
  const float* bias = nullptr;
  if (changes) {
    if (p.repetition) rep = p.repetition[b];
    if (p.presence) pres = p.presence[b];
    if (p.frequency) freq = p.frequency[b];
    if (p.bias_count) bias = p.bias_values + b * p.bias_stride;
    __syncthreads();  // (the table is zeros)
    auto place_of = [&](int t) { return t >= 0 && t < p.V && t >= base && t - base < kSpan ? t - base : -1; };
    auto touch = [&](int at) { atomicOr(&sh.touched[at / kChunk][at & 31], 1u << (at / 32 & 31)); };
    for (int i = tid; i < p.bias_count; i += kLogitThreads) {
      const int at = place_of(p.bias_tokens[b * p.bias_stride + i]);
      if (at < 0) continue;
      if (own_biases) {
        atomicMax(&bias_at[at], (uint32_t)i + 1u);
        atomicOr(&sh.table[at], kBiased);
      } else {  // (the table holds nothing else yet: the largest is the last of the token's)
        atomicMax(&sh.table[at], kBiased | ((uint32_t)i + 1u) << kBiasShift);
      }
      touch(at);
    }
    if (p.bias_count) __syncthreads();
    const int drafts = p.draft_tokens ? p.R - 1 : 0;  // draft[n], 1 <= n <= drafts: token of node n
    for (int n = 1 + tid; n <= drafts; n += kLogitThreads) {
      const int t = p.tree ? p.draft_tokens[(int64_t)b * p.R + n] : p.draft_tokens[(int64_t)b * (p.R - 1) + n - 1];
      sh.draft[n] = t;
      const int at = place_of(t);
      if (at < 0) continue;
      atomicOr(&sh.table[at], kDrafted);
      touch(at);
    }
    if (p.history) {
      int n = p.history_lens ? p.history_lens[b] : p.history_width;
      n = max(0, min(n, p.history_width));
      const int prompt = p.prompt_lens ? p.prompt_lens[b] : 0;
      const int32_t* h = p.history + (int64_t)b * p.history_width;
      for (int i0 = tid; i0 < p.history_width && (i0 < 8 * kLogitThreads || i0 < n); i0 += 8 * kLogitThreads) {
        int t[8];  // (asked for before the length is known to be so: the entries up to the width are there)
#pragma unroll
        for (int k = 0; k < 8; ++k) t[k] = i0 + k * kLogitThreads < p.history_width ? h[i0 + k * kLogitThreads] : -1;
#pragma unroll
        for (int k = 0; k < 8; ++k)
          if (i0 + k * kLogitThreads >= n) t[k] = -1;
#pragma unroll
        for (int k = 0; k < 8; ++k) {
          const int at = place_of(t[k]);
          if (at < 0) continue;
          atomicOr(&sh.table[at], kSeen);
          if (i0 + k * kLogitThreads >= prompt) atomicAdd(&sh.table[at], 1u);
          touch(at);
        }
      }
    }
    __syncthreads();
  }
  const double rep_inverse = 1.0 / (double)rep;
  const uint32_t count_bits = p.long_history ? kLongCount : kShortCount;
  // The logit x of the table's token `at` on the block's row r.
  auto changed = [&](float x, int at, int r) {
    const uint32_t e = sh.table[at];
    uint32_t c = e & count_bits;
    bool seen = (e & kSeen) != 0;
    if (e & kDrafted) {  // a drafted token counts if it is on the path to this row
      for (int m = row0 + r; m > 0; m = p.tree ? sh.parent[m] : m - 1) c += sh.draft[m] == at + base;
      seen |= c > 0;
    }
    if (seen) {
      // (a product in 64 bits for the quotient: rounded once like it, without a branch between the two)
      if (p.repetition) x = (float)((double)x * (x > 0.0f ? rep_inverse : (double)rep));
      if (c) x -= fmaf(freq, (float)c, pres);
    }
    if (e & kBiased) x += bias[(p.long_history ? bias_at[at] : e >> kBiasShift & 0xFFFFu) - 1];
    return x;
  };

  if (p.in_place && !p.mask) {  // the listed tokens alone
    if (!changes) return;
    for (int l = warp; l < kLists; l += 2 * kLogitWarps) {
      for (int r = 0; r < rows; ++r) {
        const int lead = lead_of(r);
        for (uint32_t left = sh.touched[l][lane]; left; left &= left - 1) {
          const int at = l * kChunk + lane + 32 * (__ffs(left) - 1), t = at + base;
          if (t < s0 - lead || t >= s0 - lead + kSlice) continue;  // (in this row the token is in another block's slice)
          T* x = out0 + r * p.ld_out + t;
          *x = from_float<T>(changed(to_float(*x), at, r));
        }
      }
    }
    return;
  }

  // A sequence's frequent tokens lie close together.  Of the chunk with the most of them, from kMany on, the warps
  // without a chunk take their share in every row, or its own warp would hold up the block (4 us for each row with
  // histories of 3000 tokens).
  int shared_chunk = -1;
  // (not looked for where rows times tokens are few: 4.05 us instead of 4.25 for a row with 208 tokens; without `changes`
  // there are no lists, and no changes of the chunk's own warp for the others to meet it at)
  if (kFew && changes && (int64_t)rows * (p.history_width + p.bias_count) >= 4 * kMany) {
    if (warp < kLogitWarps) {
      const int n = __reduce_add_sync(0xFFFFFFFFu, __popc(sh.touched[warp][lane]));
      if (lane == 0) sh.listed[warp] = n;
    }
    __syncthreads();
    int most = kMany - 1;
#pragma unroll
    for (int w = 0; w < kLogitWarps; ++w)
      if (sh.listed[w] > most) most = sh.listed[w], shared_chunk = w;
  }
  // The tokens of list l, of every `step`-th 32 from `from` on, in a chunk of row r.
  auto change_listed = [&](T* x, int chunk_start, int l, int from, int step, int r) {
    uint32_t mine = sh.touched[l][lane];
    if (step > 1) {
      uint32_t pattern = 0;
#pragma unroll
      for (int i = 0; i < 32; i += kSharers) pattern |= 1u << i;
      mine &= pattern << from;
    }
    for (uint32_t left = mine; left; left &= left - 1) {
      const int at = l * kChunk + lane + 32 * (__ffs(left) - 1), in_chunk = at + base - chunk_start;
      if (kVary && (in_chunk < 0 || in_chunk >= kChunk)) continue;
      x[in_chunk] = from_float<T>(changed(to_float(x[in_chunk]), at, r));
    }
  };
  auto sharers_sync = [](int barrier) { asm volatile("bar.sync %0, %1;" ::"r"(barrier), "n"(32 * kSharers) : "memory"); };
  auto landed = [&](int w, int r) {
    const uint32_t full = shared_address(&sh.full[w][r % kRing]), parity = (uint32_t)(r / kRing) & 1;
    uint32_t ok = 0;
    for (int i = 0; i < (1 << 22) && !ok; ++i)
      asm volatile("{\n\t.reg .pred p;\n\tmbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\n\tselp.b32 %0, 1, 0, p;\n\t}"
                   : "=r"(ok)
                   : "r"(full), "r"(parity)
                   : "memory");
    return __all_sync(0xFFFFFFFFu, ok);
  };
  if (!streams) {
    if (kFew && shared_chunk >= 0)
      for (int r = 0; r < rows; ++r) {
        sharers_sync(1);
        landed(shared_chunk, r);  // (the copy's bytes are there: its own warp has seen it; this thread sees them by this)
        change_listed(sh.ring[shared_chunk][r % kRing], s0 - lead_of(r) + shared_chunk * kChunk, shared_chunk, 1 + warp - kLogitWarps, kSharers, r);
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
        sharers_sync(2);
      }
    return;
  }
  for (int r = 0; r < rows; ++r) {
    const Piece c = kVary ? piece_of(r) : first;
    T* x = sh.ring[warp][r % kRing];
    // (a copy that never lands: seen by whoever reads the row)
    if (!landed(warp, r)) {
      for (int i = lane; i < kChunk; i += 32) x[i] = from_float<T>(__uint_as_float(0x7FC00000u));
    }
    __syncwarp();
    // ---- the listed tokens
    if (changes) {
      if (kFew && warp == shared_chunk) sharers_sync(1);
      change_listed(x, c.start, warp, 0, kFew && warp == shared_chunk ? kSharers : 1, r);
      if (kVary) change_listed(x, c.start, warp + 1, 0, 1, r);
      if (kFew && warp == shared_chunk) sharers_sync(2);
      __syncwarp();
    }
    const uint32_t bits = bits_of(r);
    // ---- the mask: 32 tokens to a lane, which start at different ones of their 16-byte pieces (other banks)
    if (p.mask && bits != 0xFFFFFFFFu) {
      uint4* mine = (uint4*)(x + lane * 32);
      constexpr int kPieces = 2 * (int)sizeof(T);
#pragma unroll
      for (int j = 0; j < kPieces; ++j) {
        const int k = (j + (lane >> (sizeof(T) == 2 ? 1 : 0))) & (kPieces - 1);
        const uint32_t ok = bits >> (k * kPer16);
        uint4 w = mine[k];
        uint32_t v[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          if constexpr (sizeof(T) == 4) {
            v[i] = ok >> i & 1u ? v[i] : 0xFF800000u;
          } else {
            // (all bits of a half as its token's bit, which the shifts bring to the top)
            const uint32_t keep = spread_tops(ok << (30 - 2 * i), ok << (31 - 2 * i));
            v[i] = (v[i] & keep) | (0xFF80FF80u & ~keep);
          }
        }
        mine[k] = make_uint4(v[0], v[1], v[2], v[3]);
      }
    }
    // ---- the next row to ask for takes the place of the one before this, which has been taken away meanwhile
    ask_mask(r + kMaskRing - 1);
    if (r + kRing - 1 < rows) {
      asm volatile("cp.async.wait_group %0;" ::"n"(kMaskRing - kRing) : "memory");
      if (lane == 0) asm volatile("cp.async.bulk.wait_group.read 0;" ::: "memory");
      __syncwarp();
      load(r + kRing - 1, bits_of(r + kRing - 1));
    }
    T* out = out0 + r * p.ld_out;
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    __syncwarp();
    if (((uintptr_t)(out + c.a) & 15) == 0) {
      if (lane == 0) {
        if (c.z > c.a) bulk_store(out + c.a, x + (c.a - c.start), (uint32_t)(c.z - c.a) * (uint32_t)sizeof(T));
        asm volatile("cp.async.bulk.commit_group;" ::: "memory");
      }
      if (c.a > c.lo || c.z < c.hi) {
        for (int t = c.lo + lane; t < min(c.a, c.hi); t += 32) out[t] = x[t - c.start];
        for (int t = max(c.z, c.lo) + lane; t < c.hi; t += 32) out[t] = x[t - c.start];
      }
    } else {  // rows of logits and out at different distances from a 16-byte boundary
      for (int t = c.lo + lane; t < c.hi; t += 32) out[t] = x[t - c.start];
    }
    __syncwarp();
  }
  if (lane == 0) asm volatile("cp.async.bulk.wait_group 0;" ::: "memory");  // (shared memory goes with the block)
}

// What a build (one of eight) needs before its first launch on a device: room for the call that needs the most shared
// memory.  (Set to a call's own need it would change under another thread's launch.)
int prepare_build(const void* kernel, int at, size_t most) {
  static std::mutex m;
  static uint64_t ready[8];  // a bit for each device
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess) return cuda_fail(e);
  if (dev < 0 || dev >= 64) return ERSD_EUNSUPPORTED;
  std::lock_guard<std::mutex> lock(m);
  if (ready[at] >> dev & 1) return ERSD_OK;
  e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)most);
  if (e != cudaSuccess) return cuda_fail(e);
  ready[at] |= (uint64_t)1 << dev;
  return ERSD_OK;
}

}  // namespace

}  // namespace ersd

extern "C" int ersd_process_logits(const void* logits, void* out, ersd_dtype dt, int B, int R, int V, const ersd_logit_opts* opts,
                                   void* cuda_stream) {
  using namespace ersd;
  const ersd_logit_opts o = read_struct(opts);
  if (!logits || !out || B < 1 || R < 1 || V < 1 || (dt != ERSD_F32 && dt != ERSD_BF16)) return ERSD_EINVAL;
  if (o.ld_in < 0 || o.ld_out < 0 || (o.ld_in && o.ld_in < V) || (o.ld_out && o.ld_out < V)) return ERSD_EINVAL;
  if (o.history_width < 0 || (o.history && o.history_width < 1) || (!o.history && (o.history_lens || o.prompt_lens))) return ERSD_EINVAL;
  if (o.bias_count < 0 || o.bias_stride < 0 || (o.bias_count && (!o.bias_tokens || !o.bias_values))) return ERSD_EINVAL;
  if (!o.bias_count && (o.bias_tokens || o.bias_values)) return ERSD_EINVAL;
  if (o.mask_stride_b < 0 || o.mask_stride_r < 0) return ERSD_EINVAL;
  const size_t size = dt == ERSD_BF16 ? 2 : 4;
  if (!aligned_to(logits, size) || !aligned_to(out, size)) return ERSD_EALIGN;
  const void* words[] = {o.history, o.history_lens, o.prompt_lens, o.draft_tokens, o.repetition, o.presence, o.frequency, o.bias_tokens,
                         o.bias_values, o.mask};
  for (const void* w : words)
    if (!aligned_to(w, 4)) return ERSD_EALIGN;
  if (B > 65535 || R > 65535 || V > kMaxVocab || o.bias_count > ERSD_MAX_BIASES || (o.history && o.history_width > (int)kLongCount) || (o.draft_tokens && R > ERSD_MAX_ROWS)) return ERSD_EUNSUPPORTED;
  if (o.draft_tokens && o.parent && !is_tree(o.parent, R)) return ERSD_EINVAL;
  LogitParams p;
  memset(&p, 0, sizeof p);
  p.in = logits;
  p.out = out;
  p.ld_in = o.ld_in ? o.ld_in : V;
  p.ld_out = o.ld_out ? o.ld_out : V;
  p.in_place = out == logits;
  if (p.in_place && p.ld_in != p.ld_out) return ERSD_EINVAL;
  p.B = B;
  p.R = R;
  p.V = V;
  p.history = o.history;
  p.history_lens = o.history_lens;
  p.prompt_lens = o.prompt_lens;
  p.history_width = o.history ? o.history_width : 0;  // (a width alone plays no part)
  p.draft_tokens = R > 1 ? o.draft_tokens : nullptr;
  p.tree = o.draft_tokens && o.parent;
  if (p.tree)
    for (int n = 1; n < R; ++n) p.parent[n] = (uint8_t)o.parent[n];
  p.repetition = o.repetition;
  p.presence = o.presence;
  p.frequency = o.frequency;
  p.bias_tokens = o.bias_tokens;
  p.bias_values = o.bias_values;
  p.bias_stride = o.bias_stride;
  p.bias_count = o.bias_count;
  p.mask = o.mask;
  p.mask_stride_b = o.mask_stride_b;
  p.mask_stride_r = o.mask_stride_r;
  const unsigned slices = (unsigned)(((int64_t)V + kLead - 1 + kSlice - 1) / kSlice);
  const bool vary = (int64_t)B * R > 1 && (p.ld_in * (int64_t)size & 15) != 0;
  size_t smem = dt == ERSD_BF16 ? sizeof(LogitShared<__nv_bfloat16>) : sizeof(LogitShared<float>);
  p.long_history = o.history && o.history_width > (int)kShortCount;
  const bool lead = vary || !aligned_to(logits, 16);
  const size_t most = smem + kBiasBytes + 2 * kMaskBytes;
  smem += (p.bias_count && p.long_history ? kBiasBytes : 0) + (p.mask ? (lead ? 2 : 1) * kMaskBytes : 0);
  const bool few = (int64_t)B * slices <= kFewBlocks * sm_count();
  const auto build = [&](auto is_few) {
    constexpr bool kFew = decltype(is_few)::value;
    return dt == ERSD_BF16 ? (vary ? process_logits_kernel<__nv_bfloat16, true, kFew> : process_logits_kernel<__nv_bfloat16, false, kFew>)
                           : (vary ? process_logits_kernel<float, true, kFew> : process_logits_kernel<float, false, kFew>);
  };
  const auto kernel = few ? build(std::true_type()) : build(std::false_type());
  const int status = prepare_build((const void*)kernel, (dt == ERSD_BF16 ? 4 : 0) + (vary ? 2 : 0) + (few ? 1 : 0), most);
  if (status != ERSD_OK) return status;
  // Blocks share the rows while there are fewer than two to an SM (each counts the slice's history for itself).
  unsigned shares = 1;
  while (few && (int64_t)B * slices * shares * 2 <= 2 * sm_count() && (int)shares * 4 <= R) shares *= 2;
  note_launch("process_logits_kernel<%s>: %d threads x (%d, %u, %u) blocks", dt == ERSD_BF16 ? "bf16" : "f32", kLogitThreads, B, slices, shares);
  // (all sequences' first slices before the next: frequent tokens have low numbers, their blocks the most to change)
  Launch l(dim3((unsigned)B, slices, shares), kLogitThreads, smem, (cudaStream_t)cuda_stream);
  const cudaError_t e = cudaLaunchKernelEx(&l.cfg, kernel, p);
  return e == cudaSuccess ? ERSD_OK : cuda_fail(e);
}
