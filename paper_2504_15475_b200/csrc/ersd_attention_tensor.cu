// ersd_chunk_attention on tensor cores: bfloat16 caches with heads of 64 or 128.
//
// A thread block takes a tile of packed rows of one kv head (see AttentionParams) through its keys.  A warp each
// copies keys and values page by page with TMA into rings of shared memory, another issues the products
// (tcgen05.mma), and groups of four warps do the softmax, a thread to a row: scores come out of tensor memory,
// weights go back there as bfloat16 over scores they came from, and the second product takes them from there.
// Two builds:
//   Few<D>   up to 128 packed rows (decoding, drafts), where the cache's bytes bound the call; scores have two or three
//            buffers, so that the next products of scores run during a softmax, and a warp each issues the two
//            products, since what bounds a tile is the waits of the one that issues.  Either 64 slots at a time
//            with half of an SM's shared and tensor memory, so that two blocks share an SM and one's start and end
//            hide behind the other; or, for calls of no more blocks than SMs, 128 slots at a time with longer rings,
//            four warps that copy and q in tensor memory, which leaves shared memory and its rate to them (a step of 16
//            by itself: 64 cycles for 128 columns from either; for 64 columns 48 from shared memory, 32 from there).  The product has 128 rows whether they are there or not: up to 32 rows are put there
//            four times, up to 64 twice, and each copy's warps take a part of the slots, which divides the softmax's
//            time (a warp's powers of two for 64 slots alone take 512 cycles) by as much; the copies' outputs are
//            joined at the end.
//   Many<D>  256 packed rows (long chunks), where products and powers of two do: two streams of 128 rows with a
//            softmax group each, 128 slots at a time (with 64 the first operand is read again for every 64 columns: a
//            score product by itself takes 384 cycles for 64 slots, 512 for 128, and the kernel 2545 against 3660); one's
//            products run while the other's softmax does, and half of a tile's weights go ahead of the rest.
//            No unit is at its limit: of 3170 cycles for a tile of heads of 128 the tensor cores are busy 2048 (scores and
//            outputs of a stream 512 each, measured by themselves), powers of two take 2048, shared memory's traffic at
//            128 bytes a cycle 2048.  What takes the time is a stream's chain, whose scores take the place of its weights:
//            scores 512, softmax 1850 to 1950, the second half of the outputs 256, and waits for the other stream's
//            products in the one queue.  (Over the prompt below the tensor cores are busy 57 % of the cycles in which an SM has a block,
//            which is 85 % of the call: 512 blocks of unlike length, 3.5 to an SM.)  With heads of 64 a tile takes 2970, products 1024 and powers of two 2048 of them.
//            (q in tensor memory, which has room for it beside 64 slots: 683 us instead of 580 for the prompt below.)
// Measured on one B200 (several of them where a range is given): 32 trees of 17 nodes behind 3100 positions on average
// (32/8 heads of 128) 79 to 91 us, 4.6 to 5.3 TB/s; one token each in 18 sequences behind 64000 positions 702 us, 6.7 TB/s
// (behind 32000 to 64000: 568 to 592 us, 6.1 to 6.3); one token behind 1000 positions 9.2 to 9.5 us, behind 64000 54 to 60 us; 2 x
// 2048 rows behind up to 8192 positions 519 to 607 us, 0.91 to 1.06 PFLOP/s (heads of 64: 481 us).
//
// The second product takes both operands in one type, and values are bfloat16: weights are rounded to bfloat16 for it, by
// 2^-8 of each at most.  Sums are of the unrounded weights (of the rounded ones the result is as far off).  Against 64 bits
// the result is 1.2 to 1.4 times as far off as its own rounding to bfloat16 leaves it; weights in two parts would
// take that product twice.  kernel_path = 1 rounds no weight.
//
// The output's accumulator stays in tensor memory.  It is scaled only when a row's maximum has risen by more than
// 2^8 since the last time (weights are then at most 2^8, which bfloat16 and the 32-bit sums hold as well as 1);
// the end divides by a sum formed with the same maximum, so this changes no result beyond rounding.
//
// `split` blocks of a cluster share the keys and join their outputs through distributed shared memory.
#include <cooperative_groups.h>
#include <cuda.h>
#include <cuda_bf16.h>
#include <math.h>

#include <mutex>
#include <type_traits>

#include "ersd_attention.cuh"

namespace cg = cooperative_groups;

namespace ersd {

namespace {

constexpr float kRise = 8.0f;         // a row's maximum may rise by 2^8 before its output is scaled

template <int D_, int kBlocks_>
struct Few {
  static constexpr int D = D_, kStreams = 1, kN = kBlocks_ == 1 ? 128 : 64, kBuffers = kBlocks_ == 2 && D == 64 ? 3 : 2;
  static constexpr int kStages = kBlocks_ == 2 ? (D == 64 ? 4 : 2) : (D == 64 ? 7 : 3);  // of each ring
  static constexpr bool kQInTmem = kBlocks_ == 1;
  static constexpr int kWarps = 4, kCopyWarps = kBlocks_ == 1 ? 4 : 2, kThreads = 192 + 32 * kCopyWarps, kBlocks = kBlocks_, kColumns = 512 / kBlocks_;
};
template <int D_>
struct Many {
  static constexpr int D = D_, kStreams = 2, kN = 128, kBuffers = 2;  // (a stream has one)
  static constexpr int kStages = D == 64 ? 5 : 2;
  static constexpr bool kQInTmem = false;
  // (the last four warps are a group that gives its registers to the others)
  static constexpr int kWarps = 8, kCopyWarps = 2, kThreads = 384, kBlocks = 1, kColumns = 512;
  static constexpr int kRegistersSoftmax = 200, kRegistersOthers = 104;  // 2 * 200 + 104 = 3 * 168, what a launch gives
};

struct Ring {  // of keys or values
  uint64_t full[8], empty[8];
};
struct Misc {  // behind the rings
  Ring ring[2];                  // keys, values
  uint64_t scores[4];            // of a buffer (of the stream, or of a stream) are in tensor memory
  uint64_t half[2];              // with 128 slots: the weights of the first 64 are
  uint64_t weights[4];           // and all weights, which take the scores' place.  (A buffer's own: with one barrier for both
                                 // a quick warp's next tile would count for a slow warp's last.)
  uint64_t rest[4];              // Few: the product with a buffer's weights is done
  uint64_t done;                 // all products
  uint64_t q_there;              // q's rows are in shared memory
  uint32_t tmem;
  uint32_t gave_up;              // a wait ran out: nothing that follows it can be trusted
  uint8_t parent[ERSD_MAX_ROWS], depth[ERSD_MAX_ROWS];
};
static_assert(sizeof(Misc) <= 2048, "");

template <typename C>
struct Plan : C {
  static constexpr int D = C::D, kN = C::kN;
  static constexpr int kRows = C::kStreams * 128;
  static constexpr int kStageBytes = kN * D * 2;  // keys or values of a tile
  static constexpr int kQBytes = C::kQInTmem ? 0 : kRows * D * 2;
  static constexpr int kSmem = kQBytes + 2 * C::kStages * kStageBytes + 2048;
  static constexpr int kOutputs = C::kBuffers * kN;  // first column of the outputs
  static constexpr int kQColumn = kOutputs + C::kStreams * D;
  static constexpr int kPartRow = D + 4;  // floats of a row of partial output: 16 bytes on, so that rows fall on other banks
  static_assert(kRows * (kPartRow + 2) * 4 <= kQBytes + 2 * C::kStages * kStageBytes, "");
  static_assert(kQColumn + (C::kQInTmem ? D / 2 : 0) <= C::kColumns, "");
  // No more than kBlocks blocks fit on an SM by shared memory, and their tensor memory fits with them: a block
  // never waits for another's tensor memory, which could not be given up by one that waits for it in a cluster.
  static_assert((kSmem + 1024) * C::kBlocks <= 228 * 1024 && (kSmem + 1024) * (C::kBlocks + 1) > 228 * 1024, "");
  static_assert(C::kBlocks * C::kColumns <= 512, "");
};

__device__ __forceinline__ uint32_t smem_address(const void* p) { return (uint32_t)__cvta_generic_to_shared(p); }

__device__ __forceinline__ void barrier_init(uint64_t* b, uint32_t count) {
  asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(smem_address(b)), "r"(count) : "memory");
}
__device__ __forceinline__ void barrier_arrive(uint64_t* b) {
  asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(smem_address(b)) : "memory");
}
__device__ __forceinline__ void barrier_expect(uint64_t* b, uint32_t bytes) {
  asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(smem_address(b)), "r"(bytes) : "memory");
}
__device__ __forceinline__ bool barrier_try(uint64_t* b, uint32_t parity) {
  uint32_t ok;
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\n\t"
      "selp.b32 %0, 1, 0, p;\n\t}"
      : "=r"(ok)
      : "r"(smem_address(b)), "r"(parity)
      : "memory");
  return ok != 0;
}
// For a whole warp: whether the phase ended; false when it did not within some seconds, or another wait of the block
// ran out.  (The vote keeps the warp together, and tells the compiler so: what one thread issues later comes from
// registers that the warp shares.)
__device__ __forceinline__ bool barrier_wait(uint64_t* b, uint32_t parity, uint32_t* gave_up) {
  for (int i = 0; i < (1 << 22); ++i) {
    if (__all_sync(0xFFFFFFFFu, barrier_try(b, parity))) return true;
    if (__any_sync(0xFFFFFFFFu, *(volatile uint32_t*)gave_up != 0)) return false;
  }
  *(volatile uint32_t*)gave_up = 1;
  return false;
}
__device__ __forceinline__ bool elected() {  // one thread of the warp
  uint32_t one;
  asm volatile("{\n\t.reg .pred p;\n\telect.sync _|p, 0xFFFFFFFF;\n\tselp.b32 %0, 1, 0, p;\n\t}" : "=r"(one));
  return one != 0;
}

__device__ __forceinline__ void tma_box(uint32_t to, const CUtensorMap* map, int x, int token, int head, int page, uint64_t* full) {
  asm volatile(
      "cp.async.bulk.tensor.4d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4, %5}], [%6];" ::"r"(to),
      "l"(map), "r"(x), "r"(token), "r"(head), "r"(page), "r"(smem_address(full))
      : "memory");
}

// Descriptor of an operand in shared memory, in rows of 128 bytes with their 16-byte pieces swizzled in groups of
// eight rows (1024 bytes apart); `lead`: bytes between panels of 64 elements along the row where the rows run
// along the operand's outer dimension.
__device__ __forceinline__ uint64_t operand(uint32_t address, uint32_t lead) {
  return (uint64_t)((address & 0x3FFFF) >> 4) | (uint64_t)(lead >> 4) << 16 | (uint64_t)(1024 >> 4) << 32 | (uint64_t)1 << 46 | (uint64_t)2 << 61;
}
// Instruction descriptor: bfloat16 times bfloat16 into 32 bits, 128 x n; `outer`: B's rows run along n.
__host__ __device__ constexpr uint32_t instruction(int n, bool outer) {
  return 1u << 4 | 1u << 7 | 1u << 10 | (outer ? 1u << 16 : 0u) | (uint32_t)(n >> 3) << 17 | (uint32_t)(128 >> 4) << 24;
}
__device__ __forceinline__ void mma_shared(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t add) {
  asm volatile(
      "{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\t"
      "tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n\t}" ::"r"(d),
      "l"(a), "l"(b), "r"(idesc), "r"(add)
      : "memory");
}
__device__ __forceinline__ void mma_tmem(uint32_t d, uint32_t a, uint64_t b, uint32_t idesc, uint32_t add) {
  asm volatile(
      "{\n\t.reg .pred p;\n\tsetp.ne.b32 p, %4, 0;\n\t"
      "tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}" ::"r"(d),
      "r"(a), "l"(b), "r"(idesc), "r"(add)
      : "memory");
}
__device__ __forceinline__ void mma_commit(uint64_t* b) {
  asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(smem_address(b)) : "memory");
}
__device__ __forceinline__ void before_sync() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void after_sync() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }

#define R8(a, i) "=r"(a[i]), "=r"(a[i + 1]), "=r"(a[i + 2]), "=r"(a[i + 3]), "=r"(a[i + 4]), "=r"(a[i + 5]), "=r"(a[i + 6]), "=r"(a[i + 7])
#define S8(a, i) "r"(a[i]), "r"(a[i + 1]), "r"(a[i + 2]), "r"(a[i + 3]), "r"(a[i + 4]), "r"(a[i + 5]), "r"(a[i + 6]), "r"(a[i + 7])
// 32 columns of this warp's 32 rows of tensor memory
__device__ __forceinline__ void tmem_load(uint32_t at, uint32_t* r) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, "
      "%16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31}, [%32];"
      : R8(r, 0), R8(r, 8), R8(r, 16), R8(r, 24)
      : "r"(at));
}
__device__ __forceinline__ void tmem_load_16(uint32_t at, uint32_t* r) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, [%16];"
      : R8(r, 0), R8(r, 8)
      : "r"(at));
}
__device__ __forceinline__ void tmem_store(uint32_t at, const uint32_t* r) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x32.b32 [%32], {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, "
      "%16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31};" ::S8(r, 0),
      S8(r, 8), S8(r, 16), S8(r, 24), "r"(at)
      : "memory");
}
__device__ __forceinline__ void tmem_store_8(uint32_t at, const uint32_t* r) {
  asm volatile("tcgen05.st.sync.aligned.32x32b.x8.b32 [%8], {%0, %1, %2, %3, %4, %5, %6, %7};" ::S8(r, 0), "r"(at) : "memory");
}
__device__ __forceinline__ void tmem_store_16(uint32_t at, const uint32_t* r) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x16.b32 [%16], {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15};" ::S8(r, 0),
      S8(r, 8), "r"(at)
      : "memory");
}
__device__ __forceinline__ void tmem_loaded() { asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ void tmem_stored() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }

__device__ __forceinline__ float power_of_two(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
__device__ __forceinline__ uint32_t pair(float lo, float hi) {
  uint32_t y;
  asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(y) : "f"(hi), "f"(lo));
  return y;
}

__device__ __forceinline__ float max3(float a, float b, float c) {
  float y;
  asm("max.f32 %0, %1, %2, %3;" : "=f"(y) : "f"(a), "f"(b), "f"(c));
  return y;
}
// Two 32-bit floats in a register pair, and what is done to both at once.
__device__ __forceinline__ uint64_t two(float a, float b) {
  uint64_t y;
  asm("mov.b64 %0, {%1, %2};" : "=l"(y) : "f"(a), "f"(b));
  return y;
}
__device__ __forceinline__ void apart(uint64_t x, float& a, float& b) { asm("mov.b64 {%0, %1}, %2;" : "=f"(a), "=f"(b) : "l"(x)); }
__device__ __forceinline__ uint64_t fma_two(uint64_t a, uint64_t b, uint64_t c) {
  uint64_t y;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(y) : "l"(a), "l"(b), "l"(c));
  return y;
}
__device__ __forceinline__ uint64_t add_two(uint64_t a, uint64_t b) {
  uint64_t y;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(y) : "l"(a), "l"(b));
  return y;
}

// Bits [a, b) of a word, both cut to 0..32.
__device__ __forceinline__ uint32_t bits_between(int a, int b) {
  a = max(a, 0);
  b = min(b, 32);
  if (a >= b) return 0u;
  return (0xFFFFFFFFu >> (32 - (b - a))) << a;
}

template <typename C>
__global__ void __launch_bounds__(C::kThreads, C::kBlocks)
    attention_tensor_kernel(const __grid_constant__ AttentionParams p, const __grid_constant__ CUtensorMap k_map,
                            const __grid_constant__ CUtensorMap v_map, const int box) {
  using P = Plan<C>;
  constexpr int D = P::D, kN = P::kN, kStreams = C::kStreams, kBuffers = C::kBuffers, kStages = C::kStages;
  constexpr int kPanel = kN * 128, kQPanel = 128 * 128;  // bytes of a panel: rows of 64 elements
  constexpr int kSoftmaxThreads = C::kWarps * 32, kCopies = C::kWarps, kProducts = kCopies + C::kCopyWarps;  // (the last two: warps)
  extern __shared__ __align__(1024) char raw[];
  char* q_tile = raw;
  char* key_ring = q_tile + P::kQBytes;
  char* value_ring = key_ring + kStages * P::kStageBytes;
  Misc& sh = *(Misc*)(value_ring + kStages * P::kStageBytes);
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int kv_head = blockIdx.y, b = blockIdx.z;
  // (a chunk's later rows see more keys: their tiles go first)
  const int tile = p.row_tiles - 1 - (int)blockIdx.x / p.split, part = (int)blockIdx.x % p.split;

  // ---- what needs nothing of the kernel before this one on the stream
  if (tid == 0) {
    for (int i = 0; i < 8; ++i)
      for (int s = 0; s < 2; ++s) {
        barrier_init(&sh.ring[s].full[i], 1);
        barrier_init(&sh.ring[s].empty[i], 1);
      }
    for (int i = 0; i < kBuffers; ++i) {
      barrier_init(&sh.scores[i], 1);
      barrier_init(&sh.rest[i], 1);
    }
    barrier_init(&sh.done, 1);
    barrier_init(&sh.q_there, C::kWarps);
    sh.gave_up = (smem_address(raw) & 1023) != 0;  // (the operands' layout wants it so)
    asm volatile("prefetch.tensormap [%0];" ::"l"(&k_map) : "memory");
    asm volatile("prefetch.tensormap [%0];" ::"l"(&v_map) : "memory");
  }
  if (warp == kProducts) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_address(&sh.tmem)), "n"(C::kColumns) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  if (p.tree)
    for (int n = tid; n < ERSD_MAX_ROWS; n += C::kThreads) {
      sh.parent[n] = p.parent[n];
      sh.depth[n] = p.depth[n];
    }
  asm volatile("griddepcontrol.wait;" ::: "memory");
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");

  // ---- q's rows are asked for while the lengths are on their way
  const int m0 = tile * P::kRows;
  const __nv_bfloat16* q = (const __nv_bfloat16*)p.q + b * p.q_b;
  const bool q_wide = ((p.q_b | p.q_r | p.q_h) & 7) == 0 && ((uintptr_t)p.q & 15) == 0;
  const uint32_t flip = p.scale_log2 < 0.0f ? 0x80008000u : 0u;  // (the softmax takes a positive scale)
  constexpr int kPieces = D / 8;  // of a row, of 16 bytes
  auto q_row = [&](int m) {
    const int r = (m0 + m) / p.group;
    return q + r * p.q_r + (kv_head * p.group + m0 + m - r * p.group) * p.q_h;
  };
  auto load_piece = [&](const __nv_bfloat16* at) {
    if (q_wide) return *(const uint4*)at;
    const unsigned short* e = (const unsigned short*)at;
    return make_uint4(e[0] | (uint32_t)e[1] << 16, e[2] | (uint32_t)e[3] << 16, e[4] | (uint32_t)e[5] << 16, e[6] | (uint32_t)e[7] << 16);
  };
  auto load_q = [&](int i) { return load_piece(q_row(i / kPieces) + i % kPieces * 8); };
  const int most_rows = min(P::kRows, p.R * p.group - m0);  // (some of them may not count)
  const int copies = kStreams == 2 || most_rows > 64 ? 1 : most_rows > 32 ? 2 : 4, copy_rows = 128 / copies;  // how often the rows are there
  const int place = tid & 127, copy = place / copy_rows;  // a softmax thread's
  constexpr int kEarly = C::kQInTmem ? kPieces : 4;  // pieces asked for early by a thread: its own row, or any
  uint4 early[kEarly];
  if (warp < C::kWarps) {
    if constexpr (C::kQInTmem) {
      const int m = place % copy_rows;
      const __nv_bfloat16* at = q_row(min(m, most_rows - 1));
#pragma unroll
      for (int j = 0; j < kEarly; ++j) early[j] = load_piece(at + j * 8);
    } else {
#pragma unroll
      for (int j = 0; j < kEarly; ++j)
        if (tid + j * kSoftmaxThreads < most_rows * kPieces) early[j] = load_q(tid + j * kSoftmaxThreads);
    }
  }

  int rows = p.row_counts ? p.row_counts[b] : p.R;
  const int ctx = context_of(p, b);
  rows = max(0, min(rows, p.R));
  const int m1 = max(m0, min(m0 + P::kRows, rows * p.group));  // (no rows: the same for every block of the cluster)
  const int r0 = m0 / p.group, r1 = max(r0, (m1 - 1) / p.group + 1);
  // the warps of each stream with rows
  const int warps0 = copies > 1 && m1 > m0 ? 4 : (min(m1 - m0, 128) + 31) / 32;
  const int warps1 = kStreams == 1 ? 0 : (max(m1 - m0 - 128, 0) + 31) / 32;
  int min_depth = r0;
  if (p.tree && m1 > m0) {
    min_depth = p.depth[r0];
    for (int r = r0 + 1; r < r1; ++r) min_depth = min(min_depth, (int)p.depth[r]);
  }
  const KeyRange keys = key_range<kN>(p, ctx, r1, min_depth);
  const int all_tiles = m1 > m0 ? keys.tiles : 0;
  const int t0 = all_tiles * part / p.split, t1 = all_tiles * (part + 1) / p.split;  // (at most 2^24 tiles, 16 parts)
  const int tiles = t1 - t0;
  if (tid == 0) {
    for (int i = 0; i < kBuffers; ++i) {
      if (kStreams == 2) barrier_init(&sh.half[i], (uint32_t)max(1, i == 0 ? warps0 : warps1));
      barrier_init(&sh.weights[i], (uint32_t)max(1, kStreams == 1 || i == 0 ? warps0 : warps1));
    }
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  before_sync();
  __syncthreads();
  after_sync();
  const uint32_t tmem = sh.tmem;
  uint32_t* const gave_up = &sh.gave_up;

  float* parts = (float*)q_tile;                        // [rows][kPartRow]
  float* tops = parts + P::kRows * P::kPartRow;        // [rows]
  float* sums = tops + P::kRows;                       // [rows]
  const bool joins = copies > 1 || p.split > 1;  // whether outputs go through shared memory
  // Four columns of a row's joined output.
  const bool out_wide = ((p.o_b | p.o_r | p.o_h) & 3) == 0 && ((uintptr_t)p.out & 7) == 0;
  auto write_row = [&](int row, int d, const float4& y, float total) {
    const float inv = total == 0.f ? 0.f : 1.f / total;
    const int r = (m0 + row) / p.group, g = m0 + row - r * p.group;
    __nv_bfloat16* at = (__nv_bfloat16*)p.out + b * p.o_b + r * p.o_r + (kv_head * p.group + g) * p.o_h + d;
    const uint2 x = make_uint2(pair(y.x * inv, y.y * inv), pair(y.z * inv, y.w * inv));
    if (out_wide) {
      *(uint2*)at = x;
    } else {
      const uint32_t w[2] = {x.x, x.y};
#pragma unroll
      for (int j = 0; j < 4; ++j) ((unsigned short*)at)[j] = (unsigned short)(w[j >> 1] >> (16 * (j & 1)));
    }
  };
  auto products_done = [&]() {
    // (asked for in every case: after a wait that ran out, products may still be under way)
    if (tiles > 0)
      for (int i = 0; i < (1 << 22) && !barrier_try(&sh.done, 0); ++i) {
      }
    __syncwarp();
    after_sync();
  };
  if (warp >= C::kWarps) {
    if constexpr (kStreams == 2) asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(Many<D>::kRegistersOthers));
    if (warp < kProducts) {
      // ---- copies of keys, of values: a lane has a box (`box` slots by 64 elements) of every tile, or the two of its
      // slots.  64 entries of the block table are in the warp's registers, the later 32 asked for 32 pages before
      // they are needed.  All that a tile's copies need is worked out before the wait for their place.
      const bool values = (warp - kCopies) & 1;
      constexpr int kStep = C::kCopyWarps / 2;  // warps that take turns at the tiles of keys, of values
      const CUtensorMap* map = values ? &v_map : &k_map;
      char* const places = values ? value_ring : key_ring;
      Ring& ring = sh.ring[values];
      const int groups = kN / box, boxes = groups * (D / 64), shift = __ffs(groups) - 1;
      const int group = lane & (groups - 1), panel = lane >> shift;
      const int32_t* table = p.table + b * p.table_stride;
      const int last_entry = page_of(p, p.capacity - 1);
      auto entry = [&](int i) { return table[min(i, last_entry)]; };
      int first_entry = 0;
      int32_t near = 0, far = 0;  // entries first_entry + lane, and 32 on
      auto refill = [&](int from) {
        first_entry = from;
        near = entry(from + lane);
        far = entry(from + 32 + lane);
      };
      if (tiles > 0) refill(page_of(p, tile_start<kN>(keys, t0)));
      int t = (warp - kCopies) >> 1, stage = t;
      uint32_t parity = 1;  // of the ring's round before: nothing to wait for in the first
      for (; t < tiles; t += kStep) {
        const int start = tile_start<kN>(keys, t0 + t), end_entry = page_of(p, min(start + kN, p.capacity) - 1);
        if (end_entry >= first_entry + 64) {
          if (page_of(p, start) >= first_entry + 32 && end_entry < first_entry + 96) {
            first_entry += 32;
            near = far;
            far = entry(first_entry + 32 + lane);
          } else {  // behind a gap between first tokens and window (64 entries hold any tile: pages are of four slots and more)
            refill(page_of(p, start));
          }
        }
        const int slot = start + group * box, at = page_of(p, min(slot, p.capacity - 1));
        const int32_t page_near = __shfl_sync(0xFFFFFFFFu, near, at - first_entry & 31), page_far = __shfl_sync(0xFFFFFFFFu, far, at - first_entry & 31);
        int page = at - first_entry < 32 ? page_near : page_far;
        if (page < 0 || page >= p.num_pages) page = p.num_pages;  // (outside the cache: such a page gives zeros)
        const int token = slot - at * p.page_size;
        const bool needed = lane < boxes && slot < keys.hi && !(slot >= keys.sink_hi && slot + box <= keys.lo);
        const uint32_t bytes = (uint32_t)__popc(__ballot_sync(0xFFFFFFFFu, needed)) * (uint32_t)box * (boxes > 32 ? 256u : 128u);
        uint64_t* full = &ring.full[stage];
        const uint32_t to = smem_address(places + stage * P::kStageBytes) + group * box * 128;
        if (t >= kStages && !barrier_wait(&ring.empty[stage], parity, gave_up)) break;
        if (lane == 0) barrier_expect(full, bytes);
        __syncwarp();
        if (needed) {
          tma_box(to + panel * kPanel, map, panel * 64, token, kv_head, page, full);
          if (boxes > 32) tma_box(to + kPanel, map, 64, token, kv_head, page, full);
        }
        __syncwarp();
        if ((stage += kStep) >= kStages) {
          stage -= kStages;
          parity ^= 1;
        }
      }
      // every copy has landed before the block ends, even where the products gave up
      if (*(volatile uint32_t*)gave_up)
        for (int x = max(t - kStep, 0), n = 0; x >= 0 && n < kStages; x -= kStep, n += kStep)
          for (int i = 0; i < (1 << 22) && x < tiles && !barrier_try(&ring.full[x % kStages], (uint32_t)(x / kStages) & 1); ++i) {
          }
      __syncwarp();
    } else if (warp == kProducts || (kStreams == 1 && warp == kProducts + 1)) {
      // ---- products: a warp stays together, one thread issues.  Few: a warp for the scores, a warp for the outputs.
      // Many: one warp for both, since a stream's scores take the place of the weights that the product before uses.
      constexpr uint32_t kScores = instruction(kN, false), kOutput = instruction(D, true);
      const int streams = kStreams == 2 && warps1 > 0 ? 2 : 1;
      const bool leader = elected();
      const uint64_t q_operand = operand(smem_address(q_tile), 16), key_operand = operand(smem_address(key_ring), 16),
                     value_operand = operand(smem_address(value_ring), kPanel);
      int key_stage = 0, value_stage = 0;
      uint32_t key_parity = 0, value_parity = 0;
      // Scores of stream s into `buffer`.  (Addresses are in steps of 16 bytes in an operand's lowest bits.)
      auto score = [&](int s, int buffer) {
        if (s == 0 && !barrier_wait(&sh.ring[0].full[key_stage], key_parity, gave_up)) return false;
        after_sync();
        const uint64_t a = q_operand + (uint32_t)(s * (128 * D * 2 >> 4)), k = key_operand + (uint32_t)(key_stage * (P::kStageBytes >> 4));
        if (leader) {
#pragma unroll
          for (int j = 0; j < D / 16; ++j)
            if constexpr (C::kQInTmem)
              mma_tmem(tmem + buffer * kN, tmem + P::kQColumn + j * 8, k + (uint32_t)(((j >> 2) * kPanel + (j & 3) * 32) >> 4), kScores, j > 0);
            else mma_shared(tmem + buffer * kN, a + (uint32_t)(((j >> 2) * kQPanel + (j & 3) * 32) >> 4),
                       k + (uint32_t)(((j >> 2) * kPanel + (j & 3) * 32) >> 4), kScores, j > 0);
          mma_commit(&sh.scores[buffer]);
          if (s == streams - 1) mma_commit(&sh.ring[0].empty[key_stage]);
        }
        __syncwarp();
        if (s == streams - 1 && ++key_stage == kStages) {
          key_stage = 0;
          key_parity ^= 1;
        }
        return true;
      };
      // The output of stream s from four of the tile's steps of 16 slots, from step `from` on.
      auto output = [&](int s, int t, int buffer, int from) {
        after_sync();
        const uint64_t v = value_operand + (uint32_t)(value_stage * (P::kStageBytes >> 4));
        if (leader) {
#pragma unroll
          for (int j = 0; j < 4; ++j)
            mma_tmem(tmem + P::kOutputs + s * D, tmem + buffer * kN + (from + j) * 8, v + (uint32_t)((from + j) * 16 * 128 >> 4), kOutput,
                     t > 0 || from + j > 0);
        }
        __syncwarp();
      };
      bool ok = true;
      if constexpr (kStreams == 1) {
        if (warp == kProducts) {
          ok = barrier_wait(&sh.q_there, 0, gave_up);
          int buffer = 0;
          uint32_t round = 1;  // parity of the round of buffers before
          for (int t = 0; ok && t < tiles; ++t) {
            // (the weights that were in this buffer are used up)
            if (t >= kBuffers) ok = barrier_wait(&sh.rest[buffer], round, gave_up);
            ok = ok && score(0, buffer);
            if (++buffer == kBuffers) {
              buffer = 0;
              round ^= 1;
            }
          }
        } else if (tiles > 0) {
          int buffer = 0;
          uint32_t round = 0;
          for (int t = 0; t < tiles; ++t) {
            ok = barrier_wait(&sh.ring[1].full[value_stage], value_parity, gave_up) && barrier_wait(&sh.weights[buffer], round, gave_up);
            if (!ok) break;
            output(0, t, buffer, 0);
            if (kN == 128) output(0, t, buffer, 4);
            if (leader) {
              mma_commit(&sh.rest[buffer]);
              mma_commit(&sh.ring[1].empty[value_stage]);
            }
            __syncwarp();
            if (++buffer == kBuffers) {
              buffer = 0;
              round ^= 1;
            }
            if (++value_stage == kStages) {
              value_stage = 0;
              value_parity ^= 1;
            }
          }
          if (leader) mma_commit(&sh.done);
          __syncwarp();
        }
      } else if (tiles > 0) {
        ok = barrier_wait(&sh.q_there, 0, gave_up);
        for (int s = 0; ok && s < streams; ++s) ok = score(s, s);
        for (int t = 0; ok && t < tiles; ++t) {
          for (int s = 0; ok && s < streams; ++s) {
            if (s == 0) ok = barrier_wait(&sh.ring[1].full[value_stage], value_parity, gave_up);
            ok = ok && barrier_wait(&sh.half[s], (uint32_t)t & 1, gave_up);
            if (!ok) break;
            output(s, t, s, 0);
            ok = barrier_wait(&sh.weights[s], (uint32_t)t & 1, gave_up);
            if (!ok) break;
            output(s, t, s, 4);
            if (s == streams - 1) {
              if (leader) mma_commit(&sh.ring[1].empty[value_stage]);
              __syncwarp();
            }
            if (t + 1 < tiles) ok = score(s, s);
          }
          if (++value_stage == kStages) {
            value_stage = 0;
            value_parity ^= 1;
          }
        }
        if (leader) mma_commit(&sh.done);
        __syncwarp();
      }
    }
    products_done();
  } else {
    // ---- softmax: a thread has one row
    if constexpr (kStreams == 2) asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(Many<D>::kRegistersSoftmax));
    if constexpr (C::kQInTmem) {
#pragma unroll
      for (int j = 0; j < kPieces; j += 8) {
        uint32_t w[32];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          w[4 * i] = early[j + i].x ^ flip;
          w[4 * i + 1] = early[j + i].y ^ flip;
          w[4 * i + 2] = early[j + i].z ^ flip;
          w[4 * i + 3] = early[j + i].w ^ flip;
        }
        tmem_store(tmem + ((uint32_t)((warp & 3) * 32) << 16) + P::kQColumn + j * 4, w);
      }
      tmem_stored();
      before_sync();
    } else {  // rows of q that are not there stay as they are: their scores go nowhere
      const int pieces = (m1 - m0) * kPieces;
      auto store_q = [&](int i, const uint4& x) {  // in the operand's layout
        const int m = i / kPieces, c = i % kPieces;
        for (int row = m & 127; row < 128; row += copy_rows)
          *(uint4*)(q_tile + (m >> 7) * (128 * D * 2) + (c >> 3) * kQPanel + row * 128 + (((c & 7) ^ (row & 7)) << 4)) =
              make_uint4(x.x ^ flip, x.y ^ flip, x.z ^ flip, x.w ^ flip);
      };
#pragma unroll
      for (int j = 0; j < kEarly; ++j)
        if (tid + j * kSoftmaxThreads < pieces) store_q(tid + j * kSoftmaxThreads, early[j]);
      for (int i = tid + kEarly * kSoftmaxThreads; i < pieces; i += kSoftmaxThreads) store_q(i, load_q(i));
      asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    }
    __syncwarp();
    if (lane == 0) barrier_arrive(&sh.q_there);
    const int s = warp >> 2, quarter = warp & 3, my_warps = s ? warps1 : warps0;
    const int m = m0 + s * 128 + place % copy_rows;
    float top = -INFINITY, sum = 0.f;  // the maximum that the row's weights were formed with, their sum
    const uint32_t lanes = (uint32_t)(quarter * 32) << 16, output = tmem + lanes + P::kOutputs + s * D;

    // The tiles of keys, W = kN / copies slots of each.
    auto all_tiles_of = [&](auto width) {
      constexpr int W = decltype(width)::value;
      const float scale = fabsf(p.scale_log2);
      const int r = min(m, m1 - 1) / p.group;  // (rows behind the last: as the last, and not written)
      const int depth = p.tree ? (int)sh.depth[r] : r;
      const int lo = p.window ? max(0, ctx + depth - p.window + 1) : 0;   // cached slots from lo on, and below `sinks`
      const int hi = min(keys.hi, p.tree ? ctx : ctx + r + 1);
      const int sinks = p.window ? min(p.sinks, hi) : 0;
      // what the first and the last row of the stream see of the cache bounds the tiles that need no mask
      const int first_m = m0 + s * 128, last_m = min(first_m + 128, m1) - 1;
      const int all_hi = min(keys.hi, p.tree ? ctx : ctx + first_m / p.group + 1);
      const int all_lo = p.window ? ctx + (p.tree ? p.R - 1 : last_m / p.group) - p.window + 1 : 0;
      int buffer = s;
      uint32_t round = 0;  // parity of the buffer's turn
      for (int t = 0; t < tiles; ++t) {
        const int tile_at = tile_start<kN>(keys, t0 + t), start = tile_at + copy * W;
        const uint32_t scores = tmem + lanes + buffer * kN;
        if (!barrier_wait(&sh.scores[buffer], round, gave_up)) break;
        after_sync();
        uint32_t x[W];
        if constexpr (W == 16) {
          tmem_load_16(scores + copy * W, x);
        } else {
#pragma unroll
          for (int c = 0; c < W; c += 32) tmem_load(scores + copy * W + c, x + c);
        }
        tmem_loaded();
        const bool whole = tile_at + kN <= all_hi && (tile_at >= all_lo || tile_at + kN <= p.sinks);
        if (!whole) {
          uint32_t see[(W + 31) / 32];
#pragma unroll
          for (int w = 0; w < (W + 31) / 32; ++w) {
            const int at = start + 32 * w;
            see[w] = bits_between(lo - at, hi - at) | bits_between(-at, sinks - at);
          }
          if (p.tree) {
            for (int n = r;; n = sh.parent[n]) {
              const int pos = ctx + (int)sh.depth[n], at = ctx + n - start;
              if (at >= 0 && at < W && ctx + n < keys.hi && (!p.window || pos >= lo || pos < p.sinks)) {
                const uint32_t bit = 1u << (at & 31);
#pragma unroll
                for (int w = 0; w < (W + 31) / 32; ++w) see[w] |= (at >> 5) == w ? bit : 0u;
              }
              if (n == 0) break;
            }
            __syncwarp();
          }
#pragma unroll
          for (int c = 0; c < W; ++c) x[c] = see[c >> 5] >> (c & 31) & 1u ? x[c] : 0xFF800000u;
          // Values of slots that no row of the block sees are whatever was there: 0 * NaN is no 0.  (Both streams
          // may write the same zeros.)
          bool any_dead = keys.dead(tile_at) || keys.dead(tile_at + kN - 1);
          if (!any_dead) any_dead = keys.sink_hi < keys.lo && keys.sink_hi < tile_at + kN && keys.lo > tile_at;
          if (any_dead) {
            if (!barrier_wait(&sh.ring[1].full[t % kStages], (uint32_t)(t / kStages) & 1, gave_up)) break;
            // the stream's warps share the tile's rows
            for (int n = place; n < kN; n += my_warps * 32)
              if (keys.dead(tile_at + n)) {
                char* v = value_ring + (t % kStages) * P::kStageBytes + n * 128;
#pragma unroll
                for (int c = 0; c < D / 64; ++c)
#pragma unroll
                  for (int j = 0; j < 8; ++j) *(uint4*)(v + c * kPanel + j * 16) = make_uint4(0, 0, 0, 0);
              }
            asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
            __syncwarp();
          }
        }
        float a[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
        for (int c = 0; c < W; c += 8)
#pragma unroll
          for (int j = 0; j < 4; ++j) a[j] = max3(a[j], __uint_as_float(x[c + 2 * j]), __uint_as_float(x[c + 2 * j + 1]));
        const float now = max3(fmaxf(a[0], a[1]), a[2], a[3]) * scale;
        const bool rise = now > top + kRise;  // (also from nothing seen to something)
        if (t == 0) {
          top = now;
        } else if (__any_sync(0xFFFFFFFFu, rise)) {
          // The output has to be at rest.  (In Many it is: this tile's scores come after the product with the last
          // weights.)
          if (kStreams == 1) {
            if (!barrier_wait(&sh.rest[buffer ? buffer - 1 : kBuffers - 1], buffer ? round : round ^ 1, gave_up)) break;
            after_sync();
          }
          const float f = rise ? power_of_two(top - now) : 1.0f;
          sum *= f;
          if (rise) top = now;
#pragma unroll 1
          for (int c = 0; c < D; c += 16) {
            uint32_t o[16];
            tmem_load_16(output + c, o);
            tmem_loaded();
#pragma unroll
            for (int j = 0; j < 16; ++j) o[j] = __float_as_uint(__uint_as_float(o[j]) * f);
            tmem_store_16(output + c, o);
          }
        }
        const float minus = top == -INFINITY ? 0.f : -top;
        const uint64_t scale_two = two(scale, scale), minus_two = two(minus, minus);
        uint64_t both[2] = {0, 0};
        constexpr int kStep = W == 16 ? 16 : 32;
#pragma unroll
        for (int c0 = 0; c0 < W; c0 += kStep) {
          uint32_t w[kStep / 2];
#pragma unroll
          for (int c = 0; c < kStep; c += 2) {
            float e0, e1;
            apart(fma_two(two(__uint_as_float(x[c0 + c]), __uint_as_float(x[c0 + c + 1])), scale_two, minus_two), e0, e1);
            e0 = power_of_two(e0);
            e1 = power_of_two(e1);
            both[c >> 1 & 1] = add_two(both[c >> 1 & 1], two(e0, e1));
            w[c >> 1] = pair(e0, e1);
          }
          if constexpr (W == 16) tmem_store_8(scores + copy * W / 2, w);
          else tmem_store_16(scores + (copy * W + c0) / 2, w);
          if (kStreams == 2 && c0 == 32) {
            tmem_stored();
            before_sync();
            __syncwarp();
            if (lane == 0) barrier_arrive(&sh.half[s]);
          }
        }
        // the other copies' slots have no weight in this one
        if (W < kN) {
          const uint32_t none[16] = {0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0};
#pragma unroll
          for (int c0 = 0; c0 < kN; c0 += kStep)
            if (c0 / W != copy) {
              if constexpr (W == 16) tmem_store_8(scores + c0 / 2, none);
              else tmem_store_16(scores + c0 / 2, none);
            }
        }
        float s0, s1;
        apart(add_two(both[0], both[1]), s0, s1);
        sum += s0 + s1;
        tmem_stored();
        before_sync();
        __syncwarp();
        if (lane == 0) barrier_arrive(&sh.weights[buffer]);
        if (kStreams == 2) {
          round ^= 1;
        } else if (++buffer == kBuffers) {
          buffer = 0;
          round ^= 1;
        }
      }
    };
    if (quarter < my_warps) {
      if constexpr (kStreams == 1) {
        if (copies == 4) all_tiles_of(std::integral_constant<int, kN / 4>());
        else if (copies == 2) all_tiles_of(std::integral_constant<int, kN / 2>());
        else all_tiles_of(std::integral_constant<int, kN>());
      } else {
        all_tiles_of(std::integral_constant<int, kN>());
      }
    }
    // ---- the end: every product is done, q's rows and the ring are free
    products_done();
    const bool wide = ((p.o_b | p.o_r | p.o_h) & 7) == 0 && ((uintptr_t)p.out & 15) == 0;
    if (quarter < my_warps) {
      if (*(volatile uint32_t*)gave_up) sum = __uint_as_float(0x7FC00000u);  // NaN: seen by whoever reads the output
      const float inv = sum == 0.f ? 0.f : 1.f / sum;
      const int r = m / p.group, g = m - r * p.group, at = s * 128 + place;
      __nv_bfloat16* out = (__nv_bfloat16*)p.out + b * p.o_b + r * p.o_r + (kv_head * p.group + g) * p.o_h;
#pragma unroll
      for (int c0 = 0; c0 < D; c0 += 64) {
        uint32_t o[64];
        if (tiles > 0) {
          tmem_load(output + c0, o);
          tmem_load(output + c0 + 32, o + 32);
          tmem_loaded();
        } else {
#pragma unroll
          for (int c = 0; c < 64; ++c) o[c] = 0;
        }
        if (m >= m1) continue;
        if (joins) {
#pragma unroll
          for (int c = 0; c < 64; c += 4) *(uint4*)(parts + at * P::kPartRow + c0 + c) = make_uint4(o[c], o[c + 1], o[c + 2], o[c + 3]);
        } else {
#pragma unroll
          for (int c = 0; c < 64; c += 8) {
            uint32_t w[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) w[j] = pair(__uint_as_float(o[c + 2 * j]) * inv, __uint_as_float(o[c + 2 * j + 1]) * inv);
            if (wide) {
              *(uint4*)(out + c0 + c) = make_uint4(w[0], w[1], w[2], w[3]);
            } else {
#pragma unroll
              for (int j = 0; j < 8; ++j) ((unsigned short*)out)[c0 + c + j] = (unsigned short)(w[j >> 1] >> (16 * (j & 1)));
            }
          }
        }
      }
      if (joins) {
        tops[at] = top;
        sums[at] = sum;
      }
    }
  }

  // ---- the copies' outputs into the first copy's place: out = sum_c 2^(top_c - top) o_c, and so the sums
  if (copies > 1) {
    __syncthreads();
    for (int i = tid; i < (m1 - m0) * (D / 4); i += C::kThreads) {  // (D / 4 divides 32: a row's threads are in one warp)
      const int row = i / (D / 4), d = (i % (D / 4)) * 4;
      float most = -INFINITY, total = 0.f;
      for (int c = 0; c < copies; ++c) most = fmaxf(most, tops[row + c * copy_rows]);
      const float from = most == -INFINITY ? 0.f : most;
      float4 y = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
      for (int c = 0; c < 4; ++c) {
        if (c >= copies) break;
        const float theirs = sums[row + c * copy_rows];
        if (theirs == 0.f) continue;  // saw nothing
        const float f = power_of_two(tops[row + c * copy_rows] - from);
        const float4 x = *(const float4*)(parts + (row + c * copy_rows) * P::kPartRow + d);
        total = fmaf(f, theirs, total);
        y.x = fmaf(f, x.x, y.x);
        y.y = fmaf(f, x.y, y.y);
        y.z = fmaf(f, x.z, y.z);
        y.w = fmaf(f, x.w, y.w);
      }
      if (p.split > 1) {
        __syncwarp(D == 128 ? 0xFFFFFFFFu : lane < 16 ? 0xFFFFu : 0xFFFF0000u);  // (all have read the row's tops and sums)
        *(float4*)(parts + row * P::kPartRow + d) = y;
        if (d == 0) {
          tops[row] = most;
          sums[row] = total;
        }
      } else {
        write_row(row, d, y, total);
      }
    }
  }
  if (p.split > 1) {
    cg::cluster_group cluster = cg::this_cluster();
    __syncwarp();
    cluster.sync();
    // Join the blocks' outputs: out = sum_c 2^(top_c - top) o_c / sum_c 2^(top_c - top) sum_c.  Rows are dealt out
    // over the cluster's warps; lane c works out block c's factor, then a lane joins four columns (or, where a head
    // has 64, half a warp a row's half of the blocks).
    constexpr int kD4 = D / 4, kGroups = 32 / kD4;
    for (int row = warp * p.split + part; row < m1 - m0; row += (C::kThreads / 32) * p.split) {
      float their_top = -INFINITY, their_sum = 0.f;
      if (lane < p.split) {
        their_top = *cluster.map_shared_rank(&tops[row], lane);
        their_sum = *cluster.map_shared_rank(&sums[row], lane);
      }
      float most = their_top;
#pragma unroll
      for (int w = 8; w; w >>= 1) most = fmaxf(most, __shfl_xor_sync(0xFFFFFFFFu, most, w));
      if (most == -INFINITY) most = 0.f;
      float f = lane < p.split && their_sum != 0.f ? power_of_two(their_top - most) : 0.f;  // (0: saw nothing)
      float total = f != 0.f || their_sum != their_sum ? f * their_sum : 0.f;
#pragma unroll
      for (int w = 8; w; w >>= 1) total += __shfl_xor_sync(0xFFFFFFFFu, total, w);
      total = __shfl_sync(0xFFFFFFFFu, total, 0);  // (lanes 0 to 15 hold the sum)
      const int d = (lane % kD4) * 4, first = lane / kD4;
      float4 y = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 4
      for (int c0 = 0; c0 < p.split; c0 += kGroups) {
        const int c = c0 + first;
        const float g = __shfl_sync(0xFFFFFFFFu, f, c & 31);
        if (c < p.split && g != 0.f) {
          const float4 x = *(const float4*)cluster.map_shared_rank(&parts[row * P::kPartRow + d], c);
          y.x = fmaf(g, x.x, y.x);
          y.y = fmaf(g, x.y, y.y);
          y.z = fmaf(g, x.z, y.z);
          y.w = fmaf(g, x.w, y.w);
        }
      }
      if (kGroups == 2) {
        y.x += __shfl_xor_sync(0xFFFFFFFFu, y.x, 16);
        y.y += __shfl_xor_sync(0xFFFFFFFFu, y.y, 16);
        y.z += __shfl_xor_sync(0xFFFFFFFFu, y.z, 16);
        y.w += __shfl_xor_sync(0xFFFFFFFFu, y.w, 16);
      }
      if (first == 0) write_row(row, d, y, total);
    }
    __syncwarp();
    cluster.sync();  // (no block ends while another reads its shared memory)
  }
  before_sync();
  __syncthreads();
  if (warp == kProducts) {
    after_sync();
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "n"(C::kColumns) : "memory");
  }
}

// ---------------------------------------------------------------------------------------------------- host side
using Encode = decltype(&cuTensorMapEncodeTiled);

Encode encode_function() {
  static Encode f = [] {
    void* at = nullptr;
    cudaDriverEntryPointQueryResult r;
    if (cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &at, cudaEnableDefault, &r) != cudaSuccess || r != cudaDriverEntryPointSuccess) {
      (void)cudaGetLastError();
      at = nullptr;
    }
    return (Encode)at;
  }();
  return f;
}

// The map of one side of the cache: [pages, heads, positions of a page, D], boxes of `box` positions by 64 elements.
bool encode(CUtensorMap* map, const void* at, int D, const AttentionParams& p, int64_t token, int64_t head, int64_t page, int box) {
  const cuuint64_t dims[4] = {(cuuint64_t)D, (cuuint64_t)p.page_size, (cuuint64_t)p.heads, (cuuint64_t)p.num_pages};
  // (the stride of a dimension of one is free: the map wants a multiple of 16 bytes all the same)
  if (p.heads == 1) head = D;
  if (p.num_pages == 1) page = D;
  if (token <= 0 || head <= 0 || page <= 0 || ((token | head | page) & 7) || !aligned_to(at, 16)) return false;
  const cuuint64_t strides[3] = {(cuuint64_t)token * 2, (cuuint64_t)head * 2, (cuuint64_t)page * 2};
  const cuuint32_t boxes[4] = {64, (cuuint32_t)box, 1, 1}, steps[4] = {1, 1, 1, 1};
  for (const cuuint64_t s : strides)
    if (s >= (cuuint64_t)1 << 40) return false;
  return encode_function()(map, CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 4, const_cast<void*>(at), dims, strides, boxes, steps,
                           CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                           CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

struct TensorBuild {
  const void* kernel;
  int smem, rows, threads, slots;
};
template <typename C>
TensorBuild tensor_build() {
  return {(const void*)attention_tensor_kernel<C>, Plan<C>::kSmem, Plan<C>::kRows, C::kThreads, C::kN};
}

// What a build needs before its first launch on a device; clusters[n]: how many clusters of n blocks, n <= 16, the
// device holds at a time.
int prepare_build(const TensorBuild& k, int at, const int** clusters) {
  static std::mutex m;
  static int known[6][64][17];
  int dev = 0;
  cudaError_t e = cudaGetDevice(&dev);
  if (e != cudaSuccess) return cuda_fail(e);
  if (dev < 0 || dev >= 64) return ERSD_EUNSUPPORTED;
  std::lock_guard<std::mutex> lock(m);
  int* n = known[at][dev];
  if (!n[0]) {
    e = cudaFuncSetAttribute(k.kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, k.smem);
    if (e != cudaSuccess) return cuda_fail(e);
    (void)cudaFuncSetAttribute(k.kernel, cudaFuncAttributeNonPortableClusterSizeAllowed, 1);
    for (int i = 2; i <= 16; ++i) {
      Launch l(dim3((unsigned)i, 1, 1), (unsigned)k.threads, (size_t)k.smem, nullptr, (unsigned)i);
      l.cfg.attrs = &l.at[1];  // (the cluster's size alone)
      l.cfg.numAttrs = 1;
      if (cudaOccupancyMaxActiveClusters(&n[i], k.kernel, &l.cfg) != cudaSuccess) n[i] = 0;
    }
    (void)cudaGetLastError();  // a size that is refused fits no time
    n[0] = 1;
  }
  *clusters = n;
  return ERSD_OK;
}

}  // namespace

int launch_attention_tensor(AttentionParams& p, int max_context, cudaStream_t st) {
  if ((p.dim != 64 && p.dim != 128) || p.page_size % 4 || !encode_function()) return ERSD_EUNSUPPORTED;
  const int64_t sms = sm_count();
  const bool many = (int64_t)p.R * p.group > 128;
  p.row_tiles = (int)(((int64_t)p.R * p.group + (many ? 255 : 127)) / (many ? 256 : 128));
  const int64_t units = (int64_t)p.row_tiles * p.heads * p.B;
  // Blocks with a long ring while no more than one goes to an SM (18 sequences of 32000 to 64000 positions, 144
  // blocks, when the two were compared: 620 us, and 1150 with the shorter rings and one block to an SM),
  // else two to an SM.
  const bool alone = many || units * (p.split ? p.split : 1) <= sms;
  const int at = (p.dim == 64 ? 0 : 3) + (many ? 2 : alone ? 1 : 0);
  const TensorBuild builds[6] = {tensor_build<Few<64, 2>>(),  tensor_build<Few<64, 1>>(),  tensor_build<Many<64>>(),
                                 tensor_build<Few<128, 2>>(), tensor_build<Few<128, 1>>(), tensor_build<Many<128>>()};
  const TensorBuild& k = builds[at];
  int box = 4;
  while (box < k.slots && p.page_size % (box * 2) == 0) box *= 2;
  CUtensorMap k_map, v_map;
  if (!encode(&k_map, p.k, p.dim, p, p.k_token, p.k_head, p.k_page, box) || !encode(&v_map, p.v, p.dim, p, p.v_token, p.v_head, p.v_page, box))
    return ERSD_EUNSUPPORTED;
  const int* clusters;
  const int status = prepare_build(k, at, &clusters);
  if (status != ERSD_OK) return status;
  if (!p.split) {
    // as many blocks as SMs, with a tile of keys at least for each, and no cluster that has to wait for another
    int64_t reach = (int64_t)max_context + p.R;
    if (p.window && reach > (int64_t)p.window + p.sinks + p.R) reach = (int64_t)p.window + p.sinks + p.R;
    const int64_t tiles = (reach + k.slots - 1) / k.slots;
    p.split = 1;
    for (int n = 2; n <= 16 && units * n <= sms && n <= tiles; ++n)
      if (units <= clusters[n]) p.split = n;
  }
  while (p.split > 1 && !clusters[p.split]) --p.split;
  note_launch("attention_tensor_kernel<%d, %d rows>: %d threads x (%d, %d, %d) blocks, %d to a tile of rows, boxes of %d", p.dim, k.rows,
              k.threads, p.row_tiles * p.split, p.heads, p.B, p.split, box);
  Launch l(dim3((unsigned)(p.row_tiles * p.split), (unsigned)p.heads, (unsigned)p.B), (unsigned)k.threads, (size_t)k.smem, st, (unsigned)p.split);
  void* args[] = {(void*)&p, (void*)&k_map, (void*)&v_map, (void*)&box};
  const cudaError_t e = cudaLaunchKernelExC(&l.cfg, k.kernel, args);
  return e == cudaSuccess ? ERSD_OK : cuda_fail(e);
}

}  // namespace ersd
