// ersd_chunk_attention: checks, the choice of the kernel, and the kernels of 32-bit arithmetic.
//
// Up to 48 packed rows (see AttentionParams and few_rows), where the cache's bytes are to bound the call: rows_kernel takes four.
// L lanes share a slot, eight elements of its key and value in registers each, so that a warp has 32 / L slots at a
// time and every warp goes through its own slots without waiting for another: the lanes' parts of the scores are
// summed and dealt out by a few exchanges (lane r ends with row r's), lane r weighs row r's, and each lane adds its
// part of the value to its part of the outputs.  What the slots' lanes, the warps and, with
// `split` blocks to a cluster, the blocks have is joined at the end through shared memory.
//
// More rows, where the multiplications do: tile_kernel takes 64 rows through the keys, kNK slots at a time: keys and
// values are copied to shared memory as floats, a thread forms the scores of four slots with four rows, the
// softmax's running maximum and sum live in shared memory, and a thread holds four columns of several rows of the
// output in registers.  `split` blocks join their partial results through distributed shared memory.
//
// Measured on one B200, float32, 8 sequences behind up to 777 positions, 16 heads of 64: chains of five rows 25 us (their
// bytes 6: warps wait, a third of the time for memory, 8 of them to an SM, and five rows go through the cache twice; an
// instruction is issued in a quarter of the cycles), 30 rows 51 us.  tile_kernel: 2 x 700 rows behind 2000 positions, 16 heads
// of 64, 604 us, 15 TFLOP/s; 16/4 heads of 128 1052 us, 17.
#include <cooperative_groups.h>
#include <cuda_bf16.h>
#include <math.h>

#include "ersd_attention.cuh"

namespace cg = cooperative_groups;

namespace ersd {

namespace {

constexpr int kNK = 64;       // slots of a tile
constexpr int kThreads = 256;

template <typename T>
__device__ __forceinline__ float as_float(T x);
template <>
__device__ __forceinline__ float as_float<float>(float x) { return x; }
template <>
__device__ __forceinline__ float as_float<__nv_bfloat16>(__nv_bfloat16 x) { return __bfloat162float(x); }

// Four elements from `at` on as floats; `wide`: all four exist and lie on a boundary of their size.
template <typename T>
__device__ __forceinline__ float4 four(const T* at, int left, bool wide) {
  float4 f = make_float4(0.f, 0.f, 0.f, 0.f);
  if (wide) {
    if constexpr (sizeof(T) == 4) {
      f = *(const float4*)at;
    } else {
      const uint2 w = *(const uint2*)at;
      f.x = __uint_as_float(w.x << 16);
      f.y = __uint_as_float(w.x & 0xFFFF0000u);
      f.z = __uint_as_float(w.y << 16);
      f.w = __uint_as_float(w.y & 0xFFFF0000u);
    }
  } else {
    if (left > 0) f.x = as_float(at[0]);
    if (left > 1) f.y = as_float(at[1]);
    if (left > 2) f.z = as_float(at[2]);
    if (left > 3) f.w = as_float(at[3]);
  }
  return f;
}

// Whether row r (-1: none) sees a slot; `above`: a tree's nodes that it sees.
__device__ __forceinline__ bool sees(const AttentionParams& p, const KeyRange& keys, int ctx, int slot, int r, const uint32_t* above) {
  if (r < 0 || slot >= keys.hi) return false;
  if (!p.tree) return slot <= ctx + r && (!p.window || slot > ctx + r - p.window || slot < p.sinks);
  if (slot < ctx) return !p.window || slot > ctx + (int)p.depth[r] - p.window || slot < p.sinks;
  const int node = slot - ctx;
  return above[node >> 5] >> (node & 31) & 1u;
}
// The nodes of a tree that row r sees.
__device__ __forceinline__ void nodes_above(const AttentionParams& p, int ctx, int r, uint32_t* above) {
  uint32_t w[ERSD_MAX_ROWS / 32];
#pragma unroll
  for (int j = 0; j < ERSD_MAX_ROWS / 32; ++j) w[j] = 0;
  if (r >= 0) {
    for (int n = r;; n = p.parent[n]) {
      const int pos = ctx + p.depth[n];
      if (!p.window || p.depth[n] > (int)p.depth[r] - p.window || pos < p.sinks) w[n >> 5] |= 1u << (n & 31);
      if (n == 0) break;
    }
  }
#pragma unroll
  for (int j = 0; j < ERSD_MAX_ROWS / 32; ++j) above[j] = w[j];
}

template <int MR, int DP>
struct Shared {
  float q[MR][DP + 4];   // (+4: a warp's 16-byte reads of several rows or slots fall on other banks)
  float k[kNK][DP + 4];
  float v[kNK][DP];
  float s[MR][kNK + 4];
  float top[MR], sum[MR], factor[MR];  // running maximum, sum, and what the output is scaled by this tile
  int row[MR];                         // row of the chunk, or -1
  uint32_t above[MR][ERSD_MAX_ROWS / 32];  // tree: nodes the row sees
};

// MR packed rows, DP >= dim columns (a multiple of 64).
template <typename T, int MR, int DP>
__global__ void __launch_bounds__(kThreads) tile_kernel(const AttentionParams p, bool wide) {
  extern __shared__ __align__(16) char raw[];
  Shared<MR, DP>& sh = *(Shared<MR, DP>*)raw;
  const int tid = threadIdx.x, kv_head = blockIdx.y, b = blockIdx.z;
  const int tile = blockIdx.x / p.split, part = blockIdx.x - tile * p.split;
  asm volatile("griddepcontrol.wait;" ::: "memory");
  int rows = p.row_counts ? p.row_counts[b] : p.R;
  rows = max(0, min(rows, p.R));
  const int m0 = tile * MR, m1 = min(m0 + MR, rows * p.group);
  if (m0 >= m1) return;  // (the same for every block of the cluster)
  const int ctx = context_of(p, b);
  const int r0 = m0 / p.group, r1 = (m1 - 1) / p.group + 1;

  constexpr int kD4 = DP / 4;
  for (int i = tid; i < MR * kD4; i += kThreads) {
    const int m = i / kD4, d = (i - m * kD4) * 4, r = (m0 + m) / p.group, g = m0 + m - r * p.group;
    float4 f = make_float4(0.f, 0.f, 0.f, 0.f);
    if (m0 + m < m1)
      f = four((const T*)p.q + b * p.q_b + r * p.q_r + (kv_head * p.group + g) * p.q_h + d, p.dim - d, wide && d + 4 <= p.dim);
    f.x *= p.scale_log2;
    f.y *= p.scale_log2;
    f.z *= p.scale_log2;
    f.w *= p.scale_log2;
    *(float4*)&sh.q[m][d] = f;
  }
  for (int m = tid; m < MR; m += kThreads) {
    const int r = m0 + m < m1 ? (m0 + m) / p.group : -1;
    sh.row[m] = r;
    sh.top[m] = -INFINITY;
    sh.sum[m] = 0.f;
    sh.factor[m] = 0.f;
    if (p.tree) nodes_above(p, ctx, r, sh.above[m]);
  }
  int min_depth = r0;
  if (p.tree) {
    min_depth = p.depth[r0];
    for (int r = r0 + 1; r < r1; ++r) min_depth = min(min_depth, (int)p.depth[r]);
  }
  const KeyRange keys = key_range<kNK>(p, ctx, r1, min_depth);
  const int t0 = (int)((int64_t)keys.tiles * part / p.split), t1 = (int)((int64_t)keys.tiles * (part + 1) / p.split);
  const int32_t* table = p.table + b * p.table_stride;
  const T* K = (const T*)p.k + kv_head * p.k_head;
  const T* V = (const T*)p.v + kv_head * p.v_head;

  // a thread's part of the output: four columns of every kRowStep-th row
  constexpr int kRowStep = kThreads / kD4, kOut = (MR + kRowStep - 1) / kRowStep;
  const int oc = (tid % kD4) * 4, om = tid / kD4;
  float4 o[kOut];
#pragma unroll
  for (int i = 0; i < kOut; ++i) o[i] = make_float4(0.f, 0.f, 0.f, 0.f);
  __syncthreads();

  for (int t = t0; t < t1; ++t) {
    const int start = tile_start<kNK>(keys, t);
    // slots that no row sees are not read: their values could be anything, and 0 * NaN is no 0
    for (int i = tid; i < kNK * kD4; i += kThreads) {
      const int n = i / kD4, d = (i - n * kD4) * 4, slot = start + n;
      float4 fk = make_float4(0.f, 0.f, 0.f, 0.f), fv = fk;
      if (!keys.dead(slot)) {
        const int entry = page_of(p, slot), page = table[entry];
        if (page >= 0 && page < p.num_pages) {
          const int in_page = slot - entry * p.page_size;
          fk = four(K + page * p.k_page + in_page * p.k_token + d, p.dim - d, wide && d + 4 <= p.dim);
          fv = four(V + page * p.v_page + in_page * p.v_token + d, p.dim - d, wide && d + 4 <= p.dim);
        }
      }
      *(float4*)&sh.k[n][d] = fk;
      *(float4*)&sh.v[n][d] = fv;
    }
    __syncthreads();
    {
      // a thread: slots x, x + 16, ..; rows 4 y to 4 y + 3
      static_assert(MR == 64 && kNK == 64 && kThreads == 256, "");
      const int x = tid & 15, y = tid >> 4;
      float s[4][4];
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) s[i][j] = 0.f;
      for (int d = 0; d < DP; d += 4) {
        float4 fq[4], fk[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) fq[i] = *(const float4*)&sh.q[y * 4 + i][d];
#pragma unroll
        for (int j = 0; j < 4; ++j) fk[j] = *(const float4*)&sh.k[x + 16 * j][d];
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            s[i][j] = fmaf(fq[i].x, fk[j].x, s[i][j]);
            s[i][j] = fmaf(fq[i].y, fk[j].y, s[i][j]);
            s[i][j] = fmaf(fq[i].z, fk[j].z, s[i][j]);
            s[i][j] = fmaf(fq[i].w, fk[j].w, s[i][j]);
          }
      }
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const int m = y * 4 + i, n = x + 16 * j;
          sh.s[m][n] = sees(p, keys, ctx, start + n, sh.row[m], sh.above[m]) ? s[i][j] : -INFINITY;
        }
    }
    __syncthreads();
    // a warp takes whole rows: maximum, weights, sum
    for (int m = tid >> 5; m < MR; m += kThreads / 32) {
      const int lane = tid & 31;
      float a = sh.s[m][lane], c = sh.s[m][lane + 32];
      float top = fmaxf(a, c);
#pragma unroll
      for (int w = 16; w; w >>= 1) top = fmaxf(top, __shfl_xor_sync(0xFFFFFFFFu, top, w));
      const float before = sh.top[m];
      top = fmaxf(top, before);
      const float at = top == -INFINITY ? 0.f : top;  // (nothing seen yet: weights of 0, not NaN)
      a = exp2f(a - at);
      c = exp2f(c - at);
      float sum = a + c;
#pragma unroll
      for (int w = 16; w; w >>= 1) sum += __shfl_xor_sync(0xFFFFFFFFu, sum, w);
      sh.s[m][lane] = a;
      sh.s[m][lane + 32] = c;
      __syncwarp();
      if (lane == 0) {
        const float f = exp2f(before - at);
        sh.factor[m] = f;
        sh.sum[m] = sh.sum[m] * f + sum;
        sh.top[m] = top;
      }
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < kOut; ++i) {
      const int m = om + i * kRowStep;
      const float f = m < MR ? sh.factor[m] : 0.f;
      o[i].x *= f;
      o[i].y *= f;
      o[i].z *= f;
      o[i].w *= f;
    }
    for (int n = 0; n < kNK; n += 4) {
      float4 fv[4];
#pragma unroll
      for (int j = 0; j < 4; ++j) fv[j] = *(const float4*)&sh.v[n + j][oc];
#pragma unroll
      for (int i = 0; i < kOut; ++i) {
        const int m = om + i * kRowStep;
        if (MR % kRowStep && m >= MR) continue;
        const float4 w = *(const float4*)&sh.s[m][n];
        const float ws[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          o[i].x = fmaf(ws[j], fv[j].x, o[i].x);
          o[i].y = fmaf(ws[j], fv[j].y, o[i].y);
          o[i].z = fmaf(ws[j], fv[j].z, o[i].z);
          o[i].w = fmaf(ws[j], fv[j].w, o[i].w);
        }
      }
    }
    __syncthreads();
  }

  // Join the parts: out = sum_c 2^(top_c - top) o_c / sum_c 2^(top_c - top) sum_c.
  float* mine = &sh.k[0][0];  // [MR][DP] of this block, where the keys and values were
  static_assert(sizeof(float) * MR * DP <= sizeof sh.k + sizeof sh.v, "");
  if (p.split > 1) {
    cg::cluster_group cluster = cg::this_cluster();
#pragma unroll
    for (int i = 0; i < kOut; ++i) {
      const int m = om + i * kRowStep;
      if (m < MR) *(float4*)&mine[m * DP + oc] = o[i];
    }
    cluster.sync();
    // rows are dealt out over the cluster's blocks; a thread joins its four columns
    for (int i = tid + part * kThreads; i < (m1 - m0) * kD4; i += kThreads * p.split) {
      const int m = i / kD4, d = (i - m * kD4) * 4;
      float top = -INFINITY;
      for (int c = 0; c < p.split; ++c) top = fmaxf(top, *cluster.map_shared_rank(&sh.top[m], c));
      if (top == -INFINITY) top = 0.f;
      float sum = 0.f;
      float4 a = make_float4(0.f, 0.f, 0.f, 0.f);
      for (int c = 0; c < p.split; ++c) {
        const float theirs = *cluster.map_shared_rank(&sh.sum[m], c);
        if (theirs == 0.f) continue;  // saw nothing
        const float f = exp2f(*cluster.map_shared_rank(&sh.top[m], c) - top);
        sum = fmaf(f, theirs, sum);
        const float4 x = *(const float4*)cluster.map_shared_rank(&mine[m * DP + d], c);
        a.x = fmaf(f, x.x, a.x);
        a.y = fmaf(f, x.y, a.y);
        a.z = fmaf(f, x.z, a.z);
        a.w = fmaf(f, x.w, a.w);
      }
      const float inv = sum > 0.f || sum != sum ? 1.f / sum : 0.f;
      const int r = (m0 + m) / p.group, g = m0 + m - r * p.group;
      T* out = (T*)p.out + b * p.o_b + r * p.o_r + (kv_head * p.group + g) * p.o_h + d;
      const float x[4] = {a.x * inv, a.y * inv, a.z * inv, a.w * inv};
      for (int j = 0; j < 4; ++j)
        if (d + j < p.dim) out[j] = (T)x[j];
    }
    cluster.sync();  // (no block ends while another reads its shared memory)
    return;
  }
#pragma unroll
  for (int i = 0; i < kOut; ++i) {
    const int m = om + i * kRowStep;
    if (m >= m1 - m0) continue;
    const float sum = sh.sum[m], inv = sum > 0.f || sum != sum ? 1.f / sum : 0.f;
    const int r = (m0 + m) / p.group, g = m0 + m - r * p.group;
    T* out = (T*)p.out + b * p.o_b + r * p.o_r + (kv_head * p.group + g) * p.o_h + oc;
    const float x[4] = {o[i].x * inv, o[i].y * inv, o[i].z * inv, o[i].w * inv};
    for (int j = 0; j < 4; ++j)
      if (oc + j < p.dim) out[j] = (T)x[j];
  }
}

// ---- few rows
// (eight rows to a warp: 30 us instead of 24 for chains of five, for want of registers)
constexpr int kRows = 4, kRowWarps = 4, kAhead = 2;  // kAhead: steps whose keys and values a warp asks for at once

template <int L, int MR>
struct RowShared {
  static constexpr int kParts = kRowWarps * (32 / L), DP = 8 * L;
  float o[kParts][MR][DP];
  float top[kParts][MR], sum[kParts][MR];
  float joined[MR][DP];
  float joined_top[MR], joined_sum[MR];
  int row[MR];
  uint32_t above[MR][ERSD_MAX_ROWS / 32];
};

// Eight elements of a row from `at` on as floats; `wide`: on a boundary of 16 bytes (and the row goes on that far).
template <typename T>
__device__ __forceinline__ void eight(const T* at, int left, bool wide, float* f) {
  if (wide && left >= 8) {
    if constexpr (sizeof(T) == 4) {
      const float4 a = *(const float4*)at, b = *((const float4*)at + 1);
      f[0] = a.x, f[1] = a.y, f[2] = a.z, f[3] = a.w, f[4] = b.x, f[5] = b.y, f[6] = b.z, f[7] = b.w;
    } else {
      const uint4 w = *(const uint4*)at;
      const uint32_t v[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        f[2 * i] = __uint_as_float(v[i] << 16);
        f[2 * i + 1] = __uint_as_float(v[i] & 0xFFFF0000u);
      }
    }
  } else {
#pragma unroll
    for (int i = 0; i < 8; ++i) f[i] = i < left ? as_float(at[i]) : 0.f;
  }
}

// MR packed rows, heads of up to 8 L.
template <typename T, int L, int MR>
__global__ void __launch_bounds__(32 * kRowWarps, 4) rows_kernel(const AttentionParams p, bool wide) {
  constexpr int kSlots = 32 / L, kTile = kSlots * kRowWarps * kAhead, DP = 8 * L;
  extern __shared__ __align__(16) char raw[];
  RowShared<L, MR>& sh = *(RowShared<L, MR>*)raw;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, kv_head = blockIdx.y, b = blockIdx.z;
  const int j = lane % L, g = lane / L, first_lane = lane - j;  // part of the slot's elements, slot of the step
  const int tile = blockIdx.x / p.split, part = blockIdx.x - tile * p.split;
  asm volatile("griddepcontrol.wait;" ::: "memory");
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  int rows = p.row_counts ? p.row_counts[b] : p.R;
  const int ctx = context_of(p, b);
  rows = max(0, min(rows, p.R));
  const int m0 = tile * MR, m1 = min(m0 + MR, rows * p.group);
  if (m0 >= m1) return;  // (the same for every block of the cluster)
  const int r0 = m0 / p.group, r1 = (m1 - 1) / p.group + 1;
  float q[MR][8];
#pragma unroll
  for (int m = 0; m < MR; ++m) {
    const int r = (m0 + m) / p.group, h = kv_head * p.group + m0 + m - r * p.group;
    const bool there = m0 + m < m1;
    eight((const T*)p.q + b * p.q_b + (there ? r * p.q_r + h * p.q_h : 0) + j * 8, there ? p.dim - j * 8 : 0, wide, q[m]);
#pragma unroll
    for (int i = 0; i < 8; ++i) q[m][i] = there ? q[m][i] * p.scale_log2 : 0.f;
  }
  if (tid < MR) {
    const int r = m0 + tid < m1 ? (m0 + tid) / p.group : -1;
    sh.row[tid] = r;
    if (p.tree) nodes_above(p, ctx, r, sh.above[tid]);
  }
  int min_depth = r0;
  if (p.tree) {
    min_depth = p.depth[r0];
    for (int r = r0 + 1; r < r1; ++r) min_depth = min(min_depth, (int)p.depth[r]);
  }
  __syncthreads();
  const KeyRange keys = key_range<kTile>(p, ctx, r1, min_depth);
  const int t0 = (int)((int64_t)keys.tiles * part / p.split), t1 = (int)((int64_t)keys.tiles * (part + 1) / p.split);
  const int32_t* table = p.table + b * p.table_stride;
  const T* K = (const T*)p.k + kv_head * p.k_head + j * 8;
  const T* V = (const T*)p.v + kv_head * p.v_head + j * 8;
  const int my_row = sh.row[j & (MR - 1)];
  const uint32_t* above = sh.above[j & (MR - 1)];
  // step u of tile t: slot of this lane, and its page (-1: none, or no row sees it)
  auto slot_of = [&](int t, int u) { return tile_start<kTile>(keys, t) + (u * kRowWarps + warp) * kSlots + g; };
  auto page_at = [&](int t, int u) {
    if (t >= t1) return -1;
    const int slot = slot_of(t, u);
    if (keys.dead(slot)) return -1;
    const int page = table[page_of(p, slot)];
    return page < p.num_pages ? max(page, -1) : -1;
  };
  float o[MR][8];
#pragma unroll
  for (int m = 0; m < MR; ++m)
#pragma unroll
    for (int i = 0; i < 8; ++i) o[m][i] = 0.f;
  float top = -INFINITY, sum = 0.f;  // of row j & (MR - 1) over this lane's slots
  int page[kAhead];
#pragma unroll
  for (int u = 0; u < kAhead; ++u) page[u] = page_at(t0, u);
  for (int t = t0; t < t1; ++t) {
    float k[kAhead][8], v[kAhead][8];
#pragma unroll
    for (int u = 0; u < kAhead; ++u) {
      // (slots that no row sees are not read: their values could be anything, and 0 * NaN is no 0)
      const int slot = slot_of(t, u), token = page[u] < 0 ? 0 : slot - page_of(p, slot) * p.page_size, left = page[u] < 0 ? 0 : p.dim - j * 8;
      const int64_t at = max(page[u], 0);
      eight(K + at * p.k_page + token * p.k_token, left, wide, k[u]);
      eight(V + at * p.v_page + token * p.v_token, left, wide, v[u]);
    }
#pragma unroll
    for (int u = 0; u < kAhead; ++u) page[u] = page_at(t + 1, u);
#pragma unroll
    for (int u = 0; u < kAhead; ++u) {
      const int slot = slot_of(t, u);
      float s[MR];
#pragma unroll
      for (int m = 0; m < MR; ++m) {
        s[m] = q[m][0] * k[u][0];
#pragma unroll
        for (int i = 1; i < 8; ++i) s[m] = fmaf(q[m][i], k[u][i], s[m]);
      }
      // sums over the slot's lanes, row r's to lanes r, r + MR, ..
#pragma unroll
      for (int half = MR / 2; half; half >>= 1) {
        const bool upper = j & half;
#pragma unroll
        for (int m = 0; m < half; ++m) {
          const float send = upper ? s[m] : s[m + half], keep = upper ? s[m + half] : s[m];
          s[m] = keep + __shfl_xor_sync(0xFFFFFFFFu, send, half);
        }
      }
#pragma unroll
      for (int w = MR; w < L; w <<= 1) s[0] += __shfl_xor_sync(0xFFFFFFFFu, s[0], w);
      const float x = sees(p, keys, ctx, slot, my_row, above) ? s[0] : -INFINITY;
      // the output is scaled only when a maximum has risen by more than 2^8: weights are then 2^8 at most
      const bool rise = x > top + 8.0f;
      if (__any_sync(0xFFFFFFFFu, rise)) {
        const float f = rise ? exp2f(top - x) : 1.0f;
        sum *= f;
        if (rise) top = x;
#pragma unroll
        for (int m = 0; m < MR; ++m) {
          const float fm = __shfl_sync(0xFFFFFFFFu, f, first_lane + m);
#pragma unroll
          for (int i = 0; i < 8; ++i) o[m][i] *= fm;
        }
      }
      const float weight = exp2f(x - (top == -INFINITY ? 0.f : top));
      sum += weight;
#pragma unroll
      for (int m = 0; m < MR; ++m) {
        const float w = __shfl_sync(0xFFFFFFFFu, weight, first_lane + m);
#pragma unroll
        for (int i = 0; i < 8; ++i) o[m][i] = fmaf(w, v[u][i], o[m][i]);
      }
    }
  }

  // Join: out = sum_c 2^(top_c - top) o_c / sum_c 2^(top_c - top) sum_c over the slots' lanes and the warps ...
  {
    const int c = warp * kSlots + g;
#pragma unroll
    for (int m = 0; m < MR; ++m)
#pragma unroll
      for (int i = 0; i < 8; i += 4) *(float4*)&sh.o[c][m][j * 8 + i] = make_float4(o[m][i], o[m][i + 1], o[m][i + 2], o[m][i + 3]);
    if (j < MR) {
      sh.top[c][j] = top;
      sh.sum[c][j] = sum;
    }
  }
  __syncthreads();
  auto write = [&](int m, int d, const float4& y, float total) {
    const float inv = total == 0.f ? 0.f : 1.f / total;
    const int r = (m0 + m) / p.group, h = kv_head * p.group + m0 + m - r * p.group;
    T* out = (T*)p.out + b * p.o_b + r * p.o_r + h * p.o_h + d;
    const float x[4] = {y.x * inv, y.y * inv, y.z * inv, y.w * inv};
#pragma unroll
    for (int i = 0; i < 4; ++i)
      if (d + i < p.dim) out[i] = (T)x[i];
  };
  for (int i = tid; i < (m1 - m0) * (DP / 4); i += 32 * kRowWarps) {
    const int m = i / (DP / 4), d = (i - m * (DP / 4)) * 4;
    float most = -INFINITY, total = 0.f;
#pragma unroll
    for (int c = 0; c < RowShared<L, MR>::kParts; ++c) most = fmaxf(most, sh.top[c][m]);
    const float from = most == -INFINITY ? 0.f : most;
    float4 y = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
    for (int c = 0; c < RowShared<L, MR>::kParts; ++c) {
      const float theirs = sh.sum[c][m];
      if (theirs == 0.f) continue;  // saw nothing
      const float f = exp2f(sh.top[c][m] - from);
      const float4 x = *(const float4*)&sh.o[c][m][d];
      total = fmaf(f, theirs, total);
      y.x = fmaf(f, x.x, y.x);
      y.y = fmaf(f, x.y, y.y);
      y.z = fmaf(f, x.z, y.z);
      y.w = fmaf(f, x.w, y.w);
    }
    if (p.split == 1) {
      write(m, d, y, total);
    } else {
      *(float4*)&sh.joined[m][d] = y;
      sh.joined_top[m] = most;  // (all threads of the row the same)
      sh.joined_sum[m] = total;
    }
  }
  if (p.split == 1) return;
  // ... and over the blocks of the cluster, whose warps share the rows.
  cg::cluster_group cluster = cg::this_cluster();
  cluster.sync();
  for (int i = tid + part * 32 * kRowWarps; i < (m1 - m0) * (DP / 4); i += 32 * kRowWarps * p.split) {
    const int m = i / (DP / 4), d = (i - m * (DP / 4)) * 4;
    float most = -INFINITY, total = 0.f;
#pragma unroll 4
    for (int c = 0; c < p.split; ++c) most = fmaxf(most, *cluster.map_shared_rank(&sh.joined_top[m], c));
    const float from = most == -INFINITY ? 0.f : most;
    float4 y = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 4
    for (int c = 0; c < p.split; ++c) {
      const float theirs = *cluster.map_shared_rank(&sh.joined_sum[m], c), at = *cluster.map_shared_rank(&sh.joined_top[m], c);
      const float4 x = *(const float4*)cluster.map_shared_rank(&sh.joined[m][d], c);
      const float f = theirs == 0.f ? 0.f : exp2f(at - from);
      total = fmaf(f, theirs, total);
      y.x = fmaf(f, x.x, y.x);
      y.y = fmaf(f, x.y, y.y);
      y.z = fmaf(f, x.z, y.z);
      y.w = fmaf(f, x.w, y.w);
    }
    write(m, d, y, total);
  }
  cluster.sync();  // (no block ends while another reads its shared memory)
}

// Up to how many packed rows of a kv head rows_kernel takes, which goes through the cache once for every four, while
// tile_kernel's tiles are of 64 whether the rows are there or not, and no more than eight blocks share one.  `heads`: of
// all sequences (rows_kernel / tile_kernel, us):
//                                            36 rows        48 rows      bfloat16: 36 rows    48 rows
//   1 x 20000 positions, 2 heads of 96       135 / 509      133 / 510        162 / 568        162 / 569
//   1 x 2000, 8 heads of 96                   54 / 57        57 / 58          68 / 63          69 / 64
//   1 x 8000, 8 heads of 256                 330 / 466      355 / 472        411 / 407        493 / 409
//   2 x 300, 8 heads of 64                    11 / 23        13 / 23          13 / 24          15 / 24
//   2 x 2000, 8 heads of 256                 153 / 200      174 / 203        201 / 215        218 / 219
//   4 x 2000, 8 heads of 96                  108 / 169      204 / 171        131 / 188        253 / 190
//   4 x 1500, 8 heads of 128                  69 / 131      125 / 133         87 / 142        166 / 144
//   4 x 1500, 8 heads of 256                 141 / 276      277 / 286        167 / 250        325 / 254
//   8 x 1500, 8 heads of 80                  159 / 166      310 / 169        193 / 183        368 / 184
//   8 x 777, 16 heads of 64                   72 / 91       103 / 91          93 / 93         136 / 94
//   16 x 3000, 8 heads of 128                544 / 756      776 / 759        938 / 899       1375 / 900
//   32 x 3000, 8 heads of 64                 549 / 651      788 / 652        949 / 704       1359 / 701
constexpr int few_rows(bool bf16, int64_t heads) { return bf16 && heads > 16 ? 36 : 48; }

struct Build {
  const void* kernel;
  size_t smem;
  int rows, threads, slots;
};
template <typename T, int MR>
Build rows_build(int dim) {
  constexpr int kThreadsFew = 32 * kRowWarps, kSlots = kRowWarps * kAhead;  // slots of a tile: times 32 / L
  if (dim <= 64) return {(const void*)rows_kernel<T, 8, MR>, sizeof(RowShared<8, MR>), MR, kThreadsFew, kSlots * 4};
  if (dim <= 128) return {(const void*)rows_kernel<T, 16, MR>, sizeof(RowShared<16, MR>), MR, kThreadsFew, kSlots * 2};
  return {(const void*)rows_kernel<T, 32, MR>, sizeof(RowShared<32, MR>), MR, kThreadsFew, kSlots};
}
template <typename T>
Build build_of(bool few, int dim) {
  if (few) return rows_build<T, kRows>(dim);
  if (dim <= 64) return {(const void*)tile_kernel<T, 64, 64>, sizeof(Shared<64, 64>), 64, kThreads, kNK};
  if (dim <= 128) return {(const void*)tile_kernel<T, 64, 128>, sizeof(Shared<64, 128>), 64, kThreads, kNK};
  return {(const void*)tile_kernel<T, 64, 256>, sizeof(Shared<64, 256>), 64, kThreads, kNK};
}

int launch_attention_f32(AttentionParams& p, bool bf16, int max_context, cudaStream_t st) {
  const bool few = (int64_t)p.R * p.group <= few_rows(bf16, (int64_t)p.heads * p.B);
  const Build k = bf16 ? build_of<__nv_bfloat16>(few, p.dim) : build_of<float>(few, p.dim);
  p.row_tiles = (int)(((int64_t)p.R * p.group + k.rows - 1) / k.rows);
  const int64_t units = (int64_t)p.row_tiles * p.heads * p.B;
  if (!p.split) {
    // three or four blocks to an SM (one or two of 64 rows), of eight steps at least
    int64_t reach = (int64_t)max_context + p.R;
    if (p.window && reach > (int64_t)p.window + p.sinks + p.R) reach = (int64_t)p.window + p.sinks + p.R;
    const int64_t tiles = (reach + k.slots - 1) / k.slots;
    p.split = 1;
    while (p.split < (few ? 16 : 8) && units * p.split * 2 <= (few ? 4 : 2) * sm_count() && p.split * (few ? 8 : 2) <= tiles) p.split *= 2;
  }
  if (p.split > 8 && !few) p.split = 8;  // (a block of 64 rows takes half of an SM's shared memory and more)
  cudaError_t e = cudaFuncSetAttribute(k.kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)k.smem);
  if (e == cudaSuccess && p.split > 8) e = cudaFuncSetAttribute(k.kernel, cudaFuncAttributeNonPortableClusterSizeAllowed, 1);
  if (e != cudaSuccess) return cuda_fail(e);
  note_launch("attention %s_kernel<%s, %d rows>: %d threads x (%d, %d, %d) blocks, %d to a tile of rows", few ? "rows" : "tile", bf16 ? "bf16" : "f32",
              k.rows, k.threads, p.row_tiles * p.split, p.heads, p.B, p.split);
  Launch l(dim3((unsigned)(p.row_tiles * p.split), (unsigned)p.heads, (unsigned)p.B), (unsigned)k.threads, k.smem, st, (unsigned)p.split);
  // whether rows start on boundaries of the reads: four elements, or with few rows 16 bytes
  const int64_t all = p.q_b | p.q_r | p.q_h | p.k_page | p.k_token | p.k_head | p.v_page | p.v_token | p.v_head;
  const size_t bytes = bf16 && !few ? 8 : 16;
  bool wide = all % (int64_t)(bytes / (bf16 ? 2 : 4)) == 0 && aligned_to(p.q, bytes) && aligned_to(p.k, bytes) && aligned_to(p.v, bytes);
  void* args[] = {(void*)&p, (void*)&wide};
  e = cudaLaunchKernelExC(&l.cfg, k.kernel, args);
  return e == cudaSuccess ? ERSD_OK : cuda_fail(e);
}

}  // namespace

}  // namespace ersd

extern "C" int ersd_chunk_attention(const ersd_cache* cache, const void* q, void* out, const int32_t* context_lens, int B, int R, int Hq,
                                    const ersd_chunk_opts* opts, void* cuda_stream) {
  using namespace ersd;
  if (!cache) return ERSD_EINVAL;
  const ersd_cache c = read_struct(cache);
  const ersd_chunk_opts o = read_struct(opts);
  if (!c.k || !c.v || !c.block_table || (c.dtype != ERSD_F32 && c.dtype != ERSD_BF16)) return ERSD_EINVAL;
  if (c.num_pages < 1 || c.page_size < 1 || c.heads < 1 || c.head_dim < 1 || c.layers < 1 || c.max_pages < 1) return ERSD_EINVAL;
  if (!q || !out || !context_lens || B < 1 || R < 1 || Hq < 1 || Hq % c.heads) return ERSD_EINVAL;
  if (o.window < 0 || o.sinks < 0 || o.max_context < 0 || !(fabsf(o.scale) <= 2.3e38f) || o.kernel_path > 2) return ERSD_EINVAL;
  if (o.split < 0 || o.split > 16) return ERSD_EINVAL;
  const size_t size = c.dtype == ERSD_BF16 ? 2 : 4;
  if (!aligned_to(c.k, size) || !aligned_to(c.v, size) || !aligned_to(q, size) || !aligned_to(out, size)) return ERSD_EALIGN;
  if (!aligned_to(c.block_table, 4) || !aligned_to(context_lens, 4) || !aligned_to(o.row_counts, 4)) return ERSD_EALIGN;
  if (c.head_dim > ERSD_MAX_HEAD_DIM || B > 65535 || c.heads > 65535 || (o.parent && R > ERSD_MAX_ROWS)) return ERSD_EUNSUPPORTED;
  if ((int64_t)R * Hq > (1 << 30) || (int64_t)c.max_pages * c.page_size > (1 << 30)) return ERSD_EUNSUPPORTED;
  if (o.parent && !is_tree(o.parent, R)) return ERSD_EINVAL;
  const bool qs = o.a_stride_b || o.a_stride_r || o.a_stride_h, os = o.b_stride_b || o.b_stride_r || o.b_stride_h;
  if (os && ((B > 1 && !o.b_stride_b) || (R > 1 && !o.b_stride_r) || (Hq > 1 && !o.b_stride_h))) return ERSD_EINVAL;  // (rows written over one another)
  AttentionParams p;
  memset(&p, 0, sizeof p);
  const int64_t d = c.head_dim;
  p.q = q;
  p.k = c.k;
  p.v = c.v;
  p.out = out;
  p.table = c.block_table;
  p.context_lens = context_lens;
  p.row_counts = o.row_counts;
  p.table_stride = c.table_stride;
  p.q_b = qs ? o.a_stride_b : R * Hq * d;
  p.q_r = qs ? o.a_stride_r : Hq * d;
  p.q_h = qs ? o.a_stride_h : d;
  p.o_b = os ? o.b_stride_b : R * Hq * d;
  p.o_r = os ? o.b_stride_r : Hq * d;
  p.o_h = os ? o.b_stride_h : d;
  p.k_page = c.k_stride_page;
  p.k_token = c.k_stride_token;
  p.k_head = c.k_stride_head;
  p.v_page = c.v_stride_page;
  p.v_token = c.v_stride_token;
  p.v_head = c.v_stride_head;
  p.B = B;
  p.R = R;
  p.heads = c.heads;
  p.group = Hq / c.heads;
  p.dim = c.head_dim;
  set_page_size(p, c.page_size);
  p.num_pages = c.num_pages;
  p.capacity = c.max_pages * c.page_size;
  p.window = o.window;
  p.sinks = o.sinks;
  p.scale_log2 = (o.scale != 0.0f ? o.scale : 1.0f / sqrtf((float)c.head_dim)) * 1.4426950408889634f;
  p.split = o.split;
  p.tree = o.parent != nullptr;
  if (o.parent)
    for (int n = 1; n < R; ++n) {
      p.parent[n] = (uint8_t)o.parent[n];
      p.depth[n] = (uint8_t)(p.depth[o.parent[n]] + 1);
    }
  int max_context = o.max_context;
  if (!max_context || max_context > p.capacity) max_context = p.capacity;
  cudaStream_t st = (cudaStream_t)cuda_stream;
  if (o.kernel_path != 1) {
    const int status = c.dtype == ERSD_BF16 ? launch_attention_tensor(p, max_context, st) : ERSD_EUNSUPPORTED;
    if (status != ERSD_EUNSUPPORTED || o.kernel_path == 2) return status;
    p.split = o.split;
  }
  return launch_attention_f32(p, c.dtype == ERSD_BF16, max_context, st);
}
