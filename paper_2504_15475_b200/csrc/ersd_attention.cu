// ersd_chunk_attention: checks, the choice of the kernel, and the kernel of 32-bit arithmetic.
//
// The kernel of 32-bit arithmetic takes a tile of MR packed rows of one kv head through the keys, kNK slots at a
// time: keys and values are copied to shared memory as floats, a thread forms the scores of one slot with several
// rows, the softmax's running maximum and sum live in shared memory, and a thread holds four columns of a few
// rows of the output in registers.  `split` thread blocks of a cluster share the keys of a tile of rows and join
// their partial results through distributed shared memory, so that a few rows over a long cache use many SMs.
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

template <int MR, int DP>
struct Shared {
  float q[MR][DP];
  float k[kNK][DP + 4];  // (+4: a warp's 16-byte reads of 32 slots fall on all banks)
  float v[kNK][DP];
  float s[MR][kNK + 4];
  float top[MR], sum[MR], factor[MR];  // running maximum, sum, and what the output is scaled by this tile
  int row[MR];                         // row of the chunk, or -1
  uint32_t above[MR][ERSD_MAX_ROWS / 32];  // tree: nodes the row sees
};

// MR packed rows, DP >= dim columns (a multiple of 64).
template <typename T, int MR, int DP>
__global__ void __launch_bounds__(kThreads) attention_kernel(const AttentionParams p, bool wide) {
  extern __shared__ __align__(16) char raw[];
  Shared<MR, DP>& sh = *(Shared<MR, DP>*)raw;
  const int tid = threadIdx.x, kv_head = blockIdx.y, b = blockIdx.z;
  const int tile = blockIdx.x / p.split, part = blockIdx.x - tile * p.split;
  asm volatile("griddepcontrol.wait;" ::: "memory");
  int rows = p.row_counts ? p.row_counts[b] : p.R;
  rows = max(0, min(rows, p.R));
  const int m0 = tile * MR, m1 = min(m0 + MR, rows * p.group);
  if (m0 >= m1) return;  // (the same for every block of the cluster)
  const int ctx = max(0, p.context_lens[b]);
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
    if (p.tree) {
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
      for (int j = 0; j < ERSD_MAX_ROWS / 32; ++j) sh.above[m][j] = w[j];
    }
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
      constexpr int kParts = kThreads / kNK, kRows = MR / kParts;  // a thread: one slot, kRows rows
      const int n = tid % kNK, part_of = tid / kNK, slot = start + n;
      float s[kRows];
#pragma unroll
      for (int i = 0; i < kRows; ++i) s[i] = 0.f;
      for (int d = 0; d < DP; d += 4) {
        const float4 fk = *(const float4*)&sh.k[n][d];
#pragma unroll
        for (int i = 0; i < kRows; ++i) {
          const float4 fq = *(const float4*)&sh.q[part_of * kRows + i][d];
          s[i] = fmaf(fq.x, fk.x, s[i]);
          s[i] = fmaf(fq.y, fk.y, s[i]);
          s[i] = fmaf(fq.z, fk.z, s[i]);
          s[i] = fmaf(fq.w, fk.w, s[i]);
        }
      }
#pragma unroll
      for (int i = 0; i < kRows; ++i) {
        const int m = part_of * kRows + i, r = sh.row[m];
        bool see = r >= 0 && slot < keys.hi;
        if (see) {
          if (!p.tree) {
            see = slot <= ctx + r && (!p.window || slot > ctx + r - p.window || slot < p.sinks);
          } else if (slot < ctx) {
            see = !p.window || slot > ctx + (int)p.depth[r] - p.window || slot < p.sinks;
          } else {
            const int node = slot - ctx;
            see = sh.above[m][node >> 5] >> (node & 31) & 1u;
          }
        }
        sh.s[m][n] = see ? s[i] : -INFINITY;
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

struct Build {
  const void* kernel;
  size_t smem;
  int rows;
};
template <typename T, int MR>
Build build_of(int dim) {
  if (dim <= 64) return {(const void*)attention_kernel<T, MR, 64>, sizeof(Shared<MR, 64>), MR};
  if (dim <= 128) return {(const void*)attention_kernel<T, MR, 128>, sizeof(Shared<MR, 128>), MR};
  return {(const void*)attention_kernel<T, MR, 256>, sizeof(Shared<MR, 256>), MR};
}

int launch_attention_f32(AttentionParams& p, bool bf16, int max_context, cudaStream_t st) {
  // Tiles of 16 packed rows where there are few: a tile of 64 would spend four times the arithmetic on rows that
  // are not there.
  const bool few = (int64_t)p.R * p.group <= 32;
  const Build k = bf16 ? (few ? build_of<__nv_bfloat16, 16>(p.dim) : build_of<__nv_bfloat16, 64>(p.dim))
                       : (few ? build_of<float, 16>(p.dim) : build_of<float, 64>(p.dim));
  p.row_tiles = (int)(((int64_t)p.R * p.group + k.rows - 1) / k.rows);
  const int64_t units = (int64_t)p.row_tiles * p.heads * p.B;
  if (!p.split) {
    int64_t reach = (int64_t)max_context + p.R;
    if (p.window && reach > (int64_t)p.window + p.sinks + p.R) reach = (int64_t)p.window + p.sinks + p.R;
    const int64_t tiles = (reach + kNK - 1) / kNK;
    p.split = 1;
    while (p.split < 8 && units * p.split < 2 * sm_count() && p.split * 2 <= tiles) p.split *= 2;
  }
  if (p.split > 8) p.split = 8;
  cudaError_t e = cudaFuncSetAttribute(k.kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)k.smem);
  if (e != cudaSuccess) return cuda_fail(e);
  note_launch("attention_kernel<%s, %d rows>: %d threads x (%d, %d, %d) blocks, %d to a tile of rows", bf16 ? "bf16" : "f32", k.rows, kThreads,
              p.row_tiles * p.split, p.heads, p.B, p.split);
  Launch l(dim3((unsigned)(p.row_tiles * p.split), (unsigned)p.heads, (unsigned)p.B), kThreads, k.smem, st, (unsigned)p.split);
  const int64_t align = bf16 ? 4 : 4;  // elements of a 16-byte (8-byte) read
  const int64_t all = p.q_b | p.q_r | p.q_h | p.k_page | p.k_token | p.k_head | p.v_page | p.v_token | p.v_head;
  const size_t bytes = bf16 ? 8 : 16;
  bool wide = all % align == 0 && aligned_to(p.q, bytes) && aligned_to(p.k, bytes) && aligned_to(p.v, bytes);
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
  if (o.window < 0 || o.sinks < 0 || o.max_context < 0 || !(fabsf(o.scale) <= 3e38f) || o.kernel_path > 2) return ERSD_EINVAL;
  if (o.split < 0 || o.split > 16) return ERSD_EINVAL;
  const size_t size = c.dtype == ERSD_BF16 ? 2 : 4;
  if (!aligned_to(c.k, size) || !aligned_to(c.v, size) || !aligned_to(q, size) || !aligned_to(out, size)) return ERSD_EALIGN;
  if (!aligned_to(c.block_table, 4) || !aligned_to(context_lens, 4) || !aligned_to(o.row_counts, 4)) return ERSD_EALIGN;
  if (c.head_dim > ERSD_MAX_HEAD_DIM || B > 65535 || c.heads > 65535 || (o.parent && R > ERSD_MAX_ROWS)) return ERSD_EUNSUPPORTED;
  if ((int64_t)R * Hq > (1 << 30) || (int64_t)c.max_pages * c.page_size > (1 << 30)) return ERSD_EUNSUPPORTED;
  if (o.parent && !is_tree(o.parent, R)) return ERSD_EINVAL;
  AttentionParams p;
  memset(&p, 0, sizeof p);
  const int64_t d = c.head_dim;
  const bool qs = o.a_stride_b || o.a_stride_r || o.a_stride_h, os = o.b_stride_b || o.b_stride_r || o.b_stride_h;
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
