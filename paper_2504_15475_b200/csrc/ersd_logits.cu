// Penalties, biases and masks on logits: ersd_process_logits.
//
// Bytes bound the operator: every row is read and written once.  What a token's logit is changed by is the
// same for all rows of a sequence, up to the drafted tokens on a row's path, so one block takes a slice of the
// vocabulary for ALL rows of a sequence: it counts the history's tokens that fall into the slice in shared
// memory (integers: no order of the atomics changes a result) and then streams the slice of each row past the
// table.  A token's bit in a bitmap says whether anything but the mask touches it; a group of eight tokens
// without such a bit and with all mask bits set goes through unchanged, one with no mask bit set is written
// without being read.
#include <cuda_bf16.h>
#include <math.h>

#include "ersd_host.h"

namespace ersd {

namespace {

constexpr int kGroup = 8;            // consecutive tokens a thread takes at a time
constexpr int kAhead = 4;            // groups whose loads a thread issues before it works on the first
constexpr int kLogitThreads = 256;
constexpr uint32_t kSeen = 1u << 31;     // in the history
constexpr uint32_t kDrafted = 1u << 30;  // among the sequence's drafted tokens: its count depends on the row
constexpr uint32_t kCount = kDrafted - 1;

struct LogitParams {
  const void* in;
  void* out;
  int64_t ld_in, ld_out;
  int B, R, V, slice;
  int in_place;
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

template <typename T>
struct alignas(16) Group {
  T x[kGroup];
};

// Eight bits from bit position `at` on of a bitmap whose words past `last` do not exist.
__device__ __forceinline__ uint32_t bits_at(const uint32_t* words, int at, int last) {
  const int w = at >> 5;
  const uint32_t lo = words[w], hi = (at & 31) > 24 && w < last ? words[w + 1] : 0u;
  return __funnelshift_r(lo, hi, at & 31) & 0xFFu;
}

template <typename T>
__global__ void __launch_bounds__(kLogitThreads) process_logits_kernel(const LogitParams p) {
  extern __shared__ uint32_t shared[];
  const int b = blockIdx.y, tid = threadIdx.x;
  const int s0 = (int)blockIdx.x * p.slice;       // this block: groups whose last token is in [s0, s0 + slice)
  const int base = s0 - kGroup, span = p.slice + kGroup;  // tokens base .. base + span
  uint32_t* table = shared;                        // [span] counts and flags
  uint32_t* touched = table + span;                // [span / 32 + 2] bit per token
  uint32_t* bias_at = touched + span / 32 + 2;     // [span] 1 + index of the token's bias, where biases are given
  __shared__ int32_t draft[ERSD_MAX_ROWS];
  __shared__ uint8_t parent[ERSD_MAX_ROWS];
  const int words = span / 32 + 2;
  for (int i = tid; i < span + words + (p.bias_count ? span : 0); i += kLogitThreads) shared[i] = 0;
  for (int n = tid; n < ERSD_MAX_ROWS; n += kLogitThreads) parent[n] = p.parent[n];
  asm volatile("griddepcontrol.wait;" ::: "memory");
  __syncthreads();

  if (p.history) {
    int n = p.history_lens ? p.history_lens[b] : p.history_width;
    n = max(0, min(n, p.history_width));
    const int prompt = p.prompt_lens ? p.prompt_lens[b] : 0;
    const int32_t* h = p.history + (int64_t)b * p.history_width;
#pragma unroll 4
    for (int i = tid; i < n; i += kLogitThreads) {
      const int t = h[i], at = t - base;
      if (t >= 0 && t < p.V && at >= 0 && at < span) {
        atomicOr(&table[at], kSeen);
        if (i >= prompt) atomicAdd(&table[at], 1u);
        atomicOr(&touched[at >> 5], 1u << (at & 31));
      }
    }
  }
  const int drafts = p.draft_tokens ? p.R - 1 : 0;  // draft[n], 1 <= n <= drafts: token of node n
  for (int n = 1 + tid; n <= drafts; n += kLogitThreads) {
    const int t = p.tree ? p.draft_tokens[(int64_t)b * p.R + n] : p.draft_tokens[(int64_t)b * (p.R - 1) + n - 1];
    draft[n] = t;
    const int at = t - base;
    if (t >= 0 && t < p.V && at >= 0 && at < span) {
      atomicOr(&table[at], kDrafted);
      atomicOr(&touched[at >> 5], 1u << (at & 31));
    }
  }
  for (int i = tid; i < p.bias_count; i += kLogitThreads) {
    const int t = p.bias_tokens[b * p.bias_stride + i], at = t - base;
    if (t >= 0 && t < p.V && at >= 0 && at < span) {
      atomicMax(&bias_at[at], (uint32_t)i + 1u);
      atomicOr(&touched[at >> 5], 1u << (at & 31));
    }
  }
  const float rep = p.repetition ? p.repetition[b] : 1.0f;
  const float pres = p.presence ? p.presence[b] : 0.0f;
  const float freq = p.frequency ? p.frequency[b] : 0.0f;
  const float* bias = p.bias_count ? p.bias_values + b * p.bias_stride : nullptr;
  __syncthreads();

  const int mask_last = (p.V - 1) >> 5;
  const float minus_inf = -INFINITY;
  // A token's logit on row r.  The table's entry says what the history holds; a drafted token counts if it is
  // on the path to this row.
  auto change = [&](float x, int at, int r) {
    uint32_t e = table[at];
    uint32_t c = e & kCount;
    bool seen = (e & kSeen) != 0;
    if (e & kDrafted) {
      for (int n = r; n > 0; n = p.tree ? parent[n] : n - 1) c += draft[n] == at + base;
      seen |= c > 0;
    }
    if (seen) {
      if (p.repetition) x = x > 0.0f ? __fdiv_rn(x, rep) : x * rep;
      if (c) x = x - freq * (float)c - pres;
    }
    if (bias) {
      const uint32_t k = bias_at[at];
      if (k) x += bias[k - 1];
    }
    return x;
  };

  constexpr int kPer16 = 16 / (int)sizeof(T);
  for (int r = 0; r < p.R; ++r) {
    const T* in = (const T*)p.in + ((int64_t)b * p.R + r) * p.ld_in;
    T* out = (T*)p.out + ((int64_t)b * p.R + r) * p.ld_out;
    // groups start on 16-byte boundaries of the input: lead tokens before the slice's first
    const int lead = (int)(((uintptr_t)in / sizeof(T)) & (kPer16 - 1));
    const bool wide_out = (((uintptr_t)(out - lead)) & 15) == 0;
    const uint32_t* mask = p.mask ? p.mask + b * p.mask_stride_b + r * p.mask_stride_r : nullptr;
    for (int g0 = tid; g0 < p.slice / kGroup; g0 += kLogitThreads * kAhead) {
      Group<T> x[kAhead];
      uint32_t allow[kAhead], hit[kAhead];
      // 0: outside the row, 1: whole, 2: cut by the row's ends
      int kind[kAhead];
#pragma unroll
      for (int k = 0; k < kAhead; ++k) {
        const int g = g0 + k * kLogitThreads, t = s0 - lead + g * kGroup;
        kind[k] = g >= p.slice / kGroup || t >= p.V || t + kGroup <= 0 ? 0 : t < 0 || t + kGroup > p.V ? 2 : 1;
        allow[k] = 0xFFu;
        if (kind[k] == 1 && mask) allow[k] = bits_at(mask, t, mask_last);
      }
#pragma unroll
      for (int k = 0; k < kAhead; ++k) {
        const int g = g0 + k * kLogitThreads, t = s0 - lead + g * kGroup;
        hit[k] = 0;
        if (kind[k] != 1) continue;
        hit[k] = bits_at(touched, t - base, words - 1);
        if (allow[k] && (!p.in_place || (hit[k] | (allow[k] ^ 0xFFu)))) {
          const int4* src = (const int4*)(in + t);
          int4* dst = (int4*)&x[k];
#pragma unroll
          for (int j = 0; j < (int)sizeof(Group<T>) / 16; ++j) dst[j] = __ldcs(src + j);
        }
      }
#pragma unroll
      for (int k = 0; k < kAhead; ++k) {
        const int g = g0 + k * kLogitThreads, t = s0 - lead + g * kGroup;
        if (kind[k] == 0) continue;
        if (kind[k] == 2) {
          for (int e = 0; e < kGroup; ++e) {
            const int i = t + e;
            if (i < 0 || i >= p.V) continue;
            const bool ok = !mask || (mask[i >> 5] >> (i & 31) & 1u);
            out[i] = from_float<T>(ok ? change(to_float(in[i]), i - base, r) : minus_inf);
          }
          continue;
        }
        if (hit[k] | (allow[k] ^ 0xFFu)) {
#pragma unroll
          for (int e = 0; e < kGroup; ++e) {
            if (!(allow[k] >> e & 1u)) x[k].x[e] = from_float<T>(minus_inf);
            else if (hit[k] >> e & 1u) x[k].x[e] = from_float<T>(change(to_float(x[k].x[e]), t + e - base, r));
          }
        } else if (p.in_place) {
          continue;
        }
        if (wide_out) {
#pragma unroll
          for (int j = 0; j < (int)sizeof(Group<T>) / 16; ++j) __stcs((int4*)(out + t) + j, ((const int4*)&x[k])[j]);
        } else {
#pragma unroll
          for (int e = 0; e < kGroup; ++e) out[t + e] = x[k].x[e];
        }
      }
    }
  }
}

size_t logit_smem(int slice, bool biases) {
  const size_t span = (size_t)slice + kGroup;
  return 4 * (span + span / 32 + 2 + (biases ? span : 0));
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
  if (o.parent && !o.draft_tokens) return ERSD_EINVAL;
  const size_t size = dt == ERSD_BF16 ? 2 : 4;
  if (!aligned_to(logits, size) || !aligned_to(out, size)) return ERSD_EALIGN;
  const void* words[] = {o.history, o.history_lens, o.prompt_lens, o.draft_tokens, o.repetition, o.presence, o.frequency, o.bias_tokens,
                         o.bias_values, o.mask};
  for (const void* w : words)
    if (!aligned_to(w, 4)) return ERSD_EALIGN;
  if (B > 65535 || V > 0x7FFF0000 || o.bias_count > ERSD_MAX_BIASES || (o.draft_tokens && R > ERSD_MAX_ROWS)) return ERSD_EUNSUPPORTED;
  if (o.parent && !is_tree(o.parent, R)) return ERSD_EINVAL;
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
  p.history_width = o.history_width;
  p.draft_tokens = R > 1 ? o.draft_tokens : nullptr;
  p.tree = o.parent != nullptr;
  if (o.parent)
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
  // Slices as long as the shared table allows while there are four blocks to an SM, shorter ones for few sequences.
  p.slice = 8192;
  while (p.slice > 2048 && (int64_t)B * ((V + p.slice - 1) / p.slice) < 4 * sm_count()) p.slice /= 2;
  const unsigned slices = (unsigned)(((int64_t)V + kGroup - 1 + p.slice - 1) / p.slice);
  const size_t smem = logit_smem(p.slice, p.bias_count != 0);
  const auto kernel = dt == ERSD_BF16 ? process_logits_kernel<__nv_bfloat16> : process_logits_kernel<float>;
  cudaError_t e = cudaSuccess;
  if (smem > 48 * 1024) e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
  if (e != cudaSuccess) return cuda_fail(e);
  note_launch("process_logits_kernel<%s>: %d threads x (%u, %d) blocks, slices of %d tokens", dt == ERSD_BF16 ? "bf16" : "f32", kLogitThreads,
              slices, B, p.slice);
  Launch l(dim3(slices, (unsigned)B, 1), kLogitThreads, smem, (cudaStream_t)cuda_stream);
  e = cudaLaunchKernelEx(&l.cfg, kernel, p);
  return e == cudaSuccess ? ERSD_OK : cuda_fail(e);
}
