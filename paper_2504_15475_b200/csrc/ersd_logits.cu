// Penalties, biases and masks on logits: ersd_process_logits.
//
// Bytes bound the operator: every row is read and written once.  Few tokens are changed by more than the mask,
// and which ones is the same for all rows of a sequence, up to the drafted tokens on a row's path.  So one block
// takes a slice of the vocabulary for ALL rows of a sequence.  It copies the slice of every row, with -inf where
// the mask forbids a token (eight tokens that are all forbidden are not read), counts the history's tokens that
// fall into the slice in shared memory (integers: no order of the atomics changes a result), lists the tokens
// that occur, and writes those of every row again, each from its own logit.  Changing them while copying would
// cost a warp the work for every token that any of its 256 is listed for: 303 us instead of 62 for 64 sequences
// of nine rows with histories of 3000 tokens.
#include <cuda_bf16.h>
#include <math.h>

#include "ersd_host.h"

namespace ersd {

namespace {

constexpr int kGroup = 8;            // consecutive tokens a thread takes at a time
constexpr int kAhead = 4;            // groups whose loads a thread issues before it works on the first
constexpr int kLogitThreads = 512;
constexpr uint32_t kSeen = 1u << 31;     // in the history
constexpr uint32_t kDrafted = 1u << 30;  // among the sequence's drafted tokens: its count depends on the row
constexpr uint32_t kBiased = 1u << 29;
constexpr uint32_t kCount = kBiased - 1;

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

// Eight bits from bit position `at` on of a bitmap whose words past `last` do not exist.
__device__ __forceinline__ uint32_t bits_at(const uint32_t* words, int at, int last) {
  const int w = at >> 5;
  const uint32_t lo = words[w], hi = (at & 31) > 24 && w < last ? words[w + 1] : 0u;
  return __funnelshift_r(lo, hi, at & 31) & 0xFFu;
}

template <typename T>
struct alignas(16) Group {
  static constexpr int kWords = kGroup * (int)sizeof(T) / 4;
  uint32_t w[kWords];
  __device__ __forceinline__ void forbid(uint32_t allow) {  // -inf where a bit is 0
#pragma unroll
    for (int j = 0; j < kWords; ++j) {
      if constexpr (sizeof(T) == 4) {
        if (!(allow >> j & 1u)) w[j] = 0xFF800000u;
      } else {
        if (!(allow >> (2 * j) & 1u)) w[j] = (w[j] & 0xFFFF0000u) | 0xFF80u;
        if (!(allow >> (2 * j) & 2u)) w[j] = (w[j] & 0xFFFFu) | 0xFF800000u;
      }
    }
  }
};

template <typename T>
__global__ void __launch_bounds__(kLogitThreads) process_logits_kernel(const LogitParams p) {
  extern __shared__ uint32_t shared[];
  const int b = blockIdx.x, tid = threadIdx.x;
  const int s0 = (int)blockIdx.y * p.slice;               // this block: groups whose last token is in [s0, s0 + slice)
  const int base = s0 - kGroup, span = p.slice + kGroup;  // tokens base .. base + span
  uint32_t* table = shared;                               // [span] counts and flags
  uint16_t* list = (uint16_t*)(table + span);             // [span] tokens of the table that occur
  uint32_t* bias_at = table + span + span / 2;            // [span] 1 + index of the token's bias, where biases are given
  __shared__ int32_t draft[ERSD_MAX_ROWS];
  __shared__ uint8_t parent[ERSD_MAX_ROWS];
  __shared__ int listed;
  const bool changes = p.history || p.draft_tokens || p.bias_count;
  if (changes) {
    for (int i = tid; i < span; i += kLogitThreads) table[i] = 0;
    if (p.bias_count)
      for (int i = tid; i < span; i += kLogitThreads) bias_at[i] = 0;
    if (p.tree)
      for (int n = tid; n < ERSD_MAX_ROWS; n += kLogitThreads) parent[n] = p.parent[n];
    if (tid == 0) listed = 0;
  }
  asm volatile("griddepcontrol.wait;" ::: "memory");

  // ---- the copy
  constexpr int kPer16 = 16 / (int)sizeof(T);
  const int mask_last = (p.V - 1) >> 5, groups = p.slice / kGroup, shift = __ffs(groups) - 1;
  if (!p.in_place || p.mask) {
    const int64_t items = (int64_t)p.R * groups;
    for (int64_t i0 = tid; i0 < items; i0 += kLogitThreads * kAhead) {
      Group<T> x[kAhead];
      uint32_t allow[kAhead];
      int t[kAhead];
      const T* in[kAhead];
      // groups start on 16-byte boundaries of the input: `lead` tokens before the slice's first
#pragma unroll
      for (int k = 0; k < kAhead; ++k) {
        const int64_t i = i0 + k * kLogitThreads;
        const int r = (int)(i >> shift), g = (int)(i & (groups - 1));
        in[k] = (const T*)p.in + ((int64_t)b * p.R + r) * p.ld_in;
        t[k] = i < items ? s0 - (int)(((uintptr_t)in[k] / sizeof(T)) & (kPer16 - 1)) + g * kGroup : p.V;
        allow[k] = 0xFFu;
        if (p.mask && t[k] >= 0 && t[k] + kGroup <= p.V)
          allow[k] = bits_at(p.mask + b * p.mask_stride_b + r * p.mask_stride_r, t[k], mask_last);
      }
#pragma unroll
      for (int k = 0; k < kAhead; ++k)
        if (t[k] >= 0 && t[k] + kGroup <= p.V && allow[k] && (!p.in_place || allow[k] != 0xFFu)) {
#pragma unroll
          for (int j = 0; j < Group<T>::kWords / 4; ++j) ((int4*)&x[k])[j] = __ldg((const int4*)(in[k] + t[k]) + j);
        }
#pragma unroll
      for (int k = 0; k < kAhead; ++k) {
        if (t[k] >= p.V || t[k] + kGroup <= 0) continue;
        const int r = (int)((i0 + k * kLogitThreads) >> shift);
        T* out = (T*)p.out + ((int64_t)b * p.R + r) * p.ld_out;
        if (t[k] < 0 || t[k] + kGroup > p.V) {  // cut by the row's ends
          const uint32_t* mask = p.mask ? p.mask + b * p.mask_stride_b + r * p.mask_stride_r : nullptr;
          for (int i = max(t[k], 0); i < min(t[k] + kGroup, p.V); ++i)
            out[i] = !mask || (mask[i >> 5] >> (i & 31) & 1u) ? in[k][i] : from_float<T>(-INFINITY);
          continue;
        }
        if (p.in_place && allow[k] == 0xFFu) continue;
        x[k].forbid(allow[k]);
        if (((uintptr_t)(out + t[k]) & 15) == 0) {
#pragma unroll
          for (int j = 0; j < Group<T>::kWords / 4; ++j) ((int4*)(out + t[k]))[j] = ((const int4*)&x[k])[j];
        } else {
#pragma unroll
          for (int e = 0; e < kGroup; ++e) out[t[k] + e] = ((const T*)&x[k])[e];
        }
      }
    }
  }
  if (!changes) return;
  __syncthreads();  // (the table is zeros)

  // ---- the tokens that are changed
  auto put = [&](int t, uint32_t flags, uint32_t count) {
    const int at = t - base;
    if (t < 0 || t >= p.V || at < 0 || at >= span) return;
    if (atomicOr(&table[at], flags) == 0) list[atomicAdd(&listed, 1)] = (uint16_t)at;
    if (count) atomicAdd(&table[at], count);
  };
  if (p.history) {
    int n = p.history_lens ? p.history_lens[b] : p.history_width;
    n = max(0, min(n, p.history_width));
    const int prompt = p.prompt_lens ? p.prompt_lens[b] : 0;
    const int32_t* h = p.history + (int64_t)b * p.history_width;
#pragma unroll 4
    for (int i = tid; i < n; i += kLogitThreads) put(h[i], kSeen, i >= prompt);
  }
  const int drafts = p.draft_tokens ? p.R - 1 : 0;  // draft[n], 1 <= n <= drafts: token of node n
  for (int n = 1 + tid; n <= drafts; n += kLogitThreads) {
    const int t = p.tree ? p.draft_tokens[(int64_t)b * p.R + n] : p.draft_tokens[(int64_t)b * (p.R - 1) + n - 1];
    draft[n] = t;
    put(t, kDrafted, 0);
  }
  for (int i = tid; i < p.bias_count; i += kLogitThreads) {
    const int t = p.bias_tokens[b * p.bias_stride + i], at = t - base;
    if (t >= 0 && t < p.V && at >= 0 && at < span) atomicMax(&bias_at[at], (uint32_t)i + 1u);
    put(t, kBiased, 0);
  }
  const float rep = p.repetition ? p.repetition[b] : 1.0f;
  const float pres = p.presence ? p.presence[b] : 0.0f;
  const float freq = p.frequency ? p.frequency[b] : 0.0f;
  const float* bias = p.bias_count ? p.bias_values + b * p.bias_stride : nullptr;
  __syncthreads();  // (the list; and the copies of other threads, which are written over)
  const int n = listed;
  const int items = n * p.R;  // (at most 4104 * 65535)
  for (int i0 = tid; i0 < items; i0 += kLogitThreads * kAhead) {
    float x[kAhead];
    int r[kAhead], at[kAhead];
#pragma unroll
    for (int k = 0; k < kAhead; ++k) {
      const int i = i0 + k * kLogitThreads;
      at[k] = -1;
      if (i >= items) continue;
      r[k] = i / n;
      const int found = list[i - r[k] * n], t = found + base;
      const T* in = (const T*)p.in + ((int64_t)b * p.R + r[k]) * p.ld_in;
      // the token's group may belong to the block before or behind this one in this row
      const int lead = (int)(((uintptr_t)in / sizeof(T)) & (kPer16 - 1));
      if (t < s0 - lead || t >= s0 - lead + p.slice) continue;
      if (p.mask && !(p.mask[b * p.mask_stride_b + r[k] * p.mask_stride_r + (t >> 5)] >> (t & 31) & 1u)) continue;
      at[k] = found;
      x[k] = to_float(in[t]);
    }
#pragma unroll
    for (int k = 0; k < kAhead; ++k) {
      if (at[k] < 0) continue;
      const int t = at[k] + base;
      const uint32_t e = table[at[k]];
      uint32_t c = e & kCount;
      bool seen = (e & kSeen) != 0;
      if (e & kDrafted) {  // a drafted token counts if it is on the path to this row
        for (int m = r[k]; m > 0; m = p.tree ? parent[m] : m - 1) c += draft[m] == t;
        seen |= c > 0;
      }
      float y = x[k];
      if (seen) {
        if (p.repetition) y = y > 0.0f ? __fdiv_rn(y, rep) : y * rep;
        if (c) y = y - freq * (float)c - pres;
      }
      if (e & kBiased) y += bias[bias_at[at[k]] - 1];
      ((T*)p.out + ((int64_t)b * p.R + r[k]) * p.ld_out)[t] = from_float<T>(y);
    }
  }
}

size_t logit_smem(int slice, bool biases) {
  const size_t span = (size_t)slice + kGroup;
  return 4 * (span + span / 2 + (biases ? span : 0));
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
  if (B > 65535 || R > 65535 || V > (1 << 28) || o.bias_count > ERSD_MAX_BIASES || (o.draft_tokens && R > ERSD_MAX_ROWS)) return ERSD_EUNSUPPORTED;
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
  p.history_width = o.history_width;
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
  // Long slices while there are four blocks to an SM (every block reads the sequence's whole history), shorter ones
  // for few sequences.
  p.slice = 4096;
  while (p.slice > 1024 && (int64_t)B * ((V + p.slice - 1) / p.slice) < 4 * sm_count()) p.slice /= 2;
  const unsigned slices = (unsigned)(((int64_t)V + kGroup - 1 + p.slice - 1) / p.slice);
  const size_t smem = logit_smem(p.slice, p.bias_count != 0);
  const auto kernel = dt == ERSD_BF16 ? process_logits_kernel<__nv_bfloat16> : process_logits_kernel<float>;
  cudaError_t e = cudaSuccess;
  if (smem > 48 * 1024) e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
  if (e != cudaSuccess) return cuda_fail(e);
  note_launch("process_logits_kernel<%s>: %d threads x (%d, %u) blocks, slices of %d tokens", dt == ERSD_BF16 ? "bf16" : "f32", kLogitThreads,
              B, slices, p.slice);
  // (all sequences' first slices before the next: frequent tokens have low numbers, their blocks the most to change)
  Launch l(dim3((unsigned)B, slices, 1), kLogitThreads, smem, (cudaStream_t)cuda_stream);
  e = cudaLaunchKernelEx(&l.cfg, kernel, p);
  return e == cudaSuccess ? ERSD_OK : cuda_fail(e);
}
