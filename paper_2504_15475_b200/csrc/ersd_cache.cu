// The paged cache's writes: ersd_cache_append and ersd_cache_commit.  Both are copies, bound by bytes (large
// calls) or by one launch and two dependent reads (small ones).  Measured on one B200, 8 heads of 128 in bfloat16: 8 x up to
// 2048 rows appended in 16 us (67 MB moved, 4.2 TB/s with ragged counts; 134 MB in 23 us, 5.9, when every row counts: the
// blocks of rows that do not count are launched all the same, and index arithmetic fills two thirds of the issue slots), 64 x 1 row in
// 1.8 us, accepted paths of 32 sequences in 32 layers in 6 us.
#include "ersd_host.h"

namespace ersd {

namespace {

struct Side {  // keys or values
  char* cache;
  const char* rows;  // append: the new rows
  int64_t layer, page, token, head;  // strides of the cache, in bytes
  int64_t row_b, row_r, row_h;       // and of the rows
};

struct CacheParams {
  Side side[2];
  const int32_t *table, *context_lens, *row_counts, *path, *accept_len;
  int32_t* out_context_lens;
  int64_t table_stride;
  int R, heads, pieces;  // pieces: copies of N bytes in a head's row
  int page_size, num_pages, max_pages, depth;
};

// Byte offset of slot `at` of a sequence in one side of the cache, or -1 where there is no such slot.
__device__ __forceinline__ int64_t slot_offset(const CacheParams& p, const Side& s, const int32_t* table, int64_t at) {
  if (at < 0 || at >= (int64_t)p.max_pages * p.page_size) return -1;
  const int entry = (int)at / p.page_size, page = table[entry];
  if (page < 0 || page >= p.num_pages) return -1;
  return page * s.page + ((int)at - entry * p.page_size) * s.token;
}

constexpr int kAtOnce = 2;  // pieces of keys, and of values, that a thread asks for before it writes the first

// Rows of one sequence (blockIdx.y): a thread copies pieces of rows' keys and the same pieces of their values.
template <typename Piece>
__global__ void __launch_bounds__(256) cache_append_kernel(const CacheParams p) {
  asm volatile("griddepcontrol.wait;" ::: "memory");
  const int b = blockIdx.y, per_row = p.heads * p.pieces;
  const int64_t i0 = (int64_t)blockIdx.x * (256 * kAtOnce) + threadIdx.x;
  int rows = p.row_counts ? p.row_counts[b] : p.R;
  rows = max(0, min(rows, p.R));
  const int64_t ctx = max(0, p.context_lens[b]);
  const int32_t* table = p.table + b * p.table_stride;
  Piece v[kAtOnce][2];
  int r[kAtOnce], h[kAtOnce], d[kAtOnce];
#pragma unroll
  for (int k = 0; k < kAtOnce; ++k) {
    const int64_t i = i0 + 256 * k;
    // (a 64-bit division takes longer than the copy)
    r[k] = i < 0x7FFFFFFF ? (int)i / per_row : (int)min(i / per_row, (int64_t)p.R);
    const int x = (int)(i - (int64_t)r[k] * per_row);
    h[k] = x / p.pieces;
    d[k] = x - h[k] * p.pieces;
    if (r[k] >= rows) continue;
#pragma unroll
    for (int s = 0; s < 2; ++s)
      v[k][s] = ((const Piece*)(p.side[s].rows + b * p.side[s].row_b + r[k] * p.side[s].row_r + h[k] * p.side[s].row_h))[d[k]];
  }
#pragma unroll
  for (int k = 0; k < kAtOnce; ++k) {
    if (r[k] >= rows) continue;
#pragma unroll
    for (int s = 0; s < 2; ++s) {
      const int64_t at = slot_offset(p, p.side[s], table, ctx + r[k]);
      if (at >= 0) ((Piece*)(p.side[s].cache + at + h[k] * p.side[s].head))[d[k]] = v[k][s];
    }
  }
}

constexpr int kMoves = 8;  // rows of a path that a thread reads before it writes the first

// One block: one layer's keys or values of one sequence (blockIdx.y).  A path ascends, so path[j] >= j: the slot
// that move j fills can be the source of an earlier move but of no later one.  A thread keeps to its own pieces
// and reads a group of rows before it writes them, so no move overwrites what another still has to read.
template <typename Piece>
__global__ void __launch_bounds__(256) cache_commit_kernel(const CacheParams p) {
  asm volatile("griddepcontrol.wait;" ::: "memory");
  const int b = blockIdx.y, layer = blockIdx.x >> 1;
  const Side& s = p.side[blockIdx.x & 1];
  const int64_t ctx = max(0, p.context_lens[b]);
  const int accepted = min(p.accept_len[b], p.depth);
  if (blockIdx.x == 0 && threadIdx.x == 0 && p.out_context_lens) p.out_context_lens[b] = (int32_t)(ctx + max(accepted, -1) + 1);
  const int32_t* table = p.table + b * p.table_stride;
  const int32_t* path = p.path + (int64_t)b * (p.depth + 1);
  char* cache = s.cache + layer * s.layer;
  for (int x = threadIdx.x; x < p.heads * p.pieces; x += blockDim.x) {
    const int h = x / p.pieces, d = x - h * p.pieces;
    const int64_t in_row = h * s.head + (int64_t)d * (int64_t)sizeof(Piece);
    for (int j0 = 0; j0 <= accepted; j0 += kMoves) {
      Piece v[kMoves];
      int64_t to[kMoves];
#pragma unroll
      for (int k = 0; k < kMoves; ++k) {
        const int j = j0 + k;
        to[k] = -1;
        const int node = j <= accepted ? path[j] : j;
        if (node <= j) continue;  // in its place, or no node
        const int64_t from = slot_offset(p, s, table, ctx + node);
        to[k] = from < 0 ? -1 : slot_offset(p, s, table, ctx + j);
        if (to[k] >= 0) v[k] = *(const Piece*)(cache + from + in_row);
      }
#pragma unroll
      for (int k = 0; k < kMoves; ++k)
        if (to[k] >= 0) *(Piece*)(cache + to[k] + in_row) = v[k];
    }
  }
}

// Checks what the calls over a cache share; the cache's sides in bytes.
int read_cache(const ersd_cache* cache, ersd_cache* c, CacheParams* p) {
  if (!cache) return ERSD_EINVAL;
  *c = read_struct(cache);
  if (!c->k || !c->v || !c->block_table || (c->dtype != ERSD_F32 && c->dtype != ERSD_BF16)) return ERSD_EINVAL;
  if (c->num_pages < 1 || c->page_size < 1 || c->heads < 1 || c->head_dim < 1 || c->layers < 1 || c->max_pages < 1) return ERSD_EINVAL;
  const size_t size = c->dtype == ERSD_BF16 ? 2 : 4;
  if (!aligned_to(c->k, size) || !aligned_to(c->v, size) || !aligned_to(c->block_table, 4)) return ERSD_EALIGN;
  if ((int64_t)c->max_pages * c->page_size > (1 << 30) || c->head_dim > (1 << 20) || c->heads > 65535) return ERSD_EUNSUPPORTED;
  memset(p, 0, sizeof *p);
  const int64_t z = (int64_t)size;
  p->side[0] = Side{(char*)c->k, nullptr, c->k_stride_layer * z, c->k_stride_page * z, c->k_stride_token * z, c->k_stride_head * z, 0, 0, 0};
  p->side[1] = Side{(char*)c->v, nullptr, c->v_stride_layer * z, c->v_stride_page * z, c->v_stride_token * z, c->v_stride_head * z, 0, 0, 0};
  p->table = c->block_table;
  p->table_stride = c->table_stride;
  p->heads = c->heads;
  p->page_size = c->page_size;
  p->num_pages = c->num_pages;
  p->max_pages = c->max_pages;
  return ERSD_OK;
}

// Whether every row of a head starts on a 16-byte boundary and is a multiple of 16 bytes long.
bool pieces_of_16(const Side& s, int64_t row_bytes) {
  const int64_t all = s.layer | s.page | s.token | s.head | s.row_b | s.row_r | s.row_h | row_bytes;
  return (all & 15) == 0 && aligned_to(s.cache, 16) && aligned_to(s.rows, 16);
}

// Whether two rows of a side that is written lie in the same place for want of a stride.
bool shares_rows(const ersd_cache& c, const Side& s) {
  return (c.heads > 1 && !s.head) || (c.page_size > 1 && !s.token) || (c.num_pages > 1 && !s.page);
}

// Whether n numbers from a on and m from b on have any in common.
bool meet(const int32_t* a, int64_t n, const int32_t* b, int64_t m) {
  const uintptr_t x = (uintptr_t)a, y = (uintptr_t)b;
  return x < y + 4 * (uintptr_t)m && y < x + 4 * (uintptr_t)n;
}

}  // namespace

}  // namespace ersd

extern "C" int ersd_cache_append(const ersd_cache* cache, const void* k_new, const void* v_new, const int32_t* context_lens, int B, int R,
                                 const ersd_chunk_opts* opts, void* cuda_stream) {
  using namespace ersd;
  ersd_cache c;
  CacheParams p;
  const int st = read_cache(cache, &c, &p);
  if (st != ERSD_OK) return st;
  const ersd_chunk_opts o = read_struct(opts);
  if (!k_new || !v_new || !context_lens || B < 1 || R < 1) return ERSD_EINVAL;
  const int64_t size = c.dtype == ERSD_BF16 ? 2 : 4;
  if (!aligned_to(k_new, size) || !aligned_to(v_new, size) || !aligned_to(context_lens, 4) || !aligned_to(o.row_counts, 4)) return ERSD_EALIGN;
  if (B > 65535 || (int64_t)R * c.heads > (1 << 30)) return ERSD_EUNSUPPORTED;
  const int64_t d = c.head_dim;
  const bool ka = o.a_stride_b || o.a_stride_r || o.a_stride_h, vb = o.b_stride_b || o.b_stride_r || o.b_stride_h;
  p.side[0].rows = (const char*)k_new;
  p.side[0].row_b = (ka ? o.a_stride_b : R * c.heads * d) * size;
  p.side[0].row_r = (ka ? o.a_stride_r : c.heads * d) * size;
  p.side[0].row_h = (ka ? o.a_stride_h : d) * size;
  p.side[1].rows = (const char*)v_new;
  p.side[1].row_b = (vb ? o.b_stride_b : R * c.heads * d) * size;
  p.side[1].row_r = (vb ? o.b_stride_r : c.heads * d) * size;
  p.side[1].row_h = (vb ? o.b_stride_h : d) * size;
  if (shares_rows(c, p.side[0]) || shares_rows(c, p.side[1])) return ERSD_EINVAL;
  p.context_lens = context_lens;
  p.row_counts = o.row_counts;
  p.R = R;
  p.side[0].layer = p.side[1].layer = 0;
  const bool wide = pieces_of_16(p.side[0], d * size) && pieces_of_16(p.side[1], d * size);
  p.pieces = (int)(wide ? d * size / 16 : d);
  const auto kernel = wide ? cache_append_kernel<uint4> : size == 2 ? cache_append_kernel<uint16_t> : cache_append_kernel<uint32_t>;
  const int64_t blocks = ((int64_t)R * c.heads * p.pieces + 256 * kAtOnce - 1) / (256 * kAtOnce);
  if (blocks > 0x7FFFFFFF || (int64_t)c.heads * p.pieces > 0x7FFFFFFF) return ERSD_EUNSUPPORTED;
  note_launch("cache_append_kernel<%s>: 256 threads x (%lld, %d) blocks", wide ? "16 bytes" : "an element", (long long)blocks, B);
  Launch l(dim3((unsigned)blocks, (unsigned)B, 1), 256, 0, (cudaStream_t)cuda_stream);
  const cudaError_t e = cudaLaunchKernelEx(&l.cfg, kernel, p);
  return e == cudaSuccess ? ERSD_OK : cuda_fail(e);
}

extern "C" int ersd_cache_commit(const ersd_cache* cache, const int32_t* context_lens, const int32_t* path, const int32_t* accept_len, int B,
                                 int D, int32_t* out_context_lens, void* cuda_stream) {
  using namespace ersd;
  ersd_cache c;
  CacheParams p;
  const int st = read_cache(cache, &c, &p);
  if (st != ERSD_OK) return st;
  if (!context_lens || !path || !accept_len || B < 1 || D < 0) return ERSD_EINVAL;
  if (!aligned_to(context_lens, 4) || !aligned_to(path, 4) || !aligned_to(accept_len, 4) || !aligned_to(out_context_lens, 4)) return ERSD_EALIGN;
  // (a sequence's other blocks may still have to read what its first would write over)
  if (out_context_lens && (meet(out_context_lens, B, context_lens, B) || meet(out_context_lens, B, accept_len, B) ||
                           meet(out_context_lens, B, path, (int64_t)B * ((int64_t)D + 1))))
    return ERSD_EINVAL;
  if (B > 65535 || D >= ERSD_MAX_ROWS || c.layers > (1 << 20)) return ERSD_EUNSUPPORTED;
  if (shares_rows(c, p.side[0]) || shares_rows(c, p.side[1]) || (c.layers > 1 && (!p.side[0].layer || !p.side[1].layer))) return ERSD_EINVAL;
  const int64_t size = c.dtype == ERSD_BF16 ? 2 : 4, d = c.head_dim;
  p.context_lens = context_lens;
  p.path = path;
  p.accept_len = accept_len;
  p.out_context_lens = out_context_lens;
  p.depth = D;
  const bool wide = pieces_of_16(p.side[0], d * size) && pieces_of_16(p.side[1], d * size);
  p.pieces = (int)(wide ? d * size / 16 : d);
  if ((int64_t)c.heads * p.pieces > 0x7FFFFFFF) return ERSD_EUNSUPPORTED;
  const auto kernel = wide ? cache_commit_kernel<uint4> : size == 2 ? cache_commit_kernel<uint16_t> : cache_commit_kernel<uint32_t>;
  const int work = c.heads * p.pieces, threads = work >= 256 ? 256 : (work + 31) / 32 * 32;
  note_launch("cache_commit_kernel<%s>: %d threads x (%d, %d) blocks", wide ? "16 bytes" : "an element", threads, 2 * c.layers, B);
  Launch l(dim3(2u * (unsigned)c.layers, (unsigned)B, 1), (unsigned)threads, 0, (cudaStream_t)cuda_stream);
  const cudaError_t e = cudaLaunchKernelEx(&l.cfg, kernel, p);
  return e == cudaSuccess ? ERSD_OK : cuda_fail(e);
}
