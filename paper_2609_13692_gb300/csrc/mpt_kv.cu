// C ABI of the paged-cache operators (include/mpt_kv.h): argument checks,
// tensor maps and launches.
#include <cmath>
#include <cstring>

#include "kv_pages.cuh"
#include "kv_report.h"

namespace mpt {
namespace {

bool page_log2(int page_size, int* log2) {
  for (int l = 3; l <= 8; ++l)
    if (page_size == 1 << l) {
      *log2 = l;
      return true;
    }
  return false;
}

bool aligned(const void* p, uintptr_t a) { return ((uintptr_t)p & (a - 1)) == 0; }
bool stride_ok(int64_t s, int64_t entries) {
  return entries == 1 || (s > 0 && s % 8 == 0 && s < (int64_t)1 << 38);
}

mpt_status check_cache(const mpt_kv_cache* c, int64_t tokens, int* log2) {
  if (!c || !c->k || !c->v || !aligned(c->k, 16) || !aligned(c->v, 16)) return MPT_ERR_INVALID_ARG;
  if (c->type != MPT_KV_BF16 && c->type != MPT_KV_F16) return MPT_ERR_INVALID_ARG;
  if (!page_log2(c->page_size, log2) || c->n_pages < 1 || c->kv_heads < 1 || c->batch < 0 || c->table_width < 1)
    return MPT_ERR_INVALID_ARG;
  if (c->head_dim < 8 || c->head_dim % 8 != 0 || tokens < 0) return MPT_ERR_INVALID_ARG;
  if (c->head_dim > 256 || c->kv_heads > 1024 || c->batch > 1 << 20 || tokens > INT32_MAX) return MPT_ERR_TOO_LARGE;
  if ((int64_t)c->table_width << *log2 > INT32_MAX) return MPT_ERR_TOO_LARGE;
  // a stride of 0 only along an axis of one entry
  const int entries[3] = {c->n_pages, c->page_size, c->kv_heads};
  for (int i = 0; i < 3; ++i)
    if (!stride_ok(c->k_stride[i], entries[i]) || !stride_ok(c->v_stride[i], entries[i])) return MPT_ERR_INVALID_ARG;
  if (c->batch > 0 && (!c->page_table || !c->q_offsets || !c->kv_lens || c->table_stride < c->table_width))
    return MPT_ERR_INVALID_ARG;
  if (!aligned(c->page_table, 4) || !aligned(c->q_offsets, 4) || !aligned(c->kv_lens, 4)) return MPT_ERR_INVALID_ARG;
  return MPT_OK;
}

using EncodeTiled = CUresult (*)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*,
                                 const cuuint64_t*, const cuuint32_t*, const cuuint32_t*, CUtensorMapInterleave,
                                 CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

EncodeTiled encode_tiled() {
  static const EncodeTiled fn = [] {
    void* f = nullptr;
    cudaDriverEntryPointQueryResult found;
    if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &f, 12000, cudaEnableDefault, &found) != cudaSuccess ||
        found != cudaDriverEntryPointSuccess)
      f = nullptr;
    return (EncodeTiled)f;
  }();
  return fn;
}

// Reads go to L2 in pieces of 256 bytes where a head's elements are whole such
// pieces, else of 128: larger ones fetch a neighbouring head's bytes too (64
// requests of 2,000 to 6,000 keys, 16 heads of 64: 259 against 203 us; heads of
// 96: 89 against 76), smaller ones cost heads of 128 a hundredth.
CUtensorMapL2promotion promotion(int dim) {
  return dim * 2 % 256 == 0 ? CU_TENSOR_MAP_L2_PROMOTION_L2_256B : CU_TENSOR_MAP_L2_PROMOTION_L2_128B;
}

// (element, slot, KV head, page) of K or V, copied `box` slots of 64 elements
// at a time into rows of 128 bytes with their 16-byte pieces permuted by row.
bool make_map(CUtensorMap* map, const mpt_kv_cache& c, const void* at, const int64_t* stride, int box) {
  const EncodeTiled fn = encode_tiled();
  if (!fn) return false;
  const cuuint64_t dims[4] = {(cuuint64_t)c.head_dim, (cuuint64_t)c.page_size, (cuuint64_t)c.kv_heads, (cuuint64_t)c.n_pages};
  // a stride along an axis of one entry is never used, whatever the caller has there
  const cuuint64_t strides[3] = {(cuuint64_t)stride[1] * 2, c.kv_heads > 1 ? (cuuint64_t)stride[2] * 2 : 16,
                                 c.n_pages > 1 ? (cuuint64_t)stride[0] * 2 : 16};
  const cuuint32_t boxes[4] = {64, (cuuint32_t)box, 1, 1}, ones[4] = {1, 1, 1, 1};
  return fn(map, c.type == MPT_KV_F16 ? CU_TENSOR_MAP_DATA_TYPE_FLOAT16 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 4,
            const_cast<void*>(at), dims, strides, boxes, ones, CU_TENSOR_MAP_INTERLEAVE_NONE,
            CU_TENSOR_MAP_SWIZZLE_128B, promotion(c.head_dim), CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// (element, query head, token) of the queries, copied as whole tokens' heads
// of one KV head, at most 128 rows at a time.
bool make_query_map(CUtensorMap* map, const AttnParams& p, bool f16) {
  const EncodeTiled fn = encode_tiled();
  if (!fn) return false;
  const cuuint64_t dims[3] = {(cuuint64_t)p.dim, (cuuint64_t)p.heads, (cuuint64_t)p.tokens};
  const cuuint64_t strides[2] = {p.heads > 1 ? (cuuint64_t)p.q_head * 2 : 16, p.tokens > 1 ? (cuuint64_t)p.q_tok * 2 : 16};
  const cuuint32_t boxes[3] = {64, (cuuint32_t)p.group, (cuuint32_t)(128 / p.group)}, ones[3] = {1, 1, 1};
  return fn(map, f16 ? CU_TENSOR_MAP_DATA_TYPE_FLOAT16 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16, 3, const_cast<char*>(p.q), dims,
            strides, boxes, ones, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
            promotion(p.dim), CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// Whether [a, a + an) and [b, b + bn) share a byte.
bool overlap(const void* a, int64_t an, const void* b, int64_t bn) {
  const uintptr_t x = (uintptr_t)a, y = (uintptr_t)b;
  return x < y ? y - x < (uint64_t)an : x - y < (uint64_t)bn;
}

size_t attend_workspace(int sms) {
  const size_t few = attend_few_workspace(sms), tile = attend_tile_workspace(sms);
  return few > tile ? few : tile;
}

}  // namespace
}  // namespace mpt

extern "C" {

mpt_status mpt_kv_attend_workspace_bytes(int32_t head_dim, size_t* bytes) {
  if (!bytes || head_dim < 8 || head_dim > 256 || head_dim % 8 != 0) return MPT_ERR_INVALID_ARG;
  int device = 0;
  *bytes = mpt::attend_workspace(mpt::kv_sm_count(&device));
  return MPT_OK;
}

mpt_status mpt_kv_attend(const mpt_kv_cache* c, const void* q, const int64_t* q_stride, int64_t tokens, int32_t heads,
                         int32_t max_q_len, int32_t causal, float scale, void* out, const int64_t* out_stride,
                         float* lse, void* workspace, size_t workspace_bytes, void* stream_ptr) {
  int log2 = 0;
  const mpt_status st = mpt::check_cache(c, tokens, &log2);
  if (st != MPT_OK) return st;
  if (heads < 1 || heads % c->kv_heads != 0 || max_q_len < 0 || !std::isfinite(scale) || !(scale > 0.f) || !q_stride || !out_stride)
    return MPT_ERR_INVALID_ARG;
  if (heads / c->kv_heads > 128 || tokens * (heads / c->kv_heads) > INT32_MAX) return MPT_ERR_TOO_LARGE;
  const int64_t entries[2] = {tokens, heads};
  for (int i = 0; i < 2; ++i)
    if (!mpt::stride_ok(q_stride[i], entries[i]) || !mpt::stride_ok(out_stride[i], entries[i])) return MPT_ERR_INVALID_ARG;
  if (tokens == 0 || c->batch == 0) return MPT_OK;
  if (!q || !out || !mpt::aligned(q, 16) || !mpt::aligned(out, 16) || !mpt::aligned(lse, 4)) return MPT_ERR_INVALID_ARG;
  int device = 0;
  const int sms = mpt::kv_sm_count(&device);
  if (!workspace || !mpt::aligned(workspace, 256)) return MPT_ERR_INVALID_ARG;
  if (workspace_bytes < mpt::attend_workspace(sms)) return MPT_ERR_WORKSPACE_TOO_SMALL;

  mpt::AttnParams p;
  std::memset((void*)&p, 0, sizeof(p));
  p.q = (const char*)q;
  p.out = (char*)out;
  p.lse = lse;
  p.q_tok = q_stride[0], p.q_head = q_stride[1], p.out_tok = out_stride[0], p.out_head = out_stride[1];
  p.table = c->page_table;
  p.table_stride = c->table_stride;
  p.q_offsets = c->q_offsets;
  p.kv_lens = c->kv_lens;
  p.desc = (int4*)workspace;
  p.part = (float*)((char*)workspace + ((size_t)sms * mpt::kFewPerSm * sizeof(int4) + 255) / 256 * 256);
  p.tokens = tokens;
  p.width = c->table_width;
  p.n_pages = c->n_pages;
  p.page_log2 = log2;
  p.batch = c->batch;
  p.heads = heads;
  p.kv_heads = c->kv_heads;
  p.group = heads / c->kv_heads;
  p.dim = c->head_dim;
  p.toks = 128 / p.group;
  p.item_toks = p.toks * (p.dim > 128 ? 1 : 2);
  p.wide = p.dim % 16 == 0 && mpt::aligned(out, 32) && (heads == 1 || p.out_head % 16 == 0) && (tokens == 1 || p.out_tok % 16 == 0);
  p.causal = causal != 0;
  p.scale_log2 = scale * 1.4426950408889634f;
  cudaStream_t stream = (cudaStream_t)stream_ptr;
  const bool f16 = c->type == MPT_KV_F16;
  p.k = (const char*)c->k, p.v = (const char*)c->v;
  p.k_page = c->k_stride[0], p.k_slot = c->k_stride[1], p.k_head = c->k_stride[2];
  p.v_page = c->v_stride[0], p.v_slot = c->v_stride[1], p.v_head = c->v_stride[2];
  // Few rows per KV head: 16 of them fill the smaller kernel's products.  Where
  // the caller does not say, as many tokens as requests are taken for one each.
  const int64_t most = max_q_len > 0 ? max_q_len : tokens <= c->batch ? 1 : 129;
  const bool tile = most * p.group > 16 && c->batch <= mpt::kTileBatch;
  const int keys = tile ? 128 : 64;
  p.box = c->page_size < keys ? c->page_size : keys;
  if (!mpt::make_map(&p.map_k, *c, c->k, c->k_stride, p.box) || !mpt::make_map(&p.map_v, *c, c->v, c->v_stride, p.box) ||
      (tile && !mpt::make_query_map(&p.map_q, p, f16)))
    return MPT_ERR_CUDA;
  const cudaError_t e = tile ? mpt::launch_attend_tile(p, f16, sms, device, stream)
                             : mpt::launch_attend_few(p, f16, most * p.group < 16 ? (int)(most * p.group) : 16, sms, device, stream);
  return e == cudaSuccess ? MPT_OK : MPT_ERR_CUDA;
}

mpt_status mpt_kv_merge(const void* const* outs, const float* const* lses, int32_t n_parts, int64_t rows,
                        int32_t head_dim, int32_t type, void* out, float* lse, void* stream) {
  if (!outs || !lses || n_parts < 1 || rows < 0 || head_dim < 8 || head_dim % 8 != 0) return MPT_ERR_INVALID_ARG;
  if (type != MPT_KV_BF16 && type != MPT_KV_F16 && type != MPT_KV_F32) return MPT_ERR_INVALID_ARG;
  if (n_parts > mpt::kMergeParts || head_dim > 1024 || rows > (int64_t)1 << 40) return MPT_ERR_TOO_LARGE;
  if (rows == 0) return MPT_OK;
  if (!out || !mpt::aligned(out, 16) || !mpt::aligned(lse, 4)) return MPT_ERR_INVALID_ARG;
  mpt::MergeParams p;
  std::memset(&p, 0, sizeof(p));
  // A thread reads its own 16 bytes of every part's out and writes them at one
  // address: out may be a part.  A row's sums are read by all its threads.
  const int64_t out_bytes = rows * head_dim * (type == MPT_KV_F32 ? 4 : 2), lse_bytes = rows * (int64_t)sizeof(float);
  if (lse && mpt::overlap(out, out_bytes, lse, lse_bytes)) return MPT_ERR_INVALID_ARG;
  for (int i = 0; i < n_parts; ++i) {
    if (!outs[i] || !lses[i] || !mpt::aligned(outs[i], 16) || !mpt::aligned(lses[i], 4)) return MPT_ERR_INVALID_ARG;
    if ((outs[i] != out && mpt::overlap(outs[i], out_bytes, out, out_bytes)) || mpt::overlap(lses[i], lse_bytes, out, out_bytes))
      return MPT_ERR_INVALID_ARG;
    if (lse && (mpt::overlap(lses[i], lse_bytes, lse, lse_bytes) || mpt::overlap(outs[i], out_bytes, lse, lse_bytes)))
      return MPT_ERR_INVALID_ARG;
    p.outs[i] = outs[i];
    p.lses[i] = lses[i];
  }
  p.out = out;
  p.lse = lse;
  p.rows = rows;
  p.vecs = head_dim / (type == MPT_KV_F32 ? 4 : 8);
  p.n = n_parts;
  return mpt::launch_kv_merge(p, type, (cudaStream_t)stream) == cudaSuccess ? MPT_OK : MPT_ERR_CUDA;
}

mpt_status mpt_kv_write(const mpt_kv_cache* c, const void* k_new, const int64_t* k_stride, const void* v_new,
                        const int64_t* v_stride, int64_t tokens, void* stream) {
  int log2 = 0;
  const mpt_status st = mpt::check_cache(c, tokens, &log2);
  if (st != MPT_OK) return st;
  if (!k_stride || !v_stride) return MPT_ERR_INVALID_ARG;
  const int64_t entries[2] = {tokens, c->kv_heads};
  for (int i = 0; i < 2; ++i)
    if (!mpt::stride_ok(k_stride[i], entries[i]) || !mpt::stride_ok(v_stride[i], entries[i])) return MPT_ERR_INVALID_ARG;
  if (tokens == 0 || c->batch == 0) return MPT_OK;
  if (!k_new || !v_new || !mpt::aligned(k_new, 16) || !mpt::aligned(v_new, 16)) return MPT_ERR_INVALID_ARG;
  mpt::WriteParams p;
  std::memset(&p, 0, sizeof(p));
  p.k_new = (const char*)k_new, p.v_new = (const char*)v_new, p.k = (char*)c->k, p.v = (char*)c->v;
  p.k_new_tok = k_stride[0] / 8, p.k_new_head = k_stride[1] / 8, p.v_new_tok = v_stride[0] / 8, p.v_new_head = v_stride[1] / 8;
  p.k_page = c->k_stride[0] / 8, p.k_slot = c->k_stride[1] / 8, p.k_head = c->k_stride[2] / 8;
  p.v_page = c->v_stride[0] / 8, p.v_slot = c->v_stride[1] / 8, p.v_head = c->v_stride[2] / 8;
  p.table = c->page_table, p.table_stride = c->table_stride, p.q_offsets = c->q_offsets, p.kv_lens = c->kv_lens;
  p.tokens = tokens, p.width = c->table_width, p.n_pages = c->n_pages, p.page_log2 = log2, p.batch = c->batch;
  p.kv_heads = c->kv_heads, p.vecs = c->head_dim / 8;
  return mpt::launch_kv_write(p, (cudaStream_t)stream) == cudaSuccess ? MPT_OK : MPT_ERR_CUDA;
}

}  // extern "C"

namespace mpt {
namespace {

mpt_status check_book(const mpt_kv_book* b, int32_t n, int* log2) {
  if (!b || !b->table || !b->lens || !b->refs || b->width < 1 || b->rows < 1 || b->n_pages < 1 || b->table_stride < b->width || n < 0 ||
      !page_log2(b->page_size, log2))
    return MPT_ERR_INVALID_ARG;
  if (!aligned(b->table, 4) || !aligned(b->lens, 4) || !aligned(b->refs, 4)) return MPT_ERR_INVALID_ARG;
  if (b->rows > 1 << 20 || b->n_pages >= 1 << 30 || (int64_t)b->width << *log2 > INT32_MAX || n > b->rows || n > kBookList)
    return MPT_ERR_TOO_LARGE;
  return MPT_OK;
}

mpt_status run_book(const mpt_kv_book* b, BookOp op, const int32_t* l0, const int32_t* l1, const int32_t* l2, int32_t lists,
                    int32_t n, int32_t* copy_src, int32_t* copy_dst, int32_t* status, void* stream) {
  int log2 = 0;
  const mpt_status st = check_book(b, n, &log2);
  if (st != MPT_OK) return st;
  const int32_t* list[3] = {l0, l1, l2};
  for (int i = 0; i < lists; ++i)
    if (n > 0 && (!list[i] || !aligned(list[i], 4))) return MPT_ERR_INVALID_ARG;
  const bool copies = op == kBookFork ? n > 0 : op == kBookCompact && b->n_pages > 1;
  if (copies && (!copy_src || !copy_dst || !aligned(copy_src, 4) || !aligned(copy_dst, 4) || copy_src == copy_dst)) return MPT_ERR_INVALID_ARG;
  if (!status || !aligned(status, 4)) return MPT_ERR_INVALID_ARG;
  BookParams p;
  std::memset(&p, 0, sizeof(p));
  p.b = *b;
  p.page_log2 = log2;
  p.n = n;
  p.l0 = l0, p.l1 = l1, p.l2 = l2;
  p.copy_src = copy_src, p.copy_dst = copy_dst, p.status = status;
  return launch_kv_book(p, op, (cudaStream_t)stream) == cudaSuccess ? MPT_OK : MPT_ERR_CUDA;
}

}  // namespace
}  // namespace mpt

extern "C" {

mpt_status mpt_kv_fork(const mpt_kv_book* book, const int32_t* src, const int32_t* dst, const int32_t* keep, int32_t n,
                       int32_t* copy_src, int32_t* copy_dst, int32_t* status, void* stream) {
  return mpt::run_book(book, mpt::kBookFork, src, dst, keep, 3, n, copy_src, copy_dst, status, stream);
}

mpt_status mpt_kv_extend(const mpt_kv_book* book, const int32_t* rows, const int32_t* more, int32_t n, int32_t* status,
                         void* stream) {
  return mpt::run_book(book, mpt::kBookExtend, rows, more, nullptr, 2, n, nullptr, nullptr, status, stream);
}

mpt_status mpt_kv_free(const mpt_kv_book* book, const int32_t* rows, int32_t n, int32_t* status, void* stream) {
  return mpt::run_book(book, mpt::kBookFree, rows, nullptr, nullptr, 1, n, nullptr, nullptr, status, stream);
}

mpt_status mpt_kv_compact(const mpt_kv_book* book, int32_t* copy_src, int32_t* copy_dst, int32_t* status, void* stream) {
  return mpt::run_book(book, mpt::kBookCompact, nullptr, nullptr, nullptr, 0, 0, copy_src, copy_dst, status, stream);
}

mpt_status mpt_kv_copy_pages(void* pool, int32_t planes, int64_t plane_stride, int32_t n_pages, int64_t page_stride,
                             int64_t page_bytes, const int32_t* src, const int32_t* dst, int32_t n, void* stream) {
  if (!pool || planes < 1 || n_pages < 1 || n < 0 || page_bytes < 16 || page_stride < page_bytes || plane_stride < 0)
    return MPT_ERR_INVALID_ARG;
  if (!mpt::aligned(pool, 16) || plane_stride % 16 || page_stride % 16 || page_bytes % 16) return MPT_ERR_INVALID_ARG;
  if (n_pages >= 1 << 30 || n >= 1 << 30 || planes > 1 << 16 || page_bytes > (int64_t)1 << 32 || page_stride > (int64_t)1 << 32 ||
      plane_stride > (int64_t)1 << 46 || (int64_t)n * planes > (INT64_MAX >> 1) / mpt::copy_segments(page_bytes))
    return MPT_ERR_TOO_LARGE;
  if (n == 0) return MPT_OK;
  if (!src || !dst || !mpt::aligned(src, 4) || !mpt::aligned(dst, 4)) return MPT_ERR_INVALID_ARG;
  mpt::CopyParams p;
  p.pool = (char*)pool;
  p.plane_stride = plane_stride, p.page_stride = page_stride, p.page_bytes = page_bytes;
  p.src = src, p.dst = dst;
  p.planes = planes, p.n_pages = n_pages, p.n = n;
  return mpt::launch_kv_copy_pages(p, (cudaStream_t)stream) == cudaSuccess ? MPT_OK : MPT_ERR_CUDA;
}

mpt_status mpt_kv_check(void* stream_ptr) {
  static mpt::Reported few, tile, outside[3];
  cudaStream_t stream = (cudaStream_t)stream_ptr;
  uint32_t f[mpt::kKvCounts], t[mpt::kKvCounts], g[mpt::kKvCounts];
  int device = 0;
  if (cudaGetDevice(&device) != cudaSuccess || mpt::attend_few_counts(stream, f) != cudaSuccess ||
      mpt::attend_tile_counts(stream, t) != cudaSuccess || mpt::kv_pages_counts(stream, g) != cudaSuccess || cudaStreamSynchronize(stream) != cudaSuccess)
    return MPT_ERR_CUDA;
  const bool in_few = few.news(device, f[mpt::kKvGaveUp]), in_tile = tile.news(device, t[mpt::kKvGaveUp]);
  bool bad = false;
  const uint32_t* const counts[3] = {f, t, g};
  for (int i = 0; i < 3; ++i) bad |= outside[i].news(device, counts[i][mpt::kKvOutside]);
  return bad ? MPT_ERR_INTERNAL : in_few || in_tile ? MPT_ERR_TIMEOUT : MPT_OK;
}

}  // extern "C"
