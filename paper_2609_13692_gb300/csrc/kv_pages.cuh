// Launchers of the page operators (k_kv_pages.cu), called by mpt_kv.cu.
#pragma once

#include "kv_internal.cuh"

namespace mpt {

constexpr int kMergeParts = 16;

struct MergeParams {
  const void* outs[kMergeParts];
  const float* lses[kMergeParts];
  void* out;
  float* lse;  // or nullptr
  int64_t rows;
  int32_t vecs;  // 16-byte pieces of a row
  int32_t n;
};
cudaError_t launch_kv_merge(const MergeParams& p, int type, cudaStream_t stream);

struct WriteParams {
  const char *k_new, *v_new;
  char *k, *v;  // everything below in 16-byte pieces
  int64_t k_new_tok, k_new_head, v_new_tok, v_new_head, k_page, k_slot, k_head, v_page, v_slot, v_head;
  const int32_t* table;
  int64_t table_stride;
  const int32_t* q_offsets;
  const int32_t* kv_lens;
  int64_t tokens;
  int32_t width, n_pages, page_log2, batch, kv_heads, vecs;  // vecs: pieces of a head
};
cudaError_t launch_kv_write(const WriteParams& p, cudaStream_t stream);

struct CopyParams {
  char* pool;
  int64_t plane_stride, page_stride, page_bytes;
  const int32_t *src, *dst;
  int32_t planes, n_pages, n;
};
constexpr int kCopyThreads = 256, kCopyVecs = 4, kCopySeg = kCopyThreads * kCopyVecs * 16;
// Units of a page in one plane; the units of all pairs and planes are counted in 64 bits.
__host__ __device__ constexpr int64_t copy_segments(int64_t page_bytes) { return (page_bytes + kCopySeg - 1) / kCopySeg; }
cudaError_t launch_kv_copy_pages(const CopyParams& p, cudaStream_t stream);

struct BookParams {
  mpt_kv_book b;
  int32_t page_log2, n;
  const int32_t *l0, *l1, *l2;  // fork: src, dst, keep; extend: rows, more; free: rows
  int32_t *copy_src, *copy_dst, *status;
};
constexpr int kBookList = 16384;  // entries of a list, at most: 4 bytes of shared memory each, beside a bit per row
enum BookOp { kBookFork, kBookExtend, kBookFree, kBookCompact };
cudaError_t launch_kv_book(const BookParams& p, BookOp op, cudaStream_t stream);

// The kernels' counts (in the default build they have none to make).
cudaError_t kv_pages_counts(cudaStream_t stream, uint32_t* counts);

}  // namespace mpt
