// A cache of keys and values in pages, and the sequences of one step over it: what the append and the attention share.
// Everything the device is told by device memory (row ranges, lengths, page numbers) is checked there before it becomes an address.
#pragma once
#include <cuda_bf16.h>

#include <utility>

#include "mst_internal.cuh"
#include "mst_paged_list.h"

namespace mst_paged {

struct Cache {
  __nv_bfloat16 *K, *V;
  int64_t page_stride, token_stride, head_stride;
  int num_pages, page_size, kv_heads, D;
  Divider by_page;
};
struct Batch {
  const int32_t *first, *len, *table;
  int batch, tokens, table_stride;
};

inline mst_status_t check(const mst_paged_cache_t* c, const mst_paged_batch_t* b, Cache* cache, Batch* batch) {
  if (!c || !b || !c->K || !c->V) return MST_ERR_INVALID_ARG;
  if (c->num_pages < 0 || c->page_size <= 0 || c->kv_heads <= 0 || c->head_dim <= 0 || b->batch < 0 || b->tokens < 0 || b->table_stride < 0 ||
      b->max_new < 0 || b->max_len < 0)
    return MST_ERR_INVALID_ARG;
  if (b->batch > 0 && (!b->first || !b->len || (!b->page_table && b->table_stride > 0))) return MST_ERR_INVALID_ARG;
  if (c->kv_heads > 65535 || b->batch > 65535) return MST_ERR_SHAPE;
  if (c->page_stride < 0 || c->token_stride < 0 || c->head_stride < 0 || c->page_stride % 8 != 0 || c->token_stride % 8 != 0 ||
      c->head_stride % 8 != 0)
    return MST_ERR_SHAPE;
  // Rows of different slots or heads do not overlap: with strides in ascending order each is at least what those before it span.  And a cache
  // lies within an address space of 57 bits: products of strides and counts stay in 64
  struct { int64_t stride, n; } dims[3] = {{c->head_stride, c->kv_heads}, {c->token_stride, c->page_size}, {c->page_stride, c->num_pages}};
  for (int i = 0; i < 2; ++i)
    for (int k = 0; k < 2; ++k)
      if (dims[k + 1].stride < dims[k].stride) std::swap(dims[k], dims[k + 1]);
  int64_t span = c->head_dim;
  for (const auto& x : dims) {
    if (x.n <= 1) continue;
    if (x.stride < span || x.stride > ((INT64_C(1) << 56) - span) / (x.n - 1)) return MST_ERR_SHAPE;
    span += x.stride * (x.n - 1);
  }
  if (((reinterpret_cast<uintptr_t>(c->K) | reinterpret_cast<uintptr_t>(c->V)) & 15u) != 0 ||
      ((reinterpret_cast<uintptr_t>(b->first) | reinterpret_cast<uintptr_t>(b->len) | reinterpret_cast<uintptr_t>(b->page_table)) & 3u) != 0)
    return MST_ERR_SHAPE;
  *cache = Cache{(__nv_bfloat16*)c->K, (__nv_bfloat16*)c->V, c->page_stride, c->token_stride, c->head_stride,
                 c->num_pages, c->page_size, c->kv_heads, c->head_dim, Divider::of((uint32_t)c->page_size)};
  *batch = Batch{b->first, b->len, b->page_table, b->batch, b->tokens, b->table_stride};
  return MST_OK;
}

#ifdef __CUDACC__
struct Slot {
  bool exists;
  int64_t at;    // element of the slot's first head
};
// Slot of position p (p >= 0) of sequence b.  `flag`: the file's own word for pages that do not exist
__device__ __forceinline__ Slot slot_of(const Cache& C, const Batch& B, int b, int p, int* flag) {
  int slot;
  const int id = page_of(B.table + (int64_t)b * B.table_stride, B.table_stride, C.by_page, C.num_pages, p, slot);
  if (id < 0) {
    *flag = 1;
    return Slot{false, 0};
  }
  return Slot{true, (int64_t)id * C.page_stride + (int64_t)slot * C.token_stride};
}
// The sequence that a row belongs to (a warp's question, all lanes the same row): how many sequences end at or before it.  -1: none, or one that
// RowsOf gives no rows.  `flag`: the file's own word for sequences with rows outside 0 .. tokens - 1
__device__ __forceinline__ int sequence_of(const Batch& B, int row, int lane, int* flag) {
  int before = 0;
  for (int i0 = 0; i0 < B.batch; i0 += 32) {
    const int end = i0 + lane < B.batch ? B.first[i0 + lane + 1] : INT32_MIN;
    if (end > B.tokens) *flag = 1;
    before += __popc(__ballot_sync(0xffffffffu, i0 + lane < B.batch && end <= row));
  }
  if (before >= B.batch) return -1;
  const int first = B.first[before];
  if (first < 0) *flag = 1;
  return first >= 0 && first <= row && row < B.first[before + 1] ? before : -1;
}
// The position of row `row` of sequence b, below 0 where the sequence is shorter than its new tokens
__device__ __forceinline__ int position_of(const Batch& B, int b, int row) {
  const int64_t p = (int64_t)B.len[b] - B.first[b + 1] + row;
  return p < 0 ? -1 : (int)p;
}
// A file's word for pages that do not exist, or for rows: its value, and zero from then on
inline mst_status_t take_flag(const void* symbol, int32_t* flag) {
  int v = 0;
  MST_CUDA_TRY(cudaMemcpyFromSymbol(&v, symbol, sizeof(int)));
  const int zero = 0;
  if (v) MST_CUDA_TRY(cudaMemcpyToSymbol(symbol, &zero, sizeof(int)));
  *flag = v;
  return MST_OK;
}
#endif

}  // namespace mst_paged
