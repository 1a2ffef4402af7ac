// pages_internal.h -- what the paged cache's translation units share.
#pragma once

#include "ckv_internal.h"

namespace ckv {

inline int page_elem_bytes(int dtype) {
  return dtype == CKV_DTYPE_F32 ? 4 : dtype == CKV_DTYPE_BF16 ? 2 : 1;
}
inline int64_t page_bytes_of(const ckv_page_pool* p) {
  return (int64_t)p->page_size * p->n_kv_heads * p->head_dim * page_elem_bytes(p->dtype);
}
inline int64_t page_stride_bytes(const ckv_page_pool* p) {
  return p->page_stride ? p->page_stride * page_elem_bytes(p->dtype) : page_bytes_of(p);
}

// An array of a call: `n` rows of `bytes` bytes each, `stride` bytes apart.
struct MemRows {
  const void* at;
  int64_t n, bytes, stride;
};
inline MemRows mem_array(const void* at, int64_t bytes) { return MemRows{at, at ? 1 : 0, bytes, bytes}; }
// Whether an array that is written shares a byte with one that is read, or with another that is written
// (rows of one may lie between those of another); up to kMostArrays of each.
constexpr int kMostArrays = 16;
bool writes_overlap(const MemRows* writes, int n_writes, const MemRows* reads, int n_reads);

// A launch has fewer than 2^32 threads along x: workgroups of 256 threads at most.
constexpr int64_t kMaxGrid = int64_t(1) << 24;

// Validate a pool's and a batch's host fields (with_pointers: those of device
// memory too); CKV_OK, or the code of the first fault, with its reason recorded.
ckv_status check_pool(const ckv_page_pool* p, bool with_pointers);
ckv_status check_batch(const ckv_page_batch* b, bool with_pointers);
ckv_status check_groups(const ckv_page_groups* g, const ckv_page_batch* b, bool with_pointers);

// A batch as kernels read it.
struct PageSeqs {
  const int32_t* table;
  const int32_t* lens;
  const int32_t* tok_off;
  int64_t table_stride;
  int64_t n_tokens;
  int32_t n_seqs, max_pages;
};
inline PageSeqs page_seqs(const ckv_page_batch* b) {
  return PageSeqs{b->table, b->lens, b->tok_off, b->table_stride ? b->table_stride : b->max_pages,
                  b->n_tokens, b->n_seqs, b->max_pages};
}

// Sequence b's token rows [first, first + count), whatever tok_off holds inside
// the token tensors, and its length.
struct SeqSpan {
  int64_t first;
  int32_t count, len;
};
__device__ __forceinline__ SeqSpan seq_span(const PageSeqs& s, int b) {
  const int64_t lo = min<int64_t>(max(s.tok_off[b], 0), s.n_tokens);
  const int64_t hi = min<int64_t>(max(s.tok_off[b + 1], 0), s.n_tokens);
  return SeqSpan{lo, (int32_t)max<int64_t>(hi - lo, 0), s.lens[b]};
}

// The last b of n sequences (or groups) with start(b) <= k, -1 if there is none; start must not fall.  A whole
// wave calls it: 64 sequences are looked at at a time (one round of loads for 64 of them, two
// for 4,096).
// Work that the sequences have in parts is numbered so: sequence b's parts from start(b) on,
// where start(b + 1) - start(b) is at least their number and follows from the offsets alone;
// a number past a sequence's last part has no work.
template <class F>
__device__ __forceinline__ int find_seq(int n, int64_t k, F&& start) {
  const int lane = threadIdx.x & 63;
  int lo = 0;
  do {
    const int step = (n + 63) / 64;
    const uint64_t at_most = __ballot(lane * step < n && start(lo + min(lane * step, n - 1)) <= k);
    if (!at_most) return -1;
    const int at = (63 - __builtin_clzll(at_most)) * step;
    lo += at;
    n = min(step, n - at);
  } while (n > 1);
  return lo;
}
// tok_off[b] inside the token tensors.
__device__ __forceinline__ int64_t token_of(const PageSeqs& s, int b) {
  return min<int64_t>(max(s.tok_off[b], 0), s.n_tokens);
}

// The scale of an E4M3 page from its byte: 2^(e - 127), finite whatever the byte (a page
// that no query sees may hold any; its cleared rows then stay 0).
__device__ __forceinline__ float scale_of(uint32_t byte) {
  return __uint_as_float(min(byte, 254u) << 23);
}

}  // namespace ckv
