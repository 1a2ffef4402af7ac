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

// A launch has fewer than 2^32 threads along x: workgroups of 256 threads at most.
constexpr int64_t kMaxGrid = int64_t(1) << 24;

// Validate a pool's and a batch's host fields (with_pointers: those of device
// memory too); CKV_OK, or the code of the first fault, with its reason recorded.
ckv_status check_pool(const ckv_page_pool* p, bool with_pointers);
ckv_status check_batch(const ckv_page_batch* b, bool with_pointers);

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
  const int64_t n = min<int64_t>(s.n_tokens, INT32_MAX);
  const int64_t lo = min<int64_t>(max(s.tok_off[b], 0), n), hi = min<int64_t>(max(s.tok_off[b + 1], 0), n);
  return SeqSpan{lo, (int32_t)max<int64_t>(hi - lo, 0), s.lens[b]};
}

// Work that the sequences have in parts, parts(span) of them each, numbered sequence by
// sequence: the sequence b of part `want`, its span, and the part's number inside it (in
// want).  b = -1 past the last part.  A whole wave calls it: 64 sequences at a time, by a
// running sum over the lanes.
template <class F>
__device__ __forceinline__ int find_part(const PageSeqs& s, F&& parts, int64_t& want, SeqSpan& span) {
  const int lane = threadIdx.x & 63;
  for (int b0 = 0; b0 < s.n_seqs; b0 += 64) {
    SeqSpan mine{0, 0, 0};
    int n = 0;
    if (b0 + lane < s.n_seqs) {
      mine = seq_span(s, b0 + lane);
      if (mine.count > 0) n = parts(mine);
    }
    int sum = n;  // up to this lane
#pragma unroll
    for (int x = 1; x < 64; x <<= 1) {
      const int y = __shfl_up(sum, x);
      if (lane >= x) sum += y;
    }
    const uint64_t past = __ballot((int64_t)sum > want);
    if (past) {
      const int at = __builtin_ctzll(past);
      want -= __builtin_amdgcn_readlane(sum - n, at);
      span.first = (int64_t)__builtin_amdgcn_readlane((int)mine.first, at);  // (below 2^31)
      span.count = __builtin_amdgcn_readlane(mine.count, at);
      span.len = __builtin_amdgcn_readlane(mine.len, at);
      return b0 + at;
    }
    want -= __builtin_amdgcn_readlane(sum, 63);
  }
  return -1;
}

// The scale of an E4M3 page from its byte: 2^(e - 127), finite whatever the byte (a page
// that no query sees may hold any; its cleared rows then stay 0).
__device__ __forceinline__ float scale_of(uint32_t byte) {
  return __uint_as_float(min(byte, 254u) << 23);
}

}  // namespace ckv
