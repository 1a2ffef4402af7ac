// page_tables.hip -- the tables of a paged cache's sequences for gfx950: what groups share, forks
// after a step's parents, pages and slots of a step's new tokens.
//
// Integers throughout: page numbers, lengths, use counts.  A call moves a megabyte or two at
// most, in the L2s' reach: launches and the dependent loads of a workgroup (a length, a table
// entry, that page's count) are what it takes.  Sums are of integers, so atomics leave the
// same result in any order.  Measured: shares of four sequences 3.4 us, of 48 on 30,000 tokens 8.8; a
// fork of 256 sequences of 500 pages 7.8 (3.0 and 4.3 in its two kernels); a step of as many on
// 65,536 pages 11.4 (7.9 and 3.7), 40 prompts of up to 6,000 tokens 9.8.

#include "pages_internal.h"

namespace ckv {

ckv_status check_groups(const ckv_page_groups* g, const ckv_page_batch* b, bool with_pointers) {
  if (!g) CKV_FAIL(CKV_EINVAL, "groups is NULL");
  if (g->n_groups < 0 || g->n_groups > (1 << 20))
    CKV_FAIL(CKV_EINVAL, "n_groups must be in [0, 2^20] (got %d)", g->n_groups);
  if (g->max_tokens < 0 || g->max_shared < 0) CKV_FAIL(CKV_EINVAL, "max_tokens and max_shared must be >= 0");
  if (with_pointers && g->n_groups > 0 && b->n_seqs > 0 && b->n_tokens > 0 && (!g->grp_off || !g->shared))
    CKV_FAIL(CKV_EINVAL, "NULL groups pointer");
  return CKV_OK;
}

namespace {

// ---- block-wide sums ------------------------------------------------------------------

// Inclusive sums over a wave's lanes, by moves between lanes (a row of 16, then the last lane
// of each row to the next rows).
template <int CTRL, int ROWS>
__device__ __forceinline__ int moved(int x, int none = 0) {
  return __builtin_amdgcn_update_dpp(none, x, CTRL, ROWS, 0xF, false);
}
template <int CTRL, int ROWS>
__device__ __forceinline__ int64_t moved(int64_t x) {
  return (int64_t)join64((uint32_t)moved<CTRL, ROWS>((int)(x >> 32)), (uint32_t)moved<CTRL, ROWS>((int)x));
}
template <class T>
__device__ __forceinline__ T wave_upto(T x) {
  x += moved<kDppRowShr1, 0xF>(x);
  x += moved<kDppRowShr2, 0xF>(x);
  x += moved<kDppRowShr4, 0xF>(x);
  x += moved<kDppRowShr8, 0xF>(x);
  x += moved<0x142, 0xA>(x);  // lane 15 of rows 0 and 2 to rows 1 and 3
  x += moved<0x143, 0xC>(x);  // lane 31 to rows 2 and 3
  return x;
}
// The least of a wave's lanes, for all of them.
__device__ __forceinline__ int wave_least(int x) {
  x = min(x, moved<kDppRowShr1, 0xF>(x, INT32_MAX));
  x = min(x, moved<kDppRowShr2, 0xF>(x, INT32_MAX));
  x = min(x, moved<kDppRowShr4, 0xF>(x, INT32_MAX));
  x = min(x, moved<kDppRowShr8, 0xF>(x, INT32_MAX));
  x = min(x, moved<0x142, 0xA>(x, INT32_MAX));
  x = min(x, moved<0x143, 0xC>(x, INT32_MAX));
  return __builtin_amdgcn_readlane(x, 63);
}
// The sum of x over all threads, for all of them.
template <int kThreads>
__device__ __forceinline__ int block_total(int x) {
  __shared__ int part[kThreads / 64];
  x = wave_upto(x);
  if ((threadIdx.x & 63) == 63) part[threadIdx.x >> 6] = x;
  __syncthreads();
  const int lane = threadIdx.x & 63;
  x = wave_upto(lane < kThreads / 64 ? part[lane] : 0);
  __syncthreads();
  return __builtin_amdgcn_readlane(x, 63);
}
// Each x becomes its sum over the threads before this one; `total` gets those of all.
template <int kThreads, int N, class T>
__device__ __forceinline__ void block_before(T (&x)[N], T (&total)[N]) {
  constexpr int kWaves = kThreads / 64;
  static_assert(kWaves <= 64);
  __shared__ T part[N][kWaves];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  T upto[N];
#pragma unroll
  for (int i = 0; i < N; ++i) {
    upto[i] = wave_upto(x[i]);
    if (lane == 63) part[i][wave] = upto[i];
  }
  __syncthreads();
#pragma unroll
  for (int i = 0; i < N; ++i) {
    const T p = lane < kWaves ? part[i][lane] : T(0), w = wave_upto(p);
    total[i] = __shfl(w, kWaves - 1);
    x[i] = __shfl(w - p, wave) + upto[i] - x[i];
  }
  __syncthreads();
}

// ---- share ----------------------------------------------------------------------------

struct ShareArgs {
  PageSeqs s;
  const int32_t* grp_off;
  int32_t* shared;  // [n_groups] tokens, [n_groups] leaders, [n_seqs] tokens
  int n_groups, c;
};

// A workgroup per group: its waves go over the sequences in turn, lanes along the table,
// against the first sequence with tokens.  One more for the sequences of no group.
// Its time is that of the loads' rounds, one after the other (offsets, lengths, tables: four sequences of
// 65 pages 3.4 us), and of one CU's misses (48 of 970 pages 8.8; a sequence of a wave at a time 11.4).
constexpr int kShareThreads = 1024, kShareBatch = 16, kShareSeqs = 4;
__global__ __launch_bounds__(kShareThreads) void share_kernel(ShareArgs a) {
  const auto begin_of = [&](int g) { return min(max(a.grp_off[g], 0), a.s.n_seqs); };
  const int g = blockIdx.x, tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  int32_t* const of_seq = a.shared + 2 * (int64_t)a.n_groups;
  if (g == a.n_groups) {
    const int lo = begin_of(0), hi = begin_of(a.n_groups);
    for (int b = tid; b < a.s.n_seqs; b += kShareThreads)
      if (b < lo || b >= hi) of_seq[b] = 0;
    return;
  }
  const int f = begin_of(g), l = begin_of(g + 1);
  constexpr int kWavesOf = kShareThreads / 64;
  __shared__ int common;
  // Every wave goes over the group's sequences itself, 64 at a time: no wave waits for another.
  int leader = INT32_MAX, least = INT32_MAX;
  uint64_t active = 0;  // of the first 64
  for (int b0 = f; b0 < l; b0 += 64) {
    const int b = min(b0 + lane, l - 1);
    const SeqSpan sp = seq_span(a.s, b);
    const uint64_t some = __ballot(b0 + lane < l && sp.count > 0);
    least = min(least, some >> lane & 1 ? sp.len - sp.count + 1 : INT32_MAX);
    if (some && leader == INT32_MAX) leader = b0 + __builtin_ctzll(some);
    if (b0 == f) active = some;
  }
  least = wave_least(least);
  const int seen = leader == INT32_MAX ? 0 : (int)min((int64_t)max(least, 0), (int64_t)a.s.max_pages * a.c);
  const int slots = (seen + a.c - 1) / a.c;
  if (tid == 0) common = slots;
  __syncthreads();
  const int32_t* const first = a.s.table + (int64_t)min(leader, a.s.n_seqs - 1) * a.s.table_stride;
  for (int b0 = f + wave; b0 < l && slots > 0; b0 += kWavesOf * kShareSeqs) {
    // (a sequence that is not there or has no tokens: the first one again)
    const int32_t* mine[kShareSeqs];
#pragma unroll
    for (int i = 0; i < kShareSeqs; ++i) {
      const int b = b0 + i * kWavesOf;
      const bool there = b < l && (b - f < 64 ? active >> (b - f & 63) & 1 : seq_span(a.s, min(b, l - 1)).count > 0);
      mine[i] = there ? a.s.table + (int64_t)b * a.s.table_stride : first;
    }
    for (int s0 = 0; s0 < slots; s0 += 64 * kShareBatch) {
      int x[kShareBatch], y[kShareSeqs][kShareBatch];
#pragma unroll
      for (int k = 0; k < kShareBatch; ++k) {
        const int at = min(s0 + 64 * k + lane, slots - 1);
        x[k] = first[at];
#pragma unroll
        for (int i = 0; i < kShareSeqs; ++i) y[i][k] = mine[i][at];
      }
      int differ = INT32_MAX;
#pragma unroll
      for (int k = kShareBatch - 1; k >= 0; --k)
#pragma unroll
        for (int i = 0; i < kShareSeqs; ++i)
          if (x[k] != y[i][k]) differ = min(s0 + 64 * k + lane, slots - 1);
      if (!__any(differ != INT32_MAX)) continue;
      differ = wave_least(differ);
      if (lane == 0) atomicMin(&common, differ);
      break;
    }
  }
  __syncthreads();
  const int e = (int)min((int64_t)common * a.c, (int64_t)seen) / 32 * 32;
  if (tid == 0) {
    a.shared[g] = e;
    a.shared[a.n_groups + g] = leader == INT32_MAX ? f : leader;
  }
  for (int b = f + tid; b < l; b += kShareThreads) of_seq[b] = e;
}

// ---- tables -----------------------------------------------------------------------------

struct Tables {
  const int32_t* table;
  int32_t* table_out;
  const int32_t* lens;
  int32_t* lens_out;
  const int32_t* refs;
  int32_t* refs_out;
  int64_t table_stride, table_out_stride;
  int32_t n_pages, n_seqs, n_out, max_pages, c;
  __device__ __forceinline__ int length(int len) const {
    return (int)min((int64_t)max(len, 0), (int64_t)max_pages * c);
  }
  __device__ __forceinline__ int pages(int tokens) const { return (int)((uint32_t)(tokens + c - 1) / (uint32_t)c); }
  __device__ __forceinline__ bool names_page(int e) const { return e >= 0 && e < n_pages; }
};

constexpr int kThreads = 256;
constexpr int kPiece = 1024;      // table entries of a workgroup
constexpr int kRowPiece = 4096;   // bytes of a state's row

struct StateRows {
  const char* src;
  char* dst;
  int64_t row_bytes, src_stride, dst_stride;
  int32_t pieces, word;  // word: bytes of a load, 16, 4 or 1
};
struct ForkArgs {
  Tables t;
  const int32_t* parents;
  StateRows states[CKV_MAX_SEQ_ROWS];
  int n_states;
  int table_pieces;
  int64_t table_blocks, state_blocks;  // of the grid; the rest copies use counts
};

template <class W>
__device__ __forceinline__ void copy_piece(const char* src, char* dst, int64_t from, int64_t to) {
  for (int64_t o = from + threadIdx.x * sizeof(W); o < to; o += kThreads * sizeof(W))
    *reinterpret_cast<W*>(dst + o) = *reinterpret_cast<const W*>(src + o);
}

// Everything but the change of the use counts, which follows in a launch of its own: a page's
// holders lie anywhere in the tables, so its count is set first and added to then.
__global__ __launch_bounds__(kThreads) void fork_copy_kernel(ForkArgs a) {
  const Tables& t = a.t;
  int64_t w = blockIdx.x;
  if (w < a.table_blocks) {
    const int i = (int)(w / a.table_pieces), piece = (int)(w % a.table_pieces);
    const int p = a.parents[i];
    const bool there = p >= 0 && p < t.n_seqs;
    const int len = there ? t.length(t.lens[p]) : 0, held = t.pages(len);
    if (piece == 0 && threadIdx.x == 0) t.lens_out[i] = len;
    const int32_t* const from = t.table + (int64_t)(there ? p : 0) * t.table_stride;
    int32_t* const to = t.table_out + (int64_t)i * t.table_out_stride;
    int e[kPiece / kThreads];
#pragma unroll
    for (int k = 0; k < kPiece / kThreads; ++k) {
      const int at = piece * kPiece + k * kThreads + (int)threadIdx.x;
      e[k] = at < held ? from[at] : -1;
    }
#pragma unroll
    for (int k = 0; k < kPiece / kThreads; ++k) {
      const int at = piece * kPiece + k * kThreads + (int)threadIdx.x;
      if (at < t.max_pages) to[at] = e[k];
    }
    return;
  }
  w -= a.table_blocks;
  if (w < a.state_blocks) {
    int s = 0;
    while (w >= (int64_t)a.states[s].pieces * t.n_out) w -= (int64_t)a.states[s++].pieces * t.n_out;
    const StateRows& r = a.states[s];
    const int i = (int)(w / r.pieces);
    const int p = a.parents[i];
    if (p < 0 || p >= t.n_seqs) return;
    const int64_t from = w % r.pieces * kRowPiece, to = min(from + kRowPiece, r.row_bytes);
    const char* src = r.src + p * r.src_stride;
    char* dst = r.dst + i * r.dst_stride;
    if (r.word == 16)
      copy_piece<u32x4>(src, dst, from, to);
    else if (r.word == 4)
      copy_piece<uint32_t>(src, dst, from, to);
    else
      copy_piece<uint8_t>(src, dst, from, to);
    return;
  }
  w -= a.state_blocks;
#pragma unroll
  for (int k = 0; k < kPiece / kThreads; ++k) {
    const int64_t p = w * kPiece + k * kThreads + threadIdx.x;
    if (p < t.n_pages) t.refs_out[p] = t.refs[p];
  }
}

__global__ __launch_bounds__(kThreads) void fork_count_kernel(ForkArgs a) {
  const Tables& t = a.t;
  const int b = blockIdx.x / a.table_pieces, piece = blockIdx.x % a.table_pieces;
  const int32_t* const from = t.table + (int64_t)b * t.table_stride;
  const int len = t.lens[b];
  int e[kPiece / kThreads];  // (all loads together, past the held ones too)
#pragma unroll
  for (int k = 0; k < kPiece / kThreads; ++k)
    e[k] = from[min(piece * kPiece + k * kThreads + (int)threadIdx.x, t.max_pages - 1)];
  int children = 0;
#pragma unroll 4
  for (int i = threadIdx.x; i < t.n_out; i += kThreads) children += a.parents[i] == b;
  const int held = t.pages(t.length(len)), by = block_total<kThreads>(children) - 1;
  if (by == 0) return;
#pragma unroll
  for (int k = 0; k < kPiece / kThreads; ++k)
    if (piece * kPiece + k * kThreads + (int)threadIdx.x < held && t.names_page(e[k])) atomicAdd(&t.refs_out[e[k]], by);
}

// ---- extend -------------------------------------------------------------------------------

// The plan: list[r], the r-th free page; of each sequence its old length, the rank of its
// first page and tok_off; pages to copy.  The second launch writes what follows from it, so
// that nothing of the plan is read from arrays that the call may write in place.
constexpr int kPlanThreads = 1024, kPlanPer = 4, kPlanPages = kPlanThreads * kPlanPer;
constexpr int kSelfCounted = 16;  // blocks of pages up to which each counts all below it
struct ExtendArgs {
  Tables t;
  const int32_t* n_new;
  ckv_page_step o;
  int32_t* counts;   // [plan blocks]: free pages of each
  int32_t* list;     // [n_pages]
  int32_t* first;    // [n_seqs]
  int32_t* old_len;  // [n_seqs]
  int plan_blocks;
  int table_pieces;
  int64_t table_blocks;
};

// Use counts of four pages, this thread's p0 .. p0 + 3 or, where they would reach past the last
// page, the last four of all (n_pages is at least 4): no branch keeps one load waiting for another.
// `first` gets which of them are this thread's, from first on.
__device__ __forceinline__ void load_four(const Tables& t, int p0, int32_t (&refs)[kPlanPer], int& first) {
  const uint32_t at = (uint32_t)min(p0, t.n_pages - kPlanPer);  // (2^26 pages at most)
  first = min(p0 - (int)at, kPlanPer);
  __builtin_memcpy(refs, reinterpret_cast<const char*>(t.refs) + at * 4, sizeof refs);
}
// The same in their places; 1 past the last page.
__device__ __forceinline__ void load_refs(const Tables& t, int64_t p0, int32_t (&refs)[kPlanPer]) {
#pragma unroll
  for (int i = 0; i < kPlanPer; ++i) refs[i] = p0 + i < t.n_pages ? t.refs[p0 + i] : 1;
}
__device__ __forceinline__ int free_of(const int32_t (&refs)[kPlanPer]) {
  int n = 0;
#pragma unroll
  for (int i = 0; i < kPlanPer; ++i) n += refs[i] <= 0;
  return n;
}

__global__ __launch_bounds__(kPlanThreads) void extend_count_kernel(ExtendArgs a) {
  int32_t refs[kPlanPer];
  load_refs(a.t, (int64_t)blockIdx.x * kPlanPages + threadIdx.x * kPlanPer, refs);
  const int n = block_total<kPlanThreads>(free_of(refs));
  if (threadIdx.x == 0) a.counts[blockIdx.x] = n;
}

// This thread's share of the free pages of the first `blocks` blocks.  kCounted: their counts
// are there; else every workgroup goes over their use counts itself.
template <bool kCounted>
__device__ __forceinline__ int free_below(const ExtendArgs& a, int blocks) {
  const Tables& t = a.t;
  int n = 0;
  if constexpr (kCounted) {
    for (int i = threadIdx.x; i < blocks; i += kPlanThreads) n += a.counts[i];
  } else {
    constexpr int kAtOnce = 8;  // (32 registers of the 128 that 16 waves leave each)
#pragma unroll 1
    for (int i0 = 0; i0 < blocks; i0 += kAtOnce) {
      int32_t refs[kAtOnce][kPlanPer];
      int first[kAtOnce];
#pragma unroll
      for (int i = 0; i < kAtOnce; ++i)
        load_four(t, min(i0 + i, blocks - 1) * kPlanPages + (int)threadIdx.x * kPlanPer, refs[i], first[i]);
#pragma unroll
      for (int i = 0; i < kAtOnce; ++i)
#pragma unroll
        for (int k = 0; k < kPlanPer; ++k) n += i0 + i < blocks && k >= first[i] && refs[i][k] <= 0;
    }
  }
  return n;
}

template <bool kCounted>
__global__ __launch_bounds__(kPlanThreads) void extend_plan_kernel(ExtendArgs a) {
  const Tables& t = a.t;
  if ((int)blockIdx.x < a.plan_blocks) {
    const int64_t p0 = (int64_t)blockIdx.x * kPlanPages + threadIdx.x * kPlanPer;
    int32_t refs[kPlanPer];
    load_refs(t, p0, refs);
    int sums[2] = {free_below<kCounted>(a, blockIdx.x), free_of(refs)}, all[2];
    block_before<kPlanThreads>(sums, all);
    int rank = all[0] + sums[1];
#pragma unroll
    for (int i = 0; i < kPlanPer; ++i) {
      if (p0 + i >= t.n_pages) break;
      if (refs[i] <= 0) a.list[rank++] = (int32_t)(p0 + i);
      if (t.refs_out != t.refs) t.refs_out[p0 + i] = refs[i];
    }
    return;
  }
  // the sequences, in their order
  int64_t n_free = free_below<kCounted>(a, a.plan_blocks);  // (this thread's share; of all from the first sums on)
  int64_t needed = 0, asked = 0, taken = 0, tokens = 0;
  int refused = 0;  // of this thread's sequences
  if (threadIdx.x == 0) a.o.tok_off[0] = 0;
  for (int b0 = 0; b0 < t.n_seqs; b0 += kPlanThreads) {
    const int b = b0 + threadIdx.x;
    int64_t need = 0, add = 0;
    int len = 0, tail = -1;
    bool no = false;
    if (b < t.n_seqs) {
      const int said = t.lens[b], more = a.n_new[b];
      len = t.length(said);
      add = max(more, 0);
      const int held = t.pages(len);
      const int64_t upto = (int64_t)len + add;
      no = upto > (int64_t)t.max_pages * t.c;
      if (no) {
        add = 0;
      } else if (add > 0) {
        if (held * t.c != len) {
          tail = t.table[(int64_t)b * t.table_stride + held - 1];
          if (!t.names_page(tail) || t.refs[tail] <= 1) tail = -1;
        }
        need = t.pages((int)upto) - held + (tail >= 0);
      }
    }
    int64_t x[3] = {need, add, b0 == 0 ? n_free : 0}, total[3];
    block_before<kPlanThreads>(x, total);
    if (b0 == 0) n_free = total[2];
    const int64_t need_before = needed, add_before = asked;
    needed += total[0];
    asked += total[1];
    if (needed > n_free || asked > a.o.n_tokens) {  // some are refused
      if ((need > 0 && need_before + x[0] + need > n_free) || (add > 0 && add_before + x[1] + add > a.o.n_tokens)) {
        no = true;
        need = add = 0;
        tail = -1;
      }
      x[0] = need;
      x[1] = add;
      block_before<kPlanThreads>(x, total);
    }
    refused += no;
    if (b < t.n_seqs) {
      a.first[b] = (int32_t)(taken + x[0]);
      a.old_len[b] = len;
      a.o.tok_off[b + 1] = (int32_t)(tokens + x[1] + add);
      a.o.copy_src[b] = tail;
    }
    taken += total[0];
    tokens += total[1];
  }
  if (t.n_seqs == 0) n_free = block_total<kPlanThreads>((int)n_free);
  refused = block_total<kPlanThreads>(refused);
  if (threadIdx.x == 0) {
    a.o.counts[0] = (int32_t)tokens;
    a.o.counts[1] = (int32_t)taken;
    a.o.counts[2] = (int32_t)(n_free - taken);
    a.o.counts[3] = refused;
  }
}

__global__ __launch_bounds__(kThreads) void extend_write_kernel(ExtendArgs a) {
  const Tables& t = a.t;
  // entry `slot` of a sequence whose pages from `from` on are new
  const auto entry = [&](int b, int slot, int from, int first) {
    return slot >= from ? a.list[first + slot - from] : t.table[(int64_t)b * t.table_stride + slot];
  };
  if (blockIdx.x < a.table_blocks) {
    const int b = blockIdx.x / a.table_pieces, piece = blockIdx.x % a.table_pieces;
    const int len = a.old_len[b], add = a.o.tok_off[b + 1] - a.o.tok_off[b], first = a.first[b];
    const int src = a.o.copy_src[b];
    const int from = t.pages(len) - (src >= 0), upto = add > 0 ? t.pages(len + add) : from;
    int32_t* const to = t.table_out + (int64_t)b * t.table_out_stride;
    if (piece == 0 && threadIdx.x == 0) {
      t.lens_out[b] = len + add;
      a.o.copy_dst[b] = src >= 0 ? a.list[first] : -1;
      if (src >= 0) atomicSub(&t.refs_out[src], 1);
    }
    const bool in_place = t.table_out == t.table;
    const int lo = max(in_place ? from : 0, piece * kPiece);
    const int hi = min(in_place ? upto : t.max_pages, (piece + 1) * kPiece);
#pragma unroll 4
    for (int s = lo + (int)threadIdx.x; s < hi; s += kThreads) {
      const bool is_new = s >= from && s < upto;
      const int e = is_new ? a.list[first + s - from] : t.table[(int64_t)b * t.table_stride + s];
      to[s] = e;
      if (is_new) t.refs_out[e] = 1;
    }
    return;
  }
  // token rows: a lane finds its sequence among those of the workgroup's rows
  constexpr int kCached = 512;
  __shared__ int32_t off[kCached];
  const int64_t t0 = ((int64_t)blockIdx.x - a.table_blocks) * kThreads, row = t0 + threadIdx.x;
  const int total = t.n_seqs > 0 ? a.o.tok_off[t.n_seqs] : 0;
  const auto start = [&](int q) -> int64_t { return a.o.tok_off[q]; };
  int b = 0;
  if (t0 < total) {  // (uniform)
    const int64_t last = min(t0 + kThreads, (int64_t)total) - 1;
    const int lo = find_seq(t.n_seqs, t0, start), n = find_seq(t.n_seqs, last, start) - lo + 1;
    const bool cached = n <= kCached;
    if (cached)
      for (int i = threadIdx.x; i < n; i += kThreads) off[i] = a.o.tok_off[lo + i];
    __syncthreads();
    int below = 0, upto = n;  // the last of the n that begins at or before the row
    while (upto - below > 1) {
      const int mid = (below + upto) >> 1;
      const int32_t at = cached ? off[mid] : a.o.tok_off[lo + mid];
      if (at <= row)
        below = mid;
      else
        upto = mid;
    }
    b = lo + below;
  }
  if (row >= a.o.n_tokens) return;
  int64_t slot = -1;
  int pos = -1;
  if (row < total) {
    const int len = a.old_len[b];
    pos = len + (int)(row - a.o.tok_off[b]);
    const int e = entry(b, pos / t.c, t.pages(len) - (a.o.copy_src[b] >= 0), a.first[b]);
    slot = t.names_page(e) ? (int64_t)e * t.c + pos % t.c : -1;
  }
  if (a.o.slots) a.o.slots[row] = slot;
  if (a.o.positions) a.o.positions[row] = pos;
  if (a.o.seqs) a.o.seqs[row] = row < total ? b : -1;
}

struct ExtendLayout {
  size_t counts, list, first, old_len, bytes;
};
ExtendLayout extend_layout(int64_t n_pages, int64_t n_seqs) {
  ExtendLayout l{};
  size_t off = 0;
  auto take = [&](int64_t n) {
    const size_t at = off;
    off = align_up(off + (size_t)std::max<int64_t>(n, 1) * sizeof(int32_t), 256);
    return at;
  };
  l.counts = take(ceil_div(n_pages, kPlanPages));
  l.list = take(n_pages);
  l.first = take(n_seqs);
  l.old_len = take(n_seqs);
  l.bytes = off;
  return l;
}

ckv_status check_page_size(int c) {
  if (c < 1) CKV_FAIL(CKV_EINVAL, "page_size must be >= 1 (got %d)", c);
  if (!(c == 8 || c == 16 || c % 32 == 0))
    CKV_FAIL(CKV_EUNSUPPORTED, "page_size must be 8, 16 or a multiple of 32 (got %d)", c);
  return CKV_OK;
}

ckv_status check_tables(const ckv_page_tables* t, Tables& x) {
  if (!t) CKV_FAIL(CKV_EINVAL, "tables is NULL");
  if (ckv_status s = check_page_size(t->page_size); s != CKV_OK) return s;
  if (t->n_seqs < 0 || t->n_seqs > (1 << 20) || t->n_out < 0 || t->n_out > (1 << 20))
    CKV_FAIL(CKV_EINVAL, "n_seqs and n_out must be in [0, 2^20] (got %d, %d)", t->n_seqs, t->n_out);
  if (t->n_pages < 1 || t->n_pages > INT32_MAX)
    CKV_FAIL(CKV_EINVAL, "n_pages must be in [1, 2^31-1] (got %lld)", (long long)t->n_pages);
  if (t->n_pages > (int64_t(1) << 26)) CKV_FAIL(CKV_EUNSUPPORTED, "more than 2^26 pages");
  if (t->max_pages < 1) CKV_FAIL(CKV_EINVAL, "max_pages must be >= 1 (got %d)", t->max_pages);
  if ((int64_t)t->max_pages * t->page_size > (1 << 30))
    CKV_FAIL(CKV_EUNSUPPORTED, "tables of more than 2^30 tokens");
  if ((t->table_stride != 0 && t->table_stride < t->max_pages) ||
      (t->table_out_stride != 0 && t->table_out_stride < t->max_pages))
    CKV_FAIL(CKV_EINVAL, "a table's stride must be 0 or at least max_pages");
  if (!t->refs || !t->refs_out || (t->n_seqs > 0 && (!t->table || !t->lens)) ||
      (t->n_out > 0 && (!t->table_out || !t->lens_out)))
    CKV_FAIL(CKV_EINVAL, "NULL tables pointer");
  x = Tables{t->table, t->table_out, t->lens, t->lens_out, t->refs, t->refs_out,
             t->table_stride ? t->table_stride : t->max_pages,
             t->table_out_stride ? t->table_out_stride : t->max_pages, (int32_t)t->n_pages, t->n_seqs, t->n_out,
             t->max_pages, t->page_size};
  return CKV_OK;
}

constexpr int kInt = sizeof(int32_t);
MemRows table_rows(const int32_t* at, int64_t n, const Tables& t, int64_t stride) {
  return MemRows{at, n, (int64_t)t.max_pages * kInt, std::min(stride, INT64_MAX / kInt) * kInt};
}

}  // namespace
}  // namespace ckv

using namespace ckv;

#define CKV_REQUIRE(cond, ...)                      \
  do {                                              \
    if (!(cond)) CKV_FAIL(CKV_EINVAL, __VA_ARGS__); \
  } while (0)

#define CKV_CHECK(expr)            \
  do {                             \
    ckv_status s_ = (expr);        \
    if (s_ != CKV_OK) return s_;   \
  } while (0)

extern "C" {

int64_t ckv_page_share_ints(int32_t n_groups, int32_t n_seqs) {
  if (n_groups < 0 || n_groups > (1 << 20) || n_seqs < 0 || n_seqs > (1 << 20)) return 0;
  return 2 * (int64_t)n_groups + n_seqs;
}

ckv_status ckv_page_share(int32_t page_size, const ckv_page_batch* batch, const ckv_page_groups* groups,
                          void* stream) {
  clear_error();
  CKV_CHECK(check_page_size(page_size));
  CKV_CHECK(check_batch(batch, true));
  CKV_CHECK(check_groups(groups, batch, true));
  if (batch->n_seqs == 0 || batch->n_tokens == 0 || groups->n_groups == 0) return CKV_OK;
  if ((int64_t)batch->max_pages * page_size > (1 << 30))
    CKV_FAIL(CKV_EUNSUPPORTED, "tables of more than 2^30 tokens");
  const ShareArgs a{page_seqs(batch), groups->grp_off, groups->shared, groups->n_groups, page_size};
  hipLaunchKernelGGL(share_kernel, dim3((unsigned)groups->n_groups + 1), dim3(kShareThreads), 0,
                     (hipStream_t)stream, a);
  CKV_HIP(hipGetLastError());
  return CKV_OK;
}

ckv_status ckv_page_fork(const ckv_page_tables* tables, const int32_t* parents, const ckv_seq_rows* states,
                         int32_t n_states, void* stream) {
  clear_error();
  ForkArgs a{};
  CKV_CHECK(check_tables(tables, a.t));
  CKV_REQUIRE(n_states >= 0 && n_states <= CKV_MAX_SEQ_ROWS, "n_states must be in [0, %d] (got %d)",
              CKV_MAX_SEQ_ROWS, n_states);
  CKV_REQUIRE(n_states == 0 || states, "states is NULL");
  CKV_REQUIRE(a.t.n_out == 0 || parents, "parents is NULL");
  CKV_REQUIRE(a.t.n_out == 0 || a.t.n_seqs == 0 || (a.t.table_out != a.t.table && a.t.lens_out != a.t.lens),
              "tables and lengths must go to other buffers than they come from");
  a.parents = parents;
  a.n_states = n_states;
  a.table_pieces = (int)ceil_div(a.t.max_pages, kPiece);
  a.table_blocks = (int64_t)a.t.n_out * a.table_pieces;
  for (int i = 0; i < n_states; ++i) {
    const ckv_seq_rows& r = states[i];
    CKV_REQUIRE(r.row_bytes >= 1 && r.row_bytes <= (int64_t(1) << 40), "row_bytes must be in [1, 2^40]");
    CKV_REQUIRE((r.src_stride == 0 || r.src_stride >= r.row_bytes) && (r.dst_stride == 0 || r.dst_stride >= r.row_bytes),
                "a state's rows must not overlap");
    if (a.t.n_out == 0 || a.t.n_seqs == 0) continue;
    CKV_REQUIRE(r.src && r.dst, "NULL state pointer");
    CKV_REQUIRE(r.src != r.dst, "a state's rows must go to another buffer than they come from");
    StateRows& x = a.states[i];
    x.src = static_cast<const char*>(r.src);
    x.dst = static_cast<char*>(r.dst);
    x.row_bytes = r.row_bytes;
    x.src_stride = r.src_stride ? r.src_stride : r.row_bytes;
    x.dst_stride = r.dst_stride ? r.dst_stride : r.row_bytes;
    const uint64_t all = reinterpret_cast<uintptr_t>(r.src) | reinterpret_cast<uintptr_t>(r.dst) | (uint64_t)r.row_bytes |
                         (uint64_t)x.src_stride | (uint64_t)x.dst_stride;
    x.word = all % 16 == 0 ? 16 : all % 4 == 0 ? 4 : 1;
    x.pieces = (int32_t)ceil_div(r.row_bytes, kRowPiece);
    a.state_blocks += (int64_t)x.pieces * a.t.n_out;
  }
  // Workgroups read what others write, in no order: only the counts may be in place.
  MemRows reads[4 + CKV_MAX_SEQ_ROWS] = {table_rows(a.t.table, a.t.n_seqs, a.t, a.t.table_stride),
                                         mem_array(a.t.lens, (int64_t)a.t.n_seqs * kInt),
                                         mem_array(parents, (int64_t)a.t.n_out * kInt),
                                         mem_array(a.t.refs_out == a.t.refs ? nullptr : a.t.refs, a.t.n_pages * kInt)};
  MemRows writes[3 + CKV_MAX_SEQ_ROWS] = {table_rows(a.t.table_out, a.t.n_out, a.t, a.t.table_out_stride),
                                          mem_array(a.t.lens_out, (int64_t)a.t.n_out * kInt),
                                          mem_array(a.t.refs_out, a.t.n_pages * kInt)};
  for (int i = 0; i < n_states; ++i) {
    const StateRows& x = a.states[i];
    reads[4 + i] = MemRows{x.src, x.src ? a.t.n_seqs : 0, x.row_bytes, x.src_stride};
    writes[3 + i] = MemRows{x.dst, x.dst ? a.t.n_out : 0, x.row_bytes, x.dst_stride};
  }
  CKV_REQUIRE(!writes_overlap(writes, 3 + n_states, reads, 4 + n_states),
              "an array that is written overlaps another one (only refs_out may be refs)");
  const int64_t ref_blocks = a.t.refs_out != a.t.refs ? ceil_div(a.t.n_pages, kPiece) : 0;
  const int64_t grid = a.table_blocks + a.state_blocks + ref_blocks, counts = (int64_t)a.t.n_seqs * a.table_pieces;
  if (grid >= kMaxGrid || counts >= kMaxGrid) CKV_FAIL(CKV_EUNSUPPORTED, "batch too large");
  const hipStream_t st = (hipStream_t)stream;
  if (grid > 0) {
    hipLaunchKernelGGL(fork_copy_kernel, dim3((unsigned)grid), dim3(kThreads), 0, st, a);
    CKV_HIP(hipGetLastError());
  }
  if (counts > 0) {
    hipLaunchKernelGGL(fork_count_kernel, dim3((unsigned)counts), dim3(kThreads), 0, st, a);
    CKV_HIP(hipGetLastError());
  }
  return CKV_OK;
}

size_t ckv_page_extend_workspace_bytes(int64_t n_pages, int32_t n_seqs) {
  if (n_pages < 1 || n_pages > (int64_t(1) << 26) || n_seqs < 0 || n_seqs > (1 << 20)) return 0;
  return extend_layout(n_pages, n_seqs).bytes;
}

ckv_status ckv_page_extend(const ckv_page_tables* tables, const int32_t* n_new, const ckv_page_step* step,
                           void* ws, size_t ws_bytes, void* stream) {
  clear_error();
  ExtendArgs a{};
  CKV_CHECK(check_tables(tables, a.t));
  CKV_REQUIRE(step, "step is NULL");
  CKV_REQUIRE(a.t.n_out == a.t.n_seqs, "n_out must be n_seqs (%d, got %d)", a.t.n_seqs, a.t.n_out);
  CKV_REQUIRE(step->n_tokens >= 0 && step->n_tokens <= INT32_MAX, "n_tokens must be in [0, 2^31-1] (got %lld)",
              (long long)step->n_tokens);
  CKV_REQUIRE(step->tok_off && step->counts && ws, "NULL pointer argument");
  CKV_REQUIRE(a.t.n_seqs == 0 || (n_new && step->copy_src && step->copy_dst), "NULL pointer argument");
  CKV_REQUIRE(a.t.n_seqs == 0 || a.t.table_out != a.t.table || a.t.table_out_stride == a.t.table_stride,
              "a table written in place has one stride");
  const ExtendLayout l = extend_layout(a.t.n_pages, a.t.n_seqs);
  CKV_REQUIRE(ws_bytes >= l.bytes, "workspace too small: %zu < %zu", ws_bytes, l.bytes);
  CKV_REQUIRE(aligned16(ws), "pointers must be 16-byte aligned");
  {
    const int64_t n = (int64_t)a.t.n_seqs * kInt;
    const MemRows reads[4] = {
        table_rows(a.t.table, a.t.table_out == a.t.table ? 0 : a.t.n_seqs, a.t, a.t.table_stride),
        mem_array(a.t.lens_out == a.t.lens ? nullptr : a.t.lens, n),
        mem_array(a.t.refs_out == a.t.refs ? nullptr : a.t.refs, a.t.n_pages * kInt), mem_array(n_new, n)};
    const MemRows writes[11] = {table_rows(a.t.table_out, a.t.n_out, a.t, a.t.table_out_stride),
                                mem_array(a.t.lens_out, n),
                                mem_array(a.t.refs_out, a.t.n_pages * kInt),
                                mem_array(step->tok_off, n + kInt),
                                mem_array(step->copy_src, n),
                                mem_array(step->copy_dst, n),
                                mem_array(step->counts, 4 * kInt),
                                mem_array(step->slots, step->n_tokens * (int64_t)sizeof(int64_t)),
                                mem_array(step->positions, step->n_tokens * kInt),
                                mem_array(step->seqs, step->n_tokens * kInt),
                                mem_array(ws, (int64_t)l.bytes)};
    CKV_REQUIRE(!writes_overlap(writes, 11, reads, 4),
                "an array that is written overlaps another one (only the table, lengths and counts may be in place)");
  }
  auto at = [&](size_t off) { return reinterpret_cast<int32_t*>(static_cast<char*>(ws) + off); };
  a.n_new = n_new;
  a.o = *step;
  a.counts = at(l.counts);
  a.list = at(l.list);
  a.first = at(l.first);
  a.old_len = at(l.old_len);
  a.plan_blocks = (int)ceil_div(a.t.n_pages, kPlanPages);
  a.table_pieces = (int)ceil_div(a.t.max_pages, kPiece);
  a.table_blocks = (int64_t)a.t.n_seqs * a.table_pieces;
  const bool rows = step->slots || step->positions || step->seqs;
  const int64_t grid = a.table_blocks + (rows ? ceil_div(step->n_tokens, kThreads) : 0);
  if (grid >= kMaxGrid) CKV_FAIL(CKV_EUNSUPPORTED, "batch too large");
  const hipStream_t st = (hipStream_t)stream;
  if (a.plan_blocks <= kSelfCounted && a.t.n_pages >= kPlanPer) {
    hipLaunchKernelGGL(extend_plan_kernel<false>, dim3(a.plan_blocks + 1), dim3(kPlanThreads), 0, st, a);
  } else {
    hipLaunchKernelGGL(extend_count_kernel, dim3(a.plan_blocks), dim3(kPlanThreads), 0, st, a);
    CKV_HIP(hipGetLastError());
    hipLaunchKernelGGL(extend_plan_kernel<true>, dim3(a.plan_blocks + 1), dim3(kPlanThreads), 0, st, a);
  }
  CKV_HIP(hipGetLastError());
  if (grid > 0) {
    hipLaunchKernelGGL(extend_write_kernel, dim3((unsigned)grid), dim3(kThreads), 0, st, a);
    CKV_HIP(hipGetLastError());
  }
  return CKV_OK;
}

}  // extern "C"
