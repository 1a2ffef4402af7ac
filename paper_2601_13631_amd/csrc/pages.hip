// pages.hip -- the paged cache's writer and movers for gfx950: append, copy, compact.
//
// All three move bytes, each 16-byte piece read once and written once: memory bounds the
// large calls, launch and latency the small ones.  Measured: the rows of four prompts (15,300
// tokens of 4 heads of 128, bf16 to 8 bits, 47 MB) 12.5 us, of one step of 64 sequences 5.2; the
// same prompts into a bf16 pool (63 MB) 14.7, the step 5.2; eight pages copied in 28 layers
// (15 MB) 6 us; 850 of 4,000 pages of 8 KB moved in 28 layers (780 MB read + written) 173 us,
// 4.5 TB/s (a copy of 4 GiB: 4.8).

#include "pages_internal.h"

namespace ckv {

namespace {
using Wide = __int128;  // (rows times strides pass 64 bits)
Wide floor_div(Wide a, Wide b) { return a / b - (a % b < 0 ? 1 : 0); }  // b > 0
Wide begin_of(const MemRows& x) { return (Wide) reinterpret_cast<uintptr_t>(x.at); }
// Whether bytes [lo, hi) meet a row of x.
bool meets(Wide lo, Wide hi, const MemRows& x) {
  // rows j with j stride + bytes > lo and j stride < hi, from x's begin
  const Wide from = std::max<Wide>(floor_div(lo - begin_of(x) - x.bytes, x.stride) + 1, 0);
  const Wide upto = std::min<Wide>(floor_div(hi - 1 - begin_of(x), x.stride), x.n - 1);
  return from <= upto;
}
// Whether arrays whose bytes from the first to the last meet share one.
bool rows_overlap(const MemRows& a, const MemRows& b) {
  const MemRows &few = a.n <= b.n ? a : b, &many = a.n <= b.n ? b : a;
  if (few.n > 1 && few.stride == many.stride) {
    // Row i of `few` begins `off` bytes into a step of `many`, alike for all i.
    const Wide d = begin_of(few) - begin_of(many), off = d - floor_div(d, few.stride) * few.stride;
    if (off >= many.bytes && off + few.bytes <= few.stride) return false;
  }
  for (int64_t i = 0; i < few.n; ++i) {
    const Wide lo = begin_of(few) + (Wide)i * few.stride;
    if (meets(lo, lo + few.bytes, many)) return true;
  }
  return false;
}
// The address behind the last byte; the first one's of an empty array.
uint64_t end_of(const MemRows& x) {
  const uint64_t at = reinterpret_cast<uintptr_t>(x.at);
  if (x.n <= 0 || x.bytes <= 0) return at;
  const Wide end = (Wide)at + (Wide)(x.n - 1) * x.stride + x.bytes;
  return end < (Wide)UINT64_MAX ? (uint64_t)end : UINT64_MAX;
}
}  // namespace

bool writes_overlap(const MemRows* writes, int n_writes, const MemRows* reads, int n_reads) {
  // (mostly no two come near each other: an allocation each)
  uint64_t read_end[kMostArrays], write_end[kMostArrays];
  for (int k = 0; k < n_reads; ++k) read_end[k] = end_of(reads[k]);
  for (int k = 0; k < n_writes; ++k) write_end[k] = end_of(writes[k]);
  const auto meet = [](const MemRows& a, uint64_t a1, const MemRows& b, uint64_t b1) {
    const uint64_t a0 = reinterpret_cast<uintptr_t>(a.at), b0 = reinterpret_cast<uintptr_t>(b.at);
    return a0 < b1 && b0 < a1 && a0 < a1 && b0 < b1 && rows_overlap(a, b);
  };
  for (int i = 0; i < n_writes; ++i) {
    for (int k = 0; k < n_reads; ++k)
      if (meet(writes[i], write_end[i], reads[k], read_end[k])) return true;
    for (int k = i + 1; k < n_writes; ++k)
      if (meet(writes[i], write_end[i], writes[k], write_end[k])) return true;
  }
  return false;
}

ckv_status check_pool(const ckv_page_pool* p, bool with_pointers) {
  if (!p) CKV_FAIL(CKV_EINVAL, "pool is NULL");
  if (p->dtype != CKV_DTYPE_F32 && p->dtype != CKV_DTYPE_BF16 && p->dtype != CKV_DTYPE_E4M3)
    CKV_FAIL(CKV_EINVAL, "unknown page dtype %d", p->dtype);
  if (p->n_pages < 1 || p->n_pages > INT32_MAX)
    CKV_FAIL(CKV_EINVAL, "n_pages must be in [1, 2^31-1] (got %lld)", (long long)p->n_pages);
  if (p->n_kv_heads < 1) CKV_FAIL(CKV_EINVAL, "n_kv_heads must be >= 1 (got %d)", p->n_kv_heads);
  if (p->page_size < 1) CKV_FAIL(CKV_EINVAL, "page_size must be >= 1 (got %d)", p->page_size);
  if (p->head_dim < 1) CKV_FAIL(CKV_EINVAL, "head_dim must be >= 1");
  if (p->head_dim != 64 && !(p->head_dim == 128 && p->dtype != CKV_DTYPE_F32))
    CKV_FAIL(CKV_EUNSUPPORTED, "pages support head_dim 64, and 128 but for fp32 (got %d)", p->head_dim);
  const int c = p->page_size;
  if (!(c == 8 || c == 16 || c % 32 == 0))
    CKV_FAIL(CKV_EUNSUPPORTED, "page_size must be 8, 16 or a multiple of 32 (got %d)", c);
  if (p->n_kv_heads > 65535 ||
      (int64_t)c * p->n_kv_heads > ((int64_t(1) << 30) / (p->head_dim * page_elem_bytes(p->dtype))))
    CKV_FAIL(CKV_EUNSUPPORTED, "page too large");
  const int64_t dense = (int64_t)c * p->n_kv_heads * p->head_dim;
  if (p->page_stride != 0 && (p->page_stride < dense || p->page_stride > (int64_t(1) << 40) ||
                              p->page_stride * page_elem_bytes(p->dtype) % 16))
    CKV_FAIL(CKV_EINVAL, "page_stride must be 0, or at least %lld and a whole number of 16 bytes (got %lld)",
             (long long)dense, (long long)p->page_stride);
  if (!with_pointers) return CKV_OK;
  if (!p->k || !p->v) CKV_FAIL(CKV_EINVAL, "NULL pool pointer");
  if (!aligned16(p->k) || !aligned16(p->v)) CKV_FAIL(CKV_EINVAL, "pointers must be 16-byte aligned");
  if (p->dtype == CKV_DTYPE_E4M3 && (!p->k_scale || !p->v_scale))
    CKV_FAIL(CKV_EINVAL, "an E4M3 pool needs k_scale and v_scale");
  if (p->dtype != CKV_DTYPE_E4M3 && (p->k_scale || p->v_scale))
    CKV_FAIL(CKV_EINVAL, "scales belong to E4M3 pools only");
  return CKV_OK;
}

ckv_status check_batch(const ckv_page_batch* b, bool with_pointers) {
  if (!b) CKV_FAIL(CKV_EINVAL, "batch is NULL");
  if (b->n_seqs < 0 || b->n_seqs > (1 << 20))
    CKV_FAIL(CKV_EINVAL, "n_seqs must be in [0, 2^20] (got %d)", b->n_seqs);
  if (b->n_tokens < 0 || b->n_tokens > INT32_MAX)
    CKV_FAIL(CKV_EINVAL, "n_tokens must be in [0, 2^31-1] (got %lld)", (long long)b->n_tokens);
  if (b->max_pages < 1) CKV_FAIL(CKV_EINVAL, "max_pages must be >= 1 (got %d)", b->max_pages);
  if (b->table_stride != 0 && b->table_stride < b->max_pages)
    CKV_FAIL(CKV_EINVAL, "table_stride must be 0 or at least max_pages");
  if (b->max_tokens < 0 || b->max_len < 0) CKV_FAIL(CKV_EINVAL, "max_tokens and max_len must be >= 0");
  if (with_pointers && b->n_seqs > 0 && b->n_tokens > 0 && (!b->table || !b->lens || !b->tok_off))
    CKV_FAIL(CKV_EINVAL, "NULL batch pointer");
  return CKV_OK;
}

namespace {

constexpr int kThreads = 256;

// ---- append ---------------------------------------------------------------------

// Rows of a pool that takes them as they are: a thread per 16 bytes of a token's K
// (grid z 0) or V row.
struct AppendArgs {
  PageSeqs s;
  const char* k_new;
  const char* v_new;
  char* k;
  char* v;
  uint8_t* k_scale;
  uint8_t* v_scale;
  int64_t page_stride;  // bytes
  int64_t n_pages;
  int c, Hkv, row_bytes;  // of a pool row (all heads)
  int by_token;           // numbering of the pages written to, see append_start
};

// Pages that the call writes to, as find_seq numbers them: n tokens of a sequence lie in at
// most min(n, n / c + 2) pages, so either from its first token's number on, or from that
// number / c + 2 per sequence before; the host takes the one with the lower end.
__device__ __forceinline__ int64_t append_start(const AppendArgs& a, int b) {
  const int64_t t = token_of(a.s, b);
  return a.by_token ? t : t / a.c + 2 * (int64_t)b;
}

// The sequence whose rows hold token t: the last b with tok_off[b] <= t (those
// before it that are empty share its offset); -1 if it is in none.
__device__ __forceinline__ int seq_of_token(const PageSeqs& s, int64_t t) {
  int lo = 0, hi = s.n_seqs;  // first b with tok_off[b + 1] > t
  while (lo < hi) {
    const int mid = (lo + hi) >> 1;
    if (s.tok_off[mid + 1] > t)
      hi = mid;
    else
      lo = mid + 1;
  }
  return lo < s.n_seqs && s.tok_off[lo] <= t ? lo : -1;
}

__global__ __launch_bounds__(kThreads) void append_kernel(AppendArgs a) {
  const int per_row = a.row_bytes / 16;
  const int64_t i = (int64_t)blockIdx.x * kThreads + threadIdx.x;
  const int64_t t = i / per_row;
  if (t >= a.s.n_tokens) return;
  const int piece = (int)(i % per_row);
  const char* src = blockIdx.z ? a.v_new : a.k_new;
  const u32x4 x = *reinterpret_cast<const u32x4*>(src + t * a.row_bytes + piece * 16);
  const int b = seq_of_token(a.s, t);
  if (b < 0) return;
  const SeqSpan sp = seq_span(a.s, b);
  const int64_t pos = (int64_t)sp.len - sp.count + (t - sp.first);
  if (t < sp.first || t >= sp.first + sp.count || pos < 0 || pos / a.c >= a.s.max_pages) return;
  const int page = a.s.table[(int64_t)b * a.s.table_stride + pos / a.c];
  if (page < 0 || page >= a.n_pages) return;
  char* dst = (blockIdx.z ? a.v : a.k) + (int64_t)page * a.page_stride + pos % a.c * a.row_bytes;
  *reinterpret_cast<u32x4*>(dst + piece * 16) = x;
}

// The byte of the least power of two s with amax <= 448 s (448 = 1.75 * 2^8).
__device__ __forceinline__ uint32_t scale_byte(float amax) {
  const uint32_t b = __float_as_uint(amax);
  const int e = (int)(b >> 23) - 8 + ((b & 0x7fffffu) > 0x600000u ? 1 : 0);
  return (uint32_t)max(e, 10);
}

// Two e4m3 codes of x and y (each |x| <= 448, an infinity, or NaN).
__device__ __forceinline__ uint32_t codes2(float x, float y) {
  // min and max of a NaN and a number are the number: a NaN goes past them
  const float cx = x != x ? x : fminf(fmaxf(x, -448.f), 448.f);
  const float cy = y != y ? y : fminf(fmaxf(y, -448.f), 448.f);
  return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(cx, cy, 0, false) & 0xffffu;
}

// 8-bit rows.  A wave owns one (page that the call writes to, KV head) of K (grid
// z 0) or V: it takes the largest finite magnitude of the page's new rows, sets the
// scale, rounds the page's older rows again if that rose, and writes the new rows.
// Lanes hold 8 elements each, D / 8 lanes per row.
//
template <int D>
__global__ __launch_bounds__(64) void append_e4m3_kernel(AppendArgs a) {
  constexpr int kLanes = D / 8, kRows = 64 / kLanes;
  const int lane = threadIdx.x, g = blockIdx.y;
  const int b = find_seq(a.s.n_seqs, blockIdx.x, [&](int q) { return append_start(a, q); });
  if (b < 0) return;
  const SeqSpan sp = seq_span(a.s, b);
  const int64_t start = (int64_t)sp.len - sp.count;  // position of the call's first token
  const int64_t slot = max<int64_t>(start, 0) / a.c + ((int64_t)blockIdx.x - append_start(a, b));
  if (sp.count == 0 || slot * a.c >= sp.len || slot >= a.s.max_pages) return;
  const int page = a.s.table[(int64_t)b * a.s.table_stride + slot];
  if (page < 0 || page >= a.n_pages) return;

  const char* src = blockIdx.z ? a.v_new : a.k_new;  // bf16
  char* dst = (blockIdx.z ? a.v : a.k) + (int64_t)page * a.page_stride + g * D;
  uint8_t* scale = (blockIdx.z ? a.v_scale : a.k_scale) + (int64_t)page * a.Hkv + g;
  const int64_t base = slot * a.c;
  const int r0 = (int)(max(start, base) - base), r1 = (int)(min<int64_t>(sp.len, base + a.c) - base);
  const int col = lane % kLanes * 8, sub = lane / kLanes;
  auto new_row = [&](int r) {  // 8 elements of the page's row r
    const int64_t t = sp.first + (base + r - start);
    return *reinterpret_cast<const bf16x8*>(src + ((t * a.Hkv + g) * D + col) * 2);
  };

  // the first kBatch rows per lane stay in registers, all in flight together
  constexpr int kBatch = 8;
  bf16x8 x[kBatch];
#pragma unroll
  for (int i = 0; i < kBatch; ++i) x[i] = new_row(min(r0 + sub + i * kRows, r1 - 1));
  float amax = 0.f;
  auto look = [&](const bf16x8& y) {
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const float z = fabsf((float)y[e]);
      if (z < INFINITY) amax = fmaxf(amax, z);
    }
  };
#pragma unroll
  for (int i = 0; i < kBatch; ++i) look(x[i]);  // (a row past the end is the last one again)
  for (int r = r0 + sub + kBatch * kRows; r < r1; r += kRows) look(new_row(r));
#pragma unroll
  for (int x = 1; x < 64; x <<= 1) amax = fmaxf(amax, __shfl_xor(amax, x));
  uint32_t to = scale_byte(amax);
  if (r0 > 0) {
    const uint32_t from = *scale;
    to = max(to, from);
    if (to > from) {
      // (2^-127 and less leaves no code)
      const float f = scale_of((uint32_t)max(127 + (int)from - (int)to, 0));
      for (int r = sub; r < r0; r += kRows) {
        uint2* at = reinterpret_cast<uint2*>(dst + (int64_t)r * a.row_bytes + col);
        const uint2 w = *at;
        uint32_t z[2] = {w.x, w.y};
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          const auto lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)z[i], false);
          const auto hi = __builtin_amdgcn_cvt_pk_f32_fp8((int)z[i], true);
          z[i] = codes2(lo[0] * f, lo[1] * f) | codes2(hi[0] * f, hi[1] * f) << 16;
        }
        *at = make_uint2(z[0], z[1]);
      }
    }
  }
  // 1 / scale is a power of two of its own (a byte of 10 to 247 gives 2^117 to 2^-120)
  const float inv = scale_of(254 - to);
  auto write = [&](int r, const bf16x8& y) {
    uint32_t z[2];
#pragma unroll
    for (int i = 0; i < 2; ++i)
      z[i] = codes2((float)y[4 * i] * inv, (float)y[4 * i + 1] * inv) |
             codes2((float)y[4 * i + 2] * inv, (float)y[4 * i + 3] * inv) << 16;
    *reinterpret_cast<uint2*>(dst + (int64_t)r * a.row_bytes + col) = make_uint2(z[0], z[1]);
  };
#pragma unroll
  for (int i = 0; i < kBatch; ++i)
    if (const int r = r0 + sub + i * kRows; r < r1) write(r, x[i]);
  for (int r = r0 + sub + kBatch * kRows; r < r1; r += kRows) write(r, new_row(r));
  // every lane has read the old scale: the wave runs in step
  if (lane == 0) *scale = (uint8_t)to;
}

// ---- copy and compact ---------------------------------------------------------------

// The pools of one launch, by value in the kernel's arguments.
constexpr int kMaxPools = 64;
struct PoolTable {
  char* k[kMaxPools];
  char* v[kMaxPools];
  uint8_t* k_scale[kMaxPools];
  uint8_t* v_scale[kMaxPools];
  int n;
};

struct MoveArgs {
  int64_t n_pages, page_stride, page_bytes;
  int Hkv;
  int pieces;  // of piece_bytes(kUnroll) per page
};
constexpr int64_t piece_bytes(int unroll) { return (int64_t)kThreads * unroll * 16; }
// 16-byte loads per thread and piece: 1, 2 or 4, the most that a page has for all threads.
inline int unroll_of(int64_t page_bytes) {
  return page_bytes >= piece_bytes(4) ? 4 : page_bytes >= piece_bytes(2) ? 2 : 1;
}

// Piece w of a page moved from src to dst: w counts pieces, then K and V, then pools.
template <int kUnroll>
__device__ __forceinline__ void move_piece(const PoolTable& t, const MoveArgs& a, int64_t src,
                                           int64_t dst, int w) {
  const int piece = w % a.pieces, kv = w / a.pieces & 1, pool = w / a.pieces / 2;
  char* base = kv ? t.v[pool] : t.k[pool];
  const char* s = base + src * a.page_stride;
  char* d = base + dst * a.page_stride;
  const int64_t at = piece * piece_bytes(kUnroll) + (int64_t)threadIdx.x * 16;
  u32x4 x[kUnroll];
  // unconditional loads at offsets clamped into the page, so that all are in flight
#pragma unroll
  for (int p = 0; p < kUnroll; ++p)
    x[p] = *reinterpret_cast<const u32x4*>(s + min(at + (int64_t)p * kThreads * 16, a.page_bytes - 16));
#pragma unroll
  for (int p = 0; p < kUnroll; ++p) {
    const int64_t o = at + (int64_t)p * kThreads * 16;
    if (o < a.page_bytes) *reinterpret_cast<u32x4*>(d + o) = x[p];
  }
  uint8_t* scale = kv ? t.v_scale[pool] : t.k_scale[pool];
  if (scale && piece == 0)
    for (int g = threadIdx.x; g < a.Hkv; g += kThreads) scale[dst * a.Hkv + g] = scale[src * a.Hkv + g];
}

template <int kUnroll>
__global__ __launch_bounds__(kThreads) void copy_pages_kernel(PoolTable t, MoveArgs a,
                                                              const int32_t* __restrict__ src,
                                                              const int32_t* __restrict__ dst,
                                                              int64_t count) {
  const int per_pair = a.pieces * 2 * t.n;
  const int64_t total = count * per_pair;
  for (int64_t w = blockIdx.x; w < total; w += gridDim.x) {
    const int64_t i = w / per_pair;
    const int64_t s = src[i], d = dst[i];
    if (s < 0 || d < 0 || s >= a.n_pages || d >= a.n_pages) continue;
    move_piece<kUnroll>(t, a, s, d, (int)(w % per_pair));
  }
}

// Compaction's plan.  live(p): refs[p] > 0; before(p): pages in use below p; L: all of
// them.  A free page p < L is hole p - before(p); a page in use p >= L is mover
// before(p) - before(L).  Workspace: rank[p] = before(p) of a page in use, ~(p -
// before(p)) of a free one; hole[i]; mover[before(p)] and its use count; {L,
// before(L)}; the pages in use of each block of kPlan pages.
constexpr int kPlanThreads = 256, kPlanPer = 8, kPlan = kPlanThreads * kPlanPer;
struct PlanArgs {
  const int32_t* refs;
  int64_t n_pages;
  int32_t* counts;  // [blocks]
  int32_t* rank;    // [n_pages]
  int32_t* hole;
  int32_t* mover;
  int32_t* mover_refs;
  int32_t* head;    // {L, before(L)}
  int32_t* n_live;
};

__device__ __forceinline__ int block_sum(int x) {
  __shared__ int part[kPlanThreads / 64];
#pragma unroll
  for (int i = 1; i < 64; i <<= 1) x += __shfl_xor(x, i);
  if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = x;
  __syncthreads();
  x = 0;
#pragma unroll
  for (int i = 0; i < kPlanThreads / 64; ++i) x += part[i];
  __syncthreads();
  return x;
}

__global__ __launch_bounds__(kPlanThreads) void compact_count_kernel(PlanArgs a) {
  int n = 0;
#pragma unroll
  for (int i = 0; i < kPlanPer; ++i) {
    const int64_t p = (int64_t)blockIdx.x * kPlan + i * kPlanThreads + threadIdx.x;
    n += p < a.n_pages && a.refs[p] > 0;
  }
  n = block_sum(n);
  if (threadIdx.x == 0) a.counts[blockIdx.x] = n;
}

// kCount: no counts yet, every workgroup goes over all use counts itself.
template <bool kCount>
__global__ __launch_bounds__(kPlanThreads) void compact_rank_kernel(PlanArgs a) {
  __shared__ int waves[kPlanThreads / 64];
  int below = 0, all = 0;
  if constexpr (kCount) {
    for (int64_t p0 = threadIdx.x; p0 < a.n_pages; p0 += kPlan) {
      int32_t refs[kPlanPer];
#pragma unroll
      for (int i = 0; i < kPlanPer; ++i) refs[i] = a.refs[min<int64_t>(p0 + i * kPlanThreads, a.n_pages - 1)];
      int n = 0;
#pragma unroll
      for (int i = 0; i < kPlanPer; ++i) n += p0 + i * kPlanThreads < a.n_pages && refs[i] > 0;
      all += n;
      if (p0 < (int64_t)blockIdx.x * kPlan) below += n;
    }
  } else {
    for (int i = threadIdx.x; i < (int)gridDim.x; i += kPlanThreads) {
      const int n = a.counts[i];
      all += n;
      if (i < (int)blockIdx.x) below += n;
    }
  }
  below = block_sum(below);
  const int64_t L = block_sum(all);
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
#pragma unroll 1
  for (int i = 0; i < kPlanPer; ++i) {
    const int64_t p = (int64_t)blockIdx.x * kPlan + i * kPlanThreads + threadIdx.x;
    const int refs = p < a.n_pages ? a.refs[p] : 0;
    const bool live = refs > 0;
    const uint64_t mask = __ballot(live);
    if (lane == 0) waves[wave] = __builtin_popcountll(mask);
    __syncthreads();
    int before = below + __builtin_popcountll(mask & ((1ull << lane) - 1)), row = 0;
    for (int w = 0; w < kPlanThreads / 64; ++w) {
      if (w < wave) before += waves[w];
      row += waves[w];
    }
    below += row;
    __syncthreads();
    if (p >= a.n_pages) continue;
    a.rank[p] = live ? before : (int32_t)~(p - before);
    if (live && p >= L) {
      a.mover[before] = (int32_t)p;
      a.mover_refs[before] = refs;
    }
    if (!live && p < L) a.hole[p - before] = (int32_t)p;
    // before(L): of page L, or all of them where every page is in use
    if (p == L || (L == a.n_pages && p == L - 1)) {
      a.head[0] = (int32_t)L;
      a.head[1] = p == L ? before : (int32_t)L;
      *a.n_live = (int32_t)L;
    }
  }
}

struct FollowArgs {
  const int32_t* refs;
  int32_t* refs_out;
  const int32_t* table;
  int32_t* table_out;
  int64_t n_entries;
  int64_t follow_blocks;  // the grid's first blocks write counts and tables, the others move
};

template <int kUnroll>
__global__ __launch_bounds__(kThreads) void compact_move_kernel(PoolTable t, MoveArgs a, PlanArgs pl,
                                                                FollowArgs f) {
  const int64_t L = pl.head[0], base = pl.head[1];
  if (blockIdx.x < f.follow_blocks) {
    const int64_t step = f.follow_blocks * kThreads;
    for (int64_t p = (int64_t)blockIdx.x * kThreads + threadIdx.x; p < pl.n_pages; p += step) {
      const int r = pl.rank[p];
      f.refs_out[p] = p >= L ? 0 : r >= 0 ? f.refs[p] : pl.mover_refs[base + ~r];
    }
    for (int64_t i = (int64_t)blockIdx.x * kThreads + threadIdx.x; i < f.n_entries; i += step) {
      int32_t e = f.table[i];
      if (e >= 0 && e < pl.n_pages) {
        const int r = pl.rank[e];
        e = r < 0 ? -1 : e < L ? e : pl.hole[r - base];
      }
      f.table_out[i] = e;
    }
    return;
  }
  const int per_pair = a.pieces * 2 * t.n;
  const int64_t total = (L - base) * per_pair;
  for (int64_t w = blockIdx.x - f.follow_blocks; w < total; w += gridDim.x - f.follow_blocks) {
    const int64_t i = w / per_pair;
    move_piece<kUnroll>(t, a, pl.mover[base + i], pl.hole[i], (int)(w % per_pair));
  }
}

// The pools' shapes agree; MoveArgs from the first.
ckv_status check_pools(const ckv_page_pool* pools, int32_t n_pools, MoveArgs& a) {
  if (n_pools < 0) CKV_FAIL(CKV_EINVAL, "n_pools must be >= 0 (got %d)", n_pools);
  if (n_pools > 0 && !pools) CKV_FAIL(CKV_EINVAL, "pools is NULL");
  a = MoveArgs{};
  for (int i = 0; i < n_pools; ++i) {
    const ckv_page_pool &p = pools[i], &q = pools[0];
    if (ckv_status s = check_pool(&p, true); s != CKV_OK) return s;
    if (p.n_pages != q.n_pages || page_stride_bytes(&p) != page_stride_bytes(&q) ||
        p.page_size != q.page_size || p.n_kv_heads != q.n_kv_heads || p.head_dim != q.head_dim ||
        p.dtype != q.dtype)
      CKV_FAIL(CKV_EINVAL, "pool %d differs in shape from pool 0", i);
  }
  if (n_pools == 0) return CKV_OK;
  a.n_pages = pools[0].n_pages;
  a.page_stride = page_stride_bytes(&pools[0]);
  a.page_bytes = page_bytes_of(&pools[0]);
  a.Hkv = pools[0].n_kv_heads;
  a.pieces = (int)ceil_div(a.page_bytes, piece_bytes(unroll_of(a.page_bytes)));
  return CKV_OK;
}

void fill_table(PoolTable& t, const ckv_page_pool* pools, int n) {
  t.n = n;
  for (int i = 0; i < n; ++i) {
    t.k[i] = static_cast<char*>(pools[i].k);
    t.v[i] = static_cast<char*>(pools[i].v);
    t.k_scale[i] = pools[i].k_scale;
    t.v_scale[i] = pools[i].v_scale;
  }
}

// Workgroups that a mover takes at most: four rounds of every CU's 8, so that the last
// ones spread (one round: 181 us where this took 176, half a round: 191).
constexpr int64_t kMoveBlocks = 8192;

struct PlanLayout {
  size_t counts, rank, hole, mover, mover_refs, head, bytes;
};
PlanLayout plan_layout(int64_t n_pages) {
  PlanLayout l{};
  size_t off = 0;
  auto take = [&](int64_t n) {
    const size_t at = off;
    off = align_up(off + (size_t)n * sizeof(int32_t), 256);
    return at;
  };
  l.counts = take(ceil_div(n_pages, kPlan));
  l.rank = take(n_pages);
  l.hole = take(n_pages);
  l.mover = take(n_pages);
  l.mover_refs = take(n_pages);
  l.head = take(2);
  l.bytes = off;
  return l;
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

ckv_status ckv_page_append(const ckv_page_pool* pool, const ckv_page_batch* batch,
                           const void* k_new, const void* v_new, void* stream) {
  clear_error();
  CKV_CHECK(check_pool(pool, true));
  CKV_CHECK(check_batch(batch, true));
  if (batch->n_seqs == 0 || batch->n_tokens == 0) return CKV_OK;
  CKV_REQUIRE(k_new && v_new, "NULL pointer argument");
  CKV_REQUIRE(aligned16(k_new) && aligned16(v_new), "pointers must be 16-byte aligned");
  AppendArgs a;
  a.s = page_seqs(batch);
  a.k_new = static_cast<const char*>(k_new);
  a.v_new = static_cast<const char*>(v_new);
  a.k = static_cast<char*>(pool->k);
  a.v = static_cast<char*>(pool->v);
  a.k_scale = pool->k_scale;
  a.v_scale = pool->v_scale;
  a.page_stride = page_stride_bytes(pool);
  a.n_pages = pool->n_pages;
  a.c = pool->page_size;
  a.Hkv = pool->n_kv_heads;
  a.row_bytes = pool->n_kv_heads * pool->head_dim * page_elem_bytes(pool->dtype);
  const hipStream_t st = (hipStream_t)stream;
  if (pool->dtype == CKV_DTYPE_E4M3) {
    const int64_t by_page = batch->n_tokens / a.c + 2 * (int64_t)batch->n_seqs;
    a.by_token = batch->n_tokens <= by_page ? 1 : 0;
    const int64_t waves = std::min(batch->n_tokens, by_page);
    if (waves >= kMaxGrid) CKV_FAIL(CKV_EUNSUPPORTED, "too many rows in one call");
    const dim3 grid((unsigned)waves, (unsigned)a.Hkv, 2);
    if (pool->head_dim == 128)
      hipLaunchKernelGGL(append_e4m3_kernel<128>, grid, dim3(64), 0, st, a);
    else
      hipLaunchKernelGGL(append_e4m3_kernel<64>, grid, dim3(64), 0, st, a);
  } else {
    const int64_t blocks = ceil_div(batch->n_tokens * (a.row_bytes / 16), kThreads);
    if (blocks >= kMaxGrid) CKV_FAIL(CKV_EUNSUPPORTED, "too many rows in one call");
    hipLaunchKernelGGL(append_kernel, dim3((unsigned)blocks, 1, 2), dim3(kThreads), 0, st, a);
  }
  CKV_HIP(hipGetLastError());
  return CKV_OK;
}

ckv_status ckv_page_copy(const ckv_page_pool* pools, int32_t n_pools, const int32_t* src,
                         const int32_t* dst, int64_t count, void* stream) {
  clear_error();
  MoveArgs a;
  CKV_CHECK(check_pools(pools, n_pools, a));
  CKV_REQUIRE(count >= 0, "count must be >= 0 (got %lld)", (long long)count);
  if (count == 0 || n_pools == 0) return CKV_OK;
  CKV_REQUIRE(count <= INT32_MAX, "too many pairs");
  CKV_REQUIRE(src && dst, "NULL pointer argument");
  for (int p0 = 0; p0 < n_pools; p0 += kMaxPools) {
    PoolTable t;
    fill_table(t, pools + p0, std::min(kMaxPools, n_pools - p0));
    const int64_t work = count * a.pieces * 2 * t.n;
    const int u = unroll_of(a.page_bytes);
    const auto kernel = u == 4 ? copy_pages_kernel<4> : u == 2 ? copy_pages_kernel<2> : copy_pages_kernel<1>;
    hipLaunchKernelGGL(kernel, dim3((unsigned)std::min(work, kMoveBlocks)), dim3(kThreads),
                       0, (hipStream_t)stream, t, a, src, dst, count);
    CKV_HIP(hipGetLastError());
  }
  return CKV_OK;
}

size_t ckv_page_compact_workspace_bytes(int64_t n_pages) {
  return n_pages < 1 || n_pages > INT32_MAX ? 0 : plan_layout(n_pages).bytes;
}

ckv_status ckv_page_compact(const ckv_page_pool* pools, int32_t n_pools, const int32_t* refs,
                            int32_t* refs_out, int64_t n_pages, const int32_t* table,
                            int32_t* table_out, int64_t n_entries, int32_t* n_live, void* ws,
                            size_t ws_bytes, void* stream) {
  clear_error();
  MoveArgs a;
  CKV_CHECK(check_pools(pools, n_pools, a));
  CKV_REQUIRE(n_pages >= 1 && n_pages <= INT32_MAX, "n_pages must be in [1, 2^31-1] (got %lld)",
              (long long)n_pages);
  // (its plan goes over the blocks' counts from every block)
  if (n_pages > (int64_t(1) << 26)) CKV_FAIL(CKV_EUNSUPPORTED, "more than 2^26 pages to compact");
  CKV_REQUIRE(n_pools == 0 || n_pages == a.n_pages, "the pools hold %lld pages, not %lld",
              (long long)a.n_pages, (long long)n_pages);
  CKV_REQUIRE(n_entries >= 0, "n_entries must be >= 0 (got %lld)", (long long)n_entries);
  CKV_REQUIRE(refs && refs_out && n_live && ws, "NULL pointer argument");
  CKV_REQUIRE(n_entries == 0 || (table && table_out), "NULL table with entries");
  const PlanLayout l = plan_layout(n_pages);
  CKV_REQUIRE(ws_bytes >= l.bytes, "workspace too small: %zu < %zu", ws_bytes, l.bytes);
  CKV_REQUIRE(aligned16(ws), "pointers must be 16-byte aligned");
  auto at = [&](size_t off) { return reinterpret_cast<int32_t*>(static_cast<char*>(ws) + off); };
  const PlanArgs pl{refs, n_pages, at(l.counts), at(l.rank), at(l.hole), at(l.mover),
                    at(l.mover_refs), at(l.head), n_live};
  const hipStream_t st = (hipStream_t)stream;
  const unsigned blocks = (unsigned)ceil_div(n_pages, kPlan);
  // Up to 4 workgroups each count all pages themselves: 4,000 pages in one launch of 6.2 us
  // instead of two of 5.2 and 5.4; more of them go by the counts.
  if (blocks <= 4) {
    hipLaunchKernelGGL(compact_rank_kernel<true>, dim3(blocks), dim3(kPlanThreads), 0, st, pl);
  } else {
    hipLaunchKernelGGL(compact_count_kernel, dim3(blocks), dim3(kPlanThreads), 0, st, pl);
    CKV_HIP(hipGetLastError());
    hipLaunchKernelGGL(compact_rank_kernel<false>, dim3(blocks), dim3(kPlanThreads), 0, st, pl);
  }
  CKV_HIP(hipGetLastError());
  for (int p0 = 0; p0 == 0 || p0 < n_pools; p0 += kMaxPools) {
    PoolTable t;
    fill_table(t, pools + p0, std::min(kMaxPools, n_pools - p0));
    FollowArgs f{refs, refs_out, table, table_out, n_entries, 0};
    if (p0 == 0)  // once
      f.follow_blocks = std::min<int64_t>(256, ceil_div(std::max(n_pages, n_entries), kThreads));
    // at most half the pages move
    const int64_t work = n_pages / 2 * a.pieces * 2 * t.n;
    const unsigned grid = (unsigned)(f.follow_blocks + std::min(work, kMoveBlocks));
    if (grid == 0) continue;
    const int u = unroll_of(a.page_bytes);
    const auto kernel = u == 4 ? compact_move_kernel<4> : u == 2 ? compact_move_kernel<2> : compact_move_kernel<1>;
    hipLaunchKernelGGL(kernel, dim3(grid), dim3(kThreads), 0, st, t, a, pl, f);
    CKV_HIP(hipGetLastError());
  }
  return CKV_OK;
}

}  // extern "C"
