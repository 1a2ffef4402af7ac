// page_attn.hip -- attention over a paged KV cache for gfx950: decoding and prefill,
// a sliding window with the first tokens kept visible, pages in fp32, bf16 or 8 bits.
//
// For a query at position p of its sequence and the keys j that it sees,
//   out = sum_j exp(s_j - m) v_j / sum_j exp(s_j - m),  s_j = sm_scale q.k_j,
// for any reference m.  A key is seen if j <= p, its page is there, and (window > 0)
// j > p - window or j < n_sinks.  An 8-bit row is code * 2^(byte - 127), which bf16 holds
// exactly but for the largest (finite_codes): what follows the conversion is the bf16 computation.
//
// A sequence of few rows (query x head of one KV head) is bound by reading its K and V once:
// page_rows_kernel, 16 rows per workgroup, many splits of the keys.  One of many rows by its
// products: page_tile_kernel, 128 rows against tiles in LDS.  A call takes the second from
// 33 rows per KV head on (one sequence of 33,000 tokens in 8 bits, 28 heads on 4, at 3, 4, 5, 7
// and 18 tokens of 7 rows: rows 16.7, 17.0, 23.8, 26.3 and 46.3 us, tiles 22.5, 22.7, 23.1, 23.7
// and 27.7; 16 sequences of up to 8,000 in bf16 with up to as many: 43.1, 43.6, 46.2, 57.3 and
// 83.5, 46.4, 44.5, 45.1, 48.5 and 52.9).  fp32 has the first only: 128 tokens on 4,096 14.1 us,
// 1,000 on 4,000 59 (3.6 GFLOP; a product of 8,192 reaches 154 TFLOP/s).  Splits (by each
// sequence's own length) leave partials in fp32 that page_combine_kernel joins in split order.
//
// Measured, join included: 64 sequences of 1,024 to 16,384 tokens in 8 bits, 40 heads on 8,
// 163 us, 4.8 TB/s (a kernel that only reads such pages reaches 5.6 to 6.0); 48 of up to 30,011
// with a window of 4,096 in bf16 80 us, 4.6 TB/s; 512 tokens on 32,768 others, 28 heads on 4:
// 239 to 254 us by the card, 955 to 1,010 TFLOP/s, in bf16 and 8 bits alike (a matrix product of
// 8,192 reaches 1,210 to 1,230); five prompts of up to 2,048 tokens with a window of 1,000 130 us, 766.
//
// Groups of sequences that share their first pages (page_parts_kernel): the softmax is taken in two
// parts, over the shared keys for all rows of a group at once and over each sequence's own keys
// behind them, each against its own reference; the join of the splits makes one of both, for any
// references.  48 sequences on 30,011 shared tokens in bf16, 28 heads on 4: 51 us a layer, where each
// sequence by itself reads 3 GB; eight groups of eight on up to 16,384 in 8 bits, 40 heads on 8: 60 us,
// 3.3 TB/s of bytes read once; 24 prompts of up to 48 tokens on 32,768 in 8 bits: 335 to 369 us by the card, 925
// to 1,020 TFLOP/s, apart 541.

#include <type_traits>

#include "attn_tile.h"
#include "pages_internal.h"

namespace ckv {
namespace {

constexpr int kTile = 32;  // keys per step of a wave
constexpr int kRows = 16;  // query rows (query x head of one KV head) per workgroup
constexpr float kNone = -3.4028234663852886e38f;  // reference of a row that has seen no key
// A row's reference follows its maximum once that is 8 log2 units above it: sums and
// outputs stay below 2^8 times what the maximum itself would give, and a rescaling
// of the outputs is rare.
constexpr float kSlack = 8.f;
// An exponent s c1 - m in one fused step leaves the maximum itself, whose m is rounded, at up to half a
// step of m: a quarter below 2^23, powers of two that pass the range from 2^30 on.  Rows whose
// reference is past this take s c1 as rounded too, which the maximum is then exactly (page_rows_kernel;
// page_tile_kernel when it does a split again).
constexpr float kFar = 0x1p23f;

struct PageAttnArgs {
  PageSeqs s;
  const char* k;
  const char* v;
  const uint8_t* k_scale;
  const uint8_t* v_scale;
  int64_t page_stride;  // bytes
  int64_t n_pages;
  const void* q;        // [n_tokens][Hq][D]
  void* out;
  float* o_part;        // [splits][n_tokens][Hq][D]
  float2* ml_part;      // [splits][n_tokens][Hq]: (reference, sum)
  int32_t* n_parts;     // [n_tokens]: splits that the token's sequence takes
  int c, log2c;         // log2c: -1 if c is no power of two
  int Hkv, Hq, G;
  int window, sinks, n_splits;
  uint32_t n_blocks;    // blocks of 128 rows, at most (page_tile_kernel)
  int slice;            // steps that a sequence takes another split for
  float c1;
  // groups that share a prefix (parts below)
  const int32_t* grp_off;  // [n_groups + 1]
  const int32_t* shared;   // [n_groups] tokens, [n_groups] leaders, [n_seqs] tokens
  int n_groups;
  int n_wgs;               // workgroups of few rows for the shared keys of one KV head, about
  const int32_t* shared_parts;  // the join: splits of the shared keys by token
  int shared_splits;            //   and the places that they have;
  int first_places;             //   places up to which most rows have all of theirs
};

// What a launch attends over: whole sequences; or, where groups of them share a prefix, in one
// launch the shared keys for all rows of a group, in another each sequence's own keys behind
// them.  The parts meet in the join of the splits.  kAlone: whole sequences in fp32, their
// exponents as those of the parts (rows_part).
enum Part { kWhole, kShared, kOwn, kAlone };
constexpr bool is_whole(int part) { return part == kWhole || part == kAlone; }

// The rows and keys of one unit of a launch's work: a sequence, or a group (kShared), whose
// rows are those of its sequences.
struct Unit {
  SeqSpan sp;          // its token rows
  const int32_t* tab;  // its table
  int first, kv_end;   // its keys' positions; `first` is a whole number of kTile
  int p_base;          // the first row's position
};
template <int P>
__device__ __forceinline__ int n_units(const PageAttnArgs& a) {
  return P == kShared ? a.n_groups : a.s.n_seqs;
}
// The first sequence of a group, inside the batch whatever grp_off holds.
__device__ __forceinline__ int group_begin(const PageAttnArgs& a, int g) {
  return min(max(a.grp_off[g], 0), a.s.n_seqs);
}
template <int P>
__device__ __forceinline__ int64_t unit_token(const PageAttnArgs& a, int u) {
  return token_of(a.s, P == kShared ? group_begin(a, u) : u);
}
// Shared tokens as ckv_page_share left them, inside the table whatever they are.
__device__ __forceinline__ int shared_tokens(const PageAttnArgs& a, int at) {
  return (int)min((int64_t)max(a.shared[at], 0), (int64_t)a.s.max_pages * a.c) & ~31;
}
template <int P>
__device__ __forceinline__ Unit unit_of(const PageAttnArgs& a, int u) {
  Unit x;
  if constexpr (P == kShared) {
    const int64_t lo = unit_token<P>(a, u), hi = unit_token<P>(a, u + 1);
    x.kv_end = shared_tokens(a, u);
    x.p_base = x.kv_end;  // past every key: nothing is hidden
    x.sp = SeqSpan{lo, (int32_t)max<int64_t>(hi - lo, 0), x.kv_end};
    x.tab = a.s.table + (int64_t)min(max(a.shared[a.n_groups + u], 0), a.s.n_seqs - 1) * a.s.table_stride;
    x.first = 0;
  } else {
    x.sp = seq_span(a.s, u);
    x.tab = a.s.table + (int64_t)u * a.s.table_stride;
    x.kv_end = (int)min<int64_t>(max(x.sp.len, 0), (int64_t)a.s.max_pages * a.c);
    x.first = P == kOwn ? shared_tokens(a, 2 * a.n_groups + u) : 0;
    x.p_base = x.sp.len - x.sp.count;
  }
  return x;
}
// Splits of a unit of so many steps.  A whole sequence without a key has one, which writes its
// rows' zeros; a part that another one completes has none.
template <int P>
__device__ __forceinline__ int parts_of(const PageAttnArgs& a, const Unit& x, int steps, int slice) {
  const int least = is_whole(P) || (P == kOwn && x.first == 0) ? 1 : 0;
  return min(max((steps + slice - 1) / slice, least), a.n_splits);
}
// Steps of a split of shared keys, so that the groups' splits together are a.n_wgs at most (for
// one KV head), as many as run at once, however unequal the groups are; a.slice at least.
__device__ __forceinline__ int shared_slice(const PageAttnArgs& a) {
  const int more = a.n_wgs - a.n_groups;  // splits beside each group's first
  if (more <= 0) return 1 << 30;
  int64_t steps = 0;
  for (int g0 = 0; g0 < a.n_groups; g0 += 64) {
    const int g = g0 + (int)(threadIdx.x & 63);
    int x = g < a.n_groups ? shared_tokens(a, g) / kTile : 0;
#pragma unroll
    for (int i = 1; i < 64; i <<= 1) x += __shfl_xor(x, i);
    steps += x;
  }
  return __builtin_amdgcn_readfirstlane((int)max((steps + more - 1) / more, (int64_t)a.slice));
}
// What the join reads of a token's sequence: its splits and, of kOwn, whether shared ones go before.
constexpr int kAfterShared = 1 << 30;
template <int P>
__device__ __forceinline__ int parts_note(const Unit& x, int n_parts) {
  return P == kOwn && x.first > 0 ? n_parts | kAfterShared : n_parts;
}

// The keys of a block of rows as steps of kTile: those that hold the sinks, then those
// from the window's begin on.
struct Steps {
  int n_sink, first, n;  // step i: tile i < n_sink ? i : first + i - n_sink
  __device__ __forceinline__ int tile(int i) const { return i < n_sink ? i : first + (i - n_sink); }
};
// For queries at positions p0 .. p1 of a sequence with keys below kv_end.
template <int P>
__device__ __forceinline__ Steps steps_of(const PageAttnArgs& a, int p0, int p1, int first, int kv_end) {
  Steps s{0, P == kOwn ? first / kTile : 0, 0};
  const int hi = min(p1 + 1, kv_end);
  if (hi <= 0) return s;
  const int tiles = (hi + kTile - 1) / kTile;
  if (P == kWhole && a.window > 0) {
    const int lo = max(p0 - a.window + 1, 0);
    s.n_sink = (min(min(a.sinks, lo), hi) + kTile - 1) / kTile;
    s.first = max(lo / kTile, s.n_sink);
  }
  s.n = s.n_sink + max(tiles - s.first, 0);
  return s;
}

// The same keys as groups of 8, which lie in one page each: those that hold the sinks, then
// those from the window's begin on, without a gap between.
struct Groups {
  int n_sink, first, n;
  __device__ __forceinline__ int pos(int i) const { return 8 * (i < n_sink ? i : first + (i - n_sink)); }
};
template <int P>
__device__ __forceinline__ Groups groups_of(const PageAttnArgs& a, int p0, int p1, int first, int kv_end) {
  Groups s{0, P == kOwn ? first / 8 : 0, 0};
  const int hi = min(p1 + 1, kv_end);
  if (hi <= 0) return s;
  if (P == kWhole && a.window > 0) {
    const int lo = max(p0 - a.window + 1, 0);
    s.n_sink = (min(min(a.sinks, lo), hi) + 7) / 8;
    s.first = max(lo / 8, s.n_sink);
  }
  s.n = s.n_sink + max((hi + 7) / 8 - s.first, 0);
  return s;
}

// The entry of a slot of a sequence's table (past its end: of its last slot, whose
// page then counts as not there).
__device__ __forceinline__ int entry_of(const PageAttnArgs& a, const int32_t* tab, int slot) {
  return tab[min(slot, a.s.max_pages - 1)];
}
// The same, for a slot that is one for the wave: a scalar load, which the wait for
// rows in flight does not include.
__device__ __forceinline__ int entry_of_uniform(const PageAttnArgs& a, const int32_t* tab, int slot) {
  return *(const __attribute__((address_space(4))) int32_t*)(tab + min(slot, a.s.max_pages - 1));
}
__device__ __forceinline__ bool names_page(const PageAttnArgs& a, int entry) {
  return entry >= 0 && entry < a.n_pages;
}

template <int T>
struct Elem;  // the cache's element
template <>
struct Elem<CKV_DTYPE_F32> {
  static constexpr int kBytes = 4;
  using Q = float;
};
template <>
struct Elem<CKV_DTYPE_BF16> {
  static constexpr int kBytes = 2;
  using Q = __bf16;
};
template <>
struct Elem<CKV_DTYPE_E4M3> {
  static constexpr int kBytes = 1;
  using Q = __bf16;
};

// What a wave holds of a step: the table entries of its 16-key (kSmall: 8-key) groups and
// where these begin in the pool, and its V rows and scales as loaded.
template <bool kSmall>
struct Pages {
  __attribute__((ext_vector_type(kSmall ? 4 : 2))) int e;
  __attribute__((ext_vector_type(kSmall ? 4 : 2))) int64_t at;
};
template <int D, int T>
struct Step {
  uint32_t v[2][4][D / 16 * Elem<T>::kBytes / 4];
  uint32_t ks[2], vs[2];
};

__device__ __forceinline__ uint32_t bf16_pair(float x, float y) {
  const bf16x2 b = {(__bf16)x, (__bf16)y};
  return __builtin_bit_cast(uint32_t, b);
}

// l plus both numbers of a packed pair.  A row's sum takes its numerators as they are
// rounded for the product with V, so that a key that outweighs the others keeps its exact
// weight (500 tokens on 4,000: 2.34e-3 -> 2.22e-3 off 64 bits, 1.66e-3 of it the output's
// own rounding; the product with ones also takes one instruction in place of two).
__device__ __forceinline__ float add_pair(uint32_t pair, float l) {
  const bf16x2 ones = {(__bf16)1.f, (__bf16)1.f};
  return __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2, pair), ones, l, false);
}

// 8 codes (two dwords) as bf16, each times the scale.
__device__ __forceinline__ bf16x8 bf16_of_codes(uint32_t w0, uint32_t w1, float scale) {
  u32x4 r;
  r[0] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w0, scale, false));
  r[1] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w0, scale, true));
  r[2] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w1, scale, false));
  r[3] = __builtin_bit_cast(uint32_t, __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w1, scale, true));
  return __builtin_bit_cast(bf16x8, r);
}

// s_waitcnt: vmcnt(0); lgkmcnt(0).
__device__ __forceinline__ void wait_loads() { __builtin_amdgcn_s_waitcnt(0x0f70); }
__device__ __forceinline__ void wait_lds() { __builtin_amdgcn_s_waitcnt(0xc07f); }

// 4 codes of a page whose scale byte is kTopByte or more.  There 256 times the scale is 2^128,
// which bf16 does not hold: codes of 256 and more are taken for 240, the largest below (a
// finite number appended is then read within the half step that its rounding is off by).
// Bytes 0x78 to 0x7e become 0x77; 0x7f, a NaN, stays.
constexpr uint32_t kTopByte = 247;
__device__ __forceinline__ uint32_t finite_codes(uint32_t w) {
  const uint32_t big = w >> 3 & w >> 4 & w >> 5 & w >> 6 & 0x01010101u, top = big & ~(w & w >> 1 & w >> 2);
  return (w & ~(top * 0x7fu)) | top * 0x77u;
}

// Few rows: where the waves' K rows lie in LDS, after the last step their outputs with references and sums,
// and the query rows: its own memory, or that of another kernel's part in one launch.
template <int D, int T, int kWaves, int kBlocks>
struct RowsLds {
  // 8 waves have about two steps each (a launch of so few workgroups has splits of 16): both
  // are loaded before the first is waited for (one sequence of 32,801 tokens in 8 bits 14.5 ->
  // 14.1 us, 16 of up to 8,000 11.4 -> 11.1).
  static constexpr bool kPairs = kWaves == 8;
  static constexpr int kBuf = (kPairs ? 2 : 1) * kTile * D * Elem<T>::kBytes;  // of a wave
  static constexpr int kOut = kRows * (D + 4) * (int)sizeof(float);
  static constexpr int kJoined = kWaves * (kOut + kRows * (int)sizeof(float2));
  static constexpr int kQRow = D + 8;  // of the query rows: 16 lanes in a column of pieces meet all banks
  static constexpr int kQ = kBlocks > 1 ? kBlocks * kRows * kQRow * 2 : 0;
  static constexpr int kBytes = kJoined > kWaves * kBuf ? kJoined : kWaves * kBuf;
  char* lds;
  uint16_t* q;
  __device__ __forceinline__ char* mine_k(int wave) const { return lds + wave * kBuf; }
  __device__ __forceinline__ float* mine_o(int wave) const { return o(wave); }
  __device__ __forceinline__ float* o(int w) const { return reinterpret_cast<float*>(lds + w * kOut); }
  __device__ __forceinline__ float2* ml(int w) const { return reinterpret_cast<float2*>(lds + kWaves * kOut) + w * kRows; }
};

// Few rows: a workgroup owns 16 query rows of one KV head and one split of their
// steps, its 4 or 8 waves step by step in turn:
//   S^T = K Q^T    MFMA 16x16 (bf16: x32, fp32: x4), two groups of 16 keys; lane l
//                  then holds row l % 16 and keys 4 (l / 16) + 0..3 of each group
//   O^T += V^T P^T the contraction's 8 (bf16) keys per lane are those it holds, so
//                  P^T goes from the softmax registers to the MFMA as it is; lane l
//                  loads D/16 elements from l % 16 * D/16 on of its 8 keys' V rows, and
//                  product i of D/16 takes element i of each (8 keys x D/16 elements
//                  are turned over in registers).
// V rows go straight to registers, 16 lanes a row.  The K operand wants neighbouring
// lanes in different rows, which read so cost the cache an access per 16 bytes: K rows go
// whole to LDS, a step ahead, into a buffer of the wave's own (64 sequences in 8 bits: 173 us
// with K read to registers, 165 so).  The waves' outputs are joined through LDS.
// Bound by memory, and by latency where there is little of it: a decoding step of one
// sequence of 1,000 tokens takes 6.6 us: four dependent round trips, two steps per wave of 0.9,
// the waves' join 0.4.
// kSmall: pages of 8 tokens, four in a step (else at least 16 keys share a page).
// kBlocks: 16-row blocks of a workgroup, which share the keys as loaded, converted and turned over;
// their query rows then come from LDS.  Up to 48 rows of a group go so (32 in bf16 at head_dim 128,
// where three blocks take every register): eight groups of 40 rows in 8 bits, with 1,024 workgroups
// each, shared keys alone 67 us in 128-row tiles, 52 in three blocks; four groups' 42 rows in bf16
// 63 in tiles, 68 in three blocks.  More rows in several such workgroups: 336 rows 49 to 53 us where
// the tiles take 44.
// The workgroup is (bx, by) of a grid gy high.
template <int D, int T, bool kSmall, int kWaves, int P, int kBlocks, class Lds>
__device__ __forceinline__ void rows_part(const PageAttnArgs& a, uint32_t bx, uint32_t by, uint32_t gy, const Lds& lds) {
  using E = Elem<T>;
  using QT = typename E::Q;
  constexpr bool kF32 = T == CKV_DTYPE_F32, kE4 = T == CKV_DTYPE_E4M3;
  static_assert(kBlocks == 1 || !kF32);
  // In fp32, but for ckv_page_attn, an exponent s c1 - m is rounded once (up to kFar), so that keys near
  // the maximum, which count, lose nothing to the size of s c1, and a logit is the sum of four parts:
  // 12 cases of logits around 10 are 1.8e-7 to 5.8e-7 off 64 bits, 2.9e-7 to 1.3e-6 without.
  constexpr bool kFused = kF32 && P != kWhole;
  constexpr int kVec = D / 16;                    // elements of a V row per lane, and products of O
  constexpr int kRow = D * E::kBytes;             // bytes of a K row in LDS
  constexpr int kPieces = kRow / 64;              // 16-byte pieces of a K row per lane
  constexpr int kVWords = kVec * E::kBytes / 4;   // dwords of a V row per lane

  // The KV heads of one slice of keys are neighbours on one XCD, where together they read
  // whole token rows.  The slices go round the XCDs, every sequence's first ones before the
  // second ones and so on, turned by one from split to split: long sequences spread.
  const uint32_t pair = bx / 8 / a.Hkv * 8 + (bx & 7), units = n_units<P>(a);
  if (pair >= units * a.n_splits) return;
  const int g = (int)(bx / 8 % a.Hkv), split = (int)(pair / units);
  const int b = (int)((pair + split) % units);
  const int lane = threadIdx.x & 63, n16 = lane & 15, j4 = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const Unit unit = unit_of<P>(a, b);
  const SeqSpan& sp = unit.sp;
  if (sp.count == 0) return;
  const int32_t* tab = unit.tab;
  const int kv_end = unit.kv_end;
  const int row_bytes = a.Hkv * kRow, kvh = g, g_bytes = g * kRow;
  const int rows = sp.count * a.G;
  const int p_base = unit.p_base;
  // this sequence's own number of splits, by its length
  const int all_steps = steps_of<P>(a, p_base, p_base + sp.count - 1, unit.first, kv_end).n;
  const int n_parts = parts_of<P>(a, unit, all_steps, P == kShared ? shared_slice(a) : a.slice);
  if ((!is_whole(P) || a.n_splits > 1) && split == 0 && g == 0 && by == 0)
    for (int i = threadIdx.x; i < sp.count; i += 64 * kWaves) a.n_parts[sp.first + i] = parts_note<P>(unit, n_parts);
  if (split >= n_parts) return;

  constexpr bool kPairs = kWaves == 8;
  char* const lds_k = lds.mine_k(wave);
  // A load to LDS moves kLoadRows rows, lane l 16 bytes of row l / kSegs: the segment at
  // position s of row r is segment s ^ swz(r), so that 16 lanes that read one piece of 16
  // rows each meet 64 different banks.
  constexpr int kSegs = kRow / 16, kLoadRows = 64 / kSegs, kLoads = kTile / kLoadRows;
  constexpr auto swz = [](int r) { return kSegs == 16 ? r & 15 : kSegs == 8 ? r >> 1 & 7 : r >> 2 & 3; };
  const uint32_t k_col = (uint32_t)(lane / kSegs * row_bytes + g_bytes + ((lane % kSegs) ^ swz(lane / kSegs)) * 16);
  uint32_t k_at[kPieces];  // this lane's pieces of row n16
#pragma unroll
  for (int y = 0; y < kPieces; ++y) k_at[y] = (uint32_t)(n16 * kRow + (((j4 + 4 * y) ^ swz(n16)) * 16));
  const uint32_t v_col = (uint32_t)(4 * j4 * row_bytes + g_bytes + n16 * kVec * E::kBytes);

  constexpr int kQRow = D + 8;

  for (int rb = by; rb * (kRows * kBlocks) < rows; rb += gy) {
    const int r_first = rb * (kRows * kBlocks), r_last = min(rows, r_first + kRows * kBlocks) - 1;
    const int p0 = p_base + r_first / a.G, p1 = p_base + r_last / a.G;
    const Steps steps = steps_of<P>(a, p0, p1, unit.first, kv_end);
    const int per = steps.n / n_parts, over = steps.n % n_parts;  // the first `over` splits: one more
    const int begin = split * per + min(split, over), end = begin + per + (split < over ? 1 : 0);

    // this lane's row of each block: its query (position p) and head
    int p[kBlocks];
    const QT* q[kBlocks];
#pragma unroll
    for (int k = 0; k < kBlocks; ++k) {
      const int r = min(r_first + kRows * k + n16, r_last);
      const int64_t tok = sp.first + r / a.G;
      const int head = g * a.G + r % a.G;
      p[k] = p_base + r / a.G;
      q[k] = static_cast<const QT*>(a.q) + (tok * a.Hq + head) * D;
    }
    // Q^T operands in the order of the K pieces
    f32x4 qf[kF32 ? kPieces : 1];
    bf16x8 qb[kF32 || kBlocks > 1 ? 1 : D / 32];
    const auto q_piece = [&](int i) { return kE4 ? 64 * (i >> 1) + 16 * j4 + 8 * (i & 1) : 32 * i + 8 * j4; };
    if constexpr (kF32) {
#pragma unroll
      for (int i = 0; i < kPieces; ++i) qf[i] = *reinterpret_cast<const f32x4*>(q[0] + 16 * i + 4 * j4);
    } else if constexpr (kBlocks == 1) {
#pragma unroll
      for (int i = 0; i < D / 32; ++i) qb[i] = *reinterpret_cast<const bf16x8*>(q[0] + q_piece(i));
    } else {
      // each wave brings some of the rows
      constexpr int kSegsQ = D / 8;
      for (int i = threadIdx.x; i < kBlocks * kRows * kSegsQ; i += 64 * kWaves) {
        const int r = min(r_first + i / kSegsQ, r_last);
        const QT* from = static_cast<const QT*>(a.q) + ((sp.first + r / a.G) * a.Hq + g * a.G + r % a.G) * D;
        *reinterpret_cast<u32x4*>(lds.q + i / kSegsQ * kQRow + i % kSegsQ * 8) =
            *reinterpret_cast<const u32x4*>(from + i % kSegsQ * 8);
      }
      __syncthreads();
    }
    const auto query = [&](int k, int i) __attribute__((always_inline)) {
      if constexpr (kBlocks == 1)
        return qb[i];
      else
        return *reinterpret_cast<const bf16x8*>(lds.q + (kRows * k + n16) * kQRow + q_piece(i));
    };

    f32x4 o[kBlocks][kVec];
    float ref[kBlocks], l[kBlocks];
#pragma unroll
    for (int k = 0; k < kBlocks; ++k) {
      ref[k] = kNone;
      l[k] = 0.f;
#pragma unroll
      for (int i = 0; i < kVec; ++i) o[k][i] = f32x4{0.f, 0.f, 0.f, 0.f};
    }

    // The table entries of a step's groups of keys.
    constexpr int kGroup = kSmall ? 8 : 16;
    auto pages_of = [&](int st, Pages<kSmall>& x) __attribute__((always_inline)) {
      const int pos0 = steps.tile(st) * kTile;
#pragma unroll
      for (int i = 0; i < kTile / kGroup; ++i) {
        const int pos = pos0 + kGroup * i;
        x.e[i] = entry_of_uniform(a, tab, kSmall ? pos >> 3 : a.log2c >= 0 ? pos >> a.log2c
                                                                           : (int)((uint32_t)pos / (uint32_t)a.c));
      }
    };
    // (a missing page: page 0, and its keys count for nothing)
    auto locate = [&](int st, Pages<kSmall>& x) __attribute__((always_inline)) {
      const int pos0 = steps.tile(st) * kTile;
#pragma unroll
      for (int i = 0; i < kTile / kGroup; ++i) {
        const int pos = pos0 + kGroup * i;
        const int r0 = kSmall ? 0 : a.log2c >= 0 ? pos & (a.c - 1) : (int)((uint32_t)pos % (uint32_t)a.c);
        x.at[i] = (int64_t)(names_page(a, x.e[i]) ? x.e[i] : 0) * a.page_stride + (int64_t)r0 * row_bytes;
      }
    };
    auto load_k = [&](const Pages<kSmall>& x, char* to) __attribute__((always_inline)) {
#pragma unroll
      for (int i = 0; i < kLoads; ++i) {
        constexpr int kPer = kLoadRows > kGroup ? kLoadRows / kGroup : 1;  // groups of a load: 2 at most
        const uint32_t col = k_col ^ (uint32_t)(64 * (i & (kSegs / 4 - 1)));
#pragma unroll
        for (int h = 0; h < kPer; ++h) {
          const int key = i * kLoadRows + h * kGroup;
          const __amdgpu_buffer_rsrc_t rsrc = tile::raw_rsrc(a.k + x.at[key / kGroup], 0xffffffffu);
          // (the second half of a load has the second group: 8 rows back in the lanes' offsets)
          const uint32_t in_group = (uint32_t)(key % kGroup * row_bytes);
          if (kPer == 1 || lane >> 5 == h)
            __builtin_amdgcn_raw_ptr_buffer_load_lds(rsrc, (tile::LdsPtr)(to + i * kLoadRows * kRow), 16,
                                                     col - (uint32_t)(h * kGroup * row_bytes), in_group, 0, 0);
        }
      }
    };
    auto load_v = [&](const Pages<kSmall>& x, Step<D, T>& y) __attribute__((always_inline)) {
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        if constexpr (kE4) {  // pages of K row 16 i + n16, V rows 16 i + 4 j4 ..
          int pk = x.e[kSmall ? 2 * i : i], pv = pk;
          if constexpr (kSmall) {
            pk = n16 & 8 ? x.e[2 * i + 1] : pk;
            pv = j4 & 2 ? x.e[2 * i + 1] : pv;
          }
          y.ks[i] = a.k_scale[(int64_t)(names_page(a, pk) ? pk : 0) * a.Hkv + kvh];
          y.vs[i] = a.v_scale[(int64_t)(names_page(a, pv) ? pv : 0) * a.Hkv + kvh];
        }
      }
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        if constexpr (kSmall) {
          const int64_t lo = x.at[2 * i], hi = x.at[2 * i + 1] - 8 * (int64_t)row_bytes;
          const char* at = a.v + (j4 & 2 ? hi : lo) + v_col;
#pragma unroll
          for (int k = 0; k < 4; ++k) {
            if constexpr (kVWords == 4)
              *reinterpret_cast<u32x4*>(y.v[i][k]) = *reinterpret_cast<const u32x4*>(at + k * row_bytes);
            else if constexpr (kVWords == 2)
              *reinterpret_cast<uint2*>(y.v[i][k]) = *reinterpret_cast<const uint2*>(at + k * row_bytes);
            else
              y.v[i][k][0] = *reinterpret_cast<const uint32_t*>(at + k * row_bytes);
          }
        } else {
          const __amdgpu_buffer_rsrc_t rsrc = tile::raw_rsrc(a.v + x.at[i], 0xffffffffu);
#pragma unroll
          for (int k = 0; k < 4; ++k) {
            if constexpr (kVWords == 4)
              *reinterpret_cast<u32x4*>(y.v[i][k]) =
                  __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(rsrc, v_col, k * row_bytes, 0));
            else if constexpr (kVWords == 2)
              *reinterpret_cast<uint2*>(y.v[i][k]) =
                  __builtin_bit_cast(uint2, __builtin_amdgcn_raw_buffer_load_b64(rsrc, v_col, k * row_bytes, 0));
            else
              y.v[i][k][0] = __builtin_amdgcn_raw_buffer_load_b32(rsrc, v_col, k * row_bytes, 0);
          }
        }
      }
    };
    auto attend = [&](int st, const Pages<kSmall>& e, u32x4 (&kw)[2][kPieces], Step<D, T>& x)
        __attribute__((always_inline)) {
      const int pos0 = steps.tile(st) * kTile;
      float ks[2], vs[2];
      if constexpr (kE4) {
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          ks[i] = scale_of(x.ks[i]);
          vs[i] = scale_of(x.vs[i]);
        }
        if (__builtin_expect(__any(max(max(x.ks[0], x.ks[1]), max(x.vs[0], x.vs[1])) >= kTopByte), 0)) {
#pragma unroll
          for (int i = 0; i < 2; ++i) {
            if (x.ks[i] >= kTopByte)
#pragma unroll
              for (int y = 0; y < kPieces; ++y)
#pragma unroll
                for (int w = 0; w < 4; ++w) kw[i][y][w] = finite_codes(kw[i][y][w]);
            if (x.vs[i] >= kTopByte)
#pragma unroll
              for (int k = 0; k < 4; ++k)
#pragma unroll
                for (int w = 0; w < kVWords; ++w) x.v[i][k][w] = finite_codes(x.v[i][k][w]);
          }
        }
      }
      f32x4 s[kBlocks][2];
#pragma unroll
      for (int k = 0; k < kBlocks; ++k)
#pragma unroll
        for (int i = 0; i < 2; ++i) s[k][i] = f32x4{0.f, 0.f, 0.f, 0.f};
      if constexpr (kFused) {
        // (a sum for each quarter of the products: half the roundings in a row, and no product waits
        // for the one before)
        f32x4 part[kPieces][2];
#pragma unroll
        for (int y = 0; y < kPieces; ++y)
#pragma unroll
          for (int i = 0; i < 2; ++i) part[y][i] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int z = 0; z < 4; ++z)
#pragma unroll
          for (int y = 0; y < kPieces; ++y)
#pragma unroll
            for (int i = 0; i < 2; ++i)
              part[y][i] = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(kw[i][y][z]), qf[y][z], part[y][i], 0, 0, 0);
#pragma unroll
        for (int i = 0; i < 2; ++i) s[0][i] = (part[0][i] + part[1][i]) + (part[2][i] + part[3][i]);
      } else if constexpr (kF32) {
#pragma unroll
        for (int y = 0; y < kPieces; ++y)
#pragma unroll
          for (int z = 0; z < 4; ++z)
#pragma unroll
            for (int i = 0; i < 2; ++i)
              s[0][i] = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(kw[i][y][z]), qf[y][z], s[0][i], 0, 0, 0);
      } else {
#pragma unroll
        for (int y = 0; y < D / 32; ++y) {
          bf16x8 kb[2];
#pragma unroll
          for (int i = 0; i < 2; ++i) {
            if constexpr (kE4)
              kb[i] = bf16_of_codes(kw[i][y >> 1][2 * (y & 1)], kw[i][y >> 1][2 * (y & 1) + 1], ks[i]);
            else
              kb[i] = __builtin_bit_cast(bf16x8, kw[i][y]);
          }
#pragma unroll
          for (int k = 0; k < kBlocks; ++k) {
            const bf16x8 qy = query(k, y);
#pragma unroll
            for (int i = 0; i < 2; ++i)
              s[k][i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kb[i], qy, s[k][i], 0, 0, 0);
          }
        }
      }
      // what some row of the block must not see
      const int last = pos0 + kTile;
      bool all = last <= min(p0 + 1, kv_end) &&
                 (a.window <= 0 || pos0 > p1 - a.window || last <= a.sinks);
#pragma unroll
      for (int i = 0; i < kTile / kGroup; ++i) all = all && names_page(a, e.e[i]);
      if (!all) {
        const int lo = a.window > 0 ? p0 - a.window : -1;  // the block's first row sees keys past it
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          int page = e.e[kSmall ? 2 * i : i];
          if constexpr (kSmall) page = j4 & 2 ? e.e[2 * i + 1] : page;
#pragma unroll
          for (int y = 0; y < 4; ++y) {
            const int pos = pos0 + 16 * i + 4 * j4 + y;
            const bool there = names_page(a, page) && pos < kv_end;
#pragma unroll
            for (int k = 0; k < kBlocks; ++k)
              if (!(there && pos <= p[k] && (a.window <= 0 || pos > p[k] - a.window || pos < a.sinks)))
                s[k][i][y] = -INFINITY;
            // a weight of 0 does not undo a NaN: rows that no query of the block sees are cleared
            if (!(there && pos <= p1 && (pos > lo || pos < a.sinks)))
#pragma unroll
              for (int w = 0; w < kVWords; ++w) x.v[i][y][w] = 0u;
          }
        }
      }
      u32x4 pb[kF32 ? 1 : kBlocks];
#pragma unroll
      for (int k = 0; k < kBlocks; ++k) {
        float mx = -INFINITY;
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
          for (int y = 0; y < 4; ++y) {
            if constexpr (kFused) {
              mx = fmaxf(mx, s[k][i][y] * a.c1);
            } else {
              s[k][i][y] *= a.c1;
              mx = fmaxf(mx, s[k][i][y]);
            }
          }
        if (__any(mx > ref[k] + kSlack)) {
          mx = fmaxf(mx, __shfl_xor(mx, 16));
          mx = fmaxf(mx, __shfl_xor(mx, 32));
          const float to = fmaxf(mx, ref[k]), f = __builtin_amdgcn_exp2f(ref[k] - to);
          ref[k] = to;
          l[k] *= f;
#pragma unroll
          for (int i = 0; i < kVec; ++i) o[k][i] *= f;
        }
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
          for (int y = 0; y < 4; ++y) {
            if constexpr (kFused) {
              const bool far = fabsf(ref[k]) >= kFar;
              s[k][i][y] = fmaf(far ? s[k][i][y] * a.c1 : s[k][i][y], far ? 1.f : a.c1, -ref[k]);
            } else {
              s[k][i][y] -= ref[k];
            }
            s[k][i][y] = __builtin_amdgcn_exp2f(s[k][i][y]);
            if constexpr (kF32) l[k] += s[k][i][y];
          }
        if constexpr (!kF32)
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            pb[k][i] = bf16_pair(s[k][i >> 1][2 * (i & 1)], s[k][i >> 1][2 * (i & 1) + 1]);
            l[k] = add_pair(pb[k][i], l[k]);
          }
      }
      if constexpr (kF32) {
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
          for (int y = 0; y < 4; ++y)
#pragma unroll
            for (int e = 0; e < kVec; ++e)
              o[0][e] = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(x.v[i][y][e]), s[0][i][y], o[0][e], 0, 0, 0);
      } else {
#pragma unroll
        for (int e = 0; e < kVec; ++e) {
          u32x4 vt;  // element e of the 8 keys
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const uint32_t* r0 = x.v[i >> 1][2 * (i & 1)];
            const uint32_t* r1 = x.v[i >> 1][2 * (i & 1) + 1];
            if constexpr (kE4) {
              // codes of elements 2 (e / 2) and + 1 of both keys, then the pair of element e
              const uint32_t w = __builtin_amdgcn_perm(r1[e >> 2], r0[e >> 2], e & 2 ? 0x07030602u : 0x05010400u);
              vt[i] = __builtin_bit_cast(
                  uint32_t, e & 1 ? __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, vs[i >> 1], true)
                                  : __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, vs[i >> 1], false));
            } else {
              vt[i] = __builtin_amdgcn_perm(r1[e >> 1], r0[e >> 1], e & 1 ? 0x07060302u : 0x05040100u);
            }
          }
#pragma unroll
          for (int k = 0; k < kBlocks; ++k)
            o[k][e] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, vt),
                                                              __builtin_bit_cast(bf16x8, pb[k]), o[k][e], 0, 0, 0);
        }
      }
    };

    int st = begin + wave;
    if constexpr (kPairs) {
      if (st < end) {
        Pages<kSmall> ga, gb;
        Step<D, T> xa, xb;
        pages_of(st, ga);
        pages_of(min(st + kWaves, end - 1), gb);
        auto read_k = [&](const char* from, u32x4 (&kw)[2][kPieces]) __attribute__((always_inline)) {
#pragma unroll
          for (int i = 0; i < 2; ++i)
#pragma unroll
            for (int y = 0; y < kPieces; ++y)
              kw[i][y] = *reinterpret_cast<const u32x4*>(from + i * 16 * kRow + k_at[y]);
        };
        while (true) {
          const bool two = st + kWaves < end;
          locate(st, ga);
          load_k(ga, lds_k);
          load_v(ga, xa);
          if (two) {
            locate(st + kWaves, gb);
            load_k(gb, lds_k + kTile * kRow);
            load_v(gb, xb);
          }
          __builtin_amdgcn_sched_barrier(0);
          wait_loads();
          __builtin_amdgcn_sched_barrier(0);
          u32x4 kw[2][kPieces];
          read_k(lds_k, kw);
          attend(st, ga, kw, xa);
          if (!two) break;
          read_k(lds_k + kTile * kRow, kw);
          attend(st + kWaves, gb, kw, xb);
          st += 2 * kWaves;
          if (st >= end) break;
          pages_of(st, ga);
          pages_of(min(st + kWaves, end - 1), gb);
          wait_lds();  // read: the next steps' rows may come
          __builtin_amdgcn_sched_barrier(0);
        }
      }
    } else if (st < end) {
      // A step's rows load during the step before, its table entries two steps before.
      Pages<kSmall> ga, gb;
      Step<D, T> xa, xb;
      pages_of(st, ga);
      pages_of(min(st + kWaves, end - 1), gb);
      locate(st, ga);
      load_k(ga, lds_k);
      load_v(ga, xa);
      __builtin_amdgcn_sched_barrier(0);
      auto turn = [&](Pages<kSmall>& g, Step<D, T>& x, Pages<kSmall>& gn, Step<D, T>& xn)
          __attribute__((always_inline)) {
        wait_loads();  // the K rows are in LDS
        __builtin_amdgcn_sched_barrier(0);
        u32x4 kw[2][kPieces];
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
          for (int y = 0; y < kPieces; ++y)
            kw[i][y] = *reinterpret_cast<const u32x4*>(lds_k + i * 16 * kRow + k_at[y]);
        wait_lds();  // read: the next step's may come
        __builtin_amdgcn_sched_barrier(0);
        locate(min(st + kWaves, end - 1), gn);
        if (st + kWaves < end) {
          load_k(gn, lds_k);
          load_v(gn, xn);
        }
        Pages<kSmall> after;
        pages_of(min(st + 2 * kWaves, end - 1), after);
        attend(st, g, kw, x);
        g = after;
        st += kWaves;
        __builtin_amdgcn_sched_barrier(0);
      };
      while (true) {
        turn(ga, xa, gb, xb);
        if (st >= end) break;
        turn(gb, xb, ga, xa);
        if (st >= end) break;
      }
    }

#pragma unroll
    for (int k = 0; k < kBlocks; ++k) {
      l[k] += __shfl_xor(l[k], 16);
      l[k] += __shfl_xor(l[k], 32);
      __syncthreads();  // every wave is through with its K rows (the block before is written)
      // o[x][v] holds element kVec (4 j4 + v) + x of row n16
#pragma unroll
      for (int v = 0; v < 4; ++v)
#pragma unroll
        for (int x = 0; x < kVec; ++x) lds.mine_o(wave)[n16 * (D + 4) + kVec * (4 * j4 + v) + x] = o[k][x][v];
      if (lane < kRows) lds.ml(wave)[lane] = make_float2(ref[k], l[k]);
      __syncthreads();
      // 16 threads per row, D / 16 elements each
      const int row = threadIdx.x >> 4, col = (threadIdx.x & 15) * kVec;
      const int rr = r_first + kRows * k + row;
      if (row < kRows && rr <= r_last) {
        float M = kNone, L = 0.f, f[kWaves], acc[kVec];
#pragma unroll
        for (int w = 0; w < kWaves; ++w) M = fmaxf(M, lds.ml(w)[row].x);
#pragma unroll
        for (int w = 0; w < kWaves; ++w) {
          f[w] = __builtin_amdgcn_exp2f(lds.ml(w)[row].x - M);
          L += f[w] * lds.ml(w)[row].y;
        }
#pragma unroll
        for (int x = 0; x < kVec; ++x) {
          acc[x] = 0.f;
#pragma unroll
          for (int w = 0; w < kWaves; ++w) acc[x] += f[w] * lds.o(w)[row * (D + 4) + col + x];
        }
        const int64_t at = (sp.first + rr / a.G) * a.Hq + g * a.G + rr % a.G;
        if (P == kShared || n_parts > 1 || (P == kOwn && unit.first > 0)) {
          const int64_t prow = (int64_t)split * a.s.n_tokens * a.Hq + at;
          float* dst = a.o_part + prow * D + col;
#pragma unroll
          for (int x = 0; x < kVec; x += 4)
            *reinterpret_cast<f32x4*>(dst + x) = f32x4{acc[x], acc[x + 1], acc[x + 2], acc[x + 3]};
          if (col == 0) a.ml_part[prow] = make_float2(M, L);
        } else {
          const float inv = L > 0.f ? 1.f / L : 0.f;
          QT y[kVec];
#pragma unroll
          for (int x = 0; x < kVec; ++x) y[x] = (QT)(acc[x] * inv);
          char* dst = reinterpret_cast<char*>(static_cast<QT*>(a.out) + at * D + col);
          if constexpr (sizeof y == 16)
            *reinterpret_cast<uint4*>(dst) = *reinterpret_cast<const uint4*>(y);
          else
            *reinterpret_cast<uint2*>(dst) = *reinterpret_cast<const uint2*>(y);
        }
      }
    }
    if (rb + (int)gy < (rows + kRows * kBlocks - 1) / (kRows * kBlocks))
      __syncthreads();  // read, before the next block's K rows come
  }
}

template <int D, int T, bool kSmall, int kWaves, int P>
__global__ __launch_bounds__(64 * kWaves, 8 / kWaves) void page_rows_kernel(PageAttnArgs a) {
  using Lds = RowsLds<D, T, kWaves, 1>;
  __shared__ __attribute__((aligned(16))) char lds[Lds::kBytes];
  rows_part<D, T, kSmall, kWaves, P, 1>(a, blockIdx.x, blockIdx.y, gridDim.y, Lds{lds, nullptr});
}

// The numerators exp2(c1 s - m) of 32 keys in 16 / E + 2 steps, which are issued between
// MFMAs: step i scales the E logits of group i, takes the exponentials of group i - 1, and
// packs those of group i - 2 to bf16 pairs (P^T), which as rounded are added to the row's sums.
// The empty asm keeps a step in its place.
template <int E, int i>
__device__ __forceinline__ void rounded_step(f32x16& s, float c1, float m, float (&l)[2], u32x4 (&pb)[2]) {
  constexpr int kGroups = 16 / E;
  if constexpr (i < 0 || i > kGroups + 1) return;
#pragma unroll
  for (int e = 0; e < E; ++e) {
    if (i < kGroups) s[E * i + e] = fmaf(s[E * i + e], c1, -m);
    if (i >= 1 && i <= kGroups) s[E * (i - 1) + e] = __builtin_amdgcn_exp2f(s[E * (i - 1) + e]);
    const int v = E * (i - 2) + e;
    if (i < 2 || i > kGroups + 1) continue;
    if (v & 1) {
      uint32_t w = bf16_pair(s[v - 1], s[v]);
      asm volatile("" : "+v"(w));
      float& sum = l[v >> 1 & 1];
      sum = add_pair(w, sum);
      asm volatile("" : "+v"(sum));
      pb[v >> 3][(v & 7) >> 1] = w;
    }
  }
}

// Many rows: a workgroup owns 128 query rows (4 waves x 32) of one KV head and one split
// of their 64-key stages; K and V go through LDS as bf16, two stages of buffers:
//   S^T = K Q^T   MFMA 32x32x16 in two halves of 32 keys: a lane owns one row, 16 keys
//   O^T += V^T P^T  V^T by transposing LDS reads, P^T from the softmax registers
// bf16 rows go from memory straight to LDS, a page per load (8 keys of a stage lie in
// one page).  8-bit rows come through registers, a stage further ahead, and are written
// as bf16.  A row's reference is the maximum of the first keys that it sees; where it is
// followed later it moves by whole log2 units, so that numerators already rounded are scaled
// by a power of two and lose nothing.
// Bound by what the two waves of a SIMD issue beside their products: 32 MFMAs of 33 cycles a
// stage, three VALU instructions per logit and lane (one an exponential, 8 cycles) and the
// stage's own work, and the two pipes overlap in part only (two waves with 1 MFMA and 8 FMAs
// each, in a loop of these: 87 cycles where the MFMAs take 67 and the FMAs 47).  A wave
// alone issues an instruction in 5 cycles.  Hence no maximum in the loop (a chain from the
// products to the exponentials), pages found by the lanes for the 64 groups of 8 stages at
// once (for a stage: 258 us where this took 243), masks and their conditions in the stages
// that need some only (243 -> 235), and conversions beside the first run of products.
// k0 .. v1: kKeys * D numbers in LDS each.
template <int D, int T, int P>
__device__ __forceinline__ void tile_part(const PageAttnArgs& a, uint32_t bx, uint16_t* k0, uint16_t* k1, uint16_t* v0,
                                          uint16_t* v1) {
  using namespace tile;
  using St = Stage<D>;
  constexpr int kKeys = tile::kTile;
  constexpr bool kE4 = T == CKV_DTYPE_E4M3;
  // Blocks of rows that read the same keys (of one head and split: a stream) share an
  // XCD's L2: eight streams at a time, one per XCD.  Of the streams left over, 1, 2 or 4
  // have 8, 4 or 2 XCDs each, their blocks in turn; 3, 5, 6 or 7 are cut into eight runs of
  // blocks.  The last rows see the most keys: first.
  const uint32_t streams = a.Hkv * a.n_splits, xcd = bx & 7, idx = bx >> 3;
  const uint32_t whole = streams / 8 * a.n_blocks, rest = streams % 8;
  uint32_t stream, blk;
  if (idx < whole) {
    stream = idx / a.n_blocks * 8 + xcd;
    blk = idx % a.n_blocks;
  } else if (8 % rest == 0) {
    stream = streams - rest + xcd % rest;
    blk = (idx - whole) * (8 / rest) + xcd / rest;
  } else {
    const uint32_t run = (rest * a.n_blocks + 7) / 8, j = xcd * run + (idx - whole);
    stream = streams - rest + j / a.n_blocks;
    blk = j % a.n_blocks;
    if (idx - whole >= run) return;
  }
  if (stream >= streams || blk >= a.n_blocks) return;
  const int g = (int)(stream % a.Hkv), split = (int)(stream / a.Hkv);
  // n tokens of a sequence are ceil(n G / 128) blocks: numbered from floor(t G / 128) + 1 per
  // sequence before, t its first token
  const auto block_start = [&](int q) { return unit_token<P>(a, q) * a.G / kBlockRows + q; };
  const int64_t block = a.n_blocks - 1 - blk;
  const int b = find_seq(n_units<P>(a), block, block_start);
  if (b < 0) return;
  const Unit unit = unit_of<P>(a, b);
  const SeqSpan& sp = unit.sp;
  const int rb = (int)(block - block_start(b));
  if ((int64_t)rb * kBlockRows >= (int64_t)sp.count * a.G) return;
  const int lane = threadIdx.x & 63, half = lane >> 5;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int32_t* tab = unit.tab;
  const int kv_end = unit.kv_end;
  const int rows = sp.count * a.G, r_first = rb * kBlockRows, r_last = min(rows, r_first + kBlockRows) - 1;
  const int p_base = unit.p_base;
  const int p0 = p_base + r_first / a.G, p1 = p_base + r_last / a.G;
  const int all_steps = (groups_of<P>(a, p_base, p_base + sp.count - 1, unit.first, kv_end).n + 7) / 8;
  const int n_parts = parts_of<P>(a, unit, all_steps, a.slice);
  if ((P != kWhole || a.n_splits > 1) && split == 0 && g == 0)
    for (int i = r_first / a.G + (int)threadIdx.x; i <= r_last / a.G; i += 256)
      a.n_parts[sp.first + i] = parts_note<P>(unit, n_parts);
  if (split >= n_parts) return;
  const Groups groups = groups_of<P>(a, p0, p1, unit.first, kv_end);  // a stage: 8 of them
  const int stages = (groups.n + 7) / 8;
  const int per = stages / n_parts, over = stages % n_parts;  // the first `over` splits: one more
  const int begin = split * per + min(split, over), end = begin + per + (split < over ? 1 : 0);

  // this lane's row
  const int row = r_first + wave * kWaveRows + (lane & 31);
  const bool row_ok = row <= r_last;
  const int rt = (row_ok ? row : r_last) / a.G;
  const int p = p_base + rt;  // (a row past the last goes like the last one, and is not written)
  const int64_t out_row = (sp.first + rt) * a.Hq + g * a.G + (row_ok ? row : r_last) % a.G;
  bf16x8 qf[D / 16];
  {
    const __bf16* q = static_cast<const __bf16*>(a.q) + out_row * D + 8 * half;
#pragma unroll
    for (int i = 0; i < D / 16; ++i) qf[i] = *reinterpret_cast<const bf16x8*>(q + 16 * i);
  }

  // The pages of 8 stages at a time: lane l has group l of them, its table entry in the 8
  // stages before, then where it begins in the pool (a missing page: page 0) and its scale
  // bytes.  A load takes its group's by readlane.
  const int row_bytes = a.Hkv * D * Elem<T>::kBytes;
  struct Eight {
    int next;        // entry of group l of the 8 stages after
    int64_t of;
    uint64_t there;  // bit l: group l's page is there
    uint32_t ks, vs;
  };
  auto group_pos = [&](int st) __attribute__((always_inline)) { return groups.pos(min(8 * st + lane, 8 * end - 1)); };
  auto entries = [&](int st) __attribute__((always_inline)) {
    const int pos = group_pos(st);
    return entry_of(a, tab, a.log2c >= 0 ? pos >> a.log2c : (int)((uint32_t)pos / (uint32_t)a.c));
  };
  auto enter = [&](int st, Eight& x) __attribute__((always_inline)) {  // the 8 stages from st on
    const int pos = group_pos(st), r = a.log2c >= 0 ? pos & (a.c - 1) : (int)((uint32_t)pos % (uint32_t)a.c);
    const bool ok = names_page(a, x.next);
    const int page = ok ? x.next : 0;
    x.of = (int64_t)page * a.page_stride + (int64_t)r * row_bytes;
    x.there = __ballot(ok);
    if constexpr (kE4) {
      x.ks = a.k_scale[(int64_t)page * a.Hkv + g];
      x.vs = a.v_scale[(int64_t)page * a.Hkv + g];
    }
    x.next = entries(st + 8);
  };
  // Before a stage's loads, stages in order; gives the bits of its 8 pages.
  auto at_stage = [&](int st, Eight& x) __attribute__((always_inline)) {
    const int i = (st - begin) & 7;
    if (i == 0) enter(st, x);
    return (uint32_t)(x.there >> (8 * i)) & 0xffu;
  };
  auto place = [&](const Eight& x, int st, int group) __attribute__((always_inline)) {
    const int l = 8 * ((st - begin) & 7) + group;
    return (int64_t)((uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)(x.of >> 32), l) << 32 |
                     (uint32_t)__builtin_amdgcn_readlane((int)x.of, l));
  };

  // bf16: this lane's byte of the rows that a load moves (the LDS permutation undone)
  const int key0 = wave * St::kRowsPerLoad + lane / St::kSegs;
  const uint32_t rcol = (uint32_t)(((wave * St::kRowsPerLoad & 7) + lane / St::kSegs) * row_bytes);
  const uint32_t kcol = rcol + (uint32_t)(2 * (g * D + ((lane % St::kSegs ^ k_swz<D>(key0)) << 3)));
  const uint32_t vcol = rcol + (uint32_t)(2 * (g * D + ((lane % St::kSegs ^ v_swz<D>(key0)) << 3)));
  auto load_direct = [&](const Eight& x, int st, uint16_t* dk, uint16_t* dv) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < St::kPer; ++i) {
      const int key = i * St::kKeyStep + wave * St::kRowsPerLoad;
      const int64_t off = place(x, st, key >> 3);
      buffer_to_lds(raw_rsrc(a.k + off, 0xffffffffu), kcol, 0, dk + key * D);
      buffer_to_lds(raw_rsrc(a.v + off, 0xffffffffu), vcol, 0, dv + key * D);
    }
  };
  // 8 bits: 16 codes of a row per lane and load, kLoads loads of kERows rows per wave
  constexpr int kELanes = D / 16, kERows = 64 / kELanes, kLoads = kKeys / (4 * kERows);
  struct Codes {
    u32x4 k[kLoads], v[kLoads];
  };
  const uint32_t ecol = (uint32_t)((lane / kELanes & 7) * row_bytes + g * D + lane % kELanes * 16);
  auto load_codes = [&](const Eight& e, int st, Codes& x) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < kLoads; ++i) {
      const int group = (4 * i + wave) * kERows >> 3;
      if constexpr (kERows == 8) {
        const int64_t off = place(e, st, group);
        x.k[i] = __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(raw_rsrc(a.k + off, 0xffffffffu), ecol, 0, 0));
        x.v[i] = __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(raw_rsrc(a.v + off, 0xffffffffu), ecol, 0, 0));
      } else {  // (at D = 64 a load has rows of two groups)
        const int64_t lo = place(e, st, group), hi = place(e, st, group + 1), off = (lane >> 5 ? hi : lo) + ecol;
        x.k[i] = *reinterpret_cast<const u32x4*>(a.k + off);
        x.v[i] = *reinterpret_cast<const u32x4*>(a.v + off);
      }
    }
  };
  // Piece n < 4 kLoads of a stage's codes as bf16 in LDS: half n % 2 of load n / 4, K then V.
  auto write_codes = [&](auto n, const Eight& e, int st, const Codes& x, uint16_t* dk, uint16_t* dv)
      __attribute__((always_inline)) {
    constexpr int i = n / 4, kv = n / 2 % 2, h = n % 2;
    const int first = (4 * i + wave) * kERows, key = first + lane / kELanes;
    const int l = 8 * ((st - begin) & 7) + (first >> 3);
    const uint32_t bytes = kv ? e.vs : e.ks;
    uint32_t byte = (uint32_t)__builtin_amdgcn_readlane(bytes, l);
    if constexpr (kERows == 16) {
      const uint32_t up = (uint32_t)__builtin_amdgcn_readlane(bytes, l + 1);
      byte = lane >> 5 ? up : byte;
    }
    const int seg = (2 * (lane % kELanes) + h) ^ (kv ? v_swz<D>(key) : k_swz<D>(key));
    const u32x4& w = kv ? x.v[i] : x.k[i];
    *reinterpret_cast<bf16x8*>((kv ? dv : dk) + key * D + (seg << 3)) =
        bf16_of_codes(w[2 * h], w[2 * h + 1], scale_of(byte));
  };
  // finite_codes for what this lane has written of a stage, where one of the pages of its 8 has such
  // a byte: codes past what bf16 holds are infinities by now, and become 240 * 2^120.  (On the codes
  // in registers, for which there is no room, the long prefill takes 2% more, so 1%.)
  auto any_top = [&](const Eight& x) __attribute__((always_inline)) { return __any(max(x.ks, x.vs) >= kTopByte) != 0; };
  auto keep_finite = [&](uint16_t* dk, uint16_t* dv) __attribute__((always_inline)) {
#pragma unroll 1
    for (int n = 0; n < 4 * kLoads; ++n) {
      const int key = (4 * (n / 4) + wave) * kERows + lane / kELanes;
      const int seg = (2 * (lane % kELanes) + n % 2) ^ (n & 2 ? v_swz<D>(key) : k_swz<D>(key));
      u32x4& w = *reinterpret_cast<u32x4*>((n & 2 ? dv : dk) + key * D + (seg << 3));
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const uint32_t x = w[j], y = (x & 0x7fffu) == 0x7f80u ? x - 0x10u : x;
        w[j] = (y & 0x7fff0000u) == 0x7f800000u ? y - 0x100000u : y;
      }
    }
  };

  // byte offsets of the operand reads (the same for every stage)
  const int kr = kappa(lane & 31);
  const uint32_t kfo = 2 * (kr * D + ((half ^ k_swz<D>(kr)) << 3));
  const int s16 = lane & 15, g4 = (lane >> 4) & 1;
  const uint32_t voff = 2 * (v_off<D>(8 * half + (s16 >> 2), 2 * g4 + ((s16 & 3) >> 1)) + 4 * (s16 & 1));

  constexpr int kG = D / 16;  // MFMAs of one 32-key product, and of one O update
  constexpr int kE = 256 / D; // logits per numerator step: kG + 2 steps per half
  static_assert(!kE4 || 4 * kLoads == kG);
  f32x16 o[D / 32];
  float l[2], ref;

  // Stages all of whose keys every row sees, as far as their pages are there, take no masks:
  // `n_clear` of them from `clear_from` on, past the sinks' groups, in the window of the last
  // row and below the position of the first one, but for the split's first stage (in whose
  // keys the reference is looked for).
  const int whole_groups = max(min(p0 + 1, kv_end), 0) >> 3;
  const int below = whole_groups <= groups.n_sink ? whole_groups : groups.n_sink + max(whole_groups - groups.first, 0);
  const int in_window = a.window > 0 ? max(groups.n_sink, groups.n_sink + ((p1 - a.window) >> 3) - groups.first + 1) : 0;
  const int clear_from = max((in_window + 7) >> 3, begin + 1), n_clear = max((below >> 3) - clear_from, 0);

  // -inf where this lane's row must not see a key of half `sub` of stage st: keys past its
  // own position or the sequence's end, keys before its window, keys of a missing page
  // (`there`: bit i, the page of the stage's group i), as far as the stage has any.
  // Registers 8 i .. + 7 hold the keys of group 4 sub + 2 i + half.
  const int upper = min(p, kv_end - 1);
  auto mask = [&](int st, int sub, uint32_t there, bool up, bool low, f32x16& s) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const int group = 4 * sub + 2 * i + half, pos = groups.pos(8 * st + group);
      if (up) {
        const int most = upper - pos;
#pragma unroll
        for (int v = 0; v < 8; ++v) s[8 * i + v] = v <= most ? s[8 * i + v] : -INFINITY;
      }
      if (low) {
        const int least = p - a.window - pos, first = a.sinks - pos;  // sees above, and below
#pragma unroll
        for (int v = 0; v < 8; ++v) s[8 * i + v] = v > least || v < first ? s[8 * i + v] : -INFINITY;
      }
      if (there != 0xffu && !(there >> group & 1)) {
#pragma unroll
        for (int v = 0; v < 8; ++v) s[8 * i + v] = -INFINITY;
      }
    }
  };
  float c1;  // of the logits: a.c1, or 1 where they are scaled already
  // The reference follows the logits of a half.  `before`: the half whose numerators are
  // under way, pb where they go; of its groups of kE the last has only its exponents, the
  // one before it is not yet added or packed.
  auto follow = [&](const f32x16& s, f32x16* before, u32x4* pb) __attribute__((always_inline)) {
    float mx = max16(s) * c1;
    if (!__any(mx > ref + kSlack)) return;
    mx = fmaxf(mx, partner_f(mx));
    // (a rise of 2^23 and more is itself rounded, and leaves nothing of what was before)
    const float rise = fmaxf(ceilf(mx - ref), 0.f);
    const float to = ref == kNone ? fmaxf(mx, kNone) : rise < kFar ? ref + rise : mx;
    const float by = ref - to, f = __builtin_amdgcn_exp2f(by);
    ref = to;
    l[0] *= f;
    l[1] *= f;
#pragma unroll
    for (int db = 0; db < D / 32; ++db)
#pragma unroll
      for (int v = 0; v < 16; ++v) o[db][v] *= f;
    if (!before) return;
#pragma unroll
    for (int e = 0; e < kE; ++e) {
      (*before)[kE * (kG - 1) + e] += by;
      (*before)[kE * (kG - 2) + e] *= f;
    }
#pragma unroll
    for (int i = 0; i < kE * (kG - 2) / 2; ++i) {
      const uint32_t w = pb[i >> 2][i & 3];
      const uint32_t lo = __float_as_uint(__uint_as_float(w << 16) * f);
      const uint32_t hi = __float_as_uint(__uint_as_float(w & 0xffff0000u) * f);
      pb[i >> 2][i & 3] = (hi & 0xffff0000u) | lo >> 16;
    }
  };

  auto scale = [&](f32x16& s) __attribute__((always_inline)) {
#pragma unroll
    for (int v = 0; v < 16; ++v) s[v] *= a.c1;
  };

  // The reference is looked at in the first stage and in those where some row sees only a
  // part: the first keys that a row sees are in one of them.  In the others it is left: only
  // a logit 120 log2 units above all earlier ones does harm, which the sums then show, and
  // the split is done again with every stage looked at.  So it is where a reference is past kFar, the
  // logits scaled and rounded before the exponents.
  for (bool look = false;; look = true) {
    c1 = __uint_as_float(__builtin_amdgcn_readfirstlane(__float_as_uint(look ? 1.f : a.c1)));
#pragma unroll
    for (int db = 0; db < D / 32; ++db)
#pragma unroll
      for (int v = 0; v < 16; ++v) o[db][v] = 0.f;
    l[0] = l[1] = 0.f;
    ref = kNone;
    if (begin < end) {
      Eight pages;
      pages.next = entries(begin);
      // the bits of the current stage's pages and of the next one's
      uint32_t there = at_stage(begin, pages), there1 = 0xffu;
      Codes codes;
      if constexpr (kE4) {
        load_codes(pages, begin, codes);
        static_for<4 * kLoads>([&](auto n) { write_codes(n, pages, begin, codes, k0, v0); });
        if (any_top(pages)) keep_finite(k0, v0);
        if (begin + 1 < end) {
          there1 = at_stage(begin + 1, pages);
          load_codes(pages, begin + 1, codes);
        }
      } else {
        load_direct(pages, begin, k0, v0);
      }
      stage_barrier();
      bf16x8 ka[kG];  // K fragments of the current stage's first 32 keys
#pragma unroll
      for (int i = 0; i < kG; ++i) ka[i] = read_k<D>(k0, kfo, 0, i);

      auto stage = [&](int st, uint16_t* lk, uint16_t* lv, uint16_t* nk, uint16_t* nv)
          __attribute__((always_inline)) {
        uint32_t ko = kfo, vo = voff;
        asm volatile("" : "+v"(ko), "+v"(vo));
        // what some row of the block must not see: keys past its position, keys before its
        // window; and V rows that no row sees
        const bool clear = (uint32_t)(st - clear_from) < (uint32_t)n_clear && there == 0xffu;
        bool up = false, low = false, hide = false;
        if (!clear) {
          const int pos0 = groups.pos(8 * st), last = groups.pos(8 * st + 7) + 8;
          const bool sinks = 8 * st < groups.n_sink;  // the first groups are of the sinks
          up = last > min(p0 + 1, kv_end);
          low = a.window > 0 && (sinks || pos0 <= p1 - a.window) && last > a.sinks;
          hide = there != 0xffu || last > min(p1 + 1, kv_end) ||
                 (a.window > 0 && (sinks || pos0 <= p0 - a.window) && last > a.sinks);
        }
        const bool top = kE4 && any_top(pages);  // (of the next stage's eight)
        const bool check = !clear || look || top;
        uint32_t after = 0xffu;
        if constexpr (!kE4)
          if (st + 1 < end) {
            after = at_stage(st + 1, pages);
            load_direct(pages, st + 1, nk, nv);
          }
        if (hide) {
          // a weight of 0 does not undo a NaN: V rows that no query of the block sees are cleared
          const int key = (int)threadIdx.x >> 2, pos = groups.pos(8 * st + (key >> 3)) + (key & 7);  // four threads a row
          if (!((there >> (key >> 3) & 1) && pos < kv_end && pos <= p1 &&
                (a.window <= 0 || pos > p0 - a.window || pos < a.sinks)))
#pragma unroll
            for (int i = 0; i < D / 32; ++i)
              *reinterpret_cast<u32x4*>(lv + key * D + ((int)(threadIdx.x & 3) * (D / 32) + i) * 8) = u32x4{0u, 0u, 0u, 0u};
          __syncthreads();
        }
        bf16x8 kb[kG], va[2][D / 32], vb[2][D / 32];
        f32x16 s0, s1;
        u32x4 p0b[2], p1b[2];
#pragma unroll
        for (int v = 0; v < 16; ++v) s0[v] = s1[v] = 0.f;
        __builtin_amdgcn_sched_barrier(0);
        // The runs with numerators beside the products go before the other wave's runs of
        // products alone (512 tokens on 32K in 8 bits: 276 -> 264 us).
        __builtin_amdgcn_s_setprio(0);
        static_for<kG>([&](auto i) __attribute__((always_inline)) {
          kb[i] = read_k<D>(lk, ko, 1, i);
          s0 = __builtin_amdgcn_mfma_f32_32x32x16_bf16(ka[i], qf[i], s0, 0, 0, 0);
          // (kG pieces: the stage after the last one is written as well, and not used)
          if constexpr (kE4) write_codes(i, pages, st + 1, codes, nk, nv);
          __builtin_amdgcn_sched_barrier(0);
        });
        __builtin_amdgcn_s_setprio(1);
        if constexpr (kE4)
          if (st + 2 < end) {
            after = at_stage(st + 2, pages);
            load_codes(pages, st + 2, codes);
          }
        if (check) {
          if constexpr (kE4)
            if (top) keep_finite(nk, nv);
          if (look) scale(s0);
          mask(st, 0, there, up, low, s0);
          follow(s0, nullptr, nullptr);
        }
        __builtin_amdgcn_sched_barrier(0);
        static_for<kG>([&](auto i) __attribute__((always_inline)) {
          constexpr int kk = i / (D / 32), db = i % (D / 32);
          va[kk][db] = read_v<D>(lv, vo, 0, kk, db);
          s1 = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kb[i], qf[i], s1, 0, 0, 0);
          rounded_step<kE, i>(s0, c1, ref, l, p0b);
          __builtin_amdgcn_sched_barrier(0);
        });
        if (check) {
          if (look) scale(s1);
          mask(st, 1, there, up, low, s1);
          follow(s1, &s0, p0b);
        }
        __builtin_amdgcn_sched_barrier(0);
        static_for<kG>([&](auto i) __attribute__((always_inline)) {
          constexpr int kk = i / (D / 32), db = i % (D / 32);
          vb[kk][db] = read_v<D>(lv, vo, 1, kk, db);
          if constexpr (i < 2) rounded_step<kE, kG + i>(s0, c1, ref, l, p0b);
          o[db] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(va[kk][db], __builtin_bit_cast(bf16x8, p0b[kk]),
                                                          o[db], 0, 0, 0);
          rounded_step<kE, i>(s1, c1, ref, l, p1b);
          __builtin_amdgcn_sched_barrier(0);
        });
        if constexpr (kE4) {  // the next stage's rows are written; loads stay in flight
          __builtin_amdgcn_fence(__ATOMIC_RELEASE, "workgroup", "local");
          __builtin_amdgcn_s_barrier();
          __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "workgroup", "local");
        } else {
          stage_barrier();  // the next stage has landed; this one's buffers are read
        }
        __builtin_amdgcn_sched_barrier(0);
        __builtin_amdgcn_s_setprio(0);
        static_for<kG>([&](auto i) __attribute__((always_inline)) {
          constexpr int kk = i / (D / 32), db = i % (D / 32);
          ka[i] = read_k<D>(nk, ko, 0, i);  // (after the last stage: read and not used)
          if constexpr (i < 2) rounded_step<kE, kG + i>(s1, c1, ref, l, p1b);
          o[db] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vb[kk][db], __builtin_bit_cast(bf16x8, p1b[kk]),
                                                          o[db], 0, 0, 0);
          __builtin_amdgcn_sched_barrier(0);
        });
        there = kE4 ? there1 : after;
        there1 = after;
      };
      for (int st = begin; st < end; st += 2) {
        stage(st, k0, v0, k1, v1);
        if (st + 1 >= end) break;
        stage(st + 1, k1, v1, k0, v0);
      }
    }
    l[0] += l[1];
    l[0] += partner_f(l[0]);
    if (look) break;
    float any[4] = {0.f, 0.f, 0.f, 0.f};  // (a sum over the outputs is inf or NaN if one of them is)
#pragma unroll
    for (int db = 0; db < D / 32; ++db)
#pragma unroll
      for (int v = 0; v < 16; ++v) any[v & 3] += o[db][v];
    const uint32_t total = __float_as_uint((any[0] + any[1]) + (any[2] + any[3]));
    const bool bad = (total & 0x7f800000u) == 0x7f800000u ||
                     (__float_as_uint(l[0]) & 0x7fffffffu) > __float_as_uint(0x1p120f) ||
                     (fabsf(ref) >= kFar && ref != kNone);
    if (!__builtin_amdgcn_readfirstlane(__syncthreads_or(bad))) break;
  }

  // o[db][v] holds d = 32*db + 8*(v/4) + 4*half + v%4 of this lane's row
  if (P == kShared || n_parts > 1 || (P == kOwn && unit.first > 0)) {
    if (!row_ok) return;
    // The sum in [1, 2), so that outputs are of V's size whatever the reference was; but for one past
    // kFar, which has no room for the change and was followed to the maximum.
    const int e = l[0] > 0.f && fabsf(ref) < kFar ? (int)(__float_as_uint(l[0]) >> 23) - 127 : 0;
    const float f = __uint_as_float((uint32_t)(127 - e) << 23);
    const int64_t prow = (int64_t)split * a.s.n_tokens * a.Hq + out_row;
    float* dst = a.o_part + prow * D + 4 * half;
#pragma unroll
    for (int db = 0; db < D / 32; ++db)
#pragma unroll
      for (int q = 0; q < 4; ++q)
        *reinterpret_cast<f32x4*>(dst + 32 * db + 8 * q) =
            f32x4{o[db][4 * q] * f, o[db][4 * q + 1] * f, o[db][4 * q + 2] * f, o[db][4 * q + 3] * f};
    if (half == 0) a.ml_part[prow] = make_float2(ref + (float)e, l[0] * f);
    return;
  }
  // Output rows through LDS, so that a store is a whole 16-byte piece of a row and 16 lanes
  // cover a row: the wave's rows go to a stage buffer of its own, which no wave reads for
  // its values any more.
  const float inv = l[0] > 0.f ? 1.f / l[0] : 0.f;
  constexpr int kRow = D + 8, kSegs = D / 8, kRowsPerPass = 64 / kSegs;
  uint16_t* rows_of = wave == 0 ? k0 : wave == 1 ? k1 : wave == 2 ? v0 : v1;
#pragma unroll
  for (int db = 0; db < D / 32; ++db)
#pragma unroll
    for (int q = 0; q < 4; ++q)
      *reinterpret_cast<uint2*>(rows_of + (lane & 31) * kRow + 32 * db + 8 * q + 4 * half) =
          make_uint2(bf16_pair(o[db][4 * q] * inv, o[db][4 * q + 1] * inv),
                     bf16_pair(o[db][4 * q + 2] * inv, o[db][4 * q + 3] * inv));
#pragma unroll
  for (int r0 = 0; r0 < kWaveRows; r0 += kRowsPerPass) {
    const int rr = r0 + lane / kSegs;
    const uint4 x = *reinterpret_cast<const uint4*>(rows_of + rr * kRow + lane % kSegs * 8);
    const int64_t at = __shfl(out_row, rr);
    if (r_first + wave * kWaveRows + rr <= r_last)
      *reinterpret_cast<uint4*>(static_cast<uint16_t*>(a.out) + at * D + lane % kSegs * 8) = x;
  }
}

template <int D, int T, int P>
__global__ __launch_bounds__(256, 2) void page_tile_kernel(PageAttnArgs a) {
  __shared__ __attribute__((aligned(16))) uint16_t k0[tile::kTile * D], k1[tile::kTile * D];
  __shared__ __attribute__((aligned(16))) uint16_t v0[tile::kTile * D], v1[tile::kTile * D];
  tile_part<D, T, P>(a, blockIdx.x, k0, k1, v0, v1);
}

// The shared keys and the sequences' own in one launch, the shared ones first: the own keys, few
// and read by workgroups of a few steps each, then fill what the others leave idle (48 sequences on
// a document: two launches 55.5 us a layer, one 45.8; eight groups of eight 77 and 67).
// Bound by latency where a group has few rows: a wave has one step of keys under way, 2,048 waves 16
// MB, and they wait for 7,000 cycles a step.
// kBlocks: of rows_part for the shared keys; 0: tile_part, in whose memory the own ones' waves
// have a buffer each.
struct TileRowsLds {
  char* mine;  // this wave's
  uint16_t *k0, *k1, *v0, *v1;
  float2* sums;
  uint16_t* q;
  __device__ __forceinline__ char* mine_k(int) const { return mine; }
  __device__ __forceinline__ float* mine_o(int) const { return reinterpret_cast<float*>(mine); }
  __device__ __forceinline__ float* o(int w) const {  // (w: a constant)
    return reinterpret_cast<float*>(w == 0 ? k0 : w == 1 ? k1 : w == 2 ? v0 : v1);
  }
  __device__ __forceinline__ float2* ml(int w) const { return sums + w * kRows; }
};
template <int D, int T, bool kSmall, int kBlocks>
__global__ __launch_bounds__(256, 2) void page_parts_kernel(PageAttnArgs shared, PageAttnArgs own, uint32_t shared_x,
                                                            uint32_t shared_y, uint32_t own_x, uint32_t own_y) {
  // (x is a multiple of 8: the XCDs stay in turn)
  const bool is_shared = blockIdx.x < shared_x * shared_y;
  const uint32_t i = is_shared ? blockIdx.x : blockIdx.x - shared_x * shared_y;
  if constexpr (kBlocks == 0) {
    static_assert(kTile * D * Elem<T>::kBytes <= tile::kTile * D * 2 && kRows * (D + 4) * 4 <= tile::kTile * D * 2);
    __shared__ __attribute__((aligned(16))) uint16_t k0[tile::kTile * D], k1[tile::kTile * D];
    __shared__ __attribute__((aligned(16))) uint16_t v0[tile::kTile * D], v1[tile::kTile * D];
    __shared__ float2 sums[4 * kRows];
    if (is_shared)
      tile_part<D, T, kShared>(shared, i, k0, k1, v0, v1);
    else {
      const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
      uint16_t* const mine = wave == 0 ? k0 : wave == 1 ? k1 : wave == 2 ? v0 : v1;
      rows_part<D, T, kSmall, 4, kOwn, 1>(own, i % own_x, i / own_x, own_y,
                                          TileRowsLds{reinterpret_cast<char*>(mine), k0, k1, v0, v1, sums, nullptr});
    }
  } else {
    using Lds = RowsLds<D, T, 4, kBlocks>;
    using OwnLds = RowsLds<D, T, 4, 1>;
    __shared__ __attribute__((aligned(16))) char lds[Lds::kBytes];
    __shared__ __attribute__((aligned(16))) uint16_t q[Lds::kQ / 2 + 8];
    if (is_shared)
      rows_part<D, T, kSmall, 4, kShared, kBlocks>(shared, i % shared_x, i / shared_x, shared_y, Lds{lds, q});
    else
      rows_part<D, T, kSmall, 4, kOwn, 1>(own, i % own_x, i / own_x, own_y, OwnLds{lds, nullptr});
  }
}

// Joins the splits of a row: kGroups groups of D / 4 threads take them in turn, 4 elements
// a thread, and meet in LDS, all in a fixed order.  One group (and several rows per
// workgroup) up to kJoinBatch splits, whose loads are all in flight together; else the
// whole workgroup.
// kParts: the first `shared_splits` places are of the shared keys, the others of the sequences' own.
constexpr int kJoinBatch = 8;
template <int D, class QT, int kGroups, bool kParts>
__global__ __launch_bounds__(256) void page_combine_kernel(PageAttnArgs a) {
  constexpr int kCols = D / 4, kRowsPer = 256 / kCols / kGroups;
  const int64_t n_rows = a.s.n_tokens * a.Hq;
  int64_t row = (int64_t)blockIdx.x * kRowsPer + threadIdx.x / (kCols * kGroups);
  // A workgroup that has one row leaves as a whole; of several rows, joined in groups, all stay.
  constexpr bool kStay = kGroups > 1 && kRowsPer > 1;
  bool mine = row < n_rows;
  if (!kStay && !mine) return;
  if (kStay) row = min(row, n_rows - 1);
  const int tok = (int)row / a.Hq;  // (at most 2^26 rows)
  const int col = threadIdx.x % kCols * 4, grp = threadIdx.x / kCols % kGroups;
  float2 ml[kJoinBatch];
  f32x4 x[kJoinBatch];
  auto load = [&](int s0, int n) __attribute__((always_inline)) {
#pragma unroll
    for (int k = 0; k < kJoinBatch; ++k) {
      const int64_t at = (int64_t)min(s0 + k * kGroups, n - 1) * n_rows + row;
      ml[k] = a.ml_part[at];
      x[k] = *reinterpret_cast<const f32x4*>(a.o_part + at * D + col);
    }
  };
  // the first splits come together with the number of them (those past it hold anything; of parts, the
  // places that few rows have come after it)
  const int usual = kParts ? a.first_places : a.n_splits;
  load(grp, usual);
  const int first_tok = a.s.tok_off[0], end_tok = a.s.tok_off[a.s.n_seqs];
  int n_parts, n_shared = 0, own_from = 0;  // places [0, n_shared) and [own_from, n_parts) are this row's
  if constexpr (kParts) {
    const int own = a.n_parts[tok], shared = a.shared_parts[tok];
    own_from = a.shared_splits;
    n_parts = own_from + min(own & (kAfterShared - 1), a.n_splits - own_from);
    n_shared = own & kAfterShared ? min(shared, own_from) : 0;
    if (tok < first_tok || tok >= end_tok || (!(own & kAfterShared) && n_parts - own_from <= 1)) mine = false;
    if (!kStay && !mine) return;
  } else {
    n_parts = min(a.n_parts[tok], a.n_splits);
    if (tok < first_tok || tok >= end_tok || n_parts <= 1) return;  // of no sequence, or written already
  }
  float M = kNone, L = 0.f;
  f32x4 acc{0.f, 0.f, 0.f, 0.f};
  for (int s0 = grp; s0 < n_parts; s0 += kGroups * kJoinBatch) {
    if (s0 != grp || (kParts && n_parts > usual)) load(s0, n_parts);
    float to = M;
#pragma unroll
    for (int k = 0; k < kJoinBatch; ++k) {
      const int at = s0 + k * kGroups;
      if (at >= n_parts || (kParts && at >= n_shared && at < own_from)) {
        ml[k] = make_float2(kNone, 0.f);
        x[k] = f32x4{0.f, 0.f, 0.f, 0.f};
      }
      to = fmaxf(to, ml[k].x);
    }
    const float f = __builtin_amdgcn_exp2f(M - to);
    M = to;
    L *= f;
    acc *= f;
#pragma unroll
    for (int k = 0; k < kJoinBatch; ++k) {
      const float w = __builtin_amdgcn_exp2f(ml[k].x - to);
      L += ml[k].y * w;
      acc += x[k] * w;  // (a split that saw no key wrote zeros)
    }
  }
  if constexpr (kGroups > 1) {
    __shared__ f32x4 part[kRowsPer][kGroups][kCols];
    __shared__ float2 part_ml[kRowsPer][kGroups];
    const int at = threadIdx.x / (kCols * kGroups), c = threadIdx.x % kCols;
    part[at][grp][c] = acc;
    if (col == 0) part_ml[at][grp] = make_float2(M, L);
    __syncthreads();
    if (grp > 0 || (kRowsPer > 1 && !mine)) return;
#pragma unroll
    for (int k = 1; k < kGroups; ++k) M = fmaxf(M, part_ml[at][k].x);
    L = 0.f;
    acc = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int k = 0; k < kGroups; ++k) {
      const float w = __builtin_amdgcn_exp2f(part_ml[at][k].x - M);
      L += part_ml[at][k].y * w;
      acc += part[at][k][c] * w;
    }
  }
  const float inv = L > 0.f ? 1.f / L : 0.f;
  QT y[4];
#pragma unroll
  for (int k = 0; k < 4; ++k) y[k] = (QT)(acc[k] * inv);
  char* dst = reinterpret_cast<char*>(static_cast<QT*>(a.out) + row * D + col);
  if constexpr (sizeof y == 16)
    *reinterpret_cast<uint4*>(dst) = *reinterpret_cast<const uint4*>(y);
  else
    *reinterpret_cast<uint2*>(dst) = *reinterpret_cast<const uint2*>(y);
}

constexpr int kFewRows = 32;  // rows of a sequence that page_rows_kernel takes (top of the file)
// Workgroups that read shared keys for 17 to 48 rows: most of the 512 that run at once, which leaves
// room for the sequences' own keys (eight groups of eight in 8 bits, 8,192 to 16,384 shared tokens: 320
// of them 68.7 us, 384 63.7, 416 59.3, 448 61.7, 512 68.5; in bf16 28 heads on 4, groups of four: 52.5,
// 49.4, 49.2, 51.4, 52.9).
constexpr int64_t kSharedBlocks = 416;
// Bytes of shared pages read again and again that are worth the parts' launch and join.  Decoding, 28 heads
// on 4 in bf16: 4 sequences on 4,000 tokens (25 MB) apart 12.7 us, in parts 14.7; 2 groups of 2 on 8,000 in 8
// bits, 40 heads on 8 (33 MB) 18.6, 17.2; 4 on 8,000 (49 MB) 18.6, 15.1; 8 on 4,000 (57 MB) 18.7, 15.2; but 16 on
// 2,000 (61 MB) 13.1, 15.5: bytes alone do not part many short sequences from these.  Prompts gain by fuller
// tiles only: 8 of 30 tokens on 4,000 (57 MB) 34.7, 39.6; 8 of 30 on 16,000 in 8 bits (114 MB) 73.9, 69.7; 16 of 8
// on 16,000 (491 MB) 79.1, 45.2.
constexpr int64_t kWorthParts = int64_t(40) << 20, kWorthPrompts = int64_t(96) << 20;

// Own keys behind shared ones: places for the longest sequence as far as they are this many workgroups (those of
// 128-row tiles fewer), from 16 steps a place on; the join loads the usual ones with the first round.  48 sequences
// on 30,011 tokens beside one of 30,000 in no group, 28 heads on 4 in bf16: 199 us with the places of the others,
// 113 with 512 workgroups, 71 with 1,024, 82 with 2,048, each by itself 163; without that one 49.7, 50.0, 50.5, 50.8.
// 8 prompts of 48 on 32,768 in 8 bits beside two of 20,000: 580, with 256 of tiles 403, 384 347, 512 328, each by
// itself 314; 8 of 30 on 16,000 in bf16 alone 82.4, 82.7, 82.7, 86.1.
constexpr int64_t kOwnWorkgroups = 1024, kOwnTiles = 384;
constexpr int kOwnSlice = 16;

struct PageAttnPlan {
  bool wide;       // page_tile_kernel
  int n_splits, slice;
  int row_blocks;  // page_rows_kernel: grid y, and its kBlocks
  int per_block;
  int n_wgs;
  int64_t blocks;  // page_tile_kernel: blocks of rows, at most
  size_t off_ml, off_n, bytes;
};

// About the most rows' tokens of one of n_units units: some unit has at least the mean,
// whatever the caller says (0: not known).
int64_t most_tokens(int64_t said, int64_t n_tokens, int n_units) {
  return said > 0 ? std::min(std::max<int64_t>(said, ceil_div(n_tokens, std::max(n_units, 1))), n_tokens) : n_tokens;
}
int64_t longest(const ckv_page_pool* pool, const ckv_page_batch* b) {
  const int64_t len = (int64_t)b->max_pages * pool->page_size;
  return b->max_len > 0 ? std::min<int64_t>(len, b->max_len) : len;
}

// The launch for n_units units of up to `most` of the n_tokens tokens, which see up to `len`
// keys; tile_blocks: about how many blocks of 128 rows they are; few_rows: rows of a unit up to which
// page_rows_kernel's steps are taken.
PageAttnPlan plan_units(const ckv_page_pool* pool, int Hq, int n_units, int64_t n_tokens, int64_t most, int64_t len,
                        int64_t tile_blocks, int window, int sinks, int few_rows, bool shared, int64_t split_steps = 16) {
  PageAttnPlan p{};
  const int G = Hq / pool->n_kv_heads;
  // (both sides: top of the file; one kernel for the call, by its longest sequence)
  p.wide = pool->dtype != CKV_DTYPE_F32 && most * G > few_rows;
  p.per_block = !shared || p.wide || pool->dtype == CKV_DTYPE_F32 ? 1 : (int)std::max<int64_t>(2, ceil_div(most * G, kRows));
  if (p.wide) {
    p.blocks = n_tokens * G / tile::kBlockRows + n_units;
    if (window > 0) len = std::min<int64_t>(len, (int64_t)window + ceil_div(tile::kBlockRows, G) + sinks + 16);
    const int64_t steps = ceil_div(len, tile::kTile);
    // The splits that cost least by a model of the launch, in cycles at 1.85 GHz: 512
    // workgroups run at once, two per CU, each for its stages (3,440 cycles a stage for two,
    // 2,100 for one alone on its CU) and a fixed part; a split's partials are written and
    // read again.  (2,341 tokens x 28 heads, 516 blocks, after 30,427 others: 1,543 us in
    // one split, 1,148 in 4, 1,125 in 6; after a window of 1,000: 67 us in one, 86 in 2.)
    constexpr double kFixed = 15000, kStage = 3440, kFixedAlone = 12500, kStageAlone = 2100;
    constexpr double kJoin = 5500, kJoinBytes = 2500;
    const int64_t wgs = tile_blocks * pool->n_kv_heads;
    const double join = (double)n_tokens * Hq * pool->head_dim * 2 * sizeof(float) / kJoinBytes;
    double best = 0;
    for (int64_t n0 = 1; n0 <= 64 && n0 * 4 <= std::max<int64_t>(steps, 4); ++n0) {
      const int64_t per = ceil_div(steps, n0), n = ceil_div(steps, per), rem = wgs * n % 512;
      double cost = (double)(wgs * n / 512) * (kFixed + kStage * (double)per);
      if (rem > 0)
        cost += rem <= 256 ? kFixedAlone + kStageAlone * (double)per : kFixed + kStage * (double)per;
      if (n > 1) cost += kJoin + join * (double)n;
      if (n0 == 1 || cost < best) {
        best = cost;
        p.n_splits = (int)n;
        p.slice = (int)per;
      }
    }
  } else {
    p.row_blocks = (int)std::min<int64_t>(65535, std::max<int64_t>(1, ceil_div(most * G, kRows * p.per_block)));
    if (window > 0) len = std::min<int64_t>(len, (int64_t)window + most + sinks + 2 * kTile);
    const int64_t steps = ceil_div(len, kTile);
    const int64_t wgs = (int64_t)n_units * pool->n_kv_heads * p.row_blocks;
    // Splits of 16 steps or more (a sequence of 1,026 steps: 14.0 us; of 12: 15.8, of 24: 14.5),
    // up to 4,096 workgroups, so that sequences of unequal lengths spread over the chip (64
    // of 1,024 to 16,384 tokens: 165 us; up to 2,048: 183, up to 8,192: 170).
    // Of shared keys a unit has places for twice the mean of kSharedBlocks, and takes as many as the
    // others leave (shared_slice).
    const int64_t most_wgs = shared ? kSharedBlocks * (n_units > 1 ? 2 : 1) : 4096;
    p.n_splits = (int)std::max<int64_t>(1, std::min(most_wgs / std::max<int64_t>(wgs, 1), steps / split_steps));
    p.slice = shared ? 16 : (int)std::max<int64_t>(1, ceil_div(steps, p.n_splits));
    p.n_wgs = (int)(kSharedBlocks / std::max<int64_t>(1, (int64_t)pool->n_kv_heads * p.row_blocks));
  }
  if (n_tokens * Hq >= kMaxGrid) p.n_splits = 1;  // (the join has a workgroup per row)
  return p;
}

PageAttnPlan make_plan(const ckv_page_pool* pool, const ckv_page_batch* b, int Hq, int window, int sinks,
                       int64_t split_steps = 16) {
  // (sequences' last blocks are taken as full: many short ones are more workgroups than this)
  const int64_t blocks = b->n_tokens * (Hq / pool->n_kv_heads) / tile::kBlockRows + 1;
  PageAttnPlan p = plan_units(pool, Hq, b->n_seqs, b->n_tokens, most_tokens(b->max_tokens, b->n_tokens, b->n_seqs),
                              longest(pool, b), blocks, window, sinks, kFewRows, false,
                              split_steps);
  const size_t rows = (size_t)b->n_tokens * Hq;
  if (p.n_splits > 1) {
    p.off_ml = align_up((size_t)p.n_splits * rows * pool->head_dim * sizeof(float), 256);
    p.off_n = align_up(p.off_ml + (size_t)p.n_splits * rows * sizeof(float2), 256);
    p.bytes = align_up(p.off_n + (size_t)b->n_tokens * sizeof(int32_t), 256);
  }
  return p;
}

// Attention of groups: a launch over the shared keys, one over the sequences' own, the join.
struct SharedPlan {
  bool apart;  // in parts; false: every sequence by itself is less work than those and their join
  PageAttnPlan whole, shared, own;
  int first_places;  // of the shared keys and, as most sequences have them, of the own ones
  size_t off_ml, off_shared, off_own, bytes;
};

SharedPlan make_shared_plan(const ckv_page_pool* pool, const ckv_page_batch* b, const ckv_page_groups* g, int Hq) {
  SharedPlan p{};
  const int G = Hq / pool->n_kv_heads;
  const int64_t len = longest(pool, b);
  const int64_t shared_len = g->max_shared > 0 ? std::min<int64_t>(len, g->max_shared) : len;
  const int64_t most = most_tokens(b->max_tokens, b->n_tokens, b->n_seqs);
  const int64_t saved = ((int64_t)b->n_seqs - g->n_groups) * shared_len * 2 * pool->n_kv_heads * pool->head_dim *
                        page_elem_bytes(pool->dtype);
  const bool prompts = pool->dtype != CKV_DTYPE_F32 && most * G > kFewRows;
  p.apart = g->n_groups > 0 && saved >= (prompts ? kWorthPrompts : kWorthParts);
  if (!p.apart) {
    // A few short sequences: a step for each of a workgroup's 8 waves where that is a workgroup per CU
    // at most (15 sequences of 1,100 keys in fp32, splits of 16 steps 14.2 us, of 8 11.3; two of 4,000 in
    // bf16 11.4 and 10.5); at head_dim 64 in 16 and 8 bits five steps a wave before the join is worth
    // its launch (four sequences of 1,040 keys: 16 steps 9.9 us, 8 9.2, all of them 8.4; of 1,640 10.1, 10.0
    // with all).
    const int64_t steps = ceil_div(len, kTile);
    int64_t split_steps = 16;
    if (pool->dtype != CKV_DTYPE_F32 && pool->head_dim == 64 && steps <= 40)
      split_steps = steps + 1;
    else if ((int64_t)b->n_seqs * pool->n_kv_heads * ceil_div(most * G, kRows) * ceil_div(steps, 8) <= 256)
      split_steps = 8;
    p.whole = make_plan(pool, b, Hq, 0, 0, split_steps);
    p.bytes = p.whole.bytes;
    return p;
  }
  const auto blocks = [&](int units, int64_t most_of) {
    return std::min(b->n_tokens * G / tile::kBlockRows + units, units * ceil_div(most_of * G, tile::kBlockRows));
  };
  // The sequences' own keys: splits for what the longest sequence has behind the longest prefix (a page at
  // least), and some more places for one whose keys are all its own: in no group, in one of a shorter prefix, or
  // where it is not known how much is shared.
  const int64_t own_len = std::max<int64_t>(len - shared_len, pool->page_size), own_blocks = blocks(b->n_seqs, most);
  p.own = plan_units(pool, Hq, b->n_seqs, b->n_tokens, most, own_len, own_blocks, 0, 0, kFewRows, false);
  const int64_t own_wgs = pool->n_kv_heads * (p.own.wide ? own_blocks : (int64_t)b->n_seqs * p.own.row_blocks);
  const int own_usual = p.own.n_splits;
  p.own.slice = std::max(p.own.slice, kOwnSlice);
  p.own.n_splits = (int)std::max<int64_t>(
      p.own.n_splits, std::min(ceil_div(ceil_div(len, p.own.wide ? tile::kTile : kTile), p.own.slice),
                               (p.own.wide ? kOwnTiles : kOwnWorkgroups) / std::max<int64_t>(own_wgs, 1)));
  const int64_t most_group = most_tokens(g->max_tokens, b->n_tokens, g->n_groups);
  const int few_rows = p.own.wide ? 0 : pool->dtype == CKV_DTYPE_BF16 && pool->head_dim == 128 ? 32 : 48;
  p.shared = plan_units(pool, Hq, g->n_groups, b->n_tokens, most_group, shared_len, blocks(g->n_groups, most_group), 0, 0,
                        few_rows, true);
  p.first_places = p.shared.n_splits + own_usual;
  const size_t rows = (size_t)b->n_tokens * Hq, places = (size_t)p.shared.n_splits + p.own.n_splits;
  p.off_ml = align_up(places * rows * pool->head_dim * sizeof(float), 256);
  p.off_shared = align_up(p.off_ml + places * rows * sizeof(float2), 256);
  p.off_own = align_up(p.off_shared + (size_t)b->n_tokens * sizeof(int32_t), 256);
  p.bytes = align_up(p.off_own + (size_t)b->n_tokens * sizeof(int32_t), 256);
  return p;
}

ckv_status check_attn(const ckv_page_pool* pool, const ckv_page_batch* b, int Hq, int window, int sinks,
                      bool with_pointers) {
  if (ckv_status s = check_pool(pool, with_pointers); s != CKV_OK) return s;
  if (ckv_status s = check_batch(b, with_pointers); s != CKV_OK) return s;
  if (Hq < 1 || Hq % pool->n_kv_heads)
    CKV_FAIL(CKV_EINVAL, "n_q_heads (%d) must be a positive multiple of n_kv_heads (%d)", Hq,
             pool->n_kv_heads);
  if (window < 0 || sinks < 0) CKV_FAIL(CKV_EINVAL, "window and n_sinks must be >= 0");
  if ((int64_t)b->max_pages * pool->page_size > (1 << 30))
    CKV_FAIL(CKV_EUNSUPPORTED, "tables of more than 2^30 tokens");
  if (window > (1 << 30) || sinks > (1 << 30)) CKV_FAIL(CKV_EUNSUPPORTED, "window or n_sinks past 2^30");
  return CKV_OK;
}

// Workgroups of a plan's launch: x by y, x a multiple of 8.
struct Grid {
  int64_t x, y;
};
ckv_status grid_of(PageAttnArgs& a, const PageAttnPlan& p, int units, Grid& g) {
  if (p.wide) {
    const int64_t streams = (int64_t)a.Hkv * a.n_splits;
    const int64_t rest = streams % 8;
    g = Grid{8 * (streams / 8 * p.blocks + ceil_div(rest * p.blocks, 8)), 1};
    a.n_blocks = (uint32_t)p.blocks;
  } else {
    g = Grid{(int64_t)align_up((size_t)units * a.n_splits, 8) * a.Hkv, p.row_blocks};
  }
  if (g.x >= kMaxGrid) CKV_FAIL(CKV_EUNSUPPORTED, "batch too large");
  return CKV_OK;
}

template <int D, int T, int P>
ckv_status launch_units(PageAttnArgs& a, const PageAttnPlan& p, hipStream_t st) {
  Grid g;
  if (ckv_status s = grid_of(a, p, P == kShared ? a.n_groups : a.s.n_seqs, g); s != CKV_OK) return s;
  if (p.wide) {
    if constexpr (T != CKV_DTYPE_F32)
      hipLaunchKernelGGL((page_tile_kernel<D, T, P>), dim3((unsigned)g.x), dim3(256), 0, st, a);
  } else if constexpr (is_whole(P)) {
    // A launch of at most a workgroup per CU has 8 waves in each, whose fewer steps follow
    // one another (16 sequences of 4 tokens: 13.1 -> 11.7 us, fp32 prompts 8.7 -> 8.0); where
    // there are more, 4 (48 sequences: 80 us, with 8: 94).
    const bool eight = g.x * g.y <= 256;
    const auto kernel = a.c == 8 ? (eight ? page_rows_kernel<D, T, true, 8, P> : page_rows_kernel<D, T, true, 4, P>)
                                 : (eight ? page_rows_kernel<D, T, false, 8, P> : page_rows_kernel<D, T, false, 4, P>);
    hipLaunchKernelGGL(kernel, dim3((unsigned)g.x, (unsigned)g.y), dim3(eight ? 512 : 256), 0, st, a);
  }
  CKV_HIP(hipGetLastError());
  return CKV_OK;
}

// The shared keys and, of few rows each, the sequences' own.
template <int D, int T, int kBlocks>
ckv_status launch_parts(PageAttnArgs& shared, PageAttnArgs& own, const SharedPlan& p, hipStream_t st) {
  Grid x, y;
  if (ckv_status s = grid_of(shared, p.shared, shared.n_groups, x); s != CKV_OK) return s;
  if (ckv_status s = grid_of(own, p.own, own.s.n_seqs, y); s != CKV_OK) return s;
  // (a workgroup goes on to the row blocks that a lower grid leaves)
  if (x.x * x.y + y.x * y.y >= kMaxGrid) {
    x.y = std::min(x.y, std::max<int64_t>(1, kMaxGrid / 2 / x.x - 1));
    y.y = std::min(y.y, std::max<int64_t>(1, kMaxGrid / 2 / y.x - 1));
  }
  const int64_t all = x.x * x.y + y.x * y.y;
  if (all >= kMaxGrid) CKV_FAIL(CKV_EUNSUPPORTED, "batch too large");
  const auto kernel = own.c == 8 ? page_parts_kernel<D, T, true, kBlocks> : page_parts_kernel<D, T, false, kBlocks>;
  hipLaunchKernelGGL(kernel, dim3((unsigned)all), dim3(256), 0, st, shared, own, (uint32_t)x.x, (uint32_t)x.y,
                     (uint32_t)y.x, (uint32_t)y.y);
  CKV_HIP(hipGetLastError());
  return CKV_OK;
}

// Joins the a.n_splits places of every row.
template <int D, int T, bool kParts>
ckv_status launch_join(const PageAttnArgs& a, hipStream_t st) {
  using QT = typename Elem<T>::Q;
  constexpr int kUnits = 256 / (D / 4);
  const int64_t rows = a.s.n_tokens * a.Hq;
  // Groups that take kJoinBatch places each at once, no more than there are places for: loads past
  // the last place are made all the same (2,560 rows of 9 places: 9.9 us with 8 groups, 5.4 with 2).
  int groups = 1;
  while (groups < kUnits && groups * kJoinBatch < a.n_splits) groups *= kParts ? 2 : kUnits;
  auto kernel = groups == 1 ? page_combine_kernel<D, QT, 1, kParts> : page_combine_kernel<D, QT, kUnits, kParts>;
  if constexpr (kParts) {
    if (groups == 2) kernel = page_combine_kernel<D, QT, 2, true>;
    if (groups == 4) kernel = page_combine_kernel<D, QT, 4, true>;
    if (groups == 8) kernel = page_combine_kernel<D, QT, 8, true>;
  }
  hipLaunchKernelGGL(kernel, dim3((unsigned)ceil_div(rows * groups, kUnits)), dim3(256), 0, st, a);
  CKV_HIP(hipGetLastError());
  return CKV_OK;
}

template <int D, int T, int P>
ckv_status launch_page_attn(PageAttnArgs& a, const PageAttnPlan& p, hipStream_t st) {
  if (ckv_status s = launch_units<D, T, P>(a, p, st); s != CKV_OK) return s;
  return a.n_splits > 1 ? launch_join<D, T, false>(a, st) : CKV_OK;
}

template <int D, int T>
ckv_status launch_shared_attn(PageAttnArgs& a, const SharedPlan& p, char* ws, hipStream_t st) {
  const size_t rows = (size_t)a.s.n_tokens * a.Hq;
  float* const o_part = reinterpret_cast<float*>(ws);
  float2* const ml_part = reinterpret_cast<float2*>(ws + p.off_ml);
  int32_t* const shared_parts = reinterpret_cast<int32_t*>(ws + p.off_shared);
  a.o_part = o_part;
  a.ml_part = ml_part;
  a.n_parts = shared_parts;
  a.n_splits = p.shared.n_splits;
  a.slice = p.shared.slice;
  a.n_wgs = p.shared.n_wgs;
  PageAttnArgs own = a;
  own.o_part = o_part + (size_t)p.shared.n_splits * rows * D;
  own.ml_part = ml_part + (size_t)p.shared.n_splits * rows;
  own.n_parts = reinterpret_cast<int32_t*>(ws + p.off_own);
  own.n_splits = p.own.n_splits;
  own.slice = p.own.slice;
  ckv_status s = CKV_OK;
  if constexpr (T == CKV_DTYPE_F32) {
    s = launch_parts<D, T, 1>(a, own, p, st);
  } else if (p.own.wide) {
    s = launch_units<D, T, kShared>(a, p.shared, st);
    if (s == CKV_OK) s = launch_units<D, T, kOwn>(own, p.own, st);
  } else if (p.shared.wide) {
    s = launch_parts<D, T, 0>(a, own, p, st);
  } else if (p.shared.per_block == 2) {
    s = launch_parts<D, T, 2>(a, own, p, st);
  } else if constexpr (T == CKV_DTYPE_E4M3 || D == 64) {
    s = launch_parts<D, T, 3>(a, own, p, st);
  }
  if (s != CKV_OK) return s;
  a.n_parts = own.n_parts;
  a.o_part = o_part;
  a.ml_part = ml_part;
  a.shared_parts = shared_parts;
  a.shared_splits = p.shared.n_splits;
  a.first_places = p.first_places;
  a.n_splits = p.shared.n_splits + p.own.n_splits;
  return launch_join<D, T, true>(a, st);
}

// f(D, T) of a pool, as integral constants.
template <class F>
ckv_status for_pool(const ckv_page_pool* pool, F&& f) {
  using std::integral_constant;
  if (pool->dtype == CKV_DTYPE_F32) return f(integral_constant<int, 64>{}, integral_constant<int, CKV_DTYPE_F32>{});
  if (pool->dtype == CKV_DTYPE_BF16)
    return pool->head_dim == 128 ? f(integral_constant<int, 128>{}, integral_constant<int, CKV_DTYPE_BF16>{})
                                 : f(integral_constant<int, 64>{}, integral_constant<int, CKV_DTYPE_BF16>{});
  return pool->head_dim == 128 ? f(integral_constant<int, 128>{}, integral_constant<int, CKV_DTYPE_E4M3>{})
                               : f(integral_constant<int, 64>{}, integral_constant<int, CKV_DTYPE_E4M3>{});
}

// What both calls need of q, out and ws, and the kernels' arguments but for their plan's.
ckv_status check_rows(const ckv_page_batch* batch, const void* q, int32_t n_q_heads, const void* out, const void* ws) {
  if (!q || !out) CKV_FAIL(CKV_EINVAL, "NULL pointer argument");
  if (!aligned16(q) || !aligned16(out) || !aligned16(ws))
    CKV_FAIL(CKV_EINVAL, "pointers must be 16-byte aligned");
  if (batch->n_tokens * n_q_heads > (int64_t(1) << 26))
    CKV_FAIL(CKV_EUNSUPPORTED, "more than 2^26 query rows in one call");
  return CKV_OK;
}
ckv_status check_scale(float sm_scale) {
  if (!(sm_scale >= 0.f) || std::isinf(sm_scale)) CKV_FAIL(CKV_EINVAL, "sm_scale must be finite and >= 0");
  return CKV_OK;
}
PageAttnArgs attn_args(const ckv_page_pool* pool, const ckv_page_batch* batch, const void* q, int32_t n_q_heads,
                       float sm_scale, void* out) {
  PageAttnArgs a{};
  a.s = page_seqs(batch);
  a.k = static_cast<const char*>(pool->k);
  a.v = static_cast<const char*>(pool->v);
  a.k_scale = pool->k_scale;
  a.v_scale = pool->v_scale;
  a.page_stride = page_stride_bytes(pool);
  a.n_pages = pool->n_pages;
  a.q = q;
  a.out = out;
  a.c = pool->page_size;
  a.log2c = (a.c & (a.c - 1)) == 0 ? __builtin_ctz(a.c) : -1;
  a.Hkv = pool->n_kv_heads;
  a.Hq = n_q_heads;
  a.G = n_q_heads / pool->n_kv_heads;
  a.c1 = (sm_scale > 0.f ? sm_scale : 1.0f / sqrtf((float)pool->head_dim)) * 1.4426950408889634f;
  return a;
}
void set_plan(PageAttnArgs& a, const PageAttnPlan& p, void* ws) {
  a.o_part = static_cast<float*>(ws);
  a.ml_part = p.bytes ? reinterpret_cast<float2*>(static_cast<char*>(ws) + p.off_ml) : nullptr;
  a.n_parts = p.bytes ? reinterpret_cast<int32_t*>(static_cast<char*>(ws) + p.off_n) : nullptr;
  a.slice = p.slice;
  a.n_splits = p.n_splits;
}

}  // namespace
}  // namespace ckv

using namespace ckv;

extern "C" {

size_t ckv_page_attn_workspace_bytes(const ckv_page_pool* pool, const ckv_page_batch* batch,
                                     int32_t n_q_heads, int32_t window, int32_t n_sinks) {
  if (check_attn(pool, batch, n_q_heads, window, n_sinks, false) != CKV_OK) return 0;
  return make_plan(pool, batch, n_q_heads, window, n_sinks).bytes;
}

ckv_status ckv_page_attn(const ckv_page_pool* pool, const ckv_page_batch* batch, const void* q,
                         int32_t n_q_heads, float sm_scale, int32_t window, int32_t n_sinks,
                         void* out, void* ws, size_t ws_bytes, void* stream) {
  clear_error();
  if (ckv_status s = check_attn(pool, batch, n_q_heads, window, n_sinks, true); s != CKV_OK) return s;
  if (ckv_status s = check_scale(sm_scale); s != CKV_OK) return s;
  if (batch->n_seqs == 0 || batch->n_tokens == 0) return CKV_OK;
  if (ckv_status s = check_rows(batch, q, n_q_heads, out, ws); s != CKV_OK) return s;
  const PageAttnPlan p = make_plan(pool, batch, n_q_heads, window, n_sinks);
  if (p.bytes && (!ws || ws_bytes < p.bytes))
    CKV_FAIL(CKV_EINVAL, "workspace too small: %zu < %zu", ws ? ws_bytes : (size_t)0, p.bytes);
  PageAttnArgs a = attn_args(pool, batch, q, n_q_heads, sm_scale, out);
  set_plan(a, p, ws);
  a.window = window;
  a.sinks = window > 0 ? n_sinks : 0;
  return for_pool(pool, [&](auto d, auto t) { return launch_page_attn<d, t, kWhole>(a, p, (hipStream_t)stream); });
}

size_t ckv_page_attn_shared_workspace_bytes(const ckv_page_pool* pool, const ckv_page_batch* batch,
                                            const ckv_page_groups* groups, int32_t n_q_heads) {
  if (check_attn(pool, batch, n_q_heads, 0, 0, false) != CKV_OK) return 0;
  if (check_groups(groups, batch, false) != CKV_OK) return 0;
  return make_shared_plan(pool, batch, groups, n_q_heads).bytes;
}

ckv_status ckv_page_attn_shared(const ckv_page_pool* pool, const ckv_page_batch* batch,
                                const ckv_page_groups* groups, const void* q, int32_t n_q_heads,
                                float sm_scale, void* out, void* ws, size_t ws_bytes, void* stream) {
  clear_error();
  if (ckv_status s = check_attn(pool, batch, n_q_heads, 0, 0, true); s != CKV_OK) return s;
  if (ckv_status s = check_groups(groups, batch, true); s != CKV_OK) return s;
  if (ckv_status s = check_scale(sm_scale); s != CKV_OK) return s;
  if (batch->n_seqs == 0 || batch->n_tokens == 0) return CKV_OK;
  if (ckv_status s = check_rows(batch, q, n_q_heads, out, ws); s != CKV_OK) return s;
  const SharedPlan p = make_shared_plan(pool, batch, groups, n_q_heads);
  if (p.bytes && (!ws || ws_bytes < p.bytes))
    CKV_FAIL(CKV_EINVAL, "workspace too small: %zu < %zu", ws ? ws_bytes : (size_t)0, p.bytes);
  PageAttnArgs a = attn_args(pool, batch, q, n_q_heads, sm_scale, out);
  if (!p.apart) {
    set_plan(a, p.whole, ws);
    return for_pool(pool, [&](auto d, auto t) {
      return launch_page_attn<d, t, t == CKV_DTYPE_F32 ? kAlone : kWhole>(a, p.whole, (hipStream_t)stream);
    });
  }
  a.grp_off = groups->grp_off;
  a.shared = groups->shared;
  a.n_groups = groups->n_groups;
  return for_pool(pool, [&](auto d, auto t) {
    return launch_shared_attn<d, t>(a, p, static_cast<char*>(ws), (hipStream_t)stream);
  });
}

}  // extern "C"
