// beam.hip -- the continuations of beams for gfx950.
//
// A live beam's token v has score c + x_v - log sum_u exp(x_u); the `keep` best of a request's
// beams go on.  Within a beam the scores fall with the logits, so the keep largest logits of
// each beam are enough, and the logits are read once:
//   beam_scan_kernel   a workgroup per slice of a beam's vocabulary: the sum of the exponentials
//                      against the slice's maximum, and its keep largest logits
//   beam_join_kernel   a workgroup per request: the slices of each beam, then the beams
// The scan is bound by reading the logits, and by what its waves do after the last of them: 256 beams
// over 131,072 tokens in bf16 (60 MB of live ones) 20.6 us, of which 14 with the reading alone, 1.5 for
// the exponentials and 5 for the choice; 104 of 100,003 in fp32 (41 MB) 16 us; 4 of 32,000 6.3.  The join
// takes 5.4 to 7.6 us, a chain of loads, a logarithm and merges.  A call of few beams is bound by its
// own two launches and checks on the host: 11 us.

#include <type_traits>

#include "pages_internal.h"

namespace ckv {
namespace {

constexpr int kMost = 64;  // beams of a request, and continuations that are kept: lanes of a wave
constexpr float kLowest = -3.4028234663852886e38f;
constexpr double kNoRef = -1e300;  // reference of an empty sum

// A logit and its token as one number: larger for a larger logit, then for a lower token.
// 0: none; numbers up to kNoKey are of logits that are -infinity.
constexpr uint64_t kNoKey = uint64_t(0x007fffff) << 32 | 0xffffffffu;
__device__ __forceinline__ uint64_t key_of(float x, int token) {
  const uint32_t b = __float_as_uint(x + 0.f);  // (-0 is 0)
  return join64(b ^ ((uint32_t)((int32_t)b >> 31) | 0x80000000u), ~(uint32_t)token);
}
__device__ __forceinline__ float value_of(uint64_t key) {
  const uint32_t b = (uint32_t)(key >> 32);
  return __uint_as_float(b & 0x80000000u ? b ^ 0x80000000u : ~b);
}
__device__ __forceinline__ int token_of_key(uint64_t key) { return (int)~(uint32_t)key; }

// The key of lane ^ X.
template <int X>
__device__ __forceinline__ uint64_t other(uint64_t k) {
  if constexpr (X == 1) return dpp64<kDppQuadXor1>(k);
  if constexpr (X == 2) return dpp64<kDppQuadXor2>(k);
  if constexpr (X == 4) return dpp64<0x1B>(dpp64<kDppRowHalfMirror>(k));  // (lane ^ 7) ^ 3
  if constexpr (X == 8) return dpp64<0x128>(k);                           // rotated by 8 in 16
  uint64_t a, b;
  swap_pair64<X>(k, a, b);
  return a ^ b ^ k;  // (a, b: own and partner's)
}
// One step of a bitonic network: of each pair lane, lane ^ X the lower lane of a descending
// run keeps the larger.  Runs of R lanes alternate; the last ones go down, with kUp up.
template <int X, int R, bool kUp>
__device__ __forceinline__ uint64_t exchange(uint64_t k) {
  const int lane = threadIdx.x & 63;
  const uint64_t o = other<X>(k);
  const bool larger = (((lane & X) == 0) == ((lane & R) == 0)) != kUp;
  return (k > o) == larger ? k : o;
}
template <int X, int R, bool kUp>
__device__ __forceinline__ uint64_t merge_runs(uint64_t k) {
  k = exchange<X, R, kUp>(k);
  if constexpr (X > 1) k = merge_runs<X / 2, R, kUp>(k);
  return k;
}
// A wave's 64 keys in descending (kUp: ascending) order.
template <bool kUp>
__device__ __forceinline__ uint64_t sorted(uint64_t k) {
  k = merge_runs<1, 2, kUp>(k);
  k = merge_runs<2, 4, kUp>(k);
  k = merge_runs<4, 8, kUp>(k);
  k = merge_runs<8, 16, kUp>(k);
  k = merge_runs<16, 32, kUp>(k);
  return merge_runs<32, 64, kUp>(k);
}
// The 64 largest of two runs, the first in descending, the second in ascending order.
__device__ __forceinline__ uint64_t largest(uint64_t k, uint64_t ascending) {
  return merge_runs<32, 64, false>(k > ascending ? k : ascending);
}
__device__ __forceinline__ uint64_t lane_of(uint64_t k, int lane) {  // (lane: one for the wave)
  return join64((uint32_t)__builtin_amdgcn_readlane((int)(k >> 32), lane),
                (uint32_t)__builtin_amdgcn_readlane((int)k, lane));
}

// What the wave's lanes wrote to LDS is there for its other lanes.
__device__ __forceinline__ void wave_sync() {
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  __builtin_amdgcn_wave_barrier();
}

struct BeamArgs {
  const char* logits;
  const float* scores;
  const uint8_t* done;
  int64_t row_stride;  // elements
  int32_t n_reqs, n_beams, vocab, keep, eos;
  int32_t slices, slice;  // of a beam, and batches (of 64 lanes' pieces) of one
  double* ref;            // [rows][slices]: the sum is of exp(x - ref)
  double* sum;            // [rows][slices]
  uint64_t* keys;         // [rows][slices][keep], descending, 0 behind the last
  int32_t* parent;
  int32_t* token;
  float* score;
  uint8_t* done_out;
};

constexpr int kWaves = 4;
constexpr int kPieces = 4;  // 16-byte pieces of a lane per batch
constexpr int64_t kScanBlocks = 1024;  // workgroups of a scan, about: 4 per CU
constexpr int64_t kMaxScanGrid = int64_t(1) << 24;

// The largest of three; of a NaN and numbers a number, or a NaN (which the sum then shows).
__device__ __forceinline__ float max3(float x, float y, float z) {
  float m;
  asm("v_max3_f32 %0, %1, %2, %3" : "=v"(m) : "v"(x), "v"(y), "v"(z));
  return m;
}

// 16 bytes from any element on.
__device__ __forceinline__ u32x4 piece_at(const char* p) {
  u32x4 x;
  __builtin_memcpy(&x, p, sizeof x);
  return x;
}

// An element of a piece (four words).
template <bool kBf16>
__device__ __forceinline__ float element(const uint32_t* w, int e) {
  if constexpr (kBf16) return __uint_as_float(e & 1 ? w[e >> 1] & 0xffff0000u : w[e >> 1] << 16);
  return __uint_as_float(w[e]);
}

// A wave goes over its batches, the next ones' loads under way, and takes of each the sum of the
// exponentials and every lane's largest element: no more, so that the memory is kept busy.
// Then keep lanes or so have all that can be among its keep largest: the lanes whose largest is
// no less than the keep-th largest of the lanes'.  Their elements are read again (from the L2),
// and those that are no less are collected in LDS.  64 collected are sorted and merged into the
// list that the lanes hold: mostly a workgroup's waves together find fewer, and one sort at
// the end does.
// kTiny: fewer tokens than a piece.
template <bool kBf16, bool kTiny>
__global__ __launch_bounds__(64 * kWaves, 4) void beam_scan_kernel(BeamArgs a) {
  constexpr int kPer = kBf16 ? 8 : 4, kBytes = kBf16 ? 2 : 4;  // elements of a piece, bytes of one
  constexpr int64_t kBatch = 64 * kPieces * kPer;
  __shared__ int32_t lanes[kWaves][64];
  __shared__ uint64_t found[kWaves][64 * (1 + kPer)];  // a piece of every lane has room behind 63
  __shared__ double sums[kWaves], refs[kWaves];
  __shared__ int32_t counts[kWaves];
  const int64_t row = blockIdx.x / a.slices;
  const int slice = blockIdx.x % a.slices;
  const float cum = a.scores[row];
  if (!(cum > -INFINITY) || (a.done && a.done[row])) return;  // offers no token: the join knows
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  // Pieces count from the row's begin, wherever that lies: rows of equal logits are then added up
  // alike, and their scores tie as they should.
  const char* const base = a.logits + row * a.row_stride * kBytes;
  const int64_t end = a.vocab;
  const int64_t batches = (end + kBatch - 1) / kBatch;
  const int64_t b0 = (int64_t)slice * a.slice + wave, b1 = min((int64_t)(slice + 1) * a.slice, batches);
  const int n_batches = b0 < b1 ? (int)((b1 - b0 + kWaves - 1) / kWaves) : 0;  // this wave's: b0, b0 + kWaves ..
  const int keep = a.keep;

  // Element e of a piece that begins at p0 is of token token_at(p0) + e: a piece that would
  // reach past the row is the row's last one, where those before p0 count for nothing.
  using Batch = u32x4[kPieces];
  auto piece_of = [&](int64_t batch, int i, int l) __attribute__((always_inline)) {
    return batch * kBatch + (int64_t)(i * 64 + l) * kPer;
  };
  auto token_at = [&](int64_t p0) __attribute__((always_inline)) { return kTiny ? 0 : min(p0, end - kPer); };
  auto load = [&](int64_t p0) __attribute__((always_inline)) {
    if constexpr (!kTiny) return piece_at(base + token_at(p0) * kBytes);
    u32x4 x{0u, 0u, 0u, 0u};
    for (int e = 0; e < (int)end; ++e) {
      if constexpr (kBf16)
        x[e >> 1] |= (uint32_t)reinterpret_cast<const uint16_t*>(base)[e] << 16 * (e & 1);
      else
        x[e] = reinterpret_cast<const uint32_t*>(base)[e];
    }
    return x;
  };
  // -infinity outside the piece's own tokens and, if `careful`, for NaN; the largest number for an infinity.
  auto mend = [&](int64_t p0, bool outside, bool careful, u32x4& x) __attribute__((always_inline)) {
    const int64_t at = token_at(p0);
    const int from = (int)min(p0 - at, (int64_t)kPer), upto = (int)min(end - at, (int64_t)kPer);
#pragma unroll
    for (int e = 0; e < kPer; ++e) {
      const bool drop = outside && (e < from || e >= upto);
      if constexpr (kBf16) {
        uint32_t h = x[e >> 1] >> 16 * (e & 1) & 0xffffu;
        if (careful) h = (h & 0x7fffu) > 0x7f80u ? 0xff80u : h == 0x7f80u ? 0x7f7fu : h;
        h = drop ? 0xff80u : h;
        x[e >> 1] = e & 1 ? (x[e >> 1] & 0xffffu) | h << 16 : (x[e >> 1] & 0xffff0000u) | h;
      } else {
        uint32_t h = x[e];
        if (careful) h = (h & 0x7fffffffu) > 0x7f800000u ? 0xff800000u : h == 0x7f800000u ? 0x7f7fffffu : h;
        x[e] = drop ? 0xff800000u : h;
      }
    }
  };

  double ref, sum;  // of exp(x - ref)
  float mx;         // this lane's largest
  // The exponent x log2(e) - c is one fused step with c = log2(e) max, rounded: the reference is
  // c / log2(e) exactly, and what the factor's own rounding leaves, kOff x, is taken back for
  // x = max, off by kOff (max - x) for the others, a term that is as far below the largest.
  // `careful`: as in mend, and the exponent is (x - max) log2(e), as c may be past what 32 bits
  // hold.  Such logits show in the sum, after which the slice is done again.
  constexpr float kLog2e = 1.4426950408889634f;
  constexpr double kOff = 1.0 - (double)kLog2e / 1.4426950408889634074;
  float top, c;
  auto clear = [&](float from) __attribute__((always_inline)) {
    top = from;
    c = top * kLog2e;
    sum = 0;
    mx = -INFINITY;
  };
  auto take = [&](const Batch& x, auto careful) __attribute__((always_inline)) {
    float v[kPieces * kPer];
#pragma unroll
    for (int i = 0; i < kPieces; ++i) {
      const uint32_t w[4] = {x[i][0], x[i][1], x[i][2], x[i][3]};
#pragma unroll
      for (int e = 0; e < kPer; ++e) v[i * kPer + e] = element<kBf16>(w, e);
    }
#pragma unroll
    for (int e = 0; e < kPieces * kPer; e += 2) mx = max3(mx, v[e], v[e + 1]);
    if (__any(mx > top)) {
      // (no product of this block may go into a fused step: sums are carried from the rounded c to the
      // rounded next one, and what one unrounded would be off by grows with c: 8e-6 in the logarithm for
      // logits around 500)
#pragma clang fp contract(off)
      float to = mx;
#pragma unroll
      for (int i = 1; i < 64; i <<= 1) to = fmaxf(to, __shfl_xor(to, i));
      const float next = to * kLog2e;
      sum *= (double)__builtin_amdgcn_exp2f(careful ? (top - to) * kLog2e : c - next);
      top = to;
      c = next;
    }
    float part[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int e = 0; e < kPieces * kPer; ++e)
      part[e & 3] += __builtin_amdgcn_exp2f(careful ? (v[e] - top) * kLog2e : fmaf(v[e], kLog2e, -c));
    sum += (double)((part[0] + part[1]) + (part[2] + part[3]));
  };
  auto take_slow = [&](int n, auto careful) __attribute__((always_inline)) {
    const int64_t batch = b0 + (int64_t)n * kWaves;
    Batch x;
#pragma unroll
    for (int i = 0; i < kPieces; ++i) {
      x[i] = load(piece_of(batch, i, lane));
      mend(piece_of(batch, i, lane), true, careful, x[i]);
    }
    take(x, careful);
  };
  auto all_lanes = [&]() __attribute__((always_inline)) {
#pragma unroll
    for (int i = 1; i < 64; i <<= 1) sum += __shfl_xor(sum, i);
  };
  clear(-0x1p125f);
  {
    // whole batches, two of them under way; the lanes' addresses are a common one and 16 bytes each
    const int64_t last = b0 + (int64_t)(n_batches - 1) * kWaves;
    const int n_whole = n_batches > 0 && (last + 1) * kBatch > end ? n_batches - 1 : n_batches;
    auto fetch = [&](int n, Batch& x) __attribute__((always_inline)) {  // (past the last: that one again)
      const char* from = base + (b0 + (int64_t)min(n, n_whole - 1) * kWaves) * (kBatch * kBytes);
#pragma unroll
      for (int i = 0; i < kPieces; ++i) x[i] = piece_at(from + (uint32_t)(lane * 16) + i * 1024);
    };
    constexpr std::false_type plain{};
    if (n_whole > 0) {
      Batch x, y, z;
      fetch(0, x);
      fetch(1, y);
      for (int n = 0;; n += 3) {
        fetch(n + 2, z);
        take(x, plain);
        if (n + 1 >= n_whole) break;
        fetch(n + 3, x);
        take(y, plain);
        if (n + 2 >= n_whole) break;
        fetch(n + 4, y);
        take(z, plain);
        if (n + 3 >= n_whole) break;
      }
    }
    if (n_whole < n_batches) take_slow(n_batches - 1, plain);
    all_lanes();
  }
  ref = (double)c * 0.69314718055994530942 + kOff * (double)top;
  const bool careful = __any(!__builtin_isfinite(sum) || (sum == 0 && mx > -INFINITY));
  if (careful) {
    clear(kLowest);
    for (int n = 0; n < n_batches; ++n) take_slow(n, std::true_type{});
    all_lanes();
    ref = (double)top;
  }
  if (sum == 0) ref = kNoRef;

  // Bit by bit the largest number that keep lanes' largest reach, or one a little below it (as
  // upper halves of keys); every number above -infinity where fewer lanes have any.
  const uint32_t mine = (uint32_t)(key_of(mx, 0) >> 32);
  uint32_t kth = 0;
#pragma unroll
  for (int bit = 31; bit >= (kBf16 ? 16 : 12); --bit) {
    const uint32_t to = kth | 1u << bit;
    if (__builtin_popcountll(__ballot(mine >= to)) >= keep) kth = to;
  }
  uint64_t least = max((uint64_t)kth << 32, kNoKey + 1);  // what the best have at least
  uint64_t list = 0;                                      // this lane's of the 64 best so far
  int n_found = 0;
  bool flushed = false;  // the list has some
  const uint64_t hit = __ballot(mine >= (uint32_t)(least >> 32));
  if (hit >> lane & 1) lanes[wave][__builtin_amdgcn_mbcnt_hi(hit >> 32, __builtin_amdgcn_mbcnt_lo((uint32_t)hit, 0))] = lane;
  wave_sync();
  const int per_lane = n_batches * kPieces, total = __builtin_popcountll(hit) * per_lane;
  for (int at = lane; at - lane < total; at += 64) {
    const int l = min(at / max(per_lane, 1), 63), piece = at % max(per_lane, 1);
    const int64_t p0 = piece_of(b0 + (int64_t)(piece / kPieces) * kWaves, piece % kPieces, lanes[wave][l]);
    u32x4 x{0u, 0u, 0u, 0u};
    if (at < total) {
      x = load(p0);
      mend(p0, true, careful, x);
    }
    const uint32_t w[4] = {x[0], x[1], x[2], x[3]};
    const int first = (int)token_at(p0);
#pragma unroll
    for (int e = 0; e < kPer; ++e) {
      const uint64_t k = key_of(element<kBf16>(w, e), first + e);
      const uint64_t yes = __ballot(at < total && k >= least);
      if (!yes) continue;
      if (yes >> lane & 1)
        found[wave][n_found + __builtin_amdgcn_mbcnt_hi(yes >> 32, __builtin_amdgcn_mbcnt_lo((uint32_t)yes, 0))] = k;
      n_found += __builtin_popcountll(yes);
    }
    while (n_found >= 64) {  // the last 64 found
      n_found -= 64;
      wave_sync();
      list = largest(list, sorted<true>(found[wave][n_found + lane]));
      wave_sync();
      const uint64_t last = lane_of(list, keep - 1);
      least = last > least ? last : least;
      flushed = true;
    }
  }

  // The waves' parts.  What they found is mostly 64 keys at most: one wave then sorts it all.
  if (lane == 0) {
    sums[wave] = sum;
    refs[wave] = ref;
    counts[wave] = flushed ? 65 : n_found;
  }
  __syncthreads();
  int before[kWaves + 1] = {0};
#pragma unroll
  for (int w = 0; w < kWaves; ++w) before[w + 1] = before[w] + counts[w];
  if (before[kWaves] > 64) {  // (the same for all waves)
    list = largest(list, sorted<true>(lane < n_found ? found[wave][lane] : 0));
    wave_sync();
    found[wave][lane] = list;
    __syncthreads();
    if (wave > 0) return;
#pragma unroll
    for (int w = 1; w < kWaves; ++w) list = largest(list, found[w][63 - lane]);
  } else {
    if (wave > 0) return;
    uint64_t k = 0;
#pragma unroll
    for (int w = 0; w < kWaves; ++w)
      if (lane >= before[w] && lane < before[w + 1]) k = found[w][lane - before[w]];
    list = sorted<false>(k);
  }
  ref = refs[lane & (kWaves - 1)];
  double most = ref;
#pragma unroll
  for (int i = 1; i < kWaves; i <<= 1) most = fmax(most, __shfl_xor(most, i));
  sum = sums[lane & (kWaves - 1)] * exp(ref - most);
#pragma unroll
  for (int i = 1; i < kWaves; i <<= 1) sum += __shfl_xor(sum, i);
  const int64_t at = row * a.slices + slice;
  if (lane == 0) {
    a.ref[at] = most;
    a.sum[at] = sum;
  }
  if (lane < keep) a.keys[at * keep + lane] = list;
}

// A wave per beam in turn joins its slices' sums and lists; then the beams' lists, which fall,
// are merged by counting what goes before each entry: equal scores go to the lower beam.
constexpr int kJoinWaves = 8;
__global__ __launch_bounds__(64 * kJoinWaves) void beam_join_kernel(BeamArgs a) {
  extern __shared__ double scores[];  // [n_beams][keep], then tokens, then entries of each beam
  int32_t* const tokens = reinterpret_cast<int32_t*>(scores + a.n_beams * a.keep);
  int32_t* const entries = tokens + a.n_beams * a.keep;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int64_t row0 = (int64_t)blockIdx.x * a.n_beams;
  const int keep = a.keep;
  for (int b = wave; b < a.n_beams; b += kJoinWaves) {
    const int64_t row = row0 + b, at = row * a.slices;
    // (all loads together: those of a beam that the scan left out hold anything)
    const uint64_t* const keys = a.keys + at * keep;
    const int up = 63 - lane;
    uint64_t list = lane < keep ? keys[lane] : 0, next = a.slices > 1 && up < keep ? keys[keep + up] : 0;
    const double ref = lane < a.slices ? a.ref[at + lane] : kNoRef;
    double sum = lane < a.slices ? a.sum[at + lane] : 0;
    const float c = a.scores[row];
    const uint8_t ended = a.done ? a.done[row] : 0;
    const bool live = c > -INFINITY, done = live && ended;
    int n = 0;
    if (done) {
      n = 1;
      if (lane == 0) {
        scores[b * keep] = (double)c;
        tokens[b * keep] = a.eos;
      }
    } else if (live) {
      // (every lane is to have the same sum: a product fused into one lane's addition and rounded for the
      // other's would part their scores by 2^-40 once in thousands of rows, and break ties)
#pragma clang fp contract(off)
      double top = ref;
#pragma unroll
      for (int i = 1; i < 64; i <<= 1) top = fmax(top, __shfl_xor(top, i));
      sum *= exp(ref - top);
#pragma unroll
      for (int i = 1; i < 64; i <<= 1) sum += __shfl_xor(sum, i);
      for (int s = 1; s < a.slices; ++s) {
        const uint64_t x = next;
        next = s + 1 < a.slices && up < keep ? keys[(int64_t)(s + 1) * keep + up] : 0;
        list = largest(list, x);
      }
      // A whole number of 2^-40, finer than the exponentials are: what is added to it in 64 bits
      // (logits and scores below 2^12 that are whole numbers of it as well) is added exactly, so
      // that scores which are equal by arithmetic compare equal.
      // (Past 2^20 the logarithm is not to be lost in the reference.)
      const double rest = log(sum), all = rint((top + rest) * 0x1p40) * 0x1p-40;
      const bool far = fabs(top) > 0x1p20;
      n = __builtin_popcountll(__ballot(lane < keep && list != 0));
      if (lane < n) {
        const double x = (double)value_of(list);
        scores[b * keep + lane] = (far ? (x - top) - rest : x - all) + (double)c;
        tokens[b * keep + lane] = token_of_key(list);
      }
    }
    if (lane == 0) entries[b] = n;
  }
  __syncthreads();
  int total = 0;
  for (int b = 0; b < a.n_beams; ++b) total += entries[b];
  const int64_t out0 = (int64_t)blockIdx.x * keep;
  for (int i = threadIdx.x; i < a.n_beams * keep; i += 64 * kJoinWaves) {
    const int b = i / keep;
    if (i % keep >= entries[b]) continue;
    const double s = scores[i];
    int rank = i % keep;
    for (int o = 0; o < a.n_beams && rank < keep; ++o) {
      if (o == b) continue;
      int lo = 0, hi = entries[o];  // the first entry of beam o that does not go before
      while (lo < hi) {
        const int mid = (lo + hi) >> 1;
        const double x = scores[o * keep + mid];
        if (x > s || (x == s && o < b))
          lo = mid + 1;
        else
          hi = mid;
      }
      rank += lo;
    }
    if (rank >= keep) continue;
    const int64_t row = row0 + b;
    a.parent[out0 + rank] = (int32_t)row;
    a.token[out0 + rank] = tokens[i];
    a.score[out0 + rank] = (float)s;
    if (a.done_out) a.done_out[out0 + rank] = tokens[i] == a.eos || (a.done && a.done[row]) ? 1 : 0;
  }
  for (int i = total + (int)threadIdx.x; i < keep; i += 64 * kJoinWaves) {
    a.parent[out0 + i] = -1;
    a.token[out0 + i] = -1;
    a.score[out0 + i] = -INFINITY;
    if (a.done_out) a.done_out[out0 + i] = 0;
  }
}

struct BeamPlan {
  int32_t slices, slice;
  size_t off_sum, off_keys, bytes;
};

BeamPlan make_beam_plan(const ckv_beams* b) {
  BeamPlan p{};
  const int64_t rows = (int64_t)b->n_reqs * b->n_beams;
  const int64_t batch = 64 * kPieces * (b->dtype == CKV_DTYPE_BF16 ? 8 : 4);
  const int64_t batches = ceil_div(b->vocab, batch);
  const int64_t most = std::min<int64_t>(kMost, ceil_div(batches, kWaves));
  const int64_t want = std::max<int64_t>(1, std::min(most, ceil_div(kScanBlocks, std::max<int64_t>(rows, 1))));
  p.slice = (int32_t)ceil_div(batches, want);
  p.slices = (int32_t)ceil_div(batches, p.slice);
  p.off_sum = align_up((size_t)rows * p.slices * sizeof(double), 256);
  p.off_keys = align_up(p.off_sum + (size_t)rows * p.slices * sizeof(double), 256);
  p.bytes = align_up(p.off_keys + (size_t)rows * p.slices * b->keep * sizeof(uint64_t), 256);
  return p;
}

ckv_status check_beams(const ckv_beams* b, bool with_pointers) {
  if (!b) CKV_FAIL(CKV_EINVAL, "beams is NULL");
  if (b->dtype != CKV_DTYPE_F32 && b->dtype != CKV_DTYPE_BF16) CKV_FAIL(CKV_EINVAL, "logits are fp32 or bf16");
  if (b->n_reqs < 0 || b->n_reqs > (1 << 20))
    CKV_FAIL(CKV_EINVAL, "n_reqs must be in [0, 2^20] (got %d)", b->n_reqs);
  if (b->n_beams < 1 || b->keep < 1) CKV_FAIL(CKV_EINVAL, "n_beams and keep must be >= 1");
  if (b->n_beams > kMost || b->keep > kMost)
    CKV_FAIL(CKV_EUNSUPPORTED, "more than %d beams or continuations (%d, %d)", kMost, b->n_beams, b->keep);
  if ((int64_t)b->n_reqs * b->n_beams > (1 << 20)) CKV_FAIL(CKV_EUNSUPPORTED, "more than 2^20 beams in one call");
  if (b->vocab < 1) CKV_FAIL(CKV_EINVAL, "vocab must be >= 1 (got %d)", b->vocab);
  if (b->vocab > (1 << 30)) CKV_FAIL(CKV_EUNSUPPORTED, "vocab past 2^30");
  if (b->row_stride != 0 && (b->row_stride < b->vocab || b->row_stride > (int64_t(1) << 40)))
    CKV_FAIL(CKV_EINVAL, "row_stride must be 0 or at least vocab");
  if (b->eos < -1 || b->eos >= b->vocab) CKV_FAIL(CKV_EINVAL, "eos must be -1 or below vocab (got %d)", b->eos);
  if (b->done && b->eos < 0) CKV_FAIL(CKV_EINVAL, "beams that are done need eos");
  if (!with_pointers || b->n_reqs == 0) return CKV_OK;
  if (!b->logits || !b->scores) CKV_FAIL(CKV_EINVAL, "NULL beams pointer");
  if (reinterpret_cast<uintptr_t>(b->logits) % elem_bytes(b->dtype))
    CKV_FAIL(CKV_EINVAL, "logits must be aligned to an element");
  return CKV_OK;
}

}  // namespace
}  // namespace ckv

using namespace ckv;

extern "C" {

size_t ckv_beam_select_workspace_bytes(const ckv_beams* beams) {
  return check_beams(beams, false) == CKV_OK ? make_beam_plan(beams).bytes : 0;
}

ckv_status ckv_beam_select(const ckv_beams* beams, int32_t* parent, int32_t* token, float* score, uint8_t* done,
                           void* ws, size_t ws_bytes, void* stream) {
  clear_error();
  if (ckv_status s = check_beams(beams, true); s != CKV_OK) return s;
  if (beams->n_reqs == 0) return CKV_OK;
  if (!parent || !token || !score || !ws) CKV_FAIL(CKV_EINVAL, "NULL pointer argument");
  if (score == beams->scores || (done && done == beams->done))
    CKV_FAIL(CKV_EINVAL, "the outputs must be other buffers than the beams'");
  const BeamPlan p = make_beam_plan(beams);
  if (ws_bytes < p.bytes) CKV_FAIL(CKV_EINVAL, "workspace too small: %zu < %zu", ws_bytes, p.bytes);
  if (!aligned16(ws)) CKV_FAIL(CKV_EINVAL, "pointers must be 16-byte aligned");
  {
    const int64_t rows = (int64_t)beams->n_reqs * beams->n_beams, kept = (int64_t)beams->n_reqs * beams->keep;
    const int bytes = elem_bytes(beams->dtype);
    const MemRows reads[3] = {
        MemRows{beams->logits, rows, (int64_t)beams->vocab * bytes,
                (beams->row_stride ? beams->row_stride : beams->vocab) * bytes},
        mem_array(beams->scores, rows * (int64_t)sizeof(float)), mem_array(beams->done, rows)};
    const MemRows writes[5] = {mem_array(parent, kept * (int64_t)sizeof(int32_t)),
                               mem_array(token, kept * (int64_t)sizeof(int32_t)),
                               mem_array(score, kept * (int64_t)sizeof(float)), mem_array(done, kept),
                               mem_array(ws, (int64_t)p.bytes)};
    if (writes_overlap(writes, 5, reads, 3))
      CKV_FAIL(CKV_EINVAL, "the outputs must be other buffers than each other and the beams'");
  }
  char* const w = static_cast<char*>(ws);
  const BeamArgs a{static_cast<const char*>(beams->logits), beams->scores, beams->done,
                   beams->row_stride ? beams->row_stride : beams->vocab, beams->n_reqs, beams->n_beams,
                   beams->vocab, beams->keep, beams->eos, p.slices, p.slice, reinterpret_cast<double*>(w),
                   reinterpret_cast<double*>(w + p.off_sum), reinterpret_cast<uint64_t*>(w + p.off_keys),
                   parent, token, score, done};
  const int64_t grid = (int64_t)beams->n_reqs * beams->n_beams * p.slices;
  if (grid >= kMaxScanGrid) CKV_FAIL(CKV_EUNSUPPORTED, "batch too large");
  const hipStream_t st = (hipStream_t)stream;
  const auto kernel = beams->dtype == CKV_DTYPE_BF16
                          ? (beams->vocab < 8 ? beam_scan_kernel<true, true> : beam_scan_kernel<true, false>)
                          : (beams->vocab < 4 ? beam_scan_kernel<false, true> : beam_scan_kernel<false, false>);
  hipLaunchKernelGGL(kernel, dim3((unsigned)grid), dim3(64 * kWaves), 0, st, a);
  CKV_HIP(hipGetLastError());
  const size_t lds = (size_t)a.n_beams * (a.keep * (sizeof(double) + sizeof(int32_t)) + sizeof(int32_t));
  hipLaunchKernelGGL(beam_join_kernel, dim3((unsigned)beams->n_reqs), dim3(64 * kJoinWaves), lds, st, a);
  CKV_HIP(hipGetLastError());
  return CKV_OK;
}

}  // extern "C"
