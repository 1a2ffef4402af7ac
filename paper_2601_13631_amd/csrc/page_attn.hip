// page_attn.hip -- attention over a paged KV cache for gfx950: decoding and prefill,
// a sliding window with the first tokens kept visible, pages in fp32, bf16 or 8 bits.
//
// For a query at position p of its sequence and the keys j that it sees,
//   out = sum_j exp(s_j - m) v_j / sum_j exp(s_j - m),  s_j = sm_scale q.k_j,
// for any reference m.  A key is seen if j <= p, its page is there, and (window > 0)
// j > p - window or j < n_sinks.

#include "pages_internal.h"

namespace ckv {
namespace {

constexpr int kTile = 32;  // keys per step of a wave
constexpr int kRows = 16;  // query rows (query x head of one KV head) per workgroup
constexpr int kWaves = 4;
constexpr float kNone = -3.4028234663852886e38f;  // reference of a row that has seen no key
// A row's reference follows its maximum once that is 8 log2 units above it: sums and
// outputs stay below 2^8 times what the maximum itself would give, and a rescaling
// of the outputs is rare.
constexpr float kSlack = 8.f;

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
  int c, log2c;         // log2c: -1 if c is no power of two
  int Hkv, Hq, G;
  int window, sinks, n_splits;
  float c1;
};

// The keys of a block of rows as steps of kTile: those that hold the sinks, then those
// from the window's begin on.
struct Steps {
  int n_sink, first, n;  // step i: tile i < n_sink ? i : first + i - n_sink
  __device__ __forceinline__ int tile(int i) const { return i < n_sink ? i : first + (i - n_sink); }
};
// For queries at positions p0 .. p1 of a sequence with keys below kv_end.
__device__ __forceinline__ Steps steps_of(const PageAttnArgs& a, int p0, int p1, int kv_end) {
  Steps s{0, 0, 0};
  const int hi = min(p1 + 1, kv_end);
  if (hi <= 0) return s;
  const int tiles = (hi + kTile - 1) / kTile;
  if (a.window > 0) {
    const int lo = max(p0 - a.window + 1, 0);
    s.n_sink = (min(min(a.sinks, lo), hi) + kTile - 1) / kTile;
    s.first = max(lo / kTile, s.n_sink);
  }
  s.n = s.n_sink + max(tiles - s.first, 0);
  return s;
}

// Page and row inside it of the key at position pos of sequence table `tab`; page -1
// where there is none.
__device__ __forceinline__ int page_of(const PageAttnArgs& a, const int32_t* tab, int slot) {
  const int page = slot < a.s.max_pages ? tab[slot] : -1;
  return page >= 0 && page < a.n_pages ? page : -1;
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

__device__ __forceinline__ uint32_t bf16_pair(float x, float y) {
  const bf16x2 b = {(__bf16)x, (__bf16)y};
  return __builtin_bit_cast(uint32_t, b);
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

// Few rows: a workgroup owns 16 query rows of one KV head and one split of their
// steps, each wave every fourth step of it, straight from memory to registers:
//   S^T = K Q^T    MFMA 16x16 (bf16: x32, fp32: x4), two groups of 16 keys; lane l
//                  then holds row l % 16 and keys 4 (l / 16) + 0..3 of each group
//   O^T += V^T P^T the contraction's 8 (bf16) keys per lane are those it holds, so
//                  P^T goes from the softmax registers to the MFMA as it is; lane l
//                  loads D/16 elements from l % 16 * D/16 on of its 8 keys' V rows, and
//                  product i of D/16 takes element i of each (8 keys x D/16 elements
//                  are turned over in registers).
// The waves' outputs are joined through LDS, the splits' by page_combine_kernel.
template <int D, int T>
__global__ __launch_bounds__(64 * kWaves) void page_rows_kernel(PageAttnArgs a) {
  using E = Elem<T>;
  using QT = typename E::Q;
  constexpr bool kF32 = T == CKV_DTYPE_F32, kE4 = T == CKV_DTYPE_E4M3;
  constexpr int kVec = D / 16;                    // elements of a V row per lane, and products of O
  constexpr int kPieces = D * E::kBytes / 64;     // 16-byte pieces of a K row per lane
  constexpr int kVWords = kVec * E::kBytes / 4;   // dwords of a V row per lane

  const int split = (int)(blockIdx.x / a.Hkv) % a.n_splits, g = (int)(blockIdx.x % a.Hkv);
  const int b = (int)(blockIdx.x / ((uint32_t)a.Hkv * a.n_splits));
  const int lane = threadIdx.x & 63, n16 = lane & 15, j4 = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const SeqSpan sp = seq_span(a.s, b);
  if (sp.count == 0) return;
  const int32_t* tab = a.s.table + (int64_t)b * a.s.table_stride;
  const int kv_end = (int)min<int64_t>(max(sp.len, 0), (int64_t)a.s.max_pages * a.c);
  const int row_bytes = a.Hkv * D * E::kBytes;
  const int64_t rows = (int64_t)sp.count * a.G;

  __shared__ float lds_o[kWaves][kRows][D + 4];
  __shared__ float2 lds_ml[kWaves][kRows];

  for (int64_t rb = blockIdx.y; rb * kRows < rows; rb += gridDim.y) {
    const int64_t r_first = rb * kRows, r_last = min<int64_t>(rows, r_first + kRows) - 1;
    const int p_base = sp.len - sp.count;
    const int p0 = p_base + (int)(r_first / a.G), p1 = p_base + (int)(r_last / a.G);
    const Steps steps = steps_of(a, p0, p1, kv_end);
    const int begin = (int)((int64_t)steps.n * split / a.n_splits);
    const int end = (int)((int64_t)steps.n * (split + 1) / a.n_splits);

    // this lane's row: its query (position p) and head
    const int64_t r = min<int64_t>(r_first + n16, r_last);
    const int64_t tok = sp.first + r / a.G;
    const int head = g * a.G + (int)(r % a.G), p = p_base + (int)(r / a.G);
    const QT* q = static_cast<const QT*>(a.q) + (tok * a.Hq + head) * D;
    // Q^T operands in the order of the K pieces
    f32x4 qf[kF32 ? kPieces : 1];
    bf16x8 qb[kF32 ? 1 : D / 32];
    if constexpr (kF32) {
#pragma unroll
      for (int i = 0; i < kPieces; ++i) qf[i] = *reinterpret_cast<const f32x4*>(q + 16 * i + 4 * j4);
    } else if constexpr (kE4) {
#pragma unroll
      for (int i = 0; i < D / 32; ++i)
        qb[i] = *reinterpret_cast<const bf16x8*>(q + 64 * (i >> 1) + 16 * j4 + 8 * (i & 1));
    } else {
#pragma unroll
      for (int i = 0; i < D / 32; ++i) qb[i] = *reinterpret_cast<const bf16x8*>(q + 32 * i + 8 * j4);
    }

    f32x4 o[kVec];
#pragma unroll
    for (int i = 0; i < kVec; ++i) o[i] = f32x4{0.f, 0.f, 0.f, 0.f};
    float ref = kNone, l = 0.f;

    for (int st = begin + wave; st < end; st += kWaves) {
      const int tile = steps.tile(st), pos0 = tile * kTile;
      // pages of this lane's keys: K rows 16 i + n16, V rows 16 i + 4 j4 + 0..3
      int kp[2], vp[2], kr[2], vr[2];
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const int pos = pos0 + 16 * i;
        if (a.c >= 16) {
          const int slot = a.log2c >= 0 ? pos >> a.log2c : (int)((uint32_t)pos / (uint32_t)a.c);
          kp[i] = vp[i] = page_of(a, tab, slot);
          kr[i] = pos - slot * a.c + n16;
          vr[i] = pos - slot * a.c + 4 * j4;
        } else {
          kp[i] = page_of(a, tab, (pos + n16) >> 3);
          vp[i] = page_of(a, tab, (pos + 4 * j4) >> 3);
          kr[i] = n16 & 7;
          vr[i] = (4 * j4) & 7;
        }
      }
      // a key that is not there reads page 0 and counts for nothing
      u32x4 kw[2][kPieces];
      uint32_t vw[2][4][kVWords];
      float ks[2], vs[2];
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const char* kr_at = a.k + (int64_t)max(kp[i], 0) * a.page_stride +
                            (int64_t)kr[i] * row_bytes + g * D * E::kBytes + 16 * j4;
#pragma unroll
        for (int x = 0; x < kPieces; ++x) kw[i][x] = *reinterpret_cast<const u32x4*>(kr_at + 64 * x);
        const char* vr_at = a.v + (int64_t)max(vp[i], 0) * a.page_stride +
                            (int64_t)vr[i] * row_bytes + (g * D + n16 * kVec) * E::kBytes;
#pragma unroll
        for (int y = 0; y < 4; ++y) {
          if constexpr (kVWords == 4)
            *reinterpret_cast<u32x4*>(vw[i][y]) = *reinterpret_cast<const u32x4*>(vr_at + y * row_bytes);
          else if constexpr (kVWords == 2)
            *reinterpret_cast<uint2*>(vw[i][y]) = *reinterpret_cast<const uint2*>(vr_at + y * row_bytes);
          else
            vw[i][y][0] = *reinterpret_cast<const uint32_t*>(vr_at + y * row_bytes);
        }
        if constexpr (kE4) {
          ks[i] = scale_of(a.k_scale[(int64_t)max(kp[i], 0) * a.Hkv + g]);
          vs[i] = scale_of(a.v_scale[(int64_t)max(vp[i], 0) * a.Hkv + g]);
        }
      }
      // logits
      f32x4 s[2];
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        s[i] = f32x4{0.f, 0.f, 0.f, 0.f};
        if constexpr (kF32) {
#pragma unroll
          for (int x = 0; x < kPieces; ++x)
#pragma unroll
            for (int e = 0; e < 4; ++e)
              s[i] = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(kw[i][x][e]), qf[x][e], s[i], 0, 0, 0);
        } else if constexpr (kE4) {
#pragma unroll
          for (int x = 0; x < D / 32; ++x)
            s[i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(
                bf16_of_codes(kw[i][x >> 1][2 * (x & 1)], kw[i][x >> 1][2 * (x & 1) + 1], ks[i]), qb[x],
                s[i], 0, 0, 0);
        } else {
#pragma unroll
          for (int x = 0; x < D / 32; ++x)
            s[i] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, kw[i][x]), qb[x],
                                                           s[i], 0, 0, 0);
        }
      }
      // what some row of the block must not see
      const int last = pos0 + kTile;
      const bool all = last <= min(p0 + 1, kv_end) &&
                       (a.window <= 0 || pos0 > p1 - a.window || last <= a.sinks);
      if (!all || __any(vp[0] < 0 || vp[1] < 0)) {
        const int lo = a.window > 0 ? p0 - a.window : -1;  // the block's first row sees keys past it
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
          for (int y = 0; y < 4; ++y) {
            const int pos = pos0 + 16 * i + 4 * j4 + y;
            const bool there = vp[i] >= 0 && pos < kv_end;
            if (!(there && pos <= p && (a.window <= 0 || pos > p - a.window || pos < a.sinks)))
              s[i][y] = -INFINITY;
            // a weight of 0 does not undo a NaN: rows that no query of the block sees are cleared
            if (!(there && pos <= p1 && (pos > lo || pos < a.sinks)))
#pragma unroll
              for (int w = 0; w < kVWords; ++w) vw[i][y][w] = 0u;
          }
      }
      float mx = -INFINITY;
#pragma unroll
      for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int y = 0; y < 4; ++y) {
          s[i][y] *= a.c1;
          mx = fmaxf(mx, s[i][y]);
        }
      if (__any(mx > ref + kSlack)) {
        mx = fmaxf(mx, __shfl_xor(mx, 16));
        mx = fmaxf(mx, __shfl_xor(mx, 32));
        const float to = fmaxf(mx, ref), f = __builtin_amdgcn_exp2f(ref - to);
        ref = to;
        l *= f;
#pragma unroll
        for (int i = 0; i < kVec; ++i) o[i] *= f;
      }
#pragma unroll
      for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int y = 0; y < 4; ++y) {
          s[i][y] = __builtin_amdgcn_exp2f(s[i][y] - ref);
          l += s[i][y];
        }
      if constexpr (kF32) {
#pragma unroll
        for (int i = 0; i < 2; ++i)
#pragma unroll
          for (int y = 0; y < 4; ++y)
#pragma unroll
            for (int x = 0; x < kVec; ++x)
              o[x] = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(vw[i][y][x]), s[i][y], o[x], 0, 0, 0);
      } else {
        u32x4 pb;
#pragma unroll
        for (int i = 0; i < 4; ++i) pb[i] = bf16_pair(s[i >> 1][2 * (i & 1)], s[i >> 1][2 * (i & 1) + 1]);
#pragma unroll
        for (int x = 0; x < kVec; ++x) {
          u32x4 vt;  // element x of the 8 keys
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const uint32_t* r0 = vw[i >> 1][2 * (i & 1)];
            const uint32_t* r1 = vw[i >> 1][2 * (i & 1) + 1];
            if constexpr (kE4) {
              // codes of elements 2 (x / 2) and + 1 of both keys, then the pair of element x
              const uint32_t w = __builtin_amdgcn_perm(r1[x >> 2], r0[x >> 2], x & 2 ? 0x07030602u : 0x05010400u);
              vt[i] = __builtin_bit_cast(
                  uint32_t, x & 1 ? __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, vs[i >> 1], true)
                                  : __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, vs[i >> 1], false));
            } else {
              vt[i] = __builtin_amdgcn_perm(r1[x >> 1], r0[x >> 1], x & 1 ? 0x07060302u : 0x05040100u);
            }
          }
          o[x] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, vt),
                                                         __builtin_bit_cast(bf16x8, pb), o[x], 0, 0, 0);
        }
      }
    }

    l += __shfl_xor(l, 16);
    l += __shfl_xor(l, 32);
    if (rb > (int64_t)blockIdx.y) __syncthreads();  // the last block's rows have been read
    // o[x][v] holds element kVec (4 j4 + v) + x of row n16
#pragma unroll
    for (int v = 0; v < 4; ++v)
#pragma unroll
      for (int x = 0; x < kVec; ++x) lds_o[wave][n16][kVec * (4 * j4 + v) + x] = o[x][v];
    if (lane < kRows) lds_ml[wave][lane] = make_float2(ref, l);
    __syncthreads();
    // 16 threads per row, D / 16 elements each
    const int row = threadIdx.x >> 4, col = (threadIdx.x & 15) * kVec;
    const int64_t rr = r_first + row;
    if (rr <= r_last) {
      float M = kNone, L = 0.f, f[kWaves], acc[kVec];
#pragma unroll
      for (int w = 0; w < kWaves; ++w) M = fmaxf(M, lds_ml[w][row].x);
#pragma unroll
      for (int w = 0; w < kWaves; ++w) {
        f[w] = __builtin_amdgcn_exp2f(lds_ml[w][row].x - M);
        L += f[w] * lds_ml[w][row].y;
      }
#pragma unroll
      for (int x = 0; x < kVec; ++x) {
        acc[x] = 0.f;
#pragma unroll
        for (int w = 0; w < kWaves; ++w) acc[x] += f[w] * lds_o[w][row][col + x];
      }
      const int64_t at = (sp.first + rr / a.G) * a.Hq + g * a.G + rr % a.G;
      if (a.n_splits > 1) {
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
}

// Joins the splits of each row in split order.  D / 4 threads per row.
template <int D, class QT>
__global__ __launch_bounds__(256) void page_combine_kernel(PageAttnArgs a) {
  const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x, row = i / (D / 4);
  const int col = (int)(i % (D / 4)) * 4;
  const int64_t n_rows = a.s.n_tokens * a.Hq, tok = row / a.Hq;
  if (row >= n_rows) return;
  if (tok < a.s.tok_off[0] || tok >= a.s.tok_off[a.s.n_seqs]) return;  // of no sequence
  float M = kNone, L = 0.f;
  f32x4 acc{0.f, 0.f, 0.f, 0.f};
  constexpr int kBatch = 8;  // splits whose loads are in flight together
  for (int s0 = 0; s0 < a.n_splits; s0 += kBatch) {
    float2 ml[kBatch];
    f32x4 x[kBatch];
#pragma unroll
    for (int k = 0; k < kBatch; ++k) {
      const int64_t at = (int64_t)min(s0 + k, a.n_splits - 1) * n_rows + row;
      ml[k] = a.ml_part[at];
      x[k] = *reinterpret_cast<const f32x4*>(a.o_part + at * D + col);
    }
#pragma unroll
    for (int k = 0; k < kBatch; ++k) {
      if (s0 + k >= a.n_splits || !(ml[k].y > 0.f)) continue;
      const float to = fmaxf(M, ml[k].x);
      const float f = __builtin_amdgcn_exp2f(M - to), w = __builtin_amdgcn_exp2f(ml[k].x - to);
      M = to;
      L = L * f + ml[k].y * w;
      acc = acc * f + x[k] * w;
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

struct PageAttnPlan {
  int n_splits;
  int row_blocks;  // grid y
  size_t off_ml, bytes;
};

PageAttnPlan make_plan(const ckv_page_pool* pool, const ckv_page_batch* b, int Hq, int window, int sinks) {
  PageAttnPlan p{};
  const int G = Hq / pool->n_kv_heads;
  const int64_t most = b->max_tokens > 0 ? std::min<int64_t>(b->max_tokens, b->n_tokens) : b->n_tokens;
  p.row_blocks = (int)std::min<int64_t>(65535, std::max<int64_t>(1, ceil_div(most * G, kRows)));
  int64_t len = (int64_t)b->max_pages * pool->page_size;
  if (b->max_len > 0) len = std::min<int64_t>(len, b->max_len);
  if (window > 0) len = std::min<int64_t>(len, (int64_t)window + most + sinks + 2 * kTile);
  const int64_t steps = ceil_div(len, kTile), wgs = (int64_t)b->n_seqs * pool->n_kv_heads * p.row_blocks;
  p.n_splits = (int)std::max<int64_t>(1, std::min(1024 / std::max<int64_t>(wgs, 1), steps / 8));
  const size_t rows = (size_t)b->n_tokens * Hq;
  if (p.n_splits > 1) {
    p.off_ml = align_up((size_t)p.n_splits * rows * pool->head_dim * sizeof(float), 256);
    p.bytes = align_up(p.off_ml + (size_t)p.n_splits * rows * sizeof(float2), 256);
  }
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

template <int D, int T>
ckv_status launch_page_attn(const PageAttnArgs& a, const PageAttnPlan& p, hipStream_t st) {
  const int64_t wgs = (int64_t)a.s.n_seqs * a.Hkv * a.n_splits;
  if (wgs >= kMaxGrid) CKV_FAIL(CKV_EUNSUPPORTED, "batch too large");
  hipLaunchKernelGGL((page_rows_kernel<D, T>), dim3((unsigned)wgs, (unsigned)p.row_blocks),
                     dim3(64 * kWaves), 0, st, a);
  CKV_HIP(hipGetLastError());
  if (a.n_splits > 1) {
    const int64_t blocks = ceil_div(a.s.n_tokens * a.Hq * (D / 4), 256);
    hipLaunchKernelGGL((page_combine_kernel<D, typename Elem<T>::Q>), dim3((unsigned)blocks), dim3(256),
                       0, st, a);
    CKV_HIP(hipGetLastError());
  }
  return CKV_OK;
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
  if (!(sm_scale >= 0.f) || std::isinf(sm_scale)) CKV_FAIL(CKV_EINVAL, "sm_scale must be finite and >= 0");
  if (batch->n_seqs == 0 || batch->n_tokens == 0) return CKV_OK;
  if (!q || !out) CKV_FAIL(CKV_EINVAL, "NULL pointer argument");
  if (!aligned16(q) || !aligned16(out) || !aligned16(ws))
    CKV_FAIL(CKV_EINVAL, "pointers must be 16-byte aligned");
  if (batch->n_tokens * n_q_heads > (int64_t(1) << 26))
    CKV_FAIL(CKV_EUNSUPPORTED, "more than 2^26 query rows in one call");
  const PageAttnPlan p = make_plan(pool, batch, n_q_heads, window, n_sinks);
  if (p.bytes && (!ws || ws_bytes < p.bytes))
    CKV_FAIL(CKV_EINVAL, "workspace too small: %zu < %zu", ws ? ws_bytes : (size_t)0, p.bytes);
  PageAttnArgs a;
  a.s = page_seqs(batch);
  a.k = static_cast<const char*>(pool->k);
  a.v = static_cast<const char*>(pool->v);
  a.k_scale = pool->k_scale;
  a.v_scale = pool->v_scale;
  a.page_stride = page_stride_bytes(pool);
  a.n_pages = pool->n_pages;
  a.q = q;
  a.out = out;
  a.o_part = static_cast<float*>(ws);
  a.ml_part = p.bytes ? reinterpret_cast<float2*>(static_cast<char*>(ws) + p.off_ml) : nullptr;
  a.c = pool->page_size;
  a.log2c = (a.c & (a.c - 1)) == 0 ? __builtin_ctz(a.c) : -1;
  a.Hkv = pool->n_kv_heads;
  a.Hq = n_q_heads;
  a.G = n_q_heads / pool->n_kv_heads;
  a.window = window;
  a.sinks = window > 0 ? n_sinks : 0;
  a.n_splits = p.n_splits;
  a.c1 = (sm_scale > 0.f ? sm_scale : 1.0f / sqrtf((float)pool->head_dim)) * 1.4426950408889634f;
  const hipStream_t st = (hipStream_t)stream;
  if (pool->dtype == CKV_DTYPE_F32) return launch_page_attn<64, CKV_DTYPE_F32>(a, p, st);
  if (pool->dtype == CKV_DTYPE_BF16)
    return pool->head_dim == 128 ? launch_page_attn<128, CKV_DTYPE_BF16>(a, p, st)
                                 : launch_page_attn<64, CKV_DTYPE_BF16>(a, p, st);
  return pool->head_dim == 128 ? launch_page_attn<128, CKV_DTYPE_E4M3>(a, p, st)
                               : launch_page_attn<64, CKV_DTYPE_E4M3>(a, p, st);
}

}  // extern "C"
