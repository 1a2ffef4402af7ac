// attn_tile.h -- the parts of an attention tile of 128 query rows (4 waves x 32) against
// 64-key stages of K and V in LDS, which the kernels that run such tiles share.
#pragma once

#include <type_traits>
#include <utility>

#include "ckv_internal.h"

namespace ckv::tile {

constexpr int kWaves = 4;
constexpr int kWaveRows = 32;
constexpr int kBlockRows = kWaves * kWaveRows;  // 128
constexpr int kTile = 64;                       // keys per LDS stage
constexpr int kSub = 32;                        // keys per MFMA product
// MFMA row p of the K operand holds key kappa(p); afterwards register v of a
// lane in half h holds key 16*(v/8) + 8*h + v%8.
__device__ __forceinline__ int kappa(int p) {
  const int i = p >> 3, h = (p >> 2) & 1, j = p & 3;
  return 16 * (i >> 1) + 8 * h + 4 * (i & 1) + j;
}

// LDS stages hold kTile rows of D bf16, unpadded (the direct-to-LDS loads write
// lane i's 16 bytes at base + 16 i), with the 16-byte segments of a row
// permuted by an XOR that depends on the row: segment s of row r sits at
// position s ^ swz(r).  K: any 16 consecutive MFMA rows (kappa) then read one
// segment column from all 64 banks.
template <int D>
__device__ __forceinline__ int k_swz(int row) {
  return D == 128 ? (row & 15) : ((row >> 1) & 7);
}

// V: conflict-free for the transposing reads.
template <int D>
__device__ __forceinline__ int v_swz(int row) {
  if constexpr (D == 128)
    return ((row & 1) ? 4 : 0) ^ ((row & 2) ? 10 : 0);
  else
    return ((row & 1) ? 2 : 0) ^ ((row & 2) ? 4 : 0);
}
template <int D>
__device__ __forceinline__ int v_off(int row, int seg) { return row * D + ((seg ^ v_swz<D>(row)) << 3); }

__device__ __forceinline__ float partner_f(float x) {
  int v = __float_as_int(x);
  auto r = __builtin_amdgcn_permlane32_swap(v, v, false, false);
  return __int_as_float(threadIdx.x & 32 ? r[0] : r[1]);
}

// Buffer resource over `bytes` bytes from p (raw loads; offsets past the end read 0).
__device__ __forceinline__ __amdgpu_buffer_rsrc_t raw_rsrc(const void* p, uint32_t bytes) {
  return __builtin_amdgcn_make_buffer_rsrc(const_cast<void*>(p), (short)0, (int)bytes, 0x00020000);
}

// The direct-to-LDS loads of one 64-key stage: instruction p of wave w moves
// the K (or V) rows of keys p*kKeyStep + w*kRowsPerLoad .. +kRowsPerLoad-1,
// kSegs lanes per row.
template <int D>
struct Stage {
  static constexpr int kSegs = D / 8;
  static constexpr int kRowsPerLoad = 64 / kSegs;
  static constexpr int kKeyStep = kWaves * kRowsPerLoad;
  static constexpr int kPer = kTile / kKeyStep;
};

using LdsPtr = __attribute__((address_space(3))) void*;

// 16 bytes per lane from memory to lds + 16 * lane (lds is uniform).  Buffer
// loads only: a global load to LDS counts as a FLAT access, after which the
// compiler no longer counts the LDS reads in flight and waits for all of them.
__device__ __forceinline__ void buffer_to_lds(__amdgpu_buffer_rsrc_t r, uint32_t voff, uint32_t soff,
                                              uint16_t* lds) {
  __builtin_amdgcn_raw_ptr_buffer_load_lds(r, (LdsPtr)lds, 16, voff, soff, 0, 0);
}

// Every wave's stage loads have landed in LDS (and the LDS reads before this
// are done): each wave waits for its own, then for the others.
__device__ __forceinline__ void stage_barrier() {
  __builtin_amdgcn_s_waitcnt(0x0070);  // vmcnt(0) lgkmcnt(0)
  __syncthreads();
}

// K operand fragment ks of 32 keys: kfo is this lane's byte offset of segment
// `half` of its row; segment 2 ks + half sits at that offset ^ 32 ks.
template <int D>
__device__ __forceinline__ bf16x8 read_k(const uint16_t* lk, uint32_t kfo, int sub, int ks) {
  return *reinterpret_cast<const bf16x8*>(reinterpret_cast<const char*>(lk) + (kfo ^ (32u * ks)) +
                                          sub * kSub * D * 2);
}

// V^T operand fragment (kb, db) of 32 keys: voff is the byte offset for db = 0,
// that of db is voff ^ 64 db, and (sub, kb, rd) add whole rows.
template <int D>
__device__ __forceinline__ bf16x8 read_v(const uint16_t* lv, uint32_t voff, int sub, int kb, int db) {
  bf16x8 vf;
#pragma unroll
  for (int rd = 0; rd < 2; ++rd)
    *(reinterpret_cast<s16x4*>(&vf) + rd) = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
        (__attribute__((address_space(3))) s16x4*)(reinterpret_cast<const char*>(lv) +
                                                   (voff ^ (64u * db)) +
                                                   (sub * kSub + 16 * kb + 4 * rd) * D * 2));
  return vf;
}

__device__ __forceinline__ float max16(const f32x16& s) {
  float mx = s[0];
#pragma unroll
  for (int v = 1; v < 16; ++v) mx = fmaxf(mx, s[v]);
  return mx;
}

// f(0), f(1), ... with compile-time arguments.
template <class F, int... I>
__device__ __forceinline__ void for_each_of(std::integer_sequence<int, I...>, F&& f) {
  (f(std::integral_constant<int, I>{}), ...);
}
template <int N, class F>
__device__ __forceinline__ void static_for(F&& f) {
  for_each_of(std::make_integer_sequence<int, N>{}, f);
}

}  // namespace ckv::tile
