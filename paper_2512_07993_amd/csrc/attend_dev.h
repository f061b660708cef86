// Device-side helpers shared by the two attention kernels over the 8-bit cache.
#pragma once

#include "quant_dev.h"

namespace skipkv {

constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;
constexpr float kSlack = 8.f;  // the reference may lag behind the maximum by this much (log2): weights up to 2^8, no less accurate

__device__ __forceinline__ float nan32() { return __uint_as_float(0x7FC00000u); }

// Keys that query row r_last of a head sees, of n keys of a sequence with m query tokens; the rows before it see no more.
__device__ __forceinline__ int rows_see(const AttendArgs &a, int m, int n, int r_last) {
  return max(0, min(n, n - m + r_last / a.group + 1));
}
__device__ __forceinline__ bool seq_queries(const AttendArgs &a, int b, int *q0, int *m) {
  const int lo = a.q_off[b], hi = a.q_off[b + 1];
  *q0 = lo;
  *m = hi - lo;
  return lo >= 0 && hi >= lo && hi <= a.total_q && hi - lo <= a.max_q;
}
__device__ __forceinline__ bool length_ok(const AttendArgs &a, int n) {
  return n >= 0 && n <= a.max_len && n <= (a.table_stride << a.block_log2);
}

__device__ __forceinline__ int lanes_before_and_here(int v) {  // inclusive prefix sum over the wave
#define SKIPKV_ROW_STEP(CTRL, ROWS) v += __builtin_amdgcn_update_dpp(0, v, CTRL, ROWS, 0xf, true)
  SKIPKV_ROW_STEP(0x111, 0xf);  // within rows of 16 lanes: from 1, 2, 4 and 8 lanes before
  SKIPKV_ROW_STEP(0x112, 0xf);
  SKIPKV_ROW_STEP(0x114, 0xf);
  SKIPKV_ROW_STEP(0x118, 0xf);
  SKIPKV_ROW_STEP(0x142, 0xa);  // the sums of rows 0 and 2 for the rows behind them, then that of the first two
  SKIPKV_ROW_STEP(0x143, 0xc);
#undef SKIPKV_ROW_STEP
  return v;
}
// x as a sum of N bf16 numbers, the rest of each in the next; pairs of x, y packed.
template <int N>
__device__ __forceinline__ void split_bf16(float x, float y, uint32_t (&out)[N]) {
#pragma unroll
  for (int i = 0; i < N; ++i) {
    out[i] = pack_bf16x2(x, y);
    if (i + 1 < N) {
      x -= __uint_as_float(out[i] << 16);
      y -= __uint_as_float(out[i] & 0xFFFF0000u);
    }
  }
}
__device__ __forceinline__ bf16x8 frag(uint32_t a, uint32_t b, uint32_t c, uint32_t d) { return __builtin_bit_cast(bf16x8, make_uint4(a, b, c, d)); }

// Codes that are no finite bf16 number: NaN (0x7F, 0xFF) and, with a block's scale byte e from 247 on, what reaches 2^128 (from code 256 =
// 0x78 on at 2^120, eight codes fewer for each further power).  room_of: what their magnitudes lack to 0x80, in every byte.
__device__ __forceinline__ uint32_t room_of(uint32_t e) { return 0x01010101u * (e < 247u ? 1u : 8u * (e - 246u)); }
__device__ __forceinline__ uint32_t over_bits(uint32_t w, uint32_t room) { return ((w & 0x7F7F7F7Fu) + room) & 0x80808080u; }  // (at most 0x7F + 72: no carry leaves a byte)
// Their bytes, as 0xFF.
__device__ __forceinline__ uint32_t infinite_bytes(uint32_t w, uint32_t room) {
  const uint32_t high = over_bits(w, room);
  return (high << 1) - (high >> 7);
}

// Four dimensions of a finished row (d = 0: and its lse): v / all, rounded once.
template <int DT>
__device__ __forceinline__ void store_row(const AttendArgs &a, int tok, int head, int d, float4 v, float top, float all) {
  const bool none = all == 0.f;  // the row sees no key
  const float f = none ? 0.f : 1.f / all;
  const float4 y = none ? make_float4(0.f, 0.f, 0.f, 0.f) : make_float4(v.x * f, v.y * f, v.z * f, v.w * f);
  const int64_t at = tok * a.out_stride_tok + head * a.out_stride_head + d;
  if constexpr (DT == SKIPKV_BF16) *reinterpret_cast<uint2 *>(static_cast<uint16_t *>(a.out) + at) = make_uint2(pack_bf16x2(y.x, y.y), pack_bf16x2(y.z, y.w));
  else *reinterpret_cast<float4 *>(static_cast<float *>(a.out) + at) = y;
  if (d == 0 && a.lse) a.lse[(int64_t)tok * a.n_kv_heads * a.group + head] = none ? -__builtin_inff() : (top + log2f(all)) * kLn2;
}

}  // namespace skipkv
