// Rows of a dense cache to and from the 8-bit one: per block of tokens and head, e4m3 codes with one power-of-two scale.
//
// Storing a block: a = largest finite magnitude of its new rows, scale 2^e with the least e for which a <= 448 * 2^e
// (no value is clipped, and half the range of the format is used at least), code = x * 2^-e rounded once.  (From 248 * 2^120
// on that is 2^128, an infinity to whoever reads it: numbers of 4 significant bits have no other neighbour there at any scale.)  A power of two costs no
// accuracy - e4m3 has 4 significant bits at every normal magnitude - and buys exactness afterwards: codes that move between blocks with
// a compression step are not rounded a second time, and the attention's bf16 operands are the stored values themselves.
// A block that already holds rows keeps the larger scale; its old codes are read and written only where the new rows
// need a larger one.
//
// Bound by memory: a row is read and written once.
#include <algorithm>
#include <type_traits>

#include "quant_dev.h"

namespace skipkv {

namespace {

constexpr int kLoadAhead = 2;  // positions of a lane that are under way together in a load (64 x 4 heads of 1152 tokens, us, 1 / 2 / 4: 106 / 95 / 102)

// A head's share of the call: positions begin .. end-1 of sequence b, whose first row is seq_off[b].
struct HeadRange {
  int begin, end, row0;
};
// False: nothing to do, or a range that does not fit (reported).
__device__ __forceinline__ bool head_range(const QuantRowsArgs &a, int lh, int b, bool report, HeadRange *out) {
  const int row0 = a.seq_off[b], room = a.seq_off[b + 1] - row0;
  const int begin = a.begin ? a.begin[(int64_t)lh * a.batch + b] : 0;
  const int64_t end = a.end ? (int64_t)a.end[(int64_t)lh * a.batch + b] : (int64_t)begin + room;
  const int64_t cap = (int64_t)a.table_stride << a.block_log2;
  const bool ok = begin >= 0 && end >= begin && end <= cap && end - begin <= room && row0 >= 0 && (int64_t)row0 + (end - begin) <= a.total_tokens;
  if (!ok && report && a.dev_status) atomicOr(a.dev_status, SKIPKV_DEV_BAD_LENGTHS);
  out->begin = begin;
  out->end = (int)end;
  out->row0 = row0;
  return ok && end > begin;
}

__device__ __forceinline__ void bad_block(const QuantRowsArgs &a) {
  if (a.dev_status) atomicOr(a.dev_status, SKIPKV_DEV_BAD_BLOCK_TABLE);
}

// grid = (x, batch, 2 * layers * heads): K of all heads, then V.  A workgroup of four waves takes kBpw blocks at a time; a wave
// holds 16 rows of a block of up to 64 slots in registers between the maximum and the conversion, 32 of one of 128.
template <int DT, int LBS>
__global__ void __launch_bounds__(256) k_quant_store(QuantRowsArgs a) {
  constexpr int BS = 1 << LBS, kWpb = BS / 16 < 4 ? BS / 16 : 4, kBpw = 4 / kWpb, kRowsW = BS / kWpb, NL = kRowsW / 4;
  constexpr int ESZ = DT == SKIPKV_BF16 ? 2 : 4;
  __shared__ float team_max[2][4];
  const int n_lh = a.n_layers * a.n_kv_heads, b = blockIdx.y;
  const bool is_v = (int)blockIdx.z >= n_lh;
  const int lh = blockIdx.z - (is_v ? n_lh : 0), l = lh / a.n_kv_heads, h = lh % a.n_kv_heads;
  HeadRange r;
  if (!head_range(a, lh, b, blockIdx.x == 0 && threadIdx.x == 0, &r)) return;
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, team = wave / kWpb, tw = wave % kWpb, piece = lane & 15;
  uint8_t *pool = static_cast<uint8_t *>(is_v ? a.v : a.k) + l * a.stride_layer + h * a.stride_head;
  uint8_t *exps = (is_v ? a.v_exp : a.k_exp) + (int64_t)lh * a.n_blocks;
  const char *src = static_cast<const char *>(is_v ? a.rv : a.rk) +
                    (l * a.r_stride_layer + h * a.r_stride_head + (int64_t)r.row0 * a.r_stride_tok) * ESZ + piece * 8 * ESZ;
  const int32_t *table = a.block_table + (int64_t)b * a.table_stride;
  const int j_end = ((r.end - 1) >> LBS) + 1;
  int par = 0;
  for (int j0 = (r.begin >> LBS) + (int)blockIdx.x * kBpw; j0 < j_end; j0 += gridDim.x * kBpw, par ^= 1) {
    const int j = j0 + team;
    const bool in = j < j_end;
    const int id = in ? table[j] : -1;
    const bool good = in && id >= 0 && id < a.n_blocks;
    if (in && !good && lane == 0) bad_block(a);
    const int t0 = j * BS + tw * kRowsW + (lane >> 4);
    float x[NL][8];
    float amax = 0.f;
#pragma unroll
    for (int i = 0; i < NL; ++i) {
      const int t = t0 + 4 * i;
      if (good && t >= r.begin && t < r.end) {
        const char *p = src + (int64_t)(t - r.begin) * a.r_stride_tok * ESZ;
        if constexpr (DT == SKIPKV_BF16) {
          const uint4 w = *reinterpret_cast<const uint4 *>(p);
          const uint32_t u[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            x[i][2 * e] = __uint_as_float(u[e] << 16);
            x[i][2 * e + 1] = __uint_as_float(u[e] & 0xFFFF0000u);
          }
        } else {
          const float4 u = reinterpret_cast<const float4 *>(p)[0], w = reinterpret_cast<const float4 *>(p)[1];
          x[i][0] = u.x, x[i][1] = u.y, x[i][2] = u.z, x[i][3] = u.w;
          x[i][4] = w.x, x[i][5] = w.y, x[i][6] = w.z, x[i][7] = w.w;
        }
      } else {
#pragma unroll
        for (int e = 0; e < 8; ++e) x[i][e] = 0.f;
      }
    }
#pragma unroll
    for (int i = 0; i < NL; ++i)
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        x[i][e] = finite_or_nan(x[i][e]);
        amax = fmaxf(amax, fabsf(x[i][e]));  // a NaN does not count
      }
    amax = row16_max(amax);
    amax = fmaxf(amax, __shfl_xor(amax, 16));
    amax = fmaxf(amax, __shfl_xor(amax, 32));
    const bool has_old = j * BS < r.begin;
    const int e_old = good && has_old ? exps[id] : 0;
    if constexpr (kWpb > 1) {
      if (lane == 0) team_max[par][wave] = amax;
      __syncthreads();  // (two buffers: the next iteration's writes are behind its own barrier's predecessor)
#pragma unroll
      for (int w = 0; w < kWpb; ++w) amax = fmaxf(amax, team_max[par][team * kWpb + w]);
    }
    if (!good) continue;
    const int need = scale_byte_for(amax), byte = has_old ? max(e_old, need) : need;
    const float inv = scale_of_byte(254 - byte);  // 2^(127 - byte)
    uint8_t *dst = pool + (int64_t)id * a.stride_block + piece * 8;
#pragma unroll
    for (int i = 0; i < NL; ++i) {
      const int t = t0 + 4 * i;
      if (t >= r.begin && t < r.end) {
        uint2 w;
        w.x = to_e4m3<true>(x[i][2] * inv, x[i][3] * inv, to_e4m3<false>(x[i][0] * inv, x[i][1] * inv, 0));
        w.y = to_e4m3<true>(x[i][6] * inv, x[i][7] * inv, to_e4m3<false>(x[i][4] * inv, x[i][5] * inv, 0));
        *reinterpret_cast<uint2 *>(dst + (int64_t)(t & (BS - 1)) * a.stride_tok) = w;
      }
    }
    if (has_old && byte > e_old) {
      const float shrink = scale_of_byte((uint32_t)max(127 + e_old - byte, 1));  // at 2^-126 every code becomes 0 as it should
#pragma unroll 1
      for (int t = t0; t < min(r.begin, j * BS + (tw + 1) * kRowsW); t += 4) {
        uint2 *p = reinterpret_cast<uint2 *>(dst + (int64_t)(t & (BS - 1)) * a.stride_tok);
        const uint2 c = *p;
        uint32_t w[2] = {c.x, c.y};
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          const uint32_t lo = e4m3_to_bf16x2<false>(w[e], shrink), hi = e4m3_to_bf16x2<true>(w[e], shrink);
          w[e] = to_e4m3<true>(__uint_as_float(hi << 16), __uint_as_float(hi & 0xFFFF0000u),
                               to_e4m3<false>(__uint_as_float(lo << 16), __uint_as_float(lo & 0xFFFF0000u), 0));
        }
        *p = make_uint2(w[0], w[1]);
      }
    }
    if (tw == 0 && lane == 0) exps[id] = (uint8_t)byte;
  }
}

// grid = (x, batch, 2 * layers * heads / HW).  A lane writes 16 bytes: 16 lanes per bf16 row, 32 per fp32 row.  HW heads side by side,
// whose rows of a slot are neighbours in memory; kLoadAhead positions of a lane are under way at a time.
template <int DT, int HW>
__global__ void __launch_bounds__(256) k_quant_load(QuantRowsArgs a) {
  constexpr int ESZ = DT == SKIPKV_BF16 ? 2 : 4, kCodes = 16 / ESZ, kLanes = kD / kCodes, kPos = 256 / kLanes / HW, kAhead = kLoadAhead;
  const int n_lh = a.n_layers * a.n_kv_heads, b = blockIdx.y;
  const bool is_v = (int)blockIdx.z >= n_lh / HW;
  const int row = threadIdx.x / kLanes, piece = threadIdx.x % kLanes, pos = row / HW;
  const int lh = (blockIdx.z - (is_v ? n_lh / HW : 0)) * HW + row % HW, l = lh / a.n_kv_heads, h = lh - l * a.n_kv_heads;
  HeadRange r;
  if (!head_range(a, lh, b, blockIdx.x == 0 && pos == 0 && piece == 0, &r)) return;
  const uint8_t *pool = static_cast<const uint8_t *>(is_v ? a.v : a.k) + l * a.stride_layer + h * a.stride_head + piece * kCodes;
  const uint8_t *exps = (is_v ? a.v_exp : a.k_exp) + (int64_t)lh * a.n_blocks;
  char *dst = static_cast<char *>(const_cast<void *>(is_v ? a.rv : a.rk)) +
              (l * a.r_stride_layer + h * a.r_stride_head + (int64_t)r.row0 * a.r_stride_tok) * ESZ + piece * 16;
  const int32_t *table = a.block_table + (int64_t)b * a.table_stride;
  const int mask = (1 << a.block_log2) - 1;
  bool bad = false;
  for (int64_t t0 = r.begin + (int64_t)blockIdx.x * (kAhead * kPos) + pos; t0 < r.end; t0 += (int64_t)gridDim.x * (kAhead * kPos)) {
    uint32_t w[kAhead][2], e[kAhead];
    bool in[kAhead];
#pragma unroll
    for (int i = 0; i < kAhead; ++i) {
      const int64_t t = t0 + i * kPos;
      int id = t < r.end ? table[t >> a.block_log2] : -1;
      in[i] = id >= 0 && id < a.n_blocks;
      bad |= t < r.end && !in[i];
      if (in[i]) {
        const uint8_t *p = pool + (int64_t)id * a.stride_block + (int64_t)((int)t & mask) * a.stride_tok;
        w[i][0] = *reinterpret_cast<const uint32_t *>(p);
        if constexpr (kCodes == 8) w[i][1] = *reinterpret_cast<const uint32_t *>(p + 4);
        e[i] = exps[id];
      }
    }
#pragma unroll
    for (int i = 0; i < kAhead; ++i) {
      if (!in[i]) continue;
      const float s = scale_of_byte(e[i]);
      float x[kCodes];
#pragma unroll
      for (int k = 0; k < kCodes / 4; ++k) {  // codes to fp32 first: the product with the scale is the one rounding
        const uint32_t lo = e4m3_to_bf16x2<false>(w[i][k], 1.f), hi = e4m3_to_bf16x2<true>(w[i][k], 1.f);
        x[4 * k] = __uint_as_float(lo << 16) * s;
        x[4 * k + 1] = __uint_as_float(lo & 0xFFFF0000u) * s;
        x[4 * k + 2] = __uint_as_float(hi << 16) * s;
        x[4 * k + 3] = __uint_as_float(hi & 0xFFFF0000u) * s;
      }
      char *o = dst + (t0 + i * kPos - r.begin) * a.r_stride_tok * ESZ;
      if constexpr (DT == SKIPKV_BF16)
        *reinterpret_cast<uint4 *>(o) = make_uint4(pack_bf16x2(x[0], x[1]), pack_bf16x2(x[2], x[3]), pack_bf16x2(x[4], x[5]), pack_bf16x2(x[6], x[7]));
      else
        *reinterpret_cast<float4 *>(o) = make_float4(x[0], x[1], x[2], x[3]);
    }
  }
  if (bad) bad_block(a);
}

// Workgroups along a sequence: as many as its share of the rows asks for, at least one, some `all` in the call.  They walk the
// sequence in steps of the grid, so that one sequence may be much longer than the mean.
unsigned along(const QuantRowsArgs &a, int64_t columns, int64_t rows_per_wg, int64_t all) {
  const int64_t longest = (a.total_tokens + rows_per_wg - 1) / rows_per_wg + 1;
  return (unsigned)std::max<int64_t>(1, std::min(longest, (all + columns - 1) / columns));
}

}  // namespace

hipError_t launch_quant_store(const QuantRowsArgs &a, hipStream_t st) {
  auto go = [&](auto dt, auto lbs) {
    constexpr int DT = decltype(dt)::value, LBS = decltype(lbs)::value;
    const int heads = 2 * a.n_layers * a.n_kv_heads;
    // 16 x 8 heads of 2048-16384 tokens, us, with 2048 / 8192 / 16384 / 32768 workgroups: 253 / 191 / 181 / 179
    const dim3 grid(along(a, (int64_t)heads * a.batch, std::max(64, 1 << LBS), 32768), a.batch, heads);
    hipLaunchKernelGGL((k_quant_store<DT, LBS>), grid, dim3(256), 0, st, a);
  };
  auto of_size = [&](auto dt) {
    switch (a.block_log2) {
      case 4: go(dt, std::integral_constant<int, 4>{}); break;
      case 5: go(dt, std::integral_constant<int, 5>{}); break;
      case 6: go(dt, std::integral_constant<int, 6>{}); break;
      default: go(dt, std::integral_constant<int, 7>{}); break;
    }
  };
  if (a.dtype == SKIPKV_BF16) of_size(std::integral_constant<int, SKIPKV_BF16>{});
  else of_size(std::integral_constant<int, SKIPKV_F32>{});
  return hipGetLastError();
}

hipError_t launch_quant_load(const QuantRowsArgs &a, hipStream_t st) {
  auto go = [&](auto dt, auto hw) {
    constexpr int DT = decltype(dt)::value, HW = decltype(hw)::value;
    const int groups = 2 * a.n_layers * a.n_kv_heads / HW;
    const dim3 grid(along(a, (int64_t)groups * a.batch, kLoadAhead * 256 / (DT == SKIPKV_BF16 ? 16 : 32) / HW, 16384), a.batch, groups);
    hipLaunchKernelGGL((k_quant_load<DT, HW>), grid, dim3(256), 0, st, a);
  };
  auto of_heads = [&](auto dt) {
    if (a.n_kv_heads % 4 == 0) go(dt, std::integral_constant<int, 4>{});
    else if (a.n_kv_heads % 2 == 0) go(dt, std::integral_constant<int, 2>{});
    else go(dt, std::integral_constant<int, 1>{});
  };
  if (a.dtype == SKIPKV_BF16) of_heads(std::integral_constant<int, SKIPKV_BF16>{});
  else of_heads(std::integral_constant<int, SKIPKV_F32>{});
  return hipGetLastError();
}

}  // namespace skipkv
