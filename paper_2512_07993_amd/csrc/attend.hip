// Attention over the 8-bit cache: for every query row r of a (sequence, KV head), out = sum_t p_t v_t with
// p = softmax(scale * q.k_t) over the keys that the row sees, in one pass over K and V with a running reference and sum.
//
// Everything is computed transposed, so that nothing has to change lanes between the two products: S^T = K Q^T leaves lane (g, c)
// of a 16 x 16 tile (g = lane / 16, c = lane % 16) with the logits of query row c for keys 4g .. 4g+3, and O^T = V^T P^T wants from that
// lane the weights of query row c for 8 keys of its choice: those of two tiles, 4g .. 4g+3 of each.  A row's reference, sum and
// rescaling stay in its lanes.
//  - K: lane (g, c) loads 16-byte pieces g and g + 4 of key c's row: 8 codes each are the lane's slice of the head
//    dimension in one matrix instruction (the order within the sum is free, Q follows it).
//  - V: lane (g, c) loads 8 codes, dimensions 8c .. 8c+7, of each of its 8 keys; byte j of those is its operand for the tile of
//    dimensions { 8m + j }: a byte permutation brings the codes of two keys together.
// So codes go from memory to registers and, converted there, straight into the matrix cores; shared memory is used
// once, to merge the waves at the end.  The conversion multiplies by the block's scale and is exact.
#include <algorithm>
#include <type_traits>

#include "quant_dev.h"

namespace skipkv {

namespace {

constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;
constexpr float kSlack = 8.f;  // the reference may lag behind the maximum by this much (log2): weights up to 2^8, no less accurate
constexpr int kOPitch = kD + 4;  // floats per row of the merge buffer: 16 rows start at different banks

// How many keys the rows r0 .. r1-1 of a head see: the last of them sees the most.
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

__device__ __forceinline__ float nan32() { return __uint_as_float(0x7FC00000u); }
// Bytes of w that are a NaN code (0x7F, 0xFF), as 0xFF.
__device__ __forceinline__ uint32_t nan_bytes(uint32_t w) {
  const uint32_t high = ((w & 0x7F7F7F7Fu) + 0x01010101u) & 0x80808080u;  // 0x7F + 1: no carry leaves a byte
  return (high >> 7) * 0xFFu;
}
__device__ __forceinline__ bool has_nan(uint32_t w) { return (((w & 0x7F7F7F7Fu) + 0x01010101u) & 0x80808080u) != 0; }

// Four dimensions of a finished row (d = 0: and its lse): v / all, rounded once.
template <int DT>
__device__ __forceinline__ void store_row(const AttendArgs &a, int tok, int head, int64_t row, int d, float4 v, float top, float all) {
  const bool none = all == 0.f;  // the row sees no key
  const float f = none ? 0.f : 1.f / all;
  const float4 y = none ? make_float4(0.f, 0.f, 0.f, 0.f) : make_float4(v.x * f, v.y * f, v.z * f, v.w * f);
  const int64_t at = tok * a.out_stride_tok + head * a.out_stride_head + d;
  if constexpr (DT == SKIPKV_BF16) *reinterpret_cast<uint2 *>(static_cast<uint16_t *>(a.out) + at) = make_uint2(pack_bf16x2(y.x, y.y), pack_bf16x2(y.z, y.w));
  else *reinterpret_cast<float4 *>(static_cast<float *>(a.out) + at) = y;
  if (d == 0 && a.lse) a.lse[row] = none ? -__builtin_inff() : (top + log2f(all)) * kLn2;
}

// 32 keys of a wave: two tiles of 16, each within one block.
struct Keys {
  uint4 k[2][2];  // [tile][piece]
  uint2 v[2][4];  // [tile][key 4g + i]
};

// DT: type of q and out.  QT: tiles of 16 query rows.  W: waves, which take the steps of 32 keys in turn.
// Accuracy: stored keys and values are bf16 numbers.  bf16 queries enter as they are; fp32 ones as three bf16 parts (24 bits).  Weights
// enter the second product as two parts (16 bits) with bf16 outputs, three with fp32 ones.  Everything else is fp32.
template <int DT, int QT, int W>
__global__ void __launch_bounds__(64 * W) k_attend(AttendArgs a) {
  constexpr int NQ = DT == SKIPKV_BF16 ? 1 : 3, NP = DT == SKIPKV_BF16 ? 2 : 3;
  constexpr int ESZ = DT == SKIPKV_BF16 ? 2 : 4;
  __shared__ __align__(16) float o_part[W][16][kOPitch];
  __shared__ float2 ml_part[W][16];
  const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63, g = lane >> 4, c = lane & 15;
  // ---- which rows and keys
  uint32_t x = blockIdx.x;
  const int h = x % a.n_kv_heads;
  x /= a.n_kv_heads;
  const int split = x % a.n_split;
  x /= a.n_split;
  const int rb = x % a.n_rb, b = x / a.n_rb;
  int q0, m;
  if (!seq_queries(a, b, &q0, &m)) {
    if (split == 0 && rb == 0 && tid == 0 && a.dev_status) atomicOr(a.dev_status, SKIPKV_DEV_BAD_LENGTHS);
    return;
  }
  const int r0 = rb * a.rows, r1 = min(r0 + a.rows, m * a.group);
  if (r0 >= r1) return;
  const int n = a.len[h * a.batch + b];
  const bool n_ok = length_ok(a, n);
  if (!n_ok) {
    if (split > 0) return;
    if (tid == 0 && a.dev_status) atomicOr(a.dev_status, SKIPKV_DEV_BAD_LENGTHS);
  }
  const int k_end_all = n_ok ? rows_see(a, m, n, r1 - 1) : 0;
  const int n_chunks = max(1, (k_end_all + a.chunk - 1) / a.chunk);
  if (split >= n_chunks) return;
  const int k_begin = split * a.chunk, k_end = min(k_end_all, k_begin + a.chunk);

  // ---- queries: lane (g, c) holds dimensions 64 i + 16 g + 8 half + (0 .. 7) of row c of every tile
  bf16x8 qf[QT][NQ][4];
  int sees[QT];  // keys that row c of the tile sees
#pragma unroll
  for (int t = 0; t < QT; ++t) {
    const int r = r0 + 16 * t + c;
    const bool in = r < r1;
    const int j = r / a.group, i = r - j * a.group;
    sees[t] = in ? n - m + j + 1 : 0x7FFFFFFF;
    const char *p = static_cast<const char *>(a.q) + ((q0 + j) * a.q_stride_tok + (h * a.group + i) * a.q_stride_head + 16 * g) * ESZ;
#pragma unroll
    for (int s = 0; s < 4; ++s) {
      uint32_t w[NQ][4] = {};
      if (in) {
        const char *src = p + (64 * (s >> 1) + 8 * (s & 1)) * ESZ;
        if constexpr (DT == SKIPKV_BF16) {
          const uint4 u = *reinterpret_cast<const uint4 *>(src);
          w[0][0] = u.x, w[0][1] = u.y, w[0][2] = u.z, w[0][3] = u.w;
        } else {
          const float4 u = reinterpret_cast<const float4 *>(src)[0], v = reinterpret_cast<const float4 *>(src)[1];
          const float f[8] = {u.x, u.y, u.z, u.w, v.x, v.y, v.z, v.w};
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            uint32_t parts[NQ];
            split_bf16(f[2 * e], f[2 * e + 1], parts);
#pragma unroll
            for (int k = 0; k < NQ; ++k) w[k][e] = parts[k];
          }
        }
      }
#pragma unroll
      for (int k = 0; k < NQ; ++k) qf[t][k][s] = frag(w[k][0], w[k][1], w[k][2], w[k][3]);
    }
  }
  const int all_see = max(0, n - m + r0 / a.group + 1);  // keys below this are seen by every row

  f32x4 o[QT][8];
  float ref[QT], sum[QT];
#pragma unroll
  for (int t = 0; t < QT; ++t) {
    ref[t] = kRefInit;
    sum[t] = 0.f;
#pragma unroll
    for (int j = 0; j < 8; ++j) o[t][j] = f32x4{0.f, 0.f, 0.f, 0.f};
  }
  const float to_log2 = a.scale * kLog2e;
  bool poison = !n_ok;

  const uint8_t *kbase = a.k + h * a.stride_head, *vbase = a.v + h * a.stride_head;
  const uint8_t *kexp = a.k_exp + (int64_t)h * a.n_blocks, *vexp = a.v_exp + (int64_t)h * a.n_blocks;
  const int32_t *table = a.block_table + (int64_t)b * a.table_stride;
  const int bmask = (1 << a.block_log2) - 1;
  const uint32_t k_lane = (uint32_t)c * (uint32_t)a.stride_tok + 16 * g;
  const uint32_t v_lane = (uint32_t)(4 * g) * (uint32_t)a.stride_tok + 8 * c;
  const int steps_all = (k_end - k_begin + 31) / 32;
  const int steps = wave < steps_all ? (steps_all - wave + W - 1) / W : 0;  // of this wave

  // Up to 32 steps at a time: lane i looks up the block of tile i & 1 of step i >> 1, and its scales.
  for (int s0 = 0; s0 < steps; s0 += 32) {
    int id = 0;
    float ks = 1.f, vs = 1.f;
    {
      const int key = k_begin + ((s0 + (lane >> 1)) * W + wave) * 32 + (lane & 1) * 16;
      if (key < k_end) {
        id = table[key >> a.block_log2];
        if (id < 0 || id >= a.n_blocks) {
          poison = true;
          id = 0;
        }
        ks = scale_of_byte(kexp[id]);
        vs = scale_of_byte(vexp[id]);
      }
    }
    auto load = [&](int s) {  // (tiles that lie behind the last key read block 0)
      Keys kv;
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        const int key = k_begin + ((s0 + s) * W + wave) * 32 + t * 16;
        const int64_t row = (int64_t)__builtin_amdgcn_readlane(id, 2 * s + t) * a.stride_block + (int64_t)(key & bmask) * a.stride_tok;
        const uint8_t *kp = kbase + row, *vp = vbase + row;
        kv.k[t][0] = *reinterpret_cast<const uint4 *>(kp + k_lane);
        kv.k[t][1] = *reinterpret_cast<const uint4 *>(kp + k_lane + 64);
#pragma unroll
        for (int i = 0; i < 4; ++i) kv.v[t][i] = *reinterpret_cast<const uint2 *>(vp + v_lane + (uint32_t)i * (uint32_t)a.stride_tok);
      }
      return kv;
    };
    const int here = min(32, steps - s0);
    Keys next = load(0);
    for (int s = 0; s < here; ++s) {
      Keys kv = next;
      if (s + 1 < here) next = load(s + 1);
      const int key0 = k_begin + ((s0 + s) * W + wave) * 32;
      const float ks2[2] = {__uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(ks), 2 * s)), __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(ks), 2 * s + 1))};
      const float vs2[2] = {__uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(vs), 2 * s)), __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(vs), 2 * s + 1))};
      const bool whole = key0 + 32 <= min(all_see, k_end);  // every row sees every key
      // ---- logits
      f32x4 acc[QT][2];
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        bf16x8 kf[4];
#pragma unroll
        for (int s4 = 0; s4 < 4; ++s4) {
          const uint4 u = kv.k[t][s4 >> 1];
          const uint32_t w0 = s4 & 1 ? u.z : u.x, w1 = s4 & 1 ? u.w : u.y;
          kf[s4] = frag(e4m3_to_bf16x2<false>(w0, ks2[t]), e4m3_to_bf16x2<true>(w0, ks2[t]), e4m3_to_bf16x2<false>(w1, ks2[t]), e4m3_to_bf16x2<true>(w1, ks2[t]));
        }
#pragma unroll
        for (int q = 0; q < QT; ++q) {
          f32x4 z = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
          for (int k = NQ - 1; k >= 0; --k)
#pragma unroll
            for (int s4 = 0; s4 < 4; ++s4) z = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf[s4], qf[q][k][s4], z, 0, 0, 0);
          acc[q][t] = z * to_log2;
        }
      }
      // ---- what is not seen
      bool v_nan = false;
      if (!whole) {
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const int key = key0 + 16 * t + 4 * g + i;
            if (key >= k_end) kv.v[t][i] = make_uint2(0, 0);
            v_nan |= has_nan(kv.v[t][i].x) || has_nan(kv.v[t][i].y);
#pragma unroll
            for (int q = 0; q < QT; ++q)
              if (key >= min(sees[q], k_end)) acc[q][t][i] = -__builtin_inff();
          }
        v_nan = __any(v_nan);
      }
      // ---- weights
      uint32_t pf[QT][NP][4];
#pragma unroll
      for (int q = 0; q < QT; ++q) {
        float top = acc[q][0][0];
#pragma unroll
        for (int i = 1; i < 8; ++i) top = fmaxf(top, acc[q][i >> 2][i & 3]);
        if (__any(top > ref[q] + kSlack)) {
          top = fmaxf(top, __shfl_xor(top, 16));
          top = fmaxf(top, __shfl_xor(top, 32));
          const float now = fmaxf(ref[q], top), f = __builtin_amdgcn_exp2f(ref[q] - now);
          ref[q] = now;
          sum[q] *= f;
#pragma unroll
          for (int j = 0; j < 8; ++j) o[q][j] *= f;
        }
        float p[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          p[i] = __builtin_amdgcn_exp2f(acc[q][i >> 2][i & 3] - ref[q]);
          sum[q] += p[i];
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          uint32_t parts[NP];
          split_bf16(p[2 * i], p[2 * i + 1], parts);
#pragma unroll
          for (int k = 0; k < NP; ++k) pf[q][k][i] = parts[k];
        }
      }
      // ---- values, and where a NaN among them is seen
      auto product = [&](auto &&use) {
#pragma unroll
        for (int half = 0; half < 2; ++half) {  // dimensions 8c + 4 half + (0 .. 3)
          uint32_t w[4][2];  // [pair of keys][two dimensions]: codes of both keys side by side
#pragma unroll
          for (int pr = 0; pr < 4; ++pr) {
            const uint2 u0 = kv.v[pr >> 1][2 * (pr & 1)], u1 = kv.v[pr >> 1][2 * (pr & 1) + 1];
            const uint32_t a0 = half ? u0.y : u0.x, a1 = half ? u1.y : u1.x;
            w[pr][0] = __builtin_amdgcn_perm(a1, a0, 0x05010400u);
            w[pr][1] = __builtin_amdgcn_perm(a1, a0, 0x07030602u);
          }
#pragma unroll
          for (int d = 0; d < 4; ++d) {
            uint32_t f[4];
#pragma unroll
            for (int pr = 0; pr < 4; ++pr) f[pr] = d & 1 ? e4m3_to_bf16x2<true>(w[pr][d >> 1], vs2[pr >> 1]) : e4m3_to_bf16x2<false>(w[pr][d >> 1], vs2[pr >> 1]);
            use(4 * half + d, frag(f[0], f[1], f[2], f[3]));
          }
        }
      };
      if (v_nan) {
        // A weight of 0 does not undo a NaN in a matrix product, so here NaN are taken out of the values and counted apart, with
        // weight 1 for the rows that see them.
        Keys clean = kv;
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            clean.v[t][i] = make_uint2(kv.v[t][i].x & ~nan_bytes(kv.v[t][i].x), kv.v[t][i].y & ~nan_bytes(kv.v[t][i].y));
            kv.v[t][i] = make_uint2(nan_bytes(kv.v[t][i].x) & 0x38383838u, nan_bytes(kv.v[t][i].y) & 0x38383838u);  // 0x38: 1.0
          }
        product([&](int j, bf16x8 vf) {
#pragma unroll
          for (int q = 0; q < QT; ++q) {
            uint32_t one[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              const int key = key0 + 16 * (i >> 1) + 4 * g + 2 * (i & 1);
              one[i] = (key < min(sees[q], k_end) ? 0x3F80u : 0u) | (key + 1 < min(sees[q], k_end) ? 0x3F800000u : 0u);
            }
            const f32x4 z = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vf, frag(one[0], one[1], one[2], one[3]), f32x4{0.f, 0.f, 0.f, 0.f}, 0, 0, 0);
#pragma unroll
            for (int i = 0; i < 4; ++i)
              if (z[i] > 0.f) o[q][j][i] = nan32();
          }
        });
        kv = clean;
      }
      product([&](int j, bf16x8 vf) {
#pragma unroll
        for (int q = 0; q < QT; ++q)
#pragma unroll
          for (int k = NP - 1; k >= 0; --k)
            o[q][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vf, frag(pf[q][k][0], pf[q][k][1], pf[q][k][2], pf[q][k][3]), o[q][j], 0, 0, 0);
      });
    }
  }
  poison = __any(poison);
  if (poison && n_ok && lane == 0 && a.dev_status) atomicOr(a.dev_status, SKIPKV_DEV_BAD_BLOCK_TABLE);

  // ---- merge of the waves, a tile of rows at a time
#pragma unroll
  for (int t = 0; t < QT; ++t) {
    if (t) __syncthreads();
    float l = sum[t];
    l += __shfl_xor(l, 16);
    l += __shfl_xor(l, 32);
    if (g == 0) ml_part[wave][c] = make_float2(ref[t], poison ? nan32() : l);
    // lane (g, c): row c, dimensions 32 g + 8 i + j
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int j4 = 0; j4 < 2; ++j4)
        *reinterpret_cast<float4 *>(&o_part[wave][c][32 * g + 8 * i + 4 * j4]) = make_float4(o[t][4 * j4][i], o[t][4 * j4 + 1][i], o[t][4 * j4 + 2][i], o[t][4 * j4 + 3][i]);
    __syncthreads();
    for (int item = tid; item < 16 * (kD / 4); item += 64 * W) {
      const int row = item / (kD / 4), d = 4 * (item % (kD / 4)), r = r0 + 16 * t + row;
      if (r >= r1) break;
      float top = kRefInit;
#pragma unroll
      for (int w = 0; w < W; ++w) top = fmaxf(top, ml_part[w][row].x);
      float all = 0.f;
      float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
      for (int w = 0; w < W; ++w) {
        const float2 ml = ml_part[w][row];
        const float f = __builtin_amdgcn_exp2f(ml.x - top);
        const float4 u = *reinterpret_cast<const float4 *>(&o_part[w][row][d]);
        all += ml.y * f;
        v.x += u.x * f, v.y += u.y * f, v.z += u.z * f, v.w += u.w * f;
      }
      const int j = r / a.group, head = h * a.group + r - j * a.group;
      const int64_t row_all = (int64_t)(q0 + j) * a.n_kv_heads * a.group + head;
      if (n_chunks > 1) {
        const int64_t at = (int64_t)split * a.total_q * a.n_kv_heads * a.group + row_all;
        *reinterpret_cast<float4 *>(a.part_o + at * kD + d) = v;
        if (d == 0) a.part_ml[at] = make_float2(top, all);
      } else {
        store_row<DT>(a, q0 + j, head, row_all, d, v, top, all);
      }
    }
  }
}

// Rows whose keys were cut into chunks: a wave per row, two dimensions per lane.
template <int DT>
__global__ void __launch_bounds__(256) k_attend_join(AttendArgs a) {
  const int n_heads = a.n_kv_heads * a.group, lane = threadIdx.x & 63;
  const int64_t rows = (int64_t)a.total_q * n_heads, row = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
  if (row >= rows) return;
  const int tok = (int)(row / n_heads), head = (int)(row - (int64_t)tok * n_heads);
  int lo = 0, hi = a.batch;  // the last sequence that begins at or before the token
  while (hi - lo > 1) {
    const int mid = (lo + hi) / 2;
    if (a.q_off[mid] <= tok) lo = mid;
    else hi = mid;
  }
  int q0, m;
  if (!seq_queries(a, lo, &q0, &m) || tok < q0 || tok >= q0 + m) return;
  const int h = head / a.group, n = a.len[h * a.batch + lo];
  if (!length_ok(a, n)) return;
  const int r = (tok - q0) * a.group + head % a.group, r1 = min((r / a.rows + 1) * a.rows, m * a.group);
  const int n_chunks = (rows_see(a, m, n, r1 - 1) + a.chunk - 1) / a.chunk;
  if (n_chunks <= 1) return;
  float top = kRefInit, all = 0.f;
  for (int s = 0; s < n_chunks; ++s) top = fmaxf(top, a.part_ml[s * rows + row].x);
  float2 v = make_float2(0.f, 0.f);
  for (int s = 0; s < n_chunks; ++s) {
    const float2 ml = a.part_ml[s * rows + row];
    const float f = __builtin_amdgcn_exp2f(ml.x - top);
    const float2 u = *reinterpret_cast<const float2 *>(a.part_o + (s * rows + row) * kD + 2 * lane);
    all += ml.y * f;
    v.x += u.x * f, v.y += u.y * f;
  }
  const float4 w = make_float4(v.x, v.y, __shfl_down(v.x, 1), __shfl_down(v.y, 1));
  if (!(lane & 1)) store_row<DT>(a, tok, head, row, 2 * lane, w, top, all);
}

}  // namespace

void plan_attend(AttendArgs *a) {
  a->rows = a->dtype == SKIPKV_BF16 && (int64_t)a->max_q * a->group > 16 ? 32 : 16;
  a->n_rb = (int32_t)(((int64_t)a->max_q * a->group + a->rows - 1) / a->rows);
  // chunks so that some 1024 workgroups work at a time, of 256 keys at least
  const int64_t columns = std::max<int64_t>(1, (int64_t)a->batch * a->n_kv_heads * a->n_rb);
  const int64_t want = std::max<int64_t>(1, 1024 / columns);
  const int64_t chunk = ((a->max_len + want - 1) / want + 255) / 256 * 256;
  a->chunk = (int32_t)std::min<int64_t>(std::max<int64_t>(chunk, 256), 1 << 30);
  a->n_split = std::max(1, (a->max_len + a->chunk - 1) / a->chunk);
}

hipError_t launch_attend(const AttendArgs &a, hipStream_t st) {
  const unsigned grid = (unsigned)((int64_t)a.batch * a.n_rb * a.n_split * a.n_kv_heads);
  if (a.dtype == SKIPKV_F32) hipLaunchKernelGGL((k_attend<SKIPKV_F32, 1, 4>), dim3(grid), dim3(256), 0, st, a);
  else if (a.rows == 16) hipLaunchKernelGGL((k_attend<SKIPKV_BF16, 1, 4>), dim3(grid), dim3(256), 0, st, a);
  else hipLaunchKernelGGL((k_attend<SKIPKV_BF16, 2, 4>), dim3(grid), dim3(256), 0, st, a);
  if (a.n_split > 1) {
    const unsigned join = (unsigned)(((int64_t)a.total_q * a.n_kv_heads * a.group + 3) / 4);
    if (a.dtype == SKIPKV_F32) hipLaunchKernelGGL(k_attend_join<SKIPKV_F32>, dim3(join), dim3(256), 0, st, a);
    else hipLaunchKernelGGL(k_attend_join<SKIPKV_BF16>, dim3(join), dim3(256), 0, st, a);
  }
  return hipGetLastError();
}

}  // namespace skipkv
