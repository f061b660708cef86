// Attention over the 8-bit cache: for every query row r of a (sequence, KV head), out = sum_t p_t v_t with
// p = softmax(scale * q.k_t) over the keys that the row sees, in one pass over K and V with a running reference and sum.
// This file: 16 or 32 rows at a time (decode, drafted tokens), where the cache's bytes are what counts.
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

#include "attend_dev.h"

namespace skipkv {

namespace {

constexpr int kOPitch = kD + 4;  // floats per row of the merge buffer: 16 rows start at different banks
constexpr int kWaves = 8;        // per workgroup; two workgroups share a CU (one with fp32 queries or 32 rows)
// 32 keys of a wave: two tiles of 16, each within one block.
struct Keys {
  uint4 k[2][2];  // [tile][piece]
};
struct Values {
  uint2 v[2][4];  // [tile][key 4g + i]
};

// The 8 operands (tiles of dimensions { 8m + j }) that a wave's values make.
template <class Use>
__device__ __forceinline__ void value_frags(const Values &kv, const float (&scale)[2], Use &&use) {
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
      for (int pr = 0; pr < 4; ++pr)
        f[pr] = d & 1 ? e4m3_to_bf16x2<true>(w[pr][d >> 1], scale[pr >> 1]) : e4m3_to_bf16x2<false>(w[pr][d >> 1], scale[pr >> 1]);
      use(4 * half + d, frag(f[0], f[1], f[2], f[3]));
      if (d & 1) __builtin_amdgcn_sched_barrier(0);
    }
  }
}

// The work of a call dealt out by its lengths: all entries' keys in chunks of one length, about the shortest for which there are no more
// chunks than workgroups, so that no CU is left without work by sequences that are shorter than the longest.  Every wave works this
// out for itself, with up to kDealt entries (of one block of rows) in each lane, from the same numbers; the first one writes it down
// for the joining kernel.
template <int HW>
__device__ __forceinline__ bool deal(const AttendArgs &a, int wg, bool publish, int *b, int *hg, int *split, int *chunk) {
  constexpr int kUnit = 32 * kWaves / HW;  // keys of a step
  const int n_hg = a.n_kv_heads / HW, n = (int)a.n_entries, lane = threadIdx.x & 63, per = (n + 63) / 64;
  const float per_hg = 1.f / (float)n_hg;
  auto seq_of = [&](int e) { return (int)(((float)e + 0.5f) * per_hg); };  // e / n_hg (both are small)
  int u[kDealt];  // steps of an entry, one at least; 0: no such entry
  float all = 0.f;
#pragma unroll
  for (int i = 0; i < kDealt; ++i) {
    const int e = lane * per + i;
    u[i] = 0;
    if (i < per && e < n) {
      const int seq = seq_of(e);
      int most = 1;
#pragma unroll
      for (int x = 0; x < HW; ++x) {
        const int len = a.len[((e - seq * n_hg) * HW + x) * a.batch + seq];
        if (length_ok(a, len)) most = max(most, len);
      }
      u[i] = (most + kUnit - 1) / kUnit;
      all += (float)u[i];
    }
  }
  all = row16_sum_fast(all);
  auto lane_of = [](float v, int l) { return __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(v), l)); };
  all = lane_of(all, 0) + lane_of(all, 16) + lane_of(all, 32) + lane_of(all, 48);
  int c = __builtin_amdgcn_readfirstlane(max(1, (int)(all / (float)a.dealt))), cnt, upto;
  for (;;) {
    cnt = 0;
#pragma unroll
    for (int i = 0; i < kDealt; ++i)
      if (i < per) cnt += (u[i] + c - 1) / c;
    upto = lanes_before_and_here(cnt);
    if (__builtin_amdgcn_readlane(upto, 63) <= a.dealt) break;
    c += max(1, c / 32);
  }
  *chunk = c * kUnit;
  if (publish) {
    int first = upto - cnt;
    if (lane == 0) a.deal[0] = *chunk;
#pragma unroll
    for (int i = 0; i < kDealt; ++i)
      if (i < per && lane * per + i < n) {
        a.deal[1 + lane * per + i] = first;
        first += (u[i] + c - 1) / c;
      }
  }
  const uint64_t behind = __ballot(upto > wg);
  if (!behind) return false;  // fewer chunks than workgroups
  const int at = __builtin_ctzll(behind);
  int first = __builtin_amdgcn_readlane(upto - cnt, at), entry = at * per;
#pragma unroll
  for (int i = 0; i < kDealt - 1; ++i)
    if (i < per - 1) {
      const int k = (__builtin_amdgcn_readlane(u[i], at) + c - 1) / c;
      if (wg >= first + k && entry == at * per + i) {
        ++entry;
        first += k;
      }
    }
  *split = wg - first;
  *b = __builtin_amdgcn_readfirstlane(seq_of(entry));
  *hg = entry - *b * n_hg;
  return true;
}

// HW: heads side by side (their rows of a slot are neighbours in memory: 512 bytes at a time come faster than 128), one or more waves to
// each, which take steps of 32 keys in turn.  RT: tiles of 16 query rows, which share the keys' and values' conversion.  DT: type of q and out.
// Accuracy: stored keys and values are bf16 numbers.  bf16 queries enter as they are; fp32 ones as three bf16 parts (24 bits).  Weights
// enter the second product as two parts (16 bits) with bf16 outputs, three with fp32 ones.  Everything else is fp32.
template <int DT, int HW, int RT>
__global__ void __launch_bounds__(64 * kWaves, DT == SKIPKV_F32 || RT > 1 ? 2 : 4) k_attend(AttendArgs a) {
  constexpr int KW = kWaves / HW;
  constexpr int NQ = DT == SKIPKV_BF16 ? 1 : 3, NP = DT == SKIPKV_BF16 ? 2 : 3;
  constexpr int ESZ = DT == SKIPKV_BF16 ? 2 : 4;
  __shared__ __align__(16) float o_part[kWaves][16][kOPitch];
  __shared__ float2 ml_part[kWaves][16];
  const int tid = threadIdx.x, wave_all = __builtin_amdgcn_readfirstlane(tid >> 6), kw = wave_all / HW, hw = wave_all % HW;
  const int lane = tid & 63, g = lane >> 4, c = lane & 15;
  const int bmask = (1 << a.block_log2) - 1;
  const int n_hg = a.n_kv_heads / HW;
  int split, hg, rb = 0, b, chunk = a.chunk;
  if (a.dealt) {
    if (!deal<HW>(a, blockIdx.x, blockIdx.x == 0 && wave_all == 0, &b, &hg, &split, &chunk)) return;
  } else {
    split = blockIdx.x / n_hg;
    hg = blockIdx.x - split * n_hg;
    rb = blockIdx.y;
    b = blockIdx.z;
  }
  const int h = hg * HW + hw;
  const int k_begin = split * chunk;
  const int32_t *table = a.block_table + (int64_t)b * a.table_stride;
  // Up to 32 steps at a time: lane i looks up the block of tile i & 1 of step i >> 1.  The first look-up waits for nothing: what it
  // finds behind the last key is put right below.
  auto tile_key = [&](int s0) { return k_begin + ((s0 + (lane >> 1)) * KW + kw) * 32 + (lane & 1) * 16; };
  int id = 0;
  {
    const int at = tile_key(0) >> a.block_log2;
    if (at < a.table_stride) id = table[at];
  }
  int n = 0, most = 0;  // keys of this head; keys that some head of the group sees
  bool n_ok = true;
  int q0, m;
  const bool q_ok = seq_queries(a, b, &q0, &m);
  const int r0 = rb * a.rows, r1 = min(r0 + a.rows, m * a.group);
#pragma unroll
  for (int i = 0; i < HW; ++i) {
    const int ni = a.len[(hg * HW + i) * a.batch + b];
    const bool ok = length_ok(a, ni);
    most = max(most, ok ? rows_see(a, m, ni, r1 - 1) : 0);
    if (i == hw) {
      n = ni;
      n_ok = ok;
    }
  }
  const int n_chunks = max(1, (most + chunk - 1) / chunk);
  if (!q_ok || r0 >= r1 || split >= n_chunks) {
    if (!q_ok && split == 0 && rb == 0 && lane == 0 && a.dev_status) atomicOr(a.dev_status, SKIPKV_DEV_BAD_LENGTHS);
    return;
  }
  if (!n_ok && split == 0 && lane == 0 && a.dev_status) atomicOr(a.dev_status, SKIPKV_DEV_BAD_LENGTHS);
  const int k_end = min(n_ok ? rows_see(a, m, n, r1 - 1) : 0, k_begin + chunk);
  const int steps_all = max(0, (k_end - k_begin + 31) / 32);
  const int steps = kw < steps_all ? (steps_all - kw + KW - 1) / KW : 0;  // of this wave
  bool poison = !n_ok;
  auto check_id = [&](int s0) {
    const bool in = tile_key(s0) < k_end, good = id >= 0 && id < a.n_blocks;
    poison |= in && !good;
    if (!in || !good) id = 0;
  };
  check_id(0);
  const uint8_t *kbase = a.k + h * a.stride_head, *vbase = a.v + h * a.stride_head;
  const uint8_t *kexp = a.k_exp + (int64_t)h * a.n_blocks, *vexp = a.v_exp + (int64_t)h * a.n_blocks;
  const uint32_t k_lane = (uint32_t)c * (uint32_t)a.stride_tok + 16 * g;
  const uint32_t v_lane = (uint32_t)(4 * g) * (uint32_t)a.stride_tok + 8 * c;
  auto row_of = [&](int s0, int s, int t) {  // (tiles that lie behind the last key read block 0)
    const int key = k_begin + ((s0 + s) * KW + kw) * 32 + t * 16;
    return (int64_t)__builtin_amdgcn_readlane(id, 2 * s + t) * a.stride_block + (int64_t)(key & bmask) * a.stride_tok;
  };
  Keys kk;
  Values kv;
  auto load_k = [&](int s0, int s) {
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      const uint8_t *p = kbase + row_of(s0, s, t);
      kk.k[t][0] = *reinterpret_cast<const uint4 *>(p + k_lane);
      kk.k[t][1] = *reinterpret_cast<const uint4 *>(p + k_lane + 64);
    }
  };
  auto load_v = [&](int s0, int s) {
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      const uint8_t *p = vbase + row_of(s0, s, t);
#pragma unroll
      for (int i = 0; i < 4; ++i) kv.v[t][i] = *reinterpret_cast<const uint2 *>(p + v_lane + (uint32_t)i * (uint32_t)a.stride_tok);
    }
  };
  load_k(0, 0);
  load_v(0, 0);
  // (behind the last key that of 1: a block to which nobody has stored may have any, and some make a NaN of 0)
  auto value_scale = [&](int s0) -> uint32_t { return tile_key(s0) < k_end ? vexp[id] : 127u; };
  uint32_t ke = kexp[id], ve = value_scale(0);

  // ---- queries: lane (g, c) holds dimensions 64 i + 16 g + 8 half + (0 .. 7) of row c
  bf16x8 qf[RT][NQ][4];
  int sees[RT];  // keys that row 16 rt + c sees
#pragma unroll
  for (int rt = 0; rt < RT; ++rt) {
    const uint32_t q_sign = a.scale < 0.f ? 0x80008000u : 0u;
    const int r = r0 + 16 * rt + c, j = r / a.group, i = r - j * a.group;
    const bool in = r < r1;
    sees[rt] = in ? n - m + j + 1 : 0x7FFFFFFF;
    const char *p = static_cast<const char *>(a.q) + ((q0 + j) * a.q_stride_tok + (h * a.group + i) * a.q_stride_head + 16 * g) * ESZ;
#pragma unroll
    for (int s = 0; s < 4; ++s) {
      uint32_t w[NQ][4] = {};
      if (in) {
        const char *src = p + (64 * (s >> 1) + 8 * (s & 1)) * ESZ;
        if constexpr (DT == SKIPKV_BF16) {
          const uint4 x = *reinterpret_cast<const uint4 *>(src);
          w[0][0] = x.x, w[0][1] = x.y, w[0][2] = x.z, w[0][3] = x.w;
        } else {
          const float4 x = reinterpret_cast<const float4 *>(src)[0], y = reinterpret_cast<const float4 *>(src)[1];
          const float f[8] = {x.x, x.y, x.z, x.w, y.x, y.y, y.z, y.w};
#pragma unroll
          for (int i4 = 0; i4 < 4; ++i4) {
            uint32_t parts[NQ];
            split_bf16(f[2 * i4], f[2 * i4 + 1], parts);
#pragma unroll
            for (int k = 0; k < NQ; ++k) w[k][i4] = parts[k];
          }
        }
      }
#pragma unroll
      for (int k = 0; k < NQ; ++k) qf[rt][k][s] = frag(w[k][0] ^ q_sign, w[k][1] ^ q_sign, w[k][2] ^ q_sign, w[k][3] ^ q_sign);
    }
  }
  const int all_see = max(0, n - m + r0 / a.group + 1);  // keys below this are seen by every row

  f32x4 o[RT][8];
  float ref[RT], sum[RT];
#pragma unroll
  for (int rt = 0; rt < RT; ++rt) {
#pragma unroll
    for (int j = 0; j < 8; ++j) o[rt][j] = f32x4{0.f, 0.f, 0.f, 0.f};
    ref[rt] = kRefInit;
    sum[rt] = 0.f;
  }
  // (the scale's sign has gone into the queries; not 0, so that what is not seen stays -inf)
  const float to_log2 = fmaxf(fabsf(a.scale) * kLog2e, 1e-45f);
  int inf_from = 0x7FFFFFFF;  // first step of the wave with a NaN or an infinity that only some rows see
  for (int s0 = 0; s0 < steps; s0 += 32) {
    if (s0 > 0) {
      const int key = tile_key(s0);
      id = key < k_end ? table[key >> a.block_log2] : 0;
      check_id(s0);
      load_k(s0, 0);
      load_v(s0, 0);
      ke = kexp[id];
      ve = value_scale(s0);
    }
    const int here = min(32, steps - s0);
    for (int s = 0; s < here; ++s) {
      const int after = min(s + 1, here - 1);  // loaded as soon as the registers are free (the last one again)
      const int key0 = k_begin + ((s0 + s) * KW + kw) * 32;
      const float ks2[2] = {scale_of_byte(__builtin_amdgcn_readlane(ke, 2 * s)), scale_of_byte(__builtin_amdgcn_readlane(ke, 2 * s + 1))};
      const float vs2[2] = {scale_of_byte(__builtin_amdgcn_readlane(ve, 2 * s)), scale_of_byte(__builtin_amdgcn_readlane(ve, 2 * s + 1))};
      const bool all_seen = key0 + 32 <= min(all_see, k_end);
      // ---- logits
      f32x4 acc[RT][2];
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        bf16x8 kf[4];
#pragma unroll
        for (int s4 = 0; s4 < 4; ++s4) {
          const uint4 x = kk.k[t][s4 >> 1];
          const uint32_t w0 = s4 & 1 ? x.z : x.x, w1 = s4 & 1 ? x.w : x.y;
          kf[s4] = frag(e4m3_to_bf16x2<false>(w0, ks2[t]), e4m3_to_bf16x2<true>(w0, ks2[t]), e4m3_to_bf16x2<false>(w1, ks2[t]), e4m3_to_bf16x2<true>(w1, ks2[t]));
        }
#pragma unroll
        for (int rt = 0; rt < RT; ++rt) {
          f32x4 z = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
          for (int k = NQ - 1; k >= 0; --k)
#pragma unroll
            for (int s4 = 0; s4 < 4; ++s4) z = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kf[s4], qf[rt][k][s4], z, 0, 0, 0);
          acc[rt][t] = z;
        }
        __builtin_amdgcn_sched_barrier(0);  // (few registers: four waves share a SIMD)
      }
      load_k(s0, after);
      // ---- what is not seen
      if (!all_seen) {
        asm volatile("");  // (a branch: this is not worth computing for every step)
        uint32_t over = 0;
#pragma unroll
        for (int t = 0; t < 2; ++t) {
          const uint32_t room = room_of(__builtin_amdgcn_readlane(ve, 2 * s + t));
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const int key = key0 + 16 * t + 4 * g + i;
            uint2 &x = kv.v[t][i];
            if (key >= k_end) x = make_uint2(0, 0);
            over |= over_bits(x.x, room) | over_bits(x.y, room);
            x = make_uint2(x.x & ~infinite_bytes(x.x, room), x.y & ~infinite_bytes(x.y, room));  // (see below)
#pragma unroll
            for (int rt = 0; rt < RT; ++rt)
              if (key >= min(sees[rt], k_end)) acc[rt][t][i] = -__builtin_inff();
          }
        }
        if (__any(over != 0)) inf_from = min(inf_from, s0 + s);
      }
      // ---- weights
      uint32_t pf[RT][NP][4];
#pragma unroll
      for (int rt = 0; rt < RT; ++rt) {
        float top = acc[rt][0][0];
#pragma unroll
        for (int i = 1; i < 8; ++i) top = fmaxf(top, acc[rt][i >> 2][i & 3]);
        top *= to_log2;
        if (__any(top > ref[rt] + kSlack)) {
          asm volatile("");
          top = fmaxf(top, __shfl_xor(top, 16));
          top = fmaxf(top, __shfl_xor(top, 32));
          const float now = fmaxf(ref[rt], top), f = __builtin_amdgcn_exp2f(ref[rt] - now);
          ref[rt] = now;
          sum[rt] *= f;
#pragma unroll
          for (int j = 0; j < 8; ++j) o[rt][j] *= f;
        }
        float p[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          p[i] = __builtin_amdgcn_exp2f(fmaf(acc[rt][i >> 2][i & 3], to_log2, -ref[rt]));
          sum[rt] += p[i];
        }
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          uint32_t parts[NP];
          split_bf16(p[2 * i], p[2 * i + 1], parts);
#pragma unroll
          for (int k = 0; k < NP; ++k) pf[rt][k][i] = parts[k];
        }
      }
      // ---- values
      value_frags(kv, vs2, [&](int j, bf16x8 vf) {
#pragma unroll
        for (int rt = 0; rt < RT; ++rt)
#pragma unroll
          for (int k = NP - 1; k >= 0; --k) o[rt][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vf, frag(pf[rt][k][0], pf[rt][k][1], pf[rt][k][2], pf[rt][k][3]), o[rt][j], 0, 0, 0);
      });
      load_v(s0, after);
      __builtin_amdgcn_sched_barrier(0);
    }
  }
  // A weight of 0 does not undo a NaN or an infinity in a matrix product, so these have been taken out of the values of the steps that not
  // every row sees in full; here they are counted, with weight 1 for the rows that see them.
  for (int s = inf_from; s < steps; ++s) {
    const int key0 = k_begin + (s * KW + kw) * 32;
#pragma unroll
    for (int t = 0; t < 2; ++t)
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int key = key0 + 16 * t + 4 * g + i;
        const int p = key < k_end ? table[key >> a.block_log2] : -1;
        kv.v[t][i] = make_uint2(0, 0);
        if (p >= 0 && p < a.n_blocks) {
          const uint2 x = *reinterpret_cast<const uint2 *>(vbase + p * a.stride_block + (int64_t)(key & bmask) * a.stride_tok + 8 * c);
          const uint32_t room = room_of(vexp[p]);
          kv.v[t][i] = make_uint2(infinite_bytes(x.x, room) & 0x38383838u, infinite_bytes(x.y, room) & 0x38383838u);  // the code of 1
        }
      }
    const float unscaled[2] = {1.f, 1.f};
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
      uint32_t one[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int key = key0 + 16 * (i >> 1) + 4 * g + 2 * (i & 1);
        one[i] = (key < min(sees[rt], k_end) ? 0x3F80u : 0u) | (key + 1 < min(sees[rt], k_end) ? 0x3F800000u : 0u);
      }
      value_frags(kv, unscaled, [&](int j, bf16x8 vf) {
        const f32x4 z = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vf, frag(one[0], one[1], one[2], one[3]), f32x4{0.f, 0.f, 0.f, 0.f}, 0, 0, 0);
#pragma unroll
        for (int i = 0; i < 4; ++i)
          if (z[i] > 0.f) o[rt][j][i] = nan32();
      });
    }
  }
  poison = __any(poison);
  if (poison && n_ok && lane == 0 && a.dev_status) atomicOr(a.dev_status, SKIPKV_DEV_BAD_BLOCK_TABLE);

  // ---- merge of a head's waves, 16 rows at a time: lane (g, c) has row c, dimensions 32 g + 8 i + j
  const int64_t part = a.dealt ? (int64_t)blockIdx.x : (int64_t)((b * a.n_rb + rb) * n_hg + hg) * a.n_split + split;
#pragma unroll
  for (int rt = 0; rt < RT; ++rt) {
    if (rt > 0) __syncthreads();  // (the rows before are read)
    sum[rt] += __shfl_xor(sum[rt], 16);
    sum[rt] += __shfl_xor(sum[rt], 32);
    if (g == 0) ml_part[wave_all][c] = make_float2(ref[rt], poison ? nan32() : sum[rt]);
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int j4 = 0; j4 < 2; ++j4)
        *reinterpret_cast<float4 *>(&o_part[wave_all][c][32 * g + 8 * i + 4 * j4]) = make_float4(o[rt][4 * j4][i], o[rt][4 * j4 + 1][i], o[rt][4 * j4 + 2][i], o[rt][4 * j4 + 3][i]);
    __syncthreads();
    const int rows = min(16, r1 - r0 - 16 * rt);  // (negative: none)
    for (int item = kw * 64 + lane; item < rows * (kD / 4); item += 64 * KW) {
      const int row = item / (kD / 4), d = 4 * (item % (kD / 4)), r = r0 + 16 * rt + row;
      float top = kRefInit;
#pragma unroll
      for (int w = 0; w < KW; ++w) top = fmaxf(top, ml_part[w * HW + hw][row].x);
      float all = 0.f;
      float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
      for (int w = 0; w < KW; ++w) {
        const float2 ml = ml_part[w * HW + hw][row];
        const float f = __builtin_amdgcn_exp2f(ml.x - top);
        const float4 x = *reinterpret_cast<const float4 *>(&o_part[w * HW + hw][row][d]);
        all += ml.y * f;
        v.x += x.x * f, v.y += x.y * f, v.z += x.z * f, v.w += x.w * f;
      }
      if (n_chunks == 1) {
        const int j = r / a.group;
        store_row<DT>(a, q0 + j, h * a.group + r - j * a.group, d, v, top, all);
      } else {
        const int64_t at = (part * HW + hw) * a.part_rows + 16 * rt + row;
        *reinterpret_cast<float4 *>(a.part_o + at * kD + d) = v;
        if (d == 0) a.part_ml[at] = make_float2(top, all);
      }
    }
  }
}

// Entries (sequence, block of rows, group of heads) of several chunks: 32 lanes per chunk of a row, four dimensions each, GR chunks at a
// time; a workgroup has 8 / GR rows.  What it costs is waiting for memory, so all chunks up to 8 * GR are under way together,
// before it is known how many there are.
template <int DT, int GR>
__global__ void __launch_bounds__(256) k_attend_join(AttendArgs a) {
  __shared__ float4 v_part[8][32];
  __shared__ float2 ml_part[8];
  const int tid = threadIdx.x, d = tid & 31, grp = (tid >> 5) % GR, n_hg = a.n_kv_heads / a.hw;
  const int64_t row_at = (int64_t)blockIdx.x * (8 / GR) + (tid >> 5) / GR;  // (entry, head of the group, row)
  const int per_entry = a.hw * a.part_rows;
  const int64_t entry = row_at / per_entry;
  const int in_entry = (int)(row_at - entry * per_entry);
  const bool in = entry < a.n_entries;
  const int chunk = a.dealt ? a.deal[0] : a.chunk;
  const int64_t first = !in ? 0 : a.dealt ? a.deal[1 + entry] : entry * a.n_split, bound = a.dealt ? a.n_parts : first + a.n_split;
  constexpr int AHEAD = 8;
  float2 ml[AHEAD];
  float4 x[AHEAD];
  auto fetch = [&](int s0) {
#pragma unroll
    for (int i = 0; i < AHEAD; ++i) {
      const int s = s0 + i * GR + grp;
      if (in && first + s < bound) {
        const int64_t at = (first + s) * per_entry + in_entry;
        ml[i] = a.part_ml[at];
        x[i] = *reinterpret_cast<const float4 *>(a.part_o + at * kD + 4 * d);
      }
    }
  };
  fetch(0);
  const int hw = in_entry / a.part_rows, hg = (int)(entry % n_hg), b = (int)(entry / n_hg / a.n_rb), rb = (int)(entry / n_hg % a.n_rb);
  const int r = rb * a.rows + in_entry - hw * a.part_rows;
  int n_chunks = 0, q0 = 0;
  if (in) {
    int m;
    const bool q_ok = seq_queries(a, b, &q0, &m);
    const int r1 = min((rb + 1) * a.rows, m * a.group);
    int most = 0;
    for (int i = 0; i < a.hw; ++i) {
      const int n = a.len[(hg * a.hw + i) * a.batch + b];
      if (length_ok(a, n)) most = max(most, rows_see(a, m, n, r1 - 1));
    }
    if (q_ok && r < r1) n_chunks = (most + chunk - 1) / chunk;
  }
  if (n_chunks <= 1) n_chunks = 0;  // written already
  if (GR == 8 && n_chunks == 0) return;
  float top = kRefInit, all = 0.f;
  float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
  for (int s0 = 0; s0 < n_chunks;) {
    float now = top;
#pragma unroll
    for (int i = 0; i < AHEAD; ++i)
      if (s0 + i * GR + grp < n_chunks) now = fmaxf(now, ml[i].x);
    const float back = __builtin_amdgcn_exp2f(top - now);
    top = now;
    all *= back;
    v.x *= back, v.y *= back, v.z *= back, v.w *= back;
#pragma unroll
    for (int i = 0; i < AHEAD; ++i)
      if (s0 + i * GR + grp < n_chunks) {
        const float f = __builtin_amdgcn_exp2f(ml[i].x - now);
        all += ml[i].y * f;
        v.x += x[i].x * f, v.y += x[i].y * f, v.z += x[i].z * f, v.w += x[i].w * f;
      }
    s0 += AHEAD * GR;
    if (s0 < n_chunks) fetch(s0);
  }
  if constexpr (GR > 1) {
    v_part[tid >> 5][d] = v;
    if (d == 0) ml_part[tid >> 5] = make_float2(top, all);
    __syncthreads();
    if (grp > 0) return;
    const int g0 = tid >> 5;
#pragma unroll
    for (int i = 1; i < GR; ++i) top = fmaxf(top, ml_part[g0 + i].x);
    all = 0.f;
    v = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
    for (int i = 0; i < GR; ++i) {
      const float f = __builtin_amdgcn_exp2f(ml_part[g0 + i].x - top);
      const float4 w = v_part[g0 + i][d];
      all += ml_part[g0 + i].y * f;
      v.x += w.x * f, v.y += w.y * f, v.z += w.z * f, v.w += w.w * f;
    }
  }
  if (n_chunks == 0) return;
  const int j = r / a.group;
  store_row<DT>(a, q0 + j, (hg * a.hw + hw) * a.group + r - j * a.group, 4 * d, v, top, all);
}

}  // namespace

// How the work is laid out: rows per workgroup, heads side by side, and chunks per entry.  Taken is what comes out shortest if all
// lengths were max_len, by these times (us, all of them measured when the whole chip is at work):
//   16 or 32 rows: a workgroup's unit is one step of its 8 waves, 64 KB of codes whatever their number of heads: 2.9 where four
//     heads' rows lie together, 3.05 and 3.3 with two and one; 2.2 and 2.4 where several blocks of 16 and 32 rows read the same codes; the
//     way to the first unit and from the last 4; a row of partial results, written and read again, 0.0003, the launch that joins them 5;
//   256 rows (k_attend_rows; bf16, from 33 rows on): a tile of 64 keys 0.9 to 1.8, the way to the first one 8, pieces as above.
// Measured, us, one head / four heads side by side:
//   64 x 4 heads, 1152 keys 15.8 / 22.5;  50 x 8 heads, 400-830 keys 18.6 / 22.8;  8 x 8 heads, 32896 keys 127 / 104;  18 x 8 heads, 10 K keys 110 / 74;
// rows of 16 / 32 / 256:
//   20 rows, 16 x 8 heads, 4200 keys 45 / 39 / -;  32 rows, 64 x 4 heads, 1152 keys 28 / 19 / 29;  32 rows, 16 x 8 heads, 1000 keys 12.7 / 16.2 / 20;
//   80 rows, 4 x 8 heads, 1100 keys 11.9 / 15.4 / 17.5;  160 rows 18.6 / 16.0 / 22.9;  48 rows, 30 x 4 heads, 300-2000 keys 27.7 / 22.5 / 28.2;
//   128 rows, 64 x 8 heads, 1152 keys 123 / 106 / 69;  64 rows, 8 x 8 heads, 32000 keys 264 / 166 / 156.
// Without the time of partial results, which made the chunks shorter: 1 x 8 heads, 4224 keys, one token 12.2 instead of 10.8.
void plan_attend(AttendArgs *a) {
  const int64_t head_rows = (int64_t)a->max_q * a->group;
  const bool bf16 = a->dtype == SKIPKV_BF16;
  constexpr double kPartRow = 0.0003, kJoin = 5;
  double best = 0;
  int steps = 0;  // of a workgroup
  for (const int rows : {16, 32}) {
    if (rows == 32 && (!bf16 || head_rows <= 16)) continue;
    const int64_t n_rb = (head_rows + rows - 1) / rows;
    if (bf16 && n_rb > 16) continue;
    const int part_rows = (int)std::min<int64_t>(rows, head_rows);
    for (const int hw : {4, 2, 1}) {
      if (a->n_kv_heads % hw) continue;
      const int unit = 32 * kWaves / hw, units = std::max(1, (a->max_len + unit - 1) / unit);
      const int64_t entries = (int64_t)a->batch * n_rb * (a->n_kv_heads / hw);
      const double unit_us = bf16 && n_rb > 1 ? (rows == 32 ? 2.4 : 2.2) : hw == 4 ? 2.9 : hw == 2 ? 3.05 : 3.3;
      for (int turn = 0; turn <= 4; ++turn) {  // one workgroup per entry, or as many as fill the CUs so many times
        const int64_t want = turn == 0 ? 1 : std::min<int64_t>(units, 256 * turn / entries);
        if (want < 1) continue;
        const int per = (int)((units + want - 1) / want), split = (units + per - 1) / per;  // units per workgroup
        const double turns = (double)((entries * split + 255) / 256);
        const double us = turns * (per * unit_us + 4) + (split > 1 ? kJoin + kPartRow * (double)(entries * split * hw * part_rows) : 0);
        if (best == 0 || us < best) {
          best = us;
          a->rows = rows;
          a->n_rb = (int32_t)n_rb;
          a->part_rows = part_rows;
          a->hw = hw;
          a->chunk = per * unit;
          a->n_split = split;
          a->n_entries = entries;
          steps = per;
        }
      }
    }
  }
  a->n_parts = a->n_entries * a->n_split;
  if (bf16 && head_rows > 32) {
    const int64_t n_rb = (head_rows + 255) / 256, entries = (int64_t)a->batch * n_rb * a->n_kv_heads;
    const int part_rows = (int)std::min<int64_t>(256, head_rows);
    // Up to 128 blocks of rows are cut alike, into pieces of less than 2048 keys; others are dealt out by what the sequences have, us, as cut here / dealt: 8 x 8 heads, 100-400
    // query tokens over 2-6 K keys 215 / 180;  4 x 8 heads, 700-1500 tokens 295 / 282;  30 x 8 heads, 20-40 tokens 133 / 136;  and
    // 32 blocks in all 23.2 / 26.4.
    const int64_t blocks = std::min<int64_t>((int64_t)a->batch * n_rb, ((int64_t)a->total_q * a->group + 255) / 256 + a->batch) * a->n_kv_heads;
    const int64_t want = std::max<int64_t>(1, 256 / entries);
    int chunk = (int)std::max<int64_t>(256, ((a->max_len + want - 1) / want + 63) / 64 * 64);
    const bool dealt = (entries > 128 || chunk >= 2048) && a->batch <= 64 * kDealt && blocks < (1 << 22);  // (a grid has fewer than 2^32 threads)
    if (dealt) chunk = a->max_len;
    const int split = dealt ? 1 : std::max(1, (a->max_len + chunk - 1) / chunk);
    const double tile_us = 0.9 + 0.9 * part_rows / 256, turns = (double)blocks / 256;
    const double us = dealt ? std::max(0.125, turns) * (a->max_len / 64 + 1) * tile_us + std::max(1., turns) * 8 + kJoin + kPartRow * 256 * part_rows
                            : (double)((entries * split + 255) / 256) * ((chunk / 64 + 1) * tile_us + 8) +
                                  (split > 1 ? kJoin + kPartRow * (double)(entries * split * part_rows) : 0);
    if (best == 0 || us < best) {
      a->rows = 256;
      a->n_rb = (int32_t)n_rb;
      a->part_rows = part_rows;
      a->hw = 1;
      a->chunk = chunk;
      a->n_split = split;
      a->n_entries = entries;
      a->n_parts = dealt ? kRowParts : entries * split;
      a->dealt = dealt ? (int32_t)blocks + kRowParts : 0;
      return;
    }
  }
  // Dealing costs a workgroup 2 us before its first key and pays where lengths differ, us, as planned for equal lengths / dealt:
  //   steps  8: 16 x 8 heads, 512-4096 keys 22.6 / 23.4;  8 x 8 heads, 1-8 K 22.0 / 22.4
  //   steps 16: 16 x 8 heads, 1-8 K 39.5 / 36.1;  8 x 8 heads, 2-16 K 39.3 / 37.0;  all 4000-4500 35.3 / 36.4
  //   steps 32 and more: 16 x 8 heads, 2-16 K 65.2 / 57.0;  60 x 4 heads, 2-16 K 122 / 105;  all 32896 103.9 / 106.2
  // It also pays where max_len is the room that a sequence has rather than its length, one sequence's too.
  if (a->n_split > 1 && steps >= 12 && a->n_rb == 1 && a->n_entries <= 64 * kDealt)
    a->dealt = (int32_t)(a->n_parts = (a->n_parts + 255) / 256 * 256);
}

// Rows of partial results for which a call and every smaller one (fewer sequences, query tokens or keys, the heads alike) have room: the
// most that plan_attend makes of them.  Its choices rise and fall with the sizes (one token of 8 heads: 1.06 MB at 32 K keys, 2.08 at
// some shorter ones), and a workspace of the largest call has to serve the others.
//   16 or 32 rows at a time: keys that are cut make at most four turns of 256 workgroups, dealt out or not, of hw heads' rows each;
//   256 rows at a time: at most kRowParts pieces dealt out, 256 cut alike.
int64_t attend_room(const AttendArgs &a) {
  const int64_t head_rows = (int64_t)a.max_q * a.group;
  const bool bf16 = a.dtype == SKIPKV_BF16;
  const int hw = a.n_kv_heads % 4 == 0 ? 4 : a.n_kv_heads % 2 == 0 ? 2 : 1;
  const int64_t few = a.max_len > 32 * kWaves / hw ? 256 * 4 * hw * std::min<int64_t>(bf16 ? 32 : 16, head_rows) : 0;  // (else one unit, which is not cut)
  const int64_t many = bf16 && head_rows > 32 ? kRowParts * std::min<int64_t>(256, head_rows) : 0;
  return std::max(few, many);
}

hipError_t launch_attend(const AttendArgs &a, hipStream_t st) {
  const dim3 grid = a.dealt ? dim3((unsigned)a.dealt) : dim3(a.n_split * (a.n_kv_heads / a.hw), a.n_rb, a.batch);
  hipError_t err = hipSuccess;
  auto go = [&](auto dt) {
    constexpr int DT = decltype(dt)::value;
    auto few = [&](auto rt) {
      constexpr int RT = decltype(rt)::value;
      if (a.hw == 4) hipLaunchKernelGGL((k_attend<DT, 4, RT>), grid, dim3(64 * kWaves), 0, st, a);
      else if (a.hw == 2) hipLaunchKernelGGL((k_attend<DT, 2, RT>), grid, dim3(64 * kWaves), 0, st, a);
      else hipLaunchKernelGGL((k_attend<DT, 1, RT>), grid, dim3(64 * kWaves), 0, st, a);
    };
    if (a.rows == 16) few(std::integral_constant<int, 1>{});
    else if constexpr (DT == SKIPKV_BF16) {
      if (a.rows == 32) few(std::integral_constant<int, 2>{});
      else err = launch_attend_rows(a, st);
    }
    if (err == hipSuccess) err = hipGetLastError();  // (asking for an error takes it away)
    if (a.n_split == 1 || err != hipSuccess) return;  // (or joined already)
    const int64_t rows = a.n_entries * a.hw * a.part_rows;
    // eight chunks of a row at a time from nine on; dealt out, a row may have more than the mean: from eight on (16 x 8 heads, 2-16 K keys: 57.0
    // us instead of 59.0; four on average, 32 x 8 heads, 1-8 K: 66.4 instead of 64.4)
    if (a.dealt ? a.n_parts >= 8 * a.n_entries : a.n_split > 8) hipLaunchKernelGGL((k_attend_join<DT, 8>), dim3((unsigned)rows), dim3(256), 0, st, a);
    else hipLaunchKernelGGL((k_attend_join<DT, 1>), dim3((unsigned)((rows + 7) / 8)), dim3(256), 0, st, a);
    err = hipGetLastError();
  };
  if (a.dtype == SKIPKV_F32) go(std::integral_constant<int, SKIPKV_F32>{});
  else go(std::integral_constant<int, SKIPKV_BF16>{});
  return err;
}

}  // namespace skipkv
