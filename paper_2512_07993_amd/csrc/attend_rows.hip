// Attention over the 8-bit cache with many query rows (pieces of prompts): the matrix cores count here, not the cache's bytes.
//
// A workgroup of eight waves owns 256 query rows of a head, 32 per wave, and walks the keys in tiles of 64.  A tile's codes are converted
// once, with their blocks' scales, into bf16 in shared memory, from where all waves read their operands; the next tile's codes are on
// their way meanwhile.  As with few rows, everything is computed transposed: S^T = K Q^T (32 x 32 tiles) leaves lane (hi, c)
// (hi = lane / 32, c = lane % 32) with the logits of query row c for keys 8a + 4 hi + (0 .. 3), a = 0 .. 3, and O^T = V^T P^T takes the
// weights from there as they lie: the keys of a matrix instruction are 16 k + 4 hi + (0 .. 3) and 8 further on, which transposing
// reads of V's rows deliver in that order.
//
// What bounds it: per matrix instruction of 32 cycles 68 pass on a SIMD, 35 of which issue vector instructions (per weight an fma, an
// exponential of two issue slots, an addition, half a conversion and half a maximum, besides the staging: 6.6 per matrix instruction).  The
// matrix pipe is busy for 47 % of the time and vector instructions are issued for 50 %, which is what two engines look like that take turns;
// a wave waits 29 % of its time for LDS, memory or the barrier and 35 % for its turn to issue.  (Without memory, six independent vector
// instructions beside each matrix instruction take 18.8 ns instead of 15.5, eight 23: this does not reach that.)  So everything but the
// matrix instructions is dealt out evenly among them; operands are in registers a block of 32 keys ahead; rows in shared memory are
// padded, not swizzled, so that addresses are immediates.  4 sequences of 3.5-4.3 K keys, 1.0-1.5 K query tokens, 8 x 4 heads (256 GFLOP):
// 280 to 304 us from run to run, 840-915 TFLOP/s (a library's product of square matrices reaches 1.2-1.3 PFLOP/s); before blocks were dealt
// out 294 to 316: 11 us less each time; before that, with all weights before the product and swizzled addresses 7 % more, without
// the pipeline across blocks 15 % more.  32 x 32 tiles with 64 rows per wave need more registers than two waves on a
// SIMD have (544 us).
//
// Weights enter the product with V rounded to one bf16 number (half a step, 2^-8 of each at most; their sum is of the unrounded ones).  Two
// numbers, as with few rows, take eight more matrix instructions and some 40 vector instructions per block: 380 us instead of 280 in the case
// above.  The error against 64 bits, of the result's norm (300 tokens over 3.5-4 K keys): 1.99e-3 instead of 1.64e-3, which rounding the
// result to bf16 makes by itself.
#include <algorithm>
#include <type_traits>

#include "attend_dev.h"

namespace skipkv {

namespace {

typedef __attribute__((__vector_size__(16 * sizeof(float)))) float f32x16;
constexpr int kTile = 64;      // keys
// A tile in shared memory: rows of 128 bf16 numbers and a little room, so that the rows that are read together start at
// different banks: eight rows of K by 16 bytes, four of V by 32.
constexpr int kPitchK = 2 * kD + 16, kPitchV = 2 * kD + 32;
constexpr int kTileB = kTile * (kPitchK + kPitchV), kTileV = kTile * kPitchK;  // bytes of a tile; where its V begins
constexpr int kRowWaves = 8;  // of 32 rows each
static_assert(kTile * 8 == 64 * kRowWaves, "a thread moves two pieces of K and of V per tile");

// Codes 8 j .. and 64 + 8 j .. of a key to their places in its row (eight lanes write 128 bytes side by side).
__device__ __forceinline__ void put_codes(char *row, int j, uint4 c, float scale) {
  const uint32_t w[4] = {c.x, c.y, c.z, c.w};
#pragma unroll
  for (int i = 0; i < 2; ++i)
    *reinterpret_cast<uint4 *>(row + 16 * j + 128 * i) = make_uint4(e4m3_to_bf16x2<false>(w[2 * i], scale), e4m3_to_bf16x2<true>(w[2 * i], scale),
                                                                   e4m3_to_bf16x2<false>(w[2 * i + 1], scale), e4m3_to_bf16x2<true>(w[2 * i + 1], scale));
}
__device__ __forceinline__ uint4 load_codes(const uint8_t *p) {
  const uint2 x = *reinterpret_cast<const uint2 *>(p), y = *reinterpret_cast<const uint2 *>(p + 64);
  return make_uint4(x.x, x.y, y.x, y.y);
}

// Keys of a piece: whole tiles.
__device__ __forceinline__ int piece_keys(int keys, int pieces) { return max(1, ((keys + kTile - 1) / kTile + pieces - 1) / pieces) * kTile; }

// Blocks of 256 rows dealt out: as many as make whole turns of the 256 CUs run over all their keys; the others, which would leave CUs
// without work at the end, are cut into `pieces` along the keys, as many as come out shortest.  (600 blocks of 53 tiles: three turns take
// 161 tiles' time, 88 blocks in two pieces 139, an even share of all would be 125.)
struct RowDeal {
  int blocks, whole, pieces;  // blocks of all sequences and heads; those that are not cut
};
__device__ __forceinline__ bool deal_rows(const AttendArgs &a, int wg, bool publish, int *b, int *rb, int *h, RowDeal *deal, int *piece) {
  const int lane = threadIdx.x & 63, per = (a.batch + 63) / 64;
  int cnt = 0, u[kDealt];
  float keys = 0.f;
  bool bad = false;
#pragma unroll
  for (int i = 0; i < kDealt; ++i) {
    const int seq = lane * per + i;
    u[i] = 0;
    if (i < per && seq < a.batch) {
      int q0, m;
      const int len = a.len[seq];
      if (!seq_queries(a, seq, &q0, &m)) bad = true;
      else u[i] = (m * a.group + a.rows - 1) / a.rows;
      if (length_ok(a, len)) keys += (float)u[i] * (float)len;
      cnt += u[i];
    }
  }
  const int upto = lanes_before_and_here(cnt), n = __builtin_amdgcn_readlane(upto, 63);
  keys = row16_sum_fast(keys);
  auto lane_of = [](float v, int l) { return __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(v), l)); };
  keys = lane_of(keys, 0) + lane_of(keys, 16) + lane_of(keys, 32) + lane_of(keys, 48);
  const int blocks = n * a.n_kv_heads, whole = blocks / 256 * 256, rest = blocks - whole;
  // us: a tile of 64 keys 1.9 and three of them before the first one; a piece's partial results 0.05, their joining 5
  int pieces = 1;
  if (rest > 0) {
    const float tiles = keys / (64.f * (float)max(n, 1));  // of a block, about
    float best = 0.f;
    for (int p = 1; p <= 8 && p * rest <= kRowParts && (p == 1 || tiles >= 4.f * (float)p); ++p) {
      const float us = (float)((rest * p + 255) / 256) * (tiles / (float)p + 3.f) * 1.9f + (p > 1 ? 5.f + 0.05f * (float)(rest * p) : 0.f);
      if (p == 1 || us < best) {
        best = us;
        pieces = p;
      }
    }
  }
  pieces = __builtin_amdgcn_readfirstlane(pieces);
  *deal = RowDeal{blocks, whole, pieces};
  if (publish) {
    int first = upto - cnt;
    // (offsets that descend can make more blocks than the call has workgroups: nothing is joined of pieces that nobody forms)
    if (lane == 0) a.deal[0] = whole, a.deal[1] = whole + rest * pieces <= (int)gridDim.x ? pieces : 1;
#pragma unroll
    for (int i = 0; i < kDealt; ++i)
      if (i < per && lane * per + i < a.batch) a.deal[2 + lane * per + i] = (first += u[i]);
    if (bad && a.dev_status) atomicOr(a.dev_status, SKIPKV_DEV_BAD_LENGTHS);
  }
  const int block = wg < whole ? wg : whole + (wg - whole) / pieces;
  *piece = wg < whole ? 0 : (wg - whole) % pieces;
  if (block >= blocks) return false;
  const int at_block = block / a.n_kv_heads;
  *h = block - at_block * a.n_kv_heads;
  const int at = __builtin_ctzll(__ballot(upto > at_block));
  int first = __builtin_amdgcn_readlane(upto - cnt, at), seq = at * per;
#pragma unroll
  for (int i = 0; i < kDealt - 1; ++i) {
    const int k = __builtin_amdgcn_readlane(u[i], at);
    if (i < per - 1 && at_block >= first + k && seq == at * per + i) {
      ++seq;
      first += k;
    }
  }
  const int of_seq = __builtin_amdgcn_readlane(u[0], at);
  int mine = of_seq;  // blocks of the sequence
#pragma unroll
  for (int i = 1; i < kDealt; ++i)
    if (seq == at * per + i) mine = __builtin_amdgcn_readlane(u[i], at);
  *b = seq;
  *rb = mine - 1 - (at_block - first);  // the rows that see most first
  return true;
}

__global__ void __launch_bounds__(64 * kRowWaves, 2) k_attend_rows(AttendArgs a) {
  __shared__ __align__(256) char tiles[3][kTileB];
  __shared__ int inf_tile;                              // first tile with a NaN or an infinity in V that only some rows see
  const int tid = threadIdx.x, wave = __builtin_amdgcn_readfirstlane(tid >> 6), lane = tid & 63, hi = lane >> 5, c = lane & 31;
  const int bmask = (1 << a.block_log2) - 1;
  int split, h, rb, b;
  RowDeal dealt{0, 0, 1};
  if (a.dealt) {
    if (!deal_rows(a, blockIdx.x, blockIdx.x == 0 && wave == 0, &b, &rb, &h, &dealt, &split)) return;
  } else {
    split = blockIdx.x / a.n_kv_heads;
    h = blockIdx.x - split * a.n_kv_heads;
    rb = a.n_rb - 1 - blockIdx.y;  // (the rows that see most first)
    b = blockIdx.z;
  }
  int q0, m;
  const bool q_ok = seq_queries(a, b, &q0, &m);
  const int n = a.len[h * a.batch + b];
  const int r0 = rb * a.rows, r1 = min(r0 + a.rows, m * a.group);
  if (!q_ok || r0 >= r1) {
    if (!q_ok && split == 0 && rb == 0 && tid == 0 && a.dev_status) atomicOr(a.dev_status, SKIPKV_DEV_BAD_LENGTHS);
    return;
  }
  const bool n_ok = length_ok(a, n);
  if (!n_ok && split == 0 && tid == 0 && a.dev_status) atomicOr(a.dev_status, SKIPKV_DEV_BAD_LENGTHS);
  const int most = n_ok ? rows_see(a, m, n, r1 - 1) : 0;
  const int chunk = !a.dealt ? a.chunk : (int)blockIdx.x < dealt.whole ? max(most, 1) : piece_keys(most, dealt.pieces);
  const int n_chunks = max(1, (most + chunk - 1) / chunk);
  if (split >= n_chunks) return;
  const int k_begin = split * chunk, k_end = min(most, k_begin + chunk);
  const int n_tiles = (k_end - k_begin + kTile - 1) / kTile;
  const int all_see = max(0, n - m + r0 / a.group + 1);  // keys below this are seen by every row of the workgroup
  if (tid == 0) inf_tile = 0x7FFFFFFF;

  // ---- queries: lane (hi, c) holds dimensions 16 s + 8 hi + (0 .. 7) of row c
  const int w0 = r0 + 32 * wave;  // the wave's first row
  bf16x8 qf[8];
  int sees = 0x7FFFFFFF;
  {
    const uint32_t q_sign = a.scale < 0.f ? 0x80008000u : 0u;
    const int r = w0 + c, j = r / a.group, i = r - j * a.group;
    const bool in = r < r1;
    if (in) sees = n - m + j + 1;
    const uint16_t *p = static_cast<const uint16_t *>(a.q) + (q0 + j) * a.q_stride_tok + (h * a.group + i) * a.q_stride_head + 8 * hi;
#pragma unroll
    for (int s = 0; s < 8; ++s) {
      uint4 x = make_uint4(0, 0, 0, 0);
      if (in) x = *reinterpret_cast<const uint4 *>(p + 16 * s);
      qf[s] = frag(x.x ^ q_sign, x.y ^ q_sign, x.z ^ q_sign, x.w ^ q_sign);
    }
  }
  // keys that the wave's rows see: all of them below w_all, none of them from w_end on
  const int w_last = min(w0 + 32, r1) - 1;
  const int w_end = w0 < r1 ? min(k_end, rows_see(a, m, n, w_last)) : 0, w_all = min(w_end, max(0, n - m + w0 / a.group + 1));

  f32x16 o[4];
  float ref = kRefInit, sum = 0.f, part = 0.f;  // the sum is kept in two parts
#pragma unroll
  for (int d = 0; d < 4; ++d)
#pragma unroll
    for (int i = 0; i < 16; ++i) o[d][i] = 0.f;
  const float to_log2 = fmaxf(fabsf(a.scale) * kLog2e, 1e-45f);
  bool poison = !n_ok;

  // ---- staging: thread (key, j) moves codes 16 j .. 16 j + 15 of a tile's key, of K and of V
  const int s_key = tid >> 3, s_j = tid & 7;
  const int32_t *table = a.block_table + (int64_t)b * a.table_stride;
  const uint8_t *kbase = a.k + h * a.stride_head + 8 * s_j, *vbase = a.v + h * a.stride_head + 8 * s_j;
  const uint8_t *kexp = a.k_exp + (int64_t)h * a.n_blocks, *vexp = a.v_exp + (int64_t)h * a.n_blocks;
  uint4 kc, vc;
  uint32_t ke, ve;
  int id_next = 0;
  auto look_up = [&](int tile) {
    const int key = k_begin + tile * kTile + s_key;
    id_next = key < k_end ? table[key >> a.block_log2] : 0;
  };
  auto fetch = [&](int tile) {  // (of the block that look_up found; behind the last key, and for a bad id, of block 0)
    const bool good = (uint32_t)id_next < (uint32_t)a.n_blocks;
    poison |= !good;
    const int id = good ? id_next : 0;
    const int64_t row = (int64_t)id * a.stride_block + (int64_t)((k_begin + tile * kTile + s_key) & bmask) * a.stride_tok;
    kc = load_codes(kbase + row);
    vc = load_codes(vbase + row);
    ke = kexp[id];
    ve = vexp[id];
  };
  auto commit = [&](int tile, char *to) {
    const int key0 = k_begin + tile * kTile;
    if (key0 + kTile > min(all_see, k_end)) {  // some row does not see all of it
      asm volatile("");
      if (key0 + s_key >= k_end) {  // (a block to which nobody has stored may have any scale, and some make a NaN of 0)
        vc = make_uint4(0, 0, 0, 0);
        ve = 127;
      }
      const uint32_t room = room_of(ve);
      if (over_bits(vc.x, room) | over_bits(vc.y, room) | over_bits(vc.z, room) | over_bits(vc.w, room)) {  // counted below
        atomicMin(&inf_tile, tile);
        vc = make_uint4(vc.x & ~infinite_bytes(vc.x, room), vc.y & ~infinite_bytes(vc.y, room), vc.z & ~infinite_bytes(vc.z, room), vc.w & ~infinite_bytes(vc.w, room));
      }
    }
    put_codes(to + s_key * kPitchK, s_j, kc, scale_of_byte(ke));
    put_codes(to + kTileV + s_key * kPitchV, s_j, vc, scale_of_byte(ve));
  };
  // operand addresses in a tile: K: key c, 16 bytes; V: the group of 16 lanes reads 4 keys x 16 dimensions
  typedef const __attribute__((address_space(3))) char *LdsPtr;
  const LdsPtr lds0 = (LdsPtr)(uintptr_t)lds_addr(tiles);
  const uint32_t k_at = (uint32_t)(c * kPitchK + hi * 16), v_at = (uint32_t)(kTileV + (((lane & 15) >> 2) + 4 * hi) * kPitchV + ((lane >> 4) & 1) * 32 + (lane & 3) * 8);
  // dimensions 32 d .. 32 d + 31, keys 32 half + 16 k + 4 hi + (0 .. 3) and 8 further on
  auto value_frag = [&](LdsPtr base, int half, int d, int k) {
    uint2 x[2];
#pragma unroll
    for (int i = 0; i < 2; ++i)
      x[i] = __builtin_bit_cast(uint2, __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) i16x4 *)(base + ((32 * half + 16 * k + 8 * i) * kPitchV + 64 * d))));
    return frag(x[0].x, x[0].y, x[1].x, x[1].y);
  };
  auto key_frag = [&](LdsPtr base, int half, int sl) { return *(const __attribute__((address_space(3))) bf16x8 *)(base + (32 * half * kPitchK + 32 * sl)); };
  f32x16 s0, s1;  // logits of the even and of the odd blocks of 32 keys
  bf16x8 kf[8], vf[8];
  uint32_t pf[8];
  auto mask = [&](int key0, f32x16 &x) {  // keys that a row does not see
    if (key0 + 32 > w_all) {
      asm volatile("");
#pragma unroll
      for (int e = 0; e < 16; ++e) {
        const int key = key0 + 8 * (e >> 2) + 4 * hi + (e & 3);
        if (key >= min(sees, k_end)) x[e] = -__builtin_inff();
      }
    }
  };
  auto raise = [&](float top) {  // the reference, where a block's logits are far above it
    top *= to_log2;
    asm volatile("");
    {
      const float now = fmaxf(ref, fmaxf(top, __shfl_xor(top, 32))), f = __builtin_amdgcn_exp2f(ref - now);
      ref = now;
      sum *= f;
      part *= f;
#pragma unroll
      for (int d = 0; d < 4; ++d) o[d] *= f;
    }
  };
  // A block of 32 keys takes 16 matrix instructions: 8 for the logits of the next block, whose operands of K are there, and 8 for its own
  // product with V.  Everything else of the block is issued among them, evenly: its weights (in time for the half of the product that takes
  // them), the operands of V and those of K for the block behind the next one, and the largest logits of the next block.
  // A pair of weights takes three slots, so that no instruction waits for the one before it.
  float wx[8], wy[8];
  auto weights_in_slot = [&](const f32x16 &cur, int slot) {
    constexpr int kFirst[8] = {0, 1, 2, 3, 5, 6, 8, 9};
#pragma unroll
    for (int p = 0; p < 8; ++p) {
      if (slot == kFirst[p]) {
        wx[p] = fmaf(cur[2 * p], to_log2, -ref);
        wy[p] = fmaf(cur[2 * p + 1], to_log2, -ref);
      } else if (slot == kFirst[p] + 1) {
        wx[p] = __builtin_amdgcn_exp2f(wx[p]);
        wy[p] = __builtin_amdgcn_exp2f(wy[p]);
      } else if (slot == kFirst[p] + 2) {
        part += wx[p];
        pf[p] = pack_bf16x2(wx[p], wy[p]);
        sum += wy[p];
      }
    }
  };
  auto weights = [&](const f32x16 &cur, f32x16 &nxt, LdsPtr v_base, int half) {
#pragma unroll
    for (int e = 0; e < 16; ++e) nxt[e] = 0.f;
#pragma unroll
    for (int sl = 0; sl < 8; ++sl) {
      nxt = __builtin_amdgcn_mfma_f32_32x32x16_bf16(kf[sl], qf[sl], nxt, 0, 0, 0);
      weights_in_slot(cur, sl);
      vf[sl] = value_frag(v_base, half, sl & 3, sl >> 2);
      __builtin_amdgcn_sched_barrier(0);
    }
  };
  auto product = [&](auto masked, const f32x16 &cur, f32x16 &nxt, int key0, LdsPtr k_base, int half) {
    if (decltype(masked)::value) mask(key0, nxt);
    float top = kRefInit;
    bool above = false;
#pragma unroll
    for (int x = 0; x < 8; ++x) {
      const int k = x >> 2, d = x & 3;
      o[d] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(vf[x], frag(pf[4 * k], pf[4 * k + 1], pf[4 * k + 2], pf[4 * k + 3]), o[d], 0, 0, 0);
      weights_in_slot(cur, 8 + x);
      if (x >= 2 && x < 6)
#pragma unroll
        for (int e = 4 * (x - 2); e < 4 * (x - 1); ++e) top = fmaxf(top, nxt[e]);
      if (x == 6) above = __any(top * to_log2 > ref + kSlack);
      kf[x] = key_frag(k_base, half, x);
      __builtin_amdgcn_sched_barrier(0);
    }
    if (above) raise(top);
  };

  look_up(0);
  fetch(0);
  look_up(1);
  __syncthreads();  // (inf_tile)
  char *here = tiles[0], *there = tiles[1], *then = tiles[2];  // buffers of this tile, the next one, the one behind it
  auto lds_of = [](const char *p) { return (LdsPtr)(uintptr_t)lds_addr(p); };
  if (n_tiles > 0) {
    commit(0, here);
    fetch(1);
    look_up(2);
    lds_barrier();
    float top = kRefInit;
#pragma unroll
    for (int e = 0; e < 16; ++e) s0[e] = 0.f;
#pragma unroll
    for (int sl = 0; sl < 8; ++sl) s0 = __builtin_amdgcn_mfma_f32_32x32x16_bf16(key_frag(lds_of(here) + k_at, 0, sl), qf[sl], s0, 0, 0, 0);
#pragma unroll
    for (int sl = 0; sl < 8; ++sl) kf[sl] = key_frag(lds_of(here) + k_at, 1, sl);
    mask(k_begin, s0);
#pragma unroll
    for (int e = 0; e < 16; ++e) top = fmaxf(top, s0[e]);
    raise(top);
  }
  auto step = [&](auto masked, int tile) {
    const int key0 = k_begin + tile * kTile;
    const LdsPtr v_here = lds_of(here) + v_at, k_there = lds_of(there) + k_at;
    weights(s0, s1, v_here, 0);
    // Three buffers, one barrier per tile: what is written here was last read two tiles ago, before the barrier of the last tile.
    commit(tile + 1, there);
    fetch(tile + 2);
    look_up(tile + 3);
    lds_barrier();
    product(masked, s0, s1, key0 + 32, k_there, 0);
    weights(s1, s0, v_here, 1);
    product(masked, s1, s0, key0 + 64, k_there, 1);
    char *const t = here;
    here = there;
    there = then;
    then = t;
  };
  // tiles after which the wave's rows see the next two blocks in full, then the others
  const int n_free = max(0, min(n_tiles, (w_all - k_begin - 96) / kTile + (w_all - k_begin >= 96)));
  if (w0 >= r1) {  // no rows: this wave only moves its share of the tiles
    for (int tile = 0; tile < n_tiles; ++tile) {
      commit(tile + 1, there);
      fetch(tile + 2);
      look_up(tile + 3);
      lds_barrier();
      char *const t = here;
      here = there;
      there = then;
      then = t;
    }
  } else {
    for (int tile = 0; tile < n_free; ++tile) step(std::false_type{}, tile);
    for (int tile = n_free; tile < n_tiles; ++tile) step(std::true_type{}, tile);
  }
  // ---- NaN and infinities among the values of tiles that only some rows see: counted with weight 1 for the rows that see them
  __syncthreads();
  for (int tile = inf_tile; tile < n_tiles; ++tile) {
    __syncthreads();
    look_up(tile);
    fetch(tile);
    const uint32_t room = room_of(ve);
    const auto ones = [&](uint32_t w) { return k_begin + tile * kTile + s_key < k_end ? infinite_bytes(w, room) & 0x38383838u : 0u; };  // the code of 1
    put_codes(tiles[0] + kTileV + s_key * kPitchV, s_j, make_uint4(ones(vc.x), ones(vc.y), ones(vc.z), ones(vc.w)), 1.f);
    __syncthreads();
#pragma unroll
    for (int half = 0; half < kTile / 32; ++half) {
      const int key0 = k_begin + tile * kTile + 32 * half;
      const LdsPtr vt = lds0 + v_at;
      uint32_t one[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const int key = key0 + 8 * (i >> 1) + 4 * hi + 2 * (i & 1);
        one[i] = (key < min(sees, k_end) ? 0x3F80u : 0u) | (key + 1 < min(sees, k_end) ? 0x3F800000u : 0u);
      }
#pragma unroll
      for (int d = 0; d < 4; ++d) {
        f32x16 z;
#pragma unroll
        for (int i = 0; i < 16; ++i) z[i] = 0.f;
#pragma unroll
        for (int k = 0; k < 2; ++k) z = __builtin_amdgcn_mfma_f32_32x32x16_bf16(value_frag(vt, half, d, k), frag(one[4 * k], one[4 * k + 1], one[4 * k + 2], one[4 * k + 3]), z, 0, 0, 0);
#pragma unroll
        for (int i = 0; i < 16; ++i)
          if (z[i] > 0.f) o[d][i] = nan32();
      }
    }
  }
  poison = __syncthreads_or(poison) != 0;
  if (poison && n_ok && tid == 0 && a.dev_status) atomicOr(a.dev_status, SKIPKV_DEV_BAD_BLOCK_TABLE);

  // ---- lane (hi, c): row c, dimensions 32 d + 8 i + 4 hi + (0 .. 3)
  const int r = w0 + c;
  sum += part;
  const float all = poison ? nan32() : sum + __shfl_xor(sum, 32);
  if (r >= r1) return;
  const int j = r / a.group, head = h * a.group + r - j * a.group;
  const int64_t place = a.dealt ? (int64_t)((int)blockIdx.x - dealt.whole) : ((int64_t)(b * a.n_rb + rb) * a.n_kv_heads + h) * a.n_split + split;
  const int64_t at = place * a.part_rows + (r - r0);
#pragma unroll
  for (int d = 0; d < 4; ++d)
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const float4 v = make_float4(o[d][4 * i], o[d][4 * i + 1], o[d][4 * i + 2], o[d][4 * i + 3]);
      const int dim = 32 * d + 8 * i + 4 * hi;
      if (n_chunks == 1) {
        store_row<SKIPKV_BF16>(a, q0 + j, head, dim, v, ref, all);
      } else {
        *reinterpret_cast<float4 *>(a.part_o + at * kD + dim) = v;
        if (dim == 0) a.part_ml[at] = make_float2(ref, all);
      }
    }
}

// Joins the pieces of the blocks that were cut: 32 lanes per row, four dimensions each.
__global__ void __launch_bounds__(256) k_attend_join_rows(AttendArgs a) {
  const int whole = a.deal[0], pieces = a.deal[1], rest = a.deal[1 + a.batch] * a.n_kv_heads - whole, d = threadIdx.x & 31;
  if (pieces <= 1) return;
  for (int item = blockIdx.x * 8 + (threadIdx.x >> 5); item < rest * a.part_rows; item += gridDim.x * 8) {
    const int cut = item / a.part_rows, row = item - cut * a.part_rows, at_block = (whole + cut) / a.n_kv_heads, h = whole + cut - at_block * a.n_kv_heads;
    float2 ml[8];
    float4 x[8];
#pragma unroll
    for (int i = 0; i < 8; ++i)  // (under way before it is known how many there are)
      if (i < pieces) {
        const int64_t at = (int64_t)(cut * pieces + i) * a.part_rows + row;
        ml[i] = a.part_ml[at];
        x[i] = *reinterpret_cast<const float4 *>(a.part_o + at * kD + 4 * d);
      }
    int lo = 0, hi = a.batch - 1;  // the first sequence whose blocks end behind this one
    while (lo < hi) {
      const int mid = (lo + hi) / 2;
      if (a.deal[2 + mid] > at_block) hi = mid;
      else lo = mid + 1;
    }
    int q0, m;
    (void)seq_queries(a, lo, &q0, &m);
    const int rb = a.deal[2 + lo] - 1 - at_block, r0 = rb * a.rows, r1 = min(r0 + a.rows, m * a.group), r = r0 + row, n = a.len[h * a.batch + lo];
    if (r >= r1) continue;
    const int most = length_ok(a, n) ? rows_see(a, m, n, r1 - 1) : 0, chunk = piece_keys(most, pieces), n_chunks = (most + chunk - 1) / chunk;
    if (n_chunks <= 1) continue;  // written already
    float top = kRefInit, all = 0.f;
    float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (i < n_chunks) top = fmaxf(top, ml[i].x);
#pragma unroll
    for (int i = 0; i < 8; ++i)
      if (i < n_chunks) {
        const float f = __builtin_amdgcn_exp2f(ml[i].x - top);
        all += ml[i].y * f;
        v.x += x[i].x * f, v.y += x[i].y * f, v.z += x[i].z * f, v.w += x[i].w * f;
      }
    const int j = r / a.group;
    store_row<SKIPKV_BF16>(a, q0 + j, h * a.group + r - j * a.group, 4 * d, v, top, all);
  }
}

}  // namespace

hipError_t launch_attend_rows(const AttendArgs &a, hipStream_t st) {
  const dim3 grid = a.dealt ? dim3((unsigned)a.dealt) : dim3(a.n_split * a.n_kv_heads, a.n_rb, a.batch);
  hipLaunchKernelGGL(k_attend_rows, grid, dim3(64 * kRowWaves), 0, st, a);
  const hipError_t err = hipGetLastError();
  if (!a.dealt || err != hipSuccess) return err;
  hipLaunchKernelGGL(k_attend_join_rows, dim3(1024), dim3(256), 0, st, a);
  return hipGetLastError();
}

}  // namespace skipkv
