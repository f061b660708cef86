// Block tables of a paged cache: blocks given back by sequences that became shorter, blocks taken by those that grow, and the
// slots of the new tokens, from the lengths on the GPU.
//
// With P the prefix sums over sequences of the blocks given back, the stack of free blocks after all releases is the old one with
// entry need_b + i of sequence b's table row at n_free + P_b + i; with G those of the blocks wanted, sequence b's i-th new block is the
// one at top - 1 - G_b - i, and it is served iff its end G_b + grow_b is at most top.  Every workgroup of the second kernel forms both
// sums for itself (a few thousand numbers), so that nothing is passed between workgroups: an entry on top of the old stack is read from
// the table row that gives it back, not from the stack, and rows that give back are not written.  The result does not depend on any
// order.
//
// Three kernels: the blocks that every sequence needs, the blocks moved, the slots.  A kernel of its own for the slots reads finished
// tables; with the slots in the second one, whose workgroups then look up each grown block in the prefix sums, a call takes 17 instead
// of 13 us (64 sequences, one token, 112 rows) and 53 instead of 34 us (256 sequences, 342 tokens each, 256 rows: 90 MB of slots).
// Bound by the latency of the launches and of their chains of loads (some 12 us), and by the slots' writes where there are many
// new tokens: 22 us for the 90 MB.
#include <algorithm>

#include "common.h"

namespace skipkv {

namespace {

static_assert(SKIPKV_MAX_PAGES_BATCH * 12 + 2048 <= 64 * 1024, "three numbers per sequence in shared memory");
constexpr int kSeqs = 16;  // sequences per workgroup of the first kernel

// Blocks that every sequence needs, and a copy of the counts that the second kernel replaces.
__global__ void __launch_bounds__(256) k_pages_need(PagesArgs a) {
  __shared__ int32_t part[16][kSeqs];
  const int b = blockIdx.x * kSeqs + (threadIdx.x & 15), group = threadIdx.x >> 4;
  int top = 0;
  bool bad = false;
  if (b < a.batch) {
#pragma unroll 8
    for (int r = group; r < a.n_rows; r += 16) {
      const int n = a.len[(int64_t)r * a.batch + b];
      bad |= n < 0;
      top = max(top, n);
    }
  }
  part[group][threadIdx.x & 15] = bad ? -1 : top;
  __syncthreads();
  if (group == 0 && b < a.batch) {
    for (int i = 1; i < 16; ++i) {
      const int p = part[i][threadIdx.x];
      bad |= p < 0;
      top = max(top, p);
    }
    const int64_t fresh = a.new_off ? (int64_t)a.new_off[b + 1] - a.new_off[b] : 0;
    bad |= fresh < 0;
    const int64_t need = ((int64_t)top + fresh + a.block_size - 1) / a.block_size;
    a.need[b] = bad ? -1 : (int)std::min<int64_t>(need, 0x7FFFFFFF);
    a.was_held[b] = a.n_held[b];
    if (bad && a.dev_status) atomicOr(a.dev_status, SKIPKV_DEV_BAD_LENGTHS);
  }
  if (blockIdx.x == 0 && threadIdx.x == 0) a.was_held[a.batch] = *a.n_free;
}

// Inclusive prefix sum over the workgroup's 256 threads of two counts at once; *total: of all.
__device__ __forceinline__ longlong2 scan256(longlong2 v, longlong2 (&wave_total)[4], longlong2 *total) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
#pragma unroll
  for (int d = 1; d < 64; d *= 2) {
    const long long x = __shfl_up(v.x, d), y = __shfl_up(v.y, d);
    if (lane >= d) {
      v.x += x;
      v.y += y;
    }
  }
  if (lane == 63) wave_total[wave] = v;
  __syncthreads();
  longlong2 all{0, 0};
#pragma unroll
  for (int w = 0; w < 4; ++w) {
    if (w < wave) {
      v.x += wave_total[w].x;
      v.y += wave_total[w].y;
    }
    all.x += wave_total[w].x;
    all.y += wave_total[w].y;
  }
  *total = all;
  return v;
}

// Blocks given back and taken: table rows, counts and the stack.  Shared memory: three numbers per sequence.
__global__ void __launch_bounds__(256) k_pages_move(PagesArgs a) {
  extern __shared__ int32_t shared[];
  __shared__ longlong2 wave_total[4];
  __shared__ int any_bad;
  const int tid = threadIdx.x, n = a.batch, wg = blockIdx.x, n_wg = gridDim.x;
  int32_t *const s_held = shared;                                  // blocks held before
  int32_t *const s_back = shared + n, *const s_want = shared + 2 * n;  // prefix sums up to and including the sequence: blocks given back, blocks wanted
  const int free0 = a.was_held[n];
  if (tid == 0) any_bad = free0 < 0 || free0 > a.n_blocks;
  __syncthreads();
  // ---- both prefix sums: each thread its stretch, then the threads' totals
  const int per = (n + 255) / 256, lo = min(tid * per, n), hi = min(lo + per, n);
  longlong2 sums{0, 0};
  bool bad = false, short_row = false;
  for (int b = lo; b < hi; ++b) {
    const int held = a.was_held[b];
    int need = a.need[b];
    bad |= held < 0 || held > a.table_stride;
    short_row |= need > a.table_stride;
    if (need < 0 || need > a.table_stride) need = held;
    s_held[b] = held;
    s_back[b] = max(held - need, 0);
    s_want[b] = max(need - held, 0);
    sums.x += s_back[b];
    sums.y += s_want[b];
  }
  if (bad) any_bad = 1;  // every writer stores the same value
  longlong2 total;
  const longlong2 upto = scan256(sums, wave_total, &total);  // (its barrier is behind the writes of any_bad)
  const long long total_back = total.x;
  const bool refused = any_bad || free0 + total_back > a.n_blocks;
  if (wg == 0 && tid == 0) {
    a.was_held[n + 1] = refused;
    if (refused && a.dev_status) atomicOr(a.dev_status, SKIPKV_DEV_BAD_BLOCK_TABLE);
  }
  if (refused) return;
  const int top = free0 + (int)total_back;  // (at most n_blocks)
  long long back = upto.x - sums.x, want = upto.y - sums.y;
  for (int b = lo; b < hi; ++b) {
    back += s_back[b];
    want += s_want[b];
    s_back[b] = (int)back;
    s_want[b] = (int)min(want, (long long)0x7FFFFFFF);
  }
  __syncthreads();
  auto first_above = [&](const int32_t *of, int x) {  // first sequence whose sum exceeds x
    int l = 0, h = n;
    while (l < h) {
      const int mid = (l + h) / 2;
      if (of[mid] > x) h = mid;
      else l = mid + 1;
    }
    return l;
  };
  // sequences from here on do not grow, those before it take all that they want
  const int n_served = total.y <= top ? n : first_above(s_want, top);
  const int taken = n_served > 0 ? s_want[n_served - 1] : 0;
  const int left = top - taken;
  auto at = [&](int pos) -> int32_t {  // entry of the stack after all releases
    if (pos < free0) return a.free_list[pos];
    const int q = pos - free0, b = first_above(s_back, q);
    return a.block_table[(int64_t)b * a.table_stride + s_held[b] - s_back[b] + q];
  };
  auto before = [&](const int32_t *of, int b) { return b > 0 ? of[b - 1] : 0; };
  auto grown_at = [&](int b, int i) { return at(top - 1 - before(s_want, b) - (i - s_held[b])); };
  auto held_after = [&](int b) {  // (a sequence that gives back wants none)
    return s_held[b] - (s_back[b] - before(s_back, b)) + (b < n_served ? s_want[b] - before(s_want, b) : 0);
  };
  if (wg == 0) {
    if (tid == 0) *a.n_free = left;
    if (a.dev_status && (short_row || (tid == 0 && total.y > taken))) atomicOr(a.dev_status, SKIPKV_DEV_OUT_OF_BLOCKS);
  }
  // (an id that does not exist is moved like any other, and reported)
  bool no_block = false;
  auto moved = [&](int32_t id) {
    no_block |= (uint32_t)id >= (uint32_t)a.n_blocks;
    return id;
  };
  // ---- blocks of the sequences that grow (entries behind n_held), a wave to each
  for (int b = wg * 4 + (tid >> 6); b < n; b += n_wg * 4) {
    const int held = s_held[b], now = held_after(b);
    for (int i = held + (tid & 63); i < now; i += 64) a.block_table[(int64_t)b * a.table_stride + i] = moved(grown_at(b, i));
    if ((tid & 63) == 0 && now != held) a.n_held[b] = now;
  }
  // ---- what stays on the stack of the blocks given back
  for (int i = free0 + wg * 256 + tid; i < left; i += n_wg * 256) a.free_list[i] = moved(at(i));
  if (no_block && a.dev_status) atomicOr(a.dev_status, SKIPKV_DEV_BAD_BLOCK_TABLE);
}

// Slots of the new tokens, from the tables as they are now.  grid = (tokens / 256, rows / rows_per_wg): a thread has one token in
// several rows.
__global__ void __launch_bounds__(256) k_pages_slots(PagesArgs a, int rows_per_wg, uint32_t div_mul, int div_shift) {
  __shared__ int wave_seq[4];
  __shared__ int32_t s_seq[256];  // a sequence whose tokens begin here (plus one), 0: none does
  const int tid = threadIdx.x, n = a.batch, tok0 = blockIdx.x * 256, tok = tok0 + tid;
  const bool refused = a.was_held[n + 1] != 0;
  s_seq[tid] = 0;
  __syncthreads();
  for (int b = tid; b < n; b += 256) {
    const int first = a.new_off[b], end = a.new_off[b + 1], need = a.need[b];
    if (need >= 0 && first < end && first < tok0 + 256ll && end > tok0) atomicMax(&s_seq[max(first, tok0) - tok0], b + 1);
  }
  __syncthreads();
  // the sequence of the thread's token: the last one that begins at or before it
  int seq = s_seq[tid];
#pragma unroll
  for (int d = 1; d < 64; d *= 2) {
    const int x = __shfl_up(seq, d);
    if ((tid & 63) >= d) seq = max(seq, x);
  }
  if ((tid & 63) == 63) wave_seq[tid >> 6] = seq;
  __syncthreads();
  for (int w = 0; w < (tid >> 6); ++w) seq = max(seq, wave_seq[w]);
  if (tok >= a.total_new) return;
  const int l = max(seq - 1, 0);
  const int64_t ahead = (int64_t)tok - a.new_off[l];
  const bool known = seq > 0 && !refused && ahead >= 0 && ahead <= 0x7FFFFFFF && tok < a.new_off[l + 1];
  const int held = known ? a.n_held[l] : 0;
  const int32_t *row = a.block_table + (int64_t)l * a.table_stride;
  // eight rows at a time: their lengths, then their entries of the table, then the slots, so that the loads overlap
  constexpr int kRows = 8;
  bool no_block = false;
  const int r1 = min((int)(blockIdx.y + 1) * rows_per_wg, a.n_rows);
  for (int r0 = blockIdx.y * rows_per_wg; r0 < r1; r0 += kRows) {
    uint32_t pos[kRows], bi[kRows];
    int32_t id[kRows];
#pragma unroll
    for (int i = 0; i < kRows; ++i) {
      const int len = (a.len + (int64_t)min(r0 + i, r1 - 1) * n)[l];
      pos[i] = len >= 0 && known ? (uint32_t)len + (uint32_t)ahead : 0xFFFFFFFFu;
    }
#pragma unroll
    for (int i = 0; i < kRows; ++i) {
      bi[i] = pos[i] <= 0x7FFFFFFFu ? __umulhi(pos[i] * 2, div_mul) >> div_shift : 0xFFFFFFFFu;
      id[i] = bi[i] < (uint32_t)held ? row[bi[i]] : 0;
    }
#pragma unroll
    for (int i = 0; i < kRows; ++i) {
      const uint32_t slot = (uint32_t)id[i] * (uint32_t)a.block_size + (pos[i] - bi[i] * (uint32_t)a.block_size);
      const bool exists = (uint32_t)id[i] < (uint32_t)a.n_blocks;
      no_block |= !exists;  // (0 where the sequence holds none, and the last row again)
      if (r0 + i < r1) (a.slot_map + (int64_t)(r0 + i) * a.total_new)[tok] = bi[i] < (uint32_t)held && exists ? (int32_t)slot : -1;
    }
  }
  if (no_block && a.dev_status) atomicOr(a.dev_status, SKIPKV_DEV_BAD_BLOCK_TABLE);
}

}  // namespace

hipError_t launch_pages_update(const PagesArgs &a, hipStream_t st) {
  hipLaunchKernelGGL(k_pages_need, dim3((a.batch + kSeqs - 1) / kSeqs), dim3(256), 0, st, a);
  // four sequences to a workgroup, a wave to each
  hipLaunchKernelGGL(k_pages_move, dim3(std::max(1, std::min(256, a.batch / 4))), dim3(256), (size_t)a.batch * 12, st, a);
  if (!a.slot_map) return hipGetLastError();
  // pos / d for pos < 2^31 as pos * m >> 31 + s, with 2^s >= d and m = 2^(31 + s) / d rounded up, e = m d - 2^(31 + s) < 2^s: the
  // product is above the quotient by pos e / (2^(31 + s) d) < 1 / d
  int div_shift = 0;
  while ((1ll << div_shift) < a.block_size) ++div_shift;
  const uint32_t div_mul = (uint32_t)(((1ull << (31 + div_shift)) + a.block_size - 1) / a.block_size);
  // eight rows to a thread, or a multiple of eight that leaves some 2048 workgroups
  const unsigned x = (unsigned)((a.total_new + 255ll) / 256);
  const int rows = (int)std::max<int64_t>(1, ((int64_t)a.n_rows * x + 2048 * 8 - 1) / (2048 * 8)) * 8;
  hipLaunchKernelGGL(k_pages_slots, dim3(x, (unsigned)((a.n_rows + rows - 1) / rows)), dim3(256), 0, st, a, rows, div_mul, div_shift);
  return hipGetLastError();
}

}  // namespace skipkv
