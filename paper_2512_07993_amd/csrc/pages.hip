// Block tables of a paged cache: blocks given back by sequences that became shorter, blocks taken by those that grow, and the
// slots of the new tokens, from the lengths on the GPU.
//
// With P the prefix sums over sequences of the blocks given back, the stack of free blocks after all releases is the old one with
// entry need_b + i of sequence b's table row at n_free + P_b + i; with G those of the blocks wanted, sequence b's i-th new block is the
// one at top - 1 - G_b - i, and it is served iff its end G_b + grow_b is at most top.  Every workgroup forms both sums for itself (a few
// thousand numbers), so that nothing is passed between workgroups: an entry on top of the old stack is read from the
// table row that gives it back, not from the stack, and rows that give back are not written.  The result does not depend on any order.
//
// Bound by the two launches, and by the slots' writes where there are many new tokens.
#include <algorithm>

#include "common.h"

namespace skipkv {

namespace {

static_assert(SKIPKV_MAX_PAGES_BATCH * 16 <= 64 * 1024, "four numbers per sequence in shared memory");
constexpr int kSeqs = 16;  // sequences per workgroup of the first kernel

// Blocks that every sequence needs, and a copy of the counts that the second kernel replaces.
__global__ void __launch_bounds__(256) k_pages_need(PagesArgs a) {
  __shared__ int32_t part[16][kSeqs];
  const int b = blockIdx.x * kSeqs + (threadIdx.x & 15), group = threadIdx.x >> 4;
  int top = 0;
  bool bad = false;
  if (b < a.batch) {
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

// grid = (tokens of the slot map / 256, rows of it / rows_per_wg).  Shared memory: four numbers per sequence.
__global__ void __launch_bounds__(256) k_pages_move(PagesArgs a, int rows_per_wg) {
  extern __shared__ int32_t shared[];
  __shared__ longlong2 wave_total[4];
  __shared__ int any_bad;
  const int tid = threadIdx.x, n = a.batch, wg = blockIdx.y * gridDim.x + blockIdx.x, n_wg = gridDim.x * gridDim.y;
  int32_t *const s_held = shared, *const s_need = shared + n;             // before; after (equal where a sequence stays as it is)
  int32_t *const s_back = shared + 2 * n, *const s_want = shared + 3 * n;  // prefix sums up to and including the sequence: blocks given back, blocks wanted
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
    s_need[b] = need;
    sums.x += max(held - need, 0);
    sums.y += max(need - held, 0);
  }
  if (bad) any_bad = 1;  // every writer stores the same value
  longlong2 total;
  const longlong2 upto = scan256(sums, wave_total, &total);  // (its barrier is behind the writes of any_bad)
  const long long total_back = total.x;
  if (any_bad || free0 + total_back > a.n_blocks) {
    if (wg == 0 && tid == 0 && a.dev_status) atomicOr(a.dev_status, SKIPKV_DEV_BAD_BLOCK_TABLE);
    if (a.slot_map)
      for (int64_t i = (int64_t)wg * 256 + tid; i < (int64_t)a.n_rows * a.total_new; i += (int64_t)n_wg * 256) a.slot_map[i] = -1;
    return;
  }
  const int top = free0 + (int)total_back;  // (at most n_blocks)
  long long back = upto.x - sums.x, want = upto.y - sums.y;
  for (int b = lo; b < hi; ++b) {
    back += max(s_held[b] - s_need[b], 0);
    want += max(s_need[b] - s_held[b], 0);
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
    return a.block_table[(int64_t)b * a.table_stride + s_need[b] + q - (b > 0 ? s_back[b - 1] : 0)];
  };
  auto grown_at = [&](int b, int i) { return at(top - 1 - (b > 0 ? s_want[b - 1] : 0) - (i - s_held[b])); };
  auto held_after = [&](int b) { return s_need[b] > s_held[b] && b >= n_served ? s_held[b] : s_need[b]; };
  if (wg == 0) {
    if (tid == 0) *a.n_free = left;
    if (a.dev_status && (short_row || (tid == 0 && total.y > taken))) atomicOr(a.dev_status, SKIPKV_DEV_OUT_OF_BLOCKS);
  }
  // ---- blocks of the sequences that grow (entries behind n_held), a wave to each
  for (int b = wg * 4 + (tid >> 6); b < n; b += n_wg * 4) {
    const int held = s_held[b], now = held_after(b);
    for (int i = held + (tid & 63); i < now; i += 64) a.block_table[(int64_t)b * a.table_stride + i] = grown_at(b, i);
    if ((tid & 63) == 0 && now != held) a.n_held[b] = now;
  }
  // ---- what stays on the stack of the blocks given back
  for (int i = free0 + wg * 256 + tid; i < left; i += n_wg * 256) a.free_list[i] = at(i);
  // ---- slots of the new tokens: a thread has one token in several rows
  const int tok = blockIdx.x * 256 + tid;
  if (!a.slot_map || tok >= a.total_new) return;
  int l = 0, h = n;  // the sequence: the last whose first new token is at or before this one
  while (h - l > 1) {
    const int mid = (l + h) / 2;
    if (a.new_off[mid] <= tok) l = mid;
    else h = mid;
  }
  const int ahead = tok - a.new_off[l], now = held_after(l), was = s_held[l];
  const bool known = a.need[l] >= 0 && ahead >= 0;
  const int32_t *row = a.block_table + (int64_t)l * a.table_stride;
  const int r1 = min((int)(blockIdx.y + 1) * rows_per_wg, a.n_rows);
#pragma unroll 4
  for (int r = blockIdx.y * rows_per_wg; r < r1; ++r) {
    const int64_t pos = (int64_t)a.len[(int64_t)r * n + l] + ahead;
    int32_t slot = -1;
    if (known && pos >= 0 && pos <= 0x7FFFFFFF) {
      const uint32_t bi = (uint32_t)pos / (uint32_t)a.block_size;
      if (bi < (uint32_t)now) {
        const int32_t id = bi < (uint32_t)was ? row[bi] : grown_at(l, (int)bi);
        slot = (int32_t)((uint32_t)id * (uint32_t)a.block_size + ((uint32_t)pos - bi * (uint32_t)a.block_size));
      }
    }
    a.slot_map[(int64_t)r * a.total_new + tok] = slot;
  }
}

}  // namespace

hipError_t launch_pages_update(const PagesArgs &a, hipStream_t st) {
  hipLaunchKernelGGL(k_pages_need, dim3((a.batch + kSeqs - 1) / kSeqs), dim3(256), 0, st, a);
  // a thread per new token and 8 rows of the slot map, or as many rows as leave some 2048 workgroups; without a slot map a
  // workgroup per 16 sequences
  unsigned x = (unsigned)std::max(1, std::min(256, a.batch / 16)), y = 1;
  int rows = 1;
  if (a.slot_map) {
    x = (unsigned)((a.total_new + 255) / 256);
    rows = (int)std::max<int64_t>(8, ((int64_t)a.n_rows * x + 2047) / 2048);
    y = (unsigned)((a.n_rows + rows - 1) / rows);
  }
  hipLaunchKernelGGL(k_pages_move, dim3(x, y), dim3(256), (size_t)a.batch * 16, st, a, rows);
  return hipGetLastError();
}

}  // namespace skipkv
