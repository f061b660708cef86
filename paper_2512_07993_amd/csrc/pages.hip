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

constexpr int kMaxB = SKIPKV_MAX_PAGES_BATCH;
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

struct Tables {
  int32_t held[kMaxB], need[kMaxB];      // before; after (equal where a sequence stays as it is)
  int32_t back[kMaxB], want[kMaxB];      // prefix sums up to and including the sequence: blocks given back, blocks wanted
  int64_t tsum[2][256];
  int32_t bad;
};

__global__ void __launch_bounds__(256) k_pages_move(PagesArgs a) {
  __shared__ Tables s;
  const int tid = threadIdx.x, n = a.batch;
  const int free0 = a.was_held[n];
  if (tid == 0) s.bad = free0 < 0 || free0 > a.n_blocks;
  __syncthreads();
  // ---- both prefix sums: each thread its stretch, then the threads' totals
  const int per = (n + 255) / 256, lo = min(tid * per, n), hi = min(lo + per, n);
  int64_t back = 0, want = 0;
  bool bad = false, short_row = false;
  for (int b = lo; b < hi; ++b) {
    const int held = a.was_held[b];
    int need = a.need[b];
    bad |= held < 0 || held > a.table_stride;
    short_row |= need > a.table_stride;
    if (need < 0 || need > a.table_stride) need = held;
    s.held[b] = held;
    s.need[b] = need;
    back += max(held - need, 0);
    want += max(need - held, 0);
  }
  if (bad) s.bad = 1;  // every writer stores the same value
  s.tsum[0][tid] = back;
  s.tsum[1][tid] = want;
  __syncthreads();
  int64_t off[2] = {0, 0}, total_back = 0;
  for (int i = 0; i < 256; ++i) {
    if (i < tid) {
      off[0] += s.tsum[0][i];
      off[1] += s.tsum[1][i];
    }
    total_back += s.tsum[0][i];
  }
  const bool corrupt = s.bad || free0 + total_back > a.n_blocks;
  if (corrupt) {
    if (blockIdx.x == 0 && tid == 0 && a.dev_status) atomicOr(a.dev_status, SKIPKV_DEV_BAD_BLOCK_TABLE);
    if (a.slot_map)
      for (int64_t i = (int64_t)blockIdx.x * 256 + tid; i < (int64_t)a.n_rows * a.total_new; i += (int64_t)gridDim.x * 256) a.slot_map[i] = -1;
    return;
  }
  const int top = free0 + (int)total_back;  // (at most n_blocks)
  for (int b = lo; b < hi; ++b) {
    off[0] += max(s.held[b] - s.need[b], 0);
    off[1] += max(s.need[b] - s.held[b], 0);
    s.back[b] = (int)off[0];
    s.want[b] = (int)std::min<int64_t>(off[1], 0x7FFFFFFF);
  }
  __syncthreads();
  // blocks that are taken: those of the last sequence that is served (the sums only rise)
  auto first_above = [&](const int32_t *sums, int x) {  // first sequence whose sum exceeds x
    int l = 0, h = n;
    while (l < h) {
      const int mid = (l + h) / 2;
      if (sums[mid] > x) h = mid;
      else l = mid + 1;
    }
    return l;
  };
  const int n_served = first_above(s.want, top);  // sequences from here on do not grow
  const int taken = n_served > 0 ? s.want[n_served - 1] : 0;
  const int left = top - taken;
  auto at = [&](int pos) -> int32_t {  // entry of the stack after all releases
    if (pos < free0) return a.free_list[pos];
    const int q = pos - free0, b = first_above(s.back, q);
    return a.block_table[(int64_t)b * a.table_stride + s.need[b] + q - (b > 0 ? s.back[b - 1] : 0)];
  };
  auto grown_at = [&](int b, int i) { return at(top - 1 - (b > 0 ? s.want[b - 1] : 0) - (i - s.held[b])); };
  auto held_after = [&](int b) { return s.need[b] > s.held[b] && b >= n_served ? s.held[b] : s.need[b]; };
  if (blockIdx.x == 0) {
    if (tid == 0) *a.n_free = left;
    if (a.dev_status && (short_row || (tid == 0 && n_served < n && s.want[n - 1] > taken))) atomicOr(a.dev_status, SKIPKV_DEV_OUT_OF_BLOCKS);
  }
  // ---- blocks of the sequences that grow (entries behind n_held), a wave to each
  for (int b = blockIdx.x * 4 + (tid >> 6); b < n; b += gridDim.x * 4) {
    const int held = s.held[b], now = held_after(b);
    for (int i = held + (tid & 63); i < now; i += 64) a.block_table[(int64_t)b * a.table_stride + i] = grown_at(b, i);
    if ((tid & 63) == 0 && now != held) a.n_held[b] = now;
  }
  // ---- what stays on the stack of the blocks given back
  for (int i = free0 + blockIdx.x * 256 + tid; i < left; i += gridDim.x * 256) a.free_list[i] = at(i);
  // ---- slots of the new tokens
  if (!a.slot_map) return;
  const int64_t slots = (int64_t)a.n_rows * a.total_new;
  for (int64_t i = (int64_t)blockIdx.x * 256 + tid; i < slots; i += (int64_t)gridDim.x * 256) {
    const int r = (int)(i / a.total_new), tok = (int)(i - (int64_t)r * a.total_new);
    int l = 0, h = n;  // the sequence: the last whose first new token is at or before this one
    while (h - l > 1) {
      const int mid = (l + h) / 2;
      if (a.new_off[mid] <= tok) l = mid;
      else h = mid;
    }
    const int64_t pos = (int64_t)a.len[(int64_t)r * n + l] + tok - a.new_off[l];
    const int64_t bi = pos / a.block_size;
    int32_t slot = -1;
    if (a.need[l] >= 0 && tok >= a.new_off[l] && pos >= 0 && bi < held_after(l)) {
      const int32_t id = bi < s.held[l] ? a.block_table[(int64_t)l * a.table_stride + bi] : grown_at(l, (int)bi);
      slot = (int32_t)((int64_t)id * a.block_size + pos - bi * a.block_size);
    }
    a.slot_map[i] = slot;
  }
}

}  // namespace

hipError_t launch_pages_update(const PagesArgs &a, hipStream_t st) {
  hipLaunchKernelGGL(k_pages_need, dim3((a.batch + kSeqs - 1) / kSeqs), dim3(256), 0, st, a);
  // a workgroup per 4096 slots or 16 sequences, up to one per CU and then some
  const int64_t by_slots = a.slot_map ? (int64_t)a.n_rows * a.total_new / 4096 : 0;
  const unsigned grid = (unsigned)std::max<int64_t>(1, std::min<int64_t>(512, std::max<int64_t>(by_slots, a.batch / 16)));
  hipLaunchKernelGGL(k_pages_move, dim3(grid), dim3(256), 0, st, a);
  return hipGetLastError();
}

}  // namespace skipkv
