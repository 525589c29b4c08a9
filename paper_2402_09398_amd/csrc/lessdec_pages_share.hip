// Paged cache: what neighbouring slots have in common, as a plan for attention that reads it once.
//
// Slots that were forked from one another name the same pages from the beginning of their table rows on.  With a[k] the number of leading
// entries that the k-th slot that has rows shares with the one before it, the runs of slots that share more than their surroundings are the
// intervals of a (from one entry that is smaller than all within to the next), nested like the forks were: a node for each.  A node covers
// the entries from where the node around it ends up to the least a within it, and a slot's own part begins where its innermost node ends.
//
// Entries count as shared where the slots that see any of the page's tokens name the same page.  Of a window's pages every slot
// has let go what it no longer sees itself, so that one slot may name a page and the next one none; the slot whose rows lie furthest back sees all that
// any of them sees, and its row is the one that is read for the node.
//
// Made once a step for all layers, from a few bytes a page and slot: bound by the latency of its dependent steps.  No atomics but a minimum in the
// LDS; the same tables give the same plan.
#include "lessdec_pages.h"

namespace lessdec {
namespace {

constexpr int kMaxSlots = LESSDEC_MAX_SLOTS, kNever = 1 << 30;

// A slot as far as sharing goes.  entries: -1: no rows, not there; 0: shares nothing.
struct Sharer { int entries, seen_from, sinks, lo; };
__device__ inline Sharer sharer_of(const Pages &c, const int *start, int rows, int s)
{
  const Rows r = slot_rows(start, s, rows);
  const int len = slot_length(c, s), lo = len - r.count > 0 ? len - r.count : 0;
  Sharer x = {-1, 0, 0, lo};
  if (r.count == 0) return x;
  // (from 128 query columns on a slot's tiles are full by themselves)
  x.entries = r.count * c.q_per_kv >= kTrunkTile ? 0 : (len + c.page_tokens - 1) / c.page_tokens;
  if (c.window > 0 && lo >= c.window) {
    x.seen_from = (lo - c.window + 1) / c.page_tokens;
    x.sinks = (int)(((long)c.sinks + c.page_tokens - 1) / c.page_tokens);
  }
  return x;
}

// For every slot with rows the first entry, among a workgroup's, in which it differs from the one with rows before it.  A thread has a
// column of the table and goes down the slots with the page that was named last by one that sees it.
__global__ __launch_bounds__(256) void agree_kernel(Pages c, const int *start, int rows, Plan plan)
{
  extern __shared__ int shared[];
  int *entries = shared, *seen_from = shared + c.slots, *differs = shared + 2 * c.slots;
  __shared__ int most;
  const int tid = threadIdx.x, lane = tid & 63;
  if (tid == 0) most = 0;
  __syncthreads();
  int sinks = 0;
  for (int s = tid; s < c.slots; s += 256) {
    const Sharer x = sharer_of(c, start, rows, s);
    entries[s] = x.entries;
    seen_from[s] = x.seen_from;
    differs[s] = kNever;
    atomicMax(&most, x.entries);
    sinks = max(sinks, x.sinks);
  }
  // positions of the rows of the slots that can share
  for (int s = blockIdx.x; s < c.slots; s += gridDim.x) {
    const Rows r = slot_rows(start, s, rows);
    if (r.count == 0 || r.count * c.q_per_kv >= kTrunkTile) continue;
    const int before = slot_length(c, s) - r.count;
    for (int i = tid; i < r.count; i += 256) plan.pos[r.first + i] = before + i;
  }
  sinks = c.window > 0 ? (int)(((long)c.sinks + c.page_tokens - 1) / c.page_tokens) : 0;
  __syncthreads();
  for (int base = blockIdx.x * 256; base < most; base += gridDim.x * 256) {
    const int j = base + tid;
    const int *column = c.table + min(j, c.table_len - 1);
    constexpr int kAny = -2;
    int state = kAny, before = 0;                    // entries of the slot before
    for (int s0 = 0; s0 < c.slots; s0 += 16) {
      int page[16];
#pragma unroll
      for (int i = 0; i < 16; ++i) page[i] = column[(size_t)min(s0 + i, c.slots - 1) * c.table_len];
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        const int s = s0 + i;
        if (s >= c.slots || entries[s] < 0) continue;                  // (the same for all threads)
        const int now = (unsigned)page[i] < (unsigned)c.pages ? page[i] : -1;
        const bool sees = j >= seen_from[s] || j < sinks;
        const bool same = j < before && j < entries[s] && (!sees || state == kAny || state == now);
        if (sees || j >= entries[s]) state = now;
        before = entries[s];
        const unsigned long long not_same = __ballot(!same);
        if (not_same && lane == 0) atomicMin(differs + s, base + (tid & ~63) + __ffsll(not_same) - 1);
      }
    }
  }
  __syncthreads();
  for (int s = tid; s < c.slots; s += 256) plan.apart[(long)blockIdx.x * c.slots + s] = differs[s];
}

constexpr int kThreads = 1024, kWaves = kThreads / kWave, kTurns = kMaxSlots / kThreads;
// A node is worth its shares and their joining from so many tokens on, that it saves reading (tokens that it has, times slots but one).
constexpr int kLeastSaved = 256;

__device__ inline int scan_before(int x, int *sums, int &total)
{
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  int upto = x;
  for (int d = 1; d < kWave; d <<= 1) {
    const int y = __shfl_up(upto, d, kWave);
    if (lane >= d) upto += y;
  }
  __syncthreads();
  if (lane == 63) sums[wave] = upto;
  __syncthreads();
  int before = upto - x;
  total = 0;
  for (int w = 0; w < kWaves; ++w) {
    if (w < wave) before += sums[w];
    total += sums[w];
  }
  return before;
}

// Blocks that rows at lo .. hi see some token of, of those in [first, last).
__device__ inline int seen_blocks(const Pages &c, int lo, int hi, int first, int last)
{
  const int end = min(last, hi / kBlock + 1);
  if (c.window == 0 || lo < c.window) return max(end - first, 0);
  const int window = (lo - c.window + 1) / kBlock, sinks = (int)min(((long)c.sinks + kBlock - 1) / kBlock, (long)window);
  return max(min(end, sinks) - first, 0) + max(end - max(first, window), 0);
}

// One workgroup.  All arrays are indexed by the slots that have rows, in order: entry k and the boundary between the (k-1)-th and the k-th.
__global__ __launch_bounds__(kThreads) void plan_kernel(Pages c, const int *start, int rows, Plan plan, int agree_workers, int most_items, long most_columns)
{
  extern __shared__ int shared[];
  int *a = shared;                                   // entries in common across the boundary
  short *slot = reinterpret_cast<short *>(shared + c.slots), *left = slot + c.slots, *right = left + c.slots;
  short *same = right + c.slots;                     // the first boundary of the node
  short *around = same + c.slots;                    // that of the node around it, -1: none; later of the nearest one that is kept
  short *index = around + c.slots;                   // of the node in the plan, -1: not kept
  __shared__ int sums[kWaves], found;
  const int tid = threadIdx.x;
  int n = 0;
#pragma unroll
  for (int t = 0; t < kTurns; ++t) {
    if (t * kThreads >= c.slots) break;
    const int s = tid + t * kThreads;
    const bool there = s < c.slots && slot_rows(start, s, rows).count > 0;
    if (s < c.slots && !there) *reinterpret_cast<int2 *>(plan.slot + 2L * s) = make_int2(-1, 0);
    int all;
    const int at = n + scan_before(there, sums, all);
    if (there) slot[at] = (short)s;
    n += all;
  }
  __syncthreads();
  for (int k = tid; k < n; k += kThreads) {
    if (k == 0) { a[0] = 0; continue; }
    int x = min(sharer_of(c, start, rows, slot[k]).entries, sharer_of(c, start, rows, slot[k - 1]).entries);
    for (int w = 0; w < agree_workers; w += 8) {
      int y[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) y[i] = plan.apart[(long)min(w + i, agree_workers - 1) * c.slots + slot[k]];
#pragma unroll
      for (int i = 0; i < 8; ++i) x = min(x, y[i]);
    }
    a[k] = x;
  }
  __syncthreads();
  // intervals: from the boundary to the left that is smaller (one as large: the same node as that) to the one on the right
  for (int k = tid; k < n; k += kThreads) {
    same[k] = left[k] = right[k] = around[k] = index[k] = -1;
    if (a[k] == 0) continue;
    int i = k - 1;
    while (a[i] > a[k]) --i;                         // (a[0] is 0)
    same[k] = (short)(a[i] == a[k] ? i : k);
    if (same[k] != k) continue;
    left[k] = (short)i;
    int j = k + 1;
    while (j < n && a[j] >= a[k]) ++j;
    right[k] = (short)j;
  }
  __syncthreads();
  for (;;) {                                         // the chains of `same`, halved at a time
    bool more = false;
    short next[kTurns];
#pragma unroll
    for (int t = 0; t < kTurns; ++t) {
      const int k = tid + t * kThreads;
      next[t] = -1;
      if (k < n && same[k] >= 0) {
        next[t] = same[same[k]];
        more |= next[t] != same[k];
      }
    }
    more = __syncthreads_or(more);
#pragma unroll
    for (int t = 0; t < kTurns; ++t)
      if (next[t] >= 0) same[tid + t * kThreads] = next[t];
    __syncthreads();
    if (!more) break;
  }
  // which nodes are worth it, and what is around them
  for (int k = tid; k < n; k += kThreads) {
    if (same[k] != k) continue;
    const int l = left[k], r = right[k], below = r < n ? a[r] : 0, from = max(a[l], below);
    if (from > 0) around[k] = same[a[l] >= below ? l : r];
    int lo = kNever, hi = 0;
    for (int i = l; i < r; ++i) {
      const int s = slot[i], len = slot_length(c, s), count = slot_rows(start, s, rows).count;
      lo = min(lo, max(len - count, 0));
      hi = max(hi, len - 1);
      if (c.window == 0) break;                      // (nothing below asks for the others)
    }
    const long saved = (long)seen_blocks(c, lo, c.window ? hi : kNever, from * page_blocks(c), a[k] * page_blocks(c)) * kBlock * (r - l - 1);
    index[k] = saved >= kLeastSaved ? 0 : -1;
  }
  __syncthreads();
  short keep[kTurns], near[kTurns];
#pragma unroll
  for (int t = 0; t < kTurns; ++t) {
    const int k = tid + t * kThreads;
    keep[t] = 0;
    near[t] = -1;
    if (k >= n || same[k] != k) continue;
    // the nodes around it that are worth it, the outermost kTrunkDepth of which are kept
    int depth = 0;
    for (int i = around[k]; i >= 0; i = around[i]) depth += index[i] >= 0;
    keep[t] = index[k] >= 0 && depth < kTrunkDepth;
    int past = max(depth - kTrunkDepth, 0);
    for (int i = around[k]; i >= 0; i = around[i]) {
      if (index[i] < 0) continue;
      if (past == 0) { near[t] = (short)i; break; }
      --past;
    }
  }
  __syncthreads();
  int nodes = 0;
#pragma unroll
  for (int t = 0; t < kTurns; ++t) {
    if (t * kThreads >= n) break;
    const int k = tid + t * kThreads;
    int all;
    const int at = nodes + scan_before(keep[t], sums, all);
    if (k < n && same[k] == k) {
      index[k] = keep[t] ? (short)at : (short)-1;
      around[k] = near[t];
    }
    nodes += all;
  }
  __syncthreads();
  // records of the nodes
  const int per = page_blocks(c);
  for (int k = tid; k < n; k += kThreads) {
    if (same[k] != k || index[k] < 0) continue;
    const int l = left[k], r = right[k], up = around[k];
    const int row = slot_rows(start, slot[l], rows).first;
    int lo = kNever, hi = 0, read = slot[l], end = row;
    for (int i = l; i < r; ++i) {
      const Rows x = slot_rows(start, slot[i], rows);
      const int len = slot_length(c, slot[i]), from = max(len - x.count, 0);
      if (from < lo) { lo = from; read = slot[i]; }
      hi = max(hi, len - 1);
      end = max(end, x.first + x.count);
    }
    int *f = plan.node + (long)index[k] * kNodeInts;
    f[0] = read; f[1] = row; f[3] = lo; f[4] = hi;
    f[2] = (long)(end - row) * c.q_per_kv <= (r - l) * (kTrunkTile - 1) ? end - row : 0;       // (not for a start that does not ascend)
    f[5] = (up < 0 ? 0 : a[up]) * per;
    f[6] = a[k] * per;
    f[8] = up < 0 ? -1 : index[up];
  }
  // the slots': their innermost node is that of the larger of their two boundaries
  for (int k = tid; k < n; k += kThreads) {
    const int b = k + 1 < n && a[k + 1] > a[k] ? k + 1 : k;
    int i = same[b];
    if (i >= 0 && index[i] < 0) i = around[i];
    *reinterpret_cast<int2 *>(plan.slot + 2 * slot[k]) = i >= 0 ? make_int2(index[i], a[i] * per) : make_int2(-1, 0);
  }
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
  __syncthreads();
  // Splits: tiles of 64 tokens to an item, the fewest with which the items of all heads do not outnumber the workgroups (where that can be)
  const int most = max(kTrunkWorkers / c.heads, 1);
  int node_tiles[kTurns], columns[kTurns], length = 0;
#pragma unroll
  for (int t = 0; t < kTurns; ++t) {
    const int i = tid + t * kThreads;
    node_tiles[t] = columns[t] = 0;
    if (i >= nodes) continue;
    const int *f = plan.node + (long)i * kNodeInts;
    columns[t] = f[2] * c.q_per_kv;
    node_tiles[t] = (seen_blocks(c, f[3], f[4], f[5], f[6]) + 3) / 4;
  }
  auto total_of = [&](auto of) {
    int x = 0;
#pragma unroll
    for (int t = 0; t < kTurns; ++t) x += of(t);
    int all;
    scan_before(x, sums, all);
    return all;
  };
  auto tall = [&](int t) { return (columns[t] + kTrunkTile - 1) / kTrunkTile; };
  if (tid == 0) found = 0;
  __syncthreads();
#pragma unroll
  for (int t = 0; t < kTurns; ++t)
    if (node_tiles[t]) atomicMax(&found, node_tiles[t]);
  __syncthreads();
  const int longest = found;
  // bisection: how many items there are falls with the length
  int few = 2, many = max(longest, 2);
  while (few < many) {
    length = (few + many) / 2;
    if (total_of([&](int t) { return tall(t) * ((node_tiles[t] + length - 1) / length); }) <= most) many = length;
    else few = length + 1;
  }
  length = many;
  int items = 0;
  long in_all = 0;
#pragma unroll
  for (int t = 0; t < kTurns; ++t) {
    if (t * kThreads >= nodes) break;
    const int i = tid + t * kThreads, splits = (node_tiles[t] + length - 1) / length;
    int all, wide;
    const int at = items + scan_before(tall(t) * splits, sums, all);
    const long base = in_all + scan_before(columns[t] * splits, sums, wide);
    if (i < nodes) {
      int *f = plan.node + (long)i * kNodeInts;
      const bool fits = base + (long)columns[t] * splits <= most_columns && at + tall(t) * splits <= most_items;
      f[7] = (int)base;
      f[9] = fits ? splits : 0;
      f[10] = at;
    }
    items += all;
    in_all += wide;
  }
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
  __syncthreads();
  // the items: a wave has a node, neighbours are the tiles of columns over the same tokens
  for (int i = tid / kWave; i < nodes; i += kWaves) {
    const int *f = plan.node + (long)i * kNodeInts;
    const int wide = (f[2] * c.q_per_kv + kTrunkTile - 1) / kTrunkTile, splits = f[9], tiles = (seen_blocks(c, f[3], f[4], f[5], f[6]) + 3) / 4;
    for (int e = tid & 63; e < wide * splits; e += kWave) {
      const int split = e / wide, column = e - split * wide;
      *reinterpret_cast<int4 *>(plan.item + 4L * (f[10] + e)) = make_int4(i, column | split << 16, split * length, min(tiles, (split + 1) * length));
    }
  }
  if (tid == 0) {
    plan.head[kPlanNodes] = nodes;
    plan.head[kPlanItems] = min(items, most_items);
    plan.head[kPlanColumns] = (int)in_all;
    plan.head[kPlanRows] = rows;
  }
}

}  // namespace

hipError_t launch_pages_share(const Pages &c, const int *start, int rows, const Plan &plan, int items, long columns, hipStream_t st)
{
  const int wide = (c.table_len + 255) / 256, workers = wide < kAgreeWorkers ? wide : kAgreeWorkers;
  agree_kernel<<<workers, 256, (size_t)c.slots * 3 * sizeof(int), st>>>(c, start, rows, plan);
  const size_t lds = (size_t)c.slots * (sizeof(int) + 6 * sizeof(short));
  if (lds > 60000) {
    const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void *>(plan_kernel), hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds);
    if (e != hipSuccess) return e;
  }
  plan_kernel<<<1, kThreads, lds, st>>>(c, start, rows, plan, workers, items, columns);
  return hipGetLastError();
}

}  // namespace lessdec
