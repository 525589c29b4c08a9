// Paged cache: what neighbouring slots have in common, as a plan for attention that reads it once.
//
// Slots that were forked from one another name the same pages from the beginning of their table rows on.  With a[k] the number of leading
// entries that the k-th slot that has rows shares with the one before it, the runs of slots that share more than their surroundings are the
// intervals of a (from one entry that is smaller than all within to the next), nested like the forks were: a node for each.  A node covers
// the entries from where the node around it ends up to the least a within it; what is behind a slot's innermost node is a node of its own.
//
// Entries count as shared where the slots that see any of the page's tokens name the same page.  What a slot names that it does not see says
// nothing: it may have let go of it or not.  So neighbours are compared where both see the page, and what a slot sees and the one before it does not
// is compared with the last slot before that which does: where these differ, they have no node with the entry, and one of the boundaries between them is
// cut.  The slot whose rows lie furthest back sees all that any of them sees, and its row is the one that is read for the node.
//
// Made once a step for all layers, from a few bytes a page and slot: bound by the latency of its dependent steps.  The same tables give
// the same plan.
#include "lessdec_pages.h"

namespace lessdec {
namespace {

// A slot as far as sharing goes.  entries: 0: shares nothing.
struct Sharer { Rows rows; int len, lo, entries; };
__device__ inline Sharer sharer_of(const Pages &c, const int *start, int rows, int s)
{
  Sharer x;
  x.rows = slot_rows(start, s, rows);
  x.len = slot_length(c, s);
  x.lo = max(x.len - x.rows.count, 0);
  // (from 128 query columns on a slot's tiles are full by themselves)
  x.entries = x.rows.count * c.q_per_kv >= kTrunkTile ? 0 : (x.len + c.page_tokens - 1) / c.page_tokens;
  return x;
}
// the first entry behind those of the first tokens that rows from position lo on see
__device__ inline int first_seen(const Pages &c, int lo)
{
  if (c.window == 0 || lo < c.window) return 0;
  return max((lo - c.window + 1) / c.page_tokens, (int)min(((long)c.sinks + c.page_tokens - 1) / c.page_tokens, (long)c.table_len));
}
__device__ inline bool sees_entry(const Pages &c, int lo, int j) { return j >= first_seen(c, lo) || (long)j * c.page_tokens < c.sinks; }

// A wave for every slot: positions of its rows, and how many leading entries it shares with the slot that has rows before it, up to the first that both
// see and name differently, sixteen entries a lane on their way; with a window also the first that it sees and the slot before it does not, and that the last one
// before which does names differently, and that one (of several the nearest), or -1.
// 64 slots of up to 8192 tokens: 4.8 us; with a window and lengths that all differ 8.0.
constexpr int kEach = 16;
__device__ inline int2 *cuts_of(const Plan &plan) { return reinterpret_cast<int2 *>(plan.few); }       // (not made yet)
__global__ __launch_bounds__(256) void agree_kernel(Pages c, const int *start, int rows, Plan plan)
{
  const int s = __builtin_amdgcn_readfirstlane((blockIdx.x * 256 + threadIdx.x) / kWave), lane = threadIdx.x & 63;
  if (s >= c.slots) return;
  const Sharer me = sharer_of(c, start, rows, s);
  int same = 0;
  int2 cut = make_int2(-1, -1);
  if (me.rows.count > 0 && me.entries > 0) {
    for (int i = lane; i < me.rows.count; i += kWave) plan.pos[me.rows.first + i] = me.len - me.rows.count + i;
    // the slot with rows before x, -1: none
    auto before = [&](int x) {
      for (; x > 0; x -= kWave) {
        const int i = x - 1 - lane;
        const unsigned long long there = __ballot(i >= 0 && slot_rows(start, max(i, 0), rows).count > 0);
        if (there) return x - __ffsll(there);
      }
      return -1;
    };
    const int first = before(s);
    const Sharer other = sharer_of(c, start, rows, max(first, 0));
    const int most = first < 0 ? 0 : min(me.entries, other.entries);
    const int *mine = c.table + (size_t)s * c.table_len, *theirs = c.table + (size_t)max(first, 0) * c.table_len;
    auto page_of = [&](int x) { return (unsigned)x < (unsigned)c.pages ? x : -1; };
    same = most;
    for (int base = 0; base < most; base += kEach * kWave) {
      int x[kEach], y[kEach];
#pragma unroll
      for (int i = 0; i < kEach; ++i) {
        const int j = min(base + i * kWave + lane, most - 1);
        x[i] = mine[j];
        y[i] = theirs[j];
      }
      unsigned apart = 0;
#pragma unroll
      for (int i = 0; i < kEach; ++i) apart |= (unsigned)(page_of(x[i]) != page_of(y[i])) << i;
      if (!__ballot(apart)) continue;
      int differs = most;
      for (int i = 0; i < kEach && differs == most; ++i) {
        const int j = base + i * kWave + lane;
        const bool differ = (apart >> i & 1) && j < most && sees_entry(c, me.lo, j) && sees_entry(c, other.lo, j);
        const unsigned long long who = __ballot(differ);
        if (who) differs = base + i * kWave + __ffsll(who) - 1;
      }
      if (differs < most) { same = differs; break; }
    }
    const int to = first < 0 ? 0 : min(first_seen(c, other.lo), same);
    for (int base = first_seen(c, me.lo); base < to; base += kWave) {
      const int j = base + lane;
      bool asking = j < to;
      int asked = -1;                                // the last slot that sees the entry, if a node could have both
      for (int end = first; __ballot(asking); end -= kWave) {          // 64 slots at a time, from registers
        const Sharer z = sharer_of(c, start, rows, max(end - 1 - lane, 0));
        const int seen = first_seen(c, z.lo);
        for (int l = 0; l < kWave && __ballot(asking); ++l) {
          const int at = end - 1 - l, entries = __builtin_amdgcn_readlane(z.entries, l), from = __builtin_amdgcn_readlane(seen, l);
          if (at >= 0 && __builtin_amdgcn_readlane(z.rows.count, l) == 0) continue;
          if (at < 0 || entries == 0) {              // (no one sees it; or no run reaches past that slot)
            asking = false;
          } else if (asking && from <= j) {
            if (j < entries) asked = at;
            asking = false;
          }
        }
      }
      if (asked >= 0 && page_of(mine[j]) == page_of(c.table[(size_t)asked * c.table_len + j])) asked = -1;
      const unsigned long long who = __ballot(asked >= 0);
      if (!who) continue;
      if (cut.x < 0) cut.x = base + __ffsll(who) - 1;
      for (int d = 1; d < kWave; d <<= 1) asked = max(asked, __shfl_xor(asked, d, kWave));
      cut.y = max(cut.y, asked);
    }
  }
  if (lane == 0) {
    plan.apart[s] = same;
    if (c.window > 0) cuts_of(plan)[s] = cut;
  }
}

constexpr int kThreads = 512, kWaves = kThreads / kWave;
// A node is worth its shares and their joining from so many tokens on, that it saves reading (tokens that it has, times slots but one).  Pairs of slots
// that have 128 tokens in common behind 4096 of all 64, 8 heads: with 4 query heads 27.0 us as nodes and 28.3 without, with 16 of them 59.8 and 48.6;
// 256 tokens: 27.7 and 28.8; 512: 30.8 and 48.
constexpr int kLeastSaved = 256;
// All of them together are worth it from so many bytes of a layer on that are not read.  16 MB (64 slots, a window of 2044, one head of 64): 25.4 us shared,
// 24.4 with the same launches and nothing shared; 25 MB (4 slots, 1030 tokens, 32 heads): 19.8 and 17.8; 63 MB (16 slots, 2048 tokens, 8 heads): 15.7, 18.9 apart;
// 528 MB (64 slots, 8192 tokens): 34, 132 apart.
constexpr long kLeastBytes = 32L << 20;

// Blocks that rows at lo .. hi see some token of, of those in [first, last).
__device__ inline int seen_blocks(const Pages &c, int lo, int hi, int first, int last)
{
  const int end = min(last, hi / kBlock + 1);
  if (hi < 0) return 0;
  if (c.window == 0 || lo < c.window) return max(end - first, 0);
  const int window = (lo - c.window + 1) / kBlock, sinks = (int)min(((long)c.sinks + kBlock - 1) / kBlock, (long)window);
  return max(min(end, sinks) - first, 0) + max(end - max(first, window), 0);
}

// What the plan kernel keeps of the slots that have rows, in order: entry k, and the boundary between the (k-1)-th and the k-th.
struct Runs {
  int *a;                                            // entries in common across the boundary
  int *hi, *row, *rows;                              // of the slot: largest position, first row, how many
  short *slot, *left, *right;                        // the slot; the boundaries around the node
  short *same;                                       // the first boundary of the node
  short *around;                                     // that of the node around it, -1: none
  short *worth;                                      // whether the node is worth its shares
  short *near;                                       // the nearest node around it that is kept
  short *index;                                      // of the node in the plan, -1: not kept
};
constexpr int kRunBytes = 4 * sizeof(int) + 8 * sizeof(short);

__global__ __launch_bounds__(kThreads) void plan_kernel(Pages c, const int *start, int rows, Plan plan, long most_columns, long least_bytes)
{
  extern __shared__ int shared[];
  __shared__ long sums[2][kWaves];
  __shared__ unsigned long long saved_in_all;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, N = c.slots, per = page_blocks(c), G = c.q_per_kv;
  Runs r;
  r.a = shared; r.hi = r.a + N; r.row = r.hi + N; r.rows = r.row + N;
  r.left = reinterpret_cast<short *>(r.rows + N);
  r.right = r.left + N; r.around = r.right + N; r.worth = r.around + N; r.slot = r.worth + N; r.same = r.slot + N; r.near = r.same + N; r.index = r.near + N;
  int *unit = r.rows + N;                            // of the plan's nodes, two a slot at most, once the four above are done with
  auto lo_of = [&](int k) { return max(r.hi[k] + 1 - r.rows[k], 0); };
  // sum over the threads before this one, and over all; sums are held twice, so that one barrier a call is enough
  int which = 0;
  auto scan = [&](auto x, auto &total) {
    auto upto = x;
    for (int d = 1; d < kWave; d <<= 1) {
      const auto y = __shfl_up(upto, d, kWave);
      if (lane >= d) upto += y;
    }
    if (lane == 63) sums[which][wave] = upto;
    __syncthreads();
    auto before = upto - x;
    total = 0;
    for (int w = 0; w < kWaves; ++w) {
      const auto y = (decltype(x))sums[which][w];
      if (w < wave) before += y;
      total += y;
    }
    which ^= 1;
    return before;
  };

  if (tid == 0) saved_in_all = 0;
  int n = 0;
  bool cut = false;
  for (int base = 0; base < N; base += kThreads) {
    const int s = base + tid;
    Sharer x;
    x.rows = Rows{0, 0};
    int same = 0;
    if (s < N) {
      x = sharer_of(c, start, rows, s);
      same = plan.apart[s];
      if (c.window > 0) cut |= cuts_of(plan)[s].x >= 0;
      *reinterpret_cast<int4 *>(plan.chain + 4L * (kTrunkDepth + 1) * s) = make_int4(-1, 0, 0, 0);
    }
    int all;
    const int at = n + scan((int)(x.rows.count > 0), all);
    if (x.rows.count > 0) {
      r.slot[at] = (short)s;
      r.a[at] = at == 0 ? 0 : same;
      r.hi[at] = x.len - 1;
      r.row[at] = x.rows.first;
      r.rows[at] = x.rows.count;
    }
    n += all;
  }
  if (__syncthreads_or(cut)) {
    // Of the boundaries between a slot and the one that it was compared with the one with the least in common is cut, unless that is no more than the entry
    // already (of equal ones the last): most likely that between two prompts.
    int *least = unit;                               // (what follows there is not in use yet)
    for (int k = tid; k < n; k += kThreads) least[k] = r.a[k];
    __syncthreads();
    for (int k = tid; k < n; k += kThreads) {
      const int2 x = cuts_of(plan)[r.slot[k]];
      if (x.x < 0) continue;
      int at = k;
      for (int i = k - 1; i > 0 && r.slot[i] > x.y; --i) at = r.a[i] < r.a[at] ? i : at;
      if (r.a[at] > x.x) atomicMin(least + at, x.x);
    }
    __syncthreads();
    for (int k = tid; k < n; k += kThreads) r.a[k] = least[k];
    __syncthreads();
  }
  // intervals: from the boundary to the left that is smaller (one as large: the same node as that) to the one on the right
  for (int base = wave * kWave; base < n; base += kThreads) {
    const int k = base + lane, mine = k < n ? r.a[k] : 0;
    // among the wave's 64, from which of them are smaller or as large, a bit each
    unsigned smaller[2], like[2];
#pragma unroll
    for (int half = 0; half < 2; ++half) {
      smaller[half] = like[half] = 0;
      for (int eight = 0; eight < 32 && half * 32 + eight < n - base; eight += 8)
#pragma unroll
        for (int q = eight; q < eight + 8; ++q) {
          const int x = __builtin_amdgcn_readlane(mine, half * 32 + q);
          smaller[half] |= (unsigned)(x < mine) << q;
          like[half] |= (unsigned)(x == mine) << q;
        }
    }
    if (k >= n) continue;
    r.same[k] = r.left[k] = r.right[k] = r.around[k] = r.worth[k] = r.near[k] = r.index[k] = -1;
    if (mine == 0) continue;
    const unsigned long long less = (unsigned long long)smaller[1] << 32 | smaller[0], before = less & ((1ull << lane) - 1), after = less & ~((2ull << lane) - 1);
    const int below = 63 - __clzll(before);          // (-1: none)
    const unsigned long long equal = ((unsigned long long)like[1] << 32 | like[0]) & ((1ull << lane) - 1) & ~((1ull << (below + 1)) - 1);
    int i = base + below, same = equal ? base + __ffsll(equal) - 1 : k;
    // and on through those before and behind, eight at a time
    for (bool more = same == k && !before; more;) {
      int x[8];
#pragma unroll
      for (int q = 0; q < 8; ++q) x[q] = r.a[max(i - q, 0)];
#pragma unroll
      for (int q = 0; q < 8; ++q) {                  // (a[0] is 0)
        more = more && x[q] >= mine;
        same = more && x[q] == mine ? i : same;
        i -= more;
      }
      more = more && same == k;
    }
    r.same[k] = (short)same;
    if (same != k) continue;
    int j = after ? base + __ffsll(after) - 1 : base + kWave;
    for (bool more = !after; more && j < n;) {
      int x[8];
#pragma unroll
      for (int q = 0; q < 8; ++q) x[q] = r.a[min(j + q, n - 1)];
#pragma unroll
      for (int q = 0; q < 8; ++q) {
        more = more && j < n && x[q] >= mine;
        j += more;
      }
    }
    r.left[k] = (short)i;
    r.right[k] = (short)min(j, n);
  }
  __syncthreads();
  for (bool more = n > kWave; more;) {               // the chains of `same` across waves, shortened until they have one link
    more = false;
    for (int k = tid; k < n; k += kThreads) {
      const int x = r.same[k], y = x >= 0 ? r.same[x] : -1;            // (whichever thread goes first, y is on k's chain)
      if (y != x) { r.same[k] = (short)y; more = true; }
    }
    more = __syncthreads_or(more);
  }
  // the slots of a run: least and largest position, and the first that has the least
  auto extent = [&](int l, int e, int &lo, int &hi, int &read) {
    lo = INT_MAX; hi = -1;
    int at = l;
#pragma unroll 8
    for (int i = l; i < e; ++i) {
      const int x = lo_of(i);
      at = x < lo ? i : at;
      lo = min(lo, x);
      hi = max(hi, r.hi[i]);
    }
    read = r.slot[at];
  };
  // which nodes are worth it, and what is around them; a thread's first node keeps its extent in registers
  int lo0 = 0, hi0 = 0, read0 = 0;
  for (int k = tid; k < n; k += kThreads) {
    if (r.same[k] != k) continue;
    const int l = r.left[k], e = r.right[k], below = e < n ? r.a[e] : 0, from = max(r.a[l], below);
    int lo, hi, read;
    extent(l, e, lo, hi, read);
    if (k == tid) { lo0 = lo; hi0 = hi; read0 = read; }
    const long saved = (long)seen_blocks(c, lo, hi, from * per, r.a[k] * per) * kBlock * (e - l - 1);
    if (from > 0) r.around[k] = r.same[r.a[l] >= below ? l : e];
    r.worth[k] = saved >= (least_bytes < 0 ? kLeastSaved : 1);
    if (r.worth[k]) atomicAdd(&saved_in_all, (unsigned long long)saved);
  }
  __syncthreads();
  const bool none = saved_in_all * (2ull * c.heads * c.head_dim) < (unsigned long long)(least_bytes < 0 ? kLeastBytes : least_bytes);
  // the outermost kTrunkDepth of the nodes around a slot are kept
  int nodes = 0;
  for (int base = 0; base < n; base += kThreads) {
    const int k = base + tid;
    bool keep = false;
    if (k < n && r.same[k] == k) {
      int depth = 0;
      for (int i = r.around[k]; i >= 0; i = r.around[i]) depth += r.worth[i];
      int past = max(depth - kTrunkDepth, 0);
      for (int i = r.around[k]; i >= 0; i = r.around[i])
        if (r.worth[i] && past-- == 0) { r.near[k] = (short)i; break; }
      keep = !none && r.worth[k] && depth < kTrunkDepth;
    }
    int all;
    const int at = nodes + scan((int)keep, all);
    if (keep) r.index[k] = (short)at;
    nodes += all;
  }
  __syncthreads();
  auto record = [&](int i, int read, int row, int count, int lo, int hi, int first, int last, int before) {
    int4 *f = reinterpret_cast<int4 *>(plan.node + (long)i * kNodeInts);
    f[0] = make_int4(read, row, count, lo);
    f[1] = make_int4(hi, first, last, before);
  };
  for (int k = tid; k < n; k += kThreads) {
    if (r.same[k] != k || r.index[k] < 0) continue;
    const int l = r.left[k], e = r.right[k], up = r.near[k], row = r.row[l], end = r.row[e - 1] + r.rows[e - 1];
    int lo = lo0, hi = hi0, read = read0;
    if (k != tid) extent(l, e, lo, hi, read);
    // (a start that does not ascend gives a node without rows)
    const int count = end > row && (long)(end - row) * G <= (e - l) * (kTrunkTile - 1) ? end - row : 0;
    record(r.index[k], read, row, count, lo, hi, (up < 0 ? 0 : r.a[up]) * per, r.a[k] * per, up < 0 ? -1 : r.index[up]);
  }
  // a slot's own part, behind its innermost node, which is that of the larger of its two boundaries
  int all_nodes = nodes, few = 0, short_ones = 0;
  long few_steps = 0;
  // an entry of few columns for those threads that have one; all threads call it
  auto list = [&](bool mine, int blocks, int read, int row, int count, int lo, int hi, int first, int last, int column, bool several) {
    const bool brief = blocks <= kShortBlocks;
    // three sums in one word: entries, short ones, steps
    long all;
    const long before = scan(!mine ? 0L : brief ? 1L << 14 : 1L | (long)((blocks + kFewBlocks - 1) / kFewBlocks) << 28, all);
    const int at = brief ? 3 * N - 1 - (short_ones + (int)(before >> 14 & 16383)) : few + (int)(before & 16383);
    few += (int)(all & 16383);
    short_ones += (int)(all >> 14 & 16383);
    few_steps += all >> 28;
    if (!mine) return;
    int4 *f = reinterpret_cast<int4 *>(plan.few + (long)at * kNodeInts);
    const int step = brief ? 2 : kFewBlocks;
    f[0] = make_int4(max((blocks + step - 1) / step, 1), read, row, count);
    f[1] = make_int4(lo, hi, first, last);
    f[2] = make_int4(column, several, 0, 0);
  };
  for (int base = 0; base < n; base += kThreads) {
    const int k = base + tid;
    int i = -1;
    if (k < n) {
      i = r.same[k + 1 < n && r.a[k + 1] > r.a[k] ? k + 1 : k];
      if (i >= 0 && r.index[i] < 0) i = r.near[i];
    }
    if (none) i = -1;
    // one that shares nothing has a node all the same if its columns are too many for the list of few and too few for tiles of its own
    const int columns = k < n ? r.rows[k] * G : 0;
    const bool own = i >= 0 || (columns > kFewColumns && columns < kTrunkTile);
    int all;
    const int at = all_nodes + scan((int)own, all);
    if (own) {
      record(at, r.slot[k], r.row[k], r.rows[k], lo_of(k), r.hi[k], i >= 0 ? r.a[i] * per : 0, kEndless, i >= 0 ? r.index[i] : -1);
      plan.chain[4L * (kTrunkDepth + 1) * r.slot[k] + 3] = at;
    }
    all_nodes += all;
    const bool direct = k < n && !own && columns <= kFewColumns;
    const int at_k = min(k, n - 1), lo = lo_of(at_k), hi = r.hi[at_k];
    list(direct, seen_blocks(c, lo, hi, 0, kEndless), r.slot[at_k], r.row[at_k], r.rows[at_k], lo, hi, 0, kEndless, -1, false);
  }
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
  __syncthreads();
  // tiles of the nodes of more than kFewColumns columns, steps of the others
  long tiles = 0, columns_of_tiles = 0;              // of a head: tiles, and columns of 128 that have some
  for (int base = 0; base < all_nodes; base += kThreads) {
    const int i = base + tid;
    int *f = plan.node + (long)min(i, all_nodes - 1) * kNodeInts;
    int mine = 0, wide = 0, narrow = 0;
    if (i < all_nodes) {
      const int columns = f[2] * G, blocks = columns > 0 ? seen_blocks(c, f[3], f[4], f[5], f[6]) : 0;
      if (columns > kFewColumns) { mine = (blocks + 3) / 4; wide = (columns + kTrunkTile - 1) / kTrunkTile; }
      else narrow = blocks;
    }
    long sum;
    scan((long)mine * wide << 20 | (mine ? wide : 0), sum);
    if (i < all_nodes) {
      f[9] = mine;
      f[11] = narrow;
    }
    tiles += sum >> 20;
    columns_of_tiles += sum & 1048575;
    // (columns of the plan follow)
    list(narrow > 0, narrow, f[0], f[1], f[2], f[3], f[4], f[5], f[6], i, i < nodes);
  }
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
  __syncthreads();
  // columns: as many times a node's as workgroups may have a piece of it
  // How many workgroups for the entries of few, which also has those of the nodes: the longer of the two kinds of work is to be short.  In units of
  // 1/8 us, measured: a short entry by a head 15 us for each of the waves that has one, a step of a long one 0.6, a piece 11 and 2.2 a tile.
  const unsigned all_tiles = (unsigned)(tiles * c.heads), begun = (unsigned)(tiles + columns_of_tiles * kBegin) * c.heads;     // (begun: in units, a chunk a column)
  Trunk trunk{0, 8, 1};
  int few_workers = 0;
  if (few_steps || short_ones) {
    unsigned best = ~0u;
#pragma unroll 1
    for (int s = 5; 1 << s <= kSharedWorkers; ++s) {
      const int f = 1 << s;
      if (f == kSharedWorkers && tiles) break;
      const unsigned waves = 4 * f, a = (((unsigned)short_ones * c.heads + waves - 1) >> (s + 2)) * 120 + (unsigned)min(few_steps * c.heads >> s, 1L << 26) * 5;
      const unsigned b = tiles ? 88 + min(begun / max(kSharedWorkers - f, 8) + 1, 1u << 26) * 18 : 0, time = max(a, b);
      if (time < best) { best = time; few_workers = f; }
    }
  }
  trunk.workers = max(min(kSharedWorkers - few_workers, (int)min(all_tiles / 2, 4096u)) & ~7, 8);
  // Whole chunks: their length.
  int length = max((int)((all_tiles + trunk.workers - 1) / trunk.workers), 2), chunks_of_head = 0;
  bool whole = false;
  // a thread's first node stays in registers
  const int columns0 = tid < all_nodes ? plan.node[(long)tid * kNodeInts + 2] * G : 0, tiles0 = tid < all_nodes ? plan.node[(long)tid * kNodeInts + 9] : 0;
#pragma unroll 1
  for (int turn = 0; turn < 5 && tiles; ++turn) {
    int x = 0;
    for (int i = tid; i < all_nodes; i += kThreads) {
      const int *f = plan.node + (long)i * kNodeInts, columns = i == tid ? columns0 : f[2] * G, n = i == tid ? tiles0 : f[9];
      x += min((columns + kTrunkTile - 1) / kTrunkTile * ((n + length - 1) / length), 1 << 20);
    }
    scan(x, chunks_of_head);
    const long all = (long)chunks_of_head * c.heads;
    whole = all <= trunk.workers;
    if (whole) break;
    length = max(length + 1, (int)min((float)length * (float)all / (float)trunk.workers, (float)kEndless));
  }
  const int part = (int)(begun / trunk.workers);
  whole = whole && length < part + kBegin;
  trunk.chunk = whole ? length : Trunk::chunk_of(all_tiles, part, trunk.workers);
  if (whole) trunk.workers = chunks_of_head * c.heads;
  long columns = 0;
  int units = 0;                                     // or chunks, where workers have whole ones
  for (int base = 0; base < all_nodes; base += kThreads) {
    const int i = base + tid;
    int *f = plan.node + (long)min(i, all_nodes - 1) * kNodeInts;
    const int pieces = i >= all_nodes ? 0 : f[9] ? (whole ? 1 : 2) * trunk.chunks(f[9]) : f[11] > 0;
    const int mine = i >= all_nodes ? 0 : whole ? (f[9] ? (f[2] * G + kTrunkTile - 1) / kTrunkTile * pieces : 0) : trunk.units(f[9], f[2] * G);
    int upto;
    const int at_unit = units + scan(mine, upto);
    units += upto;
    int all;
    const long at = columns + scan(i < all_nodes ? pieces * f[2] * G : 0, all);
    const bool fits = at + (long)pieces * f[2] * G <= most_columns;    // (it does: plan_columns)
    if (i < all_nodes) {
      f[8] = unit[i] = at_unit;
      f[10] = fits ? (int)at : -1;
      f[11] = fits ? pieces : 0;
    }
    columns += all;
  }
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
  __syncthreads();
  // the columns of the entries of few, which have their node's number there
  for (int i = tid; i < few + short_ones; i += kThreads) {
    int *f = plan.few + (long)(i < few ? i : 3 * N - 1 - (i - few)) * kNodeInts + 8;
    if (*f >= 0) *f = plan.node[(long)*f * kNodeInts + 10];
  }
  // the workers' first pieces: the last node that begins no later
  trunk.total = (unsigned)units * c.heads;
  if (tiles)
    for (int w = tid; w < trunk.workers; w += kThreads) {
      const unsigned at = whole ? w : trunk.first(w), end = whole ? w + 1 : trunk.first(w + 1);
      const unsigned head = at / (unsigned)units;
      const int in_head = (int)(at - head * units);
      int low = 0;
      for (int high = all_nodes; high - low > 1;) {
        const int mid = (low + high) / 2;
        if (unit[mid] <= in_head) low = mid;
        else high = mid;
      }
      const int4 *f = reinterpret_cast<const int4 *>(plan.node + (long)low * kNodeInts);
      int4 *to = reinterpret_cast<int4 *>(plan.first + w * kFirstInts);
      const int4 x = f[0], y = f[1], z = f[2];
      const int in_node = in_head - z.x;
      to[0] = x; to[1] = y; to[2] = z;
      if (whole) {
        const int n = max(z.y, 1), tall = max((x.z * G + kTrunkTile - 1) / kTrunkTile, 1), each = (n + trunk.chunks(n) - 1) / trunk.chunks(n), k = in_node / tall;
        to[3] = make_int4((int)head, (in_node - k * tall) * kTrunkTile, k * each, min(n, (k + 1) * each));
        to[4] = make_int4(k, 0, 1, 0);
      } else {
        const Trunk::Dealt p = trunk.dealt(z.y, x.z * G, in_node, (int)(end - at));
        to[3] = make_int4((int)head, p.column, p.from, p.to);
        to[4] = make_int4(p.piece, p.only, p.units, 0);
      }
    }
  // what a slot's rows are joined from
  for (int k = tid; k < n; k += kThreads) {
    int4 *chain = reinterpret_cast<int4 *>(plan.chain) + (kTrunkDepth + 1L) * r.slot[k];
    const int columns = r.rows[k] * G;
    int i = r.same[k + 1 < n && r.a[k + 1] > r.a[k] ? k + 1 : k];
    if (i >= 0 && r.index[i] < 0) i = r.near[i];
    if (none) i = -1;
    if (i < 0 && (columns <= kFewColumns || columns >= kTrunkTile)) continue;
    int node = chain[0].w;
    for (int d = 0; d <= kTrunkDepth; ++d) {
      int4 x = make_int4(0, 0, 0, 0);
      if (node >= 0) {
        const int *f = plan.node + (long)node * kNodeInts;
        x = make_int4(f[10] + (r.row[k] - f[1]) * G, f[2] * G, f[11], 0);
        node = f[7];
      }
      chain[d] = x;
    }
  }
  if (tid == 0) {
    plan.head[kPlanNodes] = all_nodes;
    plan.head[kPlanUnits] = units;
    plan.head[kPlanFew] = few;
    plan.head[kPlanShort] = short_ones;
    plan.head[kPlanRows] = rows;
    plan.head[kPlanWorkers] = trunk.workers | few_workers << kPlanFewShift;
    plan.head[kPlanChunk] = trunk.chunk;
    plan.head[kPlanShape] = 2 * N | whole;
  }
}

}  // namespace

hipError_t launch_pages_share(const Pages &c, const int *start, int rows, const Plan &plan, long columns, long least_bytes, hipStream_t st)
{
  agree_kernel<<<(c.slots + 3) / 4, 256, 0, st>>>(c, start, rows, plan);
  const size_t lds = (size_t)c.slots * kRunBytes;
  if (lds > 60000) {
    const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void *>(plan_kernel), hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds);
    if (e != hipSuccess) return e;
  }
  plan_kernel<<<1, kThreads, lds, st>>>(c, start, rows, plan, columns, least_bytes);
  return hipGetLastError();
}

}  // namespace lessdec
