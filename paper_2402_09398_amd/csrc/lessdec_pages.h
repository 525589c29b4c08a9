// Paged cache in 8 bits: what its kernels share, and the launch interfaces between the C ABI (lessdec_pages_api.hip) and the
// kernel files.
#pragma once

#include <hip/hip_bfloat16.h>

#include "lessdec_common.h"
#include "lessdec.h"

namespace lessdec {

constexpr int kBlock = LESSDEC_PAGE_BLOCK;           // tokens that share an exponent

// A layer of the cache, as a kernel argument.  k, v, exps point at the layer.
struct Pages {
  int slots, pages, page_tokens, table_len, heads, head_dim, q_per_kv, sinks, window;
  unsigned inverse;                                  // 2^32 / (blocks of a page), rounded up; 0: a page is a block
  float scale_log2;                                  // of the scores, times log2 e
  unsigned char *k, *v;
  int8_t *exps;
  int *table, *length, *refs;
};

__device__ inline int page_blocks(const Pages &c) { return c.page_tokens / kBlock; }
__device__ inline int slot_length(const Pages &c, int s)
{
  const int n = c.length[s], most = c.table_len * c.page_tokens;
  return n < 0 ? 0 : n < most ? n : most;
}
// [first, first + count): a slot's rows
struct Rows { int first, count; };
__device__ inline Rows slot_rows(const int *start, int s, int rows)
{
  const int a = start[s], b = start[s + 1];
  Rows r;
  r.first = a < 0 ? 0 : a < rows ? a : rows;
  const int end = b < 0 ? 0 : b < rows ? b : rows;
  r.count = end > r.first ? end - r.first : 0;
  return r;
}
// table entry of a slot's block: block / page_blocks, exact for the 2^26 blocks that a slot can have
__device__ inline int entry_of(const Pages &c, int block) { return c.inverse ? (int)__umulhi((unsigned)block, c.inverse) : block; }
// index of a block in its layer (a layer has less than 2^31), or -1 where page is none of the pool's
__device__ inline int block_in(const Pages &c, int page, int head, int block)
{
  const int per = page_blocks(c);
  return (unsigned)page < (unsigned)c.pages ? (page * c.heads + head) * per + (block - entry_of(c, block) * per) : -1;
}
__device__ inline int block_index(const Pages &c, int s, int head, int block)
{
  return block_in(c, c.table[(size_t)s * c.table_len + entry_of(c, block)], head, block);
}

// The last i in [0, n) whose base(i) is at most x, likewise, for any n.
template <typename F>
__device__ inline int last_at(int n, long x, F base)
{
  const int lane = threadIdx.x & 63;
  int from = 0;
  int step = 1;
  while ((long)step * kWave < n) step *= kWave;
  for (;; step /= kWave) {
    const long i = from + (long)lane * step;
    const int there = __popcll(__ballot(i < n && base((int)(i < n ? i : 0)) <= x));
    from += (there > 0 ? there - 1 : 0) * step;
    if (step == 1) return from;
  }
}

// The last slot s in [0, slots) whose base(s) is at most x, for a base that does not fall with s: 64 lanes ask at a time, so that
// up to 4096 slots cost two rounds of loads.  All lanes of a wave call it with the same x.
template <typename F>
__device__ inline int last_slot_at(int slots, long x, F base)
{
  const int lane = threadIdx.x & 63, step = (slots + 63) / 64;
  int s = lane * step;
  int n = __popcll(__ballot(s < slots && base(s < slots ? s : 0) <= x));
  const int from = (n > 0 ? n - 1 : 0) * step;
  if (step == 1) return from;
  s = from + lane;
  n = __popcll(__ballot(lane < step && s < slots && base(s < slots ? s : 0) <= x));
  return from + (n > 0 ? n - 1 : 0);
}

// LDS traffic between the lanes of one wave: the accesses behind it see those before it
__device__ inline void wave_lds_sync()
{
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront", "local");
  __builtin_amdgcn_wave_barrier();
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront", "local");
}

// 2^e for -126 <= e <= 127
__device__ inline float pow2(int e) { return __uint_as_float((unsigned)(e + 127) << 23); }

// launches (host)
hipError_t launch_pages_reset(const Pages &c, hipStream_t st);
hipError_t launch_pages_reserve(const Pages &c, const int *n_new, int *granted, int *plan, int *free_list, hipStream_t st);
hipError_t launch_pages_select(const Pages &c, const int *from, hipStream_t st);
hipError_t launch_pages_compact(const Pages &c, int *plan, int *moved, hipStream_t st);
hipError_t launch_pages_copy(const Pages &c, int layers, const int *plan, int max_pairs, hipStream_t st);

struct AppendArgs {
  const void *k, *v;
  long stride;
  const int *start;
  int rows;
};
hipError_t launch_pages_append(const Pages &c, int dtype, const AppendArgs &a, hipStream_t st);

struct ReadArgs {
  const int *slots;
  int n, first, count;
  void *k, *v;
};
hipError_t launch_pages_read(const Pages &c, int dtype, const ReadArgs &a, hipStream_t st);

struct AttendArgs {
  const void *q;
  long stride;
  void *out;
  float *lse;
  const int *start;
  int rows, max_new;
  int *counters;                                     // [3 kPagesWorkers], 0 before and after a call
  float *parts;
};
constexpr int kPagesWorkers = 768;                   // workgroups of the kernel of few rows: three to a compute unit
hipError_t launch_pages_attend(const Pages &c, int dtype, const AttendArgs &a, hipStream_t st);

// What neighbouring slots have in common, for a call's rows (lessdec_pages_share.hip), in the caller's memory.
//  head  [8]: nodes, units of a head, entries of few, rows that it was made for, workers of the nodes and (kPlanFewShift) of the entries of few, tiles of a
//        chunk, short entries, slots and (the last bit) whether workers have whole chunks
//  node  [3 slots][kNodeInts]: slot whose table row is read, first row, rows, least and largest position of them, blocks [first, last), node before it
//        (-1: none), its first unit (or chunk, where workers have whole ones) among a head's, tiles (of 64 tokens; 0: few columns, or nothing of its own), first column (-1: none), shares of a column.
//        First the nodes of several slots, then a slot's own part, which reaches to kEndless.
//  few   [3 slots][kNodeInts]: of nodes of up to kFewColumns columns, and of slots of so many that share nothing: steps, slot whose table row is
//        read, first row, rows, least and largest position, blocks [first, last), first column of the plan (-1: the rows are stored), rows of several slots.
//        From the front, in steps of kFewBlocks blocks, for a workgroup each; from the back, in steps of two, the short ones, for a wave each
//  chain [slots][kTrunkDepth + 1][4]: of its own node and those around it, the first column of the plan that is its first row's, columns from a share to
//        the next, shares (0: no more nodes; with -1 in the first the slot is not in any, and an entry of few or of 128 columns and more)
//  first [kSharedWorkers][kFirstInts]: a worker's first piece: its node as above, then head, first column, tiles [from, to), piece, whether it is a whole chunk, units
//  pos   [rows]: positions of the rows
//  apart [slots]: scratch
// A (head, column of the plan) has a sum of D floats, a maximum and a total in the workspace.
constexpr int kPlanNodes = 0, kPlanUnits = 1, kPlanFew = 2, kPlanRows = 3, kPlanWorkers = 4, kPlanChunk = 5, kPlanShort = 6, kPlanShape = 7, kPlanHead = 8, kNodeInts = 12, kFirstInts = 20, kEndless = 1 << 30;
constexpr int kPlanFewShift = 16;
constexpr int kFewColumns = 16, kFewBlocks = 8;      // columns of the kernel of few rows, and its blocks a step
// Up to how many blocks an entry of few is a wave's by itself.  64 beams with up to 300 tokens of their own, 8 heads: 34 us a layer, 60 with 8 blocks (a
// workgroup has an entry's beginning and end to itself), 33 with 128; but 8 slots with 100, 32 heads: 26, 26 and 50, few waves with long lists.
constexpr int kShortBlocks = 32;
// Nodes around a slot (instructions, a prompt, its samples' fork).  Samples of 16 prompts behind the same instructions: 39 us a layer with 3 and with 2,
// 89 with 1.
constexpr int kTrunkDepth = 3;
constexpr int kTrunkTile = 128;                      // columns of a tile
constexpr int kSharedWorkers = 512;                  // workgroups of the launch, two to a compute unit, multiples of 8 of them for either kind of work
struct Plan {
  int *head, *node, *chain, *few, *first, *apart, *pos;
};
// The nodes' tiles as the workers get them, in one of two ways.  Whole chunks: the tiles of a node's 128 columns by one head are cut into chunks of
// the same length, the least with which there are no more chunks than workers, and each worker has one.  Or, where that would leave workers idle for
// longer than a second beginning and end take: the chunks of all heads and nodes, one behind the other, are dealt out evenly, in units of a tile's
// time.  A chunk begins with kBegin units that stand for what a piece costs beside its tiles, so that a worker of many short parts has no more to do
// than one of a long one; worker w has [first(w), first(w + 1)).  32 questions of 24 tokens behind 16384, 32 heads: 393 us dealt
// by tiles alone, 277 so, 285 and 290 with 5 and 8 units; behind 8192: 277, 160, 167 and 177.
// Within a node and head the order is by chunks of tokens, in a chunk by tiles of 128 columns, so that neighbouring workers read the same tokens at the
// same time.  A chunk has no more tiles than any worker has units: what it has of 128 columns is cut into two pieces at most.
constexpr int kBegin = 3;
struct Trunk {
  unsigned total;                                    // units of all heads, less than 2^31
  int workers, chunk;                                // tiles of a chunk
  __host__ __device__ inline unsigned first(unsigned w) const
  {
    const unsigned each = total / workers, more = total - each * workers;
    return w * each + (w < more ? w : more);
  }
  // where workers have `part` units at least: those less what a piece costs, but so many that all tiles make no more than two chunks a worker, which there
  // is room for
  __host__ __device__ static inline int chunk_of(unsigned tiles, int part, int workers)
  {
    const int least = (int)((tiles + 2u * workers - 1) / (2u * workers)), most = part - kBegin;
    return most > least ? most : least > 1 ? least : 1;
  }
  __host__ __device__ inline int chunks(int n) const { return (n + chunk - 1) / chunk; }        // of n tiles of 128 columns
  __host__ __device__ inline int units(int n, int columns) const // of a node by a head
  {
    return n ? (columns + kTrunkTile - 1) / kTrunkTile * (n + kBegin * chunks(n)) : 0;
  }
  // The piece of a node of n tiles at unit `at` of the node's, up to `left` units of it: 128 columns from `column` on, tiles [from, to), which may be none.
  struct Dealt { int column, from, to, piece, only, units; };
  __device__ inline Dealt dealt(int n, int columns, int at, int left) const
  {
    const int tall = (columns + kTrunkTile - 1) / kTrunkTile, k = at / max((chunk + kBegin) * tall, 1), in_chunk = at - k * (chunk + kBegin) * tall;
    const int len = max(min(chunk, n - k * chunk), 0), column = in_chunk / (len + kBegin), done = in_chunk - column * (len + kBegin);
    Dealt x;
    x.units = min(len + kBegin - done, left);
    x.column = column * kTrunkTile;
    const int from = max(done - kBegin, 0), to = max(done + x.units - kBegin, 0);
    x.from = k * chunk + from;
    x.to = k * chunk + to;
    x.piece = 2 * k + (from > 0);
    x.only = from == 0 && to == len;
    return x;
  }
};
// Slots of up to 127 query columns share.  A row is in kTrunkDepth nodes and one of its own at most, each of which has room for two pieces, and
// for as many more as chunks are (n tiles have n / chunk + 1 at most, and all tiles make two chunks a worker at most).
inline long plan_columns(int slots, int heads, int q_per_kv, long rows)
{
  const long n = rows * q_per_kv, most = (long)slots * kTrunkTile;
  return 2 * (kTrunkDepth + 1) * (n < most ? n : most) + 4L * kTrunkTile * (kSharedWorkers / heads + 1);
}
// units of all heads and nodes, at most
inline double plan_units(int slots, int heads, int q_per_kv, long rows, long tokens)
{
  const double n = (double)rows * q_per_kv, most = (double)slots * kTrunkTile;
  return heads * ((kTrunkDepth + 1) * (n < most ? n : most) / kTrunkTile + 2.0 * slots) * (tokens / 64 + 1 + kBegin) + 2.0 * kBegin * kSharedWorkers;
}
inline long plan_ints(int slots, long rows) { return kPlanHead + kSharedWorkers * kFirstInts + (long)slots * (6 * kNodeInts + 4 * (kTrunkDepth + 1) + 1) + rows; }
inline Plan plan_at(int *p, int slots)
{
  Plan x;
  x.head = p;
  x.node = x.head + kPlanHead;                       // (16-byte aligned)
  x.chain = x.node + 3L * slots * kNodeInts;
  x.few = x.chain + 4L * (kTrunkDepth + 1) * slots;
  x.first = x.few + 3L * slots * kNodeInts;
  x.apart = x.first + kSharedWorkers * kFirstInts;
  x.pos = x.apart + slots;
  return x;
}
struct SharedArgs : AttendArgs {
  Plan plan;
  float *trunk;                                      // [heads][columns][D] sums, [heads][columns] maxima, [heads][columns] totals
  long columns;
};
hipError_t launch_pages_attend_shared(const Pages &c, int dtype, const SharedArgs &a, hipStream_t st);
hipError_t launch_pages_share(const Pages &c, const int *start, int rows, const Plan &plan, long columns, long least_bytes, hipStream_t st);

// floats of AttendArgs::parts for up to `rows` rows
size_t pages_attend_floats(int slots, int heads, int q_per_kv, int head_dim, long tokens, int rows);

}  // namespace lessdec
