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
// floats of AttendArgs::parts for up to `rows` rows
size_t pages_attend_floats(int slots, int heads, int q_per_kv, int head_dim, long tokens, int rows);

}  // namespace lessdec
