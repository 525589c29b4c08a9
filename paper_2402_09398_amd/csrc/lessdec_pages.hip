// Bookkeeping of the paged cache: making room, forking, freeing, compacting, and the copies that these ask for.
//
// Tables, lengths and reference counts live on the device, so that a generation step can be captured in a graph; everything here
// but the copy touches a few bytes a slot or page and is bound by the latency of its dependent loads.  What has an order
// (which free page goes to which slot) is settled by prefix sums over slots and pages in one workgroup, never by the order in
// which atomics arrive: the same state gives the same pages every time.  Counts change by integer atomics, which commute.
// Measured: 64 beams of 2050 tokens on pages of 16: select 4.1 us, reserve 8.4, their 64 copies in four layers 3.8; compacting a pool of 5000 pages:
// 11.6 us to find what moves, 4.5 to rename it, 56 for the copies (305 MB, 5.5 TB/s).
#include "lessdec_pages.h"

namespace lessdec {
namespace {

constexpr int kThreads = 1024, kWaves = kThreads / kWave;
constexpr int kSpan = kWave * 16;                    // pages that a wave looks at in one turn: sixteen ballots
constexpr int kMaxSlots = LESSDEC_MAX_SLOTS, kTurns = kMaxSlots / kThreads;

// refs are changed by atomics, which work in the L2: read there, past this compute unit's own cache
__device__ inline int count_of(const int *refs, int p)
{
  return __hip_atomic_load(refs + p, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}

// The counts of the wave's next kSpan pages from `first` on, sixteen a lane.  Every load is made (of the last page behind the end): sixteen
// conditional ones wait for one another (a pool of 17000 pages: the search took 8 us, now 2.2).
__device__ inline void load_counts(const Pages &c, int first, int (&count)[16])
{
#pragma unroll
  for (int k = 0; k < 16; ++k) count[k] = count_of(c.refs, min(first + k * kWave + (int)(threadIdx.x & 63), c.pages - 1));
}

// sum over the threads before this one; total: over all of them
template <typename T>
__device__ inline T scan_exclusive(T x, T *shared, T &total)
{
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  T upto = x;
  for (int d = 1; d < kWave; d <<= 1) {
    const T y = __shfl_up(upto, d, kWave);
    if (lane >= d) upto += y;
  }
  __syncthreads();
  if (lane == 63) shared[wave] = upto;
  __syncthreads();
  T before = 0;
  total = 0;
  for (int w = 0; w < kWaves; ++w) {
    if (w == wave) before = total;
    total += shared[w];
  }
  return before + upto - x;
}

__global__ void reset_kernel(Pages c)
{
  const long n = (long)c.slots * c.table_len, at = (long)blockIdx.x * blockDim.x + threadIdx.x;
  const long stride = (long)gridDim.x * blockDim.x;
  for (long i = at; i < n; i += stride) c.table[i] = -1;
  for (long i = at; i < c.pages; i += stride) c.refs[i] = 0;
  for (long i = at; i < c.slots; i += stride) c.length[i] = 0;
}

// One workgroup.  free_list: [pages], the free pages from the kMaxSlots-th on (those before stay in the LDS).
__global__ __launch_bounds__(kThreads) void reserve_kernel(Pages c, const int *n_new, int *granted, int *plan, int *free_list)
{
  __shared__ __align__(16) int open_page[kMaxSlots]; // the page that the slot goes on filling, or -1; later the first of the free pages
  __shared__ int upto[kMaxSlots];                    // pages needed by the slots up to this one
  __shared__ int want[kMaxSlots];                    // pages needed by this one
  __shared__ long sums[kWaves];
  __shared__ int page_sums[kWaves], pairs;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, pt = c.page_tokens;
  const long room = (long)c.table_len * pt;
  if (tid == 0) pairs = 0;

  // pages behind the window: from the newest down to the last that was let go, 64 at a time
  if (c.window > 0) {
    const int a = (int)(((long)c.sinks + pt - 1) / pt);
    for (int s = wave; s < c.slots; s += kWaves) {
      const int n = n_new[s], len = slot_length(c, s);
      if (n <= 0 || len + (long)n > room || len < c.window) continue;
      for (int j = (len - c.window + 1) / pt - 1; j >= a; j -= kWave) {
        const int i = j - lane;
        int *at = c.table + (size_t)s * c.table_len + i;
        const int p = i >= a ? *at : -1;
        if (p >= 0) {
          if (p < c.pages) atomicSub(c.refs + p, 1);
          *at = -1;
        }
        if (__ballot(p < 0)) break;
      }
    }
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
    __syncthreads();
  }
  int counts[16];                                    // of the pages looked at first: on their way meanwhile
  load_counts(c, wave * kSpan, counts);

  // what each slot needs; a thread has the slots tid, tid + kThreads, ..
  int wanted[kTurns], length[kTurns], old_page[kTurns], pair[kTurns];
#pragma unroll
  for (int t = 0; t < kTurns; ++t) {
    const int s = tid + t * kThreads;
    old_page[t] = pair[t] = -1;
    wanted[t] = length[t] = 0;
    if (s >= c.slots) continue;
    const int n = n_new[s], len = slot_length(c, s);
    wanted[t] = n > 0 && len + (long)n <= room ? n : 0;
    length[t] = len;
    if (wanted[t] && len % pt) {
      const int p = c.table[(size_t)s * c.table_len + len / pt];
      old_page[t] = (unsigned)p < (unsigned)c.pages ? p : -1;
    }
    open_page[s] = old_page[t];
  }
  __syncthreads();
  long before_turn = 0;
#pragma unroll
  for (int t = 0; t < kTurns; ++t) {
    if (t * kThreads >= c.slots) break;
    const int s = tid + t * kThreads;
    int need = 0, copies = 0;
    if (wanted[t]) {
      const int n = wanted[t], len = length[t];
      if (len % pt) {
        const int p = old_page[t], sharers = p >= 0 ? count_of(c.refs, p) : 0;
        if (sharers > 1) {
          int before = 0;                            // slots before this one that write to the same page
          for (int i = 0; i < s; i += 16) {
            int4 o[4];
#pragma unroll
            for (int q = 0; q < 4; ++q) o[q] = reinterpret_cast<const int4 *>(open_page + i)[q];
#pragma unroll
            for (int q = 0; q < 4; ++q) {
              const int at = i + 4 * q;
              before += (at < s && o[q].x == p) + (at + 1 < s && o[q].y == p) + (at + 2 < s && o[q].z == p) + (at + 3 < s && o[q].w == p);
            }
          }
          copies = sharers - before > 1;
        }
      }
      // (`copies`: a new page in the place of the partly filled one.  None where the table names none there: what an earlier
      // sequence left on it would be read as this one's older tokens.)
      need = (int)((len + (long)n + pt - 1) / pt) - (len + pt - 1) / pt + copies;
    }
    long all;                                        // both sums in one word: 2^12 slots of less than 2^27 pages each
    const long x = scan_exclusive<long>(need | (long)copies << 48, sums, all) + before_turn;
    before_turn += all;
    if (copies) pair[t] = (int)(x >> 48);
    if (s < c.slots) {
      const long u = (x & ((1L << 48) - 1)) + need;
      upto[s] = u < (1 << 30) ? (int)u : 1 << 30;
      want[s] = need;
    }
  }
  const int total = (int)min(before_turn & ((1L << 48) - 1), (long)c.pages);           // (more than there are do not come)

  // the first free pages, in order (the scan above has synchronised: no one looks for an open page any more)
  int *first_free = open_page, found = 0;
  for (int base = 0; base < c.pages && found < total; base += kWaves * kSpan) {
    int count = 0;
    const int first = base + wave * kSpan;
    if (base) load_counts(c, first, counts);
#pragma unroll
    for (int k = 0; k < 16; ++k) count += __popcll(__ballot(counts[k] == 0 && first + k * kWave + lane < c.pages));
    __syncthreads();
    if (lane == 0) page_sums[wave] = count;
    __syncthreads();
    int at = found;
    for (int w = 0; w < kWaves; ++w) {
      if (w < wave) at += page_sums[w];
      found += page_sums[w];
    }
    if (at < total)                                  // (most waves are past the last page that is wanted)
#pragma unroll
      for (int k = 0; k < 16; ++k) {
        const unsigned long long free_of = __ballot(counts[k] == 0 && first + k * kWave + lane < c.pages);
        const int mine = at + __popcll(free_of & ((1ull << lane) - 1));
        if ((free_of >> lane & 1) && mine < total) (mine < kMaxSlots ? first_free : free_list)[mine] = first + k * kWave + lane;
        at += __popcll(free_of);
      }
  }
  __syncthreads();                                   // the free pages and want, upto
  auto free_page = [&](int i) { return i < kMaxSlots ? first_free[i] : free_list[i]; };

  // tables: by the slot's thread where few pages are wanted, else by a wave
  auto take = [&](int s, int j, int need, int end) {
    const int p = free_page(upto[s] - need + j);
    c.table[(size_t)s * c.table_len + end - need + j] = p;
    c.refs[p] = 1;
  };
#pragma unroll
  for (int t = 0; t < kTurns; ++t) {
    const int s = tid + t * kThreads;
    if (s >= c.slots) continue;
    const int n = wanted[t], len = length[t], need = want[s];
    const bool fits = n && upto[s] <= found;
    if (granted) granted[s] = fits ? n : 0;
    if (!fits) {
      want[s] = 0;
      continue;
    }
    const int end = (int)((len + (long)n + pt - 1) / pt);
    if (need <= 4)
      for (int j = 0; j < need; ++j) take(s, j, need, end);
    if (pair[t] >= 0) {
      atomicSub(c.refs + old_page[t], 1);
      plan[1 + 2 * pair[t]] = old_page[t];
      plan[2 + 2 * pair[t]] = free_page(upto[s] - need);
      atomicMax(&pairs, pair[t] + 1);
    }
  }
  __syncthreads();
  for (int base = 0; base < c.slots; base += kThreads) {
    const int mine = base + lane * kWaves + wave;    // neighbours to different waves
    unsigned long long many = __ballot(mine < c.slots && want[mine < c.slots ? mine : 0] > 4);
    for (; many; many &= many - 1) {
      const int s = base + (__ffsll(many) - 1) * kWaves + wave, need = want[s];
      const int end = (int)((slot_length(c, s) + (long)n_new[s] + pt - 1) / pt);
      for (int j = lane; j < need; j += kWave) take(s, j, need, end);
    }
  }
  if (tid == 0) plan[0] = pairs;
  __syncthreads();                                   // lengths are read up to here
#pragma unroll
  for (int t = 0; t < kTurns; ++t) {
    const int s = tid + t * kThreads;
    if (wanted[t] && upto[s] <= found) c.length[s] = length[t] + wanted[t];
  }
}

// A workgroup has 1 << shift columns of the table, all slots of them, so that every old entry is read before one is written; the
// last workgroup has the lengths.  Loads are made four at a time, none of them conditional (64 slots of 133 entries: 4.2 us, 6.5 one by one).
__global__ __launch_bounds__(256) void select_kernel(Pages c, const int *from, int shift)
{
  extern __shared__ int shared[];
  const bool lengths = blockIdx.x == gridDim.x - 1;
  if (lengths) shift = 0;
  const int base = blockIdx.x << shift, mask = (1 << shift) - 1, last = c.table_len - 1, n = c.slots << shift;
  // more[f]: slots that get slot f's entries, less f itself if it loses them
  int *old = shared, *source = shared + n, *more = source + c.slots;
  for (int s = threadIdx.x; s < c.slots; s += 256) {
    const int f = from[s];
    source[s] = f < -1 || f >= c.slots ? s : f;
    more[s] = 0;
  }
  for (int i = threadIdx.x; i < n; i += 4 * 256) {
    int x[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const int e = min(i + k * 256, n - 1), s = e >> shift;
      x[k] = *(lengths ? c.length + s : c.table + (size_t)s * c.table_len + min(base + (e & mask), last));
    }
#pragma unroll
    for (int k = 0; k < 4; ++k)
      if (i + k * 256 < n) old[i + k * 256] = x[k];
  }
  __syncthreads();
  for (int s = threadIdx.x; s < c.slots; s += 256) {
    const int f = source[s];
    if (f == s) continue;
    atomicSub(more + s, 1);
    if (f >= 0) atomicAdd(more + f, 1);
  }
  __syncthreads();
  for (int i = threadIdx.x; i < n; i += 256) {
    const int s = i >> shift, j = base + (i & mask), f = source[s], was = old[i];
    if (!lengths && j > last) continue;
    if (!lengths && more[s] && (unsigned)was < (unsigned)c.pages) atomicAdd(c.refs + was, more[s]);
    if (f == s) continue;
    const int now = f < 0 ? (lengths ? 0 : -1) : old[(f << shift) + (i & mask)];
    if (lengths) c.length[s] = now;
    else c.table[(size_t)s * c.table_len + j] = now;
  }
}

// One workgroup.  moved[p], p >= pages in use: where page p goes (-1: nothing there); moved[0]: pages in use.
__global__ __launch_bounds__(kThreads) void compact_kernel(Pages c, int *plan, int *moved)
{
  __shared__ int sums[kWaves], sums2[kWaves];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  int mine = 0, count[16], used;
  for (int base = 0; base < c.pages; base += kWaves * kSpan) {
    const int first = base + wave * kSpan;
    load_counts(c, first, count);
#pragma unroll
    for (int k = 0; k < 16; ++k) mine += count[k] != 0 && first + k * kWave + lane < c.pages;
  }
  scan_exclusive<int>(mine, sums, used);
  int sources = 0, places = 0;
  for (int base = 0; base < c.pages; base += kWaves * kSpan) {
    unsigned long long in_use[16];
    int above = 0, below = 0;
    load_counts(c, base + wave * kSpan, count);
#pragma unroll
    for (int k = 0; k < 16; ++k) {
      const int p = base + wave * kSpan + k * kWave + lane;
      in_use[k] = __ballot(p < c.pages && count[k] != 0);
      const unsigned long long high = __ballot(p >= used), low = __ballot(p < used);
      above += __popcll(in_use[k] & high);
      below += __popcll(~in_use[k] & low);
    }
    __syncthreads();
    if (lane == 0) { sums[wave] = above; sums2[wave] = below; }
    __syncthreads();
    int a = sources, b = places;
    for (int w = 0; w < kWaves; ++w) {
      if (w < wave) { a += sums[w]; b += sums2[w]; }
      sources += sums[w];
      places += sums2[w];
    }
#pragma unroll
    for (int k = 0; k < 16; ++k) {
      const int p = base + wave * kSpan + k * kWave + lane;
      const unsigned long long from = in_use[k] & __ballot(p >= used), to = ~in_use[k] & __ballot(p < used);
      const unsigned long long below_me = (1ull << lane) - 1;
      if (from >> lane & 1) plan[1 + 2 * (a + __popcll(from & below_me))] = p;
      else if (p >= used && p < c.pages) moved[p] = -1;
      if (to >> lane & 1) plan[2 + 2 * (b + __popcll(to & below_me))] = p;
      a += __popcll(from);
      b += __popcll(to);
    }
  }
  __syncthreads();
  for (int i = tid; i < sources; i += kThreads) {
    const int p = plan[1 + 2 * i], to = plan[2 + 2 * i];
    c.refs[to] = c.refs[p];
    c.refs[p] = 0;
    moved[p] = to;
  }
  if (tid == 0) {
    plan[0] = sources;
    if (used > 0) moved[0] = used;
  }
}

__global__ void rename_kernel(Pages c, const int *moved)
{
  const long n = (long)c.slots * c.table_len;
  const int used = moved[0];
  for (long i = (long)blockIdx.x * blockDim.x + threadIdx.x; i < n; i += (long)gridDim.x * blockDim.x) {
    const int p = c.table[i];
    if ((unsigned)p < (unsigned)c.pages && p >= used) c.table[i] = moved[p];
  }
}

// 16 KiB of a page's keys and as much of its values to a workgroup at a time, 128 bytes a thread in flight; non-temporal, as nothing of it is
// read again soon.
constexpr int kPiece = 16384;
typedef unsigned u4 __attribute__((ext_vector_type(4)));
__global__ __launch_bounds__(256) void copy_kernel(Pages c, int layers, const int *plan, int max_pairs)
{
  const int n = plan[0] < max_pairs ? plan[0] : max_pairs;
  const long page = (long)c.heads * c.page_tokens * c.head_dim, scales = (long)c.heads * page_blocks(c);
  const int pieces = (int)((page + kPiece - 1) / kPiece);
  const long total = (long)(n > 0 ? n : 0) * layers * pieces;
  for (long item = blockIdx.x; item < total; item += gridDim.x) {
    const int piece = (int)(item % pieces), layer = (int)(item / pieces % layers), pair = (int)(item / pieces / layers);
    const int from = plan[1 + 2 * pair], to = plan[2 + 2 * pair];
    if ((unsigned)from >= (unsigned)c.pages || (unsigned)to >= (unsigned)c.pages) continue;
    const long a = ((long)layer * c.pages + from) * page, b = ((long)layer * c.pages + to) * page;
    u4 x[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const long at = (long)piece * kPiece + (i / 2) * 4096 + threadIdx.x * 16;
      if (at < page) x[i] = __builtin_nontemporal_load(reinterpret_cast<const u4 *>((i & 1 ? c.v : c.k) + a + at));
    }
#pragma unroll
    for (int i = 0; i < 8; ++i) {
      const long at = (long)piece * kPiece + (i / 2) * 4096 + threadIdx.x * 16;
      if (at < page) __builtin_nontemporal_store(x[i], reinterpret_cast<u4 *>((i & 1 ? c.v : c.k) + b + at));
    }
    if (piece == 0) {
      const unsigned short *e = reinterpret_cast<const unsigned short *>(c.exps) + ((long)layer * c.pages + from) * scales;
      unsigned short *f = reinterpret_cast<unsigned short *>(c.exps) + ((long)layer * c.pages + to) * scales;
      for (long i = threadIdx.x; i < scales; i += 256) f[i] = e[i];
    }
  }
}

int blocks_for(long n, int threads, int most)
{
  const long b = (n + threads - 1) / threads;
  return (int)(b < 1 ? 1 : b < most ? b : most);
}

}  // namespace

hipError_t launch_pages_reset(const Pages &c, hipStream_t st)
{
  const long table = (long)c.slots * c.table_len;
  reset_kernel<<<blocks_for(table > c.pages ? table : c.pages, 256, 2048), 256, 0, st>>>(c);
  return hipGetLastError();
}

hipError_t launch_pages_reserve(const Pages &c, const int *n_new, int *granted, int *plan, int *free_list, hipStream_t st)
{
  reserve_kernel<<<1, kThreads, 0, st>>>(c, n_new, granted, plan, free_list);
  return hipGetLastError();
}

hipError_t launch_pages_select(const Pages &c, const int *from, hipStream_t st)
{
  int shift = 4;                                     // 64 bytes of a row where 64 KiB of LDS hold them (of 4096 slots: two entries)
  while ((size_t)c.slots * ((1 << shift) + 2) * sizeof(int) > 65536) --shift;
  select_kernel<<<((c.table_len - 1) >> shift) + 2, 256, (size_t)c.slots * ((1 << shift) + 2) * sizeof(int), st>>>(c, from, shift);
  return hipGetLastError();
}

hipError_t launch_pages_compact(const Pages &c, int *plan, int *moved, hipStream_t st)
{
  compact_kernel<<<1, kThreads, 0, st>>>(c, plan, moved);
  rename_kernel<<<blocks_for((long)c.slots * c.table_len, 256, 2048), 256, 0, st>>>(c, moved);
  return hipGetLastError();
}

hipError_t launch_pages_copy(const Pages &c, int layers, const int *plan, int max_pairs, hipStream_t st)
{
  const long page = (long)c.heads * c.page_tokens * c.head_dim;
  const long items = (long)max_pairs * layers * ((page + kPiece - 1) / kPiece);
  copy_kernel<<<(unsigned)(items < 16384 ? items : 16384), 256, 0, st>>>(c, layers, plan, max_pairs);
  return hipGetLastError();
}

}  // namespace lessdec
