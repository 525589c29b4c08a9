// Paged cache: attention of the slots' last tokens over their cached ones.
//
// A row's output is sum_j 2^{t_j} c_j / sum_j 2^{t_j - e_j} with t_j = log2(e) scale 2^{k_j} (q . kc_j) + e_j, where kc_j, c_j are the
// e4m3 codes of token j's key and value and k_j, e_j their blocks' exponents.  With the values' exponents in t, the product with the
// values takes bare codes, which fp16 holds exactly, and weights 2^{t_j - M} <= 1 relative to the largest contribution so far (not
// the largest score), so that fp16 holds the weights for any exponents: |e_j| <= 40 also keeps both sums within fp32.
//
// One pass over the tokens with the running maximum M and both sums (fp32).  M follows the maximum only where a weight would pass
// 2^kSlack (a wave asks once per tile); until then the weights' range in fp16 above 1 takes it up and nothing is rescaled.
//
// M is held in two parts, the score S and the value exponent E of the token that M was taken from.  Far from 0 an fp32 holds neither the exact
// product behind a score nor a score and an exponent in one, so there a weight is 2^((s_j - S) + (e_j - E)), with s_j rounded as S was: the largest
// token's weight is 2^kBase, and tokens of one score have one weight, wherever the scores lie.  Up to |S| = kNear one fma in
// place of the three operations is off by 2^-13 at most, less than the weights' rounding to fp16.  Sums that leave a wave's registers are taken times 2^E, so
// that S alone goes with them.
//
// Both kernels form the scores transposed, S^T = K Q^T, with tokens along the rows of a matrix tile: a lane's accumulator
// registers are then tokens of one query column, and just those tokens are what the lane has to bring to the second product, O^T = V^T P^T,
// so the weights never leave their registers.  They are rounded to fp16 for it, the sum's are not: fp16 outputs are off by 2.6e-4 of their size in place of the
// 2.1e-4 of fp32 weights and the output's own rounding, bfloat16 ones by 1.7e-3 either way (the cases of perf/operators.py; those of perf/more_operators.py,
// where slots share pages: 2.3e-4 to 2.9e-4, 1.7e-3).  A query column is a (row, query head of the group) pair: the heads of a group share the
// cached keys and values that a tile has loaded.
#include <type_traits>

#include "lessdec_pages.h"

namespace lessdec {
namespace {

typedef _Float16 half2v __attribute__((ext_vector_type(2)));
typedef _Float16 half8 __attribute__((ext_vector_type(8)));
typedef __bf16 bf2v __attribute__((ext_vector_type(2)));
typedef __bf16 bf8 __attribute__((ext_vector_type(8)));
typedef float f4 __attribute__((ext_vector_type(4)));
typedef float f16v __attribute__((ext_vector_type(16)));
typedef unsigned u4 __attribute__((ext_vector_type(4)));

constexpr float kLowest = -3.402823466e38f;
constexpr float kSlack = 8.f, kBase = 6.f;           // weights reach 2^(kBase + kSlack) = 2^14 (fp16: below 2^16), normal down to 2^-14
constexpr float kMost = 32768.f;                     // of a sum of weights: no one is more
constexpr float kNear = 1024.f;                      // scores (base 2) for which fp32 holds a score and a value's exponent in one
constexpr float kFirstE = 40.f - kBase;              // of M before its first token: no exponent is larger

// A lane's 16 bytes at a scalar address.  The asm keeps the address from being added to the lane's offset in vector registers, which loads in
// flight would then be waited for; the pointer says that it is global memory, which the compiler no longer sees.
typedef const __attribute__((address_space(1))) unsigned char *Bytes;
typedef const __attribute__((address_space(1))) u4 *Pieces;
__device__ inline Bytes scalar_bytes(const unsigned char *base, long offset)
{
  Bytes p = (Bytes)base + offset;
  asm("" : "+s"(p));
  return p;
}

template <bool BF16> struct Operand;
template <> struct Operand<false> {
  typedef half8 Vec;
  __device__ static inline unsigned pair(unsigned w, bool high)
  {
    const half2v x = high ? __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w, 1.f, true) : __builtin_amdgcn_cvt_scalef32_pk_f16_fp8(w, 1.f, false);
    return __builtin_bit_cast(unsigned, x);
  }
  __device__ static inline f4 mma16(u4 a, u4 b, f4 c)
  {
    return __builtin_amdgcn_mfma_f32_16x16x32_f16(__builtin_bit_cast(half8, a), __builtin_bit_cast(half8, b), c, 0, 0, 0);
  }
  __device__ static inline f16v mma32(u4 a, u4 b, f16v c)
  {
    return __builtin_amdgcn_mfma_f32_32x32x16_f16(__builtin_bit_cast(half8, a), __builtin_bit_cast(half8, b), c, 0, 0, 0);
  }
  __device__ static inline unsigned short store(float x) { return __half_as_ushort(__float2half_rn(x)); }
};
template <> struct Operand<true> {
  typedef bf8 Vec;
  __device__ static inline unsigned pair(unsigned w, bool high)
  {
    const bf2v x = high ? __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, 1.f, true) : __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, 1.f, false);
    return __builtin_bit_cast(unsigned, x);
  }
  __device__ static inline f4 mma16(u4 a, u4 b, f4 c)
  {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf8, a), __builtin_bit_cast(bf8, b), c, 0, 0, 0);
  }
  __device__ static inline f16v mma32(u4 a, u4 b, f16v c)
  {
    return __builtin_amdgcn_mfma_f32_32x32x16_bf16(__builtin_bit_cast(bf8, a), __builtin_bit_cast(bf8, b), c, 0, 0, 0);
  }
  __device__ static inline unsigned short store(float x) { return __builtin_bit_cast(unsigned short, (__bf16)x); }
};
// eight codes as an operand
template <bool BF16> __device__ inline u4 widen(unsigned a, unsigned b)
{
  return u4{Operand<BF16>::pair(a, false), Operand<BF16>::pair(a, true), Operand<BF16>::pair(b, false), Operand<BF16>::pair(b, true)};
}
__device__ inline unsigned half_pair(float a, float b)
{
  return __builtin_bit_cast(unsigned, half2v{(_Float16)a, (_Float16)b});
}
__device__ inline unsigned code_nans(unsigned w)     // 0xff where one of four codes is a NaN
{
  return ((((w & 0x7f7f7f7fu) + 0x01010101u) & 0x80808080u) >> 7) * 255u;
}
// x / l as x * r, 0 for a row that sees nothing (whose x is NaN if values that it sees with weight 0 are)
__device__ inline float share_of(float x, float l, float r) { return l == 0.f ? 0.f : x * r; }
__device__ inline float exp2_fast(float x) { return __builtin_amdgcn_exp2f(x); }
__device__ inline float product(float a, float b)   // rounded by itself, not within an fma
{
#pragma clang fp contract(off)
  return a * b;
}

// M: the score and the value exponent, less kBase, of the token with the largest t so far.
struct Top {
  float s, e;
  __device__ inline float above(float score, float exponent) const { return (score - s) + (exponent - e); }
  __device__ inline void raise(float score, float exponent)
  {
    const bool more = above(score, exponent) > 0;
    s = more ? score : s;
    e = more ? exponent : e;
  }
  // the larger of two lanes' that lie Distance apart, in both; the swap has the lower lane's in one result and the upper one's in the other
  template <int Distance> __device__ inline void raise_over()
  {
    auto swapped = [](float x) {
      const unsigned bits = __float_as_uint(x);
      return Distance == 32 ? __builtin_amdgcn_permlane32_swap(bits, bits, false, false) : __builtin_amdgcn_permlane16_swap(bits, bits, false, false);
    };
    const auto scores = swapped(s), exponents = swapped(e);
    s = __uint_as_float(scores[0]);
    e = __uint_as_float(exponents[0]);
    raise(__uint_as_float(scores[1]), __uint_as_float(exponents[1]));
  }
  __device__ inline float unit() const { return pow2((int)e); }
};

// The blocks of 16 tokens that rows at positions lo .. hi see some token of, as a list: the first ones, then those of the window.
struct Span {
  int sinks, window, count;                          // blocks of the first tokens; the window's first block; blocks in all
  __device__ inline int block(int i) const { return i < sinks ? i : i - sinks + window; }
};
// Some of such a list.
struct Cut : Span {
  int skip;                                          // blocks before its first
  __device__ inline int block(int i) const { return Span::block(i + skip); }
  __device__ inline int place(int block) const { return min(block, sinks) + max(block - window, 0); }       // blocks of the whole list before this one
  __device__ inline Cut() {}
  __device__ inline Cut(const Span &whole, int first, int last) : Span(whole) // those of blocks first .. last - 1
  {
    skip = min(place(first), count);
    count = max(min(place(last), count) - skip, 0);
  }
};
__device__ inline Span span_of(const Pages &c, int lo, int hi)
{
  Span s = {0, 0, 0};
  if (hi < 0) return s;
  const int last = hi / kBlock;
  if (c.window > 0 && lo >= c.window) {
    const int w = (lo - c.window + 1) / kBlock, n = (int)min(((long)c.sinks + kBlock - 1) / kBlock, (long)last + 1);
    if (w > n) { s.sinks = n; s.window = w; }
  }
  s.count = s.sinks + last - s.window + 1;
  return s;
}
__device__ inline bool sees(const Pages &c, int p, int token)
{
  return token <= p && (c.window == 0 || token > p - c.window || token < c.sinks);
}
// whether rows at lo .. hi all see all of a block
__device__ inline bool all_see(const Pages &c, int lo, int hi, int t0)
{
  return t0 + kBlock - 1 <= lo && (c.window == 0 || t0 > hi - c.window || t0 + kBlock <= c.sinks);
}

// Tiles of four blocks that rows up to position hi, from position lo on, see in full: from this one on, and before this one.  (The first
// tokens' blocks before a window are not among them.)
__device__ inline int inner_first(const Pages &c, const Span &s, int hi)
{
  if (c.window == 0 || hi < c.window) return 0;
  const int block = (hi - c.window + kBlock) / kBlock;                 // the first whose tokens are all > hi - window
  return (max(block - s.window, 0) + s.sinks + 3) / 4;
}
__device__ inline int inner_last(const Span &s, int lo) { return max((lo + 1) / kBlock - s.window + s.sinks, 0) / 4; }
// (of some of a list, which may end before the rows do)
__device__ inline int inner_first(const Pages &c, const Cut &s, int hi)
{
  if (c.window == 0 || hi < c.window) return 0;
  const int block = (hi - c.window + kBlock) / kBlock;
  return (max(max(block - s.window, 0) + s.sinks - s.skip, 0) + 3) / 4;
}
__device__ inline int inner_last(const Cut &s, int lo) { return min(max((lo + 1) / kBlock - s.window + s.sinks - s.skip, 0), s.count) / 4; }
__device__ inline float read_lane(float x, int lane) { return __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(x), lane)); }

// ---- slots that share pages --------------------------------------------------------------------------------------------
//
// What neighbouring slots have in common (a node of the plan) is gone through once, for the rows of all of them, and what is behind it a slot at a
// time, by the same two kernels' work in one launch; a second one joins a row's sums.  Sums lie at [head][column of the plan].
//
// Nodes of more than 16 columns are tiles of 128 columns by 64 tokens, as below: bound by the instruction streams where they are long, else by what a
// piece costs beside its tiles (11 us: the plan's record, the table, keys, values, then 64 KB of sums) and by the second launch, which reads
// the sums again.  Both kinds of work are in one launch as neither fills the chip: 64 beams of 8192 tokens, 8 heads, 4 query heads each: 27 + 7 us a layer
// (132 apart); one document of 131072, 24 slots, 5 query heads: 103 + 9 (930 apart), 625 TFLOP/s; 32 questions of 24 tokens behind 16384, 32 heads: 306 + 22
// (785), 685 TFLOP/s, call by call (at clocks that have settled the pass takes 292 with its plan); 64 samples of 16 prompts behind 1000 tokens: 34 + 6 (73).
template <typename Args> constexpr bool kShares = false;
template <> constexpr bool kShares<SharedArgs> = true;

// of a value that is the same in all lanes: in a scalar register, where loads from memory that the kernel also writes are not by themselves
__device__ inline int same(int v) { return __builtin_amdgcn_readfirstlane(v); }

// Work that a kernel does piece by piece: what depends on the thread alone is not to be kept in registers over all of them (it would be
// computed before the first, and spilled).
template <typename Args> __device__ inline int thread_of()
{
  int x = threadIdx.x;
  if constexpr (kShares<Args>) asm volatile("" : "+v"(x));
  return x;
}

struct Node {
  int slot, row, rows, lo, hi, first, last, before, unit, tiles, base, shares;
  int cols;
};
// (f: the same in all lanes)
__device__ inline Node node_of(const Pages &c, const SharedArgs &a, const int *record)
{
  const int4 *f = reinterpret_cast<const int4 *>(record);
  const int4 x = f[0], y = f[1], z = f[2];
  const int most = c.table_len * c.page_tokens;
  Node n;
  n.slot = min(max(same(x.x), 0), c.slots - 1);
  n.row = min(max(same(x.y), 0), a.rows);
  n.rows = min(max(same(x.z), 0), a.rows - n.row);
  n.lo = min(max(same(x.w), 0), most - 1);
  n.hi = min(max(same(y.x), -1), most - 1);
  n.first = max(same(y.y), 0);
  n.last = min(max(same(y.z), 0), c.table_len * page_blocks(c));
  n.before = same(y.w);
  n.unit = same(z.x); n.tiles = max(same(z.y), 0); n.base = same(z.z); n.shares = max(same(z.w), 0);
  n.cols = n.rows * c.q_per_kv;
  return n;
}
// whether it was made for so many rows and slots
__device__ inline bool plan_holds(const Pages &c, const SharedArgs &a)
{
  return same(a.plan.head[kPlanRows]) == a.rows && same(a.plan.head[kPlanShape]) >> 1 == c.slots;
}

// ---- few rows a slot: up to 16 query columns -----------------------------------------------------------------------------
//
// Bound by the read of the cache.  The work is a list of steps, 128 tokens of a slot and head each, that is dealt out evenly to as many
// workgroups as the chip holds at once, whatever the slots' lengths; every workgroup finds its part from the lengths.  A
// step is 32 tokens for each of four waves, which stay apart until the workgroup leaves a (slot, head).  What a
// workgroup has of a (slot, head) that it shares with others goes to memory, past the L2 of its die, and the last of them to arrive joins
// the shares in the order of the tokens: 32 neighbours first, then the joined ones, so that one sequence can be spread over the chip.

// Measured: 64 slots of up to 8192 tokens, 8 heads, 4 query heads each: 107 us, 5.7 TB/s; one of 131072, 8 heads, 5 query heads each: 52 us,
// 5.2 TB/s; one of 1025, 32 heads: 10.5 us, the latency of its chain of loads (start and length, table, codes, shares).
// 16 columns is one matrix tile, and where the kernels meet: 64 slots of 8192, 8 heads, 16 columns 206 us here, 249 in the other.

constexpr int kCols = 16, kStepBlocks = 8;
constexpr int kGroup = 32;
// Three workgroups to a compute unit; where that would make more than 32 shares of a (slot, head) down to one, which reads as
// fast (one sequence of 131072 tokens, 8 heads: 54 us with 256 workgroups, 61 with 512, 64 with 768).  Counted are the slots that the cache
// has, as lengths are on the device: the same sequence alone in a cache of 64 slots takes 60 us, in one of its own 52.
inline int few_workers(long items) { return (int)(items * kGroup < 256 ? 256 : items * kGroup < kPagesWorkers ? items * kGroup : kPagesWorkers); }

__device__ inline int steps_of(const Pages &c, const AttendArgs &a, int s)
{
  const Rows r = slot_rows(a.start, s, a.rows);
  if (r.count == 0 || r.count * c.q_per_kv > kCols) return 0;
  const int len = slot_length(c, s);
  const int n = (span_of(c, len - r.count, len - 1).count + kStepBlocks - 1) / kStepBlocks;
  return n > 0 ? n : 1;                              // (rows that see nothing are written too)
}
// where slots share pages, entries of the plan: slots that share nothing, and nodes of few columns
__device__ inline int steps_of(const Pages &c, const SharedArgs &a, int i)
{
  return min(max(a.plan.few[(long)i * kNodeInts], 0), c.table_len * page_blocks(c) / kStepBlocks + 1);
}
__device__ inline int few_entries(const Pages &c, const AttendArgs &) { return c.slots; }
__device__ inline int few_entries(const Pages &c, const SharedArgs &a) { return min(max(same(a.plan.head[kPlanFew]), 0), 3 * c.slots); }

// Worker w's part [begin, end) of the steps, and where it begins: slot, and step among the slot's (head by head).
struct Part {
  long begin, end, per;
  int slot;
  long in_slot;
  bool whole;                                        // the slots (by head) that begin in the part are all its own, to their end
};
template <typename Args> __device__ inline Part part_of(const Pages &c, const Args &a, int w, int workers)
{
  __shared__ long sums[4], found_at;
  __shared__ int found, most;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, entries = few_entries(c, a);
  int largest = 0;
  auto scan = [&](int base, long &n, long &upto, long &at) {           // at: the sum before this chunk, then behind it
    const int s = base + tid;
    const int steps = s < entries ? steps_of(c, a, s) : 0;
    n = (long)steps * c.heads;
    if constexpr (kShares<Args>) largest = max(largest, steps);
    upto = n;
    for (int d = 1; d < kWave; d <<= 1) {
      const long y = __shfl_up(upto, d, kWave);
      if (lane >= d) upto += y;
    }
    if (base) __syncthreads();
    if (lane == 63) sums[wave] = upto;
    __syncthreads();
    long before = at;
    for (int i = 0; i < 4; ++i) {
      if (i < wave) before += sums[i];
      at += sums[i];
    }
    upto += before;
  };
  Part p;
  long total = 0, n, upto;
  for (int base = 0; base < entries; base += 256) scan(base, n, upto, total);
  p.per = (total + workers - 1) / workers;
  p.whole = false;
  if constexpr (kShares<Args>) {
    // Where none is longer than a part, parts that meet at slots have nothing to join.
    if (tid == 0) most = 0;
    __syncthreads();
    atomicMax(&most, largest);
    __syncthreads();
    p.whole = most <= p.per;
  }
  p.begin = w * p.per;
  p.end = p.begin + p.per < total ? p.begin + p.per : total;
  if (p.begin >= p.end) return p;
  auto look = [&](int base) {
    if (n > 0 && p.begin >= upto - n && p.begin < upto) {
      found = base + tid;
      found_at = p.begin - (upto - n);
    }
  };
  if (entries <= 256) {
    look(0);
  } else {
    long at = 0;
    for (int base = 0; base < entries && at <= p.begin; base += 256) {
      __syncthreads();
      scan(base, n, upto, at);
      look(base);
    }
  }
  __syncthreads();
  p.slot = __builtin_amdgcn_readfirstlane(found);
  p.in_slot = found_at;
  return p;
}

// A share: [columns][D] sums, maxima, totals.  Stored and loaded past the caches that other dies do not see.
constexpr int part_floats(int D) { return kCols * (D + 2); }
__host__ __device__ constexpr long few_floats(int G, int D) { return G <= kCols ? (long)kPagesWorkers * 2 * part_floats(D) : 0; }
__device__ inline void put(float *p, float x, float y)
{
  const unsigned long long v = (unsigned long long)__float_as_uint(y) << 32 | __float_as_uint(x);
  __hip_atomic_store(reinterpret_cast<unsigned long long *>(p), v, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
}
__device__ inline float2 get(const float *p)
{
  const unsigned long long v =
      __hip_atomic_load(reinterpret_cast<const unsigned long long *>(p), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  return make_float2(__uint_as_float((unsigned)v), __uint_as_float((unsigned)(v >> 32)));
}
__device__ inline void put(float *p, float x) { __hip_atomic_store(p, x, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); }
__device__ inline float get1(const float *p) { return __hip_atomic_load(p, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); }

// Whether this workgroup is the last of n to arrive; the counter is 0 again then.  The shares go past the L2 of the die both ways (put,
// get), so that all it takes is that a wave's stores are done before it is counted.  Ordered by acquire and release instead, every
// arrival writes back and invalidates the L2 under the other workgroups' reads: 64 slots of up to 8192 tokens took 160 us, in place of 111.
__device__ inline bool last_to_arrive(int *counter, int n)
{
  __shared__ int arrived;
  asm volatile("s_waitcnt vmcnt(0)" : : : "memory");
  __syncthreads();
  if (threadIdx.x == 0) {
    arrived = __hip_atomic_fetch_add(counter, 1, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) + 1;
    if (arrived == n) __hip_atomic_store(counter, 0, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  }
  __syncthreads();
  const bool last = arrived == n;
  __syncthreads();
  return last;
}

// Joins n shares; done(column, channel, sum, sum of the next channel, maximum, total).
template <int D, typename Share, typename Done>
__device__ inline void join(int n, int cols, Share share, Done done)
{
  for (int i = threadIdx.x; i < cols * (D / 2); i += 256) {
    const int col = i / (D / 2), d = i % (D / 2) * 2;
    float top = kLowest, l = 0, x = 0, y = 0;
    for (int k = 0; k < n; k += 8) {                 // eight at a time on their way
      float m[8], t[8];
      float2 v[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const float *f = share(k + j < n ? k + j : k);
        m[j] = get1(f + kCols * D + col);
        t[j] = get1(f + kCols * (D + 1) + col);
        v[j] = get(f + col * D + d);
      }
      float now = top;
#pragma unroll
      for (int j = 0; j < 8; ++j) now = fmaxf(now, m[j]);
      const float f = exp2_fast(top - now);
      top = now;
      l *= f; x *= f; y *= f;
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        if (k + j >= n) break;
        const float e = exp2_fast(m[j] - top);
        l = fmaf(t[j], e, l);
        x = fmaf(v[j].x, e, x);
        y = fmaf(v[j].y, e, y);
      }
    }
    done(col, d, x, y, top, l);
  }
}

template <int D> struct FewShared {
  float sums[4][kCols][D + 4], tops[4][kCols], totals[4][kCols];
};
// kAlone: a wave has a (slot, head) of a short list by itself, in steps of 32 tokens, and no part in other waves' work.
template <bool BF16, int D, bool kAlone = false, typename Args>
__device__ __forceinline__ void few_rows(const Pages &c, const Args &a, int worker, int workers, FewShared<D> &shared)
{
  constexpr int H = D / 64, T = D / 16, kBlocks = kAlone ? 2 : kStepBlocks;
  auto &sums = shared.sums;
  auto &tops = shared.tops, &totals = shared.totals;
  const int wave = __builtin_amdgcn_readfirstlane(thread_of<Args>() >> 6), lane = thread_of<Args>() & 63, n = lane & 15, g = lane >> 4;
  const int G = c.q_per_kv;
  Part part;
  if constexpr (kAlone) {
    // units to the waves of all workgroups, the workgroups first
    part.begin = worker + wave * workers;
    part.end = (long)min(max(same(a.plan.head[kPlanShort]), 0), 3 * c.slots) * c.heads;
  } else {
    part = part_of(c, a, worker, workers);
  }
  if (part.begin >= part.end) return;
  int s = part.slot;
  long in_slot = part.in_slot;
  for (long pos = part.begin; pos < part.end;) {
    int steps = 0, head, from, to;
    if constexpr (kAlone) {
      s = same((int)((unsigned)pos / (unsigned)c.heads));
      head = same((int)pos - s * c.heads);
      from = to = 0;
    } else {
      steps = steps_of(c, a, s);
      if constexpr (kShares<Args>) steps = same(steps);
      if (steps == 0) { ++s; in_slot = 0; continue; }
      head = (int)((unsigned long)in_slot >> 32 ? in_slot / steps : (unsigned)in_slot / (unsigned)steps);
      from = (int)(in_slot - (long)head * steps);
      to = kShares<Args> && part.whole ? steps : (int)min((long)steps, from + (part.end - pos));
      if (kShares<Args> && part.whole && from > 0) { // another worker's
        pos += to - from;
        in_slot += to - from;
        if (in_slot == (long)steps * c.heads) { ++s; in_slot = 0; }
        continue;
      }
    }

    Rows rows;
    int lo, hi, p, read = s, base_column = -1;
    std::conditional_t<kShares<Args>, Cut, Span> span;
    if constexpr (kShares<Args>) {
      const int4 *f = reinterpret_cast<const int4 *>(a.plan.few + (long)(kAlone ? 3 * c.slots - 1 - s : s) * kNodeInts);
      const int4 x = f[0], y = f[1], z = f[2];
      const int most = c.table_len * c.page_tokens;
      if constexpr (kAlone) to = steps = min(max(same(x.x), 1), kShortBlocks / 2);
      read = min(max(same(x.y), 0), c.slots - 1);
      rows.first = min(max(same(x.z), 0), a.rows);
      rows.count = min(max(same(x.w), 0), a.rows - rows.first);
      lo = min(max(same(y.x), 0), most - 1);
      hi = min(max(same(y.y), -1), most - 1);
      span = Cut(span_of(c, lo, hi), max(same(y.z), 0), min(max(same(y.w), 0), c.table_len * page_blocks(c)));
      base_column = same(z.x);
      p = hi + 1 - rows.count + n / G;
      if (same(z.y)) p = n < rows.count * G ? min(max(a.plan.pos[rows.first + n / G], -1), most - 1) : -1;
    } else {
      rows = slot_rows(a.start, read, a.rows);
      const int len = slot_length(c, read);
      lo = len - rows.count;
      hi = len - 1;
      span = span_of(c, lo, hi);
      p = lo + n / G;
    }
    const int cols = kShares<Args> ? min(rows.count * G, kCols) : rows.count * G, mine = kAlone ? 0 : wave * 2;
    u4 q[H][2];
#pragma unroll
    for (int h = 0; h < H; ++h)
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        q[h][i] = u4{0, 0, 0, 0};
        if (n < cols)
          q[h][i] = reinterpret_cast<const u4 *>(a.q)[(rows.first + n / G) * (a.stride / 8) + (head * G + n % G) * (D / 8) + h * 8 + g * 2 + i];
      }

    // A wave's blocks are looked up 64 at a time, a lane each: two of every step.  The next step's keys are requested as soon as this one's
    // are multiplied, its values likewise; every load is made (of the last step's blocks behind it, of the pool's first block where
    // there is none): with a branch around it the compiler would wait for all loads where it means to wait for the older ones.
    const int *table = c.table + (size_t)read * c.table_len;
    u4 k[2][H], v[2][H];
    int ats, exs, base, end;                         // the lane's block in the pool, or -1, and its exponents; steps [base, end)
    auto look = [&](int step) {
      base = step;
      end = min(to, base + kWave / 2);
      const int i = (base + lane / 2) * kBlocks + mine + (lane & 1), block = span.block(i);
      const bool there = base + lane / 2 < to && i < span.count;
      const int page = table[there ? entry_of(c, block) : 0];
      ats = there ? block_in(c, page, head, block) : -1;
      exs = reinterpret_cast<const unsigned short *>(c.exps)[max(ats, 0)];
    };
    auto request = [&](u4 (&x)[2][H], const unsigned char *codes, int step) {
#pragma unroll
      for (int b = 0; b < 2; ++b) {
        const int at = max(__builtin_amdgcn_readlane(ats, (min(step, end - 1) - base) * 2 + b), 0);
        const Bytes block = scalar_bytes(codes, at * ((long)kBlock * D));
#pragma unroll
        for (int h = 0; h < H; ++h) x[b][h] = __builtin_nontemporal_load((Pieces)(block + (unsigned)(h * kWave + lane) * 16));
      }
    };
    auto tokens_of = [&](int step, int b) {          // the first token of a block, -1: not there
      const int at = __builtin_amdgcn_readlane(ats, (step - base) * 2 + b);
      return at >= 0 ? span.block(step * kBlocks + mine + b) * kBlock : -1;
    };

    f4 acc[T];
#pragma unroll
    for (int t = 0; t < T; ++t) acc[t] = f4{0, 0, 0, 0};
    Top top = {kLowest, kFirstE};
    float total = 0;
    bool spoiled = false;
    auto attend_to = [&](int step) {
      const int t0[2] = {tokens_of(step, 0), tokens_of(step, 1)};
      int ex[2];
#pragma unroll
      for (int b = 0; b < 2; ++b) ex[b] = t0[b] < 0 ? 0 : __builtin_amdgcn_readlane(exs, (step - base) * 2 + b);
      f4 x[2];
#pragma unroll
      for (int b = 0; b < 2; ++b) {
        x[b] = f4{0, 0, 0, 0};
#pragma unroll
        for (int h = 0; h < H; ++h)
#pragma unroll
          for (int i = 0; i < 2; ++i) x[b] = Operand<BF16>::mma16(widen<BF16>(k[b][h][2 * i], k[b][h][2 * i + 1]), q[h][i], x[b]);
      }
      request(k, c.k, step + 1);
#pragma unroll
      for (int b = 0; b < 2; ++b)
        if (t0[b] < 0 || !all_see(c, lo, hi, t0[b])) {
          // What no row sees is taken out, and where rows see different tokens NaN values are too (0 * NaN is NaN); those that some row
          // sees are given to it in the end.
          unsigned keep = 0;
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const int token = t0[b] + 4 * g + i;
            x[b][i] = t0[b] >= 0 && sees(c, p, token) ? x[b][i] : -__builtin_inff();
            if (t0[b] >= 0 && token <= hi && (c.window == 0 || token + c.window > lo || token < c.sinks)) keep |= 255u << 8 * i;
          }
#pragma unroll
          for (int h = 0; h < H; ++h) {
            v[b][h] &= keep;
            if (rows.count > 1)
#pragma unroll
              for (int i = 0; i < 4; ++i) {
                const unsigned bad = code_nans(v[b][h][i]);
                spoiled |= bad != 0;
                v[b][h][i] &= ~bad;
              }
          }
        }
      // the factor is positive, so a block's largest x gives its largest score
      float ve[2], y[2];
#pragma unroll
      for (int b = 0; b < 2; ++b) {
        const float factor = pow2((signed char)ex[b]) * c.scale_log2;
        ve[b] = (float)(signed char)(ex[b] >> 8);
#pragma unroll
        for (int i = 0; i < 4; ++i) x[b][i] = product(x[b][i], factor);
        y[b] = fmaxf(fmaxf(x[b][0], x[b][1]), fmaxf(x[b][2], x[b][3]));
      }
      if (__ballot(fmaxf(top.above(y[0], ve[0]), top.above(y[1], ve[1])) > kBase + kSlack)) {
        Top most = {y[0], ve[0] - kBase};
        most.raise(y[1], ve[1] - kBase);
        most.raise_over<16>();
        most.raise_over<32>();
        const Top was = top;
        top.raise(most.s, most.e);
        const float f = exp2_fast(top.above(was.s, was.e));
        total *= f;
#pragma unroll
        for (int i = 0; i < T; ++i) acc[i] *= f;
      }
      u4 weights;
#pragma unroll
      for (int b = 0; b < 2; ++b) {
        float w[4];
        const float zero = ve[b] - top.e;
#pragma unroll
        for (int i = 0; i < 4; ++i) w[i] = exp2_fast((x[b][i] - top.s) + zero);
        total = fmaf((w[0] + w[1]) + (w[2] + w[3]), pow2(-(signed char)(ex[b] >> 8)), total);
        weights[2 * b] = half_pair(w[0], w[1]);
        weights[2 * b + 1] = half_pair(w[2], w[3]);
      }
#pragma unroll
      for (int h = 0; h < H; ++h)
#pragma unroll
        for (int i = 0; i < 4; ++i)
          acc[h * 4 + i] = Operand<false>::mma16(widen<false>(v[0][h][i], v[1][h][i]), weights, acc[h * 4 + i]);
      request(v, c.v, step + 1);
    };
    for (int chunk = from; chunk < to; chunk += kWave / 2) {
      look(chunk);
      request(k, c.k, chunk);
      request(v, c.v, chunk);
      for (int step = chunk; step < end; ++step) attend_to(step);
    }
    if (__ballot(spoiled))                           // the NaN that were taken out, counted for the rows that see them
#pragma unroll 1
      for (int step = from; step < to; ++step) {
        look(step);
        request(v, c.v, step);
        half8 seen;
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const int t0 = tokens_of(step, i / 4);
          seen[i] = t0 >= 0 && !all_see(c, lo, hi, t0) && sees(c, p, t0 + 4 * g + i % 4) ? 1 : 0;
        }
#pragma unroll
        for (int h = 0; h < H; ++h)
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const u4 ones = widen<false>(code_nans(v[0][h][i]) & 0x38383838u, code_nans(v[1][h][i]) & 0x38383838u);    // the code of 1
            const f4 count = Operand<false>::mma16(ones, __builtin_bit_cast(u4, seen), f4{0, 0, 0, 0});
#pragma unroll
            for (int j = 0; j < 4; ++j) acc[h * 4 + i][j] = count[j] > 0 ? __builtin_nanf("") : acc[h * 4 + i][j];
          }
      }

    // the four waves' sums, relative to the largest of their scores
    total += __shfl_xor(total, 16, kWave);
    total += __shfl_xor(total, 32, kWave);
    if constexpr (kAlone) {
      pos += 4 * workers;
      if (n >= cols) continue;
      if (base_column < 0) {
        const long to_row = (long)(rows.first + n / G) * c.heads * G + head * G + n % G;
        const float r = 1.f / total;
#pragma unroll
        for (int t = 0; t < T; ++t) {
          auto stored = [&](int j) { return (unsigned)Operand<BF16>::store(share_of(acc[t][j], total, r)); };
          reinterpret_cast<uint2 *>(a.out)[to_row * (D / 4) + t * 4 + g] = make_uint2(stored(0) | stored(1) << 16, stored(2) | stored(3) << 16);
        }
        if (a.lse && g == 0) a.lse[to_row] = total == 0.f ? -__builtin_inff() : (top.s + (top.e + __builtin_log2f(total))) * 0.6931471805599453f;
      } else if (base_column + n < a.columns) {
        const long at = (long)head * a.columns + base_column + n;
        const float unit_of_e = top.unit();
#pragma unroll
        for (int t = 0; t < T; ++t) *reinterpret_cast<f4 *>(a.trunk + at * D + t * 16 + g * 4) = acc[t] * unit_of_e;
        float *tops_at = a.trunk + c.heads * a.columns * D + at;
        if (g == 0) {
          tops_at[0] = top.s == kLowest ? -__builtin_inff() : top.s;
          tops_at[c.heads * a.columns] = total * unit_of_e;
        }
      }
      continue;
    } else {
    if (g == 0) { tops[wave][n] = top.s; totals[wave][n] = total * top.unit(); }
    __syncthreads();
    const float largest = fmaxf(fmaxf(tops[0][n], tops[1][n]), fmaxf(tops[2][n], tops[3][n])), f = exp2_fast(top.s - largest) * top.unit();
    if (n < cols)
#pragma unroll
      for (int t = 0; t < T; ++t) *reinterpret_cast<f4 *>(&sums[wave][n][t * 16 + g * 4]) = acc[t] * f;
    __syncthreads();
    auto finish = [&](int col, int d, float x, float y, float m, float l) {
      if constexpr (kShares<Args>)
        if (base_column >= 0) {
          const long at = (long)head * a.columns + base_column + col;
          if ((long)base_column + col >= a.columns) return;
          *reinterpret_cast<float2 *>(a.trunk + at * D + d) = make_float2(x, y);
          float *tops = a.trunk + c.heads * a.columns * D;
          if (d == 0) { tops[at] = l == 0.f && m == kLowest ? -__builtin_inff() : m; tops[c.heads * a.columns + at] = l; }
          return;
        }
      const float r = 1.f / l;
      const long at = (long)(rows.first + col / G) * c.heads * G + head * G + col % G;
      reinterpret_cast<unsigned *>(a.out)[at * (D / 2) + d / 2] =
          (unsigned)Operand<BF16>::store(share_of(x, l, r)) | (unsigned)Operand<BF16>::store(share_of(y, l, r)) << 16;
      if (a.lse && d == 0) a.lse[at] = l == 0.f ? -__builtin_inff() : (m + __builtin_log2f(l)) * 0.6931471805599453f;
    };
    const bool whole = from == 0 && to == steps;
    // this share is number i of the (slot, head), which begins in worker w0; share 0 lies in that worker's second place, the others in the first
    const long first = pos - from;
    const int w0 = (int)(first / part.per), shares = (int)((first + steps - 1) / part.per) - w0 + 1, i = worker - w0;
    auto share = [&](int k) { return a.parts + ((long)(w0 + k) * 2 + (k == 0)) * part_floats(D); };
    auto store = [&](float *to_share) {
      return [=](int col, int d, float x, float y, float m, float l) {
        put(to_share + col * D + d, x, y);
        if (d == 0) { put(to_share + kCols * D + col, m); put(to_share + kCols * (D + 1) + col, l); }
      };
    };
    const auto to_mine = store(share(i));
    for (int at = threadIdx.x; at < cols * (D / 2); at += 256) {
      const int col = at / (D / 2), d = at % (D / 2) * 2;
      const float m = fmaxf(fmaxf(tops[0][col], tops[1][col]), fmaxf(tops[2][col], tops[3][col]));
      float l = 0, x = 0, y = 0;
#pragma unroll
      for (int wv = 0; wv < 4; ++wv) {
        l += totals[wv][col] * exp2_fast(tops[wv][col] - m);
        x += sums[wv][col][d];
        y += sums[wv][col][d + 1];
      }
      if (whole) finish(col, d, x, y, m, l);
      else to_mine(col, d, x, y, m, l);
    }
    if (!whole) {
      // counters of a worker: of the (slot, head) that begins in it, of one that goes on, of the groups
      const int group = i / kGroup, members = min(kGroup, shares - group * kGroup), groups = (shares + kGroup - 1) / kGroup;
      int *counters = a.counters + 3 * (w0 + group * kGroup);
      if (last_to_arrive(counters + (group > 0), members)) {
        auto mine = [&](int k) { return share(group * kGroup + k); };
        if (groups == 1) {
          join<D>(members, cols, mine, finish);
        } else {
          join<D>(members, cols, mine, [&](int col, int d, float x, float y, float m, float l) {
            *reinterpret_cast<float2 *>(&sums[0][col][d]) = make_float2(x, y);
            if (d == 0) { tops[0][col] = m; totals[0][col] = l; }
          });
          __syncthreads();                           // every share is read: the first one's place is free
          const auto to_first = store(share(group * kGroup));
          for (int at = threadIdx.x; at < cols * (D / 2); at += 256) {
            const int col = at / (D / 2), d = at % (D / 2) * 2;
            to_first(col, d, sums[0][col][d], sums[0][col][d + 1], tops[0][col], totals[0][col]);
          }
          if (last_to_arrive(a.counters + 3 * w0 + 2, groups)) join<D>(groups, cols, [&](int k) { return share(k * kGroup); }, finish);
        }
      }
    }
    __syncthreads();
    pos += to - from;
    in_slot += to - from;
    if (in_slot == (long)steps * c.heads) { ++s; in_slot = 0; }
    }
  }
}

template <bool BF16, int D>
__global__ __launch_bounds__(256, 3) void few_kernel(Pages c, AttendArgs a)
{
  __shared__ FewShared<D> shared;
  few_rows<BF16, D>(c, a, blockIdx.x, gridDim.x, shared);
}

// ---- many rows a slot ---------------------------------------------------------------------------------------------------
//
// Bound by the matrix and vector instructions.  A workgroup has 128 query columns of a (slot, head), 32 to a wave, and goes through the
// tokens in tiles of 64: the codes of the tile after the next are on their way from memory, those of the next are widened once for
// all four waves and put into the LDS in the order in which the matrix operands read them (whole lines, no padding), one
// barrier a tile.  Where there are too few workgroups for the chip, several share a (slot, head, 128 columns), each some
// of its tiles, and a second launch joins them.
//
// Measured: 32 heads of a prompt of 8192 tokens 561 us (980 TFLOP/s of the visible pairs; a large library product reaches 1184), the
// matrix cores busy for 46 % of the cycles and the vector units about as long (6 of their instructions a product: widening, exponentials,
// sums), half of it at the same time; 4 x 4096 tokens, 40 heads, a window of 820: 403 us (617), 10 of their instructions a product.
// Two workgroups are what the registers hold of a compute unit at D = 128, three at 64 (167 registers; 8192 tokens, 32 heads: 351 us, 365 with two);
// eight waves of 16 columns to a workgroup took 605 us in place of 591, four of 64 columns spilled.

constexpr int kWide = 128, kTile = 64;               // columns and tokens
// Workgroups that are enough not to split: two to a compute unit.  128 rows over 8192 tokens, 32 heads: 54 us (67 with 256, 46 with
// 1024, 191 unsplit); 1024 rows: 182 us (247, 195, 246); 64 slots of 71 columns over 8192 tokens: 51 us (67, 49, 137).  The host counts a tile for every
// slot that the cache has: 256 rows of one slot over 8192 tokens, 8 heads, take 35 us in a cache of one slot and, unsplit, 182 in one of 64.
constexpr int kEnough = 512;
// Slots of few rows in such a call: their steps are dealt out to this many workgroups behind the others of the launch, where they read memory
// while the last tiles are multiplied.  32 slots, half of them prompts: 197 us (256 or 768 of them 195 and 196), 211 in front of the
// others, 215 as a launch of their own, whose 4 us a call without such slots would pay as well.
constexpr int kFewBeside = 512;

__host__ __device__ inline long wide_items(int slots, int q_per_kv, long rows) { return rows * q_per_kv / kWide + slots; }
inline int wide_splits(long items, long tokens)
{
  const long most = (tokens / kTile + 3) / 2;        // two tiles each, at least
  const long n = items >= kEnough ? 1 : (kEnough + items - 1) / items;
  return (int)(n < most ? n : most);
}
constexpr int wide_floats(int D) { return kWide * (D + 2); }

// Column tile x of the list over all slots, those of up to 16 columns left out (they are the other kernel's).  Up to 64 slots, and where
// tiles are not split, every wave has all of them in its lanes, one load deep, and the list has their tiles alone, longest slot first:
// the last workgroups to begin are short ones.  Else slot s has its tiles from floor(start[s] G / 128) + s on,
// which leaves each as many as it can have.  32 slots of 537 to 4096 tokens, 8 heads: 201 us, as the slots are 247; 64 slots of 2048: 204 and
// 233; 4 slots of 4096: 830 and 816.  Split tiles have a second launch that would do all of this again: 64 slots, 24 us as they are, 30 in order.
struct Columns { int slot, first, count, len; };     // first column, columns of the slot in all; its tokens
// (where slots share pages, those of 128 columns and more are what is left to wide_kernel)
template <typename Args> constexpr int kLeast = kShares<Args> ? kTrunkTile : kCols + 1;
template <typename Args> __device__ inline bool columns_of(const Pages &c, const Args &a, int x, bool sorted, Columns &t, Rows &rows)
{
  const int G = c.q_per_kv, lane = threadIdx.x & 63;
  int i;
  if (sorted) {
    const int s = min(lane, c.slots - 1);
    const Rows r = slot_rows(a.start, s, a.rows);
    const int len = slot_length(c, s), n = lane < c.slots && r.count * G >= kLeast<Args> ? (r.count * G + kWide - 1) / kWide : 0;
    const int seen = c.window > 0 ? min(len, min(c.window, len) + r.count) : len;
    const int key = (seen / kTile << 6) + 63 - lane;   // tokens that a tile sees, in tiles; ties as the slots are
    int before = 0;
    for (int base = 0; base < c.slots; base += 8)
#pragma unroll
      for (int j = base; j < base + 8; ++j)
        before += __builtin_amdgcn_readlane(n, j) & -(int)(__builtin_amdgcn_readlane(key, j) > key);
    const unsigned long long found = __ballot((unsigned)(x - before) < (unsigned)n);
    if (!found) return false;
    t.slot = __ffsll(found) - 1;
    rows.first = __builtin_amdgcn_readlane(r.first, t.slot);
    rows.count = __builtin_amdgcn_readlane(r.count, t.slot);
    t.len = __builtin_amdgcn_readlane(len, t.slot);
    i = x - __builtin_amdgcn_readlane(before, t.slot);
  } else {
    auto base = [&](int s) {
      const int f = a.start[s];
      return (long)(f < 0 ? 0 : f < a.rows ? f : a.rows) * G / kWide + s;
    };
    t.slot = __builtin_amdgcn_readfirstlane(last_slot_at(c.slots, x, base));
    rows = slot_rows(a.start, t.slot, a.rows);
    t.len = slot_length(c, t.slot);
    i = (int)(x - base(t.slot));
  }
  t.count = rows.count * G;
  const int n = (t.count + kWide - 1) / kWide;
  if (i < 0 || i >= n || t.count < kLeast<Args>) return false;               // (i < 0: before the first slot's rows)
  t.slot = __builtin_amdgcn_readfirstlane(t.slot);
  t.count = __builtin_amdgcn_readfirstlane(t.count);
  t.len = __builtin_amdgcn_readfirstlane(t.len);
  rows.first = __builtin_amdgcn_readfirstlane(rows.first);
  rows.count = __builtin_amdgcn_readfirstlane(rows.count);
  t.first = __builtin_amdgcn_readfirstlane((n - 1 - i) * kWide);       // the longest first
  return true;
}

template <int D> using Tiles = u4[4][kTile * D / 8];  // of keys, two, and of values
// A piece of the nodes' tiles: 128 columns of a node by one head, tiles [from, to), the piece-th of these columns.
struct Piece {
  Node node;
  int column, head, from, to, piece;
  bool only;                                         // the chunk has no second piece
};

template <bool BF16, int D, typename Args>
__global__ __launch_bounds__(256, 2) void wide_kernel(Pages c, Args a, unsigned items, int splits)
{
  __shared__ __align__(16) Tiles<D> tiles_of;
  __shared__ int spoiled;
  if constexpr (kShares<Args>)
    if (!plan_holds(c, a)) return;
  const unsigned total = items * c.heads * splits;
  if (blockIdx.x >= total) {
    static_assert(sizeof(FewShared<D>) <= sizeof tiles_of, "the slots of few rows work in the same LDS");
    if constexpr (!kShares<Args>) few_rows<BF16, D>(c, a, blockIdx.x - total, gridDim.x - total, reinterpret_cast<FewShared<D> &>(tiles_of));
    return;
  }
  // Where the workgroups divide by the dies, each die works through neighbouring items, head by head, and what a (slot, head) has cached stays in
  // its L2: 32 heads of 8192 tokens 555 us, 684 in their order; 32 uneven slots, 8 heads 170 and 200; with 2 or 4 heads, which put long rows on one die
  // and short ones on another, no slower: 8191 rows, 4 heads of 8 557 and 557, 4095 rows, 2 heads of 16 150 and 150.
  unsigned id = blockIdx.x;
  if (total % 8 == 0) id = id % 8 * (total / 8) + id / 8;
  constexpr bool kTrunk = false;
  constexpr Piece trunk = {};
#include "lessdec_pages_wide.h"
}

// A piece of the nodes' tiles.
template <bool BF16, int D>
__device__ __forceinline__ void wide_piece(const Pages &c, const SharedArgs &a, const Piece &trunk, Tiles<D> &tiles_of, int &spoiled)
{
  using Args = SharedArgs;
  constexpr bool kTrunk = true;
  constexpr unsigned id = 0, items = 1;
  constexpr int splits = 1;
#include "lessdec_pages_wide.h"
}

// Worker w's pieces of the nodes' tiles.
template <bool BF16, int D>
__device__ __forceinline__ void trunk_pieces(const Pages &c, const SharedArgs &a, unsigned w, int workers, Tiles<D> &tiles_of, int &spoiled)
{
  // (the first piece is loaded before what says whether there is one)
  const int *mine = a.plan.first + w * kFirstInts;
  Piece x;
  x.node = node_of(c, a, mine);
  const int4 f = reinterpret_cast<const int4 *>(mine)[3], g = reinterpret_cast<const int4 *>(mine)[4];
  const int units = max(same(a.plan.head[kPlanUnits]), 0), nodes = min(max(same(a.plan.head[kPlanNodes]), 0), 3 * c.slots);
  if (units == 0 || nodes == 0) return;
  const Trunk all{(unsigned)units * c.heads, max(workers, 1), max(same(a.plan.head[kPlanChunk]), 1)};
  const bool whole = same(a.plan.head[kPlanShape]) & 1;
  const unsigned end = whole ? w + 1 : all.first(w + 1);
  x.head = same(f.x); x.column = same(f.y); x.from = same(f.z); x.to = same(f.w); x.piece = same(g.x); x.only = same(g.y);
  int now = same(g.z);
  for (unsigned at = whole ? w : all.first(w); at < end;) {
    // (no plan of this library's fails here)
    if ((unsigned)x.head >= (unsigned)c.heads || (unsigned)x.column >= (unsigned)x.node.cols || x.from < 0 || x.piece < 0 || now <= 0 ||
        x.to > c.table_len * page_blocks(c) / 4 + 1) return;
    if (x.from < x.to) wide_piece<BF16, D>(c, a, x, tiles_of, spoiled);
    at += now;
    if (at >= end || whole) return;
    __syncthreads();
    x.head = same((int)(at / (unsigned)units));
    const int in_head = (int)(at - (unsigned)x.head * units);
    const int i = last_at(nodes, in_head, [&](int k) { return (long)a.plan.node[(long)k * kNodeInts + 8]; });
    x.node = node_of(c, a, a.plan.node + (long)same(i) * kNodeInts);
    if (in_head < x.node.unit) return;
    const Trunk::Dealt y = all.dealt(x.node.tiles, x.node.cols, in_head - x.node.unit, (int)(end - at));
    x.column = same(y.column); x.from = same(y.from); x.to = same(y.to); x.piece = same(y.piece); x.only = same(y.only);
    now = same(y.units);
  }
}

// The plan's work: entries of few columns by the first workgroups, nodes by those behind them.
template <bool BF16, int D>
__global__ __launch_bounds__(256, 2) void shared_kernel(Pages c, SharedArgs a)
{
  __shared__ __align__(16) Tiles<D> tiles_of;
  __shared__ int spoiled;
  if (!plan_holds(c, a)) return;
  const int both = same(a.plan.head[kPlanWorkers]), few = both >> kPlanFewShift, workers = both & ((1 << kPlanFewShift) - 1);
  if ((int)blockIdx.x < few) {
    auto &parts = reinterpret_cast<FewShared<D> &>(tiles_of);
    few_rows<BF16, D, true>(c, a, blockIdx.x, few, parts);
    if (same(a.plan.head[kPlanFew]) > 0) few_rows<BF16, D>(c, a, blockIdx.x, few, parts);
  } else {
    unsigned w = blockIdx.x - few;
    if ((int)w >= workers) return;
    if (workers % 8 == 0) w = w % 8 * (workers / 8) + w / 8;           // (neighbours on one die)
    trunk_pieces<BF16, D>(c, a, w, workers, tiles_of, spoiled);
  }
}

// A wave joins a row's sums by one query head: those of its slot's own part and of the nodes around it, a lane a share for their maxima and totals, then
// four channels a lane, of two shares (four where D is 64) at a time.  Bound by its chain of loads (slot, columns, maxima, sums), where there are many
// rows by memory.  64 rows of 32 heads, 23 shares each: 7.2 us; 768 rows of 32 heads: 22 (24 with a share at a time, 34 with sixteen loads on their way:
// 127 registers).
template <bool BF16, int D>
__global__ __launch_bounds__(256) void shared_join_kernel(Pages c, SharedArgs a)
{
  constexpr int kNodes = kTrunkDepth + 1, kLanes = D / 4, kBeside = kWave / kLanes, kLoads = 8;      // lanes of a share, shares of a load
  const int G = c.q_per_kv, heads = c.heads * G, lane = threadIdx.x & 63;
  const int slot = blockIdx.y, id = same((int)(blockIdx.x * 4 + threadIdx.x / kWave));
  const Rows rows = slot_rows(a.start, slot, a.rows);
  int4 chain[kNodes];
#pragma unroll
  for (int d = 0; d < kNodes; ++d) {
    chain[d] = reinterpret_cast<const int4 *>(a.plan.chain)[(long)kNodes * slot + d];
    chain[d].y = max(chain[d].y, 0);
  }
  const int in_slot = id / heads, q_head = id - in_slot * heads, head = q_head / G, g = q_head - head * G;
  if (in_slot >= rows.count || !plan_holds(c, a) || chain[0].x < 0) return;
  int upto[kNodes];                                  // shares of the nodes so far
#pragma unroll
  for (int d = 0; d < kNodes; ++d) {
    const long last = (long)max(chain[d].x, 0) + (long)chain[d].y * max(chain[d].z - 1, 0) + in_slot * G + g;
    upto[d] = (d ? upto[d - 1] : 0) + (last < a.columns ? max(chain[d].z, 0) : 0);
  }
  const float *tops = a.trunk + c.heads * a.columns * D + (long)head * a.columns, *totals = tops + c.heads * a.columns;
  const float *sums = a.trunk + (long)head * a.columns * D + lane % kLanes * 4;
  float top = kLowest, l = 0;
  f4 x = f4{0, 0, 0, 0};
  for (int from = 0; from < upto[kNodes - 1]; from += kWave) {
    const int k = from + lane;
    int column = max(chain[0].x, 0) + k * chain[0].y;
#pragma unroll
    for (int d = 1; d < kNodes; ++d)
      if (k >= upto[d - 1]) column = max(chain[d].x, 0) + (k - upto[d - 1]) * chain[d].y;
    const bool there = k < upto[kNodes - 1];
    column = there ? column + in_slot * G + g : 0;
    float m = tops[column], u = totals[column];
    if (!there) m = -__builtin_inff();
    float now = fmaxf(top, m);
#pragma unroll
    for (int d = 1; d < kWave; d <<= 1) now = fmaxf(now, __shfl_xor(now, d, kWave));
    const bool some = m != -__builtin_inff();        // (no tiles, nothing written)
    const float less = exp2_fast(top - now);
    float f = some ? exp2_fast(m - now) : 0.f;
    top = now;
    u = some ? u * f : 0.f;
#pragma unroll
    for (int d = 1; d < kWave; d <<= 1) u += __shfl_xor(u, d, kWave);
    l = fmaf(l, less, u);
    x *= less;
    // those that are there come first
    const unsigned long long who = __ballot(some);
    const int before = __builtin_amdgcn_mbcnt_hi((unsigned)(who >> 32), __builtin_amdgcn_mbcnt_lo((unsigned)who, 0)), count = __popcll(who);
    const int to = (some ? before : count + lane - before) * 4;
    column = __builtin_amdgcn_ds_permute(to, column);
    f = __int_as_float(__builtin_amdgcn_ds_permute(to, __float_as_int(f)));
    for (int base = 0; base < count; base += kLoads * kBeside) {
      f4 v[kLoads];
#pragma unroll
      for (int j = 0; j < kLoads; ++j)
        v[j] = *reinterpret_cast<const f4 *>(sums + (long)__shfl(column, min(base + j * kBeside + lane / kLanes, count - 1), kWave) * D);
#pragma unroll
      for (int j = 0; j < kLoads; ++j) {
        const int share = base + j * kBeside + lane / kLanes;
        const float w = __shfl(f, share & (kWave - 1), kWave);
        const f4 y = share < count ? v[j] : f4{0, 0, 0, 0};
#pragma unroll
        for (int e = 0; e < 4; ++e) x[e] = fmaf(y[e], share < count ? w : 0.f, x[e]);
      }
    }
  }
#pragma unroll
  for (int d = kLanes; d < kWave; d <<= 1)
#pragma unroll
    for (int e = 0; e < 4; ++e) x[e] += __shfl_xor(x[e], d, kWave);
  const float r = 1.f / l;
  const long to = (long)(rows.first + in_slot) * heads + q_head;
  auto stored = [&](int e) { return (unsigned)Operand<BF16>::store(share_of(x[e], l, r)); };
  const uint2 y = make_uint2(stored(0) | stored(1) << 16, stored(2) | stored(3) << 16);
  if (lane < kLanes) reinterpret_cast<uint2 *>(a.out)[to * kLanes + lane] = y;
  if (a.lse && lane == 0) a.lse[to] = l == 0.f ? -__builtin_inff() : (top + __builtin_log2f(l)) * 0.6931471805599453f;
}

// Eight columns of an item to a workgroup, eight shares on their way at a time.
constexpr int kJoinColumns = 8;
template <bool BF16, int D, typename Args>
__global__ __launch_bounds__(256) void wide_join_kernel(Pages c, Args a, unsigned items, int splits)
{
  const int G = c.q_per_kv;
  const unsigned item = blockIdx.x;
  const int head = item / items;
  Columns t;
  Rows rows;
  if constexpr (kShares<Args>)
    if (!plan_holds(c, a)) return;
  if (!columns_of(c, a, item % items, false, t, rows)) return;
  const float *base = a.parts + few_floats(G, D) + (long)item * splits * wide_floats(D);
  for (int i = threadIdx.x; i < kJoinColumns * (D / 2); i += 256) {
    const int at = blockIdx.y * kJoinColumns + i / (D / 2), d = i % (D / 2) * 2, col = t.first + at;
    if (col >= t.count) return;
    float top = kLowest, l = 0, x = 0, y = 0;
    for (int k = 0; k < splits; k += 8) {
      float m[8], u[8];
      float2 v[8];
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const float *f = base + (long)min(k + j, splits - 1) * wide_floats(D);
        m[j] = k + j < splits ? f[kWide * D + at] : -__builtin_inff();
        u[j] = f[kWide * (D + 1) + at];
        v[j] = *reinterpret_cast<const float2 *>(f + at * D + d);
      }
      float now = top;
#pragma unroll
      for (int j = 0; j < 8; ++j) now = fmaxf(now, m[j]);
      const float less = exp2_fast(top - now);
      top = now;
      l *= less; x *= less; y *= less;
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        if (m[j] == -__builtin_inff()) continue;     // no tiles, nothing written
        const float e = exp2_fast(m[j] - top);
        l = fmaf(u[j], e, l);
        x = fmaf(v[j].x, e, x);
        y = fmaf(v[j].y, e, y);
      }
    }
    const float r = 1.f / l;
    const long to = (long)(rows.first + col / G) * c.heads * G + head * G + col % G;
    reinterpret_cast<unsigned *>(a.out)[to * (D / 2) + d / 2] =
        (unsigned)Operand<BF16>::store(share_of(x, l, r)) | (unsigned)Operand<BF16>::store(share_of(y, l, r)) << 16;
    if (a.lse && d == 0) a.lse[to] = l == 0.f ? -__builtin_inff() : (top + __builtin_log2f(l)) * 0.6931471805599453f;
  }
}

template <bool BF16, int D, typename Args>
hipError_t attend(const Pages &c, const Args &a, hipStream_t st)
{
  const long pairs = (long)c.slots * c.heads;
  if constexpr (kShares<Args>) {
    shared_kernel<BF16, D><<<kSharedWorkers, 256, 0, st>>>(c, a);
    const long columns = (long)a.max_new * c.q_per_kv < kTrunkTile ? (long)a.max_new * c.q_per_kv : kTrunkTile - 1;
    shared_join_kernel<BF16, D><<<dim3((unsigned)((columns * c.heads + 3) / 4), (unsigned)c.slots), 256, 0, st>>>(c, a);
    if ((long)a.max_new * c.q_per_kv < kTrunkTile) return hipGetLastError();
  } else if ((long)a.max_new * c.q_per_kv <= kCols) {
    few_kernel<BF16, D><<<few_workers(pairs), 256, 0, st>>>(c, a);
    return hipGetLastError();
  }
  const long items = wide_items(c.slots, c.q_per_kv, a.rows);
  const int splits = wide_splits(items * c.heads, (long)c.table_len * c.page_tokens);
  const int few = c.q_per_kv <= kCols && !kShares<Args> ? min(few_workers(pairs), kFewBeside) : 0;
  wide_kernel<BF16, D, Args><<<(unsigned)(items * c.heads * splits + few), 256, 0, st>>>(c, a, (unsigned)items, splits);
  if (splits > 1) wide_join_kernel<BF16, D, Args><<<dim3((unsigned)(items * c.heads), kWide / kJoinColumns), 256, 0, st>>>(c, a, (unsigned)items, splits);
  return hipGetLastError();
}

}  // namespace

size_t pages_attend_floats(int slots, int heads, int q_per_kv, int head_dim, long tokens, int rows)
{
  size_t n = (size_t)few_floats(q_per_kv, head_dim);
  if ((long)rows * q_per_kv > kCols) {
    long items = wide_items(slots, q_per_kv, rows) * heads, fewest = wide_items(slots, q_per_kv, 0) * heads;
    if (fewest < kEnough) {
      // splits items: less than kEnough + items workgroups, for any number of rows up to this one
      const long most = wide_splits(fewest, tokens), now = items < kEnough ? items : kEnough - 1;
      long parts = now * most < kEnough + now ? now * most : kEnough + now;
      n += (size_t)parts * wide_floats(head_dim);
    }
  }
  return n;
}

template <typename Args> static hipError_t attend_any(const Pages &c, int dtype, const Args &a, hipStream_t st)
{
  const bool bf16 = dtype == LESSDEC_DTYPE_BF16;
  if (c.head_dim == 128) return bf16 ? attend<true, 128>(c, a, st) : attend<false, 128>(c, a, st);
  return bf16 ? attend<true, 64>(c, a, st) : attend<false, 64>(c, a, st);
}
hipError_t launch_pages_attend(const Pages &c, int dtype, const AttendArgs &a, hipStream_t st) { return attend_any(c, dtype, a, st); }
hipError_t launch_pages_attend_shared(const Pages &c, int dtype, const SharedArgs &a, hipStream_t st) { return attend_any(c, dtype, a, st); }

}  // namespace lessdec
