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
// 2.1e-4 of fp32 weights and the output's own rounding, bfloat16 ones by 1.7e-3 either way (the cases of perf/operators.py).  A query column is a (row, query head of the group) pair: the heads of a group share the
// cached keys and values that a tile has loaded.
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
__device__ inline float read_lane(float x, int lane) { return __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(x), lane)); }

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

// Worker w's part [begin, end) of the steps, and where it begins: slot, and step among the slot's (head by head).
struct Part {
  long begin, end, per;
  int slot;
  long in_slot;
};
__device__ inline Part part_of(const Pages &c, const AttendArgs &a, int w, int workers)
{
  __shared__ long sums[4], found_at;
  __shared__ int found;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  auto scan = [&](int base, long &n, long &upto, long &at) {           // at: the sum before this chunk, then behind it
    const int s = base + tid;
    n = s < c.slots ? (long)steps_of(c, a, s) * c.heads : 0;
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
  for (int base = 0; base < c.slots; base += 256) scan(base, n, upto, total);
  p.per = (total + workers - 1) / workers;
  p.begin = w * p.per;
  p.end = p.begin + p.per < total ? p.begin + p.per : total;
  if (p.begin >= p.end) return p;
  auto look = [&](int base) {
    if (n > 0 && p.begin >= upto - n && p.begin < upto) {
      found = base + tid;
      found_at = p.begin - (upto - n);
    }
  };
  if (c.slots <= 256) {
    look(0);
  } else {
    long at = 0;
    for (int base = 0; base < c.slots && at <= p.begin; base += 256) {
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
template <bool BF16, int D>
__device__ __forceinline__ void few_rows(const Pages &c, const AttendArgs &a, int worker, int workers, FewShared<D> &shared)
{
  constexpr int H = D / 64, T = D / 16;
  auto &sums = shared.sums;
  auto &tops = shared.tops, &totals = shared.totals;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63, n = lane & 15, g = lane >> 4;
  const int G = c.q_per_kv;
  const Part part = part_of(c, a, worker, workers);
  if (part.begin >= part.end) return;
  int s = part.slot;
  long in_slot = part.in_slot;
  for (long pos = part.begin; pos < part.end;) {
    const int steps = steps_of(c, a, s);
    if (steps == 0) { ++s; in_slot = 0; continue; }
    const int head = (int)((unsigned long)in_slot >> 32 ? in_slot / steps : (unsigned)in_slot / (unsigned)steps);
    const int from = (int)(in_slot - (long)head * steps);
    const int to = (int)min((long)steps, from + (part.end - pos));

    const Rows rows = slot_rows(a.start, s, a.rows);
    const int len = slot_length(c, s), lo = len - rows.count, hi = len - 1, cols = rows.count * G;
    const Span span = span_of(c, lo, hi);
    const int p = lo + n / G;
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
    const int *table = c.table + (size_t)s * c.table_len;
    u4 k[2][H], v[2][H];
    int ats, exs, base, end;                         // the lane's block in the pool, or -1, and its exponents; steps [base, end)
    auto look = [&](int step) {
      base = step;
      end = min(to, base + kWave / 2);
      const int i = (base + lane / 2) * kStepBlocks + wave * 2 + (lane & 1), block = span.block(i);
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
      return at >= 0 ? span.block(step * kStepBlocks + wave * 2 + b) * kBlock : -1;
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
    if (g == 0) { tops[wave][n] = top.s; totals[wave][n] = total * top.unit(); }
    __syncthreads();
    const float largest = fmaxf(fmaxf(tops[0][n], tops[1][n]), fmaxf(tops[2][n], tops[3][n])), f = exp2_fast(top.s - largest) * top.unit();
    if (n < cols)
#pragma unroll
      for (int t = 0; t < T; ++t) *reinterpret_cast<f4 *>(&sums[wave][n][t * 16 + g * 4]) = acc[t] * f;
    __syncthreads();
    auto finish = [&](int col, int d, float x, float y, float m, float l) {
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
__device__ inline bool columns_of(const Pages &c, const AttendArgs &a, int x, bool sorted, Columns &t, Rows &rows)
{
  const int G = c.q_per_kv, lane = threadIdx.x & 63;
  int i;
  if (sorted) {
    const int s = min(lane, c.slots - 1);
    const Rows r = slot_rows(a.start, s, a.rows);
    const int len = slot_length(c, s), n = lane < c.slots && r.count * G > kCols ? (r.count * G + kWide - 1) / kWide : 0;
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
  if (i < 0 || i >= n || t.count <= kCols) return false;               // (i < 0: before the first slot's rows)
  t.slot = __builtin_amdgcn_readfirstlane(t.slot);
  t.count = __builtin_amdgcn_readfirstlane(t.count);
  t.len = __builtin_amdgcn_readfirstlane(t.len);
  rows.first = __builtin_amdgcn_readfirstlane(rows.first);
  rows.count = __builtin_amdgcn_readfirstlane(rows.count);
  t.first = __builtin_amdgcn_readfirstlane((n - 1 - i) * kWide);       // the longest first
  return true;
}

template <bool BF16, int D>
__global__ __launch_bounds__(256, 2) void wide_kernel(Pages c, AttendArgs a, unsigned items, int splits)
{
  constexpr int H = D / 64, KK = D / 16, OB = D / 32;
  __shared__ __align__(16) u4 tiles_of[4][kTile * D / 8];
  __shared__ int spoiled;
  const unsigned total = items * c.heads * splits;
  if (blockIdx.x >= total) {
    static_assert(sizeof(FewShared<D>) <= sizeof tiles_of, "the slots of few rows work in the same LDS");
    few_rows<BF16, D>(c, a, blockIdx.x - total, gridDim.x - total, reinterpret_cast<FewShared<D> &>(tiles_of));
    return;
  }
  auto keys = tiles_of, values = tiles_of + 2;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63, n = lane & 31, h = lane >> 5;
  const int G = c.q_per_kv;
  // Where the workgroups divide by the dies, each die works through neighbouring items, head by head, and what a (slot, head) has cached stays in
  // its L2: 32 heads of 8192 tokens 555 us, 684 in their order; 32 uneven slots, 8 heads 170 and 200; with 2 or 4 heads, which put long rows on one die
  // and short ones on another, no slower: 8191 rows, 4 heads of 8 557 and 557, 4095 rows, 2 heads of 16 150 and 150.
  unsigned id = blockIdx.x;
  if (total % 8 == 0) id = id % 8 * (total / 8) + id / 8;
  const int split = id % (unsigned)splits;
  const unsigned item = id / (unsigned)splits;
  const int head = item / items;
  Columns t;
  Rows rows;
  if (!columns_of(c, a, item % items, splits == 1 && c.slots <= kWave, t, rows)) return;
  const int len = t.len, before = len - rows.count;
  const int last_col = min(t.first + kWide, t.count) - 1;
  const int lo = before + t.first / G, hi = before + last_col / G;
  const Span span = span_of(c, lo, hi);
  const int tiles = (span.count + 3) / 4, each = max(2, (tiles + splits - 1) / splits);
  const int from = split * each, to = min(tiles, from + each);

  // this wave's columns
  const int col = t.first + wave * 32 + n;
  const int wave_last = min(t.first + wave * 32 + 31, last_col);
  const int wave_lo = before + (t.first + wave * 32) / G, wave_hi = before + wave_last / G;
  const bool have = t.first + wave * 32 <= last_col;
  const int row = rows.first + col / G, q_head = head * G + col % G;
  // the row, at p, sees the tokens from_token .. p and those before first_tokens
  const int p = col <= last_col ? before + col / G : -1;
  const int from_token = c.window > 0 ? max(max(p, 0) - c.window + 1, 0) : 0, first_tokens = c.window > 0 ? min(c.sinks, p + 1) : 0;
  u4 q[KK];
#pragma unroll
  for (int k = 0; k < KK; ++k) {
    q[k] = u4{0, 0, 0, 0};
    if (col <= last_col) q[k] = reinterpret_cast<const u4 *>(a.q)[row * (a.stride / 8) + q_head * (D / 8) + k * 2 + h];
  }

  // Tiles that all rows of the workgroup, of this wave, see in full: a range [first, last) of the list, none where a page of the
  // slot is missing (which the look-ups below find before such a tile is reached).
  const int all_first = inner_first(c, span, hi), mine_first = inner_first(c, span, wave_hi);
  int all_last = inner_last(span, lo), mine_last = inner_last(span, wave_lo);

  // Blocks are looked up for sixteen tiles at a time, a lane each: the table a chunk ahead, the exponents half a chunk ahead.
  constexpr int kChunk = kWave / 4;
  const int *table = c.table + (size_t)t.slot * c.table_len;
  int chunk = from, page, at, at_next, exps_next;    // at: the lane's block in the pool, -1: not there
  float factor, shift, unit;                         // of the lane's block: t = factor x + shift; its weights add to the sum times unit
  auto look = [&](int tile) {                        // of the chunk that begins with this tile
    const int i = tile * 4 + lane;
    page = table[i < to * 4 && i < span.count ? entry_of(c, span.block(i)) : 0];      // (not looked at here: it is on its way)
  };
  auto place = [&](int tile) {
    const int i = tile * 4 + lane;
    at_next = i < to * 4 && i < span.count ? block_in(c, page, head, span.block(i)) : -1;
    exps_next = reinterpret_cast<const unsigned short *>(c.exps)[max(at_next, 0)];
    if (__ballot(at_next < 0 && i < to * 4 && i < span.count)) all_last = mine_last = 0;
  };
  auto turn = [&] {
    at = at_next;
    const int ex = at < 0 ? 0 : exps_next;           // (of what is not there the load gave any block's: powers of two that are no numbers, perhaps)
    factor = pow2((signed char)ex) * c.scale_log2;
    const int e = (signed char)(ex >> 8);
    shift = (float)e;
    unit = pow2(-e);
  };
  auto at_of = [&](int tile, int b) {
    const int i = tile - chunk;
    return __builtin_amdgcn_readlane(i < kChunk ? at : at_next, i % kChunk * 4 + b);
  };

  // Staging.  A wave brings halves of 64 channels of a block: D = 128 two of them (blocks wave / 2 and wave / 2 + 2), D = 64 one.  Every load
  // is made (of the pool's first block where there is none to read).
  u4 kc[H], vc[H];
  auto piece_block = [&](int j) { return H == 2 ? wave / 2 + 2 * j : wave; };
  const int half = H == 2 ? wave % 2 : 0;
  auto request = [&](int tile) {
    if (tile >= to) return;
#pragma unroll
    for (int j = 0; j < H; ++j) {
      const int block = max(at_of(tile, piece_block(j)), 0);
      const Bytes k = scalar_bytes(c.k, block * ((long)kBlock * D)), v = scalar_bytes(c.v, block * ((long)kBlock * D));
      kc[j] = *(Pieces)(k + (unsigned)(half * kWave + lane) * 16);
      vc[j] = *(Pieces)(v + (unsigned)(half * kWave + lane) * 16);
    }
  };
  // where a word of four tokens' codes of channel 64 half + 16 i + (lane & 15) goes: [block][32 channels][which eight of the 16
  // tokens][channel], tokens 0-3 and 8-11, or 4-7 and 12-15
  auto value_at = [&](int j, int i) {
    const int d = half * 64 + i * 16 + (lane & 15), g = lane >> 4;
    return (((piece_block(j) * OB + d / 32) * 2 + (g & 1)) * 32 + d % 32) * 2 + (g >> 1);
  };
  bool mine_spoiled = false;
  auto stage = [&](int tile, int buf) {
    const int tok = lane & 15, g = lane >> 4;
    // what no row sees is left out, and a NaN among values that only some rows see is taken out (0 * NaN is NaN) and given to those
    // that see it in the end
    if (tile < all_first || tile >= all_last) {
#pragma unroll
      for (int j = 0; j < H; ++j) {
        const bool there = at_of(tile, piece_block(j)) >= 0;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const unsigned bad = code_nans(vc[j][i]);
          mine_spoiled |= there && bad != 0;
          vc[j][i] = there ? vc[j][i] & ~bad : 0;
        }
      }
    }
#pragma unroll
    for (int j = 0; j < H; ++j) {
      const int b = piece_block(j);
      // key operands: [32 tokens][16 channels][half of 8 channels][token]
#pragma unroll
      for (int e = 0; e < 2; ++e)
        keys[buf][(((b >> 1) * KK + half * 4 + g) * 2 + e) * 32 + (b & 1) * 16 + tok] = widen<BF16>(kc[j][2 * e], kc[j][2 * e + 1]);
#pragma unroll
      for (int i = 0; i < 4; ++i)
        reinterpret_cast<uint2 *>(values[buf])[value_at(j, i)] = make_uint2(Operand<false>::pair(vc[j][i], false), Operand<false>::pair(vc[j][i], true));
    }
  };

  f16v acc[OB];
#pragma unroll
  for (int o = 0; o < OB; ++o) acc[o] = f16v{0};
  Top top = {kLowest, kFirstE};
  float level = kLowest;                             // M less kBase, in one
  unsigned long long far = 0;                        // lanes whose M is beyond kNear (as a bool 587 us at 8192 tokens, 32 heads, so 571)
  float sum = 0;
  if (threadIdx.x == 0) spoiled = 0;
  if (from < to) {
    look(from);
    place(from);
    turn();
    look(from + kChunk);
    request(from);
    stage(from, from & 1);
    request(from + 1);
  }

  // A tile's 64 tokens are worked on as two halves: the scores of the second are multiplied while the weights of the first are
  // computed, and its weights while the first half's go into the values.
  bool whole, active;
  float f[4], add[4], units[4];
  f16v x[2];
  auto enter = [&](int tile) {
    const int i = (tile - chunk) * 4;
    whole = tile >= mine_first && tile < mine_last;
    active = have;
    if (!whole) {
      bool some = false;
#pragma unroll
      for (int b = 0; b < 4; ++b) {
        const int t0 = span.block(tile * 4 + b) * kBlock;
        some |= at_of(tile, b) >= 0 && t0 <= wave_hi && (c.window == 0 || t0 + kBlock + c.window > wave_lo || t0 < c.sinks);
      }
      active &= some;
    }
#pragma unroll
    for (int b = 0; b < 4; ++b) {
      f[b] = read_lane(factor, i + b);
      add[b] = read_lane(shift, i + b);
      units[b] = read_lane(unit, i + b);
    }
  };
  // The operands of a product are read from the LDS ahead of what comes before it, so that it does not wait (8192 tokens, 32 heads, a call
  // at a time: 624 us; with the first half of them ahead 631.  Each read as soon as the product before has used its registers: 628, and 657
  // with the barrier before a tile's last product, which then meets no wait for the LDS at all).
  static_assert(KK == 2 * OB, "as many operands of keys as of values");
  u4 ahead[KK];
  auto keys_ahead = [&](int buf, int m) {
#pragma unroll
    for (int k = 0; k < KK; ++k) ahead[k] = keys[buf][(m * KK + k) * 64 + lane];
  };
  auto values_ahead = [&](int buf, int m) {
#pragma unroll
    for (int o = 0; o < KK; ++o) ahead[o] = values[buf][(m * KK + o) * 64 + lane];
  };
  auto scores = [&](int m) {
    x[m] = f16v{0};
#pragma unroll
    for (int k = 0; k < KK; ++k) x[m] = Operand<BF16>::mma32(ahead[k], q[k], x[m]);
  };
  // Which of the lane's eight tokens of a block the row sees is a word of bits (four compares a score took 470
  // us at 40 heads, 4 x 4096 tokens, a window of 820, two 440, this 415).
  auto mask = [&](int tile, int m) {
    auto below = [](int n) { return (1u << min(max(n, 0), 12)) - 1; };
#pragma unroll
    for (int b = 2 * m; b < 2 * m + 2; ++b) {
      const int t0 = span.block(tile * 4 + b) * kBlock + 4 * h;        // the lane has t0 .. t0 + 3 and t0 + 8 .. t0 + 11
      unsigned seen = (below(p + 1 - t0) & ~below(from_token - t0)) | below(first_tokens - t0);
      if (at_of(tile, b) < 0) seen = 0;
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const unsigned all = (unsigned)((int)(seen << (31 - (i & 3) - 8 * (i >> 2))) >> 31);
        x[m][b % 2 * 8 + i] = __uint_as_float((__float_as_uint(x[m][b % 2 * 8 + i]) & all) | (0xff800000u & ~all));
      }
    }
  };
  // Weights of half m, and what they add to the sum (before 2^-e).  Whether one is too large for fp16 shows in these, so the maximum is
  // only looked for where one is, or where scores are far from 0: then M is moved and the weights are computed again, each step rounded by itself.
  u4 weights[2];
  float part[2];
  auto weigh = [&](int m) {
#pragma unroll
    for (int b = 0; b < 2; ++b) {
      const float zero = add[2 * m + b] - level;
      part[b] = 0;
#pragma unroll
      for (int i = 0; i < 8; i += 2) {
        const float y = exp2_fast(fmaf(x[m][b * 8 + i], f[2 * m + b], zero)), z = exp2_fast(fmaf(x[m][b * 8 + i + 1], f[2 * m + b], zero));
        part[b] += y + z;
        weights[b][i / 2] = half_pair(y, z);
      }
    }
  };
  auto weigh_exactly = [&](int m) {
#pragma unroll
    for (int b = 0; b < 2; ++b) {
      const float factor = f[2 * m + b], e = add[2 * m + b] - top.e;
      part[b] = 0;
#pragma unroll
      for (int i = 0; i < 8; i += 2) {
        const float y = exp2_fast((product(x[m][b * 8 + i], factor) - top.s) + e), z = exp2_fast((product(x[m][b * 8 + i + 1], factor) - top.s) + e);
        part[b] += y + z;
        weights[b][i / 2] = half_pair(y, z);
      }
    }
  };
  auto settle = [&](int m) {
    if (far | __ballot(fmaxf(part[0], part[1]) > kMost)) {
      Top most;
#pragma unroll
      for (int b = 0; b < 2; ++b) {
        float y = x[m][b * 8];
#pragma unroll
        for (int i = 1; i < 8; ++i) y = fmaxf(y, x[m][b * 8 + i]);      // (the factor is positive)
        const float score = product(y, f[2 * m + b]), e = add[2 * m + b] - kBase;
        if (b == 0) most = Top{score, e};
        else most.raise(score, e);
      }
      most.raise_over<32>();
      const Top was = top;
      top.raise(most.s, most.e);
      const float less = exp2_fast(top.above(was.s, was.e));
      level = top.s + top.e;
      far = __ballot(fabsf(top.s) > kNear && top.s > kLowest);
      sum *= less;
#pragma unroll
      for (int o = 0; o < OB; ++o) acc[o] *= less;
      weigh_exactly(m);
    }
#pragma unroll
    for (int b = 0; b < 2; ++b) sum = fmaf(part[b], units[2 * m + b], sum);
  };
  auto gather = [&](const u4 (&w)[2]) {
#pragma unroll
    for (int o = 0; o < KK; ++o) acc[o % OB] = Operand<false>::mma32(ahead[o], w[o / OB], acc[o % OB]);
  };
#pragma unroll
  for (int k = 0; k < KK; ++k) asm volatile("" : "+v"(q[k]));          // the queries are waited for here, not (with all codes requested since) in the loop
  __syncthreads();
  if (from < to) {
    enter(from);
    if (active) {
      keys_ahead(from & 1, 0);
      scores(0);
      if (!whole) mask(from, 0);
    }
  }
  for (int tile = from; tile < to; ++tile) {
    const int buf = tile & 1;
    __builtin_amdgcn_s_setprio(0);
    keys_ahead(buf, 1);
    if (tile - chunk == kChunk / 2) place(chunk + kChunk);
    if (tile + 1 < to) {                             // (requested a round ago)
      stage(tile + 1, buf ^ 1);
      request(tile + 2);
    }
    if (active) {
      // products before the other workgroup's staging: 661 -> 621 us at 32 heads x 8192 tokens, clocks settled
      __builtin_amdgcn_s_setprio(1);
      scores(1);
      weigh(0);
      values_ahead(buf, 0);
      settle(0);
      if (!whole) mask(tile, 1);
      const u4 first[2] = {weights[0], weights[1]};
      gather(first);
      weigh(1);
      values_ahead(buf, 1);
      settle(1);
      gather(weights);
    }
    if (tile + 1 == to) break;
    if (tile + 1 - chunk == kChunk) {
      turn();
      chunk += kChunk;
      look(chunk + kChunk);
    }
    enter(tile + 1);
    __syncthreads();
    if (active) {
      keys_ahead(buf ^ 1, 0);
      scores(0);
      if (!whole) mask(tile + 1, 0);
    }
  }

  if (mine_spoiled) spoiled = 1;
  __syncthreads();
  if (spoiled)                                       // the NaN that were taken out, counted for the rows that see them
    for (int tile = from; tile < to; ++tile) {
      chunk = tile;
      look(tile);
      place(tile);
      at = at_next;
      if (tile >= all_first && tile < all_last) continue;
      request(tile);
#pragma unroll
      for (int j = 0; j < H; ++j)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const unsigned one = code_nans(vc[j][i]) & 0x38383838u;      // the code of 1
          reinterpret_cast<uint2 *>(values[0])[value_at(j, i)] = make_uint2(Operand<false>::pair(one, false), Operand<false>::pair(one, true));
        }
      __syncthreads();
#pragma unroll
      for (int b = 0; b < 4; ++b) {
        const int t0 = span.block(tile * 4 + b) * kBlock;
        half8 seen;
#pragma unroll
        for (int i = 0; i < 8; ++i) seen[i] = at_of(tile, b) >= 0 && sees(c, p, t0 + (i & 3) + 4 * h + 8 * (i >> 2)) ? 1 : 0;
#pragma unroll
        for (int o = 0; o < OB; ++o) {
          const f16v count = Operand<false>::mma32(values[0][(b * OB + o) * 64 + lane], __builtin_bit_cast(u4, seen), f16v{0});
#pragma unroll
          for (int i = 0; i < 16; ++i) acc[o][i] = count[i] > 0 ? __builtin_nanf("") : acc[o][i];
        }
      }
      __syncthreads();
    }

  sum += __shfl_xor(sum, 32, kWave);
  if (splits > 1) {
    float *share = a.parts + few_floats(G, D) + (long)id * wide_floats(D);
    const int mine = wave * 32 + n;
    const float unit_of_e = top.unit();
    if (from < to)
#pragma unroll
      for (int o = 0; o < OB; ++o)
#pragma unroll
        for (int i = 0; i < 4; ++i)
          *reinterpret_cast<f4 *>(share + mine * D + o * 32 + i * 8 + h * 4) =
              f4{acc[o][4 * i], acc[o][4 * i + 1], acc[o][4 * i + 2], acc[o][4 * i + 3]} * unit_of_e;
    if (h == 0) { share[kWide * D + mine] = from < to ? top.s : -__builtin_inff(); share[kWide * (D + 1) + mine] = sum * unit_of_e; }
    return;
  }
  if (col > last_col) return;
  const float r = 1.f / sum;
  const long to_row = (long)row * c.heads * G + q_head;
#pragma unroll
  for (int o = 0; o < OB; ++o)
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      auto stored = [&](int j) { return (unsigned)Operand<BF16>::store(share_of(acc[o][4 * i + j], sum, r)); };
      const uint2 y = make_uint2(stored(0) | stored(1) << 16, stored(2) | stored(3) << 16);
      reinterpret_cast<uint2 *>(a.out)[to_row * (D / 4) + o * 8 + i * 2 + h] = y;
    }
  if (a.lse && h == 0) a.lse[to_row] = sum == 0.f ? -__builtin_inff() : (top.s + (top.e + __builtin_log2f(sum))) * 0.6931471805599453f;
}

// Eight columns of an item to a workgroup, eight shares on their way at a time.
constexpr int kJoinColumns = 8;
template <bool BF16, int D>
__global__ __launch_bounds__(256) void wide_join_kernel(Pages c, AttendArgs a, unsigned items, int splits)
{
  const int G = c.q_per_kv;
  const unsigned item = blockIdx.x;
  const int head = item / items;
  Columns t;
  Rows rows;
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

template <bool BF16, int D>
hipError_t attend(const Pages &c, const AttendArgs &a, hipStream_t st)
{
  const long pairs = (long)c.slots * c.heads;
  if ((long)a.max_new * c.q_per_kv <= kCols) {
    few_kernel<BF16, D><<<few_workers(pairs), 256, 0, st>>>(c, a);
    return hipGetLastError();
  }
  const long items = wide_items(c.slots, c.q_per_kv, a.rows);
  const int splits = wide_splits(items * c.heads, (long)c.table_len * c.page_tokens);
  const int few = c.q_per_kv <= kCols ? min(few_workers(pairs), kFewBeside) : 0;
  wide_kernel<BF16, D><<<(unsigned)(items * c.heads * splits + few), 256, 0, st>>>(c, a, (unsigned)items, splits);
  if (splits > 1) wide_join_kernel<BF16, D><<<dim3((unsigned)(items * c.heads), kWide / kJoinColumns), 256, 0, st>>>(c, a, (unsigned)items, splits);
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

hipError_t launch_pages_attend(const Pages &c, int dtype, const AttendArgs &a, hipStream_t st)
{
  const bool bf16 = dtype == LESSDEC_DTYPE_BF16;
  if (c.head_dim == 128) return bf16 ? attend<true, 128>(c, a, st) : attend<false, 128>(c, a, st);
  return bf16 ? attend<true, 64>(c, a, st) : attend<false, 64>(c, a, st);
}

}  // namespace lessdec
