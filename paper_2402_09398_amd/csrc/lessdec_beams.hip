// Choice of the next beams: of every (beam, token) pair of a prompt the best by score + log-probability.
//
// With x the logits of a beam's row, c = score + (x_v - lse), lse = ln sum_v e^{x_v}.  Within a row c rises with x, so a row's best
// pairs are its largest logits (ties: the lower token), found exactly and without any exponential; lse is only needed to compare beams.
// It decides between them, so it is formed in fp64, like everything here that decides, and so that a number added to all of a row's logits changes nothing.
//
// One pass over the logits.  A workgroup has a part of a row, its waves take turns at tiles of 512 logits.  A wave keeps the sum of e^{x - m},
// where m is 0 (fp64 takes e^{+-350}) unless logits lie further out, from the first logit above -inf on, and a list of candidates in the LDS: what is larger than a lower bound of the
// K-th largest so far joins it, and when it is full it is cut to the K largest.  The last workgroup of
// a row joins the parts, the last of a prompt joins its rows, all in the one launch; every sum has an order of its own that depends on
// sizes alone, and rows of the same logits have the same lse to the bit.
//
// Bound by the vector instructions of the exponentials, 18 a logit (65 us and 41 by a polynomial of degree 10 alone, 50 and 27 with remainders in fp32,
// whose error of 1e-10 was not wanted); small calls by a chain of latencies.  64 prompts of 4 beams, 128256 logits in bfloat16: 45 us (1.5 TB/s); 16 of
// 8, 50257 in fp32, 16 picks: 28; one of 4, 32000 in fp16: 14.  The largest with half of the logits masked by -inf: 36, by the type's lowest value 55; with all
// of them below -250: 73.
#include "lessdec_beams.h"

namespace lessdec {
namespace {

typedef unsigned long long u64;
typedef unsigned u4 __attribute__((ext_vector_type(4)));
typedef unsigned u4a2 __attribute__((ext_vector_type(4), aligned(2)));
typedef unsigned u4a4 __attribute__((ext_vector_type(4), aligned(4)));

constexpr int kThreads = 256, kWaves = kThreads / kWave, kRoom = 4 * kWave, kEach = kBeamTile / kWave;
static_assert(kEach == 8, "eight logits a lane and tile");
// Where m is 0, logits in [-kLeast, kFar] are taken as they are and what lies further below counts as e^-kLeast: less than e^-100 of one that the wave has
// seen, as m is 0 only once there is one in [-kFar, kFar].  What comes before a wave's first logit above -inf is not in its sum at all.
constexpr float kFar = 250.f, kLeast = 350.f;

// ---- e^x in fp64 -----------------------------------------------------------------------------------------------------------
// 2^{y / 512} with y = 512 x / ln 2 = n + r, |r| <= 1/2: a table of 2^{i / 512}, i = n mod 512, times a polynomial of degree 3 for 2^{r / 512}
// (its next term is 8.8e-15 at most), times 2^{n / 512 - i / 512} by addition to the exponent.  -kLeast <= x <= 2 kFar.
constexpr int kTable = 512;
struct Exponentials {
  double table[kTable];
  __device__ inline void fill()
  {
    for (int i = threadIdx.x; i < kTable; i += kThreads) table[i] = exp2((double)i / kTable);
  }
  __device__ inline double of(double x) const
  {
    constexpr double kRound = 6755399441055744.0;    // 1.5 * 2^52: its sum with y has n in the low word
    constexpr double kPer = 738.65986093514926;      // 512 / ln 2
    constexpr double c1 = 1.3538030870311431e-03, c2 = 9.1639139924594288e-07, c3 = 4.1353744987218336e-10;    // (ln 2 / 512)^i / i!
    const double s = fma(x, kPer, kRound);
    const int n = (int)__double2loint(s);
    const double r = fma(x, kPer, kRound - s), p = r * fma(r, fma(r, c3, c2), c1);
    const double power = table[n & (kTable - 1)], e = fma(power, p, power);
    return __hiloint2double(__double2hiint(e) + (int)((unsigned)(n & ~(kTable - 1)) << 11), __double2loint(e));
  }
};

// ---- keys ------------------------------------------------------------------------------------------------------------------
// A logit and its token as a number that is larger for the better of two: the larger logit (-0 is 0), then the lower token.
__device__ inline u64 key_of(float x, int token)
{
  const unsigned u = __float_as_uint(x + 0.f);
  return (u64)(u ^ ((unsigned)((int)u >> 31) | 0x80000000u)) << 32 | (unsigned)~token;
}
__device__ inline float logit_of(u64 key)
{
  const unsigned u = (unsigned)(key >> 32);
  return __uint_as_float(u & 0x80000000u ? u ^ 0x80000000u : ~u);
}
__device__ inline int token_of(u64 key) { return (int)~(unsigned)key; }
// likewise of a candidate's c; 0 (that of no number) for what is none
__device__ inline u64 key_of(double c)
{
  if (!(c > -__builtin_inf())) return 0;
  const u64 u = __double_as_longlong(c + 0.0);
  return u ^ ((u64)((long long)u >> 63) | 1ull << 63);
}
__device__ inline double score_of(u64 key) { return __longlong_as_double(key >> 63 ? key ^ 1ull << 63 : ~key); }

__device__ inline u64 read_lane(u64 x, int lane)
{
  return (u64)(unsigned)__builtin_amdgcn_readlane((int)(x >> 32), lane) << 32 | (unsigned)__builtin_amdgcn_readlane((int)x, lane);
}
__device__ inline void put(u64 *p, u64 x) { __hip_atomic_store(p, x, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); }
__device__ inline u64 get(const u64 *p) { return __hip_atomic_load(p, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT); }
__device__ inline void lds_sync()                    // between the lanes of a wave
{
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront", "local");
  __builtin_amdgcn_wave_barrier();
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront", "local");
}

// A wave's candidates: up to kRoom keys in the LDS, in any order.  Keys of one list differ, or else (kTied) the one with the lower mark comes
// first.  Everything but the lanes' own values is the same in all lanes.
template <bool kTied> struct Candidates {
  u64 *keys;
  unsigned short *marks;                             // with kTied
  int count, most;                                   // how many there are, how many are wanted
  u64 least;                                         // of those that were kept at the last cut: what is below is not wanted

  __device__ inline void start(u64 *k, unsigned short *m, int wanted) { keys = k; marks = m; count = 0; most = wanted; least = 1; }
  __device__ inline void add(bool wanted, u64 key, int mark)
  {
    const u64 who = __ballot(wanted);
    if (!who) return;
    if (count > kRoom - kWave) cut();
    if (wanted) {
      const int at = count + __builtin_amdgcn_mbcnt_hi((unsigned)(who >> 32), __builtin_amdgcn_mbcnt_lo((unsigned)who, 0));
      keys[at] = key;
      if constexpr (kTied) marks[at] = (unsigned short)mark;
    }
    count += __popcll(who);
  }
  // the `most` best stay: bit by bit the largest t that so many keys reach
  __device__ inline void cut()
  {
    if (count <= most) return;
    lds_sync();
    const int lane = threadIdx.x & 63;
    u64 k[kRoom / kWave];
    int m[kRoom / kWave];
    unsigned differ = 0;                             // bits of the upper words that are not the same in all
#pragma unroll
    for (int j = 0; j < kRoom / kWave; ++j) {
      const int i = j * kWave + lane;
      k[j] = i < count ? keys[i] : 0;
      m[j] = kTied && i < count ? marks[i] : 0;
      if (i < count) differ |= (unsigned)(k[j] >> 32) ^ (unsigned)__builtin_amdgcn_readfirstlane((int)(k[0] >> 32));
    }
    for (int d = 1; d < kWave; d <<= 1) differ |= __shfl_xor(differ, d, kWave);
    auto reach = [&](u64 t) {
      int n = 0;
#pragma unroll
      for (int j = 0; j < kRoom / kWave; ++j) n += __popcll(__ballot(k[j] >= t));
      return n;
    };
    // (from the first bit that differs on)
    int bit = differ ? 63 - __clz(differ) : 31;
    u64 t = read_lane(k[0], 0) & ~((2ull << bit) - 1);
    int n = count;
    for (; bit >= 0 && n != most; --bit) {
      const u64 higher = t | 1ull << bit;
      const int there = reach(higher);
      if (there >= most) { t = higher; n = there; }
    }
    int last = 1 << 16;                              // of the ties at t: those with lower marks stay
    if constexpr (kTied)
      if (n != most) {
        const int above = reach(t + 1);
        int low = 0;                                 // the largest number that at most (most - above) marks lie below
        for (int bit = 15; bit >= 0; --bit) {
          int below = 0;
#pragma unroll
          for (int j = 0; j < kRoom / kWave; ++j) below += __popcll(__ballot(k[j] == t && m[j] < (low | 1 << bit)));
          if (below <= most - above) low |= 1 << bit;
        }
        last = low;
      }
    lds_sync();
    count = 0;
#pragma unroll
    for (int j = 0; j < kRoom / kWave; ++j) {
      const bool stays = k[j] > t || (k[j] == t && t && (!kTied || m[j] < last));
      const u64 who = __ballot(stays);
      if (stays) {
        const int at = count + __builtin_amdgcn_mbcnt_hi((unsigned)(who >> 32), __builtin_amdgcn_mbcnt_lo((unsigned)who, 0));
        keys[at] = k[j];
        if constexpr (kTied) marks[at] = (unsigned short)m[j];
      }
      count += __popcll(who);
    }
    least = t;
    lds_sync();
  }
  // the lane's key, mark and place among up to 64
  __device__ inline void rank(u64 &key, int &mark, int &place)
  {
    lds_sync();
    const int lane = threadIdx.x & 63;
    key = lane < count ? keys[lane] : 0;
    mark = kTied && lane < count ? marks[lane] : 0;
    place = 0;
    for (int i = 0; i < count; ++i) {
      const u64 other = read_lane(key, i);
      place += other > key || (kTied && other == key && __builtin_amdgcn_readlane(mark, i) < mark);
    }
    if (lane >= count) place = lane;
  }
};

struct Shared {
  Exponentials exponentials;
  u64 keys[kWaves][kRoom];
  unsigned short marks[kWaves][kRoom];
  int counts[kWaves];
  double sums[kWaves], tops[kWaves];
  int arrived;
};

__device__ inline bool last_to_arrive(int *counter, int n, int &arrived)
{
  // (what the others have stored goes past the L2 of the die both ways, so that the stores being done is all it takes)
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

// The waves' lists as one, in wave 0, cut to the best; the other waves' are gone.  All threads call it.
template <bool kTied> __device__ inline void join_waves(Shared &s, Candidates<kTied> &mine)
{
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
  if (mine.count > kWave) mine.cut();
  if (lane == 0) s.counts[wave] = mine.count;
  __syncthreads();
  if (wave == 0) {
    for (int w = 1; w < kWaves; ++w) {
      const bool there = lane < s.counts[w];
      mine.add(there, there ? s.keys[w][lane] : 0, kTied && there ? s.marks[w][lane] : 0);
    }
    if (mine.count > kWave) mine.cut();              // (up to 64 are ranked as they are)
  }
}

template <int DTYPE> struct Logits;
template <> struct Logits<LESSDEC_DTYPE_F32> {
  typedef float T;
  u4 a, b;
  __device__ inline void load(const T *p)
  {
    a = __builtin_nontemporal_load(reinterpret_cast<const u4a4 *>(p));
    b = __builtin_nontemporal_load(reinterpret_cast<const u4a4 *>(p) + 1);
  }
  __device__ inline float get(int i) const { return __uint_as_float(i < 4 ? a[i & 3] : b[i & 3]); }
  __device__ inline void set(int i, T x) { (i < 4 ? a : b)[i & 3] = __float_as_uint(x); }
  static __device__ inline T none() { return -__builtin_inff(); }
};
template <> struct Logits<LESSDEC_DTYPE_F16> {
  typedef unsigned short T;
  u4 a;
  __device__ inline void load(const T *p) { a = __builtin_nontemporal_load(reinterpret_cast<const u4a2 *>(p)); }
  __device__ inline float get(int i) const { return __half2float(__ushort_as_half((unsigned short)(a[i / 2] >> (i % 2 * 16)))); }
  __device__ inline void set(int i, T x) { a[i / 2] = i % 2 ? (a[i / 2] & 0xffffu) | (unsigned)x << 16 : (a[i / 2] & 0xffff0000u) | x; }
  static __device__ inline T none() { return 0xfc00; }
};
template <> struct Logits<LESSDEC_DTYPE_BF16> {
  typedef unsigned short T;
  u4 a;
  __device__ inline void load(const T *p) { a = __builtin_nontemporal_load(reinterpret_cast<const u4a2 *>(p)); }
  __device__ inline float get(int i) const { return __uint_as_float(i % 2 ? a[i / 2] & 0xffff0000u : a[i / 2] << 16); }
  __device__ inline void set(int i, T x) { a[i / 2] = i % 2 ? (a[i / 2] & 0xffffu) | (unsigned)x << 16 : (a[i / 2] & 0xffff0000u) | x; }
  static __device__ inline T none() { return 0xff80; }
};

__device__ inline double lane_sum(double x)
{
  for (int d = 1; d < kWave; d <<= 1) x += __shfl_xor(x, d, kWave);
  return x;
}
__device__ inline float lane_max(float x)
{
  for (int d = 1; d < kWave; d <<= 1) x = fmaxf(x, __shfl_xor(x, d, kWave));
  return x;
}

// A part of a row: the sum of e^{x - m} and the row's best candidates there, to the workspace.
template <int DTYPE> __device__ inline void scan_part(const BeamArgs &a, int row, int part, Shared &s)
{
  typedef Logits<DTYPE> L;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63;
  const typename L::T *x = static_cast<const typename L::T *>(a.logits) + row * a.stride;
  const int from = part * a.per, to = min(a.vocab, from + a.per);
  auto load = [&](L &l, int v) {                     // the lane's eight from v on
    if (v + kEach <= to) {
      l.load(x + v);
    } else {
#pragma unroll
      for (int i = 0; i < kEach; ++i) {
        typename L::T y = L::none();
        if (v + i < to) y = x[v + i];
        l.set(i, y);
      }
    }
  };
  Candidates<false> best;
  best.start(s.keys[wave], nullptr, a.picks);
  float limit = -__builtin_inff(), m = 0;            // the K-th largest so far, or less; what exponents are relative to
  float seen = -__builtin_inff();                    // the lane's largest
  int tile = 0, look = 0;
  double sum = 0;
  bool bad = false, any = false;                     // (any: a logit above -inf; until then m means nothing and the sum is 0)
  // m is 0 unless a logit lies beyond kFar, or all so far below -kFar; a mask of finite values is left behind with the first tile that has others
  auto reference = [&](float now) {
    now = fabsf(now) > kFar && fabsf(now) < __builtin_inff() ? now : 0.f;              // (not finite: the row has no sum, `bad`)
    if (sum != 0) sum *= exp((double)m - now);
    m = now;
  };
  auto work = [&](const L &l, int v) {
    float y[kEach];
#pragma unroll
    for (int i = 0; i < kEach; ++i) y[i] = l.get(i);
    bool more = false;
#pragma unroll
    for (int i = 0; i < kEach; ++i) more |= !(y[i] <= limit);
    if (__ballot(more)) {
      float top = y[0];
#pragma unroll
      for (int i = 1; i < kEach; ++i) top = fmaxf(top, y[i]);
      seen = fmaxf(seen, top);
      if (!any && __ballot(top >= -kFar) == 0) reference(lane_max(top));
      any = true;
      if (__ballot(top > m + kFar)) reference(lane_max(top));
      if (tile >= look) {
        // the K-th largest of the lanes' largest is reached by K logits at least: asked for after 1, 2, 4, .. tiles
        look = 2 * tile + 1;
        const unsigned k = (unsigned)(key_of(seen, 0) >> 32);
        unsigned t = 0;
        for (int bit = 31; bit >= 0; --bit)
          if (__popcll(__ballot(k >= (t | 1u << bit))) >= a.picks) t |= 1u << bit;
        // just below, which of 0 is not the -0 that comes before it in these numbers; -inf at least
        limit = fmaxf(limit, logit_of((u64)(t > 0x007fffffu ? t - 1 - (t == 0x80000000u) : 0x007fffffu) << 32));
      }
#pragma unroll
      for (int i = 0; i < kEach; ++i) {
        const bool wanted = !(y[i] <= limit);
        if (!__ballot(wanted)) continue;
        bad |= wanted && !(y[i] < __builtin_inff());                   // NaN or infinite
        const u64 key = key_of(y[i], v + i);
        best.add(wanted && key >= best.least, key, 0);
      }
      // (only now, as tokens of a tile do not come in order; those of later tiles lose a tie)
      if (best.least > 1) limit = fmaxf(limit, logit_of(best.least));
    }
    if (!any) return;
    if (m == 0.f) {
#pragma unroll
      for (int i = 0; i < kEach; ++i) sum += s.exponentials.of(__builtin_amdgcn_fmed3f(y[i], -kLeast, kFar));
    } else {
      // (differences need not be fp32's; they are 256 at most, as m + kFar is rounded.  Half of 128256 logits masked by -1e4: 55 us, 71 by the library's
      // exponential, with all eight at once 52, but 46 in place of 45 where nothing is masked)
#pragma unroll 2
      for (int i = 0; i < kEach; ++i) sum += s.exponentials.of(fmax((double)y[i] - m, (double)-kLeast));
    }
  };
  const int step = kWaves * kBeamTile;
  int v = from + wave * kBeamTile;
  L now, next;
  if (v < to) load(now, v + lane * kEach);
  for (; v < to; v += step) {
    if (v + step < to) load(next, v + step + lane * kEach);
    work(now, v + lane * kEach);
    ++tile;
    now = next;
  }
  sum = lane_sum(sum);
  if (__ballot(bad)) sum = __builtin_nan("");
  if (lane == 0) { s.sums[wave] = sum; s.tops[wave] = any ? m : -__builtin_inf(); }
  join_waves(s, best);
  if (wave) return;
  u64 key;
  int mark, place;
  best.rank(key, mark, place);
  const long at = (long)row * a.parts + part;
  if (place < a.picks) put(a.lists + at * a.picks + place, key);
  if (lane == 0) {
    double top = s.tops[0], total = 0;
    for (int w = 1; w < kWaves; ++w) top = fmax(top, s.tops[w]);
    for (int w = 0; w < kWaves; ++w)
      if (s.tops[w] > -__builtin_inf()) total += s.sums[w] * exp(s.tops[w] - top);
    put(a.sums + 2 * at, __double_as_longlong(top));
    put(a.sums + 2 * at + 1, __double_as_longlong(total));
  }
}

// A row's candidates, from its parts: c and token, the best first.
__device__ inline void join_parts(const BeamArgs &a, int row, bool ended, Shared &s)
{
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
  u64 *scores = a.scores + (long)row * a.picks;
  int *tokens = a.tokens + (long)row * a.picks;
  const double score = a.score[row];
  if (ended) {
    if (threadIdx.x < a.picks) {
      put(scores + threadIdx.x, threadIdx.x == 0 ? key_of(score) : 0);
      __hip_atomic_store(tokens + threadIdx.x, a.end_token, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    }
    return;
  }
  const u64 *sums = a.sums + 2 * (long)row * a.parts;
  const u64 m_of = get(sums + 2 * min(lane, a.parts - 1)), part_of = get(sums + 2 * min(lane, a.parts - 1) + 1);
  const u64 *lists = a.lists + (long)row * a.parts * a.picks;
  const int n = a.parts * a.picks;
  Candidates<false> best;
  best.start(s.keys[wave], nullptr, a.picks);
  for (int base = 0; base < n; base += kThreads) {
    const int i = base + threadIdx.x;
    const u64 key = i < n ? get(lists + i) : 0;
    best.add(key >= best.least, key, 0);
  }
  join_waves(s, best);
  if (wave) return;
  const double m = lane < a.parts ? __longlong_as_double(m_of) : -__builtin_inf(), part = lane < a.parts ? __longlong_as_double(part_of) : 0;
  double top = m;
  for (int d = 1; d < kWave; d <<= 1) top = fmax(top, __shfl_xor(top, d, kWave));
  const double log_sum = log(lane_sum(lane < a.parts ? part * exp(m - top) : 0)), lse = top + log_sum;
  const bool far = fabs(top) > 65536;                // where lse would lose log_sum (fp16 does not come so far)
  u64 key;
  int mark, place;
  best.rank(key, mark, place);
  if (place < a.picks) {
    put(scores + place, key ? key_of(score + (far ? (logit_of(key) - top) - log_sum : logit_of(key) - lse)) : 0);
    __hip_atomic_store(tokens + place, token_of(key), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  }
}

// A prompt's picks, from its rows' candidates.
__device__ inline void join_rows(const BeamArgs &a, int group, Shared &s)
{
  const int wave = threadIdx.x >> 6;
  const long first = (long)group * a.beams * a.picks;
  const int n = a.beams * a.picks;
  Candidates<true> best;
  best.start(s.keys[wave], s.marks[wave], a.picks);
  for (int base = 0; base < n; base += kThreads) {
    const int i = base + threadIdx.x;
    const u64 key = i < n ? get(a.scores + first + i) : 0;
    best.add(key >= best.least, key, i);
  }
  join_waves(s, best);
  if (wave) return;
  u64 key;
  int mark, place;
  best.rank(key, mark, place);
  if (place >= a.picks) return;
  const long to = (long)group * a.picks + place;
  const int token = key ? __hip_atomic_load(a.tokens + first + mark, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) : -1;
  a.parent[to] = key ? group * a.beams + mark / a.picks : -1;
  a.token[to] = token;
  a.next_score[to] = key ? (float)score_of(key) : -__builtin_inff();
  if (a.next_ended) a.next_ended[to] = key && token == a.end_token;
}

template <int DTYPE> __global__ __launch_bounds__(kThreads, 5) void beam_kernel(BeamArgs a)
{
  __shared__ Shared s;
  const int row = blockIdx.x / (unsigned)a.parts, part = blockIdx.x % (unsigned)a.parts, group = row / a.beams;
  const bool ended = a.ended && a.ended[row];
  if (!ended) {
    s.exponentials.fill();
    __syncthreads();
    scan_part<DTYPE>(a, row, part, s);
  }
  if (!last_to_arrive(a.counters + row, a.parts, s.arrived)) return;
  join_parts(a, row, ended, s);
  if (!last_to_arrive(a.counters + (long)a.groups * a.beams + group, a.beams, s.arrived)) return;
  join_rows(a, group, s);
}

}  // namespace

hipError_t launch_beam_select(const BeamArgs &a, int dtype, hipStream_t st)
{
  const unsigned grid = (unsigned)((long)a.groups * a.beams * a.parts);
  if (dtype == LESSDEC_DTYPE_F32) beam_kernel<LESSDEC_DTYPE_F32><<<grid, kThreads, 0, st>>>(a);
  else if (dtype == LESSDEC_DTYPE_F16) beam_kernel<LESSDEC_DTYPE_F16><<<grid, kThreads, 0, st>>>(a);
  else beam_kernel<LESSDEC_DTYPE_BF16><<<grid, kThreads, 0, st>>>(a);
  return hipGetLastError();
}

}  // namespace lessdec
