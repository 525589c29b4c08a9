// Paged cache: keys and values into the cache (append) and back out of it (read).
//
// Both are bound by memory: a token of a head is 2 D elements of two bytes on one side and 2 D bytes on the other.  A wave has one
// block of 16 tokens of one head, keys and values, so that the block's exponents are the wave's own reduction, nothing is
// shared and no wave waits for another.  Eight lanes have a line of 128 bytes of a token's row, so that rows are read and written by whole
// lines, past the caches; the values are turned into the cache's order in the LDS.  32 heads, D = 128, bf16: 15581 tokens of 16 prompts in,
// 383 MB, 78 us (4.9 TB/s); 16 times 2049 out, 806 MB, 128 us (6.3 TB/s).  Four lanes to a line took 253 us for both, not 209, and
// non-temporal access by less than a line 447.  A token a slot is a chain of latencies: 5.3 us in, 4.0 out.
#include "lessdec_pages.h"

namespace lessdec {
namespace {

constexpr int kTop = 40;                             // exponents lie within +-kTop

// Raw 16-bit elements as fp32.
template <bool BF16> __device__ inline float element(unsigned short x)
{
  if constexpr (BF16) return __uint_as_float((unsigned)x << 16);
  else return __half2float(__ushort_as_half(x));
}
template <bool BF16> __device__ inline unsigned short rounded(float x)
{
  if constexpr (BF16) {
    const unsigned b = __float_as_uint(x);
    if ((b & 0x7fffffffu) > 0x7f800000u) return 0x7fc0;
    return (unsigned short)((b + 0x7fffu + (b >> 16 & 1)) >> 16);
  } else {
    return __half_as_ushort(__float2half_rn(x));
  }
}

__device__ inline unsigned magnitude(float x)        // bits of |x|, 0 where x is not finite
{
  const unsigned b = __float_as_uint(x) & 0x7fffffffu;
  return b < 0x7f800000u ? b : 0;
}

// The least e with x <= 448 * 2^e = 1.75 * 2^(e + 8), within +-kTop; x by its bits.
__device__ inline int exponent_of(unsigned bits)
{
  const int e = (int)(bits >> 23) - 127 - 8 + ((bits & 0x7fffffu) > 0x600000u);
  return e < -kTop ? -kTop : e < kTop ? e : kTop;
}

__device__ inline unsigned wave_max(unsigned x)
{
#pragma unroll
  for (int d = 1; d < kWave; d <<= 1) {
    const unsigned y = __shfl_xor(x, d, kWave);
    x = y > x ? y : x;
  }
  return x;
}

// x / 2^e for the conversion: at most 448 (more only at e = kTop), NaN where x is not finite
__device__ inline float scaled(float x, float inverse)
{
  const float y = fminf(fmaxf(x * inverse, -448.f), 448.f);
  return magnitude(x) || x == 0.f ? y : __builtin_nanf("");
}
__device__ inline unsigned four_codes(float a, float b, float c, float d)
{
  int w = __builtin_amdgcn_cvt_pk_fp8_f32(a, b, 0, false);
  return (unsigned)__builtin_amdgcn_cvt_pk_fp8_f32(c, d, w, true);
}
typedef unsigned short us2 __attribute__((ext_vector_type(2)));
typedef short s2 __attribute__((ext_vector_type(2)));
// codes of four elements over a power of two, none of them beyond 448 times it
template <bool BF16> __device__ inline unsigned four_codes(unsigned a, unsigned b, float scale)
{
  s2 w = {0, 0};
  if constexpr (BF16) {
    typedef __bf16 v2 __attribute__((ext_vector_type(2)));
    w = __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(w, __builtin_bit_cast(v2, a), scale, false);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp8_bf16(w, __builtin_bit_cast(v2, b), scale, true);
  } else {
    typedef _Float16 v2 __attribute__((ext_vector_type(2)));
    w = __builtin_amdgcn_cvt_scalef32_pk_fp8_f16(w, __builtin_bit_cast(v2, a), scale, false);
    w = __builtin_amdgcn_cvt_scalef32_pk_fp8_f16(w, __builtin_bit_cast(v2, b), scale, true);
  }
  return __builtin_bit_cast(unsigned, w);
}
// four codes, rounded again for an exponent that is larger by shift (factor = 2^-shift)
__device__ inline unsigned again(unsigned w, float factor)
{
  const auto a = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, false), b = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, true);
  return four_codes(a[0] * factor, a[1] * factor, b[0] * factor, b[1] * factor);
}

// whole lines of rows that are read, or written, once
typedef unsigned u4 __attribute__((ext_vector_type(4)));
__device__ inline uint4 load_once(const uint4 *p) { return __builtin_bit_cast(uint4, __builtin_nontemporal_load(reinterpret_cast<const u4 *>(p))); }
__device__ inline void store_once(uint4 *p, uint4 x) { __builtin_nontemporal_store(__builtin_bit_cast(u4, x), reinterpret_cast<u4 *>(p)); }

constexpr int kRowPad = 16;                          // bytes behind a token's codes in the LDS: the four tokens of a group in other banks

// Block b of a slot's new tokens: the wave's index less start[s] / 16 + 2 s, which leaves every slot as many waves as it can
// touch blocks (count / 16 + 2) without a prefix sum over the slots.
template <bool BF16, int D>
__global__ __launch_bounds__(256) void append_kernel(Pages c, AppendArgs a)
{
  constexpr int H = D / 64;
  __shared__ __align__(16) unsigned char turned[4][kBlock * (D + kRowPad)];
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, head = blockIdx.y;
  const long w = (long)blockIdx.x * 4 + wave;
  auto base = [&](int s) {
    const int f = a.start[s];
    return (long)((f < 0 ? 0 : f < a.rows ? f : a.rows) / kBlock) + 2 * (long)s;
  };
  const int s = last_slot_at(c.slots, w, base);
  const Rows r = slot_rows(a.start, s, a.rows);
  const int len = slot_length(c, s), begin = len > r.count ? len - r.count : 0;
  const int row0 = r.first + r.count - (len - begin);                  // row of the token at position begin
  const long nth = w - base(s), b = begin / kBlock + nth;              // (below 0: a wave before the first slot's rows)
  if (r.count == 0 || nth < 0 || b * kBlock >= len) return;
  const int t0 = (int)b * kBlock;
  const int page = c.table[(size_t)s * c.table_len + entry_of(c, (int)b)];           // (on its way beside the rows)
  const int off = begin > t0 ? begin - t0 : 0;                         // older tokens of the block

  // A lane has eight channels of two tokens (of every 64 channels), eight lanes a line of a token's row; of the cache a piece of 16 bytes of
  // every half block: of the values four channels of four tokens.
  const int piece = lane & 7, g = lane >> 4;
  int tok[2];
  bool fresh[2];
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    tok[i] = (lane >> 3) + 8 * i;
    fresh[i] = tok[i] >= off && t0 + tok[i] < len;
  }
  uint4 x[2][H][2];
#pragma unroll
  for (int which = 0; which < 2; ++which)
#pragma unroll
    for (int h = 0; h < H; ++h)
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        x[which][h][i] = make_uint4(0, 0, 0, 0);
        if (fresh[i])
          x[which][h][i] = load_once(reinterpret_cast<const uint4 *>(which ? a.v : a.k) + (long)(row0 + t0 + tok[i] - begin) * (a.stride / 8) + head * (D / 8) + h * 8 + piece);
      }
  const int block = block_in(c, page, head, (int)b);
  if (block < 0) return;
  unsigned short *exps = reinterpret_cast<unsigned short *>(c.exps) + block;
  unsigned char *kb = c.k + block * ((long)kBlock * D);
  uint4 *vb = reinterpret_cast<uint4 *>(c.v + block * ((long)kBlock * D)) + lane;
  auto key_at = [&](int h, int i) { return reinterpret_cast<uint2 *>(kb + h * 1024 + ((piece >> 1) * 16 + tok[i]) * 16 + (piece & 1) * 8); };
  uint4 old[H];
  const bool mixed = off > 0 && 4 * g + 3 >= off && t0 + 4 * g < len;  // the lane's four tokens of a value piece are not all older
#pragma unroll
  for (int h = 0; h < H; ++h) {
    old[h] = make_uint4(0, 0, 0, 0);
    if (mixed) old[h] = vb[h * kWave];
  }
  const unsigned was = off > 0 ? *exps : 0;

  // The largest magnitude, on the elements' bits, two at a time; where one is not finite, once more without those.
  constexpr unsigned kInf = BF16 ? 0x7f80u : 0x7c00u;
  int e[2], shift[2];
  bool odd[2];                                       // a block with elements that are not finite, or beyond the largest exponent
#pragma unroll
  for (int which = 0; which < 2; ++which) {
    us2 most = {0, 0};
#pragma unroll
    for (int h = 0; h < H; ++h)
#pragma unroll
      for (int i = 0; i < 8; ++i)
        most = __builtin_elementwise_max(most, __builtin_bit_cast(us2, (&x[which][h][i / 4].x)[i % 4] & 0x7fff7fffu));
    unsigned m = wave_max(most[0] > most[1] ? most[0] : most[1]);
    odd[which] = m >= kInf;
    if (odd[which]) {
      m = 0;
#pragma unroll
      for (int h = 0; h < H; ++h)
#pragma unroll
        for (int i = 0; i < 16; ++i) {
          const unsigned y = (&x[which][h][i / 8].x)[i / 2 % 4] >> 16 * (i % 2) & 0x7fffu;
          m = y < kInf && y > m ? y : m;
        }
      m = wave_max(m);
    }
    e[which] = exponent_of(__float_as_uint(element<BF16>((unsigned short)m)));
    odd[which] |= e[which] == kTop;
    shift[which] = 0;
    if (off > 0) {
      int before = (signed char)(which ? was >> 8 : was);
      before = before < -kTop ? -kTop : before < kTop ? before : kTop;
      if (e[which] > before) shift[which] = e[which] - before;
      else e[which] = before;
    }
  }
  if (lane == 0) *exps = (unsigned short)((e[0] & 255) | (e[1] & 255) << 8);

  // codes of the lane's eight channels of a token
  uint2 code[2][H][2];
#pragma unroll
  for (int which = 0; which < 2; ++which) {
    const float scale = pow2(e[which]), inverse = pow2(-e[which]);
#pragma unroll
    for (int h = 0; h < H; ++h)
#pragma unroll
      for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          const unsigned p = (&x[which][h][i].x)[2 * j], q = (&x[which][h][i].x)[2 * j + 1];
          unsigned &w = (&code[which][h][i].x)[j];
          if (!odd[which])
            w = four_codes<BF16>(p, q, scale);
          else
            w = four_codes(scaled(element<BF16>((unsigned short)p), inverse), scaled(element<BF16>((unsigned short)(p >> 16)), inverse),
                           scaled(element<BF16>((unsigned short)q), inverse), scaled(element<BF16>((unsigned short)(q >> 16)), inverse));
        }
  }

#pragma unroll
  for (int i = 0; i < 2; ++i) {
    if (fresh[i] || off == 0) {                                        // (the rest of a new block: zeros)
#pragma unroll
      for (int h = 0; h < H; ++h) *key_at(h, i) = code[0][h][i];
    } else if (shift[0] && tok[i] < off) {
      const float factor = pow2(-shift[0]);
#pragma unroll
      for (int h = 0; h < H; ++h) {
        const uint2 k = *key_at(h, i);
        *key_at(h, i) = make_uint2(again(k.x, factor), again(k.y, factor));
      }
    }
  }

  // the values' codes are turned in the LDS
  unsigned char *mine = turned[wave];
#pragma unroll
  for (int h = 0; h < H; ++h)
#pragma unroll
    for (int i = 0; i < 2; ++i) *reinterpret_cast<uint2 *>(mine + tok[i] * (D + kRowPad) + h * 64 + piece * 8) = code[1][h][i];
  wave_lds_sync();
  const bool rescale = off > 0 && shift[1] > 0;
  if (off == 0 || mixed || rescale) {
    const float factor = pow2(-shift[1]);
    unsigned keep = 0;                                                 // bytes of tokens that are not new
#pragma unroll
    for (int j = 0; j < 4; ++j)
      if (4 * g + j < off || (off > 0 && t0 + 4 * g + j >= len)) keep |= 255u << 8 * j;
#pragma unroll
    for (int h = 0; h < H; ++h) {
      if (rescale && !mixed) old[h] = vb[h * kWave];
      uint4 v;
#pragma unroll
      for (int t = 0; t < 4; ++t) {
        unsigned word = 0;
#pragma unroll
        for (int j = 0; j < 4; ++j)
          word |= (unsigned)mine[(4 * g + j) * (D + kRowPad) + h * 64 + t * 16 + (lane & 15)] << 8 * j;
        unsigned before = (&old[h].x)[t];
        if (rescale) before = again(before, factor);
        (&v.x)[t] = (word & ~keep) | (before & keep);
      }
      vb[h * kWave] = v;
    }
  }
}

// A wave has a block of the cache and writes those of its tokens that are asked for.
template <bool BF16, int D>
__global__ __launch_bounds__(256) void read_kernel(Pages c, ReadArgs a)
{
  constexpr int H = D / 64;
  __shared__ __align__(16) unsigned char turned[4][kBlock * (D + kRowPad)];
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, head = blockIdx.y, i = blockIdx.z;
  const int s = a.slots[i];
  const bool there = (unsigned)s < (unsigned)c.slots;
  const int len = there ? slot_length(c, s) : 0;
  const long first = a.first >= 0 ? a.first : (long)len + a.first;
  const long b = (first >> 4) + (long)blockIdx.x * 4 + wave;           // (floor: first may be negative)
  if (b * kBlock >= first + a.count) return;
  const long t0 = b * kBlock;
  const int block = t0 >= 0 && t0 < len ? block_index(c, s, head, (int)b) : -1;
  // of the cache and of the rows a lane has what it has when they are stored
  const int piece = lane & 7, g = lane >> 4;
  uint2 k[H][2], v[H][2];
  uint4 turn[H];
  unsigned e = 0;
#pragma unroll
  for (int h = 0; h < H; ++h) {
    turn[h] = make_uint4(0, 0, 0, 0);
    k[h][0] = k[h][1] = make_uint2(0, 0);
  }
  if (block >= 0) {
    e = reinterpret_cast<const unsigned short *>(c.exps)[block];
    const unsigned char *kb = c.k + block * ((long)kBlock * D);
#pragma unroll
    for (int h = 0; h < H; ++h) {
#pragma unroll
      for (int i = 0; i < 2; ++i)
        k[h][i] = *reinterpret_cast<const uint2 *>(kb + h * 1024 + ((piece >> 1) * 16 + (lane >> 3) + 8 * i) * 16 + (piece & 1) * 8);
      turn[h] = reinterpret_cast<const uint4 *>(c.v + block * ((long)kBlock * D))[h * kWave + lane];
    }
  }
  unsigned char *mine = turned[wave];
#pragma unroll
  for (int h = 0; h < H; ++h)
#pragma unroll
    for (int t = 0; t < 4; ++t)
#pragma unroll
      for (int j = 0; j < 4; ++j)
        mine[(4 * g + j) * (D + kRowPad) + h * 64 + t * 16 + (lane & 15)] = (unsigned char)((&turn[h].x)[t] >> 8 * j);
  wave_lds_sync();
  const float most = BF16 ? __uint_as_float(0x7f7f0000u) : 65504.f;
#pragma unroll
  for (int half = 0; half < 2; ++half) {
    const int tok = (lane >> 3) + 8 * half;
    const long at = t0 + tok - first;
    if (at < 0 || at >= a.count) continue;
    const bool held = block >= 0 && t0 + tok < len;
    const long row = (((long)i * c.heads + head) * a.count + at) * (D / 8);
#pragma unroll
    for (int h = 0; h < H; ++h) v[h][half] = *reinterpret_cast<const uint2 *>(mine + tok * (D + kRowPad) + h * 64 + piece * 8);
#pragma unroll
    for (int which = 0; which < 2; ++which) {
      int ex = (signed char)(which ? e >> 8 : e);
      ex = ex < -kTop ? -kTop : ex < kTop ? ex : kTop;
      const float scale = pow2(ex);
#pragma unroll
      for (int h = 0; h < H; ++h) {
        uint4 out;
#pragma unroll
        for (int n = 0; n < 4; ++n) {
          const uint2 &x = which ? v[h][half] : k[h][half];
          const unsigned word = (&x.x)[n / 2];
          const auto p = n % 2 ? __builtin_amdgcn_cvt_pk_f32_fp8((int)word, true) : __builtin_amdgcn_cvt_pk_f32_fp8((int)word, false);
          unsigned pair = 0;
#pragma unroll
          for (int j = 0; j < 2; ++j) {
            float y = held ? p[j] * scale : 0.f;
            y = y > most ? most : y < -most ? -most : y;               // (NaN stays)
            pair |= (unsigned)rounded<BF16>(y) << 16 * j;
          }
          (&out.x)[n] = pair;
        }
        store_once(reinterpret_cast<uint4 *>(which ? a.v : a.k) + row + h * 8 + piece, out);
      }
    }
  }
}

}  // namespace

hipError_t launch_pages_append(const Pages &c, int dtype, const AppendArgs &a, hipStream_t st)
{
  const long waves = a.rows / kBlock + 2 * (long)c.slots;
  const dim3 grid((unsigned)((waves + 3) / 4), (unsigned)c.heads);
  const bool bf16 = dtype == LESSDEC_DTYPE_BF16;
  if (c.head_dim == 128) bf16 ? append_kernel<true, 128><<<grid, 256, 0, st>>>(c, a) : append_kernel<false, 128><<<grid, 256, 0, st>>>(c, a);
  else bf16 ? append_kernel<true, 64><<<grid, 256, 0, st>>>(c, a) : append_kernel<false, 64><<<grid, 256, 0, st>>>(c, a);
  return hipGetLastError();
}

hipError_t launch_pages_read(const Pages &c, int dtype, const ReadArgs &a, hipStream_t st)
{
  const long blocks = a.count / kBlock + 2;
  const dim3 grid((unsigned)((blocks + 3) / 4), (unsigned)c.heads, (unsigned)a.n);
  const bool bf16 = dtype == LESSDEC_DTYPE_BF16;
  if (c.head_dim == 128) bf16 ? read_kernel<true, 128><<<grid, 256, 0, st>>>(c, a) : read_kernel<false, 128><<<grid, 256, 0, st>>>(c, a);
  else bf16 ? read_kernel<true, 64><<<grid, 256, 0, st>>>(c, a) : read_kernel<false, 64><<<grid, 256, 0, st>>>(c, a);
  return hipGetLastError();
}

}  // namespace lessdec
