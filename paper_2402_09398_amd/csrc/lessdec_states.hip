// Compressed states that follow their sequences: batch row b of all state arrays becomes what row from[b] was, in place.
//
// Bound by memory: every row that another one gets is read once, every row that changes is written once.  As rows may be read
// and written at once (beams whose parents are each other), a workgroup takes some columns of an array in all of the rows that are
// read, brings them into the LDS, and only then writes: no order of rows, no second copy of the state, one launch.  Which rows are read, and
// which change, every workgroup works out for itself from the 4 bytes a row of from.
//
// Measured: 32 rows of 40 heads, 408 tokens: 86 us (4.7 TB/s of bytes read and written; a large copy reaches 4.95); 64 rows of 32 heads, 102 tokens:
// 32.5 (4.3); 8 of them: 10.5, the latency of the lists, the reads and the writes.
#include "lessdec_common.h"
#include "lessdec_internal.h"

namespace lessdec {
namespace {

typedef unsigned u4 __attribute__((ext_vector_type(4)));

constexpr int kThreads = 256, kMost = LESSDEC_MAX_SLOTS, kInFlight = 8;

// LDS: columns of the rows that are read, then for every row of the batch the place of the row that it gets (-1: none, it becomes
// empty), then the rows that change, then those that are read.
struct Lists {
  short *place, *change, *read;
  int changes, reads;
};

// at: places of the set flags in ascending order of the rows, of which a thread has neighbours; returns how many are set
__device__ inline int scan_flags(int *counts, const bool (&flags)[kMost / kThreads], int (&at)[kMost / kThreads])
{
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  int mine = 0;
#pragma unroll
  for (int t = 0; t < kMost / kThreads; ++t) mine += flags[t];
  int upto = mine;
  for (int d = 1; d < kWave; d <<= 1) {
    const int y = __shfl_up(upto, d, kWave);
    if (lane >= d) upto += y;
  }
  __syncthreads();
  if (lane == 63) counts[wave] = upto;
  __syncthreads();
  int before = upto - mine, total = 0;
  for (int w = 0; w < kThreads / kWave; ++w) {
    if (w < wave) before += counts[w];
    total += counts[w];
  }
#pragma unroll
  for (int t = 0; t < kMost / kThreads; ++t) {
    at[t] = before;
    before += flags[t];
  }
  return total;
}

template <typename T>
__device__ inline void move_columns(const SelectArray &a, const Lists &l, long column, int shift, T *staged)
{
  // 1 << shift pieces of T of a row, from byte `column` on
  const int per = 1 << shift, mask = per - 1;
  const long left = (a.row_bytes - column) / (long)sizeof(T);
  const int pieces = l.reads << shift;
  for (int base = 0; base < pieces; base += kThreads * kInFlight) {
    T x[kInFlight];
#pragma unroll
    for (int i = 0; i < kInFlight; ++i) {
      const int at = base + i * kThreads + threadIdx.x, c = at & mask;
      if (at < pieces && c < left)
        x[i] = __builtin_nontemporal_load(reinterpret_cast<const T *>(a.p + l.read[at >> shift] * a.row_bytes + column) + c);
    }
#pragma unroll
    for (int i = 0; i < kInFlight; ++i) {
      const int at = base + i * kThreads + threadIdx.x;
      if (at < pieces) staged[at] = x[i];
    }
  }
  __syncthreads();
  const int stores = l.changes << shift;
  for (int at = threadIdx.x; at < stores; at += kThreads) {
    const int row = l.change[at >> shift], c = at & mask, from = l.place[row];
    if (c >= left || (from < 0 && !a.emptied)) continue;
    T x;
    if (from >= 0) x = staged[(from << shift) + c];
    else if constexpr (sizeof(T) == 16) x = T{a.empty, a.empty, a.empty, a.empty};
    else x = a.empty;
    __builtin_nontemporal_store(x, reinterpret_cast<T *>(a.p + row * a.row_bytes + column) + c);
  }
  __syncthreads();
}

__global__ __launch_bounds__(kThreads) void state_select_kernel(SelectArgs s, int staged_bytes)
{
  extern __shared__ __align__(16) unsigned char shared[];
  __shared__ int counts[kThreads / kWave];
  const int B = s.batch, turns = (B + kThreads - 1) / kThreads;
  Lists l;
  l.place = reinterpret_cast<short *>(shared + staged_bytes);
  l.change = l.place + B;
  l.read = l.change + B;
  // a thread has the rows [tid turns, tid turns + turns)
  for (int b = threadIdx.x; b < B; b += kThreads) l.read[b] = 0;
  __syncthreads();
  bool flags[kMost / kThreads];
  int at[kMost / kThreads], from[kMost / kThreads];
#pragma unroll
  for (int t = 0; t < kMost / kThreads; ++t) {
    const int b = threadIdx.x * turns + t;
    flags[t] = false;
    if (t >= turns || b >= B) continue;
    const int f = s.from[b];
    from[t] = f < -1 || f >= B ? b : f;
    flags[t] = from[t] != b;
    if (flags[t] && from[t] >= 0) l.read[from[t]] = 1;
  }
  l.changes = scan_flags(counts, flags, at);
#pragma unroll
  for (int t = 0; t < kMost / kThreads; ++t)
    if (flags[t]) l.change[at[t]] = (short)(threadIdx.x * turns + t);
  bool is_read[kMost / kThreads];
#pragma unroll
  for (int t = 0; t < kMost / kThreads; ++t) {
    const int b = threadIdx.x * turns + t;
    is_read[t] = t < turns && b < B && l.read[b] != 0;
  }
  l.reads = scan_flags(counts, is_read, at);
#pragma unroll
  for (int t = 0; t < kMost / kThreads; ++t)
    if (is_read[t]) {
      const int b = threadIdx.x * turns + t;
      l.read[at[t]] = (short)b;
      l.place[b] = (short)at[t];                     // (of a row that is read, for now)
    }
  __syncthreads();
  short places[kMost / kThreads];
#pragma unroll
  for (int t = 0; t < kMost / kThreads; ++t) places[t] = flags[t] && from[t] >= 0 ? l.place[from[t]] : (short)-1;
  __syncthreads();
#pragma unroll
  for (int t = 0; t < kMost / kThreads; ++t)
    if (flags[t]) l.place[threadIdx.x * turns + t] = places[t];
  __syncthreads();
  if (l.changes == 0) return;

  // as many columns at a time as the LDS holds of the rows that are read
  int bytes = 2048;
  while (bytes > 16 && bytes * l.reads > staged_bytes) bytes >>= 1;
  const int shift16 = __ffs(bytes) - 5;
  long tile = blockIdx.x;
#pragma unroll 1
  for (int i = 0; i < kSelectArrays; ++i) {
    const SelectArray a = s.array[i];
    const long tiles = (a.row_bytes + bytes - 1) / bytes;
    for (; tile < tiles; tile += gridDim.x) {
      if (a.wide) move_columns<u4>(a, l, tile * bytes, shift16, reinterpret_cast<u4 *>(shared));
      else move_columns<unsigned>(a, l, tile * bytes, shift16 + 2, reinterpret_cast<unsigned *>(shared));
    }
    tile -= tiles;
  }
}

}  // namespace

hipError_t launch_state_select(const SelectArgs &s, hipStream_t st)
{
  // 16 bytes of every row, at least.  Four workgroups to a compute unit; 16 KB: 86.7 us in place of 85.8 for the larger case above, 64 KB: 89.0 (15.1 in
  // place of 10.6 for the smallest).  512 workgroups 90.7, 2048 92.5 (16.7 for the smallest); 1024 bytes of a row at a time in place of 2048: 86.7 (11.3).
  const int staged = s.batch <= 2048 ? 32768 : 65536;
  const size_t lds = (size_t)staged + (size_t)s.batch * 3 * sizeof(short);
  if (lds > 65536) {
    const hipError_t e = hipFuncSetAttribute(reinterpret_cast<const void *>(state_select_kernel), hipFuncAttributeMaxDynamicSharedMemorySize, (int)lds);
    if (e != hipSuccess) return e;
  }
  state_select_kernel<<<1024, kThreads, lds, st>>>(s, staged);
  return hipGetLastError();
}

}  // namespace lessdec
