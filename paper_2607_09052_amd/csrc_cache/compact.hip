// The kept tokens of a cache moved together (cobs_compact_cache): a copy of
// rows, bound by HBM.
//
// To another cache every (destination position, K or V) is independent.  In place
// a row may land where another row still has to be read from.  With entries
// that ascend strictly and kept[j] >= first + j, a position below first + j1 is the
// source of no entry from j1 on, so a workgroup that owns a column slice of one
// (batch row, KV head) walks the entries in order, reads a batch of rows into
// registers, waits, and writes it while the next batch is read: no write meets a
// later read.
//
// Measured with weights, bf16, d 128: to another cache 32 units of up to 8192 rows, 271 MB
// read and written, in 47 us from the last-level cache and 55 from memory (4.9 TB/s, the rate
// of a large copy); in place 32 units of 8192 rows in 76 us (3.5 TB/s), 8 units in 36, bound
// by a batch's chain of loads (entry, row, barrier).
#include <algorithm>

#include "cache_device.h"

namespace cobs {

constexpr int kCompactThreads = 256;

__device__ __forceinline__ int kept_at(const CompactParams& p, int b, int h, int j) {
  return p.kept[(p.per_head ? ((int64_t)b * p.hkv + h) : (int64_t)b) * p.num_kept + j];
}

// Destination of entry j, position t, and its source; false when the entry moves nothing.
__device__ __forceinline__ bool move_of(const CompactParams& p, int b, int h, int T, int first, int j, int t,
                                        int64_t& from, int64_t& to) {
  if (t < 0 || t >= T || j >= p.dst_max - first) return false;
  from = kv_offset(p.src, b, h, t);
  to = kv_offset(p.dst, b, h, first + j);
  return from >= 0 && to >= 0;
}

// Out of place: the first `row_blocks` workgroups of a (row, KV head) move rows, one
// thread per 16 bytes of K and of V (and the row's weight); the others clear the
// weights behind the last entry, 4 a thread.
template <int CPR>
__global__ __launch_bounds__(kCompactThreads) void compact_copy_kernel(CompactParams p, int row_blocks) {
  const int h = blockIdx.y, b = blockIdx.z, es = p.kv_f32 ? 4 : 2;
  const int T = clamp_len(p.seq_lens[b], p.tmax);
  const int first = p.first ? clamp_len(p.first[b], p.dst_max) : 0;
  const int64_t u = (int64_t)b * p.hkv + h;
  if ((int)blockIdx.x >= row_blocks) {
    const int j0 = p.num_kept + ((int)blockIdx.x - row_blocks) * 4 * kCompactThreads + threadIdx.x;
    const int end = min(T, p.dst_max) - first;
    for (int j = j0; j < min(end, j0 + 4 * kCompactThreads); j += kCompactThreads)
      p.weights_out[u * p.dst_max + first + j] = 0.0f;
    return;
  }
  const int row = ((int)blockIdx.x * kCompactThreads + threadIdx.x) / CPR, ch = threadIdx.x % CPR;
  if (row >= p.num_kept) return;
  int64_t from, to;
  const bool ok = move_of(p, b, h, T, first, row, kept_at(p, b, h, row), from, to);
  if (ok) {
    const uint4 k = reinterpret_cast<const uint4*>(static_cast<const char*>(p.src.k) + from * es)[ch];
    const uint4 v = reinterpret_cast<const uint4*>(static_cast<const char*>(p.src.v) + from * es)[ch];
    reinterpret_cast<uint4*>(static_cast<char*>(const_cast<void*>(p.dst.k)) + to * es)[ch] = k;
    reinterpret_cast<uint4*>(static_cast<char*>(const_cast<void*>(p.dst.v)) + to * es)[ch] = v;
  }
  if (p.weights && ch == 0 && row < p.dst_max - first)
    p.weights_out[u * p.dst_max + first + row] = ok ? p.weights[u * p.tmax + kept_at(p, b, h, row)] : 0.0f;
}

// in place: blockIdx.x = slice of a row's 16-byte chunks (SC of them, K then V),
// and one more for the weights
template <int CPR, int SC>
__global__ __launch_bounds__(kCompactThreads, 4) void compact_in_place_kernel(CompactParams p) {
  constexpr int NS = CPR / SC, RPP = kCompactThreads / SC, U = 8;
  const int h = blockIdx.y, b = blockIdx.z, es = p.kv_f32 ? 4 : 2, tid = threadIdx.x;
  const int T = clamp_len(p.seq_lens[b], p.tmax);
  const int first = p.first ? clamp_len(p.first[b], p.dst_max) : 0;
  const int slice = blockIdx.x;
  if (slice == 2 * NS) {
    const int64_t u = ((int64_t)b * p.hkv + h) * p.tmax;
    const int end = p.num_kept > T - first ? p.num_kept : T - first;
    for (int j0 = 0; j0 < end; j0 += kCompactThreads * U) {
      float w[U];
#pragma unroll
      for (int i = 0; i < U; ++i) {
        const int j = j0 + i * kCompactThreads + tid;
        int64_t from, to;
        w[i] = 0.0f;
        if (j < p.num_kept && move_of(p, b, h, T, first, j, kept_at(p, b, h, j), from, to)) w[i] = p.weights[u + kept_at(p, b, h, j)];
      }
      __syncthreads();
#pragma unroll
      for (int i = 0; i < U; ++i) {
        const int j = j0 + i * kCompactThreads + tid;
        if (j < end && j < p.dst_max - first) p.weights_out[u + first + j] = w[i];
      }
      __syncthreads();
    }
    return;
  }
  // A batch's rows are in registers before the workgroup's barrier; then the next batch's, which
  // no write of this one meets, are under way while this one is written.
  char* base = static_cast<char*>(const_cast<void*>(slice < NS ? p.src.k : p.src.v));
  const int ch = (slice % NS) * SC + tid % SC, jt = tid / SC;
  int t[U];
  uint4 x[U] = {}, y[U] = {};
  int64_t to[U], to_y[U];
  auto entries = [&](int j0) {
#pragma unroll
    for (int i = 0; i < U; ++i) {
      const int j = j0 + i * RPP + jt;
      t[i] = j < p.num_kept ? kept_at(p, b, h, j) : -1;
    }
  };
  auto read = [&](int j0, uint4 (&r)[U], int64_t (&at)[U]) {
#pragma unroll
    for (int i = 0; i < U; ++i) {
      int64_t from;
      if (move_of(p, b, h, T, first, j0 + i * RPP + jt, t[i], from, at[i])) r[i] = reinterpret_cast<const uint4*>(base + from * es)[ch];
      else at[i] = -1;
    }
  };
  entries(0);
  read(0, x, to);
  entries(RPP * U);
  for (int j0 = 0; j0 < p.num_kept; j0 += RPP * U) {
#pragma unroll
    for (int i = 0; i < U; ++i) asm volatile("" : "+v"(x[i].x), "+v"(x[i].y), "+v"(x[i].z), "+v"(x[i].w));   // arrived
    __syncthreads();
    read(j0 + RPP * U, y, to_y);
    entries(j0 + 2 * RPP * U);
#pragma unroll
    for (int i = 0; i < U; ++i)
      if (to[i] >= 0) reinterpret_cast<uint4*>(base + to[i] * es)[ch] = x[i];
#pragma unroll
    for (int i = 0; i < U; ++i) {
      x[i] = y[i];
      to[i] = to_y[i];
    }
  }
}

template <int CPR>
static hipError_t launch_compact_rows(const CompactParams& p, hipStream_t st) {
  if (p.in_place) {
    // Slices of a 128-byte line where they are 128 workgroups, else of half a line (which two XCDs
    // then read): 32 units of 8192 rows 76 and 91 us, 128 of 2048 49 and 71, but 8 of 8192 66 and 36.
    const int more = p.weights ? 1 : 0;
    if ((int64_t)p.B * p.hkv * (2 * CPR / 8) >= 128)
      hipLaunchKernelGGL((compact_in_place_kernel<CPR, 8>), dim3(2 * CPR / 8 + more, p.hkv, p.B), dim3(kCompactThreads), 0, st, p);
    else
      hipLaunchKernelGGL((compact_in_place_kernel<CPR, 4>), dim3(2 * CPR / 4 + more, p.hkv, p.B), dim3(kCompactThreads), 0, st, p);
    return hipGetLastError();
  }
  const int rpw = kCompactThreads / CPR;
  const int rows = (p.num_kept + rpw - 1) / rpw;
  const int left = p.weights ? std::min(p.tmax, p.dst_max) - p.num_kept : 0;       // weights to clear, at most
  const int tail = left > 0 ? (left + 4 * kCompactThreads - 1) / (4 * kCompactThreads) : 0;
  if (rows + tail == 0) return hipSuccess;
  hipLaunchKernelGGL(compact_copy_kernel<CPR>, dim3(rows + tail, p.hkv, p.B), dim3(kCompactThreads), 0, st, p, rows);
  return hipGetLastError();
}

hipError_t launch_compact(const CompactParams& p, hipStream_t st) {
  if (p.num_kept == 0 && !p.weights) return hipSuccess;
  switch (p.d * (p.kv_f32 ? 4 : 2) / 16) {
    case 8: return launch_compact_rows<8>(p, st);
    case 16: return launch_compact_rows<16>(p, st);
    default: return launch_compact_rows<32>(p, st);
  }
}

}  // namespace cobs
