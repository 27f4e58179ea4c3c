// Device helpers of the cache operators.
#pragma once

#include "cache_kernels.h"

namespace cobs {

// The tokens of one (batch row, KV head) that queries attend to, as frames:
// aligned runs of 32 positions a .. a + 31, of which lo .. hi - 1 take part.
// First the frames of the valid selected blocks (tokens before the window start
// ws), then those from ws to the end E = C + n of the context and the draft
// (with the whole cache attended, ws = 0 and there are no blocks).  A frame
// lies within one block, so within one page, and wholly inside the cache (whose
// capacity is a multiple of 32).  Its tokens at positions below C are attended to
// by every query, those from C on by the queries with their bit set.
struct Attended {
  int C, n, E, ws;       // context, drafted tokens, their sum, window start
  int nq;                // live queries
  int nsel, fpb;         // valid selected blocks, frames of a block
  int lsh;
  const int32_t* sel;
  __device__ __forceinline__ int sel_frames() const { return nsel * fpb; }
  __device__ __forceinline__ int frames() const {
    return sel_frames() + (E > ws ? ((E + kFrame - 1) / kFrame - ws / kFrame) : 0);
  }
  __device__ __forceinline__ void frame(int f, int& a, int& lo, int& hi) const {
    const int ns = sel_frames();
    if (f < ns) {
      a = (sel[f / fpb] << lsh) + kFrame * (f % fpb);
      lo = a;
      hi = min(a + kFrame, ws);
    } else {
      a = (ws / kFrame + (f - ns)) * kFrame;
      lo = max(a, ws);
      hi = min(a + kFrame, E);
    }
  }
};

// Called by every thread of a workgroup of NT threads (with a barrier inside
// when there is a selection); `red`: NT / 64 ints of LDS.
template <int NT>
__device__ __forceinline__ Attended attended(const AttendParams& p, int b, int h, int* red) {
  Attended x;
  x.C = clamp_len(p.seq_lens[b], p.tmax);
  x.n = 0;
  x.nq = p.N;
  if (p.mask) {
    x.n = clamp_len(p.draft_lens[b], min(p.N, p.tmax - x.C));
    x.nq = x.n;
  }
  x.E = x.C + x.n;
  x.ws = p.sparse ? max(0, x.C - p.w) : 0;
  x.lsh = p.lsh;
  x.fpb = (1 << p.lsh) / kFrame;
  x.nsel = 0;
  x.sel = p.sel + ((int64_t)b * p.hkv + h) * p.s;
  if (p.sparse && p.s > 0) {
    const int nc = blocks_of(x.ws, p.lsh);
    int valid = p.s;                      // first entry that breaks the ascending run of candidates
    for (int i = threadIdx.x; i < p.s; i += NT) {
      const int bi = x.sel[i], prev = x.sel[i > 0 ? i - 1 : 0];
      if (bi < 0 || bi >= nc || (i > 0 && bi <= prev)) valid = min(valid, i);
    }
#pragma unroll
    for (int o = 32; o >= 1; o >>= 1) valid = min(valid, __shfl_xor(valid, o, 64));
    if ((threadIdx.x & 63) == 0) red[threadIdx.x >> 6] = valid;
    __syncthreads();
    valid = red[0];
#pragma unroll
    for (int i = 1; i < NT / 64; ++i) valid = min(valid, red[i]);
    x.nsel = valid;
  }
  return x;
}

// Parts that the rows' contexts are split into, where the `parts` B parts of a KV head go to the rows by
// their frames, at most one for each `step` frames of a row (its passes: a part without one would write and be joined
// for nothing): lane b has those of row b and of the rows before it.  So a row's parts, and the order
// of its sums, go by the other rows' lengths too.  (Alike in every kernel of a call; all lanes active.)
__device__ __forceinline__ void row_parts(const AttendParams& a, int parts, int step, int& n, int& before) {
  const int b = threadIdx.x & 63;
  uint32_t frames = 0;
  if (b < a.B) {
    const int C = clamp_len(a.seq_lens[b], a.tmax);
    const int drafted = a.mask ? clamp_len(a.draft_lens[b], min(a.N, a.tmax - C)) : 0;
    frames = (uint32_t)(C + drafted + kFrame - 1) / kFrame;
  }
  const uint32_t all = (uint32_t)__builtin_amdgcn_readlane(wave_incl_scan((int)frames), 63);
  // (at most 64 rows of 128 parts and 2^15 frames: below 2^32)
  n = 1 + (int)((uint32_t)(a.B * (parts - 1)) * frames / max(all, 1u));
  n = b < a.B ? min(n, max(1, (int)(frames + step - 1) / step)) : 0;
  before = wave_incl_scan(n) - n;
}

// What a workgroup does: part `split` of the `n` of (row b, KV head h), whose first is number `first` of all.
struct TreePart {
  int b, h, split, n;
  int64_t first;
};

// The part of workgroup `group` of units nsplit; false if it has none.  Of equal splits, the draft's frames
// and the longer parts first.
__device__ __forceinline__ bool tree_part(const TreeParams& p, int group, TreePart& t) {
  const int hkv = p.a.hkv;
  if (!p.even) {
    const int unit = group % p.units;
    t = {unit / hkv, unit % hkv, p.nsplit - 1 - group / p.units, p.nsplit, (int64_t)unit * p.nsplit};
    return true;
  }
  int n, before;
  row_parts(p.a, p.nsplit, p.step, n, before);
  t.h = group % hkv;
  const int j = group / hkv;
  const unsigned long long mine = __ballot(j >= before && j < before + n);
  if (mine == 0) return false;
  t.b = __builtin_ctzll(mine);
  const int skip = __builtin_amdgcn_readlane(before, t.b);
  t.split = j - skip;
  t.n = __builtin_amdgcn_readlane(n, t.b);
  t.first = (int64_t)t.h * p.a.B * p.nsplit + skip;
  return true;
}

__device__ __forceinline__ int wave_uniform32(int x) { return __builtin_amdgcn_readfirstlane(x); }

// The value that the lane of the other half of the wave (l ^ 32) holds.
__device__ __forceinline__ float other_half(float x) {
  const uint32_t u = __float_as_uint(x);
  const auto s = __builtin_amdgcn_permlane32_swap(u, u, false, false);
  return __uint_as_float((threadIdx.x & 32) ? s[0] : s[1]);
}

// Transposing LDS read of bf16: the 16 lanes of a group give the addresses of 4
// rows by four 8-byte pieces; lane i gets column i of the 4 rows.
__device__ __forceinline__ auto tr_read(const char* p) {
  typedef short s16x4 __attribute__((ext_vector_type(4)));
  return __builtin_amdgcn_ds_read_tr16_b64_v4i16(
      (__attribute__((address_space(3))) s16x4*)(const_cast<char*>(p)));
}

// Four outputs sum / total at element `i` (a multiple of 4) in the outputs' type; 0 for a total of 0.
__device__ __forceinline__ void store_row4(void* out, int64_t i, float4 sum, float total, int bf16) {
  const float f = total != 0.0f ? 1.0f / total : 0.0f;
  if (total == 0.0f) sum = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
  const float4 y = make_float4(sum.x * f, sum.y * f, sum.z * f, sum.w * f);
  if (bf16) {
    *reinterpret_cast<uint2*>(static_cast<uint16_t*>(out) + i) =
        make_uint2(f32x2_to_bf16x2_rne(y.x, y.y), f32x2_to_bf16x2_rne(y.z, y.w));
  } else {
    *reinterpret_cast<float4*>(static_cast<float*>(out) + i) = y;
  }
}

// The kernel's parameter block (its only argument) as it stands in memory: what a rare path at a kernel's end reads from
// there takes no scalar registers before.
template <typename P>
__device__ __forceinline__ const P& kernel_params() {
  uint64_t at = (uint64_t)__builtin_amdgcn_kernarg_segment_ptr();
  asm volatile("" : "+s"(at));
  return *reinterpret_cast<const P*>(at);
}

__device__ __forceinline__ float load_elem(const void* p, int64_t i, bool f32) {
  if (f32) return static_cast<const float*>(p)[i];
  return bf16_lo((uint32_t) static_cast<const uint16_t*>(p)[i]);
}

__device__ __forceinline__ void store_elem(void* p, int64_t i, float v, bool f32) {
  if (f32) static_cast<float*>(p)[i] = v;
  else static_cast<uint16_t*>(p)[i] = (uint16_t)f32_to_bf16_rne(v);
}

}  // namespace cobs
