// cobs_append8: new tokens' keys (rotated) and values into a cache of 8-bit floats with one scale for
// each block and KV head; their queries rotated beside (append_body.h).
//
// The unit of work is (row b, block, KV head, keys or values): the largest magnitude among the block's new tokens sets
// its scale, so a unit holds its tokens in registers between that maximum and their encoding, and memory is
// read once.  D / 16 lanes take a token's head, 16 elements each.  A unit is taken by
//   a workgroup   (many new tokens; 256 lanes, PASSES times 16 elements each), which takes several heads in turn, so
//                 that the cosines and sines of its tokens stay in registers, or in LDS;
//   a wave        (up to 8 new tokens a row, 16 of 64-element heads);
//   D / 16 lanes  (one new token a row: a decode step, 8 or 16 units a wave).
// Scales are powers of two, so a grown scale changes the exponents of the block's earlier codes and nothing else
// (but for the smallest ones, which are rounded again).
//
// Measured (d 128, 8 KV and 32 query heads, bf16): four prompts of 8k to 16k tokens in 272 us with their queries, 1.34 GB, 4.9 TB/s (HBM, the
// rate of a large copy being 5.0); without queries 89 us, 4.1 TB/s read (a token's heads are apart by the queries') and written, waiting
// for a block's maximum between; in blocks of 128 tokens 132 us, as a lane's four rows take 232 registers, for two workgroups a CU.  One
// token of 64 rows: 5.6 us, a chain of loads (length, page, row, scale), if no block's scale grows.  The D / 16 lanes of a unit encode its earlier tokens again
// one after the other, a memory round trip each: where all 1024 units grow 31 us (blocks of 128: 50), and with scales that come from the tokens
// that the blocks hold (normal ones) 16 us on average over a block's steps (15).  Eight tokens of 64 rows, by a wave a unit: 7.5 us without, 9.5 with
// such scales, 11.4 if all grow.
#include "append_body.h"

namespace cobs {

// Query heads from which on a launch of their own rotates them: the workgroups that encode leave a CU three or four at a time, too few
// for a copy (q and all: 446 us for four prompts of 16k tokens, 8 KV and 32 query heads).
constexpr int64_t kApart = 1 << 15;
constexpr int kMostItems = 64;         // (head, keys or values) pairs that a workgroup takes in turn

// The smallest power of two s, 2^-100 at least, with top / s <= 448 = 1.75 * 2^8: a mantissa above 1.75 carries
// into the exponent.
__device__ __forceinline__ float scale_for(float top) {
  const int e = (int)((__float_as_uint(top) + 0x1fffffu) >> 23) - 8;
  return __uint_as_float((uint32_t)max(e, 27) << 23);
}

// Four codes of x * inv (at most 448 in magnitude, or NaN), the lowest byte first.  The hardware rounds to nearest even and
// keeps denormals.
__device__ __forceinline__ uint32_t codes4(const float* x, float inv) {
  int r = __builtin_amdgcn_cvt_pk_fp8_f32(x[0] * inv, x[1] * inv, 0, false);
  return (uint32_t)__builtin_amdgcn_cvt_pk_fp8_f32(x[2] * inv, x[3] * inv, r, true);
}

__device__ __forceinline__ void values4(uint32_t w, float* x) {
  const auto a = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, false), b = __builtin_amdgcn_cvt_pk_f32_fp8((int)w, true);
  x[0] = a[0]; x[1] = a[1]; x[2] = b[0]; x[3] = b[1];
}

// Whether a workgroup's cosines and sines are in LDS instead of registers, for four workgroups a CU in place of three (four prompts of
// 8k to 16k tokens 272 us for 285, without queries 89 for 102; fp32, which spills for it, four of 16k without queries 157 for 145).
template <int LANES, int PASSES, bool F32>
constexpr bool kTurnsShared = LANES == kHeadThreads && PASSES == 2 && !F32;

template <int D, int LANES, int PASSES, bool F32>
__global__ __launch_bounds__(kHeadThreads, (kTurnsShared<LANES, PASSES, F32> ? 4 : 1)) void append8_kernel(Append8Params p) {
  constexpr int TPR = D / 16, RP = LANES / TPR, UNITS = kHeadThreads / LANES;
  constexpr bool GROUP = LANES == kHeadThreads;
  static_assert(GROUP || LANES <= 64, "a workgroup, or lanes of a wave");
  __shared__ HeadsShared hs;
  __shared__ float s_top[2][kHeadThreads / 64], s_held[kMostItems];
  if (blockIdx.x == 0) write_lens(p.t);
  if ((int)blockIdx.x < p.q_groups) {
    heads_body<D, false>(p.t, nullptr, false, blockIdx.x, p.per_wg, p.slots, p.slot_groups, hs);
    return;
  }
  const int tid = threadIdx.x, H2 = 2 * p.t.hkv;
  // items: (head, K or V), keys first, `items` of them a workgroup (LANES < 256: one a unit)
  const int per = GROUP ? p.items : 1, groups = (H2 + per - 1) / per;
  const int64_t unit = (int64_t)((int)blockIdx.x - p.q_groups) * UNITS + tid / LANES;
  const int64_t units = (int64_t)p.t.B * p.blocks * groups;
  if (unit >= units) return;                           // (LANES == 256: the whole workgroup)
  const int it0 = (int)(unit % groups) * per, it1 = min(H2, it0 + per);
  const int bj = (int)(unit / groups), b = bj / p.blocks;
  const NewRow r = new_row(p.t, b);
  const int lsh = p.kv.lsh;
  const int n = min(r.n, p.t.tmax - r.T);               // tokens that the cache has room for
  const int j = (r.T >> lsh) + bj % p.blocks;           // the block
  const int t0 = max(j << lsh, r.T), t1 = min((j + 1) << lsh, r.T + n);     // its new tokens
  if (t0 >= t1) return;
  const int earlier = t0 - (j << lsh);                  // tokens that it holds
  const int64_t base = kv_offset(p.kv, b, 0, j << lsh);
  if (base < 0) return;
  const int64_t rs = p.kv.table ? D : p.kv.st, hs_step = p.kv.table ? ((int64_t)D << lsh) : p.kv.sh;
  const int64_t srow = p.kv.table ? base / ((int64_t)p.t.hkv * D << lsh) * p.t.hkv : (int64_t)b * p.t.hkv * p.kv.nbmax + j;
  const int64_t sstep = p.kv.table ? 1 : p.kv.nbmax;

  const int lane = tid % LANES, row = lane / TPR, piece = lane % TPR;
  const Piece e = piece_of<D>(p.t.rope, piece), straight = {16 * piece, 16 * piece + 8, false};
  // the new tokens' rows of an item as they come; the next item's are loaded while one is encoded
  Raw8 raw[PASSES][2];
  auto load = [&](int it) {
    const bool key = it < p.t.hkv;
    const HeadsView& from = key ? p.t.k : p.t.v;
    const Piece c = key ? e : straight;
#pragma unroll
    for (int k = 0; k < PASSES; ++k) {
      const int t = t0 + row + k * RP;
      if (t < t1) {
        const int64_t at = b * from.sb + (t - r.T) * from.sn + (key ? it : it - p.t.hkv) * from.sh;
        raw[k][0] = load_raw8(from.p, at + c.e0, F32);
        raw[k][1] = load_raw8(from.p, at + c.e1, F32);
      }
    }
  };
  auto scale_of = [&](int it) { return (it < p.t.hkv ? p.k_scale + it * sstep : p.v_scale + (it - p.t.hkv) * sstep) + srow; };
  // (workgroups begin with different heads, as those of one head of all tokens may lie in few memory channels: fp32 prompts 145 us for 165)
  const int items = it1 - it0, shift = GROUP ? bj % items : 0;
  auto item = [&](int i) { return it0 + (i + shift < items ? i + shift : i + shift - items); };
  load(item(0));
  if (GROUP && earlier > 0 && tid < items) s_held[tid] = *scale_of(it0 + tid);
  // (in LDS by token and pair; twos of pairs change places by the token, so that eight tokens are read from different banks)
  constexpr bool SHARED = kTurnsShared<LANES, PASSES, F32>;
  __shared__ __align__(16) float2 turn[SHARED ? PASSES * RP * (D / 2) : 1];
  auto turn_at = [&](int k, int x) { return &turn[(k * RP + row) * (D / 2) + ((8 * piece + x) ^ (2 * (row & 3)))]; };
  float2 cs[SHARED ? 1 : PASSES][8];
  if (e.turned && it0 < p.t.hkv) {
#pragma unroll
    for (int k = 0; k < PASSES; ++k) {
      const int t = t0 + row + k * RP;
      if (t < t1) {
        const int i = t - r.T, at = p.t.rope.positions ? p.t.rope.positions[(int64_t)b * p.t.N + i] : t;
#pragma unroll
        for (int x = 0; x < 8; ++x) {
          const float2 c = turn_of(p.t.rope, at, pair_of(p.t.rope, piece, x));
          if constexpr (SHARED) *turn_at(k, x) = c;        // (read by this lane alone)
          else cs[k][x] = c;
        }
      }
    }
  }
  for (int i = 0; i < items; ++i) {
    const int it = item(i);
    const bool key = it < p.t.hkv;
    const int h = key ? it : it - p.t.hkv;
    const Piece c = key ? e : straight;
    float x[PASSES][16];
    float top = 0.0f;
#pragma unroll
    for (int k = 0; k < PASSES; ++k) {
      if (t0 + row + k * RP < t1) {
        widen8(raw[k][0], F32, x[k]);
        widen8(raw[k][1], F32, x[k] + 8);
        if (c.turned) {
          if constexpr (SHARED) {
#pragma unroll
            for (int i = 0; i < 8; i += 2) {
              const float2* const two = turn_at(k, i);
              cs[0][i] = two[0];
              cs[0][i + 1] = two[1];
            }
          }
          turn16(x[k], cs[SHARED ? 0 : k], p.t.rope.interleaved);
        }
#pragma unroll
        for (int y = 0; y < 16; ++y) top = fmaxf(top, fabsf(x[k][y]));      // (NaN leaves it)
      }
    }
    if (__ballot(top == INFINITY)) {                    // rare: infinities become NaN and do not count
      top = 0.0f;
#pragma unroll
      for (int k = 0; k < PASSES; ++k)
#pragma unroll
        for (int y = 0; y < 16; ++y) {
          if (t0 + row + k * RP >= t1) continue;
          x[k][y] = fabsf(x[k][y]) < INFINITY ? x[k][y] : __uint_as_float(0x7fc00000u);
          top = fmaxf(top, fabsf(x[k][y]));
        }
    }
    if (i + 1 < items) load(item(i + 1));
    float* const scale = scale_of(it);
    float held = 0.0f;
    if constexpr (GROUP) {
      top = wave_max_rows(top);
      const int buf = i & 1;                   // (a barrier lies between a buffer's use and its next writing)
      if ((tid & 63) == 0) s_top[buf][tid >> 6] = top;
      __syncthreads();
#pragma unroll
      for (int w = 0; w < kHeadThreads / 64; ++w) top = fmaxf(top, s_top[buf][w]);
      if (earlier > 0) held = s_held[it - it0];
    } else {
#pragma unroll
      for (int o = LANES / 2; o >= 1; o >>= 1) top = fmaxf(top, __shfl_xor(top, o, 64));
      if (earlier > 0) held = *scale;
    }
    const float need = scale_for(top);
    const float now = earlier > 0 && held >= need ? held : need, inv = 1.0f / now;
    uint8_t* const codes = static_cast<uint8_t*>(const_cast<void*>(key ? p.kv.k : p.kv.v)) + base + h * hs_step;
    if (earlier > 0 && now != held) {
      const float ratio = held * inv;
      for (int t = row; t < earlier; t += RP) {
        uint4* const at = reinterpret_cast<uint4*>(codes + t * rs + 16 * piece);
        const uint4 w = *at;
        float y[16];
        values4(w.x, y); values4(w.y, y + 4); values4(w.z, y + 8); values4(w.w, y + 12);
        *at = make_uint4(codes4(y, ratio), codes4(y + 4, ratio), codes4(y + 8, ratio), codes4(y + 12, ratio));
      }
    }
#pragma unroll
    for (int k = 0; k < PASSES; ++k) {
      const int t = t0 + row + k * RP;
      if (t < t1) {
        uint8_t* const at = codes + (t - (j << lsh)) * rs;
        *reinterpret_cast<uint2*>(at + c.e0) = make_uint2(codes4(x[k], inv), codes4(x[k] + 4, inv));
        *reinterpret_cast<uint2*>(at + c.e1) = make_uint2(codes4(x[k] + 8, inv), codes4(x[k] + 12, inv));
      }
    }
    if (lane == 0) *scale = now;
  }
}

template <int D, bool F32>
static hipError_t launch_d(Append8Params p, hipStream_t st) {
  constexpr int TPR = D / 16;
  const int L = 1 << p.kv.lsh;
  p.q_groups = p.per_wg = p.slots = p.slot_groups = 0;
  const int64_t tokens = (int64_t)p.t.B * p.t.N;
  if (p.t.hq > 0 && tokens * p.t.hq >= kApart) {
    AppendParams q = {};
    q.t = p.t;
    q.t.hkv = 0;
    q.t.new_seq_lens = nullptr;
    const hipError_t e = launch_append(q, st);
    if (e != hipSuccess) return e;
  } else if (p.t.hq > 0) {
    plan_heads(tokens, p.t.hq, D, &p.per_wg, &p.slots, &p.slot_groups);
    const int64_t g = (tokens + p.per_wg - 1) / p.per_wg * p.slot_groups;
    if (g > 0x3fffffff) return hipErrorInvalidValue;
    p.q_groups = (int)g;
  }
  const int most = p.t.N < L ? p.t.N : L;               // new tokens of a block
  p.blocks = (p.t.N + L - 2) / L + 1;
  const int lanes = most == 1 ? TPR : (most <= 64 / TPR ? 64 : kHeadThreads);
  p.items = 1;
  if (lanes == kHeadThreads) {
    // Heads of a workgroup, which share their tokens' cosines and sines: as many as leave two workgroups a CU, keys and values apart
    // (16000 tokens in blocks of 128, 8 heads: 26 us; by 2048 workgroups of one head each 38; 49000 tokens by workgroups of
    // 8 heads' keys or values 89, when those took 102 by workgroups of both 130).
    const int64_t all = (int64_t)p.t.B * p.blocks * 2 * p.t.hkv;
    const int top = p.t.hkv < kMostItems ? p.t.hkv : kMostItems;
    p.items = (int)(all / 512 < top ? all / 512 : top);
    if (p.items < 1) p.items = 1;
  }
  const int64_t units = (int64_t)p.t.B * p.blocks * ((2 * p.t.hkv + p.items - 1) / p.items);
  const int per_group = kHeadThreads / lanes;
  const int64_t grid = p.q_groups + (units + per_group - 1) / per_group;
  if (grid > 0x7fffffff) return hipErrorInvalidValue;
  const dim3 g((uint32_t)grid), t(kHeadThreads);
  const int rows = kHeadThreads / TPR;                  // tokens of a workgroup's pass
  if (lanes == TPR) hipLaunchKernelGGL((append8_kernel<D, TPR, 1, F32>), g, t, 0, st, p);
  else if (lanes == 64) hipLaunchKernelGGL((append8_kernel<D, 64, 1, F32>), g, t, 0, st, p);
  else if (most <= rows) hipLaunchKernelGGL((append8_kernel<D, kHeadThreads, 1, F32>), g, t, 0, st, p);
  else if (most <= 2 * rows) hipLaunchKernelGGL((append8_kernel<D, kHeadThreads, 2, F32>), g, t, 0, st, p);
  else if constexpr (D == 128) hipLaunchKernelGGL((append8_kernel<D, kHeadThreads, 4, F32>), g, t, 0, st, p);
  return hipGetLastError();
}

hipError_t launch_append8(const Append8Params& p, hipStream_t st) {
  if (p.t.k.f32) return p.t.d == 64 ? launch_d<64, true>(p, st) : launch_d<128, true>(p, st);
  return p.t.d == 64 ? launch_d<64, false>(p, st) : launch_d<128, false>(p, st);
}

}  // namespace cobs
