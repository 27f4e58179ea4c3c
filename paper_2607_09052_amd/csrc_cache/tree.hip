// cobs_tree_decode: the plan of a call, its launches, and the kernel that joins
// the parts of a split context.  The attention itself is in tree_kernel.h.
#include "cache_device.h"

namespace cobs {

constexpr int kMergeThreads = 256;

struct MergeRow {
  int64_t first, at;   // its first part; its row of out and lse
  int n;               // parts
  bool live;           // of a query that is there
};
// (every lane of the wave calls it)
__device__ __forceinline__ MergeRow merge_row(const TreeParams& p, uint32_t idx) {
  const AttendParams& a = p.a;
  const uint32_t M = a.N * a.G;
  const int unit = idx / M, row = idx % M, b = unit / a.hkv, h = unit % a.hkv, i = row / a.G;
  const int C = clamp_len(a.seq_lens[b], a.tmax);
  const int nq = a.mask ? clamp_len(a.draft_lens[b], min(a.N, a.tmax - C)) : a.N;
  int n = p.nsplit;
  int64_t first = (int64_t)unit * p.nsplit;
  if (p.even) {
    int parts, before;
    row_parts(a, p.nsplit, p.step, parts, before);
    n = __shfl(parts, b, 64);
    first = (int64_t)h * a.B * p.nsplit + __shfl(before, b, 64);
  }
  return {first * M + row, ((int64_t)b * a.N + i) * a.hq + h * a.G + (row - i * a.G), n, i < nq};
}

// Parts joined with the weights 2^(m_k - max m).  A row of up to kFewParts parts by D / 4 threads,
// 4 outputs a thread, all loads in one batch: many rows, bound by HBM (2 parts of 32768 rows of
// 128: 9 us, 4.7 TB/s; by four groups 36 us, as two of them have nothing to do).
constexpr int kFewParts = 4;
template <int D>
__global__ __launch_bounds__(kMergeThreads) void tree_merge_few_kernel(TreeParams p) {
  constexpr int TPR = D / 4, RPB = kMergeThreads / TPR;
  const int M = p.a.N * p.a.G, d4 = threadIdx.x % TPR;
  const uint32_t idx = blockIdx.x * RPB + threadIdx.x / TPR;
  const bool here = idx < (uint32_t)(p.units * M);
  const MergeRow r = merge_row(p, here ? idx : 0);
  if (!here) return;
  float2 ml[kFewParts];
  float4 o[kFewParts];
#pragma unroll
  for (int k = 0; k < kFewParts; ++k) {
    if (k < r.n) {                                       // (of a query that is not there: read, not used)
      const int64_t at = r.first + (int64_t)k * M;
      ml[k] = *reinterpret_cast<const float2*>(p.part_ml + 2 * at);
      o[k] = *reinterpret_cast<const float4*>(p.part_o + at * D + 4 * d4);
    } else {
      ml[k] = make_float2(-INFINITY, 0.0f);
      o[k] = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
    }
  }
  float top = -INFINITY, total = 0.0f;
#pragma unroll
  for (int k = 0; k < kFewParts; ++k) top = fmaxf(top, ml[k].x);
  const float ref = top == -INFINITY ? 0.0f : top;
  float4 sum = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
#pragma unroll
  for (int k = 0; k < kFewParts; ++k) {
    const float f = __builtin_amdgcn_exp2f(ml[k].x - ref);
    total += f * ml[k].y;
    sum.x += f * o[k].x; sum.y += f * o[k].y; sum.z += f * o[k].z; sum.w += f * o[k].w;
  }
  if (!r.live) {
    total = 0.0f;
    sum = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
  }
  store_row4(p.out, r.at * D + 4 * d4, sum, total, p.a.io_bf16);
  if (d4 == 0 && p.lse) p.lse[r.at] = total != 0.0f ? ref * 0.6931471805599453f + logf(total) : -INFINITY;
}

// A row of more parts by kMergeGroups groups of D / 4 threads: group g takes the
// parts g, g + 4, ... (their loads in flight together), and the groups' sums meet
// in LDS in group order.  Few rows, bound by the chain of loads: 3 to 4 us of 32 parts of
// 32 to 256 rows.
constexpr int kMergeGroups = 4;
template <int D>
__global__ __launch_bounds__(kMergeThreads) void tree_merge_kernel(TreeParams p) {
  constexpr int TPR = D / 4, RPB = kMergeThreads / (TPR * kMergeGroups), U = 8;
  __shared__ float4 s_sum[RPB][kMergeGroups][TPR];
  __shared__ float s_total[RPB][kMergeGroups];
  const int M = p.a.N * p.a.G;
  const int rb = threadIdx.x / (TPR * kMergeGroups), g = threadIdx.x / TPR % kMergeGroups, d4 = threadIdx.x % TPR;
  const uint32_t idx = blockIdx.x * RPB + rb;
  const bool here = idx < (uint32_t)(p.units * M);
  const MergeRow r = merge_row(p, here ? idx : 0);
  const int n = here && r.live ? r.n : 0;
  // the parts' maxima: each thread of a group loads its share
  float top = -INFINITY;
  for (int k = d4; k < n; k += TPR) top = fmaxf(top, p.part_ml[2 * (r.first + (int64_t)k * M)]);
#pragma unroll
  for (int o = TPR / 2; o >= 1; o >>= 1) top = fmaxf(top, __shfl_xor(top, o, 64));
  const float ref = top == -INFINITY ? 0.0f : top;
  float total = 0.0f;
  float4 sum = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
  for (int k0 = g; k0 < n; k0 += U * kMergeGroups) {
    float2 ml[U];
    float4 o[U];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int k = k0 + u * kMergeGroups;
      const int64_t at = r.first + (int64_t)(k < n ? k : g) * M;
      ml[u] = *reinterpret_cast<const float2*>(p.part_ml + 2 * at);
      o[u] = *reinterpret_cast<const float4*>(p.part_o + at * D + 4 * d4);
    }
#pragma unroll
    for (int u = 0; u < U; ++u) {
      if (k0 + u * kMergeGroups < n) {
        const float f = __builtin_amdgcn_exp2f(ml[u].x - ref);
        total += f * ml[u].y;
        sum.x += f * o[u].x; sum.y += f * o[u].y; sum.z += f * o[u].z; sum.w += f * o[u].w;
      }
    }
  }
  s_sum[rb][g][d4] = sum;
  if (d4 == 0) s_total[rb][g] = total;
  __syncthreads();
  if (g != 0 || !here) return;
#pragma unroll
  for (int k = 1; k < kMergeGroups; ++k) {
    const float4 o = s_sum[rb][k][d4];
    sum.x += o.x; sum.y += o.y; sum.z += o.z; sum.w += o.w;
    total += s_total[rb][k];
  }
  store_row4(p.out, r.at * D + 4 * d4, sum, total, p.a.io_bf16);
  if (d4 == 0 && p.lse) p.lse[r.at] = total != 0.0f ? ref * 0.6931471805599453f + logf(total) : -INFINITY;
}

template <int D>
static hipError_t launch_merge(const TreeParams& p, hipStream_t st) {
  const bool few = p.nsplit <= kFewParts && !p.even;
  const uint32_t rows = (uint32_t)(p.units * p.a.N * p.a.G), per = kMergeThreads / (D / 4 * (few ? 1 : kMergeGroups));
  const dim3 g((rows + per - 1) / per), t(kMergeThreads);
  if (few) hipLaunchKernelGGL(tree_merge_few_kernel<D>, g, t, 0, st, p);
  else hipLaunchKernelGGL(tree_merge_kernel<D>, g, t, 0, st, p);
  return hipGetLastError();
}

hipError_t launch_tree_merge(const TreeParams& p, hipStream_t st) {
  return p.a.d == 64 ? launch_merge<64>(p, st) : launch_merge<128>(p, st);
}

hipError_t launch_tree_bf16_d64(const TreeParams& p, int wq, int grid, hipStream_t st);
hipError_t launch_tree_bf16_d128(const TreeParams& p, int wq, int grid, hipStream_t st);
hipError_t launch_tree_f32_d64(const TreeParams& p, int wq, int grid, hipStream_t st);
hipError_t launch_tree_f32_d128(const TreeParams& p, int wq, int grid, hipStream_t st);

// Frames of a pass of a workgroup's waves (STEP of the kernels).
static int pass_frames(const AttendParams& a, int wq) { return wq == 1 ? 4 : (wq == 2 || !a.kv_f32 ? 2 : 1); }

void tree_plan(const AttendParams& a, int* wq, int* mtiles, int* nsplit) {
  const int M = a.N * a.G;
  *wq = M <= 32 ? 1 : (M <= 64 ? 2 : 4);
  // Tiles of 256 rows (tree_wide.h) where they pad no more than tiles of 128 and a workgroup has some 64 frames
  // or more (us with tiles of 128 and of 256: 512 rows over 8 x 32k tokens 873, 804; 256 rows over 32 x 4k 245, 233,
  // over 32k 77, 77, over 16 x 2k 79, 80).
  const int64_t units = (int64_t)a.B * a.hkv, tiles = (M + 255) / 256;
  if (a.io_bf16 && !a.kv_f32 && a.d == 128 && (M + 127) / 128 == 2 * tiles && max_frames(a) * units * tiles >= 64 * 256) *wq = 8;
  *mtiles = (M + *wq * 32 - 1) / (*wq * 32);
  // the longest row's frames, by a pass of a workgroup's waves at a time
  const int step = pass_frames(a, *wq);
  const int64_t passes = (max_frames(a) + step - 1) / step;
  *nsplit = parts_of(passes, units * *mtiles, *wq == 8 ? 1.0 : 2.0, 1 << 30, 128, 0, *wq == 8 ? 256 : 512);
}

// Enough for both attended sets and types of q.
size_t tree_workspace(const AttendParams& a) {
  int wq, mtiles, nsplit = 1;
  for (int form = 0; form < 4; ++form) {
    AttendParams x = a;
    x.sparse = form & 1;
    x.io_bf16 = form >> 1;
    int n;
    tree_plan(x, &wq, &mtiles, &n);
    nsplit = n > nsplit ? n : nsplit;
  }
  const size_t rows = (size_t)a.B * a.hkv * nsplit * a.N * a.G;
  const size_t ml = (rows * 2 * sizeof(float) + 255) / 256 * 256;
  return ml + (rows * a.d * sizeof(float) + 255) / 256 * 256;
}

hipError_t launch_tree(const TreeParams& q, hipStream_t st) {
  TreeParams p = q;
  int wq;
  tree_plan(p.a, &wq, &p.mtiles, &p.nsplit);
  p.units = p.a.B * p.a.hkv;
  // Parts by the rows' lengths, which a wave's lanes hold: 128 rows over 4 contexts of 8k to 32k tokens, on pages,
  // 133 us (139 with as many parts a row), 32 rows over 16 contexts 284 (301).  Contexts of one length pay 1 to 2 us
  // for finding their part, so not for short ones, nor where few parts a row are dealt too coarsely (512 rows over
  // 8 contexts of 2 parts: 800 us, 722 with 2 for each).
  p.even = parts_by_length(p.a, p.nsplit);
  p.step = pass_frames(p.a, wq);
  const size_t rows = (size_t)p.units * p.nsplit * p.a.N * p.a.G;
  p.part_o = p.part_ml + (rows * 2 * sizeof(float) + 255) / 256 * 256 / sizeof(float);
  // eight XCDs: a multiple of 8 workgroup slots (see tree_kernel)
  const int64_t groups = ((int64_t)p.units * p.nsplit + 7) / 8 * 8, grid = groups * p.mtiles;
  if (grid > 0x7fffffff) return hipErrorInvalidValue;
  const int g = (int)grid;
  hipError_t e;
  if (p.a.kv_f32) e = p.a.d == 64 ? launch_tree_f32_d64(p, wq, g, st) : launch_tree_f32_d128(p, wq, g, st);
  else e = p.a.d == 64 ? launch_tree_bf16_d64(p, wq, g, st) : launch_tree_bf16_d128(p, wq, g, st);
  if (e != hipSuccess || p.nsplit == 1) return e;
  return launch_tree_merge(p, st);
}

}  // namespace cobs
