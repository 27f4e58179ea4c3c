// cobs_tree_decode: the plan of a call, its launches, and the kernel that joins
// the parts of a split context.  The attention itself is in tree_kernel.h.
#include "cache_device.h"

namespace cobs {

constexpr int kMergeThreads = 256;

// One thread per 4 outputs of a query row: the parts' weights 2^(m_k - max m) and
// sums in split order.
template <int D>
__global__ __launch_bounds__(kMergeThreads) void tree_merge_kernel(TreeParams p) {
  constexpr int TPR = D / 4;
  const AttendParams& a = p.a;
  const int M = a.N * a.G;
  const int64_t idx = (int64_t)blockIdx.x * (kMergeThreads / TPR) + threadIdx.x / TPR;
  const int d4 = threadIdx.x % TPR;
  if (idx >= (int64_t)p.units * M) return;
  const int unit = (int)(idx / M), row = (int)(idx % M), b = unit / a.hkv, h = unit % a.hkv;
  const int i = row / a.G;
  const int64_t at = ((int64_t)b * a.N + i) * a.hq + h * a.G + (row - i * a.G);
  const int C = clamp_len(a.seq_lens[b], a.tmax);
  const int nq = a.mask ? clamp_len(a.draft_lens[b], min(a.N, a.tmax - C)) : a.N;
  float top = -INFINITY, total = 0.0f;
  float4 sum = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
  if (i < nq) {
    const int64_t first = (int64_t)unit * p.nsplit * M + row;
    for (int k = 0; k < p.nsplit; ++k) top = fmaxf(top, p.part_ml[2 * (first + (int64_t)k * M)]);
    const float ref = top == -INFINITY ? 0.0f : top;
    for (int k = 0; k < p.nsplit; ++k) {
      const int64_t r = first + (int64_t)k * M;
      const float2 ml = *reinterpret_cast<const float2*>(p.part_ml + 2 * r);
      const float f = __builtin_amdgcn_exp2f(ml.x - ref);
      const float4 o = *reinterpret_cast<const float4*>(p.part_o + r * D + 4 * d4);
      total += f * ml.y;
      sum.x += f * o.x; sum.y += f * o.y; sum.z += f * o.z; sum.w += f * o.w;
    }
    top = ref;
  }
  store_row4(p.out, at * D + 4 * d4, sum, total, a.io_bf16);
  if (d4 == 0 && p.lse) p.lse[at] = total != 0.0f ? top * 0.6931471805599453f + logf(total) : -INFINITY;
}

hipError_t launch_tree_bf16_d64(const TreeParams& p, int wq, int grid, hipStream_t st);
hipError_t launch_tree_bf16_d128(const TreeParams& p, int wq, int grid, hipStream_t st);
hipError_t launch_tree_f32_d64(const TreeParams& p, int wq, int grid, hipStream_t st);
hipError_t launch_tree_f32_d128(const TreeParams& p, int wq, int grid, hipStream_t st);

void tree_plan(const AttendParams& a, int* wq, int* mtiles, int* nsplit) {
  const int M = a.N * a.G;
  *wq = M <= 32 ? 1 : (M <= 64 ? 2 : 4);
  *mtiles = (M + *wq * 32 - 1) / (*wq * 32);
  // frames of the longest row, and as many splits as give the chip's 256 CUs two
  // workgroups each, of at least 8 frames
  const int64_t frames = max_frames(a);
  const int64_t tiles = (int64_t)a.B * a.hkv * *mtiles;
  int64_t n = (512 + tiles - 1) / tiles;
  n = n < frames / 8 ? n : frames / 8;
  *nsplit = (int)(n < 1 ? 1 : (n > 128 ? 128 : n));
}

// Enough for both attended sets.
size_t tree_workspace(const AttendParams& a) {
  int wq, mtiles, nsplit = 1;
  for (int sparse = 0; sparse < 2; ++sparse) {
    AttendParams x = a;
    x.sparse = sparse;
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
  const int64_t rows_out = (int64_t)p.units * p.a.N * p.a.G, per = kMergeThreads / (p.a.d / 4);
  const dim3 mg((unsigned)((rows_out + per - 1) / per));
  if (p.a.d == 64) hipLaunchKernelGGL(tree_merge_kernel<64>, mg, dim3(kMergeThreads), 0, st, p);
  else hipLaunchKernelGGL(tree_merge_kernel<128>, mg, dim3(kMergeThreads), 0, st, p);
  return hipGetLastError();
}

}  // namespace cobs
