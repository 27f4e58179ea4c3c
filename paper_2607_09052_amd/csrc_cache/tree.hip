// Attention of several query tokens a row over the cache and their draft
// (cobs_tree_decode).  One workgroup per (query, query head); its four waves
// take the frames of the attended tokens round-robin, each with a running
// maximum, sum and output, which they merge through LDS at the end.  Per frame
// lane l scores token l & 31 over half l >> 5 of the head dimension.
#include "cache_device.h"

namespace cobs {

template <int D>
__global__ __launch_bounds__(256) void tree_plain_kernel(TreeParams p) {
  constexpr int CPL = D / 64;
  __shared__ float qs[D];
  __shared__ float wm[4], wl[4], wo[4][D];
  __shared__ int red[4];
  const AttendParams& a = p.a;
  const int hq = blockIdx.x, i = blockIdx.y, b = blockIdx.z;
  const int h = hq / a.G, tid = threadIdx.x, wave = tid >> 6, lane = tid & 63;
  const Attended x = attended<256>(a, b, h, red);
  const int64_t row = ((int64_t)b * a.N + i) * a.hq + hq;
  for (int e = tid; e < D; e += 256) qs[e] = load_elem(a.q, row * D + e, !a.io_bf16) * a.c;
  __syncthreads();
  float m = -INFINITY, l = 0.0f, o[CPL];
#pragma unroll
  for (int j = 0; j < CPL; ++j) o[j] = 0.0f;
  const uint64_t bits = a.mask ? a.mask[(int64_t)b * a.N + i] : 0;
  const int64_t rs = a.kv.table ? a.kv.d : a.kv.st;
  const bool f32 = a.kv_f32 != 0;
  const int nf = i < x.nq ? x.frames() : 0;
  for (int f = wave; f < nf; f += 4) {
    int t0, lo, hi;
    x.frame(f, t0, lo, hi);
    const int64_t base = hi > lo ? kv_offset(a.kv, b, h, t0) : -1;
    if (base < 0) continue;
    const int t = t0 + (lane & 31), half = lane >> 5;
    const bool seen = t >= lo && t < hi && (t < x.C || ((bits >> (t - x.C)) & 1));
    float sc = 0.0f;
    if (seen)
      for (int e = half * (D / 2); e < (half + 1) * (D / 2); ++e)
        sc += qs[e] * load_elem(a.kv.k, base + (t - t0) * rs + e, f32);
    sc += __shfl_xor(sc, 32, 64);
    if (!seen) sc = -INFINITY;
    const float mn = fmaxf(m, wave_max(sc));
    const float ref = mn == -INFINITY ? 0.0f : mn;
    const float alpha = __expf(m - ref), pr = seen ? __expf(sc - ref) : 0.0f;
    l = l * alpha + 0.5f * wave_sum(pr);
    m = mn;
#pragma unroll
    for (int j = 0; j < CPL; ++j) o[j] *= alpha;
    for (int r = 0; r < kFrame; ++r) {
      if (!__shfl((int)seen, r, 64)) continue;
      const float pt = __shfl(pr, r, 64);
#pragma unroll
      for (int j = 0; j < CPL; ++j) o[j] += pt * load_elem(a.kv.v, base + r * rs + j * 64 + lane, f32);
    }
  }
  if (lane == 0) { wm[wave] = m; wl[wave] = l; }
#pragma unroll
  for (int j = 0; j < CPL; ++j) wo[wave][j * 64 + lane] = o[j];
  __syncthreads();
  const float top = fmaxf(fmaxf(wm[0], wm[1]), fmaxf(wm[2], wm[3])), M = top == -INFINITY ? 0.0f : top;
  float L = 0.0f, f[4];
#pragma unroll
  for (int k = 0; k < 4; ++k) {
    f[k] = __expf(wm[k] - M);
    L += f[k] * wl[k];
  }
  for (int e = tid; e < D; e += 256) {
    float s = 0.0f;
#pragma unroll
    for (int k = 0; k < 4; ++k) s += f[k] * wo[k][e];
    store_elem(p.out, row * D + e, L != 0.0f ? s / L : 0.0f, !a.io_bf16);
  }
  if (p.lse && tid == 0) p.lse[row] = L != 0.0f ? M + logf(L) : -INFINITY;
}

size_t tree_workspace(const AttendParams&) { return 256; }

hipError_t launch_tree(const TreeParams& p, hipStream_t st) {
  const dim3 grid(p.a.hq, p.a.N, p.a.B);
  if (p.a.d == 128) hipLaunchKernelGGL(tree_plain_kernel<128>, grid, dim3(256), 0, st, p);
  else hipLaunchKernelGGL(tree_plain_kernel<64>, grid, dim3(256), 0, st, p);
  return hipGetLastError();
}

}  // namespace cobs
