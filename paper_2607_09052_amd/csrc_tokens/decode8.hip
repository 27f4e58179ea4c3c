// cobs_decode8: the plan of a call and its launches.  The attention itself is in decode8_kernel.h, the
// kernels that join the parts of a split context are cobs_tree_decode's.
#include "tokens_kernels.h"

namespace cobs {

hipError_t launch_decode8_bf16_d64(const Decode8Params& p, int tiles, int grid, hipStream_t st);
hipError_t launch_decode8_bf16_d128(const Decode8Params& p, int tiles, int grid, hipStream_t st);
hipError_t launch_decode8_f32_d64(const Decode8Params& p, int tiles, int grid, hipStream_t st);
hipError_t launch_decode8_f32_d128(const Decode8Params& p, int tiles, int grid, hipStream_t st);

// Tiles of 16 query rows that a workgroup takes: 1 or 2 (decode8_kernel), 4 or 8 (decode8_many_kernel); frames that its
// waves take at a time.
static int row_tiles(const AttendParams& a) {
  const int M = a.N * a.G;
  const bool two = a.d == 64 || a.io_bf16;              // tiles a wave
  return M <= 16 ? 1 : (M <= 32 && two ? 2 : (M <= 64 || !two ? 4 : 8));
}
static int pass_frames(int tiles) { return tiles <= 2 ? 4 : 2; }

static void decode8_plan(const AttendParams& a, int* tiles, int* mtiles, int* nsplit) {
  *tiles = row_tiles(a);
  *mtiles = (a.N * a.G + *tiles * 16 - 1) / (*tiles * 16);
  const int step = pass_frames(*tiles);
  const int64_t passes = (max_frames(a) + step - 1) / step;
  *nsplit = parts_of(passes, (int64_t)a.B * a.hkv * *mtiles, 2.0, 1 << 30, 128);
}

static size_t ml_bytes(size_t rows) { return (rows * 2 * sizeof(float) + 255) / 256 * 256; }

// Enough for both attended sets and types of q.
size_t decode8_workspace(const AttendParams& a) {
  int tiles, mtiles, nsplit = 1;
  for (int form = 0; form < 4; ++form) {
    AttendParams x = a;
    x.sparse = form & 1;
    x.io_bf16 = form >> 1;
    int n;
    decode8_plan(x, &tiles, &mtiles, &n);
    nsplit = n > nsplit ? n : nsplit;
  }
  const size_t rows = (size_t)a.B * a.hkv * nsplit * a.N * a.G;
  return ml_bytes(rows) + (rows * a.d * sizeof(float) + 255) / 256 * 256;
}

hipError_t launch_decode8(const Decode8Params& q, hipStream_t st) {
  Decode8Params p = q;
  TreeParams& t = p.t;
  int tiles;
  decode8_plan(t.a, &tiles, &t.mtiles, &t.nsplit);
  t.units = t.a.B * t.a.hkv;
  t.even = parts_by_length(t.a, t.nsplit);
  t.step = pass_frames(tiles);
  t.part_o = t.part_ml + ml_bytes((size_t)t.units * t.nsplit * t.a.N * t.a.G) / sizeof(float);
  // eight XCDs: a multiple of 8 workgroup slots (see decode8_kernel)
  const int64_t groups = ((int64_t)t.units * t.nsplit + 7) / 8 * 8, grid = groups * t.mtiles;
  if (grid > 0x7fffffff) return hipErrorInvalidValue;
  const int g = (int)grid;
  hipError_t e;
  if (t.a.io_bf16) e = t.a.d == 64 ? launch_decode8_bf16_d64(p, tiles, g, st) : launch_decode8_bf16_d128(p, tiles, g, st);
  else e = t.a.d == 64 ? launch_decode8_f32_d64(p, tiles, g, st) : launch_decode8_f32_d128(p, tiles, g, st);
  if (e != hipSuccess || t.nsplit == 1) return e;
  return launch_tree_merge(t, st);
}

}  // namespace cobs
