// cobs_decode8: the plan of a call and its launches.  The attention itself is in decode8_kernel.h.  The parts of a
// split context are joined there by the last workgroup to leave one (few rows), or by cobs_tree_decode's kernels.
#include "tokens_kernels.h"

namespace cobs {

hipError_t launch_decode8_bf16_d64(const Decode8Params& p, int rows, int grid, hipStream_t st);
hipError_t launch_decode8_bf16_d128(const Decode8Params& p, int rows, int grid, hipStream_t st);
hipError_t launch_decode8_f32_d64(const Decode8Params& p, int rows, int grid, hipStream_t st);
hipError_t launch_decode8_f32_d128(const Decode8Params& p, int rows, int grid, hipStream_t st);

constexpr int kFramesOfPass = 4;       // a workgroup's waves take a frame each

// Query rows of a workgroup, their tiles, and the workgroups that a context is split over.
static void decode8_plan(const AttendParams& a, int* rows, int* mtiles, int* nsplit) {
  const int M = a.N * a.G;
  *rows = M <= 16 ? 16 : 32;
  *mtiles = (M + *rows - 1) / *rows;
  // (three workgroups a CU, or two: kWorkgroups8)
  const int64_t slots = a.d == 64 && (a.io_bf16 || *rows == 16) ? 768 : 512;
  const int64_t passes = (max_frames(a) + kFramesOfPass - 1) / kFramesOfPass;
  *nsplit = parts_of(passes, (int64_t)a.B * a.hkv * *mtiles, 2.0, 1 << 30, 128, 0, slots);
}

// Arrival counters at the workspace's start: as many for every shape, so that calls of different shapes may use it in turn.
constexpr int kCounters = 4096;
constexpr size_t kCounterBytes = kCounters * sizeof(unsigned);

// Whether the last workgroup of a (row, KV head) joins its parts: few of them, as it reads them all alone (16 rows over 1000 tokens,
// 8 parts: 11.9 us a call, 13.7 with a launch for it; over 4000 tokens, 32 parts: 20.7 and 13.7).  It goes by the average: with parts by the rows' lengths a long row
// among short ones has more (8 rows of 8 KV heads, one of 32k tokens and 7 below 100: 4 query rows 26.6 us and 21.6, 16 query rows 36.0 and 22.4; 64 rows of one
// KV head 86 and 23; 8 rows alike 96 and 97, 16 from 2k to 32k 111 and 112).
static bool joined_by_last(const TreeParams& t) {
  return t.nsplit > 1 && t.mtiles == 1 && t.units <= kCounters && t.nsplit * t.a.N * t.a.G <= 128;
}

static size_t ml_bytes(size_t rows) { return (rows * 2 * sizeof(float) + 255) / 256 * 256; }

// Enough for both attended sets and types of q.
size_t decode8_workspace(const AttendParams& a) {
  int tile, mtiles, nsplit = 1;
  for (int form = 0; form < 4; ++form) {
    AttendParams x = a;
    x.sparse = form & 1;
    x.io_bf16 = form >> 1;
    int n;
    decode8_plan(x, &tile, &mtiles, &n);
    nsplit = n > nsplit ? n : nsplit;
  }
  const size_t rows = (size_t)a.B * a.hkv * nsplit * a.N * a.G;
  return kCounterBytes + ml_bytes(rows) + (rows * a.d * sizeof(float) + 255) / 256 * 256;
}

hipError_t launch_decode8(const Decode8Params& q, hipStream_t st) {
  Decode8Params p = q;
  TreeParams& t = p.t;
  int rows;
  decode8_plan(t.a, &rows, &t.mtiles, &t.nsplit);
  t.units = t.a.B * t.a.hkv;
  t.even = parts_by_length(t.a, t.nsplit);
  t.step = kFramesOfPass;
  p.counters = joined_by_last(t) ? reinterpret_cast<unsigned*>(t.part_ml) : nullptr;
  t.part_ml += kCounterBytes / sizeof(float);
  t.part_o = t.part_ml + ml_bytes((size_t)t.units * t.nsplit * t.a.N * t.a.G) / sizeof(float);
  // eight XCDs: a multiple of 8 workgroup slots (see decode8_kernel)
  const int64_t groups = ((int64_t)t.units * t.nsplit + 7) / 8 * 8, grid = groups * t.mtiles;
  if (grid > 0x7fffffff) return hipErrorInvalidValue;
  const int g = (int)grid;
  hipError_t e;
  if (t.a.io_bf16) e = t.a.d == 64 ? launch_decode8_bf16_d64(p, rows, g, st) : launch_decode8_bf16_d128(p, rows, g, st);
  else e = t.a.d == 64 ? launch_decode8_f32_d64(p, rows, g, st) : launch_decode8_f32_d128(p, rows, g, st);
  if (e != hipSuccess || t.nsplit == 1 || p.counters) return e;
  return launch_tree_merge(t, st);
}

}  // namespace cobs
