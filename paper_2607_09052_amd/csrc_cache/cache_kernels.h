// Launch interface between the host side of the cache operators and their kernels.
#pragma once

#include "cobs_device.h"

namespace cobs {

constexpr int kMaxQueries = 64;      // query tokens per row: the bits of a tree mask word
constexpr int kFrame = 32;           // tokens of a frame (see Attended)

// What the query tokens of a call attend to (include/cobs_cache.h), and the sizes.
struct AttendParams {
  KvView kv;
  const void* q;                // [B, N, Hq, d], fp32 or bf16
  const int32_t* seq_lens;
  const int32_t* draft_lens;    // null: no draft
  const uint64_t* mask;
  const int32_t* sel;
  int sparse;
  int B, hkv, hq, G, N, d, tmax, s, w, lsh;
  int kv_f32, io_bf16;
  float c;
};

// Frames of the longest row that a call can attend to.
inline int max_frames(const AttendParams& a) {
  const int64_t dense = (a.tmax + kFrame - 1) / kFrame;
  const int64_t sparse = (int64_t)a.s * ((1 << a.lsh) / kFrame) + ((int64_t)a.w + a.N) / kFrame + 2;
  // (a selected block that the window start cuts has frames on both sides of it)
  return (int)(a.sparse && sparse < dense + 4 ? sparse : dense + (a.sparse ? 4 : 0));
}

// Workgroups that each of `units` pieces of work of `passes` passes is split over: at most `parts`, with
// at most `most` passes each, on `slots` (256 CUs, two workgroups each, as most of the kernels fit: tree_kernel
// for fp32 caches of 128-element heads, and for up to 32 rows of fp32 queries over bf16 ones, fits one; for 64-element
// bf16 caches three).  The split with the least
// time of its rounds: a pass takes `pass_us`, and a workgroup 4 us more (measured: 3 to 5 us of
// dependent loads before the first product).  The longest parts go first, so that only with one round
// does a part's last, uneven pass show.  `taken`: workgroups besides that the launch has.
inline int parts_of(int64_t passes, int64_t units, double pass_us, int64_t most, int64_t parts, int64_t taken = 0, int64_t slots = 512) {
  int64_t best = 0;
  double cost = 0.0;
  for (int64_t rounds = 1; rounds <= 64; ++rounds) {
    int64_t n = (slots * rounds - taken) / units;
    n = n < 1 ? 1 : n;
    n = n < parts ? n : parts;
    n = n < passes ? n : passes;
    const int64_t per = (passes + n - 1) / n, r = (units * n + taken + slots - 1) / slots;
    const double mean = (double)passes / (double)n;
    const double c = r * (mean * pass_us + 4.0) + (r == 1 ? (per - mean) * pass_us : 0.0);
    if (per <= most && (best == 0 || c < cost)) { best = n; cost = c; }
    if (per == 1) break;
  }
  return (int)(best > 0 ? best : (passes + most - 1) / most);
}

// Whether a batch's parts go to its rows by their lengths (row_parts) rather than `parts` to each.
inline bool parts_by_length(const AttendParams& a, int parts) {
  return !a.sparse && a.B > 1 && a.B <= 64 && parts >= 4 && parts <= 128 && max_frames(a) >= 32 * parts;
}

// Pass that part `i` of `n` begins with when `passes` are dealt evenly.
__host__ __device__ inline int first_pass(int passes, int i, int n) { return (int)((int64_t)passes * i / n); }

struct TreeParams {
  AttendParams a;
  void* out;
  float* lse;
  // parts of a context that is split over workgroups (tree_workspace): per (unit, split,
  // query row) the log2-domain maximum and sum, and D unnormalised outputs
  float* part_ml;
  float* part_o;
  int units, mtiles, nsplit;    // (row, KV head) pairs, query row tiles, splits
  int even, step;               // whether rows get parts by their length (row_parts); frames of a workgroup's pass
};

struct WeightsParams {
  AttendParams a;
  const float* lse;
  const float* prev;
  float* weights;
  // set by the launcher: workgroups of a (row, KV head), on average if `even` (row_parts); log2 of G
  int parts, lg, even;
};

// What a launch of an eviction leaves for the next, per chunk: the digits found and the keys still
// needed (the same in each chunk), the chunk's keys above those digits.
struct EvictState {
  uint32_t prefix;
  int need, over, unused;
};

struct EvictParams {
  const float* weights;
  const int32_t* seq_lens;
  int32_t* kept;
  int32_t* new_lens;
  int B, hkv, tmax, keep, sinks, recent;
  uint16_t* hist;               // digit histograms of the chunks, then their states (evict_workspace)
  EvictState* state;
  int chunks;                   // chunks of the longest row (set by the launcher)
};

struct CompactParams {
  KvView src, dst;
  const int32_t* kept;
  const int32_t* seq_lens;
  const int32_t* first;
  const float* weights;
  float* weights_out;
  int per_head, num_kept, B, hkv, d, tmax, dst_max, kv_f32, in_place;
};

// Row tiles and splits of a call, from its shape alone (so that a workspace's size depends on nothing else).
void tree_plan(const AttendParams& a, int* wq, int* mtiles, int* nsplit);
size_t tree_workspace(const AttendParams& a);
hipError_t launch_tree(const TreeParams& p, hipStream_t st);
hipError_t launch_weights(const WeightsParams& p, hipStream_t st);
size_t evict_workspace(int B, int hkv, int tmax);
hipError_t launch_evict(const EvictParams& p, hipStream_t st);
hipError_t launch_compact(const CompactParams& p, hipStream_t st);

}  // namespace cobs
