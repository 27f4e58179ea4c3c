// Launch interface between the host side of the token operators and their kernels.
#pragma once

#include "cache_kernels.h"

namespace cobs {

// Workgroups of a launch: HIP takes fewer than 2^32 threads in a dimension, and a workgroup has 256.  A call of more takes several launches.
constexpr int64_t kLaunchGroups = 1 << 23;

// Heads of tokens by their strides, in elements.
struct HeadsView {
  void* p;
  int64_t sb, sn, sh;
  int f32;
};

struct RopeView {
  const float* freq;
  const int32_t* positions;     // [B, N]; null: the token's place in the cache
  int half;                     // pairs; 0: no rotation
  int interleaved;
  float scale;
};

// New tokens (include/cobs_tokens.h): queries to rotate (hq = 0: none), keys and values to append
// (hkv = 0: none).
struct NewTokens {
  RopeView rope;
  HeadsView q, q_out, k, v;
  const int32_t* seq_lens;      // null: no cache, every token is live
  const int32_t* new_lens;      // null: N
  int32_t* new_seq_lens;        // optional
  int B, N, hq, hkv, d, tmax;
};

struct AppendParams {
  NewTokens t;
  KvView kv;
  int kv_f32;
  int per_wg, slots, slot_groups;    // tokens and heads of a workgroup, groups of heads (set by the launcher)
  int first_wg;                 // the launch's first workgroup
};

struct Append8Params {
  NewTokens t;
  KvView kv;
  float* k_scale;
  float* v_scale;
  // set by the launcher
  int q_groups, per_wg, slots, slot_groups;     // workgroups that rotate queries, as above
  int blocks, items;            // blocks that a row's new tokens can touch; (head, K or V) items of a workgroup
};

struct Unpack8Params {
  KvView src, dst;
  const float* k_scale;
  const float* v_scale;
  const int32_t* seq_lens;
  int B, hkv, d, tmax, first, num, f32;
  int first_row;                // the launch's first row (set by the launcher)
};

struct Decode8Params {
  TreeParams t;                 // (kv: places of codes, one byte an element)
  const float* k_scale;
  const float* v_scale;
  unsigned* counters;           // of each (row, KV head), if the last workgroup joins its parts; else null
};

hipError_t launch_append(const AppendParams& p, hipStream_t st);
hipError_t launch_append8(const Append8Params& p, hipStream_t st);
hipError_t launch_unpack8(const Unpack8Params& p, hipStream_t st);
// Row tiles, splits and workspace of a call, from its shape alone.
size_t decode8_workspace(const AttendParams& a);
hipError_t launch_decode8(const Decode8Params& p, hipStream_t st);

}  // namespace cobs
