// Which tokens a cache keeps (cobs_evict): per (batch row, KV head) the first and
// the last tokens and the `need` largest weights of those between, in order.
//
// Radix search over order-preserving 32-bit keys in digits of 11, 11 and 10 bits
// from the top: the histogram of the keys that share the digits found so far gives
// the digit of the need-th largest key and how many keys above it are kept.  After
// three digits the key itself is known; every larger one is kept, and the first
// of the equal ones.
//
// A workgroup of 16 waves holds a chunk of up to 32768 keys in registers (wave w a
// run of 64 KPT positions, so ranks come from ballots and one sum over waves).
// Rows of up to 32768 positions are done by one launch.  Longer ones take four: each
// writes the chunks' histograms of one digit (16-bit counts, 4 KB a chunk), and the
// next sums them in every workgroup, which costs less than a wait between
// workgroups, needs no atomics across them and no cleared memory; what it found
// goes on to the launch after it in a state per chunk.  The last one's sums over
// the chunks before a workgroup's own are its ranks.
//
// Bound by what one CU does with its chunk (loads, atomics in LDS, barriers): 9 to 16
// us a launch with chunks of 32768, whatever the rows; so few rows take smaller
// chunks, as long as there is a CU for each (evict_keys).  64 rows of 131072:
// 47.6 us, the four reads at 2.8 TB/s; 8 rows: 23 us (38 with chunks of 32768).
// Many long rows: 256 of 131072 in 166 us, 3.2 TB/s.
#include "cache_device.h"

namespace cobs {

constexpr int kEvictThreads = 1024, kEvictWaves = 16;
constexpr int kEvictRow = 32768;                             // the longest row of one launch
constexpr int kBins = 2048;                                  // of a digit; the last has 1024
constexpr int kChunkHist = (2 * kBins + kBins / 2);          // 16-bit counts of a chunk: three digits
__device__ __forceinline__ int digit_shift(int lv) { return lv == 0 ? 21 : (lv == 1 ? 10 : 0); }
__device__ __forceinline__ int digit_bins(int lv) { return lv == 2 ? kBins / 2 : kBins; }

// Larger weight, larger key; NaN with -inf.  -0 and 0 are one weight.
__device__ __forceinline__ uint32_t weight_key(float w) {
  if (w != w) w = -INFINITY;
  return order_key(w + 0.0f);
}

// Set bits of a ballot below this lane.
__device__ __forceinline__ int lanes_below(unsigned long long m) {
  return __builtin_amdgcn_mbcnt_hi((uint32_t)(m >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)m, 0));
}

// Sum over the wave, in every lane; all lanes active.
__device__ __forceinline__ int wave_total(int x) { return __builtin_amdgcn_readlane(wave_incl_scan(x), 63); }

static_assert(kBins == 2 * kEvictThreads, "two 16-bit counts a thread");
struct EvictShared {
  int hist[kBins];
  int wsum[kEvictWaves];
  int digit, left;
};

// Sum over the workgroup of x, and over the waves before this one (barriers inside).
__device__ __forceinline__ int sum_before(int x, int* wsum, int wave, int lane, int& before) {
  const int inc = wave_incl_scan(x);
  if (lane == 63) wsum[wave] = inc;
  __syncthreads();
  int all = 0;
  before = 0;
#pragma unroll
  for (int i = 0; i < kEvictWaves; ++i) {
    const int v = wsum[i];
    before += i < wave ? v : 0;
    all += v;
  }
  __syncthreads();
  return all;
}

constexpr int kBpt = kBins / kEvictThreads;                  // bins of a thread: kBpt tid ..

// The digit that holds the need-th largest key, from this thread's counts of its bins; `need` becomes
// what is still needed of that digit's keys.
__device__ __forceinline__ int find_digit(const int (&c)[kBpt], int& need, EvictShared& s, int wave, int lane) {
  int v = 0;
#pragma unroll
  for (int i = 0; i < kBpt; ++i) v += c[i];
  const int inc = wave_incl_scan(v);
  int before;
  const int all = sum_before(v, s.wsum, wave, lane, before);
  int after = all - before - inc;                            // keys in higher bins than this thread's
  if (after < need && need <= after + v) {
#pragma unroll
    for (int i = kBpt - 1; i >= 0; --i) {
      if (after < need && need <= after + c[i]) {
        s.digit = kBpt * threadIdx.x + i;
        s.left = need - after;
      }
      after += c[i];
    }
  }
  __syncthreads();
  const int d = s.digit;
  need = s.left;
  __syncthreads();
  return d;
}

// LV 0..2: the launch of that digit; 3: the last launch; 4: all of it for rows of one chunk.
template <int KPT, int LV>
__global__ __launch_bounds__(kEvictThreads) void evict_kernel(EvictParams p) {
  __shared__ EvictShared s;
  const int chunk = blockIdx.x, h = blockIdx.y, b = blockIdx.z;
  const int tid = threadIdx.x, lane = tid & 63, wave = wave_uniform32(tid >> 6);
  const int T = clamp_len(p.seq_lens[b], p.tmax), unit = b * p.hkv + h;
  const float* w = p.weights + (int64_t)unit * p.tmax;
  int32_t* out = p.kept + (int64_t)unit * p.keep;
  constexpr bool LAST = LV >= 3;
  if (LAST && p.new_lens && chunk == 0 && h == 0 && tid == 0) p.new_lens[b] = min(T, p.keep);
  if (T <= p.keep) {
    if (LAST)
      for (int j = chunk * kEvictThreads + tid; j < p.keep; j += gridDim.x * kEvictThreads) out[j] = j < T ? j : -1;
    return;
  }
  constexpr int CHUNK = KPT * kEvictThreads;
  const int t_first = chunk * CHUNK;
  if (t_first >= T) return;
  const int nch = (T + CHUNK - 1) / CHUNK;
  const int lo = p.sinks, hi = T - p.recent;                 // the tokens to choose from
  int need = p.keep - p.sinks - p.recent;                    // fewer than those: T > keep
  const bool choose = need > 0;

  // (the weights' bits until the digits are found, so that their loads run meanwhile)
  uint32_t key[KPT];
  const int t_wave = t_first + wave * 64 * KPT, t0 = t_wave + lane;
  const bool inner = t_wave >= lo && t_wave + 64 * KPT <= hi;        // the wave's positions are all to choose from
  if (inner) {
#pragma unroll
    for (int i = 0; i < KPT; ++i) key[i] = __float_as_uint(w[t0 + 64 * i]);
  } else {
#pragma unroll
    for (int i = 0; i < KPT; ++i) {
      const int t = t0 + 64 * i;
      key[i] = (t >= lo && t < hi) ? __float_as_uint(w[t]) : 0;
    }
  }

  auto make_keys = [&] {
#pragma unroll
    for (int i = 0; i < KPT; ++i) key[i] = weight_key(__uint_as_float(key[i]));
  };
  if (LV == 4) make_keys();

  // histogram of digit `lv` of the chunk's keys that share the digits above it, in s.hist
  auto count = [&](int lv, uint32_t prefix) {
    for (int i = tid; i < kBins; i += kEvictThreads) s.hist[i] = 0;
    __syncthreads();
    const int sh = digit_shift(lv), up = sh + (lv == 2 ? 10 : 11);
#pragma unroll
    for (int i = 0; i < KPT; ++i) {
      const int t = t0 + 64 * i;
      const bool in = (inner || (t >= lo && t < hi)) && (lv == 0 || (key[i] >> up) == (prefix >> up));
      if (in) atomicAdd(&s.hist[(key[i] >> sh) & (digit_bins(lv) - 1)], 1);
    }
    __syncthreads();
  };
  uint32_t prefix = 0;
  int above = 0, equal = 0;                                  // kept, and equal keys, of the chunks before
  uint16_t* hists = p.hist + (int64_t)unit * p.chunks * kChunkHist;
  EvictState* const states = p.state + (int64_t)unit * p.chunks;
  if (choose) {
    int over_here = 0;                                       // the chunk's keys above the digits found by earlier launches
    if (LV == 2 || LV == 3) {
      const EvictState e = states[chunk];
      prefix = e.prefix;
      need = e.need;
      over_here = e.over;
    }
#pragma unroll 1
    for (int lv = LV == 4 || LV == 0 ? 0 : LV - 1; lv < (LV == 4 ? 3 : LV); ++lv) {
      int c[kBpt], before_c[kBpt], own_c[kBpt];              // all chunks; those before this one; this one
#pragma unroll
      for (int i = 0; i < kBpt; ++i) c[i] = before_c[i] = own_c[i] = 0;
      if (LV == 4) {
        count(lv, prefix);
#pragma unroll
        for (int i = 0; i < kBpt; ++i) c[i] = s.hist[kBpt * tid + i];
      } else if (kBpt * tid < digit_bins(lv)) {
#pragma unroll 4
        for (int k = 0; k < nch; ++k) {
          const uint32_t x = reinterpret_cast<const uint32_t*>(hists + k * kChunkHist + lv * kBins)[tid];
          const int n[kBpt] = {(int)(x & 0xffff), (int)(x >> 16)};
#pragma unroll
          for (int i = 0; i < kBpt; ++i) {
            c[i] += n[i];
            before_c[i] += k < chunk ? n[i] : 0;
            own_c[i] += k == chunk ? n[i] : 0;
          }
        }
      }
      const int d = find_digit(c, need, s, wave, lane);
      prefix |= (uint32_t)d << digit_shift(lv);
      if (LV == 1 || LV == 2) {
        // what the launches after need of this digit
        int over = 0, before;
#pragma unroll
        for (int i = 0; i < kBpt; ++i) over += kBpt * tid + i > d ? own_c[i] : 0;
        over = sum_before(over, s.wsum, wave, lane, before);
        if (tid == 0) states[chunk] = {prefix, need, over_here + over, 0};
      }
      if (LV == 3) {
        int over = 0, same = 0, before;
#pragma unroll
        for (int i = 0; i < kBpt; ++i) {
          over += kBpt * tid + i > d ? before_c[i] : 0;
          same += kBpt * tid + i == d ? before_c[i] : 0;
        }
        for (int k = tid; k < chunk; k += kEvictThreads) over += states[k].over;
        above = sum_before(over, s.wsum, wave, lane, before);
        equal = sum_before(same, s.wsum, wave, lane, before);
      }
    }
    if (LV < 4) make_keys();
    if (LV < 3) {
      count(LV, prefix);
      if (kBpt * tid < digit_bins(LV)) {
        const int* n = s.hist + kBpt * tid;
        reinterpret_cast<uint32_t*>(hists + chunk * kChunkHist + LV * kBins)[tid] = (uint32_t)n[0] | ((uint32_t)n[1] << 16);
      }
      return;
    }
  }
  if constexpr (LAST) {
    // Keep the ends, every key above `prefix` and the first `need` equal to it.  Bit i
    // of a lane's masks is its key i; ranks inside a wave go by i, then by lane.
    uint32_t take = 0, same = 0;
    if (inner && choose) {
#pragma unroll
      for (int i = 0; i < KPT; ++i) {
        take |= (key[i] > prefix ? 1u : 0u) << i;
        same |= (key[i] == prefix ? 1u : 0u) << i;
      }
    } else {
#pragma unroll
    for (int i = 0; i < KPT; ++i) {
      const int t = t0 + 64 * i;
      const bool mid = t >= lo && t < hi;
      take |= (t < T && (!mid || (choose && key[i] > prefix)) ? 1u : 0u) << i;
      same |= (choose && mid && key[i] == prefix ? 1u : 0u) << i;
    }
    }
    const int mine = wave_total(__popc(same));
    int eq;
    sum_before(lane == 0 ? mine : 0, s.wsum, wave, lane, eq);
    eq += equal;
    if (mine > 0 && eq < need) {
      if (eq + mine <= need) {
        take |= same;
      } else {                                   // the wave where they run out
#pragma unroll
        for (int i = 0; i < KPT; ++i) {
          const unsigned long long eqs = __ballot((same >> i) & 1u);
          if (((same >> i) & 1u) && eq + lanes_below(eqs) < need) take |= 1u << i;
          eq += __popcll(eqs);
        }
      }
    }
    const int taken = wave_total(__popc(take));
    int at;
    sum_before(lane == 0 ? taken : 0, s.wsum, wave, lane, at);
    // chunks before this one: their ends, keys above and kept equal ones
    if (chunk > 0) at += min(lo, t_first) + max(0, t_first - hi) + above + min(equal, choose ? need : 0);
#pragma unroll
    for (int i = 0; i < KPT; ++i) {
      const unsigned long long tk = __ballot((take >> i) & 1u);
      if ((take >> i) & 1u) out[at + lanes_below(tk)] = t0 + 64 * i;
      at += __popcll(tk);
    }
  }
}

// Keys of a thread: the smallest chunks that are one a CU and at most 32 a row, whose histograms
// every workgroup of the row sums.  (us with chunks of 8192, 16384, 32768: 8 rows of 131072 23, 26, 38;
// 64 of 65000 32, 29, 40, and of 131072 62, 53, 48; 1 of 500000 38, 33, 37; 256 of 131072 200, 164, 166.)
static int evict_keys(int B, int hkv, int tmax) {
  if (tmax <= kEvictRow) return tmax <= 4 * kEvictThreads ? 4 : (tmax <= 16 * kEvictThreads ? 16 : 32);
  for (int keys = 8; keys < 32; keys *= 2) {
    const int64_t n = (tmax + keys * kEvictThreads - 1) / (keys * kEvictThreads);
    if (n <= 32 && n * B * hkv <= 256) return keys;
  }
  return 32;
}

static int evict_chunks(int B, int hkv, int tmax) {
  const int chunk = evict_keys(B, hkv, tmax) * kEvictThreads;
  return (tmax + chunk - 1) / chunk;
}

size_t evict_workspace(int B, int hkv, int tmax) {
  const int n = evict_chunks(B, hkv, tmax);
  return n == 1 ? 0 : ((size_t)B * hkv * n * (kChunkHist * sizeof(uint16_t) + sizeof(EvictState)) + 255) / 256 * 256;
}

template <int KPT>
static hipError_t launch_long_rows(const EvictParams& p, dim3 grid, hipStream_t st) {
  const dim3 t(kEvictThreads);
  hipLaunchKernelGGL((evict_kernel<KPT, 0>), grid, t, 0, st, p);
  hipLaunchKernelGGL((evict_kernel<KPT, 1>), grid, t, 0, st, p);
  hipLaunchKernelGGL((evict_kernel<KPT, 2>), grid, t, 0, st, p);
  hipLaunchKernelGGL((evict_kernel<KPT, 3>), grid, t, 0, st, p);
  return hipGetLastError();
}

hipError_t launch_evict(const EvictParams& q, hipStream_t st) {
  EvictParams p = q;
  const int keys = evict_keys(p.B, p.hkv, p.tmax);
  p.chunks = evict_chunks(p.B, p.hkv, p.tmax);
  const dim3 grid(p.chunks, p.hkv, p.B), t(kEvictThreads);
  if (p.chunks == 1) {
    if (keys == 4) hipLaunchKernelGGL((evict_kernel<4, 4>), grid, t, 0, st, p);
    else if (keys == 16) hipLaunchKernelGGL((evict_kernel<16, 4>), grid, t, 0, st, p);
    else hipLaunchKernelGGL((evict_kernel<32, 4>), grid, t, 0, st, p);
    return hipGetLastError();
  }
  p.state = reinterpret_cast<EvictState*>(p.hist + (size_t)p.B * p.hkv * p.chunks * kChunkHist);
  if (keys == 8) return launch_long_rows<8>(p, grid, st);
  if (keys == 16) return launch_long_rows<16>(p, grid, st);
  return launch_long_rows<32>(p, grid, st);
}

}  // namespace cobs
