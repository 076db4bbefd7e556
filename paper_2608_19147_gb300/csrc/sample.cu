// Sampling from logits with given random numbers (include/head.h).
//
// A row belongs to a cluster of CTAs and is read once: its logits stay in shared
// memory, and all later passes go over those.  With x the logits and m their
// maximum, a token weighs w(x) = 2^((x - m) log2(e) / T), as a whole number of 2^-44
// parts of the largest, so that sums are exact and no split of the row changes
// them.  The kept tokens are a prefix of the order by falling logit and rising id:
// a threshold `edge`, and how many of its ties.
//   1. maximum, minimum, greedy token
//   2. a histogram of count (top_k) or of count and mass (top_p) over the values;
//      if the bins that may hold kept tokens have no more than 512, these go to one
//      CTA, which ranks them and draws
//   3. otherwise the thresholds of min_p, top_k and top_p in turn, each by
//      histograms within the bin where it lies, until all of a bin are equal, and
//      the mass of what is kept
//   4. the first id whose cumulated kept mass exceeds u times all of it
// What the CTAs tell each other goes by cluster barriers and reads of the others'
// shared memory.
//
// Measured (GB300, calls replayed, rows of 128256): one row with top_k 50 and top_p 0.9
// 12.5 us, 16 rows with settings of their own 52.5, 256 rows of bf16 with top_p 0.95 and
// min_p 0.02 118 (0.55 TB/s), 16 rows without filters 24, with top_p 0.9 alone 80.  A row's
// chain of barriers and passes bounds it, not memory: a cluster barrier is 900 cycles, the
// first histogram of a CTA's 8192 tokens 2500 (its atomics), a pass over exact weights 14000.
// 64 registers, so that two CTAs fit an SM, spill 128 to 152 bytes a thread, also in the
// launches that have one CTA to an SM.
#include <cooperative_groups.h>
#include <cuda_bf16.h>

#include <algorithm>
#include <atomic>
#include <cmath>
#include <cstdarg>
#include <cstdio>

#include "../../include/head.h"
#include "launch.cuh"
#include "sample.cuh"

namespace shard {
int shard_fail_msg(int code, const char* msg);
}  // namespace shard

using namespace shard;
namespace cg = cooperative_groups;

namespace {

constexpr int kThreads = 512, kWarps = kThreads / 32, kMaxCluster = 16;
constexpr int kBlock = 4 * kThreads, kMaxBlocks = 16;  // tokens per block; blocks per CTA
constexpr int kBins = kThreads;  // a thread each; the last one is for what lies below the others
constexpr int kList = kThreads;  // candidates that one CTA ranks, a thread each
constexpr int kScale = 44;  // the largest weight is 2^44: 2^19 of them fit
static_assert(HEAD_MAX_SAMPLE_VOCAB == kBlock * kMaxBlocks * kMaxCluster, "a row's logits in shared memory");

// Order of the values as whole numbers.
__device__ __forceinline__ uint32_t key_of(float x) {
  const uint32_t u = __float_as_uint(x);
  return u ^ ((uint32_t)((int32_t)u >> 31) | 0x80000000u);
}
__device__ __forceinline__ float of_key(uint32_t k) { return __uint_as_float(k & 0x80000000u ? k ^ 0x80000000u : ~k); }
constexpr uint32_t kKeyNone = 0x007FFFFFu;  // of minus infinity: never chosen

// 2^x with relative error 2^-22.
__device__ __forceinline__ float exp2_rough(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

// Weights: 2^(k / 64 + r) with k whole and |r| <= 1/128, 2^(k mod 64 / 64) as two
// floats from a table and 2^r - 1 by its series (the table-driven exponential
// of P. T. P. Tang, ACM TOMS 15, 1989).  The argument is kept in two floats.  Errors relative to the weight: 2^-30.2 of r
// log(2) and 2^-30 of the series in 32 bits, 2^-31 of its product with the table's value: under 2^-28.7, and half a unit of
// 2^-44.  A weight comes as two whole numbers of 22 bits and a sign: integer instructions run at half the rate of
// 32-bit floats or less, and 64-bit shifts and sums take several (256 rows of 16 bits without filters 133 -> 127 us).
// Whole numbers come from the low bits of a float around 1.5 * 2^23.
struct Weights {
  float max, c_hi, c_lo;  // c: log2(e) / T
  const float2* table;    // [64] in shared memory
  struct Parts {          // high * 2^kLow + low, |low| < 2^kLow
    int high, low;
  };
  static constexpr int kLow = kScale / 2, kMagicBits = 0x4B400000;
  static_assert(kScale == 2 * kLow, "parts of the same size");
  __device__ __forceinline__ Parts parts(float x) const {
    constexpr float kMagic = 12582912.f;
    const float s = __fadd_rn(x, -max), b = __fadd_rn(s, -x);
    const float e = __fadd_rn(__fadd_rn(x, -__fadd_rn(s, -b)), -__fadd_rn(max, b));  // x - max is s + e
    const float t = __fmul_rn(s, c_hi);
    const float lo = __fmaf_rn(e, c_hi, __fmaf_rn(s, c_lo, __fmaf_rn(s, c_hi, -t)));
    const float kf = __fmaf_rn(t, 64.f, kMagic);
    const float y = __fmul_rn(__fadd_rn(__fmaf_rn(__fadd_rn(kf, -kMagic), -1.f / 64.f, t), lo), 0.693147180559945f);
    const float series = __fmul_rn(y, __fmaf_rn(y, __fmaf_rn(y, 1.f / 6.f, 0.5f), 1.f));
    const uint32_t k = __float_as_uint(kf);
    const float2 base = table[k & 63];
    const float scale = __uint_as_float(((k << 17) & 0xFF800000u) + ((127u + kLow) << 23));  // 2^kLow of it
    const float rest = __fmaf_rn(base.x, series, base.y), v = __fadd_rn(base.x, rest), v_lo = __fadd_rn(rest, -__fadd_rn(v, -base.x));
    const float up = __fmul_rn(v, scale), high = __fadd_rn(up, kMagic);
    const float down = __fadd_rn(__fadd_rn(up, -__fadd_rn(high, -kMagic)), __fmul_rn(v_lo, scale));
    const float low = __fmaf_rn(down, (float)(1 << kLow), kMagic);
    const bool any = t > -46.f;  // else under half a unit, or what is no number here
    return Parts{any ? __float_as_int(high) - kMagicBits : 0, any ? __float_as_int(low) - kMagicBits : 0};
  }
  static __device__ __forceinline__ uint64_t joined(int high, int low) { return (uint64_t)(((int64_t)high << kLow) + low); }
  __device__ __forceinline__ uint64_t operator()(float x) const {
    const Parts p = parts(x);
    return joined(p.high, p.low);
  }
};

// Sum over the lanes of values below 2^63 / 32 in three parts: a reduction of 32 bits is one instruction, a shuffle of
// 64 takes ten.
__device__ __forceinline__ uint64_t warp_sum(uint64_t v) {
  const uint32_t a = __reduce_add_sync(0xffffffffu, (uint32_t)v & 0xFFFFFFu), b = __reduce_add_sync(0xffffffffu, (uint32_t)(v >> 24) & 0xFFFFFFu),
                 c = __reduce_add_sync(0xffffffffu, (uint32_t)(v >> 48));
  return a + ((uint64_t)b << 24) + ((uint64_t)c << 48);
}
// Inclusive sums over the lanes.
template <class T>
__device__ __forceinline__ T warp_scan(T v, int lane) {
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const T x = __shfl_up_sync(0xffffffffu, v, o);
    if (lane >= o) v += x;
  }
  return v;
}

// floor or ceiling of v * share, share in [0, 1) a float
__device__ __forceinline__ uint64_t share_of(uint64_t v, float share, bool up) {
  const uint32_t bits = __float_as_uint(share);
  const int shift = (int)(bits >> 23) - 86;  // share = mantissa * 2^(shift - 64)
  const uint64_t mantissa = bits & 0x7FFFFFu | 0x800000u, q = shift >= 0 ? mantissa << shift : shift > -24 ? mantissa >> -shift : 0;
  return __umul64hi(v, q) + (up && v * q != 0);
}

// A logit: minus infinity for NaN, and one zero.
__device__ __forceinline__ float plain(float x) { return fmaxf(x, -INFINITY) + 0.f; }
template <int kType>
__device__ __forceinline__ float logit(const void* row, int v) {
  if (kType == SHARD_F32) return plain(__ldg(static_cast<const float*>(row) + v));
  if (kType == SHARD_F16) return plain(__half2float(static_cast<const __half*>(row)[v]));
  return plain(__bfloat162float(static_cast<const __nv_bfloat16*>(row)[v]));
}

// Four tokens in shared memory, in the logits' own bits.
template <int kType>
struct Four {
  using T = uint2;
  static __device__ __forceinline__ float4 get(uint2 v) {
    if (kType == SHARD_F16) {
      const float2 a = __half22float2(*reinterpret_cast<const __half2*>(&v.x)), b = __half22float2(*reinterpret_cast<const __half2*>(&v.y));
      return make_float4(a.x, a.y, b.x, b.y);
    }
    return make_float4(__uint_as_float(v.x << 16), __uint_as_float(v.x & 0xFFFF0000u), __uint_as_float(v.y << 16),
                       __uint_as_float(v.y & 0xFFFF0000u));
  }
  static __device__ __forceinline__ uint2 put(float4 f) {  // of values that the type has
    if (kType == SHARD_F16) {
      const __half2 a = __floats2half2_rn(f.x, f.y), b = __floats2half2_rn(f.z, f.w);
      return make_uint2(*reinterpret_cast<const uint32_t*>(&a), *reinterpret_cast<const uint32_t*>(&b));
    }
    return make_uint2(__byte_perm(__float_as_uint(f.x), __float_as_uint(f.y), 0x7632),
                      __byte_perm(__float_as_uint(f.z), __float_as_uint(f.w), 0x7632));
  }
};
template <>
struct Four<SHARD_F32> {
  using T = float4;
  static __device__ __forceinline__ float4 get(float4 v) { return v; }
  static __device__ __forceinline__ float4 put(float4 f) { return f; }
};

struct SampleArgs {
  const void* logits;
  int V, blocks;
  long long ld;
  head_sampling s;
  int32_t* token;
  float* p;
  int32_t* n_kept;
  const int* failed;  // nonzero: the logits are not to be used
};

// What a CTA (first a lane, then a warp) tells the others.
struct Told {
  uint64_t mass[2];
  uint32_t count[2], hi, lo;
  int id;  // the lowest that has hi
};
constexpr uint32_t kAll = 0xffffffffu;
__device__ __forceinline__ Told nothing() { return Told{{0, 0}, {0, 0}, 0, kAll, 0x7fffffff}; }
// Over the lanes: sums, the largest hi, the smallest lo; the rest is not looked at.
enum { kBounds = 1, kIds = 2, kCount = 4, kMass = 8, kAllMass = 16 };
template <int kWhat>
__device__ __forceinline__ Told join(Told t) {
  if (kWhat & kMass) t.mass[0] = warp_sum(t.mass[0]);
  if (kWhat & kAllMass) t.mass[1] = warp_sum(t.mass[1]), t.count[1] = __reduce_add_sync(0xffffffffu, t.count[1]);
  if (kWhat & kCount) t.count[0] = __reduce_add_sync(0xffffffffu, t.count[0]);
  if (kWhat & (kBounds | kIds)) {
    const uint32_t hi = __reduce_max_sync(0xffffffffu, t.hi);
    if (kWhat & kIds) t.id = __reduce_min_sync(0xffffffffu, t.hi == hi ? t.id : 0x7fffffff);
    t.hi = hi;
    t.lo = __reduce_min_sync(0xffffffffu, t.lo);
  }
  return t;
}

struct Shared {
  float2 table[64];
  Weights w;
  Told told[2];  // in turn: an exchange is over before the next but one is written
  Told warp[kWarps], sum, lower;
  double bound;    // T log(min_p)
  uint32_t least;  // the min_p threshold
  struct Hist {
    uint32_t count[kBins], limb[3][kBins];  // mass in 16-bit parts: 2^16 additions fit
  } hist[2];
  uint32_t count[kBins], part_count[kBins];  // of the row; of one bin in one CTA
  uint64_t mass[kBins], part_mass[kBins];
  uint64_t scan_mass[kWarps], found_mass, all_mass;
  uint32_t scan_count[kWarps], found, found_count, found_there, n_list;
  uint64_t part[kMaxBlocks][kWarps];  // kept mass of a block's warps
  uint32_t ties[kMaxBlocks][kWarps];  // ties of lower ids than a block's warp has
  struct Candidate {
    uint32_t key;
    int id;
    uint64_t weight;
  } list[kList];
  uint32_t own[kList];  // this CTA's keys of one bin
};

__device__ __forceinline__ void sync_row(const cg::cluster_group& cluster, int n_cta) {
  if (n_cta > 1) cluster.sync();
  else __syncthreads();
}

// Every lane's `mine` over the row: sh.sum is all of it, sh.lower that of the CTAs of lower rank.
template <int kWhat>
__device__ __noinline__ void exchange(Shared& sh, int turn, Told mine, int n_cta, int rank) {
  const cg::cluster_group cluster = cg::this_cluster();
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  mine = join<kWhat>(mine);
  if (lane == 0) sh.warp[warp] = mine;
  __syncthreads();
  if (warp == 0) {
    const Told t = join<kWhat>(lane < kWarps ? sh.warp[lane] : nothing());
    if (lane == 0) {
      sh.told[turn] = t;
      if (n_cta == 1) sh.sum = t, sh.lower = nothing();
    }
  }
  if (n_cta > 1) {
    cluster.sync();
    if (warp < 2) {
      const bool take = warp == 0 ? lane < n_cta : lane < rank;
      const Told t = join<kWhat>(take ? *cluster.map_shared_rank(&sh.told[turn], lane) : nothing());
      if (lane == 0) (warp == 0 ? sh.sum : sh.lower) = t;
    }
  }
  __syncthreads();
}

// Bins of the keys of [lo, hi] by value: the first and the last of them have one at least unless all are equal, so
// that every level narrows.
struct Bins {
  uint32_t lo, hi;
  float x_hi, per_value;
  __device__ __forceinline__ Bins(uint32_t lo, uint32_t hi) : lo(lo), hi(hi), x_hi(of_key(hi)) {
    per_value = 0.5f * (kBins - 1) / (0.5f * x_hi - 0.5f * of_key(lo));
  }
  __device__ __forceinline__ uint32_t operator()(float v) const {
    return lo == hi ? 0u : min((uint32_t)(kBins - 2), __float2uint_rz((x_hi - v) * per_value));
  }
  // No value of the bin is below `least` or above `most`: the product above is off by 2^-23 of it at most, the terms here
  // by less than the margin (1e-35 covers what underflows).
  __device__ __forceinline__ float margin(float way) const { return fmaf(way, 0x1p-20f, fmaf(fabsf(x_hi), 0x1p-20f, 1e-35f)); }
  __device__ __forceinline__ float least(int bin) const {
    const float way = (float)(bin + 1) / per_value;
    return bin >= kBins - 2 ? of_key(lo) : fmaxf(of_key(lo), x_hi - way - margin(way));
  }
  __device__ __forceinline__ float most(int bin) const {
    const float way = (float)bin / per_value;
    return fminf(x_hi, x_hi - way + margin(way));
  }
};

// sh.count and, by mass, sh.mass: those of the row's bins.  In the last bin the mass of the keys below lo, roughly, and in
// place of their count a bound of its error in parts of 2^12.  With t = (x - max) c in 32 bits, a weight 2^t is off by
// 2.5 |t| log(2) 2^-24 (the difference, the product and c) and the instruction's 2^-22, sums of 18 terms by 17 * 2^-24:
// (2 |t| + 24) 2^-24 of it; the sum of |t| 2^t is taken along.
template <class F>
__device__ __noinline__ void histogram(Shared& sh, const typename F::T* xs, int blocks, uint32_t lo, uint32_t hi, bool by_mass, int level,
                                       int n_cta, int rank) {
  const cg::cluster_group cluster = cg::this_cluster();
  const int tid = threadIdx.x, lane = tid & 31;
  const Bins bins(lo, hi);
  const Weights w = sh.w;
  Shared::Hist& h = sh.hist[level & 1];
  h.count[tid] = h.limb[0][tid] = h.limb[1][tid] = h.limb[2][tid] = 0;
  if (tid == 0) sh.n_list = 0;
  __syncthreads();
  const float x_lo = of_key(lo), x_hi = of_key(hi);
  float rest[4] = {0.f, 0.f, 0.f, 0.f}, rest_t[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll 1
  for (int j = 0; j < blocks; ++j) {
    const float4 f = F::get(xs[j * kThreads + tid]);
    const float x[4] = {f.x, f.y, f.z, f.w};
    if (by_mass) {
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const float t = fmaxf((x[e] - w.max) * w.c_hi, -127.f), y = exp2_rough(t);
        if (x[e] < x_lo) rest[e] += y, rest_t[e] = fmaf(t, y, rest_t[e]);
      }
    }
    if (!__any_sync(0xffffffffu, fmaxf(fmaxf(x[0], x[1]), fmaxf(x[2], x[3])) >= x_lo)) continue;
    bool in[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) in[e] = x[e] >= x_lo && x[e] <= x_hi;
    uint64_t one[4];
    if (by_mass)
#pragma unroll
      for (int e = 0; e < 4; ++e) one[e] = w(x[e]);
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      if (!in[e]) continue;
      const uint32_t bin = bins(x[e]);
      atomicAdd(&h.count[bin], 1u);
      if (by_mass) {
        atomicAdd(&h.limb[0][bin], (uint32_t)one[e] & 0xFFFFu);
        atomicAdd(&h.limb[1][bin], (uint32_t)(one[e] >> 16) & 0xFFFFu);
        atomicAdd(&h.limb[2][bin], (uint32_t)(one[e] >> 32));
      }
    }
  }
  if (by_mass) {
    const float all = (rest[0] + rest[1]) + (rest[2] + rest[3]), all_t = (rest_t[0] + rest_t[1]) + (rest_t[2] + rest_t[3]);
    const uint64_t mass = warp_sum((uint64_t)(all * (float)(1ull << kScale)));
    const uint32_t off = __reduce_add_sync(0xffffffffu, __float2uint_ru(fmaf(-2.f, all_t, 24.f * all) * (float)(1 << (kScale - 24 - 12))));
    if (lane == 0 && off) {
      atomicAdd(&h.limb[0][kBins - 1], (uint32_t)mass & 0xFFFFu);
      atomicAdd(&h.limb[1][kBins - 1], (uint32_t)(mass >> 16) & 0xFFFFu);
      atomicAdd(&h.limb[2][kBins - 1], (uint32_t)(mass >> 32));
      atomicAdd(&h.count[kBins - 1], off);
    }
  }
  sync_row(cluster, n_cta);
  // This CTA adds up its share of the bins, a thread for each CTA's part of each, and tells all of them the sums.
  const int per = kBins / n_cta, i = tid % per, r = tid / per, bin = rank * per + i;
  const Shared::Hist* o = cluster.map_shared_rank(&h, r);
  uint32_t c = o->count[bin];
  uint64_t mass = by_mass ? o->limb[0][bin] + ((uint64_t)o->limb[1][bin] << 16) + ((uint64_t)o->limb[2][bin] << 32) : 0;
  if (n_cta > 1) {
    sh.part_count[tid] = c;
    sh.part_mass[tid] = mass;
    __syncthreads();
    c = 0;
    mass = 0;
#pragma unroll
    for (int q = 0; q < kMaxCluster; ++q)
      if (q < n_cta) c += sh.part_count[q * per + i], mass += sh.part_mass[q * per + i];
  }
  Shared* to = cluster.map_shared_rank(&sh, r);
  to->count[bin] = c;
  to->mass[bin] = mass;
  sync_row(cluster, n_cta);
}

// The CTAs' keys (sh.own, sh.n_list) into sh.list, kList at most in all, after a sync_row; the next one comes before
// one's keys may change.  (An atomic of another CTA's counter takes a round trip.)
__device__ __noinline__ void gather(Shared& sh, int n_cta) {
  const cg::cluster_group cluster = cg::this_cluster();
  const int tid = threadIdx.x, lane = tid & 31;
  const uint32_t there = lane < n_cta ? *cluster.map_shared_rank(&sh.n_list, lane) : 0, upto = warp_scan(there, lane);
  int r = 0;
  uint32_t base = 0;
#pragma unroll
  for (int i = 0; i < kMaxCluster; ++i) {
    const uint32_t end = __shfl_sync(0xffffffffu, upto, i);
    if ((uint32_t)tid >= end) ++r, base = end;
  }
  if (r < n_cta) sh.list[tid].key = *cluster.map_shared_rank(&sh.own[tid - base], r);
  __syncthreads();
}

// The sum over the row of all weights, by one CTA, from memory.
template <int kType>
__device__ __noinline__ uint64_t sum_of_row(Shared& sh, const char* row, int V) {
  const Weights w = sh.w;
  uint64_t s = 0;
#pragma unroll 1
  for (int v = threadIdx.x; v < V; v += 8 * kThreads) {
    float x[8];
#pragma unroll
    for (int i = 0; i < 8; ++i) x[i] = v + i * kThreads < V ? logit<kType>(row, v + i * kThreads) : -INFINITY;
#pragma unroll
    for (int i = 0; i < 8; ++i) s += x[i] > -INFINITY ? w(x[i]) : 0;
  }
  s = warp_sum(s);
  __syncthreads();
  if (threadIdx.x % 32 == 0) sh.scan_mass[threadIdx.x / 32] = s;
  __syncthreads();
  s = 0;
  for (int i = 0; i < kWarps; ++i) s += sh.scan_mass[i];
  __syncthreads();
  return s;
}

// The bin where the rank or the mass is reached, among those of sh.count and sh.mass: sh.found, with its count, and the
// count and mass above it; kBins where it is not.
__device__ __noinline__ void reach(Shared& sh, bool by_mass, uint32_t above, uint64_t above_mass, uint32_t rank_goal, uint64_t mass_goal) {
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const uint32_t c = sh.count[tid], uc = warp_scan(c, lane);
  const uint64_t m = sh.mass[tid], um = warp_scan(m, lane);
  if (lane == 31) sh.scan_count[warp] = uc, sh.scan_mass[warp] = um;
  if (tid == 0) sh.found = kBins;
  __syncthreads();
  uint32_t pc = above + uc - c;
  uint64_t pm = above_mass + um - m;
#pragma unroll
  for (int i = 0; i < kWarps - 1; ++i)
    if (i < warp) pc += sh.scan_count[i], pm += sh.scan_mass[i];
  if (by_mass ? pm < mass_goal && pm + m >= mass_goal : pc < rank_goal && pc + c >= rank_goal) {
    sh.found = tid;
    sh.found_there = c;
    sh.found_count = pc;
    sh.found_mass = pm;
  }
  __syncthreads();
}

// A row per cluster.  CTA `rank` has `blocks` blocks of 2048 tokens; thread t's of block j are first + 4 (512 j + t) + e.
template <int kType>
__global__ void __launch_bounds__(kThreads, 2) sample_kernel(const __grid_constant__ SampleArgs a) {
  using F = Four<kType>;
  extern __shared__ __align__(16) uint8_t dynamic[];
  typename F::T* xs = reinterpret_cast<typename F::T*>(dynamic);  // [blocks][thread]: each thread reads what it wrote
  __shared__ Shared sh;
  const cg::cluster_group cluster = cg::this_cluster();
  const int n_cta = (int)cluster.num_blocks(), rank = (int)cluster.block_rank(), blocks = a.blocks;
  const int m = blockIdx.x / n_cta, tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int first = rank * blocks * kBlock;
  constexpr int kSize = kType == SHARD_F32 ? 4 : 2;
  const char* row = static_cast<const char*>(a.logits) + (long long)m * a.ld * kSize;
  if (tid < 64) sh.table[tid] = kSampleTable[tid];
  if (tid == 0) sh.n_list = 0;
  const float T = a.s.temperature ? __ldg(a.s.temperature + m) : 1.f, top_p = a.s.top_p ? __ldg(a.s.top_p + m) : 1.f,
              min_p = a.s.min_p ? __ldg(a.s.min_p + m) : 0.f, u = __ldg(a.s.u + m);
  const int top_k = a.s.top_k ? __ldg(a.s.top_k + m) : 0;
  if (tid == kThreads - 1) {  // by one thread, under the loads: 64-bit arithmetic by all of them took 9000 cycles
    const double c = fmin(1.4426950408889634 / (double)T, 1e30);
    sh.w.c_hi = (float)c;
    sh.w.c_lo = (float)(c - (double)(float)c);
    sh.w.table = sh.table;
    if (min_p > 0.f) sh.bound = (double)T * log((double)min_p);
  }

  // ---- 1. the row's logits (minus infinity for NaN and behind the end, one zero); the maximum, and the smallest that
  // is not minus infinity ----
  const bool vec = reinterpret_cast<uintptr_t>(row) % (4 * kSize) == 0;
  if (vec) {
#pragma unroll 1
    for (int j = 0; j < blocks; ++j) {
      const int v = first + 4 * (j * kThreads + tid);
      if (v + 4 > a.V) break;
      const uint32_t to = smem_addr(xs + j * kThreads + tid);
      if (kSize == 4) asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(to), "l"(row + (size_t)v * 4) : "memory");
      else asm volatile("cp.async.ca.shared.global [%0], [%1], 8;" ::"r"(to), "l"(row + (size_t)v * 2) : "memory");
    }
    asm volatile("cp.async.wait_all;" ::: "memory");
  }
  float most_x = -INFINITY, least_x = INFINITY;
#pragma unroll 1
  for (int j = 0; j < blocks; ++j) {
    const int v = first + 4 * (j * kThreads + tid);
    float x[4];
    if (vec && v + 4 <= a.V) {
      const float4 f = F::get(xs[j * kThreads + tid]);
      x[0] = f.x, x[1] = f.y, x[2] = f.z, x[3] = f.w;
    } else {
#pragma unroll
      for (int e = 0; e < 4; ++e) x[e] = v + e < a.V ? logit<kType>(row, v + e) : -INFINITY;
    }
#pragma unroll
    for (int e = 0; e < 4; ++e) x[e] = plain(x[e]);
    most_x = fmaxf(fmaxf(most_x, fmaxf(x[0], x[1])), fmaxf(x[2], x[3]));
    const float low = fminf(fminf(x[0], x[1]), fminf(x[2], x[3]));
    if (low > -INFINITY) {
      least_x = fminf(least_x, low);
    } else {
#pragma unroll
      for (int e = 0; e < 4; ++e)
        if (x[e] > -INFINITY) least_x = fminf(least_x, x[e]);
    }
    xs[j * kThreads + tid] = F::put(make_float4(x[0], x[1], x[2], x[3]));
  }
  const bool valid = T >= 0.f && T < INFINITY && top_k >= 0 && top_p > 0.f && top_p <= 1.f && min_p >= 0.f &&
                     min_p <= 1.f && u >= 0.f && u < 1.f && !(a.failed && *a.failed);
  int turn = 0;
  Told mine = nothing();
  mine.hi = key_of(most_x);
  mine.lo = key_of(least_x);
  exchange<kBounds>(sh, turn, mine, n_cta, rank);
  uint32_t top = sh.sum.hi, bottom = sh.sum.lo;
  if (!valid || top <= kKeyNone || T == 0.f) {
    if (valid && top > kKeyNone) {  // the lowest id of the largest
      mine = nothing();
#pragma unroll 1
      for (int j = blocks - 1; j >= 0; --j) {
        const float4 f = F::get(xs[j * kThreads + tid]);
        const float x[4] = {f.x, f.y, f.z, f.w};
#pragma unroll
        for (int e = 3; e >= 0; --e)
          if (key_of(x[e]) == top) mine.hi = top, mine.id = first + 4 * (j * kThreads + tid) + e;
      }
      exchange<kIds>(sh, turn ^= 1, mine, n_cta, rank);
    }
    if (rank == 0 && tid == 0) {
      const bool none = !valid || top <= kKeyNone;
      a.token[m] = none ? -1 : sh.sum.id;
      if (a.p) a.p[m] = none ? __int_as_float(0x7fc00000) : 1.f;
      if (a.n_kept) a.n_kept[m] = none ? 0 : 1;
    }
    if (n_cta > 1) cluster.sync();  // the others may still read this CTA's shared memory
    return;
  }
  const bool infinite = top == key_of(INFINITY);
  if (infinite) {  // the infinite ones alone have weight, all the same
    for (int j = 0; j < blocks; ++j) {
      float4 f = F::get(xs[j * kThreads + tid]);
      f.x = f.x == INFINITY ? 0.f : -INFINITY, f.y = f.y == INFINITY ? 0.f : -INFINITY;
      f.z = f.z == INFINITY ? 0.f : -INFINITY, f.w = f.w == INFINITY ? 0.f : -INFINITY;
      xs[j * kThreads + tid] = F::put(f);
    }
    top = bottom = key_of(0.f);
  }
  if (tid == 0) {
    sh.w.max = of_key(top);
    sh.least = min_p > 0.f ? key_of(__double2float_ru((double)of_key(top) + sh.bound) + 0.f) : 0;
  }
  __syncthreads();
  const Weights w = sh.w;
  // this thread's tokens, block by block
  auto each = [&](auto&& body) {
#pragma unroll 1
    for (int j = 0; j < blocks; ++j) {
      const float4 f = F::get(xs[j * kThreads + tid]);
      const float x[4] = {f.x, f.y, f.z, f.w};
      body(j, x);
    }
  };

  // Kept: the keys above `edge`, and of those that are `edge` the first `ties` by id.
  uint32_t edge = kKeyNone + 1, ties = kAll;
  edge = max(edge, sh.least);
  const uint32_t least = edge;
  const bool cut = edge > kKeyNone + 1;
  uint64_t mass = 0, lower = 0, whole = 0;  // kept; kept by the CTAs of lower rank; what top_p is a share of
  uint32_t count = 0, choices = 0;          // kept; all that can be chosen
  bool probe = false, fewer = false;  // fewer: top_k is known to cut
  int level = 0;

  uint32_t first_lo = 0;  // the first histogram's bounds are this and top;
  int have = 0;           // sh.count (1), and sh.mass (2), are still its

  // ---- 2. few enough to rank: the candidates go to the first CTA, which finishes alone ----
  if (top_k > 0 || top_p < 1.f || cut) {
    const bool by_rank = top_k > 0, by_mass = !by_rank && top_p < 1.f;
    const bool drop = cut && (!by_rank || top_p >= 1.f);  // what lies below min_p's threshold has no part in a sum
    // down to min_p's threshold, or to weights of 2^-20: the rest only has to be known roughly
    const uint32_t lo = min(top, max(bottom, drop ? edge : key_of(w.max - 20.f / w.c_hi)));
    first_lo = lo;
    have = by_mass ? 2 : 1;
    histogram<F>(sh, xs, blocks, lo, top, by_mass, level++, n_cta, rank);
    uint64_t all = 0, slack = 0, most = 1;
    if (by_mass) {
      // what top_p is a share of, give or take the rest's error, and one of less than a part for each token
      const uint64_t part = warp_sum(sh.mass[tid]);
      if (lane == 0) sh.part[0][warp] = part;
      __syncthreads();
      for (int i = 0; i < kWarps; ++i) all += sh.part[0][i];
      slack = ((uint64_t)sh.count[kBins - 1] << 12) + (uint32_t)a.V;
      most = share_of(all + slack, top_p, true) + 1;
    }
    const Bins bins(lo, top);
    uint32_t last = kBins - 2;
    if (by_rank || by_mass) {
      reach(sh, by_mass, 0, 0, (uint32_t)top_k, most);
      // the min_p threshold alone, where that cuts more
      last = drop ? min(sh.found, (uint32_t)(kBins - 2)) : sh.found;
    }
    fewer = by_rank && !cut && sh.found < kBins - 1;
    uint32_t n = kList + 1;
    if (last < kBins - 1) {
      n = __reduce_add_sync(0xffffffffu, tid <= (int)last ? sh.count[tid] : 0);
      if (lane == 0) sh.part_count[warp] = n;
      __syncthreads();
      n = 0;
      for (int i = 0; i < kWarps; ++i) n += sh.part_count[i];
    }
    if (n <= kList) {
      Shared* to = cluster.map_shared_rank(&sh, 0);
      const float from = bins.least((int)last);
      each([&](int j, const float (&x)[4]) {
        if (fmaxf(fmaxf(x[0], x[1]), fmaxf(x[2], x[3])) < from) return;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          if (x[e] < from || bins(x[e]) > last) continue;
          const uint32_t at = atomicAdd(&to->n_list, 1u);
          to->list[at].key = key_of(x[e]);
          to->list[at].id = first + 4 * (j * kThreads + tid) + e;
        }
      });
      sync_row(cluster, n_cta);
      if (rank != 0) return;  // nothing of this CTA is read any more
      // its rank and the mass before it, then what is kept, then the mass up to its id: as many threads to a candidate
      // as there are, the first of which has it
      if (tid < (int)n) sh.list[tid].weight = w(of_key(sh.list[tid].key));
      const int by = min(5, 31 - __clz(kThreads / (int)n)), share = 1 << by, c = tid >> by, sub = tid & (share - 1);
      const bool real = c < (int)n, owner = real && sub == 0;
      __syncthreads();
      const uint32_t key = sh.list[real ? c : 0].key;
      const int id = sh.list[real ? c : 0].id;
      const uint64_t one = owner ? sh.list[c].weight : 0;
      uint32_t place = 0;
      uint64_t ahead = 0;
      if (real)
#pragma unroll 4
        for (int i = sub; i < (int)n; i += share) {
          const Shared::Candidate o = sh.list[i];
          const bool before = o.key > key || (o.key == key && o.id < id);
          place += before;
          ahead += before ? o.weight : 0;
        }
      for (int o = 1; o < share; o *= 2) {
        place += __shfl_xor_sync(0xffffffffu, place, o);
        ahead += __shfl_xor_sync(0xffffffffu, ahead, o);
      }
      bool keep = owner && key >= edge && (!by_rank || place < (uint32_t)top_k);
      if (top_p < 1.f) {
        uint64_t goal = most;
        if (by_rank) {  // a share of the first top_k
          const uint64_t part = warp_sum(place < (uint32_t)top_k ? one : 0);
          if (lane == 0) sh.scan_mass[warp] = part;
          __syncthreads();
          all = 0;
          for (int i = 0; i < kWarps; ++i) all += sh.scan_mass[i];
          goal = max(share_of(all, top_p, true), (uint64_t)1);
        } else {
          // where a candidate's mass lies within what is not known of the goal, all weights are summed up
          const uint64_t least = share_of(all > slack ? all - slack : 0, top_p, false);
          const bool sum = __syncthreads_or(keep && ahead >= least && ahead <= most) && !infinite;
          goal = max(share_of(sum ? sum_of_row<kType>(sh, row, a.V) : all, top_p, true), (uint64_t)1);
        }
        keep = keep && ahead < goal;
      }
      __syncthreads();
      if (owner) sh.list[c].weight = keep ? one : 0;
      const uint64_t part = warp_sum(keep ? one : 0);
      const uint32_t kept = __popc(__ballot_sync(0xffffffffu, keep));
      if (lane == 0) sh.part[0][warp] = part, sh.scan_count[warp] = kept;
      __syncthreads();
      uint64_t mass = 0, upto = 0;
      uint32_t count = 0;
      for (int i = 0; i < kWarps; ++i) mass += sh.part[0][i], count += sh.scan_count[i];
      if (tid == 0 && a.n_kept) a.n_kept[m] = (int32_t)count;
      if (real)
#pragma unroll 4
        for (int i = sub; i < (int)n; i += share) {
          const Shared::Candidate o = sh.list[i];
          upto += o.id <= id ? o.weight : 0;
        }
      for (int o = 1; o < share; o *= 2) upto += __shfl_xor_sync(0xffffffffu, upto, o);
      const uint64_t goal = share_of(mass, u, false);
      if (keep && upto > goal && upto - one <= goal) {
        a.token[m] = id;
        if (a.p) a.p[m] = (float)((double)one / (double)mass);
      }
      return;
    }
  }

  // ---- 3. otherwise the thresholds one by one ----
  // First the min_p threshold; then, each where it cuts more, that of top_k and that of top_p. Where min_p keeps fewer
  // than top_k, top_p is a share of the top_k all the same: their mass is found, and the min_p threshold taken back.
#pragma unroll 1
  for (int step = 0; step < 4; ++step) {
    const bool by_mass = step == 3;
    uint32_t rank_goal = (uint32_t)top_k, lo = edge, hi = top;
    uint64_t mass_goal = 0;
    bool find = false;
    if (step == 0 && top_k > 0) {  // only how many they are
      if (fewer) continue;
      mine = nothing();
      const float at_edge = of_key(edge);
      each([&](int, const float (&x)[4]) {
#pragma unroll
        for (int e = 0; e < 4; ++e) mine.count[0] += x[e] >= at_edge, mine.count[1] += x[e] > -INFINITY;
      });
      exchange<kCount | kAllMass>(sh, turn ^= 1, mine, n_cta, rank);
      count = sh.sum.count[0];
      choices = sh.sum.count[1];
      continue;
    }
    if (step == 1) {
      if (top_k == 0) continue;
      fewer = fewer || rank_goal < count;
      probe = !fewer && top_p < 1.f && rank_goal < choices;
      if (probe) lo = bottom;
      find = fewer || probe;
    } else if (step == 2) {
      if (!probe) continue;
      edge = least;
      ties = kAll;
    } else if (by_mass) {
      if (!(top_p < 1.f)) continue;
      mass_goal = max(share_of(whole, top_p, true), (uint64_t)1);
      if (mass_goal > mass) continue;
      find = true;
    }
    if (find) {
      // where the rank (or the mass) is reached among the keys of [lo, hi]
      uint32_t above = 0, there = 0;
      uint64_t above_mass = 0;
      bool again = have == (by_mass ? 2 : 1);  // the first histogram will do, if the goal is in it
#pragma unroll 1
      for (int tries = 0; tries < 1024; ++tries) {  // (each narrows the bounds)
        const Bins bins(again ? first_lo : lo, hi);
        if (!again) {
          histogram<F>(sh, xs, blocks, lo, hi, by_mass, level++, n_cta, rank);
          have = 0;
        }
        reach(sh, by_mass, above, above_mass, rank_goal, mass_goal);
        if (again && sh.found >= kBins - 1) {
          again = false;
          continue;
        }
        again = false;
        const uint32_t bin = sh.found;
        above = sh.found_count;
        above_mass = sh.found_mass;
        const float from = bins.least((int)bin), to = bins.most((int)bin);
        if (sh.found_there <= kList) {
          // few in the bin: all CTAs get them
          each([&](int, const float (&x)[4]) {
#pragma unroll
            for (int e = 0; e < 4; ++e)
              if (x[e] >= from && x[e] <= to && bins(x[e]) == bin) sh.own[atomicAdd(&sh.n_list, 1u)] = key_of(x[e]);
          });
          sync_row(cluster, n_cta);
          gather(sh, n_cta);
          const int n = (int)sh.found_there;
          const uint32_t key = tid < n ? sh.list[tid].key : 0;
          const uint64_t one = tid < n && by_mass ? w(of_key(key)) : 0;
          sh.list[tid].weight = one;
          __syncthreads();
          if (tid < n) {
            uint32_t c = above, equal = 0;
            uint64_t s = above_mass;
#pragma unroll 8
            for (int i = 0; i < n; ++i) {
              const Shared::Candidate o = sh.list[i];
              c += o.key > key;
              s += o.key > key ? o.weight : 0;
              equal += o.key == key;
            }
            if (by_mass ? s < mass_goal && s + equal * one >= mass_goal : c < rank_goal && c + equal >= rank_goal) {
              sh.found = key;
              sh.found_there = equal;
              sh.found_count = c;
              sh.found_mass = s;
            }
          }
          __syncthreads();
          lo = sh.found;
          there = sh.found_there;
          above = sh.found_count;
          above_mass = sh.found_mass;
          break;
        }
        // the bin's own bounds
        mine = nothing();
        each([&](int, const float (&x)[4]) {
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            if (!(x[e] >= from && x[e] <= to && bins(x[e]) == bin)) continue;
            const uint32_t k = key_of(x[e]);
            mine.hi = max(mine.hi, k);
            mine.lo = min(mine.lo, k);
            ++mine.count[0];
          }
        });
        exchange<kBounds | kCount>(sh, turn ^= 1, mine, n_cta, rank);
        lo = sh.sum.lo;
        hi = sh.sum.hi;
        there = sh.sum.count[0];
        if (lo >= hi) break;
      }
      uint64_t take = rank_goal - above;
      if (by_mass) {
        const uint64_t one = max(w(of_key(lo)), (uint64_t)1);
        take = (mass_goal - above_mass + one - 1) / one;
      }
      edge = lo;
      ties = take < there ? (uint32_t)take : kAll;
      count = above + (uint32_t)min(take, (uint64_t)there);
      if (ties != kAll) {
        // ties of lower ids than each warp of a block has
        mine = nothing();
        each([&](int j, const float (&x)[4]) {
          uint32_t here = 0;
#pragma unroll
          for (int e = 0; e < 4; ++e) here += key_of(x[e]) == edge;
          here = __reduce_add_sync(0xffffffffu, here);
          if (lane == 0) sh.ties[j][warp] = here, mine.count[0] += here;
        });
        exchange<kCount>(sh, turn ^= 1, mine, n_cta, rank);
        if (warp == 0) {
          uint32_t base = sh.lower.count[0];
          for (int j = 0; j < blocks; ++j) {
            const uint32_t here = lane < kWarps ? sh.ties[j][lane] : 0, upto = warp_scan(here, lane);
            if (lane < kWarps) sh.ties[j][lane] = base + upto - here;
            base += __shfl_sync(0xffffffffu, upto, 31);
          }
        }
        __syncthreads();
      }
    }
    // the mass of what is kept
    const bool first_time = step == 0 || (step == 1 && !find), all = first_time && cut && top_p < 1.f;  // and of all that can be chosen
    mine = nothing();
    const float at_edge = of_key(edge);
    int kept_high = 0, kept_low = 0, all_high = 0, all_low = 0;  // a thread's 64 tokens at most, 2^22 each
    each([&](int j, const float (&x)[4]) {
      uint32_t tie = 0;
      if (ties != kAll) {
        uint32_t here = 0;
#pragma unroll
        for (int e = 0; e < 4; ++e) here += key_of(x[e]) == edge;
        tie = sh.ties[j][warp] + warp_scan(here, lane) - here;
      }
      bool keep[4], weigh[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        keep[e] = x[e] > at_edge || (x[e] == at_edge && tie++ < ties);
        weigh[e] = keep[e] || (all && x[e] > -INFINITY);
      }
      int high = 0, low = 0;
      if (__any_sync(0xffffffffu, weigh[0] | weigh[1] | weigh[2] | weigh[3])) {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const Weights::Parts one = w.parts(x[e]);
          if (all && weigh[e]) all_high += one.high, all_low += one.low;
          if (keep[e]) high += one.high, low += one.low, ++mine.count[0];
        }
        kept_high += high;
        kept_low += low;
        high = __reduce_add_sync(0xffffffffu, high);
        low = __reduce_add_sync(0xffffffffu, low);
      }
      if (lane == 0) sh.part[j][warp] = Weights::joined(high, low);
    });
    mine.mass[0] = Weights::joined(kept_high, kept_low);
    mine.mass[1] = Weights::joined(all_high, all_low);
    if (all) exchange<kMass | kCount | kAllMass>(sh, turn ^= 1, mine, n_cta, rank);
    else exchange<kMass | kCount>(sh, turn ^= 1, mine, n_cta, rank);
    mass = sh.sum.mass[0];
    lower = sh.lower.mass[0];
    if (step != 1 || !probe) count = sh.sum.count[0];
    if (step < 2) whole = all ? sh.sum.mass[1] : mass;
  }

  // ---- 4. the first id whose cumulated mass exceeds u times all of it ----
  const uint64_t goal = share_of(mass, u, false);
  if (goal >= lower) {
    uint64_t left = goal - lower;
#pragma unroll 1
    for (int j = 0; j < blocks; ++j) {
      const uint64_t of_warp = lane < kWarps ? sh.part[j][lane] : 0, upto = warp_scan(of_warp, lane), all = __shfl_sync(0xffffffffu, upto, 31);
      if (left >= all) {
        left -= all;
        continue;
      }
      const int in_warp = __ffs(__ballot_sync(0xffffffffu, upto > left)) - 1;
      left -= __shfl_sync(0xffffffffu, upto - of_warp, in_warp);
      if (warp != in_warp) break;
      const float4 f = F::get(xs[j * kThreads + tid]);
      const float x[4] = {f.x, f.y, f.z, f.w};
      uint32_t tie = 0;
      if (ties != kAll) {
        uint32_t here = 0;
#pragma unroll
        for (int e = 0; e < 4; ++e) here += key_of(x[e]) == edge;
        tie = sh.ties[j][warp] + warp_scan(here, lane) - here;
      }
      uint64_t one[4], kept = 0;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const uint32_t k = key_of(x[e]);
        one[e] = k > edge || (k == edge && tie++ < ties) ? w(x[e]) : 0;
        kept += one[e];
      }
      uint64_t cum = warp_scan(kept, lane) - kept;
      if (cum <= left && left < cum + kept) {
        int e = 0;
#pragma unroll
        for (; e < 3; ++e) {
          if (left < cum + one[e]) break;
          cum += one[e];
        }
        a.token[m] = first + 4 * (j * kThreads + tid) + e;
        if (a.p) a.p[m] = (float)((double)(e == 0 ? one[0] : e == 1 ? one[1] : e == 2 ? one[2] : one[3]) / (double)mass);
      }
      break;
    }
  }
  if (rank == 0 && tid == 0 && a.n_kept) a.n_kept[m] = (int32_t)count;
  if (n_cta > 1) cluster.sync();  // the others may still read this CTA's shared memory
}

int fail(int code, const char* fmt, ...) __attribute__((format(printf, 2, 3)));
int fail(int code, const char* fmt, ...) {
  char buf[512];
  va_list ap;
  va_start(ap, fmt);
  vsnprintf(buf, sizeof(buf), fmt, ap);
  va_end(ap);
  return shard_fail_msg(code, buf);
}

template <int kType>
cudaError_t launch_type(SampleArgs a, int M, int sms, cudaStream_t s) {
  static std::atomic<uint64_t> ready{0};  // devices whose limits are raised
  int device;
  cudaError_t e = cudaGetDevice(&device);
  if (e != cudaSuccess) return e;
  if (device >= 64 || !(ready.load() >> device & 1)) {
    e = cudaFuncSetAttribute(sample_kernel<kType>, cudaFuncAttributeNonPortableClusterSizeAllowed, 1);
    if (e == cudaSuccess)
      e = cudaFuncSetAttribute(sample_kernel<kType>, cudaFuncAttributeMaxDynamicSharedMemorySize, kMaxBlocks * kThreads * sizeof(typename Four<kType>::T));
    if (e != cudaSuccess) return e;
    if (device < 64) ready.fetch_or(1ull << device);
  }
  // The fewest blocks per CTA, and so the most CTAs to a row, with which all rows run at once, a CTA to an SM; with more
  // rows, the 64 KB that leave room for two CTAs (32 / 64 KB, 48 rows of 32 bits 49 / 32 us; 256 rows of 16 bits 156 / 118).
  // Two to an SM for fewer rows as well, 16 of them: with settings of their own 53 -> 45 us, where top_p keeps thousands 80
  // -> 73, but with top_k of 2000 73 -> 90 and a few left by min_p 47 -> 56 (14 clusters of 16 run at once).
  constexpr int kCell = sizeof(typename Four<kType>::T);
  int n_cta = 1;
  for (a.blocks = 1;; ++a.blocks) {
    for (n_cta = 1; (long long)n_cta * a.blocks * kBlock < a.V;) n_cta *= 2;
    if (n_cta <= kMaxCluster && ((long long)M * n_cta <= sms || a.blocks * kThreads * kCell >= 64 << 10)) break;
  }
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3((unsigned)M * n_cta);
  cfg.blockDim = dim3(kThreads);
  cfg.dynamicSmemBytes = (size_t)a.blocks * kThreads * kCell;
  cfg.stream = s;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeClusterDimension;
  attr[0].val.clusterDim.x = n_cta;
  attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  return cudaLaunchKernelEx(&cfg, sample_kernel<kType>, a);
}

}  // namespace

namespace shard {

bool sampling_aligned(const head_sampling& s, const int32_t* token, const float* p, const int32_t* n_kept) {
  return aligned4(s.temperature, s.top_k, s.top_p, s.min_p, s.u, token, p, n_kept);
}

cudaError_t launch_sample(const void* logits, int type, int M, int V, long long ld, const head_sampling& s, int32_t* token,
                          float* p, int32_t* n_kept, const int* failed, int sms, cudaStream_t stream) {
  const SampleArgs a{logits, V, 0, ld, s, token, p, n_kept, failed};
  return type == SHARD_F32   ? launch_type<SHARD_F32>(a, M, sms, stream)
         : type == SHARD_F16 ? launch_type<SHARD_F16>(a, M, sms, stream)
                             : launch_type<SHARD_BF16>(a, M, sms, stream);
}

}  // namespace shard

extern "C" int head_sample_logits(const void* logits, int type, int M, int V, long long ld,
                                  const head_sampling* sampling, int32_t* token, float* p, int32_t* n_kept,
                                  void* cuda_stream) {
  if (!logits || !sampling || !sampling->u || !token) return fail(SHARD_EINVAL, "head_sample_logits: null argument");
  if (type < SHARD_F32 || type > SHARD_BF16) return fail(SHARD_EINVAL, "head_sample_logits: type %d", type);
  if (M < 1 || V < 1 || ld < V) return fail(SHARD_EINVAL, "head_sample_logits: M %d, V %d or ld %lld out of range", M, V, ld);
  if (reinterpret_cast<uintptr_t>(logits) % (type == SHARD_F32 ? 4 : 2))
    return fail(SHARD_EINVAL, "head_sample_logits: logits is not aligned to its values");
  if (!sampling_aligned(*sampling, token, p, n_kept))
    return fail(SHARD_EINVAL, "head_sample_logits: an array is not aligned to its values");
  if (V > HEAD_MAX_SAMPLE_VOCAB || M > HEAD_MAX_SAMPLE_ROWS)
    return fail(SHARD_EUNSUPPORTED, "head_sample_logits: V %d > %d or M %d > %d", V, HEAD_MAX_SAMPLE_VOCAB, M, HEAD_MAX_SAMPLE_ROWS);
  OnDeviceOf on(logits);
  if (on.error()) return fail(SHARD_EINVAL, "head_sample_logits: logits is not device memory");
  const cudaError_t e = launch_sample(logits, type, M, V, ld, *sampling, token, p, n_kept, nullptr, sms_of(on.device()),
                                      static_cast<cudaStream_t>(cuda_stream));
  return e == cudaSuccess ? SHARD_OK : fail(SHARD_ECUDA, "head_sample_logits: %s", cudaGetErrorString(e));
}
