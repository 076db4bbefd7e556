// Attention of drafted trees over their requests' caches (include/shard.h) on the
// tensor cores.
//
// For a request and a kv head, the query rows of all its nodes and of the heads
// that share the kv head form one matrix Q (rows (node, head)), and
//   O = softmax(scale Q K^T + visibility) V
// is computed over tiles of 128 entries with a running maximum m and sum l per
// row: S = Q K^T, P = 2^((S - m) c), l += sum P, O += P V, all in tensor memory.  A
// row sees a cache entry by the mask, a node's entry by its ancestor bits.  The maximum
// is one of S itself: with a rounded product m c, S c - m c is off by half a step of it,
// which makes weights overflow from 2^27 on (an addition more for two entries, 1.5 % of
// the time of the trees of 64 below).
//
// Work split: an item is (request, kv head, up to 256 rows), its units the tiles
// of entries; the units of all items, laid end to end, are cut into one equal run
// per CTA, so that ragged requests load every SM alike.  A CTA whose run holds an
// item whole writes its output; of an item cut between CTAs each leaves m, l and
// O, and tree_combine_kernel joins them in order.
//
// A CTA has two streams of softmax (four warps each, a row per thread).  An item
// of more than 128 rows gives each 128 of them over the same tiles; a smaller one
// gives both the same rows and every other tile, joined when the item ends.  A
// stream takes a tile in two steps of 64 entries with an S each, so that the
// products of the step before and of the one after run under its exponentials.
// Roles: warp 0 copies K and V tiles (tensor copies, a ring of slots), warps 1 and
// 2 issue the streams' products, warp 3 copies the queries and makes V tiles safe
// (below), warps 4..11 are the two streams.
//
// P times V would give NaN for a weight of 0 times an infinity or NaN, so V
// entries that no row sees are set to zero in shared memory, and values of the
// tree's own entries that are not finite too; those are added to the rows that
// see them when O is read.
//
// P is rounded to the cache's type for its product, 2^-8 (bf16) or 2^-11 of a
// weight at most, as the values are; 32-bit queries and their P go as two parts of fp16 or
// three of bf16, 22 or 24 bits, the small parts' products first (queries of 32 bits
// on 500 to 900 entries: 5.5e-7 of the result off, with the large ones first 9e-7 and
// 13e-7).  Three parts of P fit into tensor memory with one stream only (S, P and O of
// two fill it): the second has no tiles then (16-bit outputs: 278 us instead of 180 for
// fp16 on 95000 entries, 48 instead of 40 for 16 requests).
//
// Measured (GB300, calls replayed): one node on 100 entries 9.2 us, 16 requests of
// 5 nodes on 128 to 2048 entries 28.8 (65 MB), 4 trees of 64 at 64 / 8 heads on 4096
// entries 54.7 (34.6 GFLOP), the same two on 60000 entries 225 (1120 TFLOP/s), 2 of
// 32 at 32 / 8 heads on 95000 entries 131 (5.8 TB/s).  Long caches are bound by
// memory; many rows by the chain S, softmax, P V of a stream's steps (the tensor
// unit is 40 to 60 % busy); the rest by the kernels' starts, pieces' output and join.
#include <algorithm>
#include <atomic>
#include <cmath>

#include <cuda_bf16.h>

#include "launch.cuh"
#include "tcgen05.cuh"
#include "tree.cuh"

namespace shard {
namespace {

constexpr int kTile = 128;      // entries per tile, rows per stream
constexpr int kStep = 64;       // entries per step
constexpr int kThreads = 384;
constexpr int kSoftWarp0 = 4;   // first softmax warp
constexpr int kSoft = 256;      // softmax threads
// Weights are kept times 2^6, and the maximum they are relative to is raised only
// when it has been passed by 2^8: a weight is below 2^14, within fp16, and fp16
// still holds weights 2^-20 of the largest with all its bits.
constexpr float kLift = 6.f, kLag = 8.f;
constexpr float kMost = 3.402823466e38f;  // the largest finite value

struct Params {
  shard_tree_attn a;
  CUtensorMap kmap, vmap;  // {head_dim, capacity, kv heads, requests}, box 64 x 128
  CUtensorMap qmap;        // 16-bit queries: {head_dim, heads, nodes}, box 64 x heads of a kv head x 128 rows' nodes
  int g_shift;             // log2 of query heads per kv head
  int rows_max;            // rows of an item in `work`
  int act_order;
  float c;                 // scale * log2(e), finite
  int* plan;               // work: per request {first unit, first item, tiles, nodes}, then {all units, all items, CTAs, -}
  float4* ml;              // work: [2 * CTAs][rows_max] maximum, sum, and what scores are times
  float* o;                // work: [2 * CTAs][rows_max][D]
  float4* taken;           // work: [CTAs][2][taken_rows / 32][D / 4][32], a stream's O taken over (head_dim 128, two streams)
  int taken_rows;          // rows of a stream at most, in whole warps
  int fold;                // steps between two of these
};

// kRows: rows of an item at most.  128 where the requests have no more (or 32-bit queries take the second
// tile's place): it leaves room for another slot, and what a CTA has in flight bounds long caches (slots 4 -> 5,
// two caches of 95000 entries with 128 rows each).  256 where they have more: each tile then serves twice the rows.
template <int D, bool kF32, bool kBf16, int kRows_>
struct Geo {
  static constexpr int kRows = kRows_;
  static_assert(!kF32 || kRows == kTile, "the other tiles hold the lower parts");
  static constexpr int kParts = !kF32 ? 1 : kBf16 ? 3 : 2;  // of 11 or 8 bits of a 32-bit value
  static constexpr bool kSingle = kParts == 3;              // one stream: the other's S is where the third parts of P go
  static constexpr bool kSpare = kSingle || D == 64;        // tensor memory has room for the sums that O is taken over into
  // The tensor unit cuts off the bits that a sum of 32 bits has no room for, always toward zero: O loses some 2^-25 of itself
  // with each product added, 3e-5 over 64 tiles of three parts.  So a stream takes its O over into a sum of its own, rounded
  // to nearest, after kFold32 tiles with 32-bit queries and outputs (error 5.4e-7 to 7e-7 of the result on one to 256 tiles
  // per CTA, 8.2e-7 by two tiles, where it was 2.7e-5 after 64 and 1e-4 after 256), else after kFold (some 1000 products or
  // 1500: 3e-5 to 5e-5, which the weights' or the outputs' rounding covers).  The sum is in tensor memory where that has
  // room (head_dim 64; one stream, whose sums the idle warps of the other take), else in `work`.  Two caches of 95000
  // entries, 32-bit queries and outputs, without and with it: fp16 179 / 225 us (every tile 256), bf16 257 / 283; head_dim 64,
  // fp16, 114 / 135; 5 nodes instead of 32, fp16, 158 / 174.
  static constexpr int kFold32 = kSpare ? 1 : 2, kFold = kParts == 1 ? 128 : 64;
  static constexpr int kQTiles = kF32 ? kParts : kRows / kTile;
  static constexpr uint32_t kBlock = kTile * 128;        // 64 columns of a tile of K, V or Q
  static constexpr uint32_t kSlot = kBlock * (D / 64);   // a tile
  static constexpr int kSlots = D == 128 ? (kQTiles == 1 ? 5 : kQTiles == 2 ? 4 : 3) : (kQTiles == 1 ? 10 : 8);
  static constexpr size_t kQ = 0;                        // rows 0..127 and 128..255, or a 32-bit value's parts
  static constexpr size_t kRing = kQTiles * kSlot;
  static constexpr size_t kReq = kRing + kSlots * kSlot;            // each request, and the end
  static constexpr size_t kAnc = kReq + 16 * (SHARD_MAX_TREES + 1) + 16;
  static constexpr size_t kJump = kAnc + SHARD_MAX_TREE * 32;
  static constexpr size_t kMl = kJump + SHARD_MAX_TREE * 4;
  static constexpr size_t kStage = kMl + 2 * 2 * kTile * 8;         // per softmax warp, 32 rows of 64 bytes on their way out
  static constexpr size_t kTotal = kStage + 8 * 2048 + 1024;        // + alignment slack
  static_assert(kTotal + 512 <= 232448, "shared memory");
};

// The cut of `units` units into n equal runs, n <= units: run c begins at floor(units * c / n), in 32 bits.
struct Runs {
  uint32_t each, rest, n, units;
  __device__ __forceinline__ Runs(uint32_t units, uint32_t n) : each(units / n), rest(units - units / n * n), n(n), units(units) {}
  __device__ __forceinline__ uint32_t start(uint32_t c) const { return each * c + rest * c / n; }
  __device__ __forceinline__ uint32_t of(uint32_t unit) const {  // the run that has a unit
    uint32_t c = min(n - 1, (uint32_t)(((float)unit + 0.5f) * (float)n / (float)units));
    while (start(c) > unit) --c;
    while (c + 1 < n && start(c + 1) <= unit) ++c;
    return c;
  }
};

__device__ __forceinline__ float exp2_fast(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
// The largest of three; NaN if one is.
__device__ __forceinline__ float max3(float a, float b, float c) {
  float d;
  asm("max.NaN.f32 %0, %1, %2, %3;" : "=f"(d) : "f"(a), "f"(b), "f"(c));
  return d;
}

// Two 32-bit values in a register pair.
typedef unsigned long long f32x2;
__device__ __forceinline__ f32x2 pair(float a, float b) {
  f32x2 r;
  asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(a), "f"(b));
  return r;
}
__device__ __forceinline__ float2 halves(f32x2 v) {
  float2 r;
  asm("mov.b64 {%0, %1}, %2;" : "=f"(r.x), "=f"(r.y) : "l"(v));
  return r;
}
__device__ __forceinline__ f32x2 fma2(f32x2 a, f32x2 b, f32x2 c) {
  f32x2 d;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(d) : "l"(a), "l"(b), "l"(c));
  return d;
}
__device__ __forceinline__ f32x2 add2(f32x2 a, f32x2 b) {
  f32x2 d;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(a), "l"(b));
  return d;
}
__device__ __forceinline__ void fence_async_proxy() { asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); }
__device__ __forceinline__ bool bar_any(int id, int threads, bool v) {
  uint32_t r;
  asm volatile(
      "{\n .reg .pred p, q;\n setp.ne.u32 p, %1, 0;\n barrier.cta.red.or.pred q, %2, %3, p;\n selp.u32 %0, 1, 0, q;\n}\n"
      : "=r"(r)
      : "r"((uint32_t)v), "r"(id), "r"(threads)
      : "memory");
  return r != 0;
}

template <bool kBf16>
__device__ __forceinline__ uint32_t pack2(float lo, float hi) {
  if (kBf16) {
    const __nv_bfloat162 v = __floats2bfloat162_rn(lo, hi);
    return *reinterpret_cast<const uint32_t*>(&v);
  }
  const __half2 v = __floats2half2_rn(lo, hi);
  return *reinterpret_cast<const uint32_t*>(&v);
}
template <bool kBf16>
__device__ __forceinline__ float2 unpack2(uint32_t u) {
  if (kBf16) return make_float2(__uint_as_float(u << 16), __uint_as_float(u & 0xFFFF0000u));
  return __half22float2(*reinterpret_cast<const __half2*>(&u));
}
// Whether either of two 16-bit values is infinite or NaN.
template <bool kBf16>
__device__ __forceinline__ bool odd2(uint32_t u) {
  constexpr uint32_t lo = kBf16 ? 0x7F80u : 0x7C00u, hi = lo << 16;
  return (u & lo) == lo || (u & hi) == hi;
}

// a pair of 16-bit values times zero, plus b
template <bool kBf16>
__device__ __forceinline__ uint32_t times_zero(uint32_t a, uint32_t b) {
  uint32_t d;
  if (kBf16) asm("fma.rn.bf16x2 %0, %1, %2, %3;" : "=r"(d) : "r"(a), "r"(0u), "r"(b));
  else asm("fma.rn.f16x2 %0, %1, %2, %3;" : "=r"(d) : "r"(a), "r"(0u), "r"(b));
  return d;
}

// One piece of a CTA's run: tiles [t0, t1) of an item.
struct Piece {
  int b, h, row0, rows, t0, t1, tiles;  // rows row0 .. row0 + rows - 1 of the item's request and kv head
  int P, n, start;
  bool pair;   // more than 128 rows: a stream for each 128
};

// Walks a CTA's run piece by piece; every role has its own.
struct Walk {
  const shard_tree_attn* a;
  const int4* req;        // first unit, cache entries, nodes, first node of each request; behind the last, all units
  int rows_item, g_shift;
  int b, h, part, t0;     // where the next piece begins
  uint32_t left;          // units
  __device__ __forceinline__ bool next(Piece& p) {
    if (left == 0) return false;
    const int4 r = req[b];
    p.b = b;
    p.h = h;
    p.P = r.y;
    p.n = r.z;
    p.start = r.w;
    p.tiles = (p.P + p.n + kTile - 1) / kTile;
    p.t0 = t0;
    p.t1 = min(p.tiles, t0 + (int)left);
    p.row0 = part * rows_item;
    p.rows = min(rows_item, (p.n << g_shift) - p.row0);
    p.pair = p.rows > kTile;
    left -= p.t1 - p.t0;
    t0 = 0;
    ++part;
    if (part * rows_item >= p.n << g_shift) {
      part = 0;
      if (++h == a->n_kv_heads) {
        h = 0;
        do ++b;
        while (left > 0 && req[b + 1].x == req[b].x);
      }
    }
    return true;
  }
};
// Steps of stream s in a piece: two per tile, but for an item's last one that needs one only.  A stream takes every tile
// (of rows of its own, or with the other idle) or every other one.
template <bool kSingle>
__device__ __forceinline__ int steps_of(const Piece& q, int s) {
  const int nt = q.t1 - q.t0, todo = q.pair ? nt : kSingle ? (s ? 0 : nt) : (nt + 1 - s) / 2,
            last = q.t0 + (q.pair || kSingle ? todo - 1 : 2 * (todo - 1) + s);
  return 2 * todo - (todo > 0 && q.P + q.n - last * kTile <= kStep);
}

// A row of O into the sum of those taken over, that times f, to the place of the one or the other.  Out of line: the loop
// around it has no registers for this, which comes once in many steps; here all of a row's reads of `work` are on their way
// together.
template <int D, bool kSpare>
__device__ __noinline__ void take_rows(uint32_t O, uint32_t T, float4* in_work, float f, bool there, bool first, bool back) {
  if (kSpare) {
#pragma unroll 1
    for (int c = 0; c < D; c += 32) {
      uint32_t x[32], t[32];
      tc_ld32(O + c, x);
      tc_ld32(T + c, t);
      tc_ld_wait(x);
      tc_ld_wait(t);
      if (!first)
#pragma unroll
        for (int e = 0; e < 32; ++e) x[e] = __float_as_uint(fmaf(__uint_as_float(t[e]), f, __uint_as_float(x[e])));
      tc_st32((back ? O : T) + c, x);
    }
    tc_st_wait();
    return;
  }
  constexpr int kHalf = D / 8;  // of a row's float4
#pragma unroll 1
  for (int h = 0; h < 2; ++h) {
    float4 t[kHalf];
#pragma unroll
    for (int k = 0; k < kHalf; ++k) t[k] = there && !first ? __ldcg(in_work + 32 * (h * kHalf + k)) : make_float4(0.f, 0.f, 0.f, 0.f);
    __syncwarp();
#pragma unroll
    for (int c = 0; c < kHalf / 4; ++c) {
      uint32_t x[16];
      tc_ld(O + 4 * h * kHalf + 16 * c, x);
      tc_ld_wait(x);
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        float4& o = t[4 * c + k];
        o = make_float4(fmaf(o.x, f, __uint_as_float(x[4 * k])), fmaf(o.y, f, __uint_as_float(x[4 * k + 1])),
                        fmaf(o.z, f, __uint_as_float(x[4 * k + 2])), fmaf(o.w, f, __uint_as_float(x[4 * k + 3])));
        x[4 * k] = __float_as_uint(o.x), x[4 * k + 1] = __float_as_uint(o.y), x[4 * k + 2] = __float_as_uint(o.z), x[4 * k + 3] = __float_as_uint(o.w);
      }
      if (back) tc_st16(O + 4 * h * kHalf + 16 * c, x);
    }
    if (there && !back)
#pragma unroll
      for (int k = 0; k < kHalf; ++k) __stcg(in_work + 32 * (h * kHalf + k), t[k]);
    __syncwarp();
  }
  if (back) tc_st_wait();
}

// kTake: a stream's tiles may be more than p.fold.
template <int D, bool kF32, bool kBf16, int kRows, bool kTake>
__global__ void __launch_bounds__(kThreads, 1) tree_attention_kernel(const __grid_constant__ Params p) {
  using L = Geo<D, kF32, kBf16, kRows>;
  constexpr uint32_t kIdescS = (1u << 4) | ((uint32_t)kBf16 << 7) | ((uint32_t)kBf16 << 10) | ((uint32_t)(kStep >> 3) << 17) |
                               ((uint32_t)(kTile >> 4) << 24);
  constexpr uint32_t kIdescO = (1u << 4) | ((uint32_t)kBf16 << 7) | ((uint32_t)kBf16 << 10) | (1u << 16) |
                               ((uint32_t)(D >> 3) << 17) | ((uint32_t)(kTile >> 4) << 24);
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
  // full, empty: a slot's tile has come, has been used by both streams; v_ready: a V tile (by its place among
  // the V tiles) is safe; q_full, q_free: the piece's queries are in place, have been used by both streams;
  // s_full, p_ready, o_done: a step's S is computed, its P written, P V added (in turn for a stream's steps);
  // o_free: all have read a stream's O of a piece in which it has steps (a stream goes by its own pieces: one that
  // counted the others' too would not follow the phases of those, and take an old one for the piece before); o_full,
  // o_taken: one stream's O is ready for the other's warps, has been taken over by them (a phase for each time: by o_done,
  // which has one for each step, they would miss some); at_end: a stream's last product is done
  __shared__ uint64_t full[2 * L::kSlots], empty[L::kSlots], v_ready[L::kSlots], q_full, q_free, s_full[2][2], p_ready[2][2],
      o_done[2][2], o_free[2], o_full, o_taken, at_end[2];
  __shared__ uint32_t s_tmem;
  // pieces (counted from 1) whose tree entries hold a V that is not finite; V tiles run at most kSlots pieces ahead
  __shared__ volatile int s_odd[2 * L::kSlots];
  const shard_tree_attn& a = p.a;
  const int tid = threadIdx.x, warp = __shfl_sync(0xffffffffu, tid >> 5, 0), lane = tid & 31;
  int4* s_req = reinterpret_cast<int4*>(smem + L::kReq);
  uint32_t* s_anc = reinterpret_cast<uint32_t*>(smem + L::kAnc);  // [node][8]
  int* s_jump = reinterpret_cast<int*>(smem + L::kJump);
  float2* s_ml = reinterpret_cast<float2*>(smem + L::kMl);        // [piece % 2][stream][row]
  if (tid < 16) {
    if (tid < L::kSlots) {
      mbar_init(&full[2 * tid], 1);
      mbar_init(&full[2 * tid + 1], 1);
      mbar_init(&empty[tid], 2);
      mbar_init(&v_ready[tid], 1);
      s_odd[2 * tid] = s_odd[2 * tid + 1] = 0;
    }
    static_assert(L::kSlots <= 16, "a thread per slot");
    if (tid < 4) {
      mbar_init(&s_full[0][0] + tid, 1);
      mbar_init(&p_ready[0][0] + tid, 4);
      mbar_init(&o_done[0][0] + tid, 1);
    }
    if (tid == 0) {
      mbar_init(&q_full, kF32 ? kSoft : 1);
      mbar_init(&q_free, 2);
      mbar_init(&o_free[0], 8);
      mbar_init(&o_free[1], 8);
      mbar_init(&o_full, 1);
      mbar_init(&o_taken, 4);
      mbar_init(&at_end[0], 1);
      mbar_init(&at_end[1], 1);
    }
    mbar_fence_init();
  }
  if (warp == 1) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_addr(&s_tmem)), "r"(512u) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  pdl_wait();
  pdl_launch_dependents();

  // ---- the batch: every request's first unit; each warp for itself, 32 requests at a time ----
  uint32_t units_all = 0, items_all = 0;
  {
    int bad = 0;
#pragma unroll 1
    for (int b0 = 0; b0 < a.B; b0 += 32) {
      const int b = b0 + lane;
      uint32_t items = 0, tiles = 0;
      int n = 0, s = 0, P = 0;
      if (b < a.B) {
        const int e = __ldg(a.tree_start + b + 1);
        s = __ldg(a.tree_start + b);
        P = __ldg(a.lens + b);
        if (s < 0 || e < s || e > a.N || e - s > SHARD_MAX_TREE) {
          bad |= SHARD_TREE_START;
        } else if (P < 0 || P > a.capacity - (e - s) || (a.mask && P > a.mask_stride)) {
          bad |= SHARD_TREE_LENGTH;
        } else {
          n = e - s;
          tiles = (P + n + kTile - 1) / kTile;
          items = a.n_kv_heads * (((n << p.g_shift) + kRows - 1) / kRows);
        }
      }
      const uint32_t units = items * tiles;
      uint32_t upto = units, iupto = items;
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const uint32_t x = __shfl_up_sync(0xffffffffu, upto, o), y = __shfl_up_sync(0xffffffffu, iupto, o);
        if (lane >= o) upto += x, iupto += y;
      }
      if (warp == 0 && b < a.B) {
        s_req[b] = make_int4((int)(units_all + upto - units), P, n, s);
        if (blockIdx.x == 0)
          reinterpret_cast<int4*>(p.plan)[b] =
              make_int4((int)(units_all + upto - units), (int)(items_all + iupto - items), (int)tiles, n);
      }
      units_all += __shfl_sync(0xffffffffu, upto, 31);
      items_all += __shfl_sync(0xffffffffu, iupto, 31);
    }
    if (warp == 0) {
      if (lane == 0) s_req[a.B] = make_int4((int)units_all, 0, 0, 0);
      if (blockIdx.x == 0) {
        if (lane == 0)
          reinterpret_cast<int4*>(p.plan)[a.B] = make_int4((int)units_all, (int)items_all, (int)min(units_all, gridDim.x), 0);
        if (bad && a.status) atomicOr(a.status, bad);
      }
    }
  }
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  const uint32_t tmem = s_tmem;
  Walk walk{&a, s_req, kRows, p.g_shift, 0, 0, 0, 0, 0};
  {
    const uint32_t n_cta = min(units_all, gridDim.x);
    if (blockIdx.x < n_cta) {
      const Runs runs(units_all, n_cta);
      const uint32_t at = runs.start(blockIdx.x);
      walk.left = runs.start(blockIdx.x + 1) - at;
      int lo = 0, hi = a.B;  // the request: the last that begins at `at` or before
      while (hi - lo > 1) {
        const int mid = (lo + hi) / 2;
        if ((uint32_t)s_req[mid].x <= at) lo = mid;
        else hi = mid;
      }
      walk.b = lo;
      const int n = s_req[lo].z;
      const uint32_t tiles = (s_req[lo].y + n + kTile - 1) / kTile, u = at - (uint32_t)s_req[lo].x, item = u / tiles;
      const uint32_t parts = ((n << p.g_shift) + kRows - 1) / kRows;
      walk.t0 = u - item * tiles;
      walk.h = item / parts;
      walk.part = item - walk.h * parts;
    }
  }
  // false once a wait gave up: the copies and products stop, the streams go on to their
  // end without waiting
  bool ok = true;
  auto wait = [&](uint64_t* bar, uint32_t parity) {
    if (!ok) return;
    uint32_t it = 0;
    while (!mbar_test_wait(bar, parity))
      if (++it > (1u << 26)) {
        ok = false;
        break;
      }
  };
  // Whatever came before: what this role has under way is not left behind when the CTA ends.
  auto drain = [](uint64_t* bar, uint32_t parity) {
    for (uint32_t it = 0; it < (1u << 26) && !mbar_test_wait(bar, parity);) ++it;
  };
  // the product of a stream's step; two steps back, it has been waited for before a step's S was begun
  auto wait_o = [&](int s, uint32_t step) { wait(&o_done[s][step & 1], (step >> 1) & 1); };
  // Order of a piece's tiles in the ring.  A stream for each half of the rows, or one only: K(0) V(0) K(1) V(1) ..;
  // tiles in turn: K(0) K(1) V(0) V(1) K(2) ..
  auto k_seq = [](bool every, int t) { return every ? 2 * t : 4 * (t >> 1) + (t & 1); };
  auto v_seq = [](bool every, int t, int nt) { return every ? 2 * t + 1 : 4 * (t >> 1) + ((t | 1) < nt ? 2 : 1) + (t & 1); };
  auto slot_of = [](uint32_t seq) { return seq % L::kSlots; };
  auto turn_of = [](uint32_t seq) { return (seq / L::kSlots) & 1; };
  // A slot's uses take two barriers in turn: a role waits for its own tiles only, and may begin to while the
  // slot's last tile, the other stream's, is still coming; the one before that has been used (whatever it
  // waited for last is at most kSlots places back, and came after that tile was released).
  auto full_of = [&](uint32_t seq) { return &full[2 * (seq % L::kSlots) + ((seq / L::kSlots) & 1)]; };
  auto full_turn = [](uint32_t seq) { return (seq / (2 * L::kSlots)) & 1; };

  // The code is kept short rather than unrolled: most of it runs a few times a launch, and instructions for one
  // use are fetched from memory for it (102 KB of them before, 24 KB now).
  if (warp == 0) {
    // ---- copies ----
    if (lane == 0) {
      Piece q;
      uint32_t seq = 0;
      while (ok && walk.next(q)) {
        const int nt = q.t1 - q.t0;
#pragma unroll 1
        for (int i = 0; i < 2 * nt; ++i, ++seq) {
          // place i of the piece: which tile, and of K or V
          const int two = (i >> 2) * 2 + 1 < nt ? 2 : 1, r = i & 3;
          const bool every = q.pair || L::kSingle, v = every ? i & 1 : r >= two;
          const int t = q.t0 + (every ? i >> 1 : (i >> 2) * 2 + (v ? r - two : r));
          if (seq >= L::kSlots) wait(&empty[slot_of(seq)], turn_of(seq) ^ 1);
          if (!ok) break;
          mbar_arrive_expect_tx(full_of(seq), L::kSlot);
#pragma unroll
          for (int c = 0; c < D / 64; ++c)
            tma_load_4d(smem + L::kRing + (size_t)slot_of(seq) * L::kSlot + c * L::kBlock, v ? &p.vmap : &p.kmap, 64 * c, t * kTile,
                        q.h, q.b, full_of(seq));
        }
      }
      for (uint32_t i = seq > L::kSlots ? seq - L::kSlots : 0; i < seq; ++i) drain(full_of(i), full_turn(i));
    }
  } else if (warp < 3) {
    // ---- products, a warp per stream ----
    // A thread alone took ~1150 cycles to issue 8 products against 520 of tensor time when their operands
    // were computed under its branch; the whole warp goes along, a stream each.
    const int s = warp - 1;
    const bool leader = elect_one();
    const uint32_t S = tmem + s * kTile, O = tmem + 2 * kTile + s * kTile;
    const uint32_t ring = smem_addr(smem + L::kRing);
    Piece q;
    uint32_t base = 0, piece = 0, mine = 0, taken = 0, n = 0;  // first ring place of the piece; before it the stream's pieces, its O's taken over, its steps
    while (ok && walk.next(q)) {
      const int nt = __shfl_sync(0xffffffffu, q.t1 - q.t0, 0), steps = __shfl_sync(0xffffffffu, steps_of<L::kSingle>(q, s), 0);
      const bool pair = __shfl_sync(0xffffffffu, (int)q.pair, 0), every = pair || L::kSingle;
      const int entries = __shfl_sync(0xffffffffu, q.P + q.n, 0), t0 = __shfl_sync(0xffffffffu, q.t0, 0);
      const uint64_t Q = smem_desc_sw128(smem_addr(smem + L::kQ) + (pair && s ? L::kSlot : 0));
      wait(&q_full, piece & 1);
      // the slot of a tile that this stream has used
      auto release = [&](uint32_t slot) {
        if (!pair) mbar_arrive(&empty[slot]);  // the other stream has no use for it
        tc_commit(&empty[slot]);
      };
      // the S of a step is begun before the product of the step before
#pragma unroll 1
      for (int k = 0; k < steps + 2 && steps > 0; ++k) {
        if (k >= 2) {
          const int i = k - 2, t = every ? i >> 1 : 2 * (i >> 1) + s, half = i & 1;
          const uint32_t seq = base + v_seq(every, t, nt), nv = base / 2 + t, buf = (n + i) & 1, P = S + kStep * buf;
          const uint64_t V = smem_desc_sw128_mn(ring + slot_of(seq) * L::kSlot + half * (kStep * 128), L::kBlock);
          const int there = entries - (t0 + t) * kTile - half * kStep;  // entries from the step's first on
          if (i == 0 && mine) wait(&o_free[s], (mine - 1) & 1);
          if (kTake && L::kSingle && i > 0 && (i & (p.fold - 1)) == 0) wait(&o_taken, taken++ & 1);
          if (!half) {
            wait(full_of(seq), full_turn(seq));
            wait(&v_ready[slot_of(nv)], turn_of(nv));
          }
          wait(&p_ready[s][buf], ((n + i) >> 1) & 1);
          __syncwarp();
          tc_fence_after();
          if (ok && leader) {
            auto add = [&](int x) {
              const bool more = (kTake ? i & (p.fold - 1) : i) != 0 || x > 0;
              if (L::kSingle) tc_mma(O, tmem + kTile + 32 * buf + 8 * x, V + ((x * 2048) >> 4), kIdescO, more);
              if (kF32) tc_mma(O, P + 32 * (x >> 1) + 16 + 8 * (x & 1), V + ((x * 2048) >> 4), kIdescO, L::kSingle || more);
              tc_mma(O, P + 32 * (x >> 1) + 8 * (x & 1), V + ((x * 2048) >> 4), kIdescO, kF32 || more);
            };
            if (there >= kStep) {
#pragma unroll
              for (int x = 0; x < kStep / 16; ++x) add(x);
            } else {  // nothing behind the item's last entry
#pragma unroll 1
              for (int x = 0; 16 * x < there; ++x) add(x);
            }
            tc_commit(&o_done[s][buf]);
            if (kTake && L::kSingle && steps > p.fold && (((i + 1) & (p.fold - 1)) == 0 || i == steps - 1)) tc_commit(&o_full);
            if (half || i == steps - 1) release(slot_of(seq));
          }
          __syncwarp();
        }
        if (k < steps) {
          const int t = every ? k >> 1 : 2 * (k >> 1) + s, half = k & 1;
          const uint32_t seq = base + k_seq(every, t), buf = (n + k) & 1;
          const uint64_t K = smem_desc_sw128(ring + slot_of(seq) * L::kSlot + half * (kStep * 128));
          if (!half) wait(full_of(seq), full_turn(seq));
          // S holds the P of two steps ago until its product is done; at the piece's first, the last one's is
          if (k != 1 && n + k) wait_o(s, k ? n + k - 2 : n - 1);
          __syncwarp();
          tc_fence_after();
          if (ok && leader) {
#pragma unroll
            for (int part = L::kParts - 1; part >= 0; --part)
#pragma unroll
              for (int x = 0; x < D / 16; ++x)
                tc_mma_ss(S + kStep * buf, Q + ((part * L::kSlot + (x >> 2) * L::kBlock + (x & 3) * 32) >> 4),
                          K + (((x >> 2) * L::kBlock + (x & 3) * 32) >> 4), kIdescS, part < L::kParts - 1 || x > 0);
            tc_commit(&s_full[s][buf]);
            if (half || k == steps - 1) release(slot_of(seq));
            if (k == steps - 1) tc_commit(&q_free);
          }
          __syncwarp();
        }
      }
      if (steps == 0 && leader) mbar_arrive(&q_free);
      n += steps;
      mine += steps > 0;
      base += 2 * nt;
      ++piece;
    }
    if (leader) {
      tc_commit(&at_end[s]);
      drain(&at_end[s], 0);
    }
    __syncwarp();
  } else if (warp < kSoftWarp0) {
    // ---- queries; V tiles: zero what no row sees, and what is not finite ----
    Piece q;
    uint32_t base = 0, piece = 0, copied = 0;  // copied: pieces whose queries have been asked for
    while (ok && walk.next(q)) {
      const int nt = q.t1 - q.t0;
      if (!kF32) {
        if (piece) wait(&q_free, (piece - 1) & 1);
        copied += ok;
        if (ok && lane == 0) {
          mbar_arrive_expect_tx(&q_full, (q.pair ? 2 : 1) * L::kSlot);
          for (int r = 0; r < (q.pair ? 2 : 1); ++r)
#pragma unroll
            for (int k = 0; k < D / 64; ++k)
              tma_load_3d(smem + L::kQ + r * L::kSlot + k * L::kBlock, &p.qmap, 64 * k, q.h << p.g_shift,
                          q.start + ((q.row0 + r * kTile) >> p.g_shift), &q_full);
        }
        __syncwarp();
      }
      const uint8_t* mask = a.mask ? a.mask + (size_t)q.b * a.mask_stride : nullptr;
      // bit w: no row sees entry 32 w + lane of the tile
      auto hidden_of = [&](int t) {
        uint32_t bits = 0;
#pragma unroll
        for (int w = 0; w < 4; ++w) {
          const int j = t * kTile + 32 * w + lane;
          if (j >= q.P ? j >= q.P + q.n : mask && !__ldg(mask + j)) bits |= 1u << w;
        }
        return bits;
      };
      uint32_t next_hidden = hidden_of(q.t0);
#pragma unroll 1
      for (int i = 0; i < nt && ok; ++i) {
        const uint32_t seq = base + v_seq(q.pair || L::kSingle, i, nt), hidden = next_hidden;
        const int j0 = (q.t0 + i) * kTile;
        if (i + 1 < nt) next_hidden = hidden_of(q.t0 + i + 1);
        wait(full_of(seq), full_turn(seq));
        __syncwarp();
        // a lane per entry, its 16-byte pieces in an order that spreads the lanes over the banks
        uint8_t* v = smem + L::kRing + (size_t)slot_of(seq) * L::kSlot + lane * 128;
        const int there = q.P + q.n - j0;  // products read up to the next multiple of 16
        if (__any_sync(0xffffffffu, hidden != 0) || there < kTile || j0 + kTile > q.P) {
#pragma unroll 1
          for (int w = 0; w < 4 && 32 * w < there; ++w, v += 32 * 128) {
            const int j = 32 * w + lane, node = j0 + j - q.P;
            if ((hidden >> w & 1) && j < (there + 15) / 16 * 16) {
#pragma unroll
              for (int c = 0; c < D / 8; ++c)
                *reinterpret_cast<uint4*>(v + (c >> 3) * L::kBlock + (((c + lane) & 7) << 4)) = make_uint4(0, 0, 0, 0);
            }
            if (j0 + 32 * w + 32 > q.P) {
              const bool mine = node >= 0 && j < there;
              uint32_t sum = 0;  // NaN where a value is not finite: times zero
              if (mine)
#pragma unroll 8
                for (int c = 0; c < D / 8; ++c) {
                  const uint4 u = *reinterpret_cast<const uint4*>(v + (c >> 3) * L::kBlock + (((c + lane) & 7) << 4));
                  sum = times_zero<kBf16>(u.x, times_zero<kBf16>(u.y, times_zero<kBf16>(u.z, times_zero<kBf16>(u.w, sum))));
                }
              if (odd2<kBf16>(sum)) {
#pragma unroll 1
                for (int c = 0; c < D / 8; ++c) {
                  uint4* at = reinterpret_cast<uint4*>(v + (c >> 3) * L::kBlock + (((c + lane) & 7) << 4));
                  auto finite = [](uint32_t x) {
                    return (odd2<kBf16>(x & 0xFFFFu) ? 0 : x & 0xFFFFu) | (odd2<kBf16>(x & 0xFFFF0000u) ? 0 : x & 0xFFFF0000u);
                  };
                  const uint4 u = *at;
                  *at = make_uint4(finite(u.x), finite(u.y), finite(u.z), finite(u.w));
                }
                s_odd[piece % (2 * L::kSlots)] = (int)piece + 1;
              }
            }
          }
          fence_async_proxy();
          __syncwarp();
        }
        if (ok && lane == 0) mbar_arrive(&v_ready[slot_of(base / 2 + i)]);
      }
      base += 2 * nt;
      ++piece;
    }
    if (lane == 0 && copied) drain(&q_full, (copied - 1) & 1);
    __syncwarp();
  } else {
    // ---- the two streams ----
    const int s = (warp - kSoftWarp0) >> 2, quad = warp & 3, row = 32 * quad + lane, st = tid - kSoftWarp0 * 32;
    const uint32_t lanes = tmem + ((uint32_t)(32 * quad) << 16);
    const int G = 1 << p.g_shift;
    Piece q;
    uint32_t piece = 0, n_s = 0, n_o[2] = {0, 0}, n_full = 0;  // steps of this stream; of both, up to the piece's end; O's taken over from the other
    float scores = p.c;  // from this row's products to exponents of two
    int anc_of = -1;  // the request whose ancestors are in shared memory
    // 32-bit queries of a piece into shared memory, in parts; rows behind its last zero.  A row is taken times the power of
    // two that brings its largest value to 2^13 (fp16: above 2^16 the first part is infinite, below 2^-3 the second loses
    // bits) or 2^-20 (bf16: whose range the values of K may take up), and the inverse goes into the row's scale of scores,
    // left in row_c for the row's threads.
    auto load_q = [&](const Piece& q, float2* row_c) {
      constexpr int kPieces = D / 8;  // pieces of 8 values to a row
      constexpr int kTop = kBf16 ? -20 : 13;
      constexpr int kPass = kSoft / kPieces;  // rows at a time
      const int passes = (q.rows + kPass - 1) / kPass;
      int e = st;
#pragma unroll 2
      for (int pass = 0; pass < passes; ++pass, e += kSoft) {
        const int r = e / kPieces, c = e % kPieces, gr = q.row0 + r;
        float4 x = make_float4(0.f, 0.f, 0.f, 0.f), y = x;
        if (r < q.rows) {
          const float4* at = reinterpret_cast<const float4*>(
              static_cast<const float*>(a.q) + (q.start + (gr >> p.g_shift)) * a.q_stride + (q.h * G + (gr & (G - 1))) * D + 8 * c);
          x = __ldg(at);
          y = __ldg(at + 1);
        }
        float rest[8] = {x.x, x.y, x.z, x.w, y.x, y.y, y.z, y.w}, top = 0.f;
#pragma unroll
        for (int i = 0; i < 8; ++i) top = fmaxf(top, fabsf(rest[i]));
#pragma unroll
        for (int o = kPieces / 2; o > 0; o >>= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
        const int exponent = (int)(__float_as_uint(top) >> 23);  // biased; a row of zeros or with an infinity stays as it is
        const int up = top == 0.f || exponent == 255 ? 127 : max(1, min(253, 254 + kTop - exponent));
        const float times = __uint_as_float((uint32_t)up << 23);
#pragma unroll
        for (int i = 0; i < 8; ++i) rest[i] *= times;
        if (c == 0) {
          // (not 0, so that minus infinity stays; what is cut off is of scores below 2^-80)
          const float row = fminf(fmaxf(p.c * __uint_as_float((uint32_t)(254 - up) << 23), 0x1p-126f), kMost);
          row_c[r].x = row_c[kTile + r].x = row;
        }
        uint8_t* to = smem + L::kQ + (c >> 3) * L::kBlock + r * 128 + (((c & 7) ^ (r & 7)) << 4);
#pragma unroll
        for (int part = 0; part < L::kParts; ++part) {
          uint32_t w[4];
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            w[i] = pack2<kBf16>(rest[2 * i], rest[2 * i + 1]);
            const float2 b = unpack2<kBf16>(w[i]);
            rest[2 * i] -= b.x, rest[2 * i + 1] -= b.y;
          }
          *reinterpret_cast<uint4*>(to + part * L::kSlot) = make_uint4(w[0], w[1], w[2], w[3]);
        }
      }
#pragma unroll 1
      for (; e < kTile * kPieces; e += kSoft) {
        const int r = e / kPieces, c = e % kPieces;
#pragma unroll
        for (int part = 0; part < L::kParts; ++part)
          *reinterpret_cast<uint4*>(smem + L::kQ + part * L::kSlot + (c >> 3) * L::kBlock + r * 128 + (((c & 7) ^ (r & 7)) << 4)) =
              make_uint4(0, 0, 0, 0);
        if (c == 0) row_c[r].x = row_c[kTile + r].x = p.c;
      }
      fence_async_proxy();
      mbar_arrive(&q_full);
    };
    while (walk.next(q)) {
      if (kF32) {
        // Both product warps have passed the piece before: one without steps in it has no other tie to the streams, and
        // would miss a phase of q_full
        if (piece) wait(&q_free, (piece - 1) & 1);
        float2* row_c = s_ml + (piece & 1) * 2 * kTile;  // in the place of the maximum that this thread leaves at the piece's end
        load_q(q, row_c);
        named_bar_sync(1, kSoft);
        scores = row_c[s * kTile + row].x;
      }
      const int nt = q.t1 - q.t0, steps = steps_of<L::kSingle>(q, s);
      const int row_item = (q.pair ? s * kTile : 0) + row, grow = q.row0 + row_item;  // row of the item; of the request and kv head
      const int node = min(grow >> p.g_shift, q.n - 1);
      const uint8_t* mask = a.mask ? a.mask + (size_t)q.b * a.mask_stride : nullptr;
      const bool in_tree = q.t1 * kTile > q.P;  // the piece has entries of the tree
      if (in_tree && anc_of != q.b) {
        // ancestors of every node, doubling the reach each time: anc(i) |= anc(jump(i)), jump(i) = jump(jump(i))
        anc_of = q.b;
        int jump = -1;
        if (st < q.n) {
          jump = __ldg(a.parents + q.start + st);
          if (jump < -1 || jump >= st) {
            jump = -1;
            if (a.status) atomicOr(a.status, SHARD_TREE_PARENT);
          }
        }
        named_bar_sync(1, kSoft);
        uint4 w[2];
        uint4* mine = reinterpret_cast<uint4*>(s_anc + 8 * st);
        w[0] = make_uint4(st >> 5 == 0, st >> 5 == 1, st >> 5 == 2, st >> 5 == 3);
        w[1] = make_uint4(st >> 5 == 4, st >> 5 == 5, st >> 5 == 6, st >> 5 == 7);
#pragma unroll
        for (int k = 0; k < 2; ++k) w[k].x <<= st & 31, w[k].y <<= st & 31, w[k].z <<= st & 31, w[k].w <<= st & 31;
#pragma unroll 1
        while (true) {
          mine[0] = w[0];
          mine[1] = w[1];
          s_jump[st] = jump;
          if (!bar_any(1, kSoft, jump >= 0)) break;
          if (jump >= 0) {
#pragma unroll
            for (int k = 0; k < 2; ++k) {
              const uint4 x = *reinterpret_cast<const uint4*>(s_anc + 8 * jump + 4 * k);
              w[k].x |= x.x, w[k].y |= x.y, w[k].z |= x.z, w[k].w |= x.w;
            }
            jump = s_jump[jump];
          }
          named_bar_sync(1, kSoft);
        }
      }
      // the words of a step that say which entries this thread's row sees
      auto load_mask = [&](int j0, uint8_t (&m)[2]) {
#pragma unroll
        for (int w = 0; w < 2; ++w) {
          const int j = j0 + 32 * w + lane;
          m[w] = j < q.P ? (mask ? __ldg(mask + j) : 1) : 0;
        }
      };
      auto first_of = [&](int i) { return (q.t0 + (q.pair || L::kSingle ? i >> 1 : 2 * (i >> 1) + s)) * kTile + (i & 1) * kStep; };
      float m = -kMost, l = 0.f;  // the score that weights are relative to (the lowest finite one until any is seen); their sum
      uint8_t mb[2];
      if (steps > 0) load_mask(first_of(0), mb);
      // This row's sum of O's taken over, and O, to the place of the one or the other: the sum is relative to the score
      // taken_m, O to m_now.
      const uint32_t O_own = lanes + 2 * kTile + (L::kSingle ? 0 : s * kTile), T_own = O_own + (D == 64 ? 64 : kTile);
      float4* in_work = p.taken + ((size_t)(2 * blockIdx.x + s) * p.taken_rows + 32 * quad) * (D / 4) + lane;
      float taken_m = 0.f;
      auto take_over = [&](uint64_t* ready, uint32_t parity, auto&& m_of, bool first, bool back) {
        wait(ready, parity);
        __syncwarp();
        tc_fence_after();
        if (row_item - lane >= q.rows) return;  // nobody's rows
        const float m_now = m_of(), f = taken_m == m_now ? 1.f : exp2_fast((taken_m - m_now) * scores);
        taken_m = m_now;
        take_rows<D, L::kSpare>(O_own, T_own, in_work, f, row_item < q.rows, first, back);
        tc_fence_before();
      };
      float* s_m = reinterpret_cast<float*>(s_jump);  // [group of steps % 2][row]: one stream's m, for the other's warps
      if (kTake && L::kSingle && s == 1) {
        const int all = steps_of<L::kSingle>(q, 0);
        if (all > p.fold)
#pragma unroll 1
          for (int end = p.fold, group = 0;; end += p.fold, ++group) {
            take_over(&o_full, n_full++ & 1, [&] { return s_m[group % 2 * kTile + row]; }, group == 0, end >= all);
            __syncwarp();
            if (end >= all) break;
            if (lane == 0) mbar_arrive(&o_taken);
          }
      }
#pragma unroll 1
      for (int i = 0;; ++i, ++n_s) {
        const bool fresh = kTake && (i & (p.fold - 1)) == 0;  // O begins anew
        if (kTake && !L::kSingle && i > 0 && steps > p.fold && (fresh || i == steps))
          take_over(&o_done[s][(n_s - 1) & 1], ((n_s - 1) >> 1) & 1, [&] { return m; }, i == p.fold, i == steps);
        if (i >= steps) break;
        const int j0 = first_of(i);
        uint32_t see[2];
#pragma unroll
        for (int w = 0; w < 2; ++w) see[w] = __ballot_sync(0xffffffffu, mb[w] != 0);
        if (i + 1 < steps) load_mask(first_of(i + 1), mb);
        if (j0 + kStep > q.P) {
#pragma unroll
          for (int w = 0; w < 2; ++w) {
            const int at = j0 + 32 * w - q.P, k = at >> 5;  // node of the word's first entry
            const uint32_t* anc = s_anc + 8 * node;
            const uint32_t x = k >= 0 && k < 8 ? anc[k] : 0, y = k >= -1 && k < 7 ? anc[k + 1] : 0;
            see[w] |= __funnelshift_r(x, y, at & 31);
          }
        }
        const uint32_t S = lanes + s * kTile + (n_s & 1) * kStep;
        wait(&s_full[s][n_s & 1], (n_s >> 1) & 1);
        __syncwarp();
        tc_fence_after();
        uint32_t v[2][32];
        tc_ld32(S, v[0]);
        tc_ld32(S + 32, v[1]);
        tc_ld_wait(v[0]);
        tc_ld_wait(v[1]);
        float top[2] = {-kMost, -kMost};
#pragma unroll
        for (int w = 0; w < 2; ++w) {
          if (!__all_sync(0xffffffffu, see[w] == 0xffffffffu)) {
#pragma unroll
            for (int e = 0; e < 32; ++e)
              if (!(see[w] >> e & 1)) v[w][e] = 0xFF800000u;  // minus infinity
          }
#pragma unroll
          for (int e = 0; e < 32; e += 4) {
            top[0] = max3(top[0], __uint_as_float(v[w][e]), __uint_as_float(v[w][e + 1]));
            top[1] = max3(top[1], __uint_as_float(v[w][e + 2]), __uint_as_float(v[w][e + 3]));
          }
        }
        const float mx = max3(top[0], top[1], top[1]);
        const bool raise = !((mx - m) * scores <= kLag);  // or NaN
        if (i == 0) {
          m = mx;
        } else if (__any_sync(0xffffffffu, raise)) {
          const float f = raise ? exp2_fast((m - mx) * scores) : 1.f;
          if (raise) m = mx;
          l *= f;
          if (!fresh) {
            wait_o(s, n_s - 1);
            __syncwarp();
            tc_fence_after();
#pragma unroll 1
            for (int w = 0; w < D / 16; ++w) {
              uint32_t x[16];
              tc_ld(O_own + 16 * w, x);
              tc_ld_wait(x);
#pragma unroll
              for (int e = 0; e < 16; ++e) x[e] = __float_as_uint(__uint_as_float(x[e]) * f);
              tc_st16(O_own + 16 * w, x);
            }
            tc_st_wait();
          }
        }
        // an infinite maximum makes the row NaN
        const f32x2 c2 = pair(scores, scores), lift2 = pair(kLift, kLift), less2 = pair(-m, -m);
        f32x2 sum[2] = {0, 0};
#pragma unroll
        for (int w = 0; w < 2; ++w) {
          uint32_t h[16], lo[16], least[16];
#pragma unroll
          for (int e = 0; e < 16; ++e) {
            const f32x2 x = fma2(add2(pair(__uint_as_float(v[w][2 * e]), __uint_as_float(v[w][2 * e + 1])), less2), c2, lift2);
            const float2 t = halves(x), y = make_float2(exp2_fast(t.x), exp2_fast(t.y));
            sum[e & 1] = add2(sum[e & 1], pair(y.x, y.y));
            h[e] = pack2<kBf16>(y.x, y.y);
            if (kF32) {
              const float2 b = unpack2<kBf16>(h[e]), r = make_float2(y.x - b.x, y.y - b.y);
              lo[e] = pack2<kBf16>(r.x, r.y);
              if (L::kSingle) {
                const float2 c = unpack2<kBf16>(lo[e]);
                least[e] = pack2<kBf16>(r.x - c.x, r.y - c.y);
              }
            }
          }
          tc_st16(S + 32 * w, h);
          if (kF32) tc_st16(S + 32 * w + 16, lo);
          if (L::kSingle) tc_st16(lanes + kTile + (n_s & 1) * 32 + 16 * w, least);
        }
        const float2 all = halves(add2(sum[0], sum[1]));
        l += all.x + all.y;
        tc_st_wait();
        tc_fence_before();
        if (kTake && L::kSingle && (((i + 1) & (p.fold - 1)) == 0 || i + 1 == steps)) s_m[(i & p.fold ? kTile : 0) + row] = m;
        __syncwarp();
        if (lane == 0) mbar_arrive(&p_ready[s][n_s & 1]);
      }
      // ---- the piece's end ----
      float2* ml = s_ml + (piece & 1) * 2 * kTile;
      ml[s * kTile + row] = make_float2(m, l);
      named_bar_sync(1, kSoft);
      const bool both = !q.pair && !L::kSingle && nt > 1;  // two streams of the same rows
      float w0 = 1.f, w1 = 0.f, M = m, sum = l;
      if (!q.pair) {
        const float2 x = ml[row], y = ml[kTile + row];
        M = both ? max3(x.x, y.x, y.x) : x.x;
        w0 = x.x == M ? 1.f : exp2_fast((x.x - M) * scores);
        w1 = !both ? 0.f : y.x == M ? 1.f : exp2_fast((y.x - M) * scores);
        sum = both ? x.y * w0 + y.y * w1 : x.y;
      }
      const int steps_1 = steps_of<L::kSingle>(q, 1);
      n_o[0] += steps_of<L::kSingle>(q, 0);
      n_o[1] += steps_1;
      if (!q.pair || s == 0) wait_o(0, n_o[0] - 1);
      if (q.pair ? s == 1 : both) wait_o(1, n_o[1] - 1);
      __syncwarp();
      tc_fence_after();
      const bool whole = q.t0 == 0 && q.t1 == q.tiles;
      const uint32_t O = lanes + 2 * kTile + (q.pair ? s * kTile : 0);
      const int c0 = q.pair ? 0 : s * (D / 2), c1 = q.pair ? D : c0 + D / 2;
      const bool odd = in_tree && s_odd[piece % (2 * L::kSlots)] == (int)piece + 1;
      const size_t slot = (2 * (size_t)blockIdx.x + (piece > 0)) * p.rows_max;  // of a piece of an item that is cut
      if (!whole && row_item < q.rows && c0 == 0) p.ml[slot + row_item] = make_float4(M, sum, scores, 0.f);
      if (whole) {
        const float inv = 1.f / sum;
        w0 *= inv;
        w1 *= inv;
      }
      const bool out16 = whole && a.out_type != SHARD_F32;
      const int first_row = row_item - lane;
      uint8_t* stage = smem + L::kStage + (warp - kSoftWarp0) * 2048;
      // Through shared memory, so that a row's 64 (32) bytes go out together: a warp's store of 16 bytes to each of 32
      // rows took eight times as long. This lane's rows and 16-byte unit of them on the way out:
      const int u_shift = out16 ? 1 : 2, unit = lane & ((1 << u_shift) - 1), r_step = 32 >> u_shift;
      uint8_t* to[4];
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const int ri = first_row + (lane >> u_shift) + k * r_step, g = q.row0 + ri;
        to[k] = nullptr;
        if (ri >= q.rows || k >> u_shift) continue;
        const long long at = (q.start + (g >> p.g_shift)) * a.out_stride + (q.h * G + (g & (G - 1))) * D;
        to[k] = !whole  ? reinterpret_cast<uint8_t*>(p.o + (slot + ri) * D) + 16 * unit
                : out16 ? static_cast<uint8_t*>(a.out) + 2 * at + (p.act_order ? 32 : 16) * unit
                        : static_cast<uint8_t*>(a.out) + 4 * at + 16 * unit;
      }
      if (first_row < q.rows) {
        uint32_t v[16], u[16], v1[16], u1[16];
        tc_ld(O + c0, v1);
        if (both) tc_ld(O + kTile + c0, u1);
#pragma unroll 1
        for (int c = c0; c < c1; c += 16) {
          tc_ld_wait(v1);
          if (both) tc_ld_wait(u1);
#pragma unroll
          for (int e = 0; e < 16; ++e) v[e] = v1[e], u[e] = u1[e];
          if (c + 16 < c1) {
            tc_ld(O + c + 16, v1);
            if (both) tc_ld(O + kTile + c + 16, u1);
          }
#pragma unroll
          for (int e = 0; e < 16; ++e)
            v[e] = __float_as_uint(__uint_as_float(v[e]) * w0 + (both ? __uint_as_float(u[e]) * w1 : 0.f));
          if (odd && row_item < q.rows) {
            // what the tree's entries hold that is not finite, for the rows that see it
            for (int i = max(0, q.t0 * kTile - q.P); i < min(q.n, q.t1 * kTile - q.P); ++i) {
              if (!(s_anc[8 * node + (i >> 5)] >> (i & 31) & 1)) continue;
              const uint32_t* x = reinterpret_cast<const uint32_t*>(
                  static_cast<const uint16_t*>(a.v) + q.b * a.kv_request + q.h * a.kv_head + (long long)(q.P + i) * a.kv_entry + c);
#pragma unroll
              for (int e = 0; e < 8; ++e) {
                const uint32_t two = __ldg(x + e);
                const float2 f = unpack2<kBf16>(two);
                if (odd2<kBf16>(two & 0xFFFFu)) v[2 * e] = __float_as_uint(__uint_as_float(v[2 * e]) + f.x);
                if (odd2<kBf16>(two & 0xFFFF0000u)) v[2 * e + 1] = __float_as_uint(__uint_as_float(v[2 * e + 1]) + f.y);
              }
            }
          }
          if (out16) {
#pragma unroll
            for (int e = 0; e < 8; ++e) {
              const float x = __uint_as_float(v[2 * e]), y = __uint_as_float(v[2 * e + 1]);
              v[e] = a.out_type == SHARD_F16 ? pack2<false>(x, y) : pack2<true>(x, y);
            }
            if (p.act_order) {  // inputs 0..3 and 8..11 lie together, and 4..7 and 12..15, 16 values further
              const uint32_t x = v[2], y = v[3];
              v[2] = v[4], v[3] = v[5], v[4] = x, v[5] = y;
            }
          }
          __syncwarp();  // the last one's reads
#pragma unroll
          for (int e = 0; e < 4; ++e)
            if (!(e >> u_shift))
              *reinterpret_cast<uint4*>(stage + lane * 64 + ((e ^ ((lane >> 1) & 3)) << 4)) =
                  make_uint4(v[4 * e], v[4 * e + 1], v[4 * e + 2], v[4 * e + 3]);
          __syncwarp();
          const int col = !out16 ? 4 * c : p.act_order ? 2 * ((c & ~31) + (c & 16) / 2) : 2 * c;  // bytes
#pragma unroll
          for (int k = 0; k < 4; ++k) {
            const int r = (lane >> u_shift) + k * r_step;
            if (to[k]) *reinterpret_cast<uint4*>(to[k] + col) = *reinterpret_cast<const uint4*>(stage + r * 64 + ((unit ^ ((r >> 1) & 3)) << 4));
          }
        }
      }
      tc_fence_before();
      __syncwarp();
      if (lane == 0) {
        mbar_arrive(&o_free[0]);  // the first stream has steps in every piece
        if (steps_1 > 0) mbar_arrive(&o_free[1]);
      }
      ++piece;
    }
  }
  if (!ok && a.status) atomicOr(a.status, ST_WAIT_TIMEOUT);
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  if (warp == 1)
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "r"(512u) : "memory");
}

// Rows of items that were cut: sum_i 2^((m_i - M) c) O_i over sum_i 2^((m_i - M) c) l_i, the
// pieces in order.  Bound by latency: the plan, then maxima and values together.  A warp per row of the batch (request,
// kv head, node, head): with a grid of items by their most rows, CTAs for rows that are not there took 3 us for 16
// requests of 5 nodes, and the join 17 us instead of 13 after 64 items of 256 rows.
constexpr int kJoinWarps = 16, kJoinPieces = 4;  // rows per CTA; pieces of a row in flight
template <int D>
__global__ void __launch_bounds__(kJoinWarps * 32) tree_combine_kernel(const __grid_constant__ Params p, int rows_item) {
  __shared__ int4 s_plan[SHARD_MAX_TREES];
  __shared__ int s_start[SHARD_MAX_TREES + 1];
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, B = p.a.B;
  static_assert(kJoinWarps * 32 > SHARD_MAX_TREES, "a thread per request");
  pdl_wait();
  pdl_launch_dependents();
  const int4* plan = reinterpret_cast<const int4*>(p.plan);
  const int4 all = __ldcg(plan + B);
  if (tid < B) s_plan[tid] = __ldcg(plan + tid);
  if (tid <= B) s_start[tid] = __ldg(p.a.tree_start + tid);
  if (all.z < 2) return;
  __syncthreads();
  const int G = 1 << p.g_shift;
  const uint32_t batch_row = blockIdx.x * kJoinWarps + warp, heads = (uint32_t)p.a.n_kv_heads << p.g_shift;
  const int node0 = (int)(batch_row / heads);
  int b = -1;  // the request of this row's node
#pragma unroll 1
  for (int b0 = 0; b0 < B && b < 0; b0 += 32) {
    const int at = b0 + lane;
    const uint32_t here = __ballot_sync(0xffffffffu, at < B && s_plan[at].w > 0 && s_start[at] <= node0 && node0 < s_start[at + 1]);
    if (here) b = b0 + __ffs(here) - 1;
  }
  if (b < 0) return;
  const int4 r = s_plan[b];
  const int start = s_start[b], rows = r.w << p.g_shift, parts = (rows + rows_item - 1) / rows_item;
  const int in_request = (int)(batch_row - start * heads), h = in_request / rows, grow = in_request - h * rows;
  const int part = grow / rows_item, row = grow - part * rows_item;  // its item of the kv head, and its row there
  const Runs runs(all.x, all.z);
  const uint32_t u0 = (uint32_t)r.x + (uint32_t)(h * parts + part) * r.z;
  const uint32_t cta0 = runs.of(u0), n = runs.of(u0 + r.z - 1) - cta0 + 1;  // its pieces, a CTA's each
  if (n == 1) return;
  const uint32_t first = 2 * cta0 + (runs.start(cta0) < u0);  // only the first run can begin earlier
  auto slot = [&](uint32_t i) { return (size_t)(i == 0 ? first : 2 * (cta0 + i)) * p.rows_max + row; };
  constexpr int kPer = D / 32;
  const int c = kPer * lane;
  float v[kJoinPieces][kPer];
  auto fetch = [&](uint32_t i0) {
#pragma unroll
    for (int i = 0; i < kJoinPieces; ++i) {
      if (i0 + i >= n) continue;
      const float* o = p.o + slot(i0 + i) * D + c;
      if (kPer == 4) *reinterpret_cast<float4*>(v[i]) = __ldcg(reinterpret_cast<const float4*>(o));
      else *reinterpret_cast<float2*>(v[i]) = __ldcg(reinterpret_cast<const float2*>(o));
    }
  };
  float4 ml = make_float4(-kMost, 0.f, 0.f, 0.f);
  if (lane < n) ml = __ldcg(&p.ml[slot(lane)]);
  fetch(0);
  float M = ml.x;
  const float scores = __shfl_sync(0xffffffffu, ml.z, 0);
  for (uint32_t i = lane + 32; i < n; i += 32) M = fmaxf(M, __ldcg(&p.ml[slot(i)]).x);
#pragma unroll
  for (int o = 16; o > 0; o >>= 1) M = fmaxf(M, __shfl_xor_sync(0xffffffffu, M, o));
  float acc[kPer], sum = 0.f, w = 0.f, l = 0.f;
#pragma unroll
  for (int k = 0; k < kPer; ++k) acc[k] = 0.f;
#pragma unroll 1
  for (uint32_t i0 = 0; i0 < n; i0 += kJoinPieces) {
    if (i0 > 0) fetch(i0);
    if (i0 % 32 == 0) {
      if (i0 > 0) ml = i0 + lane < n ? __ldcg(&p.ml[slot(i0 + lane)]) : make_float4(-kMost, 0.f, 0.f, 0.f);
      w = ml.x == M ? 1.f : exp2_fast((ml.x - M) * scores);
      l = ml.y * w;
    }
#pragma unroll
    for (int i = 0; i < kJoinPieces; ++i) {
      const float wi = __shfl_sync(0xffffffffu, w, (i0 + i) % 32), li = __shfl_sync(0xffffffffu, l, (i0 + i) % 32);
      if (i0 + i >= n) continue;
      sum += li;
      if (wi == 0.f) continue;  // nothing of it is seen, or it is too far below
#pragma unroll
      for (int k = 0; k < kPer; ++k) acc[k] += v[i][k] * wi;
    }
  }
  const float inv = 1.f / sum;
  const long long out = (long long)(start + (grow >> p.g_shift)) * p.a.out_stride + (h * G + (grow & (G - 1))) * D;
  const long long at = out + (p.act_order ? (c & ~31) + act_pos(c & 31) : c);
  if (p.a.out_type == SHARD_F32) {
#pragma unroll
    for (int k = 0; k < kPer; ++k) static_cast<float*>(p.a.out)[at + k] = acc[k] * inv;
  } else {
    uint32_t* o = reinterpret_cast<uint32_t*>(static_cast<uint16_t*>(p.a.out) + at);
#pragma unroll
    for (int k = 0; k < kPer / 2; ++k)
      o[k] = p.a.out_type == SHARD_F16 ? pack2<false>(acc[2 * k] * inv, acc[2 * k + 1] * inv)
                                       : pack2<true>(acc[2 * k] * inv, acc[2 * k + 1] * inv);
  }
}

constexpr size_t kPlanBytes = (16 * (SHARD_MAX_TREES + 1) + 127) / 128 * 128;

template <int D, bool kF32, bool kBf16, int kRows, bool kTake>
cudaError_t launch_kernel(const Params& p, int device, int grid, cudaStream_t s) {
  using L = Geo<D, kF32, kBf16, kRows>;
  static std::atomic<uint64_t> ready{0};  // devices whose limit is raised
  if (device >= 64 || !(ready.load() >> device & 1)) {
    const cudaError_t e = cudaFuncSetAttribute(tree_attention_kernel<D, kF32, kBf16, kRows, kTake>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                               (int)L::kTotal);
    if (e != cudaSuccess) return e;
    if (device < 64) ready.fetch_or(1ull << device);
  }
  return launch_behind(tree_attention_kernel<D, kF32, kBf16, kRows, kTake>, grid, kThreads, L::kTotal, s, p);
}

// units: no fewer than there are
template <int D, bool kF32, bool kBf16, int kRows>
cudaError_t launch(Params& p, int device, int grid, long long units, cudaStream_t s) {
  using L = Geo<D, kF32, kBf16, kRows>;
  const int tiles = kF32 && p.a.out_type == SHARD_F32 ? L::kFold32 : L::kFold;
  p.fold = 2 * tiles;
  // A piece's tiles are no more than the cache's and than a CTA's, and two streams share those of 128 rows.  Where a
  // stream's are within p.fold, the kernel without the code for more (without / with: two caches of 95000 entries 131 / 135
  // us, one stream 257 / 278; trees of 64 on 60000 entries 214 to 225 / 222 to 226).
  const long long piece = std::min<long long>((p.a.capacity + kTile - 1) / kTile, (units + grid - 1) / grid);
  const bool take = (kRows == kTile && !L::kSingle ? (piece + 1) / 2 : piece) > tiles;
  cudaError_t e = take ? launch_kernel<D, kF32, kBf16, kRows, true>(p, device, grid, s) : launch_kernel<D, kF32, kBf16, kRows, false>(p, device, grid, s);
  if (e != cudaSuccess || grid < 2) return e;
  const long long rows = ((long long)p.a.N * p.a.n_kv_heads) << p.g_shift;
  return launch_behind(tree_combine_kernel<D>, dim3((unsigned)((rows + kJoinWarps - 1) / kJoinWarps)), kJoinWarps * 32, 0, s, p, kRows);
}

int taken_rows_of(int rows) { return std::min((rows + 31) / 32 * 32, kTile); }
int rows_of(int N, int G) { return std::min(256, std::min(N, SHARD_MAX_TREE) * G); }

}  // namespace

cudaError_t tree_attention_work(int N, int n_heads, int n_kv_heads, int head_dim, long long* bytes) {
  int device;
  const cudaError_t e = cudaGetDevice(&device);
  if (e != cudaSuccess) return e;
  const int rows = rows_of(N, n_heads / n_kv_heads);
  *bytes = kPlanBytes + 2ll * sms_of(device) * (rows * (head_dim * 4ll + 16) + (head_dim == 64 ? 0 : taken_rows_of(rows) * (head_dim * 4ll)));
  return cudaSuccess;
}

cudaError_t launch_tree_attention(const shard_tree_attn& a, bool act_order, cudaStream_t s) {
  int device;
  cudaError_t e = cudaGetDevice(&device);
  if (e != cudaSuccess) return e;
  EncodeTiledFn enc = encode_tiled();
  const int sms = sms_of(device);
  if (!enc || !sms) return cudaErrorNotSupported;
  Params p;
  p.a = a;
  const int G = a.n_heads / a.n_kv_heads;
  p.g_shift = G == 1 ? 0 : G == 2 ? 1 : G == 4 ? 2 : G == 8 ? 3 : 4;
  p.rows_max = rows_of(a.N, G);
  p.act_order = act_order;
  p.c = std::min(a.scale * 1.44269504f, kMost);
  uint8_t* w = static_cast<uint8_t*>(a.work);
  const size_t rows = 2ull * sms * p.rows_max;
  p.plan = reinterpret_cast<int*>(w);
  p.ml = reinterpret_cast<float4*>(w + kPlanBytes);
  p.o = reinterpret_cast<float*>(w + kPlanBytes + rows * 16);
  p.taken = reinterpret_cast<float4*>(w + kPlanBytes + rows * (16 + 4ull * a.head_dim));
  p.taken_rows = taken_rows_of(p.rows_max);
  // a dimension of one value may have any stride: one that the map takes
  const cuuint64_t dims[4] = {(cuuint64_t)a.head_dim, (cuuint64_t)a.capacity, (cuuint64_t)a.n_kv_heads, (cuuint64_t)a.B};
  const cuuint64_t entry = (cuuint64_t)a.kv_entry * 2;
  const cuuint64_t strides[3] = {entry, a.n_kv_heads > 1 ? (cuuint64_t)a.kv_head * 2 : entry, a.B > 1 ? (cuuint64_t)a.kv_request * 2 : entry};
  const cuuint32_t box[4] = {64, kTile, 1, 1}, one[4] = {1, 1, 1, 1};
  for (int i = 0; i < 2; ++i)
    if (enc(i ? &p.vmap : &p.kmap, a.kv_type == SHARD_BF16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT16, 4,
            const_cast<void*>(i ? a.v : a.k), dims, strides, box, one, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
            CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) != CUDA_SUCCESS)
      return cudaErrorInvalidValue;
  if (a.q_type != SHARD_F32) {
    const cuuint64_t qdims[3] = {(cuuint64_t)a.head_dim, (cuuint64_t)a.n_heads, (cuuint64_t)a.N};
    const cuuint64_t qstrides[2] = {(cuuint64_t)a.head_dim * 2, (cuuint64_t)a.q_stride * 2};
    const cuuint32_t qbox[3] = {64, (cuuint32_t)G, (cuuint32_t)(kTile / G)};
    if (enc(&p.qmap, a.kv_type == SHARD_BF16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT16, 3,
            const_cast<void*>(a.q), qdims, qstrides, qbox, one, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
            CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) != CUDA_SUCCESS)
      return cudaErrorInvalidValue;
  }
  // Items of 256 rows where the requests have more than 128 on the whole: half the reads of a cache that L2 does not hold
  // (256 / 128: two trees of 64 with 8 heads to a kv head on 60000 entries 219 / 301 us, on 4096 entries 54 / 55; 128 rows
  // on 95000 entries 141 / 131, for the slot less).
  const long long nodes = std::min<long long>(a.N, (long long)a.B * SHARD_MAX_TREE);  // of trees; the others are nobody's
  const bool f32 = a.q_type == SHARD_F32, bf = a.kv_type == SHARD_BF16, wide = !f32 && nodes * G > 128ll * a.B;
  const long long items = a.n_kv_heads * ((long long)std::min(a.B, a.N) + nodes * G / (wide ? 256 : 128));
  const long long units = items * ((a.capacity + kTile - 1) / kTile);
  if (units >= (1ll << 31)) return cudaErrorInvalidValue;
  const int grid = (int)std::min<long long>(sms, units);
#define A(D)                                                                                                            \
  if (f32) return bf ? launch<D, true, true, 128>(p, device, grid, units, s) : launch<D, true, false, 128>(p, device, grid, units, s); \
  if (wide) return bf ? launch<D, false, true, 256>(p, device, grid, units, s) : launch<D, false, false, 256>(p, device, grid, units, s); \
  return bf ? launch<D, false, true, 128>(p, device, grid, units, s) : launch<D, false, false, 128>(p, device, grid, units, s);
  if (a.head_dim == 128) { A(128) }
  A(64)
#undef A
}

}  // namespace shard
