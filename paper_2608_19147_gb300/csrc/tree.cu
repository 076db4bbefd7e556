// Drafted trees (include/shard.h): the entry points and the acceptance of the
// drafts; the attention is tree_attn.cu.
#include <algorithm>
#include <cmath>
#include <cstdarg>
#include <cstdio>

#include "../../include/shard.h"
#include "launch.cuh"
#include "tree.cuh"

namespace shard {
int shard_fail_msg(int code, const char* msg);
}  // namespace shard

using namespace shard;

namespace {

// One CTA per request, a thread per node. Of a node's children that feed its
// target, the first; then the path is a walk along these from node 0 by one
// thread (30 cycles a node). Bound by the kernel's start: 2.3 us for 16 trees, 2.5
// for 64.
__global__ void __launch_bounds__(SHARD_MAX_TREE) tree_accept_kernel(
    int B, int N, const int32_t* tree_start, const int32_t* parents, const int32_t* drafts, const int32_t* targets,
    int path_stride, int32_t* path, int32_t* tokens, int32_t* count, const int32_t* lens, uint8_t* mask, int mask_stride,
    int32_t* status) {
  __shared__ int s_target[SHARD_MAX_TREE], s_next[SHARD_MAX_TREE], s_path[SHARD_MAX_TREE], s_count;
  __shared__ uint8_t s_kept[SHARD_MAX_TREE];
  const int b = blockIdx.x, i = threadIdx.x;
  const int start = tree_start[b], end = tree_start[b + 1];
  int bad = 0;
  if (start < 0 || end < start || end > N || end - start > min(path_stride, SHARD_MAX_TREE)) bad = SHARD_TREE_START;
  const int n = bad ? 0 : end - start, P = mask ? lens[b] : 0;
  if (!bad && mask && (P < 0 || P > mask_stride - n)) bad = SHARD_TREE_LENGTH;
  if (bad) {
    if (i == 0) {
      count[b] = 0;
      if (status) atomicOr(status, bad);
    }
    return;
  }
  if (i < n) s_target[i] = targets[start + i];
  s_next[i] = n;
  s_kept[i] = 0;
  __syncthreads();
  if (i < n) {
    const int p = parents[start + i];
    if (p < -1 || p >= i) {
      if (status) atomicOr(status, SHARD_TREE_PARENT);
    } else if (p >= 0 && drafts[start + i] == s_target[p]) {
      atomicMin(&s_next[p], i);
    }
  }
  __syncthreads();
  if (i == 0) {
    int k = 0;
    for (int at = 0; at < n; at = s_next[at]) s_path[k++] = at, s_kept[at] = 1;
    s_count = k;
    count[b] = k;
  }
  __syncthreads();
  const int k = s_count;
  for (int c = i; c < path_stride; c += blockDim.x) {
    path[(size_t)b * path_stride + c] = c < k ? s_path[c] : -1;
    tokens[(size_t)b * path_stride + c] = c < k ? s_target[s_path[c]] : -1;
  }
  if (!mask) return;
  uint8_t* row = mask + (size_t)b * mask_stride + P;
  if (i < n) row[i] = s_kept[i];
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

#define TREE_CUDA_TRY(expr)                                                                        \
  do {                                                                                             \
    cudaError_t _e = (expr);                                                                       \
    if (_e != cudaSuccess)                                                                         \
      return fail(_e == cudaErrorMemoryAllocation ? SHARD_ENOMEM : SHARD_ECUDA, "%s: %s (%s:%d)", #expr, \
                  cudaGetErrorString(_e), __FILE__, __LINE__);                                     \
  } while (0)

}  // namespace

extern "C" {

int shard_tree_attention_work(int N, int n_heads, int n_kv_heads, int head_dim, long long* bytes) {
  if (!bytes || N < 1 || n_heads < 1 || n_kv_heads < 1 || n_heads % n_kv_heads || (head_dim != 64 && head_dim != 128))
    return fail(SHARD_EINVAL, "shard_tree_attention_work: bad argument");
  TREE_CUDA_TRY(tree_attention_work(N, n_heads, n_kv_heads, head_dim, bytes));
  return SHARD_OK;
}

int shard_tree_attention(const shard_tree_attn* args, void* cuda_stream) {
  if (!args) return fail(SHARD_EINVAL, "shard_tree_attention: null argument");
  shard_tree_attn a = *args;
  if (!a.q || !a.k || !a.v || !a.out || !a.tree_start || !a.parents || !a.lens || !a.work)
    return fail(SHARD_EINVAL, "shard_tree_attention: null pointer");
  if (a.B < 1 || a.B > SHARD_MAX_TREES || a.N < 1 || a.capacity < 1 || a.n_heads < 1 || a.n_kv_heads < 1 ||
      (a.mask && a.mask_stride < 1))
    return fail(SHARD_EINVAL, "shard_tree_attention: B %d (1..%d), N %d, capacity %d, heads %d / %d or mask_stride %d out of range",
                a.B, SHARD_MAX_TREES, a.N, a.capacity, a.n_heads, a.n_kv_heads, a.mask_stride);
  const int G = a.n_heads / a.n_kv_heads;
  if (a.n_heads % a.n_kv_heads || (G != 1 && G != 2 && G != 4 && G != 8 && G != 16) ||
      (a.head_dim != 64 && a.head_dim != 128))
    return fail(SHARD_EUNSUPPORTED, "shard_tree_attention: %d / %d heads of %d (supported: 1, 2, 4, 8 or 16 query heads per kv head, head_dim 64 or 128)",
                a.n_heads, a.n_kv_heads, a.head_dim);
  if (a.q_type < SHARD_F32 || a.q_type > SHARD_BF16 || a.out_type < SHARD_F32 || a.out_type > SHARD_BF16 ||
      (a.kv_type != SHARD_F16 && a.kv_type != SHARD_BF16) || (a.q_type != SHARD_F32 && a.q_type != a.kv_type))
    return fail(SHARD_EUNSUPPORTED, "shard_tree_attention: types q %d, cache %d, out %d", a.q_type, a.kv_type, a.out_type);
  const long long row = (long long)a.n_heads * a.head_dim;
  if (!a.q_stride) a.q_stride = row;
  if (!a.out_stride) a.out_stride = row;
  const int q_size = a.q_type == SHARD_F32 ? 4 : 2, out_size = a.out_type == SHARD_F32 ? 4 : 2;
  if (a.q_stride < row || a.out_stride < row || a.kv_request < 0 || a.kv_head < 0 || a.kv_entry < a.head_dim)
    return fail(SHARD_EINVAL, "shard_tree_attention: a stride is negative or too small");
  auto bits = [](const void* p) { return reinterpret_cast<uintptr_t>(p); };
  if ((bits(a.q) | bits(a.k) | bits(a.v) | bits(a.out) | bits(a.work)) % 16 || a.q_stride * q_size % 16 ||
      a.out_stride * out_size % 16 || a.kv_request % 8 || a.kv_head % 8 || a.kv_entry % 8)
    return fail(SHARD_EINVAL, "shard_tree_attention: a pointer or stride is not a multiple of 16 bytes");
  if (!aligned4(a.tree_start, a.parents, a.lens, a.status))
    return fail(SHARD_EINVAL, "shard_tree_attention: an int32 array is not aligned to its values");
  if (a.scale == 0.f) a.scale = 1.f / sqrtf((float)a.head_dim);
  if (!(a.scale > 0.f && a.scale < INFINITY)) return fail(SHARD_EINVAL, "shard_tree_attention: scale %g", (double)a.scale);
  if ((a.n_kv_heads > 1 && !a.kv_head) || (a.B > 1 && !a.kv_request))
    return fail(SHARD_EINVAL, "shard_tree_attention: a stride of 0");
  // Tiles of entries times items are counted in 32 bits, of trees that may overlap where tree_start is not as it should be.
  const long long tiles = (a.capacity + 127ll) / 128, items = a.n_kv_heads * (long long)a.B * (1 + 2 * G);
  if (a.capacity > (1 << 30) || items >= (1ll << 31) || items * tiles >= (1ll << 31) || (long long)a.N * a.n_heads >= (1ll << 31) || std::max({a.kv_request, a.kv_head, a.kv_entry}) >= (1ll << 39))
    return fail(SHARD_EUNSUPPORTED, "shard_tree_attention: too large a batch or cache");
  OnDeviceOf on(a.q);
  if (on.error()) return fail(SHARD_EINVAL, "shard_tree_attention: q is not device memory");
  long long need;
  TREE_CUDA_TRY(tree_attention_work(a.N, a.n_heads, a.n_kv_heads, a.head_dim, &need));
  if (a.work_bytes < need)
    return fail(SHARD_EINVAL, "shard_tree_attention: work of %lld bytes, %lld needed", a.work_bytes, need);
  TREE_CUDA_TRY(launch_tree_attention(a, false, static_cast<cudaStream_t>(cuda_stream)));
  return SHARD_OK;
}

int shard_tree_accept(int B, int N, const int32_t* tree_start, const int32_t* parents, const int32_t* drafts,
                      const int32_t* targets, int path_stride, int32_t* path, int32_t* tokens, int32_t* count,
                      const int32_t* lens, uint8_t* attention_mask, int mask_stride, int32_t* status,
                      void* cuda_stream) {
  if (!tree_start || !parents || !drafts || !targets || !path || !tokens || !count)
    return fail(SHARD_EINVAL, "shard_tree_accept: null pointer");
  if ((lens == nullptr) != (attention_mask == nullptr))
    return fail(SHARD_EINVAL, "shard_tree_accept: lens and attention_mask go together");
  if (B < 1 || B > SHARD_MAX_TREES || N < 1 || path_stride < 1 || (attention_mask && mask_stride < 1))
    return fail(SHARD_EINVAL, "shard_tree_accept: B %d (1..%d), N %d, path_stride %d or mask_stride %d out of range", B,
                SHARD_MAX_TREES, N, path_stride, mask_stride);
  if (!aligned4(tree_start, parents, drafts, targets, path, tokens, count, lens, status))
    return fail(SHARD_EINVAL, "shard_tree_accept: an int32 array is not aligned to its values");
  OnDeviceOf on(parents);
  if (on.error()) return fail(SHARD_EINVAL, "shard_tree_accept: parents is not device memory");
  tree_accept_kernel<<<B, SHARD_MAX_TREE, 0, static_cast<cudaStream_t>(cuda_stream)>>>(
      B, N, tree_start, parents, drafts, targets, path_stride, path, tokens, count, lens, attention_mask, mask_stride, status);
  TREE_CUDA_TRY(cudaGetLastError());
  return SHARD_OK;
}

}  // extern "C"
