// Attention of a tree of drafted tokens over a paged cache (tq_attend_tree).
#include <algorithm>

#include "tq_cache_view.h"

namespace tq {
namespace {

constexpr int kTreeThreads = 256;
constexpr float kLog2e = 1.4426950408889634f;

struct TreeView {
  const void* q;
  uint16_t* out;
  const int32_t *seqs, *lengths, *sizes;
  const uint64_t* masks;
  uint64_t q_stride, out_stride;
  float scale;         // times log2(e)
  uint32_t trees, nodes, heads, group, q16;
};

// What a tree's nodes attend to: slots below `length`, then slots length + j with bit j of a node's mask, below `end`.
struct Seen {
  uint32_t seq, length, end, size;
};
__device__ __forceinline__ Seen seen_by(const CacheView& c, const TreeView& a, uint32_t t) {
  const int32_t s = a.seqs ? a.seqs[t] : (int32_t)t;
  const uint32_t size = a.sizes ? (uint32_t)min(max(a.sizes[t], 0), (int32_t)a.nodes) : a.nodes, length = (uint32_t)max(a.lengths[t], 0);
  if ((uint32_t)s >= c.n_seqs) return Seen{0, 0, 0, size};
  return Seen{(uint32_t)s, min(length, c.capacity), (uint32_t)min((uint64_t)length + size, (uint64_t)c.capacity), size};
}

template <bool INT8>
__device__ __forceinline__ float value_at(const char* from, uint32_t d) {
  if constexpr (INT8) return (float)((const int8_t*)from)[d];
  else return bf16_value(((const uint16_t*)from)[d]);
}

// One head of one node: a token per thread, then a dim per thread.
template <bool INT8>
__global__ __launch_bounds__(kTreeThreads) void k_attend_tree(CacheView c, TreeView a) {
  __shared__ float lds_q[256], lds_p[kTreeThreads], lds_sum[kTreeThreads], lds_wave[2][kTreeThreads / 64];
  __shared__ uint64_t lds_at[kTreeThreads];
  const uint32_t h = blockIdx.x, i = blockIdx.y, t = blockIdx.z, tid = threadIdx.x, D = c.head_dim, kv = h / a.group;
  const Seen s = seen_by(c, a, t);
  const uint64_t row = (uint64_t)t * a.nodes + i, mask = i < s.size ? a.masks[row] : 0;
  const uint32_t end = i < s.size ? s.end : 0;
  if (tid < D) lds_q[tid] = (a.q16 ? bf16_value(((const uint16_t*)a.q)[row * a.q_stride + h * D + tid]) : ((const float*)a.q)[row * a.q_stride + h * D + tid]) * a.scale;
  uint32_t lanes = 16;
  while (lanes < D) lanes *= 2;
  const uint32_t d = tid % lanes, of_group = tid / lanes, groups = kTreeThreads / lanes;
  float top = -INFINITY, total = 0.f, sum = 0.f;
  for (uint32_t begin = 0; begin < end; begin += kTreeThreads) {
    const uint32_t slot = begin + tid;
    uint32_t page = c.n_pages;
    if (slot < end && (slot < s.length || mask >> (slot - s.length) & 1)) page = (uint32_t)c.tables[(uint64_t)s.seq * c.table_stride + (slot >> c.page_shift)];
    const bool there = page < c.n_pages;
    const uint32_t in_page = slot & ((1u << c.page_shift) - 1);
    const uint64_t at = (INT8 ? 1 : 2) * ((uint64_t)(there ? page : 0) * c.page_stride + kv * c.head_stride + in_page * c.slot_stride);
    const uint64_t mark = (((uint64_t)(there ? page : 0) * c.kv_heads + kv) << c.page_shift) + in_page;
    __syncthreads();
    float l = -INFINITY;
    if (there) {
      const float scale = INT8 ? c.k_scale[mark] : 1.f;
      const bool after = fabsf(scale) < INFINITY;   // (an infinite scale makes NaN of a level of zero)
      l = 0.f;
      for (uint32_t x = 0; x < D; ++x) l = fmaf(lds_q[x], after ? value_at<INT8>(c.k + at, x) : value_at<INT8>(c.k + at, x) * scale, l);
      if (after) l *= scale;
    }
    float m = group_max<64>(l);
    if (tid % 64 == 0) lds_wave[0][tid / 64] = m;
    __syncthreads();
    m = top;
    for (int w = 0; w < kTreeThreads / 64; ++w) m = fmaxf(m, lds_wave[0][w]);
    const float base = m == -INFINITY ? 0.f : m, shrink = exp2f(top - base), p = there ? exp2f(l - base) : 0.f;
    top = m;
    const float of_wave = group_sum<64>(p);
    if (tid % 64 == 0) lds_wave[1][tid / 64] = of_wave;
    lds_p[tid] = there && INT8 ? p * c.v_scale[mark] : p;
    lds_at[tid] = there ? at : ~0ull;
    __syncthreads();
    total *= shrink;
    for (int w = 0; w < kTreeThreads / 64; ++w) total += lds_wave[1][w];
    sum *= shrink;
    if (d < D)
      for (uint32_t n = of_group; n < kTreeThreads; n += groups)
        if (lds_at[n] != ~0ull) sum = fmaf(lds_p[n], value_at<INT8>(c.v + lds_at[n], d), sum);
  }
  lds_sum[tid] = sum;
  __syncthreads();
  if (tid >= D) return;
  for (uint32_t g = 1; g < groups; ++g) sum += lds_sum[g * lanes + d];
  a.out[row * a.out_stride + h * D + d] = (uint16_t)pack_bf16(total == 0.f ? 0.f : sum / total, 0.f);
}

int check_tree(const std::string& who, const tq_cache* cache, const tq_tree_args* a, CacheView* c, uint64_t* bytes) {
  if (int rc = view_cache(who, cache, c)) return rc;
  if (!a) return refuse(TQ_E_INVALID_ARG, who + ": null argument");
  if (a->q_type != TQ_FP32 && a->q_type != TQ_BF16) return refuse(TQ_E_UNSUPPORTED, who + ": q is TQ_FP32 or TQ_BF16");
  if (a->heads == 0 || a->heads > 65535 || a->heads % c->kv_heads) return refuse(TQ_E_INVALID_ARG, who + ": heads must be a multiple of kv_heads up to 65535");
  if (a->nodes == 0 || a->nodes > TQ_MAX_NODES) return refuse(TQ_E_UNSUPPORTED, who + ": a tree has 1..64 nodes");
  if (a->trees > 65535) return refuse(TQ_E_UNSUPPORTED, who + ": more than 65535 trees");
  if (!a->seqs && a->trees > c->n_seqs) return refuse(TQ_E_INVALID_ARG, who + ": more trees than sequences, and no seqs");
  if (!(a->scale > 0.f) || !(a->scale < INFINITY)) return refuse(TQ_E_INVALID_ARG, who + ": scale must be positive");
  *bytes = 256;
  return TQ_OK;
}

int attend_tree(const tq_cache* cache, const tq_tree_args* a, void* stream) {
  const std::string who = "tq_attend_tree";
  CacheView c;
  uint64_t bytes = 0;
  if (int rc = check_tree(who, cache, a, &c, &bytes)) return rc;
  if (a->trees == 0) return TQ_OK;
  if (!a->q || !a->out || !a->lengths || !a->masks || !a->workspace) return refuse(TQ_E_INVALID_ARG, who + ": null pointer");
  const uint64_t row = (uint64_t)a->heads * c.head_dim;
  const bool q16 = a->q_type == TQ_BF16;
  if (!aligned_to(a->q, q16 ? 2 : 4) || !aligned_to(a->out, 2) || !aligned_to(a->seqs, 4) || !aligned_to(a->lengths, 4) || !aligned_to(a->sizes, 4) ||
      !aligned_to(a->masks, 8) || !aligned_to(a->workspace, 16))
    return refuse(TQ_E_INVALID_ARG, who + ": a pointer is not aligned to its type (workspace: 16 bytes)");
  if ((a->q_stride && a->q_stride < row) || (a->out_stride && a->out_stride < row)) return refuse(TQ_E_INVALID_ARG, who + ": a stride is smaller than a row");
  if (a->workspace_bytes < bytes)
    return refuse(TQ_E_INVALID_ARG, who + ": the workspace has " + std::to_string(a->workspace_bytes) + " bytes, " + std::to_string(bytes) + " are needed");
  const TreeView v{a->q, (uint16_t*)a->out, a->seqs, a->lengths, a->sizes, a->masks, a->q_stride ? a->q_stride : row, a->out_stride ? a->out_stride : row,
                   a->scale * kLog2e, a->trees, a->nodes, a->heads, a->heads / c.kv_heads, q16};
  auto go = [&](auto kernel) { hipLaunchKernelGGL(kernel, dim3(a->heads, a->nodes, a->trees), dim3(kTreeThreads), 0, (hipStream_t)stream, c, v); };
  cache->type == TQ_INT8 ? go(k_attend_tree<true>) : go(k_attend_tree<false>);
  return launched("tq_attend_tree");
}

}  // namespace
}  // namespace tq

extern "C" int tq_attend_tree(const tq_cache* cache, const tq_tree_args* args, void* stream) {
  return tq::contained("tq_attend_tree", [&] { return tq::attend_tree(cache, args, stream); });
}

extern "C" int tq_attend_tree_workspace(const tq_cache* cache, const tq_tree_args* args, uint64_t* bytes) {
  return tq::contained("tq_attend_tree_workspace", [&] {
    if (!bytes) return tq::refuse(TQ_E_INVALID_ARG, "tq_attend_tree_workspace: null argument");
    tq::CacheView c;
    return tq::check_tree("tq_attend_tree_workspace", cache, args, &c, bytes);
  });
}
