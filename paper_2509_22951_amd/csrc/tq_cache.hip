// The paged cache: new tokens go in (tq_cache_append), tokens with little attention weight go out (tq_cache_evict).
#include <algorithm>

#include "tq_cache_view.h"

namespace tq {
namespace {

struct AppendView {
  const float *q, *k, *v;
  void* q_out;
  const int32_t *seqs, *slots, *positions;
  const float *cos, *sin;
  uint64_t q_stride, k_stride, v_stride, q_out_stride;
  uint32_t heads, rotary_dim, n_positions, adjacent;
  bool by4;   // every row starts on 16 bytes
};

// One workgroup takes some of the heads (query, key and value heads in this order) of one row; LANES lanes of a wavefront take a
// head, 4 values each.  A pair of the halves rotation lies head_dim / 2 values apart: its other half comes from another lane of
// the same group, so a wavefront has read all of its values before it writes any (q_out may be q), and 8 bits' absmax is a
// maximum over the group.
//
// Bound: device memory for prompts; for a few rows the chain slot -> page -> store, beside slot -> angles -> rotation.
template <int LANES, bool INT8, bool Q16>
__global__ __launch_bounds__(256) void k_cache_append(CacheView c, AppendView a) {
  const uint32_t r = blockIdx.x, D = c.head_dim;
  const uint32_t t = threadIdx.x % LANES, head = (blockIdx.y * 256 + threadIdx.x) / LANES;
  const uint32_t n_heads = a.heads + 2 * c.kv_heads;
  const int32_t seq = a.seqs ? a.seqs[r] : (int32_t)r, slot = a.slots[r], pos = a.positions ? a.positions[r] : slot;
  const bool there = (uint32_t)seq < c.n_seqs && (uint32_t)slot < c.capacity && (a.rotary_dim == 0 || (uint32_t)pos < a.n_positions);
  const uint32_t i = 4 * t;
  const bool mine = head < n_heads && i < D;
  const bool is_q = head < a.heads, is_v = head >= a.heads + c.kv_heads;
  const uint32_t h = is_q ? head : is_v ? head - a.heads - c.kv_heads : head - a.heads;
  float x[4] = {0.f, 0.f, 0.f, 0.f};
  if (mine && there) {
    const float* from = (is_q ? a.q + r * a.q_stride : is_v ? a.v + r * a.v_stride : a.k + r * a.k_stride) + h * D + i;
    if (a.by4) {
      const float4 d = *(const float4*)from;
      x[0] = d.x, x[1] = d.y, x[2] = d.z, x[3] = d.w;
    } else {
#pragma unroll
      for (int j = 0; j < 4; ++j) x[j] = from[j];
    }
  }
  if (a.rotary_dim && there) {   // the same for the whole workgroup
    const uint32_t half = a.rotary_dim / 2;
    const bool turned = mine && !is_v && i < a.rotary_dim;
    const float *cs = a.cos + (uint64_t)(uint32_t)pos * half, *sn = a.sin + (uint64_t)(uint32_t)pos * half;
    if (a.adjacent) {
      if (turned) {
        const float c0 = cs[i / 2], s0 = sn[i / 2], c1 = cs[i / 2 + 1], s1 = sn[i / 2 + 1];
        const float y[4] = {x[0] * c0 - x[1] * s0, x[0] * s0 + x[1] * c0, x[2] * c1 - x[3] * s1, x[2] * s1 + x[3] * c1};
#pragma unroll
        for (int j = 0; j < 4; ++j) x[j] = y[j];
      }
    } else {
      const bool second = i >= half;
      const int other = (int)(threadIdx.x & 63) + (second ? -(int)(half / 4) : (int)(half / 4));
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const float y = __shfl(x[j], other & 63);
        const uint32_t at = second ? i + j - half : i + j;
        if (turned) x[j] = second ? y * sn[at] + x[j] * cs[at] : x[j] * cs[at] - y * sn[at];
      }
    }
  }
  if (is_q) {
    if (!mine) return;   // (a group is whole: its lanes of unused places hold nothing that the others need from here on)
    if constexpr (Q16) {
      uint16_t* to = (uint16_t*)a.q_out + r * a.q_out_stride + h * D + i;
      const uint32_t lo = pack_bf16(x[0], x[1]), hi = pack_bf16(x[2], x[3]);
      if (a.by4) *(uint2*)to = make_uint2(lo, hi);
      else to[0] = (uint16_t)lo, to[1] = (uint16_t)(lo >> 16), to[2] = (uint16_t)hi, to[3] = (uint16_t)(hi >> 16);
    } else {
      float* to = (float*)a.q_out + r * a.q_out_stride + h * D + i;
      if (a.by4) *(float4*)to = make_float4(x[0], x[1], x[2], x[3]);
      else
#pragma unroll
        for (int j = 0; j < 4; ++j) to[j] = x[j];
    }
    return;
  }
  if (!there) return;
  const uint32_t page = (uint32_t)c.tables[(uint64_t)(uint32_t)seq * c.table_stride + ((uint32_t)slot >> c.page_shift)];
  const uint32_t in_page = (uint32_t)slot & ((1u << c.page_shift) - 1);
  float scale = 0.f;
  if constexpr (INT8) {
    float top = 0.f;
#pragma unroll
    for (int j = 0; j < 4; ++j) top = max_or_nan(top, fabsf(x[j]));
#pragma unroll
    for (int d = 1; d < LANES; d *= 2) top = max_or_nan(top, __shfl_xor(top, d));
    scale = scale_of(top);
  }
  if (!mine || page >= c.n_pages) return;
  const uint64_t at = (uint64_t)page * c.page_stride + h * c.head_stride + in_page * c.slot_stride + i;
  char* pool = is_v ? c.v : c.k;
  if constexpr (INT8) {
    *(uint32_t*)(pool + at) = (uint32_t)(quantized(x[0], scale) & 255) | (uint32_t)(quantized(x[1], scale) & 255) << 8 |
                              (uint32_t)(quantized(x[2], scale) & 255) << 16 | (uint32_t)quantized(x[3], scale) << 24;
    if (t == 0) (is_v ? c.v_scale : c.k_scale)[(((uint64_t)page * c.kv_heads + h) << c.page_shift) + in_page] = scale;
  } else {
    *(uint2*)(pool + 2 * at) = make_uint2(pack_bf16(x[0], x[1]), pack_bf16(x[2], x[3]));
  }
  if (t == 0 && !is_v) {
    const uint64_t mark = ((uint64_t)(uint32_t)seq * c.kv_heads + h) * c.capacity + (uint32_t)slot;
    if (c.scores) c.scores[mark] = 0.f;
    if (c.positions) c.positions[mark] = pos;
  }
}

int cache_append(const tq_cache* cache, const tq_append_args* a, void* stream) {
  const std::string who = "tq_cache_append";
  CacheView c;
  if (int rc = view_cache(who, cache, &c)) return rc;
  if (!a) return refuse(TQ_E_INVALID_ARG, who + ": null argument");
  if (a->q_out_type != TQ_FP32 && a->q_out_type != TQ_BF16) return refuse(TQ_E_UNSUPPORTED, who + ": q_out is TQ_FP32 or TQ_BF16");
  if (a->pairing > TQ_ROTARY_ADJACENT) return refuse(TQ_E_UNSUPPORTED, who + ": unknown pairing");
  if (a->rotary_dim % 8 || a->rotary_dim > c.head_dim) return refuse(TQ_E_UNSUPPORTED, who + ": rotary_dim must be a multiple of 8 up to head_dim");
  if (a->heads == 0 || a->heads > 65535) return refuse(TQ_E_INVALID_ARG, who + ": heads must be in 1..65535");
  if (a->rows == 0) return TQ_OK;
  if (a->rows > 0x7FFFFFFFu) return refuse(TQ_E_UNSUPPORTED, who + ": too many rows");
  if (!a->q || !a->k || !a->v || !a->q_out || !a->slots || (a->rotary_dim && (!a->cos || !a->sin))) return refuse(TQ_E_INVALID_ARG, who + ": null pointer");
  if (!a->seqs && a->rows > c.n_seqs) return refuse(TQ_E_INVALID_ARG, who + ": more rows than sequences, and no seqs");
  const uint64_t q_row = (uint64_t)a->heads * c.head_dim, kv_row = (uint64_t)c.kv_heads * c.head_dim;
  AppendView v{a->q, a->k, a->v, a->q_out, a->seqs, a->slots, a->positions, a->cos, a->sin, a->q_stride ? a->q_stride : q_row,
               a->k_stride ? a->k_stride : kv_row, a->v_stride ? a->v_stride : kv_row, a->q_out_stride ? a->q_out_stride : q_row,
               a->heads, a->rotary_dim, a->n_positions, a->pairing, false};
  if (v.q_stride < q_row || v.k_stride < kv_row || v.v_stride < kv_row || v.q_out_stride < q_row)
    return refuse(TQ_E_INVALID_ARG, who + ": a stride is smaller than a row");
  const bool q16 = a->q_out_type == TQ_BF16;
  if (a->q_out == (const void*)a->q && (q16 || v.q_out_stride != v.q_stride))
    return refuse(TQ_E_INVALID_ARG, who + ": q_out is q, with another type or stride");
  if (!aligned_to(a->q, 4) || !aligned_to(a->k, 4) || !aligned_to(a->v, 4) || !aligned_to(a->q_out, q16 ? 2 : 4) || !aligned_to(a->seqs, 4) ||
      !aligned_to(a->slots, 4) || !aligned_to(a->positions, 4) || !aligned_to(a->cos, 4) || !aligned_to(a->sin, 4))
    return refuse(TQ_E_INVALID_ARG, who + ": a pointer is not aligned to its type");
  auto fours = [](const void* p, uint64_t stride, size_t size) { return stride % 4 == 0 && aligned_to(p, 4 * size); };
  v.by4 = fours(v.q, v.q_stride, 4) && fours(v.k, v.k_stride, 4) && fours(v.v, v.v_stride, 4) && fours(v.q_out, v.q_out_stride, q16 ? 2 : 4);
  const bool int8 = cache->type == TQ_INT8;
  const uint32_t lanes = c.head_dim <= 16 ? 4 : c.head_dim <= 32 ? 8 : c.head_dim <= 64 ? 16 : c.head_dim <= 128 ? 32 : 64;
  const uint32_t n_heads = a->heads + 2 * c.kv_heads, blocks = (n_heads * lanes + 255) / 256;
  auto go = [&](auto kernel) { hipLaunchKernelGGL(kernel, dim3(a->rows, blocks), dim3(256), 0, (hipStream_t)stream, c, v); };
  auto of = [&](auto n) {
    constexpr int L = decltype(n)::value;
    if (int8) q16 ? go(k_cache_append<L, true, true>) : go(k_cache_append<L, true, false>);
    else q16 ? go(k_cache_append<L, false, true>) : go(k_cache_append<L, false, false>);
  };
  if (lanes == 4) of(std::integral_constant<int, 4>());
  else if (lanes == 8) of(std::integral_constant<int, 8>());
  else if (lanes == 16) of(std::integral_constant<int, 16>());
  else if (lanes == 32) of(std::integral_constant<int, 32>());
  else of(std::integral_constant<int, 64>());
  return launched("tq_cache_append");
}

// ---- eviction --------------------------------------------------------------------------------------------------------

struct EvictView {
  const int32_t *lengths, *since;
  int32_t* lengths_out;
  float* scores_out;
  int32_t* positions_out;
  uint32_t* counts;   // [seq][head]: tokens to move
  uint2* moves;       // [seq][head][keep]: slot to fill, slot it is filled from
  uint32_t keep;
};

constexpr int kSelectThreads = 1024, kMoveThreads = 256;
constexpr uint32_t kProtected = 0xFFFFFFFFu;

// Numbers that compare as the scores do: NaN lowest, the two zeros equal, protected tokens above +infinity.
__device__ __forceinline__ uint32_t rank_of(float score, bool is_protected) {
  if (is_protected) return kProtected;
  if (score != score) return 0;
  const uint32_t b = __float_as_uint(score + 0.f);
  return b & 0x80000000u ? ~b : b | 0x80000000u;
}

// Sum over lower threads of the workgroup, and over all of them; totals: one word per wavefront.
__device__ __forceinline__ uint32_t sum_below(bool v, uint32_t* totals, uint32_t* all) {
  const uint64_t ballot = __ballot(v);
  const uint32_t lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  __syncthreads();
  if (lane == 0) totals[wave] = __popcll(ballot);
  __syncthreads();
  uint32_t below = __popcll(ballot & ((1ull << lane) - 1)), sum = 0;
  for (uint32_t w = 0; w < kSelectThreads / 64; ++w) {
    below += w < wave ? totals[w] : 0;
    sum += totals[w];
  }
  *all = sum;
  return below;
}

// Which tokens of a (sequence, head) stay: the `keep` highest ranks, found 8 bits at a time from the top (a histogram of the
// next 8 bits over those that agree with the bits found), then one pass in the order of the slots that numbers the equal ones at
// the limit, the free slots below `keep` and the kept ones above.
__global__ __launch_bounds__(kSelectThreads) void k_evict_select(CacheView c, EvictView e) {
  __shared__ uint32_t bins[256], totals[kSelectThreads / 64], found[2];
  const uint32_t h = blockIdx.x, s = blockIdx.y, list = s * c.kv_heads + h;
  const uint64_t row = (uint64_t)list * c.capacity;
  const uint32_t length = (uint32_t)min(max(e.lengths[s], 0), (int32_t)c.capacity);
  const int32_t since = e.since ? e.since[s] : 0;
  const bool out_of_place = e.scores_out != c.scores, positions_too = e.positions_out != c.positions;
  auto stay = [&](uint32_t slot) {
    if (out_of_place) e.scores_out[row + slot] = c.scores[row + slot];
    if (positions_too) e.positions_out[row + slot] = c.positions[row + slot];
  };
  if (length <= e.keep) {
    if (threadIdx.x == 0) e.counts[list] = 0;
    for (uint32_t i = threadIdx.x; i < length; i += kSelectThreads) stay(i);
    return;
  }
  auto rank_at = [&](uint32_t i) { return rank_of(c.scores[row + i], e.since && c.positions[row + i] >= since); };
  uint32_t prefix = 0, left = e.keep;   // `left` of those that agree with the prefix stay
  for (int shift = 24; shift >= 0; shift -= 8) {
    if (threadIdx.x < 256) bins[threadIdx.x] = 0;
    __syncthreads();
    for (uint32_t i = threadIdx.x; i < length; i += kSelectThreads) {
      const uint32_t k = rank_at(i);
      if (shift == 24 || (k ^ prefix) >> (shift + 8) == 0) atomicAdd(&bins[k >> shift & 255], 1u);
    }
    __syncthreads();
    if (threadIdx.x == 0) {
      uint32_t b = 255, over = 0;
      while (over + bins[b] < left) over += bins[b--];
      found[0] = b, found[1] = over;
    }
    __syncthreads();
    prefix |= found[0] << shift;
    left -= found[1];
  }
  uint32_t equal = 0, freed = 0, taken = 0;   // numbered so far
  uint2* moves = e.moves + (uint64_t)list * e.keep;
  for (uint32_t first = 0; first < length; first += kSelectThreads) {
    const uint32_t i = first + threadIdx.x;
    const uint32_t k = i < length ? rank_at(i) : 0;
    uint32_t all;
    const bool at_limit = i < length && k == prefix;
    const uint32_t before = equal + sum_below(at_limit, totals, &all);
    equal += all;
    const bool kept = i < length && (k > prefix || (at_limit && before < left));
    const bool frees = i < e.keep && !kept, takes = i >= e.keep && kept;
    const uint32_t f = freed + sum_below(frees, totals, &all);
    freed += all;
    const uint32_t t = taken + sum_below(takes, totals, &all);
    taken += all;
    if (frees) moves[f].x = i;
    if (takes) moves[t].y = i;
    if (kept && i < e.keep) stay(i);
  }
  if (threadIdx.x == 0) e.counts[list] = freed;
}

// Moves keys, values, scales and marks: a group of 16 lanes per token.  No slot is both written and read.
template <bool INT8>
__global__ __launch_bounds__(kMoveThreads) void k_evict_move(CacheView c, EvictView e) {
  const uint32_t h = blockIdx.y, s = blockIdx.z, list = s * c.kv_heads + h;
  if (blockIdx.x == 0 && h == 0 && threadIdx.x == 0) {
    const int32_t length = e.lengths[s];
    e.lengths_out[s] = min(length, (int32_t)min(e.keep, 0x7FFFFFFFu));
  }
  const uint32_t n = e.counts[list];
  const uint64_t row = (uint64_t)list * c.capacity;
  const uint2* moves = e.moves + (uint64_t)list * e.keep;
  const uint32_t lane = threadIdx.x % 16, bytes = c.head_dim * (INT8 ? 1 : 2), mask = (1u << c.page_shift) - 1;
  const int32_t* table = c.tables + (uint64_t)s * c.table_stride;
  for (uint32_t m = (blockIdx.x * kMoveThreads + threadIdx.x) / 16; m < n; m += gridDim.x * (kMoveThreads / 16)) {
    const uint2 mv = moves[m];
    if (lane == 0) {
      e.scores_out[row + mv.x] = c.scores[row + mv.y];
      if (c.positions) e.positions_out[row + mv.x] = c.positions[row + mv.y];
    }
    const uint32_t to = (uint32_t)table[mv.x >> c.page_shift], of = (uint32_t)table[mv.y >> c.page_shift];
    if (to >= c.n_pages || of >= c.n_pages) continue;
    const uint64_t size = INT8 ? 1 : 2;
    const uint64_t d = size * (to * c.page_stride + h * c.head_stride + (mv.x & mask) * c.slot_stride);
    const uint64_t f = size * (of * c.page_stride + h * c.head_stride + (mv.y & mask) * c.slot_stride);
    for (uint32_t b = lane * 16; b < bytes; b += 256) {
      const uint4 k = *(const uint4*)(c.k + f + b), v = *(const uint4*)(c.v + f + b);
      *(uint4*)(c.k + d + b) = k;
      *(uint4*)(c.v + d + b) = v;
    }
    if (INT8 && lane == 0) {
      const uint64_t sd = (((uint64_t)to * c.kv_heads + h) << c.page_shift) + (mv.x & mask), sf = (((uint64_t)of * c.kv_heads + h) << c.page_shift) + (mv.y & mask);
      c.k_scale[sd] = c.k_scale[sf];
      c.v_scale[sd] = c.v_scale[sf];
    }
  }
}

uint64_t evict_counts_bytes(const CacheView& c) { return ((uint64_t)c.n_seqs * c.kv_heads * 4 + 255) / 256 * 256; }

int check_evict(const std::string& who, const tq_cache* cache, const tq_evict_args* a, CacheView* c, uint64_t* bytes) {
  if (int rc = view_cache(who, cache, c)) return rc;
  if (!a) return refuse(TQ_E_INVALID_ARG, who + ": null argument");
  if (a->keep == 0) return refuse(TQ_E_INVALID_ARG, who + ": keep must be at least 1");
  if (!c->scores) return refuse(TQ_E_INVALID_ARG, who + ": the cache has no scores");
  if (a->since && !c->positions) return refuse(TQ_E_INVALID_ARG, who + ": since needs the cache's positions");
  if ((a->positions_out && !c->positions)) return refuse(TQ_E_INVALID_ARG, who + ": positions_out needs the cache's positions");
  *bytes = evict_counts_bytes(*c) + (uint64_t)c->n_seqs * c->kv_heads * std::min(a->keep, c->capacity) * sizeof(uint2);
  return TQ_OK;
}

int cache_evict(const tq_cache* cache, const tq_evict_args* a, void* stream) {
  const std::string who = "tq_cache_evict";
  CacheView c;
  uint64_t need = 0;
  if (int rc = check_evict(who, cache, a, &c, &need)) return rc;
  if (!a->lengths || !a->workspace) return refuse(TQ_E_INVALID_ARG, who + ": null pointer");
  if (a->workspace_bytes < need) return refuse(TQ_E_INVALID_ARG, who + ": the workspace has " + std::to_string(a->workspace_bytes) + " bytes, " + std::to_string(need) + " are needed");
  if (!aligned_to(a->lengths, 4) || !aligned_to(a->lengths_out, 4) || !aligned_to(a->since, 4) || !aligned_to(a->scores_out, 4) ||
      !aligned_to(a->positions_out, 4) || !aligned_to(a->workspace, 16))
    return refuse(TQ_E_INVALID_ARG, who + ": a pointer is not aligned to its type (workspace: 16 bytes)");
  const uint32_t keep = std::min(a->keep, c.capacity);
  EvictView e{a->lengths, a->since, a->lengths_out ? a->lengths_out : a->lengths, a->scores_out ? a->scores_out : c.scores,
              a->positions_out ? a->positions_out : c.positions, (uint32_t*)a->workspace, (uint2*)((char*)a->workspace + evict_counts_bytes(c)), keep};
  hipLaunchKernelGGL(k_evict_select, dim3(c.kv_heads, c.n_seqs), dim3(kSelectThreads), 0, (hipStream_t)stream, c, e);
  const uint32_t most = std::min(keep, c.capacity - keep), groups = kMoveThreads / 16;
  const uint32_t parts = std::max(1u, std::min((most + groups - 1) / groups, std::max(1u, 4096u / (c.kv_heads * c.n_seqs))));
  const dim3 grid(parts, c.kv_heads, c.n_seqs);
  if (cache->type == TQ_INT8) hipLaunchKernelGGL(k_evict_move<true>, grid, dim3(kMoveThreads), 0, (hipStream_t)stream, c, e);
  else hipLaunchKernelGGL(k_evict_move<false>, grid, dim3(kMoveThreads), 0, (hipStream_t)stream, c, e);
  return launched("tq_cache_evict");
}

}  // namespace
}  // namespace tq

extern "C" int tq_cache_append(const tq_cache* cache, const tq_append_args* args, void* stream) {
  return tq::contained("tq_cache_append", [&] { return tq::cache_append(cache, args, stream); });
}

extern "C" int tq_cache_evict(const tq_cache* cache, const tq_evict_args* args, void* stream) {
  return tq::contained("tq_cache_evict", [&] { return tq::cache_evict(cache, args, stream); });
}

extern "C" int tq_cache_evict_workspace(const tq_cache* cache, const tq_evict_args* args, uint64_t* bytes) {
  return tq::contained("tq_cache_evict_workspace", [&] {
    if (!bytes) return tq::refuse(TQ_E_INVALID_ARG, "tq_cache_evict_workspace: null argument");
    tq::CacheView c;
    return tq::check_evict("tq_cache_evict_workspace", cache, args, &c, bytes);
  });
}
