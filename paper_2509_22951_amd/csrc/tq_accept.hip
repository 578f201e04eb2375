// The accepted branch of a tree of drafted tokens, and its keys and values moved together in every layer (tq_tree_accept).
#include <algorithm>
#include <vector>

#include "tq_cache_view.h"

namespace tq {
namespace {

constexpr uint32_t kAcceptThreads = 256, kCaches = 32, kBatch = 8;   // caches of a launch, as many as its arguments hold; tokens in registers

struct AcceptView {
  const uint64_t* masks;
  const int32_t *sizes, *seqs, *lengths, *drafted, *sampled;
  int32_t *path, *accepted, *next, *lengths_out;
  uint32_t trees, nodes, writes;   // writes: this launch writes the branches
};

struct CacheList {
  CacheView of[kCaches];
  uint32_t int8;   // a bit per cache
};

static_assert(sizeof(CacheList) + sizeof(AcceptView) <= 4096, "the arguments of a launch");

// A workgroup takes kAcceptThreads pieces of one cache's tokens of one tree.  Every wavefront finds the branch by itself, a lane per node: a step is one comparison in all
// lanes.  Then lane i looks up the pages of the i-th accepted token, and a thread moves its own piece (16 bytes of a key or value of a head; a scale, score or position)
// of all of them, in order.  A token moves to a slot no higher than its own: what a thread has written no later token of the branch is read from, and within kBatch tokens
// it reads before it writes.  So the move works in place, without a barrier.
//
// Bound: launch, and the chain masks -> branch -> page -> piece -> store: 16 layers of one tree of 8 nodes, 8 heads of 64, 4.2 us (least: 1.8); 28 layers of 16 trees of 64 nodes, 8 heads of 128, 9.0 us (8.6).  A launch per
// layer would cost 28 times the first of these.
__global__ __launch_bounds__(kAcceptThreads) void k_tree_accept(CacheList caches, AcceptView a) {
  const uint32_t lane = threadIdx.x & 63, t = blockIdx.z;
  const uint64_t row = (uint64_t)t * a.nodes;
  const uint32_t size = a.sizes ? (uint32_t)min(max(a.sizes[t], 0), (int32_t)a.nodes) : a.nodes;
  const int32_t length = max(a.lengths[t], 0);
  uint64_t mask = 0;
  int32_t drafted = 0, sampled = 0;
  if (lane < size) mask = a.masks[row + lane], drafted = a.drafted[row + lane], sampled = a.sampled[row + lane];
  uint32_t at = 0, n = size ? 1 : 0, mine = 0;   // mine: the node of the lane-th accepted token
  while (n) {
    const uint64_t up = (uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)mask, at) | (uint64_t)(uint32_t)__builtin_amdgcn_readlane((int)(mask >> 32), at) << 32;
    const int32_t word = __builtin_amdgcn_readlane(sampled, at);
    const uint64_t children = __ballot(lane > at && lane < size && mask == (up | 1ull << lane) && drafted == word);
    if (!children) break;
    at = (uint32_t)__builtin_ctzll(children);
    if (lane == n) mine = at;
    ++n;
  }
  if (a.writes && blockIdx.x == 0 && blockIdx.y == 0 && threadIdx.x < 64) {
    if (lane < a.nodes) a.path[row + lane] = lane < n ? (int32_t)mine : -1;
    if (lane == at) a.next[t] = n ? sampled : -1;
    if (lane == 0) a.accepted[t] = (int32_t)n, a.lengths_out[t] = (int32_t)((uint32_t)length + n);
  }
  if (n < 2) return;

  const CacheView& c = caches.of[blockIdx.y];
  const bool int8 = caches.int8 >> blockIdx.y & 1;
  const int32_t seq = a.seqs ? a.seqs[t] : (int32_t)t;
  if (!c.k || (uint32_t)seq >= c.n_seqs) return;   // (no caches at all: one that is zero)
  __shared__ uint32_t lds_to[64], lds_from[64], lds_to_page[64], lds_from_page[64], lds_moving;
  if (threadIdx.x < 64) {
    const uint32_t to = (uint32_t)length + lane, from = (uint32_t)length + mine;   // (both below 2^32)
    uint32_t to_page = c.n_pages, from_page = c.n_pages;
    if (lane < n && mine != lane && from < c.capacity) {
      const int32_t* table = c.tables + (uint64_t)(uint32_t)seq * c.table_stride;
      to_page = (uint32_t)table[to >> c.page_shift], from_page = (uint32_t)table[from >> c.page_shift];
    }
    const bool moves = to_page < c.n_pages && from_page < c.n_pages;
    const uint64_t moving = __ballot(moves);
    if (moves) {
      const uint32_t i = (uint32_t)__builtin_popcountll(moving & ((1ull << lane) - 1));
      lds_to[i] = to, lds_from[i] = from, lds_to_page[i] = to_page, lds_from_page[i] = from_page;
    }
    if (lane == 0) lds_moving = (uint32_t)__builtin_popcountll(moving);
  }
  __syncthreads();
  const uint32_t moving = lds_moving, in_page = (1u << c.page_shift) - 1, piece = blockIdx.x * kAcceptThreads + threadIdx.x;
  auto each = [&](auto place, auto* pool) {   // place(page, slot) -> element of the pool
    std::remove_pointer_t<decltype(pool)> held[kBatch];
    for (uint32_t i = 0; i < moving; i += kBatch) {
#pragma unroll
      for (uint32_t b = 0; b < kBatch; ++b)
        if (i + b < moving) held[b] = pool[place(lds_from_page[i + b], lds_from[i + b])];
#pragma unroll
      for (uint32_t b = 0; b < kBatch; ++b)
        if (i + b < moving) pool[place(lds_to_page[i + b], lds_to[i + b])] = held[b];
    }
  };
  const uint32_t size_of = int8 ? 1 : 2, of_head = size_of * c.head_dim / 16, wide = 2 * c.kv_heads * of_head, marks = 2 * c.kv_heads;
  if (piece < wide) {
    const bool of_v = piece / of_head >= c.kv_heads;
    const uint32_t head = piece / of_head % c.kv_heads, part = piece % of_head;
    each([&](uint32_t page, uint32_t slot) { return size_of * ((uint64_t)page * c.page_stride + head * c.head_stride + (slot & in_page) * c.slot_stride) / 16 + part; },
         (uint4*)(of_v ? c.v : c.k));
  } else if (piece < wide + marks) {
    const uint32_t p = piece - wide, head = p % c.kv_heads;
    if (int8) each([&](uint32_t page, uint32_t slot) { return (((uint64_t)page * c.kv_heads + head) << c.page_shift) + (slot & in_page); }, (uint32_t*)(p / c.kv_heads ? c.v_scale : c.k_scale));
  } else if (piece < wide + 2 * marks) {
    const uint32_t p = piece - wide - marks, head = p % c.kv_heads;
    uint32_t* of = p / c.kv_heads ? (uint32_t*)c.positions : (uint32_t*)c.scores;
    if (of) each([&](uint32_t, uint32_t slot) { return ((uint64_t)(uint32_t)seq * c.kv_heads + head) * c.capacity + slot; }, of);
  }
}

int tree_accept(uint32_t n, const tq_cache* const* caches, const tq_accept_args* a, void* stream) {
  const std::string who = "tq_tree_accept";
  if (!a || (n && !caches)) return refuse(TQ_E_INVALID_ARG, who + ": null argument");
  if (n > 4096) return refuse(TQ_E_UNSUPPORTED, who + ": more than 4096 caches");
  if (a->nodes == 0 || a->nodes > TQ_MAX_NODES) return refuse(TQ_E_UNSUPPORTED, who + ": a tree has 1..64 nodes");
  if (a->trees > 65535) return refuse(TQ_E_UNSUPPORTED, who + ": more than 65535 trees");
  for (uint32_t i = 0; i < n; ++i) {
    CacheView c;
    if (int rc = view_cache(who, caches[i], &c)) return rc;
    if (!a->seqs && a->trees > c.n_seqs) return refuse(TQ_E_INVALID_ARG, who + ": more trees than sequences, and no seqs");
  }
  // (layers that share their keys would have them moved twice, at the same time)
  std::vector<std::pair<const void*, const void*>> pools(n);
  for (uint32_t i = 0; i < n; ++i) pools[i] = {caches[i]->k, caches[i]->tables};
  std::sort(pools.begin(), pools.end());
  if (std::adjacent_find(pools.begin(), pools.end()) != pools.end()) return refuse(TQ_E_INVALID_ARG, who + ": a cache is there twice");
  if (a->trees == 0) return TQ_OK;
  if (!a->masks || !a->lengths || !a->drafted || !a->sampled || !a->path || !a->accepted || !a->next || !a->lengths_out)
    return refuse(TQ_E_INVALID_ARG, who + ": null pointer");
  if (!aligned_to(a->masks, 8)) return refuse(TQ_E_INVALID_ARG, who + ": masks must be 8-byte aligned");
  for (const void* p : {(const void*)a->sizes, (const void*)a->seqs, (const void*)a->lengths, (const void*)a->drafted, (const void*)a->sampled, (const void*)a->path,
                        (const void*)a->accepted, (const void*)a->next, (const void*)a->lengths_out})
    if (!aligned_to(p, 4)) return refuse(TQ_E_INVALID_ARG, who + ": a pointer is not aligned to its type");
  if (a->lengths_out == a->lengths) return refuse(TQ_E_INVALID_ARG, who + ": lengths_out is lengths, which other workgroups read");
  AcceptView v{a->masks, a->sizes, a->seqs, a->lengths, a->drafted, a->sampled, a->path, a->accepted, a->next, a->lengths_out, a->trees, a->nodes, 1};
  // Scores or positions that several layers share move once, with the first of these: a move in place reads slots that a second one would find moved.
  std::vector<const void*> moving;
  auto first_of = [&](auto*& marks) {
    if (!marks) return;
    const auto at = std::lower_bound(moving.begin(), moving.end(), (const void*)marks);
    if (at != moving.end() && *at == marks) marks = nullptr;
    else moving.insert(at, marks);
  };
  uint32_t done = 0;
  do {
    CacheList list{};
    const uint32_t now = std::min(n - done, kCaches);
    uint32_t groups = 1;
    for (uint32_t i = 0; i < now; ++i) {
      if (int rc = view_cache(who, caches[done + i], &list.of[i])) return rc;
      first_of(list.of[i].scores), first_of(list.of[i].positions);
      const bool int8 = caches[done + i]->type == TQ_INT8;
      list.int8 |= (uint32_t)int8 << i;
      const uint64_t pieces = 2ull * list.of[i].kv_heads * ((int8 ? 1 : 2) * list.of[i].head_dim / 16 + 2);
      groups = std::max(groups, (uint32_t)((pieces + kAcceptThreads - 1) / kAcceptThreads));
    }
    hipLaunchKernelGGL(k_tree_accept, dim3(groups, std::max(now, 1u), a->trees), dim3(kAcceptThreads), 0, (hipStream_t)stream, list, v);
    v.writes = 0;
    done += now;
  } while (done < n);
  return launched("tq_tree_accept");
}

}  // namespace
}  // namespace tq

extern "C" int tq_tree_accept(uint32_t n, const tq_cache* const* caches, const tq_accept_args* args, void* stream) {
  return tq::contained("tq_tree_accept", [&] { return tq::tree_accept(n, caches, args, stream); });
}
