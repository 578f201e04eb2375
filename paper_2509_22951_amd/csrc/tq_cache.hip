// The paged cache: new tokens go in (tq_cache_append), tokens with little attention weight go out (tq_cache_evict).
#include <algorithm>

#include "tq_cache_view.h"

namespace tq {
namespace {

constexpr int kAppendThreads = 256, kMostItems = 6;

struct AppendView {
  const float *q, *k, *v;
  void* q_out;
  const int32_t *seqs, *slots, *positions;
  const float *cos, *sin;
  uint64_t q_stride, k_stride, v_stride, q_out_stride;
  uint32_t heads, rotary_dim, n_positions, adjacent, items;
};

// One workgroup takes a.items * kAppendThreads / LANES of the heads (query, key and value heads in this order) of one row; LANES lanes of a
// wavefront take a head, 4 values each, and a.items heads one after another, all of them requested ahead.  A pair of the halves
// rotation lies rotary_dim / 2 values apart: its other half comes from another lane of the same group, so a wavefront has read all
// of a head before it writes any (q_out may be q), and 8 bits' absmax is a maximum over the group.
//
// Bound: device memory for prompts (8192 rows of 40 heads of 128 to 8 bits, bf16 q: 56 us); for a few rows the chain slot -> page -> store,
// beside slot -> angles -> rotation.
template <int LANES, bool INT8, bool Q16>
__global__ __launch_bounds__(kAppendThreads) void k_cache_append(CacheView c, AppendView a) {
  constexpr uint32_t kGroups = kAppendThreads / LANES;
  const uint32_t r = blockIdx.x, D = c.head_dim;
  const uint32_t t = threadIdx.x % LANES, i = 4 * t, first_head = blockIdx.y * (a.items * kGroups) + threadIdx.x / LANES;
  const uint32_t n_heads = a.heads + 2 * c.kv_heads;
  const int32_t seq = a.seqs ? ((constant_i32*)a.seqs)[r] : (int32_t)r, slot = ((constant_i32*)a.slots)[r], pos = a.positions ? ((constant_i32*)a.positions)[r] : slot;
  const bool there = (uint32_t)seq < c.n_seqs && (uint32_t)slot < c.capacity && (a.rotary_dim == 0 || (uint32_t)pos < a.n_positions);
  f32x4_any x[kMostItems];   // ahead of what decides whether the row is there; read once (512 rows of 40 heads of 128: 8.7 us, past the caches 7.9)
#pragma unroll
  for (int k = 0; k < kMostItems; ++k) {
    if (k && k >= (int)a.items) break;
    const uint32_t head = first_head + k * kGroups < n_heads ? first_head + k * kGroups : 0;
    const bool is_q = head < a.heads, is_v = head >= a.heads + c.kv_heads;
    const uint32_t h = is_q ? head : is_v ? head - a.heads - c.kv_heads : head - a.heads;
    x[k] = __builtin_nontemporal_load((const f32x4_any*)((is_q ? a.q + r * a.q_stride : is_v ? a.v + r * a.v_stride : a.k + r * a.k_stride) + h * D + (i < D ? i : 0)));
  }
  uint32_t page = c.n_pages;
  if (there) page = (uint32_t)((constant_i32*)c.tables)[(uint64_t)(uint32_t)seq * c.table_stride + ((uint32_t)slot >> c.page_shift)];
  const uint32_t half = a.rotary_dim / 2, in_page = (uint32_t)slot & ((1u << c.page_shift) - 1);
  const bool turned = i < a.rotary_dim, second = !a.adjacent && i >= half;
  float cs[4] = {1.f, 1.f, 1.f, 1.f}, sn[4] = {0.f, 0.f, 0.f, 0.f};   // of this lane's values (adjacent pairs: of pairs 0 and 1)
  if (turned && there) {
    const uint64_t at = (uint64_t)(uint32_t)pos * half + (a.adjacent ? i / 2 : second ? i - half : i);
    if (a.adjacent) {
      cs[0] = a.cos[at], cs[1] = a.cos[at + 1], sn[0] = a.sin[at], sn[1] = a.sin[at + 1];
    } else {
      const f32x4_any d = *(const f32x4_any*)(a.cos + at), e = *(const f32x4_any*)(a.sin + at);
#pragma unroll
      for (int j = 0; j < 4; ++j) cs[j] = d[j], sn[j] = e[j];
    }
  }
  const int other = ((int)(threadIdx.x & 63) + (second ? -(int)(half / 4) : (int)(half / 4))) & 63;
#pragma unroll
  for (int k = 0; k < kMostItems; ++k) {
    if (k && k >= (int)a.items) break;
    const uint32_t head = first_head + k * kGroups;
    const bool is_q = head < a.heads, is_v = head >= a.heads + c.kv_heads, mine = head < n_heads && i < D;
    const uint32_t h = is_q ? head : is_v ? head - a.heads - c.kv_heads : head - a.heads;
    float y[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) y[j] = mine && there ? x[k][j] : 0.f;
    if (a.adjacent) {
      if (turned && !is_v) {
        const float z[4] = {y[0] * cs[0] - y[1] * sn[0], y[0] * sn[0] + y[1] * cs[0], y[2] * cs[1] - y[3] * sn[1], y[2] * sn[1] + y[3] * cs[1]};
#pragma unroll
        for (int j = 0; j < 4; ++j) y[j] = z[j];
      }
    } else if (half) {
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const float z = __shfl(y[j], other);
        if (turned && !is_v) y[j] = second ? z * sn[j] + y[j] * cs[j] : y[j] * cs[j] - z * sn[j];
      }
    }
    float scale = 0.f;
    if constexpr (INT8) {
      float top = 0.f;
#pragma unroll
      for (int j = 0; j < 4; ++j) top = max_or_nan(top, fabsf(y[j]));
#pragma unroll
      for (int d = 1; d < LANES; d *= 2) top = max_or_nan(top, __shfl_xor(top, d));
      scale = scale_of(top);
    }
    if (!mine) continue;
    if (is_q) {
      const uint64_t at = r * a.q_out_stride + h * D + i;
      if constexpr (Q16) {
        uint16_t* to = (uint16_t*)a.q_out + at;
        const uint32_t lo = pack_bf16(y[0], y[1]), hi = pack_bf16(y[2], y[3]);
        *(u32x2_any*)to = u32x2_any{lo, hi};
      } else {
        float* to = (float*)a.q_out + at;
        *(f32x4_any*)to = f32x4_any{y[0], y[1], y[2], y[3]};
      }
      continue;
    }
    if (page < c.n_pages) {
      const uint64_t at = (uint64_t)page * c.page_stride + h * c.head_stride + in_page * c.slot_stride + i;
      char* pool = is_v ? c.v : c.k;
      if constexpr (INT8) {
        *(uint32_t*)(pool + at) = (uint32_t)(quantized(y[0], scale) & 255) | (uint32_t)(quantized(y[1], scale) & 255) << 8 |
                                  (uint32_t)(quantized(y[2], scale) & 255) << 16 | (uint32_t)quantized(y[3], scale) << 24;
        if (t == 0) (is_v ? c.v_scale : c.k_scale)[(((uint64_t)page * c.kv_heads + h) << c.page_shift) + in_page] = scale;
      } else {
        *(uint2*)(pool + 2 * at) = make_uint2(pack_bf16(y[0], y[1]), pack_bf16(y[2], y[3]));
      }
      if (t == 0 && !is_v) {
        const uint64_t mark = ((uint64_t)(uint32_t)seq * c.kv_heads + h) * c.capacity + (uint32_t)slot;
        if (c.scores) c.scores[mark] = 0.f;
        if (c.positions) c.positions[mark] = pos;
      }
    }
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
  if ((uint64_t)a->rows * kAppendThreads > 0xFFFFFFFFu) return refuse(TQ_E_UNSUPPORTED, who + ": too many rows for one launch");
  if (!a->q || !a->k || !a->v || !a->q_out || !a->slots || (a->rotary_dim && (!a->cos || !a->sin))) return refuse(TQ_E_INVALID_ARG, who + ": null pointer");
  if (!a->seqs && a->rows > c.n_seqs) return refuse(TQ_E_INVALID_ARG, who + ": more rows than sequences, and no seqs");
  const uint64_t q_row = (uint64_t)a->heads * c.head_dim, kv_row = (uint64_t)c.kv_heads * c.head_dim;
  AppendView v{a->q, a->k, a->v, a->q_out, a->seqs, a->slots, a->positions, a->cos, a->sin, a->q_stride ? a->q_stride : q_row,
               a->k_stride ? a->k_stride : kv_row, a->v_stride ? a->v_stride : kv_row, a->q_out_stride ? a->q_out_stride : q_row,
               a->heads, a->rotary_dim, a->n_positions, a->pairing};
  if (v.q_stride < q_row || v.k_stride < kv_row || v.v_stride < kv_row || v.q_out_stride < q_row)
    return refuse(TQ_E_INVALID_ARG, who + ": a stride is smaller than a row");
  const bool q16 = a->q_out_type == TQ_BF16;
  if (a->q_out == (const void*)a->q && (q16 || v.q_out_stride != v.q_stride))
    return refuse(TQ_E_INVALID_ARG, who + ": q_out is q, with another type or stride");
  if (!aligned_to(a->q, 4) || !aligned_to(a->k, 4) || !aligned_to(a->v, 4) || !aligned_to(a->q_out, q16 ? 2 : 4) || !aligned_to(a->seqs, 4) ||
      !aligned_to(a->slots, 4) || !aligned_to(a->positions, 4) || !aligned_to(a->cos, 4) || !aligned_to(a->sin, 4))
    return refuse(TQ_E_INVALID_ARG, who + ": a pointer is not aligned to its type");
  const bool int8 = cache->type == TQ_INT8;
  const uint32_t lanes = c.head_dim <= 16 ? 4 : c.head_dim <= 32 ? 8 : c.head_dim <= 64 ? 16 : c.head_dim <= 128 ? 32 : 64;
  const uint32_t n_heads = a->heads + 2 * c.kv_heads, groups = kAppendThreads / lanes, rounds = (n_heads + groups - 1) / groups;
  // A head per group of lanes, until there are many more workgroups than the GPU holds; then several per group, so that their loads are on
  // their way together, and as evenly as they divide, since a group without a head waits with the others (40 heads of 128 in 8 bits, through
  // the caches: 8192 rows 75 us with one, 68 with four and one in turn, 62 with five; 1024 rows 12.6 with one, 13.7 with five).
  const uint32_t most = (uint64_t)a->rows * rounds > 16384 ? kMostItems : 1, parts = (rounds + most - 1) / most;
  v.items = (rounds + parts - 1) / parts;
  auto go = [&](auto kernel) { hipLaunchKernelGGL(kernel, dim3(a->rows, parts), dim3(kAppendThreads), 0, (hipStream_t)stream, c, v); };
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
  uint32_t *to, *from;   // [seq][head][keep]: slots to fill, and the slots they are filled from (slices: the last one first)
  uint32_t keep;
  // lists that are cut into slices
  uint32_t slices;         // of a list; 0: not cut
  uint32_t* histograms;    // [round % 2][seq][head][slice][256]
  uint32_t* above;         // [seq][head][slice]: tokens above what is found of the limit
  uint2* found;            // [round][seq][head]: upper bits of the limit, tokens with these bits that stay
};

constexpr int kMoveThreads = 256, kMoveAhead = 2;   // (64 lists, 3000 rows of 128 bytes each: 25.6 us; with four together 26.1, one 28.6)
constexpr uint32_t kMovesInSelect = 512;   // tokens of a list, half of it with fewer than kManyLists lists
constexpr uint32_t kManyLists = 64;
constexpr uint32_t kSlicesTogether = 512;      // workgroups
constexpr uint32_t kListInWorkgroup = 16384;   // slots: one workgroup takes 8 lists of 16384 in 20 us, slices 29; of 20000 it took 44, slices 28
constexpr uint32_t kProtected = 0xFFFFFFFFu;
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

// Numbers that compare as the scores do: NaN lowest, the two zeros equal, protected tokens above +infinity.
__device__ __forceinline__ uint32_t rank_of(float score, bool is_protected) {
  if (is_protected) return kProtected;
  if (score != score) return 0;
  const uint32_t b = __float_as_uint(score + 0.f);
  return b & 0x80000000u ? ~b : b | 0x80000000u;
}

// The ranks of slots first + k * stride .. + 3 of a list, whose slots begin at `row`; those from `length` on are read as the list's first
// ones.  All loads are requested before any of them is used, and without a condition: behind one they would come one after another (8 lists
// of 16384 slots, all of the call: 24.1 us in place of 19.9).  copies: what stays in its place goes to scores_out and positions_out, with
// what will be written over there by a token that is moved.
template <int STRIDES>
__device__ __forceinline__ void ranks_at(const CacheView& c, const EvictView& e, uint64_t row, uint32_t first, uint32_t stride, uint32_t length, int32_t since, bool copies,
                                         uint32_t (&rank)[STRIDES][4]) {
  f32x4_any v[STRIDES];
  i32x4_any p[STRIDES];
  const float* scores = c.scores + row;
  const int32_t* positions = (c.positions ? c.positions : (const int32_t*)c.scores) + row;   // (no use is made of them without positions)
#pragma unroll
  for (int k = 0; k < STRIDES; ++k) {
    const uint32_t i = first + k * stride, at = i < length ? i : 0;   // (a list's room is a multiple of 16 slots)
    v[k] = *(const f32x4_any*)(scores + at), p[k] = *(const i32x4_any*)(positions + at);
  }
  if (copies) {
    const uint32_t stay = min(length, e.keep);
#pragma unroll
    for (int k = 0; k < STRIDES; ++k) {
      const uint32_t i = first + k * stride;
      if (i + 4 <= stay) {
        if (e.scores_out != c.scores) *(f32x4_any*)(e.scores_out + row + i) = v[k];
        if (e.positions_out != c.positions) *(i32x4_any*)(e.positions_out + row + i) = p[k];
      } else {
#pragma unroll
        for (int j = 0; j < 4; ++j)
          if (i + j < stay) {
            if (e.scores_out != c.scores) e.scores_out[row + i + j] = v[k][j];
            if (e.positions_out != c.positions) e.positions_out[row + i + j] = p[k][j];
          }
      }
    }
  }
#pragma unroll
  for (int k = 0; k < STRIDES; ++k)
#pragma unroll
    for (int j = 0; j < 4; ++j) rank[k][j] = rank_of(v[k][j], e.since && p[k][j] >= since);
}

// The bin, from the top, in which the `left`-th token lies; `over` lie above it.  sums: of 256 bins, the highest first.
struct Bin {
  uint32_t bin, over, in;
};
__device__ __forceinline__ Bin find_bin(const uint32_t* sums, uint32_t left) {   // every wavefront for itself
  const uint32_t lane = threadIdx.x & 63;
  const uint4 v = *(const uint4*)&sums[4 * lane];
  const uint32_t n = v.x + v.y + v.z + v.w, upto = wave_prefix_sum(n), before = upto - n;
  const uint64_t at = __ballot(before < left && left <= upto);
  uint32_t over = before, b = 4 * lane, in = v.x;
  if (over + in < left) over += in, in = v.y, ++b;
  if (over + in < left) over += in, in = v.z, ++b;
  if (over + in < left) over += in, in = v.w, ++b;
  const int one = at ? __builtin_ctzll(at) : 63;   // (there is one)
  return {255 - (uint32_t)__builtin_amdgcn_readlane((int)b, one), (uint32_t)__builtin_amdgcn_readlane((int)over, one), (uint32_t)__builtin_amdgcn_readlane((int)in, one)};
}

// Moves keys, values, scales and marks of a list's tokens: a group of 16 lanes per token, first, first + step, ..., AHEAD of them together (a
// token is a chain of list, page tables, then its bytes).  No slot is both written and read.  Bound: memory, for many tokens (16 x 8 lists,
// 4096 rows of 256 bytes of keys and of values each: 117 us, 4.6 TB/s read and written).
template <bool INT8, uint32_t AHEAD>
__device__ __forceinline__ void move_tokens(const CacheView& c, const EvictView& e, uint32_t s, uint32_t h, const uint32_t* slots_to, const uint32_t* slots_from, uint32_t n,
                                            uint32_t first, uint32_t step) {
  const uint32_t list = s * c.kv_heads + h, lane = threadIdx.x % 16, pieces = c.head_dim * (INT8 ? 1 : 2) / 16, mask = (1u << c.page_shift) - 1;
  const uint64_t row = (uint64_t)list * c.capacity, size = INT8 ? 1 : 2;
  const int32_t* table = c.tables + (uint64_t)s * c.table_stride;
  for (uint32_t m = first; m < n; m += AHEAD * step) {
    uint32_t to[AHEAD], of[AHEAD], to_page[AHEAD], of_page[AHEAD];
    bool there[AHEAD];
#pragma unroll
    for (uint32_t i = 0; i < AHEAD; ++i) {
      const uint32_t at = min(m + i * step, n - 1);
      to[i] = min(slots_to[at], c.capacity - 1), of[i] = min(slots_from[e.slices ? n - 1 - at : at], c.capacity - 1);   // (lengths that change)
    }
#pragma unroll
    for (uint32_t i = 0; i < AHEAD; ++i) {
      to_page[i] = (uint32_t)table[to[i] >> c.page_shift], of_page[i] = (uint32_t)table[of[i] >> c.page_shift];
      there[i] = m + i * step < n && to_page[i] < c.n_pages && of_page[i] < c.n_pages;
    }
    auto place = [&](uint32_t page, uint32_t slot) { return size * (page * c.page_stride + h * c.head_stride + (slot & mask) * c.slot_stride); };
    auto mark = [&](uint32_t page, uint32_t slot) { return (((uint64_t)page * c.kv_heads + h) << c.page_shift) + (slot & mask); };
    // a lane's pieces of 16 bytes: of the key's, then of the value's
    for (uint32_t p0 = lane; p0 - lane < 2 * pieces; p0 += 32) {
      u32x4 x[AHEAD][2];
      const bool more = p0 - lane + 16 < 2 * pieces;
      auto piece = [&](uint32_t p) { return p < pieces ? c.k + 16 * p : c.v + 16 * (p - pieces); };
      auto load = [&](int half) {   // (in place of a token that is not moved, one of page 0)
        const uint32_t p = p0 + 16 * half;
        const char* from = piece(p < 2 * pieces ? p : 0);
#pragma unroll
        for (uint32_t i = 0; i < AHEAD; ++i) x[i][half] = __builtin_nontemporal_load((const u32x4*)(from + place(there[i] ? of_page[i] : 0, of[i])));
      };
      auto store = [&](int half) {
        const uint32_t p = p0 + 16 * half;
        char* to_piece = piece(p);
#pragma unroll
        for (uint32_t i = 0; i < AHEAD; ++i)
          if (there[i] && p < 2 * pieces) __builtin_nontemporal_store(x[i][half], (u32x4*)(to_piece + place(to_page[i], to[i])));
      };
      load(0);
      if (more) load(1);
      store(0);
      if (more) store(1);
    }
    if (lane < AHEAD && m + lane * step < n) {   // a lane per token
      uint32_t t = to[0], f = of[0], tp = to_page[0], fp = of_page[0];
#pragma unroll
      for (uint32_t i = 1; i < AHEAD; ++i)
        if (lane == i) t = to[i], f = of[i], tp = to_page[i], fp = of_page[i];
      e.scores_out[row + t] = c.scores[row + f];
      if (c.positions) e.positions_out[row + t] = c.positions[row + f];
      if (INT8 && tp < c.n_pages && fp < c.n_pages) {
        c.k_scale[mark(tp, t)] = c.k_scale[mark(fp, f)];
        c.v_scale[mark(tp, t)] = c.v_scale[mark(fp, f)];
      }
    }
  }
}

// Which tokens of a (sequence, head) stay: the `keep` highest ranks, found 8 bits at a time from the top (a histogram of the next
// 8 bits over those that agree with the bits found), then one look in the order of the slots that numbers the equal ones at the
// limit, the free slots below `keep` and the kept ones above.
//
// A workgroup per list; a thread has 4 neighbouring slots of every kStride, and their ranks in registers.  Scores share few exponents, so
// that a histogram of the top 8 bits would have a wavefront's lanes add to few words one after another: there are several copies of it.
// Bound: one workgroup's chain of loads, four rounds of histogram and look, numbering: 8 lists of 1152 slots 6.7 us with their 128 moves, of
// 16384 18.  MOVES: the tokens are moved here too (lengths_out is not lengths, and there are few of them).
template <int THREADS, int STRIDES, bool INT8, bool MOVES>
__global__ __launch_bounds__(THREADS) void k_evict_select(CacheView c, EvictView e) {
  constexpr int kWaves = THREADS / 64, kCopies = kWaves < 8 ? kWaves : 8;   // (a copy per lane: 16384 slots 19.9 -> 22.8 us, to clear and add up)
  __shared__ __attribute__((aligned(16))) uint32_t bins[256 * kCopies], sums[256], totals[2][64];
  constexpr uint32_t kStride = THREADS * 4;
  const uint32_t h = blockIdx.x, s = blockIdx.y, list = s * c.kv_heads + h, lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const uint64_t row = (uint64_t)list * c.capacity;
  const uint32_t length = (uint32_t)min(max(e.lengths[s], 0), (int32_t)c.capacity);
  const int32_t since = e.since ? e.since[s] : 0;
  const uint32_t stay = min(length, e.keep);
  uint32_t rank[STRIDES][4];
  auto slot_of = [&](int k) { return k * kStride + threadIdx.x * 4; };
  const bool copies = e.scores_out != c.scores || e.positions_out != c.positions;
  if (MOVES && h == 0 && threadIdx.x == 0) e.lengths_out[s] = min(e.lengths[s], (int32_t)min(e.keep, 0x7FFFFFFFu));
  if (length <= e.keep) {
    if (threadIdx.x == 0) e.counts[list] = 0;
    if (copies) ranks_at<STRIDES>(c, e, row, slot_of(0), kStride, length, since, true, rank);
    return;
  }
  if (threadIdx.x < 64 * kCopies) *(uint4*)&bins[threadIdx.x * 4] = make_uint4(0, 0, 0, 0);
  static_assert(64 * kCopies <= THREADS && kCopies % 4 == 0, "a thread clears four words, of one bin");
  ranks_at<STRIDES>(c, e, row, slot_of(0), kStride, length, since, copies, rank);
  __syncthreads();
  uint32_t prefix = 0, left = e.keep;   // `left` of those that agree with the prefix stay
  for (int shift = 24; shift >= 0; shift -= 8) {
#pragma unroll
    for (int k = 0; k < STRIDES; ++k) {
      const uint32_t i = slot_of(k);
#pragma unroll
      for (int j = 0; j < 4; ++j)
        if (i + j < length && (shift == 24 || (rank[k][j] ^ prefix) >> ((shift + 8) & 31) == 0))
          atomicAdd(&bins[(rank[k][j] >> shift & 255) * kCopies + (lane & (kCopies - 1))], 1u);
    }
    __syncthreads();
    if (threadIdx.x < 64 * kCopies) {   // kCopies / 4 lanes per bin
      const uint4 v = *(const uint4*)&bins[threadIdx.x * 4];
      *(uint4*)&bins[threadIdx.x * 4] = make_uint4(0, 0, 0, 0);
      uint32_t n = v.x + v.y + v.z + v.w;
#pragma unroll
      for (int d = 1; d < kCopies / 4; d *= 2) n += __shfl_xor(n, d);
      if (threadIdx.x % (kCopies / 4) == 0) sums[255 - threadIdx.x / (kCopies / 4)] = n;   // from the top
    }
    __syncthreads();
    const Bin found = find_bin(sums, left);
    prefix |= found.bin << shift;
    left -= found.over;
    if (found.in == left) break;   // all of these stay
  }
  // The numbering.  Sums over all wavefronts and strides before this wavefront's: totals has a word for each, in that order.
  static_assert(STRIDES * kWaves <= 64, "a lane per word");
  auto before_each = [&](uint32_t word, uint32_t (&at)[STRIDES]) {
    const uint32_t upto = wave_prefix_sum(word), below = upto - word;
#pragma unroll
    for (int k = 0; k < STRIDES; ++k) at[k] = (uint32_t)__builtin_amdgcn_readlane((int)below, k * kWaves + wave);
    return (uint32_t)__builtin_amdgcn_readlane((int)upto, 63);
  };
  __shared__ uint32_t few[2][MOVES ? kMovesInSelect : 1];   // the list, where it is used here
  uint32_t *to = MOVES ? few[0] : e.to + (uint64_t)list * e.keep, *from = MOVES ? few[1] : e.from + (uint64_t)list * e.keep;
  if (threadIdx.x < 64) totals[0][threadIdx.x] = totals[1][threadIdx.x] = 0;   // (more than there are of them with one stride)
  __syncthreads();
  uint32_t eq[STRIDES], at[STRIDES];
#pragma unroll
  for (int k = 0; k < STRIDES; ++k) {
    uint32_t n = 0;
#pragma unroll
    for (int j = 0; j < 4; ++j) n += slot_of(k) + j < length && rank[k][j] == prefix;
    const uint32_t upto = wave_prefix_sum(n);
    if (lane == 63) totals[0][k * kWaves + wave] = upto;
    eq[k] = upto - n;
  }
  __syncthreads();
  before_each(totals[0][lane], at);
  uint32_t packed[STRIDES], upto[STRIDES];   // a bit per slot: 0..3 it becomes free, 4..7 its token moves; both counts, up to and with this lane
#pragma unroll
  for (int k = 0; k < STRIDES; ++k) {
    const uint32_t i = slot_of(k);
    uint32_t before = at[k] + eq[k];
    packed[k] = 0;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const bool here = i + j < length, tie = here && rank[k][j] == prefix, kept = here && (rank[k][j] > prefix || (tie && before < left));
      before += tie;
      packed[k] |= (uint32_t)(i + j < stay && !kept) << j | (uint32_t)(i + j >= e.keep && kept) << (4 + j);
    }
    upto[k] = wave_prefix_sum((uint32_t)__builtin_popcount(packed[k] & 15) << 16 | (uint32_t)__builtin_popcount(packed[k] >> 4));
    if (lane == 63) totals[1][k * kWaves + wave] = upto[k];
  }
  __syncthreads();
  static_assert(kStride * STRIDES <= 1u << 15, "either count in 16 bits: at most half of the slots move");
  const uint32_t moves = before_each(totals[1][lane], at) & 0xFFFF;
#pragma unroll
  for (int k = 0; k < STRIDES; ++k) {
    const uint32_t i = slot_of(k), frees = packed[k] & 15, takes = packed[k] >> 4, below = at[k] + upto[k];
    uint32_t f = (below >> 16) - (uint32_t)__builtin_popcount(frees), t = (below & 0xFFFF) - (uint32_t)__builtin_popcount(takes);
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      if (frees >> j & 1) to[f++] = i + j;
      if (takes >> j & 1) from[t++] = i + j;
    }
  }
  if constexpr (MOVES) {
    __syncthreads();
    move_tokens<INT8, 4>(c, e, s, h, few[0], few[1], moves, threadIdx.x / 16, THREADS / 16);
  } else if (threadIdx.x == 0) {
    e.counts[list] = moves;
  }
}

// The same for lists that are more than a workgroup has registers for: a workgroup per slice, a launch per 8 bits of the limit (rounds
// 0..3: the slice's histogram of these bits) and one that numbers (round 4).  Each begins with the sum of the slices' histograms of the
// launch before.  With K kept tokens before it, a free slot i below `keep` is the list's (i - K)-th, and a kept one at or above `keep` the
// (keep - 1 - K)-th from the end of those that move, so that K is all a slice has to know of the others.
constexpr int kSliceThreads = 1024;
template <int STRIDES>
__global__ __launch_bounds__(kSliceThreads) void k_evict_slice(CacheView c, EvictView e, uint32_t round) {
  constexpr int kWaves = kSliceThreads / 64, kCopies = 16;
  constexpr uint32_t kStride = kSliceThreads * 4, kSlice = kStride * STRIDES;
  __shared__ __attribute__((aligned(16))) uint32_t bins[256 * kCopies], sums[256], totals[4][64];
  const uint32_t slice = blockIdx.x, h = blockIdx.y, s = blockIdx.z, list = s * c.kv_heads + h, lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const uint32_t lists = c.n_seqs * c.kv_heads, length = (uint32_t)min(max(e.lengths[s], 0), (int32_t)c.capacity);
  if (length <= e.keep && slice == 0 && threadIdx.x == 0) e.counts[list] = 0;
  if (slice * kSlice >= length || (length <= e.keep && round)) return;
  auto slot_of = [&](int k) { return slice * kSlice + k * kStride + threadIdx.x * 4; };
  uint32_t rank[STRIDES][4];
  ranks_at<STRIDES>(c, e, (uint64_t)list * c.capacity, slot_of(0), kStride, length, e.since ? e.since[s] : 0, round == 0 && (e.scores_out != c.scores || e.positions_out != c.positions), rank);
  if (length <= e.keep) return;
  const uint32_t slices = (length + kSlice - 1) / kSlice;
  auto histogram_of = [&](uint32_t r, uint32_t q) { return (uint4*)(e.histograms + (((uint64_t)(r % 2) * lists + list) * e.slices + q) * 256); };
  uint32_t prefix = 0, left = e.keep, above = 0;   // `left` of those that agree with the prefix stay; the slice's tokens above it
  uint32_t bin = 0;
  if (round) {
    if (round > 1) {
      const uint2 f = e.found[(uint64_t)(round - 1) * lists + list];
      prefix = f.x, left = f.y;
    }
    uint4 n = make_uint4(0, 0, 0, 0);
    for (uint32_t q = wave; q < slices; q += kWaves) {
      const uint4 v = histogram_of(round - 1, q)[lane];
      n.x += v.x, n.y += v.y, n.z += v.z, n.w += v.w;
    }
    *(uint4*)&bins[wave * 256 + 4 * lane] = n;
    __syncthreads();
    if (threadIdx.x < 256) {
      uint32_t sum = 0;
#pragma unroll
      for (int w = 0; w < kWaves; ++w) sum += bins[w * 256 + threadIdx.x];
      sums[255 - threadIdx.x] = sum;
    }
    __syncthreads();
    const Bin found = find_bin(sums, left);
    bin = found.bin;
    prefix |= bin << (32 - 8 * round);
    left -= found.over;
  }
  auto above_in = [&](uint4 v) { return (4 * lane > bin ? v.x : 0u) + (4 * lane + 1 > bin ? v.y : 0u) + (4 * lane + 2 > bin ? v.z : 0u) + (4 * lane + 3 > bin ? v.w : 0u); };
  if (round < 4) {
    *(uint4*)&bins[threadIdx.x * 4] = make_uint4(0, 0, 0, 0);
    static_assert(256 * kCopies == kSliceThreads * 4 && kWaves <= kCopies, "a thread clears four words, of one bin; a wavefront's sums fit");
    if (round && wave == 0) {
      above = above_in(histogram_of(round - 1, slice)[lane]);
      above = (uint32_t)__builtin_amdgcn_readlane((int)wave_prefix_sum(above), 63);
      if (lane == 0) {
        uint32_t* to = e.above + (uint64_t)list * e.slices + slice;
        *to = above + (round > 1 ? *to : 0);
        if (slice == 0) e.found[(uint64_t)round * lists + list] = make_uint2(prefix, left);
      }
    }
    __syncthreads();
    const uint32_t shift = 24 - 8 * round;
#pragma unroll
    for (int k = 0; k < STRIDES; ++k)
#pragma unroll
      for (int j = 0; j < 4; ++j)
        if (slot_of(k) + j < length && (round == 0 || (rank[k][j] ^ prefix) >> ((shift + 8) & 31) == 0))
          atomicAdd(&bins[(rank[k][j] >> shift & 255) * kCopies + (lane & (kCopies - 1))], 1u);
    __syncthreads();
    const uint4 v = *(const uint4*)&bins[threadIdx.x * 4];
    uint32_t n = v.x + v.y + v.z + v.w;
#pragma unroll
    for (int d = 1; d < kCopies / 4; d *= 2) n += __shfl_xor(n, d);
    if (threadIdx.x % (kCopies / 4) == 0) ((uint32_t*)histogram_of(round, slice))[threadIdx.x / (kCopies / 4)] = n;
    return;
  }
  // what the slices before this one have above the limit and at it
  uint32_t over = 0, equal = 0;
  for (uint32_t q = wave; q < slice; q += kWaves) {
    const uint4 v = histogram_of(3, q)[lane];
    over += above_in(v) + (lane == 0 ? e.above[(uint64_t)list * e.slices + q] : 0);
    equal += 4 * lane == (bin & ~3u) ? (bin & 2 ? bin & 1 ? v.w : v.z : bin & 1 ? v.y : v.x) : 0;
  }
  over = wave_prefix_sum(over), equal = wave_prefix_sum(equal);
  if (threadIdx.x < 4 * 64) totals[threadIdx.x / 64][lane] = 0;   // (with fewer strides there are fewer of them)
  __syncthreads();
  if (lane == 63) totals[0][wave] = over, totals[1][wave] = equal;
  static_assert(STRIDES * kWaves <= 64, "a lane per word");
  auto before_each = [&](uint32_t word, uint32_t (&at)[STRIDES]) {   // over all wavefronts and strides before this wavefront's
    const uint32_t below = wave_prefix_sum(word) - word;
#pragma unroll
    for (int k = 0; k < STRIDES; ++k) at[k] = (uint32_t)__builtin_amdgcn_readlane((int)below, k * kWaves + wave);
  };
  uint32_t tie[STRIDES], kept[STRIDES], before[STRIDES], at[STRIDES];
#pragma unroll
  for (int k = 0; k < STRIDES; ++k) {
    uint32_t n = 0;
#pragma unroll
    for (int j = 0; j < 4; ++j) n += slot_of(k) + j < length && rank[k][j] == prefix;
    const uint32_t upto = wave_prefix_sum(n);
    if (lane == 63) totals[2][k * kWaves + wave] = upto;
    tie[k] = upto - n;
  }
  __syncthreads();
  const uint32_t over_before = (uint32_t)__builtin_amdgcn_readlane((int)wave_prefix_sum(totals[0][lane]), 63);
  const uint32_t equal_before = (uint32_t)__builtin_amdgcn_readlane((int)wave_prefix_sum(totals[1][lane]), 63);
  before_each(totals[2][lane], at);
#pragma unroll
  for (int k = 0; k < STRIDES; ++k) {
    uint32_t order = equal_before + at[k] + tie[k];
    kept[k] = 0;   // a bit per slot
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const bool here = slot_of(k) + j < length, same = here && rank[k][j] == prefix;
      kept[k] |= (uint32_t)(here && (rank[k][j] > prefix || (same && order < left))) << j;
      order += same;
    }
    const uint32_t n = (uint32_t)__builtin_popcount(kept[k]), upto = wave_prefix_sum(n);
    if (lane == 63) totals[3][k * kWaves + wave] = upto;
    before[k] = upto - n;
  }
  __syncthreads();
  before_each(totals[3][lane], at);
  uint32_t *to = e.to + (uint64_t)list * e.keep, *from = e.from + (uint64_t)list * e.keep;
#pragma unroll
  for (int k = 0; k < STRIDES; ++k) {
    uint32_t n = over_before + min(equal_before, left) + at[k] + before[k];   // kept tokens before slot i
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const uint32_t i = slot_of(k) + j;
      const bool stays = kept[k] >> j & 1;
      if (i < e.keep && !stays && n <= i) to[i - n] = i;   // (the bounds: lengths that change under the call)
      if (i >= e.keep && stays && n < e.keep) from[e.keep - 1 - n] = i;
      n += stays;
      if (i + 1 == e.keep) e.counts[list] = e.keep - min(n, e.keep);
    }
  }
}

template <bool INT8>
__global__ __launch_bounds__(kMoveThreads) void k_evict_move(CacheView c, EvictView e) {
  const uint32_t h = blockIdx.y, s = blockIdx.z;
  if (blockIdx.x == 0 && h == 0 && threadIdx.x == 0) {
    const int32_t length = e.lengths[s];
    e.lengths_out[s] = min(length, (int32_t)min(e.keep, 0x7FFFFFFFu));
  }
  const uint32_t list = s * c.kv_heads + h;
  move_tokens<INT8, kMoveAhead>(c, e, s, h, e.to + (uint64_t)list * e.keep, e.from + (uint64_t)list * e.keep, e.counts[list], (blockIdx.x * kMoveThreads + threadIdx.x) / 16, gridDim.x * (kMoveThreads / 16));
}

uint64_t evict_counts_bytes(const CacheView& c) { return ((uint64_t)c.n_seqs * c.kv_heads * 4 + 255) / 256 * 256; }

uint64_t evict_moves_bytes(const CacheView& c, uint32_t keep) { return ((uint64_t)c.n_seqs * c.kv_heads * std::min(keep, c.capacity) * sizeof(uint2) + 255) / 256 * 256; }
// A slice has as few strides as let all workgroups be on the GPU together (two per compute unit): 8 lists of 20000 slots 28 us with one stride
// and 32 with two, 128 of them 74 and 69, of 32768 95 and 81.
uint32_t evict_strides(const CacheView& c) {
  const uint64_t pieces = (uint64_t)c.n_seqs * c.kv_heads * ((c.capacity + 4 * kSliceThreads - 1) / (4 * kSliceThreads));
  return pieces <= kSlicesTogether ? 1 : pieces <= 2 * kSlicesTogether ? 2 : 4;
}
// Slices of a list, or 0 where a workgroup takes the whole of it
uint32_t evict_slices(const CacheView& c) {
  const uint32_t slots = 4 * kSliceThreads * evict_strides(c);
  return c.capacity <= kListInWorkgroup ? 0 : (c.capacity + slots - 1) / slots;
}
uint64_t evict_slices_bytes(const CacheView& c) {   // histograms of two rounds, above, found
  const uint64_t lists = (uint64_t)c.n_seqs * c.kv_heads, slices = evict_slices(c);
  return slices ? lists * (slices * (2 * 256 + 1) * sizeof(uint32_t) + 4 * sizeof(uint2)) : 0;
}

int check_evict(const std::string& who, const tq_cache* cache, const tq_evict_args* a, CacheView* c, uint64_t* bytes) {
  if (int rc = view_cache(who, cache, c)) return rc;
  if (!a) return refuse(TQ_E_INVALID_ARG, who + ": null argument");
  if (a->keep == 0) return refuse(TQ_E_INVALID_ARG, who + ": keep must be at least 1");
  if (!c->scores) return refuse(TQ_E_INVALID_ARG, who + ": the cache has no scores");
  if (a->since && !c->positions) return refuse(TQ_E_INVALID_ARG, who + ": since needs the cache's positions");
  if ((a->positions_out && !c->positions)) return refuse(TQ_E_INVALID_ARG, who + ": positions_out needs the cache's positions");
  *bytes = evict_counts_bytes(*c) + evict_moves_bytes(*c, a->keep) + evict_slices_bytes(*c);
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
              a->positions_out ? a->positions_out : c.positions, (uint32_t*)a->workspace, (uint32_t*)((char*)a->workspace + evict_counts_bytes(c)), nullptr, keep};
  const uint64_t n_lists = (uint64_t)c.n_seqs * c.kv_heads;
  e.from = e.to + n_lists * keep;
  e.slices = evict_slices(c);
  e.found = (uint2*)((char*)a->workspace + evict_counts_bytes(c) + evict_moves_bytes(c, keep));
  e.histograms = (uint32_t*)(e.found + 4 * n_lists);
  e.above = e.histograms + 2 * n_lists * e.slices * 256;
  const bool int8 = cache->type == TQ_INT8;
  const uint32_t most = std::min(keep, c.capacity - keep);   // tokens to move, of a list
  // Few of them are moved by the workgroup that has found them, unless others may still have to read the lengths that it writes: 8 lists of
  // 1152 slots, 128 moves 6.7 us in place of 8.7, 400 moves 10.4 in place of 9.0; 128 lists of them 8.6 in place of 12.6, 13.2 in place of 17.8.
  const bool moves = !e.slices && e.lengths_out != e.lengths && most <= (c.n_seqs * c.kv_heads < kManyLists ? kMovesInSelect / 2 : kMovesInSelect);
  const dim3 lists(c.kv_heads, c.n_seqs);
  hipStream_t st = (hipStream_t)stream;
  auto select = [&](auto threads, auto strides) {
    constexpr int T = decltype(threads)::value, S = decltype(strides)::value;
    auto go = [&](auto kernel) { hipLaunchKernelGGL(kernel, lists, dim3(T), 0, st, c, e); };
    if (moves) int8 ? go(k_evict_select<T, S, true, true>) : go(k_evict_select<T, S, false, true>);
    else go(k_evict_select<T, S, false, false>);
  };
  // As many threads as a list has fours of slots, as far as there are: a barrier among fewer wavefronts is shorter (8 lists of 1152 slots:
  // 512 threads 7.7 us, 1024 9.4), and as few strides (8 lists of 8000 slots with four, two of them empty: 16.4 us in place of 12.5).
  if (c.capacity <= 1024) select(std::integral_constant<int, 256>(), std::integral_constant<int, 1>());
  else if (c.capacity <= 2048) select(std::integral_constant<int, 512>(), std::integral_constant<int, 1>());
  else if (c.capacity <= 4096) select(std::integral_constant<int, 1024>(), std::integral_constant<int, 1>());
  else if (c.capacity <= 8192) select(std::integral_constant<int, 1024>(), std::integral_constant<int, 2>());
  else if (!e.slices) select(std::integral_constant<int, 1024>(), std::integral_constant<int, 4>());
  else
    for (uint32_t round = 0; round <= 4; ++round) {
      auto go = [&](auto kernel) { hipLaunchKernelGGL(kernel, dim3(e.slices, c.kv_heads, c.n_seqs), dim3(kSliceThreads), 0, st, c, e, round); };
      const uint32_t strides = evict_strides(c);
      strides == 1 ? go(k_evict_slice<1>) : strides == 2 ? go(k_evict_slice<2>) : go(k_evict_slice<4>);
    }
  if (!moves) {
    const uint32_t groups = kMoveThreads / 16 * kMoveAhead;
    const uint32_t parts = std::max(1u, std::min((most + groups - 1) / groups, std::max(1u, 4096u / (c.kv_heads * c.n_seqs))));
    const dim3 grid(parts, c.kv_heads, c.n_seqs);
    if (int8) hipLaunchKernelGGL(k_evict_move<true>, grid, dim3(kMoveThreads), 0, st, c, e);
    else hipLaunchKernelGGL(k_evict_move<false>, grid, dim3(kMoveThreads), 0, st, c, e);
  }
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
