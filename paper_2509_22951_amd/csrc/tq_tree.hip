// Attention of a tree of drafted tokens over a paged cache (tq_attend_tree).
//
// All nodes of a tree and all query heads that share a key/value head are columns of one product, so that a token's key and value are read once for all of them.  A
// workgroup takes up to 12 tiles of 16 columns and a stage of tokens at a time: keys and values go from memory to LDS as they are, and a
// wavefront per column tile, or several that share out its tokens, reads them in the shape of the 16 x 16 matrix instructions:
//   logits [token][column] = K [token][dim] Q^T: lane l supplies 16 bytes of token l % 16.
//   out^T [dim][column] = V^T [dim][token] P^T: the lane that got the logits of tokens 4g..4g+3 of both 16-token blocks (g = l / 16) supplies the same tokens as its 8
//   values of the contraction, so P is already where it is needed; V is transposed on its way out of LDS.
// bf16: q (if fp32) and the weights enter as three bf16 parts each, all of fp32's 24 bits.  8 bits: q as a whole number of 24 bits, in units of a row's largest value / (127 * 2^16),
// whose three digits of 8 bits meet the keys in integer products, which are exact; values become bf16 in registers, which is exact too, and meet weights (times the
// values' scales) of three bf16 parts.  (q loses up to 2^-24 of its largest value in every dim: over 256 dims that is 2^-8 of what
// the rounding of a key to 8 bits in the one dim of that value can be.  Weights are never brought to one exponent like that: in a dim where the tokens
// of the largest ones have values of zero, the small ones are all there is.  Parts end at 2^-133, bf16's last step: a weight times a scale has all 24 bits from 2^-110 on.)
#include <algorithm>

#include "tq_cache_view.h"
#include "tq_strip_decode.h"

namespace tq {
namespace {

constexpr int kLoaders = 8, kTile = 32;   // wavefronts that load; tokens that a wavefront multiplies at a time
template <int DIM>
constexpr int kTreeWaves = DIM == 256 ? 8 : 12;   // two or three per SIMD: q and the sums take 160 or 80 registers
constexpr uint32_t kMaxGroups = 256;      // workgroups of a launch: one per compute unit
constexpr float kLog2e = 1.4426950408889634f;

struct TreeView {
  const void* q;
  uint16_t* out;
  const int32_t *seqs, *lengths, *sizes;
  const uint64_t* masks;
  float* partials;     // [workgroup][2]: [column tile][block of 16 dims][lane] four sums, then [column] maximum and total
  uint64_t q_stride, out_stride;
  float scale;         // times log2(e)
  uint32_t trees, nodes, heads, group, columns, tiles, chunks;   // columns of a key/value head; column tiles of a chunk; chunks per key/value head
  uint32_t groups;     // workgroups of the main launch
};

// What a tree's nodes attend to: slots below `length`, then slots length + j with bit j of a node's mask, below `end`.
struct Seen {
  uint32_t seq, length, end, size;
};
template <typename C, typename A>
__device__ __forceinline__ Seen seen_by(C& c, A& a, uint32_t t) {
  // (three loads at once, where a condition would put them behind each other)
  const int32_t *lengths = a.lengths, *seqs = a.seqs ? a.seqs : lengths, *sizes = a.sizes ? a.sizes : lengths;
  const int32_t of_lengths = lengths[t], of_seqs = seqs[t], of_sizes = sizes[t];
  const int32_t s = a.seqs ? of_seqs : (int32_t)t;
  const uint32_t size = a.sizes ? (uint32_t)min(max(of_sizes, 0), (int32_t)a.nodes) : a.nodes, length = (uint32_t)max(of_lengths, 0);
  if ((uint32_t)s >= c.n_seqs || size == 0) return Seen{0, 0, 0, size};
  return Seen{(uint32_t)s, min(length, c.capacity), (uint32_t)min((uint64_t)length + size, (uint64_t)c.capacity), size};
}

template <bool INT8>
__device__ __forceinline__ float value_at(const char* from, uint32_t d) {
  if constexpr (INT8) return (float)((const int8_t*)from)[d];
  else return bf16_value(((const uint16_t*)from)[d]);
}

// Four dims of a row's head, divided by the weights' total.
template <typename A>
__device__ __forceinline__ void write_out(A& a, uint32_t size, uint32_t t, uint32_t node, uint32_t head, uint32_t D, uint32_t d0, float4 sum, float total) {
  if (d0 >= D) return;
  const float inv = total == 0.f || node >= size ? 0.f : 1.f / total;
  if (node >= size) sum = make_float4(0.f, 0.f, 0.f, 0.f);
  uint16_t* to = a.out + ((uint64_t)t * a.nodes + node) * a.out_stride + head * D + d0;
  const uint32_t lo = pack_bf16(sum.x * inv, sum.y * inv), hi = pack_bf16(sum.z * inv, sum.w * inv);
  *(u32x2_any*)to = u32x2_any{lo, hi};
}

typedef int i32x4 __attribute__((ext_vector_type(4)));

template <int DIM, bool INT8>
struct Shape {
  static constexpr int kWaves = kTreeWaves<DIM>, kThreads = kWaves * 64;
  static constexpr int kSize = INT8 ? 1 : 2, kRow = DIM * kSize, kPieces = kRow / 16;   // bytes of a row, in memory and in LDS; its 16-byte pieces
  static constexpr int kTokens = 32768 / kRow, kTiles = kTokens / kTile;   // of a stage: 32 KB of keys and as much of values in LDS
  static constexpr int kSteps = DIM / (INT8 ? 64 : 32), kBlocks = DIM / 16; // contraction steps of the logits, blocks of 16 dims
  static constexpr int kOwnRows = kTokens / kLoaders, kRows = 64 / kPieces, kLoads = kOwnRows / kRows;   // rows that a wavefront loads of a stage, and at a time
  static constexpr int kOwnBlocks = kOwnRows > 16 ? kOwnRows / 16 : 1, kPerBlock = kLoads / kOwnBlocks;
  // Piece p of row r lies in place p ^ key_swizzle(r), or p ^ value_swizzle(r), so that the lanes of a read are spread over the banks.  Keys are read as 16 rows' same
  // piece.  Values are transposed as they are read: bf16 by 16 lanes from 4 rows' two neighbouring pieces, 8 bits by 32 lanes from rows 0..7 and 16..23, or 8..15 and 24..31, of one.
  static constexpr int kShift = DIM == 64 ? 2 : DIM == 128 ? 1 : 0;   // (8 bits: as many rows' bits of a number lie side by side in the 64 banks)
  static __device__ constexpr uint32_t key_swizzle(uint32_t r) { return INT8 ? (r >> kShift) & (kPieces - 1) : r & 7; }
  static __device__ constexpr uint32_t value_swizzle(uint32_t r) { return INT8 ? ((r >> kShift) & ((8 >> kShift) - 1)) | (r >> 4 & 1) << (3 - kShift) : (r & 3) << 1; }
  static constexpr int places(int period) { return kRows >= period ? 1 : period / kRows < kLoads ? period / kRows : kLoads; }
  static constexpr int kKeyPlaces = places(INT8 ? 16 : 8), kValuePlaces = places(INT8 ? 32 : 4);   // loads after which a lane's piece is the same again
  static_assert(kOwnRows % 8 == 0, "a loader begins where the places of bf16 pieces do");
  static constexpr uint32_t kPartial = kBlocks * 256 + 32;                    // floats of a column tile's partial
};

template <int TOKENS>
__device__ __forceinline__ uint32_t units_of(uint32_t end) { return max((end + TOKENS - 1) / TOKENS, 1u); }   // (a tree without tokens is written too)

// All (tree, key/value head, chunk, unit of a stage) in this order are one line, cut into equal shares, one per workgroup.  What lies in several shares leaves its parts
// in memory, and k_join_tree joins them.
//
// A workgroup that has the end of one (tree, head, chunk) and the start of another finishes one and takes up the other's queries in between, which costs about two stages.
// Where there are no more of them than workgroups, and shares need not be longer than by two units for it, every one of them is rounded up to whole shares, so that
// no workgroup has two (8 trees of 15 nodes, ragged up to 6001 tokens, 24 heads on 8: 66 us cut anywhere, 37 so).
struct Cutting {
  uint32_t share;
  bool whole;   // rounded up
};
__device__ __forceinline__ uint32_t wave_total(uint32_t v) { return (uint32_t)__builtin_amdgcn_readlane((int)wave_prefix_sum(v), 63); }
// all: units of all trees; units: of tree threadIdx.x % 64, if there are no more than 64 trees.
__device__ __forceinline__ Cutting cutting_of(uint32_t all, uint32_t units, uint32_t trees, uint32_t pairs, uint32_t groups) {
  const uint32_t even = (all * pairs + groups - 1) / groups;
  if (trees <= 64 && trees * pairs <= groups) {   // (few units in all then: below 2^31, as is their number times two)
    for (uint32_t share = even; share <= even + 2; ++share)
      if (wave_total((units + share - 1) / share) * pairs <= groups) return Cutting{share, true};
  }
  return Cutting{even, false};
}
__device__ __forceinline__ uint32_t rounded(uint32_t units, const Cutting& cut) { return cut.whole ? (units + cut.share - 1) / cut.share * cut.share : units; }

// Bound: reading the cache while there are few columns, the matrix and vector units from two or three column tiles on.  24 heads on 8, 128 dims, bf16, 16 x 16384 tokens (171 us at the
// 6.3 TB/s of a read stream): 5 nodes, one tile, 202 us, 5.3 TB/s; 16 nodes, three, 246; 20 nodes, four, 280.  1 x 131000 tokens, 64 nodes, 12 tiles: 280 us, with q in bf16 224: three parts
// of q and three of the weights are 6 products where 2 would be the least; the matrix units are busy 62 % of the time.  16 x 32700 tokens in 8 bits (176 us): 5 nodes 235, 16 nodes 369: vector
// instructions are issued 79 % of the time (weights of two f16 parts, at one exponent for all of a column's: 236, 351; what is 2^-37 of the largest then begins to be lost).
//
// Why so: 12 wavefronts, because of the 168 registers that leaves each (8 of them with everything in registers and no LDS: 80 us for the ragged batch, 368, 462; 4 with three column tiles each and
// 512 registers: 131, 420, 813; the sums' copies between the two halves of the register file cost more than the reads that were saved).  Two stages of 64 KB: what is on its way
// meanwhile, 16 MB on the card, is more than memory's latency times its rate; cut in halves with two barriers a stage it was no faster (77, 298, 470).  Loads go to LDS directly, since a
// stage in registers on its way spills.
template <int DIM, bool INT8, bool Q16>
__global__ __launch_bounds__((Shape<DIM, INT8>::kThreads)) void k_attend_tree(CacheView c, TreeView a) {
  using S = Shape<DIM, INT8>;
  constexpr int kParts = Q16 && !INT8 ? 1 : 3;
  typedef std::conditional_t<INT8, i32x4, bf16x8> key8;      // what a lane supplies of a row of keys or q
  typedef std::conditional_t<INT8, i32x4, f32x4> logits4;
  auto multiply_keys = [](key8 of_rows, key8 of_columns, logits4 sum) __attribute__((always_inline)) {
    if constexpr (INT8) return __builtin_amdgcn_mfma_i32_16x16x64_i8(of_rows, of_columns, sum, 0, 0, 0);
    else return __builtin_amdgcn_mfma_f32_16x16x32_bf16(of_rows, of_columns, sum, 0, 0, 0);
  };
  constexpr uint32_t kT = S::kTokens, kBytes = kT * S::kRow, kAll = 64, kNobody = 65;
  // Keys, then values of a stage; those of the next one are on their way into lds_1, or lds_0.
  // (Arrays of their own, so that the compiler sees that a read of one does not wait for loads into the other.)
  __shared__ __attribute__((aligned(16))) char lds_0[2 * kBytes], lds_1[2 * kBytes];
  __shared__ __attribute__((aligned(16))) uint32_t lds_kind[2][kT];     // j: of node j; kAll: of the context, kNobody
  __shared__ __attribute__((aligned(16))) float lds_scale_0[2][INT8 ? kT : 4], lds_scale_1[2][INT8 ? kT : 4];   // of keys, of values
  __shared__ float lds_max[S::kWaves * 16], lds_total[S::kWaves * 16], lds_weight[256];
  __shared__ uint64_t lds_at[256];
  __shared__ __attribute__((aligned(16))) uint32_t lds_some[2][kLoaders];   // a loader's rows of a stage: some of them are not of the context, and their kinds are told
  __shared__ uint32_t lds_odd, lds_odd_column[S::kWaves * 16];
  const uint32_t tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), D = c.head_dim;
  auto scalar = [](uint32_t v) { return (uint32_t)__builtin_amdgcn_readfirstlane((int)v); };
  // A thread's number that looks new each time: what is made of it is made where it is used, and takes no registers from the products.
  auto anew = [](uint32_t v) {
    asm volatile("" : "+v"(v));
    return v;
  };
  auto stage = [&](auto b) -> char* { return decltype(b)::value ? lds_1 : lds_0; };
  auto scales = [&](auto b, int of_values) -> float* { return decltype(b)::value ? lds_scale_1[of_values] : lds_scale_0[of_values]; };

  // The arguments, read again where they are used once in a while: the loop over the stages has no registers for all of them.
  typedef __attribute__((address_space(4))) const char constant_char;
  typedef __attribute__((address_space(4))) const CacheView constant_cache;
  typedef __attribute__((address_space(4))) const TreeView constant_tree;
  static_assert(sizeof(CacheView) % alignof(TreeView) == 0, "the kernel's arguments lie side by side");
  auto arguments = [] {
    constant_char* at = (constant_char*)__builtin_amdgcn_kernarg_segment_ptr();
    asm volatile("" : "+s"(at));
    return at;
  };
#define ARGUMENTS_ANEW                            \
  constant_char* arguments_at = arguments();      \
  constant_cache& c = *(constant_cache*)arguments_at; \
  constant_tree& a = *(constant_tree*)(arguments_at + sizeof(CacheView))

  // this workgroup's share, and the tree it begins in
  uint32_t lane_units = 0;   // of tree (t & ~63) + lane
  auto look_at = [&](uint32_t first) __attribute__((always_inline)) {
    ARGUMENTS_ANEW;
    lane_units = first + lane < a.trees ? units_of<kT>(seen_by(c, a, first + lane).end) : 0u;
    return wave_prefix_sum(lane_units);
  };
  const uint32_t pairs = c.kv_heads * a.chunks;
  uint32_t all = 0, upto = 0;
  for (uint32_t first = (a.trees - 1) & ~63u;; first -= 64) {   // (the first trees last: they stay in the lanes)
    upto = look_at(first);
    all += (uint32_t)__builtin_amdgcn_readlane((int)upto, 63);
    if (first == 0) break;
  }
  const Cutting cutting = cutting_of(all, lane_units, a.trees, pairs, gridDim.x);
  const uint32_t share = cutting.share;
  if (cutting.whole) upto = wave_prefix_sum(rounded(lane_units, cutting)), all = (uint32_t)__builtin_amdgcn_readlane((int)upto, 63);
  all *= pairs;
  uint32_t pos = blockIdx.x * share;
  const uint32_t stop = min(pos + share, all);
  if (pos >= stop) return;
  uint32_t t = 0, tree_first = 0;
  for (;;) {   // (all > pos: the tree is found)
    const uint64_t beyond = __ballot(tree_first + upto * pairs > pos);
    if (beyond) {
      const uint32_t at = (uint32_t)__builtin_ctzll(beyond);
      t += at;
      if (at) tree_first += (uint32_t)__builtin_amdgcn_readlane((int)upto, at - 1) * pairs;
      break;
    }
    tree_first += (uint32_t)__builtin_amdgcn_readlane((int)upto, 63) * pairs;
    t += 64;
    if (t >= a.trees) return;   // (lengths that change under the call)
    upto = look_at(t);
  }

  struct Segment {   // the part of a (tree, key/value head, chunk) that lies in this share
    Seen of;
    uint32_t t, kv, first_column, unit, n_units, first, units;   // first: where the whole of it begins on the line, units long
  };
  auto next_segment = [&]() __attribute__((always_inline)) {
    ARGUMENTS_ANEW;
    Segment s;
    s.t = t, s.of = seen_by(c, a, t);
    s.of.seq = scalar(s.of.seq), s.of.length = scalar(s.of.length), s.of.end = scalar(s.of.end), s.of.size = scalar(s.of.size);
    s.units = (uint32_t)__builtin_amdgcn_readlane((int)lane_units, t & 63);
    const uint32_t on_line = rounded(s.units, cutting), pair = (pos - tree_first) / on_line;
    s.first = tree_first + pair * on_line;
    s.kv = pair / a.chunks, s.first_column = pair % a.chunks * a.tiles * 16;
    s.unit = pos - s.first, s.n_units = min(s.units - s.unit, stop - pos);
    pos += min(on_line - s.unit, stop - pos);
    if (pos == tree_first + on_line * (c.kv_heads * a.chunks)) {
      tree_first = pos, ++t;
      if ((t & 63) == 0 && pos < stop) look_at(t);
    }
    return s;
  };

  // ---- from memory to LDS ----
  // A loader takes kOwnRows rows of a stage; 16 tokens lie in one page.  The pages are looked up ahead of the barrier in front of the loads.
  struct Place {   // a stage: of a segment, or none
    Segment s;
    uint32_t unit;
    bool there;
  };
  auto after = [&](const Place& p) __attribute__((always_inline)) {
    Place n = p;
    ++n.unit;
    if (p.there && n.unit == p.s.n_units) {
      n.unit = 0, n.there = pos < stop;
      if (n.there) n.s = next_segment();
    }
    return n;
  };
  const bool loads = wave < kLoaders;
  const uint32_t slot_bytes = S::kSize * (uint32_t)c.slot_stride;
  const uint64_t page_bytes = S::kSize * c.page_stride;
  typedef __attribute__((address_space(1))) const uint32_t global_cu32;
  typedef __attribute__((address_space(3))) uint32_t lds_mu32;
  uint32_t ids[S::kOwnBlocks];
  auto look_up = [&](const Place& p) __attribute__((always_inline)) {
    constant_i32* table = (constant_i32*)(c.tables + (uint64_t)p.s.of.seq * c.table_stride);
    const uint32_t newest = max(p.s.of.end, 1u) - 1, slot = (p.s.unit + p.unit) * kT + wave * S::kOwnRows;
#pragma unroll
    for (int b = 0; b < S::kOwnBlocks; ++b) ids[b] = (uint32_t)table[min(slot + 16 * b, newest) >> c.page_shift];
  };
  auto fetch = [&](const Place& p, auto buffer) __attribute__((always_inline)) {
    constexpr int kBuffer = decltype(buffer)::value;
    if (!loads) return;
    const uint32_t lane = anew(tid) & 63;
    // The piece of a row that a lane loads with the i-th group of rows (of dims that a head does not have: its first one, against zeros of q).
    const uint32_t place = lane % S::kPieces, row_of_lane = lane / S::kPieces;
    auto piece_at = [&](uint32_t swizzle) __attribute__((always_inline)) {
      const uint32_t of = (place ^ swizzle) * 16;
      return of < S::kSize * D ? of : 0;
    };
    uint32_t key_from[S::kKeyPlaces], value_from[S::kValuePlaces];
#pragma unroll
    for (int i = 0; i < S::kKeyPlaces; ++i) key_from[i] = piece_at(S::key_swizzle(wave * S::kOwnRows + i * S::kRows + row_of_lane));
#pragma unroll
    for (int i = 0; i < S::kValuePlaces; ++i) value_from[i] = piece_at(S::value_swizzle(wave * S::kOwnRows + i * S::kRows + row_of_lane));
    const uint32_t first = (p.s.unit + p.unit) * kT + wave * S::kOwnRows, page_mask = (1u << c.page_shift) - 1;
    char* to = stage(buffer) + wave * S::kOwnRows * S::kPieces * 16;
    bool some = first + S::kOwnRows > p.s.of.length;
    uint32_t limit_of_lane = 0;   // of the 16 tokens that token first + lane is one of: how many are there
    uint64_t mark_of_lane = 0;
#pragma unroll
    for (int b = 0; b < S::kOwnBlocks; ++b) {
      // In place of rows that are not there the block's first one comes again, so that beside a weight of zero lies what is attended to anyway; in place of a page that is not there, page 0: if that
      // holds something that is not finite, the tokens are taken again.
      const uint32_t newest = max(p.s.of.end, 1u) - 1, slot = first + 16 * b, from = min(slot, newest & ~(uint32_t)(S::kOwnRows < 16 ? S::kOwnRows - 1 : 15)), id = scalar(ids[b]);
      const uint32_t page = id < c.n_pages ? id : 0, in_page = from & page_mask, limit = id < c.n_pages && slot < p.s.of.end ? min(p.s.of.end - slot, 16u) : 0u;
      some |= id >= c.n_pages;
      const uint64_t at = page * page_bytes + (uint64_t)(p.s.kv * c.head_stride) * S::kSize + (uint64_t)in_page * slot_bytes;
#pragma unroll
      for (int j = 0; j < S::kPerBlock; ++j) {
        const int i = b * S::kPerBlock + j;
        const uint32_t row = j * S::kRows + row_of_lane, row_at = row < limit ? row * slot_bytes : 0;
        __builtin_amdgcn_global_load_lds((global_cu32*)(c.k + at + (row_at + key_from[i % S::kKeyPlaces])), (lds_mu32*)(to + i * 1024), 16, 0, 0);
        __builtin_amdgcn_global_load_lds((global_cu32*)(c.v + at + (row_at + value_from[i % S::kValuePlaces])), (lds_mu32*)(to + i * 1024 + kT * S::kPieces * 16), 16, 0, 0);
      }
      if (S::kOwnBlocks == 1 || (int)(lane / 16) == b) {
        limit_of_lane = limit;
        mark_of_lane = (((uint64_t)page * c.kv_heads + p.s.kv) << c.page_shift) + in_page + (lane % 16 < limit ? lane % 16 : 0);
      }
    }
    if constexpr (INT8) {
      if (lane < S::kOwnRows) {   // (the wavefront's rows' scales, a lane each)
        __builtin_amdgcn_global_load_lds((global_cu32*)(c.k_scale + mark_of_lane), (lds_mu32*)&scales(buffer, 0)[wave * S::kOwnRows], 4, 0, 0);
        __builtin_amdgcn_global_load_lds((global_cu32*)(c.v_scale + mark_of_lane), (lds_mu32*)&scales(buffer, 1)[wave * S::kOwnRows], 4, 0, 0);
      }
    }
    if (lane == 0) lds_some[kBuffer][wave] = some;
    if (__builtin_expect(some, 0)) {
      const uint32_t slot = first + lane;
      if (lane < S::kOwnRows) lds_kind[kBuffer][wave * S::kOwnRows + lane] = lane % 16 >= limit_of_lane ? kNobody : slot < p.s.of.length ? kAll : slot - p.s.of.length;
    }
  };

  // ---- a column tile per wavefront, or for several, that share out the tiles of tokens ----
  uint32_t over = 1;
  while (over < (uint32_t)S::kTiles && 2 * over * a.tiles <= (uint32_t)S::kWaves) over *= 2;
  const uint32_t of_tile = wave % a.tiles, of_tokens = wave / a.tiles;
  const bool works = of_tokens < over;
  key8 q[kParts][S::kSteps];   // 8 bits: three digits of a whole number, in units of the largest value / 127.0, that logits are multiplied by
  float logit_scale = a.scale;
  __shared__ uint64_t lds_mask[S::kWaves * 16];
  auto column_of = [&](const Segment& s, uint32_t column, uint32_t* node) {   // -> query head
    constant_tree& a = *(constant_tree*)(arguments() + sizeof(CacheView));
    *node = column / a.group;
    return s.kv * a.group + column % a.group;
  };
  auto load_q = [&](const Segment& s) __attribute__((always_inline)) {
    ARGUMENTS_ANEW;
    const uint32_t D = c.head_dim;
    const uint32_t lane = anew(threadIdx.x) & 63, g = lane / 16, n = lane % 16;
    const uint32_t column = s.first_column + of_tile * 16 + n;
    const bool has = works && column < a.columns;
    uint32_t node, head = column_of(s, has ? column : 0, &node);
    const uint64_t row = (uint64_t)s.t * a.nodes + node;
    if (of_tokens == 0 && g == 0) lds_mask[of_tile * 16 + n] = has && node < s.of.size ? a.masks[row] : 0;   // (a barrier ahead of the next stage's weights)
    auto read = [&](uint32_t d, float* v) __attribute__((always_inline)) {   // eight
      const bool own = has && d < D;
      const uint64_t at = row * a.q_stride + head * D + (own ? d : 0);
      if constexpr (Q16) {
        const u16x4_any lo = *(const u16x4_any*)((const uint16_t*)a.q + at), hi = *(const u16x4_any*)((const uint16_t*)a.q + at + 4);
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = own ? bf16_value(j < 4 ? lo[j % 4] : hi[j % 4]) : 0.f;
      } else {
        const f32x4_any lo = *(const f32x4_any*)((const float*)a.q + at), hi = *(const f32x4_any*)((const float*)a.q + at + 4);
#pragma unroll
        for (int j = 0; j < 8; ++j) v[j] = own ? (j < 4 ? lo[j % 4] : hi[j % 4]) : 0.f;
      }
    };
    if constexpr (INT8) {
      float v[S::kSteps][16], most = 0.f, odd = 0.f;
#pragma unroll
      for (int i = 0; i < S::kSteps; ++i) {
        read(i * 64 + 16 * g, &v[i][0]), read(i * 64 + 16 * g + 8, &v[i][8]);
#pragma unroll
        for (int j = 0; j < 16; ++j) most = fmaxf(most, fabsf(v[i][j])), odd = fmaf(v[i][j], 0.f, odd);
      }
      most = fmaxf(most, __shfl_xor(most, 16)), most = fmaxf(most, __shfl_xor(most, 32));
      odd += __shfl_xor(odd, 16), odd += __shfl_xor(odd, 32);
      const float up = fminf(127.f * 65536.f / most, 0x1p126f);   // (of nothing but zeros: zeros)
      logit_scale = a.scale / up + odd;                    // (a query that is not finite: NaN, so that the tokens are taken again)
#pragma unroll
      for (int i = 0; i < S::kSteps; ++i)
#pragma unroll
        for (int w = 0; w < 4; ++w) {
          uint32_t digits[3] = {0, 0, 0};
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            const int32_t whole = odd == 0.f ? (int32_t)rintf(v[i][4 * w + j] * up) : 0;
            const uint32_t u = (uint32_t)(whole + 0x8080);   // digits of -128..127: those of 0..255, less 128, and the upper one as it is
            digits[0] |= (u >> 16 & 255) << (8 * j), digits[1] |= ((u >> 8 & 255) ^ 128) << (8 * j), digits[2] |= ((u & 255) ^ 128) << (8 * j);
          }
#pragma unroll
          for (int k = 0; k < 3; ++k) q[k][i][w] = (int)digits[k];
        }
    } else {
#pragma unroll
      for (int i = 0; i < S::kSteps; ++i) {
        float v[8];
        read(i * 32 + 8 * g, v);
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          float left = v[j];
#pragma unroll
          for (int k = 0; k < kParts; ++k) {
            q[k][i][j] = (__bf16)left;
            left -= (float)q[k][i][j];
          }
        }
      }
    }
  };

  f32x4 o[S::kBlocks];
  float top = -INFINITY, total = 0.f;
  constexpr float kMostScale = 0x1p80f;   // of an 8-bit key (sums of levels and digits are below 2^39)
  auto take_tile = [&](auto buffer, uint32_t tile, bool some) __attribute__((always_inline)) {
    constexpr int kBuffer = decltype(buffer)::value;
    const char* keys = stage(buffer) + tile * kTile * S::kRow;
    const char* values = keys + kBytes;
    const uint32_t g = lane / 16, n = lane % 16;
    const uint32_t key_at = n * S::kRow, key_place = g ^ S::key_swizzle(n);
    logits4 l[2] = {{0, 0, 0, 0}, {0, 0, 0, 0}}, less[2] = {{0, 0, 0, 0}, {0, 0, 0, 0}};
    constexpr int kKeySteps = S::kSteps < 2 ? S::kSteps : 2;   // of which all keys are asked for at once
    auto key_of = [&](int i, int b) __attribute__((always_inline)) { return *(const key8*)(keys + b * 16 * S::kRow + key_at + ((key_place ^ (4 * i)) * 16)); };
    if constexpr (INT8) {   // the sums of the lowest digits, and 256 times the upper ones' and the middle ones'
      key8 key[S::kSteps][2];
#pragma unroll
      for (int i = 0; i < S::kSteps; ++i)
#pragma unroll
        for (int b = 0; b < 2; ++b) key[i][b] = key_of(i, b);
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int part = 0; part < 3; ++part) {
#pragma unroll
        for (int i = 0; i < S::kSteps; ++i)
#pragma unroll
          for (int b = 0; b < 2; ++b) (part == 1 ? less : l)[b] = multiply_keys(key[i][b], q[part == 0 ? 0 : 3 - part][i], (part == 1 ? less : l)[b]);
        if (part == 1)
#pragma unroll
          for (int b = 0; b < 2; ++b) l[b] <<= 8;   // (below 2^22 of 256 dims)
      }
    } else {
#pragma unroll
      for (int first = 0; first < S::kSteps; first += kKeySteps) {
        key8 key[kKeySteps][2];
#pragma unroll
        for (int i = 0; i < kKeySteps; ++i)
#pragma unroll
          for (int b = 0; b < 2; ++b) key[i][b] = key_of(first + i, b);
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int i = 0; i < kKeySteps; ++i)
#pragma unroll
          for (int part = 0; part < kParts; ++part)
#pragma unroll
            for (int b = 0; b < 2; ++b) l[b] = multiply_keys(key[i][b], q[part][first + i], l[b]);
      }
    }
    // The values are asked for ahead of what the weights take.
    typedef short s16x4 __attribute__((ext_vector_type(4)));
    typedef __attribute__((address_space(3))) s16x4 lds_s16x4;
    typedef int i32x2 __attribute__((ext_vector_type(2)));
    typedef __attribute__((address_space(3))) i32x2 lds_i32x2;
    const uint32_t value_row = INT8 ? 4 * g + n / 2 % 4 + n / 8 * 16 : 4 * g + n / 4;
    const uint32_t value_at0 = value_row * S::kRow + S::value_swizzle(value_row) * 16 + (INT8 ? n % 2 : n % 4) * 8;
    std::conditional_t<INT8, i32x2, bf16x8> asked[S::kBlocks];
    auto ask = [&](int b) __attribute__((always_inline)) {
      const char* from = values + (value_at0 ^ (b * 16 * S::kSize));
      if constexpr (INT8) {
        asked[b] = __builtin_amdgcn_ds_read_tr8_b64_v2i32((lds_i32x2*)from);
      } else {
        const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)from), hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(from + 16 * S::kRow));
        asked[b] = __builtin_bit_cast(bf16x8, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
      }
    };
    auto value_of = [&](int b) __attribute__((always_inline)) {
      if constexpr (INT8) return i8x8_to_bf16x8(make_uint2((uint32_t)asked[b][0], (uint32_t)asked[b][1]));
      else return asked[b];
    };
    constexpr int kEarly = INT8 ? 4 : 2;
#pragma unroll
    for (int b = 0; b < kEarly; ++b) ask(b);
    float p[8], most_scale = 0.f;   // logits, without `logit_scale`
    float4 vs[2];
#pragma unroll
    for (int b = 0; b < 2; ++b) {
      if constexpr (INT8) {
        const float4 ks = *(const float4*)&scales(buffer, 0)[tile * kTile + 16 * b + 4 * g];
        vs[b] = *(const float4*)&scales(buffer, 1)[tile * kTile + 16 * b + 4 * g];
#pragma unroll
        for (int j = 0; j < 4; ++j) p[4 * b + j] = fmaf((float)l[b][j], 256.f, (float)less[b][j]) * (&ks.x)[j], most_scale = fmaxf(most_scale, fabsf((&ks.x)[j]));
      } else {
#pragma unroll
        for (int j = 0; j < 4; ++j) p[4 * b + j] = l[b][j];
      }
    }
    if (some) {
      const uint64_t mask = lds_mask[of_tile * 16 + n];
#pragma unroll
      for (int b = 0; b < 2; ++b) {
        const uint32_t row = tile * kTile + 16 * b + 4 * g;
        uint4 kind = *(const uint4*)&lds_kind[kBuffer][row];
        if (!lds_some[kBuffer][row / S::kOwnRows]) kind = make_uint4(kAll, kAll, kAll, kAll);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const uint32_t k = (&kind.x)[j], word = k & 32 ? (uint32_t)(mask >> 32) : (uint32_t)mask;
          const uint32_t sees = (k == kAll ? 1u : 0u) | (k < kAll ? word >> (k & 31) & 1u : 0u);
          p[4 * b + j] = sees ? p[4 * b + j] : -INFINITY;
          if constexpr (INT8) (&vs[b].x)[j] = sees ? (&vs[b].x)[j] : 0.f;
        }
      }
    }
    float m = p[0];
#pragma unroll
    for (int i = 1; i < 8; ++i) m = fmaxf(m, p[i]);
    const float scale = INT8 ? logit_scale : a.scale;
    m *= scale;
    // The weights' reference follows the maximum when that has grown by more than 8 (2^8 is far from any bound of fp32).
    if (__any(m > top + 8.f || (INT8 && !(most_scale < kMostScale)))) {
      // (an infinite scale of a key makes NaN of a level of zero, and one this large could make an infinity of a logit that is none: the tokens are taken again)
      if (INT8 && !(most_scale < kMostScale)) total = __builtin_nanf("");
      m = fmaxf(m, top);
      m = fmaxf(m, __shfl_xor(m, 16));
      m = fmaxf(m, __shfl_xor(m, 32));
      const float shrink = __builtin_amdgcn_exp2f(top - (m == -INFINITY ? 0.f : m));
      top = m, total *= shrink;
#pragma unroll
      for (int b = 0; b < S::kBlocks; ++b) o[b] *= shrink;
    }
    const float base = top == -INFINITY ? 0.f : top;
    uint32_t part[3][4];
#pragma unroll
    for (int i = 0; i < 8; i += 2) {
      float w[2];
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        w[j] = __builtin_amdgcn_exp2f(fmaf(p[i + j], scale, -base));
        total += w[j];
        if constexpr (INT8) w[j] *= (&vs[i / 4].x)[i % 4 + j];
      }
#pragma unroll
      for (int k = 0; k < 3; ++k) {   // the upper 8 bits of the mantissas, the next 8, the last 8
        const uint32_t lo = __float_as_uint(w[0]), hi = __float_as_uint(w[1]);
        part[k][i / 2] = __builtin_amdgcn_perm(hi, lo, 0x07060302u);
        w[0] -= __uint_as_float(lo & 0xFFFF0000u), w[1] -= __uint_as_float(hi & 0xFFFF0000u);
      }
    }
#pragma unroll
    for (int first = 0; first < S::kBlocks; first += kEarly) {
      if (first)
#pragma unroll
        for (int b = 0; b < kEarly; ++b) ask(first + b);
      bf16x8 value[kEarly];
#pragma unroll
      for (int b = 0; b < kEarly; ++b) value[b] = value_of(first + b);
#pragma unroll
      for (int k = 0; k < 3; ++k)
#pragma unroll
        for (int b = 0; b < kEarly; ++b)
          o[first + b] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(value[b], __builtin_bit_cast(bf16x8, make_uint4(part[k][0], part[k][1], part[k][2], part[k][3])), o[first + b], 0, 0, 0);
    }
  };

  // A column's tokens of a segment once more, a product per value as the formula has them, so that infinities give what they give there: only for what is not finite, and
  // slow.  256 threads take a token each, then all of them a dim of every so-manieth token; the sums go to `sums`, LDS of 32 KB at least.
  auto take_again = [&](const Segment& s, uint32_t col, float* sums) __attribute__((always_inline)) {
    constexpr uint32_t kN = 256, kTeams = S::kThreads / DIM;
    constexpr uint64_t kNothing = 1ull << 63;
    ARGUMENTS_ANEW;
    const uint32_t D = c.head_dim;
    const uint32_t tid = anew(threadIdx.x), team = tid / DIM, dim = tid % DIM;
    const uint32_t begin = s.unit * kT, end = min(s.of.end, (s.unit + s.n_units) * kT);
    uint32_t node, head = column_of(s, s.first_column + col, &node);
    const uint64_t row = (uint64_t)s.t * a.nodes + node, sees = node < s.of.size ? a.masks[row] : 0;
    const uint64_t q_at = row * a.q_stride + head * D;
    float *lds_q = sums, *slots = sums + DIM, *of_teams = sums + 2 * DIM;
    if (tid < D) lds_q[tid] = (Q16 ? bf16_value(((const uint16_t*)a.q)[q_at + tid]) : ((const float*)a.q)[q_at + tid]) * a.scale;
    __syncthreads();
    // over the 256 tokens, in the same order every time
    auto over_all = [&](float v, auto join) __attribute__((always_inline)) {
#pragma unroll
      for (int d = 1; d < 64; d *= 2) v = join(v, __shfl_xor(v, d));
      __syncthreads();
      if (tid < kN && tid % 64 == 0) slots[tid / 64] = v;
      __syncthreads();
      return join(join(slots[0], slots[1]), join(slots[2], slots[3]));
    };
    float m = -INFINITY, sum_p = 0.f, sum = 0.f;
    for (uint32_t first = begin; first < end && node < s.of.size; first += kN) {
      const uint32_t slot = first + tid;
      uint32_t page = c.n_pages;
      if (tid < kN && slot < end && (slot < s.of.length || sees >> (slot - s.of.length) & 1)) page = (uint32_t)c.tables[(uint64_t)s.of.seq * c.table_stride + (slot >> c.page_shift)];
      const bool there = page < c.n_pages;
      const uint32_t in_page = slot & ((1u << c.page_shift) - 1);
      const uint64_t at = S::kSize * ((uint64_t)(there ? page : 0) * c.page_stride + s.kv * c.head_stride + in_page * c.slot_stride);
      const uint64_t mark = (((uint64_t)(there ? page : 0) * c.kv_heads + s.kv) << c.page_shift) + in_page;
      float l = -INFINITY;
      if (there) {
        const float scale = INT8 ? c.k_scale[mark] : 1.f;
        const bool after = fabsf(scale) < INFINITY;   // (an infinite scale makes NaN of a level of zero)
        l = 0.f;
        for (uint32_t x = 0; x < D; x += 16 / S::kSize) {
          const uint4 piece = *(const uint4*)(c.k + at + x * S::kSize);
#pragma unroll
          for (int j = 0; j < 16 / S::kSize; ++j) {
            const float value = value_at<INT8>((const char*)&piece, j);
            l = fmaf(lds_q[x + j], after ? value : value * scale, l);
          }
        }
        if (after) l *= scale;
      }
      const float most = fmaxf(m, over_all(l, [](float x, float y) { return fmaxf(x, y); })), base = most == -INFINITY ? 0.f : most, shrink = __builtin_amdgcn_exp2f(m - base);
      const float p = there ? __builtin_amdgcn_exp2f(l - base) : 0.f;
      m = most, sum *= shrink;
      sum_p = fmaf(sum_p, shrink, over_all(p, [](float x, float y) { return x + y; }));
      if (tid < kN) lds_weight[tid] = there && INT8 ? p * c.v_scale[mark] : p, lds_at[tid] = there ? at : at | kNothing;
      __syncthreads();
      if (dim < D) {
#pragma unroll 8
        for (uint32_t i = team; i < kN; i += kTeams) {
          const uint64_t from = lds_at[i];
          const float value = value_at<INT8>(c.v + (from & ~kNothing), dim);
          sum = from & kNothing ? sum : fmaf(lds_weight[i], value, sum);
        }
      }
    }
    of_teams[tid] = sum;   // (kTeams * DIM are all threads)
    __syncthreads();
    if (tid < DIM) {
      sum = of_teams[tid];
#pragma unroll
      for (uint32_t i = 1; i < kTeams; ++i) sum += of_teams[i * DIM + tid];
      sums[tid] = sum;   // (everyone is done with q)
    }
    if (tid == 0) lds_max[col] = m, lds_total[col] = sum_p;
    __syncthreads();
  };

  // The end of a segment: the wavefronts of a column tile join, in LDS that its last stage took, and the first of them writes.
  auto finish = [&](const Segment& s, float* sums) __attribute__((always_inline)) {
    ARGUMENTS_ANEW;
    const uint32_t D = c.head_dim;
    const uint32_t tid = anew(threadIdx.x), lane = tid & 63, g = lane / 16, n = lane % 16;
    total += __shfl_xor(total, 16);
    total += __shfl_xor(total, 32);
    if (tid == 0) lds_odd = 0;
    if (tid < S::kWaves * 16) lds_odd_column[tid] = 0;
    __syncthreads();   // everyone is done with the stage
    for (uint32_t half = over / 2; half; half /= 2) {
      if (works && of_tokens >= half && of_tokens < 2 * half) {
        const uint32_t at = (of_tokens - half) * a.tiles + of_tile;
#pragma unroll
        for (int b = 0; b < S::kBlocks; ++b) *(f32x4*)&sums[((at * S::kBlocks + b) * 64 + lane) * 4] = o[b];
        if (g == 0) lds_max[at * 16 + n] = top, lds_total[at * 16 + n] = total;
      }
      __syncthreads();
      if (of_tokens < half) {
        const uint32_t at = of_tokens * a.tiles + of_tile;
        const float other = lds_max[at * 16 + n], m = fmaxf(top, other), base = m == -INFINITY ? 0.f : m;
        const float e = __builtin_amdgcn_exp2f(top - base), f = __builtin_amdgcn_exp2f(other - base);
        total = fmaf(f, lds_total[at * 16 + n], total * e), top = m;
#pragma unroll
        for (int b = 0; b < S::kBlocks; ++b) {
          const f32x4 v = *(const f32x4*)&sums[((at * S::kBlocks + b) * 64 + lane) * 4];
#pragma unroll
          for (int j = 0; j < 4; ++j) o[b][j] = fmaf(f, v[j], o[b][j] * e);
        }
      }
      __syncthreads();
    }
    const uint32_t column = s.first_column + of_tile * 16 + n;
    const bool mine = of_tokens == 0 && column < a.columns;
    float odd = total * 0.f;   // a query, key or value that is not finite leaves no total or sum finite that it went into
#pragma unroll
    for (int b = 0; b < S::kBlocks; ++b)
#pragma unroll
      for (int j = 0; j < 4; ++j) odd = fmaf(o[b][j], 0.f, odd);
    if (mine && !(odd == 0.f)) lds_odd = lds_odd_column[of_tile * 16 + n] = 1;
    __syncthreads();
    if (__builtin_expect(lds_odd, 0)) {
#pragma unroll 1
      for (uint32_t col = 0; col < a.tiles * 16; ++col) {
        if (!lds_odd_column[col]) continue;
        take_again(s, col, sums);
        if (of_tokens == 0 && of_tile * 16 + n == col) {
          top = lds_max[col], total = lds_total[col];
#pragma unroll
          for (int b = 0; b < S::kBlocks; ++b) o[b] = *(const f32x4*)&sums[16 * b + 4 * g];
        }
        __syncthreads();
      }
    }
    if (of_tokens != 0) return;
    if (s.n_units == s.units) {
      if (!mine) return;
      uint32_t node, head = column_of(s, column, &node);
#pragma unroll
      for (int b = 0; b < S::kBlocks; ++b) write_out(a, s.of.size, s.t, node, head, D, 16 * b + 4 * g, make_float4(o[b][0], o[b][1], o[b][2], o[b][3]), total);
    } else {
      float* to = a.partials + (uint64_t)(2 * blockIdx.x + (blockIdx.x * share >= s.first ? 0 : 1)) * (a.tiles * S::kPartial) + of_tile * S::kPartial;
#pragma unroll
      for (int b = 0; b < S::kBlocks; ++b) *(f32x4*)&to[(b * 64 + lane) * 4] = o[b];
      if (g == 0) *(float2*)&to[S::kBlocks * 256 + 2 * n] = make_float2(top, total);
    }
  };

  typedef std::integral_constant<int, 0> First;
  typedef std::integral_constant<int, 1> Second;
  Place now{next_segment(), 0, true};
  look_up(now);
  fetch(now, First());
  Place next = after(now);
  look_up(next);
  load_q(now.s);
  auto take = [&](auto buffer, auto other) __attribute__((always_inline)) {
    __builtin_amdgcn_s_waitcnt(0x0F70);   // vmcnt(0): this stage's loads
    __syncthreads();
    if (next.there) fetch(next, other);
    if (works) {
      constexpr int kBuffer = decltype(buffer)::value;
      const uint4 x = *(const uint4*)&lds_some[kBuffer][0], y = *(const uint4*)&lds_some[kBuffer][4];
      const bool some = scalar(x.x | x.y | x.z | x.w | y.x | y.y | y.z | y.w) != 0;
      for (uint32_t tile = of_tokens; tile < (uint32_t)S::kTiles; tile += over) take_tile(buffer, tile, some);
    }
  };
  auto step = [&](auto buffer, auto other) __attribute__((always_inline)) {
    if (now.unit == 0) {
      top = -INFINITY, total = 0.f;
#pragma unroll
      for (int b = 0; b < S::kBlocks; ++b) o[b] = f32x4{0.f, 0.f, 0.f, 0.f};
    }
    take(buffer, other);
    if (now.unit + 1 == now.s.n_units) {
      finish(now.s, (float*)stage(buffer));
      if (!next.there) return true;
      load_q(next.s);
    }
    now = next, next = after(next);
    look_up(next);
    return false;
  };
  // (Two steps a turn, so that the compiler knows of each read which of the stages on their way it could meet, and waits for none.)
  while (!step(First(), Second()) && !step(Second(), First())) {}
}

#undef ARGUMENTS_ANEW

// The parts of what lies in more than one share, joined in the order of the line: a wavefront per 16 columns and 16 dims.  A launch of its own, which a sequence that can not be longer than a stage
// does without: the last workgroup to arrive would join alone what all of them share here.  Bound: its launch and three waits behind each other, 5.1 us (least: 4.8) for the ragged batch of 8 x 15 nodes; the parts, 25 MB written and
// read, 11.4 us (9.6) for 64 nodes over 131000 tokens.
template <int DIM, bool INT8>
__global__ __launch_bounds__(256) void k_join_tree(CacheView c, TreeView a) {
  using S = Shape<DIM, INT8>;
  const uint32_t lane = threadIdx.x & 63, wave = threadIdx.x >> 6, g = lane / 16, n = lane % 16, pairs = c.kv_heads * a.chunks, D = c.head_dim, blocks = (D + 15) / 16;
  const uint32_t per_tree = pairs * a.tiles * blocks, pieces = a.trees * per_tree;   // (below 2^31)
  for (uint32_t of = blockIdx.x * 4 + wave; of < pieces; of += gridDim.x * 4) {
    const uint32_t t = of / per_tree, rest = of % per_tree, b = rest % blocks, tile = rest / blocks % a.tiles, pair = rest / blocks / a.tiles;
    uint32_t all = 0, before = 0, units = 0;
    for (uint32_t first = 0; first < a.trees; first += 64) {
      units = first + lane < a.trees ? units_of<S::kTokens>(seen_by(c, a, first + lane).end) : 0u;
      all += wave_total(units), before += wave_total(first + lane < t ? units : 0u);
    }
    const Cutting cutting = cutting_of(all, units, a.trees, pairs, a.groups);
    if (cutting.whole) before = wave_total(lane < t ? rounded(units, cutting) : 0u);
    const Seen seen = seen_by(c, a, t);
    units = units_of<S::kTokens>(seen.end);
    const uint32_t share = cutting.share, first = before * pairs + pair * rounded(units, cutting);
    const uint32_t group0 = first / share, group1 = (first + units - 1) / share;
    if (group0 == group1) continue;
    auto part_of = [&](uint32_t group) { return a.partials + ((uint64_t)(2 * group + (group * share >= first ? 0 : 1)) * a.tiles + tile) * S::kPartial; };
    float m = -INFINITY, sum_p = 0.f;
    float4 sum = make_float4(0.f, 0.f, 0.f, 0.f);
    constexpr uint32_t kAhead = 8;   // (four, sixteen: ragged batch 5.4, 6.4 us at the least in place of 4.9; 64 nodes over 131000 tokens 14.2, 11.0 in place of 9.8)
    for (uint32_t group = group0; group <= group1; group += kAhead) {
      float4 v[kAhead];
      float2 st[kAhead];
#pragma unroll
      for (uint32_t i = 0; i < kAhead; ++i) {
        const float* from = part_of(min(group + i, group1));
        v[i] = *(const float4*)&from[(b * 64 + lane) * 4], st[i] = *(const float2*)&from[S::kBlocks * 256 + 2 * n];
      }
#pragma unroll
      for (uint32_t i = 0; i < kAhead; ++i) {
        if (group + i > group1) continue;
        const float to = fmaxf(m, st[i].x), base = to == -INFINITY ? 0.f : to, e = __builtin_amdgcn_exp2f(m - base), f = __builtin_amdgcn_exp2f(st[i].x - base);
        m = to, sum_p = fmaf(f, st[i].y, sum_p * e);
        sum.x = fmaf(f, v[i].x, sum.x * e), sum.y = fmaf(f, v[i].y, sum.y * e), sum.z = fmaf(f, v[i].z, sum.z * e), sum.w = fmaf(f, v[i].w, sum.w * e);
      }
    }
    const uint32_t column = (pair % a.chunks * a.tiles + tile) * 16 + n;
    if (column < a.columns) write_out(a, seen.size, t, column / a.group, pair / a.chunks * a.group + column % a.group, D, 16 * b + 4 * g, sum, sum_p);
  }
}

struct Layout {
  uint32_t columns, tiles, chunks, units, groups;   // as in TreeView; units: of a full sequence
  uint64_t bytes;
};

int check_tree(const std::string& who, const tq_cache* cache, const tq_tree_args* a, CacheView* c, Layout* l) {
  if (int rc = view_cache(who, cache, c)) return rc;
  if (!a) return refuse(TQ_E_INVALID_ARG, who + ": null argument");
  if (a->q_type != TQ_FP32 && a->q_type != TQ_BF16) return refuse(TQ_E_UNSUPPORTED, who + ": q is TQ_FP32 or TQ_BF16");
  if (a->heads == 0 || a->heads > 65535 || a->heads % c->kv_heads) return refuse(TQ_E_INVALID_ARG, who + ": heads must be a multiple of kv_heads up to 65535");
  if (a->nodes == 0 || a->nodes > TQ_MAX_NODES) return refuse(TQ_E_UNSUPPORTED, who + ": a tree has 1..64 nodes");
  if (a->trees > 65535) return refuse(TQ_E_UNSUPPORTED, who + ": more than 65535 trees");
  if (!a->seqs && a->trees > c->n_seqs) return refuse(TQ_E_INVALID_ARG, who + ": more trees than sequences, and no seqs");
  if (!(a->scale > 0.f) || !(a->scale < INFINITY)) return refuse(TQ_E_INVALID_ARG, who + ": scale must be positive");
  const uint32_t group = a->heads / c->kv_heads, dim = c->head_dim <= 64 ? 64 : c->head_dim <= 128 ? 128 : 256, tokens = (cache->type == TQ_INT8 ? 32768 : 16384) / dim;   // of a stage
  l->columns = a->nodes * group;
  const uint32_t all_tiles = (l->columns + 15) / 16, most = dim == 256 ? kTreeWaves<256> : kTreeWaves<64>;
  l->chunks = (all_tiles + most - 1) / most;
  l->tiles = (all_tiles + l->chunks - 1) / l->chunks;
  l->units = (c->capacity + tokens - 1) / tokens;
  const uint64_t line = (uint64_t)a->trees * c->kv_heads * l->chunks * l->units;   // if all sequences are full
  if (line >= (1u << 31) - kMaxGroups || (uint64_t)a->trees * c->kv_heads * l->chunks * l->tiles * 16 >= (1u << 31) - 65536) return refuse(TQ_E_UNSUPPORTED, who + ": trees * heads * capacity is beyond what one call takes");
  l->groups = (uint32_t)std::min<uint64_t>(kMaxGroups, std::max<uint64_t>(1, line));
  l->bytes = l->units > 1 ? (uint64_t)l->groups * 2 * l->tiles * 16 * (dim + 2) * 4 : 16;
  return TQ_OK;
}

int attend_tree(const tq_cache* cache, const tq_tree_args* a, void* stream) {
  const std::string who = "tq_attend_tree";
  CacheView c;
  Layout l{};
  if (int rc = check_tree(who, cache, a, &c, &l)) return rc;
  if (a->trees == 0) return TQ_OK;
  if (!a->q || !a->out || !a->lengths || !a->masks || !a->workspace) return refuse(TQ_E_INVALID_ARG, who + ": null pointer");
  const uint64_t row = (uint64_t)a->heads * c.head_dim;
  const bool q16 = a->q_type == TQ_BF16;
  if (!aligned_to(a->q, q16 ? 2 : 4) || !aligned_to(a->out, 2) || !aligned_to(a->seqs, 4) || !aligned_to(a->lengths, 4) || !aligned_to(a->sizes, 4) ||
      !aligned_to(a->masks, 8) || !aligned_to(a->workspace, 16))
    return refuse(TQ_E_INVALID_ARG, who + ": a pointer is not aligned to its type (workspace: 16 bytes)");
  if ((a->q_stride && a->q_stride < row) || (a->out_stride && a->out_stride < row)) return refuse(TQ_E_INVALID_ARG, who + ": a stride is smaller than a row");
  if (a->workspace_bytes < l.bytes)
    return refuse(TQ_E_INVALID_ARG, who + ": the workspace has " + std::to_string(a->workspace_bytes) + " bytes, " + std::to_string(l.bytes) + " are needed");
  const TreeView v{a->q, (uint16_t*)a->out, a->seqs, a->lengths, a->sizes, a->masks, (float*)a->workspace, a->q_stride ? a->q_stride : row, a->out_stride ? a->out_stride : row,
                   a->scale * kLog2e, a->trees, a->nodes, a->heads, a->heads / c.kv_heads, l.columns, l.tiles, l.chunks, l.groups};
  hipStream_t st = (hipStream_t)stream;
  auto of = [&](auto dim) {
    constexpr int kDim = decltype(dim)::value;
    auto go = [&](auto kernel) { hipLaunchKernelGGL(kernel, dim3(l.groups), dim3(kTreeWaves<kDim> * 64), 0, st, c, v); };
    if (cache->type == TQ_INT8) q16 ? go(k_attend_tree<kDim, true, true>) : go(k_attend_tree<kDim, true, false>);
    else q16 ? go(k_attend_tree<kDim, false, true>) : go(k_attend_tree<kDim, false, false>);
    if (l.units == 1) return;   // nothing is cut
    const uint64_t waves = (uint64_t)a->trees * c.kv_heads * l.chunks * l.tiles * ((c.head_dim + 15) / 16);
    hipLaunchKernelGGL((cache->type == TQ_INT8 ? k_join_tree<kDim, true> : k_join_tree<kDim, false>), dim3((uint32_t)std::min<uint64_t>((waves + 3) / 4, 16384)), dim3(256), 0, st, c, v);
  };
  if (c.head_dim <= 64) of(std::integral_constant<int, 64>());
  else if (c.head_dim <= 128) of(std::integral_constant<int, 128>());
  else of(std::integral_constant<int, 256>());
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
    tq::Layout l{};
    const int rc = tq::check_tree("tq_attend_tree_workspace", cache, args, &c, &l);
    if (rc == TQ_OK) *bytes = l.bytes;
    return rc;
  });
}
