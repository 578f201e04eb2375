// Attention of a tree of drafted tokens over a paged cache (tq_attend_tree).
//
// All nodes of a tree and all query heads that share a key/value head are columns of one product, so that a token's key and value are read once for all of them.  A
// workgroup takes up to 8 tiles of 16 columns and a stage of tokens at a time: keys and values go from memory through registers (8 bits become bf16 there) to LDS, and a
// wavefront per column tile, or several that share out the tokens, reads them in the shape of v_mfma_f32_16x16x32_bf16:
//   logits [token][column] = K [token][dim] Q^T: lane l supplies token l % 16 and 8 neighbouring dims.
//   out^T [dim][column] = V^T [dim][token] P^T: the lane that got the logits of tokens 4g..4g+3 of both 16-token blocks (g = l / 16) supplies the same tokens as its 8
//   values of the contraction, so P is already where it is needed; V is transposed on its way out of LDS.
// q and p enter as three bf16 parts each, all of fp32's 24 bits.
#include <algorithm>

#include "tq_cache_view.h"
#include "tq_strip_decode.h"

namespace tq {
namespace {

constexpr int kTreeWaves = 8, kTreeThreads = kTreeWaves * 64, kMostTiles = 8, kTile = 32;
constexpr uint32_t kMaxGroups = 256;      // workgroups of a launch: one per compute unit
constexpr float kLog2e = 1.4426950408889634f;

struct TreeView {
  const void* q;
  uint16_t* out;
  const int32_t *seqs, *lengths, *sizes;
  const uint64_t* masks;
  float* partials;     // [workgroup][2]: [column][DIM] sums, then maximum and total of every column
  uint64_t q_stride, out_stride;
  float scale;         // times log2(e)
  uint32_t trees, nodes, heads, group, columns, tiles, chunks;   // columns of a key/value head; column tiles of a chunk; chunks per key/value head
  uint32_t groups;     // workgroups of the main launch
};

// What a tree's nodes attend to: slots below `length`, then slots length + j with bit j of a node's mask, below `end`.
struct Seen {
  uint32_t seq, length, end, size;
};
__device__ __forceinline__ Seen seen_by(const CacheView& c, const TreeView& a, uint32_t t) {
  const int32_t s = a.seqs ? a.seqs[t] : (int32_t)t;
  const uint32_t size = a.sizes ? (uint32_t)min(max(a.sizes[t], 0), (int32_t)a.nodes) : a.nodes, length = (uint32_t)max(a.lengths[t], 0);
  if ((uint32_t)s >= c.n_seqs || size == 0) return Seen{0, 0, 0, size};
  return Seen{(uint32_t)s, min(length, c.capacity), (uint32_t)min((uint64_t)length + size, (uint64_t)c.capacity), size};
}

template <bool INT8>
__device__ __forceinline__ float value_at(const char* from, uint32_t d) {
  if constexpr (INT8) return (float)((const int8_t*)from)[d];
  else return bf16_value(((const uint16_t*)from)[d]);
}

// Four dims of a row's head, divided by the weights' total.
__device__ __forceinline__ void write_out(const TreeView& a, uint32_t size, uint32_t t, uint32_t node, uint32_t head, uint32_t D, uint32_t d0, float4 sum, float total) {
  if (d0 >= D) return;
  const float inv = total == 0.f || node >= size ? 0.f : 1.f / total;
  if (node >= size) sum = make_float4(0.f, 0.f, 0.f, 0.f);
  uint16_t* to = a.out + ((uint64_t)t * a.nodes + node) * a.out_stride + head * D + d0;
  const uint32_t lo = pack_bf16(sum.x * inv, sum.y * inv), hi = pack_bf16(sum.z * inv, sum.w * inv);
  *(u32x2_any*)to = u32x2_any{lo, hi};
}

template <int DIM, bool INT8>
struct Shape {
  static constexpr int kTokens = 16384 / DIM, kTiles = kTokens / kTile;      // of a stage: 32 KB of keys and as much of values in LDS
  static constexpr int kSteps = DIM / 32, kBlocks = DIM / 16, kRow = DIM * 2; // contraction steps of the logits, blocks of 16 dims, bytes of a row in LDS
  static constexpr int kSize = INT8 ? 1 : 2, kPieces = DIM * kSize / 16;      // 16-byte pieces of a row in memory
  static constexpr int kLoads = kTokens * kPieces / kTreeThreads, kRows = 64 / kPieces;   // loads of a lane for a stage; rows that a wavefront loads at a time
};

// All (tree, key/value head, chunk, unit of a stage) in this order are one line, cut into equal shares, one per workgroup.
struct Line {
  uint32_t all, share;
};
template <int TOKENS>
__device__ __forceinline__ uint32_t units_of(uint32_t end) { return max((end + TOKENS - 1) / TOKENS, 1u); }   // (a tree without tokens is written too)

template <int DIM, bool INT8, bool Q16>
__global__ __launch_bounds__(kTreeThreads, 2) void k_attend_tree(CacheView c, TreeView a) {
  using S = Shape<DIM, INT8>;
  constexpr int kParts = Q16 ? 1 : 3;
  constexpr uint32_t kT = S::kTokens, kBytes = kT * S::kRow, kJoin = kTreeWaves * 16 * (DIM + 4) * 4;
  __shared__ __attribute__((aligned(16))) char lds[(4 * kBytes > kJoin ? 4 * kBytes : kJoin)];   // keys, values, keys, values; at a segment's end [wave][column][DIM + 4] sums
  __shared__ __attribute__((aligned(16))) uint32_t lds_kind[2][kT];     // 0: of the context, 1 + j: node j, kNobody
  __shared__ __attribute__((aligned(16))) float lds_scale[2][2][INT8 ? kT : 4];
  __shared__ float lds_max[kTreeWaves * 16], lds_total[kTreeWaves * 16], lds_weight[kTreeThreads];
  __shared__ uint64_t lds_at[kTreeThreads];
  __shared__ uint32_t lds_odd, lds_odd_column[kMostTiles * 16];
  constexpr uint32_t kNobody = 255;
  const uint32_t tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6), g = lane / 16, n = lane % 16, D = c.head_dim;
  auto scalar = [](uint32_t v) { return (uint32_t)__builtin_amdgcn_readfirstlane((int)v); };

  // this workgroup's share, and the tree it begins in
  uint32_t lane_units = 0;   // of tree (t & ~63) + lane
  auto look_at = [&](uint32_t first) {
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
  all *= pairs;
  const uint32_t share = (all + gridDim.x - 1) / gridDim.x;
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
  auto next_segment = [&] {
    Segment s;
    s.t = t, s.of = seen_by(c, a, t);
    s.of.seq = scalar(s.of.seq), s.of.length = scalar(s.of.length), s.of.end = scalar(s.of.end), s.of.size = scalar(s.of.size);
    s.units = (uint32_t)__builtin_amdgcn_readlane((int)lane_units, t & 63);
    const uint32_t pair = (pos - tree_first) / s.units;
    s.first = tree_first + pair * s.units;
    s.kv = pair / a.chunks, s.first_column = pair % a.chunks * a.tiles * 16;
    s.unit = pos - s.first, s.n_units = min(s.units - s.unit, stop - pos);
    pos += s.n_units;
    if (pos == tree_first + s.units * pairs) {
      tree_first = pos, ++t;
      if ((t & 63) == 0 && pos < stop) look_at(t);
    }
    return s;
  };

  // ---- from memory to registers ----
  const uint32_t piece = lane % S::kPieces, row_of_lane = lane / S::kPieces;
  const uint32_t slot_bytes = S::kSize * (uint32_t)c.slot_stride;
  const uint32_t lane_at = row_of_lane * slot_bytes + (16 * piece < S::kSize * D ? 16 * piece : 0);   // (dims that a head does not have: its first ones, against zeros of q)
  uint4 in_k[S::kLoads], in_v[S::kLoads];
  float in_ks[S::kLoads], in_vs[S::kLoads];
  uint32_t in_limit[S::kLoads], in_first[S::kLoads], in_length = 0;   // rows of a load that are there; their first slot
  auto fetch_one = [&](const Segment& s, uint32_t unit, int i) {
    constant_i32* table = (constant_i32*)(c.tables + (uint64_t)s.of.seq * c.table_stride);
    const uint32_t newest = max(s.of.end, 1u) - 1, slot = unit * kT + (i * kTreeWaves + wave) * S::kRows, from = min(slot, newest & ~(uint32_t)(S::kRows - 1));
    const uint32_t id = scalar((uint32_t)table[from >> c.page_shift]), page = id < c.n_pages ? id : 0, in_page = from & ((1u << c.page_shift) - 1);
    in_first[i] = slot;
    in_limit[i] = id < c.n_pages && slot < s.of.end ? min(s.of.end - slot, (uint32_t)S::kRows) : 0u;
    const uint64_t at = S::kSize * ((uint64_t)page * c.page_stride + s.kv * c.head_stride + in_page * c.slot_stride);
    in_k[i] = *(const uint4*)(c.k + at + lane_at);
    in_v[i] = *(const uint4*)(c.v + at + lane_at);
    if constexpr (INT8) {
      const uint64_t mark = (((uint64_t)page * c.kv_heads + s.kv) << c.page_shift) + in_page + row_of_lane;
      in_ks[i] = c.k_scale[mark], in_vs[i] = c.v_scale[mark];
    }
  };
  // ---- from registers to LDS: rows of pieces of 8 dims, in places that spread the lanes of a read over the banks ----
  auto store_one = [&](uint32_t buffer, int i) {
    const uint32_t row = (i * kTreeWaves + wave) * S::kRows + row_of_lane;
    const bool there = row_of_lane < in_limit[i];
    char* keys = lds + buffer * 2 * kBytes + row * S::kRow;
    char* values = keys + kBytes;
    constexpr uint32_t kKeyMask = DIM == 64 ? 7 : 15, kValueMask = DIM == 64 ? 3 : 7;
    auto put = [&](uint32_t p, uint4 k, uint4 v) {
      *(uint4*)(keys + ((p ^ (row & kKeyMask)) * 16)) = k;
      *(uint4*)(values + ((p ^ ((row & kValueMask) << 1)) * 16)) = v;
    };
    const uint4 none = make_uint4(0, 0, 0, 0);
    const uint4 k = there ? in_k[i] : none, v = there ? in_v[i] : none;
    if constexpr (INT8) {
      auto wide = [](uint32_t x, uint32_t y) { return __builtin_bit_cast(uint4, i8x8_to_bf16x8(make_uint2(x, y))); };
      put(2 * piece, wide(k.x, k.y), wide(v.x, v.y));
      put(2 * piece + 1, wide(k.z, k.w), wide(v.z, v.w));
    } else {
      put(piece, k, v);
    }
    if (piece == 0) {
      const uint32_t slot = in_first[i] + row_of_lane;
      lds_kind[buffer][row] = !there ? kNobody : slot < in_length ? 0u : 1 + slot - in_length;
      // (an infinite scale of a key makes NaN of a level of zero, and is NaN here, so that the tokens are taken again)
      if constexpr (INT8) lds_scale[buffer][0][row] = there ? fmaf(in_ks[i], a.scale, in_ks[i] * 0.f) : 0.f, lds_scale[buffer][1][row] = there ? in_vs[i] : 0.f;
    }
  };

  const uint32_t over = min((uint32_t)(kTreeWaves / a.tiles), (uint32_t)S::kTiles);   // wavefronts that share out the tokens of a column tile
  const uint32_t of_tile = wave % a.tiles, of_tokens = wave / a.tiles;
  const bool works = of_tokens < over;
  const uint32_t key_at = n * S::kRow, key_swizzle = g ^ (n & (DIM == 64 ? 7 : 15));
  const uint32_t value_row = 4 * g + n / 4, value_at0 = value_row * S::kRow + ((value_row & (DIM == 64 ? 3 : 7)) * 32) + n % 4 * 8;
  bf16x8 q[kParts][S::kSteps];
  uint64_t mask = 0;
  auto column_of = [&](const Segment& s, uint32_t column, uint32_t* node) {   // -> query head
    *node = column / a.group;
    return s.kv * a.group + column % a.group;
  };
  auto load_q = [&](const Segment& s) {
    const uint32_t column = s.first_column + of_tile * 16 + n;
    const bool has = works && column < a.columns;
    uint32_t node, head = column_of(s, has ? column : 0, &node);
    const uint64_t row = (uint64_t)s.t * a.nodes + node;
    mask = has && node < s.of.size ? a.masks[row] : 0;
#pragma unroll
    for (int i = 0; i < S::kSteps; ++i) {
      const uint32_t d = i * 32 + 8 * g;
      const bool own = has && d < D;
      const uint64_t at = row * a.q_stride + head * D + (own ? d : 0);
      if constexpr (Q16) {
        const u16x4_any lo = *(const u16x4_any*)((const uint16_t*)a.q + at), hi = *(const u16x4_any*)((const uint16_t*)a.q + at + 4);
#pragma unroll
        for (int j = 0; j < 8; ++j) q[0][i][j] = own ? __builtin_bit_cast(__bf16, (uint16_t)(j < 4 ? lo[j % 4] : hi[j % 4])) : (__bf16)0.f;
      } else {
        const f32x4_any lo = *(const f32x4_any*)((const float*)a.q + at), hi = *(const f32x4_any*)((const float*)a.q + at + 4);
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          const float v = own ? (j < 4 ? lo[j % 4] : hi[j % 4]) : 0.f;
          const __bf16 upper = (__bf16)v, middle = (__bf16)(v - (float)upper);
          q[0][i][j] = upper, q[kParts > 1][i][j] = middle, q[kParts - 1][i][j] = (__bf16)(v - (float)upper - (float)middle);
        }
      }
    }
  };

  f32x4 o[S::kBlocks];
  float top = -INFINITY, total = 0.f;
  auto take_tile = [&](uint32_t buffer, uint32_t tile) {
    const char* keys = lds + buffer * 2 * kBytes + tile * kTile * S::kRow;
    const char* values = keys + kBytes;
    f32x4 l[2] = {{0.f, 0.f, 0.f, 0.f}, {0.f, 0.f, 0.f, 0.f}};
#pragma unroll
    for (int i = 0; i < S::kSteps; ++i) {
      bf16x8 key[2];
#pragma unroll
      for (int b = 0; b < 2; ++b) key[b] = *(const bf16x8*)(keys + b * 16 * S::kRow + key_at + ((key_swizzle ^ (4 * i)) * 16));
#pragma unroll
      for (int part = 0; part < kParts; ++part)
#pragma unroll
        for (int b = 0; b < 2; ++b) l[b] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(key[b], q[part][i], l[b], 0, 0, 0);
    }
    float p[8];
    uint4 kind[2];
    float4 vs[2];
#pragma unroll
    for (int b = 0; b < 2; ++b) {
      kind[b] = *(const uint4*)&lds_kind[buffer][tile * kTile + 16 * b + 4 * g];
      float4 ks = make_float4(a.scale, a.scale, a.scale, a.scale);
      if constexpr (INT8) {
        ks = *(const float4*)&lds_scale[buffer][0][tile * kTile + 16 * b + 4 * g];
        vs[b] = *(const float4*)&lds_scale[buffer][1][tile * kTile + 16 * b + 4 * g];
      }
#pragma unroll
      for (int j = 0; j < 4; ++j) p[4 * b + j] = l[b][j] * (&ks.x)[j];
    }
    if (__any((kind[0].x | kind[0].y | kind[0].z | kind[0].w | kind[1].x | kind[1].y | kind[1].z | kind[1].w) != 0)) {
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const uint32_t k = (&kind[i / 4].x)[i % 4];
        if (!(k == 0 || (k != kNobody && mask >> (k - 1) & 1))) p[i] = -INFINITY;
      }
    }
    float m = p[0];
#pragma unroll
    for (int i = 1; i < 8; ++i) m = fmaxf(m, p[i]);
    // The weights' reference follows the maximum when that has grown by more than 8 (2^8 is far from any bound of fp32).
    if (__any(m > top + 8.f)) {
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
        w[j] = __builtin_amdgcn_exp2f(p[i + j] - base);
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
    typedef short s16x4 __attribute__((ext_vector_type(4)));
    typedef __attribute__((address_space(3))) s16x4 lds_s16x4;
#pragma unroll
    for (int b = 0; b < S::kBlocks; ++b) {
      const char* from = values + (value_at0 ^ (b * 32));
      const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)from), hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((lds_s16x4*)(from + 16 * S::kRow));
      const bf16x8 value = __builtin_bit_cast(bf16x8, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
#pragma unroll
      for (int k = 0; k < 3; ++k)
        o[b] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(value, __builtin_bit_cast(bf16x8, make_uint4(part[k][0], part[k][1], part[k][2], part[k][3])), o[b], 0, 0, 0);
    }
  };

  // A segment's tokens once more, a product per value as the formula has them, so that infinities give what they give there: only for what is not finite, and
  // slow.  Its results replace those in LDS.
  auto take_again = [&](const Segment& s, float* sums) {
    const uint32_t begin = s.unit * kT, end = min(s.of.end, (s.unit + s.n_units) * kT), mine = min(a.columns - s.first_column, a.tiles * 16);
    for (uint32_t col = 0; col < mine; ++col) {
      if (!lds_odd_column[col]) continue;
      uint32_t node, head = column_of(s, s.first_column + col, &node);
      const uint64_t row = (uint64_t)s.t * a.nodes + node, sees = a.masks[row];
      const uint64_t q_at = row * a.q_stride + head * D;
      float m = -INFINITY, sum_p = 0.f, sum = 0.f;
      for (uint32_t first = begin; first < end && node < s.of.size; first += kTreeThreads) {
        const uint32_t slot = first + tid;
        uint32_t page = c.n_pages;
        if (slot < end && (slot < s.of.length || sees >> (slot - s.of.length) & 1)) page = (uint32_t)c.tables[(uint64_t)s.of.seq * c.table_stride + (slot >> c.page_shift)];
        const bool there = page < c.n_pages;
        const uint32_t in_page = slot & ((1u << c.page_shift) - 1);
        const uint64_t at = S::kSize * ((uint64_t)(there ? page : 0) * c.page_stride + s.kv * c.head_stride + in_page * c.slot_stride);
        const uint64_t mark = (((uint64_t)(there ? page : 0) * c.kv_heads + s.kv) << c.page_shift) + in_page;
        float l = -INFINITY;
        if (there) {
          const float scale = INT8 ? c.k_scale[mark] : 1.f;
          const bool after = fabsf(scale) < INFINITY;   // (an infinite scale makes NaN of a level of zero)
          l = 0.f;
          for (uint32_t x = 0; x < D; ++x) {
            const float of_q = (Q16 ? bf16_value(((const uint16_t*)a.q)[q_at + x]) : ((const float*)a.q)[q_at + x]) * a.scale;
            l = fmaf(of_q, after ? value_at<INT8>(c.k + at, x) : value_at<INT8>(c.k + at, x) * scale, l);
          }
          if (after) l *= scale;
        }
        __syncthreads();
        lds_weight[tid] = l, lds_at[tid] = there ? at : ~0ull;
        __syncthreads();
        float most = m;
        for (uint32_t i = 0; i < kTreeThreads; ++i) most = fmaxf(most, lds_weight[i]);
        const float base = most == -INFINITY ? 0.f : most, shrink = exp2f(m - base);
        m = most, sum_p *= shrink, sum *= shrink;
        const float p = there ? exp2f(l - base) : 0.f, with_scale = there && INT8 ? p * c.v_scale[mark] : p;
        __syncthreads();
        lds_weight[tid] = p;
        __syncthreads();
        for (uint32_t i = 0; i < kTreeThreads; ++i) sum_p += lds_weight[i];
        __syncthreads();
        lds_weight[tid] = with_scale;
        __syncthreads();
        if (tid < D)
          for (uint32_t i = 0; i < kTreeThreads; ++i)
            if (lds_at[i] != ~0ull) sum = fmaf(lds_weight[i], value_at<INT8>(c.v + lds_at[i], tid), sum);
      }
      // the first of the wavefronts that share this tile has it all, the others nothing
      for (uint32_t w = 0; w < over; ++w) {
        const uint32_t at = (col / 16 + w * a.tiles) * 16 + col % 16;
        if (tid < DIM) sums[at * (DIM + 4) + tid] = w ? 0.f : sum;
        if (tid == 0) lds_max[at] = w ? -INFINITY : m, lds_total[at] = w ? 0.f : sum_p;
      }
    }
  };

  auto finish = [&](const Segment& s) {
    float* sums = (float*)lds;
    total += __shfl_xor(total, 16);
    total += __shfl_xor(total, 32);
    float odd = total * 0.f;   // a query, key or value that is not finite leaves no total or sum finite that it went into
#pragma unroll
    for (int b = 0; b < S::kBlocks; ++b)
#pragma unroll
      for (int j = 0; j < 4; ++j) odd = fmaf(o[b][j], 0.f, odd);
    if (tid == 0) lds_odd = 0;
    if (tid < kMostTiles * 16) lds_odd_column[tid] = 0;
    __syncthreads();   // everyone is done with the stages
    if (works) {
#pragma unroll
      for (int b = 0; b < S::kBlocks; ++b) *(f32x4*)&sums[(wave * 16 + n) * (DIM + 4) + b * 16 + 4 * g] = o[b];
      if (g == 0) lds_max[wave * 16 + n] = top, lds_total[wave * 16 + n] = total;
      if (!(odd == 0.f)) lds_odd = lds_odd_column[of_tile * 16 + n] = 1;
    }
    __syncthreads();
    if (__builtin_expect(lds_odd, 0)) {
      take_again(s, sums);
      __syncthreads();
    }
    constexpr uint32_t kLanes = DIM / 4, kAtATime = kTreeThreads / kLanes;   // lanes of a column, four dims each
    const uint32_t d0 = tid % kLanes * 4, mine = min(a.columns - s.first_column, a.tiles * 16);
    const bool whole = s.n_units == s.units;
    float* to_part = a.partials + (uint64_t)(2 * blockIdx.x + (blockIdx.x * share >= s.first ? 0 : 1)) * (a.tiles * 16 * (DIM + 2));
    for (uint32_t col = tid / kLanes; col < mine; col += kAtATime) {
      float m = -INFINITY, sum_p = 0.f;
      float4 sum = make_float4(0.f, 0.f, 0.f, 0.f);
      for (uint32_t w = 0; w < over; ++w) m = fmaxf(m, lds_max[(col / 16 + w * a.tiles) * 16 + col % 16]);
      const float base = m == -INFINITY ? 0.f : m;
      for (uint32_t w = 0; w < over; ++w) {
        const uint32_t at = (col / 16 + w * a.tiles) * 16 + col % 16;
        const float f = __builtin_amdgcn_exp2f(lds_max[at] - base);
        const float4 v = *(const float4*)&sums[at * (DIM + 4) + d0];
        sum_p = fmaf(f, lds_total[at], sum_p);
        sum.x = fmaf(f, v.x, sum.x), sum.y = fmaf(f, v.y, sum.y), sum.z = fmaf(f, v.z, sum.z), sum.w = fmaf(f, v.w, sum.w);
      }
      if (whole) {
        uint32_t node, head = column_of(s, s.first_column + col, &node);
        write_out(a, s.of.size, s.t, node, head, D, d0, sum, sum_p);
      } else {
        *(float4*)&to_part[col * DIM + d0] = sum;
        if (d0 == 0) *(float2*)&to_part[a.tiles * 16 * DIM + 2 * col] = make_float2(m, sum_p);
      }
    }
    __syncthreads();   // LDS is free again
  };

  Segment s = next_segment(), next = s;
  uint32_t unit = 0, buffer = 0;
  in_length = s.of.length;
#pragma unroll
  for (int i = 0; i < S::kLoads; ++i) fetch_one(s, s.unit, i);
  load_q(s);
  for (;;) {
    if (unit == 0) {
      top = -INFINITY, total = 0.f;
#pragma unroll
      for (int b = 0; b < S::kBlocks; ++b) o[b] = f32x4{0.f, 0.f, 0.f, 0.f};
    }
    const bool last = unit + 1 == s.n_units, more = pos < stop;
#pragma unroll
    for (int i = 0; i < S::kLoads; ++i) store_one(buffer, i);
    if (last && more) next = next_segment();
    if (!last || more) {
      in_length = next.of.length;
      const uint32_t at = last ? next.unit : s.unit + unit + 1;
#pragma unroll
      for (int i = 0; i < S::kLoads; ++i) fetch_one(last ? next : s, at, i);
    }
    __syncthreads();
    if (works)
      for (uint32_t tile = of_tokens; tile < (uint32_t)S::kTiles; tile += over) take_tile(buffer, tile);
    buffer ^= 1, ++unit;
    if (!last) continue;
    finish(s);
    if (!more) break;
    s = next, unit = 0;
    load_q(s);
  }
}

// The parts of what lies in more than one share, joined in the order of the line.  A wavefront takes a column, all lanes four dims at a time.
template <int DIM, int TOKENS>
__global__ __launch_bounds__(256) void k_join_tree(CacheView c, TreeView a) {
  const uint32_t lane = threadIdx.x & 63, wave = threadIdx.x >> 6, pairs = c.kv_heads * a.chunks, D = c.head_dim;
  const uint32_t per_tree = c.kv_heads * a.columns;
  for (uint64_t of = (uint64_t)blockIdx.x * 4 + wave; of < (uint64_t)a.trees * per_tree; of += (uint64_t)gridDim.x * 4) {
    const uint32_t t = (uint32_t)(of / per_tree), kv = (uint32_t)(of % per_tree) / a.columns, column = (uint32_t)of % per_tree % a.columns;
    uint32_t all = 0, before = 0;
    for (uint32_t first = 0; first < a.trees; first += 64) {
      const uint32_t units = first + lane < a.trees ? units_of<TOKENS>(seen_by(c, a, first + lane).end) : 0u;
      all += units;
      if (first + lane < t) before += units;
    }
#pragma unroll
    for (int d = 1; d < 64; d *= 2) all += __shfl_xor(all, d), before += __shfl_xor(before, d);
    const Seen seen = seen_by(c, a, t);
    const uint32_t units = units_of<TOKENS>(seen.end), share = (all * pairs + a.groups - 1) / a.groups;
    const uint32_t chunk = column / (a.tiles * 16), col = column % (a.tiles * 16), first = before * pairs + (kv * a.chunks + chunk) * units;
    const uint32_t group0 = first / share, group1 = (first + units - 1) / share;
    if (group0 == group1) continue;
    auto part_of = [&](uint32_t group) { return a.partials + (uint64_t)(2 * group + (group * share >= first ? 0 : 1)) * (a.tiles * 16 * (DIM + 2)); };
    float m = -INFINITY, sum_p = 0.f;
    for (uint32_t group = group0; group <= group1; ++group) m = fmaxf(m, part_of(group)[a.tiles * 16 * DIM + 2 * col]);
    const float base = m == -INFINITY ? 0.f : m;
    float4 sum = make_float4(0.f, 0.f, 0.f, 0.f);
    const uint32_t d0 = 4 * lane < DIM ? 4 * lane : 0;
    for (uint32_t group = group0; group <= group1; ++group) {
      const float* from = part_of(group);
      const float2 st = *(const float2*)&from[a.tiles * 16 * DIM + 2 * col];
      const float f = __builtin_amdgcn_exp2f(st.x - base);
      const float4 v = *(const float4*)&from[col * DIM + d0];
      sum_p = fmaf(f, st.y, sum_p);
      sum.x = fmaf(f, v.x, sum.x), sum.y = fmaf(f, v.y, sum.y), sum.z = fmaf(f, v.z, sum.z), sum.w = fmaf(f, v.w, sum.w);
    }
    if (4 * lane < DIM) write_out(a, seen.size, t, column / a.group, kv * a.group + column % a.group, D, d0, sum, sum_p);
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
  const uint32_t group = a->heads / c->kv_heads, dim = c->head_dim <= 64 ? 64 : c->head_dim <= 128 ? 128 : 256, tokens = 16384 / dim;
  l->columns = a->nodes * group;
  const uint32_t all_tiles = (l->columns + 15) / 16;
  l->chunks = (all_tiles + kMostTiles - 1) / kMostTiles;
  l->tiles = (all_tiles + l->chunks - 1) / l->chunks;
  l->units = (c->capacity + tokens - 1) / tokens;
  const uint64_t most = (uint64_t)a->trees * c->kv_heads * l->chunks * l->units;   // if all sequences are full
  if (most >= (1u << 31) - kMaxGroups) return refuse(TQ_E_UNSUPPORTED, who + ": trees * heads * capacity is beyond what one call takes");
  l->groups = (uint32_t)std::min<uint64_t>(kMaxGroups, std::max<uint64_t>(1, most));
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
  auto go = [&](auto dim, auto kernel) {
    constexpr int kDim = decltype(dim)::value;
    hipLaunchKernelGGL(kernel, dim3(l.groups), dim3(kTreeThreads), 0, st, c, v);
    if (l.units == 1) return;   // nothing is cut
    const uint64_t columns = (uint64_t)a->trees * c.kv_heads * l.columns;
    hipLaunchKernelGGL((k_join_tree<kDim, 16384 / kDim>), dim3((uint32_t)std::min<uint64_t>((columns + 3) / 4, 16384)), dim3(256), 0, st, c, v);
  };
  auto of = [&](auto dim) {
    constexpr int kDim = decltype(dim)::value;
    if (cache->type == TQ_INT8) q16 ? go(dim, k_attend_tree<kDim, true, true>) : go(dim, k_attend_tree<kDim, true, false>);
    else q16 ? go(dim, k_attend_tree<kDim, false, true>) : go(dim, k_attend_tree<kDim, false, false>);
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
